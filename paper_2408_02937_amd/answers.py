"""The index and the cache together: requests are answered behind the passages that a search finds (`bench.py --study answers`).

Passages are embedded vectors in an index and token sequences whose keys and values lie in the cache, written once.  A batch of
requests is searched for; each request forks the sequence of its best passage (pages are shared, nothing is copied but a last
page that is part full), appends its question (a short prompt) and decodes tokens in a recorded HIP graph; then its pages are
freed.  Some passages are replaced in between, and the pages compacted.  The network is a stack of attention layers
with random weights: what is timed is the path, not what it says.

The same network answers by trees of drafted tokens too: each token's most likely followers, as `score` last gave them, make a tree behind
the token that was chosen last; one pass attends to all of it, the path that the choices follow stays in the cache, the rest is cut.
"""
from __future__ import annotations

import time

import torch

from . import rtams, synth
from .cache import Cache
from .logits import score


class Stack:
    """Layers of attention over a cache and of a small perceptron, random weights, bfloat16."""

    def __init__(self, layers: int, heads: int, kv_heads: int, head_dim: int, vocab: int, device, seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)
        width = heads * head_dim
        w = lambda i, o: (torch.randn((i, o), device=device, generator=g) * i ** -0.5).bfloat16()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.tokens = w(width, vocab).t().contiguous()
        self.layers = [{"qkv": w(width, (heads + 2 * kv_heads) * head_dim), "out": w(width, width), "up": w(width, 2 * width),
                        "down": w(2 * width, width)} for _ in range(layers)]

    def __call__(self, cache: Cache, ids: torch.Tensor, seqs: torch.Tensor, starts=None, max_new=None, tree=None) -> torch.Tensor:
        """The rows' states after all layers; room for them has been made.  tree: what drafted rows see of each other."""
        norm = lambda x: torch.nn.functional.layer_norm(x, x.shape[-1:])
        x = self.tokens[ids]
        for i, w in enumerate(self.layers):
            qkv = (norm(x) @ w["qkv"]).view(len(ids), -1, self.head_dim)  # queries, keys and values are views of one tensor
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
            cache.write(i, k, v, seqs, starts, max_new)
            a = cache.attend(i, q, seqs, starts, max_new, tree=tree)
            x = x + a.view(len(ids), -1) @ w["out"]
            x = x + torch.nn.functional.gelu(norm(x) @ w["up"]) @ w["down"]
        return norm(x)

    def next_ids(self, x: torch.Tensor) -> torch.Tensor:
        return (x @ self.tokens.t()).argmax(-1)


# A draft: node 0 is the token chosen last; node j follows node PARENTS[j] and is its RANKS[j]-th most likely follower.
PARENTS = (-1, 0, 0, 1, 2, 3, 1)
RANKS = (0, 0, 1, 0, 0, 0, 1)


class Drafts:
    """Answers by trees of drafted tokens: the state of some requests, and a step that can be recorded."""

    def __init__(self, net: Stack, cache: Cache, seqs: torch.Tensor, ids: torch.Tensor, vocab: int):
        dev, n, nodes = ids.device, len(ids), len(PARENTS)
        self.net, self.cache, self.seqs, self.ids = net, cache, seqs, ids  # ids: the tokens chosen last, int32
        self.followers = torch.zeros((n, vocab, max(RANKS) + 1), dtype=torch.int32, device=dev)  # of each request's tokens
        self.parents = _ints(PARENTS * n, dev)
        self.starts = _ints(range(0, n * nodes + 1, nodes), dev)
        self.request = torch.arange(n, device=dev)
        self.drafted = torch.zeros((n, nodes), dtype=torch.int32, device=dev)
        self.chosen, self.path = (torch.zeros((n, nodes), dtype=torch.int32, device=dev) for _ in range(2))
        self.kept = torch.zeros(n, dtype=torch.int32, device=dev)
        self.logprobs = torch.zeros((n, nodes), device=dev)

    def step(self) -> None:
        args = (self.seqs, self.starts, len(PARENTS))
        self.drafted[:, 0] = self.ids
        for j in range(1, len(PARENTS)):
            self.drafted[:, j] = self.followers[self.request, self.drafted[:, PARENTS[j]].long(), RANKS[j]]
        self.cache.extend(self.seqs, self.starts)
        tree, _ = self.cache.tree(self.parents, *args)
        x = self.net(self.cache, self.drafted.flatten().long(), *args, tree=tree)
        said = score(x @ self.net.tokens.t(), top=max(RANKS) + 1)
        top = said.top.view(*self.drafted.shape, -1)
        for j in range(len(PARENTS)):  # (one node after the other: of a token that is there twice the last one counts)
            self.followers[self.request, self.drafted[:, j].long()] = top[:, j]
        self.chosen.copy_(top[..., 0])
        self.logprobs.copy_(said.top_logprobs[:, 0].view_as(self.logprobs))
        path, kept, following = self.cache.walk(self.parents, self.drafted.flatten(), self.chosen.flatten(), self.starts, len(PARENTS))
        self.cache.keep(path, kept, *args)
        self.path.copy_(path.view_as(self.path))
        self.kept.copy_(kept)
        self.ids.copy_(following)


def drafted_answers(net: Stack, requests: int, steps: int, page_tokens: int, vocab: int, record: bool = True, seed: int = 7) -> dict:
    """Prompts answered a token at a time, and by drafts from the same pages."""
    dev = net.tokens.device
    rng = torch.Generator().manual_seed(seed)
    text = torch.Generator(device=dev).manual_seed(seed)
    counts = torch.randint(50, 240, (requests,), generator=rng).tolist()
    longest = 240 + 4 * steps + len(PARENTS)  # a step keeps four tokens at most
    wide = -(-longest // page_tokens)
    cache = Cache(net.kv_heads, net.head_dim, layers=len(net.layers), page_tokens=page_tokens, pages=2 * requests * wide, max_seqs=2 * requests, max_pages=wide, device=dev)
    plain, mine = _ints(range(requests), dev), _ints(range(requests, 2 * requests), dev)
    st = _starts(counts, dev)
    cache.extend(plain, st)
    x = net(cache, torch.randint(0, vocab, (sum(counts),), device=dev, generator=text), plain, st, max(counts))
    first = score(x[st[1:].long() - 1] @ net.tokens.t(), top=1).top[:, 0].contiguous()
    cache.fork(plain, mine)

    def timed(step, keep):
        step()
        keep(0)
        torch.cuda.synchronize()
        graph = None
        if record:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        t0 = time.perf_counter()
        for i in range(1, steps):
            graph.replay() if graph else step()
            keep(i)
        torch.cuda.synchronize()
        return (time.perf_counter() - t0) * 1e3 / max(1, steps - 1)

    ids = first.clone()
    one = torch.zeros((steps, requests), dtype=torch.int32, device=dev)

    def step():
        cache.extend(plain)
        ids.copy_(score(net(cache, ids.long(), plain) @ net.tokens.t(), top=1).top[:, 0])

    ms_one = timed(step, lambda i: one[i].copy_(ids))
    d = Drafts(net, cache, mine, first.clone(), vocab)
    chosen, path = (torch.zeros((steps, *d.drafted.shape), dtype=torch.int32, device=dev) for _ in range(2))
    logprobs = torch.zeros((steps, *d.drafted.shape), device=dev)

    def keep(i):
        chosen[i], path[i], logprobs[i] = d.chosen, d.path, d.logprobs

    ms = timed(d.step, keep)
    assert cache.poll_error() == rtams.OK, cache.poll_error()
    one, chosen, path, logprobs = one.t().tolist(), chosen.tolist(), path.tolist(), logprobs.tolist()
    said = [[chosen[i][r][j] for i in range(steps) for j in path[i][r] if j >= 0] for r in range(requests)]
    sure = [logprobs[i][r][j] for r in range(requests) for i in range(steps) for j in path[i][r] if j >= 0]
    tokens = sum(len(x) for x in said)
    alike = sum(next((i for i, (a, b) in enumerate(zip(x, y)) if a != b), min(len(x), len(y))) for x, y in zip(said, one))
    out = {"requests": requests, "steps": steps, "nodes": len(PARENTS), "ms_per_step_of_one": ms_one, "ms_per_step": ms, "tokens_per_step": tokens / (steps * requests),
           "tokens_per_s_of_one": requests / (ms_one * 1e-3), "tokens_per_s": tokens / steps / (ms * 1e-3), "mean_logprob": sum(sure) / max(1, len(sure)),
           "alike_before_the_first_difference": alike / max(1, sum(min(len(x), len(y)) for x, y in zip(said, one))), "said_sum": sum(map(sum, said)),
           "lengths": cache.lengths[requests:].tolist(), "prompts": counts, "said": said}
    cache.close()
    return out


def _ints(values, device):
    return torch.tensor(list(values), dtype=torch.int32, device=device)


def _starts(counts, device):
    return torch.nn.functional.pad(torch.tensor(list(counts), device=device).cumsum(0), (1, 0)).to(torch.int32)


def answers_study(scale: float = 1.0, layers: int = 4, heads: int = 16, kv_heads: int = 4, head_dim: int = 64, requests: int = 32,
                  steps: int = 32, rounds: int = 4, page_tokens: int = 64, record: bool = True, seed: int = 7) -> dict:
    dev = torch.device("cuda:0")
    rng = torch.Generator().manual_seed(seed)
    text = torch.Generator(device=dev).manual_seed(seed)
    pick = lambda lo, hi, n: torch.randint(lo, hi, (n,), generator=rng).tolist()
    # passages: vectors shaped like text embeddings, and tokens
    w = synth.config(4, scale=0.01 * scale)
    n = min(len(w.base), max(requests, int(512 * scale)))
    vectors, queries = torch.from_numpy(w.base[:n].copy()).to(dev), torch.from_numpy(w.queries).to(dev)
    index = rtams.Index(w.d, w.nlist, w.metric, w.block_vecs, pool_blocks=n // w.block_vecs + 2 * w.nlist + 64, max_batch=requests,
                        max_k=4, max_nprobe=min(32, w.nlist), candidates_per_query=n + 64)
    index.set_centroids(torch.from_numpy(w.centroids).to(dev))
    index.add(vectors)
    net = Stack(layers, heads, kv_heads, head_dim, 4096, dev, seed)
    lengths, vocab = pick(40, 200, n), 4096
    seqs_all = n + requests
    longest = 200 + 40 + steps
    pages = sum(-(-x // page_tokens) for x in lengths) + requests * (2 + (40 + steps) // page_tokens) + 64
    cache = Cache(kv_heads, head_dim, layers=layers, page_tokens=page_tokens, pages=pages, max_seqs=seqs_all, max_pages=-(-longest // page_tokens), device=dev)

    def read_passages(which):
        counts = [lengths[i] for i in which]
        s, st = _ints(which, dev), _starts(counts, dev)
        cache.extend(s, st)
        net(cache, torch.randint(0, vocab, (sum(counts),), device=dev, generator=text), s, st, max(counts))

    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for at in range(0, n, 64):
        read_passages(range(at, min(n, at + 64)))
    torch.cuda.synchronize()
    out = {"study": "answers", "passages": n, "passage_tokens": sum(lengths), "layers": layers, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
           "page_tokens": page_tokens, "pages": pages, "cache_bytes": cache.pages.numel(), "read_passages_s": time.perf_counter() - t0, "rounds": []}

    mine = _ints(range(n, seqs_all), dev)
    ids = torch.zeros(requests, dtype=torch.int64, device=dev)
    said = torch.zeros((steps, requests), dtype=torch.int64, device=dev)

    def step():
        cache.extend(mine)
        ids.copy_(net.next_ids(net(cache, ids, mine)))

    graph = None
    for r in range(rounds):
        q = queries[(torch.arange(requests, device=dev) + r * requests) % len(queries)]
        t = [time.perf_counter()]

        def lap():
            torch.cuda.synchronize()
            t.append(time.perf_counter())

        found = index.search(q, 4, min(32, w.nlist))[1][:, 0].clamp(min=0).to(torch.int32)
        lap()
        cache.fork(found, mine)
        shared = int((cache.refs > 1).sum())
        lap()
        counts = pick(8, 40, requests)
        st = _starts(counts, dev)
        cache.extend(mine, st)
        x = net(cache, torch.randint(0, vocab, (sum(counts),), device=dev, generator=text), mine, st, max(counts))
        ids.copy_(net.next_ids(x[st[1:].long() - 1]))
        lap()
        if record and graph is None:  # (a step that has run once is recorded)
            step()
            said[0] = ids
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            done = 1
            t[-1] = time.perf_counter()
        else:
            done = 0
        for i in range(done, steps):
            graph.replay() if graph else step()
            said[i] = ids
        lap()
        used = pages - cache.free_pages
        cache.trim(mine)
        gone = sorted(set(pick(0, n, max(1, n // 16))))  # some passages are replaced by shorter ones
        cache.trim(_ints(gone, dev))
        cache.compact()
        for i, length in zip(gone, pick(40, 200, len(gone))):
            lengths[i] = min(length, lengths[i])
        read_passages(gone)
        lap()
        out["rounds"].append({"search_ms": (t[1] - t[0]) * 1e3, "fork_ms": (t[2] - t[1]) * 1e3, "questions_ms": (t[3] - t[2]) * 1e3,
                              "ms_per_step": (t[4] - t[3]) * 1e3 / max(1, steps - done), "replace_ms": (t[5] - t[4]) * 1e3, "question_tokens": sum(counts),
                              "pages_shared": shared, "pages_in_use": used, "said": said.flatten()[:8].tolist(), "said_sum": int(said.sum())})
    assert cache.poll_error() == rtams.OK, cache.poll_error()
    last = out["rounds"][-1]
    out["tokens_per_s"] = requests / (last["ms_per_step"] * 1e-3)
    index.close()
    cache.close()
    drafted = drafted_answers(net, requests, steps, page_tokens, vocab, record, seed)
    out["drafted"] = {k: v for k, v in drafted.items() if k not in ("lengths", "prompts", "said")}
    return out
