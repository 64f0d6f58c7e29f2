"""Answers by trees of drafted tokens: recorded steps say what steps one by one say, every sequence holds what was kept, and the answers are
those of the network a token at a time wherever its choice is not within roundings of another."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_drafted_answers():
    from paper_2408_02937_amd import answers
    dev = torch.device("cuda:0")
    net = answers.Stack(2, 8, 2, 64, 512, dev, seed=3)
    print("[case] drafted answers, recorded and not", flush=True)
    a, b = (answers.drafted_answers(net, requests=6, steps=12, page_tokens=32, vocab=512, record=r) for r in (True, False))
    assert a["said"] == b["said"] and a["lengths"] == b["lengths"] and a["said_sum"] == b["said_sum"]
    for said, length, prompt in zip(a["said"], a["lengths"], a["prompts"]):
        assert 12 <= len(said) <= 48 and length == prompt + len(said)
        assert all(0 <= t < 512 for t in said)
    assert a["tokens_per_step"] >= 1.0 and a["mean_logprob"] <= 0.0


def test_a_drafted_step_chooses_what_the_network_says():
    """One step of drafts against the same network run over the kept tokens as a plain prompt, in a cache of its own."""
    from paper_2408_02937_amd import answers
    from paper_2408_02937_amd.cache import Cache
    dev = torch.device("cuda:0")
    net = answers.Stack(2, 8, 2, 64, 512, dev, seed=4)
    n, prompt = 3, 40
    g = torch.Generator(device=dev).manual_seed(5)
    ids = torch.randint(0, 512, (n, prompt), device=dev, generator=g)
    ints = lambda v: torch.tensor(list(v), dtype=torch.int32, device=dev)
    cache = Cache(2, 64, layers=2, page_tokens=32, pages=40, max_seqs=n, device=dev)
    seqs = ints(range(n))
    cache.extend(seqs, ints(range(0, n * prompt + 1, prompt)))
    net(cache, ids.flatten(), seqs, ints(range(0, n * prompt + 1, prompt)), prompt)
    d = answers.Drafts(net, cache, seqs, ints([3, 5, 7]), 512)
    held = [list(x) for x in ids.tolist()]
    for step in range(4):
        d.followers.random_(0, 512, generator=g)
        d.step()
        torch.cuda.synchronize()
        drafted, chosen, path = d.drafted.tolist(), d.chosen.tolist(), d.path.tolist()
        for r in range(n):
            held[r] += [drafted[r][j] for j in path[r] if j >= 0]
            c = Cache(2, 64, layers=2, page_tokens=32, pages=20, max_seqs=1, device=dev)
            st = ints([0, len(held[r])])
            c.extend(starts=st)
            x = net(c, torch.tensor(held[r], device=dev), ints([0]), st, len(held[r]))
            logits = (x @ net.tokens.t()).float()
            for i, j in enumerate([j for j in path[r] if j >= 0]):
                row = logits[len(held[r]) - sum(p >= 0 for p in path[r]) + i]
                # two runs of the network in bfloat16: each of its some ten roundings in a row's path is 2^-9 of what it rounds
                assert row[chosen[r][j]] >= row.max() - 20 * 2.0 ** -9 * row.abs().max()
    assert cache.lengths.tolist() == [len(h) for h in held] and cache.poll_error() == 0
