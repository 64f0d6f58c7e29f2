"""The operators of answering by trees of drafted tokens, as cases that can be timed: attention of a tree and attention of a
window with first tokens that stay visible, both over the cache of keys and values in 4 bits, what a drafted step does to the
cache beside the network, and the scores of logits.

A case is a dict of plain values:
  op       "attend": one layer's attention of new rows whose window leaves the first `sinks` positions visible
           "tree":   one layer's attention of drafted rows: each sees what lies before them (window, sinks) and its ancestors
           "accept": a drafted step beside the network: room for the rows, the trees' words and positions, keys and values of all
                     layers written, the path that the model's choices follow, its rows kept, and the last rows read back
           "score":  log probabilities of given tokens, entropy and the most likely tokens of rows of logits
  n        sequences; length: of the longest, with its new rows; ragged: the others are shorter, down to an eighth; new: rows each
  q_heads, kv_heads, head_dim, page (tokens), window, sinks, dtype ("bf16", "f16", "f32"); layers
  rows, vocab, top, tokens (given for each row), scale, masked (nine logits of ten are -inf), pad (elements between rows): of "score"
The plain form keeps 4-bit codes two to a byte in pages of its own, with a step and a lowest value for 32 channels.
"""
import math
import random

import torch

DEV = "cuda:0"
GROUP = 32     # channels that share a step and a lowest value
MOST = 60000.0  # what a channel is clamped to
DRAFTED = 4096  # tokens that drafts are made of
own = False


def _case(name, op, n, length, new, q_heads, kv_heads, head_dim, page, dtype="bf16", ragged=True, window=0, sinks=0, layers=1):
    return {"name": name, "op": op, "n": n, "length": length, "new": new, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "page": page, "dtype": dtype, "ragged": ragged, "window": window, "sinks": sinks, "layers": layers}


def _score(name, rows, vocab, top, tokens, dtype="bf16", scale=1.0, masked=False, pad=0):
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "top": top, "tokens": tokens, "dtype": dtype, "scale": scale,
            "masked": masked, "pad": pad}


def listed():
    return [
        # one interactive token of a session that has outgrown its window: a chain of latencies
        _case("sinks_short", "attend", 1, 333, 1, 8, 2, 64, 64, window=100, sinks=4),
        # a serving batch of long sessions, one token each
        _case("sinks_batch64", "attend", 64, 20_001, 1, 32, 8, 128, 64, window=2048, sinks=4, dtype="f16"),
        # a long prompt read under the window that its answer will have
        _case("sinks_prompt", "attend", 1, 8192, 8192, 32, 8, 128, 128, window=1000, sinks=64),
        # a few drafted tokens behind a short passage
        _case("tree5_short", "tree", 1, 205, 5, 8, 2, 64, 64),
        # a batch of answers, a dozen drafted tokens each
        _case("tree13_batch", "tree", 16, 6001, 13, 32, 8, 128, 64),
        # few requests behind long contexts with wide trees
        _case("tree63_long", "tree", 4, 60_063, 63, 32, 8, 128, 128, dtype="f16"),
        # the step of one request, two layers
        _case("accept_one", "accept", 1, 206, 6, 2, 2, 64, 64, layers=2),
        # a batch with wide trees, many layers
        _case("accept_batch", "accept", 48, 2031, 31, 8, 8, 128, 64, layers=8, dtype="f16"),
        # the next token of one request
        _score("score_one", 1, 4096, 5, 1),
        # the next tokens of a batch over many tokens, logits in 32 bits, at a temperature
        _score("score_batch", 64, 131_072, 20, 1, dtype="f32", scale=1.25),
        # texts that are scored token by token
        _score("score_texts", 4095, 50_001, 0, 1),
        # the rows of drafted trees, of which a grammar allows a tenth
        _score("score_trees", 1000, 32_768, 4, 3, dtype="f16", masked=True, pad=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["attend", "prompt", "tree", "tree", "accept", "score", "score"])
    if op == "score":
        vocab = _log(rng, 300, 200_000)
        rows = _log(rng, 1, min(4096, (1 << 28) // vocab))
        c = _score("", rows, vocab, rng.choice([0, 1, _log(rng, 2, 64)]), rng.choice([0, 1, 1, 4]), rng.choice(["bf16", "f16", "f32"]),
                   rng.choice([1.0, 1.0, 0.7, 1.6]), rng.random() < 0.25, rng.choice([0, 0, 1, 24]))
        if c["top"] == 0 and c["tokens"] == 0:
            c["tokens"] = 1
        return _drop(c)
    dim = rng.choice([64, 96, 128, 256])
    q_heads, kv_heads = rng.choice([(8, 8), (32, 8), (16, 2), (16, 1), (12, 12), (28, 4), (64, 8)])
    page = rng.choice([32, 64, 96, 128, 256])
    dtype = rng.choice(["bf16", "f16"])
    row = kv_heads * dim  # channels of a token
    sinks = rng.choice([1, 4, 4, 16, _log(rng, 1, 300)])
    if op == "prompt":
        n = _log(rng, 1, 8)
        length = _log(rng, 200, 8192 // n if n > 1 else 6000)
        most = int(4 * 10**8 / (q_heads * n * length))  # scores of the plain form
        new = min(length, max(33, min(int(length * rng.choice([1.0, 1.0, 0.5, 0.2])), most)))
        return _drop(_case("", "attend", n, length, new, q_heads, kv_heads, dim, page, dtype, rng.random() < 0.5, _log(rng, 16, 2048), sinks))
    if op == "accept":
        n, layers = _log(rng, 1, 48), _log(rng, 1, 8)
        new = _log(rng, 2, 64)
        length = new + _log(rng, 8, max(64, min(8000, (1 << 28) // (n * layers * row))))
        return _drop(_case("", "accept", n, length, new, kv_heads, kv_heads, dim, page, dtype, True, layers=layers))
    n = _log(rng, 1, 64)
    length = _log(rng, 80, max(100, min(131_072, (1 << 28) // (row * n))))
    if op == "attend":
        return _drop(_case("", "attend", n, length, min(length, rng.choice([1, 1, 1, 2, 5, 16])), q_heads, kv_heads, dim, page, dtype, rng.random() < 0.75,
                           _log(rng, 16, 8192), sinks))
    new = max(2, min(_log(rng, 2, 200), length // 2, int(4 * 10**8 / (q_heads * n * length))))
    window = rng.choice([0, 0, 0, _log(rng, 16, 8192)])
    return _drop(_case("", "tree", n, length, new, q_heads, kv_heads, dim, page, dtype, rng.random() < 0.75, window, sinks if window else 0))


def _drop(c):
    del c["name"]
    return c


# ------------------------------------------------------------------ sizes that follow from a case
def _lengths(case):
    """Of each sequence, its new rows among them."""
    n, top = case["n"], case["length"]
    if not case["ragged"]:
        return [top] * n
    return [max(1, top - (top * 7 * ((i * 37) % 64)) // (64 * 8)) for i in range(n)]


def _new(case):
    return [min(case["new"], x) for x in _lengths(case)]


def _starts(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _pages_of(case, length):
    return -(-length // case["page"])


def _drafted(case):
    return case["op"] in ("tree", "accept")


def _parents(case, seed):
    """Of each sequence's rows: drafts of up to eight branches; a row behind its parent, row 0 in front of all."""
    rng = random.Random(seed * 7919 + 11)
    return [[-1] + [rng.randint(max(0, j - 8), j - 1) for j in range(1, c)] for c in _new(case)]


def _ancestors(parents):
    """Of each row of one tree, itself among them."""
    out = []
    for j, p in enumerate(parents):
        out.append((out[p] if p >= 0 else []) + [j])
    return out


def _tail(case):
    """Rows of each sequence that "accept" reads back."""
    return [min(x - c + 1, c + 3) for x, c in zip(_lengths(case), _new(case))]


def _itemsize(case):
    return 4 if case["dtype"] == "f32" else 2


def work(case):
    if case["op"] == "score":
        rows = case["rows"]
        return {"bytes": rows * (case["vocab"] * _itemsize(case) + 8 * case["tokens"] + 8 * case["top"] + 8.0), "flops": 5.0 * rows * case["vocab"]}
    lengths, new = _lengths(case), _new(case)
    row, dim, heads = case["kv_heads"] * case["head_dim"], case["head_dim"], case["q_heads"]
    if case["op"] == "accept":
        rows, tail = sum(new), sum(_tail(case))  # rows in as they are, into the cache, a third of them moved, the last ones out of it
        return {"bytes": case["layers"] * row * (rows * (4 + 1.25) + rows / 3 * 2.5 + tail * (1.25 + 4)) + 24.0 * rows,
                "flops": 12.0 * case["layers"] * (rows + tail) * row}
    out = {"bytes": 0.0, "flops": 0.0}
    trees = [_ancestors(p) for p in _parents(case, 1)] if case["op"] == "tree" else [None] * case["n"]
    for length, c, tree in zip(lengths, new, trees):
        base, seen, low = length - c, 0, length
        for j in range(c):
            path = len(tree[j]) if tree else j + 1
            first = max(0, base + path - case["window"]) if case["window"] else 0
            first = min(first, base) if tree else first
            head = min(case["sinks"], first)
            seen += (base - first + path if tree else base + path - first) + head
            low = min(low, first)
        held = length - low + min(case["sinks"], low)
        out["bytes"] += held * row * 1.25 + 2 * c * heads * dim * 2
        out["flops"] += 4.0 * seen * heads * dim
    return out


# ------------------------------------------------------------------ inputs
def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(seed * 1_000_003 + stream)


def _dtype(case):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[case["dtype"]]


def _rows(case, seed, stream, rows, spread):
    """Keys or values: channels have means and widths of their own."""
    g = _gen(seed, stream)
    shape = (case["kv_heads"], case["head_dim"])
    mean = torch.randn(shape, device=DEV, generator=g) * 0.5
    width = torch.exp(torch.randn(shape, device=DEV, generator=g) * spread)
    x = torch.empty((rows, *shape), device=DEV, dtype=_dtype(case))
    piece = max(1, (1 << 28) // (shape[0] * shape[1]))
    for at in range(0, rows, piece):
        m = min(piece, rows - at)
        x[at:at + m] = torch.randn((m, *shape), device=DEV, generator=g) * width + mean
    return x


def _queries(case, seed, rows):
    g = _gen(seed, 3)
    return (torch.randn((rows, case["q_heads"], case["head_dim"]), device=DEV, generator=g) * 1.5).to(_dtype(case))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _words(case, seed):
    """Bit i of a row's words: it sees row i of its item."""
    wide, flat = -(-max(_new(case)) // 32), []
    for parents in _parents(case, seed):
        for seen in _ancestors(parents):
            w = [0] * wide
            for i in seen:
                w[i // 32] |= 1 << (i % 32)
            flat.append([x - (1 << 32) if x >> 31 else x for x in w])
    return _ints(flat)


def _logits(case, seed):
    g = _gen(seed, 8)
    x = torch.empty((case["rows"], case["vocab"] + case["pad"]), dtype=_dtype(case), device=DEV)[:, :case["vocab"]]
    piece = max(1, (1 << 26) // case["vocab"])
    for at in range(0, case["rows"], piece):
        m = min(piece, case["rows"] - at)
        f = torch.randn((m, case["vocab"]), device=DEV, generator=g)
        f = f * 2.0 + f * f * f * 0.3  # a few stand out
        if case["masked"]:
            f.masked_fill_(torch.rand((m, case["vocab"]), device=DEV, generator=g) < 0.9, float("-inf"))
        x[at:at + m] = f
    return x


def prepare(case, seed):
    if case["op"] == "score":
        g = _gen(seed, 9)
        given = torch.randint(0, case["vocab"], (case["rows"], case["tokens"]), dtype=torch.int32, device=DEV, generator=g) if case["tokens"] else None
        return {"case": case, "logits": _logits(case, seed), "given": given}
    return _prepare_cache(case, seed)


def _held_rows(case, seed):
    """(keys, values) of all that the cache holds before a pass, by layer."""
    lengths, new = _lengths(case), _new(case)
    rows = sum(lengths) if case["op"] != "accept" else sum(lengths) - sum(new)
    return [(_rows(case, seed, 20 + 4 * i, rows, 0.4), _rows(case, seed, 21 + 4 * i, rows, 0.2)) for i in range(case["layers"])]


def _drafted_rows(case, seed):
    """(keys, values) that "accept" writes, by layer."""
    rows = sum(_new(case))
    return [(_rows(case, seed, 22 + 4 * i, rows, 0.4), _rows(case, seed, 23 + 4 * i, rows, 0.2)) for i in range(case["layers"])]


def _choices(case, seed):
    """(drafted token of each row, token that the model chose behind it): three times of four that of a child."""
    rng = random.Random(seed * 104_729 + 5)
    drafted, chosen = [], []
    for parents in _parents(case, seed):
        t = [rng.randrange(DRAFTED) for _ in parents]
        c = [rng.randrange(DRAFTED) for _ in parents]
        for j in range(len(parents) - 1, 0, -1):
            if rng.random() < 0.75:
                c[parents[j]] = t[j]
        drafted += t
        chosen += c
    return drafted, chosen


def _prepare_cache(case, seed):
    lengths, new = _lengths(case), _new(case)
    accept = case["op"] == "accept"
    held = [x - c for x, c in zip(lengths, new)] if accept else lengths
    s = {"case": case, "lengths": lengths, "max_new": max(new), "starts": None if max(new) == 1 else _ints(_starts(new)), "scale": case["head_dim"] ** -0.5}
    if accept:
        s["starts"] = _ints(_starts(new))
        s["rows"] = _drafted_rows(case, seed)
        s["parents"] = _ints(sum(_parents(case, seed), []))
        s["drafted"], s["chosen"] = (_ints(x) for x in _choices(case, seed))
        s["before"] = _ints(held)
        s["tail"] = _tail(case)
        s["tail_starts"] = _ints(_starts(s["tail"]))
    else:
        s["q"] = _queries(case, seed, sum(new))
    if case["op"] == "tree":
        s["tree"] = _words(case, seed)
    wide, pages = _pages_of(case, max(lengths)), sum(_pages_of(case, x) for x in lengths) + case["n"]
    every = _ints(_starts(held))
    rows = _held_rows(case, seed)
    if own:
        from paper_2408_02937_amd.cache import Cache
        c = s["cache"] = Cache(case["kv_heads"], case["head_dim"], layers=case["layers"], page_tokens=case["page"], pages=pages, max_seqs=case["n"], max_pages=wide, device=DEV)
        c.extend(starts=_ints(_starts([x // 2 for x in held])))  # in two turns, so that pages of different sequences lie side by side
        c.extend(starts=_ints(_starts([x - x // 2 for x in held])))
        for i, (k, v) in enumerate(rows):
            if max(held):
                c.write(i, k, v, starts=every, max_new=max(held))
        return s
    order = torch.randperm(pages, device=DEV, generator=_gen(seed, 6)).to(torch.int32)
    table = torch.full((case["n"], wide), -1, dtype=torch.int32, device=DEV)
    within = torch.arange(wide, device=DEV)[None, :] < torch.tensor([_pages_of(case, x) for x in lengths], device=DEV)[:, None]
    table[within] = order[: int(within.sum())]
    s["table"], s["length"] = table, torch.tensor(held, device=DEV)
    slots = _slots(s, torch.repeat_interleave(torch.arange(case["n"], device=DEV), s["length"]),
                   torch.arange(sum(held), device=DEV) - torch.repeat_interleave(every[:-1].long(), s["length"]))
    heads, dim = case["kv_heads"], case["head_dim"]
    s["codes"] = torch.zeros((case["layers"], 2, pages * case["page"], heads, dim // 2), dtype=torch.uint8, device=DEV)
    s["meta"] = torch.zeros((case["layers"], 2, pages * case["page"], heads, dim // GROUP, 2), dtype=torch.float16, device=DEV)
    piece = max(1, (1 << 28) // (heads * dim))
    for i, kv in enumerate(rows):
        for which in (0, 1):
            for at in range(0, sum(held), piece):
                _put(s, i, which, slots[at:at + piece], kv[which][at:at + piece])
    return s


# ------------------------------------------------------------------ the plain form
def _quantised(x):
    """(codes two to a byte, (step, lowest value)) of rows [...][head_dim]."""
    f = torch.nan_to_num(x.float(), nan=0.0, posinf=MOST, neginf=-MOST).clamp(-MOST, MOST)
    f = f.reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = f.amin(-1), f.amax(-1)
    step, zero = ((hi - lo) / 15.0).half(), lo.half()
    inv = torch.where(step > 0, 1.0 / step.float(), torch.zeros_like(lo))
    code = torch.round((f - zero.float()[..., None]) * inv[..., None]).clamp(0.0, 15.0).to(torch.uint8).reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.stack([step, zero], -1)


def _values(codes, meta):
    """Back again, in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1, GROUP).float()
    m = meta.float()
    return (c * m[..., 0:1] + m[..., 1:2]).reshape(*codes.shape[:-1], -1)


def _slots(s, seq, pos):
    page = s["case"]["page"]
    return s["table"][seq, pos // page].long() * page + pos % page


def _put(s, layer, which, slots, x):
    codes, meta = _quantised(x)
    s["codes"][layer, which, slots] = codes
    s["meta"][layer, which, slots] = meta


def _of_rows(case, length):
    """Sequence and place among its sequence's new rows, of each new row, and new rows of each sequence."""
    count = torch.clamp(torch.full_like(length, case["new"]), max=length)
    seq = torch.repeat_interleave(torch.arange(case["n"], device=DEV), count)
    return seq, torch.arange(seq.numel(), device=DEV) - (torch.cumsum(count, 0) - count)[seq], count


def _attend(s):
    case, length = s["case"], s["length"]
    n, heads, kv, dim, sinks, window = case["n"], case["q_heads"], case["kv_heads"], case["head_dim"], case["sinks"], case["window"]
    seq, nth, count = _of_rows(case, length)
    base, most, longest = length - count, s["max_new"], max(s["lengths"])
    # positions that some row may see: the first ones, and from the first row's window on
    if window and window + most + sinks < longest:
        first = (base - window + 1).clamp(min=0)
        t = torch.cat([torch.arange(sinks, device=DEV).expand(n, -1), first[:, None] + torch.arange(window + most, device=DEV)], 1)
        there = t < length[:, None]
        there[:, :sinks] &= t[:, :sinks] < first[:, None]
    else:
        t = torch.arange(longest, device=DEV).expand(n, -1)
        there = t < length[:, None]
    slot = _slots(s, torch.arange(n, device=DEV)[:, None], torch.where(there, t, torch.zeros_like(t)))
    k = _values(s["codes"][0, 0, slot], s["meta"][0, 0, slot]).permute(0, 2, 3, 1).contiguous()  # [n][kv][dim][t]
    v = _values(s["codes"][0, 1, slot], s["meta"][0, 1, slot]).permute(0, 2, 1, 3).contiguous()  # [n][kv][t][dim]
    q = torch.zeros((n, most, heads, dim), device=DEV)
    q[seq, nth] = s["q"].float()
    # what each row sees, [n][most][t]
    if case["op"] == "tree":
        bits = ((s["tree"][:, :, None] >> torch.arange(32, device=DEV)) & 1).flatten(1)[:, :most] > 0
        seen = torch.zeros((n, most, most), dtype=torch.bool, device=DEV)
        seen[seq, nth] = bits
        at = base[:, None] + seen.sum(-1) - 1
        behind = t - base[:, None]
        among = torch.gather(seen, 2, behind.clamp(0, most - 1)[:, None, :].expand(-1, most, -1))
        new = (behind >= 0)[:, None, :]
    else:
        at = base[:, None] + torch.arange(most, device=DEV)
        new, among = torch.zeros((), dtype=torch.bool, device=DEV), torch.zeros((), dtype=torch.bool, device=DEV)
    see = there[:, None, :] & (t[:, None, :] <= at[:, :, None])
    if window:
        see = see & ((t[:, None, :] > at[:, :, None] - window) | (t < sinks)[:, None, :])
    see = torch.where(new, among & there[:, None, :], see)
    q = q.reshape(n, most, kv, heads // kv, dim).permute(0, 2, 1, 3, 4).reshape(n, kv, -1, dim)
    score = torch.matmul(q, k).mul_(s["scale"]).reshape(n, kv, most, heads // kv, -1)
    score.masked_fill_(~see[:, None, :, None, :], float("-inf"))
    m = score.amax(-1, keepdim=True)
    score = score.sub_(torch.where(torch.isinf(m), torch.zeros_like(m), m)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.reshape(n, kv, -1, t.shape[1]), v).reshape(n, kv, most, heads // kv, dim)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 2, 1, 3, 4).reshape(n, most, heads, dim)
    return {"out": o[seq, nth].to(_dtype(case))}


def _accept(s):
    case = s["case"]
    n, most = case["n"], s["max_new"]
    counts = torch.diff(s["starts"]).long()
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), counts)
    nth = torch.arange(seq.numel(), device=DEV) - s["starts"][seq].long()
    base = s["before"].long()
    slots = _slots(s, seq, base[seq] + nth)
    for i, (k, v) in enumerate(s["rows"]):
        _put(s, i, 0, slots, k)
        _put(s, i, 1, slots, v)
    # rows that each row sees: parents' parents, twice as far each time
    real = torch.zeros((n, most), dtype=torch.bool, device=DEV)
    real[seq, nth] = True
    pad = lambda x, fill: torch.full((n, most), fill, dtype=torch.long, device=DEV).index_put_((seq, nth), x.long())
    parent, drafted, chosen = pad(s["parents"], -1), pad(s["drafted"], -1), pad(s["chosen"], -2)
    rows = torch.arange(most, device=DEV)
    reach = ((parent[:, :, None] == rows) | (rows[:, None] == rows)).float()
    for _ in range(max(1, most - 1).bit_length()):
        reach = (torch.bmm(reach, reach) > 0).float()
    reach = (reach > 0) & real[:, :, None]
    wide = -(-most // 32)
    bits = torch.nn.functional.pad(reach, (0, wide * 32 - most)).reshape(n, most, wide, 32).long()
    words = (bits << torch.arange(32, device=DEV)).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)[seq, nth]
    positions = (base[:, None] + reach.sum(-1) - 1).to(torch.int32)[seq, nth]
    # a row is on the path where it and its ancestors, but the first row, are the first children with the token that was chosen
    right = (parent >= 0) & (drafted == torch.gather(chosen, 1, parent.clamp(min=0)))
    earlier = (parent[:, :, None] == parent[:, None, :]) & right[:, None, :] & (rows[:, None] > rows)
    good = (right & ~earlier.any(-1)) | (rows == 0)
    on = real & ~(reach & ~good[:, None, :]).any(-1) & (reach[:, :, 0])
    kept = on.sum(-1)
    path = torch.where(on, rows, torch.full_like(rows, most)).sort(-1).values
    path = torch.where(path < most, path, torch.full_like(path, -1))
    last = torch.gather(path, 1, (kept - 1)[:, None])
    following = torch.gather(chosen, 1, last).squeeze(1).to(torch.int32)
    # its rows move to the front
    held = path >= 0
    item = torch.arange(n, device=DEV)[:, None].expand(-1, most)[held]
    src = _slots(s, item, base[item] + path[held])
    dst = _slots(s, item, base[item] + rows.expand(n, -1)[held])
    s["codes"][:, :, dst] = s["codes"][:, :, src]
    s["meta"][:, :, dst] = s["meta"][:, :, src]
    length = base + kept
    tail = torch.diff(s["tail_starts"]).long()
    seq2 = torch.repeat_interleave(torch.arange(n, device=DEV), tail)
    back = length[seq2] - tail[seq2] + torch.arange(seq2.numel(), device=DEV) - s["tail_starts"][seq2].long()
    slots = _slots(s, seq2, back)
    out = _values(s["codes"][:, :, slots], s["meta"][:, :, slots]).half()
    return {"words": words, "positions": positions, "path": path[seq, nth].to(torch.int32), "kept": kept.to(torch.int32), "following": following,
            "length": length.to(torch.int32), "rows": [(out[i, 0], out[i, 1]) for i in range(case["layers"])]}


def _scores(s):
    case, x = s["case"], s["logits"].float()
    out = {}
    if case["top"]:
        # whole numbers in the order of the logits, and of two alike the lower index in front
        i = (x + 0.0).view(torch.int32)
        key = ((i ^ ((i >> 31) & 0x7fffffff)).long() << 32) + torch.arange(case["vocab"] - 1, -1, -1, device=DEV)
        at = case["vocab"] - 1 - (torch.topk(key, case["top"]).values & 0xffffffff)
        best = torch.gather(x, 1, at)
        out["top"] = torch.where(torch.isinf(best), torch.full_like(at, -1), at).to(torch.int32)
    x = x * case["scale"]
    m = x.amax(-1, keepdim=True)
    z = x - m
    e = z.exp()
    total = e.sum(-1)
    log_total = total.log()
    out["entropy"] = log_total - (e * torch.where(e > 0, z, torch.zeros_like(z))).sum(-1) / total
    if case["tokens"]:
        out["logprobs"] = torch.gather(z, 1, s["given"].long()) - log_total[:, None]
    if case["top"]:
        out["top_logprobs"] = best * case["scale"] - m - log_total[:, None]
    return out


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return _scores(s) if op == "score" else _accept(s) if op == "accept" else _attend(s)
    if op == "score":
        from paper_2408_02937_amd.logits import score
        r = score(s["logits"], s["given"], top=case["top"], scale=case["scale"])
        out = {}
        if case["top"]:
            out["top"] = r.top
        out["entropy"] = r.entropy
        if case["tokens"]:
            out["logprobs"] = r.logprobs
        if case["top"]:
            out["top_logprobs"] = r.top_logprobs
        return out
    c = s["cache"]
    if op != "accept":
        return {"out": c.attend(0, s["q"], starts=s["starts"], max_new=s["max_new"], scale=s["scale"], window=case["window"], sinks=case["sinks"], tree=s.get("tree"))}
    c.trim(lengths=s["before"])
    c.extend(starts=s["starts"])
    words, positions = c.tree(s["parents"], starts=s["starts"], max_new=s["max_new"])
    for i, (k, v) in enumerate(s["rows"]):
        c.write(i, k, v, starts=s["starts"], max_new=s["max_new"])
    path, kept, following = c.walk(s["parents"], s["drafted"], s["chosen"], starts=s["starts"], max_new=s["max_new"])
    c.keep(path, kept, starts=s["starts"], max_new=s["max_new"])
    rows = [c.read(i, sum(s["tail"]), starts=s["tail_starts"], max_new=max(s["tail"]), dtype=torch.float16) for i in range(case["layers"])]
    return {"words": words, "positions": positions, "path": path, "kept": kept, "following": following, "length": c.lengths, "rows": rows}


# ------------------------------------------------------------------ the same in 64 bits, from the definition
def _held(x):
    """What the cache stands for after x went in: one of 16 values between a group's lowest and highest."""
    x = x.double()
    x[x.isnan()] = 0.0
    g = x.clamp_(-MOST, MOST).unflatten(-1, (-1, GROUP))
    low = g.min(-1, keepdim=True).values
    width = ((g.max(-1, keepdim=True).values - low) / 15).float().half().double()
    low = low.half().double()
    level = torch.where(width > 0, (g - low) / width.clamp(min=1e-30), torch.zeros_like(g)).round().clamp(0, 15)
    return (low + width * level).flatten(-2)


def exact(case, seed):
    if case["op"] == "score":
        return _exact_scores(case, seed)
    lengths, new = _lengths(case), _new(case)
    if case["op"] == "accept":
        return _exact_accept(case, seed)
    k, v = _held_rows(case, seed)[0]
    q = _queries(case, seed, sum(new)).double() * case["head_dim"] ** -0.5
    out = torch.zeros_like(q)
    share = case["q_heads"] // case["kv_heads"]
    trees = [_ancestors(p) for p in _parents(case, seed)] if case["op"] == "tree" else [None] * case["n"]
    row = at = 0
    for length, c, tree in zip(lengths, new, trees):
        ks, vs = k[row:row + length], v[row:row + length]
        row += length
        base = length - c
        t = torch.arange(length, device=DEV)
        pos = torch.tensor([base + len(x) - 1 for x in tree] if tree else list(range(base, length)), device=DEV)[:, None]
        see = t <= pos
        if case["window"]:
            see &= (t > pos - case["window"]) | (t < case["sinks"])
        if tree:
            see[:, base:] = False
            see[[j for j, x in enumerate(tree) for _ in x], [base + i for x in tree for i in x]] = True
        for h in range(case["kv_heads"]):
            kh, vh = _held(ks[:, h]), _held(vs[:, h])
            for j in range(share):
                w = q[at:at + c, h * share + j] @ kh.t()
                w = torch.softmax(w.masked_fill_(~see, float("-inf")), -1)
                out[at:at + c, h * share + j] = w @ vh
        at += c
    return {"out": out}


def _exact_accept(case, seed):
    lengths, new, tail = _lengths(case), _new(case), _tail(case)
    held, drafted = _held_rows(case, seed), _drafted_rows(case, seed)
    tokens, chosen = _choices(case, seed)
    before, fresh = _starts([x - c for x, c in zip(lengths, new)]), _starts(new)
    old_at, new_at = [], []  # for each row that is read back: its place among the held rows, or among the drafted ones
    for i, parents in enumerate(_parents(case, seed)):
        at, path = fresh[i], [0]
        while True:
            child = [j for j in range(len(parents)) if parents[j] == path[-1] and tokens[at + j] == chosen[at + path[-1]]]
            if not child:
                break
            path.append(child[0])
        rows = [(x, -1) for x in range(before[i], before[i + 1])] + [(-1, at + j) for j in path]
        for x, y in rows[len(rows) - tail[i]:]:
            old_at.append(x)
            new_at.append(y)
    old_at, new_at = torch.tensor(old_at, device=DEV), torch.tensor(new_at, device=DEV)
    pick = lambda a, b: torch.where((old_at >= 0)[:, None, None], a[old_at.clamp(min=0)], b[new_at.clamp(min=0)])
    rows = [(_held(pick(k0, k1)), _held(pick(v0, v1))) for (k0, v0), (k1, v1) in zip(held, drafted)]
    return {"words": None, "positions": None, "path": None, "kept": None, "following": None, "length": None, "rows": rows}


def _exact_scores(case, seed):
    x = _logits(case, seed)
    given = prepare(case, seed)["given"] if case["tokens"] else None
    out = {"entropy": torch.zeros(case["rows"], dtype=torch.float64, device=DEV)}
    if case["top"]:
        out = {"top": None, **out}
    if case["tokens"]:
        out["logprobs"] = torch.zeros((case["rows"], case["tokens"]), dtype=torch.float64, device=DEV)
    if case["top"]:
        out["top_logprobs"] = torch.zeros((case["rows"], case["top"]), dtype=torch.float64, device=DEV)
    piece = max(1, (1 << 25) // case["vocab"])
    for at in range(0, case["rows"], piece):
        to = min(case["rows"], at + piece)
        p = torch.log_softmax(x[at:to].double() * case["scale"], -1)
        out["entropy"][at:to] = torch.special.entr(p.exp()).sum(-1)
        if case["tokens"]:
            out["logprobs"][at:to] = torch.gather(p, 1, given[at:to].long())
        if case["top"]:
            out["top_logprobs"][at:to] = p.sort(-1, descending=True).values[:, :case["top"]]
    return out
