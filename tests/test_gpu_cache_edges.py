"""The cache where its calls could go wrong at the edges of what they take: sums beyond 32 bits, items that are not what a call asks for, probabilities
far below the largest, arguments that another stream reads, strides that say nothing.  Plain implementations and bounds: test_gpu_cache.py."""
import numpy as np
import pytest
import torch

from paper_2408_02937_amd import rtams
from paper_2408_02937_amd.cache import Cache
from tests.test_gpu_cache import DEV, Filled, check_attention, floats, ints, starts_of, unit_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ pages
def test_copies_of_a_long_sequence_are_counted_beyond_32_bits():
    """1,024 copies of 2^22 pages are 2^32, of a page more 2^32 + 1,024: far more than are free, and nothing changes."""
    n, long = 1024, 1 << 22
    c = Cache(1, 64, page_tokens=32, pages=long + 2000, max_seqs=n + 1, max_pages=long + 1, device=DEV)
    c.extend(ints([0]), ints([0, long * 32]))
    for _ in range(2):
        free = c.free_pages
        refs = c.refs.clone()
        c.fork(ints([0] * n), ints(range(1, n + 1)), copy=True)
        torch.cuda.synchronize()
        assert c.poll_error() == rtams.EPOOL and c.free_pages == free
        assert torch.equal(c.refs, refs) and not c.lengths[1:].any() and (c.table[1:, :3] == -1).all() and (c.table[1:, -3:] == -1).all()
        c.clear_error()
        c.extend(ints([0]))  # the last page
    assert c.free_pages == 1999
    c.trim(ints([0]), ints([5 * 32]))  # ... and what there is room for is copied
    c.fork(ints([0] * n), ints(range(1, n + 1)), copy=True)
    torch.cuda.synchronize()
    assert c.poll_error() == 0 and c.free_pages == long + 2000 - 5 * (n + 1)
    assert c.table[1:, :5].flatten().tolist() == list(range(5, 5 * (n + 1)))


# ------------------------------------------------------------------ items that attention refuses
@pytest.mark.parametrize("lengths,counts,heads,kv,dim", [([0, 40, 9], [1, 1, 1], 4, 2, 64), ([3, 40, 0], [5, 5, 2], 4, 2, 128), ([3, 70], [17, 16], 4, 1, 256),
                                                         ([30, 200, 64], [90, 100, 65], 4, 2, 64), ([69, 300], [70, 70], 2, 2, 256)])
@pytest.mark.parametrize("window", [0, 20])
def test_more_causal_rows_than_tokens_are_refused_and_left(lengths, counts, heads, kv, dim, window):
    """The item's rows and logarithms stay what they were, the other items' are theirs; without a causal mask rows have no places and any number is answered."""
    f = Filled(lengths, kv, dim, seed=40)
    q = f.query(counts, heads)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 5.0, device=DEV)
    at = np.concatenate([[0], np.cumsum(counts)])
    one = all(c == 1 for c in counts)
    args = (ints(range(len(lengths))), None if one else starts_of(counts), None if one else max(counts))
    f.cache.attend(0, q, *args, window=window, out=out, lse=lse)
    torch.cuda.synchronize()
    assert f.cache.poll_error() == rtams.EINVAL
    f.cache.clear_error()
    want = f.want(q, counts, dim ** -0.5, window=window)
    for i, (n, c) in enumerate(zip(lengths, counts)):
        rows = slice(at[i], at[i + 1])
        if c > n:
            assert (out[rows] == 7.0).all() and (lse[rows] == 5.0).all(), i
        else:
            check_attention(out[rows], lse[rows], [x[rows] for x in want], unit_of(q.dtype))
    if not window:
        out = f.cache.attend(0, q, *args, causal=False, lse=lse)
        check_attention(out, lse, f.want(q, counts, dim ** -0.5, causal=False), unit_of(q.dtype))
        assert f.cache.poll_error() == 0


def test_more_causal_rows_than_tokens_among_many_prompts():
    lengths = [(i * 37) % 90 + 40 for i in range(300)]
    f = Filled(lengths, 4, 64, page=32, seed=41)
    counts = [36 + i % 9 for i in range(300)]
    counts[7], counts[299] = lengths[7] + 1, lengths[299] + 30
    q = f.query(counts, 8)
    out = torch.full_like(q, 7.0)
    f.cache.attend(0, q, starts=starts_of(counts), max_new=max(counts), out=out)
    torch.cuda.synchronize()
    assert f.cache.poll_error() == rtams.EINVAL
    at = np.concatenate([[0], np.cumsum(counts)])
    for i in range(300):
        assert bool((out[at[i]:at[i + 1]] == 7.0).all()) == (i in (7, 299)), i


# ------------------------------------------------------------------ sequences named twice
@pytest.mark.parametrize("n", [2, 5, 257, 300, 1024, 1025, 1500])
@pytest.mark.parametrize("single", [True, False])
def test_a_sequence_named_twice_is_not_written(n, single):
    """Its items are left out, with an error; the others are written."""
    rng = np.random.default_rng(n)
    c = Cache(2, 64, page_tokens=32, pages=n, max_seqs=n, max_pages=1, device=DEV)
    length = 5
    every = starts_of([length] * n)
    g = torch.Generator(device=DEV).manual_seed(n)
    old = [torch.randn((n * length, 2, 64), device=DEV, generator=g).half() for _ in range(2)]
    c.extend(starts=every)
    c.write(0, *old, starts=every, max_new=length)
    was = [x.view(n, length, 2, 64).clone() for x in c.read(0, n * length, starts=every, max_new=length)]
    seqs = rng.permutation(n)
    seqs[n - 1] = seqs[0]
    if n > 4:
        seqs[n // 2] = seqs[n // 2 - 1]
    counts = [1] * n if single else [int(x) for x in rng.integers(0, length + 1, n)]
    counts[0] = counts[n - 1] = 1 if single else 3
    new = [torch.randn((sum(counts), 2, 64), device=DEV, generator=g).half() for _ in range(2)]
    args = (ints(seqs), None if single else starts_of(counts), length)
    c.write(0, *new, *args)
    got = [x.view(n, length, 2, 64) for x in c.read(0, n * length, starts=every, max_new=length)]
    torch.cuda.synchronize()
    assert c.poll_error() == rtams.EINVAL
    c.clear_error()
    twice = {s for s in seqs if (seqs == s).sum() > 1}
    alone = [x.clone() for x in was]
    at = 0
    for s, m in zip(seqs, counts):
        if s not in twice and m:
            one = Cache(2, 64, page_tokens=32, pages=1, max_seqs=1, device=DEV) if s == seqs[1] else None
            if one is not None:  # (what a single sequence's write leaves)
                one.extend(starts=ints([0, m]))
                one.write(0, *(x[at:at + m] for x in new), starts=ints([0, m]), max_new=m)
                for x, y in zip(alone, one.read(0, m, starts=ints([0, m]), max_new=m)):
                    assert torch.equal(got[0 if x is alone[0] else 1][s, length - m:], y)
            for x, y in zip(alone, got):
                assert not torch.equal(x[s, length - m:], y[s, length - m:])
                x[s, length - m:] = y[s, length - m:]
        at += m
    for x, y in zip(alone, got):  # nothing else changed
        assert torch.equal(x, y)
    some = rng.permutation(n)[:max(1, n - 1)]
    c.write(0, old[0][:len(some)], old[1][:len(some)], ints(some))
    torch.cuda.synchronize()
    assert c.poll_error() == 0


# ------------------------------------------------------------------ numbers
UP = 7  # a row's largest probability is at least 2^UP when it is rounded to a half


@pytest.mark.parametrize("depth", [12.0, 20.0, 24.5, 25.2, 28.0])
@pytest.mark.parametrize("dim,count", [(64, 1), (64, 40), (64, 90), (96, 1), (96, 70), (128, 1), (128, 90), (256, 1), (256, 20), (256, 70)])
@pytest.mark.parametrize("spread", [0.0, 1.0])
def test_a_long_tail_behind_a_sink(dim, count, depth, spread):
    """One token with nearly all the weight and a value of 0; what comes out is the tail's, whose probabilities are 2^-depth of it (spread: a factor of two
    among them).  A half of 2^UP times that is off by 2^-25 at most, and by 2^-11 of itself; scores of up to 25 in 32 bits are off by 2^-20."""
    tokens = 64
    g = np.random.default_rng(int(depth * 10) + dim)
    c = -(depth + spread * (g.random(tokens) - 0.5)) * np.log(2) / dim
    c[0] = 0.0
    k = torch.tensor(c, device=DEV).half()[:, None, None].expand(tokens, 1, dim).contiguous()
    v = torch.full((tokens, 1, dim), 1024.0, dtype=torch.float16, device=DEV)
    v[0] = 0.0
    cache = Cache(1, dim, page_tokens=64, pages=1, max_seqs=1, device=DEV)
    st = ints([0, tokens])
    cache.extend(starts=st)
    cache.write(0, k, v, starts=st, max_new=tokens)
    q = torch.ones((count, 1, dim), dtype=torch.float16, device=DEV)
    lse = torch.empty((count, 1), device=DEV)
    out = cache.attend(0, q, starts=ints([0, count]), max_new=count, scale=1.0, causal=False, lse=lse).double().cpu().numpy()
    p = np.exp(floats(k[:, 0, 0]).astype(np.float64) * dim)
    want = 1024.0 * p[1:].sum() / p.sum()
    rel = 2.0 ** -25 / (2.0 ** UP * p[1:].min()) if 2.0 ** UP * p[1:].min() < 2.0 ** -14 else 2.0 ** -11
    assert rel < 0.2
    bound = want * (rel + 2.0 ** -11 + 2.0 ** -16) + 2.0 ** -25  # (the last: of an output that is below a half's normal range)
    assert np.abs(out - want).max() <= bound, (out.flat[0], want)
    assert abs(lse.cpu().numpy() - np.log(p.sum())).max() <= 2.0 ** -16 + 2.0 ** -10 * p[1:].sum()


def test_a_long_tail_adds_up():
    """Thousands of tokens behind a sink, each of them below a half's normal range at 2^UP times its probability: their sum is in the logarithm.  A
    half below the normal range is off by 2^-25, as often up as down; what is left of that in a sum of so many is far less than all off alike, the bound."""
    tokens, heads, dim, depth = 4097, 256, 64, 22.3
    c = np.full(tokens, -depth * np.log(2) / dim)
    c[0] = 0.0
    k = torch.tensor(c, device=DEV).half()[:, None, None].expand(tokens, heads, dim).contiguous()
    v = torch.full((tokens, heads, dim), 1024.0, dtype=torch.float16, device=DEV)
    v[0] = 0.0
    cache = Cache(heads, dim, page_tokens=64, pages=65, max_seqs=1, device=DEV)
    st = ints([0, tokens])
    cache.extend(starts=st)
    cache.write(0, k, v, starts=st, max_new=tokens)
    p = np.exp(floats(k[:, 0, 0]).astype(np.float64) * dim)
    tail = p[1:].sum()
    rel = 2.0 ** -25 / (2.0 ** UP * p[1])
    assert 2.0 ** UP * p[1] < 2.0 ** -14 and rel < 2.0 ** -9 and tail > 2.0 ** -11
    for count in (1, 70):
        q = torch.ones((count, heads, dim), dtype=torch.float16, device=DEV)
        lse = torch.empty((count, heads), device=DEV)
        out = cache.attend(0, q, starts=ints([0, count]), max_new=count, scale=1.0, causal=False, lse=lse).double().cpu().numpy()
        assert np.abs(lse.double().cpu().numpy() - np.log1p(tail)).max() <= rel * tail + 2.0 ** -16
        want = 1024.0 * tail / (1 + tail)
        assert np.abs(out - want).max() <= want * (rel + 2.0 ** -11 + 2.0 ** -16)


# ------------------------------------------------------------------ streams
@pytest.mark.parametrize("call", ["extend", "write", "read", "attend", "fork", "trim"])
def test_what_another_stream_reads_is_not_given_out_again(call):
    """Arguments that die right after a call on a stream that is busy: their memory is not a new tensor's."""
    f = Filled([300, 200], 2, 64, seed=42, max_seqs=4, extra_pages=20)
    s = torch.cuda.Stream()
    a = torch.randn((4096, 4096), device=DEV)
    b = torch.empty_like(a)
    q, k, v = f.query([1, 1], 4), f.k[:2].clone(), f.v[:2].clone()
    x, y, st = ints([0, 1]), ints([2, 3]), ints([0, 1, 2])
    lens = ints([300, 200])
    out, lse = torch.empty_like(q), torch.empty((2, 4), device=DEV)
    with torch.cuda.stream(s):  # everything has run once
        torch.mm(a, a, out=b)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(1500):
            torch.mm(a, a, out=b)
    done = torch.cuda.Event()
    given = {"extend": lambda: (f.cache.extend(x, st, stream=s), [x, st]),
             "write": lambda: (f.cache.write(0, k, v, x, st, max_new=1, stream=s), [k, v, x, st]),
             "read": lambda: (f.cache.read(0, 2, x, st, max_new=1, stream=s), [x, st]),
             "attend": lambda: (f.cache.attend(0, q, x, st, max_new=1, out=out, lse=lse, stream=s), [q, x, st, out, lse]),
             "fork": lambda: (f.cache.fork(x, y, stream=s), [x, y]),
             "trim": lambda: (f.cache.trim(x, lens, stream=s), [x, lens])}[call]
    result, mine = given()
    at = [(t.data_ptr(), t.numel() * t.element_size()) for t in mine]
    del result, mine, given, q, k, v, x, y, st, lens, out, lse
    done.record(s)
    fresh = [torch.empty(n, dtype=torch.uint8, device=DEV) for _, n in at for _ in range(500)]
    again = {t.data_ptr() for t in fresh} & {p for p, _ in at}
    assert not done.query(), "the stream was to be busy all the while"
    torch.cuda.synchronize()
    assert not again
    assert f.cache.poll_error() == 0


@pytest.mark.parametrize("call", ["read", "attend"])
def test_outputs_on_another_stream_take_no_memory_that_is_still_read(call):
    """A tensor that the current stream has yet to read is dropped: its memory is not the output's that another stream writes at once; and an output that
    the current stream has yet to read is dropped: the other stream does not get it again."""
    rows, heads = 4000, 8
    f = Filled([rows], heads, 64, page=64, seed=47)
    st = ints([0, rows])
    s = torch.cuda.Stream()
    run = {"attend": lambda: f.cache.attend(0, f.k, starts=st, max_new=rows, stream=s), "read": lambda: f.cache.read(0, rows, starts=st, max_new=rows, dtype=torch.bfloat16, stream=s)[0]}[call]
    want = run()
    a = torch.randn((4096, 4096), device=DEV)
    b = torch.mm(a, a)
    torch.cuda.synchronize()
    x = torch.full_like(want, 3.0)
    at = x.data_ptr()
    for _ in range(200):
        torch.mm(a, a, out=b)
    y = x.clone()
    del x
    got = run()
    assert got.data_ptr() != at
    s.synchronize()
    del want
    for _ in range(200):
        torch.mm(a, a, out=b)
    z, at = got.clone(), got.data_ptr()
    del got
    more = [run() for _ in range(4)]
    assert not torch.cuda.current_stream().query(), "the stream was to be busy all the while"
    assert at not in {t.data_ptr() for t in more}
    torch.cuda.synchronize()
    assert (y == 3.0).all() and torch.equal(z, more[0]) and f.cache.poll_error() == 0


# ------------------------------------------------------------------ gradients
def test_what_asks_for_a_gradient_is_refused():
    f = Filled([40, 20], 2, 64, seed=43)
    q, k, v = f.query([1, 1], 4), f.k[:2].clone(), f.v[:2].clone()
    want = f.cache.attend(0, q)
    for t in (q, k, v):
        t.requires_grad_()
    for call in (lambda: f.cache.attend(0, q), lambda: f.cache.attend(0, q * 2), lambda: f.cache.write(0, k, v.detach()), lambda: f.cache.write(0, k.detach(), v),
                 lambda: f.cache.attend(0, q.detach(), out=q)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert torch.equal(f.cache.attend(0, q.detach()), want)
    with torch.no_grad():
        assert torch.equal(f.cache.attend(0, q), want)
        f.cache.write(0, k, v)
    with torch.inference_mode():
        f.cache.attend(0, q)


# ------------------------------------------------------------------ many items, and a long one among them
def test_a_long_piece_among_many_sequences():
    """Workgroups are counted by the longest item: more of them than a launch takes."""
    n, rows, heads, kv, dim = 512, 32_768, 32, 8, 64
    lengths = [rows] + [(i * 7) % 50 + 1 for i in range(1, n)]
    c = Cache(kv, dim, page_tokens=64, pages=sum(-(-x // 64) for x in lengths), max_seqs=n, max_pages=rows // 64, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(44)
    st = starts_of(lengths)
    c.extend(starts=st)
    k, v = (torch.randn((sum(lengths), kv, dim), device=DEV, generator=g).bfloat16() for _ in range(2))
    c.write(0, k, v, starts=st, max_new=rows)
    counts = [rows] + [1] * (n - 1)
    q = torch.randn((sum(counts), heads, dim), device=DEV, generator=g).bfloat16()
    out = torch.full_like(q, 7.0)
    c.attend(0, q, starts=starts_of(counts), max_new=rows, out=out)
    alone = c.attend(0, q[:rows], ints([0]), ints([0, rows]), max_new=rows)
    single = c.attend(0, q[rows:], ints(range(1, n)))
    torch.cuda.synchronize()
    assert c.poll_error() == 0
    assert torch.equal(out[:rows], alone)
    # two kernels: each off by its own roundings (of probabilities, keys and values 2^-11 of a value of up to 5, and the output's)
    assert (out[rows:].float() - single.float()).abs().max() <= 5 * (3 * 2.0 ** -11 + 2.0 ** -8)


# ------------------------------------------------------------------ strides
def test_strides_that_no_place_depends_on():
    """Of one row, and of one head, the stride says nothing; heads may lie as far apart as they do."""
    g = torch.Generator(device=DEV).manual_seed(45)
    base = [torch.randn((2, 1, 64), device=DEV, generator=g).bfloat16() for _ in range(2)]
    c, want = (Cache(1, 64, page_tokens=32, pages=2, max_seqs=2, device=DEV) for _ in range(2))
    for x in (c, want):
        x.extend(n=2)
    want.write(0, *base)
    one = [x[1:2].as_strided((1, 1, 64), (1 << 26, 1 << 25, 1)) for x in base]
    c.write(0, base[0][:1].as_strided((1, 1, 64), (7, 3, 1)), base[1][:1].as_strided((1, 1, 64), (64, 1 << 30, 1)), ints([0]))
    c.write(0, *one, ints([1]))
    two = [torch.empty((2, 1, 64), dtype=torch.bfloat16, device=DEV).as_strided((2, 1, 64), (64, s, 1)).copy_(x) for s, x in zip((1 << 28, 5), base)]
    for _ in range(2):
        for x, y in zip(c.read(0, 2), want.read(0, 2)):
            assert torch.equal(x, y)
        c.write(0, *two)
    assert c.poll_error() == 0
    far = torch.empty((2, 131_072, 128), dtype=torch.float16, device=DEV)[:, -40:]  # heads 2^24 elements apart
    far.copy_(torch.randn((2, 40, 128), device=DEV, generator=g))
    c, want = (Cache(2, 128, page_tokens=32, pages=2, max_seqs=1, device=DEV) for _ in range(2))
    st = ints([0, 40])
    for x, t in ((c, far.transpose(0, 1)), (want, far.transpose(0, 1).contiguous())):
        x.extend(starts=st)
        x.write(0, t, t, starts=st, max_new=40)
    for x, y in zip(c.read(0, 40, starts=st, max_new=40), want.read(0, 40, starts=st, max_new=40)):
        assert torch.equal(x, y)
    q = far.transpose(0, 1)
    assert torch.equal(c.attend(0, q, starts=st, max_new=40), want.attend(0, q.contiguous(), starts=st, max_new=40))


def test_keys_and_values_of_different_strides():
    """Keys that were turned, values still in the fused projection; also on another stream, whose keys are only made there."""
    g = torch.Generator(device=DEV).manual_seed(46)
    rows, h, d = 41, 4, 64
    fused = torch.randn((rows, 3 * h * d), device=DEV, generator=g).half()
    k, v = fused[:, h * d:2 * h * d].view(rows, h, d), fused[:, 2 * h * d:].view(rows, h, d)
    st = ints([0, rows])
    caches = [Cache(h, d, page_tokens=32, pages=3, max_seqs=1, device=DEV) for _ in range(4)]
    for c in caches:
        c.extend(starts=st)
    caches[0].write(0, k.contiguous(), v.contiguous(), starts=st, max_new=rows)
    caches[1].write(0, k.contiguous(), v, starts=st, max_new=rows)
    caches[2].write(0, k, v.permute(1, 0, 2).contiguous().permute(1, 0, 2), starts=st, max_new=rows)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a = torch.randn((4096, 4096), device=DEV)
    with torch.cuda.stream(s):
        for _ in range(20):
            a @ a
        late = torch.zeros_like(v.contiguous())
        late.copy_(v)
    caches[3].write(0, k, late, starts=st, max_new=rows, stream=s)
    torch.cuda.synchronize()
    want = caches[0].read(0, rows, starts=st, max_new=rows)
    for c in caches[1:]:
        assert c.poll_error() == 0
        for x, y in zip(c.read(0, rows, starts=st, max_new=rows), want):
            assert torch.equal(x, y)


# ------------------------------------------------------------------ what no test looked at
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_values_read_back_in_fewer_bits(dim, dtype):
    """The values in 32 bits, rounded once to the nearest."""
    f = Filled([70, 1, 33], 3, dim, page=64, dtype=dtype, seed=dim)
    f.cache.write(0, f.k * 50, f.v * 1e-6, starts=starts_of(f.lengths), max_new=70)
    args = dict(starts=starts_of([69, 1, 20]), max_new=69)
    for x, y in zip(f.cache.read(0, 90, dtype=dtype, **args), f.cache.read(0, 90, **args)):
        assert x.dtype == dtype and torch.equal(x, y.to(dtype))
    assert f.cache.poll_error() == 0


def test_a_token_past_a_sequences_last_page():
    """Among others that have room, without starts: nothing changes, and the error says which it was."""
    c = Cache(1, 64, page_tokens=32, pages=9, max_seqs=4, max_pages=2, device=DEV)
    c.extend(starts=ints([0, 64, 94, 126, 126]))
    state = [x.clone() for x in (c.table, c.lengths, c.refs)]
    for call in (lambda: c.extend(n=4), lambda: c.extend(ints([1, 0])), lambda: c.extend(ints([0]), ints([0, 1]))):
        call()
        torch.cuda.synchronize()
        assert c.poll_error() == rtams.EINVAL
        assert all(torch.equal(x, y) for x, y in zip(state, (c.table, c.lengths, c.refs)))
        c.clear_error()
    c.extend(ints([1, 2, 3]))
    assert c.lengths.tolist() == [64, 31, 33, 1] and c.poll_error() == 0


# ------------------------------------------------------------------ scratch
@pytest.mark.parametrize("dim,kv,n,share,count,tokens", [(64, 100, 12, 1, 1, 17 * 128), (64, 100, 7, 4, 8, 9 * 128), (96, 50, 20, 2, 1, 12 * 128), (96, 50, 10, 4, 8, 8 * 128),
                                                         (128, 50, 14, 4, 1, 12 * 128), (128, 50, 10, 8, 8, 7 * 128), (256, 50, 5, 2, 1, 12 * 128), (256, 31, 2, 8, 8, 9 * 128),
                                                         (64, 50, 5, 1, 100, 9 * 128), (96, 50, 5, 1, 256, 9 * 128), (128, 31, 8, 4, 64, 1100), (256, 31, 8, 2, 64, 1000)])
def test_parts_of_rows_stay_in_their_scratch(dim, kv, n, share, count, tokens, monkeypatch):
    """Pieces a little shorter than what they are cut from, so that parts are as many as they can be: what lies behind the scratch is not touched, and a call
    gives what its items give one by one, but for the order of sums."""
    from paper_2408_02937_amd import cache as module
    kept = []

    def more(nbytes, device):
        kept.append(torch.full((nbytes + (64 << 20),), 0x5A, dtype=torch.uint8, device=device))
        return kept[-1][:nbytes]

    monkeypatch.setattr(module, "_device_bytes", more)
    c = Cache(kv, dim, page_tokens=128, pages=n * -(-tokens // 128), max_seqs=n, max_pages=-(-tokens // 128), device=DEV)
    scratch = c.scratch.numel()
    st = starts_of([tokens] * n)
    c.extend(starts=st)
    g = torch.Generator(device=DEV).manual_seed(48)
    k, v = (torch.randn((n * tokens, kv, dim), device=DEV, generator=g).half() for _ in range(2))
    c.write(0, k, v, starts=st, max_new=tokens)
    q = torch.randn((n * count, kv * share, dim), device=DEV, generator=g).half()
    out = c.attend(0, q, starts=starts_of([count] * n), max_new=count, causal=False)
    apart = torch.cat([c.attend(0, q[i * count:(i + 1) * count], ints([i]), ints([0, count]), max_new=count, causal=False) for i in range(n)])
    torch.cuda.synchronize()
    assert c.poll_error() == 0 and kept[1].numel() == scratch + (64 << 20)
    assert (kept[1][scratch:] == 0x5A).all()
    # (probabilities of one part or another relative to another maximum: each rounded to 2^-11 of itself, times values of up to 5; and the outputs')
    assert (out.float() - apart.float()).abs().max() <= 5 * (2 * 2.0 ** -11) + 2.0 ** -9
