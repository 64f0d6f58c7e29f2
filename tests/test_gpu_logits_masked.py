"""Scores of rows of which most logits are equal: masked with the type's lowest number, or with few that stand above the others in few lanes.  The
bounds are those of test_gpu_logits.py."""
import pytest
import torch

from paper_2408_02937_amd.logits import score
from tests.test_gpu_logits import DEV, TYPES, check, gen

pytestmark = pytest.mark.gpu


def masked(rows, vocab, dtype, allowed, low, where="spread", seed=1):
    """Rows of which `allowed` tokens are allowed: spread, behind one another, or those of one lane and the next ones."""
    f = torch.randn((rows, vocab), device=DEV, generator=gen(seed))
    if where == "spread":
        at = torch.rand((rows, vocab), device=DEV, generator=gen(seed + 1)).topk(allowed, 1).indices if allowed else None
    else:
        each = 4 if dtype == torch.float32 else 8
        t = torch.arange(allowed, device=DEV)
        at = (t + vocab // 3 if where == "beside" else t // each * (256 * each) + t % each).expand(rows, allowed) % vocab
    x = torch.full((rows, vocab), low, dtype=dtype, device=DEV)
    if allowed:
        x.scatter_(1, at, f.gather(1, at).to(dtype))
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("where", ["spread", "beside", "lane"])
@pytest.mark.parametrize("rows,vocab", [(3, 32_768), (5, 33_000), (1100, 9_001)])
def test_masks_of_the_lowest_number(dtype, where, rows, vocab):
    for allowed in (0, 1, 19, 20, 21, 63, 64, 200, 700) if rows < 100 else (0, 19, 64, 700):
        x = masked(rows, vocab, dtype, allowed, torch.finfo(dtype).min, where, seed=allowed)
        for top in (1, 20, 64):
            check(x, None, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lanes", [5, 6, 20, 60])
def test_few_lanes_that_have_the_most_likely(dtype, lanes):
    """More logits stand above the others than are ranked at once, all of them different or some alike."""
    vocab = 70_000
    each = 4 if dtype == torch.float32 else 8
    t = torch.arange(vocab, device=DEV)
    g = torch.randn((4, vocab), device=DEV, generator=gen(lanes))
    g[1] = (g[1] * 8).round() / 8
    g[2] = g[2].abs() + 1
    g[3] = g[3].round()
    x = torch.where(t % (256 * each) < lanes * each, g, torch.full((), -9.0, device=DEV)).to(dtype)
    for y in (x, x[:, :19_000].repeat(260, 1)):
        for top in (1, 33, 64):
            check(y, None, top)


def least_time(f):
    for _ in range(3):
        f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            f()
    graph.replay()
    times = []
    for _ in range(7):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("allowed", [2, 19, 50])
@pytest.mark.parametrize("rows,vocab", [(1, 32_768), (1000, 32_768)])
def test_a_mask_of_the_lowest_number_costs_about_what_one_of_infinity_does(rows, vocab, allowed):
    """(A search for the tie, bit by bit, made it seven to seventeen times that.)"""
    x, y = (masked(rows, vocab, torch.float16, allowed, low) for low in (float("-inf"), torch.finfo(torch.float16).min))
    assert least_time(lambda: score(y, top=20)) < 5 * least_time(lambda: score(x, top=20))
