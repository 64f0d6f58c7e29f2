"""The cache where its calls could go wrong at the edges of what they take: sums beyond 32 bits, items that are not what a call asks for, probabilities
far below the largest, arguments that another stream reads, strides that say nothing.  Plain implementations and bounds: test_gpu_cache.py."""
import pytest
import torch

from paper_2408_02937_amd import rtams
from paper_2408_02937_amd.cache import Cache
from tests.test_gpu_cache import DEV, ints

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
    assert c.poll_error() == 0 and c.free_pages == long + 2000 - 5 * (n + 1)
    assert c.table[1:, :5].flatten().tolist() == list(range(5, 5 * (n + 1)))
