"""The cache's boundary without a GPU: size arithmetic and the refusals of the host."""
import ctypes as C

import pytest

from paper_2408_02937_amd import rtams


def cfg(**kw):
    base = dict(layers=2, kv_heads=4, head_dim=128, page_tokens=64, max_seqs=16, max_pages=32)
    base.update(kw)
    return rtams.CacheConfig(**base)


def test_a_page_takes_five_bits_a_channel():
    L = rtams.lib()
    size = lambda c, n: L.rtams_cache_pool_bytes_for(C.byref(c), n)
    for c in (cfg(), cfg(head_dim=64, layers=1), cfg(head_dim=96, page_tokens=32, kv_heads=1), cfg(head_dim=256, layers=5)):
        page = c.layers * c.page_tokens * c.kv_heads * c.head_dim * 5 // 4
        # codes, steps and zeros; a bit and five words of tables for each page, in whole 256 bytes
        assert size(c, 4096) - size(c, 2048) == 2048 * page + 2048 // 8 + 2048 * 5 * 4


def test_tables_grow_with_the_sequences():
    L = rtams.lib()
    size = lambda c: L.rtams_cache_pool_bytes_for(C.byref(c), 64)
    assert size(cfg(max_seqs=128)) - size(cfg(max_seqs=64)) == 64 * (4 + 32 * 4 + 32)


@pytest.mark.parametrize("bad", [dict(layers=0), dict(kv_heads=0), dict(head_dim=80), dict(head_dim=0), dict(page_tokens=48), dict(page_tokens=0),
                                 dict(page_tokens=2048), dict(max_seqs=0), dict(max_seqs=65537), dict(max_pages=0), dict(max_pages=1 << 25)])
def test_bad_configurations_are_refused(bad):
    L = rtams.lib()
    c = cfg(**bad)
    assert L.rtams_cache_pool_bytes_for(C.byref(c), 10) == 0 and L.rtams_cache_scratch_bytes_for(C.byref(c)) == 0
    h = C.c_void_p()
    assert L.rtams_cache_create(C.byref(c), C.byref(h)) == rtams.EINVAL and not h.value
    assert list(bad)[0].encode() in L.rtams_last_error()


def test_create_asks_for_memory():
    L = rtams.lib()
    h = C.c_void_p()
    c = cfg()
    assert L.rtams_cache_create(C.byref(c), C.byref(h)) == rtams.EINVAL and b"pool and scratch" in L.rtams_last_error()
    c.d_pool, c.d_scratch = 0x10010, 0x20000
    assert L.rtams_cache_create(C.byref(c), C.byref(h)) == rtams.EINVAL and b"aligned" in L.rtams_last_error()
    c.d_pool, c.pool_bytes = 0x10000, 100
    assert L.rtams_cache_create(C.byref(c), C.byref(h)) == rtams.EINVAL and b"holds no page" in L.rtams_last_error()
    c.pool_bytes, c.scratch_bytes = L.rtams_cache_pool_bytes_for(C.byref(c), 3), 100
    assert L.rtams_cache_create(C.byref(c), C.byref(h)) == rtams.EINVAL and b"scratch_bytes" in L.rtams_last_error()
    assert L.rtams_cache_create(None, C.byref(h)) == rtams.EINVAL and L.rtams_cache_create(C.byref(c), None) == rtams.EINVAL


def test_calls_without_a_cache_are_refused():
    L = rtams.lib()
    q, v, n = rtams.CacheQuery(), rtams.CacheView(), C.c_int64()
    for rc in (L.rtams_cache_extend(None, 1, None, None, None), L.rtams_cache_write(None, 0, 1, None, None, 1, 1, None, None, 0, 0, 0, None),
               L.rtams_cache_read(None, 0, 1, None, None, 1, 1, None, None, 0, None), L.rtams_cache_attend(None, C.byref(q), 1, None, None, 1, None),
               L.rtams_cache_fork(None, 1, None, None, 0, None), L.rtams_cache_trim(None, 1, None, None, None), L.rtams_cache_compact(None, None),
               L.rtams_cache_layout(None, C.byref(v)), L.rtams_cache_free_pages(None, C.byref(n)), L.rtams_cache_poll_error(None), L.rtams_cache_clear_error(None)):
        assert rc == rtams.EINVAL
    assert L.rtams_cache_destroy(None) == rtams.OK


@pytest.fixture(scope="module")
def records():
    from tests.test_kernel_resources import code_objects, kernels
    with open(rtams.LIB_PATH, "rb") as f:
        blob = f.read()
    return {k[".name"]: k for e in code_objects(blob) for k in kernels(e)}


# wavefronts of a workgroup and workgroups that are to run at once on a compute unit: four SIMDs of 512 registers, 160 KiB of LDS
@pytest.mark.parametrize("name,waves,groups,lds", [
    ("14k_cache_attendILi64ELi1E", 4, 5, 21 * 1024), ("14k_cache_attendILi64ELi2E", 4, 3, 22 * 1024), ("14k_cache_attendILi96ELi1E", 4, 4, 31 * 1024),
    ("14k_cache_attendILi96ELi2E", 4, 2, 32 * 1024), ("14k_cache_attendILi128ELi1E", 4, 3, 42 * 1024), ("14k_cache_attendILi128ELi2E", 4, 2, 42 * 1024),
    ("14k_cache_attendILi256ELi1E", 4, 1, 83 * 1024), ("14k_cache_promptILi64ELi8E", 8, 1, 32 * 1024), ("14k_cache_promptILi96ELi8E", 8, 1, 48 * 1024),
    ("14k_cache_promptILi128ELi8E", 8, 1, 64 * 1024), ("14k_cache_promptILi256ELi4E", 4, 1, 64 * 1024),
])
def test_attention_runs_as_many_workgroups_at_once_as_it_plans_for(records, name, waves, groups, lds):
    mine = [k for n, k in records.items() if name in n]
    assert len(mine) == 1
    assert (mine[0][".vgpr_count"] + 7) // 8 * 8 * ((waves * groups + 3) // 4) <= 512
    assert groups * (mine[0][".group_segment_fixed_size"] + lds) <= 160 * 1024
