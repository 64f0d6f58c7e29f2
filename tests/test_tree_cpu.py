"""Trees over the cache and scores of logits without a GPU: sizes, structures and the refusals of the host."""
import ctypes as C

import pytest

from paper_2408_02937_amd import rtams
from paper_2408_02937_amd.rtams import LogitsQuery


def query(**kw):
    base = dict(rows=3, row_stride=100, vocab=100, type=0, top=4, tokens=1, scale=1.0, d_logits=0x1000, d_tokens=0x2000, d_logprobs=0x3000, d_top=0x4000)
    base.update(kw)
    return LogitsQuery(**base)


def test_calls_without_a_cache_are_refused():
    L = rtams.lib()
    q, g = rtams.CacheQuery(), rtams.CacheSight()
    for rc in (L.rtams_cache_attend_sight(None, C.byref(q), C.byref(g), 1, None, None, 1, None), L.rtams_cache_tree(None, 1, None, None, 1, 1, None, None, 1, None, None),
               L.rtams_cache_walk(None, 1, None, 1, 1, None, None, None, None, None, None, None), L.rtams_cache_keep(None, 1, None, None, 1, 1, None, None, None)):
        assert rc == rtams.EINVAL


@pytest.mark.parametrize("bad,word", [(dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=1 << 30), "vocab"), (dict(type=3), "type"),
                                      (dict(type=-1), "type"), (dict(top=-1), "top"), (dict(top=65), "top"), (dict(tokens=-1), "tokens"), (dict(scale=0.0), "scale"),
                                      (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(scale=2e30), "scale"),
                                      (dict(row_stride=-1), "row_stride"), (dict(row_stride=1 << 40), "row_stride")])
def test_bad_queries_are_refused(bad, word):
    L = rtams.lib()
    q = query(**bad)
    assert L.rtams_logits_scratch_bytes_for(C.byref(q)) == C.c_size_t(-1).value and word.encode() in L.rtams_last_error()
    assert L.rtams_logits_score(C.byref(q), None) == rtams.EINVAL and word.encode() in L.rtams_last_error()


@pytest.mark.parametrize("bad,word", [(dict(d_logits=0), "NULL"), (dict(d_tokens=0), "NULL"), (dict(d_logprobs=0), "NULL"), (dict(d_top=0), "NULL"), (dict(d_logits=0x1001), "aligned"),
                                      (dict(type=2, d_logits=0x1002), "aligned"), (dict(d_tokens=0x2002), "aligned"), (dict(d_lse=0x5001), "aligned"), (dict(d_entropy=0x5002), "aligned"),
                                      (dict(d_top=0x4002), "aligned"), (dict(d_top_logprobs=0x4003), "aligned"),
                                      (dict(rows=1, vocab=200_000), "scratch_bytes"), (dict(rows=1, vocab=200_000, d_scratch=0x6000, scratch_bytes=16), "scratch_bytes"),
                                      (dict(rows=1, vocab=200_000, d_scratch=0x6008, scratch_bytes=1 << 20), "aligned")])
def test_bad_memory_is_refused(bad, word):
    L = rtams.lib()
    q = query(**bad)
    assert L.rtams_logits_score(C.byref(q), None) == rtams.EINVAL and word.encode() in L.rtams_last_error()


def test_scratch_is_asked_for_where_rows_are_few():
    L = rtams.lib()
    size = lambda **kw: L.rtams_logits_scratch_bytes_for(C.byref(query(**kw)))
    assert size(rows=0) == 0 and size(rows=1) == 0 and size(rows=4096, vocab=200_000) == 0
    one = size(rows=1, vocab=200_000, top=0)
    assert one > 0 and one % 16 == 0 and size(rows=2, vocab=200_000, top=0) == 2 * one
    assert size(rows=1, vocab=200_000, top=8) == one // 16 * (16 + 64)
    assert L.rtams_logits_score(None, None) == rtams.EINVAL
    assert L.rtams_logits_score(C.byref(query(rows=0, d_logits=0)), None) == rtams.OK


@pytest.fixture(scope="module")
def records():
    from tests.test_kernel_resources import code_objects, kernels
    with open(rtams.LIB_PATH, "rb") as f:
        blob = f.read()
    return {k[".name"]: k for e in code_objects(blob) for k in kernels(e)}


# wavefronts of a workgroup and workgroups that are to run at once on a compute unit: four SIMDs of 512 registers, 160 KiB of LDS.  Dynamic LDS of many
# rows: two tiles of halves and four of codes, of 64 tokens (32 where workgroups have 4 wavefronts).
@pytest.mark.parametrize("name,waves,groups,lds", [
    ("13k_cache_sightILi64ELi1E", 4, 5, 21 * 1024), ("13k_cache_sightILi64ELi2E", 4, 3, 22 * 1024), ("13k_cache_sightILi96ELi1E", 4, 4, 31 * 1024),
    ("13k_cache_sightILi96ELi2E", 4, 2, 32 * 1024), ("13k_cache_sightILi128ELi1E", 4, 3, 42 * 1024), ("13k_cache_sightILi128ELi2E", 4, 2, 42 * 1024),
    ("13k_cache_sightILi256ELi1E", 4, 1, 83 * 1024),
    ("20k_cache_prompt_sightILi64ELi8ELi2E", 8, 1, 52 * 1024), ("20k_cache_prompt_sightILi64ELi4ELi1E", 4, 2, 26 * 1024),
    ("20k_cache_prompt_sightILi96ELi8ELi2E", 8, 1, 78 * 1024), ("20k_cache_prompt_sightILi96ELi4ELi1E", 4, 2, 39 * 1024),
    ("20k_cache_prompt_sightILi128ELi8ELi2E", 8, 1, 104 * 1024), ("20k_cache_prompt_sightILi128ELi4ELi1E", 4, 2, 52 * 1024),
    ("20k_cache_prompt_sightILi256ELi4ELi1E", 4, 1, 104 * 1024), ("14k_cache_promptILi128ELi8E", 8, 1, 104 * 1024), ("14k_cache_promptILi256ELi4E", 4, 1, 104 * 1024),
    ("8k_logitsILi0E", 4, 4, 0), ("8k_logitsILi1E", 4, 4, 0), ("8k_logitsILi2E", 4, 4, 0),
])
def test_as_many_workgroups_run_at_once_as_are_planned_for(records, name, waves, groups, lds):
    mine = [k for n, k in records.items() if name in n]
    assert len(mine) == 1
    assert (mine[0][".vgpr_count"] + 7) // 8 * 8 * ((waves * groups + 3) // 4) <= 512
    assert groups * (mine[0][".group_segment_fixed_size"] + lds) <= 160 * 1024
