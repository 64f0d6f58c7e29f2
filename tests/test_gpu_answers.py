"""The index and the cache together, on a shrunken workload: the recorded steps say what the steps one by one say, and
pages come and go as the passages and requests do."""
import pytest

pytestmark = pytest.mark.gpu


def test_answers_study_small():
    from paper_2408_02937_amd import answers
    print("[case] answers study, scale 0.2, recorded and not", flush=True)
    kw = dict(scale=0.2, layers=2, heads=8, kv_heads=2, requests=12, steps=10, rounds=3, page_tokens=32)
    a, b = (answers.answers_study(record=r, **kw) for r in (True, False))
    for x, y in zip(a["rounds"], b["rounds"]):
        assert x["said"] == y["said"] and x["said_sum"] == y["said_sum"]
        assert x["pages_shared"] == y["pages_shared"] > 0 and x["pages_in_use"] == y["pages_in_use"] <= a["pages"]
    assert a["tokens_per_s"] > 0
