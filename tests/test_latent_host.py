"""Latent caches: what the host refuses and sizes (no GPU)."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "tests"))

import latent_ref as R


@pytest.fixture(scope="module")
def pask():
    subprocess.run(["python", os.path.join(ROOT, "paper_2608_28276_b200", "build.py"), "--if-stale"], check=True, capture_output=True)
    import paper_2608_28276_b200 as P
    return P


def test_sizes(pask):
    for bits, row in ((4, 288 + 36), (0, 288 + 36), (8, 576 + 36), (2, 144 + 36)):
        s = pask.pask_cache_sizes(pask.CacheDesc(2, 128, 1, 576, 16, 4, 1024, 1024, 5, 7, 0, bits))
        assert s.high_page_bytes == 16 * 1152 and s.low_page_bytes == 16 * row
        assert s.pool_high_bytes == 5 * s.high_page_bytes and s.pool_low_bytes == 7 * s.low_page_bytes
    # the low-precision row costs codes plus one bf16 scale per 32 values: what pask_budget_state charges
    assert 16 * 324 == pask.pask_cache_sizes(pask.CacheDesc(1, 1, 1, 576, 16, 1, 1, 1, 1, 1)).low_page_bytes


def test_unsupported_shapes(pask):
    D = pask.CacheDesc
    for bad in (D(1, 16, 2, 576, 16, 4, 64, 64, 8, 8), D(1, 129, 1, 576, 16, 4, 64, 64, 8, 8), D(1, 0, 1, 576, 16, 4, 64, 64, 8, 8),
                D(1, 16, 1, 576, 32, 4, 64, 64, 8, 8), D(1, 16, 1, 576, 16, 4, 64, 64, 8, 8, 16), D(1, 16, 1, 512, 16, 4, 64, 64, 8, 8)):
        with pytest.raises(pask.PaskError) as e:
            pask.pask_cache_sizes(bad)
        assert e.value.status == pask.ERR_UNSUPPORTED_SHAPE
    with pytest.raises(pask.PaskError) as e:
        pask.pask_cache_sizes(D(1, 16, 1, 576, 16, 4, 64, 64, 8, 8, 0, 6))
    assert e.value.status == pask.ERR_INVALID_ARG


def test_null_and_malformed_arguments(pask):
    L = pask._lib
    assert L.pask_append_latent(None, 0, 1, 1, 16, 16, 16, 16, None, None, None) == pask.ERR_INVALID_ARG
    assert L.pask_read_latent(None, 0, 1, 1, 16, 16, 16, None, None) == pask.ERR_INVALID_ARG
    assert L.pask_decode_attention_latent(None, 0, 1, 16, 16, 1.0, 16, None, 256, 256, None) == pask.ERR_INVALID_ARG
    ok = dict(n=1, tq=4, tk=4, h=2, cq=16, ck=16, q=16, kv=16, r=16, st=64, sc=0.1, o=16, l=None)

    def prompt(**kw):
        a = {**ok, **kw}
        return L.pask_prompt_attention_latent(a["n"], a["tq"], a["tk"], a["h"], a["cq"], a["ck"], a["q"], a["kv"], a["r"], a["st"], a["sc"],
                                              a["o"], a["l"], None)

    for kw in (dict(n=0), dict(n=1025), dict(tq=-1), dict(tk=-1), dict(cq=None), dict(ck=None), dict(q=None), dict(kv=None), dict(r=None),
               dict(o=None), dict(st=56), dict(st=65), dict(q=24), dict(kv=8), dict(r=2), dict(o=4), dict(l=2), dict(cq=1),
               dict(sc=0.0), dict(sc=-1.0), dict(sc=float("nan")), dict(sc=float("inf"))):
        assert prompt(**kw) == pask.ERR_INVALID_ARG, kw
    for kw in (dict(h=0), dict(h=129)):
        assert prompt(**kw) == pask.ERR_UNSUPPORTED_SHAPE, kw
    assert prompt(tq=0) == pask.OK              # nothing to do


def test_tensors_are_checked(pask):
    cpu = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(pask.PaskError) as e:
        pask.pask_append_latent(1, 0, cpu[:1], cpu[:2], torch.zeros((1, 576), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.uint8))
    assert e.value.status == pask.ERR_INVALID_ARG


def test_model_of_the_format():
    # ties to even, scale of a group below 2^-126, and the largest finite values
    x = torch.zeros((1, 576), dtype=torch.bfloat16)
    x[0, 0], x[0, 1], x[0, 2] = 7.0, 2.5, -3.5
    x[0, 32], x[0, 33] = 2.0 ** -126, -2.0 ** -127
    x[0, 64], x[0, 65] = 3.38e38, -1.0e38
    v = R.stored_low(x, 4)[0].double()
    assert v[:3].tolist() == [7.0, 2.0, -4.0] and v[32:34].tolist() == [0.0, 0.0] and bool(torch.isfinite(v).all())
    assert R.stored_low(x, 2)[0, 32].double() == 2.0 ** -126
