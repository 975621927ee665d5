"""Latent calls: what the host refuses (no GPU)."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def pask():
    subprocess.run([sys.executable, os.path.join(ROOT, "paper_2608_28276_b200", "build.py"), "--if-stale"], check=True, capture_output=True)
    import paper_2608_28276_b200 as P
    return P


def test_prompt_wait_limits(pask):
    for limit, surplus in ((0, 0), (-1, 0), (99_999, 0), (10 ** 12 + 1, 0), (10 ** 6, 8), (10 ** 6, 65552)):
        with pytest.raises(pask.PaskError) as e:
            pask.pask_debug_set_prompt_wait(limit, surplus)
        assert e.value.status == pask.ERR_INVALID_ARG
    pask.pask_debug_set_prompt_wait(100_000, 65536)
    pask.pask_debug_set_prompt_wait()


def test_tensors_of_another_rank_are_refused(pask):
    # one dimension too few in each tensor whose sizes a call goes by
    ids, cu, bf = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), dict(dtype=torch.bfloat16)
    u8, ws = torch.zeros(1, dtype=torch.uint8), torch.zeros(256, dtype=torch.uint8)
    row, q, kv, rope = torch.zeros((1, 576), **bf), torch.zeros((1, 2, 192), **bf), torch.zeros((1, 2, 256), **bf), torch.zeros((1, 64), **bf)
    out = torch.zeros((1, 2, 128), **bf)
    for call in (lambda: pask.pask_append_latent(0, 0, ids, cu, row[0, 0], u8), lambda: pask.pask_append_latent(0, 0, ids, cu, row[0], u8),
                 lambda: pask.pask_read_latent(0, 0, ids, cu, row[0, 0]), lambda: pask.pask_decode_attention_latent(0, 0, ids, row[0], 1.0, out, None, ws),
                 lambda: pask.pask_prompt_attention_latent(cu, cu, q[0, 0], kv, rope, 1.0, out),
                 lambda: pask.pask_prompt_attention_latent(cu, cu, q[0, 0, 0], kv, rope, 1.0, out),
                 lambda: pask.pask_prompt_attention_latent(cu, cu, q, kv[0, 0, 0], rope, 1.0, out),
                 lambda: pask.pask_prompt_attention_latent(cu, cu, q, kv, rope[0], 1.0, out)):
        with pytest.raises(pask.PaskError) as e:
            call()
        assert e.value.status == pask.ERR_INVALID_ARG


@pytest.mark.parametrize("stride", [2 ** 31, 2 ** 31 + 64, 2 ** 32 + 64])
def test_rope_rows_further_apart_than_the_call_can_say_are_refused(pask, stride):
    # the C call's stride is an int32: the lower half of a larger one is another stride (2^32 + 64: adjacent rows)
    cu, bf = torch.zeros(2, dtype=torch.int32), dict(dtype=torch.bfloat16)
    rope = torch.empty_strided((2, 64), (stride, 1), dtype=torch.bfloat16, device="meta")
    with pytest.raises(pask.PaskError, match="k_rope") as e:
        pask.pask_prompt_attention_latent(cu, cu, torch.zeros((2, 2, 192), **bf), torch.zeros((2, 2, 256), **bf), rope, 1.0, torch.zeros((2, 2, 128), **bf))
    assert e.value.status == pask.ERR_INVALID_ARG


def test_the_stride_of_a_single_rope_row_does_not_matter(pask):
    cu, bf = torch.zeros(2, dtype=torch.int32), dict(dtype=torch.bfloat16)
    rope = torch.empty_strided((1, 64), (2 ** 40, 1), dtype=torch.bfloat16, device="meta")
    with pytest.raises(pask.PaskError, match="CUDA device"):                                  # as far as a call without a GPU gets
        pask.pask_prompt_attention_latent(cu, cu, torch.zeros((1, 2, 192), **bf), torch.zeros((1, 2, 256), **bf), rope, 1.0, torch.zeros((1, 2, 128), **bf))
