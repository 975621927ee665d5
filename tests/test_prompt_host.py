"""Refusals of pask_prompt_attention that come before anything touches a GPU, and the size of its workspace."""
import ctypes as C

import pytest
import torch

import prompt_ref as R


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def test_no_cache_is_refused(P):
    assert P._lib.pask_prompt_attention(None, 0, 1, 1, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000, None, 0x1000, 1 << 30, None) == P.ERR_INVALID_ARG
    assert P._lib.pask_prompt_workspace_bytes(None, 1, 1) == 0


def test_binding_refuses_what_is_not_on_a_gpu(P):
    q, k = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    ids, cu = torch.zeros(1, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32)
    with pytest.raises(P.PaskError) as e:
        P.pask_prompt_attention(1, 0, ids, cu, q, k, k, q.clone(), None, torch.zeros(256, dtype=torch.uint8))
    assert e.value.status == P.ERR_INVALID_ARG


def test_model_of_the_format_against_whole_numbers():
    """bf16(code * scale) of the model, for rows whose scale is a power of two: the codes are what is left."""
    for bits, levels in R.LEVELS.items():
        codes = torch.arange(-levels, levels + 1)
        codes = codes[torch.arange(4 * 32) % codes.numel()].reshape(1, 1, 128).clone()
        codes[..., ::32] = levels                  # each group's largest
        x = (codes.float() * 0.25).to(torch.bfloat16)
        assert torch.equal(R.stored_low(x, bits).float(), codes.float() * 0.25)
