"""pask_rotary at the largest number of tokens that its arguments hold."""
import pytest
import torch

import rotary_ref as R

pytestmark = pytest.mark.gpu


def test_as_many_tokens_as_an_int_holds():
    """One pair a token, all tokens with the same input (a stride of zero): 9 GB of positions, 9 of results."""
    import paper_2608_28276_b200 as P
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of free memory")
    n = 2 ** 31 - 1
    table, freq = P.pask_rotary_table(2, 10000.0), R.frequencies(2, 10000.0)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    x = torch.tensor([[[0.8, -0.6]]], dtype=torch.bfloat16, device="cuda").expand(n, 1, 2)
    y = torch.full((n, 1, 2), float("nan"), dtype=torch.bfloat16, device="cuda")
    P.pask_rotary(pos, table, [(x, y)])
    for a, b in ((0, 4000), (2 ** 30 - 2000, 2 ** 30 + 2000), (n - 4001, n)):
        off = (y[a:b].double() - R.rotate(x[a:b], pos[a:b], freq)).abs() - R.bound(x[a:b], freq, False, 1.0, x.dtype)
        assert off.max().item() <= 0
    for a in range(0, n, 1 << 28):
        assert not bool(torch.isnan(y[a:a + (1 << 28)]).any())
