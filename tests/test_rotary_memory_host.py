"""pask_rotary refuses outputs in memory that the call uses otherwise, before anything touches a GPU.  Made-up addresses: refused calls only."""
import pytest

IN, OUT, POS, TABLE = 0x100000, 0x200000, 0x1000, 0x2000
TOKENS, HEADS, DIM, ROW = 5, 4, 128, 512           # bf16: a row of 1024 bytes, a tensor of 5120


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def call(P, *tensors, n=TOKENS, pos=POS, table=TABLE):
    ts = (P.RotaryTensor * len(tensors))(*[P.RotaryTensor(**{**dict(src=IN, dst=OUT, in_token_stride=ROW, in_head_stride=DIM, out_token_stride=ROW,
                                                                    out_head_stride=DIM, n_heads=HEADS, head_dim=DIM), **t}) for t in tensors])
    return P._lib.pask_rotary(n, pos, table, 64, 0, 0, 1.0, 0, len(tensors), ts, None)


SECOND = dict(src=0x300000, dst=0x400000)


@pytest.mark.parametrize("tensors, kw", [
    ([dict(dst=IN + 2)], {}), ([dict(dst=IN - 2)], {}), ([dict(dst=IN + 256)], {}), ([dict(dst=IN + 5118)], {}), ([dict(dst=IN - 5118)], {}),      # shifted
    ([dict(dst=IN + 1024)], {}),                                                                                  # a token on
    ([dict(n_heads=1, in_token_stride=1000, out_token_stride=1000, dst=IN + 254)], {}),                           # rows of a wider tensor, by an element
    ([dict(n_heads=1, in_token_stride=1000, out_token_stride=1000, dst=IN + 2000 * 4 - 254)], {}),
    ([dict(in_head_stride=192, out_head_stride=192, in_token_stride=800, out_token_stride=800, dst=IN + 1600 + 384 + 254)], {}),
    ([dict(dst=IN + 64, in_token_stride=700)], {}),                                                               # a whole range against wider rows
    ([{}, dict(src=0x300000, dst=OUT + 5118)], {}), ([{}, dict(src=0x300000, dst=IN)], {}), ([{}, dict(src=OUT + 1024, dst=0x400000)], {}),       # two tensors
    ([dict(dst=IN), dict(src=IN, dst=0x400000)], {}), ([dict(dst=IN), dict(dst=IN)], {}),                         # the same one in place and beside it, or twice
    ([SECOND], dict(pos=0x400000 + 4)), ([SECOND], dict(pos=0x400000 - 16)), ([SECOND], dict(table=0x400000 + 5112)), ([SECOND], dict(table=0x400000 - 120)),
    ([dict(n_heads=1, head_dim=64, dst=IN + 2, src=IN)], dict(n=1)),
    ([dict(in_token_stride=2 ** 40, in_head_stride=2 ** 40)], dict(n=2 ** 31 - 1)),                               # no memory reaches that far
])
def test_memory_that_is_in_use_is_refused(P, tensors, kw):
    assert call(P, *tensors, **kw) == P.ERR_INVALID_ARG


def test_too_many_heads_are_refused(P):
    assert call(P, dict(n_heads=2 ** 20 + 1, out_token_stride=2 ** 28, in_token_stride=2 ** 28)) == P.ERR_UNSUPPORTED_SHAPE
