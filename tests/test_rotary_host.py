"""pask_rotary_table against its formulas, and the refusals of both rotary calls (all of them come before anything touches a GPU)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import rotary_ref as R


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


CASES = [dict(rot=128, base=1e6), dict(rot=64, base=10000.0, scaling=1, factor=4.0), dict(rot=128, base=1e6, scaling=2, factor=8.0, context=4096.0),
         dict(rot=64, base=10000.0, scaling=3, factor=40.0, context=4096.0), dict(rot=2, base=500000.0),
         dict(rot=256, base=10000.0, scaling=2, factor=8.0, context=8192.0, few=1.0, many=4.0),
         dict(rot=64, base=10000.0, scaling=3, factor=4.0, context=100.0)]          # lo = 0, the mixture starts at pair 0


@pytest.mark.parametrize("kw", CASES)
def test_table_holds_the_formulas_as_parts_of_a_turn(P, kw):
    got = P.pask_rotary_table(kw["rot"], kw["base"], kw.get("scaling", 0), kw.get("factor", 1.0), kw.get("context", 0.0), kw.get("few", 1.0),
                              kw.get("many", 32.0), device="cpu").numpy().view(np.uint64)
    want = R.frequencies(**kw)
    assert got.shape == (kw["rot"] // 2,)
    for g, w in zip(got.tolist(), want.tolist()):
        # the formulas above are in doubles: a power and a few products, 2^-50 relative, and the table's own 2^-65 of a turn
        assert abs(g / 2.0 ** 64 - w / (2 * math.pi)) <= w * 2.0 ** -50 + 2.0 ** -64


def test_table_keeps_frequencies_above_a_turn_modulo_one(P):
    got = P.pask_rotary_table(2, 10000.0, P.ROTARY_LINEAR, 0.1, device="cpu").numpy().view(np.uint64)
    assert abs(got[0] / 2.0 ** 64 - (10.0 / (2 * math.pi)) % 1.0) < 2.0 ** -50       # 10 rad a position


@pytest.mark.parametrize("kw, status", [
    (dict(rot_dim=0), -3), (dict(rot_dim=7), -3), (dict(rot_dim=258), -3), (dict(rot_dim=-2), -3), (dict(scaling=4), -1), (dict(scaling=-1), -1),
    (dict(base=1.0), -1), (dict(base=float("nan")), -1), (dict(base=float("inf")), -1), (dict(scaling=1, factor=0.0), -1),
    (dict(scaling=1, factor=float("nan")), -1), (dict(scaling=2, factor=2.0, context=0.0), -1), (dict(scaling=2, factor=2.0, context=4096.0, few=0.0), -1),
    (dict(scaling=3, factor=2.0, context=4096.0, few=32.0, many=32.0), -1), (dict(scaling=3, factor=2.0, context=4096.0, many=float("inf")), -1)])
def test_table_refuses(P, kw, status):
    with pytest.raises(P.PaskError) as e:
        P.pask_rotary_table(**{**dict(rot_dim=64, base=10000.0), **kw}, device="cpu")
    assert e.value.status == status


def call(P, n=5, pos=0x1000, table=0x2000, rot=64, inter=0, trans=0, mag=1.0, dtype=0, count=None, tensors=None, **kw):
    """The C call with made-up addresses: only for calls that it refuses (or that have no tokens)."""
    one = dict(src=0x10000, dst=0x20000, in_token_stride=512, in_head_stride=128, out_token_stride=512, out_head_stride=128, n_heads=4, head_dim=128)
    one.update(kw)
    ts = (P.RotaryTensor * 1)(P.RotaryTensor(**one)) if tensors is None else tensors
    return P._lib.pask_rotary(n, pos, table, rot, inter, trans, mag, dtype, 1 if count is None else count, ts, None)


@pytest.mark.parametrize("kw, status", [
    (dict(n=-1), -1), (dict(pos=None), -1), (dict(pos=0x1002), -1), (dict(table=None), -1), (dict(table=0x2004), -1), (dict(rot=0), -3),
    (dict(rot=63), -3), (dict(rot=130), -3), (dict(rot=258), -3), (dict(inter=2), -1), (dict(trans=-1), -1), (dict(mag=float("nan")), -1),
    (dict(mag=float("inf")), -1), (dict(dtype=3), -1), (dict(dtype=-1), -1), (dict(count=0), -1), (dict(count=5), -1), (dict(src=None), -1),
    (dict(dst=None), -1), (dict(src=0x10001), -1), (dict(dtype=2, dst=0x20002), -1), (dict(n_heads=0), -1), (dict(head_dim=257), -3),
    (dict(in_token_stride=-512), -1), (dict(out_head_stride=-1), -1), (dict(in_token_stride=2 ** 41), -1),
    (dict(out_head_stride=64), -1), (dict(out_head_stride=0), -1), (dict(out_token_stride=0), -1),               # heads, tokens share elements
    (dict(out_token_stride=256), -1),                                                                             # tokens reach into heads
    (dict(n=2 ** 31 - 1, out_token_stride=2 ** 40, out_head_stride=2 ** 40), -1),
    (dict(dst=0x10000, out_token_stride=1024), -1)])                                                              # in place with other strides
def test_rotary_refuses(P, kw, status):
    assert call(P, **kw) == status


def test_no_tokens_is_nothing_to_do(P):
    assert call(P, n=0, pos=None, src=None, dst=None) == 0
    assert P._lib.pask_rotary(0, None, 0x2000, 64, 0, 0, 1.0, 0, 1, None, None) == -1


def test_binding_refuses_what_does_not_fit(P):
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    pos, table = torch.zeros(3, dtype=torch.int32), P.pask_rotary_table(64, device="cpu")
    for args in [(pos, table, []), (pos, table, [(x, x)] * 5), (pos, table, [(x.double(), x.double())]), (pos, table, [(x, x.float())]),
                 (pos, table, [(x, x[:2])]), (pos, table, [(x[0], x[0])]), (pos[:2], table, [(x, x)]), (pos, table, [(x, x)])]:      # (the last: not on a GPU)
        with pytest.raises(P.PaskError) as e:
            P.pask_rotary(*args)
        assert e.value.status == P.ERR_INVALID_ARG
