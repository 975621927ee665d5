"""pask_rotary on pieces of one buffer that lie side by side, between one another or on top of one another: what shares nothing is
computed, what shares an element is refused (where strides are equal or a piece has no gaps) and leaves the buffer alone."""
import random

import pytest
import torch

import rotary_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def check(got, x, pos, freq):
    off = (got.double() - R.rotate(x, pos, freq)).abs() - R.bound(x, freq, False, 1.0, x.dtype)
    assert off.max().item() <= 0 and torch.equal(got[..., 2 * freq.numel():], x[..., 2 * freq.numel():])


def test_slices_between_one_another(P):
    """Input and output are interleaved in the same rows, or in the same heads; two tensors write what lies between a third one's rows."""
    n, table, freq = 21, P.pask_rotary_table(64), R.frequencies(64, 10000.0)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 37
    buf = torch.randn(n, 12, 192, device="cuda").to(torch.bfloat16)
    for ins, outs in (([buf[:, :4]], [buf[:, 8:]]), ([buf[:, :, 128:]], [buf[:, :, 64:128]]), ([buf[:, :1, :64], buf[:, 1:2, :64]], [buf[:, 2:3, 64:128], buf[:, 2:3, 128:]]),
                      ([buf[:, ::2, :64]], [buf[:, 1::2, :64]]), ([buf[:1, :3]], [buf[:1, 3:6]])):
        old, p = [x.clone() for x in ins], pos[:ins[0].shape[0]]
        P.pask_rotary(p, table, list(zip(ins, outs)))
        for x, y in zip(old, outs):
            check(y, x, p, freq)


@pytest.mark.parametrize("n", [1, 2, 33])
@pytest.mark.parametrize("heads_k", [1, 2, 8])
def test_queries_and_keys_in_place_in_one_projection(P, n, heads_k):
    """Two tensors of the same rows, each its own input, values behind them left alone."""
    table, freq = P.pask_rotary_table(128), R.frequencies(128, 10000.0)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 301
    rows = torch.randn(n, 8 + 2 * heads_k, 128, device="cuda").to(torch.bfloat16)
    q, k, old = rows[:, :8], rows[:, 8:8 + heads_k], rows.clone()
    P.pask_rotary(pos, table, [(q, q), (k, k)])
    check(rows[:, :8 + heads_k], old[:, :8 + heads_k], pos, freq)
    assert torch.equal(rows[:, 8 + heads_k:], old[:, 8 + heads_k:])


@pytest.mark.parametrize("seed", range(8))
def test_drawn_pieces_of_one_buffer(P, seed):
    r, table, freq = random.Random(seed), P.pask_rotary_table(16), R.frequencies(16, 10000.0)
    buf = torch.randn(4000, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)
    seen = [0, 0]
    for _ in range(150):
        n, heads, dim = r.randint(1, 5), r.randint(1, 4), r.randint(16, 24)
        pos = torch.randint(0, 5000, (n,), device="cuda", dtype=torch.int32)
        hs = dim + r.choice([0, 0, 1, 30])
        ts = hs * heads + r.choice([0, 7, 100])
        views, places = [], []
        for _ in range(2):
            at = r.randint(0, r.choice([40, 2000]))
            views.append(buf.as_strided((n, heads, dim), (ts, hs, 1), at))
            places.append({at + t * ts + h * hs + d for t in range(n) for h in range(heads) for d in range(dim)})
        shared = places[0] != places[1] and bool(places[0] & places[1])
        old, before = views[0].clone(), buf.clone()
        if shared:
            with pytest.raises(P.PaskError) as e:
                P.pask_rotary(pos, table, [tuple(views)])
            assert e.value.status == P.ERR_INVALID_ARG and torch.equal(buf, before)
        else:
            P.pask_rotary(pos, table, [tuple(views)])
            check(views[1], old, pos, freq)
            rest = torch.ones(4000, dtype=torch.bool, device="cuda")
            rest[torch.tensor(sorted(places[1]), device="cuda")] = False
            assert torch.equal(buf[rest], before[rest])
        seen[shared] += 1
    assert min(seen) > 10
