"""pask_rotary against rotations in 64 bits: layouts, parts of a head, types, strides, far positions, the transpose as gradient."""
import math
import pytest
import torch

import rotary_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def positions(n, far, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, far, (n,), generator=g, dtype=torch.int64).to(torch.int32).cuda()


def normal(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.float32).to(dtype)


def check(got, x, pos, freq, inter=False, trans=False, mag=1.0):
    want = R.rotate(x, pos, freq, inter, trans, mag)
    off = (got.double() - want).abs() - R.bound(x, freq, inter, mag, x.dtype)
    assert off.max().item() <= 0.0, (off.max().item(), got.shape, got.dtype)
    assert torch.equal(got[..., 2 * freq.numel():], x[..., 2 * freq.numel():])       # what is not rotated is copied


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot, dim", [(128, 128), (64, 128), (16, 64), (2, 64), (96, 96), (40, 80), (18, 19), (256, 256), (2, 256), (64, 65)])
def test_layouts_types_and_parts_of_a_head(P, dtype, inter, rot, dim):
    n, far = 37, 70000
    pos, table, freq = positions(n, far, rot), P.pask_rotary_table(rot, 1e6), R.frequencies(rot, 1e6)
    q, k = normal((n, 5, dim), 1, dtype), normal((n, 2, dim), 2, dtype)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    P.pask_rotary(pos, table, [(q, qo), (k, ko)], interleaved=inter, magnitude=1.3)
    check(qo, q, pos, freq, inter, mag=1.3)
    check(ko, k, pos, freq, inter, mag=1.3)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 1183, 1185, 5000, 20011])
def test_numbers_of_tokens(P, n):
    pos, table, freq = positions(n, 1 << 20, n), P.pask_rotary_table(128, 1e6), R.frequencies(128, 1e6)
    q, k = normal((n, 7, 128), 3, torch.bfloat16), normal((n, 1, 128), 4, torch.bfloat16)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    P.pask_rotary(pos, table, [(q, qo), (k, ko)])
    if n:
        check(qo, q, pos, freq)
        check(ko, k, pos, freq)


def test_positions_to_both_ends_of_32_bits(P):
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 16777217 * 100, 123456789], dtype=torch.int32, device="cuda")
    # frequencies that 64-bit products with positions of 2^31 carry without loss: sums of few powers of two of a turn
    table = torch.tensor([1 << 62, 3 << 40, (1 << 33) + 1, 1, -(1 << 50)], dtype=torch.int64, device="cuda")
    x = normal((8, 3, 10), 5, torch.float32)
    y = torch.empty_like(x)
    P.pask_rotary(pos, table, [(x, y)])
    turns = [[(int(p) * (int(f) % 2 ** 64)) % 2 ** 64 / 2.0 ** 64 for f in table.tolist()] for p in pos.tolist()]       # exact in whole numbers
    ang = torch.tensor(turns, dtype=torch.float64, device="cuda")[:, None] * 2 * math.pi
    a, b = x[..., :5].double(), x[..., 5:].double()
    want = torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)
    assert ((y.double() - want).abs() - R.bound(x, torch.zeros(5), False, 1.0, x.dtype)).max().item() <= 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_views_of_wider_rows_and_other_orders(P, dtype):
    n, freq, table = 50, R.frequencies(64, 10000.0), P.pask_rotary_table(64)
    pos = positions(n, 5000, 9)
    fused = normal((n, 10, 128), 6, dtype)
    lat, wide = normal((n, 1, 576), 7, dtype), normal((n, 4, 192), 8, dtype)
    odd = normal((n, 3, 131), 10, dtype)
    cases = [(fused[:, :6], torch.empty(n, 6, 128, dtype=dtype, device="cuda")),                          # part of a projection's rows
             (lat[:, :, 512:], torch.empty(n, 1, 64, dtype=dtype, device="cuda")),                        # rotary dims of latent rows
             (wide[:, :, 128:], torch.empty(4, n, 64, dtype=dtype, device="cuda").transpose(0, 1)),       # output with heads outside
             (odd[:, :, 1:129], torch.empty(n, 3, 129, dtype=dtype, device="cuda")[:, :, 1:]),            # not aligned
             (fused[:, 3:4].expand(n, 5, 128), torch.empty(n, 5, 128, dtype=dtype, device="cuda")),       # one head for five
             (fused[::2][:25], torch.empty(25, 10, 128, dtype=dtype, device="cuda"))]
    for i, (x, y) in enumerate(cases):
        y.fill_(float("nan"))
        p = pos[:x.shape[0]]
        P.pask_rotary(p, table, [(x, y)], interleaved=bool(i & 1))
        check(y, x, p, freq, bool(i & 1))


def test_in_place_touches_only_the_rotated_dims(P):
    n, freq, table = 33, R.frequencies(64, 10000.0), P.pask_rotary_table(64)
    pos, rows = positions(n, 100000, 11), normal((n, 576), 12, torch.bfloat16)
    q = normal((n, 8, 192), 13, torch.bfloat16)
    before, qb = rows.clone(), q.clone()
    P.pask_rotary(pos, table, [(q[:, :, 128:],) * 2, (rows[:, None, 512:],) * 2], interleaved=True)
    check(rows[:, None, 512:], before[:, None, 512:], pos, freq, True)
    check(q[:, :, 128:], qb[:, :, 128:], pos, freq, True)
    assert torch.equal(rows[:, :512], before[:, :512]) and torch.equal(q[:, :, :128], qb[:, :, :128])
    part = normal((n, 2, 128), 14, torch.bfloat16)                    # in place with a tail behind the rotated dims
    pb = part.clone()
    P.pask_rotary(pos, table, [(part, part)])
    check(part, pb, pos, freq)


def test_four_tensors_of_different_heads_in_one_launch(P):
    n, freq, table = 41, R.frequencies(64, 10000.0), P.pask_rotary_table(64)
    pos = positions(n, 3000, 15)
    xs = [normal((n, h, d), 20 + h, torch.bfloat16) for h, d in ((9, 64), (1, 128), (33, 72), (2, 256))]
    ys = [torch.full_like(x, float("nan")) for x in xs]
    P.pask_rotary(pos, table, list(zip(xs, ys)))
    for x, y in zip(xs, ys):
        check(y, x, pos, freq)


@pytest.mark.parametrize("inter", [False, True])
def test_transpose_is_the_gradient(P, inter):
    """<R x, g> = <x, R^T g> for the call and its transpose, and R^T g against differences of <R x, g>: R is linear, so a difference over any
    step is exact but for rounding, a step of 2^-21 of |a| + |b| for each of the 2 * 24 products behind a value."""
    n, rot, dim = 6, 24, 32
    pos, table = positions(n, 9000, 30), P.pask_rotary_table(rot, 1000.0)
    x, g = normal((n, 2, dim), 31, torch.float32), normal((n, 2, dim), 32, torch.float32)
    y, gx = torch.empty_like(x), torch.empty_like(x)
    P.pask_rotary(pos, table, [(x, y)], interleaved=inter, magnitude=0.7)
    P.pask_rotary(pos, table, [(g, gx)], interleaved=inter, transpose=True, magnitude=0.7)
    check(gx, g, pos, R.frequencies(rot, 1000.0), inter, True, 0.7)
    slack = (x.double().abs().sum() * g.abs().max().double()).item() * 2.0 ** -20
    assert abs((y.double() * g).sum().item() - (x.double() * gx).sum().item()) <= slack
    for t, h, d in ((0, 0, 0), (3, 1, 5), (5, 0, 23), (2, 1, 30)):
        z = x.clone()
        z[t, h, d] += 1.0
        up = torch.empty_like(x)
        P.pask_rotary(pos, table, [(z, up)], interleaved=inter, magnitude=0.7)
        slope = ((up.double() - y.double()) * g.double())[t, h].sum().item()
        assert abs(slope - gx[t, h, d].item()) <= 2 * dim * 2.0 ** -21 * (1 + x[t, h].abs().max().item() * 4) * g[t, h].abs().max().item()
    back = torch.empty_like(x)
    P.pask_rotary(pos, table, [(y, back)], interleaved=inter, transpose=True, magnitude=1 / 0.7)
    assert (back - x).abs().max().item() <= 2.0 ** -18 * x.abs().max().item()        # there and back: two calls' bounds, |a| + |b| twice


def test_infinities_and_nan_stay_in_their_pairs(P):
    n, table = 4, P.pask_rotary_table(64)
    x = normal((n, 2, 64), 33, torch.bfloat16)
    x[1, 0, 3], x[2, 1, 40] = float("inf"), float("nan")
    y = torch.empty_like(x)
    P.pask_rotary(positions(n, 100, 34), table, [(x, y)])
    bad = ~torch.isfinite(y)
    assert set(map(tuple, bad.nonzero().tolist())) <= {(1, 0, 3), (1, 0, 35), (2, 1, 8), (2, 1, 40)} and bad.any()


def test_on_another_stream_and_captured(P):
    n, freq, table = 64, R.frequencies(128, 1e6), P.pask_rotary_table(128, 1e6)
    pos, x = positions(n, 8192, 35), normal((n, 40, 128), 36, torch.bfloat16)
    y, s = torch.empty_like(x), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    P.pask_rotary(pos, table, [(x, y)], stream=s)
    s.synchronize()
    check(y, x, pos, freq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.pask_rotary(pos, table, [(x, y)])
    for seed in (37, 38):
        x.copy_(normal(x.shape, seed, torch.bfloat16))
        pos.copy_(positions(n, 8192, seed))
        graph.replay()
        check(y, x, pos, freq)
