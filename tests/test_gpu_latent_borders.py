"""Latent caches on the GPU, at the borders of what their calls are documented to do."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "tests"))

import latent_ref as R
from test_gpu_latent import Both, D, SCALE, normal, tags_of

pytestmark = pytest.mark.gpu

LUT3 = [[2], [1], [0]]


@pytest.fixture(scope="module")
def pask():
    import paper_2608_28276_b200 as P
    return P


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=D)


# ------------------------------------------------------------------------------------------- read back

def read_and_check(pask, b, ids, cu, total):
    """Every sequence whose own range is in order, inside the buffer and long enough is written there; nothing else is."""
    want, bad = torch.full((total, 576), 7.0, dtype=torch.bfloat16), False
    for s, r0, r1 in zip(ids, cu, cu[1:]):
        kept = b.ref.rows(0, s)
        if 0 <= r0 <= r1 <= total and r1 - r0 >= kept.shape[0]:
            want[r0:r0 + kept.shape[0]] = kept
        else:
            bad = True
    rows = torch.full((total, 576), 7.0, dtype=torch.bfloat16, device=D)
    lens = torch.full((len(ids), 2), -1, dtype=torch.int32, device=D)
    pask.pask_read_latent(b.h, 0, i32(ids), i32(cu), rows, lens)
    assert torch.equal(rows.cpu(), want)
    assert lens.cpu().tolist() == [b.ref.lens(0, s) for s in ids]
    assert b.status() == (pask.DEV_BAD_RAGGED if bad else 0)


@pytest.mark.parametrize("case", ["too large in the middle", "descending first", "behind a descending one, overlapping", "negative first",
                                  "too short between others", "extremes", "descending without a page", "all good"])
def test_read_leaves_only_malformed_ranges_out(pask, case):
    g = torch.Generator().manual_seed(40)
    b = Both(pask, n_layers=1, lut=LUT3, max_append=4000, pages=300)
    lens = [700, 650, 40, 900]
    b.append(0, [0, 1, 2, 3], [normal(g, n, 576) for n in lens], [tags_of(g, n, 3) for n in lens])
    n0, n1, n2, n3 = (b.ref.rows(0, s).shape[0] for s in range(4))
    total = n0 + n1 + n2 + n3 + 500
    ids, cu = {
        "too large in the middle": ([0, 1, 2, 3], [0, n0, total + 1, n0 + 7, n0 + 7 + n3]),
        "descending first": ([0, 1], [n1 + 50, 0, n1]),
        "behind a descending one, overlapping": ([0, 1, 2], [0, n0 + 200, n0, n0 + n2 + 1]),     # ranges overlap, rows do not
        "negative first": ([3, 0, 1], [-5, 20, 20 + n0, 20 + n0 + n1]),
        "too short between others": ([0, 1, 2, 3], [3, 3 + n0, 3 + n0, 3 + n0 + n2, total]),
        "extremes": ([0, 1, 3, 2], [n3 + 40, n3 + 40 + n0, -2 ** 31, 2 ** 31 - 1, 0]),
        "descending without a page": ([0, 3, 1], [0, n0, 2 * 16, 2 * 16]),
        "all good": ([3, 1, 0, 2], [11, 11 + n3, 40 + n3 + n1, 41 + n3 + n1 + n0, total]),
    }[case]
    read_and_check(pask, b, ids, cu, total)


def test_read_of_a_thousand_ranges_in_descending_order(pask):
    # every second range runs backwards; sequences are named many times
    g = torch.Generator().manual_seed(41)
    b = Both(pask, n_layers=1, lut=LUT3, max_append=4000, pages=300)
    lens = [70, 1, 18, 33]
    b.append(0, [0, 1, 2, 3], [normal(g, n, 576) for n in lens], [tags_of(g, n, 3) for n in lens])
    ids, cu, places = [], [], []
    at = 0
    for k in range(512):
        n = b.ref.rows(0, k % 4).shape[0]
        places.append((at, at + n))
        at += n + k % 3
    for k in reversed(range(512)):
        ids += [k % 4, (k + 1) % 4]
        cu += places[k]
    read_and_check(pask, b, ids, cu + [0], at)


# ------------------------------------------------------------------------------------------- the largest finite values

TOP = 2.0 ** 120              # the last binade of bf16: 128 .. 255 times this


def low_values(x, bits):
    """What RETAIN-LOW stands for, in 64 bits: the largest scale is the one whose value of the last level is finite."""
    levels = R.LEVELS[bits]
    v = x.double().reshape(-1, 32)
    s = (v.abs().amax(1, keepdim=True) / levels).to(torch.bfloat16).double()
    s = s.clamp_max({1: 255 * TOP, 7: 36.25 * TOP, 127: 2 * TOP}[levels])
    assert bool(torch.isfinite((s * levels).to(torch.bfloat16)).all())
    code = torch.round(v / s).clamp(-levels, levels)
    return (code * s).to(torch.bfloat16).reshape(-1, 576)


@pytest.mark.parametrize("bits", [2, 4, 8])
def test_finite_values_stay_finite(pask, bits):
    # every mantissa of the last binade as a group's largest value, both signs, other values of the group anywhere below it
    g = torch.Generator().manual_seed(60)
    m = torch.arange(128, 256).repeat_interleave(4)
    x = torch.randint(-255, 256, (512, 576), generator=g).double() * TOP * (torch.arange(512)[:, None] % 2 + 1) / 2
    x = torch.minimum(torch.maximum(x, -m[:, None].double() * TOP), m[:, None].double() * TOP).to(torch.bfloat16)
    x[:, ::32] = (m * torch.tensor([1, -1, 1, -1]).repeat(128)).double()[:, None].to(torch.bfloat16) * TOP
    x[-1] = torch.finfo(torch.bfloat16).max
    x[-2] = -x[-1]
    want = low_values(x, bits)
    assert bool(torch.isfinite(want).all())
    b = Both(pask, bits, n_layers=1, lut=[[1]])
    tags = torch.zeros(512, dtype=torch.uint8, device=D)
    pask.pask_append_latent(b.h, 0, i32([0]), i32([0, 512]), x.to(D), tags)                   # two kernels
    for at in range(0, 512, 128):                                                             # one launch
        pask.pask_append_latent(b.h, 0, i32([1]), i32([0, 128]), x[at:at + 128].to(D), tags[:128])
    rows = torch.zeros((1024, 576), dtype=torch.bfloat16, device=D)
    pask.pask_read_latent(b.h, 0, i32([0, 1]), i32([0, 512, 1024]), rows)
    assert torch.equal(rows[:512].cpu(), want) and torch.equal(rows[512:].cpu(), want)
    # a row alone with a zero query: its values come out as they are stored
    pask.pask_append_latent(b.h, 0, i32([2]), i32([0, 1]), x[-1:].to(D), tags[:1])
    out, lse = b.decode(0, [2], torch.zeros((1, 16, 576), dtype=torch.bfloat16))
    assert torch.equal(out[0].cpu(), want[-1, :512].expand(16, 512)) and bool((lse == 0).all())
    assert b.status() == 0


# ------------------------------------------------------------------------------------------- prompts: waits that run out

# the first shape has more blocks of queries than SMs (a CTA that gives up has already accepted its next block); the others
# split the keys of a block over a cluster, of two to eight CTAs, some parts without a key
@pytest.mark.parametrize("heads,nq,nk", [(16, [256] * 40, [256 - 6 * i for i in range(40)]), (24, [512], [2100]), (30, [200], [2000]),
                                         (16, [200], [2000]), (5, [3], [6000]), (6, [300, 40, 2], [280, 900, 1])])
def test_prompt_wait_that_runs_out_leaves_nan(pask, heads, nq, nk):
    g = torch.Generator().manual_seed(70)
    tq, tk = sum(nq) + 2, sum(nk)
    q, kv, rope = normal(g, tq, heads, 192).to(D), normal(g, tk, heads, 256).to(D), normal(g, tk, 64).to(D)
    cq, ck = (i32([0] + torch.tensor(n).cumsum(0).tolist()) for n in (nq, nk))

    def run():
        out, lse = torch.full((tq, heads, 128), 7.0, dtype=torch.bfloat16, device=D), torch.full((tq, heads), 7.0, device=D)
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        pask.pask_prompt_attention_latent(cq, ck, q, kv, rope, SCALE, out, lse)
        t1.record()
        torch.cuda.synchronize()
        assert t0.elapsed_time(t1) < 1000.0
        return out, lse

    want, want_l = run()
    assert not bool(torch.isnan(want).any())
    pask.pask_debug_set_prompt_wait(1_000_000, 16)
    try:
        got, got_l = run()
    finally:
        pask.pask_debug_set_prompt_wait()
    nan = torch.isnan(got).all(-1) & torch.isnan(got_l)
    right = (got == want).all(-1) & (got_l == want_l)
    assert bool((nan | right)[:-2].all()), "neither finished nor marked"
    assert bool(nan.any()) and bool(right[:-2].any())
    assert bool((got[-2:] == 7.0).all()) and bool((got_l[-2:] == 7.0).all())                 # rows of no sequence
    again, again_l = run()
    assert torch.equal(again, want) and torch.equal(again_l, want_l)


# ------------------------------------------------------------------------------------------- workspaces and streams

def test_workspaces_are_not_shared(pask):
    b = Both(pask, heads=40)
    ws = [b.gpu.workspace(1) for _ in range(3)]
    assert len({w.data_ptr() for w in ws}) == 3 and all(w.numel() >= pask.pask_workspace_bytes(b.h, 1) for w in ws)


def test_decode_refuses_a_workspace_that_is_too_small(pask):
    b = Both(pask, heads=16)
    q, out = torch.zeros((2, 16, 576), dtype=torch.bfloat16, device=D), torch.full((2, 16, 512), 7.0, dtype=torch.bfloat16, device=D)
    ws = b.gpu.workspace(2)
    for n in (256, ws.numel() - 1):
        with pytest.raises(pask.PaskError) as e:
            pask.pask_decode_attention_latent(b.h, 0, i32([0, 1]), q, SCALE, out, None, ws[:n])
        assert e.value.status == pask.ERR_WORKSPACE
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


def test_two_streams_with_a_workspace_each(pask):
    g = torch.Generator().manual_seed(80)
    b = Both(pask, heads=40)
    for s, n in ((0, 1900), (1, 1700)):
        b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n)])
    ids, q = [i32([0, 1]), i32([1])], [normal(g, 2, 40, 576).to(D), normal(g, 1, 40, 576).to(D)]
    ws = [b.gpu.workspace(n.numel()) for n in ids]
    assert ws[0].data_ptr() != ws[1].data_ptr()
    rounds = 30
    out = [[torch.zeros((n.numel(), 40, 512), dtype=torch.bfloat16, device=D) for _ in range(rounds + 1)] for n in ids]
    lse = [[torch.zeros((n.numel(), 40), device=D) for _ in range(rounds + 1)] for n in ids]
    for i in (0, 1):
        pask.pask_decode_attention_latent(b.h, 0, ids[i], q[i], SCALE, out[i][rounds], lse[i][rounds], ws[i])
        rows = b.ref.rows(0, 1)
        R.check(out[i][rounds][-1], lse[i][rounds][-1], R.attend(q[i][-1].cpu(), rows[None], rows[None, :, :512], SCALE))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ids]
    for r in range(rounds):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                pask.pask_decode_attention_latent(b.h, 0, ids[i], q[i], SCALE, out[i][r], lse[i][r], ws[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        for r in range(rounds):
            assert torch.equal(out[i][r], out[i][rounds]) and torch.equal(lse[i][r], lse[i][rounds]), (i, r)


def test_a_workspace_dropped_at_once_outlives_the_call(pask):
    g = torch.Generator().manual_seed(81)
    b = Both(pask, heads=16, n_layers=1)
    b.append(0, [0], [normal(g, 1500, 576)], [tags_of(g, 1500)])
    q = normal(g, 1, 16, 576).to(D)
    want, want_l = b.decode(0, [0], q)
    out, lse, st = torch.empty_like(want), torch.empty_like(want_l), torch.cuda.Stream()
    n = pask.pask_workspace_bytes(b.h, 1)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        torch.cuda._sleep(20_000_000)                                                          # the call waits its turn there
    ids = i32([0])
    torch.cuda.current_stream().synchronize()
    lent = b.gpu.workspace(1)
    at = lent.data_ptr()
    pask.pask_decode_attention_latent(b.h, 0, ids, q, SCALE, out, lse, lent, stream=st)
    del lent
    others = [torch.empty(n, dtype=torch.uint8, device=D) for _ in range(4)]
    assert all(t.data_ptr() != at for t in others)
    st.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_l)


# ------------------------------------------------------------------------------------------- every row counts

# Gaussian rows against a bound for the whole sum do not show a row that is left out among thousands: each row in turn gets a query
# along itself, whose weight it then has nearly to itself.
@pytest.mark.parametrize("mix", [(3, 0, 2), (9, 0, 1), (1, 1, 1), (1, 0, 0), (0, 0, 1)])
@pytest.mark.parametrize("ctas", [148, 5])
def test_decode_finds_every_row(pask, mix, ctas):
    g = torch.Generator().manual_seed(90 + sum(mix))
    lut = [[2]] * mix[0] + [[0]] * mix[1] + [[1]] * mix[2]
    b = Both(pask, heads=40, max_seqs=2, n_layers=1, lut=lut, max_tokens=6000, pages=800)
    for s, n in ((0, 5201), (1, 77)):
        b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n, len(lut))])
    pask.pask_debug_set_attention_ctas(b.h, ctas)
    for s in (0, 1):
        rows = b.ref.rows(0, s)
        m = rows.shape[0]
        n = (m + 39) // 40
        q = rows[torch.arange(40 * n).clamp_max(m - 1)].view(n, 40, 576)
        dev = rows.to(D)
        out, lse = b.decode(0, [s] * n, q)
        for i in range(n):
            ref = [t.cpu() for t in R.attend(q[i].to(D), dev[None], dev[None, :, :512], SCALE)]
            R.check(out[i], lse[i], ref, f"rows from {40 * i}")
            # the tolerance sees the row: its weight is more than nine tenths, and it is far longer than the bound
            own = rows[40 * i:40 * i + 40].double()[:, :512]
            assert bool((own.abs().amax(-1) > 4 * ref[2][:own.shape[0]].amax(-1)).all())
    assert b.status() == 0


@pytest.mark.parametrize("heads,nq,nk", [(2, 40, 3001), (40, 300, 1500), (3, 700, 700)])
def test_prompt_finds_every_key(pask, heads, nq, nk):
    # the same for prompts: query t of head h looks along key (t * heads + h) * step, whichever it can see
    g = torch.Generator().manual_seed(95)
    kv, rope = normal(g, nk, heads, 256), normal(g, nk, 64)
    first = nk - nq
    at = (torch.arange(nq)[:, None] * heads + torch.arange(heads)[None, :]) * 7 % nk
    at = torch.minimum(at, first + torch.arange(nq)[:, None])
    q = torch.cat([kv[at, torch.arange(heads)[None, :], :128], rope[at]], -1)
    out, lse = torch.empty((nq, heads, 128), dtype=torch.bfloat16, device=D), torch.empty((nq, heads), device=D)
    pask.pask_prompt_attention_latent(i32([0, nq]), i32([0, nk]), q.to(D), kv.to(D), rope.to(D), 2 * SCALE, out, lse)
    k = torch.cat([kv[:, :, :128], rope[:, None].expand(-1, heads, -1)], -1).transpose(0, 1)
    R.check(out, lse, R.attend(q, k, kv[:, :, 128:].transpose(0, 1), 2 * SCALE, torch.arange(nq) + 1 + first), "needles")


def test_workspace_does_not_grow_with_the_batch_and_holds_what_is_written(pask):
    # two partial results a share at most; the bytes behind the workspace stay as they were in batches of every shape
    g = torch.Generator().manual_seed(82)
    b = Both(pask, heads=72, max_seqs=5, n_layers=1, lut=LUT3, pages=800)
    lens = [1000, 1, 333, 90]
    b.append(0, [0, 1, 3, 4], [normal(g, n, 576) for n in lens], [tags_of(g, n, 3) for n in lens])
    for ctas in (148, 2, 6, 40):
        pask.pask_debug_set_attention_ctas(b.h, ctas)
        assert pask.pask_workspace_bytes(b.h, 1024) - pask.pask_workspace_bytes(b.h, 1) <= 1024 * 16
        for seqs in ([0], [0, 0], [1, 0, 2, 3, 4], [1, 1, 0, 1, 0, 3] * 8, [4] * 60):
            n = pask.pask_workspace_bytes(b.h, len(seqs))
            room = torch.full((n + 65536,), 0xA5, dtype=torch.uint8, device=D)
            q = normal(g, len(seqs), 72, 576)
            out, lse = torch.empty((len(seqs), 72, 512), dtype=torch.bfloat16, device=D), torch.empty((len(seqs), 72), device=D)
            pask.pask_decode_attention_latent(b.h, 0, i32(seqs), q.to(D), SCALE, out, lse, room[:n])
            for i, s in enumerate(seqs):
                rows = b.ref.rows(0, s)
                R.check(out[i], lse[i], R.attend(q[i], rows[None], rows[None, :, :512], SCALE), f"{ctas} CTAs, {seqs}")
            assert bool((room[n:] == 0xA5).all())
    assert b.status() == 0
