"""Latent caches on the GPU against the plain 64-bit model (latent_ref): append, read-back, decode and prompt attention."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "tests"))

import latent_ref as R

pytestmark = pytest.mark.gpu

D = "cuda"
LUT = [[0, 2], [1, 0], [2, 1], [1, 2], [0, 1]]          # action of (tag, group); group 0 and 1 differ everywhere
SCALE = 192 ** -0.5


@pytest.fixture(scope="module")
def pask():
    import paper_2608_28276_b200 as P
    return P


def normal(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float32).to(torch.bfloat16)


class Both:
    """A latent cache beside its model; pools start out full of NaN patterns, as memory that was used before may be."""

    def __init__(self, pask, bits=4, heads=16, max_seqs=4, max_tokens=2048, max_append=8192, pages=400, n_layers=2, lut=LUT):
        self.P, self.bits, self.heads = pask, bits, heads
        lg = [0, 1, 1][:n_layers] if n_layers > 1 else [0]
        lut = [row[:max(lg) + 1] for row in lut]
        self.gpu = pask.LatentCache(R.blob(lut, n_layers, lg, bits), n_layers, heads, max_seqs, max_tokens, max_append, pages, pages,
                                    low_bits=bits)
        self.gpu.pool_high.fill_(0xFF)
        self.gpu.pool_low.fill_(0xFF)
        self.ref = R.Ref(lut, lg, bits)
        self.h = self.gpu.handle

    def append(self, layer, seqs, xs, tags, actions=None):
        cu = torch.tensor(np.concatenate([[0], np.cumsum([x.shape[0] for x in xs])]), dtype=torch.int32, device=D)
        n = int(cu[-1])
        out = torch.full((n,), 0xEE, dtype=torch.uint8, device=D)
        self.P.pask_append_latent(self.h, layer, torch.tensor(seqs, dtype=torch.int32, device=D), cu, torch.cat(xs).to(D),
                                  torch.cat(tags).to(D), actions=actions, actions_out=out)
        at = 0
        for s, x, t in zip(seqs, xs, tags):
            dec = None if actions is None else actions[at:at + x.shape[0], self.ref.lg[layer]].cpu().numpy()
            a = self.ref.append(layer, s, x, t.numpy(), dec)
            assert torch.equal(out[at:at + x.shape[0]].cpu(), a)
            at += x.shape[0]

    def read(self, layer, seqs, spare=0):
        """Rows of the sequences; `spare` rows are left behind each and checked to be untouched."""
        lens = [sum(self.ref.lens(layer, s)) for s in seqs]
        cu = np.concatenate([[0], np.cumsum([n + spare for n in lens])])
        rows = torch.full((int(cu[-1]) + 3, 576), 7.0, dtype=torch.bfloat16, device=D)
        out_lens = torch.full((len(seqs), 2), -1, dtype=torch.int32, device=D)
        self.P.pask_read_latent(self.h, layer, torch.tensor(seqs, dtype=torch.int32, device=D),
                                torch.tensor(cu, dtype=torch.int32, device=D), rows, out_lens)
        assert out_lens.cpu().tolist() == [self.ref.lens(layer, s) for s in seqs]
        rows = rows.cpu()
        for c, n in zip(cu, lens):
            assert bool((rows[c + n:c + n + spare] == 7.0).all())
        assert bool((rows[int(cu[-1]):] == 7.0).all())
        return [rows[c:c + n] for c, n in zip(cu, lens)]

    def check_rows(self, layer, seqs, spare=0):
        for s, got in zip(seqs, self.read(layer, seqs, spare)):
            assert torch.equal(got.view(torch.int16), self.ref.rows(layer, s).view(torch.int16)) or \
                torch.equal(got, self.ref.rows(layer, s)), f"layer {layer} sequence {s}"

    def decode(self, layer, seqs, q, scale=SCALE, lse=True):
        n = len(seqs)
        out = torch.full((n, self.heads, 512), float("nan"), dtype=torch.bfloat16, device=D)
        l = torch.full((n, self.heads), float("nan"), dtype=torch.float32, device=D) if lse else None
        ws = self.gpu.workspace(n)
        ws.fill_(0xFF)
        self.P.pask_decode_attention_latent(self.h, layer, torch.tensor(seqs, dtype=torch.int32, device=D), q.to(D), scale, out, l, ws)
        return out, l

    def check_decode(self, layer, seqs, q, scale=SCALE):
        out, lse = self.decode(layer, seqs, q, scale)
        for i, s in enumerate(seqs):
            rows = self.ref.rows(layer, s)
            R.check(out[i], lse[i], R.attend(q[i], rows[None], rows[None, :, :512], scale), f"sequence {s}")

    def status(self):
        return self.P.pask_budget_state(self.h, 0).device_status


def tags_of(g, n, choices=5):
    return torch.randint(0, choices, (n,), generator=g, dtype=torch.uint8)


# ------------------------------------------------------------------------------------------- append and read back

@pytest.mark.parametrize("bits", [2, 4, 8])
def test_append_in_pieces_reads_back(pask, bits):
    g = torch.Generator().manual_seed(100 + bits)
    b = Both(pask, bits)
    for lens in ([1, 1, 1], [0, 5, 1], [17, 300, 0], [1, 0, 1], [513, 2, 64], [1, 1, 1]):
        for layer in (0, 1):
            b.append(layer, [2, 0, 3], [normal(g, n, 576) for n in lens], [tags_of(g, n) for n in lens])
            b.check_rows(layer, [0, 3, 2], spare=5)
    assert b.status() == 0
    # the budget state charges what was kept
    for s in (0, 2, 3):
        st = pask.pask_budget_state(b.h, s)
        nh, nl = (sum(b.ref.lens(l, s)[k] for l in (0, 1)) for k in (0, 1))
        assert st.retained_bytes == nh * 1152 + nl * (72 * bits + 36)
        assert sum(st.n_high) == nh and sum(st.n_low) == nl and st.full_bytes == sum(st.n_seen) * 1152
    # forgetting a sequence: its pages come back and are written over
    pask.pask_seq_reset(b.h, 3)
    b.ref.reset(3)
    assert b.read(0, [3])[0].shape[0] == 0
    b.append(0, [3, 1], [normal(g, 40, 576), normal(g, 19, 576)], [tags_of(g, 40), tags_of(g, 19)])
    b.check_rows(0, [1, 3, 0, 2, 3])
    assert b.status() == 0


@pytest.mark.parametrize("bits", [2, 4, 8])
def test_stored_values_at_the_borders(pask, bits):
    g = torch.Generator().manual_seed(7)
    lv = R.LEVELS[bits]
    x = normal(g, 12, 576)
    x[0] = 0.0
    x[1] = torch.tensor(2.0) ** torch.randint(-133, 120, (576,), generator=g).float()          # every magnitude, subnormals too
    x[2] = (torch.randint(-2 * lv, 2 * lv + 1, (576,), generator=g).float() / 2).to(torch.bfloat16)   # exact ties
    x[2].view(18, 32)[:, 0] = lv
    x[3] = x[2] * 2.0 ** -60
    x[4] = 3.3e38
    x[5] = normal(g, 576) * 1e37
    x[6] = 2.0 ** -126 * lv                                                                       # the smallest scale that is kept
    x[7] = (torch.tensor(2.0 ** -127 * lv)).to(torch.bfloat16)                                    # and one that is not
    x[8].view(18, 32)[:, 1:] = 0.0
    x[9] = normal(g, 576) * 1e-38
    tags = torch.full((12,), 1, dtype=torch.uint8)
    tags[11] = 0
    x[11] = float("nan")                                                                          # released: never looked at
    b = Both(pask, bits)
    b.append(0, [1], [x], [tags])
    b.check_rows(0, [1])
    keep = normal(g, 3, 576)
    b.append(1, [1], [torch.cat([keep, torch.full((1, 576), float("nan"), dtype=torch.bfloat16)])], [torch.tensor([3, 0, 0, 1], dtype=torch.uint8)])
    b.check_rows(1, [1])


def test_random_groups_round_exactly(pask):
    # many scales and quotients near a rounding border: every code must be that of the exact quotient
    g = torch.Generator().manual_seed(8)
    for bits in (4, 8):
        x = (torch.randint(128, 256, (600, 576), generator=g).float() * torch.tensor(2.0) ** torch.randint(-5, 1, (600, 576), generator=g).float())
        x = (x * (torch.randint(0, 2, (600, 576), generator=g) * 2 - 1)).to(torch.bfloat16)
        b = Both(pask, bits)
        b.append(0, [0], [x], [torch.full((600,), 1, dtype=torch.uint8)])
        b.check_rows(0, [0])


def test_decided_actions_and_protected_tags(pask):
    g = torch.Generator().manual_seed(9)
    b = Both(pask)
    n = 75
    tags = tags_of(g, n)
    tags[::7] = 255
    tags[3] = 200                                            # unknown: kept in bf16, counted
    cu = torch.tensor([0, 30, n], dtype=torch.int32, device=D)
    ids = torch.tensor([1, 2], dtype=torch.int32, device=D)
    acts = torch.empty((n, 2), dtype=torch.uint8, device=D)
    pask.pask_decide(b.h, ids, cu, tags.to(D), None, acts)
    x = [normal(g, 30, 576), normal(g, n - 30, 576)]
    for layer in (0, 1):
        b.append(layer, [1, 2], x, [tags[:30], tags[30:]], actions=acts)
        b.check_rows(layer, [1, 2])
    st = pask.pask_budget_state(b.h, 1)
    assert st.bad_tags == 2 and st.decided_retained_bytes == st.retained_bytes and st.device_status == 0
    with pytest.raises(pask.PaskError):
        pask.pask_append_latent(b.h, 0, ids, cu, torch.cat(x).to(D), tags.to(D), actions=acts[:, :1].contiguous())


def test_append_is_refused_as_a_whole(pask):
    g = torch.Generator().manual_seed(10)
    b = Both(pask, pages=6, max_tokens=64)
    b.append(0, [0], [normal(g, 20, 576)], [tags_of(g, 20)])
    keep = b.read(0, [0])[0]
    ids = torch.tensor([0, 1], dtype=torch.int32, device=D)

    def attempt(ids, lens, tag, bit, cu=None):
        n = sum(lens)
        cu = torch.tensor([0, lens[0], n], dtype=torch.int32, device=D) if cu is None else cu
        pask.pask_append_latent(b.h, 0, ids, cu, normal(g, n, 576).to(D), torch.full((n,), tag, dtype=torch.uint8, device=D))
        assert b.status() & bit
        assert torch.equal(b.read(0, [0])[0], keep)

    attempt(ids, [60, 60], 2, pask.DEV_POOL_EXHAUSTED)
    attempt(ids, [80, 1], 2, pask.DEV_SEQ_OVERFLOW)          # the page table holds 64 tokens of a stream
    attempt(torch.tensor([0, 0], dtype=torch.int32, device=D), [1, 1], 2, pask.DEV_BAD_SEQ)
    attempt(torch.tensor([0, 9], dtype=torch.int32, device=D), [1, 1], 2, pask.DEV_BAD_SEQ)
    attempt(ids, [1, 1], 2, pask.DEV_BAD_RAGGED, cu=torch.tensor([0, 2, 1], dtype=torch.int32, device=D))


def test_read_refusals(pask):
    g = torch.Generator().manual_seed(11)
    b = Both(pask)
    b.append(0, [0, 1, 2], [normal(g, n, 576) for n in (40, 50, 3)], [tags_of(g, n) for n in (40, 50, 3)])
    n0, n1, n2 = (sum(b.ref.lens(0, s)) for s in (0, 1, 2))
    rows = torch.full((n0 + n1 + n2, 576), 7.0, dtype=torch.bfloat16, device=D)
    lens = torch.empty((4, 2), dtype=torch.int32, device=D)

    def read(ids, cu):
        rows.fill_(7.0)
        pask.pask_read_latent(b.h, 0, torch.tensor(ids, dtype=torch.int32, device=D), torch.tensor(cu, dtype=torch.int32, device=D), rows,
                              lens[:len(ids)])
        return rows.cpu()

    got = read([0, 1, 2], [0, n0, n0 + n1 - 1, n0 + n1 + n2])              # one row short: that sequence is left out
    assert torch.equal(got[:n0], b.ref.rows(0, 0)) and bool((got[n0:n0 + n1 - 1] == 7.0).all())
    assert torch.equal(got[n0 + n1 - 1:n0 + n1 - 1 + n2], b.ref.rows(0, 2))
    assert b.status() == pask.DEV_BAD_RAGGED
    pask.pask_cache_reset(b.h)
    b.ref.__init__(LUT, [0, 1], 4)
    b.append(0, [0], [normal(g, 40, 576)], [tags_of(g, 40)])
    n0 = sum(b.ref.lens(0, 0))
    got = read([0, 77, -1], [0, n0, n0, n0])
    assert torch.equal(got[:n0], b.ref.rows(0, 0)) and lens[1:3].cpu().tolist() == [[0, 0], [0, 0]]
    assert b.status() == pask.DEV_BAD_SEQ
    got = read([0, 3], [0, n0, rows.shape[0] + 1])                          # beyond the buffer
    assert torch.equal(got[:n0], b.ref.rows(0, 0)) and b.status() & pask.DEV_BAD_RAGGED
    empty = torch.empty((0, 576), dtype=torch.bfloat16, device=D)
    pask.pask_read_latent(b.h, 0, torch.tensor([1], dtype=torch.int32, device=D), torch.tensor([0, 0], dtype=torch.int32, device=D), empty, lens[:1])
    assert lens[0].cpu().tolist() == [0, 0]


def test_other_calls_refuse_a_latent_cache(pask):
    b = Both(pask)
    ids, cu = torch.tensor([0], dtype=torch.int32, device=D), torch.tensor([0, 1], dtype=torch.int32, device=D)
    kv, q = torch.zeros((1, 1, 128), dtype=torch.bfloat16, device=D), torch.zeros((1, 4, 128), dtype=torch.bfloat16, device=D)
    out, ws = torch.zeros((1, 4, 128), device=D), b.gpu.workspace(1)
    tags = torch.zeros(1, dtype=torch.uint8, device=D)
    acts = torch.zeros((1, 2), dtype=torch.uint8, device=D)
    host = torch.zeros(4096, dtype=torch.uint8)
    calls = [
        lambda: pask.pask_append_kv(b.h, 0, ids, cu, kv, kv, tags),
        lambda: pask.pask_append_kv_decided(b.h, 0, ids, cu, kv, kv, tags, acts),
        lambda: pask.pask_append_attend(b.h, 0, ids, cu, kv, kv, tags, q, out, None, ws),
        lambda: pask.pask_decode_attention(b.h, 0, ids, q, out, None, ws),
        lambda: pask.pask_decode_attention_full(b.h, 0, ids, q, out, None, ws),
        lambda: pask.pask_decode_attention_static(b.h, 0, ids, q, out, None),
        lambda: pask.pask_plan_ahead(b.h, 0, ids, ws),
        lambda: pask.pask_decode_step_ahead(b.h, 0, ids, kv, kv, tags, q, out, None, ws, ws),
        lambda: pask.pask_decode_step_packed(b.h, 0, 1, host, host.view(torch.float32), ws, ws),
        lambda: pask.pask_decode_step_pipelined(b.h, 0, 1, host, host.view(torch.float32), ws, ws),
        lambda: pask.pask_step_packed_layout(b.h, 1),
        lambda: pask.pask_debug_dump_high(b.h, 0, 0, 1),
        lambda: pask.pask_debug_dump_low(b.h, 0, 0, 1),
        lambda: pask.pask_debug_plan_order_span(b.h, 1, 0, 0),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(pask.PaskError) as e:
            call()
        assert e.value.status == pask.ERR_UNSUPPORTED_SHAPE, i
    assert pask.pask_plan_area_bytes(b.h, 1) == 0 and pask.pask_step_staging_bytes(b.h, 1) == 0
    kvc = pask.Cache(R.blob([[2]], 1, [0]), 1, 4, 1, 1, 64, 64, 4, 4)
    lat, q576 = torch.zeros((1, 576), dtype=torch.bfloat16, device=D), torch.zeros((1, 4, 576), dtype=torch.bfloat16, device=D)
    o512 = torch.zeros((1, 4, 512), dtype=torch.bfloat16, device=D)
    for call in (lambda: pask.pask_append_latent(kvc.handle, 0, ids, cu, lat, tags),
                 lambda: pask.pask_read_latent(kvc.handle, 0, ids, cu, lat),
                 lambda: pask.pask_decode_attention_latent(kvc.handle, 0, ids, q576, SCALE, torch.cat([o512] * 1), None, ws)):
        with pytest.raises(pask.PaskError) as e:
            call()
        assert e.value.status in (pask.ERR_UNSUPPORTED_SHAPE, pask.ERR_INVALID_ARG)


def test_latent_calls_check_their_arguments(pask):
    b = Both(pask, heads=16)
    ids, cu = torch.tensor([0, 1], dtype=torch.int32, device=D), torch.tensor([0, 1, 2], dtype=torch.int32, device=D)
    x, tags = torch.zeros((2, 576), dtype=torch.bfloat16, device=D), torch.zeros(2, dtype=torch.uint8, device=D)
    q, out, ws = torch.zeros((2, 16, 576), dtype=torch.bfloat16, device=D), torch.zeros((2, 16, 512), dtype=torch.bfloat16, device=D), b.gpu.workspace(2)
    lse = torch.zeros((2, 16), device=D)
    A, Rd, Dc = pask.pask_append_latent, pask.pask_read_latent, pask.pask_decode_attention_latent
    for call in (lambda: A(b.h, 0, ids, cu[:2], x, tags), lambda: A(b.h, 0, ids, cu, x[:, :512], tags), lambda: A(b.h, 0, ids, cu, x.float(), tags),
                 lambda: A(b.h, 0, ids, cu, x, tags[:1]), lambda: A(b.h, 2, ids, cu, x, tags), lambda: A(b.h, -1, ids, cu, x, tags),
                 lambda: A(b.h, 0, ids, cu, x, tags, actions=tags.view(2, 1)), lambda: A(b.h, 0, ids.long(), cu, x, tags),
                 lambda: A(b.h, 0, ids[:0], cu[:1], x, tags), lambda: A(b.h, 0, ids.cpu(), cu, x, tags),
                 lambda: Rd(b.h, 0, ids, cu[:2], x), lambda: Rd(b.h, 0, ids, cu, x.float()), lambda: Rd(b.h, 0, ids, cu, x, cu), lambda: Rd(b.h, 5, ids, cu, x),
                 lambda: Dc(b.h, 0, ids, q[:, :8].contiguous(), SCALE, out, lse, ws), lambda: Dc(b.h, 0, ids, q, 0.0, out, lse, ws),
                 lambda: Dc(b.h, 0, ids, q, float("nan"), out, lse, ws), lambda: Dc(b.h, 0, ids, q, SCALE, out.float(), lse, ws),
                 lambda: Dc(b.h, 0, ids, q, SCALE, out[:1], lse, ws), lambda: Dc(b.h, 0, ids, q, SCALE, out, lse[:, :8], ws),
                 lambda: Dc(b.h, 0, ids, q.transpose(0, 1), SCALE, out, lse, ws), lambda: Dc(b.h, 9, ids, q, SCALE, out, lse, ws)):
        with pytest.raises(pask.PaskError) as e:
            call()
        assert e.value.status == pask.ERR_INVALID_ARG
    with pytest.raises(pask.PaskError) as e:
        Dc(b.h, 0, ids, q, SCALE, out, lse, ws[:0].new_zeros(128))
    assert e.value.status in (pask.ERR_WORKSPACE, pask.ERR_INVALID_ARG)
    assert b.status() == 0


# ------------------------------------------------------------------------------------------- decode attention

LENGTHS = [0, 1, 15, 16, 17, 63, 64, 65, 129, 500]


@pytest.mark.parametrize("heads", [1, 5, 16, 17, 32, 40, 64, 65, 96, 128])
def test_decode_heads(pask, heads):
    g = torch.Generator().manual_seed(heads)
    b = Both(pask, heads=heads, max_seqs=len(LENGTHS), n_layers=1, pages=800)
    for s, n in enumerate(LENGTHS):
        if n:
            b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n)])
    b.check_decode(0, list(range(len(LENGTHS))), normal(g, len(LENGTHS), heads, 576))
    b.check_decode(0, [9, 1, 9], normal(g, 3, heads, 576))              # a sequence twice, another order
    assert b.status() == 0


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("kind", ["low", "high", "mixed"])
def test_decode_formats(pask, bits, kind):
    g = torch.Generator().manual_seed(bits)
    lut = {"low": [[1]], "high": [[2]], "mixed": [[0], [1], [2]]}[kind]
    lens = [1, 33, 64, 127, 700, 16]
    b = Both(pask, bits, heads=24, max_seqs=6, n_layers=1, lut=lut)
    for s, n in enumerate(lens):
        b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n, len(lut))])
    b.check_decode(0, list(range(6)), normal(g, 6, 24, 576))


@pytest.mark.parametrize("ctas", [1, 2, 7, 40, 148, 300])
def test_decode_splits(pask, ctas):
    g = torch.Generator().manual_seed(3)
    b = Both(pask, heads=72, max_seqs=5, n_layers=1, pages=800)
    for s, n in enumerate([1000, 1, 0, 333, 90]):
        if n:
            b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n)])
    pask.pask_debug_set_attention_ctas(b.h, ctas)
    b.check_decode(0, [0, 1, 2, 3, 4], normal(g, 5, 72, 576))
    b.check_decode(0, [1, 4, 1, 2, 1, 0, 1, 1], normal(g, 8, 72, 576))       # many short parts in a share
    assert b.status() == 0


def test_decode_peaked_and_rising_scores(pask):
    # the running maximum moves with nearly every tile, and one row dominates
    g = torch.Generator().manual_seed(4)
    b = Both(pask, heads=16, n_layers=1, lut=[[2], [1]])
    x = normal(g, 1200, 576)
    x = (x.float() * torch.linspace(0.05, 6.0, 1200)[:, None]).to(torch.bfloat16)
    b.append(0, [0], [x], [(torch.arange(1200) % 2).to(torch.uint8)])
    b.append(0, [1], [x.flip(0)], [(torch.arange(1200) % 2).to(torch.uint8)])
    for scale in (1e-4, SCALE, 1.0):
        b.check_decode(0, [0, 1], normal(g, 2, 16, 576), scale)


def test_decode_after_growth_and_reuse(pask):
    # pages that end inside a tile, grown token by token, then handed to another sequence
    g = torch.Generator().manual_seed(5)
    b = Both(pask, heads=8, n_layers=1, lut=[[2], [1]], pages=8, max_tokens=128)
    for n in range(1, 36):
        b.append(0, [0, 1], [normal(g, 1, 576) * 50, normal(g, 1, 576)], [tags_of(g, 1, 2), tags_of(g, 1, 2)])
        b.check_decode(0, [0, 1], normal(g, 2, 8, 576))
    pask.pask_seq_reset(b.h, 0)
    b.ref.reset(0)
    b.append(0, [2], [normal(g, 9, 576)], [tags_of(g, 9, 2)])
    b.check_decode(0, [2, 0, 1], normal(g, 3, 8, 576))
    assert b.status() == 0


@pytest.mark.parametrize("mix", [(3, 0, 2), (1, 0, 9), (9, 0, 1), (1, 1, 1)])
def test_decode_long_shares_of_both_formats(pask, mix):
    # dozens of tiles in a share, formats alternating in every rhythm: neither producer may outrun the other's barriers
    g = torch.Generator().manual_seed(14)
    lut = [[2]] * mix[0] + [[0]] * mix[1] + [[1]] * mix[2]
    b = Both(pask, heads=40, max_seqs=2, n_layers=1, lut=lut, max_tokens=6000, pages=800)
    for s, n in enumerate([5200, 3100]):
        b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n, len(lut))])
    for ctas in (2, 5):
        pask.pask_debug_set_attention_ctas(b.h, ctas)
        b.gpu._ws = None
        b.check_decode(0, [0, 1], normal(g, 2, 40, 576))
        assert b.status() == 0


def test_many_sequences(pask):
    # more than a one-launch append takes, up to the largest call: single tokens, then a ragged second call
    g = torch.Generator().manual_seed(15)
    n = 1024
    b = Both(pask, heads=3, max_seqs=n, max_tokens=64, max_append=40000, pages=3000, n_layers=1, lut=[[2], [1], [0]])
    for lens in ([1] * n, [(7 * i) % 31 for i in range(n)]):
        b.append(0, list(range(n)), [normal(g, k, 576) for k in lens], [tags_of(g, k, 3) for k in lens])
    order = [(5 * i + 3) % n for i in range(n)]
    b.check_rows(0, order[:400])
    q = normal(g, n, 3, 576)
    out, lse = b.decode(0, order, q)
    for i in range(0, n, 7):
        rows = b.ref.rows(0, order[i])
        R.check(out[i], lse[i], R.attend(q[i], rows[None], rows[None, :, :512], SCALE), f"sequence {order[i]}")
    assert b.status() == 0


def test_decode_wait_that_runs_out_reports(pask):
    # the first copy announces bytes it does not bring: the waits give up after the limit, nothing hangs, the cache stays usable
    g = torch.Generator().manual_seed(16)
    b = Both(pask, heads=70, max_seqs=3, n_layers=1, lut=[[2], [2], [1]])
    x = [normal(g, n, 576) for n in (700, 90, 300)]
    t = [tags_of(g, n, 3) for n in (700, 90, 300)]
    b.append(0, [0, 1, 2], x, t)
    q = normal(g, 3, 70, 576)
    b.check_decode(0, [0, 1, 2], q)
    pask.pask_debug_set_wait(b.h, 100_000, 16)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    b.decode(0, [0, 1, 2], q)
    t0.record()
    b.decode(0, [0, 1, 2], q)
    t1.record()
    torch.cuda.synchronize()
    assert t0.elapsed_time(t1) < 1000.0
    assert b.status() & pask.DEV_TIMEOUT
    pask.pask_debug_set_wait(b.h)
    pask.pask_cache_reset(b.h)
    b.ref.__init__([[2], [2], [1]], [0], 4)
    b.append(0, [0, 1, 2], x, t)
    b.check_decode(0, [0, 1, 2], q)
    assert b.status() == 0


def test_decode_timing_hooks(pask):
    g = torch.Generator().manual_seed(17)
    b = Both(pask, heads=16, n_layers=1)
    b.append(0, [0], [normal(g, 900, 576)], [tags_of(g, 900)])
    q = normal(g, 1, 16, 576)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for e in ev:
        e.record()
    span = torch.tensor([-1, 0], dtype=torch.int64, device=D)
    pask.pask_cache_set_timing_events(b.h, *ev)
    pask.pask_cache_set_timing_span(b.h, span)
    b.check_decode(0, [0], q)
    torch.cuda.synchronize()
    lo, hi = span.tolist()
    assert 0 < hi - lo < 10_000_000 and 0.0 < ev[0].elapsed_time(ev[1]) < 1000.0


def test_decode_bad_ids_and_no_lse(pask):
    g = torch.Generator().manual_seed(6)
    b = Both(pask, heads=16, n_layers=1)
    b.append(0, [1], [normal(g, 70, 576)], [tags_of(g, 70)])
    q = normal(g, 3, 16, 576)
    out, lse = b.decode(0, [4, 1, -5], q)
    assert b.status() == pask.DEV_BAD_SEQ
    rows = b.ref.rows(0, 1)
    R.check(out[1], lse[1], R.attend(q[1], rows[None], rows[None, :, :512], SCALE))
    for i in (0, 2):
        assert bool((out[i] == 0).all()) and bool((lse[i] == -math.inf).all())
    again, _ = b.decode(0, [4, 1, -5], q, lse=False)
    assert torch.equal(again, out)


def test_decode_nan_query_stays_in_its_row(pask):
    g = torch.Generator().manual_seed(12)
    b = Both(pask, heads=16, n_layers=1)
    b.append(0, [0, 1], [normal(g, 90, 576), normal(g, 90, 576)], [tags_of(g, 90), tags_of(g, 90)])
    q = normal(g, 2, 16, 576)
    want, want_l = b.decode(0, [0, 1], q)
    q2 = q.clone()
    q2[0, 3, 5] = float("nan")
    q2[0, 4, 7] = float("inf")
    got, got_l = b.decode(0, [0, 1], q2)
    keep = [h for h in range(16) if h not in (3, 4)]
    assert torch.equal(got[1], want[1]) and torch.equal(got_l[1], want_l[1])
    assert torch.equal(got[0, keep], want[0, keep]) and torch.equal(got_l[0, keep], want_l[0, keep])
    assert bool(torch.isnan(got[0, 3]).all())


def test_decode_repeats_bit_for_bit_in_a_graph_and_on_a_stream(pask):
    g = torch.Generator().manual_seed(13)
    b = Both(pask, heads=80, max_seqs=3, n_layers=1)
    for s, n in enumerate([700, 40, 1]):
        b.append(0, [s], [normal(g, n, 576)], [tags_of(g, n)])
    q = normal(g, 3, 80, 576)
    want, want_l = b.decode(0, [0, 1, 2], q)
    ids, qd = torch.arange(3, dtype=torch.int32, device=D), q.to(D)
    out, lse, ws = torch.empty_like(want), torch.empty_like(want_l), torch.empty_like(b.gpu.workspace(3))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        pask.pask_decode_attention_latent(b.h, 0, ids, qd, SCALE, out, lse, ws)
    st.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_l)
    # one step captured: append a token, read back, attend; the replay works on what the buffers hold then
    x, tags = normal(g, 3, 576).to(D), torch.full((3,), 2, dtype=torch.uint8, device=D)
    cu = torch.arange(4, dtype=torch.int32, device=D)
    rows = torch.zeros((800, 576), dtype=torch.bfloat16, device=D)
    cu_rows = torch.tensor([0, 720, 790, 800], dtype=torch.int32, device=D)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pask.pask_append_latent(b.h, 0, ids, cu, x, tags)
        pask.pask_decode_attention_latent(b.h, 0, ids, qd, SCALE, out, lse, ws)
        pask.pask_read_latent(b.h, 0, ids, cu_rows, rows)
    for _ in range(3):
        nx = normal(g, 3, 576)
        x.copy_(nx)
        graph.replay()
        for s in range(3):
            b.ref.append(0, s, nx[s:s + 1], [2])
            r = b.ref.rows(0, s)
            R.check(out[s], lse[s], R.attend(q[s], r[None], r[None, :, :512], SCALE))
            at = int(cu_rows[s])
            assert torch.equal(rows[at:at + r.shape[0]].cpu(), r)
    assert b.status() == 0


# ------------------------------------------------------------------------------------------- prompt attention

def prompt(pask, nq, nk, heads, g, scale=SCALE, strided=False, junk=0, lse=True, factor=1.0):
    """Runs the call on a ragged batch with `junk` rows of NaN between the sequences' rows and checks it."""
    def layout(lens):
        cu, rows = [], 0
        for n in lens:
            cu.append(rows)
            rows += n
        return cu + [rows]
    tq, tk = sum(nq) + junk, sum(nk) + junk
    q, kv, latent = normal(g, tq, heads, 192) * factor, normal(g, tk, heads, 256), normal(g, tk, 576)
    for t, n in ((q, sum(nq)), (kv, sum(nk)), (latent, sum(nk))):
        t[n:] = float("nan")
    latent[:, :512] = float("nan")
    rope = latent.to(D)[:, 512:] if strided else latent[:, 512:].contiguous().to(D)
    out = torch.full((tq, heads, 128), 7.0, dtype=torch.bfloat16, device=D)
    l = torch.full((tq, heads), 7.0, device=D) if lse else None
    cq, ck = layout(nq), layout(nk)
    pask.pask_prompt_attention_latent(torch.tensor(cq, dtype=torch.int32, device=D), torch.tensor(ck, dtype=torch.int32, device=D), q.to(D),
                                      kv.to(D), rope, scale, out, l)
    out = out.cpu()
    assert bool((out[sum(nq):] == 7.0).all()) and (l is None or bool((l[sum(nq):] == 7.0).all()))
    for i, (a, b) in enumerate(zip(nq, nk)):
        if a == 0:
            continue
        k = torch.cat([kv[ck[i]:ck[i] + b, :, :128], latent[ck[i]:ck[i] + b, None, 512:].expand(-1, heads, -1)], -1).transpose(0, 1)
        ref = R.attend(q[cq[i]:cq[i] + a], k, kv[ck[i]:ck[i] + b, :, 128:].transpose(0, 1), scale,
                       torch.arange(a) + 1 + b - a if b else None) if b else \
            (torch.zeros((a, heads, 128), dtype=torch.float64), torch.full((a, heads), -math.inf, dtype=torch.float64), torch.zeros((a, heads, 128)), torch.zeros((a, heads)))
        R.check(out[cq[i]:cq[i] + a], l[cq[i]:cq[i] + a] if lse else ref[1], ref, f"sequence {i}: {a} queries, {b} keys")
    return out


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 400])
def test_prompt_lengths(pask, n):
    prompt(pask, [n], [n], 2, torch.Generator().manual_seed(n))


@pytest.mark.parametrize("heads", [1, 3, 16, 128])
def test_prompt_ragged_batch(pask, heads):
    g = torch.Generator().manual_seed(heads)
    n = [33, 1, 0, 150, 64] if heads == 128 else [130, 1, 0, 257, 64, 300]
    prompt(pask, n, n, heads, g, junk=5, strided=True)


@pytest.mark.parametrize("nq,nk", [([1], [300]), ([129], [500]), ([3, 200, 1, 7], [131, 129, 1, 0]), ([300, 5], [40, 2]), ([260], [259]),
                                   ([1, 1, 1], [128, 129, 127]), ([256], [513]), ([128, 128], [128, 384]), ([0, 0, 2], [5, 0, 2])])
def test_prompt_history_and_rows_that_see_nothing(pask, nq, nk):
    prompt(pask, nq, nk, 3, torch.Generator().manual_seed(sum(nq) + 7 * sum(nk)), junk=3)


@pytest.mark.parametrize("n_seqs", [33, 70])
def test_prompt_many_sequences(pask, n_seqs):
    # beyond 32 sequences the blocks go in the order of the batch
    g = torch.Generator().manual_seed(n_seqs)
    nq = [(37 * i) % 301 for i in range(n_seqs)]
    prompt(pask, nq, [n + (i % 3) * 40 for i, n in enumerate(nq)], 2, g, junk=2)


def test_prompt_without_any_keys(pask):
    prompt(pask, [5, 300], [0, 0], 2, torch.Generator().manual_seed(23))


def test_prompt_in_a_graph_and_on_a_stream(pask):
    g = torch.Generator().manual_seed(24)
    n, h = 700, 24
    q, kv, rope = normal(g, n, h, 192).to(D), normal(g, n, h, 256).to(D), normal(g, n, 64).to(D)
    cu = torch.tensor([0, 650, n], dtype=torch.int32, device=D)
    want, want_l = torch.empty((n, h, 128), dtype=torch.bfloat16, device=D), torch.empty((n, h), device=D)
    pask.pask_prompt_attention_latent(cu, cu, q, kv, rope, SCALE, want, want_l)
    torch.cuda.synchronize()
    out, lse = torch.zeros_like(want), torch.zeros_like(want_l)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        pask.pask_prompt_attention_latent(cu, cu, q, kv, rope, SCALE, out, lse)
    st.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pask.pask_prompt_attention_latent(cu, cu, q, kv, rope, SCALE, out, lse)
    q.mul_(0.5)
    pask.pask_prompt_attention_latent(cu, cu, q, kv, rope, SCALE, want, want_l)
    for _ in range(2):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_l)


# few blocks of queries: the keys of each are split over two, four or eight CTAs; parts without a key, queries without one,
# more blocks than fit at a time
@pytest.mark.parametrize("heads,nq,nk", [(5, [3], [6000]), (16, [200], [2000]), (24, [512], [2100]), (8, [2500], [2500]), (4, [900], [700]),
                                         (3, [3, 1, 250, 2, 0], [4000, 1, 100, 0, 300]), (2, [1] * 40, [700 + 13 * i for i in range(40)]),
                                         (1, [257, 255], [1025, 1023]), (20, [129], [1281])])
def test_prompt_splits_long_keys(pask, heads, nq, nk):
    prompt(pask, nq, nk, heads, torch.Generator().manual_seed(heads + sum(nk)), junk=2)


def test_prompt_split_scores_that_rise_along_the_keys(pask):
    # each part's reference maximum differs by far from the others'
    g = torch.Generator().manual_seed(25)
    prompt(pask, [60], [4000], 6, g, factor=20.0)
    nq, nk, h = 60, 4000, 6
    q, kv, rope = normal(g, nq, h, 192), normal(g, nk, h, 256), normal(g, nk, 64)
    q[:, :, 128:] = 1.0
    rope[:] = torch.linspace(-8, 8, nk)[:, None].to(torch.bfloat16)
    out, lse = torch.empty((nq, h, 128), dtype=torch.bfloat16, device=D), torch.empty((nq, h), device=D)
    pask.pask_prompt_attention_latent(torch.tensor([0, nq], dtype=torch.int32, device=D), torch.tensor([0, nk], dtype=torch.int32, device=D),
                                      q.to(D), kv.to(D), rope.to(D), SCALE, out, lse)
    kk = torch.cat([kv[:, :, :128], rope[:, None, :].expand(-1, h, -1)], -1).transpose(0, 1)
    R.check(out, lse, R.attend(q, kk, kv[:, :, 128:].transpose(0, 1), SCALE, torch.arange(nq) + 1 + nk - nq), "rising")


def test_prompt_split_repeats_bit_for_bit_in_a_graph_and_on_a_stream(pask):
    g = torch.Generator().manual_seed(26)
    nq, nk, h = 40, 3333, 8
    q, kv, rope = normal(g, nq, h, 192).to(D), normal(g, nk, h, 256).to(D), normal(g, nk, 64).to(D)
    cq, ck = (torch.tensor([0, n], dtype=torch.int32, device=D) for n in (nq, nk))
    want, want_l = torch.empty((nq, h, 128), dtype=torch.bfloat16, device=D), torch.empty((nq, h), device=D)
    pask.pask_prompt_attention_latent(cq, ck, q, kv, rope, SCALE, want, want_l)
    torch.cuda.synchronize()
    out, lse = torch.zeros_like(want), torch.zeros_like(want_l)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for _ in range(20):
            pask.pask_prompt_attention_latent(cq, ck, q, kv, rope, SCALE, out, lse)
    st.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pask.pask_prompt_attention_latent(cq, ck, q, kv, rope, SCALE, out, lse)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_l)


def test_prompt_scales_and_no_lse(pask):
    g = torch.Generator().manual_seed(21)
    for scale, factor in ((1.0, 1.0), (1e-4, 1.0), (SCALE, 30.0)):
        prompt(pask, [300], [300], 2, g, scale=scale, factor=factor)
    prompt(pask, [70], [70], 2, g, lse=False)


def test_prompt_malformed_ranges_are_left_out(pask):
    g = torch.Generator().manual_seed(22)
    q, kv, rope = normal(g, 100, 2, 192).to(D), normal(g, 100, 2, 256).to(D), normal(g, 100, 64).to(D)

    def run(cq, ck):
        out = torch.full((100, 2, 128), 7.0, dtype=torch.bfloat16, device=D)
        pask.pask_prompt_attention_latent(torch.tensor(cq, dtype=torch.int32, device=D), torch.tensor(ck, dtype=torch.int32, device=D), q, kv, rope, SCALE, out)
        return out

    good = run([0, 50, 100], [0, 50, 100])
    for cq, ck in (([0, 50, 101], [0, 50, 100]), ([0, 50, 100], [0, 50, 101]), ([0, 50, 100], [0, 50, 40]), ([0, 50, 20], [0, 50, 100])):
        out = run(cq, ck)
        assert torch.equal(out[:50], good[:50]) and bool((out[50:] == 7.0).all()), (cq, ck)


# ------------------------------------------------------------------------------------------- all of them together

def test_prompt_chunks_then_decode(pask):
    """A model's layer as it would use the calls: a first chunk attended and appended, a second chunk that reads the stored
    history back and expands it, then decode steps whose absorbed form equals the expanded one."""
    g = torch.Generator().manual_seed(30)
    heads, n1, n2 = 4, 150, 40
    b = Both(pask, heads=heads, n_layers=1, lut=[[2], [1], [0]])
    w = normal(g, 512, heads * 256) * 512 ** -0.5                  # up-projection: latent -> (key 128 | value 128) per head

    def expand(rows):
        return (rows[:, :512].to(D).float() @ w.to(D).float()).to(torch.bfloat16).view(-1, heads, 256)

    chunks = [normal(g, n1, 576), normal(g, n2, 576)]
    tags = [tags_of(g, n, 3) for n in (n1, n2)]
    for i, (x, t) in enumerate(zip(chunks, tags)):
        nh, nl = b.ref.lens(0, 2)
        hist = torch.empty((nh + nl, 576), dtype=torch.bfloat16, device=D)
        ids = torch.tensor([2], dtype=torch.int32, device=D)
        pask.pask_read_latent(b.h, 0, ids, torch.tensor([0, nh + nl], dtype=torch.int32, device=D), hist)
        keys = torch.cat([hist, x.to(D)])
        kv, q = expand(keys), normal(g, x.shape[0], heads, 192)
        out, lse = torch.empty((x.shape[0], heads, 128), dtype=torch.bfloat16, device=D), torch.empty((x.shape[0], heads), device=D)
        n, m = x.shape[0], keys.shape[0]
        pask.pask_prompt_attention_latent(torch.tensor([0, n], dtype=torch.int32, device=D), torch.tensor([0, m], dtype=torch.int32, device=D),
                                          q.to(D), kv, keys[:, 512:], SCALE, out, lse)
        kk = torch.cat([kv.cpu()[:, :, :128], keys.cpu()[:, None, 512:].expand(-1, heads, -1)], -1).transpose(0, 1)
        R.check(out, lse, R.attend(q, kk, kv.cpu()[:, :, 128:].transpose(0, 1), SCALE, torch.arange(n) + 1 + m - n), f"chunk {i}")
        b.append(0, [2], [x], [t])
        b.check_rows(0, [2])
    wk = w.view(512, heads, 256)[:, :, :128].float()
    for _ in range(3):
        x = normal(g, 1, 576)
        b.append(0, [2], [x], [torch.tensor([1], dtype=torch.uint8)])
        qe = normal(g, heads, 192)
        q = torch.cat([torch.einsum("hd,lhd->hl", qe[:, :128].float(), wk), qe[:, 128:].float()], -1).to(torch.bfloat16)[None]
        b.check_decode(0, [2], q)
        # the expanded form on the read-back rows gives the same log-sum-exp up to the rounding of q and of the keys to bf16
        rows = b.read(0, [2])[0]
        kv = expand(rows)
        out, lse = torch.empty((1, heads, 128), dtype=torch.bfloat16, device=D), torch.empty((1, heads), device=D)
        pask.pask_prompt_attention_latent(torch.tensor([0, 1], dtype=torch.int32, device=D), torch.tensor([0, len(rows)], dtype=torch.int32, device=D),
                                          qe[None].to(D), kv, rows.to(D)[:, 512:], SCALE, out, lse)
        _, l = b.decode(0, [2], q)
        # each side's score is off by at most one rounding of 2^-8 of each product's terms
        mag = float((q[0].double().abs() @ rows.double().abs().T).max() + (qe[:, :128].double().abs() @ kv.cpu().double()[:, :, :128].abs().amax(0).T).max()) * SCALE
        assert float((lse[0] - l[0]).abs().max()) <= 2 * R.BF16_HALF_STEP * mag
    assert b.status() == 0


FIRST_CALLS = """
import os, sys, torch
sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]
import paper_2608_28276_b200 as pask
import latent_ref as R
i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
c = pask.LatentCache(R.blob([[2], [1], [0]], 1, [0], 4), 1, 20, 4, 2048, 2048, 400, 400)
x = torch.randn(1300, 576, device="cuda").bfloat16()
tags = (torch.arange(1300, device="cuda") % 3).to(torch.uint8)
ids, cu, ids1, cu1 = i32(0, 2), i32(0, 600, 1300), i32(1), i32(0, 40)
rows, lens = torch.zeros(1300, 576, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda")
cu_rows = i32(0, 600, 1300)
qd, od, ws = torch.randn(2, 20, 576, device="cuda").bfloat16(), torch.zeros(2, 20, 512, dtype=torch.bfloat16, device="cuda"), c.workspace(2)
q, kv = torch.randn(300, 4, 192, device="cuda").bfloat16(), torch.randn(1300, 4, 256, device="cuda").bfloat16()
outs = [torch.zeros(n, 4, 128, dtype=torch.bfloat16, device="cuda") for n in (300, 300)]
one, cq, ck = i32(0, 100), i32(0, 300), i32(0, 1300)
def step():
    pask.pask_append_latent(c.handle, 0, ids, cu, x, tags)
    pask.pask_append_latent(c.handle, 0, ids1, cu1, x[:40], tags[:40])
    pask.pask_read_latent(c.handle, 0, ids, cu_rows, rows, lens)
    pask.pask_decode_attention_latent(c.handle, 0, ids, qd, 0.07, od, None, ws)
    pask.pask_prompt_attention_latent(cq, cq, q, kv[:300], x[:300, 512:], 0.07, outs[0])
    pask.pask_prompt_attention_latent(cq, ck, q, kv, x[:, 512:], 0.07, outs[1])
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (rows, lens, od, *outs)]
assert all(bool(t.any()) for t in got)
pask.pask_cache_reset(c.handle)
for t in (rows, lens, od, *outs):
    t.zero_()
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (rows, lens, od, *outs)))
print("same")
"""


def test_first_calls_of_a_process_can_be_captured():
    r = subprocess.run([sys.executable, "-c", f"ROOT = {ROOT!r}" + FIRST_CALLS], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


def test_calls_of_two_streams_side_by_side(pask):
    # each with its own workspace; prompts have nothing to share
    g = torch.Generator().manual_seed(33)
    b = Both(pask, heads=40)
    for s in (0, 1):
        b.append(0, [s], [normal(g, 900, 576)], [tags_of(g, 900, 5)])
    ids = [torch.tensor([s], dtype=torch.int32, device=D) for s in (0, 1)]
    q = [normal(g, 1, 40, 576).to(D) for _ in ids]
    ws = [b.gpu.workspace(1) for _ in ids]
    pq, pkv, pr = normal(g, 50, 4, 192).to(D), normal(g, 3000, 4, 256).to(D), normal(g, 3000, 64).to(D)
    cq, ck = (torch.tensor([0, n], dtype=torch.int32, device=D) for n in (50, 3000))
    new = lambda: ([torch.zeros((1, 40, 512), dtype=torch.bfloat16, device=D) for _ in ids], [torch.zeros((50, 4, 128), dtype=torch.bfloat16, device=D) for _ in ids])

    def go(i, out):
        pask.pask_decode_attention_latent(b.h, 0, ids[i], q[i], 0.06, out[0][i], None, ws[i])
        pask.pask_prompt_attention_latent(cq, ck, pq, pkv, pr, SCALE, out[1][i])

    want, got = new(), new()
    for i in (0, 1):
        go(i, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ids]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                go(i, got)
    torch.cuda.synchronize()
    for a, c in zip(want[0] + want[1], got[0] + got[1]):
        assert torch.equal(a, c)
