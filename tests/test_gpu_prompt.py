"""pask_prompt_attention against attention in 64 bits over what the table retains: head counts, code widths, lengths around every tile's
border, the protected window, single tokens and long prompts, and what callers may do with it (streams, graphs, repeated sequences)."""
import pytest
import torch

import prompt_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def normal(shape, g, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(torch.bfloat16)


def cu_of(lens):
    return torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


class Case:
    """A cache filled with histories of the given lengths, and the model of it."""

    def __init__(self, P, hist, n_kv=2, bits=4, window=0, mix=(0.3, 0.4), seed=1, n_layers=1, layer=0, chunk=None):
        self.P, self.n_kv, self.n_q, self.layer = P, n_kv, 4 * n_kv, layer
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        most = max(max(hist), 1)
        pages = sum((h + 15) // 16 + 1 for h in hist) + 8
        self.cache = P.Cache(R.blob(bits, window, n_layers), n_layers, self.n_q, n_kv, len(hist), most, max(1, chunk or most), pages, pages,
                             recent_window=window, low_bits=bits)
        self.cache.pool_high.fill_(255)            # NaN in every place that no token is written to
        self.cache.pool_low.fill_(255)
        self.ref = R.Ref(n_kv, bits, window)
        for s, n in enumerate(hist):
            for a in range(0, n, chunk or max(n, 1)):
                self.append(s, min(n - a, chunk or n), mix)

    def tags(self, n, mix):
        u = torch.rand(n, generator=self.g, device="cuda")
        return torch.where(u < mix[0], 2, torch.where(u < mix[0] + mix[1], 1, 0)).to(torch.uint8)

    def append(self, s, n, mix, k=None, v=None):
        k = normal((n, self.n_kv, 128), self.g) if k is None else k
        v = normal((n, self.n_kv, 128), self.g) if v is None else v
        t = self.tags(n, mix)
        self.P.pask_append_kv(self.cache.handle, self.layer, torch.tensor([s], dtype=torch.int32, device="cuda"), cu_of([n]), k, v, t)
        self.ref.append(s, k, v, t)

    def inputs(self, nq, scale=1.0):
        t = sum(nq)
        return normal((t, self.n_q, 128), self.g, scale), normal((t, self.n_kv, 128), self.g), normal((t, self.n_kv, 128), self.g)

    def call(self, ids, nq, q, k, v, lse=True, cu=None, ws=None):
        total = q.shape[0]
        out = torch.full((total, self.n_q, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        l = torch.full((total, self.n_q), float("nan"), dtype=torch.float32, device="cuda") if lse else None
        self.P.pask_prompt_attention(self.cache.handle, self.layer, torch.tensor(ids, dtype=torch.int32, device="cuda"), cu_of(nq) if cu is None else cu,
                                     q, k, v, out, l, self.cache.prompt_workspace(len(ids), total) if ws is None else ws)
        return out, l

    def verify(self, ids, nq, q, k, v, out, lse, where=""):
        at = 0
        for s, n in zip(ids, nq):
            if n:
                hk, hv = self.ref.rows(s)
                ref = R.attend(q[at:at + n], torch.cat([hk, k[at:at + n]]), torch.cat([hv, v[at:at + n]]), hk.shape[0])
                R.check(out[at:at + n], ref[1].float() if lse is None else lse[at:at + n], ref, f"{where} sequence {s}, {n} tokens behind {hk.shape[0]}")
            at += n
        assert self.status() == 0

    def status(self):
        return self.P.pask_budget_state(self.cache.handle, 0).device_status

    def run(self, nq, ids=None, scale=1.0, where=""):
        ids = list(range(len(nq))) if ids is None else ids
        q, k, v = self.inputs(nq, scale)
        out, lse = self.call(ids, nq, q, k, v)
        self.verify(ids, nq, q, k, v, out, lse, where)
        return q, k, v, out, lse


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 500])
def test_a_prompt_on_its_own(P, n):
    Case(P, [0], n_kv=2).run([n])


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("hist", [1, 15, 16, 17, 127, 128, 129, 400])
def test_a_token_behind_a_history(P, bits, hist):
    for mix in ((1.0, 0.0), (0.0, 1.0), (0.3, 0.4)):
        Case(P, [hist], n_kv=1, bits=bits, mix=mix).run([1], where=f"mix {mix}")


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("n_kv", [1, 2, 4, 8])
def test_ragged_batches(P, bits, n_kv):
    c = Case(P, [0, 1, 40, 700, 129, 0, 2000, 333], n_kv=n_kv, bits=bits, seed=n_kv)
    c.run([5, 64, 1, 130, 33, 300, 17, 96])
    c.run([1] * 8)
    c.run([0, 70, 0, 0, 65, 0, 1, 0])


@pytest.mark.parametrize("window", [16, 64, 256])
@pytest.mark.parametrize("bits", [2, 4, 8])
def test_protected_window(P, window, bits):
    c = Case(P, [0, 1, 15, 63, 64, 65, 256, 300, 1000], n_kv=2, bits=bits, window=window, seed=window)
    c.run([3, 40, 1, 65, 2, 7, 33, 5, 100])
    for s in range(9):                             # the ring goes round token by token
        for _ in range(3):
            c.append(s, 1, (0.3, 0.4))
    c.run([1, 2, 3, 4, 5, 6, 7, 8, 9])


def test_nothing_retained(P):
    Case(P, [300, 20], mix=(0.0, 0.0)).run([40, 1])


def test_more_items_than_ctas(P):
    c = Case(P, [i * 37 % 900 for i in range(70)], n_kv=8, seed=3)
    c.run([1 + i * 13 % 9 for i in range(70)])
    c.run([1 + i * 29 % 150 for i in range(70)])


def test_one_long_history_among_many_short_ones(P):
    c = Case(P, [20000] + [5] * 39, n_kv=8, seed=4)
    c.run([3] * 40)


def test_a_thousand_sequences(P):
    c = Case(P, [i % 50 for i in range(1024)], n_kv=1, seed=5)
    c.run([1 + i % 3 for i in range(1024)])


@pytest.mark.parametrize("n, hist", [(1, 33000), (17, 33000), (700, 9000), (5000, 0), (3001, 2500)])
def test_long(P, n, hist):
    Case(P, [hist], n_kv=2, seed=6).run([n])


def test_growing_chunk_by_chunk_equals_one_prompt(P):
    """Rotated, attended, appended: with a table that keeps everything in bf16, chunks of any size give what one prompt gives."""
    n, c, one = 700, Case(P, [0], n_kv=2, mix=(1.0, 0.0), chunk=800), Case(P, [0], n_kv=2)
    big = P.Cache(R.blob(), 1, 8, 2, 1, 800, 800, 64, 64)
    qkv = normal((n, 12, 128), c.g)
    pos, table = torch.arange(n, dtype=torch.int32, device="cuda"), P.pask_rotary_table(128, 1e6)
    q, k, v = torch.empty(n, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 2, 128, dtype=torch.bfloat16, device="cuda"), qkv[:, 10:].contiguous()
    P.pask_rotary(pos, table, [(qkv[:, :8], q), (qkv[:, 8:10], k)])
    whole = one.call([0], [n], q, k, v)
    one.verify([0], [n], q, k, v, *whole)
    at, ids = 0, torch.zeros(1, dtype=torch.int32, device="cuda")
    ref = R.attend(q, k, v, 0)
    for step in (1, 64, 200, 5, 129, 1, 300):
        s = slice(at, at + step)
        out, lse = torch.empty(step, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(step, 8, dtype=torch.float32, device="cuda")
        P.pask_prompt_attention(big.handle, 0, ids, cu_of([step]), q[s], k[s], v[s], out, lse, big.prompt_workspace(1, step))
        P.pask_append_kv(big.handle, 0, ids, cu_of([step]), k[s], v[s], torch.full((step,), 255, dtype=torch.uint8, device="cuda"))
        R.check(out, lse, tuple(x[s] for x in ref), f"tokens {at} ..")
        at += step
    assert at == n
    # and the next token as a decode step sees the same history: append, then attend with its query
    x = normal((1, 12, 128), c.g)
    qn, kn = torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    P.pask_rotary(torch.full((1,), n, dtype=torch.int32, device="cuda"), table, [(x[:, :8], qn), (x[:, 8:10], kn)])
    vn = x[:, 10:].contiguous()
    out, lse = torch.empty_like(qn), torch.empty(1, 8, dtype=torch.float32, device="cuda")
    P.pask_prompt_attention(big.handle, 0, ids, cu_of([1]), qn, kn, vn, out, lse, big.prompt_workspace(1, 1))
    P.pask_append_kv(big.handle, 0, ids, cu_of([1]), kn, vn, torch.full((1,), 255, dtype=torch.uint8, device="cuda"))
    d_out, d_lse = torch.empty(1, 8, 128, dtype=torch.float32, device="cuda"), torch.empty(1, 8, dtype=torch.float32, device="cuda")
    P.pask_decode_attention(big.handle, 0, ids, qn, d_out, d_lse, big.workspace(1))
    ref = R.attend(qn, torch.cat([k, kn]), torch.cat([v, vn]), n)
    R.check(out, lse, ref)
    R.check(d_out, d_lse, ref, "decode")


def test_layers_are_apart(P):
    a = Case(P, [300, 90], n_layers=3, layer=2, seed=7)
    a.run([10, 70])
    a.layer, a.ref = 1, R.Ref(2, 4, 0)             # nothing there
    a.run([10, 70])


def test_the_same_sequence_twice_and_any_order(P):
    c = Case(P, [500, 0, 77], n_kv=4, seed=8)
    c.run([9, 9, 40, 3], ids=[2, 0, 2, 1])


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("tokens", [8, 9, 16, 17, 32, 33])
def test_few_tokens_behind_long_histories(P, bits, tokens):
    """On both sides of where another number of tokens shares a tile; histories that end inside blocks, halves of blocks and pages."""
    c = Case(P, [1500, 64, 65, 2049, 1023, 130], n_kv=2, bits=bits, seed=tokens + bits)
    c.run([tokens] * 6)
    c.run([max(1, tokens - i) for i in range(6)])


def test_a_graph_recorded_before_anything_was_appended(P):
    """What was recorded is the variant for prompts without a history; replayed behind one it is as right as any."""
    for bits in (2, 4, 8):
        c = Case(P, [0, 0, 0], n_kv=2, bits=bits, window=16, seed=20 + bits, chunk=1000)
        nq = [100, 40, 130]
        q, k, v = c.inputs(nq)
        out, lse, ws = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"), c.cache.prompt_workspace(3, sum(nq))
        ids, cu = torch.arange(3, dtype=torch.int32, device="cuda"), cu_of(nq)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            P.pask_prompt_attention(c.cache.handle, 0, ids, cu, q, k, v, out, lse, ws)
        graph.replay()
        c.verify([0, 1, 2], nq, q, k, v, out, lse, "nothing there")
        for s in range(3):
            c.append(s, 1, (0.0, 0.0))
        graph.replay()
        c.verify([0, 1, 2], nq, q, k, v, out, lse, "a token each")
    c = Case(P, [900, 0, 77], n_kv=2, seed=24)     # and a cache that is filled, reset, recorded on and filled again
    P.pask_cache_reset(c.cache.handle)
    c.ref = R.Ref(2, 4, 0)
    q, k, v = c.inputs([100, 40, 130])
    out, lse, ws = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"), c.cache.prompt_workspace(3, 270)
    ids, cu = torch.arange(3, dtype=torch.int32, device="cuda"), cu_of([100, 40, 130])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.pask_prompt_attention(c.cache.handle, 0, ids, cu, q, k, v, out, lse, ws)
    for s, n in enumerate((900, 300, 77)):
        c.append(s, n, (0.3, 0.4))
    graph.replay()
    c.verify([0, 1, 2], [100, 40, 130], q, k, v, out, lse, "behind histories")


@pytest.mark.parametrize("seed", range(24))
def test_drawn_batches(P, seed):
    import random
    r = random.Random(seed)
    n = r.choice([1, 1, 2, 3, 7, 20, 45])
    window, bits, n_kv = r.choice([0, 0, 16, 64]), r.choice([2, 4, 8]), r.choice([1, 2, 4, 8])
    most = r.choice([1, 40, 300, 2500])
    hist = [r.choice([0, r.randint(0, most), r.randint(0, most)]) for _ in range(n)]
    longest = r.choice([1, 6, 14, 30, 70, 400])
    mix = r.choice([(1.0, 0.0), (0.0, 1.0), (0.2, 0.5), (0.05, 0.1)])
    c = Case(P, hist, n_kv=n_kv, bits=bits, window=window, mix=mix, seed=100 + seed)
    c.run([r.randint(0 if n > 1 and i else 1, longest) for i in range(n)], scale=r.choice([1.0, 4.0]), where=f"seed {seed}")


def test_large_and_small_scores(P):
    for scale in (0.0, 1e-3, 8.0, 30.0):
        Case(P, [400], seed=9).run([70], scale=scale, where=f"scale {scale}")


def test_scores_that_rise_by_much_in_the_last_keys(P):
    """The reference maximum moves at a late block, the early ones' weights fall below anything."""
    c = Case(P, [700], n_kv=1, mix=(1.0, 0.0), seed=10)
    q, k, v = c.inputs([130])
    k[100:] = 0
    k[120] = (q[125, 0].float() * 3).to(torch.bfloat16)
    out, lse = c.call([0], [130], q, k, v)
    c.verify([0], [130], q, k, v, out, lse)


def test_rows_outside_every_sequence(P):
    c = Case(P, [200, 50], seed=11)
    q, k, v = c.inputs([10, 7, 30, 3, 60])
    for x in (q, k, v):                            # rows 10 .. 16 and 47 .. 49 belong to nobody
        x[10:17], x[47:50] = float("nan"), float("inf")
    cu = torch.tensor([0, 10, 17, 47], dtype=torch.int32, device="cuda")
    ids = [0, 1, 1]
    out, lse = c.call(ids, None, q, k, v, cu=torch.tensor([0, 10, 10, 10], dtype=torch.int32, device="cuda"))
    c.verify([0], [10], q, k, v, out, lse)
    assert bool(torch.isnan(out[10:]).all()) and bool(torch.isnan(lse[10:]).all())
    pieces = torch.tensor([17, 47, 47, 47], dtype=torch.int32, device="cuda")
    out, lse = c.call(ids, None, q, k, v, cu=pieces)
    hk, hv = c.ref.rows(0)
    ref = R.attend(q[17:47], torch.cat([hk, k[17:47]]), torch.cat([hv, v[17:47]]), hk.shape[0])
    R.check(out[17:47], lse[17:47], ref)
    assert bool(torch.isnan(out[:17]).all()) and bool(torch.isnan(out[47:]).all())
    del cu


def test_without_lse(P):
    c = Case(P, [333], seed=12)
    q, k, v = c.inputs([20])
    out, _ = c.call([0], [20], q, k, v, lse=False)
    c.verify([0], [20], q, k, v, out, None)


def test_the_same_bits_every_time(P):
    c = Case(P, [i * 91 % 3000 for i in range(30)], n_kv=8, seed=13)
    nq = [1 + i * 7 % 40 for i in range(30)]
    q, k, v = c.inputs(nq)
    first = c.call(list(range(30)), nq, q, k, v)
    for _ in range(5):
        again = c.call(list(range(30)), nq, q, k, v)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_unknown_sequences_and_malformed_ranges(P):
    c = Case(P, [200, 50], seed=14)
    nq = [10, 70, 5, 6]
    q, k, v = c.inputs(nq)
    out, lse = c.call([0, 2, 1, -1], nq, q, k, v)
    assert c.status() == P.DEV_BAD_SEQ
    assert bool((out[10:80] == 0).all()) and bool((lse[10:80] == -float("inf")).all()) and bool((out[85:] == 0).all())
    P.pask_cache_reset(c.cache.handle)
    c.ref = R.Ref(2, 4, 0)
    c.append(0, 200, (0.3, 0.4)), c.append(1, 50, (0.3, 0.4))
    for at, s, n in ((0, 0, 10), (80, 1, 5)):
        hk, hv = c.ref.rows(s)
        o, l = c.call([s], None, q, k, v, cu=torch.tensor([at, at + n], dtype=torch.int32, device="cuda"))
        R.check(o[at:at + n], l[at:at + n], R.attend(q[at:at + n], torch.cat([hk, k[at:at + n]]), torch.cat([hv, v[at:at + n]]), hk.shape[0]))
    for cu, written in (([0, 10, 5, 91], (0, 10)), ([-3, 10, 10, 10], (0, 0)), ([0, 0, 92, 92], (0, 0)), ([5, 5, 5, 2 ** 31 - 1], (0, 0))):
        out, lse = c.call([0, 1, 0], None, q, k, v, cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        assert c.status() == P.DEV_BAD_RAGGED
        assert bool(torch.isfinite(out[written[0]:written[1]]).all())
        if cu[3] != 91:
            assert bool(torch.isnan(out[written[1]:]).all())
        P.pask_cache_reset(c.cache.handle)
        c.append(0, 200, (0.3, 0.4))


def test_two_streams_side_by_side_and_a_graph(P):
    c = Case(P, [900, 2000], n_kv=8, seed=15)
    jobs = []
    for s in range(2):
        q, k, v = c.inputs([40, 9])
        jobs.append((q, k, v, torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"), c.cache.prompt_workspace(2, 49), torch.cuda.Stream()))
    ids, cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda"), cu_of([40, 9])
    torch.cuda.synchronize()
    for _ in range(10):
        for q, k, v, out, lse, ws, st in jobs:
            P.pask_prompt_attention(c.cache.handle, 0, ids, cu, q, k, v, out, lse, ws, stream=st)
    torch.cuda.synchronize()
    for q, k, v, out, lse, ws, st in jobs:
        c.verify([0, 1], [40, 9], q, k, v, out, lse)
    q, k, v, out, lse, ws, st = jobs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.pask_prompt_attention(c.cache.handle, 0, ids, cu, q, k, v, out, lse, ws)
    for _ in range(3):                             # new inputs, a longer history, another split of the rows
        for x in (q, k, v):
            x.copy_(normal(x.shape, c.g))
        cu.copy_(cu_of([30, 19]))
        out.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        c.verify([0, 1], [30, 19], q, k, v, out, lse, "replayed")


def test_a_wait_that_runs_out_reports_and_leaves_the_cache_usable(P):
    c = Case(P, [900, 300], n_kv=2, seed=16)
    P.pask_debug_set_wait(c.cache.handle, 100_000, 16)
    q, k, v = c.inputs([40, 200])
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    c.call([0, 1], [40, 200], q, k, v)
    t1.record()
    torch.cuda.synchronize()
    assert t0.elapsed_time(t1) < 1000.0 and c.status() == P.DEV_TIMEOUT
    P.pask_debug_set_wait(c.cache.handle)
    P.pask_cache_reset(c.cache.handle)
    c.ref = R.Ref(2, 4, 0)
    c.append(0, 900, (0.3, 0.4)), c.append(1, 300, (0.3, 0.4))
    c.run([40, 200])


def test_refusals(P):
    c = Case(P, [20], n_kv=2, seed=17)
    h = c.cache.handle
    q, k, v = c.inputs([5])
    out, lse, ws = torch.empty_like(q), torch.empty(5, 8, dtype=torch.float32, device="cuda"), c.cache.prompt_workspace(1, 5)
    ids, cu = torch.zeros(1, dtype=torch.int32, device="cuda"), cu_of([5])
    need = P.pask_prompt_workspace_bytes(h, 1, 5)

    def raw(layer=0, n=1, total=5, i=ids.data_ptr(), u=cu.data_ptr(), qq=q.data_ptr(), kk=k.data_ptr(), vv=v.data_ptr(), o=out.data_ptr(),
            l=lse.data_ptr(), w=ws.data_ptr(), b=need, cache=h):
        return P._lib.pask_prompt_attention(cache, layer, n, total, i, u, qq, kk, vv, o, l, w, b, torch.cuda.current_stream().cuda_stream)

    bad = [dict(layer=-1), dict(layer=1), dict(n=0), dict(n=1025), dict(total=-1), dict(i=None), dict(u=None), dict(qq=None), dict(kk=None), dict(vv=None),
           dict(o=None), dict(w=None), dict(i=ids.data_ptr() + 2), dict(l=lse.data_ptr() + 2), dict(qq=q.data_ptr() + 8), dict(kk=k.data_ptr() + 2),
           dict(o=out.data_ptr() + 8), dict(w=ws.data_ptr() + 16), dict(o=q.data_ptr()), dict(o=k.data_ptr()), dict(o=v.data_ptr()),
           dict(o=q.data_ptr() + q.numel() * 2 - 16), dict(o=k.data_ptr() - q.numel() * 2 + 16)]
    assert all(raw(**x) == P.ERR_INVALID_ARG for x in bad)
    assert raw(b=need - 1) == P.ERR_WORKSPACE and raw(total=0, qq=None, o=None, w=None) == P.OK
    latent = P.LatentCache(R.blob(), 1, 16, 1, 16, 16, 4, 4)
    assert raw(cache=latent.handle) == P.ERR_UNSUPPORTED_SHAPE and P.pask_prompt_workspace_bytes(latent.handle, 1, 5) == 0
    for args in [(q.float(), k, v, out, lse), (q[:, :4], k, v, out, lse), (q, k[:4], v, out, lse), (q, k, v[:, :1], out, lse), (q, k, v, out[:, ::2], lse),
                 (q, k, v, out, lse.double()), (q.transpose(0, 1), k, v, out, lse), (q[0], k, v, out, lse), (q, k.cpu(), v, out, lse)]:
        with pytest.raises(P.PaskError) as e:
            P.pask_prompt_attention(h, 0, ids, cu, *args, ws)
        assert e.value.status == P.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert c.status() == 0
