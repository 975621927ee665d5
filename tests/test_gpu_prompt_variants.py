"""pask_prompt_attention's variants with and without pages to expand: which of them does the work goes by what the cache holds when the
call runs on the GPU, in calls of long sequences (both are launched) and of short ones, called and replayed."""
import pytest
import torch

import prompt_ref as R
from test_gpu_prompt import Case, cu_of

pytestmark = pytest.mark.gpu

LONG = [2500, 1900, 2300]                          # a mean above the border of 2048


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def empty(P, n_seqs, bits, window, seed, n_kv=1):
    c = Case(P, [700] * n_seqs, n_kv=n_kv, bits=bits, window=window, mix=(0.0, 0.0), seed=seed)
    P.pask_cache_reset(c.cache.handle)
    c.ref = R.Ref(n_kv, bits, window)
    return c


@pytest.mark.parametrize("nq", [LONG, [2047] * 3, [2048] * 3, [100, 40, 130]])
@pytest.mark.parametrize("bits, window", [(4, 0), (2, 16), (8, 64)])
def test_recorded_once_replayed_behind_anything(P, bits, window, nq):
    """Nothing there, a token each, histories, nothing again after a reset that was issued and one that was recorded."""
    c = empty(P, 3, bits, window, sum(nq) + bits)
    q, k, v = c.inputs(nq)
    out, lse, ws = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"), c.cache.prompt_workspace(3, sum(nq))
    ids, cu = torch.arange(3, dtype=torch.int32, device="cuda"), cu_of(nq)
    graph, wipe = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.pask_prompt_attention(c.cache.handle, 0, ids, cu, q, k, v, out, lse, ws)
    with torch.cuda.graph(wipe):
        P.pask_cache_reset(c.cache.handle)

    def replay(where):
        out.fill_(float("nan")), ws.fill_(255)
        graph.replay()
        c.verify([0, 1, 2], nq, q, k, v, out, lse, where)

    replay("nothing there")
    for s in range(3):
        c.append(s, 1, (0.0, 0.0))
    replay("a released token each")
    c.append(1, 500, (0.3, 0.4))
    replay("a history behind one sequence")
    c.append(0, 33, (1.0, 0.0)), c.append(2, 200, (0.0, 1.0))
    replay("histories")
    for reset in (lambda: P.pask_cache_reset(c.cache.handle), wipe.replay):
        reset()
        c.ref = R.Ref(1, bits, window)
        replay("nothing left")
        c.append(2, 300, (0.3, 0.4))
        replay("a history again")


@pytest.mark.parametrize("ids, nq", [([0, 1, 2], [2600, 2300, 2000]), ([2, 0, 1], [0, 4200, 2200]), ([1, 9, 0], [2400, 2100, 2200]), ([1], [6001])])
def test_long_sequences_some_with_a_history(P, ids, nq):
    """Sequence 2 alone has one: it asks for tokens, or for none, or another one is unknown."""
    c = empty(P, 3, 4, 0, 40 + len(ids), n_kv=2)
    c.append(2, 400, (0.3, 0.4))
    q, k, v = c.inputs(nq)
    out, lse = c.call(ids, nq, q, k, v)
    at = 0
    for s, n in zip(ids, nq):
        if s == 9:
            assert bool((out[at:at + n] == 0).all()) and bool((lse[at:at + n] == -float("inf")).all())
        elif n:
            hk, hv = c.ref.rows(s)
            R.check(out[at:at + n], lse[at:at + n], R.attend(q[at:at + n], torch.cat([hk, k[at:at + n]]), torch.cat([hv, v[at:at + n]]), hk.shape[0]), f"sequence {s}")
        at += n
    assert c.status() == (P.DEV_BAD_SEQ if 9 in ids else 0)


@pytest.mark.parametrize("nq", [[2200, 2000], [300, 200], [20, 25], [12, 12], [5, 3]])
@pytest.mark.parametrize("hist", [0, 600])
def test_a_wait_that_runs_out_in_any_variant(P, hist, nq):
    c = empty(P, 2, 4, 0, 50)
    if hist:
        c.append(0, hist, (0.3, 0.4))
    q, k, v = c.inputs(nq)
    P.pask_debug_set_wait(c.cache.handle, 100_000, 16)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    c.call([0, 1], nq, q, k, v)
    t1.record()
    torch.cuda.synchronize()
    assert t0.elapsed_time(t1) < 1000.0 and c.status() == P.DEV_TIMEOUT
    P.pask_debug_set_wait(c.cache.handle)
    P.pask_cache_reset(c.cache.handle)
    c.ref = R.Ref(1, 4, 0)
    if hist:
        c.append(0, hist, (0.3, 0.4))
    out, lse = c.call([0, 1], nq, q, k, v)
    c.verify([0, 1], nq, q, k, v, out, lse)
