"""pask_prompt_attention refuses calls whose outputs share memory with what other parts of the call still read or write."""
import pytest
import torch

from test_gpu_prompt import Case, cu_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def test_outputs_that_share_memory_are_refused(P):
    total, n_kv, n_q = 5, 2, 8
    c = Case(P, [20, 3], n_kv=n_kv, seed=31)
    q, k, v = c.inputs([4, 1])
    out, lse = torch.empty_like(q), torch.empty(total, n_q, dtype=torch.float32, device="cuda")
    ids, cu, ws = torch.arange(2, dtype=torch.int32, device="cuda"), cu_of([4, 1]), c.cache.prompt_workspace(2, total)
    need = P.pask_prompt_workspace_bytes(c.cache.handle, 2, total)

    def call(**kw):
        at = dict(i=ids.data_ptr(), u=cu.data_ptr(), q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), o=out.data_ptr(), l=lse.data_ptr(), w=ws.data_ptr(), b=need)
        at.update(kw)
        return P._lib.pask_prompt_attention(c.cache.handle, 0, 2, total, at["i"], at["u"], at["q"], at["k"], at["v"], at["o"], at["l"], at["w"], at["b"],
                                            torch.cuda.current_stream().cuda_stream)

    q_bytes, kv_bytes, l_bytes = q.numel() * 2, k.numel() * 2, lse.numel() * 4
    for name, t, size in (("q", q, q_bytes), ("k", k, kv_bytes), ("v", v, kv_bytes), ("o", out, q_bytes), ("w", ws, need), ("i", ids, 8), ("u", cu, 12)):
        for at in (t.data_ptr(), t.data_ptr() + size - 4, t.data_ptr() - l_bytes + 4):
            assert call(l=at) == P.ERR_INVALID_ARG, ("lse", name, at - t.data_ptr())
        if name not in "ow":
            assert call(o=t.data_ptr() // 16 * 16) == P.ERR_INVALID_ARG, ("out", name)
        if name != "w":
            assert call(w=t.data_ptr() // 256 * 256) == P.ERR_INVALID_ARG, ("workspace", name)
    torch.cuda.synchronize()
    assert c.status() == 0


def test_neighbours_in_one_buffer_are_not(P):
    """Everything of a call cut out of one allocation, one piece right behind the other."""
    total, n_kv, n_q = 5, 2, 8
    c = Case(P, [20, 3], n_kv=n_kv, seed=32)
    q, k, v = c.inputs([4, 1])
    need = P.pask_prompt_workspace_bytes(c.cache.handle, 2, total)
    buf = torch.empty(need + 2 * q.numel() * 2 + 2 * k.numel() * 2 + total * n_q * 4 + 20, dtype=torch.uint8, device="cuda")
    at = need
    ws, views = buf[:need], []
    for shape, dtype in ((q.shape, torch.bfloat16), (k.shape, torch.bfloat16), (v.shape, torch.bfloat16), (q.shape, torch.bfloat16),
                         ((total, n_q), torch.float32), ((2,), torch.int32), ((3,), torch.int32)):
        size = torch.empty(0, dtype=dtype).element_size() * torch.Size(shape).numel()
        views.append(buf[at:at + size].view(dtype).view(shape))
        at += size
    assert at == buf.numel()
    bq, bk, bv, out, lse, ids, cu = views
    bq.copy_(q), bk.copy_(k), bv.copy_(v), ids.copy_(torch.arange(2)), cu.copy_(cu_of([4, 1]))
    P.pask_prompt_attention(c.cache.handle, 0, ids, cu, bq, bk, bv, out, lse, ws)
    c.verify([0, 1], [4, 1], q, k, v, out, lse)


def test_workspace_of_as_many_tokens_as_an_int_holds(P):
    """It depends on the tokens only by their mean, and that is as large as it gets from 33 on."""
    c = Case(P, [3], seed=33)
    for n in (1, 7, 1024):
        assert P.pask_prompt_workspace_bytes(c.cache.handle, n, 2 ** 31 - 1) == P.pask_prompt_workspace_bytes(c.cache.handle, n, 64 * n)
        assert P.pask_prompt_workspace_bytes(c.cache.handle, n, 64 * n) > P.pask_prompt_workspace_bytes(c.cache.handle, n, 8 * n) > 0
