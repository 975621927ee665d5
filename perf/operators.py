"""The latent-cache operators as workloads: their plain forms, the library's calls, and the exact results.

A latent cache holds one row of 576 values per token and layer (a 512-wide compressed key/value vector and the 64
rotary key dimensions all heads share) under the library's persistence table: released, kept in low precision
(2, 4 or 8 bits with one bf16 scale per 32 values) or kept in bf16.  Four operators work on it:

  write   pask_append_latent then pask_read_latent: rows are decided, quantised and compacted, and read back
  read    pask_read_latent: a sequence's retained rows as bf16, its bf16 stream first, then the low-precision one
  decode  pask_decode_attention_latent: one new query per sequence against the stored rows (absorbed form; the 512
          leading values of a row are its value vector for every head)
  prompt  pask_prompt_attention_latent: causal attention of a ragged batch with keys and values expanded per head

`own` selects the library's calls; otherwise the operators are computed with elementary torch operations in 32 bits.
"""
import math
import struct

import torch

own = False

ROW, LATENT, ROPE, GROUP = 576, 512, 64, 32
NOPE, VDIM, QDIM = 128, 128, 192
LEVELS = {2: 1, 4: 7, 8: 127}
RELEASE, LOW, HIGH = 0, 1, 2                      # tag == action in the table written by `_policy`
PAGE = 16


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one decode step's rows of a batch of 64 sequences: the smallest write, launches and latency only
        dict(name="write-step-b64", op="write", n_seqs=64, len_lo=1, len_hi=1, high=0.25, low=0.5, bits=4),
        # prompts of 2K tokens of a batch of 8, ragged, at the balanced mix of a third of the bytes kept
        dict(name="write-prompt-b8", op="write", n_seqs=8, len_lo=1777, len_hi=2305, high=0.25, low=0.4, bits=4),
        # the whole history of the 64-sequence batch with 2K to 8K tokens each: a bulk fill bound by bandwidth
        dict(name="write-bulk-b64", op="write", n_seqs=64, len_lo=2048, len_hi=8192, high=0.25, low=0.4, bits=4),
        # one short conversation read back before its next prompt chunk
        dict(name="read-one", op="read", n_seqs=1, len_lo=777, len_hi=777, high=0.4, low=0.5, bits=4),
        # 8 sequences of 8K + 1K tokens, eight-bit codes, read back for a chunk that follows
        dict(name="read-b8-9k", op="read", n_seqs=8, len_lo=8192, len_hi=9216, high=0.3, low=0.6, bits=8),
        # decode: a single user, a kilotoken of history all in bf16, 16 heads: latency and a deep split
        dict(name="decode-one-1k", op="decode", n_seqs=1, len_lo=1023, len_hi=1023, high=1.0, low=0.0, bits=4, heads=16),
        # decode: 8 sequences of 8K + 1K tokens, 32 heads, a third of the bytes kept
        dict(name="decode-b8-9k", op="decode", n_seqs=8, len_lo=8192, len_hi=9216, high=0.25, low=0.4, bits=4, heads=32),
        # decode: the 64-sequence batch of 2K to 8K tokens, full-precision cache, 128 heads: bytes and products both count
        dict(name="decode-b64-high", op="decode", n_seqs=64, len_lo=2048, len_hi=8192, high=1.0, low=0.0, bits=4, heads=128),
        # decode: 128 sequences of 16K tokens, most of them released, 64 heads
        dict(name="decode-b128-16k", op="decode", n_seqs=128, len_lo=15000, len_hi=16384, high=0.2, low=0.3, bits=4, heads=64),
        # prompt: one short question, 16 heads
        dict(name="prompt-one-short", op="prompt", n_seqs=1, q_lo=131, q_hi=131, hist=0, heads=16),
        # prompt: chunks of 512 tokens that follow a history read back from the cache, 32 heads
        dict(name="prompt-chunk-b4", op="prompt", n_seqs=4, q_lo=480, q_hi=512, hist=3333, heads=32),
        # prompt: a ragged batch of first prompts up to 8K tokens, 16 heads: bound by the matrix products
        dict(name="prompt-b4-8k", op="prompt", n_seqs=4, q_lo=4096, q_hi=8192, hist=0, heads=16),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, odd ones as they fall, never above the largest listed case."""
    op = rng.choice(["write", "read", "decode", "prompt"])
    if op == "prompt":
        heads = rng.choice([5, 8, 16, 24, 32])
        while True:
            n_seqs, q_hi, hist = _logint(rng, 1, 12), _logint(rng, 1, 8000), rng.choice([0, 0, _logint(rng, 1, 6000)])
            case = dict(op=op, n_seqs=n_seqs, q_lo=max(1, int(q_hi * rng.uniform(0.3, 1.0))), q_hi=q_hi, hist=hist, heads=heads)
            if work(case)["flops"] <= 8e11 and n_seqs * (q_hi + hist) <= 40000:
                return case
    while True:
        high = rng.choice([0.0, 1.0, rng.uniform(0.05, 0.9)])
        low = 0.0 if high == 1.0 else rng.uniform(0.1, 1.0 - high)
        # a decode or a read-back finds at least a few rows in every sequence
        n_seqs, len_hi = _logint(rng, 1, 160), _logint(rng, 1 if op == "write" else 40, 20000)
        len_lo = max(1 if op == "write" else 24, int(len_hi * rng.uniform(0.3, 1.0)))
        case = dict(op=op, n_seqs=n_seqs, len_lo=len_lo, len_hi=len_hi, high=high, low=low, bits=rng.choice([2, 4, 4, 8]))
        if op == "decode":
            case["heads"] = rng.choice([1, 8, 16, 20, 32, 40, 64, 96, 128])
        if n_seqs * len_hi >= 32 and work(case)["bytes"] <= 6e8 and work(case)["flops"] <= 1.3e11:
            return case


def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly spaced, in an order that mixes short and long ones; fixed by the case alone."""
    vals = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]
    return vals[::2] + vals[1::2][::-1]


def _counts(case):
    """Per sequence: tokens, those kept in bf16, those kept in low precision (the shares hold over the whole batch)."""
    out, seen, sum_h, sum_l = [], 0, 0, 0
    for n in _spread(case["len_lo"], case["len_hi"], case["n_seqs"]):
        seen += n
        nh = min(n, int(seen * case["high"] + 0.5) - sum_h)
        nl = max(0, min(n - nh, int(seen * case["low"] + 0.5) - sum_l))
        sum_h, sum_l = sum_h + nh, sum_l + nl
        out.append((n, nh, nl))
    return out


def _low_bytes(bits):
    return ROW * bits // 8 + 2 * ROW // GROUP


def work(case):
    """Inputs read once, outputs written once; products of the attention forms at two operations per multiply-add."""
    if case["op"] == "prompt":
        h, byts, flops = case["heads"], 0, 0
        for nq in _spread(case["q_lo"], case["q_hi"], case["n_seqs"]):
            nk = nq + case["hist"]
            pairs = nq * case["hist"] + nq * (nq + 1) // 2
            flops += 2 * pairs * (QDIM + VDIM) * h
            byts += nq * h * (QDIM + VDIM) * 2 + nq * h * 4 + nk * (h * (NOPE + VDIM) + ROPE) * 2
        return {"bytes": byts, "flops": flops}
    c = _counts(case)
    tok, nh, nl = sum(x[0] for x in c), sum(x[1] for x in c), sum(x[2] for x in c)
    stored = nh * 2 * ROW + nl * _low_bytes(case["bits"])
    if case["op"] == "write":      # retained rows and all tags in; stored bytes out; and read back
        return {"bytes": (nh + nl) * 2 * ROW + 2 * tok + 2 * stored + (nh + nl) * 2 * ROW, "flops": 4 * nl * ROW}
    if case["op"] == "read":
        return {"bytes": stored + (nh + nl) * 2 * ROW, "flops": nl * ROW}
    h, b = case["heads"], case["n_seqs"]
    return {"bytes": stored + b * h * (ROW * 2 + LATENT * 2 + 4), "flops": 2 * (nh + nl) * h * (ROW + LATENT)}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(0x5EED ^ (seed * 2654435761 & 0x7FFFFFFF))
    return g


def _normal(shape, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _tags(n, nh, nl, g):
    t = torch.zeros(n, dtype=torch.uint8, device="cuda")
    perm = torch.randperm(n, generator=g, device="cuda")
    t[perm[:nh]] = HIGH
    t[perm[nh:nh + nl]] = LOW
    return t


def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _policy(bits):
    """A table of three tags in one layer group: tag a takes action a."""
    blob = b"PASK" + struct.pack("<9I", 1, 3, 1, 1, 0, 65536, 0, bits, GROUP) + b"\0\0\0\0"
    for a in (RELEASE, LOW, HIGH):
        blob += struct.pack("<BBHff", a, 0, 0, 1.0, 1.0)
    return blob


def _library_cache(case, heads, max_append):
    import paper_2608_28276_b200 as pask
    counts = _counts(case)
    pages_h = sum((nh + PAGE - 1) // PAGE for _, nh, _ in counts)
    pages_l = sum((nl + PAGE - 1) // PAGE for _, _, nl in counts)
    return pask.LatentCache(_policy(case["bits"]), 1, heads, case["n_seqs"], max(n for n, _, _ in counts), max_append, pages_h, pages_l,
                            low_bits=case["bits"])


def _rows_inputs(case, seed):
    """Latent rows and tags of every sequence, in turn (generated as they are asked for)."""
    g = _gen(seed)
    for n, nh, nl in _counts(case):
        yield _normal((n, ROW), g), _tags(n, nh, nl, g)


def _quantise(x, bits):
    """Codes around zero (int8) and bf16 scales of rows x [n][576], groups of 32 values: scale = bf16(amax / levels), zero
    if that is not a normal number; code = x / scale rounded to the nearest whole number, ties to even."""
    v = x.float().view(-1, ROW // GROUP, GROUP)
    a = v.abs().amax(-1)
    s = (a / torch.full_like(a, float(LEVELS[bits]))).to(torch.bfloat16)
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    q = v.double() / s.double().clamp_min(2.0 ** -126).unsqueeze(-1)    # 64 bits: values next to a rounding border
    q = torch.where((s == 0).unsqueeze(-1), torch.zeros_like(q), q)
    return q.round().to(torch.int8), s


def _dequantise(codes, scales):
    return (codes.float() * scales.float().unsqueeze(-1)).to(torch.bfloat16).view(-1, ROW)


def prepare(case, seed):
    op = case["op"]
    if op == "prompt":
        g, h = _gen(seed), case["heads"]
        nq = _spread(case["q_lo"], case["q_hi"], case["n_seqs"])
        nk = [n + case["hist"] for n in nq]
        tq, tk = sum(nq), sum(nk)
        st = dict(case=case, nq=nq, nk=nk, cu_q=_cu(nq), cu_k=_cu(nk), scale=QDIM ** -0.5, q=_normal((tq, h, QDIM), g),
                  kv=_normal((tk, h, NOPE + VDIM), g), k_rope=_normal((tk, ROPE), g))
        if own:
            st["out"] = torch.empty((tq, h, VDIM), dtype=torch.bfloat16, device="cuda")
            st["lse"] = torch.empty((tq, h), dtype=torch.float32, device="cuda")
        return st
    counts = _counts(case)
    st = dict(case=case, kept=[nh + nl for _, nh, nl in counts])
    st["cu_rows"] = _cu(st["kept"])
    ids = torch.arange(case["n_seqs"], dtype=torch.int32, device="cuda")
    if op == "write":
        rows, tags = zip(*_rows_inputs(case, seed))
        st.update(latent=torch.cat(rows), tags=torch.cat(tags), cu=_cu([n for n, _, _ in counts]), ids=ids)
        if own:
            total = st["latent"].shape[0]
            st["cache"] = _library_cache(case, 16, total)
            st["actions"] = torch.empty(total, dtype=torch.uint8, device="cuda")
        else:
            st["lut"] = torch.tensor([RELEASE, LOW, HIGH], dtype=torch.uint8, device="cuda")
    elif own:
        import paper_2608_28276_b200 as pask
        st["ids"], st["cache"] = ids, _library_cache(case, case.get("heads", 16), max(n for n, _, _ in counts))
        for i, (x, t) in enumerate(_rows_inputs(case, seed)):
            pask.pask_append_latent(st["cache"].handle, 0, ids[i:i + 1].clone(), _cu([x.shape[0]]), x, t)
    else:
        st["hist"] = []
        for x, t in _rows_inputs(case, seed):
            codes, scales = _quantise(x[t == LOW], case["bits"])
            st["hist"].append((x[t == HIGH], codes, scales))
    if own and op != "decode":
        st["rows"] = torch.empty((sum(st["kept"]), ROW), dtype=torch.bfloat16, device="cuda")
        st["lens"] = torch.empty((case["n_seqs"], 2), dtype=torch.int32, device="cuda")
    if op == "decode":
        g = _gen(seed + 7919)
        h = case["heads"]
        st["q"], st["scale"] = _normal((case["n_seqs"], h, ROW), g), QDIM ** -0.5
        if own:
            st["out"] = torch.empty((case["n_seqs"], h, LATENT), dtype=torch.bfloat16, device="cuda")
            st["lse"] = torch.empty((case["n_seqs"], h), dtype=torch.float32, device="cuda")
            st["ws"] = st["cache"].workspace(case["n_seqs"])
    return st


# ------------------------------------------------------------------------------------------------ one pass

def _run_own(st):
    import paper_2608_28276_b200 as pask
    op = st["case"]["op"]
    if op == "prompt":
        pask.pask_prompt_attention_latent(st["cu_q"], st["cu_k"], st["q"], st["kv"], st["k_rope"], st["scale"], st["out"], st["lse"])
        return st["out"], st["lse"]
    cache = st["cache"].handle
    if op == "decode":
        pask.pask_decode_attention_latent(cache, 0, st["ids"], st["q"], st["scale"], st["out"], st["lse"], st["ws"])
        return st["out"], st["lse"]
    if op == "write":
        pask.pask_cache_reset(cache)               # the sequences start afresh, as a new batch of prompts does
        pask.pask_append_latent(cache, 0, st["ids"], st["cu"], st["latent"], st["tags"], actions_out=st["actions"])
    pask.pask_read_latent(cache, 0, st["ids"], st["cu_rows"], st["rows"], st["lens"])
    return (st["actions"], st["rows"], st["lens"]) if op == "write" else (st["rows"], st["lens"])


def _attend(q, k, v, scale, mask=None):
    """Softmax attention of heads q [h][n][d] with k [h or 1][m][d], v [h or 1][m][e] in 32 bits; out and log-sum-exp."""
    s = torch.matmul(q, k.transpose(-1, -2)) * scale
    if mask is not None:
        s = s.masked_fill(~mask, float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / l, (m + torch.log(l)).squeeze(-1)


def run(st):
    if own:
        return _run_own(st)
    case, op = st["case"], st["case"]["op"]
    if op == "prompt":
        outs, lses, oq, ok = [], [], 0, 0
        for nq, nk in zip(st["nq"], st["nk"]):
            q = st["q"][oq:oq + nq].float().transpose(0, 1)
            kv = st["kv"][ok:ok + nk].float().transpose(0, 1)
            rope = st["k_rope"][ok:ok + nk].float()
            mask = torch.arange(nk, device="cuda")[None, :] <= torch.arange(nq, device="cuda")[:, None] + (nk - nq)
            o = torch.empty((nq, case["heads"], VDIM), dtype=torch.bfloat16, device="cuda")
            l = torch.empty((nq, case["heads"]), dtype=torch.float32, device="cuda")
            step = max(1, int(2e9 // (4 * nq * nk)))               # heads at a time, to bound the scores' memory
            for h in range(0, case["heads"], step):
                kk = torch.cat([kv[h:h + step, :, :NOPE], rope.expand(kv[h:h + step].shape[0], -1, -1)], -1)
                oo, ll = _attend(q[h:h + step], kk, kv[h:h + step, :, NOPE:], st["scale"], mask)
                o[:, h:h + step] = oo.transpose(0, 1).to(torch.bfloat16)
                l[:, h:h + step] = ll.transpose(0, 1)
            outs.append(o)
            lses.append(l)
            oq, ok = oq + nq, ok + nk
        return torch.cat(outs), torch.cat(lses)
    if op == "decode":
        outs, lses = [], []
        for i, (hi, codes, scales) in enumerate(st["hist"]):
            rows = torch.cat([hi, _dequantise(codes, scales)]).float()
            o, l = _attend(st["q"][i].float(), rows, rows[:, :LATENT], st["scale"])
            outs.append(o.to(torch.bfloat16))
            lses.append(l)
        return torch.stack(outs), torch.stack(lses)
    if op == "read":
        lens = torch.tensor([[h.shape[0], c.shape[0]] for h, c, _ in st["hist"]], dtype=torch.int32, device="cuda")
        return torch.cat([r for h, c, s in st["hist"] for r in (h, _dequantise(c, s))]), lens
    # write: look the actions up, bring each sequence's bf16 rows before its low-precision ones, quantise those
    x, actions, cu = st["latent"], st["lut"][st["tags"].long()], st["cu"].long()
    seq = torch.searchsorted(cu[1:], torch.arange(x.shape[0], device="cuda"), right=True)
    n = case["n_seqs"]
    lens = torch.stack([torch.zeros(n, dtype=torch.int32, device="cuda").index_add_(0, seq, (actions == a).int()) for a in (HIGH, LOW)], 1)
    key = torch.where(actions == RELEASE, torch.full_like(seq, 2 * n), 2 * seq + (actions == LOW).long())
    order = torch.argsort(key, stable=True)[:sum(st["kept"])]
    kept, low = x[order], (actions[order] == LOW)
    return actions, torch.where(low[:, None], _dequantise(*_quantise(kept, case["bits"])), kept), lens


# ------------------------------------------------------------------------------------------------ exact results

def _stored_rows_exact(x, t, bits):
    """The rows of one sequence that the cache holds, in 64 bits, from the format's definition."""
    lo = x[t == LOW].double().reshape(-1, GROUP)
    amax = lo.abs().max(dim=1, keepdim=True).values if lo.numel() else lo[:, :1]
    s = (amax / LEVELS[bits]).to(torch.bfloat16).double()
    s[s < 2.0 ** -126] = 0.0
    code = torch.where(s > 0, torch.round(lo / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(lo))
    low_rows = (code * s).to(torch.bfloat16).double().reshape(-1, ROW)
    return torch.cat([x[t == HIGH].double(), low_rows])


def exact(case, seed):
    op = case["op"]
    if op == "prompt":
        h = case["heads"]
        if work(case)["flops"] > 6e12:
            return None
        g = _gen(seed)
        nq = _spread(case["q_lo"], case["q_hi"], case["n_seqs"])
        nk = [n + case["hist"] for n in nq]
        q, kv, rope = _normal((sum(nq), h, QDIM), g), _normal((sum(nk), h, NOPE + VDIM), g), _normal((sum(nk), ROPE), g)
        out, lse = torch.empty((sum(nq), h, VDIM), dtype=torch.float64, device="cuda"), torch.empty((sum(nq), h), dtype=torch.float64, device="cuda")
        oq = ok = 0
        for a, b in zip(nq, nk):
            hidden = torch.ones((a, b), dtype=torch.bool, device="cuda").triu(b - a + 1)
            for i in range(h):
                s = q[oq:oq + a, i, :NOPE].double() @ kv[ok:ok + b, i, :NOPE].double().T
                s = (s + q[oq:oq + a, i, NOPE:].double() @ rope[ok:ok + b].double().T) / math.sqrt(QDIM)
                s[hidden] = float("-inf")
                lse[oq:oq + a, i] = torch.logsumexp(s, dim=1)
                out[oq:oq + a, i] = torch.exp(s - lse[oq:oq + a, i, None]) @ kv[ok:ok + b, i, NOPE:].double()
            oq, ok = oq + a, ok + b
        return out, lse
    rows, acts = [], []
    outs, lses = [], []
    q = _normal((case["n_seqs"], case["heads"], ROW), _gen(seed + 7919)).double() / math.sqrt(QDIM) if op == "decode" else None
    for i, (x, t) in enumerate(_rows_inputs(case, seed)):
        r = _stored_rows_exact(x, t, case["bits"])
        if op == "decode":
            s = q[i] @ r.T
            lse = torch.logsumexp(s, dim=1)
            outs.append(torch.exp(s - lse[:, None]) @ r[:, :LATENT])
            lses.append(lse)
        else:
            rows.append(r)
            acts.append(t)
    if op == "decode":
        return torch.stack(outs), torch.stack(lses)
    lens = torch.tensor([[nh, nl] for _, nh, nl in _counts(case)], dtype=torch.int32, device="cuda")
    return (torch.cat(acts), torch.cat(rows), lens) if op == "write" else (torch.cat(rows), lens)
