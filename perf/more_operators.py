"""Rotary positions and prompt attention over a mixed-precision cache as workloads: plain forms, the library's calls, exact results.

A layer's step in front of the cache is: project to q, k, v; rotate q and k by their tokens' positions; attend; persist k and
v as the table decides.  Two operators of that step:

  rotary  pask_rotary: q and k of a ragged batch rotated pair by pair by position times frequency.  Pairs are the two halves of the
          rotated dims or neighbours; the rotated dims may be a part of the head; frequencies may be scaled for long contexts; the
          transposed rotation is the gradient.
  prompt  pask_prompt_attention: causal attention of the tokens of a ragged batch (whole prompts, chunks of one, forced or drafted
          tokens of a decode step), as given, behind what the cache retains of their sequences: bf16 rows, rows of 2, 4 or
          8 bits (whose values enter rounded to bf16), and the protected window of the last tokens.

`own` selects the library's calls; otherwise the operators are computed with elementary torch operations in 32 bits (angles in 64).
"""
import math
import struct

import torch

own = False

DIM = 128                                         # head dims of the cache
GQA = 4                                           # query heads of a key / value head
GROUP = 32                                        # values with a scale in common
LEVELS = {2: 1, 4: 7, 8: 127}
RELEASE, LOW, HIGH = 0, 1, 2                      # tag == action in the table written by `_policy`
PAGE = 16
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BASE = 1000000.0


# ------------------------------------------------------------------------------------------------ cases

def listed():
    rot = dict(op="rotary", heads_q=32, heads_k=8, dim=128, rot=128, pairs=False, dtype="bf16", transpose=False, rule="plain", factor=1.0,
               source="fused")
    pro = dict(op="prompt", n_kv=8, high=0.25, low=0.4, bits=4, window=0)
    return [
        # one token of one sequence: launch latency
        dict(rot, name="rotary-step-one", tokens=1, far=8191),
        # a decode step of the 64-sequence batch
        dict(rot, name="rotary-step-b64", tokens=64, far=8192),
        # prompts of 17 thousand tokens in all at far positions of a long context, frequencies scaled by their rotations
        dict(rot, name="rotary-prompt-17k", tokens=17001, far=262144, rule="rotations", factor=8.0),
        # the rotary dims of a latent model's queries (the last 64 of 192) and rows (the last 64 of 576), neighbours paired
        dict(rot, name="rotary-latent-16k", tokens=16000, far=131072, heads_q=32, heads_k=1, dim=64, rot=64, pairs=True, rule="index", factor=40.0,
             source="latent"),
        # the gradient of a rotation of a quarter of the head, in fp32
        dict(rot, name="rotary-grad-part-fp32", tokens=4099, far=32768, heads_q=16, heads_k=4, rot=32, dtype="fp32", transpose=True, source="rows"),
        # one short question on its own
        dict(pro, name="prompt-one-short", n_seqs=1, q_lo=131, q_hi=131, hist_lo=0, hist_hi=0),
        # tokens that the grammar forces, behind the 32K-token history of a single user, two-bit codes
        dict(pro, name="prompt-forced-one-32k", n_seqs=1, q_lo=17, q_hi=17, hist_lo=32768, hist_hi=32768, bits=2),
        # five drafted tokens for each of 64 sequences of 2K to 8K tokens, a third of the bytes kept: bound by the cache's bytes
        dict(pro, name="prompt-draft-b64", n_seqs=64, q_lo=5, q_hi=5, hist_lo=2048, hist_hi=8192),
        # ragged short chunks behind a history with a protected window, two key / value heads
        dict(pro, name="prompt-window-b16", n_seqs=16, n_kv=2, q_lo=33, q_hi=120, hist_lo=2500, hist_hi=3333, window=64),
        # chunks of 512 tokens of 8 sequences behind 8K + 1K tokens, eight-bit codes
        dict(pro, name="prompt-chunk-b8-9k", n_seqs=8, q_lo=480, q_hi=512, hist_lo=8192, hist_hi=9216, high=0.3, low=0.6, bits=8),
        # a ragged batch of first prompts of 4K to 8K tokens: bound by the matrix products
        dict(pro, name="prompt-b4-8k", n_seqs=4, q_lo=4096, q_hi=8192, hist_lo=0, hist_hi=0),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, odd ones as they fall, never above the largest listed case."""
    if rng.random() < 0.4:
        while True:
            source = rng.choice(["fused", "rows", "latent"])
            dim = 64 if source == "latent" else rng.choice([64, 80, 96, 128, 128, 192])
            rot = dim if source == "latent" else rng.choice([dim, dim, dim // 2, dim // 4])
            heads_k = 1 if source == "latent" else rng.choice([1, 2, 4, 8])
            case = dict(op="rotary", tokens=_logint(rng, 1, 40000), far=_logint(rng, 100, 1000000), heads_q=rng.choice([4, 7, 16, 32, 40]), heads_k=heads_k,
                        dim=dim, rot=rot, pairs=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), transpose=rng.random() < 0.3,
                        rule=rng.choice(["plain", "linear", "rotations", "index"]), factor=float(rng.choice([1, 2, 4, 8, 40])), source=source)
            if work(case)["bytes"] <= 6e8:
                return case
    while True:
        high = rng.choice([0.0, 1.0, rng.uniform(0.05, 0.9)])
        low = 0.0 if high == 1.0 else rng.uniform(0.1, 1.0 - high)
        q_hi, hist_hi = _logint(rng, 1, 8000), rng.choice([0, _logint(rng, 1, 20000), _logint(rng, 1, 20000)])
        case = dict(op="prompt", n_seqs=_logint(rng, 1, 80), n_kv=rng.choice([1, 2, 4, 8]), q_lo=max(1, int(q_hi * rng.uniform(0.3, 1.0))), q_hi=q_hi,
                    hist_lo=int(hist_hi * rng.uniform(0.3, 1.0)), hist_hi=hist_hi, high=high, low=low, bits=rng.choice([2, 4, 4, 8]),
                    window=rng.choice([0, 0, 0, 16, 64, 256]))
        w = work(case)
        if w["bytes"] <= 5e8 and w["flops"] <= 9e11 and case["n_seqs"] * q_hi <= 40000 and case["n_seqs"] * hist_hi <= 600000:
            return case


def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly spaced, in an order that mixes short and long ones; fixed by the case alone."""
    vals = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]
    return vals[::2] + vals[1::2][::-1]


def _counts(case):
    """Per sequence: tokens of history, those kept in bf16, those kept in low precision (the shares hold over the whole batch)."""
    out, seen, sum_h, sum_l = [], 0, 0, 0
    for n in _spread(case["hist_lo"], case["hist_hi"], case["n_seqs"]):
        seen += n
        nh = min(n, int(seen * case["high"] + 0.5) - sum_h)
        nl = max(0, min(n - nh, int(seen * case["low"] + 0.5) - sum_l))
        sum_h, sum_l = sum_h + nh, sum_l + nl
        out.append((n, nh, nl))
    return out


def work(case):
    """Inputs read once, outputs written once; products of attention at two operations per multiply-add."""
    if case["op"] == "rotary":
        values = case["tokens"] * (case["heads_q"] + case["heads_k"]) * case["dim"]
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": 2 * values * size + 4 * case["tokens"] + 8 * case["rot"] // 2, "flops": 3 * values * case["rot"] // case["dim"]}
    n_kv, byts, flops = case["n_kv"], 0.0, 0
    for nq, (n, nh, nl) in zip(_spread(case["q_lo"], case["q_hi"], case["n_seqs"]), _counts(case)):
        w = min(n, case["window"])
        rest = (n - w) / n if n else 0.0          # share of the streams that the window does not stand in for
        keys = w + rest * (nh + nl)
        byts += n_kv * ((w + rest * nh) * 4 * DIM + rest * nl * 2 * (DIM * case["bits"] // 8 + DIM // GROUP * 2))
        byts += nq * n_kv * (GQA * (4 * DIM + 4) + 4 * DIM)
        flops += 4 * DIM * GQA * n_kv * (nq * keys + nq * (nq + 1) // 2)
    return {"bytes": int(byts), "flops": int(flops)}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(0x70717 ^ (seed * 2654435761 & 0x7FFFFFFF))
    return g


def _normal(shape, g, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _cu(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _rotary_inputs(case, seed):
    """positions int32 [tokens]; q [tokens][heads_q][dim] and k [tokens][heads_k][dim] as a model has them: views of wider rows."""
    g, t, dt = _gen(seed), case["tokens"], TYPES[case["dtype"]]
    hq, hk, d = case["heads_q"], case["heads_k"], case["dim"]
    # runs of consecutive positions, as the prompts of a batch have them (single positions in a decode step)
    run = max(1, t // 8)
    first = torch.randint(0, max(1, case["far"] - run + 1), ((t + run - 1) // run,), generator=g, device="cuda")
    pos = (first.repeat_interleave(run)[:t] + torch.arange(t, device="cuda") % run).to(torch.int32)
    if case["source"] == "latent":                # the last dims of queries of 128 + 64 and of rows of 512 + 64
        return pos, _normal((t, hq, 192), g, dt)[:, :, 128:], _normal((t, 1, 576), g, dt)[:, :, 512:]
    if case["source"] == "fused":                 # one projection's output: queries, keys, values
        row = _normal((t, hq + 2 * hk, d), g, dt)
        return pos, row[:, :hq], row[:, hq:hq + hk]
    return pos, _normal((t, hq, d), g, dt), _normal((t, hk, d), g, dt)


CONTEXT, FEW, MANY = 4096, 1.0, 32.0              # trained context; rotations over it below / above which a pair counts as slow / fast


def _frequencies(case):
    """Radians a position of each pair: base^(-2i/rot), those that turn slowly divided by the factor."""
    n, out = case["rot"] // 2, []
    for i in range(n):
        f = BASE ** (-2.0 * i / case["rot"])
        if case["rule"] == "linear":
            f /= case["factor"]
        elif case["rule"] == "rotations":         # share kept: linear in the rotations over the trained context
            r = CONTEXT * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (r - FEW) / (MANY - FEW)))
            f = f * keep + f / case["factor"] * (1 - keep)
        elif case["rule"] == "index":             # linear in the pair's index, between the (whole) indexes with MANY and FEW rotations
            at = [case["rot"] * math.log(CONTEXT / (x * 2 * math.pi)) / (2 * math.log(BASE)) for x in (MANY, FEW)]
            lo, hi = max(0, math.floor(at[0])), min(case["rot"] - 1, math.ceil(at[1]))
            keep = 1 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            f = f * keep + f / case["factor"] * (1 - keep)
        out.append(f)
    return out


def _magnitude(case):
    return 1.0 if case["rule"] in ("plain", "linear") else 0.1 * math.log(case["factor"]) + 1.0


def _policy(bits, window):
    """A table of three tags in one layer group: tag a takes action a."""
    blob = b"PASK" + struct.pack("<9I", 1, 3, 1, 1, 0, 65536, window, bits, GROUP) + b"\0\0\0\0"
    for a in (RELEASE, LOW, HIGH):
        blob += struct.pack("<BBHff", a, 0, 0, 1.0, 1.0)
    return blob


def _history(case, seed):
    """k, v [n][n_kv][128] and tags of every sequence's history, in turn (generated as they are asked for)."""
    g = _gen(seed + 101)
    for n, nh, nl in _counts(case):
        t = torch.zeros(n, dtype=torch.uint8, device="cuda")
        perm = torch.randperm(n, generator=g, device="cuda")
        t[perm[:nh]] = HIGH
        t[perm[nh:nh + nl]] = LOW
        yield _normal((n, case["n_kv"], DIM), g), _normal((n, case["n_kv"], DIM), g), t


def _prompt_inputs(case, seed):
    g, nq = _gen(seed), _spread(case["q_lo"], case["q_hi"], case["n_seqs"])
    t = sum(nq)
    return nq, _normal((t, GQA * case["n_kv"], DIM), g), _normal((t, case["n_kv"], DIM), g), _normal((t, case["n_kv"], DIM), g)


def _quantise(x, bits):
    """Codes around zero (int8) and fp16 scales of rows x [n][heads][128], groups of 32 values: scale = fp16(amax / levels), code =
    x times the scale's reciprocal, rounded to the nearest whole number, ties to even."""
    v = x.float().view(*x.shape[:-1], DIM // GROUP, GROUP)
    a = v.abs().amax(-1)
    s = (a / torch.full_like(a, float(LEVELS[bits]))).clamp_max(65504.0).to(torch.float16)
    f = s.float()
    inv = torch.where(f > 0, torch.ones_like(f) / f, torch.zeros_like(f))
    return (v * inv.unsqueeze(-1)).round().clamp(-LEVELS[bits], LEVELS[bits]).to(torch.int8), s


def _dequantise(codes, scales):
    return (codes.float() * scales.float().unsqueeze(-1)).to(torch.bfloat16).flatten(-2)


def _library_cache(case):
    import paper_2608_28276_b200 as pask
    counts = _counts(case)
    pages_h = sum((nh + PAGE - 1) // PAGE for _, nh, _ in counts)
    pages_l = sum((nl + PAGE - 1) // PAGE for _, _, nl in counts)
    most = max(1, max(n for n, _, _ in counts))
    return pask.Cache(_policy(case["bits"], case["window"]), 1, GQA * case["n_kv"], case["n_kv"], case["n_seqs"], most, most, pages_h, pages_l,
                      recent_window=case["window"], low_bits=case["bits"])


def _rows(parts):
    """Rows of every sequence [n][...] as one padded tensor [sequences][longest][...]."""
    return torch.nn.utils.rnn.pad_sequence(parts, batch_first=True)


def prepare(case, seed):
    if case["op"] == "rotary":
        pos, q, k = _rotary_inputs(case, seed)
        st = dict(case=case, pos=pos, q=q, k=k)
        if own:
            import paper_2608_28276_b200 as pask
            scaling = {"plain": pask.ROTARY_PLAIN, "linear": pask.ROTARY_LINEAR, "rotations": pask.ROTARY_ROTATIONS, "index": pask.ROTARY_INDEX}
            st["table"] = pask.pask_rotary_table(case["rot"], BASE, scaling[case["rule"]], case["factor"], CONTEXT, FEW, MANY)
            st["q_out"], st["k_out"] = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda")
        else:
            st["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        return st
    nq, q, k, v = _prompt_inputs(case, seed)
    st = dict(case=case, nq=nq, cu=_cu(nq), q=q, k=k, v=v)
    if own:
        import paper_2608_28276_b200 as pask
        st["ids"] = torch.arange(case["n_seqs"], dtype=torch.int32, device="cuda")
        st["cache"] = _library_cache(case)
        for i, (hk, hv, t) in enumerate(_history(case, seed)):
            if t.numel():
                pask.pask_append_kv(st["cache"].handle, 0, st["ids"][i:i + 1].clone(), _cu([t.numel()]), hk, hv, t)
        st["out"] = torch.empty_like(q)
        st["lse"] = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        st["ws"] = st["cache"].prompt_workspace(case["n_seqs"], q.shape[0])
        return st
    whole, codes = ([], []), ([], [], [], [])
    for hk, hv, t in _history(case, seed):
        n = t.numel()
        recent = torch.arange(n, device="cuda") >= n - case["window"]
        keep, low = recent | (t == HIGH), ~recent & (t == LOW)
        whole[0].append(hk[keep])
        whole[1].append(hv[keep])
        for at, part in zip((0, 2), (hk, hv)):
            c, s = _quantise(part[low], case["bits"])
            codes[at].append(c)
            codes[at + 1].append(s)
    st["n_whole"], st["n_low"] = [x.shape[0] for x in whole[0]], [x.shape[0] for x in codes[0]]
    st["whole"], st["codes"] = [_rows(x) for x in whole], [_rows(x) for x in codes]
    return st


# ------------------------------------------------------------------------------------------------ one pass

def _run_own(st):
    import paper_2608_28276_b200 as pask
    case = st["case"]
    if case["op"] == "rotary":
        pask.pask_rotary(st["pos"], st["table"], [(st["q"], st["q_out"]), (st["k"], st["k_out"])], interleaved=case["pairs"],
                         transpose=case["transpose"], magnitude=_magnitude(case))
        return st["q_out"], st["k_out"]
    pask.pask_prompt_attention(st["cache"].handle, 0, st["ids"], st["cu"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["ws"])
    return st["out"], st["lse"]


def _rotate(x, cos, sin, case):
    rot = case["rot"]
    f, out = x.float(), torch.empty(x.shape, dtype=x.dtype, device="cuda")
    a, b = (f[..., 0:rot:2], f[..., 1:rot:2]) if case["pairs"] else (f[..., :rot // 2], f[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    if case["pairs"]:
        out[..., 0:rot:2], out[..., 1:rot:2] = ra.to(x.dtype), rb.to(x.dtype)
    else:
        out[..., :rot // 2], out[..., rot // 2:rot] = ra.to(x.dtype), rb.to(x.dtype)
    out[..., rot:] = x[..., rot:]
    return out


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    if case["op"] == "rotary":
        ang = st["pos"].double()[:, None] * st["freq"]
        cos, sin = (torch.cos(ang) * _magnitude(case)).float()[:, None], (torch.sin(ang) * _magnitude(case)).float()[:, None]
        if case["transpose"]:
            sin = -sin
        return _rotate(st["q"], cos, sin, case), _rotate(st["k"], cos, sin, case)
    n_kv, nq, total = case["n_kv"], st["nq"], st["q"].shape[0]
    out, lse = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
    most = [max(nq), max(st["n_whole"]), max(st["n_low"])]
    per = 4 * GQA * n_kv * most[0] * (most[0] + most[1] + most[2])     # bytes of a sequence's scores
    step, heads = max(1, int(4e9 // per)), max(1, min(n_kv, int(4e9 * n_kv // per)))
    for s in range(0, len(nq), step):                                  # as many sequences and heads at a time as memory is good for
        e = min(len(nq), s + step)
        mq, mw, ml = max(nq[s:e]), max(st["n_whole"][s:e]), max(st["n_low"][s:e])
        cu, at = st["cu"].long(), torch.arange(max(mq, mw, ml), device="cuda")
        mine = at[None, :mq] < (cu[s + 1:e + 1] - cu[s:e])[:, None]
        idx = (cu[s:e, None] + at[None, :mq]).clamp_max(total - 1)
        seen = torch.cat([at[None, :mw] < torch.tensor(st["n_whole"][s:e], device="cuda")[:, None],
                          at[None, :ml] < torch.tensor(st["n_low"][s:e], device="cuda")[:, None]], 1)
        mask = torch.cat([seen[:, None].expand(-1, mq, -1), (at[None, :mq] <= at[:mq, None]).expand(e - s, -1, -1)], 2)[:, None]
        low = [_dequantise(c[s:e, :ml], d[s:e, :ml]) for c, d in (st["codes"][:2], st["codes"][2:])]
        keys = torch.cat([st["whole"][0][s:e, :mw], low[0], st["k"][idx]], 1)
        values = torch.cat([st["whole"][1][s:e, :mw], low[1], st["v"][idx]], 1)
        for h in range(0, n_kv, heads):
            kk, vv = keys[:, :, h:h + heads].float().transpose(1, 2), values[:, :, h:h + heads].float().transpose(1, 2)
            qq = st["q"][idx][:, :, GQA * h:GQA * (h + heads)].float().transpose(1, 2).unflatten(1, (-1, GQA)).flatten(2, 3)
            x = torch.matmul(qq, kk.transpose(-1, -2)) * DIM ** -0.5   # [sequence][kv head][query head, token][key]
            x = x.unflatten(2, (GQA, -1)).masked_fill(~mask[:, :, None], float("-inf")).flatten(2, 3)
            m = x.amax(-1, keepdim=True)
            p = torch.exp(x - m)
            l = p.sum(-1, keepdim=True)
            o = (torch.matmul(p, vv) / l).unflatten(2, (GQA, -1)).flatten(1, 2).transpose(1, 2)
            b = (m + torch.log(l)).squeeze(-1).unflatten(2, (GQA, -1)).flatten(1, 2).transpose(1, 2)
            rows = slice(sum(nq[:s]), sum(nq[:e]))
            out[rows, GQA * h:GQA * (h + heads)] = o[mine].to(out.dtype)
            lse[rows, GQA * h:GQA * (h + heads)] = b[mine]
    return out, lse


# ------------------------------------------------------------------------------------------------ exact results

def _exact_rotation(x, pos, freq, case):
    """Pairs as complex numbers times magnitude e^(i position frequency) (its conjugate for the transpose)."""
    rot, n = case["rot"], case["rot"] // 2
    y = x.double().clone()
    head = y[..., :rot].reshape(*y.shape[:-1], n, 2) if case["pairs"] else y[..., :rot].reshape(*y.shape[:-1], 2, n).transpose(-1, -2)
    turn = torch.polar(torch.full((pos.numel(), n), _magnitude(case), dtype=torch.float64, device="cuda"), torch.outer(pos.double(), freq))
    z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * (turn.conj().resolve_conj() if case["transpose"] else turn)[:, None])
    y[..., :rot] = z.reshape(*y.shape[:-1], rot) if case["pairs"] else z.transpose(-1, -2).reshape(*y.shape[:-1], rot)
    return y


def _stored_exact(x, bits):
    """What low-precision rows stand for, in 64 bits, from the format's definition: bf16(code * scale)."""
    g = x.reshape(-1, GROUP)
    top = g.abs().max(dim=1, keepdim=True).values.float() if g.numel() else g[:, :1].float()
    s = torch.minimum(top / torch.full_like(top, LEVELS[bits]), torch.full_like(top, 65504.0)).half()
    r = torch.reciprocal(s.float())
    c = torch.clamp(torch.round(g.float() * r), -LEVELS[bits], LEVELS[bits])
    c = torch.where(s > 0, c, torch.zeros_like(c))
    return (c.double() * s.double()).to(torch.bfloat16).double().reshape(x.shape)


def exact(case, seed):
    if case["op"] == "rotary":
        pos, q, k = _rotary_inputs(case, seed)
        freq = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
        return _exact_rotation(q, pos, freq, case), _exact_rotation(k, pos, freq, case)
    if work(case)["flops"] > 6e12:
        return None
    nq, q, k, v = _prompt_inputs(case, seed)
    out, lse = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    a = 0
    for n, (hk, hv, t) in zip(nq, _history(case, seed)):
        old = max(0, t.numel() - case["window"])
        kept = [torch.cat([h[old:].double(), h[:old][t[:old] == HIGH].double(), _stored_exact(h[:old][t[:old] == LOW], case["bits"])]) for h in (hk, hv)]
        m = kept[0].shape[0]
        hidden = torch.ones((n, m + n), dtype=torch.bool, device="cuda").triu(m + 1)
        for h in range(q.shape[1]):
            keys, values = (torch.cat([part[:, h // GQA], new[a:a + n, h // GQA].double()]) for part, new in zip(kept, (k, v)))
            x = (q[a:a + n, h].double() @ keys.T) / math.sqrt(DIM)
            x[hidden] = float("-inf")
            lse[a:a + n, h] = torch.logsumexp(x, dim=1)
            out[a:a + n, h] = torch.exp(x - lse[a:a + n, h, None]) @ values
        a += n
    return out, lse
