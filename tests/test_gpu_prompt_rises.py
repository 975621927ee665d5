"""pask_prompt_attention where a row's largest score rises late and by much, so that outputs so far are rescaled between the products of two
blocks of keys: in either half of a block of 128, in every one or with blocks between that do not rise, for every number of tokens
that shares a tile and every format of the history."""
import pytest
import torch

import prompt_ref as R
from test_gpu_prompt import Case

pytestmark = pytest.mark.gpu

BLOCK, STEP = 128, 7.0                             # keys of a block; rise of the largest score a step (e^7: more than the 2^8 that are let pass)


@pytest.fixture(scope="module")
def P():
    import paper_2608_28276_b200 as pask
    return pask


def rising_keys(n, n_kv, slots, g):
    """Keys of n tokens that score little, but those at `slots`: each STEP above the one before.  And the direction that they score in."""
    u = (torch.randint(0, 2, (n_kv, 128), generator=g, device="cuda") * 2 - 1).float()
    k = torch.randn((n, n_kv, 128), generator=g, device="cuda") * 0.3
    for i, s in enumerate(slots):
        k[s] = u * (STEP * (i + 1) / 128 ** 0.5)   # u u / sqrt(128) = sqrt(128)
    return k.to(torch.bfloat16), u


def slots_of(i, n, half, blocks):
    """Sequence i: one late block alone, or every first, second, third one."""
    at = [i] if i < blocks else list(range(0, blocks, i - blocks + 1))
    return [s for s in (BLOCK * b + 64 * half + (13 * b + 7 * i) % 64 for b in at) if s < n]


def queries(us, nq, g):
    """[tokens][query heads][128] that look in their key head's direction."""
    rows = torch.cat([u.repeat_interleave(4, 0)[None].expand(n, -1, -1) for u, n in zip(us, nq)])
    return (rows + 0.1 * torch.randn(rows.shape, generator=g, device="cuda")).to(torch.bfloat16)


def verify_every_time(c, ids, nq, q, k, v, where):
    first = c.call(ids, nq, q, k, v)
    c.verify(ids, nq, q, k, v, *first, where)
    for _ in range(4):
        again = c.call(ids, nq, q, k, v)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]), where


@pytest.mark.parametrize("half", [0, 1])
@pytest.mark.parametrize("tokens", [5, 12, 17, 20, 32, 40])
@pytest.mark.parametrize("bits, mix", [(4, (1.0, 0.0)), (2, (0.0, 1.0)), (4, (0.0, 1.0)), (8, (0.0, 1.0))])
def test_scores_that_rise_in_late_blocks(P, bits, mix, tokens, half):
    """As many items as there are CTAs, nearly: each has all blocks of its keys."""
    n, blocks, n_kv = 2000, 15, 8
    c = Case(P, [n] * 18, n_kv=n_kv, bits=bits, mix=(0.0, 0.0), seed=10 * tokens + half, chunk=4000)
    c.ref = R.Ref(n_kv, bits, 0)
    P.pask_cache_reset(c.cache.handle)
    us = []
    for s in range(18):
        k, u = rising_keys(n, n_kv, slots_of(s, n, half, blocks), c.g)
        c.append(s, n, mix, k=k)
        us.append(u)
    nq = [tokens] * 18
    _, k, v = c.inputs(nq)
    verify_every_time(c, list(range(18)), nq, queries(us, nq, c.g), k, v, f"bits {bits}, mix {mix}, {tokens} tokens, half {half}")


@pytest.mark.parametrize("tokens", [6, 14, 30])
@pytest.mark.parametrize("bits", [2, 4, 8])
def test_scores_that_rise_anywhere(P, bits, tokens):
    """More items than CTAs, cut anywhere; all kinds of pages in one sequence, the window's too; chunks of unequal length that end in the call's own rises."""
    n_kv, window = 8, 64
    hist = [1 + 211 * i % 2300 for i in range(40)]
    c = Case(P, hist, n_kv=n_kv, bits=bits, window=window, mix=(0.0, 0.0), seed=tokens, chunk=4000)
    c.ref = R.Ref(n_kv, bits, window)
    P.pask_cache_reset(c.cache.handle)
    us = []
    for s, n in enumerate(hist):
        k, u = rising_keys(n, n_kv, sorted((n * (2 * i + 1) // 14 + 5 * s) % n for i in range(7)), c.g)
        c.append(s, n, (0.35, 0.5), k=k)
        us.append(u)
    nq = [max(1, tokens + (i % 5 - 2) * tokens // 3) for i in range(40)]
    nq[3] += 2 * tokens                            # (the mean stays in its range: 40 sequences)
    _, k, v = c.inputs(nq)
    at = 0
    for n, u in zip(nq, us):                       # the last own key is above all of the history
        k[at + n - 1] = (u * (STEP * 9 / 128 ** 0.5)).to(torch.bfloat16)
        at += n
    verify_every_time(c, list(range(40)), nq, queries(us, nq, c.g), k, v, f"bits {bits}, {tokens} tokens")
