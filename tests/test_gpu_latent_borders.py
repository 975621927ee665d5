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
