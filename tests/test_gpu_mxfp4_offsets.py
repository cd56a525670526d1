"""Offsets of the experts' rows that go back or past the rows: they are reported, and an expert whose rows one of them begins or ends,
or that begins inside another one's rows, has none; the others' results are what they are with offsets in order."""

import numpy as np
import pytest
import torch

from oracle import layer_steps_ref as ref
from paper_2609_07536_b200 import binding as B
from tests.gpu_common import handle
from tests.test_gpu_layer_steps import WIDE_N, check_product, f64, half_step, ints, normal, product_case, status, wide_case, TINY

pytestmark = pytest.mark.gpu


def intact(offsets, rows):
    """Which experts have rows."""
    top, have = 0, []
    for begin, end in zip(offsets, offsets[1:]):
        fine = 0 <= begin <= end <= rows
        have.append(fine and begin >= top)
        top = max(top, end) if fine else top
    return have


def reported(st):
    torch.cuda.synchronize()
    return B.moe_get_status(handle(), st, check=False).code == B.MOE_DEV_OOB


LARGE, SMALL = 2 ** 31 - 1, -2 ** 31
BAD = [
    ([0, 4, 8, 12], [0, 1000, 8, 12], [False, False, True]),
    ([0, 4, 8, 12], [0, 4, 8, 13], [True, True, False]),
    ([0, 4, 8, 12], [-1, 4, 8, 12], [False, True, True]),
    ([0, 4, 8, 12], [0, 4, 2, 12], [True, False, False]),           # the third would begin inside the first
    ([0, 4, 8, 12], [0, SMALL, 8, 12], [False, False, True]),
    ([0, 4, 8, 12], [0, 4, LARGE, 12], [True, False, False]),
    ([0, 4, 8, 12], [SMALL, LARGE, 8, 12], [False, False, True]),
    ([0, 8, 8, 8, 12], [0, 8, 4, 8, 12], [True, False, False, True]),
    ([0, 300, 300, 700, 900], [0, 300, 5000, 700, 900], [True, False, False, True]),
    ([0, 300, 300, 700, 900], [0, 300, 300, 701, 700], [True, True, True, False]),
]


def check_experts(out, xv, wv, good, bad, have):
    """Rows of the experts that have some against their definition, the rest as they were."""
    mine = np.zeros(out.shape[0], dtype=bool)
    got, eps = f64(out), torch.finfo(out.dtype).eps / 2
    for e, ok in enumerate(have):
        if ok and bad[e:e + 2] == good[e:e + 2]:
            rows = slice(good[e], good[e + 1])
            x = xv[rows]
            want, mag = x @ wv[e].T, np.abs(x) @ np.abs(wv[e]).T
            assert (np.abs(got[rows] - want) <= eps * np.abs(want) + TINY[out.dtype] / 2 + x.shape[1] * 2.0 ** -23 * mag).all(), e
        if ok:
            mine[bad[e]:bad[e + 1]] = True
    assert (got[~mine] == 7.0).all()


@pytest.mark.parametrize("good, bad, have", BAD)
def test_product_skips_experts_without_a_place(good, bad, have):
    assert intact(bad, good[-1]) == have
    N, K = 136, 96
    xc, xs, wc, ws, xv, wv = product_case(good, good[-1], N, K, 3)
    for dtype in (torch.bfloat16, torch.float16):
        out, st = torch.full((good[-1], N), 7.0, dtype=dtype, device="cuda"), status()
        B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(bad), out, st)
        assert reported(st)
        check_experts(out, xv, wv, good, bad, have)


@pytest.mark.parametrize("E", [20, 415, 416, 1000])
@pytest.mark.parametrize("at, value", [(0, -5), (7, LARGE), (13, 0), (-2, 10 ** 6), (-1, 3)])
def test_product_of_many_experts_skips_those_without_a_place(E, at, value):
    N, K = 16, 64
    counts = np.random.default_rng(E).integers(1, 4, size=E)
    good = [0] + np.cumsum(counts).tolist()
    bad = list(good)
    bad[at] = value
    xc, xs, wc, ws, xv, wv = product_case(good, good[-1], N, K, 3)
    out, st = torch.full((good[-1], N), 7.0, dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(bad), out, st)
    assert reported(st)
    have = intact(bad, good[-1])
    assert E - 2 <= sum(have) <= E - 1
    check_experts(out, xv, wv, good, bad, have)


def test_wide_tiles_skip_experts_without_a_place():
    good, bad, K = [0, 300, 500, 1100, 1400], [0, 300, 5000, 1100, 1400], 96
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = torch.randn((1400, K), device="cuda", generator=g), 0.05 * torch.randn((4 * WIDE_N, K), device="cuda", generator=g)
    xc, xs, wc, ws, xv, wv = wide_case(good, x, w, 4)
    out, st = torch.full((1400, WIDE_N), 7.0, dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(bad), out, st)
    assert reported(st)
    check_experts(out, xv.cpu().numpy(), wv.cpu().numpy(), good, bad, [True, False, False, True])
