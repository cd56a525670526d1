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


# ----------------------------------------------------------------------------- quantisation and back

def places(bad, have, K):
    """{row: bytes of its exponents} of the rows that have a place."""
    at = {}
    for e, ok in enumerate(have):
        for r in range(bad[e], bad[e + 1]) if ok else ():
            i = r - bad[e]
            block = bad[e] // 128 + e + i // 128
            at[r] = [(block * -(-K // 128) + s // 4) * 512 + 16 * (i % 32) + 4 * (i % 128 // 32) + s % 4 for s in range(K // 32)]
    return at


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("good, bad, have", BAD)
def test_quantisation_skips_groups_without_a_place(good, bad, have, gather):
    rows, K, groups = good[-1], 96, len(good) - 1
    x = normal((rows // 2 if gather else rows, K), torch.bfloat16, 5)
    inv = torch.randperm(rows, generator=torch.Generator().manual_seed(2)).to(torch.int32).reshape(-1, 2)
    codes = torch.full((rows, K // 2), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.moe_mxfp4_scale_bytes(rows, K, groups),), 0x5A, dtype=torch.uint8, device="cuda")
    st = status()
    B.moe_mxfp4_quantize(handle(), x.cuda(), codes, scales, groups, st, offsets=ints(bad), inv_perm=inv.cuda() if gather else None)
    assert reported(st)
    xv = ref.permute(f64(x), inv.numpy(), np.zeros((rows, K))) if gather else f64(x)
    want_codes, want_e = ref.quantize(xv)
    at = places(bad, have, K)
    want, buf = np.full((rows, K // 2), 0x5A, np.uint8), scales.cpu().numpy()
    for r, where in at.items():
        want[r] = want_codes[r]
        assert np.array_equal(buf[where], want_e[r]), r
    assert np.array_equal(codes.cpu().numpy(), want)
    # a row's exponents are words of four bytes
    assert (buf != 0x5A).sum() <= 4 * len(at) and len({w for v in at.values() for w in v}) == len(at) * (K // 32)
    out, st = torch.full((rows, K), 7.0, device="cuda"), status()
    B.moe_mxfp4_dequantize(handle(), codes, scales, groups, out, st, offsets=ints(bad))
    assert reported(st)
    back = np.full((rows, K), 7.0)
    keep = sorted(at)
    back[keep] = ref.dequantize(want_codes, want_e)[keep]
    assert np.array_equal(f64(out), back)


def many_groups(groups):
    counts = np.random.default_rng(groups).integers(0, 4, size=groups)
    counts[groups // 2] = 300
    return [0] + np.cumsum(counts).tolist()


@pytest.mark.parametrize("groups", [1023, 1024, 1025, 1500])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_more_groups_than_are_held(groups, dtype):
    offsets, K = many_groups(groups), 160
    n = offsets[-1]
    x, off = normal((n, K), dtype, 1), ints(offsets)
    codes = torch.full((n + 2, K // 2), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.moe_mxfp4_scale_bytes(n + 2, K, groups),), 0x5A, dtype=torch.uint8, device="cuda")
    st = status()
    B.moe_mxfp4_quantize(handle(), torch.cat([x, x[:2]]).cuda(), codes, scales, groups, st, offsets=off)
    want_codes, want_e = ref.quantize(f64(x))
    at = places(offsets, [True] * groups, K)
    assert np.array_equal(codes.cpu().numpy()[:n], want_codes) and (codes.cpu().numpy()[n:] == 0x5A).all()
    assert np.array_equal(scales.cpu().numpy()[np.array([at[r] for r in range(n)])], want_e)
    out = torch.full((n + 2, K), 7.0, dtype=dtype, device="cuda")
    B.moe_mxfp4_dequantize(handle(), codes, scales, groups, out, st, offsets=off)
    want = ref.dequantize(want_codes, want_e)
    assert (np.abs(f64(out)[:n] - want) <= half_step(dtype, want)).all() and (f64(out)[n:] == 7.0).all()
    assert st.tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("at, value", [(3, LARGE), (700, SMALL), (700, 0), (-1, 10 ** 6), (-1, 5)])
def test_more_groups_than_are_held_with_one_without_a_place(at, value):
    # the rows of every group beside the bad offset are left alone; no row gets a place that is not its own
    groups, K = 1500, 64
    good = many_groups(groups)
    n, bad = good[-1], list(good)
    bad[at] = value
    x = normal((n, K), torch.bfloat16, 1)
    codes = torch.full((n, K // 2), 0x5A, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.moe_mxfp4_scale_bytes(n, K, groups),), 0x5A, dtype=torch.uint8, device="cuda")
    st = status()
    B.moe_mxfp4_quantize(handle(), x.cuda(), codes, scales, groups, st, offsets=ints(bad))
    assert reported(st)
    want_codes, want_e = ref.quantize(f64(x))
    got, buf = codes.cpu().numpy(), scales.cpu().numpy()
    at_bad = places(bad, intact(bad, n), K)
    written = ~(got == 0x5A).all(1)
    for r in np.flatnonzero(written):
        assert r in at_bad and np.array_equal(got[r], want_codes[r]) and np.array_equal(buf[at_bad[r]], want_e[r])
    beside = set(range(min(max(good[at - 1], 0), n), good[at + 1] if at != -1 else n))
    assert not beside & set(np.flatnonzero(written).tolist())
    out, st = torch.full((n, K), 7.0, device="cuda"), status()
    B.moe_mxfp4_dequantize(handle(), codes, scales, groups, out, st, offsets=ints(bad))
    assert reported(st)
    assert np.array_equal((f64(out) == 7.0).all(1), ~written)
