"""The grouped 4-bit product on each family of its tiles: (64, 128) where experts have few rows, (192, 128), and (192, 256) by pairs of CTAs.
Every test says which family its sizes are for, so that a change of the rule that chooses it does not leave one untested.

Tolerances as in tests/test_gpu_layer_steps.py."""

import numpy as np
import pytest
import torch

from oracle import layer_steps_ref as ref
from paper_2609_07536_b200 import binding as B
from tests import test_gpu_layer_steps as steps
from tests.gpu_common import handle
from tests.test_gpu_layer_steps import WIDE_N, check_product, check_wide, f64, gen, ints, normal, pitched, quantized, status, wide_case

pytestmark = pytest.mark.gpu

FEW, ONE, PAIR = (64, 128), (192, 128), (192, 256)


def select(rows, E, N):
    return B.moe_mxfp4_select_tile(handle(), rows, E, N)


def test_which_tiles():
    assert select(16 * 66 + 65, 66, 2816) == FEW and select(17 * 66, 66, 2816) == ONE
    assert select(0, 1, 8) == FEW and select(16, 1, 8) == FEW and select(17, 1, 8) == ONE
    # pairs from 128 rows an expert on, where each of the pairs that fit the device has eleven tiles
    assert select(127 * 66, 66, 2816) == ONE and select(128 * 66, 66, 2816) == PAIR
    assert select(40 * 300, 40, 1536) == ONE and select(60 * 300, 60, 1536) == PAIR
    for args in ((-1, 4, 8), (4, 0, 8), (4, 1025, 8), (4, 4, 12), (4, 1024, 1 << 20)):
        with pytest.raises(B.MoeError) as e:
            select(*args)
        assert e.value.code == B.MOE_ERR_SHAPE


def test_the_sizes_of_the_other_tests_reach_every_family():
    assert {select(rows, len(offsets) - 1, N) for offsets, rows, N, K in steps.PRODUCTS} == {FEW, ONE}
    assert select(9 + 385, 3, 128) == ONE and select(9 + 1, 3, 128) == FEW
    for M in (1, 385):
        assert select(800 + M, 3, WIDE_N) == PAIR
    assert select(1100, 2, WIDE_N) == PAIR and select(1400, 4, WIDE_N) == PAIR and select(900, 3, WIDE_N) == PAIR
    assert select(800000, 4, 2816) == PAIR and select(127000, 1000, 16960) == ONE


def far(rows, K, seed):
    """Every row and block of 32 columns has another exponent, from far below to far above."""
    ex = torch.randint(-30, 30, (rows, K // 32, 1), generator=gen(seed)).float()
    return (normal((rows, K // 32, 32), torch.float32, seed + 1) * torch.exp2(ex)).reshape(rows, K)


# N mod 256: the second CTA of a pair has 8, 40, 72 or 120 of its 128 columns; K mod 256: a last stage of one to three MMAs, the last of them half empty or not
@pytest.mark.parametrize("over, K, dtype", [(136, 288, torch.bfloat16), (168, 416, torch.float16), (200, 192, torch.bfloat16), (248, 160, torch.float16),
                                            (136, 704, torch.bfloat16), (248, 1440, torch.bfloat16)])
def test_pairs_whose_second_cta_has_part_of_its_columns(over, K, dtype):
    N, E, offsets = 29952 - 256 + over, 2, [0, 333, 1100]
    assert N % 256 == over and select(1100, E, N) == PAIR
    g = torch.Generator(device="cuda").manual_seed(K)
    spread = lambda n: (torch.randn((n, K // 32, 32), device="cuda", generator=g) * torch.exp2(torch.randint(-30, 30, (n, K // 32, 1), device="cuda", generator=g).float())).reshape(n, K)  # noqa: E731
    xc, xs, wc, ws, xv, wv = wide_case(offsets, spread(1100), spread(E * N), E)
    out, st = pitched(torch.full((1103, N), 7.0, dtype=torch.float32).to(dtype), N + 8), status()
    # fp16 does not hold results of such exponents: their powers of two are moved down for it
    if dtype == torch.float16:
        ws = (ws.to(torch.int32) - 60).clamp(min=0).to(torch.uint8)
        wv = torch.zeros((E * N, K), device="cuda")
        B.moe_mxfp4_dequantize(handle(), wc.reshape(E * N, K // 2), ws, E, wv, st)
        wv = wv.double().reshape(E, N, K)
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out[:1100], st)
    assert st.tolist() == [0, 0, 0, 0]
    check_wide(out, xv, wv, offsets, K)
    assert torch.isfinite(out).all()
    assert torch.isnan(out.as_strided((1102, 8), (N + 8, 1), N)).all()      # between the rows
    assert (out[1100:] == 7.0).all()                                        # behind them


def few_offsets(M):
    """20 experts, one with 5 rows, one with M, one with 1."""
    return [0] * 3 + [5] + [5 + M] * 8 + [6 + M] * 9


@pytest.mark.parametrize("offsets, tile", [(few_offsets(65), FEW), (few_offsets(200), FEW), (few_offsets(1), FEW), ([0, 150, 300], ONE), ([0, 250, 600], ONE)])
@pytest.mark.parametrize("K", [512, 2720])
def test_exponents_far_apart(offsets, tile, K):
    N, E, rows = 264, len(offsets) - 1, offsets[-1]
    assert select(rows, E, N) == tile
    x, w = far(rows, K, 1), far(E * N, K, 5)
    xc, xs, _ = quantized(x.cuda(), E, ints(offsets))
    wc, ws, _ = quantized(w.cuda(), E)
    out, st = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc.reshape(E, N, K // 2), ws, ints(offsets), out, st)
    assert st.tolist() == [0, 0, 0, 0]
    check_product(out, ref.dequantize(*ref.quantize(f64(x))), ref.dequantize(*ref.quantize(f64(w))).reshape(E, N, K), offsets, K, torch.bfloat16)


@pytest.mark.parametrize("offsets, tile", [(few_offsets(70), FEW), (few_offsets(200), FEW), ([0] * 3 + [5] + [300] * 8 + [420] * 9, ONE)])
def test_no_number_stays_in_its_row_and_column(offsets, tile):
    N, K, E, rows = 136, 2720, 20, offsets[-1]
    assert select(rows, E, N) == tile
    x, w = normal((rows, K), torch.float32, 1), normal((E * N, K), torch.float32, 2)
    x[60, 40], w[3 * N + 5, 2719] = float("nan"), float("inf")      # the expert with most rows, the fourth: a row, a column
    xc, xs, _ = quantized(x.cuda(), E, ints(offsets))
    wc, ws, _ = quantized(w.cuda(), E)
    out, st = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc.reshape(E, N, K // 2), ws, ints(offsets), out, st)
    bad = np.isnan(f64(out))
    mine = offsets[4] - offsets[3]
    assert bad[60].all() and bad[offsets[3]:offsets[4], 5].all() and bad.sum() == N + mine - 1 and st.tolist() == [0, 0, 0, 0]


def test_all_families_on_streams_of_their_own():
    # against the same calls one after the other
    jobs = []
    for offsets, N, K, tile in (([0, 5, 9, 30], 264, 2720, FEW), ([0, 100, 101, 400], 1032, 320, ONE), ([0, 400, 401, 900], WIDE_N, 320, PAIR)):
        assert select(offsets[-1], 3, N) == tile
        g = torch.Generator(device="cuda").manual_seed(N)
        xc, xs, wc, ws, xv, wv = wide_case(offsets, torch.randn((offsets[-1], K), device="cuda", generator=g), torch.randn((3 * N, K), device="cuda", generator=g), 3)
        jobs.append((offsets, xc, xs, wc, ws, xv, wv, ints(offsets), [torch.zeros((offsets[-1], N), dtype=torch.bfloat16, device="cuda") for _ in range(2)], status(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for which in range(2):
        for _ in range(20 if which else 1):
            for _, xc, xs, wc, ws, _, _, off, out, st, stream in jobs:
                with torch.cuda.stream(stream if which else torch.cuda.current_stream()):
                    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, off, out[which], st)
        torch.cuda.synchronize()
    for offsets, _, _, _, _, xv, wv, _, out, st, _ in jobs:
        check_wide(out[0], xv, wv, offsets, xv.shape[1])
        assert torch.equal(*out) and st.tolist() == [0, 0, 0, 0]


# ----------------------------------------------------------------------------- waits that run out

# Sizes whose tiles take several times the 64 polls (90 us) after which a wait looks at its limit, three and more tiles for a CTA or pair: the results'
# warps give up in the first, the issuer and the loaders where those no longer hand accumulators and stages back.
LONG = [(16, 444 * 128, 1 << 17, FEW), (4100, 21 * 128, 1 << 18, ONE), (5400, 29 * 256, 1 << 18, PAIR)]
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


@pytest.mark.parametrize("rows, N, K, tile", LONG)
def test_a_wait_that_runs_out_is_reported_and_the_context_survives(rows, N, K, tile):
    assert select(rows, 1, N) == tile
    # row r of x is one value all along, column n of the weights another: every partial sum is 1, 3 or 9 times a power of two times up to 2^18, exact in fp32
    code = lambda n: (torch.arange(n, device="cuda") % 8 * 17).to(torch.uint8).reshape(-1, 1).expand(n, K // 2).contiguous()  # noqa: E731
    scales = lambda n: torch.full((B.moe_mxfp4_scale_bytes(n, K, 1),), 127, dtype=torch.uint8, device="cuda")  # noqa: E731
    xc, wc, xs, ws, off = code(rows), code(N).reshape(1, N, K // 2), scales(rows), scales(N), ints([0, rows])
    out, st = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda"), status()
    B.moe_set_wait_limit_ns(handle(), 1000)
    try:
        B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, off, out, st)
        torch.cuda.synchronize()
    finally:
        B.moe_set_wait_limit_ns(handle(), 2_000_000_000)
    assert B.moe_get_status(handle(), st, check=False).code == B.MOE_DEV_TIMEOUT
    v = torch.tensor(VALUES, device="cuda")
    want = v[torch.arange(rows, device="cuda") % 8].reshape(-1, 1) * v[torch.arange(N, device="cuda") % 8] * K
    # what was written before the limit is right, and not all of it was
    assert ((out == 7.0) | (out == want)).all() and (out == 7.0).any()
    for _ in range(2):
        st = status()
        B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, off, out, st)
        assert st.tolist() == [0, 0, 0, 0] and (out == want).all()
