"""The expert products' waits run out while operands and MMAs are on their way: the call reports it, and the same workspace and context then
give the results that they gave before.  (The combine's waits: tests/test_gpu_fused.py, the 4-bit product's: tests/test_gpu_mxfp4_tiles.py.)

A wait looks at its limit after 64 polls, 90 us: the sizes have tiles that take several times as long, and three or more for every CTA or
pair, so that the warps of the results give up in the first and the others where nothing is handed back to them."""

from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2609_07536_b200 import binding as B
from paper_2609_07536_b200 import workloads as wl
from tests import gpu_common as G

pytestmark = pytest.mark.gpu


def normal(*shape, seed):
    return torch.randn(shape, device="cuda", dtype=torch.bfloat16, generator=torch.Generator(device="cuda").manual_seed(seed))


def with_a_limit(call):
    B.moe_set_wait_limit_ns(G.handle(), 1000)
    try:
        return call()
    finally:
        B.moe_set_wait_limit_ns(G.handle(), 2_000_000_000)


@pytest.mark.parametrize("tile_m", [128, 256])
def test_gemm1_that_runs_out_of_time(tile_m):
    w = replace(wl.TINY, name="long", T=2816, E=1, k=1, H=1 << 17, I=21 * 128, EP=1, tile_m=tile_m, tile_n=256)
    ws, idx, S = G.build_routing(w, np.zeros((w.T, 1), np.int32))
    hidden, W1 = normal(w.T, w.H, seed=1), normal(1, 2, w.I, w.H, seed=2) * 2.0 ** -8
    hr = torch.empty(B.moe_gemm1_workspace_bytes(ws.shape), dtype=torch.uint8, device="cuda")

    def run():
        x = torch.full((w.R, w.I), 7.0, dtype=torch.bfloat16, device="cuda")
        B.moe_clear_status(G.handle(), ws.status)
        B.moe_gemm1_act(G.handle(), hidden, W1, ws.shape, tile_m, ws.routing, S, hr, x, ws.status)
        torch.cuda.synchronize()
        return x, B.moe_get_status(G.handle(), ws.status, check=False).code

    want, code = run()
    assert code == 0
    x, code = with_a_limit(run)
    assert code == B.MOE_DEV_TIMEOUT and ((x == want) | (x == 7.0)).all() and not torch.equal(x, want)
    for _ in range(2):
        x, code = run()
        assert code == 0 and torch.equal(x, want)


@pytest.mark.parametrize("tile", [(128, 256), (256, 256)])
def test_gemm2_that_runs_out_of_time(tile):
    w = replace(wl.TINY, name="long", T=2816, E=1, k=1, H=21 * 256, I=1 << 17, EP=1, tile_m=tile[0], tile_n=tile[1])
    idx, wt = np.zeros((w.T, 1), np.int32), np.ones((w.T, 1), np.float32)
    x, W2 = normal(w.R, w.I, seed=1), normal(1, w.H, w.I, seed=2) * 2.0 ** -8
    want, plan, ws, S, st = G.run_layer(w, idx, wt, x, W2, force_C=2)
    assert st.code == 0
    *_, st = with_a_limit(lambda: G.run_layer(w, idx, wt, x, W2, force_C=2, mode=B.MOE_MODE_GEMM_ONLY, ws=ws, check_status=False))
    assert st.code == B.MOE_DEV_TIMEOUT and st.where in (10, 11, 20, 21, 30, 31, 32)
    for _ in range(2):
        again, *_, st = G.run_layer(w, idx, wt, x, W2, force_C=2, ws=ws)
        assert st.code == 0 and np.array_equal(again[0], want[0])
