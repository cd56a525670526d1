"""The layer's steps at the limits of what they take: gates whose exponential leaves the range of fp32.

Tolerances as in tests/test_gpu_layer_steps.py."""

import numpy as np
import pytest
import torch

from oracle import layer_steps_ref as ref
from paper_2609_07536_b200 import binding as B
from tests.gpu_common import handle
from tests.test_gpu_layer_steps import act_slack, f64, half_step

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------- gated activation

def subnormal_slack(dtype, g, y, factor):
    # beside the slack of the other tests, without its room for small results: exp(-|g|) below 2^-126 is a subnormal number, to a step of
    # 2^-149 at most, which the gate (with 1 in the derivative) and `factor` multiply
    return half_step(dtype, y) + 2.0 ** -20 * (1.0 + np.abs(g)) * np.abs(y) + 2.0 ** -148 * (1.0 + np.abs(g)) * np.abs(factor)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gates_far_from_zero_with_large_factors(dtype):
    # silu(-88) is -5e-37, a normal number of both types, and the other factor makes it an ordinary one
    gates = torch.arange(-108.0, 108.5, 0.5)[:432].reshape(27, 16).to(dtype)
    for up in (1.0, 2.0 ** 90, -(2.0 ** 120)):
        x = torch.cat([gates, torch.full_like(gates, up)], 1)
        act = torch.empty(gates.shape, dtype=dtype, device="cuda")
        B.moe_gated_act(handle(), x.cuda(), act)
        g, u = f64(gates), np.full(gates.shape, up)
        want = ref.gated_act(g, u)
        assert (np.abs(f64(act) - want) <= subnormal_slack(dtype, g, want, u)).all(), up


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_at_gates_far_from_zero(dtype):
    # gates that the 8-bit copy holds exactly
    gates = torch.tensor([-112.0, -104.0, -96.0, -88.0, -80.0, -72.0, -64.0, -8.0, 8.0, 64.0, 72.0, 80.0, 88.0, 96.0, 104.0, 112.0]).reshape(1, 16).repeat(4, 2)
    ups, d = torch.full((4, 32), 2.0 ** 40), torch.tensor([1.0, 2.0 ** 50, -(2.0 ** 60), 2.0 ** -30]).reshape(4, 1).expand(4, 32)
    x, act = torch.cat([gates, ups], 1).to(dtype).cuda(), torch.empty((4, 32), dtype=dtype, device="cuda")
    codes, scales = torch.empty((4, 64), dtype=torch.uint8, device="cuda"), torch.empty((4, 2), dtype=torch.uint8, device="cuda")
    B.moe_gated_act(handle(), x, act, codes, scales)
    grad, again = torch.empty((4, 64), dtype=dtype, device="cuda"), torch.empty((4, 32), dtype=dtype, device="cuda")
    B.moe_gated_act_grad(handle(), d.to(dtype).contiguous().cuda(), codes, scales, grad, again)
    g, u, dv = f64(gates), f64(ups), f64(d)
    want_g, want_u = ref.gated_act_grad(dv, g, u)
    terms = np.abs(dv * u * ref.sigmoid(g)) * (1.0 + np.abs(g))
    slack_g = half_step(dtype, want_g) + 2.0 ** -20 * (1.0 + np.abs(g)) * terms + 2.0 ** -148 * (1.0 + np.abs(g)) * np.abs(dv * u)
    assert (np.abs(f64(grad)[:, :32] - want_g) <= slack_g).all()
    assert (np.abs(f64(grad)[:, 32:] - want_u) <= subnormal_slack(dtype, g, want_u, dv)).all()
    want = ref.gated_act(g, u)
    assert (np.abs(f64(again) - want) <= subnormal_slack(dtype, g, want, u)).all()


def test_infinite_gates():
    gates = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0]).repeat(4).reshape(1, 16)
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        act = torch.empty((1, 16), dtype=dtype, device="cuda")
        B.moe_gated_act(handle(), torch.cat([gates, torch.full_like(gates, 2.0)], 1).to(dtype).cuda(), act)
        got = f64(act).reshape(4, 4)
        # x / (1 + exp(-x)) in IEEE arithmetic: a quotient of infinities is no number
        assert (got[:, 0] == np.inf).all() and np.isnan(got[:, 1:3]).all()
        assert (np.abs(got[:, 3] - ref.gated_act(3.0, 2.0)) <= act_slack(dtype, 3.0, ref.gated_act(3.0, 2.0))).all()
