"""The 64-bit definitions of the layer's steps, pinned by what they have to satisfy, and what the library refuses of their arguments
before it touches a device."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import layer_steps_ref as ref
from paper_2609_07536_b200 import binding as B


def _inv_perm(rng, T, k, E, drop=0.0):
    e = rng.integers(0, E, size=(T, k)).reshape(-1)
    e[rng.random(T * k) < drop] = E
    order = np.argsort(e, kind="stable")
    inv = np.empty(T * k, dtype=np.int64)
    inv[order] = np.arange(T * k)
    inv[e == E] = -1
    return inv.reshape(T, k)


def test_sums_are_the_transposes_of_the_copies():
    # <permute(a), b> = <a, permute_grad(b)>, and the same for the weighted way back
    rng = np.random.default_rng(0)
    T, k, H = 7, 3, 8
    inv = _inv_perm(rng, T, k, 4, drop=0.3)
    a, b, w = rng.standard_normal((T, H)), rng.standard_normal((T * k, H)), rng.standard_normal((T, k))
    rows = ref.permute(a, inv, np.zeros((T * k, H)))
    assert np.isclose((rows * b).sum(), (a * ref.unpermute(b, inv)[0]).sum(), rtol=1e-12)
    d_rows, d_w, _ = ref.unpermute_grad(a, b, inv, w, np.zeros((T * k, H)))
    assert np.isclose((ref.unpermute(b, inv, w)[0] * a).sum(), (d_rows * b).sum(), rtol=1e-12)
    assert np.isclose((ref.unpermute(b, inv, w)[0] * a).sum(), (d_w * w).sum(), rtol=1e-12)


def test_activation_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(1)
    g, u, d = rng.standard_normal((3, 50)) * np.array([[4.0], [1.0], [1.0]])
    dg, du = ref.gated_act_grad(d, g, u)
    h = 1e-6          # central differences: h^2 f''' / 6 + 2^-53 |f| / h, both below 1e-9 at these sizes
    assert np.allclose(dg, d * (ref.gated_act(g + h, u) - ref.gated_act(g - h, u)) / (2 * h), atol=1e-8)
    assert np.allclose(du, d * (ref.gated_act(g, u + h) - ref.gated_act(g, u - h)) / (2 * h), atol=1e-8)


def test_checkpoint_codes_are_the_types_own_rounding():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((40, 96)) * np.exp2(rng.integers(-20, 20, size=(40, 1)))
    x = x.astype(np.float32)
    q, e = ref.checkpoint(x)
    amax = np.abs(x.reshape(40, 3, 32)).max(-1)
    assert (amax <= 448.0 * np.exp2(e)).all() and (amax > 448.0 * np.exp2(e - 1.0)).all()
    scaled = torch.from_numpy(x.reshape(40, 3, 32) * np.exp2(-e)[..., None].astype(np.float32))
    want = scaled.to(torch.float8_e4m3fn).float().numpy().reshape(40, 96)
    assert np.array_equal(q, want)
    err = np.abs(ref.checkpoint_values(q, e) - x)
    # half a step: 2^-4 of the value, or of the smallest normal code
    assert (err <= 2.0 ** -4 * np.maximum(np.abs(x), np.repeat(np.exp2(e - 6.0), 32, 1))).all()


@pytest.mark.parametrize("exact", [448.0, 449.0, 224.0, 225.0, 256.0, 255.0, 1.75, 1.7500001])
def test_checkpoint_exponent_at_its_borders(exact):
    x = np.zeros((1, 32), dtype=np.float32)
    x[0, 5] = exact
    q, e = ref.checkpoint(x)
    assert np.float32(exact) <= 448.0 * 2.0 ** float(e[0, 0]) and np.float32(exact) > 448.0 * 2.0 ** (float(e[0, 0]) - 1)


def test_four_bit_codes_are_the_nearest_values():
    v = np.linspace(-6.0, 6.0, 32)
    codes, e = ref.quantize(v.reshape(1, 32))
    assert e[0, 0] == 127                                                # 6 = 1.5 * 2^2: exponent 0
    back = ref.dequantize(codes, e)[0]
    grid = np.concatenate([-ref.E2M1, ref.E2M1])
    assert np.allclose(np.abs(back - v), np.abs(v[:, None] - grid).min(1))
    # ties go to the even code, beyond 6 it saturates, a block with no number is none
    t = np.zeros((3, 32))
    t[0, :8] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    t[1, :2] = [7.9, -7.9]
    t[2, 7] = np.inf
    codes, e = ref.quantize(t)
    assert ref.dequantize(codes, e)[0, :8].tolist() == [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]
    assert ref.dequantize(codes, e)[1, :2].tolist() == [6.0, -6.0]
    assert e[2, 0] == 255 and np.isnan(ref.dequantize(codes, e)[2]).all()


@pytest.mark.parametrize("offsets", [[0, 1], [0, 128, 256], [0, 127, 127, 128, 400], [0, 0, 0, 5, 133, 261, 262, 700]])
@pytest.mark.parametrize("K", [32, 128, 160])
def test_exponents_have_places_of_their_own_inside_the_buffer(offsets, K):
    at = ref.scale_places(offsets, K)
    assert len(np.unique(at)) == at.size
    assert at.min() >= 0 and at.max() < B.moe_mxfp4_scale_bytes(offsets[-1], K, len(offsets) - 1)


# ----------------------------------------------------------------------------- refusals, without a device

def _fake_handle():
    # refused before the handle is looked at: zeros stand in for one where there is no device to make it on
    return C.create_string_buffer(1 << 16)


OK_SHAPE = (4, 64, 32, 8, 2, 1, 1, 1)


@pytest.mark.parametrize("change, code", [
    (dict(h=None), B.MOE_ERR_NULL), (dict(tokens=None), B.MOE_ERR_NULL), (dict(rows=None), B.MOE_ERR_NULL), (dict(inv=None), B.MOE_ERR_NULL),
    (dict(status=None), B.MOE_ERR_NULL), (dict(tokens=8), B.MOE_ERR_ALIGN), (dict(rows=4096 + 2), B.MOE_ERR_ALIGN),
    (dict(ld_tokens=63), B.MOE_ERR_SHAPE), (dict(ld_rows=68), B.MOE_ERR_SHAPE), (dict(dtype=3), B.MOE_ERR_UNSUPPORTED), (dict(dtype=-1), B.MOE_ERR_UNSUPPORTED),
    (dict(shape=(4, 60, 32, 8, 2, 1, 1, 1)), B.MOE_ERR_SHAPE), (dict(shape=(-1, 64, 32, 8, 2, 1, 1, 1)), B.MOE_ERR_SHAPE),
    (dict(shape=(4, 64, 32, 8, 33, 1, 1, 1)), B.MOE_ERR_SHAPE), (dict(shape=(1 << 29, 64, 32, 8, 2, 1, 1, 1)), B.MOE_ERR_SHAPE),
    (dict(shape=(0, 64, 32, 8, 2, 1, 1, 1), tokens=None, rows=None), B.MOE_OK),
])
def test_permute_and_its_relatives_refuse(change, code):
    a = dict(h=_fake_handle(), tokens=4096, rows=8192, inv=4096, status=4096, ld_tokens=64, ld_rows=64, dtype=0, shape=OK_SHAPE, w=4096)
    a.update(change)
    L, s = B.lib(), C.byref(B.make_shape(*a["shape"]))
    assert L.moe_permute(a["h"], a["tokens"], a["ld_tokens"], a["inv"], s, a["dtype"], a["rows"], a["ld_rows"], a["status"], None) == code
    assert L.moe_permute_grad(a["h"], a["rows"], a["ld_rows"], a["inv"], s, a["dtype"], a["tokens"], a["ld_tokens"], a["status"], None) == code
    assert L.moe_unpermute(a["h"], a["rows"], a["ld_rows"], a["inv"], a["w"], s, a["dtype"], a["tokens"], a["ld_tokens"], a["status"], None) == code
    assert L.moe_unpermute_grad(a["h"], a["tokens"], a["ld_tokens"], a["rows"], a["ld_rows"], a["inv"], a["w"], s, a["dtype"], a["rows"], a["ld_rows"], a["w"],
                                a["status"], None) == code


def test_weights_and_their_gradient_are_required():
    L, s, h = B.lib(), C.byref(B.make_shape(*OK_SHAPE)), _fake_handle()
    assert L.moe_unpermute(h, 4096, 64, 4096, None, s, 0, 4096, 64, 4096, None) == B.MOE_ERR_NULL
    for w, d_rows, ld, d_w, code in ((None, 4096, 64, 4096, B.MOE_ERR_NULL), (4096, None, 64, 4096, B.MOE_ERR_NULL), (4096, 4096, 64, None, B.MOE_ERR_NULL),
                                     (4096, 4098, 64, 4096, B.MOE_ERR_ALIGN), (4096, 4096, 56, 4096, B.MOE_ERR_SHAPE)):
        assert L.moe_unpermute_grad(h, 4096, 64, 4096, 64, 4096, w, s, 0, d_rows, ld, d_w, 4096, None) == code


@pytest.mark.parametrize("change, code", [
    (dict(h=None), B.MOE_ERR_NULL), (dict(src=None), B.MOE_ERR_NULL), (dict(act=None), B.MOE_ERR_NULL), (dict(codes=None), B.MOE_ERR_NULL),
    (dict(scales=None), B.MOE_ERR_NULL), (dict(src=4104), B.MOE_ERR_ALIGN), (dict(act=4100), B.MOE_ERR_ALIGN), (dict(codes=4104), B.MOE_ERR_ALIGN),
    (dict(I=40), B.MOE_ERR_SHAPE), (dict(I=0), B.MOE_ERR_SHAPE), (dict(rows=-1), B.MOE_ERR_SHAPE), (dict(rows=1 << 30), B.MOE_ERR_SHAPE),
    (dict(ld=126), B.MOE_ERR_SHAPE), (dict(ld=132), B.MOE_ERR_SHAPE), (dict(ld_act=56), B.MOE_ERR_SHAPE), (dict(dtype=7), B.MOE_ERR_UNSUPPORTED),
    (dict(rows=0, src=None, act=None, codes=None, scales=None), B.MOE_OK),
])
def test_gated_activation_refuses(change, code):
    a = dict(h=_fake_handle(), src=4096, act=4096, codes=4096, scales=4096, rows=5, I=64, ld=128, ld_act=64, dtype=0)
    a.update(change)
    L = B.lib()
    assert L.moe_gated_act(a["h"], a["src"], a["ld"], a["rows"], a["I"], a["dtype"], a["act"], a["ld_act"], a["codes"], a["scales"], None) == code
    assert L.moe_gated_act_grad(a["h"], a["act"], a["ld_act"], a["codes"], a["scales"], a["rows"], a["I"], a["dtype"], a["src"], a["ld"], None, 0, None) == code


@pytest.mark.parametrize("change, code", [
    (dict(h=None), B.MOE_ERR_NULL), (dict(src=None), B.MOE_ERR_NULL), (dict(codes=None), B.MOE_ERR_NULL), (dict(scales=None), B.MOE_ERR_NULL),
    (dict(status=None), B.MOE_ERR_NULL), (dict(src=4104), B.MOE_ERR_ALIGN), (dict(codes=4104), B.MOE_ERR_ALIGN), (dict(scales=4100), B.MOE_ERR_ALIGN),
    (dict(K=48), B.MOE_ERR_SHAPE), (dict(K=0), B.MOE_ERR_SHAPE), (dict(rows=-6), B.MOE_ERR_SHAPE), (dict(groups=0), B.MOE_ERR_SHAPE),
    (dict(groups=4), B.MOE_ERR_SHAPE), (dict(ld=60), B.MOE_ERR_SHAPE), (dict(dtype=5), B.MOE_ERR_UNSUPPORTED),
    (dict(rows=0, src=None, codes=None, scales=None), B.MOE_OK),
])
def test_quantisation_refuses(change, code):
    a = dict(h=_fake_handle(), src=4096, codes=4096, scales=4096, status=4096, rows=6, K=64, ld=64, groups=3, dtype=0)
    a.update(change)
    L = B.lib()
    assert L.moe_mxfp4_quantize(a["h"], a["src"], a["ld"], a["dtype"], a["rows"], a["K"], a["groups"], None, None, 1, a["codes"], a["scales"], a["status"], None) == code
    assert L.moe_mxfp4_dequantize(a["h"], a["codes"], a["scales"], a["rows"], a["K"], a["groups"], None, a["dtype"], a["src"], a["ld"], a["status"], None) == code


def test_copies_go_with_the_rows_they_name():
    L, h = B.lib(), _fake_handle()
    for inv, copies in ((None, 2), (None, 0), (4096, 0), (4096, 33), (4096, 4)):
        assert L.moe_mxfp4_quantize(h, 4096, 64, 0, 6, 64, 3, 4096, inv, copies, 4096, 4096, 4096, None) == B.MOE_ERR_SHAPE


@pytest.mark.parametrize("change, code", [
    (dict(h=None), B.MOE_ERR_NULL), (dict(x=None), B.MOE_ERR_NULL), (dict(xs=None), B.MOE_ERR_NULL), (dict(w=None), B.MOE_ERR_NULL), (dict(ws=None), B.MOE_ERR_NULL),
    (dict(off=None), B.MOE_ERR_NULL), (dict(out=None), B.MOE_ERR_NULL), (dict(status=None), B.MOE_ERR_NULL),
    (dict(x=4104), B.MOE_ERR_ALIGN), (dict(ws=4104), B.MOE_ERR_ALIGN), (dict(out=4098), B.MOE_ERR_ALIGN),
    (dict(N=12), B.MOE_ERR_SHAPE), (dict(N=0), B.MOE_ERR_SHAPE), (dict(K=80), B.MOE_ERR_SHAPE), (dict(E=0), B.MOE_ERR_SHAPE), (dict(E=1025), B.MOE_ERR_SHAPE),
    (dict(rows=-1), B.MOE_ERR_SHAPE), (dict(ld=8), B.MOE_ERR_SHAPE), (dict(dtype=B.MOE_FP32), B.MOE_ERR_UNSUPPORTED), (dict(dtype=9), B.MOE_ERR_UNSUPPORTED),
    (dict(rows=0, x=None, out=None), B.MOE_OK),
])
def test_grouped_product_refuses(change, code):
    a = dict(h=_fake_handle(), x=4096, xs=4096, w=4096, ws=4096, off=4096, rows=6, E=3, N=16, K=64, dtype=0, out=4096, ld=16, status=4096)
    a.update(change)
    assert B.lib().moe_mxfp4_gemm(a["h"], a["x"], a["xs"], a["w"], a["ws"], a["off"], a["rows"], a["E"], a["N"], a["K"], a["dtype"], a["out"], a["ld"], a["status"],
                                  None) == code


def test_scale_bytes():
    assert B.moe_mxfp4_scale_bytes(1, 32, 1) == 512 and B.moe_mxfp4_scale_bytes(128, 128, 1) == 1024 and B.moe_mxfp4_scale_bytes(300, 160, 5) == 7 * 2 * 512
    assert B.moe_mxfp4_scale_bytes(0, 32, 4) == 4 * 512
    for rows, K, groups in ((-1, 32, 1), (5, 33, 1), (5, 0, 1), (5, 32, 0)):
        with pytest.raises(B.MoeError) as e:
            B.moe_mxfp4_scale_bytes(rows, K, groups)
        assert e.value.code == B.MOE_ERR_SHAPE
    assert B.lib().moe_mxfp4_scale_bytes(1, 32, 1, None) == B.MOE_ERR_NULL
