"""The steps of the layer as operators of their own against their 64-bit definitions (oracle/layer_steps_ref.py).

Tolerances.  A result is rounded once to its type: half a step, `eps / 2` relative to the value (and half the smallest subnormal).
fp32 sums of n terms, in any order, are within n 2^-24 of the sum of the terms' magnitudes; every product in them adds 2^-24 of itself."""

import numpy as np
import pytest
import torch

from oracle import layer_steps_ref as ref
from oracle import routing_ref as rr
from paper_2609_07536_b200 import binding as B
from tests.gpu_common import handle

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}


def half_step(t, ref_value):
    return torch.finfo(t).eps / 2 * np.abs(ref_value) + TINY[t] / 2


def gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def normal(shape, dtype, seed, std=1.0):
    return (torch.randn(shape, generator=gen(seed), dtype=torch.float32) * std).to(dtype)


def pitched(t, ld):
    """The same matrix on the GPU with `ld` elements between rows; what lies between them is no number."""
    buf = torch.full((t.shape[0], ld), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t.cuda()
    return buf[:, :t.shape[1]]


def f64(t):
    return t.detach().cpu().double().numpy()


def status():
    return torch.zeros(4, dtype=torch.int32, device="cuda")


def shape_of(T, k, H):
    return B.make_shape(T, H, 32, 8, k, 1, 1, 1)


def inv_perm_of(T, k, E, seed, drop=0.0):
    rng = np.random.default_rng(seed)
    e = rng.integers(0, E, size=T * k)
    if drop:
        e[rng.random(T * k) < drop] = E
        e[:k] = E                                       # the first token has no row at all
    order = np.argsort(e, kind="stable")
    inv = np.empty(T * k, dtype=np.int32)
    inv[order] = np.arange(T * k, dtype=np.int32)
    inv[e == E] = -1
    return inv.reshape(T, k)


# ----------------------------------------------------------------------------- tokens to rows and back

ROWS = [(1, 1, 8, 1, 0), (1, 8, 2048, 8, 0), (3, 2, 264, 4, 8), (5, 32, 72, 40, 0), (130, 8, 1536, 40, 16), (257, 6, 520, 64, 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("drop", [0.0, 0.3])
@pytest.mark.parametrize("T, k, H, E, pad", ROWS)
def test_rows_and_back(T, k, H, E, pad, drop, dtype):
    h, s, st = handle(), shape_of(T, k, H), status()
    inv = inv_perm_of(T, k, E, T + k, drop)
    tokens, rows, d_out = normal((T, H), dtype, 1), normal((T * k, H), dtype, 2), normal((T, H), dtype, 3)
    w = torch.rand((T, k), generator=gen(4))
    inv_d, w_d, ld = torch.from_numpy(inv).cuda(), w.cuda(), H + pad
    new = lambda n: pitched(torch.full((n, H), 7.0, dtype=dtype), ld)  # noqa: E731
    x, d_tokens, out, d_rows, d_w = new(T * k), new(T), new(T), new(T * k), torch.full((T, k), 9.0, device="cuda")
    tokens_d, rows_d, d_out_d = pitched(tokens, ld), pitched(rows, ld), pitched(d_out, ld)
    B.moe_permute(h, tokens_d, inv_d, s, x, st)
    B.moe_permute_grad(h, rows_d, inv_d, s, d_tokens, st)
    B.moe_unpermute(h, rows_d, inv_d, w_d, s, out, st)
    B.moe_unpermute_grad(h, d_out_d, rows_d, inv_d, w_d, s, d_rows, d_w, st)
    assert st.tolist() == [0, 0, 0, 0]
    sevens = np.full((T * k, H), 7.0)
    assert np.array_equal(f64(x), ref.permute(f64(tokens), inv, sevens))
    want, mag = ref.unpermute(f64(rows), inv)
    assert (np.abs(f64(d_tokens) - want) <= half_step(dtype, want) + k * 2.0 ** -24 * mag).all()
    want, mag = ref.unpermute(f64(rows), inv, f64(w))
    assert (np.abs(f64(out) - want) <= half_step(dtype, want) + (k + 1) * 2.0 ** -24 * mag).all()
    want_rows, want_w, mag = ref.unpermute_grad(f64(d_out), f64(rows), inv, f64(w), sevens)
    assert (np.abs(f64(d_rows) - want_rows) <= half_step(dtype, want_rows) + 2.0 ** -24 * np.abs(want_rows)).all()
    assert (np.abs(f64(d_w) - want_w) <= (H + 1) * 2.0 ** -24 * mag).all()
    if drop:
        assert f64(out)[0].tolist() == [0.0] * H and f64(d_w)[0].tolist() == [0.0] * k
    # what lies between the rows is as it was
    if pad:
        for t in (x, d_tokens, out, d_rows):
            assert torch.isnan(t.as_strided((t.shape[0] - 1, pad), (ld, 1), t.storage_offset() + H)).all()
    # in place, and the same bits again
    rows_in = rows_d.clone(memory_format=torch.preserve_format) if pad == 0 else pitched(rows, ld)
    again = torch.empty_like(d_w)
    B.moe_unpermute_grad(h, d_out_d, rows_in, inv_d, w_d, s, rows_in, again, st)
    kept = torch.from_numpy(inv[inv >= 0].astype(np.int64)).cuda()
    assert torch.equal(rows_in[kept], d_rows[kept]) and torch.equal(again, d_w)


def test_no_number_stays_in_its_token():
    T, k, H = 6, 3, 64
    h, s, st = handle(), shape_of(T, k, H), status()
    inv = inv_perm_of(T, k, 4, 0, 0.2)
    rows = normal((T * k, H), torch.bfloat16, 5)
    free = sorted(set(range(T * k)) - set(inv[inv >= 0].tolist()))
    rows[free] = float("nan")                           # rows that no assignment names are not read
    hurt = 3
    rows[inv[hurt][inv[hurt] >= 0][0], 5] = float("inf")
    out, w = torch.empty((T, H), dtype=torch.bfloat16, device="cuda"), torch.rand((T, k), generator=gen(6)) + 0.1
    B.moe_unpermute(h, rows.cuda(), torch.from_numpy(inv).cuda(), w.cuda(), s, out, st)
    bad = ~np.isfinite(f64(out))
    assert bad[hurt, 5] and bad.sum() == 1


def test_indices_out_of_range_are_reported_and_skipped():
    T, k, H = 4, 2, 64
    h, s = handle(), shape_of(T, k, H)
    inv = inv_perm_of(T, k, 4, 1)
    bad = inv.copy()
    bad[1, 0], bad[2, 1] = T * k, -2
    good = bad.copy()
    good[1, 0] = good[2, 1] = -1
    tokens, rows = normal((T, H), torch.float32, 1), normal((T * k, H), torch.float32, 2)
    w = torch.rand((T, k), generator=gen(4)).cuda()
    for call in ("permute", "permute_grad", "unpermute", "unpermute_grad"):
        got = []
        for i in (bad, good):
            st, inv_d = status(), torch.from_numpy(i).cuda()
            x, o, dw = torch.zeros((T * k, H), device="cuda"), torch.zeros((T, H), device="cuda"), torch.zeros((T, k), device="cuda")
            if call == "permute":
                B.moe_permute(h, tokens.cuda(), inv_d, s, x, st)
            elif call == "permute_grad":
                B.moe_permute_grad(h, rows.cuda(), inv_d, s, o, st)
            elif call == "unpermute":
                B.moe_unpermute(h, rows.cuda(), inv_d, w, s, o, st)
            else:
                B.moe_unpermute_grad(h, tokens.cuda(), rows.cuda(), inv_d, w, s, x, dw, st)
            torch.cuda.synchronize()
            assert B.moe_get_status(h, st, check=False).code == (B.MOE_DEV_OOB if i is bad else 0)
            got.append((x, o, dw))
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_offsets_past_32_bits():
    # 1.2 million rows of 2048 columns: 2.4e9 elements, 4.9 GB
    T, k, H = 150001, 8, 2048
    h, s, st = handle(), shape_of(T, k, H), status()
    inv = torch.randperm(T * k, device="cuda", dtype=torch.int32).reshape(T, k)
    tokens = torch.randn((T, H), device="cuda", dtype=torch.bfloat16)
    rows = torch.empty((T * k, H), device="cuda", dtype=torch.bfloat16)
    B.moe_permute(h, tokens, inv, s, rows, st)
    for t in (0, 1, T // 2, T - 2, T - 1):
        assert torch.equal(rows[inv[t].long()], tokens[t].expand(k, H))
    out, w = torch.empty_like(tokens), torch.full((T, k), 0.125, device="cuda")
    B.moe_unpermute(h, rows, inv, w, s, out, st)
    assert torch.equal(out, tokens)                     # eight equal rows of an eighth each: exact
    d_w = torch.empty((T, k), device="cuda")
    B.moe_unpermute_grad(h, tokens, rows, inv, w, s, rows, d_w, st)
    assert torch.equal(rows[inv[T - 1].long()], (tokens[T - 1] * 0.125).expand(k, H))
    want = tokens[-64:].double().square().sum(1, keepdim=True).expand(64, k)
    assert ((d_w[-64:].double() - want).abs() <= (H + 1) * 2.0 ** -24 * want).all()
    assert st.tolist() == [0, 0, 0, 0]


# ----------------------------------------------------------------------------- gated activation

def act_slack(dtype, g, y):
    # exp to 2^-22 (1 + |g|) of itself (the fast one scales its argument by 1 / ln 2 in fp32, the result has 2^-22), a sum, a quotient to 2^-22 and
    # two products: 2^-20 (1 + |g|) of the result covers them; the fast quotient takes what is below 2^-118 for zero
    return half_step(dtype, y) + 2.0 ** -20 * (1.0 + np.abs(g)) * np.abs(y) + 2.0 ** -110


ACT = [(1, 16, 0), (1, 1408, 0), (7, 48, 8), (33, 512, 16), (129, 144, 0), (700, 1408, 0)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R, I, pad", ACT)
def test_gated_activation_and_its_checkpoint(R, I, pad, dtype):
    h = handle()
    x = normal((R, 2 * I), dtype, R + I, std=2.0)
    if R > 6:
        x[1] = 0.0                                      # blocks of zeros
        x[2] *= 2.0 ** -14                              # (subnormal in fp16)
        x[3] *= 2.0 ** 12
        x[4, :32] = 448.0                               # exactly at the border
        x[5, :16] = -449.0 if dtype == torch.float32 else -450.0
    nb = (I + 31) // 32
    x_d, act = pitched(x, 2 * I + pad), pitched(torch.zeros((R, I), dtype=dtype), I + pad)
    codes, scales = torch.full((R, 2 * I), 0x55, dtype=torch.uint8, device="cuda"), torch.full((R, 2 * nb), 0x55, dtype=torch.uint8, device="cuda")
    B.moe_gated_act(h, x_d, act, codes, scales)
    g, u = f64(x)[:, :I], f64(x)[:, I:]
    want = ref.gated_act(g, u)
    fits = np.abs(want) < torch.finfo(dtype).max
    assert (np.abs(f64(act) - want) <= act_slack(dtype, g, want))[fits].all()
    assert np.isinf(f64(act)[~fits]).all()
    (gq, ge), (uq, ue) = ref.checkpoint(g), ref.checkpoint(u)
    assert np.array_equal(f64(codes.view(torch.float8_e4m3fn).float()), np.concatenate([gq, uq], 1))
    assert np.array_equal(scales.cpu().numpy(), np.concatenate([ge, ue], 1) + 127)
    # without a checkpoint: the same activation
    plain = pitched(torch.zeros((R, I), dtype=dtype), I + pad)
    B.moe_gated_act(h, x_d, plain)
    assert torch.equal(plain, act)
    # backward pass, from the copy alone
    d = normal((R, I), dtype, 3)
    gv, uv = ref.checkpoint_values(gq, ge), ref.checkpoint_values(uq, ue)
    for want_act in (True, False):
        d_gu, again = pitched(torch.zeros((R, 2 * I), dtype=dtype), 2 * I + pad), pitched(torch.full((R, I), 7.0, dtype=dtype), I + pad)
        B.moe_gated_act_grad(h, pitched(d, I + pad), codes, scales, d_gu, again if want_act else None)
        dg, du = ref.gated_act_grad(f64(d), gv, uv)
        got = f64(d_gu)
        # the gate's gradient is a product with 1 + g (1 - s), which may cancel: its error goes by the terms' magnitude
        terms = np.abs(f64(d) * uv * ref.sigmoid(gv)) * (1.0 + np.abs(gv))
        with np.errstate(invalid="ignore"):
            ok_g = np.abs(got[:, :I] - dg) <= half_step(dtype, dg) + 2.0 ** -20 * (1.0 + np.abs(gv)) * terms + 2.0 ** -110
            ok_u = np.abs(got[:, I:] - du) <= act_slack(dtype, gv, du)
            ok_a = np.abs(f64(again) - ref.gated_act(gv, uv)) <= act_slack(dtype, gv, ref.gated_act(gv, uv))
        top = torch.finfo(dtype).max
        assert (ok_g | (np.abs(dg) >= top)).all() and (ok_u | (np.abs(du) >= top)).all()
        if want_act:
            assert (ok_a | (np.abs(ref.gated_act(gv, uv)) >= top)).all()
        else:
            assert (f64(again) == 7.0).all()


def test_gradient_is_the_difference_quotient_of_the_activation():
    # fp32 end to end on values that the 8-bit copy holds exactly, so that it is the activation's own derivative
    h, R, I = handle(), 4, 32
    grid = torch.tensor([0.5, -0.5, 1.0, -1.25, 2.0, -3.0, 0.875, 4.0]).repeat(R, 4)
    x = torch.cat([grid, grid.roll(3, 1)], 1).cuda()
    d = normal((R, I), torch.float32, 8).cuda()
    act, codes, scales = torch.empty((R, I), device="cuda"), torch.empty((R, 2 * I), dtype=torch.uint8, device="cuda"), torch.empty((R, 2), dtype=torch.uint8, device="cuda")
    grad = torch.empty((R, 2 * I), device="cuda")
    B.moe_gated_act(h, x, act, codes, scales)
    B.moe_gated_act_grad(h, d, codes, scales, grad)
    step, g, u = 1e-6, f64(x)[:, :I], f64(x)[:, I:]
    want_g = f64(d) * (ref.gated_act(g + step, u) - ref.gated_act(g - step, u)) / (2 * step)
    want_u = f64(d) * (ref.gated_act(g, u + step) - ref.gated_act(g, u - step)) / (2 * step)
    # fp32 arithmetic, 2^-22 of terms |d| |u| s (1 + |g|) < 5 * 4 * 5 (the exponential's argument is at most 4); the quotients are good to 1e-8
    assert np.abs(f64(grad) - np.concatenate([want_g, want_u], 1)).max() <= 100 * 2.0 ** -22 + 1e-7


@pytest.mark.parametrize("dtype", DTYPES)
def test_checkpoint_of_what_is_no_number(dtype):
    h, R, I = handle(), 3, 64
    x = normal((R, 2 * I), dtype, 9)
    x[0, 3], x[1, I + 40], x[2, 63], x[2, 62] = float("nan"), float("inf"), float("-inf"), float("nan")
    act, codes, scales = torch.empty((R, I), dtype=dtype, device="cuda"), torch.empty((R, 2 * I), dtype=torch.uint8, device="cuda"), torch.empty((R, 4), dtype=torch.uint8, device="cuda")
    B.moe_gated_act(h, x.cuda(), act, codes, scales)
    (gq, ge), (uq, ue) = ref.checkpoint(f64(x)[:, :I]), ref.checkpoint(f64(x)[:, I:])
    want = np.concatenate([gq, uq], 1)
    got = f64(codes.view(torch.float8_e4m3fn).float())
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).sum() == 4
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
    assert np.array_equal(scales.cpu().numpy(), np.concatenate([ge, ue], 1) + 127)
    grad = torch.empty((R, 2 * I), dtype=dtype, device="cuda")
    B.moe_gated_act_grad(h, torch.ones((R, I), dtype=dtype, device="cuda"), codes, scales, grad)
    # the gate's gradient takes both values, the up projection's the gate alone
    hurt = np.concatenate([np.isnan(want[:, :I]) | np.isnan(want[:, I:]), np.isnan(want[:, :I])], 1)
    assert np.array_equal(np.isnan(f64(grad)), hurt)


def test_gated_activation_past_32_bits():
    R, I = 800003, 1408                                 # 2.25e9 elements of gate and up
    h = handle()
    x = torch.empty((R, 2 * I), dtype=torch.bfloat16, device="cuda").normal_()
    act = torch.empty((R, I), dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.empty((R, 2 * I), dtype=torch.uint8, device="cuda"), torch.empty((R, 88), dtype=torch.uint8, device="cuda")
    B.moe_gated_act(h, x, act, codes, scales)
    d_gu = torch.empty_like(x)
    B.moe_gated_act_grad(h, act, codes, scales, d_gu)
    tail = slice(R - 3, R)
    small = [torch.empty((3, n), dtype=t, device="cuda") for n, t in ((I, torch.bfloat16), (2 * I, torch.uint8), (88, torch.uint8), (2 * I, torch.bfloat16))]
    B.moe_gated_act(h, x[tail], *small[:3])
    B.moe_gated_act_grad(h, small[0], small[1], small[2], small[3])
    for big, few in ((act, small[0]), (codes, small[1]), (scales, small[2]), (d_gu, small[3])):
        assert torch.equal(big[tail], few)


# ----------------------------------------------------------------------------- microscaled 4 bits

def quantized(x, groups, offsets=None, inv=None, rows=None, fill=0xFF):
    """(codes, scales, status) of the library; both buffers full of `fill` beforehand."""
    rows = x.shape[0] if rows is None else rows
    K = x.shape[1]
    codes = torch.full((rows, K // 2), fill, dtype=torch.uint8, device="cuda")
    scales = torch.full((B.moe_mxfp4_scale_bytes(rows, K, groups),), fill, dtype=torch.uint8, device="cuda")
    st = status()
    B.moe_mxfp4_quantize(handle(), x, codes, scales, groups, st, offsets=offsets, inv_perm=inv)
    return codes, scales, st


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def matrix_with_everything(rows, K, dtype, seed):
    x = normal((rows, K), torch.float32, seed) * torch.exp2(torch.randint(-10, 10, (rows, 1), generator=gen(seed + 1)).float())
    x[0, :] = 0.0
    if rows > 4:
        x[1, :16] = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -4.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0])
        x[1, 16:32] = 0.0
        x[2, :32] = 7.99
        x[3, :32] = 2.0 ** -20
    x = x.to(dtype)
    if rows > 4:
        x[4, :32] = torch.finfo(dtype).max
        x[3, 0] = torch.finfo(dtype).tiny / 2           # subnormal
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", [32, 96, 128, 1408])
@pytest.mark.parametrize("offsets, rows, even", [([0, 1], 1, True), ([0, 5, 10, 15], 15, True), ([0, 0, 3, 131, 131, 260], 270, False), ([0, 128, 192], 192, False)])
def test_quantisation_and_back(offsets, rows, even, K, dtype):
    groups, n = len(offsets) - 1, offsets[-1]
    x = matrix_with_everything(rows, K, dtype, K + rows)
    x_d = pitched(x, K + 8)
    off = None if even else ints(offsets)
    codes, scales, st = quantized(x_d, groups, off)
    want_codes, want_e = ref.quantize(f64(x)[:n])
    assert np.array_equal(codes.cpu().numpy()[:n], want_codes)
    at = ref.scale_places(offsets, K)
    buf = scales.cpu().numpy()
    assert np.array_equal(buf[at], want_e)
    # exponents of columns past K are zero, nothing else is written, and no row behind the last group
    row_bytes = {int(a) // 4 * 4 for a in at[:, 0]}
    for base in list(row_bytes)[:50]:
        last = base + (-(-K // 128) - 1) * 512
        used = (K // 32 - 1) % 4 + 1
        assert (buf[last + used:last + 4] == 0).all()
    assert (buf == 0xFF).sum() >= buf.size - len(row_bytes) * 4 * -(-K // 128)
    assert (codes.cpu().numpy()[n:] == 0xFF).all()
    for out_type in DTYPES:
        out = pitched(torch.full((rows, K), 7.0, dtype=out_type), K + 8)
        B.moe_mxfp4_dequantize(handle(), codes, scales, groups, out, st, offsets=off)
        want = ref.dequantize(want_codes, want_e)
        got = f64(out)
        fits = np.abs(want) <= torch.finfo(out_type).max
        assert (np.abs(got[:n] - want) <= half_step(out_type, want))[fits].all()
        assert (got[n:] == 7.0).all()
    assert st.tolist() == [0, 0, 0, 0]


def test_blocks_with_no_number():
    x = normal((3, 96), torch.float32, 3)
    x[0, 33], x[1, 0], x[2, 95] = float("nan"), float("inf"), float("-inf")
    codes, scales, st = quantized(x.cuda(), 1)
    want_codes, want_e = ref.quantize(f64(x))
    assert np.array_equal(codes.cpu().numpy(), want_codes) and np.array_equal(scales.cpu().numpy()[ref.scale_places([0, 3], 96)], want_e)
    out = torch.empty((3, 96), device="cuda")
    B.moe_mxfp4_dequantize(handle(), codes, scales, 1, out, st)
    assert np.array_equal(np.isnan(f64(out)), np.isnan(ref.dequantize(want_codes, want_e))) and np.isnan(f64(out)).sum() == 96


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T, k, E, K, drop", [(1, 1, 1, 32, 0.0), (1, 8, 64, 2048, 0.0), (37, 6, 64, 160, 0.25), (300, 8, 5, 256, 0.0)])
def test_quantisation_into_routed_order(T, k, E, K, drop, dtype):
    inv = inv_perm_of(T, k, E, 5, drop)
    n = int((inv >= 0).sum())
    counts = np.sort(np.random.default_rng(0).integers(0, n + 1, size=E - 1))
    offsets = [0] + counts.tolist() + [n]
    x = normal((T, K), dtype, 2)
    codes, scales, st = quantized(x.cuda(), E, ints(offsets), torch.from_numpy(inv).cuda(), rows=T * k)
    rows = ref.permute(f64(x), inv, np.zeros((T * k, K)))[:n]
    want_codes, want_e = ref.quantize(rows) if n else (np.zeros((0, K // 2), np.uint8), np.zeros((0, K // 32), np.uint8))
    assert np.array_equal(codes.cpu().numpy()[:n], want_codes) and (codes.cpu().numpy()[n:] == 0xFF).all()
    if n:
        assert np.array_equal(scales.cpu().numpy()[ref.scale_places(offsets, K)], want_e)
    assert st.tolist() == [0, 0, 0, 0]


def test_quantisation_reports_rows_that_do_not_exist():
    x, inv = normal((2, 64), torch.float32, 1).cuda(), ints([[0, 4], [1, -3]])
    codes, scales, st = quantized(x, 1, ints([0, 4]), inv, rows=4)
    torch.cuda.synchronize()
    assert B.moe_get_status(handle(), st, check=False).code == B.MOE_DEV_OOB
    want, _ = ref.quantize(f64(x))
    assert np.array_equal(codes.cpu().numpy()[:2], want) and (codes.cpu().numpy()[2:] == 0xFF).all()
    # groups that begin behind their rows
    codes, scales, st = quantized(x, 2, ints([1, 2, 2]))
    torch.cuda.synchronize()
    assert B.moe_get_status(handle(), st, check=False).code == B.MOE_DEV_OOB


# ----------------------------------------------------------------------------- grouped product

def product_case(offsets, rows, N, K, seed, std=1.0):
    E = len(offsets) - 1
    x, w = normal((rows, K), torch.bfloat16, seed, std), normal((E * N, K), torch.bfloat16, seed + 1, 0.05)
    xc, xs, _ = quantized(x.cuda(), E, ints(offsets))
    wc, ws, _ = quantized(w.cuda(), E)
    xv = ref.dequantize(*ref.quantize(f64(x)))[:offsets[-1]]
    wv = ref.dequantize(*ref.quantize(f64(w))).reshape(E, N, K)
    return xc, xs, wc.reshape(E, N, K // 2), ws, xv, wv


def check_product(out, xv, wv, offsets, K, dtype):
    want, mag = ref.grouped_product(xv, wv, offsets)
    n = offsets[-1]
    # products are exact; K additions to fp32, each to a step (not half of one) of the sum of magnitudes
    err = np.abs(f64(out)[:n] - want)
    assert (err <= half_step(dtype, want) + K * 2.0 ** -23 * mag).all(), float((err - half_step(dtype, want)).max())


PRODUCTS = [
    ([0, 1], 1, 8, 32), ([0, 1], 1, 128, 256), ([0, 3, 3, 4], 4, 24, 64), ([0, 16, 33], 40, 136, 96), ([0, 64, 64, 129], 129, 256, 160),
    ([0, 191, 383, 576], 576, 128, 256), ([0, 193, 193, 600], 640, 264, 288), ([0, 193, 193, 700], 800, 264, 288), ([0, 400, 1003], 1003, 1408, 512), ([0, 0, 0, 7], 7, 2048, 1408),
    ([0] + list(range(1, 67)), 66, 384, 1280),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("offsets, rows, N, K", PRODUCTS)
def test_grouped_product(offsets, rows, N, K, dtype):
    xc, xs, wc, ws, xv, wv = product_case(offsets, rows, N, K, rows + N)
    out, st = pitched(torch.full((rows, N), 7.0, dtype=dtype), N + 8), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
    assert st.tolist() == [0, 0, 0, 0]
    check_product(out, xv, wv, offsets, K, dtype)
    assert (f64(out)[offsets[-1]:] == 7.0).all()
    if rows > 1:
        assert torch.isnan(out.as_strided((rows - 1, 8), (N + 8, 1), out.storage_offset() + N)).all()
    again = torch.empty((rows, N), dtype=dtype, device="cuda")
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), again, st)
    assert torch.equal(again[:offsets[-1]], out[:offsets[-1]])


@pytest.mark.parametrize("M", [1, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 160, 192, 256, 320, 321, 385])
def test_product_at_row_counts_around_the_steps(M):
    offsets, N, K = [0, 5, 5 + M, 9 + M], 128, 384
    xc, xs, wc, ws, xv, wv = product_case(offsets, 9 + M, N, K, M)
    out, st = torch.empty((9 + M, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
    check_product(out, xv, wv, offsets, K, torch.bfloat16)


@pytest.mark.parametrize("M", [1, 15, 16, 17, 31, 33, 48, 63, 64, 65, 127, 128, 129, 192, 200])
def test_few_rows_an_expert_with_one_that_has_more(M):
    # tiles of 64 rows in more stages: the longest sequences of stages (K = 2720: eleven), more than one tile for an expert
    E, N, K = 20, 264, 2720
    offsets = [0] * 3 + [5] + [5 + M] * 8 + [6 + M] * 9
    assert len(offsets) == E + 1 and offsets[-1] // E <= 16
    xc, xs, wc, ws, xv, wv = product_case(offsets, offsets[-1], N, K, M)
    out, st = torch.empty((offsets[-1], N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
    assert st.tolist() == [0, 0, 0, 0]
    check_product(out, xv, wv, offsets, K, torch.bfloat16)


# Tiles of 256 columns by two CTAs are for many rows an expert and many tiles: tests of them have many columns, and take their reference
# on the GPU, in 64 bits from the values that the quantisation (tested above) left.
WIDE_N = 29960                                          # 117 tiles of 256 columns and one of 8; with seven tiles of rows, eleven for each of 74 pairs


def wide_case(offsets, x, w, E):
    rows, K = x.shape
    xc, xs, st1 = quantized(x.cuda(), E, ints(offsets))
    wc, ws, st2 = quantized(w.cuda(), E)
    xv, wv = torch.zeros((rows, K), device="cuda"), torch.empty((w.shape[0], K), device="cuda")
    B.moe_mxfp4_dequantize(handle(), xc, xs, E, xv, st1, offsets=ints(offsets))
    B.moe_mxfp4_dequantize(handle(), wc, ws, E, wv, st2)
    return xc, xs, wc.reshape(E, -1, K // 2), ws, xv.double(), wv.double().reshape(E, -1, K)


def check_wide(out, xv, wv, offsets, K):
    eps = torch.finfo(out.dtype).eps / 2
    for e in range(len(offsets) - 1):
        x, got = xv[offsets[e]:offsets[e + 1]], out[offsets[e]:offsets[e + 1]].double()
        want, mag = x @ wv[e].t(), x.abs() @ wv[e].abs().t()
        assert ((got - want).abs() <= eps * want.abs() + TINY[out.dtype] / 2 + K * 2.0 ** -23 * mag).all(), e


@pytest.mark.parametrize("M", [1, 15, 17, 31, 32, 33, 63, 64, 65, 96, 97, 128, 129, 191, 192, 193, 256, 257, 320, 321, 385])
@pytest.mark.parametrize("K, dtype", [(384, torch.bfloat16), (1504, torch.float16)])
def test_wide_tiles_at_row_counts_around_the_steps(M, K, dtype):
    offsets, E = [0, 300, 300 + M, 800 + M], 3
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn((800 + M, K), device="cuda", generator=g), 0.05 * torch.randn((E * WIDE_N, K), device="cuda", generator=g)
    xc, xs, wc, ws, xv, wv = wide_case(offsets, x, w, E)
    out, st = pitched(torch.full((803 + M, WIDE_N), 7.0, dtype=dtype), WIDE_N + 8)[:800 + M], status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
    assert st.tolist() == [0, 0, 0, 0]
    check_wide(out, xv, wv, offsets, K)
    assert torch.isnan(out.as_strided((799 + M, 8), (WIDE_N + 8, 1), WIDE_N)).all()      # between the rows
    assert (out.as_strided((3, WIDE_N), (WIDE_N + 8, 1), (800 + M) * (WIDE_N + 8)) == 7.0).all()      # behind them


def test_wide_tiles_with_exponents_far_apart_and_no_numbers():
    offsets, K, E = [0, 250, 1100], 512, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    far = lambda n: torch.randn((n, K // 32, 32), device="cuda", generator=g) * torch.exp2(torch.randint(-30, 30, (n, K // 32, 1), device="cuda", generator=g).float())  # noqa: E731
    x, w = far(1100).reshape(1100, K), far(E * WIDE_N).reshape(E * WIDE_N, K)
    xc, xs, wc, ws, xv, wv = wide_case(offsets, x, w, E)
    out, st = torch.empty((1100, WIDE_N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
    check_wide(out, xv, wv, offsets, K)
    x[300, 40], w[5, 200] = float("nan"), float("inf")  # expert 1; expert 0, column 5
    xc, xs, wc, ws, _, _ = wide_case(offsets, x, w, E)
    hurt = torch.empty_like(out)
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), hurt, st)
    bad = torch.isnan(hurt)
    assert bad[300].all() and bad[:250, 5].all() and int(bad.sum()) == WIDE_N + 250
    assert torch.equal(hurt[~bad], out[~bad]) and st.tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("offsets, rows", [([0, 150, 300], 300), ([0, 250, 600], 600)])
def test_product_with_exponents_far_apart(offsets, rows):
    # exponents from far below to far above, every row and block another one: none is mixed up
    N, K, E = 136, 512, 2
    ex = torch.randint(-30, 30, (rows, K // 32, 1), generator=gen(1)).float()
    x = (normal((rows, K // 32, 32), torch.float32, 2) * torch.exp2(ex)).reshape(rows, K)
    ew = torch.randint(-30, 30, (E * N, K // 32, 1), generator=gen(3)).float()
    w = (normal((E * N, K // 32, 32), torch.float32, 4) * torch.exp2(ew)).reshape(E * N, K)
    xc, xs, _ = quantized(x.cuda(), E, ints(offsets))
    wc, ws, _ = quantized(w.cuda(), E)
    out, st = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc.reshape(E, N, K // 2), ws, ints(offsets), out, st)
    check_product(out, ref.dequantize(*ref.quantize(f64(x))), ref.dequantize(*ref.quantize(f64(w))).reshape(E, N, K), offsets, K, torch.bfloat16)


@pytest.mark.parametrize("far", [0, 500])
def test_no_number_in_a_product_stays_in_its_row_and_column(far):
    rows = 200 + far                                    # (few rows an expert, many)
    offsets, N, K = [0, 70, rows], 136, 256
    x, w = normal((rows, K), torch.float32, 1), normal((2 * N, K), torch.float32, 2)
    x[90, 40] = float("nan")                            # expert 1
    w[5, 200] = float("inf")                            # expert 0, column 5
    xc, xs, _ = quantized(x.cuda(), 2, ints(offsets))
    wc, ws, _ = quantized(w.cuda(), 2)
    out, st = torch.empty((rows, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc.reshape(2, N, K // 2), ws, ints(offsets), out, st)
    bad = np.isnan(f64(out))
    assert bad[90].all() and bad[:70, 5].all() and bad.sum() == N + 70


def test_more_experts_than_threads():
    E, N, K = 1000, 16, 64
    counts = np.random.default_rng(0).integers(0, 4, size=E)
    offsets = [0] + np.cumsum(counts).tolist()
    xc, xs, wc, ws, xv, wv = product_case(offsets, offsets[-1] + 3, N, K, 3)
    out, st = torch.full((offsets[-1] + 3, N), 7.0, dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
    assert st.tolist() == [0, 0, 0, 0]
    check_product(out, xv, wv, offsets, K, torch.bfloat16)
    assert (f64(out)[offsets[-1]:] == 7.0).all()


def test_product_reports_offsets_that_go_back():
    N, K = 16, 64
    xc, xs, wc, ws, xv, wv = product_case([0, 4, 8, 12], 12, N, K, 3)
    for offsets in ([0, 4, 2, 12], [0, 4, 8, 13], [-1, 4, 8, 12]):
        out, st = torch.zeros((12, N), dtype=torch.bfloat16, device="cuda"), status()
        B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, ints(offsets), out, st)
        torch.cuda.synchronize()
        assert B.moe_get_status(handle(), st, check=False).code == B.MOE_DEV_OOB


def test_product_past_32_bits():
    R, N, K, E = 800000, 2816, 32, 4                    # 2.25e9 elements out
    offsets = ints([0, 100, 400001, 799990, R])
    codes = torch.randint(0, 256, (R, K // 2), dtype=torch.uint8, device="cuda")
    xs = torch.full((B.moe_mxfp4_scale_bytes(R, K, E),), 127, dtype=torch.uint8, device="cuda")
    wc = torch.randint(0, 256, (E, N, K // 2), dtype=torch.uint8, device="cuda")
    ws = torch.full((B.moe_mxfp4_scale_bytes(E * N, K, E),), 127, dtype=torch.uint8, device="cuda")
    out, st = torch.empty((R, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), codes, xs, wc, ws, offsets, out, st)
    for e, at in ((0, 3), (1, 399990), (2, 799980), (3, R - 5)):
        x = ref.dequantize(codes[at:at + 5].cpu().numpy(), np.full((5, 1), 127, np.uint8))
        w = ref.dequantize(wc[e].cpu().numpy(), np.full((N, 1), 127, np.uint8))
        want = x @ w.T                                  # multiples of 1/4 below 2^11: exact in fp32
        assert (np.abs(f64(out[at:at + 5]) - want) <= half_step(torch.bfloat16, want)).all()
    assert st.tolist() == [0, 0, 0, 0]


def test_product_of_many_experts_past_32_bits():
    R, N, K, E = 127000, 16960, 32, 1000                # 2.15e9 elements out, 127 rows an expert: tiles of one CTA
    offsets = ints([127 * e for e in range(E + 1)])
    codes = torch.randint(0, 256, (R, K // 2), dtype=torch.uint8, device="cuda")
    xs = torch.full((B.moe_mxfp4_scale_bytes(R, K, E),), 127, dtype=torch.uint8, device="cuda")
    wc = torch.randint(0, 256, (E, N, K // 2), dtype=torch.uint8, device="cuda")
    ws = torch.full((B.moe_mxfp4_scale_bytes(E * N, K, E),), 127, dtype=torch.uint8, device="cuda")
    out, st = torch.empty((R, N), dtype=torch.bfloat16, device="cuda"), status()
    B.moe_mxfp4_gemm(handle(), codes, xs, wc, ws, offsets, out, st)
    for e in (0, 500, 999):
        at = 127 * e + 122
        x = ref.dequantize(codes[at:at + 5].cpu().numpy(), np.full((5, 1), 127, np.uint8))
        want = x @ ref.dequantize(wc[e].cpu().numpy(), np.full((N, 1), 127, np.uint8)).T     # multiples of 1/4 below 2^11: exact in fp32
        assert (np.abs(f64(out[at:at + 5]) - want) <= half_step(torch.bfloat16, want)).all()
    assert st.tolist() == [0, 0, 0, 0]


# ----------------------------------------------------------------------------- together

def routed(T, k, E, seed):
    """The library's own routing build of random choices: (routing workspace, inv_perm, offsets, choices)."""
    idx = np.stack([np.random.default_rng(seed + t).permutation(E)[:k] for t in range(T)]).astype(np.int32)
    s = B.make_shape(T, 64, 32, E, k, 1, 1, 1)
    ws = torch.empty(B.moe_workspace_bytes(s, 128, 64)[0], dtype=torch.uint8, device="cuda")
    r, st = B.moe_routing_view(ws, s, 128), status()
    B.moe_build_routing(handle(), torch.from_numpy(idx).cuda(), s, 128, r, None, st)
    view = lambda p, n: ws[p - ws.data_ptr():p - ws.data_ptr() + 4 * n].view(torch.int32)  # noqa: E731
    return ws, view(r.inv_perm, T * k).reshape(T, k), view(r.offsets, E + 1), idx


@pytest.mark.parametrize("T, k, E, H, I", [(1, 2, 8, 64, 32), (50, 4, 16, 256, 160)])
def test_a_layer_in_four_bits(T, k, E, H, I):
    # sort and quantise -> gate and up projection -> activation -> quantise -> down projection -> back, each step against
    # its definition on what the step before left
    h, st, R = handle(), status(), T * k
    ws_keep, inv, offsets, idx = routed(T, k, E, 7)
    off = offsets.cpu().tolist()
    assert np.array_equal(inv.cpu().numpy(), rr.build_routing(idx, E, 128)["inv_perm"].reshape(T, k))
    hidden = normal((T, H), torch.bfloat16, 1).cuda()
    W1, W2 = normal((E * 2 * I, H), torch.bfloat16, 2, 0.1), normal((E * H, I), torch.bfloat16, 3, 0.1)
    w1c, w1s, _ = quantized(W1.cuda(), E)
    w2c, w2s, _ = quantized(W2.cuda(), E)
    xc, xs, st1 = quantized(hidden, E, offsets, inv, rows=R)
    gate_up, act = (torch.empty((R, n), dtype=torch.bfloat16, device="cuda") for n in (2 * I, I))
    B.moe_mxfp4_gemm(h, xc, xs, w1c.reshape(E, 2 * I, H // 2), w1s, offsets, gate_up, st)
    B.moe_gated_act(h, gate_up, act)
    ac, as_, st2 = quantized(act, E, offsets)
    y, out = torch.empty((R, H), dtype=torch.bfloat16, device="cuda"), torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
    B.moe_mxfp4_gemm(h, ac, as_, w2c.reshape(E, H, I // 2), w2s, offsets, y, st)
    w = torch.softmax(torch.rand((T, k), generator=gen(9)), 1)
    B.moe_unpermute(h, y, inv, w.cuda(), shape_of(T, k, H), out, st)
    assert (st + st1 + st2).tolist() == [0, 0, 0, 0]
    inv_n = inv.cpu().numpy()
    x_rows = ref.permute(f64(hidden), inv_n, np.zeros((R, H)))
    q = lambda v: ref.dequantize(*ref.quantize(v))  # noqa: E731
    check_product(gate_up, q(x_rows), q(f64(W1)).reshape(E, 2 * I, H), off, H, torch.bfloat16)
    g, u = f64(gate_up)[:, :I], f64(gate_up)[:, I:]
    assert (np.abs(f64(act) - ref.gated_act(g, u)) <= act_slack(torch.bfloat16, g, ref.gated_act(g, u))).all()
    check_product(y, q(f64(act)), q(f64(W2)).reshape(E, H, I), off, I, torch.bfloat16)
    want, mag = ref.unpermute(f64(y), inv_n, f64(w))
    assert (np.abs(f64(out) - want) <= half_step(torch.bfloat16, want) + (k + 1) * 2.0 ** -24 * mag).all()


def training_step(T, k, E, H, I, inv, offsets, hidden, W1, W2, w, d_out, st, buf):
    """Forward and backward pass of a layer: the library's steps around plain products.  Returns (out, d_hidden, d_w)."""
    h, s = handle(), shape_of(T, k, H)
    B.moe_permute(h, hidden, inv, s, buf["x"], st)
    torch.bmm(buf["x"].view(E, -1, H), W1.transpose(1, 2), out=buf["gu"].view(E, -1, 2 * I))
    B.moe_gated_act(h, buf["gu"], buf["act"], buf["codes"], buf["scales"])
    torch.bmm(buf["act"].view(E, -1, I), W2.transpose(1, 2), out=buf["y"].view(E, -1, H))
    B.moe_unpermute(h, buf["y"], inv, w, s, buf["out"], st)
    B.moe_unpermute_grad(h, d_out, buf["y"], inv, w, s, buf["dy"], buf["dw"], st)
    torch.bmm(buf["dy"].view(E, -1, H), W2, out=buf["dact"].view(E, -1, I))
    B.moe_gated_act_grad(h, buf["dact"], buf["codes"], buf["scales"], buf["dgu"], buf["act2"])
    torch.bmm(buf["dgu"].view(E, -1, 2 * I), W1, out=buf["dx"].view(E, -1, H))
    B.moe_permute_grad(h, buf["dx"], inv, s, buf["dh"], st)


def training_buffers(T, k, H, I):
    R, new = T * k, lambda *s, t=torch.float32: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    return dict(x=new(R, H), gu=new(R, 2 * I), act=new(R, I), codes=new(R, 2 * I, t=torch.uint8), scales=new(R, 2 * ((I + 31) // 32), t=torch.uint8),
                y=new(R, H), out=new(T, H), dy=new(R, H), dw=new(T, k), dact=new(R, I), dgu=new(R, 2 * I), act2=new(R, I), dx=new(R, H), dh=new(T, H))


def balanced(T, k, E, seed):
    """Choices that give every expert equally many rows, so that the products between the steps are batched ones."""
    flat = torch.arange(T * k) % E
    inv = torch.empty(T * k, dtype=torch.int32)
    order = torch.sort(flat, stable=True).indices
    inv[order] = torch.arange(T * k, dtype=torch.int32)
    return inv.reshape(T, k).cuda()


def test_a_training_step_has_the_gradients_of_its_formula():
    T, k, E, H, I = 32, 2, 4, 64, 48
    inv, st = balanced(T, k, E, 0), status()
    hidden, d_out, w = (normal(s, torch.float32, i) for i, s in ((1, (T, H)), (2, (T, H)), (3, (T, k))))
    W1, W2 = normal((E, 2 * I, H), torch.float32, 4, 0.2), normal((E, H, I), torch.float32, 5, 0.2)
    buf = training_buffers(T, k, H, I)
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        training_step(T, k, E, H, I, inv, None, hidden.cuda(), W1.cuda(), W2.cuda(), w.cuda(), d_out.cuda(), st, buf)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = before
    # autograd in 64 bits of the same layer; its activation's derivative is taken at the values that the 8-bit copy holds
    hv, wv = hidden.double().requires_grad_(), w.double().requires_grad_()
    flat = inv.cpu().long().reshape(-1)
    perm = torch.empty_like(flat)
    perm[flat] = torch.arange(T * k)
    x = hv[perm // k].reshape(E, -1, H)
    gu = (x @ W1.double().transpose(1, 2)).reshape(T * k, 2 * I)
    kept = np.concatenate([ref.checkpoint_values(*ref.checkpoint(f64(buf["gu"])[:, a:a + I])) for a in (0, I)], 1)

    class Act(torch.autograd.Function):
        @staticmethod
        def forward(ctx, v):
            return v[:, :I] * torch.sigmoid(v[:, :I]) * v[:, I:]

        @staticmethod
        def backward(ctx, d):
            return torch.from_numpy(np.concatenate(ref.gated_act_grad(d.numpy(), kept[:, :I], kept[:, I:]), 1))

    y = (Act.apply(gu).reshape(E, -1, I) @ W2.double().transpose(1, 2)).reshape(T * k, H)
    out = (y[flat].reshape(T, k, H) * wv.unsqueeze(-1)).sum(1)
    out.backward(d_out.double())
    # fp32 throughout: chains of at most H + 2 I + I + k = 210 additions, each to 2^-24, on magnitudes within 64 of the results' rms
    for got, want in ((buf["out"], out), (buf["dh"], hv.grad), (buf["dw"], wv.grad)):
        want = f64(want)
        assert np.abs(f64(got) - want).max() <= 210 * 2.0 ** -24 * 64 * np.sqrt(np.mean(want ** 2))
    # and against the derivative at the values before they were rounded to 8 bits: 2^-4 relative a value, so that the gradient is off by
    # no more than a few times that of its norm
    hv2 = hidden.double().requires_grad_()
    gu = (hv2[perm // k].reshape(E, -1, H) @ W1.double().transpose(1, 2)).reshape(T * k, 2 * I)
    a = gu[:, :I] * torch.sigmoid(gu[:, :I]) * gu[:, I:]
    y = (a.reshape(E, -1, I) @ W2.double().transpose(1, 2)).reshape(T * k, H)
    (y[flat].reshape(T, k, H) * w.double().unsqueeze(-1)).sum(1).backward(d_out.double())
    exact = f64(hv2.grad)
    assert np.linalg.norm(f64(buf["dh"]) - exact) <= 3 * 2.0 ** -4 * np.linalg.norm(exact)
    assert st.tolist() == [0, 0, 0, 0]


def chain(T, k, I, inv, tokens, w, d_out, st, buf):
    """All six steps of the training path, one behind the other: rows [gate | up] go straight into the activation."""
    h, wide, narrow = handle(), shape_of(T, k, 2 * I), shape_of(T, k, I)
    B.moe_permute(h, tokens, inv, wide, buf["x"], st)
    B.moe_gated_act(h, buf["x"], buf["act"], buf["codes"], buf["scales"])
    B.moe_unpermute(h, buf["act"], inv, w, narrow, buf["out"], st)
    B.moe_unpermute_grad(h, d_out, buf["act"], inv, w, narrow, buf["d_act"], buf["dw"], st)
    B.moe_gated_act_grad(h, buf["d_act"], buf["codes"], buf["scales"], buf["dx"], buf["act2"])
    B.moe_permute_grad(h, buf["dx"], inv, wide, buf["d_tokens"], st)


def chain_buffers(T, k, I):
    R, new = T * k, lambda *s, t=torch.bfloat16: torch.full(s, 7, dtype=t, device="cuda")  # noqa: E731
    return dict(x=new(R, 2 * I), act=new(R, I), codes=new(R, 2 * I, t=torch.uint8), scales=new(R, 2 * ((I + 31) // 32), t=torch.uint8), out=new(T, I),
                d_act=new(R, I), dw=new(T, k, t=torch.float32), dx=new(R, 2 * I), act2=new(R, I), d_tokens=new(T, 2 * I))


def test_steps_in_graphs_on_streams_of_their_own():
    # two graphs of all steps, captured on other streams, replayed at once on new inputs, against eager calls on the default stream
    T, k, I = 64, 4, 144
    inv, jobs = balanced(T, k, 8, 0), []
    for n in range(2):
        tokens, d_out, w = torch.zeros((T, 2 * I), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, I), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, k), device="cuda")
        st, buf, stream, graph = status(), chain_buffers(T, k, I), torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            chain(T, k, I, inv, tokens, w, d_out, st, buf)
        jobs.append((tokens, d_out, w, st, buf, stream, graph))
    for rnd in range(2):
        for n, (tokens, d_out, w, *_) in enumerate(jobs):
            for i, t in enumerate((tokens, d_out, w)):
                t.copy_(normal(tuple(t.shape), t.dtype, 100 * rnd + 10 * n + i))
        torch.cuda.synchronize()
        for *_, stream, graph in jobs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for tokens, d_out, w, st, buf, stream, graph in jobs:
            want = chain_buffers(T, k, I)
            chain(T, k, I, inv, tokens, w, d_out, st, want)
            for name in want:
                assert torch.equal(want[name], buf[name]), name
            assert st.tolist() == [0, 0, 0, 0]


def test_four_bit_steps_in_a_graph():
    offsets, N, K = [0, 100, 100, 333], 136, 256
    E = 3
    x, w = torch.zeros((333, K), dtype=torch.bfloat16, device="cuda"), normal((E * N, K), torch.bfloat16, 2, 0.1)
    wc, ws, st = quantized(w.cuda(), E)
    off = ints(offsets)
    xc, xs = torch.empty((333, K // 2), dtype=torch.uint8, device="cuda"), torch.empty(B.moe_mxfp4_scale_bytes(333, K, E), dtype=torch.uint8, device="cuda")
    out = torch.empty((333, N), dtype=torch.bfloat16, device="cuda")

    def step():
        B.moe_mxfp4_quantize(handle(), x, xc, xs, E, st, offsets=off)
        B.moe_mxfp4_gemm(handle(), xc, xs, wc.reshape(E, N, K // 2), ws, off, out, st)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        x.copy_(normal((333, K), torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        check_product(out, ref.dequantize(*ref.quantize(f64(x))), ref.dequantize(*ref.quantize(f64(w))).reshape(E, N, K), offsets, K, torch.bfloat16)


# ----------------------------------------------------------------------------- refusals of the binding

def test_tensors_that_do_not_fit_together_are_refused():
    h, s, st = handle(), shape_of(4, 2, 64), status()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    tokens, rows, inv = torch.zeros((4, 64), **bf), torch.zeros((8, 64), **bf), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    w = torch.zeros((4, 2), device="cuda")

    def refused(code, call, *args, **more):
        with pytest.raises(B.MoeError) as e:
            call(h, *args, **more)
        assert e.value.code == code

    refused(B.MOE_ERR_SHAPE, B.moe_permute, tokens[:3], inv, s, rows, st)
    refused(B.MOE_ERR_SHAPE, B.moe_permute, tokens, inv, s, rows[:, :56], st)
    refused(B.MOE_ERR_SHAPE, B.moe_permute, torch.zeros((64, 4), **bf).t(), inv, s, rows, st)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_permute, tokens, inv, s, rows.float(), st)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_permute, tokens.double(), inv, s, rows.double(), st)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_permute, tokens, inv.long(), s, rows, st)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_permute, tokens.cpu(), inv, s, rows, st)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_permute, tokens, inv.cpu(), s, rows, st)
    refused(B.MOE_ERR_SHAPE, B.moe_permute, tokens[:1].expand(4, 64), inv, s, rows, st)
    refused(B.MOE_ERR_ALIGN, B.moe_permute, torch.zeros(4 * 64 + 1, **bf)[1:].view(4, 64), inv, s, rows, st)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_unpermute, rows, inv, w.bfloat16(), s, tokens, st)
    refused(B.MOE_ERR_SHAPE, B.moe_unpermute, rows, inv, w.t(), s, tokens, st)
    refused(B.MOE_ERR_NULL, B.moe_unpermute_grad, tokens, rows, inv, w, s, rows, None, st)
    codes, scales = torch.zeros((8, 64), dtype=torch.uint8, device="cuda"), torch.zeros((8, 2), dtype=torch.uint8, device="cuda")
    refused(B.MOE_ERR_SHAPE, B.moe_gated_act, rows, torch.zeros((8, 64), **bf))
    refused(B.MOE_ERR_NULL, B.moe_gated_act, rows, rows[:, :32].contiguous(), codes)
    refused(B.MOE_ERR_SHAPE, B.moe_gated_act, rows, rows[:, :32].contiguous(), codes, scales[:4])
    refused(B.MOE_ERR_SHAPE, B.moe_gated_act_grad, rows, codes[:2], scales, torch.zeros((8, 128), **bf))
    mx = torch.zeros(B.moe_mxfp4_scale_bytes(8, 64, 2), dtype=torch.uint8, device="cuda")
    half = torch.zeros((8, 32), dtype=torch.uint8, device="cuda")
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_quantize, rows, half, mx[:512], 2, st)
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_quantize, rows, half, mx, 3, st)
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_quantize, tokens, half, mx, 2, st, offsets=ints([0, 4, 8]))
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_quantize, tokens, half, mx, 2, st, offsets=ints([0, 8]), inv_perm=inv)
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_mxfp4_quantize, rows, half.char(), mx, 2, st)
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_dequantize, half, mx, 2, tokens, st)
    wc, wsc = torch.zeros((2, 16, 16), dtype=torch.uint8, device="cuda"), torch.zeros(B.moe_mxfp4_scale_bytes(32, 32, 2), dtype=torch.uint8, device="cuda")
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_gemm, half, mx, wc, wsc, ints([0, 4, 8]), torch.zeros((8, 16), **bf), st)
    wc, wsc = torch.zeros((2, 16, 32), dtype=torch.uint8, device="cuda"), torch.zeros(B.moe_mxfp4_scale_bytes(32, 64, 2), dtype=torch.uint8, device="cuda")
    refused(B.MOE_ERR_UNSUPPORTED, B.moe_mxfp4_gemm, half, mx, wc, wsc, ints([0, 4, 8]), torch.zeros((8, 16), device="cuda"), st)
    refused(B.MOE_ERR_SHAPE, B.moe_mxfp4_gemm, half, mx, wc, wsc, ints([0, 8]), torch.zeros((8, 16), **bf), st)
    B.moe_mxfp4_gemm(h, half, mx, wc, wsc, ints([0, 4, 8]), torch.zeros((8, 16), **bf), st)


def test_addresses_in_place_of_index_tensors():
    # the routing arrays as the library's own view names them: by address
    T, k, E, H = 40, 3, 7, 96
    h, s, st = handle(), shape_of(T, k, H), status()
    ws_keep, inv, offsets, _ = routed(T, k, E, 3)
    tokens = normal((T, H), torch.bfloat16, 1).cuda()
    rows = [torch.zeros((T * k, H), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.moe_permute(h, tokens, inv, s, rows[0], st)
    B.moe_permute(h, tokens, inv.data_ptr(), s, rows[1], st)
    assert torch.equal(*rows)
    codes = [torch.zeros((T * k, H // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(B.moe_mxfp4_scale_bytes(T * k, H, E), dtype=torch.uint8, device="cuda") for _ in range(2)]
    B.moe_mxfp4_quantize(h, tokens, codes[0], scales[0], E, st, offsets=offsets, inv_perm=inv)
    B.moe_mxfp4_quantize(h, tokens, codes[1], scales[1], E, st, offsets=offsets.data_ptr(), inv_perm=inv.data_ptr(), copies=k)
    assert torch.equal(*codes) and torch.equal(*scales) and st.tolist() == [0, 0, 0, 0]


def test_nothing_to_do():
    h, st = handle(), status()
    none = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    s = shape_of(0, 4, 64)
    B.moe_permute(h, none(0, 64), none(0, 4, dtype=torch.int32), s, none(0, 64), st)
    B.moe_unpermute_grad(h, none(0, 64), none(0, 64), none(0, 4, dtype=torch.int32), none(0, 4, dtype=torch.float32), s, none(0, 64), none(0, 4, dtype=torch.float32), st)
    B.moe_gated_act(h, none(0, 64), none(0, 32), none(0, 64, dtype=torch.uint8), none(0, 2, dtype=torch.uint8))
    scales = none(B.moe_mxfp4_scale_bytes(0, 64, 2), dtype=torch.uint8)
    B.moe_mxfp4_quantize(h, none(0, 64), none(0, 32, dtype=torch.uint8), scales, 2, st, offsets=ints([0, 0, 0]))
    w, ws = none(2, 16, 32, dtype=torch.uint8), none(B.moe_mxfp4_scale_bytes(32, 64, 2), dtype=torch.uint8)
    B.moe_mxfp4_gemm(h, none(0, 32, dtype=torch.uint8), scales, w, ws, ints([0, 0, 0]), none(0, 16), st)
    # rows that there are, but none of them in a group
    out = torch.full((5, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    x, xs = torch.zeros((5, 32), dtype=torch.uint8, device="cuda"), torch.zeros(B.moe_mxfp4_scale_bytes(5, 64, 2), dtype=torch.uint8, device="cuda")
    B.moe_mxfp4_gemm(h, x, xs, w, ws, ints([0, 0, 0]), out, st)
    assert (out == 7.0).all() and st.tolist() == [0, 0, 0, 0]


def test_a_status_buffer_on_the_host_is_refused():
    h, s = handle(), shape_of(4, 2, 64)
    tokens, rows, inv = torch.zeros((4, 64), device="cuda"), torch.zeros((8, 64), device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(B.MoeError) as e:
        B.moe_permute(h, tokens, inv, s, rows, torch.zeros(4, dtype=torch.int32))
    assert e.value.code == B.MOE_ERR_UNSUPPORTED


def test_products_on_two_streams_at_once():
    # both families of tiles beside each other and beside the row kernels, against the same calls one after the other
    small, large = [0, 5, 9, 30], [0, 400, 401, 900]
    jobs = []
    for offsets, N, K, seed in ((small, 264, 320, 1), (large, WIDE_N, 320, 2)):
        g = torch.Generator(device="cuda").manual_seed(seed)
        xc, xs, wc, ws, _, _ = wide_case(offsets, torch.randn((offsets[-1], K), device="cuda", generator=g), torch.randn((3 * N, K), device="cuda", generator=g), 3)
        jobs.append((xc, xs, wc, ws, ints(offsets), [torch.zeros((offsets[-1], N), dtype=torch.bfloat16, device="cuda") for _ in range(2)], status(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for which in range(2):
        for _ in range(20 if which else 1):
            for xc, xs, wc, ws, off, out, st, stream in jobs:
                with torch.cuda.stream(stream if which else torch.cuda.current_stream()):
                    B.moe_mxfp4_gemm(handle(), xc, xs, wc, ws, off, out[which], st)
        torch.cuda.synchronize()
    for *_, out, st, stream in jobs:
        assert torch.equal(*out) and st.tolist() == [0, 0, 0, 0]
