"""The steps of a mixture-of-experts layer, each from its definition, in 64 bits with numpy: tokens to expert rows and back with
their gradients, the gated activation with its 8-bit copy and its backward pass, microscaled 4-bit floating point and the grouped
product.  Written for clarity; the CUDA path shares nothing with it."""

from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ----------------------------------------------------------------------------- tokens to rows and back

def permute(tokens, inv_perm, rows_before):
    """rows[inv_perm[t][j]] = tokens[t]; the other rows as they were."""
    out = np.array(rows_before, dtype=np.float64)
    for t in range(inv_perm.shape[0]):
        for r in inv_perm[t]:
            if r >= 0:
                out[r] = tokens[t]
    return out


def unpermute(rows, inv_perm, w=None):
    """out[t] = sum_j w[t][j] rows[inv_perm[t][j]], and the sum of the magnitudes that were added."""
    T, k = inv_perm.shape
    out = np.zeros((T, rows.shape[1]))
    mag = np.zeros_like(out)
    for t in range(T):
        for j in range(k):
            r = inv_perm[t, j]
            if r >= 0:
                v = np.asarray(rows[r], dtype=np.float64) * (1.0 if w is None else float(w[t, j]))
                out[t] += v
                mag[t] += np.abs(v)
    return out, mag


def unpermute_grad(d_out, rows, inv_perm, w, d_rows_before):
    """(d_rows, d_w, sum of the magnitudes behind d_w)."""
    T, k = inv_perm.shape
    d_rows = np.array(d_rows_before, dtype=np.float64)
    d_w, mag = np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            r = inv_perm[t, j]
            if r >= 0:
                d = np.asarray(d_out[t], dtype=np.float64)
                prod = d * rows[r]
                d_rows[r] = float(w[t, j]) * d
                d_w[t, j], mag[t, j] = prod.sum(), np.abs(prod).sum()
    return d_rows, d_w, mag


# ----------------------------------------------------------------------------- gated activation

def sigmoid(g):
    g = np.asarray(g, dtype=np.float64)
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def gated_act(gate, up):
    return gate * sigmoid(gate) * up


def gated_act_grad(d_act, gate, up):
    """(d_gate, d_up)."""
    s = sigmoid(gate)
    return d_act * up * s * (1.0 + gate * sigmoid(-np.asarray(gate, dtype=np.float64))), d_act * gate * s


def _in_blocks(x):
    """[rows, n] -> [rows, ceil(n / 32), 32], zeros behind the last column."""
    rows, n = x.shape
    return np.concatenate([x, np.zeros((rows, -n % 32))], axis=1).reshape(rows, -1, 32)


def round_to(v, mantissa, smallest):
    """Nearest value with `mantissa` bits behind the leading one (fixed point below the exponent `smallest`), ties to even."""
    _, e = np.frexp(np.where(v == 0, 1.0, np.abs(v)))
    step = np.exp2(np.maximum(e - 1.0, smallest) - mantissa)
    return np.rint(v / step) * step


def checkpoint(x):
    """(values of the e4m3 codes, exponents): the smallest exponent >= -127 at which no finite value of 32 exceeds 448; values that are
    not finite are no number."""
    b = _in_blocks(np.asarray(x, dtype=np.float64))
    fine = np.isfinite(b)
    amax = np.where(fine, np.abs(b), 0.0).max(-1)
    e = np.where(amax > 0, np.ceil(np.log2(np.where(amax > 0, amax, 1.0) / 448.0)), -127)
    for _ in range(2):                                                   # (the logarithm may be off by a unit where it is near a whole number)
        e = np.where(amax > 448.0 * np.exp2(e), e + 1, e)
        e = np.where((amax <= 448.0 * np.exp2(e - 1)) & (e > -127), e - 1, e)
    e = np.maximum(e, -127)
    q = round_to(np.where(fine, b, 0.0) * np.exp2(-e)[..., None], 3, -6)
    q = np.where(fine, q, np.nan)
    return q.reshape(x.shape[0], -1)[:, :x.shape[1]], e.astype(np.int64)


def checkpoint_values(q, e):
    return (_in_blocks(q) * np.exp2(e.astype(np.float64))[..., None]).reshape(q.shape[0], -1)[:, :q.shape[1]]


# ----------------------------------------------------------------------------- microscaled 4 bits

def quantize(x):
    """x [rows, K] -> codes uint8 [rows, K / 2], biased exponents uint8 [rows, K / 32]."""
    rows, K = x.shape
    b = np.asarray(x, dtype=np.float64).reshape(rows, K // 32, 32)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    amax = np.abs(b).max(-1)
    e = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 3, -127)
    e = np.clip(e, -127, 127)
    v = b * np.exp2(-e.astype(np.float64))[..., None]
    mag = np.abs(v)
    dist = np.abs(mag[..., None] - E2M1)                                 # nearest of the eight; of two equally near ones the even code
    best = dist.min(-1, keepdims=True)
    near = dist == best
    code = np.where(near[..., ::2].any(-1), near[..., ::2].argmax(-1) * 2, near[..., 1::2].argmax(-1) * 2 + 1)
    code = code + 8 * np.signbit(v)
    code = np.where(bad[..., None], 0, code).reshape(rows, K)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def dequantize(codes, exponents):
    rows = codes.shape[0]
    c = np.stack([codes & 15, codes >> 4], -1).reshape(rows, exponents.shape[1], 32)
    v = np.where(c >= 8, -E2M1[c & 7], E2M1[c & 7])
    scale = np.where(exponents == 255, np.nan, np.exp2(exponents.astype(np.float64) - 127.0))
    return (v * scale[..., None]).reshape(rows, -1)


def scale_place(r, offsets, K, s):
    """Byte of the exponent of row r, columns 32 s .. 32 s + 31."""
    g = max(i for i in range(len(offsets) - 1) if offsets[i] <= r)
    i = r - offsets[g]
    block = offsets[g] // 128 + g + i // 128
    i %= 128
    return (block * (-(-K // 128)) + s // 4) * 512 + 16 * (i % 32) + 4 * (i // 32) + s % 4


def scale_places(offsets, K):
    """[rows of all groups, K / 32]"""
    n = offsets[-1]
    return np.array([[scale_place(r, offsets, K, s) for s in range(K // 32)] for r in range(n)], dtype=np.int64).reshape(n, K // 32)


def grouped_product(x, w, offsets):
    """out[r] = w[e] x[r], and the sum of the magnitudes that were added."""
    out, mag = [], []
    for e in range(len(offsets) - 1):
        xe = x[offsets[e]:offsets[e + 1]]
        out.append(xe @ w[e].T)
        mag.append(np.abs(xe) @ np.abs(w[e]).T)
    return np.concatenate(out), np.concatenate(mag)
