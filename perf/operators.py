"""The steps of a mixture-of-experts layer as operators of their own, as cases that can be timed and compared.

A case names an operator, the sizes of one MoE layer and the options in use:

  op "sort"     tokens sorted by expert: routing build from the router's choices, then every token's row copied to the rows of
                its experts; with `grad` the way back of a gradient as well (a token gets the sum of its rows').
     "back"     expert rows back to token order with the routing weights applied; with `grad` the gradients of the rows and of
                the weights.  `drop`: share of the assignments that have no row (an expert's capacity ran out).
     "act"      gated activation silu(gate) * up of the routed rows; with `train` it keeps gate and up as 8-bit floating
                point with a power of two per 32 values, and the backward pass reads that copy.
     "quant"    microscaled 4-bit floating point (32 values share a power of two): quantisation and back, of the experts'
                weights ("weights") or of tokens that are put in routed order on the way ("tokens").
     "product"  grouped product of routed rows and expert weights, both in microscaled 4 bits: gate and up projections in one
                ("up": N = 2 I, K = H) or the down projection ("down": N = H, K = I).
  skew  0: all experts equally popular; s > 0: expert popularity follows Zipf(s), softened by per-token noise so that the
        busiest expert gets about 2.5 to 3 times the mean load.

Sizes are the repository's four configurations (tiny, Granite-3-MoE-, Qwen1.5-MoE- and DeepSeek-V2-Lite-shaped) with one token
(a single stream decoding) to a 16384-token prefill or training batch.

Microscaled formats.  4 bits (e2m1): the shared exponent of 32 values is floor(log2(amax)) - 2, values are rounded to the nearest,
ties to even, and saturate at 6; two codes a byte, the even column in the low half.  The exponents (a byte each, biased by 127)
lie as the tensor cores take them: blocks of 128 rows x 128 columns are 512 bytes, the byte of row i and columns 32 s to 32 s + 31
at 16 (i % 32) + 4 (i / 32) + s; row r of group g (an expert), whose rows begin at o, is row (r - o) % 128 of row block
o / 128 + g + (r - o) / 128.  8 bits (e4m3): the shared exponent is the smallest at which nothing saturates.
"""

import torch

own = False

#: name -> (H, I, routed experts, experts per token, shared experts, Zipf exponent, noise that softens it)
FAMILIES = {
    "tiny": (256, 128, 8, 2, 0, 1.0, 3.2),
    "granite": (1536, 512, 40, 8, 0, 1.0, 3.2),
    "qwen": (2048, 1408, 60, 4, 0, 1.0, 5.8),
    "dsv2lite": (2048, 1408, 64, 6, 2, 1.2, 4.9),
}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _case(op, family, T, dtype="bf16", skewed=True, name=None, **options):
    H, I, E, k, shared, s, noise = FAMILIES[family]
    c = dict(op=op, T=T, H=H, I=I, E=E, k=k, shared=shared, dtype=dtype, skew=s if skewed else 0.0, noise=noise if skewed else 1.0, **options)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a small serving batch enters its experts: launches are all there is
        _case("sort", "dsv2lite", 16, grad=False, name="sort_decode_16"),
        # a training micro-batch, forward and backward
        _case("sort", "granite", 4096, grad=True, name="sort_train_4096"),
        # one stream decoding: one token's expert rows are added up
        _case("back", "dsv2lite", 1, skewed=False, grad=False, drop=0.0, name="back_decode_1"),
        # a training batch with capacity drops, forward and backward
        _case("back", "qwen", 8192, grad=True, drop=0.05, name="back_train_8192"),
        # a ragged prefill chunk, half precision, serving: nothing is kept
        _case("act", "granite", 1003, dtype="fp16", train=False, name="act_chunk_1003"),
        # the activation of a training batch with its 8-bit copy and its backward pass
        _case("act", "dsv2lite", 16384, train=True, name="act_train_16384"),
        # a serving batch's hidden states, quantised into routed order
        _case("quant", "dsv2lite", 256, what="tokens", name="quant_tokens_256"),
        # a checkpoint's expert weights, once when a model is loaded
        _case("quant", "qwen", 1, what="weights", name="quant_weights_qwen"),
        # one stream decoding: one token's experts are read
        _case("product", "dsv2lite", 1, skewed=False, proj="up", name="product_decode_1"),
        # a serving batch: nearly all experts' weights for a few rows each
        _case("product", "qwen", 48, proj="down", name="product_decode_48"),
        # a ragged prefill chunk
        _case("product", "granite", 1003, dtype="fp16", proj="up", name="product_chunk_1003"),
        # the largest: gate and up projections of a 16384-token prefill
        _case("product", "dsv2lite", 16384, proj="up", name="product_prefill_16384"),
    ]


def _log_int(rng, lo, hi):
    """Integer in [lo, hi], even over its logarithm; odd and ragged values come as they fall."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["sort", "back", "act", "quant", "product", "product"])
    family = rng.choice(["tiny", "granite", "qwen", "dsv2lite", "granite", "qwen", "dsv2lite"])
    T = _log_int(rng, 1, 16384)
    dtype = rng.choice(["bf16", "bf16", "fp16"] if op == "product" or T > 4096 else ["bf16", "fp16", "fp32"])
    more = {"sort": dict(grad=rng.random() < 0.6), "back": dict(grad=rng.random() < 0.6, drop=rng.choice([0.0, round(0.3 * rng.random(), 3)])),
            "act": dict(train=rng.random() < 0.6), "quant": dict(what=rng.choice(["tokens", "tokens", "weights"])),
            "product": dict(proj=rng.choice(["up", "down"]))}[op]
    return _case(op, family, T, dtype=dtype, skewed=rng.random() < 0.7, **more)


# ----------------------------------------------------------------------------- inputs

def _normal(gen, shape, std, dtype):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def _route(c, gen):
    """Top-k of noisy logits and the softmax of the selected ones; shared experts with weight one behind them."""
    T, E, k = c["T"], c["E"], c["k"]
    if c["skew"] > 0:
        rank = torch.randperm(E, generator=gen, device="cuda") + 1
        logits = c["noise"] * torch.randn((T, E), generator=gen, device="cuda") - c["skew"] * torch.log(rank.float())
    else:
        logits = torch.rand((T, E), generator=gen, device="cuda")
    top, idx = torch.topk(logits, k, dim=1)
    w = torch.softmax(top, dim=1)
    if c["shared"]:
        more = torch.arange(E, E + c["shared"], device="cuda").expand(T, -1)
        idx = torch.cat([idx, more], dim=1)
        w = torch.cat([w, torch.ones((T, c["shared"]), device="cuda")], dim=1)
    return idx.to(torch.int32).contiguous(), w.to(torch.float32).contiguous()


def _sorted(idx, E_tot, dropped=None):
    """Row of every assignment (-1: none) in the stable order by expert, and where each expert's rows begin."""
    e = idx.reshape(-1).long()
    if dropped is not None:
        e = torch.where(dropped.reshape(-1), E_tot, e)
    order = torch.sort(e, stable=True).indices
    inv = torch.empty_like(order)
    inv[order] = torch.arange(order.numel(), device=order.device)
    inv = torch.where(e < E_tot, inv, -1)
    counts = torch.bincount(e, minlength=E_tot + 1)[:E_tot]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return inv.reshape(idx.shape).to(torch.int32), offsets.to(torch.int32)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _fp4_of(x):
    """x [rows, K] -> codes [rows, K / 2] and biased exponents [rows, K / 32], both bytes."""
    rows, K = x.shape
    b = x.float().reshape(rows, K // 32, 32)
    amax = b.abs().amax(-1)
    ex = (torch.frexp(amax).exponent - 3).clamp(-127, 127)              # frexp's mantissa is in [0.5, 1)
    ex = torch.where(amax > 0, ex, -127)
    v = torch.ldexp(b, -ex.unsqueeze(-1)).reshape(rows, K)
    a = v.abs()
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code |= torch.signbit(v).to(torch.uint8) << 3
    return code[:, 0::2] | (code[:, 1::2] << 4), (ex + 127).to(torch.uint8)


def _blocks(rows, groups):
    return rows // 128 + groups


def _places(offsets, rows, K):
    """Where the exponents of [rows, K / 32] lie in the buffer; rows behind the last group have no place of their own (-1)."""
    o = offsets.long()
    r = torch.arange(rows, device=o.device)
    g = torch.searchsorted(o, r, right=True) - 1
    inside = r < o[-1]
    g = g.clamp(0, o.numel() - 2)
    i = r - o[g]
    block = torch.div(o[g], 128, rounding_mode="floor") + g + torch.div(i, 128, rounding_mode="floor")
    i = i % 128
    s = torch.arange(K // 32, device=o.device)
    per_row = (K + 127) // 128
    at = (block[:, None] * per_row + s[None, :] // 4) * 512 + (i % 32)[:, None] * 16 + (i // 32)[:, None] * 4 + (s % 4)[None, :]
    return torch.where(inside[:, None], at, -1)


def _laid_out(exponents, offsets, K):
    rows, groups = exponents.shape[0], offsets.numel() - 1
    buf = torch.zeros(_blocks(rows, groups) * ((K + 127) // 128) * 512 + 1, dtype=torch.uint8, device="cuda")
    buf[_places(offsets, rows, K).reshape(-1)] = exponents.reshape(-1)
    return buf[:-1]


def _even_offsets(groups, n):
    return torch.arange(groups + 1, device="cuda", dtype=torch.int32) * n


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    E_tot, k_tot, dt = c["E"] + c["shared"], c["k"] + c["shared"], DTYPES[c["dtype"]]
    T, H, I = c["T"], c["H"], c["I"]
    R = T * k_tot
    st = dict(case=c, E_tot=E_tot, k_tot=k_tot, dt=dt, R=R)
    if c["op"] == "act":
        st["gate_up"] = _normal(gen, (R, 2 * I), 1.0, dt)
        if c["train"]:
            st["d_act"] = _normal(gen, (R, I), 0.02, dt)
        return st
    if c["op"] == "quant" and c["what"] == "weights":
        st["src"] = _normal(gen, (E_tot * H, I), 0.02, dt)
        st["offsets"] = _even_offsets(E_tot, H)
        return st
    idx, w = _route(c, gen)
    if c["op"] == "sort":
        st.update(idx=idx, hidden=_normal(gen, (T, H), 1.0, dt))
        if c["grad"]:
            st["d_rows"] = _normal(gen, (R, H), 0.02, dt)
        return st
    dropped = torch.rand(idx.shape, generator=gen, device="cuda") < c["drop"] if c["op"] == "back" and c["drop"] > 0 else None
    st["inv_perm"], st["offsets"] = _sorted(idx, E_tot, dropped)
    if c["op"] == "back":
        st.update(w=w, rows=_normal(gen, (R, H), 1.0, dt))
        if c["grad"]:
            st["d_out"] = _normal(gen, (T, H), 0.02, dt)
    elif c["op"] == "quant":
        st["src"] = _normal(gen, (T, H), 1.0, dt)
    else:
        N, K = (2 * I, H) if c["proj"] == "up" else (H, I)
        codes, ex = _fp4_of(_normal(gen, (R, K), 1.0, torch.bfloat16))
        st["x_codes"], st["x_scales"] = codes, _laid_out(ex, st["offsets"], K)
        codes, ex = _fp4_of(_normal(gen, (E_tot * N, K), 0.02, torch.bfloat16))
        st["w_codes"], st["w_scales"] = codes.reshape(E_tot, N, K // 2), _laid_out(ex, _even_offsets(E_tot, N), K)
        st["counts"] = st["offsets"].diff().tolist()
    return st


# ----------------------------------------------------------------------------- the plain forms

def _e4m3_of(x):
    """x [rows, n] -> codes as float8 values, and biased exponents of every 32 columns."""
    rows, n = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -n % 32)).reshape(rows, -1, 32)
    amax = b.abs().amax(-1)
    m, ex = torch.frexp(amax)
    ex = (ex - 1 - 8 + (m > 0.875)).clamp(-127, 127)                    # m 2^ex = (2 m) 2^(ex - 1); 448 = 1.75 2^8
    ex = torch.where(amax > 0, ex, -127)
    v = torch.ldexp(b, -ex.unsqueeze(-1)).reshape(rows, -1)[:, :n]
    return v.to(torch.float8_e4m3fn), (ex + 127).to(torch.uint8)


def _e4m3_back(codes, exponents):
    n = codes.shape[1]
    return torch.ldexp(codes.float(), (exponents.int() - 127).repeat_interleave(32, 1)[:, :n])


def _fp4_values(codes, exponents):
    """fp32 values of codes [rows, K / 2] with their biased exponents [rows, K / 32]."""
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1)
    ex = exponents.int() - 127
    return torch.ldexp(v.reshape(*ex.shape, 32), ex.unsqueeze(-1)).reshape(codes.shape[0], -1)


def _fp4_back(codes, scales, offsets, K):
    return _fp4_values(codes, scales[_places(offsets, codes.shape[0], K)])


def _plain(s):
    c, dt = s["case"], s["dt"]
    if c["op"] == "sort":
        perm = torch.sort(s["idx"].reshape(-1), stable=True).indices
        inv = torch.empty_like(perm)
        inv[perm] = torch.arange(perm.numel(), device=perm.device)
        out = [inv.to(torch.int32).reshape(s["idx"].shape), s["hidden"][torch.div(perm, s["k_tot"], rounding_mode="floor")]]
        if c["grad"]:
            out.append(s["d_rows"].float()[inv].reshape(c["T"], s["k_tot"], c["H"]).sum(1).to(dt))
        return out
    if c["op"] == "back":
        flat = s["inv_perm"].reshape(-1).long()
        kept = flat >= 0
        y = s["rows"].float()[flat.clamp(min=0)] * kept[:, None]
        y = y.reshape(c["T"], s["k_tot"], c["H"])
        out = [(y * s["w"].unsqueeze(-1)).sum(1).to(dt)]
        if c["grad"]:
            d = s["d_out"].float().unsqueeze(1)
            d_rows = torch.zeros_like(s["rows"])
            d_rows[flat[kept]] = (d * s["w"].unsqueeze(-1)).reshape(-1, c["H"])[kept].to(dt)
            out += [d_rows, (d * y).sum(-1)]
        return out
    if c["op"] == "act":
        g, u = s["gate_up"][:, :c["I"]], s["gate_up"][:, c["I"]:]
        gf, uf = g.float(), u.float()
        act = (gf / (1.0 + torch.exp(-gf)) * uf).to(dt)
        if not c["train"]:
            return act
        (gc, gx), (uc, ux) = _e4m3_of(g), _e4m3_of(u)
        gf, uf, d = _e4m3_back(gc, gx), _e4m3_back(uc, ux), s["d_act"].float()
        sg = 1.0 / (1.0 + torch.exp(-gf))
        silu = gf * sg
        d_gate_up = torch.cat([d * uf * (sg * (1.0 + gf * (1.0 - sg))), d * silu], 1).to(dt)
        codes = torch.cat([gc.view(torch.uint8), uc.view(torch.uint8)], 1).view(torch.float8_e4m3fn)
        return [act, codes, torch.cat([gx, ux], 1), d_gate_up, (silu * uf).to(dt)]
    if c["op"] == "quant":
        src = s["src"]
        if c["what"] == "tokens":
            flat = s["inv_perm"].reshape(-1).long()
            perm = torch.empty_like(flat)
            perm[flat] = torch.arange(flat.numel(), device=flat.device)
            src = src[torch.div(perm, s["k_tot"], rounding_mode="floor")]
        codes, ex = _fp4_of(src)
        K = src.shape[1]
        return _fp4_back(codes, _laid_out(ex, s["offsets"], K), s["offsets"], K).to(torch.bfloat16)
    E, N, K2 = s["w_codes"].shape
    x = _fp4_back(s["x_codes"], s["x_scales"], s["offsets"], 2 * K2)
    used = torch.tensor([e for e, n in enumerate(s["counts"]) if n], device="cuda")
    at = _places(_even_offsets(E, N), E * N, 2 * K2).reshape(E, N, -1)[used].reshape(used.numel() * N, -1)
    w = _fp4_values(s["w_codes"][used].reshape(-1, K2), s["w_scales"][at]).reshape(-1, N, 2 * K2)
    out = torch.empty((s["R"], N), dtype=dt, device="cuda")
    at = 0
    for n, w_e in zip([n for n in s["counts"] if n], w):                 # the groups are ragged: one product for each that has rows
        out[at:at + n] = x[at:at + n] @ w_e.t()
        at += n
    return out


# ----------------------------------------------------------------------------- the framework's calls

_handles = {}


def _handle():
    """One handle per process and device, as a serving or training program keeps it."""
    from paper_2609_07536_b200 import binding as B
    dev = torch.cuda.current_device()
    if dev not in _handles:
        _handles[dev] = B.moe_create(dev)
    return _handles[dev]


def _kept(s):
    """The buffers that a user's program keeps between passes: results, routing workspace, status."""
    if "kept" in s:
        return s["kept"]
    from paper_2609_07536_b200 import binding as B
    c, dt = s["case"], s["dt"]
    T, H, I, R = c["T"], c["H"], c["I"], s["R"]
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    b = dict(B=B, h=_handle(), status=torch.zeros(4, dtype=torch.int32, device="cuda"),
             shape=B.make_shape(T, H, I, s["E_tot"], s["k_tot"], 1, 1, 1))
    if c["op"] == "sort":
        b["ws"] = torch.empty(B.moe_workspace_bytes(b["shape"], 128, 128)[0], dtype=torch.uint8, device="cuda")
        b["routing"] = B.moe_routing_view(b["ws"], b["shape"], 128)
        at = b["routing"].inv_perm - b["ws"].data_ptr()
        b["inv_perm"] = b["ws"][at:at + 4 * R].view(torch.int32).reshape(T, s["k_tot"])
        b["rows"] = new(R, H)
        b["result"] = [b["inv_perm"], b["rows"]]
        if c["grad"]:
            b["d_tokens"] = new(T, H)
            b["result"].append(b["d_tokens"])
    elif c["op"] == "back":
        b["out"] = new(T, H)
        b["result"] = [b["out"]]
        if c["grad"]:
            b["d_rows"], b["d_w"] = new(R, H).zero_(), new(T, s["k_tot"], dtype=torch.float32)
            b["result"] += [b["d_rows"], b["d_w"]]
    elif c["op"] == "act":
        b["act"] = new(R, I)
        b["result"] = b["act"]
        if c["train"]:
            b["codes"] = new(R, 2 * I, dtype=torch.uint8)
            b["scales"] = new(R, 2 * ((I + 31) // 32), dtype=torch.uint8)
            b["d_gate_up"], b["act_again"] = new(R, 2 * I), new(R, I)
            b["result"] = [b["act"], b["codes"].view(torch.float8_e4m3fn), b["scales"], b["d_gate_up"], b["act_again"]]
    elif c["op"] == "quant":
        rows, K = (R, H) if c["what"] == "tokens" else s["src"].shape
        b["codes"] = new(rows, K // 2, dtype=torch.uint8)
        b["scales"] = new(B.moe_mxfp4_scale_bytes(rows, K, s["E_tot"]), dtype=torch.uint8)
        b["result"] = new(rows, K, dtype=torch.bfloat16)
    else:
        b["result"] = new(R, s["w_codes"].shape[1])
    s["kept"] = b
    return b


def run(state):
    s = state
    if not own:
        return _plain(s)
    c, b = s["case"], _kept(s)
    B, h, shape, status = b["B"], b["h"], b["shape"], b["status"]
    if c["op"] == "sort":
        B.moe_build_routing(h, s["idx"], shape, 128, b["routing"], None, status)
        B.moe_permute(h, s["hidden"], b["inv_perm"], shape, b["rows"], status)
        if c["grad"]:
            B.moe_permute_grad(h, s["d_rows"], b["inv_perm"], shape, b["d_tokens"], status)
    elif c["op"] == "back":
        B.moe_unpermute(h, s["rows"], s["inv_perm"], s["w"], shape, b["out"], status)
        if c["grad"]:
            B.moe_unpermute_grad(h, s["d_out"], s["rows"], s["inv_perm"], s["w"], shape, b["d_rows"], b["d_w"], status)
    elif c["op"] == "act":
        if c["train"]:
            B.moe_gated_act(h, s["gate_up"], b["act"], b["codes"], b["scales"])
            B.moe_gated_act_grad(h, s["d_act"], b["codes"], b["scales"], b["d_gate_up"], b["act_again"])
        else:
            B.moe_gated_act(h, s["gate_up"], b["act"])
    elif c["op"] == "quant":
        if c["what"] == "tokens":
            B.moe_mxfp4_quantize(h, s["src"], b["codes"], b["scales"], s["E_tot"], status, offsets=s["offsets"], inv_perm=s["inv_perm"])
            B.moe_mxfp4_dequantize(h, b["codes"], b["scales"], s["E_tot"], b["result"], status, offsets=s["offsets"])
        else:
            B.moe_mxfp4_quantize(h, s["src"], b["codes"], b["scales"], s["E_tot"], status)
            B.moe_mxfp4_dequantize(h, b["codes"], b["scales"], s["E_tot"], b["result"], status)
    else:
        B.moe_mxfp4_gemm(h, s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["offsets"], b["result"], status)
    return b["result"]


# ----------------------------------------------------------------------------- what a pass needs

def work(case):
    """Bytes: every input once and every output once; of the weights, those of the experts that some token chose (expected
    number, experts equally popular).  Flops: products only."""
    c = case
    k_tot, E_tot = c["k"] + c["shared"], c["E"] + c["shared"]
    T, H, I = c["T"], c["H"], c["I"]
    R, size = T * k_tot, DTYPES[c["dtype"]].itemsize
    if c["op"] == "sort":
        n = T * H * size + R * H * size + 2 * R * 4
        return {"bytes": float(2 * n - R * 4 if c["grad"] else n), "flops": float(R * H if c["grad"] else 0)}
    if c["op"] == "back":
        kept = R * (1.0 - c["drop"])
        n = kept * H * size + T * H * size + R * 8
        if c["grad"]:
            n += T * H * size + kept * H * size + R * 4
        return {"bytes": float(n), "flops": float((5 if c["grad"] else 2) * kept * H)}
    if c["op"] == "act":
        n = 3 * R * I * size
        if c["train"]:
            n += 2 * R * I + R * 2 * ((I + 31) // 32) + 4 * R * I * size
        return {"bytes": float(n), "flops": float((20 if c["train"] else 5) * R * I)}
    if c["op"] == "quant":
        rows, K, read = (R, H, T) if c["what"] == "tokens" else (E_tot * H, I, E_tot * H)
        return {"bytes": float(read * K * size + rows * (K / 2 + K / 32) + rows * K * 2), "flops": float(2 * rows * K)}
    N, K = (2 * I, H) if c["proj"] == "up" else (H, I)
    used = c["E"] * (1.0 - (1.0 - c["k"] / c["E"]) ** T) + c["shared"]
    per = K / 2 + K / 32
    return {"bytes": float(R * per + used * N * per + R * N * 2 + 4 * (E_tot + 1)), "flops": 2.0 * R * N * K}


# ----------------------------------------------------------------------------- the definitions in 64 bits

def _power(x):
    """floor(log2(x)) of positive doubles, exactly."""
    return torch.frexp(x).exponent.double() - 1.0


def _rounded(x, step):
    return torch.round(x / step) * step                                 # ties to even


def _exact_e4m3(x):
    n = x.shape[1]
    b = torch.nn.functional.pad(x.double(), (0, -n % 32)).reshape(x.shape[0], -1, 32)
    amax = b.abs().amax(-1, keepdim=True)
    ex = _power(amax.clamp(min=2.0 ** -300)) - 8.0
    ex = torch.where(amax > 448.0 * torch.exp2(ex), ex + 1.0, ex).clamp(-127.0, 127.0)
    v = b * torch.exp2(-ex)
    q = _rounded(v, torch.exp2(_power(v.abs().clamp(min=2.0 ** -6)) - 3.0))
    return q.reshape(x.shape[0], -1)[:, :n], (q * torch.exp2(ex)).reshape(x.shape[0], -1)[:, :n]


def _exact_fp4(x):
    b = x.double().reshape(x.shape[0], -1, 32)
    ex = (_power(b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -300)) - 2.0).clamp(-127.0, 127.0)
    v = b * torch.exp2(-ex)
    q = _rounded(v, torch.exp2(_power(v.abs().clamp(min=1.0)) - 1.0)).clamp(-6.0, 6.0)
    return (q * torch.exp2(ex)).reshape(x.shape)


def _exact_decode(codes, scales, offsets, K):
    rows = codes.shape[0]
    c = torch.stack([codes % 16, codes // 16], -1).reshape(rows, K).double()
    neg, c = c >= 8, c % 8
    e, m = torch.floor(c / 2), c % 2
    v = torch.where(e > 0, (1.0 + m / 2) * torch.exp2(e - 1.0), m / 2)
    ex = scales[_places(offsets, rows, K)].double() - 127.0
    return torch.where(neg, -v, v) * torch.exp2(ex).repeat_interleave(32, 1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    T, H, I, k = c["T"], c["H"], c["I"], s["k_tot"]
    if c["op"] in ("sort", "back"):
        if c["op"] == "sort":
            e = s["idx"].reshape(-1).double() * s["R"] + torch.arange(s["R"], device="cuda")
            rows_of = torch.argsort(e)                                  # by expert, then by place: all keys differ
            x = s["hidden"].double().repeat_interleave(k, 0)[rows_of]
            if not c["grad"]:
                return [None, x]
            back = torch.empty_like(s["d_rows"], dtype=torch.float64)
            back[rows_of] = s["d_rows"].double()
            return [None, x, back.reshape(T, k, H).sum(1)]
        flat = s["inv_perm"].reshape(-1).long()
        ext = torch.cat([s["rows"].double(), s["rows"].new_zeros((1, H), dtype=torch.float64)])   # row -1: zeros
        y, w = ext[flat].reshape(T, k, H), s["w"].double()
        out = [torch.einsum("tkh,tk->th", y, w)]
        if c["grad"]:
            d = s["d_out"].double()
            d_rows = torch.zeros_like(ext)
            d_rows[flat] = torch.einsum("th,tk->tkh", d, w).reshape(-1, H)
            out += [d_rows[:-1], torch.einsum("tkh,th->tk", y, d)]
        return out
    if c["op"] == "act":
        sig = torch.sigmoid
        g, u = s["gate_up"].double().split(I, 1)
        act = g * sig(g) * u
        if not c["train"]:
            return act
        (gq, gv), (uq, uv), d = _exact_e4m3(g), _exact_e4m3(u), s["d_act"].double()
        sg = sig(gv)
        return [act, torch.cat([gq, uq], 1), None, torch.cat([d * uv * sg * (1.0 + gv * sig(-gv)), d * gv * sg], 1), gv * sg * uv]
    if c["op"] == "quant":
        v = _exact_fp4(s["src"])
        if c["what"] == "weights":
            return v
        out = torch.empty((s["R"], H), dtype=torch.float64, device="cuda")
        out[s["inv_perm"].reshape(-1).long()] = v.repeat_interleave(k, 0)
        return out
    E, N, K2 = s["w_codes"].shape
    even = _even_offsets(1, N)
    x = _exact_decode(s["x_codes"], s["x_scales"], s["offsets"], 2 * K2)
    out, at, per_row = [], 0, (2 * K2 + 127) // 128 * 512
    for e, n in enumerate(s["counts"]):
        if n:
            first = (e * N // 128 + e) * per_row
            w = _exact_decode(s["w_codes"][e], s["w_scales"][first:first + _blocks(N, 1) * per_row], even, 2 * K2)
            out.append(x[at:at + n] @ w.t())
        at += n
    return torch.cat(out)
