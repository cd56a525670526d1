// Gated activation between the two expert products (Section II-A), act = silu(gate) * up, on rows [gate | up], with gate and up kept in
// 8 bits for the backward pass, and that backward pass, which reads nothing but the 8-bit copy:
//   s = 1 / (1 + exp(-g)),  silu = g s,  d_up = d_act silu,  d_gate = d_act u s (1 + g (1 - s)),  act = silu u.
// The copy: e4m3 codes, and for every 32 columns of gate and of up one byte e, the power of two 2^(e - 127) that the codes are
// multiplied by: the smallest at which the largest magnitude of the 32 does not exceed e4m3's 448 (not floor(log2(amax)) - 8, at
// which values up to an eighth beyond 448 would saturate).  The scaling is exact, so that a value's one rounding is the
// code's, half a step of 2^-3 of it.  A value that is infinite or no number becomes the code for no number, alone.
// Bound by HBM: 2 I elements in, I out, 2 I + I / 16 bytes of copy; the backward pass reads I elements and the copy and writes 2 I
// elements (and the I of act, which the gradient of the next weights needs and which is not kept).  A thread has 16 (backward
// pass: 8) columns of gate and the same of up.

#include <cuda_fp8.h>

#include "rows_device.cuh"
#include "sm100_device.cuh"

namespace moe {
namespace {

constexpr int kActThreads = 256;

struct GatedAct {
    long long ld_in, ld_act, ld_d_act, ld_out;   // elements: gate_up, act, d_act, d_gate_up
    uint8_t *codes, *scales;
    int32_t rows, I, lanes;            // lanes: threads of a row, two per 32 columns (backward pass: four)
    int32_t rows_per_cta, wide;        // wide: 16 columns of the matrices are on 32-byte boundaries
    Divisor by_lanes;
};

// x / (1 + exp(-g)), down to fp32's smallest numbers: at g = -88.7, where exp(-g) leaves the range of fp32, silu(g) is -3e-37, a normal
// number, and another factor may make it an ordinary one.  fp32: of exp(-|g|), which is at most 1.  16-bit results do not see the
// approximations' last bits: 2^-24 / (2^-24 + 2^(-24 - g log2(e))), whose exponential ends where the quotient does, at 2^150, and costs no
// instruction more.  Absolute error of the quotient where it is subnormal: a step of 2^-149.
template <class E>
__device__ __forceinline__ float sigmoid_times(float x, float g)
{
    if constexpr (sizeof(E) == 4) {
        const float e = expf(-fabsf(g));
        return (g < 0.0f ? x * e : x) / (1.0f + e);
    } else {
        float e, r;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fmaf(-g, 1.44269504f, -24.0f)));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(0x1p-24f + e));
        return x * (r * 0x1p-24f);
    }
}

// sixteen codes of x * 2^-e, x = 0 .. 448 * 2^e in magnitude
__device__ __forceinline__ uint4 e4m3_codes(const float (&x)[16], int e)
{
    const float inv = power_of_two(-e);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i] * inv, x[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2] * inv, x[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | (hi << 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Where a value is not finite: the largest finite magnitude, and the code for no number in the place of such values
__device__ __forceinline__ float finite_magnitude(const float (&x)[16])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (fabsf(x[i]) <= 3.402823466e38f) m = fmaxf(m, fabsf(x[i]));
    return m;
}
__device__ __forceinline__ uint4 mark_not_finite(const float (&x)[16], uint4 codes)
{
    uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (!(fabsf(x[i]) <= 3.402823466e38f)) w[i >> 2] |= 0x7Fu << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// the exponent for a largest magnitude: smallest e >= -127 with amax <= 448 * 2^e = 1.75 * 2^(e + 8)
__device__ __forceinline__ int e4m3_exponent(uint32_t amax_bits)
{
    return max(-127, (int)((amax_bits + 0x1FFFFFu) >> 23) - 127 - 8);
}
__device__ __forceinline__ void e4m3_values(uint2 c, float scale, float (&x)[8])
{
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[2 * i] = f.x * scale;
        x[2 * i + 1] = f.y * scale;
    }
}

// Two threads share the exponents of 32 columns.  What costs besides the bytes is the issue of the instructions that make the copy: a
// thread takes 16 columns, so that addresses and exponents are worked out once for them, and finds its largest magnitudes in the
// 16-bit patterns, two values a step.  131072 rows of 2 x 1408 in bf16: 226 us, 101 % of the measured copy bandwidth (8 columns a thread and
// magnitudes in fp32: 304); without the copy 163 us.
template <class E, bool kKeep>
__global__ void __launch_bounds__(kActThreads, 4) gated_act_kernel(const __grid_constant__ GatedAct p, const E *gate_up, E *act)
{
    grid_dependency_wait();
    const long long row0 = (long long)blockIdx.x * p.rows_per_cta;
    const int items = (int)min((long long)p.rows_per_cta, p.rows - row0) * p.lanes;
    for (int base = (int)(threadIdx.x & ~31u); base < items; base += kActThreads) {
        const int it = base + (int)(threadIdx.x & 31u), r = quotient(p.by_lanes, it), q = it - r * p.lanes;
        const long long row = row0 + r;
        const bool live = it < items && q * 16 < p.I;
        Raw16<E> rg = {}, ru = {};
        float g[16], u[16];
        if (live) {
            const E *src = gate_up + row * p.ld_in + q * 16;
            load16<E>(src, p.wide, rg);
            load16<E>(src + p.I, p.wide, ru);
        }
        values16<E>(rg, g);
        values16<E>(ru, u);
        const auto activate = [&]() {
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = sigmoid_times<E>(g[i], g[i]) * u[i];
            store16<E>(act + row * p.ld_act + q * 16, p.wide, y);
        };
        if (!kKeep) {
            if (live) activate();
            continue;
        }
        uint32_t mg = magnitude16<E>(rg), mu = magnitude16<E>(ru);
        if constexpr (sizeof(E) == 2) {
            uint32_t both = mg | (mu << 16);
            both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 1));
            mg = both & 0xffffu;
            mu = both >> 16;
        } else {
            mg = max(mg, __shfl_xor_sync(0xffffffffu, mg, 1));
            mu = max(mu, __shfl_xor_sync(0xffffffffu, mu, 1));
        }
        uint32_t bg = magnitude_bits<E>(mg), bu = magnitude_bits<E>(mu);
        const bool hurt = mg >= kNotFinite<E> || mu >= kNotFinite<E>;
        if (__any_sync(0xffffffffu, hurt)) {
            float fg = finite_magnitude(g), fu = finite_magnitude(u);
            bg = __float_as_uint(fmaxf(fg, __shfl_xor_sync(0xffffffffu, fg, 1)));
            bu = __float_as_uint(fmaxf(fu, __shfl_xor_sync(0xffffffffu, fu, 1)));
        }
        if (!live) continue;
        const int eg = e4m3_exponent(bg), eu = e4m3_exponent(bu), blocks = p.lanes >> 1;
        uint4 cg = e4m3_codes(g, eg), cu = e4m3_codes(u, eu);
        if (hurt) {
            cg = mark_not_finite(g, cg);
            cu = mark_not_finite(u, cu);
        }
        uint8_t *c = p.codes + row * 2 * p.I + q * 16;
        st_row_v4(c, cg);
        st_row_v4(c + p.I, cu);
        activate();                            // (behind the copy: in front of it, it held values in registers that spilled)
        if ((q & 1) == 0) {
            uint8_t *sc = p.scales + row * 2 * blocks + (q >> 1);
            sc[0] = (uint8_t)(eg + 127);
            sc[blocks] = (uint8_t)(eu + 127);
        }
    }
}

// 131072 rows of 2 x 1408 in bf16, the activation written again: 280 us, 1.86 GB at the measured copy bandwidth.
template <class E>
__global__ void __launch_bounds__(kActThreads) gated_act_grad_kernel(const __grid_constant__ GatedAct p, const E *d_act, E *d_gate_up, E *act)
{
    grid_dependency_wait();
    const long long row0 = (long long)blockIdx.x * p.rows_per_cta;
    const int items = (int)min((long long)p.rows_per_cta, p.rows - row0) * p.lanes, blocks = p.lanes >> 2;
    for (int it = (int)threadIdx.x; it < items; it += kActThreads) {
        const int r = quotient(p.by_lanes, it), q = it - r * p.lanes;
        if (q * 8 >= p.I) continue;
        const long long row = row0 + r;
        const uint8_t *c = p.codes + row * 2 * p.I + q * 8, *sc = p.scales + row * 2 * blocks + (q >> 2);
        const uint2 cg = ld_row_v2(c), cu = ld_row_v2(c + p.I);
        const float sg = power_of_two((int)ld_row_u8(sc) - 127), su = power_of_two((int)ld_row_u8(sc + blocks) - 127);
        float d[8], g[8], u[8];
        load8<E>(d_act + row * p.ld_d_act + q * 8, d);
        e4m3_values(cg, sg, g);
        e4m3_values(cu, su, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = sigmoid_times<E>(1.0f, g[i]), silu = g[i] * s;
            const float dg = d[i] * u[i] * (s * fmaf(g[i], 1.0f - s, 1.0f));
            u[i] *= silu;                   // act
            d[i] *= silu;                   // d_up
            g[i] = dg;
        }
        E *dst = d_gate_up + row * p.ld_out + q * 8;
        store8<E>(dst, g);
        store8<E>(dst + p.I, d);
        if (act) store8<E>(act + row * p.ld_act + q * 8, u);
    }
}

bool sizes_ok(int32_t rows, int32_t I) { return rows >= 0 && rows < 1 << 30 && I >= 16 && I % 16 == 0 && I <= 1 << 20; }

GatedAct describe(const moe_handle *h, int32_t rows, int32_t I, int lanes_per_block, int rows_per_cta)
{
    GatedAct p = {};
    p.rows = rows;
    p.I = I;
    p.lanes = (I + 31) / 32 * lanes_per_block;
    p.by_lanes = divisor_of(p.lanes);
    // rows a block: many fill its passes of 256 threads, few let the next block start sooner, fewer still where that leaves SMs without one
    p.rows_per_cta = rows_per_cta;
    while (p.rows_per_cta > 1 && (int64_t)rows < (int64_t)p.rows_per_cta * 4 * h->G) p.rows_per_cta /= 2;
    return p;
}

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" int32_t moe_gated_act(moe_handle *h, const void *gate_up, int64_t ld_gate_up, int32_t rows, int32_t I, int32_t dtype, void *act,
                                 int64_t ld_act, void *codes_or_null, void *scales_or_null, void *stream)
{
    if (!h) return MOE_ERR_NULL;
    if (!sizes_ok(rows, I)) return MOE_ERR_SHAPE;
    if (!row_type_ok(dtype)) return MOE_ERR_UNSUPPORTED;
    if (!pitch_ok(ld_gate_up, 2 * (int64_t)I) || !pitch_ok(ld_act, I)) return MOE_ERR_SHAPE;
    if (rows == 0) return MOE_OK;
    if (!gate_up || !act || !codes_or_null != !scales_or_null) return MOE_ERR_NULL;
    if (!rows_aligned(gate_up) || !rows_aligned(act) || !rows_aligned(codes_or_null)) return MOE_ERR_ALIGN;
    if (const int32_t rc = require_handle_device(h, "moe_gated_act")) return rc;
    GatedAct p = describe(h, rows, I, 2, 8);     // 16 / 8 / 4 / 2 rows: 63.5 / 61.0 / 64.8 / 66.1 us at 32768 rows of 2 x 1408
    p.wide = rows_wide(gate_up, ld_gate_up, dtype) && rows_wide(act, ld_act, dtype);
    p.ld_in = ld_gate_up;
    p.ld_act = ld_act;
    p.codes = static_cast<uint8_t *>(codes_or_null);
    p.scales = static_cast<uint8_t *>(scales_or_null);
    const unsigned grid = (unsigned)((rows + p.rows_per_cta - 1) / p.rows_per_cta);
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const E *in = static_cast<const E *>(gate_up);
        E *out = static_cast<E *>(act);
        const cudaError_t err = launch_chained(codes_or_null ? gated_act_kernel<E, true> : gated_act_kernel<E, false>, grid, kActThreads, 0,
                                               static_cast<cudaStream_t>(stream), p, in, out);
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "gated activation launch");
    });
}

extern "C" int32_t moe_gated_act_grad(moe_handle *h, const void *d_act, int64_t ld_d_act, const void *codes, const void *scales, int32_t rows,
                                      int32_t I, int32_t dtype, void *d_gate_up, int64_t ld_d_gate_up, void *act_or_null, int64_t ld_act, void *stream)
{
    if (!h) return MOE_ERR_NULL;
    if (!sizes_ok(rows, I)) return MOE_ERR_SHAPE;
    if (!row_type_ok(dtype)) return MOE_ERR_UNSUPPORTED;
    if (!pitch_ok(ld_d_gate_up, 2 * (int64_t)I) || !pitch_ok(ld_d_act, I) || (act_or_null && !pitch_ok(ld_act, I))) return MOE_ERR_SHAPE;
    if (rows == 0) return MOE_OK;
    if (!d_act || !codes || !scales || !d_gate_up) return MOE_ERR_NULL;
    if (!rows_aligned(d_act) || !rows_aligned(codes) || !rows_aligned(d_gate_up) || !rows_aligned(act_or_null)) return MOE_ERR_ALIGN;
    if (const int32_t rc = require_handle_device(h, "moe_gated_act_grad")) return rc;
    GatedAct p = describe(h, rows, I, 4, 4);     // 16 / 8 / 4 / 2 rows: 80.8 / 75.6 / 72.9 / 74.4 us at 32768 rows of 2 x 1408
    p.ld_act = ld_act;
    p.ld_d_act = ld_d_act;
    p.ld_out = ld_d_gate_up;
    p.codes = static_cast<uint8_t *>(const_cast<void *>(codes));
    p.scales = static_cast<uint8_t *>(const_cast<void *>(scales));
    const unsigned grid = (unsigned)((rows + p.rows_per_cta - 1) / p.rows_per_cta);
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const E *in = static_cast<const E *>(d_act);
        E *out = static_cast<E *>(d_gate_up), *again = static_cast<E *>(act_or_null);
        const cudaError_t err = launch_chained(gated_act_grad_kernel<E>, grid, kActThreads, 0, static_cast<cudaStream_t>(stream), p, in, out, again);
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "gated activation gradient launch");
    });
}
