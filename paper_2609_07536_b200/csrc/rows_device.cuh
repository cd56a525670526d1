// Device-side building blocks of the operators that work on rows of 16- or 32-bit floating point: eight columns of a row in one
// thread, loaded and stored with 16-byte accesses, computed in fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "moe_internal.h"

namespace moe {
namespace {

// 16 bytes that are read once.  An ordinary load (not the read-only path, which may be moved above the wait for a predecessor).
__device__ __forceinline__ uint4 ld_row_v4(const void *p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_row_v2(const void *p)
{
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_row_u8(const void *p)
{
    uint32_t v;
    asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st_row_v4(void *p, uint4 v)
{
    asm volatile("st.global.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// kVec elements of type E are 16 bytes
template <class E> struct RowType;
template <> struct RowType<__nv_bfloat16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float2 two(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        uint32_t w;
        memcpy(&w, &h, 4);
        return w;
    }
};
template <> struct RowType<__half> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float2 two(uint32_t w)
    {
        __half2 h;
        memcpy(&h, &w, 4);
        return __half22float2(h);
    }
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const __half2 h = __floats2half2_rn(a, b);
        uint32_t w;
        memcpy(&w, &h, 4);
        return w;
    }
};
template <> struct RowType<float> {
    static constexpr int kVec = 4;
};

// the values of 16 bytes
template <class E>
__device__ __forceinline__ void unpack16(uint4 v, float (&x)[RowType<E>::kVec])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else {
            const float2 f = RowType<E>::two(w[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}
template <class E>
__device__ __forceinline__ uint4 pack16(const float (&x)[RowType<E>::kVec])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) w[i] = __float_as_uint(x[i]);
        else w[i] = RowType<E>::pack(x[2 * i], x[2 * i + 1]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// eight columns, whatever the type
template <class E>
__device__ __forceinline__ void load8(const E *p, float (&x)[8])
{
    if constexpr (sizeof(E) == 4) {
        float a[4], b[4];
        unpack16<E>(ld_row_v4(p), a);
        unpack16<E>(ld_row_v4(p + 4), b);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        unpack16<E>(ld_row_v4(p), x);
    }
}
template <class E>
__device__ __forceinline__ void store8(E *p, const float (&x)[8])
{
    if constexpr (sizeof(E) == 4) {
        const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
        st_row_v4(p, pack16<E>(a));
        st_row_v4(p + 4, pack16<E>(b));
    } else {
        st_row_v4(p, pack16<E>(x));
    }
}

// Sixteen columns as they lie in memory.  `wide`: the address is on a 32-byte boundary
template <class E> struct Raw16 {
    static constexpr int kWords = 4 * (int)sizeof(E);
    uint32_t w[kWords];
};
__device__ __forceinline__ void ld_row_v8(const void *p, uint32_t *w)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
template <class E>
__device__ __forceinline__ void load16(const E *p, bool wide, Raw16<E> &r)
{
    if (wide) {
#pragma unroll
        for (int i = 0; i < Raw16<E>::kWords; i += 8) ld_row_v8(reinterpret_cast<const uint32_t *>(p) + i, &r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < Raw16<E>::kWords; i += 4) {
            const uint4 v = ld_row_v4(reinterpret_cast<const uint32_t *>(p) + i);
            r.w[i] = v.x;
            r.w[i + 1] = v.y;
            r.w[i + 2] = v.z;
            r.w[i + 3] = v.w;
        }
    }
}
template <class E>
__device__ __forceinline__ void values16(const Raw16<E> &r, float (&x)[16])
{
#pragma unroll
    for (int i = 0; i < Raw16<E>::kWords; ++i) {
        if constexpr (sizeof(E) == 4) {
            x[i] = __uint_as_float(r.w[i]);
        } else {
            const float2 f = RowType<E>::two(r.w[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}
template <class E>
__device__ __forceinline__ void store16(E *p, bool wide, const float (&x)[16])
{
    uint32_t w[Raw16<E>::kWords];
#pragma unroll
    for (int i = 0; i < Raw16<E>::kWords; ++i) {
        if constexpr (sizeof(E) == 4) w[i] = __float_as_uint(x[i]);
        else w[i] = RowType<E>::pack(x[2 * i], x[2 * i + 1]);
    }
    uint32_t *q = reinterpret_cast<uint32_t *>(p);
#pragma unroll
    for (int i = 0; i < Raw16<E>::kWords; i += 8) {
        if (wide) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q + i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]),
                         "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7]) : "memory");
        } else {
            st_row_v4(q + i, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
            st_row_v4(q + i + 4, make_uint4(w[i + 4], w[i + 5], w[i + 6], w[i + 7]));
        }
    }
}
// The largest magnitude of sixteen values, as the bits of the type without the sign: integers that are ordered as the values are, an
// infinity above the finite ones and what is no number above that.  16-bit types: two values a step.
template <class E>
__device__ __forceinline__ uint32_t magnitude16(const Raw16<E> &r)
{
    if constexpr (sizeof(E) == 4) {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, r.w[i] & 0x7fffffffu);
        return m;
    } else {
        uint32_t m = r.w[0] & 0x7fff7fffu;
#pragma unroll
        for (int i = 1; i < 8; ++i) m = __vmaxu2(m, r.w[i] & 0x7fff7fffu);
        return max(m & 0xffffu, m >> 16);
    }
}
// ... as a float's bits; finite magnitudes only
template <class E> __device__ __forceinline__ uint32_t magnitude_bits(uint32_t m);
template <> __device__ __forceinline__ uint32_t magnitude_bits<float>(uint32_t m) { return m; }
template <> __device__ __forceinline__ uint32_t magnitude_bits<__nv_bfloat16>(uint32_t m) { return m << 16; }
template <> __device__ __forceinline__ uint32_t magnitude_bits<__half>(uint32_t m)
{
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
}
// the magnitudes from here on are an infinity or no number
template <class E> constexpr uint32_t kNotFinite = 0x7f800000u;
template <> constexpr uint32_t kNotFinite<__nv_bfloat16> = 0x7f80u;
template <> constexpr uint32_t kNotFinite<__half> = 0x7c00u;
// 2^e for -127 <= e <= 127 (2^-127 is subnormal)
__device__ __forceinline__ float power_of_two(int e) { return e > -127 ? __uint_as_float((uint32_t)(e + 127) << 23) : __uint_as_float(1u << 22); }

}  // namespace

// the element type of a call -> the kernel's: fn is called with a null pointer of that type
template <class Fn>
inline int32_t with_row_type(int32_t dtype, Fn fn)
{
    switch (dtype) {
        case MOE_BF16: return fn(static_cast<__nv_bfloat16 *>(nullptr));
        case MOE_FP16: return fn(static_cast<__half *>(nullptr));
        case MOE_FP32: return fn(static_cast<float *>(nullptr));
        default: return MOE_ERR_UNSUPPORTED;
    }
}
inline size_t row_type_bytes(int32_t dtype) { return dtype == MOE_FP32 ? 4 : 2; }
inline bool row_type_ok(int32_t dtype) { return dtype == MOE_BF16 || dtype == MOE_FP16 || dtype == MOE_FP32; }
inline bool rows_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// every 16 columns of the matrix on a 32-byte boundary
inline bool rows_wide(const void *p, int64_t ld, int32_t dtype)
{
    return (reinterpret_cast<uintptr_t>(p) & 31u) == 0 && (ld * (int64_t)row_type_bytes(dtype)) % 32 == 0;
}
// distance of two rows, in elements: no overlap, every row on a 16-byte boundary
inline bool pitch_ok(int64_t ld, int64_t cols) { return ld >= cols && ld % 8 == 0 && ld < (int64_t)1 << 29; }

// A launch that may start beside its predecessor's end.  Kernels launched with it wait before they touch global memory.
template <class... Args>
inline cudaError_t launch_chained(void (*kernel)(Args...), unsigned grid, unsigned block, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1] = {chained_launch_attribute()};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace moe
