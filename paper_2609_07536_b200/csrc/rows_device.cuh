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
__device__ __forceinline__ uint32_t ld_row_u32(const void *p)
{
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
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

// the largest finite magnitude of eight values; `bad`: bit i, value i is an infinity or no number
__device__ __forceinline__ float finite_amax8(const float (&x)[8], uint32_t &bad)
{
    float m = 0.0f;
    bad = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(x[i]);
        if (a <= 3.402823466e38f) m = fmaxf(m, a);
        else bad |= 1u << i;
    }
    return m;
}
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
// distance of two rows, in elements: no overlap, every row on a 16-byte boundary
inline bool pitch_ok(int64_t ld, int64_t cols) { return ld >= cols && ld % 8 == 0 && ld < (int64_t)1 << 40; }

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
