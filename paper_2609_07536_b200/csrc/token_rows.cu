// Tokens to expert rows and back, and the gradients of both (Section II-A: the gather in front of the expert products and the
// weighted combine behind them, as steps of their own).  With r = inv_perm[t][j], the row of token t's j-th assignment
// (-1: it has none):
//   moe_permute          rows[r]   = tokens[t]
//   moe_permute_grad     d_tokens[t] = sum_j d_rows[r_j]
//   moe_unpermute        out[t]    = sum_j w[t][j] rows[r_j]
//   moe_unpermute_grad   d_rows[r] = w[t][j] d_out[t],   d_w[t][j] = <d_out[t], rows[r]>
// All four move bytes and compute next to nothing: the bound is HBM, R rows read or written once and T token rows once.  So a
// token's columns are read once and stored k_tot times (spread), or k_tot rows are read and one is written (gather), by a
// warp per token and 512 bytes of columns: the assignments of the token sit in its lanes, no division per element, no
// atomics, a fixed order of the sum over j.  Sums are fp32, rounded once.

#include "rows_device.cuh"
#include "sm100_device.cuh"

namespace moe {
namespace {

constexpr int kRowThreads = 128, kRowWarps = kRowThreads / 32;
constexpr int kGradThreads = 64, kGradWarps = kGradThreads / 32;       // the way back's gradient

struct TokenRows {
    const int32_t *inv_perm;
    const float *w;                // [T, k_tot], or nullptr: weights of one
    uint32_t *status;
    long long ld_tokens, ld_rows, ld_d_rows;   // elements
    long long pieces;              // T * parts, less than 2^32 (gradient of the way back: assignments)
    int32_t R, k_tot, vecs;        // 16-byte vectors of a row
    int32_t parts;                 // pieces of 512 bytes of a token's row
};

// The row of assignment `f` (bounds checked: -1 where there is none)
__device__ __forceinline__ int row_of(const TokenRows &p, long long f)
{
    const int r = ld_chained(p.inv_perm + f);
    if (r >= p.R || r < -1) {
        report(p.status, MOE_DEV_OOB, (uint32_t)f, 60u);
        return -1;
    }
    return r;
}

// A warp has one piece: what is in flight are stores, which nothing waits for.  (Blocks that stay, with the next piece loaded ahead as
// in the gather below: 16384 tokens, 8 rows each of 4 KB, 113 us instead of 99; 1 KB a warp and token: 106.)
template <class E>
__global__ void __launch_bounds__(kRowThreads) spread_kernel(const __grid_constant__ TokenRows p, const E *tokens, E *rows)
{
    grid_dependency_wait();
    constexpr int kVec = RowType<E>::kVec;
    const int lane = threadIdx.x & 31;
    for (long long piece = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5); piece < p.pieces; piece += (long long)gridDim.x * kRowWarps) {
        const long long t = piece / p.parts;
        const int v = (int)(piece - t * p.parts) * 32 + lane;
        const int mine = lane < p.k_tot ? row_of(p, t * p.k_tot + lane) : -1;
        const bool live = v < p.vecs;
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (live) x = ld_row_v4(tokens + t * p.ld_tokens + (long long)v * kVec);
        for (int j = 0; j < p.k_tot; ++j) {
            const int r = __shfl_sync(0xffffffffu, mine, j);
            if (live && r >= 0) st_row_v4(rows + (long long)r * p.ld_rows + (long long)v * kVec, x);
        }
    }
}

// kAhead loads in flight a thread.  The blocks stay: a warp looks up the indexes of its next piece while the rows of this one are on their
// way, so that the one latency does not lie in front of the other in every piece (16384 tokens, 8 rows each of 4 KB: 95 us, 98 % of the
// measured copy bandwidth; a block for every eight pieces 107).  Eight loads from five rows a token on: four leave more blocks to an SM, but
// then take two turns.  Four / eight, us, 16384 tokens of 4 KB, 1 / 2 / 4 / 5 / 6 / 8 / 12 rows each: 33.1/47.4  40.1/51.4  54.9/62.2  70.6/69.0
// 78.6/77.1  95.8/95.4  137.2/140.0; 1003 tokens of 3 KB, 4 / 5 / 6 / 8 rows: 4.1/4.1  4.1/4.6  4.8/4.8  6.2/5.5 (five rows of few tokens and twelve
// of many lose 0.5 and 3 us by the rule).
template <class E, bool kWeighted, int kAhead>
__global__ void __launch_bounds__(kRowThreads, kAhead == 8 ? 6 : 8) gather_kernel(const __grid_constant__ TokenRows p, const E *rows, E *tokens)
{
    grid_dependency_wait();
    constexpr int kVec = RowType<E>::kVec;
    const int lane = threadIdx.x & 31;
    const uint32_t stride = gridDim.x * kRowWarps;
    const char *base = reinterpret_cast<const char *>(rows) + lane * 16;
    const uint32_t pitch = (uint32_t)p.ld_rows * (uint32_t)sizeof(E);
    int t, v0, mine;
    float w;
    const auto look_up = [&](uint32_t piece) {
        t = (int)(piece / (uint32_t)p.parts);
        v0 = (int)(piece - (uint32_t)t * (uint32_t)p.parts) * 32;
        mine = -1;
        if (lane < p.k_tot) {
            if (kWeighted) w = ld_chained(p.w + (long long)t * p.k_tot + lane);    // (in front of the index, whose check waits for it)
            mine = row_of(p, (long long)t * p.k_tot + lane);
        }
    };
    uint32_t piece = blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    if (piece < (uint32_t)p.pieces) look_up(piece);
    while (piece < (uint32_t)p.pieces) {
        const int t_now = t, v_now = v0, r_now = mine;
        const float w_now = w;
        const bool live = v_now + lane < p.vecs;
        float acc[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) acc[i] = 0.0f;
        for (int j0 = 0; j0 < p.k_tot; j0 += kAhead) {
            uint4 x[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int r = j0 + a < p.k_tot ? __shfl_sync(0xffffffffu, r_now, j0 + a) : -1;
                if (live && r >= 0) x[a] = ld_row_v4(base + (unsigned long long)(uint32_t)r * pitch + (long long)v_now * 16);
            }
            if (j0 == 0) {
                piece = piece + stride >= piece ? piece + stride : 0xffffffffu;
                if (piece < (uint32_t)p.pieces) look_up(piece);
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                if (j0 + a >= p.k_tot) break;
                const int r = __shfl_sync(0xffffffffu, r_now, j0 + a);
                const float wj = kWeighted ? __shfl_sync(0xffffffffu, w_now, j0 + a) : 1.0f;
                if (r < 0) continue;
                float y[kVec];
                unpack16<E>(x[a], y);
#pragma unroll
                for (int i = 0; i < kVec; ++i) acc[i] = kWeighted ? fmaf(wj, y[i], acc[i]) : acc[i] + y[i];
            }
        }
        if (live) st_row_v4(tokens + t_now * p.ld_tokens + (long long)(v_now + lane) * kVec, pack16<E>(acc));
    }
}

// A warp per assignment, four vectors of both inputs in flight a thread: blocks of two warps start as soon as two others
// are done (16384 tokens, 8 rows each of 4 KB: 174 us at the measured copy bandwidth; eight warps a block 178, one vector at a time 206).
template <class E>
__global__ void __launch_bounds__(kGradThreads) spread_grad_kernel(const __grid_constant__ TokenRows p, const E *d_out, const E *rows, E *d_rows, float *d_w)
{
    grid_dependency_wait();
    constexpr int kVec = RowType<E>::kVec, kAhead = 4;
    const int lane = threadIdx.x & 31;
    for (long long f = (long long)blockIdx.x * kGradWarps + (threadIdx.x >> 5); f < p.pieces; f += (long long)gridDim.x * kGradWarps) {
        const long long t = f / p.k_tot;
        const int r = __shfl_sync(0xffffffffu, lane == 0 ? row_of(p, f) : 0, 0);
        float dot = 0.0f;
        if (r >= 0) {
            const float w = ld_chained(p.w + f);
            for (int v = lane; v - lane < p.vecs; v += 32 * kAhead) {
                uint4 dx[kAhead], yx[kAhead];
#pragma unroll
                for (int a = 0; a < kAhead; ++a)
                    if (v + 32 * a < p.vecs) {
                        yx[a] = ld_row_v4(rows + (long long)r * p.ld_rows + (long long)(v + 32 * a) * kVec);
                        dx[a] = ld_row_v4(d_out + t * p.ld_tokens + (long long)(v + 32 * a) * kVec);
                    }
#pragma unroll
                for (int a = 0; a < kAhead; ++a) {
                    if (v + 32 * a >= p.vecs) continue;
                    float d[kVec], y[kVec];
                    unpack16<E>(dx[a], d);
                    unpack16<E>(yx[a], y);
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        dot = fmaf(d[i], y[i], dot);
                        d[i] *= w;
                    }
                    st_row_v4(d_rows + (long long)r * p.ld_d_rows + (long long)(v + 32 * a) * kVec, pack16<E>(d));
                }
            }
        }
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, m);
        if (lane == 0) d_w[f] = dot;
    }
}

// What the four calls check alike; `done`: nothing to do
int32_t token_rows_args(moe_handle *h, const moe_shape *s, int32_t dtype, const void *tokens, int64_t ld_tokens, const void *rows,
                        int64_t ld_rows, const int32_t *inv_perm, uint32_t *status, TokenRows *p, bool *done)
{
    *done = false;
    if (!h || !s || !status) return MOE_ERR_NULL;
    if (s->T < 0 || s->H < 8 || s->H % 8 != 0 || s->k_tot < 1 || s->k_tot > 32 || (int64_t)s->T * s->k_tot >= (int64_t)1 << 30) return MOE_ERR_SHAPE;
    if (!row_type_ok(dtype)) return MOE_ERR_UNSUPPORTED;
    if (!pitch_ok(ld_tokens, s->H) || !pitch_ok(ld_rows, s->H)) return MOE_ERR_SHAPE;
    if (s->T == 0) {
        *done = true;
        return MOE_OK;
    }
    if (!tokens || !rows || !inv_perm) return MOE_ERR_NULL;
    if (!rows_aligned(tokens) || !rows_aligned(rows) || !rows_aligned(status)) return MOE_ERR_ALIGN;
    p->inv_perm = inv_perm;
    p->w = nullptr;
    p->status = status;
    p->ld_tokens = ld_tokens;
    p->ld_rows = p->ld_d_rows = ld_rows;
    p->R = s->T * s->k_tot;
    p->k_tot = s->k_tot;
    p->vecs = (int32_t)((int64_t)s->H * (int64_t)row_type_bytes(dtype) / 16);
    p->parts = (p->vecs + 31) / 32;
    p->pieces = (int64_t)s->T * p->parts;
    if (p->pieces >= (int64_t)1 << 32) return MOE_ERR_SHAPE;
    return MOE_OK;
}
unsigned row_grid(const TokenRows &p, int warps = kRowWarps)
{
    const long long blocks = (p.pieces + warps - 1) / warps;
    return (unsigned)(blocks < (1ll << 30) ? blocks : 1ll << 30);
}

// as many blocks as the SMs hold at once (`held` each), or as there are pieces for
unsigned staying_grid(const moe_handle *h, const TokenRows &p, unsigned held)
{
    const unsigned all = row_grid(p), most = (unsigned)h->G * held;
    return all < most ? all : most;
}

template <class E>
E *typed(void *p) { return static_cast<E *>(p); }
template <class E>
const E *typed(const void *p) { return static_cast<const E *>(p); }

}  // namespace
}  // namespace moe

using namespace moe;

extern "C" int32_t moe_permute(moe_handle *h, const void *tokens, int64_t ld_tokens, const int32_t *inv_perm, const moe_shape *s,
                               int32_t dtype, void *rows, int64_t ld_rows, uint32_t *status_dev, void *stream)
{
    TokenRows p;
    bool done;
    int32_t rc = token_rows_args(h, s, dtype, tokens, ld_tokens, rows, ld_rows, inv_perm, status_dev, &p, &done);
    if (rc != MOE_OK || done) return rc;
    if ((rc = require_handle_device(h, "moe_permute")) != MOE_OK) return rc;
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const cudaError_t err = launch_chained(spread_kernel<E>, row_grid(p), kRowThreads, 0, static_cast<cudaStream_t>(stream), p, typed<E>(tokens), typed<E>(rows));
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "permute launch");
    });
}

extern "C" int32_t moe_permute_grad(moe_handle *h, const void *d_rows, int64_t ld_rows, const int32_t *inv_perm, const moe_shape *s,
                                    int32_t dtype, void *d_tokens, int64_t ld_tokens, uint32_t *status_dev, void *stream)
{
    TokenRows p;
    bool done;
    int32_t rc = token_rows_args(h, s, dtype, d_tokens, ld_tokens, d_rows, ld_rows, inv_perm, status_dev, &p, &done);
    if (rc != MOE_OK || done) return rc;
    if ((rc = require_handle_device(h, "moe_permute_grad")) != MOE_OK) return rc;
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const cudaError_t err = launch_chained(p.k_tot > 4 ? gather_kernel<E, false, 8> : gather_kernel<E, false, 4>, staying_grid(h, p, p.k_tot > 4 ? 6 : 8), kRowThreads, 0, static_cast<cudaStream_t>(stream), p, typed<E>(d_rows), typed<E>(d_tokens));
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "permute gradient launch");
    });
}

extern "C" int32_t moe_unpermute(moe_handle *h, const void *rows, int64_t ld_rows, const int32_t *inv_perm, const float *topk_w,
                                 const moe_shape *s, int32_t dtype, void *out, int64_t ld_out, uint32_t *status_dev, void *stream)
{
    TokenRows p;
    bool done;
    int32_t rc = token_rows_args(h, s, dtype, out, ld_out, rows, ld_rows, inv_perm, status_dev, &p, &done);
    if (rc != MOE_OK || done) return rc;
    if (!topk_w) return MOE_ERR_NULL;
    p.w = topk_w;
    if ((rc = require_handle_device(h, "moe_unpermute")) != MOE_OK) return rc;
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const cudaError_t err = launch_chained(p.k_tot > 4 ? gather_kernel<E, true, 8> : gather_kernel<E, true, 4>, staying_grid(h, p, p.k_tot > 4 ? 6 : 8), kRowThreads, 0, static_cast<cudaStream_t>(stream), p, typed<E>(rows), typed<E>(out));
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "unpermute launch");
    });
}

extern "C" int32_t moe_unpermute_grad(moe_handle *h, const void *d_out, int64_t ld_out, const void *rows, int64_t ld_rows, const int32_t *inv_perm,
                                      const float *topk_w, const moe_shape *s, int32_t dtype, void *d_rows, int64_t ld_d_rows, float *d_topk_w,
                                      uint32_t *status_dev, void *stream)
{
    TokenRows p;
    bool done;
    int32_t rc = token_rows_args(h, s, dtype, d_out, ld_out, rows, ld_rows, inv_perm, status_dev, &p, &done);
    if (rc != MOE_OK || done) return rc;
    if (!topk_w || !d_rows || !d_topk_w) return MOE_ERR_NULL;
    if (!pitch_ok(ld_d_rows, s->H)) return MOE_ERR_SHAPE;
    if (!rows_aligned(d_rows)) return MOE_ERR_ALIGN;
    p.w = topk_w;
    p.ld_d_rows = ld_d_rows;
    p.pieces = p.R;
    if ((rc = require_handle_device(h, "moe_unpermute_grad")) != MOE_OK) return rc;
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const cudaError_t err = launch_chained(spread_grad_kernel<E>, row_grid(p, kGradWarps), kGradThreads, 0, static_cast<cudaStream_t>(stream), p, typed<E>(d_out), typed<E>(rows), typed<E>(d_rows), d_topk_w);
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "unpermute gradient launch");
    });
}
