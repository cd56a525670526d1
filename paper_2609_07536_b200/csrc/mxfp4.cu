// Microscaled 4-bit floating point for the expert products: quantisation, its inverse, and the grouped product of routed rows
// and expert weights that are both held in it.
//
// Format: a value is an e2m1 code (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign) times 2^(e - 127), with one exponent byte e for 32 consecutive
// columns: e - 127 = floor(log2(amax)) - 2, clamped to [-127, 127]; codes are rounded to the nearest, ties to even, and saturate at
// 6.  A block with an infinity or no number gets e = 255, the code for no number, as a whole.
// Codes lie [rows, K / 2], the even column in the low half of its byte.  Exponents lie as the tensor cores take them: blocks of
// 128 rows x 128 columns are 512 bytes, row i, columns 32 s.. at 16 (i % 32) + 4 (i / 32) + s, so that the product copies them
// from global memory through shared memory into TMEM as they are.  Rows come in groups (experts); row r of the group g whose rows
// begin at o lies in row block o / 128 + g + (r - o) / 128: the blocks of two groups never meet, and no prefix over the groups is
// needed to find them.

#include <cuda_fp4.h>

#include <cstring>

#include "rows_device.cuh"
#include "sm100_device.cuh"

namespace moe {
namespace {

constexpr int kMxBlock = 32;           // columns that share an exponent
constexpr int kMxTile = 128;           // rows and columns of an exponent block
constexpr int kMxTileBytes = 512;

// --------------------------------------------------------------------------- quantisation and back

constexpr int kQuantThreads = 256;
constexpr int kQuantRowsMax = 16, kQuantTokensMax = 2, kQuantEntriesMax = kQuantTokensMax * 32;   // source rows of a block; rows they go to
static_assert(kQuantEntriesMax >= kQuantRowsMax, "a place for every row of a block");

struct Quant {
    const int32_t *offsets;        // [groups + 1], or nullptr: groups of n_even rows each
    const int32_t *inv_perm;       // [src_rows, copies], or nullptr: row r from source row r
    uint32_t *status;
    uint8_t *codes, *scales;
    long long ld, blocks;          // elements of the 16- or 32-bit matrix; row blocks of the exponents
    int32_t rows, src_rows, copies, groups, n_even;
    int32_t K, KQ, lanes, rows_per_cta;   // KQ = ceil(K / 128); lanes: threads of a row, 8 per 128 columns
    int32_t wide;                  // 16 columns of the 16- or 32-bit matrix are on 32-byte boundaries
    Divisor by_lanes, by_n;
};
struct QuantRow {
    uint8_t *codes, *scales;       // the row's codes (nullptr: it has no place), its first exponent byte
};
// the groups' offsets in shared memory, up to this many (more are looked up where they are)
constexpr int kQuantGroupsHeld = 1024;
__device__ __forceinline__ void hold_offsets(const Quant &p, int32_t *held)
{
    if (p.offsets && p.groups <= kQuantGroupsHeld)
        for (int g = threadIdx.x; g <= p.groups; g += kQuantThreads) held[g] = ld_chained(p.offsets + g);
}
// 0 <= begin <= end <= rows
__device__ __forceinline__ bool ordered(const Quant &p, int begin, int end) { return (uint32_t)begin <= (uint32_t)end && (uint32_t)end <= (uint32_t)p.rows; }
// All threads meet here; false: offsets that are not in order, or more than are held.  The last threads look them over, while the first
// ones find their rows.
__device__ __forceinline__ bool meet_with_offsets_ordered(const Quant &p, const int32_t *held)
{
    if (!p.offsets) {
        __syncthreads();
        return true;
    }
    bool fine = p.groups <= kQuantGroupsHeld;
    if (fine)
        for (int g = kQuantThreads - 1 - (int)threadIdx.x; g < p.groups; g += kQuantThreads) fine = fine && ordered(p, held[g], held[g + 1]);
    return __syncthreads_and(fine) != 0;
}

// Row `r` of group `g`, whose rows begin at `o`
__device__ __forceinline__ QuantRow row_in_group(const Quant &p, int r, int g, int o, uint32_t what)
{
    QuantRow q = {nullptr, nullptr};
    const int i = r - o;
    const long long block = (long long)(o / kMxTile) + g + i / kMxTile;
    if (o < 0 || i < 0 || block >= p.blocks) {
        report(p.status, MOE_DEV_OOB, what, 62u);
        return q;
    }
    q.codes = p.codes + (long long)r * (p.K / 2);
    q.scales = p.scales + block * p.KQ * kMxTileBytes + (i & 31) * 16 + ((i & 127) >> 5) * 4;
    return q;
}
// the last group that begins at or before r: the one with rows among equals
template <class Offset>
__device__ __forceinline__ int bisect(const Quant &p, int r, Offset offset)
{
    int lo = 0, hi = p.groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (offset(mid) <= r) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
// Where row `r` lies, by offsets that are held and in order (of others, it has a place found again below); rows behind the last group have no place
__device__ __forceinline__ QuantRow quant_row(const Quant &p, const int32_t *held, int r, uint32_t what)
{
    int g, o;
    if (p.offsets) {
        if (r < 0 || p.groups > kQuantGroupsHeld || r >= held[p.groups]) return {nullptr, nullptr};
        g = bisect(p, r, [&](int i) { return held[i]; });
        o = held[g];
    } else {
        if (r < 0) return {nullptr, nullptr};
        g = quotient(p.by_n, r);
        o = g * p.n_even;
    }
    return row_in_group(p, r, g, o, what);
}
// Where the rows of a block lie (row0: the first of the source; gather: by inv_perm) by offsets that are not in order, or more than are held.
// A group has rows where its two offsets are in order and it begins behind the rows of all such groups before it, as in the product.  Of
// more than are held, a row has the group that the bisection finds, where that and the offset before it are in order; the blocks look the
// offsets over together.  Out of line, and the caller loads its columns again: inlined, or with them kept across the call, it took
// registers that cost weights 5 of 70 us.
__device__ __noinline__ void find_places_again(const Quant &p, const int32_t *held, QuantRow *where, int row0, int n, bool gather)
{
    const bool all = p.groups <= kQuantGroupsHeld;
    const auto offset = [&](int i) { return all ? held[i] : ld_chained(p.offsets + i); };
    if (!all || blockIdx.x == 0)
        for (long long g = (long long)blockIdx.x * kQuantThreads + threadIdx.x; g < p.groups; g += (all ? 1ll : (long long)gridDim.x) * kQuantThreads)
            if (!ordered(p, offset((int)g), offset((int)g + 1))) report(p.status, MOE_DEV_OOB, (uint32_t)g, 63u);
    for (int k = threadIdx.x; k < n; k += kQuantThreads) {
        const long long f = (long long)row0 * (gather ? p.copies : 1) + k;
        const int r = gather ? ld_chained(p.inv_perm + f) : (int)f;
        int found = -1;
        if (!all && r >= 0 && r < p.rows) {
            const int g = bisect(p, r, offset);
            if (ordered(p, offset(g), offset(g + 1)) && r < offset(g + 1) && (g == 0 || offset(g - 1) <= offset(g))) found = g;
        }
        for (int g = 0, top = 0; all && g < p.groups; ++g) {
            if (!ordered(p, held[g], held[g + 1])) continue;
            if (held[g] >= top && held[g] <= r && r < held[g + 1]) found = g;
            top = max(top, held[g + 1]);
        }
        QuantRow q = {nullptr, nullptr};
        if (found >= 0) q = row_in_group(p, r, found, offset(found), (uint32_t)f);
        where[k] = q;
    }
    __syncthreads();
}

// e2m1 codes of eight values times `inv`, the first in the lowest four bits
__device__ __forceinline__ uint32_t e2m1_codes(const float *x, float inv)
{
    uint32_t w = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(x[2 * i] * inv, x[2 * i + 1] * inv), __NV_E2M1, cudaRoundNearest) << (8 * i);
    return w;
}

// A thread has 16 columns, two threads share an exponent, eight write the four exponents of 128 columns as one word.  Besides the
// bytes, the issue of instructions costs: with 8 columns a thread, and magnitudes found in fp32 one by one, weights of 60 x 2048 x 1408
// took 126 us, now 71 (6.2 TB/s).  A block's first columns, its rows' numbers and the groups' offsets are fetched side by side: one
// behind the other they were most of what a small batch took, and of tokens into routed order, whose blocks are many and short (16384
// tokens, 8 rows each: 52 us, now 43, of which the codes are 15, the exponents' scattered words 9).
template <class E, bool kGather>
__global__ void __launch_bounds__(kQuantThreads, sizeof(E) == 2 ? 8 : 6) quantize_kernel(const __grid_constant__ Quant p, const E *src)
{
    __shared__ QuantRow where[kQuantEntriesMax];
    __shared__ int32_t held[kQuantGroupsHeld + 1];
    grid_dependency_wait();
    const int row0 = (int)blockIdx.x * p.rows_per_cta, n = min(p.rows_per_cta, p.src_rows - row0), items = n * p.lanes, tid = (int)threadIdx.x;
    // this thread's item `it`: row it / lanes, columns 16 (it % lanes) ..
    Raw16<E> raw = {};
    int i = quotient(p.by_lanes, tid), q = tid - i * p.lanes;
    const auto fetch = [&](int it) {
        i = quotient(p.by_lanes, it);
        q = it - i * p.lanes;
        raw = {};
        if (it < items && q * 16 < p.K) load16<E>(src + (long long)(row0 + i) * p.ld + q * 16, p.wide, raw);
    };
    int r = kGather ? -1 : row0 + tid;
    if (kGather && tid < n * p.copies) r = ld_chained(p.inv_perm + (long long)row0 * p.copies + tid);
    fetch(tid);
    hold_offsets(p, held);
    __syncthreads();
    for (int k = tid; k < n * p.copies; k += kQuantThreads) {
        const long long f = (long long)row0 * p.copies + k;
        if (kGather) {
            if (k != tid) r = ld_chained(p.inv_perm + f);
            if (r < -1 || r >= p.rows) {
                report(p.status, MOE_DEV_OOB, (uint32_t)f, 61u);
                r = -1;
            }
        }
        where[k] = quant_row(p, held, r, (uint32_t)f);
    }
    if (!meet_with_offsets_ordered(p, held)) {
        find_places_again(p, held, where, row0, n * p.copies, kGather);
        fetch(tid);
    }
    for (int base = tid & ~31; base < items; base += kQuantThreads) {
        const int it = base + (tid & 31);
        if (base >= kQuantThreads) fetch(it);
        const bool in = it < items, live = in && q * 16 < p.K;
        uint32_t m = magnitude16<E>(raw);
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        // floor(log2(amax)) - 2, biased: the exponent field less 2; 255: no number
        const bool none = m >= kNotFinite<E>;
        const int e = none ? 255 : max(0, (int)(magnitude_bits<E>(m) >> 23) - 2);
        float x[16];
        values16<E>(raw, x);
        const float inv = power_of_two(127 - e);
        uint2 codes = make_uint2(e2m1_codes(x, inv), e2m1_codes(x + 8, inv));
        if (none) codes = make_uint2(0u, 0u);
        uint32_t bytes = live ? (uint32_t)e << (8 * ((q >> 1) & 3)) : 0u;
#pragma unroll
        for (int d = 2; d < 8; d *= 2) bytes |= __shfl_xor_sync(0xffffffffu, bytes, d);
        if (!in) continue;
        for (int j = 0; j < (kGather ? p.copies : 1); ++j) {
            const QuantRow w = where[kGather ? i * p.copies + j : i];
            if (!w.codes) continue;
            if (live) *reinterpret_cast<uint2 *>(w.codes + q * 8) = codes;
            if ((q & 7) == 0) *reinterpret_cast<uint32_t *>(w.scales + (q >> 3) * kMxTileBytes) = bytes;
        }
    }
}

template <class E>
__global__ void __launch_bounds__(kQuantThreads) dequantize_kernel(const __grid_constant__ Quant p, E *dst)
{
    __shared__ QuantRow where[kQuantRowsMax];
    __shared__ int32_t held[kQuantGroupsHeld + 1];
    grid_dependency_wait();
    const int row0 = (int)blockIdx.x * p.rows_per_cta, n = min(p.rows_per_cta, p.rows - row0);
    hold_offsets(p, held);
    __syncthreads();
    if ((int)threadIdx.x < n) where[threadIdx.x] = quant_row(p, held, row0 + (int)threadIdx.x, (uint32_t)(row0 + (int)threadIdx.x));
    if (!meet_with_offsets_ordered(p, held)) find_places_again(p, held, where, row0, n, false);
    const int items = n * p.lanes;
    for (int it = (int)threadIdx.x; it < items; it += kQuantThreads) {
        const int i = quotient(p.by_lanes, it), q = it - i * p.lanes;
        const QuantRow w = where[i];
        if (!w.codes || q * 16 >= p.K) continue;
        const uint2 c = ld_row_v2(w.codes + q * 8);
        const int e = (int)ld_row_u8(w.scales + (q >> 3) * kMxTileBytes + ((q >> 1) & 3));
        const float scale = e == 255 ? __uint_as_float(0x7fffffffu) : power_of_two(e - 127);
        float x[16];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)((k < 4 ? c.x : c.y) >> (8 * (k & 3))), __NV_E2M1);
            const float2 f = __half22float2(__half2(h));
            x[2 * k] = f.x * scale;
            x[2 * k + 1] = f.y * scale;
        }
        store16<E>(dst + (long long)(row0 + i) * p.ld + q * 16, p.wide, x);
    }
}

// --------------------------------------------------------------------------- grouped product
//
// out[r][n] = sum_k x[r][k] w[e][n][k] for the rows r of expert e, fp32 accumulation in TMEM, one rounding at the end.
// The weights are on the M side of the MMA and the rows on its N side, as in the other products here: a tile costs what its rows cost.
// Tile: 128 columns of the output x up to 192 rows, or, computed by a pair of CTAs (cta_group::2), 256 columns x up to 192 rows: each CTA
// then loads its own 128 rows of the weights and half of the rows of x, 31 KB a stage instead of 43 for the same products.  Where experts
// have few rows: 128 columns x up to 64 rows, in eight stages instead of five.
// TMEM holds two accumulators of 192 columns and, for five stages, 24 columns of exponents (128 rows of weights: 4 per 128
// columns of K; 256 rows of x: 8; a pair's CTAs each have those of all rows of x); that is 504 of its 512 columns, and why a tile has
// 192 rows and not 256.  A stage is 256 columns of K: 128 bytes of codes a row, a swizzle row.
//   warps 0, 2, 3, 12  loaders: codes of the weights, of the rows, and the exponents of both as they lie;
//   warp 1      copies the exponents to TMEM (tcgen05.cp, each of the four lane quarters gets them) and issues
//               tcgen05.mma.kind::mxf4.block_scale (K = 64, two exponents a row); both are issued by one lane of the converged
//               warp (pair: of the first CTA) and run in order;
//   warps 4-11  epilogue: pieces of 32 rows x 32 columns, 16-bit, transposed in registers, 64 contiguous bytes a row; a pair's, where all
//               32 rows are the tile's: two warps put 64 columns together in shared memory, which leave as whole lines by a tiled copy
//               (131072 rows, N 2816, K 2048: 407 -> 386 us at the power limit; half lines straight from registers cost 80 of 407).
// What bounds a large product: shared memory.  In a stage of a pair the MMAs read 40 KB (4 KB of weights and 6 KB of rows each), the copies
// write 31, results pass through with 12: 83 KB at 128 bytes a cycle are 650 cycles, where the MMAs alone take 400.  131072 rows, N 2816,
// K 2048: MMAs alone 185 us, copies of the weights and of the rows +45 each, results +65: 342 us, 4.4 PFLOP/s; 386 us at the 1000 W limit,
// where clocks fall to 1.6 GHz.  With few rows an expert it is HBM: 85 to 90 % of the measured copy bandwidth.

constexpr int kPrThreads = 416, kPrEpiWarps = 8;
constexpr int kPrN = 128;                                   // output columns of a CTA's part of a tile (M of the MMA: a pair's twice that)
constexpr int kPrK = 256, kPrStepK = 64;                    // columns of K of a stage, of an MMA
constexpr int kPrWBytes = kPrN * kPrK / 2;
constexpr int kPrWScaleBytes = 2 * kMxTileBytes, kPrXScaleBytes = 4 * kMxTileBytes;      // x: row block 0 of both 128s of K, then row block 1
constexpr int kPrScaleCols = 24;                            // TMEM columns of a stage's exponents: weights 2 x 4, rows 2 x 8
constexpr int kPrTmemCols = 512;
constexpr int kPrMaxStages = 8;
constexpr int kMaxExperts = 1024;
// results on their way out: 32 rows x 64 columns, two of them for every two epilogue warps
constexpr int kPrOutRows = 32, kPrOutCols = 64, kPrOutBytes = kPrOutRows * kPrOutCols * 2, kPrOutUnits = kPrEpiWarps / 2;
// Families of tiles: one CTA; a pair; one CTA where an expert has few rows: 64 rows of x at most leave shared memory and TMEM for eight
// stages, and it is bytes in flight that a product of few rows lives on
enum { kOneTiles, kPairTiles, kFewTiles };
template <int kKind>
struct PrCfg {
    static constexpr bool kPair = kKind == kPairTiles, kFew = kKind == kFewTiles;
    static constexpr int kTileN = kPair ? 2 * kPrN : kPrN;
    static constexpr int kRows = kFew ? 64 : 192;                                        // rows of a tile (N of the MMA)
    static constexpr int kXRows = kPair ? kRows / 2 : kRows;                             // rows of x that a CTA holds
    static constexpr int kXBytes = kXRows * kPrK / 2;
    static constexpr int kXsBytes = kFew ? kPrXScaleBytes / 2 : kPrXScaleBytes;          // what comes of the exponents: 64 rows lie in one row block
    static constexpr int kStageBytes = kPrWBytes + kXBytes + kPrWScaleBytes + kPrXScaleBytes;
    static constexpr int kStages = kFew ? kPrMaxStages : 5;
    static constexpr int kOutBytes = kPair ? kPrOutUnits * 2 * kPrOutBytes : 0;
    static constexpr int kRound = kPair ? 32 : 16;                                       // N of the MMA is a multiple of this
    static_assert(kStageBytes % 1024 == 0, "stages are 1024-byte aligned");
    static_assert(2 * kRows + kStages * kPrScaleCols <= kPrTmemCols, "accumulators and exponents exceed TMEM");
};

struct alignas(64) ProductParams {
    CUtensorMap tmW;               // codes [E][N][K / 2]   box 128 bytes x 128 rows, 128B swizzle
    CUtensorMap tmX[3];            // codes [R][K / 2]      box 128 bytes x 192, 64, 16 rows (pair: 96, 32; few rows: 64, 16)
    CUtensorMap tmOut;             // (pair) out [R][N]     box 64 columns x 32 rows, 128B swizzle
    CUtensorMap tmWs, tmXs;        // exponents [row blocks][KQ][512 bytes]   box 1 (x: 2; few rows: 1) row blocks x 2 x 512 bytes
    const int32_t *offsets;        // [E + 1]
    void *out;
    long long ld_out;              // elements
    uint32_t *status;
    unsigned long long wait_ns;
    int32_t R, E, N, KQ, num_kb, last_steps, NT;
    Divisor by_NT;
};
struct ProductControl {
    unsigned long long full[kPrMaxStages], empty[kPrMaxStages], tmem_full[2], tmem_empty[2], drain;
    uint32_t tmem_base;
    volatile uint32_t abort;
    int32_t warp_tiles[kPrThreads / 32];
    int32_t first[kMaxExperts + 1];       // the offsets, as they are
    int32_t tiles[kMaxExperts + 1];       // row tiles of the experts before
};

__device__ __forceinline__ bool pr_wait(uint32_t bar, uint32_t parity, ProductControl *ctl, unsigned long long deadline, uint32_t *status,
                                        uint32_t detail, uint32_t where)
{
    if (mbar_test_wait(bar, parity)) return true;
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++spins & 63u) == 0u) {
            if (ctl->abort) return false;
            if (globaltimer_ns() > deadline) {
                ctl->abort = 1u;
                report(status, MOE_DEV_TIMEOUT, detail, where);
                return false;
            }
        }
    }
    return true;
}

// The tiles of a CTA (of a pair): row tile outer, column tile inner, dealt one by one.  The expert is found by a vote of the warp for the first
// tile and by steps from there on (found by bisection for every tile, and the addresses worked out from nothing, a tile's start cost
// 1500 cycles in every role, of 9000 that a tile of 2048 columns took).
struct ProductTile {
    int e, row0, valid, local, n0;     // local: first row inside the expert
};
template <int kKind>
struct ProductWalk {
    static constexpr bool kPair = kKind == kPairTiles;
    int g, e;
    // (the whole warp)
    __device__ __forceinline__ ProductWalk(const ProductParams &P, const ProductControl *ctl) : g((int)blockIdx.x >> (kPair ? 1 : 0)), e(-1)
    {
        const int mu = quotient(P.by_NT, g), lane = threadIdx.x & 31;
        for (int i = 0; i < P.E; i += 32) e += __popc(__ballot_sync(0xffffffffu, i + lane < P.E && ctl->tiles[i + lane] <= mu));
    }
    __device__ __forceinline__ void next() { g += (int)gridDim.x >> (kPair ? 1 : 0); }
    __device__ __forceinline__ ProductTile tile(const ProductParams &P, const ProductControl *ctl)
    {
        const int mu = quotient(P.by_NT, g);
        while (ctl->tiles[e + 1] <= mu) ++e;       // (g is a tile that there is)
        ProductTile t;
        t.e = e;
        t.local = (mu - ctl->tiles[e]) * PrCfg<kKind>::kRows;
        t.row0 = ctl->first[e] + t.local;
        t.valid = min(PrCfg<kKind>::kRows, ctl->first[e + 1] - t.row0);
        t.n0 = (g - mu * P.NT) * PrCfg<kKind>::kTileN;
        return t;
    }
};

// Instruction descriptor, kind::mxf4: e2m1 operands, K-major, M x N, exponents of type ue8m0, exponent pair `half` of the column's four bytes
__device__ __forceinline__ uint32_t mxf4_idesc(uint32_t m, uint32_t n, uint32_t half)
{
    return (2u * half << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((m >> 4) << 24) | (2u * half << 29);
}
// Exponents, shared memory -> TMEM: 512 contiguous bytes are 32 rows of 16, which become 32 lanes x 4 columns in each of the four lane
// quarters.  Descriptor: no swizzle, eights of rows 128 bytes apart (stride offset), version 1; its low word is smem_desc_lo's.
constexpr uint32_t kScaleDescHi = (128u >> 4) | (1u << 14);
// One stage of operands in one statement: the exponents' copies (`two`: two row blocks of x), the MMAs and the commit that hands the
// stage back, to both CTAs of a pair.  All of them are issued by one thread and run in order.  First the exponents of the first 128
// columns, then of the second; 64 columns of codes are 32 bytes further along the swizzle row.  AT1, AT2, AT3, T2: predicates
// of the last stage, which may have fewer than four MMAs.
#define MOE_MXF4_STAGE(GROUP, AT1, AT2, AT3, T2, COMMIT) \
    asm volatile( \
        "{\n\t.reg .pred p, q, t, t1, s1, s2, s3;\n\t.reg .b64 da, db;\n\t.reg .b32 al, bl, sa, sb, sc;\n\t" \
        "setp.ne.b32 p, %11, 0;\n\t" \
        "setp.eq.b32 q, %11, %11;\n\t" \
        "setp.ne.b32 t, %8, 0;\n\t" \
        "setp.gt.u32 s1, %12, 1;\n\t" \
        "setp.gt.u32 s2, %12, 2;\n\t" \
        "setp.gt.u32 s3, %12, 3;\n\t" \
        "and.pred t1, t, s2;\n\t" \
        "add.u32 sa, %5, 4;\n\t" \
        "add.u32 sb, %6, %7;\n\t" \
        "add.u32 sc, sb, 8;\n\t" \
        "mov.b64 da, {%3, %15};\n\t" \
        "tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [%5], da;\n\t" \
        "mov.b64 da, {%4, %15};\n\t" \
        "tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [%6], da;\n\t" \
        "add.u32 al, %4, 64;\n\tadd.u32 bl, %6, 4;\n\t" \
        "mov.b64 da, {al, %15};\n\t" \
        "@t tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [bl], da;\n\t" \
        "add.u32 al, %3, 32;\n\t" \
        "mov.b64 da, {al, %15};\n\t" \
        AT2 "tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [sa], da;\n\t" \
        "add.u32 al, %4, 32;\n\tadd.u32 bl, %6, 8;\n\t" \
        "mov.b64 da, {al, %15};\n\t" \
        AT2 "tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [bl], da;\n\t" \
        "add.u32 al, %4, 96;\n\tadd.u32 bl, %6, 12;\n\t" \
        "mov.b64 da, {al, %15};\n\t" \
        T2 "tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [bl], da;\n\t" \
        "mov.b64 da, {%1, %14};\n\tmov.b64 db, {%2, %14};\n\t" \
        "tcgen05.mma.cta_group::" GROUP ".kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %9, [%5], [sb], p;\n\t" \
        "add.u32 al, %1, 2;\n\tadd.u32 bl, %2, 2;\n\t" \
        "mov.b64 da, {al, %14};\n\tmov.b64 db, {bl, %14};\n\t" \
        AT1 "tcgen05.mma.cta_group::" GROUP ".kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %10, [%5], [sb], q;\n\t" \
        "add.u32 al, %1, 4;\n\tadd.u32 bl, %2, 4;\n\t" \
        "mov.b64 da, {al, %14};\n\tmov.b64 db, {bl, %14};\n\t" \
        AT2 "tcgen05.mma.cta_group::" GROUP ".kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %9, [sa], [sc], q;\n\t" \
        "add.u32 al, %1, 6;\n\tadd.u32 bl, %2, 6;\n\t" \
        "mov.b64 da, {al, %14};\n\tmov.b64 db, {bl, %14};\n\t" \
        AT3 "tcgen05.mma.cta_group::" GROUP ".kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %10, [sa], [sc], q;\n\t" \
        COMMIT "\n\t}" \
        ::"r"(d_tmem), "r"(w_lo), "r"(x_lo), "r"(ws_lo), "r"(xs_lo), "r"(sw), "r"(sx), "r"(shift), "r"(two), "r"(idesc0), "r"(idesc1), "r"(accumulate), \
        "r"(steps), "r"(empty_bar), "r"(kSmemDescHi), "r"(kScaleDescHi), "h"((uint16_t)3) \
        : "memory")
#define MOE_COMMIT_PAIR "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%13], %16;"
#define MOE_COMMIT_ONE "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%13];"
template <bool kPair, bool kWhole>
__device__ __forceinline__ void tc_stage_mxf4(uint32_t d_tmem, uint32_t w_lo, uint32_t x_lo, uint32_t ws_lo, uint32_t xs_lo, uint32_t sw, uint32_t sx,
                                              uint32_t shift, uint32_t two, uint32_t idesc0, uint32_t idesc1, uint32_t accumulate, uint32_t steps,
                                              uint32_t empty_bar)
{
    if constexpr (kPair && kWhole) MOE_MXF4_STAGE("2", "", "", "", "@t ", MOE_COMMIT_PAIR);
    else if constexpr (kPair) MOE_MXF4_STAGE("2", "@s1 ", "@s2 ", "@s3 ", "@t1 ", MOE_COMMIT_PAIR);
    else if constexpr (kWhole) MOE_MXF4_STAGE("1", "", "", "", "@t ", MOE_COMMIT_ONE);
    else MOE_MXF4_STAGE("1", "@s1 ", "@s2 ", "@s3 ", "@t1 ", MOE_COMMIT_ONE);
}
#undef MOE_MXF4_STAGE
#undef MOE_COMMIT_PAIR
#undef MOE_COMMIT_ONE
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"((unsigned long long)map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// 32 rows x 32 columns of an accumulator -> 16 bits, one store instruction 64 contiguous bytes of eight rows.  `dst`: lane i, where the
// first of the columns of row i goes (nullptr: nowhere); `cols`: columns that exist (a multiple of 8)
template <class E>
__device__ __forceinline__ void store_piece(const uint32_t (&lo)[16], const uint32_t (&hi)[16], E *dst, int cols)
{
    const int lane = threadIdx.x & 31, c = lane & 3;
    const auto pack = [](uint32_t a, uint32_t b) { return RowType<E>::pack(__uint_as_float(a), __uint_as_float(b)); };
#pragma unroll
    for (int j = 0; j < 4; ++j) {                // rows 8j..8j+7; this lane: row 8j + lane / 4
        uint32_t v[4] = {transpose_8x8(pack(lo[4 * j], lo[4 * j + 1])), transpose_8x8(pack(lo[4 * j + 2], lo[4 * j + 3])),
                         transpose_8x8(pack(hi[4 * j], hi[4 * j + 1])), transpose_8x8(pack(hi[4 * j + 2], hi[4 * j + 3]))};
        // v[m]: columns 8m + 2c and the next one -> v[k]: columns 8c + 2k and the next one
#pragma unroll
        for (int d = 1; d < 4; d *= 2)
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                if (m & d) continue;
                const bool up = (c & d) != 0;
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? v[m] : v[m + d], d);
                if (up) v[m] = got;
                else v[m + d] = got;
            }
        E *row = reinterpret_cast<E *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), 8 * j + (lane >> 2)));
        if (row != nullptr && c * 8 < cols) st_row_v4(row + c * 8, make_uint4(v[0], v[1], v[2], v[3]));
    }
}

// A loader: one copy a stage, codes of the weights or of the rows, or the exponents of either.  The warp runs the loop converged and one
// elected lane issues, as in the loop that issues the MMAs; operands advance by additions, the next stage's barrier is looked at early.  (One
// thread, addresses worked out from the stage's number: 500 cycles a stage and copy, two copies 750, where the MMAs of a full stage
// take 400; an untiled copy takes longer than a tiled one.)  Pair: every copy completes on the first CTA's barrier, at the same
// offset there, and that CTA's loaders arm it for both.
enum { kLoadW, kLoadX, kLoadWs, kLoadXs };
template <int kKind, int kWhat>
__device__ __forceinline__ void product_loader(const ProductParams &P, ProductControl *ctl, ProductWalk<kKind> walk, int total, unsigned long long deadline,
                                               uint32_t rank, uint8_t *ring)
{
    using C = PrCfg<kKind>;
    constexpr bool kPair = C::kPair;
    constexpr uint32_t kAt = kWhat == kLoadW ? 0 : kWhat == kLoadX ? kPrWBytes : kWhat == kLoadWs ? kPrWBytes + C::kXBytes : kPrWBytes + C::kXBytes + kPrWScaleBytes;
    constexpr int kStep = kWhat == kLoadW || kWhat == kLoadX ? kPrK / 2 : 2;
    const uint32_t dst0 = smem_u32(ring) + kAt, empty0 = smem_u32(&ctl->empty[0]), full0 = smem_u32(&ctl->full[0]);
    uint32_t dst = dst0, empty_bar = empty0, full_bar = full0, phase = 0;
    bool ok = true, ready = true;                              // (all stages are free at first)
    for (; walk.g < total && ok; walk.next()) {
        const ProductTile t = walk.tile(P, ctl);
        const CUtensorMap *map;
        int y, z = 0, boxes = 1;
        uint32_t bytes;
        if (kWhat == kLoadW) {
            map = &P.tmW;
            bytes = kPrWBytes;
            y = t.n0 + (int)rank * kPrN;
            z = t.e;
        } else if (kWhat == kLoadX) {
            // rows that this CTA holds of the tile: in one box, or in two of 64; those behind the tile's own are read for nothing
            const int held = kPair ? ((t.valid + C::kRound - 1) & -C::kRound) / 2 : t.valid;
            const int which = kPair ? (held > 32 ? 0 : 1) : C::kFew ? (held > 16 ? 0 : 1) : held > 128 ? 0 : held > 16 ? 1 : 2;
            boxes = kKind == kOneTiles && which == 1 && held > 64 ? 2 : 1;
            map = &P.tmX[which];
            bytes = (which == 0 ? C::kXRows : which == 2 || C::kFew ? 16u : kPair ? 32u : 64u) * (kPrK / 2);
            y = t.row0 + (int)rank * held;
        } else if (kWhat == kLoadWs) {
            map = &P.tmWs;
            bytes = kPrWScaleBytes;
            y = t.e * P.N / kMxTile + t.e + t.n0 / kMxTile + (int)rank;
        } else {
            // the row block that the quantisation put the tile's first row into: by the expert's first row (row0 - local)
            map = &P.tmXs;
            bytes = C::kXsBytes;
            y = (t.row0 - t.local) / kMxTile + t.e + t.local / kMxTile;
        }
        const uint32_t expected = (kPair ? 2u : 1u) * (uint32_t)boxes * bytes;
        int x = 0;
        for (int kb = 0; kb < P.num_kb; ++kb) {
            if (!__all_sync(0xffffffffu, ready)) {
                ok = __all_sync(0xffffffffu, pr_wait(empty_bar, phase ^ 1u, ctl, deadline, P.status, (uint32_t)walk.g, 70u + kWhat));
                if (!ok) break;
            }
            if (elect_one_sync()) {
                if (!kPair || rank == 0) mbar_arrive_expect_tx(full_bar, expected);
                const uint32_t bar = kPair ? full_bar & 0xFEFFFFFFu : full_bar;
                if (kWhat == kLoadX) {
                    if (kPair) tma_load_2d_pair(dst, map, bar, x, y);
                    else tma_load_2d(dst, map, bar, x, y);
                    if (kKind == kOneTiles && boxes == 2) tma_load_2d(dst + bytes, map, bar, x, y + 64);
                } else if (kWhat == kLoadW) {
                    if (kPair) tma_load_3d_pair(dst, map, bar, x, y, z);
                    else tma_load_3d(dst, map, bar, x, y, z);
                } else {
                    if (kPair) tma_load_3d_pair(dst, map, bar, 0, x, y);
                    else tma_load_3d(dst, map, bar, 0, x, y);
                }
            }
            x += kStep;
            dst += (uint32_t)C::kStageBytes;
            empty_bar += 8u;
            full_bar += 8u;
            if (empty_bar == empty0 + 8u * C::kStages) {
                dst = dst0;
                empty_bar = empty0;
                full_bar = full0;
                phase ^= 1u;
            }
            ready = mbar_test_wait(empty_bar, phase ^ 1u);
        }
    }
    __syncwarp();
}

// The same piece into shared memory: rows of 128 bytes, 128B swizzle, `half` the columns 32 half .. of the 64
template <class E>
__device__ __forceinline__ void stage_piece(const uint32_t (&lo)[16], const uint32_t (&hi)[16], uint32_t buf, int half)
{
    const int lane = threadIdx.x & 31, r = lane & 7, chunk = half * 4 + (lane >> 3);
    const auto pack = [](uint32_t a, uint32_t b) { return RowType<E>::pack(__uint_as_float(a), __uint_as_float(b)); };
#pragma unroll
    for (int j = 0; j < 4; ++j)                  // rows 8j..8j+7: four blocks of 8 x 8, stored transposed
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                     ::"r"(buf + (uint32_t)((8 * j + r) * 128 + ((chunk ^ r) << 4))), "r"(pack(lo[4 * j], lo[4 * j + 1])), "r"(pack(lo[4 * j + 2], lo[4 * j + 3])),
                     "r"(pack(hi[4 * j], hi[4 * j + 1])), "r"(pack(hi[4 * j + 2], hi[4 * j + 3]))
                     : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"((unsigned long long)map), "r"(src), "r"(x), "r"(y) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

// Row tiles counted by one warp, whatever the offsets and however many.  An expert has rows where its two offsets are in order and within
// the rows, and where it begins behind the rows of all such experts before it; tiles of any other are never walked to.
__device__ __noinline__ void count_tiles(const ProductParams &P, ProductControl *ctl, int lane, int tile_rows)
{
    int tiles = 0, top = 0;                      // of the experts before these 32: their tiles, where their rows end
    for (int e0 = 0; e0 <= P.E; e0 += 32) {
        const int e = e0 + lane, begin = ctl->first[min(e, P.E)], end = ctl->first[min(e + 1, P.E)];
        const bool ordered = begin >= 0 && begin <= end && end <= P.R;
        if (e <= P.E && !ordered && blockIdx.x == 0) report(P.status, MOE_DEV_OOB, (uint32_t)e, 63u);
        int ends = ordered ? end : 0;            // running maximum of the ends up to this expert
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, ends, d);
            if (lane >= d) ends = max(ends, u);
        }
        int before = __shfl_up_sync(0xffffffffu, ends, 1);
        before = lane == 0 ? top : max(before, top);
        const int own = e < P.E && ordered && begin >= before ? (end - begin + tile_rows - 1) / tile_rows : 0;
        int t = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, t, d);
            if (lane >= d) t += u;
        }
        if (e <= P.E) ctl->tiles[e] = tiles + t - own;
        top = max(top, __shfl_sync(0xffffffffu, ends, 31));
        tiles += __shfl_sync(0xffffffffu, t, 31);
    }
}

// After a wait that ran out, roles have left without waiting for one another: the MMAs that were issued finish, and the copies that are on
// their way land, before TMEM and shared memory are given back.  By the warp that issues the MMAs, in each CTA of a pair: a pair's copies
// complete on the first CTA's barriers, so that the second has none to wait on, and every CTA waits for a time that copies do not take.
template <bool kPair>
__device__ __noinline__ void finish_in_flight(ProductControl *ctl, uint32_t rank)
{
    const unsigned long long now = globaltimer_ns();
    if (rank == 0) {
        if (elect_one_sync()) {
            if (kPair) tc_commit_pair(smem_u32(&ctl->drain));
            else tc_commit(smem_u32(&ctl->drain));
        }
        __syncwarp();
        while (!mbar_try_wait(smem_u32(&ctl->drain), 0u) && globaltimer_ns() < now + 4 * kLandNs) {}
    }
    wait_for_what_is_in_flight();
}

template <class E, int kKind>
__global__ void __launch_bounds__(kPrThreads, 1) mxfp4_product_kernel(const __grid_constant__ ProductParams P)
{
    using C = PrCfg<kKind>;
    constexpr bool kPair = C::kPair;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    ProductControl *ctl = reinterpret_cast<ProductControl *>(ring + C::kStages * C::kStageBytes + C::kOutBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kPair ? cluster_ctarank() : 0u;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(smem_u32(&ctl->full[i]), 4);            // the four loaders (pair: the first CTA's, which arm it for both)
            mbar_init(smem_u32(&ctl->empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ctl->tmem_full[i]), 1);
            mbar_init(smem_u32(&ctl->tmem_empty[i]), (kPair ? 2 : 1) * kPrEpiWarps);
        }
        mbar_init(smem_u32(&ctl->drain), 1);
        ctl->abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        prefetch_tensormap(&P.tmW);
        prefetch_tensormap(&P.tmX[0]);
        prefetch_tensormap(&P.tmWs);
        prefetch_tensormap(&P.tmXs);
    }
    if (warp == 1) {
        if (kPair) tmem_alloc_pair(smem_u32(&ctl->tmem_base), kPrTmemCols);
        else tmem_alloc(smem_u32(&ctl->tmem_base), kPrTmemCols);
    }
    grid_dependency_wait();
    // Where the experts' rows begin and how many row tiles lie before them.  A thread has an expert; offsets that go back or past the rows
    // are reported, and the experts beside them have no rows.
    if (P.E <= kPrThreads - 1) {
        const int e = (int)threadIdx.x;
        const int o = ld_chained(P.offsets + min(e, P.E)), next = ld_chained(P.offsets + min(e + 1, P.E));
        int t = e < P.E ? (int)(((uint32_t)next - (uint32_t)o + (uint32_t)(C::kRows - 1)) / (uint32_t)C::kRows) : 0;      // (in order: as below)
        const int own = t;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, t, d);
            if (lane >= d) t += u;
        }
        if (e <= P.E) ctl->first[e] = o;
        if (lane == 31) ctl->warp_tiles[warp] = t;
        tc_fence_before();
        const bool fine = __syncthreads_and(o >= 0 && o <= next && next <= P.R) != 0;
        tc_fence_after();
        if (fine && 32 * warp <= P.E) {
            int base = 0;
            for (int w = 0; w < warp; ++w) base += ctl->warp_tiles[w];
            if (e <= P.E) ctl->tiles[e] = base + t - own;
        } else if (!fine && warp == 3) {
            count_tiles(P, ctl, lane, C::kRows);
        }
    } else {
        for (int e = threadIdx.x; e <= P.E; e += kPrThreads) ctl->first[e] = ld_chained(P.offsets + e);
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == 3) count_tiles(P, ctl, lane, C::kRows);
    }
    __syncthreads();
    if (kPair) cluster_sync_all();     // the other CTA's barriers exist before anything arrives on them
    const uint32_t tmem_base = ctl->tmem_base;
    const int total = ctl->tiles[P.E] * P.NT;
    const unsigned long long deadline = globaltimer_ns() + P.wait_ns;
    ProductWalk<kKind> walk(P, ctl);

    if (warp == 0) product_loader<kKind, kLoadW>(P, ctl, walk, total, deadline, rank, ring);
    else if (warp == 2) product_loader<kKind, kLoadX>(P, ctl, walk, total, deadline, rank, ring);
    else if (warp == 3) product_loader<kKind, kLoadWs>(P, ctl, walk, total, deadline, rank, ring);
    else if (warp == 4 + kPrEpiWarps) product_loader<kKind, kLoadXs>(P, ctl, walk, total, deadline, rank, ring);
    else if (warp == 1 && rank == 0) {
        // The whole warp runs the loop, converged, and one elected lane issues: warp-uniform operands, addresses that advance by additions,
        // the next stage's barrier looked at before this one's MMAs are issued.  The thread that issues paces the tensor pipe: with a
        // wait that starts at the head of a stage, a second one for columns of exponents in shorter supply than stages, and addresses from
        // the stage's number, it needed 450 cycles a stage without a single MMA; the MMAs take 400.
        constexpr uint32_t kLoStage = (uint32_t)(C::kStageBytes >> 4), kLoX = (uint32_t)(kPrWBytes >> 4), kLoWs = (uint32_t)((kPrWBytes + C::kXBytes) >> 4),
                           kLoXs = kLoWs + (uint32_t)(kPrWScaleBytes >> 4);
        const uint32_t lo0 = smem_desc_lo(smem_u32(ring)), full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
        const uint32_t sw0 = tmem_base + (uint32_t)(2 * C::kRows);
        uint32_t w_lo = lo0, full_bar = full0, empty_bar = empty0, sw = sw0, phase = 0;
        int it = 0;
        bool ok = true, ready = mbar_test_wait(full0, 0u);
        const auto wait_stage = [&]() {
            if (__all_sync(0xffffffffu, ready)) return;
            ok = __all_sync(0xffffffffu, pr_wait(full_bar, phase, ctl, deadline, P.status, (uint32_t)walk.g, 76u));
        };
        const auto advance = [&]() {
            w_lo += kLoStage;
            full_bar += 8u;
            empty_bar += 8u;
            sw += (uint32_t)kPrScaleCols;
            if (full_bar == full0 + 8u * C::kStages) {
                w_lo = lo0;
                full_bar = full0;
                empty_bar = empty0;
                sw = sw0;
                phase ^= 1u;
            }
        };
        // the next stage's barrier, looked at early
        const auto look = [&]() {
            const bool wraps = full_bar == full0 + 8u * (C::kStages - 1);
            ready = mbar_test_wait(wraps ? full0 : full_bar + 8u, wraps ? phase ^ 1u : phase);
        };
        for (; walk.g < total && ok; walk.next(), ++it) {
            const ProductTile t = walk.tile(P, ctl);
            const int a = it & 1;
            const uint32_t shift = __reduce_max_sync(0xffffffffu, (uint32_t)(t.local & (kMxTile - 1)) >> 5);     // 0 or 2 columns: first row inside its row block
            const uint32_t n = __reduce_max_sync(0xffffffffu, (uint32_t)((t.valid + C::kRound - 1) & -C::kRound)), two = 32u * shift + n > (uint32_t)kMxTile ? 1u : 0u;
            const uint32_t idesc0 = mxf4_idesc((uint32_t)C::kTileN, n, 0u), idesc1 = mxf4_idesc((uint32_t)C::kTileN, n, 1u);
            const uint32_t parity = ((uint32_t)(it >> 1) & 1u) ^ 1u;
            if (!__all_sync(0xffffffffu, mbar_test_wait(smem_u32(&ctl->tmem_empty[a]), parity))) {
                ok = __all_sync(0xffffffffu, pr_wait(smem_u32(&ctl->tmem_empty[a]), parity, ctl, deadline, P.status, (uint32_t)walk.g, 75u));
                if (!ok) break;
            }
            const uint32_t d_tmem = tmem_base + (uint32_t)(a * C::kRows);
            uint32_t accumulate = 0u;
            for (int kb = 1; kb < P.num_kb; ++kb) {
                wait_stage();
                if (!ok) break;
                tc_fence_after();
                look();
                if (elect_one_sync())
                    tc_stage_mxf4<kPair, true>(d_tmem, w_lo, w_lo + kLoX, w_lo + kLoWs, w_lo + kLoXs, sw, sw + 8u, shift, two, idesc0, idesc1, accumulate, 4u, empty_bar);
                accumulate = 1u;
                advance();
            }
            if (!ok) break;
            wait_stage();
            if (!ok) break;
            tc_fence_after();
            look();
            if (elect_one_sync()) {
                tc_stage_mxf4<kPair, false>(d_tmem, w_lo, w_lo + kLoX, w_lo + kLoWs, w_lo + kLoXs, sw, sw + 8u, shift, two, idesc0, idesc1, accumulate,
                                            (uint32_t)P.last_steps, empty_bar);
                if (kPair) tc_commit_pair(smem_u32(&ctl->tmem_full[a]));
                else tc_commit(smem_u32(&ctl->tmem_full[a]));
            }
            advance();
        }
        __syncwarp();
    } else if (warp >= 4 && warp < 4 + kPrEpiWarps) {
        const int q4 = warp & 3, grp = (warp - 4) >> 2;
        int it = 0;
        // a pair: the two warps of 64 columns (a barrier of their own, 1 to 4), and which of their two buffers is next
        const int unit = 2 * grp + (q4 >> 1);
        const uint32_t out0 = smem_u32(ring + C::kStages * C::kStageBytes) + (uint32_t)(unit * 2 * kPrOutBytes);
        uint32_t flip = 0;
        for (; walk.g < total; walk.next(), ++it) {
            const ProductTile t = walk.tile(P, ctl);
            const int a = it & 1, pieces = (t.valid + 31) >> 5, col = t.n0 + (int)rank * kPrN + q4 * 32, cols = P.N - col;
            uint32_t ok = 1u;
            if (lane == 0) ok = pr_wait(smem_u32(&ctl->tmem_full[a]), (uint32_t)(it >> 1) & 1u, ctl, deadline, P.status, (uint32_t)walk.g, 77u) ? 1u : 0u;
            ok = __shfl_sync(0xffffffffu, ok, 0);
            // (the two warps of a unit leave together: each waits for the other in every piece)
            if (kPair)
                asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %0, 0;\n\tbar.red.and.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "+r"(ok) : "r"(1 + unit) : "memory");
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(q4 * 32) << 16) + (uint32_t)(a * C::kRows);
            const auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (kPair) mbar_arrive_cluster_relaxed(mapa_u32(smem_u32(&ctl->tmem_empty[a]), 0u));   // the first CTA's barrier
                    else mbar_arrive(smem_u32(&ctl->tmem_empty[a]));
                }
            };
            if (grp >= pieces) release();
#pragma unroll 1
            for (int piece = grp; piece < pieces; piece += kPrEpiWarps / 4) {
                uint32_t lo[16], hi[16];
                tmem_ld_16x256_x4(taddr + (uint32_t)(piece * 32), lo);
                tmem_ld_16x256_x4(taddr + (16u << 16) + (uint32_t)(piece * 32), hi);
                tmem_ld_wait(lo);
                tmem_ld_wait(hi);
                if (piece + kPrEpiWarps / 4 >= pieces) release();
                if (kPair && piece * 32 + 32 <= t.valid) {
                    const int first = col - (q4 & 1) * 32;                     // of the 64 columns
                    if (first >= P.N) continue;
                    const bool issues = (q4 & 1) == 0 && lane == 0;
                    const uint32_t buf = out0 + flip * (uint32_t)kPrOutBytes;
                    if (issues) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");       // this buffer's last copy has been read
                    asm volatile("bar.sync %0, 64;" ::"r"(1 + unit) : "memory");
                    stage_piece<E>(lo, hi, buf, q4 & 1);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    asm volatile("bar.sync %0, 64;" ::"r"(1 + unit) : "memory");
                    if (issues) tma_store_2d(&P.tmOut, buf, first, t.row0 + piece * 32);
                    flip ^= 1u;
                    continue;
                }
                const int row = piece * 32 + lane;
                E *dst = row < t.valid && cols > 0 ? static_cast<E *>(P.out) + (long long)(t.row0 + row) * P.ld_out + col : nullptr;
                store_piece<E>(lo, hi, dst, cols);
            }
        }
        if (kPair && (q4 & 1) == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1 && ctl->abort) finish_in_flight<kPair>(ctl, rank);
    // (pair: nobody leaves while the other CTA may still touch its memory)
    if (kPair) cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        if (kPair) tmem_dealloc_pair(tmem_base, kPrTmemCols);
        else tmem_dealloc(tmem_base, kPrTmemCols);
    }
}

template <int kKind>
constexpr size_t pr_smem_bytes() { return (size_t)PrCfg<kKind>::kStages * PrCfg<kKind>::kStageBytes + PrCfg<kKind>::kOutBytes + 1024 + ((sizeof(ProductControl) + 127) & ~(size_t)127); }
static_assert(pr_smem_bytes<kOneTiles>() <= 227 * 1024 && pr_smem_bytes<kPairTiles>() <= 227 * 1024 && pr_smem_bytes<kFewTiles>() <= 227 * 1024, "the product's stages exceed the shared memory of an SM");

// Tiles by pairs of CTAs read less per product, but there are half as many places for them.  They pay from this many rows per expert
// on, where every pair then has this many tiles.  One CTA / pair, us, skewed routing, at the rows per expert (tiles a pair) given:
//   N 2816, K 2048   84 (14) 44.4/45.0   121 (17) 48.7/48.1   157 (18) 53.4/52.1   181 (19) 57.5/55.2   248 (22) 69.2/64.4   992 (61) 210/183
//   N 2048, K 1408  100 (10) 26.3/26.9   136 (11) 29.8/29.8   157 (13) 35.3/33.9   181 (14) 36.1/35.0   248 (16) 42.9/40.9   992 (44) 132/113
//   N 1536, K 512   200 (6) 14.4/15.0    300 (8) 17.5/18.6    409 (10) 20.6/21.5   520 (12) 22.7/23.4   819 (17) 30.8/30.8   1638 (31) 52.0/49.5
//   N 1024, K 1536  200 (4) 17.5/18.5    300 (6) 20.5/20.7    409 (7) 23.2/22.8    819 (11) 35.7/34.0   1638 (20) 62.7/56.5
// Within 2 % of the line either side may be ahead: the rule loses 3 % at N 1536, K 512 with 12 tiles, whose short K hides a pair's start least.
constexpr int32_t kPairRowsPerExpert = 128, kPairTilesEach = 11;
// Mean rows per expert up to which tiles of 64 rows in eight stages pay: with up to 16 rows in a tile 160 KB are on their way to an SM instead of 105
// (with 64 rows 208 instead of 135), but an expert of 65 rows reads its weights twice.  192 / 64 rows, us, at 1 / 4 to 6 / 7 to 8 / 15 to 17 / 48 rows per expert:
//   N 2816, K 2048   22.8/21.9  34.2/33.8  35.9/36.4  36.9/37.6  40.5/42.2
//   N 2048, K 1408   16.4/15.4  20.8/19.2  22.5/21.0  23.8/22.2  25.8/24.7
//   N 1024, K 1536    9.4/9.3   11.3/10.9  12.0/11.6  12.2/11.9  12.7/12.3
// The rule goes by rows alone, and loses 1 to 2 % where the weights are largest (N 2816, K 2048 from seven rows on), as it leaves 4 % at 48 rows elsewhere.
constexpr int32_t kFewRowsPerExpert = 16;

// tiles of a launch, whatever the offsets
int64_t tiles_at_most(int32_t rows, int32_t E_tot, int32_t tile_rows, int32_t NT)
{
    const int64_t used = rows < E_tot ? rows : E_tot;
    return ((rows - used) / tile_rows + used) * NT;
}
int product_kind(const moe_handle *h, int32_t rows, int32_t E_tot, int32_t N)
{
    using Pair = PrCfg<kPairTiles>;
    if (h->max_pairs > 0 && rows / E_tot >= kPairRowsPerExpert &&
        tiles_at_most(rows, E_tot, Pair::kRows, (N + Pair::kTileN - 1) / Pair::kTileN) >= (int64_t)kPairTilesEach * h->max_pairs)
        return kPairTiles;
    return rows / E_tot <= kFewRowsPerExpert ? kFewTiles : kOneTiles;
}
bool product_sizes_ok(int32_t rows, int32_t E_tot, int32_t N)
{
    return rows >= 0 && rows < 1 << 30 && E_tot >= 1 && E_tot <= kMaxExperts && N >= 8 && N % 8 == 0 && (int64_t)E_tot * N < 1 << 30;
}

bool columns_ok(int32_t K) { return K >= kMxBlock && K % kMxBlock == 0 && K <= 1 << 20; }
int64_t scale_blocks(int64_t rows, int32_t groups) { return rows / kMxTile + groups; }

int32_t describe(moe_handle *h, const char *who, int32_t rows, int32_t src_rows, int32_t copies, int32_t K, int32_t groups, int32_t dtype, int64_t ld,
                 const int32_t *offsets, const int32_t *inv_perm, const void *matrix, const void *codes, const void *scales, uint32_t *status, Quant *p)
{
    if (!h || !status) return MOE_ERR_NULL;
    if (rows < 0 || rows >= 1 << 30 || groups < 1 || groups > (1 << 20) || !columns_ok(K) || !pitch_ok(ld, K)) return MOE_ERR_SHAPE;
    if (!offsets && rows % groups != 0) return MOE_ERR_SHAPE;
    if (!row_type_ok(dtype)) return MOE_ERR_UNSUPPORTED;
    p->rows = 0;
    if (rows == 0) return MOE_OK;
    if (!matrix || !codes || !scales) return MOE_ERR_NULL;
    if (!rows_aligned(matrix) || !rows_aligned(codes) || !rows_aligned(scales) || !rows_aligned(status)) return MOE_ERR_ALIGN;
    if (const int32_t rc = require_handle_device(h, who)) return rc;
    memset(p, 0, sizeof *p);
    p->codes = static_cast<uint8_t *>(const_cast<void *>(codes));
    p->scales = static_cast<uint8_t *>(const_cast<void *>(scales));
    p->offsets = offsets;
    p->inv_perm = inv_perm;
    p->status = status;
    p->ld = ld;
    p->blocks = scale_blocks(rows, groups);
    p->rows = rows;
    p->src_rows = src_rows;
    p->copies = copies;
    p->groups = groups;
    p->n_even = rows / groups > 0 ? rows / groups : 1;
    p->K = K;
    p->KQ = (K + kMxTile - 1) / kMxTile;
    p->lanes = p->KQ * 8;
    p->wide = rows_wide(matrix, ld, dtype);
    p->by_lanes = divisor_of(p->lanes);
    p->by_n = divisor_of(p->n_even);
    // (tokens into routed order: 16 a block 51 us, 4 46, 2 42, 1 44 at 16384 tokens; weights: the same from 16 down to 2)
    p->rows_per_cta = inv_perm ? kQuantTokensMax : kQuantRowsMax;
    while (p->rows_per_cta > 1 && (int64_t)src_rows < (int64_t)p->rows_per_cta * 4 * h->G) p->rows_per_cta /= 2;
    return MOE_OK;
}

}  // namespace
}  // namespace moe

using namespace moe;

template <int kKind>
static cudaError_t prepare_product()
{
    const cudaError_t e = cudaFuncSetAttribute(mxfp4_product_kernel<__nv_bfloat16, kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pr_smem_bytes<kKind>());
    return e != cudaSuccess ? e : cudaFuncSetAttribute(mxfp4_product_kernel<__half, kKind>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pr_smem_bytes<kKind>());
}
cudaError_t moe::mxfp4_prepare()
{
    cudaError_t e = prepare_product<kOneTiles>();
    if (e == cudaSuccess) e = prepare_product<kPairTiles>();
    return e != cudaSuccess ? e : prepare_product<kFewTiles>();
}

extern "C" int32_t moe_mxfp4_scale_bytes(int32_t rows, int32_t K, int32_t groups, size_t *bytes)
{
    if (!bytes) return MOE_ERR_NULL;
    if (rows < 0 || rows >= 1 << 30 || groups < 1 || groups > 1 << 20 || !columns_ok(K)) return MOE_ERR_SHAPE;
    *bytes = (size_t)scale_blocks(rows, groups) * (size_t)((K + kMxTile - 1) / kMxTile) * kMxTileBytes;
    return MOE_OK;
}

extern "C" int32_t moe_mxfp4_quantize(moe_handle *h, const void *src, int64_t ld_src, int32_t dtype, int32_t rows, int32_t K, int32_t groups,
                                      const int32_t *offsets_or_null, const int32_t *inv_perm_or_null, int32_t copies, void *codes, void *scales,
                                      uint32_t *status_dev, void *stream)
{
    if (inv_perm_or_null ? copies < 1 || copies > 32 || rows % copies != 0 : copies != 1) return MOE_ERR_SHAPE;
    Quant p;
    const int32_t rc = describe(h, "moe_mxfp4_quantize", rows, rows / copies, copies, K, groups, dtype, ld_src, offsets_or_null, inv_perm_or_null, src, codes, scales,
                                status_dev, &p);
    if (rc != MOE_OK || p.rows == 0) return rc;
    const unsigned grid = (unsigned)((p.src_rows + p.rows_per_cta - 1) / p.rows_per_cta);
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const cudaError_t err = launch_chained(inv_perm_or_null ? quantize_kernel<E, true> : quantize_kernel<E, false>, grid, kQuantThreads, 0,
                                               static_cast<cudaStream_t>(stream), p, static_cast<const E *>(src));
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "quantisation launch");
    });
}

extern "C" int32_t moe_mxfp4_dequantize(moe_handle *h, const void *codes, const void *scales, int32_t rows, int32_t K, int32_t groups,
                                        const int32_t *offsets_or_null, int32_t dtype, void *out, int64_t ld_out, uint32_t *status_dev, void *stream)
{
    Quant p;
    const int32_t rc = describe(h, "moe_mxfp4_dequantize", rows, rows, 1, K, groups, dtype, ld_out, offsets_or_null, nullptr, out, codes, scales, status_dev, &p);
    if (rc != MOE_OK || p.rows == 0) return rc;
    const unsigned grid = (unsigned)((rows + p.rows_per_cta - 1) / p.rows_per_cta);
    return with_row_type(dtype, [&](auto *e) -> int32_t {
        using E = std::remove_pointer_t<decltype(e)>;
        const cudaError_t err = launch_chained(dequantize_kernel<E>, grid, kQuantThreads, 0, static_cast<cudaStream_t>(stream), p, static_cast<E *>(out));
        return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "dequantisation launch");
    });
}

extern "C" int32_t moe_mxfp4_select_tile(moe_handle *h, int32_t rows, int32_t E_tot, int32_t N, int32_t *tile_rows, int32_t *tile_cols)
{
    if (!h || !tile_rows || !tile_cols) return MOE_ERR_NULL;
    if (!product_sizes_ok(rows, E_tot, N)) return MOE_ERR_SHAPE;
    const int kind = product_kind(h, rows, E_tot, N);
    *tile_rows = kind == kFewTiles ? PrCfg<kFewTiles>::kRows : PrCfg<kOneTiles>::kRows;
    *tile_cols = kind == kPairTiles ? PrCfg<kPairTiles>::kTileN : kPrN;
    return MOE_OK;
}

extern "C" int32_t moe_mxfp4_gemm(moe_handle *h, const void *x_codes, const void *x_scales, const void *w_codes, const void *w_scales,
                                  const int32_t *offsets, int32_t rows, int32_t E_tot, int32_t N, int32_t K, int32_t dtype, void *out, int64_t ld_out,
                                  uint32_t *status_dev, void *stream)
{
    if (!h || !status_dev) return MOE_ERR_NULL;
    if (!product_sizes_ok(rows, E_tot, N) || !columns_ok(K) || !pitch_ok(ld_out, N)) return MOE_ERR_SHAPE;
    if (dtype != MOE_BF16 && dtype != MOE_FP16) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    if (!x_codes || !x_scales || !w_codes || !w_scales || !offsets || !out) return MOE_ERR_NULL;
    if (!rows_aligned(x_codes) || !rows_aligned(x_scales) || !rows_aligned(w_codes) || !rows_aligned(w_scales) || !rows_aligned(out) ||
        !rows_aligned(status_dev))
        return MOE_ERR_ALIGN;
    if (const int32_t rc = require_handle_device(h, "moe_mxfp4_gemm")) return rc;
    ProductParams p;
    memset(&p, 0, sizeof p);
    p.offsets = offsets;
    p.out = out;
    p.ld_out = ld_out;
    p.status = status_dev;
    p.wait_ns = h->wait_ns;
    p.R = rows;
    p.E = E_tot;
    p.N = N;
    p.KQ = (K + kMxTile - 1) / kMxTile;
    p.num_kb = (K + kPrK - 1) / kPrK;
    p.last_steps = (K - (p.num_kb - 1) * kPrK + kPrStepK - 1) / kPrStepK;
    const int kind = product_kind(h, rows, E_tot, N);
    const bool pair = kind == kPairTiles, few = kind == kFewTiles;
    const int32_t tile_n = pair ? PrCfg<kPairTiles>::kTileN : kPrN, tile_rows = few ? PrCfg<kFewTiles>::kRows : PrCfg<kOneTiles>::kRows;
    p.NT = (N + tile_n - 1) / tile_n;
    p.by_NT = divisor_of(p.NT);
    const int64_t tiles = tiles_at_most(rows, E_tot, tile_rows, p.NT);
    if (tiles >= (int64_t)1 << 31) return MOE_ERR_SHAPE;
    const int32_t boxes[3][3] = {{PrCfg<kOneTiles>::kXRows, 64, 16}, {PrCfg<kPairTiles>::kXRows, 32, 0}, {PrCfg<kFewTiles>::kXRows, 16, 0}};
    for (int i = 0; i < 3 && boxes[kind][i]; ++i)
        if (!code_map(h, &p.tmX[i], x_codes, 0, rows, K / 2, boxes[kind][i], "x_codes")) return MOE_ERR_CUDA;
    if (pair && !out_map(h, &p.tmOut, out, rows, N, ld_out, kPrOutCols, kPrOutRows, "out")) return MOE_ERR_CUDA;
    if (!code_map(h, &p.tmW, w_codes, E_tot, N, K / 2, kPrN, "w_codes") ||
        !scale_map(h, &p.tmXs, x_scales, scale_blocks(rows, E_tot), p.KQ, few ? 1 : 2, "x_scales") ||
        !scale_map(h, &p.tmWs, w_scales, scale_blocks((int64_t)E_tot * N, E_tot), p.KQ, 1, "w_scales"))
        return MOE_ERR_CUDA;
    const int64_t slots = pair ? h->max_pairs : h->G, grid = tiles < slots ? tiles : slots;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2] = {chained_launch_attribute()};
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pair ? 2 : 1;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.gridDim = dim3((unsigned)(pair ? 2 * grid : grid));
    cfg.blockDim = dim3(kPrThreads);
    cfg.dynamicSmemBytes = pair ? pr_smem_bytes<kPairTiles>() : few ? pr_smem_bytes<kFewTiles>() : pr_smem_bytes<kOneTiles>();
    const bool half = dtype == MOE_FP16;
    const auto launch = [&](auto one, auto two, auto three) { return cudaLaunchKernelEx(&cfg, pair ? two : few ? three : one, p); };
    const cudaError_t err =
        half ? launch(mxfp4_product_kernel<__half, kOneTiles>, mxfp4_product_kernel<__half, kPairTiles>, mxfp4_product_kernel<__half, kFewTiles>)
             : launch(mxfp4_product_kernel<__nv_bfloat16, kOneTiles>, mxfp4_product_kernel<__nv_bfloat16, kPairTiles>, mxfp4_product_kernel<__nv_bfloat16, kFewTiles>);
    return err == cudaSuccess ? MOE_OK : cuda_fail(h, err, "grouped 4-bit product launch");
}
