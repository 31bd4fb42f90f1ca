// Products of 16-bit codes (binary16 or bfloat16 words) whose sums go through an epilogue of the caller's choice instead of
// to memory as they are: the frame that qfmt_linear_act and qfmt_linear_cross_entropy share.
//
// One persistent kernel.  For large products one CTA pair per two SMs and 256 x 256 tiles: each CTA stages its own 128 rows of op(A) and its own 128
// columns of op(B) by TMA (64 K elements, 32 KB a stage), the leader's MMA thread issues tcgen05.mma.cta_group::2 kind::f16
// with M = 256, N = 256, K = 16, and each CTA's tensor memory receives its 128 x 256 half of the tile, in one of two 256-column
// accumulators, so the sixteen epilogue warps work on one tile while the next one is summed in the other.
//
// Accuracy.  Sums are fp32, and the tensor core truncates one once per 16 products, by at most 2^-23 of sum |a||b| and always towards zero, so
// a sum of one sign drifts by its length.  After 8192 elements it is closed (kLong): its epilogue warps add it to what the ones before it
// came to, rounded to nearest, while the next 8192 are summed in the other accumulator.  So a sum is off by at most
//     (min(K, 8192) / 16 + K / 16384) 2^-23 of sum |a||b|
// and what the few additions of an epilogue lose: 2^-14 at K = 8192, 2^-13.8 at 2^20, 2^-12.4 at 2^24, against the half step of 2^-12 that
// binary16 has.  (qfmt_gemm_packed16 hands out fp32 sums and takes them in three levels instead, 2^-20, which costs it a third of its
// rate.)  The closed sums are 256 bytes a thread of local memory.  Kernels of their own, since the epilogues have no registers to spare: with
// the same code for all, 8192 x 1024 x 4096 with GELU took 86 instead of 81 us.
//
// Products that leave pairs without a tile run on single CTAs with 128 x 256 tiles (cta_group::1, 48 KB a stage): twice as many workers
// for half the rows each, at one and a half times the operand traffic (rule: plan_product).
//
// Roles: warps 0 and 3 fill alternate stages, warp 1 issues the MMAs (leader CTA), warp 2 idles, warps 4-19 run the epilogue:
// warp w has rows 32 (w % 4) .. + 31 and columns 64 ((w - 4) / 4) .. + 63 of its CTA's half, one row a lane, 32 columns at a time.  (With
// eight epilogue warps of 128 columns each an activation's epilogue took longer than a contraction over 1024 elements, waiting on its own
// loads and conversions; 96 registers a thread are enough for 32 columns.)
//
// Rows may be counted on the device (ProductParams::count): tiles beyond the count are left out, and an operand that was
// gathered is read in place if every row counts (alt).  Every wait is bounded; on expiry the status area reports
// QFMT_ERR_TIMEOUT and all roles leave.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "activation.cuh"
#include "common.cuh"
#include "ptx.cuh"
#include "tiles.cuh"

namespace qfmt {
namespace p16 {

constexpr int kRows = 128, kTileN = 256, kStageK = 64;  // rows of a CTA's tile, columns of a tile, K elements of a stage
// kPair: shared memory holds half of a tile's columns of B and five stages (three: 64 us for 8192 x 1024 x 4096 without an activation, four
// 58.6, five 56.9, six 56.4, at the expense of what the epilogues' loads keep in the first-level cache: 84 against 91 us for the backward
// pass through GELU); otherwise all of them and four stages.
template <bool kPair>
struct Staging {
    static constexpr int kStages = kPair ? 5 : 4, kColumns = kPair ? 128 : 256;
    static constexpr uint32_t kA = kRows * kStageK * 2, kB = kColumns * kStageK * 2, kBytes = kA + kB;
};
constexpr int kThreads = 640, kEpiWarps = 16;
constexpr uint32_t kBoxBytes = 2048;       // 32 rows x 64 bytes per epilogue warp, 16-byte chunks swizzled with the row
template <bool kPair>
constexpr uint32_t smem_bytes() { return Staging<kPair>::kStages * Staging<kPair>::kBytes + kEpiWarps * kBoxBytes + 256 + 1024; }
static_assert(smem_bytes<true>() <= 232448 && smem_bytes<false>() <= 232448, "shared memory");
constexpr uint32_t kAccCols = 256, kTmemCols = 512;
constexpr uint32_t kWaitLimit = 1u << 31;  // SM cycles, about a second
constexpr int kCloseK = 8192, kCloseStages = kCloseK / kStageK;  // elements and stages of a sum before it is closed

enum : int { kFixed = 0, kCountM = 1, kCountK = 2 };  // which extent the device's count replaces
enum : int { kAltNone = 0, kAltA = 1, kAltB = 2 };    // which operand has a second place

struct ProductParams {
    int M, N, K;             // M or K is the upper bound where the device counts
    const int* count;        // device word, read where dyn != kFixed or alt != kAltNone
    int dyn, alt, alt_rows;  // the second map is read if *count == alt_rows
    int a_mn, b_mn;          // operand stored with M / N contiguous
    int a_blocked, b_blocked;
    int bf16;
    int splits, kb_per_split;
    unsigned long long* status;
    unsigned long long tag;
};

// What an epilogue warp gets to see of a tile.
struct Patch {
    int lane, quad, warp;    // warp: 0 .. 15 of the epilogue warps
    int row0;                // row of lane 0; lane l has row row0 + l
    int rows;                // M as counted
    int col0, cols;          // first of the 64 columns, N
    int split, tile_m, tile_n;
    uint32_t tmem;           // accumulator address of (row0, col0)
    bool empty;              // nothing was summed: the sums are zero
    float* closed;           // the closed sums of the lane's row, 64 columns; null without any
    uint8_t* box;

    __device__ __forceinline__ void load32(int block, uint32_t (&r)[32]) const {
        if (empty) {
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = 0u;
        } else {
            ptx::tmem_load_32cols(tmem + block * 32, r);
        }
    }
    // Waits for what load32 has asked for and adds the closed sums.
    __device__ __forceinline__ void finish(int block, uint32_t (&r)[32]) const {
        if (!empty) ptx::tmem_load_wait_for(r);
        if (closed != nullptr) {
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__fadd_rn(closed[block * 32 + j], __uint_as_float(r[j])));
        }
    }
    // Puts the accumulator on top of the closed sums.
    __device__ __forceinline__ void close(float (&sums)[64]) {
#pragma unroll 1
        for (int block = 0; block < 2; ++block) {
            uint32_t r[32];
            load32(block, r);
            finish(block, r);
#pragma unroll
            for (int j = 0; j < 32; ++j) sums[block * 32 + j] = __uint_as_float(r[j]);
        }
        closed = sums;
    }
    // Block of 32 columns in pairs, complete on return; kBias: plus a vector of the columns, of which the lane brings its column's value.
    // (It goes round through the box.)
    template <bool kBias>
    __device__ __forceinline__ void load_pairs(int block, pair_t (&v)[16], float bias = 0.0f) const {
        uint32_t r[32];
        load32(block, r);
        if (kBias) {
            reinterpret_cast<float*>(box)[lane] = bias;
            __syncwarp();
        }
        finish(block, r);
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            v[j / 2] = make_pair(__uint_as_float(r[j]), __uint_as_float(r[j + 1]));
            v[j / 2 + 1] = make_pair(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3]));
            if (kBias) {
                const float4 b = *reinterpret_cast<const float4*>(box + j * 4);
                v[j / 2] = add2(v[j / 2], make_pair(b.x, b.y));
                v[j / 2 + 1] = add2(v[j / 2 + 1], make_pair(b.z, b.w));
            }
        }
        if (kBias) __syncwarp();
    }
    // The lane's value of a vector of columns in each of the two blocks; zero beyond N and without a vector.
    __device__ __forceinline__ void columns(const float* v, float (&out)[2]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = col0 + i * 32 + lane;
            out[i] = v != nullptr && c < cols ? v[c] : 0.0f;
        }
    }
};

// ---- the box: 32 columns of 16 bits or 16 of 32 bits per row, written and read a row a lane on one side and in whole
// 64-byte rows on the other, so that global memory is touched in full sectors
__device__ __forceinline__ uint4* box_at(uint8_t* box, int row, int chunk) {
    return reinterpret_cast<uint4*>(box + row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4));
}
// box -> global.  vec: base and pitch are multiples of 16 bytes.
template <typename T>
__device__ __forceinline__ void box_store(uint8_t* box, T* base, int64_t ld, int row0, int rows, int col0, int cols, int lane, bool vec) {
    constexpr int per = 16 / (int)sizeof(T), width = 64 / (int)sizeof(T);
    if (vec) {
        const int c = lane & 3, col = col0 + c * per;
        T* g = base + (int64_t)(row0 + (lane >> 2)) * ld + col;
#pragma unroll
        for (int i = 0; i < 4; ++i, g += 8 * ld) {
            const int r = i * 8 + (lane >> 2);
            if (row0 + r < rows && col < cols) {
                if (col + per <= cols) {
                    *reinterpret_cast<uint4*>(g) = *box_at(box, r, c);
                } else {
                    const T* e = reinterpret_cast<const T*>(box_at(box, r, c));
                    for (int k = 0; k < cols - col; ++k) g[k] = e[k];
                }
            }
        }
    } else {
        constexpr int rows_at_once = 32 / width;  // one (codes) or two (fp32)
        const int j = lane % width, r_end = rows - row0 < 32 ? rows - row0 : 32;
        if (col0 + j < cols) {
            T* g = base + (int64_t)(row0 + lane / width) * ld + col0 + j;
            for (int r = lane / width; r < r_end; r += rows_at_once, g += rows_at_once * ld)
                *g = reinterpret_cast<const T*>(box_at(box, r, j / per))[j % per];
        }
    }
}
// global -> box in two steps, so that the loads are on their way while something else is done: pieces of 16 bytes in registers (vec
// and a whole row of the box inside the matrix), else elements when they are put.  Zeros beyond the matrix.
struct Fetched {
    uint4 v[4];
};
template <typename T>
__device__ __forceinline__ bool fetch_whole(int col0, int cols, bool vec) { return vec && col0 + 64 / (int)sizeof(T) <= cols; }
template <typename T>
__device__ __forceinline__ void box_fetch(Fetched& f, const T* base, int64_t ld, int row0, int rows, int col0, int cols, int lane, bool vec) {
    if (!fetch_whole<T>(col0, cols, vec)) return;
    const T* g = base + (int64_t)(row0 + (lane >> 2)) * ld + col0 + (lane & 3) * (16 / (int)sizeof(T));
#pragma unroll
    for (int i = 0; i < 4; ++i, g += 8 * ld)
        f.v[i] = row0 + i * 8 + (lane >> 2) < rows ? *reinterpret_cast<const uint4*>(g) : make_uint4(0, 0, 0, 0);
}
template <typename T>
__device__ __forceinline__ void box_put(uint8_t* box, const Fetched& f, const T* base, int64_t ld, int row0, int rows, int col0, int cols,
                                        int lane, bool vec) {
    constexpr int per = 16 / (int)sizeof(T), width = 64 / (int)sizeof(T);
    if (fetch_whole<T>(col0, cols, vec)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *box_at(box, i * 8 + (lane >> 2), lane & 3) = f.v[i];
    } else {
        constexpr int rows_at_once = 32 / width;
        const int j = lane % width;
        const bool there = col0 + j < cols;
        const T* g = base + (int64_t)(row0 + lane / width) * ld + col0 + j;
#pragma unroll 8
        for (int r = lane / width; r < 32; r += rows_at_once, g += rows_at_once * ld) {
            T e = T(0.0f);
            if (there && row0 + r < rows) e = *g;
            reinterpret_cast<T*>(box_at(box, r, j / per))[j % per] = e;
        }
    }
}
// fp32 pairs to two codes and back, rounded to nearest even
template <typename T>
__device__ __forceinline__ uint32_t pack_codes(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack_codes<__half>(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack_codes<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ float2 unpack_codes(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack_codes<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <>
__device__ __forceinline__ float2 unpack_codes<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
// the lane's row of 32 fp32 values, in pairs -> box, as codes
template <typename T>
__device__ __forceinline__ uint32_t pack_pair(pair_t v) {
    const float2 f = split_pair(v);
    return pack_codes<T>(f.x, f.y);
}
template <typename T>
__device__ __forceinline__ void box_put_codes(uint8_t* box, int lane, const pair_t (&v)[16]) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *box_at(box, lane, c) = make_uint4(pack_pair<T>(v[c * 4]), pack_pair<T>(v[c * 4 + 1]), pack_pair<T>(v[c * 4 + 2]), pack_pair<T>(v[c * 4 + 3]));
}
// box -> the lane's row of 32 codes, two at a time: f(pair's index, values)
template <typename T, typename F>
__device__ __forceinline__ void box_each(uint8_t* box, int lane, F f) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint4 w = *box_at(box, lane, c);
        f(c * 4, unpack_codes<T>(w.x));
        f(c * 4 + 1, unpack_codes<T>(w.y));
        f(c * 4 + 2, unpack_codes<T>(w.z));
        f(c * 4 + 3, unpack_codes<T>(w.w));
    }
}
// Sums over the warp's 32 rows of its 32 columns; lane l returns the sum of column l, in a fixed order.  Through the box, 16 columns
// at a time: a lane puts its row, then adds two columns of eight rows, and three other lanes have the other rows.  (56 instructions;
// exchanging halves by shuffles takes 124.)
__device__ __forceinline__ float column_sum(uint8_t* box, int lane, const pair_t (&v)[16]) {
    float mine = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 a = split_pair(v[h * 8 + k * 2]), b = split_pair(v[h * 8 + k * 2 + 1]);
            *reinterpret_cast<float4*>(box_at(box, lane, k)) = make_float4(a.x, a.y, b.x, b.y);
        }
        __syncwarp();
        // columns 2 (lane % 8), + 1; rows lane / 8, + 4, ...: the eight lanes of a row read its 64 bytes
        const int two = lane & 7;
        pair_t s = 0ull;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = (lane >> 3) + i * 4;
            const pair_t w = reinterpret_cast<const pair_t*>(box_at(box, row, two >> 1))[two & 1];
            s = i == 0 ? w : add2(s, w);
        }
        float2 f = split_pair(s);
        f.x = __fadd_rn(f.x, __shfl_xor_sync(0xFFFFFFFFu, f.x, 8));
        f.y = __fadd_rn(f.y, __shfl_xor_sync(0xFFFFFFFFu, f.y, 8));
        f.x = __fadd_rn(f.x, __shfl_xor_sync(0xFFFFFFFFu, f.x, 16));
        f.y = __fadd_rn(f.y, __shfl_xor_sync(0xFFFFFFFFu, f.y, 16));
        // column 16 h + c to lane 16 h + c: it is with lane c / 2, as its c % 2
        const float x = __shfl_sync(0xFFFFFFFFu, f.x, (lane & 15) >> 1), y = __shfl_sync(0xFFFFFFFFu, f.y, (lane & 15) >> 1);
        if ((lane >> 4) == h) mine = (lane & 1) ? y : x;
        __syncwarp();
    }
    return mine;
}

template <bool kPair>
__device__ __forceinline__ uint32_t make_idesc(int a_mn, int b_mn, int bf16) {
    const uint32_t ab = bf16 ? 1u : 0u;
    return (1u << 4) | (ab << 7) | (ab << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(kTileN >> 3) << 17) |
           ((uint32_t)((kPair ? 2 * kRows : kRows) >> 4) << 24);
}

template <typename Epi, bool kPair, bool kLong>
__device__ __forceinline__ void product16_body(const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_alt,
                                               const ProductParams& p, const typename Epi::Params& ep) {
    using S = Staging<kPair>;
    constexpr int kStages = S::kStages, kTileM = kPair ? 2 * kRows : kRows;
    constexpr uint32_t kStageBytes = S::kBytes, kStageA = S::kA;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = ptx::smem_addr(smem_raw);
    const uint32_t tiles = (raw + 1023u) & ~1023u;
    const uint32_t boxes = tiles + kStages * kStageBytes, bars = boxes + kEpiWarps * kBoxBytes;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (kStages + s); };
    auto acc_full_bar = [&](int a) { return bars + 8u * (2 * kStages + a); };
    auto acc_empty_bar = [&](int a) { return bars + 8u * (2 * kStages + 2 + a); };
    uint8_t* const gen_bars = smem_raw + (bars - raw);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(gen_bars + 8 * (2 * kStages + 4));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(gen_bars + 8 * (2 * kStages + 4) + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = kPair ? ptx::cluster_ctarank() : 0u;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            ptx::mbar_init(full_bar(s), kPair ? 2 : 1);
            ptx::mbar_init(empty_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            ptx::mbar_init(acc_full_bar(a), 1);
            ptx::mbar_init(acc_empty_bar(a), (kPair ? 2 : 1) * kEpiWarps);
        }
        *abort_flag = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 1) {
        const uint32_t slot = ptx::smem_addr(const_cast<uint32_t*>(tmem_slot));
        if (kPair) {
            ptx::tmem_alloc_pair(slot, kTmemCols);
            ptx::tmem_relinquish_pair();
        } else {
            ptx::tmem_alloc(slot, kTmemCols);
            ptx::tmem_relinquish();
        }
    }
    // global memory from here on
    grid_dependency_wait();
    announce_launch(p.status, p.tag);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (kPair) ptx::cluster_sync();  // the peer's barriers exist before anything is signalled to them
    ptx::tc_fence_after_sync();
    grid_launch_dependents();
    const uint32_t tmem_base = *tmem_slot;

    const int count = p.dyn != kFixed || p.alt != kAltNone ? *p.count : 0;
    const int M = p.dyn == kCountM ? count : p.M, K = p.dyn == kCountK ? count : p.K;
    const bool use_alt = p.alt != kAltNone && count == p.alt_rows;
    const int tiles_m = (M + kTileM - 1) / kTileM, tiles_n = (p.N + kTileN - 1) / kTileN;
    const int kb_total = (K + kStageK - 1) / kStageK;
    const int items = tiles_m * tiles_n * p.splits;
    const int workers = kPair ? gridDim.x >> 1 : gridDim.x, first = kPair ? blockIdx.x >> 1 : blockIdx.x;
    // item t: tile t % (tiles_m tiles_n), rows of tiles first so that pairs side by side read the same columns of B
    auto stages_of = [&](int t, int* begin) {
        const int split = t / (tiles_m * tiles_n);
        *begin = split * p.kb_per_split;
        const int left = kb_total - *begin;
        return left < 0 ? 0 : (left < p.kb_per_split ? left : p.kb_per_split);
    };

    if (warp == 0 || warp == 3) {
        if (lane == 0) {
            const CUtensorMap* const ma = use_alt && p.alt == kAltA ? &map_alt : &map_a;
            const CUtensorMap* const mb = use_alt && p.alt == kAltB ? &map_alt : &map_b;
            const uint32_t who = warp == 0 ? 0u : 1u;
            uint32_t seq = 0, phase = 0;
            int stage = 0;
            bool dead = false;
            for (int t = first; t < items && !dead && !*abort_flag; t += workers) {
                const int tile = t % (tiles_m * tiles_n);
                const int m0 = (tile % tiles_m) * kTileM + (int)rank * kRows, n0 = (tile / tiles_m) * kTileN + (int)rank * S::kColumns;
                int kb0;
                const int nkb = stages_of(t, &kb0);
                for (int kb = kb0; kb < kb0 + nkb; ++kb) {
                    if ((seq++ & 1u) != who) {  // the other producer's stage
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                        continue;
                    }
                    if (!ptx::mbar_wait_bounded(empty_bar(stage), phase ^ 1u, kWaitLimit)) {
                        raise_timeout(p.status, p.tag, abort_flag);
                        dead = true;
                        break;
                    }
                    const uint32_t sa = tiles + stage * kStageBytes, sb = sa + kStageA;
                    const uint32_t bar = kPair ? ptx::map_to_cta(full_bar(stage), 0) : full_bar(stage);
                    const int k0 = kb * kStageK;
                    if (kPair) ptx::mbar_expect_tx_cluster(bar, kStageBytes);
                    else ptx::mbar_expect_tx(bar, kStageBytes);
                    auto load = [&](uint32_t dst, const CUtensorMap* m, int columns, int x0, bool mn, bool blocked) {
                        if (blocked) {
                            if (kPair) ptx::tma_load_3d_pair(dst, m, bar, 0, k0, x0 >> 6);
                            else ptx::tma_load_3d(dst, m, bar, 0, k0, x0 >> 6);
                        } else if (mn) {
                            for (int c = 0; c < columns / 64; ++c) {
                                if (kPair) ptx::tma_load_2d_pair(dst + c * 8192u, m, bar, x0 + c * 64, k0);
                                else ptx::tma_load_2d(dst + c * 8192u, m, bar, x0 + c * 64, k0);
                            }
                        } else {
                            if (kPair) ptx::tma_load_2d_pair(dst, m, bar, k0, x0);
                            else ptx::tma_load_2d(dst, m, bar, k0, x0);
                        }
                    };
                    load(sa, ma, kRows, m0, p.a_mn != 0, p.a_blocked != 0);
                    load(sb, mb, S::kColumns, n0, p.b_mn != 0, p.b_blocked != 0);
                    if (++stage == kStages) { stage = 0; phase ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = make_idesc<kPair>(p.a_mn, p.b_mn, p.bf16);
            // K-major tile: 128-byte rows, 32 bytes a step.  MN-major: blocks of 64 columns x 64 K rows (8192 bytes), 16 K
            // rows a step.
            const uint32_t a_step = (p.a_mn ? 2048u : 32u) >> 4, b_step = (p.b_mn ? 2048u : 32u) >> 4;
            const uint32_t hi = desc_hi(1024u, kLayoutSw128);
            const uint32_t a_lo = desc_lo(tiles, p.a_mn ? 8192u : 16u), b_lo = desc_lo(tiles + kStageA, p.b_mn ? 8192u : 16u);
            int stage = 0;
            uint32_t phase = 0, it = 0;
            bool dead = false;
            for (int t = first; t < items && !dead; t += workers) {
                int kb0;
                const int nkb = stages_of(t, &kb0);
                for (int from = 0; from < nkb && !dead; from += kLong ? kCloseStages : nkb) {
                    const int until = kLong && nkb - from > kCloseStages ? kCloseStages : nkb - from;
                    const uint32_t acc = it & 1u, acc_phase = (it >> 1) & 1u;
                    ++it;
                    if (!ptx::mbar_wait_bounded(acc_empty_bar(acc), acc_phase ^ 1u, kWaitLimit)) {
                        raise_timeout(p.status, p.tag, abort_flag);
                        dead = true;
                        break;
                    }
                    ptx::tc_fence_after_sync();
                    const uint32_t d = tmem_base + acc * kAccCols;
                    for (int kb = 0; kb < until; ++kb) {
                        if (!ptx::mbar_wait_bounded(full_bar(stage), phase, kWaitLimit)) {
                            raise_timeout(p.status, p.tag, abort_flag);
                            dead = true;
                            break;
                        }
                        ptx::tc_fence_after_sync();
                        const uint32_t off = (uint32_t)stage * (kStageBytes >> 4);
#pragma unroll
                        for (int k = 0; k < kStageK / 16; ++k) {
                            const uint64_t da = desc_join(hi, a_lo + off + k * a_step), db = desc_join(hi, b_lo + off + k * b_step);
                            if (kPair) ptx::mma_f16_pair(d, da, db, idesc, (kb | k) != 0 ? 1u : 0u);
                            else ptx::mma_f16(d, da, db, idesc, (kb | k) != 0 ? 1u : 0u);
                        }
                        if (kPair) ptx::mma_commit_pair(empty_bar(stage), 3);
                        else ptx::mma_commit(empty_bar(stage));
                        if (++stage == kStages) { stage = 0; phase ^= 1u; }
                    }
                    if (dead) break;
                    if (kPair) ptx::mma_commit_pair(acc_full_bar(acc), 3);
                    else ptx::mma_commit(acc_full_bar(acc));
                }
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        Patch pt;
        pt.lane = lane;
        pt.quad = warp & 3;
        pt.warp = warp - 4;
        pt.box = smem_raw + (boxes - raw) + pt.warp * kBoxBytes;
        pt.rows = M;
        pt.cols = p.N;
        float sums[kLong ? 64 : 1];
        pt.closed = nullptr;
        const int quarter = pt.warp >> 2;
        uint32_t it = 0;
        for (int t = first; t < items; t += workers) {
            const int tile = t % (tiles_m * tiles_n);
            int kb0;
            const int nkb = stages_of(t, &kb0);
            pt.split = t / (tiles_m * tiles_n);
            pt.tile_m = tile % tiles_m;
            pt.tile_n = tile / tiles_m;
            pt.row0 = pt.tile_m * kTileM + (int)rank * kRows + pt.quad * 32;
            pt.col0 = pt.tile_n * kTileN + quarter * 64;
            pt.empty = nkb == 0;
            uint32_t acc = it & 1u, acc_phase = (it >> 1) & 1u;
            pt.tmem = tmem_base + ((uint32_t)(pt.quad * 32) << 16) + acc * kAccCols + (uint32_t)quarter * 64u;
            typename Epi::Ahead ahead;
            Epi::before(pt, ep, ahead);
            auto complete = [&] {  // waits for the accumulator
                ++it;
                bool ok = true;
                if (lane == 0) ok = ptx::mbar_wait_bounded(acc_full_bar(acc), acc_phase, kWaitLimit);
                ok = __shfl_sync(0xFFFFFFFFu, ok ? 1 : 0, 0) != 0;
                if (!ok && lane == 0) raise_timeout(p.status, p.tag, abort_flag);
                if (!ok || *abort_flag) return false;
                ptx::tc_fence_after_sync();
                return true;
            };
            auto release = [&](uint32_t bar) {  // the accumulator has been read
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if (kPair) ptx::mbar_arrive_cluster(bar);
                    else ptx::mbar_arrive(bar);
                }
            };
            auto empty_of = [&] { return kPair ? ptx::map_to_cta(acc_empty_bar(acc), 0) : acc_empty_bar(acc); };
            if (nkb != 0 && !complete()) break;
            if constexpr (kLong) {
                pt.closed = nullptr;
                bool ok = true;
                for (int left = nkb; left > kCloseStages && ok; left -= kCloseStages) {
                    pt.close(sums);
                    release(empty_of());
                    acc = it & 1u;
                    acc_phase = (it >> 1) & 1u;
                    pt.tmem = tmem_base + ((uint32_t)(pt.quad * 32) << 16) + acc * kAccCols + (uint32_t)quarter * 64u;
                    ok = complete();
                }
                if (!ok) break;
            }
            const uint32_t bar = empty_of();
            Epi::run(pt, ep, ahead, [&] {
                if (nkb != 0) release(bar);
            });
        }
        __syncwarp();
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {  // copies in flight land before the shared memory goes
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
    if (kPair) ptx::cluster_sync();  // neither CTA leaves while the other may still signal it
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        if (kPair) ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
        else ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

template <typename Epi, bool kLong>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
product16_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                      const __grid_constant__ CUtensorMap map_alt, const ProductParams p, const typename Epi::Params ep) {
    product16_body<Epi, true, kLong>(map_a, map_b, map_alt, p, ep);
}
template <typename Epi, bool kLong>
__global__ void __launch_bounds__(kThreads, 1)
product16_single_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                        const __grid_constant__ CUtensorMap map_alt, const ProductParams p, const typename Epi::Params ep) {
    product16_body<Epi, false, kLong>(map_a, map_b, map_alt, p, ep);
}

// ---- host side --------------------------------------------------------------------------------------------------------

// How a product is laid over the GPU: CTA pairs or single CTAs, and parts of K.
struct ProductPlan {
    bool pair;
    int splits, kb_per_split;
};
constexpr int64_t kPairs = 74, kSingles = 148;  // the plan goes by a whole GPU, so that workspaces are sized without asking a device
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t pair_tiles(int64_t M, int64_t N) { return ceil_div(M, 2 * kRows) * ceil_div(N, kTileN); }
inline int64_t single_tiles(int64_t M, int64_t N) { return ceil_div(M, kRows) * ceil_div(N, kTileN); }

// Single CTAs where every tile of theirs is worked on at once, or where they need at least a quarter fewer rounds.
// A product of fewer tiles than workers shares its K among them (if `share`), in pieces of at least four stages (256 elements) and at most
// 16: shorter ones would cost more in moving fp32 sums than they save.
inline ProductPlan plan_product(int64_t M, int64_t N, int64_t K, bool share) {
    ProductPlan plan;
    const int64_t pairs = pair_tiles(M, N), singles = single_tiles(M, N), stages = ceil_div(K, kStageK);
    const int64_t pair_rounds = ceil_div(pairs, kPairs), single_rounds = ceil_div(singles, kSingles);
    plan.pair = singles > kSingles && 4 * single_rounds > 3 * pair_rounds;
    const int64_t tiles = plan.pair ? pairs : singles, workers = plan.pair ? kPairs : kSingles;
    int64_t n = !share || tiles == 0 ? 1 : workers / tiles;
    if (n > stages / 4) n = stages / 4;
    if (n > 16) n = 16;
    if (n < 1) n = 1;
    plan.kb_per_split = (int)ceil_div(stages, n);
    plan.splits = plan.kb_per_split > 0 ? (int)ceil_div(stages, plan.kb_per_split) : 1;
    return plan;
}

// An operand of M (or N) x K elements as the kernel fetches it; *blocked: see make_operand_map16.
struct Operand {
    CUtensorMap map;
    int mn, blocked;
};
inline int make_operand(Operand* o, bool is_b, bool pair, const void* ptr, bool mn, int64_t extent, int64_t k, int64_t ld) {
    o->mn = mn ? 1 : 0;
    return make_operand_map16(&o->map, reinterpret_cast<const uint16_t*>(ptr), mn, (uint64_t)extent, (uint64_t)k, (uint64_t)ld,
                              is_b && !pair ? kTileN : kRows, &o->blocked);
}

template <typename Epi, bool kLong>
int launch_product_of(bool pair, const Operand& a, const Operand& b, const CUtensorMap& alt, const ProductParams& p, const typename Epi::Params& ep,
                      const DeviceInfo& dev, cudaStream_t stream) {
    static std::atomic<bool> ready[64];
    const bool known = dev.ordinal >= 0 && dev.ordinal < 64;
    auto* const pairs = product16_pair_kernel<Epi, kLong>;
    auto* const singles = product16_single_kernel<Epi, kLong>;
    if (!known || !ready[dev.ordinal].load()) {
        QFMT_CUDA_TRY(cudaFuncSetAttribute(pairs, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<true>()));
        QFMT_CUDA_TRY(cudaFuncSetAttribute(singles, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<false>()));
        if (known) ready[dev.ordinal].store(true);
    }
    const int64_t items = (pair ? pair_tiles(p.M, p.N) : single_tiles(p.M, p.N)) * p.splits;
    const int64_t most = pair ? dev.sm_count / 2 : dev.sm_count, workers = items < most ? items : most;
    if (workers == 0) return QFMT_OK;
    if (pair) QFMT_CUDA_TRY(launch_overlapping(pairs, (unsigned)(2 * workers), (unsigned)kThreads, smem_bytes<true>(), stream, a.map, b.map, alt, p, ep));
    else QFMT_CUDA_TRY(launch_overlapping(singles, (unsigned)workers, (unsigned)kThreads, smem_bytes<false>(), stream, a.map, b.map, alt, p, ep));
    return QFMT_OK;
}

// Workspace words, statuses and operands are the caller's; the plan's splits are in p.
template <typename Epi>
int launch_product(bool pair, const Operand& a, const Operand& b, const Operand* alt, ProductParams p, const typename Epi::Params& ep,
                   const DeviceInfo& dev, cudaStream_t stream) {
    p.a_mn = a.mn;
    p.b_mn = b.mn;
    p.a_blocked = a.blocked;
    p.b_blocked = b.blocked;
    const CUtensorMap& other = alt != nullptr ? alt->map : a.map;
    if (p.kb_per_split > kCloseStages) return launch_product_of<Epi, true>(pair, a, b, other, p, ep, dev, stream);
    return launch_product_of<Epi, false>(pair, a, b, other, p, ep, dev, stream);
}

}  // namespace p16
}  // namespace qfmt
