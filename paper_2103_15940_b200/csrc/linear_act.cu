// Products of 16-bit codes with bias, activation and residual in the epilogue, their backward pass, and the pass over a gradient
// that is there already:
//     z = X W + bias,  y = act(z) + residual;      dz = (dY W^T + residual) act'(z),  dbias = column sums of dz.
// Formulas: activation.cuh; the product's frame: product16.cuh.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "activation.cuh"
#include "columns.cuh"
#include "common.cuh"
#include "product16.cuh"
#include "skinny16.cuh"

namespace qfmt {
namespace {

using p16::Patch;

struct Nothing {};

// ---- epilogues of the product -------------------------------------------------------------------------------------------

template <typename T, int kAct>
struct ForwardEpilogue {
    struct Params {
        const float* bias;
        const T* residual;
        T *z, *y;
        int64_t ld_residual, ld_z, ld_y;
        int vec_residual, vec_z, vec_y;
    };
    struct Ahead {
        p16::Fetched residual;
        float bias[2];
    };
    static __device__ __forceinline__ void fetch(const Patch& p, const Params& e, Ahead& a, int col0) {
        if (e.residual != nullptr)
            p16::box_fetch<T>(a.residual, e.residual, e.ld_residual, p.row0, p.rows, col0, p.cols, p.lane, e.vec_residual != 0);
    }
    static __device__ __forceinline__ void before(const Patch& p, const Params& e, Ahead& a) {
        p.columns(e.bias, a.bias);
        fetch(p, e, a, p.col0);
    }
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead& a, F release) {
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            const int col0 = p.col0 + c * 32;
            pair_t v[16];
            p.load_pairs<true>(c, v, c == 0 ? a.bias[0] : a.bias[1]);
            if (c == 1) release();
            if (col0 >= p.cols || p.row0 >= p.rows) continue;
            if (e.z != nullptr) {
                p16::box_put_codes<T>(p.box, p.lane, v);
                __syncwarp();
                p16::box_store<T>(p.box, e.z, e.ld_z, p.row0, p.rows, col0, p.cols, p.lane, e.vec_z != 0);
                __syncwarp();
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = activate2<kAct>(v[j]);
            if (e.residual != nullptr) {
                p16::box_put<T>(p.box, a.residual, e.residual, e.ld_residual, p.row0, p.rows, col0, p.cols, p.lane, e.vec_residual != 0);
                __syncwarp();
                if (c == 0) fetch(p, e, a, col0 + 32);
                p16::box_each<T>(p.box, p.lane, [&](int j, float2 r) { v[j] = add2(v[j], make_pair(r.x, r.y)); });
                __syncwarp();
            }
            p16::box_put_codes<T>(p.box, p.lane, v);
            __syncwarp();
            p16::box_store<T>(p.box, e.y, e.ld_y, p.row0, p.rows, col0, p.cols, p.lane, e.vec_y != 0);
            __syncwarp();
        }
    }
};

template <typename T, int kAct>
struct BackwardEpilogue {
    struct Params {
        const T *residual, *z;
        T* dz;
        float* parts;  // [32-row groups][pitch] column sums, or null
        int64_t ld_residual, ld_z, ld_dz, pitch;
        int vec_residual, vec_z, vec_dz;
    };
    // z is on its way while the tile is summed; the residual where there is no z (both would not fit the registers)
    struct Ahead {
        p16::Fetched f;
    };
    static __device__ __forceinline__ void fetch_residual(const Patch& p, const Params& e, p16::Fetched& f, int col0) {
        p16::box_fetch<T>(f, e.residual, e.ld_residual, p.row0, p.rows, col0, p.cols, p.lane, e.vec_residual != 0);
    }
    static __device__ __forceinline__ void fetch(const Patch& p, const Params& e, Ahead& a, int col0) {
        if (kAct != QFMT_ACT_NONE) p16::box_fetch<T>(a.f, e.z, e.ld_z, p.row0, p.rows, col0, p.cols, p.lane, e.vec_z != 0);
        else if (e.residual != nullptr) fetch_residual(p, e, a.f, col0);
    }
    static __device__ __forceinline__ void before(const Patch& p, const Params& e, Ahead& a) { fetch(p, e, a, p.col0); }
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead& a, F release) {
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            const int col0 = p.col0 + c * 32;
            pair_t v[16];
            p.load_pairs<false>(c, v);
            if (c == 1) release();
            if (col0 >= p.cols) continue;
            if (p.row0 + p.lane >= p.rows) {  // rows beyond the matrix are zeros, but not their products with infinite weights
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = 0ull;
            }
            if (e.residual != nullptr) {
                p16::Fetched late;
                if (kAct != QFMT_ACT_NONE) fetch_residual(p, e, late, col0);
                p16::box_put<T>(p.box, kAct != QFMT_ACT_NONE ? late : a.f, e.residual, e.ld_residual, p.row0, p.rows, col0, p.cols, p.lane,
                                e.vec_residual != 0);
                __syncwarp();
                p16::box_each<T>(p.box, p.lane, [&](int j, float2 r) { v[j] = add2(v[j], make_pair(r.x, r.y)); });
                __syncwarp();
            }
            if (kAct != QFMT_ACT_NONE) {
                p16::box_put<T>(p.box, a.f, e.z, e.ld_z, p.row0, p.rows, col0, p.cols, p.lane, e.vec_z != 0);
                __syncwarp();
            }
            if (c == 0) fetch(p, e, a, col0 + 32);
            if (kAct != QFMT_ACT_NONE) {
                p16::box_each<T>(p.box, p.lane, [&](int j, float2 z) { v[j] = mul2(v[j], slope2<kAct>(z.x, z.y)); });
                __syncwarp();
            }
            p16::box_put_codes<T>(p.box, p.lane, v);
            __syncwarp();
            p16::box_store<T>(p.box, e.dz, e.ld_dz, p.row0, p.rows, col0, p.cols, p.lane, e.vec_dz != 0);
            __syncwarp();
            if (e.parts != nullptr) {
                const float s = p16::column_sum(p.box, p.lane, v);
                if (col0 + p.lane < p.cols) e.parts[(int64_t)(p.row0 >> 5) * e.pitch + col0 + p.lane] = s;
            }
        }
    }
};

// Sums as they are, in fp32, to [split][M][pitch]: products of few tiles whose K is shared.
struct PartEpilogue {
    struct Params {
        float* parts;
        int64_t pitch, split_stride;
    };
    using Ahead = Nothing;
    static __device__ __forceinline__ void before(const Patch&, const Params&, Ahead&) {}
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead&, F release) {
        float* base = e.parts + (int64_t)p.split * e.split_stride;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            uint32_t a[32];
            p.load32(c, a);
            p.finish(c, a);
            if (c == 1) release();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col0 = p.col0 + c * 32 + h * 16;
                if (p.row0 >= p.rows || col0 >= p.cols) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *p16::box_at(p.box, p.lane, k) = make_uint4(a[16 * h + 4 * k], a[16 * h + 4 * k + 1], a[16 * h + 4 * k + 2], a[16 * h + 4 * k + 3]);
                __syncwarp();
                p16::box_store<float>(p.box, base, e.pitch, p.row0, p.rows, col0, p.cols, p.lane, true);
                __syncwarp();
            }
        }
    }
};

// ---- the pass over rows -------------------------------------------------------------------------------------------------
// Finishes a product whose K was shared (kParts: the source is [splits][rows][pitch] fp32) or works on a gradient that is in
// memory.  A block has a strip of 256 columns and a range of rows, a warp a row at a time and a lane eight columns of it: whole
// 16-byte pieces (32 bytes of containers) if everything is aligned (kVec), else every 32nd element so that accesses still join.
// Column sums stay in registers down the rows and are joined across the block's eight warps, then across blocks by
// join_columns_kernel.  Bound by memory: with two tensors read and one written 8192 x 4096 bfloat16 moves 201 MB.
struct RowPass {
    const float* parts;
    int splits;
    int64_t split_stride, pitch;       // pitch of the fp32 sources, and of the column sums
    const void *dy, *residual, *z_in;
    void *out, *z_out;
    const float* bias;
    float* sums;                       // [row blocks][pitch], or null
    int64_t ld_dy, ld_residual, ld_z, ld_out;
    int64_t rows, cols;
    int strips;
    int64_t rows_per_block;
};

template <typename T, bool kVec>
__device__ __forceinline__ int64_t pass_col(int lane, int k) { return kVec ? lane * 8 + k : k * 32 + lane; }

// A lane's eight elements of a row; `p` is the row's first element of the strip and `there` says which of them exist (bit k; in
// whole pieces all or none).
template <typename T, bool kVec>
__device__ __forceinline__ void pass_load(const T* p, unsigned there, int lane, float (&v)[8]) {
    if (kVec) {
        if (!there) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
        } else {
            const uint4* q = reinterpret_cast<const uint4*>(p + lane * 8);
            uint4 w[sizeof(T) / 2];
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = q[i];
            const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = (float)e[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (there >> k) & 1u ? (float)p[k * 32 + lane] : 0.0f;
    }
}
__device__ __forceinline__ float to_type(float v, float) { return v; }
__device__ __forceinline__ __half to_type(float v, __half) { return __float2half_rn(v); }
__device__ __forceinline__ __nv_bfloat16 to_type(float v, __nv_bfloat16) { return __float2bfloat16_rn(v); }

template <typename T, bool kVec>
__device__ __forceinline__ void pass_store(T* p, unsigned there, int lane, const float (&v)[8]) {
    if (kVec) {
        if (!there) return;
        uint4 w[sizeof(T) / 2];
        T* e = reinterpret_cast<T*>(w);
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = to_type(v[k], T());
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p + lane * 8)[i] = w[i];
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if ((there >> k) & 1u) p[k * 32 + lane] = to_type(v[k], T());
        }
    }
}

constexpr int kPassWarps = 8, kPassPerSm = 4;

// Whole pieces of a gradient come through a ring in shared memory, a lane's own pieces at its own place, so that several rows of every warp
// are on their way at all times without holding registers: with the loads of one row at a time 8192 x 4096 bfloat16 takes 54 to 56 us,
// whether with 16, 32 or 48 warps an SM.
template <typename T, int kAct, bool kBackward, bool kParts, bool kVec>
__global__ void __launch_bounds__(kPassWarps * 32, 4)
row_pass_kernel(const RowPass a) {
    constexpr bool kPrecise = sizeof(T) == 4, kRing = kVec && !kParts, kZ = kAct != QFMT_ACT_NONE;
    constexpr int kPieces = (int)sizeof(T) / 2 * (kZ ? 2 : 1);   // 16-byte pieces of a row and lane
    constexpr int kDepth = 8 / kPieces;                          // rows on their way
    __shared__ float sums[kPassWarps][256];
    __shared__ uint4 ring[kRing ? kDepth : 1][kPieces][kPassWarps * 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col0 = (int64_t)(blockIdx.x % a.strips) * 256;
    const int64_t block = blockIdx.x / a.strips, first = block * a.rows_per_block;
    const int64_t end = first + a.rows_per_block < a.rows ? first + a.rows_per_block : a.rows;
    unsigned there = 0u;
#pragma unroll
    for (int k = 0; k < 8; ++k) there |= col0 + pass_col<T, kVec>(lane, k) < a.cols ? 1u << k : 0u;
    grid_dependency_wait();
    grid_launch_dependents();
    float bias[8], total[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        bias[k] = !kBackward && a.bias != nullptr && ((there >> k) & 1u) ? a.bias[col0 + pass_col<T, kVec>(lane, k)] : 0.0f;
        total[k] = 0.0f;
    }
    const T *residual = static_cast<const T*>(a.residual), *z_in = static_cast<const T*>(a.z_in);
    T *out = static_cast<T*>(a.out), *z_out = static_cast<T*>(a.z_out);
    const T* const dy = static_cast<const T*>(a.dy);
    auto ask = [&](int64_t row, int slot) {
        if (row < end && there) {
            const T* p = dy + row * a.ld_dy + col0 + lane * 8;
            const T* q = kZ ? z_in + row * a.ld_z + col0 + lane * 8 : nullptr;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint4* from = i < (int)sizeof(T) / 2 ? reinterpret_cast<const uint4*>(p) + i : reinterpret_cast<const uint4*>(q) + (i - (int)sizeof(T) / 2);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_addr(&ring[slot][i][threadIdx.x])), "l"(from) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");  // committed even when empty: the waits count groups
    };
    int slot = 0;
    if constexpr (kRing) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) ask(first + warp + i * kPassWarps, i);
    }
#pragma unroll 1
    for (int64_t row = first + warp; row < end; row += kPassWarps) {
        float v[8], z[8];
        if constexpr (kRing) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
            uint4 w[kPieces];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) w[i] = ring[slot][i][threadIdx.x];
            ask(row + kDepth * kPassWarps, slot);
            slot = slot + 1 == kDepth ? 0 : slot + 1;
            const T* e = reinterpret_cast<const T*>(w);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = (float)e[k];
                if (kZ) z[k] = (float)e[8 + k];
            }
        } else if constexpr (kParts) {
            const float* part = a.parts + row * a.pitch + col0;
            pass_load<float, kVec>(part, there, lane, v);
#pragma unroll 2
            for (int s = 1; s < a.splits; ++s) {
                float w[8];
                part += a.split_stride;
                pass_load<float, kVec>(part, there, lane, w);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __fadd_rn(v[k], w[k]);
            }
        } else {
            pass_load<T, kVec>(dy + row * a.ld_dy + col0, there, lane, v);
        }
        float r[8];
        if (kBackward) {
            if constexpr (kAct != QFMT_ACT_NONE) {
                if constexpr (!kRing) pass_load<T, kVec>(z_in + row * a.ld_z + col0, there, lane, z);
                if (residual != nullptr) {
                    pass_load<T, kVec>(residual + row * a.ld_residual + col0, there, lane, r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = __fadd_rn(v[k], r[k]);
                }
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const float2 s = kPrecise ? make_float2(slope<kAct>(z[k]), slope<kAct>(z[k + 1])) : split_pair(slope2<kAct>(z[k], z[k + 1]));
                    v[k] = __fmul_rn(v[k], s.x);
                    v[k + 1] = __fmul_rn(v[k + 1], s.y);
                }
            } else if (residual != nullptr) {
                pass_load<T, kVec>(residual + row * a.ld_residual + col0, there, lane, r);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __fadd_rn(v[k], r[k]);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) total[k] = __fadd_rn(total[k], v[k]);
        } else {
            if (residual != nullptr) pass_load<T, kVec>(residual + row * a.ld_residual + col0, there, lane, r);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __fadd_rn(v[k], bias[k]);
            if (z_out != nullptr) pass_store<T, kVec>(z_out + row * a.ld_z + col0, there, lane, v);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float2 f = split_pair(activate2<kAct>(make_pair(v[k], v[k + 1])));
                v[k] = f.x;
                v[k + 1] = f.y;
            }
            if (residual != nullptr) {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __fadd_rn(v[k], r[k]);
            }
        }
        if (out != nullptr) pass_store<T, kVec>(out + row * a.ld_out + col0, there, lane, v);
    }
    if constexpr (kBackward) {
        if (a.sums == nullptr) return;
#pragma unroll
        for (int k = 0; k < 8; ++k) sums[warp][pass_col<T, kVec>(lane, k)] = total[k];
        __syncthreads();
        const int64_t col = col0 + threadIdx.x;
        if (col < a.cols) {
            float s = sums[0][threadIdx.x];
            for (int w = 1; w < kPassWarps; ++w) s = __fadd_rn(s, sums[w][threadIdx.x]);
            a.sums[block * a.pitch + col] = s;
        }
    }
}

// ---- small products ---------------------------------------------------------------------------------------------------------
// One launch: a block takes 32 rows and 16 (weights stored by output) or 64 outputs (by K), its warps share K, and up to eight blocks of a cluster share
// it again where that leaves more of the GPU with work.  The warps' sums meet in shared memory and the blocks' in the first one's, both
// in order; the epilogue takes two outputs a thread.
struct FewRows {
    skinny::Operands o;
    const float* bias;
    const void* residual;
    const void* z_in;
    void *out, *z_out;
    float* sums;  // column sums: of all rows, or [blocks of 32 rows][pitch]
    int64_t ld_residual, ld_z, ld_out, pitch;
    int k_warp;  // K elements of a warp, a multiple of 32
    unsigned long long* status;
    unsigned long long tag;
};
constexpr int kFewWarps = 8;

template <typename T, int kAct, bool kBackward, bool kByK, int kBlocks>
__global__ void __launch_bounds__(kFewWarps * 32, kByK || kBlocks > 2 ? 2 : 3)
few_rows_kernel(FewRows f) {
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    constexpr int kOutputs = kByK ? 64 : 16, kRows = kByK ? 16 * kBlocks : 8 * kBlocks, kPitch = kOutputs + 2, kElements = kRows * kPitch;
    extern __shared__ float few_sums[];  // [warps][rows][outputs]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    uint32_t rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    const int n0 = (int)(blockIdx.x / size) * kOutputs;
    {  // the block's rows as a matrix of its own
        const int64_t r0 = (int64_t)blockIdx.y * skinny::kMostRows;
        f.o.a += r0 * f.o.lda;
        f.o.rows = f.o.rows - r0 < skinny::kMostRows ? (int)(f.o.rows - r0) : skinny::kMostRows;
        f.residual = f.residual != nullptr ? static_cast<const T*>(f.residual) + r0 * f.ld_residual : nullptr;
        f.z_in = f.z_in != nullptr ? static_cast<const T*>(f.z_in) + r0 * f.ld_z : nullptr;
        f.z_out = f.z_out != nullptr ? static_cast<T*>(f.z_out) + r0 * f.ld_z : nullptr;
        f.out = static_cast<T*>(f.out) + r0 * f.ld_out;
        if (f.sums != nullptr) f.sums += blockIdx.y * f.pitch;
    }
    const int k0 = ((int)rank * kFewWarps + warp) * f.k_warp;
    skinny::prefetch_weights<kByK>(f.o, n0, k0, k0 + f.k_warp, lane);
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.y == 0) announce_launch(f.status, f.tag);
    float* mine = few_sums + warp * kElements;
    // what the epilogue of the thread's first two outputs needs is on its way meanwhile
    const T *residual = static_cast<const T*>(f.residual), *z_in = static_cast<const T*>(f.z_in);
    struct Two {
        float b0, b1, r0, r1, z0, z1;
    };
    auto operands = [&](int e) {
        Two v = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        const int row = e / (kOutputs / 2), n = n0 + e % (kOutputs / 2) * 2;
        if (row >= f.o.rows || n >= f.o.n) return v;
        const bool second = n + 1 < f.o.n;
        if (!kBackward && f.bias != nullptr) {
            v.b0 = f.bias[n];
            if (second) v.b1 = f.bias[n + 1];
        }
        if (residual != nullptr) {
            v.r0 = (float)residual[row * f.ld_residual + n];
            if (second) v.r1 = (float)residual[row * f.ld_residual + n + 1];
        }
        if (kBackward && kAct != QFMT_ACT_NONE) {
            v.z0 = (float)z_in[row * f.ld_z + n];
            if (second) v.z1 = (float)z_in[row * f.ld_z + n + 1];
        }
        return v;
    };
    Two first_two = operands(threadIdx.x);
    if constexpr (kByK) {
        float d[kBlocks][8][4] = {};
        skinny::by_k<kBf16, kBlocks, 1>(f.o, n0, k0, k0 + f.k_warp, lane, d);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float* p = mine + (b * 16 + g) * kPitch + 16 * t + i;
                p[0] = d[b][i][0];
                p[8] = d[b][i][1];
                p[8 * kPitch] = d[b][i][2];
                p[8 * kPitch + 8] = d[b][i][3];
            }
        }
    } else {
        float d[kBlocks][4] = {};
        skinny::by_output<kBf16, kBlocks, (kBlocks == 1 ? 4 : 2)>(f.o, n0, k0, k0 + f.k_warp, lane, d);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            float* p = mine + (b * 8 + 2 * t) * kPitch + g;
            p[0] = d[b][0];
            p[kPitch] = d[b][1];
            p[8] = d[b][2];
            p[kPitch + 8] = d[b][3];
        }
    }
    __syncthreads();
    const int rows = f.o.rows;
    for (int e = threadIdx.x; e < rows * kOutputs; e += kFewWarps * 32) {  // every element is one thread's
        float* p = few_sums + e / kOutputs * kPitch + e % kOutputs;
        float s = p[0];
#pragma unroll
        for (int w = 1; w < kFewWarps; ++w) s = __fadd_rn(s, p[w * kElements]);
        p[0] = s;
    }
    if (size > 1) {
        ptx::cluster_sync();
        if (rank == 0) {
            for (int e = threadIdx.x; e < rows * kOutputs; e += kFewWarps * 32) {
                float* p = few_sums + e / kOutputs * kPitch + e % kOutputs;
                const uint32_t at = ptx::smem_addr(p);
                float part[8], s = *p;
#pragma unroll
                for (int r = 1; r < 8; ++r) {
                    part[r] = 0.0f;
                    if (r < (int)size) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part[r]) : "r"(ptx::map_to_cta(at, r)) : "memory");
                }
#pragma unroll
                for (int r = 1; r < 8; ++r) {
                    if (r < (int)size) s = __fadd_rn(s, part[r]);
                }
                *p = s;
            }
        }
        ptx::cluster_sync();  // the other blocks' shared memory has been read
        if (rank != 0) return;
    }
    __syncthreads();
    T *out = static_cast<T*>(f.out), *z_out = static_cast<T*>(f.z_out);
    for (int e = threadIdx.x; e < rows * (kOutputs / 2); e += kFewWarps * 32) {
        const int row = e / (kOutputs / 2), c = e % (kOutputs / 2) * 2, n = n0 + c;
        if (n >= f.o.n) continue;
        const Two w = e < kFewWarps * 32 ? first_two : operands(e);
        const bool second = n + 1 < f.o.n;
        float* p = few_sums + row * kPitch + c;
        float v0 = p[0], v1 = p[1];
        if (kBackward) {
            v0 = __fadd_rn(v0, w.r0);
            v1 = __fadd_rn(v1, w.r1);
            if constexpr (kAct != QFMT_ACT_NONE) {
                const float2 s = split_pair(slope2<kAct>(w.z0, w.z1));
                v0 = __fmul_rn(v0, s.x);
                v1 = __fmul_rn(v1, s.y);
            }
            p[0] = v0;
            p[1] = v1;
        } else {
            v0 = __fadd_rn(v0, w.b0);
            v1 = __fadd_rn(v1, w.b1);
            if (z_out != nullptr) {
                T* z = z_out + row * f.ld_z + n;
                z[0] = to_type(v0, T());
                if (second) z[1] = to_type(v1, T());
            }
            const float2 a = split_pair(activate2<kAct>(make_pair(v0, v1)));
            v0 = residual != nullptr ? __fadd_rn(a.x, w.r0) : a.x;
            v1 = residual != nullptr ? __fadd_rn(a.y, w.r1) : a.y;
        }
        T* y = out + row * f.ld_out + n;
        y[0] = to_type(v0, T());
        if (second) y[1] = to_type(v1, T());
    }
    if (kBackward && f.sums != nullptr) {
        __syncthreads();
        if (threadIdx.x < kOutputs && n0 + (int)threadIdx.x < f.o.n) {
            float s = few_sums[threadIdx.x];
            for (int row = 1; row < rows; ++row) s = __fadd_rn(s, few_sums[row * kPitch + threadIdx.x]);
            f.sums[n0 + threadIdx.x] = s;
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------------

// Columns of fp32 working matrices are padded so that rows start on 32 bytes.
int64_t padded(int64_t cols) { return (cols + 7) / 8 * 8; }

// Blocks of rows of a pass: as many blocks as are on the GPU at a time, none of fewer than eight rows (one a warp).
constexpr int64_t kPassBlocks = 148 * kPassPerSm;
int64_t pass_row_blocks(int64_t rows, int64_t cols) {
    const int64_t strips = (cols + 255) / 256, most = (rows + 7) / 8;
    int64_t want = kPassBlocks / strips;
    if (want < 1) want = 1;
    return want < most ? want : most;
}

template <typename T, int kAct, bool kBackward, bool kParts>
int launch_row_pass(RowPass a, bool vec, cudaStream_t stream) {
    a.strips = (int)((a.cols + 255) / 256);
    const int64_t blocks = pass_row_blocks(a.rows, a.cols);
    a.rows_per_block = (a.rows + blocks - 1) / blocks;
    const unsigned grid = (unsigned)(a.strips * ((a.rows + a.rows_per_block - 1) / a.rows_per_block));
    if (vec) QFMT_CUDA_TRY(launch_overlapping(row_pass_kernel<T, kAct, kBackward, kParts, true>, grid, kPassWarps * 32u, 0, stream, a));
    else QFMT_CUDA_TRY(launch_overlapping(row_pass_kernel<T, kAct, kBackward, kParts, false>, grid, kPassWarps * 32u, 0, stream, a));
    return QFMT_OK;
}

bool misaligned(const void* p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }
// Whether rows can be moved in 16-byte pieces.
bool whole(const void* p, int64_t ld, int64_t size) { return p == nullptr || (!misaligned(p, 16) && (ld * size) % 16 == 0); }

struct Shape {
    int64_t M, N, K;
};
int product_shape(const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, Shape* s) {
    if (A == nullptr || B == nullptr) return QFMT_ERR_BAD_ARG;
    if (A->rows < 0 || A->cols < 0 || B->rows < 0 || B->cols < 0) return QFMT_ERR_BAD_ARG;
    s->M = A->trans ? A->cols : A->rows;
    s->K = A->trans ? A->rows : A->cols;
    s->N = B->trans ? B->rows : B->cols;
    if (s->K != (B->trans ? B->cols : B->rows)) return QFMT_ERR_BAD_ARG;
    if (s->M > (1 << 30) || s->N > (1 << 30) || s->K > (1 << 30)) return QFMT_ERR_BAD_ARG;
    if (p16::single_tiles(s->M, s->N) > (1 << 26)) return QFMT_ERR_BAD_ARG;  // work items are counted in 32 bits
    return QFMT_OK;
}

// Products that go over the weights in few_rows_kernel: up to 2^27 multiplications, which tiles cannot spread over the GPU, and up to 32 rows
// of any size if the weights are stored by output.  Measured against tiles, with GELU: 128 x 256 x 512 3.0 us by output and 5.1 by K against 11.4,
// 512 x 512 x 512 7.2 and 7.3 against 10.8; at 2^28 256 x 1024 x 1024 9.5 and 11.3 against 11.8, 1024 x 512 x 512 13.1 and 10.8 against 11.7;
// 32 x 4096 x 4096 13.8 and 25.8 against 17.4.  A's K must be contiguous, and short enough that none of the eight warps sums more than
// tiles do before they close a sum.
constexpr int64_t kFewWork = 1ll << 27;
bool few_rows(const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const Shape& s) {
    if (A->trans != 0 || s.K > kFewWarps * p16::kCloseK) return false;
    if (B->trans != 0 && s.M <= skinny::kMostRows) return true;
    return s.M <= 1024 && s.M * s.N <= kFewWork && s.M * s.N * s.K <= kFewWork;
}

constexpr size_t kHeader = 256;
size_t sums_bytes(const Shape& s) {  // column sums by groups of 32 rows of whole tiles, or by the row blocks of a pass
    const int64_t groups = p16::ceil_div(s.M, 2 * p16::kRows) * 2 * p16::kRows / 32, blocks = s.N > 0 ? pass_row_blocks(s.M, s.N) : 0;
    return (size_t)(groups > blocks ? groups : blocks) * (size_t)padded(s.N) * sizeof(float);
}
size_t part_bytes(const Shape& s, int splits) { return (size_t)splits * (size_t)s.M * (size_t)padded(s.N) * sizeof(float); }

struct Call {
    Shape s;
    int act;
    int64_t ld_residual, ld_z;
    DeviceInfo dev;
    p16::Operand a, b;
    p16::ProductParams p;
    bool pair;
    int splits;
    float *sums, *parts;
};

// Everything the two directions check and set up alike.  On QFMT_OK with *work false there is nothing to compute.
int prepare_call(Call* c, bool backward, const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* e, const void* d_out, int64_t ld_out,
                 const float* d_dbias, int32_t dtype, void* d_workspace, size_t workspace_bytes, bool* work) {
    *work = false;
    int rc = product_shape(A, B, &c->s);
    if (rc != QFMT_OK) return rc;
    const Shape& s = c->s;
    if (e == nullptr || (dtype != QFMT_F16 && dtype != QFMT_BF16)) return QFMT_ERR_BAD_ARG;
    if (e->act < QFMT_ACT_NONE || e->act > QFMT_ACT_SILU) return QFMT_ERR_BAD_ARG;
    c->act = e->act;
    c->ld_residual = e->ld_residual == 0 ? s.N : e->ld_residual;
    c->ld_z = e->ld_z == 0 ? s.N : e->ld_z;
    if (A->ld < A->cols || B->ld < B->cols || ld_out < s.N || c->ld_residual < s.N || c->ld_z < s.N) return QFMT_ERR_BAD_ARG;
    if (misaligned(e->d_bias, 4) || misaligned(e->d_residual, 2) || misaligned(e->d_z, 2) || misaligned(d_out, 2) || misaligned(d_dbias, 4))
        return QFMT_ERR_BAD_ARG;
    if (d_workspace == nullptr || misaligned(d_workspace, 16) || workspace_bytes < kHeader) return QFMT_ERR_BAD_ARG;
    const size_t sums = d_dbias != nullptr ? sums_bytes(s) : 0;
    if (workspace_bytes < kHeader + sums) return QFMT_ERR_BAD_ARG;
    if (s.M == 0 || s.N == 0) return QFMT_OK;
    if (d_out == nullptr || (backward && e->act != QFMT_ACT_NONE && e->d_z == nullptr)) return QFMT_ERR_BAD_ARG;
    if (s.K != 0) {
        if (A->ptr == nullptr || B->ptr == nullptr || misaligned(A->ptr, 16) || misaligned(B->ptr, 16) || (A->ld & 7) || (B->ld & 7))
            return QFMT_ERR_BAD_ARG;  // TMA: 16-byte aligned bases and row pitches
    }
    rc = current_device(&c->dev);
    if (rc != QFMT_OK) return rc;
    p16::ProductPlan plan = p16::plan_product(s.M, s.N, s.K, true);
    while (plan.splits > 1 && kHeader + sums + part_bytes(s, plan.splits) > workspace_bytes) --plan.splits;
    const int stages = (int)p16::ceil_div(s.K, p16::kStageK);
    plan.kb_per_split = (stages + plan.splits - 1) / plan.splits;
    if (plan.splits > 1) plan.splits = (stages + plan.kb_per_split - 1) / plan.kb_per_split;
    c->pair = plan.pair;
    c->splits = plan.splits;
    c->a = p16::Operand{};
    c->b = p16::Operand{};
    if (s.K != 0 && !few_rows(A, B, s)) {
        rc = p16::make_operand(&c->a, false, plan.pair, A->ptr, A->trans != 0, s.M, s.K, A->ld);
        if (rc != QFMT_OK) return rc;
        rc = p16::make_operand(&c->b, true, plan.pair, B->ptr, B->trans == 0, s.N, s.K, B->ld);
        if (rc != QFMT_OK) return rc;
    }
    p16::ProductParams& p = c->p;
    p = p16::ProductParams{};
    p.M = (int)s.M;
    p.N = (int)s.N;
    p.K = (int)s.K;
    p.bf16 = dtype == QFMT_BF16;
    p.kb_per_split = plan.kb_per_split;
    p.splits = plan.splits;
    p.status = static_cast<unsigned long long*>(d_workspace);
    p.tag = next_launch_tag();
    c->sums = reinterpret_cast<float*>(static_cast<char*>(d_workspace) + kHeader);
    c->parts = reinterpret_cast<float*>(static_cast<char*>(d_workspace) + kHeader + sums);
    *work = true;
    return QFMT_OK;
}

int launch_parts(const Call& c, RowPass* a, cudaStream_t stream) {
    typename PartEpilogue::Params pe = {c.parts, padded(c.s.N), c.s.M * padded(c.s.N)};
    *a = RowPass{};
    a->parts = c.parts;
    a->splits = c.splits;
    a->split_stride = pe.split_stride;
    a->pitch = pe.pitch;
    a->rows = c.s.M;
    a->cols = c.s.N;
    return p16::launch_product<PartEpilogue>(c.pair, c.a, c.b, nullptr, c.p, pe, c.dev, stream);
}

template <typename T, int kAct, bool kBackward, bool kByK, int kBlocks>
int launch_few_rows(const FewRows& f0, const DeviceInfo& dev, cudaStream_t stream) {
    FewRows f = f0;
    constexpr int kOutputs = kByK ? 64 : 16, kRows = kByK ? 16 * kBlocks : 8 * kBlocks;
    constexpr size_t smem = (size_t)kFewWarps * kRows * (kOutputs + 2) * sizeof(float);
    auto* kernel = few_rows_kernel<T, kAct, kBackward, kByK, kBlocks>;
    if (smem > 48 * 1024) {
        static std::atomic<bool> ready[64];
        const bool known = dev.ordinal >= 0 && dev.ordinal < 64;
        if (!known || !ready[dev.ordinal].load()) {
            QFMT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
            if (known) ready[dev.ordinal].store(true);
        }
    }
    // blocks to a cluster: while there are processors without a block and a warp keeps 64 elements of K
    const int groups = (f.o.n + kOutputs - 1) / kOutputs, row_blocks = (f.o.rows + skinny::kMostRows - 1) / skinny::kMostRows;
    int size = 1;
    while (size < 8 && groups * row_blocks * size * 2 <= dev.sm_count && f.o.k >= size * 2 * kFewWarps * 64) size *= 2;
    const int per = (f.o.k + size * kFewWarps - 1) / (size * kFewWarps);
    f.k_warp = (per + 31) / 32 * 32;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * size), (unsigned)row_blocks, 1);
    cfg.blockDim = dim3(kFewWarps * 32, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)size;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    QFMT_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, f));
    return QFMT_OK;
}

template <typename T, int kAct, bool kBackward>
int few_rows_call(const Call& c, const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* e, void* d_out, int64_t ld_out,
                  float* d_dbias, cudaStream_t stream) {
    FewRows f = {};
    f.o = skinny::Operands{A->ptr, B->ptr, A->ld, B->ld, (int)c.s.M, (int)c.s.N, (int)c.s.K};
    f.bias = e->d_bias;
    f.residual = e->d_residual;
    f.ld_residual = c.ld_residual;
    f.z_in = f.z_out = e->d_z;
    f.ld_z = c.ld_z;
    f.out = d_out;
    f.ld_out = ld_out;
    const bool join = c.s.M > skinny::kMostRows && d_dbias != nullptr;
    f.sums = join ? c.sums : d_dbias;
    f.pitch = padded(c.s.N);
    f.status = c.p.status;
    f.tag = c.p.tag;
    int rc;
    if (B->trans != 0) {
        if (c.s.M <= 8) rc = launch_few_rows<T, kAct, kBackward, false, 1>(f, c.dev, stream);
        else if (c.s.M <= 16) rc = launch_few_rows<T, kAct, kBackward, false, 2>(f, c.dev, stream);
        else rc = launch_few_rows<T, kAct, kBackward, false, 4>(f, c.dev, stream);
    } else {
        if (c.s.M <= 16) rc = launch_few_rows<T, kAct, kBackward, true, 1>(f, c.dev, stream);
        else rc = launch_few_rows<T, kAct, kBackward, true, 2>(f, c.dev, stream);
    }
    if (rc != QFMT_OK || !join) return rc;
    return launch_join_columns(c.sums, f.pitch, (c.s.M + skinny::kMostRows - 1) / skinny::kMostRows, nullptr, 0, nullptr, d_dbias, c.s.N, stream);
}

template <typename T, int kAct>
int forward_call(const Call& c, const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* e, void* d_y, int64_t ldy, cudaStream_t stream) {
    if (few_rows(A, B, c.s)) return few_rows_call<T, kAct, false>(c, A, B, e, d_y, ldy, nullptr, stream);
    const bool vr = whole(e->d_residual, c.ld_residual, 2), vz = whole(e->d_z, c.ld_z, 2), vy = whole(d_y, ldy, 2);
    if (c.splits > 1) {
        RowPass a;
        const int rc = launch_parts(c, &a, stream);
        if (rc != QFMT_OK) return rc;
        a.bias = e->d_bias;
        a.residual = e->d_residual;
        a.ld_residual = c.ld_residual;
        a.z_out = e->d_z;
        a.ld_z = c.ld_z;
        a.out = d_y;
        a.ld_out = ldy;
        return launch_row_pass<T, kAct, false, true>(a, vr && vz && vy && c.s.N % 8 == 0, stream);
    }
    using Epi = ForwardEpilogue<T, kAct>;
    typename Epi::Params ep = {e->d_bias, static_cast<const T*>(e->d_residual), static_cast<T*>(e->d_z), static_cast<T*>(d_y),
                               c.ld_residual, c.ld_z, ldy, vr, vz, vy};
    return p16::launch_product<Epi>(c.pair, c.a, c.b, nullptr, c.p, ep, c.dev, stream);
}

template <typename T, int kAct>
int backward_call(const Call& c, const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* e, void* d_dz, int64_t ld_dz,
                  float* d_dbias, cudaStream_t stream) {
    if (few_rows(A, B, c.s)) return few_rows_call<T, kAct, true>(c, A, B, e, d_dz, ld_dz, d_dbias, stream);
    const bool vr = whole(e->d_residual, c.ld_residual, 2), vz = whole(e->d_z, c.ld_z, 2), vd = whole(d_dz, ld_dz, 2);
    const int64_t pitch = padded(c.s.N);
    const int64_t tile_rows = c.pair ? 2 * p16::kRows : p16::kRows;
    int64_t n_parts = p16::ceil_div(c.s.M, tile_rows) * tile_rows / 32;
    int rc;
    if (c.splits > 1) {
        RowPass a;
        rc = launch_parts(c, &a, stream);
        if (rc != QFMT_OK) return rc;
        a.residual = e->d_residual;
        a.ld_residual = c.ld_residual;
        a.z_in = e->d_z;
        a.ld_z = c.ld_z;
        a.out = d_dz;
        a.ld_out = ld_dz;
        a.sums = d_dbias != nullptr ? c.sums : nullptr;
        rc = launch_row_pass<T, kAct, true, true>(a, vr && vz && vd && c.s.N % 8 == 0, stream);
        const int64_t blocks = pass_row_blocks(c.s.M, c.s.N), per = (c.s.M + blocks - 1) / blocks;
        n_parts = (c.s.M + per - 1) / per;
    } else {
        using Epi = BackwardEpilogue<T, kAct>;
        typename Epi::Params ep = {static_cast<const T*>(e->d_residual), static_cast<const T*>(e->d_z), static_cast<T*>(d_dz),
                                   d_dbias != nullptr ? c.sums : nullptr, c.ld_residual, c.ld_z, ld_dz, pitch, vr, vz, vd};
        rc = p16::launch_product<Epi>(c.pair, c.a, c.b, nullptr, c.p, ep, c.dev, stream);
    }
    if (rc != QFMT_OK || d_dbias == nullptr) return rc;
    return launch_join_columns(c.sums, pitch, n_parts, nullptr, 0, nullptr, d_dbias, c.s.N, stream);
}

template <typename T, int kAct>
int act_backward_call(RowPass a, bool vec, float* d_dbias, cudaStream_t stream) {
    int rc = launch_row_pass<T, kAct, true, false>(a, vec, stream);
    if (rc != QFMT_OK || d_dbias == nullptr) return rc;
    const int64_t blocks = pass_row_blocks(a.rows, a.cols), per = (a.rows + blocks - 1) / blocks;
    return launch_join_columns(a.sums, a.pitch, (a.rows + per - 1) / per, nullptr, 0, nullptr, d_dbias, a.cols, stream);
}

#define BY_ACT(act, call)                                              \
    switch (act) {                                                     \
        case QFMT_ACT_RELU: { constexpr int kA = QFMT_ACT_RELU; return call; }         \
        case QFMT_ACT_GELU: { constexpr int kA = QFMT_ACT_GELU; return call; }         \
        case QFMT_ACT_GELU_TANH: { constexpr int kA = QFMT_ACT_GELU_TANH; return call; } \
        case QFMT_ACT_SILU: { constexpr int kA = QFMT_ACT_SILU; return call; }         \
        default: { constexpr int kA = QFMT_ACT_NONE; return call; }    \
    }

template <typename T>
int forward_typed(const Call& c, const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* e, void* d_y, int64_t ldy,
                  cudaStream_t stream) {
    BY_ACT(c.act, (forward_call<T, kA>(c, A, B, e, d_y, ldy, stream)))
}
template <typename T>
int backward_typed(const Call& c, const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* e, void* d_dz, int64_t ld_dz,
                   float* d_dbias, cudaStream_t stream) {
    BY_ACT(c.act, (backward_call<T, kA>(c, A, B, e, d_dz, ld_dz, d_dbias, stream)))
}
template <typename T>
int act_backward_typed(int act, const RowPass& a, bool vec, float* d_dbias, cudaStream_t stream) {
    BY_ACT(act, (act_backward_call<T, kA>(a, vec, d_dbias, stream)))
}

}  // namespace
}  // namespace qfmt

extern "C" size_t qfmt_linear_act_workspace_bytes(const qfmt_matrix16_t* A, const qfmt_matrix16_t* B) {
    qfmt::Shape s;
    if (qfmt::product_shape(A, B, &s) != QFMT_OK) return 0;
    const int splits = qfmt::p16::plan_product(s.M, s.N, s.K, true).splits;
    return qfmt::kHeader + qfmt::sums_bytes(s) + (splits > 1 ? qfmt::part_bytes(s, splits) : 0);
}

extern "C" int qfmt_linear_act(const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* epilogue, void* d_y, int64_t ldy,
                               int32_t dtype, void* d_workspace, size_t workspace_bytes, void* stream) {
    qfmt::Call c;
    bool work;
    const int rc = qfmt::prepare_call(&c, false, A, B, epilogue, d_y, ldy, nullptr, dtype, d_workspace, workspace_bytes, &work);
    if (rc != QFMT_OK || !work) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == QFMT_F16) return qfmt::forward_typed<__half>(c, A, B, epilogue, d_y, ldy, st);
    return qfmt::forward_typed<__nv_bfloat16>(c, A, B, epilogue, d_y, ldy, st);
}

extern "C" int qfmt_linear_act_backward(const qfmt_matrix16_t* A, const qfmt_matrix16_t* B, const qfmt_epilogue_t* epilogue, void* d_dz,
                                        int64_t ld_dz, float* d_dbias, int32_t dtype, void* d_workspace, size_t workspace_bytes,
                                        void* stream) {
    qfmt::Call c;
    bool work;
    const int rc = qfmt::prepare_call(&c, true, A, B, epilogue, d_dz, ld_dz, d_dbias, dtype, d_workspace, workspace_bytes, &work);
    if (rc != QFMT_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!work) {
        if (d_dbias != nullptr && c.s.N > 0) {
            qfmt::DeviceInfo dev;
            const int ok = qfmt::current_device(&dev);
            if (ok != QFMT_OK) return ok;
            QFMT_CUDA_TRY(cudaMemsetAsync(d_dbias, 0, (size_t)c.s.N * sizeof(float), st));
        }
        return QFMT_OK;
    }
    if (dtype == QFMT_F16) return qfmt::backward_typed<__half>(c, A, B, epilogue, d_dz, ld_dz, d_dbias, st);
    return qfmt::backward_typed<__nv_bfloat16>(c, A, B, epilogue, d_dz, ld_dz, d_dbias, st);
}

extern "C" size_t qfmt_act_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31)) return 0;
    return qfmt::kHeader + (size_t)qfmt::pass_row_blocks(rows, cols > 0 ? cols : 1) * (size_t)qfmt::padded(cols) * sizeof(float);
}

extern "C" int qfmt_act_backward(const void* d_dy, int64_t ld_dy, const void* d_z, int64_t ld_z, void* d_dz, int64_t ld_dz, float* d_dbias,
                                 int64_t rows, int64_t cols, int32_t dtype, int32_t act, void* d_workspace, size_t workspace_bytes,
                                 void* stream) {
    using namespace qfmt;
    if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31)) return QFMT_ERR_BAD_ARG;
    if (dtype != QFMT_F32 && dtype != QFMT_F16 && dtype != QFMT_BF16) return QFMT_ERR_BAD_ARG;
    if (act < QFMT_ACT_NONE || act > QFMT_ACT_SILU) return QFMT_ERR_BAD_ARG;
    const int64_t size = dtype == QFMT_F32 ? 4 : 2;
    if (ld_dy == 0) ld_dy = cols;
    if (ld_z == 0) ld_z = cols;
    if (ld_dz == 0) ld_dz = cols;
    if (ld_dy < cols || ld_z < cols || ld_dz < cols) return QFMT_ERR_BAD_ARG;
    if (misaligned(d_dy, size) || misaligned(d_z, size) || misaligned(d_dz, size) || misaligned(d_dbias, 4)) return QFMT_ERR_BAD_ARG;
    if (d_dbias != nullptr && rows > 0 && cols > 0) {
        if (d_workspace == nullptr || misaligned(d_workspace, 16) || workspace_bytes < qfmt_act_backward_workspace_bytes(rows, cols))
            return QFMT_ERR_BAD_ARG;
    }
    if (rows > 0 && cols > 0 && (d_dy == nullptr || (act != QFMT_ACT_NONE && d_z == nullptr))) return QFMT_ERR_BAD_ARG;
    DeviceInfo dev;
    const int rc = current_device(&dev);
    if (rc != QFMT_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0 || cols == 0) {
        if (d_dbias != nullptr && cols > 0) QFMT_CUDA_TRY(cudaMemsetAsync(d_dbias, 0, (size_t)cols * sizeof(float), st));
        return QFMT_OK;
    }
    if (d_dz == nullptr && d_dbias == nullptr) return QFMT_OK;
    RowPass a = {};
    a.dy = d_dy;
    a.ld_dy = ld_dy;
    a.z_in = d_z;
    a.ld_z = ld_z;
    a.out = d_dz;
    a.ld_out = ld_dz;
    // behind the status area, which is another call's if the workspace is shared
    a.sums = d_dbias != nullptr ? reinterpret_cast<float*>(static_cast<char*>(d_workspace) + kHeader) : nullptr;
    a.pitch = padded(cols);
    a.rows = rows;
    a.cols = cols;
    const bool vec = whole(d_dy, ld_dy, size) && (act == QFMT_ACT_NONE || whole(d_z, ld_z, size)) && whole(d_dz, ld_dz, size) &&
                     cols % 8 == 0;
    if (dtype == QFMT_F32) return act_backward_typed<float>(act, a, vec, d_dbias, st);
    if (dtype == QFMT_F16) return act_backward_typed<__half>(act, a, vec, d_dbias, st);
    return act_backward_typed<__nv_bfloat16>(act, a, vec, d_dbias, st);
}
