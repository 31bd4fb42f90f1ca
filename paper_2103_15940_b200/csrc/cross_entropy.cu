// Softmax cross entropy on top of the product that makes the logits, forward and backward, without the logits in memory:
//     logits = H W + bias,  lse = log sum exp(logits),  loss = lse - logits_target,
//     d = g (exp(logits - lse) - onehot),  dH = d W^T,  dW = H^T d,  dbias = column sums of d.
//
// In the backward pass g is a row's dloss alone (1 without one), times a power of two.  What all rows share (1 / rows that count, the loss
// scale) multiplies the sums: rounded into the codes of d it would be off by up to half a step in every row alike, which does not average
// out (binary16, 333 x 520 over 10007 words: gradients 3.0e-4 of their size off against 2.2e-4, of which their own rounding is 2.1e-4; 11 x 809
// over 112272 3.7e-4 against 2.1e-4).
//
// Rows that do not count are taken out first: compact_kernel numbers the others, and the products run over as many rows as it
// found (the host never learns the number).  If all count, H is read in place.  Forward, the product's epilogue reduces each row's
// 64 logits to their maximum and the sum of exponentials relative to it (base 2, one pass: a later maximum rescales the sum),
// and join_rows_kernel joins the pieces.  Backward, the vocabulary is walked in pieces: the product again, its epilogue forming d in
// codes in a buffer that stays in the second-level cache, then the two products that read it.  dH is added up in fp32 over the pieces.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "activation.cuh"
#include "columns.cuh"
#include "common.cuh"
#include "product16.cuh"
#include "skinny16.cuh"

namespace qfmt {
namespace {

using p16::Patch;

struct Nothing {};

// Head of the workspace behind the status area: what compact_kernel finds out.
struct Found {
    int count;       // rows that count
    float unscale;   // what sums of d are multiplied by: the factors that all rows share, without the power of two that d is given
};

// ---- rows that count ----------------------------------------------------------------------------------------------------
struct Compact {
    const int64_t* targets;
    int64_t ignore;
    int rows, vocab;
    Found* found;
    int *index, *target;      // compact row -> row, target (-1: not a word)
    // forward: results of rows that do not count
    float *loss, *lse_out;
    // backward: what d needs of a compact row
    const float *lse, *dloss;
    const qfmt_dls_t* dls;
    float *lse_of, *g;
    int mean;
    // H and its compact copy; dH, whose rows that do not count are zeros
    const uint16_t* h;
    int64_t ld_h;
    uint16_t* copy;
    int64_t ld_copy;
    uint16_t* dh;
    int64_t ld_dh;
    int hidden;
    int rows_per_block;
};

constexpr int kCompactThreads = 1024;  // a warp a row of a block's 32, so that the copies of all are on their way at once

template <typename V>
__device__ __forceinline__ V block_sum(V v, V* scratch) {  // scratch: one per warp; every thread gets the sum
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[threadIdx.x & 31];
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// A block has rows_per_block rows and finds the place of its first by counting all rows itself (targets are a few bytes a row
// and lie in the second-level cache), so blocks need not wait for one another.
template <bool kBackward>
__global__ void __launch_bounds__(kCompactThreads)
compact_kernel(const Compact c, unsigned long long* status, unsigned long long tag) {
    __shared__ int scratch[kCompactThreads / 32], place[kCompactThreads];
    __shared__ float most[kCompactThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    announce_launch(status, tag);
    const int first = (int)blockIdx.x * c.rows_per_block;
    const int end = first + c.rows_per_block < c.rows ? first + c.rows_per_block : c.rows;
    int before = 0, total = 0;
#pragma unroll 8
    for (int i = tid; i < c.rows; i += kCompactThreads) {
        const int counts = c.targets[i] != c.ignore ? 1 : 0;
        total += counts;
        before += i < first ? counts : 0;
    }
    before = block_sum(before, scratch);
    total = block_sum(total, scratch);
    const bool last = end == c.rows;
    float scale = 1.0f, shared = 1.0f;
    if (kBackward) {
        if (c.mean) shared = __frcp_rn((float)(total > 0 ? total : 1));
        if (c.dls != nullptr) shared = __fmul_rn(shared, c.dls->scale);
        // |d| <= |g|, so the largest |g| scaled to 2^13 .. 2^14 leaves room above and, in binary16, 37 binades below
        float m = c.dloss != nullptr ? 0.0f : 1.0f;
        if (c.dloss != nullptr) {
            for (int i = tid; i < c.rows; i += kCompactThreads) {
                const float v = c.targets[i] != c.ignore ? fabsf(c.dloss[i]) : 0.0f;
                m = v > m ? v : m;
            }
            for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            if (lane == 0) most[warp] = m;
            __syncthreads();
            m = most[0];
            for (int w = 1; w < kCompactThreads / 32; ++w) m = fmaxf(m, most[w]);
        }
        uint32_t exponent = __float_as_uint(m) >> 23;
        if (exponent < 13u) exponent = 13u;  // the power has to be a number
        if (exponent != 255u) scale = __uint_as_float((267u - exponent) << 23);
    }
    if (last && tid == 0) {
        c.found->count = total;
        c.found->unscale = __fmul_rn(shared, __frcp_rn(scale));
    }
    const bool copy = total != c.rows;
    const int whole = c.hidden & ~7;
    for (int seg = first; seg < end; seg += kCompactThreads) {
        const int row = seg + tid;
        int64_t target = c.ignore;
        if (row < end) target = c.targets[row];
        const bool counts = row < end && target != c.ignore;
        const unsigned mask = __ballot_sync(0xFFFFFFFFu, counts);
        __syncthreads();
        if (lane == 0) scratch[warp] = __popc(mask);
        __syncthreads();
        int sum = scratch[lane];  // of the warps up to this lane's
        for (int o = 1; o < 32; o <<= 1) {
            const int below = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += below;
        }
        const int at = before + __shfl_sync(0xFFFFFFFFu, sum, warp) - __popc(mask) + __popc(mask & ((1u << lane) - 1u));
        before += __shfl_sync(0xFFFFFFFFu, sum, 31);
        place[tid] = counts ? at : -1;
        if (counts) {
            c.index[at] = row;
            c.target[at] = target >= 0 && target < c.vocab ? (int)target : -1;
            if (kBackward) {
                c.lse_of[at] = c.lse[row];
                c.g[at] = c.dloss != nullptr ? __fmul_rn(c.dloss[row], scale) : scale;
            }
        } else if (!kBackward && row < end) {
            if (c.loss != nullptr) c.loss[row] = 0.0f;
            if (c.lse_out != nullptr) c.lse_out[row] = 0.0f;
        }
        __syncthreads();
        if (!copy) continue;
        const int n = end - seg < kCompactThreads ? end - seg : kCompactThreads;
        for (int r = warp; r < n; r += kCompactThreads / 32) {
            const int to = place[r];
            if (to >= 0) {
                const uint16_t* src = c.h + (int64_t)(seg + r) * c.ld_h;
                uint16_t* dst = c.copy + (int64_t)to * c.ld_copy;
#pragma unroll 4
                for (int j = lane * 8; j < whole; j += 256) *reinterpret_cast<uint4*>(dst + j) = *reinterpret_cast<const uint4*>(src + j);
                if (lane < c.hidden - whole) dst[whole + lane] = src[whole + lane];
            } else if (kBackward && c.dh != nullptr) {
                uint16_t* dst = c.dh + (int64_t)(seg + r) * c.ld_dh;
                if ((reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
                    for (int j = lane * 8; j < whole; j += 256) *reinterpret_cast<uint4*>(dst + j) = make_uint4(0, 0, 0, 0);
                    if (lane < c.hidden - whole) dst[whole + lane] = 0;
                } else {
                    for (int j = lane; j < c.hidden; j += 32) dst[j] = 0;
                }
            }
        }
    }
    if (last && copy) {  // the weight gradient's products read whole stages of 64 rows
        const int pad = (total + 63) / 64 * 64;
        for (int r = total + warp; r < pad; r += kCompactThreads / 32)
            for (int j = lane; j < c.hidden; j += 32) c.copy[(int64_t)r * c.ld_copy + j] = 0;
    }
}

// ---- epilogues ------------------------------------------------------------------------------------------------------------

// Per row and 64 columns: m = the largest logit, s = sum exp(logit - m), and the target's logit.  The exponentials are
// 2^(logit log2 e - shift), one fused operation and one of the special function unit each, with shift = m log2 e rounded; what the rounding
// took off is put back by one factor per 32 columns.  Logits whose product with log2 e overflows have m subtracted first.
struct RowSumEpilogue {
    struct Params {
        const float* bias;
        const int* target;
        float2* parts;  // [64-column groups][pitch]
        float* picked;  // the target's logit of a compact row
        int64_t pitch;
    };
    struct Ahead {
        int target;
        float bias[2];
    };
    static __device__ __forceinline__ void before(const Patch& p, const Params& e, Ahead& a) {
        p.columns(e.bias, a.bias);
        a.target = p.row0 + p.lane < p.rows ? e.target[p.row0 + p.lane] - p.col0 : -1;
    }
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead& a, F release) {
        const int row = p.row0 + p.lane;
        float most = -INFINITY, sum = 0.0f;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            pair_t v[16];
            p.load_pairs<true>(c, v, c == 0 ? a.bias[0] : a.bias[1]);
            if (c == 1) release();
            const int left = p.cols - p.col0 - c * 32;
            if (left <= 0) continue;
            if (left < 32) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float2 f = split_pair(v[j]);
                    v[j] = make_pair(2 * j < left ? f.x : -INFINITY, 2 * j + 1 < left ? f.y : -INFINITY);
                }
            }
            if ((a.target >> 5) == c) {  // by halves: an index would put the values into memory
                pair_t w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (a.target & 16) ? v[j + 8] : v[j];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = (a.target & 8) ? w[j + 4] : w[j];
                w[0] = (a.target & 4) ? w[2] : w[0];
                w[1] = (a.target & 4) ? w[3] : w[1];
                const float2 f = split_pair((a.target & 2) ? w[1] : w[0]);
                e.picked[row] = (a.target & 1) ? f.y : f.x;
            }
            float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float2 f = split_pair(v[j]);
                m0 = fmaxf(m0, f.x);
                m1 = fmaxf(m1, f.y);
            }
            const float now = fmaxf(most, fmaxf(m0, m1));
            float shift = __fmul_rn(now, kLog2E), back = 1.0f;
            if (isinf(shift)) {
                if (now != -INFINITY) {  // else nothing but -infinity yet: all terms are zero
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = add2(v[j], both(-now));
                }
                shift = 0.0f;
            } else {
                back = fast_exp2(-__fmaf_rn(now, kLog2E, -shift));
            }
            if (now != -INFINITY) sum = __fmul_rn(sum, fast_exp2(__fmul_rn(__fsub_rn(most, now), kLog2E)));
            pair_t s0 = 0ull, s1 = 0ull;
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const float2 x = split_pair(fma2(v[j], both(kLog2E), both(-shift))), y = split_pair(fma2(v[j + 1], both(kLog2E), both(-shift)));
                s0 = add2(s0, make_pair(fast_exp2(x.x), fast_exp2(x.y)));
                s1 = add2(s1, make_pair(fast_exp2(y.x), fast_exp2(y.y)));
            }
            const float2 s = split_pair(add2(s0, s1));
            sum = __fmaf_rn(__fadd_rn(s.x, s.y), back, sum);
            most = now;
        }
        if (row < p.rows && p.col0 < p.cols) e.parts[(int64_t)(p.col0 >> 6) * e.pitch + row] = make_float2(most, sum);
    }
};

// d = g (exp(logit - lse) - onehot) in codes, zeros beyond the rows and the words; column sums of the 32-bit values.
template <typename T>
struct GradEpilogue {
    struct Params {
        const float* bias;
        const int* target;
        const float *lse, *g;
        T* d;             // [rows of whole tiles][pitch]
        float* parts;     // [32-row groups][pitch], or null
        int64_t pitch;
        int first_word;   // of this piece of the vocabulary
    };
    struct Ahead {
        int target;
        float lse, lse2, g, gp;  // lse2 = lse log2 e rounded; gp = g times what the rounding took off
        float bias[2];
    };
    static __device__ __forceinline__ void before(const Patch& p, const Params& e, Ahead& a) {
        p.columns(e.bias, a.bias);
        const int row = p.row0 + p.lane;
        const bool there = row < p.rows;
        a.target = there ? e.target[row] - e.first_word - p.col0 : -1;
        a.lse = there ? e.lse[row] : 0.0f;
        a.g = there ? e.g[row] : 0.0f;
        a.lse2 = __fmul_rn(a.lse, kLog2E);
        a.gp = a.g;
        if (isfinite(a.lse2)) a.gp = __fmul_rn(a.g, fast_exp2(-__fmaf_rn(a.lse, kLog2E, -a.lse2)));
    }
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead& a, F release) {
        const bool there = p.row0 + p.lane < p.rows;
        const bool huge = __any_sync(0xFFFFFFFFu, isinf(a.lse2));  // lse log2 e overflows: subtract first
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            pair_t v[16];
            p.load_pairs<true>(c, v, c == 0 ? a.bias[0] : a.bias[1]);
            if (c == 1) release();
            const int col0 = p.col0 + c * 32, left = p.cols - col0;
            if (!huge) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float2 x = split_pair(fma2(v[j], both(kLog2E), both(-a.lse2)));
                    v[j] = mul2(make_pair(fast_exp2(x.x), fast_exp2(x.y)), both(a.gp));
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float2 x = split_pair(mul2(add2(v[j], both(-a.lse)), both(kLog2E)));
                    v[j] = mul2(make_pair(fast_exp2(x.x), fast_exp2(x.y)), both(a.g));
                }
            }
            if ((a.target >> 5) == c) {
                const int at = (a.target & 31) >> 1;
                const pair_t minus = (a.target & 1) ? make_pair(0.0f, -a.g) : make_pair(-a.g, 0.0f);
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = at == j ? add2(v[j], minus) : v[j];
            }
            if (left < 32 || p.row0 + 32 > p.rows) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float2 x = split_pair(v[j]);
                    v[j] = make_pair(there && 2 * j < left ? x.x : 0.0f, there && 2 * j + 1 < left ? x.y : 0.0f);
                }
            }
            p16::box_put_codes<T>(p.box, p.lane, v);
            __syncwarp();
            p16::box_store<T>(p.box, e.d, e.pitch, p.row0, p.row0 + 32, col0, (int)e.pitch, p.lane, true);
            __syncwarp();
            if (e.parts != nullptr) {
                const float s = p16::column_sum(p.box, p.lane, v);
                e.parts[(int64_t)(p.row0 >> 5) * e.pitch + col0 + p.lane] = s;
            }
        }
    }
};

// The sums times a factor, in codes: dW.
template <typename T>
struct ScaledEpilogue {
    struct Params {
        const float* factor;
        T* out;
        int64_t ld;
        int vec;
    };
    struct Ahead {
        float factor;
    };
    static __device__ __forceinline__ void before(const Patch&, const Params& e, Ahead& a) { a.factor = *e.factor; }
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead& a, F release) {
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            pair_t v[16];
            p.load_pairs<false>(c, v);
            if (c == 1) release();
            const int col0 = p.col0 + c * 32;
            if (p.row0 >= p.rows || col0 >= p.cols) continue;
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = mul2(v[j], both(a.factor));
            p16::box_put_codes<T>(p.box, p.lane, v);
            __syncwarp();
            p16::box_store<T>(p.box, e.out, e.ld, p.row0, p.rows, col0, p.cols, p.lane, e.vec != 0);
            __syncwarp();
        }
    }
};

// The sums added to what the pieces before left, in fp32, one place per split of K: dH.
struct AddEpilogue {
    struct Params {
        float* sums;
        int64_t pitch, split_stride;
        int add;  // 0: the first piece
    };
    using Ahead = Nothing;
    static __device__ __forceinline__ void before(const Patch&, const Params&, Ahead&) {}
    template <typename F>
    static __device__ __forceinline__ void run(const Patch& p, const Params& e, Ahead&, F release) {
        float* base = e.sums + (int64_t)p.split * e.split_stride;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
            p16::Fetched f[2];
            if (e.add) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    p16::box_fetch<float>(f[h], base, e.pitch, p.row0, p.rows, p.col0 + c * 32 + h * 16, p.cols, p.lane, true);
            }
            uint32_t r[32];
            p.load32(c, r);
            p.finish(c, r);
            if (c == 1) release();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col0 = p.col0 + c * 32 + h * 16;
                if (p.row0 >= p.rows || col0 >= p.cols) continue;
                if (e.add) {
                    p16::box_put<float>(p.box, f[h], base, e.pitch, p.row0, p.rows, col0, p.cols, p.lane, true);
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float4 w = *reinterpret_cast<const float4*>(p16::box_at(p.box, p.lane, k));
                        const float s[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) r[16 * h + 4 * k + j] = __float_as_uint(__fadd_rn(s[j], __uint_as_float(r[16 * h + 4 * k + j])));
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *p16::box_at(p.box, p.lane, k) = make_uint4(r[16 * h + 4 * k], r[16 * h + 4 * k + 1], r[16 * h + 4 * k + 2], r[16 * h + 4 * k + 3]);
                __syncwarp();
                p16::box_store<float>(p.box, base, e.pitch, p.row0, p.rows, col0, p.cols, p.lane, true);
                __syncwarp();
            }
        }
    }
};

// ---- joining ----------------------------------------------------------------------------------------------------------------

// lse - logit in 64 bits: rounded to 32 before the subtraction, lse takes half a step of the largest logit's size from every loss (2e-6 where
// logits are around 50, all of a small loss).
__device__ __forceinline__ float loss_of(float most, float log, float picked) { return (float)((double)most + (double)log - (double)picked); }

constexpr int kJoinRows = 32, kJoinParts = 32;

// Block of 32 rows x 32 groups: group q joins a row's parts q, q + 32, ..., then a warp a row joins the groups' (halves onto halves).
__global__ void __launch_bounds__(kJoinRows * kJoinParts)
join_rows_kernel(const float2* __restrict__ parts, int64_t pitch, int n_parts, const Found* found, const int* __restrict__ index,
                 const int* __restrict__ target, const float* __restrict__ picked, float* loss, float* lse_out, float* compact_loss,
                 float* mean) {
    __shared__ float2 joined[kJoinParts][kJoinRows + 1];
    __shared__ float losses[kJoinRows];
    const int r = threadIdx.x % kJoinRows, q = threadIdx.x / kJoinRows, row = (int)blockIdx.x * kJoinRows + r;
    grid_dependency_wait();
    grid_launch_dependents();
    const int count = found->count;
    float m = -INFINITY, s = 0.0f;
    auto join = [&](float2 v) {
        const float now = fmaxf(m, v.x);
        if (now == -INFINITY) {
            s = __fadd_rn(s, v.y);  // zero, or NaN where all of a part's logits are
            return;
        }
        s = __fmaf_rn(v.y, fast_exp2(__fmul_rn(__fsub_rn(v.x, now), kLog2E)), __fmul_rn(s, fast_exp2(__fmul_rn(__fsub_rn(m, now), kLog2E))));
        m = now;
    };
    if (row < count) {
#pragma unroll 4
        for (int i = q; i < n_parts; i += kJoinParts) join(parts[(int64_t)i * pitch + row]);
    }
    joined[q][r] = make_float2(m, s);
    __syncthreads();
    // now thread (r, q) is lane r of warp q: the warp has row q of the block, the lane group r
    const int mine = (int)blockIdx.x * kJoinRows + q;
    float2 v = joined[r][q];
    m = v.x;
    s = v.y;
    for (int o = 16; o > 0; o >>= 1) join(make_float2(__shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o)));
    if (r == 0) {
        float l = 0.0f;
        if (mine < count) {
            const float log = logf(s);
            float lse = __fadd_rn(m, log);
            l = loss_of(m, log, picked[mine]);
            if (target[mine] < 0) l = lse = __int_as_float(0x7FC00000);  // the target is not a word
            const int to = index[mine];
            if (loss != nullptr) loss[to] = l;
            if (lse_out != nullptr) lse_out[to] = lse;
            if (compact_loss != nullptr) compact_loss[mine] = l;
        }
        losses[q] = l;
    }
    if (mean == nullptr) return;  // else this is the only block
    __syncthreads();
    if (q == 0) {
        double total = losses[r];
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
        if (r == 0) *mean = (float)(total / (count > 0 ? count : 1));
    }
}

__global__ void __launch_bounds__(1024)
mean_kernel(const float* __restrict__ loss, const Found* found, float* mean) {
    __shared__ double sums[32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int count = found->count;
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += 1024) s += loss[i];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 32; ++w) s += sums[w];
        *mean = (float)(s / (count > 0 ? count : 1));
    }
}

// dH: the splits of a compact row added in order, scaled back, rounded and put where the row came from.  A warp 128 columns of a row
// at a time.
template <typename T>
__global__ void __launch_bounds__(256)
scatter_kernel(const float* __restrict__ sums, int splits, int64_t split_stride, int64_t pitch, const Found* found,
               const int* __restrict__ index, T* dh, int64_t ld, int hidden, int vec) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, chunks = (hidden + 127) / 128;
    const int64_t units = (int64_t)found->count * chunks;
    const float factor = found->unscale;
    for (int64_t u = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * 8) {
        const int row = (int)(u / chunks), j = (int)(u % chunks) * 128 + lane * 4;
        if (j >= hidden) continue;
        const float* src = sums + (int64_t)row * pitch + j;  // rows are padded to whole pieces
        T* dst = dh + (int64_t)index[row] * ld + j;
        float4 v = *reinterpret_cast<const float4*>(src);
#pragma unroll 8
        for (int s = 1; s < splits; ++s) {
            const float4 w = *reinterpret_cast<const float4*>(src + s * split_stride);
            v = make_float4(__fadd_rn(v.x, w.x), __fadd_rn(v.y, w.y), __fadd_rn(v.z, w.z), __fadd_rn(v.w, w.w));
        }
        const uint32_t lo = p16::pack_codes<T>(__fmul_rn(v.x, factor), __fmul_rn(v.y, factor));
        const uint32_t hi = p16::pack_codes<T>(__fmul_rn(v.z, factor), __fmul_rn(v.w, factor));
        if (vec && j + 4 <= hidden) {
            *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
        } else {
            const uint32_t words[2] = {lo, hi};
            const T* e = reinterpret_cast<const T*>(words);
            for (int k = 0; k < 4 && j + k < hidden; ++k) dst[k] = e[k];
        }
    }
}

// ---- few rows ---------------------------------------------------------------------------------------------------------------
// The forward pass as a pass over a W that is stored by word: a warp takes 16 words at a time and the whole of K, and keeps a maximum and a
// sum for every row that a lane's words belong to; the block leaves one pair a row.  Rows that do not count ride along: they are read and
// multiplied, and their results are left out.
struct FewRows {
    skinny::Operands o;
    const float* bias;
    const int64_t* targets;
    float2* parts;  // [blocks][rows]
    float* picked;
    unsigned long long* status;
    unsigned long long tag;
};
constexpr int kFewWarps = 2, kFirst = 256;  // K elements that are asked for ahead of the kernel before

struct Running {  // sum exp(logit - most)
    float most = -INFINITY, sum = 0.0f;
    __device__ __forceinline__ void join(float m, float s) {
        const float now = fmaxf(most, m);
        if (now == -INFINITY) {
            sum = __fadd_rn(sum, s);  // zero, or NaN where all logits are
            return;
        }
        sum = __fmaf_rn(s, fast_exp2(__fmul_rn(__fsub_rn(m, now), kLog2E)), __fmul_rn(sum, fast_exp2(__fmul_rn(__fsub_rn(most, now), kLog2E))));
        most = now;
    }
    template <int kN>
    __device__ __forceinline__ void add(const float (&logits)[kN]) {
        float now = most;
#pragma unroll
        for (int i = 0; i < kN; ++i) now = fmaxf(now, logits[i]);
        if (now == -INFINITY) {
#pragma unroll
            for (int i = 0; i < kN; ++i) sum = logits[i] != logits[i] ? logits[i] : sum;
            return;
        }
        sum = __fmul_rn(sum, fast_exp2(__fmul_rn(__fsub_rn(most, now), kLog2E)));
        most = now;
#pragma unroll
        for (int i = 0; i < kN; ++i) sum = __fadd_rn(sum, fast_exp2(__fmul_rn(__fsub_rn(logits[i], now), kLog2E)));
    }
};

// kLong: sums over K are closed as those of tiles are (product16.cuh); on its own since the loop costs the others up to a tenth of their time.
template <bool kBf16, int kBlocks, bool kLong>
__global__ void __launch_bounds__(kFewWarps * 32, 8)
few_rows_kernel(const FewRows f) {
    constexpr int kWords = 16, kRows = 8 * kBlocks, kLane = 2 * kBlocks;  // kLane: rows of a lane
    __shared__ float2 joined[kFewWarps][kRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int groups = (f.o.n + kWords - 1) / kWords;
    {
        const int n0 = ((int)blockIdx.x * kFewWarps + warp) * kWords;
        if (n0 < f.o.n) skinny::prefetch_weights<false>(f.o, n0, 0, f.o.k < kFirst ? f.o.k : kFirst, lane);
    }
    grid_dependency_wait();
    grid_launch_dependents();
    announce_launch(f.status, f.tag);
    auto row_of = [&](int j) { return (j >> 1) * 8 + 2 * t + (j & 1); };
    int target[kLane];
    Running run[kLane];
#pragma unroll
    for (int j = 0; j < kLane; ++j) {
        const int64_t word = row_of(j) < f.o.rows ? f.targets[row_of(j)] : -1;
        target[j] = word >= 0 && word < f.o.n ? (int)word : -1;
    }
    auto logit = [&](int j, int word, float sum) {
        if (word >= f.o.n) return -INFINITY;
        const float l = f.bias != nullptr ? __fadd_rn(sum, f.bias[word]) : sum;
        if (word == target[j]) f.picked[row_of(j)] = l;
        return l;
    };
    for (int group = (int)blockIdx.x * kFewWarps + warp; group < groups; group += (int)gridDim.x * kFewWarps) {
        const int n0 = group * kWords;
        float d[kBlocks][4] = {};
        if constexpr (kLong) {
#pragma unroll 1
            for (int k = 0; k < f.o.k; k += p16::kCloseK) {
                float part[kBlocks][4] = {};
                skinny::by_output<kBf16, kBlocks, (kBlocks > 1 ? 2 : 4)>(f.o, n0, k, k + p16::kCloseK, lane, part);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[b][i] = __fadd_rn(d[b][i], part[b][i]);
                }
            }
        } else {
            skinny::by_output<kBf16, kBlocks, (kBlocks > 1 ? 2 : 4)>(f.o, n0, 0, f.o.k, lane, d);
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float l[2] = {logit(2 * b + h, n0 + g, d[b][h]), logit(2 * b + h, n0 + g + 8, d[b][2 + h])};
                run[2 * b + h].add(l);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kLane; ++j) {  // over the lanes that have other words of the same row
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) run[j].join(__shfl_xor_sync(0xFFFFFFFFu, run[j].most, o), __shfl_xor_sync(0xFFFFFFFFu, run[j].sum, o));
        if (g == 0) joined[warp][row_of(j)] = make_float2(run[j].most, run[j].sum);
    }
    __syncthreads();
    if ((int)threadIdx.x < f.o.rows) {  // at most 32
        Running all;
        for (int w = 0; w < kFewWarps; ++w) all.join(joined[w][threadIdx.x].x, joined[w][threadIdx.x].y);
        f.parts[(int64_t)blockIdx.x * f.o.rows + threadIdx.x] = make_float2(all.most, all.sum);
    }
}

// A team of warps a row over the blocks' pairs (`team` warps: 32 for one row, one for 32 rows), then a warp a row over its team's; the
// mean of the rows that count.
__global__ void __launch_bounds__(1024)
few_rows_join_kernel(const float2* __restrict__ parts, int n_parts, int rows, int team, int vocab, const int64_t* __restrict__ targets,
                     int64_t ignore, const float* __restrict__ picked, float* loss, float* lse_out, float* mean) {
    __shared__ float2 joined[32];
    __shared__ float losses[32];
    __shared__ int counted[32];
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp / team, member = warp % team;
    Running run;
    if (mine < rows) {
#pragma unroll 4
        for (int i = member * 32 + lane; i < n_parts; i += team * 32) {
            const float2 v = parts[(int64_t)i * rows + mine];
            run.join(v.x, v.y);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) run.join(__shfl_xor_sync(0xFFFFFFFFu, run.most, o), __shfl_xor_sync(0xFFFFFFFFu, run.sum, o));
    if (lane == 0) {
        joined[warp] = make_float2(run.most, run.sum);
        losses[warp] = 0.0f;
        counted[warp] = 0;
    }
    __syncthreads();
    const int row = warp;
    if (row < rows) {
        Running all;
        if (lane < team) {
            all.most = joined[row * team + lane].x;
            all.sum = joined[row * team + lane].y;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all.join(__shfl_xor_sync(0xFFFFFFFFu, all.most, o), __shfl_xor_sync(0xFFFFFFFFu, all.sum, o));
        if (lane == 0) {
            const int64_t target = targets[row];
            float lse = 0.0f, l = 0.0f;
            if (target != ignore) {
                const float log = logf(all.sum);
                lse = __fadd_rn(all.most, log);
                if (target >= 0 && target < vocab) l = loss_of(all.most, log, picked[row]);
                else l = lse = __int_as_float(0x7FC00000);  // the target is not a word
                counted[row] = 1;
            }
            if (loss != nullptr) loss[row] = l;
            if (lse_out != nullptr) lse_out[row] = lse;
            losses[row] = l;
        }
    }
    if (mean == nullptr) return;
    __syncthreads();
    if (row == 0) {
        double total = losses[lane];
        int count = counted[lane];
        for (int o = 16; o > 0; o >>= 1) {
            total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
            count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
        }
        if (lane == 0) *mean = (float)(total / (count > 0 ? count : 1));
    }
}

// ---- host side --------------------------------------------------------------------------------------------------------------

bool misaligned(const void* p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }
bool whole(const void* p, int64_t ld, int64_t size) { return !misaligned(p, 16) && (ld * size) % 16 == 0; }
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct Sizes {
    int64_t rows, hidden, vocab;
    bool stored_words;  // W stored with words as rows
};
int loss_sizes(const qfmt_matrix16_t* H, const qfmt_matrix16_t* W, Sizes* s) {
    if (H == nullptr || W == nullptr || H->trans != 0) return QFMT_ERR_BAD_ARG;
    s->stored_words = W->trans != 0;
    s->rows = H->rows;
    s->hidden = H->cols;
    s->vocab = s->stored_words ? W->rows : W->cols;
    if (s->hidden != (s->stored_words ? W->cols : W->rows)) return QFMT_ERR_BAD_ARG;
    if (s->rows < 0 || s->hidden < 1 || s->vocab < 1) return QFMT_ERR_BAD_ARG;
    if (s->rows > (1 << 24) || s->hidden > (1 << 24) || s->vocab > (1 << 28)) return QFMT_ERR_BAD_ARG;
    if (p16::single_tiles(s->rows, s->vocab) > (1 << 26)) return QFMT_ERR_BAD_ARG;
    return QFMT_OK;
}

// How the backward pass walks the vocabulary.  A piece's d (rows x piece, 2 bytes each) should stay in the second-level cache (126 MB)
// between the product that writes it and the two that read it; and pieces of at least 1024 words keep those products whole.  Within
// that a piece has as many 256-word tiles as let the weight gradient's tiles fill whole rounds of the CTA pairs.
constexpr int64_t kPieceBytes = 80ll << 20;
struct Plan {
    int64_t tile_rows;   // rows of whole tiles
    int64_t piece;       // words, a multiple of 256
    int splits;          // of a piece's words in the product for dH
    int64_t pitch_h;     // of the fp32 dH and the compact H
};
Plan plan_backward(const Sizes& s) {
    Plan p;
    p.tile_rows = up(s.rows > 0 ? s.rows : 1, 2 * p16::kRows);
    int64_t most = kPieceBytes / (p.tile_rows * 2) / p16::kTileN;  // tiles of words
    if (most < 4) most = 4;
    const int64_t all = (s.vocab + p16::kTileN - 1) / p16::kTileN, across = up(s.hidden, p16::kTileN) / p16::kTileN;
    if (most < all) {
        const int64_t fill = most * across / p16::kPairs * p16::kPairs / across;  // the most whose tiles make whole rounds
        if (fill > 0) most = fill;
    }
    const int64_t pieces = (all + most - 1) / most;
    p.piece = (all + pieces - 1) / pieces * p16::kTileN;
    p.pitch_h = up(s.hidden, 8);
    p.splits = p16::plan_product(s.rows, s.hidden, p.piece, true).splits;
    return p;
}

// Forward passes that go over W in few_rows_kernel, if it is stored by word: up to eight rows, or up to 32 and 2^25 multiplications
// (measured against tiles: 8 x 1024 x 30522 24.0 against 26.6 us, 16 27.8 against 26.5; 16 x 256 x 4000 9.6 against 12.6, 32 x 256 x 8000
// 15.3 against 13.2; a W stored by K took longer than tiles at nearly every size).  D of at most 2^15: a warp then has
// four closed sums at most.
bool few_rows(const Sizes& s) {
    return s.stored_words && s.hidden <= 1 << 15 && (s.rows <= 8 || (s.rows <= skinny::kMostRows && s.rows * s.vocab * s.hidden <= 1ll << 25));
}

// The workspace's parts, in order; every one starts on 256 bytes.
struct Layout {
    size_t size = 0;
    size_t take(size_t bytes) {
        const size_t at = size;
        size += (bytes + 255) / 256 * 256;
        return at;
    }
};
struct Places {
    size_t found, index, target, compact_h;
    size_t parts, picked, compact_loss;            // forward
    size_t lse_of, g, d, column_parts, sums;         // backward
    size_t total;
};
Places places(const Sizes& s, const Plan& plan, bool backward) {
    Layout l;
    Places p = {};
    l.take(256);  // the status area, Found behind it
    p.found = 64;
    p.index = l.take((size_t)s.rows * 4);
    p.target = l.take((size_t)s.rows * 4);
    p.compact_h = l.take((size_t)up(s.rows, 64) * plan.pitch_h * 2);
    if (!backward) {
        // a pair a row for every 64 words of a tile, or for every block of at least 16 words
        const int64_t words = few_rows(s) ? 16 : 64;
        p.parts = l.take((size_t)(up(s.vocab, words) / words) * s.rows * sizeof(float2));
        p.picked = l.take((size_t)s.rows * 4);
        p.compact_loss = l.take((size_t)s.rows * 4);
    } else {
        p.lse_of = l.take((size_t)s.rows * 4);
        p.g = l.take((size_t)s.rows * 4);
        p.d = l.take((size_t)plan.tile_rows * plan.piece * 2);
        p.column_parts = l.take((size_t)(plan.tile_rows / 32) * plan.piece * 4);
        p.sums = l.take((size_t)plan.splits * s.rows * plan.pitch_h * 4);
    }
    p.total = l.size;
    return p;
}

template <typename T>
T* at(void* workspace, size_t place) { return reinterpret_cast<T*>(static_cast<char*>(workspace) + place); }

int check_loss(const qfmt_matrix16_t* H, const qfmt_matrix16_t* W, const qfmt_cross_entropy_t* kind, const float* d_bias,
               const int64_t* d_targets, void* d_workspace, size_t workspace_bytes, bool backward, Sizes* s) {
    const int rc = loss_sizes(H, W, s);
    if (rc != QFMT_OK) return rc;
    if (kind == nullptr || (kind->dtype != QFMT_F16 && kind->dtype != QFMT_BF16) || (kind->mean != 0 && kind->mean != 1)) return QFMT_ERR_BAD_ARG;
    if (H->ld < H->cols || W->ld < W->cols || misaligned(d_bias, 4) || misaligned(d_targets, 8)) return QFMT_ERR_BAD_ARG;
    if (W->ptr == nullptr || misaligned(W->ptr, 16) || (W->ld & 7)) return QFMT_ERR_BAD_ARG;
    if (s->rows > 0 && (H->ptr == nullptr || misaligned(H->ptr, 16) || (H->ld & 7) || d_targets == nullptr)) return QFMT_ERR_BAD_ARG;
    if (d_workspace == nullptr || misaligned(d_workspace, 16) || workspace_bytes < places(*s, plan_backward(*s), backward).total)
        return QFMT_ERR_BAD_ARG;
    return QFMT_OK;
}

Compact compact_args(const qfmt_matrix16_t* H, const qfmt_cross_entropy_t* kind, const int64_t* d_targets, const Sizes& s,
                     const Plan& plan, const Places& pl, void* ws) {
    Compact c = {};
    c.targets = d_targets;
    c.ignore = kind->ignore_index;
    c.rows = (int)s.rows;
    c.vocab = (int)s.vocab;
    c.found = at<Found>(ws, pl.found);
    c.index = at<int>(ws, pl.index);
    c.target = at<int>(ws, pl.target);
    c.mean = kind->mean;
    c.h = H->ptr;
    c.ld_h = H->ld;
    c.copy = at<uint16_t>(ws, pl.compact_h);
    c.ld_copy = plan.pitch_h;
    c.hidden = (int)s.hidden;
    return c;
}
template <bool kBackward>
int launch_compact(Compact c, const p16::ProductParams& p, const DeviceInfo& dev, cudaStream_t stream) {
    const int most = 2 * dev.sm_count;
    int blocks = (c.rows + 31) / 32;
    if (blocks > most) blocks = most;
    c.rows_per_block = (c.rows + blocks - 1) / blocks;
    blocks = (c.rows + c.rows_per_block - 1) / c.rows_per_block;
    QFMT_CUDA_TRY(launch_overlapping(compact_kernel<kBackward>, (unsigned)blocks, (unsigned)kCompactThreads, 0, stream, c, p.status, p.tag));
    return QFMT_OK;
}

// W's words first .. first + n - 1 as an operand: `words`: the words are the extent (logits), else they are K (dH).
int word_operand(p16::Operand* o, bool pair, const qfmt_matrix16_t* W, const Sizes& s, bool words, int64_t first, int64_t n) {
    const uint16_t* base = W->ptr + (s.stored_words ? first * W->ld : first);
    return p16::make_operand(o, true, pair, base, words != s.stored_words, words ? n : s.hidden, words ? s.hidden : n, W->ld);
}

template <bool kBf16, bool kLong>
int launch_few_rows(const FewRows& f, const DeviceInfo& dev, unsigned* blocks, cudaStream_t stream) {
    const unsigned want = (unsigned)((f.o.n + 16 * kFewWarps - 1) / (16 * kFewWarps)), most = 8u * dev.sm_count;
    *blocks = want < most ? want : most;
    auto* kernel = f.o.rows <= 8    ? few_rows_kernel<kBf16, 1, kLong>
                   : f.o.rows <= 16 ? few_rows_kernel<kBf16, 2, kLong>
                                    : few_rows_kernel<kBf16, 4, kLong>;
    QFMT_CUDA_TRY(launch_overlapping(kernel, *blocks, kFewWarps * 32u, 0, stream, f));
    return QFMT_OK;
}

// H in the compact copy or in place, as rows of the logits' product or as the K of the weight gradient's.
struct Tokens {
    p16::Operand copy, whole;
};
int token_operand(Tokens* o, bool is_b, bool pair, const qfmt_matrix16_t* H, const Sizes& s, const Plan& plan, const uint16_t* copy, bool rows) {
    const int64_t n = rows ? up(s.rows, 64) : s.hidden, k = rows ? s.hidden : up(s.rows, 64);
    const int rc = p16::make_operand(&o->copy, is_b, pair, copy, !rows, n, k, plan.pitch_h);
    if (rc != QFMT_OK) return rc;
    return p16::make_operand(&o->whole, is_b, pair, H->ptr, !rows, rows ? s.rows : s.hidden, rows ? s.hidden : s.rows, H->ld);
}

template <typename T>
int backward_pieces(const qfmt_matrix16_t* H, const qfmt_matrix16_t* W, const float* d_bias, const Sizes& s, const Plan& plan, const Places& pl,
                    void* ws, p16::ProductParams base, void* d_dh, int64_t ld_dh, void* d_dw, int64_t ld_dw, float* d_dbias,
                    const DeviceInfo& dev, cudaStream_t stream) {
    const Found* found = at<Found>(ws, pl.found);
    const uint16_t* copy = at<uint16_t>(ws, pl.compact_h);
    T* d = at<T>(ws, pl.d);
    float* column_parts = at<float>(ws, pl.column_parts);
    float* sums = at<float>(ws, pl.sums);
    int rc;
    for (int64_t first = 0; first < s.vocab; first += plan.piece) {
        const int64_t n = first + plan.piece < s.vocab ? plan.piece : s.vocab - first, n64 = up(n, 64);
        // d of this piece
        Tokens h;
        p16::Operand w, g;
        p16::ProductPlan pp = p16::plan_product(s.rows, n, s.hidden, false);
        rc = token_operand(&h, false, pp.pair, H, s, plan, copy, true);
        if (rc == QFMT_OK) rc = word_operand(&w, pp.pair, W, s, true, first, n);
        if (rc != QFMT_OK) return rc;
        p16::ProductParams p = base;
        p.M = (int)s.rows;
        p.N = (int)n;
        p.K = (int)s.hidden;
        p.dyn = p16::kCountM;
        p.alt = p16::kAltA;
        p.splits = 1;
        p.kb_per_split = pp.kb_per_split;
        typename GradEpilogue<T>::Params ge = {d_bias != nullptr ? d_bias + first : nullptr, at<int>(ws, pl.target), at<float>(ws, pl.lse_of),
                                               at<float>(ws, pl.g), d, d_dbias != nullptr ? column_parts : nullptr, plan.piece, (int)first};
        rc = p16::launch_product<GradEpilogue<T>>(pp.pair, h.copy, w, &h.whole, p, ge, dev, stream);
        if (rc != QFMT_OK) return rc;
        if (d_dbias != nullptr) {
            rc = launch_join_columns(column_parts, plan.piece, plan.tile_rows / 32, &found->count, pp.pair ? 2 * p16::kRows : p16::kRows,
                                     &found->unscale, d_dbias + first, n, stream);
            if (rc != QFMT_OK) return rc;
        }
        if (d_dw != nullptr) {
            p.M = (int)(s.stored_words ? n : s.hidden);
            p.N = (int)(s.stored_words ? s.hidden : n);
            p.K = (int)s.rows;
            p.dyn = p16::kCountK;
            p.alt = s.stored_words ? p16::kAltB : p16::kAltA;
            pp = p16::plan_product(p.M, p.N, s.rows, false);
            p.kb_per_split = pp.kb_per_split;
            rc = token_operand(&h, s.stored_words, pp.pair, H, s, plan, copy, false);
            if (rc == QFMT_OK) rc = p16::make_operand(&g, !s.stored_words, pp.pair, d, true, n64, plan.tile_rows, plan.piece);
            if (rc != QFMT_OK) return rc;
            T* out = static_cast<T*>(d_dw) + (s.stored_words ? first * ld_dw : first);
            typename ScaledEpilogue<T>::Params se = {&found->unscale, out, ld_dw, whole(out, ld_dw, 2)};
            if (s.stored_words) rc = p16::launch_product<ScaledEpilogue<T>>(pp.pair, g, h.copy, &h.whole, p, se, dev, stream);
            else rc = p16::launch_product<ScaledEpilogue<T>>(pp.pair, h.copy, g, &h.whole, p, se, dev, stream);
            if (rc != QFMT_OK) return rc;
        }
        if (d_dh != nullptr) {
            p.M = (int)s.rows;
            p.N = (int)s.hidden;
            p.K = (int)n;
            p.dyn = p16::kCountM;
            p.alt = p16::kAltNone;
            pp = p16::plan_product(s.rows, s.hidden, plan.piece, true);
            p.splits = plan.splits;
            // a short last piece is shared as finely: some splits may be left without work and add zeros
            p.kb_per_split = (int)p16::ceil_div(p16::ceil_div(n, p16::kStageK), plan.splits);
            rc = p16::make_operand(&g, false, pp.pair, d, false, plan.tile_rows, n64, plan.piece);
            if (rc == QFMT_OK) rc = word_operand(&w, pp.pair, W, s, false, first, n);
            if (rc != QFMT_OK) return rc;
            typename AddEpilogue::Params ae = {sums, plan.pitch_h, s.rows * plan.pitch_h, first > 0 ? 1 : 0};
            rc = p16::launch_product<AddEpilogue>(pp.pair, g, w, nullptr, p, ae, dev, stream);
            if (rc != QFMT_OK) return rc;
        }
    }
    if (d_dh != nullptr) {
        const int64_t want = (s.rows * ((s.hidden + 127) / 128) + 7) / 8, most = (int64_t)dev.sm_count * 8;
        QFMT_CUDA_TRY(launch_overlapping(scatter_kernel<T>, (unsigned)(want < most ? want : most), 256u, 0, stream, (const float*)sums, plan.splits,
                                         s.rows * plan.pitch_h, plan.pitch_h, found, (const int*)at<int>(ws, pl.index), static_cast<T*>(d_dh),
                                         ld_dh, (int)s.hidden, (int)(!misaligned(d_dh, 8) && ld_dh % 4 == 0)));
    }
    return QFMT_OK;
}

}  // namespace
}  // namespace qfmt

extern "C" size_t qfmt_linear_cross_entropy_workspace_bytes(const qfmt_matrix16_t* H, const qfmt_matrix16_t* W, int backward) {
    qfmt::Sizes s;
    if (qfmt::loss_sizes(H, W, &s) != QFMT_OK) return 0;
    return qfmt::places(s, qfmt::plan_backward(s), backward != 0).total;
}

extern "C" int qfmt_linear_cross_entropy(const qfmt_matrix16_t* H, const qfmt_matrix16_t* W, const qfmt_cross_entropy_t* kind,
                                         const float* d_bias, const int64_t* d_targets, float* d_loss, float* d_lse, float* d_mean,
                                         void* d_workspace, size_t workspace_bytes, void* stream) {
    using namespace qfmt;
    Sizes s;
    int rc = check_loss(H, W, kind, d_bias, d_targets, d_workspace, workspace_bytes, false, &s);
    if (rc != QFMT_OK) return rc;
    if (misaligned(d_loss, 4) || misaligned(d_lse, 4) || misaligned(d_mean, 4)) return QFMT_ERR_BAD_ARG;
    DeviceInfo dev;
    rc = current_device(&dev);
    if (rc != QFMT_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (s.rows == 0) {
        if (d_mean != nullptr) QFMT_CUDA_TRY(cudaMemsetAsync(d_mean, 0, sizeof(float), st));
        return QFMT_OK;
    }
    const Plan plan = plan_backward(s);
    const Places pl = places(s, plan, false);
    if (few_rows(s)) {
        FewRows f = {skinny::Operands{H->ptr, W->ptr, H->ld, W->ld, (int)s.rows, (int)s.vocab, (int)s.hidden}, d_bias, d_targets,
                     at<float2>(d_workspace, pl.parts), at<float>(d_workspace, pl.picked), static_cast<unsigned long long*>(d_workspace),
                     next_launch_tag()};
        unsigned blocks = 0;
        const bool closed = s.hidden > p16::kCloseK;
        if (kind->dtype == QFMT_BF16) rc = closed ? launch_few_rows<true, true>(f, dev, &blocks, st) : launch_few_rows<true, false>(f, dev, &blocks, st);
        else rc = closed ? launch_few_rows<false, true>(f, dev, &blocks, st) : launch_few_rows<false, false>(f, dev, &blocks, st);
        if (rc != QFMT_OK) return rc;
        int team = 32;
        while (team > 1 && team * s.rows > 32) team /= 2;
        QFMT_CUDA_TRY(launch_overlapping(few_rows_join_kernel, 1u, 1024u, 0, st, (const float2*)f.parts, (int)blocks, (int)s.rows, team, (int)s.vocab,
                                         d_targets, kind->ignore_index, (const float*)f.picked, d_loss, d_lse, d_mean));
        return QFMT_OK;
    }
    const p16::ProductPlan pp = p16::plan_product(s.rows, s.vocab, s.hidden, false);
    Tokens h;
    p16::Operand w;
    rc = token_operand(&h, false, pp.pair, H, s, plan, at<uint16_t>(d_workspace, pl.compact_h), true);
    if (rc == QFMT_OK) rc = word_operand(&w, pp.pair, W, s, true, 0, s.vocab);
    if (rc != QFMT_OK) return rc;
    Compact c = compact_args(H, kind, d_targets, s, plan, pl, d_workspace);
    c.loss = d_loss;
    c.lse_out = d_lse;
    p16::ProductParams p = {};
    p.M = (int)s.rows;
    p.N = (int)s.vocab;
    p.K = (int)s.hidden;
    p.count = &c.found->count;
    p.dyn = p16::kCountM;
    p.alt = p16::kAltA;
    p.alt_rows = (int)s.rows;
    p.bf16 = kind->dtype == QFMT_BF16;
    p.splits = 1;
    p.kb_per_split = (int)(up(s.hidden, p16::kStageK) / p16::kStageK);
    p.status = static_cast<unsigned long long*>(d_workspace);
    p.tag = next_launch_tag();
    rc = launch_compact<false>(c, p, dev, st);
    if (rc != QFMT_OK) return rc;
    typename RowSumEpilogue::Params re = {d_bias, c.target, at<float2>(d_workspace, pl.parts), at<float>(d_workspace, pl.picked), s.rows};
    rc = p16::launch_product<RowSumEpilogue>(pp.pair, h.copy, w, &h.whole, p, re, dev, st);
    if (rc != QFMT_OK) return rc;
    const unsigned blocks = (unsigned)((s.rows + kJoinRows - 1) / kJoinRows);
    float* compact_loss = d_mean != nullptr && blocks > 1 ? at<float>(d_workspace, pl.compact_loss) : nullptr;
    QFMT_CUDA_TRY(launch_overlapping(join_rows_kernel, blocks, (unsigned)(kJoinRows * kJoinParts), 0, st, (const float2*)re.parts, s.rows,
                                     (int)(up(s.vocab, 64) / 64), (const Found*)c.found, (const int*)c.index, (const int*)c.target,
                                     (const float*)re.picked, d_loss, d_lse, compact_loss, blocks == 1 ? d_mean : (float*)nullptr));
    if (compact_loss != nullptr)
        QFMT_CUDA_TRY(launch_overlapping(mean_kernel, 1u, 1024u, 0, st, (const float*)compact_loss, (const Found*)c.found, d_mean));
    return QFMT_OK;
}

extern "C" int qfmt_linear_cross_entropy_backward(const qfmt_matrix16_t* H, const qfmt_matrix16_t* W, const qfmt_cross_entropy_t* kind,
                                                  const float* d_bias, const int64_t* d_targets, const float* d_lse, const float* d_dloss,
                                                  const qfmt_dls_t* d_dls, void* d_dh, int64_t ld_dh, void* d_dw, int64_t ld_dw,
                                                  float* d_dbias, void* d_workspace, size_t workspace_bytes, void* stream) {
    using namespace qfmt;
    Sizes s;
    int rc = check_loss(H, W, kind, d_bias, d_targets, d_workspace, workspace_bytes, true, &s);
    if (rc != QFMT_OK) return rc;
    if (misaligned(d_lse, 4) || misaligned(d_dloss, 4) || misaligned(d_dls, 8) || misaligned(d_dh, 2) || misaligned(d_dw, 2) ||
        misaligned(d_dbias, 4))
        return QFMT_ERR_BAD_ARG;
    if (s.rows > 0 && d_lse == nullptr) return QFMT_ERR_BAD_ARG;
    if ((d_dh != nullptr && ld_dh < s.hidden) || (d_dw != nullptr && ld_dw < W->cols)) return QFMT_ERR_BAD_ARG;
    DeviceInfo dev;
    rc = current_device(&dev);
    if (rc != QFMT_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (s.rows == 0) {
        if (d_dw != nullptr) QFMT_CUDA_TRY(cudaMemset2DAsync(d_dw, (size_t)ld_dw * 2, 0, (size_t)W->cols * 2, (size_t)W->rows, st));
        if (d_dbias != nullptr) QFMT_CUDA_TRY(cudaMemsetAsync(d_dbias, 0, (size_t)s.vocab * sizeof(float), st));
        return QFMT_OK;
    }
    const Plan plan = plan_backward(s);
    const Places pl = places(s, plan, true);
    Compact c = compact_args(H, kind, d_targets, s, plan, pl, d_workspace);
    c.lse = d_lse;
    c.dloss = d_dloss;
    c.dls = d_dls;
    c.lse_of = at<float>(d_workspace, pl.lse_of);
    c.g = at<float>(d_workspace, pl.g);
    c.dh = static_cast<uint16_t*>(d_dh);
    c.ld_dh = ld_dh;
    p16::ProductParams p = {};
    p.count = &c.found->count;
    p.alt_rows = (int)s.rows;
    p.bf16 = kind->dtype == QFMT_BF16;
    p.status = static_cast<unsigned long long*>(d_workspace);
    p.tag = next_launch_tag();
    rc = launch_compact<true>(c, p, dev, st);
    if (rc != QFMT_OK) return rc;
    if (kind->dtype == QFMT_F16)
        return backward_pieces<__half>(H, W, d_bias, s, plan, pl, d_workspace, p, d_dh, ld_dh, d_dw, ld_dw, d_dbias, dev, st);
    return backward_pieces<__nv_bfloat16>(H, W, d_bias, s, plan, pl, d_workspace, p, d_dh, ld_dh, d_dw, ld_dw, d_dbias, dev, st);
}
