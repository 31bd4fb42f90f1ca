// Layer normalisation, and its fused form y = LN(residual + D(x)), forward and backward.
//
//   mean = sum_c h / n        rstd = 1 / sqrt(sum_c (h - mean)^2 / n + eps)
//   y    = (h - mean) rstd w + b
//   xhat = (h - mean) rstd,  g = w dy
//   dh   = rstd (g - sum_c g / n - xhat sum_c (g xhat) / n)        dw = sum_r dy xhat        db = sum_r dy
//
// Everything is held in 32 bits between the loads and the one rounding of each stored value; the forward pass
// normalises the 32-bit sum, not the stored h.
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

#include "common.cuh"
#include "elements.cuh"

namespace qfmt {
namespace {

template <int kType>
struct ForwardArgs {
    using W = typename Word<kType>::type;
    const W* x;
    const W* residual;  // or NULL
    const float* weight;
    const float* bias;
    W* h;  // or NULL
    W* y;
    float* mean;
    float* rstd;
    int64_t ld_x, ld_residual, ld_h, ld_y;
    int64_t rows, cols;
    float eps;
    bool vec;
    bool fmt;  // quant holds a format to round to
    DropParams drop;
    QuantParams quant;
    qfmt_stats_t* stats;
};

template <int kType>
struct BackwardArgs {
    using W = typename Word<kType>::type;
    const W* dy;
    const W* dh;  // gradient that reaches h by another path, or NULL
    const W* h;
    const float* mean;
    const float* rstd;
    const float* weight;
    W* dx;         // or NULL
    W* dresidual;  // or NULL
    float* partial;  // [parts][2][cols] sums of dy xhat and dy over a part of the rows, or NULL
    int64_t ld_dy, ld_dh, ld_h, ld_dx, ld_dresidual;
    int64_t rows, cols;
    bool vec;
    bool fmt;  // quant holds a format to round to
    DropParams drop;
    QuantParams quant;
    qfmt_stats_t* stats;
};

__device__ __forceinline__ int granule_columns(int64_t cols, int64_t col) {
    const int64_t left = cols - col;
    return left < kGranule ? (int)left : kGranule;
}

// h of one granule: x, or residual + D(x).
template <int kType, bool kFused>
__device__ __forceinline__ void load_h(const ForwardArgs<kType>& a, int64_t row, uint32_t g, int n, uint64_t offset,
                                       float (&v)[kGranule]) {
    const int64_t col = (int64_t)g * kGranule;
    load_granule<kType>(a.x + row * a.ld_x + col, n, a.vec, v);
    if constexpr (kFused) {
        if (a.drop.threshold != 0u) drop_granule(a.drop, offset, (uint32_t)row, g, v);
        if (a.residual != nullptr) {
            float r[kGranule];
            load_granule<kType>(a.residual + row * a.ld_residual + col, n, a.vec, r);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) v[j] = add_ieee(r[j], v[j]);
        }
    }
}

// `n` entries of a vector of one value per column, or `fill` where there is none.  kVec: all eight, aligned.
template <bool kVec>
__device__ __forceinline__ void load_columns(const float* p, int64_t col, int n, float fill, float (&v)[kGranule]) {
    if (kVec && p != nullptr) {
        const float4 lo = __ldg(reinterpret_cast<const float4*>(p + col)), hi = __ldg(reinterpret_cast<const float4*>(p + col) + 1);
        v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w;
        v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
    } else {
#pragma unroll
        for (int j = 0; j < kGranule; ++j) v[j] = p != nullptr && j < n ? __ldg(p + col + j) : fill;
    }
}

// Sum over the block in every thread, in a fixed order.  `scratch` holds one entry per warp.
__device__ __forceinline__ float2 block_sum(float2 s, float2* scratch) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, off);
        s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, off);
    }
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    s = lane < warps ? scratch[lane] : make_float2(0.0f, 0.0f);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, off);
        s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, off);
    }
    __syncthreads();  // the scratch may be written again
    return s;
}

constexpr int kLoopThreads = 512;

// A block takes a row at a time and reads it three times: for the mean, for the variance, for the result.
template <int kType, bool kFused, bool kFmt>
__global__ void __launch_bounds__(kLoopThreads) norm_forward_loop_kernel(const ForwardArgs<kType> a) {
    extern __shared__ uint32_t lane_hist[];
    __shared__ float2 scratch[32];
    uint32_t* hist = kFmt && a.stats != nullptr ? lane_hist : nullptr;
    if (hist != nullptr) clear_hist(hist, a.quant);
    const uint32_t granules = (uint32_t)((a.cols + kGranule - 1) / kGranule);
    const float count = (float)a.cols;
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f;
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            const int n = granule_columns(a.cols, (int64_t)g * kGranule);
            float v[kGranule];
            load_h<kType, kFused>(a, row, g, n, offset, v);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) sum += v[j];
        }
        const float mean = block_sum(make_float2(sum, 0.0f), scratch).x / count;
        float square = 0.0f;
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            const int n = granule_columns(a.cols, (int64_t)g * kGranule);
            float v[kGranule];
            load_h<kType, kFused>(a, row, g, n, offset, v);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) {
                const float d = j < n ? v[j] - mean : 0.0f;
                square = __fmaf_rn(d, d, square);
            }
        }
        const float rstd = 1.0f / sqrtf(block_sum(make_float2(square, 0.0f), scratch).x / count + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean != nullptr) a.mean[row] = mean;
            if (a.rstd != nullptr) a.rstd[row] = rstd;
        }
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            const int64_t col = (int64_t)g * kGranule;
            const int n = granule_columns(a.cols, col);
            float v[kGranule], w[kGranule], b[kGranule];
            load_h<kType, kFused>(a, row, g, n, offset, v);
            if (kFused && a.h != nullptr)
                store_granule<kType>(a.h + row * a.ld_h + col, n, a.vec, finish<kType, false>(v, n, a.quant, nullptr));
            load_columns<false>(a.weight, col, n, 1.0f, w);
            load_columns<false>(a.bias, col, n, 0.0f, b);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) v[j] = __fmaf_rn((v[j] - mean) * rstd, w[j], b[j]);
            store_granule<kType>(a.y + row * a.ld_y + col, n, a.vec, finish<kType, kFmt>(v, n, a.quant, hist));
        }
    }
    if (hist != nullptr) flush_hist(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
}

// Teams: the threads that share a row.  A team of up to 32 threads is an aligned part of a warp; a larger
// one is whole warps.  Granule k * team + t of the row is thread t's k-th.

// Sum over a team in every thread, in a fixed order.  scratch: 16 entries per team, of which those past the
// team's warps are zero; one barrier, so the next sum needs another scratch.
__device__ __forceinline__ float2 team_sum(float2 s, int team, int t, int barrier, float2* scratch) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        if (off < team) {
            s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, off);
            s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, off);
        }
    }
    if (team > 32) {
        if ((t & 31) == 0) scratch[t >> 5] = s;
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(team) : "memory");
        const float4* q = reinterpret_cast<const float4*>(scratch);
        s = make_float2(0.0f, 0.0f);
        for (int i = 0; i < team; i += 128) {  // four warps' entries
            const float4 u = q[i / 64], v = q[i / 64 + 1];
            s.x += (u.x + u.z) + (v.x + v.z);
            s.y += (u.y + u.w) + (v.y + v.w);
        }
    }
    return s;
}

constexpr int kRowThreads = 512;

// A row is read once and stays in its team's registers.
template <int kType, int V, bool kFused, bool kVec>
__global__ void __launch_bounds__(kRowThreads) norm_forward_rows_kernel(const ForwardArgs<kType> a, int team) {
    extern __shared__ uint32_t lane_hist[];
    __shared__ float2 scratch[2][16];
    uint32_t* hist = a.stats != nullptr ? lane_hist : nullptr;
    if (team > 32) {
        if (threadIdx.x < 32) scratch[threadIdx.x >> 4][threadIdx.x & 15] = make_float2(0.0f, 0.0f);
        __syncthreads();
    }
    if (hist != nullptr) clear_hist(hist, a.quant);
    const int t = team > 32 ? (int)threadIdx.x : (int)threadIdx.x & (team - 1);
    const int teams = blockDim.x / team;
    const float inverse = 1.0f / (float)a.cols;
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    // the last teams of a warp may have no row while its other teams have one: they go through the motions
    for (int64_t base = (int64_t)blockIdx.x * teams; base < a.rows; base += (int64_t)gridDim.x * teams) {
        const int64_t row = base + threadIdx.x / team;
        float v[V][kGranule];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int64_t col = (int64_t)(k * team + t) * kGranule;
            const int n = row < a.rows && col < a.cols ? granule_columns(a.cols, col) : 0;
#pragma unroll
            for (int j = 0; j < kGranule; ++j) v[k][j] = 0.0f;
            if (n > 0) load_granule<kType, kVec>(a.x + row * a.ld_x + col, n, v[k]);
        }
        if constexpr (kFused) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int64_t col = (int64_t)(k * team + t) * kGranule;
                const int n = row < a.rows && col < a.cols ? granule_columns(a.cols, col) : 0;
                if (n > 0) {
                    float r[kGranule];
                    if (a.residual != nullptr) load_granule<kType, kVec>(a.residual + row * a.ld_residual + col, n, r);
                    if (a.drop.threshold != 0u) drop_granule(a.drop, offset, (uint32_t)row, k * team + t, v[k]);
                    if (a.residual != nullptr) {
#pragma unroll
                        for (int j = 0; j < kGranule; ++j) v[k][j] = add_ieee(r[j], v[k][j]);
                    }
                    if (a.h != nullptr)
                        store_granule<kType, kVec>(a.h + row * a.ld_h + col, n, finish<kType, false>(v[k], n, a.quant, nullptr));
                }
            }
        }
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int j = 0; j < kGranule; ++j) s.x += v[k][j];
        const float mean = team_sum(s, team, t, 1, scratch[0]).x * inverse;
        s.x = 0.0f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int64_t col = (int64_t)(k * team + t) * kGranule;
#pragma unroll
            for (int j = 0; j < kGranule; ++j) {
                v[k][j] = col + j < a.cols ? v[k][j] - mean : 0.0f;
                s.x = __fmaf_rn(v[k][j], v[k][j], s.x);
            }
        }
        const float rstd = 1.0f / sqrtf(team_sum(s, team, t, 1, scratch[1]).x * inverse + a.eps);
        if (t == 0 && row < a.rows) {
            if (a.mean != nullptr) a.mean[row] = mean;
            if (a.rstd != nullptr) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int64_t col = (int64_t)(k * team + t) * kGranule;
            const int n = row < a.rows && col < a.cols ? granule_columns(a.cols, col) : 0;
            if (n > 0) {
                float w[kGranule], b[kGranule];
                load_columns<kVec>(a.weight, col, n, 1.0f, w);
                load_columns<kVec>(a.bias, col, n, 0.0f, b);
#pragma unroll
                for (int j = 0; j < kGranule; ++j) v[k][j] = __fmaf_rn(v[k][j] * rstd, w[j], b[j]);
                store_granule<kType, kVec>(a.y + row * a.ld_y + col, n,
                                           a.fmt ? finish<kType, true>(v[k], n, a.quant, hist) : finish<kType, false>(v[k], n, a.quant, nullptr));
            }
        }
    }
    if (hist != nullptr) flush_hist(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
}

template <int kType>
__device__ __forceinline__ void load_xhat_dy(const BackwardArgs<kType>& a, int64_t row, int64_t col, int n, float mean, float rstd,
                                             float (&xhat)[kGranule], float (&dy)[kGranule]) {
    load_granule<kType>(a.h + row * a.ld_h + col, n, a.vec, xhat);
    load_granule<kType>(a.dy + row * a.ld_dy + col, n, a.vec, dy);
#pragma unroll
    for (int j = 0; j < kGranule; ++j) xhat[j] = j < n ? (xhat[j] - mean) * rstd : 0.0f;
}

// The gradient of h, and D of it: a block takes a row at a time and reads it twice.
template <int kType, bool kFused, bool kFmt>
__global__ void __launch_bounds__(kLoopThreads) norm_backward_loop_kernel(const BackwardArgs<kType> a) {
    extern __shared__ uint32_t lane_hist[];
    __shared__ float2 scratch[32];
    uint32_t* hist = kFmt && a.stats != nullptr ? lane_hist : nullptr;
    if (hist != nullptr) clear_hist(hist, a.quant);
    const uint32_t granules = (uint32_t)((a.cols + kGranule - 1) / kGranule);
    const float count = (float)a.cols;
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float2 s = make_float2(0.0f, 0.0f);
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            const int64_t col = (int64_t)g * kGranule;
            const int n = granule_columns(a.cols, col);
            float xhat[kGranule], dy[kGranule], w[kGranule];
            load_xhat_dy<kType>(a, row, col, n, mean, rstd, xhat, dy);
            load_columns<false>(a.weight, col, n, 1.0f, w);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) {
                const float t = dy[j] * w[j];
                s.x += t;
                s.y = __fmaf_rn(t, xhat[j], s.y);
            }
        }
        s = block_sum(s, scratch);
        const float c1 = s.x / count, c2 = s.y / count;
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            const int64_t col = (int64_t)g * kGranule;
            const int n = granule_columns(a.cols, col);
            float xhat[kGranule], dy[kGranule], w[kGranule];
            load_xhat_dy<kType>(a, row, col, n, mean, rstd, xhat, dy);
            load_columns<false>(a.weight, col, n, 1.0f, w);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) dy[j] = rstd * (__fmaf_rn(dy[j], w[j], -c1) - xhat[j] * c2);
            if (kFused) {
                if (a.dh != nullptr) {
                    float more[kGranule];
                    load_granule<kType>(a.dh + row * a.ld_dh + col, n, a.vec, more);
#pragma unroll
                    for (int j = 0; j < kGranule; ++j) dy[j] += more[j];
                }
                if (a.dresidual != nullptr)
                    store_granule<kType>(a.dresidual + row * a.ld_dresidual + col, n, a.vec, finish<kType, false>(dy, n, a.quant, nullptr));
                if (a.drop.threshold != 0u && a.dx != nullptr) drop_granule(a.drop, offset, (uint32_t)row, g, dy);
            }
            if (a.dx != nullptr)
                store_granule<kType>(a.dx + row * a.ld_dx + col, n, a.vec, finish<kType, kFmt>(dy, n, a.quant, hist));
        }
    }
    if (hist != nullptr) flush_hist(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
}

// Sums over rows for the gradients of weight and bias: a block takes 32 granules of columns and one part of
// the rows, its eight warps every eighth row; their sums are joined in a fixed order.
constexpr int kColumnWarps = 8;
template <int kType>
__global__ void __launch_bounds__(32 * kColumnWarps) norm_column_sums_kernel(const BackwardArgs<kType> a) {
    __shared__ float part[kColumnWarps][2][kGranule][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = ((int64_t)blockIdx.x * 32 + lane) * kGranule;
    const int n = col < a.cols ? granule_columns(a.cols, col) : 0;
    float dw[kGranule] = {}, db[kGranule] = {};
    if (n > 0) {
        for (int64_t row = (int64_t)blockIdx.y * kColumnWarps + warp; row < a.rows; row += (int64_t)gridDim.y * kColumnWarps) {
            float xhat[kGranule], dy[kGranule];
            load_xhat_dy<kType>(a, row, col, n, a.mean[row], a.rstd[row], xhat, dy);
#pragma unroll
            for (int j = 0; j < kGranule; ++j) {
                dw[j] = __fmaf_rn(dy[j], xhat[j], dw[j]);
                db[j] += dy[j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kGranule; ++j) {
        part[warp][0][j][lane] = dw[j];
        part[warp][1][j][lane] = db[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kGranule * 32; i += 32 * kColumnWarps) {
        const int which = i / (kGranule * 32), l = i % (kGranule * 32) / kGranule, j = i % kGranule;
        const int64_t c = ((int64_t)blockIdx.x * 32 + l) * kGranule + j;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kColumnWarps; ++w) s += part[w][which][j][l];
        if (c < a.cols) a.partial[((int64_t)blockIdx.y * 2 + which) * a.cols + c] = s;
    }
}

// Joins the parts in a fixed order: a block takes 32 columns, its eight warps every eighth part.
__global__ void __launch_bounds__(32 * kColumnWarps)
norm_join_parts_kernel(const float* __restrict__ partial, int parts, int64_t cols, float* dweight, float* dbias) {
    __shared__ float sums[kColumnWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float* const out = blockIdx.y == 0 ? dweight : dbias;
    if (out == nullptr) return;
    float s = 0.0f;
    if (c < cols)
        for (int k = warp; k < parts; k += kColumnWarps) s += partial[((int64_t)k * 2 + blockIdx.y) * cols + c];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < cols) {
#pragma unroll
        for (int w = 1; w < kColumnWarps; ++w) s += sums[w][lane];
        out[c] = s;
    }
}

// Parts the rows are summed in for the gradients of weight and bias.
int row_parts(int64_t rows) {
    const int64_t want = (rows + 8 * kColumnWarps - 1) / (8 * kColumnWarps);
    return (int)(want < 64 ? (want > 0 ? want : 1) : 64);
}

struct Call {  // what every entry point checks and works out once
    qfmt_norm_t norm;
    DropParams drop;
    QuantParams quant;
    DeviceInfo dev;
    size_t hist_bytes;
    bool fmt;
};

int prepare_call(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, const qfmt_format_t* fmt, const qfmt_stats_t* d_stats,
                 int accumulate, Call* c) {
    if (norm == nullptr) return QFMT_ERR_BAD_ARG;
    c->norm = *norm;
    qfmt_norm_t& s = c->norm;
    if (s.rows < 0 || s.cols < 0 || s.rows > 0x7FFFFFFF || s.cols > 0x7FFFFFFF) return QFMT_ERR_BAD_ARG;
    if (s.dtype < QFMT_F32 || s.dtype > QFMT_BF16 || !(s.eps >= 0.0f) || !std::isfinite(s.eps)) return QFMT_ERR_BAD_ARG;
    for (int64_t* ld : {&s.ld_x, &s.ld_residual, &s.ld_h, &s.ld_y, &s.ld_dy, &s.ld_dh, &s.ld_dx, &s.ld_dresidual}) {
        if (*ld == 0) *ld = s.cols;
        if (*ld < s.cols) return QFMT_ERR_BAD_ARG;
    }
    int rc = make_drop_params(drop, &c->drop);
    if (rc != QFMT_OK) return rc;
    if (accumulate != 0 && accumulate != 1) return QFMT_ERR_BAD_ARG;
    c->fmt = fmt != nullptr;
    c->quant = QuantParams{};
    c->hist_bytes = 0;
    if (fmt != nullptr) {
        rc = validate_format(fmt);
        if (rc != QFMT_OK) return rc;
        if (fmt->loss_scale != 1.0f) return QFMT_ERR_BAD_FORMAT;
        if (s.dtype == QFMT_F16 && (fmt->e != 5 || fmt->m != 10)) return QFMT_ERR_BAD_FORMAT;
        if (s.dtype == QFMT_BF16 && (fmt->e != 8 || fmt->m != 7)) return QFMT_ERR_BAD_FORMAT;
        c->quant = make_params(*fmt);
        if (d_stats != nullptr) c->hist_bytes = (size_t)(c->quant.top + kExtraBins) * 32 * sizeof(uint32_t);
    } else if (d_stats != nullptr) {
        return QFMT_ERR_BAD_ARG;  // bins are those of a format
    }
    if (reinterpret_cast<uintptr_t>(d_stats) & 7u) return QFMT_ERR_BAD_ARG;
    return QFMT_OK;
}

bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Threads that share a row and the granules each of them holds: the fewest that cover it with at most four
// granules a thread (fewer barriers and shuffles per element than one granule a thread).
struct Team {
    int threads, granules;
};
Team forward_team(int64_t cols) {
    const int64_t g = (cols + kGranule - 1) / kGranule;
    if (g > 4 * kRowThreads) return {0, 0};
    if (g <= 32) {
        int threads = 1;
        while (threads < g) threads *= 2;
        return {threads, 1};
    }
    if (g <= 64) return {32, 2};
    return {(int)((g + 127) / 128) * 32, 4};
}

bool column_aligned(const float* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <int kType, bool kFused>
int launch_forward(const Call& c, const ForwardArgs<kType>& a, cudaStream_t stream) {
    const Team team = forward_team(a.cols);
    if (team.threads != 0) {
        const bool vec = a.vec && a.cols % kGranule == 0 && column_aligned(a.weight) && column_aligned(a.bias);
        const unsigned block = team.threads > 32 ? team.threads : 128;
        const int64_t want = (a.rows * team.threads + block - 1) / block, cap = (int64_t)c.dev.sm_count * 32;
        const auto kern = vec ? (team.granules == 1   ? norm_forward_rows_kernel<kType, 1, kFused, true>
                                 : team.granules == 2 ? norm_forward_rows_kernel<kType, 2, kFused, true>
                                                      : norm_forward_rows_kernel<kType, 4, kFused, true>)
                              : (team.granules == 1   ? norm_forward_rows_kernel<kType, 1, kFused, false>
                                 : team.granules == 2 ? norm_forward_rows_kernel<kType, 2, kFused, false>
                                                      : norm_forward_rows_kernel<kType, 4, kFused, false>);
        kern<<<(unsigned)(want < cap ? want : cap), block, c.hist_bytes, stream>>>(a, team.threads);
    } else {
        const int64_t cap = (int64_t)c.dev.sm_count * 4;
        const auto kern = c.fmt ? norm_forward_loop_kernel<kType, kFused, true> : norm_forward_loop_kernel<kType, kFused, false>;
        kern<<<(unsigned)(a.rows < cap ? a.rows : cap), kLoopThreads, c.hist_bytes, stream>>>(a);
    }
    QFMT_CUDA_TRY(cudaGetLastError());
    return QFMT_OK;
}

template <int kType, bool kFused>
int forward(const Call& c, const void* d_x, const void* d_residual, const float* d_weight, const float* d_bias, void* d_h,
            void* d_y, float* d_mean, float* d_rstd, qfmt_stats_t* d_stats, cudaStream_t stream) {
    using W = typename Word<kType>::type;
    ForwardArgs<kType> a;
    a.x = static_cast<const W*>(d_x);
    a.residual = static_cast<const W*>(d_residual);
    a.weight = d_weight;
    a.bias = d_bias;
    a.h = static_cast<W*>(d_h);
    a.y = static_cast<W*>(d_y);
    a.mean = d_mean;
    a.rstd = d_rstd;
    a.ld_x = c.norm.ld_x;
    a.ld_residual = c.norm.ld_residual;
    a.ld_h = c.norm.ld_h;
    a.ld_y = c.norm.ld_y;
    a.rows = c.norm.rows;
    a.cols = c.norm.cols;
    a.eps = c.norm.eps;
    a.vec = granule_aligned(d_x, a.ld_x, kType) && granule_aligned(d_residual, a.ld_residual, kType) &&
            granule_aligned(d_h, a.ld_h, kType) && granule_aligned(d_y, a.ld_y, kType);
    a.fmt = c.fmt;
    a.drop = c.drop;
    a.quant = c.quant;
    a.stats = d_stats;
    return launch_forward<kType, kFused>(c, a, stream);
}

int forward_entry(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, bool fused, const void* d_x, const void* d_residual,
                  const float* d_weight, const float* d_bias, void* d_h, void* d_y, float* d_mean, float* d_rstd,
                  const qfmt_format_t* fmt, qfmt_stats_t* d_stats, int accumulate, cudaStream_t stream) {
    Call c;
    int rc = prepare_call(norm, drop, fmt, d_stats, accumulate, &c);
    if (rc != QFMT_OK) return rc;
    const int32_t t = c.norm.dtype;
    const bool empty = c.norm.rows == 0 || c.norm.cols == 0;
    if (!empty && (d_x == nullptr || d_y == nullptr)) return QFMT_ERR_BAD_ARG;
    if (!element_aligned(d_x, t) || !element_aligned(d_residual, t) || !element_aligned(d_h, t) || !element_aligned(d_y, t) ||
        !float_aligned(d_weight) || !float_aligned(d_bias) || !float_aligned(d_mean) || !float_aligned(d_rstd))
        return QFMT_ERR_BAD_ARG;
    rc = current_device(&c.dev);
    if (rc != QFMT_OK) return rc;
    if (d_stats != nullptr && accumulate == 0) QFMT_CUDA_TRY(cudaMemsetAsync(d_stats, 0, sizeof(qfmt_stats_t), stream));
    if (empty) return QFMT_OK;
    const auto run = fused ? (t == QFMT_F32 ? forward<QFMT_F32, true> : t == QFMT_F16 ? forward<QFMT_F16, true> : forward<QFMT_BF16, true>)
                           : (t == QFMT_F32 ? forward<QFMT_F32, false> : t == QFMT_F16 ? forward<QFMT_F16, false> : forward<QFMT_BF16, false>);
    return run(c, d_x, d_residual, d_weight, d_bias, d_h, d_y, d_mean, d_rstd, d_stats, stream);
}

template <int kType, bool kFused, bool kFmt>
int launch_backward(const Call& c, const BackwardArgs<kType>& a, float* d_dweight, float* d_dbias, cudaStream_t stream) {
    if (a.partial != nullptr) {  // before the row pass, which may overwrite dy
        const int parts = row_parts(a.rows);
        const dim3 grid((unsigned)((a.cols + 32 * kGranule - 1) / (32 * kGranule)), (unsigned)parts);
        norm_column_sums_kernel<kType><<<grid, 32 * kColumnWarps, 0, stream>>>(a);
        const dim3 join((unsigned)((a.cols + 31) / 32), 2);
        norm_join_parts_kernel<<<join, 32 * kColumnWarps, 0, stream>>>(a.partial, parts, a.cols, d_dweight, d_dbias);
        QFMT_CUDA_TRY(cudaGetLastError());
    }
    if (a.rows != 0 && (a.dx != nullptr || a.dresidual != nullptr)) {
        const int64_t cap = (int64_t)c.dev.sm_count * 4;
        norm_backward_loop_kernel<kType, kFused, kFmt><<<(unsigned)(a.rows < cap ? a.rows : cap), kLoopThreads, c.hist_bytes, stream>>>(a);
        QFMT_CUDA_TRY(cudaGetLastError());
    }
    return QFMT_OK;
}

template <int kType, bool kFused>
int backward(const Call& c, const void* d_dy, const void* d_dh, const void* d_h, int64_t ld_h, const float* d_mean,
             const float* d_rstd, const float* d_weight, void* d_dx, void* d_dresidual, float* d_dweight, float* d_dbias,
             qfmt_stats_t* d_stats, float* partial, cudaStream_t stream) {
    using W = typename Word<kType>::type;
    BackwardArgs<kType> a;
    a.dy = static_cast<const W*>(d_dy);
    a.dh = static_cast<const W*>(d_dh);
    a.h = static_cast<const W*>(d_h);
    a.mean = d_mean;
    a.rstd = d_rstd;
    a.weight = d_weight;
    a.dx = static_cast<W*>(d_dx);
    a.dresidual = static_cast<W*>(d_dresidual);
    a.partial = partial;
    a.ld_dy = c.norm.ld_dy;
    a.ld_dh = c.norm.ld_dh;
    a.ld_h = ld_h;
    a.ld_dx = c.norm.ld_dx;
    a.ld_dresidual = c.norm.ld_dresidual;
    a.rows = c.norm.rows;
    a.cols = c.norm.cols;
    a.vec = granule_aligned(d_dy, a.ld_dy, kType) && granule_aligned(d_dh, a.ld_dh, kType) && granule_aligned(d_h, a.ld_h, kType) &&
            granule_aligned(d_dx, a.ld_dx, kType) && granule_aligned(d_dresidual, a.ld_dresidual, kType);
    a.fmt = c.fmt;
    a.drop = c.drop;
    a.quant = c.quant;
    a.stats = d_stats;
    return c.fmt ? launch_backward<kType, kFused, true>(c, a, d_dweight, d_dbias, stream)
                 : launch_backward<kType, kFused, false>(c, a, d_dweight, d_dbias, stream);
}

int backward_entry(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, bool fused, const void* d_dy, const void* d_dh,
                   const void* d_h, const float* d_mean, const float* d_rstd, const float* d_weight, void* d_dx,
                   void* d_dresidual, float* d_dweight, float* d_dbias, const qfmt_format_t* fmt, qfmt_stats_t* d_stats,
                   int accumulate, void* d_workspace, size_t workspace_bytes, cudaStream_t stream) {
    Call c;
    int rc = prepare_call(norm, drop, fmt, d_stats, accumulate, &c);
    if (rc != QFMT_OK) return rc;
    const int32_t t = c.norm.dtype;
    const bool empty = c.norm.rows == 0 || c.norm.cols == 0;
    const bool columns = (d_dweight != nullptr || d_dbias != nullptr) && c.norm.cols != 0;
    if (!empty && (d_dy == nullptr || d_h == nullptr || d_mean == nullptr || d_rstd == nullptr)) return QFMT_ERR_BAD_ARG;
    if (d_stats != nullptr && d_dx == nullptr && !empty) return QFMT_ERR_BAD_ARG;  // the record is dx's
    if (!element_aligned(d_dy, t) || !element_aligned(d_dh, t) || !element_aligned(d_h, t) || !element_aligned(d_dx, t) ||
        !element_aligned(d_dresidual, t) || !float_aligned(d_mean) || !float_aligned(d_rstd) || !float_aligned(d_weight) ||
        !float_aligned(d_dweight) || !float_aligned(d_dbias))
        return QFMT_ERR_BAD_ARG;
    if (!empty && d_dx != nullptr && d_dx == d_dresidual) return QFMT_ERR_BAD_ARG;
    if (columns && (d_workspace == nullptr || (reinterpret_cast<uintptr_t>(d_workspace) & 15u) ||
                    workspace_bytes < qfmt_layer_norm_workspace_bytes(norm)))
        return QFMT_ERR_BAD_ARG;
    rc = current_device(&c.dev);
    if (rc != QFMT_OK) return rc;
    if (d_stats != nullptr && accumulate == 0) QFMT_CUDA_TRY(cudaMemsetAsync(d_stats, 0, sizeof(qfmt_stats_t), stream));
    if (c.norm.cols == 0 || (empty && !columns)) return QFMT_OK;
    const int64_t ld_h = fused ? c.norm.ld_h : c.norm.ld_x;
    const auto run = fused ? (t == QFMT_F32 ? backward<QFMT_F32, true> : t == QFMT_F16 ? backward<QFMT_F16, true> : backward<QFMT_BF16, true>)
                           : (t == QFMT_F32 ? backward<QFMT_F32, false> : t == QFMT_F16 ? backward<QFMT_F16, false> : backward<QFMT_BF16, false>);
    return run(c, d_dy, d_dh, d_h, ld_h, d_mean, d_rstd, d_weight, d_dx, d_dresidual, d_dweight, d_dbias, d_stats,
               columns ? static_cast<float*>(d_workspace) : nullptr, stream);
}

}  // namespace
}  // namespace qfmt

extern "C" size_t qfmt_layer_norm_workspace_bytes(const qfmt_norm_t* norm) {
    if (norm == nullptr || norm->rows < 0 || norm->cols < 0 || norm->rows > 0x7FFFFFFF || norm->cols > 0x7FFFFFFF) return 0;
    return (size_t)qfmt::row_parts(norm->rows) * 2 * (size_t)norm->cols * sizeof(float);
}

extern "C" int qfmt_layer_norm(const qfmt_norm_t* norm, const void* d_x, const float* d_weight, const float* d_bias, void* d_y,
                               float* d_mean, float* d_rstd, const qfmt_format_t* fmt, qfmt_stats_t* d_stats, int accumulate,
                               void* stream) {
    return qfmt::forward_entry(norm, nullptr, false, d_x, nullptr, d_weight, d_bias, nullptr, d_y, d_mean, d_rstd, fmt, d_stats,
                               accumulate, (cudaStream_t)stream);
}

extern "C" int qfmt_layer_norm_backward(const qfmt_norm_t* norm, const void* d_dy, const void* d_x, const float* d_mean,
                                        const float* d_rstd, const float* d_weight, void* d_dx, float* d_dweight,
                                        float* d_dbias, const qfmt_format_t* fmt, qfmt_stats_t* d_stats, int accumulate,
                                        void* d_workspace, size_t workspace_bytes, void* stream) {
    return qfmt::backward_entry(norm, nullptr, false, d_dy, nullptr, d_x, d_mean, d_rstd, d_weight, d_dx, nullptr, d_dweight,
                                d_dbias, fmt, d_stats, accumulate, d_workspace, workspace_bytes, (cudaStream_t)stream);
}

extern "C" int qfmt_dropout_add_layer_norm(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, const void* d_x,
                                           const void* d_residual, const float* d_weight, const float* d_bias, void* d_h,
                                           void* d_y, float* d_mean, float* d_rstd, const qfmt_format_t* fmt,
                                           qfmt_stats_t* d_stats, int accumulate, void* stream) {
    return qfmt::forward_entry(norm, drop, true, d_x, d_residual, d_weight, d_bias, d_h, d_y, d_mean, d_rstd, fmt, d_stats,
                               accumulate, (cudaStream_t)stream);
}

extern "C" int qfmt_dropout_add_layer_norm_backward(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, const void* d_dy,
                                                    const void* d_dh, const void* d_h, const float* d_mean,
                                                    const float* d_rstd, const float* d_weight, void* d_dx, void* d_dresidual,
                                                    float* d_dweight, float* d_dbias, const qfmt_format_t* fmt,
                                                    qfmt_stats_t* d_stats, int accumulate, void* d_workspace,
                                                    size_t workspace_bytes, void* stream) {
    return qfmt::backward_entry(norm, drop, true, d_dy, d_dh, d_h, d_mean, d_rstd, d_weight, d_dx, d_dresidual, d_dweight, d_dbias,
                                fmt, d_stats, accumulate, d_workspace, workspace_bytes, (cudaStream_t)stream);
}
