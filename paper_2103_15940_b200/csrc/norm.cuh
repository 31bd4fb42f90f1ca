// What the forward and the backward pass of layer normalisation (and of its fused form y = LN(residual + D(x))) share.
//
//   mean = sum_c h / n        rstd = 1 / sqrt(sum_c (h - mean)^2 / n + eps)
//   y    = (h - mean) rstd w + b
//   xhat = (h - mean) rstd,  g = w dy
//   dh   = rstd (g - sum_c g / n - xhat sum_c (g xhat) / n)        dw = sum_r dy xhat        db = sum_r dy
//
// Everything is held in 32 bits between the loads and the one rounding of each stored value; the forward pass
// normalises the 32-bit sum, not the stored h.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <initializer_list>

#include "common.cuh"
#include "elements.cuh"

namespace qfmt {
namespace {

// Columns of granule g that exist, 0..8.
__device__ __forceinline__ int granule_columns(int64_t cols, int64_t g) {
    const int64_t left = cols - g * kGranule;
    return left >= kGranule ? kGranule : left > 0 ? (int)left : 0;
}

// Zeros from column n of a granule on.
__device__ __forceinline__ void clear_from(Granule& v, int n) {
#pragma unroll
    for (int j = 0; j < kGranule; ++j)
        if (j >= n) v.at(j) = 0.0f;
}

// `n` entries of granule g of a vector of one value per column, or `fill` where there is none.
__device__ __forceinline__ Granule load_columns(const float* p, int64_t g, int n, float fill) {
    Granule v = splat(fill);
    if (p == nullptr) return v;
    p += g * kGranule;
    if (n == kGranule && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
        const float4 lo = reinterpret_cast<const float4*>(p)[0], hi = reinterpret_cast<const float4*>(p)[1];
        v.p[0] = make_float2(lo.x, lo.y), v.p[1] = make_float2(lo.z, lo.w);
        v.p[2] = make_float2(hi.x, hi.y), v.p[3] = make_float2(hi.z, hi.w);
    } else {
#pragma unroll
        for (int j = 0; j < kGranule; ++j)
            if (j < n) v.at(j) = p[j];
    }
    return v;
}

// Column i of dweight and dbias laid side by side, each padded to whole granules.  In 64 bits: i runs to twice the
// padded columns, and a row may have 2^31 - 1.
struct JoinedColumn {
    bool second;  // of dbias
    int64_t c;    // may lie in the padding
};
__host__ __device__ __forceinline__ JoinedColumn joined_column(int64_t i, int64_t padded) { return {i >= padded, i >= padded ? i - padded : i}; }

template <int kType, bool kPlain, int kLanes = kHistLanes, typename Args>
__device__ __forceinline__ Raw<kType> finish_output(const Args& a, const Granule& v, int n, uint32_t* hist) {
    return !kPlain && a.fmt ? finish_format<kType, kLanes>(v, n, a.quant, hist) : finish<kType>(v);
}

constexpr int kLoopThreads = 512;

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

// Teams: the threads that share a row.  Up to 32 of them are an aligned part of a warp, more are whole warps.  Granule
// k * team + t of the row is thread t's k-th, k < V.
constexpr int kMaxTeam = 512;

__device__ __forceinline__ float across(float s, int off) { return s + __shfl_xor_sync(0xFFFFFFFFu, s, off); }

// What the warps of a team left in scratch, 16 entries for each of kValues values, those past the team's warps zero.
// Up to four warps every thread adds the entries up; more would be 15 additions a value in every thread, so the lanes
// of each warp share them (always in the order of the shuffles, whatever kValues is).
template <int kValues>
__device__ __forceinline__ void sum_entries(const float* scratch, int team, float (&s)[kValues]) {
    if (team <= 128) {
#pragma unroll
        for (int i = 0; i < kValues; ++i) {
            const float4 q = *reinterpret_cast<const float4*>(scratch + 16 * i);
            s[i] = (q.x + q.y) + (q.z + q.w);
        }
        return;
    }
    const int lane = threadIdx.x & 31;
    constexpr int kLanes = kValues == 4 ? 8 : 16;  // that share a value
    const int value = lane / kLanes % kValues;
    float u = scratch[16 * value + lane % kLanes];
    if (kLanes == 8) u += scratch[16 * value + 8 + lane % 8];
    else u = across(u, 8);
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) u = across(u, off);
    if constexpr (kValues == 1) {
        s[0] = u;
    } else {
#pragma unroll
        for (int i = 0; i < kValues; ++i) s[i] = __shfl_sync(0xFFFFFFFFu, u, i * kLanes);
    }
}

// How a pass runs: the threads that share a row and the granules each of them holds.  The fewest granules a thread
// with which a team of at most 512 covers the row, but in the forward pass two rather than one beyond a warp (fewer
// shuffles and barriers per element; the backward pass has no registers for that beside the column sums of its rows).
struct Plan {
    int team, granules;  // team 0: the row does not fit a team
};
inline Plan make_plan(int64_t cols, int least, int most) {
    const int64_t g = (cols + kGranule - 1) / kGranule;
    if (g <= 32) {
        int team = 1;
        while (team < g) team *= 2;
        return {team, 1};
    }
    for (int v = least; v <= most; ++v)
        if (g <= (int64_t)v * kMaxTeam) return {(int)((g + 32 * v - 1) / (32 * v)) * 32, v};
    return {0, 0};
}

struct Call {  // what every entry point checks and works out once
    qfmt_norm_t norm;
    DropParams drop;
    QuantParams quant;
    DeviceInfo dev;
    size_t hist_bytes;
    bool fmt;
};

inline int prepare_call(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, const qfmt_format_t* fmt, const qfmt_stats_t* d_stats,
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
        if (d_stats != nullptr) c->hist_bytes = (size_t)(c->quant.top + kExtraBins) * kHistLanes * sizeof(uint32_t);
    } else if (d_stats != nullptr) {
        return QFMT_ERR_BAD_ARG;  // bins are those of a format
    }
    if (reinterpret_cast<uintptr_t>(d_stats) & 7u) return QFMT_ERR_BAD_ARG;
    return QFMT_OK;
}

inline bool float_aligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Whether every granule of every tensor is whole and aligned.
inline bool plain_layout(int64_t cols, std::initializer_list<bool> whole) {
    return cols % kGranule == 0 && std::all_of(whole.begin(), whole.end(), [](bool w) { return w; });
}

constexpr size_t kMostShared = 216 * 1024;  // dynamic, beside the kernels' own few KiB

// Raises a kernel's limit of dynamic shared memory, once on every GPU.
template <typename K>
int allow_shared(K kernel, size_t bytes, const DeviceInfo& dev, std::atomic<bool>* allowed) {
    const bool known = dev.ordinal >= 0 && dev.ordinal < 64;
    if (known && allowed[dev.ordinal].load()) return QFMT_OK;
    QFMT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (known) allowed[dev.ordinal].store(true);
    return QFMT_OK;
}

}  // namespace
}  // namespace qfmt
