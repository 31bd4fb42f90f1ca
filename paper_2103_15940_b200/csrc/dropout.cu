// Dropout from a counter-based generator: out = residual + D(x), with the mask recomputed from (seed, offset,
// row, column) wherever it is needed and never stored.
//
// One read and one write per element (two reads with a residual) and, per granule of eight columns, one
// Philox block: 20 wide products, against 32 bytes of traffic for 16-bit codes.
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "elements.cuh"

namespace qfmt {
namespace {

constexpr int kDropThreads = 256;

template <int kType>
struct DropArgs {
    Source<kType> x, residual;
    Target<kType> out;
    int64_t cols;
    uint32_t granules;    // per row
    uint64_t total;       // rows * granules
    uint32_t step_rows, step_granules;  // the grid's threads as whole rows and granules beyond them
    DropParams drop;
};

// A thread takes granules a grid's width apart, kAhead of them at a time.  kPlain: every granule whole and aligned.
template <int kType, bool kResidual, bool kPlain>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs<kType> a) {
    constexpr int kAhead = !kPlain ? 1 : (kType == QFMT_F32) + kResidual == 2 ? 2 : 4;
    grid_launch_dependents();
    grid_dependency_wait();
    const uint64_t offset = drop_offset(a.drop);
    const int lane = threadIdx.x & 31;
    const uint64_t step = (uint64_t)gridDim.x * kDropThreads;
    uint64_t at = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x;
    uint32_t row = (uint32_t)(at / a.granules), g = (uint32_t)(at - (uint64_t)row * a.granules);
    for (; at - lane < a.total; at += kAhead * step) {  // whole warps
        Raw<kType> x[kAhead], r[kAhead];
        uint32_t rows[kAhead], gs[kAhead];
        int n[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            rows[i] = row;
            gs[i] = g;
            const int64_t col = (int64_t)g * kGranule, left = a.cols - col;
            n[i] = at + i * step < a.total ? (kPlain || left > kGranule ? kGranule : (int)left) : 0;
            const auto* px = a.x.p + row * a.x.ld + col;
            if constexpr (kPlain) x[i] = load_raw<kType>(px, n[i] > 0);
            else x[i] = load_any<kType>(px, n[i], a.x);
            if constexpr (kResidual) {
                const auto* pr = a.residual.p + row * a.residual.ld + col;
                if constexpr (kPlain) r[i] = load_raw<kType>(pr, n[i] > 0);
                else r[i] = load_any<kType>(pr, n[i], a.residual);
            }
            row += a.step_rows;
            g += a.step_granules;
            if (g >= a.granules) {
                g -= a.granules;
                ++row;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (kPlain && n[i] == 0) continue;
            Granule v = widen_raw<kType>(x[i]);
            if (a.drop.active) drop_granule(a.drop, offset, rows[i], gs[i], v);
            if constexpr (kResidual) {
                const Granule u = widen_raw<kType>(r[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) v.p[j] = add2(u.p[j], v.p[j]);
            }
            auto* po = a.out.p + rows[i] * a.out.ld + (int64_t)gs[i] * kGranule;
            if constexpr (kPlain) store_raw<kType>(po, finish<kType>(v));
            else store_any<kType>(po, n[i], a.out, finish<kType>(v), lane != 0 && gs[i] != 0, lane != 31 && gs[i] + 1 < a.granules);
        }
    }
}

template <int kType>
int launch_dropout(const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, void* d_out, int64_t ld_out,
                   int64_t rows, int64_t cols, const DropParams& drop, const DeviceInfo& dev, cudaStream_t stream) {
    DropArgs<kType> a;
    a.x = make_source<kType>(d_x, ld_x, rows, cols);
    a.residual = make_source<kType>(d_residual, ld_residual, rows, cols);
    a.out = make_target<kType>(d_out, ld_out);
    a.cols = cols;
    a.granules = (uint32_t)((cols + kGranule - 1) / kGranule);
    a.total = (uint64_t)rows * a.granules;
    a.drop = drop;
    const uint64_t want = (a.total + kDropThreads - 1) / kDropThreads, cap = (uint64_t)dev.sm_count * 8;
    const unsigned blocks = (unsigned)(want < cap ? want : cap);
    const uint64_t threads = (uint64_t)blocks * kDropThreads;
    a.step_rows = (uint32_t)(threads / a.granules);
    a.step_granules = (uint32_t)(threads % a.granules);
    const bool plain = cols % kGranule == 0 && a.x.whole && a.residual.whole && a.out.whole;
    const auto kern = d_residual != nullptr ? (plain ? dropout_kernel<kType, true, true> : dropout_kernel<kType, true, false>)
                                            : (plain ? dropout_kernel<kType, false, true> : dropout_kernel<kType, false, false>);
    QFMT_CUDA_TRY(launch_overlapping(kern, blocks, kDropThreads, 0, stream, a));
    return QFMT_OK;
}

}  // namespace
}  // namespace qfmt

extern "C" int qfmt_dropout(const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, void* d_out,
                            int64_t ld_out, int64_t rows, int64_t cols, int32_t dtype, const qfmt_dropout_t* drop,
                            void* stream) {
    using namespace qfmt;
    if (drop == nullptr || dtype < QFMT_F32 || dtype > QFMT_BF16) return QFMT_ERR_BAD_ARG;
    DropParams params;
    int rc = make_drop_params(drop, &params);
    if (rc != QFMT_OK) return rc;
    if (rows < 0 || cols < 0 || rows > 0x7FFFFFFF || cols > 0x7FFFFFFF) return QFMT_ERR_BAD_ARG;
    ld_x = ld_x ? ld_x : cols;
    ld_residual = ld_residual ? ld_residual : cols;
    ld_out = ld_out ? ld_out : cols;
    if (ld_x < cols || ld_out < cols || (d_residual != nullptr && ld_residual < cols)) return QFMT_ERR_BAD_ARG;
    if (rows != 0 && cols != 0 && (d_x == nullptr || d_out == nullptr)) return QFMT_ERR_BAD_ARG;
    if (!element_aligned(d_x, dtype) || !element_aligned(d_residual, dtype) || !element_aligned(d_out, dtype)) return QFMT_ERR_BAD_ARG;
    DeviceInfo dev;
    rc = current_device(&dev);
    if (rc != QFMT_OK) return rc;
    if (rows == 0 || cols == 0) return QFMT_OK;
    const auto launch = dtype == QFMT_F32 ? launch_dropout<QFMT_F32> : dtype == QFMT_F16 ? launch_dropout<QFMT_F16> : launch_dropout<QFMT_BF16>;
    return launch(d_x, ld_x, d_residual, ld_residual, d_out, ld_out, rows, cols, params, dev, (cudaStream_t)stream);
}
