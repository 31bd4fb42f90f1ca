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
    uint32_t rows, granules;  // per row
    uint32_t step;            // rows from a thread's granule to its next one
    uint32_t turns;           // granules of a thread down the rows
    int64_t step_x, step_residual, step_out;  // the same step in elements
    DropParams drop;
};

// A thread keeps its granule of columns and walks down the rows, so that the first round of the generator and half of
// the second are the same all the way; kAhead granules are loaded at a time.  kPlain: every granule whole and aligned.
template <int kType, bool kResidual, bool kPlain>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs<kType> a) {
    constexpr int kAhead = !kPlain || (kType == QFMT_F32 && kResidual) ? 2 : 4;
    grid_launch_dependents();
    grid_dependency_wait();
    const uint64_t offset = drop_offset(a.drop);
    const uint32_t threads = gridDim.x * kDropThreads, id = blockIdx.x * kDropThreads + threadIdx.x;
    const int lane = threadIdx.x & 31;
    const uint32_t row0 = id / a.granules, g0 = id - row0 * a.granules;
    for (uint32_t g = g0; g - g0 < a.granules; g += threads) {  // once, unless a row is longer than the grid
        const int64_t col = (int64_t)g * kGranule, left = a.cols - col;
        const int columns = row0 >= a.step || left <= 0 ? 0 : kPlain || left > kGranule ? kGranule : (int)left;
        const auto* px = a.x.p + row0 * a.x.ld + col;
        const auto* pr = a.residual.p + row0 * a.residual.ld + col;
        auto* po = a.out.p + row0 * a.out.ld + col;
        uint32_t row = row0;
        for (uint32_t turn = 0; turn < a.turns; turn += kAhead) {  // whole warps
            Raw<kType> x[kAhead], r[kAhead];
            int n[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                n[i] = row + i * a.step < a.rows ? columns : 0;
                if constexpr (kPlain) x[i] = load_raw<kType>(px, n[i] > 0);
                else x[i] = load_any<kType>(px, n[i], a.x);
                px += a.step_x;
                if constexpr (kResidual) {
                    if constexpr (kPlain) r[i] = load_raw<kType>(pr, n[i] > 0);
                    else r[i] = load_any<kType>(pr, n[i], a.residual);
                    pr += a.step_residual;
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                Granule v = widen_raw<kType>(x[i]);
                if (a.drop.active) drop_granule(a.drop, offset, row, g, v);
                if constexpr (kResidual) {
                    const Granule u = widen_raw<kType>(r[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v.p[j] = add2(u.p[j], v.p[j]);
                }
                if constexpr (!kPlain) store_any<kType>(po, n[i], a.out, finish<kType>(v), lane != 0 && g != 0, lane != 31 && g + 1 < a.granules);
                else if (n[i] > 0) store_raw<kType>(po, finish<kType>(v));
                po += a.step_out;
                row += a.step;
            }
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
    a.rows = (uint32_t)rows;
    a.granules = (uint32_t)((cols + kGranule - 1) / kGranule);
    a.drop = drop;
    const bool plain = cols % kGranule == 0 && a.x.whole && a.residual.whole && a.out.whole;
    const int variant = 2 * (d_residual != nullptr) + plain;
    const auto kern = variant == 3   ? dropout_kernel<kType, true, true>
                      : variant == 2 ? dropout_kernel<kType, true, false>
                      : variant == 1 ? dropout_kernel<kType, false, true>
                                     : dropout_kernel<kType, false, false>;
    static std::atomic<int> known[4][kDropThreads / 32 + 1];
    int resident = 0;
    const int rc = resident_blocks(kern, kDropThreads, 0, known[variant], &resident);
    if (rc != QFMT_OK) return rc;
    const uint64_t want = ((uint64_t)rows * a.granules + kDropThreads - 1) / kDropThreads, cap = (uint64_t)dev.sm_count * resident;
    const unsigned blocks = (unsigned)(want < cap ? want : cap);
    const uint32_t step = blocks * kDropThreads / a.granules;
    a.step = step > 0 ? step : 1;
    a.turns = (a.rows + a.step - 1) / a.step;
    a.step_x = a.step * ld_x;
    a.step_residual = a.step * ld_residual;
    a.step_out = a.step * ld_out;
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
