// Dropout from a counter-based generator: out = residual + D(x), with the mask recomputed from (seed, offset,
// row, column) wherever it is needed and never stored.
//
// One read and one write per element (two reads with a residual): bound by memory, with the integer pipe not far
// behind.  A granule of eight columns costs one generator block of 20 wide products and 20 three-way xors; with the
// rest a warp issues 93 instructions for 32 granules of codes (137 before a thread kept its columns and the round keys
// came as constants, 28 us against 24 on 8192 x 4096 bfloat16).  Sixteen bits an element, not 32, because two blocks a
// granule would make the integer pipe the bound; so p is held in steps of 2^-16 and the scale belongs to the step taken.
// Measured: 8192 x 4096 bfloat16 24.0 us (5.6 TB/s, 0.87 of the measured copy rate), 16384 x 4096 fp32 92 us (5.8 TB/s),
// 16 Mi elements in one row of bfloat16 13.5 us, 4099 x 1021 fp32 with a residual into dense rows 10.7 us (4.7 TB/s); all on sets
// of tensors larger than L2 in turn.
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
    uint32_t inner;           // inner_rows()
    uint32_t turns;           // granules that a thread takes one after the other ...
    uint32_t step;            // ... this many rows apart, or in rows longer than the grid this many granules
    int64_t step_x, step_residual, step_out;  // the same step in elements
    DropParams drop;
};

// kDown: a thread keeps its granule of columns and walks down the rows, so that the first round of the generator and
// half of the second are the same all the way.  Otherwise (rows longer than the grid, a flat tensor) it walks along
// one row after the other.  kAhead granules are loaded at a time.  kPlain: every granule whole and aligned.
template <int kType, bool kResidual, bool kDown, bool kPlain>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs<kType> a) {
    constexpr int kAhead = !kPlain ? 1 : kType == QFMT_F32 && kResidual ? 2 : 4;
    grid_launch_dependents();
    grid_dependency_wait();
    const uint64_t offset = drop_offset(a.drop);
    const uint32_t id = blockIdx.x * kDropThreads + threadIdx.x;
    const int lane = threadIdx.x & 31;
    uint32_t row = kDown ? id / a.granules : 0u;
    const uint32_t g0 = id - row * a.granules;
    const bool mine = !kDown || row < a.step;
    for (uint32_t first = 0; first < (kDown ? 1u : a.rows); ++first, row = first) {
        uint32_t g = g0;
        const auto* px = a.x.p + row * a.x.ld + (int64_t)g * kGranule;
        const auto* pr = a.residual.p + row * a.residual.ld + (int64_t)g * kGranule;
        auto* po = a.out.p + row * a.out.ld + (int64_t)g * kGranule;
        for (uint32_t turn = 0; turn < a.turns; turn += kAhead) {  // whole warps
            OnItsWay<kType, kPlain> x[kAhead], r[kAhead];
            int n[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const uint32_t at_row = kDown ? row + i * a.step : row, at_g = kDown ? g : g + i * a.step;
                const int64_t left = a.cols - (int64_t)at_g * kGranule;
                n[i] = !mine || at_row >= a.rows || left <= 0 ? 0 : kPlain || left > kGranule ? kGranule : (int)left;
                const bool edge = at_edge(a.cols, at_g);
                x[i] = start<kType, kPlain>(px + i * a.step_x, n[i], at_row, a.rows, edge, a.inner);
                if (kResidual) r[i] = start<kType, kPlain>(pr + i * a.step_residual, n[i], at_row, a.rows, edge, a.inner);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                Granule v = widen_raw<kType>(words<kType, kPlain>(x[i], px, n[i]));
                if (a.drop.active) drop_granule(a.drop, offset, row, g, v);
                if constexpr (kResidual) {
                    const Granule u = widen_raw<kType>(words<kType, kPlain>(r[i], pr, n[i]));
#pragma unroll
                    for (int j = 0; j < 4; ++j) v.p[j] = add2(u.p[j], v.p[j]);
                }
                put<kType, kPlain>(po, n[i], a.out, finish<kType>(v), lane != 0 && g != 0, lane != 31 && g + 1 < a.granules);
                px += a.step_x;
                pr += a.step_residual;
                po += a.step_out;
                if (kDown) row += a.step;
                else g += a.step;
            }
        }
    }
}

template <int kType>
int launch_dropout(const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, void* d_out, int64_t ld_out,
                   int64_t rows, int64_t cols, const DropParams& drop, const DeviceInfo& dev, cudaStream_t stream) {
    DropArgs<kType> a;
    a.x = make_source<kType>(d_x, ld_x);
    a.residual = make_source<kType>(d_residual, ld_residual);
    a.out = make_target<kType>(d_out, ld_out);
    a.cols = cols;
    a.rows = (uint32_t)rows;
    a.inner = inner_rows(cols, rows);
    a.granules = (uint32_t)((cols + kGranule - 1) / kGranule);
    a.drop = drop;
    const bool plain = cols % kGranule == 0 && a.x.whole && a.residual.whole && a.out.whole;
    const bool down = a.granules <= (uint32_t)dev.sm_count * kDropThreads;  // a row is no longer than the smallest grid
    const int variant = 4 * (d_residual != nullptr) + 2 * down + plain;
    void (*const kernels[8])(DropArgs<kType>) = {
        dropout_kernel<kType, false, false, false>, dropout_kernel<kType, false, false, true>,
        dropout_kernel<kType, false, true, false>,  dropout_kernel<kType, false, true, true>,
        dropout_kernel<kType, true, false, false>,  dropout_kernel<kType, true, false, true>,
        dropout_kernel<kType, true, true, false>,   dropout_kernel<kType, true, true, true>};
    static std::atomic<uint64_t> known[8][kDropThreads / 32 + 1];
    int resident = 0;
    const int rc = resident_blocks(kernels[variant], kDropThreads, 0, known[variant], &resident);
    if (rc != QFMT_OK) return rc;
    const uint64_t want = ((uint64_t)rows * a.granules + kDropThreads - 1) / kDropThreads, cap = (uint64_t)dev.sm_count * resident;
    const unsigned blocks = (unsigned)(want < cap ? want : cap);
    const uint32_t threads = blocks * kDropThreads;
    a.step = down ? threads / a.granules : threads;
    a.turns = down ? (a.rows + a.step - 1) / a.step : (a.granules + threads - 1) / threads;
    a.step_x = (int64_t)a.step * (down ? ld_x : kGranule);
    a.step_residual = (int64_t)a.step * (down ? ld_residual : kGranule);
    a.step_out = (int64_t)a.step * (down ? ld_out : kGranule);
    QFMT_CUDA_TRY(launch_overlapping(kernels[variant], blocks, kDropThreads, 0, stream, a));
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
