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
    Source<kType> x, residual;  // residual.p may be NULL
    Target<kType> out;
    int64_t cols;
    uint32_t granules;  // per row
    uint64_t total;     // rows * granules
    DropParams drop;
};

template <int kType>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs<kType> a) {
    grid_launch_dependents();
    grid_dependency_wait();
    const uint64_t offset = drop_offset(a.drop);
    const int lane = threadIdx.x & 31;
    const uint64_t step = (uint64_t)gridDim.x * kDropThreads;
    for (uint64_t base = (uint64_t)blockIdx.x * kDropThreads; base < a.total; base += step) {  // whole warps
        const uint64_t i = base + threadIdx.x;
        const uint64_t row = i / a.granules;
        const uint32_t g = (uint32_t)(i - row * a.granules);
        const int64_t col = (int64_t)g * kGranule;
        const int n = i < a.total ? (int)(a.cols - col < kGranule ? a.cols - col : kGranule) : 0;
        Granule v = widen_raw<kType>(load_any<kType>(a.x.p + row * a.x.ld + col, n, a.x));
        if (a.drop.active) drop_granule(a.drop, offset, (uint32_t)row, g, v);
        if (a.residual.p != nullptr) {
            const Granule r = widen_raw<kType>(load_any<kType>(a.residual.p + row * a.residual.ld + col, n, a.residual));
#pragma unroll
            for (int j = 0; j < 4; ++j) v.p[j] = add2(r.p[j], v.p[j]);
        }
        store_any<kType>(a.out.p + row * a.out.ld + col, n, a.out, finish<kType>(v), lane != 0 && g != 0, lane != 31 && g + 1 < a.granules);
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
    const uint64_t blocks = (a.total + kDropThreads - 1) / kDropThreads;
    const uint64_t cap = (uint64_t)dev.sm_count * 16;
    QFMT_CUDA_TRY(launch_overlapping(dropout_kernel<kType>, (unsigned)(blocks < cap ? blocks : cap), kDropThreads, 0, stream, a));
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
