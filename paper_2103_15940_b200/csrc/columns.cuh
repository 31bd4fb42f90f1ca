// Sums of a matrix' columns from parts: [parts][pitch] fp32, part by part in a fixed order.
#pragma once

#include "common.cuh"

namespace qfmt {

constexpr int kJoinCols = 32, kJoinGroups = 32;

// Block of 32 columns x 32 groups: group g adds parts g, g + 32, ..., then a warp a column adds the groups (halves onto halves).  `count`
// (or NULL) holds the rows counted on the device: only the parts of whole tiles of tile_rows that hold some of them were written, one for
// 32 rows.  `scale` (or NULL): what the sums are multiplied by.
static __global__ void __launch_bounds__(kJoinCols * kJoinGroups)
join_columns_kernel(const float* __restrict__ parts, int64_t pitch, int n_parts, const int* count, int tile_rows,
                    const float* scale, float* __restrict__ out, int cols) {
    __shared__ float sums[kJoinGroups][kJoinCols + 1];
    grid_dependency_wait();
    grid_launch_dependents();
    if (count != nullptr) n_parts = (*count + tile_rows - 1) / tile_rows * (tile_rows / 32);
    const int c = threadIdx.x % kJoinCols, g = threadIdx.x / kJoinCols, col = blockIdx.x * kJoinCols + c;
    float s = 0.0f;
    if (col < cols) {
#pragma unroll 4
        for (int i = g; i < n_parts; i += kJoinGroups) s = __fadd_rn(s, parts[(int64_t)i * pitch + col]);
    }
    sums[g][c] = s;
    __syncthreads();
    s = sums[c][g];  // now the warp has column g of the block and the lane group c
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(0xFFFFFFFFu, s, o));
    const int mine = blockIdx.x * kJoinCols + g;
    if (c == 0 && mine < cols) out[mine] = scale != nullptr ? __fmul_rn(s, *scale) : s;
}

inline int launch_join_columns(const float* parts, int64_t pitch, int64_t n_parts, const int* count, int tile_rows,
                               const float* scale, float* out, int64_t cols, cudaStream_t stream) {
    QFMT_CUDA_TRY(launch_overlapping(join_columns_kernel, (unsigned)((cols + kJoinCols - 1) / kJoinCols), (unsigned)(kJoinCols * kJoinGroups),
                                     0, stream, parts, pitch, (int)n_parts, count, tile_rows, scale, out, (int)cols));
    return QFMT_OK;
}

}  // namespace qfmt
