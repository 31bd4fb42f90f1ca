// What the tensor-core kernels share: shared-memory matrix descriptors, the status area of a launch and the tensor maps of
// 16-bit operands.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "common.cuh"

namespace qfmt {

// Shared-memory matrix descriptor.  Addresses and offsets are stored in 16-byte units.
//   K-major tile (layout 2, 128-byte swizzle of 16-byte chunks): rows of 128 bytes (32 K
//       elements), 8-row groups 1024 bytes apart (stride offset); leading offset unused.
//   MN-major tile (layout 1, 128-byte swizzle of 32-byte chunks: the one layout 32-bit
//       operands may use when M/N is the contiguous dimension): blocks of [32 K-rows][128
//       bytes = 32 M/N elements]; leading offset = distance between blocks, stride offset =
//       distance between groups of 4 K-rows (512 bytes).
constexpr uint32_t kLayoutSw128 = 2, kLayoutSw128Base32 = 1;
// Field positions: start address bits 0-13, leading offset bits 16-29, stride offset bits 32-45,
// descriptor version (1 on sm_100) bits 46-47, layout bits 61-63.  The descriptor is kept as a
// constant high word and a low word to which the tile's offset (in 16-byte units) is added, so
// that the MMA thread spends one add per operand per MMA.
__device__ __forceinline__ uint32_t desc_hi(uint32_t sbo_bytes, uint32_t layout) {
    return ((sbo_bytes >> 4) & 0x3FFFu) | (1u << 14) | (layout << 29);
}
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo_bytes) {
    return ((saddr & 0x3FFFFu) >> 4) | (((lbo_bytes >> 4) & 0x3FFFu) << 16);
}
__device__ __forceinline__ uint64_t desc_join(uint32_t hi, uint32_t lo) {
    return ((uint64_t)hi << 32) | lo;
}

// Status area at the head of a workspace: two 64-bit words.  Word 1 receives the launch's tag, word 0 an error as (tag << 16) |
// code, which counts only under that launch's tag.
// What a role does when one of its bounded waits runs out: the CTA-wide flag tells the other roles
// to stop at their next check, the status area (first error of the launch wins) tells the host.
__device__ __forceinline__ void raise_timeout(unsigned long long* status, unsigned long long tag, volatile int* abort_flag) {
    *abort_flag = 1;
    const unsigned long long seen = *reinterpret_cast<volatile unsigned long long*>(status);
    if ((seen >> 16) != tag)  // no error of this launch yet; if another role gets in first, its error stands
        atomicCAS(status, seen, (tag << 16) | (unsigned long long)(-(int)QFMT_ERR_TIMEOUT));
}
// The first thread of the grid names the launch in the status area.
__device__ __forceinline__ void announce_launch(unsigned long long* status, unsigned long long tag) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<volatile unsigned long long*>(status + 1) = tag;
}

// ---- host side

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    if (fn == nullptr) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(sym);
    }
    return fn;
}

// Map over packed 16-bit codes (plain 128-byte swizzle): rank 2 or 3, strides in elements.
inline int make_map16(CUtensorMap* map, const uint16_t* base, int rank, const uint64_t* dims, const uint64_t* strides_elems,
               const uint32_t* box) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (fn == nullptr) { set_last_cuda_error((int)cudaErrorSymbolNotFound); return QFMT_ERR_CUDA; }
    cuuint64_t d[3], st[2];
    cuuint32_t bx[3], estr[3] = {1, 1, 1};
    for (int i = 0; i < rank; ++i) { d[i] = dims[i]; bx[i] = box[i]; }
    for (int i = 0; i + 1 < rank; ++i) st[i] = strides_elems[i] * sizeof(uint16_t);
    CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, (cuuint32_t)rank, const_cast<uint16_t*>(base), d, st, bx, estr,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) { set_last_cuda_error(100000 + (int)r); return QFMT_ERR_CUDA; }
    return QFMT_OK;
}
// One operand of the packed contraction.  `extent` is its M (or N) size and `tile` the rows of it a
// CTA stages (128).  K-major: {K, extent} with 64 x tile boxes.  MN-major: 64-wide column blocks of
// 64 K rows; {64, K, extent / 64} with one box per stage when the extent is a multiple of 64
// (*blocked = 1), else the plain {extent, K} map, one 64 x 64 box per block, zero-filled past the end.
inline int make_operand_map16(CUtensorMap* map, const uint16_t* base, bool mn_major, uint64_t extent, uint64_t k, uint64_t ld,
                       uint32_t tile, int* blocked) {
    *blocked = 0;
    if (!mn_major) {
        const uint64_t dims[2] = {k, extent}, strides[1] = {ld};
        const uint32_t box[2] = {64, tile};
        return make_map16(map, base, 2, dims, strides, box);
    }
    if (extent % 64 == 0) {
        *blocked = 1;
        const uint64_t dims[3] = {64, k, extent / 64}, strides[2] = {ld, 64};
        const uint32_t box[3] = {64, 64, tile / 64};
        return make_map16(map, base, 3, dims, strides, box);
    }
    const uint64_t dims[2] = {extent, k}, strides[1] = {ld};
    const uint32_t box[2] = {64, 64};
    return make_map16(map, base, 2, dims, strides, box);
}

}  // namespace qfmt
