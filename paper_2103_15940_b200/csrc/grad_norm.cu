// The global norm of a list of tensors and clipping by it:
//     norm = sqrt(sum (g / scale)^2),  dst = src min(1, max_norm / norm) / scale.
//
// Sums are in 64 bits, and squares too unless eight of codes add up in 32 bits without leaving its range: the square of any 32-bit
// value is exact and finite in 64 bits, so nothing overflows or vanishes and a sum is not finite exactly if an element is not.  Only then
// are elements looked at one by one for the counts.
//
// The list's chunks (at most 8192 elements of one tensor) form one sequence, cut into equal ranges among the blocks; a block finds its
// first tensor by bisection and walks on from there.  Every block leaves one partial sum and one more block adds those up, so the order
// depends on sizes alone.  Clipping walks each range backwards: what the norm read last is what the second-level cache still holds.
// Bound by memory: two reads and one write of every element.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"

namespace qfmt {
namespace {

constexpr int kChunk = 8192, kThreads = 256, kBlocksPerSm = 6;

struct Partial {
    double sum;
    unsigned long long n_nan, n_inf;
};

template <typename T>
__device__ __forceinline__ void unpack16(uint4 w, float* v);  // the 16 / sizeof(T) values of a piece
template <>
__device__ __forceinline__ void unpack16<float>(uint4 w, float* v) {
    v[0] = __uint_as_float(w.x);
    v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z);
    v[3] = __uint_as_float(w.w);
}
template <>
__device__ __forceinline__ void unpack16<__half>(uint4 w, float* v) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
template <>
__device__ __forceinline__ void unpack16<__nv_bfloat16>(uint4 w, float* v) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x[i] << 16);
        v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ float rounded(float v, float) { return v; }
__device__ __forceinline__ __half rounded(float v, __half) { return __float2half_rn(v); }
__device__ __forceinline__ __nv_bfloat16 rounded(float v, __nv_bfloat16) { return __float2bfloat16_rn(v); }

// The last tensor whose first chunk is not behind `chunk` (empty tensors share theirs with the next).  Each step of the search looks at
// 32 places at once, a lane each: a list of a thousand tensors takes two dependent loads, not ten.
__device__ __forceinline__ int tensor_of(const qfmt_tensor_t* tensors, int count, long long chunk) {
    const int lane = threadIdx.x & 31;
    int lo = 0, n = count;  // the answer is in lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) / 32, at = lane * step;
        const bool here = at < n && tensors[lo + at].first_chunk <= chunk;
        const int last = 31 - __clz(__ballot_sync(0xFFFFFFFFu, here) | 1u);
        lo += last * step;
        n = n - last * step < step ? n - last * step : step;
    }
    return lo;
}

template <typename T>
__device__ __forceinline__ void chunk_square(const T* p, int n, Partial& total) {
    constexpr int per = 16 / (int)sizeof(T);
    const int tid = threadIdx.x;
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
    if (head > n) head = n;
    const int pieces = (n - head) / per, tail = head + pieces * per;
    const uint4* body = reinterpret_cast<const uint4*>(p + head);
    double s0 = 0.0, s1 = 0.0;
    if (tid < head) {
        const double x = (double)(float)p[tid];
        s0 = x * x;
    }
    if (tid < n - tail) {
        const double x = (double)(float)p[tail + tid];
        s1 = x * x;
    }
    for (int i0 = tid; i0 < pieces; i0 += 4 * kThreads) {
        uint4 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = i0 + j * kThreads < pieces ? body[i0 + j * kThreads] : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[per];
            unpack16<T>(w[j], v);
            if constexpr (sizeof(T) == 2) {
                // Eight squares in 32 bits (a code's square is exact there, the sum off by 2^-22 at most) where they are in range:
                // conversions to 64 bits take eight times as long as the additions, and one for eight codes keeps up with memory.
                float q0 = __fmul_rn(v[0], v[0]), q1 = __fmul_rn(v[1], v[1]);
#pragma unroll
                for (int k = 2; k < per; k += 2) {
                    q0 = __fmaf_rn(v[k], v[k], q0);
                    q1 = __fmaf_rn(v[k + 1], v[k + 1], q1);
                }
                const float q = __fadd_rn(q0, q1);
                const bool zero = ((w[j].x | w[j].y | w[j].z | w[j].w) & 0x7FFF7FFFu) == 0u;
                if ((q >= 1e-25f && q <= 1e37f) || zero) {
                    s0 += (double)q;
                    continue;
                }
            }
#pragma unroll
            for (int k = 0; k < per; k += 2) {
                const double a = (double)v[k], b = (double)v[k + 1];
                s0 = __fma_rn(a, a, s0);
                s1 = __fma_rn(b, b, s1);
            }
        }
    }
    const double s = s0 + s1;
    if (!isfinite(s)) {
        auto look = [&](float x) {
            if (x != x) total.n_nan += 1;
            else if (isinf(x)) total.n_inf += 1;
        };
        if (tid < head) look((float)p[tid]);
        if (tid < n - tail) look((float)p[tail + tid]);
        for (int i = tid; i < pieces; i += kThreads)
            for (int k = 0; k < per; ++k) look((float)p[head + i * per + k]);
    }
    total.sum += s;
}

__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
norm_kernel(const qfmt_tensor_t* __restrict__ tensors, int count, long long chunks, Partial* __restrict__ partials) {
    __shared__ Partial sums[kThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    long long chunk = chunks * blockIdx.x / gridDim.x;
    const long long end = chunks * (blockIdx.x + 1) / gridDim.x;
    int t = tensor_of(tensors, count, chunk);
    Partial total = {0.0, 0ull, 0ull};
    qfmt_tensor_t r = tensors[t];
    for (; chunk < end; ++chunk) {
        while ((chunk - r.first_chunk) * kChunk >= r.n) r = tensors[++t];
        const long long at = (chunk - r.first_chunk) * kChunk;
        const int n = r.n - at < kChunk ? (int)(r.n - at) : kChunk;
        if (r.dtype == QFMT_F32) chunk_square(static_cast<const float*>(r.src) + at, n, total);
        else if (r.dtype == QFMT_F16) chunk_square(static_cast<const __half*>(r.src) + at, n, total);
        else chunk_square(static_cast<const __nv_bfloat16*>(r.src) + at, n, total);
    }
    for (int o = 16; o > 0; o >>= 1) {
        total.sum += __shfl_xor_sync(0xFFFFFFFFu, total.sum, o);
        total.n_nan += __shfl_xor_sync(0xFFFFFFFFu, total.n_nan, o);
        total.n_inf += __shfl_xor_sync(0xFFFFFFFFu, total.n_inf, o);
    }
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = total;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kThreads / 32; ++w) {
        total.sum += sums[w].sum;
        total.n_nan += sums[w].n_nan;
        total.n_inf += sums[w].n_inf;
    }
    partials[blockIdx.x] = total;
}

__global__ void __launch_bounds__(kThreads)
finish_kernel(const Partial* __restrict__ partials, int n, const qfmt_tensor_t* __restrict__ tensors, int count, float max_norm,
              const qfmt_dls_t* dls, qfmt_grad_norm_t* out, qfmt_stats_t* stats) {
    __shared__ Partial sums[kThreads / 32];
    __shared__ unsigned long long elements[kThreads / 32];
    grid_dependency_wait();
    grid_launch_dependents();
    Partial total = {0.0, 0ull, 0ull};
    unsigned long long all = 0ull;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        total.sum += partials[i].sum;
        total.n_nan += partials[i].n_nan;
        total.n_inf += partials[i].n_inf;
    }
    if (stats != nullptr) {
        for (int i = threadIdx.x; i < count; i += kThreads) all += (unsigned long long)tensors[i].n;
    }
    for (int o = 16; o > 0; o >>= 1) {
        total.sum += __shfl_xor_sync(0xFFFFFFFFu, total.sum, o);
        total.n_nan += __shfl_xor_sync(0xFFFFFFFFu, total.n_nan, o);
        total.n_inf += __shfl_xor_sync(0xFFFFFFFFu, total.n_inf, o);
        all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
    }
    if ((threadIdx.x & 31) == 0) {
        sums[threadIdx.x >> 5] = total;
        elements[threadIdx.x >> 5] = all;
    }
    if (stats != nullptr) {
        unsigned long long* words = reinterpret_cast<unsigned long long*>(stats);
        for (int i = threadIdx.x; i < (int)(sizeof(qfmt_stats_t) / 8); i += kThreads) words[i] = 0ull;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < kThreads / 32; ++w) {
        total.sum += sums[w].sum;
        total.n_nan += sums[w].n_nan;
        total.n_inf += sums[w].n_inf;
        all += elements[w];
    }
    const double scale = dls != nullptr ? (double)dls->scale : 1.0;
    const double norm = sqrt(total.sum) / scale;
    double factor = 1.0;
    if (total.n_nan + total.n_inf == 0ull) factor = (norm > (double)max_norm ? (double)max_norm / norm : 1.0) / scale;
    out->norm = (float)norm;
    out->factor = (float)factor;
    out->n_nonfinite = total.n_nan + total.n_inf;
    if (stats != nullptr) {
        stats->n_total = all;
        stats->n_nan = total.n_nan;
        stats->n_inf_in = total.n_inf;
    }
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* p, T* q, int n, float factor) {
    constexpr int per = 16 / (int)sizeof(T);
    const int tid = threadIdx.x;
    if (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) != 0) {  // not in the same place of a piece
#pragma unroll 4
        for (int i = tid; i < n; i += kThreads) q[i] = rounded(__fmul_rn((float)p[i], factor), T());
        return;
    }
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
    if (head > n) head = n;
    const int pieces = (n - head) / per, tail = head + pieces * per;
    if (tid < head) q[tid] = rounded(__fmul_rn((float)p[tid], factor), T());
    if (tid < n - tail) q[tail + tid] = rounded(__fmul_rn((float)p[tail + tid], factor), T());
    const uint4* from = reinterpret_cast<const uint4*>(p + head);
    uint4* to = reinterpret_cast<uint4*>(q + head);
#pragma unroll 4
    for (int i = tid; i < pieces; i += kThreads) {
        float v[per];
        unpack16<T>(from[i], v);
        uint4 w;
        T* e = reinterpret_cast<T*>(&w);
#pragma unroll
        for (int k = 0; k < per; ++k) e[k] = rounded(__fmul_rn(v[k], factor), T());
        to[i] = w;
    }
}

__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
clip_kernel(const qfmt_tensor_t* tensors, int count, long long chunks, const qfmt_grad_norm_t* norm) {
    grid_dependency_wait();
    grid_launch_dependents();
    const float factor = norm->factor;
    const long long first = chunks * blockIdx.x / gridDim.x;
    long long chunk = chunks * (blockIdx.x + 1) / gridDim.x - 1;
    if (chunk < first) return;
    int t = tensor_of(tensors, count, chunk);
    qfmt_tensor_t r = tensors[t];
    for (; chunk >= first; --chunk) {
        while (r.n == 0 || chunk < r.first_chunk) r = tensors[--t];
        if (r.dst == nullptr || (r.dst == r.src && factor == 1.0f)) continue;
        const long long at = (chunk - r.first_chunk) * kChunk;
        const int n = r.n - at < kChunk ? (int)(r.n - at) : kChunk;
        if (r.dtype == QFMT_F32) chunk_scale(static_cast<const float*>(r.src) + at, static_cast<float*>(r.dst) + at, n, factor);
        else if (r.dtype == QFMT_F16) chunk_scale(static_cast<const __half*>(r.src) + at, static_cast<__half*>(r.dst) + at, n, factor);
        else chunk_scale(static_cast<const __nv_bfloat16*>(r.src) + at, static_cast<__nv_bfloat16*>(r.dst) + at, n, factor);
    }
}

// Blocks of a list: never more than its chunks.
int64_t list_blocks(int64_t chunks, const DeviceInfo& dev) {
    const int64_t most = (int64_t)dev.sm_count * kBlocksPerSm;
    return chunks < most ? chunks : most;
}
constexpr int64_t kMostBlocks = 256 * kBlocksPerSm;  // workspaces are sized without asking a device
constexpr size_t kHeader = 256;                      // the status area, which is another call's if the workspace is shared

bool misaligned(const void* p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }
bool list_ok(const qfmt_tensor_t* d_tensors, int64_t count, int64_t chunks) {
    if (count < 0 || chunks < 0 || count >= (1ll << 31) || (count == 0 && chunks != 0)) return false;
    return (count == 0 || d_tensors != nullptr) && !misaligned(d_tensors, 8);
}

}  // namespace
}  // namespace qfmt

extern "C" int64_t qfmt_plan_tensors(qfmt_tensor_t* h_tensors, int64_t count) {
    if (count < 0 || count >= (1ll << 31) || (count > 0 && h_tensors == nullptr)) return QFMT_ERR_BAD_ARG;
    int64_t chunks = 0;
    for (int64_t i = 0; i < count; ++i) {
        qfmt_tensor_t& r = h_tensors[i];
        if (r.dtype != QFMT_F32 && r.dtype != QFMT_F16 && r.dtype != QFMT_BF16) return QFMT_ERR_BAD_ARG;
        const uintptr_t size = r.dtype == QFMT_F32 ? 4 : 2;
        if (r.n < 0 || r.n > (1ll << 46) || (r.n > 0 && r.src == nullptr)) return QFMT_ERR_BAD_ARG;
        if (qfmt::misaligned(r.src, size) || qfmt::misaligned(r.dst, size)) return QFMT_ERR_BAD_ARG;
        r.first_chunk = chunks;
        chunks += (r.n + qfmt::kChunk - 1) / qfmt::kChunk;
        if (chunks > (1ll << 46)) return QFMT_ERR_BAD_ARG;
    }
    return chunks;
}

extern "C" size_t qfmt_grad_norm_workspace_bytes(int64_t count, int64_t chunks) {
    if (count < 0 || chunks < 0) return 0;
    const int64_t blocks = chunks < qfmt::kMostBlocks ? chunks : qfmt::kMostBlocks;
    return qfmt::kHeader + (size_t)blocks * sizeof(qfmt::Partial);
}

extern "C" int qfmt_grad_norm(const qfmt_tensor_t* d_tensors, int64_t count, int64_t chunks, float max_norm, const qfmt_dls_t* d_dls,
                              qfmt_grad_norm_t* d_norm, qfmt_stats_t* d_stats, void* d_workspace, size_t workspace_bytes, void* stream) {
    using namespace qfmt;
    if (!list_ok(d_tensors, count, chunks) || !(max_norm > 0.0f)) return QFMT_ERR_BAD_ARG;
    if (misaligned(d_dls, 8) || d_norm == nullptr || misaligned(d_norm, 8) || misaligned(d_stats, 8)) return QFMT_ERR_BAD_ARG;
    if (d_workspace == nullptr || misaligned(d_workspace, 16) || workspace_bytes < qfmt_grad_norm_workspace_bytes(count, chunks))
        return QFMT_ERR_BAD_ARG;
    DeviceInfo dev;
    const int rc = current_device(&dev);
    if (rc != QFMT_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    int64_t blocks = list_blocks(chunks, dev);
    if (blocks > kMostBlocks) blocks = kMostBlocks;
    Partial* partials = reinterpret_cast<Partial*>(static_cast<char*>(d_workspace) + kHeader);
    if (blocks > 0)
        QFMT_CUDA_TRY(launch_overlapping(norm_kernel, (unsigned)blocks, (unsigned)kThreads, 0, st, d_tensors, (int)count, (long long)chunks, partials));
    QFMT_CUDA_TRY(launch_overlapping(finish_kernel, 1u, (unsigned)kThreads, 0, st, (const Partial*)partials, (int)blocks, d_tensors, (int)count,
                                     max_norm, d_dls, d_norm, d_stats));
    return QFMT_OK;
}

extern "C" int qfmt_grad_clip(const qfmt_tensor_t* d_tensors, int64_t count, int64_t chunks, const qfmt_grad_norm_t* d_norm, void* stream) {
    using namespace qfmt;
    if (!list_ok(d_tensors, count, chunks) || d_norm == nullptr || misaligned(d_norm, 8)) return QFMT_ERR_BAD_ARG;
    DeviceInfo dev;
    const int rc = current_device(&dev);
    if (rc != QFMT_OK) return rc;
    if (chunks == 0) return QFMT_OK;
    QFMT_CUDA_TRY(launch_overlapping(clip_kernel, (unsigned)list_blocks(chunks, dev), (unsigned)kThreads, 0, static_cast<cudaStream_t>(stream),
                                     d_tensors, (int)count, (long long)chunks, d_norm));
    return QFMT_OK;
}
