// Products of 16-bit codes with few rows, or with little work at all: a weight is used for at most 32 rows at a time, so the product is a
// pass over the weights, bound by memory or by latency, and tiles of 128 x 256 would leave most of the GPU idle.
//
// A warp takes 16 (weights stored by output) or 64 (stored by K) outputs and walks K; the weights go from memory straight into the
// registers that mma.sync reads.  The order of K within an MMA is free as long as both operands agree, so it is chosen such that a lane's
// registers are 16 contiguous bytes:
//   by output  (W [N][K])  m16n8k16, the outputs are M and the rows of A are N: lane (g, t) loads 8 K elements 8 t .. of outputs g and g + 8 and
//              of row g of A, which is two MMAs;
//   by K       (W [K][N])  m16n8k16, the rows of A are M and the outputs are N: lane (g, t) loads outputs 8 g .. + 7 at K = 8 t .. 8 t + 7 and
//              those K of rows g and g + 8 of A, which is two times eight MMAs: element i of the weights goes to the i-th, whose column g
//              is output 8 g + i.
// A (at most 32 rows) is read by every warp from the caches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace qfmt {
namespace skinny {

constexpr int kMostRows = 32;

template <bool kBf16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (kBf16) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    } else {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
}

// The operands: A is rows x K with K contiguous, W as above.  Both start on 16 bytes and have pitches that are multiples of 8.
struct Operands {
    const uint16_t* a;
    const uint16_t* w;
    int64_t lda, ldw;
    int rows, n, k;
};

// Eight codes at p of which `left` are in the row, zeros for the others (what lies behind a row is not its own, and may be no memory).
__device__ __forceinline__ uint4 piece(const uint16_t* p, int left) {
    if (left >= 8) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) w[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Asks the second-level cache for the weights of outputs n0 .. and K elements [k0, k1).  A kernel does this while the one before it in the
// stream may still run, before it waits for it: what is prefetched is not read, and whatever that kernel writes there is seen.
template <bool kByK>
__device__ __forceinline__ void prefetch_weights(const Operands& o, int n0, int k0, int k1, int lane) {
    const int end = k1 < o.k ? k1 : o.k, width = end - k0;
    if (width <= 0) return;
    auto ask = [](const uint16_t* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); };
    if (kByK) {
        for (int r = lane; r < width; r += 32) ask(o.w + (int64_t)(k0 + r) * o.ldw + (n0 < o.n ? n0 : 0));
    } else {
        const int lines = (width + 63) / 64;
        for (int i = lane; i < 16 * lines; i += 32) {
            const int n = n0 + i / lines;
            if (n < o.n) ask(o.w + (int64_t)n * o.ldw + k0 + i % lines * 64);
        }
    }
}

// By output: sums over K elements [k0, k1) (k0 a multiple of 32) for outputs n0 .. n0 + 15.  d[b][0 .. 3]: row 8 b + 2 t (0, 2) and
// + 1 (1, 3) of A, output n0 + g (0, 1) and n0 + g + 8 (2, 3).
// kAhead: 32-element steps whose weights are on their way together.
template <bool kBf16, int kBlocks, int kAhead>
__device__ __forceinline__ void by_output(const Operands& o, int n0, int k0, int k1, int lane, float (&d)[kBlocks][4]) {
    const int g = lane >> 2, t = lane & 3, end = k1 < o.k ? k1 : o.k;
    // outputs and rows beyond the last read the last one's: what comes of them is nobody's
    const uint16_t* w0 = o.w + (int64_t)(n0 + g < o.n ? n0 + g : o.n - 1) * o.ldw + t * 8;
    const uint16_t* w1 = o.w + (int64_t)(n0 + g + 8 < o.n ? n0 + g + 8 : o.n - 1) * o.ldw + t * 8;
    const uint16_t* a[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) a[b] = o.a + (int64_t)(b * 8 + g < o.rows ? b * 8 + g : o.rows - 1) * o.lda + t * 8;
    auto multiply = [&](uint4 x, uint4 y, const uint4 (&r)[kBlocks]) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            mma<kBf16>(d[b], x.x, y.x, x.y, y.y, r[b].x, r[b].y);
            mma<kBf16>(d[b], x.z, y.z, x.w, y.w, r[b].z, r[b].w);
        }
    };
    int k = k0;
    for (; k + 32 * kAhead <= end; k += 32 * kAhead) {
        uint4 x[kAhead], y[kAhead], r[kAhead][kBlocks];
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            x[s] = *reinterpret_cast<const uint4*>(w0 + k + s * 32);
            y[s] = *reinterpret_cast<const uint4*>(w1 + k + s * 32);
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) r[s][b] = *reinterpret_cast<const uint4*>(a[b] + k + s * 32);
        }
#pragma unroll
        for (int s = 0; s < kAhead; ++s) multiply(x[s], y[s], r[s]);
    }
    for (; k < end; k += 32) {
        const int left = end - k - t * 8;
        uint4 r[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) r[b] = piece(a[b] + k, left);
        multiply(piece(w0 + k, left), piece(w1 + k, left), r);
    }
}

// By K: sums over [k0, k1) (k0 a multiple of 32) for outputs n0 .. n0 + 63.  d[b][i][0 .. 3]: row 16 b + g (0, 1) and + 8 (2, 3) of A,
// output n0 + 16 t + i (0, 2) and n0 + 16 t + 8 + i (1, 3).  kAhead: 32-element steps whose weights are on their way together.
template <bool kBf16, int kBlocks, int kAhead>
__device__ __forceinline__ void by_k(const Operands& o, int n0, int k0, int k1, int lane, float (&d)[kBlocks][8][4]) {
    const int g = lane >> 2, t = lane & 3, n = n0 + 8 * g, end = k1 < o.k ? k1 : o.k;
    // rows beyond the last read the last one's: what comes of them is nobody's
    const uint16_t* a[kBlocks][2];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = b * 16 + h * 8 + g;
            a[b][h] = o.a + (int64_t)(row < o.rows ? row : o.rows - 1) * o.lda + t * 8;
        }
    }
    auto multiply = [&](const uint4 (&w)[8], const uint4 (&r)[kBlocks][2]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t p0[4] = {w[4 * s].x, w[4 * s].y, w[4 * s].z, w[4 * s].w}, p1[4] = {w[4 * s + 1].x, w[4 * s + 1].y, w[4 * s + 1].z, w[4 * s + 1].w};
            const uint32_t p2[4] = {w[4 * s + 2].x, w[4 * s + 2].y, w[4 * s + 2].z, w[4 * s + 2].w};
            const uint32_t p3[4] = {w[4 * s + 3].x, w[4 * s + 3].y, w[4 * s + 3].z, w[4 * s + 3].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t pick = i & 1 ? 0x7632u : 0x5410u;
                const uint32_t b0 = __byte_perm(p0[i >> 1], p1[i >> 1], pick), b1 = __byte_perm(p2[i >> 1], p3[i >> 1], pick);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    if (s == 0) mma<kBf16>(d[b][i], r[b][0].x, r[b][1].x, r[b][0].y, r[b][1].y, b0, b1);
                    else mma<kBf16>(d[b][i], r[b][0].z, r[b][1].z, r[b][0].w, r[b][1].w, b0, b1);
                }
            }
        }
    };
    int k = k0;
    {
        // A piece that reaches beyond the outputs lies before the next row, so it is memory unless the row is the last; outputs beyond the last
        // piece read that one.
        const int whole = n0 + 64 <= o.n ? o.k : o.k - 1, limit = end < whole ? end : whole;
        const uint16_t* w0 = o.w + (int64_t)t * 8 * o.ldw + (n < o.n ? n : (o.n - 1) & ~7);
        for (; k + 32 * kAhead <= limit; k += 32 * kAhead) {
            uint4 w[kAhead][8], r[kAhead][kBlocks][2];
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
                const uint16_t* p = w0 + (int64_t)(k + s * 32) * o.ldw;
#pragma unroll
                for (int j = 0; j < 8; ++j, p += o.ldw) w[s][j] = *reinterpret_cast<const uint4*>(p);
            }
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    r[s][b][0] = *reinterpret_cast<const uint4*>(a[b][0] + k + s * 32);
                    r[s][b][1] = *reinterpret_cast<const uint4*>(a[b][1] + k + s * 32);
                }
            }
#pragma unroll
            for (int s = 0; s < kAhead; ++s) multiply(w[s], r[s]);
        }
    }
    for (; k < end; k += 32) {
        const int left = end - k - t * 8;
        uint4 w[8], r[kBlocks][2];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[j] = j < left && n < o.n ? piece(o.w + (int64_t)(k + t * 8 + j) * o.ldw + n, o.n - n) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            r[b][0] = piece(a[b][0] + k, left);
            r[b][1] = piece(a[b][1] + k, left);
        }
        multiply(w, r);
    }
}

}  // namespace skinny
}  // namespace qfmt
