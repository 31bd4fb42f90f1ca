// Typed access to rows of fp32 containers, binary16 codes and bfloat16 codes in granules of eight
// columns, the dropout mask, and the rounding of finished values, shared by the passes that work on
// whole layer outputs (dropout, layer normalisation).
//
// A granule is the unit everything here is laid out by: eight 16-bit codes are one 128-bit access, eight
// containers one 256-bit access, and eight columns take the 128 random bits of one Philox block, so a
// thread that owns a granule never shares a block of random bits with another one.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "qfmt.h"
#include "round.cuh"

namespace qfmt {
namespace {

constexpr int kGranule = 8;

template <int kType>
struct Word {
    using type = uint16_t;
};
template <>
struct Word<QFMT_F32> {
    using type = uint32_t;
};

template <int kType>
__device__ __forceinline__ float widen(typename Word<kType>::type w) {
    if constexpr (kType == QFMT_F32) {
        return __uint_as_float(w);
    } else if constexpr (kType == QFMT_BF16) {
        return __uint_as_float((uint32_t)w << 16);
    } else {
        float f;
        asm("cvt.f32.f16 %0, %1;" : "=f"(f) : "h"(w));
        return f;
    }
}

// The words of a granule as they lie in memory: eight for containers, four for codes.
template <int kType>
struct Raw {
    uint32_t w[kType == QFMT_F32 ? 8 : 4];
};

// A whole granule where it is there (n > 0) and its row is one (row < rows), zeros elsewhere.  A predicate on the load,
// not a branch around it.
template <int kType>
__device__ __forceinline__ Raw<kType> load_raw(const typename Word<kType>::type* p, int n, uint32_t row, uint32_t rows) {
    Raw<kType> r;
#pragma unroll
    for (uint32_t& w : r.w) w = 0u;
    if constexpr (kType == QFMT_F32) {
        asm volatile("{ .reg .pred q, s; setp.lt.u32 s, %10, %11; setp.ne.and.s32 q, %9, 0, s;"
                     " @q ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8]; }"
                     : "+r"(r.w[0]), "+r"(r.w[1]), "+r"(r.w[2]), "+r"(r.w[3]), "+r"(r.w[4]), "+r"(r.w[5]), "+r"(r.w[6]),
                       "+r"(r.w[7])
                     : "l"(p), "r"(n), "r"(row), "r"(rows));
    } else {
        asm volatile("{ .reg .pred q, s; setp.lt.u32 s, %6, %7; setp.ne.and.s32 q, %5, 0, s;"
                     " @q ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4]; }"
                     : "+r"(r.w[0]), "+r"(r.w[1]), "+r"(r.w[2]), "+r"(r.w[3]) : "l"(p), "r"(n), "r"(row), "r"(rows));
    }
    return r;
}

template <int kType>
__device__ __forceinline__ void store_raw(typename Word<kType>::type* p, const Raw<kType>& r) {
    if constexpr (kType == QFMT_F32) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     :: "l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]),
                     "r"(r.w[7]) : "memory");
    } else {
        asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};"
                     :: "l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]) : "memory");
    }
}

// The eight columns of a granule as four pairs: additions and products on pairs issue as one instruction each
// (two IEEE results), which halves what the passes issue per element.
struct Granule {
    float2 p[4];
    __device__ __forceinline__ float& at(int j) { return j & 1 ? p[j / 2].y : p[j / 2].x; }
    __device__ __forceinline__ float at(int j) const { return j & 1 ? p[j / 2].y : p[j / 2].x; }
};

__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{ .reg .b64 a, b, r; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; add.rn.f32x2 r, a, b; mov.b64 {%0, %1}, r; }"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{ .reg .b64 a, b, r; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mul.rn.f32x2 r, a, b; mov.b64 {%0, %1}, r; }"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{ .reg .b64 a, b, c, r; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mov.b64 c, {%6, %7}; fma.rn.f32x2 r, a, b, c;"
        " mov.b64 {%0, %1}, r; }"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

__device__ __forceinline__ Granule splat(float v) {
    Granule g;
#pragma unroll
    for (int j = 0; j < 4; ++j) g.p[j] = both(v);
    return g;
}

template <int kType>
__device__ __forceinline__ Granule widen_raw(const Raw<kType>& r) {
    Granule g;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (kType == QFMT_F32) {
            g.p[j] = make_float2(__uint_as_float(r.w[2 * j]), __uint_as_float(r.w[2 * j + 1]));
        } else if constexpr (kType == QFMT_BF16) {
            g.p[j] = make_float2(__uint_as_float(r.w[j] << 16), __uint_as_float(r.w[j] & 0xFFFF0000u));
        } else {
            asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi; }"
                : "=f"(g.p[j].x), "=f"(g.p[j].y) : "r"(r.w[j]));
        }
    }
    return g;
}

// A matrix that is read or written in granules.  whole: every row starts on a granule boundary of memory.
template <int kType>
struct Source {
    const typename Word<kType>::type* p;
    int64_t ld;
    bool whole;
};
template <int kType>
struct Target {
    typename Word<kType>::type* p;
    int64_t ld;
    bool whole;
};

template <int kType>
__device__ __forceinline__ uint32_t word_of(const Raw<kType>& r, int j) {
    if constexpr (kType == QFMT_F32) return r.w[j];
    else return j & 1 ? r.w[j / 2] >> 16 : r.w[j / 2] & 0xFFFFu;
}

// A granule's words from element `first` of w on; the elements are 32 or 16 bits wide.  `first` is the same in all of a
// row, so this branches on it: a selection per word and stage would keep the integer pipe four times as busy.
template <int kType, int kWord, int kFrom>
__device__ __forceinline__ void take_from(Raw<kType>& r, const uint32_t (&w)[kFrom], uint32_t odd) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.w) / 4); ++i) {
        if (kType == QFMT_F32) r.w[i] = w[kWord + i];
        else asm volatile("shf.r.wrap.b32 %0, %1, %2, %3;" : "=r"(r.w[i]) : "r"(w[kWord + i]), "r"(w[(kWord + i + 1) % kFrom]), "r"(odd));
    }
}
template <int kType, int kFrom>
__device__ __forceinline__ Raw<kType> shifted(const uint32_t (&w)[kFrom], uint32_t first) {
    Raw<kType> r;
    const uint32_t odd = kType == QFMT_F32 ? 0u : (first & 1u) * 16u;
    switch (kType == QFMT_F32 ? first : first >> 1) {
        case 0: take_from<kType, 0>(r, w, odd); break;
        case 1: take_from<kType, 1>(r, w, odd); break;
        case 2: take_from<kType, 2>(r, w, odd); break;
        default: take_from<kType, 3>(r, w, odd); break;
    }
    return r;
}

// Four words of w from word `first` (0..3) on.
struct Four {
    uint32_t w[4];
};
__device__ __forceinline__ Four shifted_words(const uint32_t (&v)[8], int first) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = v[i];
#pragma unroll
    for (int by = 2; by > 0; by /= 2) {
#pragma unroll
        for (int i = 0; i + by < 8; ++i) w[i] = first & by ? w[i + by] : w[i];
    }
    return {{w[0], w[1], w[2], w[3]}};
}

// A granule of any alignment on its way: the aligned 16-byte pieces that hold it.
template <int kType>
struct Pieces {
    uint32_t w[kType == QFMT_F32 ? 12 : 8];
    bool inside;  // they lie in the matrix
};

// The pieces of a granule hold up to 7 elements on either side of it, so they can reach beyond the matrix where it lies at an
// edge of its row (at_edge) in the first or last row, or, where rows may lie closer together than that, in any row.  Rows 1 ..
// inner_rows() are those whose pieces cannot.
__host__ __device__ __forceinline__ bool at_edge(int64_t cols, int64_t g) { return g == 0 || (g + 2) * kGranule > cols + 1; }
__host__ __device__ __forceinline__ uint32_t inner_rows(int64_t cols, int64_t rows) { return cols < kGranule || rows < 3 ? 0u : (uint32_t)rows - 2u; }
__host__ __device__ __forceinline__ bool pieces_inside(bool edge, uint32_t row, uint32_t inner) { return !edge || row - 1u < inner; }

// Starts to load `n` columns (0..8) of a granule at p: loads under a predicate, nothing waits and nothing branches.
// What the pieces hold beyond the columns is thrown away later; where they could reach beyond the matrix (`inside`
// false) the granule is left to arrive().
template <int kType>
__device__ __forceinline__ Pieces<kType> start_any(const typename Word<kType>::type* p, int n, bool inside) {
    constexpr int kPer = kType == QFMT_F32 ? 4 : 8;
    Pieces<kType> r;
    const int first = (int)(reinterpret_cast<uintptr_t>(p) & 15u) / (16 / kPer);
    const auto* base = p - first;
    const int reach = inside && n > 0 ? first + n : 0;
    r.inside = inside;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.w) / 16); ++i)
        asm volatile("{ .reg .pred q; setp.gt.s32 q, %5, %6; @q ld.global.v4.b32 {%0,%1,%2,%3}, [%4]; }"
                     : "=r"(r.w[4 * i]), "=r"(r.w[4 * i + 1]), "=r"(r.w[4 * i + 2]), "=r"(r.w[4 * i + 3])
                     : "l"(base + i * kPer), "r"(reach), "r"(i * kPer));
    return r;
}
// Its words, zero where there is no column.
template <int kType>
__device__ __forceinline__ Raw<kType> arrive(const Pieces<kType>& q, const typename Word<kType>::type* p, int n) {
    constexpr int kPer = kType == QFMT_F32 ? 4 : 8;
    const uint32_t first = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) / (16 / kPer);
    Raw<kType> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.w) / 4); ++i) r.w[i] = q.w[i];
    if (first != 0) r = shifted<kType>(q.w, first);
    if (n != kGranule || !q.inside) {
        const bool read = n > 0 && !q.inside;
#pragma unroll
        for (int j = 0; j < kGranule; ++j) {
            uint32_t w = word_of<kType>(r, j);
            if (read && j < n) w = (uint32_t)p[j];
            if (j >= n) w = 0u;
            if constexpr (kType == QFMT_F32) r.w[j] = w;
            else r.w[j / 2] = j & 1 ? (r.w[j / 2] & 0xFFFFu) | (w << 16) : (r.w[j / 2] & 0xFFFF0000u) | w;
        }
    }
    return r;
}
template <int kType>
__device__ __forceinline__ Raw<kType> load_any(const typename Word<kType>::type* p, int n, bool inside) {
    return arrive<kType>(start_any<kType>(p, n, inside), p, n);
}

// Writes `n` columns (0..8) of a granule at p.  Called by whole warps.  `from` and `to`: the lane before this one holds
// the granule before this one, the lane after it the next.  Where rows do not start on granule boundaries a lane
// writes the aligned 16-byte pieces that begin inside its granule, the last one with words of the next lane, and only
// the ends of a warp's stretch are written by elements.
template <int kType>
__device__ __forceinline__ void store_any(typename Word<kType>::type* p, int n, const Target<kType>& m, const Raw<kType>& r, bool from,
                                          bool to) {
    constexpr int kPer = kType == QFMT_F32 ? 4 : 8;
    uint32_t left = (1u << n) - 1u;  // columns that no aligned piece covers
    if (m.whole) {
        if (n == kGranule) {
            store_raw<kType>(p, r);
            left = 0u;
        }
    } else {
        const int following = __shfl_down_sync(0xFFFFFFFFu, n, 1);
        uint32_t w[8];  // the last 16 bytes of this granule and the first 16 of the next
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = r.w[kType == QFMT_F32 ? 4 + i : i];
            w[4 + i] = __shfl_down_sync(0xFFFFFFFFu, r.w[i], 1);
        }
        const int skew = (int)(reinterpret_cast<uintptr_t>(p) & 15u) / (16 / kPer);
        const int first = (kPer - skew) & (kPer - 1);  // columns before the first piece that begins here
        const uint32_t before = (1u << first) - 1u;
        if (from && n >= first) left &= ~before;
        const bool full = n == kGranule;
        const bool last = skew != 0 ? to && following >= first : full;  // the piece that may need the next lane's words
        Four q;
        if constexpr (kType == QFMT_F32) {
            if (full) {  // a piece in the middle is all this lane's
                const uint32_t own[8] = {r.w[0], r.w[1], r.w[2], r.w[3], r.w[4], r.w[5], r.w[6], r.w[7]};
                q = shifted_words(own, first);
                asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(p + first), "r"(q.w[0]), "r"(q.w[1]), "r"(q.w[2]), "r"(q.w[3]) : "memory");
                left &= ~(0xFu << first);
            }
            q = shifted_words(w, first);
        } else {
            const Raw<kType> s = shifted<kType>(w, first);
            q = {{s.w[0], s.w[1], s.w[2], s.w[3]}};
        }
        if (last) {
            constexpr int kMiddle = kType == QFMT_F32 ? 4 : 0;
            asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};" ::"l"(p + first + kMiddle), "r"(q.w[0]), "r"(q.w[1]), "r"(q.w[2]), "r"(q.w[3]) : "memory");
            left &= (1u << (first + kMiddle)) - 1u;
        }
    }
    if (left != 0u) {
#pragma unroll
        for (int j = 0; j < kGranule; ++j)
            if (left >> j & 1u) p[j] = (typename Word<kType>::type)word_of<kType>(r, j);
    }
}

// Eight finished values to words, rounded once to the storage type (nearest, ties to even).
template <int kType>
__device__ __forceinline__ Raw<kType> finish(const Granule& v) {
    Raw<kType> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (kType == QFMT_F32) {
            r.w[2 * j] = __float_as_uint(v.p[j].x);
            r.w[2 * j + 1] = __float_as_uint(v.p[j].y);
        } else if constexpr (kType == QFMT_BF16) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w[j]) : "f"(v.p[j].y), "f"(v.p[j].x));
        } else {
            asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r.w[j]) : "f"(v.p[j].y), "f"(v.p[j].x));
        }
    }
    return r;
}

// The same rounded to the format *p (for codes, the one of their storage type); the bins of the first `n`
// columns are counted in the per-lane histogram `hist` when there is one.
template <int kType, int kLanes>
__device__ __forceinline__ Raw<kType> finish_format(const Granule& v, int n, const QuantParams& p, uint32_t* hist) {
    Raw<kType> r;
    int bin[kGranule];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t x = __float_as_uint(v.p[j].x), y = __float_as_uint(v.p[j].y);
        if constexpr (kType == QFMT_F32) {
            r.w[2 * j] = quantize_one<false>(x, p, bin[2 * j]);
            r.w[2 * j + 1] = quantize_one<false>(y, p, bin[2 * j + 1]);
        } else {
            r.w[j] = quantize_pack_pair_native<false, kType == QFMT_BF16>(x, y, p, bin[2 * j], bin[2 * j + 1]);
        }
    }
    if (hist != nullptr) {
        const int lane = threadIdx.x & (kLanes - 1);
#pragma unroll
        for (int j = 0; j < kGranule; ++j)
            if (j < n) atomicAdd(&hist[bin[j] * kLanes + lane], 1u);
    }
    return r;
}

// A granule of n columns at p, in row `row` of `rows`, on its way, and its words: zeros where there is nothing.
// kPlain: whole and aligned, or not there at all.  edge: at_edge() of the granule, inner: inner_rows().
template <int kType, bool kPlain>
using OnItsWay = std::conditional_t<kPlain, Raw<kType>, Pieces<kType>>;
template <int kType, bool kPlain>
__device__ __forceinline__ OnItsWay<kType, kPlain> start(const typename Word<kType>::type* p, int n, uint32_t row, uint32_t rows, bool edge,
                                                           uint32_t inner) {
    if constexpr (kPlain) return load_raw<kType>(p, n, row, rows);
    else return start_any<kType>(p, row < rows ? n : 0, pieces_inside(edge, row, inner));
}
template <int kType, bool kPlain>
__device__ __forceinline__ Raw<kType> words(const OnItsWay<kType, kPlain>& q, const typename Word<kType>::type* p, int n) {
    if constexpr (kPlain) return q;
    else return arrive<kType>(q, p, n);
}
template <int kType, bool kPlain>
__device__ __forceinline__ void put(typename Word<kType>::type* p, int n, const Target<kType>& m, const Raw<kType>& r, bool from, bool to) {
    if constexpr (kPlain) {
        if (n > 0) store_raw<kType>(p, r);
    } else {
        store_any<kType>(p, n, m, r, from, to);
    }
}

struct DropParams {
    uint32_t active;  // 0: nothing is dropped
    uint32_t limit;   // 65536 t - 1: 16 random bits, moved to the top of a word, at or below this drop their element
    float scale;      // 65536 / (65536 - t): the mean is kept exactly for the threshold in use
    uint32_t key[10][2];  // of every round
    uint64_t offset;
    const uint64_t* d_offset;  // added to offset when the kernel runs, or NULL
};

// Rows of containers of any alignment through shared memory: a team copies a row there asynchronously, in 16-byte pieces and
// as many words past a 16-byte boundary as it starts in global memory (its skew), word by word what is before the first and
// behind the last whole piece.  (All of a skewed row word by word: 16384 x 1021 forward 34 us against 31, backward of 16384 x
// 4093 250 against 211.)
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
inline __host__ __device__ uint32_t staged_row_bytes(int64_t cols) { return (uint32_t)((cols + kGranule - 1) / kGranule * kGranule * 4 + 16); }
__device__ __forceinline__ int row_skew(const uint32_t* row) { return (int)(reinterpret_cast<uintptr_t>(row) >> 2 & 3u); }
__device__ __forceinline__ void stage_row(uint32_t shared, const uint32_t* row, int cols, int t, int team) {
    const int skew = row_skew(row), start = min(cols, -skew & 3), end = start + (cols - start) / 4 * 4;
    shared += 4 * skew;
    for (int i = start + 4 * t; i < end; i += 4 * team)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared + 4 * i), "l"(row + i) : "memory");
    for (int i = t; i < start + cols - end; i += team) {
        const int c = i < start ? i : i - start + end;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(shared + 4 * c), "l"(row + c) : "memory");
    }
}
__device__ __forceinline__ void stage_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stage_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }  // this thread's copies

// n columns (0..8) of granule g of a staged row, zeros where there are none.
__device__ __forceinline__ Raw<QFMT_F32> staged_granule(uint32_t shared, int skew, int g, int n) {
    Raw<QFMT_F32> r;
#pragma unroll
    for (uint32_t& w : r.w) w = 0u;
    if (n <= 0) return r;
    const uint32_t at = shared + (uint32_t)g * 32;
    uint32_t q[12];
    const auto load = [&](int i) {
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(q[i]), "=r"(q[i + 1]), "=r"(q[i + 2]), "=r"(q[i + 3]) : "r"(at + 4 * i) : "memory");
    };
    load(0), load(4);
    const auto take = [&](int first) {
#pragma unroll
        for (int j = 0; j < kGranule; ++j) r.w[j] = j < n ? q[first + j] : 0u;
    };
    if (skew == 0) {
        take(0);
        return r;
    }
    load(8);
    if (skew == 1) take(1);
    else if (skew == 2) take(2);
    else take(3);
    return r;
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten
// rounds of two 32 x 32 -> 64-bit products on a counter of four words, each with its key.
__device__ __forceinline__ uint4 philox4x32_10(uint4 c, const DropParams& d) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
        c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ d.key[r][0], (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ d.key[r][1], (uint32_t)a);
    }
    return c;
}

__device__ __forceinline__ uint64_t drop_offset(const DropParams& d) {
    return d.offset + (d.d_offset != nullptr ? *d.d_offset : 0ull);
}

// D(v) of the granule of columns 8 * granule .. of a row.  A dropped element is zero whatever it held (a
// selection, not a product: inf and NaN do not get through).  The upper half of a random word is compared in
// place (its lower half cannot reach the limit's ones), the lower half after a shift.
__device__ __forceinline__ void drop_granule(const DropParams& d, uint64_t offset, uint32_t row, uint32_t granule, Granule& v) {
    const uint4 r = philox4x32_10(make_uint4(granule, row, (uint32_t)offset, (uint32_t)(offset >> 32)), d);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 s = mul2(v.p[j], both(d.scale));
        v.p[j].x = (w[j] << 16) > d.limit ? s.x : 0.0f;
        v.p[j].y = w[j] > d.limit ? s.y : 0.0f;
    }
}

// Per-lane histogram [bin][lane] in shared memory: cleared by the whole block, merged into the device
// record by the whole block at the end (round.cuh).  kLanes: counters of a bin, 32 (no two lanes of a warp meet) or 16 where
// shared memory is short.
constexpr int kHistLanes = 32;
template <int kLanes = kHistLanes>
__device__ __forceinline__ void clear_hist(uint32_t* hist, const QuantParams& p) {
    for (int i = threadIdx.x; i < (p.top + kExtraBins) * kLanes; i += blockDim.x) hist[i] = 0u;
    __syncthreads();
}
template <int kLanes = kHistLanes>
__device__ __forceinline__ void flush_hist(const uint32_t* hist, const QuantParams& p, qfmt_stats_t* stats, uint64_t n_total) {
    __syncthreads();
    const int lane = threadIdx.x & 31;
    for (int b = (threadIdx.x >> 5) + 1; b < p.top + kExtraBins; b += blockDim.x >> 5) {  // bin 0 is never used
        const uint32_t c = __reduce_add_sync(0xFFFFFFFFu, lane < kLanes ? hist[b * kLanes + lane] : 0u);
        if (lane == 0 && c != 0u) merge_bin(stats, p, b, c);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicAdd((unsigned long long*)&stats->n_total, (unsigned long long)n_total);
}

// Host side -----------------------------------------------------------------------------------------------

inline size_t element_size(int32_t dtype) { return dtype == QFMT_F32 ? 4 : 2; }
inline size_t granule_bytes(int32_t dtype) { return kGranule * element_size(dtype); }
inline bool element_aligned(const void* p, int32_t dtype) { return (reinterpret_cast<uintptr_t>(p) & (element_size(dtype) - 1)) == 0; }
// Whether every row of a matrix starts on a granule boundary.
inline bool granule_aligned(const void* p, int64_t ld, int32_t dtype) {
    return (reinterpret_cast<uintptr_t>(p) & (granule_bytes(dtype) - 1)) == 0 && ld % kGranule == 0;
}
template <int kType>
Source<kType> make_source(const void* p, int64_t ld) {
    return {static_cast<const typename Word<kType>::type*>(p), ld, granule_aligned(p, ld, kType)};
}
template <int kType>
Target<kType> make_target(void* p, int64_t ld) {
    return {static_cast<typename Word<kType>::type*>(p), ld, granule_aligned(p, ld, kType)};
}

inline int make_drop_params(const qfmt_dropout_t* d, DropParams* out) {
    *out = DropParams{};
    if (d == nullptr) return QFMT_OK;
    if (!(d->p >= 0.0f && d->p <= 1.0f) || (reinterpret_cast<uintptr_t>(d->d_offset) & 7u)) return QFMT_ERR_BAD_ARG;
    const uint32_t t = (uint32_t)((double)d->p * 65536.0 + 0.5);
    out->active = t != 0u;
    out->limit = (t << 16) - 1u;  // t = 65536: all ones, which nothing exceeds
    out->scale = t < 65536u ? (float)(65536.0 / (65536.0 - (double)t)) : 0.0f;
    for (int r = 0; r < 10; ++r) {
        out->key[r][0] = (uint32_t)d->seed + (uint32_t)r * 0x9E3779B9u;
        out->key[r][1] = (uint32_t)(d->seed >> 32) + (uint32_t)r * 0xBB67AE85u;
    }
    out->offset = d->offset;
    out->d_offset = d->d_offset;
    return QFMT_OK;
}

// Blocks of a kernel that an SM holds at once.  `known` remembers the last answer for every block size (with the bytes
// of shared memory it was for), since asking takes as long as a launch.
template <typename K>
int resident_blocks(K kernel, unsigned block, size_t smem, std::atomic<uint64_t>* known, int* out) {
    std::atomic<uint64_t>& slot = known[block / 32];
    const uint64_t seen = slot.load(), key = (uint64_t)smem << 8 | 0x80u;
    if ((seen & ~(uint64_t)0x7Fu) == key) {
        *out = (int)(seen & 0x7Fu);
        return QFMT_OK;
    }
    QFMT_CUDA_TRY(cudaOccupancyMaxActiveBlocksPerMultiprocessor(out, kernel, (int)block, smem));
    if (*out < 1) *out = 1;
    slot.store(key | (uint64_t)*out);
    return QFMT_OK;
}

}  // namespace
}  // namespace qfmt
