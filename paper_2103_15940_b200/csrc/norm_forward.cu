// Layer normalisation and its fused form, forward: y = LN(x), or h = residual + D(x) and y = LN(h) in one pass.
//
// Bound by memory: every element is read once and written once.  What stands in the way is the number of instructions
// and the two sums a row needs one after the other (the variance is taken about the mean: a one-pass formula would lose
// rows whose mean is large against their spread), so
//   * a row stays in registers, two granules a thread, and additions and products issue in pairs: 118 instructions a
//     granule and warp, against 186 with branches around loads and 64-bit row arithmetic (76 us -> 59 us on the first case below);
//   * two rows at a time share the barriers, and five shuffles reduce both rows' sums (79 instructions, 59 -> 48 us);
//   * weight and bias stay in registers from row to row; four granules a thread without them took 75 us (their
//     reads from L1 are four times the row's);
//   * the next rows' granules are loaded while these are worked on.
// Measured (replayed from a graph, on sets of tensors larger than L2 in turn, as all figures here that do not say otherwise):
// 16384 x 4096 bfloat16 46.9 us (5.7 TB/s, 0.89 of the measured copy rate), 4096 x 768 fp32 6.3 us (4.8 in L2), fused 8192 x 1024
// bfloat16 14.6 us (4.6 TB/s), fused 16384 x 4096 bfloat16 89 us (6.0 TB/s), fp32 182 us (5.9 TB/s).
#include <cuda_runtime.h>
#include <stdint.h>

#include "norm.cuh"

namespace qfmt {
namespace {

template <int kType>
struct ForwardArgs {
    Source<kType> x, residual;  // residual.p may be NULL
    const float* weight;
    const float* bias;
    Target<kType> h, y;  // h.p may be NULL
    float* mean;
    float* rstd;
    int64_t rows, cols;
    uint32_t inner;  // inner_rows()
    float eps;
    float inverse;  // 1 / cols
    bool fmt;       // quant holds a format to round to
    DropParams drop;
    QuantParams quant;
    qfmt_stats_t* stats;
};

// residual + D(x)
template <int kType, bool kFused>
__device__ __forceinline__ Granule join_h(const ForwardArgs<kType>& a, const Raw<kType>& x, const Raw<kType>& r, uint64_t offset, uint32_t row,
                                          uint32_t g) {
    Granule v = widen_raw<kType>(x);
    if constexpr (kFused) {
        if (a.drop.active) drop_granule(a.drop, offset, row, g, v);
        if (a.residual.p != nullptr) {
            const Granule u = widen_raw<kType>(r);
#pragma unroll
            for (int j = 0; j < 4; ++j) v.p[j] = add2(u.p[j], v.p[j]);
        }
    }
    return v;
}

__device__ __forceinline__ float sum8(const Granule& v) {
    const float2 s = add2(add2(v.p[0], v.p[1]), add2(v.p[2], v.p[3]));
    return s.x + s.y;
}
// v - mean where a column exists, 0 elsewhere; the sum of its squares.  kPlain: all eight exist or (v = 0) none.
template <bool kPlain>
__device__ __forceinline__ float centre(Granule& v, float mean, int n) {
    const float2 shift = both(kPlain && n == 0 ? 0.0f : -mean);
#pragma unroll
    for (int j = 0; j < 4; ++j) v.p[j] = add2(v.p[j], shift);
    if (!kPlain && n < kGranule) clear_from(v, n);
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < 4; ++j) s = fma2(v.p[j], v.p[j], s);
    return s.x + s.y;
}

// 1 / sqrt(v): the hardware's approximation, within 2^-22.9 of it.
__device__ __forceinline__ float inverse_root(float v) {
    float r;
    asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Rows too long for a team's registers: a block takes a row at a time and reads it three times, for the mean,
// for the variance and for the result.  A thread adds up a granule in 32 bits and the granules in 64, since it has cols / 4096 of them:
// in 32 bits the mean of 4 Mi equal columns was off by 170 roundings.
template <int kType, bool kFused>
__global__ void __launch_bounds__(kLoopThreads) norm_forward_loop_kernel(const ForwardArgs<kType> a) {
    extern __shared__ uint32_t lane_hist[];
    __shared__ float2 scratch[32];
    grid_dependency_wait();
    uint32_t* hist = a.stats != nullptr ? lane_hist : nullptr;
    if (hist != nullptr) clear_hist(hist, a.quant);
    const uint32_t granules = (uint32_t)((a.cols + kGranule - 1) / kGranule);
    const float count = (float)a.cols;
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    const bool from = threadIdx.x & 31, to = (threadIdx.x & 31) != 31;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const auto h = [&](uint32_t g, int n) {
            const int64_t col = (int64_t)g * kGranule;
            const bool inside = pieces_inside(at_edge(a.cols, g), (uint32_t)row, a.inner);
            const Raw<kType> res = kFused && a.residual.p != nullptr
                                       ? load_any<kType>(a.residual.p + row * a.residual.ld + col, n, inside) : Raw<kType>();
            return join_h<kType, kFused>(a, load_any<kType>(a.x.p + row * a.x.ld + col, n, inside), res, offset, (uint32_t)row, g);
        };
        double sum = 0.0;
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) sum += (double)sum8(h(g, granule_columns(a.cols, g)));
        const float mean = block_sum(make_float2((float)sum, 0.0f), scratch).x / count;
        sum = 0.0;
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            const int n = granule_columns(a.cols, g);
            Granule v = h(g, n);
            sum += (double)centre<false>(v, mean, n);
        }
        const float rstd = inverse_root(block_sum(make_float2((float)sum, 0.0f), scratch).x / count + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean != nullptr) a.mean[row] = mean;
            if (a.rstd != nullptr) a.rstd[row] = rstd;
        }
        for (uint32_t g0 = 0; g0 < granules; g0 += kLoopThreads) {  // whole warps
            const uint32_t g = g0 + threadIdx.x;
            const int64_t col = (int64_t)g * kGranule;
            const int n = granule_columns(a.cols, g);
            Granule v = h(g, n);
            if (kFused && a.h.p != nullptr) store_any<kType>(a.h.p + row * a.h.ld + col, n, a.h, finish<kType>(v), from, to);
            const Granule w = load_columns(a.weight, g, n, 1.0f), b = load_columns(a.bias, g, n, 0.0f);
#pragma unroll
            for (int j = 0; j < 4; ++j) v.p[j] = fma2(mul2(add2(v.p[j], both(-mean)), both(rstd)), w.p[j], b.p[j]);
            store_any<kType>(a.y.p + row * a.y.ld + col, n, a.y, finish_output<kType, false>(a, v, n, hist), from, to);
        }
    }
    if (hist != nullptr) flush_hist(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
}

// Sums over a team, in every thread and in a fixed order: of one value, or of two at once.  kBlock: the team is the
// block.  One barrier, so the next sum needs another scratch.
template <bool kBlock>
__device__ __forceinline__ void team_sum(float (&s)[1], int team, int t, float* scratch) {
    if constexpr (!kBlock) {
        for (int off = team >> 1; off > 0; off >>= 1) s[0] = across(s[0], off);
    } else {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s[0] = across(s[0], off);
        if (team == 32) return;
        if ((t & 31) == 0) scratch[t >> 5] = s[0];
        __syncthreads();
        sum_entries<1>(scratch, team, s);
    }
}
// Two values: after one exchange the lower half of a warp holds the first value's partial sums and the upper half
// the second's, so five shuffles do for both.
template <bool kBlock>
__device__ __forceinline__ void team_sum(float (&s)[2], int team, int t, float* scratch) {
    if constexpr (!kBlock) {
        for (int off = team >> 1; off > 0; off >>= 1) s[0] = across(s[0], off), s[1] = across(s[1], off);
    } else {
        const bool upper = t & 16;
        float u = (upper ? s[1] : s[0]) + __shfl_xor_sync(0xFFFFFFFFu, upper ? s[0] : s[1], 16);
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) u = across(u, off);
        if (team == 32) {
            const float v = __shfl_xor_sync(0xFFFFFFFFu, u, 16);
            s[0] = upper ? v : u;
            s[1] = upper ? u : v;
            return;
        }
        if ((t & 15) == 0) scratch[(t & 16) + (t >> 5)] = u;
        __syncthreads();
        sum_entries<2>(scratch, team, s);
    }
}

// Elements from a row of a team to its next one.
struct ForwardSteps {
    int64_t x, residual, h, y;
};

// R rows at a time are read once and stay in their team's registers.  V <= 2: so do the team's weight and bias,
// from row to row; of longer rows where they fit (kKeep).
// kPlain: every granule whole and aligned, no format; granules go straight to registers, with V <= 2 those of the next
// rows while these are worked on.  Otherwise any layout and an optional format: codes come as aligned pieces that are
// shifted into place; rows of containers (kStaged) go through shared memory behind the histogram, where the next row
// is copied as soon as this one has been read from there by its whole team.  fp32 16384 x 1021 takes 39 us shifted and 30
// staged; codes were staged only word by word (31 us against 23 shifted, in L2), not in pieces as containers are now.
// Registers: 128 for a team of 512; fewer where more blocks on an SM are worth more, the general variant without dropout.  With
// 128 against these: fp32 16384 x 4093 133 and 123 us; bfloat16 16384 x 4093 121 and 121, x 2049 76 and 62, x 1021 31 and 27, 2048 x
// 10237 50 and 42.  (Bfloat16 at 96, 80, 72: x 4093 120, 109, 127, x 2049 62, 71, 74.  With dropout they spill: bfloat16
// 16384 x 4093 at 128, 80: 206, 240.)
constexpr int forward_registers(int type, int v, bool fused, bool plain) {
    if (plain || fused || v == 4) return 128;
    if (v == 1) return 64;
    return type == QFMT_F32 ? (v == 2 ? 80 : 64) : (v == 2 ? 96 : 72);
}
template <int kType, int V, int R, bool kFused, bool kPlain>
__global__ void __maxnreg__((forward_registers(kType, V, kFused, kPlain)))
norm_forward_rows_kernel(const ForwardArgs<kType> a, int team, const ForwardSteps step, int hist_words) {
    // Wide rows keep the weights where that leaves the blocks of an SM as many as before.  2048 rows, kept against read again, us:
    // of 16384 bfloat16 41 against 50 / fused 64 against 68, fp32 53 against 62 / fused 105 against 89; of 12288 fused bfloat16 50
    // against 54, fp32 67 against 71.  Of 9216 bfloat16 without dropout 30 against 25, which the rule goes by; towards 12288
    // columns it turns (35 against 42, fp32 46 against 52).
    constexpr bool kKeep = V <= 2 || (V == 3 ? kFused && (kPlain || kType == QFMT_F32) : !(kFused && kType == QFMT_F32));
    constexpr bool kAhead = V <= 2 && kPlain, kStaged = !kPlain && kType == QFMT_F32;
    extern __shared__ __align__(16) uint32_t dynamic[];
    __shared__ __align__(16) float scratch[2][R][16];
    grid_launch_dependents();
    grid_dependency_wait();
    uint32_t* hist = !kPlain && a.stats != nullptr ? dynamic : nullptr;
    if (V > 1) {
        for (int i = threadIdx.x; i < 2 * R * 16; i += blockDim.x) (&scratch[0][0][0])[i] = 0.0f;
        __syncthreads();
    }
    if (hist != nullptr) clear_hist(hist, a.quant);
    const int mine = V > 1 ? 0 : threadIdx.x / team, t = threadIdx.x - mine * team, teams = V > 1 ? 1 : blockDim.x / team;
    const bool from = (t & 31) != 0, to = (t & 31) != 31 && t + 1 < team;  // the lanes before and after hold neighbours
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    const bool residual = kFused && a.residual.p != nullptr;
    const int next = team * kGranule;  // elements between a thread's granules
    int n[V];                          // columns of each granule
#pragma unroll
    for (int k = 0; k < V; ++k) n[k] = granule_columns(a.cols, k * team + t);

    // A team past the last row, whose warp has teams with one, keeps in step with them and stores nothing.
    const uint32_t rows = (uint32_t)a.rows, stride = gridDim.x * teams * R;
    uint32_t row = (blockIdx.x * teams + mine) * R;
    const auto* px = a.x.p + row * a.x.ld + (kStaged ? 0 : t * kGranule);
    const auto* pr = a.residual.p + row * a.residual.ld + (kStaged ? 0 : t * kGranule);
    auto* ph = a.h.p + row * a.h.ld + t * kGranule;
    auto* py = a.y.p + row * a.y.ld + t * kGranule;
    OnItsWay<kType, kPlain || kStaged> x[R][V], r[R][V];
    const auto fetch_rows = [&](uint32_t at) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const bool edge = at_edge(a.cols, k * team + t);
                x[i][k] = start<kType, kPlain || kStaged>(px + i * a.x.ld + k * next, n[k], at + i, rows, edge, a.inner);
                if (kFused)
                    r[i][k] = start<kType, kPlain || kStaged>(pr + i * a.residual.ld + k * next, residual ? n[k] : 0, at + i, rows, edge, a.inner);
            }
        }
        if (kAhead) px += step.x, pr += step.residual;
    };
    const uint32_t row_bytes = staged_row_bytes(a.cols);
    const uint32_t place = shared_address(dynamic + hist_words) + mine * (kFused ? 2 : 1) * row_bytes;  // of the team
    [[maybe_unused]] int skew_x = 0, skew_r = 0;
    const auto stage_next = [&]([[maybe_unused]] uint32_t at) {  // the next row through shared memory
        if constexpr (kStaged) {
            skew_x = row_skew(px), skew_r = row_skew(pr);
            if (at < rows) {
                stage_row(place, px, (int)a.cols, t, team);
                if (residual) stage_row(place + row_bytes, pr, (int)a.cols, t, team);
            }
            stage_end();
            px += step.x;
            pr += step.residual;
        }
    };
    if (kAhead) fetch_rows(row);
    stage_next(row);
    Granule w[kKeep ? V : 1], b[kKeep ? V : 1];
    if constexpr (kKeep) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            w[k] = load_columns(a.weight, k * team + t, n[k], 1.0f);
            b[k] = load_columns(a.bias, k * team + t, n[k], 0.0f);
        }
    }
    for (; row - mine * R < rows; row += stride) {
        if constexpr (kStaged) {
            stage_wait();
            if (V > 1) __syncthreads();
            else __syncwarp();
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int there = row < rows ? n[k] : 0;
                x[0][k] = staged_granule(place, skew_x, k * team + t, there);
                if (kFused) r[0][k] = staged_granule(place + row_bytes, skew_r, k * team + t, residual ? there : 0);
            }
        } else if (!kAhead) {
            fetch_rows(row);
        }
        Granule v[R][V];
        float mean[R], rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int there = row + i < rows ? n[k] : 0;
                const Raw<kType> xs = words<kType, kPlain || kStaged>(x[i][k], px + i * a.x.ld + k * next, there);
                const Raw<kType> rs = kFused ? words<kType, kPlain || kStaged>(r[i][k], pr + i * a.residual.ld + k * next, residual ? there : 0)
                                             : Raw<kType>();
                v[i][k] = join_h<kType, kFused>(a, xs, rs, offset, row + i, k * team + t);
            }
        if (kAhead) fetch_rows(row + stride);
        else if (!kStaged) px += step.x, pr += step.residual;
        if (kFused && a.h.p != nullptr) {
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    put<kType, kPlain>(ph + i * a.h.ld + k * next, row + i < rows ? n[k] : 0, a.h, finish<kType>(v[i][k]), from, to);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mean[i] = sum8(v[i][0]);
#pragma unroll
            for (int k = 1; k < V; ++k) mean[i] += sum8(v[i][k]);
        }
        team_sum<(V > 1)>(mean, team, t, scratch[0][0]);
        if (V == 1 || team == 32) __syncwarp();  // the sum of one warp or less is shuffles, which order no memory
        stage_next(row + stride);  // behind the sum's barrier: everyone has read the place
#pragma unroll
        for (int i = 0; i < R; ++i) {
            mean[i] *= a.inverse;
            rstd[i] = centre<kPlain>(v[i][0], mean[i], n[0]);
#pragma unroll
            for (int k = 1; k < V; ++k) rstd[i] += centre<kPlain>(v[i][k], mean[i], n[k]);
        }
        team_sum<(V > 1)>(rstd, team, t, scratch[1][0]);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            rstd[i] = inverse_root(rstd[i] * a.inverse + a.eps);
            if (t == 0 && row + i < rows) {
                if (a.mean != nullptr) a.mean[row + i] = mean[i];
                if (a.rstd != nullptr) a.rstd[row + i] = rstd[i];
            }
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if constexpr (!kKeep) {
                w[0] = load_columns(a.weight, k * team + t, n[k], 1.0f);
                b[0] = load_columns(a.bias, k * team + t, n[k], 0.0f);
            }
            const Granule& wk = w[kKeep ? k : 0];
            const Granule& bk = b[kKeep ? k : 0];
#pragma unroll
            for (int i = 0; i < R; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][k].p[j] = fma2(mul2(v[i][k].p[j], both(rstd[i])), wk.p[j], bk.p[j]);
                const int there = row + i < rows ? n[k] : 0;
                put<kType, kPlain>(py + i * a.y.ld + k * next, there, a.y, finish_output<kType, kPlain>(a, v[i][k], there, hist), from, to);
            }
        }
        ph += step.h;
        py += step.y;
    }
    if (hist != nullptr) flush_hist(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
}

Plan forward_plan(int64_t cols) { return make_plan(cols, 2, 4); }

template <int kType, int V, int R, bool kFused, bool kPlain>
int launch_forward_rows(const Call& c, const ForwardArgs<kType>& a, int team, cudaStream_t stream) {
    static std::atomic<uint64_t> known[kMaxTeam / 32 + 1];
    const auto kern = norm_forward_rows_kernel<kType, V, R, kFused, kPlain>;
    const unsigned teams = V > 1 ? 1 : 128 / team, block = teams * team;
    constexpr bool kStaged = !kPlain && kType == QFMT_F32;
    const size_t smem = c.hist_bytes + (kStaged ? (size_t)teams * (kFused ? 2 : 1) * staged_row_bytes(a.cols) : 0);
    static std::atomic<bool> allowed[64];
    if (kStaged) {
        const int rc = allow_shared(kern, kMostShared, c.dev, allowed);
        if (rc != QFMT_OK) return rc;
    }
    int resident = 0;
    const int rc = resident_blocks(kern, block, smem, known, &resident);
    if (rc != QFMT_OK) return rc;
    const int64_t want = (a.rows + teams * R - 1) / (teams * R), cap = (int64_t)c.dev.sm_count * resident;
    // Two rows at a time only where every team has them, and not where the mask's arithmetic already fills a small team's
    // time.  Fused bfloat16, two against one: 8192 x 1024 on the same tensors in L2 12.6 against 11.2 us; from memory 14.6 against
    // 14.4, 65536 x 512 49.0 against 47.8, but 16384 x 1024 25.6 against 26.2 and x 768 21.6 against 23.2.  Teams of more than 64:
    // 8192 x 4096 45.6 against 50.1 (in L2).
    if constexpr (R == 2) {
        if (want < cap || (kFused && V == 2 && team <= 64)) return launch_forward_rows<kType, V, 1, kFused, kPlain>(c, a, team, stream);
    }
    const unsigned blocks = (unsigned)(want < cap ? want : cap);
    const int64_t stride = (int64_t)blocks * teams * R;
    const ForwardSteps step = {stride * a.x.ld, stride * a.residual.ld, stride * a.h.ld, stride * a.y.ld};
    QFMT_CUDA_TRY(launch_overlapping(kern, blocks, block, smem, stream, a, team, step, (int)(c.hist_bytes / 4)));
    return QFMT_OK;
}

template <int kType, bool kFused>
int launch_forward(const Call& c, const ForwardArgs<kType>& a, cudaStream_t stream) {
    const Plan plan = forward_plan(a.cols);
    if (plan.team != 0) {
        const bool plain = plain_layout(a.cols, {a.x.whole, a.residual.whole, a.h.whole, a.y.whole}) && !a.fmt;
        constexpr int kRows = kFused && kType == QFMT_F32 ? 1 : 2;  // two wide fp32 rows of x and residual do not fit
        const auto run = plain ? (plan.granules == 1   ? launch_forward_rows<kType, 1, 2, kFused, true>
                                  : plan.granules == 2 ? launch_forward_rows<kType, 2, kRows, kFused, true>
                                  : plan.granules == 3 ? launch_forward_rows<kType, 3, 1, kFused, true>
                                                       : launch_forward_rows<kType, 4, 1, kFused, true>)
                               : (plan.granules == 1   ? launch_forward_rows<kType, 1, 1, kFused, false>
                                  : plan.granules == 2 ? launch_forward_rows<kType, 2, 1, kFused, false>
                                  : plan.granules == 3 ? launch_forward_rows<kType, 3, 1, kFused, false>
                                                       : launch_forward_rows<kType, 4, 1, kFused, false>);
        return run(c, a, plan.team, stream);
    }
    const int64_t cap = (int64_t)c.dev.sm_count * 4;
    QFMT_CUDA_TRY(launch_overlapping(norm_forward_loop_kernel<kType, kFused>, (unsigned)(a.rows < cap ? a.rows : cap), kLoopThreads,
                                     c.hist_bytes, stream, a));
    return QFMT_OK;
}

template <int kType, bool kFused>
int forward(const Call& c, const void* d_x, const void* d_residual, const float* d_weight, const float* d_bias, void* d_h,
            void* d_y, float* d_mean, float* d_rstd, qfmt_stats_t* d_stats, cudaStream_t stream) {
    const qfmt_norm_t& s = c.norm;
    ForwardArgs<kType> a;
    a.x = make_source<kType>(d_x, s.ld_x);
    a.residual = make_source<kType>(d_residual, s.ld_residual);
    a.weight = d_weight;
    a.bias = d_bias;
    a.h = make_target<kType>(d_h, s.ld_h);
    a.y = make_target<kType>(d_y, s.ld_y);
    a.mean = d_mean;
    a.rstd = d_rstd;
    a.rows = s.rows;
    a.cols = s.cols;
    a.inner = inner_rows(s.cols, s.rows);
    a.eps = s.eps;
    a.inverse = 1.0f / (float)a.cols;
    a.fmt = c.fmt;
    a.drop = c.drop;
    a.quant = c.quant;
    a.stats = d_stats;
    return launch_forward<kType, kFused>(c, a, stream);
}

int forward_entry(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, bool fused, const void* d_x, const void* d_residual,
                  const float* d_weight, const float* d_bias, void* d_h, void* d_y, float* d_mean, float* d_rstd,
                  const qfmt_format_t* fmt, qfmt_stats_t* d_stats, int accumulate, cudaStream_t stream) {
    Call c;
    int rc = prepare_call(norm, drop, fmt, d_stats, accumulate, &c);
    if (rc != QFMT_OK) return rc;
    const int32_t t = c.norm.dtype;
    const bool empty = c.norm.rows == 0 || c.norm.cols == 0;
    if (!empty && (d_x == nullptr || d_y == nullptr)) return QFMT_ERR_BAD_ARG;
    if (!element_aligned(d_x, t) || !element_aligned(d_residual, t) || !element_aligned(d_h, t) || !element_aligned(d_y, t) ||
        !float_aligned(d_weight) || !float_aligned(d_bias) || !float_aligned(d_mean) || !float_aligned(d_rstd))
        return QFMT_ERR_BAD_ARG;
    rc = current_device(&c.dev);
    if (rc != QFMT_OK) return rc;
    if (d_stats != nullptr && accumulate == 0)
        QFMT_CUDA_TRY(launch_overlapping(zero_words_kernel, 1u, 256u, 0, stream, reinterpret_cast<int*>(d_stats),
                                         (int)(sizeof(qfmt_stats_t) / sizeof(int))));
    if (empty) return QFMT_OK;
    const auto run = fused ? (t == QFMT_F32 ? forward<QFMT_F32, true> : t == QFMT_F16 ? forward<QFMT_F16, true> : forward<QFMT_BF16, true>)
                           : (t == QFMT_F32 ? forward<QFMT_F32, false> : t == QFMT_F16 ? forward<QFMT_F16, false> : forward<QFMT_BF16, false>);
    return run(c, d_x, d_residual, d_weight, d_bias, d_h, d_y, d_mean, d_rstd, d_stats, stream);
}

}  // namespace
}  // namespace qfmt

extern "C" int qfmt_layer_norm(const qfmt_norm_t* norm, const void* d_x, const float* d_weight, const float* d_bias, void* d_y,
                               float* d_mean, float* d_rstd, const qfmt_format_t* fmt, qfmt_stats_t* d_stats, int accumulate,
                               void* stream) {
    return qfmt::forward_entry(norm, nullptr, false, d_x, nullptr, d_weight, d_bias, nullptr, d_y, d_mean, d_rstd, fmt, d_stats,
                               accumulate, (cudaStream_t)stream);
}

extern "C" int qfmt_dropout_add_layer_norm(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, const void* d_x,
                                           const void* d_residual, const float* d_weight, const float* d_bias, void* d_h,
                                           void* d_y, float* d_mean, float* d_rstd, const qfmt_format_t* fmt,
                                           qfmt_stats_t* d_stats, int accumulate, void* stream) {
    return qfmt::forward_entry(norm, drop, true, d_x, d_residual, d_weight, d_bias, d_h, d_y, d_mean, d_rstd, fmt, d_stats,
                               accumulate, (cudaStream_t)stream);
}
