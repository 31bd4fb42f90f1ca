// Layer normalisation and its fused form, backward: the gradients of the input, the residual, the weight and the bias.
//
// Bound by memory: dy and h are read once, each gradient is written once.  The sums over rows for the weight and the
// bias run along with the rows, in the registers of the thread that owns the columns, so nothing is read again for
// them; each SM's one block of 512 threads leaves one part of 2 n sums and a second kernel joins them (up to 148; the one part
// of a few rows is the result), in an order that depends on sizes alone.  Measured choices:
//   * up to 1280 columns one granule a thread and two rows at a time: 35.5 us for dx and the sums of 16384 x 1024 fp32; wider
//     rows by the rule at backward_plan;
//   * teams of one block, joined through its shared memory: small blocks in clusters that add up their sums through
//     distributed shared memory took 4 to 5 us more at the end of every call;
//   * with one granule a thread the sums are registers; with more, the registers hold the row and the sums lie in shared memory.
// Measured (replayed from a graph, on sets of tensors larger than L2 in turn, as all figures here that do not say otherwise):
// fused 8192 x 1024 fp32 26.6 us (5.0 TB/s, 0.78 of the measured copy rate), fused 8192 x 4096 bfloat16 53.0 us (5.1 TB/s), fused
// 16384 x 4096 fp32 187 us (5.8 TB/s), 4096 x 768 binary16 9.1 us (7.8 with three sets, partly in L2), of which joining takes 3.
#include <cuda_runtime.h>
#include <stdint.h>

#include "norm.cuh"

namespace qfmt {
namespace {

template <int kType>
struct BackwardArgs {
    Source<kType> dy, dh, h;  // dh: gradient that reaches h by another path, or NULL
    const float* mean;
    const float* rstd;
    const float* weight;
    Target<kType> dx, dresidual;  // or NULL
    float* partial;  // [parts][2][padded columns] sums of dy xhat and dy over a part of the rows, or NULL
    float* dweight;  // where a single part goes at once; both NULL with several parts
    float* dbias;
    int64_t rows, cols;
    uint32_t inner;  // inner_rows()
    float inverse;
    bool fmt;
    DropParams drop;
    QuantParams quant;
    qfmt_stats_t* stats;
};

// xhat of a granule; 0 where there is no column.  kPlain: all eight exist or (v = 0) none.
template <bool kPlain>
__device__ __forceinline__ Granule normalise(Granule v, float mean, float rstd, int n) {
    const float2 shift = both(kPlain && n == 0 ? 0.0f : -mean);
#pragma unroll
    for (int j = 0; j < 4; ++j) v.p[j] = mul2(add2(v.p[j], shift), both(rstd));
    if (!kPlain && n < kGranule) clear_from(v, n);
    return v;
}

// The row's two sums over one granule: g = w dy and g xhat.
__device__ __forceinline__ float2 row_sums(const Granule& dy, const Granule& xhat, const Granule& w) {
    float2 s = make_float2(0.0f, 0.0f), q = s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 g = mul2(dy.p[j], w.p[j]);
        s = add2(s, g);
        q = fma2(g, xhat.p[j], q);
    }
    return make_float2(s.x + s.y, q.x + q.y);
}

// Where the gradients of a row go, at a thread's first granule (and, i rows on, those of the next ones).
template <int kType>
struct GradientRow {
    const typename Word<kType>::type* dh;
    typename Word<kType>::type* dx;
    typename Word<kType>::type* dresidual;
    __device__ __forceinline__ GradientRow(const BackwardArgs<kType>& a, int64_t row, int64_t col)
        : dh(a.dh.p + row * a.dh.ld + col), dx(a.dx.p + row * a.dx.ld + col), dresidual(a.dresidual.p + row * a.dresidual.ld + col) {}
};

// What a granule's gradients become: dh (with what arrives by another path) to dresidual, D of it to dx.
template <int kType, bool kFused, bool kPlain, int kLanes = kHistLanes>
__device__ __forceinline__ void store_gradients(const BackwardArgs<kType>& a, const GradientRow<kType>& to, int i, int64_t at, const Granule& dy,
                                                const Granule& xhat, const Granule& w, float rstd, float c1, float c2, uint32_t row,
                                                uint32_t g, int n, bool from, bool after, uint64_t offset,
                                                uint32_t* hist) {
    Granule d;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        d.p[j] = mul2(fma2(xhat.p[j], both(-c2), fma2(dy.p[j], w.p[j], both(-c1))), both(rstd));
    if constexpr (kFused) {
        if (a.dh.p != nullptr) {
            const auto* p = to.dh + i * a.dh.ld + at;
            const Granule more = widen_raw<kType>(kPlain ? load_raw<kType>(p, n, 0, 1)
                                                         : load_any<kType>(p, n, pieces_inside(at_edge(a.cols, g), row, a.inner)));
#pragma unroll
            for (int j = 0; j < 4; ++j) d.p[j] = add2(d.p[j], more.p[j]);
        }
        if (a.dresidual.p != nullptr) put<kType, kPlain>(to.dresidual + i * a.dresidual.ld + at, n, a.dresidual, finish<kType>(d), from, after);
        if (a.drop.active && a.dx.p != nullptr) drop_granule(a.drop, offset, row, g, d);
    }
    if (a.dx.p != nullptr)
        put<kType, kPlain>(to.dx + i * a.dx.ld + at, n, a.dx, finish_output<kType, kPlain, kLanes>(a, d, n, hist), from, after);
}

// Long rows: a block takes a row at a time and reads it twice; a thread adds up its granules' sums in 64 bits, as in the forward
// pass.
template <int kType, bool kFused>
__global__ void __launch_bounds__(kLoopThreads) norm_backward_loop_kernel(const BackwardArgs<kType> a) {
    extern __shared__ uint32_t lane_hist[];
    __shared__ float2 scratch[32];
    uint32_t* hist = a.stats != nullptr ? lane_hist : nullptr;
    if (hist != nullptr) clear_hist(hist, a.quant);
    const uint32_t granules = (uint32_t)((a.cols + kGranule - 1) / kGranule);
    const float count = (float)a.cols;
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        const auto load = [&](uint32_t g, int n, Granule& dy, Granule& xhat, Granule& w) {
            const bool inside = pieces_inside(at_edge(a.cols, g), (uint32_t)row, a.inner);
            dy = widen_raw<kType>(load_any<kType>(a.dy.p + row * a.dy.ld + (int64_t)g * kGranule, n, inside));
            xhat = normalise<false>(widen_raw<kType>(load_any<kType>(a.h.p + row * a.h.ld + (int64_t)g * kGranule, n, inside)), mean, rstd, n);
            w = load_columns(a.weight, g, n, 1.0f);
        };
        double sum_g = 0.0, sum_gx = 0.0;
        Granule dy, xhat, w;
        for (uint32_t g = threadIdx.x; g < granules; g += kLoopThreads) {
            load(g, granule_columns(a.cols, g), dy, xhat, w);
            const float2 one = row_sums(dy, xhat, w);
            sum_g += (double)one.x;
            sum_gx += (double)one.y;
        }
        const float2 s = block_sum(make_float2((float)sum_g, (float)sum_gx), scratch);
        for (uint32_t g0 = 0; g0 < granules; g0 += kLoopThreads) {  // whole warps
            const uint32_t g = g0 + threadIdx.x;
            const int n = granule_columns(a.cols, g);
            load(g, n, dy, xhat, w);
            store_gradients<kType, kFused, false>(a, GradientRow<kType>(a, row, 0), 0, (int64_t)g * kGranule, dy, xhat, w, rstd, s.x / count,
                                                  s.y / count, (uint32_t)row, g, n, threadIdx.x & 31, (threadIdx.x & 31) != 31, offset, hist);
        }
    }
    if (hist != nullptr) flush_hist(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
}

// Sums over rows for the gradients of weight and bias of long rows: a block takes 32 granules of columns and
// one part of the rows, its eight warps every eighth row; their sums are joined in a fixed order.
constexpr int kColumnWarps = 8;
template <int kType>
__global__ void __launch_bounds__(32 * kColumnWarps) norm_column_sums_kernel(const BackwardArgs<kType> a) {
    __shared__ float part[kColumnWarps][2][kGranule][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t g = blockIdx.x * 32 + lane;
    const int n = granule_columns(a.cols, g);
    Granule dw = splat(0.0f), db = splat(0.0f);
    if (n > 0) {
        for (int64_t row = (int64_t)blockIdx.y * kColumnWarps + warp; row < a.rows; row += (int64_t)gridDim.y * kColumnWarps) {
            const bool inside = pieces_inside(at_edge(a.cols, g), (uint32_t)row, a.inner);
            const Granule dy = widen_raw<kType>(load_any<kType>(a.dy.p + row * a.dy.ld + (int64_t)g * kGranule, n, inside));
            const Granule xhat = normalise<false>(widen_raw<kType>(load_any<kType>(a.h.p + row * a.h.ld + (int64_t)g * kGranule, n, inside)), a.mean[row], a.rstd[row], n);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dw.p[j] = fma2(dy.p[j], xhat.p[j], dw.p[j]);
                db.p[j] = add2(db.p[j], dy.p[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kGranule; ++j) {
        part[warp][0][j][lane] = dw.at(j);
        part[warp][1][j][lane] = db.at(j);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kGranule * 32; i += 32 * kColumnWarps) {
        const int which = i / (kGranule * 32), l = i % (kGranule * 32) / kGranule, j = i % kGranule;
        const int64_t c = ((int64_t)blockIdx.x * 32 + l) * kGranule + j;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kColumnWarps; ++w) s += part[w][which][j][l];
        if (c < a.cols) a.partial[((int64_t)blockIdx.y * 2 + which) * ((a.cols + kGranule - 1) / kGranule * kGranule) + c] = s;
    }
}

// Elements from a row of a team to its next one.
struct BackwardSteps {
    int64_t dy, h, dh, dx, dresidual;
};

// Two sums of each of R rows over a team of whole warps that is one of several in its block, in every thread and in
// a fixed order.  With every exchange a lane gives up half of the values it holds, so six shuffles do for four values.
template <int R>
__device__ __forceinline__ void team_sums(float2 (&s)[R], int team, int t, int barrier, float* scratch) {
    const bool upper = t & 16, odd = t & 8;
    float u[R];
#pragma unroll
    for (int i = 0; i < R; ++i) u[i] = (upper ? s[i].y : s[i].x) + __shfl_xor_sync(0xFFFFFFFFu, upper ? s[i].x : s[i].y, 16);
    float v;
    if constexpr (R == 2) v = (odd ? u[1] : u[0]) + __shfl_xor_sync(0xFFFFFFFFu, odd ? u[0] : u[1], 8);
    else v = across(u[0], 8);
#pragma unroll
    for (int off = 4; off > 0; off >>= 1) v = across(v, off);
    // value 0 of row 0, 0 of row 1, 1 of row 0, 1 of row 1 in lanes 0, 8, 16, 24; with one row in lanes 0 and 16
    if ((t & 7) == 0 && (R == 2 || !odd)) scratch[(t & 24) * R + (t >> 5)] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(team) : "memory");
    float total[2 * R];
    sum_entries<2 * R>(scratch, team, total);
#pragma unroll
    for (int i = 0; i < R; ++i) s[i] = make_float2(total[i], total[R + i]);
}

// Column sums of one more row: dweight += dy xhat, dbias += dy.
__device__ __forceinline__ void add_columns(Granule& dw, Granule& db, const Granule& dy, const Granule& xhat) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        dw.p[j] = fma2(dy.p[j], xhat.p[j], dw.p[j]);
        db.p[j] = add2(db.p[j], dy.p[j]);
    }
}
__device__ __forceinline__ float4 quad(const Granule& v, int i) { return make_float4(v.p[2 * i].x, v.p[2 * i].y, v.p[2 * i + 1].x, v.p[2 * i + 1].y); }
__device__ __forceinline__ Granule from_quads(float4 a, float4 b) {
    return {{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}
__device__ __forceinline__ float4 sum_of(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

// Four columns of dweight and dbias laid side by side, from column 4 i on.
__device__ __forceinline__ void put_columns(int i, float4 s, int padded, int cols, float* dweight, float* dbias) {
    const bool second = 4 * i >= padded;
    float* const out = second ? dbias : dweight;
    const int c = 4 * i - (second ? padded : 0);
    const float v[4] = {s.x, s.y, s.z, s.w};
    if (out == nullptr) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < cols) out[c + j] = v[j];
}

// Counters of a bin.  The sums of the widest containers and a place for one row leave 24 KB for the histogram, whose 262 bins
// of 32 would take 33: a call with statistics would have to add up in the order of another kernel.
__host__ __device__ constexpr int backward_hist_lanes(int type, int v) { return type == QFMT_F32 && v == 4 ? kHistLanes / 2 : kHistLanes; }
static_assert((255 + kExtraBins) * backward_hist_lanes(QFMT_F32, 4) * 4 + 4 * kMaxTeam * 64 + 4 * kMaxTeam * kGranule * 4 + 16 <= kMostShared,
              "histogram, column sums and one place of the widest rows");

// The backward pass of rows that a team holds in registers, R at a time: dy and h are read once, the sums over rows
// stay in the registers of the thread that owns their columns from row to row, and a block leaves one part.
// kParts: a team is a part of a warp (or all of it), otherwise whole warps; a block has 512 threads' worth of teams.
// V > 1 (wide rows): the column sums lie in shared memory, each thread's its own, since the registers hold V granules of
// dy and h; V > 2: the team is the block; with V = 4 the weight is read from the cache as well.
// kPlain and kStaged as in the forward pass (16384 x 1021 bfloat16 takes 43 us in shifted pieces; staged word by word, before rows
// were staged in pieces, 75); with registers to spare (kAhead) the next rows are on their way while these are worked on.  Staged rows have two
// places a team, or one for h and dy in turn; the next ones are copied as soon as they have been read.
// A team takes `group` neighbouring rows (R, or R = 1 at a time), then the group that is a step away.
template <int kType, int V, int R, bool kParts, bool kFused, bool kPlain>
__global__ void __launch_bounds__(kMaxTeam)
norm_backward_rows_kernel(const BackwardArgs<kType> a, int team, int group, const BackwardSteps step, int hist_words, int sum_words,
                          int slots) {
    constexpr bool kStaged = !kPlain && kType == QFMT_F32;
    constexpr bool kAhead = (kPlain && V <= 2) || (!kPlain && !kStaged && V == 1);
    constexpr int kLanes = backward_hist_lanes(kType, V);
    extern __shared__ __align__(16) uint32_t dynamic[];  // [hist_words] histogram, [sum_words] the block's column sums, places for rows
    __shared__ __align__(16) float scratch[kParts ? 1 : kMaxTeam / 64][2][64];
    grid_launch_dependents();
    grid_dependency_wait();
    uint32_t* hist = !kPlain && a.stats != nullptr ? dynamic : nullptr;
    if constexpr (!kParts) {
        for (int i = threadIdx.x; i < kMaxTeam * 2; i += blockDim.x) (&scratch[0][0][0])[i] = 0.0f;
        __syncthreads();
    }
    if (hist != nullptr) clear_hist<kLanes>(hist, a.quant);
    // (the shuffle tells the compiler that a warp belongs to one team)
    const int mine = V > 2 ? 0 : kParts ? threadIdx.x / team : __shfl_sync(0xFFFFFFFFu, threadIdx.x / team, 0);
    const int t = threadIdx.x - mine * team, teams = V > 2 ? 1 : blockDim.x / team;
    const bool from = (t & 31) != 0, after = (t & 31) != 31 && t + 1 < team;
    const uint64_t offset = kFused ? drop_offset(a.drop) : 0ull;
    const int next = team * kGranule;  // elements between a thread's granules
    int n[V];
    Granule w[V <= 3 ? V : 1], dw = splat(0.0f), db = splat(0.0f);  // the sums with V = 1
    float4* const sums_in_shared = reinterpret_cast<float4*>(dynamic + hist_words) + (V == 2 ? mine * V * 4 * team : 0);  // with V > 1: [teams][V][4][team]
#pragma unroll
    for (int k = 0; k < V; ++k) {
        n[k] = granule_columns(a.cols, k * team + t);
        if (V > 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sums_in_shared[(4 * k + i) * team + t] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    }
    const uint32_t rows = (uint32_t)a.rows, stride = gridDim.x * teams * group;
    uint32_t row = (blockIdx.x * teams + mine) * group;
    const auto* pdy = a.dy.p + row * a.dy.ld + (kStaged ? 0 : t * kGranule);
    const auto* ph = a.h.p + row * a.h.ld + (kStaged ? 0 : t * kGranule);
    GradientRow<kType> to(a, row, t * kGranule);
    OnItsWay<kType, kPlain || kStaged> raw_dy[R][V], raw_h[R][V];
    float mean[R], rstd[R];
    const auto fetch_rows = [&](uint32_t at) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool there = at + i < rows;
            mean[i] = there ? a.mean[at + i] : 0.0f;
            rstd[i] = there ? a.rstd[at + i] : 0.0f;
            if constexpr (!kStaged) {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const bool edge = at_edge(a.cols, k * team + t);
                    raw_dy[i][k] = start<kType, kPlain>(pdy + i * a.dy.ld + k * next, n[k], at + i, rows, edge, a.inner);
                    raw_h[i][k] = start<kType, kPlain>(ph + i * a.h.ld + k * next, n[k], at + i, rows, edge, a.inner);
                }
            }
        }
    };
    const uint32_t row_bytes = staged_row_bytes(a.cols);
    const uint32_t places = shared_address(dynamic + hist_words + sum_words) + mine * slots * row_bytes;
    const auto stage = [&](uint32_t at, uint32_t place, const auto* p) {
        if constexpr (kStaged) if (at < rows) stage_row(place, p, (int)a.cols, t, team);
    };
    const auto arrived = [&]() {  // every thread's copies, for the whole team
        if constexpr (V > 2) __syncthreads();
        else if constexpr (kParts) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(team) : "memory");
    };
    // rows to the next one: a step, or with R = 1 one row within a group
    const bool pairs = R == 1 && group == 2;
    const auto advance = [&](bool second, auto*& p, int64_t ld, int64_t by) { p += pairs ? (second ? by - ld : ld) : by; };
    if (kAhead) fetch_rows(row);
    [[maybe_unused]] int skew_h = 0, skew_dy = 0;
    const auto stage_next = [&](uint32_t at) {
        if constexpr (kStaged) {
            skew_h = row_skew(ph), skew_dy = row_skew(pdy);
            stage(at, places, ph);
            if (slots == 2) stage(at, places + row_bytes, pdy);
            stage_end();
        }
    };
    stage_next(row);
#pragma unroll
    for (int k = 0; k < (V <= 3 ? V : 0); ++k) w[k] = load_columns(a.weight, k * team + t, n[k], 1.0f);
    int parity = 0;
    bool second = false;
    for (uint32_t first = blockIdx.x * teams * group; first < rows; parity ^= 1) {  // the row of the block's first team
        const uint32_t by = pairs ? (second ? stride - 1 : 1) : stride;
        if (!kAhead) fetch_rows(row);
        if constexpr (kStaged) {
            const bool there = row < rows;
            stage_wait();
            arrived();
#pragma unroll
            for (int k = 0; k < V; ++k) raw_h[0][k] = staged_granule(places, skew_h, k * team + t, there ? n[k] : 0);
            if (slots == 1) {
                arrived();  // h has been read by everyone
                stage(row, places, pdy);
                stage_end();
                stage_wait();
                arrived();
            }
            const uint32_t place = slots == 2 ? places + row_bytes : places;
#pragma unroll
            for (int k = 0; k < V; ++k) raw_dy[0][k] = staged_granule(place, skew_dy, k * team + t, there ? n[k] : 0);
        }
        Granule dy[R][V], xhat[R][V];
        float2 s[R];
        float this_rstd[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            this_rstd[i] = rstd[i];
            s[i] = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int there = row + i < rows ? n[k] : 0;  // a row that does not exist adds nothing to the column sums
                const Raw<kType> ds = words<kType, kPlain || kStaged>(raw_dy[i][k], pdy + i * a.dy.ld + k * next, there);
                const Raw<kType> hs = words<kType, kPlain || kStaged>(raw_h[i][k], ph + i * a.h.ld + k * next, there);
                dy[i][k] = widen_raw<kType>(ds);
                xhat[i][k] = normalise<kPlain>(widen_raw<kType>(hs), mean[i], rstd[i], there);
                if (V > 3) w[0] = load_columns(a.weight, k * team + t, n[k], 1.0f);
                s[i] = add2(s[i], row_sums(dy[i][k], xhat[i][k], w[V <= 3 ? k : 0]));
                if constexpr (V == 1) {
                    add_columns(dw, db, dy[i][k], xhat[i][k]);
                } else {
                    float4* const q = sums_in_shared + 4 * k * team + t;
                    Granule u = from_quads(q[0], q[team]), v = from_quads(q[2 * team], q[3 * team]);
                    add_columns(u, v, dy[i][k], xhat[i][k]);
                    q[0] = quad(u, 0), q[team] = quad(u, 1), q[2 * team] = quad(v, 0), q[3 * team] = quad(v, 1);
                }
            }
        }
        advance(second, pdy, a.dy.ld, step.dy);
        advance(second, ph, a.h.ld, step.h);
        if (kAhead) fetch_rows(row + by);
        if constexpr (kParts) {
            for (int off = team >> 1; off > 0; off >>= 1) {
#pragma unroll
                for (int i = 0; i < R; ++i) s[i] = make_float2(across(s[i].x, off), across(s[i].y, off));
            }
        } else {
            team_sums<R>(s, team, t, 1 + mine, scratch[mine][parity]);
        }
        if (kParts) __syncwarp();
        stage_next(row + by);  // behind the sums' barrier: everyone has read the places
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float c1 = s[i].x * a.inverse, c2 = s[i].y * a.inverse;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (V > 3) w[0] = load_columns(a.weight, k * team + t, n[k], 1.0f);
                store_gradients<kType, kFused, kPlain, kLanes>(a, to, i, k * next, dy[i][k], xhat[i][k], w[V <= 3 ? k : 0], this_rstd[i], c1, c2,
                                                               row + i, k * team + t, row + i < rows ? n[k] : 0, from, after, offset, hist);
            }
        }
        advance(second, to.dh, a.dh.ld, step.dh);
        advance(second, to.dx, a.dx.ld, step.dx);
        advance(second, to.dresidual, a.dresidual.ld, step.dresidual);
        row += by;
        first += by;
        second = pairs && !second;
    }
    if (hist != nullptr) flush_hist<kLanes>(hist, a.quant, a.stats, (uint64_t)a.rows * (uint64_t)a.cols);
    const bool alone = a.dweight != nullptr || a.dbias != nullptr;  // this block's part is the result
    if (kStaged) stage_wait();
    if (a.partial == nullptr) return;
    // [dweight, dbias][padded columns]
    const int padded = ((int)a.cols + kGranule - 1) / kGranule * kGranule, quads = padded / 2;
    float4* const part = reinterpret_cast<float4*>(a.partial) + (int64_t)blockIdx.x * quads;
    if constexpr (V > 1) {  // the sum of every team's
        __syncthreads();
        const float4* const sums = reinterpret_cast<const float4*>(dynamic + hist_words);
        for (int i = threadIdx.x; i < V * 4 * team; i += blockDim.x) {
            const int g = i / (4 * team) * team + i % team, which = i / team % 4;
            if (g >= padded / kGranule) continue;
            float4 s = sums[i];
            for (int u = 1; u < teams; ++u) s = sum_of(s, sums[u * V * 4 * team + i]);
            const int at = g * 2 + (which & 1) + (which >= 2 ? quads / 2 : 0);
            if (alone) put_columns(at, s, padded, (int)a.cols, a.dweight, a.dbias);
            else part[at] = s;
        }
        return;
    }
    // that of every warp of small teams, or of every team; then their sum
    const int units = kParts ? blockDim.x / 32 : teams;
    float4* const sums = units > 1 ? reinterpret_cast<float4*>(dynamic + hist_words) : part;
    float4* const own = sums + (kParts ? threadIdx.x / 32 : mine) * quads;
    if constexpr (kParts) {
        for (int off = 16; off >= team; off >>= 1) {  // the teams of a warp
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dw.p[j] = make_float2(across(dw.p[j].x, off), across(dw.p[j].y, off));
                db.p[j] = make_float2(across(db.p[j].x, off), across(db.p[j].y, off));
            }
        }
    }
    if (!(kParts && (threadIdx.x & 31) >= team) && n[0] != 0) {
        float4* const q = own + t * 2;
        q[0] = quad(dw, 0), q[1] = quad(dw, 1);
        q[quads / 2] = quad(db, 0), q[quads / 2 + 1] = quad(db, 1);
    }
    if (units == 1 && !alone) return;
    __syncthreads();
    for (int i = threadIdx.x; i < quads; i += blockDim.x) {
        float4 s = sums[i];
        for (int u = 1; u < units; ++u) s = sum_of(s, sums[u * quads + i]);
        if (alone) put_columns(i, s, padded, (int)a.cols, a.dweight, a.dbias);
        else part[i] = s;
    }
}

// Joins the parts in a fixed order: a block takes 128 columns of dweight and dbias side by side, its warps every 32nd
// part, four columns a lane.  148 parts of 1024 columns are 1.2 MB that lie in L2: what it takes (3 us behind the rows
// kernel) is its launch and two dependent reads; one column a lane took 17 us instead of 10 at 16384 columns.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps)
norm_join_parts_kernel(const float4* partial, int parts, int64_t padded, int64_t cols, float* dweight, float* dbias) {
    __shared__ float4 sums[kJoinWarps][32];
    grid_launch_dependents();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t quads = (uint32_t)(padded / 2), q = blockIdx.x * 32 + lane;  // at most 2^30
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (q < quads) {
        const float4* p = partial + (int64_t)warp * quads + q;
        const int64_t step = (int64_t)kJoinWarps * quads;
#pragma unroll 5
        for (int k = warp; k < parts; k += kJoinWarps, p += step) s = sum_of(s, *p);
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (threadIdx.x >= 128) return;
    float u = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) u += reinterpret_cast<const float*>(sums[w])[threadIdx.x];
    const JoinedColumn at = joined_column((int64_t)blockIdx.x * 128 + threadIdx.x, padded);
    float* const out = at.second ? dbias : dweight;
    if (out != nullptr && at.c < cols) out[at.c] = u;
}

// One granule a thread; two and more, teams half as large, beyond 1280 columns where there are enough rows (16 a block of
// containers, 32 of codes) and it pays: with containers (fused: unless the larger teams fill 512 threads), with codes where the
// larger teams leave three eighths of 512 without work (2049 to 2560 columns).  dx and the sums / fused, two granules against
// one, us: fp32 16384 x 1536 50 against 57 / 72 against 75, x 2048 63 against 68 / 97 against 89, x 2560 78 against 110 / 118
// against 145, ragged x 2556 121 against 198 / 159 against 202, x 3496 109 against 134 / 157 against 175, x 4096 120 against 143
// / 190 against 187, 3000 x 2560 20 against 27 / 25 against 33.  bfloat16 16384 x 2560 53 against 62 / 67 against 75, ragged
// x 2556 113 against 131 / 185 against 161 (registers spill).  Where the rule keeps one, in L2: fp32 16384 x 1024 36 against 36 / 49
// against 46, 2048 x 2560 13.7 against 12.8 / 16.4 against 18.3, 400 x 2560 8.1 against 7.6 / 8.9 against 8.3; bfloat16 9899 x 2816
// 41.7 against 40.1 / 52 against 50, 16384 x 4096 79 against 77 / 100 against 99, 2000 x 2560 11.4 against 10.4 / 14.6 against 13.9.
constexpr int kMaxParts = 148;  // the blocks of the rows kernel, one on each of a B200's SMs
Plan backward_plan(const qfmt_norm_t& s, bool fused) {
    const Plan one = make_plan(s.cols, 1, 4);
    if (one.granules != 1 || one.team <= 160) return one;
    const int used = kMaxTeam / one.team * one.team;
    const bool containers = s.dtype == QFMT_F32;
    const bool pays = containers ? !fused || used < kMaxTeam : used <= kMaxTeam - 3 * kMaxTeam / 8;
    return pays && s.rows >= (containers ? 16 : 32) * kMaxParts ? make_plan(s.cols, 2, 4) : one;
}

// Parts that the backward pass leaves for the gradients of weight and bias: one per block of the rows kernel, or a
// share of the rows for long rows.
int row_parts(const qfmt_norm_t& s) {
    if (backward_plan(s, false).team != 0) return kMaxParts;  // more than the loop would need
    const int64_t want = (s.rows + 8 * kColumnWarps - 1) / (8 * kColumnWarps);
    return (int)(want < 64 ? (want > 0 ? want : 1) : 64);
}

int64_t padded_columns(int64_t cols) { return (cols + kGranule - 1) / kGranule * kGranule; }

int join_parts(const float* partial, int parts, int64_t cols, float* d_dweight, float* d_dbias, cudaStream_t stream) {
    const int64_t padded = padded_columns(cols);
    QFMT_CUDA_TRY(launch_overlapping(norm_join_parts_kernel, (unsigned)((2 * padded + 127) / 128), 32u * kJoinWarps, 0, stream,
                                     reinterpret_cast<const float4*>(partial), parts, padded, cols, d_dweight, d_dbias));
    return QFMT_OK;
}

// Shared memory for the column sums of a block of the backward pass.
size_t backward_sum_bytes(int v, bool parts, int team, int64_t cols) {
    if (v > 1) return (size_t)(kMaxTeam / team) * team * v * 64;
    const int units = parts ? kMaxTeam / team * team / 32 : kMaxTeam / team;
    return units > 1 ? 2 * sizeof(float) * (size_t)padded_columns(cols) * units : 0;
}

template <int kType, int V, int R, bool kParts, bool kFused, bool kPlain>
int launch_backward_rows(const Call& c, BackwardArgs<kType> a, int team, int group, int blocks, float* d_dweight, float* d_dbias,
                         cudaStream_t stream) {
    const int teams = kMaxTeam / team, block = teams * team;
    const bool alone = a.partial != nullptr && blocks == 1;
    if (alone) a.dweight = d_dweight, a.dbias = d_dbias;
    const auto kern = norm_backward_rows_kernel<kType, V, R, kParts, kFused, kPlain>;
    constexpr bool kStaged = !kPlain && kType == QFMT_F32;
    const size_t place = (size_t)teams * staged_row_bytes(a.cols), hist = c.hist_bytes / kHistLanes * backward_hist_lanes(kType, V);
    const size_t sums = backward_sum_bytes(V, kParts, team, a.cols), rest = hist + sums;
    const int slots = !kStaged ? 0 : rest + 2 * place <= kMostShared ? 2 : 1;
    // More than half of what an SM has: its one block must not be joined by a second of the same launch, which would
    // leave another SM without work (launches overlap, so SMs come free at different times).
    const size_t smem = std::max(rest + slots * place, (size_t)116 * 1024);
    static std::atomic<bool> allowed[64];
    const int rc = allow_shared(kern, kMostShared, c.dev, allowed);
    if (rc != QFMT_OK) return rc;
    const int64_t stride = (int64_t)blocks * teams * group;
    const BackwardSteps step = {stride * a.dy.ld, stride * a.h.ld, stride * a.dh.ld, stride * a.dx.ld, stride * a.dresidual.ld};
    QFMT_CUDA_TRY(launch_overlapping(kern, blocks, block, smem, stream, a, team, group, step, (int)(hist / 4), (int)(sums / 4), slots));
    return a.partial != nullptr && !alone ? join_parts(a.partial, (int)blocks, a.cols, d_dweight, d_dbias, stream) : QFMT_OK;
}

template <int kType, bool kFused>
int launch_backward(const Call& c, const BackwardArgs<kType>& a, float* d_dweight, float* d_dbias, cudaStream_t stream) {
    if (a.rows == 0) return join_parts(a.partial, 0, a.cols, d_dweight, d_dbias, stream);  // zeros
    const Plan plan = backward_plan(c.norm, kFused);
    const bool plain = plain_layout(a.cols, {a.dy.whole, a.dh.whole, a.h.whole, a.dx.whole, a.dresidual.whole}) && !a.fmt;
    if (plan.team != 0) {
        // Two neighbouring rows to a team where every team gets some: a rule on sizes alone, since it decides the order
        // of the sums over rows.  Whether the two are worked on at once does not.
        // So is a single block where that takes one turn of pairs, or two of narrow rows: its part is the result, and no
        // second kernel runs (8 rows of 1024 fp32 3.6 us against 4.1 in a graph; 16 rows 4.7 against 4.2, bfloat16 3.9 against 4.0, but
        // 6.1 against 8.7 when calls are launched one by one; four turns would take 5.5).
        const int teams = kMaxTeam / plan.team, cap = std::min(c.dev.sm_count, kMaxParts);
        const bool few = plan.granules == 1 && a.partial != nullptr && a.rows <= (plan.team <= 128 ? 4 : 2) * teams;
        const int group = plan.granules == 1 && (few || a.rows > 2 * ((int64_t)teams * cap - 1)) ? 2 : 1;
        // With one granule as few blocks as take no more turns, so fewer parts are joined (in L2: 5000 x 256 bfloat16 6.6 -> 5.8 us,
        // 700 x 2048 6.9 -> 6.5, 400 x 4096 fp32 9.0 -> 8.7, 8192 x 1024 bfloat16 11.0 -> 11.2, wide rows mixed: 331 x 8192 11.4 ->
        // 11.8; from memory 6.5 -> 6.4, 9.1 -> 9.0, 10.2 -> 10.4, 14.0 -> 14.0).
        const int64_t units = (a.rows + (int64_t)teams * group - 1) / ((int64_t)teams * group);
        const int64_t turns = plan.granules == 1 ? (units + cap - 1) / cap : 1;
        const int blocks = few ? 1 : (int)std::min<int64_t>((units + turns - 1) / turns, cap);
        const auto run = plan.granules == 3   ? (plain ? launch_backward_rows<kType, 3, 1, false, kFused, true>
                                                       : launch_backward_rows<kType, 3, 1, false, kFused, false>)
                         : plan.granules == 4 ? (plain ? launch_backward_rows<kType, 4, 1, false, kFused, true>
                                                       : launch_backward_rows<kType, 4, 1, false, kFused, false>)
                         : plan.granules == 2 ? (plain ? launch_backward_rows<kType, 2, 1, false, kFused, true>
                                                       : launch_backward_rows<kType, 2, 1, false, kFused, false>)
                         : plan.team > 32   ? (!plain       ? launch_backward_rows<kType, 1, 1, false, kFused, false>
                                               : group == 2 ? launch_backward_rows<kType, 1, 2, false, kFused, true>
                                                            : launch_backward_rows<kType, 1, 1, false, kFused, true>)
                                            : (!plain       ? launch_backward_rows<kType, 1, 1, true, kFused, false>
                                               : group == 2 ? launch_backward_rows<kType, 1, 2, true, kFused, true>
                                                            : launch_backward_rows<kType, 1, 1, true, kFused, true>);
        return run(c, a, plan.team, group, blocks, d_dweight, d_dbias, stream);
    }
    if (a.partial != nullptr) {  // before the row pass, which may overwrite dy
        const int parts = row_parts(c.norm);
        const dim3 grid((unsigned)((a.cols + 32 * kGranule - 1) / (32 * kGranule)), (unsigned)parts);
        norm_column_sums_kernel<kType><<<grid, 32 * kColumnWarps, 0, stream>>>(a);
        QFMT_CUDA_TRY(cudaGetLastError());
        const int rc = join_parts(a.partial, parts, a.cols, d_dweight, d_dbias, stream);
        if (rc != QFMT_OK) return rc;
    }
    if (a.dx.p != nullptr || a.dresidual.p != nullptr) {
        const int64_t cap = (int64_t)c.dev.sm_count * 4;
        norm_backward_loop_kernel<kType, kFused><<<(unsigned)(a.rows < cap ? a.rows : cap), kLoopThreads, c.hist_bytes, stream>>>(a);
        QFMT_CUDA_TRY(cudaGetLastError());
    }
    return QFMT_OK;
}

template <int kType, bool kFused>
int backward(const Call& c, const void* d_dy, const void* d_dh, const void* d_h, int64_t ld_h, const float* d_mean,
             const float* d_rstd, const float* d_weight, void* d_dx, void* d_dresidual, float* d_dweight, float* d_dbias,
             qfmt_stats_t* d_stats, float* partial, cudaStream_t stream) {
    const qfmt_norm_t& s = c.norm;
    BackwardArgs<kType> a;
    a.dy = make_source<kType>(d_dy, s.ld_dy);
    a.dh = make_source<kType>(d_dh, s.ld_dh);
    a.h = make_source<kType>(d_h, ld_h);
    a.mean = d_mean;
    a.rstd = d_rstd;
    a.weight = d_weight;
    a.dx = make_target<kType>(d_dx, s.ld_dx);
    a.dresidual = make_target<kType>(d_dresidual, s.ld_dresidual);
    a.partial = partial;
    a.dweight = a.dbias = nullptr;
    a.rows = s.rows;
    a.cols = s.cols;
    a.inner = inner_rows(s.cols, s.rows);
    a.inverse = 1.0f / (float)a.cols;
    a.fmt = c.fmt;
    a.drop = c.drop;
    a.quant = c.quant;
    a.stats = d_stats;
    return launch_backward<kType, kFused>(c, a, d_dweight, d_dbias, stream);
}

int backward_entry(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, bool fused, const void* d_dy, const void* d_dh,
                   const void* d_h, const float* d_mean, const float* d_rstd, const float* d_weight, void* d_dx,
                   void* d_dresidual, float* d_dweight, float* d_dbias, const qfmt_format_t* fmt, qfmt_stats_t* d_stats,
                   int accumulate, void* d_workspace, size_t workspace_bytes, cudaStream_t stream) {
    Call c;
    int rc = prepare_call(norm, drop, fmt, d_stats, accumulate, &c);
    if (rc != QFMT_OK) return rc;
    const int32_t t = c.norm.dtype;
    const bool empty = c.norm.rows == 0 || c.norm.cols == 0;
    const bool columns = (d_dweight != nullptr || d_dbias != nullptr) && c.norm.cols != 0;
    if (!empty && (d_dy == nullptr || d_h == nullptr || d_mean == nullptr || d_rstd == nullptr)) return QFMT_ERR_BAD_ARG;
    if (d_stats != nullptr && d_dx == nullptr && !empty) return QFMT_ERR_BAD_ARG;  // the record is dx's
    if (!element_aligned(d_dy, t) || !element_aligned(d_dh, t) || !element_aligned(d_h, t) || !element_aligned(d_dx, t) ||
        !element_aligned(d_dresidual, t) || !float_aligned(d_mean) || !float_aligned(d_rstd) || !float_aligned(d_weight) ||
        !float_aligned(d_dweight) || !float_aligned(d_dbias))
        return QFMT_ERR_BAD_ARG;
    if (!empty && d_dx != nullptr && d_dx == d_dresidual) return QFMT_ERR_BAD_ARG;
    if (columns && (d_workspace == nullptr || (reinterpret_cast<uintptr_t>(d_workspace) & 15u) ||
                    workspace_bytes < qfmt_layer_norm_workspace_bytes(norm)))
        return QFMT_ERR_BAD_ARG;
    rc = current_device(&c.dev);
    if (rc != QFMT_OK) return rc;
    if (d_stats != nullptr && accumulate == 0)
        QFMT_CUDA_TRY(launch_overlapping(zero_words_kernel, 1u, 256u, 0, stream, reinterpret_cast<int*>(d_stats),
                                         (int)(sizeof(qfmt_stats_t) / sizeof(int))));
    if (c.norm.cols == 0 || (empty && !columns)) return QFMT_OK;
    const int64_t ld_h = fused ? c.norm.ld_h : c.norm.ld_x;
    const auto run = fused ? (t == QFMT_F32 ? backward<QFMT_F32, true> : t == QFMT_F16 ? backward<QFMT_F16, true> : backward<QFMT_BF16, true>)
                           : (t == QFMT_F32 ? backward<QFMT_F32, false> : t == QFMT_F16 ? backward<QFMT_F16, false> : backward<QFMT_BF16, false>);
    return run(c, d_dy, d_dh, d_h, ld_h, d_mean, d_rstd, d_weight, d_dx, d_dresidual, d_dweight, d_dbias, d_stats,
               columns ? static_cast<float*>(d_workspace) : nullptr, stream);
}

}  // namespace
}  // namespace qfmt

extern "C" size_t qfmt_layer_norm_workspace_bytes(const qfmt_norm_t* norm) {
    if (norm == nullptr || norm->rows < 0 || norm->cols < 0 || norm->rows > 0x7FFFFFFF || norm->cols > 0x7FFFFFFF) return 0;
    return (size_t)qfmt::row_parts(*norm) * 2 * (size_t)qfmt::padded_columns(norm->cols) * sizeof(float);
}

extern "C" int qfmt_layer_norm_backward(const qfmt_norm_t* norm, const void* d_dy, const void* d_x, const float* d_mean,
                                        const float* d_rstd, const float* d_weight, void* d_dx, float* d_dweight,
                                        float* d_dbias, const qfmt_format_t* fmt, qfmt_stats_t* d_stats, int accumulate,
                                        void* d_workspace, size_t workspace_bytes, void* stream) {
    return qfmt::backward_entry(norm, nullptr, false, d_dy, nullptr, d_x, d_mean, d_rstd, d_weight, d_dx, nullptr, d_dweight,
                                d_dbias, fmt, d_stats, accumulate, d_workspace, workspace_bytes, (cudaStream_t)stream);
}

extern "C" int qfmt_dropout_add_layer_norm_backward(const qfmt_norm_t* norm, const qfmt_dropout_t* drop, const void* d_dy,
                                                    const void* d_dh, const void* d_h, const float* d_mean,
                                                    const float* d_rstd, const float* d_weight, void* d_dx, void* d_dresidual,
                                                    float* d_dweight, float* d_dbias, const qfmt_format_t* fmt,
                                                    qfmt_stats_t* d_stats, int accumulate, void* d_workspace,
                                                    size_t workspace_bytes, void* stream) {
    return qfmt::backward_entry(norm, drop, true, d_dy, d_dh, d_h, d_mean, d_rstd, d_weight, d_dx, d_dresidual, d_dweight, d_dbias,
                                fmt, d_stats, accumulate, d_workspace, workspace_bytes, (cudaStream_t)stream);
}
