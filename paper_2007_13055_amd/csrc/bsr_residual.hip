// The norms around a block, with its gate and the residual's scales:
//
//     b = post(B)      S' = beta S + alpha gate b      U = pre(S')
//
// post and pre: none, x / sqrt(mean(x^2) + eps), or (x - mean) / sqrt(var + eps), times a weight, plus a bias.  U is taken of
// S' before its rounding.  And the gradient: with g = GS + pre'(GU) the gradient of S',
//
//     dS = beta g      t = alpha gate g      dB = post'(t)
//     norm'(G) = r (Gw - mean(Gw) - x r c),  x the (centred) input, r = 1 / sqrt(mean(x^2) + eps), Gw = G weight,
//                c = r mean(Gw x); without the mean of Gw for the root mean square
//     sums over the rows: of GU x r and GU (pre's weight and bias), alpha g post(B) (gate), t x r and t (post's)
//
// Work split: T lanes share a row, eight neighbouring columns a lane (T = 8 to 64: several rows a wavefront; 128 to 512: a
// workgroup a row), two or four runs of eight where a row has more than 4096, so a row is read once and stays in registers through
// its norms.  A workgroup walks over rows and keeps the five vectors' parts -- and in the backward pass the five sums -- of its
// columns in registers, with the next row's reads under way while one is summed.  Not so in rows of more than 4096 columns, whose
// registers hold one row alone: the forward pass reads the vectors again in every row (7400 x 9683 f16 with all five: 293 us, a
// copy's time is 110), and the backward pass keeps 1 to 190 of its registers in memory.  Its sums are written once, and a second
// launch adds the workgroups' in a fixed order (no atomics: the same bits every time).  In the backward pass the sums of more than
// 8192 columns do not fit a workgroup's registers: one launch makes the rows' means and a second, eight columns a lane, the
// gradients from them.
#include <algorithm>

#include "bsr_rows.h"

using namespace bsr_dev;

namespace {

constexpr int V = 8;                                  // neighbouring columns of a lane
constexpr int kMostCols = 16384;
constexpr int kMostSummed = 8192;                     // columns of a row whose sums the gradient's kernel keeps in registers
constexpr int kSums = 5;                              // post's weight and bias, gate, pre's weight and bias
constexpr int kStats = 8;                             // floats a row that the two-launch gradient passes on

struct norm_args {
    int post, pre;
    const void* vec[kSums];
    float eps, alpha, beta, over_n;                   // over_n = 1 / n
};

constexpr int kMostAtOnce = 4;                        // values a call adds: the areas' size
// T lanes' sums of N values; `slots`: two areas of kMostAtOnce floats a wavefront, used in turn by the calls of a workgroup (of
// one size whatever N is: a call that takes fewer must not reach into the area of the call before, which may still be read).
template <int T, int N> struct row_sums {
    static constexpr int WAVES = T > 64 ? T / 64 : 1;
    static_assert(N <= kMostAtOnce, "an area holds them");
    __device__ __forceinline__ static void add(float (&v)[N], float* slots, int& phase)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lane_sum<(T > 64 ? 64 : T)>(v[i]);
        if constexpr (T > 64) {
            float* const at = slots + phase * (WAVES * kMostAtOnce);
            phase ^= 1;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) at[(threadIdx.x >> 6) * N + i] = v[i];
            }
            __syncthreads();                          // (who writes this area next has passed the other area's barrier, behind these reads)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += at[w * N + i];
        }
    }
};

// 1 / sqrt(mean_square + eps): the instruction's, which is up to 2^-22 off, and a Newton step (gradients of rows of a few columns
// cancel to a small part of their terms).  A sum of 0 or infinity keeps the instruction's.
__device__ __forceinline__ float inverse_root(float mean_square, float eps)
{
    const float v = mean_square + eps, r = __builtin_amdgcn_rsqf(v), off = fmaf(-(v * r), r, 1.f);
    return fabsf(off) < 1.f ? fmaf(0.5f * r, off, r) : r;
}

template <typename WT> __device__ __forceinline__ void load_vec(any_run<WT, V>& r, const void* p, int col, int count, float absent)
{
    if (p) {
        r.load(static_cast<const WT*>(p) + col, count);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) r.set(e, absent);
    }
}

// Rows of K runs a lane.  ST: S's type, XT: B's and U's, WT: the vectors'.
template <typename ST, typename XT, typename WT, int T, int K>
__global__ __launch_bounds__(T <= 64 ? 256 : T) void bsr_norm_rows(const ST* S, const XT* B, ST* S_out, XT* U, int m, int n, int per, norm_args a)
{
    constexpr int TEAMS = T <= 64 ? 256 / T : 1;
    __shared__ float slots[T > 64 ? 2 * (T / 64) * kMostAtOnce : 1];
    int phase = 0;
    const int t = (int)threadIdx.x % T, team = (int)threadIdx.x / T;
    int col[K], count[K];
    any_run<WT, V> wp[K], bp[K], gate[K], wq[K], bq[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        col[j] = (t + T * j) * V;
        count[j] = max(n - col[j], 0);
        if (count[j] == 0) col[j] = 0;
    }
    auto vectors = [&](int j) {
        load_vec<WT>(wp[j], a.vec[0], col[j], count[j], 1.f);
        load_vec<WT>(bp[j], a.vec[1], col[j], count[j], 0.f);
        load_vec<WT>(gate[j], a.vec[2], col[j], count[j], 1.f);
        load_vec<WT>(wq[j], a.vec[3], col[j], count[j], 1.f);
        load_vec<WT>(bq[j], a.vec[4], col[j], count[j], 0.f);
    };
    if constexpr (K == 1) vectors(0);
    any_run<ST, V> s_in[K];
    any_run<XT, V> b_in[K];
    const int first = ((int)blockIdx.x * per) * TEAMS + team;
    auto fetch = [&](int i) {                         // of a row behind the last one: nothing
        const size_t row = (size_t)min(i, m - 1) * (size_t)n;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int there = i < m ? count[j] : 0;
            s_in[j].load(S + row + col[j], there);
            if (B) b_in[j].load(B + row + col[j], there);
        }
    };
    constexpr bool kAhead = K == 1;                   // (longer rows' registers hold one row)
    if (kAhead) fetch(first);
    for (int q = 0; q < per; ++q) {
        const int i = first + q * TEAMS;
        if (!kAhead) fetch(i);
        float s[K][V], b[K][V];
#pragma unroll
        for (int j = 0; j < K; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                s[j][e] = a.beta * s_in[j][e];
                b[j][e] = B ? b_in[j][e] : 0.f;
            }
        if (kAhead && q + 1 < per) fetch(i + TEAMS);
        // x - mean, or x; elements behind the row's end stay zeros
        auto centre = [&](float (&x)[K][V]) {
            float sum[1] = {0.f};
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[0] += x[j][e];
            row_sums<T, 1>::add(sum, slots, phase);
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) x[j][e] = e < count[j] ? x[j][e] - sum[0] * a.over_n : 0.f;
        };
        auto root = [&](const float (&x)[K][V]) {
            float sum[1] = {0.f};
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[0] = fmaf(x[j][e], x[j][e], sum[0]);
            row_sums<T, 1>::add(sum, slots, phase);
            return inverse_root(sum[0] * a.over_n, a.eps);
        };
        if (B) {
            float r = 1.f;
            if (a.post == BSR_NORM_LAYER) centre(b);
            if (a.post != BSR_NORM_NONE) r = root(b);
#pragma unroll
            for (int j = 0; j < K; ++j) {
                if constexpr (K > 1) vectors(j);
#pragma unroll
                for (int e = 0; e < V; ++e) s[j][e] = fmaf(a.alpha * gate[j][e], fmaf(b[j][e] * r, wp[j][e], bp[j][e]), s[j][e]);
            }
        }
        const size_t row = (size_t)i * (size_t)n;
        if (S_out && i < m)
#pragma unroll
            for (int j = 0; j < K; ++j) {
                any_run<ST, V> out;
#pragma unroll
                for (int e = 0; e < V; ++e) out.set(e, s[j][e]);
                out.store(S_out + row + col[j], count[j]);
            }
        if (!U) continue;
#pragma unroll
        for (int j = 0; j < K; ++j)                   // (a bias has filled what is behind the end)
#pragma unroll
            for (int e = 0; e < V; ++e) s[j][e] = e < count[j] ? s[j][e] : 0.f;
        if (a.pre == BSR_NORM_LAYER) centre(s);
        const float r = root(s);
        if (i < m)
#pragma unroll
            for (int j = 0; j < K; ++j) {
                any_run<XT, V> out;
                if constexpr (K > 1) {
                    load_vec<WT>(wq[j], a.vec[3], col[j], count[j], 1.f);
                    load_vec<WT>(bq[j], a.vec[4], col[j], count[j], 0.f);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) out.set(e, fmaf(s[j][e] * r, wq[j][e], bq[j][e]));
                out.store(U + row + col[j], count[j]);
            }
    }
}

// What the gradients of a row's columns are made of.
struct row_stats { float mean, r, c, shift; };        // of the input; r and c as above; shift: mean of Gw (layer norm)

// A product; PIN: rounded wherever it is taken, so that what a mean subtracts is what the mean was made of: a row of one column
// has a layer norm's gradient of exactly 0, rows of a few lose no more than the formulas do.  (Not in rows of more than 4096 columns,
// whose sums have no such cancellation and whose registers are short: pinned products wait there, in memory, from one use to the next.
// 12598 x 6886 bf16, fp32 weights 564 us pinned, 429 not; 4096 x 8192 fp32 335, 232; 4096 x 12288 bf16 445, 359.)
template <bool PIN> __device__ __forceinline__ float rounded_product(float a, float b)
{
    float p = a * b;
    if constexpr (PIN) asm("" : "+v"(p));
    return p;
}
// The gradient of S' in one column, from gw = GU weight.
template <bool PIN> __device__ __forceinline__ float sum_gradient(const norm_args& a, const row_stats& pre, float x, float gw, float gs)
{
    if (a.pre == BSR_NORM_NONE) return gs;
    if constexpr (PIN) return fmaf(pre.r, fmaf(-rounded_product<PIN>(x - pre.mean, pre.r), pre.c, gw - pre.shift), gs);
    return fmaf(pre.r, fmaf(-(x - pre.mean), pre.r * pre.c, gw - pre.shift), gs);
}

// One column's part: from x, GU, GS, b to g, dS, dB and what the five sums get.
struct column_parts { float ds, db, sum[kSums]; };
template <bool PIN>
__device__ __forceinline__ column_parts column_gradient(const norm_args& a, const row_stats& pre, const row_stats& post, float x, float gu, float gs,
                                                        float b, float wp, float bp, float gate, float wq)
{
    column_parts out;
    const float xm = x - pre.mean;
    const float g = sum_gradient<PIN>(a, pre, x, rounded_product<PIN>(gu, wq), gs);
    out.sum[3] = gu * (xm * pre.r);
    out.sum[4] = gu;
    out.ds = a.beta * g;
    const float bh = rounded_product<PIN>(b - post.mean, post.r), ag = rounded_product<PIN>(a.alpha, g);
    out.sum[2] = ag * fmaf(bh, wp, bp);
    const float t = rounded_product<PIN>(ag, gate);
    out.sum[0] = t * bh;
    out.sum[1] = t;
    out.db = a.post == BSR_NORM_NONE ? t : post.r * fmaf(-bh, post.c, rounded_product<PIN>(t, wp) - post.shift);
    return out;
}

// The backward pass.  K < 4: all of it; `partial`: [workgroups][sums wanted][n].  K == 4: the rows' means alone, into `stats`.
struct grad_ptrs { int at[kSums]; };                  // place of each sum among those wanted, -1: not wanted
template <typename ST, typename XT, typename WT, int T, int K>
__global__ __launch_bounds__(T <= 64 ? 256 : T) void bsr_norm_grad_rows(const ST* S, const XT* B, const ST* GS, const XT* GU, ST* DS, XT* DB,
                                                                        float* __restrict__ partial, float* __restrict__ stats, int m, int n, int per,
                                                                        int wanted, grad_ptrs place, norm_args a)
{
    constexpr int BLOCK = T <= 64 ? 256 : T, TEAMS = BLOCK / T;
    __shared__ float slots[T > 64 ? 2 * (T / 64) * kMostAtOnce : 1];
    __shared__ float red[TEAMS > 1 ? BLOCK * V : 1];
    constexpr bool kAll = K < 4, PIN = K == 1;
    int phase = 0;
    const int t = (int)threadIdx.x % T, team = (int)threadIdx.x / T;
    int col[K], count[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        col[j] = (t + T * j) * V;
        count[j] = max(n - col[j], 0);
        if (count[j] == 0) col[j] = 0;
    }
    any_run<WT, V> wp[K], bp[K], gate[K], wq[K];
    auto vectors = [&](int j) {
        load_vec<WT>(wp[j], a.vec[0], col[j], count[j], 1.f);
        load_vec<WT>(bp[j], a.vec[1], col[j], count[j], 0.f);
        load_vec<WT>(gate[j], a.vec[2], col[j], count[j], 1.f);
        load_vec<WT>(wq[j], a.vec[3], col[j], count[j], 1.f);
    };
#pragma unroll
    for (int j = 0; j < K; ++j) vectors(j);
    float sum[kSums][kAll ? K : 1][V];
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int j = 0; j < (kAll ? K : 1); ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[k][j][e] = 0.f;
    any_run<ST, V> s_in[K], gs_in[K];
    any_run<XT, V> b_in[K], gu_in[K];
    const int first = ((int)blockIdx.x * per) * TEAMS + team;
    auto fetch = [&](int i) {
        const size_t row = (size_t)min(i, m - 1) * (size_t)n;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int there = i < m ? count[j] : 0;
            const size_t at = row + (size_t)col[j];
            // (null: zeros)
            s_in[j].load(S + at, S ? there : 0);
            b_in[j].load(B + at, B ? there : 0);
            gs_in[j].load(GS + at, GS ? there : 0);
            gu_in[j].load(GU + at, GU ? there : 0);
        }
    };
    constexpr bool kAhead = K == 1;
    if (kAhead) fetch(first);
    for (int q = 0; q < per; ++q) {
        const int i = first + q * TEAMS;
        if (!kAhead) fetch(i);
        any_run<ST, V> x[K], gs[K];
        any_run<XT, V> b[K], gu[K];
#pragma unroll
        for (int j = 0; j < K; ++j) { x[j] = s_in[j]; gs[j] = gs_in[j]; b[j] = b_in[j]; gu[j] = gu_in[j]; }
        if (kAhead && q + 1 < per) fetch(i + TEAMS);
        row_stats pre{0.f, 0.f, 0.f, 0.f}, post{0.f, 1.f, 0.f, 0.f};
        auto each = [&](auto f) {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) f(j, e);
        };
        if (a.pre == BSR_NORM_LAYER || a.post == BSR_NORM_LAYER) {
            float v[2] = {0.f, 0.f};
            each([&](int j, int e) { v[0] += x[j][e]; v[1] += b[j][e]; });
            row_sums<T, 2>::add(v, slots, phase);
            if (a.pre == BSR_NORM_LAYER) pre.mean = v[0] * a.over_n;
            if (a.post == BSR_NORM_LAYER) post.mean = v[1] * a.over_n;
        }
        if (a.pre != BSR_NORM_NONE || a.post != BSR_NORM_NONE) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            each([&](int j, int e) {
                const bool there = e < count[j];
                const float xm = there ? x[j][e] - pre.mean : 0.f, bm = there ? b[j][e] - post.mean : 0.f, gw = rounded_product<PIN>(gu[j][e], wq[j][e]);
                v[0] = fmaf(xm, xm, v[0]);
                v[1] = fmaf(gw, xm, v[1]);
                v[2] += gw;
                v[3] = fmaf(bm, bm, v[3]);
            });
            row_sums<T, 4>::add(v, slots, phase);
            if (a.pre != BSR_NORM_NONE) {
                pre.r = inverse_root(v[0] * a.over_n, a.eps);
                pre.c = pre.r * (v[1] * a.over_n);
                if (a.pre == BSR_NORM_LAYER) pre.shift = v[2] * a.over_n;
            }
            if (a.post != BSR_NORM_NONE) post.r = inverse_root(v[3] * a.over_n, a.eps);
        }
        if (a.post != BSR_NORM_NONE) {
            float v[2] = {0.f, 0.f};
            each([&](int j, int e) {
                const bool there = e < count[j];
                const float bm = there ? b[j][e] - post.mean : 0.f;
                const float g = sum_gradient<PIN>(a, pre, x[j][e], rounded_product<PIN>(gu[j][e], wq[j][e]), gs[j][e]);
                const float gw = there ? rounded_product<PIN>(rounded_product<PIN>(rounded_product<PIN>(a.alpha, g), gate[j][e]), wp[j][e]) : 0.f;
                v[0] = fmaf(gw, bm, v[0]);
                v[1] += gw;
            });
            row_sums<T, 2>::add(v, slots, phase);
            post.c = post.r * (v[0] * a.over_n);
            if (a.post == BSR_NORM_LAYER) post.shift = v[1] * a.over_n;
        }
        if constexpr (!kAll) {
            if (t == 0 && i < m) {
                float* const to = stats + (size_t)i * kStats;
                to[0] = pre.mean; to[1] = pre.r; to[2] = pre.c; to[3] = pre.shift;
                to[4] = post.mean; to[5] = post.r; to[6] = post.c; to[7] = post.shift;
            }
        } else {
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const size_t at = (size_t)i * (size_t)n + (size_t)col[j];
                const int there = i < m ? count[j] : 0;
                any_run<ST, V> ds;
                any_run<XT, V> db;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const column_parts p =
                        column_gradient<PIN>(a, pre, post, x[j][e], gu[j][e], gs[j][e], b[j][e], wp[j][e], bp[j][e], gate[j][e], wq[j][e]);
                    ds.set(e, p.ds);
                    db.set(e, p.db);
#pragma unroll
                    for (int k = 0; k < kSums; ++k) sum[k][j][e] += i < m ? p.sum[k] : 0.f;
                }
                if (DS && there) ds.store(DS + at, there);
                if (DB && there) db.store(DB + at, there);
            }
        }
    }
    if constexpr (kAll) {
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            if (place.at[k] < 0) continue;            // uniform
            float* const out = partial + ((size_t)blockIdx.x * (size_t)wanted + (size_t)place.at[k]) * (size_t)n;
            if constexpr (TEAMS > 1) {                // the teams' sums, in their order
                __syncthreads();
#pragma unroll
                for (int e = 0; e < V; ++e) red[threadIdx.x * V + e] = sum[k][0][e];
                __syncthreads();
                if (team == 0 && count[0] > 0)
                    for (int e = 0; e < V && e < count[0]; ++e) {
                        float v = 0.f;
                        for (int w = 0; w < TEAMS; ++w) v += red[(w * T + t) * V + e];
                        out[col[0] + e] = v;
                    }
            } else {
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    any_run<float, V> v;
#pragma unroll
                    for (int e = 0; e < V; ++e) v.v[e] = sum[k][j][e];
                    if (count[j] > 0) v.store(out + col[j], count[j]);
                }
            }
        }
    }
}

// The gradients of rows whose means are known: a lane takes eight columns down the rows of its chunk.
template <typename ST, typename XT, typename WT>
__global__ __launch_bounds__(256) void bsr_norm_grad_cols(const ST* S, const XT* B, const ST* GS, const XT* GU, ST* DS, XT* DB, float* __restrict__ partial,
                                                          const float* __restrict__ stats, int m, int n, int rows, int wanted, grad_ptrs place, norm_args a)
{
    const int col = (int)(blockIdx.x * 256 + threadIdx.x) * V, count = n - col;
    if (count <= 0) return;
    any_run<WT, V> wp, bp, gate, wq;
    load_vec<WT>(wp, a.vec[0], col, count, 1.f);
    load_vec<WT>(bp, a.vec[1], col, count, 0.f);
    load_vec<WT>(gate, a.vec[2], col, count, 1.f);
    load_vec<WT>(wq, a.vec[3], col, count, 1.f);
    float sum[kSums][V];
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[k][e] = 0.f;
    const int first = (int)blockIdx.y * rows, end = min(first + rows, m);
    for (int i = first; i < end; ++i) {
        const float* const from = stats + (size_t)i * kStats;
        const row_stats pre{from[0], from[1], from[2], from[3]}, post{from[4], from[5], from[6], from[7]};
        const size_t at = (size_t)i * (size_t)n + (size_t)col;
        any_run<ST, V> x, gs, ds;
        any_run<XT, V> b, gu, db;
        x.load(S + at, S ? count : 0);
        b.load(B + at, B ? count : 0);
        gs.load(GS + at, GS ? count : 0);
        gu.load(GU + at, GU ? count : 0);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const column_parts p = column_gradient<false>(a, pre, post, x[e], gu[e], gs[e], b[e], wp[e], bp[e], gate[e], wq[e]);
            ds.set(e, p.ds);
            db.set(e, p.db);
#pragma unroll
            for (int k = 0; k < kSums; ++k) sum[k][e] += p.sum[k];
        }
        if (DS) ds.store(DS + at, count);
        if (DB) db.store(DB + at, count);
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (place.at[k] < 0) continue;
        any_run<float, V> v;
#pragma unroll
        for (int e = 0; e < V; ++e) v.v[e] = sum[k][e];
        v.store(partial + ((size_t)blockIdx.y * (size_t)wanted + (size_t)place.at[k]) * (size_t)n + (size_t)col, count);
    }
}

// out[k][j] = sum of partial[c][k][j] over the workgroups c: 16 columns a workgroup, 16 shares of them.
struct sum_outputs { float* to[kSums]; };
__global__ __launch_bounds__(256) void bsr_norm_sums(const float* __restrict__ partial, sum_outputs out, int n, int chunks, int wanted)
{
    __shared__ float red[16][16];
    const int at = threadIdx.x % 16, share = threadIdx.x / 16, col = (int)blockIdx.x * 16 + at;
    const size_t step = (size_t)wanted * (size_t)n;
    const float* const from = partial + (size_t)blockIdx.y * (size_t)n + (size_t)col;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (col < n) {
        int c = share;
        for (; c + 48 < chunks; c += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += from[(size_t)(c + 16 * u) * step];
        for (; c < chunks; c += 16) v[0] += from[(size_t)c * step];
    }
    red[share][at] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (share == 0 && col < n) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 4) s += (red[i][at] + red[i + 1][at]) + (red[i + 2][at] + red[i + 3][at]);
        out.to[blockIdx.y][col] = s;
    }
}

// How rows are shared out.
struct row_split {
    int t;                                            // lanes of a row
    int runs;                                         // of eight columns a lane: 1, 2 or 4
    int per;                                          // rows that a team walks over
    int groups;                                       // workgroups
};
row_split split_rows(int64_t m, int64_t n, int most_groups)
{
    row_split s{8, 1, 1, 1};
    while (s.t < 512 && (int64_t)s.t * V < n) s.t *= 2;
    while ((int64_t)s.t * V * s.runs < n) s.runs *= 2;
    const int64_t teams = s.t <= 64 ? 256 / s.t : 1;
    const int64_t all = (m + teams - 1) / teams;
    s.per = (int)std::max<int64_t>((all + most_groups - 1) / most_groups, 1);
    s.groups = (int)((all + s.per - 1) / s.per);
    return s;
}
// Workgroups of a launch: as many as the CUs hold at once, so that each walks over as many rows as there are.
int most_groups_forward(int64_t n) { return n <= 2048 ? 2048 : 1024; }
int most_groups_backward(int64_t n) { return n <= 2048 ? 1024 : 512; }

constexpr int kChunks = 256;                          // of rows, in the column pass
struct column_split { int rows, chunks; };
column_split split_columns(int64_t m)
{
    const int64_t rows = std::max<int64_t>((m + kChunks - 1) / kChunks, 4);
    return {(int)rows, (int)((m + rows - 1) / rows)};
}

bool sizes_fit(int64_t m, int64_t n) { return m >= 0 && n >= 0 && m < ((int64_t)1 << 30) && n <= kMostCols; }
size_t round_up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
size_t stats_bytes(int64_t m, int64_t n) { return n > kMostSummed ? round_up((size_t)m * kStats * sizeof(float)) : 0; }
size_t partial_bytes(int64_t m, int64_t n, int wanted)
{
    const int chunks = n > kMostSummed ? split_columns(m).chunks : split_rows(m, n, most_groups_backward(n)).groups;
    return round_up((size_t)chunks * (size_t)wanted * (size_t)n * sizeof(float));
}
size_t size_of(bsr_dtype t) { return t == BSR_F32 ? 4 : 2; }
bool known(bsr_dtype t) { return (int)t >= (int)BSR_F32 && (int)t <= (int)BSR_BF16; }
bool known_norm(bsr_norm k) { return (int)k >= (int)BSR_NORM_NONE && (int)k <= (int)BSR_NORM_LAYER; }

// Calls f(lanes of a row, runs) with the split's as constants.
template <typename F> bsr_status with_team(const row_split& s, F f)
{
    using std::integral_constant;
    switch (s.t) {
        case 8: return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
        case 16: return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
        case 32: return f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
        case 64: return f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
        case 128: return f(integral_constant<int, 128>{}, integral_constant<int, 1>{});
        case 256: return f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    }
    if (s.runs == 1) return f(integral_constant<int, 512>{}, integral_constant<int, 1>{});
    if (s.runs == 2) return f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    return f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
}
// Calls f(S's type, B's, the vectors').
template <typename F> bsr_status with_types(bsr_dtype s, bsr_dtype x, bsr_dtype w, F f)
{
    auto vectors = [&](auto st, auto xt) {
        if (w == BSR_F32) return f(st, xt, 0.f);
        return f(st, xt, xt);
    };
    if (x == BSR_F32) return f(0.f, 0.f, 0.f);
    if (x == BSR_F16) return s == BSR_F32 ? vectors(0.f, f16_t{}) : vectors(f16_t{}, f16_t{});
    return s == BSR_F32 ? vectors(0.f, bf16_t{}) : vectors(bf16_t{}, bf16_t{});
}

bsr_status launched() { return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP; }

bsr_status check_how(int64_t m, int64_t n, bsr_dtype s_dtype, bsr_dtype b_dtype, const bsr_residual* how)
{
    if (!how) return BSR_ERR_NULL;
    if (!sizes_fit(m, n)) return BSR_ERR_SHAPE;
    if (!known(s_dtype) || !known(b_dtype) || (s_dtype != b_dtype && s_dtype != BSR_F32) || !known_norm(how->post) || !known_norm(how->pre) ||
        (how->w_dtype != b_dtype && how->w_dtype != BSR_F32)) return BSR_ERR_DTYPE;
    if (!(how->eps >= 0)) return BSR_ERR_SHAPE;       // (NaN too)
    for (const void* p : {how->post_weight_dev, how->post_bias_dev, how->gate_dev, how->pre_weight_dev, how->pre_bias_dev})
        if (!aligned16(p)) return BSR_ERR_ALIGN;
    return BSR_OK;
}

norm_args args_of(const bsr_residual& h, int64_t n, bool branch)
{
    norm_args a{};
    a.post = branch ? h.post : BSR_NORM_NONE;
    a.pre = h.pre;
    if (a.post != BSR_NORM_NONE) { a.vec[0] = h.post_weight_dev; a.vec[1] = h.post_bias_dev; }
    if (branch) a.vec[2] = h.gate_dev;
    if (a.pre != BSR_NORM_NONE) { a.vec[3] = h.pre_weight_dev; a.vec[4] = h.pre_bias_dev; }
    a.eps = (float)h.eps;
    a.alpha = h.branch_scale;
    a.beta = h.stream_scale;
    a.over_n = (float)(1.0 / (double)n);
    return a;
}

// Whether `out` lies over one of the inputs, but for the places it may take (null: none).
bool covers(const byte_range& out, std::initializer_list<byte_range> in, const void* in_place0 = nullptr, const void* in_place1 = nullptr)
{
    for (const byte_range& r : in)
        if (overlap(out, r) && !(out.p == r.p && out.bytes == r.bytes && (out.p == in_place0 || out.p == in_place1))) return true;
    return false;
}

}  // namespace

extern "C" {

bsr_status bsr_residual_norm(int64_t m, int64_t n, bsr_dtype s_dtype, const void* S_dev, bsr_dtype b_dtype, const void* B_dev, void* S_out_dev,
                             void* U_dev, const bsr_residual* how, void* hip_stream)
{
    const bsr_status st = check_how(m, n, s_dtype, b_dtype, how);
    if (st != BSR_OK) return st;
    if (m == 0 || n == 0) return BSR_OK;
    if (!S_dev || (!S_out_dev && !U_dev)) return BSR_ERR_NULL;
    if (U_dev && how->pre == BSR_NORM_NONE) return BSR_ERR_UNSUPPORTED;
    for (const void* p : {S_dev, B_dev, (const void*)S_out_dev, (const void*)U_dev})
        if (!aligned16(p)) return BSR_ERR_ALIGN;
    const size_t elements = (size_t)m * (size_t)n, w = (size_t)n * size_of(how->w_dtype);
    const byte_range s{S_dev, elements * size_of(s_dtype)}, b{B_dev, elements * size_of(b_dtype)}, s_out{S_out_dev, elements * size_of(s_dtype)},
        u{U_dev, elements * size_of(b_dtype)};
    const byte_range vec[kSums] = {{how->post_weight_dev, w}, {how->post_bias_dev, w}, {how->gate_dev, w}, {how->pre_weight_dev, w}, {how->pre_bias_dev, w}};
    if (overlap(s_out, u) || covers(s_out, {s, b}, S_dev) || covers(u, {s, b}, B_dev)) return BSR_ERR_OVERLAP;
    for (const byte_range& r : vec)
        if (overlap(s_out, r) || overlap(u, r)) return BSR_ERR_OVERLAP;
    const norm_args a = args_of(*how, n, B_dev != nullptr);
    const row_split split = split_rows(m, n, most_groups_forward(n));
    return with_types(s_dtype, b_dtype, how->w_dtype, [&](auto s_type, auto x_type, auto w_type) {
        typedef decltype(s_type) ST;
        typedef decltype(x_type) XT;
        typedef decltype(w_type) WT;
        return with_team(split, [&](auto team, auto runs) {
            constexpr int T = decltype(team)::value, K = decltype(runs)::value;
            hipLaunchKernelGGL((bsr_norm_rows<ST, XT, WT, T, K>), dim3((unsigned)split.groups), dim3(T <= 64 ? 256 : T), 0, (hipStream_t)hip_stream,
                               (const ST*)S_dev, (const XT*)B_dev, (ST*)S_out_dev, (XT*)U_dev, (int)m, (int)n, split.per, a);
            return launched();
        });
    });
}

bsr_status bsr_residual_norm_backward_workspace_size(int64_t m, int64_t n, size_t* bytes)
{
    if (!bytes) return BSR_ERR_NULL;
    *bytes = 0;
    if (!sizes_fit(m, n)) return BSR_ERR_SHAPE;
    if (m > 0 && n > 0) *bytes = stats_bytes(m, n) + partial_bytes(m, n, kSums);
    return BSR_OK;
}

bsr_status bsr_residual_norm_backward(int64_t m, int64_t n, bsr_dtype s_dtype, const void* S_dev, bsr_dtype b_dtype, const void* B_dev,
                                      const void* GS_dev, const void* GU_dev, void* DS_dev, void* DB_dev, const bsr_residual* how,
                                      const bsr_residual_grads* grads, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    const bsr_status st = check_how(m, n, s_dtype, b_dtype, how);
    if (st != BSR_OK) return st;
    if (n == 0) return BSR_OK;
    const bool branch = B_dev != nullptr || m == 0;
    const bsr_residual_grads none{};
    const bsr_residual_grads& g = grads ? *grads : none;
    float* const to[kSums] = {g.post_weight_dev, g.post_bias_dev, g.gate_dev, g.pre_weight_dev, g.pre_bias_dev};
    if ((!branch && (to[0] || to[1] || to[2] || DB_dev)) || (how->post == BSR_NORM_NONE && (to[0] || to[1])) ||
        (how->pre == BSR_NORM_NONE && (to[3] || to[4] || GU_dev))) return BSR_ERR_UNSUPPORTED;
    sum_outputs out{};
    grad_ptrs place;
    int wanted = 0;
    for (int k = 0; k < kSums; ++k) {
        place.at[k] = to[k] ? wanted : -1;
        if (to[k]) out.to[wanted++] = to[k];
    }
    for (const void* p : {S_dev, B_dev, GS_dev, GU_dev, (const void*)DS_dev, (const void*)DB_dev, (const void*)to[0], (const void*)to[1], (const void*)to[2],
                          (const void*)to[3], (const void*)to[4], (const void*)workspace_dev})
        if (!aligned16(p)) return BSR_ERR_ALIGN;
    hipStream_t stream = (hipStream_t)hip_stream;
    if (m > 0 && !S_dev && how->pre != BSR_NORM_NONE) return BSR_ERR_NULL;
    if (!DS_dev && !DB_dev && !wanted) return BSR_ERR_NULL;
    const size_t vector = (size_t)n * sizeof(float), w = (size_t)n * size_of(how->w_dtype), elements = (size_t)m * (size_t)n;
    const size_t need = m > 0 ? stats_bytes(m, n) + (wanted ? partial_bytes(m, n, wanted) : 0) : 0;
    if (need && (stats_bytes(m, n) || wanted) && (!workspace_dev || workspace_bytes < need)) return BSR_ERR_WORKSPACE;
    const byte_range s{how->pre != BSR_NORM_NONE ? S_dev : nullptr, elements * size_of(s_dtype)}, b{B_dev, elements * size_of(b_dtype)},
        gs{GS_dev, elements * size_of(s_dtype)}, gu{GU_dev, elements * size_of(b_dtype)}, ds{DS_dev, elements * size_of(s_dtype)},
        db{DB_dev, elements * size_of(b_dtype)}, ws{need ? workspace_dev : nullptr, need};
    if (overlap(ds, db) || covers(ds, {s, b, gs, gu}, GS_dev, S_dev) || covers(db, {s, b, gs, gu}, GU_dev, B_dev)) return BSR_ERR_OVERLAP;
    const byte_range vec[kSums] = {{how->post_weight_dev, w}, {how->post_bias_dev, w}, {how->gate_dev, w}, {how->pre_weight_dev, w}, {how->pre_bias_dev, w}};
    for (const byte_range& r : vec)
        if (overlap(ds, r) || overlap(db, r) || overlap(ws, r)) return BSR_ERR_OVERLAP;
    for (int k = 0; k < kSums; ++k) {
        const byte_range mine{to[k], vector};
        for (const byte_range& r : {s, b, gs, gu, ds, db, ws, vec[0], vec[1], vec[2], vec[3], vec[4]})
            if (overlap(mine, r)) return BSR_ERR_OVERLAP;
        for (int other = 0; other < k; ++other)
            if (overlap(mine, {to[other], vector})) return BSR_ERR_OVERLAP;
    }
    for (const byte_range& r : {s, b, gs, gu, ds, db})
        if (overlap(ws, r)) return BSR_ERR_OVERLAP;
    float* const stats = static_cast<float*>(workspace_dev);
    float* const partial = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + stats_bytes(m, n));
    int chunks = 0;
    if (m > 0) {
        const norm_args a = args_of(*how, n, branch);
        const row_split split = split_rows(m, n, most_groups_backward(n));
        const column_split columns = split_columns(m);
        chunks = n > kMostSummed ? columns.chunks : split.groups;
        const void* const sum = how->pre != BSR_NORM_NONE ? S_dev : nullptr;
        const bsr_status done = with_types(s_dtype, b_dtype, how->w_dtype, [&](auto s_type, auto x_type, auto w_type) {
            typedef decltype(s_type) ST;
            typedef decltype(x_type) XT;
            typedef decltype(w_type) WT;
            const bsr_status rows = with_team(split, [&](auto team, auto runs) {
                constexpr int T = decltype(team)::value, K = decltype(runs)::value;
                hipLaunchKernelGGL((bsr_norm_grad_rows<ST, XT, WT, T, K>), dim3((unsigned)split.groups), dim3(T <= 64 ? 256 : T), 0, stream,
                                   (const ST*)sum, (const XT*)B_dev, (const ST*)GS_dev, (const XT*)GU_dev, (ST*)DS_dev, (XT*)DB_dev, partial, stats,
                                   (int)m, (int)n, split.per, wanted, place, a);
                return launched();
            });
            if (rows != BSR_OK || n <= kMostSummed) return rows;
            hipLaunchKernelGGL((bsr_norm_grad_cols<ST, XT, WT>), dim3((unsigned)((n + 256 * V - 1) / (256 * V)), (unsigned)columns.chunks), dim3(256), 0, stream,
                               (const ST*)sum, (const XT*)B_dev, (const ST*)GS_dev, (const XT*)GU_dev, (ST*)DS_dev, (XT*)DB_dev, partial, stats, (int)m,
                               (int)n, columns.rows, wanted, place, a);
            return launched();
        });
        if (done != BSR_OK) return done;
    }
    if (!wanted) return BSR_OK;
    hipLaunchKernelGGL(bsr_norm_sums, dim3((unsigned)((n + 15) / 16), (unsigned)wanted), dim3(256), 0, stream, partial, out, (int)n, chunks, wanted);
    return launched();
}

}  // extern "C"
