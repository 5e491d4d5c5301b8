// One step over the stored blocks of many matrices whose update is orthogonalised block by block:
//
//     M = mu M + g      V = g + mu M or M      X = V / (|V| + eps)
//     ns_steps times    X = a X + b (X X^T) X + c (X X^T)^2 X
//     p = p (1 - lr decay) - lr scale X        and the stored values of W^T
//
// A wavefront takes a block from its first read to its last write; between them the block stays in registers as 16x16 tiles of
// the matrix cores' results (lane l holds column l mod 16, rows 4 (l / 16) .. + 3), fp32, zeros where its sides end before a
// tile does (they stay zeros).  The steps are written with W, the block turned so that its longer side runs down the rows, L x S:
//     G = W^T W      P = b G + c G^2      W = a W + W P
// and fed without moving anything, because the order in which a product's terms are added is free: as terms 4h + e (h the lane's
// quarter, e = 0 .. 3) a lane's four result rows are its four operands.  G's two operands are both W's tiles as they are; G is
// symmetric, so that its tiles serve as either operand of G^2; P's tiles are W P's right operand.  Its left one is W^T's tiles,
// which W passes through LDS for, written once a step by columns and read back 16 bytes a lane; the wavefront's own area, no barrier.
//
// What bounds it (40 million elements, bf16 with a master copy, 805 MB; a large copy moves 5.2 bytes a ps): memory, beside it in
// 16x16 blocks the vector units (splitting into parts), in the largest blocks registers, which leave two wavefronts a SIMD to cover its
// latency; 64x64 blocks are 30 short of them, which wait in memory (100 bytes a lane; 900 where bs_c is no multiple of 4).  With 0
// and 5 steps, us: 16x16 147, 198; 32x32 158, 191; 64x32 165, 176 to 192; 64x64 215, 285.  (16x16 with products of fp32 numbers 235;
// 64x64, fp32 gradients and W^T's copy with it, 312, and 456 with products of three bf16 parts.)
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <stdexcept>

#include "bsr_optimizer.h"

using namespace bsr_dev;
using namespace bsr_list;

namespace {

constexpr int kMostSide = 64;
constexpr int kMostSteps = 16;

// A tensor as the kernels see it.
struct muon_desc {
    void* param;
    float* master;
    const void* grad;
    float* momentum;
    void* transposed;                                 // null: none
    const int32_t* place;                             // [blocks]: where each block's transpose goes
    int64_t blocks;
    float decay, scale;
    uint32_t number;                                  // in the caller's list
    int32_t bs_r, bs_c;
    int32_t dtype, grad_dtype;
    int32_t pad;
};
static_assert(sizeof(muon_desc) == 88, "uploaded as words");

struct muon_args {
    float lr, mu, eps, a, b, c, grad_scale;
    int32_t ns_steps, nesterov;
    int32_t small;                                    // the steps' numbers stay in fp16's range
    uint32_t key;                                     // of the seed and the step
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale_dev;
};

// Wavefronts of a workgroup, a block each: as many as 64 KB of LDS hold, four at most.
constexpr int waves_of(int rt, int ct) { return rt * ct > 8 ? 2 : 4; }

// Where four neighbouring elements of a lane are: `count` of them belong to the block, from `at` on.
struct run_at { size_t at; int count; };

// Tiles of a tensor of type T as fp32 numbers, zeros where a run ends.  All reads are under way before the first is used.  WHOLE: runs
// hold four elements or none, at a multiple of their size; `safe`: an element to read where there is none.
template <typename T, bool WHOLE, int CT, int RT, typename F>
__device__ __forceinline__ void load_runs(f32x4 (&v)[CT][RT], const void* p, size_t safe, F run_of)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    const T* const from = static_cast<const T*>(p);
    if constexpr (WHOLE) {
        t4 raw[CT][RT];
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) {
                const run_at r = run_of(J, I);
                raw[J][I] = *reinterpret_cast<const t4*>(from + (r.count >= 4 ? r.at : safe));
            }
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[J][I][e] = run_of(J, I).count >= 4 ? (float)raw[J][I][e] : 0.f;
    } else {
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const run_at r = run_of(J, I, e);
                    const float x = (float)from[r.count > 0 ? r.at : safe];
                    v[J][I][e] = r.count > 0 ? x : 0.f;
                }
    }
}
template <typename T, bool WHOLE, typename F> __device__ __forceinline__ void store_run4(T* to, const T (&v)[4], int J, int I, F run_of)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    if constexpr (WHOLE) {
        const run_at r = run_of(J, I);
        if (r.count >= 4) *reinterpret_cast<t4*>(to + r.at) = t4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const run_at r = run_of(J, I, e);
            if (r.count > 0) to[r.at] = v[e];
        }
    }
}

__device__ __forceinline__ double shared_sum(double v, int lane_xor)
{
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const int lo = __shfl_xor((int)(unsigned)u, lane_xor), hi = __shfl_xor((int)(unsigned)(u >> 32), lane_xor);
    return v + __builtin_bit_cast(double, (unsigned long long)(unsigned)lo | ((unsigned long long)(unsigned)hi << 32));
}

__device__ __forceinline__ bool finite_sum(double sum) { return sum - sum == 0.0; }
// held / (|V| + eps) from the sum of squares; NaN where V is not finite (an infinity's 0 would leave the block's other elements 0)
__device__ __forceinline__ float inverse_norm(double sum, float eps, float held)
{
    return (float)((double)held / (sqrt(sum + (sum - sum)) + (double)eps));
}

// fp32 products on the 16-bit matrix cores, which take a sixteenth of the time.  A lane's eight terms are those of two tiles, four each.
// F16: x = hi + lo, two fp16 numbers, to 2^-23 of x's power of two, and of the four products of two such sums the three largest (the
// fourth is below 2^-22 of hi hi); for numbers that are known to stay in fp16's range.  Else: x = hi + mid + lo, three bf16 numbers,
// exactly (8 of its 24 bits each), and of the nine products the six largest; the others are below 2^-26 of the whole.
template <bool F16> struct parts { u32x4 p[F16 ? 2 : 3]; };                  // the largest first
template <bool F16> __device__ __forceinline__ parts<F16> parts_of(const f32x4& a, const f32x4& b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    parts<F16> out;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f32x2 x = q < 2 ? f32x2{a[2 * q], a[2 * q + 1]} : f32x2{b[2 * q - 4], b[2 * q - 3]};
        if constexpr (F16) {
            const f16x2 hi = __builtin_convertvector(x, f16x2);
            float minus = -1.f;                       // (unknown to the compiler, which then takes one instruction that reads fp16)
            asm("" : "+s"(minus));
            const f32x2 rest = {fmaf((float)hi.x, minus, x.x), fmaf((float)hi.y, minus, x.y)};
            out.p[0][q] = __builtin_bit_cast(uint32_t, hi);
            out.p[1][q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, f16x2));
        } else {
#pragma unroll
            for (int part = 0; part < 3; ++part) {
                const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
                out.p[part][q] = w;
                if (part < 2) {
                    x.x -= __builtin_bit_cast(float, w << 16);
                    x.y -= __builtin_bit_cast(float, w & 0xFFFF0000u);
                }
            }
        }
    }
    return out;
}
// acc[t] += left^T right[t], the small products first
template <bool F16, int S> __device__ __forceinline__ void add_row(f32x4 (&acc)[S], const parts<F16>& left, const parts<F16> (&right)[S])
{
    auto add = [&](int u, int v) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < S; ++t) {
            if constexpr (F16)
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, left.p[u]), __builtin_bit_cast(f16x8, right[t].p[v]), acc[t], 0, 0, 0);
            else
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, left.p[u]), __builtin_bit_cast(bf16x8, right[t].p[v]), acc[t], 0, 0, 0);
        }
    };
    if constexpr (!F16) {
        add(2, 0);
        add(0, 2);
        add(1, 1);
    }
    add(1, 0);
    add(0, 1);
    add(0, 0);
}
// acc[s][t] += operand(s)^T operand(t)
template <bool F16, int R, int S, typename F> __device__ __forceinline__ void add_product(f32x4 (&acc)[R][S], F operand)
{
    parts<F16> x[S];
#pragma unroll
    for (int s = 0; s < S; ++s) x[s] = operand(s);
#pragma unroll
    for (int s = 0; s < R; ++s) add_row<F16, S>(acc[s], x[s], x);
}

// acc += left^T right for single tiles: as their fp16 parts fill half of the eight terms each, two instructions take all four products.
struct stacked { u32x4 both, hi, lo; };               // {hi, lo}, {hi, hi}, {lo, lo}
__device__ __forceinline__ stacked stacked_of(const f32x4& a)
{
    const parts<true> x = parts_of<true>(a, a);       // (the second half's arithmetic is the first's)
    return {u32x4{x.p[0][0], x.p[0][1], x.p[1][0], x.p[1][1]}, u32x4{x.p[0][0], x.p[0][1], x.p[0][0], x.p[0][1]},
            u32x4{x.p[1][0], x.p[1][1], x.p[1][0], x.p[1][1]}};
}
__device__ __forceinline__ void add_tile(f32x4& acc, const u32x4& left, const stacked& right)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, left), __builtin_bit_cast(f16x8, right.lo), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, left), __builtin_bit_cast(f16x8, right.hi), acc, 0, 0, 0);
}
// ... and in fp32.
__device__ __forceinline__ void add_tile(f32x4& acc, const f32x4& left, const f32x4& right)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(left[e], right[e], acc, 0, 0, 0);
}

// RT, CT: 16x16 tiles of a block down and across.  MODE: 0 a block a wavefront; where the smaller side is 8 at most, as many as fit
// 16 beside one another along it, 1 down (bs_r <= bs_c), 2 across: G then holds their products with one another, too, which are
// dropped, and P keeps them apart.  WHOLE: a lane's runs are four neighbouring elements of a block's row, or none.  F16: the steps'
// products are of fp16 parts, and W is held 64 times as large, G thus 4096 times, so that the small parts of theirs stay above fp16's
// smallest numbers; |X| <= 3.9 keeps them below the largest (stays_small()).
template <int RT, int CT, int MODE, bool WHOLE, bool F16>
__global__ __launch_bounds__(64 * waves_of(RT, CT), 2) void bsr_muon_blocks(const muon_desc* __restrict__ tensors, const int2* __restrict__ chunks, muon_args h)
{
    constexpr int WAVES = waves_of(RT, CT);
    constexpr bool TALL = RT > CT || MODE == 2;
    constexpr int L = TALL ? RT : CT, S = TALL ? CT : RT;
    static_assert(MODE == 0 || S == 1, "blocks beside one another fill one tile");
    constexpr float kHeld = F16 ? 64.f : 1.f;         // W's scale
    const float b = h.b / (kHeld * kHeld), c = h.c / (kHeld * kHeld * kHeld * kHeld);
    constexpr int PW = S * 16 + 4, PY = RT * 16 + 4;  // pitches in LDS of W [L * 16][], of the block's transpose [CT * 16][]
    constexpr int AREA = std::max(L * 16 * PW, CT * 16 * PY);
    __shared__ __attribute__((aligned(16))) float areas[WAVES][AREA];
    const int lane = threadIdx.x & 63, i = lane & 15, c0 = (lane >> 4) * 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int2 where = chunks[blockIdx.x];            // {tensor, first block}
    const muon_desc& d = tensors[where.x];
    const int bs_r = d.bs_r, bs_c = d.bs_c, size = bs_r * bs_c;
    const int small = MODE == 1 ? bs_r : bs_c, beside = MODE == 0 ? 1 : 16 / small;   // blocks of a wavefront
    const int64_t block0 = (int64_t)where.y + (int64_t)wave * beside;
    if (block0 >= d.blocks) return;                   // (no barrier below)
    const int here = (int)min((int64_t)beside, d.blocks - block0);
    float* const area = areas[wave];

    float lr = h.lr, grad_scale = h.grad_scale;
    uint32_t key = h.key;
    if (h.grad_scale_dev) {
        grad_scale = *h.grad_scale_dev;
        if (grad_scale == 0.f) return;                // the step is skipped
    }
    if (h.lr_dev) lr = *h.lr_dev;
    if (h.step_dev) {
        const int64_t t = *h.step_dev;
        if (t < 1) return;                            // no such step
        key = step_key(h.seed, (uint64_t)t);
    }

    const size_t first = (size_t)block0 * (size_t)size;
    // a lane's elements of tile (J, I): row 16 I + i, columns 16 J + c0 .. + 3, of the block or of the blocks beside one another
    const int mine = MODE == 1 ? i / bs_r : 0, row0 = MODE == 1 ? i - mine * bs_r : i;
    auto row_of = [&](int I) __attribute__((always_inline)) { return 16 * I + row0; };
    auto run_of = [&](int J, int I, int e = 0) __attribute__((always_inline)) {
        int b = mine, col = 16 * J + c0 + e;
        if constexpr (MODE == 2) {
            b = col / bs_c;
            col -= b * bs_c;
        }
        const bool there = row_of(I) < bs_r && b < here;
        return run_at{first + (size_t)(b * size + row_of(I) * bs_c + col), there ? bs_c - col : 0};
    };
    uint32_t mask = 0;                                // bit e: row c0 + e of G and this lane's column are of one block
    if constexpr (MODE != 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) mask |= (uint32_t)((c0 + e) / small == i / small) << e;

    f32x4 y[CT][RT];                                  // the block's transpose in result tiles
    auto read = [&](f32x4 (&v)[CT][RT], const void* p, int dtype) __attribute__((always_inline)) {   // dtype: uniform
        if (dtype == BSR_F32) load_runs<float, WHOLE>(v, p, first, run_of);
        else if (dtype == BSR_F16) load_runs<f16_t, WHOLE>(v, p, first, run_of);
        else load_runs<bf16_t, WHOLE>(v, p, first, run_of);
    };
    constexpr bool kEarly = RT * CT <= 4;             // the parameter is read with the rest; larger blocks' registers are full until the steps are done
    f32x4 param[CT][RT];
    auto read_param = [&]() __attribute__((always_inline)) {
        if (d.master) read(param, d.master, BSR_F32);
        else read(param, d.param, d.dtype);
    };
    {
        f32x4 m[CT][RT];
        read(m, d.momentum, BSR_F32);
        if (kEarly) read_param();
        read(y, d.grad, d.grad_dtype);
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) {
                float mv[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float g = y[J][I][e] * grad_scale;
                    mv[e] = fmaf(h.mu, m[J][I][e], g);
                    y[J][I][e] = h.nesterov ? fmaf(h.mu, mv[e], g) : mv[e];
                }
                store_run4<float, WHOLE>(d.momentum, mv, J, I, run_of);
            }
    }
    // A block that is not finite ends as NaN (by |V|, so that it does with no steps, too).  It takes no part in the steps of those
    // beside it, whose zeros its numbers would meet.
    uint32_t spoilt = 0;                              // bit e: column c0 + e is of such a block
    // |V|: squares and their sum in 64 bits, which hold those of any fp32 numbers
    {
        float over[4];                                // of the lane's four columns (MODE 2: they may be of four blocks)
        auto inverse = [&](double sum) { return inverse_norm(sum, h.eps, kHeld); };
        if constexpr (MODE == 2) {
            double* const sums = reinterpret_cast<double*>(area);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                double sum = 0.0;
#pragma unroll
                for (int I = 0; I < RT; ++I) sum += (double)y[0][I][e] * (double)y[0][I][e];
                for (int x = 1; x < 16; x *= 2) sum = shared_sum(sum, x);
                if (i == 0) sums[c0 + e] = sum;       // of column c0 + e
            }
            wave_lds_fence();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int b = (c0 + e) / bs_c;
                double sum = 0.0;
                if (b < here)
                    for (int q = 0; q < bs_c; ++q) sum += sums[b * bs_c + q];
                over[e] = inverse(sum);
                spoilt |= (uint32_t)!finite_sum(sum) << e;
            }
            wave_lds_fence();
        } else {
            double sum = 0.0;
#pragma unroll
            for (int J = 0; J < CT; ++J)
#pragma unroll
                for (int I = 0; I < RT; ++I)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum += (double)y[J][I][e] * (double)y[J][I][e];
            for (int x = MODE == 1 ? 16 : 1; x < 64; x *= 2) sum = shared_sum(sum, x);
            if constexpr (MODE == 1) {                // of row i so far
                double* const sums = reinterpret_cast<double*>(area);
                if (lane < 16) sums[i] = sum;
                wave_lds_fence();
                sum = 0.0;
                if (mine < here)
                    for (int q = 0; q < bs_r; ++q) sum += sums[mine * bs_r + q];
                wave_lds_fence();
                spoilt = finite_sum(sum) ? 0u : 15u;
            }
            over[0] = over[1] = over[2] = over[3] = inverse(sum);
        }
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[J][I][e] = MODE != 0 && ((spoilt >> e) & 1) ? 0.f : y[J][I][e] * over[e];
    }

    f32x4 w[L][S];
    auto put_y = [&]() __attribute__((always_inline)) {                              // and read turned_y: the tiles of its transpose
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) area[(16 * J + c0 + e) * PY + 16 * I + i] = y[J][I][e];
        wave_lds_fence();
    };
    auto turned_y = [&](int I, int J) __attribute__((always_inline)) { return *reinterpret_cast<const f32x4*>(&area[(16 * J + i) * PY + 16 * I + c0]); };
    if constexpr (TALL) {
        put_y();
#pragma unroll
        for (int I = 0; I < RT; ++I)
#pragma unroll
            for (int J = 0; J < CT; ++J) w[I][J] = turned_y(I, J);
    } else {
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) w[J][I] = y[J][I];
    }
    auto put_w = [&]() __attribute__((always_inline)) {
        wave_lds_fence();                             // the other lanes have read what was there
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) area[(16 * l + c0 + e) * PW + 16 * s + i] = w[l][s][e];
        wave_lds_fence();
    };
    auto turned = [&](int s, int l) __attribute__((always_inline)) { return *reinterpret_cast<const f32x4*>(&area[(16 * l + i) * PW + 16 * s + c0]); };   // tile (s, l) of W^T

    for (int step = 0; step < h.ns_steps; ++step) {
        put_w();
        f32x4 g[S][S], p[S][S];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int t = 0; t < S; ++t) g[s][t] = p[s][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (S == 1) {
            auto square = [&](f32x4& to, const f32x4& x) __attribute__((always_inline)) {
                if constexpr (F16) {
                    const stacked v = stacked_of(x);
                    add_tile(to, v.both, v);
                } else {
                    add_tile(to, x, x);
                }
            };
#pragma unroll
            for (int l = 0; l < L; ++l) square(g[0][0], w[l][0]);
            if constexpr (MODE != 0) {                // what is of two blocks is no part of either
#pragma unroll
                for (int e = 0; e < 4; ++e) g[0][0][e] = ((mask >> e) & 1) ? g[0][0][e] : 0.f;
            }
            square(p[0][0], g[0][0]);
        } else {
#pragma unroll
            for (int k = 0; k < L; k += 2) add_product<F16, S, S>(g, [&](int s) __attribute__((always_inline)) { return parts_of<F16>(w[k][s], k + 1 < L ? w[k + 1][s] : f32x4{}); });
#pragma unroll
            for (int k = 0; k < S; k += 2) add_product<F16, S, S>(p, [&](int s) __attribute__((always_inline)) { return parts_of<F16>(g[k][s], k + 1 < S ? g[k + 1][s] : f32x4{}); });
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int t = 0; t < S; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[s][t][e] = fmaf(b, g[s][t][e], c * p[s][t][e]);
        if constexpr (S == 1) {
            stacked right{};
            if constexpr (F16) right = stacked_of(p[0][0]);
#pragma unroll
            for (int l = 0; l < L; ++l) {
                const f32x4 wt = turned(0, l);
                w[l][0] *= h.a;
                if constexpr (F16) add_tile(w[l][0], stacked_of(wt).both, right);
                else add_tile(w[l][0], wt, p[0][0]);
            }
        } else {
            // (a W from LDS: its registers were G^2's in the meantime)
#pragma unroll
            for (int l = 0; l < L; ++l)
#pragma unroll
                for (int t = 0; t < S; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[l][t][e] = h.a * area[(16 * l + c0 + e) * PW + 16 * t + i];
#pragma unroll
            for (int k = 0; k < S; k += 2) {
                parts<F16> right[S];
#pragma unroll
                for (int t = 0; t < S; ++t) right[t] = parts_of<F16>(p[k][t], k + 1 < S ? p[k + 1][t] : f32x4{});
#pragma unroll
                for (int l = 0; l < L; ++l) {
                    const parts<F16> left = parts_of<F16>(turned(k, l), k + 1 < S ? turned(k + 1, l) : f32x4{});
                    add_row<F16, S>(w[l], left, right);
                }
            }
        }
    }
    if constexpr (TALL) {
        put_w();
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) y[J][I] = turned(J, I);
    } else {
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) y[J][I] = w[J][I];
    }

    if (MODE != 0 && spoilt)
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[J][I][e] = (spoilt >> e) & 1 ? __builtin_nanf("") : y[J][I][e];

    const float keep = 1.f - lr * d.decay, rate = lr * d.scale / kHeld;
    const uint32_t base = mix(d.number + key);
    // the transposed copy: its rows by way of LDS, four neighbouring elements a lane, where they are whole runs of a block
    const bool through = MODE != 2 && (bs_r & 3) == 0;
    auto update = [&](auto type, auto has_master) __attribute__((always_inline)) {
        typedef decltype(type) T;
        typedef T t4 __attribute__((ext_vector_type(4)));
        constexpr bool MASTER = decltype(has_master)::value;
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) {
                float v[4];
                T out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = fmaf(-rate, y[J][I][e], param[J][I][e] * keep);
                    asm("" : "+v"(v[e]));             // an fp32 number, of which the stored one is the rounding
                    if constexpr (MASTER || std::is_same<T, float>::value) out[e] = from_f32<T>(v[e]);
                    else out[e] = round_at_random(T{}, v[e], mix(base + (uint32_t)run_of(J, I, e).at));
                    y[J][I][e] = (float)out[e];
                }
                store_run4<T, WHOLE>(static_cast<T*>(d.param), out, J, I, run_of);
                if constexpr (MASTER) store_run4<float, WHOLE>(d.master, v, J, I, run_of);
            }
        if (!d.transposed) return;                    // uniform
        T* const t = static_cast<T*>(d.transposed);
        if (through) {
            wave_lds_fence();
            put_y();
#pragma unroll
            for (int J = 0; J < CT; ++J)
#pragma unroll
                for (int I = 0; I < RT; ++I) {
                    const f32x4 v = turned_y(I, J);
                    const int c = 16 * J + i, at = 16 * I + c0, b = MODE == 1 ? at / bs_r : 0, a = at - b * bs_r;
                    if (c < bs_c && a < bs_r && b < here)
                        *reinterpret_cast<t4*>(t + (size_t)d.place[block0 + b] * (size_t)size + (size_t)(c * bs_r + a)) =
                            t4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
                }
        } else {
#pragma unroll
            for (int J = 0; J < CT; ++J)
#pragma unroll
                for (int I = 0; I < RT; ++I)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int all = 16 * J + c0 + e, b = MODE == 2 ? all / bs_c : mine, c = MODE == 2 ? all - b * bs_c : all;
                        if (c < bs_c && row_of(I) < bs_r && b < here)
                            t[(size_t)d.place[block0 + b] * (size_t)size + (size_t)(c * bs_r + row_of(I))] = (T)y[J][I][e];
                    }
        }
    };
    if (!kEarly) read_param();
    auto update_type = [&](auto type) __attribute__((always_inline)) {
        if (d.master) update(type, std::true_type{});
        else update(type, std::false_type{});
    };
    if (d.dtype == BSR_F32) update(0.f, std::false_type{});
    else if (d.dtype == BSR_F16) update_type(f16_t{});
    else update_type(bf16_t{});
}

// The same for blocks of three and four tiles both ways, whose tiles are too many for a wavefront to hold with others beside it: a
// block a workgroup, row l of W's tiles wavefront l's.  Each of W, G and P is split into its fp16 parts once, by the wavefronts that
// have it, and read by all of them as operands from LDS, two regions in turn: between a region's reads and its next writes there
// is a barrier, and three barriers make a step.  What bounds it where there are many blocks is LDS, which a wavefront a block reads
// less of; where there are few it is the chain of a block.  fp32 64x64, us: 10 blocks 15.0, 1024 42, 2400 81 (a wavefront a block: 10
// of f16 with W^T 37.8, 1030 50, 2400 84); 9828 blocks of bf16 with a master copy 326 and 285.
template <int RT, int CT, bool WHOLE>
__global__ __launch_bounds__(64 * std::max(RT, CT), 3) void bsr_muon_team(const muon_desc* __restrict__ tensors, const int2* __restrict__ chunks, muon_args h)
{
    constexpr bool TALL = RT > CT;
    constexpr int L = TALL ? RT : CT, S = TALL ? CT : RT;
    constexpr int PITCH = S * 16 + 4;
    constexpr float kHeld = 64.f;                     // W's scale, as above
    const float b = h.b / (kHeld * kHeld), c = h.c / (kHeld * kHeld * kHeld * kHeld);
    __shared__ u32x4 operands[2][2][2][S][64];        // [region][hi, lo][two rows of tiles][column of tiles][lane]
    __shared__ __attribute__((aligned(16))) float areas[L][16 * PITCH];
    __shared__ double sums[L];
    const int lane = threadIdx.x & 63, i = lane & 15, c0 = (lane >> 4) * 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int PER = waves_of(RT, CT);             // blocks of a chunk
    const int2 where = chunks[blockIdx.x / PER];
    const muon_desc& d = tensors[where.x];
    const int bs_r = d.bs_r, bs_c = d.bs_c, size = bs_r * bs_c;
    const int64_t block = (int64_t)where.y + (int64_t)(blockIdx.x % PER);
    if (block >= d.blocks) return;                    // whole workgroup, as the returns below

    float lr = h.lr, grad_scale = h.grad_scale;
    uint32_t key = h.key;
    if (h.grad_scale_dev) {
        grad_scale = *h.grad_scale_dev;
        if (grad_scale == 0.f) return;
    }
    if (h.lr_dev) lr = *h.lr_dev;
    if (h.step_dev) {
        const int64_t t = *h.step_dev;
        if (t < 1) return;
        key = step_key(h.seed, (uint64_t)t);
    }

    // tile s of this wavefront's row of W: the block's rows 16 row_tile(s) + i, columns 16 col_tile(s) + c0 .. + 3 in a lane
    const size_t first = (size_t)block * (size_t)size;
    auto row_of = [&](int s) __attribute__((always_inline)) { return 16 * (TALL ? wave : s) + i; };
    auto col_of = [&](int s) __attribute__((always_inline)) { return 16 * (TALL ? s : wave) + c0; };
    auto run_of = [&](int s, int, int e = 0) __attribute__((always_inline)) {
        const int row = row_of(s), col = col_of(s) + e;
        return run_at{first + (size_t)(row * bs_c + col), row < bs_r ? bs_c - col : 0};
    };
    auto read = [&](f32x4 (&v)[S][1], const void* p, int dtype) __attribute__((always_inline)) {
        if (dtype == BSR_F32) load_runs<float, WHOLE>(v, p, first, run_of);
        else if (dtype == BSR_F16) load_runs<f16_t, WHOLE>(v, p, first, run_of);
        else load_runs<bf16_t, WHOLE>(v, p, first, run_of);
    };
    float* const area = areas[wave];
    // each tile's transpose, by way of the wavefront's own area
    auto turn = [&](f32x4 (&to)[S], const f32x4 (&v)[S]) __attribute__((always_inline)) {
        wave_lds_fence();
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) area[(c0 + e) * PITCH + 16 * s + i] = v[s][e];
        wave_lds_fence();
#pragma unroll
        for (int s = 0; s < S; ++s) to[s] = *reinterpret_cast<const f32x4*>(&area[i * PITCH + 16 * s + c0]);
    };
    auto barrier = []() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };   // (of LDS alone)

    f32x4 w[S], param[S][1];
    {
        f32x4 m[S][1], g[S][1];
        read(m, d.momentum, BSR_F32);
        if (d.master) read(param, d.master, BSR_F32);
        else read(param, d.param, d.dtype);
        read(g, d.grad, d.grad_dtype);
        double sum = 0.0;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float mv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = g[s][0][e] * grad_scale;
                mv[e] = fmaf(h.mu, m[s][0][e], x);
                w[s][e] = h.nesterov ? fmaf(h.mu, mv[e], x) : mv[e];
                sum += (double)w[s][e] * (double)w[s][e];
            }
            store_run4<float, WHOLE>(d.momentum, mv, s, 0, run_of);
        }
        for (int x = 1; x < 64; x *= 2) sum = shared_sum(sum, x);
        if (lane == 0) sums[wave] = sum;
        barrier();
        sum = 0.0;
#pragma unroll
        for (int l = 0; l < L; ++l) sum += sums[l];
        const float over = inverse_norm(sum, h.eps, kHeld);
#pragma unroll
        for (int s = 0; s < S; ++s) w[s] *= over;
    }
    if constexpr (TALL) turn(w, w);

    int region = 0;
    // This wavefront's row of tiles into the region that is next, of a matrix of `rows` rows of tiles (an odd last one with zeros).
    auto put = [&](const f32x4 (&v)[S], auto rows) __attribute__((always_inline)) {
        constexpr int R = decltype(rows)::value;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const parts<true> x = parts_of<true>(v[s], f32x4{});
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                u32x4* const at = &operands[region][part][wave >> 1][s][lane];
                if (R % 2 == 1 && wave == R - 1) *at = x.p[part];
                else reinterpret_cast<u32x2*>(at)[wave & 1] = u32x2{x.p[part][0], x.p[part][1]};
            }
        }
    };
    auto operand = [&](int k, int s) __attribute__((always_inline)) { return parts<true>{{operands[region][0][k][s][lane], operands[region][1][k][s][lane]}}; };
    // acc[t] += sum over the region's matrix's rows k of left(k)^T (its tile (k, t))
    auto add = [&](f32x4 (&acc)[S], auto rows, auto left) __attribute__((always_inline)) {
        constexpr int R = decltype(rows)::value;
#pragma unroll
        for (int k = 0; k < (R + 1) / 2; ++k) {
            parts<true> right[S];
#pragma unroll
            for (int t = 0; t < S; ++t) right[t] = operand(k, t);
            add_row<true, S>(acc, left(k), right);
        }
    };
    const std::integral_constant<int, L> l_rows{};
    const std::integral_constant<int, S> s_rows{};
    for (int step = 0; step < h.ns_steps; ++step) {
        put(w, l_rows);
        barrier();
        f32x4 wt[S], g[S], p[S];
        turn(wt, w);
        if (wave < S) {                               // row `wave` of G
#pragma unroll
            for (int t = 0; t < S; ++t) g[t] = p[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            add(g, l_rows, [&](int k) __attribute__((always_inline)) { return operand(k, wave); });
        }
        region ^= 1;
        if (wave < S) put(g, s_rows);
        barrier();
        if (wave < S) {
            add(p, s_rows, [&](int k) __attribute__((always_inline)) { return operand(k, wave); });
#pragma unroll
            for (int t = 0; t < S; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[t][e] = fmaf(b, g[t][e], c * p[t][e]);
        }
        region ^= 1;
        if (wave < S) put(p, s_rows);
        barrier();
#pragma unroll
        for (int t = 0; t < S; ++t) w[t] *= h.a;
        add(w, s_rows, [&](int k) __attribute__((always_inline)) { return parts_of<true>(wt[2 * k], 2 * k + 1 < S ? wt[2 * k + 1] : f32x4{}); });
        region ^= 1;
    }
    if constexpr (TALL) turn(w, w);

    const float keep = 1.f - lr * d.decay, rate = lr * d.scale / kHeld;
    const uint32_t base = mix(d.number + key);
    auto update = [&](auto type, auto has_master) __attribute__((always_inline)) {
        typedef decltype(type) T;
        typedef T t4 __attribute__((ext_vector_type(4)));
        constexpr bool MASTER = decltype(has_master)::value;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float v[4];
            T out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = fmaf(-rate, w[s][e], param[s][0][e] * keep);
                asm("" : "+v"(v[e]));                 // an fp32 number, of which the stored one is the rounding
                if constexpr (MASTER || std::is_same<T, float>::value) out[e] = from_f32<T>(v[e]);
                else out[e] = round_at_random(T{}, v[e], mix(base + (uint32_t)run_of(s, 0, e).at));
                w[s][e] = (float)out[e];
            }
            store_run4<T, WHOLE>(static_cast<T*>(d.param), out, s, 0, run_of);
            if constexpr (MASTER) store_run4<float, WHOLE>(d.master, v, s, 0, run_of);
        }
        if (!d.transposed) return;                    // uniform
        T* const t = static_cast<T*>(d.transposed) + (size_t)d.place[block] * (size_t)size;
        if ((bs_r & 3) == 0) {                        // four neighbouring elements of a row of the transpose a lane
            f32x4 turned[S];
            turn(turned, w);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int col = 16 * (TALL ? s : wave) + i, row = 16 * (TALL ? wave : s) + c0;
                if (col < bs_c && row < bs_r)
                    *reinterpret_cast<t4*>(t + (size_t)(col * bs_r + row)) = t4{(T)turned[s][0], (T)turned[s][1], (T)turned[s][2], (T)turned[s][3]};
            }
        } else {
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col_of(s) + e < bs_c && row_of(s) < bs_r) t[(size_t)((col_of(s) + e) * bs_r + row_of(s))] = (T)w[s][e];
        }
    };
    auto update_type = [&](auto type) __attribute__((always_inline)) {
        if (d.master) update(type, std::true_type{});
        else update(type, std::false_type{});
    };
    if (d.dtype == BSR_F32) update(0.f, std::false_type{});
    else if (d.dtype == BSR_F16) update_type(f16_t{});
    else update_type(bf16_t{});
}

// Whether X's singular values, 1 at most, stay below 3.9 through the steps, and P's below 2^15: the steps take a singular value s to
// a s + b s^3 + c s^5, whose largest value over 0 .. s is at the end or where its slope a + 3 b s^2 + 5 c s^4 is 0.  And a is 1 at
// least, so that small ones do not shrink from step to step below what fp16 parts tell apart (near 0 they become a s).
bool stays_small(const bsr_muon_hyper& y)
{
    const double a = y.a, b = y.b, c = y.c;
    if (std::fabs(a) < 1.0) return false;
    double most = 1.0 + 0x1p-10;                      // (roundings)
    for (int step = 0; step < y.ns_steps; ++step) {
        if (std::fabs(b) * most * most + std::fabs(c) * most * most * most * most > 0x1p15) return false;
        double next = 0.0;
        auto at = [&](double q) {                     // q: s^2
            if (q >= 0.0 && q <= most * most) next = std::max(next, std::sqrt(q) * std::fabs(a + q * (b + q * c)));
        };
        at(most * most);
        const double inside = 9.0 * b * b - 20.0 * a * c;
        if (c != 0.0 && inside >= 0.0) {
            at((-3.0 * b + std::sqrt(inside)) / (10.0 * c));
            at((-3.0 * b - std::sqrt(inside)) / (10.0 * c));
        }
        if (b != 0.0) at(-a / (3.0 * b));             // c = 0, or so small that the roots above lose it
        most = next * (1.0 + 0x1p-10);
        if (!(most <= 3.9)) return false;
    }
    return true;
}

int tiles_of(int32_t side) { return (side + 15) / 16; }
// Blocks that stand beside one another: along rows (1) or columns (2) of 8 at most, else none (0).
int mode_of(const bsr_muon_tensor& t) { return t.bs_r <= t.bs_c ? (t.bs_r <= 8 ? 1 : 0) : t.bs_c <= 8 ? 2 : 0; }
bool whole_of(const bsr_muon_tensor& t) { return mode_of(t) != 2 && t.bs_c % 4 == 0; }
int kind_of(const bsr_muon_tensor& t) { return ((mode_of(t) * 4 + tiles_of(t.bs_r) - 1) * 4 + tiles_of(t.bs_c) - 1) * 2 + whole_of(t); }
int chunk_of(const bsr_muon_tensor& t)                // blocks of a workgroup
{
    return waves_of(tiles_of(t.bs_r), tiles_of(t.bs_c)) * (mode_of(t) ? 16 / std::min(t.bs_r, t.bs_c) : 1);
}
int64_t chunks_of(const bsr_muon_tensor& t) { return (t.blocks + chunk_of(t) - 1) / chunk_of(t); }
size_t elements_of(const bsr_muon_tensor& t) { return (size_t)t.blocks * (size_t)t.bs_r * (size_t)t.bs_c; }

bsr_status check_sizes(int64_t n, const bsr_muon_tensor* tensors)
{
    if (n < 0 || n >= ((int64_t)1 << 24)) return BSR_ERR_SHAPE;
    if (n > 0 && !tensors) return BSR_ERR_NULL;
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        const bsr_muon_tensor& t = tensors[i];
        if (t.blocks < 0 || t.blocks >= ((int64_t)1 << 31) || t.bs_r < 1 || t.bs_c < 1 || t.bs_r > kMostSide || t.bs_c > kMostSide) return BSR_ERR_SHAPE;
        if (!known(t.dtype) || (t.grad_dtype != t.dtype && t.grad_dtype != BSR_F32) || (t.master_dev && t.dtype == BSR_F32)) return BSR_ERR_DTYPE;
        chunks += chunks_of(t);
        if (chunks >= ((int64_t)1 << 24)) return BSR_ERR_SHAPE;   // a launch has below 2^32 threads
    }
    return BSR_OK;
}

size_t table_words(int64_t n) { return words_of((size_t)n * sizeof(muon_desc)); }
size_t workspace_words(int64_t n, const bsr_muon_tensor* tensors)
{
    size_t words = table_words(n), chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        chunks += (size_t)chunks_of(tensors[i]);
        if (tensors[i].t_param_dev) words += words_of((size_t)tensors[i].blocks * 4);
    }
    return std::max<size_t>(words + words_of(chunks * sizeof(int2)), 64);
}

}  // namespace

struct bsr_muon {
    int device = 0;
    struct launch_t { int kind; int32_t first, count; };
    std::vector<launch_t> launches;
    const muon_desc* descs = nullptr;                 // device
    const int2* chunks = nullptr;
    std::vector<int32_t> host;                        // kept for the asynchronous upload
    hipEvent_t uploaded = nullptr;
    mutable std::atomic<bool> landed{false};
};

namespace {

bsr_status create_muon(bsr_muon** out, int64_t n, const bsr_muon_tensor* tensors, void* workspace_dev, size_t workspace_bytes, hipStream_t stream)
{
    const bsr_status st = check_sizes(n, tensors);
    if (st != BSR_OK) return st;
    if (!workspace_dev) return BSR_ERR_NULL;
    if (!aligned16(workspace_dev)) return BSR_ERR_ALIGN;
    const size_t words = workspace_words(n, tensors);
    if (workspace_bytes < words * 4) return BSR_ERR_WORKSPACE;
    std::vector<used_range> ranges;
    add_range(ranges, workspace_dev, words * 4, true);
    for (int64_t i = 0; i < n; ++i) {
        const bsr_muon_tensor& t = tensors[i];
        if (t.blocks == 0) continue;
        if (!t.param_dev || !t.grad_dev || !t.momentum_dev || (t.t_param_dev && !t.t_perm_host)) return BSR_ERR_NULL;
        for (const void* p : {(const void*)t.param_dev, (const void*)t.master_dev, t.grad_dev, (const void*)t.momentum_dev, (const void*)t.t_param_dev})
            if (!aligned16(p)) return BSR_ERR_ALIGN;
        const size_t c = elements_of(t), s = size_of(t.dtype);
        add_range(ranges, t.param_dev, c * s, true);
        add_range(ranges, t.t_param_dev, c * s, true);
        add_range(ranges, t.master_dev, c * 4, true);
        add_range(ranges, t.momentum_dev, c * 4, true);
        add_range(ranges, t.grad_dev, c * size_of(t.grad_dtype), false);
    }
    std::sort(ranges.begin(), ranges.end(), by_start);
    if (!apart(ranges)) return BSR_ERR_OVERLAP;
    std::unique_ptr<bsr_muon> opt(new bsr_muon);
    std::vector<int64_t> order((size_t)n);
    for (int64_t i = 0; i < n; ++i) order[(size_t)i] = i;
    std::stable_sort(order.begin(), order.end(), [&](int64_t a, int64_t b) { return kind_of(tensors[a]) < kind_of(tensors[b]); });
    opt->host.assign(words, 0);
    int32_t* const dev = static_cast<int32_t*>(workspace_dev);
    const size_t chunks_at = table_words(n);
    size_t chunk = 0, total = 0;
    for (int64_t i = 0; i < n; ++i) total += (size_t)chunks_of(tensors[i]);
    size_t at = chunks_at + words_of(total * sizeof(int2));
    for (int64_t s = 0; s < n; ++s) {
        const bsr_muon_tensor& t = tensors[order[(size_t)s]];
        const int64_t mine = chunks_of(t);
        if (mine) {
            if (opt->launches.empty() || opt->launches.back().kind != kind_of(t)) opt->launches.push_back({kind_of(t), (int32_t)chunk, 0});
            opt->launches.back().count += (int32_t)mine;
        }
        for (int64_t c = 0; c < mine; ++c, ++chunk) {
            opt->host[chunks_at + 2 * chunk] = (int32_t)s;
            opt->host[chunks_at + 2 * chunk + 1] = (int32_t)(c * chunk_of(t));
        }
        muon_desc d{};
        d.param = t.param_dev; d.master = t.master_dev; d.grad = t.grad_dev; d.momentum = t.momentum_dev; d.blocks = t.blocks;
        d.decay = t.weight_decay; d.scale = t.scale; d.number = (uint32_t)order[(size_t)s]; d.bs_r = t.bs_r; d.bs_c = t.bs_c;
        d.dtype = t.dtype; d.grad_dtype = t.grad_dtype;
        if (t.t_param_dev && t.blocks) {
            d.transposed = t.t_param_dev;
            d.place = dev + at;
            std::vector<char> seen((size_t)t.blocks, 0);
            for (int64_t q = 0; q < t.blocks; ++q) {  // block perm[q] of W goes to place q of W^T
                const int32_t p = t.t_perm_host[q];
                if (p < 0 || p >= t.blocks || seen[(size_t)p]) return BSR_ERR_INDEX;
                seen[(size_t)p] = 1;
                opt->host[at + (size_t)p] = (int32_t)q;
            }
        }
        if (t.t_param_dev) at += words_of((size_t)t.blocks * 4);
        std::memcpy(opt->host.data() + (size_t)s * (sizeof(muon_desc) / 4), &d, sizeof d);
    }
    opt->descs = reinterpret_cast<const muon_desc*>(dev);
    opt->chunks = reinterpret_cast<const int2*>(dev + chunks_at);
    if (hipGetDevice(&opt->device) != hipSuccess) return BSR_ERR_HIP;
    if (n > 0 && (is_capturing(stream) || !upload_words(dev, opt->host, stream, opt->uploaded, opt->landed))) {
        if (opt->uploaded) (void)hipEventDestroy(opt->uploaded);
        (void)hipGetLastError();
        return BSR_ERR_HIP;
    }
    *out = opt.release();
    return BSR_OK;
}

// Up to so many chunks of two large blocks, which do not fill the CUs with a wavefront each, a block has a workgroup (both sides: at
// bsr_muon_team).  The two add a product's terms in another order: which one a tensor gets depends on the list's blocks of its tiles.
constexpr int kFewChunks = 512;
template <int RT, int CT, int MODE> bsr_status launch_tiles(const bsr_muon* opt, const bsr_muon::launch_t& l, const muon_args& h, hipStream_t stream)
{
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.count), dim3(64 * waves_of(RT, CT)), 0, stream, opt->descs, opt->chunks + l.first, h);
        return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
    };
    const bool whole = l.kind % 2;
    if constexpr (RT > 2 && CT > 2)
        if (h.small && l.count <= kFewChunks) {
            auto team = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3((unsigned)l.count * waves_of(RT, CT)), dim3(64 * std::max(RT, CT)), 0, stream, opt->descs, opt->chunks + l.first, h);
                return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
            };
            return whole ? team(bsr_muon_team<RT, CT, true>) : team(bsr_muon_team<RT, CT, false>);
        }
    if constexpr (MODE != 2)
        if (whole) return h.small ? go(bsr_muon_blocks<RT, CT, MODE, true, true>) : go(bsr_muon_blocks<RT, CT, MODE, true, false>);
    return h.small ? go(bsr_muon_blocks<RT, CT, MODE, false, true>) : go(bsr_muon_blocks<RT, CT, MODE, false, false>);
}
template <int RT> bsr_status launch_rows(const bsr_muon* opt, const bsr_muon::launch_t& l, const muon_args& h, hipStream_t stream)
{
    switch (l.kind / 2 % 4) {
        case 0: return launch_tiles<RT, 1, 0>(opt, l, h, stream);
        case 1: return launch_tiles<RT, 2, 0>(opt, l, h, stream);
        case 2: return launch_tiles<RT, 3, 0>(opt, l, h, stream);
    }
    return launch_tiles<RT, 4, 0>(opt, l, h, stream);
}
bsr_status launch_kind(const bsr_muon* opt, const bsr_muon::launch_t& l, const muon_args& h, hipStream_t stream)
{
    const int mode = l.kind / 32, rt = l.kind / 8 % 4, ct = l.kind / 2 % 4;
    if (mode == 1) return ct == 0 ? launch_tiles<1, 1, 1>(opt, l, h, stream) : ct == 1 ? launch_tiles<1, 2, 1>(opt, l, h, stream)
                        : ct == 2 ? launch_tiles<1, 3, 1>(opt, l, h, stream) : launch_tiles<1, 4, 1>(opt, l, h, stream);
    if (mode == 2) return rt == 0 ? launch_tiles<1, 1, 2>(opt, l, h, stream) : rt == 1 ? launch_tiles<2, 1, 2>(opt, l, h, stream)
                        : rt == 2 ? launch_tiles<3, 1, 2>(opt, l, h, stream) : launch_tiles<4, 1, 2>(opt, l, h, stream);
    return rt == 0 ? launch_rows<1>(opt, l, h, stream) : rt == 1 ? launch_rows<2>(opt, l, h, stream)
         : rt == 2 ? launch_rows<3>(opt, l, h, stream) : launch_rows<4>(opt, l, h, stream);
}

}  // namespace

extern "C" {

bsr_status bsr_muon_workspace_size(int64_t n_tensors, const bsr_muon_tensor* tensors, size_t* bytes)
{
    if (!bytes) return BSR_ERR_NULL;
    *bytes = 0;
    const bsr_status st = check_sizes(n_tensors, tensors);
    if (st == BSR_OK) *bytes = workspace_words(n_tensors, tensors) * 4;
    return st;
}

bsr_status bsr_muon_create(bsr_muon** out, int64_t n_tensors, const bsr_muon_tensor* tensors, void* workspace_dev, size_t workspace_bytes,
                           void* hip_stream)
{
    if (!out) return BSR_ERR_NULL;
    *out = nullptr;
    try {
        return create_muon(out, n_tensors, tensors, workspace_dev, workspace_bytes, (hipStream_t)hip_stream);
    } catch (const std::bad_alloc&) {                 // no host memory for the tables
        return BSR_ERR_HIP;
    } catch (const std::length_error&) {
        return BSR_ERR_SHAPE;
    }
}

void bsr_muon_destroy(bsr_muon* opt)
{
    if (!opt) return;
    if (opt->uploaded) {                              // the upload reads the handle's host buffer
        (void)hipEventSynchronize(opt->uploaded);
        (void)hipEventDestroy(opt->uploaded);
        (void)hipGetLastError();
    }
    delete opt;
}

bsr_status bsr_muon_step(const bsr_muon* opt, const bsr_muon_hyper* hyper, void* hip_stream)
{
    if (!opt || !hyper) return BSR_ERR_NULL;
    const bsr_muon_hyper& y = *hyper;
    // (negated: NaN is refused too)
    if (!(y.momentum >= 0 && y.momentum < 1) || !(y.eps >= 0x1p-100 && y.eps <= 1) || !std::isfinite(y.a) || !std::isfinite(y.b) || !std::isfinite(y.c) ||
        y.ns_steps < 0 || y.ns_steps > kMostSteps || (!y.step_dev && y.step < 1) || (!y.lr_dev && !(y.lr >= 0))) return BSR_ERR_SHAPE;
    const float size = std::fabs(y.grad_scale);
    if (!y.grad_scale_dev && !(size == 0.f || (size >= 0x1p-40f && size <= 0x1p40f))) return BSR_ERR_SHAPE;
    for (const void* p : {(const void*)y.lr_dev, (const void*)y.grad_scale_dev})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return BSR_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(y.step_dev) & 7u) return BSR_ERR_ALIGN;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev != opt->device) return BSR_ERR_DEVICE;
    hipStream_t stream = (hipStream_t)hip_stream;
    ready_for(opt->uploaded, opt->landed, stream);
    if (!y.grad_scale_dev && y.grad_scale == 0.f) return BSR_OK;
    muon_args h{};
    h.lr = (float)y.lr;
    h.mu = (float)y.momentum;
    h.eps = (float)y.eps;
    h.a = y.a;
    h.b = y.b;
    h.c = y.c;
    h.grad_scale = y.grad_scale;
    h.ns_steps = y.ns_steps;
    h.nesterov = y.nesterov != 0;
    h.small = stays_small(y);
    if (!y.step_dev) h.key = step_key(y.seed, (uint64_t)y.step);
    h.seed = y.seed;
    h.lr_dev = y.lr_dev;
    h.step_dev = y.step_dev;
    h.grad_scale_dev = y.grad_scale_dev;
    for (const auto& l : opt->launches) {
        const bsr_status st = launch_kind(opt, l, h, stream);
        if (st != BSR_OK) return st;
    }
    return BSR_OK;
}

}  // extern "C"
