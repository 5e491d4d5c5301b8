// What a product does with its sums before they are stored (bsr_spmm_epilogue):
//
//     z = sum + bias[j]         Z[i][j] = z, if wanted
//     y = act(z)                or, with `through`, z * act'(Z0[i][j])
//     Y[i][j] = y + R[i][j]
//
// Every kernel of the product is built twice: with `no_epilogue`, as bsr_spmm() runs it, and with `epilogue_args`.  All of it
// happens in fp32 on the accumulated sum; a 16-bit result is rounded once, on its way to Y (and z once, on its way to Z).
//
// Activations, with e = 2^(-y log2 e) from the hardware's exponential and its reciprocal (both within an ulp):
//   silu       x s(x),   s(x) = 1 / (1 + exp(-x))
//   gelu_tanh  x s(2 u), u = sqrt(2 / pi) (x + 0.044715 x^3): tanh(u) = 2 s(2 u) - 1
//   gelu       x Phi(x) = max(x, 0) - |x| Q(|x|),  Q(a) = erfc(a / sqrt 2) / 2 = exp(-a^2 / 2) P(a):  P(a) = t S(t) with
//              t = 1 / (1 + 0.24 a), S of degree 7, fitted to least relative error with P(0) = 1/2 held, so that the slope has
//              no jump at 0 (4.4e-7 over a in [0, 40], with the coefficients as fp32 holds them).  Written so, a negative x
//              keeps its relative accuracy, which 1 + erf(x / sqrt 2) loses by cancellation.  In fp32 the relative error of
//              Q is below 1.5e-6 + 2^-23 a^2 while Q is a normal number (a < 12.9): besides the fit, t's two roundings (P
//              follows t with a power of up to 3.3), the exponential's ulp and three products', 1e-6; and what the argument
//              y^2, y = a sqrt(log2(e) / 2), is off by, 2^-24 for the constant and for y, twice each, and for the square, of
//              which a^2 / 2 becomes a relative error.  (x^2 times a constant has one rounding less, and its products are
//              ordered otherwise by the compiler: 4096 x (1024, 4096) bf16 16x16 20 % 32.8 us, this way 31.9.)
// A NaN stays one; at infinite z the limits are taken (0 or z, slopes 0 or 1) in place of the NaN of 0 * inf.
#pragma once

#include "bsr_mfma_common.h"

// `e` as the kernels take it; null pointers: that part is left out.
struct epilogue_args {
    static constexpr bool on = true, gated = false;
    const void* bias;                                 // [n], W's type or fp32
    const void* residual;                             // [m] rows of n elements of Y's type, residual_ld apart
    const void* through;                              // Z0 [m][n], Y's type
    void* z;                                          // Z [m][n], Y's type
    int64_t residual_ld;
    int32_t act;
    int32_t bias_f32;
    int32_t once;                                     // residual and Z0 are read past the caches
};
struct no_epilogue {
    static constexpr bool on = false, gated = false;
};

// The gated product's last stage (bsr_spmm_gated): a workgroup has the sums of block-rows 2r and 2r + 1, z_g and z_u,
//     z += bias         Z = z, if wanted         H = act(z_g) z_u
// n is W's, twice H's; a half's columns stand together in units of bs_r.
struct gated_args {
    typedef bsr_dev::i32x4 i32x4;
    static constexpr bool on = false, gated = true;
    const void* bias;                                 // [n], W's type or fp32, in W's order
    void* z;                                          // Z [m][n], H's type
    const int32_t* indptr;                            // W's
    const i32x4* pairs;                               // W's gate_pairs
    int32_t act;
    int32_t bias_f32;
};

// Calls launch(no_epilogue) or launch(epilogue_args), as the product asks for.
template <typename F>
bsr_status with_epilogue(const spmm_args& a, F launch)
{
    if (!a.epilogue) return launch(no_epilogue{});
    const bsr_epilogue& e = *a.epilogue;
    const int32_t act = e.act;
    // Where neither is in the 256 MB cache behind the L2s, both ways take as long (within 3 % from 34 to 134 MB).  A residual that
    // the kernel that wrote it left there is read faster through the caches (two 105 MB ones in turn: 89 us, past them 99;
    // 34 MB: 30 and 36), unless it pushes the result and itself out: two of 134 MB, 154 us, past the caches 136.  The rule knows
    // the result's size alone.  A residual of 126 MB that the kernel before has just written, one set over and over (k = 1024,
    // 10 %), is read either way as long with 64x64 f16 blocks (67 us) and faster through the caches with 32x32 f16 (79 us, past them 98),
    // 16x16 f16 with fp32 results (68, 74) and fp32 blocks (134 MB, 32x32: 104, 116); two sets in turn of the same past
    // them (f16 16x16 87, through them 94; 32x32 98, 99); 201 MB is faster past them in all of these (103 and 112, 146 and 162).
    const bool once = (int64_t)a.m * a.W->n * (a.y_dtype == BSR_F32 ? 4 : 2) > ((int64_t)112 << 20);
    return launch(epilogue_args{e.bias_dev, e.residual_dev, act == BSR_ACT_NONE ? nullptr : e.through_dev, e.z_dev,
                                e.residual_ld ? e.residual_ld : a.W->n, act, e.bias_dtype == BSR_F32, once});
}

// The same, in the kernels that also finish gated products.
template <typename F>
bsr_status with_epilogue_or_gate(const spmm_args& a, F launch)
{
    if (!a.gated) return with_epilogue(a, launch);
    const bsr_gated& e = *a.gated;
    return launch(gated_args{e.bias_dev, e.z_dev, a.W->indptr, reinterpret_cast<const bsr_dev::i32x4*>(a.W->gate_pairs), (int32_t)e.act, e.bias_dtype == BSR_F32});
}

namespace bsr_dev {

constexpr float kLog2e = 1.44269504f;

__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x)); }
// share * x; 0 where share is, at infinite x too (0 * inf is no part of a limit).  A NaN x has made `share` one.
constexpr float kMost = 3.40282347e+38f;
__device__ __forceinline__ float share_of(float share, float x) { return share * __builtin_amdgcn_fmed3f(x, -kMost, __builtin_inff()); }

__device__ __forceinline__ float finite(float x) { return __builtin_amdgcn_fmed3f(x, -kMost, kMost); }

// exp(-x^2 / 2) and Q(|x|)
__device__ __forceinline__ void normal_tail(float x, float& e, float& q)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.24f, fabsf(x), 1.f)), y = x * 0.849321800f;   // sqrt(log2(e) / 2)
    float s = -0.0530403703f;
    s = fmaf(s, t, 0.152946189f);
    s = fmaf(s, t, -0.0658932477f);
    s = fmaf(s, t, 0.11851076f);
    s = fmaf(s, t, 0.0633547232f);
    s = fmaf(s, t, 0.0928467363f);
    s = fmaf(s, t, 0.0955213904f);
    s = fmaf(s, t, 0.0957538188f);
    e = __builtin_amdgcn_exp2f(-y * y);
    q = e * (t * s);
}

constexpr float kGeluA = 1.59576912f, kGeluB = 0.044715f;          // 2 sqrt(2 / pi)
__device__ __forceinline__ float gelu_share(float x, float xx)      // s(2 u)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * fmaf(-kLog2e * kGeluA * kGeluB, xx, -kLog2e * kGeluA)));
}

template <int ACT> __device__ __forceinline__ float act_value(float x)
{
    if constexpr (ACT == BSR_ACT_RELU) return x < 0.f ? 0.f : x;
    if constexpr (ACT == BSR_ACT_GELU) {
        float e, q;
        normal_tail(x, e, q);
        // med3 for the minimum and the maximum, which cost an instruction more each (of 17); a NaN x has made q one
        return fmaf(-q, __builtin_amdgcn_fmed3f(fabsf(x), -kMost, kMost), __builtin_amdgcn_fmed3f(x, 0.f, __builtin_inff()));
    }
    if constexpr (ACT == BSR_ACT_GELU_TANH) return share_of(gelu_share(x, x * x), x);
    if constexpr (ACT == BSR_ACT_SILU) return share_of(logistic(x), x);
    return x;
}

template <int ACT> __device__ __forceinline__ float act_slope(float x)
{
    if constexpr (ACT == BSR_ACT_RELU) return x > 0.f ? 1.f : x != x ? x : 0.f;
    if constexpr (ACT == BSR_ACT_GELU) {
        float e, q;
        normal_tail(x, e, q);
        return fmaf(e * 0.398942280f, finite(x), x < 0.f ? q : 1.f - q);   // x phi(x) + Phi(x)
    }
    if constexpr (ACT == BSR_ACT_GELU_TANH) {
        const float xx = x * x, s = gelu_share(x, xx);
        return fmaf(s * (1.f - s), finite(x * fmaf(3.f * kGeluA * kGeluB, xx, kGeluA)), s);
    }
    if constexpr (ACT == BSR_ACT_SILU) {
        const float s = logistic(x);
        return fmaf(s * (1.f - s), finite(x), s);
    }
    return 1.f;
}

// The activation is the same for a whole launch: one uniform branch around all of a lane's values.
template <typename F> __device__ __forceinline__ void with_act(int act, F f)
{
    if (act == BSR_ACT_RELU) f(std::integral_constant<int, BSR_ACT_RELU>{});
    else if (act == BSR_ACT_GELU) f(std::integral_constant<int, BSR_ACT_GELU>{});
    else if (act == BSR_ACT_GELU_TANH) f(std::integral_constant<int, BSR_ACT_GELU_TANH>{});
    else if (act == BSR_ACT_SILU) f(std::integral_constant<int, BSR_ACT_SILU>{});
}

// The same where there may be none.
template <typename F> __device__ __forceinline__ void with_act_or_none(int act, F f)
{
    if (act == BSR_ACT_NONE) f(std::integral_constant<int, BSR_ACT_NONE>{});
    else with_act(act, f);
}

// N consecutive elements (1, 4 or 8) as loaded, at an address that is a multiple of their size up to 16 bytes.
template <typename T, int N> struct run_of {
    static constexpr int K = (int)(16 / sizeof(T)) < N ? (int)(16 / sizeof(T)) : N;   // of a load
    typedef T vec_t __attribute__((ext_vector_type(K)));
    vec_t part[N / K];
    __device__ __forceinline__ void load(const T* __restrict__ p, bool once = false)   // uniform
    {
#pragma unroll
        for (int i = 0; i < N / K; ++i) {
            const vec_t* at = reinterpret_cast<const vec_t*>(p + i * K);
            // (the comments in the code keep the compiler from making one ordinary load of the two)
            if (once) {
                asm volatile("; read once");
                part[i] = __builtin_nontemporal_load(at);
                asm volatile("; read once");
            } else {
                part[i] = *at;
            }
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return (float)part[e / K][e % K]; }
};
template <typename T, int N> __device__ __forceinline__ void load_run(float (&v)[N], const T* __restrict__ p)
{
    run_of<T, N> r;
    r.load(p);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = r[e];
}
template <bool NT = false, typename O, int N> __device__ __forceinline__ void store_run(O* __restrict__ p, const float (&v)[N])
{
    constexpr int K = run_of<O, N>::K;
#pragma unroll
    for (int i = 0; i < N; i += K) {
        typename run_of<O, N>::vec_t t;
#pragma unroll
        for (int e = 0; e < K; ++e) t[e] = from_f32<O>(v[i + e]);
        auto* at = reinterpret_cast<typename run_of<O, N>::vec_t*>(p + i);
        if constexpr (NT) __builtin_nontemporal_store(t, at);
        else *at = t;
    }
}

// What the sums of columns j .. j + N - 1 meet, T: W's type, O: Y's: the bias, and row i's part of what is read once per
// result.  Apart from finish(), so that a kernel can have the reads under way before it has its sums.
template <typename T, int N> struct bias_run {
    float b[N];
    template <typename E> __device__ __forceinline__ void fetch(const E& ep, int j)   // epilogue_args or gated_args
    {
#pragma unroll
        for (int e = 0; e < N; ++e) b[e] = 0.f;
        if (!ep.bias) return;
        if (std::is_same<T, float>::value || ep.bias_f32) load_run<float>(b, static_cast<const float*>(ep.bias) + j);
        else load_run<T>(b, static_cast<const T*>(ep.bias) + j);
    }
};
template <typename O, int N> struct result_reads {
    run_of<O, N> z0, r;
    __device__ __forceinline__ void fetch(const epilogue_args& ep, int i, int j, int n)
    {
        if (ep.through) z0.load(static_cast<const O*>(ep.through) + (size_t)i * (size_t)n + (size_t)j, ep.once);
        if (ep.residual) r.load(static_cast<const O*>(ep.residual) + (size_t)i * (size_t)ep.residual_ld + (size_t)j, ep.once);
    }
};

// Sums of columns j .. j + N - 1 of row i, as they are to be stored.
template <typename T, typename O, int N>
__device__ __forceinline__ void finish(const epilogue_args& ep, const bias_run<T, N>& bias, const result_reads<O, N>& reads, float (&v)[N], int i,
                                       int j, int n)
{
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] += bias.b[e];
    if (ep.z) store_run<true>(static_cast<O*>(ep.z) + (size_t)i * (size_t)n + (size_t)j, v);
    if (ep.through) {
        with_act(ep.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] *= act_slope<decltype(act)::value>(reads.z0[e]);
        });
    } else {
        with_act(ep.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = act_value<decltype(act)::value>(v[e]);
        });
    }
    if (ep.residual) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += reads.r[e];
    }
}
template <typename T, typename O, int N>
__device__ __forceinline__ void finish(const epilogue_args& ep, float (&v)[N], int i, int j, int n)
{
    bias_run<T, N> bias;
    result_reads<O, N> reads;
    bias.fetch(ep, j);
    reads.fetch(ep, i, j, n);
    finish<T, O>(ep, bias, reads, v, i, j, n);
}

// Gated sums g, u of a piece of row i, whose columns in W's order begin at j and j + unit: Z stored if wanted, H into g.  NT: past
// the caches, for kernels whose pieces of a half are 64 bytes or more beside one another; shorter ones become lines in L2 (bf16
// 16x16, 4096 x (1024, 2 x 4096): 51.6 us, past it 55.9).
template <typename T, typename O, bool NT = false, int N>
__device__ __forceinline__ void finish_gate(const gated_args& ep, const bias_run<T, N>& bg, const bias_run<T, N>& bu, float (&g)[N], float (&u)[N], int i,
                                            int j, int unit, int n)
{
#pragma unroll
    for (int e = 0; e < N; ++e) {
        g[e] += bg.b[e];
        u[e] += bu.b[e];
    }
    if (ep.z) {
        O* const z = static_cast<O*>(ep.z) + (size_t)i * (size_t)n + (size_t)j;
        store_run<NT>(z, g);
        store_run<NT>(z + unit, u);
    }
    with_act_or_none(ep.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            g[e] = act_value<decltype(act)::value>(g[e]) * u[e];
            asm("" : "+v"(g[e]));                     // an fp32 number: left to itself the compiler rounds the exact product to fp16
        }
    });
}

// As store4: 4 consecutive columns of row i.
template <typename T, typename O, typename E>
__device__ __forceinline__ void finish_store4(const E& ep, O* __restrict__ Y, int i, int j, int n, float v0, float v1, float v2, float v3)
{
    O* dst = Y + (size_t)i * (size_t)n + (size_t)j;
    if constexpr (E::on) {
        float v[4] = {v0, v1, v2, v3};
        finish<T, O>(ep, v, i, j, n);
        store_run(dst, v);
    } else {
        store4<O>(dst, v0, v1, v2, v3);
    }
}

}  // namespace bsr_dev
