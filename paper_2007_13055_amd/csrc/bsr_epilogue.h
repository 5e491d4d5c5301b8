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
//              t = 1 / (1 + 0.24 a), S of degree 7, fitted to least relative error (4.3e-7 over a in [0, 40]; in fp32 8e-7).
//              Written so, a negative x keeps its relative accuracy, which 1 + erf(x / sqrt 2) loses by cancellation.
// A NaN stays one; at infinite z the limits are taken (0 or z, slopes 0 or 1) in place of the NaN of 0 * inf.
#pragma once

#include "bsr_mfma_common.h"

// `e` as the kernels take it; null pointers: that part is left out.
struct epilogue_args {
    static constexpr bool on = true;
    const void* bias;                                 // [n], W's type or fp32
    const void* residual;                             // [m] rows of n elements of Y's type, residual_ld apart
    const void* through;                              // Z0 [m][n], Y's type
    void* z;                                          // Z [m][n], Y's type
    int64_t residual_ld;
    int32_t act;
    int32_t bias_f32;
};
struct no_epilogue {
    static constexpr bool on = false;
};

// Calls launch(no_epilogue) or launch(epilogue_args), as the product asks for.
template <typename F>
bsr_status with_epilogue(const spmm_args& a, F launch)
{
    if (!a.epilogue) return launch(no_epilogue{});
    const bsr_epilogue& e = *a.epilogue;
    const int32_t act = e.act;
    return launch(epilogue_args{e.bias_dev, e.residual_dev, act == BSR_ACT_NONE ? nullptr : e.through_dev, e.z_dev,
                                e.residual_ld ? e.residual_ld : a.W->n, act, e.bias_dtype == BSR_F32});
}

namespace bsr_dev {

constexpr float kLog2e = 1.44269504f;

__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * x)); }
// 0 where `share` is, whatever x is (0 * inf is no part of a limit)
__device__ __forceinline__ float share_of(float share, float x) { return share == 0.f ? 0.f : share * x; }

// exp(-a^2 / 2) and Q(a) of a = |x|
__device__ __forceinline__ void normal_tail(float a, float& e, float& q)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.24f, a, 1.f));
    float s = -0.0529904738f;
    s = fmaf(s, t, 0.152789459f);
    s = fmaf(s, t, -0.0656933263f);
    s = fmaf(s, t, 0.118379995f);
    s = fmaf(s, t, 0.0634018406f);
    s = fmaf(s, t, 0.0928374827f);
    s = fmaf(s, t, 0.0955223069f);
    s = fmaf(s, t, 0.0957537889f);
    e = __builtin_amdgcn_exp2f(a * a * (-0.5f * kLog2e));
    q = e * (t * s);
}

constexpr float kGeluA = 1.59576912f, kGeluB = 0.044715f;          // 2 sqrt(2 / pi)

template <int ACT> __device__ __forceinline__ float act_value(float x)
{
    if constexpr (ACT == BSR_ACT_RELU) return x < 0.f ? 0.f : x;
    if constexpr (ACT == BSR_ACT_GELU) {
        float e, q;
        normal_tail(fabsf(x), e, q);
        return (x < 0.f ? 0.f : x) - share_of(q, fabsf(x));
    }
    if constexpr (ACT == BSR_ACT_GELU_TANH) return share_of(logistic(kGeluA * x * fmaf(kGeluB, x * x, 1.f)), x);
    if constexpr (ACT == BSR_ACT_SILU) return share_of(logistic(x), x);
    return x;
}

template <int ACT> __device__ __forceinline__ float act_slope(float x)
{
    if constexpr (ACT == BSR_ACT_RELU) return x > 0.f ? 1.f : x != x ? x : 0.f;
    if constexpr (ACT == BSR_ACT_GELU) {
        float e, q;
        normal_tail(fabsf(x), e, q);
        return (x < 0.f ? q : 1.f - q) + share_of(e, x * 0.398942280f);   // Phi(x) + x phi(x)
    }
    if constexpr (ACT == BSR_ACT_GELU_TANH) {
        const float xx = x * x, s = logistic(kGeluA * x * fmaf(kGeluB, xx, 1.f));
        return s + share_of(s * (1.f - s), kGeluA * x * fmaf(3.f * kGeluB, xx, 1.f));
    }
    if constexpr (ACT == BSR_ACT_SILU) {
        const float s = logistic(x);
        return s + share_of(s * (1.f - s), x);
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

// N consecutive elements (1, 4 or 8), at an address that is a multiple of their size up to 16 bytes.
template <typename T, int N> __device__ __forceinline__ void load_run(float (&v)[N], const T* __restrict__ p)
{
    if constexpr (N == 1) {
        v[0] = (float)*p;
    } else {
        constexpr int K = (int)(16 / sizeof(T)) < N ? (int)(16 / sizeof(T)) : N;
        typedef T vec_t __attribute__((ext_vector_type(K)));
#pragma unroll
        for (int i = 0; i < N; i += K) {
            const vec_t t = *reinterpret_cast<const vec_t*>(p + i);
#pragma unroll
            for (int e = 0; e < K; ++e) v[i + e] = (float)t[e];
        }
    }
}
template <typename O, int N> __device__ __forceinline__ void store_run(O* __restrict__ p, const float (&v)[N])
{
    if constexpr (N == 1) {
        *p = from_f32<O>(v[0]);
    } else {
        constexpr int K = (int)(16 / sizeof(O)) < N ? (int)(16 / sizeof(O)) : N;
        typedef O vec_t __attribute__((ext_vector_type(K)));
#pragma unroll
        for (int i = 0; i < N; i += K) {
            vec_t t;
#pragma unroll
            for (int e = 0; e < K; ++e) t[e] = from_f32<O>(v[i + e]);
            *reinterpret_cast<vec_t*>(p + i) = t;
        }
    }
}

// Sums of columns j .. j + N - 1 of row i, as they are to be stored.  T: W's type, O: Y's.
template <typename T, typename O, int N>
__device__ __forceinline__ void finish(const epilogue_args& ep, float (&v)[N], int i, int j, int n)
{
    const size_t at = (size_t)i * (size_t)n + (size_t)j;
    if (ep.bias) {
        float b[N];
        if (std::is_same<T, float>::value || ep.bias_f32) load_run<float>(b, static_cast<const float*>(ep.bias) + j);
        else load_run<T>(b, static_cast<const T*>(ep.bias) + j);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += b[e];
    }
    if (ep.z) store_run<O>(static_cast<O*>(ep.z) + at, v);
    if (ep.through) {
        float z0[N];
        load_run<O>(z0, static_cast<const O*>(ep.through) + at);
        with_act(ep.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] *= act_slope<decltype(act)::value>(z0[e]);
        });
    } else {
        with_act(ep.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = act_value<decltype(act)::value>(v[e]);
        });
    }
    if (ep.residual) {
        float r[N];
        load_run<O>(r, static_cast<const O*>(ep.residual) + (size_t)i * (size_t)ep.residual_ld + (size_t)j);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += r[e];
    }
}
template <typename T, typename O, int N> __device__ __forceinline__ void finish(const no_epilogue&, float (&)[N], int, int, int) {}

// As store4: 4 consecutive columns of row i.
template <typename T, typename O, typename E>
__device__ __forceinline__ void finish_store4(const E& ep, O* __restrict__ Y, int i, int j, int n, float v0, float v1, float v2, float v3)
{
    O* dst = Y + (size_t)i * (size_t)n + (size_t)j;
    if constexpr (E::on) {
        float v[4] = {v0, v1, v2, v3};
        finish<T, O>(ep, v, i, j, n);
        store_run<O>(dst, v);
    } else {
        store4<O>(dst, v0, v1, v2, v3);
    }
}

}  // namespace bsr_dev
