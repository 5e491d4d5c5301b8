// Rows of any width and alignment: vectors of elements at any multiple of their size, and sums over the lanes that share a row.
#pragma once

#include "bsr_mfma_common.h"

namespace bsr_dev {

// V elements at any multiple of their size, of which `count` are there (the others as zeros, and not stored).
template <typename T, int V> struct any_run {
    typedef T vec_t __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    vec_t v;
    __device__ __forceinline__ void load(const T* p, int count)
    {
        if (count >= V) {
            v = *reinterpret_cast<const vec_t*>(p);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = e < count ? p[e] : (T)0.f;
        }
    }
    __device__ __forceinline__ void store(T* p, int count) const
    {
        if (count >= V) {
            *reinterpret_cast<vec_t*>(p) = v;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < count) p[e] = v[e];
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return (float)v[e]; }
    __device__ __forceinline__ void set(int e, float x) { v[e] = from_f32<T>(x); }
};

template <int CTRL> __device__ __forceinline__ float dpp_f32(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}

// Sum over T neighbouring lanes (T = 8, 16, 32 or 64), the same in all of them; every lane of the wavefront takes part.
template <int T> __device__ __forceinline__ float lane_sum(float v)
{
    v += dpp_f32<0xB1>(v);                            // lanes 1 apart, 2 apart, the halves of 8, of 16
    v += dpp_f32<0x4E>(v);
    v += dpp_f32<0x141>(v);
    if constexpr (T >= 16) v += dpp_f32<0x140>(v);
    if constexpr (T >= 32) v += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F));
    if constexpr (T >= 64)
        v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 0)) +
            __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 32));
    return v;
}

}  // namespace bsr_dev
