// What the steps over lists of tensors share (bsr_adamw.hip, bsr_muon.hip): random bits and roundings, and on the host the
// checks of a list's buffers and the wait for its tables.
#pragma once

#include <algorithm>

#include "bsr_mfma_common.h"

namespace bsr_dev {

// Two rounds of xor-shift and multiply.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0xBB67AE85u;
    x ^= x >> 15;
    x *= 0x6A09E667u;
    return x ^ (x >> 16);
}
__host__ __device__ __forceinline__ uint32_t step_key(uint32_t seed, uint64_t step) { return mix(seed + 0x9E3779B1u * (uint32_t)step); }

template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false); }
// Largest v of the wavefront (the steps of a sum over 64 lanes).  On the bits of numbers that are not negative, whose order
// theirs is: a maximum of floats costs another instruction for each operand, to quieten a NaN.
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = max(v, dpp<0xB1>(v));
    v = max(v, dpp<0x4E>(v));
    v = max(v, dpp<0x141>(v));
    v = max(v, dpp<0x140>(v));
    v = max(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x401F));
    return max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 32));
}
__device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float float_of(uint32_t v) { return __builtin_bit_cast(float, v); }

// fp32 to 16 bits, away from zero with the probability that keeps the mean; `random`: 16 random bits.
__device__ __forceinline__ bf16_t round_at_random(bf16_t, float x, uint32_t random)
{
    // an infinity's low bits are zeros and stay below the place; of a NaN the arithmetic has set the highest bit, which stays
    const uint32_t u = bits_of(x) + (x == x ? random & 0xFFFFu : 0u);
    return __builtin_bit_cast(bf16_t, (uint16_t)(u >> 16));
}
__device__ __forceinline__ f16_t round_at_random(f16_t, float x, uint32_t random)
{
    // steps of fp16 at x: 2^(exponent - 10), 2^-24 among its subnormal numbers; x in such steps keeps 13 bits behind the point
    const int exponent = max((int)((__builtin_bit_cast(uint32_t, x) >> 23) & 255u) - 127, -14);
    if (exponent > 15) return (f16_t)x;
    const float steps = ldexpf(fabsf(x), 10 - exponent);
    const float whole = floorf(steps + (float)(random & 0x1FFFu) * (1.f / 8192.f));
    return (f16_t)copysignf(ldexpf(whole, exponent - 10), x);
}

}  // namespace bsr_dev

namespace bsr_list {

inline size_t size_of(bsr_dtype t) { return t == BSR_F32 ? 4 : 2; }
inline bool known(bsr_dtype t) { return (int)t >= (int)BSR_F32 && (int)t <= (int)BSR_BF16; }
inline size_t words_of(size_t bytes) { return (bytes + 255) / 256 * 64; }

struct used_range { uintptr_t from, to; bool written; };
inline void add_range(std::vector<used_range>& all, const void* p, size_t bytes, bool written)
{
    if (p && bytes) all.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
}
inline bool by_start(const used_range& a, const used_range& b) { return a.from < b.from; }
// Whether all that is written is apart from everything else of these, which are in order.
inline bool apart(const std::vector<used_range>& all)
{
    uintptr_t end = 0, written_end = 0;               // of what begins before
    for (const used_range& x : all) {
        if (x.from < (x.written ? end : written_end)) return false;
        end = std::max(end, x.to);
        if (x.written) written_end = std::max(written_end, x.to);
    }
    return true;
}

// The tables are there for what `stream` is given next.  What is recorded into a graph cannot wait for an upload outside of
// it, so a capture right behind the list's creation waits here, on the host.
inline void ready_for(hipEvent_t uploaded, std::atomic<bool>& landed, hipStream_t stream)
{
    if (uploaded && is_capturing(stream) && !upload_landed(uploaded, landed)) {
        hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;      // in the default mode the wait would end the capture
        const bool swapped = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
        if (hipEventSynchronize(uploaded) == hipSuccess) landed.store(true, std::memory_order_release);
        if (swapped) (void)hipThreadExchangeStreamCaptureMode(&mode);
        (void)hipGetLastError();
    }
    order_after_upload(stream, uploaded, landed);
}

}  // namespace bsr_list
