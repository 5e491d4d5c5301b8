// One AdamW step over many tensors at once: the step that turns the gradients of the stored blocks (bsr_sddmm) into the
// blocks that the next product reads (bsr_spmm), and the stored values of W^T with them (bsr_transpose_values).
//
//     m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
//     p = p (1 - lr decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Work split: the tensors are cut into chunks of 4096 elements (1024 where there are few), a workgroup each, listed in a table that bsr_adamw_create()
// uploads once; a launch takes all the chunks of one kind (type, gradient's type, master copy or not), so a model of one kind
// is one launch however many tensors it has.  A wavefront takes 256 elements at a time, four neighbouring ones a lane.
//
// 8-bit moments.  The 256 elements of a wavefront share three fp32 scales:
//   m   e4m3 code times scale, scale = (largest |m|) / 448, rounded to nearest-even (a step changes m by a tenth of g - m,
//       above half a step of the code).  All zeros where the largest is below 2^-100.
//   v   code c: 0 is zero, 1 .. 255 are low * 2^((c - 1) spacing): evenly spaced in log2 v from the smallest positive v of the
//       256 (at least 2^-40 of the largest, and 2^-120) to the largest, so no larger v becomes 0, which would blow its update
//       up (and where eps would not hold that back, the elements below get no update).  A step
//       changes v by 0.1 % of g^2 - v (beta2 = 0.999), while codes are some 1 to 10 % apart: rounded to nearest, v would stop
//       after its first few dozen steps.  Between two codes the upper one is taken with the probability that keeps the mean.
// A 16-bit parameter without a master copy is rounded the same way: an update is mostly below half its last place.  The random
// bits are a hash of the seed, the step, the tensor's number and the element's, so a step can be repeated bit for bit.
//
// The stored values of W^T: the chunk's new values pass through LDS and leave in the order of W^T's blocks, 16 bytes a
// thread, where a block's size divides the chunk; for other blocks bsr_transpose_values() is launched behind.
//
// What bounds it: memory, 28 bytes an element with a master copy and fp32 moments of bf16 parameters, 30 with W^T: 40 million
// elements in 231 us, a large copy's rate.  8-bit moments without a master copy move 10, 12 with W^T, and are bound by the vector units
// (hash, logarithms, exponentials): 120 us, 93 at that rate.  0.95 million elements: 6.0 us, of which the launch is a third.
#include <algorithm>
#include <cmath>
#include <limits>
#include <memory>
#include <new>
#include <stdexcept>

#include "bsr_mfma_common.h"

using namespace bsr_dev;

namespace {

constexpr int kThreads = 256;
constexpr int kPass = 4 * kThreads;                   // elements that a workgroup takes at a time
constexpr int kPasses = 4;                            // of a chunk, one where there are few chunks
constexpr int kChunk = kPasses * kPass;
constexpr int kShared = 256;                          // elements that share scales: a wavefront's at a time
constexpr float kTop8 = 448.f;                        // largest e4m3 number
constexpr float kLeast = 0x1p-120f;                   // smallest v that 8 bits hold

// A tensor as the kernels see it.
struct tensor_desc {
    void* param;
    float* master;
    const void* grad;
    void* m;
    void* v;
    float* scales;
    void* transposed;                                 // null: none, or not written here
    const int32_t* place;                             // [stored blocks]: where each block's transpose goes
    int64_t count;
    float decay;
    uint32_t number;                                  // in the caller's list
    int32_t r_log, c_log;                             // log2 of the block's sides
    int64_t pad;
};
static_assert(sizeof(tensor_desc) == 96, "uploaded as words");

struct step_args {
    float lr, beta1, beta2, one1, one2, eps;          // one1 = 1 - beta1
    float rate, root;                                 // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t); where step_dev is null
    float log1, log2;                                 // natural logarithms of the betas
    float grad_scale;
    uint32_t key;                                     // of the seed and the step
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale_dev;
};

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

// Four neighbouring elements as loaded.  FULL: all of them are there, else the first n (any n; the others as zeros).
template <typename T> struct run4 {
    typedef T vec_t __attribute__((ext_vector_type(4)));
    vec_t v;
    template <bool FULL> __device__ __forceinline__ void load(const T* p, int n)
    {
        if (FULL || n >= 4) {
            v = *reinterpret_cast<const vec_t*>(p);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = e < n ? p[e] : (T)0;
        }
    }
    template <bool FULL> __device__ __forceinline__ void store(T* p, int n) const
    {
        if (FULL || n >= 4) {
            *reinterpret_cast<vec_t*>(p) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) p[e] = v[e];
        }
    }
};
typedef run4<uint8_t> codes4;
__device__ __forceinline__ uint32_t word_of(const codes4& c) { return __builtin_bit_cast(uint32_t, c.v); }
__device__ __forceinline__ codes4 codes_of(uint32_t w) { codes4 c; c.v = __builtin_bit_cast(codes4::vec_t, w); return c; }

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void decode_first(float (&m)[4], uint32_t codes, float scale)
{
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    m[0] = a.x * scale; m[1] = a.y * scale; m[2] = b.x * scale; m[3] = b.y * scale;
}
// (the argument's product and sum rounded each, as where a code is chosen)
__device__ __forceinline__ float second_of(float at, float start, float spacing)
{
#pragma clang fp contract(off)
    return __builtin_amdgcn_exp2f(at * spacing + start);
}
__device__ __forceinline__ void decode_second(float (&v)[4], uint32_t codes, float start, float spacing)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float c = (float)((codes >> (8 * e)) & 255u);
        v[e] = c > 0.f ? second_of(c - 1.f, start, spacing) : 0.f;
    }
}

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

// What a wavefront reads for 256 elements.  T: the parameter's type, GT: the gradient's, BITS: of the moments.
template <typename T, typename GT, int BITS, bool MASTER> struct pass_reads {
    typedef std::conditional_t<MASTER, float, T> P;   // what the parameter is read from
    typedef std::conditional_t<BITS == 32, float, uint8_t> S;
    run4<P> p;
    run4<GT> g;
    run4<S> m, v;
    float scale[3];

    template <bool FULL> __device__ __forceinline__ void fetch(const tensor_desc& d, int64_t first, int at, int n)
    {
        p.template load<FULL>(static_cast<const P*>(MASTER ? (const void*)d.master : d.param) + first + at, n);
        g.template load<FULL>(static_cast<const GT*>(d.grad) + first + at, n);
        m.template load<FULL>(static_cast<const S*>(d.m) + first + at, n);
        v.template load<FULL>(static_cast<const S*>(d.v) + first + at, n);
        if constexpr (BITS == 8)
#pragma unroll
            for (int e = 0; e < 3; ++e) scale[e] = d.scales[3 * ((first + at) / kShared) + e];
    }
};

// a x + b y, each operation rounded: moments that are held in 8 bits.  Their codes are up to a twelfth of m and a twentieth of
// v apart, so a last bit that is rounded another way can move the next update by that much.  With the sums, the arguments of
// exponentials and the quotients rounded as the formulas are written, plain fp32 arithmetic finds the same codes (of 45
// million one differed).  With fmas and reciprocals 2 of 100 000 v and 2 of a million m did, for 10 of 120 us.
__device__ __forceinline__ float weighted(float a, float x, float b, float y)
{
#pragma clang fp contract(off)
    return a * x + b * y;
}

struct step_now {                                     // a step's settings as a chunk uses them
    float beta1, beta2, eps, rate, root, keep;
    float one1, one2;                                 // (1 - beta1) scale, (1 - beta2) scale^2 for gradients times scale
    uint32_t base;
};

template <typename T, typename GT, int BITS, bool MASTER, bool FULL>
__device__ __forceinline__ void step_pass(const tensor_desc& d, const step_now& h, const pass_reads<T, GT, BITS, MASTER>& in, int64_t first, int at, int n,
                                          T* turned)
{
    float p[4], m[4], v[4];
    run4<T> stored;
    uint32_t random[4];
    if constexpr (BITS == 8) {
        decode_first(m, word_of(in.m), in.scale[0]);
        decode_second(v, word_of(in.v), in.scale[1], in.scale[2]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) { m[e] = in.m.v[e]; v[e] = in.v.v[e]; }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float g = (float)in.g.v[e];
        m[e] = BITS == 8 ? weighted(h.beta1, m[e], h.one1, g) : fmaf(h.one1, g, m[e] * h.beta1);
        v[e] = BITS == 8 ? weighted(h.beta2, v[e], h.one2 * g, g) : fmaf(h.one2 * g, g, v[e] * h.beta2);
        float size = __builtin_amdgcn_sqrtf(v[e]);
        // the root of a subnormal v would be 0 here; 2^-63, what it is below, keeps m / 0 (and 0 / 0) out where eps does not
        if constexpr (BITS == 32) size = v[e] < 0x1p-126f ? 0x1p-63f : size;
        float over = __builtin_amdgcn_rcpf(fmaf(size, h.root, h.eps));
        // what is held as 0 in 8 bits, m not: below 2^-55 or so, and nothing beside a larger eps
        if constexpr (BITS == 8)
            if (h.eps < 0x1p-40f) over = v[e] < kLeast ? 0.f : over;   // uniform
        p[e] = fmaf(-h.rate * m[e], over, (float)in.p.v[e] * h.keep);
        // fp32 numbers, of which the stored ones are roundings: left to itself the compiler rounds the exact sum to fp16
        asm("" : "+v"(p[e]));
        random[e] = mix(h.base + (uint32_t)(at + e));
        if constexpr (MASTER || std::is_same<T, float>::value) stored.v[e] = from_f32<T>(p[e]);
        else stored.v[e] = round_at_random(T{}, p[e], mix(random[e] + 0x3C6EF373u));
    }
    if (FULL || n > 0) {
        stored.template store<FULL>(static_cast<T*>(d.param) + first + at, n);
        if constexpr (MASTER) {
            run4<float> w;
            w.v = run4<float>::vec_t{p[0], p[1], p[2], p[3]};
            w.template store<FULL>(d.master + first + at, n);
        }
    }
    if (d.transposed) *reinterpret_cast<typename run4<T>::vec_t*>(turned + at) = stored.v;   // uniform
    if constexpr (BITS == 32) {
        if (FULL || n > 0) {
            run4<float> w;
            w.v = run4<float>::vec_t{m[0], m[1], m[2], m[3]};
            w.template store<FULL>(static_cast<float*>(d.m) + first + at, n);
            w.v = run4<float>::vec_t{v[0], v[1], v[2], v[3]};
            w.template store<FULL>(static_cast<float*>(d.v) + first + at, n);
        }
    } else {
        constexpr float kMost = 0x1.fffffep+127f;
        float top = 0.f;
        uint32_t top_v = 0, low_v = 0;                // low_v: the largest complement
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool mine = FULL || e < n;
            top = mine ? fmaxf(top, fabsf(m[e])) : top;
            top_v = max(top_v, mine ? bits_of(v[e]) : 0u);
            low_v = max(low_v, mine && v[e] >= kLeast ? ~bits_of(v[e]) : 0u);
        }
        const float top_m = float_of(wave_max(bits_of(top))), most = float_of(wave_max(top_v)), least = float_of(~wave_max(low_v));
        float scale[3] = {0.f, 0.f, 0x1p-12f};
        float inverse = 0.f;
        if (top_m >= 0x1p-100f) {                     // uniform
            scale[0] = top_m * (1.f / kTop8);
            inverse = __builtin_amdgcn_rcpf(scale[0]);
            inverse = fmaf(fmaf(-scale[0], inverse, 1.f), inverse, inverse);
        }
        auto quotient = [&](float x) {                // x / scale
            const float q = x * inverse;
            return fmaf(fmaf(-q, scale[0], x), inverse, q);
        };
        int packed = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(m[0]), quotient(m[1]), 0, false);
        packed = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(m[2]), quotient(m[3]), packed, true);
        if (!(most <= kMost)) {                       // a gradient that is not finite: so are the values of the whole group
            scale[1] = most;
        } else if (most >= kLeast) {                  // uniform
            scale[1] = __builtin_amdgcn_logf(fmaxf(least, most * 0x1p-40f));         // log2
            scale[2] = fmaxf((__builtin_amdgcn_logf(most) - scale[1]) * (1.f / 254.f), 0x1p-12f);
        }
        const float per = __builtin_amdgcn_rcpf(scale[2]), offset = -scale[1] * per;
        const float step = 0x1p24f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(scale[2]) - 1.f);
        uint32_t codes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float at_code = __builtin_amdgcn_fmed3f(floorf(fmaf(__builtin_amdgcn_logf(v[e]), per, offset)), 0.f, 253.f);
            // where v lies from one code to the next, times 2^24; the quotient v / below
            const float below = second_of(at_code, scale[1], scale[2]), r = __builtin_amdgcn_rcpf(below), q = v[e] * r;
            const float up = (fmaf(fmaf(-q, below, v[e]), r, q) - 1.f) * step;
            const uint32_t code = (uint32_t)at_code + 1u + ((float)(random[e] >> 8) < up ? 1u : 0u);
            codes |= (v[e] < kLeast ? 0u : code) << (8 * e);   // (a NaN has a code, of which its scales make one again)
        }
        if (FULL || n > 0) {
            codes_of((uint32_t)packed).template store<FULL>(static_cast<uint8_t*>(d.m) + first + at, n);
            codes_of(codes).template store<FULL>(static_cast<uint8_t*>(d.v) + first + at, n);
        }
        const int lane = threadIdx.x & 63;
        if (lane < 3) d.scales[3 * ((first + at) / kShared) + lane] = lane == 0 ? scale[0] : lane == 1 ? scale[1] : scale[2];
    }
}

// `passes`: of a chunk, 1024 elements each.
template <typename T, typename GT, int BITS, bool MASTER>
__global__ __launch_bounds__(kThreads) void bsr_adamw_chunks(const tensor_desc* __restrict__ tensors, const int2* __restrict__ chunks, int passes,
                                                             step_args a)
{
    __shared__ __attribute__((aligned(16))) T turned[kChunk];
    const int2 where = chunks[blockIdx.x];            // {tensor, chunk of it}
    const tensor_desc& d = tensors[where.x];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first = (int64_t)where.y * (passes * kPass);
    const int there = (int)min(d.count - first, (int64_t)(passes * kPass));   // elements of this chunk
    const int at = wave * kShared + lane * 4;         // of this lane in the first pass

    // A whole chunk's reads are all on their way before the first is used.
    typedef pass_reads<T, GT, BITS, MASTER> reads_t;
    reads_t in[kPasses];
    const bool whole = there == kChunk;
    if (whole)
#pragma unroll
        for (int q = 0; q < kPasses; ++q) in[q].template fetch<true>(d, first, at + q * kPass, 4);

    step_now h{a.beta1, a.beta2, a.eps, a.rate, a.root, 0.f, 0.f, 0.f, 0u};
    float lr = a.lr, grad_scale = a.grad_scale;
    uint32_t key = a.key;
    if (a.grad_scale_dev) {
        grad_scale = *a.grad_scale_dev;
        if (grad_scale == 0.f) return;                // the step is skipped: the whole grid leaves
    }
    h.one1 = a.one1 * grad_scale;
    h.one2 = a.one2 * grad_scale * grad_scale;
    if (a.lr_dev) lr = *a.lr_dev;
    if (a.step_dev) {
        const int64_t t = *a.step_dev;
        if (t < 1) return;                            // no such step (its corrections divide by 0): skipped, as for a scale of 0
        h.root = __builtin_amdgcn_rsqf(-expm1f((float)t * a.log2));
        h.rate = -1.f / expm1f((float)t * a.log1);
        key = step_key(a.seed, (uint64_t)t);
    }
    h.rate *= lr;
    h.keep = 1.f - lr * d.decay;
    h.base = mix(d.number + key) + (uint32_t)first;

    if (whole) {
#pragma unroll
        for (int q = 0; q < kPasses; ++q) step_pass<T, GT, BITS, MASTER, true>(d, h, in[q], first, at + q * kPass, 4, turned);
    } else {
        for (int q = 0; q < passes; ++q) {
            const int left = there - (q * kPass + wave * kShared);
            if (left <= 0) break;                     // uniform
            const int here = at + q * kPass;
            if (left >= kShared) {
                in[0].template fetch<true>(d, first, here, 4);
                step_pass<T, GT, BITS, MASTER, true>(d, h, in[0], first, here, 4, turned);
            } else {
                in[0].template fetch<false>(d, first, here, there - here);
                step_pass<T, GT, BITS, MASTER, false>(d, h, in[0], first, here, there - here, turned);
            }
        }
    }
    if (!d.transposed) return;                        // uniform
    __syncthreads();
    // Blocks are whole in the chunk.  Element e of a block of W^T is (c, a) = (e / bs_r, e mod bs_r).
    constexpr int V = 16 / (int)sizeof(T);
    const int r_log = d.r_log, c_log = d.c_log, e_log = r_log + c_log;
    T* const out = static_cast<T*>(d.transposed);
    const int64_t block0 = first >> e_log;
    if ((1 << r_log) >= V) {
        for (int u = threadIdx.x * V; u < there; u += kThreads * V) {
            const int b = u >> e_log, e = u & ((1 << e_log) - 1), c = e >> r_log, a = e & ((1 << r_log) - 1);
            typedef T tv __attribute__((ext_vector_type(V)));
            tv w;
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = turned[(b << e_log) + ((a + i) << c_log) + c];
            *reinterpret_cast<tv*>(out + ((int64_t)d.place[block0 + b] << e_log) + e) = w;
        }
    } else {
        for (int u = threadIdx.x; u < there; u += kThreads) {
            const int b = u >> e_log, e = u & ((1 << e_log) - 1), c = e >> r_log, a = e & ((1 << r_log) - 1);
            out[((int64_t)d.place[block0 + b] << e_log) + e] = turned[(b << e_log) + (a << c_log) + c];
        }
    }
}

constexpr int kOutputs = 64;                          // tensors of a launch
struct output_ptrs { void* m[kOutputs]; void* v[kOutputs]; };

// The moments as values of type O.
template <typename O, int BITS>
__global__ __launch_bounds__(kThreads) void bsr_adamw_values(const tensor_desc* __restrict__ tensors, const int2* __restrict__ chunks, int passes,
                                                             int first_tensor, output_ptrs outs)
{
    typedef std::conditional_t<BITS == 32, float, uint8_t> S;
    const int2 where = chunks[blockIdx.x];
    const tensor_desc& d = tensors[where.x];
    O* const m_out = static_cast<O*>(outs.m[where.x - first_tensor]);
    O* const v_out = static_cast<O*>(outs.v[where.x - first_tensor]);
    const int64_t first = (int64_t)where.y * (passes * kPass);
    const int there = (int)min(d.count - first, (int64_t)(passes * kPass));
    struct reads_t {
        run4<S> m, v;
        float scale[3];
    };
    auto fetch = [&](auto full, reads_t& in, int at, int n) {
        in.m.template load<decltype(full)::value>(static_cast<const S*>(d.m) + first + at, n);
        in.v.template load<decltype(full)::value>(static_cast<const S*>(d.v) + first + at, n);
        if constexpr (BITS == 8)
#pragma unroll
            for (int e = 0; e < 3; ++e) in.scale[e] = d.scales[3 * ((first + at) / kShared) + e];
    };
    auto put = [&](auto full, const reads_t& in, int at, int n) {
        float m[4], v[4];
        if constexpr (BITS == 32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { m[e] = in.m.v[e]; v[e] = in.v.v[e]; }
        } else {
            decode_first(m, word_of(in.m), in.scale[0]);
            decode_second(v, word_of(in.v), in.scale[1], in.scale[2]);
        }
        run4<O> a, b;
#pragma unroll
        for (int e = 0; e < 4; ++e) { a.v[e] = from_f32<O>(m[e]); b.v[e] = from_f32<O>(v[e]); }
        if (m_out) a.template store<decltype(full)::value>(m_out + first + at, n);
        if (v_out) b.template store<decltype(full)::value>(v_out + first + at, n);
    };
    // 256 elements a wavefront, whose scales are the same address for all lanes
    const int mine = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kShared + ((int)threadIdx.x & 63) * 4;
    if (there == kChunk) {
        reads_t in[kPasses];
#pragma unroll
        for (int q = 0; q < kPasses; ++q) fetch(std::true_type{}, in[q], mine + q * kPass, 4);
#pragma unroll
        for (int q = 0; q < kPasses; ++q) put(std::true_type{}, in[q], mine + q * kPass, 4);
        return;
    }
    for (int at = mine; at < there; at += kPass) {
        reads_t in;
        fetch(std::false_type{}, in, at, there - at);
        put(std::false_type{}, in, at, there - at);
    }
}

size_t size_of(bsr_dtype t) { return t == BSR_F32 ? 4 : 2; }
bool known(bsr_dtype t) { return (int)t >= (int)BSR_F32 && (int)t <= (int)BSR_BF16; }
size_t words_of(size_t bytes) { return (bytes + 255) / 256 * 64; }
int log2_of(int64_t v) { int l = 0; while (((int64_t)1 << l) < v) ++l; return l; }
// Whether the step's own kernel writes the transposes of such blocks: they are whole in a chunk.
bool turns(const bsr_adamw_tensor& t) { return kChunk % ((int64_t)t.bs_r * t.bs_c) == 0; }
int64_t chunks_of(int64_t count, int passes) { return (count + passes * kPass - 1) / (passes * kPass); }
// Passes of a chunk of this list: one where there would be fewer than four workgroups a CU else and every transposed block
// fits (an fp32 layer of 0.95 M elements, 30 MB: 10.8 us a call with four, 7.5 with one).
int passes_of(int64_t n, const bsr_adamw_tensor* tensors)
{
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        chunks += chunks_of(tensors[i].count, kPasses);
        if (tensors[i].t_param_dev && turns(tensors[i]) && kPass % ((int64_t)tensors[i].bs_r * tensors[i].bs_c) != 0) return kPasses;
    }
    return chunks < 1024 ? 1 : kPasses;
}
// Whether bsr_transpose_values() takes them: sides of whole 16-byte pieces, or blocks that fit its LDS.
bool transposable(const bsr_adamw_tensor& t)
{
    const int64_t u = 16 / (int64_t)size_of(t.dtype), block = (int64_t)t.bs_r * t.bs_c;
    if (t.bs_r % u == 0 && t.bs_c % u == 0 && t.count / (u * u) < ((int64_t)1 << 31)) return true;
    return block <= 32 * 1024 && (size_t)t.bs_r * (size_t)(t.bs_c + 1) * size_of(t.dtype) <= 64 * 1024;
}

struct used_range { uintptr_t from, to; bool written; };
void add_range(std::vector<used_range>& all, const void* p, size_t bytes, bool written)
{
    if (p && bytes) all.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
}
bool by_start(const used_range& a, const used_range& b) { return a.from < b.from; }
// Whether all that is written is apart from everything else of these, which are in order.
bool apart(const std::vector<used_range>& all)
{
    uintptr_t end = 0, written_end = 0;               // of what begins before
    for (const used_range& x : all) {
        if (x.from < (x.written ? end : written_end)) return false;
        end = std::max(end, x.to);
        if (x.written) written_end = std::max(written_end, x.to);
    }
    return true;
}

}  // namespace

struct bsr_adamw {
    int bits = 32, passes = kPasses, device = 0;
    std::vector<bsr_adamw_tensor> tensors;            // the caller's, in the order of the table (by kind)
    std::vector<int64_t> number;                      // their places in the caller's list
    std::vector<int32_t> first_chunk;                 // of each, and the end
    struct launch_t { int kind; int32_t first, count; };
    std::vector<launch_t> launches;
    struct behind_t { size_t tensor; const int32_t* perm; };   // transposes that are launches of their own
    std::vector<behind_t> behind;
    std::vector<used_range> ranges;                   // all buffers of the list
    const tensor_desc* descs = nullptr;               // device
    const int2* chunks = nullptr;
    std::vector<int32_t> host;                        // kept for the asynchronous upload
    hipEvent_t uploaded = nullptr;
    mutable std::atomic<bool> landed{false};
};

namespace {

// {type, gradient in fp32, master copy}
int kind_of(const bsr_adamw_tensor& t) { return ((int)t.dtype * 2 + (t.grad_dtype == BSR_F32)) * 2 + (t.master_dev != nullptr); }

bsr_status check_sizes(int64_t n, const bsr_adamw_tensor* tensors, int32_t state_bits)
{
    if (n < 0 || n >= ((int64_t)1 << 24)) return BSR_ERR_SHAPE;
    if (n > 0 && !tensors) return BSR_ERR_NULL;
    if (state_bits != 32 && state_bits != 8) return BSR_ERR_DTYPE;
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        const bsr_adamw_tensor& t = tensors[i];
        if (t.count < 0 || t.count >= ((int64_t)1 << 40)) return BSR_ERR_SHAPE;
        if (!known(t.dtype) || (t.grad_dtype != t.dtype && t.grad_dtype != BSR_F32) || (t.master_dev && t.dtype == BSR_F32)) return BSR_ERR_DTYPE;
        if (t.t_param_dev) {
            if (t.bs_r <= 0 || t.bs_c <= 0 || t.count % ((int64_t)t.bs_r * t.bs_c) != 0 ||
                t.count / ((int64_t)t.bs_r * t.bs_c) >= ((int64_t)1 << 31)) return BSR_ERR_SHAPE;
            if (!turns(t) && !transposable(t)) return BSR_ERR_UNSUPPORTED;
        }
        chunks += chunks_of(t.count, kPasses);
        if (chunks >= ((int64_t)1 << 24)) return BSR_ERR_SHAPE;   // a launch has below 2^32 threads
    }
    return BSR_OK;
}

size_t workspace_words(int64_t n, const bsr_adamw_tensor* tensors)
{
    size_t words = words_of((size_t)n * sizeof(tensor_desc)), chunks = 0;
    const int passes = passes_of(n, tensors);
    for (int64_t i = 0; i < n; ++i) {
        const bsr_adamw_tensor& t = tensors[i];
        chunks += (size_t)chunks_of(t.count, passes);
        if (t.t_param_dev) words += words_of((size_t)(t.count / ((int64_t)t.bs_r * t.bs_c)) * 4);
    }
    return std::max<size_t>(words + words_of(chunks * sizeof(int2)), 64);
}

// The buffers of a list, in order.
std::vector<used_range> ranges_of(int64_t n, const bsr_adamw_tensor* tensors, int32_t bits, const byte_range& workspace)
{
    std::vector<used_range> all;
    auto add = [&](const void* p, size_t bytes, bool written) { add_range(all, p, bytes, written); };
    add(workspace.p, workspace.bytes, true);
    for (int64_t i = 0; i < n; ++i) {
        const bsr_adamw_tensor& t = tensors[i];
        const size_t c = (size_t)t.count, s = size_of(t.dtype);
        add(t.param_dev, c * s, true);
        add(t.t_param_dev, c * s, true);
        add(t.master_dev, c * 4, true);
        add(t.exp_avg_dev, c * (size_t)(bits / 8), true);
        add(t.exp_avg_sq_dev, c * (size_t)(bits / 8), true);
        if (bits == 8) add(t.scales_dev, (c + kShared - 1) / kShared * 12, true);
        add(t.grad_dev, c * size_of(t.grad_dtype), false);
    }
    std::sort(all.begin(), all.end(), by_start);
    return all;
}

bsr_status create_adamw(bsr_adamw** out, int64_t n, const bsr_adamw_tensor* tensors, int32_t state_bits, void* workspace_dev,
                        size_t workspace_bytes, hipStream_t stream)
{
    bsr_status st = check_sizes(n, tensors, state_bits);
    if (st != BSR_OK) return st;
    if (!workspace_dev) return BSR_ERR_NULL;
    if (!aligned16(workspace_dev)) return BSR_ERR_ALIGN;
    const size_t words = workspace_words(n, tensors);
    if (workspace_bytes < words * 4) return BSR_ERR_WORKSPACE;
    for (int64_t i = 0; i < n; ++i) {
        const bsr_adamw_tensor& t = tensors[i];
        if (t.count == 0) continue;
        if (!t.param_dev || !t.grad_dev || !t.exp_avg_dev || !t.exp_avg_sq_dev || (state_bits == 8 && !t.scales_dev) ||
            (t.t_param_dev && !t.t_perm_host)) return BSR_ERR_NULL;
        for (const void* p : {(const void*)t.param_dev, (const void*)t.master_dev, t.grad_dev, (const void*)t.exp_avg_dev,
                              (const void*)t.exp_avg_sq_dev, (const void*)t.t_param_dev})
            if (!aligned16(p)) return BSR_ERR_ALIGN;
        if (reinterpret_cast<uintptr_t>(t.scales_dev) & 3u) return BSR_ERR_ALIGN;
    }
    std::unique_ptr<bsr_adamw> opt(new bsr_adamw);
    opt->ranges = ranges_of(n, tensors, state_bits, {workspace_dev, words * 4});
    if (!apart(opt->ranges)) return BSR_ERR_OVERLAP;
    opt->bits = state_bits;
    opt->passes = passes_of(n, tensors);
    std::vector<int64_t> order((size_t)n);
    for (int64_t i = 0; i < n; ++i) order[(size_t)i] = i;
    std::stable_sort(order.begin(), order.end(), [&](int64_t a, int64_t b) { return kind_of(tensors[a]) < kind_of(tensors[b]); });
    opt->host.assign(words, 0);
    int32_t* const dev = static_cast<int32_t*>(workspace_dev);
    const size_t chunks_at = words_of((size_t)n * sizeof(tensor_desc));
    size_t chunk = 0, total = 0;
    for (int64_t i = 0; i < n; ++i) total += (size_t)chunks_of(tensors[i].count, opt->passes);
    size_t at = chunks_at + words_of(total * sizeof(int2));
    for (int64_t s = 0; s < n; ++s) {
        const bsr_adamw_tensor& t = tensors[order[(size_t)s]];
        opt->first_chunk.push_back((int32_t)chunk);
        const int32_t mine = (int32_t)chunks_of(t.count, opt->passes);
        for (int32_t c = 0; c < mine; ++c, ++chunk) {
            opt->host[chunks_at + 2 * chunk] = (int32_t)s;
            opt->host[chunks_at + 2 * chunk + 1] = c;
        }
        if (mine) {
            if (opt->launches.empty() || opt->launches.back().kind != kind_of(t)) opt->launches.push_back({kind_of(t), (int32_t)chunk - mine, 0});
            opt->launches.back().count += mine;
        }
        tensor_desc d{};
        d.param = t.param_dev; d.master = t.master_dev; d.grad = t.grad_dev; d.m = t.exp_avg_dev; d.v = t.exp_avg_sq_dev;
        d.scales = t.scales_dev; d.count = t.count; d.decay = t.weight_decay; d.number = (uint32_t)order[(size_t)s];
        if (t.t_param_dev && t.count) {
            const int64_t blocks = t.count / ((int64_t)t.bs_r * t.bs_c);
            std::vector<char> seen((size_t)blocks, 0);
            const bool here = turns(t);
            for (int64_t q = 0; q < blocks; ++q) {    // block perm[q] of W goes to place q of W^T
                const int32_t p = t.t_perm_host[q];
                if (p < 0 || p >= blocks || seen[(size_t)p]) return BSR_ERR_INDEX;
                seen[(size_t)p] = 1;
                if (here) opt->host[at + (size_t)p] = (int32_t)q;
                else opt->host[at + (size_t)q] = p;
            }
            if (here) {
                d.transposed = t.t_param_dev;
                d.place = dev + at;
                d.r_log = log2_of(t.bs_r);
                d.c_log = log2_of(t.bs_c);
            } else {
                opt->behind.push_back({(size_t)s, dev + at});
            }
            at += words_of((size_t)blocks * 4);
        }
        std::memcpy(opt->host.data() + (size_t)s * (sizeof(tensor_desc) / 4), &d, sizeof d);
        opt->tensors.push_back(t);
        opt->tensors.back().t_perm_host = nullptr;    // read during the call only
        opt->number.push_back(order[(size_t)s]);
    }
    opt->first_chunk.push_back((int32_t)chunk);
    opt->descs = reinterpret_cast<const tensor_desc*>(dev);
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

template <typename T, typename GT, bool MASTER>
bsr_status launch_kind(const bsr_adamw* opt, const bsr_adamw::launch_t& l, const step_args& h, hipStream_t stream)
{
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.count), dim3(kThreads), 0, stream, opt->descs, opt->chunks + l.first, opt->passes, h);
        return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
    };
    return opt->bits == 8 ? go(bsr_adamw_chunks<T, GT, 8, MASTER>) : go(bsr_adamw_chunks<T, GT, 32, MASTER>);
}

template <typename T>
bsr_status launch_type(const bsr_adamw* opt, const bsr_adamw::launch_t& l, const step_args& h, hipStream_t stream)
{
    const bool f32_grad = (l.kind >> 1) & 1, master = l.kind & 1;
    if (master) return f32_grad ? launch_kind<T, float, true>(opt, l, h, stream) : launch_kind<T, T, true>(opt, l, h, stream);
    return f32_grad ? launch_kind<T, float, false>(opt, l, h, stream) : launch_kind<T, T, false>(opt, l, h, stream);
}

// The tables are there for what `stream` is given next.  What is recorded into a graph cannot wait for an upload outside of
// it, so a capture right behind bsr_adamw_create() waits here, on the host.
void ready_for(const bsr_adamw* opt, hipStream_t stream)
{
    if (opt->uploaded && is_capturing(stream) && !upload_landed(opt->uploaded, opt->landed)) {
        hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;      // in the default mode the wait would end the capture
        const bool swapped = hipThreadExchangeStreamCaptureMode(&mode) == hipSuccess;
        if (hipEventSynchronize(opt->uploaded) == hipSuccess) opt->landed.store(true, std::memory_order_release);
        if (swapped) (void)hipThreadExchangeStreamCaptureMode(&mode);
        (void)hipGetLastError();
    }
    order_after_upload(stream, opt->uploaded, opt->landed);
}

bool on_its_device(const bsr_adamw* opt)
{
    int dev = -1;
    return hipGetDevice(&dev) == hipSuccess && dev == opt->device;
}

}  // namespace

extern "C" {

bsr_status bsr_adamw_workspace_size(int64_t n_tensors, const bsr_adamw_tensor* tensors, int32_t state_bits, size_t* bytes)
{
    if (!bytes) return BSR_ERR_NULL;
    *bytes = 0;
    const bsr_status st = check_sizes(n_tensors, tensors, state_bits);
    if (st == BSR_OK) *bytes = workspace_words(n_tensors, tensors) * 4;
    return st;
}

bsr_status bsr_adamw_create(bsr_adamw** out, int64_t n_tensors, const bsr_adamw_tensor* tensors, int32_t state_bits, void* workspace_dev,
                            size_t workspace_bytes, void* hip_stream)
{
    if (!out) return BSR_ERR_NULL;
    *out = nullptr;
    try {
        return create_adamw(out, n_tensors, tensors, state_bits, workspace_dev, workspace_bytes, (hipStream_t)hip_stream);
    } catch (const std::bad_alloc&) {                 // no host memory for the tables
        return BSR_ERR_HIP;
    } catch (const std::length_error&) {
        return BSR_ERR_SHAPE;
    }
}

void bsr_adamw_destroy(bsr_adamw* opt)
{
    if (!opt) return;
    if (opt->uploaded) {                              // the upload reads the handle's host buffer
        (void)hipEventSynchronize(opt->uploaded);
        (void)hipEventDestroy(opt->uploaded);
        (void)hipGetLastError();
    }
    delete opt;
}

bsr_status bsr_adamw_step(const bsr_adamw* opt, const bsr_adamw_hyper* hyper, void* hip_stream)
{
    if (!opt || !hyper) return BSR_ERR_NULL;
    const bsr_adamw_hyper& y = *hyper;
    // (negated: NaN is refused too)
    if (!(y.beta1 >= 0 && y.beta1 < 1) || !(y.beta2 >= 0 && y.beta2 < 1) || !(y.eps >= 0) || (!y.step_dev && y.step < 1) ||
        (!y.lr_dev && !(y.lr >= 0))) return BSR_ERR_SHAPE;
    const float size = std::fabs(y.grad_scale);       // its square has to be an fp32 number, with room for 1 - beta2
    if (!y.grad_scale_dev && !(size == 0.f || (size >= 0x1p-40f && size <= 0x1p40f))) return BSR_ERR_SHAPE;
    for (const void* p : {(const void*)y.lr_dev, (const void*)y.grad_scale_dev})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return BSR_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(y.step_dev) & 7u) return BSR_ERR_ALIGN;
    if (!on_its_device(opt)) return BSR_ERR_DEVICE;
    hipStream_t stream = (hipStream_t)hip_stream;
    ready_for(opt, stream);
    step_args h{};
    h.lr = (float)y.lr;
    h.beta1 = (float)y.beta1;
    h.beta2 = (float)y.beta2;
    h.one1 = (float)(1.0 - y.beta1);
    h.one2 = (float)(1.0 - y.beta2);
    h.eps = (float)y.eps;
    h.log1 = (float)std::log(y.beta1);
    h.log2 = (float)std::log(y.beta2);
    if (!y.step_dev) {
        h.rate = (float)(1.0 / (1.0 - std::pow(y.beta1, (double)y.step)));
        h.root = (float)(1.0 / std::sqrt(1.0 - std::pow(y.beta2, (double)y.step)));
        h.key = step_key(y.seed, (uint64_t)y.step);
    }
    h.grad_scale = y.grad_scale;
    h.seed = y.seed;
    h.lr_dev = y.lr_dev;
    h.step_dev = y.step_dev;
    h.grad_scale_dev = y.grad_scale_dev;
    if (!y.grad_scale_dev && y.grad_scale == 0.f) return BSR_OK;
    for (const auto& l : opt->launches) {
        const int type = l.kind >> 2;
        const bsr_status st = type == BSR_F32 ? launch_kind<float, float, false>(opt, l, h, stream)
                            : type == BSR_F16 ? launch_type<f16_t>(opt, l, h, stream) : launch_type<bf16_t>(opt, l, h, stream);
        if (st != BSR_OK) return st;
    }
    for (const auto& b : opt->behind) {
        const bsr_adamw_tensor& t = opt->tensors[b.tensor];
        const bsr_status st = bsr_transpose_values(t.dtype, t.bs_r, t.bs_c, t.count / ((int64_t)t.bs_r * t.bs_c), b.perm, t.param_dev,
                                                   t.t_param_dev, hip_stream);
        if (st != BSR_OK) return st;
    }
    return BSR_OK;
}

bsr_status bsr_adamw_moments(const bsr_adamw* opt, bsr_dtype dtype, void* const* exp_avg_out, void* const* exp_avg_sq_out, void* hip_stream)
{
    if (!opt || !exp_avg_out || !exp_avg_sq_out) return BSR_ERR_NULL;
    if (!known(dtype)) return BSR_ERR_DTYPE;
    const size_t n = opt->tensors.size();
    for (size_t i = 0; i < n; ++i)
        if (!aligned16(exp_avg_out[i]) || !aligned16(exp_avg_sq_out[i])) return BSR_ERR_ALIGN;
    try {
        std::vector<used_range> outs, all;
        for (size_t i = 0; i < n; ++i)
            for (const void* p : {(const void*)exp_avg_out[opt->number[i]], (const void*)exp_avg_sq_out[opt->number[i]]})
                add_range(outs, p, (size_t)opt->tensors[i].count * size_of(dtype), true);
        std::sort(outs.begin(), outs.end(), by_start);
        all.resize(outs.size() + opt->ranges.size());
        std::merge(outs.begin(), outs.end(), opt->ranges.begin(), opt->ranges.end(), all.begin(), by_start);
        if (!apart(all)) return BSR_ERR_OVERLAP;
    } catch (const std::bad_alloc&) {
        return BSR_ERR_HIP;
    }
    if (!on_its_device(opt)) return BSR_ERR_DEVICE;
    hipStream_t stream = (hipStream_t)hip_stream;
    ready_for(opt, stream);
    for (size_t s = 0; s < n; s += kOutputs) {
        const size_t end = std::min(n, s + kOutputs);
        const int32_t first = opt->first_chunk[s], count = opt->first_chunk[end] - first;
        if (count == 0) continue;
        output_ptrs outs{};
        for (size_t i = s; i < end; ++i) {
            outs.m[i - s] = exp_avg_out[opt->number[i]];
            outs.v[i - s] = exp_avg_sq_out[opt->number[i]];
        }
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(kThreads), 0, stream, opt->descs, opt->chunks + first, opt->passes, (int)s, outs);
            return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
        };
        const bool eight = opt->bits == 8;
        const bsr_status st = dtype == BSR_F32 ? (eight ? go(bsr_adamw_values<float, 8>) : go(bsr_adamw_values<float, 32>))
                            : dtype == BSR_F16 ? (eight ? go(bsr_adamw_values<f16_t, 8>) : go(bsr_adamw_values<f16_t, 32>))
                                               : (eight ? go(bsr_adamw_values<bf16_t, 8>) : go(bsr_adamw_values<bf16_t, 32>));
        if (st != BSR_OK) return st;
    }
    return BSR_OK;
}

}  // extern "C"
