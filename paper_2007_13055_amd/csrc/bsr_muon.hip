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
// What bounds it: up to 16x16 blocks memory (22 bytes an element for bf16 with a master copy and W^T), beyond that the matrix
// cores' fp32 rate: 5 (4 L S^2 + 2 S^3) operations a block.
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
    uint32_t key;                                     // of the seed and the step
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale_dev;
};

// Wavefronts of a workgroup, a block each: as many as 64 KB of LDS hold, four at most.
constexpr int waves_of(int rt, int ct) { return rt * ct > 8 ? 2 : 4; }

template <typename T> __device__ __forceinline__ f32x4 load_as(const void* p, size_t at, int count, bool whole)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    const T* const from = static_cast<const T*>(p) + at;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (whole) {
        if (count >= 4) {
            const t4 t = *reinterpret_cast<const t4*>(from);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (float)t[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < count) v[e] = (float)from[e];
    }
    return v;
}
// Up to four neighbouring elements of a tensor of any type; `whole`: four or none, at a multiple of their size.
__device__ __forceinline__ f32x4 load4(const void* p, int dtype, size_t at, int count, bool whole)
{
    if (dtype == BSR_F32) return load_as<float>(p, at, count, whole);    // uniform
    if (dtype == BSR_F16) return load_as<f16_t>(p, at, count, whole);
    return load_as<bf16_t>(p, at, count, whole);
}
template <typename T> __device__ __forceinline__ void put4(T* to, const T (&v)[4], int count, bool whole)
{
    typedef T t4 __attribute__((ext_vector_type(4)));
    if (whole) {
        if (count >= 4) *reinterpret_cast<t4*>(to) = t4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < count) to[e] = v[e];
    }
}

// RT, CT: 16x16 tiles of a block down and across.
template <int RT, int CT>
__global__ __launch_bounds__(64 * waves_of(RT, CT)) void bsr_muon_blocks(const muon_desc* __restrict__ tensors, const int2* __restrict__ chunks, muon_args h)
{
    constexpr int WAVES = waves_of(RT, CT);
    constexpr bool TALL = RT > CT;
    constexpr int L = TALL ? RT : CT, S = TALL ? CT : RT;
    constexpr int PW = S * 16 + 4, PY = RT * 16 + 4;  // pitches in LDS of W [L * 16][] and, where the block is turned, of its transpose
    constexpr int AREA = std::max(L * 16 * PW, TALL ? CT * 16 * PY : 0);
    __shared__ __attribute__((aligned(16))) float areas[WAVES][AREA];
    const int lane = threadIdx.x & 63, i = lane & 15, c0 = (lane >> 4) * 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int2 where = chunks[blockIdx.x];            // {tensor, first block}
    const muon_desc& d = tensors[where.x];
    const int64_t block = (int64_t)where.y + wave;
    if (block >= d.blocks) return;                    // (no barrier below)
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

    const int bs_r = d.bs_r, bs_c = d.bs_c;
    const size_t first = (size_t)block * (size_t)(bs_r * bs_c);
    const bool whole = (bs_c & 3) == 0;
    // a lane's elements of tile (J, I): row 16 I + i of the block, columns 16 J + c0 .. + 3
    auto count_of = [&](int J, int I) { return 16 * I + i < bs_r ? bs_c - (16 * J + c0) : 0; };
    auto place_of = [&](int J, int I) { return (16 * I + i) * bs_c + 16 * J + c0; };

    f32x4 y[CT][RT];                                  // the block's transpose in result tiles
    uint32_t top = 0;
#pragma unroll
    for (int J = 0; J < CT; ++J)
#pragma unroll
        for (int I = 0; I < RT; ++I) {
            const int count = count_of(J, I);
            const size_t at = first + (size_t)place_of(J, I);
            f32x4 g = load4(d.grad, d.grad_dtype, at, count, whole), m = load4(d.momentum, BSR_F32, at, count, whole);
            float mv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g[e] *= grad_scale;
                mv[e] = fmaf(h.mu, m[e], g[e]);
                y[J][I][e] = h.nesterov ? fmaf(h.mu, mv[e], g[e]) : mv[e];
                top = max(top, bits_of(fabsf(y[J][I][e])));
            }
            put4(d.momentum + at, mv, count, whole);
        }
    // |V|, of V times a power of two that keeps the squares fp32 numbers
    {
        const int exponent = __builtin_amdgcn_frexp_expf(float_of(wave_max(top)));
        float sum = 0.f;
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = ldexpf(y[J][I][e], -exponent);
                    sum = fmaf(v, v, sum);
                }
        sum += __builtin_bit_cast(float, dpp<0xB1>(bits_of(sum)));
        sum += __builtin_bit_cast(float, dpp<0x4E>(bits_of(sum)));
        sum += __builtin_bit_cast(float, dpp<0x141>(bits_of(sum)));
        sum += __builtin_bit_cast(float, dpp<0x140>(bits_of(sum)));
        sum += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle((int)bits_of(sum), 0x401F));
        sum = __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)bits_of(sum), 0)) +
              __builtin_bit_cast(float, __builtin_amdgcn_readlane((int)bits_of(sum), 32));
        const float inverse = 1.f / (ldexpf(sqrtf(sum), exponent) + h.eps);
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) y[J][I] *= inverse;
    }

    f32x4 w[L][S];
    if constexpr (TALL) {
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I)
#pragma unroll
                for (int e = 0; e < 4; ++e) area[(16 * J + c0 + e) * PY + 16 * I + i] = y[J][I][e];
        wave_lds_fence();
#pragma unroll
        for (int I = 0; I < RT; ++I)
#pragma unroll
            for (int J = 0; J < CT; ++J) w[I][J] = *reinterpret_cast<const f32x4*>(&area[(16 * J + i) * PY + 16 * I + c0]);
        wave_lds_fence();
    } else {
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) w[J][I] = y[J][I];
    }
    auto put_w = [&]() {
        wave_lds_fence();                             // the other lanes have read what was there
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) area[(16 * l + c0 + e) * PW + 16 * s + i] = w[l][s][e];
        wave_lds_fence();
    };
    auto turned = [&](int s, int l) { return *reinterpret_cast<const f32x4*>(&area[(16 * l + i) * PW + 16 * s + c0]); };   // tile (s, l) of W^T

    for (int step = 0; step < h.ns_steps; ++step) {
        put_w();
        f32x4 g[S][S], p[S][S];
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int t = 0; t < S; ++t) g[s][t] = p[s][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int l = 0; l < L; ++l)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int s = 0; s < S; ++s)
#pragma unroll
                    for (int t = 0; t < S; ++t) g[s][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[l][s][e], w[l][t][e], g[s][t], 0, 0, 0);
#pragma unroll
        for (int k = 0; k < S; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int s = 0; s < S; ++s)
#pragma unroll
                    for (int t = 0; t < S; ++t) p[s][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(g[k][s][e], g[k][t][e], p[s][t], 0, 0, 0);
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int t = 0; t < S; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) p[s][t][e] = fmaf(h.b, g[s][t][e], h.c * p[s][t][e]);
#pragma unroll
        for (int l = 0; l < L; ++l) {
            f32x4 wt[S];
#pragma unroll
            for (int k = 0; k < S; ++k) wt[k] = turned(k, l);
#pragma unroll
            for (int t = 0; t < S; ++t) w[l][t] *= h.a;
#pragma unroll
            for (int k = 0; k < S; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t = 0; t < S; ++t) w[l][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(wt[k][e], p[k][t][e], w[l][t], 0, 0, 0);
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

    const float keep = 1.f - lr * d.decay, rate = lr * d.scale;
    const uint32_t base = mix(d.number + key) + (uint32_t)first;
    const size_t to = d.transposed ? (size_t)d.place[block] * (size_t)(bs_r * bs_c) : 0;
    auto update = [&](auto type, auto has_master) {
        typedef decltype(type) T;
        constexpr bool MASTER = decltype(has_master)::value;
#pragma unroll
        for (int J = 0; J < CT; ++J)
#pragma unroll
            for (int I = 0; I < RT; ++I) {
                const int count = count_of(J, I), place = place_of(J, I);
                const size_t at = first + (size_t)place;
                const f32x4 p = load_as<std::conditional_t<MASTER, float, T>>(MASTER ? (const void*)d.master : d.param, at, count, whole);
                float v[4];
                T out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = fmaf(-rate, y[J][I][e], p[e] * keep);
                    asm("" : "+v"(v[e]));             // an fp32 number, of which the stored one is the rounding
                    if constexpr (MASTER || std::is_same<T, float>::value) out[e] = from_f32<T>(v[e]);
                    else out[e] = round_at_random(T{}, v[e], mix(base + (uint32_t)(place + e)));
                }
                put4(static_cast<T*>(d.param) + at, out, count, whole);
                if constexpr (MASTER) put4(d.master + at, v, count, whole);
                if (d.transposed) {                   // uniform
                    T* const t = static_cast<T*>(d.transposed) + to + (size_t)((16 * J + c0) * bs_r + 16 * I + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < count) t[e * bs_r] = out[e];
                }
            }
    };
    auto update_type = [&](auto type) {
        if (d.master) update(type, std::true_type{});
        else update(type, std::false_type{});
    };
    if (d.dtype == BSR_F32) update(0.f, std::false_type{});
    else if (d.dtype == BSR_F16) update_type(f16_t{});
    else update_type(bf16_t{});
}

int tiles_of(int32_t side) { return (side + 15) / 16; }
int kind_of(const bsr_muon_tensor& t) { return (tiles_of(t.bs_r) - 1) * 4 + tiles_of(t.bs_c) - 1; }
int chunk_of(const bsr_muon_tensor& t) { return waves_of(tiles_of(t.bs_r), tiles_of(t.bs_c)); }   // blocks of a workgroup
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

template <int RT, int CT> bsr_status launch_tiles(const bsr_muon* opt, const bsr_muon::launch_t& l, const muon_args& h, hipStream_t stream)
{
    hipLaunchKernelGGL((bsr_muon_blocks<RT, CT>), dim3((unsigned)l.count), dim3(64 * waves_of(RT, CT)), 0, stream, opt->descs, opt->chunks + l.first, h);
    return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
}
template <int RT> bsr_status launch_rows(const bsr_muon* opt, const bsr_muon::launch_t& l, const muon_args& h, hipStream_t stream)
{
    switch (l.kind % 4) {
        case 0: return launch_tiles<RT, 1>(opt, l, h, stream);
        case 1: return launch_tiles<RT, 2>(opt, l, h, stream);
        case 2: return launch_tiles<RT, 3>(opt, l, h, stream);
    }
    return launch_tiles<RT, 4>(opt, l, h, stream);
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
    if (!y.step_dev) h.key = step_key(y.seed, (uint64_t)y.step);
    h.seed = y.seed;
    h.lr_dev = y.lr_dev;
    h.step_dev = y.step_dev;
    h.grad_scale_dev = y.grad_scale_dev;
    for (const auto& l : opt->launches) {
        const int rt = l.kind / 4;
        const bsr_status st = rt == 0 ? launch_rows<1>(opt, l, h, stream) : rt == 1 ? launch_rows<2>(opt, l, h, stream)
                            : rt == 2 ? launch_rows<3>(opt, l, h, stream) : launch_rows<4>(opt, l, h, stream);
        if (st != BSR_OK) return st;
    }
    return BSR_OK;
}

}  // extern "C"
