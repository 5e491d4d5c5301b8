// The gradient of the product's epilogue:  dZ = G * act'(Z),  db[j] = sum over i of dZ[i][j]  (fp32, before its rounding).
//
// One pass over G and Z: a lane keeps V neighbouring columns, 16 bytes of G, and walks down the rows of its workgroup's chunk,
// storing dZ and adding up V sums in registers.  A strip of columns is 256 bytes wide (fp32: 512), so that a workgroup has 16
// (8) rows in flight and leaves one partial sum for all of them: the fewer partial sums, the less the second launch has to
// read, which adds them in a fixed order (no atomics, the same bits every time).  Rows need not begin at multiples of 16 bytes;
// the lane at their end takes its last elements one by one.
//
// What bounds it: memory.  It moves 2 or 3 matrices and computes some 25 operations an element.  Measured, gelu, us (and of
// the rate of a large copy, 5.2 TB/s): 8192 x 8192 bf16 84 (93 %), fp32 145 (107 %), 4096 x 4096 bf16 25.5 (76 %), 16384 x 1024
// f16 27 (71 %), 2048 x 2048 bf16 10.6 (46 %: two launches, 2 us each by themselves).  Strips of 1024 bytes: 92, 163, 28, 37, 15.
// Chunks for 1024 workgroups in place of 4096: 92, 147, 26, 27, 11; four rows' loads in flight in place of two: no gain.  Rows
// that begin anywhere take longer, their pieces crossing lines: 8191 x 8191 bf16 168 (element by element 228).
#include <algorithm>

#include "bsr_epilogue.h"

using namespace bsr_dev;

namespace {

constexpr int kThreads = 256;

struct backward_shape {
    int lpr_log;                                      // log2 of the lanes of a row of a strip
    int strips, chunks, rows;                         // workgroups along n and m, rows of a chunk
};

constexpr int kMostChunks = 256;

// The split of an m x n matrix, v columns a lane.
backward_shape split(int64_t m, int64_t n, int v)
{
    backward_shape s{0, 1, 1, 0};
    const int64_t units = (n + v - 1) / v;
    while (s.lpr_log < (v == 8 ? 4 : 5) && (1 << s.lpr_log) < units) ++s.lpr_log;
    s.strips = (int)((units + (1 << s.lpr_log) - 1) >> s.lpr_log);
    const int64_t slots = kThreads >> s.lpr_log;      // rows in flight
    // up to 4096 workgroups of at least four rows a lane; two where there would not be two workgroups a CU else
    auto at_least = [&](int64_t rows) { return (m + rows * slots - 1) / (rows * slots); };
    int64_t chunks = std::min<int64_t>(std::max(4096 / s.strips, 1), at_least(4));
    chunks = std::max<int64_t>(chunks, std::min<int64_t>(512 / s.strips, at_least(2)));
    chunks = std::min<int64_t>(std::max<int64_t>(chunks, 1), kMostChunks);
    s.rows = (int)((m + chunks - 1) / chunks);
    s.rows = (int)((s.rows + slots - 1) / slots * slots);
    s.chunks = (int)((m + s.rows - 1) / s.rows);
    return s;
}

// V elements at any multiple of their size, of which `count` are there (the others as zeros, and not stored).
template <typename T, int V> __device__ __forceinline__ void load_any(float (&v)[V], const T* p, int count)
{
    typedef T vec_t __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (count >= V) {
        const vec_t t = *reinterpret_cast<const vec_t*>(p);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (float)t[e];
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = e < count ? (float)p[e] : 0.f;
    }
}
template <typename T, int V> __device__ __forceinline__ void store_any(T* p, const float (&v)[V], int count)
{
    typedef T vec_t __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    if (count >= V) {
        vec_t t;
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = from_f32<T>(v[e]);
        *reinterpret_cast<vec_t*>(p) = t;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e < count) p[e] = from_f32<T>(v[e]);
    }
}

template <typename G, typename O, bool SUMS>
__global__ __launch_bounds__(kThreads) void bsr_backward_pass(const G* g, const G* z, O* dz, float* __restrict__ partial,
                                                              int m, int n, int lpr_log, int rows, int act)
{
    constexpr int V = 16 / (int)sizeof(G);
    __shared__ float red[SUMS ? kThreads * V : 1];
    const int tid = threadIdx.x, lpr = 1 << lpr_log, slots = kThreads >> lpr_log;
    const int col = (int)((blockIdx.x << lpr_log) + (tid & (lpr - 1))) * V, count = n - col;
    const int first = (int)blockIdx.y * rows, end = min(first + rows, m);
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    if (count > 0) {
        constexpr int U = 2;                          // rows whose loads are in flight
        const int step = slots;
        int i = first + (tid >> lpr_log);
        auto rows_of = [&](auto k, int i) {
            constexpr int K = decltype(k)::value;
            float gv[K][V], zv[K][V];
#pragma unroll
            for (int u = 0; u < K; ++u) {
                const size_t at = (size_t)(i + u * step) * (size_t)n + (size_t)col;
                load_any(gv[u], g + at, count);
                if (z) load_any(zv[u], z + at, count);
            }
            if (z)
                with_act(act, [&](auto a) {
#pragma unroll
                    for (int u = 0; u < K; ++u)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            gv[u][e] *= act_slope<decltype(a)::value>(zv[u][e]);
                            // an fp32 number whether or not it is summed: without the sums the compiler would round the
                            // exact product to fp16 in one instruction, and dZ would hang on what else is wanted
                            asm("" : "+v"(gv[u][e]));
                        }
                });
#pragma unroll
            for (int u = 0; u < K; ++u) {
                if (dz) store_any(dz + (size_t)(i + u * step) * (size_t)n + (size_t)col, gv[u], count);
                if constexpr (SUMS)
#pragma unroll
                    for (int e = 0; e < V; ++e) sum[e] += gv[u][e];
            }
        };
        for (; i + (U - 1) * step < end; i += U * step) rows_of(std::integral_constant<int, U>{}, i);
        for (; i < end; i += step) rows_of(std::integral_constant<int, 1>{}, i);
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int e = 0; e < V; ++e) red[tid * V + e] = sum[e];
        for (int half = kThreads / 2; half >= lpr; half >>= 1) {
            __syncthreads();
            if (tid < half)
#pragma unroll
                for (int e = 0; e < V; ++e) red[tid * V + e] += red[(tid + half) * V + e];
        }
        __syncthreads();
        for (int t = tid; t < lpr * V; t += kThreads) {
            const int c = (int)(blockIdx.x << lpr_log) * V + t;
            if (c < n) partial[(size_t)blockIdx.y * (size_t)n + c] = red[t];
        }
    }
}

// db[j] = sum of partial[c][j] over the chunks: 16 columns a workgroup, 16 shares of the chunks.
constexpr int kSumCols = 16;
__global__ __launch_bounds__(256) void bsr_backward_sums(const float* __restrict__ partial, float* __restrict__ db, int n, int chunks)
{
    __shared__ float red[16][kSumCols];
    const int at = threadIdx.x % kSumCols, share = threadIdx.x / kSumCols, col = (int)blockIdx.x * kSumCols + at;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (col < n) {
        int c = share;
        for (; c + 48 < chunks; c += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] += partial[(size_t)(c + 16 * u) * (size_t)n + col];
        for (; c < chunks; c += 16) v[0] += partial[(size_t)c * (size_t)n + col];
    }
    red[share][at] = (v[0] + v[1]) + (v[2] + v[3]);
    __syncthreads();
    if (share == 0 && col < n) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 4) s += (red[i][at] + red[i + 1][at]) + (red[i + 2][at] + red[i + 3][at]);
        db[col] = s;
    }
}

template <typename G, typename O>
bsr_status launch_types(const backward_shape& s, int64_t m, int64_t n, bsr_act act, const void* g, const void* z, void* dz, float* db,
                        float* ws, hipStream_t stream)
{
    float* out = s.chunks > 1 ? ws : db;
    auto go = [&](auto sums) -> bsr_status {
        hipLaunchKernelGGL((bsr_backward_pass<G, O, decltype(sums)::value>), dim3((unsigned)s.strips, (unsigned)s.chunks), dim3(kThreads), 0,
                           stream, (const G*)g, (const G*)z, (O*)dz, out, (int)m, (int)n, s.lpr_log, s.rows, (int)act);
        return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
    };
    const bsr_status st = db ? go(std::true_type{}) : go(std::false_type{});
    if (st != BSR_OK || !db || s.chunks == 1) return st;
    hipLaunchKernelGGL(bsr_backward_sums, dim3((unsigned)((n + kSumCols - 1) / kSumCols)), dim3(256), 0, stream, ws, db, (int)n, s.chunks);
    return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
}

bool sizes_fit(int64_t m, int64_t n) { return m >= 0 && n >= 0 && m < ((int64_t)1 << 30) && n < ((int64_t)1 << 28); }

}  // namespace

extern "C" {

bsr_status bsr_epilogue_backward_workspace_size(int64_t m, int64_t n, size_t* bytes)
{
    if (!bytes) return BSR_ERR_NULL;
    *bytes = 0;
    if (!sizes_fit(m, n)) return BSR_ERR_SHAPE;
    if (m == 0 || n == 0) return BSR_OK;
    const int chunks = std::max(split(m, n, 4).chunks, split(m, n, 8).chunks);   // whatever the type
    if (chunks > 1) *bytes = ((size_t)chunks * (size_t)n * sizeof(float) + 255) & ~(size_t)255;
    return BSR_OK;
}

bsr_status bsr_epilogue_backward(int64_t m, int64_t n, bsr_act act, bsr_dtype g_dtype, const void* G_dev, const void* Z_dev,
                                 bsr_dtype dz_dtype, void* DZ_dev, float* DB_dev, void* workspace_dev, size_t workspace_bytes,
                                 void* hip_stream)
{
    if (!sizes_fit(m, n)) return BSR_ERR_SHAPE;
    if ((int)g_dtype < 0 || (int)g_dtype > (int)BSR_BF16 || (int)dz_dtype < 0 || (int)dz_dtype > (int)BSR_BF16 || !known_act(act))
        return BSR_ERR_DTYPE;
    if (dz_dtype != g_dtype && g_dtype != BSR_F32) return BSR_ERR_DTYPE;
    if (n == 0) return BSR_OK;
    if (m > 0 && (!G_dev || (act != BSR_ACT_NONE && !Z_dev))) return BSR_ERR_NULL;
    if (!DZ_dev && !DB_dev) return BSR_ERR_NULL;
    if (m > 0 && n >= ((int64_t)1 << 40) / m) return BSR_ERR_SHAPE;
    const void* Z = act == BSR_ACT_NONE ? nullptr : Z_dev;
    for (const void* p : {G_dev, Z, (const void*)DZ_dev, (const void*)DB_dev, (const void*)workspace_dev})
        if (!aligned16(p)) return BSR_ERR_ALIGN;
    hipStream_t stream = (hipStream_t)hip_stream;
    if (m == 0) {                                     // no rows: the sums are zero
        if (!DB_dev) return BSR_OK;
        hipLaunchKernelGGL(bsr_backward_sums, dim3((unsigned)((n + kSumCols - 1) / kSumCols)), dim3(256), 0, stream, DB_dev, DB_dev, (int)n, 0);
        return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
    }
    const backward_shape s = split(m, n, g_dtype == BSR_F32 ? 4 : 8);
    size_t need = DB_dev && s.chunks > 1 ? (size_t)s.chunks * (size_t)n * sizeof(float) : 0;
    if (need && (!workspace_dev || workspace_bytes < need)) return BSR_ERR_WORKSPACE;
    const size_t elements = (size_t)m * (size_t)n, g_size = g_dtype == BSR_F32 ? 4 : 2, dz_size = dz_dtype == BSR_F32 ? 4 : 2;
    const byte_range g{G_dev, elements * g_size}, z{Z, elements * g_size}, dz{DZ_dev, elements * dz_size},
        db{DB_dev, (size_t)n * sizeof(float)}, ws{need ? workspace_dev : nullptr, need};
    // dZ may take the place of G or of Z, element by element
    const bool in_place = dz_dtype == g_dtype;
    if ((overlap(dz, g) && !(in_place && DZ_dev == G_dev)) || (overlap(dz, z) && !(in_place && DZ_dev == Z))) return BSR_ERR_OVERLAP;
    for (const byte_range& r : {g, z, dz})
        if (overlap(db, r) || overlap(ws, r)) return BSR_ERR_OVERLAP;
    if (overlap(db, ws)) return BSR_ERR_OVERLAP;
    float* part = static_cast<float*>(workspace_dev);
    if (g_dtype == BSR_F16) return launch_types<f16_t, f16_t>(s, m, n, act, G_dev, Z, DZ_dev, DB_dev, part, stream);
    if (g_dtype == BSR_BF16) return launch_types<bf16_t, bf16_t>(s, m, n, act, G_dev, Z, DZ_dev, DB_dev, part, stream);
    if (dz_dtype == BSR_F16) return launch_types<float, f16_t>(s, m, n, act, G_dev, Z, DZ_dev, DB_dev, part, stream);
    if (dz_dtype == BSR_BF16) return launch_types<float, bf16_t>(s, m, n, act, G_dev, Z, DZ_dev, DB_dev, part, stream);
    return launch_types<float, float>(s, m, n, act, G_dev, Z, DZ_dev, DB_dev, part, stream);
}

}  // extern "C"
