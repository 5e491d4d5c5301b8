// A gate and what it multiplies, H = act(z_g) z_u, where a product has left both in memory; and its gradient,
//
//     dz_g = G z_u act'(z_g)      dz_u = G act(z_g)      db[j] = sum over i of dZ[i][j]      (fp32, before its rounding).
//
// z is kept in the order of W's block-rows, `unit` columns of z_g and `unit` of z_u in turn, so a lane that takes V
// neighbouring columns of H (V divides unit: 16 bytes of G where it can) reads and writes three runs at offsets that it works
// out once; it walks down the rows of its workgroup's chunk with them.  The gradient adds up 2 V sums in registers; a workgroup
// leaves one partial sum for its rows, and a second launch adds those in a fixed order (no atomics).
//
// What bounds both: memory.
#include <algorithm>

#include "bsr_epilogue.h"

using namespace bsr_dev;

namespace {

constexpr int kThreads = 256;
constexpr int kMostChunks = 256;

struct gate_shape {
    int lpr_log;                                      // log2 of the lanes of a row of a strip
    int strips, chunks, rows;                         // workgroups along n and m, rows of a chunk
};

// The split of m x n results, v columns a lane.
gate_shape split(int64_t m, int64_t n, int v)
{
    gate_shape s{0, 1, 1, 0};
    const int64_t units = n / v;                      // v divides n
    while (s.lpr_log < 5 && (1 << s.lpr_log) < units) ++s.lpr_log;
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

// Columns a lane: the largest power of two that divides unit, 16 bytes of the narrower type at most.
int run_of_unit(int64_t unit, int most)
{
    int v = 1;
    while (v < most && unit % (2 * v) == 0) v *= 2;
    return v;
}

// V elements, at a multiple of their size.
template <typename T, int V> __device__ __forceinline__ void load_v(float (&v)[V], const T* p)
{
    typedef T vec_t __attribute__((ext_vector_type(V)));
    const vec_t t = *reinterpret_cast<const vec_t*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (float)t[e];
}
template <typename T> __device__ __forceinline__ void load_v(float (&v)[1], const T* p) { v[0] = (float)*p; }
template <typename T, int V> __device__ __forceinline__ void store_v(T* p, const float (&v)[V])
{
    typedef T vec_t __attribute__((ext_vector_type(V)));
    vec_t t;
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = from_f32<T>(v[e]);
    *reinterpret_cast<vec_t*>(p) = t;
}
template <typename T> __device__ __forceinline__ void store_v(T* p, const float (&v)[1]) { *p = from_f32<T>(v[0]); }

// Z's fp32 sums to H and, rounded, to z_out.
template <typename O, int V>
__global__ __launch_bounds__(kThreads) void bsr_gate_pass(const float* __restrict__ z, O* __restrict__ h, O* __restrict__ z_out, int m, int n, int unit,
                                                          int lpr_log, int rows, int act)
{
    const int lpr = 1 << lpr_log, slots = kThreads >> lpr_log;
    const int col = (int)((blockIdx.x << lpr_log) + (threadIdx.x & (lpr - 1))) * V;
    if (col >= n) return;
    const int gate = col / unit * unit + col;         // 2 unit (col / unit) + col mod unit
    const int first = (int)blockIdx.y * rows, end = min(first + rows, m);
    with_act_or_none(act, [&](auto a) {
        for (int i = first + (int)(threadIdx.x >> lpr_log); i < end; i += slots) {
            const size_t row = (size_t)i * (size_t)n;
            float g[V], u[V], y[V];
            load_v(g, z + 2 * row + gate);
            load_v(u, z + 2 * row + gate + unit);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                y[e] = act_value<decltype(a)::value>(g[e]) * u[e];
                asm("" : "+v"(y[e]));                 // an fp32 number: left to itself the compiler rounds the exact product to fp16
            }
            store_v(h + row + col, y);
            if (z_out) {
                store_v(z_out + 2 * row + gate, g);
                store_v(z_out + 2 * row + gate + unit, u);
            }
        }
    });
}

template <typename G, typename O, int V, bool SUMS>
__global__ __launch_bounds__(kThreads) void bsr_gated_backward_pass(const G* g, const G* z, O* dz, float* __restrict__ partial, int m, int n, int unit,
                                                                    int lpr_log, int rows, int act)
{
    __shared__ float red[SUMS ? kThreads * V : 1];
    const int tid = threadIdx.x, lpr = 1 << lpr_log, slots = kThreads >> lpr_log;
    const int col = (int)((blockIdx.x << lpr_log) + (tid & (lpr - 1))) * V;
    const int gate = col < n ? col / unit * unit + col : 0;
    const int first = (int)blockIdx.y * rows, end = min(first + rows, m);
    float sum[2][V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[0][e] = sum[1][e] = 0.f;
    if (col < n)
        with_act_or_none(act, [&](auto a) {
            constexpr int U = 2;                      // rows whose loads are in flight
            const int step = slots;
            int i = first + (tid >> lpr_log);
            auto rows_of = [&](auto k, int i) {
                constexpr int K = decltype(k)::value;
                float gv[K][V], zg[K][V], zu[K][V];
#pragma unroll
                for (int q = 0; q < K; ++q) {
                    const size_t row = (size_t)(i + q * step) * (size_t)n;
                    load_v(gv[q], g + row + col);
                    load_v(zg[q], z + 2 * row + gate);
                    load_v(zu[q], z + 2 * row + gate + unit);
                }
#pragma unroll
                for (int q = 0; q < K; ++q) {
                    float dg[V], du[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        dg[e] = gv[q][e] * zu[q][e] * act_slope<decltype(a)::value>(zg[q][e]);
                        du[e] = gv[q][e] * act_value<decltype(a)::value>(zg[q][e]);
                        asm("" : "+v"(dg[e]), "+v"(du[e]));   // fp32 numbers, whether or not they are summed
                    }
                    if (dz) {
                        const size_t row = 2 * (size_t)(i + q * step) * (size_t)n;
                        store_v(dz + row + gate, dg);
                        store_v(dz + row + gate + unit, du);
                    }
                    if constexpr (SUMS)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            sum[0][e] += dg[e];
                            sum[1][e] += du[e];
                        }
                }
            };
            for (; i + (U - 1) * step < end; i += U * step) rows_of(std::integral_constant<int, U>{}, i);
            for (; i < end; i += step) rows_of(std::integral_constant<int, 1>{}, i);
        });
    if constexpr (SUMS) {
#pragma unroll
        for (int half_z = 0; half_z < 2; ++half_z) {
            if (half_z) __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) red[tid * V + e] = sum[half_z][e];
            for (int half = kThreads / 2; half >= lpr; half >>= 1) {
                __syncthreads();
                if (tid < half)
#pragma unroll
                    for (int e = 0; e < V; ++e) red[tid * V + e] += red[(tid + half) * V + e];
            }
            __syncthreads();
            for (int t = tid; t < lpr * V; t += kThreads) {
                const int c = (int)(blockIdx.x << lpr_log) * V + t;
                if (c < n) partial[2 * (size_t)blockIdx.y * (size_t)n + (size_t)(c / unit * unit + c + half_z * unit)] = red[t];
            }
        }
    }
}

// Calls f(columns a lane as a constant).
template <int MOST, typename F> bsr_status with_run(int v, F f)
{
    if constexpr (MOST >= 8)
        if (v == 8) return f(std::integral_constant<int, 8>{});
    if (v == 4) return f(std::integral_constant<int, 4>{});
    if (v == 2) return f(std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1>{});
}

template <typename G, typename O>
bsr_status launch_types(const gate_shape& s, int v, int64_t m, int64_t n, int32_t unit, bsr_act act, const void* g, const void* z, void* dz, float* db,
                        float* ws, hipStream_t stream)
{
    float* out = s.chunks > 1 ? ws : db;
    const bsr_status st = with_run<sizeof(G) == 4 ? 4 : 8>(v, [&](auto run) {
        constexpr int V = decltype(run)::value;
        auto go = [&](auto sums) -> bsr_status {
            hipLaunchKernelGGL((bsr_gated_backward_pass<G, O, V, decltype(sums)::value>), dim3((unsigned)s.strips, (unsigned)s.chunks), dim3(kThreads), 0,
                               stream, (const G*)g, (const G*)z, (O*)dz, out, (int)m, (int)n, (int)unit, s.lpr_log, s.rows, (int)act);
            return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
        };
        return db ? go(std::true_type{}) : go(std::false_type{});
    });
    if (st != BSR_OK || !db || s.chunks == 1) return st;
    return launch_backward_sums(ws, db, 2 * n, s.chunks, stream);
}

bool sizes_fit(int64_t m, int64_t n, int32_t unit)
{
    return m >= 0 && n >= 0 && unit >= 1 && m < ((int64_t)1 << 30) && n < ((int64_t)1 << 27) && n % unit == 0;
}

}  // namespace

bsr_status launch_gate_pass(int64_t m, int64_t n, int32_t unit, bsr_act act, const float* z, bsr_dtype h_dtype, void* h, void* z_out, hipStream_t stream)
{
    const int v = run_of_unit(unit, 4);
    const gate_shape s = split(m, n, v);
    auto go = [&](auto type) {
        typedef decltype(type) O;
        return with_run<4>(v, [&](auto run) {
            hipLaunchKernelGGL((bsr_gate_pass<O, decltype(run)::value>), dim3((unsigned)s.strips, (unsigned)s.chunks), dim3(kThreads), 0, stream, z, (O*)h,
                               (O*)z_out, (int)m, (int)n, (int)unit, s.lpr_log, s.rows, (int)act);
            return hipGetLastError() == hipSuccess ? BSR_OK : BSR_ERR_HIP;
        });
    };
    return h_dtype == BSR_F32 ? go(0.f) : h_dtype == BSR_F16 ? go(f16_t{}) : go(bf16_t{});
}

extern "C" {

bsr_status bsr_gated_backward_workspace_size(int64_t m, int64_t n, int32_t unit, size_t* bytes)
{
    if (!bytes) return BSR_ERR_NULL;
    *bytes = 0;
    if (!sizes_fit(m, n, unit)) return BSR_ERR_SHAPE;
    if (m == 0 || n == 0) return BSR_OK;
    const int chunks = std::max(split(m, n, run_of_unit(unit, 4)).chunks, split(m, n, run_of_unit(unit, 8)).chunks);   // whatever the type
    if (chunks > 1) *bytes = ((size_t)chunks * (size_t)n * 2 * sizeof(float) + 255) & ~(size_t)255;
    return BSR_OK;
}

bsr_status bsr_gated_backward(int64_t m, int64_t n, int32_t unit, bsr_act act, bsr_dtype g_dtype, const void* G_dev, const void* Z_dev,
                              bsr_dtype dz_dtype, void* DZ_dev, float* DB_dev, void* workspace_dev, size_t workspace_bytes, void* hip_stream)
{
    if (!sizes_fit(m, n, unit)) return BSR_ERR_SHAPE;
    if ((int)g_dtype < 0 || (int)g_dtype > (int)BSR_BF16 || (int)dz_dtype < 0 || (int)dz_dtype > (int)BSR_BF16 || !known_act(act)) return BSR_ERR_DTYPE;
    if (dz_dtype != g_dtype && g_dtype != BSR_F32) return BSR_ERR_DTYPE;
    if (n == 0) return BSR_OK;
    if ((m > 0 && (!G_dev || !Z_dev)) || (!DZ_dev && !DB_dev)) return BSR_ERR_NULL;
    if (m > 0 && n >= ((int64_t)1 << 39) / m) return BSR_ERR_SHAPE;
    for (const void* p : {G_dev, Z_dev, (const void*)DZ_dev, (const void*)DB_dev, (const void*)workspace_dev})
        if (!aligned16(p)) return BSR_ERR_ALIGN;
    hipStream_t stream = (hipStream_t)hip_stream;
    if (m == 0) return DB_dev ? launch_backward_sums(DB_dev, DB_dev, 2 * n, 0, stream) : BSR_OK;   // no rows: the sums are zero
    const int v = run_of_unit(unit, g_dtype == BSR_F32 ? 4 : 8);
    const gate_shape s = split(m, n, v);
    const size_t need = DB_dev && s.chunks > 1 ? (size_t)s.chunks * (size_t)n * 2 * sizeof(float) : 0;
    if (need && (!workspace_dev || workspace_bytes < need)) return BSR_ERR_WORKSPACE;
    const size_t elements = (size_t)m * (size_t)n, g_size = g_dtype == BSR_F32 ? 4 : 2, dz_size = dz_dtype == BSR_F32 ? 4 : 2;
    const byte_range g{G_dev, elements * g_size}, z{Z_dev, 2 * elements * g_size}, dz{DZ_dev, 2 * elements * dz_size},
        db{DB_dev, (size_t)n * 2 * sizeof(float)}, ws{need ? workspace_dev : nullptr, need};
    // dZ may take the place of Z, element by element
    if (overlap(dz, g) || (overlap(dz, z) && !(dz_dtype == g_dtype && DZ_dev == Z_dev))) return BSR_ERR_OVERLAP;
    for (const byte_range& r : {g, z, dz})
        if (overlap(db, r) || overlap(ws, r)) return BSR_ERR_OVERLAP;
    if (overlap(db, ws)) return BSR_ERR_OVERLAP;
    float* part = static_cast<float*>(workspace_dev);
    if (g_dtype == BSR_F16) return launch_types<f16_t, f16_t>(s, v, m, n, unit, act, G_dev, Z_dev, DZ_dev, DB_dev, part, stream);
    if (g_dtype == BSR_BF16) return launch_types<bf16_t, bf16_t>(s, v, m, n, unit, act, G_dev, Z_dev, DZ_dev, DB_dev, part, stream);
    if (dz_dtype == BSR_F16) return launch_types<float, f16_t>(s, v, m, n, unit, act, G_dev, Z_dev, DZ_dev, DB_dev, part, stream);
    if (dz_dtype == BSR_BF16) return launch_types<float, bf16_t>(s, v, m, n, unit, act, G_dev, Z_dev, DZ_dev, DB_dev, part, stream);
    return launch_types<float, float>(s, v, m, n, unit, act, G_dev, Z_dev, DZ_dev, DB_dev, part, stream);
}

}  // extern "C"
