// The layer norm of rows and its gradient.
#include "layer_internal.cuh"

namespace {

// A team of threads has a row: a warp (8 rows a block) or the whole block.  Its threads hold the row as accesses of N elements, NV each,
// a team's width apart.
constexpr int kWarps = 8;

// The sums of a[0] .. a[M - 1] over the team, the same in every thread, in an order that the team's size alone decides.
// sum: kM x 32 floats of shared memory; two calls in a row use different ones.
template <bool kWarp, int M>
__device__ __forceinline__ void team_sums(float (&a)[M], float* sum)
{
#pragma unroll
    for (int m = 0; m < M; ++m) a[m] = layer_warp_sum(a[m]);
    if constexpr (!kWarp) {
        const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
        if (lane == 0) {
#pragma unroll
            for (int m = 0; m < M; ++m) sum[m * 32 + warp] = a[m];
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) a[m] = layer_warp_sum(lane < warps ? sum[m * 32 + lane] : 0.0f);
    }
}

// N parameters from element `at` on, of which n are there, as binary32; `otherwise` where there is no array.
template <int N>
__device__ __forceinline__ void load_params(float (&p)[N], const void* a, uint32_t ptype, uint64_t at, int n, float otherwise)
{
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = otherwise;
    if (a == nullptr) return;
    if (ptype == PEARL_F32) {
        const float* f = (const float*)a + at;
        if (N >= 4 && n >= N && ((uintptr_t)f & 15u) == 0) {
#pragma unroll
            for (int i = 0; i + 3 < N; i += 4) {
                const float4 v = *reinterpret_cast<const float4*>(f + i);
                p[i] = v.x; p[i + 1] = v.y; p[i + 2] = v.z; p[i + 3] = v.w;
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = f[i];
        return;
    }
    const uint16_t* b = (const uint16_t*)a + at;
    if (N == 8 && n >= N && ((uintptr_t)b & 15u) == 0) {
        const uint4 v = *reinterpret_cast<const uint4*>(b);
        const uint32_t w[4] = { v.x, v.y, v.z, v.w };
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 f = ptype == PEARL_F16 ? RowsElem<__half>::up2(w[i]) : RowsElem<__nv_bfloat16>::up2(w[i]);
            p[2 * i] = f.x;
            p[2 * i + 1] = f.y;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) p[i] = ptype == PEARL_F16 ? __half2float(__ushort_as_half(b[i])) : __uint_as_float((uint32_t)b[i] << 16);
}

// ---- forward ---------------------------------------------------------------------------------------------------------
// One pass over memory: a row is in registers while its mean, then the mean of the squared differences from it, are formed.
template <typename E, int N, int NV, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kWarps * 32 : 1024) norm_kernel(uint32_t T, uint32_t D, const E* x, uint64_t ld_x, uint32_t ptype,
                                                                          const void* gamma, const void* beta, float eps, E* y, uint64_t ld_y,
                                                                          float* mean_out, float* rstd_out)
{
    __shared__ float sums[2 * 32];
    rows_begin();
    const uint32_t team = kWarp ? 32u : blockDim.x, me = kWarp ? threadIdx.x & 31u : threadIdx.x;
    const uint64_t t = kWarp ? (uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5) : blockIdx.x;
    if (kWarp && t >= T) return;
    RowsVec<E, N> v[NV];
    const E* row = x + t * ld_x;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const uint32_t at = (j * team + me) * N;
        v[j] = layer_load_part<E, N>(row + at, (int)D - (int)at);
    }
    float s[1] = { 0.0f };
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] += v[j].get(i);
    team_sums<kWarp>(s, sums);
    const float mean = s[0] / (float)D;
    s[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int n = (int)D - (int)((j * team + me) * N);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = v[j].get(i) - mean;
            if (i < n) s[0] = __fmaf_rn(d, d, s[0]);
        }
    }
    team_sums<kWarp>(s, sums + 32);
    const float rstd = 1.0f / sqrtf(s[0] / (float)D + eps);
    if (me == 0) {
        if (mean_out) mean_out[t] = mean;
        if (rstd_out) rstd_out[t] = rstd;
    }
    E* to = y + t * ld_y;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const uint32_t at = (j * team + me) * N;
        const int n = (int)D - (int)at;
        if (n <= 0) continue;
        float g[N], b[N];
        load_params<N>(g, gamma, ptype, at, n, 1.0f);
        load_params<N>(b, beta, ptype, at, n, 0.0f);
        float out[N];
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = __fmaf_rn((v[j].get(i) - mean) * rstd, g[i], b[i]);
        RowsVec<E, N> o;
        o.set(out);
        layer_store_part<E, N>(to + at, o, n);
    }
}

// Rows that are too long for a block's registers: read three times.
template <typename E, int N>
__global__ void __launch_bounds__(1024) norm_long_kernel(uint32_t D, const E* x, uint64_t ld_x, uint32_t ptype, const void* gamma,
                                                         const void* beta, float eps, E* y, uint64_t ld_y, float* mean_out, float* rstd_out)
{
    __shared__ float sums[2 * 32];
    rows_begin();
    const uint64_t t = blockIdx.x;
    const E* row = x + t * ld_x;
    float s[1] = { 0.0f };
    for (uint32_t at = threadIdx.x * N; at < D; at += blockDim.x * N) {
        const RowsVec<E, N> v = layer_load_part<E, N>(row + at, (int)D - (int)at);
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] += v.get(i);
    }
    team_sums<false>(s, sums);
    const float mean = s[0] / (float)D;
    s[0] = 0.0f;
    for (uint32_t at = threadIdx.x * N; at < D; at += blockDim.x * N) {
        const RowsVec<E, N> v = layer_load_part<E, N>(row + at, (int)D - (int)at);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = v.get(i) - mean;
            if (i < (int)D - (int)at) s[0] = __fmaf_rn(d, d, s[0]);
        }
    }
    team_sums<false>(s, sums + 32);
    const float rstd = 1.0f / sqrtf(s[0] / (float)D + eps);
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[t] = mean;
        if (rstd_out) rstd_out[t] = rstd;
    }
    for (uint32_t at = threadIdx.x * N; at < D; at += blockDim.x * N) {
        const int n = (int)D - (int)at;
        const RowsVec<E, N> v = layer_load_part<E, N>(row + at, n);
        float g[N], b[N], out[N];
        load_params<N>(g, gamma, ptype, at, n, 1.0f);
        load_params<N>(b, beta, ptype, at, n, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = __fmaf_rn((v.get(i) - mean) * rstd, g[i], b[i]);
        RowsVec<E, N> o;
        o.set(out);
        layer_store_part<E, N>(y + t * ld_y + at, o, n);
    }
}

// ---- gradient --------------------------------------------------------------------------------------------------------
// A block goes over every gridDim.x-th row (or group of kWarps rows); its threads hold the sums of dy * n and dy of their columns, which
// end as the block's line of `work`: [blocks][2][D].
template <typename E, int N, int NV, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kWarps * 32 : 1024)
    norm_grad_kernel(unsigned* status, uint32_t T, uint32_t D, const E* dy, uint64_t ld_dy, const E* x, uint64_t ld_x, const float* mean,
                     const float* rstd, uint32_t ptype, const void* gamma, E* dx, uint64_t ld_dx, float* work, const float* work_end)
{
    extern __shared__ float shared[];                  // kWarp: 2 * D for the warps' sums
    __shared__ float sums[2][2 * 32];
    rows_begin();
    const uint32_t team = kWarp ? 32u : blockDim.x, me = kWarp ? threadIdx.x & 31u : threadIdx.x;
    const uint64_t step = (uint64_t)gridDim.x * (kWarp ? kWarps : 1);
    uint64_t t = kWarp ? (uint64_t)blockIdx.x * kWarps + (threadIdx.x >> 5) : blockIdx.x;
    float dg[NV][N], db[NV][N];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) dg[j][i] = db[j][i] = 0.0f;
    const float part = 1.0f / (float)D;
    for (uint32_t odd = 0; t < T; t += step, odd ^= 1u) {
        RowsVec<E, N> a[NV], b[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t at = (j * team + me) * N;
            a[j] = layer_load_part<E, N>(dy + t * ld_dy + at, (int)D - (int)at);
            b[j] = layer_load_part<E, N>(x + t * ld_x + at, (int)D - (int)at);
        }
        const float m = mean[t], r = rstd[t];
        float s[2] = { 0.0f, 0.0f };
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t at = (j * team + me) * N;
            const int n = (int)D - (int)at;
            float g[N];
            load_params<N>(g, gamma, ptype, at, n, 1.0f);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i >= n) break;
                const float d = a[j].get(i), norm = (b[j].get(i) - m) * r, w = d * g[i];
                dg[j][i] = __fmaf_rn(d, norm, dg[j][i]);
                db[j][i] += d;
                s[0] += w;
                s[1] = __fmaf_rn(w, norm, s[1]);
            }
        }
        if (dx == nullptr) continue;
        team_sums<kWarp>(s, sums[odd]);
        const float along = s[1] * part, off = s[0] * part;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t at = (j * team + me) * N;
            const int n = (int)D - (int)at;
            if (n <= 0) continue;
            float g[N], out[N];
            load_params<N>(g, gamma, ptype, at, n, 1.0f);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float norm = (b[j].get(i) - m) * r;
                out[i] = r * (__fmaf_rn(a[j].get(i), g[i], -off) - norm * along);
            }
            RowsVec<E, N> o;
            o.set(out);
            layer_store_part<E, N>(dx + t * ld_dx + at, o, n);
        }
    }
    if (work == nullptr) return;
    float* line = work + (uint64_t)blockIdx.x * 2 * D;
    if constexpr (kWarp) {
        for (uint32_t w = 0; w < kWarps; ++w) {            // the warps' sums, one warp after the other
            if (threadIdx.x >> 5 == w) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const uint32_t c = (j * 32 + me) * N + i;
                        if (c >= D) continue;
                        shared[c] = w ? shared[c] + dg[j][i] : dg[j][i];
                        shared[D + c] = w ? shared[D + c] + db[j][i] : db[j][i];
                    }
            }
            __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < 2 * D; c += blockDim.x)
            if (ROWS_IN_ARRAY(status, line + c, 4, work, work_end)) line[c] = shared[c];
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t c = (j * team + me) * N + i;
                if (c >= D || !ROWS_IN_ARRAY(status, line + D + c, 4, work, work_end)) continue;
                line[c] = dg[j][i];
                line[D + c] = db[j][i];
            }
    }
}

// Rows that are too long for a block's registers: read twice; the columns' sums are the block's line of `work` itself.
template <typename E, int N>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(unsigned* status, uint32_t T, uint32_t D, const E* dy, uint64_t ld_dy, const E* x,
                                                              uint64_t ld_x, const float* mean, const float* rstd, uint32_t ptype,
                                                              const void* gamma, E* dx, uint64_t ld_dx, float* work, const float* work_end)
{
    __shared__ float sums[2][2 * 32];
    rows_begin();
    const float part = 1.0f / (float)D;
    float* line = work + (uint64_t)blockIdx.x * 2 * D;
    bool first = true;
    uint32_t odd = 0;
    for (uint64_t t = blockIdx.x; t < T; t += gridDim.x, odd ^= 1u) {
        const float m = mean[t], r = rstd[t];
        float s[2] = { 0.0f, 0.0f };
        for (uint32_t at = threadIdx.x * N; at < D; at += blockDim.x * N) {
            const int n = (int)D - (int)at;
            const RowsVec<E, N> a = layer_load_part<E, N>(dy + t * ld_dy + at, n), b = layer_load_part<E, N>(x + t * ld_x + at, n);
            float g[N];
            load_params<N>(g, gamma, ptype, at, n, 1.0f);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i >= n) break;
                const float d = a.get(i), norm = (b.get(i) - m) * r, w = d * g[i];
                s[0] += w;
                s[1] = __fmaf_rn(w, norm, s[1]);
                if (work && ROWS_IN_ARRAY(status, line + D + at + i, 4, work, work_end)) {
                    line[at + i] = __fmaf_rn(d, norm, first ? 0.0f : line[at + i]);
                    line[D + at + i] = d + (first ? 0.0f : line[D + at + i]);
                }
            }
        }
        first = false;
        if (dx == nullptr) continue;
        team_sums<false>(s, sums[odd]);
        const float along = s[1] * part, off = s[0] * part;
        for (uint32_t at = threadIdx.x * N; at < D; at += blockDim.x * N) {
            const int n = (int)D - (int)at;
            const RowsVec<E, N> a = layer_load_part<E, N>(dy + t * ld_dy + at, n), b = layer_load_part<E, N>(x + t * ld_x + at, n);
            float g[N], out[N];
            load_params<N>(g, gamma, ptype, at, n, 1.0f);
#pragma unroll
            for (int i = 0; i < N; ++i) out[i] = r * (__fmaf_rn(a.get(i), g[i], -off) - (b.get(i) - m) * r * along);
            RowsVec<E, N> o;
            o.set(out);
            layer_store_part<E, N>(dx + t * ld_dx + at, o, n);
        }
    }
}

// dgamma and dbeta: the blocks' lines added up.  A block has 32 columns of the two; its 32 warps take every 32nd line each, then one adds
// the warps' sums in order.
__global__ void __launch_bounds__(1024) norm_params_kernel(uint32_t D, uint32_t lines, const float* work, float* dgamma, float* dbeta)
{
    __shared__ float sums[32][33];
    rows_begin();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t c = blockIdx.x * 32 + lane;
    const bool bias = blockIdx.y != 0;
    float s = 0.0f;
    if (c < D)
        for (uint32_t l = warp; l < lines; l += 32) s += work[((uint64_t)l * 2 + bias) * D + c];
    sums[warp][lane] = s;
    __syncthreads();
    s = layer_warp_sum(sums[lane][warp]);
    const uint32_t col = blockIdx.x * 32 + warp;
    float* to = bias ? dbeta : dgamma;
    if (lane == 0 && col < D && to) to[col] = s;
}

// ---- which kernel ----------------------------------------------------------------------------------------------------
// How a row of `cols` accesses is held.
struct Shape {
    int nv;                 // accesses of a thread; 0: too many
    bool warp;
    uint32_t threads;       // of a block
};
Shape shape_of(uint32_t cols, int most)
{
    if (cols <= 32) return { 1, true, kWarps * 32 };
    if (cols <= 128) return { 4, true, kWarps * 32 };
    int nv = 1;
    while (nv < most && cols > 512u * nv) nv *= 2;
    const uint32_t threads = ((cols + nv - 1) / nv + 31) / 32 * 32;
    return threads <= 1024 ? Shape{ nv, false, threads } : Shape{ 0, false, 1024 };
}

struct NormArgs {
    uint32_t T, D, ptype;
    const void *x, *gamma, *beta;
    uint64_t ld_x, ld_y;
    float eps;
    void* y;
    float *mean, *rstd;
};
template <typename E, int N> int norm_as(const NormArgs& a, cudaStream_t s)
{
    const Shape f = shape_of((a.D + N - 1) / N, 8);
    const uint32_t blocks = f.warp ? (uint32_t)(((uint64_t)a.T + kWarps - 1) / kWarps) : a.T;
#define NORM(NV, WARP)                                                                                                                       \
    rows_launch(norm_kernel<E, N, NV, WARP>, dim3(blocks), dim3(f.threads), 0, s, 0, a.T, a.D, (const E*)a.x, a.ld_x, a.ptype, a.gamma, a.beta, \
                a.eps, (E*)a.y, a.ld_y, a.mean, a.rstd)
    if (f.warp) return f.nv == 1 ? NORM(1, true) : NORM(4, true);
    switch (f.nv) {
        case 1: return NORM(1, false);
        case 2: return NORM(2, false);
        case 4: return NORM(4, false);
        case 8: return NORM(8, false);
    }
#undef NORM
    return rows_launch(norm_long_kernel<E, N>, dim3(a.T), dim3(1024), 0, s, 0, a.D, (const E*)a.x, a.ld_x, a.ptype, a.gamma, a.beta, a.eps, (E*)a.y,
                       a.ld_y, a.mean, a.rstd);
}

struct GradArgs {
    uint32_t T, D, ptype;
    const void *dy, *x, *gamma;
    uint64_t ld_dy, ld_x, ld_dx;
    const float *mean, *rstd;
    void* dx;
    float *dgamma, *dbeta, *work;
    const float* work_end;
    unsigned* status;
};
constexpr uint32_t kLines = 296;       // of work at most: two blocks for each of 148 SMs

template <typename E, int N> int grad_as(const GradArgs& a, cudaStream_t s)
{
    const Shape f = shape_of((a.D + N - 1) / N, 4);
    const bool params = a.dgamma || a.dbeta;
    const uint64_t groups = f.warp ? ((uint64_t)a.T + kWarps - 1) / kWarps : a.T;
    const uint32_t lines = (uint32_t)(groups < kLines ? groups : kLines);
    int n = 0;
    if (lines) {
        float* work = params ? a.work : nullptr;
#define GRAD(NV, WARP)                                                                                                                            \
    rows_launch(norm_grad_kernel<E, N, NV, WARP>, dim3(lines), dim3(f.threads), WARP ? 2 * a.D * sizeof(float) : 0, s, 0, a.status, a.T, a.D,      \
                (const E*)a.dy, a.ld_dy, (const E*)a.x, a.ld_x, a.mean, a.rstd, a.ptype, a.gamma, (E*)a.dx, a.ld_dx, work, a.work_end)
        if (f.warp) n = f.nv == 1 ? GRAD(1, true) : GRAD(4, true);
        else if (f.nv == 1) n = GRAD(1, false);
        else if (f.nv == 2) n = GRAD(2, false);
        else if (f.nv == 4) n = GRAD(4, false);
        else
            n = rows_launch(norm_grad_long_kernel<E, N>, dim3(lines), dim3(1024), 0, s, 0, a.status, a.T, a.D, (const E*)a.dy, a.ld_dy, (const E*)a.x,
                            a.ld_x, a.mean, a.rstd, a.ptype, a.gamma, (E*)a.dx, a.ld_dx, work, a.work_end);
#undef GRAD
        if (n < 0) return n;
    }
    if (!params) return n;
    const int m = rows_launch(norm_params_kernel, dim3((a.D + 31) / 32, 2), dim3(1024), 0, s, 0, a.D, lines, (const float*)a.work, a.dgamma, a.dbeta);
    return m < 0 ? m : n + m;
}

// Runs CALL(type, elements of an access) for rows whose addresses and distances are multiples of `granule` bytes.
#define WITH_ACCESS(dtype, granule, CALL)                          \
    do {                                                           \
        if ((dtype) == PEARL_F32) {                                \
            if ((granule) >= 16) { CALL(float, 4); }               \
            else { CALL(float, 1); }                               \
        } else if ((dtype) == PEARL_F16) {                         \
            if ((granule) >= 16) { CALL(__half, 8); }              \
            else if ((granule) >= 4) { CALL(__half, 2); }          \
            else { CALL(__half, 1); }                              \
        } else {                                                   \
            if ((granule) >= 16) { CALL(__nv_bfloat16, 8); }       \
            else if ((granule) >= 4) { CALL(__nv_bfloat16, 2); }   \
            else { CALL(__nv_bfloat16, 1); }                       \
        }                                                          \
    } while (0)

}  // namespace

int layer_launch_norm(uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, uint32_t ptype, const void* gamma, const void* beta,
                      float eps, void* y, uint64_t ld_y, float* mean, float* rstd, cudaStream_t s)
{
    const NormArgs a = { T, D, ptype, x, gamma, beta, ld_x, ld_y, eps, y, mean, rstd };
    const uint32_t S = rows_elem_bytes(dtype), granule = rows_granule((uintptr_t)x, (uintptr_t)y, ld_x * S, ld_y * S);
#define NORM_AS(E, N) return norm_as<E, N>(a, s)
    WITH_ACCESS(dtype, granule, NORM_AS);
#undef NORM_AS
}

uint64_t layer_norm_grad_work_bytes(uint32_t T, uint32_t D) { return (T < 1 ? 1u : T < kLines ? T : kLines) * 2ull * D * sizeof(float); }

int layer_launch_norm_grad(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x,
                           const float* mean, const float* rstd, uint32_t ptype, const void* gamma, void* dx, uint64_t ld_dx, float* dgamma,
                           float* dbeta, float* work, uint64_t work_bytes, cudaStream_t s)
{
    const GradArgs a = { T, D, ptype, dy, x, gamma, ld_dy, ld_x, ld_dx, mean, rstd, dx, dgamma, dbeta, work,
                         (const float*)((const char*)work + work_bytes), status };
    const uint32_t S = rows_elem_bytes(dtype);
    const uint32_t granule = rows_granule((uintptr_t)dy | (uintptr_t)x, (uintptr_t)dx, ld_dy * S, ld_x * S, ld_dx * S);
#define GRAD_AS(E, N) return grad_as<E, N>(a, s)
    WITH_ACCESS(dtype, granule, GRAD_AS);
#undef GRAD_AS
}
