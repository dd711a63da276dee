// Rows to the experts and back: dispatch, combine and the gradient of combine.
#include "rows_internal.cuh"

namespace {

constexpr uint32_t kThreads = 256;

// How a block of threads covers rows of `cols` accesses each: `across` threads along a row, `down` rows; where a row has more
// than a block's threads the grid's y covers its parts, all of one length within an access.
struct Tiling {
    uint32_t across, down, parts;
    dim3 grid, block;
};
Tiling tile(uint32_t rows, uint32_t cols)
{
    Tiling t;
    t.parts = (cols + kThreads - 1) / kThreads;
    t.across = (cols + t.parts - 1) / t.parts;
    t.down = kThreads / t.across;
    t.grid = dim3((rows + t.down - 1) / t.down, t.parts);
    t.block = dim3((t.across * t.down + 31) / 32 * 32);
    return t;
}

// The places of KC slots from `first` on, -1 where there is none or it is out of range (which is reported once a slot).
template <int KC>
__device__ __forceinline__ void load_places(unsigned* status, const int32_t* place, uint32_t n, uint32_t sorted_rows, bool report,
                                            int32_t (&at)[KC])
{
    bool bad = false;
#pragma unroll
    for (int j = 0; j < KC; ++j) at[j] = rows_read_if((uint32_t)j < n, place + j, -1);
#pragma unroll
    for (int j = 0; j < KC; ++j)
        if ((uint32_t)at[j] >= sorted_rows) {
            bad |= at[j] != -1;
            at[j] = -1;
        }
    if (bad && report) atomicOr(status, PEARL_ST_BAD_INDEX);
}

// ---- dispatch --------------------------------------------------------------------------------------------------------
// xs[place[t, j]] = x[t].  A thread reads its access of row t once and writes it k times: (1 + k) rows of traffic for k
// copies, bound by HBM's writes: 131048 rows of 4 KB from 16381 in 96 us, 6.3 TB/s.  (Two or four rows a thread: 99 us; 16-byte accesses:
// 101.)
template <int B, int KC>
__global__ void __launch_bounds__(kThreads) dispatch_kernel(unsigned* status, uint32_t T, uint32_t k, uint32_t cols, uint32_t across,
                                                            uint32_t down, const unsigned char* x, uint64_t ld_x,
                                                            const int32_t* place, uint32_t sorted_rows,
                                                            unsigned char* xs)
{
    rows_begin();
    const uint32_t in = threadIdx.x / across;
    const uint32_t col = threadIdx.x - in * across + blockIdx.y * across;
    const uint64_t t = (uint64_t)blockIdx.x * down + in;
    if (in >= down || t >= T || col >= cols) return;
    RowsRaw<B> v;
    rows_load_if<false>(true, v, x + t * ld_x + (uint64_t)col * B);
    for (uint32_t j0 = 0; j0 < k; j0 += KC) {
        int32_t at[KC];
        load_places<KC>(status, place + t * k + j0, k - j0, sorted_rows, col == 0, at);
#pragma unroll
        for (int j = 0; j < KC; ++j)
            if (at[j] >= 0) rows_store(xs + ((uint64_t)(uint32_t)at[j] * cols + col) * B, v);
    }
}

// The same where rows start at odd bytes or odd 2-byte places: a thread has a 16-byte word of each of the k destinations.
template <int S, int KC>
__global__ void __launch_bounds__(kThreads) dispatch_any_kernel(unsigned* status, uint32_t T, uint32_t k, uint32_t row_bytes, uint32_t cols, uint32_t across,
                                                                uint32_t down, const unsigned char* x, uint64_t ld_x,
                                                                const int32_t* place, uint32_t sorted_rows, unsigned char* xs)
{
    rows_begin();
    const uint32_t in = threadIdx.x / across;
    const uint32_t col = threadIdx.x - in * across + blockIdx.y * across;
    const uint64_t t = (uint64_t)blockIdx.x * down + in;
    if (in >= down || t >= T || col >= cols) return;
    const unsigned char *row = x + t * ld_x, *end = x + (T - 1) * ld_x + row_bytes;
    for (uint32_t j0 = 0; j0 < k; j0 += KC) {
        int32_t at[KC];
        load_places<KC>(status, place + t * k + j0, k - j0, sorted_rows, col == 0, at);
        RowsAny<S> v[KC];
        int shift[KC];
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            // the word's first byte is byte 16 col - shift of the row
            shift[j] = at[j] < 0 ? 0 : (int)((uint32_t)(uintptr_t)(xs + (uint64_t)(uint32_t)at[j] * row_bytes) & 15u);
            if (at[j] >= 0 && (int)(col * 16) - shift[j] >= (int)row_bytes) at[j] = -1;
            v[j].fetch(status, at[j] >= 0, row + (int)(col * 16) - shift[j], x, end);
        }
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            if (at[j] < 0) continue;
            const int first = (int)(col * 16) - shift[j];
            rows_store_part<S>(status, xs + (uint64_t)(uint32_t)at[j] * row_bytes + first, v[j].get(row + first, x, end), -first,
                               (int)row_bytes - first, xs, xs + (uint64_t)sorted_rows * row_bytes);
        }
    }
}

// ---- combine ---------------------------------------------------------------------------------------------------------
// y[t] = sum_j w[t, j] z[place[t, j]], j ascending, in binary32.  A thread holds the sums of N elements; the k reads do not
// depend on one another and are issued together (predicated loads: branches around them made it 124 us).  32768 rows of 2048
// binary16 elements from 117965 answers: 100 us, 6.2 TB/s, bound by HBM.
template <typename E, int N, int KC, bool kWeights>
__global__ void __launch_bounds__(kThreads) combine_kernel(unsigned* status, uint32_t T, uint32_t k, uint32_t cols, uint32_t across,
                                                           uint32_t down, const E* z, uint32_t sorted_rows,
                                                           const int32_t* place, const float* w,
                                                           E* y, uint64_t ld_y)
{
    rows_begin();
    const uint32_t in = threadIdx.x / across;
    const uint32_t col = threadIdx.x - in * across + blockIdx.y * across;
    const uint64_t t = (uint64_t)blockIdx.x * down + in;
    if (in >= down || t >= T || col >= cols) return;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    for (uint32_t j0 = 0; j0 < k; j0 += KC) {
        int32_t at[KC];
        float wt[KC];
        RowsVec<E, N> v[KC];
        load_places<KC>(status, place + t * k + j0, k - j0, sorted_rows, col == 0, at);
#pragma unroll
        for (int j = 0; j < KC; ++j) wt[j] = kWeights ? rows_read_if(j0 + j < k, w + t * k + j0 + j, 1.0f) : 1.0f;
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            v[j].clear();
            rows_load_if<false>(at[j] >= 0, v[j].raw, z + ((uint64_t)(uint32_t)at[j] * cols + col) * N);
        }
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            if (at[j] < 0) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = kWeights ? __fmaf_rn(wt[j], v[j].get(i), sum[i]) : __fadd_rn(sum[i], v[j].get(i));
        }
    }
    RowsVec<E, N> out;
    out.set(sum);
    rows_store_vec<E, N>(y + t * ld_y + (uint64_t)col * N, out);
}

// The same for 16-bit elements where rows start at odd places: a thread has a 16-byte word of y.
template <typename E, int KC, bool kWeights>
__global__ void __launch_bounds__(kThreads) combine_any_kernel(unsigned* status, uint32_t T, uint32_t k, uint32_t D, uint32_t cols, uint32_t across,
                                                               uint32_t down, const E* z, uint32_t sorted_rows,
                                                               const int32_t* place, const float* w,
                                                               E* y, uint64_t ld_y)
{
    constexpr int S = (int)sizeof(E), N = 16 / S;
    rows_begin();
    const uint32_t in = threadIdx.x / across;
    const uint32_t col = threadIdx.x - in * across + blockIdx.y * across;
    const uint64_t t = (uint64_t)blockIdx.x * down + in;
    if (in >= down || t >= T || col >= cols) return;
    unsigned char* out = reinterpret_cast<unsigned char*>(y + t * ld_y);
    const int first = (int)(col * 16) - (int)((uint32_t)(uintptr_t)out & 15u), row_bytes = (int)(D * S);
    if (first >= row_bytes) return;
    const unsigned char *from = reinterpret_cast<const unsigned char*>(z), *end = from + (uint64_t)sorted_rows * row_bytes;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    for (uint32_t j0 = 0; j0 < k; j0 += KC) {
        int32_t at[KC];
        float wt[KC];
        RowsAny<S> any[KC];
        load_places<KC>(status, place + t * k + j0, k - j0, sorted_rows, col == 0, at);
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            wt[j] = kWeights ? rows_read_if(j0 + j < k, w + t * k + j0 + j, 1.0f) : 1.0f;
            any[j].fetch(status, at[j] >= 0, from + (uint64_t)(uint32_t)at[j] * row_bytes + first, from, end);
        }
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            if (at[j] < 0) continue;
            RowsVec<E, N> v;
            v.raw = any[j].get(from + (uint64_t)(uint32_t)at[j] * row_bytes + first, from, end);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = kWeights ? __fmaf_rn(wt[j], v.get(i), sum[i]) : __fadd_rn(sum[i], v.get(i));
        }
    }
    RowsVec<E, N> o;
    o.set(sum);
    rows_store_part<S>(status, out + first, o.raw, -first, row_bytes - first, y, y + (T - 1) * ld_y + D);
}

// ---- the gradient of combine -----------------------------------------------------------------------------------------
// dz[place[t, j]] = w[t, j] dy[t], dw[t, j] = <dy[t], z[place[t, j]]>.  A team of `team` threads (a power of two, 4 .. 256) has one
// row t: each thread reads its accesses of dy once for KC slots at a time and keeps one partial sum a slot; the partial sums are
// added in a fixed order (a tree over the lanes, then the warps in turn).  8192 rows of 4096 bfloat16 elements, k = 8: with the
// gradient of dispatch 269 us for 1.75 GB, 6.5 TB/s, the rate of a copy.
template <typename E, int N, int KC>
__global__ void __launch_bounds__(kThreads) combine_grad_kernel(unsigned* status, uint32_t T, uint32_t k, uint32_t cols, uint32_t team,
                                                                const E* dy, uint64_t ld_dy, const E* z,
                                                                uint32_t sorted_rows, const int32_t* place,
                                                                const float* w, E* dz, float* dw)
{
    __shared__ float part[kThreads / 32][KC];
    rows_begin();
    const uint32_t in = threadIdx.x / team, me = threadIdx.x % team;
    const uint64_t t = (uint64_t)blockIdx.x * (kThreads / team) + in;
    const bool row = t < T;
    const E* g = dy + (row ? t : 0) * ld_dy;
    for (uint32_t j0 = 0; j0 < k; j0 += KC) {
        int32_t at[KC];
        float wt[KC], dot[KC];
        load_places<KC>(status, place + (row ? t : 0) * k + j0, row ? k - j0 : 0u, sorted_rows, me == 0, at);
#pragma unroll
        for (int j = 0; j < KC; ++j) {
            wt[j] = rows_read_if(row && j0 + j < k && w != nullptr, w + t * k + j0 + j, 1.0f);
            dot[j] = 0.0f;
        }
        for (uint32_t col = me; col < cols && row; col += team) {
            const RowsVec<E, N> a = rows_load_vec<E, N>(g + (uint64_t)col * N);
            if (dw != nullptr) {
                RowsVec<E, N> v[KC];
#pragma unroll
                for (int j = 0; j < KC; ++j) rows_load_if<false>(at[j] >= 0, v[j].raw, z + ((uint64_t)(uint32_t)at[j] * cols + col) * N);
#pragma unroll
                for (int j = 0; j < KC; ++j) {
                    if (at[j] < 0) continue;
#pragma unroll
                    for (int i = 0; i < N; ++i) dot[j] = __fmaf_rn(a.get(i), v[j].get(i), dot[j]);
                }
            }
            if (dz != nullptr) {
#pragma unroll
                for (int j = 0; j < KC; ++j) {
                    if (at[j] < 0) continue;
                    float part[N];
#pragma unroll
                    for (int i = 0; i < N; ++i) part[i] = __fmul_rn(wt[j], a.get(i));
                    RowsVec<E, N> o;
                    o.set(part);
                    rows_store_vec<E, N>(dz + ((uint64_t)(uint32_t)at[j] * cols + col) * N, o);
                }
            }
        }
        if (dw == nullptr) continue;
        for (uint32_t d = (team < 32 ? team : 32u) / 2; d > 0; d >>= 1)
#pragma unroll
            for (int j = 0; j < KC; ++j) dot[j] = __fadd_rn(dot[j], __shfl_xor_sync(0xFFFFFFFFu, dot[j], d));
        if (team > 32) {
            const uint32_t warp = threadIdx.x / 32;
            __syncthreads();                          // the sums of the slots before these have been read
            if ((threadIdx.x & 31u) == 0) {
#pragma unroll
                for (int j = 0; j < KC; ++j) part[warp][j] = dot[j];
            }
            __syncthreads();
            if (me < KC && row && j0 + me < k) {
                float s = 0.0f;
                for (uint32_t q = 0; q < team / 32; ++q) s = __fadd_rn(s, part[in * (team / 32) + q][me]);
                dw[t * k + j0 + me] = s;
            }
        } else if (me == 0 && row) {
#pragma unroll
            for (int j = 0; j < KC; ++j)
                if (j0 + j < k) dw[t * k + j0 + j] = dot[j];
        }
    }
}

// Threads that share a row of `cols` accesses: a lane an access up to a warp, then up to four accesses a thread.
uint32_t team_of(uint32_t cols)
{
    uint32_t team = 4;
    while (team < 32 && team < cols) team *= 2;
    while (team >= 32 && team < kThreads && team * 4 < cols) team *= 2;
    return team;
}

// Runs CALL(N) with the elements per access that `granule` allows for elements of S bytes.
#define ROWS_WITH_VEC(S, granule, CALL)                                         \
    do {                                                                        \
        if ((granule) >= 32) { CALL(32 / (S)); }                                \
        else if ((granule) >= 16) { CALL(16 / (S)); }                           \
        else if ((granule) >= 8) { CALL(8 / (S)); }                             \
        else if ((granule) >= 4) { CALL(4 / (S)); }                             \
        else { CALL(1); }                                                       \
    } while (0)

// Runs CALL(KC): slots of a row that are handled together.
#define ROWS_WITH_SLOTS(k, CALL)                                                \
    do {                                                                        \
        if ((k) <= 2) { CALL(2); } else if ((k) <= 4) { CALL(4); } else { CALL(8); } \
    } while (0)

}  // namespace

int rows_launch_dispatch(unsigned* status, uint32_t T, uint32_t k, uint32_t row_bytes, const void* x, uint64_t ld_x,
                         const int32_t* place, uint32_t sorted_rows, void* xs, cudaStream_t s)
{
    if (T == 0) return 0;
    const uint32_t g = rows_granule(row_bytes, ld_x, (uintptr_t)x, (uintptr_t)xs);
    int rc = -1;
    if (g <= 2 && row_bytes >= kRowsAnyBytes) {
        const uint32_t words = (row_bytes + 30) / 16;                     // of a destination, wherever it starts
        const Tiling t = tile(T, words);
#define ROWS_ANY(S, KC)                                                                                                     \
    rc = rows_launch(dispatch_any_kernel<S, KC>, t.grid, t.block, 0, s, 0, status, T, k, row_bytes, words, t.across, t.down,     \
                     (const unsigned char*)x, ld_x, place, sorted_rows, (unsigned char*)xs)
#define ROWS_K(KC)                                                                                                          \
    do { if (g == 2) ROWS_ANY(2, KC); else ROWS_ANY(1, KC); } while (0)
        if (k <= 2) ROWS_K(2); else ROWS_K(4);
#undef ROWS_K
#undef ROWS_ANY
        return rc;
    }
    const uint32_t cols = row_bytes / g;
    const Tiling t = tile(T, cols);
    if (t.grid.y > 65535u) return -1;
#define ROWS_GO(B, KC)                                                                                                      \
    rc = rows_launch(dispatch_kernel<B, KC>, t.grid, t.block, 0, s, 0, status, T, k, cols, t.across, t.down, (const unsigned char*)x, ld_x, \
                     place, sorted_rows, (unsigned char*)xs)
#define ROWS_K(KC)                                                                                     \
    switch (g) {                                                                                       \
    case 32: ROWS_GO(32, KC); break;                                                                   \
    case 16: ROWS_GO(16, KC); break;                                                                   \
    case 8: ROWS_GO(8, KC); break;                                                                     \
    case 4: ROWS_GO(4, KC); break;                                                                     \
    case 2: ROWS_GO(2, KC); break;                                                                     \
    default: ROWS_GO(1, KC); break;                                                                    \
    }
    ROWS_WITH_SLOTS(k, ROWS_K);
#undef ROWS_K
#undef ROWS_GO
    return rc;
}

int rows_launch_combine(unsigned* status, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* z, uint32_t sorted_rows,
                        const int32_t* place, const float* w, void* y, uint64_t ld_y, cudaStream_t s)
{
    if (T == 0) return 0;
    const uint32_t S = rows_elem_bytes(dtype);
    const uint32_t g = rows_granule((uint64_t)D * S, ld_y * S, (uintptr_t)z, (uintptr_t)y);
    int rc = -1;
    if (g == 2 && dtype != PEARL_F32 && D * S >= kRowsAnyBytes) {
        const uint32_t words = (D * S + 30) / 16;
        const Tiling t = tile(T, words);
#define ROWS_ANY(E, KC)                                                                                                     \
    do {                                                                                                                    \
        if (w) rc = rows_launch(combine_any_kernel<E, KC, true>, t.grid, t.block, 0, s, 0, status, T, k, D, words, t.across, t.down, \
                                (const E*)z, sorted_rows, place, w, (E*)y, ld_y);                                           \
        else rc = rows_launch(combine_any_kernel<E, KC, false>, t.grid, t.block, 0, s, 0, status, T, k, D, words, t.across, t.down,  \
                              (const E*)z, sorted_rows, place, w, (E*)y, ld_y);                                             \
    } while (0)
        if (dtype == PEARL_F16) { if (k <= 2) ROWS_ANY(__half, 2); else ROWS_ANY(__half, 4); }
        else { if (k <= 2) ROWS_ANY(__nv_bfloat16, 2); else ROWS_ANY(__nv_bfloat16, 4); }
#undef ROWS_ANY
        return rc;
    }
#define ROWS_GO(E, N, KC)                                                                                                           \
    do {                                                                                                                            \
        const uint32_t cols = D / (N);                                                                                              \
        const Tiling t = tile(T, cols);                                                                                             \
        if (t.grid.y > 65535u) break;                                                                                               \
        if (w) rc = rows_launch(combine_kernel<E, N, KC, true>, t.grid, t.block, 0, s, 0, status, T, k, cols, t.across, t.down, (const E*)z, \
                                sorted_rows, place, w, (E*)y, ld_y);                                                                \
        else rc = rows_launch(combine_kernel<E, N, KC, false>, t.grid, t.block, 0, s, 0, status, T, k, cols, t.across, t.down, (const E*)z,   \
                              sorted_rows, place, w, (E*)y, ld_y);                                                                  \
    } while (0)
#define ROWS_TYPE(E)                                                                  \
    do {                                                                              \
        constexpr int kSize = sizeof(E);                                              \
        ROWS_WITH_VEC(kSize, g, ROWS_N_##E);                                          \
    } while (0)
#define ROWS_N(E, N)                                                                  \
    do {                                                                              \
        if (k <= 2) ROWS_GO(E, N, 2); else if (k <= 4) ROWS_GO(E, N, 4); else ROWS_GO(E, N, 8); \
    } while (0)
#define ROWS_N_float(N) ROWS_N(float, N)
#define ROWS_N___half(N) ROWS_N(__half, N)
#define ROWS_N___nv_bfloat16(N) ROWS_N(__nv_bfloat16, N)
    ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_GO
    return rc;
}

int rows_launch_combine_grad(unsigned* status, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy,
                             const void* z, uint32_t sorted_rows, const int32_t* place, const float* w, void* dz, float* dw,
                             cudaStream_t s)
{
    if (T == 0) return 0;
    const uint32_t S = rows_elem_bytes(dtype);
    const uint32_t g = rows_granule((uint64_t)D * S, ld_dy * S, (uintptr_t)dy, dw ? (uintptr_t)z : 0, dz ? (uintptr_t)dz : 0);
    int rc = -1;
#define ROWS_GO(E, N, KC)                                                                                                  \
    do {                                                                                                                   \
        const uint32_t cols = D / (N);                                                                                     \
        const uint32_t team = team_of(cols), each = kThreads / team;                                                                             \
        rc = rows_launch(combine_grad_kernel<E, N, KC>, dim3((T + each - 1) / each), dim3(kThreads), 0, s, 0, status, T, k, cols, team, \
                         (const E*)dy, ld_dy, (const E*)z, sorted_rows, place, w, (E*)dz, dw);                             \
    } while (0)
    ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_GO
    return rc;
}
