// Dropout by a counter-based generator, joined with the residual sum.
//
// Bound by memory, with the generator beside it: one counter is good for 8 elements of 16 bits each, some 60 instructions.  (32 bits an
// element would be twice that, and a 16-bit element's share of an SM's cycles is 9 instructions at the memory's rate.)  The counters are made
// while the elements are on their way.  16384 x 4096 bfloat16 elements with a residual 62 us (6.5 TB/s), without one 55 (4.9 TB/s; issue slots three
// quarters used).
#include "layer_internal.cuh"

namespace {

constexpr uint32_t kThreads = 256;
constexpr int kGroup = 8;               // columns of a counter

// Philox4x32-10 (Salmon et al., SC'11): four words of the counter (c0, c1, c2, c3) under the key.
__device__ __forceinline__ void philox4x32_10(uint32_t (&c)[4], uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint32_t hi0 = __umulhi(0xD2511F53u, c[0]), lo0 = 0xD2511F53u * c[0];
        const uint32_t hi1 = __umulhi(0xCD9E8D57u, c[2]), lo1 = 0xCD9E8D57u * c[2];
        c[0] = hi1 ^ c[1] ^ k0;
        c[1] = lo1;
        c[2] = hi0 ^ c[3] ^ k1;
        c[3] = lo0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

struct Args {
    unsigned* status;
    uint32_t T, D, below;
    float scale;
    uint64_t ld_x, ld_r, ld_y, seed, call;
    const uint64_t* calls;
};

// N elements' results from their words of x and of the residual; bits: 16 for each of 8, of which these are from `first` on.
template <typename E, int N>
__device__ __forceinline__ RowsVec<E, N> dropped(const RowsVec<E, N>& x, const RowsVec<E, N>& residual, const uint32_t (&bits)[4], int first, const Args& a)
{
    float out[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = first + i;
        const uint32_t b = e % 2 ? bits[e / 2] >> 16 : bits[e / 2] & 0xFFFFu;
        out[i] = (b >= a.below ? x.get(i) * a.scale : 0.0f) + residual.get(i);
    }
    RowsVec<E, N> o;
    o.set(out);
    return o;
}

// A thread has the 8 columns of a counter in R rows.  N: the elements of an access; `across` threads along a row, `down` rows a block
// times R.
template <typename E, int N, int R>
__global__ void __launch_bounds__(kThreads) dropout_kernel(uint32_t across, uint32_t down, const E* x, const E* residual, E* y, Args a)
{
    rows_begin();
    const uint32_t in = threadIdx.x / across;
    const uint32_t group = threadIdx.x - in * across + blockIdx.y * across, col = group * kGroup;
    const uint64_t t0 = (uint64_t)blockIdx.x * down * R + in;
    if (in >= down || col >= a.D) return;
    const int n = (int)(a.D - col);
    RowsVec<E, N> v[R][kGroup / N], r[R][kGroup / N];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
        for (int j = 0; j < kGroup / N; ++j) {
            const uint64_t t = t0 + (uint64_t)k * down;
            int there = t < a.T ? n - j * N : 0;
            const E *p = x + t * a.ld_x + col + j * N, *q = residual + t * a.ld_r + col + j * N;
            if (!layer_in_rows<N>(a.status, p, 0, there, x, layer_end(x, a.T, a.D, a.ld_x))) there = 0;
            v[k][j] = layer_load_part<E, N>(p, there);
            if (residual && layer_in_rows<N>(a.status, q, 0, there, residual, layer_end(residual, a.T, a.D, a.ld_r))) r[k][j] = layer_load_part<E, N>(q, there);
            else r[k][j].clear();
        }
    const uint64_t call = a.call + (a.calls ? *a.calls : 0);
    uint32_t c[R][4];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        c[k][0] = group;
        c[k][1] = (uint32_t)(t0 + (uint64_t)k * down);
        c[k][2] = (uint32_t)call;
        c[k][3] = (uint32_t)(call >> 32);
        philox4x32_10(c[k], (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const uint64_t t = t0 + (uint64_t)k * down;
        if (t >= a.T) break;
#pragma unroll
        for (int j = 0; j < kGroup / N; ++j) {
            E* p = y + t * a.ld_y + col + j * N;
            if (layer_in_rows<N, E>(a.status, p, 0, n - j * N, y, layer_end(y, a.T, a.D, a.ld_y)))
                layer_store_part<E, N>(p, dropped<E, N>(v[k][j], r[k][j], c[k], j * N, a), n - j * N);
        }
    }
}

// Rows that start anywhere, x, residual and y alike: a lane has 8 elements that start with a 16-byte word of memory, which are the end of one
// counter's columns and the beginning of the next one's.  It makes the latter and has the former from the lane before; a warp's first lane
// does nothing else.  8000 rows of 2047 binary16 elements and their gradient 57 us, element by element 84.
template <typename E>
__global__ void __launch_bounds__(kThreads) dropout_any_kernel(uint32_t parts, uint64_t warps, const E* x, const E* residual, E* y, Args a)
{
    constexpr int N = 16 / (int)sizeof(E), M = kGroup / N;       // elements of a word; words of a lane
    rows_begin();
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t which = (uint64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (which >= warps) return;
    const uint64_t t = which / parts;
    const int unit = (int)((uint32_t)(which - t * parts) * 31u + lane) - 1;
    const E* row = x + t * a.ld_x;
    const int off = (int)(((uint32_t)(uintptr_t)row & 15u) / sizeof(E)), e = unit * kGroup - off, D = (int)a.D;
    const bool works = lane > 0 && e < D;
    RowsVec<E, N> v[M], r[M];
    // elements [lo, hi) of the N at p
    const auto load = [&](const E* p, int lo, int hi, const E* first, uint64_t ld) {
        RowsVec<E, N> w;
        w.clear();
        if (!layer_in_rows<N>(a.status, p, lo, hi, first, layer_end(first, a.T, a.D, ld))) return w;
        if (lo <= 0 && hi >= N) {
            rows_load_if<false>(true, w.raw, p);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i < lo || i >= hi) continue;
                if constexpr (sizeof(E) == 4) w.word[i] = reinterpret_cast<const uint32_t*>(p)[i];
                else w.word[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << (i % 2 * 16);
            }
        }
        return w;
    };
#pragma unroll
    for (int j = 0; j < M; ++j) {
        const int lo = works ? -(e + j * N) : N, hi = D - (e + j * N);
        v[j] = load(row + e + j * N, lo, hi, x, a.ld_x);
        if (residual) r[j] = load(residual + t * a.ld_r + e + j * N, lo, hi, residual, a.ld_r);
        else r[j].clear();
    }
    const uint64_t call = a.call + (a.calls ? *a.calls : 0);
    uint32_t c[4] = { (uint32_t)unit, (uint32_t)t, (uint32_t)call, (uint32_t)(call >> 32) };
    philox4x32_10(c, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    // 16 times 16 bits, of which the 8 from the (8 - off)-th on are the lane's
    uint32_t w[9];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __shfl_up_sync(0xFFFFFFFFu, c[i], 1);
        w[4 + i] = c[i];
    }
    w[8] = 0;
    const uint32_t skip = kGroup - off;
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = skip & 8u ? w[i + 4] : w[i];
#pragma unroll
    for (int i = 0; i < 7; ++i) w[i] = skip & 4u && !(skip & 8u) ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = skip & 2u && !(skip & 8u) ? w[i + 1] : w[i];
    uint32_t bits[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) bits[i] = __funnelshift_r(w[i], w[i + 1], (skip & 1u) * 16u);
    if (!works) return;
#pragma unroll
    for (int j = 0; j < M; ++j) {
        const RowsVec<E, N> o = dropped<E, N>(v[j], r[j], bits, j * N, a);
        E* to = y + t * a.ld_y + e + j * N;
        const int lo = -(e + j * N), hi = D - (e + j * N);
        if (!layer_in_rows<N, E>(a.status, to, lo, hi, y, layer_end(y, a.T, a.D, a.ld_y))) continue;
        if (lo <= 0 && hi >= N) {
            rows_store(to, o.raw);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (i < lo || i >= hi) continue;
                if constexpr (sizeof(E) == 4) reinterpret_cast<uint32_t*>(to)[i] = o.word[i];
                else reinterpret_cast<uint16_t*>(to)[i] = (uint16_t)(o.word[i / 2] >> (i % 2 * 16));
            }
        }
    }
}

template <typename E, int N, int R> int dropout_as(const Args& a, const void* x, const void* residual, void* y, cudaStream_t s)
{
    const uint32_t groups = (a.D + kGroup - 1) / kGroup, parts = (groups + kThreads - 1) / kThreads, across = (groups + parts - 1) / parts;
    const uint32_t down = kThreads / across;
    const dim3 grid((uint32_t)(((uint64_t)a.T + (uint64_t)down * R - 1) / ((uint64_t)down * R)), parts), block((across * down + 31) / 32 * 32);
    return rows_launch(dropout_kernel<E, N, R>, grid, block, 0, s, 0, across, down, (const E*)x, (const E*)residual, (E*)y, a);
}
template <typename E> int dropout_of(const Args& a, const void* x, const void* residual, void* y, cudaStream_t s)
{
    constexpr uint32_t S = sizeof(E);
    constexpr int N = 16 / (int)S;
    const uint32_t granule = rows_granule((uintptr_t)x | (uintptr_t)y, residual ? (uintptr_t)residual : 0, a.ld_x * S, a.ld_y * S, residual ? a.ld_r * S : 0);
    if (S == 4 && granule >= 32) return dropout_as<E, S == 4 ? 8 : N, 1>(a, x, residual, y, s);
    // (two rows a thread from 2^20 elements on: 16384 x 4096 bfloat16 elements with a residual 62 us, with one row a thread 66; 2048 x 512 2.0 and 2.2, 256 x
    // 4096 2.0 and 2.2; 1536 x 512 2.0 and 1.9, 64 x 4096 1.6 and 1.4)
    if (granule >= 16) return (uint64_t)a.T * a.D >= 1u << 20 && S == 2 ? dropout_as<E, N, S == 2 ? 2 : 1>(a, x, residual, y, s) : dropout_as<E, N, 1>(a, x, residual, y, s);
    // (rows of an even number of elements: 2^24 of them in rows of 30 to 4094 24 us, by the other kernel 29 to 55)
    if (S == 2 && granule >= 4) return dropout_as<E, S == 2 ? 2 : 1, 1>(a, x, residual, y, s);
    const auto alike = [&](const void* p, uint64_t ld) { return (((uintptr_t)p ^ (uintptr_t)x) & 15u) == 0 && ((ld - a.ld_x) * S & 15u) == 0; };
    if (alike(y, a.ld_y) && (!residual || alike(residual, a.ld_r))) {
        const uint32_t units = (a.D + N - 1 + kGroup - 1) / kGroup, parts = (units + 30) / 31;
        const uint64_t warps = (uint64_t)a.T * parts, blocks = (warps + kThreads / 32 - 1) / (kThreads / 32);
        // Where seven tenths of the lanes have something, half of them in binary32.  2^24 bfloat16 elements in rows of 193 (eight tenths) 40 us, element by element
        // 41; of 513 (0.70) 42 and 42, of 501 (0.69) 42 and 42, of 301 (0.63) 49 and 41, of 249 (0.53) 57 and 42.  2^23 binary32 elements in rows of 257 (0.53) 29
        // and 30, of 301 (0.63) 26 and 29, of 65 (0.29) 56 and 28.
        if (blocks <= 0x7FFFFFFFu && 10 * units >= (S == 4 ? 5 : 7) * 31 * parts)
            return rows_launch(dropout_any_kernel<E>, dim3((uint32_t)blocks), dim3(kThreads), 0, s, 0, parts, warps, (const E*)x, (const E*)residual, (E*)y, a);
    }
    return dropout_as<E, 1, 1>(a, x, residual, y, s);
}

}  // namespace

int layer_launch_dropout(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, const void* residual, uint64_t ld_r, uint32_t below,
                         float scale, uint64_t seed, uint64_t call, const uint64_t* calls, void* y, uint64_t ld_y, cudaStream_t s)
{
    const Args a = { status, T, D, below, scale, ld_x, ld_r, ld_y, seed, call, calls };
#define DROP(E) return dropout_of<E>(a, x, residual, y, s)
    ROWS_WITH_TYPE(dtype, DROP);
#undef DROP
}
