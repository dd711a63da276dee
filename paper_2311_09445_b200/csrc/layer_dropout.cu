// Dropout by a counter-based generator, joined with the residual sum.
#include "layer_internal.cuh"

namespace {

constexpr uint32_t kThreads = 256;

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

// A thread has 8 columns of a row, those of one counter.  N: the elements of an access; `across` threads along a row, `down` rows a block.
template <typename E, int N>
__global__ void __launch_bounds__(kThreads) dropout_kernel(uint32_t T, uint32_t D, uint32_t across, uint32_t down, const E* x, uint64_t ld_x,
                                                           const E* residual, uint64_t ld_r, uint32_t below, float scale, uint64_t seed,
                                                           uint64_t call, const uint64_t* calls, E* y, uint64_t ld_y)
{
    rows_begin();
    const uint32_t in = threadIdx.x / across;
    const uint32_t group = threadIdx.x - in * across + blockIdx.y * across;
    const uint64_t t = (uint64_t)blockIdx.x * down + in;
    if (in >= down || t >= T || (uint64_t)group * 8 >= D) return;
    const uint32_t col = group * 8;
    const int n = (int)(D - col);
    RowsVec<E, N> a[8 / N], b[8 / N];
#pragma unroll
    for (int j = 0; j < 8 / N; ++j) {
        a[j] = layer_load_part<E, N>(x + t * ld_x + col + j * N, n - j * N);
        if (residual) b[j] = layer_load_part<E, N>(residual + t * ld_r + col + j * N, n - j * N);
        else b[j].clear();
    }
    if (calls) call += *calls;
    uint32_t c[4] = { group, (uint32_t)t, (uint32_t)call, (uint32_t)(call >> 32) };
    philox4x32_10(c, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
    for (int j = 0; j < 8 / N; ++j) {
        float out[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = j * N + i;
            const uint32_t bits = e % 2 ? c[e / 2] >> 16 : c[e / 2] & 0xFFFFu;
            out[i] = (bits >= below ? a[j].get(i) * scale : 0.0f) + b[j].get(i);
        }
        RowsVec<E, N> o;
        o.set(out);
        layer_store_part<E, N>(y + t * ld_y + col + j * N, o, n - j * N);
    }
}

}  // namespace

int layer_launch_dropout(uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, const void* residual, uint64_t ld_r, uint32_t below,
                         float scale, uint64_t seed, uint64_t call, const uint64_t* calls, void* y, uint64_t ld_y, cudaStream_t s)
{
    const uint32_t groups = (D + 7) / 8, parts = (groups + kThreads - 1) / kThreads, across = (groups + parts - 1) / parts, down = kThreads / across;
    const dim3 grid((uint32_t)(((uint64_t)T + down - 1) / down), parts), block((across * down + 31) / 32 * 32);
    const uint32_t S = rows_elem_bytes(dtype);
    const uint32_t granule = rows_granule((uintptr_t)x | (uintptr_t)y, residual ? (uintptr_t)residual : 0, ld_x * S, ld_y * S, residual ? ld_r * S : 0);
#define DROP(E, N)                                                                                                                      \
    return rows_launch(dropout_kernel<E, N>, grid, block, 0, s, 0, T, D, across, down, (const E*)x, ld_x, (const E*)residual, ld_r, below, scale, \
                       seed, call, calls, (E*)y, ld_y)
    if (dtype == PEARL_F32) {
        if (granule >= 32) DROP(float, 8);
        else if (granule >= 16) DROP(float, 4);
        else DROP(float, 1);
    } else if (dtype == PEARL_F16) {
        if (granule >= 16) DROP(__half, 8);
        else if (granule >= 4) DROP(__half, 2);
        else DROP(__half, 1);
    } else {
        if (granule >= 16) DROP(__nv_bfloat16, 8);
        else if (granule >= 4) DROP(__nv_bfloat16, 2);
        else DROP(__nv_bfloat16, 1);
    }
#undef DROP
}
