// Internal declarations shared by the translation units of a layer's operators (include/pearl_layers.h).
#pragma once
#include "../../include/pearl_layers.h"
#include "rows_internal.cuh"

// Kernel launchers; each returns the number of kernels launched (0: nothing to do), or -1 on a launch error.
int layer_launch_norm(uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, uint32_t ptype, const void* gamma, const void* beta,
                      float eps, void* y, uint64_t ld_y, float* mean, float* rstd, cudaStream_t s);
int layer_launch_norm_grad(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x,
                           const float* mean, const float* rstd, uint32_t ptype, const void* gamma, void* dx, uint64_t ld_dx, float* dgamma,
                           float* dbeta, float* work, uint64_t work_bytes, cudaStream_t s);
uint64_t layer_norm_grad_work_bytes(uint32_t T, uint32_t D);
int layer_launch_dropout(uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, const void* residual, uint64_t ld_r, uint32_t below,
                         float scale, uint64_t seed, uint64_t call, const uint64_t* calls, void* y, uint64_t ld_y, cudaStream_t s);

struct LayerExperts {
    uint32_t T, D, H, E, k, dtype, act;
    bool over_chosen;
    const void *x, *router, *up, *down;
    uint64_t ld_x, ld_y;
    float* w;
    int32_t* ids;
    void *y, *work;
};
int layer_launch_experts(unsigned* status, const LayerExperts& a, cudaStream_t s);
uint64_t layer_experts_work_bytes(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k);

#ifdef __CUDACC__

// The sum over a warp's lanes, the same in each.
__device__ __forceinline__ float layer_warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}

// Elements [0, n) of the N at p, zeros behind them; a whole access where all are there (p is aligned for one).
template <typename E, int N>
__device__ __forceinline__ RowsVec<E, N> layer_load_part(const E* p, int n)
{
    RowsVec<E, N> v;
    v.clear();
    if (n >= N) {
        rows_load_if<false>(true, v.raw, p);
    } else if (N > 1 && n > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i >= n) break;
            if constexpr (sizeof(E) == 4) {
                v.word[i] = reinterpret_cast<const uint32_t*>(p)[i];
            } else {
                v.word[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << (i % 2 * 16);
            }
        }
    }
    return v;
}
template <typename E, int N>
__device__ __forceinline__ void layer_store_part(E* p, const RowsVec<E, N>& v, int n)
{
    if (n >= N) {
        rows_store(p, v.raw);
    } else if (N > 1 && n > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i >= n) break;
            if constexpr (sizeof(E) == 4) reinterpret_cast<uint32_t*>(p)[i] = v.word[i];
            else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(v.word[i / 2] >> (i % 2 * 16));
        }
    }
}

#endif
