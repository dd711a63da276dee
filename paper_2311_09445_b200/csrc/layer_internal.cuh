// Internal declarations shared by the translation units of a layer's operators (include/pearl_layers.h).
#pragma once
#include "../../include/pearl_layers.h"
#include "rows_internal.cuh"

// Kernel launchers; each returns the number of kernels launched (0: nothing to do), or -1 on a launch error.
int layer_launch_norm(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, uint32_t ptype, const void* gamma,
                      const void* beta, float eps, void* y, uint64_t ld_y, float* mean, float* rstd, cudaStream_t s);
int layer_launch_norm_grad(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x,
                           const float* mean, const float* rstd, uint32_t ptype, const void* gamma, void* dx, uint64_t ld_dx, float* dgamma,
                           float* dbeta, float* work, uint64_t work_bytes, cudaStream_t s);
uint64_t layer_norm_grad_work_bytes(uint32_t T, uint32_t D);
int layer_launch_dropout(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, const void* residual, uint64_t ld_r,
                         uint32_t below, float scale, uint64_t seed, uint64_t call, const uint64_t* calls, void* y, uint64_t ld_y, cudaStream_t s);

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

// The checked build compares with their extents: the words of rows that the norm, its gradient and dropout load and store, the bulk copies of the gradient's
// ring (with the rest of the words that a row starts and ends in), the places of parameters in shared memory, the blocks' lines of scratch; the
// expert layer's logits, copied words, h and results of slots.
// The end of a matrix's last row.
template <typename E> __device__ __forceinline__ const E* layer_end(const E* p, uint32_t T, uint32_t D, uint64_t ld) { return p + (uint64_t)(T - 1) * ld + D; }
// Whether elements [lo, hi) of the N at p, those of them that there are, lie in a matrix.
template <int N, typename E>
__device__ __forceinline__ bool layer_in_rows(unsigned* status, const E* p, int lo, int hi, const E* first, const E* end)
{
    lo = lo > 0 ? lo : 0;
    hi = hi < N ? hi : N;
    return lo >= hi || ROWS_IN_ARRAY(status, p + lo, (hi - lo) * (int)sizeof(E), first, end);
}

// ---- two binary32 numbers at once (add, multiply and multiply-add take them in one instruction) ------------------------
struct LayerTwo {
    unsigned long long v;
    __device__ __forceinline__ LayerTwo() {}
    __device__ __forceinline__ LayerTwo(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit LayerTwo(float a) : LayerTwo(a, a) {}
    __device__ __forceinline__ float2 get() const
    {
        float2 f;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
        return f;
    }
    __device__ __forceinline__ float sum() const { const float2 f = get(); return f.x + f.y; }
};
__device__ __forceinline__ LayerTwo operator+(LayerTwo a, LayerTwo b)
{
    LayerTwo r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ LayerTwo operator*(LayerTwo a, LayerTwo b)
{
    LayerTwo r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ LayerTwo layer_fma(LayerTwo a, LayerTwo b, LayerTwo c)
{
    LayerTwo r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// The pairs of an access; the second of an odd last one is 0.
template <typename E, int N> __device__ __forceinline__ void layer_twos(LayerTwo (&t)[(N + 1) / 2], const RowsVec<E, N>& v)
{
#pragma unroll
    for (int i = 0; i < (N + 1) / 2; ++i) t[i] = LayerTwo(v.get(2 * i), 2 * i + 1 < N ? v.get(2 * i + 1 < N ? 2 * i + 1 : 0) : 0.0f);
}
template <typename E, int N> __device__ __forceinline__ RowsVec<E, N> layer_access(const LayerTwo (&t)[(N + 1) / 2])
{
    float f[(N + 1) / 2 * 2];
#pragma unroll
    for (int i = 0; i < (N + 1) / 2; ++i) { const float2 p = t[i].get(); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
    RowsVec<E, N> v;
    v.set(f);
    return v;
}

// The sum over a warp's lanes, the same in each.
__device__ __forceinline__ float layer_warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}

// ---- barriers in shared memory ----------------------------------------------------------------------------------------
constexpr uint32_t kLayerSpins = 1u << 21;           // polls of a flag in global memory at most (0.6 s); a barrier, whose polls wait 1.5 us each, has four times as many
__device__ __forceinline__ uint32_t layer_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void layer_barrier(uint64_t* barrier, uint32_t arrivals)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(layer_address(barrier)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void layer_arrive(uint64_t* barrier) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(layer_address(barrier)) : "memory"); }
__device__ __forceinline__ void layer_arrive_with(uint64_t* barrier, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(layer_address(barrier)), "r"(bytes) : "memory");
}
// Waits for the end of a barrier's phase of this parity; with a limit, and a status bit behind it.
__device__ __forceinline__ void layer_wait(unsigned* status, uint64_t* barrier, uint32_t parity)
{
    uint32_t there = 0;
    for (uint32_t spins = 0; !there; ++spins) {
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                     : "=r"(there) : "r"(layer_address(barrier)), "r"(parity & 1u) : "memory");
        if (spins > 4 * kLayerSpins) { atomicOr(status, PEARL_ST_INTERNAL); break; }
    }
}

// N elements at p, which is aligned for them, by one plain access.
template <typename E, int N> __device__ __forceinline__ RowsVec<E, N> layer_read(const void* p)
{
    RowsVec<E, N> v;
    constexpr int B = (int)sizeof(E) * N;
    if constexpr (B == 16) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        v.raw.r[0] = w.x; v.raw.r[1] = w.y; v.raw.r[2] = w.z; v.raw.r[3] = w.w;
    } else if constexpr (B == 8) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        v.raw.r[0] = w.x; v.raw.r[1] = w.y;
    } else if constexpr (B == 4) {
        v.raw.r[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        v.raw.r[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    return v;
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
