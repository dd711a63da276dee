// Internal declarations shared by the translation units of the row operators (include/pearl_rows.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/pearl_rows.h"

// The checked build (-DPEARL_CHECKED): an index into an array that the kernel computed is compared with its extent before it
// is used; one out of range raises PEARL_ST_INTERNAL and the access is skipped.  (Indices that the caller gives -- ids, places,
// parents -- are compared in every build.)
#ifdef PEARL_CHECKED
#define ROWS_IN_BOUNDS(status, cond) ((cond) ? true : (atomicOr((status), PEARL_ST_INTERNAL), false))
#else
#define ROWS_IN_BOUNDS(status, cond) (true)
#endif

// Kernel launchers; each returns the number of kernels launched (0: nothing to do), or -1 on a launch error.
int rows_launch_route(unsigned* status, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                      bool over_chosen, float* w, int32_t* ids, cudaStream_t s);
int rows_launch_route_grad(unsigned* status, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                           bool over_chosen, const float* w, const int32_t* ids, const float* dw, void* dlogits, uint64_t ld_d,
                           cudaStream_t s);
int rows_launch_sort(unsigned* status, uint32_t slots, uint32_t E, const int32_t* ids, int32_t* offsets, int32_t* order,
                     int32_t* place, cudaStream_t s);
int rows_launch_dispatch(unsigned* status, uint32_t T, uint32_t k, uint32_t row_bytes, const void* x, uint64_t ld_x,
                         const int32_t* place, uint32_t sorted_rows, void* xs, cudaStream_t s);
int rows_launch_combine(unsigned* status, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* z, uint32_t sorted_rows,
                        const int32_t* place, const float* w, void* y, uint64_t ld_y, cudaStream_t s);
int rows_launch_combine_grad(unsigned* status, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy,
                             const void* z, uint32_t sorted_rows, const int32_t* place, const float* w, void* dz, float* dw,
                             cudaStream_t s);
int rows_launch_beam_select(unsigned* status, uint32_t G, uint32_t W, uint32_t V, uint32_t C, uint32_t dtype, const void* logits,
                            uint64_t ld, const float* scores, const uint8_t* done, int32_t end_token, float* best_score,
                            int32_t* best_beam, int32_t* best_token, cudaStream_t s);
int rows_launch_beam_reorder(unsigned* status, uint32_t blocks, uint32_t G, uint32_t W, uint32_t pieces, uint64_t piece_bytes,
                             const int32_t* parent, const void* src, const pearl_states_t& sp, void* dst, const pearl_states_t& dp,
                             cudaStream_t s);

inline uint32_t rows_elem_bytes(uint32_t dtype) { return dtype == PEARL_F32 ? 4u : 2u; }

// The widest access (16, 8, 4, 2 or 1 bytes) that every one of these byte counts and addresses is a multiple of.
inline uint32_t rows_granule(uint64_t a, uint64_t b = 0, uint64_t c = 0, uint64_t d = 0, uint64_t e = 0)
{
    const uint64_t all = a | b | c | d | e | 16u;
    return (uint32_t)(all & (~all + 1u));
}

// Launches a kernel as a programmatic dependent of the one before it on the stream: its blocks may be set up while that one
// still runs; each of them waits (rows_begin) before it reads or writes anything.
template <typename... Params, typename... Args>
inline int rows_launch(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, uint32_t cluster, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster ? cluster : 1u;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster ? 2u : 1u;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) == cudaSuccess ? 1 : -1;
}

#ifdef __CUDACC__

__device__ __forceinline__ void rows_begin() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- elements --------------------------------------------------------------------------------------------------------
template <typename T> struct RowsElem;
template <> struct RowsElem<float> {
    static __device__ __forceinline__ float up(float x) { return x; }
    static __device__ __forceinline__ float down(float x) { return x; }
};
template <> struct RowsElem<__half> {
    static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
};
template <> struct RowsElem<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
};

// N consecutive elements, moved as one access (aligned to their size).
template <typename T, int N>
struct alignas(sizeof(T) * N) RowsVec {
    T e[N];
};

// A raw access of B bytes.
template <int B> struct RowsRaw;
template <> struct RowsRaw<16> { typedef uint4 type; };
template <> struct RowsRaw<8> { typedef uint2 type; };
template <> struct RowsRaw<4> { typedef uint32_t type; };
template <> struct RowsRaw<2> { typedef uint16_t type; };
template <> struct RowsRaw<1> { typedef uint8_t type; };

// A row that is read once or written once and is larger, all rows together, than the caches: L2 need not keep it.
template <typename R> __device__ __forceinline__ R rows_load(const R* p) { return __ldg(p); }
template <typename R> __device__ __forceinline__ void rows_store(R* p, R v) { *p = v; }

template <typename T, int N>
__device__ __forceinline__ RowsVec<T, N> rows_load_vec(const T* p)
{
    typedef typename RowsRaw<sizeof(T) * N>::type R;
    RowsVec<T, N> v;
    *reinterpret_cast<R*>(&v) = rows_load(reinterpret_cast<const R*>(p));
    return v;
}
template <typename T, int N>
__device__ __forceinline__ void rows_store_vec(T* p, const RowsVec<T, N>& v)
{
    typedef typename RowsRaw<sizeof(T) * N>::type R;
    rows_store(reinterpret_cast<R*>(p), *reinterpret_cast<const R*>(&v));
}

#endif  // __CUDACC__

// Runs CALL(type) for the element type named by dtype.
#define ROWS_WITH_TYPE(dtype, CALL)                                   \
    do {                                                              \
        if ((dtype) == PEARL_F32) { CALL(float); }                    \
        else if ((dtype) == PEARL_F16) { CALL(__half); }              \
        else { CALL(__nv_bfloat16); }                                 \
    } while (0)
