// Internal declarations shared by the translation units of the row operators (include/pearl_rows.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "../../include/pearl_rows.h"

// The checked build (-DPEARL_CHECKED) compares what kernels compute with the extents: the 16-byte words of rows at odd places, read and
// stored (RowsAny, rows_store_part), and the words of a selection's ring; the moved states' accesses; the router's logits and gradients at a
// row's end and its experts' places in shared memory; the sort's staged slots and places; a selection's lists; and the experts, places
// and tokens that are handed out.  One out of range raises PEARL_ST_INTERNAL and the access is skipped.  (Indices that the caller gives --
// ids, places, parents -- are compared in every build.)
#ifdef PEARL_CHECKED
#define ROWS_IN_BOUNDS(status, cond) ((cond) ? true : (atomicOr((status), PEARL_ST_INTERNAL), false))
#else
#define ROWS_IN_BOUNDS(status, cond) (true)
#endif
// Whether `bytes` bytes from p on lie in [lo, hi).
#define ROWS_IN_ARRAY(status, p, bytes, lo, hi)                                                                      \
    ROWS_IN_BOUNDS(status, (uintptr_t)(p) >= (uintptr_t)(lo) && (uintptr_t)(p) + (uintptr_t)(bytes) <= (uintptr_t)(hi))

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

// The widest access (32, 16, 8, 4, 2 or 1 bytes) that every one of these byte counts and addresses is a multiple of.
inline uint32_t rows_granule(uint64_t a, uint64_t b = 0, uint64_t c = 0, uint64_t d = 0, uint64_t e = 0)
{
    const uint64_t all = a | b | c | d | e | 32u;
    return (uint32_t)(all & (~all + 1u));
}

// The current device (0 .. 63; -1 where it cannot be told) and its SMs.
constexpr int kRowsMaxDevices = 64;
inline int rows_device()
{
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < kRowsMaxDevices ? dev : -1;
}
inline uint32_t rows_sm_count()
{
    static std::atomic<uint32_t> known[kRowsMaxDevices];
    const int dev = rows_device();
    if (dev < 0) return 148;
    if (known[dev] == 0) {
        int n = 0;
        known[dev] = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0 ? (uint32_t)n : 148u;
    }
    return known[dev];
}
// Lets a kernel be launched in clusters of more than 8 CTAs and, with smem, with that much shared memory (once per kernel and
// device; one call site per kernel).
template <typename... Params> inline bool rows_large_cluster(void (*kernel)(Params...), int smem = 0)
{
    struct Known { const void* kernel; bool done[kRowsMaxDevices]; };
    static Known known[8];
    static std::mutex lock;                  // (handles of several host threads share the table)
    const std::lock_guard<std::mutex> held(lock);
    const int dev = rows_device();
    for (Known& k : known) {
        if (k.kernel != nullptr && k.kernel != (const void*)kernel) continue;
        if (dev >= 0 && k.kernel != nullptr && k.done[dev]) return true;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return false;
        if (smem && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return false;
        k.kernel = (const void*)kernel;
        if (dev >= 0) k.done[dev] = true;
        return true;
    }
    return false;
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

// Waits for the kernel before.  What a kernel reads may still be written until then, so nothing here promises that it stays as it is
// while the kernel runs: no pointer is __restrict__ and no load goes through the read-only path, which would let it move ahead of this.
// Operands are read by plain loads, which stay behind the "memory" here, and by `volatile` ones, which stay behind this one.
__device__ __forceinline__ void rows_begin() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// *p if `there`, else `otherwise`: one predicated load.
__device__ __forceinline__ int32_t rows_read_if(bool there, const int32_t* p, int32_t otherwise)
{
    asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q ld.global.b32 %0, [%1]; }" : "+r"(otherwise) : "l"(p), "r"((uint32_t)there));
    return otherwise;
}
__device__ __forceinline__ float rows_read_if(bool there, const float* p, float otherwise)
{
    return __int_as_float(rows_read_if(there, reinterpret_cast<const int32_t*>(p), __float_as_int(otherwise)));
}

// ---- elements --------------------------------------------------------------------------------------------------------
template <typename T> struct RowsElem;
template <> struct RowsElem<float> {
    static __device__ __forceinline__ float up(float x) { return x; }
    static __device__ __forceinline__ float down(float x) { return x; }
};
template <> struct RowsElem<__half> {
    static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
    static __device__ __forceinline__ uint16_t bits(__half x) { return __half_as_ushort(x); }
    static __device__ __forceinline__ __half from_bits(uint16_t b) { return __ushort_as_half(b); }
    static __device__ __forceinline__ float2 up2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ uint32_t down2(float lo, float hi)
    {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <> struct RowsElem<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ uint16_t bits(__nv_bfloat16 x) { return __bfloat16_as_ushort(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_bits(uint16_t b) { return __ushort_as_bfloat16(b); }
    static __device__ __forceinline__ float2 up2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ uint32_t down2(float lo, float hi)
    {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

// A raw access of B bytes: what is loaded and stored at once.  sm_100 moves 32 bytes a thread: a copy of 131048 rows of 4 KB to
// eight places each runs at 6190 GB/s with them, 5980 with 16.
template <int B> struct RowsRaw {
    uint32_t r[B / 4];
};
template <> struct RowsRaw<2> {
    uint16_t r[1];
};
template <> struct RowsRaw<1> {
    uint8_t r[1];
};

// Loads *p if `there`, else leaves v as it is: a predicated load, so that several of them are in flight together.  kKept: the bytes
// may be written by this kernel (a move in place), so the loads stay in front of the stores that follow them.
template <bool kKept, int B>
__device__ __forceinline__ void rows_load_if(bool there, RowsRaw<B>& v, const void* p)
{
    if constexpr (B == 32) {
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %9, 0; @q ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8]; }"
                     : "+r"(v.r[0]), "+r"(v.r[1]), "+r"(v.r[2]), "+r"(v.r[3]), "+r"(v.r[4]), "+r"(v.r[5]), "+r"(v.r[6]), "+r"(v.r[7])
                     : "l"(p), "r"((uint32_t)there));
    } else if constexpr (B == 16) {
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %5, 0; @q ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4]; }"
                     : "+r"(v.r[0]), "+r"(v.r[1]), "+r"(v.r[2]), "+r"(v.r[3]) : "l"(p), "r"((uint32_t)there));
    } else if constexpr (B == 8) {
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %3, 0; @q ld.global.v2.b32 {%0, %1}, [%2]; }"
                     : "+r"(v.r[0]), "+r"(v.r[1]) : "l"(p), "r"((uint32_t)there));
    } else if constexpr (B == 4) {
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q ld.global.b32 %0, [%1]; }" : "+r"(v.r[0]) : "l"(p), "r"((uint32_t)there));
    } else if constexpr (B == 2) {
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q ld.global.b16 %0, [%1]; }" : "+h"(v.r[0]) : "l"(p), "r"((uint32_t)there));
    } else {
        uint32_t byte = v.r[0];
        asm volatile("{ .reg .pred q; setp.ne.u32 q, %2, 0; @q ld.global.u8 %0, [%1]; }" : "+r"(byte) : "l"(p), "r"((uint32_t)there));
        v.r[0] = (uint8_t)byte;
    }
    if constexpr (kKept) asm volatile("" ::: "memory");
}
template <int B>
__device__ __forceinline__ void rows_store(void* p, const RowsRaw<B>& v)
{
    if constexpr (B == 32)
        asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(v.r[0]), "r"(v.r[1]), "r"(v.r[2]), "r"(v.r[3]),
                     "r"(v.r[4]), "r"(v.r[5]), "r"(v.r[6]), "r"(v.r[7]), "l"(p) : "memory");
    else if constexpr (B == 16)
        *reinterpret_cast<uint4*>(p) = make_uint4(v.r[0], v.r[1], v.r[2], v.r[3]);
    else if constexpr (B == 8)
        *reinterpret_cast<uint2*>(p) = make_uint2(v.r[0], v.r[1]);
    else if constexpr (B == 4)
        *reinterpret_cast<uint32_t*>(p) = v.r[0];
    else if constexpr (B == 2)
        *reinterpret_cast<uint16_t*>(p) = v.r[0];
    else
        *reinterpret_cast<uint8_t*>(p) = v.r[0];
}

// ---- rows that do not start on 16-byte boundaries ---------------------------------------------------------------------
// Such rows are moved by whole 16-byte words of the destination: a word's bytes come from the two words of the source that hold
// them, shifted together, and only the words at a row's ends are stored in parts.  S: 1 or 2, what every address is a multiple of (rows
// on 4-byte boundaries move faster by accesses of that size: 8192 sums of 4 rows of 2047 binary16 elements 92 us by 2 bytes, 57 so;
// of 2046 elements 51 by 4 bytes, 57 so).

// The 16 bytes at p, in two steps, so that several such reads are in flight together.  Words that lie in part outside [lo, hi), the
// array that p points into, are not read as such; bytes outside it are 0.  kKept: as for rows_load_if.
template <int S, bool kKept = false>
struct RowsAny {
    RowsRaw<16> v, w;
    __device__ __forceinline__ static bool whole(const unsigned char* p, const unsigned char* lo, const unsigned char* hi)
    {
        const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
        return (p - off >= lo) & (p - off + (off ? 32 : 16) <= hi);
    }
    __device__ __forceinline__ void fetch(unsigned* status, bool there, const unsigned char* p, const unsigned char* lo, const unsigned char* hi)
    {
        const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
        bool words = there & whole(p, lo, hi);
        if (words) words = ROWS_IN_ARRAY(status, p - off, off ? 32 : 16, lo, hi);
        rows_load_if<kKept>(words, v, p - off);
        rows_load_if<kKept>(words & (off != 0), w, p - off + 16);
    }
    __device__ __forceinline__ const RowsRaw<16>& get(const unsigned char* p, const unsigned char* lo, const unsigned char* hi)
    {
        const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
        if (off & 8u) { v.r[0] = v.r[2]; v.r[1] = v.r[3]; v.r[2] = w.r[0]; v.r[3] = w.r[1]; w.r[0] = w.r[2]; w.r[1] = w.r[3]; }
        if (off & 4u) { v.r[0] = v.r[1]; v.r[1] = v.r[2]; v.r[2] = v.r[3]; v.r[3] = w.r[0]; w.r[0] = w.r[1]; }
        const uint32_t bits = (off & 3u) * 8u;
        v.r[0] = __funnelshift_r(v.r[0], v.r[1], bits);
        v.r[1] = __funnelshift_r(v.r[1], v.r[2], bits);
        v.r[2] = __funnelshift_r(v.r[2], v.r[3], bits);
        v.r[3] = __funnelshift_r(v.r[3], w.r[0], bits);
        if (!whole(p, lo, hi)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v.r[i] = 0u;
#pragma unroll
            for (int i = 0; i < 16; i += S) {
                const unsigned char* at = p + i;
                if (at < lo || at + S > hi) continue;
                if constexpr (S == 2) v.r[i / 4] |= (uint32_t)*reinterpret_cast<const uint16_t*>(at) << (i % 4 * 8);
                else v.r[i / 4] |= (uint32_t)*at << (i % 4 * 8);
            }
        }
        return v;
    }
};
// Bytes [from, to) of a word, to the 16-byte boundary p, which is in (or beside) an array [lo, hi).
template <int S>
__device__ __forceinline__ void rows_store_part(unsigned* status, unsigned char* p, const RowsRaw<16>& v, int from, int to, const void* lo, const void* hi)
{
    if (!ROWS_IN_ARRAY(status, p + (from > 0 ? from : 0), (to < 16 ? to : 16) - (from > 0 ? from : 0), lo, hi)) return;
    if (from <= 0 && to >= 16) {
        rows_store(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; i += S) {
        if (i < from || i >= to) continue;
        if constexpr (S == 2) *reinterpret_cast<uint16_t*>(p + i) = (uint16_t)(v.r[i / 4] >> (i % 4 * 8));
        else p[i] = (unsigned char)(v.r[i / 4] >> (i % 4 * 8));
    }
}
// Rows of at least this many bytes are moved so: below, the words at the ends are most of a row.
constexpr uint32_t kRowsAnyBytes = 128;

// N consecutive elements, moved as one access.
template <typename T, int N>
union RowsVec {
    RowsRaw<(int)sizeof(T) * N> raw;
    uint32_t word[(sizeof(T) * N + 3) / 4];
    __device__ __forceinline__ RowsVec() {}
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * N + 3) / 4; ++i) word[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw.r[i]);
        else if constexpr (N == 1) return RowsElem<T>::up(RowsElem<T>::from_bits(raw.r[0]));
        else { const float2 f = RowsElem<T>::up2(raw.r[i / 2]); return i % 2 ? f.y : f.x; }
    }
    __device__ __forceinline__ void set(const float* x)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i) raw.r[i] = __float_as_uint(x[i]);
        } else if constexpr (N == 1) {
            raw.r[0] = RowsElem<T>::bits(RowsElem<T>::down(x[0]));
        } else {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) raw.r[i] = RowsElem<T>::down2(x[2 * i], x[2 * i + 1]);
        }
    }
};
template <typename T, int N>
__device__ __forceinline__ RowsVec<T, N> rows_load_vec(const T* p)
{
    RowsVec<T, N> v;
    rows_load_if<false>(true, v.raw, p);
    return v;
}
template <typename T, int N>
__device__ __forceinline__ void rows_store_vec(T* p, const RowsVec<T, N>& v) { rows_store(p, v.raw); }

#endif  // __CUDACC__

// Runs CALL(type) for the element type named by dtype.
#define ROWS_WITH_TYPE(dtype, CALL)                                   \
    do {                                                              \
        if ((dtype) == PEARL_F32) { CALL(float); }                    \
        else if ((dtype) == PEARL_F16) { CALL(__half); }              \
        else { CALL(__nv_bfloat16); }                                 \
    } while (0)
