// The router: the k best of E experts with their softmax weights, and its gradient.
//
// L lanes have a row, N consecutive logits each, in registers.  The k choices are k rounds of "largest that is left": a
// maximum over the lane's logits, one over the lanes by exchanges, the first lane that has it takes its first such
// logit out.  Lanes and logits are in order, so the lower expert wins among equal ones.
#include "rows_internal.cuh"

namespace {

constexpr uint32_t kThreads = 256;
constexpr float kInf = __builtin_huge_valf();

template <int L> __device__ __forceinline__ float over_lanes_max(float v)
{
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d, L));
    return v;
}
template <int L> __device__ __forceinline__ float over_lanes_sum(float v)
{
#pragma unroll
    for (int d = L / 2; d > 0; d >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xFFFFFFFFu, v, d, L));
    return v;
}

// A lane's N elements as accesses of up to 16 bytes.
template <typename E, int N> struct Access {
    static constexpr int elements = (int)(sizeof(E) * N) <= 16 ? N : 16 / (int)sizeof(E);
};

// The lane's N logits of row t, -inf where the row has none; NaN and +inf become -inf, and are reported.
template <typename E, int N>
__device__ __forceinline__ bool load_logits(const E* row, uint32_t first, uint32_t experts, bool there, bool wide, float (&x)[N])
{
    if (wide && there && first + N <= experts) {
        constexpr int M = Access<E, N>::elements;
#pragma unroll
        for (int a = 0; a < N; a += M) {
            const RowsVec<E, M> v = rows_load_vec<E, M>(row + first + a);
#pragma unroll
            for (int i = 0; i < M; ++i) x[a + i] = v.get(i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = there && first + i < experts ? RowsElem<E>::up(row[first + i]) : -kInf;
    }
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (!(x[i] < kInf)) { bad = true; x[i] = -kInf; }
    return bad;
}

template <typename E, int L, int N>
__global__ void __launch_bounds__(kThreads) route_kernel(unsigned* status, uint32_t T, uint32_t experts, uint32_t k, const E* __restrict__ logits,
                                                         uint64_t ld, uint32_t wide, uint32_t over_chosen, float* __restrict__ w,
                                                         int32_t* __restrict__ ids)
{
    rows_begin();
    const uint32_t lane = threadIdx.x % L;
    const uint64_t t = (uint64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const bool there = t < T;
    float x[N];
    if (load_logits<E, N>(logits + (there ? t : 0) * ld, lane * N, experts, there, wide != 0, x)) atomicOr(status, PEARL_ST_BAD_SCORE);

    float best = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = fmaxf(best, x[i]);
    const float top = over_lanes_max<L>(best);
    const float shift = top == -kInf ? 0.0f : top;
    float sum = 0.0f;
    if (!over_chosen) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum = __fadd_rn(sum, __expf(__fsub_rn(x[i], shift)));
        sum = over_lanes_sum<L>(sum);
    }
    // choice j is kept by lane j % L of the row, in held[j / L]
    constexpr int kHeld = (PEARL_ROWS_MAX_CHOICES + L - 1) / L;
    float held_x[kHeld];
    int32_t held_id[kHeld];
    const uint32_t lanes = L == 32 ? 0xFFFFFFFFu : ((1u << (L & 31)) - 1u) << ((threadIdx.x & 31u) / L * L);
    float chosen_sum = 0.0f, gmax = top;
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        held_x[h] = -kInf;
        held_id[h] = -1;
        for (uint32_t j = h * L; j < (h + 1) * L && j < k; ++j) {
            const uint32_t have = __ballot_sync(0xFFFFFFFFu, best == gmax) & lanes;
            const uint32_t owner = (__ffs(have) - 1u) % L;
            int32_t at = -1;
            if (lane == owner) {
                bool found = false;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const bool hit = !found && x[i] == gmax;
                    if (hit) { at = (int32_t)(lane * N + i); x[i] = -kInf; }
                    found |= hit;
                }
                best = x[0];
#pragma unroll
                for (int i = 1; i < N; ++i) best = fmaxf(best, x[i]);
            }
            at = __shfl_sync(0xFFFFFFFFu, at, (int)owner, L);
            const bool shut = gmax == -kInf;
            if (lane == j - h * L) { held_x[h] = gmax; held_id[h] = shut ? -1 : at; }
            chosen_sum = __fadd_rn(chosen_sum, __expf(__fsub_rn(gmax, shift)));
            gmax = over_lanes_max<L>(best);
        }
    }
    if (!there) return;
    const float denominator = over_chosen ? chosen_sum : sum;
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const uint32_t j = h * L + lane;
        if (j < k) {
            ids[t * k + j] = held_id[h];
            w[t * k + j] = held_id[h] < 0 ? 0.0f : __fdiv_rn(__expf(__fsub_rn(held_x[h], shift)), denominator);
        }
    }
}

// The gradient: each lane builds its N gradients from the row's k (id, weight, dw).
template <typename E, int L, int N>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(unsigned* status, uint32_t T, uint32_t experts, uint32_t k,
                                                              const E* __restrict__ logits, uint64_t ld, uint32_t wide, uint32_t over_chosen,
                                                              const float* __restrict__ w, const int32_t* __restrict__ ids,
                                                              const float* __restrict__ dw, E* __restrict__ dlogits, uint64_t ld_d,
                                                              uint32_t wide_d)
{
    rows_begin();
    const uint32_t lane = threadIdx.x % L;
    const uint64_t t = (uint64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const bool there = t < T;
    float x[N], g[N];
#pragma unroll
    for (int i = 0; i < N; ++i) g[i] = 0.0f;
    float p_scale = 0.0f, shift = 0.0f;
    if (!over_chosen) {
        if (load_logits<E, N>(logits + (there ? t : 0) * ld, lane * N, experts, there, wide != 0, x)) atomicOr(status, PEARL_ST_BAD_SCORE);
        float best = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) best = fmaxf(best, x[i]);
        const float top = over_lanes_max<L>(best);
        shift = top == -kInf ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) sum = __fadd_rn(sum, __expf(__fsub_rn(x[i], shift)));
        sum = over_lanes_sum<L>(sum);
        p_scale = sum > 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;
    }
    if (!there) return;                     // (no exchange between lanes from here on)
    float mean = 0.0f;
    for (uint32_t j = 0; j < k; ++j)
        if ((uint32_t)ids[t * k + j] < experts) mean = __fmaf_rn(w[t * k + j], dw[t * k + j], mean);
    for (uint32_t j = 0; j < k; ++j) {
        const int32_t e = ids[t * k + j];
        if (e < -1 || e >= (int32_t)experts) {
            if (lane == 0) atomicOr(status, PEARL_ST_BAD_INDEX);
            continue;
        }
        const float d = dw[t * k + j];
        const float add = over_chosen ? __fmul_rn(w[t * k + j], __fsub_rn(d, mean)) : d;
        const uint32_t at = (uint32_t)e - lane * N;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e >= 0 && at == (uint32_t)i) g[i] = __fadd_rn(g[i], add);
    }
    constexpr int M = Access<E, N>::elements;
    RowsVec<E, M> out[N / M];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float v = over_chosen ? g[i] : __fmul_rn(__fmul_rn(__expf(__fsub_rn(x[i], shift)), p_scale), __fsub_rn(g[i], mean));
        out[i / M].put(i % M, v);
    }
    E* row = dlogits + t * ld_d;
    if (wide_d && lane * N + N <= experts) {
#pragma unroll
        for (int a = 0; a < N / M; ++a) rows_store_vec<E, M>(row + lane * N + a * M, out[a]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane * N + i < experts) row[lane * N + i] = RowsElem<E>::down(out[i / M].get(i % M));
    }
}

// Runs CALL(L, N): the lanes of a row and the logits of a lane for E experts (L * N >= E).
#define ROWS_WITH_SPREAD(E, CALL)                                               \
    do {                                                                        \
        if ((E) <= 8) { CALL(4, 2); }                                           \
        else if ((E) <= 16) { CALL(4, 4); }                                     \
        else if ((E) <= 32) { CALL(8, 4); }                                     \
        else if ((E) <= 64) { CALL(8, 8); }                                     \
        else if ((E) <= 128) { CALL(16, 8); }                                   \
        else if ((E) <= 256) { CALL(32, 8); }                                   \
        else if ((E) <= 512) { CALL(32, 16); }                                  \
        else { CALL(32, 32); }                                                  \
    } while (0)

// Whether every lane's N elements of every row can be moved as whole accesses.
template <typename E, int N> bool wide_rows(const void* p, uint64_t ld)
{
    constexpr uint64_t bytes = sizeof(E) * Access<E, N>::elements;
    return (uintptr_t)p % bytes == 0 && ld * sizeof(E) % bytes == 0;
}

}  // namespace

int rows_launch_route(unsigned* status, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                      bool over_chosen, float* w, int32_t* ids, cudaStream_t s)
{
    if (T == 0) return 0;
    int rc = -1;
#define ROWS_GO(L, N)                                                                                                        \
    do {                                                                                                                     \
        const uint32_t rows = kThreads / (L);                                                                                \
        rc = rows_launch(route_kernel<ROWS_T, L, N>, dim3((T + rows - 1) / rows), dim3(kThreads), 0, s, 0, status, T, E, k,  \
                         (const ROWS_T*)logits, ld, wide_rows<ROWS_T, N>(logits, ld) ? 1u : 0u, over_chosen ? 1u : 0u, w, ids); \
    } while (0)
#define ROWS_TYPE(X) do { typedef X ROWS_T; ROWS_WITH_SPREAD(E, ROWS_GO); } while (0)
    ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_GO
    return rc;
}

int rows_launch_route_grad(unsigned* status, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                           bool over_chosen, const float* w, const int32_t* ids, const float* dw, void* dlogits, uint64_t ld_d,
                           cudaStream_t s)
{
    if (T == 0) return 0;
    int rc = -1;
#define ROWS_GO(L, N)                                                                                                        \
    do {                                                                                                                     \
        const uint32_t rows = kThreads / (L);                                                                                \
        rc = rows_launch(route_grad_kernel<ROWS_T, L, N>, dim3((T + rows - 1) / rows), dim3(kThreads), 0, s, 0, status, T, E, k, \
                         (const ROWS_T*)logits, ld, wide_rows<ROWS_T, N>(logits, ld) ? 1u : 0u, over_chosen ? 1u : 0u, w, ids, dw, \
                         (ROWS_T*)dlogits, ld_d, wide_rows<ROWS_T, N>(dlogits, ld_d) ? 1u : 0u);                             \
    } while (0)
    ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_GO
    return rc;
}
