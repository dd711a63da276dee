// A whole expert layer for a few rows: the router's product and choice, the experts' two products, their weighted sum.
#include "layer_internal.cuh"

namespace {

constexpr uint32_t kWarps = 8;

// The parts of the scratch, in bytes from its start.
struct Layout {
    uint64_t logits, h, bytes;
};
Layout layout_of(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k)
{
    (void)D;
    Layout l;
    l.logits = 0;
    l.h = l.logits + ((uint64_t)T * E * 4 + 255) / 256 * 256;
    l.bytes = l.h + ((uint64_t)T * k * H * 4 + 255) / 256 * 256;
    return l;
}

template <typename E> __device__ __forceinline__ float element(const E* p) { return RowsElem<E>::up(*p); }

// logits[t, e]: a warp each, in binary64.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) logits_kernel(uint32_t rows, uint32_t D, uint32_t E, const T* x, uint64_t ld_x, const T* router, float* logits)
{
    rows_begin();
    const uint32_t i = blockIdx.x * kWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31u;
    if (i >= rows * E) return;
    const T *a = x + (uint64_t)(i / E) * ld_x, *b = router + (uint64_t)(i % E) * D;
    double s = 0.0;
    for (uint32_t d = lane; d < D; d += 32) s = __fma_rn((double)element(a + d), (double)element(b + d), s);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (lane == 0) logits[i] = (float)s;
}

// h[slot, j]: a warp each.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) up_kernel(unsigned* status, uint32_t D, uint32_t H, uint32_t E, uint32_t k, uint32_t act, const T* x, uint64_t ld_x,
                                                         const T* up, const int32_t* ids, float* h)
{
    rows_begin();
    const uint32_t j = blockIdx.x * kWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31u, slot = blockIdx.y;
    if (j >= H) return;
    const int32_t e = ids[slot];
    if ((uint32_t)e >= E) {
        if (e != -1 && j == 0 && lane == 0) atomicOr(status, PEARL_ST_BAD_INDEX);
        return;
    }
    const bool gated = act == PEARL_ACT_SILU_GATED;
    const T* a = x + (uint64_t)(slot / k) * ld_x;
    const T* g = up + ((uint64_t)(uint32_t)e * (gated ? 2 : 1) * H + j) * D;
    const T* v = gated ? g + (uint64_t)H * D : g;
    float sg = 0.0f, sv = 0.0f;
    for (uint32_t d = lane; d < D; d += 32) {
        const float f = element(a + d);
        sg = __fmaf_rn(f, element(g + d), sg);
        if (gated) sv = __fmaf_rn(f, element(v + d), sv);
    }
    sg = layer_warp_sum(sg);
    sv = layer_warp_sum(sv);
    if (lane == 0) h[(uint64_t)slot * H + j] = gated ? sg / (1.0f + expf(-sg)) * sv : (sg < 0.0f ? 0.0f : sg);
}

// y[t, d]: a warp each.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) down_kernel(uint32_t D, uint32_t H, uint32_t E, uint32_t k, const T* down, const float* w, const int32_t* ids,
                                                           const float* h, T* y, uint64_t ld_y)
{
    rows_begin();
    const uint32_t d = blockIdx.x * kWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31u, t = blockIdx.y;
    if (d >= D) return;
    float sum = 0.0f;
    for (uint32_t j = 0; j < k; ++j) {
        const uint32_t slot = t * k + j;
        const int32_t e = ids[slot];
        if ((uint32_t)e >= E) continue;
        const T* row = down + ((uint64_t)(uint32_t)e * D + d) * H;
        float s = 0.0f;
        for (uint32_t i = lane; i < H; i += 32) s = __fmaf_rn(h[(uint64_t)slot * H + i], element(row + i), s);
        sum = __fmaf_rn(w[slot], layer_warp_sum(s), sum);
    }
    if (lane == 0) y[(uint64_t)t * ld_y + d] = RowsElem<T>::down(sum);
}

template <typename T> int experts_as(unsigned* status, const LayerExperts& a, cudaStream_t s)
{
    const Layout l = layout_of(a.T, a.D, a.H, a.E, a.k);
    float *logits = (float*)((char*)a.work + l.logits), *h = (float*)((char*)a.work + l.h);
    int n = 0, m;
    if (a.router) {
        if ((m = rows_launch(logits_kernel<T>, dim3((a.T * a.E + kWarps - 1) / kWarps), dim3(kWarps * 32), 0, s, 0, a.T, a.D, a.E, (const T*)a.x,
                             a.ld_x, (const T*)a.router, logits)) < 0) return m;
        n += m;
        if ((m = rows_launch_route(status, a.T, a.E, a.k, PEARL_F32, logits, a.E, a.over_chosen, a.w, a.ids, s)) < 0) return m;
        n += m;
    }
    if ((m = rows_launch(up_kernel<T>, dim3((a.H + kWarps - 1) / kWarps, a.T * a.k), dim3(kWarps * 32), 0, s, 0, status, a.D, a.H, a.E, a.k, a.act,
                         (const T*)a.x, a.ld_x, (const T*)a.up, (const int32_t*)a.ids, h)) < 0) return m;
    n += m;
    if ((m = rows_launch(down_kernel<T>, dim3((a.D + kWarps - 1) / kWarps, a.T), dim3(kWarps * 32), 0, s, 0, a.D, a.H, a.E, a.k, (const T*)a.down,
                         (const float*)a.w, (const int32_t*)a.ids, (const float*)h, (T*)a.y, a.ld_y)) < 0) return m;
    return n + m;
}

}  // namespace

uint64_t layer_experts_work_bytes(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k) { return layout_of(T, D, H, E, k).bytes; }

int layer_launch_experts(unsigned* status, const LayerExperts& a, cudaStream_t s)
{
#define EXPERTS(T) return experts_as<T>(status, a, s)
    ROWS_WITH_TYPE(a.dtype, EXPERTS);
#undef EXPERTS
}
