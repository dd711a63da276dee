// Host side of the row operators: the handle, argument checks and the C ABI of include/pearl_rows.h.
#include <math.h>
#include <new>

#include "rows_handle.cuh"

namespace {

constexpr uint64_t kSlabBytes = 256;

// The bits so far, and none from here on, in one step: one that another stream raises meanwhile is among them or stays.
__global__ void take_status_kernel(unsigned* status)
{
    rows_begin();
    status[1] = atomicExch(status, 0u);
}

bool bad_slots(uint64_t T, uint64_t k) { return k < 1 || T * k > 0x7FFFFFFFull; }

// The bytes [first, last) that states of this layout occupy.
bool extent(uint32_t blocks, uint32_t G, uint32_t W, uint32_t pieces, uint64_t piece_bytes, const pearl_states_t* p, uint64_t* bytes)
{
    const long double all = (long double)(blocks - 1) * p->block_pitch + ((long double)G * W - 1) * p->state_pitch +
                            (long double)(pieces - 1) * p->piece_pitch + piece_bytes;
    if (all > 9.0e15L) return false;
    *bytes = (uint64_t)(blocks - 1) * p->block_pitch + ((uint64_t)G * W - 1) * p->state_pitch + (uint64_t)(pieces - 1) * p->piece_pitch + piece_bytes;
    return true;
}

}  // namespace

extern "C" {

uint64_t pearl_rows_slab_bytes(void) { return kSlabBytes; }

int pearl_rows_create(pearl_rows_t** out, int device, void* cuda_stream, void* slab, uint64_t slab_bytes)
{
    if (!out) return PEARL_ERR_NULL;
    if (slab && slab_bytes < kSlabBytes) return PEARL_ERR_OOM;
    if (slab && misaligned(slab, 256)) return PEARL_ERR_ALIGN;
    DeviceGuard guard(device);
    if (!guard.ok) { cudaGetLastError(); return PEARL_ERR_CUDA; }
    pearl_rows* h = new (std::nothrow) pearl_rows();
    if (!h) return PEARL_ERR_OOM;
    h->device = device;
    h->stream = (cudaStream_t)cuda_stream;
    h->launches = 0;
    h->owns_slab = slab == nullptr;
    void* p = slab;
    if (!p && cudaMalloc(&p, kSlabBytes) != cudaSuccess) { cudaGetLastError(); delete h; return PEARL_ERR_OOM; }
    h->status = (unsigned*)p;
    if (cudaMemsetAsync(p, 0, kSlabBytes, h->stream) != cudaSuccess) {
        cudaGetLastError();
        if (h->owns_slab) cudaFree(p);
        delete h;
        return PEARL_ERR_CUDA;
    }
    *out = h;
    return PEARL_OK;
}

int pearl_rows_destroy(pearl_rows_t* h)
{
    if (!h) return PEARL_ERR_NULL;
    DeviceGuard guard(h->device);
    int rc = PEARL_OK;
    if (cudaStreamSynchronize(h->stream) != cudaSuccess) rc = PEARL_ERR_CUDA;
    if (h->owns_slab && cudaFree(h->status) != cudaSuccess) rc = PEARL_ERR_CUDA;
    delete h;
    return rc;
}

int pearl_rows_route(pearl_rows_t* h, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                     int over_chosen, float* w, int32_t* ids)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || E < 1 || E > PEARL_ROWS_MAX_EXPERTS || k < 1 || k > E || k > PEARL_ROWS_MAX_CHOICES) return PEARL_ERR_BAD_ARG;
    if (bad_slots(T, k)) return PEARL_ERR_BAD_BATCH;
    if (bad_ld(T, E, ld)) return PEARL_ERR_BAD_ARG;
    if (T == 0) return PEARL_OK;
    if (!logits || !w || !ids) return PEARL_ERR_NULL;
    if (misaligned(logits, rows_elem_bytes(dtype)) || misaligned(w, 4) || misaligned(ids, 4)) return PEARL_ERR_ALIGN;
    return enqueue(h, [&] { return rows_launch_route(h->status, T, E, k, dtype, logits, ld, over_chosen != 0, w, ids, h->stream); });
}

int pearl_rows_route_grad(pearl_rows_t* h, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                          int over_chosen, const float* w, const int32_t* ids, const float* dw, void* dlogits, uint64_t ld_d)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || E < 1 || E > PEARL_ROWS_MAX_EXPERTS || k < 1 || k > E || k > PEARL_ROWS_MAX_CHOICES) return PEARL_ERR_BAD_ARG;
    if (bad_slots(T, k)) return PEARL_ERR_BAD_BATCH;
    if ((!over_chosen && bad_ld(T, E, ld)) || bad_ld(T, E, ld_d)) return PEARL_ERR_BAD_ARG;
    if (T == 0) return PEARL_OK;
    if ((!over_chosen && !logits) || !w || !ids || !dw || !dlogits) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype);
    if ((!over_chosen && misaligned(logits, S)) || misaligned(dlogits, S) || misaligned(w, 4) || misaligned(ids, 4) || misaligned(dw, 4))
        return PEARL_ERR_ALIGN;
    return enqueue(h, [&] {
        return rows_launch_route_grad(h->status, T, E, k, dtype, logits, ld, over_chosen != 0, w, ids, dw, dlogits, ld_d, h->stream);
    });
}

int pearl_rows_sort(pearl_rows_t* h, uint32_t slots, uint32_t E, const int32_t* ids, int32_t* offsets, int32_t* order, int32_t* place)
{
    if (!h) return PEARL_ERR_NULL;
    if (E < 1 || E > PEARL_ROWS_MAX_EXPERTS) return PEARL_ERR_BAD_ARG;
    if (slots > 0x7FFFFFFFu) return PEARL_ERR_BAD_BATCH;
    if (!offsets || (slots && (!ids || !place))) return PEARL_ERR_NULL;
    if (misaligned(ids, 4) || misaligned(offsets, 4) || misaligned(order, 4) || misaligned(place, 4)) return PEARL_ERR_ALIGN;
    return enqueue(h, [&] { return rows_launch_sort(h->status, slots, E, ids, offsets, order, place, h->stream); });
}

int pearl_rows_dispatch(pearl_rows_t* h, uint32_t T, uint32_t k, uint32_t row_bytes, const void* x, uint64_t ld_x, const int32_t* place,
                        uint32_t sorted_rows, void* xs)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_slots(T, k)) return PEARL_ERR_BAD_BATCH;
    if (row_bytes < 1 || row_bytes > PEARL_ROWS_MAX_ROW_BYTES || bad_ld(T, row_bytes, ld_x)) return PEARL_ERR_BAD_ARG;
    if (T == 0) return PEARL_OK;
    if (!x || !place || (!xs && sorted_rows)) return PEARL_ERR_NULL;
    if (misaligned(place, 4)) return PEARL_ERR_ALIGN;
    return enqueue(h, [&] { return rows_launch_dispatch(h->status, T, k, row_bytes, x, T > 1 ? ld_x : 0, place, sorted_rows, xs, h->stream); });
}

int pearl_rows_combine(pearl_rows_t* h, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* z, uint32_t sorted_rows,
                       const int32_t* place, const float* w, void* y, uint64_t ld_y)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || D < 1 || D > PEARL_ROWS_MAX_ROW_BYTES / rows_elem_bytes(dtype) || bad_ld(T, D, ld_y)) return PEARL_ERR_BAD_ARG;
    if (bad_slots(T, k)) return PEARL_ERR_BAD_BATCH;
    if (T == 0) return PEARL_OK;
    if ((!z && sorted_rows) || !place || !y) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype);
    if (misaligned(z, S) || misaligned(y, S) || misaligned(place, 4) || misaligned(w, 4)) return PEARL_ERR_ALIGN;
    return enqueue(h, [&] {
        return rows_launch_combine(h->status, T, k, D, dtype, z, sorted_rows, place, w, y, T > 1 ? ld_y : 0, h->stream);
    });
}

int pearl_rows_combine_grad(pearl_rows_t* h, uint32_t T, uint32_t k, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy,
                            const void* z, uint32_t sorted_rows, const int32_t* place, const float* w, void* dz, float* dw)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || D < 1 || D > PEARL_ROWS_MAX_ROW_BYTES / rows_elem_bytes(dtype) || bad_ld(T, D, ld_dy)) return PEARL_ERR_BAD_ARG;
    if (bad_slots(T, k)) return PEARL_ERR_BAD_BATCH;
    if (T == 0) return PEARL_OK;
    if (!dy || !place || (!dz && !dw && sorted_rows) || (dw && !z && sorted_rows)) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype);
    if (misaligned(dy, S) || misaligned(z, S) || misaligned(dz, S) || misaligned(place, 4) || misaligned(w, 4) || misaligned(dw, 4))
        return PEARL_ERR_ALIGN;
    return enqueue(h, [&] {
        return rows_launch_combine_grad(h->status, T, k, D, dtype, dy, T > 1 ? ld_dy : 0, z, sorted_rows, place, w, dz, dw, h->stream);
    });
}

int pearl_rows_beam_select(pearl_rows_t* h, uint32_t G, uint32_t W, uint32_t V, uint32_t C, uint32_t dtype, const void* logits,
                           uint64_t ld, const float* scores, const uint8_t* done, int32_t end_token, float* best_score,
                           int32_t* best_beam, int32_t* best_token)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || W < 1 || W > PEARL_ROWS_MAX_BEAMS || C < 1 || C > PEARL_ROWS_MAX_BEST || V < 1 || V > PEARL_ROWS_MAX_VOCAB ||
        bad_ld((uint64_t)G * W, V, ld))
        return PEARL_ERR_BAD_ARG;
    if (G > (1u << 24)) return PEARL_ERR_BAD_BATCH;
    if (G == 0) return PEARL_OK;
    if (!logits || !scores || !best_score || !best_beam || !best_token) return PEARL_ERR_NULL;
    if (misaligned(logits, rows_elem_bytes(dtype)) || misaligned(scores, 4) || misaligned(best_score, 4) || misaligned(best_beam, 4) ||
        misaligned(best_token, 4))
        return PEARL_ERR_ALIGN;
    return enqueue(h, [&] {
        return rows_launch_beam_select(h->status, G, W, V, C, dtype, logits, ld, scores, done, end_token, best_score, best_beam, best_token,
                                       h->stream);
    });
}

int pearl_rows_beam_reorder(pearl_rows_t* h, uint32_t blocks, uint32_t G, uint32_t W, uint32_t pieces, uint64_t piece_bytes,
                            const int32_t* parent, const void* src, const pearl_states_t* sp, void* dst, const pearl_states_t* dp)
{
    if (!h) return PEARL_ERR_NULL;
    if (W < 1 || W > PEARL_ROWS_MAX_BEAMS) return PEARL_ERR_BAD_ARG;
    if (blocks == 0 || G == 0 || pieces == 0 || piece_bytes == 0) return PEARL_OK;
    if ((uint64_t)blocks * G > 0x7FFFFFFFull) return PEARL_ERR_BAD_BATCH;           // (each has a block of threads at least)
    if (!parent || !src || !dst || !sp || !dp) return PEARL_ERR_NULL;
    if (misaligned(parent, 4)) return PEARL_ERR_ALIGN;
    uint64_t sb = 0, db = 0;
    if (!extent(blocks, G, W, pieces, piece_bytes, sp, &sb) || !extent(blocks, G, W, pieces, piece_bytes, dp, &db)) return PEARL_ERR_BAD_ARG;
    // The states of dst must be apart from one another: pitches sorted, each level spans less than the next one's pitch.  (States
    // between whose pieces other states' pieces lie, as in [.., heads, beams, ..], are in order too.)
    {
        uint64_t pitch[3] = { dp->piece_pitch, dp->state_pitch, dp->block_pitch };
        uint64_t count[3] = { pieces, (uint64_t)G * W, blocks };
        for (int i = 0; i < 3; ++i)
            for (int j = i + 1; j < 3; ++j)
                if (pitch[j] < pitch[i]) {
                    const uint64_t p = pitch[i], c = count[i];
                    pitch[i] = pitch[j]; count[i] = count[j];
                    pitch[j] = p; count[j] = c;
                }
        uint64_t span = piece_bytes;
        for (int i = 0; i < 3; ++i) {
            if (count[i] <= 1) continue;
            if (pitch[i] < span) return PEARL_ERR_BAD_ARG;
            span += (count[i] - 1) * pitch[i];
        }
    }
    if (src == dst) {
        if (sp->block_pitch != dp->block_pitch || sp->state_pitch != dp->state_pitch || sp->piece_pitch != dp->piece_pitch)
            return PEARL_ERR_BAD_ARG;
    } else if ((uintptr_t)src < (uintptr_t)dst + db && (uintptr_t)dst < (uintptr_t)src + sb) {
        return PEARL_ERR_BAD_ARG;
    }
    return enqueue(h, [&] { return rows_launch_beam_reorder(h->status, blocks, G, W, pieces, piece_bytes, parent, src, *sp, dst, *dp, h->stream); });
}

int pearl_rows_sync(pearl_rows_t* h, uint32_t* status_bits)
{
    if (!h) return PEARL_ERR_NULL;
    DeviceGuard guard(h->device);
    if (!guard.ok) return PEARL_ERR_CUDA;
    uint32_t st = 0;
    const auto read = [&](const unsigned* word) {
        return cudaMemcpyAsync(&st, word, 4, cudaMemcpyDeviceToHost, h->stream) == cudaSuccess && cudaStreamSynchronize(h->stream) == cudaSuccess;
    };
    if (!read(h->status)) return PEARL_ERR_CUDA;
    if (st) {
        const int n = rows_launch(take_status_kernel, dim3(1), dim3(1), 0, h->stream, 0, h->status);
        if (n < 0) { cudaGetLastError(); return PEARL_ERR_CUDA; }
        h->launches += (uint64_t)n;
        if (!read(h->status + 1)) return PEARL_ERR_CUDA;
    }
    if (status_bits) *status_bits = st;
    return PEARL_OK;
}

uint64_t pearl_rows_kernel_launches(pearl_rows_t* h) { return h ? h->launches : 0; }

}  // extern "C"
