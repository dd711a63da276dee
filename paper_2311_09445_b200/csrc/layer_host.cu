// Host side of a layer's operators: argument checks and the C ABI of include/pearl_layers.h.
#include <math.h>

#include "layer_internal.cuh"
#include "rows_handle.cuh"

namespace {

bool bad_params(uint32_t ptype, uint32_t dtype) { return ptype != PEARL_F32 && ptype != dtype; }
uint64_t apart(uint32_t T, uint64_t ld) { return T > 1 ? ld : 0; }

}  // namespace

extern "C" {

int pearl_layer_norm(pearl_rows_t* h, uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, uint32_t ptype, const void* gamma,
                     const void* beta, double eps, void* y, uint64_t ld_y, float* mean, float* rstd)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || bad_params(ptype, dtype) || D < 1 || D > PEARL_LAYER_MAX_WIDTH || bad_ld(T, D, ld_x) || bad_ld(T, D, ld_y) ||
        !(eps >= 0.0) || !(eps <= 3.0e38))
        return PEARL_ERR_BAD_ARG;
    if (T > 0x7FFFFFFFu) return PEARL_ERR_BAD_BATCH;
    if (T == 0) return PEARL_OK;
    if (!x || !y) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype), P = rows_elem_bytes(ptype);
    if (misaligned(x, S) || misaligned(y, S) || misaligned(gamma, P) || misaligned(beta, P) || misaligned(mean, 4) || misaligned(rstd, 4))
        return PEARL_ERR_ALIGN;
    return enqueue(h, [&] {
        return layer_launch_norm(h->status, T, D, dtype, x, apart(T, ld_x), ptype, gamma, beta, (float)eps, y, apart(T, ld_y), mean, rstd, h->stream);
    });
}

uint64_t pearl_layer_norm_grad_work_bytes(uint32_t T, uint32_t D)
{
    return D < 1 || D > PEARL_LAYER_MAX_WIDTH ? 0 : layer_norm_grad_work_bytes(T, D);
}

int pearl_layer_norm_grad(pearl_rows_t* h, uint32_t T, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x,
                          const float* mean, const float* rstd, uint32_t ptype, const void* gamma, void* dx, uint64_t ld_dx, float* dgamma,
                          float* dbeta, void* work, uint64_t work_bytes)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || bad_params(ptype, dtype) || D < 1 || D > PEARL_LAYER_MAX_WIDTH || bad_ld(T, D, ld_dy) || bad_ld(T, D, ld_x) ||
        (dx && bad_ld(T, D, ld_dx)))
        return PEARL_ERR_BAD_ARG;
    if (T > 0x7FFFFFFFu) return PEARL_ERR_BAD_BATCH;
    const bool params = dgamma || dbeta;
    if (!dx && !params) return PEARL_ERR_NULL;
    if (T == 0 && !params) return PEARL_OK;
    if (T && (!dy || !x || !mean || !rstd)) return PEARL_ERR_NULL;
    if (params && !work) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype);
    if (misaligned(dy, S) || misaligned(x, S) || misaligned(dx, S) || misaligned(gamma, rows_elem_bytes(ptype)) || misaligned(mean, 4) ||
        misaligned(rstd, 4) || misaligned(dgamma, 4) || misaligned(dbeta, 4) || (params && misaligned(work, 256)))
        return PEARL_ERR_ALIGN;
    if (params && work_bytes < layer_norm_grad_work_bytes(T, D)) return PEARL_ERR_OOM;
    return enqueue(h, [&] {
        return layer_launch_norm_grad(h->status, T, D, dtype, dy, apart(T, ld_dy), x, apart(T, ld_x), mean, rstd, ptype, gamma, dx,
                                      apart(T, ld_dx), dgamma, dbeta, (float*)work, work_bytes, h->stream);
    });
}

int pearl_layer_dropout(pearl_rows_t* h, uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, const void* residual,
                        uint64_t ld_r, double p, uint64_t seed, uint64_t call, const uint64_t* calls, void* y, uint64_t ld_y)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || D < 1 || D > PEARL_ROWS_MAX_ROW_BYTES / rows_elem_bytes(dtype) || bad_ld(T, D, ld_x) || bad_ld(T, D, ld_y) ||
        (residual && bad_ld(T, D, ld_r)) || !(p >= 0.0) || !(p <= 1.0))
        return PEARL_ERR_BAD_ARG;
    if (T > 0x7FFFFFFFu) return PEARL_ERR_BAD_BATCH;
    if (T == 0) return PEARL_OK;
    if (!x || !y) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype);
    if (misaligned(x, S) || misaligned(y, S) || misaligned(residual, S) || misaligned(calls, 8)) return PEARL_ERR_ALIGN;
    // In place means in place: the same rows, not rows that run into them.
    if ((y == x && T > 1 && ld_x != ld_y) || (y == residual && T > 1 && ld_r != ld_y)) return PEARL_ERR_BAD_ARG;
    const uint32_t below = (uint32_t)floor(65536.0 * p + 0.5);
    const float scale = below < 65536u ? (float)(65536.0 / (double)(65536u - below)) : 0.0f;
    return enqueue(h, [&] {
        return layer_launch_dropout(h->status, T, D, dtype, x, apart(T, ld_x), residual, apart(T, ld_r), below, scale, seed, call, calls, y,
                                    apart(T, ld_y), h->stream);
    });
}

static bool bad_layer(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k)
{
    return D < 1 || D > PEARL_LAYER_MAX_INNER || H < 1 || H > PEARL_LAYER_MAX_INNER || E < 1 || E > PEARL_ROWS_MAX_EXPERTS || k < 1 || k > E ||
           k > PEARL_ROWS_MAX_CHOICES;
}

uint64_t pearl_layer_experts_work_bytes(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k)
{
    return bad_layer(T, D, H, E, k) || T > PEARL_LAYER_MAX_FEW ? 0 : layer_experts_work_bytes(T, D, H, E, k);
}

int pearl_layer_experts(pearl_rows_t* h, uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k, uint32_t dtype, uint32_t act, const void* x,
                        uint64_t ld_x, const void* router, int over_chosen, const void* up, const void* down, float* w, int32_t* ids, void* y,
                        uint64_t ld_y, void* work, uint64_t work_bytes)
{
    if (!h) return PEARL_ERR_NULL;
    if (bad_type(dtype) || act > PEARL_ACT_RELU || bad_layer(T, D, H, E, k) || bad_ld(T, D, ld_x) || bad_ld(T, D, ld_y)) return PEARL_ERR_BAD_ARG;
    if (T > PEARL_LAYER_MAX_FEW) return PEARL_ERR_BAD_BATCH;
    if (T == 0) return PEARL_OK;
    if (!x || !up || !down || !w || !ids || !y || !work) return PEARL_ERR_NULL;
    const uint32_t S = rows_elem_bytes(dtype);
    if (misaligned(x, S) || misaligned(router, S) || misaligned(up, S) || misaligned(down, S) || misaligned(y, S) || misaligned(w, 4) ||
        misaligned(ids, 4) || misaligned(work, 256))
        return PEARL_ERR_ALIGN;
    if (work_bytes < layer_experts_work_bytes(T, D, H, E, k)) return PEARL_ERR_OOM;
    const LayerExperts a = { T, D, H, E, k, dtype, act, over_chosen != 0, x, router, up, down, apart(T, ld_x), apart(T, ld_y), w, ids, y, work };
    return enqueue(h, [&] { return layer_launch_experts(h->status, a, h->stream); });
}

}  // extern "C"
