// The handle of the row operators and what the host side of each call does with it.
#pragma once
#include "rows_internal.cuh"

struct pearl_rows {
    unsigned* status;           // two words: the status bits, and those that pearl_rows_sync() has taken
    bool owns_slab;
    int device;
    cudaStream_t stream;
    uint64_t launches;
};

namespace {

// Makes `dev` the current device for a call; the device that was current is so again afterwards.
struct DeviceGuard {
    int prev;
    bool ok, other;
    explicit DeviceGuard(int dev) : prev(-1), ok(true), other(false)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        other = prev != dev;
        if (other && cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() { if (other) cudaSetDevice(prev); }
};

bool misaligned(const void* p, uint32_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
// (a matrix of T rows of `row`, `ld` apart; one row needs no distance)
bool bad_ld(uint64_t T, uint64_t row, uint64_t ld) { return T > 1 && (ld < row || ld > (1ull << 40)); }
bool bad_type(uint32_t dtype) { return dtype > PEARL_BF16; }

// Enqueues `launch()` with the handle's device current and counts its kernels.
template <typename F> int enqueue(pearl_rows* h, F launch)
{
    DeviceGuard guard(h->device);
    if (!guard.ok) return PEARL_ERR_CUDA;
    const int n = launch();
    if (n < 0) { cudaGetLastError(); return PEARL_ERR_CUDA; }
    h->launches += (uint64_t)n;
    return PEARL_OK;
}

}  // namespace
