// Slots sorted by expert: a stable counting sort in one launch.
//
// One thread-block cluster has all the slots, each of its CTAs a run of them, each warp a run of its CTA's.  Counts per warp and
// expert lie in shared memory; the CTAs read each other's sums through it and meet at the cluster's barrier, so nothing goes
// through global memory and no CTA waits for one that may not be there.  A warp then walks its run in order, 32 slots at a
// time: the slots of one expert among them are ranked by lane, which keeps the sort stable.
#include <cooperative_groups.h>

#include "rows_internal.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr uint32_t kMostThreads = 1024;

// Shared memory: count[warps][E], total[E] (this CTA's slots per expert), start[E] (the experts' offsets), sums[32].
__global__ void __launch_bounds__(kMostThreads) sort_kernel(unsigned* status, uint32_t slots, uint32_t E, const int32_t* __restrict__ ids,
                                                            int32_t* __restrict__ offsets, int32_t* __restrict__ order,
                                                            int32_t* __restrict__ place)
{
    extern __shared__ uint32_t shared[];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ctas = cluster.num_blocks(), cta = cluster.block_rank();
    const uint32_t warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x & 31u;
    uint32_t* count = shared;
    uint32_t* total = count + warps * E;
    uint32_t* start = total + E;
    uint32_t* sums = start + E;
    for (uint32_t i = threadIdx.x; i < warps * E; i += blockDim.x) count[i] = 0;
    rows_begin();
    __syncthreads();

    // the run of this warp: whole groups of 32 slots
    const uint32_t groups = (slots + 31u) / 32u, all_warps = ctas * warps;
    const uint32_t each = (groups + all_warps - 1) / all_warps;
    const uint64_t first = (uint64_t)(cta * warps + warp) * each * 32u;
    const uint32_t begin = (uint32_t)(first < slots ? first : slots);
    const uint32_t end = (uint32_t)(first + (uint64_t)each * 32u < slots ? first + (uint64_t)each * 32u : slots);
    uint32_t* mine = count + warp * E;
    bool bad = false;
    for (uint32_t s = begin + lane; s < end; s += 32) {
        const int32_t e = __ldg(ids + s);
        if ((uint32_t)e < E) atomicAdd(mine + e, 1u);
        else bad |= e != -1;
    }
    if (bad) atomicOr(status, PEARL_ST_BAD_INDEX);
    __syncthreads();

    // per expert: the warps' counts to sums of the warps before, the CTA's total
    for (uint32_t e = threadIdx.x; e < E; e += blockDim.x) {
        uint32_t run = 0;
        for (uint32_t q = 0; q < warps; ++q) {
            const uint32_t c = count[q * E + e];
            count[q * E + e] = run;
            run += c;
        }
        total[e] = run;
    }
    cluster.sync();

    // every CTA: slots per expert over all CTAs, their exclusive sums over the experts, and the CTAs before this one
    const uint32_t per = (E + blockDim.x - 1) / blockDim.x;                   // experts a thread scans (1: E <= 1024 = the threads, or few threads)
    uint32_t here = 0;
    for (uint32_t i = 0; i < per; ++i) {
        const uint32_t e = threadIdx.x * per + i;
        uint32_t before = 0, sum = 0;
        if (e < E)
            for (uint32_t q = 0; q < ctas; ++q) {
                const uint32_t c = *cluster.map_shared_rank(total + e, q);
                if (q < cta) before += c;
                sum += c;
            }
        if (e < E) start[e] = here + before;
        // (the other CTAs read `total` until the barrier below; `sum` of this expert is kept in the running sum)
        here += sum;
    }
    uint32_t scan = here;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, scan, d);
        if (lane >= (uint32_t)d) scan += o;
    }
    if (lane == 31) sums[warp] = scan;
    __syncthreads();
    if (warp == 0) {
        uint32_t v = lane < warps ? sums[lane] : 0u;
        const uint32_t own = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, v, d);
            if (lane >= (uint32_t)d) v += o;
        }
        sums[lane] = v - own;
    }
    __syncthreads();
    const uint32_t base = sums[warp] + scan - here;
    {
        uint32_t run = base;
        for (uint32_t i = 0; i < per; ++i) {
            const uint32_t e = threadIdx.x * per + i;
            if (e >= E) break;
            start[e] += base;
            if (cta == 0) {
                offsets[e] = (int32_t)run;
                uint32_t sum = 0;
                for (uint32_t q = 0; q < ctas; ++q) sum += *cluster.map_shared_rank(total + e, q);
                run += sum;
                if (e + 1 == E) offsets[E] = (int32_t)run;
            }
        }
    }
    cluster.sync();                       // (nobody reads this CTA's memory from here on)

    for (uint32_t s0 = begin; s0 < end; s0 += 32) {
        const uint32_t s = s0 + lane;
        const int32_t e = s < end ? __ldg(ids + s) : -1;
        const bool asks = (uint32_t)e < E;
        const uint32_t peers = __match_any_sync(0xFFFFFFFFu, asks ? (uint32_t)e : 0xFFFFFFFFu);
        const uint32_t rank = __popc(peers & ((1u << lane) - 1u));
        uint32_t at = 0;
        if (asks) at = start[e] + mine[e] + rank;
        __syncwarp();
        if (asks && rank == 0) mine[e] += __popc(peers);
        __syncwarp();
        if (s < end) place[s] = asks ? (int32_t)at : -1;
        if (asks && order != nullptr && ROWS_IN_BOUNDS(status, at < slots)) order[at] = (int32_t)s;
    }
}

}  // namespace

int rows_launch_sort(unsigned* status, uint32_t slots, uint32_t E, const int32_t* ids, int32_t* offsets, int32_t* order,
                     int32_t* place, cudaStream_t s)
{
    // A warp takes at least 2 groups of 32 slots before another is added, a CTA its 32 warps before another one is.
    const uint32_t groups = (slots + 31) / 32;
    uint32_t warps = 4;
    while (warps < 32 && warps * 2 < groups) warps *= 2;
    uint32_t ctas = 1;
    while (ctas < 8 && ctas * warps * 4 < groups) ctas *= 2;
    const size_t smem = ((size_t)warps * E + 2 * E + 32) * sizeof(uint32_t);
    static bool large[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return -1;
    if (smem > 48 * 1024 && (dev >= 64 || !large[dev])) {
        if (cudaFuncSetAttribute(sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (32 * (int)PEARL_ROWS_MAX_EXPERTS + 2 * (int)PEARL_ROWS_MAX_EXPERTS + 32) * 4) != cudaSuccess)
            return -1;
        if (dev < 64) large[dev] = true;
    }
    return rows_launch(sort_kernel, dim3(ctas), dim3(warps * 32), smem, s, ctas, status, slots, E, ids, offsets, order, place);
}
