// Slots sorted by expert: a stable counting sort in one launch.
//
// One thread-block cluster has all the slots, each of its CTAs a run of them, each warp a run of its CTA's.  Counts per expert
// and warp lie in shared memory; the CTAs read each other's sums through it and meet at the cluster's barrier, so nothing goes
// through global memory and no CTA waits for one that may not be there.
//   1. A warp takes its run 32 slots at a time: every lane sets its bit in its expert's word, which then tells the lanes that share
//      it; a slot's rank is the lanes before its own and the warp's count of that expert so far.  It stays in a register (long runs: in
//      the place array).  (One vote a bit of the expert's number, or the warp's match instruction, find the same lanes, and keep the
//      SM's one unit for either busy: 131048 slots of 64 experts took 18 and 20 us with cold caches, and 13.5 this way.)
//   2. The counts become sums over the warps before, and over the CTAs before; the experts' totals become offsets.
//   3. place = offset of the expert + slots of the CTAs before + of the warps before + rank.
#include <cooperative_groups.h>

#include "rows_internal.cuh"

// What bounds it: one cluster's 16 SMs and the barriers between the steps.  131048 slots of 64 experts: 9.7 us beside the 94 of the copy of
// their rows of 4 KB; 512 slots: 3.2.  Beyond 131072 slots ranks go through the place array and `order` is written word by word: 240000
// slots 18.5 us, beside 22 for the copy of rows of 142 bytes; 524288 slots 35.5, beside 13 for rows of 68 bytes.

namespace cg = cooperative_groups;

namespace {

constexpr uint32_t kMostThreads = 1024, kMostCtas = 16;
constexpr int kHeld = 8;                 // groups of 32 slots whose ranks a lane holds

// Shared memory: tally[E][warps + 1] (x: the lanes of the running 32 slots, y: the warp's count so far), total[E] (this CTA's slots per
// expert), start[E], sums[32], and unless kLong local[E] and staged[slots of a CTA]: a CTA's slots are sorted there first, so that what
// goes to `order` is runs of an expert's slots and not single words (a warp's store to 32 places takes the SM 32 cycles).
template <bool kLong>
__global__ void __launch_bounds__(kMostThreads) sort_kernel(unsigned* status, uint32_t slots, uint32_t E, const int32_t* ids,
                                                            int32_t* offsets, int32_t* order, int32_t* place)
{
    extern __shared__ uint32_t shared[];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ctas = cluster.num_blocks(), cta = cluster.block_rank();
    const uint32_t warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x & 31u, below = (1u << lane) - 1u;
    const uint32_t pitch = warps + 1;                                          // (odd: a warp's accesses to its counts of several experts are apart)
    uint2* tally = reinterpret_cast<uint2*>(shared);
    uint32_t* total = shared + 2 * E * pitch;
    uint32_t* start = total + E;
    uint32_t* sums = start + E;
    for (uint32_t i = threadIdx.x; i < E * pitch; i += blockDim.x) tally[i] = make_uint2(0u, 0u);
    rows_begin();
    __syncthreads();

    const uint32_t groups = (slots + 31u) / 32u, all_warps = ctas * warps;
    const uint32_t each = (groups + all_warps - 1) / all_warps;                // groups of a warp's run (<= kHeld unless kLong)
    const uint64_t first = (uint64_t)(cta * warps + warp) * each * 32u;
    const uint32_t begin = (uint32_t)(first < slots ? first : slots);
    const uint32_t end = (uint32_t)(first + (uint64_t)each * 32u < slots ? first + (uint64_t)each * 32u : slots);
    int32_t e[kHeld];
    uint32_t rank[kHeld];
    bool bad = false;
    for (uint32_t s0 = begin; s0 < end; s0 += 32 * kHeld) {
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            const uint32_t s = s0 + q * 32 + lane;
            e[q] = rows_read_if(s < end, ids + s, -1);
        }
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            if (s0 + q * 32 >= end) break;
            bad |= (uint32_t)e[q] >= E && e[q] != -1;
            if ((uint32_t)e[q] >= E) e[q] = -1;
            uint2* mine = tally + (e[q] >= 0 ? (uint32_t)e[q] * pitch + warp : 0u);
            if (e[q] >= 0) atomicOr(&mine->x, 1u << lane);
            __syncwarp();
            uint2 t = make_uint2(0u, 0u);
            if (e[q] >= 0) t = *mine;
            rank[q] = __popc(t.x & below);
            __syncwarp();
            if (e[q] >= 0 && rank[q] == 0) *mine = make_uint2(0u, t.y + __popc(t.x));
            __syncwarp();
            const uint32_t before = t.y;
            rank[q] += before;
            if (kLong) {
                const uint32_t s = s0 + q * 32 + lane;
                if (s < end) place[s] = e[q] >= 0 ? (int32_t)rank[q] : -1;
            }
        }
    }
    if (bad) atomicOr(status, PEARL_ST_BAD_INDEX);
    __syncthreads();

    // per expert: the warps' counts to sums of the warps before, the CTA's total
    for (uint32_t x = warp; x < E; x += warps) {
        const uint32_t own = lane < warps ? tally[x * pitch + lane].y : 0u;
        uint32_t run = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, run, d);
            if (lane >= (uint32_t)d) run += o;
        }
        if (lane < warps) tally[x * pitch + lane].y = run - own;
        if (lane == 31) total[x] = run;
    }
    cluster.sync();

    // every CTA: the experts' totals over all CTAs, their exclusive sums, and the slots of the CTAs before this one
    const uint32_t per = (E + blockDim.x - 1) / blockDim.x;                   // experts a thread has (at most 8: the fewest threads are 128)
    uint32_t here = 0, sum[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t x = threadIdx.x * per + i;
        sum[i] = 0;
        if (i >= per || x >= E) continue;
        uint32_t before = 0, theirs[kMostCtas];
#pragma unroll
        for (uint32_t q = 0; q < kMostCtas; ++q) theirs[q] = q < ctas ? *cluster.map_shared_rank(total + x, q) : 0u;
#pragma unroll
        for (uint32_t q = 0; q < kMostCtas; ++q) {
            if (q < cta) before += theirs[q];
            sum[i] += theirs[q];
        }
        start[x] = here + before;
        here += sum[i];
    }
    uint32_t scan = here;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, scan, d);
        if (lane >= (uint32_t)d) scan += o;
    }
    if (lane == 31) sums[warp] = scan;
    cluster.sync();                       // (nobody reads this CTA's memory from here on)
    const uint32_t base = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? sums[lane] : 0u) + scan - here;
    uint32_t run = base;
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t x = threadIdx.x * per + i;
        if (i >= per || x >= E) continue;
        start[x] += base;
        if (cta == 0) {
            offsets[x] = (int32_t)run;
            run += sum[i];
            if (x + 1 == E) offsets[E] = (int32_t)run;
        }
    }
    __syncthreads();

    if (!kLong && ctas == 1) {
        // (few slots: staging them costs more than it saves; 512 slots and the copy of their rows 4.9 us without, 5.6 with)
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            const uint32_t s = begin + q * 32 + lane;
            if (s >= end) continue;
            const uint32_t at = e[q] >= 0 ? start[e[q]] + tally[(uint32_t)e[q] * pitch + warp].y + rank[q] : 0u;
            if (!ROWS_IN_BOUNDS(status, at < slots)) continue;
            place[s] = e[q] >= 0 ? (int32_t)at : -1;
            if (e[q] >= 0 && order != nullptr) order[at] = (int32_t)s;
        }
        return;
    }
    if (!kLong) {
        // where an expert's slots start among this CTA's: the exclusive sum of the CTA's totals
        uint32_t* local = sums + 32;
        uint32_t* staged = local + E;
        uint32_t own = 0;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t x = threadIdx.x * per + i;
            if (i < per && x < E) own += total[x];
        }
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= (uint32_t)d) upto += o;
        }
        __syncthreads();                                                      // (`sums` has been read)
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
        upto += __reduce_add_sync(0xFFFFFFFFu, lane < warp ? sums[lane] : 0u);
        uint32_t at = upto - own;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t x = threadIdx.x * per + i;
            if (i >= per || x >= E) continue;
            local[x] = at;
            at += total[x];
        }
        __syncthreads();
        const uint64_t cta_first = (uint64_t)cta * warps * each * 32u;
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            const uint32_t s = begin + q * 32 + lane;
            if (s >= end) continue;
            if (e[q] < 0) {
                place[s] = -1;
                continue;
            }
            const uint32_t within = tally[(uint32_t)e[q] * pitch + warp].y + rank[q], to = local[e[q]] + within;
            if (!ROWS_IN_BOUNDS(status, start[e[q]] + within < slots && to < warps * kHeld * 32u)) continue;
            place[s] = (int32_t)(start[e[q]] + within);
            staged[to] = (uint32_t)(s - cta_first) << 10 | (uint32_t)e[q];      // (at most 8192 slots, 1024 experts)
        }
        if (order == nullptr) return;
        __syncthreads();
        const uint32_t n = local[E - 1] + total[E - 1];
        for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
            const uint32_t v = staged[i], x = v & 1023u, to = start[x] + i - local[x];
            if (ROWS_IN_BOUNDS(status, x < E && to < slots && cta_first + (v >> 10) < slots)) order[to] = (int32_t)(cta_first + (v >> 10));
        }
        return;
    }
    for (uint32_t s0 = begin; s0 < end; s0 += 32 * kHeld) {
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            const uint32_t s = s0 + q * 32 + lane;
            rank[q] = s < end ? (uint32_t)place[s] : 0xFFFFFFFFu;
            e[q] = rows_read_if(s < end, ids + s, -1);
            if ((uint32_t)e[q] >= E) e[q] = -1;
        }
#pragma unroll
        for (int q = 0; q < kHeld; ++q) {
            const uint32_t s = s0 + q * 32 + lane;
            if (s >= end || e[q] < 0) continue;
            const uint32_t at = start[e[q]] + tally[(uint32_t)e[q] * pitch + warp].y + rank[q];
            if (!ROWS_IN_BOUNDS(status, at < slots)) continue;
            place[s] = (int32_t)at;
            if (order != nullptr) order[at] = (int32_t)s;
        }
    }
}

}  // namespace

int rows_launch_sort(unsigned* status, uint32_t slots, uint32_t E, const int32_t* ids, int32_t* offsets, int32_t* order,
                     int32_t* place, cudaStream_t s)
{
    // A warp has one group of 32 slots before another warp is added, a CTA's 32 warps two each before another CTA is.
    const uint32_t groups = (slots + 31) / 32, most_warps = E > 512 ? 16 : 32;              // (the tallies of 1024 experts and 16 warps are 139 KB)
    uint32_t warps = 4;
    while (warps < most_warps && warps < groups) warps *= 2;
    uint32_t ctas = 1;
    while (ctas < kMostCtas && ctas * warps * 2 < groups) ctas *= 2;
    const bool is_long = groups > ctas * warps * kHeld;
    const size_t smem = ((size_t)E * (2 * (warps + 1) + 2) + 32 + (is_long ? 0 : E + warps * kHeld * 32)) * sizeof(uint32_t);
    const auto kernel = is_long ? sort_kernel<true> : sort_kernel<false>;
    if ((smem > 48 * 1024 || ctas > 8) && !rows_large_cluster(kernel, 208 * 1024)) return -1;
    return rows_launch(kernel, dim3(ctas), dim3(warps * 32), smem, s, ctas, status, slots, E,
                       ids, offsets, order, place);
}
