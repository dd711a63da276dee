// One step of a beam search: the choice over the beams and the vocabulary, and the move of the beams' states.
#include <cooperative_groups.h>

#include "rows_internal.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.402823466e+38f;
constexpr uint32_t kMostParts = 16;
constexpr float kLog2e = 1.44269504f;

// ---- selection -------------------------------------------------------------------------------------------------------
// One thread-block cluster has a group.  A unit of work is a run of one beam's logits (the whole row, or a part of it where the
// cluster has more CTAs than the group has beams).  A unit is read once:
//   statistics   a thread keeps a reference value, the sum of exp(x - reference) and its largest logit.  The reference
//                follows the largest logit only when that is more than 8 above it (e^8 terms fit a binary32 sum easily), so a
//                logit costs one subtraction, one product, one exponential, one addition and one comparison;
//   the best C   the threads form kTeams teams.  The C-th largest of the teams' largest logits is a bound that at least C logits
//                reach, and only logits of the (at most C) teams whose largest reaches it can do so: those teams' logits -- a few
//                per cent of the unit, still in L2 -- are read again and the ones that reach the bound are sorted.
// Offers carry (logit, token) as one 64-bit key, all different, so nothing depends on the order threads arrive in.
// The CTAs then exchange row sums and sorted lists through each other's shared memory, and the rank of an offer among the
// group's is the sum over the lists of how many entries precede it: binary searches, one writer for each result.
constexpr uint32_t kThreads = 256;
constexpr uint32_t kTeams = 128;                 // >= PEARL_ROWS_MAX_BEST
constexpr uint32_t kPerTeam = kThreads / kTeams;
constexpr uint32_t kRoom = 2048;                 // offers that are sorted
constexpr uint32_t kUnroll = 4;                  // accesses a thread has in flight

// Keys that order like (larger logit, lower token); 0 stands for no offer.
__device__ __forceinline__ uint32_t rising(float x)
{
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.0f));            // (-0 becomes 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_rising(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r); }
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token)
{
    return x == -kInf ? 0ull : ((uint64_t)rising(x) << 32) | (0xFFFFFFFFu - token);
}
__device__ __forceinline__ uint64_t rising64(double x)
{
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double from_rising64(uint64_t r)
{
    return __longlong_as_double((long long)(r >> 63 ? r ^ 0x8000000000000000ull : ~r));
}

// Access v (N elements from element v*N of the run on) of a run of n elements at `run`, whose address is `off` bytes past a
// 16-byte boundary: one 16-byte load where that is 0, else the two that hold it, shifted together.  The accesses are counted from
// the run's start, not from the boundary: what a thread adds up does not depend on where the row lies in memory.  The last
// access, and the first of a shifted run, go element by element so that nothing outside the run is read.
template <typename E>
struct Run {
    static constexpr int N = 16 / (int)sizeof(E);
    const E* run;
    uint32_t n, off, accesses;
    __device__ __forceinline__ void load(uint32_t v, float (&x)[N]) const
    {
        const uint64_t at = (uint64_t)v * 16u;
        if (off == 0 ? at + 16u <= (uint64_t)n * sizeof(E) : (v > 0 && at + 32u - off <= (uint64_t)n * sizeof(E))) {
            uint32_t q[8];
            const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const unsigned char*>(run) + at - off);
            const uint4 a = __ldg(p);
            q[0] = a.x; q[1] = a.y; q[2] = a.z; q[3] = a.w;
            if (off) {
                const uint4 b = __ldg(p + 1);
                q[4] = b.x; q[5] = b.y; q[6] = b.z; q[7] = b.w;
                if (off & 8u) {
#pragma unroll
                    for (int i = 0; i < 6; ++i) q[i] = q[i + 2];
                }
                if (off & 4u) {
#pragma unroll
                    for (int i = 0; i < 5; ++i) q[i] = q[i + 1];
                }
                if (sizeof(E) == 2 && (off & 2u)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[i] = __funnelshift_r(q[i], q[i + 1], 16);
                }
            }
            const E* e = reinterpret_cast<const E*>(q);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = RowsElem<E>::up(e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = (uint64_t)v * N + i < n ? RowsElem<E>::up(run[(uint64_t)v * N + i]) : -kInf;
        }
    }
};

template <int N> __device__ __forceinline__ bool clean(float (&x)[N])
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (!(x[i] < kInf)) { bad = true; x[i] = -kInf; }
    return bad;
}

struct Stats {
    double sum;          // of exp(x - ref)
    float ref, best;     // best: the largest logit, first seen in access best_at
    uint32_t best_at;
    bool bad;
};
template <int N> __device__ __forceinline__ void take(Stats& s, float (&x)[N], uint32_t v)
{
#pragma unroll 1
    for (int again = 0; again < 2; ++again) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
        if (top < kInf) {
            if (top > __fadd_rn(s.ref, 8.0f)) {
                s.sum *= (double)exp2f(__fmul_rn(__fsub_rn(s.ref, top), kLog2e));
                s.ref = top;
            }
            float e[N];
#pragma unroll
            for (int i = 0; i < N; ++i) e[i] = exp2f(__fmul_rn(__fsub_rn(x[i], s.ref), kLog2e));
#pragma unroll
            for (int d = N / 2; d > 0; d >>= 1)
#pragma unroll
                for (int i = 0; i < d; ++i) e[i] = __fadd_rn(e[i], e[i + d]);
            if (e[0] < kInf) {                       // (a NaN among the logits makes this one)
                s.sum += (double)e[0];
                if (top > s.best) { s.best = top; s.best_at = v; }
                return;
            }
        }
        s.bad |= clean<N>(x);
    }
}

// What the CTAs of a cluster leave for one another, one entry per unit of the CTA.
struct UnitSum {
    double sum;
    float ref;
    uint32_t offers;
};

// The sorted list's place of `key` (entries that precede it): the list falls.
__device__ __forceinline__ uint32_t preceding(const uint64_t* list, uint32_t n, uint64_t key, bool equal_precedes)
{
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (list[mid] > key || (equal_precedes && list[mid] == key)) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

struct SelectArgs {
    unsigned* status;
    uint32_t W, V, C;
    uint32_t parts;             // runs a row is cut into
    uint32_t run;               // elements of a run (a multiple of 8)
    uint32_t units_per_cta;
    const void* logits;
    uint64_t ld;
    const float* scores;
    const uint8_t* done;
    int32_t end_token;
    float* best_score;
    int32_t* best_beam;
    int32_t* best_token;
};

// Dynamic shared memory: keys[units_per_cta][C] and sums[units_per_cta] (this CTA's, read by the others), then the workspace:
// kRoom offers, later all_totals[units][C], all_keys[units][C].
template <typename E>
__global__ void __launch_bounds__(kThreads) select_kernel(const SelectArgs a)
{
    extern __shared__ __align__(16) unsigned char shared[];
    __shared__ uint64_t team_best[kTeams];
    __shared__ uint32_t picked[kTeams];
    __shared__ uint32_t n_picked, n_offers;
    __shared__ uint64_t bound;
    __shared__ double warp_sum[kThreads / 32];
    __shared__ float warp_ref[kThreads / 32];
    constexpr int N = Run<E>::N;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ctas = cluster.num_blocks(), cta = cluster.block_rank(), g = blockIdx.x / ctas;
    const uint32_t units = a.W * a.parts, C = a.C, tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    uint64_t* keys = reinterpret_cast<uint64_t*>(shared);
    UnitSum* sums = reinterpret_cast<UnitSum*>(keys + a.units_per_cta * C);
    uint64_t* work = reinterpret_cast<uint64_t*>(sums + a.units_per_cta);
    rows_begin();

    for (uint32_t q = 0; q < a.units_per_cta; ++q) {
        const uint32_t u = cta * a.units_per_cta + q;
        uint64_t* mine = keys + q * C;
        if (u >= units) break;
        const uint32_t b = u / a.parts, part = u % a.parts;
        const uint64_t row = (uint64_t)g * a.W + b;
        float score = a.scores[row];
        if (!(score < kInf)) {
            if (tid == 0 && part == 0) atomicOr(a.status, PEARL_ST_BAD_SCORE);
            score = -kInf;
        }
        const bool done = a.done != nullptr && a.done[row] != 0;
        const uint64_t first = (uint64_t)part * a.run;
        if (score == -kInf || done || first >= a.V) {
            // no logits are read; a finished beam has one offer, whose key only has to be valid
            const uint32_t n = done && score > -kInf && part == 0 ? 1u : 0u;
            for (uint32_t i = tid; i < C; i += kThreads) mine[i] = i < n ? key_of(0.0f, 0u) : 0ull;
            if (tid == 0) sums[q] = UnitSum{0.0, kLowest, n};
            continue;
        }
        Run<E> r;
        r.run = reinterpret_cast<const E*>(a.logits) + row * a.ld + first;
        r.n = (uint32_t)(a.V - first < a.run ? a.V - first : a.run);
        r.off = (uint32_t)((uintptr_t)r.run & 15u);
        r.accesses = (r.n + N - 1) / N;

        Stats s{0.0, kLowest, -kInf, 0u, false};
        uint32_t v = tid;
        for (; v + (kUnroll - 1) * kThreads < r.accesses; v += kUnroll * kThreads) {
            float x[kUnroll][N];
#pragma unroll
            for (int i = 0; i < (int)kUnroll; ++i) r.load(v + i * kThreads, x[i]);
#pragma unroll
            for (int i = 0; i < (int)kUnroll; ++i) take<N>(s, x[i], v + i * kThreads);
        }
        for (; v < r.accesses; v += kThreads) {
            float x[N];
            r.load(v, x);
            take<N>(s, x, v);
        }
        if (s.bad) atomicOr(a.status, PEARL_ST_BAD_SCORE);

        // the unit's sum: relative to the largest reference, added in a fixed order
        float ref = s.ref;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xFFFFFFFFu, ref, d));
        if (lane == 0) warp_ref[warp] = ref;
        // a team's largest logit, as the smallest key that a logit of its access can have
        uint64_t key = s.best == -kInf ? 0ull : key_of(s.best, (uint32_t)first + s.best_at * N + N - 1);
#pragma unroll
        for (uint32_t d = 1; d < kPerTeam; d <<= 1) {
            const uint64_t o = __shfl_xor_sync(0xFFFFFFFFu, key, d);
            key = o > key ? o : key;
        }
        if (tid % kPerTeam == 0) team_best[tid / kPerTeam] = key;
        if (tid == 0) { n_picked = 0; n_offers = 0; bound = 1ull; }
        __syncthreads();
        ref = warp_ref[0];
#pragma unroll
        for (uint32_t i = 1; i < kThreads / 32; ++i) ref = fmaxf(ref, warp_ref[i]);
        double sum = s.sum > 0.0 ? s.sum * exp((double)s.ref - (double)ref) : 0.0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (lane == 0) warp_sum[warp] = sum;
        // the C-th largest of the teams' keys (teams without a logit have none: the bound stays at the lowest key)
        if (tid < kTeams) {
            const uint64_t k = team_best[tid];
            uint32_t ahead = 0;
            for (uint32_t i = 0; i < kTeams; ++i) ahead += team_best[i] > k || (team_best[i] == k && i < tid);
            if (ahead == C - 1 && k) bound = k;
        }
        __syncthreads();
        if (tid < kTeams && team_best[tid] && (team_best[tid] | (uint64_t)(N - 1)) >= bound) picked[atomicAdd(&n_picked, 1u)] = tid;
        __syncthreads();

        // the picked teams' logits that reach the bound.  Should they be more than there is room for, the bound is searched by
        // halving (`low`: too many reach it, `high`: fewer than C do; the keys are all different, so some key has a number between).
        const uint32_t rounds = (r.accesses + kThreads - 1) / kThreads;
        const uint64_t lowest = bound;
        uint64_t low = lowest, high = ~0ull, at_least = lowest;
        for (;;) {
            for (uint32_t p = warp; p < n_picked; p += kThreads / 32) {
                for (uint32_t i = lane; i < rounds * kPerTeam; i += 32) {
                    const uint32_t at = picked[p] * kPerTeam + i % kPerTeam + i / kPerTeam * kThreads;
                    if (at >= r.accesses) continue;
                    float x[N];
                    r.load(at, x);
                    clean<N>(x);
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const uint64_t k = key_of(x[j], (uint32_t)first + at * N + j);
                        if (k >= at_least) {
                            const uint32_t to = atomicAdd(&n_offers, 1u);
                            if (to < kRoom) work[to] = k;
                        }
                    }
                }
            }
            __syncthreads();
            const uint32_t n = n_offers;
            if (n <= kRoom && (n >= C || at_least == lowest)) break;
            if (n > kRoom) low = at_least;
            else high = at_least;
            at_least = low + (high - low) / 2;
            __syncthreads();
            if (tid == 0) n_offers = 0;
            __syncthreads();
        }
        const uint32_t n = n_offers;
        for (uint32_t i = tid; i < C; i += kThreads)
            if (i >= n) mine[i] = 0ull;
        if (n <= kThreads) {
            if (tid < n) {
                const uint64_t k = work[tid];
                uint32_t ahead = 0;
                for (uint32_t i = 0; i < n; ++i) ahead += work[i] > k;
                if (ahead < C) mine[ahead] = k;
            }
        } else {
            uint32_t size = kThreads;
            while (size < n) size *= 2;
            for (uint32_t i = n + tid; i < size; i += kThreads) work[i] = 0ull;
            for (uint32_t span = 2; span <= size; span *= 2)
                for (uint32_t step = span / 2; step > 0; step /= 2) {
                    __syncthreads();
                    for (uint32_t i = tid; i < size / 2; i += kThreads) {
                        const uint32_t x = i / step * step * 2 + i % step, y = x + step;
                        const uint64_t p = work[x], o = work[y];
                        if ((p < o) == ((x & span) == 0)) { work[x] = o; work[y] = p; }
                    }
                }
            __syncthreads();
            for (uint32_t i = tid; i < C; i += kThreads) mine[i] = work[i];
        }
        if (tid == 0) {
            double total = 0.0;
            for (uint32_t i = 0; i < kThreads / 32; ++i) total += warp_sum[i];
            sums[q] = UnitSum{total, ref, n < C ? n : C};
        }
        __syncthreads();                  // (the next unit uses the same workspace)
    }
    cluster.sync();

    // every CTA: the group's row sums and lists, copied from where they are
    __shared__ double lse[PEARL_ROWS_MAX_BEAMS];
    __shared__ uint32_t n_all;
    uint64_t* all_keys = work;
    uint64_t* all_totals = work + units * C;
    if (tid == 0) n_all = 0;
    __syncthreads();
    if (tid < a.W) {
        UnitSum part[kMostParts];
        float ref = kLowest;
        uint32_t offers = 0;
        for (uint32_t i = 0; i < a.parts; ++i) {
            const uint32_t u = tid * a.parts + i;
            part[i] = *cluster.map_shared_rank(sums + u % a.units_per_cta, u / a.units_per_cta);
            ref = fmaxf(ref, part[i].ref);
            offers += part[i].offers;
        }
        double sum = 0.0;
        for (uint32_t i = 0; i < a.parts; ++i)
            if (part[i].sum > 0.0) sum += part[i].sum * exp((double)part[i].ref - (double)ref);
        lse[tid] = (double)ref + log(sum);
        atomicAdd(&n_all, offers);
    }
    for (uint32_t i = tid; i < units * C; i += kThreads) {
        const uint32_t u = i / C;
        all_keys[i] = cluster.map_shared_rank(keys + u % a.units_per_cta * C, u / a.units_per_cta)[i % C];
    }
    cluster.sync();                       // (nobody reads this CTA's memory from here on)
    for (uint32_t i = tid; i < units * C; i += kThreads) {
        const uint32_t b = i / C / a.parts;
        const uint64_t row = (uint64_t)g * a.W + b, k = all_keys[i];
        const double score = (double)a.scores[row];
        const bool done = a.done != nullptr && a.done[row] != 0;
        all_totals[i] = k == 0 ? 0ull : rising64(done ? score : score + ((double)from_rising((uint32_t)(k >> 32)) - lse[b]));
    }
    __syncthreads();

    // the place of each offer of this CTA's units: kLanes lanes share the lists that may hold offers before it
    constexpr uint32_t kLanes = 8;
    const uint32_t own = a.units_per_cta * C;
    for (uint32_t i0 = 0; i0 < own; i0 += kThreads / kLanes) {
        const uint32_t i = i0 + tid / kLanes;
        const uint32_t u = cta * a.units_per_cta + i / C;
        const bool there = i < own && u < units && all_keys[u * C + i % C] != 0;
        const uint32_t b = u / a.parts;
        uint32_t place = 0;
        uint64_t key = 0, total = 0;
        if (there) {
            key = all_keys[u * C + i % C];
            total = all_totals[u * C + i % C];
            for (uint32_t o = tid % kLanes; o < units; o += kLanes) {
                if (o / a.parts == b) place += preceding(all_keys + o * C, C, key, false);
                else place += preceding(all_totals + o * C, C, total, o < u);
            }
        }
#pragma unroll
        for (uint32_t d = 1; d < kLanes; d <<= 1) place += __shfl_xor_sync(0xFFFFFFFFu, place, d);
        if (there && tid % kLanes == 0 && place < C) {
            const uint64_t row = (uint64_t)g * a.W + b, to = (uint64_t)g * C + place;
            const bool done = a.done != nullptr && a.done[row] != 0;
            a.best_score[to] = (float)from_rising64(total);
            a.best_beam[to] = (int32_t)b;
            a.best_token[to] = done ? a.end_token : (int32_t)(0xFFFFFFFFu - (uint32_t)key);
        }
    }
    if (cta == 0)
        for (uint32_t i = tid; i < C; i += kThreads)
            if (i >= n_all) {
                const uint64_t to = (uint64_t)g * C + i;
                a.best_score[to] = -kInf;
                a.best_beam[to] = -1;
                a.best_token[to] = -1;
            }
}

// ---- the states ------------------------------------------------------------------------------------------------------
// state[o, g, i] <- state[o, g, parent[g, i]].  A thread has one access's worth of all W states of a block and group: it reads
// what the moved states need (a state with several children comes from L1 the second time), then writes.  No other thread
// touches those bytes, so the move can be made in place.
struct ReorderArgs {
    unsigned* status;
    uint32_t G, W;
    uint64_t cols;              // accesses of a state
    uint64_t piece_cols;        // ... of a piece
    uint64_t col_blocks;
    const int32_t* parent;
    const unsigned char* src;
    unsigned char* dst;
    pearl_states_t sp, dp;
    bool in_place;
};
constexpr uint32_t kMoveThreads = 256;

template <int B, int M>
__global__ void __launch_bounds__(kMoveThreads) reorder_kernel(const ReorderArgs a)
{
    rows_begin();
    const uint64_t og = blockIdx.x / a.col_blocks;
    const uint32_t g = (uint32_t)(og % a.G);
    const uint64_t o = og / a.G;
    const uint64_t col = (blockIdx.x - og * a.col_blocks) * kMoveThreads + threadIdx.x;
    if (col >= a.cols) return;
    uint64_t piece = 0, in = col;
    if (a.piece_cols < a.cols) {
        if (a.cols >> 32) piece = col / a.piece_cols;
        else piece = (uint32_t)col / (uint32_t)a.piece_cols;
        in = col - piece * a.piece_cols;
    }
    const unsigned char* src = a.src + o * a.sp.block_pitch + (uint64_t)g * a.W * a.sp.state_pitch + piece * a.sp.piece_pitch + in * B;
    unsigned char* dst = a.dst + o * a.dp.block_pitch + (uint64_t)g * a.W * a.dp.state_pitch + piece * a.dp.piece_pitch + in * B;
    RowsRaw<B> v[M];
    int32_t from[M];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < M; ++i) from[i] = (uint32_t)i < a.W ? __ldg(a.parent + (uint64_t)g * a.W + i) : -1;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        bad |= from[i] < -1 || from[i] >= (int32_t)a.W;
        if ((uint32_t)from[i] >= a.W || (a.in_place && from[i] == i)) from[i] = -1;
        rows_load_if<true>(from[i] >= 0, v[i], src + (uint64_t)(uint32_t)from[i] * a.sp.state_pitch);
    }
#pragma unroll
    for (int i = 0; i < M; ++i)
        if (from[i] >= 0) rows_store(dst + (uint64_t)i * a.dp.state_pitch, v[i]);
    if (bad && col == 0) atomicOr(a.status, PEARL_ST_BAD_INDEX);
}

template <int B>
int launch_reorder(const ReorderArgs& a, dim3 grid, cudaStream_t s)
{
    if (a.W <= 4) return rows_launch(reorder_kernel<B, 4>, grid, dim3(kMoveThreads), 0, s, 0, a);
    if (a.W <= 8) return rows_launch(reorder_kernel<B, 8>, grid, dim3(kMoveThreads), 0, s, 0, a);
    if (a.W <= 16) return rows_launch(reorder_kernel<B, 16>, grid, dim3(kMoveThreads), 0, s, 0, a);
    return rows_launch(reorder_kernel<B, 32>, grid, dim3(kMoveThreads), 0, s, 0, a);
}

}  // namespace

int rows_launch_beam_select(unsigned* status, uint32_t G, uint32_t W, uint32_t V, uint32_t C, uint32_t dtype, const void* logits,
                            uint64_t ld, const float* scores, const uint8_t* done, int32_t end_token, float* best_score,
                            int32_t* best_beam, int32_t* best_token, cudaStream_t s)
{
    if (G == 0) return 0;
    // Rows are cut into parts where there are too few of them to occupy the GPU; a part has 2048 logits at least.
    SelectArgs a;
    const uint32_t most = 8;
    a.units_per_cta = (W + most - 1) / most;
    a.parts = 1;
    while ((a.parts + 1) * W <= most && (uint64_t)G * W * a.parts < 592 && V / (a.parts + 1) >= 2048) ++a.parts;
    a.run = ((V + a.parts - 1) / a.parts + 7) / 8 * 8;
    const uint32_t units = W * a.parts, ctas = (units + a.units_per_cta - 1) / a.units_per_cta;
    if ((uint64_t)G * ctas > 0x7FFFFFFFull) return -1;
    a.status = status; a.W = W; a.V = V; a.C = C; a.logits = logits; a.ld = ld; a.scores = scores; a.done = done; a.end_token = end_token;
    a.best_score = best_score; a.best_beam = best_beam; a.best_token = best_token;
    const size_t lists = (size_t)units * C * 16, offers = kRoom * 8;
    const size_t smem = a.units_per_cta * (C * 8 + sizeof(UnitSum)) + (lists > offers ? lists : offers);
    int rc = -1;
#define ROWS_GO(E) rc = rows_launch(select_kernel<E>, dim3(G * ctas), dim3(kThreads), smem, s, ctas, a)
    ROWS_WITH_TYPE(dtype, ROWS_GO);
#undef ROWS_GO
    return rc;
}

int rows_launch_beam_reorder(unsigned* status, uint32_t blocks, uint32_t G, uint32_t W, uint32_t pieces, uint64_t piece_bytes,
                             const int32_t* parent, const void* src, const pearl_states_t& sp, void* dst, const pearl_states_t& dp,
                             cudaStream_t s)
{
    if (blocks == 0 || G == 0 || pieces == 0 || piece_bytes == 0) return 0;
    ReorderArgs a;
    a.status = status; a.G = G; a.W = W; a.parent = parent; a.src = (const unsigned char*)src; a.dst = (unsigned char*)dst;
    a.sp = sp; a.dp = dp;
    a.in_place = src == dst;
    if (pieces > 1 && sp.piece_pitch == piece_bytes && dp.piece_pitch == piece_bytes) { piece_bytes *= pieces; pieces = 1; }
    uint64_t all = piece_bytes | (uintptr_t)src | (uintptr_t)dst | sp.state_pitch | dp.state_pitch;
    if (pieces > 1) all |= sp.piece_pitch | dp.piece_pitch;
    if (blocks > 1) all |= sp.block_pitch | dp.block_pitch;
    uint32_t g = rows_granule(all);
    if (g == 32 && W > 16) g = 16;          // (32 states of 32 bytes are more than a thread's registers)
    a.piece_cols = piece_bytes / g;
    a.cols = a.piece_cols * pieces;
    a.col_blocks = (a.cols + kMoveThreads - 1) / kMoveThreads;
    const uint64_t og = (uint64_t)blocks * G;
    if (a.col_blocks > 0x7FFFFFFFull / og) return -1;
    const dim3 grid((uint32_t)(a.col_blocks * og));
    switch (g) {
    case 32: return launch_reorder<32>(a, grid, s);
    case 16: return launch_reorder<16>(a, grid, s);
    case 8: return launch_reorder<8>(a, grid, s);
    case 4: return launch_reorder<4>(a, grid, s);
    case 2: return launch_reorder<2>(a, grid, s);
    default: return launch_reorder<1>(a, grid, s);
    }
}
