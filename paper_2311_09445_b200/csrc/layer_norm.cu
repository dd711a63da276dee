// The layer norm of rows and its gradient.
//
// Both are bound by memory: a row is read once, and everything in between is in registers.  What has to be kept small is the number of
// instructions an element (16-bit rows bring 14 elements a cycle to an SM) and what a row costs whatever its length, a sum over its
// threads: so arithmetic is on pairs, a thread has up to 32 elements of a row, and a row that a warp can hold has one warp.  Both kernels wait for
// the steps of these sums more than for memory: issue slots are 42 % used.
//
// Rows may start anywhere.  A thread has whole 16-byte words of memory, which may begin before its row does: with `off` elements of a row's first
// word before the row, word w holds the row's elements w N - off .. w N - off + N - 1.
#include "layer_internal.cuh"

namespace {

template <typename E> constexpr int kN = 16 / (int)sizeof(E);            // elements of a word
template <typename E> constexpr int kTwos = kN<E> / 2;

template <typename E> using Word = RowsVec<E, kN<E>>;
template <typename E> using Twos = LayerTwo[kTwos<E>];

// Elements before `p` in its word.
template <typename E> __host__ __device__ __forceinline__ uint32_t before(const E* p) { return ((uint32_t)(uintptr_t)p & 15u) / (uint32_t)sizeof(E); }

// Elements [lo, hi) of the word at p; zeros for the others.  Where rows start with a word and end with one (not kBroken), a word has all of them.
template <typename E, bool kBroken> __device__ __forceinline__ Word<E> load_word(const E* p, int lo, int hi)
{
    Word<E> v;
    v.clear();
    if (!kBroken || (lo <= 0 && hi >= kN<E>)) {
        rows_load_if<false>(true, v.raw, p);
    } else {
#pragma unroll
        for (int i = 0; i < kN<E>; ++i) {
            if (i < lo || i >= hi) continue;
            if constexpr (sizeof(E) == 4) v.word[i] = reinterpret_cast<const uint32_t*>(p)[i];
            else v.word[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << (i % 2 * 16);
        }
    }
    return v;
}
template <typename E, bool kBroken> __device__ __forceinline__ void store_word(E* p, const Word<E>& v, int lo, int hi)
{
    if (!kBroken || (lo <= 0 && hi >= kN<E>)) {
        rows_store(p, v.raw);
    } else {
#pragma unroll
        for (int i = 0; i < kN<E>; ++i) {
            if (i < lo || i >= hi) continue;
            if constexpr (sizeof(E) == 4) reinterpret_cast<uint32_t*>(p)[i] = v.word[i];
            else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(v.word[i / 2] >> (i % 2 * 16));
        }
    }
}
// Zeros outside [lo, hi).
template <typename E, bool kBroken> __device__ __forceinline__ void keep(Twos<E>& t, int lo, int hi)
{
    if constexpr (!kBroken) return;
    // (a vote, so that a warp without such a word jumps over this)
    if (!__any_sync(__activemask(), lo > 0 || hi < kN<E>)) return;
#pragma unroll
    for (int q = 0; q < kTwos<E>; ++q) {
        const float2 f = t[q].get();
        t[q] = LayerTwo(2 * q >= lo && 2 * q < hi ? f.x : 0.0f, 2 * q + 1 >= lo && 2 * q + 1 < hi ? f.y : 0.0f);
    }
}

// The bits of a word's elements [lo, hi).
template <typename E> __device__ __forceinline__ void bits_of(uint32_t (&mask)[4], int lo, int hi)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mask[i] = 0u;
#pragma unroll
        for (int k = 0; k < 4 / (int)sizeof(E); ++k) {
            const int e = i * (4 / (int)sizeof(E)) + k;
            if (e >= lo && e < hi) mask[i] |= sizeof(E) == 4 ? 0xFFFFFFFFu : 0xFFFFu << (k * 16);
        }
    }
}
template <typename E> __device__ __forceinline__ void mask_word(Word<E>& v, const uint32_t (&mask)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v.word[i] &= mask[i];
}

// ---- parameters in shared memory, as binary32 -----------------------------------------------------------------------------
// One behind the other where rows are whole words; else (kBroken) those of equal remainder by a word's elements, so that a warp's lanes, whose
// words are neighbours, find theirs in neighbouring places whatever `off` is.
template <typename E> __host__ __device__ constexpr uint32_t params_room(uint32_t D) { return (D / kN<E> + 3) * kN<E>; }
template <typename E, typename P, bool kBroken> __device__ __forceinline__ void bring_params(float* to, const void* from, uint32_t D, float otherwise)
{
    const uint32_t line = D / kN<E> + 3;
    if (kBroken)                            // (0 beside them: that of a word's elements which are not the row's)
        for (uint32_t e = threadIdx.x; e < kN<E>; e += blockDim.x) to[e * line] = to[e * line + (D + kN<E> - 1 - e) / kN<E> + 1] = 0.0f;
#pragma unroll 4
    for (uint32_t e = threadIdx.x; e < D; e += blockDim.x) {
        const float v = from ? RowsElem<P>::up(((const P*)from)[e]) : otherwise;
        to[kBroken ? e % kN<E> * line + e / kN<E> + 1 : e] = v;
    }
}
// Those of word w (any numbers for elements that the row does not have).
template <typename E, bool kBroken> __device__ __forceinline__ void read_params(unsigned* status, Twos<E>& p, const float* from, uint32_t w, uint32_t off, uint32_t D)
{
    if (!ROWS_IN_BOUNDS(status, kBroken ? w <= D / kN<E> + 1 : (w + 1) * kN<E> <= D)) w = 0;
    if constexpr (kBroken) {
        const uint32_t line = D / kN<E> + 3;
        float f[kN<E>];
#pragma unroll
        for (uint32_t i = 0; i < kN<E>; ++i) f[i] = from[((i - off) & (kN<E> - 1)) * line + w + (i < off ? 0 : 1)];
#pragma unroll
        for (int q = 0; q < kTwos<E>; ++q) p[q] = LayerTwo(f[2 * q], f[2 * q + 1]);
    } else {
#pragma unroll
        for (int q = 0; q < kTwos<E>; q += 2) {
            const float4 v = *reinterpret_cast<const float4*>(from + w * kN<E> + 2 * q);
            p[q] = LayerTwo(v.x, v.y);
            p[q + 1] = LayerTwo(v.z, v.w);
        }
    }
}

// ---- sums over a team -----------------------------------------------------------------------------------------------------
// A block's threads are in teams of whole warps; a team has a row.  sums: M lines of 32, one a warp of the block; two calls in a row use different
// ones.  The order of a sum depends on the team's size alone.
template <int M> __device__ __forceinline__ void team_sums(uint32_t threads, uint32_t team, float (&a)[M], float (*sums)[32])
{
    const uint32_t lane = threadIdx.x & 31u, warps = threads / 32;
#pragma unroll
    for (int m = 0; m < M; ++m) a[m] = layer_warp_sum(a[m]);
    if (warps == 1) return;
    if (lane == 0) {
#pragma unroll
        for (int m = 0; m < M; ++m) sums[m][threadIdx.x >> 5] = a[m];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(threads) : "memory");
#pragma unroll
    for (int m = 0; m < M; ++m) a[m] = layer_warp_sum(lane < warps ? sums[m][team * warps + lane] : 0.0f);
}

// ---- forward --------------------------------------------------------------------------------------------------------------
// A team goes over every so many rows; the next row's words are on their way while it forms the mean, then the mean of the squared differences,
// then the results of this one.  16381 rows of 2048 bfloat16 elements 35 us (3.9 TB/s; 465 instructions a warp and row, of which some 200 are there for any
// length), 8192 of binary32 27 (5.0 TB/s).  A block a row took 44, with four words a thread and no row ahead 34.  Words that rows
// break cost more registers than there are: four a thread spill 108 bytes (8000 rows of 2047 bfloat16 elements 34 us).
template <int NV> constexpr uint32_t kThreads = NV == 4 ? 768 : 1024;           // of a block: what the registers have room for
template <typename E, typename P, int NV, bool kBroken>
__global__ void __launch_bounds__(kThreads<NV>, 1) norm_kernel(unsigned* status, uint32_t T, uint32_t D, uint32_t threads, const E* x, uint64_t ld_x,
                                                           const void* gamma, const void* beta, float eps, E* y, uint64_t ld_y, float* mean_out, float* rstd_out)
{
    extern __shared__ __align__(16) float params[];
    __shared__ float sums[2][1][32];
    const uint32_t team = threadIdx.x / threads, me = threadIdx.x - team * threads;
    const uint64_t step = (uint64_t)gridDim.x * (blockDim.x / threads);
    rows_begin();
    float* bias = params + params_room<E>(D);
    uint64_t t = (uint64_t)blockIdx.x * (blockDim.x / threads) + team;
    Word<E> next[NV];
    const auto fetch = [&](uint64_t row) {
        const E* p = x + row * ld_x;
        const uint32_t off = kBroken ? before(p) : 0u;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (int)((j * threads + me) * kN<E>) - (int)off;
            if (row < T && e < (int)D && layer_in_rows<kN<E>>(status, p + e, -e, (int)D - e, x, layer_end(x, T, D, ld_x)))
                next[j] = load_word<E, kBroken>(p + e, -e, (int)D - e);
            else next[j].clear();
        }
    };
    fetch(t);
    bring_params<E, P, kBroken>(params, gamma, D, 1.0f);
    if (beta) bring_params<E, P, kBroken>(bias, beta, D, 0.0f);
    __syncthreads();
    const float part = 1.0f / (float)D;
    for (; t < T; t += step) {
        const uint32_t off = kBroken ? before(x + t * ld_x) : 0u;
        Twos<E> v[NV];
        LayerTwo all(0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            layer_twos<E, kN<E>>(v[j], next[j]);
#pragma unroll
            for (int q = 0; q < kTwos<E>; ++q) all = all + v[j][q];
        }
        fetch(t + step);
        float s[1] = { all.sum() };
        team_sums<1>(threads, team, s, sums[0]);
        const float mean = s[0] / (float)D;          // (times 1 / D it would be off by a unit of the last place, which a row that hardly differs from it shows)
        all = LayerTwo(0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (int)((j * threads + me) * kN<E>) - (int)off;
            if (e >= (int)D) break;
#pragma unroll
            for (int q = 0; q < kTwos<E>; ++q) v[j][q] = v[j][q] + LayerTwo(-mean);
            keep<E, kBroken>(v[j], -e, (int)D - e);
#pragma unroll
            for (int q = 0; q < kTwos<E>; ++q) all = layer_fma(v[j][q], v[j][q], all);
        }
        s[0] = all.sum();
        team_sums<1>(threads, team, s, sums[1]);
        const float rstd = 1.0f / sqrtf(__fmaf_rn(s[0], part, eps));
        if (me == 0) {
            if (mean_out) mean_out[t] = mean;
            if (rstd_out) rstd_out[t] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t w = j * threads + me;
            const int e = (int)(w * kN<E>) - (int)off;
            if (e >= (int)D) break;
            Twos<E> g, out;
            read_params<E, kBroken>(status, g, params, w, off, D);
#pragma unroll
            for (int q = 0; q < kTwos<E>; ++q) out[q] = g[q] * LayerTwo(rstd);
            if (beta) {
                read_params<E, kBroken>(status, g, bias, w, off, D);
#pragma unroll
                for (int q = 0; q < kTwos<E>; ++q) out[q] = layer_fma(v[j][q], out[q], g[q]);
            } else {
#pragma unroll
                for (int q = 0; q < kTwos<E>; ++q) out[q] = v[j][q] * out[q];
            }
            E* to = y + t * ld_y + e;
            if (layer_in_rows<kN<E>, E>(status, to, -e, (int)D - e, y, layer_end(y, T, D, ld_y)))
                store_word<E, kBroken>(to, layer_access<E, kN<E>>(out), -e, (int)D - e);
        }
    }
}

// ---- gradient --------------------------------------------------------------------------------------------------------------
// One block an SM, a row a team.  Every team has a ring in shared memory that bulk copies fill, of one row or of several that lie one
// behind the other: what is on its way (some 150 KB an SM) takes no registers.  A thread keeps to its columns -- a team's rows all start at the same
// place in a word --, so that the columns' sums of dy * n and dy stay in its registers; they end as the block's line of `work`: [blocks][2][D].
// 16384 rows of 4096 bfloat16 elements 103 us with the sum over the lines (3.9 TB/s; 7 of it the lines), 1000 of 500 binary32 elements 6.7.  Spilled
// sums made it 200 us: hence 384 threads.  Wide rows (12289 elements: 109 us for 2011) do spill,
// 440 bytes a thread, and narrow ones with broken words 40.
struct RingShape {
    uint32_t threads, teams, stages, rows;   // of a team; teams a block; stages of a team; rows of a stage
    uint32_t pitch;                          // distance of the rows of a stage
    uint32_t blocks, params;                 // of the grid; bytes of gamma, before the rings
};
constexpr uint32_t kSharedBytes = 216 * 1024, kMaxBarriers = 128;
template <int NV> constexpr int kMostThreads = NV == 4 ? 384 : 1024;      // of a block: what the registers have room for

template <typename E, typename P, int NV, bool kBroken>
__global__ void __launch_bounds__(kMostThreads<NV>, 1)
    norm_grad_kernel(unsigned* status, uint32_t T, uint32_t D, const E* dy, uint64_t ld_dy, const E* x, uint64_t ld_x, const float* mean, const float* rstd,
                     const void* gamma, E* dx, uint64_t ld_dx, float* work, const float* work_end, RingShape f)
{
    extern __shared__ __align__(128) unsigned char memory[];
    __shared__ uint64_t barriers[kMaxBarriers];
    __shared__ float sums[2][2][32];
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < f.teams * f.stages; ++i) layer_barrier(barriers + i, 1);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    const uint32_t team = threadIdx.x / f.threads, me = threadIdx.x - team * f.threads;
    const float* params = reinterpret_cast<const float*>(memory);
    unsigned char* ring = memory + f.params + team * f.stages * 2 * f.rows * f.pitch;
    uint64_t* full = barriers + team * f.stages;
    const uint64_t step = (uint64_t)gridDim.x * f.teams;
    uint64_t group = (uint64_t)blockIdx.x * f.teams + team;
    __syncthreads();
    rows_begin();
    // a team's rows all have as many elements before them (several of a group: none)
    const uint32_t off = kBroken ? before(x + group * ld_x) : 0u;
    const auto fill = [&](uint64_t g, uint32_t stage) {
        const uint64_t t = g * f.rows;
        if (t >= T) return;
        const uint32_t rows = (uint32_t)min((uint64_t)f.rows, T - t);
        const uint32_t bytes = f.rows > 1 ? rows * f.pitch : ((off + D) * (uint32_t)sizeof(E) + 15) / 16 * 16;
        // (with the rest of the words that they start and end in)
        const auto there = [&](const E* from, const E* first, uint64_t ld) {
            return ROWS_IN_ARRAY(status, from, bytes, (uintptr_t)first & ~(uintptr_t)15, ((uintptr_t)layer_end(first, T, D, ld) + 15) & ~(uintptr_t)15);
        };
        if (!there(dy + t * ld_dy - off, dy, ld_dy) || !there(x + t * ld_x - off, x, ld_x)) {
            layer_arrive(full + stage);
            return;
        }
        layer_arrive_with(full + stage, 2 * bytes);
        unsigned char* to = ring + stage * 2 * f.rows * f.pitch;
        const auto copy = [&](unsigned char* at, const E* from) {
            asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(layer_address(at)), "l"(from), "r"(bytes), "r"(layer_address(full + stage)) : "memory");
        };
        copy(to, dy + t * ld_dy - off);
        copy(to + f.rows * f.pitch, x + t * ld_x - off);
    };
    if (me == 0)
        for (uint32_t i = 0; i < f.stages; ++i) fill(group + i * step, i);
    bring_params<E, P, kBroken>(reinterpret_cast<float*>(memory), gamma, D, 1.0f);
    __syncthreads();
    LayerTwo dg[NV][kTwos<E>], db[NV][kTwos<E>];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int q = 0; q < kTwos<E>; ++q) dg[j][q] = db[j][q] = LayerTwo(0.0f);
    uint32_t head[4], end[4];
    const uint32_t last = (off + D - 1) / kN<E>;
    bits_of<E>(head, (int)off, kN<E>);
    bits_of<E>(end, last ? 0 : (int)off, (int)(off + D - last * kN<E>));
    uint32_t odd = 0, stage = 0, round = 0;
    for (; group * f.rows < T; group += step) {
        const uint32_t rows = (uint32_t)min((uint64_t)f.rows, T - group * f.rows);
        float m = mean[group * f.rows], rs = rstd[group * f.rows];
        layer_wait(status, full + stage, round);
        for (uint32_t k = 0; k < rows; ++k, odd ^= 1u) {
            const uint64_t t = group * f.rows + k;
            const unsigned char *at_dy = ring + (stage * 2 * f.rows + k) * f.pitch, *at_x = at_dy + f.rows * f.pitch;
            constexpr bool kPacked = NV == 2;            // (fewer registers: x is kept as it is, and normed again)
            Word<E> a[NV], b[kPacked ? NV : 1];
            Twos<E> p, g, n[kPacked ? 1 : NV];
            LayerTwo all(0.0f), along(0.0f);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t w = j * f.threads + me;
                const int e = (int)(w * kN<E>) - (int)off;
                if (e >= (int)D) break;
                const int i = kPacked ? 0 : j;
                a[j] = layer_read<E, kN<E>>(at_dy + w * 16);
                b[kPacked ? j : 0] = layer_read<E, kN<E>>(at_x + w * 16);
                if constexpr (kBroken) {                    // (what lies beside the row may be anything)
                    if (j == 0 && me == 0) { mask_word<E>(a[j], head); mask_word<E>(b[kPacked ? j : 0], head); }
                    if (w == last) { mask_word<E>(a[j], end); mask_word<E>(b[kPacked ? j : 0], end); }
                }
                layer_twos<E, kN<E>>(p, a[j]);
                layer_twos<E, kN<E>>(n[i], b[kPacked ? j : 0]);
                read_params<E, kBroken>(status, g, params, w, off, D);
#pragma unroll
                for (int q = 0; q < kTwos<E>; ++q) {
                    n[i][q] = (n[i][q] + LayerTwo(-m)) * LayerTwo(rs);
                    const LayerTwo u = p[q] * g[q];
                    dg[j][q] = layer_fma(p[q], n[i][q], dg[j][q]);
                    db[j][q] = db[j][q] + p[q];
                    all = all + u;
                    along = layer_fma(u, n[i][q], along);
                }
            }
            const float before_m = m, now = rs;
            if (k + 1 < rows) { m = mean[t + 1]; rs = rstd[t + 1]; }
            float s[2] = { all.sum(), along.sum() };
            team_sums<2>(f.threads, team, s, sums[odd]);
            if (k + 1 == rows) {
                // every warp of the team has read the stage
                if (f.threads == 32) __syncwarp();
                if (me == 0) fill(group + step * f.stages, stage);
                if (++stage == f.stages) { stage = 0; ++round; }
            }
            if (dx == nullptr) continue;
            const LayerTwo off_row(-s[0] / (float)D), along_row(-s[1] / (float)D);          // (divided, as the mean is)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t w = j * f.threads + me;
                const int e = (int)(w * kN<E>) - (int)off;
                if (e >= (int)D) break;
                layer_twos<E, kN<E>>(p, a[j]);
                if constexpr (kPacked) {
                    layer_twos<E, kN<E>>(n[0], b[j]);
#pragma unroll
                    for (int q = 0; q < kTwos<E>; ++q) n[0][q] = (n[0][q] + LayerTwo(-before_m)) * LayerTwo(now);
                }
                read_params<E, kBroken>(status, g, params, w, off, D);
#pragma unroll
                for (int q = 0; q < kTwos<E>; ++q) p[q] = layer_fma(n[kPacked ? 0 : j][q], along_row, layer_fma(p[q], g[q], off_row)) * LayerTwo(now);
                E* to = dx + t * ld_dx + e;
                if (layer_in_rows<kN<E>, E>(status, to, -e, (int)D - e, dx, layer_end(dx, T, D, ld_dx)))
                    store_word<E, kBroken>(to, layer_access<E, kN<E>>(p), -e, (int)D - e);
            }
        }
    }
    if (work == nullptr) return;
    // every team's sums in a place of its own, word by word; then one team after the other, column by column
    float *line = work + (uint64_t)blockIdx.x * 2 * D, *shared = reinterpret_cast<float*>(memory);
    const uint32_t words = f.threads * NV;
    __shared__ uint32_t offs[32];
    __syncthreads();
    if (me == 0) offs[team] = off;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int q = 0; q < kTwos<E>; q += 2) {
            const float2 u = dg[j][q].get(), v = dg[j][q + 1].get(), w = db[j][q].get(), z = db[j][q + 1].get();
            float* at = shared + (team * 2 * words + j * f.threads + me) * kN<E> + 2 * q;
            *reinterpret_cast<float4*>(at) = make_float4(u.x, u.y, v.x, v.y);
            *reinterpret_cast<float4*>(at + words * kN<E>) = make_float4(w.x, w.y, z.x, z.y);
        }
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 2 * D; c += blockDim.x) {
        const uint32_t which = c >= D ? 1u : 0u, col = c - which * D;
        float sum = 0.0f;
        for (uint32_t k = 0; k < f.teams; ++k) sum += shared[(k * 2 + which) * words * kN<E> + col + offs[k]];
        if (ROWS_IN_ARRAY(status, line + c, 4, work, work_end)) line[c] = sum;
    }
}

// dgamma and dbeta: the blocks' lines added up.  A block has 32 columns of the two; its 32 warps take every 32nd line each, then one adds
// the warps' sums in order.
__global__ void __launch_bounds__(1024) norm_params_kernel(uint32_t D, uint32_t lines, const float* work, float* dgamma, float* dbeta)
{
    __shared__ float sums[32][33];
    rows_begin();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t c = blockIdx.x * 32 + lane;
    const bool bias = blockIdx.y != 0;
    float s = 0.0f;
    if (c < D)
        for (uint32_t l = warp; l < lines; l += 32) s += work[((uint64_t)l * 2 + bias) * D + c];
    sums[warp][lane] = s;
    __syncthreads();
    s = layer_warp_sum(sums[lane][warp]);
    const uint32_t col = blockIdx.x * 32 + warp;
    float* to = bias ? dbeta : dgamma;
    if (lane == 0 && col < D && to) to[col] = s;
}

// ---- rows that the kernels above do not take ---------------------------------------------------------------------------------
// Too long for a block's registers, or the matrices' rows start at different places in a word: element by element, read more than once; the columns'
// sums are the block's line of `work` itself.
template <typename E, typename P> __device__ __forceinline__ float param(const void* a, uint32_t c, float otherwise)
{
    return a ? RowsElem<P>::up(((const P*)a)[c]) : otherwise;
}
__device__ __forceinline__ float block_sum(float v, float* sums)
{
    float a[1] = { v };
    team_sums<1>(1024, 0, a, reinterpret_cast<float(*)[32]>(sums));
    return a[0];
}
template <typename E, typename P>
__global__ void __launch_bounds__(1024) norm_long_kernel(uint32_t T, uint32_t D, const E* x, uint64_t ld_x, const void* gamma, const void* beta, float eps, E* y,
                                                         uint64_t ld_y, float* mean_out, float* rstd_out)
{
    __shared__ float sums[2][32];
    rows_begin();
    for (uint64_t t = blockIdx.x; t < T; t += gridDim.x) {
        const E* row = x + t * ld_x;
        float s = 0.0f;
        for (uint32_t c = threadIdx.x; c < D; c += 1024) s += RowsElem<E>::up(row[c]);
        const float mean = block_sum(s, sums[0]) / (float)D;
        s = 0.0f;
        for (uint32_t c = threadIdx.x; c < D; c += 1024) {
            const float d = RowsElem<E>::up(row[c]) - mean;
            s = __fmaf_rn(d, d, s);
        }
        const float rstd = 1.0f / sqrtf(block_sum(s, sums[1]) / (float)D + eps);
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[t] = mean;
            if (rstd_out) rstd_out[t] = rstd;
        }
        for (uint32_t c = threadIdx.x; c < D; c += 1024)
            y[t * ld_y + c] = RowsElem<E>::down(__fmaf_rn((RowsElem<E>::up(row[c]) - mean) * rstd, param<E, P>(gamma, c, 1.0f), param<E, P>(beta, c, 0.0f)));
    }
}
template <typename E, typename P>
__global__ void __launch_bounds__(1024) norm_grad_long_kernel(unsigned* status, uint32_t T, uint32_t D, const E* dy, uint64_t ld_dy, const E* x, uint64_t ld_x,
                                                              const float* mean, const float* rstd, const void* gamma, E* dx, uint64_t ld_dx, float* work,
                                                              const float* work_end)
{
    __shared__ float sums[2][2][32];
    rows_begin();
    float* line = work + (uint64_t)blockIdx.x * 2 * D;
    bool first = true;
    for (uint64_t t = blockIdx.x; t < T; t += gridDim.x, first = false) {
        const float m = mean[t], r = rstd[t];
        float s[2] = { 0.0f, 0.0f };
        for (uint32_t c = threadIdx.x; c < D; c += 1024) {
            const float d = RowsElem<E>::up(dy[t * ld_dy + c]), n = (RowsElem<E>::up(x[t * ld_x + c]) - m) * r, w = d * param<E, P>(gamma, c, 1.0f);
            s[0] += w;
            s[1] = __fmaf_rn(w, n, s[1]);
            if (work && ROWS_IN_ARRAY(status, line + D + c, 4, work, work_end)) {
                line[c] = __fmaf_rn(d, n, first ? 0.0f : line[c]);
                line[D + c] = d + (first ? 0.0f : line[D + c]);
            }
        }
        if (dx == nullptr) continue;
        team_sums<2>(1024, 0, s, sums[(t / gridDim.x) & 1]);
        const float along = s[1] / (float)D, off = s[0] / (float)D;
        for (uint32_t c = threadIdx.x; c < D; c += 1024) {
            const float n = (RowsElem<E>::up(x[t * ld_x + c]) - m) * r;
            dx[t * ld_dx + c] = RowsElem<E>::down(r * (__fmaf_rn(RowsElem<E>::up(dy[t * ld_dy + c]), param<E, P>(gamma, c, 1.0f), -off) - n * along));
        }
    }
}

// ---- which kernel ----------------------------------------------------------------------------------------------------
// Lets a kernel have that much shared memory (once a kernel and device).
template <typename... Params> bool shared_memory(void (*kernel)(Params...), std::atomic<bool> (&ready)[kRowsMaxDevices])
{
    const int dev = rows_device();
    if (dev >= 0 && ready[dev]) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedBytes) != cudaSuccess) return false;
    if (dev >= 0) ready[dev] = true;
    return true;
}
// Words of a row of D elements at most.
template <typename E> uint32_t words_of(uint32_t D, bool odd) { return (D + (odd ? kN<E> - 1 : 0) + kN<E> - 1) / kN<E>; }
// Threads of a team that has a row of so many words, nv each.
uint32_t team_of(uint32_t words, uint32_t nv) { return ((words + nv - 1) / nv + 31) / 32 * 32; }
uint32_t common_divisor(uint32_t a, uint32_t b)
{
    while (b) { const uint32_t r = a % b; a = b; b = r; }
    return a;
}
bool same_place(const void* a, uint64_t ld_a, const void* b, uint64_t ld_b, uint32_t size)
{
    return (((uintptr_t)a ^ (uintptr_t)b) & 15u) == 0 && ((ld_a - ld_b) * size & 15u) == 0;
}

struct NormArgs {
    unsigned* status;
    uint32_t T, D;
    const void *x, *gamma, *beta;
    uint64_t ld_x, ld_y;
    float eps;
    void* y;
    float *mean, *rstd;
};
template <typename E, typename P, int NV, bool kBroken> int norm_with(const NormArgs& a, uint32_t threads, uint32_t shared, cudaStream_t s)
{
    static std::atomic<bool> ready[kRowsMaxDevices];
    if (!shared_memory(norm_kernel<E, P, NV, kBroken>, ready)) return -1;
    const uint32_t whole = kThreads<NV> / threads, teams = threads > 32 && whole > 15 ? 15 : whole, most = rows_sm_count();
    const uint64_t blocks = ((uint64_t)a.T + teams - 1) / teams;
    return rows_launch(norm_kernel<E, P, NV, kBroken>, dim3((uint32_t)(blocks < most ? blocks : most)), dim3(teams * threads), shared, s, 0, a.status, a.T, a.D, threads,
                       (const E*)a.x, a.ld_x, a.gamma, a.beta, a.eps, (E*)a.y, a.ld_y, a.mean, a.rstd);
}
template <typename E, typename P> int norm_as(const NormArgs& a, cudaStream_t s)
{
    const bool odd = (((uintptr_t)a.x | a.ld_x * sizeof(E)) & 15u) != 0, broken = odd || a.D % kN<E> != 0;
    const uint32_t words = words_of<E>(a.D, odd), shared = 2 * params_room<E>(a.D) * 4;
    // words of a thread: as many as make a row a warp's, but few of a wide row.  2^25 bfloat16 elements in rows of 64 words: 2 of them 30 us, 4 34; of
    // 128: 37 and 31, of 1536: 54 and 49, of 2048: 51 and 60 (and beyond that 2 are not enough)
    const int nv = words <= 32 ? 1 : words <= 64 ? 2 : words <= 1536 ? 4 : words <= 2048 ? 2 : 4;
    const uint32_t threads = team_of(words, nv);
    if (threads <= (nv == 4 ? kThreads<4> : kThreads<2>) && shared <= kSharedBytes && same_place(a.x, a.ld_x, a.y, a.ld_y, sizeof(E))) {
#define NORM(NV) (broken ? norm_with<E, P, NV, true>(a, threads, shared, s) : norm_with<E, P, NV, false>(a, threads, shared, s))
        return nv == 1 ? NORM(1) : nv == 2 ? NORM(2) : NORM(4);
#undef NORM
    }
    const uint32_t most = 2 * rows_sm_count();
    return rows_launch(norm_long_kernel<E, P>, dim3(a.T < most ? a.T : most), dim3(1024), 0, s, 0, a.T, a.D, (const E*)a.x, a.ld_x, a.gamma, a.beta, a.eps,
                       (E*)a.y, a.ld_y, a.mean, a.rstd);
}

struct GradArgs {
    uint32_t T, D;
    const void *dy, *x, *gamma;
    uint64_t ld_dy, ld_x, ld_dx;
    const float *mean, *rstd;
    void* dx;
    float *dgamma, *dbeta, *work;
    const float* work_end;
    unsigned* status;
};
constexpr uint32_t kLines = 296;       // of work at most

template <typename E> RingShape ring_shape(const GradArgs& a, bool odd, int* nv)
{
    RingShape f = {};
    const uint32_t S = sizeof(E), words = words_of<E>(a.D, odd), sms = rows_sm_count() < kLines ? rows_sm_count() : kLines;
    // words of a thread: four, so that a row's two sums are over few threads; one where a warp has a row with that, and a wide row's two, so that one
    // block's threads have it.  2^25 bfloat16 elements in rows of 32 words: one 60 us, 4 72; of 64: one 72, 2 67, 4 62; of 1536: 4 78, 2 102
    *nv = words <= 32 ? 1 : words <= 4 * kMostThreads<4> ? 4 : 2;
    f.threads = team_of(words, *nv);
    const uint32_t whole = *nv == 4 ? kMostThreads<4> : kMostThreads<1>;
    if (f.threads > whole) return f;
    f.teams = whole / f.threads;
    if (f.threads > 32 && f.teams > 15) f.teams = 15;                  // (a named barrier each)
    f.pitch = words * 16;
    f.params = (params_room<E>(a.D) * 4 + 127) / 128 * 128;
    // several rows a copy where there are rows enough and they lie one behind the other: one takes some 200 cycles, whatever it brings
    const uint64_t each = (uint64_t)a.T / ((uint64_t)sms * f.teams * 4);
    f.rows = !odd && f.pitch == a.D * S && a.ld_x == a.D && a.ld_dy == a.D && f.pitch < 8192 ? 8192 / f.pitch : 1;
    if (f.rows > each) f.rows = each ? (uint32_t)each : 1;
    const uint32_t room = kSharedBytes - f.params, most = kMaxBarriers / f.teams;
    while (f.rows > 1 && 4 * 2 * f.teams * f.rows * f.pitch > room) f.rows /= 2;
    const uint32_t stages = room / (2 * f.teams * f.rows * f.pitch);
    f.stages = stages < most ? stages : most;
    if (f.stages > 8) f.stages = 8;
    if (f.stages < 2 || (uint64_t)f.teams * f.threads * *nv * kN<E> * 8 > kSharedBytes) { f.stages = 0; return f; }
    const uint64_t blocks = ((uint64_t)a.T + (uint64_t)f.rows * f.teams - 1) / ((uint64_t)f.rows * f.teams);
    f.blocks = blocks < sms ? (uint32_t)blocks : sms;
    if (odd && blocks > sms) {
        // teams that have several rows: rows a whole number of periods apart start at the same place
        const uint32_t apart = (uint32_t)(a.ld_x * S & 15u), period = 16 / common_divisor(16, apart ? apart : 16);
        f.blocks -= f.blocks % (period / common_divisor(period, f.teams));
    }
    return f;
}
template <typename E, typename P, int NV, bool kBroken> int ring_with(const GradArgs& a, const RingShape& f, float* work, cudaStream_t s)
{
    static std::atomic<bool> ready[kRowsMaxDevices];
    if (!shared_memory(norm_grad_kernel<E, P, NV, kBroken>, ready)) return -1;
    return rows_launch(norm_grad_kernel<E, P, NV, kBroken>, dim3(f.blocks), dim3(f.teams * f.threads), kSharedBytes, s, 0, a.status, a.T, a.D,
                       (const E*)a.dy, a.ld_dy, (const E*)a.x, a.ld_x, a.mean, a.rstd, a.gamma, (E*)a.dx, a.ld_dx, work, a.work_end, f);
}
template <typename E, typename P> int grad_as(const GradArgs& a, cudaStream_t s)
{
    const bool params = a.dgamma || a.dbeta;
    float* work = params ? a.work : nullptr;
    uint32_t lines = 0;
    int n = 0;
    if (a.T) {
        int nv = 1;
        const bool odd = (((uintptr_t)a.x | a.ld_x * sizeof(E)) & 15u) != 0;
        const bool broken = odd || a.D % kN<E> != 0;
        const bool alike = same_place(a.x, a.ld_x, a.dy, a.ld_dy, sizeof(E)) && (!a.dx || same_place(a.x, a.ld_x, a.dx, a.ld_dx, sizeof(E)));
        const RingShape f = alike ? ring_shape<E>(a, odd, &nv) : RingShape();
        if (f.stages) {
            lines = f.blocks;
#define RING(NV) (broken ? ring_with<E, P, NV, true>(a, f, work, s) : ring_with<E, P, NV, false>(a, f, work, s))
            n = nv == 1 ? RING(1) : nv == 4 ? RING(4) : RING(2);
#undef RING
        } else {
            lines = a.T < kLines ? a.T : kLines;
            n = rows_launch(norm_grad_long_kernel<E, P>, dim3(lines), dim3(1024), 0, s, 0, a.status, a.T, a.D, (const E*)a.dy, a.ld_dy, (const E*)a.x, a.ld_x,
                            a.mean, a.rstd, a.gamma, (E*)a.dx, a.ld_dx, work, a.work_end);
        }
        if (n < 0) return n;
    }
    if (!params) return n;
    const int m = rows_launch(norm_params_kernel, dim3((a.D + 31) / 32, 2), dim3(1024), 0, s, 0, a.D, lines, (const float*)a.work, a.dgamma, a.dbeta);
    return m < 0 ? m : n + m;
}

// Runs CALL(type, type of the parameters).
#define WITH_TYPES(dtype, ptype, CALL)                                                              \
    do {                                                                                            \
        if ((dtype) == PEARL_F32) { CALL(float, float); }                                           \
        else if ((dtype) == PEARL_F16) { if ((ptype) == PEARL_F32) { CALL(__half, float); } else { CALL(__half, __half); } }             \
        else { if ((ptype) == PEARL_F32) { CALL(__nv_bfloat16, float); } else { CALL(__nv_bfloat16, __nv_bfloat16); } }                  \
    } while (0)

}  // namespace

int layer_launch_norm(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* x, uint64_t ld_x, uint32_t ptype, const void* gamma, const void* beta,
                      float eps, void* y, uint64_t ld_y, float* mean, float* rstd, cudaStream_t s)
{
    const NormArgs a = { status, T, D, x, gamma, beta, ld_x, ld_y, eps, y, mean, rstd };
#define NORM_AS(E, P) return norm_as<E, P>(a, s)
    WITH_TYPES(dtype, ptype, NORM_AS);
#undef NORM_AS
}

uint64_t layer_norm_grad_work_bytes(uint32_t T, uint32_t D) { return (T < 1 ? 1u : T < kLines ? T : kLines) * 2ull * D * sizeof(float); }

int layer_launch_norm_grad(unsigned* status, uint32_t T, uint32_t D, uint32_t dtype, const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x,
                           const float* mean, const float* rstd, uint32_t ptype, const void* gamma, void* dx, uint64_t ld_dx, float* dgamma,
                           float* dbeta, float* work, uint64_t work_bytes, cudaStream_t s)
{
    const GradArgs a = { T, D, dy, x, gamma, ld_dy, ld_x, ld_dx, mean, rstd, dx, dgamma, dbeta, work, (const float*)((const char*)work + work_bytes), status };
#define GRAD_AS(E, P) return grad_as<E, P>(a, s)
    WITH_TYPES(dtype, ptype, GRAD_AS);
#undef GRAD_AS
}
