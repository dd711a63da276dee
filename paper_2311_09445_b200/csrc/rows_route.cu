// The router: the k best of E experts with their softmax weights, and its gradient.
//
// Up to 8 choices (route_kernel): L lanes have a row, N consecutive logits each.  A logit and its expert are one whole number that
// orders like (larger logit, lower expert): for 16-bit logits 32 bits, so that a comparison and exchange is one maximum and two
// multiply-adds.  A lane sorts its logits KP at a time by a network (KP: k rounded up to a power of two), keeps the KP best of them by
// bitonic merges, and merges with the other lanes' lists by exchanges.  No branch depends on the data.  65521 rows of 128 bfloat16
// logits, k = 8, over the chosen ones: 8.2 us, bound by these exchanges; the 21 MB it moves are 3.2.  Its gradient 6.1 us, the 23 MB it
// reads and writes are 3.5.  (By rounds, below, choice and gradient took 49 where this way took 13.8; they are 14.3 now.)  Over all experts
// 10.7 and 13.7 us: an exponential a logit in each.  binary32 logits cost more, because a 64-bit exchange is four such instructions and
// four multiply-adds: 65521 rows of 64, k = 6: 10.7 us.
// More choices (rounds_kernel): k rounds of "largest that is left" over the row's lanes, so bound by k chains of warp maxima: 65521 rows of 128
// bfloat16 logits 55 us with k = 16 and 103 with k = 32, of 64 binary32 ones 28 with k = 16.
#include "rows_internal.cuh"

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kRouteThreads = 128;         // of route_kernel: as many rows an SM in smaller steps (65521 rows of 64 binary32 logits: 4 % faster)
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
__global__ void __launch_bounds__(kThreads) rounds_kernel(unsigned* status, uint32_t T, uint32_t experts, uint32_t k, const E* logits,
                                                         uint64_t ld, uint32_t wide, uint32_t over_chosen, float* w,
                                                         int32_t* ids)
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
        for (int i = 0; i < N; ++i) sum = __fadd_rn(sum, expf(__fsub_rn(x[i], shift)));
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
            chosen_sum = __fadd_rn(chosen_sum, expf(__fsub_rn(gmax, shift)));
            gmax = over_lanes_max<L>(best);
        }
    }
    if (!there) return;
    const float denominator = over_chosen ? chosen_sum : sum;
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const uint32_t j = h * L + lane;
        if (j < k && ROWS_IN_BOUNDS(status, held_id[h] >= -1 && held_id[h] < (int32_t)experts)) {
            ids[t * k + j] = held_id[h];
            w[t * k + j] = held_id[h] < 0 ? 0.0f : __fdiv_rn(expf(__fsub_rn(held_x[h], shift)), denominator);
        }
    }
}

// ---- up to 8 choices -------------------------------------------------------------------------------------------------
// Keys.  16-bit logits: the logit's bits made rising in the upper half, 0xFFFF - expert in the lower; binary32: the same in 64 bits.
// Up to -infinity's key (which places behind the last expert have, too) there is nothing to choose.
template <typename E> struct Key;
template <> struct Key<float> {
    typedef uint64_t type;
    static constexpr uint32_t kNothing = 0x007FFFFFu;          // of -infinity
    static __device__ __forceinline__ uint32_t canonical(uint32_t w) { return __float_as_uint(__fadd_rn(__uint_as_float(w), 0.0f)); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        float m;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
        return __float_as_uint(m);
    }
    static __device__ __forceinline__ bool bad(uint32_t largest) { return !(__uint_as_float(largest) < kInf); }
    static __device__ __forceinline__ void mend(uint32_t& w) { if (!(__uint_as_float(w) < kInf)) w = 0xFF800000u; }
    template <int I> static __device__ __forceinline__ type of(const uint32_t* w)
    {
        const uint32_t b = w[I];
        return ((uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32) | (0xFFFFu - I);
    }
    static __device__ __forceinline__ uint32_t rising(type k) { return (uint32_t)(k >> 32); }
    static __device__ __forceinline__ float logit(type k)
    {
        const uint32_t r = rising(k);
        return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r);
    }
    static __device__ __forceinline__ float value(const uint32_t* w, int i) { return __uint_as_float(w[i]); }
};
template <typename E> struct Key16 {
    typedef uint32_t type;
    // both halves at once: a set sign flips the other bits, too (prmt spreads the two signs)
    static __device__ __forceinline__ uint32_t rising2(uint32_t w)
    {
        uint32_t signs;
        asm("prmt.b32 %0, %1, 0, 0xBB99;" : "=r"(signs) : "r"(w));
        return w ^ (signs | 0x80008000u);
    }
    template <int I> static __device__ __forceinline__ type of(const uint32_t* w)
    {
        const uint32_t r = rising2(w[I / 2]);
        return I % 2 ? (r & 0xFFFF0000u) | (0xFFFFu - I) : r * 0x10000u + (0xFFFFu - I);
    }
    static __device__ __forceinline__ uint32_t rising(type k) { return k >> 16; }
    static __device__ __forceinline__ uint16_t bits(type k) { return (uint16_t)((k >> 16) ^ (k & 0x80000000u ? 0x8000u : 0xFFFFu)); }
};
template <> struct Key<__half> : Key16<__half> {
    static constexpr uint32_t kNothing = 0x03FFu;
    static __device__ __forceinline__ __half2 as(uint32_t w) { return *reinterpret_cast<const __half2*>(&w); }
    static __device__ __forceinline__ uint32_t word(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ uint32_t canonical(uint32_t w) { return word(__hadd2_rn(as(w), as(0u))); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return word(__hmax2_nan(as(a), as(b))); }
    static __device__ __forceinline__ bool bad(uint32_t largest) { const float2 f = __half22float2(as(largest)); return !(f.x < kInf) || !(f.y < kInf); }
    static __device__ __forceinline__ void mend(uint32_t& w)
    {
        const float2 f = __half22float2(as(w));
        if (!(f.x < kInf)) w = (w & 0xFFFF0000u) | 0xFC00u;
        if (!(f.y < kInf)) w = (w & 0x0000FFFFu) | 0xFC000000u;
    }
    static __device__ __forceinline__ float logit(type k) { return __half2float(__ushort_as_half(bits(k))); }
    static __device__ __forceinline__ float value(const uint32_t* w, int i) { const float2 f = __half22float2(as(w[i / 2])); return i % 2 ? f.y : f.x; }
};
template <> struct Key<__nv_bfloat16> : Key16<__nv_bfloat16> {
    static constexpr uint32_t kNothing = 0x007Fu;
    static __device__ __forceinline__ __nv_bfloat162 as(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
    static __device__ __forceinline__ uint32_t word(__nv_bfloat162 h) { return *reinterpret_cast<const uint32_t*>(&h); }
    static __device__ __forceinline__ uint32_t canonical(uint32_t w) { return word(__hadd2_rn(as(w), as(0u))); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return word(__hmax2_nan(as(a), as(b))); }
    static __device__ __forceinline__ float2 both(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ bool bad(uint32_t largest) { const float2 f = both(largest); return !(f.x < kInf) || !(f.y < kInf); }
    static __device__ __forceinline__ void mend(uint32_t& w)
    {
        const float2 f = both(w);
        if (!(f.x < kInf)) w = (w & 0xFFFF0000u) | 0xFF80u;
        if (!(f.y < kInf)) w = (w & 0x0000FFFFu) | 0xFF800000u;
    }
    static __device__ __forceinline__ float logit(type k) { return __uint_as_float((uint32_t)bits(k) << 16); }
    static __device__ __forceinline__ float value(const uint32_t* w, int i) { const float2 f = both(w[i / 2]); return i % 2 ? f.y : f.x; }
};

// The larger first.  The smaller one is a + b - larger (modulo 2^32, word by word), by two multiply-adds: minima, maxima, comparisons and
// selections share a pipe that is the bound here, and multiply-adds have their own.  `one` is (1, -1) as an argument of the kernel, so
// that they stay what they are.  With minima 9.6 us instead of 8.3 at the size above.
__device__ __forceinline__ uint32_t other_of(uint32_t a, uint32_t b, uint32_t larger, uint2 one)
{
    uint32_t t, lo;
    asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(t) : "r"(a), "r"(one.x), "r"(b));
    asm("mad.lo.u32 %0, %1, %2, %3;" : "=r"(lo) : "r"(larger), "r"(one.y), "r"(t));
    return lo;
}
__device__ __forceinline__ void order(uint32_t& a, uint32_t& b, uint2 one)
{
    const uint32_t hi = max(a, b);
    b = other_of(a, b, hi, one);
    a = hi;
}
__device__ __forceinline__ void order(uint64_t& a, uint64_t& b, uint2 one)
{
    const uint64_t hi = a > b ? a : b;
    b = ((uint64_t)other_of((uint32_t)(a >> 32), (uint32_t)(b >> 32), (uint32_t)(hi >> 32), one) << 32) |
        other_of((uint32_t)a, (uint32_t)b, (uint32_t)hi, one);
    a = hi;
}
// Batcher's merge exchange sort (Knuth, 5.2.2), falling: 19 exchanges for 8 keys.
template <int P, typename K> __device__ __forceinline__ void sort_falling(K (&a)[P], uint2 one)
{
#pragma unroll
    for (int p = 1; p < P; p *= 2)
#pragma unroll
        for (int q = p; q >= 1; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < P; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < P && (i + j) / (2 * p) == (i + j + q) / (2 * p)) order(a[i + j], a[i + j + q], one);
}
// The P largest of two falling lists (b is handed over reversed), falling.
template <int P, typename K> __device__ __forceinline__ void merge_falling(K (&a)[P], const K (&reversed)[P], uint2 one)
{
#pragma unroll
    for (int i = 0; i < P; ++i) a[i] = a[i] > reversed[i] ? a[i] : reversed[i];
#pragma unroll
    for (int d = P / 2; d > 0; d /= 2)
#pragma unroll
        for (int i = 0; i < P; ++i)
            if ((i & d) == 0) order(a[i], a[i + d], one);
}
template <typename E, int FROM, int P, int I = 0> struct KeysOf {
    static __device__ __forceinline__ void get(const uint32_t* w, typename Key<E>::type* out)
    {
        out[I] = Key<E>::template of<FROM + I>(w);
        if constexpr (I + 1 < P) KeysOf<E, FROM, P, I + 1>::get(w, out);
    }
};
// The P best of a lane's logits FROM .. N - 1, merged into `best`.
template <typename E, int N, int P, int FROM = 0> struct Choose {
    typedef typename Key<E>::type K;
    static __device__ __forceinline__ void run(const uint32_t* w, K (&best)[P], uint2 one)
    {
        K group[P];
        KeysOf<E, FROM, P>::get(w, group);
        sort_falling<P>(group, one);
        if constexpr (FROM == 0) {
#pragma unroll
            for (int i = 0; i < P; ++i) best[i] = group[i];
        } else {
            K reversed[P];
#pragma unroll
            for (int i = 0; i < P; ++i) reversed[i] = group[P - 1 - i];
            merge_falling<P>(best, reversed, one);
        }
        if constexpr (FROM + P < N) Choose<E, N, P, FROM + P>::run(w, best, one);
    }
};

__device__ __forceinline__ uint32_t from_lane(uint32_t k, int d, int width) { return __shfl_xor_sync(0xFFFFFFFFu, k, d, width); }
__device__ __forceinline__ uint64_t from_lane(uint64_t k, int d, int width) { return __shfl_xor_sync(0xFFFFFFFFu, k, d, width); }

template <typename E, int L, int N, int P>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(unsigned* status, uint32_t T, uint32_t experts, uint32_t k, const E* logits,
                                                         uint64_t ld, uint32_t wide, uint32_t over_chosen, float* w,
                                                         int32_t* ids, uint2 one)
{
    typedef Key<E> Q;
    typedef typename Q::type K;
    constexpr int kWords = N * (int)sizeof(E) / 4, kBytes = N * (int)sizeof(E), kAccess = kBytes < 16 ? kBytes : 16;
    static_assert(N >= P && N % P == 0 && kWords >= 1, "whole groups");
    rows_begin();
    const uint32_t lane = threadIdx.x % L, first = lane * N;
    const uint64_t t = (uint64_t)blockIdx.x * (kRouteThreads / L) + threadIdx.x / L;
    const uint32_t there = t < T && first < experts ? (experts - first < (uint32_t)N ? experts - first : (uint32_t)N) : 0u;
    const E* row = logits + (t < T ? t : 0) * ld + first;
    uint32_t x[kWords];
    if (wide && there == (uint32_t)N) {
#pragma unroll
        for (int i = 0; i < kBytes / kAccess; ++i) {
            RowsRaw<kAccess> raw;
            rows_load_if<false>(true, raw, reinterpret_cast<const unsigned char*>(row) + i * kAccess);
#pragma unroll
            for (int j = 0; j < kAccess / 4; ++j) x[i * (kAccess / 4) + j] = raw.r[j];
        }
    } else if constexpr (sizeof(E) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (uint32_t)i < there ? __float_as_uint(row[i]) : 0xFF800000u;
    } else {
        const uint16_t minus_inf = RowsElem<E>::bits(RowsElem<E>::down(-kInf));
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint32_t lo = (uint32_t)(2 * i) < there ? RowsElem<E>::bits(row[2 * i]) : minus_inf;
            const uint32_t hi = (uint32_t)(2 * i + 1) < there ? RowsElem<E>::bits(row[2 * i + 1]) : minus_inf;
            x[i] = lo | hi << 16;
        }
    }
    uint32_t largest = x[0];
#pragma unroll
    for (int i = 1; i < kWords; ++i) largest = Q::larger(largest, x[i]);
    if (Q::bad(largest)) {
        atomicOr(status, PEARL_ST_BAD_SCORE);
#pragma unroll
        for (int i = 0; i < kWords; ++i) Q::mend(x[i]);
    }
#pragma unroll
    for (int i = 0; i < kWords; ++i) x[i] = Q::canonical(x[i]);           // (-0 becomes 0)

    K best[P];
    Choose<E, N, P>::run(x, best, one);
#pragma unroll
    for (int i = 0; i < P; ++i) best[i] -= first;                         // the expert's number in the row
#pragma unroll
    for (int d = 1; d < L; d *= 2) {
        K reversed[P];
#pragma unroll
        for (int i = 0; i < P; ++i) reversed[i] = from_lane(best[P - 1 - i], d, L);
        merge_falling<P>(best, reversed, one);
    }
    const float shift = Q::rising(best[0]) <= Q::kNothing ? 0.0f : Q::logit(best[0]);
    // every lane has the row's choices; each hands out its share of them
    constexpr int kEach = P / L > 0 ? P / L : 1;
    K mine[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine[i] = 0;
#pragma unroll
    for (int i = 0; i < P; ++i)
        if ((int)lane == i / kEach) mine[i % kEach] = best[i];
    float e[kEach], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (lane * kEach + i >= k || Q::rising(mine[i]) <= Q::kNothing) mine[i] = 0;
        e[i] = mine[i] ? expf(__fsub_rn(Q::logit(mine[i]), shift)) : 0.0f;
        if (over_chosen) sum = __fadd_rn(sum, e[i]);
    }
    if (!over_chosen) {
#pragma unroll
        for (int i = 0; i < N; ++i) sum = __fadd_rn(sum, expf(__fsub_rn(Q::value(x, i), shift)));
    }
    sum = over_lanes_sum<L>(sum);
    if (t >= T) return;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t j = lane * kEach + i;
        if (j < k && ROWS_IN_BOUNDS(status, !mine[i] || 0xFFFFu - (uint32_t)(mine[i] & 0xFFFFu) < experts)) {
            ids[t * k + j] = mine[i] ? (int32_t)(0xFFFFu - (uint32_t)(mine[i] & 0xFFFFu)) : -1;
            w[t * k + j] = mine[i] ? __fdiv_rn(e[i], sum) : 0.0f;
        }
    }
}

// ---- the gradient ----------------------------------------------------------------------------------------------------
// A warp has R rows at a time.  First a lane has one of a row's choices (KL lanes a row, k rounded up to a power of two): the mean
// is a sum over those lanes, and the choices' parts are laid out by expert in shared memory.  Then 32 / R lanes have a row's
// experts, 16 bytes at a time, and write the gradient: bound by the bytes of dlogits.
// B logits of a row from c on, by accesses of M (which a row's length is a multiple of): -infinity behind the last expert, and for NaN
// and +infinity, of which it tells.
template <typename E, int M, int B>
__device__ __forceinline__ bool load_block(unsigned* status, const E* x, uint32_t c, uint32_t experts, float (&v)[B])
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < B; i += M) {
        if (c + i < experts && ROWS_IN_BOUNDS(status, c + i + M <= experts)) {
            const RowsVec<E, M> a = rows_load_vec<E, M>(x + c + i);
#pragma unroll
            for (int m = 0; m < M; ++m) v[i + m] = a.get(m);
        } else {
#pragma unroll
            for (int m = 0; m < M; ++m) v[i + m] = -kInf;
        }
    }
#pragma unroll
    for (int i = 0; i < B; ++i)
        if (!(v[i] < kInf)) { bad = true; v[i] = -kInf; }
    return bad;
}
// Where the softmax runs over all experts a lane holds its logits, H = 16 or 32 of them, and then their exponentials (read again for the
// maximum, the sum and the gradient: 16.1 us instead of 12.6 for 65521 rows of 128 bfloat16 logits, when the exponentials were shorter; 13.7 now).
constexpr uint32_t kRowFloats = 1024;                // of shared memory per warp at most: R rows of the experts, rounded up to 4; so 32 a lane
template <typename E, int M, bool kChosen, int H>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(unsigned* status, uint32_t T, uint32_t experts, uint32_t k, uint32_t log_kl,
                                                              uint32_t log_r, const E* logits, uint64_t ld,
                                                              const float* w, const int32_t* ids,
                                                              const float* dw, E* dlogits, uint64_t ld_d)
{
    constexpr int B = 16 / (int)sizeof(E);
    extern __shared__ __align__(16) float shared[];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32, pitch = (experts + 3u) & ~3u, rows = 1u << log_r;
    float* g = shared + warp * rows * pitch;
    for (uint32_t i = lane * 4; i < rows * pitch; i += 128) *reinterpret_cast<float4*>(g + i) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    rows_begin();

    const uint32_t groups = (T + rows - 1) >> log_r, all_warps = gridDim.x * (kThreads / 32);
    const uint32_t r = lane >> log_kl, j = lane & ((1u << log_kl) - 1u);
    // (a lane's experts do not depend on M, the width of an access: neither does the order of the sum)
    const uint32_t log_lr = 5u - log_r, row = lane >> log_lr, step = B << log_lr, from = (lane & ((1u << log_lr) - 1u)) * B;
    int32_t next_id = -1;
    float next_weight = 0.0f, next_d = 0.0f;
    const auto fetch = [&](uint32_t group) {
        const uint64_t t = ((uint64_t)group << log_r) + r;
        const bool slot = group < groups && r < rows && t < T && j < k;
        const uint64_t at = t * k + j;
        next_id = rows_read_if(slot, ids + at, -1);
        next_weight = rows_read_if(slot, w + at, 0.0f);
        next_d = rows_read_if(slot, dw + at, 0.0f);
    };
    uint32_t group = blockIdx.x * (kThreads / 32) + warp;
    fetch(group);
    for (; group < groups; group += all_warps) {
        int32_t id = next_id;
        const float weight = next_weight, d = next_d;
        fetch(group + all_warps);                                         // (the next rows' choices are on their way meanwhile)
        if ((uint32_t)id >= experts) {
            if (id != -1) atomicOr(status, PEARL_ST_BAD_INDEX);
            id = -1;
        }
        if (id >= 0 && !ROWS_IN_BOUNDS(status, r * pitch + (uint32_t)id < rows * pitch)) id = -1;
        float mean = id >= 0 ? __fmul_rn(weight, d) : 0.0f;
        for (uint32_t q = 1; q < 1u << log_kl; q *= 2) mean = __fadd_rn(mean, __shfl_xor_sync(0xFFFFFFFFu, mean, q));
        const float add = kChosen ? __fmul_rn(weight, __fsub_rn(d, mean)) : d;
        const uint32_t to = r * pitch + (uint32_t)id;
        __syncwarp();
        // each choice leaves its lane's number (as bits) at its expert and looks whether it is still there: a hand-made row may name one twice
        if (id >= 0) g[to] = __uint_as_float(lane);
        __syncwarp();
        const bool alone = id < 0 || __float_as_uint(g[to]) == lane;
        __syncwarp();
        if (__all_sync(0xFFFFFFFFu, alone)) {
            if (id >= 0) g[to] = add;
        } else {
            if (id >= 0) g[to] = 0.0f;
            __syncwarp();
            for (uint32_t q = 0; q < 1u << log_kl; ++q) {                 // (its parts in order)
                if (j == q && id >= 0) g[to] = __fadd_rn(g[to], add);
                __syncwarp();
            }
        }
        __syncwarp();

        const uint64_t t = ((uint64_t)group << log_r) + row;
        mean = __shfl_sync(0xFFFFFFFFu, mean, (int)(row << log_kl));
        const bool there = t < T;
        float held[kChosen ? 1 : H / B][B];
        if constexpr (!kChosen) {
            float top = -kInf, sum = 0.0f;
            const E* x = logits + (there ? t : 0) * ld;
            bool bad = false;
#pragma unroll
            for (int n = 0; n < H / B; ++n) {
                const uint32_t c = from + n * step;
                if (c < experts && there) {
                    bad |= load_block<E, M, B>(status, x, c, experts, held[n]);
                } else {
#pragma unroll
                    for (int i = 0; i < B; ++i) held[n][i] = -kInf;
                }
            }
            if (bad) atomicOr(status, PEARL_ST_BAD_SCORE);
#pragma unroll
            for (int n = 0; n < H / B; ++n)
#pragma unroll
                for (int i = 0; i < B; ++i) top = fmaxf(top, held[n][i]);
            for (uint32_t q = 1; q < 1u << log_lr; q *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, q));
            const float shift = top == -kInf ? 0.0f : top;
#pragma unroll
            for (int n = 0; n < H / B; ++n)
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    held[n][i] = expf(__fsub_rn(held[n][i], shift));
                    sum = __fadd_rn(sum, held[n][i]);
                }
            for (uint32_t q = 1; q < 1u << log_lr; q *= 2) sum = __fadd_rn(sum, __shfl_xor_sync(0xFFFFFFFFu, sum, q));
            // (a product with the rounded reciprocal instead of a division a logit: one half step of binary32 more)
            const float p_scale = sum > 0.0f ? __fdiv_rn(1.0f, sum) : 0.0f;
#pragma unroll
            for (int n = 0; n < H / B; ++n)
#pragma unroll
                for (int i = 0; i < B; ++i) held[n][i] = __fmul_rn(held[n][i], p_scale);
        }
        const float* mine = g + row * pitch;
        const auto write = [&](uint32_t c, const float* p) {
            float part[B];
#pragma unroll
            for (int i = 0; i < B; i += 4) {
                float4 four = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (c + i < experts && ROWS_IN_BOUNDS(status, row * pitch + c + i + 4 <= rows * pitch)) four = *reinterpret_cast<const float4*>(mine + c + i);
                part[i] = four.x; part[i + 1] = four.y; part[i + 2] = four.z; part[i + 3] = four.w;
            }
            if (!kChosen) {
#pragma unroll
                for (int i = 0; i < B; ++i) part[i] = __fmul_rn(p[i], __fsub_rn(part[i], mean));
            }
#pragma unroll
            for (int i = 0; i < B; i += M) {
                RowsVec<E, M> out;
                out.set(part + i);
                if (c + i < experts && ROWS_IN_BOUNDS(status, c + i + M <= experts)) rows_store_vec<E, M>(dlogits + t * ld_d + c + i, out);
            }
        };
        if constexpr (kChosen) {
            for (uint32_t c = from; c < experts && there; c += step) write(c, nullptr);
        } else {
#pragma unroll
            for (int n = 0; n < H / B; ++n)
                if (from + n * step < experts && there) write(from + n * step, held[n]);
        }
        __syncwarp();
        if (id >= 0) g[to] = 0.0f;                                        // (all zeros again)
    }
}

// Runs CALL(L, N): the lanes of a row and the logits of a lane for E experts, 9 at least (L * N >= E).
#define ROWS_WITH_SPREAD(E, CALL)                                               \
    do {                                                                        \
        if ((E) <= 16) { CALL(4, 4); }                                          \
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
    if (k <= 8) {
        // P choices; a lane has P .. 32 logits.  Few rows: fewer logits a lane, so that a row's way is shorter.
        const uint32_t bytes = rows_elem_bytes(dtype);
#define ROWS_GO(L, N, P)                                                                                                      \
    do {                                                                                                                      \
        const uint32_t rows = kRouteThreads / (L);                                                                            \
        const uint32_t access = (N) * bytes < 16 ? (N) * bytes : 16;                                                          \
        const uint32_t wide = (uintptr_t)logits % access == 0 && ld * bytes % access == 0 ? 1u : 0u;                          \
        rc = rows_launch(route_kernel<ROWS_T, L, N, P>, dim3((T + rows - 1) / rows), dim3(kRouteThreads), 0, s, 0, status, T, E, k, \
                         (const ROWS_T*)logits, ld, wide, over_chosen ? 1u : 0u, w, ids, make_uint2(1u, 0xFFFFFFFFu));                                     \
    } while (0)
#define ROWS_P(P)                                                                                                             \
    do {                                                                                                                      \
        if (E <= 8) ROWS_GO(1, 8, P);                                                                                         \
        else if (E <= 16) ROWS_GO(2, 8, P);                                                                                   \
        else if (E <= 32) ROWS_GO(2, 16, P);                                                                                  \
        else if (E <= 64) ROWS_GO(4, 16, P);                                                                                  \
        else if (E <= 128) ROWS_GO(4, 32, P);                                                                                 \
        else if (E <= 256) ROWS_GO(8, 32, P);                                                                                 \
        else if (E <= 512) ROWS_GO(16, 32, P);                                                                                \
        else ROWS_GO(32, 32, P);                                                                                              \
    } while (0)
#define ROWS_TYPE(X)                                                                                                          \
    do {                                                                                                                      \
        typedef X ROWS_T;                                                                                                     \
        if (k <= 2) ROWS_P(2); else if (k <= 4) ROWS_P(4); else ROWS_P(8);                                                    \
    } while (0)
        ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_TYPE
#undef ROWS_P
#undef ROWS_GO
        return rc;
    }
#define ROWS_GO(L, N)                                                                                                        \
    do {                                                                                                                     \
        const uint32_t rows = kThreads / (L);                                                                                \
        rc = rows_launch(rounds_kernel<ROWS_T, L, N>, dim3((T + rows - 1) / rows), dim3(kThreads), 0, s, 0, status, T, E, k, \
                         (const ROWS_T*)logits, ld, wide_rows<ROWS_T, N>(logits, ld) ? 1u : 0u, over_chosen ? 1u : 0u, w, ids); \
    } while (0)
#define ROWS_TYPE(X) do { typedef X ROWS_T; ROWS_WITH_SPREAD(E, ROWS_GO); } while (0)
    ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_TYPE
#undef ROWS_GO
    return rc;
}

int rows_launch_route_grad(unsigned* status, uint32_t T, uint32_t E, uint32_t k, uint32_t dtype, const void* logits, uint64_t ld,
                           bool over_chosen, const float* w, const int32_t* ids, const float* dw, void* dlogits, uint64_t ld_d,
                           cudaStream_t s)
{
    if (T == 0) return 0;
    uint32_t log_kl = 0;
    while (1u << log_kl < k) ++log_kl;
    uint32_t log_r = 5 - log_kl;
    while (log_r > 0 && ((E + 3) / 4 * 4) << log_r > kRowFloats) --log_r;
    const uint32_t bytes = rows_elem_bytes(dtype), rows = (kThreads / 32) << log_r;
    const size_t smem = (size_t)((E + 3) / 4 * 4) * rows * sizeof(float);                      // 32 KB at most
    const uint32_t most = rows_sm_count() * 8, blocks = (T + rows - 1) / rows;
    const dim3 grid(blocks < most ? blocks : most);
    const uint32_t granule = rows_granule((uint64_t)E * bytes, (uintptr_t)dlogits, ld_d * bytes, over_chosen ? 0 : (uintptr_t)logits,
                                          over_chosen ? 0 : ld * bytes);
    int rc = -1;
#define ROWS_GO(M, CHOSEN, H)                                                                                                  \
    rc = rows_launch(route_grad_kernel<ROWS_T, M, CHOSEN, H>, grid, dim3(kThreads), smem, s, 0, status, T, E, k, log_kl, log_r, \
                     (const ROWS_T*)logits, ld, w, ids, dw, (ROWS_T*)dlogits, ld_d)
#define ROWS_WIDTH(CHOSEN, H)                                                                                                  \
    do { if (granule >= 16) ROWS_GO(kWide, CHOSEN, H); else if (granule >= 8) ROWS_GO(kWide / 2, CHOSEN, H); else ROWS_GO(1, CHOSEN, H); } while (0)
#define ROWS_TYPE(X)                                                                                                           \
    do {                                                                                                                       \
        typedef X ROWS_T;                                                                                                      \
        constexpr int kWide = 16 / (int)sizeof(ROWS_T);                                                                        \
        if (over_chosen) ROWS_WIDTH(true, 16);                                                                                 \
        else if (E <= 16u << (5 - log_r)) ROWS_WIDTH(false, 16);                                                               \
        else ROWS_WIDTH(false, 32);                                                                                            \
    } while (0)
    ROWS_WITH_TYPE(dtype, ROWS_TYPE);
#undef ROWS_TYPE
#undef ROWS_WIDTH
#undef ROWS_GO
    return rc;
}
