// One step of a beam search: the choice over the beams and the vocabulary, and the move of the beams' states.
#include <cooperative_groups.h>

#include "rows_internal.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.402823466e+38f;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// ---- selection -------------------------------------------------------------------------------------------------------
// One thread-block cluster has a group.  A unit of work is a run of one beam's logits (the whole row, or a part of it where the
// cluster has more CTAs than the group has beams).  A unit is read once, through a ring of 16-byte slots in shared memory that
// each thread fills and reads by itself (no barrier, 128 KB in flight on an SM with 64 registers a thread):
//   statistics   a thread keeps a reference value, the sum of exp(x - reference), and the largest logits of its three best pairs
//                of accesses.  The reference moves only when a pair's sum becomes large (a binary32 sum has room), so a logit costs
//                one fused operation, one exponential, one addition -- the first and the last two logits at a time -- and half a
//                comparison;
//   the best C   in each of A warps the r-th largest of the lanes' largest logits, r = ceil(C / A), is reached by r logits, so the
//                smallest of these bounds is reached by C.  Only threads whose largest logit reaches it can have such logits; they
//                read their two best pairs again (from L2), and all their logits where the third-best pair reaches the bound, too.
//                What reaches the bound -- some three times C logits -- is sorted.
// Offers carry (logit, token) as one 64-bit key, all different, so nothing depends on the order threads arrive in.
// Each CTA sends its row sums and sorted lists into the shared memory of all CTAs of the cluster, which wait for the bytes of all
// (a mbarrier each); the rank of an offer among the group's is then the sum over the lists of how many entries precede it:
// searches by halving, one writer for each result.
// What bounds it.  64 groups of 8 beams over 131072 bfloat16 logits (121 MB, 18 us at the rate of a copy): 40 us.  Reading takes
// some 26 where four CTAs share an SM, 0.84 for 16 logits of each of its threads: 114 instructions a warp, half of what the SM can issue
// in that time, and 17 for the unit of the exponentials, two thirds of what that can.  The rest are some 1700 instructions a warp in a
// row, and nothing left to hide them behind, because all CTAs run at once.  4 rows of 32003 binary32 logits: 8.8 us, which are those
// instructions.  Tried and not kept: four accesses at a time (63 us: spilled), clusters of 16 CTAs for the large case (70 us against
// 48 then), the best pairs asked for again ahead of time (49 us against 48).
constexpr uint32_t kThreads = 256, kWarps = kThreads / 32;
constexpr uint32_t kRoom = 4096;                 // offers that are sorted
constexpr uint32_t kSlots = 8;                   // of the ring, per thread
constexpr uint32_t kMostCtas = 16;

// Keys that order like (larger logit, lower token); 0 stands for no offer.
__device__ __forceinline__ uint32_t rising(float x)
{
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.0f));            // (-0 becomes 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_rising(uint32_t r) { return __uint_as_float(r & 0x80000000u ? r ^ 0x80000000u : ~r); }
// The logit of a bound; -infinity for one below every finite logit's key.
__device__ __forceinline__ float logit_of_bound(uint64_t key)
{
    const uint32_t r = (uint32_t)(key >> 32);
    return r < 0x00800000u ? -kInf : from_rising(r);
}
__device__ __forceinline__ uint64_t key_of(float x, uint32_t token) { return ((uint64_t)rising(x) << 32) | (0xFFFFFFFFu - token); }
__device__ __forceinline__ uint64_t rising64(double x)
{
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double from_rising64(uint64_t r)
{
    return __longlong_as_double((long long)(r >> 63 ? r ^ 0x8000000000000000ull : ~r));
}

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// log(x), x >= 1, by Tang's table-driven method (1990): x = 2^e m, c near 1/m from a table of 32, r = m c - 1 (|r| <= 2^-6), log x =
// e log 2 - log c + log(1 + r); beyond r the series is below 2^-12 and runs in binary32.  Within 3e-11.  A few binary64 operations
// in a row where the library's logarithm is some twenty.
__device__ __constant__ const double kLogOf[32] = {
    0.015748356968139168, 0.045962135564635756, 0.07500982100486657, 0.10275973395776894,
    0.1313017372972535, 0.15839142994391764, 0.18388527877013736, 0.21004610480880948,
    0.23443755793296864, 0.2594388601383859, 0.2824872555746769, 0.30607943759149703,
    0.33024168687057687, 0.3522205935893521, 0.3746934494414107, 0.394780208008148,
    0.415278729556489, 0.43620624966244487, 0.4575811092471784, 0.47627324225933093,
    0.4953214372300254, 0.514739523087127, 0.5312143602906321, 0.5513492686996879,
    0.5684437020589881, 0.5858354447708572, 0.6035350218702582, 0.6215535273729365,
    0.6362058041598069, 0.6548283162578087, 0.6699801212784109, 0.6853650401178903,
};        // -log of the numbers below
__device__ __constant__ const float kNear[32] = {
    504.0f / 512, 489.0f / 512, 475.0f / 512, 462.0f / 512, 449.0f / 512, 437.0f / 512, 426.0f / 512, 415.0f / 512,
    405.0f / 512, 395.0f / 512, 386.0f / 512, 377.0f / 512, 368.0f / 512, 360.0f / 512, 352.0f / 512, 345.0f / 512,
    338.0f / 512, 331.0f / 512, 324.0f / 512, 318.0f / 512, 312.0f / 512, 306.0f / 512, 301.0f / 512, 295.0f / 512,
    290.0f / 512, 285.0f / 512, 280.0f / 512, 275.0f / 512, 271.0f / 512, 266.0f / 512, 262.0f / 512, 258.0f / 512,
};        // 1 / (1 + (i + 1/2) / 32) to 9 bits
__device__ __forceinline__ double log_of(double x)
{
    const uint64_t bits = (uint64_t)__double_as_longlong(x);
    const int e = (int)(bits >> 52) - 1023;
    const double m = __longlong_as_double((long long)((bits & 0x000FFFFFFFFFFFFFull) | 0x3FF0000000000000ull));
    const uint32_t i = (uint32_t)(bits >> 47) & 31u;
    const double r = fma(m, (double)kNear[i], -1.0);
    const float f = (float)r;
    const float tail = __fmul_rn(__fmul_rn(f, f), __fmaf_rn(f, __fmaf_rn(f, __fmaf_rn(f, 0.2f, -0.25f), 0.333333343f), -0.5f));
    return fma((double)e, 0.693147180559945309417, kLogOf[i]) + (r + (double)tail);
}

// What an access of 16 bytes holds: words of one or two logits.
template <typename E> struct Word;
template <> struct Word<float> {
    static constexpr uint32_t kMinusInf = 0xFF800000u;
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
    static __device__ __forceinline__ float largest(uint32_t a) { return __uint_as_float(a); }
    static __device__ __forceinline__ uint32_t bits_of(const float* p) { return __float_as_uint(*p); }
    static __device__ __forceinline__ float get(const uint32_t (&r)[4], int i) { return __uint_as_float(r[i]); }
    static __device__ __forceinline__ void set(uint32_t (&r)[4], int i, uint32_t bits) { r[i] = bits; }
};
// (i is known to the compiler: the words stay in registers)
__device__ __forceinline__ void set_half(uint32_t (&r)[4], int i, uint32_t bits)
{
    r[i / 2] = i % 2 ? (r[i / 2] & 0x0000FFFFu) | bits << 16 : (r[i / 2] & 0xFFFF0000u) | (bits & 0xFFFFu);
}
template <> struct Word<__half> {
    static constexpr uint32_t kMinusInf = 0xFC00FC00u;
    static __device__ __forceinline__ __half2 as(uint32_t a) { return *reinterpret_cast<const __half2*>(&a); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        const __half2 m = __hmax2(as(a), as(b));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float2 both(uint32_t a) { return __half22float2(as(a)); }
    static __device__ __forceinline__ float largest(uint32_t a) { const float2 f = both(a); return fmaxf(f.x, f.y); }
    static __device__ __forceinline__ uint32_t bits_of(const __half* p) { return __half_as_ushort(*p); }
    static __device__ __forceinline__ float get(const uint32_t (&r)[4], int i) { const float2 f = both(r[i / 2]); return i % 2 ? f.y : f.x; }
    static __device__ __forceinline__ void set(uint32_t (&r)[4], int i, uint32_t bits) { set_half(r, i, bits); }
};
template <> struct Word<__nv_bfloat16> {
    static constexpr uint32_t kMinusInf = 0xFF80FF80u;
    static __device__ __forceinline__ __nv_bfloat162 as(uint32_t a) { return *reinterpret_cast<const __nv_bfloat162*>(&a); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        const __nv_bfloat162 m = __hmax2(as(a), as(b));
        return *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float2 both(uint32_t a) { return make_float2(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u)); }
    static __device__ __forceinline__ float largest(uint32_t a) { const float2 f = both(a); return fmaxf(f.x, f.y); }
    static __device__ __forceinline__ uint32_t bits_of(const __nv_bfloat16* p) { return __bfloat16_as_ushort(*p); }
    static __device__ __forceinline__ float get(const uint32_t (&r)[4], int i) { const float2 f = both(r[i / 2]); return i % 2 ? f.y : f.x; }
    static __device__ __forceinline__ void set(uint32_t (&r)[4], int i, uint32_t bits) { set_half(r, i, bits); }
};

// A run of n logits.  Its accesses (N logits each, from logit v*N on) are counted from its start, not from a 16-byte boundary:
// what a thread adds up does not depend on where a row lies in memory.  Where the start is `off` bytes past a boundary, an
// access is the two 16-byte words that hold it, shifted together; those may hold logits of the rows beside this one, and stay
// within [the first row's start, the last row's end): an access that would leave that is read logit by logit.
// What the checked build knows of the array that a run is in.
struct Extent {
#ifdef PEARL_CHECKED
    const void *lo, *hi;
    unsigned* status;
    __device__ __forceinline__ bool holds(const void* p, uint32_t bytes) const { return ROWS_IN_ARRAY(status, p, bytes, lo, hi); }
    __device__ __forceinline__ void know(const void* from, const void* to, unsigned* word) { lo = from; hi = to; status = word; }
#else
    __device__ __forceinline__ bool holds(const void*, uint32_t) const { return true; }
    __device__ __forceinline__ void know(const void*, const void*, unsigned*) {}
#endif
};
template <typename E>
struct Run : Extent {
    static constexpr int N = 16 / (int)sizeof(E);
    const E* run;
    uint32_t n, off;
    uint32_t accesses, full;        // ceil and floor of n / N
    uint32_t from, upto;            // accesses from .. upto - 1 may be read as 16-byte words

    __device__ __forceinline__ Run(const E* start, uint32_t count, const E* all, const E* all_end, unsigned* status) : run(start), n(count)
    {
        know(all, all_end, status);
        off = (uint32_t)((uintptr_t)start & 15u);
        accesses = (n + N - 1) / N;
        full = n / N;
        from = (uintptr_t)start - off < (uintptr_t)all ? 1u : 0u;
        const uint64_t room = ((uintptr_t)all_end - ((uintptr_t)start - off)) / 16u;       // 16-byte words that may be read
        const uint64_t last = off ? (room ? room - 1 : 0) : room;
        upto = last < accesses ? (uint32_t)last : accesses;
    }
    __device__ __forceinline__ bool readable(uint32_t v) const { return v >= from && v < upto; }
    __device__ __forceinline__ const unsigned char* words(uint32_t v) const
    {
        return reinterpret_cast<const unsigned char*>(run) + (uint64_t)v * 16u - off;
    }
    // The access's logits in order, in lo, from the two words that hold it.
    static __device__ __forceinline__ void shift(uint32_t off, RowsRaw<16>& lo, RowsRaw<16>& hi)
    {
        if (off & 8u) { lo.r[0] = lo.r[2]; lo.r[1] = lo.r[3]; lo.r[2] = hi.r[0]; lo.r[3] = hi.r[1]; hi.r[0] = hi.r[2]; hi.r[1] = hi.r[3]; }
        if (off & 4u) { lo.r[0] = lo.r[1]; lo.r[1] = lo.r[2]; lo.r[2] = lo.r[3]; lo.r[3] = hi.r[0]; hi.r[0] = hi.r[1]; }
        if (sizeof(E) == 2 && (off & 2u)) {
            lo.r[0] = __funnelshift_r(lo.r[0], lo.r[1], 16);
            lo.r[1] = __funnelshift_r(lo.r[1], lo.r[2], 16);
            lo.r[2] = __funnelshift_r(lo.r[2], lo.r[3], 16);
            lo.r[3] = __funnelshift_r(lo.r[3], hi.r[0], 16);
        }
    }
    // An access at an end of the run, or behind it: -infinity where there is no logit.
    __device__ __forceinline__ void mend(uint32_t v, RowsRaw<16>& w) const
    {
        const bool there = readable(v);
        const uint32_t past = v < accesses ? n - v * N : 0u;
        if (past == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w.r[i] = Word<E>::kMinusInf;
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if ((uint32_t)i >= past) Word<E>::set(w.r, i, Word<E>::kMinusInf);
            else if (!there && holds(run + (uint64_t)v * N + i, sizeof(E))) Word<E>::set(w.r, i, Word<E>::bits_of(run + (uint64_t)v * N + i));
        }
    }
    __device__ __forceinline__ bool whole(uint32_t v) const { return readable(v) && v < full; }
};

// NaN and +infinity become -infinity; true if there were any.
template <typename E> __device__ __forceinline__ bool clean(RowsRaw<16>& w)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(E); ++i)
        if (!(Word<E>::get(w.r, i) < kInf)) { bad = true; Word<E>::set(w.r, i, Word<E>::kMinusInf); }
    return bad;
}
template <typename E> __device__ __forceinline__ float largest_of(const RowsRaw<16>& w)
{
    return Word<E>::largest(Word<E>::larger(Word<E>::larger(w.r[0], w.r[1]), Word<E>::larger(w.r[2], w.r[3])));
}
// Two binary32 values in a register pair: one instruction works on both.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi)
{
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ float2 both_of(uint64_t p)
{
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(p));
    return f;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b)
{
    uint64_t c;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(c) : "l"(a), "l"(b));
    return c;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// The sum of 2^(x log2e - c) over two accesses.  kPairs: two terms an instruction, with the same results (a third fewer instructions,
// and more registers).
template <bool kPairs, typename E> __device__ __forceinline__ float exp_sum(const RowsRaw<16>& a, const RowsRaw<16>& b, float c)
{
    constexpr int P = 8 / (int)sizeof(E);                  // pairs of an access
    if constexpr (kPairs) {
        const uint64_t scale = pair_of(kLog2e, kLog2e), minus_c = pair_of(-c, -c);
        uint64_t e[2 * P];
#pragma unroll
        for (int i = 0; i < 2 * P; ++i) {
            const RowsRaw<16>& w = i % 2 ? b : a;
            const float2 x = both_of(fma_pair(pair_of(Word<E>::get(w.r, i / 2 * 2), Word<E>::get(w.r, i / 2 * 2 + 1)), scale, minus_c));
            e[i] = pair_of(exp2_of(x.x), exp2_of(x.y));
        }
#pragma unroll
        for (int d = 1; d < 2 * P; d *= 2)
#pragma unroll
            for (int i = 0; i < 2 * P; i += 2 * d) e[i] = add_pair(e[i], e[i + d]);
        const float2 f = both_of(e[0]);
        return __fadd_rn(f.x, f.y);
    } else {
        float half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float e[2 * P];
#pragma unroll
            for (int i = 0; i < 2 * P; ++i) e[i] = exp2_of(__fmaf_rn(Word<E>::get((i % 2 ? b : a).r, i / 2 * 2 + h), kLog2e, -c));
#pragma unroll
            for (int d = 1; d < 2 * P; d *= 2)
#pragma unroll
                for (int i = 0; i < 2 * P; i += 2 * d) e[i] = __fadd_rn(e[i], e[i + d]);
            half[h] = e[0];
        }
        return __fadd_rn(half[0], half[1]);
    }
}
// The sum of exp(x - ref) over an access, for any ref.
template <typename E> __device__ __forceinline__ float exp_sum_of(const RowsRaw<16>& w, float ref)
{
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(E); ++i) sum = __fadd_rn(sum, exp2_of(__fmul_rn(__fsub_rn(Word<E>::get(w.r, i), ref), kLog2e)));
    return sum;
}

// What a thread knows of its part of a run.  Its accesses are taken in pairs.  (Four at a time need a quarter fewer instructions, and
// more than the 64 registers that let four CTAs share an SM.)
struct Stats {
    double sum;                     // of exp(x - ref)
    float ref;                      // (while the run is read: c, see below)
    float best, second, third;      // the largest logits of the three pairs that have the largest
    uint32_t best_at, second_at;    // the first accesses of the two best pairs
    bool bad;
};
// While a run is read the sum is of 2^(x log2e - c), c = ref log2e rounded: one fused operation a logit, and every term off by the same
// factor, which is put right at the end.  (A difference first and then a product: 48 us instead of 40 at the size named above, the packed
// operations and the loop without branches included.)  That is good for |ref| <= kFar, where the factor is near 1.  A thread's c starts at
// that of -kFar; a logit above kFar makes it infinity, and no term counts from there on.  Where that leaves no sum -- no logit of the run is
// far above -kFar, or a thread has one above kFar -- far_sum() takes it from the logits once more.
constexpr float kFar = 1048576.0f;
constexpr float kMost = 3000.0f;    // a pair whose sum is larger moves the reference to its largest logit
template <typename E> __device__ __forceinline__ float largest_of(const RowsRaw<16>& a, const RowsRaw<16>& b)
{
    return Word<E>::largest(Word<E>::larger(Word<E>::larger(Word<E>::larger(a.r[0], a.r[1]), Word<E>::larger(a.r[2], a.r[3])),
                                            Word<E>::larger(Word<E>::larger(b.r[0], b.r[1]), Word<E>::larger(b.r[2], b.r[3]))));
}
// Pair p, whose largest logit is `top`, with its sum.
__device__ __forceinline__ void add(Stats& s, float top, float sum, uint32_t p)
{
    s.sum += (double)sum;
    s.third = fmaxf(s.third, fminf(s.second, top));
    if (top > s.best) {
        s.second_at = s.best_at;
        s.best_at = p;
    } else if (top > s.second) {
        s.second_at = p;
    }
    s.second = fmaxf(s.second, fminf(s.best, top));
    s.best = fmaxf(s.best, top);
}
// Any pair p.
template <typename E> __device__ __forceinline__ void take(Stats& s, RowsRaw<16>& a, RowsRaw<16>& b, uint32_t p)
{
    float top = 0.0f, sum = 0.0f;
#pragma unroll 1
    for (uint32_t tries = 0; tries < 4; ++tries) {           // (moved, cleaned of NaN and infinity, moved)
        top = largest_of<E>(a, b);
        sum = exp_sum<false, E>(a, b, s.ref);
        if (sum <= kMost) break;                             // (a NaN among the logits makes the sum one)
        const float to = top <= kFar ? __fmul_rn(top, kLog2e) : kInf;
        if (top < kInf && to > s.ref) {
            s.sum *= (double)exp2_of(__fsub_rn(s.ref, to));
            s.ref = to;
        } else {
            s.bad |= clean<E>(a);
            s.bad |= clean<E>(b);
        }
    }
    add(s, top, sum, p);
}

__device__ __forceinline__ void copy_16(const Extent& in, uint32_t to, const unsigned char* from)
{
    if (!in.holds(from, 16)) return;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ RowsRaw<16> ring_word(uint32_t at)
{
    RowsRaw<16> w;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.r[0]), "=r"(w.r[1]), "=r"(w.r[2]), "=r"(w.r[3]) : "r"(at) : "memory");
    return w;
}

// The sum of exp(x - best) over a thread's accesses of a run, read once more.
template <typename E>
__device__ __noinline__ double far_sum(const Run<E> r, float best)
{
    double sum = 0.0;
    if (best == -kInf) return sum;
#pragma unroll 1
    for (uint32_t v = threadIdx.x; v < r.accesses; v += kThreads) {
        RowsRaw<16> w, hi;
        rows_load_if<false>(r.readable(v) && r.holds(r.words(v), r.off ? 32 : 16), w, r.words(v));
        if (r.off) {
            rows_load_if<false>(r.readable(v) && r.holds(r.words(v), 32), hi, r.words(v) + 16);
            Run<E>::shift(r.off, w, hi);
        }
        if (!r.whole(v)) r.mend(v, w);
        clean<E>(w);
        sum += (double)exp_sum_of<E>(w, best);
    }
    return sum;
}

// A thread's way through a run: pair p is accesses tid + 2p * kThreads and the next one.  kDepth pairs are in the ring at a time;
// `ring` is the shared address of the thread's slot 0, slots are kThreads * 16 bytes apart.  Two accesses are added up at a time
// however the run lies in memory, so that equal rows have equal sums.
template <bool kShifted, typename E>
struct Stream {
    static constexpr uint32_t kWords = kShifted ? 2u : 1u, kDepth = kSlots / 2 / kWords, kStep = kWords * kThreads * 16u;
    static constexpr uint32_t kPairBytes = 2u * kThreads * 16u;
    static __device__ __forceinline__ uint32_t pairs(const Run<E>& r) { return (r.accesses + 2 * kThreads - 1) / (2 * kThreads); }
    // Pairs from .. plain() - 1 are whole accesses for every thread of the block.
    static __device__ __forceinline__ uint32_t plain(const Run<E>& r) { return (r.upto < r.full ? r.upto : r.full) / (2 * kThreads); }
    // Pair p, whose first word is at `at`, on its way into the ring (in a group of copies of its own, which may be empty).
    static __device__ __forceinline__ void issue(const Run<E>& r, uint32_t slot, uint32_t p, const unsigned char* at, bool both)
    {
#pragma unroll
        for (uint32_t i = 0; i < 2; ++i) {
            if (both || r.readable(threadIdx.x + (2 * p + i) * kThreads)) {
                copy_16(r, slot + i * kStep, at + i * kThreads * 16u);
                if (kShifted) copy_16(r, slot + i * kStep + kThreads * 16u, at + i * kThreads * 16u + 16);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    static __device__ __forceinline__ void start(const Run<E>& r, uint32_t ring)
    {
        const unsigned char* at = r.words(threadIdx.x);
#pragma unroll 1
        for (uint32_t p = 0; p < kDepth; ++p) issue(r, ring + p * 2 * kStep, p, at + p * kPairBytes, p >= r.from && p < plain(r));
    }
    static __device__ __forceinline__ void finish() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
    // The oldest pair in the ring.
    static __device__ __forceinline__ void read(uint32_t slot, uint32_t off, RowsRaw<16>& a, RowsRaw<16>& b)
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        a = ring_word(slot);
        b = ring_word(slot + kStep);
        if (kShifted) {
            RowsRaw<16> a_hi = ring_word(slot + kThreads * 16u), b_hi = ring_word(slot + kStep + kThreads * 16u);
            Run<E>::shift(off, a, a_hi);
            Run<E>::shift(off, b, b_hi);
        }
    }
    // The reference that take() gives a thread by its first pair; -kFar if that pair is out of the ordinary.
    static __device__ __forceinline__ float first_reference(uint32_t ring, uint32_t off)
    {
        RowsRaw<16> a, b;
        read(ring, off, a, b);
        const float top = largest_of<E>(a, b);
        return __fmul_rn(top > 16.0f - kFar && top <= kFar ? top : -kFar, kLog2e);
    }
    // Pairs from p on, all whole, up to `end` or to one that take() has to look at for a lane of the warp; p becomes the next pair.
    // (Accesses first .. first + span - 1 may be read as 16-byte words.)
    static __device__ __forceinline__ Stats whole_pairs(const Extent in, const unsigned char* at, uint32_t off, uint32_t first, uint32_t span, uint32_t ring, uint32_t& p,
                                                        uint32_t end, Stats s)
    {
        const uint32_t last = ring + (kDepth - 1) * 2 * kStep;
        uint32_t slot = ring + p % kDepth * 2 * kStep, v = threadIdx.x + 2 * (p + kDepth) * kThreads - first, q = p;
        at += (uint64_t)(p + kDepth) * kPairBytes;
#pragma unroll 1
        for (; q < end; ++q) {
            RowsRaw<16> a, b;
            read(slot, off, a, b);
            const float sum = exp_sum<true, E>(a, b, s.ref);
            if (__any_sync(0xFFFFFFFFu, !(sum <= kMost))) break;
            add(s, largest_of<E>(a, b), sum, q);
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)                               // (into the slots that have just been read)
                if (v + i * kThreads < span) {
                    copy_16(in, slot + i * kStep, at + i * kThreads * 16u);
                    if (kShifted) copy_16(in, slot + i * kStep + kThreads * 16u, at + i * kThreads * 16u + 16);
                }
            asm volatile("cp.async.commit_group;" ::: "memory");
            v += 2 * kThreads;
            at += kPairBytes;
            slot = slot == last ? ring : slot + 2 * kStep;
        }
        p = q;
        return s;
    }
    // Pairs p .. end - 1, of any kind.
    static __device__ __forceinline__ Stats any_pairs(const Run<E>& r, uint32_t ring, uint32_t p, uint32_t end, Stats s)
    {
        const unsigned char* at = r.words(threadIdx.x) + (uint64_t)(p + kDepth) * kPairBytes;
#pragma unroll 1
        for (; p < end; ++p) {
            const uint32_t slot = ring + p % kDepth * 2 * kStep, v = threadIdx.x + 2 * p * kThreads;
            RowsRaw<16> a, b;
            read(slot, r.off, a, b);
            if (!r.whole(v)) r.mend(v, a);
            if (!r.whole(v + kThreads)) r.mend(v + kThreads, b);
            take<E>(s, a, b, p);
            issue(r, slot, p + kDepth, at, false);
            at += kPairBytes;
        }
        return s;
    }
    static __device__ __noinline__ Stats whole_call(const Extent in, const unsigned char* at, uint32_t off, uint32_t first, uint32_t span, uint32_t ring, uint32_t& p,
                                                    uint32_t end, Stats s)
    {
        return whole_pairs(in, at, off, first, span, ring, p, end, s);
    }
    static __device__ __noinline__ Stats any_call(const Run<E> r, uint32_t ring, uint32_t p, uint32_t end, Stats s) { return any_pairs(r, ring, p, end, s); }

    template <bool kCalls> static __device__ __forceinline__ Stats walk(const Run<E>& r, uint32_t ring)
    {
        Stats s{0.0, -kFar * kLog2e, -kInf, -kInf, -kInf, 0u, 0u, false};
        const uint32_t all = pairs(r), whole = plain(r), first = kShifted ? r.from : 0u;
        constexpr uint32_t kLeast = kCalls ? kLong : 1u;                   // whole pairs that are worth a call
        if (whole && !first) s.ref = first_reference(ring, r.off);
        uint32_t p = 0;
#pragma unroll 1
        while (p < all) {
            if (p >= first && p + kLeast <= whole) {
                if constexpr (kCalls) s = whole_call(r, r.words(threadIdx.x), r.off, first, r.upto - first, ring, p, whole, s);
                else s = whole_pairs(r, r.words(threadIdx.x), r.off, first, r.upto - first, ring, p, whole, s);
            }
            if (p >= all) break;
            const uint32_t to = p + kLeast <= whole ? p + 1 : all;
            if constexpr (kCalls) s = any_call(r, ring, p, to, s);
            else s = any_pairs(r, ring, p, to, s);
            p = to;
        }
        finish();
        s.best_at = threadIdx.x + 2 * kThreads * s.best_at;
        s.second_at = threadIdx.x + 2 * kThreads * s.second_at;
        const float c = s.ref;
        if (!__syncthreads_or(c > (4.0f - kFar) * kLog2e) || c == kInf) {
            s.ref = kInf;                                                  // (for far_sum)
        } else {
            // c = ref log2e + off: the sum is 2^off too small
            s.ref = __fmul_rn(c, kLn2);
            const float off = __fmul_rn(__fmaf_rn(-s.ref, kLog2e, c), kLn2);
            const float more = __fmaf_rn(__fmul_rn(off, off), __fmaf_rn(off, 0.166666667f, 0.5f), off);       // e^off - 1, |off| < 0.1
            s.sum = fma(s.sum, (double)more, s.sum);
        }
        return s;
    }
    // Long runs call a function for the loop, because inlined the registers of what follows in the kernel are spilled inside it (42 us
    // instead of 40); short ones are a function as a whole, whose way is shorter (8.8 us for 4 rows of 32003 instead of 9.1).  From 9
    // whole pairs on a run is long: of 3, 5, 9, 17 and 33, 3 makes those rows long (9.1), and the others are within 3 % of one another from 64 x 8 rows
    // of 10000 logits to 131072.
    static constexpr uint32_t kLong = 9;
    static __device__ __noinline__ Stats short_run(const Run<E> r, uint32_t ring) { return walk<false>(r, ring); }
    static __device__ __forceinline__ Stats run(const Run<E>& r, uint32_t ring) { return plain(r) < kLong ? short_run(r, ring) : walk<true>(r, ring); }
};

// The logits of the pair of accesses that `access` is one of that reach the bound, appended to `offers`.
template <typename E>
__device__ __noinline__ void collect(const Run<E> r, uint32_t access, uint64_t at_least, uint32_t first, uint64_t* offers, uint32_t* n_offers)
{
    constexpr int N = Run<E>::N;
    access -= access / kThreads % 2u * kThreads;
    RowsRaw<16> w[2], hi[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const unsigned char* at = r.words(access + m * kThreads);
        const bool there = r.readable(access + m * kThreads) && r.holds(at, r.off ? 32 : 16);
        rows_load_if<false>(there, w[m], at);
        if (r.off) rows_load_if<false>(there, hi[m], at + 16);
    }
    // (no branch a logit: a few cycles each instead of some hundred)
    const float low = logit_of_bound(at_least), above = low > -kInf ? from_rising((uint32_t)(at_least >> 32) + 1u) : kLowest;
    const uint32_t last = 0xFFFFFFFFu - (uint32_t)at_least;               // of equal logits those up to this token, and some after it
    uint32_t reach = 0;                                                   // bit m * N + j: logit j of access m reaches the bound
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        if (r.off) Run<E>::shift(r.off, w[m], hi[m]);
        if (!r.whole(access + m * kThreads)) r.mend(access + m * kThreads, w[m]);
        const float least = low > -kInf && first + (access + m * kThreads) * N <= last ? low : above;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float x = Word<E>::get(w[m].r, j);
            if ((x >= least) & (x < kInf)) reach |= 1u << (m * N + j);
        }
    }
    uint32_t to = reach ? atomicAdd(n_offers, (uint32_t)__popc(reach)) : 0u;
    for (; reach; reach &= reach - 1u) {
        const uint32_t at = __ffs(reach) - 1u;
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at / (N / 4) == (uint32_t)i) word = w[i / 4].r[i % 4];
        float x;
        if constexpr (N == 4) x = __uint_as_float(word);
        else { const float2 f = Word<E>::both(word); x = at & 1u ? f.y : f.x; }
        if (to < kRoom) offers[to] = key_of(x, first + (access + at / N * kThreads) * N + at % N);
        ++to;
    }
}

// What the CTAs of a cluster tell one another of a unit.
struct UnitSum {
    double sum;
    float ref;
    uint32_t offers;
};

// A transfer into the shared memory of CTA `rank`: value to where this CTA has `to`, counted by that CTA's barrier.
__device__ __forceinline__ uint32_t in_cta(uint32_t at, uint32_t rank)
{
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    return there;
}
__device__ __forceinline__ void send(uint32_t to, uint32_t barrier, uint32_t rank, uint64_t value)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];"
                 ::"r"(in_cta(to, rank)), "l"(value), "r"(in_cta(barrier, rank)) : "memory");
}
__device__ __forceinline__ void send(uint32_t to, uint32_t barrier, uint32_t rank, const UnitSum& s)
{
    const uint64_t ref_offers = (uint64_t)__float_as_uint(s.ref) | (uint64_t)s.offers << 32;
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];"
                 ::"r"(in_cta(to, rank)), "l"((uint64_t)__double_as_longlong(s.sum)), "l"(ref_offers), "r"(in_cta(barrier, rank)) : "memory");
}
// Waits until all of them are here, for `polls` looks at most; the barrier's one phase.  Every CTA of the cluster sends a fixed number of
// bytes, so this ends; but a CTA whose rows have to be searched again and again may be far behind, and a CTA that left before its
// lists are here would leave them without a place to go.  So after kPolls looks the cluster's barrier is waited for, at which a CTA
// arrives once it has sent everything.  (Checked build: at once, so that this way is taken.)  Should they not be here then, PEARL_ST_INTERNAL
// tells of it, and the group's results are missing.
#ifdef PEARL_CHECKED
constexpr uint32_t kPolls = 0;
#else
constexpr uint32_t kPolls = 1u << 22;
#endif
constexpr uint32_t kLastPolls = 1u << 22;
__device__ __forceinline__ bool arrived(uint32_t barrier, uint32_t polls)
{
    for (uint32_t i = 0; i < polls; ++i) {
        uint32_t ok;
        asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0; selp.u32 %0, 1, 0, p; }"
                     : "=r"(ok) : "r"(barrier) : "memory");
        if (ok) return true;
    }
    return false;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
// (without an order on memory: what has been sent is counted by the receiver's barrier)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// The entries of a falling list of n that are larger than `bar`; `top` is the largest power of two up to n.
__device__ __forceinline__ uint32_t larger_than(const uint64_t* list, uint32_t n, uint32_t top, uint64_t bar)
{
    uint32_t at = 0;
    for (uint32_t step = top; step > 0; step >>= 1) {
        const uint32_t next = at + step;
        if (next <= n && list[next - 1] > bar) at = next;
    }
    return at;
}

struct SelectArgs {
    unsigned* status;
    uint32_t G, W, V, C;
    uint32_t parts;             // runs a row is cut into
    uint32_t run;               // logits of a run (a multiple of 8)
    uint32_t units_per_cta;
    uint32_t by_parts, by_C;    // 2^16 / parts and 2^20 / C, rounded up: (x * by_parts) >> 16 and (x * by_C) >> 20 divide what is divided here
    const void* logits;
    uint64_t ld;
    const float* scores;
    const uint8_t* done;
    int32_t end_token;
    float* best_score;
    int32_t* best_beam;
    int32_t* best_token;
};

// Dynamic shared memory: all_keys[units][C], which every CTA of the cluster writes its lists to, and a workspace that is the ring,
// then the offers to be sorted (kRoom), then all_totals[units][C].
template <typename E>
__global__ void __launch_bounds__(kThreads, 4) select_kernel(const SelectArgs a)
{
    extern __shared__ __align__(16) unsigned char shared[];
    __shared__ uint64_t barrier;
    __shared__ __align__(16) UnitSum all_sums[PEARL_ROWS_MAX_BEAMS];
    __shared__ uint64_t warp_bound[kWarps];
    __shared__ uint64_t warp_sum[kWarps];
    __shared__ float warp_ref[kWarps];
    __shared__ uint2 deep[kThreads];
    __shared__ uint32_t n_deep, n_offers, n_all;
    __shared__ float score_of[PEARL_ROWS_MAX_BEAMS];
    __shared__ uint8_t done_of[PEARL_ROWS_MAX_BEAMS];
    __shared__ double lse[PEARL_ROWS_MAX_BEAMS];
    constexpr int N = Run<E>::N;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ctas = cluster.num_blocks(), cta = cluster.block_rank(), g = blockIdx.x / ctas;
    const uint32_t units = a.W * a.parts, C = a.C, tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    uint64_t* all_keys = reinterpret_cast<uint64_t*>(shared);
    uint64_t* work = all_keys + (units * C + 1) / 2 * 2;
    const uint32_t keys_at = (uint32_t)__cvta_generic_to_shared(all_keys), sums_at = (uint32_t)__cvta_generic_to_shared(all_sums);
    const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&barrier), ring = (uint32_t)__cvta_generic_to_shared(work) + tid * 16u;
    if (tid == 0) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(units * (C * 8u + (uint32_t)sizeof(UnitSum))) : "memory");
        n_all = 0;
    }
    __syncwarp();
    cluster_arrive();
    rows_begin();

    const E* all = reinterpret_cast<const E*>(a.logits);
    const E* all_end = all + ((uint64_t)a.G * a.W - 1) * a.ld + a.V;
    for (uint32_t q = 0; q < a.units_per_cta; ++q) {
        const uint32_t u = cta * a.units_per_cta + q;
        const uint32_t b = u < units ? (u * a.by_parts) >> 16 : 0u, part = u < units ? u - b * a.parts : 0u;
        const uint64_t first = (uint64_t)part * a.run;
        const bool any = u < units && first < a.V;
        const Run<E> r(all + ((uint64_t)g * a.W + b) * a.ld + (any ? first : 0), any ? (uint32_t)(a.V - first < a.run ? a.V - first : a.run) : 0u, all,
                       all_end, a.status);
        if (r.off) Stream<true, E>::start(r, ring);
        else Stream<false, E>::start(r, ring);
        if (q == 0) {
            // (the first logits are on their way while the scores are read)
            if (tid < a.W) {
                const uint64_t row = (uint64_t)g * a.W + tid;
                float score = a.scores[row];
                done_of[tid] = a.done != nullptr && a.done[row] != 0;
                if (!(score < kInf)) {
                    if (cta == 0) atomicOr(a.status, PEARL_ST_BAD_SCORE);
                    score = -kInf;
                }
                score_of[tid] = score;
            }
            __syncwarp();
            cluster_wait();                                                           // the others' barriers may be used from here on
            __syncthreads();
        }
        if (u >= units) {
            Stream<false, E>::finish();
            break;
        }
        const uint32_t mine = keys_at + u * C * 8u;
        if (score_of[b] == -kInf || done_of[b] || !any) {
            // the logits do not matter; a finished beam has one offer, whose key only has to be valid
            Stream<false, E>::finish();
            const uint32_t n = done_of[b] && score_of[b] > -kInf && part == 0 ? 1u : 0u;
            for (uint32_t i = tid; i < C * ctas; i += kThreads) {
                const uint32_t c = (i * a.by_C) >> 20, at = i - c * C;
                send(mine + at * 8u, bar, c, at < n ? key_of(0.0f, 0u) : 0ull);
            }
            if (tid < ctas) send(sums_at + u * (uint32_t)sizeof(UnitSum), bar, tid, UnitSum{0.0, kLowest, n});
            continue;
        }
        Stats s = r.off ? Stream<true, E>::run(r, ring) : Stream<false, E>::run(r, ring);
        if (s.ref == kInf) {
            s.sum = far_sum<E>(r, s.best);
            s.ref = fmaxf(s.best, kLowest);
        }
        if (s.bad) atomicOr(a.status, PEARL_ST_BAD_SCORE);

        // a bound that C logits reach: the smallest key that the logit of its pair can have stands for it
        const uint64_t key = s.best == -kInf ? 0ull : key_of(s.best, (uint32_t)first + (s.best_at + kThreads) * N + N - 1);
        const uint32_t full_warps = r.accesses / 32u;
        const uint32_t active = full_warps < 1u ? 1u : full_warps < kWarps ? full_warps : kWarps;
        const uint32_t need = (C + active - 1) / active;
        uint64_t mark = ~0ull;
        if (warp < active) {
            uint32_t left = (uint32_t)(key >> 32), top = 0, had = 0;
            do {
                top = __reduce_max_sync(0xFFFFFFFFu, left);
                had += __popc(__ballot_sync(0xFFFFFFFFu, left == top));
                if (had < need && left == top) left = 0;
            } while (had < need && top);
            const uint32_t low = __reduce_min_sync(0xFFFFFFFFu, (uint32_t)(key >> 32) == top ? (uint32_t)key : 0xFFFFFFFFu);
            mark = top ? ((uint64_t)top << 32) | low : 1ull;                 // (too few lanes have a logit: every logit is an offer)
        }
        // the warp's sum relative to its largest reference, in fixed point (30 bits behind the point: the sum is near 1 at least if
        // there is a logit, and 2^60 of these at most): whole numbers add up in any order, three limbs of 22 bits at a time
        {
            const float ref = from_rising(__reduce_max_sync(0xFFFFFFFFu, rising(s.ref)));
            const double scaled = s.sum * (double)exp2_of(__fmul_rn(__fsub_rn(s.ref, ref), kLog2e));
            const uint64_t fixed = (uint64_t)__double2ull_rn(scaled * 1073741824.0);
            const uint64_t sum = (uint64_t)__reduce_add_sync(0xFFFFFFFFu, (uint32_t)fixed & 0x3FFFFFu) +
                                 ((uint64_t)__reduce_add_sync(0xFFFFFFFFu, (uint32_t)(fixed >> 22) & 0x3FFFFFu) << 22) +
                                 ((uint64_t)__reduce_add_sync(0xFFFFFFFFu, (uint32_t)(fixed >> 44)) << 44);
            if (lane == 0) { warp_bound[warp] = mark; warp_sum[warp] = sum; warp_ref[warp] = ref; }
        }
        if (tid == 0) { n_deep = 0; n_offers = 0; }
        __syncthreads();
        uint64_t lowest = warp_bound[0];
#pragma unroll
        for (uint32_t i = 1; i < kWarps; ++i) lowest = warp_bound[i] < lowest ? warp_bound[i] : lowest;

        // The logits that reach the bound.  Should they be more than there is room for, the bound is searched by halving (`low`: too
        // many reach it, `high`: fewer than C do; the keys are all different, so some key has a number between).
        uint64_t low = lowest, high = ~0ull, at_least = lowest;
        for (uint32_t tries = 0;; ++tries) {
            const float low_logit = logit_of_bound(at_least);
            if (s.best > -kInf && s.best >= low_logit) {
                collect<E>(r, s.best_at, at_least, (uint32_t)first, work, &n_offers);
                if (s.second > -kInf && s.second >= low_logit) collect<E>(r, s.second_at, at_least, (uint32_t)first, work, &n_offers);
                if (s.third > -kInf && s.third >= low_logit) {
                    const uint32_t to = atomicAdd(&n_deep, 1u);
                    if (ROWS_IN_BOUNDS(a.status, to < kThreads)) deep[to] = make_uint2(s.best_at, s.second_at);
                }
            }
            __syncthreads();
            const uint32_t a_thread = Stream<false, E>::pairs(r), all_deep = n_deep * a_thread;
            for (uint32_t i = tid; i < all_deep; i += kThreads) {
                const uint2 d = deep[i / a_thread];
                const uint32_t p = i % a_thread;
                if (p != d.x / (2 * kThreads) && p != d.y / (2 * kThreads))
                    collect<E>(r, d.x % kThreads + 2 * p * kThreads, at_least, (uint32_t)first, work, &n_offers);
            }
            __syncthreads();
            const uint32_t n = n_offers;
            if (n <= kRoom && (n >= C || at_least == lowest)) break;
            if (tries == 80) {                                             // (64 halvings are enough)
                if (tid == 0) atomicOr(a.status, PEARL_ST_INTERNAL);
                break;
            }
            if (n > kRoom) low = at_least;
            else high = at_least;
            at_least = low + (high - low) / 2;
            __syncthreads();
            if (tid == 0) { n_deep = 0; n_offers = 0; }
            __syncthreads();
        }
        const uint32_t n = n_offers < kRoom ? n_offers : kRoom;
        if (warp == kWarps - 1) {
            // the unit's sum, relative to the largest reference, added in a fixed order
            const float mine_ref = lane < kWarps ? warp_ref[lane] : kLowest;
            const float ref = from_rising(__reduce_max_sync(0xFFFFFFFFu, rising(mine_ref)));
            double sum = lane < kWarps ? (double)warp_sum[lane] * (1.0 / 1073741824.0) * (double)exp2_of(__fmul_rn(__fsub_rn(mine_ref, ref), kLog2e)) : 0.0;
#pragma unroll
            for (uint32_t d = 1; d < kWarps; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            sum = __shfl_sync(0xFFFFFFFFu, sum, 0);
            if (lane < ctas) send(sums_at + u * (uint32_t)sizeof(UnitSum), bar, lane, UnitSum{sum, ref, n < C ? n : C});
        }
        for (uint32_t i = n + tid; i < C; i += kThreads)
            for (uint32_t c = 0; c < ctas; ++c) send(mine + i * 8u, bar, c, 0ull);
        if (n <= kThreads) {
            // 2^shift lanes count the offers ahead of one, and hand it to the CTAs
            uint32_t shift = 5;
            while (n << shift > kThreads) --shift;
            const uint32_t each = 1u << shift, i = tid >> shift, sub = tid & (each - 1);
            const uint64_t k = i < n ? work[i] : 0ull;
            uint32_t ahead = 0;
#pragma unroll 4
            for (uint32_t o = sub; o < n; o += each) ahead += work[o] > k;
            for (uint32_t d = 1; d < each; d *= 2) ahead += __shfl_xor_sync(0xFFFFFFFFu, ahead, d);
            if (i < n && ahead < C && ROWS_IN_BOUNDS(a.status, u * C + ahead < units * C))
                for (uint32_t c = sub; c < ctas; c += each) send(mine + ahead * 8u, bar, c, k);
        } else {
            uint32_t size = kThreads;
            while (size < n) size *= 2;
            for (uint32_t i = n + tid; i < size; i += kThreads) work[i] = 0ull;
            for (uint32_t span = 2; span <= size; span *= 2)
                for (uint32_t step = span / 2; step > 0; step /= 2) {
                    __syncthreads();
                    for (uint32_t i = tid; i < size / 2; i += kThreads) {
                        const uint32_t x = (i & ~(step - 1)) * 2 + (i & (step - 1)), y = x + step;
                        const uint64_t p = work[x], o = work[y];
                        if ((p < o) == ((x & span) == 0)) { work[x] = o; work[y] = p; }
                    }
                }
            __syncthreads();
            for (uint32_t i = tid; i < C * ctas; i += kThreads) {
                const uint32_t c = (i * a.by_C) >> 20, at = i - c * C;
                send(mine + at * 8u, bar, c, work[at]);
            }
        }
        if (q + 1 < a.units_per_cta) __syncthreads();                      // (the next unit uses the same workspace)
    }
    __syncwarp();
    cluster_arrive_relaxed();                                              // (this CTA has sent everything)
    const bool late = __syncthreads_or(!arrived(bar, kPolls)) != 0;
    if (late) {
        cluster_wait();
        if (!arrived(bar, kLastPolls)) atomicOr(a.status, PEARL_ST_INTERNAL);
        __syncthreads();
    }

    if (tid < a.W) {
        float ref = kLowest;
        uint32_t offers = 0;
        for (uint32_t i = 0; i < a.parts; ++i) ref = fmaxf(ref, all_sums[tid * a.parts + i].ref);
        double sum = 0.0;
        for (uint32_t i = 0; i < a.parts; ++i) {
            const UnitSum& p = all_sums[tid * a.parts + i];
            sum += p.sum * (double)exp2_of(__fmul_rn(__fsub_rn(p.ref, ref), kLog2e));
            offers += p.offers;
        }
        lse[tid] = (double)ref + log_of(sum);
        atomicAdd(&n_all, offers);
    }
    __syncthreads();
    uint64_t* all_totals = work;
    for (uint32_t i = tid; i < units * C; i += kThreads) {
        const uint32_t b = (((i * a.by_C) >> 20) * a.by_parts) >> 16;
        const uint64_t k = all_keys[i];
        const double score = (double)score_of[b];
        all_totals[i] = k == 0 ? 0ull : rising64(done_of[b] ? score : score + ((double)from_rising((uint32_t)(k >> 32)) - lse[b]));
    }
    __syncthreads();

    // the place of each offer of this CTA's units: 2^shift lanes share the lists that may hold offers before it
    uint32_t shift = 5;
    while (shift > 0 && C << shift > kThreads) --shift;
    const uint32_t each = 1u << shift, sub = tid & (each - 1), top = 1u << (31 - __clz(C));
    for (uint32_t q = 0; q < a.units_per_cta; ++q) {
        const uint32_t u = cta * a.units_per_cta + q, b = (u * a.by_parts) >> 16, rows_from = b * a.parts, rows_to = rows_from + a.parts;
        if (u >= units) break;
        const uint64_t* mine = all_keys + u * C;
        for (uint32_t i0 = 0; i0 < C; i0 += kThreads >> shift) {
            const uint32_t i = i0 + (tid >> shift);
            const uint64_t key = i < C ? mine[i] : 0ull, total = i < C ? all_totals[u * C + i] : 0ull;
            uint32_t place = 0;
            if (key)
                for (uint32_t o = sub; o < units; o += each) {
                    // (runs of the same row by their logits and tokens, which are all different; other rows by the sums, equal ones
                    // of lower beams first)
                    const bool same = o >= rows_from && o < rows_to;
                    place += larger_than((same ? all_keys : all_totals) + o * C, C, top, same ? key : total - (o < u ? 1u : 0u));
                }
            for (uint32_t d = 1; d < each; d *= 2) place += __shfl_xor_sync(0xFFFFFFFFu, place, d);
            const uint32_t token = 0xFFFFFFFFu - (uint32_t)key;
            if (key && sub == 0 && place < C && ROWS_IN_BOUNDS(a.status, b < a.W && (done_of[b] || token < a.V))) {
                const uint64_t to = (uint64_t)g * C + place;
                a.best_score[to] = (float)from_rising64(total);
                a.best_beam[to] = (int32_t)b;
                a.best_token[to] = done_of[b] ? a.end_token : (int32_t)token;
            }
        }
    }
    if (cta == 0)
        for (uint32_t i = n_all + tid; i < C; i += kThreads) {
            const uint64_t to = (uint64_t)g * C + i;
            a.best_score[to] = -kInf;
            a.best_beam[to] = -1;
            a.best_token[to] = -1;
        }
    __syncwarp();
    if (!late) cluster_wait();                                             // (long past, where all lists are here)
}

// ---- the states ------------------------------------------------------------------------------------------------------
// state[o, g, i] <- state[o, g, parent[g, i]].  A thread has one access's worth of all W states of a block and group: it reads
// what the moved states need, all at once (a state with several children comes from a cache the second time), then writes.  No other
// thread touches those bytes, so the move can be made in place.  1 GB of states of 8 beams, 5 of which survive, in place: 230 us, in
// which DRAM moves 1.53 GB, 6.66 TB/s (branches around the loads, and 16-byte accesses: 400).
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
#ifdef PEARL_CHECKED
    const unsigned char *src_end, *dst_end;           // behind the last state's last byte
#else
    // (nobody looks at it; two members more cost the 1 GB move below 16 %)
    static constexpr const unsigned char* dst_end = nullptr;
#endif
};
constexpr uint32_t kMoveThreads = 256;

template <int B, int M>
__global__ void __launch_bounds__(kMoveThreads) reorder_kernel(const ReorderArgs a)
{
    static_assert(B < 32 || M <= 16, "32 states of 32 bytes are more than a thread's registers");
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
    for (int i = 0; i < M; ++i) from[i] = rows_read_if((uint32_t)i < a.W, a.parent + (uint64_t)g * a.W + i, -1);
#pragma unroll
    for (int i = 0; i < M; ++i) {
        bad |= from[i] < -1 || from[i] >= (int32_t)a.W;
        if ((uint32_t)from[i] >= a.W || (a.in_place && from[i] == i)) from[i] = -1;
        if (from[i] >= 0 && !ROWS_IN_ARRAY(a.status, src + (uint64_t)(uint32_t)from[i] * a.sp.state_pitch, B, a.src, a.src_end)) from[i] = -1;
        rows_load_if<true>(from[i] >= 0, v[i], src + (uint64_t)(uint32_t)from[i] * a.sp.state_pitch);
    }
#pragma unroll
    for (int i = 0; i < M; ++i)
        if (from[i] >= 0 && ROWS_IN_ARRAY(a.status, dst + (uint64_t)i * a.dp.state_pitch, B, a.dst, a.dst_end)) rows_store(dst + (uint64_t)i * a.dp.state_pitch, v[i]);
    if (bad && col == 0) atomicOr(a.status, PEARL_ST_BAD_INDEX);
}

// The same where states start at odd bytes or odd 2-byte places (67 MB of states of 4 beams in pieces of 251 x 33 binary16 elements, in
// place: 31 us, by 2 bytes 75).  A block has kAnyTile bytes of a piece of all W states of a block and group: its threads read
// what the moved states need, each thread the 16-byte words of each destination that it will store, meet, and store.  No other
// block stores to those bytes, so this move can be made in place, too.  (The first and last words of a tile hold bytes of the tiles
// beside it, which may be stored to meanwhile: those bytes are shifted out or not stored.)
constexpr uint32_t kAnyTile = (kMoveThreads - 1) * 16;
template <int S, int M>
__global__ void __launch_bounds__(kMoveThreads) reorder_any_kernel(const ReorderArgs a, uint64_t src_bytes)
{
    rows_begin();
    // (cols, piece_cols: bytes; col_blocks: tiles of all pieces of a state)
    const uint64_t og = blockIdx.x / a.col_blocks;
    const uint32_t g = (uint32_t)(og % a.G), tiles = (uint32_t)((a.piece_cols + kAnyTile - 1) / kAnyTile);
    const uint64_t o = og / a.G, of = blockIdx.x - og * a.col_blocks, piece = of / tiles;
    const uint64_t begin = (of - piece * tiles) * kAnyTile;
    const int bytes = (int)(a.piece_cols - begin < kAnyTile ? a.piece_cols - begin : kAnyTile);
    const unsigned char* src = a.src + o * a.sp.block_pitch + (uint64_t)g * a.W * a.sp.state_pitch + piece * a.sp.piece_pitch + begin;
    unsigned char* dst = a.dst + o * a.dp.block_pitch + (uint64_t)g * a.W * a.dp.state_pitch + piece * a.dp.piece_pitch + begin;
    RowsAny<S, true> v[M];
    int32_t from[M];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < M; ++i) from[i] = rows_read_if((uint32_t)i < a.W, a.parent + (uint64_t)g * a.W + i, -1);
#pragma unroll
    for (int i = 0; i < M; ++i) {
        bad |= from[i] < -1 || from[i] >= (int32_t)a.W;
        if ((uint32_t)from[i] >= a.W || (a.in_place && from[i] == i)) from[i] = -1;
        const int first = (int)(threadIdx.x * 16) - (int)((uint32_t)(uintptr_t)(dst + (uint64_t)i * a.dp.state_pitch) & 15u);
        v[i].fetch(a.status, from[i] >= 0 && first < bytes, src + (uint64_t)(uint32_t)from[i] * a.sp.state_pitch + first, a.src, a.src + src_bytes);
    }
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int first = (int)(threadIdx.x * 16) - (int)((uint32_t)(uintptr_t)(dst + (uint64_t)i * a.dp.state_pitch) & 15u);
        if (from[i] >= 0 && first < bytes)
            v[i].get(src + (uint64_t)(uint32_t)from[i] * a.sp.state_pitch + first, a.src, a.src + src_bytes);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) {
        unsigned char* to = dst + (uint64_t)i * a.dp.state_pitch;
        const int first = (int)(threadIdx.x * 16) - (int)((uint32_t)(uintptr_t)to & 15u);
        if (from[i] >= 0 && first < bytes) rows_store_part<S>(a.status, to + first, v[i].v, -first, bytes - first, a.dst, a.dst_end);
    }
    if (bad && of == 0 && threadIdx.x == 0) atomicOr(a.status, PEARL_ST_BAD_INDEX);
}
template <int S>
int launch_reorder_any(const ReorderArgs& a, uint64_t src_bytes, dim3 grid, cudaStream_t s)
{
    if (a.W <= 4) return rows_launch(reorder_any_kernel<S, 4>, grid, dim3(kMoveThreads), 0, s, 0, a, src_bytes);
    return rows_launch(reorder_any_kernel<S, 8>, grid, dim3(kMoveThreads), 0, s, 0, a, src_bytes);
}

template <int B>
int launch_reorder(const ReorderArgs& a, dim3 grid, cudaStream_t s)
{
    if (a.W <= 4) return rows_launch(reorder_kernel<B, 4>, grid, dim3(kMoveThreads), 0, s, 0, a);
    if (a.W <= 8) return rows_launch(reorder_kernel<B, 8>, grid, dim3(kMoveThreads), 0, s, 0, a);
    if (a.W <= 16) return rows_launch(reorder_kernel<B, 16>, grid, dim3(kMoveThreads), 0, s, 0, a);
    if constexpr (B < 32) return rows_launch(reorder_kernel<B, 32>, grid, dim3(kMoveThreads), 0, s, 0, a);
    else return -1;
}

}  // namespace

int rows_launch_beam_select(unsigned* status, uint32_t G, uint32_t W, uint32_t V, uint32_t C, uint32_t dtype, const void* logits,
                            uint64_t ld, const float* scores, const uint8_t* done, int32_t end_token, float* best_score,
                            int32_t* best_beam, int32_t* best_token, cudaStream_t s)
{
    if (G == 0) return 0;
    // Rows are cut into parts where there are too few of them to occupy the GPU, fewer than two an SM (148 rows of 131072 bfloat16 logits
    // 18.6 us; cut below one an SM 20.0, below four 24.8; 100 rows of 50257: 15.5, 14.5, 23.2; 296 of 131072: 24.6, 24.6, 26.5).  A part has 1024
    // logits at least (4 rows of 8000 binary32 logits 7.1 us; with 2048 7.6, with 512 7.2; 1 row of 4000: 7.1, 7.6, 7.2).
    SelectArgs a;
    const uint32_t most = (uint64_t)G * kMostCtas <= (uint64_t)rows_sm_count() && W <= kMostCtas ? kMostCtas : 8u;
    a.units_per_cta = (W + most - 1) / most;
    a.parts = 1;
    while ((a.parts + 1) * W <= most && (uint64_t)G * W * a.parts < 2u * rows_sm_count() && V / (a.parts + 1) >= 1024) ++a.parts;
    a.run = ((V + a.parts - 1) / a.parts + 7) / 8 * 8;
    const uint32_t units = W * a.parts, ctas = (units + a.units_per_cta - 1) / a.units_per_cta;
    if ((uint64_t)G * ctas > 0x7FFFFFFFull) return -1;
    a.status = status; a.G = G; a.W = W; a.V = V; a.C = C; a.logits = logits; a.ld = ld; a.scores = scores; a.done = done; a.end_token = end_token;
    a.best_score = best_score; a.best_beam = best_beam; a.best_token = best_token;
    a.by_parts = (65536u + a.parts - 1) / a.parts;
    a.by_C = ((1u << 20) + C - 1) / C;
    const size_t keys = ((size_t)units * C + 1) / 2 * 16, ring = kThreads * kSlots * 16;         // (the ring is the largest use of the workspace)
    int rc = -1;
#define ROWS_GO(E)                                                                                                                    \
    if (rows_large_cluster(select_kernel<E>, (int)(PEARL_ROWS_MAX_BEAMS * PEARL_ROWS_MAX_BEST * 8 + ring)))                             \
        rc = rows_launch(select_kernel<E>, dim3(G * ctas), dim3(kThreads), keys + ring, s, ctas, a)
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
    const auto extent = [&](const pearl_states_t& p) {
        return (uint64_t)(blocks - 1) * p.block_pitch + ((uint64_t)G * W - 1) * p.state_pitch + (uint64_t)(pieces - 1) * p.piece_pitch + piece_bytes;
    };
#ifdef PEARL_CHECKED
    a.src_end = a.src + extent(sp);
    a.dst_end = a.dst + extent(dp);
#endif
    uint64_t all = piece_bytes | (uintptr_t)src | (uintptr_t)dst | sp.state_pitch | dp.state_pitch;
    if (pieces > 1) all |= sp.piece_pitch | dp.piece_pitch;
    if (blocks > 1) all |= sp.block_pitch | dp.block_pitch;
    uint32_t g = rows_granule(all);
    if (g == 32 && W > 16) g = 16;          // (see reorder_kernel)
    if (g <= 2 && piece_bytes >= kRowsAnyBytes && W <= 8) {            // (more beams' words are more than a thread's registers)
        a.piece_cols = piece_bytes;
        a.cols = piece_bytes * pieces;
        a.col_blocks = (piece_bytes + kAnyTile - 1) / kAnyTile * pieces;
        const uint64_t groups = (uint64_t)blocks * G;
        if (a.col_blocks > 0x7FFFFFFFull / groups) return -1;
        const dim3 tiles((uint32_t)(a.col_blocks * groups));
        return g == 2 ? launch_reorder_any<2>(a, extent(sp), tiles, s) : launch_reorder_any<1>(a, extent(sp), tiles, s);
    }
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
