// A whole expert layer for a few rows: the router's product and choice, the experts' two products, their weighted sum.
//
// With few rows the layer is the reading of the weights that the rows ask for: 2 n floating-point operations for each weight where n rows
// ask for its expert.  So the weights are streamed once, straight from memory into the registers of the warps that multiply them,
// as the 16-row operand of a matrix instruction whose other operand are the expert's rows in groups of 8 columns; the sums
// are then so small that everything else is a chain of short steps.
#include "layer_internal.cuh"

namespace {

constexpr uint32_t kWarps = 8, kThreads = kWarps * 32;        // (of the experts' kernel: those that multiply; one more warp keeps the books)
constexpr uint32_t kBlockBytes = 128;         // of a weight row: what a warp takes of 16 rows in one step, 32 bytes a lane of each of two rows
constexpr uint32_t kMaxSlots = PEARL_LAYER_MAX_FEW * PEARL_ROWS_MAX_CHOICES;
constexpr uint32_t kSpins = 1u << 21;

// The parts of the scratch, in bytes from its start.  The counters are zero between calls.
struct Counters {
    uint32_t ticket, finished;
    uint32_t down;                                     // finished pieces of all second products
    uint32_t up[PEARL_ROWS_MAX_EXPERTS];               // of an expert's first product
};
struct Layout {
    uint64_t logits, h, z, bytes, pitch;
};
Layout layout_of(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k)
{
    const auto up = [](uint64_t n) { return (n + 255) / 256 * 256; };
    Layout l;
    l.pitch = 2 * ((2ull * H + 127) / 128 * 128);       // of a slot's h: two rows of 16 bits, or one of 32
    l.logits = up(sizeof(Counters));
    l.h = l.logits + up((uint64_t)T * E * 4);
    l.z = l.h + up((uint64_t)T * k * l.pitch);
    l.bytes = l.z + up((uint64_t)T * k * D * 4);
    return l;
}

template <typename E> __device__ __forceinline__ float element(const E* p) { return RowsElem<E>::up(*p); }

// ---- the router's product --------------------------------------------------------------------------------------------
// logits[t, e]: a warp each, in binary64.
template <typename T>
__global__ void __launch_bounds__(kThreads) logits_kernel(uint32_t rows, uint32_t D, uint32_t E, const T* x, uint64_t ld_x, const T* router, float* logits)
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

// ---- 32 bytes of a row ---------------------------------------------------------------------------------------------
// v = the `bytes` bytes from byte `off` of w on, zeros behind them.
__device__ __forceinline__ void shifted(RowsRaw<32>& v, uint32_t (&w)[12], uint32_t off, int bytes)
{
#pragma unroll
    for (int i = 0; i < 10; ++i) w[i] = off & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 9; ++i) w[i] = off & 4u ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v.r[i] = __funnelshift_r(w[i], w[i + 1], (off & 3u) * 8u);
        if (4 * i >= bytes) v.r[i] = 0u;
        else if (4 * i + 2 >= bytes) v.r[i] &= 0xFFFFu;
    }
}

// A lane's piece of a row of x or h: 16 (or 8) elements, of which the first `bytes` bytes are there; the others are 0.  These rows are read
// again and again, by all warps, and stay in the L1.  kAlign: what rows and their lengths are multiples of, 32 or 16 bytes; 0: nothing, the
// piece comes out of the aligned words around it.
template <int kAlign> struct Piece {
    RowsRaw<32> v;
    __device__ __forceinline__ void fetch(const unsigned char* p, int bytes, const unsigned char*, const unsigned char*)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.r[i] = 0u;
        if constexpr (kAlign == 32) {
            asm volatile("{ .reg .pred q; setp.ne.u32 q, %9, 0; @q ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8]; }"
                         : "+r"(v.r[0]), "+r"(v.r[1]), "+r"(v.r[2]), "+r"(v.r[3]), "+r"(v.r[4]), "+r"(v.r[5]), "+r"(v.r[6]), "+r"(v.r[7])
                         : "l"(p), "r"((uint32_t)(bytes > 0)) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                asm volatile("{ .reg .pred q; setp.ne.u32 q, %5, 0; @q ld.global.v4.b32 {%0, %1, %2, %3}, [%4]; }"
                             : "+r"(v.r[i]), "+r"(v.r[i + 1]), "+r"(v.r[i + 2]), "+r"(v.r[i + 3])
                             : "l"(p + i * 4), "r"((uint32_t)(bytes > i * 4)) : "memory");
        }
    }
    __device__ __forceinline__ const RowsRaw<32>& get(const unsigned char*, int, const unsigned char*, const unsigned char*) { return v; }
};
template <> struct Piece<0> {
    uint32_t w[12];
    RowsRaw<32> v;
    // [lo, hi): the array that p points into; aligned words that are not wholly in it are not read as such.
    __device__ __forceinline__ static bool whole(const unsigned char* p, const unsigned char* lo, const unsigned char* hi)
    {
        const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
        return (p - off >= lo) & (p - off + 48 <= hi);
    }
    __device__ __forceinline__ void fetch(const unsigned char* p, int bytes, const unsigned char* lo, const unsigned char* hi)
    {
        const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
        const bool words = bytes > 0 && whole(p, lo, hi);
#pragma unroll
        for (int i = 0; i < 12; ++i) w[i] = 0u;
#pragma unroll
        for (int i = 0; i < 12; i += 4)
            asm volatile("{ .reg .pred q; setp.ne.u32 q, %5, 0; @q ld.global.v4.b32 {%0, %1, %2, %3}, [%4]; }"
                         : "+r"(w[i]), "+r"(w[i + 1]), "+r"(w[i + 2]), "+r"(w[i + 3])
                         : "l"(p - off + i * 4), "r"((uint32_t)(words & (i < 8 || off > 0) & ((int)off + bytes > i * 4))) : "memory");
    }
    __device__ __forceinline__ const RowsRaw<32>& get(const unsigned char* p, int bytes, const unsigned char* lo, const unsigned char* hi)
    {
        if (bytes <= 0 || whole(p, lo, hi)) {
            shifted(v, w, (uint32_t)(uintptr_t)p & 15u, bytes);
            return v;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v.r[i] = 0u;
            if (4 * i < bytes) v.r[i] = *reinterpret_cast<const uint16_t*>(p + 4 * i);
            if (4 * i + 2 < bytes) v.r[i] |= (uint32_t) * reinterpret_cast<const uint16_t*>(p + 4 * i + 2) << 16;
        }
        return v;
    }
};

// ---- matrix instructions ----------------------------------------------------------------------------------------------
// acc += A B for 16 rows of weights and 8 columns over a block of 128 bytes of each: lane (g, t), g = lane / 4, has piece t of rows g and
// g + 8 of A and of column g of B.  Which element of a piece is which k of an instruction does not matter, as it is the same for both.
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <typename E>
__device__ __forceinline__ void block_product(float (&c)[4], const RowsRaw<32>& a, const RowsRaw<32>& b, const RowsRaw<32>& x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) mma16(c, a.r[2 * i], b.r[2 * i], a.r[2 * i + 1], b.r[2 * i + 1], x.r[2 * i], x.r[2 * i + 1], E());
}
// binary32 as the sum of two numbers of 11 bits, each rounded to nearest: what is left out of a product is 2^-22 of it.
__device__ __forceinline__ void split(RowsRaw<32>& high, RowsRaw<32>& low, const RowsRaw<32>& v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(high.r[i]) : "f"(__uint_as_float(v.r[i])));
        const float rest = __uint_as_float(v.r[i]) - __uint_as_float(high.r[i]);
        asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(low.r[i]) : "f"(rest));
    }
}

// ---- the experts' products --------------------------------------------------------------------------------------------
struct Args {
    uint32_t T, D, H, E, k, act;
    const unsigned char *x, *x_end, *up, *up_end, *down, *down_end, *h_end;
    uint64_t ld_x, ld_y, pitch;         // bytes
    const float* w;
    const int32_t* ids;
    unsigned char *y, *h;
    float* z;
    Counters* n;
    unsigned* status;
};
// What a CTA works on: some strips of 16 weight rows of one expert, with some of its slots; or a part of y.
enum Kind : uint32_t { kUp, kDown, kSum, kEnd };
struct Item {
    uint32_t kind;
    uint32_t i, piece, first, columns;          // the expert's place among those asked for; of its slots
};
// A warp's ring: stages of 16 rows of 128 bytes, 16 bytes more a row, which spreads the rows over the banks (and holds the rest of a row that
// starts between two words).
constexpr uint32_t kStages = 4, kPitch = kBlockBytes + 16, kStageBytes = 16 * kPitch;
struct Shared {
    unsigned char ring[kWarps][kStages][kStageBytes];
    float part[kWarps][2 * 128];                       // the warps' sums of 16 columns of one strip
    uint32_t count[PEARL_ROWS_MAX_EXPERTS];            // slots of an expert; then where its next one goes
    uint16_t expert[PEARL_ROWS_MAX_EXPERTS], first[PEARL_ROWS_MAX_EXPERTS + 1];       // of the experts that are asked for
    uint16_t slot[kMaxSlots];                          // by expert
    uint32_t sums[2][kWarps];
    Item item[2];                                      // what the warps work on, and what comes next
    uint32_t asked, last;
};

// The experts that are asked for, and their slots.
__device__ void plan(const Args& a, Shared& s)
{
    const uint32_t slots = a.T * a.k, tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    for (uint32_t e = tid; e < a.E; e += kThreads + 32) s.count[e] = 0;
    __syncthreads();
    for (uint32_t i = tid; i < slots; i += kThreads + 32) {
        const int32_t e = a.ids[i];
        if ((uint32_t)e < a.E) atomicAdd(&s.count[e], 1u);
        else if (e != -1 && blockIdx.x == 0) atomicOr(a.status, PEARL_ST_BAD_INDEX);
    }
    __syncthreads();
    constexpr uint32_t kEach = PEARL_ROWS_MAX_EXPERTS / kThreads;
    uint32_t mine[kEach], slots_here = 0, asked_here = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = tid * kEach + i;
        mine[i] = e < a.E ? s.count[e] : 0u;               // (the last warp has none)
        slots_here += mine[i];
        asked_here += mine[i] != 0;
    }
    uint32_t slots_to = slots_here, asked_to = asked_here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t p = __shfl_up_sync(0xFFFFFFFFu, slots_to, o), q = __shfl_up_sync(0xFFFFFFFFu, asked_to, o);
        if (lane >= (uint32_t)o) { slots_to += p; asked_to += q; }
    }
    if (lane == 31 && warp < kWarps) { s.sums[0][warp] = slots_to; s.sums[1][warp] = asked_to; }
    __syncthreads();
    uint32_t at = slots_to - slots_here, i_asked = asked_to - asked_here;
    for (uint32_t w = 0; w < min(warp, kWarps); ++w) { at += s.sums[0][w]; i_asked += s.sums[1][w]; }
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = tid * kEach + i;
        if (e >= a.E) continue;
        s.count[e] = at;
        if (mine[i]) {
            s.expert[i_asked] = (uint16_t)e;
            s.first[i_asked] = (uint16_t)at;
            at += mine[i];
            ++i_asked;
        }
    }
    if (tid == kThreads - 1) { s.asked = i_asked; s.first[i_asked] = (uint16_t)at; }
    __syncthreads();
    for (uint32_t i = tid; i < slots; i += kThreads + 32) {
        const int32_t e = a.ids[i];
        if ((uint32_t)e < a.E) s.slot[atomicAdd(&s.count[e], 1u)] = (uint16_t)i;      // (in any order: no sum runs over an expert's slots)
    }
    __syncthreads();
}

// Barriers between the warps that multiply and the one that keeps the books: items handed over, what they need there, items finished; two of
// each, for every other item.
constexpr uint32_t kFull = 1, kReady = 3, kDone = 5, kMeet = 7;
__device__ __forceinline__ void worker_waits(uint32_t id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kThreads + 32) : "memory"); }
__device__ __forceinline__ void worker_arrives(uint32_t id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kThreads + 32) : "memory"); }
__device__ __forceinline__ void books_arrive(uint32_t id) { worker_arrives(id); }
__device__ __forceinline__ void books_wait(uint32_t id) { worker_waits(id); }
__device__ __forceinline__ void workers_meet() { asm volatile("bar.sync %0, %1;" ::"n"(kMeet), "n"(kThreads) : "memory"); }

__device__ __forceinline__ uint32_t read_acquired(const uint32_t* p)
{
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// How a product is cut: pieces of `strips` strips of 16 weight rows; `ways` warps share a strip's blocks among them (strips * ways = 8).
struct Cut {
    uint32_t blocks, strips, ways, pieces;
};
__device__ __forceinline__ Cut cut_of(uint32_t rows, uint32_t row_bytes, uint32_t asked)
{
    Cut c;
    c.blocks = (row_bytes + kBlockBytes - 1) / kBlockBytes;
    const uint32_t strips = (rows + 15) / 16;
    // two pieces a CTA where there are that many strips; else a strip is shared, down to a block a warp
    c.strips = kWarps;
    while (c.strips > 1 && (uint64_t)strips * asked < 2ull * c.strips * gridDim.x) c.strips /= 2;
    c.ways = kWarps / c.strips;
    while (c.ways > 1 && c.ways / 2 >= c.blocks) c.ways /= 2;
    c.strips = kWarps / c.ways;
    c.pieces = (strips + c.strips - 1) / c.strips;
    return c;
}

__device__ __forceinline__ float activated(float gate, float value) { return gate / (1.0f + expf(-gate)) * value; }

// The weight rows of an item's strip, as the lanes copy them: lane l has word l % 8 of rows l / 8 + 4 q of a block.
template <typename E, int kAlign>
struct Strip {
    const unsigned char *low, *high;            // row 0's and row 8's first byte
    uint32_t row_bytes, blocks, rows_low, rows_high;    // rows that there are, of the first and of the last 8
    __device__ __forceinline__ Strip(const Args& a, const Shared& s, const Cut& c, const Item& it)
    {
        const bool gated = it.kind == kUp && a.act == PEARL_ACT_SILU_GATED;
        const uint32_t rows = it.kind == kDown ? a.D : a.H, strip = it.piece * c.strips + (threadIdx.x >> 5) / c.ways;
        row_bytes = (it.kind == kDown ? a.H : a.D) * (uint32_t)sizeof(E);
        blocks = c.blocks;
        const uint32_t j = strip * (gated ? 8u : 16u), k = gated ? j : j + 8;
        const unsigned char* m = (it.kind == kDown ? a.down : a.up) + (uint64_t)s.expert[it.i] * rows * (gated ? 2 : 1) * row_bytes;
        low = m + (uint64_t)j * row_bytes;
        high = m + (uint64_t)(gated ? rows + k : k) * row_bytes;
        rows_low = j < rows ? min(rows - j, 8u) : 0u;
        rows_high = k < rows ? min(rows - k, 8u) : 0u;
    }
    // Starts the copy of a block of the strip to a stage; what is not there becomes 0.
    __device__ __forceinline__ void copy(const Args& a, const Item& it, uint32_t block, unsigned char* stage) const
    {
        const uint32_t lane = threadIdx.x & 31u;
        constexpr uint32_t kWords = kPitch / 16;
        if (block >= blocks) {
        } else if constexpr (kAlign != 0) {
            const uint32_t r = lane >> 3, at = block * kBlockBytes + (lane & 7u) * 16;
            unsigned char* to = stage + r * kPitch + (lane & 7u) * 16;
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                const uint32_t row = r + q % 2 * 4;
                const bool there = at < row_bytes && row < (q < 2 ? rows_low : rows_high);
                word(a.status, to + q * 4 * kPitch, (q < 2 ? low : high) + (uint64_t)row * row_bytes + at, there ? 16u : 0u, it.kind == kDown ? a.down : a.up,
                     it.kind == kDown ? a.down_end : a.up_end);
            }
        } else {
            const unsigned char *lo = it.kind == kDown ? a.down : a.up, *hi = it.kind == kDown ? a.down_end : a.up_end;
#pragma unroll
            for (uint32_t q = 0; q < (16 * kWords + 31) / 32; ++q) {
                const uint32_t n = lane + q * 32, row = n / kWords, w = n - row * kWords;
                if (row >= 16) break;
                const unsigned char* from = (row < 8 ? low : high) + (uint64_t)(row & 7u) * row_bytes;
                const unsigned char* p = from - ((uintptr_t)from & 15u) + block * kBlockBytes + w * 16;
                const bool there = (row & 7u) < (row < 8 ? rows_low : rows_high) && p < from + row_bytes;
                unsigned char* to = stage + row * kPitch + w * 16;
                if (there && p < lo) {                       // the array's first word, of which a part is not its own
                    for (int b = 0; b < 16; b += 2)
                        *reinterpret_cast<uint16_t*>(to + b) = p + b >= lo && p + b < hi ? *reinterpret_cast<const uint16_t*>(p + b) : (uint16_t)0;
                    continue;
                }
                word(a.status, to, p, !there ? 0u : hi - p < 16 ? (uint32_t)(hi - p) : 16u, lo, hi);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // `bytes` bytes (1 .. 16) of the array [lo, hi) and zeros behind them, or 16 zeros.
    __device__ __forceinline__ static void word(unsigned* status, unsigned char* to, const unsigned char* from, uint32_t bytes, const unsigned char* lo,
                                                const unsigned char* hi)
    {
        if (bytes && ROWS_IN_ARRAY(status, from, bytes, lo, hi))
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(bytes) : "memory");
        else
            *reinterpret_cast<uint4*>(to) = make_uint4(0, 0, 0, 0);
    }
    // The lane's piece of row g of the stage (g + 8 with `upper`), of which `bytes` are there.
    __device__ __forceinline__ RowsRaw<32> piece(const unsigned char* stage, bool upper, int bytes) const
    {
        const uint32_t lane = threadIdx.x & 31u, g = lane >> 2, t = lane & 3u;
        const uint4* p = reinterpret_cast<const uint4*>(stage + (g + (upper ? 8 : 0)) * kPitch + t * 32);
        RowsRaw<32> v;
        if constexpr (kAlign != 0) {
            const uint4 x = p[0], y = p[1];
            v.r[0] = x.x; v.r[1] = x.y; v.r[2] = x.z; v.r[3] = x.w; v.r[4] = y.x; v.r[5] = y.y; v.r[6] = y.z; v.r[7] = y.w;
        } else {
            const uint32_t off = (uint32_t)(uintptr_t)((upper ? high : low) + (uint64_t)g * row_bytes) & 15u;
            const uint4 x = p[0], y = p[1], z = p[2];
            uint32_t w[12] = { x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w };
            shifted(v, w, off, bytes);
        }
        return v;
    }
};

// Starts an item's first blocks.
template <typename E, int kAlign> __device__ __forceinline__ void start(const Args& a, Shared& s, const Cut& c, const Item& it)
{
    const uint32_t warp = threadIdx.x >> 5, way = warp % c.ways;
    const Strip<E, kAlign> strip(a, s, c, it);
#pragma unroll
    for (uint32_t u = 0; u + 1 < kStages; ++u) strip.copy(a, it, way + u * c.ways, s.ring[warp][u]);
}

// One item's product; its first blocks are on their way.  next() names the item to start as soon as the ring is free.
template <typename E, int kAlign, int NT, uint32_t kKind, typename Next>
__device__ void product(const Args& a, Shared& s, const Cut& c, const Item& it, uint32_t turn, Next next)
{
    constexpr bool k32 = sizeof(E) == 4, kSecond = kKind == kDown;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3u;
    const uint32_t way = warp % c.ways;
    const bool gated = kKind == kUp && a.act == PEARL_ACT_SILU_GATED;
    const uint32_t rows = kSecond ? a.D : a.H;
    const uint32_t j0 = (it.piece * c.strips + warp / c.ways) * (gated ? 8u : 16u), ja = j0 + g, jb = gated ? ja : j0 + 8 + g;
    const Strip<E, kAlign> strip(a, s, c, it);
    const int here = (int)strip.row_bytes - (int)(t * 32);       // bytes from a lane's first piece on
    const unsigned char* px[NT];
    int lx[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t col = n * 8 + g;
        const uint32_t slot = col < it.columns ? s.slot[it.first + col] : 0u;
        px[n] = (kSecond ? a.h + slot * a.pitch : a.x + (uint64_t)(slot / a.k) * a.ld_x) + t * 32;
        lx[n] = col < it.columns ? here : 0;
    }
    const unsigned char *xlo = kSecond ? a.h : a.x, *xhi = kSecond ? a.h_end : a.x_end;
    float acc[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[n][q] = 0.0f;
    worker_waits(kReady + turn);
    uint32_t stage = 0;
    for (uint32_t block = way; block < c.blocks; block += c.ways) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        const int at = (int)(block * kBlockBytes);
        strip.copy(a, it, block + (kStages - 1) * c.ways, s.ring[warp][(stage + kStages - 1) % kStages]);
        const RowsRaw<32> va = strip.piece(s.ring[warp][stage], false, here - at), vb = strip.piece(s.ring[warp][stage], true, here - at);
        stage = (stage + 1) % kStages;
        if constexpr (k32) {
            RowsRaw<32> ah, al, bh, bl;
            split(ah, al, va);
            split(bh, bl, vb);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n > 0 && n * 8 >= (int)it.columns) break;
                Piece<kAlign> x;
                x.fetch(px[n] + at, lx[n] - at, xlo, xhi);
                RowsRaw<32> xh, xl;
                split(xh, xl, x.get(px[n] + at, lx[n] - at, xlo, xhi));
                float part[4] = { 0.0f, 0.0f, 0.0f, 0.0f };     // (the instruction cuts off where an addition rounds: sums of a block only)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    mma8(part, al.r[2 * q], bl.r[2 * q], al.r[2 * q + 1], bl.r[2 * q + 1], xh.r[2 * q], xh.r[2 * q + 1]);
                    mma8(part, ah.r[2 * q], bh.r[2 * q], ah.r[2 * q + 1], bh.r[2 * q + 1], xl.r[2 * q], xl.r[2 * q + 1]);
                    mma8(part, ah.r[2 * q], bh.r[2 * q], ah.r[2 * q + 1], bh.r[2 * q + 1], xh.r[2 * q], xh.r[2 * q + 1]);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[n][q] += part[q];
            }
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (n > 0 && n * 8 >= (int)it.columns) break;
                Piece<kAlign> x;
                x.fetch(px[n] + at, lx[n] - at, xlo, xhi);
                if constexpr (kSecond) {
                    Piece<kAlign> low;
                    low.fetch(px[n] + a.pitch / 2 + at, lx[n] - at, xlo, xhi);
                    block_product<E>(acc[n], va, vb, x.get(px[n] + at, lx[n] - at, xlo, xhi));
                    block_product<E>(acc[n], va, vb, low.get(px[n] + a.pitch / 2 + at, lx[n] - at, xlo, xhi));
                } else {
                    block_product<E>(acc[n], va, vb, x.get(px[n] + at, lx[n] - at, xlo, xhi));
                }
            }
        }
    }
    next();
    // the warps that share a strip: their sums in order, 16 columns at a time
    if (c.ways > 1) {
#pragma unroll
        for (int n0 = 0; n0 < NT; n0 += 2) {
            if (n0 > 0) workers_meet();
#pragma unroll
            for (int n = n0; n < NT && n < n0 + 2; ++n)
                *reinterpret_cast<float4*>(s.part[warp] + (n - n0) * 128 + lane * 4) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
            workers_meet();
            if (way != 0) continue;
#pragma unroll
            for (int n = n0; n < NT && n < n0 + 2; ++n)
                for (uint32_t w = 1; w < c.ways; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(s.part[warp + w] + (n - n0) * 128 + lane * 4);
                    acc[n][0] += v.x; acc[n][1] += v.y; acc[n][2] += v.z; acc[n][3] += v.w;
                }
        }
    }
    if (way == 0) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t col = n * 8 + t * 2 + q;
                if (col >= it.columns) continue;
                const uint32_t slot = s.slot[it.first + col];
                if constexpr (kSecond) {
                    float* z = a.z + (uint64_t)slot * a.D;
                    if (ja < rows) z[ja] = acc[n][q];
                    if (jb < rows) z[jb] = acc[n][q + 2];
                } else {
                    const auto store = [&](uint32_t j, float v) {
                        if (j >= rows) return;
                        if constexpr (k32) {
                            reinterpret_cast<float*>(a.h + slot * a.pitch)[j] = v;
                        } else {
                            // as the sum of two: a single one would be off by as much as the result's own rounding
                            const E high = RowsElem<E>::down(v);
                            const float rest = v - RowsElem<E>::up(high);
                            reinterpret_cast<E*>(a.h + slot * a.pitch)[j] = high;
                            reinterpret_cast<E*>(a.h + slot * a.pitch + a.pitch / 2)[j] = RowsElem<E>::down(isfinite(RowsElem<E>::up(high)) ? rest : 0.0f);
                        }
                    };
                    if (gated) {
                        store(ja, activated(acc[n][q], acc[n][q + 2]));
                    } else {
                        store(ja, acc[n][q] < 0.0f ? 0.0f : acc[n][q]);
                        store(jb, acc[n][q + 2] < 0.0f ? 0.0f : acc[n][q + 2]);
                    }
                }
            }
    }
}

template <typename E, int kAlign, uint32_t kKind, typename Next>
__device__ __forceinline__ void product_of(const Args& a, Shared& s, const Cut& c, const Item& it, uint32_t turn, Next next)
{
    if (it.columns <= 8) product<E, kAlign, 1, kKind>(a, s, c, it, turn, next);
    else if (it.columns <= 16) product<E, kAlign, 2, kKind>(a, s, c, it, turn, next);
    else if (it.columns <= 32) product<E, kAlign, 4, kKind>(a, s, c, it, turn, next);
    else product<E, kAlign, 8, kKind>(a, s, c, it, turn, next);
}

// A part of y, of `parts`: the slots' sums in the order of the choices.
template <typename E> __device__ void weighted_sums(const Args& a, uint32_t part, uint32_t parts)
{
    const uint64_t all = (uint64_t)a.T * a.D, each = (all + parts - 1) / parts, end = min(all, (part + 1) * each);
    for (uint64_t n = part * each + threadIdx.x; n < end; n += kThreads) {
        const uint32_t t = (uint32_t)(n / a.D), d = (uint32_t)(n - (uint64_t)t * a.D);
        float sum = 0.0f;
#pragma unroll 4
        for (uint32_t j = 0; j < a.k; ++j) {
            const uint32_t slot = t * a.k + j;
            if ((uint32_t)a.ids[slot] < a.E) sum = __fmaf_rn(a.w[slot], a.z[(uint64_t)slot * a.D + d], sum);
        }
        reinterpret_cast<E*>(a.y + t * a.ld_y)[d] = RowsElem<E>::down(sum);
    }
}

// The warp that keeps the books.  It takes pieces in order -- all first products' before the second ones', these before the parts of y --,
// hands them to the others, waits for what a piece needs and tells what is finished.  It alone fences, and it has no copies on their way, for
// which a fence would wait.  A CTA waits only with an earlier piece told, and each piece that it waits for is with a CTA that runs: nobody waits
// for one that is yet to be launched.
__device__ void keep_books(const Args& a, Shared& s, const Cut& up, const Cut& down, uint32_t parts)
{
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t asked = s.asked, ups = asked * up.pieces, downs = asked * down.pieces;
    uint32_t known = 0;                             // experts (in order) whose first product is known to be there
    const auto ticket = [&] { return lane == 0 ? atomicAdd(&a.n->ticket, 1u) : 0u; };
    uint32_t ahead = ticket();
    const auto item = [&] {
        Item it = { kEnd, 0, 0, 0, 0 };
        const uint32_t task = __shfl_sync(0xFFFFFFFFu, ahead, 0);
        if (task >= ups + downs + parts) return it;
        ahead = ticket();
        if (task >= ups + downs) {
            it.kind = kSum;
            it.piece = task - ups - downs;
            return it;
        }
        it.kind = task < ups ? kUp : kDown;
        const uint32_t n = task < ups ? task : task - ups, pieces = task < ups ? up.pieces : down.pieces;
        it.i = n / pieces;
        it.piece = n - it.i * pieces;
        it.first = s.first[it.i];
        it.columns = min(s.first[it.i + 1] - it.first, 64u);
        return it;
    };
    // whether what the item needs is there; `wait` for it (with a limit, and a status bit behind that)
    const auto needs = [&](const Item& it, bool wait) {
        if (it.kind == kUp || it.kind == kEnd || (it.kind == kDown && it.i < known)) return true;
        uint32_t there = 0;
        if (lane == 0) {
            const uint32_t* p = it.kind == kDown ? &a.n->up[it.i] : &a.n->down;
            const uint32_t count = it.kind == kDown ? up.pieces : downs;
            uint32_t spins = 0;
            while (!(there = read_acquired(p) >= count) && wait)
                if (++spins > kSpins) { atomicOr(a.status, PEARL_ST_INTERNAL); break; }
        }
        there = __shfl_sync(0xFFFFFFFFu, there, 0);
        if (there && it.kind == kDown) known = it.i + 1;
        return there != 0;
    };
    const auto give = [&](const Item& it, uint32_t turn) {
        if (lane == 0) s.item[turn] = it;
        __syncwarp();
        books_arrive(kFull + turn);
    };
    Item it = item();
    give(it, 0);
    bool told = false;
    for (uint32_t turn = 0;; turn ^= 1u) {
        if (!told) { needs(it, true); books_arrive(kReady + turn); }
        if (it.kind == kEnd) break;
        Item then;
        // an expert of more than 64 slots is gone over once for each 64
        const bool more = (it.kind == kUp || it.kind == kDown) && it.first + it.columns < s.first[it.i + 1];
        if (more) {
            then = it;
            then.first = it.first + it.columns;
            then.columns = min(s.first[it.i + 1] - then.first, 64u);
        } else {
            then = item();
        }
        give(then, turn ^ 1u);
        told = needs(then, false);
        if (told) books_arrive(kReady + (turn ^ 1u));
        books_wait(kDone + turn);
        if (!more && it.kind != kSum && lane == 0) {
            __threadfence();
            atomicAdd(it.kind == kUp ? &a.n->up[it.i] : &a.n->down, 1u);
        }
        it = then;
    }
}

template <typename E, int kAlign>
__global__ void __launch_bounds__(kThreads + 32, 2) experts_kernel(Args a)
{
    extern __shared__ __align__(16) unsigned char memory[];
    Shared& s = *reinterpret_cast<Shared*>(memory);
    rows_begin();
    plan(a, s);
    const uint32_t asked = s.asked;
    const bool gated = a.act == PEARL_ACT_SILU_GATED;
    const Cut up = cut_of(gated ? a.H * 2 : a.H, a.D * (uint32_t)sizeof(E), asked), down = cut_of(a.D, a.H * (uint32_t)sizeof(E), asked);
    const uint32_t parts = min(gridDim.x, (uint32_t)(((uint64_t)a.T * a.D + kThreads - 1) / kThreads));
    if (threadIdx.x >= kThreads) {
        keep_books(a, s, up, down, parts);
    } else {
        const auto begin = [&](const Item& it) {
            if (it.kind == kUp || it.kind == kDown) start<E, kAlign>(a, s, it.kind == kDown ? down : up, it);
        };
        worker_waits(kFull);
        Item it = s.item[0];
        begin(it);
        for (uint32_t turn = 0; it.kind != kEnd; turn ^= 1u) {
            Item then;
            const auto next = [&]() {
                worker_waits(kFull + (turn ^ 1u));
                then = s.item[turn ^ 1u];
                begin(then);
            };
            if (it.kind == kUp) {
                product_of<E, kAlign, kUp>(a, s, up, it, turn, next);
            } else if (it.kind == kDown) {
                product_of<E, kAlign, kDown>(a, s, down, it, turn, next);
            } else {
                next();
                worker_waits(kReady + turn);
                weighted_sums<E>(a, it.piece, parts);
            }
            worker_arrives(kDone + turn);
            it = then;
        }
    }
    // the last one out leaves the counters as they were
    __syncthreads();
    if (threadIdx.x == 0) s.last = atomicAdd(&a.n->finished, 1u) + 1 == gridDim.x;
    __syncthreads();
    if (!s.last) return;
    for (uint32_t i = threadIdx.x; i < asked; i += kThreads + 32) a.n->up[i] = 0;
    if (threadIdx.x == 0) a.n->ticket = a.n->finished = a.n->down = 0;
}

template <typename T, int kAlign> int experts_launch(const Args& a, cudaStream_t s)
{
    static std::atomic<bool> ready[kRowsMaxDevices];
    const int dev = rows_device();
    if (dev < 0 || !ready[dev]) {
        if (cudaFuncSetAttribute(experts_kernel<T, kAlign>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) != cudaSuccess) return -1;
        if (dev >= 0) ready[dev] = true;
    }
    return rows_launch(experts_kernel<T, kAlign>, dim3(2 * rows_sm_count()), dim3(kThreads + 32), sizeof(Shared), s, 0, a);
}

template <typename T> int experts_as(unsigned* status, const LayerExperts& a, cudaStream_t s)
{
    const Layout l = layout_of(a.T, a.D, a.H, a.E, a.k);
    float* logits = (float*)((char*)a.work + l.logits);
    int n = 0, m;
    if (a.router) {
        if ((m = rows_launch(logits_kernel<T>, dim3((a.T * a.E + kWarps - 1) / kWarps), dim3(kThreads), 0, s, 0, a.T, a.D, a.E, (const T*)a.x, a.ld_x,
                             (const T*)a.router, logits)) < 0) return m;
        n += m;
        if ((m = rows_launch_route(status, a.T, a.E, a.k, PEARL_F32, logits, a.E, a.over_chosen, a.w, a.ids, s)) < 0) return m;
        n += m;
    }
    constexpr uint32_t S = sizeof(T);
    unsigned char* work = (unsigned char*)a.work;
    const unsigned char* x = (const unsigned char*)a.x;
    const unsigned char *up = (const unsigned char*)a.up, *down = (const unsigned char*)a.down;
    const uint64_t matrix = (uint64_t)a.E * a.D * a.H * S;
    const Args args = { a.T, a.D, a.H, a.E, a.k, a.act, x, x + ((uint64_t)(a.T - 1) * a.ld_x + a.D) * S, up,
                        up + matrix * (a.act == PEARL_ACT_SILU_GATED ? 2 : 1), down, down + matrix, work + l.z, a.ld_x * S, a.ld_y * S, l.pitch, a.w, a.ids,
                        (unsigned char*)a.y, work + l.h, (float*)(work + l.z), (Counters*)work, status };
    const uint32_t granule = rows_granule((uintptr_t)a.x | (uintptr_t)a.up, (uintptr_t)a.down, a.ld_x * S, (uint64_t)a.D * S, (uint64_t)a.H * S);
    m = granule >= 32 ? experts_launch<T, 32>(args, s) : granule >= 16 ? experts_launch<T, 16>(args, s) : experts_launch<T, 0>(args, s);
    return m < 0 ? m : n + m;
}

}  // namespace

uint64_t layer_experts_work_bytes(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k) { return layout_of(T, D, H, E, k).bytes; }

int layer_launch_experts(unsigned* status, const LayerExperts& a, cudaStream_t s)
{
#define EXPERTS(T) return experts_as<T>(status, a, s)
    ROWS_WITH_TYPE(a.dtype, EXPERTS);
#undef EXPERTS
}
