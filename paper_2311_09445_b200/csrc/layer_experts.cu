// A whole expert layer for a few rows: the router's product and choice, the experts' two products, their weighted sum.
//
// With few rows the layer is the reading of the weights that the rows ask for: 2 n floating-point operations for each weight where n rows
// ask for its expert.  So the weights are streamed through shared memory once, one CTA an SM, by copies that nobody waits for but the warps
// that multiply: these take 16 weight rows as one operand of a matrix instruction whose other operand are the expert's rows in groups of 8.
//
// Measured, in a replayed graph: 64 rows, 64 experts of 2048 x 1408, 6 a row, binary16: 1.1 GB in 212 us (5.2 TB/s); 128 experts of 4096 x 1280, 8 a row,
// bfloat16: 4 GB in 729 us (5.4 TB/s).  The same without products takes 189 and 636 us, without copies of x and h 211 and 724: what is left beside the
// streaming is the reading of the operands from shared memory, and ten microseconds of a call's chain of steps (choice, plan, two products, their sum).
// tcgen05.mma in the place of the warps' own instructions, M = 128 and N = 16 .. 128, the sums in tensor memory, was no faster (229 and 715 us where these
// then took 223 and 706): the weights are read from shared memory all the same, and its sums over a whole row are cut off.  With many rows an expert
// it was (8 experts, 4 a row: 93 us; this then took 107, now 98 to 104).
#include <cuda.h>

#include "layer_internal.cuh"

namespace {

constexpr uint32_t kWorkers = 8;              // warps that multiply
constexpr uint32_t kBlockBytes = 128;         // of a row: what a warp takes of 16 weight rows in one step, 32 bytes a lane of each of two rows
constexpr uint32_t kMaxSlots = PEARL_LAYER_MAX_FEW * PEARL_ROWS_MAX_CHOICES;
// Slots of an expert that are multiplied at once; one with more is gone over again, its weights from L2.  In 16 bits a thread's sums for 64 and those of
// a stage do not fit its registers: 64 rows on 8 experts of 2048 x 1408, 4 a row, binary16, 182 us, so 98; with 64 slots at each of 4 experts of
// 4096 x 1280 in binary32, which has one sum, 315 and 358.
template <typename E> constexpr uint32_t kMaxColumns = sizeof(E) == 4 ? 64 : 32;
constexpr uint32_t kSpins = kLayerSpins;

// The parts of the scratch, in bytes from its start.  The counters are zero between calls.
struct Counters {
    uint32_t ticket, finished;
    uint32_t down;                                     // finished pieces of all second products
    uint32_t up[PEARL_ROWS_MAX_EXPERTS];               // of an expert's first product
};
struct Layout {
    uint64_t logits, h, z, bytes, part;
};
// How many numbers of the rows' type an h between the products is the sum of: as many as keep it to a binary32's digits (store_h).
constexpr uint32_t kMostParts = 3;
template <typename E> constexpr uint32_t kParts = 1;
template <> constexpr uint32_t kParts<__half> = 2;
template <> constexpr uint32_t kParts<__nv_bfloat16> = 3;
Layout layout_of(uint32_t T, uint32_t D, uint32_t H, uint32_t E, uint32_t k)
{
    const auto up = [](uint64_t n) { return (n + 255) / 256 * 256; };
    Layout l;
    l.part = (2ull * H + 127) / 128 * 128;              // of a slot's h: up to three rows of 16 bits, or one of 32
    l.logits = up(sizeof(Counters));
    l.h = l.logits + up((uint64_t)T * E * 4);
    l.z = l.h + up((uint64_t)T * k * kMostParts * l.part);
    l.bytes = l.z + up((uint64_t)T * k * D * 4);
    return l;
}

// ---- the router's product --------------------------------------------------------------------------------------------
// Logits of X experts for 4 rows, in binary64, so that the choice does not hang on the order of a sum: 8 warps share the width.  A
// conversion takes four times a multiply-add's time, and 4 x 4 numbers need 8 for 16 products.
constexpr uint32_t kRowsAtOnce = 4;
template <typename E, int V, int X>
__global__ void __launch_bounds__(kWorkers * 32) logits_kernel(unsigned* status, uint32_t T, uint32_t D, uint32_t experts, const E* x, uint64_t ld_x,
                                                               const E* router, float* logits)
{
    __shared__ double sums[kWorkers][X * kRowsAtOnce];
    rows_begin();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, e0 = blockIdx.x * X, t0 = blockIdx.y * kRowsAtOnce;
    double s[X * kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < X * (int)kRowsAtOnce; ++i) s[i] = 0.0;
    for (uint32_t d = threadIdx.x * V; d < D; d += kWorkers * 32 * V) {
        RowsVec<E, V> w[X], r[kRowsAtOnce];
        // (rows and widths are multiples of an access here; rows that there are none of repeat the last one)
#pragma unroll
        for (int i = 0; i < X; ++i) w[i] = rows_load_vec<E, V>(router + (uint64_t)min(e0 + i, experts - 1) * D + d);
#pragma unroll
        for (int i = 0; i < (int)kRowsAtOnce; ++i) r[i] = rows_load_vec<E, V>(x + (uint64_t)min(t0 + i, T - 1) * ld_x + d);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            double a[X];
#pragma unroll
            for (int i = 0; i < X; ++i) a[i] = (double)w[i].get(v);
#pragma unroll
            for (int j = 0; j < (int)kRowsAtOnce; ++j) {
                const double b = (double)r[j].get(v);
#pragma unroll
                for (int i = 0; i < X; ++i) s[i * kRowsAtOnce + j] = __fma_rn(a[i], b, s[i * kRowsAtOnce + j]);
            }
        }
    }
    // each step a lane hands half of its sums to another and adds the other half; what is left is one sum a lane, or a part of it
    int n = X * (int)kRowsAtOnce, which = 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        if (n > 1) {
            n /= 2;
            const bool upper = lane & o;
            which += upper ? n : 0;
#pragma unroll
            for (int i = 0; i < X * (int)kRowsAtOnce / 2; ++i) {
                if (i >= n) break;
                const double mine = upper ? s[i + n] : s[i], other = upper ? s[i] : s[i + n];
                s[i] = mine + __shfl_xor_sync(0xFFFFFFFFu, other, o);
            }
        } else {
            s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], o);
        }
    }
    sums[warp][which] = s[0];                          // (lanes that share a sum have the same)
    __syncthreads();
    if (threadIdx.x >= X * kRowsAtOnce) return;
    const uint32_t e = e0 + threadIdx.x / kRowsAtOnce, t = t0 + threadIdx.x % kRowsAtOnce;
    if (e >= experts || t >= T) return;
    double all = 0.0;
#pragma unroll
    for (int w = 0; w < (int)kWorkers; ++w) all += sums[w][threadIdx.x];
    float* to = logits + (uint64_t)t * experts + e;
    if (ROWS_IN_ARRAY(status, to, 4, logits, logits + (uint64_t)T * experts)) *to = (float)all;
}

template <typename E, int V> int logits_launch(unsigned* status, const LayerExperts& a, float* logits, cudaStream_t s)
{
    const uint32_t fours = (a.T + kRowsAtOnce - 1) / kRowsAtOnce;
#define LOGITS(X)                                                                                                                             \
    rows_launch(logits_kernel<E, V, X>, dim3((a.E + X - 1) / X, fours), dim3(kWorkers * 32), 0, s, 0, status, a.T, a.D, a.E, (const E*)a.x, a.ld_x, \
                (const E*)a.router, logits)
    // Four experts a block where there are more than two blocks an SM without that.  Whole calls, hidden 16: 64 rows and 128 experts of width 4096 52 us, with one
    // a block 57, 28 rows and 64 experts 31 and 32; 16 rows and 64 experts 26.1 and 25.9, 4 rows and 128 experts 21.3 and 20.7
    return a.E * fours > 2 * rows_sm_count() ? LOGITS(4) : LOGITS(1);
#undef LOGITS
}

// ---- matrix instructions ----------------------------------------------------------------------------------------------
// acc += A B for 16 rows of weights and 8 columns over a block of 128 bytes of each: lane (g, t), g = lane / 4, has 32 bytes, piece t, of rows g
// and g + 8 of A and of column g of B.  Which element of a piece is which k of an instruction does not matter, as it is the same for both.
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
__device__ __forceinline__ void block_product(float (&c)[4], float (&d)[4], const RowsRaw<32>& a, const RowsRaw<32>& b, const RowsRaw<32>& x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) mma16(i % 2 ? d : c, a.r[2 * i], b.r[2 * i], a.r[2 * i + 1], b.r[2 * i + 1], x.r[2 * i], x.r[2 * i + 1], E());
}
// binary32 as the sum of two numbers of 11 bits, the upper one rounded to nearest (ties away from zero), by an addition to the bits: the conversion
// instruction, at a quarter of an SM's lanes, was what the products waited for (64 experts of 2048 x 1408 for 64 rows 579 us).  What is left has
// 12 bits at most and loses the last of them: nearest would be no nearer.  So a part is off by 2^-23 of the number, and a product, with that of the
// two lower parts left out, by 2^-21.  A NaN's upper part may be anything (the addition runs over into the sign for the largest); its lower one is a
// NaN, as cutting off bits leaves that one which arithmetic gives, and so is an infinity's.
__device__ __forceinline__ void split(RowsRaw<32>& high, RowsRaw<32>& low, const RowsRaw<32>& v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        high.r[i] = (v.r[i] + 0x1000u) & 0xFFFFE000u;
        low.r[i] = __float_as_uint(__uint_as_float(v.r[i]) - __uint_as_float(high.r[i])) & 0xFFFFE000u;
    }
}

// ---- the experts' products --------------------------------------------------------------------------------------------
// How a product is cut.  A piece has `strips` strips of 16 weight rows; `ways` warps share a strip (strips * ways = 8).  A stage of the ring
// holds `chunk` bytes, `across` blocks, of each of its weight rows and of each row of x (or h): the blocks one after the other, each of them
// rows of 128 bytes, whose 16-byte words are exchanged so that 8 rows of a column of words lie in different banks; or, where rows start between
// words, whole chunks, `pitch` apart.
struct Cut {
    uint32_t row_bytes, strips, ways, across, chunk, pitch, chunks, pieces;
};
Cut cut_as(uint32_t rows, uint32_t row_bytes, uint32_t ways, uint32_t across, bool words)
{
    Cut c;
    c.row_bytes = row_bytes;
    c.ways = ways;
    while (c.ways > 1 && c.ways / 2 * kBlockBytes >= row_bytes) c.ways /= 2;
    c.strips = kWorkers / c.ways;
    c.across = across > c.ways ? across : c.ways;
    while (c.across > c.ways && c.across / 2 * kBlockBytes >= row_bytes) c.across /= 2;
    c.chunk = kBlockBytes * c.across;
    c.pitch = c.chunk + (words ? 16 : 0);          // (the rest of a row that starts between two words)
    c.chunks = (row_bytes + c.chunk - 1) / c.chunk;
    c.pieces = ((rows + 15) / 16 + c.strips - 1) / c.strips;
    return c;
}
// Pieces of 128 rows in stages of 32 KB stream fastest; where an SM would not get two pieces of every three, smaller ones.  Measured with pieces of 128,
// 64 and 32 rows: 64 experts of 2048 x 1408 for 64 rows, binary16, 211, 265 and 400 us; 24 of 2048 x 768, a row each, 45, 47 and 62; 8 of 2048 x 2048 42,
// 39 and 51; 4 of them 31, 29 and 32; 2 of 512 x 1024 for one row 19, 17 and 16.
Cut cut_of(uint32_t rows, uint32_t row_bytes, uint32_t experts, bool words)
{
    uint32_t ways = 1;
    while (ways < 4 && 3ull * experts * cut_as(rows, row_bytes, ways, 1, words).pieces < 2ull * rows_sm_count()) ways *= 2;
    return cut_as(rows, row_bytes, ways, ways == 1 ? 2 : 4, words);
}
struct Args {
    uint32_t T, D, H, E, k, act;
    Cut up_cut, down_cut;
    const unsigned char *x, *x_end, *up, *up_end, *down, *down_end;
    uint64_t ld_x, ld_y, part;          // bytes; of a part of a slot's h
    const float* w;
    const int32_t* ids;
    unsigned char *y, *h;
    float* z;
    Counters* n;
    unsigned char* work_end;
    unsigned* status;
};
// What a CTA works on: a piece of a product of one expert, 16 weight rows for each of some strips, with some of its slots; or a part of y.
enum Kind : uint32_t { kUp, kDown, kSum, kEnd };
struct Item {
    uint32_t kind;
    uint32_t i, piece, first, columns;          // the expert's place among those asked for; of its slots
};
constexpr uint32_t kQueue = 16, kMaxStages = 16, kRingBytes = 188 * 1024;
struct Shared {
    float part[2][kWorkers][2 * 128];                  // the warps' sums of 16 columns of one strip, in turn
    uint64_t full[kMaxStages], empty[kMaxStages], queued[kQueue], ready[kQueue], done[kQueue];      // barriers
    Item item[kQueue];
    uint32_t count[PEARL_ROWS_MAX_EXPERTS];            // slots of an expert; then where its next one goes
    uint16_t expert[PEARL_ROWS_MAX_EXPERTS], first[PEARL_ROWS_MAX_EXPERTS + 1];       // of the experts that are asked for
    uint16_t slot[kMaxSlots];                          // by expert
    uint32_t sums[2][32];
    uint32_t asked, most, last;                        // experts asked for; the slots of the one that most ask for
};
constexpr uint32_t kSharedBytes = (sizeof(Shared) + 1023) / 1024 * 1024;

// The experts that are asked for, and their slots.
__device__ void plan(const Args& a, Shared& s)
{
    const uint32_t slots = a.T * a.k, tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5;
    for (uint32_t e = tid; e < a.E; e += blockDim.x) s.count[e] = 0;
    if (tid == 0) s.most = 0;
    __syncthreads();
    for (uint32_t i = tid; i < slots; i += blockDim.x) {
        const int32_t e = a.ids[i];
        if ((uint32_t)e < a.E) atomicAdd(&s.count[e], 1u);
        else if (e != -1 && blockIdx.x == 0) atomicOr(a.status, PEARL_ST_BAD_INDEX);
    }
    __syncthreads();
    // experts of the first 256 threads, four each
    constexpr uint32_t kEach = PEARL_ROWS_MAX_EXPERTS / 256;
    uint32_t mine[kEach], slots_here = 0, asked_here = 0, most = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = tid * kEach + i;
        mine[i] = e < a.E ? s.count[e] : 0u;
        slots_here += mine[i];
        asked_here += mine[i] != 0;
        most = max(most, mine[i]);
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    if (lane == 0 && most) atomicMax(&s.most, most);
    uint32_t slots_to = slots_here, asked_to = asked_here;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t p = __shfl_up_sync(0xFFFFFFFFu, slots_to, o), q = __shfl_up_sync(0xFFFFFFFFu, asked_to, o);
        if (lane >= (uint32_t)o) { slots_to += p; asked_to += q; }
    }
    if (lane == 31) { s.sums[0][warp] = slots_to; s.sums[1][warp] = asked_to; }
    __syncthreads();
    uint32_t at = slots_to - slots_here, i_asked = asked_to - asked_here;
    for (uint32_t w = 0; w < warp; ++w) { at += s.sums[0][w]; i_asked += s.sums[1][w]; }
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
    if (tid == 255) { s.asked = i_asked; s.first[i_asked] = (uint16_t)at; }
    __syncthreads();
    for (uint32_t i = tid; i < slots; i += blockDim.x) {
        const int32_t e = a.ids[i];
        if ((uint32_t)e < a.E) s.slot[atomicAdd(&s.count[e], 1u)] = (uint16_t)i;      // (in any order: no sum runs over an expert's slots)
    }
    __syncthreads();
}

// ---- barriers ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void workers_meet() { asm volatile("bar.sync 1, %0;" ::"n"(kWorkers * 32) : "memory"); }
__device__ __forceinline__ uint32_t read_acquired(const uint32_t* p)
{
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Polls until *p >= count; with a limit, of more than half a second.  Once it was reached -- the scratch was not zero, or two calls share it -- the polls behind it
// soon give up, too, so that a call does not take as many limits as it has experts.
__device__ __forceinline__ void poll(unsigned* status, const uint32_t* p, uint32_t count)
{
    for (uint32_t spins = 0; read_acquired(p) < count; ++spins)
        if (spins > kSpins || (spins % 1024 == 1023 && (read_acquired(status) & PEARL_ST_INTERNAL))) {
            atomicOr(status, PEARL_ST_INTERNAL);
            break;
        }
}

// ---- copies -------------------------------------------------------------------------------------------------------------
struct Ring {
    unsigned char* base;
    uint32_t stages, bytes, x_at;       // bytes of a stage; where the rows of x are in it
    uint32_t columns;                   // rows of x (or h) that it has room for, at most
};
// (the lower parts of h lie behind all the upper ones)
template <typename E> __host__ __device__ __forceinline__ Ring ring_of(unsigned char* base, const Cut& up, const Cut& down, uint32_t most)
{
    Ring r;
    r.base = base;
    r.columns = most <= 8 ? 8u : most <= 16 ? 16u : most <= 32 ? 32u : kMaxColumns<E>;
    const uint32_t weights = up.strips * up.pitch > down.strips * down.pitch ? up.strips * up.pitch : down.strips * down.pitch;
    const uint32_t rows = up.pitch > kParts<E> * down.pitch ? up.pitch : kParts<E> * down.pitch;
    r.x_at = (weights * 16 + 1023) / 1024 * 1024;
    r.bytes = r.x_at + (r.columns * rows + 1023) / 1024 * 1024;
    r.stages = kRingBytes / r.bytes < kMaxStages ? kRingBytes / r.bytes : kMaxStages;
    return r;
}
// A place in the ring, one turn after the other.
struct Place {
    uint32_t stage, round;
    __device__ __forceinline__ void step(const Ring& r) { if (++stage == r.stages) { stage = 0; ++round; } }
};

// A box of a matrix of weights (map_of): 128 bytes of each row from row `row` of group `group` on, for as many blocks from `block` on as the
// map says; or of one, from element `column` on.
__device__ __forceinline__ void copy_blocks(uint64_t* barrier, unsigned char* to, const CUtensorMap* map, uint32_t row, uint32_t group, uint32_t block)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(layer_address(to)), "l"(map), "r"(0), "r"(row), "r"(group), "r"(block), "r"(layer_address(barrier)) : "memory");
}
__device__ __forceinline__ void copy_block(uint64_t* barrier, unsigned char* to, const CUtensorMap* map, uint32_t column, uint32_t row, uint32_t group)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(layer_address(to)), "l"(map), "r"(column), "r"(row), "r"(group), "r"(layer_address(barrier)) : "memory");
}
// The 16-byte word at `from`, of which `bytes` are read, zeros for the rest.  (A word that an array begins in is read whole.)
__device__ __forceinline__ void copy_word(uint32_t to, const unsigned char* from, uint32_t bytes, const unsigned char* lo, const unsigned char* hi,
                                          const Args& a)
{
    if (bytes == 0 || !ROWS_IN_ARRAY(a.status, from, bytes, (uintptr_t)lo & ~(uintptr_t)15, hi)) { from = (const unsigned char*)a.n; bytes = 0; }
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// An arrival when this thread's words are there.
__device__ __forceinline__ void arrive_with_words(uint64_t* barrier)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(layer_address(barrier)) : "memory");
}

// Whose rows (the first products', the second ones') are whole words: tensor copies bring them.
constexpr int kUpWhole = 1, kDownWhole = 2, kWhole = 3;
template <int kAlign> __device__ __forceinline__ bool whole_words(uint32_t kind) { return kind == kUp ? (kAlign & kUpWhole) != 0 : (kAlign & kDownWhole) != 0; }
// The warps that bring weights: one thread of one; eight warps where words have to be cut out of rows.  (21 warps then, 80 registers a thread, of which the
// products spill 0.8 to 1.7 KB: what such rows cost beside the cutting.)
template <int kAlign> constexpr uint32_t kWeightWarps = kAlign == kWhole ? 1 : 8;
// Those that bring the rows of x or h.
constexpr uint32_t kRowWarps = 4;
template <int kAlign> constexpr uint32_t kThreads = (kWorkers + 1 + kRowWarps + kWeightWarps<kAlign>) * 32;

// The rows of a stage: those of the strips one after the other; with gates, all strips' gates (8 each) before all their values.
// The first byte of row r of a piece's strips * 16, null if there is none.
template <typename E> __device__ __forceinline__ const unsigned char* weight_row(const Args& a, const Shared& s, const Cut& c, const Item& it, uint32_t r)
{
    const bool gated = it.kind == kUp && a.act == PEARL_ACT_SILU_GATED;
    const uint32_t rows = it.kind == kDown ? a.D : a.H, half = c.strips * 8;
    const bool value = gated && r >= half;
    const uint32_t j = gated ? it.piece * half + (value ? r - half : r) : it.piece * half * 2 + r;
    if (j >= rows) return nullptr;
    const unsigned char* m = (it.kind == kDown ? a.down : a.up) + (uint64_t)s.expert[it.i] * rows * (gated ? 2 : 1) * c.row_bytes;
    return m + (uint64_t)(value ? rows + j : j) * c.row_bytes;
}

// The warp (or warps) that brings weights into the ring.
template <typename E, int kAlign>
__device__ void bring_weights(const Args& a, Shared& s, const Ring& r, uint32_t warp, const CUtensorMap* up_map, const CUtensorMap* down_map)
{
    const uint32_t lane = threadIdx.x & 31u;
    Place at = { 0, 0 };
    for (uint32_t n = 0;; ++n) {
        layer_wait(a.status, s.queued + n % kQueue, n / kQueue);
        const Item it = s.item[n % kQueue];
        if (it.kind == kEnd) break;
        if (it.kind == kUp || it.kind == kDown) {
            const Cut& c = it.kind == kDown ? a.down_cut : a.up_cut;
            if (whole_words<kAlign>(it.kind)) {
                const bool gated = it.kind == kUp && a.act == PEARL_ACT_SILU_GATED;
                const uint32_t row = it.piece * c.strips * (gated ? 8 : 16), group = s.expert[it.i] * (gated ? 2 : 1);
                const bool whole = c.row_bytes % kBlockBytes == 0;
                const CUtensorMap* map = it.kind == kDown ? down_map : up_map;
                for (uint32_t k = 0; k < c.chunks; ++k, at.step(r)) {
                    layer_wait(a.status, s.empty + at.stage, at.round + 1);
                    if (warp != 0 || lane != 0) {
                        if (kAlign != kWhole) layer_arrive(s.full + at.stage);           // (as many arrive for a stage of either kind)
                        continue;
                    }
                    unsigned char* to = r.base + at.stage * r.bytes;
                    layer_arrive_with(s.full + at.stage, c.strips * 16 * c.chunk);
                    if (whole) {
                        copy_blocks(s.full + at.stage, to, map, row, group, k * c.across);
                    } else {
                        for (uint32_t b = 0; b < c.across; ++b, to += c.strips * 16 * kBlockBytes)
                            copy_block(s.full + at.stage, to, map, (k * c.across + b) * (kBlockBytes / (uint32_t)sizeof(E)), row, group);
                    }
                }
            } else if constexpr (kAlign != kWhole) {
                // a lane has a word of a block of every 32nd row, and the first of eight lanes the word behind the chunk
                const unsigned char *lo = it.kind == kDown ? a.down : a.up, *hi = it.kind == kDown ? a.down_end : a.up_end;
                const uint32_t w = lane & 7u, first = warp * 4 + (lane >> 3);
                const unsigned char* from[4];
                int here[4], left[4];                   // bytes from there on: of the row, and of the array
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    const uint32_t row = first + i * 32;
                    const unsigned char* p = row < c.strips * 16 ? weight_row<E>(a, s, c, it, row) : nullptr;
                    from[i] = p - ((uintptr_t)p & 15u) + w * 16;
                    here[i] = p ? (int)c.row_bytes + (int)((uintptr_t)p & 15u) - (int)(w * 16) : 0;
                    left[i] = p ? (int)min((long long)(hi - from[i]), (long long)1 << 30) : 0;
                }
                for (uint32_t k = 0; k < c.chunks; ++k, at.step(r)) {
                    layer_wait(a.status, s.empty + at.stage, at.round + 1);
                    const uint32_t to = layer_address(r.base) + at.stage * r.bytes + first * c.pitch + w * 16;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        for (uint32_t b = 0; b < c.across + (w == 0); ++b) {
                            const int off = (int)(k * c.chunk + b * kBlockBytes);
                            if (off < here[i]) copy_word(to + i * 32 * c.pitch + b * kBlockBytes, from[i] + off, (uint32_t)min(16, left[i] - off), lo, hi, a);
                        }
                    arrive_with_words(s.full + at.stage);
                }
            }
        }
        __syncwarp();
        if (lane == 0) layer_arrive(s.done + n % kQueue);
    }
}

// The warps that bring the rows of x or h, and wait for what items need: h for a second product, all z for a part of y.
template <typename E, int kAlign> __device__ void bring_rows(const Args& a, Shared& s, const Ring& r, uint32_t warp)
{
    const uint32_t lane = threadIdx.x & 31u;
    Place at = { 0, 0 };
    uint32_t known = 0;                             // experts (in order) whose first product is there
    bool summed = false;
    for (uint32_t n = 0;; ++n) {
        layer_wait(a.status, s.queued + n % kQueue, n / kQueue);
        const Item it = s.item[n % kQueue];
        if (it.kind == kEnd) break;
        if (it.kind == kSum) {
            if (warp == 0 && lane == 0) {
                if (!summed) poll(a.status, &a.n->down, s.asked * a.down_cut.pieces);
                layer_arrive(s.ready + n % kQueue);
            }
            summed = true;
        } else {
            if (warp == 0 && lane == 0) layer_arrive(s.ready + n % kQueue);
            if (it.kind == kDown && it.i >= known) {
                if (lane == 0) poll(a.status, &a.n->up[it.i], a.up_cut.pieces);
                __syncwarp();
                known = it.i + 1;
            }
            const Cut& c = it.kind == kDown ? a.down_cut : a.up_cut;
            const uint32_t parts = it.kind == kDown ? kParts<E> : 1u;
            // Rows that there are none of are not brought: a column of a product goes by its own row alone.
            const uint32_t rows = it.columns * parts;
            const auto part_of = [&](uint32_t row) { return (row >= it.columns ? 1u : 0u) + (row >= 2 * it.columns ? 1u : 0u); };
            const auto place_of = [&](uint32_t row) { return row + part_of(row) * (r.columns - it.columns); };
            const auto row_at = [&](uint32_t row) {
                const uint32_t part = part_of(row), slot = s.slot[it.first + row - part * it.columns];
                return it.kind == kDown ? a.h + (slot * kMostParts + part) * a.part : a.x + (uint64_t)(slot / a.k) * a.ld_x;
            };
            const unsigned char *lo = it.kind == kDown ? a.h : a.x, *hi = it.kind == kDown ? (const unsigned char*)a.z : a.x_end;
            if (whole_words<kAlign>(it.kind)) {
                // a lane's word of a block, of its first row (of 16, the four warps have four each)
                const uint32_t w = lane & 7u, first = warp * 4 + (lane >> 3), from_block = r.columns * parts * kBlockBytes;
                const unsigned char* from = first < rows ? row_at(first) + w * 16 : nullptr;
                const uint32_t place = place_of(first);
                const uint32_t to = layer_address(r.base) + r.x_at + place * kBlockBytes + ((w ^ (place & 7u)) * 16);
                for (uint32_t k = 0; k < c.chunks; ++k, at.step(r)) {
                    layer_wait(a.status, s.empty + at.stage, at.round + 1);
                    if (from) {
                        const int left = (int)(c.row_bytes - k * c.chunk - w * 16);
                        const unsigned char* p = from + k * c.chunk;
                        uint32_t q = to + at.stage * r.bytes;
#pragma unroll 2
                        for (uint32_t b = 0; b < c.across; ++b, p += kBlockBytes, q += from_block) copy_word(q, p, left > (int)(b * kBlockBytes) ? 16u : 0u, lo, hi, a);
                        for (uint32_t row = first + 16; row < rows; row += 16) {
                            const uint32_t there = place_of(row);
                            p = row_at(row) + w * 16 + k * c.chunk;
                            q = layer_address(r.base) + at.stage * r.bytes + r.x_at + there * kBlockBytes + ((w ^ (there & 7u)) * 16);
                            for (uint32_t b = 0; b < c.across; ++b, p += kBlockBytes, q += from_block) copy_word(q, p, left > (int)(b * kBlockBytes) ? 16u : 0u, lo, hi, a);
                        }
                    }
                    arrive_with_words(s.full + at.stage);
                }
            } else if constexpr (kAlign != kWhole) {
                const uint32_t w = lane & 7u, first = warp * 4 + (lane >> 3);
                const unsigned char* at_first = first < rows ? row_at(first) : nullptr;
                for (uint32_t k = 0; k < c.chunks; ++k, at.step(r)) {
                    layer_wait(a.status, s.empty + at.stage, at.round + 1);
                    const uint32_t to = layer_address(r.base) + at.stage * r.bytes + r.x_at + w * 16;
                    for (uint32_t row = first; row < rows; row += 16) {
                        const unsigned char* from = row == first ? at_first : row_at(row);
                        const unsigned char *end = from + c.row_bytes, *p = from - ((uintptr_t)from & 15u) + k * c.chunk + w * 16;
                        uint32_t q = to + place_of(row) * c.pitch;
                        for (uint32_t b = 0; b < c.across + (w == 0); ++b, p += kBlockBytes, q += kBlockBytes)
                            if (p < end) copy_word(q, p, (uint32_t)min((long long)16, (long long)(hi - p)), lo, hi, a);
                    }
                    arrive_with_words(s.full + at.stage);
                }
            }
        }
        __syncwarp();
        if (lane == 0) layer_arrive(s.done + n % kQueue);
    }
}

// ---- what the warps that multiply do ------------------------------------------------------------------------------------
// 32 bytes at p, `off` bytes further on where rows start between words; those from `bytes` on are 0 with kTail.
template <int kAlign> __device__ __forceinline__ RowsRaw<32> piece_at(const unsigned char* p, uint32_t off, int bytes, bool tail)
{
    RowsRaw<32> v;
    const uint4* q = reinterpret_cast<const uint4*>(p);
    const uint4 x = q[0], y = kAlign ? *reinterpret_cast<const uint4*>((uintptr_t)p ^ 16u) : q[1];
    if constexpr (kAlign != 0) {
        v.r[0] = x.x; v.r[1] = x.y; v.r[2] = x.z; v.r[3] = x.w; v.r[4] = y.x; v.r[5] = y.y; v.r[6] = y.z; v.r[7] = y.w;
    } else {
        const uint4 z = q[2];
        uint32_t w[12] = { x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w };
#pragma unroll
        for (int i = 0; i < 10; ++i) w[i] = off & 8u ? w[i + 2] : w[i];
#pragma unroll
        for (int i = 0; i < 9; ++i) w[i] = off & 4u ? w[i + 1] : w[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v.r[i] = __funnelshift_r(w[i], w[i + 1], (off & 3u) * 8u);
    }
    if (tail) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (4 * i >= bytes) v.r[i] = 0u;
            else if (4 * i + 2 >= bytes) v.r[i] &= 0xFFFFu;
        }
    }
    return v;
}

__device__ __forceinline__ float activated(float gate, float value) { return gate / (1.0f + expf(-gate)) * value; }

// h[slot][j] = v, as the sum of parts that keeps a binary32's digits: three of bfloat16's 8 bits each, which is all of them; two of binary16's
// 11, the second one times 2^11, so that it runs out of exponents that much later: 2^-22 of h, and 2^-36.  (With two of bfloat16 seven times as many results
// had another last place than those of a sum in 64 bits, 2.4 in 1000 of the layer of 64 rows and 128 experts of 4096 x 1280; it took 702 us, this 735.)
constexpr float kLowerHalf = 2048.0f;
template <typename E> __device__ __forceinline__ void store_h(const Args& a, uint32_t slot, uint32_t j, float v)
{
    unsigned char* row = a.h + slot * kMostParts * a.part;
    if (!ROWS_IN_ARRAY(a.status, row + (uint64_t)j * sizeof(E), (kParts<E> - 1) * a.part + sizeof(E), a.h, a.z)) return;
    if constexpr (sizeof(E) == 4) {
        reinterpret_cast<float*>(row)[j] = v;
    } else {
        E part = RowsElem<E>::down(v);
        reinterpret_cast<E*>(row)[j] = part;
        float rest = isfinite(RowsElem<E>::up(part)) ? v - RowsElem<E>::up(part) : 0.0f;
        if constexpr (kParts<E> == 2) {
            reinterpret_cast<E*>(row + a.part)[j] = RowsElem<E>::down(rest * kLowerHalf);
        } else {
            part = RowsElem<E>::down(rest);
            reinterpret_cast<E*>(row + a.part)[j] = part;
            rest -= RowsElem<E>::up(part);
            reinterpret_cast<E*>(row + 2 * a.part)[j] = RowsElem<E>::down(rest);
        }
    }
}

// A warp's share of one piece, with up to 8 NT columns.
template <typename E, int kAlign, int NT, uint32_t kKind>
__device__ __forceinline__ void product(const Args& a, Shared& s, const Ring& r, const Item& it, uint32_t number, Place& at, uint32_t& swaps)
{
    constexpr bool k32 = sizeof(E) == 4, kSecond = kKind == kDown;
    constexpr int kHow = kAlign & (kSecond ? kDownWhole : kUpWhole);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3u;
    const Cut& c = kSecond ? a.down_cut : a.up_cut;
    const uint32_t way = warp % c.ways, strip = warp / c.ways;
    const bool gated = !kSecond && a.act == PEARL_ACT_SILU_GATED;
    const uint32_t rows = kSecond ? a.D : a.H;
    const uint32_t j0 = (it.piece * c.strips + strip) * (gated ? 8u : 16u), ja = j0 + g, jb = gated ? ja : j0 + 8 + g;
    // the lane's rows in a stage
    const uint32_t ra = strip * (gated ? 8 : 16) + g, rb = gated ? ra + c.strips * 8 : ra + 8;
    // (and from one block to the next)
    const uint32_t to_a = kHow ? ra * kBlockBytes + ((2 * t) ^ g) * 16 : ra * c.pitch + t * 32, to_next = kHow ? c.strips * 16 * kBlockBytes : kBlockBytes;
    const uint32_t to_b = kHow ? rb * kBlockBytes + ((2 * t) ^ g) * 16 : rb * c.pitch + t * 32;
    uint32_t off_a = 0, off_b = 0;
    if constexpr (kHow == 0) {
        off_a = (uint32_t)(uintptr_t)weight_row<E>(a, s, c, it, ra) & 15u;
        off_b = (uint32_t)(uintptr_t)weight_row<E>(a, s, c, it, rb) & 15u;
    }
    const uint32_t pitch = kHow ? kBlockBytes : c.pitch;
    const uint32_t to_x = r.x_at + (kHow ? g * kBlockBytes + ((2 * t) ^ g) * 16 : g * pitch + t * 32);
    const uint32_t to_next_x = kHow ? r.columns * (kSecond ? kParts<E> : 1) * kBlockBytes : kBlockBytes;
    uint32_t off_x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint32_t col = n * 8 + g;
        off_x[n] = kHow || kSecond || col >= it.columns ? 0u : (uint32_t)(uintptr_t)(a.x + (uint64_t)(s.slot[it.first + col] / a.k) * a.ld_x) & 15u;
    }
    // Two sums of 16-bit products over a stage, so that an instruction need not wait for the one before (the second product's: of h's upper parts, of
    // the others).  Where a sum grows the instruction cuts off, so what a stage has is added to the sum so far by additions that round.
    float acc[NT][4], pair[NT][2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[n][q] = pair[n][0][q] = pair[n][1][q] = 0.0f;
    for (uint32_t k = 0; k < c.chunks; ++k, at.step(r)) {
        layer_wait(a.status, s.full + at.stage, at.round);
        for (uint32_t block = way; block < c.across; block += c.ways) {
            const unsigned char* stage = r.base + at.stage * r.bytes;
            const int left = (int)c.row_bytes - (int)(k * c.chunk + block * kBlockBytes);         // of the row from the block on
            if (left <= 0) break;
            const bool tail = kHow == 0 && left < (int)kBlockBytes;        // (else both sides have zeros there)
            const int here = left - (int)(t * 32);                           // from the lane's piece on
            const RowsRaw<32> va = piece_at<kHow>(stage + block * to_next + to_a, off_a, here, tail), vb = piece_at<kHow>(stage + block * to_next + to_b, off_b, here, tail);
            stage += block * to_next_x;
            RowsRaw<32> ah, al, bh, bl;
            if constexpr (k32) {
                split(ah, al, va);
                split(bh, bl, vb);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const RowsRaw<32> x = piece_at<kHow>(stage + to_x + n * 8 * pitch, off_x[n], here, tail);
                if constexpr (k32) {
                    RowsRaw<32> xh, xl;
                    split(xh, xl, x);
                    // (the instruction cuts off where an addition rounds: sums of a block only; three, which do not wait for one another)
                    float part[3][4] = {};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        mma8(part[0], al.r[2 * q], bl.r[2 * q], al.r[2 * q + 1], bl.r[2 * q + 1], xh.r[2 * q], xh.r[2 * q + 1]);
                        mma8(part[1], ah.r[2 * q], bh.r[2 * q], ah.r[2 * q + 1], bh.r[2 * q + 1], xl.r[2 * q], xl.r[2 * q + 1]);
                        mma8(part[2], ah.r[2 * q], bh.r[2 * q], ah.r[2 * q + 1], bh.r[2 * q + 1], xh.r[2 * q], xh.r[2 * q + 1]);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[n][q] += (part[0][q] + part[1][q]) + part[2][q];
                } else {
                    block_product<E>(pair[n][0], kSecond ? pair[n][0] : pair[n][1], va, vb, x);
#pragma unroll
                    for (uint32_t part = 1; kSecond && part < kParts<E>; ++part)
                        block_product<E>(pair[n][1], pair[n][1], va, vb, piece_at<kHow>(stage + to_x + (part * r.columns + n * 8) * pitch, 0u, here, tail));
                }
            }
        }
        __syncwarp();
        if (lane == 0) layer_arrive(s.empty + at.stage);
        if constexpr (!k32) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float rest = kSecond && kParts<E> == 2 ? pair[n][1][q] * (1.0f / kLowerHalf) : pair[n][1][q];
                    // (an infinite weight: what it makes of the upper part)
                    if (kSecond && !isfinite(pair[n][0][q])) rest = 0.0f;
                    acc[n][q] += pair[n][0][q] + rest;
                    pair[n][0][q] = pair[n][1][q] = 0.0f;
                }
        }
    }
    // the warps that share a strip: their sums in order, 16 columns at a time
    if (c.ways > 1) {
#pragma unroll
        for (int n0 = 0; n0 < NT; n0 += 2) {
            float(*part)[256] = s.part[swaps++ & 1u];
#pragma unroll
            for (int n = n0; n < NT && n < n0 + 2; ++n)
                *reinterpret_cast<float4*>(part[warp] + (n - n0) * 128 + lane * 4) = make_float4(acc[n][0], acc[n][1], acc[n][2], acc[n][3]);
            workers_meet();
            if (way != 0) continue;
#pragma unroll
            for (int n = n0; n < NT && n < n0 + 2; ++n)
                for (uint32_t w = 1; w < c.ways; ++w) {
                    const float4 v = *reinterpret_cast<const float4*>(part[warp + w] + (n - n0) * 128 + lane * 4);
                    acc[n][0] += v.x; acc[n][1] += v.y; acc[n][2] += v.z; acc[n][3] += v.w;
                }
        }
    }
    if (way != 0) return;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t col = n * 8 + t * 2 + q;
            if (col >= it.columns) continue;
            const uint32_t slot = s.slot[it.first + col];
            if constexpr (kSecond) {
                float* z = a.z + (uint64_t)slot * a.D;
                if (ja < rows && ROWS_IN_ARRAY(a.status, z + ja, 4, a.z, a.work_end)) z[ja] = acc[n][q];
                if (jb < rows && ROWS_IN_ARRAY(a.status, z + jb, 4, a.z, a.work_end)) z[jb] = acc[n][q + 2];
            } else {
                const auto store = [&](uint32_t j, float v) { if (j < rows) store_h<E>(a, slot, j, v); };
                if (gated) {
                    store(ja, activated(acc[n][q], acc[n][q + 2]));
                } else {
                    store(ja, acc[n][q] < 0.0f ? 0.0f : acc[n][q]);
                    store(jb, acc[n][q + 2] < 0.0f ? 0.0f : acc[n][q + 2]);
                }
            }
        }
}

template <typename E, int kAlign, uint32_t kKind>
__device__ __forceinline__ void product_of(const Args& a, Shared& s, const Ring& r, const Item& it, uint32_t number, Place& at, uint32_t& swaps)
{
    if (it.columns <= 8) product<E, kAlign, 1, kKind>(a, s, r, it, number, at, swaps);
    else if (it.columns <= 16) product<E, kAlign, 2, kKind>(a, s, r, it, number, at, swaps);
    else if (kMaxColumns<E> == 32 || it.columns <= 32) product<E, kAlign, 4, kKind>(a, s, r, it, number, at, swaps);
    else product<E, kAlign, kMaxColumns<E> / 8, kKind>(a, s, r, it, number, at, swaps);
}

// A part of y, of `parts`: the slots' sums in the order of the choices.
template <typename E> __device__ void weighted_sums(const Args& a, uint32_t part, uint32_t parts)
{
    const uint64_t all = (uint64_t)a.T * a.D, each = (all + parts - 1) / parts, end = min(all, (part + 1) * each);
    for (uint64_t n = part * each + threadIdx.x; n < end; n += kWorkers * 32) {
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

template <typename E, int kAlign>
__device__ void multiply(const Args& a, Shared& s, const Ring& r, uint32_t parts)
{
    Place at = { 0, 0 };
    uint32_t swaps = 0;
    for (uint32_t n = 0;; ++n) {
        layer_wait(a.status, s.queued + n % kQueue, n / kQueue);
        const Item it = s.item[n % kQueue];
        if (it.kind == kEnd) break;
        if (it.kind == kUp) {
            product_of<E, kAlign, kUp>(a, s, r, it, n, at, swaps);
        } else if (it.kind == kDown) {
            product_of<E, kAlign, kDown>(a, s, r, it, n, at, swaps);
        } else {
            layer_wait(a.status, s.ready + n % kQueue, n / kQueue);
            weighted_sums<E>(a, it.piece, parts);
        }
        __syncwarp();
        if ((threadIdx.x & 31u) == 0) layer_arrive(s.done + n % kQueue);
    }
}

// The thread that keeps the books.  It takes pieces in order -- all first products' before the second ones', these before the parts of y --,
// hands them to the others, some way ahead, and tells what is finished.  It alone fences, and it has no copies on their way, for which a fence
// would wait.  A CTA waits only with its earlier pieces told, and each piece that it waits for is with a CTA that runs: nobody waits for
// one that is yet to be launched.
template <typename E> __device__ void keep_books(const Args& a, Shared& s, const Ring& r, uint32_t parts, uint32_t ticket)
{
    const Cut &up = a.up_cut, &down = a.down_cut;
    const uint32_t ups = s.asked * up.pieces, downs = s.asked * down.pieces;
    Item last = { kEnd, 0, 0, 0, 0 };
    const auto more = [&](const Item& it) { return it.kind <= kDown && it.first + it.columns < s.first[it.i + 1]; };
    const auto take = [&] {
        Item it = { kEnd, 0, 0, 0, 0 };
        if (more(last)) {                    // an expert of more slots is gone over again
            it = last;
            it.first = last.first + last.columns;
            it.columns = min(s.first[it.i + 1] - it.first, kMaxColumns<E>);
            return it;
        }
        const uint32_t task = ticket;
        if (task >= ups + downs + parts) return it;
        ticket = atomicAdd(&a.n->ticket, 1u);
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
        it.columns = min(s.first[it.i + 1] - it.first, kMaxColumns<E>);
        return it;
    };
    const auto stages = [&](const Item& it) { return it.kind == kUp ? up.chunks : it.kind == kDown ? down.chunks : 0u; };
    uint32_t given = 0, told = 0, ahead = 0;             // items; stages of those given and not told
    bool ended = false;
    for (;;) {
        while (!ended && given - told < kQueue && (given == told || ahead < r.stages)) {
            last = take();
            s.item[given % kQueue] = last;
            layer_arrive(s.queued + given % kQueue);
            ++given;
            ahead += stages(last);
            ended = last.kind == kEnd;
        }
        if (ended && told + 1 == given) break;
        layer_wait(a.status, s.done + told % kQueue, told / kQueue);
        const Item it = s.item[told % kQueue];
        if (it.kind != kSum && !more(it)) {
            __threadfence();
            atomicAdd(it.kind == kUp ? &a.n->up[it.i] : &a.n->down, 1u);
        }
        ahead -= stages(it);
        ++told;
    }
}

template <typename E, int kAlign>
__global__ void __launch_bounds__(kThreads<kAlign>, 1) experts_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap up_map,
                                                                      const __grid_constant__ CUtensorMap down_map)
{
    extern __shared__ __align__(1024) unsigned char memory[];
    Shared& s = *reinterpret_cast<Shared*>(memory);
    const uint32_t warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < kMaxStages; ++i) {
            layer_barrier(s.full + i, 32 * kRowWarps + (kAlign == kWhole ? 1 : 32 * kWeightWarps<kAlign>));
            layer_barrier(s.empty + i, kWorkers);
        }
        for (uint32_t i = 0; i < kQueue; ++i) {
            layer_barrier(s.queued + i, 1);
            layer_barrier(s.ready + i, 1);
            layer_barrier(s.done + i, kWorkers + kRowWarps + kWeightWarps<kAlign>);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    rows_begin();
    uint32_t ticket = 0;
    if (threadIdx.x == kWorkers * 32) ticket = atomicAdd(&a.n->ticket, 1u);
    plan(a, s);
    const Ring r = ring_of<E>(memory + kSharedBytes, a.up_cut, a.down_cut, s.most);
    const uint32_t parts = min(gridDim.x, (uint32_t)(((uint64_t)a.T * a.D + kWorkers * 32 - 1) / (kWorkers * 32)));
    if (warp < kWorkers) multiply<E, kAlign>(a, s, r, parts);
    else if (threadIdx.x == kWorkers * 32) keep_books<E>(a, s, r, parts, ticket);
    else if (warp > kWorkers + kRowWarps) bring_weights<E, kAlign>(a, s, r, warp - kWorkers - kRowWarps - 1, &up_map, &down_map);
    else if (warp > kWorkers) bring_rows<E, kAlign>(a, s, r, warp - kWorkers - 1);
    __syncwarp();
    __syncthreads();
    // the last one out leaves the counters as they were
    if (threadIdx.x == 0) s.last = atomicAdd(&a.n->finished, 1u) + 1 == gridDim.x;
    __syncthreads();
    if (!s.last) return;
    for (uint32_t i = threadIdx.x; i < s.asked; i += blockDim.x) a.n->up[i] = 0;
    if (threadIdx.x == 0) a.n->ticket = a.n->finished = a.n->down = 0;
}

// A map of the weights' `groups` matrices of `rows` rows of `length` elements.  A box has 128 bytes of each of its rows: with rows of whole blocks
// of 128 bytes, of each of c.across blocks, brought by one operation -- one takes some 200 cycles, however much it brings (boxes of 4 KB
// instead of 16 made the streaming of 4 GB take twice as long).
bool map_of(CUtensorMap* map, uint32_t dtype, const void* base, uint64_t length, uint64_t rows, uint64_t groups, const Cut& c, uint32_t box_rows, uint32_t box_groups)
{
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<void*> known;
    void* p = known;
    if (!p) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return false;
        known = p;
    }
    const uint32_t size = rows_elem_bytes(dtype), elements = kBlockBytes / size;
    const bool whole = length % elements == 0;
    const cuuint64_t dims[4] = { whole ? elements : length, rows, groups, length / elements }, strides[3] = { length * size, rows * length * size, kBlockBytes };
    const cuuint32_t box[4] = { elements, box_rows, box_groups, c.across }, steps[4] = { 1, 1, 1, 1 };
    const CUtensorMapDataType type = dtype == PEARL_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == PEARL_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                                                             : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return ((Encode)p)(map, type, whole ? 4 : 3, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kAlign> int experts_launch(const Args& a, uint32_t dtype, cudaStream_t s)
{
    static std::atomic<bool> ready[kRowsMaxDevices];
    const int dev = rows_device();
    if (dev < 0 || !ready[dev]) {
        if (cudaFuncSetAttribute(experts_kernel<T, kAlign>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kSharedBytes + kRingBytes)) != cudaSuccess) return -1;
        if (dev >= 0) ready[dev] = true;
    }
    CUtensorMap up = {}, down = {};
    const bool gated = a.act == PEARL_ACT_SILU_GATED;
    if (((kAlign & kUpWhole) &&
         !map_of(&up, dtype, a.up, a.D, a.H, (uint64_t)a.E * (gated ? 2 : 1), a.up_cut, a.up_cut.strips * (gated ? 8 : 16), gated ? 2 : 1)) ||
        ((kAlign & kDownWhole) && !map_of(&down, dtype, a.down, a.H, a.D, a.E, a.down_cut, a.down_cut.strips * 16, 1)))
        return -1;
    return rows_launch(experts_kernel<T, kAlign>, dim3(rows_sm_count()), dim3(kThreads<kAlign>), kSharedBytes + kRingBytes, s, 0, a, up, down);
}

template <typename T> int experts_as(unsigned* status, const LayerExperts& a, cudaStream_t s)
{
    const Layout l = layout_of(a.T, a.D, a.H, a.E, a.k);
    float* logits = (float*)((char*)a.work + l.logits);
    int n = 0, m;
    if (a.router) {
        constexpr int V = 16 / (int)sizeof(T);
        const uint32_t granule = rows_granule((uintptr_t)a.x, (uintptr_t)a.router, a.ld_x * sizeof(T), (uint64_t)a.D * sizeof(T));
        if ((m = granule >= 16 ? logits_launch<T, V>(status, a, logits, s) : logits_launch<T, 1>(status, a, logits, s)) < 0) return m;
        n += m;
        if ((m = rows_launch_route(status, a.T, a.E, a.k, PEARL_F32, logits, a.E, a.over_chosen, a.w, a.ids, s)) < 0) return m;
        n += m;
    }
    constexpr uint32_t S = sizeof(T);
    unsigned char* work = (unsigned char*)a.work;
    const unsigned char* x = (const unsigned char*)a.x;
    const unsigned char *up = (const unsigned char*)a.up, *down = (const unsigned char*)a.down;
    const uint64_t matrix = (uint64_t)a.E * a.D * a.H * S;
    Args args = { a.T, a.D, a.H, a.E, a.k, a.act, Cut(), Cut(), x, x + ((uint64_t)(a.T - 1) * a.ld_x + a.D) * S, up,
                        up + matrix * (a.act == PEARL_ACT_SILU_GATED ? 2 : 1), down, down + matrix, a.ld_x * S, a.ld_y * S, l.part, a.w, a.ids,
                        (unsigned char*)a.y, work + l.h, (float*)(work + l.z), (Counters*)work, work + l.bytes, status };
    const bool gated = a.act == PEARL_ACT_SILU_GATED;
    const bool up_whole = rows_granule((uintptr_t)a.x, (uintptr_t)a.up, a.ld_x * S, (uint64_t)a.D * S) >= 16, down_whole = rows_granule((uintptr_t)a.down, (uint64_t)a.H * S) >= 16;
    const uint32_t rows = gated ? a.H * 2 : a.H, slots = a.T * a.k, experts = slots < a.E ? slots : a.E;
    args.up_cut = cut_of(rows, a.D * S, experts, !up_whole);
    args.down_cut = cut_of(a.D, a.H * S, experts, !down_whole);
    if (ring_of<T>(nullptr, args.up_cut, args.down_cut, slots).stages < 2) {       // many rows for few experts: smaller stages
        args.up_cut = cut_as(rows, a.D * S, 1, 1, !up_whole);
        args.down_cut = cut_as(a.D, a.H * S, 1, 1, !down_whole);
    }
    m = up_whole ? (down_whole ? experts_launch<T, kWhole>(args, a.dtype, s) : experts_launch<T, kUpWhole>(args, a.dtype, s))
                 : (down_whole ? experts_launch<T, kDownWhole>(args, a.dtype, s) : experts_launch<T, 0>(args, a.dtype, s));
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
