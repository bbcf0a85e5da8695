// Attention over the paged 8-bit cache for many query rows a sequence (prompt chunks): matrix products on the fifth-generation
// tensor cores, accumulators in tensor memory.
//
// A block (640 threads, one an SM) takes kTiles tiles of 128 rows of one key head - a row is one (token, query head) of the
// group - through the keys 128 at a time, in two halves of 64:
//   S = q K^T        both operands in shared memory, float16; S in tensor memory, 64 columns a half
//   softmax          a thread owns a row: reads S, writes the probabilities as float16 over the columns it has read
//   o += p V         p from tensor memory, V from shared memory, o in tensor memory
// While a tile's softmax is at one half, its products for the other half run (o for the half before, then S for the half after).
// Warpgroups 0 and 1 are the softmax of tiles 0 and 1, warpgroups 2 and 3 turn the codes of keys and of values into float16 operands
// (the scales stay out of them); in warpgroup 4 a warp for each tile issues its products and one looks up pages and scales, some steps
// ahead.  The flat order of all (sequence, head, tile, key block) is cut into one equal share a block.
//
// What bounds it: chunks of 1024 tokens over up to 8192 (32 query heads on 8, 128 dims) take 415 us, 783 TFLOP/s of the 1666 that a
// plain matrix product reaches (heads of 64: 356 us, 456 TFLOP/s; of 256: 938 us, 692).  A step of 128 keys and two tiles takes some 4500
// cycles.  The products are 2048 of tensor work, but 2560 as they are fed: a 16-deep step of S, 64 columns wide, reads 6 KB of operands
// from shared memory, 48 cycles of it for 32 of work.  The exponentials take some 2048 on the special-function units, the operands' way
// through shared memory 2600.  None of them is full (tensor pipe 38 %); the chain product - softmax - product of a tile, with the loads from
// tensor memory waited for one after the other, is what is left.  Tensor memory (512 columns: two S and two o) holds no third tile.  Tried and slower: a quarter of the exponentials as polynomials (465 us against 464), tiles that take turns
// at the softmax (544 against 475), two threads a row (538 against 487).
//
// Scales.  A page's key scale multiplies 16 or more neighbouring columns of S: it goes into the factor of the exponent's argument.
// Its value scale vs goes into the exponent: w = exp2(s + log2 vs - M), M near the running maximum of s + log2 vs, is what multiplies
// V's codes, and the softmax total sum exp2(s - M) is the sum of each page's w times 1 / vs.  So neither costs an instruction an
// element, and the operands stay exact.  (Value scales beyond kNear: the total is summed apart.)
#include "roomie_kv_attention.cuh"

namespace roomie {

// ---- tensor memory and matrix instructions ---------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t* at, uint32_t columns) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(at)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// Operands in shared memory are given by the low halves of their descriptors; the high half is the same for all (kOperandHigh).
constexpr uint32_t kOperandHigh = (1024u >> 4) | 1u << 14 | 2u << 29;
template <bool kAdd> __device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tmov.b64 x, {%1, %4};\n\tmov.b64 y, {%2, %4};\n\tsetp.ne.u32 p, %5, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "n"(kOperandHigh), "n"((int)kAdd)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tmov.b64 y, {%2, %4};\n\tsetp.ne.u32 p, %5, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "n"(kOperandHigh),
                 "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t* x) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]),
          "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(x[16]), "=r"(x[17]), "=r"(x[18]),
          "=r"(x[19]), "=r"(x[20]), "=r"(x[21]), "=r"(x[22]), "=r"(x[23]), "=r"(x[24]), "=r"(x[25]), "=r"(x[26]), "=r"(x[27]),
          "=r"(x[28]), "=r"(x[29]), "=r"(x[30]), "=r"(x[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_load16(uint32_t at, uint32_t* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]),
                   "=r"(x[9]), "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t* x) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
        "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]),
        "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(x[16]), "r"(x[17]), "r"(x[18]), "r"(x[19]), "r"(x[20]),
        "r"(x[21]), "r"(x[22]), "r"(x[23]), "r"(x[24]), "r"(x[25]), "r"(x[26]), "r"(x[27]), "r"(x[28]), "r"(x[29]), "r"(x[30]),
        "r"(x[31])
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* x) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at), "r"(x[0]),
        "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]),
        "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15])
        : "memory");
}
// The wait names the registers of the load before it: nothing that uses them may be moved in front of it.
__device__ __forceinline__ void tmem_wait16(uint32_t* x) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
          "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15])::"memory");
}
__device__ __forceinline__ void tmem_wait32(uint32_t* x) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]),
          "+r"(x[8]), "+r"(x[9]), "+r"(x[10]), "+r"(x[11]), "+r"(x[12]), "+r"(x[13]), "+r"(x[14]), "+r"(x[15]),
          "+r"(x[16]), "+r"(x[17]), "+r"(x[18]), "+r"(x[19]), "+r"(x[20]), "+r"(x[21]), "+r"(x[22]), "+r"(x[23]),
          "+r"(x[24]), "+r"(x[25]), "+r"(x[26]), "+r"(x[27]), "+r"(x[28]), "+r"(x[29]), "+r"(x[30]), "+r"(x[31])::"memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Shared-memory operand: rows of 128 bytes (64 float16), 16-byte chunks exchanged by chunk ^ (row & 7) within groups of 8 rows
// (1024 bytes apart).  `lbo`: distance of the next 64 columns where the operand's columns are the contiguous direction.
__device__ __forceinline__ uint32_t operand(uint32_t at, uint32_t lbo) { return (at & 0x3ffffu) >> 4 | (lbo >> 4) << 16; }
// float16 operands, float32 accumulator, 128 rows, n columns; `columns_contiguous`: of the second operand
__host__ __device__ constexpr uint32_t instruction(uint32_t n, bool columns_contiguous) {
    return 1u << 4 | (columns_contiguous ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}

template <int kN> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kN)); }
template <int kN> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kN)); }

// ---- shape ------------------------------------------------------------------------------------------------------------------
constexpr int kKeys = 128;                          // keys of a step
template <int DP> struct Prompt {
    static constexpr int kTiles = DP > 128 ? 1 : 2; // 512 columns of tensor memory: S 128 and o DP for each tile
    static constexpr int kStages = DP > 128 ? 1 : 2;
    static constexpr int kRows = 128 * kTiles;
    static constexpr int kHalves = DP / 64;         // 64-column slabs of an operand
    static constexpr uint32_t kSlab = 128 * 128;    // bytes: 128 rows of 64 float16
    static constexpr uint32_t kOperand = kHalves * kSlab;
    static constexpr uint32_t kSmem = kOperand * (kTiles + 2 * kStages) + 1024;
    static constexpr size_t kPartial = (size_t)kRows * (DP + 2);   // floats of a partial result: [DP/4][kRows][4], then max and total
};

// ---- the flat order of the work: sequence, key head, row tile, key block -----------------------------------------------------
// row / group by the host's 2^64 / group + 1 (exact for 32 bits; group 1 has 0 there)
__device__ __forceinline__ uint32_t token_of(const AttnArgs& a, uint32_t row) {
    return a.group_inverse ? (uint32_t)__umul64hi(row, a.group_inverse) : row;
}
struct PromptSeq {
    KvSeq s;
    uint32_t rows, tiles;                           // rows a key head
    int start;
};
template <int kRows> __device__ __forceinline__ PromptSeq prompt_seq(const AttnArgs& a, uint32_t i, bool report) {
    PromptSeq p;
    p.s = kv_seq(a.c, a.seqs, a.q_offset, a.rows, i, report);
    p.rows = p.s.count * a.group;
    p.tiles = (p.rows + kRows - 1) / kRows;
    p.start = (int)p.s.length - (int)p.s.count;
    return p;
}
// A tile's queries, first step and results cost a block about as much time as kTileCost steps: its share of the flat order has so many
// units in front, which hold no key block.  Device times, us, by that number (32 query heads on 8; tokens a chunk over context):
//        16 x 64/1024  2 x 512/4096  2048/2048  4 x 1024/8192  4 x 512/8192, heads of 256
//   0    60.0          93.5          117.6      485.6          462
//   2    53.0          84.1          89.3       485.6          445
//   4    53.1          83.4          83.1       484.3          450
//   8    49.5          90.0          90.4       482.4          467
constexpr uint32_t kTileCost = 4;
struct Blocks {
    uint32_t first, count;                          // key blocks that some row of the tile sees, at least one
    uint32_t lo, hi;                                // no row sees a key outside [lo, hi)
};
template <int kRows> __device__ __forceinline__ Blocks tile_blocks(const AttnArgs& a, const PromptSeq& p, uint32_t tile) {
    const uint32_t last_row = min((tile + 1) * kRows, p.rows) - 1;
    const int hi = max(min((int)p.s.length, p.start + (int)token_of(a, last_row) + 1), 0);
    const int lo = a.window ? min(first_seen(p.start + (int)token_of(a, tile * kRows), a.window), hi) : 0;
    Blocks b;
    b.first = (uint32_t)lo / kKeys;
    const uint32_t end = ((uint32_t)hi + kKeys - 1) / kKeys;
    b.count = end > b.first ? end - b.first : 1u;
    b.lo = (uint32_t)lo;
    b.hi = (uint32_t)hi;
    return b;
}
template <int kRows> __device__ __forceinline__ unsigned long long seq_blocks(const AttnArgs& a, const PromptSeq& p, int lane) {
    unsigned long long n = 0;                       // units of one key head; by a whole warp
    for (uint32_t t = lane; t < p.tiles; t += 32) n += tile_blocks<kRows>(a, p, t).count + kTileCost;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    return n;
}

struct Walk {                                       // where in the flat order a thread is; the same in all threads of the block
    unsigned long long at, end, total, parts;
    uint32_t seq, head, tile, unit;                 // unit: of the tile
};

struct Segment {                                    // a run of blocks of one (sequence, head, tile)
    PromptSeq p;
    uint32_t head, tile, first, count, b0, b1;      // blocks first + [b0, b1) of count
    uint32_t lo, hi;                                // keys that some row sees
    unsigned long long item;                        // flat index of the tile's first block
    uint32_t rows;                                  // of the tile
};
template <int kRows> __device__ __forceinline__ bool next_segment(const AttnArgs& a, Walk& w, Segment& s) {
    if (w.at >= w.end || w.seq >= a.num_seqs) return false;
    s.p = prompt_seq<kRows>(a, w.seq, false);
    while (s.p.tiles == 0) {
        if (++w.seq >= a.num_seqs) return false;
        s.p = prompt_seq<kRows>(a, w.seq, false);
    }
    const Blocks b = tile_blocks<kRows>(a, s.p, w.tile);
    const uint32_t until = (uint32_t)min((unsigned long long)b.count + kTileCost, (unsigned long long)w.unit + (w.end - w.at));
    s.head = w.head;
    s.tile = w.tile;
    s.first = b.first;
    s.count = b.count;
    s.lo = b.lo;
    s.hi = b.hi;
    s.b0 = max(w.unit, kTileCost) - kTileCost;
    s.b1 = max(until, kTileCost) - kTileCost;
    s.item = w.at - w.unit + kTileCost;
    s.rows = min(s.p.rows - w.tile * kRows, (uint32_t)kRows);
    w.at += until - w.unit;
    w.unit = 0;
    if (++w.tile >= s.p.tiles) {
        w.tile = 0;
        if (++w.head >= a.c.heads) {
            w.head = 0;
            ++w.seq;
        }
    }
    return s.b0 < s.b1;                             // a share can end in units without a block, but not begin and go on there
}

constexpr int kPromptThreads = 640;

template <int kRows> __device__ __forceinline__ bool walk_start(const AttnArgs& a, Walk& w, unsigned long long* sh) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    unsigned long long mine = 0;
    for (uint32_t i = wid; i < a.num_seqs; i += kPromptThreads / 32)
        mine += seq_blocks<kRows>(a, prompt_seq<kRows>(a, i, blockIdx.x == 0 && lane == 0), lane) * a.c.heads;
    if (lane == 0) sh[wid] = mine;
    __syncthreads();
    w.total = 0;
    for (int i = 0; i < kPromptThreads / 32; ++i) w.total += sh[i];
    if (w.total == 0) return false;
    w.parts = w.total < gridDim.x ? w.total : gridDim.x;
    if (blockIdx.x >= w.parts) return false;
    w.at = w.total * blockIdx.x / w.parts;
    w.end = w.total * (blockIdx.x + 1) / w.parts;
    unsigned long long before = 0;
    for (uint32_t base = 0; base < a.num_seqs; base += kPromptThreads / 32) {
        const uint32_t i = base + wid;
        const unsigned long long n = i < a.num_seqs ? seq_blocks<kRows>(a, prompt_seq<kRows>(a, i, false), lane) : 0;
        __syncthreads();
        if (lane == 0) sh[wid] = n;
        __syncthreads();
        unsigned long long first = before, all = before;
        for (int j = 0; j < kPromptThreads / 32; ++j) {
            if (j < wid) first += sh[j] * a.c.heads;
            all += sh[j] * a.c.heads;
        }
        if (n && w.at >= first && w.at < first + n * a.c.heads) {        // by the one warp whose sequence it is
            const PromptSeq p = prompt_seq<kRows>(a, i, false);
            const unsigned long long inside = w.at - first, head = inside / n;
            unsigned long long rest = inside - head * n, ahead = 0;
            for (uint32_t t0 = 0; t0 < p.tiles; t0 += 32) {
                const uint32_t t = t0 + lane, c = t < p.tiles ? tile_blocks<kRows>(a, p, t).count + kTileCost : 0u;
                unsigned long long incl = c;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, d);
                    if (lane >= d) incl += up;
                }
                const unsigned long long f = ahead + incl - c;
                if (c && rest >= f && rest < f + c) {
                    sh[20] = i; sh[21] = head; sh[22] = t; sh[23] = rest - f;
                }
                ahead += __shfl_sync(0xffffffffu, incl, 31);
                if (rest < ahead) break;
            }
        }
        before = all;
        if (w.at < before) break;
    }
    __syncthreads();
    w.seq = (uint32_t)sh[20]; w.head = (uint32_t)sh[21]; w.tile = (uint32_t)sh[22]; w.unit = (uint32_t)sh[23];
    return true;
}

// ---- shared state -----------------------------------------------------------------------------------------------------------
constexpr int kRing = 8;                            // steps whose pages and scales are looked up ahead
constexpr int kSegments = 16;                       // segments ahead: at most one a step, and the one before may still be written out
struct SegInfo {                                    // a segment as the other warps need it; steps = 0: there are no more
    uint32_t steps, rows, row0, first_row, head, key0, low_key, end_key, length, b0, count;   // keys outside [low, end) are not read
    int32_t start;                                  // position of the sequence's first row
    unsigned long long item;
};
// Barriers that are waited for once a half have one for each half of a step: a wait tells only two phases apart, and two halves may be
// on their way at once.
struct PromptShared {
    uint64_t q_full, q_empty, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2][2], p_full[2][2], o_full[2][2], look_full[kRing],
        look_free[kRing], join[2], drain;
    unsigned long long walk[24];
    long long at[kRing][8];                         // of 16 keys each: bytes from the pool's start to them (-1: none), key scale, log2
                                                    // and inverse of the value scale
    float ks[kRing][8], lvs[kRing][8], ivs[kRing][8];
    __align__(4) uint8_t wide[kRing][8];            // the value scale is beyond kNear
    float l_ref[256];                               // reference of a row's total while it is summed apart
    SegInfo seg[kSegments];
    float q_scale[2][256];                          // of a row, segments in turn: 2^e of its float16 form times scale * log2(e)
    uint32_t tmem, last, failed;
};

// By a whole warp, with one answer.  The instruction itself suspends the warp for up to the hint (20 us); a wait that runs out after
// 2^16 of them (about a second) ends the block: the flag makes its other waits give up too.  Kept to a few instructions: the roles'
// loops have to fit the instruction caches together.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, PromptShared& sh) {
    const uint32_t at = smem_addr(bar);
#pragma unroll 1
    for (uint32_t spin = 0; spin < 65536u; ++spin) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(at), "r"(parity) : "memory");
        if (__all_sync(0xffffffffu, ok != 0)) return true;
        if (*reinterpret_cast<volatile uint32_t*>(&sh.failed)) return false;
    }
    *reinterpret_cast<volatile uint32_t*>(&sh.failed) = 1u;
    return false;
}

// 16 codes to two 16-byte chunks of float16
template <int kFormat> __device__ __forceinline__ void widen(const uint4& c, uint4& x, uint4& y) {
    codes_to_f16<kFormat>(c.x, x.x, x.y);
    codes_to_f16<kFormat>(c.y, x.z, x.w);
    codes_to_f16<kFormat>(c.z, y.x, y.y);
    codes_to_f16<kFormat>(c.w, y.z, y.w);
}

// ---- warpgroups 2 and 3: operands ------------------------------------------------------------------------------------------------
// The call's rows [r0, r1) of the segment's tile, as float16 with the row's largest magnitude in [1, 2) (see few_rows_kernel).
template <int DP, class T>
__device__ __forceinline__ void feed_queries(const AttnArgs& a, PromptShared& sh, uint8_t* sq, const SegInfo& s, uint32_t which, uint32_t r0,
                                             uint32_t r1) {
    using P = Prompt<DP>;
    constexpr int kLanes = DP / 8, kPass = 128 / kLanes;         // lanes of a row side by side, 8 elements each
    const uint32_t tid = threadIdx.x & 127, c = tid % kLanes;
    r0 += tid / kLanes;
    uint8_t* to0 = sq + (c >> 3) * P::kSlab + (((c & 7) ^ (r0 & 7)) << 4);         // kPass is a multiple of 8, or r & 7 moves with it
    auto place = [&](uint32_t r) {
        return kPass % 8 == 0 ? to0 + (r >> 7) * P::kOperand + (r & 127) * 128
                              : sq + (c >> 3) * P::kSlab + (r >> 7) * P::kOperand + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4);
    };
#pragma unroll 1
    for (uint32_t r = r0; r < r1; r += kPass) {                  // as they come, all on their way together
        const uint32_t row = s.first_row + r, tok = token_of(a, row);
        const bool there = r < s.rows && 8 * c < a.c.dim;
        const T* q = static_cast<const T*>(a.q);
        if (there) q += (long long)(s.row0 + tok) * a.q_token + (long long)(s.head * a.group + row - tok * a.group) * a.q_head + 8 * c;
        if (a.q_aligned) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(place(r))), "l"(q), "r"(there ? 16u : 0u) : "memory");
        } else {
            uint4 x = make_uint4(0, 0, 0, 0);
            const unsigned short* h = reinterpret_cast<const unsigned short*>(q);
            if (there)
                x = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
            *reinterpret_cast<uint4*>(place(r)) = x;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 2
    for (uint32_t r = r0; r < r1; r += kPass) {                  // each thread its own pieces
        uint4* at = reinterpret_cast<uint4*>(place(r));
        float x[8], amax = 0.0f;
        unpack<T>(*at, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(x[k]));
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
        int e = (int)(__float_as_uint(amax) >> 23) - 127;
        e = max(min(e, 126), -126);
        const float down = pow2f(-e);
        __half2 h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2half2_rn(x[2 * k] * down, x[2 * k + 1] * down);
        *at = *reinterpret_cast<const uint4*>(h);
        if (c == 0) sh.q_scale[which][r] = pow2f(e) * a.scale_log2;
    }
}

template <int DP, int kFormat, class T>
__device__ __forceinline__ void feed(const AttnArgs& a, PromptShared& sh, uint8_t* smem, const bool keys) {
    using P = Prompt<DP>;
    constexpr int kPerRow = DP / 16;                             // 16-code units of a key
    constexpr int kUnits = kPerRow;                              // a thread's, of the 128 keys
    constexpr int kRowStep = 128 / kPerRow;                      // unit e: key row0 + e * kRowStep, codes [16 * unit, +16)
    const uint32_t tid = threadIdx.x & 127;
    uint8_t* operands = smem + (P::kTiles + (keys ? 0 : P::kStages)) * P::kOperand;
    uint64_t* full = keys ? sh.k_full : sh.v_full;
    uint64_t* empty = keys ? sh.k_empty : sh.v_empty;
    const uint32_t unit = tid % kPerRow, row0 = tid / kPerRow;
    const bool inside = 16 * unit < a.c.dim;
    // Where in an operand unit 0 goes; row0 + e * kRowStep keeps row & 7 (kRowStep is a multiple of 8).  The odd slabs store their
    // second chunk first: the eight lanes of a store then hit different banks.
    const uint32_t slab = unit / 4, swap = slab & 1, chunk = (unit & 3) * 2;
    uint8_t* to0 = operands + slab * P::kSlab + row0 * 128 + (((chunk + swap) ^ (row0 & 7)) << 4);
    const uint32_t to1 = (((chunk + 1 - swap) ^ (row0 & 7)) << 4) - (((chunk + swap) ^ (row0 & 7)) << 4);
    uint32_t step = 0;
    for (uint32_t seg = 0;; ++seg) {
        if (!warp_wait(&sh.look_full[step % kRing], (step / kRing) & 1, sh)) return;
        const SegInfo& s = sh.seg[seg % kSegments];
        const uint32_t n = s.steps;
        if (n == 0) return;
        const uint8_t* pool = (keys ? a.c.k : a.c.v) + (long long)s.head * a.c.head_step + 16 * unit + (long long)(row0 & 15) * a.c.token_step;
        int left = (int)s.end_key - (int)s.key0 - (int)row0;     // keys there from this thread's first on
        const int skip = (int)s.low_key - (int)s.key0 - (int)row0;   // and of them in front of every row's window: of the first step only
        uint4 c[kUnits];
        auto get = [&](uint32_t x, int skip) {
            const uint32_t ring = x % kRing;
#pragma unroll
            for (int e = 0; e < kUnits; ++e) {
                const long long at = sh.at[ring][(row0 + e * kRowStep) >> 4];
                c[e] = make_uint4(0, 0, 0, 0);
                if (at >= 0 && inside && e * kRowStep < left && e * kRowStep >= skip)
                    asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[e].x), "=r"(c[e].y), "=r"(c[e].z), "=r"(c[e].w)
                                 : "l"(pool + at + (kRowStep < 16 && (e & 1) ? 8 * a.c.token_step : 0u)));
            }
        };
        if (seg && !warp_wait(&sh.q_empty, (seg - 1) & 1, sh)) return;
        feed_queries<DP, T>(a, sh, smem, s, seg & 1, keys ? 0 : P::kRows / 2, keys ? P::kRows / 2 : P::kRows);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(&sh.q_full);
        get(step, skip);
        for (uint32_t j = 0; j < n; ++j) {
            const uint32_t stage = step % P::kStages, turn = step / P::kStages;
            if (turn && !warp_wait(&empty[stage], (turn - 1) & 1, sh)) return;
#pragma unroll
            for (int e = 0; e < kUnits; ++e) {
                uint4 x, y;
                widen<kFormat>(c[e], x, y);
                uint8_t* to = to0 + stage * P::kOperand + e * kRowStep * 128;
                *reinterpret_cast<uint4*>(to) = swap ? y : x;
                *reinterpret_cast<uint4*>(to + to1) = swap ? x : y;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(&full[stage]);
            ++step;
            left -= kKeys;
            if (j + 1 < n) {
                if (!warp_wait(&sh.look_full[step % kRing], (step / kRing) & 1, sh)) return;
                get(step, 0);
            }
        }
    }
}

// ---- warpgroup 4: one warp looks up pages and scales, four steps at a time ------------------------------------------------------
template <int DP>
__device__ __forceinline__ void look_up(const AttnArgs& a, PromptShared& sh, Walk w) {
    using P = Prompt<DP>;
    const KvView& kv = a.c;
    const uint32_t lane = threadIdx.x & 31, group = lane & 7;
    uint32_t step = 0, seg = 0;
    for (;; ++seg) {
        Segment s;
        const bool more = next_segment<P::kRows>(a, w, s);
        const int32_t* table = kv.pages + (more ? (size_t)s.p.s.slot * kv.max_pages : 0);
        const uint32_t n = more ? s.b1 - s.b0 : 1u;              // the end takes a step of its own
        const uint32_t low_key = more ? s.lo : 0u, end_key = more ? s.hi : 0u;
        for (uint32_t j0 = 0; j0 < n; j0 += 4) {
            const uint32_t j = j0 + (lane >> 3), x = step + j, last = step + min(j0 + 4, n) - 1;
            // products end in order: when the last slot of these four is free, all are
            if (last >= kRing && !warp_wait(&sh.look_free[last % kRing], (last / kRing - 1) & 1, sh)) return;
            if (j0 == 0) {
                if (lane == 0) {
                    SegInfo& o = sh.seg[seg % kSegments];
                    o.steps = more ? n : 0u;
                    o.rows = s.rows; o.row0 = s.p.s.row; o.first_row = s.tile * P::kRows; o.head = s.head;
                    o.key0 = (s.first + s.b0) * kKeys; o.low_key = low_key; o.end_key = end_key; o.length = s.p.s.length;
                    o.b0 = s.b0; o.count = s.count; o.start = s.p.start; o.item = s.item;
                }
                __syncwarp();
            }
            if (j < n) {
                const uint32_t key = more ? (s.first + s.b0 + j) * kKeys + 16 * group : 0u;
                int32_t id = -1;
                if (key < end_key && key + 16 > low_key) {
                    id = __ldg(table + (key >> kv.page_shift));
                    if ((uint32_t)id >= kv.num_pages) {
                        kv_flag(kv.status, ROOMIE_FLAG_KV_PAGE);
                        id = -1;
                    }
                }
                float ks = 0.0f, lvs = -INFINITY, ivs = 0.0f;    // keys that are not there weigh nothing
                if (id >= 0) {
                    ks = __ldg(kv.k_scale + (size_t)id * kv.heads + s.head);
                    const float vs = fmaxf(__ldg(kv.v_scale + (size_t)id * kv.heads + s.head), kLeastScale);
                    lvs = log2f(vs);
                    ivs = __fdiv_rn(1.0f, vs);
                }
                const uint32_t ring = x % kRing;
                sh.at[ring][group] = id < 0 ? -1ll : (long long)id * kv.page_stride + (long long)(key & (kv.page_tokens - 1)) * kv.token_step;
                sh.ks[ring][group] = ks;
                sh.lvs[ring][group] = lvs;
                sh.ivs[ring][group] = ivs;
                sh.wide[ring][group] = id >= 0 && fabsf(lvs) > kNear;
                mbar_arrive(&sh.look_full[ring]);
            }
            __syncwarp();
        }
        if (!more) return;
        step += n;
    }
}

// ---- warpgroup 4: a warp for each tile issues its products ---------------------------------------------------------------------------
// The whole warp goes through the loop, so that what does not depend on the lane stays in uniform registers; one elected lane issues.
// (A single thread's branch around all of it took 280 cycles an instruction, this some 80; the instructions themselves have 32 and 64,
// so one warp for both tiles was what the step waited for.)
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
template <int DP>
__device__ __forceinline__ void issue(PromptShared& sh, uint8_t* smem, const uint32_t t) {
    using P = Prompt<DP>;
    const uint32_t sq = smem_addr(smem), sk = sq + P::kTiles * P::kOperand, sv = sk + P::kStages * P::kOperand;
    const uint32_t q = operand(sq + t * P::kOperand, 16), k0 = operand(sk, 16), v0 = operand(sv, P::kSlab);
    const uint32_t tm = __shfl_sync(0xffffffffu, sh.tmem, 0), s_tile = tm + t * 128, o_at = tm + P::kTiles * 128 + t * DP;
    constexpr uint32_t kS = instruction(kKeys / 2, false), kO = instruction(DP, true);
    uint32_t step = 0;
    for (uint32_t seg = 0;; ++seg) {
        if (!warp_wait(&sh.look_full[step % kRing], (step / kRing) & 1, sh)) return;
        const uint32_t n = __shfl_sync(0xffffffffu, sh.seg[seg % kSegments].steps, 0);
        const bool on = __shfl_sync(0xffffffffu, sh.seg[seg % kSegments].rows, 0) > t * 128;
        if (n == 0 || !warp_wait(&sh.q_full, seg & 1, sh) || !warp_wait(&sh.k_full[step % P::kStages], (step / P::kStages) & 1, sh)) return;
        tc_fence_after();
        // Half h: o of half h - 2, then S of half h into the columns that held its p.  A tile without rows only keeps step.
        const uint32_t halves = 2 * n;
#pragma unroll 1
        for (uint32_t h = 0; h < halves + 2; ++h) {
            const uint32_t next = step + h / 2, stage = next % P::kStages;                   // keys of half h
            const uint32_t now = next - 1, old_stage = now % P::kStages, side = h & 1;       // values of half h - 2
            const uint32_t s_at = s_tile + side * 64;
            if (h >= 2) {
                if (side == 0 && !warp_wait(&sh.v_full[old_stage], (now / P::kStages) & 1, sh)) return;
                if (!warp_wait(&sh.p_full[t][side], now & 1, sh)) return;
                tc_fence_after();
                const uint32_t v = v0 + ((old_stage * P::kOperand + side * 8192) >> 4);
                if (elected()) {
                    if (on)
#pragma unroll
                        for (int i = 0; i < kKeys / 32; ++i) mma_ts(o_at, s_at + 8 * i, v + i * (2048 >> 4), kO, h > 2 || i > 0);
                    tc_commit(&sh.o_full[t][side]);
                }
                __syncwarp();
            }
            if (h < halves) {
                // S takes the columns that p was read from, by a segment's first halves the last step's of the segment before: products of
                // different shapes are not counted on to end in order (head sizes to 128: no cost; 256, with one tile: 11 %)
                if (next && !warp_wait(&sh.o_full[t][side], now & 1, sh)) return;
                if (h >= 2 && side == 0 && !warp_wait(&sh.k_full[stage], (next / P::kStages) & 1, sh)) return;
                tc_fence_after();
                const uint32_t k = k0 + ((stage * P::kOperand + side * 8192) >> 4);
                if (elected()) {
                    if (on) {
                        mma_ss<false>(s_at, q, k, kS);
#pragma unroll
                        for (int i = 1; i < DP / 16; ++i) {
                            const uint32_t off = ((i / 4) * P::kSlab + (i % 4) * 32) >> 4;
                            mma_ss<true>(s_at, q + off, k + off, kS);
                        }
                    }
                    tc_commit(&sh.s_full[t][side]);
                }
                __syncwarp();
            }
            if (side == 1 && elected()) {
                if (h >= 2) {
                    tc_commit(&sh.v_empty[old_stage]);
                    tc_commit(&sh.look_free[now % kRing]);
                }
                if (h < halves) tc_commit(&sh.k_empty[stage]);
                if (h + 1 == halves) tc_commit(&sh.q_empty);
            }
            __syncwarp();
        }
        step += n;
    }
}

// ---- one row's share of a step -----------------------------------------------------------------------------------------------------
// two float32 at a time
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) { return pair(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void split(uint64_t p, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// 2^x of 32 columns, as float16 pairs; the result is their share of the softmax total.
__device__ __forceinline__ float weights32(const uint32_t* x, uint32_t* p, const float* ivs) {
    float total = 0.0f;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float u = exp2_fast(__uint_as_float(x[16 * g + e])), v = exp2_fast(__uint_as_float(x[16 * g + e + 1]));
            sum[(e / 2) & 1] = add2(sum[(e / 2) & 1], pair(u, v));
            const __half2 h = __floats2half2_rn(u, v);
            p[8 * g + e / 2] = reinterpret_cast<const uint32_t&>(h);
        }
        float even, odd;
        split(add2(sum[0], sum[1]), even, odd);
        total = fmaf(even + odd, ivs[g], total);
    }
    return total;
}

// The same columns' share of a total that is summed apart: x holds s + log2 vs - base.
__device__ __forceinline__ float total_apart(const uint32_t* x, const float* lvs, float base, float& ref_at, float& l) {
    float add[2], ref = ref_at, top = -INFINITY, total = 0.0f;
#pragma unroll
    for (int g = 0; g < 2; ++g) add[g] = base - (lvs[g] == -INFINITY ? 0.0f : lvs[g]);
#pragma unroll
    for (int e = 0; e < 32; ++e) top = fmaxf(top, __uint_as_float(x[e]) + add[e / 16]);
    if (top > ref + kAbove) {
        if (ref != -INFINITY) l *= exp2_fast(ref - (top - kBelow));
        ref_at = ref = top - kBelow;
    }
    if (ref == -INFINITY) ref = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e) total += exp2_fast(__uint_as_float(x[e]) + add[e / 16] - ref);
    return total;
}

// Half a step of a row, 64 keys, 32 at a time: the weights exp2(f * S + log2 vs - m) go as float16 over the columns of S that have been
// read.  They are taken against an old reference m while no exponent is more than kAbove over it.  Past that m - a
// whole number - moves up to kBelow under the new maximum: the weights already written, o and the total are multiplied by a power of two.  `moved` collects that factor
// for o.  cut: some key is hidden from some row of the warp; hidden ones weigh exactly nothing.  No branch stands between the elements
// (with one, each exponential waits for the one before), and the loop is kept short because the roles share the instruction caches
// (unrolled over a whole step, a third of all stalls were for instructions).
__device__ __forceinline__ void row_half(uint32_t s_at, const float* ks, const float* lvs, const float* ivs, float q, bool cut, int k0, int lo,
                                         int hi, bool apart, float& ref, float& m, float& l, float& moved) {
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
        uint32_t x[32], p[16];
        tmem_load32(s_at + 32 * c, x);
        const float base = m == -INFINITY ? 0.0f : m;
        const float fa = q * ks[2 * c], fb = q * ks[2 * c + 1], oa = lvs[2 * c] - base, ob = lvs[2 * c + 1] - base;
        const uint64_t f2[2] = {pair(fa, fa), pair(fb, fb)}, off2[2] = {pair(oa, oa), pair(ob, ob)};
        tmem_wait32(x);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            float u, v;
            split(fma2(pair(x[e], x[e + 1]), f2[e / 16], off2[e / 16]), u, v);
            x[e] = __float_as_uint(u);
            x[e + 1] = __float_as_uint(v);
        }
        if (cut) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
                const int k = k0 + 32 * c + e;
                if (k >= hi || k < lo) x[e] = 0xff800000u;       // -inf
            }
        }
        float top[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top[i] = fmaxf(__uint_as_float(x[8 * i]), __uint_as_float(x[8 * i + 1]));
#pragma unroll
            for (int e = 2; e < 8; e += 2) top[i] = max3(top[i], __uint_as_float(x[8 * i + e]), __uint_as_float(x[8 * i + e + 1]));
        }
        const float high = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        float total = weights32(x, p, ivs + 2 * c);
        if (__any_sync(0xffffffffu, apart || high > kAbove || (m == -INFINITY && high > m))) {
            const bool none = m == -INFINITY;                    // no key so far: there is nothing to multiply
            const float up = none ? (high > m ? floorf(high) - kBelow : 0.0f) : fmaxf(floorf(high) - kBelow, 0.0f), f = none ? 1.0f : exp2_fast(-up);
            if (!none || high > m) m = base + up;
            if (!apart) l *= f;
            moved *= f;
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) - up);
            if (c) {                                             // weights already written (f may be below float16's least)
                tmem_wait_st();
                tmem_load16(s_at, p);
                tmem_wait16(p);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 w2 = __half22float2(reinterpret_cast<const __half2&>(p[e]));
                    const __half2 w = __floats2half2_rn(w2.x * f, w2.y * f);
                    p[e] = reinterpret_cast<const uint32_t&>(w);
                }
                tmem_store16(s_at, p);
            }
            total = weights32(x, p, ivs + 2 * c);
            if (apart) total = total_apart(x, lvs + 2 * c, m == -INFINITY ? 0.0f : m, ref, l);
        }
        l += total;
        tmem_store16(s_at + 16 * c, p);
    }
}

// ---- warpgroups 0 and 1: softmax, and the end of a segment ------------------------------------------------------------------------
template <int DP, class T>
__device__ __forceinline__ void softmax(const AttnArgs& a, PromptShared& sh, unsigned long long total_blocks, unsigned long long parts) {
    using P = Prompt<DP>;
    const uint32_t t = threadIdx.x >> 7, r = threadIdx.x & 127;  // tile, row
    const uint32_t lanes = (threadIdx.x & 96) << 16;             // this warp's quarter of the tensor memory's lanes
    const uint32_t s_at = sh.tmem + t * 128 + lanes, o_at = sh.tmem + P::kTiles * 128 + t * DP + lanes;
    uint32_t step = 0, joins = 0;
    for (uint32_t seg = 0;; ++seg) {
        if (!warp_wait(&sh.look_full[step % kRing], (step / kRing) & 1, sh)) return;
        const SegInfo& s = sh.seg[seg % kSegments];
        const uint32_t n = s.steps;
        if (n == 0) return;
        const bool on = t * 128 < s.rows, mine = t * 128 + r < s.rows;
        int hi = 0, lo = 0;
        if (mine) {
            const int pos = s.start + (int)token_of(a, s.first_row + t * 128 + r);
            hi = max(min(pos + 1, (int)s.length), 0);
            lo = a.window ? first_seen(pos, a.window) : 0;
        }
        float m = -INFINITY, l = 0.0f, q = 0.0f;
        float& l_ref = sh.l_ref[t * 128 + r];
        bool apart = false;
        int k0 = (int)s.key0;
        for (uint32_t h = 0; h < 2 * n; ++h, k0 += kKeys / 2) {
            const uint32_t side = h & 1, ring = step % kRing;
            if (h && !side && !warp_wait(&sh.look_full[ring], (step / kRing) & 1, sh)) return;
            if (!warp_wait(&sh.s_full[t][side], step & 1, sh)) return;
            step += side;
            if (!on) {
                mbar_arrive(&sh.p_full[t][side]);
                continue;
            }
            tc_fence_after();
            if (h == 0) q = sh.q_scale[seg & 1][t * 128 + r];
            const bool cut = __any_sync(0xffffffffu, k0 < lo || k0 + kKeys / 2 > hi);
            float moved = 1.0f;
            const bool wide = *reinterpret_cast<const uint32_t*>(sh.wide[ring] + 4 * side) != 0;
            if (wide && !apart) l_ref = m;
            apart = apart || wide;
            row_half(s_at + 64 * side, sh.ks[ring] + 4 * side, sh.lvs[ring] + 4 * side, sh.ivs[ring] + 4 * side, q, cut, k0, lo, hi, apart,
                     l_ref, m, l, moved);
            if (h && __any_sync(0xffffffffu, moved != 1.0f)) {   // o of the halves before
                if (!warp_wait(&sh.o_full[t][side ^ 1], (step - 1) & 1, sh)) return;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < DP / 32; ++c) {
                    uint32_t y[32];
                    tmem_load32(o_at + 32 * c, y);
                    tmem_wait32(y);
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * moved);
                    tmem_store32(o_at + 32 * c, y);
                }
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sh.p_full[t][side]);
        }

        float up = 1.0f;
        if (apart) one_reference(m, l, up, l_ref);
        // ---- the end of a segment: rows go out, or wait in the workspace for their other parts ---------------------------------
        const bool complete = s.b0 == 0 && n == s.count;
        const uint32_t row = s.first_row + t * 128 + r, tok = token_of(a, row), h = s.head * a.group + row - tok * a.group;
        T* out = static_cast<T*>(a.out) + (long long)(s.row0 + tok) * a.o_token + (long long)h * a.o_head;
        auto put_lse = [&](float mx, float sum) {
            if (a.lse) a.lse[(size_t)(s.row0 + tok) * a.q_heads + h] = sum > 0.0f ? (mx + log2f(sum)) * kLn2 : sum == 0.0f ? -INFINITY : sum;
        };
        auto put8 = [&](int d, const float* v) {                 // eight elements of the row
            if (d >= (int)a.c.dim) return;
            if (a.o_aligned) {
                *reinterpret_cast<uint4*>(out + d) = pack<T>(v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) out[d + i] = from_f32<T>(v[i]);
            }
        };
        float* part = a.partial + ((size_t)blockIdx.x * 2 + (s.b0 == 0 ? 1 : 0)) * P::kPartial;
        const uint32_t pr = t * 128 + r;
        if (on) {
            if (!warp_wait(&sh.o_full[t][1], (step - 1) & 1, sh)) return;
            tc_fence_after();
            const float inv = l > 0.0f ? __fdiv_rn(up, l) : l == 0.0f ? 0.0f : l;
#pragma unroll 1
            for (int c = 0; c < DP / 32; ++c) {
                uint32_t x[32];
                tmem_load32(o_at + 32 * c, x);
                tmem_wait32(x);
                if (complete) {
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = l == 0.0f ? 0.0f : __uint_as_float(x[e]) * inv;
                    if (mine)
#pragma unroll
                        for (int e = 0; e < 32; e += 8) put8(32 * c + e, v + e);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * up);
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<uint4*>(part + ((size_t)(8 * c + e / 4) * P::kRows + pr) * 4) =
                            make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                }
            }
            if (complete) {
                if (mine) put_lse(m, l);
            } else {
                part[(size_t)P::kRows * DP + 2 * pr] = m;
                part[(size_t)P::kRows * DP + 2 * pr + 1] = l;
            }
            tc_fence_before();
        }
        if (!complete) {
            const uint32_t first = (uint32_t)(((s.item + 1) * parts - 1) / total_blocks);
            const uint32_t last = (uint32_t)(((s.item + s.count) * parts - 1) / total_blocks);
            mbar_arrive(&sh.join[0]);
            if (threadIdx.x < 32) {
                if (!warp_wait(&sh.join[0], joins & 1, sh)) return;
                if (threadIdx.x == 0) {
                    const uint32_t before = count_part(a.counters + first, last - first + 1);
                    sh.last = before == last - first;
                    mbar_arrive(&sh.join[1]);
                }
            }
            if (!warp_wait(&sh.join[1], joins & 1, sh)) return;
            ++joins;
            if (sh.last && mine) {
                float mx = -INFINITY, sum = 0.0f;
                for (uint32_t b = first; b <= last; ++b) {
                    const float* pp = a.partial + ((size_t)b * 2 + (b == first ? 1 : 0)) * P::kPartial + (size_t)P::kRows * DP + 2 * pr;
                    const float mb = __ldcg(pp), lb = __ldcg(pp + 1), to = fmaxf(mx, mb);
                    // a part without keys has a total of 0, one of a query that is no number NaN: neither has a maximum
                    sum = (mx == -INFINITY ? sum : sum * exp2f(mx - to)) + (mb == -INFINITY ? lb : lb * exp2f(mb - to));
                    mx = to;
                }
                const float inv = sum > 0.0f ? __fdiv_rn(1.0f, sum) : sum == 0.0f ? 0.0f : sum;
#pragma unroll 1
                for (int d = 0; d < DP; d += 32) {
                    float v[32] = {};
                    for (uint32_t b = first; b <= last; ++b) {
                        const float* pp = a.partial + ((size_t)b * 2 + (b == first ? 1 : 0)) * P::kPartial;
                        const float mb = __ldcg(pp + (size_t)P::kRows * DP + 2 * pr);
                        float4 x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = __ldcg(reinterpret_cast<const float4*>(pp + ((size_t)(d / 4 + i) * P::kRows + pr) * 4));
                        const float f = mb == -INFINITY ? 0.0f : exp2f(mb - mx) * inv;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            v[4 * i] += f * x[i].x; v[4 * i + 1] += f * x[i].y; v[4 * i + 2] += f * x[i].z; v[4 * i + 3] += f * x[i].w;
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 8) put8(d + e, v + e);
                }
                put_lse(mx, sum);
            }
        }
    }
}

template <int DP, int kFormat, class T>
__global__ void __launch_bounds__(kPromptThreads, 1) prompt_kernel(AttnArgs a) {
    using P = Prompt<DP>;
    extern __shared__ uint8_t raw[];
    __shared__ PromptShared sh;
    uint8_t* smem = raw + ((1024u - (smem_addr(raw) & 1023u)) & 1023u);
    Walk w;
    if (!walk_start<P::kRows>(a, w, sh.walk)) return;            // the same answer in all threads
    const uint32_t wid = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(&sh.q_full, 256);
        mbar_init(&sh.q_empty, P::kTiles);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.k_full[i], 128);
            mbar_init(&sh.v_full[i], 128);
            mbar_init(&sh.k_empty[i], P::kTiles);
            mbar_init(&sh.v_empty[i], P::kTiles);
            for (int h = 0; h < 2; ++h) {
                mbar_init(&sh.s_full[i][h], 1);
                mbar_init(&sh.p_full[i][h], 128);
                mbar_init(&sh.o_full[i][h], 1);
            }
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&sh.look_full[i], 8);
            mbar_init(&sh.look_free[i], P::kTiles);
        }
        mbar_init(&sh.join[0], 128 * P::kTiles);
        mbar_init(&sh.join[1], 1);
        mbar_init(&sh.drain, P::kTiles);
        sh.failed = 0;
    }
    if (wid == 16) tmem_alloc(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // 640 threads are launched with 96 registers each; the warpgroups' shares below add up to 5 * 96.
    if (wid < 4) {
        registers_up<128>();
        softmax<DP, T>(a, sh, w.total, w.parts);
    } else if (wid < 8) {
        if constexpr (P::kTiles == 2) {
            registers_up<128>();
            softmax<DP, T>(a, sh, w.total, w.parts);
        } else {
            registers_down<40>();
        }
    } else if (wid < 16) {
        if constexpr (P::kTiles == 2) registers_down<80>();
        else registers_up<112>();
        feed<DP, kFormat, T>(a, sh, smem, wid < 12);
    } else {
        registers_down<64>();
        if (wid == 16 || (wid == 18 && P::kTiles == 2)) {
            issue<DP>(sh, smem, wid == 18);
            if (elected()) tc_commit(&sh.drain);                 // whatever was issued has ended before the memory is given back
            __syncwarp();
            warp_wait(&sh.drain, 0, sh);
        } else if (wid == 17) {
            look_up<DP>(a, sh, w);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && sh.failed) kv_flag(a.c.status, ROOMIE_FLAG_WAIT_TIMEOUT);
    if (wid == 16) tmem_free(sh.tmem, 512);
}

size_t prompt_partial_bytes(uint32_t dim) {
    const size_t floats = dim <= 64 ? Prompt<64>::kPartial : dim <= 128 ? Prompt<128>::kPartial : Prompt<256>::kPartial;
    return (size_t)sm_count() * 2 * floats * sizeof(float);
}

template <int DP, int kFormat, class T> static int launch_one(const AttnArgs& a, cudaStream_t st) {
    return launch("kv_attention", prompt_kernel<DP, kFormat, T>, dim3((uint32_t)sm_count()), dim3(kPromptThreads), Prompt<DP>::kSmem,
                  st, false, a);
}
template <int kFormat, class T> static int launch_dims(const AttnArgs& a, cudaStream_t st) {
    if (a.c.dim <= 64) return launch_one<64, kFormat, T>(a, st);
    if (a.c.dim <= 128) return launch_one<128, kFormat, T>(a, st);
    return launch_one<256, kFormat, T>(a, st);
}

int launch_prompt(const AttnArgs& a, bool half, cudaStream_t st) {
    if (a.c.format == ROOMIE_KV_E4M3)
        return half ? launch_dims<ROOMIE_KV_E4M3, __half>(a, st) : launch_dims<ROOMIE_KV_E4M3, __nv_bfloat16>(a, st);
    return half ? launch_dims<ROOMIE_KV_INT8, __half>(a, st) : launch_dims<ROOMIE_KV_INT8, __nv_bfloat16>(a, st);
}

}  // namespace roomie
