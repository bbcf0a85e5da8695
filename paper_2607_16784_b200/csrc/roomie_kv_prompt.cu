// Attention over the paged 8-bit cache for many query rows a sequence (prompt chunks): matrix products on the fifth-generation
// tensor cores, accumulators in tensor memory.
//
// A block (512 threads, one an SM) takes kTiles tiles of 128 rows of one key head - a row is one (token, query head) of the
// group - through the keys 128 at a time:
//   S = q K^T        both operands in shared memory, float16; S in tensor memory
//   softmax          a thread owns a row: reads S, writes the probabilities as float16 over the columns it has read
//   o += p V         p from tensor memory, V from shared memory, o in tensor memory
// Warpgroups 0 and 1 are the softmax of tiles 0 and 1, so that one tile's softmax overlaps the other's products; warpgroup 2
// turns codes into float16 operands (the scales stay out of them); in warpgroup 3 one thread issues the products and one warp
// looks up pages and scales, some steps ahead.
//
// Scales.  A page's key scale multiplies 16 or more neighbouring columns of S: it goes into the factor of the exponent's argument.
// Its value scale vs goes into the exponent: w = exp2(s + log2 vs - M), M the running maximum of s + log2 vs, is what multiplies
// V's codes, and the softmax total sum exp2(s - M) is the sum of each page's w times 1 / vs.  So neither costs an instruction an
// element, and the operands stay exact.
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
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
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
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// Shared-memory operand: rows of 128 bytes (64 float16), 16-byte chunks exchanged by chunk ^ (row & 7) within groups of 8 rows
// (1024 bytes apart).  `lbo`: distance of the next 64 columns where the operand's columns are the contiguous direction.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t lbo) {
    return (uint64_t)((at & 0x3ffffu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// float16 operands, float32 accumulator, 128 rows, n columns; `columns_contiguous`: of the second operand
__host__ __device__ constexpr uint32_t instruction(uint32_t n, bool columns_contiguous) {
    return 1u << 4 | (columns_contiguous ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}

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
struct Blocks {
    uint32_t first, count;                          // key blocks that some row of the tile sees, at least one
};
template <int kRows> __device__ __forceinline__ Blocks tile_blocks(const AttnArgs& a, const PromptSeq& p, uint32_t tile) {
    const uint32_t last_row = min((tile + 1) * kRows, p.rows) - 1;
    const int hi = max(min((int)p.s.length, p.start + (int)(last_row / a.group) + 1), 0);
    const int lo = a.window ? min(max(p.start + (int)(tile * kRows / a.group) - (int)a.window + 1, 0), hi) : 0;
    Blocks b;
    b.first = (uint32_t)lo / kKeys;
    const uint32_t end = ((uint32_t)hi + kKeys - 1) / kKeys;
    b.count = end > b.first ? end - b.first : 1u;
    return b;
}
template <int kRows> __device__ __forceinline__ unsigned long long seq_blocks(const AttnArgs& a, const PromptSeq& p, int lane) {
    unsigned long long n = 0;                       // of one key head; by a whole warp
    for (uint32_t t = lane; t < p.tiles; t += 32) n += tile_blocks<kRows>(a, p, t).count;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) n += __shfl_xor_sync(0xffffffffu, n, d);
    return n;
}

struct Walk {                                       // where in the flat order a thread is; the same in all threads of the block
    unsigned long long at, end, total, parts;
    uint32_t seq, head, tile, block;                // block: of the tile, from its first
};

struct Segment {                                    // a run of blocks of one (sequence, head, tile)
    PromptSeq p;
    uint32_t head, tile, first, count, b0, b1;      // blocks first + [b0, b1) of count
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
    s.head = w.head;
    s.tile = w.tile;
    s.first = b.first;
    s.count = b.count;
    s.b0 = w.block;
    s.b1 = (uint32_t)min((unsigned long long)b.count, (unsigned long long)w.block + (w.end - w.at));
    s.item = w.at - w.block;
    s.rows = min(s.p.rows - w.tile * kRows, (uint32_t)kRows);
    w.at += s.b1 - s.b0;
    w.block = 0;
    if (++w.tile >= s.p.tiles) {
        w.tile = 0;
        if (++w.head >= a.c.heads) {
            w.head = 0;
            ++w.seq;
        }
    }
    return true;
}

constexpr int kPromptThreads = 512;

template <int kRows> __device__ bool walk_start(const AttnArgs& a, Walk& w, unsigned long long* sh) {
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
                const uint32_t t = t0 + lane, c = t < p.tiles ? tile_blocks<kRows>(a, p, t).count : 0u;
                unsigned long long incl = c;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned long long up = __shfl_up_sync(0xffffffffu, incl, d);
                    if (lane >= d) incl += up;
                }
                const unsigned long long f = ahead + incl - c;
                if (c && rest >= f && rest < f + c) {
                    sh[16] = i; sh[17] = head; sh[18] = t; sh[19] = rest - f;
                }
                ahead += __shfl_sync(0xffffffffu, incl, 31);
                if (rest < ahead) break;
            }
        }
        before = all;
        if (w.at < before) break;
    }
    __syncthreads();
    w.seq = (uint32_t)sh[16]; w.head = (uint32_t)sh[17]; w.tile = (uint32_t)sh[18]; w.block = (uint32_t)sh[19];
    return true;
}

// ---- shared state -----------------------------------------------------------------------------------------------------------
constexpr int kRing = 8;                            // steps whose pages and scales are looked up ahead
struct PromptShared {
    uint64_t q_full, q_empty, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2], look_full[kRing], look_free[kRing], join[2],
        drain;
    unsigned long long walk[20];
    int32_t page[kRing][8];                         // of 16 keys each: page (-1: none), key scale, log2 and inverse of the value scale
    float ks[kRing][8], lvs[kRing][8], ivs[kRing][8];
    float q_scale[2][256];                          // of a row, segments in turn: 2^e of its float16 form times scale * log2(e)
    uint32_t tmem, last, failed;
};

// A wait that runs out (1 s) ends the block: the flag makes its other waits give up too.
__device__ __forceinline__ bool wait_on(uint64_t* bar, uint32_t parity, PromptShared& sh) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    for (uint32_t spin = 0; spin < kWaitSpins; ++spin) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*reinterpret_cast<volatile uint32_t*>(&sh.failed)) return false;
        if (global_ns() - t0 > kWaitNs) break;
    }
    *reinterpret_cast<volatile uint32_t*>(&sh.failed) = 1u;
    return false;
}

// The same by a whole warp, with one answer.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, PromptShared& sh) {
    return __all_sync(0xffffffffu, wait_on(bar, parity, sh));
}

// 16 codes to two 16-byte chunks of float16
template <int kFormat> __device__ __forceinline__ void widen(const uint4& c, uint4& x, uint4& y) {
    codes_to_f16<kFormat>(c.x, x.x, x.y);
    codes_to_f16<kFormat>(c.y, x.z, x.w);
    codes_to_f16<kFormat>(c.z, y.x, y.y);
    codes_to_f16<kFormat>(c.w, y.z, y.w);
}

// ---- warpgroup 2: operands ----------------------------------------------------------------------------------------------------
template <int DP, int kFormat, class T>
__device__ void feed(const AttnArgs& a, PromptShared& sh, uint8_t* smem, Walk w) {
    using P = Prompt<DP>;
    constexpr int kUnits = 128 * (DP / 16) / 128;                // 16-code units a thread of a 128-key operand: DP / 16
    constexpr int kPerRow = DP / 16;
    const uint32_t tid = threadIdx.x & 127;
    const KvView& kv = a.c;
    uint8_t* sq = smem;
    uint8_t* sk = smem + P::kTiles * P::kOperand;
    uint8_t* sv = sk + P::kStages * P::kOperand;
    const uint32_t unit = tid % kPerRow, row0 = tid / kPerRow;   // unit e: key row0 + e * (128 / kPerRow), codes [16 * unit, +16)
    constexpr int kRowStep = 128 / kPerRow;
    const uint32_t slab = unit / 4, chunk = (unit & 3) * 2;
    const bool inside = 16 * unit < kv.dim;
    uint32_t step = 0, seg = 0;
    Segment s;
    uint4 kr[kUnits], vr[kUnits];
    while (next_segment<P::kRows>(a, w, s)) {
        // queries: lanes of a row side by side, 8 elements each
        if (seg && !warp_wait(&sh.q_empty, (seg - 1) & 1, sh)) return;
        constexpr int kLanes = DP / 8;
        for (uint32_t r = tid / kLanes; r < (uint32_t)P::kRows; r += 128 / kLanes) {
            const uint32_t c = tid % kLanes;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
            if (r < s.rows && 8 * c < kv.dim) {
                const uint32_t row = s.tile * P::kRows + r, tok = row / a.group;
                const T* q = static_cast<const T*>(a.q) + (long long)(s.p.s.row + tok) * a.q_token +
                             (long long)(s.head * a.group + row - tok * a.group) * a.q_head + 8 * c;
                if (a.q_aligned) {
                    unpack<T>(*reinterpret_cast<const uint4*>(q), x);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = to_f32(q[i]);
                }
            }
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
            int e = (int)(__float_as_uint(amax) >> 23) - 127;    // the row's largest magnitude in [1, 2): see few_rows_kernel
            e = max(min(e, 126), -126);
            const float down = pow2f(-e);
            __half2 h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(x[2 * i] * down, x[2 * i + 1] * down);
            uint8_t* to = sq + (r >> 7) * P::kOperand + (c >> 3) * P::kSlab + (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4);
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(h);
            if (c == 0) sh.q_scale[seg & 1][r] = pow2f(e) * a.scale_log2;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(&sh.q_full);
        ++seg;

        const long long head_off = (long long)s.head * kv.head_step + 16 * unit;
        const int hi_key = (int)min((s.first + s.count) * kKeys, s.p.s.length);
        auto get = [&](const uint8_t* base, uint32_t block, uint32_t ring, uint4* to) {
#pragma unroll
            for (int e = 0; e < kUnits; ++e) {
                const int key = (int)(block * kKeys + row0 + e * kRowStep);
                const int32_t id = sh.page[ring][(row0 + e * kRowStep) >> 4];
                to[e] = make_uint4(0, 0, 0, 0);
                if (id >= 0 && inside && key < hi_key)
                    asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(to[e].x), "=r"(to[e].y), "=r"(to[e].z), "=r"(to[e].w)
                                 : "l"(base + (long long)id * kv.page_stride + head_off + (long long)(key & (kv.page_tokens - 1)) * kv.token_step));
            }
        };
        auto put = [&](uint8_t* base, const uint4* from) {
#pragma unroll
            for (int e = 0; e < kUnits; ++e) {
                const uint32_t row = row0 + e * kRowStep;
                uint4 x, y;
                widen<kFormat>(from[e], x, y);
                uint8_t* to = base + slab * P::kSlab + row * 128;
                // the odd slabs store their second chunk first: the eight lanes of a store then hit different banks
                const bool swap = slab & 1;
                *reinterpret_cast<uint4*>(to + (((chunk + swap) ^ (row & 7)) << 4)) = swap ? y : x;
                *reinterpret_cast<uint4*>(to + (((chunk + !swap) ^ (row & 7)) << 4)) = swap ? x : y;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        };
        if (!warp_wait(&sh.look_full[step % kRing], (step / kRing) & 1, sh)) return;
        get(kv.k, s.first + s.b0, step % kRing, kr);
        get(kv.v, s.first + s.b0, step % kRing, vr);
        for (uint32_t b = s.b0; b < s.b1; ++b, ++step) {
            const uint32_t stage = step % P::kStages, turn = step / P::kStages, ring = (step + 1) % kRing;
            const bool more = b + 1 < s.b1;
            if (turn && !warp_wait(&sh.k_empty[stage], (turn - 1) & 1, sh)) return;
            put(sk + stage * P::kOperand, kr);
            mbar_arrive(&sh.k_full[stage]);
            if (more) {
                if (!warp_wait(&sh.look_full[ring], ((step + 1) / kRing) & 1, sh)) return;
                get(kv.k, s.first + b + 1, ring, kr);
            }
            if (turn && !warp_wait(&sh.v_empty[stage], (turn - 1) & 1, sh)) return;
            put(sv + stage * P::kOperand, vr);
            mbar_arrive(&sh.v_full[stage]);
            if (more) get(kv.v, s.first + b + 1, ring, vr);
        }
    }
}

// ---- warpgroup 3: one warp looks up pages and scales, four steps at a time ------------------------------------------------------
template <int DP>
__device__ void look_up(const AttnArgs& a, PromptShared& sh, Walk w) {
    using P = Prompt<DP>;
    const KvView& kv = a.c;
    const uint32_t lane = threadIdx.x & 31, group = lane & 7;
    uint32_t step = 0;
    Segment s;
    while (next_segment<P::kRows>(a, w, s)) {
        const int32_t* table = kv.pages + (size_t)s.p.s.slot * kv.max_pages;
        const int hi_key = (int)min((s.first + s.count) * kKeys, s.p.s.length);
        const uint32_t n = s.b1 - s.b0;
        for (uint32_t j0 = 0; j0 < n; j0 += 4) {
            const uint32_t j = j0 + (lane >> 3), x = step + j, last = step + min(j0 + 4, n) - 1;
            // products end in order: when the last slot of these four is free, all are
            if (last >= kRing && !warp_wait(&sh.look_free[last % kRing], (last / kRing - 1) & 1, sh)) return;
            if (j < n) {
                const int key = (int)((s.first + s.b0 + j) * kKeys + 16 * group);
                int32_t id = -1;
                if (key < hi_key) {
                    id = __ldg(table + (key >> kv.page_shift));
                    if ((uint32_t)id >= kv.num_pages) {
                        kv_flag(kv.status, ROOMIE_FLAG_KV_PAGE);
                        id = -1;
                    }
                }
                float ks = 0.0f, lvs = -INFINITY, ivs = 0.0f;    // keys that are not there weigh nothing
                if (id >= 0) {
                    ks = __ldg(kv.k_scale + (size_t)id * kv.heads + s.head);
                    const float vs = fmaxf(__ldg(kv.v_scale + (size_t)id * kv.heads + s.head), 7.888609052210118e-31f);   // 2^-100
                    lvs = log2f(vs);
                    ivs = __fdiv_rn(1.0f, vs);
                }
                const uint32_t ring = x % kRing;
                sh.page[ring][group] = id;
                sh.ks[ring][group] = ks;
                sh.lvs[ring][group] = lvs;
                sh.ivs[ring][group] = ivs;
                mbar_arrive(&sh.look_full[ring]);
            }
            __syncwarp();
        }
        step += n;
    }
}

// ---- warpgroup 3: one thread issues the products --------------------------------------------------------------------------------
template <int DP>
__device__ void issue(const AttnArgs& a, PromptShared& sh, uint8_t* smem, Walk w) {
    using P = Prompt<DP>;
    const uint32_t sq = smem_addr(smem), sk = sq + P::kTiles * P::kOperand, sv = sk + P::kStages * P::kOperand;
    const uint32_t tm = sh.tmem;
    constexpr uint32_t kS = instruction(kKeys, false), kO = instruction(DP, true);
    uint32_t step = 0, seg = 0, p_turn[2] = {0, 0};
    Segment s;
    while (next_segment<P::kRows>(a, w, s)) {
        const uint32_t tiles = s.rows > 128 ? 2 : 1, n = s.b1 - s.b0;
        if (!wait_on(&sh.q_full, seg & 1, sh)) return;
        tc_fence_after();
        ++seg;
        for (uint32_t j = 0; j <= n; ++j) {                      // S of step j, o of step j - 1
            const uint32_t stage = (step + j) % P::kStages, turn = (step + j) / P::kStages;
            const uint32_t old = j ? step + j - 1 : 0, old_stage = old % P::kStages, old_turn = old / P::kStages;
            if (j < n && !wait_on(&sh.k_full[stage], turn & 1, sh)) return;
            if (j && !wait_on(&sh.v_full[old_stage], old_turn & 1, sh)) return;
            for (uint32_t t = 0; t < tiles; ++t) {
                const uint32_t s_at = tm + t * 128, o_at = tm + P::kTiles * 128 + t * DP;
                if (j) {
                    if (!wait_on(&sh.p_full[t], p_turn[t] & 1, sh)) return;
                    ++p_turn[t];
                    tc_fence_after();
#pragma unroll
                    for (int i = 0; i < kKeys / 16; ++i)
                        mma_ts(o_at, s_at + 8 * i, operand(sv + old_stage * P::kOperand + i * 2048, P::kSlab), kO, j > 1 || i > 0);
                    tc_commit(&sh.o_full[t]);
                }
                if (j < n) {
#pragma unroll
                    for (int i = 0; i < DP / 16; ++i) {
                        const uint32_t off = (i / 4) * P::kSlab + (i % 4) * 32;
                        mma_ss(s_at, operand(sq + t * P::kOperand + off, 16), operand(sk + stage * P::kOperand + off, 16), kS, i > 0);
                    }
                    tc_commit(&sh.s_full[t]);
                }
            }
            if (j) {
                tc_commit(&sh.v_empty[old_stage]);
                tc_commit(&sh.look_free[old % kRing]);
            }
            if (j < n) tc_commit(&sh.k_empty[stage]);
            if (j + 1 == n) tc_commit(&sh.q_empty);
        }
        step += n;
    }
}

// ---- warpgroups 0 and 1: softmax, and the end of a segment ------------------------------------------------------------------------
template <int DP, class T>
__device__ void softmax(const AttnArgs& a, PromptShared& sh, Walk w) {
    using P = Prompt<DP>;
    const uint32_t t = threadIdx.x >> 7, r = threadIdx.x & 127;  // tile, row
    const uint32_t lanes = (threadIdx.x & 96) << 16;             // this warp's quarter of the tensor memory's lanes
    const uint32_t s_at = sh.tmem + t * 128 + lanes, o_at = sh.tmem + P::kTiles * 128 + t * DP + lanes;
    uint32_t step = 0, s_turn = 0, o_turn = 0, seg = 0, joins = 0;
    Segment s;
    while (next_segment<P::kRows>(a, w, s)) {
        const uint32_t n = s.b1 - s.b0, row = s.tile * P::kRows + t * 128 + r;
        const bool on = t * 128 < s.rows, mine = t * 128 + r < s.rows;
        const int tok = (int)(row / a.group), pos = s.p.start + tok;
        const int hi = mine ? max(min(pos + 1, (int)s.p.s.length), 0) : 0, lo = a.window ? max(pos + 1 - (int)a.window, 0) : 0;
        float m = -INFINITY, l = 0.0f, q = 0.0f;
        for (uint32_t j = 0; on && j < n; ++j) {
            const int k0 = (int)((s.first + s.b0 + j) * kKeys);
            const uint32_t ring = (step + j) % kRing;
            if (!warp_wait(&sh.look_full[ring], ((step + j) / kRing) & 1, sh) || !warp_wait(&sh.s_full[t], s_turn & 1, sh)) return;
            ++s_turn;
            tc_fence_after();
            if (j == 0) q = sh.q_scale[seg & 1][t * 128 + r];
            const bool cut = __any_sync(0xffffffffu, k0 < lo || k0 + kKeys > hi);
            uint32_t x[32];
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                tmem_load32(s_at + 32 * c, x);
                tmem_wait_ld();
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float mx = -INFINITY;
                    if (cut) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int k = k0 + 32 * c + 16 * g + e;
                            mx = fmaxf(mx, k < hi && k >= lo ? __uint_as_float(x[16 * g + e]) : -INFINITY);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, __uint_as_float(x[16 * g + e]));
                    }
                    const float v = fmaf(mx, q * sh.ks[ring][2 * c + g], sh.lvs[ring][2 * c + g]);
                    top = fmaxf(top, mx == -INFINITY ? -INFINITY : v);
                }
            }
            // The sums are taken against an old maximum while the new one is at most 2^8 above it: probabilities then stay below
            // 2^8, far from float16's end, and o is rescaled in tensor memory only now and then.
            const bool far = top > m + 8.0f || m == -INFINITY;
            if (__any_sync(0xffffffffu, far && top > m)) {
                const float to = fmaxf(m, top), f = m == -INFINITY ? 0.0f : exp2_fast(m - to);
                m = to;
                l *= f;
                if (j) {
                    if (!warp_wait(&sh.o_full[t], (o_turn - 1) & 1, sh)) return;
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < DP / 32; ++c) {
                        tmem_load32(o_at + 32 * c, x);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
                        tmem_store32(o_at + 32 * c, x);
                    }
                    tmem_wait_st();
                }
            }
            ++o_turn;
            const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                tmem_load32(s_at + 32 * c, x);
                tmem_wait_ld();
                uint32_t p[16];
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    const float f = q * sh.ks[ring][2 * c + g], off = sh.lvs[ring][2 * c + g] - base;
                    float sum = 0.0f;
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        float u = fmaf(__uint_as_float(x[16 * g + e]), f, off), v = fmaf(__uint_as_float(x[16 * g + e + 1]), f, off);
                        if (cut) {
                            const int k = k0 + 32 * c + 16 * g + e;
                            u = k < hi && k >= lo ? u : -INFINITY;
                            v = k + 1 < hi && k + 1 >= lo ? v : -INFINITY;
                        }
                        u = exp2_fast(u);
                        v = exp2_fast(v);
                        sum += u + v;
                        const __half2 h = __floats2half2_rn(u, v);
                        p[8 * g + e / 2] = reinterpret_cast<const uint32_t&>(h);
                    }
                    l = fmaf(sum, sh.ivs[ring][2 * c + g], l);
                }
                tmem_store16(s_at + 16 * c, p);
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sh.p_full[t]);
        }
        step += n;
        ++seg;

        // ---- the end of a segment: rows go out, or wait in the workspace for their other parts ---------------------------------
        const bool complete = s.b0 == 0 && s.b1 == s.count;
        const uint32_t h = s.head * a.group + row - (uint32_t)tok * a.group;
        T* out = static_cast<T*>(a.out) + (long long)(s.p.s.row + tok) * a.o_token + (long long)h * a.o_head;
        auto put_lse = [&](float mx, float sum) {
            if (a.lse) a.lse[(size_t)(s.p.s.row + tok) * a.q_heads + h] = sum > 0.0f ? (mx + log2f(sum)) * kLn2 : sum == 0.0f ? -INFINITY : sum;
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
            if (!warp_wait(&sh.o_full[t], (o_turn - 1) & 1, sh)) return;
            tc_fence_after();
            const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == 0.0f ? 0.0f : l;
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
                uint32_t x[32];
                tmem_load32(o_at + 32 * c, x);
                tmem_wait_ld();
                if (complete) {
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = l == 0.0f ? 0.0f : __uint_as_float(x[e]) * inv;
                    if (mine)
#pragma unroll
                        for (int e = 0; e < 32; e += 8) put8(32 * c + e, v + e);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<uint4*>(part + ((size_t)(8 * c + e / 4) * P::kRows + pr) * 4) = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
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
            const uint32_t first = (uint32_t)(((s.item + 1) * w.parts - 1) / w.total);
            const uint32_t last = (uint32_t)(((s.item + s.count) * w.parts - 1) / w.total);
            __threadfence();
            mbar_arrive(&sh.join[0]);
            if (threadIdx.x < 32) {
                if (!warp_wait(&sh.join[0], joins & 1, sh)) return;
                if (threadIdx.x == 0) {
                    const uint32_t before = atomicAdd(a.counters + first, 1u);
                    sh.last = before == last - first;
                    if (before == last - first) a.counters[first] = 0;
                    mbar_arrive(&sh.join[1]);
                }
            }
            if (!warp_wait(&sh.join[1], joins & 1, sh)) return;
            ++joins;
            if (sh.last && mine) {
                __threadfence();
                float mx = -INFINITY, sum = 0.0f;
                for (uint32_t b = first; b <= last; ++b) {
                    const float* pp = a.partial + ((size_t)b * 2 + (b == first ? 1 : 0)) * P::kPartial + (size_t)P::kRows * DP + 2 * pr;
                    const float mb = __ldcg(pp), lb = __ldcg(pp + 1), to = fmaxf(mx, mb);
                    sum = (mx == -INFINITY ? 0.0f : sum * exp2f(mx - to)) + (mb == -INFINITY ? 0.0f : lb * exp2f(mb - to));
                    mx = to;
                }
                const float inv = sum > 0.0f ? __fdiv_rn(1.0f, sum) : sum == 0.0f ? 0.0f : sum;
                for (int d = 0; d < (int)a.c.dim; d += 8) {
                    float v[8] = {};
                    for (uint32_t b = first; b <= last; ++b) {
                        const float* pp = a.partial + ((size_t)b * 2 + (b == first ? 1 : 0)) * P::kPartial;
                        const float mb = __ldcg(pp + (size_t)P::kRows * DP + 2 * pr);
                        const float f = mb == -INFINITY ? 0.0f : exp2f(mb - mx) * inv;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float4 x = __ldcg(reinterpret_cast<const float4*>(pp + ((size_t)(d / 4 + i) * P::kRows + pr) * 4));
                            v[4 * i] += f * x.x; v[4 * i + 1] += f * x.y; v[4 * i + 2] += f * x.z; v[4 * i + 3] += f * x.w;
                        }
                    }
                    put8(d, v);
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
        mbar_init(&sh.q_full, 128);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.k_full[i], 128);
            mbar_init(&sh.v_full[i], 128);
            mbar_init(&sh.k_empty[i], 1);
            mbar_init(&sh.v_empty[i], 1);
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_full[i], 128);
            mbar_init(&sh.o_full[i], 1);
        }
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&sh.look_full[i], 8);
            mbar_init(&sh.look_free[i], 1);
        }
        mbar_init(&sh.join[0], 128 * P::kTiles);
        mbar_init(&sh.join[1], 1);
        mbar_init(&sh.drain, 1);
        sh.failed = 0;
    }
    if (wid == 12) tmem_alloc(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (wid < 4 * P::kTiles) {
        softmax<DP, T>(a, sh, w);
    } else if (wid >= 8 && wid < 12) {
        feed<DP, kFormat, T>(a, sh, smem, w);
    } else if (wid == 13) {
        look_up<DP>(a, sh, w);
    } else if (threadIdx.x == 12 * 32) {
        issue<DP>(a, sh, smem, w);
        tc_commit(&sh.drain);                                    // whatever was issued has ended before the memory is given back
        wait_on(&sh.drain, 0, sh);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && sh.failed) kv_flag(a.c.status, ROOMIE_FLAG_WAIT_TIMEOUT);
    if (wid == 12) tmem_free(sh.tmem, 512);
}

size_t prompt_partial_bytes(uint32_t dim) {
    const size_t floats = dim <= 64 ? Prompt<64>::kPartial : dim <= 128 ? Prompt<128>::kPartial : Prompt<256>::kPartial;
    return (size_t)sm_count() * 2 * floats * sizeof(float);
}

template <int DP, int kFormat, class T> static int launch_one(const AttnArgs& a, cudaStream_t st) {
    return launch("kv_attention_prompt", prompt_kernel<DP, kFormat, T>, dim3((uint32_t)sm_count()), dim3(kPromptThreads), Prompt<DP>::kSmem,
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
