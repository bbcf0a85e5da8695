// The attention weight that cached keys have received: for each key of a sequence and key head, the sum over the call's rows that see it of
// exp(scale * ks[page] * q_i.k_j - lse_i).
//
// Every key's sum is one thread's (or one warp's, in a fixed order): nothing is joined, and a call repeats bit for bit.
#include <cuda.h>
#include <type_traits>
#include "roomie_kv_attention.cuh"
#include "roomie_tc.cuh"

namespace roomie {

struct WeightArgs {
    KvView c;
    const int32_t *seqs, *q_offset;
    uint32_t num_seqs, rows, q_heads, group;
    uint32_t block_tokens, block_heads;              // of a block of rows: 32 / group and group, or 1 and 32
    int32_t tensor_copies;
    const void* q;
    long long q_token, q_head;
    const float* lse;                                // [rows][q_heads]
    float* weight;                                   // of the layer: [max_seqs][heads][max_tokens]
    uint32_t max_tokens, window;
    float scale_log2;
    int32_t q_aligned, fresh;
};

constexpr float kLog2e = 1.44269504088896340736f;

// ---- few rows a key head -----------------------------------------------------------------------------------------------------------
// As in attention over few rows: S^T = K q^T by 16x8x16 products, a lane's span of a key contiguous, every warp with steps of codes under way to its
// own part of shared memory.  The flat order (sequence, head, step of keys) is cut into equal shares for the call's warps.  Bound by the bytes
// of the codes: 64 sequences of up to 16384 keys (764 MB) take 145 us, 5280 GB/s; of up to 4096 (191 MB) 45, of which 10 are the way from the lengths over
// the table to the first codes.  Instructions come next (some 450 of a warp for 32 keys): with places in the flat order worked out anew for each
// step it took 60, with 12 warps an SM instead of 16 51.
constexpr int kWeightWarps = 4, kWeightThreads = 32 * kWeightWarps;

template <int DP> struct FewWeights {
    static constexpr int kGroups = DP > 128 ? 1 : 2;                // 16-key groups of a step
    static constexpr int kStep = 16 * kGroups;
    static constexpr int kSide = kStep * DP;                        // bytes of a step's keys
    static constexpr int kStages = 12288 / kSide;                   // 12 KB a warp
    static constexpr int kStage = kSide + kStep * 4 + 16;           // codes, the keys' old weights, the groups' scales
    static constexpr int kRing = kStages * kStage;
    static constexpr int kSmem = kRing * kWeightWarps;
};
constexpr int kWeightBlocks = 4;                                    // of an SM: 16 warps with 128 registers a thread

struct WeightSeq {                                   // a sequence of the call, as its warps need it
    unsigned long long first;                        // flat index of its first step
    uint32_t slot, row, count, length, step0, steps; // step0: a head's first step, of `steps`
};

// Whether the call may name a sequence twice: a bit for each slot, or for each group of slots where there are more than bits.
struct SlotBits {
    uint32_t *bits, words;
    __device__ __forceinline__ bool seen(uint32_t slot, uint32_t max_seqs) const {       // and from now on it is
        const uint32_t bit = words * 32 >= max_seqs ? slot : slot % (words * 32);
        return slot < max_seqs && (atomicOr(bits + bit / 32, 1u << (bit & 31)) >> (bit & 31) & 1);
    }
};
// All threads of the block.  A call of one `batch` is asked about when its sequences have come anyway (a pass in front of them: 0.6 us), a longer one here.
__device__ __forceinline__ bool maybe_twice(const WeightArgs& a, SlotBits& b, uint32_t batch) {
    b.words = min(b.words, (a.c.max_seqs + 31) / 32);
    for (uint32_t w = threadIdx.x; w < b.words; w += blockDim.x) b.bits[w] = 0;
    if (a.num_seqs <= batch) return false;
    __syncthreads();
    bool twice = false;
    for (uint32_t i = threadIdx.x; i < a.num_seqs; i += 8 * blockDim.x) {           // eight under way (2000 sequences: 6.5 us, one 8)
        int32_t slot[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) slot[k] = i + k * blockDim.x < a.num_seqs ? a.seqs[i + k * blockDim.x] : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) twice |= b.seen((uint32_t)slot[k], a.c.max_seqs);
    }
    return __syncthreads_or(twice) != 0;
}
// ... and if so, whether an earlier one of the call is the same as the i-th.
__device__ __forceinline__ bool named_before(const WeightArgs& a, uint32_t i, bool report) {
    const int32_t slot = a.seqs[i];
    bool before = false;
    for (uint32_t j = 0; j < i && !before; ++j) before = a.seqs[j] == slot;
    if (before && report) kv_flag(a.c.status, ROOMIE_FLAG_KV_SEQUENCE);
    return before;
}

template <int DP, int kFormat, class T>
__global__ void __launch_bounds__(kWeightThreads, kWeightBlocks) few_weights_kernel(WeightArgs a) {
    using F = FewWeights<DP>;
    constexpr int G = F::kGroups, KW = DP / 16, KS = DP / 16, kStages = F::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ WeightSeq sh_seq[kWeightThreads];
    __shared__ unsigned long long sh_sum[kWeightWarps];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const KvView& kv = a.c;
    uint8_t* ring = smem + wid * F::kRing;
    const unsigned long long me = (unsigned long long)blockIdx.x * kWeightWarps + wid, all_warps = (unsigned long long)gridDim.x * kWeightWarps;
    SlotBits slots = {reinterpret_cast<uint32_t*>(smem), F::kSmem / 4};
    bool twice = maybe_twice(a, slots, kWeightThreads);

    for (uint32_t base = 0; base < a.num_seqs; base += kWeightThreads) {
        const uint32_t here = min(a.num_seqs - base, (uint32_t)kWeightThreads);
        __syncthreads();
        unsigned long long mine = 0;
        WeightSeq w = {};
        if (threadIdx.x < here) {
            const KvSeq s = kv_seq(kv, a.seqs, a.q_offset, a.rows, base + threadIdx.x, blockIdx.x == 0);
            w.slot = s.slot; w.row = s.row; w.count = s.count; w.length = s.length;
            const int start = (int)s.length - (int)s.count;
            const uint32_t low = a.fresh ? 0u : a.window ? min((uint32_t)first_seen(start, a.window), s.length) : 0u;
            w.step0 = low / F::kStep;
            w.steps = s.count ? (s.length + F::kStep - 1) / F::kStep - w.step0 : 0u;
            mine = (unsigned long long)w.steps * kv.heads;
        }
        if (a.num_seqs > 1 && a.num_seqs <= kWeightThreads) twice = __syncthreads_or(threadIdx.x < here && slots.seen((uint32_t)a.seqs[threadIdx.x], kv.max_seqs)) != 0;
        if (twice && threadIdx.x < here && named_before(a, base + threadIdx.x, blockIdx.x == 0)) mine = w.steps = 0;
        unsigned long long upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += up;
        }
        if (lane == 31) sh_sum[wid] = upto;
        __syncthreads();
        unsigned long long total = 0;
        for (int x = 0; x < kWeightWarps; ++x) {
            if (x < wid) upto += sh_sum[x];
            total += sh_sum[x];
        }
        w.first = upto - mine;
        sh_seq[threadIdx.x] = w;
        __syncthreads();
        const unsigned long long at = total * me / all_warps, end = total * (me + 1) / all_warps;     // total < 2^50: 128 x 2^27 x 2^16
        if (at >= end) continue;
        uint32_t seq = 0;                                           // the last one whose first step is at most `at`, of those that have steps
        for (uint32_t x = lane; x < here; x += 32)
            if (sh_seq[x].steps && sh_seq[x].first <= at) seq = x;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) seq = max(seq, __shfl_xor_sync(0xffffffffu, seq, d));

        // ---- two places in the flat order: of the products, and some steps ahead of the copies ----
        struct Place {
            uint32_t seq, head, steps;                              // steps: of this (sequence, head) from here on
            unsigned long long left;                                // of the warp's share
            int key, length;                                        // first key of the step; the sequence's length
        };
        const unsigned long long inside = at - sh_seq[seq].first;
        Place now;
        now.seq = seq;
        now.head = (uint32_t)(inside / sh_seq[seq].steps);
        now.left = end - at;
        {
            const uint32_t step = (uint32_t)(inside - (unsigned long long)now.head * sh_seq[seq].steps);
            now.steps = sh_seq[seq].steps - step;
            now.key = (int)(sh_seq[seq].step0 + step) * F::kStep;
            now.length = (int)sh_seq[seq].length;
        }
        Place next = now;
        auto go_on = [&](Place& p) {                                // true: another (sequence, head)
            --p.left;
            p.key += F::kStep;
            if (--p.steps || !p.left) return false;
            if (++p.head == kv.heads) {
                p.head = 0;
                do ++p.seq; while (sh_seq[p.seq].steps == 0);
            }
            p.steps = sh_seq[p.seq].steps;
            p.key = (int)sh_seq[p.seq].step0 * F::kStep;
            p.length = (int)sh_seq[p.seq].length;
            return true;
        };
        constexpr int kChunks = DP / 16, kRowsPer = 32 / kChunks, kLoads = 16 / kRowsPer;      // of a group: row0 + i * kRowsPer
        const uint32_t chunk = lane % kChunks, row0 = lane / kChunks;
        const bool real = 16 * chunk < kv.dim;
        const uint32_t ring_at = smem_addr(ring), place0 = code_at<DP>(row0, chunk);
        const int32_t* table;                                       // of the copies' (sequence, head)
        const uint8_t* codes;
        const float *was, *scales;
        int low, known;                                             // keys before `low` no row sees; those before `known` have received something before
        auto enter = [&] {
            const WeightSeq& s = sh_seq[next.seq];
            const int start = (int)s.length - (int)s.count;
            table = kv.pages + (size_t)s.slot * kv.max_pages;
            codes = kv.k + (long long)next.head * kv.head_step + (real ? 16 * chunk : 0) + (long long)row0 * kv.token_step;
            was = a.weight + ((size_t)s.slot * kv.heads + next.head) * a.max_tokens;
            scales = kv.k_scale + next.head;
            low = a.window ? first_seen(start, a.window) : 0;
            known = a.fresh ? 0 : start;
        };
        int32_t page[G];
        auto get_pages = [&] {                                      // of the step that is copied next
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int k = next.key + 16 * g;
                page[g] = -1;
                if (next.left && k < next.length && k + 16 > low) {
                    page[g] = __ldg(table + (k >> kv.page_shift));
                    if ((uint32_t)page[g] >= kv.num_pages) {
                        if (lane == 0) kv_flag(kv.status, ROOMIE_FLAG_KV_PAGE);
                        page[g] = -1;
                    }
                }
            }
        };
        auto copy_step = [&](uint32_t to) {                         // of `next`, which moves on
            if (next.left) {
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int k = next.key + 16 * g;
                    const uint8_t* p = codes + (long long)max(page[g], 0) * kv.page_stride + (long long)(k & (int)(kv.page_tokens - 1)) * kv.token_step;
                    const int rows = page[g] >= 0 && real ? next.length - k - (int)row0 : 0;   // the rest becomes zeros
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) {
                        // row r of a step lies at code_at(r): rows kRowsPer apart differ in the chunks' exchange by those bits
                        const uint32_t d = (DP >= 128 ? place0 ^ ((kRowsPer * i & 7) << 4) : place0) + (16 * g + kRowsPer * i) * DP;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + d), "l"(p), "r"(i * kRowsPer < rows ? 16u : 0u) : "memory");
                        p += kRowsPer * kv.token_step;
                    }
                }
                if (lane < F::kStep) {
                    const int k = next.key + lane;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + F::kSide + 4 * lane), "l"(k < known ? was + k : was), "r"(k < known ? 4u : 0u)
                                 : "memory");
                }
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (lane == g) {
                        const uint32_t d = to + F::kSide + 4 * F::kStep + 4 * g;
                        if (page[g] < 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(d), "f"(-1.0f) : "memory");       // no page
                        else
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(d), "l"(scales + (size_t)page[g] * kv.heads) : "memory");
                    }
                if (go_on(next)) enter();
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        enter();
        get_pages();
#pragma unroll 1
        for (int i = 0; i < kStages; ++i) {
            copy_step(ring_at + i * F::kStage);
            get_pages();
        }

        // ---- queries of eight rows: operand b of S^T, row r of them, dims as the lane's keys ----
        uint32_t qf[KS][2];
        float qscale[2], lse2[2];
        int see_hi[2], see_lo[2];                                   // rows 2c and 2c + 1 of the eight see keys [lo, hi)
        int all_hi, all_lo;                                         // every one of the rows sees [all_lo, all_hi)
        auto load_queries = [&](const WeightSeq& s, uint32_t head, uint32_t first_row) {
            const uint32_t rows = s.count * a.group;
            all_hi = 0x7fffffff;
            all_lo = 0;
            const uint32_t row = first_row + r, tok = row / a.group;
            const bool on = row < rows;
            const T* q = static_cast<const T*>(a.q);
            if (on) q += (long long)(s.row + tok) * a.q_token + (long long)(head * a.group + row - tok * a.group) * a.q_head + c * (DP / 4);
            float x[DP / 4], amax = 0.0f;
#pragma unroll
            for (int d = 0; d < DP / 4; ++d) x[d] = 0.0f;
            if (on) {
                if (a.q_aligned) {
#pragma unroll
                    for (int d = 0; d < DP / 4; d += 8)
                        if (c * (DP / 4) + d < kv.dim) unpack<T>(*reinterpret_cast<const uint4*>(q + d), x + d);
                } else {
#pragma unroll
                    for (int d = 0; d < DP / 4; ++d)
                        if (c * (DP / 4) + d < kv.dim) x[d] = to_f32(q[d]);
                }
            }
#pragma unroll
            for (int d = 0; d < DP / 4; ++d) amax = fmaxf(amax, fabsf(x[d]));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            // To float16 with the row's largest magnitude in [1, 2): exact for float16 and bfloat16 queries but for elements below
            // 2^-14 of it, which lose at most 2^-25 of it.
            int e = (int)(__float_as_uint(amax) >> 23) - 127;
            e = max(min(e, 126), -126);
            const float down = pow2f(-e);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const __half2 lo = __floats2half2_rn(x[4 * i] * down, x[4 * i + 1] * down);
                const __half2 hi = __floats2half2_rn(x[4 * i + 2] * down, x[4 * i + 3] * down);
                qf[i][0] = reinterpret_cast<const uint32_t&>(lo);
                qf[i][1] = reinterpret_cast<const uint32_t&>(hi);
            }
            const float up = pow2f(e) * a.scale_log2;
            const float own = on ? a.lse[(size_t)(s.row + tok) * a.q_heads + head * a.group + row - tok * a.group] * kLog2e : 0.0f;
            const int start = (int)s.length - (int)s.count;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                qscale[n] = __shfl_sync(0xffffffffu, up, (2 * c + n) * 4);
                lse2[n] = __shfl_sync(0xffffffffu, own, (2 * c + n) * 4);
                const uint32_t rc = first_row + 2 * c + n;
                const int pos = start + (int)(rc / a.group);
                see_hi[n] = rc < rows ? max(min(pos + 1, (int)s.length), 0) : 0;
                see_lo[n] = a.window ? first_seen(pos, a.window) : 0;
                if (rc >= rows) lse2[n] = INFINITY;          // takes no part, whether its keys are looked at one by one or not
                else {
                    all_hi = min(all_hi, see_hi[n]);
                    all_lo = max(all_lo, see_lo[n]);
                }
            }
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, d));
                all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, d));
            }
        };

        bool fresh_queries = true;
        int stage = 0;
        float* weight = a.weight + ((size_t)sh_seq[now.seq].slot * kv.heads + now.head) * a.max_tokens;
        uint32_t rows = sh_seq[now.seq].count * a.group;
        const uint32_t place = 16 * (c >> 1) + 8 * (c & 1) + r;     // a key's rows lie in four lanes; lane c writes key r + 8 * (c & 1) of group c >> 1
        while (now.left) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            __syncwarp();
            const uint8_t* side = ring + stage * F::kStage;
            const float* old = reinterpret_cast<const float*>(side + F::kSide);
            float ks[G], sum[G][2];
            bool pages = true;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                ks[g] = old[F::kStep + g];
                pages = pages && ks[g] >= 0.0f;
                sum[g][0] = sum[g][1] = 0.0f;
            }
            for (uint32_t first_row = 0; first_row < rows; first_row += 8) {
                if (fresh_queries) load_queries(sh_seq[now.seq], now.head, first_row);
                fresh_queries = rows > 8;                             // a chunk among single tokens
                float sc[G][4];
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    sc[g][0] = sc[g][1] = sc[g][2] = sc[g][3] = 0.0f;
                    uint32_t kr[2][KW];
                    read_span<DP, KW>(kr[0], side, 16 * g + r, c * (DP / 4));
                    read_span<DP, KW>(kr[1], side, 16 * g + r + 8, c * (DP / 4));
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        uint32_t a0, a1, a2, a3;
                        codes_to_f16<kFormat>(kr[0][i], a0, a2);
                        codes_to_f16<kFormat>(kr[1][i], a1, a3);
                        mma16816(sc[g], a0, a1, a2, a3, qf[i][0], qf[i][1]);
                    }
                }
                // sc[e] is key r + 8 * (e >> 1) of the group, row 2c + (e & 1)
                const bool whole = pages && now.key >= all_lo && now.key + F::kStep <= all_hi;
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const float f = qscale[n] * ks[g];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float x = fmaf(sc[g][2 * h + n], f, -lse2[n]);
                            if (!whole) {
                                const int k = now.key + 16 * g + 8 * h + r;
                                if (k >= see_hi[n] || k < see_lo[n] || ks[g] < 0.0f) x = -INFINITY;
                            }
                            sum[g][h] += exp2_fast(x);
                        }
                    }
            }
            float mine = 0.0f;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = sum[g][h];
                    x += __shfl_xor_sync(0xffffffffu, x, 1);
                    x += __shfl_xor_sync(0xffffffffu, x, 2);
                    if (c == 2 * g + h) mine = x;
                }
            const int key = now.key + (int)place;
            if (c < 2 * G && key < now.length) weight[key] = old[place] + mine;
            __syncwarp();                                           // the stage is read
            copy_step(ring_at + stage * F::kStage);
            get_pages();
            if (++stage == kStages) stage = 0;
            if (go_on(now)) {
                fresh_queries = true;
                weight = a.weight + ((size_t)sh_seq[now.seq].slot * kv.heads + now.head) * a.max_tokens;
                rows = sh_seq[now.seq].count * a.group;
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
}

// ---- many rows a key head ----------------------------------------------------------------------------------------------------------
// Products on the fifth-generation tensor cores, transposed: S^T = K q^T with 128 keys as the accumulator's rows, so that a thread owns a key: it
// reads its key's products with 32 query rows after the other from tensor memory and adds up their exponentials.  Nothing is exchanged between
// threads, and a key's scale is a factor of its thread.  The keys are the operand that stays: widened to q's type (exactly) they lie in tensor
// memory too, so that a product reads only the queries from shared memory.
//
// A block has 128 keys of one (sequence, key head) at a time.  Warps 0 to 3 widen the codes and take the exponentials; warp 4 issues the products;
// warp 5 brings the queries, up to 32 rows at a time, by tensor copies (rows that are not aligned to 16 bytes: by hand), warp 6 the codes of the next keys
// by asynchronous copies.  What bounds it are the exponentials: 64 queries of 32 heads on 8 over four times up to 16384 keys, 87 million of them, are
// 19 us of special-function time and take 50; 1024 queries 526 (310).  Some 1700 cycles go by for a block of 32 rows, 1024 of them exponentials of the
// SM's four blocks, and 5000 for a unit's codes, widening and first product.  (Keys as shared-memory operands, 256 at a time, two blocks an SM: 63;
// queries by asynchronous copies of two warps, 2400 cycles of instructions a block: 79.)
// Four blocks share an SM (two with heads of more than 128): while one waits or widens, the others keep the
// special-function units busy.  A block of rows is whole tokens of the group, or part of one where the group has more than 32 heads.
constexpr int kManyThreads = 224, kManyRows = 32, kManyKeys = 128, kManySeqs = 128;
constexpr int kQueryStages = 4;                      // of 32 rows
constexpr int kLseStages = 8;                        // the queries are at most four blocks ahead of the products, and these at most three of the exponentials

template <int DP> struct Many {
    static constexpr uint32_t kCodes = kManyKeys * DP;              // bytes: codes of 128 keys
    static constexpr uint32_t kRowSlab = kManyRows * 128, kRowOperand = DP / 64 * kRowSlab;   // 64-column slabs of 32 query rows
    static constexpr uint32_t kSmem = kCodes + kQueryStages * kRowOperand + 1024;
    static constexpr uint32_t kColumns = DP > 128 ? 256 : 128;      // of tensor memory: two S of 32, then the keys' DP / 2
    static constexpr int kPerSm = DP > 128 ? 2 : 4;
};
struct ManyShared {
    uint64_t codes_full, codes_empty, k_full, q_full[kQueryStages], q_empty[kQueryStages], s_full[2], s_empty[2], drain;
    __align__(16) float lse[kLseStages][kManyRows];  // of the rows, negated and in powers of two; -infinity: no row
    float ks[8];                                     // of 16 keys each; -1: no page
    WeightSeq seq[kManySeqs];
    unsigned long long sum[kManyThreads / 32];
    uint32_t tmem, failed;
};

struct ManyUnit {                                    // 128 keys of a (sequence, head), and the tokens whose rows see some of them
    uint32_t seq, head, k0, t0, t1;
};
__device__ __forceinline__ ManyUnit many_unit(const WeightArgs& a, const ManyShared& sh, uint32_t here, unsigned long long at) {
    uint32_t lo = 0, hi = here;                      // the last one of those that begin at or before `at`: it is not empty
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (sh.seq[mid].first <= at) lo = mid;
        else hi = mid;
    }
    const WeightSeq& s = sh.seq[lo];
    ManyUnit u;
    const uint32_t inside = (uint32_t)(at - s.first);
    u.seq = lo;
    u.head = inside / s.steps;
    u.k0 = (s.step0 + inside - u.head * s.steps) * kManyKeys;
    const long long start = (long long)s.length - s.count, last = min(u.k0 + kManyKeys, s.length) - 1ll;
    const long long t0 = max(0ll, (long long)u.k0 - start), t1 = a.window ? min((long long)s.count, last + a.window - start) : (long long)s.count;
    u.t0 = (uint32_t)t0;
    u.t1 = t1 > t0 ? (uint32_t)t1 : u.t0;
    return u;
}
// The unit's blocks of rows: tokens [t, t + tokens), heads [h, h + heads) of the group; f(t, h).  false from f ends it.
template <class F> __device__ __forceinline__ bool row_blocks(const WeightArgs& a, uint32_t t0, uint32_t t1, F f) {
    for (uint32_t t = t0; t < t1; t += a.block_tokens)
        for (uint32_t h = 0; h < a.group; h += a.block_heads)
            if (!f(t, h)) return false;
    return true;
}

// 16 codes to eight pairs of T
template <int kFormat, class T> __device__ __forceinline__ void widen_to(const uint4& c, uint32_t* x) {
    codes_to_f16<kFormat>(c.x, x[0], x[1]);
    codes_to_f16<kFormat>(c.y, x[2], x[3]);
    codes_to_f16<kFormat>(c.z, x[4], x[5]);
    codes_to_f16<kFormat>(c.w, x[6], x[7]);
    if constexpr (!std::is_same<T, __half>::value) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = __half22float2(reinterpret_cast<const __half2&>(x[i]));
            const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
            x[i] = reinterpret_cast<const uint32_t&>(b);
        }
    }
}

// Where piece `piece` of key `row` lies among the codes: exchanged so that the 8 lanes of an access hit different banks, by rows in the reading, by
// pieces in the writing.
template <int DP> __device__ __forceinline__ uint32_t piece_at(uint32_t row, uint32_t piece) {
    if constexpr (DP == 64) return row * 64 + ((piece ^ (row >> 1 & 3)) << 4);
    return row * DP + ((piece ^ (row & 7)) << 4);
}

// Adds the exponentials of 16 products to two pairs of sums; cut: of columns [c0, c1) alone.
template <bool kCut> __device__ __forceinline__ void weigh16(const uint32_t* x, const ulonglong2* minus, uint64_t f2, int c0, int c1, uint64_t* sum) {
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        const ulonglong2 m = minus[e / 4];
#pragma unroll
        for (int o = 0; o < 4; o += 2) {
            float v, w;
            split(fma2(pair(x[e + o], x[e + o + 1]), f2, o ? m.y : m.x), v, w);
            if (kCut) {
                if (e + o < c0 || e + o >= c1) v = -INFINITY;
                if (e + o + 1 < c0 || e + o + 1 >= c1) w = -INFINITY;
            }
            sum[o / 2] = add2(sum[o / 2], pair(exp2_fast(v), exp2_fast(w)));
        }
    }
}

// warps 0 to 3
template <int DP, int kFormat, class T>
__device__ __forceinline__ void many_sums(const WeightArgs& a, ManyShared& sh, const uint8_t* codes, uint32_t here, unsigned long long at, unsigned long long end, uint32_t& block,
                                          uint32_t& units) {
    const KvView& kv = a.c;
    const uint32_t tid = threadIdx.x, tm = sh.tmem + ((tid & 96) << 16);
    for (; at < end; at += gridDim.x) {
        const ManyUnit u = many_unit(a, sh, here, at);
        const WeightSeq& s = sh.seq[u.seq];
        const int start = (int)s.length - (int)s.count;
        const uint32_t key = u.k0 + tid;
        const bool mine = key < s.length;
        float* weight = a.weight + ((size_t)s.slot * kv.heads + u.head) * a.max_tokens + key;
        const float old = mine && !a.fresh && key + s.count < s.length ? *weight : 0.0f;
        float total = 0.0f;
        if (u.t1 > u.t0) {
            if (!warp_wait(&sh.codes_full, units & 1, sh)) return;
            ++units;
            const float ks = sh.ks[tid >> 4], f = ks * a.scale_log2;
#pragma unroll
            for (int h = 0; h < DP / 64; ++h) {                      // 64 elements at a time: 32 columns
                uint32_t x[32];
#pragma unroll
                for (int e = 0; e < 4; ++e) widen_to<kFormat, T>(*reinterpret_cast<const uint4*>(codes + piece_at<DP>(tid, 4 * h + e)), x + 8 * e);
                tmem_store32(tm + 2 * kManyRows + 32 * h, x);
            }
            mbar_arrive(&sh.codes_empty);
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sh.k_full);
            // the tokens that see this key: [lo, hi)
            const int lo = max((int)key - start, 0), hi = a.window ? (int)min((long long)s.count, (long long)key + a.window - start) : (int)s.count;
            const uint64_t f2 = pair(f, f);
            uint64_t sum[2] = {0, 0};
            // 16 columns at a time: while their exponentials are taken the next 16 come, of this block or the next
            uint32_t x[2][16];
            if (!warp_wait(&sh.s_full[block & 1], (block >> 1) & 1, sh)) return;
            tc_fence_after();
            tmem_load16(tm + (block & 1) * kManyRows, x[0]);
            const bool done = row_blocks(a, u.t0, u.t1, [&](uint32_t t, uint32_t h) {
                const uint32_t side = block & 1;
                // of the block's columns, those that this key is to be weighed by: [c0, c1)
                const int tokens = (int)min(a.block_tokens, u.t1 - t), c0 = min(max(lo - (int)t, 0), (int)a.block_tokens) * (int)a.block_heads;
                int c1 = min(max(hi - (int)t, 0), tokens) * (int)a.block_heads;
                if (a.block_tokens == 1) c1 = min(c1, (int)(a.group - h));            // a part of the group's heads
                const bool cut = __any_sync(0xffffffffu, c0 > 0 || c1 < (int)(a.block_tokens * a.block_heads));
                const ulonglong2* minus = reinterpret_cast<const ulonglong2*>(sh.lse[block & (kLseStages - 1)]);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    tmem_wait16(x[half]);
                    if (half == 0) {
                        tmem_load16(tm + side * kManyRows + 16, x[1]);
                    } else {
                        tc_fence_before();
                        mbar_arrive(&sh.s_empty[side]);              // the columns are read
                        if (h + a.block_heads < a.group || t + a.block_tokens < u.t1) {
                            if (!warp_wait(&sh.s_full[side ^ 1], ((block + 1) >> 1) & 1, sh)) return false;
                            tc_fence_after();
                            tmem_load16(tm + (side ^ 1) * kManyRows, x[0]);
                        }
                    }
                    if (cut) weigh16<true>(x[half], minus + 4 * half, f2, c0 - 16 * half, c1 - 16 * half, sum);
                    else weigh16<false>(x[half], minus + 4 * half, f2, 0, 0, sum);
                }
                ++block;
                return true;
            });
            if (!done) return;
            float even, odd;
            split(add2(sum[0], sum[1]), even, odd);
            if (!(ks < 0.0f)) total = even + odd;
        }
        if (mine) *weight = old + total;
    }
}

// warp 4
template <int DP, class T>
__device__ __forceinline__ void many_issue(const WeightArgs& a, ManyShared& sh, const uint8_t* queries, uint32_t here, unsigned long long at, unsigned long long end,
                                           uint32_t& block, uint32_t& units) {
    using M = Many<DP>;
    const uint32_t q0 = operand(smem_addr(queries), 16), tm = __shfl_sync(0xffffffffu, sh.tmem, 0);
    constexpr uint32_t kS = instruction(kManyRows, false) | (std::is_same<T, __half>::value ? 0u : 1u << 7 | 1u << 10);     // both operands bfloat16
    for (; at < end; at += gridDim.x) {
        const ManyUnit u = many_unit(a, sh, here, at);
        const uint32_t t0 = __shfl_sync(0xffffffffu, u.t0, 0), t1 = __shfl_sync(0xffffffffu, u.t1, 0);
        if (t0 >= t1) continue;
        if (!warp_wait(&sh.k_full, units & 1, sh)) return;
        ++units;
        const bool done = row_blocks(a, t0, t1, [&](uint32_t, uint32_t) {
            const uint32_t side = block & 1, stage = block & (kQueryStages - 1);
            if (!warp_wait(&sh.q_full[stage], block / kQueryStages & 1, sh)) return false;
            if (block >= 2 && !warp_wait(&sh.s_empty[side], ((block >> 1) - 1) & 1, sh)) return false;
            tc_fence_after();
            const uint32_t q = q0 + stage * (M::kRowOperand >> 4), to = tm + side * kManyRows, k = tm + 2 * kManyRows;
            if (elected()) {
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) mma_ts(to, k + 8 * i, q + (((i / 4) * M::kRowSlab + (i % 4) * 32) >> 4), kS, i > 0);
                tc_commit(&sh.s_full[side]);
                tc_commit(&sh.q_empty[stage]);
                mbar_arrive(&sh.s_full[side]);                       // and hands on what came with q_full: the rows' lse
            }
            __syncwarp();
            ++block;
            return true;
        });
        if (!done) return;
    }
}

// warp 5.  The rows of a block are asked for when those kQueryStages before it have been read by their product.
template <int DP, class T>
__device__ __forceinline__ void many_queries(const WeightArgs& a, const CUtensorMap* map, ManyShared& sh, uint8_t* queries, uint32_t here, unsigned long long at,
                                             unsigned long long end, uint32_t& block) {
    using M = Many<DP>;
    const uint32_t lane = threadIdx.x & 31, token = lane / a.block_heads, head = lane - token * a.block_heads;      // of the lane's row in a block
    const bool inside = token < a.block_tokens;
    for (; at < end; at += gridDim.x) {
        const ManyUnit u = many_unit(a, sh, here, at);
        const WeightSeq& s = sh.seq[u.seq];
        const float* lse = a.lse + (size_t)(s.row + token) * a.q_heads + u.head * a.group + head;
        auto minus_at = [&](uint32_t t, uint32_t h) {
            return inside && t + token < u.t1 && h + head < a.group ? -kLog2e * lse[(size_t)t * a.q_heads + h] : -INFINITY;
        };
        float next = u.t0 < u.t1 ? minus_at(u.t0, 0) : 0.0f;
        const bool done = row_blocks(a, u.t0, u.t1, [&](uint32_t t, uint32_t h) {
            const uint32_t stage = block & (kQueryStages - 1);
            const float minus = next;
            const uint32_t h2 = h + a.block_heads < a.group ? h + a.block_heads : 0u, t2 = h2 ? t : t + a.block_tokens;
            if (t2 < u.t1) next = minus_at(t2, h2);                   // one block ahead
            if (block >= kQueryStages && !warp_wait(&sh.q_empty[stage], (block / kQueryStages - 1) & 1, sh)) return false;
            uint8_t* to = queries + stage * M::kRowOperand;
            sh.lse[block & (kLseStages - 1)][lane] = minus;
            if (a.tensor_copies) {
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_expect(&sh.q_full[stage], DP / 64 * 128 * a.block_heads * a.block_tokens);
#pragma unroll
                    for (int i = 0; i < DP / 64; ++i)
                        asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                                         smem_addr(to + i * M::kRowSlab)),
                                     "l"(map), "r"(64 * i), "r"(u.head * a.group + h), "r"(s.row + t), "r"(smem_addr(&sh.q_full[stage]))
                                     : "memory");
                }
            } else {                                                  // a lane has a row
                const bool there = inside && t + token < u.t1 && h + head < a.group;
                const T* q = static_cast<const T*>(a.q) + (there ? (long long)(s.row + t + token) * a.q_token + (long long)(u.head * a.group + h + head) * a.q_head : 0ll);
                for (uint32_t c = 0; c < DP / 8; ++c) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    const unsigned short* e = reinterpret_cast<const unsigned short*>(q) + 8 * c;
                    if (there && 8 * c < a.c.dim)
                        v = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
                    *reinterpret_cast<uint4*>(to + (c >> 3) * M::kRowSlab + lane * 128 + (((c & 7) ^ (lane & 7)) << 4)) = v;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.q_full[stage]);
            }
            ++block;
            return true;
        });
        if (!done) return;
    }
}

// warp 6
template <int DP>
__device__ __forceinline__ void many_codes(const WeightArgs& a, ManyShared& sh, uint8_t* codes, uint32_t here, unsigned long long at, unsigned long long end, uint32_t& units) {
    constexpr uint32_t kPieces = DP / 16, kPass = 32 / kPieces;       // 16-byte pieces of a key; keys of a pass: they divide 16
    const KvView& kv = a.c;
    const uint32_t lane = threadIdx.x & 31, piece = lane % kPieces, r0 = lane / kPieces;
    const bool real = 16 * piece < kv.dim;
    for (; at < end; at += gridDim.x) {
        const ManyUnit u = many_unit(a, sh, here, at);
        if (u.t0 >= u.t1) continue;
        const WeightSeq& s = sh.seq[u.seq];
        const uint32_t low = a.window ? (uint32_t)first_seen((int)s.length - (int)s.count, a.window) : 0u;
        long long from = -1;                                          // of the lane's 16 keys (lanes 0 to 7): bytes from the pool's start
        float ks = -1.0f;
        const uint32_t k = u.k0 + 16 * lane;
        if (lane < 8 && k < s.length && k + 16 > low) {
            const int32_t id = __ldg(kv.pages + (size_t)s.slot * kv.max_pages + (k >> kv.page_shift));
            if ((uint32_t)id < kv.num_pages) {
                from = (long long)id * kv.page_stride + (long long)(k & (kv.page_tokens - 1)) * kv.token_step;
                ks = __ldg(kv.k_scale + (size_t)id * kv.heads + u.head);
            } else {
                kv_flag(kv.status, ROOMIE_FLAG_KV_PAGE);
            }
        }
        if (units && !warp_wait(&sh.codes_empty, (units - 1) & 1, sh)) return;
        ++units;
        if (lane < 8) sh.ks[lane] = ks;
        const uint8_t* pool = kv.k + (long long)u.head * kv.head_step + (real ? 16 * piece : 0);
#pragma unroll 1
        for (uint32_t g = 0; g < 8; ++g) {
            const long long base = __shfl_sync(0xffffffffu, from, g);
            const uint8_t* p = pool + max(base, 0ll) + (long long)r0 * kv.token_step;
            const uint32_t keys = base >= 0 && real ? s.length - (u.k0 + 16 * g) : 0u;       // (a group with a page begins before the end)
#pragma unroll
            for (uint32_t r = 0; r < 16; r += kPass) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(codes + piece_at<DP>(16 * g + r + r0, piece))), "l"(p),
                             "r"(r + r0 < keys ? 16u : 0u) : "memory");
                p += kPass * kv.token_step;
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        mbar_arrive(&sh.codes_full);
    }
}

template <int DP, int kFormat, class T>
__global__ void __launch_bounds__(kManyThreads, Many<DP>::kPerSm) many_weights_kernel(WeightArgs a, const __grid_constant__ CUtensorMap map) {
    using M = Many<DP>;
    extern __shared__ uint8_t raw[];
    __shared__ ManyShared sh;
    uint8_t* queries = raw + ((1024u - (smem_addr(raw) & 1023u)) & 1023u);
    uint8_t* codes = queries + kQueryStages * M::kRowOperand;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(&sh.codes_full, 32);
        mbar_init(&sh.codes_empty, 128);
        mbar_init(&sh.k_full, 128);
        for (int i = 0; i < kQueryStages; ++i) {
            mbar_init(&sh.q_full[i], 1);
            mbar_init(&sh.q_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.s_full[i], 2);
            mbar_init(&sh.s_empty[i], 128);
        }
        mbar_init(&sh.drain, 1);
        sh.failed = 0;
    }
    if (wid == 4) tmem_alloc(&sh.tmem, M::kColumns);
    // rows of a block that hold none stay zero
    for (uint32_t x = threadIdx.x; x < kQueryStages * M::kRowOperand / 16; x += kManyThreads) reinterpret_cast<uint4*>(queries)[x] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    SlotBits slots = {reinterpret_cast<uint32_t*>(codes), M::kCodes / 4};
    bool twice = maybe_twice(a, slots, kManySeqs);
    uint32_t block = 0, units = 0;                                   // of this block, each role in step with the others
    unsigned long long before = 0;                                   // units of the sequences so far
    for (uint32_t base = 0; base < a.num_seqs; base += kManySeqs) {
        const uint32_t here = min(a.num_seqs - base, (uint32_t)kManySeqs);
        __syncthreads();
        unsigned long long mine = 0;
        WeightSeq w = {};
        if (threadIdx.x < here) {
            const KvSeq s = kv_seq(a.c, a.seqs, a.q_offset, a.rows, base + threadIdx.x, blockIdx.x == 0);
            w.slot = s.slot; w.row = s.row; w.count = s.count; w.length = s.length;
            const uint32_t low = a.fresh ? 0u : a.window ? min((uint32_t)first_seen((int)s.length - (int)s.count, a.window), s.length) : 0u;
            w.step0 = low / kManyKeys;
            w.steps = s.count ? (s.length + kManyKeys - 1) / kManyKeys - w.step0 : 0u;
            mine = (unsigned long long)w.steps * a.c.heads;
        }
        if (a.num_seqs > 1 && a.num_seqs <= kManySeqs) twice = __syncthreads_or(threadIdx.x < here && slots.seen((uint32_t)a.seqs[threadIdx.x], a.c.max_seqs)) != 0;
        if (twice && threadIdx.x < here && named_before(a, base + threadIdx.x, blockIdx.x == 0)) mine = w.steps = 0;
        unsigned long long upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += up;
        }
        if (lane == 31) sh.sum[wid] = upto;
        __syncthreads();
        unsigned long long total = 0;
        for (uint32_t x = 0; x < kManyThreads / 32; ++x) {
            if (x < wid) upto += sh.sum[x];
            total += sh.sum[x];
        }
        w.first = upto - mine;
        if (threadIdx.x < here) sh.seq[threadIdx.x] = w;
        __syncthreads();
        // units go round the blocks
        const unsigned long long turn = before % gridDim.x, at = blockIdx.x >= turn ? blockIdx.x - turn : blockIdx.x + gridDim.x - turn;
        before += total;
        if (wid < 4) many_sums<DP, kFormat, T>(a, sh, codes, here, at, total, block, units);
        else if (wid == 4) many_issue<DP, T>(a, sh, queries, here, at, total, block, units);
        else if (wid == 5) many_queries<DP, T>(a, &map, sh, queries, here, at, total, block);
        else many_codes<DP>(a, sh, codes, here, at, total, units);
        __syncwarp();
    }
    if (wid == 4) {
        if (elected()) tc_commit(&sh.drain);                         // whatever was issued has ended before the memory is given back
        __syncwarp();
        mbar_wait_bounded(&sh.drain, 0);
    }
    if (wid == 5 && a.tensor_copies)                                  // nor does a block that gave up end before its copies: the last of each stage
        for (uint32_t b = block > kQueryStages ? block - kQueryStages : 0; b < block; ++b) mbar_wait_bounded(&sh.q_full[b & (kQueryStages - 1)], b / kQueryStages & 1);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0 && sh.failed) kv_flag(a.c.status, ROOMIE_FLAG_WAIT_TIMEOUT);
    if (wid == 4) tmem_free(sh.tmem, M::kColumns);
}

// The queries as (dim, head, token) for tensor copies of 64 elements of a block's heads and tokens.  false: copied by hand.
static bool queries_map(const WeightArgs& a, bool half, CUtensorMap* map) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    const long long most = 1ll << 39;
    if (!encode || !a.q_aligned || (a.q_heads > 1 && (a.q_head <= 0 || a.q_head >= most / 2)) || (a.rows > 1 && (a.q_token <= 0 || a.q_token >= most / 2))) return false;
    // a stride that no step takes still has to be a legal one
    const cuuint64_t dims[3] = {a.c.dim, a.q_heads, a.rows};
    const cuuint64_t strides[2] = {2 * (cuuint64_t)(a.q_heads > 1 ? a.q_head : (long long)a.c.dim), 2 * (cuuint64_t)(a.rows > 1 ? a.q_token : (long long)a.c.dim)};
    const cuuint32_t box[3] = {64, a.block_heads, a.block_tokens}, steps[3] = {1, 1, 1};
    return encode(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DP, int kFormat, class T> static int launch_many_weights(WeightArgs a, cudaStream_t st) {
    CUtensorMap map = {};
    a.tensor_copies = queries_map(a, std::is_same<T, __half>::value, &map);
    return launch("kv_weights", many_weights_kernel<DP, kFormat, T>, dim3((uint32_t)sm_count() * Many<DP>::kPerSm), dim3(kManyThreads), Many<DP>::kSmem, st, false, a, map);
}

template <int DP, int kFormat, class T> static int weight_rows(const WeightArgs& a, bool many, cudaStream_t st) {
    if (many) return launch_many_weights<DP, kFormat, T>(a, st);
    return launch("kv_weights", few_weights_kernel<DP, kFormat, T>, dim3((uint32_t)sm_count() * kWeightBlocks), dim3(kWeightThreads), FewWeights<DP>::kSmem, st, false, a);
}
template <int kFormat, class T> static int weight_dims(const WeightArgs& a, bool many, cudaStream_t st) {
    if (a.c.dim <= 64) return weight_rows<64, kFormat, T>(a, many, st);
    if (a.c.dim <= 128) return weight_rows<128, kFormat, T>(a, many, st);
    return weight_rows<256, kFormat, T>(a, many, st);
}
template <class T> static int weight_format(const WeightArgs& a, bool many, cudaStream_t st) {
    return a.c.format == ROOMIE_KV_E4M3 ? weight_dims<ROOMIE_KV_E4M3, T>(a, many, st) : weight_dims<ROOMIE_KV_INT8, T>(a, many, st);
}

}  // namespace roomie

using namespace roomie;

extern "C" int roomie_kv_weights(const roomie_kv_cache* cache, uint32_t layer, const int32_t* seqs, uint32_t num_seqs, const int32_t* q_offset, uint32_t rows,
                                 uint32_t q_heads, const roomie_rows* q, const float* lse, float scale, uint32_t window, int fresh, float* weight, void* stream) {
    if (kv_check(cache) != ROOMIE_OK || layer >= cache->layers || q_heads == 0 || q_heads % cache->kv_heads || !(scale > 0.0f) || !(scale < INFINITY) ||
        window > 0x7fffffffu)
        return ROOMIE_ERR_INVALID_ARG;
    if (num_seqs == 0 || rows == 0) return ROOMIE_OK;
    if (!rows_valid(q) || q->type == ROOMIE_F32 || !lse || !weight || ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(weight)) & 3u))
        return ROOMIE_ERR_INVALID_ARG;
    if (!seqs || (!q_offset && rows != num_seqs) || num_seqs > 0x3fffffffu || (unsigned long long)rows * q_heads > 0x3fffffffull) return ROOMIE_ERR_INVALID_ARG;
    WeightArgs a = {};
    a.c = kv_view(cache, layer);
    a.seqs = seqs; a.q_offset = q_offset; a.num_seqs = num_seqs; a.rows = rows;
    a.q_heads = q_heads; a.group = q_heads / cache->kv_heads;
    a.block_heads = a.group < kManyRows ? a.group : kManyRows;
    a.block_tokens = kManyRows / a.block_heads;
    a.q = q->data; a.q_token = q->token_stride; a.q_head = q->head_stride;
    a.lse = lse;
    a.max_tokens = cache->max_pages * cache->page_tokens;
    if ((unsigned long long)cache->kv_heads * (a.max_tokens / kManyKeys + 1) > 0xffffffffull) return ROOMIE_ERR_INVALID_ARG;
    a.weight = weight + (size_t)layer * cache->max_seqs * cache->kv_heads * a.max_tokens;
    a.window = window;
    a.scale_log2 = scale * kLog2e;
    a.q_aligned = rows_aligned16(*q, rows, q_heads);
    a.fresh = fresh != 0;
    // Which kernel, by the rows a sequence and key head (of a mixed call: their average).  32 query heads on 8, sequences of up to 4096 keys, 16 of them
    // and 2 of them, us:
    //   rows                  4        8         16        24        32       64
    //   products by warps     16.1 8.0 18.3 10.3 26.6 15.6 88.8 21.6 110 25.6 209 45.9     (16 in one pass)
    //   on tensor memory                         25.2 9.7  25.2 9.6  23.4 9.4 27.9 10.3
    const bool many = (unsigned long long)rows * a.group > 8ull * num_seqs;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return q->type == ROOMIE_F16 ? weight_format<__half>(a, many, st) : weight_format<__nv_bfloat16>(a, many, st);
}
