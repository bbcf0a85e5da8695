// Attention over the paged 8-bit cache.
//
// o_i = sum_j p_ij * vs[page(j)] * v_j / sum_j p_ij,  p_ij = exp(scale * ks[page(j)] * q_i.k_j - max)  over the keys j that row i sees.
#include "roomie_kv_attention.cuh"

namespace roomie {

constexpr int kAttnWarps = 4, kAttnThreads = 32 * kAttnWarps;
constexpr int kJoin = 32;                                        // parts that one block adds up: a lane each (and at most 32 such groups)

// The flat order of the call's work: sequence, key head, row tile, key block.  What one sequence contributes:
struct SeqWork {
    KvSeq s;
    uint32_t first_block, blocks, tiles;     // key blocks [first_block, first_block + blocks), row tiles
};
constexpr uint32_t kWhole = 3, kMostEqual = 12; // units: see few_rows_kernel
__device__ __forceinline__ uint32_t parts_of(uint32_t blocks, uint32_t most) { return blocks <= kWhole ? 1u : (blocks + most - 1) / most; }
template <int kBlock, int kRows>
__device__ __forceinline__ SeqWork seq_work(const AttnArgs& a, uint32_t i, bool report) {
    SeqWork w;
    w.s = kv_seq(a.c, a.seqs, a.q_offset, a.rows, i, report);
    w.tiles = (w.s.count * a.group + kRows - 1) / kRows;
    const int start = (int)w.s.length - (int)w.s.count;                  // negative: leading rows that see nothing
    const int lowest = a.window ? first_seen(start, a.window) : 0;        // first key that some row may see
    w.first_block = (uint32_t)max(min(lowest, (int)w.s.length), 0) / kBlock;
    const uint32_t end = (w.s.length + kBlock - 1) / kBlock;
    w.blocks = max(end > w.first_block ? end - w.first_block : 0u, 1u);  // a sequence without keys still writes its rows
    return w;
}

// ---------------------------------------------------------------------------------------------------------------------------
// Few rows a key head (a decoding step: `group` rows for each new token).  Bound by the bytes of the codes.  The products are taken
// transposed (S^T = K q^T, o^T = V^T p^T), so that keys and values are the 16-row operand and the 8 rows of a GQA group fill the 8-wide
// one.  The contraction index of a matrix product may be permuted freely, and so may the rows of its result: a lane takes 4 bytes of its
// own contiguous span of a key for each k-step (lane quarter c of a token holds dims [c*DP/4, +DP/4)), and of a value row the dims
// [r*DP/8, +DP/8) for its result rows r: both are whole 16-byte reads of the codes as they are stored.
//
// Every warp works for itself: it has kStages steps of keys and values under way to its own part of shared memory by asynchronous
// copies (64 sequences of up to 16384 tokens in int8, 1.31 GB: 247 to 264 us from run to run, 5300 to 4960 GB/s; with one step ahead in
// registers 297).  A block walks a contiguous part of the flat order; its warps take the
// 16*kGroups-key steps in turn and meet at each (sequence, head, tile).  A part that does not hold all of a (sequence, head, tile)
// leaves its sums in the workspace, and the last part to arrive adds them in order.
//
// Scales: a page's key scale goes into the factor of the exponent's argument, its value scale vs into the exponent: the weights
// exp2(s + log2 vs - m), m near the maximum of s + log2 vs, multiply the codes, and the softmax total sums them times 1 / vs
// (or is summed apart: see kNear).
template <int DP, int NT, int kFormat, class T>
struct FewRows {
    static constexpr int kGroups = DP > 128 ? 1 : 2;               // 16-key groups a warp step
    static constexpr int kStep = 16 * kGroups;
    static constexpr int kBlock = kStep * kAttnWarps;              // keys of a flat unit
    static constexpr int kRows = 8 * NT;
    static constexpr int KS = DP / 16;
    static constexpr int KW = DP / 16;                             // words of a lane's key span
    static constexpr int VW = DP / 32;                             // words of a lane's value span
    static constexpr int kPartial = kRows * (DP + 2);              // floats of one partial result, a multiple of 4
    static constexpr int kSide = kStep * DP;                       // bytes of a step's keys
    static constexpr int kStages = 16384 / (2 * kSide);            // 16 KB a warp: 2 steps, 4 for the smallest heads
    static constexpr int kRing = kStages * 2 * kSide;
    static constexpr int kMeet = kAttnWarps * kRows * (DP + 2) * (int)sizeof(float);
    static constexpr int kSmem = kRing * kAttnWarps > kMeet ? kRing * kAttnWarps : kMeet;
};

template <class T> __device__ __forceinline__ float load_elem(const T* p) { return to_f32(*p); }

template <int DP, int NT, int kFormat, class T>
__global__ void __launch_bounds__(kAttnThreads, DP > 128 || NT > 1 ? 2 : 3) few_rows_kernel(AttnArgs a) {
    using F = FewRows<DP, NT, kFormat, T>;
    constexpr int G = F::kGroups, KW = F::KW, VW = F::VW, KS = F::KS, kStages = F::kStages;
    extern __shared__ __align__(1024) float sm[];                  // the warps' steps; then [warps][rows][DP] sums, [warps][rows][2] max and total
    __shared__ unsigned long long sh_sum[kAttnWarps], sh_first;
    __shared__ uint32_t sh_at[4];
    __shared__ float sm_row[2 * F::kRows];
    __shared__ float sh_ref[2 * NT][kAttnThreads];                 // reference of a row's total while it is summed apart
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const KvView& kv = a.c;

    // ---- where this block's part begins: a scan of the sequences' units, kept from the first pass when they are at most a block's
    // threads
    auto scan = [&](unsigned long long x, unsigned long long& all) {      // exclusive over the block
        unsigned long long upto = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned long long up = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += up;
        }
        __syncthreads();
        if (lane == 31) sh_sum[wid] = upto;
        __syncthreads();
        all = 0;
        for (int w = 0; w < kAttnWarps; ++w) {
            if (w < wid) upto += sh_sum[w];
            all += sh_sum[w];
        }
        return upto - x;
    };
    unsigned long long mine = 0, own = 0, total;
    SeqWork own_work = {};
    for (uint32_t i = threadIdx.x; i < a.num_seqs; i += kAttnThreads) {
        own_work = seq_work<F::kBlock, F::kRows>(a, i, blockIdx.x == 0);
        own = (unsigned long long)own_work.tiles * own_work.blocks * kv.heads;
        mine += own;
    }
    const unsigned long long own_first = scan(mine, total);
    if (total == 0) return;
    // Work of few units a block is not cut at any unit but into equal parts of each item, items of up to kWhole units not at all, when
    // that makes no more parts than blocks: fewer items then need joining.  Device times, us, equal parts where they fit and any cut (32
    // query heads on 8, 128 dims, page 64; units a block by `most`):
    //   sequences x keys   3 x 300    2 x 8192   16 x 4096  4 x 16384  | 64 x 2048  2 x 65536  64 x 4096  2 x 131072
    //   units a block      1          2          7          7          | 14         14         28         28
    //                      10.9 11.2  20.1 26.7  31.8 35.9  37.7 43.6  | 56.0 55.1  50.6 55.2  82.1 80.6  79.4 84.6
    // Above kMostEqual units many items lose by it and few gain.
    uint32_t most = (uint32_t)min(total / gridDim.x + 1, 1ull << 30), own_parts = 0;
    unsigned long long own_first_part = 0, parts = total < gridDim.x ? total : gridDim.x;
    bool equal = a.num_seqs <= kAttnThreads && most <= kMostEqual;
    if (equal) {                                                   // parts of at most `most`, most + 1 and most + 2 units: 21 bits each
        unsigned long long three = 0, all_three;
        if (own)                                                   // at most `own` each, which is below 2^20 here
            for (uint32_t e = 0; e < 3; ++e)
                three |= (unsigned long long)(own_work.tiles * kv.heads * parts_of(own_work.blocks, most + e)) << (21 * e);
        unsigned long long first_three = scan(three, all_three);
        equal = false;
        for (uint32_t e = 0; e < 3 && !equal; ++e, three >>= 21, first_three >>= 21, all_three >>= 21)
            if ((all_three & 0x1fffff) <= gridDim.x) {
                equal = true;
                own_parts = (uint32_t)(three & 0x1fffff);
                own_first_part = first_three & 0x1fffff;
                parts = all_three & 0x1fffff;
                most += e;
            }
    }
    if (blockIdx.x >= parts) return;
    unsigned long long at = equal ? 0 : total * blockIdx.x / parts;
    const unsigned long long end = equal ? 1 : total * (blockIdx.x + 1) / parts;

    // the sequence that holds `at`, and the flat index it begins at
    if (equal) {                                                   // seq_first: the first part of the sequence
        if (own_parts && blockIdx.x >= own_first_part && blockIdx.x < own_first_part + own_parts) {
            sh_at[0] = threadIdx.x;
            sh_first = own_first_part;
        }
    } else if (a.num_seqs <= kAttnThreads) {
        if (own && at >= own_first && at < own_first + own) {
            sh_at[0] = threadIdx.x;
            sh_first = own_first;
        }
    } else {
        unsigned long long before = 0;
        for (uint32_t base = 0; base < a.num_seqs; base += kAttnThreads) {
            const uint32_t i = base + threadIdx.x;
            unsigned long long n = 0;
            if (i < a.num_seqs) {
                const SeqWork w = seq_work<F::kBlock, F::kRows>(a, i, false);
                n = (unsigned long long)w.tiles * w.blocks * kv.heads;
            }
            unsigned long long all;
            const unsigned long long first = before + scan(n, all);
            if (n && at >= first && at < first + n) {
                sh_at[0] = i;
                sh_first = first;
            }
            before += all;
            if (at < before) break;
        }
    }
    __syncthreads();
    uint32_t seq = sh_at[0];
    unsigned long long seq_first = sh_first;

    while (at < end) {
        SeqWork w = seq_work<F::kBlock, F::kRows>(a, seq, false);
        uint32_t head, tile, b0, b1, first_part, last_part;        // the blocks that share the item
        if (equal) {
            const uint32_t cuts = parts_of(w.blocks, most), rest = blockIdx.x - (uint32_t)seq_first, which = rest / cuts, j = rest - which * cuts;
            head = which / w.tiles;
            tile = which - head * w.tiles;
            b0 = (uint32_t)((unsigned long long)w.blocks * j / cuts);
            b1 = (uint32_t)((unsigned long long)w.blocks * (j + 1) / cuts);
            first_part = blockIdx.x - j;
            last_part = first_part + cuts - 1;
        } else {
            unsigned long long n = (unsigned long long)w.tiles * w.blocks * kv.heads;
            while (at >= seq_first + n) {                          // sequences without rows contribute nothing
                seq_first += n;
                if (++seq >= a.num_seqs) return;                   // lengths changed under the call
                w = seq_work<F::kBlock, F::kRows>(a, seq, false);
                n = (unsigned long long)w.tiles * w.blocks * kv.heads;
            }
            const unsigned long long inside = at - seq_first;
            head = (uint32_t)(inside / ((unsigned long long)w.tiles * w.blocks));
            const uint32_t rest = (uint32_t)(inside - (unsigned long long)head * w.tiles * w.blocks);
            tile = rest / w.blocks;
            b0 = rest - tile * w.blocks;
            b1 = (uint32_t)min((unsigned long long)w.blocks, (unsigned long long)b0 + (end - at));
            const unsigned long long item = at - b0;               // consecutive blocks: from that of its first unit to that of its last
            first_part = (uint32_t)(((item + 1) * parts - 1) / total);
            last_part = (uint32_t)(((item + w.blocks) * parts - 1) / total);
        }
        const KvSeq& s = w.s;
        const int start = (int)s.length - (int)s.count;
        const uint32_t rows = s.count * a.group - tile * F::kRows;  // of this tile: min(rows, kRows)

        // ---- which keys the rows see; rows 2c and 2c+1 of each eight are the lane's result columns -------------------------
        int see_hi[NT][2], see_lo[NT][2];                          // row n sees keys [lo, hi)
        int tile_hi = 0, tile_lo = 0x7fffffff, all_hi = 0x7fffffff, all_lo = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const uint32_t rc = t * 8 + 2 * c + n;
                const int pos = start + (int)((tile * F::kRows + rc) / a.group);
                int hi = rc < rows ? max(min(pos + 1, (int)s.length), 0) : 0;
                int lo = a.window ? first_seen(pos, a.window) : 0;
                if (lo > hi) lo = hi;
                see_hi[t][n] = hi;
                see_lo[t][n] = lo;
                tile_hi = max(tile_hi, hi);
                if (rc < rows) {
                    if (hi > lo) tile_lo = min(tile_lo, lo);
                    all_hi = min(all_hi, hi);
                    all_lo = max(all_lo, lo);
                }
            }
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            tile_hi = max(tile_hi, __shfl_xor_sync(0xffffffffu, tile_hi, d));
            tile_lo = min(tile_lo, __shfl_xor_sync(0xffffffffu, tile_lo, d));
            all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, d));
            all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, d));
        }

        float o[NT][KS][4];
        float m[NT][2], l[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][i][e] = 0.0f;
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.0f;
        }
        bool apart = false;                                        // the totals are; the same in all lanes

        // the warp's steps: keys [k0, k0 + kStep) of this tile's blocks that some row sees
        const int part_lo = (int)((w.first_block + b0) * F::kBlock), part_hi = (int)min((w.first_block + b1) * F::kBlock, s.length);
        int lo_key = max(part_lo, tile_lo / F::kStep * F::kStep), hi_key = min(part_hi, tile_hi);
        if (lo_key >= hi_key) lo_key = hi_key = 0;
        const int32_t* table = kv.pages + (size_t)s.slot * kv.max_pages;
        const uint32_t row_step = kv.token_step;
        const long long head_off = (long long)head * kv.head_step;

        uint8_t* ring = reinterpret_cast<uint8_t*>(sm) + wid * F::kRing;
        constexpr int kChunks = DP / 16, kLoads = F::kStep * kChunks / 32;     // 16-byte copies a lane and side
        const uint32_t chunk = lane % kChunks, row0 = lane / kChunks;          // copy i: row row0 + i * (32 / kChunks)
        constexpr int kRowsPer = 32 / kChunks;
        const bool real = 16 * chunk < kv.dim;
        const long long to_v = kv.v - kv.k;
        int32_t page[G];                                           // of the step that is copied next
        auto get_pages = [&](int k0) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int k = k0 + 16 * g;
                int32_t id = -1;
                if (k < hi_key && k + 16 > tile_lo) {
                    id = __ldg(table + (k >> kv.page_shift));
                    if ((uint32_t)id >= kv.num_pages) {
                        if (lane == 0) kv_flag(kv.status, ROOMIE_FLAG_KV_PAGE);
                        id = -1;
                    }
                }
                page[g] = id;
            }
        };
        // the scales of a step are fetched with its copies and wait in registers: (key scale, value scale) of stage x, group g
        float ks_of[kStages][G], vs_of[kStages][G];
        auto copy_step = [&](int k0, int stage) {
            const uint32_t to = smem_addr(ring + stage * 2 * F::kSide);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int k = k0 + 16 * g;
                const uint8_t* p = kv.k + (long long)max(page[g], 0) * kv.page_stride + head_off +
                                   ((k & (kv.page_tokens - 1)) + row0) * row_step + 16 * chunk;
#pragma unroll
                for (int i = 0; i < kLoads / G; ++i) {
                    const uint32_t row = 16 * g + row0 + i * kRowsPer;
                    const int key = k0 + (int)row;
                    const uint32_t n = page[g] >= 0 && real && key < hi_key && key >= tile_lo ? 16u : 0u;   // the rest becomes zeros
                    const uint32_t at = to + code_at<DP>(row, chunk);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(p), "r"(n) : "memory");
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + F::kSide), "l"(p + to_v), "r"(n) : "memory");
                    p += kRowsPer * row_step;
                }
            }
        };
        auto get_scales = [&](int stage) {
#pragma unroll
            for (int s2 = 0; s2 < kStages; ++s2)
                if (s2 == stage)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        ks_of[s2][g] = 0.0f;
                        vs_of[s2][g] = -1.0f;                      // no page
                        if (page[g] >= 0) {
                            ks_of[s2][g] = __ldg(kv.k_scale + (size_t)page[g] * kv.heads + head);
                            vs_of[s2][g] = __ldg(kv.v_scale + (size_t)page[g] * kv.heads + head);
                        }
                    }
        };
        int k0 = lo_key + ((wid - lo_key / F::kStep) & (kAttnWarps - 1)) * F::kStep;   // warp w takes steps w mod 4
        get_pages(k0);
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            copy_step(k0 + i * F::kBlock, i);
            get_scales(i);
            asm volatile("cp.async.commit_group;" ::: "memory");
            get_pages(k0 + (i + 1) * F::kBlock);
        }
        // ---- queries, while the first copies are on their way: operand b of S^T; row r of the tile, dims as the lane's keys ----
        uint32_t qf[NT][KS][2];
        float qscale[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t rr = t * 8 + r;
            const bool on = rr < rows;
            const uint32_t row = tile * F::kRows + rr, tok = row / a.group;
            const T* q = static_cast<const T*>(a.q) + (long long)(s.row + tok) * a.q_token +
                         (long long)(head * a.group + row - tok * a.group) * a.q_head + c * (DP / 4);
            float x[DP / 4];
            float amax = 0.0f;
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
                        if (c * (DP / 4) + d < kv.dim) x[d] = load_elem(q + d);
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
                qf[t][i][0] = reinterpret_cast<const uint32_t&>(lo);
                qf[t][i][1] = reinterpret_cast<const uint32_t&>(hi);
            }
            const float up = pow2f(e) * a.scale_log2;
#pragma unroll
            for (int n = 0; n < 2; ++n) qscale[t][n] = __shfl_sync(0xffffffffu, up, (2 * c + n) * 4);
        }

        while (k0 < hi_key) {
#pragma unroll
            for (int stage = 0; stage < kStages; ++stage) {
                if (k0 >= hi_key) break;
                asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
                __syncwarp();
                const uint8_t* side = ring + stage * 2 * F::kSide;
                float sc[G][NT][4], ivs[G];
                bool whole = k0 >= all_lo && k0 + F::kStep <= all_hi, high = apart, wide = false;
#pragma unroll
                for (int g = 0; g < G; ++g) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[g][t][e] = 0.0f;
                    uint32_t kr[2][KW];
                    read_span<DP, KW>(kr[0], side, 16 * g + r, c * (DP / 4));
                    read_span<DP, KW>(kr[1], side, 16 * g + r + 8, c * (DP / 4));
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        uint32_t a0, a1, a2, a3;
                        codes_to_f16<kFormat>(kr[0][i], a0, a2);
                        codes_to_f16<kFormat>(kr[1][i], a1, a3);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma16816(sc[g][t], a0, a1, a2, a3, qf[t][i][0], qf[t][i][1]);
                    }
                }
                // exponents: sc[e] is key r + 8*(e >> 1) of the group, row 2c + (e & 1)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const float ks = ks_of[stage][g];
                    float vs = vs_of[stage][g], lvs = -INFINITY;   // a page that is not there weighs nothing
                    ivs[g] = 0.0f;
                    if (vs >= 0.0f) {
                        vs = fmaxf(vs, kLeastScale);
                        lvs = log2_fast(vs);
                        ivs[g] = __fdividef(1.0f, vs);
                        wide = wide || fabsf(lvs) > kNear;
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            const float f = qscale[t][n] * ks;
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float& x = sc[g][t][2 * h + n];
                                x = fmaf(x, f, lvs);
                                if (!whole) {
                                    const int k = k0 + 16 * g + 8 * h + r;
                                    if (k >= see_hi[t][n] || k < see_lo[t][n]) x = -INFINITY;
                                }
                                high = high || x > m[t][n] + kAbove;
                            }
                        }
                }
                // The maximum is looked for only when some exponent is more than kAbove over the reference m, or the totals are summed apart.
                if (__any_sync(0xffffffffu, high || wide)) {
                    if (wide && !apart) {
                        apart = true;
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int n = 0; n < 2; ++n) sh_ref[2 * t + n][threadIdx.x] = m[t][n];
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int n = 0; n < 2; ++n) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int g = 0; g < G; ++g) mx = fmaxf(mx, fmaxf(sc[g][t][n], sc[g][t][n + 2]));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                            mx = fmaxf(mx - kBelow, m[t][n]);
                            const float f = m[t][n] == -INFINITY ? 0.0f : exp2_fast(m[t][n] - mx);
                            m[t][n] = mx;
                            if (!apart) l[t][n] *= f;
#pragma unroll
                            for (int i = 0; i < KS; ++i) {
                                o[t][i][n] *= f;
                                o[t][i][n + 2] *= f;
                            }
                        }
                    if (apart) {
                        float less[G];                                 // log2 vs
#pragma unroll
                        for (int g = 0; g < G; ++g) {
                            less[g] = vs_of[stage][g] >= 0.0f ? log2_fast(fmaxf(vs_of[stage][g], kLeastScale)) : 0.0f;
                            ivs[g] = 0.0f;
                        }
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int n = 0; n < 2; ++n) {
                                float ref = sh_ref[2 * t + n][threadIdx.x], mx = -INFINITY;
#pragma unroll
                                for (int g = 0; g < G; ++g) mx = fmaxf(mx, fmaxf(sc[g][t][n], sc[g][t][n + 2]) - less[g]);
                                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                                if (mx > ref + kAbove) {
                                    if (ref != -INFINITY) l[t][n] *= exp2_fast(ref - (mx - kBelow));
                                    ref = mx - kBelow;
                                    sh_ref[2 * t + n][threadIdx.x] = ref;
                                }
                                if (ref == -INFINITY) ref = 0.0f;
#pragma unroll
                                for (int g = 0; g < G; ++g) l[t][n] += exp2_fast(sc[g][t][n] - less[g] - ref) + exp2_fast(sc[g][t][n + 2] - less[g] - ref);
                            }
                    }
                }
                // weights: rounded to float16 (11 bits) for the product with the codes, not for the total
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    uint32_t pb[NT][2];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const float m0 = m[t][0] == -INFINITY ? 0.0f : m[t][0], m1 = m[t][1] == -INFINITY ? 0.0f : m[t][1];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float p0 = exp2_fast(sc[g][t][2 * h] - m0), p1 = exp2_fast(sc[g][t][2 * h + 1] - m1);
                            l[t][0] = fmaf(p0, ivs[g], l[t][0]);
                            l[t][1] = fmaf(p1, ivs[g], l[t][1]);
                            const __half2 x = __floats2half2_rn(p0, p1);
                            pb[t][h] = transpose8x8(reinterpret_cast<const uint32_t&>(x));
                        }
                    }
                    uint32_t vr[4][VW];
#pragma unroll
                    for (int h = 0; h < 4; ++h) read_span<DP, VW>(vr[h], side + F::kSide, 16 * g + 2 * c + (h & 1) + 8 * (h >> 1), r * (DP / 8));
#pragma unroll
                    for (int j = 0; j < VW; ++j) {
                        uint32_t a0[4], a1[4];                     // [result-row pair of the word's four dims]
                        codes_to_f16<kFormat>(__byte_perm(vr[0][j], vr[1][j], 0x5140), a0[0], a0[1]);
                        codes_to_f16<kFormat>(__byte_perm(vr[0][j], vr[1][j], 0x7362), a0[2], a0[3]);
                        codes_to_f16<kFormat>(__byte_perm(vr[2][j], vr[3][j], 0x5140), a1[0], a1[1]);
                        codes_to_f16<kFormat>(__byte_perm(vr[2][j], vr[3][j], 0x7362), a1[2], a1[3]);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            mma16816(o[t][2 * j], a0[0], a0[1], a1[0], a1[1], pb[t][0], pb[t][1]);
                            mma16816(o[t][2 * j + 1], a0[2], a0[3], a1[2], a1[3], pb[t][0], pb[t][1]);
                        }
                    }
                }
                __syncwarp();                                      // the stage has been read
                copy_step(k0 + kStages * F::kBlock, stage);
                get_scales(stage);
                asm volatile("cp.async.commit_group;" ::: "memory");
                k0 += F::kBlock;
                get_pages(k0 + kStages * F::kBlock);
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");

        // ---- the warps meet --------------------------------------------------------------------------------------------
        float* sm_ml = sm + kAttnWarps * F::kRows * DP;
        if (apart) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    float up;
                    one_reference(m[t][n], l[t][n], up, sh_ref[2 * t + n][threadIdx.x]);
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        o[t][i][n] *= up;
                        o[t][i][n + 2] *= up;
                    }
                }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[t][n] += __shfl_xor_sync(0xffffffffu, l[t][n], d);
                const int row = t * 8 + 2 * c + n;
                if (r == 0) {
                    sm_ml[(wid * F::kRows + row) * 2] = m[t][n];
                    sm_ml[(wid * F::kRows + row) * 2 + 1] = l[t][n];
                }
                float* to = sm + (size_t)(wid * F::kRows + row) * DP + r * (DP / 8);
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    to[2 * i] = o[t][i][n];
                    to[2 * i + 1] = o[t][i][n + 2];
                }
            }
        __syncthreads();

        const bool complete = b0 == 0 && b1 == w.blocks;
        const uint32_t n_rows = min(rows, (uint32_t)F::kRows);
        auto put = [&](uint32_t row, uint32_t d, float mx, float sum, float value) {
            const uint32_t rr = tile * F::kRows + row, tok = rr / a.group, h = head * a.group + rr - tok * a.group;
            if (d < kv.dim)
                (static_cast<T*>(a.out) + (long long)(s.row + tok) * a.o_token + (long long)h * a.o_head)[d] =
                    from_f32<T>(sum > 0.0f ? value / sum : sum == 0.0f ? 0.0f : sum);
            if (a.lse && d == 0) a.lse[(size_t)(s.row + tok) * a.q_heads + h] = sum > 0.0f ? (mx + log2f(sum)) * kLn2 : sum == 0.0f ? -INFINITY : sum;
        };
        float* part = a.partial + ((size_t)blockIdx.x * 2 + (b0 == 0 ? 1 : 0)) * F::kPartial;
        for (uint32_t x = threadIdx.x; x < n_rows * DP; x += kAttnThreads) {
            const uint32_t row = x / DP, d = x - row * DP;
            float mx = -INFINITY;
#pragma unroll
            for (int v = 0; v < kAttnWarps; ++v) mx = fmaxf(mx, sm_ml[(v * F::kRows + row) * 2]);
            float sum = 0.0f, value = 0.0f;
#pragma unroll
            for (int v = 0; v < kAttnWarps; ++v) {
                const float mv = sm_ml[(v * F::kRows + row) * 2];
                const float f = mv == -INFINITY ? 0.0f : exp2f(mv - mx);
                sum += f * sm_ml[(v * F::kRows + row) * 2 + 1];
                value += f * sm[(size_t)(v * F::kRows + row) * DP + d];
            }
            if (complete) {
                put(row, d, mx, sum, value);
            } else {
                part[row * DP + d] = value;
                if (d == 0) {
                    part[F::kRows * DP + 2 * row] = mx;
                    part[F::kRows * DP + 2 * row + 1] = sum;
                }
            }
        }
        if (!complete) {
            // With many parts the last to arrive of each kJoin adds those up, and the last of these the sums: one block alone took 60 us
            // over 444 parts.
            const uint32_t first = first_part, last = last_part;
            const uint32_t count = last - first + 1, groups = (count + kJoin - 1) / kJoin;
            auto part_of = [&](uint32_t b) { return a.partial + ((size_t)(first + b) * 2 + (b == 0 ? 1 : 0)) * F::kPartial; };
            auto arrive = [&](uint32_t* counter, uint32_t n) {     // whether this block is the last of n
                __syncthreads();
                if (threadIdx.x == 0) sh_at[1] = count_part(counter, n) == n - 1;
                __syncthreads();
                return sh_at[1] != 0;
            };
            // parts b0, b0 + step, ...: n of them, to the results (or into the first)
            auto join = [&](uint32_t b0, uint32_t step, uint32_t n, bool end) {
                float* factor = sm;                                // [n][rows]
                for (uint32_t row = wid; row < n_rows; row += kAttnWarps) {
                    float2 ml = make_float2(-INFINITY, 0.0f);      // a lane for each part: n <= 32
                    if (lane < (int)n) ml = __ldcg(reinterpret_cast<const float2*>(part_of(b0 + lane * step) + F::kRows * DP + 2 * row));
                    float mx = ml.x;
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    const float f = ml.x == -INFINITY ? 0.0f : exp2f(ml.x - mx);
                    if (lane < (int)n) factor[lane * F::kRows + row] = f;
                    float sum = f * ml.y;
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    if (lane == 0) {
                        sm_row[2 * row] = mx;
                        sm_row[2 * row + 1] = sum;
                    }
                }
                __syncthreads();
                float* to = part_of(b0);
                for (uint32_t x = threadIdx.x; x < n_rows * (DP / 4); x += kAttnThreads) {
                    const uint32_t row = x / (DP / 4), d = 4 * (x - row * (DP / 4));
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
                    for (uint32_t b = 0; b < n; ++b) {             // many loads under way
                        const float4 y = __ldcg(reinterpret_cast<const float4*>(part_of(b0 + b * step) + row * DP + d));
                        const float f = factor[b * F::kRows + row];
                        v.x += f * y.x; v.y += f * y.y; v.z += f * y.z; v.w += f * y.w;
                    }
                    const float mx = sm_row[2 * row], sum = sm_row[2 * row + 1];
                    if (end) {
                        put(row, d, mx, sum, v.x);
                        put(row, d + 1, mx, sum, v.y);
                        put(row, d + 2, mx, sum, v.z);
                        put(row, d + 3, mx, sum, v.w);
                    } else {
                        *reinterpret_cast<float4*>(to + row * DP + d) = v;
                        if (d == 0) *reinterpret_cast<float2*>(to + F::kRows * DP + 2 * row) = make_float2(mx, sum);
                    }
                }
            };
            const uint32_t group = (blockIdx.x - first) / kJoin, in_group = min((uint32_t)kJoin, count - group * kJoin);
            bool go = true;
            if (groups > 1 && in_group > 1) {                      // (a group of one needs no counter, and the next item may have it)
                go = arrive(a.counters + gridDim.x + first + group * kJoin, in_group);
                if (go) join(group * kJoin, 1, in_group, false);
            }
            if (go && arrive(a.counters + first, groups > 1 ? groups : count)) join(0, groups > 1 ? kJoin : 1, groups > 1 ? groups : count, true);
        }
        __syncthreads();
        at += equal ? 1 : b1 - b0;
    }
}

size_t kv_attention_bytes(const roomie_kv_cache* c) {
    const uint32_t dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
    const size_t blocks = (size_t)sm_count() * kMaxAttnBlocksPerSm;
    const size_t few = blocks * 2 * (16 * (size_t)(dp + 2)) * sizeof(float), many = prompt_partial_bytes(c->head_dim);
    static_assert(2 * 512 * kMaxAttnBlocksPerSm * sizeof(uint32_t) <= ROOMIE_KV_WORKSPACE_ZEROED, "counters of up to 512 SMs");
    const size_t bytes = 2 * blocks * sizeof(uint32_t) + 256 + (few > many ? few : many);
    return (bytes + 255) / 256 * 256;
}

template <int DP, int NT, int kFormat, class T>
static int launch_few(const AttnArgs& a, cudaStream_t st) {
    using F = FewRows<DP, NT, kFormat, T>;
    const uint32_t per_sm = DP > 128 || NT > 1 ? 2 : 3;
    return launch("kv_attention", few_rows_kernel<DP, NT, kFormat, T>, dim3((uint32_t)sm_count() * per_sm), dim3(kAttnThreads),
                  F::kSmem, st, false, a);
}
template <int DP, int kFormat, class T>
static int launch_rows(const AttnArgs& a, bool eight, cudaStream_t st) {
    return eight ? launch_few<DP, 1, kFormat, T>(a, st) : launch_few<DP, 2, kFormat, T>(a, st);
}
template <int kFormat, class T>
static int launch_dim(const AttnArgs& a, bool eight, cudaStream_t st) {
    if (a.c.dim <= 64) return launch_rows<64, kFormat, T>(a, eight, st);
    if (a.c.dim <= 128) return launch_rows<128, kFormat, T>(a, eight, st);
    return launch_rows<256, kFormat, T>(a, eight, st);
}
template <class T>
static int launch_format(const AttnArgs& a, bool eight, cudaStream_t st) {
    return a.c.format == ROOMIE_KV_E4M3 ? launch_dim<ROOMIE_KV_E4M3, T>(a, eight, st) : launch_dim<ROOMIE_KV_INT8, T>(a, eight, st);
}

}  // namespace roomie

using namespace roomie;

extern "C" int roomie_kv_attention(const roomie_kv_cache* cache, uint32_t layer, const int32_t* seqs, uint32_t num_seqs,
                                   const int32_t* q_offset, uint32_t rows, uint32_t q_heads, const roomie_rows* q, float scale,
                                   uint32_t window, const roomie_rows* out, float* lse, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    if (kv_check(cache) != ROOMIE_OK || layer >= cache->layers || q_heads == 0 || q_heads % cache->kv_heads || !(scale > 0.0f) ||
        !(scale < INFINITY) || window > 0x7fffffffu)
        return ROOMIE_ERR_INVALID_ARG;
    if (num_seqs == 0 || rows == 0) return ROOMIE_OK;
    if (!rows_valid(q) || !rows_valid(out) || q->type != out->type || q->type == ROOMIE_F32 || !rows_apart(*out, rows, q_heads, cache->head_dim))
        return ROOMIE_ERR_INVALID_ARG;
    if (!seqs || (!q_offset && rows != num_seqs) || num_seqs > 0x3fffffffu || (unsigned long long)rows * q_heads > 0x3fffffffull)
        return ROOMIE_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ROOMIE_ERR_INVALID_ARG;
    if (workspace_bytes < roomie_kv_workspace_bytes(cache)) return ROOMIE_ERR_CAPACITY;
    AttnArgs a = {};
    a.c = kv_view(cache, layer);
    a.seqs = seqs; a.q_offset = q_offset; a.num_seqs = num_seqs; a.rows = rows;
    a.q_heads = q_heads; a.group = q_heads / cache->kv_heads;
    a.group_inverse = a.group > 1 ? ~0ull / a.group + 1 : 0;
    a.q = q->data; a.out = out->data; a.lse = lse;
    a.q_token = q->token_stride; a.q_head = q->head_stride; a.o_token = out->token_stride; a.o_head = out->head_stride;
    a.scale_log2 = scale * 1.44269504088896340736f;
    a.window = window;
    a.q_aligned = rows_aligned16(*q, rows, q_heads);
    a.o_aligned = rows_aligned16(*out, rows, q_heads);
    a.counters = static_cast<uint32_t*>(workspace);
    const size_t blocks = (size_t)sm_count() * kMaxAttnBlocksPerSm;
    a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + (2 * blocks * sizeof(uint32_t) + 255) / 256 * 256);
    // Which kernel, and how many rows a tile.  Measured on calls whose sequences bring alike; one that mixes single tokens with a chunk goes by
    // its average.  Rows a sequence and key head (32 query heads on 8, sequences of up to 4096 keys, 16 of them and 2 of them, us):
    //   rows        8       16      24      32      64
    //   8 a tile    36 23   57 29   57 33   82 32   117 37
    //   16 a tile   36 23   52 33   61 33   84 39   106 42
    //   prompt      82 47   82 48   83 48   83 44   82 44
    const bool eight = (unsigned long long)rows * a.group <= 8ull * num_seqs;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if ((unsigned long long)rows * a.group > 32ull * num_seqs) return launch_prompt(a, q->type == ROOMIE_F16, st);
    return q->type == ROOMIE_F16 ? launch_format<__half>(a, eight, st) : launch_format<__nv_bfloat16>(a, eight, st);
}
