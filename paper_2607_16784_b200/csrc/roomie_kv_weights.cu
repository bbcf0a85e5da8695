// The attention weight that cached keys have received: for each key of a sequence and key head, the sum over the call's rows that see it of
// exp(scale * ks[page] * q_i.k_j - lse_i).
//
// Every key's sum is one thread's (or one warp's, in a fixed order): nothing is joined, and a call repeats bit for bit.
#include "roomie_kv_attention.cuh"

namespace roomie {

struct WeightArgs {
    KvView c;
    const int32_t *seqs, *q_offset;
    uint32_t num_seqs, rows, q_heads, group;
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
// of the codes.
constexpr int kWeightWarps = 4, kWeightThreads = 32 * kWeightWarps;

template <int DP> struct FewWeights {
    static constexpr int kGroups = DP > 128 ? 1 : 2;                // 16-key groups of a step
    static constexpr int kStep = 16 * kGroups;
    static constexpr int kSide = kStep * DP;                        // bytes of a step's keys
    static constexpr int kStages = 16384 / kSide;                   // 16 KB a warp
    static constexpr int kStage = kSide + kStep * 4 + 16;           // codes, the keys' old weights, the groups' scales
    static constexpr int kRing = kStages * kStage;
    static constexpr int kSmem = kRing * kWeightWarps;
};

struct WeightSeq {                                   // a sequence of the call, as its warps need it
    unsigned long long first;                        // flat index of its first step
    uint32_t slot, row, count, length, step0, steps; // step0: a head's first step, of `steps`
};

template <int DP, int NT, int kFormat, class T>
__global__ void __launch_bounds__(kWeightThreads, 3) few_weights_kernel(WeightArgs a) {
    using F = FewWeights<DP>;
    constexpr int G = F::kGroups, KW = DP / 16, KS = DP / 16, kStages = F::kStages;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ WeightSeq sh_seq[kWeightThreads];
    __shared__ unsigned long long sh_sum[kWeightWarps];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
    const KvView& kv = a.c;
    uint8_t* ring = smem + wid * F::kRing;
    const unsigned long long me = (unsigned long long)blockIdx.x * kWeightWarps + wid, all_warps = (unsigned long long)gridDim.x * kWeightWarps;

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

        // ---- copies: a place of its own in the flat order, some steps ahead ----
        struct Place {
            uint32_t seq, head, step;
            unsigned long long left;                                // steps of the warp's share from here on
        };
        const unsigned long long inside = at - sh_seq[seq].first;
        Place now = {seq, (uint32_t)(inside / sh_seq[seq].steps), (uint32_t)(inside % sh_seq[seq].steps), end - at}, next = now;
        auto go_on = [&](Place& p) {
            --p.left;
            if (++p.step < sh_seq[p.seq].steps) return;
            p.step = 0;
            if (++p.head < kv.heads) return;
            p.head = 0;
            if (p.left) do ++p.seq; while (sh_seq[p.seq].steps == 0);
        };
        int32_t page[G];
        auto get_pages = [&] {                                      // of the place that is copied next
#pragma unroll
            for (int g = 0; g < G; ++g) page[g] = -1;
            if (!next.left) return;
            const WeightSeq& s = sh_seq[next.seq];
            const uint32_t k0 = (s.step0 + next.step) * F::kStep;
            const int start = (int)s.length - (int)s.count;
            const uint32_t low = a.window ? (uint32_t)first_seen(start, a.window) : 0u;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t k = k0 + 16 * g;
                if (k >= s.length || k + 16 <= low) continue;
                const int32_t id = __ldg(kv.pages + (size_t)s.slot * kv.max_pages + (k >> kv.page_shift));
                page[g] = id;
                if ((uint32_t)id >= kv.num_pages) {
                    if (lane == 0) kv_flag(kv.status, ROOMIE_FLAG_KV_PAGE);
                    page[g] = -1;
                }
            }
        };
        constexpr int kChunks = DP / 16, kRowsPer = 32 / kChunks, kLoads = F::kStep / kRowsPer;
        const uint32_t chunk = lane % kChunks, row0 = lane / kChunks;
        auto copy_step = [&](int stage) {                           // of `next`, which moves on
            if (next.left) {
                const WeightSeq& s = sh_seq[next.seq];
                const uint32_t k0 = (s.step0 + next.step) * F::kStep, to = smem_addr(ring + stage * F::kStage);
#pragma unroll
                for (int i = 0; i < kLoads; ++i) {
                    const uint32_t row = row0 + i * kRowsPer, key = k0 + row;
                    const int g = i * kRowsPer / 16;                // (kRowsPer divides 16)
                    const uint32_t n = page[g] >= 0 && 16 * chunk < kv.dim && key < s.length ? 16u : 0u;   // the rest becomes zeros
                    const uint8_t* p = kv.k + (long long)max(page[g], 0) * kv.page_stride + (long long)next.head * kv.head_step +
                                       (long long)(key & (kv.page_tokens - 1)) * kv.token_step + 16 * chunk;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + code_at<DP>(row, chunk)), "l"(n ? p : kv.k), "r"(n) : "memory");
                }
                if (lane < F::kStep) {
                    const uint32_t key = k0 + lane;
                    const float* p = a.weight + ((size_t)s.slot * kv.heads + next.head) * a.max_tokens + key;
                    const uint32_t n = !a.fresh && key + s.count < s.length ? 4u : 0u;      // the call's own keys have received nothing before
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + F::kSide + 4 * lane), "l"(n ? p : a.weight), "r"(n) : "memory");
                }
                float* scales = reinterpret_cast<float*>(ring + stage * F::kStage + F::kSide + 4 * F::kStep);
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (lane == g) {
                        if (page[g] < 0) scales[g] = -1.0f;         // no page
                        else
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(scales + g)),
                                         "l"(kv.k_scale + (size_t)page[g] * kv.heads + next.head) : "memory");
                    }
                go_on(next);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        get_pages();
#pragma unroll 1
        for (int i = 0; i < kStages; ++i) {
            copy_step(i);
            get_pages();
        }

        // ---- queries of a tile of rows: operand b of S^T, row r of each eight, dims as the lane's keys ----
        uint32_t qf[NT][KS][2];
        float qscale[NT][2], lse2[NT][2];
        int see_hi[NT][2], see_lo[NT][2];                           // rows 2c and 2c + 1 of each eight see keys [lo, hi)
        auto load_queries = [&](const WeightSeq& s, uint32_t head, uint32_t first_row) {
            const uint32_t rows = s.count * a.group;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const uint32_t row = first_row + t * 8 + r, tok = row / a.group;
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
                    qf[t][i][0] = reinterpret_cast<const uint32_t&>(lo);
                    qf[t][i][1] = reinterpret_cast<const uint32_t&>(hi);
                }
                const float up = pow2f(e) * a.scale_log2;
                const float own = on ? a.lse[(size_t)(s.row + tok) * a.q_heads + head * a.group + row - tok * a.group] * kLog2e : 0.0f;
                const int start = (int)s.length - (int)s.count;
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    qscale[t][n] = __shfl_sync(0xffffffffu, up, (2 * c + n) * 4);
                    lse2[t][n] = __shfl_sync(0xffffffffu, own, (2 * c + n) * 4);
                    const uint32_t rc = first_row + t * 8 + 2 * c + n;
                    const int pos = start + (int)(rc / a.group);
                    see_hi[t][n] = rc < rows ? max(min(pos + 1, (int)s.length), 0) : 0;
                    see_lo[t][n] = a.window ? first_seen(pos, a.window) : 0;
                }
            }
        };

        uint32_t q_seq = 0xffffffffu, q_head = 0;
        int stage = 0;
        while (now.left) {
            const WeightSeq& s = sh_seq[now.seq];
            const uint32_t rows = s.count * a.group, k0 = (s.step0 + now.step) * F::kStep;
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            __syncwarp();
            const uint8_t* side = ring + stage * F::kStage;
            const float* old = reinterpret_cast<const float*>(side + F::kSide);
            float ks[G], sum[G][2];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                ks[g] = old[F::kStep + g];
                sum[g][0] = sum[g][1] = 0.0f;
            }
            for (uint32_t first_row = 0; first_row < rows; first_row += 8 * NT) {
                if (rows > 8 * NT || now.seq != q_seq || now.head != q_head) {
                    load_queries(s, now.head, first_row);
                    q_seq = now.seq;
                    q_head = now.head;
                }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float sc[NT][4];
#pragma unroll
                    for (int t = 0; t < NT; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.0f;
                    uint32_t kr[2][KW];
                    read_span<DP, KW>(kr[0], side, 16 * g + r, c * (DP / 4));
                    read_span<DP, KW>(kr[1], side, 16 * g + r + 8, c * (DP / 4));
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        uint32_t a0, a1, a2, a3;
                        codes_to_f16<kFormat>(kr[0][i], a0, a2);
                        codes_to_f16<kFormat>(kr[1][i], a1, a3);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma16816(sc[t], a0, a1, a2, a3, qf[t][i][0], qf[t][i][1]);
                    }
                    // sc[e] is key r + 8 * (e >> 1) of the group, row 2c + (e & 1)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int n = e & 1, k = (int)k0 + 16 * g + 8 * (e >> 1) + r;
                            const float p = exp2_fast(fmaf(sc[t][e], qscale[t][n] * ks[g], -lse2[t][n]));
                            if (k < see_hi[t][n] && k >= see_lo[t][n] && !(ks[g] < 0.0f)) sum[g][e >> 1] += p;
                        }
                }
            }
            // a key's rows lie in four lanes; lane c writes key r + 8 * (c & 1) of group c >> 1
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
            const uint32_t place = 16 * (c >> 1) + 8 * (c & 1) + r, key = k0 + place;
            if (c < 2 * G && key < s.length) a.weight[((size_t)s.slot * kv.heads + now.head) * a.max_tokens + key] = old[place] + mine;
            __syncwarp();                                           // the stage is read
            copy_step(stage);
            get_pages();
            if (++stage == kStages) stage = 0;
            go_on(now);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
}

template <int DP, int NT, int kFormat, class T> static int launch_few_weights(const WeightArgs& a, cudaStream_t st) {
    return launch("kv_weights", few_weights_kernel<DP, NT, kFormat, T>, dim3((uint32_t)sm_count() * 3), dim3(kWeightThreads), FewWeights<DP>::kSmem, st, false, a);
}
template <int DP, int kFormat, class T> static int weight_rows(const WeightArgs& a, bool eight, cudaStream_t st) {
    return eight ? launch_few_weights<DP, 1, kFormat, T>(a, st) : launch_few_weights<DP, 2, kFormat, T>(a, st);
}
template <int kFormat, class T> static int weight_dims(const WeightArgs& a, bool eight, cudaStream_t st) {
    if (a.c.dim <= 64) return weight_rows<64, kFormat, T>(a, eight, st);
    if (a.c.dim <= 128) return weight_rows<128, kFormat, T>(a, eight, st);
    return weight_rows<256, kFormat, T>(a, eight, st);
}
template <class T> static int weight_format(const WeightArgs& a, bool eight, cudaStream_t st) {
    return a.c.format == ROOMIE_KV_E4M3 ? weight_dims<ROOMIE_KV_E4M3, T>(a, eight, st) : weight_dims<ROOMIE_KV_INT8, T>(a, eight, st);
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
    a.q = q->data; a.q_token = q->token_stride; a.q_head = q->head_stride;
    a.lse = lse;
    a.max_tokens = cache->max_pages * cache->page_tokens;
    a.weight = weight + (size_t)layer * cache->max_seqs * cache->kv_heads * a.max_tokens;
    a.window = window;
    a.scale_log2 = scale * kLog2e;
    a.q_aligned = rows_aligned16(*q, rows, q_heads);
    a.fresh = fresh != 0;
    const bool eight = (unsigned long long)rows * a.group <= 8ull * num_seqs;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return q->type == ROOMIE_F16 ? weight_format<__half>(a, eight, st) : weight_format<__nv_bfloat16>(a, eight, st);
}
