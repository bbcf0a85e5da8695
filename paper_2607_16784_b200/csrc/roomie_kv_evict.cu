// Eviction from the paged 8-bit cache: every layer and head keeps `keep` tokens - the first ones, the last ones and those that have received the most
// weight - moved together in their order.
#include "roomie_kv_pages.cuh"

namespace roomie {

// ---- the plan: which pages the kept tokens go to ---------------------------------------------------------------------------------------
// Workspace of n requests: length (-1: nothing is done), need, first, blocks that are done (n words each), the claims of max_seqs slots, the list
// of free pages (num_pages).
struct EvictView {
    int32_t *len, *need, *first, *done, *owner, *list;
};
__host__ __device__ __forceinline__ EvictView evict_view(int32_t* ws, uint32_t n, uint32_t max_seqs) {
    return {ws, ws + n, ws + 2 * (size_t)n, ws + 3 * (size_t)n, ws + 4 * (size_t)n, ws + 4 * (size_t)n + max_seqs};
}

// While the call runs, a page of the kept part that another sequence holds too stands in the table as its complement: its tokens go to a page of the
// list.  The last block of a sequence puts the new pages into the table, gives up the old ones and sets the length.
__global__ void __launch_bounds__(kPlanThreads) evict_plan_kernel(TableView t, const int32_t* seqs, uint32_t n, uint32_t keep, int32_t* ws) {
    __shared__ uint32_t sh[kPlanWarps];
    const EvictView v = evict_view(ws, n, t.max_seqs);
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, now = pages_of(t, keep);
    uint32_t bad = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads)
        if (slot_ok(t, seqs[i])) v.owner[seqs[i]] = 0x7fffffff;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads)
        if (slot_ok(t, seqs[i])) atomicMin(v.owner + seqs[i], (int32_t)i);
    __syncthreads();
    for (uint32_t i = wid; i < n; i += kPlanWarps) {
        const int32_t s = seqs[i];
        int32_t len = length_of(t, s);
        if (len < 0 || v.owner[s] != (int32_t)i) {                // no sequence, or one named before
            bad |= ROOMIE_FLAG_KV_SEQUENCE;
            len = -1;
        }
        uint32_t shared = 0;
        if (len > (int32_t)keep) {
            const int32_t* row = t.pages + (size_t)s * t.max_pages;
            bool broken = false;
            for (uint32_t e = lane; e < pages_of(t, (uint32_t)len); e += 32) {
                const int32_t id = row[e];
                const bool there = id >= 0 && (uint32_t)id < t.num_pages;
                broken = broken || !there;
                shared += e < now && there && t.refs[id] > 1;
            }
            if (__any_sync(0xffffffffu, broken)) {
                bad |= ROOMIE_FLAG_KV_PAGE;
                len = -1;
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) shared += __shfl_xor_sync(0xffffffffu, shared, d);
        } else {
            len = -1;
        }
        if (lane == 0) {
            v.len[i] = len;
            v.need[i] = len < 0 ? 0 : (int32_t)shared;
            v.done[i] = 0;
        }
    }
    __syncthreads();
    const uint32_t found = serve(t, n, v.need, v.first, v.list, t.num_pages, sh);
    __syncthreads();
    for (uint32_t i = wid; i < n; i += kPlanWarps) {
        if (v.need[i] == 0) continue;
        if ((unsigned long long)v.first[i] + (uint32_t)v.need[i] > found) {
            bad |= ROOMIE_FLAG_KV_FULL;
            if (lane == 0) v.len[i] = -1;
            continue;
        }
        int32_t* row = t.pages + (size_t)seqs[i] * t.max_pages;
        for (uint32_t e = lane; e < now; e += 32)
            if (t.refs[row[e]] > 1) row[e] = ~row[e];
    }
    if (bad) kv_flag(t.status, bad);
}

// ---- selection and move ------------------------------------------------------------------------------------------------------------------
struct EvictArgs {
    KvView c;                                       // of layer 0
    long long layer_stride;
    uint32_t layers, n, keep, first, recent, max_tokens;
    uint32_t pieces, piece_inverse;                 // 16-byte pieces of a token, and 2^20 / pieces + 1
    uint32_t pages;                                 // of a round
    const int32_t* seqs;
    int32_t* ws;
    const float* weight;
    float* weight_out;
    int32_t *refs, *pages_out, *length;
};

// A block has one (sequence, layer, head), keys and values alike.
//
// Selection: the smallest kept weight by its bits, 11, 11 and 10 at a time, from histograms in shared memory; then a bit for each token and the
// number of kept ones in front of each 128.
//
// Move: rounds of up to 256 tokens, in order.  A round's codes are read into registers (16 pieces of 16 bytes a thread: four warps have
// the keys, four the values), the pages' largest magnitudes are found, and behind a barrier the codes are written.  A token never moves up,
// so what a round writes was read by it or a round before, and no round after it reads there: tokens move inside their own pages.  Where the tokens of
// the next round come from is looked up while this round's codes arrive.
constexpr int kEvictThreads = 256, kEvictWarps = kEvictThreads / 32, kRoundTokens = 256, kPiecesEach = 16;

// One thread, after a barrier of its block: what the block read of the table comes before the count, what it writes there behind it.
__device__ __forceinline__ uint32_t count_done(int32_t* counter) {
    __threadfence();
    const uint32_t before = (uint32_t)atomicAdd(counter, 1);
    __threadfence();
    return before;
}

struct Origin {                                     // of a token of a round
    long long at;                                   // bytes from the pool's start; -1: there is none
    float ks, vs;
};
struct EvictShared {
    uint32_t hist[2048];
    Origin origin[3][kRoundTokens];                 // rounds in turn: one that is read, one that is filled, one that may still be read
    int32_t target[3][16];                          // the pages that a round's tokens go to
    uint32_t amax[3][2][16];                        // rounds in turn, side, page: bits of the largest magnitude
    uint32_t part[kEvictWarps];
    uint32_t digit, left, ties, last;
};

// bits in the order of the weights; NaN is below all, -0 is 0
__device__ __forceinline__ uint32_t weight_bits(float x) {
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// The largest magnitude of 16 codes.  Codes of e4m3 are in the order of their magnitudes but for the sign (NaN, 0x7f, counts as the largest value).
template <int kFormat> __device__ __forceinline__ float largest_of(const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t even = 0, odd = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t m;
        if constexpr (kFormat == ROOMIE_KV_E4M3) {
            m = w[i] & 0x7f7f7f7fu;
        } else {
            const uint32_t sign = (w[i] >> 7) & 0x01010101u;
            m = (w[i] ^ (sign * 0xffu)) + sign;                     // -128 becomes 128: no byte carries
        }
        even = __vmaxu2(even, m & 0x00ff00ffu);
        odd = __vmaxu2(odd, (m >> 8) & 0x00ff00ffu);
    }
    even = __vmaxu2(even, odd);
    uint32_t most = max(even & 0xffffu, even >> 16);
    if constexpr (kFormat == ROOMIE_KV_E4M3) return kv_value((uint8_t)min(most, 0x7eu), ROOMIE_KV_E4M3);
    return (float)most;
}

// 16 codes of scale `from` to codes of the power of two whose inverse is `inverse`
template <int kFormat> __device__ __forceinline__ uint4 rescaled(const uint4& x, float from, float inverse) {
    uint4 y;
    const uint32_t* w = &x.x;
    uint32_t* o = &y.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t r = 0;
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const float a = kv_value((uint8_t)(w[i] >> (8 * k)), kFormat) * from, b = kv_value((uint8_t)(w[i] >> (8 * k + 8)), kFormat) * from;
            r |= (kv_codes2(a * inverse, b * inverse, kFormat) & 0xffffu) << (8 * k);
        }
        o[i] = r;
    }
    return y;
}

template <int kFormat>
__global__ void __launch_bounds__(kEvictThreads, 2) evict_kernel(EvictArgs a) {
    extern __shared__ uint32_t bits[];              // a bit for each of max_tokens, 1: kept; then how many are kept in front of each 128
    __shared__ EvictShared sh;
    grid_dependency_wait();                         // the plan; this kernel's start overlaps its end
    const KvView& c = a.c;
    const uint32_t head = blockIdx.x % c.heads, rest = blockIdx.x / c.heads, layer = rest % a.layers, i = rest / a.layers;
    const EvictView v = evict_view(a.ws, a.n, c.max_seqs);
    const int32_t length = v.len[i];
    if (length < 0) return;
    const uint32_t tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, len = (uint32_t)length, keep = a.keep;
    const uint32_t slot = (uint32_t)a.seqs[i];
    const size_t row = (((size_t)layer * c.max_seqs + slot) * c.heads + head) * a.max_tokens;
    const float* weight = a.weight + row;
    float* weight_out = a.weight_out + row;

    // ---- selection among [first, end) of `quota` ----
    const uint32_t end = len - a.recent, quota = keep - a.first - a.recent;
    uint32_t least = 0, left = quota, ties = 0;     // kept: those above `least`, and the first `left` of the `ties` that equal it
    if (quota) {
#pragma unroll 1
        for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {       // digits [21, 32), [10, 21), [0, 10)
            for (uint32_t b = tid; b < 2048; b += kEvictThreads) sh.hist[b] = 0;
            __syncthreads();
            const uint32_t digits = shift ? 0x7ffu : 0x3ffu, above = shift == 21 ? 0u : shift == 10 ? 21u : 10u;
#pragma unroll 4
            for (uint32_t p = a.first + tid; p < end; p += kEvictThreads) {
                const uint32_t b = weight_bits(weight[p]);
                if (above == 0 || b >> above == least >> above) atomicAdd(&sh.hist[(b >> shift) & digits], 1u);
            }
            __syncthreads();
            // eight digits a thread, from the top: the one in which the left-th lies
            uint32_t mine = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) mine += sh.hist[2047 - 8 * tid - k];
            uint32_t upto = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t up = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += up;
            }
            if (lane == 31) sh.part[wid] = upto;
            __syncthreads();
            uint32_t before = upto - mine;
            for (uint32_t w = 0; w < wid; ++w) before += sh.part[w];
            if (before < left && left <= before + mine) {
                uint32_t k = 2047 - 8 * tid;
                while (before + sh.hist[k] < left) before += sh.hist[k--];
                sh.digit = k;
                sh.left = left - before;
                sh.ties = sh.hist[k];
            }
            __syncthreads();
            least |= sh.digit << shift;
            left = sh.left;
            ties = sh.ties;
        }
    }
    // ---- a bit for each token: a warp has a run of words ----
    const uint32_t words = (len + 31) / 32, each = (words + kEvictWarps - 1) / kEvictWarps, w0 = min(wid * each, words), w1 = min(w0 + each, words);
    auto look = [&](uint32_t w, bool& over, bool& same) {
        const uint32_t p = 32 * w + lane;
        const bool middle = p >= a.first && p < end;
        const uint32_t b = middle && quota ? weight_bits(weight[p]) : 0u;
        over = p < len && (!middle || (quota && b > least));
        same = middle && quota && b == least;
    };
    uint32_t take = 0xffffffffu;                    // of those that equal `least`, from this warp's first on
    if (left < ties) {
        uint32_t count = 0;
        for (uint32_t w = w0; w < w1; ++w) {
            bool over, same;
            look(w, over, same);
            count += same;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) count += __shfl_xor_sync(0xffffffffu, count, d);
        __syncthreads();
        if (lane == 0) sh.part[wid] = count;
        __syncthreads();
        take = left;
        for (uint32_t w = 0; w < wid; ++w) take = take > sh.part[w] ? take - sh.part[w] : 0u;
    }
#pragma unroll 4
    for (uint32_t w = w0; w < w1; ++w) {
        bool over, same;
        look(w, over, same);
        const uint32_t equal = __ballot_sync(0xffffffffu, same), kept = __ballot_sync(0xffffffffu, over || (same && __popc(equal & ((1u << lane) - 1)) < take));
        if (lane == 0) bits[w] = kept;
        const uint32_t n = __popc(equal);
        take = take > n ? take - n : 0u;
    }
    __syncthreads();
    // kept ones in front of each four words
    const uint32_t fours = (words + 3) / 4, run = (fours + kEvictThreads - 1) / kEvictThreads;
    uint32_t* ahead = bits + (a.max_tokens + 31) / 32;
    {
        auto of = [&](uint32_t f) {
            uint32_t n = 0;
            for (uint32_t w = 4 * f; w < min(4 * f + 4, words); ++w) n += __popc(bits[w]);
            return n;
        };
        uint32_t mine = 0;
        for (uint32_t f = tid * run; f < min((tid + 1) * run, fours); ++f) mine += of(f);
        uint32_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += up;
        }
        if (lane == 31) sh.part[wid] = upto;
        __syncthreads();
        uint32_t before = upto - mine;
        for (uint32_t w = 0; w < wid; ++w) before += sh.part[w];
        for (uint32_t f = tid * run; f < min((tid + 1) * run, fours); ++f) {
            ahead[f] = before;
            before += of(f);
        }
    }
    if (tid < 96) (&sh.amax[0][0][0])[tid] = 0;
    __syncthreads();

    // ---- move ----
    const int32_t* table = c.pages + (size_t)slot * c.max_pages;
    const uint32_t now = (keep + c.page_tokens - 1) >> c.page_shift;
    uint32_t fresh = (uint32_t)v.first[i];          // of the first warp: how many of the list's pages are taken, from the call's first on
    const size_t scale_row = (size_t)layer * c.num_pages * c.heads + head;
    const uint32_t tokens = a.pages * c.page_tokens, rounds = (keep + tokens - 1) / tokens;    // tokens of a round, at most 256
    float moved = 0.0f;                             // the weight of this thread's token of the next round
    auto origins = [&](uint32_t round) {
        const uint32_t rank = round * tokens + tid;
        if (wid == 0) {
            const uint32_t e = round * a.pages + lane;
            const int32_t id = lane < a.pages && e < now ? table[e] : 0;
            const uint32_t votes = __ballot_sync(0xffffffffu, id < 0);
            if (lane < a.pages) sh.target[round % 3][lane] = id < 0 ? v.list[fresh + __popc(votes & ((1u << lane) - 1))] : id;
            fresh += __popc(votes);
        }
        if (tid >= tokens) return;
        Origin o = {-1, 0.0f, 0.0f};
        if (rank < keep) {
            uint32_t lo = 0, hi = fours;            // ahead[lo] <= rank < ahead[hi]
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (ahead[mid] <= rank) lo = mid;
                else hi = mid;
            }
            uint32_t skip = rank - ahead[lo], w = 4 * lo;
            for (uint32_t n; skip >= (n = __popc(bits[w])); ++w) skip -= n;
            uint32_t b = bits[w];
            for (; skip; --skip) b &= b - 1;
            const uint32_t p = 32 * w + __ffs(b) - 1;
            int32_t id = table[p >> c.page_shift];
            if (id < 0) id = ~id;
            o.at = (long long)id * c.page_stride + (long long)(p & (c.page_tokens - 1)) * c.token_step;
            o.ks = c.k_scale[scale_row + (size_t)id * c.heads];
            o.vs = c.v_scale[scale_row + (size_t)id * c.heads];
            moved = weight[p];
        }
        sh.origin[round % 3][tid] = o;
    };
    origins(0);
    __syncthreads();
    const uint32_t side = wid >> 2, piece0 = (wid & 3) * 32 + lane;
    uint8_t* pool = (side ? c.v : c.k) + (long long)layer * a.layer_stride + (long long)head * c.head_step;
    float* scales = (side ? c.v_scale : c.k_scale) + scale_row;
    const uint32_t pieces = tokens * a.pieces;      // of a side and round: at most 2048
    for (uint32_t round = 0; round < rounds; ++round) {
        const Origin* from = sh.origin[round % 3];
        uint32_t* amax = sh.amax[round % 3][side];
        uint4 x[kPiecesEach];
        float scale[kPiecesEach];
        const float was = moved;
#pragma unroll
        for (int e = 0; e < kPiecesEach; ++e) {
            const uint32_t f = piece0 + e * 128, token = (f * a.piece_inverse) >> 20;
            scale[e] = -1.0f;
            if (f < pieces && from[token].at >= 0) {
                x[e] = *reinterpret_cast<const uint4*>(pool + from[token].at + 16 * (f - token * a.pieces));
                scale[e] = side ? from[token].vs : from[token].ks;
            }
        }
        if (round + 1 < rounds) origins(round + 1);
#pragma unroll
        for (int e = 0; e < kPiecesEach; ++e) {
            const uint32_t f = piece0 + e * 128, token = (f * a.piece_inverse) >> 20, page = token >> c.page_shift;
            const float m = scale[e] >= 0.0f ? largest_of<kFormat>(x[e]) * scale[e] : 0.0f;
            if (f - lane >= pieces) break;          // the same for the warp
            if (c.page_tokens * a.pieces % 32 == 0) {
                const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
                if (lane == 0 && most) atomicMax(amax + page, most);
            } else if (f < pieces) {
                atomicMax(amax + page, __float_as_uint(m));
            }
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kPiecesEach; ++e) {
            const uint32_t f = piece0 + e * 128, token = (f * a.piece_inverse) >> 20, page = token >> c.page_shift;
            if (scale[e] < 0.0f) continue;
            const int exponent = kv_scale_exponent(__uint_as_float(amax[page]), kFormat);
            const float unit = pow2f(exponent);
            const int32_t id = sh.target[round % 3][page];
            uint8_t* to = pool + (long long)id * c.page_stride + (long long)(token & (c.page_tokens - 1)) * c.token_step + 16 * (f - token * a.pieces);
            *reinterpret_cast<uint4*>(to) = scale[e] == unit ? x[e] : rescaled<kFormat>(x[e], scale[e], pow2f(-exponent));
            if ((token & (c.page_tokens - 1)) == 0 && f == token * a.pieces) scales[(size_t)id * c.heads] = unit;
        }
        if (tid < tokens && round * tokens + tid < keep) weight_out[round * tokens + tid] = was;
        if (tid < 32) (&sh.amax[(round + 2) % 3][0][0])[tid] = 0;    // read before this round's barrier, written behind the next one's
    }
    for (uint32_t p = keep + tid; p < len; p += kEvictThreads) weight_out[p] = 0.0f;

    // ---- the sequence's last block: the table ----
    __syncthreads();
    if (tid == 0) sh.last = count_done(v.done + i) == a.layers * c.heads - 1;
    __syncthreads();
    if (!sh.last) return;
    const uint32_t held = (len + c.page_tokens - 1) >> c.page_shift;
    int32_t* entries = a.pages_out + (size_t)slot * c.max_pages;
    if (wid == 0) {
        fresh = (uint32_t)v.first[i];
        for (uint32_t base = 0; base < held; base += 32) {
            const uint32_t e = base + lane;
            const int32_t id = e < held ? entries[e] : 0;
            const bool replaced = e < now && id < 0;
            const uint32_t votes = __ballot_sync(0xffffffffu, replaced);
            if (e < held && (replaced || e >= now)) {
                int32_t* count = a.refs + (replaced ? ~id : id);
                if (atomicSub(count, 1) <= 0) {
                    atomicAdd(count, 1);
                    kv_flag(c.status, ROOMIE_FLAG_KV_PAGE);
                }
                const int32_t to = replaced ? v.list[fresh + __popc(votes & ((1u << lane) - 1))] : -1;
                if (replaced) a.refs[to] = 1;
                entries[e] = to;
            }
            fresh += __popc(votes);
        }
        if (lane == 0) a.length[slot] = (int32_t)keep;
    }
}

}  // namespace roomie

using namespace roomie;

extern "C" int roomie_kv_evict(const roomie_kv_cache* cache, const int32_t* seqs, uint32_t n, const float* weight, uint32_t keep, uint32_t first,
                               uint32_t recent, float* weight_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (kv_check(cache) != ROOMIE_OK || keep == 0 || keep > 0x7fffffffu || (unsigned long long)first + recent > keep) return ROOMIE_ERR_INVALID_ARG;
    const unsigned long long tokens = (unsigned long long)cache->max_pages * cache->page_tokens;
    if (tokens > 1u << 20) return ROOMIE_ERR_INVALID_ARG;
    if (n == 0) return ROOMIE_OK;
    if (!seqs || !weight || !weight_out || n > cache->max_seqs || (reinterpret_cast<uintptr_t>(weight) & 3u) || (reinterpret_cast<uintptr_t>(weight_out) & 3u) ||
        (unsigned long long)n * cache->layers * cache->kv_heads > 0x7fffffffull)
        return ROOMIE_ERR_INVALID_ARG;
    int rc = check_workspace(cache, workspace, workspace_bytes);
    if (rc != ROOMIE_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    EvictArgs a = {};
    a.c = kv_view(cache, 0);
    a.layer_stride = cache->layer_stride;
    a.layers = cache->layers; a.n = n; a.keep = keep; a.first = first; a.recent = recent; a.max_tokens = (uint32_t)tokens;
    a.pieces = cache->head_dim / 16;
    a.piece_inverse = (1u << 20) / a.pieces + 1;
    const uint32_t most = 2048 / (cache->page_tokens * a.pieces);                  // pages whose pieces fit the block's registers
    a.pages = most < kRoundTokens / cache->page_tokens ? most : kRoundTokens / cache->page_tokens;
    a.seqs = seqs; a.ws = page_scratch(cache, workspace);
    a.weight = weight; a.weight_out = weight_out;
    a.refs = cache->refs; a.pages_out = cache->pages; a.length = cache->length;
    rc = launch("kv_evict_plan", evict_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, false, table_view(cache), seqs, n, keep, a.ws);
    if (rc != ROOMIE_OK) return rc;
    const size_t smem = ((tokens + 31) / 32 + (tokens + 127) / 128) * sizeof(uint32_t);
    const uint32_t blocks = n * cache->layers * cache->kv_heads;
    return launch("kv_evict", cache->format == ROOMIE_KV_E4M3 ? evict_kernel<ROOMIE_KV_E4M3> : evict_kernel<ROOMIE_KV_INT8>, dim3(blocks), dim3(kEvictThreads), smem, st,
                  true, a);
}
