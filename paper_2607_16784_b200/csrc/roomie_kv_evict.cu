// Eviction from the paged 8-bit cache: every layer and head keeps `keep` tokens - the first ones, the last ones and those that have received the most
// weight - moved together in their order.
#include "roomie_kv_attention.cuh"
#include "roomie_kv_pages.cuh"

namespace roomie {

// ---- the plan: which pages the kept tokens go to ---------------------------------------------------------------------------------------
// Workspace of n requests: length (-1: nothing is done), need, first, blocks that are done (n words each), the claims of max_seqs slots, the list
// of free pages and the pages that they replace (num_pages each).
struct EvictView {
    int32_t *len, *need, *first, *done, *owner, *list, *replaced;
};
__host__ __device__ __forceinline__ EvictView evict_view(int32_t* ws, uint32_t n, uint32_t max_seqs, uint32_t num_pages) {
    int32_t* list = ws + 4 * (size_t)n + max_seqs;
    return {ws, ws + n, ws + 2 * (size_t)n, ws + 3 * (size_t)n, ws + 4 * (size_t)n, list, list + num_pages};
}

// While the call runs, a page of the kept part that another sequence holds too stands in the table as the complement of its place in the list.
// The last block of a sequence puts the new pages into the table, gives up the old ones and sets the length.
__global__ void __launch_bounds__(kPlanThreads) evict_plan_kernel(TableView t, const int32_t* seqs, uint32_t n, uint32_t keep, int32_t* ws) {
    __shared__ uint32_t sh[kPlanWarps];
    const EvictView v = evict_view(ws, n, t.max_seqs, t.num_pages);
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
                const int32_t holders = id >= 0 && (uint32_t)id < t.num_pages ? t.refs[id] : 0;
                broken = broken || holders < 1;                   // no page, or one that counts as free and may be handed out here
                shared += e < now && holders > 1;
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
        uint32_t at = (uint32_t)v.first[i];
        for (uint32_t base = 0; base < now; base += 32) {
            const uint32_t e = base + lane;
            const bool shared = e < now && t.refs[row[e]] > 1;
            const uint32_t votes = __ballot_sync(0xffffffffu, shared);
            if (shared) {
                const uint32_t place = at + __popc(votes & ((1u << lane) - 1));
                v.replaced[place] = row[e];
                row[e] = ~(int32_t)place;
            }
            at += __popc(votes);
        }
    }
    if (bad) kv_flag(t.status, bad);
}

// ---- selection and move ------------------------------------------------------------------------------------------------------------------
struct EvictArgs {
    KvView c;                                       // of layer 0
    long long layer_stride;
    uint32_t layers, n, keep, first, recent, max_tokens;
    const int32_t* seqs;
    int32_t* ws;
    const float* weight;
    float* weight_out;
    int32_t *refs, *pages_out, *length;
};

// A block has one (sequence, layer, head), keys and values alike.
//
// Selection: the smallest kept weight by its bits, 11, 11 and 10 at a time, from histograms in shared memory, where the first kCached weights'
// bits lie too; then a bit for each token and the number of kept ones in front of each 128.
//
// Move: rounds of 256 tokens, in order.  A warp has the keys or the values of 32 of them: a lane looks up where one token comes from, then each token's
// 16-byte pieces are read by kLanes neighbouring lanes, all at once, into registers; the next round's tokens are looked up meanwhile.  Behind the one
// barrier of a round, when the pages' largest magnitudes are known, the codes are written.  A token never moves up, so what a round writes was read by it
// or a round before, and no round after it reads there: tokens move inside their own pages.
//
// Bound by memory, whose rows of a head are scattered 128 bytes, with the integer pipe half full: 16 sequences of up to 8192 tokens to 2048 each, 16 layers
// of 8 heads of 128 (2.2 GB read and written): 485 us, 4600 GB/s.  A few short sequences (8 of up to 1280 to 1024, 4 layers: 46 us with the plan and the
// reservation behind it) are a chain of waits: the plan 8, histograms 8, four rounds.  512 threads, two blocks an SM: one block's histograms run beside
// the other's copies.
constexpr int kEvictThreads = 512, kEvictWarps = kEvictThreads / 32, kCached = 8192;

// One thread, after a barrier of its block: what the block read of the table comes before the count, what it writes there behind it.
__device__ __forceinline__ uint32_t count_done(int32_t* counter) {
    __threadfence();
    const uint32_t before = (uint32_t)atomicAdd(counter, 1);
    __threadfence();
    return before;
}

struct EvictShared {
    uint32_t hist[2048];
    uint32_t amax[3][2][kEvictWarps];                        // rounds in turn, side, page: bits of the largest magnitude
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
// Pairs of bytes are compared by the upper one: as they are, and shifted up by one.
template <int kFormat> __device__ __forceinline__ float largest_of(const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t m;
        if constexpr (kFormat == ROOMIE_KV_E4M3) {
            m = w[i] & 0x7f7f7f7fu;
        } else {
            const uint32_t sign = (w[i] >> 7) & 0x01010101u;
            m = (w[i] ^ (sign * 0xffu)) + sign;                     // -128 becomes 128: no byte carries
        }
        most = __vimax3_u16x2(most, m, m << 8);
    }
    most = max(most >> 24, (most >> 8) & 0xffu);
    if constexpr (kFormat == ROOMIE_KV_E4M3) return kv_value((uint8_t)min(most, 0x7eu), ROOMIE_KV_E4M3);
    return (float)most;
}

// 16 codes times `ratio`, a power of two from 2^-15 to 2^7, rounded to codes.  In float16 code and product are exact: the only rounding is that to
// the code.
template <int kFormat> __device__ __forceinline__ uint4 multiplied(const uint4& x, float ratio) {
    uint4 y;
    const uint32_t* w = &x.x;
    uint32_t* o = &y.x;
    const __half2 r = __float2half2_rn(ratio);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t lo, hi;
        codes_to_f16<kFormat>(w[i], lo, hi);
        if constexpr (kFormat == ROOMIE_KV_E4M3) {
            const __half2 a = __hmul2(reinterpret_cast<const __half2&>(lo), r), b = __hmul2(reinterpret_cast<const __half2&>(hi), r);
            asm("{\n\t.reg .b16 a, b;\n\tcvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n\tcvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n\tmov.b32 %0, {a, b};\n\t}"
                : "=r"(o[i]) : "r"(reinterpret_cast<const uint32_t&>(a)), "r"(reinterpret_cast<const uint32_t&>(b)));
        } else {
            // added to 1536 the product is rounded to a whole number, whose two's complement is the low byte
            const __half2 magic = __float2half2_rn(1536.0f);
            const __half2 a = __hfma2(reinterpret_cast<const __half2&>(lo), r, magic), b = __hfma2(reinterpret_cast<const __half2&>(hi), r, magic);
            o[i] = __byte_perm(reinterpret_cast<const uint32_t&>(a), reinterpret_cast<const uint32_t&>(b), 0x6420);
        }
    }
    return y;
}

// 16 codes of scale `from`, any number, to codes of the scale whose inverse is `inverse`, a power of two
template <int kFormat> __device__ __noinline__ uint4 rescaled(uint4 x, float from, float inverse) {
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

// kLanes: the least power of two that is at least a token's pieces; also the pieces of a lane.
template <int kFormat, int kLanes>
__global__ void __launch_bounds__(kEvictThreads, kLanes == 16 ? 1 : 2) evict_kernel(EvictArgs a) {
    constexpr uint32_t kTokens = 16 * kEvictWarps, kSpan = 32 / kLanes;           // of a round; of a warp's load
    extern __shared__ uint32_t bits[];              // a bit for each of max_tokens, 1: kept; then how many are kept in front of each 128; then the
                                                    // bits of the first weights
    __shared__ EvictShared sh;
    grid_dependency_wait();                         // the plan; this kernel's start overlaps its end
    const KvView& c = a.c;
    const uint32_t head = blockIdx.x % c.heads, rest = blockIdx.x / c.heads, layer = rest % a.layers, i = rest / a.layers;
    const EvictView v = evict_view(a.ws, a.n, c.max_seqs, c.num_pages);
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
    uint32_t* ahead = bits + (a.max_tokens + 31) / 32;
    uint32_t* cached = ahead + (a.max_tokens + 127) / 128;
    auto bits_at = [&](uint32_t p) { return p < kCached ? cached[p] : weight_bits(weight[p]); };
    if (quota) {
#pragma unroll 8
        for (uint32_t p = tid; p < min(end, (uint32_t)kCached); p += kEvictThreads) cached[p] = weight_bits(weight[p]);
#pragma unroll 1
        for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift - 10) {       // digits [21, 32), [10, 21), [0, 10)
            for (uint32_t b = tid; b < 2048; b += kEvictThreads) sh.hist[b] = 0;
            __syncthreads();
            const uint32_t digits = shift ? 0x7ffu : 0x3ffu, above = shift == 21 ? 0u : shift == 10 ? 21u : 10u;
#pragma unroll 4
            for (uint32_t p = a.first + tid; p < end; p += kEvictThreads) {
                const uint32_t b = bits_at(p);
                if (above == 0 || b >> above == least >> above) atomicAdd(&sh.hist[(b >> shift) & digits], 1u);
            }
            __syncthreads();
            // some digits a thread, from the top: the one in which the left-th lies
            constexpr uint32_t kDigits = 2048 / kEvictThreads;
            uint32_t mine = 0;
#pragma unroll
            for (uint32_t k = 0; k < kDigits; ++k) mine += sh.hist[2047 - kDigits * tid - k];
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
                uint32_t k = 2047 - kDigits * tid;
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
        const uint32_t b = middle && quota ? bits_at(p) : 0u;
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
    if (tid < 6 * kEvictWarps) (&sh.amax[0][0][0])[tid] = 0;
    __syncthreads();

    // ---- move ----
    const int32_t* table = c.pages + (size_t)slot * c.max_pages;
    const uint32_t now = (keep + c.page_tokens - 1) >> c.page_shift, rounds = (keep + kTokens - 1) / kTokens;
    const uint32_t side = wid / (kEvictWarps / 2), mine = 32 * (wid % (kEvictWarps / 2)), own = mine + lane;     // this lane's token of a round
    const uint32_t piece = lane & (kLanes - 1), sub = lane / kLanes;  // load e: token e * kSpan + sub of the warp's
    const bool real = 16 * piece < c.dim, two = c.page_tokens == 16;  // two: the warp's tokens lie in two pages
    uint8_t* pool = (side ? c.v : c.k) + (long long)layer * a.layer_stride + (long long)head * c.head_step + (real ? 16 * piece : 0);
    float* scales = (side ? c.v_scale : c.k_scale) + (size_t)layer * c.num_pages * c.heads + head;
    long long from = -1;                            // of this lane's token: bytes from the pool's start, its page's scale, its weight
    float scale = 0.0f, heavy = 0.0f;
    auto look_up = [&](uint32_t round) {
        const uint32_t rank = round * kTokens + own;
        from = -1;
        if (rank >= keep) return;
        uint32_t lo = 0, hi = fours;                // ahead[lo] <= rank < ahead[hi]
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (ahead[mid] <= rank) lo = mid;
            else hi = mid;
        }
        uint32_t skip = rank - ahead[lo], w = 4 * lo;
        for (uint32_t n; skip >= (n = __popc(bits[w])); ++w) skip -= n;
        uint32_t b = bits[w], p = 32 * w;
#pragma unroll
        for (int half = 16; half > 0; half /= 2) {  // the skip-th set bit
            const uint32_t n = __popc(b & ((1u << half) - 1));
            if (skip >= n) {
                skip -= n;
                b >>= half;
                p += half;
            }
        }
        int32_t id = table[p >> c.page_shift];
        if (id < 0) id = v.replaced[~id];
        from = (long long)id * c.page_stride + (long long)(p & (c.page_tokens - 1)) * c.token_step;
        scale = scales[(size_t)id * c.heads];
        if (side == 0) heavy = weight[p];
    };
    look_up(0);
    for (uint32_t round = 0; round < rounds; ++round) {
        uint4 x[kLanes];
#pragma unroll
        for (int e = 0; e < kLanes; ++e) {
            const long long at = __shfl_sync(0xffffffffu, max(from, 0ll), e * kSpan + sub);   // some token where there is none: it counts as 0
            x[e] = __ldcs(reinterpret_cast<const uint4*>(pool + at));
        }
        const bool there = from >= 0;
        const float was = there ? scale : 0.0f, carried = heavy;
        if (round + 1 < rounds) look_up(round + 1);
        uint32_t* amax = sh.amax[round % 3][side];
        const uint32_t page = own >> c.page_shift;                    // of this lane's token, in the round
        float most[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < kLanes; ++e) {
            const float m = largest_of<kFormat>(x[e]) * __shfl_sync(0xffffffffu, was, e * kSpan + sub);
            if (kLanes == 1) most[lane >> 4] = m;
            else most[2 * e / kLanes] = fmaxf(most[2 * e / kLanes], m);
        }
        if (!real) most[0] = most[1] = 0.0f;
        if (!two) most[0] = fmaxf(most[0], most[1]);
        {
            const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(most[0]));
            if (lane == 0) atomicMax(amax + page, m);
        }
        if (two) {
            const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(most[1]));
            if (lane == 16) atomicMax(amax + page, m);
        }
        __syncthreads();
        // where this lane's token goes, and by what its codes are multiplied: a power of two near 1, or else (negative) their scale
        const int exponent = kv_scale_exponent(__uint_as_float(amax[page]), kFormat);
        const uint32_t target = round * (kTokens >> c.page_shift) + page;
        int32_t id = target < now ? table[target] : 0;
        if (id < 0) id = v.list[~id];
        float ratio = was * pow2f(-exponent);
        if ((__float_as_uint(ratio) & 0x7fffffu) != 0 || ratio < 0x1p-15f || ratio > 0x1p7f) ratio = -was;
        if (there) {
            if (side == 0) weight_out[round * kTokens + own] = carried;
            if ((own & (c.page_tokens - 1)) == 0) scales[(size_t)id * c.heads] = pow2f(exponent);
        }
        const uint32_t known = __ballot_sync(0xffffffffu, there);
        const int exponent0 = __shfl_sync(0xffffffffu, exponent, 0), exponent1 = __shfl_sync(0xffffffffu, exponent, 31);
        // the first token's page, and with `two` the last one's
        const int32_t last = __shfl_sync(0xffffffffu, id, 31);
        id = __shfl_sync(0xffffffffu, id, 0);
        uint8_t* to = pool + (long long)id * c.page_stride + (long long)((mine + sub) & (c.page_tokens - 1)) * c.token_step;
        const long long step = (long long)kSpan * c.token_step;
        if (two && kLanes == 1 && sub >= 16) to += (long long)(last - id) * c.page_stride;
#pragma unroll
        for (int e = 0; e < kLanes; ++e) {
            const uint32_t t = e * kSpan + sub;
            const float r = __shfl_sync(0xffffffffu, ratio, t);
            if (kLanes > 1 && e == kLanes / 2 && two) to += (long long)(last - id) * c.page_stride - 16ll * c.token_step;
            if ((known >> t & 1) && real) {
                if (r > 0.0f) {
                    if (r != 1.0f) x[e] = multiplied<kFormat>(x[e], r);
                } else {
                    x[e] = rescaled<kFormat>(x[e], -r, pow2f(-(t < 16 ? exponent0 : exponent1)));
                }
                __stcs(reinterpret_cast<uint4*>(to), x[e]);
            }
            to += step;
        }
        if (tid < 2 * kEvictWarps) (&sh.amax[(round + 2) % 3][0][0])[tid] = 0;    // read before this round's barrier, written behind the next one's
    }
    for (uint32_t p = keep + tid; p < len; p += kEvictThreads) weight_out[p] = 0.0f;

    // ---- the sequence's last block: the table ----
    __syncthreads();
    if (tid == 0) sh.last = count_done(v.done + i) == a.layers * c.heads - 1;
    __syncthreads();
    if (!sh.last) return;
    const uint32_t held = (len + c.page_tokens - 1) >> c.page_shift;
    int32_t* entries = a.pages_out + (size_t)slot * c.max_pages;
    for (uint32_t e = tid; e < held; e += kEvictThreads) {
        const int32_t id = entries[e];
        if (id >= 0 && e < now) continue;
        int32_t* count = a.refs + (id < 0 ? v.replaced[~id] : id);
        if (atomicSub(count, 1) <= 0) {
            atomicAdd(count, 1);
            kv_flag(c.status, ROOMIE_FLAG_KV_PAGE);
        }
        const int32_t to = id < 0 ? v.list[~id] : -1;
        if (id < 0) a.refs[to] = 1;
        entries[e] = to;
    }
    if (tid == 0) a.length[slot] = (int32_t)keep;
}
template <int kFormat> static void (*evict_kernel_for(const roomie_kv_cache* c))(EvictArgs) {
    const uint32_t pieces = c->head_dim / 16;
    if (pieces == 1) return evict_kernel<kFormat, 1>;
    if (pieces == 2) return evict_kernel<kFormat, 2>;
    if (pieces <= 4) return evict_kernel<kFormat, 4>;
    return pieces <= 8 ? evict_kernel<kFormat, 8> : evict_kernel<kFormat, 16>;
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
    a.seqs = seqs; a.ws = page_scratch(cache, workspace);
    a.weight = weight; a.weight_out = weight_out;
    a.refs = cache->refs; a.pages_out = cache->pages; a.length = cache->length;
    const size_t smem = ((tokens + 31) / 32 + (tokens + 127) / 128 + (tokens < kCached ? tokens : kCached)) * sizeof(uint32_t);
    void (*k)(EvictArgs) = cache->format == ROOMIE_KV_E4M3 ? evict_kernel_for<ROOMIE_KV_E4M3>(cache) : evict_kernel_for<ROOMIE_KV_INT8>(cache);
    rc = allow_smem(reinterpret_cast<const void*>(k), smem);      // before the plan, which marks entries of the table
    if (rc != ROOMIE_OK) return rc;
    rc = launch("kv_evict_plan", evict_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, false, table_view(cache), seqs, n, keep, a.ws);
    if (rc != ROOMIE_OK) return rc;
    return launch("kv_evict", k, dim3(n * cache->layers * cache->kv_heads), dim3(kEvictThreads), smem, st, true, a);
}
