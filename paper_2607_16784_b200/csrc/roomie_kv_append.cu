// Quantise-and-append: new keys (rotated) and values into the paged 8-bit cache, and the step's queries rotated beside them.
#include <type_traits>
#include "roomie_kv.cuh"
#include "roomie_rope.cuh"

namespace roomie {

struct AppendArgs {
    KvView c;
    const int32_t *seqs, *q_offset;
    uint32_t num_seqs, rows;
    const void *k, *v;
    long long k_token, k_head, v_token, v_head;
    RopeView rope;                 // rot = 0: keys are stored as they come
    HeadRows q;
    uint32_t q_heads, q_units, q_groups, kv_blocks;
    unsigned long long q_threads;
};

constexpr int kAppendThreads = 512, kAppendWarps = kAppendThreads / 32;

// The `j`-th (sequence, page) in which the call's sequences have new tokens: every thread of the block gets the same answer.
// false: there are fewer.
__device__ bool find_page(const AppendArgs& a, uint32_t j, KvSeq& s, uint32_t& page, uint32_t* sh) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    uint32_t before = 0;
    for (uint32_t base = 0; base < a.num_seqs; base += kAppendThreads) {
        const uint32_t i = base + threadIdx.x;
        uint32_t n = 0;
        KvSeq mine = {};
        if (i < a.num_seqs) {
            mine = kv_seq(a.c, a.seqs, a.q_offset, a.rows, i, true);
            if (mine.count > mine.length) {                               // more new tokens than the sequence has in all
                kv_flag(a.c.status, ROOMIE_FLAG_KV_SEQUENCE);
            } else if (mine.count) {
                n = ((mine.length - 1) >> a.c.page_shift) - (mine.start >> a.c.page_shift) + 1;
            }
        }
        uint32_t incl = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        if (lane == 31) sh[wid] = incl;
        __syncthreads();
        uint32_t ahead = before, all = 0;
        for (int w = 0; w < kAppendWarps; ++w) {
            if (w < wid) ahead += sh[w];
            all += sh[w];
        }
        const uint32_t first = ahead + incl - n;
        if (n && j >= first && j < first + n) {
            sh[16] = mine.slot; sh[17] = mine.row; sh[18] = mine.count; sh[19] = mine.start; sh[20] = mine.length;
            sh[21] = (mine.start >> a.c.page_shift) + (j - first);
        }
        __syncthreads();
        if (j < before + all) {
            s.slot = sh[16]; s.row = sh[17]; s.count = sh[18]; s.start = sh[19]; s.length = sh[20];
            page = sh[21];
            return true;
        }
        before += all;
        __syncthreads();
    }
    return false;
}

template <int kV> __device__ __forceinline__ void store_codes(uint8_t* to, const float* x, float inv, int32_t format) {
    if constexpr (kV == 1) {
        *to = (uint8_t)kv_codes2(x[0] * inv, 0.0f, format);
    } else {
        uint32_t w[kV / 4];
#pragma unroll
        for (int i = 0; i < kV / 4; ++i)
            w[i] = kv_codes2(x[4 * i] * inv, x[4 * i + 1] * inv, format) |
                   (kv_codes2(x[4 * i + 2] * inv, x[4 * i + 3] * inv, format) << 16);
        if constexpr (kV == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(to) = w[0];
    }
}

// NaN becomes 0, an infinity the largest float; the result is the largest magnitude.  One multiply-add an element finds both: x * 0 is
// no number for either.
template <int kN> __device__ __forceinline__ float finite(float* x, bool& odd) {
    float most = 0.0f, zero = 0.0f;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        most = fmaxf(most, fabsf(x[i]));
        zero = fmaf(x[i], 0.0f, zero);
    }
    if (zero != 0.0f) {
        odd = true;
        most = 0.0f;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -3.402823466e38f), 3.402823466e38f);
            most = fmaxf(most, fabsf(x[i]));
        }
    }
    return most;
}

// One block writes the new tokens of one page, keys or values, for all heads.  A head's new tokens have to be seen twice, for their
// largest magnitude and to be quantised: as many warps take a head as hold its tokens in registers, kHold units a thread, and the block
// takes so many heads at a time.  A thread has the same units of every head, so where they lie and their angles are worked out once.
// Larger pages (more than 512 units) are read, and turned, again.
// A row's units: `pairs` pairs of kV elements - the rotated part, or all of a row that is not rotated - then single units of what a
// partial rotation leaves.
template <class T, int kV, bool kPairs>
__device__ void append_page(const AppendArgs& a, uint32_t j, bool keys, uint32_t* sh, float* shf) {
    KvSeq s;
    uint32_t page;
    if (!find_page(a, j, s, page, sh)) return;
    const KvView& c = a.c;
    const uint32_t from = page << c.page_shift;
    const uint32_t pos0 = max(s.start, from), pos1 = min(s.length, from + c.page_tokens);
    const uint32_t tokens = pos1 - pos0, held = pos0 - from, row0 = s.row + (pos0 - s.start);
    const int32_t id = c.pages[(size_t)s.slot * c.max_pages + page];
    if (id < 0 || (uint32_t)id >= c.num_pages || (c.refs && c.refs[id] != 1)) {
        if (threadIdx.x == 0) kv_flag(c.status, ROOMIE_FLAG_KV_PAGE);
        return;
    }
    uint8_t* base = (keys ? c.k : c.v) + (long long)id * c.page_stride;
    float* scale = (keys ? c.k_scale : c.v_scale) + (size_t)id * c.heads;
    const long long x_token = keys ? a.k_token : a.v_token, x_head = keys ? a.k_head : a.v_head;
    const T* x = static_cast<const T*>(keys ? a.k : a.v) + row0 * x_token;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t rot = keys ? a.rope.rot : 0;
    const uint32_t pairs = (rot ? rot : c.dim) / 2 / kV, units = pairs + (rot ? (c.dim - rot) / kV : 0), n = tokens * units;
    const uint32_t mate = kPairs || !rot ? kV : rot / 2;                  // from a unit to the other of its pair
    constexpr int kHold = kV == 1 ? 4 : 1;
    uint32_t warps = 1;                                                   // of a head: a power of two
    while (warps < kAppendWarps && (warps * 32 * kHold < n || kAppendWarps / warps > c.heads)) warps *= 2;
    const uint32_t together = kAppendWarps / warps, group = wid / warps, team = warps * 32;
    const uint32_t me = (wid % warps) * 32 + lane;
    const bool once = n <= team * kHold;
    using Raw = typename std::conditional<kV == 1, T, uint4>::type;
    bool odd = false;

    long long src[kHold];                                                 // elements from x; bytes from the head's part of the page
    uint32_t dst[kHold];
    int kind[kHold];                                                      // 0: nothing, 1: a single, 2: a pair
    float2 w[kHold][kV];
    Raw ra[kHold], rb[kHold];
    float y[kHold][2 * kV];
    auto place = [&](uint32_t i0) {
#pragma unroll
        for (int e = 0; e < kHold; ++e) {
            const uint32_t i = i0 + e * team, t = i / units, u = i - t * units;
            kind[e] = i >= n ? 0 : u >= pairs ? 1 : 2;
            const uint32_t at = u >= pairs ? rot + (u - pairs) * kV : mate == kV ? 2 * u * kV : u * kV;
            src[e] = t * x_token + at;
            dst[e] = (held + t) * c.token_step + at;
            if (rot && kind[e] == 2)
#pragma unroll
                for (int k = 0; k < kV; ++k) w[e][k] = rope_turn(a.rope.frequency[u * kV + k], (int32_t)(pos0 + t), a.rope.amplitude);
        }
    };
    auto fetch = [&](uint32_t h) {                                        // all loads under way together
#pragma unroll
        for (int e = 0; e < kHold; ++e) {
            const T* p = x + h * x_head + src[e];
            if (kind[e]) ra[e] = *reinterpret_cast<const Raw*>(p);
            if (kind[e] == 2) rb[e] = *reinterpret_cast<const Raw*>(p + mate);
        }
    };
    auto widen = [](const Raw& r, float* to) {
        if constexpr (kV == 1) to[0] = to_f32(r);
        else unpack<T>(r, to);
    };
    auto values = [&]() {                                                 // of what was fetched; the result is their largest magnitude
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < kHold; ++e) {
            if (kind[e] == 0) continue;
            widen(ra[e], y[e]);
            if (kind[e] == 2) {
                widen(rb[e], y[e] + kV);
                if (rot) {
                    if constexpr (kPairs && kV > 1) {
#pragma unroll
                        for (int i = 0; i < kV; ++i) {                    // pairs (2i, 2i+1) of the 2*kV elements
                            const float p = y[e][2 * i], q = y[e][2 * i + 1];
                            y[e][2 * i] = __fsub_rn(__fmul_rn(p, w[e][i].x), __fmul_rn(q, w[e][i].y));
                            y[e][2 * i + 1] = __fadd_rn(__fmul_rn(q, w[e][i].x), __fmul_rn(p, w[e][i].y));
                        }
                    } else {
                        rotate_half<kV>(y[e], y[e] + kV, w[e]);
                    }
                }
            } else {
#pragma unroll
                for (int i = kV; i < 2 * kV; ++i) y[e][i] = 0.0f;
            }
            most = fmaxf(most, finite<2 * kV>(y[e], odd));
        }
        return most;
    };

    place(me);
    if (once && group < c.heads) fetch(group);
    for (uint32_t h0 = 0; h0 < c.heads; h0 += together) {
        const uint32_t h = h0 + group;
        const bool on = h < c.heads;
        const float old = on && held ? scale[h] : 0.0f;
        float amax = 0.0f;
        if (on) {
            if (once) {
                amax = values();
            } else {
                for (uint32_t i0 = me; i0 < n; i0 += kHold * team) {
                    place(i0);
                    fetch(h);
                    amax = fmaxf(amax, values());
                }
            }
        }
        if (once && h + together < c.heads) fetch(h + together);          // on their way while this head is finished
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
        __syncthreads();                                                  // shf is free again, and `old` has been read
        if (lane == 0) shf[wid] = amax;
        __syncthreads();
        if (!on) continue;
        for (uint32_t v = 0; v < warps; ++v) amax = fmaxf(amax, shf[group * warps + v]);
        const int ex = kv_scale_exponent(amax, c.format);
        float now = pow2f(ex), inv = pow2f(-ex);
        if (held && old >= now) { now = old; inv = __fdiv_rn(1.0f, old); }
        uint8_t* to = base + h * c.head_step;
        if (held && old < now) {                                          // earlier tokens of the page: to the wider scale
            const float ratio = old * inv;
            for (uint32_t i = me; i < held * (c.dim / 2); i += team) {
                const uint32_t t = i / (c.dim / 2), d = 2 * (i - t * (c.dim / 2));
                uint16_t* code2 = reinterpret_cast<uint16_t*>(to + t * c.token_step + d);
                const uint32_t code = *code2;
                *code2 = (uint16_t)kv_codes2(kv_value(code & 0xff, c.format) * ratio, kv_value(code >> 8, c.format) * ratio, c.format);
            }
        }
        if (me == 0) scale[h] = now;
        for (uint32_t i0 = me; i0 < n; i0 += kHold * team) {
            if (!once) {
                place(i0);
                fetch(h);
                values();
            }
#pragma unroll
            for (int e = 0; e < kHold; ++e) {
                if (kind[e] == 0) continue;
                store_codes<kV>(to + dst[e], y[e], inv, c.format);
                if (kind[e] == 2) store_codes<kV>(to + dst[e] + mate, y[e] + kV, inv, c.format);
            }
        }
    }
    if (odd) kv_flag(c.status, ROOMIE_FLAG_KV_NONFINITE);
}

// The queries, rotated to their rows' positions: thread `i` of those that roomie_rope would take.
template <class T, int kV, bool kPairs>
__device__ void append_queries(const AppendArgs& a, unsigned long long i) {
    if (i >= a.q_threads) return;
    const uint32_t rest = (uint32_t)(i / a.q_units), unit = (uint32_t)(i - (unsigned long long)rest * a.q_units);
    const uint32_t row = rest / a.q_groups, group = rest - row * a.q_groups;
    uint32_t s = row;                                                     // the sequence of this row: the last with offset <= row
    if (a.q_offset) {
        uint32_t lo = 0, hi = a.num_seqs;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (a.q_offset[mid] <= (int32_t)row) lo = mid;
            else hi = mid;
        }
        s = lo;
    }
    int32_t position = 0;
    bool turned = false;
    if (s < a.num_seqs) {
        const KvSeq q = kv_seq(a.c, a.seqs, a.q_offset, a.rows, s, false);
        turned = row >= q.row && row < q.row + q.count && q.count <= q.length;
        if (turned) position = (int32_t)(q.start + (row - q.row));
    }
    // a row of no sequence; a loop of its own, because a condition in the other costs 1.3 us of the 50 that 17000 rows of queries alone take
    if (!turned) return rope_copy<T, kV, kPairs>(a.q, a.rope, row, unit, group, a.q_groups, a.q_heads);
    rope_heads<T, kV, kPairs, kV == 1 ? 1 : 2>(a.q, a.rope, row, position, false, unit, group, a.q_groups, a.q_heads);
}

// Blocks [0, 2 * kv_blocks): page j of the call, keys (even) and values (odd); the rest: queries.  One launch for the three: a decoding
// step's share of each is far below a launch's cost (64 sequences: 13.5 us a call, with the queries in a launch of their own 15.4), and for
// many rows the two would follow each other, because two blocks of keys and values take all of an SM's registers (us, one launch and two;
// 32 query heads on 8, 128 dims, bfloat16, with the queries' MB):
//   rows       512 (4)      2048 (16)    4096 (32)    8192 (64)    17000 (133)
//              18.9 20.5    20.9 24.7    26.7 30.9    45.0 47.1    84.8 87.7
// (Other heads and types: as many rows as leave the last wave of blocks short lose 2 to 18 % by it, 12000 rows win up to 22 %.)
template <class T, int kV, bool kPairs>
__global__ void __launch_bounds__(kAppendThreads, 2) append_kernel(AppendArgs a) {
    __shared__ uint32_t sh[24];
    __shared__ float shf[kAppendWarps];
    if (blockIdx.x < 2 * a.kv_blocks) append_page<T, kV, kPairs>(a, blockIdx.x >> 1, (blockIdx.x & 1) == 0, sh, shf);
    else append_queries<T, kV, kPairs>(a, (unsigned long long)(blockIdx.x - 2 * a.kv_blocks) * kAppendThreads + threadIdx.x);
}

template <class T>
static int launch_append(const AppendArgs& a, bool wide, bool pairs, cudaStream_t st) {
    constexpr int v = kVecOf<T>;
    void (*k)(AppendArgs);
    if (pairs) k = wide ? append_kernel<T, v, true> : append_kernel<T, 1, true>;
    else k = wide ? append_kernel<T, v, false> : append_kernel<T, 1, false>;
    const unsigned long long queries = (a.q_threads + kAppendThreads - 1) / kAppendThreads;
    return launch("kv_append", k, dim3((uint32_t)(2 * a.kv_blocks + queries)), dim3(kAppendThreads), 0, st, false, a);
}

}  // namespace roomie

using namespace roomie;

extern "C" int roomie_kv_append(const roomie_kv_cache* cache, uint32_t layer, const int32_t* seqs, uint32_t num_seqs,
                                const int32_t* q_offset, uint32_t rows, const roomie_rows* k, const roomie_rows* v,
                                const roomie_rope_table* rope, uint32_t q_heads, const roomie_rows* q, const roomie_rows* q_out,
                                void* stream) {
    if (kv_check(cache) != ROOMIE_OK || layer >= cache->layers) return ROOMIE_ERR_INVALID_ARG;
    if (num_seqs == 0 || rows == 0) return ROOMIE_OK;
    if (!rows_valid(k) || !rows_valid(v) || k->type != v->type)
        return ROOMIE_ERR_INVALID_ARG;
    if (rope && !rope_table_valid(rope, cache->head_dim)) return ROOMIE_ERR_INVALID_ARG;
    if ((q != nullptr) != (q_out != nullptr)) return ROOMIE_ERR_INVALID_ARG;
    if (q && (!rope || q_heads == 0 || !rows_valid(q) || !rows_valid(q_out) || q->type != q_out->type || q->type != k->type ||
              !rows_apart(*q_out, rows, q_heads, cache->head_dim) ||
              (q->data == q_out->data && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride))))
        return ROOMIE_ERR_INVALID_ARG;
    if (!seqs || (!q_offset && rows != num_seqs) || rows > 0x3fffffffu || num_seqs > 0x3fffffffu ||
        (q && (unsigned long long)rows * q_heads > 0x7fffffffull))
        return ROOMIE_ERR_INVALID_ARG;
    AppendArgs a = {};
    a.c = kv_view(cache, layer);
    a.seqs = seqs; a.q_offset = q_offset; a.num_seqs = num_seqs; a.rows = rows;
    a.k = k->data; a.v = v->data;
    a.k_token = k->token_stride; a.k_head = k->head_stride; a.v_token = v->token_stride; a.v_head = v->head_stride;
    bool wide = rows_aligned16(*k, rows, cache->kv_heads) && rows_aligned16(*v, rows, cache->kv_heads);
    if (rope) {
        a.rope = {rope->frequency, rope->rotary_dim, rope->interleaved, rope->amplitude};
        wide = wide && rope_units_of_16(rope->rotary_dim, cache->head_dim, k->type, rope->interleaved);
    }
    // pages touched: at most one per page_tokens rows and two more for each sequence; never more than rows
    unsigned long long blocks = rows / cache->page_tokens + 2ull * num_seqs;
    if (blocks > rows) blocks = rows;
    a.kv_blocks = (uint32_t)blocks;
    unsigned long long q_blocks = 0;
    if (q) {
        a.q = {q->data, q_out->data, q->token_stride, q->head_stride, q_out->token_stride, q_out->head_stride};
        a.q_heads = q_heads;
        wide = wide && rows_aligned16(*q, rows, q_heads) && rows_aligned16(*q_out, rows, q_heads);
        const RopeSplit s = rope_split(rows, q_heads, cache->head_dim, rope->rotary_dim, wide ? 16u / (uint32_t)size_of_type(k->type) : 1u,
                                       q->data == q_out->data, (uint32_t)sm_count());
        a.q_units = s.units; a.q_groups = s.groups; a.q_threads = s.threads;
        q_blocks = (s.threads + kAppendThreads - 1) / kAppendThreads;
    }
    if (q_blocks + 2ull * a.kv_blocks > 0x7fffffffull) return ROOMIE_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool pairs = rope && rope->interleaved;
    if (k->type == ROOMIE_F32) return launch_append<float>(a, wide, pairs, st);
    if (k->type == ROOMIE_F16) return launch_append<__half>(a, wide, pairs, st);
    return launch_append<__nv_bfloat16>(a, wide, pairs, st);
}
