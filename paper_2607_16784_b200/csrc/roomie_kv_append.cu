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
    uint32_t q_heads, q_per_block, kv_blocks;
    int32_t q_in_place;
};

constexpr int kAppendThreads = 256, kAppendWarps = kAppendThreads / 32;

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
            sh[8] = mine.slot; sh[9] = mine.row; sh[10] = mine.count; sh[11] = mine.start; sh[12] = mine.length;
            sh[13] = (mine.start >> a.c.page_shift) + (j - first);
        }
        __syncthreads();
        if (j < before + all) {
            s.slot = sh[8]; s.row = sh[9]; s.count = sh[10]; s.start = sh[11]; s.length = sh[12];
            page = sh[13];
            return true;
        }
        before += all;
        __syncthreads();
    }
    return false;
}

// Loads unit `unit` of (row, head) as float32 - rotated pairs first, then the copied part - into x[0..kV) and, for a rotated
// unit, x[kV..2kV); at[] are the elements they belong at.
template <class T, int kV, bool kPairs>
__device__ __forceinline__ bool load_unit(const T* p, uint32_t unit, uint32_t rot, const float2* cs, float* x, uint32_t* at) {
    const uint32_t half = rot / 2, n_rot = half / kV;
    using Raw = typename std::conditional<kV == 1, T, uint4>::type;
    auto get = [](const T* from, float* to) {
        const Raw r = *reinterpret_cast<const Raw*>(from);
        if constexpr (kV == 1) to[0] = to_f32(r);
        else unpack<T>(r, to);
    };
    if (unit >= n_rot) {
        at[0] = rot + (unit - n_rot) * kV;
        get(p + at[0], x);
        return false;
    }
    at[0] = kPairs ? 2 * unit * kV : unit * kV;
    at[1] = kPairs ? at[0] + kV : at[0] + half;
    get(p + at[0], x);
    get(p + at[1], x + kV);
    const float2* w = cs + unit * kV;
    if constexpr (kPairs && kV > 1) {
#pragma unroll
        for (int i = 0; i < kV; ++i) {                                    // pairs (2i, 2i+1) of the 2*kV elements
            const float e = x[2 * i], o = x[2 * i + 1];
            x[2 * i] = __fsub_rn(__fmul_rn(e, w[i].x), __fmul_rn(o, w[i].y));
            x[2 * i + 1] = __fadd_rn(__fmul_rn(o, w[i].x), __fmul_rn(e, w[i].y));
        }
    } else {
        rotate_half<kV>(x, x + kV, w);
    }
    return true;
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

// finite magnitude of a value; NaN becomes 0, an infinity the largest float
__device__ __forceinline__ float finite(float x, bool& odd) {
    if (fabsf(x) <= 3.402823466e38f) return x;
    odd = true;
    return x != x ? 0.0f : copysignf(3.402823466e38f, x);
}

// One block writes the new tokens of one page, keys or values, for all heads.  Groups of warps take a head each: a first pass
// over the head's new tokens finds the largest magnitude, a second one quantises (it reads the tokens again, from L1/L2: a page's
// tokens of one head are 4 to 64 KB, too much for registers in general).
template <class T, int kV, bool kPairs>
__device__ void append_page(const AppendArgs& a, uint32_t j, bool keys, float2* cs, uint32_t* sh, float* shf) {
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
    const uint32_t rot = keys ? a.rope.rot : 0, half = rot / 2;
    for (uint32_t i = threadIdx.x; i < tokens * half; i += kAppendThreads) {
        const uint32_t t = i / half, p = i - t * half;
        cs[i] = rope_turn(a.rope.frequency[p], (int32_t)(pos0 + t), a.rope.amplitude);
    }
    uint8_t* base = (keys ? c.k : c.v) + (long long)id * c.page_stride;
    float* scale = (keys ? c.k_scale : c.v_scale) + (size_t)id * c.heads;
    const T* x = static_cast<const T*>(keys ? a.k : a.v);
    const long long x_token = keys ? a.k_token : a.v_token, x_head = keys ? a.k_head : a.v_head;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    uint32_t together = 1;                                                // heads at a time: a power of two
    while (together * 2 <= c.heads && together < kAppendWarps) together *= 2;
    const uint32_t warps = kAppendWarps / together, group = wid / warps, team = warps * 32;
    const uint32_t me = (wid % warps) * 32 + lane;
    const uint32_t units = half / kV + (c.dim - rot) / kV;
    bool odd = false;
    for (uint32_t h0 = 0; h0 < c.heads; h0 += together) {
        const uint32_t h = h0 + group;
        const bool on = h < c.heads;
        __syncthreads();                                                  // cs is written; shf is free again
        const float old = on && held ? scale[h] : 0.0f;
        float amax = 0.0f;
        if (on)
            for (uint32_t i = me; i < tokens * units; i += team) {
                const uint32_t t = i / units, u = i - t * units;
                float y[2 * kV];
                uint32_t at[2];
                const bool two = load_unit<T, kV, kPairs>(x + (row0 + t) * x_token + h * x_head, u, rot, cs + (size_t)t * half, y, at);
#pragma unroll
                for (int e = 0; e < kV; ++e) amax = fmaxf(amax, fabsf(finite(y[e], odd)));
                if (two)
#pragma unroll
                    for (int e = kV; e < 2 * kV; ++e) amax = fmaxf(amax, fabsf(finite(y[e], odd)));
            }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, d));
        if (lane == 0) shf[wid] = amax;
        __syncthreads();
        if (!on) continue;
        for (uint32_t w = 0; w < warps; ++w) amax = fmaxf(amax, shf[group * warps + w]);
        const int e = kv_scale_exponent(amax, c.format);
        float now = pow2f(e), inv = pow2f(-e);
        if (held && old >= now) { now = old; inv = __fdiv_rn(1.0f, old); }
        uint8_t* to = base + h * c.head_step;
        if (held && old < now) {                                          // earlier tokens of the page: to the wider scale
            const float ratio = old * inv;
            for (uint32_t i = me; i < held * (c.dim / 2); i += team) {
                const uint32_t t = i / (c.dim / 2), d = 2 * (i - t * (c.dim / 2));
                uint16_t* w = reinterpret_cast<uint16_t*>(to + t * c.token_step + d);
                const uint32_t code = *w;
                *w = (uint16_t)kv_codes2(kv_value(code & 0xff, c.format) * ratio, kv_value(code >> 8, c.format) * ratio, c.format);
            }
        }
        if (me == 0) scale[h] = now;
        for (uint32_t i = me; i < tokens * units; i += team) {
            const uint32_t t = i / units, u = i - t * units;
            float y[2 * kV];
            uint32_t at[2];
            const bool two = load_unit<T, kV, kPairs>(x + (row0 + t) * x_token + h * x_head, u, rot, cs + (size_t)t * half, y, at);
            uint8_t* q = to + (held + t) * c.token_step;
#pragma unroll
            for (int e2 = 0; e2 < kV; ++e2) y[e2] = finite(y[e2], odd);
            store_codes<kV>(q + at[0], y, inv, c.format);
            if (two) {
#pragma unroll
                for (int e2 = kV; e2 < 2 * kV; ++e2) y[e2] = finite(y[e2], odd);
                store_codes<kV>(q + at[1], y + kV, inv, c.format);
            }
        }
    }
    if (odd) kv_flag(c.status, ROOMIE_FLAG_KV_NONFINITE);
}

// The queries of q_per_block consecutive rows, rotated to their positions.
template <class T, int kV, bool kPairs>
__device__ void append_queries(const AppendArgs& a, uint32_t block, float2* cs, int32_t* pos) {
    const uint32_t first = block * a.q_per_block, tokens = min(a.q_per_block, a.rows - first), half = a.rope.rot / 2;
    if (threadIdx.x < tokens) {
        const uint32_t row = first + threadIdx.x;
        uint32_t i = row;                                                 // the sequence of this row: the last with offset <= row
        if (a.q_offset) {
            uint32_t lo = 0, hi = a.num_seqs;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) / 2;
                if (a.q_offset[mid] <= (int32_t)row) lo = mid;
                else hi = mid;
            }
            i = lo;
        }
        int32_t p = -1;
        if (i < a.num_seqs) {
            const KvSeq s = kv_seq(a.c, a.seqs, a.q_offset, a.rows, i, false);
            if (row >= s.row && row < s.row + s.count && s.count <= s.length) p = (int32_t)(s.start + (row - s.row));
        }
        pos[threadIdx.x] = p;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < tokens * half; i += kAppendThreads) {
        const uint32_t t = i / half, p = i - t * half;
        // a row that belongs to no sequence is passed on unturned
        cs[i] = pos[t] < 0 ? make_float2(1.0f, 0.0f) : rope_turn(a.rope.frequency[p], pos[t], a.rope.amplitude);
    }
    __syncthreads();
    rope_block<T, kV, kPairs, kV == 1 ? 1 : 4>(a.q, cs, first, tokens, a.q_heads, a.c.dim, a.rope.rot, a.q_in_place != 0);
}

// Blocks [0, 2 * kv_blocks): page j of the call, keys (even) and values (odd); the rest: queries.  One launch for the three, because
// a decoding step's share of each is far below a launch's cost.
template <class T, int kV, bool kPairs>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs a) {
    extern __shared__ float2 cs[];
    __shared__ uint32_t sh[16];
    __shared__ float shf[kAppendWarps];
    if (blockIdx.x < 2 * a.kv_blocks) append_page<T, kV, kPairs>(a, blockIdx.x >> 1, (blockIdx.x & 1) == 0, cs, sh, shf);
    else append_queries<T, kV, kPairs>(a, blockIdx.x - 2 * a.kv_blocks, cs, reinterpret_cast<int32_t*>(sh));
}

template <class T>
static int launch_append(const AppendArgs& a, bool wide, bool pairs, dim3 grid, size_t smem, cudaStream_t st) {
    constexpr int v = kVecOf<T>;
    void (*k)(AppendArgs);
    if (pairs) k = wide ? append_kernel<T, v, true> : append_kernel<T, 1, true>;
    else k = wide ? append_kernel<T, v, false> : append_kernel<T, 1, false>;
    return launch("kv_append", k, grid, dim3(kAppendThreads), smem, st, false, a);
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
    uint32_t q_blocks = 0;
    if (q) {
        a.q = {q->data, q_out->data, q->token_stride, q->head_stride, q_out->token_stride, q_out->head_stride};
        a.q_heads = q_heads;
        a.q_in_place = q->data == q_out->data;
        wide = wide && rows_aligned16(*q, rows, q_heads) && rows_aligned16(*q_out, rows, q_heads);
        const uint32_t full = (uint32_t)sm_count() * 8;
        a.q_per_block = rows / full < 1 ? 1 : rows / full > 8 ? 8 : rows / full;
        q_blocks = (rows + a.q_per_block - 1) / a.q_per_block;
    }
    const uint32_t half = rope ? rope->rotary_dim / 2 : 0;
    const uint32_t most = cache->page_tokens < rows ? cache->page_tokens : rows;
    const size_t smem = (size_t)(most > a.q_per_block ? most : a.q_per_block) * half * sizeof(float2);
    if (smem > 200 * 1024) return ROOMIE_ERR_CAPACITY;
    const dim3 grid(2 * a.kv_blocks + q_blocks);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool pairs = rope && rope->interleaved;
    if (k->type == ROOMIE_F32) return launch_append<float>(a, wide, pairs, grid, smem, st);
    if (k->type == ROOMIE_F16) return launch_append<__half>(a, wide, pairs, grid, smem, st);
    return launch_append<__nv_bfloat16>(a, wide, pairs, grid, smem, st);
}
