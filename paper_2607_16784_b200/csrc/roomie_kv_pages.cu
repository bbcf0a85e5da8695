// Page operations of the 8-bit cache: reserve, fork, free, copy, compact.
#include "roomie_kv_pages.cuh"

namespace roomie {

int kv_check(const roomie_kv_cache* c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->refs || !c->pages || !c->length || !c->status)
        return ROOMIE_ERR_INVALID_ARG;
    if (c->layers == 0 || c->num_pages == 0 || c->kv_heads == 0 || c->max_seqs == 0 || c->max_pages == 0 ||
        c->num_pages > 0x7fffffffu || c->max_seqs > 0x7fffffffu || c->kv_heads > 65535u ||
        (unsigned long long)c->max_pages * 128u > 0x7fffffffull)
        return ROOMIE_ERR_INVALID_ARG;
    const uint32_t t = c->page_tokens;
    if ((t != 16 && t != 32 && t != 64 && t != 128) || c->head_dim == 0 || c->head_dim % 16 || c->head_dim > 256)
        return ROOMIE_ERR_INVALID_ARG;
    if ((c->format != ROOMIE_KV_E4M3 && c->format != ROOMIE_KV_INT8) || (c->layout != ROOMIE_KV_HND && c->layout != ROOMIE_KV_NHD))
        return ROOMIE_ERR_INVALID_ARG;
    const long long page = (long long)t * c->kv_heads * c->head_dim;
    if (((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15u) || c->page_stride % 16 || c->layer_stride % 16 ||
        (c->num_pages > 1 && c->page_stride < page) || (c->layers > 1 && c->layer_stride < page) || page > 0x7fffffffll)
        return ROOMIE_ERR_INVALID_ARG;
    return ROOMIE_OK;
}

KvView kv_view(const roomie_kv_cache* c, uint32_t layer) {
    KvView v;
    v.k = static_cast<uint8_t*>(c->k) + layer * c->layer_stride;
    v.v = static_cast<uint8_t*>(c->v) + layer * c->layer_stride;
    const size_t scales = (size_t)layer * c->num_pages * c->kv_heads;
    v.k_scale = c->k_scale + scales;
    v.v_scale = c->v_scale + scales;
    v.refs = c->refs; v.pages = c->pages; v.length = c->length; v.status = c->status;
    v.page_stride = c->page_stride;
    v.num_pages = c->num_pages; v.page_tokens = c->page_tokens;
    v.page_shift = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
    v.heads = c->kv_heads; v.dim = c->head_dim; v.max_seqs = c->max_seqs; v.max_pages = c->max_pages;
    v.format = c->format;
    const bool hnd = c->layout == ROOMIE_KV_HND;
    v.token_step = hnd ? c->head_dim : c->head_dim * c->kv_heads;
    v.head_step = hnd ? c->head_dim * c->page_tokens : c->head_dim;
    return v;
}

// ---- moving pages ----------------------------------------------------------------------------------------------------
// A page of one layer is one run of bytes for keys and one for values, plus a row of scales for each.
struct CopyArgs {
    const uint8_t *sk, *sv;
    uint8_t *dk, *dv;
    const float *sks, *svs;
    float *dks, *dvs;
    long long s_layer, s_page, d_layer, d_page;
    uint32_t layers, heads, s_pages, d_pages;
    uint32_t bytes;                      // of a page of one layer, keys or values: a multiple of 256
    uint32_t n;                          // pairs, or the most of them when `count` is given
    const int32_t *src, *dst, *count;    // pair i: src[i] -> dst[i]; a pair of -1 is skipped
    uint32_t* status;
};

// Bound by memory: each unit is up to 16 KB of one run, 256 threads with four 128-bit loads in flight each, past the caches' reuse; up to
// four times the blocks that fit at once, so that the last ones end together (1.35 GB moved: 221 us, with one round of blocks 242).
constexpr uint32_t kCopyUnit = 16384;
__device__ void copy_pages(const CopyArgs& a, unsigned long long worker, unsigned long long workers) {
    const uint32_t n = a.count ? min((uint32_t)max(*a.count, 0), a.n) : a.n;
    const uint32_t parts = (a.bytes + kCopyUnit - 1) / kCopyUnit, per_pair = a.layers * 2 * parts;
    const unsigned long long units = (unsigned long long)n * per_pair;
    for (unsigned long long u = worker; u < units; u += workers) {
        const uint32_t i = (uint32_t)(u / per_pair), r = (uint32_t)(u - (unsigned long long)i * per_pair);
        const uint32_t part = r % parts, side = (r / parts) & 1, layer = r / parts / 2;
        const int32_t from = a.src[i], to = a.dst[i];
        if (from == -1 && to == -1) continue;
        if (from < 0 || to < 0 || (uint32_t)from >= a.s_pages || (uint32_t)to >= a.d_pages) {
            if (threadIdx.x == 0) kv_flag(a.status, ROOMIE_FLAG_KV_PAGE);
            continue;
        }
        const uint32_t begin = part * kCopyUnit, len = min(kCopyUnit, a.bytes - begin);
        const uint4* s = reinterpret_cast<const uint4*>((side ? a.sv : a.sk) + layer * a.s_layer + from * a.s_page + begin);
        uint4* d = reinterpret_cast<uint4*>((side ? a.dv : a.dk) + layer * a.d_layer + to * a.d_page + begin);
        const uint32_t vecs = len / 16;
        uint4 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (threadIdx.x + e * 256 < vecs) x[e] = __ldcs(s + threadIdx.x + e * 256);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (threadIdx.x + e * 256 < vecs) __stcs(d + threadIdx.x + e * 256, x[e]);
        if (part == 0) {
            const float* ss = (side ? a.svs : a.sks) + ((size_t)layer * a.s_pages + from) * a.heads;
            float* ds = (side ? a.dvs : a.dks) + ((size_t)layer * a.d_pages + to) * a.heads;
            for (uint32_t h = threadIdx.x; h < a.heads; h += 256) ds[h] = ss[h];
        }
    }
}

__global__ void __launch_bounds__(256) copy_kernel(CopyArgs a) { copy_pages(a, blockIdx.x, gridDim.x); }

static CopyArgs copy_args(const roomie_kv_cache* s, const roomie_kv_cache* d) {
    CopyArgs a = {};
    a.sk = static_cast<const uint8_t*>(s->k); a.sv = static_cast<const uint8_t*>(s->v);
    a.dk = static_cast<uint8_t*>(d->k); a.dv = static_cast<uint8_t*>(d->v);
    a.sks = s->k_scale; a.svs = s->v_scale; a.dks = d->k_scale; a.dvs = d->v_scale;
    a.s_layer = s->layer_stride; a.s_page = s->page_stride; a.d_layer = d->layer_stride; a.d_page = d->page_stride;
    a.layers = s->layers; a.heads = s->kv_heads; a.s_pages = s->num_pages; a.d_pages = d->num_pages;
    a.bytes = s->page_tokens * s->kv_heads * s->head_dim;
    a.status = d->status;
    return a;
}
static uint32_t copy_blocks(const CopyArgs& a, unsigned long long pairs) {
    const unsigned long long units = pairs * a.layers * 2 * ((a.bytes + kCopyUnit - 1) / kCopyUnit);
    const unsigned long long full = (unsigned long long)sm_count() * 32;
    return (uint32_t)(units < 1 ? 1 : units < full ? units : full);
}

// ---- reserve and fork --------------------------------------------------------------------------------------------------
// Workspace of n requests: need, first (n words each), the list of free pages (num_pages), refused (n).
__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(TableView t, const int32_t* seqs, const int32_t* want, uint32_t n,
                                                               int32_t* ws) {
    __shared__ uint32_t sh[kPlanWarps];
    int32_t *need = ws, *first = ws + n, *list = ws + 2 * n;
    uint32_t bad = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const int32_t s = seqs[i], len = length_of(t, s), w = want[i];
        int32_t x = -1;
        if (len >= 0 && w >= len && (unsigned long long)w <= ((unsigned long long)t.max_pages << t.page_shift)) {
            const uint32_t have = pages_of(t, (uint32_t)len), all = pages_of(t, (uint32_t)w);
            x = (int32_t)(all - have);
            // a sequence named twice: the first request in order claims its first new entry
            if (x) atomicMin(reinterpret_cast<uint32_t*>(t.pages) + (size_t)s * t.max_pages + have, i);
        } else {
            bad |= ROOMIE_FLAG_KV_SEQUENCE;
        }
        need[i] = x;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        first[i] = need[i];                                       // -1: refused
        if (need[i] > 0) {
            const int32_t s = seqs[i];
            const uint32_t have = pages_of(t, (uint32_t)t.length[s]);
            if ((uint32_t)t.pages[(size_t)s * t.max_pages + have] != i) {
                need[i] = 0;
                first[i] = -1;
                bad |= ROOMIE_FLAG_KV_SEQUENCE;
            }
        } else {
            need[i] = 0;
        }
    }
    __syncthreads();
    int32_t* refused = list + t.num_pages;                        // -1: refused (serve writes all of `first`)
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) refused[i] = first[i];
    __syncthreads();
    const uint32_t found = serve(t, n, need, first, list, t.num_pages, sh);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        if (refused[i] < 0) continue;
        const int32_t s = seqs[i];
        const uint32_t x = (uint32_t)need[i], at = (uint32_t)first[i];
        int32_t* row = t.pages + (size_t)s * t.max_pages;
        const uint32_t have = pages_of(t, (uint32_t)want[i]) - x;
        if (x && (unsigned long long)at + x > found) {
            bad |= ROOMIE_FLAG_KV_FULL;
            row[have] = -1;                                       // the claim is given back
            continue;
        }
        for (uint32_t e = 0; e < x; ++e) {
            row[have + e] = list[at + e];
            t.refs[list[at + e]] = 1;
        }
        atomicMax(t.length + s, want[i]);
    }
    if (bad) kv_flag(t.status, bad);
}

// Workspace of n requests: need, first, src, dst, len (n words each), the list of free pages (n).
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(TableView t, const int32_t* parents, const int32_t* children,
                                                                 uint32_t n, int32_t* ws) {
    __shared__ uint32_t sh[kPlanWarps];
    int32_t *need = ws, *first = ws + n, *src = ws + 2 * n, *dst = ws + 3 * n, *len = ws + 4 * n, *list = ws + 5 * n;
    const uint32_t inside = (1u << t.page_shift) - 1;
    uint32_t bad = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const int32_t p = parents[i], c = children[i], l = length_of(t, p);
        const bool ok = l >= 0 && slot_ok(t, c) && c != p && t.length[c] == 0;
        len[i] = ok ? l : -1;
        if (ok) atomicMin(reinterpret_cast<uint32_t*>(t.pages) + (size_t)c * t.max_pages, i);   // an empty child's first entry is -1
        else bad |= ROOMIE_FLAG_KV_SEQUENCE;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        if (len[i] >= 0 && (uint32_t)t.pages[(size_t)children[i] * t.max_pages] != i) {          // a child named before, or not empty
            len[i] = -1;
            bad |= ROOMIE_FLAG_KV_SEQUENCE;
        }
        need[i] = len[i] > 0 && ((uint32_t)len[i] & inside) ? 1 : 0;
    }
    __syncthreads();
    const uint32_t found = serve(t, n, need, first, list, min(n, t.num_pages), sh);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        src[i] = dst[i] = -1;
        if (len[i] < 0) continue;
        if (need[i]) {
            if ((uint32_t)first[i] >= found) {
                bad |= ROOMIE_FLAG_KV_FULL;
                t.pages[(size_t)children[i] * t.max_pages] = -1;
                len[i] = -1;
                continue;
            }
            src[i] = t.pages[(size_t)parents[i] * t.max_pages + ((uint32_t)len[i] >> t.page_shift)];
            dst[i] = list[first[i]];
            t.refs[dst[i]] = 1;
        }
        if (len[i] == 0) t.pages[(size_t)children[i] * t.max_pages] = -1;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads)
        if (len[i] >= 0) t.length[children[i]] = len[i];
    if (bad) kv_flag(t.status, bad);
}

// Blocks [0, n): the table row of one child; the rest: the part-filled pages.
__global__ void __launch_bounds__(256) fork_move_kernel(TableView t, const int32_t* parents, const int32_t* children, uint32_t n,
                                                        const int32_t* ws, CopyArgs copy) {
    grid_dependency_wait();                                       // the plan; this kernel's start overlaps its end
    if (blockIdx.x >= n) {
        copy_pages(copy, blockIdx.x - n, gridDim.x - n);
        return;
    }
    const uint32_t i = blockIdx.x;
    const int32_t len = ws[4 * n + i], fresh = ws[3 * n + i];
    if (len <= 0) return;
    const uint32_t held = pages_of(t, (uint32_t)len);
    const int32_t* from = t.pages + (size_t)parents[i] * t.max_pages;
    int32_t* to = t.pages + (size_t)children[i] * t.max_pages;
    for (uint32_t e = threadIdx.x; e < held; e += 256) {
        int32_t id = from[e];
        if (e + 1 == held && fresh >= 0) id = fresh;
        else if (id >= 0 && (uint32_t)id < t.num_pages) atomicAdd(t.refs + id, 1);
        else kv_flag(t.status, ROOMIE_FLAG_KV_PAGE);
        to[e] = id;
    }
}

// One warp a sequence.  A sequence named twice is empty the second time.
__global__ void __launch_bounds__(128) free_kernel(TableView t, const int32_t* seqs, uint32_t n) {
    const uint32_t i = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (i >= n) return;
    const int32_t s = seqs[i];
    if (!slot_ok(t, s)) {
        if (lane == 0) kv_flag(t.status, ROOMIE_FLAG_KV_SEQUENCE);
        return;
    }
    int32_t len = 0;
    if (lane == 0) len = atomicExch(t.length + s, 0);
    len = __shfl_sync(0xffffffffu, len, 0);
    if (len < 0 || (unsigned long long)len > ((unsigned long long)t.max_pages << t.page_shift)) {
        if (lane == 0) kv_flag(t.status, ROOMIE_FLAG_KV_SEQUENCE);
        return;
    }
    int32_t* row = t.pages + (size_t)s * t.max_pages;
    const uint32_t held = pages_of(t, (uint32_t)len);
    for (uint32_t e = lane; e < held; e += 32) {
        const int32_t id = row[e];
        row[e] = -1;
        if (id < 0 || (uint32_t)id >= t.num_pages) {
            kv_flag(t.status, ROOMIE_FLAG_KV_PAGE);
        } else if (atomicSub(t.refs + id, 1) <= 0) {
            atomicAdd(t.refs + id, 1);
            kv_flag(t.status, ROOMIE_FLAG_KV_PAGE);
        }
    }
}

// ---- reorder -----------------------------------------------------------------------------------------------------------
// Workspace of n sequences: 16 words, the first of them the widest row in use (-1: the call changes nothing); length, children, first child,
// src, dst, the list of free pages (n words each), and the claims of max_seqs slots.
struct ReorderView {
    int32_t *widest, *len, *count, *first, *src, *dst, *list, *owner;
};
__host__ __device__ __forceinline__ ReorderView reorder_view(int32_t* ws, uint32_t n) {
    int32_t* at = ws + 16;
    return {ws, at, at + n, at + 2 * (size_t)n, at + 3 * (size_t)n, at + 4 * (size_t)n, at + 5 * (size_t)n, at + 6 * (size_t)n};
}
constexpr uint32_t kReorderMost = 8192;                           // sequences of a call: a column of their rows fits shared memory

// The table's entries of the call's sequences, a sequence by a warp: `f(page, more)`, more: how many holders the page gets beyond the one that it has here.  A whole
// page has one for each child; the part-filled last page goes to the first child, and is given up when there is none.  kChanging: of the sequences alone
// where that changes anything.
template <bool kChanging, class F> __device__ __forceinline__ void held_pages(const TableView& t, const int32_t* seqs, uint32_t n, const ReorderView& v, F f) {
    const uint32_t lane = threadIdx.x & 31;
    for (uint32_t base = threadIdx.x >> 5; base < n; base += 32 * kPlanWarps) {      // 32 sequences of a warp at a time: a lane asks for each
        const uint32_t mine = base + lane * kPlanWarps;
        const int32_t my_len = mine < n ? v.len[mine] : 0, my_children = mine < n ? v.count[mine] : 0, my_slot = mine < n ? seqs[mine] : 0;
        for (uint32_t i = 0; i < 32 && base + i * kPlanWarps < n; ++i) {
            const int32_t len = __shfl_sync(0xffffffffu, my_len, i), children = __shfl_sync(0xffffffffu, my_children, i);
            const int32_t slot = __shfl_sync(0xffffffffu, my_slot, i);
            if (len <= 0 || (kChanging && children == 1)) continue;
            const uint32_t held = pages_of(t, (uint32_t)len), whole = (uint32_t)len >> t.page_shift;
            const int32_t* row = t.pages + (size_t)slot * t.max_pages;
            for (uint32_t e0 = 0; e0 < held; e0 += 128) {                            // four entries of a lane under way
                int32_t id[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) id[k] = e0 + 32 * k + lane < held ? row[e0 + 32 * k + lane] : 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t e = e0 + 32 * k + lane;
                    if (e < held) f(id[k], e < whole ? children - 1 : children ? 0 : -1);
                }
            }
        }
    }
}

// One block, for the counts' sake: they are changed, looked at, and taken back where the whole does not fit.  Bound by latency: 32 x 8 beams of 2248
// tokens take 20 us, most of it the pass over the pages that change holders and the one that looks at all.
__global__ void __launch_bounds__(kPlanThreads) reorder_plan_kernel(TableView t, const int32_t* seqs, const int32_t* parents, uint32_t n, int32_t* ws) {
    __shared__ uint32_t sh[kPlanWarps], widest;
    const ReorderView v = reorder_view(ws, n);
    const uint32_t inside = (1u << t.page_shift) - 1;
    if (threadIdx.x == 0) widest = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        if (slot_ok(t, seqs[i])) v.owner[seqs[i]] = 0x7fffffff;
        v.count[i] = 0;
        v.first[i] = 0x7fffffff;
        v.src[i] = v.dst[i] = -1;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads)
        if (slot_ok(t, seqs[i])) atomicMin(v.owner + seqs[i], (int32_t)i);
    __syncthreads();
    uint32_t bad = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const int32_t p = parents[i];
        v.len[i] = length_of(t, seqs[i]);
        if (v.len[i] < 0 || v.owner[seqs[i]] != (int32_t)i || p < -1 || p >= (int32_t)n) {
            bad |= ROOMIE_FLAG_KV_SEQUENCE;
        } else if (p >= 0) {
            atomicAdd(v.count + p, 1);
            atomicMin(v.first + p, (int32_t)i);
        }
    }
    bool refused = __syncthreads_or(bad) != 0;
    if (!refused) {
        held_pages<true>(t, seqs, n, v, [&](int32_t id, int32_t more) {
            if (more && (uint32_t)id < t.num_pages) atomicAdd(t.refs + id, more);
        });
        __syncthreads();
        // Every entry is a page, and counts for what this sequence hands on, so that none of them is among the free ones below.
        held_pages<false>(t, seqs, n, v, [&](int32_t id, int32_t more) {
            if ((uint32_t)id >= t.num_pages || t.refs[id] < more + 1) bad |= ROOMIE_FLAG_KV_PAGE;
        });
        const bool broken = __syncthreads_or(bad) != 0;
        // copies of part-filled pages, in order, to the lowest pages that are free now
        uint32_t copies = 0;
        for (uint32_t base = 0; base < n; base += kPlanThreads) {
            const uint32_t i = base + threadIdx.x;
            const int32_t p = i < n ? parents[i] : -1;
            const uint32_t copy = p >= 0 && v.len[p] > 0 && ((uint32_t)v.len[p] & inside) && v.first[p] != (int32_t)i;
            uint32_t all;
            const uint32_t at = copies + block_exclusive(copy, all, sh);
            if (copy) v.dst[i] = (int32_t)at;
            copies += all;
        }
        const uint32_t found = broken ? 0u : lowest_free(t.refs, t.num_pages, copies, v.list, sh);
        __syncthreads();
        refused = broken || found < copies;
        if (refused) {                                            // as it was
            if (!broken) bad |= ROOMIE_FLAG_KV_FULL;
            held_pages<true>(t, seqs, n, v, [&](int32_t id, int32_t more) {
                if (more && (uint32_t)id < t.num_pages) atomicSub(t.refs + id, more);
            });
        }
    }
    if (bad) kv_flag(t.status, bad);
    __syncthreads();
    if (refused) {
        if (threadIdx.x == 0) *v.widest = -1;
        return;
    }
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const int32_t p = parents[i];
        t.length[seqs[i]] = p < 0 ? 0 : v.len[p];
        atomicMax(&widest, pages_of(t, (uint32_t)v.len[i]));
        if (v.dst[i] >= 0) {
            v.src[i] = t.pages[(size_t)seqs[p] * t.max_pages + ((uint32_t)v.len[p] >> t.page_shift)];
            v.dst[i] = v.list[v.dst[i]];
            t.refs[v.dst[i]] = 1;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) *v.widest = (int32_t)widest;
}

// The first blocks: columns of the table, `columns` of them at a time: a column's entries depend on nothing but the same column.  The rest: the
// part-filled pages: 16 layers of 32 x 8 beams take 42 us behind the plan, bound by memory.
__global__ void __launch_bounds__(256) reorder_move_kernel(TableView t, const int32_t* seqs, const int32_t* parents, uint32_t n, int32_t* ws, uint32_t columns,
                                                           uint32_t table_blocks, CopyArgs copy) {
    extern __shared__ int32_t was[];                              // [n][columns]
    grid_dependency_wait();                                       // the plan; this kernel's start overlaps its end
    const ReorderView v = reorder_view(ws, n);
    const int32_t widest = *v.widest;
    if (widest < 0) return;
    if (blockIdx.x >= table_blocks) {
        copy_pages(copy, blockIdx.x - table_blocks, gridDim.x - table_blocks);
        return;
    }
    const uint32_t entries = n * columns, c = threadIdx.x % columns;       // `columns` divides the block
    for (uint32_t c0 = blockIdx.x * columns; c0 < (uint32_t)widest; c0 += table_blocks * columns) {
        const uint32_t e = c0 + c;
        for (uint32_t x = threadIdx.x; x < entries; x += 256)
            if (e < t.max_pages) was[x] = t.pages[(size_t)seqs[x / columns] * t.max_pages + e];
        __syncthreads();
        for (uint32_t x = threadIdx.x; x < entries; x += 256) {
            const uint32_t i = x / columns;
            const int32_t p = parents[i], fresh = v.dst[i], len = p < 0 ? 0 : v.len[p];
            if (p == (int32_t)i && fresh < 0) continue;
            const uint32_t held = pages_of(t, (uint32_t)len);
            if (e < max(held, pages_of(t, (uint32_t)v.len[i])))
                t.pages[(size_t)seqs[i] * t.max_pages + e] = e >= held ? -1 : e + 1 == held && fresh >= 0 ? fresh : was[(uint32_t)p * columns + c];
        }
        __syncthreads();
    }
}

// ---- compact -----------------------------------------------------------------------------------------------------------
// which of the kScan pages from p0 on are in use
__device__ __forceinline__ uint32_t used_mask(const int32_t* refs, uint32_t p0, uint32_t num_pages) {
    uint32_t m = 0;
    if (p0 < num_pages && num_pages - p0 >= kScan && (reinterpret_cast<uintptr_t>(refs) & 15u) == 0) {
#pragma unroll
        for (int e = 0; e < kScan / 4; ++e) {
            const int4 r = *reinterpret_cast<const int4*>(refs + p0 + 4 * e);
            m |= ((r.x > 0) | (r.y > 0) << 1 | (r.z > 0) << 2 | (r.w > 0) << 3) << (4 * e);
        }
    } else {
        for (int e = 0; e < kScan; ++e)
            if ((unsigned long long)p0 + e < num_pages && refs[p0 + e] > 0) m |= 1u << e;
    }
    return m;
}

// Workspace: [0] moves, [1] used pages, [2..4) unused, then source, hole, count (num_pages each) and the map of moved pages.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(TableView t, int32_t* ws, int32_t* used_out) {
    __shared__ uint32_t sh[kPlanWarps];
    const uint32_t P = t.num_pages;
    int32_t *source = ws + 4, *hole = source + P, *count = hole + P, *map = count + P;
    uint32_t mine = 0, used;
    for (uint32_t base = 0; base < P; base += kPlanThreads * kScan)
        mine += __popc(used_mask(t.refs, base + threadIdx.x * kScan, P));
    block_exclusive(mine, used, sh);
    uint32_t holes = 0, sources = 0;
    for (uint32_t base = 0; base < P; base += kPlanThreads * kScan) {
        const uint32_t p0 = base + threadIdx.x * kScan;
        const uint32_t in_use = used_mask(t.refs, p0, P), there = p0 >= P ? 0u : P - p0 >= kScan ? (1u << kScan) - 1 : (1u << (P - p0)) - 1;
        const uint32_t below = p0 >= used ? 0u : used - p0 >= kScan ? (1u << kScan) - 1 : (1u << (used - p0)) - 1;
        uint32_t hole_bits = ~in_use & there & below, source_bits = in_use & ~below, all;
        const uint32_t at = block_exclusive((uint32_t)__popc(hole_bits) | (uint32_t)__popc(source_bits) << 16, all, sh);
        uint32_t h = holes + (at & 0xffffu), s = sources + (at >> 16);
        for (uint32_t rest = there & ~below & ~in_use; rest; rest &= rest - 1) map[p0 + __ffs(rest) - 1] = -1;
        for (; hole_bits; hole_bits &= hole_bits - 1) hole[h++] = (int32_t)(p0 + __ffs(hole_bits) - 1);
        for (; source_bits; source_bits &= source_bits - 1) {
            const uint32_t p = p0 + __ffs(source_bits) - 1;
            source[s] = (int32_t)p;
            count[s++] = t.refs[p];
        }
        holes += all & 0xffffu;
        sources += all >> 16;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < sources; i += kPlanThreads) map[source[i]] = hole[i];
    if (threadIdx.x == 0) {
        ws[0] = (int32_t)sources;
        ws[1] = (int32_t)used;
        if (used_out) *used_out = (int32_t)used;
    }
}

__global__ void __launch_bounds__(256) compact_move_kernel(TableView t, const int32_t* ws, int32_t* refs_out, int32_t* pages_out,
                                                           uint32_t table_blocks, CopyArgs copy) {
    grid_dependency_wait();                                       // the plan; this kernel's start overlaps its end
    if (blockIdx.x >= table_blocks) {
        copy_pages(copy, blockIdx.x - table_blocks, gridDim.x - table_blocks);
        return;
    }
    const uint32_t P = t.num_pages, moves = (uint32_t)ws[0], used = (uint32_t)ws[1];
    const int32_t *hole = ws + 4 + P, *count = hole + P, *map = count + P;
    const uint32_t me = blockIdx.x * 256 + threadIdx.x, all = table_blocks * 256;
    // counts: below `used` every page that is in use keeps its own, the holes take their source's; past it all are free
    for (uint32_t p = me; p < P; p += all) {
        if (p >= used) refs_out[p] = 0;
        else if (t.refs[p] > 0) refs_out[p] = t.refs[p];
    }
    for (uint32_t i = me; i < moves; i += all) refs_out[hole[i]] = count[i];
    const unsigned long long entries = (unsigned long long)t.max_seqs * t.max_pages;
    for (unsigned long long e = me; e < entries; e += all) {
        int32_t id = t.pages[e];
        if (id >= 0) {
            if ((uint32_t)id >= used) id = (uint32_t)id < P ? map[id] : -1;
            if (id < 0) kv_flag(t.status, ROOMIE_FLAG_KV_PAGE);   // an entry that names a free page, or none
        }
        pages_out[e] = id;
    }
}

size_t kv_pages_bytes(const roomie_kv_cache* c) {
    const size_t words = 16 + 4 * (size_t)c->num_pages + 8 * (size_t)c->max_seqs;
    return (words * sizeof(int32_t) + 255) / 256 * 256;
}

}  // namespace roomie

using namespace roomie;

extern "C" size_t roomie_kv_workspace_bytes(const roomie_kv_cache* cache) {
    if (kv_check(cache) != ROOMIE_OK) return 0;
    return kv_attention_bytes(cache) + kv_pages_bytes(cache);
}

extern "C" int roomie_kv_reserve(const roomie_kv_cache* cache, const int32_t* seqs, const int32_t* want, uint32_t n, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (kv_check(cache) != ROOMIE_OK) return ROOMIE_ERR_INVALID_ARG;
    if (n == 0) return ROOMIE_OK;
    if (!seqs || !want || n > cache->max_seqs) return ROOMIE_ERR_INVALID_ARG;
    const int rc = check_workspace(cache, workspace, workspace_bytes);
    if (rc != ROOMIE_OK) return rc;
    return launch("kv_reserve", reserve_kernel, dim3(1), dim3(kPlanThreads), 0, static_cast<cudaStream_t>(stream), false,
                  table_view(cache), seqs, want, n, page_scratch(cache, workspace));
}

extern "C" int roomie_kv_fork(const roomie_kv_cache* cache, const int32_t* parents, const int32_t* children, uint32_t n,
                              void* workspace, size_t workspace_bytes, void* stream) {
    if (kv_check(cache) != ROOMIE_OK) return ROOMIE_ERR_INVALID_ARG;
    if (n == 0) return ROOMIE_OK;
    if (!parents || !children || n > cache->max_seqs) return ROOMIE_ERR_INVALID_ARG;
    int rc = check_workspace(cache, workspace, workspace_bytes);
    if (rc != ROOMIE_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int32_t* ws = page_scratch(cache, workspace);
    const TableView t = table_view(cache);
    rc = launch("kv_fork_plan", fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, false, t, parents, children, n, ws);
    if (rc != ROOMIE_OK) return rc;
    CopyArgs copy = copy_args(cache, cache);
    copy.n = n; copy.src = ws + 2 * (size_t)n; copy.dst = ws + 3 * (size_t)n;
    return launch("kv_fork_move", fork_move_kernel, dim3(n + copy_blocks(copy, n)), dim3(256), 0, st, true, t, parents, children, n,
                  ws, copy);
}

extern "C" int roomie_kv_reorder(const roomie_kv_cache* cache, const int32_t* seqs, const int32_t* parents, uint32_t n, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (kv_check(cache) != ROOMIE_OK) return ROOMIE_ERR_INVALID_ARG;
    if (n == 0) return ROOMIE_OK;
    if (!seqs || !parents || n > cache->max_seqs || n > kReorderMost) return ROOMIE_ERR_INVALID_ARG;
    int rc = check_workspace(cache, workspace, workspace_bytes);
    if (rc != ROOMIE_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int32_t* ws = page_scratch(cache, workspace);
    const TableView t = table_view(cache);
    uint32_t columns = 32;                                        // at most 32 KB of shared memory
    while (columns > 1 && n * columns > kReorderMost) columns /= 2;
    const size_t smem = (size_t)n * columns * sizeof(int32_t);
    rc = allow_smem(reinterpret_cast<const void*>(reorder_move_kernel), smem);   // before the plan, which changes counts and lengths: all or nothing
    if (rc != ROOMIE_OK) return rc;
    rc = launch("kv_reorder_plan", reorder_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, false, t, seqs, parents, n, ws);
    if (rc != ROOMIE_OK) return rc;
    const ReorderView v = reorder_view(ws, n);
    CopyArgs copy = copy_args(cache, cache);
    copy.n = n; copy.src = v.src; copy.dst = v.dst;
    const uint32_t all = (cache->max_pages + columns - 1) / columns, table_blocks = all < 148 ? all : 148;
    return launch("kv_reorder_move", reorder_move_kernel, dim3(table_blocks + copy_blocks(copy, n)), dim3(256), smem, st, true, t, seqs, parents, n, ws, columns,
                  table_blocks, copy);
}

extern "C" int roomie_kv_free(const roomie_kv_cache* cache, const int32_t* seqs, uint32_t n, void* stream) {
    if (kv_check(cache) != ROOMIE_OK) return ROOMIE_ERR_INVALID_ARG;
    if (n == 0) return ROOMIE_OK;
    if (!seqs || n > 0x7fffffffu) return ROOMIE_ERR_INVALID_ARG;
    return launch("kv_free", free_kernel, dim3((n + 3) / 4), dim3(128), 0, static_cast<cudaStream_t>(stream), false, table_view(cache),
                  seqs, n);
}

extern "C" int roomie_kv_copy(const roomie_kv_cache* src, const int32_t* src_pages, const roomie_kv_cache* dst,
                              const int32_t* dst_pages, uint32_t n, void* stream) {
    if (kv_check(src) != ROOMIE_OK || kv_check(dst) != ROOMIE_OK) return ROOMIE_ERR_INVALID_ARG;
    if (src->layers != dst->layers || src->page_tokens != dst->page_tokens || src->kv_heads != dst->kv_heads ||
        src->head_dim != dst->head_dim || src->format != dst->format || src->layout != dst->layout)
        return ROOMIE_ERR_INVALID_ARG;
    if (n == 0) return ROOMIE_OK;
    if (!src_pages || !dst_pages || n > 0x7fffffffu) return ROOMIE_ERR_INVALID_ARG;
    CopyArgs copy = copy_args(src, dst);
    copy.n = n; copy.src = src_pages; copy.dst = dst_pages;
    return launch("kv_copy", copy_kernel, dim3(copy_blocks(copy, n)), dim3(256), 0, static_cast<cudaStream_t>(stream), false, copy);
}

extern "C" int roomie_kv_compact(const roomie_kv_cache* cache, int32_t* refs_out, int32_t* pages_out, int32_t* used_out,
                                 void* workspace, size_t workspace_bytes, void* stream) {
    if (kv_check(cache) != ROOMIE_OK || !refs_out || !pages_out) return ROOMIE_ERR_INVALID_ARG;
    int rc = check_workspace(cache, workspace, workspace_bytes);
    if (rc != ROOMIE_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int32_t* ws = page_scratch(cache, workspace);
    const TableView t = table_view(cache);
    rc = launch("kv_compact_plan", compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, false, t, ws, used_out);
    if (rc != ROOMIE_OK) return rc;
    CopyArgs copy = copy_args(cache, cache);
    const uint32_t P = cache->num_pages;
    copy.n = P / 2; copy.count = ws; copy.src = ws + 4; copy.dst = ws + 4 + (size_t)P;
    const unsigned long long entries = (unsigned long long)cache->max_seqs * cache->max_pages + P;
    const uint32_t table_blocks = (uint32_t)(entries / 1024 < 1 ? 1 : entries / 1024 > 148 ? 148 : entries / 1024);
    return launch("kv_compact_move", compact_move_kernel, dim3(table_blocks + copy_blocks(copy, P / 2 ? P / 2 : 1)), dim3(256), 0, st,
                  true, t, ws, refs_out, pages_out, table_blocks, copy);
}
