// What the operations on the cache's pages share: the page table, a block's view of the free pages, the workspace.
#pragma once
#include "roomie_kv.cuh"

namespace roomie {

// ---- a block's view of the free pages ----------------------------------------------------------------------------------
constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;

// exclusive prefix sum over the block of one value a thread; `total` for all.  sh: kPlanWarps values.
template <class V> __device__ __forceinline__ V block_exclusive(V x, V& total, V* sh) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    V incl = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const V up = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += up;
    }
    __syncthreads();
    if (lane == 31) sh[wid] = incl;
    __syncthreads();
    if (wid == 0) {
        V w = sh[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const V up = __shfl_up_sync(0xffffffffu, w, d);
            if (lane >= d) w += up;
        }
        sh[lane] = w;
    }
    __syncthreads();
    total = sh[kPlanWarps - 1];
    return (wid ? sh[wid - 1] : V(0)) + incl - x;
}

// Writes the lowest `want` free pages to list, ascending; returns how many there are.
constexpr int kScan = 16;                                     // counts a thread looks at in one trip
static __device__ uint32_t lowest_free(const int32_t* refs, uint32_t num_pages, uint32_t want, int32_t* list, uint32_t* sh) {
    uint32_t found = 0;
    for (uint32_t base = 0; base < num_pages && found < want; base += kPlanThreads * kScan) {
        const uint32_t p0 = base + threadIdx.x * kScan;
        uint32_t free = 0;
        if (p0 + kScan <= num_pages && (reinterpret_cast<uintptr_t>(refs) & 15u) == 0) {
#pragma unroll
            for (int e = 0; e < kScan / 4; ++e) {
                const int4 r = *reinterpret_cast<const int4*>(refs + p0 + 4 * e);
                free |= ((r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3) << (4 * e);
            }
        } else {
            for (int e = 0; e < kScan; ++e)
                if (p0 + e < num_pages && refs[p0 + e] == 0) free |= 1u << e;
        }
        uint32_t all;
        uint32_t at = found + block_exclusive((uint32_t)__popc(free), all, sh);
        while (free && at < want) {
            list[at++] = (int32_t)(p0 + __ffs(free) - 1);
            free &= free - 1;
        }
        found += all;
    }
    return min(found, want);
}

// ---- the page table ----------------------------------------------------------------------------------------------------
struct TableView {
    int32_t *refs, *pages, *length;
    uint32_t* status;
    uint32_t num_pages, max_seqs, max_pages, page_shift;
};
__device__ __forceinline__ bool slot_ok(const TableView& t, int32_t s) { return s >= 0 && (uint32_t)s < t.max_seqs; }
__device__ __forceinline__ int32_t length_of(const TableView& t, int32_t s) {      // -1: not a sequence or not a length
    if (!slot_ok(t, s)) return -1;
    const int32_t n = t.length[s];
    return n >= 0 && (unsigned long long)n <= ((unsigned long long)t.max_pages << t.page_shift) ? n : -1;
}
__device__ __forceinline__ uint32_t pages_of(const TableView& t, uint32_t tokens) {
    return (tokens + (1u << t.page_shift) - 1) >> t.page_shift;
}

// One block.  need[i] = pages request i wants (0 for one that is refused, with state[i] = -1); afterwards first[i] is where its
// pages begin in list, and the return value is how many of list exist.  Sums are 64 bits wide: what is asked for may be any multiple of
// what there is.
static __device__ uint32_t serve(const TableView& t, uint32_t n, const int32_t* need, int32_t* first, int32_t* list, uint32_t limit, uint32_t* sh) {
    __shared__ unsigned long long sums[kPlanWarps];
    unsigned long long carry = 0;
    for (uint32_t base = 0; base < n; base += kPlanThreads) {
        const uint32_t i = base + threadIdx.x;
        unsigned long long all;
        const unsigned long long x = i < n ? (uint32_t)need[i] : 0u;
        const unsigned long long at = carry + block_exclusive(x, all, sums);
        if (i < n) first[i] = (int32_t)min(at, 0x7fffffffull);
        carry += all;
    }
    return lowest_free(t.refs, t.num_pages, (uint32_t)min(carry, (unsigned long long)limit), list, sh);
}

// ---- host ----------------------------------------------------------------------------------------------------------------
inline TableView table_view(const roomie_kv_cache* c) {
    const uint32_t shift = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
    return {c->refs, c->pages, c->length, c->status, c->num_pages, c->max_seqs, c->max_pages, shift};
}

inline int check_workspace(const roomie_kv_cache* c, const void* ws, size_t bytes) {
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u)) return ROOMIE_ERR_INVALID_ARG;
    return bytes < roomie_kv_workspace_bytes(c) ? ROOMIE_ERR_CAPACITY : ROOMIE_OK;
}
// the attention call's part of a workspace comes first (its counters have to stay zero), the page operations' behind it
inline int32_t* page_scratch(const roomie_kv_cache* c, void* ws) {
    return reinterpret_cast<int32_t*>(static_cast<char*>(ws) + kv_attention_bytes(c));
}

}  // namespace roomie
