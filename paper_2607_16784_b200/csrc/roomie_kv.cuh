// The paged 8-bit cache as the serving kernels see it.
#pragma once
#include "roomie_serving.cuh"

namespace roomie {

struct KvView {                     // one layer of the cache
    uint8_t *k, *v;
    float *k_scale, *v_scale;       // [num_pages][heads]
    const int32_t *refs, *pages, *length;
    uint32_t* status;
    long long page_stride;
    uint32_t num_pages, page_tokens, page_shift, heads, dim, max_seqs, max_pages;
    int32_t format;
    uint32_t token_step, head_step; // bytes between tokens and between heads inside a page
};

// roomie_kv_*.cu
int kv_check(const roomie_kv_cache* c);                       // ROOMIE_OK or ROOMIE_ERR_INVALID_ARG
KvView kv_view(const roomie_kv_cache* c, uint32_t layer);
size_t kv_attention_bytes(const roomie_kv_cache* c);
size_t kv_pages_bytes(const roomie_kv_cache* c);

__device__ __forceinline__ void kv_flag(uint32_t* status, uint32_t bits) { atomicOr(status, bits); }

// What one sequence of a call brings: rows [row, row + count) of the call at positions [start, start + count) of table row
// `slot`.  Anything out of range is reported and counts as no rows.
struct KvSeq {
    uint32_t slot, row, count, start, length;
};
__device__ __forceinline__ KvSeq kv_seq(const KvView& c, const int32_t* seqs, const int32_t* q_offset, uint32_t rows, uint32_t i,
                                        bool report) {
    KvSeq s;
    const int32_t slot = seqs[i];
    const long long lo = q_offset ? q_offset[i] : (long long)i, hi = q_offset ? q_offset[i + 1] : (long long)i + 1;
    const bool there = slot >= 0 && (uint32_t)slot < c.max_seqs;
    const int32_t len = there ? c.length[slot] : 0;
    const bool rows_ok = lo >= 0 && lo <= hi && hi <= (long long)rows;
    s.slot = there ? (uint32_t)slot : 0u;
    s.row = rows_ok ? (uint32_t)lo : 0u;
    s.count = rows_ok ? (uint32_t)(hi - lo) : 0u;
    const bool len_ok = there && len >= 0 && (unsigned long long)len <= (unsigned long long)c.max_pages * c.page_tokens;
    s.length = len_ok ? (uint32_t)len : 0u;
    s.start = s.length - s.count;                                        // may wrap: see the callers
    if (report && !(rows_ok && len_ok)) kv_flag(c.status, ROOMIE_FLAG_KV_SEQUENCE);
    return s;
}

// least power of two s with amax / s <= 448 (e4m3) or 127 (int8), from 2^-100 (values below 2^-101 of
// which are as good as zero) to 2^122 (the largest float needs no more): from the bits of amax
__device__ __forceinline__ int kv_scale_exponent(float amax, int32_t format) {
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 126;                                // amax = m * 2^e, m in [1/2, 1)
    const uint32_t m = bits & 0x7fffffu;
    int x = format == ROOMIE_KV_E4M3 ? e - 9 + (m > 0x600000u) : e - 7 + (m > 0x7e0000u);   // 448 = 0.875 * 2^9
    return x < -100 ? -100 : x > 122 ? 122 : x;
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// two values (already divided by the scale) to two codes, the first in the low byte
__device__ __forceinline__ uint32_t kv_codes2(float a, float b, int32_t format) {
    if (format == ROOMIE_KV_E4M3) return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const int x = __float2int_rn(fminf(fmaxf(a, -127.0f), 127.0f)), y = __float2int_rn(fminf(fmaxf(b, -127.0f), 127.0f));
    return (uint32_t)(x & 0xff) | ((uint32_t)(y & 0xff) << 8);
}
__device__ __forceinline__ float kv_value(uint8_t code, int32_t format) {
    if (format == ROOMIE_KV_E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw(code, __NV_E4M3)));
    return (float)(int8_t)code;
}

}  // namespace roomie
