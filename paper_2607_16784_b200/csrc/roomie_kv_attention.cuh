// What the attention kernels over the paged 8-bit cache share.
#pragma once
#include "roomie_kv.cuh"

namespace roomie {

struct AttnArgs {
    KvView c;
    const int32_t *seqs, *q_offset;
    uint32_t num_seqs, rows, q_heads, group;     // group = q_heads / kv heads
    unsigned long long group_inverse;            // 2^64 / group + 1, 0 for a group of 1
    const void* q;
    void* out;
    float* lse;
    long long q_token, q_head, o_token, o_head;
    float scale_log2;                            // scale * log2(e)
    uint32_t window;
    int32_t q_aligned, o_aligned;                // 16-byte rows
    uint32_t* counters;                          // [2][blocks] zero between calls
    float* partial;                              // [blocks][2] of (rows x (DP + 2))
};

constexpr float kLn2 = 0.693147180559945309417f;
constexpr int kMaxAttnBlocksPerSm = 4;

// Weights are float16 for the product with the codes.  They are taken against a reference that moves, to kBelow under the largest
// exponent so far, only when some exponent is more than kAbove over it: the largest weight then lies in 2^7 .. 2^15, below float16's end at
// 65504, and every weight down to 2^-21 of the largest keeps its 11 bits (with a reference at the largest itself: down to 2^-14, and a
// long flat tail behind one leading key lost 1 %).  A running maximum that is moved lazily is a published variation of the one-pass
// softmax (Milakov and Gimelshein, 2018).
constexpr float kAbove = 15.0f, kBelow = 7.0f;

// The softmax total is the weights' sum with each page's value scale divided out again.  That holds while all value scales met are
// within 2^-kNear .. 2^kNear: the largest probability's weight is then above 2^-57 and its share of the total above 2^-25, far from float32's
// end.  From the first page with another scale on, a row's total is summed apart, from exponents without log2 vs, against a reference of
// its own that moves in the same way; a page of zeros, which append gives 2^-100, would drop out of it beside a large one.  At the end both
// go to one reference between the two, where each is within float32.
constexpr float kNear = 32.0f;
constexpr float kLeastScale = 7.888609052210118e-31f;   // 2^-100: a value scale below counts as this

// sums against m (o) and ref (l): o *= up, l and m become those of one reference
__device__ __forceinline__ void one_reference(float& m, float& l, float& up, float ref) {
    up = 1.0f;
    if (m == -INFINITY) return;                         // no key
    const float d = floorf(0.5f * (m - ref));
    up = exp2f(d);
    l *= exp2f(ref - m + d);
    m -= d;
}

// The first key that a row at `position` sees.  Rows may lie before the sequence, and a window be as wide as its type: neither wraps here.
__device__ __forceinline__ int first_seen(int position, uint32_t window) { return max(max(position + 1, 0) - (int)window, 0); }

__device__ __forceinline__ float log2_fast(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// One thread counts its block's part, one of n, after a barrier at which all its threads met; the last one leaves the counter zero.  Both
// fences are this thread's: the first stands between the barrier and the count, so that what every thread wrote comes before it, the second
// between the count and the barrier behind which the other parts are read.
__device__ __forceinline__ uint32_t count_part(uint32_t* counter, uint32_t n) {
    __threadfence();
    const uint32_t before = atomicAdd(counter, 1u);
    if (before == n - 1) *counter = 0;
    __threadfence();
    return before;
}

// 16x8x16 product, float16 operands, float32 sums
__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// four codes of a word to two float16 pairs, exactly (elements 0,1 and 2,3)
template <int kFormat> __device__ __forceinline__ void codes_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    if constexpr (kFormat == ROOMIE_KV_E4M3) {
        asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
            : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        // 0x6400 | u is 1024 + u in float16; u = code + 128 (a published conversion: Kim, Henry, Fahim and Awadalla, 2022)
        const uint32_t u = w ^ 0x80808080u, bias = 0x64806480u;                   // 1152
        const uint32_t l = __byte_perm(u, 0x64646464u, 0x4140), h = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 x = __hsub2(reinterpret_cast<const __half2&>(l), reinterpret_cast<const __half2&>(bias));
        const __half2 y = __hsub2(reinterpret_cast<const __half2&>(h), reinterpret_cast<const __half2&>(bias));
        lo = reinterpret_cast<const uint32_t&>(x);
        hi = reinterpret_cast<const uint32_t&>(y);
    }
}

// Where 16-byte chunk `chunk` of row `row` of a step lies: chunks are exchanged so that neither the keys' reads (8 lanes: two rows, four
// chunks) nor the values' (four rows, two chunks) meet in a bank.
template <int DP> __device__ __forceinline__ uint32_t code_at(uint32_t row, uint32_t chunk) {
    if constexpr (DP >= 128) return row * DP + ((chunk ^ (row & 7)) << 4);
    const uint32_t line = row >> 1;                                // two rows of 64 bytes
    return line * 128 + ((((row & 1) * 4 + chunk) ^ ((line & 3) << 1)) << 4);
}
// N words from a span that starts at byte `first` of a row
template <int DP, int N> __device__ __forceinline__ void read_span(uint32_t* to, const uint8_t* side, uint32_t row, uint32_t first) {
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(side + code_at<DP>(row, first / 16 + i / 4));
            to[i] = x.x; to[i + 1] = x.y; to[i + 2] = x.z; to[i + 3] = x.w;
        }
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(side + code_at<DP>(row, first / 16) + (first & 8));
        to[0] = x.x; to[1] = x.y;
    }
}

// roomie_kv_prompt.cu: many rows a sequence, on the tensor cores' own memory
int launch_prompt(const AttnArgs& a, bool half, cudaStream_t st);
size_t prompt_partial_bytes(uint32_t dim);

}  // namespace roomie
