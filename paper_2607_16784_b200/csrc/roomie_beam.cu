// Beam search's selection: the best continuations of a request over its beams and the vocabulary.
//
//   c[b, v] = score[b] + logit[b, v] - log sum_u exp(logit[b, u]),  the `num` largest over (b, v), equal ones in the order of (b, v)
//
// Two launches.  rows_kernel: a block takes a part of a row that its threads hold in registers: the part's maximum and sum of exponentials, and
// its `num` best logits in order.  pick_kernel: a block for each request adds the parts' sums up in 64 bits and picks from their lists.
//
// Bound by the logits' bytes, with the exponentials close behind: 256 rows of 128256 in bf16, 66 MB, are 10 us and 7.5 us of special-function time.  rows_kernel
// takes 21 us for them, of which a part's block spends some 2000 cycles on the loads, 3000 on the exponentials and 2500 on its barriers and its list, four blocks
// an SM; both launches take 27.4.  pick_kernel is a chain of waits (12 cycles an instruction at its barriers).
#include <type_traits>
#include "roomie_serving.cuh"

namespace roomie {

struct BeamArgs {
    const void* logits;
    long long request_stride, beam_stride;          // elements
    const float* scores;
    const uint8_t* ended;
    uint32_t requests, beams, vocab, num, pad, splits, part;   // splits: parts of a row, of `part` elements each
    int32_t type;
    unsigned long long* keys;                       // [rows][splits][num]
    float2* sums;                                   // [rows][splits] of maximum, sum of exp(x - maximum)
    float* scores_out;
    int32_t *parent_out, *token_out;
};

// A candidate as one number: the larger is the better.  The logit's bits in the order of their values above the token's complement; 0: none.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);                    // -0 counts as 0
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ unsigned long long candidate(float x, uint32_t token) { return (unsigned long long)ordered(x) << 32 | (uint32_t)~token; }

constexpr int kBeamThreads = 256, kBeamWarps = kBeamThreads / 32, kMostNum = 128;
constexpr int kList = 1024;                         // candidates that a block looks at closely
// Of a list that ran over, so many are enough for a bound that leaves a fourth or less: each is compared with each.
__device__ __forceinline__ uint32_t sample_of(uint32_t num) { return max(4 * num, 256u); }

// Values that were widened before are widened again: kept, they would take four times the registers.
template <int kVecs> __device__ __forceinline__ void as_they_are(uint4* raw) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) asm volatile("" : "+r"(raw[i].x), "+r"(raw[i].y), "+r"(raw[i].z), "+r"(raw[i].w));
}
// the largest of a piece, NaN passed over
template <class T> __device__ __forceinline__ float largest(const uint4& raw) {
    if constexpr (sizeof(T) == 4) {
        return fmaxf(fmaxf(__uint_as_float(raw.x), __uint_as_float(raw.y)), fmaxf(__uint_as_float(raw.z), __uint_as_float(raw.w)));
    } else {
        using Two = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        const Two* e = reinterpret_cast<const Two*>(&raw);
        const Two m = __hmax2(__hmax2(e[0], e[1]), __hmax2(e[2], e[3]));
        return fmaxf(to_f32(m.x), to_f32(m.y));
    }
}
template <class T> __device__ __forceinline__ float element(const uint4& v, int i) { return to_f32(reinterpret_cast<const T*>(&v)[i]); }

constexpr int kHits = 512;                          // pieces that may hold a candidate
struct PickShared {
    unsigned long long list[kList], bound;
    uint4 hit[kHits];
    uint32_t hit_at[kHits], hits, count;
};

// The `num` best candidates of the block's pieces, in order, to out[0, num); 0 where there are fewer.  Piece i of a thread: elements base + i * step
// on, the largest of them tops[i].
//
// A bound that leaves few: the threads are 8, 16 or 32 groups (at least num) of neighbours, and the least of the groups' best is reached once in each -
// of numbers in no order about groups * log(groups) are as large; for more than 32, the num-th of the threads' best.  The pieces that may hold such a one are put into shared memory, where a thread looks at
// one element of them; candidates are listed, and each counts those above it.  (Divergent threads that looked through their own pieces took 4000 to
// 18000 cycles of a block's 15000 to 25000.)  Should the pieces or the list run over, as with rows of one number, the threads do go through their own, and the
// num-th of a full list is a higher bound.
template <class T, int kVecs>
__device__ __forceinline__ void pick_best(PickShared& sh, const uint4* raw, const float* tops, float top, uint32_t base, uint32_t num, unsigned long long* out) {
    constexpr int v = kVecOf<T>;
    constexpr uint32_t step = kBeamThreads * v;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    // a number that some of the thread's candidates reaches: its maximum at the last place of the first piece that holds it
    unsigned long long best = 0;
    if (top > -INFINITY)
#pragma unroll
        for (int i = kVecs - 1; i >= 0; --i)
            if (tops[i] == top) best = candidate(top, base + i * step + v - 1);
    unsigned long long bound;
    if (threadIdx.x == 0) sh.count = sh.hits = 0;
    if (num <= 32) {
        const uint32_t wide = num <= 8 ? 32u : num <= 16 ? 16u : 8u;  // threads of a group
#pragma unroll
        for (uint32_t d = 1; d < 32; d *= 2) {                        // the largest of a group, then the least of a warp's groups
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, d);
            if ((other > best) == (d < wide)) best = other;
        }
        if (lane == 0) sh.list[wid] = best;
        __syncthreads();
        bound = sh.list[0];
#pragma unroll
        for (int w = 1; w < kBeamWarps; ++w) bound = min(bound, sh.list[w]);
    } else {                                                          // the num-th of the threads' best (0 where fewer have one)
        sh.list[threadIdx.x] = best;
        if (threadIdx.x == 0) sh.bound = 0;
        __syncthreads();
        uint32_t above = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < kBeamThreads; ++j) above += sh.list[j] > best;
        if (above == num - 1) sh.bound = best;                        // one thread, but for 0
        __syncthreads();
        bound = sh.bound;
    }
    bound = max(bound, 1ull);
    auto put = [&](float e, uint32_t token) {
        const unsigned long long c = candidate(e, token);
        if (c >= bound && e > -INFINITY) {
            const uint32_t at = atomicAdd(&sh.count, 1u);
            if (at < kList) sh.list[at] = c;
        }
    };
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
        if (tops[i] > -INFINITY && candidate(tops[i], base + i * step) >= bound) {
            const uint32_t at = atomicAdd(&sh.hits, 1u);
            if (at < kHits) {
                sh.hit[at] = raw[i];
                sh.hit_at[at] = base + i * step;
            }
        }
    __syncthreads();
    const uint32_t hits = sh.hits;                                    // (behind this barrier nobody reads the best any more)
    if (hits <= kHits) {
        for (uint32_t x = threadIdx.x; x < hits * v; x += kBeamThreads)
            put(to_f32(reinterpret_cast<const T*>(&sh.hit[x / v])[x % v]), sh.hit_at[x / v] + x % v);
        __syncthreads();
    }
    bool full = hits <= kHits && sh.count > kList;                    // the list ran over (the same for all threads: the count is at rest)
    // Each trip with a full list leaves out sample - num candidates or more, which is 128 at least.
    constexpr uint32_t kTrips = step * kVecs / 128 + 2;
    uint32_t trip = 0;
    for (bool own = hits > kHits; (own || full) && trip < kTrips; own = false, ++trip) {
        if (full) {
            const uint32_t sample = sample_of(num);
            for (uint32_t i = threadIdx.x; i < sample; i += kBeamThreads) {
                const unsigned long long x = sh.list[i];
                uint32_t above = 0;
#pragma unroll 8
                for (uint32_t j = 0; j < sample; ++j) above += sh.list[j] > x;
                if (above == num - 1) sh.bound = x;
            }
            __syncthreads();
            bound = sh.bound;
            if (threadIdx.x == 0) sh.count = 0;
            __syncthreads();
        }
#pragma unroll 1
        for (int i = 0; i < kVecs; ++i) {
            uint4 piece = raw[0];
#pragma unroll
            for (int j = 1; j < kVecs; ++j)
                if (j == i) piece = raw[j];
#pragma unroll
            for (int k = 0; k < v; ++k) put(element<T>(piece, k), base + i * step + k);
        }
        __syncthreads();
        full = sh.count > kList;
    }
    const uint32_t n = min(sh.count, (uint32_t)kList);
    for (uint32_t i = threadIdx.x; i < n; i += kBeamThreads) {
        const unsigned long long x = sh.list[i];
        uint32_t above = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) above += sh.list[j] > x;
        if (above < num) out[above] = x;
    }
    for (uint32_t i = n + threadIdx.x; i < num; i += kBeamThreads) out[i] = 0;
}

// 16 bytes that start `shift` bytes into the 32 of a and b; shift is the same for the row
__device__ __forceinline__ uint4 joined(const uint4& a, const uint4& b, uint32_t shift) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    const uint32_t words = shift / 4, bits = 8 * (shift & 3);
    uint32_t x[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) x[i] = words == 0 ? w[i] : words == 1 ? w[i + 1] : words == 2 ? w[i + 2] : w[i + 3];
    return make_uint4(__funnelshift_r(x[0], x[1], bits), __funnelshift_r(x[1], x[2], bits), __funnelshift_r(x[2], x[3], bits), __funnelshift_r(x[3], x[4], bits));
}

// Elements [at, at + 16 bytes) of a row of any alignment, -infinity behind its end.
template <class T> __device__ __forceinline__ uint4 piece_of(const T* x, uint32_t at, uint32_t vocab, uint32_t shift) {
    constexpr int v = kVecOf<T>;
    const T* p = x + at;
    if (shift == 0 && at + v <= vocab) return __ldcs(reinterpret_cast<const uint4*>(p));
    if (shift && at && at + 2 * v <= vocab) {                         // the 32 aligned bytes around it lie inside the row
        const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) - shift);
        return joined(q[0], q[1], shift);
    }
    uint4 y;
    uint32_t* w = &y.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = at + i < vocab ? reinterpret_cast<const uint32_t*>(p)[i] : 0xff800000u;
        } else {
            const uint32_t none = std::is_same<T, __half>::value ? 0xfc00u : 0xff80u;
            const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
            w[i] = (at + 2 * i < vocab ? h[2 * i] : none) | (at + 2 * i + 1 < vocab ? (uint32_t)h[2 * i + 1] : none) << 16;
        }
    }
    return y;
}

// kVecs 16-byte pieces a thread.  The pieces are counted from the row's first element, wherever in memory that is: equal rows give equal sums.
template <class T, int kVecs>
__global__ void __launch_bounds__(kBeamThreads, 4) rows_kernel(BeamArgs a) {
    constexpr int v = kVecOf<T>;
    __shared__ PickShared sh;
    __shared__ float sh_max[kBeamWarps], sh_sum[kBeamWarps];
    const uint32_t row = blockIdx.y, request = row / a.beams, beam = row - request * a.beams;
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    if (a.ended && a.ended[row]) return;
    const T* x = static_cast<const T*>(a.logits) + (long long)request * a.request_stride + (long long)beam * a.beam_stride;
    const uint32_t shift = (uint32_t)(reinterpret_cast<uintptr_t>(x) & 15u);
    const uint32_t base = blockIdx.x * (kBeamThreads * kVecs * v) + threadIdx.x * v;    // piece i: elements base + i * kBeamThreads * v on
    uint4 raw[kVecs];
    if (shift == 0 && (blockIdx.x + 1) * (kBeamThreads * kVecs * v) <= a.vocab) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) raw[i] = __ldcs(reinterpret_cast<const uint4*>(x + base + i * (kBeamThreads * v)));
    } else {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) raw[i] = piece_of(x, base + i * (kBeamThreads * v), a.vocab, shift);
    }
    // the pieces' maxima, and the sum against the thread's own maximum.  NaN is passed over here and shows in the sum.
    float tops[kVecs], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        tops[i] = largest<T>(raw[i]);
        top = fmaxf(top, tops[i]);
    }
    as_they_are<kVecs>(raw);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int k = 0; k < v; ++k) sum[k & 3] += exp2_fast((element<T>(raw[i], k) - ref) * 1.44269504088896340736f);
    as_they_are<kVecs>(raw);
    float total = (sum[0] + sum[1]) + (sum[2] + sum[3]), most = top;
    if (total != total) most = INFINITY;                             // NaN or +infinity: the row has no probabilities
#pragma unroll
    for (int d = 1; d < 32; d *= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
    if (lane == 0) sh_max[wid] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBeamWarps; ++w) most = fmaxf(most, sh_max[w]);
    total = top == -INFINITY ? 0.0f : total * exp2_fast((top - most) * 1.44269504088896340736f);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) total += __shfl_xor_sync(0xffffffffu, total, d);
    if (lane == 0) sh_sum[wid] = total;
    const size_t part = (size_t)row * a.splits + blockIdx.x;
    pick_best<T, kVecs>(sh, raw, tops, top, base, a.num, a.keys + part * a.num);
    if (threadIdx.x == 0) {                                          // pick_best has barriers between
        total = 0.0f;
        for (int w = 0; w < kBeamWarps; ++w) total += sh_sum[w];
        a.sums[part] = make_float2(most, total);
    }
}

// ---- the requests' picks -----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned long long ordered64(double x) {
    const unsigned long long b = (unsigned long long)__double_as_longlong(x + 0.0);
    return b ^ ((unsigned long long)((long long)b >> 63) | 0x8000000000000000ull);
}

// Candidates in order of (value in 64 bits, row, token): `order` is the complement of the last two, and value 0 is none.
struct Candidate {
    unsigned long long value, order;
};
__device__ __forceinline__ bool over(const Candidate& x, const Candidate& y) { return x.value > y.value || (x.value == y.value && x.order > y.order); }

constexpr int kPickThreads = 256, kPickWarps = kPickThreads / 32;
struct PickList {
    Candidate list[kList], bound;
    unsigned long long level;
    uint32_t count, unsure, above, votes[kPickWarps], hist[256];
};

// A beam's score, the largest logit of its row (or of nothing) and the logarithm of the row's sum, as the kernel has them for each beam.  A candidate's
// value: the difference first, since logits may be of any size.
__device__ __forceinline__ unsigned long long value_of(const double* of_beam, float logit) {
    return ordered64(of_beam[0] + ((double)logit - of_beam[1] - of_beam[2]));
}
// Whether no other float32 near this logit has its value.
__device__ __forceinline__ bool only_one(const double* of_beam, uint32_t logit, unsigned long long value) {
    return value_of(of_beam, unordered(logit - 1)) < value && value_of(of_beam, unordered(logit + 1)) > value;
}

// Entry `at` of a list, a part of a beam's row.  keys: the request's.
__device__ __forceinline__ Candidate entry_of(const BeamArgs& a, const double* of_row, uint32_t request, const unsigned long long* keys, uint32_t list, uint32_t at) {
    const uint32_t b = list / a.splits, row = request * a.beams + b;
    const double score = of_row[3 * b];
    Candidate c = {0, 0};
    if (score != score) return c;
    if (a.ended && a.ended[row]) {                                   // goes on as it is, with the padding token
        if (list == b * a.splits && at == 0) c = {ordered64(score), ~((unsigned long long)b << 32 | a.pad)};
        return c;
    }
    const unsigned long long key = keys[(size_t)list * a.num + at];
    if (key) c = {value_of(of_row + 3 * b, unordered((uint32_t)(key >> 32))), ~((unsigned long long)b << 32 | (uint32_t)~(uint32_t)key)};
    return c;
}

__device__ __forceinline__ void write_pick(const BeamArgs& a, uint32_t request, uint32_t at, unsigned long long value, uint32_t beam, uint32_t token) {
    const size_t to = (size_t)request * a.num + at;
    const unsigned long long bits = value & 0x8000000000000000ull ? value ^ 0x8000000000000000ull : ~value;
    a.scores_out[to] = (float)__longlong_as_double((long long)bits);
    a.parent_out[to] = (int32_t)(request * a.beams + beam);
    a.token_out[to] = (int32_t)token;
}

// The num-th of the first n of a list, n >= num, becomes the bound: each counts those above it.
__device__ __forceinline__ void bound_of(PickList& sh, uint32_t n, uint32_t num) {
    for (uint32_t i = threadIdx.x; i < n; i += kPickThreads) {
        const Candidate x = sh.list[i];
        uint32_t above = 0, same = 0;                                // those that are none are all the same
#pragma unroll 4
        for (uint32_t j = 0; j < n; ++j) {
            above += over(sh.list[j], x);
            same += sh.list[j].value == x.value && sh.list[j].order == x.order;
        }
        if (above < num && above + same >= num) sh.bound = x;
    }
}

// The num-th value of all lists, eight bits at a time, becomes the level, and the list what lies above it: fewer than num.
__device__ __noinline__ void find_level(const BeamArgs& a, PickList& sh, const double* of_row, uint32_t request) {
    const uint32_t entries = a.beams * a.splits * a.num;
    const unsigned long long* keys = a.keys + (size_t)request * entries;
    unsigned long long level = 0;
    uint32_t left = a.num;
#pragma unroll 1
    for (int shift = 56; shift >= 0; shift -= 8) {
        sh.hist[threadIdx.x] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < entries; i += kPickThreads) {
            const unsigned long long x = entry_of(a, of_row, request, keys, i / a.num, i % a.num).value;
            if (shift == 56 || x >> (shift + 8) == level >> (shift + 8)) atomicAdd(&sh.hist[x >> shift & 255], 1u);
        }
        __syncthreads();
        uint32_t d = 255;                                            // the digit in which the left-th lies
        for (; d > 0 && sh.hist[d] < left; --d) left -= sh.hist[d];
        level |= (unsigned long long)d << shift;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        sh.level = level;
        sh.count = 0;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < entries; i += kPickThreads) {
        const Candidate c = entry_of(a, of_row, request, keys, i / a.num, i % a.num);
        if (c.value > level) {
            const uint32_t at = atomicAdd(&sh.count, 1u);
            if (at < kList) sh.list[at] = c;                         // (always, unless another call writes to the lists meanwhile)
        }
    }
    __syncthreads();
}

// The num-th of a list's n becomes the level.
__device__ __forceinline__ void level_of(PickList& sh, uint32_t n, uint32_t num) {
    for (uint32_t i = threadIdx.x; i < n; i += kPickThreads) {
        const Candidate x = sh.list[i];
        uint32_t above = 0;
        for (uint32_t j = 0; j < n; ++j) above += over(sh.list[j], x);
        if (above == num - 1) sh.level = x.value;
    }
    __syncthreads();
}

// The picks from the num-th value, the level: those above it are among the list's n, fewer than num; of those that have it the first by (beam, token) are looked for
// in the logits, in the parts whose best reaches it, of which 2 num at most are gone through, in order, up to the last one wanted.
__device__ __noinline__ void pick_by_value(const BeamArgs& a, PickList& sh, const double* of_row, uint32_t request, uint32_t n) {
    const uint32_t lane = threadIdx.x & 31, wid = threadIdx.x >> 5, lists = a.beams * a.splits;
    const unsigned long long level = sh.level;
    for (uint32_t i = threadIdx.x; i < n; i += kPickThreads) {
        const Candidate x = sh.list[i];
        if (x.value <= level) continue;
        uint32_t above = 0;
        for (uint32_t j = 0; j < n; ++j) above += over(sh.list[j], x);
        if (above < a.num) write_pick(a, request, above, x.value, (uint32_t)(~x.order >> 32), (uint32_t)~x.order);
        atomicAdd(&sh.above, 1u);
    }
    __syncthreads();
    uint32_t at = sh.above;                                          // the same in all threads, here and below
    auto ended = [&](uint32_t b) { return a.ended && a.ended[request * a.beams + b]; };
    for (uint32_t first = 0; first < lists && at < a.num; first += kPickThreads) {
        const uint32_t mine = first + threadIdx.x, b = mine / a.splits;
        bool look = false;
        if (mine < lists && of_row[3 * b] == of_row[3 * b]) {
            if (ended(b)) {
                look = mine == b * a.splits && ordered64(of_row[3 * b]) == level;
            } else {
                const unsigned long long key = a.keys[((size_t)request * lists + mine) * a.num];
                look = key && value_of(of_row + 3 * b, unordered((uint32_t)(key >> 32))) >= level;
            }
        }
        const uint32_t votes = __ballot_sync(0xffffffffu, look);
        __syncthreads();
        if (lane == 0) sh.votes[wid] = votes;
        __syncthreads();
        uint32_t chosen[kPickWarps];
#pragma unroll
        for (int w = 0; w < kPickWarps; ++w) chosen[w] = sh.votes[w];
#pragma unroll 1
        for (uint32_t x = 0; x < kPickThreads && at < a.num; ++x) {
            if (!(chosen[x >> 5] >> (x & 31) & 1)) continue;
            const uint32_t beam = (first + x) / a.splits, split = first + x - beam * a.splits;
            if (ended(beam)) {
                if (threadIdx.x == 0) write_pick(a, request, at, level, beam, a.pad);
                ++at;
                continue;
            }
            const long long row = (long long)request * a.request_stride + (long long)beam * a.beam_stride;
            const uint32_t end = min(a.vocab - split * a.part, a.part);
            for (uint32_t t0 = 0; t0 < end && at < a.num; t0 += kPickThreads) {
                const uint32_t token = split * a.part + t0 + threadIdx.x;
                bool hit = false;
                if (t0 + threadIdx.x < end) {
                    const float logit = a.type == ROOMIE_F32 ? static_cast<const float*>(a.logits)[row + token]
                                        : a.type == ROOMIE_F16 ? to_f32(static_cast<const __half*>(a.logits)[row + token])
                                                               : to_f32(static_cast<const __nv_bfloat16*>(a.logits)[row + token]);
                    hit = value_of(of_row + 3 * beam, logit) == level;
                }
                const uint32_t hits = __ballot_sync(0xffffffffu, hit);
                __syncthreads();
                if (lane == 0) sh.votes[wid] = hits;
                __syncthreads();
                uint32_t to = at + __popc(hits & ((1u << lane) - 1));
#pragma unroll
                for (int w = 0; w < kPickWarps; ++w) {
                    const uint32_t more = __popc(sh.votes[w]);
                    if (w < (int)wid) to += more;
                    at += more;
                }
                if (hit && to < a.num) write_pick(a, request, to, level, beam, token);
            }
        }
    }
}

__global__ void __launch_bounds__(kPickThreads) pick_kernel(const __grid_constant__ BeamArgs a) {
    extern __shared__ double of_row[];                               // [beams][3]: score (NaN: no candidates), largest logit, log of the sum
    __shared__ PickList sh;
    grid_dependency_wait();
    const uint32_t request = blockIdx.x, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    for (uint32_t b = wid; b < a.beams; b += kPickThreads / 32) {
        const uint32_t row = request * a.beams + b;
        const double score = a.scores[row];
        const bool live = score < INFINITY && score > -INFINITY;     // false for NaN
        double valid = __longlong_as_double(0x7ff8000000000000ll);
        if (a.ended && a.ended[row]) {
            if (live) valid = score;
        } else {
            float most = -INFINITY;
            for (uint32_t s = lane; s < a.splits; s += 32) most = fmaxf(most, a.sums[(size_t)row * a.splits + s].x);
#pragma unroll
            for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            double total = 0.0;
            for (uint32_t s = lane; s < a.splits; s += 32) {
                const float2 p = a.sums[(size_t)row * a.splits + s];
                if (p.y > 0.0f) total += (double)p.y * exp((double)p.x - (double)most);
            }
#pragma unroll
            for (int d = 16; d > 0; d /= 2) total += __shfl_xor_sync(0xffffffffu, total, d);
            if (live && most < INFINITY && most > -INFINITY) valid = score;
            if (lane == 0) {
                of_row[3 * b + 1] = most;
                of_row[3 * b + 2] = log(total);
            }
        }
        if (lane == 0) of_row[3 * b] = valid;
    }
    if (threadIdx.x == 0) {
        sh.count = sh.unsure = sh.above = 0;
        sh.level = 0;
    }
    __syncthreads();
    const uint32_t lists = a.beams * a.splits, entries = lists * a.num;
    const unsigned long long* keys = a.keys + (size_t)request * entries;
    auto entry = [&](uint32_t list, uint32_t at) { return entry_of(a, of_row, request, keys, list, at); };
    // A bound: the num-th of the leading entries of (some of) the lists, about four times num of them: what it leaves is little more than num.
    // (With num of them it left so many of 32 lists of 64 that the call took 330 us.)  Then as in pick_best.
    const uint32_t deep = min((4 * a.num + lists - 1) / lists, a.num), some = min(lists, (uint32_t)kPickThreads) * deep;   // deep > 1: lists < 4 num <= 512
    for (uint32_t i = threadIdx.x; i < some; i += kPickThreads) sh.list[i] = entry(i / deep, i % deep);
    __syncthreads();
    bound_of(sh, some, a.num);
    __syncthreads();
    const uint32_t room = sample_of(a.num);                           // more than so many: another bound
    // Lists were cut by the logit.  Where a full one's last entry may be among the picked and other logits have its value (scores so large, or logits so small, that
    // 64 bits do not tell them apart), elements that were cut may come before others by their token.
    auto unsure_behind = [&](uint32_t list) {
        const uint32_t b = list / a.splits, row = request * a.beams + b;
        if (a.ended && a.ended[row]) return false;
        const uint32_t logit = (uint32_t)(keys[(size_t)list * a.num + a.num - 1] >> 32);
        return !only_one(of_row + 3 * b, logit, value_of(of_row + 3 * b, unordered(logit)));
    };
    // One trip as a rule.  A bound may leave out little, as where the best of many lists are the last ones: after a few trips the num-th value is found by its bits,
    // in eight more (64 rising beams x 131072 words, 64 wanted: 2.3 ms, with nothing but trips 4.2; 256 x 128256 in float32, 128 wanted: 31, was 87).
    constexpr uint32_t kTrips = 16;
    for (uint32_t trip = 1;; ++trip) {
        const Candidate bound = sh.bound;
        for (uint32_t i = threadIdx.x; i < entries; i += kPickThreads) {
            const uint32_t list = i / a.num, place = i - list * a.num;
            const Candidate c = entry(list, place);
            if (c.value && c.value >= bound.value) {
                if (!over(bound, c)) {
                    const uint32_t at = atomicAdd(&sh.count, 1u);
                    if (at < room) sh.list[at] = c;
                }
                if (place == a.num - 1 && unsure_behind(list)) sh.unsure = 1;
            }
        }
        __syncthreads();
        if (sh.count <= room || trip == kTrips) break;
        __syncthreads();
        if (threadIdx.x == 0) sh.count = 0;
        bound_of(sh, room, a.num);
        __syncthreads();
    }
    const uint32_t n = sh.count;
    if (n > room) {                                                  // (the same for all threads, and below)
        find_level(a, sh, of_row, request);
        pick_by_value(a, sh, of_row, request, min(sh.count, (uint32_t)kList));
        return;
    }
    if (sh.unsure && n >= a.num) {
        level_of(sh, n, a.num);
        pick_by_value(a, sh, of_row, request, n);
        return;
    }
    for (uint32_t i = threadIdx.x; i < n; i += kPickThreads) {
        const Candidate x = sh.list[i];
        uint32_t above = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) above += over(sh.list[j], x);
        if (above < a.num) write_pick(a, request, above, x.value, (uint32_t)(~x.order >> 32), (uint32_t)~x.order);
    }
    for (uint32_t i = n + threadIdx.x; i < a.num; i += kPickThreads) {
        const size_t to = (size_t)request * a.num + i;
        a.scores_out[to] = -INFINITY;
        a.parent_out[to] = a.token_out[to] = -1;
    }
}

struct BeamShape {
    uint32_t splits, part;
    bool large;
    size_t keys, bytes;
};
// Parts of 8 pieces a thread, or of 2 where those would leave more than half of the SMs without a block.  Both launches, us (bf16; rows x vocabulary):
//      1 x 32000  1 x 128256  16 x 32000 | 16 x 128256  64 x 32000  64 x 128256  256 x 128256
//   8  8.9        10.6        10.7       | 10.8         10.8        14.9         27.3
//   2  8.5        9.4         9.9        | 17.3         11.4        23.9         49.6
static BeamShape beam_shape(uint32_t requests, uint32_t beams, uint32_t vocab, uint32_t num, int32_t type) {
    BeamShape s;
    const unsigned long long rows = (unsigned long long)requests * beams, one = (unsigned long long)kBeamThreads * 16 / size_of_type(type);
    const unsigned long long eight = (vocab + 8 * one - 1) / (8 * one), two = (vocab + 2 * one - 1) / (2 * one);
    s.large = 2 * rows * eight >= (unsigned long long)sm_count();
    s.splits = (uint32_t)(s.large ? eight : two);
    s.keys = (size_t)rows * s.splits * num * sizeof(unsigned long long);
    s.part = (uint32_t)((s.large ? 8 : 2) * one);
    s.bytes = (s.keys + (size_t)rows * s.splits * sizeof(float2) + 255) / 256 * 256;
    return s;
}
static bool beam_valid(uint32_t requests, uint32_t beams, uint32_t vocab, uint32_t num, int32_t type) {
    return beams > 0 && beams <= 256 && vocab > 0 && vocab <= 1u << 24 && num > 0 && num <= (uint32_t)kMostNum && known_type(type) &&
           (unsigned long long)requests * beams <= 65535u;
}

template <class T> static int launch_rows(const BeamArgs& a, bool large, cudaStream_t st) {
    void (*k)(BeamArgs) = large ? rows_kernel<T, 8> : rows_kernel<T, 2>;
    return launch("beam_rows", k, dim3(a.splits, a.requests * a.beams), dim3(kBeamThreads), 0, st, false, a);
}

}  // namespace roomie

using namespace roomie;

extern "C" size_t roomie_beam_workspace_bytes(uint32_t requests, uint32_t beams, uint32_t vocab, uint32_t num, int32_t type) {
    if (requests == 0 || !beam_valid(requests, beams, vocab, num, type)) return 0;
    return beam_shape(requests, beams, vocab, num, type).bytes;
}

extern "C" int roomie_beam_select(const void* logits, int32_t type, int64_t request_stride, int64_t beam_stride, uint32_t requests, uint32_t beams,
                                  uint32_t vocab, const float* scores, const uint8_t* ended, uint32_t pad, uint32_t num, float* scores_out,
                                  int32_t* parent_out, int32_t* token_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!beam_valid(requests, beams, vocab, num, type) || pad > 0x7fffffffu) return ROOMIE_ERR_INVALID_ARG;
    if (requests == 0) return ROOMIE_OK;
    if (!logits || !scores || !scores_out || !parent_out || !token_out || reinterpret_cast<uintptr_t>(logits) % size_of_type(type)) return ROOMIE_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return ROOMIE_ERR_INVALID_ARG;
    const BeamShape s = beam_shape(requests, beams, vocab, num, type);
    if (workspace_bytes < s.bytes) return ROOMIE_ERR_CAPACITY;
    BeamArgs a = {};
    a.logits = logits; a.request_stride = request_stride; a.beam_stride = beam_stride;
    a.scores = scores; a.ended = ended;
    a.requests = requests; a.beams = beams; a.vocab = vocab; a.num = num; a.pad = pad; a.splits = s.splits; a.part = s.part;
    a.type = type;
    a.keys = static_cast<unsigned long long*>(workspace);
    a.sums = reinterpret_cast<float2*>(static_cast<char*>(workspace) + s.keys);
    a.scores_out = scores_out; a.parent_out = parent_out; a.token_out = token_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int rc = type == ROOMIE_F32 ? launch_rows<float>(a, s.large, st)
             : type == ROOMIE_F16 ? launch_rows<__half>(a, s.large, st) : launch_rows<__nv_bfloat16>(a, s.large, st);
    if (rc != ROOMIE_OK) return rc;
    return launch("beam_pick", pick_kernel, dim3(requests), dim3(kPickThreads), 3 * beams * sizeof(double), st, true, a);
}
