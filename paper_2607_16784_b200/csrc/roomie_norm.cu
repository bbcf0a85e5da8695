// Norms of queries and keys for each head, with the rotary positions in the same pass, and their gradients.
//
//   y = R(position) (x * r * w),  r = (mean x^2 + eps)^(-1/2)
//   g = R^T dy,  dw = sum over rows of g * x r,  dx = r (w g - x r * mean(w g * x r))
#include <type_traits>
#include "roomie_rope.cuh"

namespace roomie {

// Rows are split like rope's: a thread has one unit - two chunks of kV elements that turn together, or two neighbouring ones of the part that
// is not turned - of some heads of one token, so its angles and weights are fetched once for all of them; the `lanes` threads of a row lie
// side by side in a warp and add their squares up by shuffles.  Queries and keys are the two sides of one launch.
struct NormSide {
    const void *x, *g, *w;          // rows, gradient of the results (backward), weights
    void* y;                        // results, or the gradient of the rows
    long long x_token, x_head, g_token, g_head, y_token, y_head;
    uint32_t heads, groups;
};
struct NormArgs {
    NormSide side[2];
    RopeView rope;
    const int32_t* positions;
    uint32_t tokens, dim, units, lanes, slots;      // slots: rows of head groups that the grid takes at a time
    int32_t weight_type;
    float eps, inverse_dim;
    float* partial;                                 // backward: [blocks][2][dim] sums of the weights' gradients
};

constexpr int kNormThreads = 128;

template <int kBytes> struct RawOf { using type = uint4; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<2> { using type = uint16_t; };
template <class T, int kV> using Raw = typename RawOf<kV * (int)sizeof(T)>::type;

// What a thread knows of its unit: where its chunks lie, and whether they are there and turn.
struct Unit {
    uint32_t a, b;
    bool on, two, turn;
};
template <int kV, bool kPairs> __device__ __forceinline__ Unit unit_of(const NormArgs& n, uint32_t unit) {
    Unit u;
    const uint32_t half = n.rope.rot / 2, n_rot = half / kV;
    u.on = unit < n.units;
    u.turn = unit < n_rot;
    u.a = u.turn ? (kPairs ? 2 * unit * kV : unit * kV) : n.rope.rot + (unit - n_rot) * 2 * kV;
    u.b = u.turn && !kPairs ? u.a + half : u.a + kV;
    u.two = u.on && u.b < n.dim;
    return u;
}

// A unit's 2 kV elements as two vectors whose i-th elements turn together (where the unit turns), two float32 a register pair.  A vector of one
// element is a pair whose second is 0.
template <int kV> constexpr int kTwos = (kV + 1) / 2;
template <int kV> struct Elements {
    uint64_t a[kTwos<kV>], b[kTwos<kV>];
};
// from a unit's elements as they lie in memory, and back
template <int kV, bool kPairs> __device__ __forceinline__ Elements<kV> vectors(const float* x) {
    Elements<kV> v;
#pragma unroll
    for (int i = 0; i < kTwos<kV>; ++i) {
        if constexpr (kV == 1) {
            v.a[0] = pair(x[0], 0.0f);
            v.b[0] = pair(x[1], 0.0f);
        } else if constexpr (kPairs) {
            v.a[i] = pair(x[4 * i], x[4 * i + 2]);
            v.b[i] = pair(x[4 * i + 1], x[4 * i + 3]);
        } else {
            v.a[i] = pair(x[2 * i], x[2 * i + 1]);
            v.b[i] = pair(x[kV + 2 * i], x[kV + 2 * i + 1]);
        }
    }
    return v;
}
template <int kV, bool kPairs> __device__ __forceinline__ void scalars(const Elements<kV>& v, float* x) {
#pragma unroll
    for (int i = 0; i < kTwos<kV>; ++i) {
        float none;
        if constexpr (kV == 1) {
            split(v.a[0], x[0], none);
            split(v.b[0], x[1], none);
        } else if constexpr (kPairs) {
            split(v.a[i], x[4 * i], x[4 * i + 2]);
            split(v.b[i], x[4 * i + 1], x[4 * i + 3]);
        } else {
            split(v.a[i], x[2 * i], x[2 * i + 1]);
            split(v.b[i], x[kV + 2 * i], x[kV + 2 * i + 1]);
        }
    }
}
template <class T, int kV> struct Loaded {
    Raw<T, kV> a, b;
};
template <class T, int kV> __device__ __forceinline__ Loaded<T, kV> load_unit(const T* p, const Unit& u) {
    Loaded<T, kV> r = {};
    if (u.on) r.a = *reinterpret_cast<const Raw<T, kV>*>(p + u.a);
    if (u.two) r.b = *reinterpret_cast<const Raw<T, kV>*>(p + u.b);
    return r;
}
template <class T, int kV, bool kPairs> __device__ __forceinline__ Elements<kV> widened(const Loaded<T, kV>& r) {
    float x[2 * kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        x[i] = to_f32(reinterpret_cast<const T*>(&r.a)[i]);
        x[kV + i] = to_f32(reinterpret_cast<const T*>(&r.b)[i]);
    }
    return vectors<kV, kPairs>(x);
}
template <class T, int kV, bool kPairs> __device__ __forceinline__ void store_unit(T* p, const Unit& u, const Elements<kV>& v) {
    float x[2 * kV];
    scalars<kV, kPairs>(v, x);
    Loaded<T, kV> r;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        reinterpret_cast<T*>(&r.a)[i] = from_f32<T>(x[i]);
        reinterpret_cast<T*>(&r.b)[i] = from_f32<T>(x[kV + i]);
    }
    if (u.on) *reinterpret_cast<Raw<T, kV>*>(p + u.a) = r.a;
    if (u.two) *reinterpret_cast<Raw<T, kV>*>(p + u.b) = r.b;
}
// kV weights in a row, 16 bytes at a time where they are aligned to that: a chunk starts at a multiple of kV.
template <class W, int kV> __device__ __forceinline__ void weights_at(const W* w, float* x) {
    if constexpr (kV * sizeof(W) >= 16) {
        if ((reinterpret_cast<uintptr_t>(w) & 15) == 0) {
#pragma unroll
            for (int i = 0; i < kV; i += 16 / (int)sizeof(W)) {
                const uint4 four = *reinterpret_cast<const uint4*>(w + i);
#pragma unroll
                for (int j = 0; j < 16 / (int)sizeof(W); ++j) x[i + j] = to_f32(reinterpret_cast<const W*>(&four)[j]);
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) x[i] = to_f32(w[i]);
}
template <class W, int kV> __device__ __forceinline__ void unit_weights(const void* w, const Unit& u, float* x) {
    if (u.on) weights_at<W, kV>(static_cast<const W*>(w) + u.a, x);
    if (u.two) weights_at<W, kV>(static_cast<const W*>(w) + u.b, x + kV);
}
template <int kV, bool kPairs> __device__ __forceinline__ Elements<kV> load_weights(const void* w, int32_t type, const Unit& u) {
    float x[2 * kV];
#pragma unroll
    for (int i = 0; i < 2 * kV; ++i) x[i] = !w && (i < kV ? u.on : u.two) ? 1.0f : 0.0f;
    if (!w) return vectors<kV, kPairs>(x);
    if (type == ROOMIE_F32) unit_weights<float, kV>(w, u, x);
    else if (type == ROOMIE_F16) unit_weights<__half, kV>(w, u, x);
    else unit_weights<__nv_bfloat16, kV>(w, u, x);
    return vectors<kV, kPairs>(x);
}
// cosines and sines of a unit's pairs; 1 and 0 where it does not turn
template <int kV> __device__ __forceinline__ Elements<kV> turns_of(const NormArgs& n, uint32_t unit, const Unit& u, int32_t position) {
    float2 cs[2 * kTwos<kV>];
#pragma unroll
    for (int i = 0; i < 2 * kTwos<kV>; ++i)
        cs[i] = u.turn && i < kV ? rope_turn(n.rope.frequency[unit * kV + i], position, n.rope.amplitude) : make_float2(1.0f, 0.0f);
    Elements<kV> v;
#pragma unroll
    for (int i = 0; i < kTwos<kV>; ++i) {
        v.a[i] = pair(cs[2 * i].x, cs[2 * i + 1].x);
        v.b[i] = pair(cs[2 * i].y, cs[2 * i + 1].y);
    }
    return v;
}
__device__ __forceinline__ uint64_t both(float x) { return pair(x, x); }
__device__ __forceinline__ uint64_t minus(uint64_t x) { return x ^ 0x8000000080000000ull; }
template <int kV> __device__ __forceinline__ void multiply(Elements<kV>& v, float f) {
#pragma unroll
    for (int i = 0; i < kTwos<kV>; ++i) {
        v.a[i] = mul2(v.a[i], both(f));
        v.b[i] = mul2(v.b[i], both(f));
    }
}
template <int kV> __device__ __forceinline__ uint64_t dot(const Elements<kV>& v, const Elements<kV>& w, uint64_t sum) {
#pragma unroll
    for (int i = 0; i < kTwos<kV>; ++i) sum = fma2(v.b[i], w.b[i], fma2(v.a[i], w.a[i], sum));
    return sum;
}

// The sum over the lanes of a row.
__device__ __forceinline__ float row_sum(uint64_t twos, uint32_t lanes, uint32_t mask) {
    float x, y;
    split(twos, x, y);
    x += y;
#pragma unroll
    for (uint32_t d = 16; d > 0; d >>= 1)
        if (d < lanes) x += __shfl_xor_sync(mask, x, d);
    return x;
}

// Squares of values above 2^64 leave float32: such a row is taken times 2^-80.
constexpr float kLess = 8.271806125530277e-25f;

// What a warp's threads know of their place: its lanes of a row, its head group and side.
struct Place {
    uint32_t first, mask, slot, group, all;
    bool second;
};
__device__ __forceinline__ Place place_of(const NormArgs& n) {
    Place p;
    const uint32_t lane = threadIdx.x & 31;
    p.first = lane & ~(n.lanes - 1);
    p.mask = n.lanes == 32 ? 0xffffffffu : ((1u << n.lanes) - 1) << p.first;
    p.all = n.side[0].groups + n.side[1].groups;
    const uint32_t flat = blockIdx.x * (kNormThreads / n.lanes) + threadIdx.x / n.lanes;
    p.slot = flat / p.all;
    p.group = flat - p.slot * p.all;
    p.second = p.group >= n.side[0].groups;
    if (p.second) p.group -= n.side[0].groups;
    return p;
}

// Bound by memory: two float32 an instruction, weights and turns multiplied once for all heads of a thread, rows under way three heads ahead (16384 tokens
// x 40 heads x 128 in bf16, 336 MB: 64 us, 5220 GB/s; the next head's row alone, in registers: 77; seven heads ahead: 87; each element on its own: 101).
// Five blocks an SM; the spills that this takes lie in front of the loop over heads (six: 69 us, eight: 94; 8-byte chunks: 125).  Of smaller chunks six,
// whose registers suffice (3001 tokens x 6 heads x 65: 18 us, with five 21).
constexpr int kAhead = 3;
template <class T, int kV, int kPer, bool kPairs>
__global__ void __launch_bounds__(kNormThreads, kV == 8 ? 5 : 6) norm_kernel(NormArgs n) {
    const Place p = place_of(n);
    if (p.slot >= n.slots) return;
    const NormSide s = p.second ? n.side[1] : n.side[0];
    Unit u[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) u[k] = unit_of<kV, kPairs>(n, (threadIdx.x & 31) - p.first + k * n.lanes);
    const long long x_step = s.groups * s.x_head, y_step = s.groups * s.y_head;
    // Chunks of 8 or 16 bytes come kAhead heads before they are needed, to a thread's own part of shared memory; smaller ones one head, to registers.
    constexpr bool kRing = kPer == 1 && sizeof(Raw<T, kV>) >= 8;
    __shared__ Raw<T, kV> ring[kRing ? kAhead + 1 : 1][2][kRing ? kNormThreads : 1];
    auto fetch = [&](const T* from, bool there, int stage) {
        if constexpr (kRing) {
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(&ring[stage][0][threadIdx.x]);
            if (there && u[0].on)
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from + u[0].a), "n"((int)sizeof(Raw<T, kV>)) : "memory");
            if (there && u[0].two)
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to + (uint32_t)(kNormThreads * sizeof(Raw<T, kV>))), "l"(from + u[0].b), "n"((int)sizeof(Raw<T, kV>)) : "memory");
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    if constexpr (kRing)
#pragma unroll
        for (int i = 0; i <= kAhead; ++i) {                          // what is not there stays 0
            if (!u[0].on) ring[i][0][threadIdx.x] = {};
            if (!u[0].two) ring[i][1][threadIdx.x] = {};
        }
    for (uint32_t token = p.slot; token < n.tokens; token += n.slots) {
        const T* x = static_cast<const T*>(s.x) + (long long)token * s.x_token + (long long)p.group * s.x_head;
        T* y = static_cast<T*>(s.y) + (long long)token * s.y_token + (long long)p.group * s.y_head;
        Loaded<T, kV> next[kPer];
        if constexpr (kRing) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(x + i * x_step, p.group + i * s.groups < s.heads, i);
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) next[k] = load_unit<T, kV>(x, u[k]);
        }
        // y_a = x_a own.a - x_b cross.b, y_b = x_b own.b + x_a cross.a, each with r
        const int32_t position = n.rope.rot ? n.positions[token] : 0;
        Elements<kV> own[kPer], cross[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const Elements<kV> w = load_weights<kV, kPairs>(s.w, n.weight_type, u[k]);
            const Elements<kV> turn = turns_of<kV>(n, (threadIdx.x & 31) - p.first + k * n.lanes, u[k], position);
#pragma unroll
            for (int i = 0; i < kTwos<kV>; ++i) {
                own[k].a[i] = mul2(turn.a[i], w.a[i]);
                own[k].b[i] = mul2(turn.a[i], w.b[i]);
                cross[k].a[i] = mul2(turn.b[i], w.a[i]);
                cross[k].b[i] = minus(mul2(turn.b[i], w.b[i]));
            }
        }
        int stage = 0;
        for (uint32_t head = p.group; head < s.heads; head += s.groups) {
            Elements<kV> v[kPer];
            uint64_t sum = 0;
            if constexpr (kRing) {
                fetch(x + kAhead * x_step, head + kAhead * s.groups < s.heads, (stage + kAhead) & kAhead);
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
                next[0].a = ring[stage][0][threadIdx.x];
                next[0].b = ring[stage][1][threadIdx.x];
                stage = (stage + 1) & kAhead;
            }
            x += x_step;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                v[k] = widened<T, kV, kPairs>(next[k]);
                if constexpr (!kRing)
                    if (head + s.groups < s.heads) next[k] = load_unit<T, kV>(x, u[k]);     // the next head's
                sum = dot<kV>(v[k], v[k], sum);
            }
            float square = row_sum(sum, n.lanes, p.mask), eps = n.eps;
            if (square == INFINITY) {                                 // the same in all lanes of the row
                sum = 0;
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    multiply<kV>(v[k], kLess);
                    sum = dot<kV>(v[k], v[k], sum);
                }
                square = row_sum(sum, n.lanes, p.mask);
                eps *= kLess * kLess;
            }
            const float r = rsqrtf(fmaf(square, n.inverse_dim, eps));
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                multiply<kV>(v[k], r);
                Elements<kV> z;
#pragma unroll
                for (int i = 0; i < kTwos<kV>; ++i) {
                    z.a[i] = fma2(v[k].a[i], own[k].a[i], mul2(v[k].b[i], cross[k].b[i]));
                    z.b[i] = fma2(v[k].b[i], own[k].b[i], mul2(v[k].a[i], cross[k].a[i]));
                }
                store_unit<T, kV, kPairs>(y, u[k], z);
            }
            y += y_step;
        }
    }
}

template <class T, int kV, int kPer, bool kPairs>
__global__ void __launch_bounds__(kNormThreads, 4) norm_grad_kernel(NormArgs n) {
    extern __shared__ float sums[];                                  // [head groups of the block][dim]
    const Place p = place_of(n);
    const NormSide s = p.second ? n.side[1] : n.side[0];
    Unit u[kPer];
    Elements<kV> w[kPer], dw[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        u[k] = unit_of<kV, kPairs>(n, (threadIdx.x & 31) - p.first + k * n.lanes);
        w[k] = load_weights<kV, kPairs>(s.w, n.weight_type, u[k]);
        dw[k] = {};
    }
    const long long x_step = s.groups * s.x_head, g_step = s.groups * s.g_head, y_step = s.groups * s.y_head;
    if (p.slot < n.slots)
        for (uint32_t token = p.slot; token < n.tokens; token += n.slots) {
            const T* x = static_cast<const T*>(s.x) + (long long)token * s.x_token + (long long)p.group * s.x_head;
            const T* g = static_cast<const T*>(s.g) + (long long)token * s.g_token + (long long)p.group * s.g_head;
            T* y = static_cast<T*>(s.y) + (long long)token * s.y_token + (long long)p.group * s.y_head;
            const int32_t position = n.rope.rot ? n.positions[token] : 0;
            Elements<kV> turn[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) turn[k] = turns_of<kV>(n, (threadIdx.x & 31) - p.first + k * n.lanes, u[k], position);
            for (uint32_t head = p.group; head < s.heads; head += s.groups) {
                Elements<kV> v[kPer], back[kPer];                     // the rows, and their gradients turned back
                uint64_t sum = 0, along = 0;
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    const Loaded<T, kV> lx = load_unit<T, kV>(x, u[k]), lg = load_unit<T, kV>(g, u[k]);
                    v[k] = widened<T, kV, kPairs>(lx);
                    const Elements<kV> d = widened<T, kV, kPairs>(lg);
#pragma unroll
                    for (int i = 0; i < kTwos<kV>; ++i) {
                        back[k].a[i] = fma2(d.a[i], turn[k].a[i], mul2(d.b[i], turn[k].b[i]));
                        back[k].b[i] = fma2(d.b[i], turn[k].a[i], minus(mul2(d.a[i], turn[k].b[i])));
                    }
                }
                auto sums_of = [&] {
                    sum = along = 0;
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {
                        sum = dot<kV>(v[k], v[k], sum);
#pragma unroll
                        for (int i = 0; i < kTwos<kV>; ++i)
                            along = fma2(mul2(back[k].a[i], w[k].a[i]), v[k].a[i], fma2(mul2(back[k].b[i], w[k].b[i]), v[k].b[i], along));
                    }
                };
                sums_of();
                float square = row_sum(sum, n.lanes, p.mask), eps = n.eps, less = 1.0f;
                if (square == INFINITY) {                             // the same in all lanes of the row
#pragma unroll
                    for (int k = 0; k < kPer; ++k) multiply<kV>(v[k], kLess);
                    sums_of();
                    square = row_sum(sum, n.lanes, p.mask);
                    less = kLess;
                    eps *= kLess * kLess;
                }
                const float r = rsqrtf(fmaf(square, n.inverse_dim, eps));
                const uint64_t mean = both(-row_sum(along, n.lanes, p.mask) * r * n.inverse_dim);
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    multiply<kV>(v[k], r);
                    Elements<kV> d;
#pragma unroll
                    for (int i = 0; i < kTwos<kV>; ++i) {
                        dw[k].a[i] = fma2(back[k].a[i], v[k].a[i], dw[k].a[i]);
                        dw[k].b[i] = fma2(back[k].b[i], v[k].b[i], dw[k].b[i]);
                        d.a[i] = fma2(v[k].a[i], mean, mul2(back[k].a[i], w[k].a[i]));
                        d.b[i] = fma2(v[k].b[i], mean, mul2(back[k].b[i], w[k].b[i]));
                    }
                    multiply<kV>(d, r * less);
                    store_unit<T, kV, kPairs>(y, u[k], d);
                }
                x += x_step;
                g += g_step;
                y += y_step;
            }
        }
    // the block's sums, head group after head group
    const uint32_t mine = threadIdx.x / n.lanes, here = kNormThreads / n.lanes;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        float d[2 * kV];
        scalars<kV, kPairs>(dw[k], d);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            if (u[k].on) sums[mine * n.dim + u[k].a + i] = d[i];
            if (u[k].two) sums[mine * n.dim + u[k].b + i] = d[kV + i];
        }
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < 2 * n.dim; d += kNormThreads) {
        const uint32_t side = d >= n.dim, at = d - side * n.dim;
        float total = 0.0f;
        for (uint32_t i = 0; i < here; ++i) {
            const uint32_t f = (blockIdx.x * here + i) % p.all;
            if ((f >= n.side[0].groups) == (side != 0)) total += sums[i * n.dim + at];
        }
        n.partial[(size_t)blockIdx.x * 2 * n.dim + d] = total;
    }
}

// The blocks' sums, 32 elements a block, in an order of their own: strides of 32 blocks, then the 32 of those.
__global__ void __launch_bounds__(1024) norm_weights_kernel(const float* partial, uint32_t blocks, uint32_t dim, void* dq, void* dk, int32_t type) {
    __shared__ float sh[32][33];
    grid_dependency_wait();
    const uint32_t c = threadIdx.x & 31, r = threadIdx.x >> 5, d = blockIdx.x * 32 + c;
    float x = 0.0f;
    if (d < 2 * dim)
#pragma unroll 8
        for (uint32_t b = r; b < blocks; b += 32) x += partial[(size_t)b * 2 * dim + d];
    sh[r][c] = x;
    __syncthreads();
    if (r) return;
    x = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) x += sh[i][c];
    if (d >= 2 * dim) return;
    void* to = d < dim ? dq : dk;
    const uint32_t at = d < dim ? d : d - dim;
    if (!to) return;
    if (type == ROOMIE_F32) static_cast<float*>(to)[at] = x;
    else if (type == ROOMIE_F16) static_cast<__half*>(to)[at] = __float2half_rn(x);
    else static_cast<__nv_bfloat16*>(to)[at] = __float2bfloat16_rn(x);
}

constexpr uint32_t kNormBlocksPerSm = 8;             // at most: the backward pass leaves a row of sums for each

template <class T, int kV, int kPer, bool kGrad> static int launch_norm(NormArgs n, uint32_t blocks, size_t smem, cudaStream_t st) {
    void (*k)(NormArgs);
    if (kGrad) k = n.rope.interleaved ? norm_grad_kernel<T, kV, kPer, true> : norm_grad_kernel<T, kV, kPer, false>;
    else k = n.rope.interleaved ? norm_kernel<T, kV, kPer, true> : norm_kernel<T, kV, kPer, false>;
    return launch(kGrad ? "qk_norm_rope_grad" : "qk_norm_rope", k, dim3(blocks), dim3(kNormThreads), smem, st, false, n);
}

// The widest chunks that divide a row's parts and that all rows are aligned to.
static uint32_t chunk_of(const NormArgs& n, uint32_t e, uint32_t align) {
    for (uint32_t bytes = 16; bytes > e; bytes /= 2) {
        const uint32_t v = bytes / e;
        if (bytes == 4 || (bytes == 8 && e == 4)) continue;
        if (align % bytes == 0 && (n.rope.rot / 2) % v == 0 && (n.dim - n.rope.rot) % v == 0) return v;
    }
    return 1;
}

template <class T, bool kGrad> static int run_norm(NormArgs n, uint32_t align, uint32_t* blocks_out, cudaStream_t st) {
    const uint32_t v = chunk_of(n, sizeof(T), align), sms = (uint32_t)sm_count();
    n.units = n.rope.rot / 2 / v + ((n.dim - n.rope.rot) / v + 1) / 2;
    n.lanes = 1;
    while (n.lanes < n.units && n.lanes < 32) n.lanes *= 2;
    // Head groups: a thread's weights and turns cost as much as some heads, so it should have eight heads or more (16384 tokens x 40 heads: with sixteen
    // 2 us more; rows one head ahead: 77, with four heads 83), unless there are too few rows to fill the GPU.
    const unsigned long long one = (unsigned long long)n.tokens * n.lanes;
    for (NormSide& s : n.side) {
        unsigned long long g = (2048ull * sms + one - 1) / one, few = 256ull * sms / one;
        if (g > s.heads / 8) g = s.heads / 8;
        if (g < few) g = few;
        if (g > s.heads) g = s.heads;
        if (kGrad && g > (unsigned long long)sms * kNormBlocksPerSm) g = (unsigned long long)sms * kNormBlocksPerSm;   // all groups fit the grid below
        s.groups = s.heads == 0 ? 0 : (uint32_t)(g < 1 ? 1 : g);
    }
    const uint32_t here = kNormThreads / n.lanes, all = n.side[0].groups + n.side[1].groups;   // here: 4 to 128
    unsigned long long blocks = ((unsigned long long)n.tokens * all + here - 1) / here;
    if (kGrad && blocks > (unsigned long long)sms * kNormBlocksPerSm) blocks = (unsigned long long)sms * kNormBlocksPerSm;
    if (blocks > 0x3fffffffull / here) return ROOMIE_ERR_INVALID_ARG;
    n.slots = (uint32_t)(blocks * here / all);
    if (blocks_out) *blocks_out = (uint32_t)blocks;
    const size_t smem = kGrad ? (size_t)here * n.dim * sizeof(float) : 0;
    if constexpr (sizeof(T) == 2) {
        if (v == 8) return launch_norm<T, 8, 1, kGrad>(n, (uint32_t)blocks, smem, st);
        if (v == 4) return launch_norm<T, 4, 1, kGrad>(n, (uint32_t)blocks, smem, st);
    } else {
        if (v == 4) return launch_norm<T, 4, 1, kGrad>(n, (uint32_t)blocks, smem, st);
    }
    return launch_norm<T, 1, 4, kGrad>(n, (uint32_t)blocks, smem, st);
}

template <bool kGrad> static int norm_type(const NormArgs& n, int32_t type, uint32_t align, uint32_t* blocks, cudaStream_t st) {
    if (type == ROOMIE_F32) return run_norm<float, kGrad>(n, align, blocks, st);
    if (type == ROOMIE_F16) return run_norm<__half, kGrad>(n, align, blocks, st);
    return run_norm<__nv_bfloat16, kGrad>(n, align, blocks, st);
}

// the largest power of two up to 16 that all of a tensor's rows are aligned to
static uint32_t rows_alignment(const roomie_rows& r, uint32_t tokens, uint32_t heads) {
    const unsigned long long e = size_of_type(r.type);
    unsigned long long bits = reinterpret_cast<uintptr_t>(r.data) | 16u;
    if (tokens > 1) bits |= (unsigned long long)r.token_stride * e;
    if (heads > 1) bits |= (unsigned long long)r.head_stride * e;
    return (uint32_t)(bits & (~bits + 1));
}

}  // namespace roomie

using namespace roomie;

static int norm_check(const roomie_rope_table* table, float eps, uint32_t head_dim, const int32_t* positions, uint32_t tokens, uint32_t q_heads,
                      uint32_t k_heads, int32_t weight_type) {
    if (head_dim == 0 || head_dim > 256 || !(eps > 0.0f) || !(eps < INFINITY) || !known_type(weight_type) || (table && !rope_table_valid(table, head_dim)))
        return ROOMIE_ERR_INVALID_ARG;
    if (tokens && q_heads + (unsigned long long)k_heads && table && !positions) return ROOMIE_ERR_INVALID_ARG;
    if (((unsigned long long)q_heads + k_heads) * (tokens ? tokens : 1) > 0x3fffffffull) return ROOMIE_ERR_INVALID_ARG;
    return ROOMIE_OK;
}
static bool weight_aligned(const void* w, int32_t type) { return reinterpret_cast<uintptr_t>(w) % size_of_type(type) == 0; }

static NormArgs norm_args(const roomie_rope_table* table, float eps, uint32_t tokens, uint32_t dim, const int32_t* positions, int32_t weight_type) {
    NormArgs n = {};
    n.rope = table ? RopeView{table->frequency, table->rotary_dim, table->interleaved, table->amplitude} : RopeView{nullptr, 0, 0, 1.0f};
    n.positions = positions;
    n.tokens = tokens;
    n.dim = dim;
    n.weight_type = weight_type;
    n.eps = eps;
    n.inverse_dim = 1.0f / (float)dim;
    return n;
}

extern "C" int roomie_qk_norm_rope(const roomie_rope_table* table, float eps, uint32_t tokens, uint32_t head_dim, const int32_t* positions,
                                   int32_t weight_type, uint32_t q_heads, const roomie_rows* q, const void* q_weight, const roomie_rows* q_out,
                                   uint32_t k_heads, const roomie_rows* k, const void* k_weight, const roomie_rows* k_out, void* stream) {
    const int rc = norm_check(table, eps, head_dim, positions, tokens, q_heads, k_heads, weight_type);
    if (rc != ROOMIE_OK) return rc;
    if (tokens == 0 || (q_heads == 0 && k_heads == 0)) return ROOMIE_OK;
    NormArgs n = norm_args(table, eps, tokens, head_dim, positions, weight_type);
    const roomie_rows *x[2] = {q, k}, *y[2] = {q_out, k_out};
    const void* w[2] = {q_weight, k_weight};
    const uint32_t heads[2] = {q_heads, k_heads};
    uint32_t align = 16;
    int32_t type = -1;
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0) continue;
        if (!rows_valid(x[i]) || !rows_valid(y[i]) || x[i]->type != y[i]->type || (type >= 0 && x[i]->type != type) || !weight_aligned(w[i], weight_type) ||
            !rows_apart(*y[i], tokens, heads[i], head_dim))
            return ROOMIE_ERR_INVALID_ARG;
        if (x[i]->data == y[i]->data && (x[i]->token_stride != y[i]->token_stride || x[i]->head_stride != y[i]->head_stride)) return ROOMIE_ERR_INVALID_ARG;
        type = x[i]->type;
        for (const roomie_rows* r : {x[i], y[i]}) {
            const uint32_t own = rows_alignment(*r, tokens, heads[i]);
            if (own < align) align = own;
        }
        NormSide& s = n.side[i];
        s.x = x[i]->data; s.y = y[i]->data; s.w = w[i]; s.heads = heads[i];
        s.x_token = x[i]->token_stride; s.x_head = x[i]->head_stride; s.y_token = y[i]->token_stride; s.y_head = y[i]->head_stride;
    }
    return norm_type<false>(n, type, align, nullptr, static_cast<cudaStream_t>(stream));
}

extern "C" size_t roomie_qk_norm_rope_workspace_bytes(uint32_t head_dim) {
    if (head_dim == 0 || head_dim > 256) return 0;
    return (size_t)sm_count() * kNormBlocksPerSm * 2 * head_dim * sizeof(float);
}

extern "C" int roomie_qk_norm_rope_grad(const roomie_rope_table* table, float eps, uint32_t tokens, uint32_t head_dim, const int32_t* positions,
                                        int32_t weight_type, uint32_t q_heads, const roomie_rows* q, const void* q_weight, const roomie_rows* gq,
                                        const roomie_rows* dq, void* dq_weight, uint32_t k_heads, const roomie_rows* k, const void* k_weight,
                                        const roomie_rows* gk, const roomie_rows* dk, void* dk_weight, void* workspace, size_t workspace_bytes,
                                        void* stream) {
    int rc = norm_check(table, eps, head_dim, positions, tokens, q_heads, k_heads, weight_type);
    if (rc != ROOMIE_OK) return rc;
    if (!weight_aligned(dq_weight, weight_type) || !weight_aligned(dk_weight, weight_type)) return ROOMIE_ERR_INVALID_ARG;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 3u)) return ROOMIE_ERR_INVALID_ARG;
    if (workspace_bytes < roomie_qk_norm_rope_workspace_bytes(head_dim)) return ROOMIE_ERR_CAPACITY;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    NormArgs n = norm_args(table, eps, tokens, head_dim, positions, weight_type);
    n.partial = static_cast<float*>(workspace);
    uint32_t blocks = 0;
    if (tokens && (q_heads || k_heads)) {
        const roomie_rows *x[2] = {q, k}, *g[2] = {gq, gk}, *d[2] = {dq, dk};
        const void* w[2] = {q_weight, k_weight};
        const uint32_t heads[2] = {q_heads, k_heads};
        uint32_t align = 16;
        int32_t type = -1;
        for (int i = 0; i < 2; ++i) {
            if (heads[i] == 0) continue;
            for (const roomie_rows* r : {x[i], g[i], d[i]}) {
                if (!rows_valid(r) || (type >= 0 && r->type != type)) return ROOMIE_ERR_INVALID_ARG;
                type = r->type;
                const uint32_t own = rows_alignment(*r, tokens, heads[i]);
                if (own < align) align = own;
            }
            if (!weight_aligned(w[i], weight_type) || !rows_apart(*d[i], tokens, heads[i], head_dim)) return ROOMIE_ERR_INVALID_ARG;
            NormSide& s = n.side[i];
            s.x = x[i]->data; s.g = g[i]->data; s.y = d[i]->data; s.w = w[i]; s.heads = heads[i];
            s.x_token = x[i]->token_stride; s.x_head = x[i]->head_stride; s.g_token = g[i]->token_stride; s.g_head = g[i]->head_stride;
            s.y_token = d[i]->token_stride; s.y_head = d[i]->head_stride;
        }
        rc = norm_type<true>(n, type, align, &blocks, st);
        if (rc != ROOMIE_OK) return rc;
    }
    if (!dq_weight && !dk_weight) return ROOMIE_OK;
    return launch("qk_norm_rope_weights", norm_weights_kernel, dim3((2 * head_dim + 31) / 32), dim3(1024), 0, st, true, n.partial, blocks, head_dim, dq_weight,
                  dk_weight, weight_type);
}
