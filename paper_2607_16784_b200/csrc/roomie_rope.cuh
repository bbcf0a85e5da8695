// Rotary positions: the body that roomie_rope's kernel and the append kernel's query part share.
#pragma once
#include "roomie_serving.cuh"

namespace roomie {

struct RopeView {
    const uint64_t* frequency;
    uint32_t rot;            // rotated elements of a head
    int32_t interleaved;
    float amplitude;
};

struct HeadRows {            // element strides
    const void* x;
    void* y;
    long long x_token, x_head, y_token, y_head;
};

// What one thread does: unit `unit` of heads head, head + step, ... of one token.  A unit is kV elements; a row has rot/(2*kV) pairs of
// units that are rotated and, unless it is done in place, (dim - rot)/kV units that are copied.  kV = 16 bytes, or 1 when some row is
// not 16-byte aligned or the parts do not divide into such units.  The thread works out its own kV cosines and sines (some 25
// instructions each) once for all its heads: nothing is shared, nobody waits.
template <class T, int kV, bool kPairs, int kUnroll>
__device__ __forceinline__ void rope_heads(const HeadRows& io, const RopeView& rope, uint32_t token, int32_t position, bool inverse,
                                           uint32_t unit, uint32_t head, uint32_t step, uint32_t heads) {
    const uint32_t half = rope.rot / 2, n_rot = half / kV;
    using Raw = typename std::conditional<kV == 1, T, uint4>::type;
    const bool turn = unit < n_rot;
    const uint32_t a = !turn ? rope.rot + (unit - n_rot) * kV : kPairs ? 2 * unit * kV : unit * kV;
    const uint32_t b = kPairs ? a + kV : a + half;
    float2 w[kV];
    if (turn)
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            w[i] = rope_turn(rope.frequency[unit * kV + i], position, rope.amplitude);
            if (inverse) w[i].y = -w[i].y;
        }
    const T* x = static_cast<const T*>(io.x) + token * io.x_token + head * io.x_head;
    T* y = static_cast<T*>(io.y) + token * io.y_token + head * io.y_head;
    for (uint32_t h = head; h < heads; h += step * kUnroll) {
        Raw ra[kUnroll], rb[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (h + u * step < heads) {
                const T* p = x + (long long)(u * step) * io.x_head;
                ra[u] = *reinterpret_cast<const Raw*>(p + a);
                if (turn) rb[u] = *reinterpret_cast<const Raw*>(p + b);
            }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (h + u * step >= heads) break;
            T* p = y + (long long)(u * step) * io.y_head;
            if (!turn) {
                *reinterpret_cast<Raw*>(p + a) = ra[u];
                continue;
            }
            if constexpr (kV == 1) {
                const float e = to_f32(ra[u]), o = to_f32(rb[u]);
                p[a] = from_f32<T>(__fsub_rn(__fmul_rn(e, w->x), __fmul_rn(o, w->y)));
                p[b] = from_f32<T>(__fadd_rn(__fmul_rn(o, w->x), __fmul_rn(e, w->y)));
            } else {
                float xa[2 * kV];
                unpack<T>(ra[u], xa);
                unpack<T>(rb[u], xa + kV);
                if constexpr (kPairs) {
#pragma unroll
                    for (int i = 0; i < kV; ++i) {                        // pairs (2i, 2i+1) of the 2*kV elements
                        const float e = xa[2 * i], o = xa[2 * i + 1];
                        xa[2 * i] = __fsub_rn(__fmul_rn(e, w[i].x), __fmul_rn(o, w[i].y));
                        xa[2 * i + 1] = __fadd_rn(__fmul_rn(o, w[i].x), __fmul_rn(e, w[i].y));
                    }
                } else {
                    rotate_half<kV>(xa, xa + kV, w);
                }
                *reinterpret_cast<uint4*>(p + a) = pack<T>(xa);
                *reinterpret_cast<uint4*>(p + b) = pack<T>(xa + kV);
            }
        }
        x += (long long)(step * kUnroll) * io.x_head;
        y += (long long)(step * kUnroll) * io.y_head;
    }
}

// The same units passed on as they are, infinities and all.
template <class T, int kV, bool kPairs>
__device__ __forceinline__ void rope_copy(const HeadRows& io, const RopeView& rope, uint32_t token, uint32_t unit, uint32_t head, uint32_t step,
                                       uint32_t heads) {
    const uint32_t half = rope.rot / 2, n_rot = half / kV;
    using Raw = typename std::conditional<kV == 1, T, uint4>::type;
    const bool turn = unit < n_rot;
    const uint32_t a = !turn ? rope.rot + (unit - n_rot) * kV : kPairs ? 2 * unit * kV : unit * kV;
    const uint32_t b = kPairs ? a + kV : a + half;
    for (uint32_t h = head; h < heads; h += step) {
        const T* x = static_cast<const T*>(io.x) + token * io.x_token + h * io.x_head;
        T* y = static_cast<T*>(io.y) + token * io.y_token + h * io.y_head;
        *reinterpret_cast<Raw*>(y + a) = *reinterpret_cast<const Raw*>(x + a);
        if (turn) *reinterpret_cast<Raw*>(y + b) = *reinterpret_cast<const Raw*>(x + b);
    }
}

// Threads are (token, head group, unit), units fastest.  Each works out its own angles, so it should have four heads or more (1000 tokens
// x 40 heads: 8.3 us, with one head a thread 10.4); up to that, groups enough for twice the GPU's threads (16384 tokens: 61.7 us, with
// half as many 64.7); and for few tokens, where only latency counts, as many groups as it takes to give every SM 256 threads.
struct RopeSplit {
    uint32_t units, groups;
    unsigned long long threads;
};
inline RopeSplit rope_split(uint32_t tokens, uint32_t heads, uint32_t dim, uint32_t rot, uint32_t kv, bool in_place, uint32_t sms) {
    RopeSplit s;
    s.units = rot / 2 / kv + (in_place ? 0 : (dim - rot) / kv);
    const unsigned long long one = (unsigned long long)tokens * s.units;
    if (one == 0) return {s.units, 1, 0};                                 // in place, and nothing is rotated
    unsigned long long g = (4096ull * sms + one - 1) / one, few = 256ull * sms / one;
    if (g > heads / 4) g = heads / 4;
    if (g < few) g = few;
    s.groups = (uint32_t)(g < 1 ? 1 : g > heads ? heads : g);
    s.threads = one * s.groups;
    return s;
}

// The parts of a row divide into units of 16 bytes.
inline bool rope_units_of_16(uint32_t rot, uint32_t dim, int32_t type, bool interleaved) {
    const uint32_t v = 16u / (uint32_t)size_of_type(type);
    return (rot / 2) % v == 0 && (dim - rot) % v == 0;
}

inline bool rope_table_valid(const roomie_rope_table* t, uint32_t head_dim) {
    return t && t->frequency && t->rotary_dim >= 2 && t->rotary_dim % 2 == 0 && t->rotary_dim <= head_dim &&
           (reinterpret_cast<uintptr_t>(t->frequency) & 7u) == 0;
}

}  // namespace roomie
