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

// Threads (chunk, row) of a 256-thread block go over the rows (token, head) of `tokens` consecutive tokens from `first`.
// cs: [tokens][rot/2] cosine and sine, in shared memory.  A unit is kV elements; a row has rot/(2*kV) unit pairs that are
// rotated and, unless it is done in place, (dim - rot)/kV units that are copied.  kV = 16 bytes, or 1 when some row is not
// 16-byte aligned or the parts do not divide into such units.
template <class T, int kV, bool kPairs, int kUnroll>
__device__ __forceinline__ void rope_block(const HeadRows& io, const float2* cs, uint32_t first, uint32_t tokens, uint32_t heads,
                                           uint32_t dim, uint32_t rot, bool in_place) {
    const uint32_t half = rot / 2, n_rot = half / kV, n_copy = in_place ? 0 : (dim - rot) / kV, units = n_rot + n_copy;
    const uint32_t width = units < blockDim.x ? units : blockDim.x, lanes = blockDim.x / width;
    const uint32_t lane = threadIdx.x / width;
    if (lane >= lanes) return;
    const uint32_t rows = tokens * heads;
    using Raw = typename std::conditional<kV == 1, T, uint4>::type;
    for (uint32_t unit = threadIdx.x % width; unit < units; unit += width) {
        const bool turn = unit < n_rot;
        const uint32_t a = !turn ? rot + (unit - n_rot) * kV : kPairs ? 2 * unit * kV : unit * kV;
        const uint32_t b = kPairs ? a + kV : a + half;
        uint32_t tok = lane / heads, head = lane % heads;
        for (uint32_t row = lane; row < rows; row += lanes * kUnroll) {
            Raw ra[kUnroll], rb[kUnroll];
            uint32_t tt[kUnroll], hh[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                tt[u] = tok;
                hh[u] = head;
                if (row + u * lanes < rows) {
                    const T* p = static_cast<const T*>(io.x) + (first + tok) * io.x_token + head * io.x_head;
                    ra[u] = *reinterpret_cast<const Raw*>(p + a);
                    if (turn) rb[u] = *reinterpret_cast<const Raw*>(p + b);
                }
                head += lanes;
                while (head >= heads) { head -= heads; ++tok; }
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (row + u * lanes >= rows) break;
                T* p = static_cast<T*>(io.y) + (first + tt[u]) * io.y_token + hh[u] * io.y_head;
                if (!turn) {
                    *reinterpret_cast<Raw*>(p + a) = ra[u];
                    continue;
                }
                const float2* w = cs + (size_t)tt[u] * half + unit * kV;
                if constexpr (kV == 1) {
                    const float x = to_f32(ra[u]), y = to_f32(rb[u]);
                    p[a] = from_f32<T>(__fsub_rn(__fmul_rn(x, w->x), __fmul_rn(y, w->y)));
                    p[b] = from_f32<T>(__fadd_rn(__fmul_rn(y, w->x), __fmul_rn(x, w->y)));
                } else {
                    float xa[kV], xb[kV];
                    unpack<T>(ra[u], xa);
                    unpack<T>(rb[u], xb);
                    if constexpr (kPairs) {
                        float e[kV], o[kV];
#pragma unroll
                        for (int i = 0; i < kV / 2; ++i) {
                            e[i] = xa[2 * i]; o[i] = xa[2 * i + 1];
                            e[kV / 2 + i] = xb[2 * i]; o[kV / 2 + i] = xb[2 * i + 1];
                        }
                        rotate_half<kV>(e, o, w);
#pragma unroll
                        for (int i = 0; i < kV / 2; ++i) {
                            xa[2 * i] = e[i]; xa[2 * i + 1] = o[i];
                            xb[2 * i] = e[kV / 2 + i]; xb[2 * i + 1] = o[kV / 2 + i];
                        }
                    } else {
                        rotate_half<kV>(xa, xb, w);
                    }
                    *reinterpret_cast<uint4*>(p + a) = pack<T>(xa);
                    *reinterpret_cast<uint4*>(p + b) = pack<T>(xb);
                }
            }
        }
    }
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
