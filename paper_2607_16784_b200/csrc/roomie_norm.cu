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

template <class T, int kV> __device__ __forceinline__ void load_chunk(const T* p, bool on, float* x) {
    using Raw = typename RawOf<kV * (int)sizeof(T)>::type;
    if (on) {
        const Raw raw = *reinterpret_cast<const Raw*>(p);
        const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
        for (int i = 0; i < kV; ++i) x[i] = to_f32(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) x[i] = 0.0f;
    }
}
template <class T, int kV> __device__ __forceinline__ void store_chunk(T* p, bool on, const float* x) {
    using Raw = typename RawOf<kV * (int)sizeof(T)>::type;
    if (!on) return;
    Raw raw;
    T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int i = 0; i < kV; ++i) e[i] = from_f32<T>(x[i]);
    *reinterpret_cast<Raw*>(p) = raw;
}
__device__ __forceinline__ float load_weight(const void* w, int32_t type, uint32_t at) {
    if (!w) return 1.0f;
    if (type == ROOMIE_F32) return static_cast<const float*>(w)[at];
    if (type == ROOMIE_F16) return __half2float(static_cast<const __half*>(w)[at]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(w)[at]);
}

// x[0, kV) and x[kV, 2 kV) are a unit's chunks; with interleaved pairs, neighbours turn together
template <int kV, bool kPairs> __device__ __forceinline__ void turn_unit(float* x, const float2* cs, float sign) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const int a = kPairs ? 2 * i : i, b = kPairs ? 2 * i + 1 : i + kV;
        const float u = x[a], v = x[b], s = cs[i].y * sign;
        x[a] = __fsub_rn(__fmul_rn(u, cs[i].x), __fmul_rn(v, s));
        x[b] = __fadd_rn(__fmul_rn(v, cs[i].x), __fmul_rn(u, s));
    }
}

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

// The sum over the lanes of a row.
__device__ __forceinline__ float row_sum(float x, uint32_t lanes, uint32_t mask) {
    for (uint32_t d = lanes / 2; d > 0; d >>= 1) x += __shfl_xor_sync(mask, x, d);
    return x;
}

// Squares of values above 2^64 leave float32: such a row is taken times 2^-80.
constexpr float kLess = 8.271806125530277e-25f;

template <class T, int kV, int kPer, bool kPairs, bool kGrad>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(NormArgs n) {
    extern __shared__ float sums[];                                  // backward: [head groups of the block][dim]
    const uint32_t lane = threadIdx.x & 31, first = lane & ~(n.lanes - 1);
    const uint32_t mask = n.lanes == 32 ? 0xffffffffu : ((1u << n.lanes) - 1) << first;
    const uint32_t all = n.side[0].groups + n.side[1].groups;
    const uint32_t flat = blockIdx.x * (kNormThreads / n.lanes) + threadIdx.x / n.lanes, slot = flat / all;
    uint32_t group = flat - slot * all;
    const bool second = group >= n.side[0].groups;
    if (second) group -= n.side[0].groups;
    const NormSide& s = n.side[second];
    Unit u[kPer];
    float w[kPer][2 * kV], dw[kPer][2 * kV];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        u[k] = unit_of<kV, kPairs>(n, lane - first + k * n.lanes);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            w[k][i] = u[k].on ? load_weight(s.w, n.weight_type, u[k].a + i) : 0.0f;
            w[k][kV + i] = u[k].two ? load_weight(s.w, n.weight_type, u[k].b + i) : 0.0f;
            if (kGrad) dw[k][i] = dw[k][kV + i] = 0.0f;
        }
    }
    if (slot < n.slots)
        for (uint32_t token = slot; token < n.tokens; token += n.slots) {
            float2 cs[kPer][kV];
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (u[k].turn)
#pragma unroll
                    for (int i = 0; i < kV; ++i)
                        cs[k][i] = rope_turn(n.rope.frequency[(lane - first + k * n.lanes) * kV + i], n.positions[token], n.rope.amplitude);
            for (uint32_t head = group; head < s.heads; head += s.groups) {
                const T* px = static_cast<const T*>(s.x) + (long long)token * s.x_token + (long long)head * s.x_head;
                const T* pg = static_cast<const T*>(s.g) + (long long)token * s.g_token + (long long)head * s.g_head;
                T* py = static_cast<T*>(s.y) + (long long)token * s.y_token + (long long)head * s.y_head;
                float x[kPer][2 * kV], g[kPer][2 * kV];
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    load_chunk<T, kV>(px + u[k].a, u[k].on, x[k]);
                    load_chunk<T, kV>(px + u[k].b, u[k].two, x[k] + kV);
                    if (kGrad) {
                        load_chunk<T, kV>(pg + u[k].a, u[k].on, g[k]);
                        load_chunk<T, kV>(pg + u[k].b, u[k].two, g[k] + kV);
                    }
                }
                if (kGrad) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k)
                        if (u[k].turn) turn_unit<kV, kPairs>(g[k], cs[k], -1.0f);
                }
                float r, less = 1.0f, along = 0.0f;
                while (true) {
                    float square = 0.0f;
                    along = 0.0f;
#pragma unroll
                    for (int k = 0; k < kPer; ++k)
#pragma unroll
                        for (int i = 0; i < 2 * kV; ++i) {
                            square = fmaf(x[k][i], x[k][i], square);
                            if (kGrad) along = fmaf(g[k][i] * w[k][i], x[k][i], along);
                        }
                    square = row_sum(square, n.lanes, mask);
                    if (kGrad) along = row_sum(along, n.lanes, mask);
                    r = __frsqrt_rn(fmaf(square, n.inverse_dim, n.eps * less * less));
                    if (less != 1.0f || square != INFINITY) break;   // the same in all lanes of the row
                    less = kLess;
#pragma unroll
                    for (int k = 0; k < kPer; ++k)
#pragma unroll
                        for (int i = 0; i < 2 * kV; ++i) x[k][i] *= kLess;
                }
#pragma unroll
                for (int k = 0; k < kPer; ++k) {
                    if (kGrad) {
                        const float mean = along * r * n.inverse_dim;
#pragma unroll
                        for (int i = 0; i < 2 * kV; ++i) {
                            const float unit = x[k][i] * r;
                            dw[k][i] = fmaf(g[k][i], unit, dw[k][i]);
                            x[k][i] = r * less * (g[k][i] * w[k][i] - unit * mean);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2 * kV; ++i) x[k][i] = x[k][i] * r * w[k][i];
                        if (u[k].turn) turn_unit<kV, kPairs>(x[k], cs[k], 1.0f);
                    }
                    store_chunk<T, kV>(py + u[k].a, u[k].on, x[k]);
                    store_chunk<T, kV>(py + u[k].b, u[k].two, x[k] + kV);
                }
            }
        }
    if (!kGrad) return;
    // the block's sums, head group after head group
    const uint32_t mine = threadIdx.x / n.lanes, here = kNormThreads / n.lanes;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            if (u[k].on) sums[mine * n.dim + u[k].a + i] = dw[k][i];
            if (u[k].two) sums[mine * n.dim + u[k].b + i] = dw[k][kV + i];
        }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < 2 * n.dim; d += kNormThreads) {
        const uint32_t side = d >= n.dim, at = d - side * n.dim;
        float total = 0.0f;
        for (uint32_t i = 0; i < here; ++i) {
            const uint32_t f = (blockIdx.x * here + i) % all;
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
    void (*k)(NormArgs) = n.rope.interleaved ? norm_kernel<T, kV, kPer, true, kGrad> : norm_kernel<T, kV, kPer, false, kGrad>;
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
    // head groups as rope's: four heads or more a thread, unless there are too few rows to fill the GPU
    const unsigned long long one = (unsigned long long)n.tokens * n.lanes;
    for (NormSide& s : n.side) {
        unsigned long long g = (4096ull * sms + one - 1) / one, few = 256ull * sms / one;
        if (g > s.heads / 4) g = s.heads / 4;
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
