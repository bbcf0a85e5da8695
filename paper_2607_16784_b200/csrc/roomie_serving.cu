// Rotary positions, and the record of the serving operators' launches.
#include <math.h>
#include <string.h>
#include <type_traits>
#include <new>
#include "roomie_rope.cuh"

namespace roomie {

// ---- recorded launches -----------------------------------------------------------------------------------------------
struct Recorded {
    const char* name;
    uint32_t grid, threads, regs, smem;
    cudaEvent_t begin, end;
};
static thread_local Recorded* t_rec = nullptr;
static thread_local uint32_t t_rec_cap = 0, t_rec_n = 0;

bool record_on() { return t_rec_n < t_rec_cap; }

void record_begin(const char* name, const void* fn, unsigned long long blocks, uint32_t threads, size_t dyn_smem,
                  cudaStream_t st) {
    Recorded& r = t_rec[t_rec_n];
    cudaFuncAttributes a;
    r.name = name;
    r.grid = (uint32_t)blocks;
    r.threads = threads;
    r.regs = r.smem = 0;
    if (cudaFuncGetAttributes(&a, fn) == cudaSuccess) {
        r.regs = (uint32_t)a.numRegs;
        r.smem = (uint32_t)(a.sharedSizeBytes + dyn_smem);
    }
    cudaEventRecord(r.begin, st);
}

void record_end(cudaStream_t st) {
    cudaEventRecord(t_rec[t_rec_n].end, st);
    ++t_rec_n;
}

static void record_drop(uint32_t made) {
    for (uint32_t i = 0; i < made; ++i) {
        cudaEventDestroy(t_rec[i].begin);
        cudaEventDestroy(t_rec[i].end);
    }
    delete[] t_rec;
    t_rec = nullptr;
    t_rec_cap = t_rec_n = 0;
}

// ---- large shared memory ---------------------------------------------------------------------------------------------
// The attribute belongs to a function and a device, for all threads of the process.  It is set to the most that there can be, once: were it set to
// what a call needs, a small call would take it away from the large ones of other threads.  A thread remembers what it has set, because setting it
// costs as much as half a launch.
int allow_smem(const void* fn, size_t bytes) {
    struct Set { const void* fn; int dev; size_t most; };
    static thread_local Set sets[64];
    int dev = 0;
    ROOMIE_CUDA_OK(cudaGetDevice(&dev));
    Set& s = sets[(reinterpret_cast<uintptr_t>(fn) >> 4) % 64];
    if (s.fn != fn || s.dev != dev) {
        int all = 0;
        cudaFuncAttributes own;
        ROOMIE_CUDA_OK(cudaDeviceGetAttribute(&all, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev));
        ROOMIE_CUDA_OK(cudaFuncGetAttributes(&own, fn));
        const size_t most = (size_t)all - own.sharedSizeBytes;
        ROOMIE_CUDA_OK(cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
        s = {fn, dev, most};
    }
    return bytes <= s.most ? ROOMIE_OK : check_cuda(cudaErrorInvalidValue);
}

// ---- rotary positions ------------------------------------------------------------------------------------------------
struct RopeArgs {
    HeadRows io;
    RopeView rope;
    const int32_t* positions;
    uint32_t heads, units, groups;
    unsigned long long threads;
    int32_t inverse;
};

constexpr int kRopeThreads = 128;

// Memory-bound: every element is read and written once.
template <class T, int kV, bool kPairs>
__global__ void __launch_bounds__(kRopeThreads, 8) rope_kernel(RopeArgs a) {
    const unsigned long long i = (unsigned long long)blockIdx.x * kRopeThreads + threadIdx.x;
    if (i >= a.threads) return;
    const uint32_t rest = (uint32_t)(i / a.units), unit = (uint32_t)(i - (unsigned long long)rest * a.units);
    const uint32_t token = rest / a.groups, group = rest - token * a.groups;
    rope_heads<T, kV, kPairs, kV == 1 ? 1 : 2>(a.io, a.rope, token, a.positions[token], a.inverse != 0, unit, group, a.groups, a.heads);
}

template <class T>
static int launch_rope(RopeArgs a, uint32_t tokens, uint32_t dim, bool in_place, bool wide, cudaStream_t st) {
    constexpr int v = kVecOf<T>;
    const RopeSplit s = rope_split(tokens, a.heads, dim, a.rope.rot, wide ? v : 1, in_place, (uint32_t)sm_count());
    if (s.threads / a.heads > 0xffffffffull) return ROOMIE_ERR_INVALID_ARG;
    a.units = s.units; a.groups = s.groups; a.threads = s.threads;
    const unsigned long long blocks = (s.threads + kRopeThreads - 1) / kRopeThreads;
    if (blocks > 0x7fffffffull) return ROOMIE_ERR_INVALID_ARG;
    void (*k)(RopeArgs);
    if (a.rope.interleaved) k = wide ? rope_kernel<T, v, true> : rope_kernel<T, 1, true>;
    else k = wide ? rope_kernel<T, v, false> : rope_kernel<T, 1, false>;
    return launch("rope", k, dim3((uint32_t)blocks), dim3(kRopeThreads), 0, st, false, a);
}

}  // namespace roomie

using namespace roomie;

extern "C" int roomie_rope_frequencies(uint32_t rotary_dim, double base, double factor, double context, double low_turns,
                                       double high_turns, uint64_t* frequency_out) {
    if (!frequency_out || rotary_dim == 0 || rotary_dim % 2 || !(base > 1.0) || !(factor >= 1.0) || !(context >= 0.0) ||
        !isfinite(base) || !isfinite(factor) || !isfinite(context))
        return ROOMIE_ERR_INVALID_ARG;
    if (context > 0.0 && !(low_turns < high_turns)) return ROOMIE_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < rotary_dim / 2; ++i) {
        const double plain = pow(base, -2.0 * i / rotary_dim) / 6.283185307179586476925286766559;
        double keep = 0.0;
        if (context > 0.0) keep = fmin(fmax((plain * context - low_turns) / (high_turns - low_turns), 0.0), 1.0);
        const double f = plain * (keep + (1.0 - keep) / factor);          // turns per position, below 0.16
        frequency_out[i] = (uint64_t)rint(ldexp(f, 64));
    }
    return ROOMIE_OK;
}

extern "C" int roomie_rope(const roomie_rope_table* table, const roomie_rows* x, const roomie_rows* y, uint32_t tokens,
                           uint32_t heads, uint32_t head_dim, const int32_t* positions, int inverse, void* stream) {
    if (!rope_table_valid(table, head_dim) || head_dim > 1024) return ROOMIE_ERR_INVALID_ARG;
    if (tokens == 0 || heads == 0) return ROOMIE_OK;
    if (!rows_valid(x) || !rows_valid(y) || x->type != y->type || !positions || !rows_apart(*y, tokens, heads, head_dim)) return ROOMIE_ERR_INVALID_ARG;
    const bool same = x->data == y->data;
    if (same && (x->token_stride != y->token_stride || x->head_stride != y->head_stride)) return ROOMIE_ERR_INVALID_ARG;
    if ((unsigned long long)tokens * heads > 0x7fffffffull) return ROOMIE_ERR_INVALID_ARG;
    RopeArgs a = {};
    a.io = {x->data, y->data, x->token_stride, x->head_stride, y->token_stride, y->head_stride};
    a.rope = {table->frequency, table->rotary_dim, table->interleaved, table->amplitude};
    a.positions = positions;
    a.heads = heads;
    a.inverse = inverse != 0;
    const bool wide = rope_units_of_16(table->rotary_dim, head_dim, x->type, table->interleaved) &&
                      rows_aligned16(*x, tokens, heads) && rows_aligned16(*y, tokens, heads);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (x->type == ROOMIE_F32) return launch_rope<float>(a, tokens, head_dim, same, wide, st);
    if (x->type == ROOMIE_F16) return launch_rope<__half>(a, tokens, head_dim, same, wide, st);
    return launch_rope<__nv_bfloat16>(a, tokens, head_dim, same, wide, st);
}

extern "C" int roomie_record_enable(uint32_t capacity) {
    if (capacity > 1u << 20) return ROOMIE_ERR_INVALID_ARG;
    if (t_rec) record_drop(t_rec_cap);
    if (capacity == 0) return ROOMIE_OK;
    t_rec = new (std::nothrow) Recorded[capacity];
    if (!t_rec) return ROOMIE_ERR_CAPACITY;
    for (uint32_t i = 0; i < capacity; ++i) {
        cudaError_t e = cudaEventCreate(&t_rec[i].begin);
        if (e == cudaSuccess && (e = cudaEventCreate(&t_rec[i].end)) != cudaSuccess) cudaEventDestroy(t_rec[i].begin);
        if (e != cudaSuccess) {
            record_drop(i);
            return check_cuda(e);
        }
    }
    t_rec_cap = capacity;
    t_rec_n = 0;
    return ROOMIE_OK;
}

extern "C" int roomie_record_read(roomie_launch* out, uint32_t capacity, uint32_t* count) {
    if (!count || (!out && capacity)) return ROOMIE_ERR_INVALID_ARG;
    *count = 0;
    for (uint32_t i = 0; i < t_rec_n && i < capacity; ++i) {
        const Recorded& r = t_rec[i];
        roomie_launch& o = out[i];
        memset(&o, 0, sizeof o);
        strncpy(o.name, r.name, sizeof(o.name) - 1);
        o.grid_blocks = r.grid; o.block_threads = r.threads; o.regs_per_thread = r.regs; o.smem_per_block = r.smem;
        ROOMIE_CUDA_OK(cudaEventSynchronize(r.end));
        ROOMIE_CUDA_OK(cudaEventElapsedTime(&o.dur_us, r.begin, r.end));
        o.dur_us *= 1000.0f;
        if (i + 1 < t_rec_n) {
            ROOMIE_CUDA_OK(cudaEventSynchronize(t_rec[i + 1].begin));
            ROOMIE_CUDA_OK(cudaEventElapsedTime(&o.gap_us, r.end, t_rec[i + 1].begin));
            o.gap_us = o.gap_us > 0.0f ? o.gap_us * 1000.0f : 0.0f;
        }
        ++*count;
    }
    t_rec_n = 0;
    return ROOMIE_OK;
}
