// Shared definitions of the serving operators: element types, vector access, rotary phases, recorded launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include "roomie_common.cuh"

namespace roomie {

// ---- launches that roomie_record_* can note (roomie_serving.cu) ---------------------------------------------------
bool record_on();
void record_begin(const char* name, const void* fn, unsigned long long blocks, uint32_t threads, size_t dyn_smem,
                  cudaStream_t st);
void record_end(cudaStream_t st);

int allow_smem(const void* fn, size_t bytes);   // so much dynamic shared memory for a kernel that may need more than 48 KB in all

// With `overlap` the kernel may start while the launch before it on the stream drains; it then waits for that launch's
// results itself (grid_dependency_wait) before it reads or writes anything another kernel touches.
template <class... KArgs, class... Args>
int launch(const char* name, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool overlap,
           Args... args) {
    const void* fn = reinterpret_cast<const void*>(kernel);
    if (smem > 16 * 1024) {                           // 48 KB less what a kernel has of its own, at most 32
        const int rc = allow_smem(fn, smem);
        if (rc != ROOMIE_OK) return rc;
    }
    const bool rec = record_on();
    if (rec) record_begin(name, fn, (unsigned long long)grid.x * grid.y * grid.z, block.x * block.y * block.z, smem, st);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
    if (rec) record_end(st);
    note_launch();
    return check_cuda(e);
}

__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ---- arithmetic -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// two float32 at a time
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
    return r;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) { return pair(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void split(uint64_t p, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// ---- element types --------------------------------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <class T> constexpr int kVecOf = 16 / (int)sizeof(T);   // elements of a 128-bit access

template <class T> __device__ __forceinline__ void unpack(const uint4& raw, float* out) {
    const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int i = 0; i < kVecOf<T>; ++i) out[i] = to_f32(e[i]);
}
template <class T> __device__ __forceinline__ uint4 pack(const float* in) {
    uint4 raw;
    T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int i = 0; i < kVecOf<T>; ++i) e[i] = from_f32<T>(in[i]);
    return raw;
}

inline size_t size_of_type(int32_t type) { return type == ROOMIE_F32 ? 4 : 2; }
inline bool known_type(int32_t type) { return type == ROOMIE_F32 || type == ROOMIE_F16 || type == ROOMIE_BF16; }
// every row of every head starts on a 16-byte boundary
inline bool rows_aligned16(const roomie_rows& r, uint32_t tokens, uint32_t heads) {
    const long long e = (long long)size_of_type(r.type);
    return (reinterpret_cast<uintptr_t>(r.data) & 15u) == 0 && (tokens <= 1 || (r.token_stride * e) % 16 == 0) &&
           (heads <= 1 || (r.head_stride * e) % 16 == 0);
}
// no two rows of an output share an element (a stride of 0, or below a row's length: several threads would write it, and one that is
// turned in place would be turned more than once)
inline bool rows_apart(const roomie_rows& r, uint32_t tokens, uint32_t heads, uint32_t dim) {
    const long long d = dim;
    return (tokens <= 1 || r.token_stride >= d || r.token_stride <= -d) && (heads <= 1 || r.head_stride >= d || r.head_stride <= -d);
}
inline bool rows_valid(const roomie_rows* r) {
    return r && r->data && known_type(r->type) && (reinterpret_cast<uintptr_t>(r->data) % size_of_type(r->type)) == 0;
}

// ---- rotary phases ---------------------------------------------------------------------------------------------------
// position * frequency modulo one turn is a 64-bit integer product that wraps: exact for any position, no range
// reduction afterwards.  Its upper 32 bits as a signed fraction of a turn round to float32 within 2^-25 turns.
__device__ __forceinline__ float2 rope_turn(uint64_t frequency, int32_t position, float amplitude) {
    const uint64_t phase = frequency * (uint64_t)(int64_t)position;
    float s, c;
    sincospif((float)(int32_t)(uint32_t)(phase >> 32) * 4.656612873077392578125e-10f, &s, &c);   // 2 * 2^-32 half turns
    return make_float2(c * amplitude, s * amplitude);
}

// One chunk pair of a row, rotated in float32.  Chunk c of the rotated part holds kV pairs: half layout elements
// [c*kV, +kV) with [c*kV + r/2, +kV); interleaved layout elements [2*c*kV, +2*kV).
template <int kV> __device__ __forceinline__ void rotate_half(float* a, float* b, const float2* cs) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const float x = a[i], y = b[i];
        a[i] = __fsub_rn(__fmul_rn(x, cs[i].x), __fmul_rn(y, cs[i].y));
        b[i] = __fadd_rn(__fmul_rn(y, cs[i].x), __fmul_rn(x, cs[i].y));
    }
}

}  // namespace roomie
