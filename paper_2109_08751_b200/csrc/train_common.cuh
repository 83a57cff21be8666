// Shared by the training operators (train_*.cu): element types
// and vector accesses, argument checks, launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "../../include/sparbit_train.h"
#include "plan_access.h"

namespace spb {

#define CU(call)                                                         \
    do {                                                                 \
        cudaError_t e_ = (call);                                         \
        if (e_ != cudaSuccess) return record_cuda_error((int)e_, #call); \
    } while (0)

// ---- host ---------------------------------------------------------------------------------------

inline size_t elem_size(int dtype) { return dtype == SPARBIT_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == SPARBIT_F32 || dtype == SPARBIT_BF16 || dtype == SPARBIT_F16; }
inline size_t round_up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// A matrix an entry point touches: `rows` rows of `width` bytes, `ld` bytes apart.
struct Region {
    const void* p;
    size_t rows, width, ld;
};

// A row stride that rows of this width cannot have: below it, or so large (a negative number taken for a size)
// that the matrix would pass 2^46 elements, more than any memory; offsets below that cannot overflow.
constexpr size_t kMostElements = (size_t)1 << 46;
inline bool bad_pitch(size_t ld, size_t width, size_t rows) {
    return ld < width || ld > kMostElements / (rows ? rows : 1);
}

// Whether two matrices share a byte.  Rows at the same pitch may interleave (the halves of one
// buffer); otherwise overlapping address ranges count as overlap.
inline bool regions_overlap(const Region& a, const Region& b) {
    if (!a.p || !b.p || !a.rows || !b.rows || !a.width || !b.width) return false;
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    if (x >= y + (b.rows - 1) * b.ld + b.width || y >= x + (a.rows - 1) * a.ld + a.width) return false;
    if (a.ld != b.ld || a.ld == 0) return true;
    const size_t d = x <= y ? (size_t)(y - x) % a.ld : (a.ld - (size_t)(x - y) % a.ld) % a.ld;
    return d < a.width || d + b.width > a.ld;
}

// Whether one of the addresses (nulls apart) is no multiple of its elements' size: such an access would fault.
inline bool misaligned(size_t size, std::initializer_list<const void*> list) {
    for (const void* p : list)
        if ((uintptr_t)p % size) return true;
    return false;
}

// The widest vector (bytes, at most `most`) that every given address and pitch is a multiple of.
inline int common_alignment(uintptr_t bits, int most) {
    int v = most;
    while (v > 1 && (bits & (uintptr_t)(v - 1))) v >>= 1;
    return v;
}

// Launch with programmatic stream serialisation: the kernel may be scheduled while its predecessor
// in the stream drains and orders itself behind it with pdl_wait().
template <typename... KArgs, typename... Args>
inline cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                          Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

// ---- device -------------------------------------------------------------------------------------

// Waits until the kernels before this one in the stream have ended and their writes are visible.
// Every kernel here calls it before it touches global memory.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets the next kernel of the stream be scheduled.
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// V elements that are read and written as one access.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

// Two numbers at a time: the packed fp32 instructions of sm_100, half the issue slots of single ones.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("mul.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long&>(r))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)),
          "l"(reinterpret_cast<unsigned long long&>(c)));
    return r;
}

// Whole-warp bit masks are written out: every lane takes part in every shuffle of these files.
constexpr unsigned kAllLanes = 0xffffffffu;

}  // namespace spb
