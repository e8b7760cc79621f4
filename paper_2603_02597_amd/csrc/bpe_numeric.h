// Element types of the operators on hidden states and logits, and their conversions.
#pragma once
#include "bpe_common.h"

namespace bpe {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));
typedef uint16_t H8 __attribute__((ext_vector_type(8)));

struct F32 { typedef float raw; static constexpr int kCode = BPE_F32; };
struct Bf16 { typedef uint16_t raw; static constexpr int kCode = BPE_BF16; };
struct F16 { typedef uint16_t raw; static constexpr int kCode = BPE_F16; };

template <class T> __device__ __forceinline__ float to_float(typename T::raw v);
template <> __device__ __forceinline__ float to_float<F32>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<Bf16>(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
template <> __device__ __forceinline__ float to_float<F16>(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }

// Rounding to the nearest, ties to even; the hardware's own conversions.
template <class T> __device__ __forceinline__ typename T::raw from_float(float v);
template <> __device__ __forceinline__ float from_float<F32>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t from_float<Bf16>(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
template <> __device__ __forceinline__ uint16_t from_float<F16>(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }

__device__ __forceinline__ float load_as_float(const void *p, int64_t i, int dtype) {
    if (dtype == BPE_F32) return ((const float *)p)[i];
    const uint16_t v = ((const uint16_t *)p)[i];
    return dtype == BPE_BF16 ? to_float<Bf16>(v) : to_float<F16>(v);
}

// What a wavefront's lanes have written to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr int64_t kMaxThreads = 1ll << 32;      // of a launch: fewer

// One launch of a kernel whose only argument is its parameter block.
template <class P>
inline int launch(void (*kernel)(P), dim3 grid, int block, P &p, void *stream, const char *what) {
    void *args[] = {&p};
    const hipError_t e = hipLaunchKernel((const void *)kernel, grid, dim3((unsigned)block), args, 0, (hipStream_t)stream);
    return e == hipSuccess ? BPE_OK : hip_fail(e, what);
}

inline int dtype_bytes(int dtype) { return dtype == BPE_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == BPE_F32 || dtype == BPE_BF16 || dtype == BPE_F16; }

}  // namespace bpe
