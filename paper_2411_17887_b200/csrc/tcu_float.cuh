// Element types of the language-model operators, and what their kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tcu {

// ---- element types -------------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// VEC elements of T, moved as one access of up to 16 bytes
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC <= 16 ? sizeof(T) * VEC : 16) Pack {
    T v[VEC];
};

// Two elements at a time: a conversion of two 16-bit ones is one instruction, and so is that of either half of a word.
template <typename T>
__device__ __forceinline__ float2 two_f32(const Pack<T, 2> &p) {
    if constexpr (sizeof(T) == 4) {
        return make_float2(p.v[0], p.v[1]);
    } else if constexpr (std::is_same_v<T, __half>) {
        return __half22float2(*reinterpret_cast<const __half2 *>(p.v));
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(p.v);
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
}
template <typename T>
__device__ __forceinline__ Pack<T, 2> two_from_f32(float a, float b) {
    Pack<T, 2> p;
    if constexpr (sizeof(T) == 4) {
        p.v[0] = a;
        p.v[1] = b;
    } else if constexpr (std::is_same_v<T, __half>) {
        *reinterpret_cast<__half2 *>(p.v) = __floats2half2_rn(a, b);
    } else {
        *reinterpret_cast<__nv_bfloat162 *>(p.v) = __floats2bfloat162_rn(a, b);
    }
    return p;
}

// The blocks of a cluster may touch one another's shared memory once all of them run: each says so when it begins, and waits before it does.
__device__ __forceinline__ void cluster_begin() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_begun() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A kernel of a sequence lets the next one be set up while it runs, and touches no memory before the one ahead of it is
// done with all of its own (which holds, in turn, for every one before).  What an earlier kernel writes is therefore not
// read through pointers that promise the compiler that nobody writes it.
__device__ __forceinline__ void begin_in_sequence() {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

}  // namespace tcu
