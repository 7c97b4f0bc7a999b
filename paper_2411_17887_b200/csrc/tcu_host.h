// What the host code of the language-model operators shares: argument checks, launches.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "tcu_lm.h"

namespace {

inline size_t float_bytes(tcu_float_t t) { return t == TCU_F32 ? 4 : 2; }
inline bool valid_float(int t) { return t == TCU_F32 || t == TCU_F16 || t == TCU_BF16; }
inline bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool overlaps(const void *a, size_t an, const void *b, size_t bn) {
    auto pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return a && b && pa < pb + bn && pb < pa + an;
}
// Whether a runtime call went well; if not, its error is taken here and is not left for the check of a later launch.
inline bool ok(cudaError_t e) {
    if (e == cudaSuccess) return true;
    (void)cudaGetLastError();
    return false;
}
inline tcu_status_t launched() { return cudaGetLastError() == cudaSuccess ? TCU_OK : TCU_ERR_CUDA; }

// Lets a kernel have as much shared memory, on the current device, as any of its launches asks for; the devices that know are remembered.
template <auto kernel>
bool allow_shared(size_t most) {
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    if (!ok(cudaGetDevice(&dev))) return false;
    const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t(1) << dev : 0;
    if (allowed.load(std::memory_order_relaxed) & bit) return true;
    if (!ok(cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, int(most)))) return false;
    allowed.fetch_or(bit, std::memory_order_relaxed);
    return true;
}

// A kernel that may be set up while the one ahead of it in the stream, of the same sequence, still runs.  A sequence ends at its
// first launch that fails: the kernels behind it index memory by what the ones before have written.
template <typename... P, typename... A>
tcu_status_t launch_next(void (*kernel)(P...), dim3 grid, dim3 block, cudaStream_t stream, A... args) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return ok(cudaLaunchKernelEx(&cfg, kernel, P(args)...)) ? TCU_OK : TCU_ERR_CUDA;
}

}  // namespace
