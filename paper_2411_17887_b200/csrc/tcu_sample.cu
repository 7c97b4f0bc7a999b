// Host side of sampling (include/tcu_lm.h): argument checks, launch.
#include "tcu_lm.h"

#include <cuda_runtime.h>

#include <initializer_list>
#include <type_traits>

#include "tcu_host.h"
#include "tcu_sample_kernel.cuh"

namespace {

using namespace tcu;

constexpr uint64_t kMostRows = ((uint64_t(1) << 31) - 1) / kSampleMaxCluster;
constexpr uint64_t kMostStride = uint64_t(1) << 38;
constexpr uint32_t kSms = 148;

// Blocks of a row: as many as hold it in parts of 32 KB, more where that leaves SMs idle and parts of 1024 tokens.
uint32_t blocks_of(uint64_t rows, uint32_t vocabulary, size_t eb) {
    uint32_t blocks = 1;
    while (blocks < kSampleMaxCluster &&
           (uint64_t(vocabulary) * eb > uint64_t(blocks) * 32768 || (rows * blocks * 2 <= kSms && vocabulary >= blocks * 2 * 1024)))
        blocks *= 2;
    return blocks;
}

template <typename T>
tcu_status_t launch(const SampleParams &p, uint32_t blocks, size_t shared, uint64_t rows, cudaStream_t stream) {
    if (!ok(cudaFuncSetAttribute(tcu_sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMostVocabulary / kSampleMaxCluster * sizeof(T) + 256)))) return TCU_ERR_CUDA;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(uint32_t(rows * blocks));
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return ok(cudaLaunchKernelEx(&cfg, tcu_sample_kernel<T>, p)) ? TCU_OK : TCU_ERR_CUDA;
}

}  // namespace

extern "C" {

tcu_status_t tcu_sample(const tcu_sample_t *a, cudaStream_t stream) {
    if (!a || a->struct_bytes != sizeof(tcu_sample_t) || !valid_float(int(a->type)) || a->vocabulary == 0) return TCU_ERR_INVALID_ARG;
    if (a->vocabulary > kMostVocabulary || a->rows > kMostRows) return TCU_ERR_UNSUPPORTED;
    const size_t eb = float_bytes(tcu_float_t(a->type)), ub = a->uniform_f64 ? 8 : 4;
    if (a->uniform_f64 > 1 || (a->rows > 1 && a->logits_stride > kMostStride)) return TCU_ERR_INVALID_ARG;
    if (!a->d_temperature && !(a->temperature >= 0.0 && a->temperature < 1e300)) return TCU_ERR_INVALID_ARG;
    if ((!a->d_top_p && a->top_p != a->top_p) || (!a->d_min_p && a->min_p != a->min_p)) return TCU_ERR_INVALID_ARG;
    for (const void *q : {static_cast<const void *>(a->d_temperature), static_cast<const void *>(a->d_top_k), static_cast<const void *>(a->d_top_p),
                          static_cast<const void *>(a->d_min_p), static_cast<const void *>(a->d_log_probs)})
        if (!aligned(q, 4)) return TCU_ERR_INVALID_ARG;
    if (a->rows == 0) return TCU_OK;
    if (!a->d_logits || !a->d_uniform || !a->d_tokens || !aligned(a->d_logits, eb) || !aligned(a->d_uniform, ub) || !aligned(a->d_tokens, 8)) return TCU_ERR_INVALID_ARG;
    const unsigned __int128 bytes = ((unsigned __int128)(a->rows - 1) * (a->rows > 1 ? a->logits_stride : 0) + a->vocabulary) * eb;
    if (bytes >> 63) return TCU_ERR_INVALID_ARG;
    struct {
        const void *p;
        size_t bytes;
    } const inputs[] = {{a->d_logits, size_t(bytes)}, {a->d_uniform, a->rows * ub}, {a->d_temperature, a->rows * 4}, {a->d_top_k, a->rows * 4}, {a->d_top_p, a->rows * 4},
                        {a->d_min_p, a->rows * 4}};
    for (const auto &in : inputs)
        if (overlaps(a->d_tokens, a->rows * 8, in.p, in.bytes) || overlaps(a->d_log_probs, a->rows * 4, in.p, in.bytes)) return TCU_ERR_INVALID_ARG;
    if (overlaps(a->d_tokens, a->rows * 8, a->d_log_probs, a->rows * 4)) return TCU_ERR_INVALID_ARG;
    SampleParams p = {};
    p.logits = a->d_logits;
    p.stride = a->logits_stride;
    p.vocabulary = a->vocabulary;
    p.uniform = a->d_uniform;
    p.uniform_f64 = int(a->uniform_f64);
    p.temperature = {a->d_temperature, a->temperature};
    p.top_k = {a->d_top_k, double(a->top_k)};
    p.top_p = {a->d_top_p, a->top_p};
    p.min_p = {a->d_min_p, a->min_p};
    p.tokens = a->d_tokens;
    p.log_probs = a->d_log_probs;
    const uint32_t blocks = blocks_of(a->rows, a->vocabulary, eb), vec = uint32_t(16 / eb);
    // the row and what may lie ahead of it on its first 16 bytes, in parts of whole 16 bytes
    p.part = ((a->vocabulary + vec - 1 + blocks - 1) / blocks + vec - 1) / vec * vec;
    const size_t shared = p.part * eb;
    if (a->type == TCU_F32) return launch<float>(p, blocks, shared, a->rows, stream);
    if (a->type == TCU_F16) return launch<__half>(p, blocks, shared, a->rows, stream);
    return launch<__nv_bfloat16>(p, blocks, shared, a->rows, stream);
}

}  // extern "C"
