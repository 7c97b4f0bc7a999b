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

// How a row is divided: 16-byte packs a thread, blocks (a power of two).  As few packs as 8 blocks do with; where that is more blocks than the SMs hold
// at once, four each, up to 64 tokens a thread, since what a thread does besides costs as much as 20 tokens: 192 rows of 50001 fp32 logits, 8 blocks of 28
// tokens a thread: top_k 42 us, top_p 102; 4 blocks of 56: 32 and 52.  More do not pay: 256 rows of 128000 bfloat16 logits, 64 tokens 75 us, 128 106.
struct Division {
    int packs;
    uint32_t blocks;
};
Division divide(uint64_t rows, uint32_t vocabulary, size_t eb) {
    const uint64_t need = vocabulary + 16 / eb - 1;                    // with what may lie ahead of the row on its first 16 bytes
    auto packs = [&](uint32_t blocks) {
        const uint64_t step = uint64_t(blocks) * kSampleThreads * (16 / eb);
        return int((need + step - 1) / step);
    };
    uint32_t blocks = kSampleMaxCluster;
    while (blocks > 1 && (packs(blocks / 2) == packs(blocks) || (rows * blocks > 4 * kSms && packs(blocks / 2) * (16 / eb) <= 64))) blocks /= 2;
    return {packs(blocks), blocks};
}

template <typename T>
tcu_status_t launch(const SampleParams &p, const Division &d, uint64_t rows, cudaStream_t stream) {
    const size_t shared = size_t(d.packs) * kSampleThreads * 16;
    constexpr size_t kMostShared = kMostVocabulary / kSampleMaxCluster * sizeof(T) + kSampleThreads * 16;
    if (shared + sizeof(SampleShared) > 48000 && !allow_shared<tcu_sample_kernel<T>>(kMostShared)) return TCU_ERR_CUDA;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = d.blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(uint32_t(rows * d.blocks));
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
    const Division d = divide(a->rows, a->vocabulary, eb);
    p.packs = d.packs;
    if (a->type == TCU_F32) return launch<float>(p, d, a->rows, stream);
    if (a->type == TCU_F16) return launch<__half>(p, d, a->rows, stream);
    return launch<__nv_bfloat16>(p, d, a->rows, stream);
}

}  // extern "C"
