// Host side of the C ABI declared in include/tcu_lm.h: argument checks, launches.
#include "tcu_lm.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <initializer_list>
#include <mutex>
#include <type_traits>

#include "tcu_embedding_kernel.cuh"
#include "tcu_linattn_kernel.cuh"

namespace {

using namespace tcu;

constexpr size_t kStatusBytes = 256;       // the header of a scan workspace: one status word is used

size_t float_bytes(tcu_float_t t) { return t == TCU_F32 ? 4 : 2; }
bool valid_float(int t) { return t == TCU_F32 || t == TCU_F16 || t == TCU_BF16; }
bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool overlaps(const void *a, size_t an, const void *b, size_t bn) {
    auto pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return a && b && pa < pb + bn && pb < pa + an;
}
// Whether a runtime call went well; if not, its error is taken here and is not left for the check of a later launch.
bool ok(cudaError_t e) {
    if (e == cudaSuccess) return true;
    (void)cudaGetLastError();
    return false;
}
tcu_status_t launched() { return cudaGetLastError() == cudaSuccess ? TCU_OK : TCU_ERR_CUDA; }

// ---- linear attention
bool has_struct(const tcu_linattn_t *a) { return a && a->struct_bytes == sizeof(tcu_linattn_t); }

// First and one-past-last byte that a token array may touch (packed: batch is 1); to the end of all addresses if it has no such last byte.
struct Span {
    uintptr_t lo, hi;
};
Span span_of(const tcu_tokens_t &x, uint64_t batch, uint64_t tokens, uint32_t heads, uint32_t width, size_t eb) {
    using Wide = unsigned __int128;
    const auto lo = reinterpret_cast<uintptr_t>(x.ptr);
    const Wide last = Wide(batch - 1) * uint64_t(x.stride_batch) + Wide(tokens - 1) * uint64_t(x.stride_token) + Wide(heads - 1) * uint64_t(x.stride_head) + width;
    const Wide end = lo + last * eb;
    return {lo, end > ~uintptr_t(0) ? ~uintptr_t(0) : uintptr_t(end)};
}
bool spans_meet(const Span &a, const Span &b) { return a.lo < b.hi && b.lo < a.hi; }

// Checks of one (batch, token, head, feature) array; written arrays may not repeat (strides of 0 with an extent above 1)
tcu_status_t check_tokens(const tcu_tokens_t &x, bool packed, uint64_t batch, uint64_t tokens, uint32_t heads, bool written) {
    if (!x.ptr || !aligned(x.ptr, 16)) return TCU_ERR_INVALID_ARG;
    const int64_t limit = int64_t(1) << 38;
    const int64_t sb = packed ? 0 : x.stride_batch;
    for (int64_t s : {sb, x.stride_token, x.stride_head})
        if (s < 0 || s >= limit || s % 8 != 0) return TCU_ERR_INVALID_ARG;
    if (tokens > 1 && x.stride_token == 0) return TCU_ERR_INVALID_ARG;
    if (written && ((!packed && batch > 1 && sb == 0) || (heads > 1 && x.stride_head == 0))) return TCU_ERR_INVALID_ARG;
    return TCU_OK;
}

MixTokens view(const tcu_tokens_t &x) { return {x.ptr, x.stride_batch, x.stride_token, x.stride_head}; }

// where a workspace keeps its status word: the header of a scan workspace, which tcu_scan_device_status reads
struct WsStatus {
    uint32_t epoch, done, error;
};

// Sequences times heads, so that three jobs of eight blocks each are a grid.  (Batch and heads alone may have a product of more than 64 bits.)
constexpr uint64_t kMostWalks = ((uint64_t(1) << 31) - 1) / 24;
bool too_many(const tcu_linattn_t *a) { return a->heads > 0 && a->batch > kMostWalks / a->heads; }
constexpr uint64_t kMostMixTokens = (uint64_t(1) << 31) - 256;

// What forward and backward share.
tcu_status_t check_linattn(const tcu_linattn_t *a, const void *d_ws, size_t ws_bytes) {
    if (!has_struct(a)) return TCU_ERR_INVALID_ARG;
    if (a->type != TCU_F16 && a->type != TCU_BF16) return TCU_ERR_INVALID_ARG;
    if (a->heads == 0 || a->dk == 0 || a->dv == 0) return TCU_ERR_INVALID_ARG;
    if (a->dk > 128 || a->dv > 128) return TCU_ERR_UNSUPPORTED;
    if (a->tokens > kMostMixTokens || too_many(a)) return TCU_ERR_UNSUPPORTED;
    if (a->batch == 0) return TCU_OK;
    if (!d_ws || ws_bytes < kStatusBytes) return TCU_ERR_WORKSPACE;
    if (!aligned(d_ws, 16) || !a->d_log_decay || !aligned(a->d_log_decay, 4)) return TCU_ERR_INVALID_ARG;
    if (a->d_offsets && !aligned(a->d_offsets, 8)) return TCU_ERR_INVALID_ARG;
    for (const void *s : {static_cast<const void *>(a->d_state_in), static_cast<const void *>(a->d_state_out),
                          static_cast<const void *>(a->d_dstate_out), static_cast<const void *>(a->d_dstate_in)})
        if (s && !aligned(s, 16)) return TCU_ERR_INVALID_ARG;
    return TCU_OK;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static std::once_flag once;
    static EncodeTiledFn fn = nullptr;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (ok(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q)) && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// (feature, token, head, sequence) view, tiles of 64 features x 128 tokens; features past the width and tokens past the end read as
// zero and are not written.  An axis along which the array repeats has an extent of 1 in the map.
bool encode_tokens(CUtensorMap *map, const tcu_linattn_t *a, const tcu_tokens_t &x, uint32_t width) {
    const bool packed = a->d_offsets != nullptr;
    const uint64_t nb = packed || x.stride_batch == 0 ? 1 : a->batch, nh = x.stride_head == 0 ? 1 : a->heads;
    const cuuint64_t dims[4] = {width, a->tokens, nh, nb};
    auto bytes = [](uint64_t extent, int64_t stride) { return extent > 1 ? cuuint64_t(stride) * 2 : cuuint64_t(16); };   // (not used when the extent is 1)
    const cuuint64_t strides[3] = {bytes(a->tokens, x.stride_token), bytes(nh, x.stride_head), bytes(nb, x.stride_batch)};
    const cuuint32_t box[4] = {64, kGroup, 1, 1}, step[4] = {1, 1, 1, 1};
    return encode_fn()(map, a->type == TCU_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, x.ptr, dims, strides, box, step,
                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count() {
    static std::atomic<int> cached{0};
    int v = cached.load();
    if (v > 0) return v;
    int dev = 0;
    if (!ok(cudaGetDevice(&dev)) || !ok(cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev))) return 0;
    cached.store(v);
    return v;
}

constexpr uint32_t kMostRanks = 8;       // blocks of a cluster, as far as every device schedules them

template <int D, typename T>
cudaLaunchConfig_t mix_config(uint32_t blocks, uint32_t ranks, cudaLaunchAttribute *attr, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kMixThreads);
    cfg.dynamicSmemBytes = kMixSmemBytes<D>;
    cfg.stream = stream;
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = ranks;
    attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ranks > 1 ? 1 : 0;
    return cfg;
}

// Into how many parts a walk is split, over the blocks of a cluster, when there are few.  A block fills an SM, and clusters of r
// blocks fill the SMs worse the larger r is (clusters of 8: 15 at a time, 120 blocks of 148).  In units of a group of the walk,
// 3.4 us: a group of the first phase takes 0.65, the exchange of states and the second start 3.  `groups` of an average walk.
// Measured: 16 heads of 8191 tokens at D = 128: 1 rank 204 us, 2 176, 3 123, 4 103, 5 86, 6 75 (taken), 8 119 (two waves); outputs and
// gradients of 64 heads of 4096 tokens, whole walks: 1 rank 316 us, 2 387, 4 457.
template <int D, typename T>
tcu_status_t choose_ranks(uint64_t units, uint64_t groups, uint32_t *ranks) {
    static std::atomic<int> configured{-1};
    static std::atomic<int> at_once[kMostRanks + 1];
    int dev = 0;
    if (!ok(cudaGetDevice(&dev))) return TCU_ERR_CUDA;
    if (configured.load() != dev) {
        if (!ok(cudaFuncSetAttribute(tcu_linattn_mix_kernel<D, T, kWhole>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMixSmemBytes<D>))) return TCU_ERR_CUDA;
        at_once[1] = sm_count();
        for (uint32_t r = 2; r <= kMostRanks; ++r) {
            cudaLaunchAttribute attr;
            const cudaLaunchConfig_t cfg = mix_config<D, T>(r, r, &attr, nullptr);
            int n = 0;
            at_once[r] = ok(cudaOccupancyMaxActiveClusters(&n, tcu_linattn_mix_kernel<D, T, kWhole>, &cfg)) ? n : 0;
        }
        configured.store(dev);
    }
    *ranks = 1;
    double best = 0;
    for (uint32_t r = 1; r <= kMostRanks && (r == 1 || groups >= 2 * r); ++r) {
        const uint64_t n = uint64_t(at_once[r].load());
        if (n == 0) continue;
        const double cost = double((units + n - 1) / n) * (r == 1 ? double(groups) : 1.65 * double((groups + r - 1) / r) + 3.0);
        if (r == 1 || cost < best) {
            best = cost;
            *ranks = r;
        }
    }
    return TCU_OK;
}

// More walks than SMs: whether they are cut into equal shares of all the groups, one for each SM, with the state handed from
// block to block, instead of running whole in waves of which the last is not full.  In units of a group: a walk costs one more to
// begin, the shares about four more in all.  Measured, bfloat16, whole against cut: gradients of 64 heads of 4096 tokens at
// 128 x 128 (192 walks) 210 us, 163; outputs of 200 heads of 2048 tokens 121, 102; of 170 heads of 8192 tokens 412, 286; of 160 heads
// of 1024 tokens at 64 x 64 51, 39; gradients of 250 heads of 300 tokens 89, 94 (whole).  Packed sequences differ in length, and a
// long one is as long in parts that wait for one another: cut as well, 24 of them with 12 heads took 164 us where whole
// walks took 153, and 137 with the long ones first.
bool cut_pays(const tcu_linattn_t *a, uint32_t jobs) {
    const uint64_t units = a->batch * a->heads * jobs, sms = uint64_t(sm_count()), places = (a->tokens + kGroup - 1) / kGroup + 1;
    return sms > 0 && units > sms && a->tokens > 0 && !a->d_offsets && units * places / sms + 4 < (units + sms - 1) / sms * places;
}
// More walks than SMs of packed sequences: the long ones first, in an order found by a kernel ahead.  Measured, bfloat16: 64 sequences
// of 50 to 3000 tokens with 16 heads 268 us as they come, 239 in order; one of 4000 after 31 of 100 with 12 heads 123, 107; 200 of 60 with
// 16 heads, where no order helps, 174, 179.
bool order_pays(const tcu_linattn_t *a, uint32_t jobs) {
    return a->d_offsets && a->tokens > 0 && a->batch > 1 && a->batch <= kMostOrdered && a->batch * a->heads * jobs > uint64_t(sm_count());
}
size_t flag_bytes() { return (size_t(sm_count()) * 4 + 255) / 256 * 256; }
size_t scratch_bytes(const tcu_linattn_t *a, uint32_t jobs) {
    return cut_pays(a, jobs) ? flag_bytes() + size_t(sm_count()) * a->dk * a->dv * 4 : order_pays(a, jobs) ? kMostOrdered * 4 : 0;
}

template <int D, typename T, int KIND>
tcu_status_t launch_kind(const MixParams &p, const cudaLaunchConfig_t &cfg) {
    static std::atomic<int> configured{-1};
    int dev = 0;
    if (!ok(cudaGetDevice(&dev))) return TCU_ERR_CUDA;
    if (configured.load() != dev) {
        if (!ok(cudaFuncSetAttribute(tcu_linattn_mix_kernel<D, T, KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMixSmemBytes<D>))) return TCU_ERR_CUDA;
        configured.store(dev);
    }
    return ok(cudaLaunchKernelEx(&cfg, tcu_linattn_mix_kernel<D, T, KIND>, p)) ? TCU_OK : TCU_ERR_CUDA;
}

template <int D, typename T>
tcu_status_t launch_mix(const tcu_linattn_t *a, MixParams &p, uint64_t groups, cudaStream_t stream) {
    const uint32_t units = p.batch * p.heads * p.jobs;
    cudaLaunchAttribute attr;
    if (a->d_scratch && cut_pays(a, p.jobs)) {
        p.ranks = 1;
        p.flags = static_cast<uint32_t *>(a->d_scratch);
        p.handed = reinterpret_cast<float *>(static_cast<uint8_t *>(a->d_scratch) + flag_bytes());
        if (!ok(cudaMemsetAsync(p.flags, 0, flag_bytes(), stream))) return TCU_ERR_CUDA;
        cudaLaunchConfig_t cfg = mix_config<D, T>(uint32_t(sm_count()), 1, &attr, stream);
        attr.id = cudaLaunchAttributeCooperative;          // blocks wait for one another: all of them run at once
        attr.val.cooperative = 1;
        cfg.numAttrs = 1;
        if (launch_kind<D, T, kCut>(p, cfg) == TCU_OK) return TCU_OK;                  // else not all SMs are this process's to use: whole walks
    }
    if (tcu_status_t st = choose_ranks<D, T>(units, groups, &p.ranks)) return st;
    const cudaLaunchConfig_t cfg = mix_config<D, T>(units * p.ranks, p.ranks, &attr, stream);
    if (a->d_scratch && p.ranks == 1 && order_pays(a, p.jobs)) {
        uint32_t *order = static_cast<uint32_t *>(a->d_scratch);
        tcu_linattn_order_kernel<<<1, kMostOrdered, 0, stream>>>(p.offsets, p.batch, order);
        if (tcu_status_t st = launched()) return st;           // the walk would take its sequences from memory that nobody has written
        p.order = order;
        cudaLaunchConfig_t next = cfg;
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        next.numAttrs = 1;
        return launch_kind<D, T, kOrdered>(p, next);
    }
    return launch_kind<D, T, kWhole>(p, cfg);
}

// `transposed`: the state that enters is stored as dv x dk.
MixJob make_job(const uint8_t (&maps)[3], uint32_t dk, uint32_t dv, bool forward, const float *init, bool transposed, float *last, float in_scale,
                float out_scale) {
    MixJob j = {};
    for (int i = 0; i < 3; ++i) j.map[i] = maps[i];
    j.init = init;
    j.last = last;
    j.init_k = transposed ? 1 : dv;
    j.init_v = transposed ? dk : 1;
    j.dk = dk;
    j.dv = dv;
    j.lead = forward ? 1 : 0;
    j.in_scale = in_scale;
    j.out_scale = out_scale;
    return j;
}

// Fills in what all jobs share and launches.  `arrays`: what the jobs' map indexes name; `outputs`: where each job writes.
tcu_status_t run_mix(const tcu_linattn_t *a, MixParams &p, const tcu_tokens_t *const *arrays, const uint32_t *widths, int count,
                     const tcu_tokens_t *const *outputs, void *d_ws, cudaStream_t stream) {
    if (a->d_scratch && (a->scratch_bytes < scratch_bytes(a, p.jobs) || !aligned(a->d_scratch, 256))) return TCU_ERR_WORKSPACE;
    if (!encode_fn()) return TCU_ERR_CUDA;
    thread_local int bound = -1;      // encoding needs a current context, which a thread that has made no CUDA call does not have
    int dev = 0;
    if (!ok(cudaGetDevice(&dev)) || (bound != dev && !ok(cudaSetDevice(dev)))) return TCU_ERR_CUDA;
    bound = dev;
    for (int i = 0; i < count; ++i)
        if (!encode_tokens(&p.map[i], a, *arrays[i], widths[i])) return TCU_ERR_CUDA;
    if (p.rounds == 0) p.rounds = kMixWaitRounds;
    p.log_decay = a->d_log_decay;
    p.offsets = a->d_offsets;
    p.error = &static_cast<WsStatus *>(d_ws)->error;
    p.tokens = a->tokens;
    p.batch = uint32_t(a->batch);
    p.heads = a->heads;
    for (uint32_t j = 0; j < p.jobs; ++j) {
        MixJob &job = p.job[j];
        for (int i = 0; i < 3; ++i) {
            job.by_batch[i] = arrays[job.map[i]]->stride_batch != 0;
            job.by_head[i] = arrays[job.map[i]]->stride_head != 0;
        }
        const tcu_tokens_t &o = *outputs[j];
        job.o = o.ptr;
        job.o_batch = o.stride_batch;
        job.o_token = o.stride_token;
        job.o_head = o.stride_head;
        job.map[3] = uint8_t(count + j);
        if (!encode_tokens(&p.map[count + j], a, o, job.dv)) return TCU_ERR_CUDA;
    }
    const bool wide = a->dk > 64 || a->dv > 64;
    const uint64_t groups = ((a->d_offsets ? a->tokens / a->batch : a->tokens) + kGroup - 1) / kGroup;
    if (a->type == TCU_F16) return wide ? launch_mix<128, __half>(a, p, groups, stream) : launch_mix<64, __half>(a, p, groups, stream);
    return wide ? launch_mix<128, __nv_bfloat16>(a, p, groups, stream) : launch_mix<64, __nv_bfloat16>(a, p, groups, stream);
}

// What a self-test changes: `rounds` and `silent` of MixParams (0: nothing).
struct Waits {
    uint32_t rounds, silent;
};

// No tokens: the state that leaves is the state that enters.
tcu_status_t copy_state(float *to, const float *from, size_t bytes, cudaStream_t stream) {
    if (!to || to == from) return TCU_OK;
    return ok(from ? cudaMemcpyAsync(to, from, bytes, cudaMemcpyDeviceToDevice, stream) : cudaMemsetAsync(to, 0, bytes, stream)) ? TCU_OK : TCU_ERR_CUDA;
}

tcu_status_t forward(const tcu_linattn_t *a, void *d_ws, size_t ws_bytes, const Waits &waits, cudaStream_t stream) {
    if (tcu_status_t st = check_linattn(a, d_ws, ws_bytes)) return st;
    if (a->batch == 0) return TCU_OK;
    const bool packed = a->d_offsets != nullptr;
    if (a->tokens > 0) {
        const tcu_tokens_t *all[4] = {&a->q, &a->k, &a->v, &a->o};
        const uint64_t nb = packed ? 1 : a->batch;
        Span at[4];
        for (int i = 0; i < 4; ++i) {
            if (tcu_status_t st = check_tokens(*all[i], packed, a->batch, a->tokens, a->heads, i == 3)) return st;
            at[i] = span_of(*all[i], nb, a->tokens, a->heads, i < 2 ? a->dk : a->dv, 2);
        }
        for (int i = 0; i < 3; ++i)
            if (spans_meet(at[i], at[3])) return TCU_ERR_INVALID_ARG;
    } else if (!a->d_state_out) {
        return TCU_OK;
    }
    const size_t state = size_t(a->batch) * a->heads * a->dk * a->dv * 4;
    if (a->d_state_out != a->d_state_in && overlaps(a->d_state_out, state, a->d_state_in, state)) return TCU_ERR_INVALID_ARG;
    if (a->tokens == 0) return copy_state(a->d_state_out, a->d_state_in, state, stream);
    const tcu_tokens_t *arrays[3] = {&a->q, &a->k, &a->v}, *outputs[1] = {&a->o};
    const uint32_t widths[3] = {a->dk, a->dk, a->dv};
    MixParams p = {};
    p.rounds = waits.rounds;
    p.silent = waits.silent;
    p.jobs = 1;
    p.job[0] = make_job({0, 1, 2}, a->dk, a->dv, true, a->d_state_in, false, a->d_state_out, 1.0f, a->scale);
    return run_mix(a, p, arrays, widths, 3, outputs, d_ws, stream);
}

tcu_status_t backward(const tcu_linattn_t *a, void *d_ws, size_t ws_bytes, const Waits &waits, cudaStream_t stream) {
    if (tcu_status_t st = check_linattn(a, d_ws, ws_bytes)) return st;
    if (a->batch == 0) return TCU_OK;
    const bool packed = a->d_offsets != nullptr;
    if (a->tokens > 0) {
        const tcu_tokens_t *all[7] = {&a->q, &a->k, &a->v, &a->d_o, &a->d_q, &a->d_k, &a->d_v};
        const uint32_t width[7] = {a->dk, a->dk, a->dv, a->dv, a->dk, a->dk, a->dv};
        const uint64_t nb = packed ? 1 : a->batch;
        Span at[7];
        for (int i = 0; i < 7; ++i) {
            if (tcu_status_t st = check_tokens(*all[i], packed, a->batch, a->tokens, a->heads, i >= 4)) return st;
            at[i] = span_of(*all[i], nb, a->tokens, a->heads, width[i], 2);
        }
        for (int i = 0; i < 4; ++i)
            for (int w = 4; w < 7; ++w)
                if (spans_meet(at[i], at[w])) return TCU_ERR_INVALID_ARG;
        // (gradients may lie between one another, as in one array of all three)
        if (a->d_q.ptr == a->d_k.ptr || a->d_q.ptr == a->d_v.ptr || a->d_k.ptr == a->d_v.ptr) return TCU_ERR_INVALID_ARG;
    } else if (!a->d_dstate_in) {
        return TCU_OK;
    }
    const size_t state = size_t(a->batch) * a->heads * a->dk * a->dv * 4;
    if (overlaps(a->d_dstate_in, state, a->d_dstate_out, state) || overlaps(a->d_dstate_in, state, a->d_state_in, state)) return TCU_ERR_INVALID_ARG;
    if (a->tokens == 0) return copy_state(a->d_dstate_in, a->d_dstate_out, state, stream);
    enum { kQ, kK, kV, kDo };
    const tcu_tokens_t *arrays[4] = {&a->q, &a->k, &a->v, &a->d_o}, *outputs[3] = {&a->d_q, &a->d_v, &a->d_k};
    const uint32_t widths[4] = {a->dk, a->dk, a->dv, a->dv};
    MixParams p = {};
    p.rounds = waits.rounds;
    p.silent = waits.silent;
    p.jobs = 3;
    p.job[0] = make_job({kDo, kV, kK}, a->dv, a->dk, true, a->d_state_in, true, nullptr, 1.0f, a->scale);
    p.job[1] = make_job({kK, kQ, kDo}, a->dk, a->dv, false, a->d_dstate_out, false, a->d_dstate_in, a->scale, 1.0f);
    p.job[2] = make_job({kV, kDo, kQ}, a->dv, a->dk, false, a->d_dstate_out, true, nullptr, a->scale, 1.0f);
    return run_mix(a, p, arrays, widths, 4, outputs, d_ws, stream);
}

}  // namespace

extern "C" {

size_t tcu_linattn_workspace_bytes(void) { return kStatusBytes; }

size_t tcu_linattn_scratch_bytes(const tcu_linattn_t *a, int backward) {
    if (!has_struct(a) || a->dk == 0 || a->dk > 128 || a->dv == 0 || a->dv > 128 || a->tokens > kMostMixTokens || too_many(a)) return 0;
    return scratch_bytes(a, backward ? 3 : 1);
}

tcu_status_t tcu_linattn_forward(const tcu_linattn_t *a, void *d_ws, size_t ws_bytes, cudaStream_t stream) {
    return forward(a, d_ws, ws_bytes, {}, stream);
}

tcu_status_t tcu_linattn_backward(const tcu_linattn_t *a, void *d_ws, size_t ws_bytes, cudaStream_t stream) {
    return backward(a, d_ws, ws_bytes, {}, stream);
}

tcu_status_t tcu_linattn_selftest_timeout(const tcu_linattn_t *a, int backward_pass, uint32_t silent_group, unsigned limit_ms, void *d_ws, size_t ws_bytes,
                                          cudaStream_t stream) {
    if (limit_ms == 0 || limit_ms > 1000 || silent_group == ~0u) return TCU_ERR_INVALID_ARG;
    const Waits waits = {limit_ms * 10, silent_group + 1};             // tries of 100 us
    return backward_pass ? backward(a, d_ws, ws_bytes, waits, stream) : forward(a, d_ws, ws_bytes, waits, stream);
}

tcu_status_t tcu_linattn_step(const tcu_linattn_t *a, cudaStream_t stream) {
    if (!has_struct(a) || (a->type != TCU_F16 && a->type != TCU_BF16)) return TCU_ERR_INVALID_ARG;
    if (a->heads == 0 || a->dk == 0 || a->dv == 0) return TCU_ERR_INVALID_ARG;
    if (a->dk > 128 || a->dv > 128) return TCU_ERR_UNSUPPORTED;
    if (a->batch > (uint64_t(1) << 31) || a->batch * a->heads > (uint64_t(1) << 31) - 1) return TCU_ERR_UNSUPPORTED;
    if (a->batch == 0) return TCU_OK;
    if (!a->d_log_decay || !a->d_state_out || !aligned(a->d_state_out, 16)) return TCU_ERR_INVALID_ARG;
    if (!a->d_slots && a->pool_slots < a->batch) return TCU_ERR_INVALID_ARG;
    if (a->d_slots && !aligned(a->d_slots, 4)) return TCU_ERR_INVALID_ARG;
    const int64_t limit = int64_t(1) << 38;
    for (const tcu_tokens_t *x : {&a->q, &a->k, &a->v, &a->o}) {
        if (!x->ptr || !aligned(x->ptr, 2)) return TCU_ERR_INVALID_ARG;
        if (x->stride_batch < 0 || x->stride_head < 0 || x->stride_batch >= limit || x->stride_head >= limit) return TCU_ERR_INVALID_ARG;
    }
    if ((a->batch > 1 && a->o.stride_batch == 0) || (a->heads > 1 && a->o.stride_head == 0)) return TCU_ERR_INVALID_ARG;
    // Each block reads q and k of its head, and v in the columns of o that it writes; a head has more than one block from dv = 65 on.
    if (a->dv > uint32_t(kStepCols) && (a->o.ptr == a->q.ptr || a->o.ptr == a->k.ptr)) return TCU_ERR_INVALID_ARG;
    StepParams p = {view(a->q), view(a->k), view(a->v), view(a->o), a->d_state_out, a->d_slots, a->d_log_decay, a->pool_slots,
                    uint32_t(a->batch), a->heads, a->dk, a->dv, a->scale};
    const dim3 grid(uint32_t(a->batch) * a->heads, (a->dv + kStepCols - 1) / kStepCols);
    const bool vec = a->dv % 4 == 0;                 // rows of the state are 16-byte aligned
    if (a->type == TCU_F16) {
        if (vec) tcu_linattn_step_kernel<__half, 4><<<grid, kStepThreads, 0, stream>>>(p);
        else tcu_linattn_step_kernel<__half, 1><<<grid, kStepThreads, 0, stream>>>(p);
    } else {
        if (vec) tcu_linattn_step_kernel<__nv_bfloat16, 4><<<grid, kStepThreads, 0, stream>>>(p);
        else tcu_linattn_step_kernel<__nv_bfloat16, 1><<<grid, kStepThreads, 0, stream>>>(p);
    }
    return launched();
}

}  // extern "C"

// ---- embedding
namespace {

constexpr uint64_t kMostTokens = (uint64_t(1) << 30) - 1;
constexpr uint64_t kMostColumns = uint64_t(1) << 20;

// Elements of an access: up to 16 bytes, as far as the row width and the addresses allow.
int vec_of(size_t d, size_t stride, size_t eb, std::initializer_list<const void *> ptrs) {
    for (int vec : {int(16 / eb), 4, 1}) {
        if (size_t(vec) * eb > 16) continue;
        bool ok = d % vec == 0 && stride % vec == 0;
        for (const void *p : ptrs) ok = ok && aligned(p, vec * eb);
        if (ok) return vec;
    }
    return 1;
}

template <typename T, typename ID>
void launch_lookup(int vec, const void *ids, uint32_t n, const void *table, uint32_t rows, uint32_t d, size_t stride, float scale, void *out,
                   cudaStream_t stream) {
    const uint32_t packs = d / vec;
    uint32_t tx = 1;
    while (tx < packs && tx < 256) tx <<= 1;
    const bool many = uint64_t(n) * packs >= uint64_t(256) * 148 * 8;          // enough for every SM with several rows a thread (at this size the same
                                                                               // 4.1 us; 32749 rows of 2048, copied: 41 us a row a thread, 32 four)
    const uint32_t rows_each = (many ? 4 : 1) * (256 / tx);
    const dim3 block(tx, 256 / tx), grid((n + rows_each - 1) / rows_each, (packs + tx - 1) / tx);
    auto go = [&](auto kernel) {
        kernel<<<grid, block, 0, stream>>>(static_cast<const ID *>(ids), n, static_cast<const T *>(table), rows, d, stride, scale, static_cast<T *>(out));
    };
    auto rows_of = [&](auto v) {
        constexpr int VEC = decltype(v)::value;
        if (many) go(tcu_embedding_lookup_kernel<T, ID, VEC, 4>);
        else go(tcu_embedding_lookup_kernel<T, ID, VEC, 1>);
    };
    if constexpr (sizeof(T) == 2) {
        if (vec == 8) return rows_of(std::integral_constant<int, 8>{});
    }
    if (vec == 4) return rows_of(std::integral_constant<int, 4>{});
    rows_of(std::integral_constant<int, 1>{});
}

bool few_tokens(size_t n, size_t rows, size_t d) { return n <= kFewTokens && (d == 0 || rows <= kFewElements / d); }

struct EmbeddingWs {
    size_t keys[2], tokens[2], counts, totals, starts, joins, join, begins, tail, head, bytes;
    uint32_t tiles, pieces;
};
EmbeddingWs embedding_ws(size_t n, size_t rows, size_t d) {
    EmbeddingWs w = {};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    w.tiles = uint32_t((n + kSortTile - 1) / kSortTile);
    w.pieces = uint32_t((n + rows + kPiece - 1) / kPiece);
    for (int i = 0; i < 2; ++i) {
        w.keys[i] = take(n * 4);
        w.tokens[i] = take(n * 4);
    }
    w.counts = take(size_t(kDigits) * w.tiles * 4);
    w.totals = take(kDigits * 4);
    w.starts = take((size_t(w.pieces) + 1) * 8);
    w.joins = take(4);
    w.join = take(size_t(w.pieces) * 8);
    w.begins = take(rows * 4);
    w.tail = take(size_t(w.pieces) * d * 4);
    w.head = take(size_t(w.pieces) * d * 4);
    w.bytes = at;
    return w;
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

// Tiles whose counts every block of the sort adds up by itself; more are scanned by a kernel between.  65536 tokens of 64 columns, 64 tiles:
// 38 us either way; 128 tiles: added 56, scanned 43.
constexpr uint32_t kMostTilesAdded = 64;

template <typename ID>
tcu_status_t sort_tokens(const void *ids, uint32_t n, uint32_t rows, const EmbeddingWs &w, uint8_t *ws, cudaStream_t stream, int &out) {
    int bits = 1;
    while (bits < 32 && (uint64_t(1) << bits) <= rows) ++bits;          // the value `rows` itself must fit
    auto at = [&](size_t o) { return reinterpret_cast<uint32_t *>(ws + o); };
    const uint32_t *keys = nullptr, *tokens = nullptr;
    const ID *id = static_cast<const ID *>(ids);
    out = 0;
    if (n <= kBlockTokens) {
        static std::atomic<int> configured{-1};
        int dev = 0;
        if (!ok(cudaGetDevice(&dev))) return TCU_ERR_CUDA;
        if (configured.load() != dev) {
            if (!ok(cudaFuncSetAttribute(tcu_sort_block_kernel<ID>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(BlockSort))))) return TCU_ERR_CUDA;
            configured.store(dev);
        }
        tcu_sort_block_kernel<ID><<<1, kBlockThreads, sizeof(BlockSort), stream>>>(id, n, rows, bits, at(w.keys[0]), at(w.tokens[0]), at(w.joins));
        return launched();
    }
    for (int shift = 0; shift < bits; shift += kDigitBits) {
        tcu_status_t st = TCU_OK;
        if (shift == 0) {
            tcu_sort_count_kernel<ID><<<w.tiles, kSortThreads, 0, stream>>>(id, keys, n, rows, shift, at(w.counts), at(w.joins));
            st = launched();
        } else {
            st = launch_next(tcu_sort_count_kernel<ID>, w.tiles, kSortThreads, stream, id, keys, n, rows, shift, at(w.counts), nullptr);
        }
        const bool scanned = w.tiles > kMostTilesAdded;
        if (st == TCU_OK && scanned) st = launch_next(tcu_sort_scan_kernel, kDigits / 32, 1024, stream, at(w.counts), w.tiles, at(w.totals));
        if (st == TCU_OK)
            st = launch_next(scanned ? tcu_sort_scatter_kernel<ID, true> : tcu_sort_scatter_kernel<ID, false>, w.tiles, kSortThreads, stream, id, keys, tokens, n, rows,
                             shift, w.tiles, at(w.counts), at(w.totals), at(w.keys[out]), at(w.tokens[out]));
        if (st != TCU_OK) return st;
        keys = at(w.keys[out]);
        tokens = at(w.tokens[out]);
        out ^= 1;
    }
    out ^= 1;
    return TCU_OK;
}

template <typename T, typename TT>
tcu_status_t launch_sum(int vec, const void *d_out, void *table, const SumParams &s, cudaStream_t stream) {
    if (tcu_status_t st = launch_next(tcu_embedding_cut_kernel, s.pieces / 4 + 1, 128, stream, s)) return st;
    auto go = [&](auto v) {
        constexpr int VEC = decltype(v)::value;
        const uint32_t packs = s.d / VEC;
        uint32_t tx = 1;                                        // a group of threads for the columns of a piece
        while (tx < packs && tx < 128) tx <<= 1;
        const dim3 block(tx, 128 / tx), grid((s.pieces + block.y - 1) / block.y, (packs + tx - 1) / tx);
        if (tcu_status_t st = launch_next(tcu_embedding_sum_kernel<T, TT, VEC>, grid, block, stream, static_cast<const T *>(d_out), static_cast<TT *>(table), s)) return st;
        return launch_next(tcu_embedding_join_kernel<TT, VEC < 4 ? VEC : 4>, 148 * 8, 128, stream, static_cast<TT *>(table), s);
    };
    if constexpr (sizeof(T) == 2) {
        if (vec == 8) return go(std::integral_constant<int, 8>{});
    }
    if (vec == 4) return go(std::integral_constant<int, 4>{});
    return go(std::integral_constant<int, 1>{});
}

template <typename T, typename TT, typename ID>
void launch_few(int vec, const void *d_out, const void *ids, void *table, uint32_t n, uint32_t rows, uint32_t d, float scale, int accumulate, cudaStream_t stream) {
    const uint32_t cols = (d + kFewCols - 1) / kFewCols;
    const uint64_t each = (uint64_t(rows) * cols + 148 * 3 - 1) / (148 * 3);       // three blocks an SM, of a row a warp to kFewRows
    const uint32_t rows_each = uint32_t(each < 8 ? 8 : each < kFewRows ? each : kFewRows);
    auto go = [&](auto kernel) {
        kernel<<<dim3((rows + rows_each - 1) / rows_each, cols), 256, 0, stream>>>(static_cast<const T *>(d_out), static_cast<const ID *>(ids), static_cast<TT *>(table), n, rows, d,
                                                                                   scale, accumulate);
    };
    if constexpr (sizeof(T) == 2) {
        if (vec == 8) return go(tcu_embedding_few_kernel<T, TT, ID, 8>);
    }
    if (vec == 4) return go(tcu_embedding_few_kernel<T, TT, ID, 4>);
    go(tcu_embedding_few_kernel<T, TT, ID, 1>);
}

}  // namespace

extern "C" {

tcu_status_t tcu_embedding_forward(const void *d_ids, int id_bytes, size_t n, const void *d_table, size_t rows, size_t d, size_t table_stride,
                                   tcu_float_t type, float scale, void *d_out, cudaStream_t stream) {
    if (!valid_float(type) || (id_bytes != 4 && id_bytes != 8)) return TCU_ERR_INVALID_ARG;
    if (table_stride < d || (rows > 1 && table_stride > uint64_t(1) << 38)) return TCU_ERR_INVALID_ARG;
    if (n > kMostTokens || rows > kMostTokens || d > kMostColumns) return TCU_ERR_UNSUPPORTED;
    if (n == 0 || d == 0) return TCU_OK;
    const size_t eb = float_bytes(type);
    if (!d_ids || !d_out || (!d_table && rows > 0)) return TCU_ERR_INVALID_ARG;
    if (!aligned(d_ids, id_bytes) || !aligned(d_table, eb) || !aligned(d_out, eb)) return TCU_ERR_INVALID_ARG;
    if (overlaps(d_out, n * d * eb, d_table, rows > 1 ? ((rows - 1) * table_stride + d) * eb : rows * d * eb) || overlaps(d_out, n * d * eb, d_ids, n * id_bytes)) return TCU_ERR_INVALID_ARG;
    const int vec = vec_of(d, table_stride, eb, {d_table, d_out});
    auto go = [&](auto t) {
        using T = decltype(t);
        if (id_bytes == 4) launch_lookup<T, int32_t>(vec, d_ids, uint32_t(n), d_table, uint32_t(rows), uint32_t(d), table_stride, scale, d_out, stream);
        else launch_lookup<T, int64_t>(vec, d_ids, uint32_t(n), d_table, uint32_t(rows), uint32_t(d), table_stride, scale, d_out, stream);
    };
    if (type == TCU_F32) go(float{});
    else if (type == TCU_F16) go(__half{});
    else go(__nv_bfloat16{});
    return launched();
}

size_t tcu_embedding_workspace_bytes(size_t n, size_t rows, size_t d) {
    if (n > kMostTokens || rows > kMostTokens) return 0;
    return few_tokens(n, rows, d) ? 256 : embedding_ws(n, rows, d).bytes;
}

tcu_status_t tcu_embedding_backward(const void *d_out, tcu_float_t type, const void *d_ids, int id_bytes, size_t n, size_t rows, size_t d, float scale,
                                    int accumulate, void *d_table, tcu_float_t table_type, void *d_ws, size_t ws_bytes, cudaStream_t stream) {
    if (!valid_float(type) || !valid_float(table_type) || (id_bytes != 4 && id_bytes != 8)) return TCU_ERR_INVALID_ARG;
    if (table_type != TCU_F32 && table_type != type) return TCU_ERR_UNSUPPORTED;
    if (n > kMostTokens || rows > kMostTokens || d > kMostColumns) return TCU_ERR_UNSUPPORTED;
    if (rows == 0 || d == 0) return TCU_OK;
    const size_t eb = float_bytes(type), tb = float_bytes(table_type);
    if (!d_table || !aligned(d_table, tb)) return TCU_ERR_INVALID_ARG;
    if (n == 0) {
        if (accumulate) return TCU_OK;
        return ok(cudaMemsetAsync(d_table, 0, rows * d * tb, stream)) ? TCU_OK : TCU_ERR_CUDA;
    }
    if (!d_out || !d_ids || !aligned(d_ids, id_bytes) || !aligned(d_out, eb)) return TCU_ERR_INVALID_ARG;
    if (!d_ws || ws_bytes < tcu_embedding_workspace_bytes(n, rows, d)) return TCU_ERR_WORKSPACE;
    if (!aligned(d_ws, 256)) return TCU_ERR_INVALID_ARG;
    if (overlaps(d_table, rows * d * tb, d_out, n * d * eb) || overlaps(d_table, rows * d * tb, d_ids, n * id_bytes)) return TCU_ERR_INVALID_ARG;
    int vec = vec_of(d, d, eb, {d_out});
    while (vec > 1 && !aligned(d_table, size_t(vec) * tb)) vec = vec == 8 ? 4 : 1;
    auto with_types = [&](auto go) {
        if (type == TCU_F32) go(float{}, float{});
        else if (type == TCU_F16 && table_type == TCU_F16) go(__half{}, __half{});
        else if (type == TCU_F16) go(__half{}, float{});
        else if (table_type == TCU_BF16) go(__nv_bfloat16{}, __nv_bfloat16{});
        else go(__nv_bfloat16{}, float{});
    };
    if (few_tokens(n, rows, d)) {
        with_types([&](auto t, auto tt) {
            using T = decltype(t);
            using TT = decltype(tt);
            if (id_bytes == 4) launch_few<T, TT, int32_t>(vec, d_out, d_ids, d_table, uint32_t(n), uint32_t(rows), uint32_t(d), scale, accumulate != 0, stream);
            else launch_few<T, TT, int64_t>(vec, d_out, d_ids, d_table, uint32_t(n), uint32_t(rows), uint32_t(d), scale, accumulate != 0, stream);
        });
        return launched();
    }
    const EmbeddingWs w = embedding_ws(n, rows, d);
    uint8_t *ws = static_cast<uint8_t *>(d_ws);
    int last = 0;
    tcu_status_t st = id_bytes == 4 ? sort_tokens<int32_t>(d_ids, uint32_t(n), uint32_t(rows), w, ws, stream, last)
                                    : sort_tokens<int64_t>(d_ids, uint32_t(n), uint32_t(rows), w, ws, stream, last);
    if (st != TCU_OK) return st;
    SumParams s = {};
    s.keys = reinterpret_cast<uint32_t *>(ws + w.keys[last]);
    s.tokens = reinterpret_cast<uint32_t *>(ws + w.tokens[last]);
    s.n = uint32_t(n);
    s.rows = uint32_t(rows);
    s.d = uint32_t(d);
    s.accumulate = accumulate != 0;
    s.pieces = uint32_t(((s.accumulate ? 0 : rows) + n + kPiece - 1) / kPiece);
    s.scale = scale;
    s.joins = reinterpret_cast<uint32_t *>(ws + w.joins);
    s.starts = reinterpret_cast<uint2 *>(ws + w.starts);
    s.join = reinterpret_cast<uint2 *>(ws + w.join);
    s.begins = reinterpret_cast<uint32_t *>(ws + w.begins);
    s.tail = reinterpret_cast<float *>(ws + w.tail);
    s.head = reinterpret_cast<float *>(ws + w.head);
    with_types([&](auto t, auto tt) { st = launch_sum<decltype(t), decltype(tt)>(vec, d_out, d_table, s, stream); });
    return st;
}

}  // extern "C"
