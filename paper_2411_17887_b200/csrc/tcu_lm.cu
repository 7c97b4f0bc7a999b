// Host side of the C ABI declared in include/tcu_lm.h: argument checks, launches.
#include "tcu_lm.h"

#include <cuda_runtime.h>

#include <initializer_list>

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
tcu_status_t launched() { return cudaGetLastError() == cudaSuccess ? TCU_OK : TCU_ERR_CUDA; }

// ---- linear attention
bool has_struct(const tcu_linattn_t *a) { return a && a->struct_bytes == sizeof(tcu_linattn_t); }

// First and one-past-last byte that a token array may touch (packed: batch is 1).
struct Span {
    uintptr_t lo, hi;
};
Span span_of(const tcu_tokens_t &x, uint64_t batch, uint64_t tokens, uint32_t heads, uint32_t width, size_t eb) {
    const uint64_t last = (batch - 1) * uint64_t(x.stride_batch) + (tokens - 1) * uint64_t(x.stride_token) + uint64_t(heads - 1) * uint64_t(x.stride_head) + width;
    const auto lo = reinterpret_cast<uintptr_t>(x.ptr);
    return {lo, lo + last * eb};
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

// What forward and backward share.  `empty` is set when there is nothing to walk (states may still have to be written).
tcu_status_t check_linattn(const tcu_linattn_t *a, const void *d_ws, size_t ws_bytes) {
    if (!has_struct(a)) return TCU_ERR_INVALID_ARG;
    if (a->type != TCU_F16 && a->type != TCU_BF16) return TCU_ERR_INVALID_ARG;
    if (a->heads == 0 || a->dk == 0 || a->dv == 0) return TCU_ERR_INVALID_ARG;
    if (a->dk > 128 || a->dv > 128) return TCU_ERR_UNSUPPORTED;
    if (a->tokens > (uint64_t(1) << 31) - 256) return TCU_ERR_UNSUPPORTED;
    if (a->batch > (uint64_t(1) << 31) || a->batch * a->heads * 3 * 8 > (uint64_t(1) << 31) - 1) return TCU_ERR_UNSUPPORTED;
    if (a->batch == 0) return TCU_OK;
    if (!d_ws || ws_bytes < kStatusBytes) return TCU_ERR_WORKSPACE;
    if (!aligned(d_ws, 16) || !a->d_log_decay || !aligned(a->d_log_decay, 4)) return TCU_ERR_INVALID_ARG;
    if (a->d_offsets && !aligned(a->d_offsets, 8)) return TCU_ERR_INVALID_ARG;
    for (const void *s : {static_cast<const void *>(a->d_state_in), static_cast<const void *>(a->d_state_out),
                          static_cast<const void *>(a->d_dstate_out), static_cast<const void *>(a->d_dstate_in)})
        if (s && !aligned(s, 16)) return TCU_ERR_INVALID_ARG;
    return TCU_OK;
}

tcu_status_t run_mix(const tcu_linattn_t *a, const MixParams &p, cudaStream_t stream) {
    const uint32_t most = a->dk > a->dv ? a->dk : a->dv;
    const dim3 grid(uint32_t(a->batch) * a->heads * p.jobs, (most + kMixCols - 1) / kMixCols);
    if (a->type == TCU_F16) tcu_linattn_mix_kernel<__half><<<grid, 128, 0, stream>>>(p);
    else tcu_linattn_mix_kernel<__nv_bfloat16><<<grid, 128, 0, stream>>>(p);
    return launched();
}

MixParams mix_params(const tcu_linattn_t *a) {
    MixParams p = {};
    p.log_decay = a->d_log_decay;
    p.offsets = a->d_offsets;
    p.tokens = a->tokens;
    p.batch = uint32_t(a->batch);
    p.heads = a->heads;
    return p;
}

}  // namespace

extern "C" {

size_t tcu_linattn_workspace_bytes(void) { return kStatusBytes; }

tcu_status_t tcu_linattn_forward(const tcu_linattn_t *a, void *d_ws, size_t ws_bytes, cudaStream_t stream) {
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
    MixParams p = mix_params(a);
    p.jobs = 1;
    p.job[0] = {view(a->q), view(a->k), view(a->v), view(a->o), a->d_state_in, a->d_state_out, a->dv, 1, a->dk, a->dv, 1, 1.0f, a->scale};
    return run_mix(a, p, stream);
}

tcu_status_t tcu_linattn_backward(const tcu_linattn_t *a, void *d_ws, size_t ws_bytes, cudaStream_t stream) {
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
    } else if (!a->d_dstate_in) {
        return TCU_OK;
    }
    const size_t state = size_t(a->batch) * a->heads * a->dk * a->dv * 4;
    if (overlaps(a->d_dstate_in, state, a->d_dstate_out, state) || overlaps(a->d_dstate_in, state, a->d_state_in, state)) return TCU_ERR_INVALID_ARG;
    MixParams p = mix_params(a);
    p.jobs = 3;
    p.job[0] = {view(a->d_o), view(a->v), view(a->k), view(a->d_q), a->d_state_in, nullptr, 1, a->dv, a->dv, a->dk, 1, 1.0f, a->scale};
    p.job[1] = {view(a->k), view(a->q), view(a->d_o), view(a->d_v), a->d_dstate_out, a->d_dstate_in, a->dv, 1, a->dk, a->dv, 0, a->scale, 1.0f};
    p.job[2] = {view(a->v), view(a->d_o), view(a->q), view(a->d_k), a->d_dstate_out, nullptr, 1, a->dv, a->dv, a->dk, 0, a->scale, 1.0f};
    return run_mix(a, p, stream);
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
void launch_lookup(int vec, const void *ids, uint64_t n, const void *table, uint32_t rows, size_t d, size_t stride, float scale, void *out,
                   cudaStream_t stream) {
    const uint32_t packs = uint32_t(d / vec);
    const uint64_t total = n * packs, blocks = (total + 255) / 256;
    const uint32_t grid = uint32_t(blocks < 148 * 64 ? blocks : 148 * 64);
    auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, stream>>>(static_cast<const ID *>(ids), n, static_cast<const T *>(table), rows, packs, stride, scale, static_cast<T *>(out));
    };
    if constexpr (sizeof(T) == 2) {
        if (vec == 8) return go(tcu_embedding_lookup_kernel<T, ID, 8>);
    }
    if (vec == 4) return go(tcu_embedding_lookup_kernel<T, ID, 4>);
    go(tcu_embedding_lookup_kernel<T, ID, 1>);
}

struct EmbeddingWs {
    size_t keys[2], tokens[2], counts, totals, tail, head, bytes;
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
    w.tail = take(size_t(w.pieces) * d * 4);
    w.head = take(size_t(w.pieces) * d * 4);
    w.bytes = at;
    return w;
}

template <typename ID>
void sort_tokens(const void *ids, uint32_t n, uint32_t rows, const EmbeddingWs &w, uint8_t *ws, cudaStream_t stream, int &out) {
    int bits = 1;
    while (bits < 32 && (uint64_t(1) << bits) <= rows) ++bits;          // the value `rows` itself must fit
    auto at = [&](size_t o) { return reinterpret_cast<uint32_t *>(ws + o); };
    const uint32_t *keys = nullptr, *tokens = nullptr;
    out = 0;
    for (int shift = 0; shift < bits; shift += kDigitBits) {
        const ID *id = static_cast<const ID *>(ids);
        tcu_sort_count_kernel<ID><<<w.tiles, kSortThreads, 0, stream>>>(id, keys, n, rows, shift, w.tiles, at(w.counts));
        tcu_sort_scan_kernel<<<kDigits, kSortThreads, 0, stream>>>(at(w.counts), w.tiles, at(w.totals));
        tcu_sort_scatter_kernel<ID><<<w.tiles, kSortThreads, 0, stream>>>(id, keys, tokens, n, rows, shift, w.tiles, at(w.counts), at(w.totals),
                                                                          at(w.keys[out]), at(w.tokens[out]));
        keys = at(w.keys[out]);
        tokens = at(w.tokens[out]);
        out ^= 1;
    }
    out ^= 1;
}

template <typename T, typename TT>
void launch_sum(int vec, const void *d_out, void *table, const SumParams &s, cudaStream_t stream) {
    auto go = [&](auto sum, auto join) {
        const uint32_t packs = s.d / vec;
        uint32_t tx = 1;
        while (tx < packs && tx < 128) tx <<= 1;
        const dim3 block(tx, 256 / tx > 0 ? 256 / tx : 1);
        const dim3 grid((s.pieces + block.y - 1) / block.y, (packs + tx - 1) / tx);
        sum<<<grid, block, 0, stream>>>(static_cast<const T *>(d_out), static_cast<TT *>(table), s);
        join<<<grid, block, 0, stream>>>(static_cast<TT *>(table), s);
    };
    if constexpr (sizeof(T) == 2) {
        if (vec == 8) return go(tcu_embedding_sum_kernel<T, TT, 8>, tcu_embedding_join_kernel<TT, 8>);
    }
    if (vec == 4) return go(tcu_embedding_sum_kernel<T, TT, 4>, tcu_embedding_join_kernel<TT, 4>);
    go(tcu_embedding_sum_kernel<T, TT, 1>, tcu_embedding_join_kernel<TT, 1>);
}

}  // namespace

extern "C" {

tcu_status_t tcu_embedding_forward(const void *d_ids, int id_bytes, size_t n, const void *d_table, size_t rows, size_t d, size_t table_stride,
                                   tcu_float_t type, float scale, void *d_out, cudaStream_t stream) {
    if (!valid_float(type) || (id_bytes != 4 && id_bytes != 8)) return TCU_ERR_INVALID_ARG;
    if (table_stride < d) return TCU_ERR_INVALID_ARG;
    if (n > kMostTokens || rows > kMostTokens || d > kMostColumns) return TCU_ERR_UNSUPPORTED;
    if (n == 0 || d == 0) return TCU_OK;
    const size_t eb = float_bytes(type);
    if (!d_ids || !d_out || (!d_table && rows > 0)) return TCU_ERR_INVALID_ARG;
    if (!aligned(d_ids, id_bytes) || !aligned(d_table, eb) || !aligned(d_out, eb)) return TCU_ERR_INVALID_ARG;
    if (overlaps(d_out, n * d * eb, d_table, rows ? ((rows - 1) * table_stride + d) * eb : 0) || overlaps(d_out, n * d * eb, d_ids, n * id_bytes)) return TCU_ERR_INVALID_ARG;
    const int vec = vec_of(d, table_stride, eb, {d_table, d_out});
    auto go = [&](auto t) {
        using T = decltype(t);
        if (id_bytes == 4) launch_lookup<T, int32_t>(vec, d_ids, n, d_table, uint32_t(rows), d, table_stride, scale, d_out, stream);
        else launch_lookup<T, int64_t>(vec, d_ids, n, d_table, uint32_t(rows), d, table_stride, scale, d_out, stream);
    };
    if (type == TCU_F32) go(float{});
    else if (type == TCU_F16) go(__half{});
    else go(__nv_bfloat16{});
    return launched();
}

size_t tcu_embedding_workspace_bytes(size_t n, size_t rows, size_t d) {
    if (n > kMostTokens || rows > kMostTokens) return 0;
    const size_t bytes = embedding_ws(n, rows, d).bytes;
    return bytes ? bytes : 256;
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
        return cudaMemsetAsync(d_table, 0, rows * d * tb, stream) == cudaSuccess ? TCU_OK : TCU_ERR_CUDA;
    }
    if (!d_out || !d_ids || !aligned(d_ids, id_bytes) || !aligned(d_out, eb)) return TCU_ERR_INVALID_ARG;
    if (!d_ws || ws_bytes < tcu_embedding_workspace_bytes(n, rows, d)) return TCU_ERR_WORKSPACE;
    if (!aligned(d_ws, 256)) return TCU_ERR_INVALID_ARG;
    if (overlaps(d_table, rows * d * tb, d_out, n * d * eb) || overlaps(d_table, rows * d * tb, d_ids, n * id_bytes)) return TCU_ERR_INVALID_ARG;
    const EmbeddingWs w = embedding_ws(n, rows, d);
    uint8_t *ws = static_cast<uint8_t *>(d_ws);
    int last = 0;
    if (id_bytes == 4) sort_tokens<int32_t>(d_ids, uint32_t(n), uint32_t(rows), w, ws, stream, last);
    else sort_tokens<int64_t>(d_ids, uint32_t(n), uint32_t(rows), w, ws, stream, last);
    SumParams s = {};
    s.keys = reinterpret_cast<uint32_t *>(ws + w.keys[last]);
    s.tokens = reinterpret_cast<uint32_t *>(ws + w.tokens[last]);
    s.n = uint32_t(n);
    s.rows = uint32_t(rows);
    s.d = uint32_t(d);
    s.accumulate = accumulate != 0;
    s.pieces = uint32_t(((s.accumulate ? 0 : rows) + n + kPiece - 1) / kPiece);
    s.scale = scale;
    s.tail = reinterpret_cast<float *>(ws + w.tail);
    s.head = reinterpret_cast<float *>(ws + w.head);
    int vec = vec_of(d, d, eb, {d_out});
    while (vec > 1 && !aligned(d_table, size_t(vec) * tb < 16 ? vec * tb : 16)) vec = vec == 8 ? 4 : 1;
    if (type == TCU_F32) launch_sum<float, float>(vec, d_out, d_table, s, stream);
    else if (type == TCU_F16 && table_type == TCU_F16) launch_sum<__half, __half>(vec, d_out, d_table, s, stream);
    else if (type == TCU_F16) launch_sum<__half, float>(vec, d_out, d_table, s, stream);
    else if (table_type == TCU_BF16) launch_sum<__nv_bfloat16, __nv_bfloat16>(vec, d_out, d_table, s, stream);
    else launch_sum<__nv_bfloat16, float>(vec, d_out, d_table, s, stream);
    return launched();
}

}  // extern "C"
