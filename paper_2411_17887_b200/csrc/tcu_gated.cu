// Host side of the gated linear recurrence (include/tcu_lm.h): argument checks, launches.
#include "tcu_lm.h"

#include <cuda_runtime.h>
#include <stddef.h>

#include <initializer_list>
#include <type_traits>

#include "tcu_gated_kernel.cuh"
#include "tcu_host.h"

namespace {

using namespace tcu;

constexpr uint64_t kMostWalks = (uint64_t(1) << 31) - 1;
constexpr uint64_t kMostTokens = (uint64_t(1) << 31) - 8192;                // (positions ahead of the last tile are 32-bit integers too)
constexpr uint32_t kMostChannels = uint32_t(1) << 30;
constexpr uint64_t kSms = 148, kSharedOfSm = 228 * 1024, kSharedOfBlock = 1024;              // (shared memory of an SM, and what a block takes of it besides its own)
constexpr int64_t kMostStride = int64_t(1) << 38;
constexpr size_t kBytesBeforeClear = offsetof(tcu_gated_t, clear_rows);     // of the structure when it ended ahead of clear_rows, which is then 0

// First and one-past-last byte that an array may touch; to the end of all addresses if it has no such last byte.
struct Span {
    uintptr_t lo, hi;
};
bool meet(const Span &a, const Span &b) { return a.lo < b.hi && b.lo < a.hi; }

struct Sizes {
    bool packed;
    uint64_t batch, tokens;
    uint32_t channels;
    size_t element;
    Span span(const tcu_rows_t &r) const {
        using Wide = unsigned __int128;
        const auto lo = reinterpret_cast<uintptr_t>(r.ptr);
        if (tokens == 0 || batch == 0) return {lo, lo};
        const Wide last = (packed ? Wide(0) : Wide(batch - 1) * uint64_t(r.stride_batch)) + Wide(tokens - 1) * uint64_t(r.stride_token) + channels;
        const Wide end = lo + last * element;
        return {lo, end > ~uintptr_t(0) ? ~uintptr_t(0) : uintptr_t(end)};
    }
    Span states(const float *s) const {
        const auto lo = reinterpret_cast<uintptr_t>(s);
        const unsigned __int128 end = (unsigned __int128)(lo) + (unsigned __int128)(batch) * channels * 4;
        return {lo, end > ~uintptr_t(0) ? ~uintptr_t(0) : uintptr_t(end)};
    }
    bool right(const tcu_rows_t &r, bool written) const {
        if (!r.ptr || !aligned(r.ptr, element)) return false;
        for (int64_t s : {packed ? 0 : r.stride_batch, r.stride_token})
            if (s < 0 || s > kMostStride) return false;
        return !written || !((!packed && batch > 1 && r.stride_batch == 0) || (tokens > 1 && r.stride_token == 0));
    }
    // `count` indices of `bytes` each, or none
    static Span indices(const void *p, uint64_t count, size_t bytes) {
        const auto lo = reinterpret_cast<uintptr_t>(p);
        const unsigned __int128 end = (unsigned __int128)(lo) + (p ? (unsigned __int128)(count) * bytes : 0);
        return {lo, end > ~uintptr_t(0) ? ~uintptr_t(0) : uintptr_t(end)};
    }
    // whether all rows of an array begin at multiples of `bytes`, and have a number of them
    bool multiples(const tcu_rows_t &r, size_t bytes) const {
        const int64_t each = int64_t(bytes / element);
        return !r.ptr || (channels % each == 0 && aligned(r.ptr, bytes) && (tokens <= 1 || r.stride_token % each == 0) && (packed || batch <= 1 || r.stride_batch % each == 0));
    }
    // How arrays are read and written: 16 bytes and two channels at a time, 4 bytes and two channels, or one channel.
    int way(std::initializer_list<const tcu_rows_t *> in, std::initializer_list<const tcu_rows_t *> out) const {
        bool sixteen = true, four = true, two = true;
        for (const tcu_rows_t *r : in) {
            sixteen = sixteen && multiples(*r, 16);
            four = four && multiples(*r, 4);
        }
        for (const tcu_rows_t *r : out) two = two && multiples(*r, 2 * element);
        return two && sixteen ? 0 : two && four ? 1 : 2;
    }
};

GatedRows rows(const tcu_rows_t &r) { return {r.ptr, r.stride_batch, r.stride_token}; }

GatedParams params(const tcu_gated_t *a) {
    GatedParams p = {};
    p.x = rows(a->x);
    p.gate = rows(a->gate);
    p.y = rows(a->y);
    p.d_y = rows(a->d_y);
    p.d_x = rows(a->d_x);
    p.d_gate = rows(a->d_gate);
    p.offsets = a->d_offsets;
    p.state_in = a->d_state_in;
    p.state_out = a->d_state_out;
    p.d_state_out = a->d_dstate_out;
    p.d_state_in = a->d_dstate_in;
    p.marks = a->d_marks;
    p.tokens = a->tokens;
    p.channels = a->channels;
    p.strips = (a->channels + kGatedChannels - 1) / kGatedChannels;
    return p;
}

tcu_status_t check(const tcu_gated_t *a, uint64_t tokens, Sizes &s) {
    if (!a || (a->struct_bytes != sizeof(tcu_gated_t) && a->struct_bytes != kBytesBeforeClear)) return TCU_ERR_INVALID_ARG;
    if (!valid_float(int(a->type)) || a->input_gate > TCU_INPUT_ROOT || a->channels == 0) return TCU_ERR_INVALID_ARG;
    if (a->channels > kMostChannels || tokens > kMostTokens) return TCU_ERR_UNSUPPORTED;
    const uint64_t strips = (uint64_t(a->channels) + kGatedChannels - 1) / kGatedChannels;
    if (a->batch > kMostWalks / strips) return TCU_ERR_UNSUPPORTED;
    if (!aligned(a->d_offsets, 8)) return TCU_ERR_INVALID_ARG;
    for (const void *q : {static_cast<const void *>(a->d_state_in), static_cast<const void *>(a->d_state_out), static_cast<const void *>(a->d_marks),
                          static_cast<const void *>(a->d_dstate_out), static_cast<const void *>(a->d_dstate_in)})
        if (!aligned(q, 4)) return TCU_ERR_INVALID_ARG;
    s = {a->d_offsets != nullptr, a->batch, tokens, a->channels, float_bytes(tcu_float_t(a->type))};
    return TCU_OK;
}

// Calls go(type, input gate) with these as types.
template <typename F>
void dispatch(const tcu_gated_t *a, F go) {
    auto input = [&](auto t) {
        if (a->input_gate == TCU_INPUT_COMPLEMENT) go(t, std::integral_constant<int, kInputComplement>{});
        else if (a->input_gate == TCU_INPUT_ONE) go(t, std::integral_constant<int, kInputOne>{});
        else go(t, std::integral_constant<int, kInputRoot>{});
    };
    if (a->type == TCU_F32) input(float{});
    else if (a->type == TCU_F16) input(__half{});
    else input(__nv_bfloat16{});
}

// Blocks that the SMs hold at once, two an SM by their registers, if their shared memory lets them.  (bytes: of it, by the blocks of a cluster)
template <auto bytes>
uint64_t blocks_at_once(uint32_t ranks) { return kSms * (2 * (bytes(ranks) + kSharedOfBlock) <= kSharedOfSm ? 2 : 1); }

// Blocks of a cluster that walk a sequence together: as many as keep all blocks on the SMs at once and have a tile each.  16383 tokens of
// 2048 channels, 32 walks: 8 blocks 61 us, 4 blocks 82; 8 x 4096 tokens, 256 walks: one block 81 us, two 111.  Gradients of 32-bit
// elements have room for two blocks an SM only where a block walks alone (off 16 bytes not even there): 8 x 4096 tokens of 1024 channels, 128 walks, one block
// 124 us, two 171; 32 walks of 16383 tokens, four blocks 175, eight 267.  Packed sequences are of lengths
// that the host does not know, and the longest alone may take most of the time: up to four times as many blocks (24 sequences of 1504 channels,
// 16001 tokens: of 0 to 3972 each, one block 61 us, two 53; of 667 each 38 and 54).
template <auto bytes>
uint32_t blocks_of_walk(uint64_t walks, const Sizes &s) {
    const uint64_t tiles = s.packed ? 4 * s.tokens / s.batch / 128 : (s.tokens + 127) / 128;
    uint32_t ranks = 1;
    while (ranks < kGatedMaxCluster && walks * ranks * 2 <= (s.packed ? 4 : 1) * blocks_at_once<bytes>(ranks * 2) && ranks * 2 <= tiles) ranks *= 2;
    return ranks;
}

template <auto kernel, auto bytes>
tcu_status_t launch_walks(const GatedParams &p, const Sizes &s, cudaStream_t stream) {
    if (!allow_shared<kernel>(bytes(kGatedMaxCluster))) return TCU_ERR_CUDA;
    GatedParams q = p;
    const uint64_t batch = s.batch;
    q.ranks = blocks_of_walk<bytes>(batch * p.strips, s);
    // Long packed sequences first, where not all blocks run at once: 24 sequences of 0 to 3972 tokens, 1504 channels, 73 -> 53 us.  Found by every block for
    // itself: 200 sequences of 100 tokens would take 87 us instead of 54, and need it less.
    if (p.offsets && batch > 1 && batch <= kGatedOrdered && batch * p.strips * q.ranks > blocks_at_once<bytes>(q.ranks)) q.ordered = int(batch);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = q.ranks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(uint32_t(batch * p.strips * q.ranks));
    cfg.blockDim = dim3(kGatedWarps * 32);
    cfg.dynamicSmemBytes = bytes(q.ranks);
    cfg.stream = stream;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return ok(cudaLaunchKernelEx(&cfg, kernel, q)) ? TCU_OK : TCU_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t tcu_gated_marks_bytes(uint64_t batch, uint64_t tokens, uint32_t channels) {
    const unsigned __int128 bytes = ((unsigned __int128)(tokens / kGatedMark) + batch) * channels * 4;
    return bytes >> 63 ? 0 : size_t(bytes);
}

tcu_status_t tcu_gated_forward(const tcu_gated_t *a, cudaStream_t stream) {
    Sizes s;
    if (tcu_status_t st = check(a, a ? a->tokens : 0, s)) return st;
    if (a->batch == 0) return TCU_OK;
    const bool tokens = a->tokens > 0;
    if (tokens && (!s.right(a->x, false) || !s.right(a->gate, false) || (a->y.ptr && !s.right(a->y, true)))) return TCU_ERR_INVALID_ARG;
    const uint64_t all = s.packed ? a->tokens : a->batch * a->tokens;
    const size_t marks = tcu_gated_marks_bytes(a->batch, all, a->channels);
    if (a->d_marks && (marks == 0 || a->marks_bytes < marks)) return TCU_ERR_WORKSPACE;
    const Span inputs[] = {s.span(a->x), s.span(a->gate), Sizes::indices(a->d_offsets, a->batch + 1, 8)};
    const Span y = a->y.ptr ? s.span(a->y) : Span{0, 0};
    const Span kept = a->d_marks ? Span{reinterpret_cast<uintptr_t>(a->d_marks), reinterpret_cast<uintptr_t>(a->d_marks) + marks} : Span{0, 0};
    const Span in = a->d_state_in ? s.states(a->d_state_in) : Span{0, 0}, out = a->d_state_out ? s.states(a->d_state_out) : Span{0, 0};
    for (const Span &w : {y, kept, out})
        for (const Span &i : inputs)
            if (meet(w, i)) return TCU_ERR_INVALID_ARG;
    if (meet(y, kept) || meet(y, out) || meet(y, in) || meet(kept, out) || meet(kept, in)) return TCU_ERR_INVALID_ARG;
    if (a->d_state_in != a->d_state_out && meet(in, out)) return TCU_ERR_INVALID_ARG;
    GatedParams p = params(a);
    tcu_status_t st = TCU_OK;
    const int way = s.way({&a->x, &a->gate}, {&a->y});
    dispatch(a, [&](auto t, auto in) {
        using T = decltype(t);
        constexpr int kInput = decltype(in)::value, kLast = sizeof(T) == 2 ? 2 : 4;
        if (way == 0) st = launch_walks<tcu_gated_forward_kernel<T, kInput, 16, true>, forward_bytes<T, 16>>(p, s, stream);
        else if (way == 1) st = launch_walks<tcu_gated_forward_kernel<T, kInput, 4, true>, forward_bytes<T, 4>>(p, s, stream);
        else st = launch_walks<tcu_gated_forward_kernel<T, kInput, kLast, false>, forward_bytes<T, kLast>>(p, s, stream);
    });
    return st;
}

tcu_status_t tcu_gated_backward(const tcu_gated_t *a, cudaStream_t stream) {
    Sizes s;
    if (tcu_status_t st = check(a, a ? a->tokens : 0, s)) return st;
    if (a->batch == 0) return TCU_OK;
    if (a->tokens > 0) {
        for (const tcu_rows_t *r : {&a->x, &a->gate, &a->d_y})
            if (!s.right(*r, false)) return TCU_ERR_INVALID_ARG;
        for (const tcu_rows_t *r : {&a->d_x, &a->d_gate})
            if (!s.right(*r, true)) return TCU_ERR_INVALID_ARG;
        if (a->d_x.ptr == a->d_gate.ptr) return TCU_ERR_INVALID_ARG;
    }
    const uint64_t clear = a->struct_bytes == kBytesBeforeClear ? 0 : a->clear_rows;
    if (clear > 1) return TCU_ERR_INVALID_ARG;
    const size_t marks = tcu_gated_marks_bytes(a->batch, s.packed ? a->tokens : a->batch * a->tokens, a->channels);
    if (!a->d_marks || marks == 0 || a->marks_bytes < marks) return TCU_ERR_WORKSPACE;
    const Span kept = {reinterpret_cast<uintptr_t>(a->d_marks), reinterpret_cast<uintptr_t>(a->d_marks) + marks};
    const Span in = a->d_dstate_out ? s.states(a->d_dstate_out) : Span{0, 0}, out = a->d_dstate_in ? s.states(a->d_dstate_in) : Span{0, 0};
    const Span inputs[] = {s.span(a->x), s.span(a->gate), s.span(a->d_y), kept, Sizes::indices(a->d_offsets, a->batch + 1, 8)};
    const Span dx = s.span(a->d_x), dg = s.span(a->d_gate);
    for (const Span &w : {dx, dg, out})
        for (const Span &i : inputs)
            if (meet(w, i)) return TCU_ERR_INVALID_ARG;
    if (meet(dx, in) || meet(dg, in) || meet(dx, out) || meet(dg, out)) return TCU_ERR_INVALID_ARG;
    if (a->d_dstate_in != a->d_dstate_out && meet(in, out)) return TCU_ERR_INVALID_ARG;
    GatedParams p = params(a);
    tcu_status_t st = TCU_OK;
    p.clear = clear && s.packed && a->tokens > 0;
    const int way = s.way({&a->x, &a->gate, &a->d_y}, {&a->d_x, &a->d_gate});
    dispatch(a, [&](auto t, auto in) {
        using T = decltype(t);
        constexpr int kInput = decltype(in)::value, kLast = sizeof(T) == 2 ? 2 : 4;
        if (way == 0) st = launch_walks<tcu_gated_backward_kernel<T, kInput, 16, true>, backward_bytes<T, 16>>(p, s, stream);
        else if (way == 1) st = launch_walks<tcu_gated_backward_kernel<T, kInput, 4, true>, backward_bytes<T, 4>>(p, s, stream);
        else st = launch_walks<tcu_gated_backward_kernel<T, kInput, kLast, false>, backward_bytes<T, kLast>>(p, s, stream);
    });
    return st;
}

tcu_status_t tcu_gated_step(const tcu_gated_t *a, cudaStream_t stream) {
    Sizes s;
    if (tcu_status_t st = check(a, 1, s)) return st;
    if (a->d_offsets) return TCU_ERR_INVALID_ARG;
    if (a->batch == 0) return TCU_OK;
    if (!s.right(a->x, false) || !s.right(a->gate, false) || !s.right(a->y, true)) return TCU_ERR_INVALID_ARG;
    if (!a->d_state_out || !aligned(a->d_slots, 4) || (!a->d_slots && a->pool_slots < a->batch)) return TCU_ERR_INVALID_ARG;
    if (a->batch > (kMostWalks * 256) / a->channels) return TCU_ERR_UNSUPPORTED;
    Sizes pool = s;
    pool.batch = a->pool_slots;
    const Span states = pool.states(a->d_state_out), y = s.span(a->y), slots = Sizes::indices(a->d_slots, a->batch, 4);
    if (meet(slots, states) || meet(slots, y)) return TCU_ERR_INVALID_ARG;
    if (meet(states, y) || meet(states, s.span(a->x)) || meet(states, s.span(a->gate))) return TCU_ERR_INVALID_ARG;
    for (const tcu_rows_t *r : {&a->x, &a->gate})
        if (meet(y, s.span(*r)) && !(r->ptr == a->y.ptr && (a->batch == 1 || r->stride_batch == a->y.stride_batch))) return TCU_ERR_INVALID_ARG;
    const GatedParams p = params(a);
    const uint64_t blocks = (a->batch * a->channels + 255) / 256;
    dispatch(a, [&](auto t, auto in) {
        tcu_gated_step_kernel<decltype(t), decltype(in)::value><<<uint32_t(blocks), 256, 0, stream>>>(p, a->d_slots, a->pool_slots, uint32_t(a->batch));
    });
    return launched();
}

}  // extern "C"
