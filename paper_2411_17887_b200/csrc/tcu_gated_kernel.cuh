// Gated linear recurrence: for every channel on its own, with f = sigmoid(gate),
//     h_t = f_t h_{t-1} + i_t x_t          i = 1 - f, 1 or sqrt(1 - f^2)
// an inclusive scan over pairs (f, b) with (f, b) before (f', b') giving (f f', f' b + b').  Its gradients are the same scan
// backward in time: with D_t the gradient with respect to h_t and C_t what flows into it from later tokens,
//     D_t = dy_t + C_t    C_{t-1} = f_t D_t    dx_t = i_t D_t    dgate_t = D_t (h_{t-1} f_t' + x_t i_t')
// where h is formed once more from the states that the forward pass leaves every kGatedMark tokens (marks).
//
// A block walks a sequence for 64 channels, a tile of 128 tokens (backward, and for 32-bit elements: 64) at a time: a warp takes 16 (8)
// tokens of it, two channels a lane, and scans them in registers; the warps' pairs go through shared memory, and what arrives at a warp from
// before is added as P_t h (P the product of the f so far): every value is read and written once.  Where there are fewer walks than
// SMs hold blocks, the blocks of a cluster walk a sequence together, a tile each, and tell one another their tiles' pairs.  The order of
// all sums follows from the sizes alone.
//
// What bounds it: instructions (28 an element forward, two of them on the special-function unit; 52 backward) and the barrier of a tile, close behind
// memory.  8 x 4096 tokens of 2048 bfloat16 channels: forward 81 us (403 MB, 4.9 TB/s, 0.75 of the copy rate), backward 148 us (671 MB, 4.5
// TB/s).  Tried: values through registers instead of shared memory (215 us, loads wait for the store of the tile before), 8 tokens a warp forward
// (110), two channels an instruction (no gain: moves into register pairs), a barrier of the block for the tile's arrival (88).
#pragma once

#include <cooperative_groups.h>

#include "tcu_float.cuh"

namespace tcu {

constexpr int kGatedMark = 64;             // tokens between marks
constexpr int kGatedWarps = 8;
constexpr int kGatedChannels = 64;
constexpr int kGatedMaxCluster = 8;
constexpr int kGatedOrdered = 64;          // packed sequences that blocks order by length

enum GatedInput { kInputComplement = 0, kInputOne = 1, kInputRoot = 2 };

struct GatedRows {
    void *ptr;
    int64_t batch, token;      // strides, in elements
};

struct GatedParams {
    GatedRows x, gate, y, d_y, d_x, d_gate;
    const int64_t *offsets;    // packed sequences, or nullptr
    const float *state_in;     // (batch, channels), or nullptr
    float *state_out;
    const float *d_state_out;
    float *d_state_in;
    float *marks;              // (tokens / kGatedMark + batch, channels): sequence b's begin at row first token / kGatedMark + b
    uint64_t tokens;           // of each sequence (dense), of all together (packed)
    uint32_t channels, strips;
    uint32_t ranks;            // blocks of a cluster
    int ordered;               // packed: so many sequences (at most kGatedOrdered) are walked in the order of their lengths; or 0
    int clear;                 // packed, backward: rows that belong to no sequence are set to zero
};

// Stores the two channels of a lane: in one access where they are aligned for it (PAIR), else one each.
template <typename T, bool PAIR>
__device__ __forceinline__ void store_two(T *p, float a, float b, bool first, bool second) {
    if constexpr (PAIR) {
        if (first) *reinterpret_cast<Pack<T, 2> *>(p) = two_from_f32<T>(a, b);
    } else {
        if (first) p[0] = from_f32<T>(a);
        if (second) p[1] = from_f32<T>(b);
    }
}

// Arithmetic on the two channels of a lane.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return make_float2(fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return make_float2(a.x * b.x, a.y * b.y); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float reciprocal(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float minus_size(float g) {              // -|g|, at least -200: exp is 0 from -104 on, and infinities would leave inf - inf
    float u;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(u) : "f"(-fabsf(g)), "f"(-200.0f));
    return u;
}

// f = sigmoid(g) and 1 - f.  The smaller of the two is a / (1 + a), a = exp(-|g|), to a few 2^-23 of itself, the larger one less it:
// f of a channel with a long memory is off by its rounding alone.  a is 2^t for the rounded product t of -|g| and log2(e); FINE, what
// the rounding leaves, -|g| - t ln 2, is added to first order.  Without it a is off by up to 1.23 |g| 2^-24 of itself besides (the product is rounded by 2^-24 of |t| at most,
// the constant by 0.23 of that, both times ln 2): below 2^-17 where |g| is at most 80, on the smaller side alone.  Whole sequences of 16-bit elements go without it, as
// their gates and outputs are rounded by 2^-9 or 2^-12: 8 x 4096 tokens of 2048 channels 81 and 148 us, with it 87 and 153.  Single tokens, bound by memory, have it.
template <bool FINE>
__device__ __forceinline__ void sigmoids(float2 g, float2 &f, float2 &rest) {
    float2 u, t;
    if constexpr (FINE) {
        u = make_float2(minus_size(g.x), minus_size(g.y));
        t = mul2(u, both(1.4426950408889634f));
    } else {
        t = make_float2(fabsf(g.x) * -1.4426950408889634f, fabsf(g.y) * -1.4426950408889634f);
    }
    float2 a;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(t.y));
    if constexpr (FINE) a = fma2(a, fma2(t, both(-0.6931471805599453f), u), a);
    const float2 sum = make_float2(1.0f + a.x, 1.0f + a.y);
    const float2 less = mul2(a, make_float2(reciprocal(sum.x), reciprocal(sum.y))), more = make_float2(1.0f - less.x, 1.0f - less.y);
    f = make_float2(g.x >= 0.0f ? more.x : less.x, g.y >= 0.0f ? more.y : less.y);
    rest = make_float2(g.x >= 0.0f ? less.x : more.x, g.y >= 0.0f ? less.y : more.y);
}

template <int INPUT>
__device__ __forceinline__ float2 input_of(float2 f, float2 rest) {
    if constexpr (INPUT == kInputComplement) return rest;
    if constexpr (INPUT == kInputOne) return both(1.0f);
    const float2 square = fma2(rest, f, rest);
    float2 i;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(i.x) : "f"(square.x));
    asm("sqrt.approx.f32 %0, %1;" : "=f"(i.y) : "f"(square.y));
    return i;
}
template <int INPUT>
__device__ __forceinline__ float2 taken_in(float2 f, float2 rest, float2 x) {
    if constexpr (INPUT == kInputOne) return x;
    else return mul2(input_of<INPUT>(f, rest), x);
}

// The gate's gradient over that of h, h_{t-1} f' + x i', from what has been taken in, i x: f' = f (1 - f), and i' is -f (1 - f), 0 or
// -f^2 i / (1 + f).
template <int INPUT>
__device__ __forceinline__ float2 gate_slope(float2 f, float2 rest, float2 before, float2 in) {
    if constexpr (INPUT == kInputComplement) return mul2(f, fma2(rest, before, make_float2(-in.x, -in.y)));
    if constexpr (INPUT == kInputOne) return mul2(f, mul2(rest, before));
    const float2 more = make_float2(f.x * reciprocal(1.0f + f.x), f.y * reciprocal(1.0f + f.y));
    return mul2(f, fma2(rest, before, mul2(more, make_float2(-in.x, -in.y))));
}

// One token of one channel.
template <int INPUT>
__device__ __forceinline__ float next_state(float g, float x, float h) {
    float2 f, rest;
    sigmoids<true>(both(g), f, rest);
    return fmaf(f.x, h, taken_in<INPUT>(f, rest, both(x)).x);
}

// One block's place: sequence, channels, tokens.
struct GatedWalk {
    uint32_t seq, c0;
    int64_t begin;             // of the sequence, in rows of the arrays (dense: 0)
    int len;
    uint64_t mark;             // row of its first mark
    // (shared: a number for each thread and one more, free again after the call)
    __device__ __forceinline__ GatedWalk(const GatedParams &p, uint32_t walk, int *shared) {
        seq = walk / p.strips;
        c0 = (walk - seq * p.strips) * kGatedChannels;
        if (!p.offsets) {
            begin = 0;
            len = int(p.tokens);
            mark = uint64_t(seq) * p.tokens / kGatedMark + seq;
            return;
        }
        if (p.ordered > 0) {           // long sequences first: the one with `seq` longer ones
            const int t = int(threadIdx.x), n = t < p.ordered ? length(p, t) : -1;
            shared[t] = n;
            __syncthreads();
            uint32_t longer = 0;
            if (t < p.ordered) {
                for (int k = 0; k < p.ordered; k += 4) {
                    const int4 m = *reinterpret_cast<const int4 *>(shared + k);
                    longer += (m.x > n || (m.x == n && k < t)) + (m.y > n || (m.y == n && k + 1 < t)) + (m.z > n || (m.z == n && k + 2 < t)) + (m.w > n || (m.w == n && k + 3 < t));
                }
            }
            if (t < p.ordered && longer == seq) shared[kGatedWarps * 32] = t;
            __syncthreads();
            seq = uint32_t(shared[kGatedWarps * 32]);
            __syncthreads();
        }
        begin = first(p, seq);
        len = length(p, seq);
        mark = uint64_t(begin) / kGatedMark + seq;
    }
    // offsets that are not as they should be may give wrong results, but no access outside the arrays
    static __device__ __forceinline__ int64_t first(const GatedParams &p, uint32_t s) { return min(max(p.offsets[s], int64_t(0)), int64_t(p.tokens)); }
    static __device__ __forceinline__ int length(const GatedParams &p, uint32_t s) {
        const int64_t b = first(p, s);
        return int(min(max(p.offsets[s + 1], b), int64_t(p.tokens)) - b);
    }
    template <typename T>
    __device__ __forceinline__ T *at(const GatedParams &p, const GatedRows &r, uint32_t c) const {
        return static_cast<T *>(r.ptr) + (p.offsets ? begin * r.token : int64_t(seq) * r.batch) + c;
    }
};

// Rows of the inputs on their way to shared memory, 16 bytes a piece.  A warp copies what it reads itself, so that no barrier of the block waits for data.
// COPY 16: all rows begin at multiples of 16 bytes.  COPY 4, 2: at multiples of that many bytes; the pieces that hold a row are copied, the last one as far
// as the row goes, and the row is read from behind what its first piece holds ahead of it (bytes of the same allocation: those begin at larger boundaries).
// Measured, 8 x 4096 tokens of 2047 bfloat16 channels: forward 139 us, backward 273; in words of 4 bytes 179 and 259.  2046: 116 and 212 (147 and 192).
// 2048 tokens of 2047 fp32: 93 and 181 (124 and 202).  Results stored in words across the lanes' pairs: 161 and 294 instead of 143 and 270.
__device__ __forceinline__ void copy_async16(void *to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(uint32_t(__cvta_generic_to_shared(to))), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async16(void *to, const void *from, uint32_t bytes) {         // the rest is set to zero
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(uint32_t(__cvta_generic_to_shared(to))), "l"(from), "r"(bytes) : "memory");
}
template <int N>
__device__ __forceinline__ void copies_but(void) {                  // waits for all but the last N commits of this thread
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <typename T, int STEPS, int COPY>
struct alignas(16) GatedRowsOf {           // of a warp
    static constexpr int kPieces = kGatedChannels * int(sizeof(T)) / 16 + (COPY == 16 ? 0 : 1);
    T v[STEPS][kPieces * 16 / sizeof(T)];
};

// One array's rows, those of a tile after those of another.  Rows that are not there, and channels, are left as they are.
template <typename T, int STEPS, int COPY>
struct GatedSource {
    using Rows = GatedRowsOf<T, STEPS, COPY>;
    static constexpr int kPieces = Rows::kPieces, kEach = 16 / int(sizeof(T)), kRows = 32 / kPieces;   // COPY 16: rows of an access
    const T *at;                           // row (COPY 16: of this lane's first piece) of the next tile
    int64_t stride, step;                  // a row to the next one, a tile to the next one (in elements)
    __device__ __forceinline__ GatedSource(const T *array, int first, int64_t stride, int tokens_on) : stride(stride) {
        at = array + (int64_t(first) + (COPY == 16 ? int((threadIdx.x & 31) / kPieces) : 0)) * stride;
        step = tokens_on * stride;
    }
    // How many bytes behind its first piece the row of token s of a tile begins, whose first row is `row`.
    static __device__ __forceinline__ uint32_t behind(const T *row, int64_t stride, int s) {
        return COPY == 16 ? 0 : (uint32_t(reinterpret_cast<uintptr_t>(row)) + uint32_t(stride) * uint32_t(sizeof(T)) * uint32_t(s)) & 15;
    }
    template <bool ALL>
    __device__ __forceinline__ void copy(Rows &rows, int n, int channels) {
        const uint32_t lane = threadIdx.x & 31;
        if constexpr (COPY == 16) {
            const int row = int(lane / kPieces), c = int(lane % kPieces) * kEach;
            const T *src = at + c;
#pragma unroll
            for (int k = 0; k < STEPS; k += kRows, src += stride * kRows)
                if ((ALL || row + k < n) && c < channels) copy_async16(&rows.v[row + k][c], src);
        } else {
            constexpr int kWhole = kPieces - 1, kAt = 32 / kWhole;             // the last piece of every row apart from the others
            const int first = int(lane / kWhole), piece = int(lane % kWhole), bytes = channels * int(sizeof(T));
            uintptr_t begin = reinterpret_cast<uintptr_t>(at + int64_t(first) * stride);
#pragma unroll
            for (int k = 0; k < STEPS; k += kAt, begin += uint64_t(stride * kAt) * sizeof(T)) {
                const int left = int(begin & 15) + bytes - 16 * piece;
                if ((ALL || first + k < n) && left > 0)
                    copy_async16(&rows.v[first + k][piece * kEach], reinterpret_cast<const void *>((begin & ~uintptr_t(15)) + 16 * piece), uint32_t(min(left, 16)));
            }
            if (int(lane) < (ALL ? STEPS : n)) {                                // (n: 0 or less, of a warp behind the end)
                begin = reinterpret_cast<uintptr_t>(at + int64_t(lane) * stride);
                const int left = int(begin & 15) + bytes - 16 * kWhole;
                if (left > 0) copy_async16(&rows.v[lane][kWhole * kEach], reinterpret_cast<const void *>((begin & ~uintptr_t(15)) + 16 * kWhole), uint32_t(left));
            }
        }
    }
    // the first n rows are there, and `channels`
    __device__ __forceinline__ void load(Rows &rows, int n, int channels) {
        if (n >= STEPS) copy<true>(rows, n, channels);
        else copy<false>(rows, n, channels);
        at += step;
    }
};

// Two channels of a token of a warp, whose row begins `behind` its first piece.
template <typename T, int STEPS, int COPY>
__device__ __forceinline__ float2 pair_of(const GatedRowsOf<T, STEPS, COPY> &rows, int s, uint32_t behind) {
    const uint32_t lane = threadIdx.x & 31;
    if constexpr (COPY == 16) {
        return two_f32<T>(*reinterpret_cast<const Pack<T, 2> *>(&rows.v[s][2 * lane]));
    } else if constexpr (sizeof(T) == 4) {
        const T *at = &rows.v[s][2 * lane] + behind / 4;
        return make_float2(at[0], at[1]);
    } else {
        const uint32_t *words = reinterpret_cast<const uint32_t *>(&rows.v[s][2 * lane]) + behind / 4;
        const uint32_t two = COPY == 2 ? __funnelshift_r(words[0], words[1], (behind & 2) * 8) : words[0];
        return two_f32<T>(*reinterpret_cast<const Pack<T, 2> *>(&two));
    }
}

// Sets the rows from n on to a value.  What the tokens that are not there look like: a gate of infinity, f = 1, and zeros, nothing that comes in,
// so that states and gradients pass them as they are.
template <typename T, int STEPS, int COPY>
__device__ __forceinline__ void fill_rows(GatedRowsOf<T, STEPS, COPY> &rows, int n, float value) {
    const uint32_t lane = threadIdx.x & 31;
    for (int s = max(n, 0); s < STEPS; ++s)
        for (uint32_t c = lane; c < sizeof(rows.v[0]) / sizeof(T); c += 32) rows.v[s][c] = from_f32<T>(value);
    __syncwarp();
}

template <typename T, bool PAIR, int STEPS>
__device__ __forceinline__ void store_rows(T *at, int64_t stride, int n, bool c0, bool c1, const float2 (&v)[STEPS]) {
    if (n >= STEPS) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s, at += stride) store_two<T, PAIR>(at, v[s].x, v[s].y, c0, c1);
    } else {
#pragma unroll
        for (int s = 0; s < STEPS; ++s, at += stride) store_two<T, PAIR>(at, v[s].x, v[s].y, s < n && c0, s < n && c1);
    }
}

// Sets the rows of d_x and d_gate that lie ahead of the first sequence and behind the last one to zero, in the channels of this block: the blocks of these channels
// take turns.  24 sequences of 16001 tokens in all, 1504 bfloat16 channels, no such row: 89 us; with both arrays cleared whole ahead of the kernel 120.
template <typename T, bool PAIR>
__device__ __forceinline__ void clear_rows(const GatedParams &p, uint32_t c, bool c0, bool c1) {
    const int64_t first = GatedWalk::first(p, 0), tokens = int64_t(p.tokens), batch = gridDim.x / (p.strips * p.ranks);
    const int64_t last = max(GatedWalk::first(p, uint32_t(batch)), first), outside = first + tokens - last;
    const int64_t place = int64_t(blockIdx.x / (p.strips * p.ranks)) * p.ranks + blockIdx.x % p.ranks;
    for (int64_t k = place * kGatedWarps + (threadIdx.x >> 5); k < outside; k += batch * p.ranks * kGatedWarps) {
        const int64_t row = k < first ? k : k - first + last;
        store_two<T, PAIR>(static_cast<T *>(p.d_x.ptr) + row * p.d_x.token + c, 0.0f, 0.0f, c0, c1);
        store_two<T, PAIR>(static_cast<T *>(p.d_gate.ptr) + row * p.d_gate.token + c, 0.0f, 0.0f, c0, c1);
    }
}

// The pairs of a lane's two channels: (f, f', b, b').
__device__ __forceinline__ float4 pairs_of(float2 f, float2 b) { return make_float4(f.x, f.y, b.x, b.y); }
__device__ __forceinline__ float2 apply(const float4 &q, float2 h) { return fma2(make_float2(q.x, q.y), h, make_float2(q.z, q.w)); }
__device__ __forceinline__ float4 after(const float4 &q, const float4 &before) {
    return pairs_of(mul2(make_float2(q.x, q.y), make_float2(before.x, before.y)), apply(q, make_float2(before.z, before.w)));
}

// Where the pairs of a tile's warps, and of the tiles that the blocks of a cluster walk at the same time, meet.  There are two sets of
// each, used in turn: who writes one again has met everybody that read it at the barrier of the other.
struct GatedMeeting {
    float4 warps[2][kGatedWarps][32];
    float4 tiles[][2][32];                         // (ranks, 2, 32)
};

// From what comes into the tiles of all blocks (`carry`, replaced by what leaves them) what comes into this warp's tokens.  In walking order, which is the order of tokens or (BACK) its reverse.
template <bool BACK>
__device__ __forceinline__ float2 meet(GatedMeeting &m, uint32_t buf, const float4 &own, uint32_t rank, uint32_t ranks, float2 &carry) {
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, place = BACK ? kGatedWarps - 1 - warp : warp;
    m.warps[buf][place][lane] = own;
    __syncthreads();
    float2 mine;
    if (ranks == 1) {
        mine = carry;
#pragma unroll
        for (uint32_t k = 0; k < kGatedWarps; ++k) {
            const float4 q = m.warps[buf][k][lane];
            if (k < place) mine = apply(q, mine);
            carry = apply(q, carry);
        }
        return mine;
    }
    auto cluster = cooperative_groups::this_cluster();
    if (warp == 0) {                               // what the warps ahead add up to, and the whole tile, for all blocks
        float4 sum = make_float4(1.0f, 1.0f, 0.0f, 0.0f);
#pragma unroll
        for (uint32_t k = 0; k < kGatedWarps; ++k) {
            const float4 q = m.warps[buf][k][lane];
            m.warps[buf][k][lane] = sum;
            sum = after(q, sum);
        }
#pragma unroll 4
        for (uint32_t k = 0; k < ranks; ++k) cluster.map_shared_rank(&m, k)->tiles[rank][buf][lane] = sum;
        asm volatile("fence.acq_rel.cluster;" ::: "memory");      // (for what this warp has told, and the block has read: the others need none)
    }
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    float2 at_tile = carry;
#pragma unroll 4
    for (uint32_t k = 0; k < ranks; ++k) {
        if (k == rank) at_tile = carry;
        carry = apply(m.tiles[k][buf][lane], carry);
    }
    return apply(m.warps[buf][place][lane], at_tile);
}

template <int COPY>
constexpr uint32_t kForwardStages = COPY == 16 ? 3 : 2;                  // (longer rows: two blocks an SM have no room for three)
constexpr uint32_t kBackwardStages = 2;
template <typename T>
constexpr int kForwardSteps = sizeof(T) == 2 ? 16 : 8;                  // tokens of a warp
constexpr int kBackwardSteps = 8;
template <typename T, int COPY>
constexpr uint32_t forward_bytes(uint32_t ranks) {
    return kForwardStages<COPY> * 2 * kGatedWarps * sizeof(GatedRowsOf<T, kForwardSteps<T>, COPY>) + sizeof(float4) * 32 * (2 * kGatedWarps + (ranks > 1 ? 2 * ranks : 0));
}
template <typename T, int COPY>
constexpr uint32_t backward_bytes(uint32_t ranks) {
    return kBackwardStages * 3 * kGatedWarps * sizeof(GatedRowsOf<T, kBackwardSteps, COPY>) + sizeof(float4) * 32 * (4 * kGatedWarps + (ranks > 1 ? 2 * ranks : 0));
}

// Blocks of a cluster walk a sequence together, block r tile r of every `ranks` tiles.
// Shared memory holds two blocks an SM.  The third one of the bound, of aligned 32-bit elements, stands for its 80 registers: 8 x 2048 tokens of 2048 channels 71.6 us, with
// 126 registers 74.6.  Off 16 bytes 80 are too few (they spill): 2047 channels 107 us, with 127 registers 93.
template <typename T, int INPUT, int COPY, bool PAIR>
__global__ void __launch_bounds__(kGatedWarps * 32, sizeof(T) == 4 && COPY == 16 ? 3 : 2) tcu_gated_forward_kernel(const GatedParams p) {
    constexpr int STEPS = kForwardSteps<T>, TILE = STEPS * kGatedWarps;
    static_assert(TILE % kGatedMark == 0 && kGatedMark % STEPS == 0, "marks lie where a warp begins");
    extern __shared__ __align__(16) uint8_t shared[];
    using Stage = GatedRowsOf<T, STEPS, COPY>[kGatedWarps];
    using Source = GatedSource<T, STEPS, COPY>;
    Stage *xs = reinterpret_cast<Stage *>(shared), *gs = xs + kForwardStages<COPY>;
    GatedMeeting &meeting = *reinterpret_cast<GatedMeeting *>(gs + kForwardStages<COPY>);
    const int warp = threadIdx.x >> 5;
    const uint32_t lane = threadIdx.x & 31, rank = blockIdx.x % p.ranks;
    if (p.ranks > 1) cluster_begin();
    const GatedWalk w(p, blockIdx.x / p.ranks, reinterpret_cast<int *>(shared));
    const uint32_t c = w.c0 + 2 * lane;
    const int wide = int(min(p.channels - w.c0, uint32_t(kGatedChannels)));
    const bool c0 = c < p.channels, c1 = c + 1 < p.channels;
    const T *px = w.at<T>(p, p.x, w.c0), *pg = w.at<T>(p, p.gate, w.c0);
    float2 carry = make_float2(0.0f, 0.0f);
    const uint64_t st = uint64_t(w.seq) * p.channels + c;
    if (p.state_in) {
        if (c0) carry.x = p.state_in[st];
        if (c1) carry.y = p.state_in[st + 1];
    }
    const int stride = int(p.ranks) * TILE;
    int t = int(rank) * TILE + warp * STEPS;                       // first token of this warp
    Source from_x(px, t, p.x.token, stride), from_g(pg, t, p.gate.token, stride);
    auto fetch = [&](uint32_t stage, int at) {
        if (at < w.len) {
            from_x.load(xs[stage][warp], w.len - at, wide);
            from_g.load(gs[stage][warp], w.len - at, wide);
        }
        commit_copies();
    };
    constexpr uint32_t kStages = kForwardStages<COPY>;
    for (uint32_t k = 0; k + 1 < kStages; ++k) fetch(k, t + int(k) * stride);
    if (p.ranks > 1) cluster_begun();
    T *py = w.at<T>(p, p.y, c) + t * p.y.token;
    uint32_t buf = 0, stage = 0;
    for (int done = 0; done < w.len; done += stride, t += stride, buf ^= 1) {
        copies_but<int(kStages) - 2>();
        __syncwarp();                                              // the rows are here, and the ones before have been read
        fetch(stage == 0 ? kStages - 1 : stage - 1, t + (int(kStages) - 1) * stride);
        const int n = w.len - t;                                   // tokens of this warp, if it has so many
        const bool here = n > 0;
        float2 prod[STEPS], local[STEPS], a = both(1.0f), b = both(0.0f);
        if (here) {
            if (n < STEPS) {
                fill_rows(xs[stage][warp], n, 0.0f);
                fill_rows(gs[stage][warp], n, INFINITY);
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const float2 x = pair_of(xs[stage][warp], s, Source::behind(px + t * p.x.token, p.x.token, s));
                const float2 g = pair_of(gs[stage][warp], s, Source::behind(pg + t * p.gate.token, p.gate.token, s));
                float2 f, rest;
                sigmoids<sizeof(T) == 4>(g, f, rest);
                a = mul2(a, f);
                b = fma2(f, b, taken_in<INPUT>(f, rest, x));
                prod[s] = a;
                local[s] = b;
            }
        }
        const float2 mine = meet<false>(meeting, buf, pairs_of(a, b), rank, p.ranks, carry);
        if (here) {
            if (p.marks && warp * STEPS % kGatedMark == 0) {
                float *m = p.marks + (w.mark + uint32_t(t) / kGatedMark) * p.channels + c;
                if (c0) m[0] = mine.x;
                if (c1) m[1] = mine.y;
            }
            if (p.y.ptr) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) local[s] = fma2(prod[s], mine, local[s]);
                store_rows<T, PAIR, STEPS>(py, p.y.token, n, c0, c1, local);
            }
        }
        py += stride * p.y.token;
        stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    if (p.ranks > 1) cooperative_groups::this_cluster().sync();           // (nobody leaves, or writes the state, before all have read)
    if (p.state_out && warp == 0 && rank == 0) {
        if (c0) p.state_out[st] = carry.x;
        if (c1) p.state_out[st + 1] = carry.y;
    }
}

template <typename T, int INPUT, int COPY, bool PAIR>
__global__ void __launch_bounds__(kGatedWarps * 32, 2) tcu_gated_backward_kernel(const GatedParams p) {
    constexpr int STEPS = kBackwardSteps, TILE = STEPS * kGatedWarps;
    static_assert(TILE == kGatedMark, "a tile begins with a mark");
    extern __shared__ __align__(16) uint8_t shared[];
    using Stage = GatedRowsOf<T, STEPS, COPY>[kGatedWarps];
    using Source = GatedSource<T, STEPS, COPY>;
    Stage *xs = reinterpret_cast<Stage *>(shared), *gs = xs + kBackwardStages, *ds = gs + kBackwardStages;
    auto *ahead = reinterpret_cast<float4(*)[kGatedWarps][32]>(ds + kBackwardStages);
    GatedMeeting &meeting = *reinterpret_cast<GatedMeeting *>(ahead + 2);
    const int warp = threadIdx.x >> 5;
    const uint32_t lane = threadIdx.x & 31, rank = blockIdx.x % p.ranks;
    if (p.ranks > 1) cluster_begin();
    const GatedWalk w(p, blockIdx.x / p.ranks, reinterpret_cast<int *>(shared));
    const uint32_t c = w.c0 + 2 * lane;
    const int wide = int(min(p.channels - w.c0, uint32_t(kGatedChannels)));
    const bool c0 = c < p.channels, c1 = c + 1 < p.channels;
    const T *px = w.at<T>(p, p.x, w.c0), *pg = w.at<T>(p, p.gate, w.c0), *pd = w.at<T>(p, p.d_y, w.c0);
    float2 flow = make_float2(0.0f, 0.0f);                                 // C at the end of the blocks' tiles
    const uint64_t st = uint64_t(w.seq) * p.channels + c;
    if (p.d_state_out) {
        if (c0) flow.x = p.d_state_out[st];
        if (c1) flow.y = p.d_state_out[st + 1];
    }
    const int tiles = (w.len + TILE - 1) / TILE, stride = int(p.ranks) * TILE;
    int t = (tiles - 1 - int(rank)) * TILE + warp * STEPS;   // first token of this warp; below 0: there is none
    Source from_x(px, t, p.x.token, -stride), from_g(pg, t, p.gate.token, -stride), from_d(pd, t, p.d_y.token, -stride);
    float2 mark = both(0.0f);                                // the state that the tile begins with
    auto fetch = [&](uint32_t stage, int at) {
        if (at >= 0) {
            from_x.load(xs[stage][warp], w.len - at, wide);
            from_g.load(gs[stage][warp], w.len - at, wide);
            from_d.load(ds[stage][warp], w.len - at, wide);
            const float *m = p.marks + (w.mark + uint32_t(at) / kGatedMark) * p.channels + c;
            if (c0) mark.x = m[0];
            if (c1) mark.y = m[1];
        }
        commit_copies();
    };
    fetch(0, t);
    if (p.ranks > 1) cluster_begun();
    T *pdx = w.at<T>(p, p.d_x, c) + t * p.d_x.token, *pdg = w.at<T>(p, p.d_gate, c) + t * p.d_gate.token;
    uint32_t buf = 0;
    for (int done = 0; done < tiles; done += int(p.ranks), t -= stride, buf ^= 1) {
        copies_but<0>();
        __syncwarp();
        float2 h = mark;
        fetch(buf ^ 1, t - stride);
        const int n = w.len - t;                             // tokens of this warp, if it has so many
        const bool here = t >= 0;
        float2 f[STEPS], rest[STEPS], in[STEPS], a = both(1.0f), b = both(0.0f), r = both(0.0f);
        if (here) {
            if (n < STEPS) {
                fill_rows(xs[buf][warp], n, 0.0f);
                fill_rows(gs[buf][warp], n, INFINITY);
                fill_rows(ds[buf][warp], n, 0.0f);
            }
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                sigmoids<sizeof(T) == 4>(pair_of(gs[buf][warp], s, Source::behind(pg + t * p.gate.token, p.gate.token, s)), f[s], rest[s]);
                in[s] = taken_in<INPUT>(f[s], rest[s], pair_of(xs[buf][warp], s, Source::behind(px + t * p.x.token, p.x.token, s)));
                a = mul2(a, f[s]);
                b = fma2(f[s], b, in[s]);
                r = fma2(a, pair_of(ds[buf][warp], s, Source::behind(pd + t * p.d_y.token, p.d_y.token, s)), r);       // of d_t flows back to the first token: d_t times all f up to its own
            }
        }
        ahead[buf][warp][lane] = pairs_of(a, b);
        float2 out = meet<true>(meeting, buf, pairs_of(a, r), rank, p.ranks, flow);
        if (here) {
#pragma unroll
            for (int k = 0; k < kGatedWarps - 1; ++k)
                if (k < warp) h = apply(ahead[buf][k][lane], h);
            float2 before[STEPS];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                before[s] = h;
                h = fma2(f[s], h, in[s]);
            }
#pragma unroll
            for (int s = STEPS - 1; s >= 0; --s) {
                const float2 grad = add2(pair_of(ds[buf][warp], s, Source::behind(pd + t * p.d_y.token, p.d_y.token, s)), out);
                out = mul2(f[s], grad);
                before[s] = mul2(grad, gate_slope<INPUT>(f[s], rest[s], before[s], in[s]));
                rest[s] = taken_in<INPUT>(f[s], rest[s], grad);
            }
            store_rows<T, PAIR, STEPS>(pdx, p.d_x.token, n, c0, c1, rest);
            store_rows<T, PAIR, STEPS>(pdg, p.d_gate.token, n, c0, c1, before);
        }
        pdx -= stride * p.d_x.token;
        pdg -= stride * p.d_gate.token;
    }
    if (p.clear) clear_rows<T, PAIR>(p, c, c0, c1);             // (ahead of the walk: 8 x 4096 tokens of 1024 channels 99 us, here 97, with or without rows to clear)
    if (p.ranks > 1) cooperative_groups::this_cluster().sync();
    if (p.d_state_in && warp == 0 && rank == 0) {
        if (c0) p.d_state_in[st] = flow.x;
        if (c1) p.d_state_in[st + 1] = flow.y;
    }
}

// One token of each sequence.  Bound by memory: 8 bytes of state and three elements a channel.
template <typename T, int INPUT>
__global__ void __launch_bounds__(256) tcu_gated_step_kernel(const GatedParams p, const int32_t *slots, uint64_t pool, uint32_t batch) {
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    const uint64_t seq = i / p.channels;
    if (seq >= batch) return;
    const uint32_t c = uint32_t(i - seq * p.channels);
    const int64_t slot = slots ? int64_t(slots[seq]) : int64_t(seq);
    T *y = static_cast<T *>(p.y.ptr) + int64_t(seq) * p.y.batch + c;
    if (slot < 0 || uint64_t(slot) >= pool) {
        *y = from_f32<T>(0.0f);
        return;
    }
    float *state = p.state_out + uint64_t(slot) * p.channels + c;
    const float g = to_f32<T>(static_cast<const T *>(p.gate.ptr)[int64_t(seq) * p.gate.batch + c]), x = to_f32<T>(static_cast<const T *>(p.x.ptr)[int64_t(seq) * p.x.batch + c]);
    const float h = next_state<INPUT>(g, x, *state);
    *state = h;
    *y = from_f32<T>(h);
}

}  // namespace tcu
