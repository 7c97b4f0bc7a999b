// Linear attention with a constant decay for each head: device code.
//
// One form, a "mixing", serves the forward pass and all three gradients.  Walking a sequence forward in time (lead = 1) or
// backward (lead = 0), with a state X of dk x dv values and a = exp(log_decay),
//     lead = 1:  X <- a X + in_scale * k_t v_t^T,   o_t = out_scale * X^T q_t
//     lead = 0:  X <- X + in_scale * k_t v_t^T,     o_t = out_scale * X^T q_t,   X <- a X
//     o  = mix(q, k, v)       forward, from the state before the first token, leaving the one after the last
//     dq = mix(do, v, k)      forward, from the transposed state
//     dv = mix(k, q, do)      backward, from the gradient of the last state, leaving the gradient of the first
//     dk = mix(v, do, q)      backward, from its transpose
// so the backward pass is one launch of three mixings for every sequence and head.
//
// In groups of L <= 128 tokens, with i, j counted in walking order inside the group and X the state that enters it,
//     o_i = in_scale * out_scale * sum_{j <= i} a^(i-j) (q_i . k_j) v_j  +  out_scale * a^(i+lead) X^T q_i
//     X  <- a^L X + in_scale * sum_j a^(L-j-lead) k_j v_j^T
// that is, per group, four products on the tensor cores (the triangular product of a scan, with powers of a below the
// diagonal in place of ones, and the carry as a matrix):
//     S = Q K^T,  O = P V with P = S * decays (rounded to the 16-bit type, A operand in tensor memory),
//     E = Q X  (X rounded to the 16-bit type),  X^T += V^T K~  with K~ = decayed keys in two 16-bit terms.
//
// A block (one job, sequence, head and - in a cluster - part of the walk) runs the groups one after another.  Roles:
//     tokens    8 warps, thread = half a token: O + decayed E -> the tile that held Q, then the next scores -> P
//     keys      8 warps, thread = half a token: K -> the terms of K~, the first in the place of K
//     state     4 warps, thread = column of v: X out of tensor memory, rounded into the operand of E, times a^L and put back
//     producer  TMA: K, Q, V of each group into a ring of tiles
//     issuers   tcgen05.mma: one warp for scores and O, one for E and the state
//     store     TMA: the outputs (stores of a row a thread, 32 bytes at a time, took 2000 cycles a group, and the load-store unit
//               from all other roles)
// What bounds it is not the tensor core (2560 of its cycles a group with D = 128) but the chain from group to group,
//     X rescaled (and, meanwhile, K~ made) -> E and the products of X (512 cycles each, and 450 until they are known to be done),
// and the elementwise work, 16 lanes a cycle and scheduler for conversions, permutations and packed arithmetic alike.  Hence the
// roles, two issuers that do not wait for one another's turn, and as few instructions an element as possible.
//
// Rounded to 16 bits are only operands of a product: P, and X as operand of E (the state itself stays in 32 bits in tensor
// memory).  K~ enters the state in two terms: 22 bits of mantissa in float16, 16 in bfloat16.  There a third term follows
// (24 bits, all that 32-bit arithmetic gives) in the groups that the decay until the end of the walk leaves above 2^-6, because
// the last state is a result in 32 bits of its own; with two terms throughout it was 2e-6 to 5e-6 off, where 32-bit sums are
// 2e-7 off.  (The rule goes by the decay alone: outputs do not depend on whether the state is asked for.)  What is left is the
// tensor core's sum in 32 bits, which drops what falls below its last bit instead of rounding it: without decay, products of one
// sign are short by 2e-8 to 3e-8 of the sum for every 16 tokens and term (4e-5 after 8192 tokens, where rounded sums are 7e-6 off;
// of either sign 1e-6), and float16 values below 2^-14 of either sign count as 2^-14 in what is dropped.  In float16 X and K~
// are brought to the type's range by powers of two found for every group, because a state without decay outgrows the type
// and the low terms of small keys fall below it; and P by one found for every token, because scores do either (products of a
// hundred features; small gradients).
//
// When there are fewer (job, sequence, head) than SMs, the walk is split over the blocks of a cluster: each block first
// forms the state that its part leaves from zero (K and V only), the blocks exchange them through distributed shared
// memory, and each walks its part from the state that enters it.  When there are more, they are cut into equal shares for the SMs,
// and a block hands the state at the end of its share to the next one through memory.
//
// Measured at D = 128: 256 heads of 4096 tokens in bfloat16, 1.08 GB, 232 us at full clock (4.7 TB/s; 4.1 us a group with all SMs in
// use), 262 to 276 (4.0) in a benchmark that keeps the device busy; 148 heads of 2048 tokens 72 to 76 us, 50 % of the memory's
// time and 33 % of the tensor pipe's, in float16 89 us (its scores and keys are read a second time, for their powers of two).
// One group takes 9.2 us with the launch.
//
// Every wait is bounded; one that runs out records TCU_ERR_TIMEOUT in the workspace and the block winds down: each role returns at
// its next wait that fails, the producer after its copies have landed, the issuers after their products have ended (drain), and a
// block whose first phase was given up leaves the second out.  tcu_linattn_selftest_timeout takes these ways.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "tcu_embedding_kernel.cuh"
#include "tcu_ptx.cuh"

namespace tcu {

constexpr int kGroup = 128;              // tokens of a group: M of the products
constexpr int kHalfBytes = 16384;        // 128 tokens x 64 features: one 128-byte-swizzled block of rows
constexpr int kMixCtlBytes = 2048;

struct MixTokens {
    const void *ptr;
    int64_t batch, token, head;          // strides in elements
};

struct MixJob {
    uint8_t map[4];                      // tensor maps of q, k, v, o
    uint8_t by_batch[3], by_head[3];     // 0 where the array repeats along that axis
    void *o;
    int64_t o_batch, o_token, o_head;    // strides in elements
    const float *init;                   // state that enters the walk, or NULL; (sequence, head) entries of dk * dv values
    float *last;                         // NULL, or receives the state that leaves it
    uint32_t init_k, init_v;             // strides of init along dk and dv (last: dv, 1)
    uint32_t dk, dv;
    uint32_t lead;                       // 1: forward in time, 0: backward
    float in_scale, out_scale;
};

struct alignas(64) MixParams {
    CUtensorMap map[7];
    MixJob job[3];
    const float *log_decay;
    const int64_t *offsets;
    uint32_t *error;                     // status word
    uint64_t tokens;
    uint32_t batch, heads, jobs, ranks;  // ranks: blocks of a cluster
    // walks cut where a block's share of all the groups ends: by block, a flag and the state that it hands to the next one
    uint32_t *flags;
    float *handed;
    const uint32_t *order;               // packed, long sequences first: which one comes where
    uint32_t rounds;                     // tries of 100 us after which a wait is given up
    uint32_t silent;                     // self-test: 0, or 1 + the group of every walk whose part of the state is never announced
};
constexpr uint32_t kMostOrdered = 512;   // sequences that are put in order

// Which groups of a walk a block takes, and how many tokens.
struct MixPart {
    uint32_t len, groups, per, first, last;   // tokens and groups of the sequence, groups per block, this block's [first, last) in walking order
    bool lead;
    __device__ __forceinline__ uint32_t in_time(uint32_t p) const { return lead ? p : groups - 1 - p; }
    __device__ __forceinline__ int tokens_of(uint32_t p) const { return int(min(len - in_time(p) * kGroup, uint32_t(kGroup))); }
    // tokens that the sequence's walk takes after group p
    __device__ __forceinline__ float tokens_after(uint32_t p) const { return float(lead ? len - min((p + 1) * kGroup, len) : in_time(p) * kGroup); }
    __device__ __forceinline__ float tokens_of_rank(uint32_t r) const {
        const uint32_t a = min(r * per, groups), b = min((r + 1) * per, groups);
        const uint32_t lo = (lead ? a : groups - b) * kGroup, hi = (lead ? b : groups - a) * kGroup;
        return float(min(hi, len) - min(lo, len));
    }
};

constexpr int kMixMostSlots = 8;
constexpr int kNear = 160 + 1 + 47;
struct MixCtl {
    uint64_t full[kMixMostSlots], empty[kMixMostSlots];      // (a tile is free when two have done with it: both issuers, or for Q one and the store)
    uint64_t qk_done;                    // S is in tensor memory
    uint64_t p_ready;                    // P is
    uint64_t pv_done;                    // O is (and S is free)
    uint64_t e_done;                     // E is
    uint64_t o_free;                     // O and E have been read
    uint64_t o_staged;                   // the outputs are in shared memory
    uint64_t x_ready;                    // X rounded into its operand, and multiplied by a^L in tensor memory
    uint64_t k_scaled;                   // float16: the power of two for K~ is known
    uint64_t k_ready;                    // two terms of K~ written (and rows past the end of V cleared)
    uint64_t first_done, third_ready;    // the first has been multiplied, and the third written in its place
    uint64_t kv_done;                    // the group is in X
    uint64_t drained[2];
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    uint32_t rounds, silent;             // as in MixParams
    MixJob job;                          // what the block works on
    MixPart part;
    uint32_t t0, b, h, count, before;    // first token of the sequence; sequence (0 when packed) and head; groups of the walk, of the first phase
    uint32_t thirds;                     // third terms of K~ in the first phase
    const uint32_t *wait_flag;           // NULL, or set once the state that enters has been handed over
    uint64_t patience;                   // nanoseconds to wait for that
    uint64_t places_from, places_to;     // what is left of the block's share
    bool none, more;                     // no walk was left; the block goes on with another
    bool hands;                          // the state is for the next block
    bool clipped;                        // dense: a store of a whole group ends where the sequence does
    bool split, entered, owns_last;      // the walk starts from a state (else from zero); its last state is wanted
    float log2_decay;
    float biggest_k[2][8], biggest_x[2][4];      // float16: largest values seen by each warp
    int scale_k[2];                      // float16: K~ is used as 2^scale_k K~
    float unscale[2];                    // float16: the factor that takes E back to the size of X
    float power[kGroup + 4];             // a^m
    alignas(16) float block[16];         // factors of P along a block of 16 tokens
    float rank_decay[8];                 // a^(tokens of a part)
    // factors of P by distance, in the order of the columns: the distance falls along a row forward in time (from 160 to -47; below
    // zero, on the wrong side of the diagonal, 0) and grows backward
    float near[kNear];
};
static_assert(sizeof(MixCtl) <= kMixCtlBytes, "control block too large");

constexpr int kTokenWarps = 8, kKeyWarps = 8, kStateWarp = kTokenWarps + kKeyWarps, kProducerWarp = kStateWarp + 4, kScoreWarp = kProducerWarp + 1,
              kProductWarp = kScoreWarp + 1, kStoreWarp = kProductWarp + 1;
constexpr int kMixThreads = 32 * (kStoreWarp + 1);
template <int D> constexpr int kMixSlots = D == 64 ? 8 : 5;                  // tiles in the ring
template <int D> constexpr int kMixTileBytes = D / 64 * kHalfBytes;
template <int D> constexpr int kMixSmemBytes = 1024 + kMixCtlBytes + (kMixSlots<D> + 1) * kMixTileBytes<D> + D * D * 2;
static_assert(kMixSmemBytes<128> <= 232448 && kMixSmemBytes<64> <= 232448, "shared memory of a block");
static_assert(kMixSlots<64> <= kMixMostSlots, "ring");

template <typename T> struct Half2Of;
template <> struct Half2Of<__nv_bfloat16> {
    static constexpr uint32_t kType = 2;             // as in make_idesc
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&p);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    using Pair = __nv_bfloat162;
};
template <> struct Half2Of<__half> {
    static constexpr uint32_t kType = 1;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 p = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&p);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
    using Pair = __half2;
};

// two products, sums at once
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z, u;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 u, x, y, z;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

// Packed arithmetic on two 16-bit values; rounded once, to nearest.
template <typename T>
struct Half2 : Half2Of<T> {
    using P = typename Half2Of<T>::Pair;
    static __device__ __forceinline__ P as(uint32_t w) { return *reinterpret_cast<const P *>(&w); }
    static __device__ __forceinline__ uint32_t bits(P p) { return *reinterpret_cast<const uint32_t *>(&p); }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b) { return bits(__hmul2_rn(as(a), as(b))); }
    static __device__ __forceinline__ uint32_t fma(uint32_t a, uint32_t b, uint32_t c) { return bits(__hfma2(as(a), as(b), as(c))); }
    static __device__ __forceinline__ uint32_t fms(uint32_t a, uint32_t b, uint32_t c) { return bits(__hfma2(as(a), as(b), __hneg2(as(c)))); }
};

__device__ __forceinline__ uint64_t global_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t) : : "memory");
    return t;
}

// Waits for the phase of a barrier; false when the wait was given up, after about a second.
constexpr uint32_t kMixWaitRounds = 10000;
__device__ __forceinline__ bool mix_wait(MixCtl *ctl, const uint64_t &barrier, uint32_t parity) {
    const bool ok = mbar_wait_bounded_at(smem_u32(&barrier), parity, smem_u32(&ctl->rounds));
    if (!ok) ctl->abort_flag = 1;
    return ok;
}
// the same for a whole warp, with one answer for all lanes
__device__ __forceinline__ bool mix_wait_warp(MixCtl *ctl, const uint64_t &barrier, uint32_t parity) {
    return __all_sync(0xffffffffu, mix_wait(ctl, barrier, parity));
}

// The same for all warps of a role that also meet at a named barrier: they get the same answer, so that they give up together.
__device__ __forceinline__ bool mix_wait_role(MixCtl *ctl, int id, int threads, const uint64_t &barrier, uint32_t parity) {
    return !named_barrier_or(id, threads, !mix_wait_warp(ctl, barrier, parity));
}

// A block, as its roles see it.  Each role is a function of its own, called for each of the two phases (a walk that is not split has
// only the second): six programs share the SM's instruction cache, and when the compiler merged and copied them the kernel was four
// times this size and spent most of its time fetching instructions.
extern __shared__ uint8_t mix_smem[];
// (an offset from the array, and found again by each role, so that the compiler knows the address space)
__device__ __forceinline__ MixCtl *mix_ctl() { return reinterpret_cast<MixCtl *>(mix_smem + (-smem_u32(mix_smem) & 1023)); }

template <int D, typename T>
struct Mix {
    using H = Half2<T>;
    static constexpr bool kIsHalf = std::is_same<T, __half>::value;
    static constexpr float kThirdFrom = -6.0f;                           // bfloat16: log2 of the decay to the end from which on K~ has a third term
    static __device__ __forceinline__ bool has_third(const MixCtl *ctl, const MixPart &part, uint32_t p) {
        return !kIsHalf && ctl->log2_decay * part.tokens_after(p) > kThirdFrom;
    }
    static constexpr uint32_t kTile = kMixTileBytes<D>, kSlots = kMixSlots<D>;
    static constexpr uint32_t kAhead = 2;                                // groups ahead of their load that tiles are brought into L2
    static constexpr int kXHalf = D * 128;                               // one 64-wide half of the operand X: D rows of 128 bytes
    static constexpr int kCols = D / 2;                                  // features of a token that a thread of the token and key roles has
    // tensor memory: S, O, E, X.  P takes the place of S: two warps share the 128 columns of a token, and each 64 columns of S
    // leave their P in their own first 32 columns.
    static constexpr uint32_t kColS = 0, kColO = 128, kColE = 256, kColX = 384, kColumns = 512;

    // shared memory: control block, ring of tiles (between the phases: D x D state totals), second term of K~, operand X
    static __device__ __forceinline__ uint32_t ring_at(const MixCtl *ctl) { return smem_u32(ctl) + kMixCtlBytes; }
    static __device__ __forceinline__ uint32_t low_at(const MixCtl *ctl) { return ring_at(ctl) + kSlots * kTile; }
    static __device__ __forceinline__ uint32_t x_at(const MixCtl *ctl) { return low_at(ctl) + kTile; }
    static __device__ __forceinline__ uint32_t slot_at(const MixCtl *ctl, uint32_t tile) { return ring_at(ctl) + tile % kSlots * kTile; }
    static __device__ __forceinline__ bool wait_full(MixCtl *ctl, uint32_t tile) { return mix_wait_warp(ctl, ctl->full[tile % kSlots], (tile / kSlots) & 1); }
    // Rows of a tile: token i of the group at i * 128 bytes, 16-byte pieces exchanged by the swizzle (piece ^ (i & 7)).
    // The 16 bytes of feature f = 64 h + 8 c are at h * kHalfBytes + (row_at(row) ^ c << 4).
    static __device__ __forceinline__ uint32_t row_at(int row) { return uint32_t(row * 128 + ((row & 7) << 4)); }
    static __device__ __forceinline__ float pow2(int n) { return __uint_as_float(uint32_t(min(max(n, -126), 127) + 127) << 23); }
    static __device__ __forceinline__ int exponent(float x) { return int((__float_as_uint(x) >> 23) & 0xFF) - 127; }

    // ---- tokens: the outputs of group i - 1, then P of group i
    static __device__ __noinline__ void tokens() {
        MixCtl *ctl = mix_ctl();
        const int warp = threadIdx.x >> 5, row0 = (warp & 3) * 32, row = row0 + (threadIdx.x & 31);
        const int side = warp >> 2;                                                // which half of the row
        const uint32_t lanes = ctl->tmem_base + (uint32_t(warp & 3) << 21);        // this warp's 32 lanes (bits 16 and up)
        const MixPart part = ctl->part;
        const uint32_t n = ctl->count;
        float2 factor[8];                                                          // of P along a block of 16 tokens
#pragma unroll
        for (int j = 0; j < 8; ++j) factor[j] = reinterpret_cast<const float2 *>(ctl->block)[j];
        // this thread's half of the row, in a tile
        const uint32_t half_at = (D == 128 ? side * kHalfBytes : 0), at_row = row_at(row) ^ (D == 128 ? 0 : side * 64);
        uint32_t tile = 2 * ctl->before + 1 - 3;                                   // of Q, of group i - 1
        float back = 1.0f;                                                         // float16: the factor that takes O back to its size
        bool ok = true;                                                            // no wait has run out (float16: two warps meet in every group, and
                                                                                   // give up there, together)
        if (n == 0) return;
#pragma unroll 1
        for (uint32_t i = 0; i <= n; ++i, tile += 3) {
            if (i > 0) {
                const uint32_t g = i - 1;
                ok = mix_wait_warp(ctl, ctl->pv_done, g & 1) && mix_wait_warp(ctl, ctl->e_done, g & 1);
                if (!ok && (!kIsHalf || i == n)) return;
            }
            if (i > 0 && ok) {
                const uint32_t g = i - 1;
                const int tokens = part.tokens_of(part.first + g), order = part.lead ? row : tokens - 1 - row;
                tc_fence_after();
                float e = ctl->job.out_scale * ctl->power[max(order, 0) + int(part.lead)];
                if (kIsHalf) e *= ctl->unscale[(ctl->before + g) & 1];
                if (g == 0 && !ctl->entered) zero_e(lanes + side * kCols);          // no state: E was not formed
                if (tokens == kGroup || ctl->clipped) {
                    const uint32_t at = slot_at(ctl, tile) + half_at;
#pragma unroll
                    for (int c = 0; c < kCols; c += 16) {
                        uint32_t out[8];
                        outputs(lanes + side * kCols + c, e, back, out);
                        st_shared_v4(at + (at_row ^ (2 * c)), out[0], out[1], out[2], out[3]);
                        st_shared_v4(at + (at_row ^ (2 * c + 16)), out[4], out[5], out[6], out[7]);
                    }
                    fence_proxy_async_smem();
                } else {
                    T *to = reinterpret_cast<T *>(ctl->job.o) + ctl->b * ctl->job.o_batch + int64_t(ctl->h) * ctl->job.o_head +
                            (ctl->t0 + part.in_time(part.first + g) * kGroup + row) * ctl->job.o_token + side * kCols;
                    write_some(to, lanes + side * kCols, e, back, row < tokens ? int(ctl->job.dv) - side * kCols : 0);
                }
                tc_fence_before();
                mbar_arrive(smem_u32(&ctl->o_free));
                mbar_arrive(smem_u32(&ctl->o_staged));
            }
            if (i < n) {
                const int tokens = part.tokens_of(part.first + i);
                ok = ok && mix_wait_warp(ctl, ctl->qk_done, i & 1);
                if (!kIsHalf && !ok) return;
                tc_fence_after();
                const uint32_t at = lanes + kColS + 64 * side;
                float up = 1.0f;
                if (kIsHalf) {
                    // float16: a token's scores are used as 2^s P with the largest near 2^14 (as they are, they can leave the type on
                    // either side).  Each half of the row leaves its largest where O will be: that was read above.
                    float big = 0.0f, other = 0.0f;
                    if (ok) {
#pragma unroll 1
                        for (int c = 64 * side, k = 0; k < 64; c += 16, k += 16) {
                            float2 x[8];
                            decayed(part.lead, row, row0, c, tokens, at + k, factor, x);
#pragma unroll
                            for (int j = 0; j < 8; ++j) big = fmaxf(big, fmaxf(fabsf(x[j].x), fabsf(x[j].y)));
                        }
                        tmem_st1(lanes + kColO + side * kCols, __float_as_uint(big));
                        tmem_st_wait();
                        tc_fence_before();
                    }
                    if (named_barrier_or(4 + (warp & 3), 64, !ok)) return;
                    tc_fence_after();
                    other = __uint_as_float(tmem_ld1(lanes + kColO + (side ^ 1) * kCols));
                    tmem_ld_wait();
                    big = fmaxf(big, other);
                    const int shift = big > 0.0f ? min(max(14 - exponent(big), -126), 126) : 0;
                    up = pow2(shift);
                    back = pow2(-shift);
                }
#pragma unroll 1
                for (int c = 64 * side, k = 0; k < 64; c += 16, k += 16) {
                    float2 x[8];
                    uint32_t out[8];
                    decayed(part.lead, row, row0, c, tokens, at + k, factor, x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (kIsHalf) x[j] = mul2(x[j], make_float2(up, up));
                        out[j] = H::pack(x[j].x, x[j].y);
                    }
                    tmem_st8(at + k / 2, out);                       // never over scores still to be read
                }
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(smem_u32(&ctl->p_ready));
            }
        }
    }
    // P, not yet rounded, of a token (`row`; the first of the warp: row0) and the 16 tokens of columns c...: all of them count, none,
    // or (around the diagonal and the end) some
    static __device__ __forceinline__ void decayed(bool lead, int row, int row0, int c, int tokens, uint32_t at, const float2 (&factor)[8], float2 (&x)[8]) {
        const MixCtl *ctl = mix_ctl();
        const int apart = lead ? row - c : c - row, apart0 = lead ? row0 - c : c - row0 - 31;     // tokens apart: of the first column; least of the warp
        const bool all = lead ? apart0 >= 15 : apart0 >= 0 && c + 15 < tokens;
        const bool none = lead ? apart0 < -31 : apart0 < -46 || c >= tokens;
        uint32_t v[16];
        if (all) {
            tmem_ld16(at, v);
            const float f = ctl->power[lead ? apart - 15 : apart];
            const float2 f2 = make_float2(f, f);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = mul2(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), mul2(f2, factor[j]));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = make_float2(0.0f, 0.0f);
            if (!none) {
                // what does not count may not be finite: it is left out, not multiplied by its factor of zero
                tmem_ld16(at, v);
                const int hi = tokens - c;                           // (past the end of a short group the factors are not zero)
                const float *near = ctl->near + (lead ? 160 - apart : 47 + apart);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float f = near[j];
                    v[j] = f != 0.0f ? __float_as_uint(__uint_as_float(v[j]) * f) : 0u;
                }
                if (!lead && hi < 16) {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (j >= hi) v[j] = 0u;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
            }
        }
    }
    // 16 features of a token: O (times `back` in float16) + e E
    static __device__ __forceinline__ void outputs(uint32_t at, float e, float back, uint32_t (&out)[8]) {
        uint32_t vo[16], ve[16];
        const float2 e2 = make_float2(e, e);
        tmem_ld16(at + kColO, vo);
        tmem_ld16(at + kColE, ve);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float2 o = make_float2(__uint_as_float(vo[2 * j]), __uint_as_float(vo[2 * j + 1]));
            if (kIsHalf) o = mul2(o, make_float2(back, back));
            const float2 x = fma2(e2, make_float2(__uint_as_float(ve[2 * j]), __uint_as_float(ve[2 * j + 1])), o);
            out[j] = H::pack(x.x, x.y);
        }
    }
    static __device__ __noinline__ void zero_e(uint32_t at) {
        const uint32_t zero[16] = {};
#pragma unroll 1
        for (int c = 0; c < kCols; c += 16) tmem_st16(at + kColE + c, zero);
        tmem_st_wait();
    }
    // the first `width` features (none when it is not positive) of this thread's half of a token
    static __device__ __noinline__ void write_some(T *to, uint32_t at, float e, float back, int width) {
#pragma unroll 1
        for (int c = 0; c < kCols; c += 16, width -= 16) {
            uint32_t out[8];
            outputs(at + c, e, back, out);
            if (width >= 8) st_global_v4(to + c, out[0], out[1], out[2], out[3]);
            if (width >= 16) st_global_v4(to + c + 8, out[4], out[5], out[6], out[7]);
            else if (width > 0) {
#pragma unroll
                for (int k = 0; k < 7; ++k) {
                    const uint32_t word = width < 8 ? out[k / 2] : out[4 + k / 2];
                    if (k < (width & 7)) reinterpret_cast<uint16_t *>(to)[c + (width & 8) + k] = uint16_t(word >> (16 * (k & 1)));
                }
            }
        }
    }

    // ---- keys.  float16: powers of two, found for every group, keep the operands inside the type: X is held as 2^s X, so that the
    // keys can be used as 2^s K~ with the largest near 2^14 (the low terms of small ones would fall below 2^-24).  What the decay takes
    // from the keys it has taken from X as well; the rest of s is at most 52: keys (with in_scale) down to 2^-55 keep both terms, and
    // states up to 2^75 stay inside 32 bits.  A group whose keys are all zero says nothing about s.
    static constexpr int kMostKeyScale = 52;
    static __device__ __noinline__ void keys(uint32_t phase) {
        MixCtl *ctl = mix_ctl();
        const int warp = (threadIdx.x >> 5) - kTokenWarps, lane = threadIdx.x & 31, row = (warp & 3) * 32 + lane;
        // this thread's half of the row, in a tile: pieces first ... first + kCols / 8 - 1 of a 64-wide half
        const uint32_t half_at = (D == 128 ? (warp >> 2) * kHalfBytes : 0), at_row = row_at(row) ^ (D == 128 ? 0 : (warp >> 2) * 64);
        const MixPart part = ctl->part;
        const uint32_t n = phase ? ctl->count : ctl->before;
        const uint32_t made = phase && n > 0 && !ctl->owns_last ? n - 1 : n;       // the last group's are not needed if its state is not
        uint32_t it = phase ? ctl->before : 0, tile = 2 * it;                      // groups before, their tiles
        uint32_t thirds = phase ? ctl->thirds : 0;
        int scale = 0;                                                             // float16: K~ is used as 2^scale K~
        auto gate = [&](const uint64_t &barrier, uint32_t parity) {
            return kIsHalf ? mix_wait_role(ctl, 2, 32 * kKeyWarps, barrier, parity) : mix_wait_warp(ctl, barrier, parity);
        };
        auto gate_full = [&](uint32_t tile) { return gate(ctl->full[tile % kSlots], (tile / kSlots) & 1); };
        // what follows the sequence may hold anything: zero times it has to be zero
        auto clear = [&](uint32_t slot) {
#pragma unroll 1
            for (uint32_t c = 0; c < kCols * 2; c += 16) st_shared_v4(slot + half_at + (at_row ^ c), 0, 0, 0, 0);
        };
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i, ++it, tile += phase + 2) {
            const uint32_t k_at = slot_at(ctl, tile) + half_at, low = low_at(ctl) + half_at;
            const int tokens = part.tokens_of(part.first + i);
            // walking order: token `row` of the group is j = row forward, tokens - 1 - row backward; a^(tokens - j - lead)
            float f = ctl->job.in_scale * ctl->power[part.lead ? max(tokens - 1 - row, 0) : row + 1];
            if (it > 0 && !gate(ctl->kv_done, (it - 1) & 1)) return;         // the buffer of the second term is free
            if (kIsHalf) {
                if (!gate_full(tile)) return;
                float big = 0.0f;
                if (row < tokens) {
#pragma unroll 1
                    for (uint32_t c = 0; c < kCols * 2; c += 16) {
                        uint32_t k4[4];
                        ld_shared_v4(k_at + (at_row ^ c), k4[0], k4[1], k4[2], k4[3]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 x = H::unpack(k4[e]);
                            big = fmaxf(big, fmaxf(fabsf(x.x), fabsf(x.y)));
                        }
                    }
                }
                __syncwarp();
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
                if (lane == 0) ctl->biggest_k[it & 1][warp] = big;
                named_barrier_sync(2, 32 * kKeyWarps);
#pragma unroll
                for (int j = 0; j < kKeyWarps; ++j) big = fmaxf(big, ctl->biggest_k[it & 1][j]);
                // the powers of a in K~ go from a^(1 - lead) to a^(tokens - lead)
                const float top = fmaxf(ctl->power[1 - int(part.lead)], ctl->power[tokens - int(part.lead)]);
                big *= fabsf(ctl->job.in_scale);
                if (big > 0.0f && top > 0.0f) scale = min(max(min(max(13 - exponent(big), -30), kMostKeyScale) - exponent(top), -126), 126);
                f *= pow2(scale);
                if (warp == 0 && lane == 0) {
                    ctl->scale_k[it & 1] = scale;
                    mbar_arrive(smem_u32(&ctl->k_scaled));
                }
            }
            if (phase && !gate(ctl->qk_done, i & 1)) return;                 // K itself has been multiplied
            if (!phase && !gate_full(tile)) return;
            if (tokens < kGroup) {
                if (!gate_full(tile + phase + 1)) return;
                if (row >= tokens) {
                    clear(slot_at(ctl, tile + phase + 1));
                    clear(slot_at(ctl, tile));
                }
            }
            const bool third = has_third(ctl, part, part.first + i);
            if (i >= made) {                                                 // (not made)
            } else if (kIsHalf) {
#pragma unroll 2
                for (uint32_t c = 0; c < kCols * 2; c += 16) split<false>(k_at + (at_row ^ c), low + (at_row ^ c), f, nullptr);
            } else if (third) {
                uint32_t rest[kCols / 2];
#pragma unroll
                for (uint32_t c = 0; c < kCols * 2; c += 16) split<true>(k_at + (at_row ^ c), low + (at_row ^ c), f, rest + c / 4);
                fence_proxy_async_smem();
                mbar_arrive(smem_u32(&ctl->k_ready));
                if (!gate(ctl->first_done, thirds & 1)) return;
                ++thirds;
#pragma unroll
                for (uint32_t c = 0; c < kCols * 2; c += 16) st_shared_v4(k_at + (at_row ^ c), rest[c / 4], rest[c / 4 + 1], rest[c / 4 + 2], rest[c / 4 + 3]);
                fence_proxy_async_smem();
                mbar_arrive(smem_u32(&ctl->third_ready));
                continue;
            } else {
                // packed arithmetic: with f = f1 + f2 in two terms, hi = k f1 rounded, its error k f1 - hi exactly (a product of two
                // 8-bit mantissas has 16 bits), and lo = k f2 + that, rounded
                const uint32_t f1 = H::pack(f, f), f2 = H::pack(f - H::unpack(f1).x, f - H::unpack(f1).x);
#pragma unroll 4
                for (uint32_t c = 0; c < kCols * 2; c += 16) {
                    uint32_t k4[4], hi[4], lo[4];
                    ld_shared_v4(k_at + (at_row ^ c), k4[0], k4[1], k4[2], k4[3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hi[e] = H::mul(k4[e], f1);
                        lo[e] = H::fma(k4[e], f2, H::fms(k4[e], f1, hi[e]));
                    }
                    st_shared_v4(k_at + (at_row ^ c), hi[0], hi[1], hi[2], hi[3]);
                    st_shared_v4(low + (at_row ^ c), lo[0], lo[1], lo[2], lo[3]);
                }
            }
            fence_proxy_async_smem();
            mbar_arrive(smem_u32(&ctl->k_ready));
        }
    }
    // eight keys times f, in 32 bits, as two terms or three
    template <bool THIRD>
    static __device__ __forceinline__ void split(uint32_t first, uint32_t second, float f, uint32_t *third) {
        uint32_t k4[4], hi[4], lo[4];
        const float2 f2 = make_float2(f, f), minus = make_float2(-1.0f, -1.0f);
        ld_shared_v4(first, k4[0], k4[1], k4[2], k4[3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 x = mul2(H::unpack(k4[e]), f2);
            hi[e] = H::pack(x.x, x.y);
            const float2 y = fma2(H::unpack(hi[e]), minus, x);
            lo[e] = H::pack(y.x, y.y);
            if (THIRD) {
                const float2 z = fma2(H::unpack(lo[e]), minus, y);
                third[e] = H::pack(z.x, z.y);
            }
        }
        st_shared_v4(first, hi[0], hi[1], hi[2], hi[3]);
        st_shared_v4(second, lo[0], lo[1], lo[2], lo[3]);
    }

    // ---- state: thread = column of v (the first D lanes)
    static __device__ __noinline__ void state(uint32_t phase) {
        MixCtl *ctl = mix_ctl();
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = (warp & 3) * 32 + lane;
        const bool holds_x = (warp & 3) * 32 < D;                            // whole warps
        const uint32_t x_lanes = ctl->tmem_base + (uint32_t(warp & 3) << 21) + kColX;
        const MixPart part = ctl->part;
        const uint32_t n = phase ? ctl->count : ctl->before, base = phase ? ctl->before : 0;
        const bool entered = phase && ctl->entered;
        const uint32_t dk = uint32_t(row) < ctl->job.dv ? ctl->job.dk : 0;   // rows of this thread's column in the states of the caller
        float *exchange = reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(ctl) + kMixCtlBytes) + row;
        int held = 0;                                                        // float16: X is held as 2^held X
        auto gate = [&](const uint64_t &barrier, uint32_t parity) {
            return kIsHalf ? mix_wait_role(ctl, 3, 128, barrier, parity) : mix_wait_warp(ctl, barrier, parity);
        };
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t it = base + i;
            const bool fresh = i == 0 && !entered;                           // X is zero: the first product does not add to it
            float shrink = 1.0f, keep = ctl->power[part.tokens_of(part.first + i)];
            if (i > 0) {
                if (!gate(ctl->kv_done, (it - 1) & 1)) return;
                tc_fence_after();
            }
            if (kIsHalf) {
                if (!gate(ctl->k_scaled, it & 1)) return;
                float big = 0.0f;
                if (!fresh && holds_x) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        uint32_t v[16];
                        tmem_ld16(x_lanes + c, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) big = fmaxf(big, fabsf(__uint_as_float(v[j])));
                    }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
                if (lane == 0) ctl->biggest_x[it & 1][warp & 3] = big;
                named_barrier_sync(3, 128);
#pragma unroll
                for (int j = 0; j < 4; ++j) big = fmaxf(big, ctl->biggest_x[it & 1][j]);
                const int ex = min(max(exponent(big), -60), 127), now = ctl->scale_k[it & 1];
                shrink = pow2(14 - ex);
                if (threadIdx.x == 32 * kStateWarp) ctl->unscale[it & 1] = pow2(ex - 14 - held);
                keep *= pow2((now - held) / 2);              // (as two factors: the powers may be 252 apart)
                keep *= pow2(now - held - (now - held) / 2);
                held = now;
            }
            if (!fresh && holds_x) {
                const float2 keep2 = make_float2(keep, keep), shrink2 = make_float2(shrink, shrink);
                const uint32_t x_row = x_at(ctl) + row * 128, swizzle = uint32_t(row & 7) << 4;
                auto step = [&](uint32_t (&v)[16], uint32_t c) {
                    if (phase) {
                        const uint32_t at = x_row + (c >> 6) * kXHalf;
#pragma unroll
                        for (uint32_t j = 0; j < 16; j += 8) {
                            uint32_t w4[4];
#pragma unroll
                            for (uint32_t e = 0; e < 4; ++e) {
                                float2 x = make_float2(__uint_as_float(v[j + 2 * e]), __uint_as_float(v[j + 2 * e + 1]));
                                if (kIsHalf) x = mul2(x, shrink2);
                                w4[e] = H::pack(x.x, x.y);
                            }
                            st_shared_v4(at + (((c * 2 + j * 2) & 127) ^ swizzle), w4[0], w4[1], w4[2], w4[3]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 16; j += 2) {
                        const float2 x = mul2(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), keep2);
                        v[j] = __float_as_uint(x.x);
                        v[j + 1] = __float_as_uint(x.y);
                    }
                    tmem_st16(x_lanes + c, v);
                };
                uint32_t v0[16], v1[16];                                     // the next columns are on their way while these are worked on
                tmem_ld16(x_lanes, v0);
#pragma unroll 1
                for (uint32_t c = 0; c < D; c += 32) {
                    tmem_ld_wait();
                    tmem_ld16(x_lanes + c + 16, v1);
                    step(v0, c);
                    tmem_ld_wait();
                    if (c + 32 < D) tmem_ld16(x_lanes + c + 32, v0);
                    step(v1, c + 16);
                }
                tmem_st_wait();
                if (phase) fence_proxy_async_smem();
            }
            tc_fence_before();
            mbar_arrive(smem_u32(&ctl->x_ready));
        }
        // the state that leaves: to the other blocks, or to the caller
        if (phase ? !ctl->owns_last : n == 0) return;
        if (n > 0 && !gate(ctl->kv_done, (base + n - 1) & 1)) return;
        tc_fence_after();
        if (!holds_x) return;
        float *to = phase ? ctl->job.last + row : exchange;
        const uint32_t pitch = phase ? ctl->job.dv : D, rows = phase ? dk : D;
        const float back = kIsHalf ? pow2(-held) : 1.0f;
#pragma unroll 1
        for (uint32_t c = 0; c < D; c += 16) {
            uint32_t v[16];
            tmem_ld16(x_lanes + c, v);
            tmem_ld_wait();
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j)
                if (c + j < rows) to[uint64_t(c + j) * pitch] = __uint_as_float(v[j]) * back;
        }
    }
    // ---- what a block works on.  One thread writes it down.
    static __device__ __forceinline__ void take(const MixParams &p, const MixPart &part, uint32_t job_index, uint32_t b, uint32_t h, int64_t begin, uint32_t rank, bool cut) {
        MixCtl *ctl = mix_ctl();
        const MixJob &job = p.job[job_index];
        const uint32_t count = part.last - part.first;
        const bool handed = cut && part.first > 0, hands = cut && part.last < part.groups;
        const uint64_t size = uint64_t(job.dk) * job.dv, state_at = (uint64_t(b) * p.heads + h) * size;
        ctl->job = job;
        if (job.init) ctl->job.init = job.init + state_at;
        if (job.last) ctl->job.last = job.last + state_at;
        if (handed) {
            ctl->job.init = p.handed + (blockIdx.x - 1) * size;
            ctl->job.init_k = job.dv;
            ctl->job.init_v = 1;
        }
        if (hands) ctl->job.last = p.handed + blockIdx.x * size;
        ctl->wait_flag = handed ? p.flags + blockIdx.x - 1 : nullptr;
        ctl->patience = 100000ull * p.rounds;
        ctl->hands = hands;
        ctl->part = part;
        ctl->t0 = uint32_t(begin);
        ctl->b = p.offsets ? 0 : b;
        ctl->clipped = !p.offsets;
        ctl->h = h;
        ctl->count = count;
        // a split walk has a first phase, over K and V only, in the blocks whose totals later blocks need
        ctl->before = p.ranks > 1 && part.last < part.groups ? count : 0;
        ctl->split = p.ranks > 1;
        ctl->log2_decay = log2_of(p.log_decay[h]);
        uint32_t lo = part.first, hi = part.first + ctl->before;           // the groups with a third term are the last ones
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (has_third(ctl, part, mid)) hi = mid;
            else lo = mid + 1;
        }
        ctl->thirds = part.first + ctl->before - lo;
        ctl->entered = job.init || part.first > 0;
        ctl->owns_last = hands || (job.last && (part.groups == 0 ? rank == 0 : (part.last == part.groups && count > 0)));
    }
    // One thread: the next walk of a block whose share is a stretch of the list of all walks, in which a walk has a place for every
    // group, and one more for what it costs to begin it.  From the last walk back to the first: what the next block waits for comes
    // first, what this one waits for last.
    static __device__ __noinline__ void next_walk(const MixParams &p) {
        MixCtl *ctl = mix_ctl();
        const uint64_t lo = ctl->places_from;
        uint64_t to = ctl->places_to, walk = 0;
        MixPart part;
        part.len = uint32_t(p.tokens);
        part.groups = (part.len + kGroup - 1) / kGroup;
        part.per = part.groups;
        do {
            ctl->none = to == lo;
            if (to == lo) return;
            walk = (to - 1) / (part.groups + 1);
            const uint64_t at = walk * (part.groups + 1), from = max(lo, at);
            part.first = min(uint32_t(from - at), part.groups);
            part.last = min(uint32_t(to - at), part.groups);
            to = from;
        } while (part.first == part.groups);         // only the place for its beginning: there is nothing to do
        const uint32_t unit = uint32_t(walk / p.jobs), job = uint32_t(walk - uint64_t(unit) * p.jobs);
        part.lead = p.job[job].lead != 0;
        ctl->more = to > lo;
        ctl->places_to = to;
        take(p, part, job, unit / p.heads, unit % p.heads, 0, 0, true);
    }
    // Whether there is another walk (all threads); if so, its barriers may be set up.
    static __device__ __forceinline__ bool goes_on() {
        MixCtl *ctl = mix_ctl();
        if (!ctl->more || ctl->abort_flag) return false;
        if (threadIdx.x == 32 * kProducerWarp)
            for (uint64_t *one = &ctl->full[0]; one <= &ctl->drained[1]; ++one)
                if (one < &ctl->full[kSlots] || (one >= &ctl->empty[0] && one < &ctl->empty[kSlots]) || one >= &ctl->qk_done) mbar_inval(smem_u32(one));
        __syncthreads();                     // everybody has seen what the next walk replaces
        return true;
    }
    // One thread.
    static __device__ __forceinline__ void begin_barriers() {
        MixCtl *ctl = mix_ctl();
        for (uint32_t i = 0; i < kSlots; ++i) {
            mbar_init(smem_u32(&ctl->full[i]), 1);
            mbar_init(smem_u32(&ctl->empty[i]), 2);
        }
        for (uint64_t *one : {&ctl->qk_done, &ctl->pv_done, &ctl->e_done, &ctl->k_scaled, &ctl->first_done, &ctl->kv_done, &ctl->drained[0], &ctl->drained[1]}) mbar_init(smem_u32(one), 1);
        mbar_init(smem_u32(&ctl->p_ready), 32 * kTokenWarps);
        mbar_init(smem_u32(&ctl->o_free), 32 * kTokenWarps);
        mbar_init(smem_u32(&ctl->o_staged), 32 * kTokenWarps);
        mbar_init(smem_u32(&ctl->x_ready), 128);
        mbar_init(smem_u32(&ctl->k_ready), 32 * kKeyWarps);
        mbar_init(smem_u32(&ctl->third_ready), 32 * kKeyWarps);
        fence_barrier_init();
    }
    // -inf becomes a value whose multiples are finite, so that a^0 = 1; a NaN stays one and reaches every output and state of its head
    static __device__ __forceinline__ float log2_of(float log_decay) {
        const float x = log_decay * 1.4426950408889634f;
        return x < -1e30f ? -1e30f : x;
    }
    // All threads: decays a^m = 2^(m log2 a)
    static __device__ __forceinline__ void tables(float log2a, bool lead, float scale, const MixPart &part) {
        MixCtl *ctl = mix_ctl();
        if (threadIdx.x < kNear) {
            const int apart = int(threadIdx.x) - 47;
            const float power = exp2f(log2a * float(max(apart, 0)));
            ctl->near[lead ? kNear - 1 - threadIdx.x : threadIdx.x] = apart >= 0 ? scale * power : 0.0f;
            if (apart >= 0 && apart <= kGroup) ctl->power[apart] = power;
            if (apart >= 0 && apart < 16) ctl->block[lead ? 15 - apart : apart] = scale * power;
        }
        if (threadIdx.x >= 256 && threadIdx.x < 264) ctl->rank_decay[threadIdx.x - 256] = exp2f(log2a * part.tokens_of_rank(threadIdx.x - 256));
    }
    // the state that enters the walk
    template <bool CUT>
    static __device__ __noinline__ void enter() {
        MixCtl *ctl = mix_ctl();
        const int warp = threadIdx.x >> 5, row = (warp & 3) * 32 + (threadIdx.x & 31);
        if (!(ctl->entered || ctl->count == 0) || (warp & 3) * 32 >= D) return;
        const bool exchanged = ctl->split && ctl->count > 0;
        const float *exchange = reinterpret_cast<const float *>(reinterpret_cast<uint8_t *>(ctl) + kMixCtlBytes) + row;
        const float *from = exchanged ? exchange : ctl->job.init + uint64_t(row) * ctl->job.init_v;
        const uint32_t pitch = exchanged ? D : ctl->job.init_k, rows = exchanged ? D : ctl->job.init && uint32_t(row) < ctl->job.dv ? ctl->job.dk : 0;
        if (CUT && ctl->wait_flag) {                 // (a block waits only for the one before it, all of them run at once, and what that
            const uint64_t from = global_ns();       // one hands over it works on first)
            while (ld_acquire_u32(ctl->wait_flag) == 0) {
                if (global_ns() - from > ctl->patience) {
                    ctl->abort_flag = 1;
                    break;
                }
                __nanosleep(200);
            }
            __syncwarp();
        }
#pragma unroll 1
        for (uint32_t c = 0; c < D; c += 16) {
            uint32_t v[16];
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) v[j] = c + j < rows ? __float_as_uint(from[uint64_t(c + j) * pitch]) : 0u;
            tmem_st16(ctl->tmem_base + (uint32_t(warp & 3) << 21) + kColX + c, v);
        }
        tmem_st_wait();
    }

    // One thread, while the block is being set up: the first group's tiles on their way into L2, and with them the descriptors.
    static __device__ __forceinline__ void first_tiles(const CUtensorMap *maps, const MixJob &job, const MixPart &part, int token, int b, int h) {
        if (part.first >= part.last) return;
        const int at = token + int(part.in_time(part.first) * kGroup);
#pragma unroll
        for (int which = 0; which < 3; ++which)
#pragma unroll
            for (int half = 0; half < D / 64; ++half)
                tma_prefetch_l2_4d(maps + job.map[which], half * 64, at, h * int(job.by_head[which]), b * int(job.by_batch[which]));
    }
    // ---- loads (one thread): K and V of the groups of the first phase; K, Q and V of those of the walk
    static __device__ __noinline__ void loads(const CUtensorMap *maps, uint32_t phase) {
        MixCtl *ctl = mix_ctl();
        const MixPart part = ctl->part;
        const uint32_t n = phase ? ctl->count : ctl->before;
        uint32_t tile = phase ? 2 * ctl->before : 0, group = 0;
#pragma unroll 1
        for (uint32_t place = 0; group < n; ++tile) {
            const uint32_t slot = tile % kSlots;
            const uint32_t ahead = group + kAhead;
            if (ahead < n) {                        // into L2, so that a load issued when its slot falls free takes less than the chain leaves it
                const uint32_t which = place == 0 ? 1 : place == 1 && phase ? 0 : 2;
#pragma unroll
                for (int half = 0; half < D / 64; ++half)
                    tma_prefetch_l2_4d(maps + ctl->job.map[which], half * 64, int(ctl->t0 + part.in_time(part.first + ahead) * kGroup), int(ctl->h * ctl->job.by_head[which]),
                                       int(ctl->b * ctl->job.by_batch[which]));
            }
            if (tile >= kSlots && !mix_wait(ctl, ctl->empty[slot], (tile / kSlots - 1) & 1)) break;
            const uint32_t which = place == 0 ? 1 : place == 1 && phase ? 0 : 2;
            const uint32_t bar = smem_u32(&ctl->full[slot]), token = ctl->t0 + part.in_time(part.first + group) * kGroup;
            mbar_expect_tx(bar, kTile);
#pragma unroll
            for (int half = 0; half < D / 64; ++half)
                tma_load_4d(ring_at(ctl) + slot * kTile + half * kHalfBytes, maps + ctl->job.map[which], half * 64, int(token), int(ctl->h * ctl->job.by_head[which]),
                            int(ctl->b * ctl->job.by_batch[which]), bar);
            if (++place == phase + 2) {
                place = 0;
                ++group;
            }
        }
        const uint32_t last = tile > kSlots ? tile - kSlots : 0;
        if (phase && group == n)                    // commits that free the last tiles arrive on barriers of this block: not after it has ended
            for (uint32_t m = last; m < tile && mix_wait(ctl, ctl->empty[m % kSlots], (m / kSlots) & 1); ++m) {}
        if (!phase || ctl->abort_flag)              // copies in flight must land before the block may exit, or (from others, in the exchange) write there
            for (uint32_t m = last; m < tile; ++m) mbar_wait_bounded(smem_u32(&ctl->full[m % kSlots]), (m / kSlots) & 1, kMixWaitRounds);
    }

    // ---- products: a whole warp walks the loop, so that descriptors stay in uniform registers; one lane issues
    static __device__ __forceinline__ void drain(MixCtl *ctl, int which) {
        if (ctl->abort_flag && elect_one()) {       // products in flight must end: tensor memory is freed afterwards
            mma_commit(smem_u32(&ctl->drained[which]));
            mbar_wait_bounded(smem_u32(&ctl->drained[which]), 0, kMixWaitRounds);
        }
        __syncwarp();
    }
    // scores of group i, then O of the group
    static __device__ __noinline__ void scores() {
        MixCtl *ctl = mix_ctl();
        const uint32_t n = ctl->count, base = ctl->before, tmem = ctl->tmem_base;
        const uint32_t short_group = ctl->part.len % kGroup == 0 ? ~0u : (ctl->part.lead ? ctl->part.groups - 1 : 0u) - ctl->part.first;
        const uint32_t idesc_s = make_idesc(H::kType, kGroup), idesc_o = make_idesc(H::kType, D) | kIdescBMn;
        uint32_t tile = 2 * base;
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i, tile += 3) {
            if (!wait_full(ctl, tile) || !wait_full(ctl, tile + 1)) break;
            if (i > 0) {
                if (!mix_wait_warp(ctl, ctl->pv_done, (i - 1) & 1)) break;                      // S holds P until it has been multiplied
                // (the key warps must not miss that the last scores were done)
                if (!mix_wait_warp(ctl, ctl->k_ready, (base + i - 1) & 1)) break;
            }
            tc_fence_after();
            if (elect_one()) {
                const uint64_t qa = make_smem_desc(slot_at(ctl, tile + 1)), kb = make_smem_desc(slot_at(ctl, tile));
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    mma_issue<false>(tmem + kColS, qa + (s / 4) * (kHalfBytes >> 4) + (s % 4) * 2, kb + (s / 4) * (kHalfBytes >> 4) + (s % 4) * 2, idesc_s, s > 0);
                mma_commit(smem_u32(&ctl->qk_done));
                mma_commit(smem_u32(&ctl->empty[tile % kSlots]));
                mma_commit(smem_u32(&ctl->empty[(tile + 1) % kSlots]));
            }
            __syncwarp();
            if (!wait_full(ctl, tile + 2) || !mix_wait_warp(ctl, ctl->p_ready, i & 1)) break;
            if (i > 0 && !mix_wait_warp(ctl, ctl->o_free, (i - 1) & 1)) break;
            if (i == short_group && !mix_wait_warp(ctl, ctl->k_ready, (base + i) & 1)) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t vb = make_smem_desc_mn(slot_at(ctl, tile + 2), kHalfBytes);
#pragma unroll
                for (int s = 0; s < kGroup / 16; ++s)
                    mma_issue_ta(tmem + kColO, tmem + kColS + (s / 4) * 64 + (s % 4) * 8, vb + s * (2048 >> 4), idesc_o, s > 0);
                mma_commit(smem_u32(&ctl->pv_done));
                mma_commit(smem_u32(&ctl->empty[(tile + 2) % kSlots]));
            }
            __syncwarp();
        }
        drain(ctl, 0);
    }
    // X^T += V^T K~, one term of K~: lanes are columns of v, columns are rows of the state.  With D = 64 the upper 64 lanes multiply
    // whatever lies behind the tile; nobody reads them.
    static __device__ __noinline__ void issue_state(uint32_t tmem, uint32_t v_slot, uint32_t term, bool onto) {
        const uint32_t idesc = make_idesc(H::kType, D) | kIdescAMn | kIdescBMn;
        const uint64_t va = make_smem_desc_mn(v_slot, kHalfBytes), ka = make_smem_desc_mn(term, kHalfBytes);
#pragma unroll
        for (int s = 0; s < kGroup / 16; ++s) mma_issue<false>(tmem + kColX, va + s * (2048 >> 4), ka + s * (2048 >> 4), idesc, onto || s > 0);
    }
    // E of group i, then its part of the state
    static __device__ __noinline__ void products(uint32_t phase) {
        MixCtl *ctl = mix_ctl();
        const uint32_t n = phase ? ctl->count : ctl->before, tmem = ctl->tmem_base;
        const bool entered = phase && ctl->entered, owns_last = !phase || ctl->owns_last;
        const uint32_t idesc_e = make_idesc(H::kType, D);
        const MixPart part = ctl->part;
        uint32_t it = phase ? ctl->before : 0, tile = 2 * it, thirds = phase ? ctl->thirds : 0;
        const uint32_t end = it + n, silent = ctl->silent;
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i, ++it, tile += phase + 2) {
            const uint32_t nv = tile + phase + 1;
            const bool fresh = i == 0 && !entered, wanted = i + 1 < n || owns_last, third = wanted && has_third(ctl, part, part.first + i);
            if (phase && (!wait_full(ctl, tile + 1) || (i > 0 && !mix_wait_warp(ctl, ctl->o_free, (i - 1) & 1)))) break;
            if (!wait_full(ctl, nv) || !mix_wait_warp(ctl, ctl->x_ready, it & 1)) break;
            tc_fence_after();
            if (phase && elect_one()) {
                if (!fresh) {
                    const uint64_t qa = make_smem_desc(slot_at(ctl, tile + 1)), xb = make_smem_desc(x_at(ctl));
#pragma unroll
                    for (int s = 0; s < D / 16; ++s)
                        mma_issue<false>(tmem + kColE, qa + (s / 4) * (kHalfBytes >> 4) + (s % 4) * 2, xb + (s / 4) * (kXHalf >> 4) + (s % 4) * 2, idesc_e, s > 0);
                }
                mma_commit(smem_u32(&ctl->e_done));
            }
            __syncwarp();
            if (!mix_wait_warp(ctl, ctl->k_ready, it & 1)) break;
            tc_fence_after();
            if (elect_one()) {
                if (wanted) {
                    issue_state(tmem, slot_at(ctl, nv), slot_at(ctl, tile), !fresh);
                    if (third) mma_commit(smem_u32(&ctl->first_done));
                    issue_state(tmem, slot_at(ctl, nv), low_at(ctl), true);
                }
            }
            __syncwarp();
            if (third) {
                if (!mix_wait_warp(ctl, ctl->third_ready, thirds & 1)) break;
                tc_fence_after();
                ++thirds;
            }
            if (elect_one()) {
                if (third) issue_state(tmem, slot_at(ctl, nv), slot_at(ctl, tile), true);
                if (it + 1 != silent) {
                    mma_commit(smem_u32(&ctl->kv_done));
                    mma_commit(smem_u32(&ctl->empty[tile % kSlots]));
                    mma_commit(smem_u32(&ctl->empty[nv % kSlots]));
                    if (!phase) {                   // (nobody else uses them)
                        mma_commit(smem_u32(&ctl->empty[tile % kSlots]));
                        mma_commit(smem_u32(&ctl->empty[nv % kSlots]));
                    }
                }
            }
            __syncwarp();
        }
        // (the last one is not waited for by anybody else when no state is wanted; the first phase's is, by the state role)
        if (phase && n > 0 && it == end) mix_wait_warp(ctl, ctl->kv_done, (it - 1) & 1);
        drain(ctl, 1);
    }

    // ---- stores (one thread)
    static __device__ __noinline__ void stores(const CUtensorMap *maps) {
        MixCtl *ctl = mix_ctl();
        const MixPart part = ctl->part;
        const uint32_t n = ctl->count;
        uint32_t tile = 2 * ctl->before + 1;
#pragma unroll 1
        for (uint32_t i = 0; i < n; ++i, tile += 3) {
            if (!mix_wait(ctl, ctl->o_staged, i & 1)) break;
            if (ctl->clipped || part.tokens_of(part.first + i) == kGroup) {
#pragma unroll
                for (int half = 0; half < D / 64; ++half)
                    if (uint32_t(half * 64) < ctl->job.dv)
                        tma_store_4d(maps + ctl->job.map[3], slot_at(ctl, tile) + half * kHalfBytes, half * 64, int(ctl->t0 + part.in_time(part.first + i) * kGroup),
                                     int(ctl->h), int(ctl->b));
                bulk_commit();
                bulk_wait_read();
            }
            mbar_arrive(smem_u32(&ctl->empty[tile % kSlots]));
        }
        bulk_wait_all();
    }

    // ---- between the phases, all threads of the cluster: element e of every part's total, in walking order; the state that enters a
    // part takes the place of its total
    static __device__ __noinline__ void exchange(uint32_t ranks, uint32_t rank) {
        MixCtl *ctl = mix_ctl();
        __syncwarp();
        cluster_sync_all();
        const MixPart part = ctl->part;
        const uint32_t at = smem_u32(ctl) + kMixCtlBytes, dk = ctl->job.dk, dv = ctl->job.dv;
        const float *init = ctl->job.init;
#pragma unroll 1
        for (uint32_t e = 4 * (rank * kMixThreads + threadIdx.x); e < D * D; e += 4 * ranks * kMixThreads) {
            const uint32_t c = e / D, r = e % D;
            float4 run = make_float4(0.0f, 0.0f, 0.0f, 0.0f), total[8];
            if (init && c < dk) {
                const float *from = init + uint64_t(c) * ctl->job.init_k;
                const uint32_t pitch = ctl->job.init_v;
                if (r < dv) run.x = from[uint64_t(r) * pitch];
                if (r + 1 < dv) run.y = from[uint64_t(r + 1) * pitch];
                if (r + 2 < dv) run.z = from[uint64_t(r + 2) * pitch];
                if (r + 3 < dv) run.w = from[uint64_t(r + 3) * pitch];
            }
#pragma unroll
            for (uint32_t s = 0; s < 8; ++s)
                if ((s + 1) * part.per < part.groups) total[s] = ld_cluster_f32x4(cluster_map(at + 4 * e, s));
#pragma unroll
            for (uint32_t s = 0; s < 8; ++s) {
                if (s >= ranks || s * part.per >= part.groups) break;
                st_cluster_f32x4(cluster_map(at + 4 * e, s), run);
                if ((s + 1) * part.per < part.groups) {
                    const float a = ctl->rank_decay[s];
                    run = make_float4(fmaf(a, run.x, total[s].x), fmaf(a, run.y, total[s].y), fmaf(a, run.z, total[s].z), fmaf(a, run.w, total[s].w));
                }
            }
        }
        cluster_sync_all();
    }
};

// The places of packed sequences, the longest first: thread i counts the sequences that come before sequence i, four at a time.
// (One block: found by every block of the walk for itself, this cost each of them 2.4 us with 200 sequences.)
__global__ void __launch_bounds__(kMostOrdered) tcu_linattn_order_kernel(const int64_t *offsets, uint32_t batch, uint32_t *order) {
    __shared__ alignas(16) uint32_t lens[kMostOrdered];
    begin_in_sequence();
    const uint32_t mine = threadIdx.x, len = mine < batch ? uint32_t(max(offsets[mine + 1] - offsets[mine], int64_t(0))) : 0;
    lens[mine] = len;
    __syncthreads();
    if (mine >= batch) return;
    uint32_t before = 0;
#pragma unroll 4
    for (uint32_t i = 0; i < batch; i += 4) {
        const uint4 other = *reinterpret_cast<const uint4 *>(lens + i);
        before += (other.x > len || (other.x == len && i < mine)) + (other.y > len || (other.y == len && i + 1 < mine)) +
                  (other.z > len || (other.z == len && i + 2 < mine)) + (other.w > len || (other.w == len && i + 3 < mine));
    }
    order[before] = mine;
}

// kWhole: a block, or a cluster of them, has one walk; kOrdered: the same with the walks of long sequences first; kCut: a block has
// a share of all walks, which begins and ends anywhere.  (A kernel that does the one or the other costs small calls 1 to 2 us.)
enum { kWhole, kOrdered, kCut };
template <int D, typename T, int KIND>
__global__ void __launch_bounds__(kMixThreads, 1) tcu_linattn_mix_kernel(const __grid_constant__ MixParams p) {
    using M = Mix<D, T>;
    MixCtl *ctl = mix_ctl();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr bool CUT = KIND == kCut;
    const uint32_t ranks = CUT ? 1 : p.ranks, rank = CUT ? 0 : blockIdx.x % p.ranks;
    if (threadIdx.x == 0) {
        ctl->abort_flag = 0;
        ctl->rounds = p.rounds;
        ctl->silent = p.silent;
        if (CUT) {
            const uint64_t places = (uint64_t(p.tokens + kGroup - 1) / kGroup + 1) * p.batch * p.heads * p.jobs;
            ctl->places_from = places * blockIdx.x / gridDim.x;
            ctl->places_to = places * (blockIdx.x + 1) / gridDim.x;
        }
        ctl->more = false;
    }
    auto allocate = [&] {
        if (warp != kProductWarp) return;
        tmem_alloc(smem_u32(&ctl->tmem_base), M::kColumns);
        tmem_relinquish();
    };
    if (CUT) allocate();
#pragma unroll 1
    do {
        if (warp == kProducerWarp && lane == 0) M::begin_barriers();
        if constexpr (CUT) {
            if (threadIdx.x == 0) M::next_walk(p);
            __syncthreads();
            if (ctl->none) break;
            M::tables(ctl->log2_decay, ctl->part.lead, ctl->job.in_scale * ctl->job.out_scale, ctl->part);
        } else {
            const uint32_t work = blockIdx.x / ranks, unit = work / p.jobs, h = unit % p.heads;
            uint32_t b = unit / p.heads;
            if (KIND == kOrdered) {
                begin_in_sequence();
                b = p.order[b];
            }
            const MixJob &job = p.job[work % p.jobs];
            // packed: whatever the offsets hold, no token outside the arrays is touched
            const int64_t most = int64_t(p.tokens), begin = p.offsets ? min(max(p.offsets[b], int64_t(0)), most) : 0;
            MixPart part;
            part.lead = job.lead != 0;
            part.len = uint32_t(p.offsets ? min(max(p.offsets[b + 1], begin), most) - begin : most);
            part.groups = (part.len + kGroup - 1) / kGroup;
            part.per = (part.groups + ranks - 1) / ranks;
            part.first = min(rank * part.per, part.groups);
            part.last = min((rank + 1) * part.per, part.groups);
            if (warp == kProducerWarp && lane == 0) M::first_tiles(p.map, job, part, int(begin), p.offsets ? 0 : int(b), int(h));
            if (threadIdx.x == 0) M::take(p, part, work % p.jobs, b, h, begin, rank, false);
            M::tables(M::log2_of(p.log_decay[h]), part.lead, job.in_scale * job.out_scale, part);
            allocate();
        }
        tc_fence_before();
        __syncthreads();
        tc_fence_after();

#pragma unroll 1
        for (uint32_t phase = ranks > 1 ? 0 : 1; phase < 2; ++phase) {
            if (phase) {
                // a first phase that was given up left the barriers anywhere: what would wait on them now could take an old phase for a new one
                if (!CUT && ranks > 1 && ctl->abort_flag) break;
                if (warp >= kStateWarp && warp < kProducerWarp) M::template enter<CUT>();
                if (ranks > 1) {
                    fence_proxy_async_smem();                               // the next writes to the exchange buffer are TMA loads
                    tc_fence_before();
                    __syncthreads();
                    tc_fence_after();
                }
            }
            if (warp < kTokenWarps) {
                if (phase) M::tokens();
            } else if (warp < kStateWarp) {
                M::keys(phase);
            } else if (warp < kProducerWarp) {
                M::state(phase);
            } else if (warp == kProducerWarp) {
                if (lane == 0) M::loads(p.map, phase);
            } else if (warp == kScoreWarp) {
                if (phase) M::scores();
            } else if (warp == kProductWarp) {
                M::products(phase);
            } else if (phase && lane == 0) {
                M::stores(p.map);
            }
            if (!CUT && !phase) M::exchange(ranks, rank);
        }
        __syncwarp();
        if (CUT) fence_proxy_async_smem();   // the next walk's tiles are TMA loads
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (CUT && threadIdx.x == 0 && ctl->hands) {
            __threadfence();
            st_release_u32(p.flags + blockIdx.x, 1);
        }
    } while (CUT && M::goes_on());
    if (warp == kProductWarp) tmem_dealloc(ctl->tmem_base, M::kColumns);
    if (threadIdx.x == 0 && ctl->abort_flag) st_system_u32(p.error, 5u);             // (it may lie on the host)
}

// ---- single tokens ---------------------------------------------------------------------------------------------------
struct StepParams {
    MixTokens q, k, v, o;
    float *pool;
    const int32_t *slots;
    const float *log_decay;
    uint64_t pool_slots;
    uint32_t batch, heads, dk, dv;
    float scale;
};

constexpr int kStepCols = 64;            // dv columns of a block
constexpr int kStepThreads = 256;

// A block updates 64 columns of one state: S <- a S + k v^T, and sums q_r S[r][c] over the rows.  VEC columns a thread (4
// where rows are 16-byte aligned), 64 / VEC threads a row.  Bound by reading and writing the state once, so every thread
// asks for all of its state before it looks at the token: 192 sequences of 16 heads at 128 x 128, 407 MB, 66.5 us
// (6.1 TB/s; 82 us with the token first, 70.5 with blocks of 32 columns); one sequence of 16 heads 4.2 us, a launch.
template <typename T, int VEC>
__global__ void __launch_bounds__(kStepThreads) tcu_linattn_step_kernel(const __grid_constant__ StepParams p) {
    constexpr int kTx = kStepCols / VEC, kTy = kStepThreads / kTx;
    __shared__ float sq[128], sk[128];
    __shared__ float part[kTy][kStepCols];
    const uint32_t b = blockIdx.x / p.heads, h = blockIdx.x % p.heads;
    const int tx = threadIdx.x % kTx, ty = threadIdx.x / kTx;
    const uint32_t col = blockIdx.y * kStepCols + tx * VEC;
    const int64_t slot = p.slots ? int64_t(p.slots[b]) : int64_t(b);
    T *o = const_cast<T *>(reinterpret_cast<const T *>(p.o.ptr)) + int64_t(b) * p.o.batch + int64_t(h) * p.o.head;
    if (slot < 0 || uint64_t(slot) >= p.pool_slots) {
        for (int c = threadIdx.x; c < kStepCols; c += kStepThreads)
            if (blockIdx.y * kStepCols + c < p.dv) o[blockIdx.y * kStepCols + c] = from_f32<T>(0.0f);
        return;
    }
    float *state = p.pool + (uint64_t(slot) * p.heads + h) * p.dk * p.dv;
    const T *q = reinterpret_cast<const T *>(p.q.ptr) + int64_t(b) * p.q.batch + int64_t(h) * p.q.head;
    const T *k = reinterpret_cast<const T *>(p.k.ptr) + int64_t(b) * p.k.batch + int64_t(h) * p.k.head;
    const T *v = reinterpret_cast<const T *>(p.v.ptr) + int64_t(b) * p.v.batch + int64_t(h) * p.v.head;
    // the state is under way before the token is looked at
    constexpr int kRows = 128 / kTy;
    const bool mine = col < p.dv;
    Pack<float, VEC> s[kRows];
#pragma unroll
    for (int j = 0; j < kRows; ++j)
        if (mine && uint32_t(ty + j * kTy) < p.dk) s[j] = *reinterpret_cast<const Pack<float, VEC> *>(state + uint64_t(ty + j * kTy) * p.dv + col);
    for (uint32_t i = threadIdx.x; i < p.dk; i += kStepThreads) {
        sq[i] = to_f32(q[i]);
        sk[i] = to_f32(k[i]);
    }
    const float a = expf(p.log_decay[h]);
    float vv[VEC], acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        vv[e] = mine ? to_f32(v[col + e]) : 0.0f;
        acc[e] = 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        const uint32_t r = ty + j * kTy;
        if (!mine || r >= p.dk) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            s[j].v[e] = fmaf(sk[r], vv[e], a * s[j].v[e]);
            acc[e] = fmaf(sq[r], s[j].v[e], acc[e]);
        }
        *reinterpret_cast<Pack<float, VEC> *>(state + uint64_t(r) * p.dv + col) = s[j];
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) part[ty][tx * VEC + e] = acc[e];
    __syncthreads();
    if (threadIdx.x < kStepCols && blockIdx.y * kStepCols + threadIdx.x < p.dv) {
        float sum = 0.0f;
#pragma unroll
        for (int y = 0; y < kTy; ++y) sum += part[y][threadIdx.x];
        o[blockIdx.y * kStepCols + threadIdx.x] = from_f32<T>(sum * p.scale);
    }
}

}  // namespace tcu
