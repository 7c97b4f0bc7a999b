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
// A block (one job, sequence, head and - in a cluster - part of the walk) runs the groups one after another.  Warps:
//     8     TMA producer: K, Q, V of each group into a ring of five tiles
//     9     tcgen05.mma issuer
//     0-3   thread = token: scores -> P, then O + decayed E -> the slot that held Q
//     4-7   thread = column of v: X out of tensor memory, rounded into the operand of E, multiplied by a^L and put back;
//           thread = token: K -> K~
//     10    TMA store of the outputs
// Rounded to 16 bits are only operands of a product: P, and X as operand of E (the state itself stays in 32 bits in tensor
// memory).  K~ enters the state in two terms, 16 bits of mantissa and more, because states are results of their own.  In
// float16 X and K~ are brought to the type's range by powers of two found for every group, because a state without decay
// outgrows the type and the low terms of small keys fall below it.
//
// When there are fewer (job, sequence, head) than SMs, the walk is split over the blocks of a cluster: each block first
// forms the state that its part leaves from zero (K and V only), the blocks exchange them through distributed shared
// memory, and each walks its part from the state that enters it.
//
// Every wait is bounded; one that runs out records TCU_ERR_TIMEOUT in the workspace and the block winds down.
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
constexpr int kMixSlots = 5;             // tiles in the ring
constexpr int kMixThreads = 352;
constexpr int kHalfBytes = 16384;        // 128 tokens x 64 features: one 128-byte-swizzled block of rows
constexpr int kMixCtlBytes = 2048;

struct MixTokens {
    const void *ptr;
    int64_t batch, token, head;          // strides in elements
};

struct MixJob {
    uint8_t map[4];                      // tensor maps of q, k, v, o
    uint8_t by_batch[4], by_head[4];     // 0 where the array repeats along that axis
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
    long long spin_limit;
};

struct MixCtl {
    uint64_t full[kMixSlots], empty[kMixSlots];
    uint64_t qk_done;                    // S is in tensor memory
    uint64_t x_ready;                    // X rounded into its operand, and multiplied by a^L in tensor memory
    uint64_t kt_ready;                   // K~ written (and rows past the end of V cleared)
    uint64_t p_ready;                    // P in tensor memory
    uint64_t o_done;                     // O and E are in tensor memory
    uint64_t o_free;                     // ... and have been read
    uint64_t kv_done;                    // the group is in X
    uint64_t o_staged;                   // output tile written to shared memory
    uint64_t drained;
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    float biggest[2][8];                 // float16: largest |k| and |X| seen by each of the four warps
    float unscale[2];                    // float16: the factor that takes E back to the size of X
    float power[kGroup + 4];             // a^m
    float block[32];                     // factors of P along a block of 32 tokens
};
static_assert(sizeof(MixCtl) <= kMixCtlBytes, "control block too large");

template <int D> constexpr int kMixTileBytes = D / 64 * kHalfBytes;
template <int D> constexpr int kMixSmemBytes = 1024 + kMixCtlBytes + (kMixSlots + 1) * kMixTileBytes<D> + D * D * 2;
static_assert(kMixSmemBytes<128> <= 232448 && 2 * (kMixSmemBytes<64> + 1024) <= 233472, "shared memory of an SM");

template <typename T> struct Half2;
template <> struct Half2<__nv_bfloat16> {
    static constexpr uint32_t kType = 2;             // as in make_idesc
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&p);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
};
template <> struct Half2<__half> {
    static constexpr uint32_t kType = 1;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 p = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&p);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
};

struct MixWaiter {
    MixCtl *ctl;
    uint32_t *error;
    long long limit;
    __device__ __forceinline__ bool wait(const uint64_t &barrier, uint32_t parity) const {
        const uint32_t bar = smem_u32(&barrier);
        if (mbar_try_wait(bar, parity)) return true;
        const long long t0 = clock64();
        uint32_t spins = 0;
        while (!mbar_try_wait(bar, parity)) {
            if ((++spins & 0xFF) == 0) {
                if (ctl->abort_flag) return false;
                if (clock64() - t0 > limit) {
                    ctl->abort_flag = 1;
                    atomicExch(error, 5u);
                    return false;
                }
            }
        }
        return true;
    }
};

// the same for a whole warp, with one answer for all lanes
__device__ __forceinline__ bool wait_warp(const MixWaiter &w, const uint64_t &barrier, uint32_t parity) {
    return __all_sync(0xffffffffu, w.wait(barrier, parity));
}

// Which groups of a walk a block takes, and how many tokens.
struct MixPart {
    uint32_t groups, per, first, last;        // groups of the sequence, per block, this block's [first, last) in walking order
    int64_t len;
    bool lead;
    __device__ __forceinline__ uint32_t in_time(uint32_t p) const { return lead ? p : groups - 1 - p; }
    __device__ __forceinline__ int tokens_of(uint32_t p) const {
        const int64_t left = len - int64_t(in_time(p)) * kGroup;
        return left < kGroup ? int(left) : kGroup;
    }
    __device__ __forceinline__ float tokens_of_rank(uint32_t r) const {
        const uint32_t a = min(r * per, groups), b = min((r + 1) * per, groups);
        const int64_t lo = int64_t(lead ? a : groups - b) * kGroup, hi = int64_t(lead ? b : groups - a) * kGroup;
        return float((hi < len ? hi : len) - (lo < len ? lo : len));
    }
};

template <int D, typename T>
__global__ void __launch_bounds__(kMixThreads, D == 64 ? 2 : 1) tcu_linattn_mix_kernel(const __grid_constant__ MixParams p) {
    using H = Half2<T>;
    constexpr bool kIsHalf = std::is_same<T, __half>::value;
    constexpr int kTile = kMixTileBytes<D>;
    constexpr int kXHalf = D * 128;                               // one 64-wide half of the operand X: D rows of 128 bytes
    // tensor memory: S (P in its first 64 columns), O, E, X.  With D = 64 O lies in the half of S that P leaves free, and two
    // blocks share an SM.
    constexpr uint32_t kColS = 0, kColO = D == 128 ? 128 : 64, kColE = D == 128 ? 256 : 128, kColX = D == 128 ? 384 : 192;
    constexpr uint32_t kColumns = D == 128 ? 512 : 256;

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    MixCtl *ctl = reinterpret_cast<MixCtl *>(smem);
    uint8_t *ring = smem + kMixCtlBytes;
    const uint32_t ring_at = smem_u32(ring), low_at = ring_at + kMixSlots * kTile, x_at = low_at + kTile;
    float *exchange = reinterpret_cast<float *>(ring);            // D x D state totals, between the two phases of a split walk

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x % p.ranks, work = blockIdx.x / p.ranks;
    const MixJob &job = p.job[work % p.jobs];
    const uint32_t unit = work / p.jobs, b = unit / p.heads, h = unit % p.heads;
    // packed: whatever the offsets hold, no token outside the arrays is touched
    const int64_t most = int64_t(p.tokens), t0 = p.offsets ? min(max(p.offsets[b], int64_t(0)), most) : 0;
    MixPart part;
    part.lead = job.lead != 0;
    part.len = p.offsets ? min(max(p.offsets[b + 1], t0), most) - t0 : most;
    part.groups = uint32_t((part.len + kGroup - 1) / kGroup);
    part.per = (part.groups + p.ranks - 1) / p.ranks;
    part.first = min(rank * part.per, part.groups);
    part.last = min((rank + 1) * part.per, part.groups);
    const uint32_t count = part.last - part.first;
    const bool split = p.ranks > 1;
    const bool totals = split && count > 0 && part.last < part.groups;       // later blocks need what this part leaves
    const bool owns_last = job.last && (part.groups == 0 ? rank == 0 : (part.last == part.groups && count > 0));
    const uint32_t before = totals ? count : 0;                              // groups of the first phase
    const uint32_t tile0 = 2 * before;                                       // tiles loaded in the first phase
    const int bz = p.offsets ? 0 : int(b);

    // decays: a^m = 2^(m log2 a); -inf becomes a value whose multiples are finite, so that a^0 = 1
    const float log2a = fmaxf(p.log_decay[h] * 1.4426950408889634f, -1e30f);
    if (threadIdx.x <= kGroup) ctl->power[threadIdx.x] = exp2f(log2a * float(threadIdx.x));
    if (threadIdx.x < 32) ctl->block[threadIdx.x] = job.in_scale * job.out_scale * exp2f(log2a * float(part.lead ? 31 - int(threadIdx.x) : int(threadIdx.x)));
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMixSlots; ++i) {
            mbar_init(smem_u32(&ctl->full[i]), 1);
            mbar_init(smem_u32(&ctl->empty[i]), 1);
        }
        mbar_init(smem_u32(&ctl->qk_done), 1);
        mbar_init(smem_u32(&ctl->x_ready), 128);
        mbar_init(smem_u32(&ctl->kt_ready), 128);
        mbar_init(smem_u32(&ctl->p_ready), 128);
        mbar_init(smem_u32(&ctl->o_done), 1);
        mbar_init(smem_u32(&ctl->o_free), 128);
        mbar_init(smem_u32(&ctl->kv_done), 1);
        mbar_init(smem_u32(&ctl->o_staged), 128);
        mbar_init(smem_u32(&ctl->drained), 1);
        ctl->abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(&ctl->tmem_base), kColumns);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem_base;
    const MixWaiter w{ctl, p.error, p.spin_limit};
    auto slot_of = [&](uint32_t n) { return ring_at + (n % kMixSlots) * kTile; };

    // ---- roles.  Each takes the groups [0, before) of phase one, then [0, count) of phase two; `it` counts both.
    // Rows of a tile: token i of the group at i * 128 bytes, 16-byte pieces exchanged by the swizzle (piece ^ (i & 7)).
    uint32_t issued = 0;                                           // producer: tiles loaded
    auto produce = [&](bool want_q) {
        const uint32_t n = want_q ? count : before;
        for (uint32_t i = 0; i < n; ++i) {
            const int token = int(t0 + int64_t(part.in_time(part.first + i)) * kGroup);
            for (int a = 0; a < 3; ++a) {
                if (a == 1 && !want_q) continue;
                const int which = a == 0 ? 1 : a == 1 ? 0 : 2;     // K, Q, V
                const uint32_t s = issued % kMixSlots;
                if (issued >= kMixSlots && !w.wait(ctl->empty[s], (issued / kMixSlots - 1) & 1)) return;
                const uint32_t bar = smem_u32(&ctl->full[s]);
                mbar_expect_tx(bar, kTile);
                for (int half = 0; half < D / 64; ++half)
                    tma_load_4d(ring_at + s * kTile + half * kHalfBytes, &p.map[job.map[which]], half * 64, token, int(h) * job.by_head[which],
                                bz * job.by_batch[which], bar);
                ++issued;
            }
        }
    };
    auto full = [&](uint32_t n) { return w.wait(ctl->full[n % kMixSlots], (n / kMixSlots) & 1); };

    // X^T += V^T K~: lanes are columns of v, columns are rows of the state.  With D = 64 the upper 64 lanes multiply whatever
    // lies behind the tile; nobody reads them.
    auto issue_state = [&](uint32_t k_slot, uint32_t v_slot) {
        const uint32_t idesc = make_idesc(H::kType, D) | kIdescAMn | kIdescBMn;
        for (int term = 0; term < 2; ++term) {
            const uint32_t kt = term == 0 ? k_slot : low_at;
            for (int s = 0; s < kGroup / 16; ++s)
                mma_issue<false>(tmem + kColX, make_smem_desc_mn(v_slot + s * 2048, kHalfBytes), make_smem_desc_mn(kt + s * 2048, kHalfBytes), idesc, 1);
        }
    };
    auto multiply = [&](bool outputs) {
        const uint32_t n = outputs ? count : before;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t it = outputs ? before + i : i;
            const bool want_state = !outputs || i + 1 < n || owns_last;
            if (outputs) {
                const uint32_t nk = tile0 + 3 * i, nq = nk + 1, nv = nk + 2;
                const uint32_t k = slot_of(nk), q = slot_of(nq), v = slot_of(nv);
                if (!full(nk) || !full(nq)) return;
                // the last group's P has been multiplied (D = 64: and its O, which lies in S, has been read)
                if (i > 0 && !w.wait(D == 64 ? ctl->o_free : ctl->o_done, (i - 1) & 1)) return;
                tc_fence_after();
                for (int half = 0; half < D / 64; ++half)
                    for (int s = 0; s < 4; ++s)
                        mma_issue<false>(tmem + kColS, make_smem_desc(q + half * kHalfBytes + s * 32), make_smem_desc(k + half * kHalfBytes + s * 32),
                                         make_idesc(H::kType, kGroup), half + s > 0);
                mma_commit(smem_u32(&ctl->qk_done));
                if (!w.wait(ctl->x_ready, it & 1)) return;
                if (D == 128 && i > 0 && !w.wait(ctl->o_free, (i - 1) & 1)) return;
                tc_fence_after();
                for (int half = 0; half < D / 64; ++half)
                    for (int s = 0; s < 4; ++s)
                        mma_issue<false>(tmem + kColE, make_smem_desc(q + half * kHalfBytes + s * 32), make_smem_desc(x_at + half * kXHalf + s * 32),
                                         make_idesc(H::kType, D), half + s > 0);
                if (part.tokens_of(part.first + i) < kGroup && !w.wait(ctl->kt_ready, it & 1)) return;
                if (!full(nv) || !w.wait(ctl->p_ready, i & 1)) return;
                tc_fence_after();
                for (int s = 0; s < kGroup / 16; ++s)
                    mma_issue_ta(tmem + kColO, tmem + kColS + s * 8, make_smem_desc_mn(v + s * 2048, kHalfBytes), make_idesc(H::kType, D) | kIdescBMn, s > 0);
                mma_commit(smem_u32(&ctl->o_done));
                if (!w.wait(ctl->kt_ready, it & 1)) return;
                tc_fence_after();
                if (want_state) issue_state(k, v);
                mma_commit(smem_u32(&ctl->kv_done));
                mma_commit(smem_u32(&ctl->empty[nk % kMixSlots]));
                mma_commit(smem_u32(&ctl->empty[nv % kMixSlots]));
            } else {
                const uint32_t nk = 2 * i, nv = nk + 1;
                if (!full(nk) || !full(nv) || !w.wait(ctl->x_ready, it & 1) || !w.wait(ctl->kt_ready, it & 1)) return;
                tc_fence_after();
                issue_state(slot_of(nk), slot_of(nv));
                mma_commit(smem_u32(&ctl->kv_done));
                mma_commit(smem_u32(&ctl->empty[nk % kMixSlots]));
                mma_commit(smem_u32(&ctl->empty[nv % kMixSlots]));
            }
        }
    };

    const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);       // this warp's 32 lanes (bits 16 and up)
    const int row = (warp & 3) * 32 + lane;                         // token of the group, or column of v
    const bool holds_x = (warp & 3) * 32 < D;                       // whole warps: X has D lanes

    // state warps: X <- values, from tensor memory or into it
    auto fill_x = [&](auto value) {
        if (holds_x) {
            for (int c = 0; c < D; c += 32) {
                uint32_t v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(value(c + j));
                tmem_st32(lanes + kColX + c, v);
            }
            tmem_st_wait();
        }
    };
    // float16 only: powers of two that keep the operands inside the type.  X is held as 2^held X, so that the decayed keys of the
    // group can be used as 2^held K~ with the largest near 2^14 (small ones would lose their low term below 2^-24).
    int held = 0;
    auto pow2 = [](int n) { return __uint_as_float(uint32_t(min(max(n, -126), 127) + 127) << 23); };
    auto exponent = [](float x) { return int((__float_as_uint(x) >> 23) & 0xFF) - 127; };
    auto biggest_x = [&]() {
        float big = 0.0f;
        if (holds_x) {
            for (int c = 0; c < D; c += 32) {
                uint32_t v[32];
                tmem_ld32(lanes + kColX + c, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) big = fmaxf(big, fabsf(__uint_as_float(v[j])));
            }
        }
        return big;
    };
    auto biggest_k = [&](uint32_t k_slot) {
        float big = 0.0f;
        for (int c = 0; c < D / 8; ++c) {
            uint32_t k4[4];
            ld_shared_v4(k_slot + (c >> 3) * kHalfBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4), k4[0], k4[1], k4[2], k4[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = H::unpack(k4[e]);
                big = fmaxf(big, fmaxf(fabsf(x.x), fabsf(x.y)));
            }
        }
        return big;
    };
    // X rounded into the operand of E, times `shrink`, and X times `keep` left in tensor memory
    auto step_x = [&](float shrink, float keep, bool operand) {
        if (holds_x) {
            for (int c = 0; c < D; c += 32) {
                uint32_t v[32];
                tmem_ld32(lanes + kColX + c, v);
                tmem_ld_wait();
                if (operand) {
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        uint32_t w4[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w4[e] = H::pack(__uint_as_float(v[j + 2 * e]) * (kIsHalf ? shrink : 1.0f), __uint_as_float(v[j + 2 * e + 1]) * (kIsHalf ? shrink : 1.0f));
                        const int piece = ((c + j) & 63) >> 3;
                        st_shared_v4(x_at + ((c + j) >> 6) * kXHalf + row * 128 + ((piece ^ (row & 7)) << 4), w4[0], w4[1], w4[2], w4[3]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * keep);
                tmem_st32(lanes + kColX + c, v);
            }
            tmem_st_wait();
        }
        if (operand) fence_proxy_async_smem();
        tc_fence_before();
        mbar_arrive(smem_u32(&ctl->x_ready));
    };
    auto step_k = [&](int tokens, uint32_t k_slot, uint32_t v_slot, bool wanted) {
        if (wanted) {
            // walking order: token `row` of the group is j = row forward, tokens - 1 - row backward; a^(tokens - j - lead)
            const float f = row < tokens ? job.in_scale * ctl->power[part.lead ? tokens - 1 - row : row + 1] * (kIsHalf ? pow2(held) : 1.0f) : 0.0f;
            for (int c = 0; c < D / 8; ++c) {
                const uint32_t at = (c >> 3) * kHalfBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4);
                uint32_t k4[4], hi[4], lo[4];
                ld_shared_v4(k_slot + at, k4[0], k4[1], k4[2], k4[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float2 x = H::unpack(k4[e]);
                    x.x = row < tokens ? x.x * f : 0.0f;
                    x.y = row < tokens ? x.y * f : 0.0f;
                    hi[e] = H::pack(x.x, x.y);
                    const float2 y = H::unpack(hi[e]);
                    lo[e] = H::pack(x.x - y.x, x.y - y.y);
                }
                st_shared_v4(k_slot + at, hi[0], hi[1], hi[2], hi[3]);
                st_shared_v4(low_at + at, lo[0], lo[1], lo[2], lo[3]);
            }
        }
        if (row >= tokens)             // what follows the sequence may hold anything: zero times it has to be zero
            for (int c = 0; c < D / 8; ++c) st_shared_v4(v_slot + (c >> 3) * kHalfBytes + row * 128 + ((c & 7) << 4), 0, 0, 0, 0);
        fence_proxy_async_smem();
        mbar_arrive(smem_u32(&ctl->kt_ready));
    };
    auto carry = [&](bool outputs) {
        const uint32_t n = outputs ? count : before;
        bool ok = true;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t it = outputs ? before + i : i;
            const uint32_t nk = outputs ? tile0 + 3 * i : 2 * i, nv = outputs ? nk + 2 : nk + 1;
            const int tokens = part.tokens_of(part.first + i);
            float big_k = 0.0f, shrink = 1.0f, keep = ctl->power[tokens];
            if (kIsHalf) {
                ok = ok && __all_sync(0xffffffffu, full(nk));
                if (ok && row < tokens) big_k = biggest_k(slot_of(nk));
                __syncwarp();
            }
            if (i > 0) {
                ok = ok && wait_warp(w, ctl->kv_done, (it - 1) & 1);
                tc_fence_after();
            }
            if (kIsHalf) {
                float big_x = ok ? biggest_x() : 0.0f;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    big_k = fmaxf(big_k, __shfl_xor_sync(0xffffffffu, big_k, o));
                    big_x = fmaxf(big_x, __shfl_xor_sync(0xffffffffu, big_x, o));
                }
                if (lane == 0) {
                    ctl->biggest[i & 1][warp & 3] = big_k;
                    ctl->biggest[i & 1][4 + (warp & 3)] = big_x;
                }
                ok = !named_barrier_or(1, 128, !ok);              // the four warps meet here, so they give up together
                if (ok) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        big_k = fmaxf(big_k, ctl->biggest[i & 1][j]);
                        big_x = fmaxf(big_x, ctl->biggest[i & 1][4 + j]);
                    }
                    const int ex = min(max(exponent(big_x), -60), 127);
                    shrink = pow2(14 - ex);
                    if (threadIdx.x == 128) ctl->unscale[i & 1] = pow2(ex - 14 - held);
                    // the powers of a in K~ go from a^(1 - lead) to a^(tokens - lead)
                    const float most = fmaxf(ctl->power[1 - job.lead], ctl->power[tokens - int(job.lead)]);
                    const int now = min(max(14 - exponent(big_k * fabsf(job.in_scale) * most), -30), 100);
                    keep *= pow2(now - held);
                    held = now;
                }
            }
            if (!ok) break;
            step_x(shrink, keep, outputs);
            ok = __all_sync(0xffffffffu, full(nk) && (tokens == kGroup || full(nv)));
            ok = ok && (!outputs || wait_warp(w, ctl->qk_done, i & 1));
            if (ok) step_k(tokens, slot_of(nk), slot_of(nv), !outputs || i + 1 < n || owns_last);
        }
        return ok;
    };

    // token warps
    auto attend = [&]() {
        for (uint32_t i = 0; i < count; ++i) {
            const int tokens = part.tokens_of(part.first + i);
            if (!wait_warp(w, ctl->qk_done, i & 1)) return;
            tc_fence_after();
            const int row0 = (warp & 3) * 32;
#pragma unroll 1
            for (int c = 0; c < kGroup; c += 32) {
                // scores of tokens c ... c + 31: all of them count, none, or (around the diagonal and the end) some
                const bool all = part.lead ? c + 31 <= row0 : c >= row0 + 31 && c + 31 < tokens;
                const bool none = part.lead ? c > row0 + 31 : c + 31 < row0 || c >= tokens;
                uint32_t out[16];
                if (none) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) out[j] = 0;
                } else {
                    uint32_t v[32];
                    tmem_ld32(lanes + kColS + c, v);
                    tmem_ld_wait();
                    if (all) {
                        const float f = ctl->power[part.lead ? row - c - 31 : c - row];
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            out[j] = H::pack(__uint_as_float(v[2 * j]) * (f * ctl->block[2 * j]), __uint_as_float(v[2 * j + 1]) * (f * ctl->block[2 * j + 1]));
                    } else {
                        const float f = job.in_scale * job.out_scale;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const int apart = part.lead ? row - (c + j) : c + j - row;
                            const bool counts = apart >= 0 && (part.lead || c + j < tokens);
                            v[j] = counts ? __float_as_uint(__uint_as_float(v[j]) * (f * ctl->power[apart])) : 0u;
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) out[j] = H::pack(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
                    }
                }
                tmem_st16(lanes + kColS + c / 2, out);         // never over scores still to be read
            }
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(smem_u32(&ctl->p_ready));

            if (!wait_warp(w, ctl->o_done, i & 1) || !wait_warp(w, ctl->x_ready, (before + i) & 1)) return;
            tc_fence_after();
            const uint32_t slot = slot_of(tile0 + 3 * i + 1);
            const int order = part.lead ? row : tokens - 1 - row;
            float e = order >= 0 ? job.out_scale * ctl->power[order + int(job.lead)] : 0.0f;
            if (kIsHalf) e *= ctl->unscale[i & 1];
            const int64_t token = t0 + int64_t(part.in_time(part.first + i)) * kGroup + row;
            T *to = reinterpret_cast<T *>(job.o) + bz * job.o_batch + token * job.o_token + int64_t(h) * job.o_head;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                uint32_t vo[32], ve[32];
                tmem_ld32(lanes + kColO + c, vo);
                tmem_ld32(lanes + kColE + c, ve);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; j += 8) {
                    uint32_t w4[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        w4[k] = H::pack(fmaf(e, __uint_as_float(ve[j + 2 * k]), __uint_as_float(vo[j + 2 * k])),
                                        fmaf(e, __uint_as_float(ve[j + 2 * k + 1]), __uint_as_float(vo[j + 2 * k + 1])));
                    if (tokens == kGroup) {
                        const int piece = ((c + j) & 63) >> 3;
                        st_shared_v4(slot + ((c + j) >> 6) * kHalfBytes + row * 128 + ((piece ^ (row & 7)) << 4), w4[0], w4[1], w4[2], w4[3]);
                    } else if (row < tokens) {
                        if (uint32_t(c + j + 8) <= job.dv) {
                            st_global_v4(to + c + j, w4[0], w4[1], w4[2], w4[3]);
                        } else {
                            const T *x = reinterpret_cast<const T *>(w4);
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (uint32_t(c + j + k) < job.dv) to[c + j + k] = x[k];
                        }
                    }
                }
            }
            tc_fence_before();
            mbar_arrive(smem_u32(&ctl->o_free));
            if (tokens == kGroup) fence_proxy_async_smem();
            mbar_arrive(smem_u32(&ctl->o_staged));
        }
    };
    auto store = [&]() {
        for (uint32_t i = 0; i < count; ++i) {
            if (!w.wait(ctl->o_staged, i & 1)) break;
            const uint32_t n = tile0 + 3 * i + 1;
            if (part.tokens_of(part.first + i) == kGroup) {
                const int token = int(t0 + int64_t(part.in_time(part.first + i)) * kGroup);
                for (int half = 0; half < D / 64; ++half)
                    if (uint32_t(half * 64) < job.dv) tma_store_4d(&p.map[job.map[3]], slot_of(n) + half * kHalfBytes, half * 64, token, int(h), bz);
                bulk_commit();
                bulk_wait_read();
            }
            mbar_arrive(smem_u32(&ctl->empty[n % kMixSlots]));
        }
        bulk_wait_all();
    };

    auto init_at = [&](int c) -> float {
        if (!job.init || uint32_t(c) >= job.dk || uint32_t(row) >= job.dv) return 0.0f;
        return job.init[uint64_t(unit) * job.dk * job.dv + uint64_t(c) * job.init_k + uint64_t(row) * job.init_v];
    };

    // ---- phase one of a split walk: what this part leaves from a state of zero, and the states that enter the parts
    if (split) {
        if (warp == 8 && lane == 0) produce(false);
        if (warp == 9 && lane == 0) multiply(false);
        if (warp >= 4 && warp < 8 && totals) {
            fill_x([](int) { return 0.0f; });
            if (carry(false) && wait_warp(w, ctl->kv_done, (before - 1) & 1)) {
                tc_fence_after();
                if (holds_x) {
                    for (int c = 0; c < D; c += 32) {
                        uint32_t v[32];
                        tmem_ld32(lanes + kColX + c, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) exchange[(c + j) * D + row] = __uint_as_float(v[j]) * (kIsHalf ? pow2(-held) : 1.0f);

                    }
                }
            }
        }
        held = 0;
        __syncwarp();
        cluster_sync_all();
        if (threadIdx.x < 256) {
            // element e of every part's total; the state that enters part r takes its place
            const uint32_t slice = D * D / p.ranks;
            for (uint32_t e = rank * slice + threadIdx.x; e < (rank + 1) * slice; e += 256) {
                const uint32_t c = e / D, r = e % D;
                float run = 0.0f;
                if (job.init && c < job.dk && r < job.dv)
                    run = job.init[uint64_t(unit) * job.dk * job.dv + uint64_t(c) * job.init_k + uint64_t(r) * job.init_v];
                float total[8];
#pragma unroll
                for (uint32_t s = 0; s < 8; ++s)
                    if (s < p.ranks && (s + 1) * part.per < part.groups) total[s] = ld_cluster_f32(cluster_map(smem_u32(exchange + e), s));
#pragma unroll
                for (uint32_t s = 0; s < 8; ++s) {
                    if (s >= p.ranks || s * part.per >= part.groups) break;
                    st_cluster_f32(cluster_map(smem_u32(exchange + e), s), run);
                    if ((s + 1) * part.per < part.groups) run = fmaf(exp2f(log2a * part.tokens_of_rank(s)), run, total[s]);
                }
            }
        }
        cluster_sync_all();
        if (warp >= 4 && warp < 8) {
            if (count > 0) fill_x([&](int c) { return exchange[c * D + row]; });
            else fill_x(init_at);
        }
        fence_proxy_async_smem();                       // the next writes to the exchange buffer are TMA loads
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    } else if (warp >= 4 && warp < 8) {
        fill_x(init_at);
    }

    // ---- the walk
    if (warp == 8) {
        if (lane == 0) {
            produce(true);
            if (ctl->abort_flag)                        // copies in flight must land before the block may exit
                for (uint32_t n = issued > kMixSlots ? issued - kMixSlots : 0; n < issued; ++n) {
                    const uint32_t bar = smem_u32(&ctl->full[n % kMixSlots]);
                    const long long since = clock64();
                    while (!mbar_try_wait(bar, (n / kMixSlots) & 1) && clock64() - since < p.spin_limit) {}
                }
        }
    } else if (warp == 9) {
        if (lane == 0) {
            multiply(true);
            if (ctl->abort_flag) {                      // so must products: tensor memory is freed below
                mma_commit(smem_u32(&ctl->drained));
                const long long since = clock64();
                while (!mbar_try_wait(smem_u32(&ctl->drained), 0) && clock64() - since < p.spin_limit) {}
            }
        }
    } else if (warp == 10) {
        if (lane == 0) store();
    } else if (warp >= 4) {
        const bool ok = carry(true);
        if (owns_last && (count == 0 || (ok && wait_warp(w, ctl->kv_done, (before + count - 1) & 1)))) {
            tc_fence_after();
            if (holds_x) {
                for (int c = 0; c < D; c += 32) {
                    uint32_t v[32];
                    tmem_ld32(lanes + kColX + c, v);
                    tmem_ld_wait();
                    float *to = job.last + uint64_t(unit) * job.dk * job.dv + row;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (uint32_t(c + j) < job.dk && uint32_t(row) < job.dv) to[uint64_t(c + j) * job.dv] = __uint_as_float(v[j]) * (kIsHalf ? pow2(-held) : 1.0f);
                }
            }
        }
    } else {
        attend();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 9) tmem_dealloc(tmem, kColumns);
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

constexpr int kStepCols = 32;            // dv columns of a block
constexpr int kStepThreads = 128;

// A block updates 32 columns of one state: S <- a S + k v^T, and sums q_r S[r][c] over the rows.  VEC columns a thread (4
// where rows are 16-byte aligned), 32 / VEC threads a row.  Bound by reading and writing the state once.
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
    for (uint32_t i = threadIdx.x; i < p.dk; i += kStepThreads) {
        sq[i] = to_f32(q[i]);
        sk[i] = to_f32(k[i]);
    }
    const float a = expf(p.log_decay[h]);
    const bool mine = col < p.dv;
    float vv[VEC], acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        vv[e] = mine ? to_f32(v[col + e]) : 0.0f;
        acc[e] = 0.0f;
    }
    __syncthreads();
    if (mine) {
#pragma unroll 8
        for (uint32_t r = ty; r < p.dk; r += kTy) {
            Pack<float, VEC> *at = reinterpret_cast<Pack<float, VEC> *>(state + uint64_t(r) * p.dv + col);
            Pack<float, VEC> s = *at;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s.v[e] = fmaf(sk[r], vv[e], a * s.v[e]);
                acc[e] = fmaf(sq[r], s.v[e], acc[e]);
            }
            *at = s;
        }
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
