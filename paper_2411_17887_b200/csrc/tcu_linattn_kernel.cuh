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
//     tokens    (8 warps, 4 when dk, dv <= 64) thread = token: scores -> P, then O + decayed E -> the slot that held Q
//     state     (as many) thread = column of v: X out of tensor memory, rounded into the operand of E, multiplied by a^L and put
//               back; thread = token: K -> K~
//     producer  TMA: K, Q, V of each group into a ring of five tiles
//     issuer    tcgen05.mma
//     store     TMA: the outputs
// Rounded to 16 bits are only operands of a product: P, and X as operand of E (the state itself stays in 32 bits in tensor
// memory).  K~ enters the state in two terms in float16, 22 bits of mantissa, and in three in bfloat16, 24 bits (two, 16
// bits, left states 2e-6 to 5e-6 off where 32-bit sums are 2e-7 off).  In float16 X and K~ are brought to the type's range by powers of two found for every group, because a state without decay
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
    uint64_t kt_ready;                   // two terms of K~ written (and rows past the end of V cleared)
    uint64_t two_done;                   // ... and multiplied
    uint64_t third_ready;                // third term written over the second
    uint64_t p_ready;                    // P in tensor memory
    uint64_t o_done;                     // O and E are in tensor memory
    uint64_t o_free;                     // ... and have been read
    uint64_t kv_done;                    // the group is in X
    uint64_t o_staged;                   // output tile written to shared memory
    uint64_t drained;
    uint32_t tmem_base;
    volatile uint32_t abort_flag;
    float biggest[2][16];                // float16: largest |k| and |X| seen by each warp
    float unscale[2];                    // float16: the factor that takes E back to the size of X
    float power[kGroup + 4];             // a^m
    alignas(16) float block[32];         // factors of P along a block of 32 tokens
    float near[32 + kGroup + 32];        // factors of P by distance, from 31 tokens on the wrong side of the diagonal (zero) on
};
static_assert(sizeof(MixCtl) <= kMixCtlBytes, "control block too large");

// warps of the token role and of the state role: a thread has 64 columns of a row, of X and of K; then producer, issuer, store
template <int D> constexpr int kMixRoleWarps = D / 16;
template <int D> constexpr int kMixThreads = 32 * (2 * kMixRoleWarps<D> + 3);
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
__global__ void __launch_bounds__(kMixThreads<D>, D == 64 ? 2 : 1) tcu_linattn_mix_kernel(const __grid_constant__ MixParams p) {
    using H = Half2<T>;
    constexpr bool kIsHalf = std::is_same<T, __half>::value;
    constexpr bool kThird = !kIsHalf;                             // K~ in three terms
    constexpr int kTile = kMixTileBytes<D>;
    constexpr int kXHalf = D * 128;                               // one 64-wide half of the operand X: D rows of 128 bytes
    constexpr int kWarps = kMixRoleWarps<D>, kRole = kWarps * 32; // warps and threads of the token role, and of the state role
    // tensor memory: S, O, E, X.  P takes the place of S; with D = 128 two warps share the 128 columns of a token, so each
    // 64 columns of S leave their P in their own first 32 columns.  With D = 64 P fills the first 64 columns of S and O the
    // others, and two blocks share an SM.
    constexpr uint32_t kColS = 0, kColO = D == 128 ? 128 : 64, kColE = D == 128 ? 256 : 128, kColX = D == 128 ? 384 : 192;
    constexpr uint32_t kColP1 = D == 128 ? 64 : 32;               // P of tokens 64 ... 127
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
    const bool entered = job.init || (split && rank > 0);                    // the walk starts from a state (else from zero)
    const uint32_t before = totals ? count : 0;                              // groups of the first phase
    const uint32_t tile0 = 2 * before;                                       // tiles loaded in the first phase
    const int bz = p.offsets ? 0 : int(b);

    // ---- loads.  Tile n of the block: K and V of the groups of the first phase, then K, Q and V of those of the walk.
    auto slot_of = [&](uint32_t n) { return ring_at + (n % kMixSlots) * kTile; };
    auto load = [&](uint32_t n) {
        const uint32_t m = n - tile0, group = n < tile0 ? n >> 1 : m / 3;
        const uint32_t which = n < tile0 ? (n & 1 ? 2 : 1) : (m % 3 == 0 ? 1 : m % 3 == 1 ? 0 : 2);
        const int token = int(t0 + int64_t(part.in_time(part.first + group)) * kGroup);
        const uint32_t bar = smem_u32(&ctl->full[n % kMixSlots]);
        mbar_expect_tx(bar, kTile);
        for (int half = 0; half < D / 64; ++half)
            tma_load_4d(slot_of(n) + half * kHalfBytes, &p.map[job.map[which]], half * 64, token, int(h) * job.by_head[which],
                        bz * job.by_batch[which], bar);
    };
    const uint32_t phase_one = split ? tile0 : tile0 + 3 * count, tiles = tile0 + 3 * count;
    uint32_t issued = 0;
    if (warp == 2 * kWarps && lane == 0) {
        for (int i = 0; i < kMixSlots; ++i) {
            mbar_init(smem_u32(&ctl->full[i]), 1);
            mbar_init(smem_u32(&ctl->empty[i]), 1);
        }
        mbar_init(smem_u32(&ctl->qk_done), 1);
        mbar_init(smem_u32(&ctl->x_ready), kRole);
        mbar_init(smem_u32(&ctl->kt_ready), kRole);
        mbar_init(smem_u32(&ctl->third_ready), kRole);
        mbar_init(smem_u32(&ctl->p_ready), kRole);
        mbar_init(smem_u32(&ctl->o_done), 1);
        mbar_init(smem_u32(&ctl->o_free), kRole);
        mbar_init(smem_u32(&ctl->two_done), 1);
        mbar_init(smem_u32(&ctl->kv_done), 1);
        mbar_init(smem_u32(&ctl->o_staged), kRole);
        mbar_init(smem_u32(&ctl->drained), 1);
        ctl->abort_flag = 0;
        fence_barrier_init();
        for (; issued < kMixSlots && issued < phase_one; ++issued) load(issued);       // the ring is empty
    }
    if (warp == 2 * kWarps + 1) {
        tmem_alloc(smem_u32(&ctl->tmem_base), kColumns);
        tmem_relinquish();
    }
    // decays: a^m = 2^(m log2 a); -inf becomes a value whose multiples are finite, so that a^0 = 1
    const float log2a = fmaxf(p.log_decay[h] * 1.4426950408889634f, -1e30f);
    if (threadIdx.x <= kGroup) ctl->power[threadIdx.x] = exp2f(log2a * float(threadIdx.x));
    if (threadIdx.x < 32) ctl->block[threadIdx.x] = job.in_scale * job.out_scale * exp2f(log2a * float(part.lead ? 31 - int(threadIdx.x) : int(threadIdx.x)));
    if (threadIdx.x < 32 + kGroup + 32) {
        const int apart = int(threadIdx.x) - 31;
        ctl->near[threadIdx.x] = apart >= 0 ? job.in_scale * job.out_scale * exp2f(log2a * float(apart)) : 0.0f;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem_base;
    const MixWaiter w{ctl, p.error, p.spin_limit};

    // ---- roles.  Each takes the groups [0, before) of the first phase, then [0, count) of the walk; `it` counts both.
    // Rows of a tile: token i of the group at i * 128 bytes, 16-byte pieces exchanged by the swizzle (piece ^ (i & 7)).
    auto produce = [&](uint32_t end) {
        for (; issued < end; ++issued) {
            if (issued >= kMixSlots && !w.wait(ctl->empty[issued % kMixSlots], (issued / kMixSlots - 1) & 1)) return;
            load(issued);
        }
    };
    auto full = [&](uint32_t n) { return w.wait(ctl->full[n % kMixSlots], (n / kMixSlots) & 1); };
    auto full_warp = [&](uint32_t n) { return wait_warp(w, ctl->full[n % kMixSlots], (n / kMixSlots) & 1); };

    // ---- the issuer: a whole warp walks the loop, so that descriptors stay in uniform registers; one lane issues
    const uint32_t idesc_s = make_idesc(H::kType, kGroup), idesc_d = make_idesc(H::kType, D);
    // X^T += V^T K~, one term of K~: lanes are columns of v, columns are rows of the state.  With D = 64 the upper 64 lanes
    // multiply whatever lies behind the tile; nobody reads them.
    auto issue_state = [&](uint32_t kt, uint32_t v_slot, bool onto) {
        const uint64_t va = make_smem_desc_mn(v_slot, kHalfBytes), kb = make_smem_desc_mn(kt, kHalfBytes);
#pragma unroll
        for (int s = 0; s < kGroup / 16; ++s)
            mma_issue<false>(tmem + kColX, va + s * (2048 >> 4), kb + s * (2048 >> 4), idesc_d | kIdescAMn | kIdescBMn, onto || s > 0);
    };
    // the state's products of group `it`, in two steps; false when a wait was given up
    auto state_two = [&](uint32_t it, uint32_t k_slot, uint32_t v_slot, bool wanted, bool onto) {
        if (!wait_warp(w, ctl->kt_ready, it & 1)) return false;
        tc_fence_after();
        if (elect_one()) {
            if (wanted) {
                issue_state(k_slot, v_slot, onto);
                issue_state(low_at, v_slot, true);
            }
            if (kThird) mma_commit(smem_u32(&ctl->two_done));
        }
        __syncwarp();
        return true;
    };
    auto state_rest = [&](uint32_t it, uint32_t nk, uint32_t nv, bool wanted) {
        if (kThird && wanted) {
            if (!wait_warp(w, ctl->third_ready, it & 1)) return false;
            tc_fence_after();
        }
        if (elect_one()) {
            if (kThird && wanted) issue_state(low_at, slot_of(nv), true);
            mma_commit(smem_u32(&ctl->kv_done));
            mma_commit(smem_u32(&ctl->empty[nk % kMixSlots]));
            mma_commit(smem_u32(&ctl->empty[nv % kMixSlots]));
        }
        __syncwarp();
        return true;
    };
    auto multiply_totals = [&]() {
        for (uint32_t i = 0; i < before; ++i) {
            const uint32_t nk = 2 * i, nv = nk + 1;
            if (!full_warp(nk) || !full_warp(nv) || !wait_warp(w, ctl->x_ready, i & 1)) return;
            if (!state_two(i, slot_of(nk), slot_of(nv), true, i > 0) || !state_rest(i, nk, nv, true)) return;
        }
    };
    auto multiply = [&]() {
        auto scores = [&](uint32_t i) {
            const uint32_t nk = tile0 + 3 * i, nq = nk + 1;
            if (!full_warp(nk) || !full_warp(nq)) return false;
            // the last group's P has been multiplied (D = 64: and its O, which lies in S, has been read)
            if (i > 0 && !wait_warp(w, D == 64 ? ctl->o_free : ctl->o_done, (i - 1) & 1)) return false;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t qa = make_smem_desc(slot_of(nq)), kb = make_smem_desc(slot_of(nk));
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    mma_issue<false>(tmem + kColS, qa + (s / 4) * (kHalfBytes >> 4) + (s % 4) * 2, kb + (s / 4) * (kHalfBytes >> 4) + (s % 4) * 2, idesc_s, s > 0);
                mma_commit(smem_u32(&ctl->qk_done));
            }
            __syncwarp();
            return true;
        };
        if (count > 0 && !scores(0)) return;
        for (uint32_t i = 0; i < count; ++i) {
            const uint32_t it = before + i;
            const uint32_t nk = tile0 + 3 * i, nq = nk + 1, nv = nk + 2;
            const bool fresh = i == 0 && !entered, wanted = i + 1 < count || owns_last;
            if (!wait_warp(w, ctl->x_ready, it & 1)) return;
            if (i > 0 && !wait_warp(w, ctl->o_free, (i - 1) & 1)) return;
            tc_fence_after();
            if (!fresh && elect_one()) {
                const uint64_t qa = make_smem_desc(slot_of(nq)), xb = make_smem_desc(x_at);
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    mma_issue<false>(tmem + kColE, qa + (s / 4) * (kHalfBytes >> 4) + (s % 4) * 2, xb + (s / 4) * (kXHalf >> 4) + (s % 4) * 2, idesc_d, s > 0);
            }
            __syncwarp();
            if (part.tokens_of(part.first + i) < kGroup && !wait_warp(w, ctl->kt_ready, it & 1)) return;
            if (!full_warp(nv) || !wait_warp(w, ctl->p_ready, i & 1)) return;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t vb = make_smem_desc_mn(slot_of(nv), kHalfBytes);
#pragma unroll
                for (int s = 0; s < kGroup / 16; ++s)
                    mma_issue_ta(tmem + kColO, tmem + kColS + (s / 4) * kColP1 + (s % 4) * 8, vb + s * (2048 >> 4), idesc_d | kIdescBMn, s > 0);
                mma_commit(smem_u32(&ctl->o_done));
            }
            __syncwarp();
            // the next scores go before the last term of the state, while the state warps write it; with D = 64 they would
            // have to wait for the outputs to be read, and the other block of the SM fills the gap
            if (!state_two(it, slot_of(nk), slot_of(nv), wanted, !fresh)) return;
            if (D == 128 && i + 1 < count && !scores(i + 1)) return;
            if (!state_rest(it, nk, nv, wanted)) return;
            if (D == 64 && i + 1 < count && !scores(i + 1)) return;
        }
    };

    const uint32_t lanes = tmem + (uint32_t(warp & 3) << 21);       // this warp's 32 lanes (bits 16 and up)
    const int row = (warp & 3) * 32 + lane;                         // token of the group, or column of v
    const int part64 = (warp % kWarps) / 4 * 64;                    // this thread's 64 columns of a row (features, or rows of the state)
    const bool holds_x = (warp & 3) * 32 < D;                       // whole warps: X has D lanes
    const uint32_t swizzled = uint32_t(row * 128), sw = uint32_t(row & 7);

    // state warps: X <- values
    auto fill_x = [&](auto value) {
        if (holds_x) {
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                uint32_t v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(value(part64 + c + j));
                tmem_st32(lanes + kColX + part64 + c, v);
            }
            tmem_st_wait();
        }
    };
    // state warps: use(column, X) for this thread's values
    auto read_x = [&](auto use) {
        if (holds_x) {
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                uint32_t v[32];
                tmem_ld32(lanes + kColX + part64 + c, v);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) use(part64 + c + j, __uint_as_float(v[j]));
            }
        }
    };
    // float16 only: powers of two that keep the operands inside the type.  X is held as 2^held X, so that the decayed keys of the
    // group can be used as 2^held K~ with the largest near 2^14 (small ones would lose their low term below 2^-24).
    int held = 0;
    auto pow2 = [](int n) { return __uint_as_float(uint32_t(min(max(n, -126), 127) + 127) << 23); };
    auto exponent = [](float x) { return int((__float_as_uint(x) >> 23) & 0xFF) - 127; };
    auto biggest_k = [&](uint32_t k_slot) {
        float big = 0.0f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            uint32_t k4[4];
            ld_shared_v4(k_slot + (part64 / 64) * kHalfBytes + swizzled + ((c ^ sw) << 4), k4[0], k4[1], k4[2], k4[3]);
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
                const float2 keep2 = make_float2(keep, keep), shrink2 = make_float2(shrink, shrink);
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                uint32_t v[32];
                tmem_ld32(lanes + kColX + part64 + c, v);
                tmem_ld_wait();
                if (operand) {
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        uint32_t w4[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float2 x = make_float2(__uint_as_float(v[j + 2 * e]), __uint_as_float(v[j + 2 * e + 1]));
                            if (kIsHalf) x = mul2(x, shrink2);
                            w4[e] = H::pack(x.x, x.y);
                        }
                        st_shared_v4(x_at + (part64 / 64) * kXHalf + swizzled + ((((c + j) >> 3) ^ sw) << 4), w4[0], w4[1], w4[2], w4[3]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    const float2 x = mul2(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), keep2);
                    v[j] = __float_as_uint(x.x);
                    v[j + 1] = __float_as_uint(x.y);
                }
                tmem_st32(lanes + kColX + part64 + c, v);
            }
            tmem_st_wait();
        }
        if (operand) fence_proxy_async_smem();
        tc_fence_before();
        mbar_arrive(smem_u32(&ctl->x_ready));
    };
    // K~ in two terms, in the place of K and in the buffer of the low terms; with three, the last one in turn takes the place
    // of the second when that has been multiplied
    auto step_k = [&](uint32_t it, int tokens, uint32_t k_slot, uint32_t v_slot, bool wanted) {
        uint32_t rest[kThird ? 32 : 1];
        if (wanted) {
            // walking order: token `row` of the group is j = row forward, tokens - 1 - row backward; a^(tokens - j - lead)
            const float f = row < tokens ? job.in_scale * ctl->power[part.lead ? tokens - 1 - row : row + 1] * (kIsHalf ? pow2(held) : 1.0f) : 0.0f;
            const float2 f2 = make_float2(f, f), minus = make_float2(-1.0f, -1.0f);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint32_t at = (part64 / 64) * kHalfBytes + swizzled + ((c ^ sw) << 4);
                uint32_t k4[4], hi[4], lo[4];
                ld_shared_v4(k_slot + at, k4[0], k4[1], k4[2], k4[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (row >= tokens) k4[e] = 0;
                    const float2 x = mul2(H::unpack(k4[e]), f2);
                    hi[e] = H::pack(x.x, x.y);
                    const float2 y = fma2(H::unpack(hi[e]), minus, x);
                    lo[e] = H::pack(y.x, y.y);
                    if (kThird) {
                        const float2 z = fma2(H::unpack(lo[e]), minus, y);
                        rest[kThird ? 4 * c + e : 0] = H::pack(z.x, z.y);
                    }
                }
                st_shared_v4(k_slot + at, hi[0], hi[1], hi[2], hi[3]);
                st_shared_v4(low_at + at, lo[0], lo[1], lo[2], lo[3]);
            }
        }
        if (row >= tokens) {           // what follows the sequence may hold anything: zero times it has to be zero
#pragma unroll
            for (int c = 0; c < 8; ++c) st_shared_v4(v_slot + (part64 / 64) * kHalfBytes + swizzled + (c << 4), 0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        mbar_arrive(smem_u32(&ctl->kt_ready));
        if (kThird && wanted) {
            if (!wait_warp(w, ctl->two_done, it & 1)) return false;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                st_shared_v4(low_at + (part64 / 64) * kHalfBytes + swizzled + ((c ^ sw) << 4), rest[kThird ? 4 * c : 0], rest[kThird ? 4 * c + 1 : 0],
                             rest[kThird ? 4 * c + 2 : 0], rest[kThird ? 4 * c + 3 : 0]);
            fence_proxy_async_smem();
            mbar_arrive(smem_u32(&ctl->third_ready));
        }
        return true;
    };
    auto carry = [&](bool outputs) {
        const uint32_t n = outputs ? count : before;
        bool ok = true;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t it = outputs ? before + i : i;
            const uint32_t nk = outputs ? tile0 + 3 * i : 2 * i, nv = outputs ? nk + 2 : nk + 1;
            const int tokens = part.tokens_of(part.first + i);
            const bool fresh = i == 0 && !(outputs && entered);            // X is zero: the first product does not add to it
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
                float big_x = 0.0f;
                if (ok && !fresh) read_x([&](int, float x) { big_x = fmaxf(big_x, fabsf(x)); });
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    big_k = fmaxf(big_k, __shfl_xor_sync(0xffffffffu, big_k, o));
                    big_x = fmaxf(big_x, __shfl_xor_sync(0xffffffffu, big_x, o));
                }
                if (lane == 0) {
                    ctl->biggest[i & 1][warp % kWarps] = big_k;
                    ctl->biggest[i & 1][kWarps + warp % kWarps] = big_x;
                }
                ok = !named_barrier_or(1, kRole, !ok);              // the warps of the role meet here, so they give up together
                if (ok) {
#pragma unroll
                    for (int j = 0; j < kWarps; ++j) {
                        big_k = fmaxf(big_k, ctl->biggest[i & 1][j]);
                        big_x = fmaxf(big_x, ctl->biggest[i & 1][kWarps + j]);
                    }
                    const int ex = min(max(exponent(big_x), -60), 127);
                    shrink = pow2(14 - ex);
                    if (threadIdx.x == kRole) ctl->unscale[i & 1] = pow2(ex - 14 - held);
                    // the powers of a in K~ go from a^(1 - lead) to a^(tokens - lead)
                    const float top = fmaxf(ctl->power[1 - job.lead], ctl->power[tokens - int(job.lead)]);
                    const int now = min(max(14 - exponent(big_k * fabsf(job.in_scale) * top), -30), 100);
                    keep *= pow2(now - held);
                    held = now;
                }
            }
            if (!ok) break;
            if (fresh) mbar_arrive(smem_u32(&ctl->x_ready));
            else step_x(shrink, keep, outputs);
            ok = __all_sync(0xffffffffu, full(nk) && (tokens == kGroup || full(nv)));
            ok = ok && (!outputs || wait_warp(w, ctl->qk_done, i & 1));
            if (ok) ok = step_k(it, tokens, slot_of(nk), slot_of(nv), !outputs || i + 1 < n || owns_last);
        }
        return ok;
    };

    // token warps
    auto attend = [&]() {
        const int row0 = (warp & 3) * 32;
        for (uint32_t i = 0; i < count; ++i) {
            const int tokens = part.tokens_of(part.first + i);
            if (!wait_warp(w, ctl->qk_done, i & 1)) return;
            tc_fence_after();
            // scores of 32 tokens at a time: all of them count, none, or (around the diagonal and the end) some
#pragma unroll 1
            for (int c = part64; c < (D == 128 ? part64 + 64 : kGroup); c += 32) {
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
                        const float2 f2 = make_float2(f, f);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float4 t = reinterpret_cast<const float4 *>(ctl->block)[j];
                            const float2 x = mul2(make_float2(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1])), mul2(f2, make_float2(t.x, t.y)));
                            const float2 y = mul2(make_float2(__uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])), mul2(f2, make_float2(t.z, t.w)));
                            out[2 * j] = H::pack(x.x, x.y);
                            out[2 * j + 1] = H::pack(y.x, y.y);
                        }
                    } else {
                        // (what does not count may not be finite: it is left out, not multiplied by zero)
                        const int apart = part.lead ? row - c : c - row;
                        const float *factor = ctl->near + 31 + apart;
                        if (part.lead) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = apart >= j ? __float_as_uint(__uint_as_float(v[j]) * factor[-j]) : 0u;
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                v[j] = apart + j >= 0 && c + j < tokens ? __float_as_uint(__uint_as_float(v[j]) * factor[j]) : 0u;
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) out[j] = H::pack(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
                    }
                }
                tmem_st16(lanes + kColS + (c / 64) * kColP1 + (c % 64) / 2, out);         // never over scores still to be read
            }
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(smem_u32(&ctl->p_ready));

            if (!wait_warp(w, ctl->o_done, i & 1) || !wait_warp(w, ctl->x_ready, (before + i) & 1)) return;
            tc_fence_after();
            const bool fresh = i == 0 && !entered;                 // no state: E was not formed
            const uint32_t slot = slot_of(tile0 + 3 * i + 1) + (part64 / 64) * kHalfBytes;
            const int order = part.lead ? row : tokens - 1 - row;
            float e = order >= 0 ? job.out_scale * ctl->power[order + int(job.lead)] : 0.0f;
            if (kIsHalf) e *= ctl->unscale[i & 1];
            const float2 e2 = make_float2(e, e);
            const int64_t token = t0 + int64_t(part.in_time(part.first + i)) * kGroup + row;
            T *to = reinterpret_cast<T *>(job.o) + bz * job.o_batch + token * job.o_token + int64_t(h) * job.o_head;
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                uint32_t vo[32], ve[32];
                tmem_ld32(lanes + kColO + part64 + c, vo);
                if (!fresh) tmem_ld32(lanes + kColE + part64 + c, ve);
                tmem_ld_wait();
                if (!fresh) {
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 x = fma2(e2, make_float2(__uint_as_float(ve[j]), __uint_as_float(ve[j + 1])), make_float2(__uint_as_float(vo[j]), __uint_as_float(vo[j + 1])));
                        vo[j] = __float_as_uint(x.x);
                        vo[j + 1] = __float_as_uint(x.y);
                    }
                }
                uint32_t out[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) out[j] = H::pack(__uint_as_float(vo[2 * j]), __uint_as_float(vo[2 * j + 1]));
                if (tokens == kGroup) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        st_shared_v4(slot + swizzled + (((c / 8 + j) ^ sw) << 4), out[4 * j], out[4 * j + 1], out[4 * j + 2], out[4 * j + 3]);
                } else if (row < tokens) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int col = part64 + c + 8 * j;
                        if (uint32_t(col + 8) <= job.dv) {
                            st_global_v4(to + col, out[4 * j], out[4 * j + 1], out[4 * j + 2], out[4 * j + 3]);
                        } else {
                            const T *x = reinterpret_cast<const T *>(out + 4 * j);
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                if (uint32_t(col + k) < job.dv) to[col + k] = x[k];
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
    const bool token_role = warp < kWarps, state_role = warp >= kWarps && warp < 2 * kWarps;

    // ---- the first phase of a split walk: what this part leaves from a state of zero, and the states that enter the parts
    if (split) {
        if (warp == 2 * kWarps && lane == 0) produce(tile0);
        if (warp == 2 * kWarps + 1) multiply_totals();
        if (state_role && totals) {
            if (carry(false) && wait_warp(w, ctl->kv_done, (before - 1) & 1)) {
                tc_fence_after();
                read_x([&](int c, float x) { exchange[c * D + row] = x * (kIsHalf ? pow2(-held) : 1.0f); });
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
        if (state_role) {
            if (count > 0 && entered) fill_x([&](int c) { return exchange[c * D + row]; });
            else if (count == 0 && owns_last) fill_x(init_at);
        }
        fence_proxy_async_smem();                       // the next writes to the exchange buffer are TMA loads
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    } else if (state_role && (entered || count == 0)) {
        fill_x(init_at);
    }

    // ---- the walk
    if (token_role) {
        attend();
    } else if (state_role) {
        const bool ok = carry(true);
        if (owns_last && (count == 0 || (ok && wait_warp(w, ctl->kv_done, (before + count - 1) & 1)))) {
            tc_fence_after();
            float *to = job.last + uint64_t(unit) * job.dk * job.dv + row;
            read_x([&](int c, float x) {
                if (uint32_t(c) < job.dk && uint32_t(row) < job.dv) to[uint64_t(c) * job.dv] = x * (kIsHalf ? pow2(-held) : 1.0f);
            });
        }
    } else if (warp == 2 * kWarps) {
        if (lane == 0) {
            produce(tiles);
            if (ctl->abort_flag)                        // copies in flight must land before the block may exit
                for (uint32_t n = issued > kMixSlots ? issued - kMixSlots : 0; n < issued; ++n) {
                    const uint32_t bar = smem_u32(&ctl->full[n % kMixSlots]);
                    const long long since = clock64();
                    while (!mbar_try_wait(bar, (n / kMixSlots) & 1) && clock64() - since < p.spin_limit) {}
                }
        }
    } else if (warp == 2 * kWarps + 1) {
        multiply();
        if (ctl->abort_flag && elect_one()) {           // so must products: tensor memory is freed below
            mma_commit(smem_u32(&ctl->drained));
            const long long since = clock64();
            while (!mbar_try_wait(smem_u32(&ctl->drained), 0) && clock64() - since < p.spin_limit) {}
        }
    } else if (lane == 0) {
        store();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 2 * kWarps + 1) tmem_dealloc(tmem, kColumns);
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
