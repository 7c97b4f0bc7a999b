// Linear attention with a constant decay for each head.
//
// One form, a "mixing", serves the forward pass and all three gradients.  Walking a sequence forward in time
// (lead = 1) or backward (lead = 0), with a state X of dk x dv values,
//     lead = 1:  X <- a X + in_scale * k_t v_t^T,   o_t = out_scale * X^T q_t
//     lead = 0:  X <- X + in_scale * k_t v_t^T,     o_t = out_scale * X^T q_t,   X <- a X
//     o  = mix(q, k, v)       forward, from the state before the first token, leaving the one after the last
//     dq = mix(do, v, k)      forward, from the transposed state
//     dv = mix(k, q, do)      backward, from the gradient of the last state, leaving the gradient of the first
//     dk = mix(v, do, q)      backward, from its transpose
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "tcu_embedding_kernel.cuh"

namespace tcu {

struct MixTokens {
    const void *ptr;
    int64_t batch, token, head;      // strides in elements
};

struct MixJob {
    MixTokens q, k, v, o;
    const float *init;               // state before the first token walked, or NULL; (sequence, head) entries of dk * dv values
    float *last;                     // NULL, or receives the state after the last
    int64_t init_k, init_v;          // strides of init along dk and dv (last: dv, 1)
    uint32_t dk, dv;
    uint32_t lead;                   // 1: forward in time, 0: backward
    float in_scale, out_scale;
};

struct MixParams {
    MixJob job[3];
    const float *log_decay;
    const int64_t *offsets;
    uint64_t tokens;
    uint32_t batch, heads, jobs;
};

constexpr int kMixCols = 32, kMixTile = 16;

// A block walks one (job, sequence, head) for 32 of its dv columns: warp w holds rows 32 w ... of the state in
// registers, lane = column; 16 tokens at a time through shared memory.
template <typename T>
__global__ void __launch_bounds__(128) tcu_linattn_mix_kernel(const __grid_constant__ MixParams p) {
    __shared__ float sq[kMixTile][128], sk[kMixTile][128], sv[kMixTile][kMixCols], part[4][kMixTile][kMixCols];
    const MixJob &j = p.job[blockIdx.x % p.jobs];
    const uint32_t unit = blockIdx.x / p.jobs, b = unit / p.heads, h = unit % p.heads;
    const uint32_t col = blockIdx.y * kMixCols;
    if (col >= j.dv) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t0 = p.offsets ? p.offsets[b] : 0, len = p.offsets ? p.offsets[b + 1] - t0 : int64_t(p.tokens);
    auto at = [&](const MixTokens &x, int64_t t) {
        return reinterpret_cast<const T *>(x.ptr) + (p.offsets ? 0 : int64_t(b) * x.batch) + (t0 + t) * x.token + int64_t(h) * x.head;
    };
    const float a = expf(p.log_decay[h]);
    const bool mine = col + lane < j.dv;
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const uint32_t r = warp * 32 + i;
        x[i] = j.init && mine && r < j.dk ? j.init[uint64_t(unit) * j.dk * j.dv + r * j.init_k + (col + lane) * j.init_v] : 0.0f;
    }
    for (int64_t base = 0; base < len; base += kMixTile) {
        const int m = int(len - base < kMixTile ? len - base : kMixTile);
        __syncthreads();
        for (int i = threadIdx.x; i < m * 128; i += 128) {
            const int t = i >> 7, c = i & 127;
            const int64_t time = j.lead ? base + t : len - 1 - base - t;
            sq[t][c] = uint32_t(c) < j.dk ? to_f32(at(j.q, time)[c]) : 0.0f;
            sk[t][c] = uint32_t(c) < j.dk ? to_f32(at(j.k, time)[c]) * j.in_scale : 0.0f;
            if (c < kMixCols) sv[t][c] = col + c < j.dv ? to_f32(at(j.v, time)[col + c]) : 0.0f;
        }
        __syncthreads();
        for (int t = 0; t < m; ++t) {
            float o = 0.0f;
            const float v = sv[t][lane];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float kv = sk[t][warp * 32 + i];
                x[i] = fmaf(kv, v, j.lead ? a * x[i] : x[i]);
                o = fmaf(sq[t][warp * 32 + i], x[i], o);
                if (!j.lead) x[i] *= a;
            }
            part[warp][t][lane] = o;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < m * kMixCols; i += 128) {
            const int t = i / kMixCols, c = i % kMixCols;
            const int64_t time = j.lead ? base + t : len - 1 - base - t;
            if (col + c < j.dv)
                const_cast<T *>(at(j.o, time))[col + c] = from_f32<T>(j.out_scale * (part[0][t][c] + part[1][t][c] + part[2][t][c] + part[3][t][c]));
        }
    }
    if (j.last && mine) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const uint32_t r = warp * 32 + i;
            if (r < j.dk) j.last[uint64_t(unit) * j.dk * j.dv + uint64_t(r) * j.dv + col + lane] = x[i];
        }
    }
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
