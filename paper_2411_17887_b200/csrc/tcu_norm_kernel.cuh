// Layer norm over the last axis, y = weight (x - mean) r + bias with r = 1 / sqrt(variance + eps), and its gradients: with
// u = (x - mean) r and e = weight dy,
//     dx = r (e - mean(e) - u mean(e u))        dweight = sum over rows of dy u        dbias = sum over rows of dy
// A row is held in registers by one warp or by one block, so that x (and dy) is read once; mean and variance are those of
// the values less a first mean, which takes what rounding of the first mean leaves out again.  A block goes through rows
// in steps of the grid and adds up its part of the parameters' gradients in registers; a second kernel adds the blocks' parts, in order.
#pragma once

#include "tcu_float.cuh"

namespace tcu {

constexpr int kNormWarpRows = 8;           // rows (a warp each) of a block, where a warp holds a row
constexpr int kNormMaxThreads = 1024;

struct NormParams {
    const void *x, *d_y, *weight, *bias;
    void *y, *d_x;
    float *parts;              // (blocks, 2, d): sums of dy u and of dy
    uint64_t x_stride, dy_stride;
    uint64_t rows;
    uint32_t d;
    int param_f32;             // weight and bias are fp32, else of the type of x
    float eps, inv_d;
};

// Sums of two values over a row's threads.
template <bool BLOCK>
__device__ __forceinline__ float2 sum_row(float a, float b, float2 *shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(~0u, a, o);
        b += __shfl_xor_sync(~0u, b, o);
    }
    if constexpr (BLOCK) {
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) shared[warp] = make_float2(a, b);
        __syncthreads();
        const float2 q = lane < blockDim.x >> 5 ? shared[lane] : make_float2(0.0f, 0.0f);
        a = q.x;
        b = q.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            a += __shfl_xor_sync(~0u, a, o);
            b += __shfl_xor_sync(~0u, b, o);
        }
    }
    return make_float2(a, b);
}

// E elements of a row, VEC at a time, held by a thread: pack j is elements ((j * threads + thread) * VEC ...) of the row.
template <typename T, int VEC, int E>
struct NormPart {
    static constexpr int kPacks = E / VEC;
    Pack<T, VEC> raw[kPacks];
    __device__ __forceinline__ void load(const T *row, uint32_t at, uint32_t step, uint32_t d) {
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
            if (at + j * step < d) raw[j] = *reinterpret_cast<const Pack<T, VEC> *>(row + at + j * step);
    }
    __device__ __forceinline__ float get(int j, int e) const { return to_f32<T>(raw[j].v[e]); }
};

template <typename T>
__device__ __forceinline__ float param(const void *p, bool f32, uint32_t i) {
    return f32 ? static_cast<const float *>(p)[i] : to_f32<T>(static_cast<const T *>(p)[i]);
}

// The row's thread, its number of threads, and the rows that it comes to.
template <bool BLOCK>
struct NormPlace {
    uint32_t thread, threads;
    uint64_t row, step;
    __device__ __forceinline__ NormPlace() {
        threads = BLOCK ? blockDim.x : 32;
        thread = BLOCK ? threadIdx.x : threadIdx.x & 31;
        row = BLOCK ? blockIdx.x : uint64_t(blockIdx.x) * kNormWarpRows + (threadIdx.x >> 5);
        step = uint64_t(gridDim.x) * (BLOCK ? 1 : kNormWarpRows);
    }
};

template <typename T, int VEC, int E, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kNormMaxThreads : kNormWarpRows * 32) tcu_norm_forward_kernel(const NormParams p) {
    constexpr int kPacks = E / VEC;
    __shared__ float2 shared[2][32];
    const NormPlace<BLOCK> place;
    const uint32_t at = place.thread * VEC, step = place.threads * VEC;
    float weight[E], bias[E];
#pragma unroll
    for (int j = 0; j < kPacks; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const uint32_t i = at + j * step + e;
            weight[j * VEC + e] = i < p.d && p.weight ? param<T>(p.weight, p.param_f32, i) : 1.0f;
            bias[j * VEC + e] = i < p.d && p.bias ? param<T>(p.bias, p.param_f32, i) : 0.0f;
        }
    for (uint64_t row = place.row; row < p.rows; row += place.step) {
        NormPart<T, VEC, E> x;
        x.load(static_cast<const T *>(p.x) + row * p.x_stride, at, step, p.d);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (at + j * step < p.d) sum += x.get(j, e);
        const float first = sum_row<BLOCK>(sum, 0.0f, shared[0]).x * p.inv_d;
        float c = 0.0f, cc = 0.0f;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (at + j * step < p.d) {
                    const float v = x.get(j, e) - first;
                    c += v;
                    cc += v * v;
                }
        const float2 s = sum_row<BLOCK>(c, cc, shared[1]);
        const float more = s.x * p.inv_d, r = rsqrtf(fmaxf(s.y * p.inv_d - more * more, 0.0f) + p.eps);
        T *y = static_cast<T *>(p.y) + row * p.d;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
            if (at + j * step < p.d) {
                Pack<T, VEC> out;
#pragma unroll
                for (int e = 0; e < VEC; ++e) out.v[e] = from_f32<T>((x.get(j, e) - first - more) * r * weight[j * VEC + e] + bias[j * VEC + e]);
                *reinterpret_cast<Pack<T, VEC> *>(y + at + j * step) = out;
            }
    }
}

template <typename T, int VEC, int E, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? kNormMaxThreads : kNormWarpRows * 32) tcu_norm_backward_kernel(const NormParams p) {
    constexpr int kPacks = E / VEC;
    __shared__ float2 shared[3][32];
    const NormPlace<BLOCK> place;
    const uint32_t at = place.thread * VEC, step = place.threads * VEC;
    float weight[E], d_weight[E], d_bias[E];
#pragma unroll
    for (int j = 0; j < kPacks; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const uint32_t i = at + j * step + e;
            weight[j * VEC + e] = i < p.d && p.weight ? param<T>(p.weight, p.param_f32, i) : 1.0f;
            d_weight[j * VEC + e] = d_bias[j * VEC + e] = 0.0f;
        }
    for (uint64_t row = place.row; row < p.rows; row += place.step) {
        NormPart<T, VEC, E> x, d_y;
        x.load(static_cast<const T *>(p.x) + row * p.x_stride, at, step, p.d);
        d_y.load(static_cast<const T *>(p.d_y) + row * p.dy_stride, at, step, p.d);
        float sum = 0.0f, sum_e = 0.0f;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (at + j * step < p.d) {
                    sum += x.get(j, e);
                    sum_e += weight[j * VEC + e] * d_y.get(j, e);
                }
        const float2 firsts = sum_row<BLOCK>(sum, sum_e, shared[0]);
        const float first = firsts.x * p.inv_d;
        float c = 0.0f, cc = 0.0f, ec = 0.0f;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (at + j * step < p.d) {
                    const float v = x.get(j, e) - first;
                    c += v;
                    cc += v * v;
                    ec += weight[j * VEC + e] * d_y.get(j, e) * v;
                }
        const float2 s = sum_row<BLOCK>(c, cc, shared[1]);
        const float sum_ec = sum_row<BLOCK>(ec, 0.0f, shared[2]).x;
        const float more = s.x * p.inv_d, r = rsqrtf(fmaxf(s.y * p.inv_d - more * more, 0.0f) + p.eps);
        const float mean_e = firsts.y * p.inv_d, mean_eu = (sum_ec - more * firsts.y) * p.inv_d * r;
        T *d_x = static_cast<T *>(p.d_x) + row * p.d;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
            if (at + j * step < p.d) {
                Pack<T, VEC> out;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float dy = d_y.get(j, e), u = (x.get(j, e) - first - more) * r;
                    out.v[e] = from_f32<T>(r * (weight[j * VEC + e] * dy - mean_e - u * mean_eu));
                    d_weight[j * VEC + e] += dy * u;
                    d_bias[j * VEC + e] += dy;
                }
                if (p.d_x) *reinterpret_cast<Pack<T, VEC> *>(d_x + at + j * step) = out;
            }
    }
    if (!p.parts) return;
    float *parts = p.parts + uint64_t(blockIdx.x) * 2 * p.d;
    if constexpr (!BLOCK) {                // the block's warps add up theirs, one after another
        __shared__ float sums[2][32 * E];
        for (int w = 0; w < kNormWarpRows; ++w) {
            if (int(threadIdx.x >> 5) == w) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float *s = &sums[0][i * 32 + place.thread], *t = &sums[1][i * 32 + place.thread];
                    *s = w ? *s + d_weight[i] : d_weight[i];
                    *t = w ? *t + d_bias[i] : d_bias[i];
                }
            }
            __syncthreads();
        }
        if (threadIdx.x >= 32) return;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            d_weight[i] = sums[0][i * 32 + place.thread];
            d_bias[i] = sums[1][i * 32 + place.thread];
        }
    }
#pragma unroll
    for (int j = 0; j < kPacks; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const uint32_t i = at + j * step + e;
            if (i < p.d) {
                parts[i] = d_weight[j * VEC + e];
                parts[p.d + i] = d_bias[j * VEC + e];
            }
        }
}

// Adds the blocks' parts: 32 columns a block, 8 groups of rows of the parts.
template <typename P>
__global__ void __launch_bounds__(256) tcu_norm_join_kernel(const float *parts, uint32_t blocks, uint32_t d, P *d_weight, P *d_bias) {
    __shared__ float sums[8][33];
    begin_in_sequence();
    const uint32_t lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint32_t i = blockIdx.x * 32 + lane;         // of 2 d columns
    float sum = 0.0f;
    if (i < 2 * d)
        for (uint32_t b = group; b < blocks; b += 8) sum += parts[uint64_t(b) * 2 * d + i];
    sums[group][lane] = sum;
    __syncthreads();
    if (group == 0 && i < 2 * d) {
        for (int g = 1; g < 8; ++g) sum += sums[g][lane];
        if (i < d) {
            if (d_weight) d_weight[i] = from_f32<P>(sum);
        } else if (d_bias) {
            d_bias[i - d] = from_f32<P>(sum);
        }
    }
}

}  // namespace tcu
