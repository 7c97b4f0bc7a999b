// Layer norm over the last axis, y = weight (x - mean) r + bias with r = 1 / sqrt(variance + eps), and its gradients: with
// u = (x - mean) r and e = weight dy,
//     dx = r (e - mean(e) - u mean(e u))        dweight = sum over rows of dy u        dbias = sum over rows of dy
// A row is held in registers, 16 elements a thread, by some lanes of a warp, a warp or a block, so that x (and dy) is read once; mean and
// variance are those of the values less a first mean, which takes what rounding of the first mean leaves out again.  A block goes through rows
// in steps of the grid - those of 16 bits, 16 elements a thread, with the next two on their way to shared memory, others with the next one on its way to registers forward and
// none backward - and adds up its part of the parameters' gradients in registers; a second
// kernel adds the blocks' parts, in order.
//
// What bounds it: forward instructions (18 an element, a quarter of them the sums over a row), close behind memory; backward (29) neither: issue slots are used in 63 % of
// the cycles, DRAM for 52 %, and of 5.7 cycles an instruction a warp waits 1.3 for shared memory and lanes, with 14 warps an SM.  32749 rows of 2048 bfloat16
// values: forward 50 us (268 MB, 5.4 TB/s, 0.82 of the copy rate), backward 91 us (402 MB, 4.4 TB/s, the joining kernel 4 us of it).  fp32: 89 and 140 us (536 and 805 MB).
// Above 8192 columns a thread holds 32 elements, which do not fit its registers: 4096 rows of 12288 bfloat16 values 81 and 149 us.
#pragma once

#include "tcu_float.cuh"

namespace tcu {

constexpr int kNormWarps = 8;              // of a block, where a warp holds one row or several
constexpr int kNormThreads = 512;          // at most, where a block holds a row: 128 registers each
// Rows in shared memory of a thread, one that it works on and the others on their way, where it holds `bytes` of each: 16 elements of 16 bits (0: none, more are too many
// for three rows of two arrays).
__host__ __device__ constexpr int norm_ahead(int bytes) { return bytes <= 32 ? 3 : 0; }

struct NormParams {
    const void *x, *d_y, *weight, *bias;
    void *y, *d_x;
    float *parts;              // (blocks, 2, d): sums of dy u and of dy
    uint64_t x_stride, dy_stride;
    uint32_t rows, d;
    int param_f32;             // weight and bias are fp32, else of the type of x
    float eps, inv_d;
};

// Sums of N values over groups of LANES lanes.  The values share the steps: at each of the first ones a lane gives half of its
// values for the other half of its partner's, so that N values cost little more than one.
template <int N, int LANES>
__device__ __forceinline__ void sum_lanes(float (&v)[N]) {
    const uint32_t lane = threadIdx.x & 31;
    if constexpr (N == 1) {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) v[0] += __shfl_xor_sync(~0u, v[0], o);
    } else {
        static_assert(N == 2 || N == 4, "a power of two");
        const bool high = lane & LANES / 2;
        float half[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) half[i] = (high ? v[i + N / 2] : v[i]) + __shfl_xor_sync(~0u, high ? v[i] : v[i + N / 2], LANES / 2);
        if constexpr (N == 4) {
            const bool odd = lane & LANES / 4;
            half[0] = (odd ? half[1] : half[0]) + __shfl_xor_sync(~0u, odd ? half[0] : half[1], LANES / 4);
        }
#pragma unroll
        for (int o = LANES / (N * 2); o > 0; o >>= 1) half[0] += __shfl_xor_sync(~0u, half[0], o);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(~0u, half[0], i * (LANES / N), LANES);
    }
}
// Sums over a row's threads: LANES lanes, or (0) a block.
// shared: N x 32 floats, of which those of warps that the block does not have are zero.
template <int N, int LANES>
__device__ __forceinline__ void sum_row(float (&v)[N], float *shared) {
    sum_lanes<N, LANES ? LANES : 32>(v);
    if constexpr (LANES == 0) {
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) shared[i * 32 + warp] = v[i];
        }
        __syncthreads();
        if (warps <= 8) {                  // four warps' sums a read
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float4 q = *reinterpret_cast<const float4 *>(shared + i * 32);
                v[i] = (q.x + q.y) + (q.z + q.w);
                if (warps > 4) {
                    const float4 s = *reinterpret_cast<const float4 *>(shared + i * 32 + 4);
                    v[i] += (s.x + s.y) + (s.z + s.w);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = shared[i * 32 + lane];
            sum_lanes<N, 32>(v);
        }
    }
}

// E elements of a row, VEC at a time, held by a thread: pack j is elements ((j * threads + thread) * VEC ...) of the row.
template <typename T, int VEC, int E>
struct NormPart {
    static constexpr int kPacks = E / VEC;
    Pack<T, VEC> raw[kPacks];
    __device__ __forceinline__ float get(int j, int e) const {
        if constexpr (VEC == 1) return to_f32<T>(raw[j].v[e]);
        const float2 two = two_f32<T>(*reinterpret_cast<const Pack<T, 2> *>(&raw[j].v[e & ~1]));
        return e & 1 ? two.y : two.x;
    }
};

// The row's thread, its number of threads, and the rows that it comes to.  (The groups of a warp go through as many rounds each, as they add
// up together: a row past the last one is read as the last one, and not written.)
template <int LANES>
struct NormPlace {
    uint32_t thread, threads, row, step, rounds;
    __device__ __forceinline__ NormPlace(uint32_t rows) {
        constexpr uint32_t kGroups = LANES ? 32 / LANES : 1;
        threads = LANES ? LANES : blockDim.x;
        thread = LANES ? threadIdx.x % threads : threadIdx.x;
        const uint32_t first = LANES ? (blockIdx.x * kNormWarps + (threadIdx.x >> 5)) * kGroups : blockIdx.x;
        row = first + (LANES ? (threadIdx.x & 31) / threads : 0);
        step = gridDim.x * (LANES ? kNormWarps * kGroups : 1);
        rounds = first < rows ? (rows - first - 1) / step + 1 : 0;
    }
};

// The rows of an array that a thread comes to, some of them on their way to shared memory while it works on one: every thread copies, and reads,
// its own elements, so that nobody waits for anybody.  Elements that cannot be copied 16 bytes at a time, or are too many, are read
// one row ahead into registers (forward), or when they are needed (backward, which has none left).  FULL: every thread has all its elements.
template <typename T, int VEC, int E, bool FULL>
struct NormAhead {
    static constexpr int kPacks = E / VEC;
    static constexpr int kRows = sizeof(Pack<T, VEC>) == 16 ? norm_ahead(E * int(sizeof(T))) : 0;
    static constexpr bool kShared = kRows > 0;
    Pack<T, VEC> *slots;                   // (kRows, packs, threads of the block)
    const T *from;                         // this thread's first element of the next row
    uint64_t stride;                       // to the one after it
    uint32_t after;                        // rows of this thread after it
    template <int LANES>
    __device__ __forceinline__ NormAhead(Pack<T, VEC> *slots, const void *array, const NormPlace<LANES> &place, uint32_t rows, uint64_t row_stride, uint32_t at)
        : slots(slots + threadIdx.x), from(static_cast<const T *>(array) + uint64_t(min(place.row, rows - 1)) * row_stride + at), stride(place.step * row_stride),
          after(place.row < rows ? (rows - 1 - place.row) / place.step : 0) {}
    __device__ __forceinline__ void next() {
        if (after > 0) {
            from += stride;
            --after;
        }
    }
    __device__ __forceinline__ void ask(uint32_t stage, uint32_t at, uint32_t step, uint32_t d) {
#pragma unroll
        for (int j = 0; j < kPacks; ++j) {
            if (FULL || at + j * step < d)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(uint32_t(__cvta_generic_to_shared(slots + (stage * kPacks + j) * blockDim.x))),
                             "l"(from + j * step) : "memory");
        }
        next();
    }
    __device__ __forceinline__ NormPart<T, VEC, E> take(uint32_t stage, uint32_t at, uint32_t step, uint32_t d) {
        NormPart<T, VEC, E> part;
#pragma unroll
        for (int j = 0; j < kPacks; ++j) {
            if constexpr (kShared) part.raw[j] = slots[(stage * kPacks + j) * blockDim.x];
            else if (FULL || at + j * step < d) part.raw[j] = *reinterpret_cast<const Pack<T, VEC> *>(from + j * step);
        }
        if constexpr (!kShared) next();
        return part;
    }
};

template <typename T, int VEC>
__device__ __forceinline__ void round_pack(Pack<T, VEC> &out, const float *v) {
    if constexpr (VEC == 1) {
        out.v[0] = from_f32<T>(v[0]);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) *reinterpret_cast<Pack<T, 2> *>(&out.v[e]) = two_from_f32<T>(v[e], v[e + 1]);
    }
}

template <typename T>
__device__ __forceinline__ float param(const void *p, bool f32, uint32_t i) {
    return f32 ? static_cast<const float *>(p)[i] : to_f32<T>(static_cast<const T *>(p)[i]);
}

template <typename T, int VEC, int E, int LANES, bool FULL>
__global__ void __launch_bounds__(LANES ? kNormWarps * 32 : kNormThreads) tcu_norm_forward_kernel(const NormParams p) {
    constexpr int kPacks = E / VEC;
    __shared__ __align__(16) float sums[2][32 * 2];
    for (uint32_t i = threadIdx.x; i < sizeof(sums) / 4; i += blockDim.x) sums[0][i] = 0.0f;
    __syncthreads();
    const NormPlace<LANES> place(p.rows);
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
    extern __shared__ __align__(16) uint8_t rows[];
    using Ahead = NormAhead<T, VEC, E, FULL>;
    constexpr uint32_t kRows = Ahead::kShared ? Ahead::kRows : 1;
    Ahead x_ahead(reinterpret_cast<Pack<T, VEC> *>(rows), p.x, place, p.rows, p.x_stride, at);
    uint32_t left = place.rounds, asked = left, stage = 0;       // rows
    uint32_t row = place.row;
    auto ask = [&](uint32_t to) {
        if constexpr (Ahead::kShared) {
            if (asked > 0) {
                x_ahead.ask(to, at, step, p.d);
                --asked;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    for (uint32_t k = 0; k + 1 < kRows; ++k) ask(k);
    NormPart<T, VEC, E> next;              // without shared memory: on its way to registers
    if (!Ahead::kShared && left > 0) next = x_ahead.take(0, at, step, p.d);
    T *y = static_cast<T *>(p.y) + uint64_t(place.row) * p.d + at;
    for (; left > 0; --left, row += place.step, y += uint64_t(place.step) * p.d) {
        if constexpr (Ahead::kShared) asm volatile("cp.async.wait_group %0;" ::"n"(int(kRows) - 2) : "memory");
        NormPart<T, VEC, E> x;
        if constexpr (Ahead::kShared) {
            x = x_ahead.take(stage, at, step, p.d);
        } else {
            x = next;
            if (left > 1) next = x_ahead.take(0, at, step, p.d);
        }
        ask(stage == 0 ? kRows - 1 : stage - 1);
        stage = stage + 1 == kRows ? 0 : stage + 1;
        float sum[1] = {0.0f}, v[E];
#pragma unroll
        for (int j = 0; j < kPacks; ++j) {
            if (FULL || at + j * step < p.d) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[j * VEC + e] = x.get(j, e);
                    sum[0] += v[j * VEC + e];
                }
            }
        }
        sum_row<1, LANES>(sum, sums[0]);
        const float first = sum[0] * p.inv_d;
        float c[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kPacks; ++j) {
            if (FULL || at + j * step < p.d) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float &w = v[j * VEC + e];
                    w -= first;
                    c[0] += w;
                    c[1] = fmaf(w, w, c[1]);
                }
            }
        }
        sum_row<2, LANES>(c, sums[1]);
        const float more = c[0] * p.inv_d, r = rsqrtf(fmaxf(c[1] * p.inv_d - more * more, 0.0f) + p.eps);
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
            if ((FULL || at + j * step < p.d) && (LANES % 32 == 0 || row < p.rows)) {
                Pack<T, VEC> out;
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[j * VEC + e] = fmaf((v[j * VEC + e] - more) * r, weight[j * VEC + e], bias[j * VEC + e]);
                round_pack(out, v + j * VEC);
                *reinterpret_cast<Pack<T, VEC> *>(y + j * step) = out;
            }
    }
}

template <typename T, int VEC, int E, int LANES, bool FULL>
__global__ void __launch_bounds__(LANES ? kNormWarps * 32 : kNormThreads) tcu_norm_backward_kernel(const NormParams p) {
    constexpr int kPacks = E / VEC;
    __shared__ __align__(16) float sums[32 * 2 + 32 * 4];
    for (uint32_t i = threadIdx.x; i < sizeof(sums) / 4; i += blockDim.x) sums[i] = 0.0f;
    __syncthreads();
    const NormPlace<LANES> place(p.rows);
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
    extern __shared__ __align__(16) uint8_t rows[];
    using Ahead = NormAhead<T, VEC, E, FULL>;
    constexpr uint32_t kRows = Ahead::kShared ? Ahead::kRows : 1;
    Ahead x_ahead(reinterpret_cast<Pack<T, VEC> *>(rows), p.x, place, p.rows, p.x_stride, at);
    Ahead d_ahead(reinterpret_cast<Pack<T, VEC> *>(rows) + Ahead::kRows * kPacks * blockDim.x, p.d_y, place, p.rows, p.dy_stride, at);
    uint32_t left = place.rounds, asked = left, stage = 0;       // rows
    uint32_t row = place.row;
    auto ask = [&](uint32_t to) {
        if constexpr (Ahead::kShared) {
            if (asked > 0) {
                x_ahead.ask(to, at, step, p.d);
                d_ahead.ask(to, at, step, p.d);
                --asked;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    for (uint32_t k = 0; k + 1 < kRows; ++k) ask(k);
    T *d_x = static_cast<T *>(p.d_x) + uint64_t(place.row) * p.d + at;
    for (; left > 0; --left, row += place.step, d_x += uint64_t(place.step) * p.d) {
        if constexpr (Ahead::kShared) asm volatile("cp.async.wait_group %0;" ::"n"(int(kRows) - 2) : "memory");
        const NormPart<T, VEC, E> x = x_ahead.take(stage, at, step, p.d), d_y = d_ahead.take(stage, at, step, p.d);
        ask(stage == 0 ? kRows - 1 : stage - 1);
        stage = stage + 1 == kRows ? 0 : stage + 1;
        float first[2] = {0.0f, 0.0f};                     // sums of x and of e
#pragma unroll
        for (int j = 0; j < kPacks; ++j) {
            if (FULL || at + j * step < p.d) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    first[0] += x.get(j, e);
                    first[1] = fmaf(weight[j * VEC + e], d_y.get(j, e), first[1]);
                }
            }
        }
        sum_row<2, LANES>(first, sums);
        const float mean = first[0] * p.inv_d;
        float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};             // of the values less the first mean, their squares, and their products with e
#pragma unroll
        for (int j = 0; j < kPacks; ++j) {
            if (FULL || at + j * step < p.d) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float v = x.get(j, e) - mean;
                    c[0] += v;
                    c[1] = fmaf(v, v, c[1]);
                    c[2] = fmaf(weight[j * VEC + e] * d_y.get(j, e), v, c[2]);
                }
            }
        }
        sum_row<4, LANES>(c, sums + 32 * 2);
        const float more = c[0] * p.inv_d, r = rsqrtf(fmaxf(c[1] * p.inv_d - more * more, 0.0f) + p.eps);
        const float mean_e = first[1] * p.inv_d, mean_eu = (c[2] - more * first[1]) * p.inv_d * r;
#pragma unroll
        for (int j = 0; j < kPacks; ++j)
            if ((FULL || at + j * step < p.d) && (LANES % 32 == 0 || row < p.rows)) {
                Pack<T, VEC> out;
                float rounded[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float dy = d_y.get(j, e), u = ((x.get(j, e) - mean) - more) * r;
                    rounded[e] = r * fmaf(-u, mean_eu, fmaf(weight[j * VEC + e], dy, -mean_e));
                    d_weight[j * VEC + e] = fmaf(dy, u, d_weight[j * VEC + e]);
                    d_bias[j * VEC + e] += dy;
                }
                round_pack(out, rounded);
                if (p.d_x) *reinterpret_cast<Pack<T, VEC> *>(d_x + j * step) = out;
            }
    }
    if (!p.parts) return;
    float *parts = p.parts + uint64_t(blockIdx.x) * 2 * p.d;
    if constexpr (LANES > 0) {             // the groups of a warp add up theirs, then the block's warps, one after another
        __shared__ float added[2][LANES * E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
#pragma unroll
            for (int o = LANES; o < 32; o <<= 1) {
                d_weight[i] += __shfl_xor_sync(~0u, d_weight[i], o);
                d_bias[i] += __shfl_xor_sync(~0u, d_bias[i], o);
            }
        }
        for (int w = 0; w < kNormWarps; ++w) {
            if (int(threadIdx.x >> 5) == w && (threadIdx.x & 31) < LANES) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    float *s = &added[0][i * LANES + place.thread], *t = &added[1][i * LANES + place.thread];
                    *s = w ? *s + d_weight[i] : d_weight[i];
                    *t = w ? *t + d_bias[i] : d_bias[i];
                }
            }
            __syncthreads();
        }
        if (threadIdx.x >= LANES) return;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            d_weight[i] = added[0][i * LANES + place.thread];
            d_bias[i] = added[1][i * LANES + place.thread];
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

// Adds the blocks' parts: 32 columns a block, 32 groups of rows of the parts.
template <typename P>
__global__ void __launch_bounds__(1024) tcu_norm_join_kernel(const float *parts, uint32_t blocks, uint32_t d, P *d_weight, P *d_bias) {
    __shared__ float sums[32][33];
    begin_in_sequence();
    const uint32_t lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const uint32_t i = blockIdx.x * 32 + lane;         // of 2 d columns
    float sum = 0.0f;
    if (i < 2 * d) {
#pragma unroll 4
        for (uint32_t b = group; b < blocks; b += 32) sum += parts[uint64_t(b) * 2 * d + i];
    }
    sums[group][lane] = sum;
    __syncthreads();
    sum = sums[lane][group];                           // of column `group` now
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    const uint32_t column = blockIdx.x * 32 + group;
    if (lane == 0 && column < 2 * d) {
        if (column < d) {
            if (d_weight) d_weight[column] = from_f32<P>(sum);
        } else if (d_bias) {
            d_bias[column - d] = from_f32<P>(sum);
        }
    }
}

}  // namespace tcu
