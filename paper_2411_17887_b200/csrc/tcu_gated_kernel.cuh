// Gated linear recurrence: for every channel on its own, with f = sigmoid(gate),
//     h_t = f_t h_{t-1} + i_t x_t          i = 1 - f, 1 or sqrt(1 - f^2)
// an inclusive scan over pairs (f, b) with (f, b) before (f', b') giving (f f', f' b + b').  Its gradients are the same scan
// backward in time: with D_t the gradient with respect to h_t and C_t what flows into it from later tokens,
//     D_t = dy_t + C_t    C_{t-1} = f_t D_t    dx_t = i_t D_t    dgate_t = D_t (h_{t-1} f_t' + x_t i_t')
// where h is formed once more from the states that the forward pass leaves every kGatedTile tokens (marks).
//
// A block walks a sequence for 64 channels, a tile of kGatedTile tokens at a time: a warp takes kGatedSteps tokens of it, two
// channels a lane, and scans them in registers; the warps' pairs go through shared memory, and what arrives at a warp from
// before is added as P_t h (P the product of the f so far): every value is read and written once.
#pragma once

#include "tcu_float.cuh"

namespace tcu {

constexpr int kGatedSteps = 8;                           // tokens of a warp
constexpr int kGatedWarps = 8;
constexpr int kGatedTile = kGatedSteps * kGatedWarps;    // tokens of a tile, and between marks
constexpr int kGatedChannels = 64;

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
    float *marks;              // (tokens / kGatedTile + batch, channels): sequence b's begin at row first token / kGatedTile + b
    uint64_t tokens;           // of each sequence (dense), of all together (packed)
    uint32_t channels, strips;
};

// The two channels of a lane: one access where they are aligned for it (PAIR), else one each.
template <typename T, bool PAIR>
struct Two {
    Pack<T, 2> raw;
    __device__ __forceinline__ void load(const T *p, bool first, bool second) {
        if constexpr (PAIR) {
            if (first) raw = *reinterpret_cast<const Pack<T, 2> *>(p);
        } else {
            if (first) raw.v[0] = p[0];
            if (second) raw.v[1] = p[1];
        }
    }
    static __device__ __forceinline__ void store(T *p, float a, float b, bool first, bool second) {
        if constexpr (PAIR) {
            if (first) *reinterpret_cast<Pack<T, 2> *>(p) = Pack<T, 2>{{from_f32<T>(a), from_f32<T>(b)}};
        } else {
            if (first) p[0] = from_f32<T>(a);
            if (second) p[1] = from_f32<T>(b);
        }
    }
    __device__ __forceinline__ float get(int c) const { return to_f32<T>(raw.v[c]); }
};

// exp(-|g|) to a few 2^-23 of itself: 2^t for the rounded product t of -|g| and log2(e), and to first order what the rounding and the
// second half of log2(e) leave.
__device__ __forceinline__ float exp_minus(float g) {
    constexpr double kLog2e = 1.4426950408889634;
    constexpr float kHigh = float(kLog2e), kLow = float(kLog2e - double(kHigh));
    const float u = -fminf(fabsf(g), 200.0f);            // (below 2^-150 either way; infinities would leave inf - inf)
    const float t = u * kHigh, left = fmaf(u, kLow, fmaf(u, kHigh, -t));
    float a;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(t));
    return fmaf(a, left * 0.69314718f, a);
}

// f = sigmoid(g) and 1 - f.  The smaller of the two is a / (1 + a), a = exp(-|g|), to a few 2^-23 of itself, the larger one less it:
// f of a channel with a long memory is off by its rounding alone.
__device__ __forceinline__ void sigmoids(float g, float &f, float &rest) {
    const float a = exp_minus(g);
    const float less = __fdividef(a, 1.0f + a), more = 1.0f - less;
    const bool keep = g >= 0.0f;
    f = keep ? more : less;
    rest = keep ? less : more;
    if (g != g) f = rest = g;                            // (fminf drops a NaN)
}

template <int INPUT>
__device__ __forceinline__ float input_of(float f, float rest) {
    if constexpr (INPUT == kInputComplement) return rest;
    if constexpr (INPUT == kInputOne) return 1.0f;
    float i;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(i) : "f"(rest * (1.0f + f)));
    return i;
}

// Derivative of the input's factor by the gate.
template <int INPUT>
__device__ __forceinline__ float input_slope(float f, float rest, float i) {
    if constexpr (INPUT == kInputComplement) return -f * rest;
    if constexpr (INPUT == kInputOne) return 0.0f;
    return -f * f * __fdividef(i, 1.0f + f);
}

// One block's place: sequence, channels, tokens.
struct GatedWalk {
    uint32_t seq, c0;
    int64_t begin, len;        // of the sequence, in rows of the arrays (packed) or of its own (dense: begin 0)
    uint64_t mark;             // row of its first mark
    __device__ __forceinline__ GatedWalk(const GatedParams &p, uint32_t walk) {
        seq = walk / p.strips;
        c0 = (walk - seq * p.strips) * kGatedChannels;
        if (p.offsets) {
            // offsets that are not as they should be may give wrong results, but no access outside the arrays
            begin = min(max(p.offsets[seq], int64_t(0)), int64_t(p.tokens));
            len = min(max(p.offsets[seq + 1], begin), int64_t(p.tokens)) - begin;
            mark = uint64_t(begin) / kGatedTile + seq;
        } else {
            begin = 0;
            len = int64_t(p.tokens);
            mark = uint64_t(seq) * p.tokens / kGatedTile + seq;
        }
    }
    template <typename T>
    __device__ __forceinline__ T *at(const GatedParams &p, const GatedRows &r, uint32_t c) const {
        return static_cast<T *>(r.ptr) + (p.offsets ? begin * r.token : int64_t(seq) * r.batch) + c;
    }
};

template <typename T, int INPUT, bool PAIR>
__global__ void __launch_bounds__(kGatedWarps * 32) tcu_gated_forward_kernel(const GatedParams p) {
    __shared__ float4 pairs[2][kGatedWarps][32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GatedWalk w(p, blockIdx.x);
    const uint32_t c = w.c0 + 2 * lane;
    const bool c0 = c < p.channels, c1 = c + 1 < p.channels;
    const T *px = w.at<T>(p, p.x, c), *pg = w.at<T>(p, p.gate, c);
    T *py = p.y.ptr ? w.at<T>(p, p.y, c) : nullptr;
    float h[2] = {0.0f, 0.0f};
    const uint64_t st = uint64_t(w.seq) * p.channels + c;
    if (p.state_in) {
        if (c0) h[0] = p.state_in[st];
        if (c1) h[1] = p.state_in[st + 1];
    }
    uint32_t buf = 0;
    for (int64_t t0 = 0; t0 < w.len; t0 += kGatedTile, buf ^= 1) {
        const int64_t t = t0 + warp * kGatedSteps;
        const int n = int(min(int64_t(kGatedSteps), w.len - t));          // tokens of this warp, or none
        Two<T, PAIR> x[kGatedSteps], g[kGatedSteps];
#pragma unroll
        for (int s = 0; s < kGatedSteps; ++s) {
            x[s].load(px + (t + s) * p.x.token, s < n && c0, s < n && c1);
            g[s].load(pg + (t + s) * p.gate.token, s < n && c0, s < n && c1);
        }
        if (p.marks && warp == 0) {
            float *m = p.marks + (w.mark + uint64_t(t0) / kGatedTile) * p.channels + c;
            if (c0) m[0] = h[0];
            if (c1) m[1] = h[1];
        }
        float prod[kGatedSteps][2], local[kGatedSteps][2], a[2] = {1.0f, 1.0f}, b[2] = {0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < kGatedSteps; ++s) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (s < n) {
                    float f, rest;
                    sigmoids(g[s].get(e), f, rest);
                    a[e] *= f;
                    b[e] = f * b[e] + input_of<INPUT>(f, rest) * x[s].get(e);
                }
                prod[s][e] = a[e];
                local[s][e] = b[e];
            }
        }
        pairs[buf][warp][lane] = make_float4(a[0], b[0], a[1], b[1]);
        __syncthreads();
        float mine[2] = {h[0], h[1]};
#pragma unroll
        for (uint32_t k = 0; k < kGatedWarps; ++k) {
            const float4 q = pairs[buf][k][lane];
            if (k == warp) mine[0] = h[0], mine[1] = h[1];
            h[0] = q.x * h[0] + q.y;
            h[1] = q.z * h[1] + q.w;
        }
        if (py) {
#pragma unroll
            for (int s = 0; s < kGatedSteps; ++s)
                Two<T, PAIR>::store(py + (t + s) * p.y.token, prod[s][0] * mine[0] + local[s][0], prod[s][1] * mine[1] + local[s][1], s < n && c0, s < n && c1);
        }
    }
    if (p.state_out && warp == 0) {
        if (c0) p.state_out[st] = h[0];
        if (c1) p.state_out[st + 1] = h[1];
    }
}

template <typename T, int INPUT, bool PAIR>
__global__ void __launch_bounds__(kGatedWarps * 32) tcu_gated_backward_kernel(const GatedParams p) {
    __shared__ float4 ahead[2][kGatedWarps][32], back[2][kGatedWarps][32];
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const GatedWalk w(p, blockIdx.x);
    const uint32_t c = w.c0 + 2 * lane;
    const bool c0 = c < p.channels, c1 = c + 1 < p.channels;
    const T *px = w.at<T>(p, p.x, c), *pg = w.at<T>(p, p.gate, c), *pd = w.at<T>(p, p.d_y, c);
    T *pdx = w.at<T>(p, p.d_x, c), *pdg = w.at<T>(p, p.d_gate, c);
    float flow[2] = {0.0f, 0.0f};                                          // C at the end of the tile
    const uint64_t st = uint64_t(w.seq) * p.channels + c;
    if (p.d_state_out) {
        if (c0) flow[0] = p.d_state_out[st];
        if (c1) flow[1] = p.d_state_out[st + 1];
    }
    uint32_t buf = 0;
    const int64_t tiles = (w.len + kGatedTile - 1) / kGatedTile;
    for (int64_t tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
        const int64_t t = tile * kGatedTile + warp * kGatedSteps;
        const int n = int(min(int64_t(kGatedSteps), w.len - t));
        Two<T, PAIR> x[kGatedSteps], g[kGatedSteps], d[kGatedSteps];
#pragma unroll
        for (int s = 0; s < kGatedSteps; ++s) {
            x[s].load(px + (t + s) * p.x.token, s < n && c0, s < n && c1);
            g[s].load(pg + (t + s) * p.gate.token, s < n && c0, s < n && c1);
            d[s].load(pd + (t + s) * p.d_y.token, s < n && c0, s < n && c1);
        }
        float h[2] = {0.0f, 0.0f};
        const float *m = p.marks + (w.mark + tile) * p.channels + c;
        if (c0) h[0] = m[0];
        if (c1) h[1] = m[1];
        float f[kGatedSteps][2], rest[kGatedSteps][2], a[2] = {1.0f, 1.0f}, b[2] = {0.0f, 0.0f}, r[2] = {0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < kGatedSteps; ++s) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                if (s < n) {
                    sigmoids(g[s].get(e), f[s][e], rest[s][e]);
                    a[e] *= f[s][e];
                    b[e] = f[s][e] * b[e] + input_of<INPUT>(f[s][e], rest[s][e]) * x[s].get(e);
                }
            }
        }
#pragma unroll
        for (int s = kGatedSteps - 1; s >= 0; --s) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (s < n) r[e] = f[s][e] * (r[e] + d[s].get(e));
        }
        ahead[buf][warp][lane] = make_float4(a[0], b[0], a[1], b[1]);
        back[buf][warp][lane] = make_float4(a[0], r[0], a[1], r[1]);
        __syncthreads();
        for (uint32_t k = 0; k < warp; ++k) {
            const float4 q = ahead[buf][k][lane];
            h[0] = q.x * h[0] + q.y;
            h[1] = q.z * h[1] + q.w;
        }
        float mine[2] = {flow[0], flow[1]};
#pragma unroll
        for (int k = kGatedWarps - 1; k >= 0; --k) {
            const float4 q = back[buf][k][lane];
            if (uint32_t(k) == warp) mine[0] = flow[0], mine[1] = flow[1];
            flow[0] = q.x * flow[0] + q.y;
            flow[1] = q.z * flow[1] + q.w;
        }
        float before[kGatedSteps][2];
#pragma unroll
        for (int s = 0; s < kGatedSteps; ++s) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                before[s][e] = h[e];
                if (s < n) h[e] = f[s][e] * h[e] + input_of<INPUT>(f[s][e], rest[s][e]) * x[s].get(e);
            }
        }
#pragma unroll
        for (int s = kGatedSteps - 1; s >= 0; --s) {
            float dx[2], dg[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                dx[e] = dg[e] = 0.0f;
                if (s < n) {
                    const float grad = d[s].get(e) + mine[e], ff = f[s][e], i = input_of<INPUT>(ff, rest[s][e]);
                    dx[e] = i * grad;
                    dg[e] = grad * (before[s][e] * (ff * rest[s][e]) + x[s].get(e) * input_slope<INPUT>(ff, rest[s][e], i));
                    mine[e] = ff * grad;
                }
            }
            Two<T, PAIR>::store(pdx + (t + s) * p.d_x.token, dx[0], dx[1], s < n && c0, s < n && c1);
            Two<T, PAIR>::store(pdg + (t + s) * p.d_gate.token, dg[0], dg[1], s < n && c0, s < n && c1);
        }
    }
    if (p.d_state_in && warp == 0) {
        if (c0) p.d_state_in[st] = flow[0];
        if (c1) p.d_state_in[st + 1] = flow[1];
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
    float f, rest;
    sigmoids(to_f32<T>(static_cast<const T *>(p.gate.ptr)[int64_t(seq) * p.gate.batch + c]), f, rest);
    const float h = f * *state + input_of<INPUT>(f, rest) * to_f32<T>(static_cast<const T *>(p.x.ptr)[int64_t(seq) * p.x.batch + c]);
    *state = h;
    *y = from_f32<T>(h);
}

}  // namespace tcu
