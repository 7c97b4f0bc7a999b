// Sampling of one token for each row of logits.  With m the largest logit of the row, every token has the weight
// w = exp((logit - m) / temperature).  In the order of falling logits, the lower token first among equals, the tokens kept are the
// first top_k, as far as w >= min_p, and of these the fewest whose weights add up to top_p times the weight of them all: a
// prefix of that order, so that it is told by its last logit and how many of the tokens with that one belong to it.  The token
// drawn is the first, in the order of tokens, up to and with which the kept weights add up to more than u times their sum.
//
// A row is read once, into the shared memory of a cluster of blocks, a part each: a warp holds consecutive tokens, so that the sums of warps and
// blocks, which tell each other theirs, are those of ranges of tokens.  Without limits a block's weights are relative to its own largest
// logit, and the blocks meet once.  The last kept logit is looked for among candidates, up to 512, which are listed and sorted: for top_k
// the tokens from the k-th of the largest logits of 64 ranges a block on (there are k of these at least), or those in the bin that a histogram
// of numbers names; for top_p the largest few hundred, found the same way, if they have the weight, or those in the bin that a histogram of weights names.  That one is of 32-bit weights, and sums of 64-bit ones say whether the
// bin is right.  Where a bin has more tokens, exact histograms of the logit's bits as an integer follow, 9 bits a time.
//
// Sums that decide which token it is are exact enough that it is the token of the definition, off its borders: weights in 64-bit floating point, in exact
// histograms in fixed point with 42 bits (three limbs of 14, each sum of at most 2^18 tokens within 32 bits), whose sums do not depend on their order.
// A weight is off by 1.3e-12 of itself (what its series leaves out), in fixed point by 2^-43 of the largest one of a bin, whose weights are at least exp(-1/64)
// of it (but in the last bin, 32 or more below the top: by less than 1e-21 in all): a quotient of two sums is off by less than 4e-12.
//
// What bounds it: instructions, 48 a token, 12 of them 64-bit arithmetic (issued in 73 % of the cycles of an SM with work; bank conflicts, those of the table, take 12 % of
// them in a shared memory that is busy for 37 %), and, with limits, the times that the blocks of a row have to meet.  256 rows of 128000 bfloat16 logits, a few of them far above the others
// (66 MB, 10 us to read): largest logit alone 28 us, temperature 75, top_k 50 58, top_p 0.9 107 (388 where it keeps 30000 tokens).  192 rows of 50001 fp32 logits:
// 18, 44, 33 and 51; top_p 0.99 at temperature 1.2, some ten thousand tokens, 145.  Tried: weights in all histograms in three limbs (top_p 284 us), logits in
// registers (they spill), weights by exp() (whole rows 203 us), all candidates sorted by every block for itself (top_k 128).
#pragma once

#include <cooperative_groups.h>

#include <type_traits>

#include "tcu_float.cuh"

namespace tcu {

constexpr int kSampleThreads = 256;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleBins = 2048, kSampleFineBits = 9, kSampleFine = 1 << kSampleFineBits;      // of a first histogram, and of those that follow
constexpr int kSampleMaxCluster = 8;
constexpr int kSampleList = 512;                      // candidates that are sorted, two a thread
constexpr int kSampleRanges = 64;                     // of a block: four lanes' tokens each
constexpr uint32_t kMostVocabulary = 1u << 18;
constexpr double kSampleFixed = 4398046511104.0;      // 2^42
constexpr int kSampleLimb = 14;
static_assert(kSampleList == 2 * kSampleThreads && kSampleRanges == 2 * 32, "two candidates each thread, two ranges each lane of a warp");

// A setting of all rows, or one for each.
template <typename T>
struct Setting {
    const T *each;
    double all;
    __device__ __forceinline__ double at(uint32_t row) const { return each ? double(each[row]) : all; }
};

struct SampleParams {
    const void *logits;
    uint64_t stride;
    uint32_t vocabulary;
    int packs;                 // 16-byte packs of a thread
    const void *uniform;
    int uniform_f64;
    Setting<float> temperature, top_p, min_p;
    Setting<int32_t> top_k;
    int64_t *tokens;
    float *log_probs;
};

// What the blocks of a cluster tell one another.
struct SampleWord {
    double a;
    uint32_t b, c;
};

struct SampleFound {
    int bin;                               // or -1
    uint64_t before, in;                   // sums ahead of the bin, of the bin
};

struct SampleShared {
    double table[32];                      // 2^(j/32)
    SampleWord slots[2][kSampleMaxCluster];
    SampleFound found[2];
    double warp_sum[kSampleWarps];
    uint64_t warp_u64[kSampleWarps];
    uint32_t warp_u32[2][kSampleWarps], warp_ties[kSampleWarps];
    float warp_max[kSampleWarps];
    uint32_t count;                        // of this block's candidates
    uint32_t counts[kSampleMaxCluster];    // of all blocks'
    uint2 list[kSampleList];               // their keys and tokens
    uint32_t ranges[kSampleRanges];        // keys of the largest logits of its ranges
    uint32_t all_ranges[kSampleMaxCluster * kSampleRanges];
    float from_k;
    union {
        uint32_t hist[kSampleBins];        // or three limbs of kSampleFine bins
        struct {
            uint64_t sorted[kSampleList];                  // all blocks' candidates, in falling order: candidate()
            uint64_t order[kSampleList];                   // those kept, in the order of tokens
        };
    };
};

__device__ __forceinline__ uint32_t sample_key(float v) {        // the order of logits as that of unsigned integers
    const uint32_t b = __float_as_uint(v);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sample_value(uint32_t key) {
    return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

constexpr uint32_t kKeyNothing = 0x007fffffu;                    // that of minus infinity

// NaN as minus infinity, no zero below zero.
__device__ __forceinline__ float sane(float v) { return fmaxf(v, -INFINITY) + 0.0f; }
template <typename T, int VEC>
__device__ __forceinline__ void sane_pack(Pack<T, VEC> &p) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.v[e] = sane(p.v[e]);
    } else if constexpr (std::is_same_v<T, __half>) {
        __half2 *two = reinterpret_cast<__half2 *>(p.v);
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) two[e] = __hadd2(__hmax2(two[e], __float2half2_rn(-INFINITY)), __float2half2_rn(0.0f));
    } else {
        __nv_bfloat162 *two = reinterpret_cast<__nv_bfloat162 *>(p.v);
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) two[e] = __hadd2(__hmax2(two[e], __float2bfloat162_rn(-INFINITY)), __float2bfloat162_rn(0.0f));
    }
}

template <typename T>
struct Sampler {
    static constexpr int kVec = 16 / sizeof(T);
    using Packed = Pack<T, kVec>;
    const SampleParams &p;
    SampleShared &s;
    Packed *held;                          // this thread's tokens, at(j) on, in steps of kSampleThreads; minus infinity where there are none
    cooperative_groups::cluster_group cluster;
    uint32_t rank, ranks, phase = 0, found_phase = 0, row;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int first;                             // token of the block's first element
    float top = 0.0f;                      // what weights are relative to
    double inverse = 1.0, parts = 1.0;         // 1 / temperature; 32 log2(e) / temperature

    __device__ Sampler(const SampleParams &p, SampleShared &s, void *held) : p(p), s(s), held(static_cast<Packed *>(held) + threadIdx.x), cluster(cooperative_groups::this_cluster()) {
        rank = cluster.block_rank();
        ranks = cluster.num_blocks();
        row = blockIdx.x / ranks;
    }
    __device__ __forceinline__ int at(int j) const { return first + ((int(warp) * p.packs + j) * 32 + int(lane)) * kVec; }
    // f(logit) for this thread's tokens.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
        for (int j = 0; j < p.packs; ++j) {
            const Packed q = held[j * kSampleThreads];
#pragma unroll
            for (int e = 0; e < kVec; ++e) f(to_f32<T>(q.v[e]));
        }
    }

    // exp((x - top) / temperature), by table (P. T. P. Tang, 1989): with y = 32 log2(e) (x - top) / temperature = k + r, k the nearest integer,
    // 2^(y/32) = 2^floor(k/32) 2^(k mod 32 / 32) exp(q), q = r ln 2 / 32 below 0.011: what the series leaves out is below 1.3e-12 of it.  (A table of 64
    // needs no shorter series, and twice the time to be read.)  Zero below 2^-1000; exactly 1 for the top itself.
    __device__ __forceinline__ double weight(float x) const {
        const double y = (double(x) - double(top)) * parts;
        constexpr double kMagic = 6755399441055744.0, kLn = 0.69314718055994530942 / 32;
        const double t = y + kMagic;
        const int k = __double2loint(t);
        const double r = y - (t - kMagic), m = s.table[k & 31];
        double poly = fma(r, kLn * kLn * kLn * kLn / 24, kLn * kLn * kLn / 6);
        poly = fma(r, poly, kLn * kLn / 2);
        poly = fma(r, poly, kLn);
        const double w = fma(m, r * poly, m);
        const bool far = uint32_t(__double2hiint(y)) > 0xC0DF4000u;                            // y below -32000
        return far ? 0.0 : __hiloint2double(__double2hiint(w) + (k >> 5) * 1048576, __double2loint(w));
    }
    __device__ __forceinline__ uint64_t fixed(float x) const { return uint64_t(__double2ll_rn(weight(x) * kSampleFixed)); }
    __device__ __forceinline__ void set_temperature(double temperature) {
        inverse = fmin(fmax(1.0 / temperature, 1e-300), 1e300);      // (0, or infinity, times nothing, or infinity, would be no number)
        parts = inverse * (32 * 1.4426950408889634074);
    }

    // Every block's word, at every block.  All threads call it; what is told has to be ready in thread 0's to kSampleMaxCluster - 1's `mine`.
    __device__ const SampleWord *exchange(const SampleWord &mine) {
        SampleWord *slots = s.slots[phase];
        phase ^= 1;
        if (threadIdx.x < ranks) cluster.map_shared_rank(slots, threadIdx.x)[rank] = mine;
        cluster.sync();
        return slots;
    }

    // The block's largest logit, from the threads'; s.ranges holds the keys of its ranges' (0 for one without a token).
    __device__ float block_max(float x) {
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, o));
        if (lane % 4 == 0) s.ranges[warp * 8 + lane / 4] = x > -INFINITY ? sample_key(x) : 0;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, o));
        if (lane == 0) s.warp_max[warp] = x;
        __syncthreads();
        x = s.warp_max[lane & (kSampleWarps - 1)];
#pragma unroll
        for (int o = kSampleWarps / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, o));
        return x;
    }
    // The least of all threads' values, of two at once.
    __device__ uint2 block_min(uint32_t a, uint32_t b) {
        a = __reduce_min_sync(~0u, a);
        b = __reduce_min_sync(~0u, b);
        __syncthreads();
        if (lane == 0) s.warp_u32[0][warp] = a, s.warp_u32[1][warp] = b;
        __syncthreads();
        return make_uint2(__reduce_min_sync(~0u, s.warp_u32[0][lane & (kSampleWarps - 1)]), __reduce_min_sync(~0u, s.warp_u32[1][lane & (kSampleWarps - 1)]));
    }
    __device__ uint2 cluster_min(uint32_t a, uint32_t b) {
        const uint2 mine = block_min(a, b);
        const SampleWord *w = exchange({0.0, mine.x, mine.y});
        uint2 least = make_uint2(w[0].b, w[0].c);
        for (uint32_t k = 1; k < ranks; ++k) least = make_uint2(min(least.x, w[k].b), min(least.y, w[k].c));
        return least;
    }
    // The sum of all threads' values, warp after warp; s.warp_sum holds the warps' sums.
    __device__ double block_sum(double x) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
        __syncthreads();
        if (lane == 0) s.warp_sum[warp] = x;
        __syncthreads();
        double sum = 0.0;
        for (int k = 0; k < kSampleWarps; ++k) sum += s.warp_sum[k];
        return sum;
    }
    // Two sums at once.
    __device__ double2 block_sums(double x, double y) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            x += __shfl_xor_sync(~0u, x, o);
            y += __shfl_xor_sync(~0u, y, o);
        }
        __syncthreads();
        if (lane == 0) {
            s.warp_sum[warp] = x;
            s.warp_u64[warp] = uint64_t(__double_as_longlong(y));
        }
        __syncthreads();
        double2 sum = make_double2(0.0, 0.0);
        for (int k = 0; k < kSampleWarps; ++k) {
            sum.x += s.warp_sum[k];
            sum.y += __longlong_as_double(int64_t(s.warp_u64[k]));
        }
        return sum;
    }
    template <typename Keep>
    __device__ double thread_sum(Keep keep) const {            // of the weights of the tokens that are kept
        double sum[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
        for (int j = 0; j < p.packs; ++j) {
            const Packed q = held[j * kSampleThreads];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float x = to_f32<T>(q.v[e]);
                if (keep(x)) sum[e & 3] += weight(x);
            }
        }
        return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }

    // Reads the block's part of the row (addresses in steps of 16 bytes, whatever the row begins at); the thread's largest logit.
    __device__ float load() {
        const T *from = static_cast<const T *>(p.logits) + uint64_t(row) * p.stride;
        first = int(rank * kSampleThreads * p.packs * kVec) - int(reinterpret_cast<uintptr_t>(from) % 16 / sizeof(T));   // (what lies ahead of the row on its first 16 bytes)
        if (threadIdx.x < 32) s.table[threadIdx.x] = exp2(threadIdx.x / 32.0);
        float most = -INFINITY;
#pragma unroll 4
        for (int j = 0; j < p.packs; ++j) {
            const int token = at(j);
            Packed q;
            if (token >= 0 && token + kVec <= int(p.vocabulary)) {
                q = *reinterpret_cast<const Packed *>(from + token);
            } else {
#pragma unroll
                for (int e = 0; e < kVec; ++e) q.v[e] = token + e >= 0 && token + e < int(p.vocabulary) ? from[token + e] : from_f32<T>(-INFINITY);
            }
            sane_pack<T, kVec>(q);
            held[j * kSampleThreads] = q;
#pragma unroll
            for (int e = 0; e < kVec; ++e) most = fmaxf(most, to_f32<T>(q.v[e]));
        }
        return most;
    }
    // An infinite logit leaves no weight to any other: it becomes 0, the others minus infinity.
    __device__ void only_infinite() {
        for (int j = 0; j < p.packs; ++j)
            for (int e = 0; e < kVec; ++e) {
                T &x = held[j * kSampleThreads].v[e];
                x = from_f32<T>(to_f32<T>(x) == INFINITY ? 0.0f : -INFINITY);
            }
    }

    // Histogram over the row's tokens of bin_of (below 0: not counted) - LIMBS 1: of what(logit); 3: of exact weights, in limbs - and the first
    // bin with which the sum reaches `target`.
    template <int LIMBS, int BINS, typename BinOf, typename What>
    __device__ SampleFound histogram(BinOf bin_of, What what, double target) {
        static_assert(LIMBS * BINS <= kSampleBins, "in shared memory");
        SampleFound *found = &s.found[found_phase];
        found_phase ^= 1;
        for (uint32_t b = threadIdx.x; b < LIMBS * BINS; b += kSampleThreads) s.hist[b] = 0;
        if (threadIdx.x == 0) found->bin = -1;
        __syncthreads();
        each([&](float x) {
            const int b = bin_of(x);
            if (b >= 0) {
                if constexpr (LIMBS == 3) {
                    const uint64_t w = fixed(x);
                    atomicAdd(&s.hist[b], uint32_t(w) & ((1u << kSampleLimb) - 1));
                    atomicAdd(&s.hist[BINS + b], uint32_t(w >> kSampleLimb) & ((1u << kSampleLimb) - 1));
                    atomicAdd(&s.hist[2 * BINS + b], uint32_t(w >> (2 * kSampleLimb)));
                } else {
                    atomicAdd(&s.hist[b], what(x));
                }
            }
        });
        cluster.sync();
        // this block's share of the bins, a few each thread
        const uint32_t share = BINS / ranks, each_thread = (share + kSampleThreads - 1) / kSampleThreads;
        const uint32_t own = rank * share + threadIdx.x * each_thread;
        const bool some = threadIdx.x * each_thread < share;
        uint64_t mine[BINS / kSampleThreads], sum = 0;
#pragma unroll
        for (uint32_t j = 0; j < BINS / kSampleThreads; ++j) mine[j] = 0;
        if (some) {
#pragma unroll
            for (uint32_t k = 0; k < kSampleMaxCluster; ++k) {           // (unrolled: all blocks' bins are on their way at once)
                if (k < ranks) {
                    const auto *h = cluster.map_shared_rank(s.hist, k) + own;
#pragma unroll
                    for (uint32_t j = 0; j < BINS / kSampleThreads; ++j)
                        if (j < each_thread) {
                            mine[j] += h[j];
                            if constexpr (LIMBS == 3) mine[j] += (uint64_t(h[BINS + j]) << kSampleLimb) + (uint64_t(h[2 * BINS + j]) << (2 * kSampleLimb));
                        }
                }
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < BINS / kSampleThreads; ++j) sum += mine[j];
        uint64_t upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t q = __shfl_up_sync(~0u, upto, o);
            if (lane >= uint32_t(o)) upto += q;
        }
        if (lane == 31) s.warp_u64[warp] = upto;
        __syncthreads();
        uint64_t ahead = upto - sum, all = 0;
        for (uint32_t k = 0; k < kSampleWarps; ++k) {
            if (k < warp) ahead += s.warp_u64[k];
            all += s.warp_u64[k];
        }
        const SampleWord *w = exchange({__longlong_as_double(int64_t(all)), 0, 0});
        for (uint32_t k = 0; k < rank; ++k) ahead += uint64_t(__double_as_longlong(w[k].a));
#pragma unroll
        for (uint32_t j = 0; j < BINS / kSampleThreads; ++j) {
            if (mine[j] && double(ahead) < target && double(ahead + mine[j]) >= target) {
                const SampleFound f = {int(own + j), ahead, mine[j]};
                for (uint32_t k = 0; k < ranks; ++k) *cluster.map_shared_rank(found, k) = f;
            }
            ahead += mine[j];
        }
        cluster.sync();
        return *found;
    }

    // A prefix of the falling order: the tokens above `edge`, and those of it - all (whole), or the first `ties`.
    struct Prefix {
        float edge;
        uint32_t ties;
        bool whole;
    };

    // Where a logit lies in the first histogram, linear in it: 64 bins to a factor of e in weight.
    __device__ __forceinline__ int bin(float x, float cut, float scale) const {
        return x < cut ? -1 : x == top ? 0 : int(fminf((top - x) * scale, float(kSampleBins - 1)));
    }

    // The prefix of the tokens from `cut` on that reaches a number of them.  False: there are fewer.
    __device__ bool reach_number(float cut, double k, Prefix &out) {
        const float scale = float(fmin(inverse * 64.0, 1e37));
        const SampleFound f = histogram<1, kSampleBins>([&](float x) { return bin(x, cut, scale); }, [](float) { return 1u; }, k);
        if (f.bin < 0) return false;
        out = in_bin<false>(cut, scale, f.bin, k - double(f.before));
        return true;
    }
    // The same for a weight, of `sum` of all that is looked at.
    __device__ bool reach_weight(float cut, double target, double sum, Prefix &out) {
        const float scale = float(fmin(inverse * 64.0, 1e37));
        // weights to about 2^-22, as parts of 2^30 of the sum
        const float to_part = float(1073741824.0 / sum), octaves = float(fmin(inverse * 1.4426950408889634, 1e37));
        const SampleFound f = histogram<1, kSampleBins>(
            [&](float x) { return bin(x, cut, scale); },
            [&](float x) {
                float w;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(fmaxf((x - top) * octaves, -1000.0f)));
                return uint32_t(__float2uint_rn(w * to_part));
            },
            target / sum * 1073741824.0);
        int at = f.bin < 0 ? bin(cut, cut, scale) : f.bin, turn = 0;
        for (;;) {
            // the sums ahead of the bin and of it; the next bins on either side that have a token
            double ahead[2] = {0.0, 0.0}, of_bin[2] = {0.0, 0.0};
            uint32_t below = ~0u, above = ~0u;
#pragma unroll 1
            for (int j = 0; j < p.packs; ++j) {
                const Packed q = held[j * kSampleThreads];
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const float x = to_f32<T>(q.v[e]);
                    const int b = bin(x, cut, scale);
                    if (b >= 0) {
                        if (b <= at) {
                            const double w = weight(x);
                            if (b < at) ahead[e & 1] += w;
                            else of_bin[e & 1] += w;
                        }
                        if (b < at) below = min(below, uint32_t(at - b));
                        if (b > at) above = min(above, uint32_t(b - at));
                    }
                }
            }
            const double2 here = block_sums(ahead[0] + ahead[1], of_bin[0] + of_bin[1]);
            const SampleWord *w = exchange({here.x, uint32_t(__double2hiint(here.y)), uint32_t(__double2loint(here.y))});
            double before = 0.0, in = 0.0;
            for (uint32_t k = 0; k < ranks; ++k) {
                before += w[k].a;
                in += __hiloint2double(int(w[k].b), int(w[k].c));
            }
            // (the bin is left in one direction only: sums that are the same but for rounding must not send it back)
            const bool down = before >= target && turn <= 0, up = before + in < target && before < target && turn >= 0;
            if (!down && !up) {
                out = in_bin<true>(cut, scale, at, fmax(target - before, 0.0));
                return true;
            }
            const uint2 next = cluster_min(below, above);
            const uint32_t by = down ? next.x : next.y;
            if (by == ~0u) return false;                     // (rounding leaves less than the target)
            turn = down ? -1 : 1;
            at += turn * int(by);
        }
    }
    // The prefix that ends in a bin: with `left` of its tokens' number, or weight.  Weights that are too many to be sorted are added up as parts of the bin's largest
    // one: 42 bits of the row's would leave a light token few (one of 1e-8, 15 of them, and of 2^18 equal ones an error of one sign: 3e-8 in all).
    template <bool WEIGHTS>
    __device__ Prefix in_bin(float cut, float scale, int which, double left) {
        const uint32_t total = list_candidates([&](float x) { return bin(x, cut, scale) == which; });
        if (total <= kSampleList) {
            sort_candidates(total);
            const Prefix out = prefix_of(total, WEIGHTS ? reach_sorted(total, 1.0, left) : uint32_t(fmin(left, double(total))));
            cluster.sync();                                  // (nobody lists others before all have read these)
            return out;
        }
        uint32_t lo = ~0u, hi_not = ~0u;                     // keys of the bin: from lo to ~hi_not
        each([&](float x) {
            if (bin(x, cut, scale) == which) {
                lo = min(lo, sample_key(x));
                hi_not = min(hi_not, ~sample_key(x));
            }
        });
        const uint2 ends = cluster_min(lo, hi_not);
        lo = ends.x;
        uint32_t hi = ~ends.y;
        const float of_row = top;
        double before = 0.0, one = 1.0, target = left, many = 1.0;
        if (WEIGHTS) {
            const double largest = weight(sample_value(hi));
            top = sample_value(hi);
            target = largest > 0.0 ? fmax(left / largest * kSampleFixed, 0.5) : 0.5;      // (less than any weight counts for: at least the first token)
        }
        do {
            const int bits = 32 - __clz(int(hi - lo)), shift = bits > kSampleFineBits ? bits - kSampleFineBits : 0;
            auto bin_of = [&](float x) {
                const uint32_t key = sample_key(x);
                return key < lo || key > hi ? -1 : int((hi - key) >> shift);
            };
            const SampleFound g = histogram<WEIGHTS ? 3 : 1, kSampleFine>(bin_of, [](float) { return 1u; }, target - before);
            if (g.bin < 0) {                                 // (rounding: the last of them)
                if (shift == 0) hi = lo;
                else hi = lo + ((hi - lo) & ((1u << shift) - 1));
            } else {
                before += double(g.before);
                hi -= uint32_t(g.bin) << shift;
                lo = max(lo, hi - ((1u << shift) - 1));
            }
            one = WEIGHTS ? double(fixed(sample_value(hi))) : 1.0;
            many = one > 0.0 ? double(g.bin < 0 ? 1 : g.in) / one : 1.0;
        } while (lo < hi);
        top = of_row;
        const uint32_t most = uint32_t(fmax(rint(many), 1.0)), ties = uint32_t(fewest(before, one, target, most));
        return {sample_value(hi), ties, ties >= most};
    }
    // The least c from 1 to `many` with before + c one >= target.
    __device__ static uint64_t fewest(double before, double one, double target, uint64_t many) {
        if (!(one > 0.0)) return 1;
        uint64_t c = uint64_t(fmin(fmax(ceil((target - before) / one), 1.0), double(many)));
        while (c > 1 && before + double(c - 1) * one >= target) --c;
        while (c < many && before + double(c) * one < target) ++c;
        return c;
    }

    // Lists this block's candidates, in any order, and tells how many the row has of them, or that they are more than kSampleList.
    template <typename Is>
    __device__ uint32_t list_candidates(Is is) {
        if (threadIdx.x == 0) s.count = 0;
        __syncthreads();
#pragma unroll 1
        for (int j = 0; j < p.packs; ++j) {
            const Packed q = held[j * kSampleThreads];
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (is(to_f32<T>(q.v[e]))) list_one(to_f32<T>(q.v[e]), at(j) + e);
        }
        __syncthreads();
        return count_candidates(0.0, 0.0f, nullptr, nullptr);
    }
    __device__ __forceinline__ void list_one(float x, int token) {
        if (*const_cast<volatile uint32_t *>(&s.count) > kSampleList) return;                // too many: no more need to be counted
        const uint32_t to = atomicAdd(&s.count, 1u);
        if (to < kSampleList) s.list[to] = make_uint2(sample_key(x), uint32_t(token));
    }
    // The row's number of candidates, and its sums of two values, the second to 2^-22.
    __device__ uint32_t count_candidates(double a, float b, double *sum_a, float *sum_b) {
        const SampleWord *w = exchange({a, s.count, __float_as_uint(b)});
        if (threadIdx.x < ranks) s.counts[threadIdx.x] = w[threadIdx.x].b;
        __syncthreads();
        uint32_t total = 0;
        for (uint32_t k = 0; k < ranks; ++k) total += w[k].b;
        if (sum_a) {
            *sum_a = 0.0;
            *sum_b = 0.0f;
            for (uint32_t k = 0; k < ranks; ++k) {
                *sum_a += w[k].a;
                *sum_b += __uint_as_float(w[k].c);
            }
        }
        return total;
    }

    // A candidate as a number: in rising order the logits fall, the lower token first among equals.  Or, for the order of tokens, turned around.
    static __device__ __forceinline__ uint64_t candidate(uint32_t key, uint32_t token) { return uint64_t(~key) << 32 | token; }
    static __device__ __forceinline__ uint64_t turned(uint64_t v) { return v << 32 | v >> 32; }
    static __device__ __forceinline__ float logit_of(uint64_t v) { return sample_value(~uint32_t(v >> 32)); }

    // Sorts the first `total` of a list (of kSampleList, two a thread), rising.  Few of them (a thread each) by counting those ahead of each: 25 steps of
    // reading four for a hundred.  More by a bitonic network over the next power of two, whose steps of up to 32 stay within a warp's 64 elements.
    __device__ void sort(uint64_t *list, uint32_t total) {
        __syncthreads();
        if (total <= 160) {
            const uint64_t mine = threadIdx.x < total ? list[threadIdx.x] : 0;
            uint32_t before = 0;
            if (threadIdx.x < total) {
                uint32_t k = 0;
                for (; k + 4 <= total; k += 4) before += (list[k] < mine) + (list[k + 1] < mine) + (list[k + 2] < mine) + (list[k + 3] < mine);
                for (; k < total; ++k) before += list[k] < mine;
            }
            __syncthreads();
            if (threadIdx.x < total) list[before] = mine;
            __syncthreads();
            return;
        }
        uint32_t n = 64;
        while (n < total) n *= 2;
        for (uint32_t i = threadIdx.x; i < n; i += kSampleThreads)
            if (i >= total) list[i] = ~0ull;
        __syncthreads();
        const bool works = 2 * threadIdx.x < n;
        for (uint32_t size = 2; size <= n; size *= 2) {
            for (uint32_t step = size / 2; step > 0; step /= 2) {
                if (works) {
                    const uint32_t low = 2 * threadIdx.x - (threadIdx.x & (step - 1)), high = low + step;
                    const uint64_t x = list[low], y = list[high];
                    if ((x > y) == ((low & size) == 0)) {
                        list[low] = y;
                        list[high] = x;
                    }
                }
                if (step > 32 || (step == 1 && size >= 64)) __syncthreads();       // (what follows reaches, or has come from, other warps' elements)
                else __syncwarp();
            }
        }
        __syncthreads();
    }
    // All blocks' `total` candidates (no more than kSampleList) to s.sorted.
    __device__ void sort_candidates(uint32_t total) {
        for (uint32_t i = threadIdx.x; i < total; i += kSampleThreads) {
            uint32_t k = 0, from = i;
            while (from >= s.counts[k]) from -= s.counts[k++];
            const uint2 q = cluster.map_shared_rank(s.list, k)[from];
            s.sorted[i] = candidate(q.x, q.y);
        }
        sort(s.sorted, total);
    }
    // This thread's two of the first m of a list, 2 i and 2 i + 1: their weights, and the sums up to them.
    struct Two {
        double w[2], upto[2], all;
    };
    template <bool TURNED>
    __device__ Two two_of(const uint64_t *list, uint32_t m) {
        Two two;
#pragma unroll
        for (uint32_t e = 0; e < 2; ++e) {
            const uint32_t i = 2 * threadIdx.x + e;
            two.w[e] = i < m ? weight(logit_of(TURNED ? turned(list[i]) : list[i])) : 0.0;
        }
        two.upto[1] = block_prefix(two.w[0] + two.w[1], two.all);
        two.upto[0] = two.upto[1] - two.w[1];
        return two;
    }
    // How many of the first `most` sorted candidates it takes until their weights reach the target (below 0: top_p of theirs).
    __device__ uint32_t reach_sorted(uint32_t most, double top_p, double target) {
        const Two two = two_of<false>(s.sorted, most);
        if (target < 0.0) target = top_p * two.all;
        const uint32_t i = 2 * threadIdx.x;
        return min(most, block_min(i < most && two.upto[0] >= target ? i : i + 1 < most && two.upto[1] >= target ? i + 1 : most - 1, 0).x + 1);
    }
    // The sum of the threads' values up to each thread's, and of all.
    __device__ double block_prefix(double x, double &all) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double q = __shfl_up_sync(~0u, x, o);
            if (lane >= uint32_t(o)) x += q;
        }
        __syncthreads();
        if (lane == 31) s.warp_sum[warp] = x;
        __syncthreads();
        double ahead = 0.0;
        all = 0.0;
        for (uint32_t k = 0; k < kSampleWarps; ++k) {
            if (k == warp) ahead = all;
            all += s.warp_sum[k];
        }
        return ahead + x;
    }
    // The prefix of the first m of `total` sorted candidates, which hold all tokens of their last one's logit.
    __device__ Prefix prefix_of(uint32_t total, uint32_t m) {
        const uint32_t key = uint32_t(s.sorted[m - 1] >> 32);
        uint32_t mine = ~0u;
        for (uint32_t i = threadIdx.x; i < total && mine == ~0u; i += kSampleThreads)
            if (uint32_t(s.sorted[i] >> 32) == key) mine = i;
        const uint32_t above = block_min(mine, 0).x;         // the first with this key
        return {sample_value(~key), m - above, m >= total || uint32_t(s.sorted[m] >> 32) != key};
    }
    // Draws from candidates that hold all tokens to be kept: the first `most` of them, and of these those that reach the target.  By one block; the
    // others lend it their lists.
    __device__ void draw_listed(uint32_t total, uint32_t most, double top_p, double target) {
        if (rank == 0) {
            sort_candidates(total);
            const uint32_t m = top_p < 1.0 ? reach_sorted(most, top_p, target) : most;
            // in the order of tokens
            for (uint32_t i = threadIdx.x; i < m; i += kSampleThreads) s.order[i] = turned(s.sorted[i]);
            sort(s.order, m);
            const Two two = two_of<true>(s.order, m);
            const double target_u = uniform() * two.all;
            const uint32_t i = 2 * threadIdx.x;
            // the first past the target; the last one with a weight, if rounding leaves none
            const uint32_t past = two.w[0] > 0.0 && two.upto[0] > target_u ? i : two.w[1] > 0.0 && two.upto[1] > target_u ? i + 1 : ~0u;
            const uint2 found = block_min(past, two.w[1] > 0.0 ? ~(i + 1) : two.w[0] > 0.0 ? ~i : ~0u);
            const uint32_t at = found.x != ~0u ? found.x : ~found.y;
            if (threadIdx.x == 0) put_drawn(int64_t(s.order[at] >> 32), logit_of(turned(s.order[at])), top, two.all);
        }
        cluster.sync();
    }

    // The least logit whose weight is at least min_p.
    __device__ float least_value(double min_p) {
        uint64_t lo = sample_key(-3.402823466e38f), hi = sample_key(top);             // hi has weight 1
        // 32 neighbours of where it should be, then, if it is not among them, 32 keys at a time
        const float guess = float(double(top) + log(min_p) / inverse);
        const uint64_t near = sample_key(fminf(fmaxf(guess, -3.402823466e38f), top));
        const uint64_t begin = near > lo + 16 ? near - 16 : lo, key = begin + lane;
        uint32_t in = __ballot_sync(~0u, key >= hi || weight(sample_value(uint32_t(key))) >= min_p);
        if (in && (!(in & 1u) || begin == lo)) return sample_value(uint32_t(min(begin + __ffs(int(in)) - 1, hi)));
        while (lo < hi) {
            const uint64_t step = (hi - lo + 31) / 32, at = lo + step * lane;
            in = __ballot_sync(~0u, at < hi && weight(sample_value(uint32_t(at))) >= min_p);
            // of the keys looked at, those from the first that is in on are in
            const uint32_t looked = __popc(__ballot_sync(~0u, at < hi)), f = in ? uint32_t(__ffs(int(in)) - 1) : looked;
            if (f < looked) hi = lo + step * f;
            if (f > 0) lo += step * (f - 1) + 1;
        }
        return sample_value(uint32_t(hi));
    }

    __device__ __forceinline__ void put(int64_t token, float log_prob) {
        p.tokens[row] = token;
        if (p.log_probs) p.log_probs[row] = log_prob;
    }
    __device__ __forceinline__ void put_drawn(int64_t token, float x, double largest, double sum) {
        put(token, float((double(x) - largest) * inverse - log(sum)));
    }

    __device__ void run() {
        cluster_begin();
        const double temperature = p.temperature.at(row), min_p = p.min_p.at(row), top_p = p.top_p.at(row), k = p.top_k.at(row);
        const float of_block = block_max(load());
        cluster_begun();
        const bool limited_k = k > 0.0 && k < double(p.vocabulary), limited_m = min_p > 0.0, limited_p = top_p < 1.0;
        if (!(temperature > 0.0) || k == 1.0 || min_p > 1.0 || top_p <= 0.0) return greedy(of_block);
        set_temperature(temperature);
        if (!limited_k && !limited_m && !limited_p) return whole(of_block);

        for (uint32_t r = threadIdx.x / kSampleRanges; r < ranks; r += kSampleThreads / kSampleRanges)        // its ranges, to all blocks
            cluster.map_shared_rank(s.all_ranges, r)[rank * kSampleRanges + threadIdx.x % kSampleRanges] = s.ranges[threadIdx.x % kSampleRanges];
        const SampleWord *w = exchange({double(of_block), 0, 0});
        top = float(w[0].a);
        for (uint32_t r = 1; r < ranks; ++r) top = fmaxf(top, float(w[r].a));
        if (top == -INFINITY) {
            if (rank == 0 && threadIdx.x == 0) put(-1, -INFINITY);
            return;
        }
        // from here on lie at least k tokens (for top_p alone: so many that most of them can be sorted)
        float from_k = top < INFINITY && (limited_k || limited_p) ? from_ranges(limited_k ? k : most_ranges()) : -INFINITY;
        if (top == INFINITY) {
            only_infinite();
            top = 0.0f;
        }
        const float low = limited_m ? least_value(min_p) : -3.402823466e38f;         // tokens below have less than min_p, or no weight
        Prefix kept = {low, 0, true};
        if (limited_k) {
            const float cut = fmaxf(low, from_k);
            if (limited_m || from_k > -INFINITY || p.vocabulary <= kSampleList) {          // (else they are too many)
                const uint32_t total = list_candidates([&](float x) { return x >= cut; });
                if (total <= kSampleList) return draw_listed(total, uint32_t(fmin(k, double(total))), top_p, -1.0);
            }
            reach_number(cut, k, kept);                      // (or there are fewer than k from `low` on: all of them)
        } else if (limited_m) {
            const uint32_t total = list_candidates([&](float x) { return x >= low; });
            if (total <= kSampleList) return draw_listed(total, total, top_p, -1.0);
        }
        if (limited_p) {
            // what top_k and min_p leave: the tokens above the edge (from the edge on), and so many of it
            const float from = kept.whole ? kept.edge : sample_value(sample_key(kept.edge) + 1);
            // their weight, and that of the largest ones, which are listed
            const float cut_list = from_k > -INFINITY || p.vocabulary <= kSampleList ? fmaxf(from, from_k) : INFINITY;
            double sums[2] = {0.0, 0.0}, large = 0.0, sum;
            float sum_large;
            if (threadIdx.x == 0) s.count = 0;
            __syncthreads();
#pragma unroll 1
            for (int j = 0; j < p.packs; ++j) {
                const Packed q = held[j * kSampleThreads];
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const float x = to_f32<T>(q.v[e]);
                    if (x >= from) {
                        const double weighs = weight(x);
                        sums[e & 1] += weighs;
                        if (x >= cut_list) {
                            large += weighs;
                            list_one(x, at(j) + e);
                        }
                    }
                }
            }
            const double2 here = block_sums(sums[0] + sums[1], large);
            const uint32_t total = count_candidates(here.x, float(here.y), &sum, &sum_large);
            const double at_edge = kept.whole ? 0.0 : weight(kept.edge), target = top_p * (sum + kept.ties * at_edge);
            if (!kept.whole && sum < target) {               // it ends within the edge
                kept.ties = uint32_t(fewest(sum, at_edge, target, kept.ties));
            } else if (total <= kSampleList && sum_large >= target * (1.0 + 1e-5)) {
                return draw_listed(total, total, top_p, target);
            } else {
                // all tokens below (1 - top_p) of the mean weight together do not make up what may be left out
                float cut = float(double(top) + log((1.0 - top_p) * sum / p.vocabulary) / inverse);
                cut -= 1e-5f * fabsf(cut) + 1e-5f / float(fmin(inverse, 1e37));                // (below it, whatever the rounding)
                cut = cut == cut ? fminf(fmaxf(cut, from), top) : from;
                reach_weight(cut, target, sum, kept);
            }
        }
        draw(kept);
    }

    // So many of the ranges' largest logits that about 130 tokens lie from the last of them on: n ranges of tokens in no order have none of m
    // tokens for a part exp(-m / n) of them.
    __device__ double most_ranges() const {
        const double n = ranks * kSampleRanges;
        return fmax(floor(n - n * exp(-130.0 / n)), 1.0);
    }
    // A logit from which on at least k tokens lie, from the largest logits of the row's ranges: by their keys' upper half; minus infinity if there are
    // fewer ranges.
    __device__ float from_ranges(double k) {
        const uint32_t n = ranks * kSampleRanges;
        if (k > n) return -INFINITY;
        if (warp == 0) {
            uint32_t mine[2 * kSampleMaxCluster];
#pragma unroll
            for (uint32_t r = 0; r < 2 * kSampleMaxCluster; ++r) mine[r] = r < 2 * ranks ? s.all_ranges[r * 32 + lane] >> 16 : 0;
            uint32_t from = 0;
            for (uint32_t bit = 1u << 15; bit; bit >>= 1) {
                uint32_t count = 0;
#pragma unroll
                for (uint32_t r = 0; r < 2 * kSampleMaxCluster; ++r) count += mine[r] >= (from | bit);
                if (double(__reduce_add_sync(~0u, count)) >= k) from |= bit;
            }
            if (lane == 0) s.from_k = from ? sample_value(max(from << 16, kKeyNothing + 1)) : -INFINITY;
        }
        __syncthreads();
        return s.from_k;
    }

    // The lowest token among those with the largest logit.
    __device__ void greedy(float of_block) {
        uint32_t token = ~0u;
#pragma unroll 1
        for (int j = 0; j < p.packs; ++j) {
            const Packed q = held[j * kSampleThreads];
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (to_f32<T>(q.v[e]) == of_block) token = min(token, uint32_t(at(j) + e));
        }
        const uint32_t lowest = block_min(token, 0).x;
        const SampleWord *w = exchange({double(of_block), lowest, 0});
        uint32_t best = 0;
        for (uint32_t k = 1; k < ranks; ++k)
            if (w[k].a > w[best].a) best = k;
        if (rank == 0 && threadIdx.x == 0) {
            if (w[best].a == -INFINITY) put(-1, -INFINITY);
            else put(w[best].b, 0.0f);
        }
    }

    // Without limits: weights relative to the block's own largest logit.
    __device__ void whole(float of_block) {
        top = of_block;
        if (top == INFINITY) {
            only_infinite();
            top = 0.0f;
        }
        const double sum = top == -INFINITY ? 0.0 : block_sum(thread_sum([](float) { return true; }));
        const SampleWord *w = exchange({sum, __float_as_uint(of_block), 0});
        float largest = -INFINITY;
        for (uint32_t k = 0; k < ranks; ++k) largest = fmaxf(largest, __uint_as_float(w[k].b));
        if (largest == -INFINITY) {
            if (rank == 0 && threadIdx.x == 0) put(-1, -INFINITY);
            return;
        }
        const float own = top;
        top = largest == INFINITY ? 0.0f : largest;
        // lane k: what block k adds, relative to the row's largest
        const float m = __uint_as_float(w[lane % ranks].b);
        const double scale = m == -INFINITY || (largest == INFINITY && m < INFINITY) ? 0.0 : m == largest ? 1.0 : weight(m);
        const Place place = place_of(lane < ranks ? w[lane % ranks].a * scale : 0.0);
        if (place.who != rank) return;
        const double largest_weighed = top;
        top = own;
        find({-3.402823466e38f, 0, true}, 0, 0.0, (place.target - place.before) / __shfl_sync(~0u, scale, place.who), place.total, largest_weighed);
    }

    // Where a random number lies among the lanes' sums: the first lane with which they pass it (the last one that adds anything, if rounding
    // leaves none), and what the lanes before it add up to.
    struct Place {
        uint32_t who;
        double before, target, total;
    };
    __device__ Place place_of(double add) const {
        double upto = add;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double q = __shfl_up_sync(~0u, upto, o);
            if (lane >= uint32_t(o)) upto += q;
        }
        Place place;
        place.total = __shfl_sync(~0u, upto, 31);
        place.target = uniform() * place.total;
        const uint32_t over = __ballot_sync(~0u, add > 0.0 && upto > place.target), any = __ballot_sync(~0u, add > 0.0);
        place.who = over ? __ffs(int(over)) - 1 : any ? 31 - __clz(int(any)) : 0;
        place.before = __shfl_sync(~0u, upto - add, place.who);
        return place;
    }

    __device__ __forceinline__ double uniform() const {
        const double u = p.uniform_f64 ? static_cast<const double *>(p.uniform)[row] : double(static_cast<const float *>(p.uniform)[row]);
        return u > 0.0 ? u : 0.0;
    }

    // Draws from a prefix.
    __device__ void draw(const Prefix &kept) {
        uint32_t ties = 0;
        if (!kept.whole) {
            each([&](float x) { ties += x == kept.edge; });
            ties = __reduce_add_sync(~0u, ties);
        }
        const double at_edge = kept.whole ? 0.0 : weight(kept.edge);
        const double sum = block_sum(thread_sum([&](float x) { return kept.whole ? x >= kept.edge : x > kept.edge; }));
        if (lane == 0) s.warp_ties[warp] = ties;
        __syncthreads();
        uint32_t here = 0;
        for (int k = 0; k < kSampleWarps; ++k) here += s.warp_ties[k];
        const SampleWord *w = exchange({sum, here, 0});
        // lane k: what block k adds, with those of the edge's tokens that belong to the prefix
        const uint32_t tied = lane < ranks ? w[lane].b : 0;
        uint32_t upto = tied;
#pragma unroll
        for (int o = 1; o < kSampleMaxCluster; o <<= 1) {
            const uint32_t q = __shfl_up_sync(~0u, upto, o);
            if (lane >= uint32_t(o)) upto += q;
        }
        const Place place = place_of(lane < ranks ? with_edge(kept, w[lane].a, upto - tied, tied, at_edge) : 0.0);
        const uint32_t ties_before = __shfl_sync(~0u, upto - tied, place.who);
        if (place.who == rank) find(kept, ties_before, at_edge, place.target - place.before, place.total, top);
    }
    // A sum with those of the edge's `here` tokens that belong to the prefix, `before` of them lying ahead.
    __device__ __forceinline__ static double with_edge(const Prefix &kept, double sum, uint32_t before, uint32_t here, double at_edge) {
        return kept.whole || before >= kept.ties ? sum : sum + double(min(kept.ties - before, here)) * at_edge;
    }

    // The block's token with which the kept weights add up to more than the target; s.warp_sum and s.warp_ties are those of its warps.
    __device__ void find(const Prefix &kept, uint32_t ties_ahead, double at_edge, double target, double total, double largest) {
        double ahead = 0.0, before = 0.0;
        uint32_t ties_before = ties_ahead, who = 0;
        bool past = false;
        for (uint32_t k = 0; k < kSampleWarps && !past; ++k) {
            const uint32_t here = kept.whole ? 0 : s.warp_ties[k];
            const double add = with_edge(kept, s.warp_sum[k], ties_ahead, here, at_edge);
            if (add > 0.0) {
                who = k;
                before = ahead;
                ties_before = ties_ahead;
                past = ahead + add > target;
            }
            ahead += add;
            ties_ahead += here;
        }
        if (who != warp) return;
        // the warp's tokens, a pack of each lane at a time: the lane in which the sum passes the target, then its token
        int token = -1;
        float chosen = 0.0f;
        past = false;
#pragma unroll 1
        for (int j = 0; j < p.packs && !past; ++j) {
            const Packed pack = held[j * kSampleThreads];
            auto value = [&](int e) { return to_f32<T>(pack.v[e]); };
            double w[kVec], sum = 0.0;
            uint32_t tied = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) tied += !kept.whole && value(e) == kept.edge;
            uint32_t upto_ties = tied;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t q = __shfl_up_sync(~0u, upto_ties, o);
                if (lane >= uint32_t(o)) upto_ties += q;
            }
            uint32_t seen = ties_before + upto_ties - tied;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const float x = value(e);
                const bool at_the_edge = !kept.whole && x == kept.edge;
                w[e] = x > kept.edge || (x == kept.edge && (kept.whole || seen < kept.ties)) ? weight(x) : 0.0;
                seen += at_the_edge;
                sum += w[e];
            }
            double upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double q = __shfl_up_sync(~0u, upto, o);
                if (lane >= uint32_t(o)) upto += q;
            }
            const uint32_t over = __ballot_sync(~0u, sum > 0.0 && before + upto > target), any = __ballot_sync(~0u, sum > 0.0);
            past = over != 0;
            const int who_lane = over ? __ffs(int(over)) - 1 : any ? 31 - __clz(int(any)) : -1;
            if (who_lane >= 0) {
                // (the lane's first token past the target, or its last one with a weight)
                double run = before + upto - sum;
                int e_found = -1;
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const bool open = e_found < 0 || !(run > target);
                    run += w[e];
                    if (open && w[e] > 0.0) e_found = e;
                }
                float x = 0.0f;
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (e == e_found) x = value(e);
                token = __shfl_sync(~0u, at(j) + e_found, who_lane);
                chosen = __shfl_sync(~0u, x, who_lane);
            }
            before += __shfl_sync(~0u, upto, 31);
            ties_before += __shfl_sync(~0u, upto_ties, 31);
        }
        if (lane == 0) put_drawn(token, chosen, largest, total);
    }
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 4) tcu_sample_kernel(const SampleParams p) {
    extern __shared__ __align__(16) uint8_t held[];
    __shared__ SampleShared shared;
    Sampler<T>(p, shared, held).run();
}

}  // namespace tcu
