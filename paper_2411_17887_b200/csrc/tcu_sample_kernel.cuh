// Sampling of one token for each row of logits.  With m the largest logit of the row, every token has the weight
// w = exp((logit - m) / temperature).  In the order of falling logits, the lower token first among equals, the tokens kept are the
// first top_k, as far as w >= min_p, and of these the fewest whose weights add up to top_p times the weight of them all: a
// prefix of that order, so that it is told by its last logit and how many of the tokens with that one belong to it.  The token
// drawn is the first, in the order of tokens, up to and with which the kept weights add up to more than u times their sum.
//
// A row is read once, into the shared memory of a cluster of blocks, a part each.  The last kept logit is found by histograms: of
// numbers of tokens for top_k, of weights for top_p - linear in the logit first, then of the logit's bits as an integer, 11 bits a time.
// Sums that decide which token it is are exact enough that it is the token of the definition: weights in 64-bit floating point, in histograms
// in fixed point with 42 bits (three limbs of 14, each sum of at most 2^18 tokens within 32 bits), whose sums do not depend on their order.
#pragma once

#include <cooperative_groups.h>

#include "tcu_float.cuh"

namespace tcu {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleBins = 2048;
constexpr int kSampleMaxCluster = 8;
constexpr uint32_t kMostVocabulary = 1u << 18;
constexpr double kSampleFixed = 4398046511104.0;      // 2^42
constexpr int kSampleLimb = 14;

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
    uint32_t vocabulary, part;             // tokens of a row, and (a multiple of 16 bytes) of a block
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
    uint32_t count;                        // of the bin (counts)
    uint64_t before, in, total;            // sums ahead of the bin, of the bin, of all bins
};

struct SampleShared {
    uint32_t hist[3][kSampleBins];
    SampleWord slots[2][kSampleMaxCluster];
    SampleFound found[2];
    double warp_sum[kSampleWarps];
    uint64_t warp_u64[kSampleWarps];
    uint32_t warp_u32[kSampleWarps], warp_ties[kSampleWarps];
    float warp_max[kSampleWarps];
    uint32_t least_key;
};

__device__ __forceinline__ uint32_t sample_key(float v) {        // the order of logits as that of unsigned integers
    const uint32_t b = __float_as_uint(v);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float sample_value(uint32_t key) {
    return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kKeyNothing = 0x007fffffu;                    // that of minus infinity

template <typename T>
struct Sampler {
    static constexpr int kVec = 16 / sizeof(T);
    const SampleParams &p;
    SampleShared &s;
    T *held;                               // this block's part of the row, minus infinity where it has no token
    cooperative_groups::cluster_group cluster;
    uint32_t rank, ranks, phase = 0, found_phase = 0;
    uint32_t row, n;
    int64_t first;                         // token of held[0]
    float top = 0.0f;
    double inverse = 1.0;                  // of the temperature

    __device__ Sampler(const SampleParams &p, SampleShared &s, T *held)
        : p(p), s(s), held(held), cluster(cooperative_groups::this_cluster()) {
        rank = cluster.block_rank();
        ranks = cluster.num_blocks();
        row = blockIdx.x / ranks;
    }

    // The weight of a token; logits at the top have 1 also where that is infinite.
    __device__ __forceinline__ double weight(float v) const { return v == top ? 1.0 : exp((double(v) - double(top)) * inverse); }
    __device__ __forceinline__ uint64_t fixed(float v) const { return uint64_t(__double2ll_rn(weight(v) * kSampleFixed)); }

    // Every block's word, at every block.  All threads call it; what is told has to be ready in thread 0's to kSampleMaxCluster - 1's `mine`.
    __device__ const SampleWord *exchange(const SampleWord &mine) {
        SampleWord *slots = s.slots[phase];
        phase ^= 1;
        if (threadIdx.x < ranks) cluster.map_shared_rank(slots, threadIdx.x)[rank] = mine;
        cluster.sync();
        return slots;
    }

    __device__ float block_max(float v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
        if ((threadIdx.x & 31) == 0) s.warp_max[threadIdx.x >> 5] = v;
        __syncthreads();
        v = s.warp_max[threadIdx.x & (kSampleWarps - 1)];
#pragma unroll
        for (int o = kSampleWarps / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
        return v;
    }
    __device__ uint32_t block_min(uint32_t v) {
        v = __reduce_min_sync(~0u, v);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) s.warp_u32[threadIdx.x >> 5] = v;
        __syncthreads();
        return __reduce_min_sync(~0u, s.warp_u32[threadIdx.x & (kSampleWarps - 1)]);
    }
    __device__ uint32_t cluster_min(uint32_t v) {
        const SampleWord *w = exchange({0.0, block_min(v), 0});
        uint32_t least = w[0].b;
        for (uint32_t k = 1; k < ranks; ++k) least = min(least, w[k].b);
        return least;
    }

    // Reads the block's part of the row (addresses in steps of 16 bytes, whatever the row begins at) and finds the largest logit.
    __device__ void load() {
        const T *at = static_cast<const T *>(p.logits) + uint64_t(row) * p.stride;
        const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(at) % 16) / sizeof(T);       // tokens ahead of the row on its first 16 bytes
        const int64_t begin = int64_t(rank) * p.part;
        first = begin - off;
        n = p.part;
        float most = -INFINITY;
        for (uint32_t i = threadIdx.x * kVec; i < n; i += kSampleThreads * kVec) {
            Pack<T, kVec> v;
            const int64_t token = first + i;
            if (token >= 0 && token + kVec <= p.vocabulary) {
                v = *reinterpret_cast<const Pack<T, kVec> *>(at + token);
            } else {
#pragma unroll
                for (int e = 0; e < kVec; ++e) v.v[e] = token + e >= 0 && token + e < p.vocabulary ? at[token + e] : from_f32<T>(-INFINITY);
            }
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                float f = to_f32<T>(v.v[e]) + 0.0f;                  // (no zero below zero: the two are equal)
                if (f != f) f = -INFINITY;
                most = fmaxf(most, f);
                v.v[e] = from_f32<T>(f);
            }
            *reinterpret_cast<Pack<T, kVec> *>(held + i) = v;
        }
        most = block_max(most);
        const SampleWord *w = exchange({double(most), 0, 0});
        top = float(w[0].a);
        for (uint32_t k = 1; k < ranks; ++k) top = fmaxf(top, float(w[k].a));
    }

    __device__ __forceinline__ float logit(uint32_t i) const { return to_f32<T>(held[i]); }

    // Histogram over the row's tokens of bin_of (below 0: not counted) - of weights, or of numbers - and the first bin with which the
    // sum from `before` on reaches `target`; the target is taken from the sum of all bins by target_of.
    template <bool WEIGHTS, typename BinOf, typename TargetOf>
    __device__ SampleFound histogram(BinOf bin_of, uint64_t before, TargetOf target_of) {
        constexpr int kLimbs = WEIGHTS ? 3 : 1;
        SampleFound *found = &s.found[found_phase];
        found_phase ^= 1;
        for (int l = 0; l < kLimbs; ++l)
            for (uint32_t b = threadIdx.x; b < kSampleBins; b += kSampleThreads) s.hist[l][b] = 0;
        if (threadIdx.x == 0) found->bin = -1;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < n; i += kSampleThreads) {
            const float v = logit(i);
            const int b = bin_of(v);
            if (b < 0) continue;
            if constexpr (WEIGHTS) {
                const uint64_t w = fixed(v);
                atomicAdd(&s.hist[0][b], uint32_t(w) & ((1u << kSampleLimb) - 1));
                atomicAdd(&s.hist[1][b], uint32_t(w >> kSampleLimb) & ((1u << kSampleLimb) - 1));
                atomicAdd(&s.hist[2][b], uint32_t(w >> (2 * kSampleLimb)));
            } else {
                atomicAdd(&s.hist[0][b], 1u);
            }
        }
        cluster.sync();
        // this block's share of the bins, a few each thread
        const uint32_t share = kSampleBins / ranks, each = (share + kSampleThreads - 1) / kSampleThreads;
        const uint32_t own = rank * share + threadIdx.x * each;
        const bool some = threadIdx.x * each < share;
        uint64_t mine[kSampleBins / kSampleThreads], sum = 0;
        for (uint32_t j = 0; j < each; ++j) {
            uint64_t v = 0;
            if (some)
                for (uint32_t k = 0; k < ranks; ++k) {
                    const auto *h = cluster.map_shared_rank(&s.hist[0][0], k) + own + j;
                    v += h[0];
                    if constexpr (WEIGHTS) v += (uint64_t(h[kSampleBins]) << kSampleLimb) + (uint64_t(h[2 * kSampleBins]) << (2 * kSampleLimb));
                }
            mine[j] = v;
            sum += v;
        }
        const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        uint64_t upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t q = __shfl_up_sync(~0u, upto, o);
            if (lane >= uint32_t(o)) upto += q;
        }
        if (lane == 31) s.warp_u64[warp] = upto;
        __syncthreads();
        uint64_t ahead = 0, all = 0;
        for (uint32_t k = 0; k < kSampleWarps; ++k) {
            if (k < warp) ahead += s.warp_u64[k];
            all += s.warp_u64[k];
        }
        ahead += upto - sum;
        const SampleWord *w = exchange({__longlong_as_double(int64_t(all)), 0, 0});
        uint64_t total = 0;
        for (uint32_t k = 0; k < ranks; ++k) {
            const uint64_t q = uint64_t(__double_as_longlong(w[k].a));
            if (k < rank) ahead += q;
            total += q;
        }
        const double target = target_of(total);
        ahead += before;
        for (uint32_t j = 0; j < each; ++j) {
            if (some && double(ahead) < target && double(ahead + mine[j]) >= target) {
                const SampleFound f = {int(own + j), 0, ahead, mine[j], total};
                for (uint32_t k = 0; k < ranks; ++k) *cluster.map_shared_rank(found, k) = f;
            }
            ahead += mine[j];
        }
        cluster.sync();
        SampleFound f = *found;
        f.total = total;
        return f;
    }

    // The prefix (in falling order) of the tokens with a key of at least `least` that reaches a target: its last key, how many of the tokens with
    // that key it takes, and whether these are all.  False: the tokens do not reach the target.
    template <bool WEIGHTS, typename TargetOf>
    __device__ bool reach(uint32_t least, TargetOf target_of, uint32_t &last, uint32_t &ties, bool &whole, uint64_t &total) {
        const float scale = float(inverse * 64.0);
        auto linear = [&](float v) {
            return sample_key(v) < least ? -1 : v == top ? 0 : int(fminf((top - v) * scale, float(kSampleBins - 1)));
        };
        SampleFound f = histogram<WEIGHTS>(linear, 0, target_of);
        total = f.total;
        if (f.bin < 0) return false;
        const double target = target_of(total);
        uint32_t lo = ~0u, hi_not = ~0u;                     // keys of the bin: from lo to ~hi_not
        for (uint32_t i = threadIdx.x; i < n; i += kSampleThreads) {
            const float v = logit(i);
            if (linear(v) != f.bin) continue;
            lo = min(lo, sample_key(v));
            hi_not = min(hi_not, ~sample_key(v));
        }
        lo = cluster_min(lo);
        uint32_t hi = ~cluster_min(hi_not);
        while (lo < hi) {
            const int bits = 32 - __clz(hi - lo), shift = bits > 11 ? bits - 11 : 0;
            const SampleFound g = histogram<WEIGHTS>(
                [&](float v) {
                    const uint32_t key = sample_key(v);
                    return key < lo || key > hi ? -1 : int((hi - key) >> shift);
                },
                f.before, [&](uint64_t) { return target; });
            if (g.bin < 0) break;                            // (not met: these bins add up to the one before)
            f = g;
            hi -= uint32_t(f.bin) << shift;
            lo = max(lo, hi - ((1u << shift) - 1));
        }
        last = hi;
        // the fewest of the tokens with this key that reach the target
        const uint64_t one = WEIGHTS ? fixed(sample_value(hi)) : 1, many = one ? f.in / one : 1;
        uint64_t c = one ? uint64_t(fmax(ceil((target - double(f.before)) / double(one)), 1.0)) : 1;
        while (c > 1 && double(f.before + (c - 1) * one) >= target) --c;
        while (c < many && double(f.before + c * one) < target) ++c;
        ties = uint32_t(c);
        whole = c >= many;
        return true;
    }

    // The least key whose weight is at least min_p: found by every warp's lanes, 32 keys at a time.
    __device__ uint32_t least_key(double min_p) {
        uint64_t lo = kKeyNothing + 1, hi = sample_key(top);             // hi has weight 1
        const uint32_t lane = threadIdx.x & 31;
        while (lo < hi) {
            const uint64_t step = (hi - lo + 31) / 32, at = lo + step * lane;
            const uint32_t in = __ballot_sync(~0u, at < hi && weight(sample_value(uint32_t(at))) >= min_p);
            // of the keys looked at, those from the first that is in on are in
            const uint32_t looked = __popc(__ballot_sync(~0u, at < hi)), f = in ? uint32_t(__ffs(int(in)) - 1) : looked;
            if (f < looked) hi = lo + step * f;
            if (f > 0) lo += step * (f - 1) + 1;
        }
        return uint32_t(hi);
    }

    __device__ void put(int64_t token, float log_prob) {
        p.tokens[row] = token;
        if (p.log_probs) p.log_probs[row] = log_prob;
    }

    __device__ void run() {
        load();
        if (top == -INFINITY) {
            if (rank == 0 && threadIdx.x == 0) put(-1, -INFINITY);
            cluster.sync();
            return;
        }
        const double temperature = p.temperature.at(row), min_p = p.min_p.at(row), top_p = p.top_p.at(row);
        const double k = p.top_k.at(row);
        const bool warm = temperature > 0.0;
        inverse = warm && top < INFINITY ? 1.0 / temperature : 1.0;      // (with an infinite logit the others have no weight at any temperature)
        if (!warm || k == 1.0 || min_p > 1.0 || top_p <= 0.0) {          // the first token alone
            uint32_t at = ~0u;
            for (uint32_t i = threadIdx.x; i < n; i += kSampleThreads)
                if (logit(i) == top) at = min(at, uint32_t(first + i));
            at = cluster_min(at);
            if (rank == 0 && threadIdx.x == 0) put(at, 0.0f);
            cluster.sync();
            return;
        }
        uint32_t least = kKeyNothing + 1, ties = 0;                      // kept: keys above `least`, and those of it, the first `ties` if not all
        bool whole = true;
        if (min_p > 0.0) least = least_key(min_p);
        uint64_t total = 0;
        bool edge = false;                                               // whether top_k ends within (or with) the tokens of key `least`
        if (k > 0.0 && k < double(p.vocabulary)) edge = reach<false>(least, [&](uint64_t) { return k; }, least, ties, whole, total);
        if (top_p < 1.0) {
            const uint64_t group = edge ? ties * fixed(sample_value(least)) : 0;
            uint32_t last = 0, some = 0;
            bool all = true;
            if (reach<true>(edge ? least + 1 : least, [&](uint64_t sum) { return top_p * double(sum + group); }, last, some, all, total)) {
                least = last;
                ties = some;
                whole = all;
            } else if (edge) {
                const uint64_t one = fixed(sample_value(least));
                const double target = top_p * double(total + group);
                uint32_t c = 1;
                if (one) c = uint32_t(fmin(fmax(ceil((target - double(total)) / double(one)), 1.0), double(ties)));
                while (c > 1 && double(total + (c - 1) * one) >= target) --c;
                while (c < ties && double(total + c * one) < target) ++c;
                whole = whole && c == ties;
                ties = c;
            }
        }
        draw(least, ties, whole);
        cluster.sync();
    }

    // Draws from the tokens with keys above `least`, and of those with it all (whole) or the first `ties`.
    __device__ void draw(uint32_t least, uint32_t ties, bool whole) {
        const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const uint32_t each = ((n + kSampleWarps - 1) / kSampleWarps + 31) / 32 * 32;         // tokens of a warp
        const uint32_t begin = min(warp * each, n), end = min(begin + each, n);
        const uint32_t edge = whole ? 0u : least;                                             // (0: no token has this key)
        const uint32_t from = whole ? least : least + 1;
        const double w_edge = whole ? 0.0 : weight(sample_value(least));
        double sum = 0.0;
        uint32_t count = 0;
        for (uint32_t i = begin + lane; i < end; i += 32) {
            const float v = logit(i);
            const uint32_t key = sample_key(v);
            if (key >= from) sum += weight(v);
            count += key == edge;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        count = __reduce_add_sync(~0u, count);
        __syncthreads();
        if (lane == 0) {
            s.warp_sum[warp] = sum;
            s.warp_ties[warp] = count;
        }
        __syncthreads();
        double block_sum = 0.0;
        uint32_t block_ties = 0;
        for (int k = 0; k < kSampleWarps; ++k) {
            block_sum += s.warp_sum[k];
            block_ties += s.warp_ties[k];
        }
        const SampleWord *words = exchange({block_sum, block_ties, 0});
        // sums with the edge's tokens that belong to it, block after block
        auto with_edge = [&](double some, uint32_t before, uint32_t here) {
            const uint32_t left = before < ties ? ties - before : 0;
            return whole ? some : some + double(min(left, here)) * w_edge;
        };
        double total = 0.0;
        uint32_t seen = 0;
        for (uint32_t k = 0; k < ranks; ++k) {
            total += with_edge(words[k].a, seen, words[k].b);
            seen += words[k].b;
        }
        double u = p.uniform_f64 ? static_cast<const double *>(p.uniform)[row] : double(static_cast<const float *>(p.uniform)[row]);
        if (!(u > 0.0)) u = 0.0;
        const double target = u * total;
        // the block, then its warp, in which the sum passes the target (the last one that adds anything, if rounding leaves none)
        double ahead = 0.0, before = 0.0;
        uint32_t ties_ahead = 0, ties_before = 0, who = 0;
        bool past = false;
        for (uint32_t k = 0; k < ranks && !past; ++k) {
            const double add = with_edge(words[k].a, ties_ahead, words[k].b);
            if (add > 0.0) {
                who = k;
                before = ahead;
                ties_before = ties_ahead;
                past = ahead + add > target;
            }
            ahead += add;
            ties_ahead += words[k].b;
        }
        if (who != rank) return;
        ahead = before;
        ties_ahead = ties_before;
        past = false;
        who = 0;
        for (uint32_t k = 0; k < kSampleWarps && !past; ++k) {
            const double add = with_edge(s.warp_sum[k], ties_ahead, s.warp_ties[k]);
            if (add > 0.0) {
                who = k;
                before = ahead;
                ties_before = ties_ahead;
                past = ahead + add > target;
            }
            ahead += add;
            ties_ahead += s.warp_ties[k];
        }
        if (who != warp) return;
        // the warp's tokens, 32 at a time
        int64_t token = -1;
        float chosen = 0.0f;
        past = false;
        for (uint32_t i0 = begin; i0 < end && !past; i0 += 32) {
            const uint32_t i = i0 + lane;
            const float v = i < end ? logit(i) : -INFINITY;
            const uint32_t key = sample_key(v);
            const uint32_t tied = __ballot_sync(~0u, key == edge);
            const bool kept = key >= from || (key == edge && ties_before + __popc(tied & ((1u << lane) - 1)) < ties);
            ties_before += __popc(tied);
            const double w = kept ? weight(v) : 0.0;
            double upto = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double q = __shfl_up_sync(~0u, upto, o);
                if (lane >= uint32_t(o)) upto += q;
            }
            const uint32_t over = __ballot_sync(~0u, w > 0.0 && before + upto > target), any = __ballot_sync(~0u, w > 0.0);
            past = over != 0;
            const int at = over ? __ffs(int(over)) - 1 : any ? 31 - __clz(int(any)) : -1;
            if (at >= 0) {
                token = first + i0 + at;
                chosen = __shfl_sync(~0u, v, at);
            }
            before += __shfl_sync(~0u, upto, 31);
        }
        if (lane == 0) put(token, float((chosen == top ? 0.0 : (double(chosen) - double(top)) * inverse) - log(total)));
    }
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) tcu_sample_kernel(const SampleParams p) {
    extern __shared__ __align__(16) uint8_t held[];
    __shared__ SampleShared shared;
    Sampler<T>(p, shared, reinterpret_cast<T *>(held)).run();
}

}  // namespace tcu
