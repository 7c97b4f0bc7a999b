// Token embedding: lookup with a scale, and the table gradient as a segmented sum over the tokens sorted by id.
//
// Lookup: out[n] = scale * table[ids[n]].  Bound by memory: every output row is written once, every row that is met is
// read from HBM once (repeated rows come from L2).  32749 skewed ids, bfloat16 rows of 2048: 34.7 us, 5.1 TB/s; a copy of
// the same rows without the scale 32.
//
// Gradient: row v of the table receives the sum of the d_out rows of the tokens that name it, in the order of the
// tokens: no atomics on sums, the result is the same from call to call.  Few tokens: one launch, in which a block owns
// some rows and picks their tokens out of all the ids.  Many: the tokens are sorted by id (least-significant-digit
// radix sort, 9 bits a pass, stable); then the rows of the table and the sorted tokens are merged into one list in which
// row v follows the last of its tokens, and the list is cut into equal pieces: a piece costs about the same whether it
// holds rows without tokens (a store of zeros each) or the many tokens of one row.  A row whose tokens end in a later
// piece leaves a partial sum, and a last kernel adds the partial sums of such rows in order.  65536 skewed tokens of 1024
// bfloat16 columns into 50000 float32 rows: 92 us, of which the sort 16 (bound by the latency of what its four
// launches read), the cuts 3, the sums 60 (339 MB, 5.6 TB/s; reading 134 MB and then clearing 205 takes 66)
// and the join 9.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tcu {

constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 512;          // as many as digits
constexpr int kSortRounds = 2;             // tokens a thread
constexpr int kSortTile = kSortThreads * kSortRounds;
constexpr int kPiece = 32;                 // entries (rows and tokens) of a piece of the merged list

// ---- element types -------------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// VEC elements of T, moved as one access of up to 16 bytes
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC <= 16 ? sizeof(T) * VEC : 16) Pack {
    T v[VEC];
};

// A kernel of a sequence lets the next one be set up while it runs, and touches no memory before the one ahead of it is
// done with all of its own (which holds, in turn, for every one before).  What an earlier kernel writes is therefore not
// read through pointers that promise the compiler that nobody writes it.
__device__ __forceinline__ void begin_in_sequence() {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <typename ID>
__device__ __forceinline__ uint32_t row_of(const ID *ids, size_t n, uint32_t rows) {
    const long long id = static_cast<long long>(ids[n]);
    return id >= 0 && id < static_cast<long long>(rows) ? static_cast<uint32_t>(id) : rows;
}

// p * scale, two elements at a time where they are 16 bits (a conversion of two is one instruction).
template <typename T, int VEC>
__device__ __forceinline__ void scale_pack(Pack<T, VEC> &p, float scale) {
    if constexpr (std::is_same_v<T, __nv_bfloat16> && VEC % 2 == 0) {
        __nv_bfloat162 *two = reinterpret_cast<__nv_bfloat162 *>(p.v);
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
            const float2 f = __bfloat1622float2(two[e]);
            two[e] = __floats2bfloat162_rn(f.x * scale, f.y * scale);
        }
    } else if constexpr (std::is_same_v<T, __half> && VEC % 2 == 0) {
        __half2 *two = reinterpret_cast<__half2 *>(p.v);
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) {
            const float2 f = __half22float2(two[e]);
            two[e] = __floats2half2_rn(f.x * scale, f.y * scale);
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.v[e] = from_f32<T>(to_f32(p.v[e]) * scale);
    }
}

// ---- lookup --------------------------------------------------------------------------------------------------------
// Threads x take the accesses of an output row, threads y rows; a thread takes one place of ROWS output rows, so that
// its loads are under way together.
template <typename T, typename ID, int VEC, int ROWS>
__global__ void __launch_bounds__(256) tcu_embedding_lookup_kernel(const ID *__restrict__ ids, uint32_t n, const T *__restrict__ table,
                                                                   uint32_t rows, uint32_t d, uint64_t table_stride, float scale,
                                                                   T *__restrict__ out) {
    const uint32_t col = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
    if (col >= d) return;
    const uint32_t first = blockIdx.x * (blockDim.y * ROWS) + threadIdx.y;
    uint32_t row[ROWS];
    Pack<T, VEC> p[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const uint32_t t = first + j * blockDim.y;
        row[j] = t < n ? row_of(ids, t, rows) : rows;
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (row[j] < rows) {
            p[j] = *reinterpret_cast<const Pack<T, VEC> *>(table + uint64_t(row[j]) * table_stride + col);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) p[j].v[e] = from_f32<T>(0.0f);
        }
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const uint32_t t = first + j * blockDim.y;
        if (t >= n) continue;
        if (row[j] < rows) scale_pack<T, VEC>(p[j], scale);
        *reinterpret_cast<Pack<T, VEC> *>(out + uint64_t(t) * d + col) = p[j];
    }
}

// ---- sort ----------------------------------------------------------------------------------------------------------
// A pass over digit `shift`: counts of every digit in every tile, then every token to its place.  The first pass reads
// the ids, later ones (row, token) pairs.
template <typename ID>
__global__ void __launch_bounds__(kSortThreads) tcu_sort_count_kernel(const ID *__restrict__ ids, const uint32_t *keys,
                                                                      uint32_t n, uint32_t rows, int shift, uint32_t *counts, uint32_t *joins) {
    __shared__ uint32_t cnt[kDigits];
    cnt[threadIdx.x] = 0;
    __syncthreads();
    begin_in_sequence();
    if (joins && blockIdx.x == 0 && threadIdx.x == 0) *joins = 0;
    const uint32_t first = blockIdx.x * kSortTile + threadIdx.x;
    uint32_t key[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const uint32_t i = first + r * kSortThreads;
        if (i < n) key[r] = keys ? keys[i] : row_of(ids, i, rows);
    }
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (first + r * kSortThreads < n) atomicAdd(&cnt[(key[r] >> shift) & (kDigits - 1)], 1u);
    __syncthreads();
    counts[size_t(blockIdx.x) * kDigits + threadIdx.x] = cnt[threadIdx.x];
}

// Exclusive scan of the counts along the tiles, in place, and the totals.  A block takes 32 digits, a warp a share of the tiles.
__global__ void __launch_bounds__(1024) tcu_sort_scan_kernel(uint32_t *counts, uint32_t tiles, uint32_t *totals) {
    __shared__ uint32_t share[32][32];
    begin_in_sequence();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t *mine = counts + blockIdx.x * 32 + lane;
    const uint32_t each = (tiles + 31) / 32, from = min(tiles, warp * each), to = min(tiles, from + each);
    uint32_t sum = 0;
#pragma unroll 8
    for (uint32_t t = from; t < to; ++t) sum += mine[size_t(t) * kDigits];
    share[warp][lane] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < warp; ++w) before += share[w][lane];
    if (warp == 31) totals[blockIdx.x * 32 + lane] = before + sum;
#pragma unroll 4
    for (uint32_t t = from; t < to; ++t) {
        const uint32_t c = mine[size_t(t) * kDigits];
        mine[size_t(t) * kDigits] = before;
        before += c;
    }
}

// SCANNED: the counts went through the scan.  Else every block adds up those of all the tiles for itself.
template <typename ID, bool SCANNED>
__global__ void __launch_bounds__(kSortThreads) tcu_sort_scatter_kernel(const ID *__restrict__ ids, const uint32_t *keys,
                                                                        const uint32_t *tokens, uint32_t n, uint32_t rows,
                                                                        int shift, uint32_t tiles, const uint32_t *counts,
                                                                        const uint32_t *totals, uint32_t *keys_out,
                                                                        uint32_t *tokens_out) {
    constexpr int kWarps = kSortThreads / 32, kRounds = kSortRounds;
    static_assert(kSortThreads == kDigits, "a thread takes a digit");
    __shared__ uint32_t base[kDigits];                 // where the tile's tokens of a digit begin
    __shared__ uint16_t seen[kWarps][kDigits];         // tokens of a digit in a warp, then in the warps before it
    __shared__ uint32_t warp_sum[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int d = threadIdx.x; d < kWarps * kDigits; d += kSortThreads) (&seen[0][0])[d] = 0;
    begin_in_sequence();
    // a warp takes consecutive tokens, 32 at a time
    const uint32_t first = blockIdx.x * kSortTile + warp * (32 * kRounds);
    uint32_t key[kRounds], token[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t i = first + r * 32 + lane;
        key[r] = i < n ? (keys ? keys[i] : row_of(ids, i, rows)) : 0;
        token[r] = tokens && i < n ? tokens[i] : i;
    }
    uint32_t total = 0, ahead_tiles = 0;               // of this thread's digit
    if (SCANNED) {
        total = totals[threadIdx.x];
        ahead_tiles = counts[size_t(blockIdx.x) * kDigits + threadIdx.x];
    } else {
        // a quarter of the tiles for each quarter of the block, four digits a thread
        constexpr uint32_t kAhead = 8;
        __shared__ uint4 sums[2][4][kDigits / 4];
        const uint32_t quarter = threadIdx.x / (kDigits / 4), four = threadIdx.x % (kDigits / 4);
        uint4 all = make_uint4(0, 0, 0, 0), ahead = all;
        auto add = [](uint4 &to, uint4 c) { to.x += c.x, to.y += c.y, to.z += c.z, to.w += c.w; };
        for (uint32_t t = quarter; t < tiles; t += 4 * kAhead) {
            uint4 c[kAhead];
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j)
                c[j] = t + 4 * j < tiles ? reinterpret_cast<const uint4 *>(counts + size_t(t + 4 * j) * kDigits)[four] : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) {
                add(all, c[j]);
                if (t + 4 * j < blockIdx.x) add(ahead, c[j]);
            }
        }
        sums[0][quarter][four] = all;
        sums[1][quarter][four] = ahead;
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            total += reinterpret_cast<const uint32_t *>(sums[0][q])[threadIdx.x];
            ahead_tiles += reinterpret_cast<const uint32_t *>(sums[1][q])[threadIdx.x];
        }
    }
    uint32_t s = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    uint32_t before = s - total;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    base[threadIdx.x] = before + ahead_tiles;
    // tokens of one digit find one another by a match
    uint32_t rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const bool valid = first + r * 32 + lane < n;
        const uint32_t digit = valid ? (key[r] >> shift) & (kDigits - 1) : uint32_t(kDigits);
        const uint32_t same = __match_any_sync(0xffffffffu, digit);
        const uint32_t ahead = __popc(same & ((1u << lane) - 1));
        uint32_t old = 0;
        if (valid) old = seen[warp][digit];
        __syncwarp();
        if (valid && ahead == 0) seen[warp][digit] = uint16_t(old + __popc(same));
        __syncwarp();
        rank[r] = old + ahead;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) {
        uint32_t sum = 0;
        for (int w = 0; w < kWarps; ++w) {
            const uint32_t c = seen[w][d];
            seen[w][d] = uint16_t(sum);
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t i = first + r * 32 + lane;
        if (i >= n) continue;
        const uint32_t digit = (key[r] >> shift) & (kDigits - 1);
        const uint32_t to = base[digit] + seen[warp][digit] + rank[r];
        keys_out[to] = key[r];
        tokens_out[to] = token[r];
    }
}

// All passes of the sort in one block, for up to kBlockTokens tokens: 1024 threads of 4 tokens, which stay in shared memory between
// the passes.  Gradient of 1025 tokens of 500 columns into 4099 rows 19 us (23 by the launches above), 4096 tokens of 1024 27 (27);
// with 8 tokens a thread 8192 tokens of 256 took 37 us, 30 by launches.
constexpr uint32_t kBlockTokens = 4096;
constexpr int kBlockThreads = 1024, kBlockRounds = kBlockTokens / kBlockThreads, kBlockWarps = kBlockThreads / 32;
struct BlockSort {
    uint32_t keys[kBlockTokens];
    uint16_t tokens[kBlockTokens];
    uint16_t seen[kBlockWarps][kDigits];               // tokens of a digit in a warp, then in the warps before it
    uint32_t base[kDigits], warp_sum[kBlockWarps];
};
template <typename ID>
__global__ void __launch_bounds__(kBlockThreads) tcu_sort_block_kernel(const ID *__restrict__ ids, uint32_t n, uint32_t rows, int bits, uint32_t *keys_out,
                                                                       uint32_t *tokens_out, uint32_t *joins) {
    extern __shared__ BlockSort block_sort[];
    BlockSort &s = block_sort[0];
    const uint32_t t = threadIdx.x, lane = t & 31, warp = t >> 5, first = warp * (32 * kBlockRounds) + lane;
    begin_in_sequence();
    if (t == 0) *joins = 0;
    uint32_t key[kBlockRounds], token[kBlockRounds], rank[kBlockRounds];
#pragma unroll
    for (int r = 0; r < kBlockRounds; ++r) {
        token[r] = first + r * 32;
        key[r] = token[r] < n ? row_of(ids, token[r], rows) : 0;
    }
    for (int shift = 0; shift < bits; shift += kDigitBits) {
        for (uint32_t i = t; i < kBlockWarps * kDigits / 2; i += kBlockThreads) reinterpret_cast<uint32_t *>(&s.seen[0][0])[i] = 0;
        __syncthreads();
        // tokens of one digit find one another by a match
#pragma unroll
        for (int r = 0; r < kBlockRounds; ++r) {
            const bool valid = first + r * 32 < n;
            const uint32_t digit = valid ? (key[r] >> shift) & (kDigits - 1) : uint32_t(kDigits);
            const uint32_t same = __match_any_sync(0xffffffffu, digit);
            const uint32_t ahead = __popc(same & ((1u << lane) - 1));
            const uint32_t old = valid ? s.seen[warp][digit] : 0;
            __syncwarp();
            if (valid && ahead == 0) s.seen[warp][digit] = uint16_t(old + __popc(same));
            __syncwarp();
            rank[r] = old + ahead;
        }
        __syncthreads();
        uint32_t total = 0;                            // of digit t
        if (t < kDigits) {
#pragma unroll 8
            for (int w = 0; w < kBlockWarps; ++w) {
                const uint32_t c = s.seen[w][t];
                s.seen[w][t] = uint16_t(total);
                total += c;
            }
        }
        uint32_t sum = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= uint32_t(o)) sum += u;
        }
        if (lane == 31) s.warp_sum[warp] = sum;
        __syncthreads();
        if (t < kDigits) {
            uint32_t before = sum - total;
            for (uint32_t w = 0; w < warp; ++w) before += s.warp_sum[w];
            s.base[t] = before;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kBlockRounds; ++r) {
            if (first + r * 32 >= n) continue;
            const uint32_t digit = (key[r] >> shift) & (kDigits - 1), to = s.base[digit] + s.seen[warp][digit] + rank[r];
            s.keys[to] = key[r];
            s.tokens[to] = uint16_t(token[r]);
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kBlockRounds; ++r) {
            if (first + r * 32 >= n) continue;
            key[r] = s.keys[first + r * 32];
            token[r] = s.tokens[first + r * 32];
        }
    }
#pragma unroll
    for (int r = 0; r < kBlockRounds; ++r) {
        if (first + r * 32 >= n) continue;
        keys_out[first + r * 32] = key[r];
        tokens_out[first + r * 32] = token[r];
    }
}

// ---- segmented sum -------------------------------------------------------------------------------------------------
struct SumParams {
    const uint32_t *keys, *tokens;     // sorted: row (or `rows` for a token that is left out) and token
    uint32_t n, rows;
    uint32_t d;                        // columns
    uint32_t pieces;
    int accumulate;
    float scale;
    float *tail, *head;                // per piece, d values: sum of the row that the piece leaves unfinished / finishes for earlier pieces
    uint2 *starts;                     // per piece, and behind the last: where it begins
    uint32_t *joins;                   // how many rows are finished for earlier pieces
    uint2 *join;                       // these, in any order: row, and the piece that finishes it
    uint32_t *begins;                  // per row that goes on in a later piece: the piece where it begins
};

// First i of lo..hi for which `holds`, which stays true from there on; hi if there is none.  A warp tries 32 places at a time.
template <typename F>
__device__ __forceinline__ uint32_t warp_first(uint32_t lo, uint32_t hi, F holds) {
    const uint32_t lane = (threadIdx.x + threadIdx.y * blockDim.x) & 31;
    while (lo < hi) {
        const uint32_t step = (hi - lo + 31) / 32;
        const uint64_t at = uint64_t(lo) + uint64_t(step) * (lane + 1) - 1;
        const uint32_t yes = __ballot_sync(0xffffffffu, at >= hi || holds(uint32_t(at)));
        if (yes == 0) return hi;
        const uint32_t f = __ffs(yes) - 1;
        const uint64_t end = uint64_t(lo) + uint64_t(step) * (f + 1) - 1;
        lo += step * f;
        if (end < hi) hi = uint32_t(end);
    }
    return hi;
}

// Where the pieces of the merged list begin: rows r and tokens n with r + n = d, where token n comes before the end of
// row r when keys[n] <= r.  When only rows with tokens are touched (accumulate), the list is the tokens alone.  A row of
// up to 32 tokens is not cut: the piece that begins it takes it to its end.  A warp a piece.
__global__ void __launch_bounds__(128) tcu_embedding_cut_kernel(const SumParams s) {
    begin_in_sequence();
    const uint32_t p = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x & 31;
    if (p > s.pieces) return;
    const uint64_t entries = (s.accumulate ? 0u : uint64_t(s.rows)) + s.n, at = uint64_t(p) * kPiece;
    const uint64_t d = at < entries ? at : entries;
    uint32_t r, n;
    if (s.accumulate) {
        n = uint32_t(d);
        r = n < s.n ? s.keys[n] : s.rows;
    } else {
        r = warp_first(uint32_t(d > s.n ? d - s.n : 0), uint32_t(d < s.rows ? d : s.rows), [&](uint32_t mid) { return s.keys[d - 1 - mid] <= mid; });
        n = uint32_t(d - r);
    }
    if (n > 0 && r < s.rows) {
        const bool before = n > lane && s.keys[n - 1 - lane] == r, after = lane < s.n - n && s.keys[n + lane] == r;
        const uint32_t b = __popc(__ballot_sync(0xffffffffu, before)), a = __popc(__ballot_sync(0xffffffffu, after));
        if (b > 0 && a + b <= 32) {
            n += a;
            r = !s.accumulate ? r + 1 : n < s.n ? s.keys[n] : s.rows;
        }
    }
    if (lane == 0) s.starts[p] = make_uint2(r, n);
}

template <typename T, int VEC>
__device__ __forceinline__ void store_pack(T *to, const Pack<T, VEC> &p) {
    if constexpr (sizeof(T) * VEC == 32) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "f"(p.v[0]), "f"(p.v[1]), "f"(p.v[2]), "f"(p.v[3]),
                     "f"(p.v[4]), "f"(p.v[5]), "f"(p.v[6]), "f"(p.v[7])
                     : "memory");
    } else {
        *reinterpret_cast<Pack<T, VEC> *>(to) = p;
    }
}

template <typename TT, int VEC>
__device__ __forceinline__ void emit_row(TT *table, uint64_t at, const float (&acc)[VEC], float scale, int accumulate) {
    Pack<TT, VEC> p;
    if (accumulate) p = *reinterpret_cast<const Pack<TT, VEC> *>(table + at);
#pragma unroll
    for (int e = 0; e < VEC; ++e) p.v[e] = from_f32<TT>((accumulate ? to_f32(p.v[e]) : 0.0f) + acc[e] * scale);
    store_pack<TT, VEC>(table + at, p);
}

template <int VEC>
__device__ __forceinline__ void store_sum(float *to, const float (&acc)[VEC]) {
    Pack<float, VEC> p;
#pragma unroll
    for (int e = 0; e < VEC; ++e) p.v[e] = acc[e];
    store_pack<float, VEC>(to, p);
}

// A group of blockDim.x threads takes a piece, VEC columns a thread; blockDim.y groups a block of 128 threads.  Bound by
// memory; pieces of 64 entries in blocks of 256 threads left a short third wave (70 us).
template <typename T, typename TT, int VEC>
__global__ void __launch_bounds__(128, 7) tcu_embedding_sum_kernel(const T *__restrict__ d_out, TT *__restrict__ table, const SumParams s) {
    begin_in_sequence();
    const uint32_t piece = blockIdx.x * blockDim.y + threadIdx.y;
    const uint32_t col = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
    if (piece >= s.pieces || col >= s.d) return;
    uint32_t row = s.starts[piece].x;
    const uint32_t n0 = s.starts[piece].y, row_end = s.starts[piece + 1].x, n1 = s.starts[piece + 1].y;
    constexpr int kAhead = 4;                       // token rows in flight; the keys and places of the next ones come meanwhile
    uint32_t key[kAhead], token[kAhead];
    auto look = [&](uint32_t n) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            key[j] = n + j < n1 ? s.keys[n + j] : s.rows;
            token[j] = n + j < n1 ? s.tokens[n + j] : 0;
        }
    };
    look(n0);
    bool continued = n0 > 0 && row < s.rows && s.keys[n0 - 1] == row;      // the first row has tokens in earlier pieces
    bool pending = false;                                                  // tokens summed for `row`, which is not finished
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
    auto finish = [&](uint32_t r) {
        if (continued) {
            store_sum<VEC>(s.head + uint64_t(piece) * s.d + col, acc);
            if (col == 0) s.join[atomicAdd(s.joins, 1u)] = make_uint2(r, piece);
            continued = false;
        } else {
            emit_row<TT, VEC>(table, uint64_t(r) * s.d + col, acc, s.scale, s.accumulate);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
        pending = false;
    };
    for (uint32_t n = n0; n < n1; n += kAhead) {
        Pack<T, VEC> val[kAhead];
        uint32_t of[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            of[j] = key[j];
            if (of[j] < s.rows) val[j] = *reinterpret_cast<const Pack<T, VEC> *>(d_out + uint64_t(token[j]) * s.d + col);
        }
        look(n + kAhead);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (of[j] >= s.rows) break;
            if (s.accumulate) {
                if (of[j] != row) {
                    finish(row);
                    row = of[j];
                }
            } else {
                for (; row < of[j]; ++row) finish(row);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[e] += to_f32(val[j].v[e]);
            pending = true;
        }
    }
    if (s.accumulate) {
        // the last row is finished here if the next piece does not go on with it
        const bool ends = n1 >= s.n || s.keys[n1] != row;
        if ((pending || continued) && row < s.rows && ends && n1 > n0) finish(row);
    } else {
        for (; row < row_end; ++row) finish(row);
    }
    if (pending) {
        store_sum<VEC>(s.tail + uint64_t(piece) * s.d + col, acc);
        if (col == 0 && !continued) s.begins[row] = piece;
    }
}

// For every row that is spread over pieces: the tails of those before the last, then the head of that.  A block takes 32
// accesses of a row, so that one with many tokens is spread over several SMs; each of its warps adds a quarter of the
// tails, in order, and the first warp adds the quarters.
template <typename TT, int VEC>
__global__ void __launch_bounds__(128) tcu_embedding_join_kernel(TT *__restrict__ table, const SumParams s) {
    __shared__ Pack<float, VEC> part[3][32];
    begin_in_sequence();
    const uint32_t shares = (s.d + 32 * VEC - 1) / (32 * VEC), joins = *s.joins;        // at most 2^15 and 2^26
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x / 32;
    for (uint64_t i = blockIdx.x; i < uint64_t(joins) * shares; i += gridDim.x) {
        const uint32_t at = uint32_t(i / shares), col = (uint32_t(i - uint64_t(at) * shares) * 32 + lane) * VEC;
        const uint2 join = s.join[at];
        const bool mine = col < s.d;
        const uint32_t first = s.begins[join.x], each = (join.y - first + 3) / 4;
        const uint32_t from = min(join.y, first + warp * each), to = min(join.y, from + each);
        Pack<float, VEC> acc, head;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc.v[e] = 0.0f;
        if (warp == 0 && mine) head = *reinterpret_cast<const Pack<float, VEC> *>(s.head + uint64_t(join.y) * s.d + col);
        constexpr uint32_t kAhead = 16;
        for (uint32_t q = from; q < to && mine; q += kAhead) {
            Pack<float, VEC> p[kAhead];
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j)
                if (q + j < to) p[j] = *reinterpret_cast<const Pack<float, VEC> *>(s.tail + uint64_t(q + j) * s.d + col);
#pragma unroll
            for (uint32_t j = 0; j < kAhead; ++j) {
                if (q + j >= to) break;
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc.v[e] += p[j].v[e];
            }
        }
        if (warp) part[warp - 1][lane] = acc;
        __syncthreads();
        if (warp == 0 && mine) {
#pragma unroll
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc.v[e] += part[w][lane].v[e];
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc.v[e] += head.v[e];
            emit_row<TT, VEC>(table, uint64_t(join.x) * s.d + col, acc.v, s.scale, s.accumulate);
        }
        __syncthreads();
    }
}

// ---- few tokens ----------------------------------------------------------------------------------------------------
// Measured, bfloat16 to float32, skewed ids: 1024 tokens of 500 columns into 4099 rows 12 us, by the sort 19; of 1024 columns
// into 4000 rows 15 against 22, 16000 rows 27 against 29, 32000 rows 42 to 65 (by device) against 45: rows reach memory out of
// order from here, which can be slow once the table does not stay in L2.  All tokens in one row: 25 us against 18.
constexpr uint32_t kFewTokens = 1024;      // at most
constexpr uint64_t kFewElements = uint64_t(1) << 24;       // of the table, at most
constexpr uint32_t kFewRows = 256;         // rows of a block, at most
constexpr uint32_t kFewCols = 256;         // columns of a block
// A row with more tokens than this is summed by the whole block: 1021 skewed tokens 10 us (23 if a warp takes every row), all of them in one
// row 27 (164).
constexpr uint32_t kFewMany = 8;

// A block of 8 warps takes every gridDim.x-th row (neighbours in a vocabulary are often alike in frequency, and would
// make some blocks slow) and 256 columns.  Every warp goes through an eighth of the ids and keeps, in order,
// those of the block's rows.  Then a warp a row; a row of many tokens takes all the warps, each with its eighth of the ids.
template <typename T, typename TT, typename ID, int VEC>
__global__ void __launch_bounds__(256, 3) tcu_embedding_few_kernel(const T *__restrict__ d_out, const ID *__restrict__ ids, TT *__restrict__ table,
                                                                uint32_t n, uint32_t rows, uint32_t d, float scale, int accumulate) {
    constexpr int kSteps = kFewCols / (32 * VEC), kIds = 4, kAhead = 4;
    __shared__ uint16_t token[kFewTokens];
    __shared__ uint8_t local[kFewTokens];
    __shared__ uint32_t kept[8], count[kFewRows];
    __shared__ __align__(32) float part[8][kFewCols];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t mine = (rows - blockIdx.x + gridDim.x - 1) / gridDim.x, col0 = blockIdx.y * kFewCols + lane * VEC;
    static_assert(kFewRows == 256, "a thread a row");
    count[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t share = (n + 255) / 256 * 32, from = min(n, warp * share), to = min(n, from + share);
    uint32_t have = 0;
    for (uint32_t base = from; base < to; base += 32 * kIds) {
        uint32_t r[kIds];
#pragma unroll
        for (int j = 0; j < kIds; ++j) {
            const uint32_t i = base + j * 32 + lane;
            r[j] = i < to ? row_of(ids, i, rows) : rows;
        }
#pragma unroll
        for (int j = 0; j < kIds; ++j) {
            const uint32_t at_row = r[j] / gridDim.x;
            const bool keep = r[j] < rows && r[j] - at_row * gridDim.x == blockIdx.x;
            const uint32_t mask = __ballot_sync(0xffffffffu, keep);
            if (keep) {
                const uint32_t at = from + have + __popc(mask & ((1u << lane) - 1));
                token[at] = uint16_t(base + j * 32 + lane);
                local[at] = uint8_t(at_row);
                atomicAdd(&count[at_row], 1u);
            }
            have += __popc(mask);
        }
    }
    if (lane == 0) kept[warp] = have;
    __syncthreads();
    float acc[kSteps][VEC];
    auto clear = [&] {
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[c][e] = 0.0f;
    };
    // adds the rows of d_out that share `w` of the ids has for row r; lanes alike
    auto add = [&](uint32_t r, uint32_t w) {
        const uint32_t begin = min(n, w * share), end = begin + kept[w];
        for (uint32_t base = begin; base < end; base += 32) {
            const uint32_t t = base + lane < end ? token[base + lane] : 0;
            uint32_t mask = __ballot_sync(0xffffffffu, base + lane < end && local[base + lane] == r);
            while (mask) {
                Pack<T, VEC> val[kAhead][kSteps];
                bool have[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    have[j] = mask != 0;
                    const uint32_t at = __shfl_sync(0xffffffffu, t, have[j] ? __ffs(mask) - 1 : 0);
                    mask &= mask - 1;
#pragma unroll
                    for (int c = 0; c < kSteps; ++c)
                        if (have[j] && col0 + c * 32 * VEC < d) val[j][c] = *reinterpret_cast<const Pack<T, VEC> *>(d_out + uint64_t(at) * d + col0 + c * 32 * VEC);
                }
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
#pragma unroll
                    for (int c = 0; c < kSteps; ++c)
                        if (have[j] && col0 + c * 32 * VEC < d) {
#pragma unroll
                            for (int e = 0; e < VEC; ++e) acc[c][e] += to_f32(val[j][c].v[e]);
                        }
            }
        }
    };
    for (uint32_t r = warp; r < mine; r += 8) {
        if (count[r] > kFewMany || (accumulate && count[r] == 0)) continue;
        clear();
        for (uint32_t w = 0; w < 8 && count[r]; ++w)
            if (kept[w]) add(r, w);
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
            if (col0 + c * 32 * VEC < d) emit_row<TT, VEC>(table, uint64_t(blockIdx.x + r * gridDim.x) * d + col0 + c * 32 * VEC, acc[c], scale, accumulate);
    }
    for (uint32_t r = 0; r < mine; ++r) {
        if (count[r] <= kFewMany) continue;             // the same for all threads
        clear();
        add(r, warp);
#pragma unroll
        for (int c = 0; c < kSteps; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) part[warp][(c * 32 + lane) * VEC + e] = acc[c][e];
        __syncthreads();
        for (uint32_t at = threadIdx.x; at < kFewCols && blockIdx.y * kFewCols + at < d; at += 256) {
            float sum[1] = {0.0f};
#pragma unroll
            for (int w = 0; w < 8; ++w) sum[0] += part[w][at];
            emit_row<TT, 1>(table, uint64_t(blockIdx.x + r * gridDim.x) * d + blockIdx.y * kFewCols + at, sum, scale, accumulate);
        }
        __syncthreads();
    }
}

}  // namespace tcu
