// Token embedding: lookup with a scale, and the table gradient as a segmented sum over the tokens sorted by id.
//
// Lookup: out[n] = scale * table[ids[n]].  Bound by memory: every output row is written once, every row that is met is
// read from HBM once (repeated rows come from L2).
//
// Gradient: row v of the table receives the sum of the d_out rows of the tokens that name it.  The tokens are sorted by
// id (least-significant-digit radix sort, 9 bits a pass, stable, so that the order of every sum is the order of the
// tokens); then the rows of the table and the sorted tokens are merged into one list in which row v follows the last of
// its tokens, and the list is cut into equal pieces: a piece costs the same whether it holds rows without tokens (a
// store of zeros each) or the many tokens of one row.  A row whose tokens end in a later piece leaves a partial sum,
// and a last kernel adds the partial sums of such rows in order.  No atomics on sums: the result is the same from call to call.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace tcu {

constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortTile = 2048;            // tokens a block sorts: 8 warps x 8 rounds of 32
constexpr int kSortThreads = 256;
constexpr int kPiece = 64;                 // entries (rows and tokens) of a piece of the merged list

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

template <typename ID>
__device__ __forceinline__ uint32_t row_of(const ID *ids, size_t n, uint32_t rows) {
    const long long id = static_cast<long long>(ids[n]);
    return id >= 0 && id < static_cast<long long>(rows) ? static_cast<uint32_t>(id) : rows;
}

// ---- lookup --------------------------------------------------------------------------------------------------------
// One thread an access; threads of a block cover `rows_per_block` output rows of `packs` accesses each.
template <typename T, typename ID, int VEC>
__global__ void __launch_bounds__(256) tcu_embedding_lookup_kernel(const ID *__restrict__ ids, uint64_t n, const T *__restrict__ table,
                                                                   uint32_t rows, uint32_t packs, uint64_t table_stride, float scale,
                                                                   T *__restrict__ out) {
    const uint64_t total = n * packs;
    for (uint64_t i = uint64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < total; i += uint64_t(gridDim.x) * blockDim.x) {
        const uint64_t t = i / packs;
        const uint32_t c = uint32_t(i - t * packs);
        const uint32_t r = row_of(ids, t, rows);
        Pack<T, VEC> p;
        if (r < rows) {
            p = *reinterpret_cast<const Pack<T, VEC> *>(table + uint64_t(r) * table_stride + uint64_t(c) * VEC);
#pragma unroll
            for (int e = 0; e < VEC; ++e) p.v[e] = from_f32<T>(to_f32(p.v[e]) * scale);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) p.v[e] = from_f32<T>(0.0f);
        }
        *reinterpret_cast<Pack<T, VEC> *>(out + i * VEC) = p;
    }
}

// ---- sort ----------------------------------------------------------------------------------------------------------
// A pass over digit `shift`: counts of every digit in every tile, their exclusive scan along the tiles (and the total
// of each digit), then every token to its place.  The first pass reads the ids, later ones (row, token) pairs.
template <typename ID>
__global__ void __launch_bounds__(kSortThreads) tcu_sort_count_kernel(const ID *__restrict__ ids, const uint32_t *__restrict__ keys,
                                                                      uint32_t n, uint32_t rows, int shift, uint32_t tiles,
                                                                      uint32_t *__restrict__ counts) {
    __shared__ uint32_t cnt[kDigits];
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) cnt[d] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * kSortTile;
    for (uint32_t i = first + threadIdx.x; i < first + kSortTile && i < n; i += kSortThreads) {
        const uint32_t key = keys ? keys[i] : row_of(ids, i, rows);
        atomicAdd(&cnt[(key >> shift) & (kDigits - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) counts[size_t(d) * tiles + blockIdx.x] = cnt[d];
}

// block d: exclusive scan of digit d's counts along the tiles, in place; the digit's total to totals[d]
__global__ void __launch_bounds__(kSortThreads) tcu_sort_scan_kernel(uint32_t *__restrict__ counts, uint32_t tiles, uint32_t *__restrict__ totals) {
    __shared__ uint32_t warp_sum[kSortThreads / 32];
    uint32_t *row = counts + size_t(blockIdx.x) * tiles;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t carry = 0;
    for (uint32_t base = 0; base < tiles; base += kSortThreads) {
        const uint32_t i = base + threadIdx.x;
        const uint32_t v = i < tiles ? row[i] : 0;
        uint32_t s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += u;
        }
        if (lane == 31) warp_sum[warp] = s;
        __syncthreads();
        uint32_t before = carry, all = 0;
        for (int w = 0; w < kSortThreads / 32; ++w) {
            if (w < warp) before += warp_sum[w];
            all += warp_sum[w];
        }
        if (i < tiles) row[i] = before + s - v;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = carry;
}

template <typename ID>
__global__ void __launch_bounds__(kSortThreads) tcu_sort_scatter_kernel(const ID *__restrict__ ids, const uint32_t *__restrict__ keys,
                                                                        const uint32_t *__restrict__ tokens, uint32_t n, uint32_t rows,
                                                                        int shift, uint32_t tiles, const uint32_t *__restrict__ counts,
                                                                        const uint32_t *__restrict__ totals, uint32_t *__restrict__ keys_out,
                                                                        uint32_t *__restrict__ tokens_out) {
    constexpr int kWarps = kSortThreads / 32, kRounds = kSortTile / kSortThreads;
    __shared__ uint32_t base[kDigits];                 // where the tile's tokens of a digit begin
    __shared__ uint16_t seen[kWarps][kDigits];         // tokens of a digit in a warp, then in the warps before it
    __shared__ uint32_t warp_sum[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int d = threadIdx.x; d < kWarps * kDigits; d += kSortThreads) (&seen[0][0])[d] = 0;
    // exclusive scan of the digits' totals: two digits a thread
    const uint32_t t0 = totals[2 * threadIdx.x], t1 = totals[2 * threadIdx.x + 1];
    uint32_t s = t0 + t1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    uint32_t before = s - t0 - t1;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    base[2 * threadIdx.x] = before + counts[size_t(2 * threadIdx.x) * tiles + blockIdx.x];
    base[2 * threadIdx.x + 1] = before + t0 + counts[size_t(2 * threadIdx.x + 1) * tiles + blockIdx.x];
    // a warp takes 256 consecutive tokens, 32 at a time; tokens of one digit find one another by a match
    const uint32_t first = blockIdx.x * kSortTile + warp * (32 * kRounds);
    uint32_t key[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint32_t i = first + r * 32 + lane;
        key[r] = i < n ? (keys ? keys[i] : row_of(ids, i, rows)) : 0;
    }
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
        tokens_out[to] = tokens ? tokens[i] : i;
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
};

// First entry of piece `p` of the merged list: rows r and tokens n with r + n = d, where token n comes before the end
// of row r when keys[n] <= r.  When only rows with tokens are touched (accumulate), the list is the tokens alone.
__device__ __forceinline__ void piece_start(const SumParams &s, uint32_t p, uint32_t &r, uint32_t &n) {
    const uint64_t entries = (s.accumulate ? 0u : uint64_t(s.rows)) + s.n;
    uint64_t d = uint64_t(p) * kPiece;
    if (d > entries) d = entries;
    if (s.accumulate) {
        n = uint32_t(d);
        r = n < s.n ? s.keys[n] : s.rows;
        return;
    }
    uint64_t lo = d > s.n ? d - s.n : 0, hi = d < s.rows ? d : s.rows;
    while (lo < hi) {
        const uint64_t mid = (lo + hi) >> 1;
        if (s.keys[d - 1 - mid] <= mid) hi = mid;
        else lo = mid + 1;
    }
    r = uint32_t(lo);
    n = uint32_t(d - lo);
}

template <typename TT, int VEC>
__device__ __forceinline__ void emit_row(TT *table, uint64_t at, const float (&acc)[VEC], float scale, int accumulate) {
    Pack<TT, VEC> p;
    Pack<TT, VEC> *to = reinterpret_cast<Pack<TT, VEC> *>(table + at);
    if (accumulate) p = *to;
#pragma unroll
    for (int e = 0; e < VEC; ++e) p.v[e] = from_f32<TT>((accumulate ? to_f32(p.v[e]) : 0.0f) + acc[e] * scale);
    *to = p;
}

// A group of blockDim.x threads takes a piece, VEC columns a thread; blockDim.y groups a block.
template <typename T, typename TT, int VEC>
__global__ void __launch_bounds__(256) tcu_embedding_sum_kernel(const T *__restrict__ d_out, TT *__restrict__ table, const SumParams s) {
    const uint32_t piece = blockIdx.x * blockDim.y + threadIdx.y;
    const uint32_t col = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
    if (piece >= s.pieces || col >= s.d) return;
    uint32_t row, n0, row_end, n1;
    piece_start(s, piece, row, n0);
    piece_start(s, piece + 1, row_end, n1);
    bool continued = n0 > 0 && row < s.rows && s.keys[n0 - 1] == row;      // the first row has tokens in earlier pieces
    bool pending = false;                                                  // tokens summed for `row`, which is not finished
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
    auto finish = [&](uint32_t r) {
        if (continued) {
            Pack<float, VEC> p;
#pragma unroll
            for (int e = 0; e < VEC; ++e) p.v[e] = acc[e];
            *reinterpret_cast<Pack<float, VEC> *>(s.head + uint64_t(piece) * s.d + col) = p;
            continued = false;
        } else {
            emit_row<TT, VEC>(table, uint64_t(r) * s.d + col, acc, s.scale, s.accumulate);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
        pending = false;
    };
    constexpr int kAhead = 8;                       // token rows in flight
    for (uint32_t n = n0; n < n1; n += kAhead) {
        Pack<T, VEC> val[kAhead];
        uint32_t key[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            key[j] = n + j < n1 ? s.keys[n + j] : s.rows;
            if (key[j] < s.rows) val[j] = *reinterpret_cast<const Pack<T, VEC> *>(d_out + uint64_t(s.tokens[n + j]) * s.d + col);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (key[j] >= s.rows) break;
            if (s.accumulate) {
                if (key[j] != row) {
                    finish(row);
                    row = key[j];
                }
            } else {
                for (; row < key[j]; ++row) finish(row);
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
        Pack<float, VEC> p;
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.v[e] = acc[e];
        *reinterpret_cast<Pack<float, VEC> *>(s.tail + uint64_t(piece) * s.d + col) = p;
    }
}

// For every piece that finishes a row begun in earlier ones: the tails of those pieces, in order, then its own head.
template <typename TT, int VEC>
__global__ void __launch_bounds__(256) tcu_embedding_join_kernel(TT *__restrict__ table, const SumParams s) {
    const uint32_t piece = blockIdx.x * blockDim.y + threadIdx.y;
    const uint32_t col = (blockIdx.y * blockDim.x + threadIdx.x) * VEC;
    if (piece >= s.pieces || piece == 0 || col >= s.d) return;
    uint32_t row, n0, row_end, n1;
    piece_start(s, piece, row, n0);
    piece_start(s, piece + 1, row_end, n1);
    if (row >= s.rows || n0 == 0 || s.keys[n0 - 1] != row) return;         // nothing from earlier pieces
    if (s.accumulate ? (n1 < s.n && s.keys[n1] == row) : row_end == row) return;       // not finished here either
    // first token of the row, and the piece that holds it
    uint32_t lo = 0, hi = n0;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (s.keys[mid] < row) lo = mid + 1;
        else hi = mid;
    }
    const uint32_t first = uint32_t(((s.accumulate ? 0u : uint64_t(row)) + lo) / kPiece);
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
    for (uint32_t q = first; q < piece; ++q) {
        const Pack<float, VEC> p = *reinterpret_cast<const Pack<float, VEC> *>(s.tail + uint64_t(q) * s.d + col);
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += p.v[e];
    }
    const Pack<float, VEC> p = *reinterpret_cast<const Pack<float, VEC> *>(s.head + uint64_t(piece) * s.d + col);
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] += p.v[e];
    emit_row<TT, VEC>(table, uint64_t(row) * s.d + col, acc, s.scale, s.accumulate);
}

}  // namespace tcu
