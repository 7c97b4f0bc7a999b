// Host side of layer norm (include/tcu_lm.h): argument checks, launches.
#include "tcu_lm.h"

#include <cuda_runtime.h>

#include <initializer_list>
#include <type_traits>
#include <utility>

#include "tcu_host.h"
#include "tcu_norm_kernel.cuh"

namespace {

using namespace tcu;

constexpr uint64_t kMostRows = (uint64_t(1) << 31) - 1;
constexpr uint64_t kMostStride = uint64_t(1) << 38;
constexpr size_t kMostWidth = size_t(kNormThreads) * 32;
constexpr uint32_t kSms = 148, kForwardThreads = 768, kForwardFull = 1024, kForwardNarrow = 512, kBackwardThreads = 512;       // of an SM, by what registers allow

bool extent(size_t rows, size_t d, size_t stride, size_t eb, size_t &bytes) {
    const unsigned __int128 n = rows == 0 ? 0 : ((unsigned __int128)(rows - 1) * stride + d) * eb;
    bytes = size_t(n);
    return !(n >> 63);
}

// How a row is divided: elements a thread holds, lanes of a row (0: a block of `threads`).  Sixteen elements a thread: the steps of a sum cost as much as
// ten elements (2048 columns, eight a thread: forward 77 us instead of 50); 32 only where a block would have more than 512 threads.
struct Shape {
    int vec, held, lanes;
    uint32_t threads;
    bool full;                 // every thread has all its elements
    uint64_t blocks;
};
// (on_sm: threads that an SM holds at once)
Shape shape_of(size_t rows, size_t d, int vec, size_t eb, uint32_t on_sm) {
    Shape s = {};
    if (vec * eb < 16 && on_sm == kForwardThreads) on_sm = kForwardNarrow;
    s.vec = vec;
    s.held = 16;
    if (d <= 32 * 16) {
        s.lanes = d <= 8 * 16 ? 8 : d <= 16 * 16 ? 16 : 32;
        s.threads = kNormWarps * 32;
        const uint64_t of_block = s.threads / s.lanes, most = kSms * (on_sm / s.threads);
        s.blocks = (rows + of_block - 1) / of_block;
        if (s.blocks > most) s.blocks = most;
        s.full = d == size_t(s.lanes) * s.held;
    } else {
        s.held = d <= kNormThreads * 16 ? 16 : 32;
        s.threads = uint32_t((d + size_t(s.held) * 32 - 1) / (size_t(s.held) * 32)) * 32;
        s.full = d == size_t(s.threads) * s.held;
        if (s.full && on_sm == kForwardThreads) on_sm = kForwardFull;
        const uint64_t most = uint64_t(kSms) * (on_sm / s.threads);
        s.blocks = rows < most ? rows : most;
    }
    return s;
}
// Elements a read: 16 bytes, 4 (two elements of 16 bits), or one element.
int vector_of(size_t eb, size_t d, std::initializer_list<size_t> strides, std::initializer_list<const void *> arrays) {
    for (size_t bytes = 16; bytes > eb; bytes = bytes == 16 && eb == 2 ? 4 : eb) {
        bool fits = d % (bytes / eb) == 0;
        for (size_t s : strides) fits = fits && s % (bytes / eb) == 0;
        for (const void *q : arrays) fits = fits && aligned(q, bytes);
        if (fits) return int(bytes / eb);
    }
    return 1;
}

// Launches a kernel with the rows that its threads have on their way, of `arrays` arrays, in shared memory.
template <auto kernel>
tcu_status_t launch(const Shape &s, size_t eb, int arrays, const NormParams &p, cudaStream_t stream) {
    const size_t of_thread = s.vec * eb == 16 ? size_t(arrays) * norm_ahead(int(s.held * eb)) * s.held * eb : 0;
    if (of_thread * kNormThreads > 32768 && !allow_shared<kernel>(of_thread * kNormThreads)) return TCU_ERR_CUDA;
    kernel<<<uint32_t(s.blocks), s.threads, of_thread * s.threads, stream>>>(p);
    return launched();
}

template <typename F>
void with_type(tcu_float_t type, F go) {
    if (type == TCU_F32) go(float{});
    else if (type == TCU_F16) go(__half{});
    else go(__nv_bfloat16{});
}

// Calls go(vector, elements held, lanes, full) with these as types.
template <typename T, typename F>
void with_shape(const Shape &s, F go) {
    constexpr int kVec = 16 / sizeof(T);
    auto divided = [&](auto vec, auto full) {
        constexpr std::integral_constant<int, 16> kHeld{};
        if (s.lanes == 8) go(vec, kHeld, std::integral_constant<int, 8>{}, full);
        else if (s.lanes == 16) go(vec, kHeld, std::integral_constant<int, 16>{}, full);
        else if (s.lanes == 32) go(vec, kHeld, std::integral_constant<int, 32>{}, full);
        else if (s.held == 16) go(vec, kHeld, std::integral_constant<int, 0>{}, full);
        else go(vec, std::integral_constant<int, 32>{}, std::integral_constant<int, 0>{}, full);
    };
    if (s.vec == kVec && s.full) return divided(std::integral_constant<int, kVec>{}, std::true_type{});
    if (s.vec == kVec) return divided(std::integral_constant<int, kVec>{}, std::false_type{});
    if constexpr (sizeof(T) == 2) {
        if (s.vec == 2) return divided(std::integral_constant<int, 2>{}, std::false_type{});
    }
    divided(std::integral_constant<int, 1>{}, std::false_type{});
}

tcu_status_t check(size_t rows, size_t d, tcu_float_t type, tcu_float_t param_type, float eps) {
    if (!valid_float(type) || !valid_float(param_type) || d == 0 || !(eps >= 0.0f) || eps > 3.0e38f) return TCU_ERR_INVALID_ARG;
    if (param_type != TCU_F32 && param_type != type) return TCU_ERR_UNSUPPORTED;
    if (d > kMostWidth || rows > kMostRows) return TCU_ERR_UNSUPPORTED;
    return TCU_OK;
}

NormParams params(size_t rows, size_t d, tcu_float_t param_type, float eps) {
    NormParams p = {};
    p.rows = uint32_t(rows);
    p.d = uint32_t(d);
    p.param_f32 = param_type == TCU_F32;
    p.eps = eps;
    p.inv_d = 1.0f / float(d);
    return p;
}

}  // namespace

extern "C" {

tcu_status_t tcu_layer_norm_forward(const void *d_x, size_t rows, size_t d, size_t x_stride, tcu_float_t type, const void *d_weight, const void *d_bias,
                                    tcu_float_t param_type, float eps, void *d_y, cudaStream_t stream) {
    if (tcu_status_t st = check(rows, d, type, param_type, eps)) return st;
    if (rows == 0) return TCU_OK;
    const size_t eb = float_bytes(type), pb = float_bytes(param_type);
    if (rows > 1 && x_stride > kMostStride) return TCU_ERR_INVALID_ARG;
    if (!d_x || !d_y || !aligned(d_x, eb) || !aligned(d_y, eb) || !aligned(d_weight, pb) || !aligned(d_bias, pb)) return TCU_ERR_INVALID_ARG;
    size_t xb, yb;
    if (!extent(rows, d, x_stride, eb, xb) || !extent(rows, d, d, eb, yb)) return TCU_ERR_INVALID_ARG;
    const bool in_place = d_x == d_y && (rows == 1 || x_stride == d);          // a row is read whole before it is written
    if ((!in_place && overlaps(d_y, yb, d_x, xb)) || overlaps(d_y, yb, d_weight, d * pb) || overlaps(d_y, yb, d_bias, d * pb)) return TCU_ERR_INVALID_ARG;
    const Shape s = shape_of(rows, d, vector_of(eb, d, {rows > 1 ? x_stride : 0}, {d_x, d_y}), eb, kForwardThreads);
    NormParams p = params(rows, d, param_type, eps);
    p.x = d_x;
    p.x_stride = x_stride;
    p.weight = d_weight;
    p.bias = d_bias;
    p.y = d_y;
    tcu_status_t st = TCU_OK;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        with_shape<T>(s, [&](auto v, auto e, auto lanes, auto full) {
            st = launch<tcu_norm_forward_kernel<T, decltype(v)::value, decltype(e)::value, decltype(lanes)::value, decltype(full)::value>>(s, eb, 1, p, stream);
        });
    });
    return st;
}

size_t tcu_layer_norm_workspace_bytes(size_t rows, size_t d) {
    if (d == 0 || d > kMostWidth || rows > kMostRows) return 0;
    return shape_of(rows, d, 1, 4, kBackwardThreads).blocks * 2 * d * 4 + 256;
}

tcu_status_t tcu_layer_norm_backward(const void *d_dy, size_t dy_stride, const void *d_x, size_t x_stride, size_t rows, size_t d, tcu_float_t type, const void *d_weight,
                                     tcu_float_t param_type, float eps, void *d_dx, void *d_dweight, void *d_dbias, void *d_ws, size_t ws_bytes, cudaStream_t stream) {
    if (tcu_status_t st = check(rows, d, type, param_type, eps)) return st;
    const size_t eb = float_bytes(type), pb = float_bytes(param_type);
    if (!aligned(d_weight, pb) || !aligned(d_dweight, pb) || !aligned(d_dbias, pb)) return TCU_ERR_INVALID_ARG;
    if (overlaps(d_dweight, d * pb, d_dbias, d * pb)) return TCU_ERR_INVALID_ARG;
    if (rows == 0) {
        for (void *q : {d_dweight, d_dbias})
            if (q && !ok(cudaMemsetAsync(q, 0, d * pb, stream))) return TCU_ERR_CUDA;
        return TCU_OK;
    }
    if (rows > 1 && (x_stride > kMostStride || dy_stride > kMostStride)) return TCU_ERR_INVALID_ARG;
    if (!d_x || !d_dy || !aligned(d_x, eb) || !aligned(d_dy, eb) || !aligned(d_dx, eb)) return TCU_ERR_INVALID_ARG;
    size_t xb, db, out;
    if (!extent(rows, d, x_stride, eb, xb) || !extent(rows, d, dy_stride, eb, db) || !extent(rows, d, d, eb, out)) return TCU_ERR_INVALID_ARG;
    const bool sums = d_dweight || d_dbias;
    if (!sums && !d_dx) return TCU_OK;
    const size_t need = sums ? tcu_layer_norm_workspace_bytes(rows, d) : 0;
    if (sums && (!d_ws || ws_bytes < need)) return TCU_ERR_WORKSPACE;
    if (sums && !aligned(d_ws, 16)) return TCU_ERR_INVALID_ARG;
    const bool in_place = d_dx == d_dy && (rows == 1 || dy_stride == d);
    for (const auto &w : {std::pair<const void *, size_t>{d_dx, out}, {d_dweight, d * pb}, {d_dbias, d * pb}, {sums ? d_ws : nullptr, need}}) {
        if (overlaps(w.first, w.second, d_x, xb) || overlaps(w.first, w.second, d_weight, d * pb)) return TCU_ERR_INVALID_ARG;
        if (!(w.first == d_dx && in_place) && overlaps(w.first, w.second, d_dy, db)) return TCU_ERR_INVALID_ARG;
    }
    for (const void *q : {static_cast<const void *>(d_dweight), static_cast<const void *>(d_dbias)})
        if (overlaps(d_dx, out, q, d * pb) || (sums && overlaps(d_ws, need, q, d * pb))) return TCU_ERR_INVALID_ARG;
    if (sums && overlaps(d_ws, need, d_dx, out)) return TCU_ERR_INVALID_ARG;
    const Shape s = shape_of(rows, d, vector_of(eb, d, {rows > 1 ? x_stride : 0, rows > 1 ? dy_stride : 0}, {d_x, d_dy, d_dx}), eb, kBackwardThreads);
    NormParams p = params(rows, d, param_type, eps);
    p.x = d_x;
    p.x_stride = x_stride;
    p.d_y = d_dy;
    p.dy_stride = dy_stride;
    p.weight = d_weight;
    p.d_x = d_dx;
    p.parts = sums ? static_cast<float *>(d_ws) : nullptr;
    tcu_status_t st = TCU_OK;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        with_shape<T>(s, [&](auto v, auto e, auto lanes, auto full) {
            st = launch<tcu_norm_backward_kernel<T, decltype(v)::value, decltype(e)::value, decltype(lanes)::value, decltype(full)::value>>(s, eb, 2, p, stream);
        });
    });
    if (st != TCU_OK || !sums) return st;
    const uint32_t joins = uint32_t((2 * d + 31) / 32);
    with_type(param_type, [&](auto t) {
        using P = decltype(t);
        st = launch_next(tcu_norm_join_kernel<P>, joins, 1024, stream, p.parts, uint32_t(s.blocks), p.d, static_cast<P *>(d_dweight), static_cast<P *>(d_dbias));
    });
    return st;
}

}  // extern "C"
