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

constexpr uint64_t kMostRows = uint64_t(1) << 40;
constexpr uint64_t kMostStride = uint64_t(1) << 38;
constexpr int kMostHeld = 32;                                        // elements of a row that a thread holds
constexpr size_t kMostWidth = size_t(kNormMaxThreads) * kMostHeld;
constexpr uint32_t kSms = 148;

bool extent(size_t rows, size_t d, size_t stride, size_t eb, size_t &bytes) {
    const unsigned __int128 n = rows == 0 ? 0 : ((unsigned __int128)(rows - 1) * stride + d) * eb;
    bytes = size_t(n);
    return !(n >> 63);
}

// How a row is divided: elements a thread holds, threads of a row, whether they are a block.
struct Shape {
    int vec, held;
    uint32_t threads;
    bool block;
    uint64_t blocks;
};
Shape shape_of(size_t rows, size_t d, int vec) {
    Shape s = {};
    s.vec = vec;
    s.held = 8;
    if (d <= 32 * 16) {
        s.held = d <= 32 * 8 ? 8 : 16;
        s.threads = 32;
        s.blocks = (rows + kNormWarpRows - 1) / kNormWarpRows;
        const uint64_t most = kSms * 8;
        if (s.blocks > most) s.blocks = most;
        return s;
    }
    while (size_t(kNormMaxThreads) * s.held < d) s.held *= 2;
    s.block = true;
    s.threads = uint32_t((d + size_t(s.held) * 32 - 1) / (size_t(s.held) * 32)) * 32;
    const uint64_t most = uint64_t(kSms) * (1024 / s.threads);
    s.blocks = rows < most ? rows : most;
    return s;
}

template <typename F>
void with_type(tcu_float_t type, F go) {
    if (type == TCU_F32) go(float{});
    else if (type == TCU_F16) go(__half{});
    else go(__nv_bfloat16{});
}

// Calls go(vector, elements held, block) with these as types.
template <typename T, typename F>
void with_shape(const Shape &s, F go) {
    constexpr int kVec = 16 / sizeof(T);
    auto held = [&](auto vec) {
        if (!s.block) {
            if (s.held == 8) go(vec, std::integral_constant<int, 8>{}, std::false_type{});
            else go(vec, std::integral_constant<int, 16>{}, std::false_type{});
        } else {
            if (s.held == 8) go(vec, std::integral_constant<int, 8>{}, std::true_type{});
            else if (s.held == 16) go(vec, std::integral_constant<int, 16>{}, std::true_type{});
            else go(vec, std::integral_constant<int, 32>{}, std::true_type{});
        }
    };
    if (s.vec > 1) held(std::integral_constant<int, kVec>{});
    else held(std::integral_constant<int, 1>{});
}

tcu_status_t check(size_t rows, size_t d, tcu_float_t type, tcu_float_t param_type, float eps) {
    if (!valid_float(type) || !valid_float(param_type) || d == 0 || !(eps >= 0.0f) || eps > 3.0e38f) return TCU_ERR_INVALID_ARG;
    if (param_type != TCU_F32 && param_type != type) return TCU_ERR_UNSUPPORTED;
    if (d > kMostWidth || rows > kMostRows) return TCU_ERR_UNSUPPORTED;
    return TCU_OK;
}

NormParams params(size_t rows, size_t d, tcu_float_t param_type, float eps) {
    NormParams p = {};
    p.rows = rows;
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
    const int vec = int(16 / eb);
    const bool wide = d % vec == 0 && (rows == 1 || x_stride % vec == 0) && aligned(d_x, 16) && aligned(d_y, 16);
    const Shape s = shape_of(rows, d, wide ? vec : 1);
    NormParams p = params(rows, d, param_type, eps);
    p.x = d_x;
    p.x_stride = x_stride;
    p.weight = d_weight;
    p.bias = d_bias;
    p.y = d_y;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        with_shape<T>(s, [&](auto v, auto e, auto block) {
            tcu_norm_forward_kernel<T, decltype(v)::value, decltype(e)::value, decltype(block)::value>
                <<<uint32_t(s.blocks), s.block ? s.threads : kNormWarpRows * 32, 0, stream>>>(p);
        });
    });
    return launched();
}

size_t tcu_layer_norm_workspace_bytes(size_t rows, size_t d) {
    if (d == 0 || d > kMostWidth || rows > kMostRows) return 0;
    return shape_of(rows, d, 1).blocks * 2 * d * 4 + 256;
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
    const int vec = int(16 / eb);
    const bool wide = d % vec == 0 && (rows == 1 || (x_stride % vec == 0 && dy_stride % vec == 0)) && aligned(d_x, 16) && aligned(d_dy, 16) && aligned(d_dx, 16);
    const Shape s = shape_of(rows, d, wide ? vec : 1);
    NormParams p = params(rows, d, param_type, eps);
    p.x = d_x;
    p.x_stride = x_stride;
    p.d_y = d_dy;
    p.dy_stride = dy_stride;
    p.weight = d_weight;
    p.d_x = d_dx;
    p.parts = sums ? static_cast<float *>(d_ws) : nullptr;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        with_shape<T>(s, [&](auto v, auto e, auto block) {
            tcu_norm_backward_kernel<T, decltype(v)::value, decltype(e)::value, decltype(block)::value>
                <<<uint32_t(s.blocks), s.block ? s.threads : kNormWarpRows * 32, 0, stream>>>(p);
        });
    });
    tcu_status_t st = launched();
    if (st != TCU_OK || !sums) return st;
    const uint32_t joins = uint32_t((2 * d + 31) / 32);
    with_type(param_type, [&](auto t) {
        using P = decltype(t);
        st = launch_next(tcu_norm_join_kernel<P>, joins, 256, stream, p.parts, uint32_t(s.blocks), p.d, static_cast<P *>(d_dweight), static_cast<P *>(d_dbias));
    });
    return st;
}

}  // extern "C"
