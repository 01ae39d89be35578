// layer_norm.cu -- layer normalisation of rows and its backward pass (include/cb_tbe.h): rows longer
// than registers hold, the join of the weight's gradient, how a call's rows are read, the entry points.
#include "layer_norm.cuh"
#include "spans.h"

#include <cmath>

namespace cbtbe {
namespace norm {

int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 152;
    return sms;
}

namespace {

// Rows longer than a block's registers hold: read again (from L2) for each sum, value by value. A rare shape.
__global__ void __launch_bounds__(kMostThreads)
layer_norm_long_kernel(const Args A) {
    __shared__ float shared[2 * kMostThreads / 32];
    begin_kernel();
    int turn = 0;
    const float inv = 1.f / static_cast<float>(A.dim);
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const int64_t x0 = row * A.x_row, y0 = row * A.out_row;
        auto value = [&](int c) { return any_value(any_bits(A.x, x0 + c, A.in_dtype), A.in_dtype); };
        float sum[1] = {0.f}, square[1] = {0.f};
        for (int c = threadIdx.x; c < A.dim; c += kMostThreads) sum[0] += value(c);
        group_sum<kMostThreads>(sum, shared, turn);
        const float mean = sum[0] * inv;
        for (int c = threadIdx.x; c < A.dim; c += kMostThreads) {
            const float d = value(c) - mean;
            square[0] = fmaf(d, d, square[0]);
        }
        group_sum<kMostThreads>(square, shared, turn);
        const float rstd = 1.f / sqrtf(fmaf(square[0], inv, A.eps));
        if (threadIdx.x == 0) {
            if (A.mean) A.mean[row] = mean;
            if (A.rstd) A.rstd[row] = rstd;
        }
        for (int c = threadIdx.x; c < A.dim; c += kMostThreads) {
            const float w = A.weight ? load_param(A.weight, c, A.weight_dtype) : 1.f;
            const float b = A.bias ? load_param(A.bias, c, A.bias_dtype) : 0.f;
            any_store(A.out, y0 + c, fmaf((value(c) - mean) * rstd, w, b), A.out_dtype);
        }
    }
}

__global__ void __launch_bounds__(kMostThreads)
layer_norm_backward_long_kernel(const Args A) {
    __shared__ float shared[4 * kMostThreads / 32];
    begin_kernel();
    int turn = 0;
    const float inv = 1.f / static_cast<float>(A.dim);
    float* mine = A.partial ? A.partial + static_cast<int64_t>(blockIdx.x) * 2 * A.dim : nullptr;
    for (int64_t row = blockIdx.x; row < A.rows; row += gridDim.x) {
        const int64_t x0 = row * A.x_row, dy0 = row * A.dy_row, dx0 = row * A.out_row;
        const float mean = A.mean[row], rstd = A.rstd[row];
        auto values = [&](int c, float& xh, float& d, float& g) {
            xh = (any_value(any_bits(A.x, x0 + c, A.in_dtype), A.in_dtype) - mean) * rstd;
            d = any_value(any_bits(A.dy, dy0 + c, A.in_dtype), A.in_dtype);
            g = d * (A.weight ? load_param(A.weight, c, A.weight_dtype) : 1.f);
        };
        float sum[2] = {0.f, 0.f};
        const bool first = row == blockIdx.x;
        for (int c = threadIdx.x; c < A.dim; c += kMostThreads) {
            float xh, d, g;
            values(c, xh, d, g);
            sum[0] += g;
            sum[1] = fmaf(g, xh, sum[1]);
            if (mine) {
                mine[c] = fmaf(d, xh, first ? 0.f : mine[c]);
                mine[A.dim + c] = d + (first ? 0.f : mine[A.dim + c]);
            }
        }
        group_sum<kMostThreads>(sum, shared, turn);
        const float m0 = sum[0] * inv, m1 = sum[1] * inv;
        for (int c = threadIdx.x; c < A.dim; c += kMostThreads) {
            float xh, d, g;
            values(c, xh, d, g);
            any_store(A.out, dx0 + c, rstd * (g - m0 - xh * m1), A.out_dtype);
        }
    }
}

// dw and db from the blocks' sums: 32 columns a block, each of its warps takes every eighth row of them.
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(kJoinWarps * 32)
layer_norm_join_kernel(const float* partial, int32_t parts, int32_t dim, float* dw, float* db) {
    __shared__ float shared[kJoinWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;  // of dw and db behind one another
    begin_kernel();
    float sum = 0.f;
    if (col < 2 * dim) {
        int p = warp;
        for (; p + 3 * kJoinWarps < parts; p += 4 * kJoinWarps) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __ldcg(partial + static_cast<int64_t>(p + k * kJoinWarps) * 2 * dim + col);
            sum += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; p < parts; p += kJoinWarps) sum += __ldcg(partial + static_cast<int64_t>(p) * 2 * dim + col);
    }
    shared[warp][lane] = sum;
    __syncthreads();
    if (warp || col >= 2 * dim) return;
#pragma unroll
    for (int k = 1; k < kJoinWarps; ++k) sum += shared[k][lane];
    if (col < dim) {
        if (dw) dw[col] = sum;
    } else if (db) {
        db[col - dim] = sum;
    }
}

bool type_ok(int t) { return t == CB_F32 || t == CB_F16 || t == CB_BF16; }
int size_of(int dtype) { return dtype == CB_F32 ? 4 : 2; }
bool aligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % size_of(dtype) == 0; }
bool sizes_ok(int64_t rows, int64_t dim) { return rows >= 0 && rows < (int64_t{1} << 40) && dim >= 0 && dim <= kMaxDim; }
bool row_ok(int64_t rows, int64_t dim, int64_t stride) {
    return rows <= 1 || (stride >= dim && stride <= (INT64_MAX >> 4) / rows);
}
// The memory of a tensor of rows; of one that is written in an input's place, of one type and layout, none.
Span span(const void* p, int dtype, int64_t rows, int64_t dim, int64_t stride) {
    return Span(p, dim * size_of(dtype)).by(rows, rows > 1 ? stride * size_of(dtype) : 0);
}
Span vector(const void* p, int dtype, int64_t n) { return Span(p, n * size_of(dtype)); }
bool in_place(const void* x, int dtype, int64_t stride, const void* out, int out_dtype, int64_t out_stride, int64_t rows) {
    return x == out && dtype == out_dtype && (rows <= 1 || stride == out_stride);
}
cb_status launched() { return cudaGetLastError() == cudaSuccess ? CB_OK : CB_ERR_CUDA; }

// Pieces of 16 bytes of the narrower type where all rows begin on them, or begin equally far behind
// one in every tensor; else value by value. Sets A's begin, and strides where there is one row.
Shape shape_of(Args& A) {
    if (A.rows <= 1) A.x_row = A.dy_row = A.out_row = A.dim;
    const int v = A.in_dtype == CB_F32 && A.out_dtype == CB_F32 ? 4 : 8;
    auto begin = [&](const void* p, int dtype) {  // values behind a piece's boundary
        return static_cast<int>(reinterpret_cast<uintptr_t>(p) / size_of(dtype) % v);
    };
    const int x = begin(A.x, A.in_dtype), y = begin(A.out, A.out_dtype), step = static_cast<int>(A.x_row % v);
    bool same = y == x && A.out_row % v == step && (!A.dy || (begin(A.dy, A.in_dtype) == x && A.dy_row % v == step));
    same = same && (A.in_dtype == A.out_dtype || A.in_dtype == CB_F32 || A.out_dtype == CB_F32);
    if (!same) return {1, group_threads(A.dim), false};
    A.begin = x;
    A.begin_step = step;
    const bool shifted = x || step || A.dim % v;
    return {v, group_threads(A.dim + (shifted ? v - 1 : 0)), shifted};
}
// The backward pass's blocks do not depend on the pointers, so that its workspace's size does not.
int64_t partial_rows(int64_t rows, int64_t dim) {
    int64_t most = 0;
    for (const int g : {group_threads(dim), group_threads(dim + 7)})
        most = std::max(most, g ? backward_blocks(rows, g) : std::min<int64_t>(rows, sm_count()));
    return most;
}

int64_t launch_any(Args& A, bool back, cudaStream_t s) {  // blocks of the backward pass
    const Shape S = shape_of(A);
    if (S.g == 0) {
        const int64_t grid = std::min<int64_t>(A.rows, sm_count());
        launch(back ? layer_norm_backward_long_kernel : layer_norm_long_kernel, dim3(static_cast<unsigned>(grid)),
               dim3(kMostThreads), 0, s, A);
        return grid;
    }
    if (S.v == 1) back ? launch_group<kAny, kAny, 1, false, true>(A, S.g, s) : launch_group<kAny, kAny, 1, false, false>(A, S.g, s);
    else if (A.in_dtype == CB_F32) launch_f32(A, S, back, s);
    else if (A.in_dtype == CB_F16) launch_f16(A, S, back, s);
    else launch_bf16(A, S, back, s);
    return back ? backward_blocks(A.rows, S.g) : 0;
}

}  // namespace
}  // namespace norm
}  // namespace cbtbe

extern "C" cb_status cb_layer_norm_forward(const void* x, cb_dtype x_dtype, int64_t rows, int64_t dim, int64_t x_row_stride,
                                           const void* weight, cb_dtype weight_dtype, const void* bias, cb_dtype bias_dtype,
                                           float eps, void* out, cb_dtype out_dtype, int64_t out_row_stride, float* mean,
                                           float* rstd, cudaStream_t stream) {
    using namespace cbtbe::norm;
    if (!sizes_ok(rows, dim) || !type_ok(x_dtype) || !type_ok(out_dtype) || !(eps >= 0.f)) return CB_ERR_INVALID_ARG;
    if (!row_ok(rows, dim, x_row_stride) || !row_ok(rows, dim, out_row_stride)) return CB_ERR_INVALID_ARG;
    if ((weight && (!type_ok(weight_dtype) || !aligned(weight, weight_dtype))) ||
        (bias && (!type_ok(bias_dtype) || !aligned(bias, bias_dtype))) || !aligned(mean, CB_F32) || !aligned(rstd, CB_F32))
        return CB_ERR_INVALID_ARG;
    if (rows == 0 || dim == 0) return CB_OK;
    if (!x || !out || !aligned(x, x_dtype) || !aligned(out, out_dtype)) return CB_ERR_INVALID_ARG;
    if (cbtbe::overlap({span(out, out_dtype, rows, dim, out_row_stride), vector(mean, CB_F32, rows), vector(rstd, CB_F32, rows)},
                       {in_place(x, x_dtype, x_row_stride, out, out_dtype, out_row_stride, rows)
                            ? cbtbe::Span()
                            : span(x, x_dtype, rows, dim, x_row_stride),
                        vector(weight, weight_dtype, dim), vector(bias, bias_dtype, dim)}))
        return CB_ERR_INVALID_ARG;
    Args A{};
    A.x = x;
    A.weight = weight;
    A.bias = bias;
    A.out = out;
    A.mean = mean;
    A.rstd = rstd;
    A.rows = rows;
    A.x_row = x_row_stride;
    A.out_row = out_row_stride;
    A.dim = static_cast<int32_t>(dim);
    A.weight_dtype = weight_dtype;
    A.bias_dtype = bias_dtype;
    A.in_dtype = x_dtype;
    A.out_dtype = out_dtype;
    A.eps = eps;
    launch_any(A, false, stream);
    return launched();
}

extern "C" int64_t cb_layer_norm_backward_workspace_bytes(int64_t rows, int64_t dim) {
    using namespace cbtbe::norm;
    if (!sizes_ok(rows, dim)) return 0;
    return partial_rows(rows, dim) * dim * 8;
}

extern "C" cb_status cb_layer_norm_backward(const void* grad_out, const void* x, cb_dtype dtype, int64_t rows, int64_t dim,
                                            int64_t grad_out_row_stride, int64_t x_row_stride, const float* mean,
                                            const float* rstd, const void* weight, cb_dtype weight_dtype, void* grad_x,
                                            cb_dtype grad_x_dtype, int64_t grad_x_row_stride, float* grad_weight,
                                            float* grad_bias, void* workspace, int64_t workspace_bytes, cudaStream_t stream) {
    using namespace cbtbe::norm;
    if (!sizes_ok(rows, dim) || !type_ok(dtype) || !type_ok(grad_x_dtype)) return CB_ERR_INVALID_ARG;
    if (!row_ok(rows, dim, grad_out_row_stride) || !row_ok(rows, dim, x_row_stride) || !row_ok(rows, dim, grad_x_row_stride))
        return CB_ERR_INVALID_ARG;
    if ((weight && (!type_ok(weight_dtype) || !aligned(weight, weight_dtype))) || !aligned(grad_weight, CB_F32) ||
        !aligned(grad_bias, CB_F32))
        return CB_ERR_INVALID_ARG;
    if (dim == 0) return CB_OK;
    if (rows > 0 && (!grad_out || !x || !grad_x || !mean || !rstd || !aligned(grad_out, dtype) || !aligned(x, dtype) ||
                     !aligned(grad_x, grad_x_dtype) || !aligned(mean, CB_F32) || !aligned(rstd, CB_F32)))
        return CB_ERR_INVALID_ARG;
    const bool sums = grad_weight || grad_bias;
    if (sums && rows > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 ||
                             workspace_bytes < cb_layer_norm_backward_workspace_bytes(rows, dim)))
        return CB_ERR_CAPACITY;
    auto input = [&](const void* p, int64_t stride) {
        return in_place(p, dtype, stride, grad_x, grad_x_dtype, grad_x_row_stride, rows) ? cbtbe::Span()
                                                                                        : span(p, dtype, rows, dim, stride);
    };
    if (cbtbe::overlap({span(grad_x, grad_x_dtype, rows, dim, grad_x_row_stride), vector(grad_weight, CB_F32, dim),
                        vector(grad_bias, CB_F32, dim),
                        {workspace, sums && rows > 0 ? cb_layer_norm_backward_workspace_bytes(rows, dim) : 0}},
                       {input(grad_out, grad_out_row_stride), input(x, x_row_stride), vector(mean, CB_F32, rows),
                        vector(rstd, CB_F32, rows), vector(weight, weight_dtype, dim)}))
        return CB_ERR_INVALID_ARG;
    Args A{};
    A.x = x;
    A.dy = grad_out;
    A.weight = weight;
    A.out = grad_x;
    A.mean = const_cast<float*>(mean);
    A.rstd = const_cast<float*>(rstd);
    A.partial = sums ? static_cast<float*>(workspace) : nullptr;
    A.rows = rows;
    A.x_row = x_row_stride;
    A.dy_row = grad_out_row_stride;
    A.out_row = grad_x_row_stride;
    A.dim = static_cast<int32_t>(dim);
    A.weight_dtype = weight_dtype;
    A.in_dtype = dtype;
    A.out_dtype = grad_x_dtype;
    const int64_t parts = rows > 0 ? launch_any(A, true, stream) : 0;
    if (sums)
        cbtbe::launch(layer_norm_join_kernel, dim3(static_cast<unsigned>((2 * dim + 31) / 32)), dim3(kJoinWarps * 32), 0,
                      stream, static_cast<const float*>(A.partial), static_cast<int32_t>(parts), A.dim, grad_weight, grad_bias);
    return launched();
}
