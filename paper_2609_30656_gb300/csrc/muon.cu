// muon.cu -- approximate orthogonalisation of matrix updates by Newton-Schulz
// products, alone and inside an optimizer step with momentum and weight decay.
//
// For a matrix G, X_0 the one of G and G^T with no more rows than columns (p <= q),
// divided by ||G||_F + eps, and for every step with its coefficients (a, b, c)
//     A = X X^T,   B = b A + c A A,   X <- a X + B X,
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the
// singular vectors as they are. A step is 3 p^2 q + p^3 operations when the symmetry of A
// and of A A is used (tiles of the lower triangle, stored to both), against p q values read
// and written: beyond sizes of a few hundred it is bound by the products.
//
// Numbers. The products take fp16 operands and sum in fp32. fp16 rather than bf16:
// both run at one rate, every matrix here is bounded (|x| <= ||X||_2 <= about 1.3 under
// the usual coefficients), so the exponent's range is not needed, and the three more
// bits are. Rounding X puts noise into its small singular directions, which every
// step multiplies by a while they are small; updates are like that, a few strong directions
// over a floor that still grows in the last step. So X is kept as the sum of two fp16 values,
// X = hi + lo, 22 bits, for the term a X, and the products take hi alone: their error is
// filtered by B, which vanishes on the small directions. B is rounded with a multiple of I added
// that keeps its diagonal small (diagonal_shift), which is taken off the term again:
//     X' = (B + s I) hi + (a - s) hi + a lo.
// Off the exact result in the 2-norm (260 matrices of random sizes, shorter side 16 to 1100, usual
// coefficients): singular values of 1 for one direction, an eighth, half or nine tenths of them over
// a floor of 1e-6 to 1e-1, at most 1.9e-3, 1.7e-3, 2.4e-3 and 2.8e-3; Gaussian matrices 2.2e-3; singular
// values all alike 2.7e-3 (the roundings of equal diagonals add up); medians 4e-4 to 1.7e-3. Constant
// matrices, all of whose roundings add up, 1.3e-2. With lo in the first two steps only and a I in
// B after them, 1.4e-2 over a floor; with no shift 4.2e-3 for values all alike; in bf16 8 times as much.
// Keeping lo throughout costs traffic in the updates' epilogues: a step of 4 x 1024 x 4096 383 -> 444 us, five
// steps of 1024 x 1024 109 -> 111, of 2048 x 2048 218 -> 231, of 4096 x 4096 1099 -> 1144, of 128 x 256
// 44 -> 47. (Times at the kernels compare forms with lo in two steps.)
// X is held times 2^10 and A and B times 2^8 (powers of two: exact), which keeps their small
// values out of fp16's subnormal range and leaves a factor of 40 and
// more below its largest value: X up to 63, A and B up to 255 in any element.
//
// The norm. Squares are summed in three classes of magnitude, each scaled to stay in
// range, so that no finite matrix overflows or underflows it; where more than one
// counts they are joined in fp64.
//
// Layout in the workspace: X as [p, q] with rows padded to 64 values, A and B as [p, p]
// likewise. The transposition of a tall matrix is done where it is read (muon_cast_kernel) and
// where the result is written (the last product's epilogue), so the products exist in
// one orientation only.
#include "muon_internal.cuh"

namespace cbtbe {
namespace muon {
namespace {

// ---------------------------------------------------------------- norm

constexpr int kNormThreads = 512;
constexpr int kNormBlocks = 304;  // most blocks (and partial sums) per matrix

// m <- beta m + g in place, and a block's part of the squares of the update u
// (g; m; or g + beta m). Blocks (x of a matrix, matrix).
template <int V>
__global__ void __launch_bounds__(kNormThreads) muon_norm_kernel(MatrixIn in, SquareSum* __restrict__ partial, int* fault) {
    begin_kernel();
    const int b = blockIdx.y;
    const char* g = static_cast<const char*>(in.g) + b * in.g_batch * dtype_bytes(in.dtype);
    float* mom = in.momentum ? in.momentum + b * in.m_batch : nullptr;
    const int vecs = in.cols / V;
    const int64_t total = static_cast<int64_t>(in.rows) * vecs;
    const int64_t step = static_cast<int64_t>(gridDim.x) * kNormThreads;
    SquareSum s;
    int64_t i = static_cast<int64_t>(blockIdx.x) * kNormThreads + threadIdx.x;
    int64_t row = i / vecs;
    int col = static_cast<int>(i - row * vecs);
    const int64_t drow = step / vecs;
    const int dcol = static_cast<int>(step - drow * vecs);
    constexpr int U = V == 8 ? 2 : 4;  // vectors in flight
    while (i < total) {
        float v[U][V], m[U][V];
        int64_t at_m[U];
        int live = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i < total) {
                live = u + 1;
                load_values<V>(g, row * in.g_row + static_cast<int64_t>(col) * V, in.dtype, v[u]);
                at_m[u] = row * in.m_row + static_cast<int64_t>(col) * V;
                if (mom) load_values<V>(mom, at_m[u], CB_F32, m[u]);
            }
            i += step;
            row += drow;
            col += dcol;
            if (col >= vecs) {
                col -= vecs;
                ++row;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u < live) {
                if (mom) {
#pragma unroll
                    for (int k = 0; k < V; ++k) v[u][k] = update_value(in, v[u][k], m[u][k]);
                    if constexpr (V == 1) {
                        mom[at_m[u]] = m[u][0];
                    } else {
#pragma unroll
                        for (int k = 0; k < V; k += 4)
                            *reinterpret_cast<float4*>(mom + at_m[u] + k) =
                                make_float4(m[u][k], m[u][k + 1], m[u][k + 2], m[u][k + 3]);
                    }
                }
                s.add(v[u]);
            }
        }
    }
    __shared__ __align__(16) unsigned char raw[kNormThreads / 32 * sizeof(SquareSum)];
    SquareSum* sh = reinterpret_cast<SquareSum*>(raw);
    s.add_lanes();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < kNormThreads / 32; ++w) s.add(sh[w]);
        partial[static_cast<int64_t>(b) * kNormBlocks + blockIdx.x] = s;
        if (b == 0 && blockIdx.x == 0) *fault = 0;  // for the call's products
    }
}

// The same from the partial sums of one matrix, by a block of 256 threads. One thread finishes
// it (every block of a large matrix does this; 140 us for 4096 x 4096 when all threads did).
__device__ __forceinline__ float2 inverse_norm(const SquareSum* partial, int blocks, float eps) {
    __shared__ __align__(16) unsigned char raw[8 * sizeof(SquareSum)];
    SquareSum* sh = reinterpret_cast<SquareSum*>(raw);
    __shared__ float2 result;
    SquareSum t;
    for (int k = threadIdx.x; k < blocks; k += 256) t.add(partial[k]);
    t.add_lanes();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < 8; ++w) t.add(sh[w]);
        result = inverse_norm(t, eps);
    }
    __syncthreads();
    return result;
}

// ---------------------------------------------------------------- cast

constexpr int kCastTile = 64;

// X_0 = kScaleX u / (||u|| + eps) as hi + lo, [p, ld] rows: u as it lies, or transposed.
// A block takes a 64 x 64 tile of u, a thread 16 values of it in runs of 4, or of 8 (V = 4 or 8: in
// one load or two each), and of X, one row of tiles after another: blocks (column tile, first row tile,
// matrix). Rows of X are padded to 64 values, so its tiles are stored whole along a row.
template <bool TRANSPOSED, int V>
__global__ void __launch_bounds__(256, 4) muon_cast_kernel(MatrixIn in, const SquareSum* __restrict__ partial, int norm_blocks,
                                                        float eps, __half* __restrict__ hi, __half* __restrict__ lo,
                                                        int ld, int64_t x_batch) {
    __shared__ float tile[TRANSPOSED ? kCastTile : 1][kCastTile + 1];
    begin_kernel();
    const int b = blockIdx.z, c0 = blockIdx.x * kCastTile;
    const char* g = static_cast<const char*>(in.g) + b * in.g_batch * dtype_bytes(in.dtype);
    const float* mom = in.momentum ? in.momentum + b * in.m_batch : nullptr;
    constexpr int N = V == 8 ? 8 : 4, R = 16 / N, kLanes = kCastTile / N, kDown = 256 / kLanes;  // R runs of N values
    const int c = threadIdx.x % kLanes * N, rq = threadIdx.x / kLanes;
    float2 f = make_float2(0.f, 0.f);
    for (int r0 = blockIdx.y * kCastTile; r0 < in.rows; r0 += gridDim.y * kCastTile) {
        float v[R][N], m[R][N];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t row = r0 + rq + kDown * k;
#pragma unroll
            for (int e = 0; e < N; ++e) v[k][e] = m[k][e] = 0.f;
            if (row >= in.rows) continue;
            if constexpr (V > 1) {
                if (c0 + c < in.cols) {
                    load_values<V>(g, row * in.g_row + c0 + c, in.dtype, v[k]);
                    if (mom) load_values<V>(mom, row * in.m_row + c0 + c, CB_F32, m[k]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (c0 + c + e < in.cols) {
                        v[k][e] = load_value(g, row * in.g_row + c0 + c + e, in.dtype);
                        if (mom) m[k][e] = mom[row * in.m_row + c0 + c + e];
                    }
            }
        }
        if (mom) {
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int e = 0; e < N; ++e) v[k][e] = in.nesterov ? mix_momentum(m[k][e], v[k][e], in.beta) : m[k][e];
        }
        if (r0 == static_cast<int>(blockIdx.y) * kCastTile)  // behind the first tile's loads
            f = inverse_norm(partial + static_cast<int64_t>(b) * kNormBlocks, norm_blocks, eps);
        auto put = [&](int64_t at, const float (&x)[N]) {
            uint32_t h[N / 2], l[N / 2];
#pragma unroll
            for (int e = 0; e < N / 2; ++e) {
                const __half2 top = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
                const float2 back = __half22float2(top);
                const __half2 rest = __floats2half2_rn(x[2 * e] - back.x, x[2 * e + 1] - back.y);
                memcpy(&h[e], &top, 4);
                memcpy(&l[e], &rest, 4);
            }
            if constexpr (N == 8) {
                *reinterpret_cast<uint4*>(hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
                *reinterpret_cast<uint4*>(lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
            } else {
                *reinterpret_cast<uint2*>(hi + at) = make_uint2(h[0], h[1]);
                *reinterpret_cast<uint2*>(lo + at) = make_uint2(l[0], l[1]);
            }
        };
        const int64_t base = b * x_batch;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int row = r0 + rq + kDown * k;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = (v[k][e] * f.x) * f.y;
                if constexpr (TRANSPOSED) tile[rq + kDown * k][c + e] = x[e];
            }
            if (!TRANSPOSED && row < in.rows) put(base + static_cast<int64_t>(row) * ld + c0 + c, x);
        }
        if constexpr (TRANSPOSED) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const int col = c0 + rq + kDown * k;  // value (row, col) of u is X[col, row]
                float x[N];
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = tile[c + e][rq + kDown * k];
                if (col < in.cols) put(base + static_cast<int64_t>(col) * ld + r0 + c, x);
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------- host

struct Workspace {
    int64_t p, q, ldx, lda;
    size_t hi[2], lo[2], gram, poly, partial, fault, bytes;
};
// Sizes come in 64 bits, so that one past 32 is refused and not cut off on its way here.
bool valid_sizes(int64_t batch, int64_t rows, int64_t cols) {
    return batch >= 0 && batch <= 65535 && rows >= 0 && rows <= (1 << 20) && cols >= 0 && cols <= (1 << 20) &&
           (batch == 0 || rows * cols <= (int64_t(1) << 38) / batch);
}
Workspace layout(int32_t batch, int32_t rows, int32_t cols) {
    Workspace w;
    w.p = rows < cols ? rows : cols;
    w.q = rows < cols ? cols : rows;
    w.ldx = round_up(w.q, 64);
    w.lda = round_up(w.p, 64);
    size_t at = 0;
    auto take = [&](int64_t bytes) {
        const size_t here = at;
        at += static_cast<size_t>(round_up(bytes, 256));
        return here;
    };
    const bool small = small_blocks(w.p, w.q) > 0;  // one kernel, which keeps all in its blocks
    const int64_t x = small ? 0 : batch * w.p * w.ldx * 2, a = small ? 0 : batch * w.p * w.lda * 2;
    w.hi[0] = take(x);
    w.hi[1] = take(x);
    w.lo[0] = take(x);
    w.lo[1] = take(x);
    w.gram = take(a);
    w.poly = take(a);
    w.partial = take(small ? 0 : static_cast<int64_t>(batch) * kNormBlocks * static_cast<int64_t>(sizeof(SquareSum)));
    w.fault = take(4);
    w.bytes = at;
    return w;
}

bool current_sms(int* sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess &&
        cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && *sms > 0)
        return true;
    cudaGetLastError();
    return false;
}

bool valid_dtype(int d) { return d == CB_F32 || d == CB_F16 || d == CB_BF16; }

struct Result {
    void* data;
    cb_dtype dtype;
    int64_t batch_stride, row_stride;
    bool weights;
    float keep, rate;
};

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

cb_status orthogonalise(const MatrixIn& in, int32_t batch, float eps, const float* coefficients, int32_t steps,
                        const Result& out, void* workspace, int64_t workspace_bytes, int* error, cudaStream_t s) {
    if (steps < 1 || steps > kMaxSteps || !coefficients || !(eps >= 0.f) || !valid_dtype(in.dtype) ||
        !valid_dtype(out.dtype))
        return CB_ERR_INVALID_ARG;
    for (int k = 0; k < 3 * steps; ++k)
        if (!std::isfinite(coefficients[k])) return CB_ERR_INVALID_ARG;
    if (batch == 0 || in.rows == 0 || in.cols == 0) return CB_OK;
    const int64_t matrix = static_cast<int64_t>(in.rows) * in.cols;
    // What is written is written by many blocks at once: no value may be two matrices'.
    if (!in.g || !out.data || in.g_row < in.cols || out.row_stride < in.cols || (batch > 1 && in.g_batch < 0) ||
        !rows_apart(batch, out.batch_stride, in.rows, out.row_stride, in.cols))
        return CB_ERR_INVALID_ARG;
    if (in.momentum && (in.m_row < in.cols || !rows_apart(batch, in.m_batch, in.rows, in.m_row, in.cols)))
        return CB_ERR_INVALID_ARG;
    if (!aligned(in.g, dtype_bytes(in.dtype)) || !aligned(out.data, dtype_bytes(out.dtype)) ||
        !aligned(in.momentum, 4) || !aligned(error, 4))
        return CB_ERR_INVALID_ARG;
    const bool tall = in.rows > in.cols;
    auto vectors_of = [&](int v) {
        return in.cols % v == 0 && in.g_row % v == 0 && (batch == 1 || in.g_batch % v == 0) &&
               aligned(in.g, min64(16, v * dtype_bytes(in.dtype))) &&
               (!in.momentum ||
                (in.m_row % v == 0 && (batch == 1 || in.m_batch % v == 0) && aligned(in.momentum, 16)));
    };
    const bool vector = vectors_of(4), wide = vectors_of(8);
    const bool user_vector = in.cols % 4 == 0 && out.row_stride % 4 == 0 && (batch == 1 || out.batch_stride % 4 == 0) &&
                             aligned(out.data, 4 * dtype_bytes(out.dtype));
    const bool user_wide = out.dtype != CB_F32 && in.cols % 8 == 0 && out.row_stride % 8 == 0 &&
                           (batch == 1 || out.batch_stride % 8 == 0) && aligned(out.data, 16);
    const int sector = 32 / dtype_bytes(out.dtype);  // values
    const bool user_sectors = !tall && in.cols % sector == 0 && out.row_stride % sector == 0 &&
                              (batch == 1 || out.batch_stride % sector == 0) && aligned(out.data, 32);
    const Workspace w = layout(batch, in.rows, in.cols);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < static_cast<int64_t>(w.bytes)) return CB_ERR_CAPACITY;
    char* base = static_cast<char*>(workspace);
    if (const int blocks = small_blocks(w.p, w.q)) {
        SmallArgs P{};
        P.p = static_cast<int32_t>(w.p);
        P.q = static_cast<int32_t>(w.q);
        P.cols = static_cast<int32_t>(round_up((w.q + blocks - 1) / blocks, 64));
        P.transposed = tall;
        P.blocks = blocks;
        P.steps = steps;
        P.eps = eps;
        for (int k = 0; k < 3 * steps; ++k) P.coefficients[k] = coefficients[k];
        for (int k = 0; k < steps; ++k) P.shift[k] = diagonal_shift(coefficients[3 * k + 1], coefficients[3 * k + 2]);
        P.user = out.data;
        P.user_batch = out.batch_stride;
        P.user_row = out.row_stride;
        P.user_dtype = out.dtype;
        P.user_vector = user_vector;
        P.in_vector = vector;
        P.weights = out.weights;
        P.keep = out.keep;
        P.rate = out.rate;
        P.error = error;
        int sms = 0;
        const bool sent = current_sms(&sms) && launch_small(in, P, batch, sms, s);
        return cudaGetLastError() == cudaSuccess && sent ? CB_OK : CB_ERR_CUDA;
    }
    int sms = 0;
    if (!current_sms(&sms) || !tensor_maps_work()) return CB_ERR_CUDA;
    __half* hi[2] = {reinterpret_cast<__half*>(base + w.hi[0]), reinterpret_cast<__half*>(base + w.hi[1])};
    __half* lo[2] = {reinterpret_cast<__half*>(base + w.lo[0]), reinterpret_cast<__half*>(base + w.lo[1])};
    __half* gram = reinterpret_cast<__half*>(base + w.gram);
    __half* poly = reinterpret_cast<__half*>(base + w.poly);
    SquareSum* partial = reinterpret_cast<SquareSum*>(base + w.partial);
    int* fault = reinterpret_cast<int*>(base + w.fault);

    Operand op_x[2], op_gram, op_poly;
    if (!op_x[0].set(hi[0], w.q, w.p, batch, w.ldx) || !op_x[1].set(hi[1], w.q, w.p, batch, w.ldx) ||
        !op_gram.set(gram, w.p, w.p, batch, w.lda) || !op_poly.set(poly, w.p, w.p, batch, w.lda))
        return CB_ERR_CUDA;

    // 8192 values a block, on up to 2 blocks per SM in all.
    const int norm_blocks = static_cast<int>(
        max64(1, min64(min64(kNormBlocks, 2 * sms / batch), (matrix + 8 * 1024 - 1) / (8 * 1024))));
    const dim3 norm_grid(norm_blocks, batch);
    if (wide) launch(muon_norm_kernel<8>, norm_grid, dim3(kNormThreads), 0, s, in, partial, fault);
    else if (vector) launch(muon_norm_kernel<4>, norm_grid, dim3(kNormThreads), 0, s, in, partial, fault);
    else launch(muon_norm_kernel<1>, norm_grid, dim3(kNormThreads), 0, s, in, partial, fault);
    const int cast_cols = (in.cols + kCastTile - 1) / kCastTile, cast_rows = (in.rows + kCastTile - 1) / kCastTile;
    const dim3 cast_grid(cast_cols,
                         static_cast<unsigned>(max64(1, min64(cast_rows, 8 * sms / (static_cast<int64_t>(cast_cols) * batch)))),
                         batch);
    const int64_t x_batch = w.p * w.ldx, a_batch = w.p * w.lda;
    const int ldx = static_cast<int>(w.ldx), lda = static_cast<int>(w.lda);
    auto cast = tall ? (wide ? muon_cast_kernel<true, 8> : vector ? muon_cast_kernel<true, 4> : muon_cast_kernel<true, 1>)
                     : (wide     ? muon_cast_kernel<false, 8>
                        : vector ? muon_cast_kernel<false, 4>
                                 : muon_cast_kernel<false, 1>);
    launch(cast, cast_grid, dim3(256), 0, s, in, static_cast<const SquareSum*>(partial), norm_blocks, eps, hi[0], lo[0], ldx,
           x_batch);

    bool sent = true;
    for (int k = 0; k < steps; ++k) {
        const int now = k & 1, next = now ^ 1;
        const float a = coefficients[3 * k], b = coefficients[3 * k + 1], c = coefficients[3 * k + 2];
        ProductArgs P{};
        P.batch = batch;
        P.error = error;
        P.fault = fault;
        P.m = P.n = static_cast<int32_t>(w.p);
        P.k = static_cast<int32_t>(w.q);
        P.parts = gram_parts(w.p, w.q);
        P.out_hi = gram;
        P.out_batch = a_batch;
        P.out_ld = lda;
        sent &= launch_product(kGram, op_x[now], op_x[now], P, sms, s);
        P.k = P.m;
        P.a = a;
        P.b = b;
        P.c = c;
        P.shift = diagonal_shift(b, c);
        P.term_hi = gram;
        P.term_batch = a_batch;
        P.term_ld = lda;
        P.out_hi = poly;
        sent &= launch_product(kPoly, op_gram, op_gram, P, sms, s);
        P.n = static_cast<int32_t>(w.q);
        P.term_hi = hi[now];
        P.term_lo = lo[now];
        P.term_batch = x_batch;
        P.term_ld = ldx;
        P.out_hi = hi[next];
        P.out_lo = lo[next];
        P.out_batch = x_batch;
        P.out_ld = ldx;
        if (k + 1 < steps) {
            sent &= launch_product(kUpdate, op_poly, op_x[now], P, sms, s);
        } else {
            P.user = out.data;
            P.user_batch = out.batch_stride;
            P.user_row = out.row_stride;
            P.user_dtype = out.dtype;
            P.transposed = tall;
            P.user_vector = user_wide ? 8 : user_vector ? 4 : 0;
            P.user_sectors = user_sectors;
            P.weights = out.weights;
            P.keep = out.keep;
            P.rate = out.rate;
            sent &= launch_product(kResult, op_poly, op_x[now], P, sms, s);
        }
    }
    return cudaGetLastError() == cudaSuccess && sent ? CB_OK : CB_ERR_CUDA;
}

}  // namespace
}  // namespace muon
}  // namespace cbtbe

extern "C" int64_t cb_muon_workspace_bytes(int64_t batch, int64_t rows, int64_t cols) {
    using namespace cbtbe::muon;
    if (!valid_sizes(batch, rows, cols) || batch == 0 || rows == 0 || cols == 0) return 0;
    return static_cast<int64_t>(
        layout(static_cast<int32_t>(batch), static_cast<int32_t>(rows), static_cast<int32_t>(cols)).bytes);
}

extern "C" cb_status cb_muon_orthogonalise(const void* g, cb_dtype g_dtype, int64_t batch, int64_t rows, int64_t cols,
                                           int64_t g_batch_stride, int64_t g_row_stride, float eps,
                                           const float* coefficients, int32_t steps, void* out, cb_dtype out_dtype,
                                           int64_t out_batch_stride, int64_t out_row_stride, void* workspace,
                                           int64_t workspace_bytes, int* error, cudaStream_t stream) {
    using namespace cbtbe::muon;
    if (!valid_sizes(batch, rows, cols)) return CB_ERR_INVALID_ARG;
    MatrixIn in{};
    in.g = g;
    in.g_batch = g_batch_stride;
    in.g_row = g_row_stride;
    in.dtype = g_dtype;
    in.rows = static_cast<int32_t>(rows);
    in.cols = static_cast<int32_t>(cols);
    const Result r{out, out_dtype, out_batch_stride, out_row_stride, false, 0.f, 0.f};
    return orthogonalise(in, static_cast<int32_t>(batch), eps, coefficients, steps, r, workspace, workspace_bytes, error, stream);
}

extern "C" cb_status cb_muon_step(void* weights, cb_dtype w_dtype, int64_t w_batch_stride, int64_t w_row_stride,
                                  const void* g, cb_dtype g_dtype, int64_t g_batch_stride, int64_t g_row_stride,
                                  float* momentum, int64_t m_batch_stride, int64_t m_row_stride, int64_t batch,
                                  int64_t rows, int64_t cols, float lr, float weight_decay, float beta, int nesterov,
                                  float eps, const float* coefficients, int32_t steps, float update_scale,
                                  void* workspace, int64_t workspace_bytes, int* error, cudaStream_t stream) {
    using namespace cbtbe::muon;
    if (!valid_sizes(batch, rows, cols) || !(lr == lr) || !(weight_decay == weight_decay) || !(beta >= 0.f) || !(update_scale == update_scale))
        return CB_ERR_INVALID_ARG;
    if (!momentum && batch > 0 && rows > 0 && cols > 0) return CB_ERR_INVALID_ARG;
    MatrixIn in{};
    in.g = g;
    in.momentum = momentum;
    in.g_batch = g_batch_stride;
    in.g_row = g_row_stride;
    in.m_batch = m_batch_stride;
    in.m_row = m_row_stride;
    in.dtype = g_dtype;
    in.rows = static_cast<int32_t>(rows);
    in.cols = static_cast<int32_t>(cols);
    in.beta = beta;
    in.nesterov = nesterov;
    const Result r{weights, w_dtype, w_batch_stride, w_row_stride, true,
                   static_cast<float>(1.0 - static_cast<double>(lr) * weight_decay),
                   static_cast<float>(static_cast<double>(lr) * update_scale)};
    return orthogonalise(in, static_cast<int32_t>(batch), eps, coefficients, steps, r, workspace, workspace_bytes, error, stream);
}
