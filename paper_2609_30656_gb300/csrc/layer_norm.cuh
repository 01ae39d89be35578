// layer_norm.cuh -- layer normalisation of rows and its backward pass: the kernels, by type of
// the rows read (one translation unit each; layer_norm.cu has the entry points).
//
//   mean = sum x / D,  r = 1 / sqrt(sum (x - mean)^2 / D + eps),  y = w (x - mean) r + b
//   g = w dy;  dx = r (g - mean(g) - xh mean(g xh)),  dw = sum over rows of dy xh,  db = sum of dy
//
// A byte or two per operation: the copy rate bounds both. A row is read once: a group of 32 to 1024
// threads keeps it in registers, so the variance is a second sum over the kept values (sum x^2 -
// mean^2 would lose what a large mean shares with them) and not a second reading, and the next row's
// values are on their way meanwhile. A thread has the same columns of every row: its weights stay in
// registers, and the gradients of weight and bias are summed there, in fp32, and joined in the order
// of the blocks (the same bits every time).
//
// Rows whose length or stride is no multiple of 16 bytes still lie at every V-th row as the first
// one does (V values in 16 bytes of the narrower type). SHIFTED kernels give each group rows of one
// such class: pieces are then aligned and a thread's columns the same for all of them, only begun
// `shift` columns before the row; the two pieces at a row's ends are written value by value (and read so in fp32).
//
// bf16 rows, 131072 of 4096: 363 us forward, 5.9 TB/s, 87 % of the copy rate; 131072 of 2048 backward: 287 us, 5.6 TB/s (one pass
// of 283 us and the join of the blocks' sums, most of it behind that). 131072 rows of 1001, SHIFTED, and of 1000: fp32 forward 166
// and 157 us, backward 302 and 303; bf16 forward 124 and 93, backward 305 and 156 (two ends of up to seven values each to write).
#pragma once

#include "token_rows.cuh"

#include <algorithm>

namespace cbtbe {
namespace norm {

constexpr int kValues = 16;  // of a row in a thread's registers
constexpr int kMostThreads = 1024;
constexpr int64_t kMaxDim = 1 << 20;
constexpr int kAny = -1;     // types looked up at run time, value by value

struct Args {
    const void* x;
    const void* dy;        // backward
    const void* weight;    // or null
    const void* bias;      // or null
    void* out;             // y, or dx
    float* mean;           // forward: or null
    float* rstd;
    float* partial;        // backward: dw and db of every block, [gridDim.x][2][dim], or null
    int64_t rows, x_row, dy_row, out_row;  // strides in values
    int32_t dim, weight_dtype, bias_dtype, in_dtype, out_dtype;
    int32_t begin, begin_step;  // SHIFTED: row r begins (begin + r * begin_step) % V values behind an aligned piece
    float eps;
};

template <int DT> constexpr int kBytes = DT == CB_F32 ? 4 : 2;
__device__ __forceinline__ float any_value(uint32_t bits, int dtype) {
    return dtype == CB_F32 ? __uint_as_float(bits) : (dtype == CB_BF16 ? widen<CB_BF16>(bits) : widen<CB_F16>(bits));
}
__device__ __forceinline__ uint32_t any_bits(const void* p, int64_t i, int dtype) {
    return dtype == CB_F32 ? static_cast<const uint32_t*>(p)[i] : static_cast<const uint16_t*>(p)[i];
}
__device__ __forceinline__ void any_store(void* p, int64_t i, float v, int dtype) {
    if (dtype == CB_F32) static_cast<float*>(p)[i] = v;
    else static_cast<uint16_t*>(p)[i] = static_cast<uint16_t>(dtype == CB_BF16 ? narrow<CB_BF16>(v) : narrow<CB_F16>(v));
}
__device__ __forceinline__ float load_param(const void* p, int64_t i, int dtype) { return any_value(any_bits(p, i, dtype), dtype); }

// The sums of N values over the G threads of a row's group (a warp, or the whole block). `turn`
// alternates: a warp may begin the next sum while another still reads this one's.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* shared, int& turn) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(kFull, v[k], off);
    if constexpr (G > 32) {
        constexpr int W = G / 32;
        float* s = shared + turn * W * N;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) s[threadIdx.x / 32 * N + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float t = (threadIdx.x & 31) < W ? s[(threadIdx.x & 31) * N + k] : 0.f;
#pragma unroll
            for (int off = W / 2; off >= 1; off >>= 1) t += __shfl_xor_sync(kFull, t, off);
            v[k] = __shfl_sync(kFull, t, 0);
        }
    }
}

template <int G> constexpr int kBlock = G == 32 ? 128 : G;

// A thread's pieces of a row: V values each, piece p G * V columns behind piece p - 1.
template <int DT, bool SHIFTED> constexpr bool kEnds = SHIFTED && (DT == CB_F16 || DT == CB_BF16);  // read whole (read_piece)
template <int DT, int V, int G, bool SHIFTED>
struct Columns {
    int first, dim;
    __device__ __forceinline__ int at(int p) const { return first + p * G * V; }
    __device__ __forceinline__ bool in(int p, int i) const {
        const int c = at(p) + i;
        return SHIFTED ? c >= 0 && c < dim : at(p) < dim;  // without a shift pieces are in whole
    }
    __device__ __forceinline__ bool whole(int p) const { return SHIFTED ? at(p) >= 0 && at(p) + V <= dim : at(p) < dim; }
    __device__ __forceinline__ bool some(int p) const { return at(p) + V > 0 && at(p) < dim; }
    // Values of a piece that are not the row's give 0.
    __device__ __forceinline__ void mask(int p, float (&f)[V]) const {
        if constexpr (kEnds<DT, SHIFTED>)
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = in(p, i) ? f[i] : 0.f;
    }
};

template <int DT, int V> struct RowPiece { Piece<DT, V> v; };
template <int V> struct RowPiece<kAny, V> { uint32_t v; };

template <int DT, int V, int G, bool SHIFTED>
__device__ __forceinline__ void read_piece(RowPiece<DT, V>& to, const Columns<DT, V, G, SHIFTED>& C, int p, const void* x,
                                           int64_t row, int64_t all, int dtype) {
    if constexpr (DT == kAny) {
        to.v = C.in(p, 0) ? any_bits(x, row + C.at(p), dtype) : 0u;
    } else {
        // Halves at a row's end are read as a whole piece too, their neighbours with them (masked where they are used), but for
        // the first and last of all, before and behind which there may be nothing: put together one by one they are waited for,
        // before the row at hand is worked on (131072 rows of 1001 bf16 backward: 446 against 305 us). Words arrive by themselves.
        const int64_t first = row + C.at(p);
        const char* at = static_cast<const char*>(x) + first * kBytes<DT>;
        if (C.whole(p) || (kEnds<DT, SHIFTED> && C.some(p) && first >= 0 && first + V <= all)) {
            to.v = load_piece<DT, V, false>(at);
        } else {
            to.v = zero_piece<DT, V>();
            if constexpr (SHIFTED)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (C.in(p, i)) {
                        const uint32_t bits = any_bits(at, i, DT);
                        if constexpr (DT == CB_F32) to.v.w[i] = bits;
                        else to.v.w[i / 2] |= i & 1 ? bits << 16 : bits;
                    }
        }
    }
}
template <int DT, int V>
__device__ __forceinline__ void piece_values(const RowPiece<DT, V>& p, float (&f)[V], int dtype) {
    if constexpr (DT == kAny) f[0] = any_value(p.v, dtype);
    else widen<DT, V>(p.v, f);
}
template <int OT, int DT, int V, int G, bool SHIFTED>
__device__ __forceinline__ void write_piece(const Columns<DT, V, G, SHIFTED>& C, int p, void* y, int64_t row, const float (&f)[V],
                                            int dtype) {
    if constexpr (OT == kAny) {
        if (C.in(p, 0)) any_store(y, row + C.at(p), f[0], dtype);
    } else {
        char* at = static_cast<char*>(y) + (row + C.at(p)) * kBytes<OT>;
        if (C.whole(p)) {
            store_piece<OT, V>(at, f);
        } else if constexpr (SHIFTED) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (C.in(p, i)) any_store(at, i, f[i], OT);
        }
    }
}

// The group's first row, and the columns of the thread.
template <int DT, int V, int G, bool SHIFTED>
__device__ __forceinline__ Columns<DT, V, G, SHIFTED> columns(const Args& A, int64_t row) {
    Columns<DT, V, G, SHIFTED> C;
    C.first = static_cast<int>(threadIdx.x) % G * V;
    C.dim = A.dim;
    if constexpr (SHIFTED) C.first -= static_cast<int>((A.begin + row % V * A.begin_step) % V);
    return C;
}

template <int DT, int OT, int V, int G, bool SHIFTED>
__global__ void __launch_bounds__(kBlock<G>)
layer_norm_kernel(const Args A) {
    constexpr int P = kValues / V, kAtOnce = kBlock<G> / G;
    __shared__ float shared[G > 32 ? 2 * G / 32 : 1];
    const int64_t step = static_cast<int64_t>(gridDim.x) * kAtOnce;
    int64_t row = static_cast<int64_t>(blockIdx.x) * kAtOnce + threadIdx.x / G;
    const auto C = columns<DT, V, G, SHIFTED>(A, row);
    begin_kernel();
    const int64_t all = (A.rows - 1) * A.x_row + A.dim;
    RowPiece<DT, V> next[P];
    auto load = [&](int64_t r) {
        if (r < A.rows)
#pragma unroll
            for (int p = 0; p < P; ++p) read_piece<DT, V, G, SHIFTED>(next[p], C, p, A.x, r * A.x_row, all, A.in_dtype);
    };
    load(row);
    float w[kValues], b[kValues];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[p * V + i] = A.weight && C.in(p, i) ? load_param(A.weight, C.at(p) + i, A.weight_dtype) : 1.f;
            b[p * V + i] = A.bias && C.in(p, i) ? load_param(A.bias, C.at(p) + i, A.bias_dtype) : 0.f;
        }
    int turn = 0;
    const float inv = 1.f / static_cast<float>(A.dim);
    for (; row < A.rows; row += step) {
        float v[kValues], sum[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float f[V];
            piece_values<DT, V>(next[p], f, A.in_dtype);
            C.mask(p, f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[p * V + i] = f[i];
                sum[0] += f[i];
            }
        }
        load(row + step);
        group_sum<G>(sum, shared, turn);
        const float mean = sum[0] * inv;
        float square[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float& x = v[p * V + i];
                x = C.in(p, i) ? x - mean : 0.f;
                square[0] = fmaf(x, x, square[0]);
            }
        group_sum<G>(square, shared, turn);
        const float rstd = 1.f / sqrtf(fmaf(square[0], inv, A.eps));
        if (threadIdx.x % G == 0) {
            if (A.mean) A.mean[row] = mean;
            if (A.rstd) A.rstd[row] = rstd;
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float f[V];
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = fmaf(v[p * V + i] * rstd, w[p * V + i], b[p * V + i]);
            write_piece<OT, DT, V, G, SHIFTED>(C, p, A.out, row * A.out_row, f, A.out_dtype);
        }
    }
}

template <int DT, int OT, int V, int G, bool SHIFTED>
__global__ void __launch_bounds__(kBlock<G>)
layer_norm_backward_kernel(const Args A) {
    constexpr int P = kValues / V, kAtOnce = kBlock<G> / G;
    __shared__ float shared[G > 32 ? 4 * G / 32 : 1];
    const int64_t step = static_cast<int64_t>(gridDim.x) * kAtOnce;
    int64_t row = static_cast<int64_t>(blockIdx.x) * kAtOnce + threadIdx.x / G;
    const auto C = columns<DT, V, G, SHIFTED>(A, row);
    begin_kernel();
    const int64_t all = (A.rows - 1) * A.x_row + A.dim, dy_all = (A.rows - 1) * A.dy_row + A.dim;
    RowPiece<DT, V> x_next[P], dy_next[P];
    float mean_next = 0.f, rstd_next = 0.f;
    auto load = [&](int64_t r) {
        if (r >= A.rows) return;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            read_piece<DT, V, G, SHIFTED>(x_next[p], C, p, A.x, r * A.x_row, all, A.in_dtype);
            read_piece<DT, V, G, SHIFTED>(dy_next[p], C, p, A.dy, r * A.dy_row, dy_all, A.in_dtype);
        }
        mean_next = A.mean[r];
        rstd_next = A.rstd[r];
    };
    load(row);
    float w[kValues], dw[kValues], db[kValues];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[p * V + i] = A.weight && C.in(p, i) ? load_param(A.weight, C.at(p) + i, A.weight_dtype) : 1.f;
            dw[p * V + i] = db[p * V + i] = 0.f;
        }
    int turn = 0;
    const float inv = 1.f / static_cast<float>(A.dim);
    for (; row < A.rows; row += step) {
        // The row's pieces stay as they were read: half the registers of their values in 32 bits.
        RowPiece<DT, V> x[P], dy[P];
        const float mean = mean_next, rstd = rstd_next;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            x[p] = x_next[p];
            dy[p] = dy_next[p];
            float f[V], d[V];
            piece_values<DT, V>(x[p], f, A.in_dtype);
            piece_values<DT, V>(dy[p], d, A.in_dtype);
            C.mask(p, d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int k = p * V + i;
                const float xh = C.in(p, i) ? (f[i] - mean) * rstd : 0.f, g = d[i] * w[k];
                dw[k] = fmaf(d[i], xh, dw[k]);
                db[k] += d[i];
                sum[0] += g;
                sum[1] = fmaf(g, xh, sum[1]);
            }
        }
        load(row + step);
        group_sum<G>(sum, shared, turn);
        const float m0 = sum[0] * inv, m1 = sum[1] * inv;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float f[V], d[V];
            piece_values<DT, V>(x[p], f, A.in_dtype);
            piece_values<DT, V>(dy[p], d, A.in_dtype);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = rstd * (fmaf(d[i], w[p * V + i], -m0) - (f[i] - mean) * rstd * m1);
            write_piece<OT, DT, V, G, SHIFTED>(C, p, A.out, row * A.out_row, f, A.out_dtype);
        }
    }
    if (!A.partial) return;
    float* mine = A.partial + static_cast<int64_t>(blockIdx.x) * 2 * A.dim;
    if constexpr (kAtOnce > 1) {  // the block's groups, joined in order
        __shared__ float joined[2 * 32 * kValues];
        for (int i = threadIdx.x; i < 2 * 32 * kValues; i += kBlock<G>) joined[i] = 0.f;
        for (int o = 0; o < kAtOnce; ++o) {
            __syncthreads();
            if (static_cast<int>(threadIdx.x) / G != o) continue;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (C.in(p, i)) {
                        joined[C.at(p) + i] += dw[p * V + i];
                        joined[32 * kValues + C.at(p) + i] += db[p * V + i];
                    }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < A.dim; i += kBlock<G>) {
            mine[i] = joined[i];
            mine[A.dim + i] = joined[32 * kValues + i];
        }
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (C.in(p, i)) {
                    mine[C.at(p) + i] = dw[p * V + i];
                    mine[A.dim + C.at(p) + i] = db[p * V + i];
                }
    }
}

// Threads for a row of `span` columns, 0 where registers do not hold it.
inline int group_threads(int64_t span) {
    int g = 32;
    while (static_cast<int64_t>(g) * kValues < span) g *= 2;
    return g <= kMostThreads ? g : 0;
}
int sm_count();
// Blocks of the backward pass: each leaves a row of sums. A multiple of 8, so that SHIFTED
// groups keep their class, unless one turn is enough.
constexpr int kBackwardThreads = 512;  // of an SM
inline int64_t backward_blocks(int64_t rows, int g) {
    const int block = g == 32 ? 128 : g, at_once = block / g;
    const int64_t most = static_cast<int64_t>(sm_count()) * std::max(1, kBackwardThreads / block) / 8 * 8;
    return std::min<int64_t>((rows + at_once - 1) / at_once, most);
}

template <int DT, int OT, int V, int G, bool SHIFTED, bool BACK>
void launch_rows(const Args& A, cudaStream_t s) {
    constexpr int block = kBlock<G>, at_once = block / G;
    if constexpr (BACK) {
        launch(layer_norm_backward_kernel<DT, OT, V, G, SHIFTED>, dim3(static_cast<unsigned>(backward_blocks(A.rows, G))),
               dim3(block), 0, s, A);
    } else {
        const int64_t most = static_cast<int64_t>(sm_count()) *
                             resident_blocks(layer_norm_kernel<DT, OT, V, G, SHIFTED>, block) / 8 * 8;
        launch(layer_norm_kernel<DT, OT, V, G, SHIFTED>,
               dim3(static_cast<unsigned>(std::min<int64_t>((A.rows + at_once - 1) / at_once, most))), dim3(block), 0, s, A);
    }
}
template <int DT, int OT, int V, bool SHIFTED, bool BACK>
void launch_group(const Args& A, int g, cudaStream_t s) {
    switch (g) {
        case 32: return launch_rows<DT, OT, V, 32, SHIFTED, BACK>(A, s);
        case 64: return launch_rows<DT, OT, V, 64, SHIFTED, BACK>(A, s);
        case 128: return launch_rows<DT, OT, V, 128, SHIFTED, BACK>(A, s);
        case 256: return launch_rows<DT, OT, V, 256, SHIFTED, BACK>(A, s);
        case 512: return launch_rows<DT, OT, V, 512, SHIFTED, BACK>(A, s);
        default: return launch_rows<DT, OT, V, 1024, SHIFTED, BACK>(A, s);
    }
}

// How a call's rows are read: V values at a time and whether they are SHIFTED; g threads a row.
struct Shape {
    int v, g;  // g = 0: rows longer than registers hold
    bool shifted;
};
template <int DT, int OT, bool BACK>
void launch_typed(const Args& A, const Shape& S, cudaStream_t s) {
    constexpr int V = DT == CB_F32 && OT == CB_F32 ? 4 : 8;
    if (S.shifted) launch_group<DT, OT, V, true, BACK>(A, S.g, s);
    else launch_group<DT, OT, V, false, BACK>(A, S.g, s);
}

// By the type of the rows read; S.v is not 1.
void launch_f32(const Args& A, const Shape& S, bool back, cudaStream_t s);
void launch_f16(const Args& A, const Shape& S, bool back, cudaStream_t s);
void launch_bf16(const Args& A, const Shape& S, bool back, cudaStream_t s);

}  // namespace norm
}  // namespace cbtbe
