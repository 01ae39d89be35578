// muon.cu -- approximate orthogonalisation of matrix updates by Newton-Schulz
// products, alone and inside an optimizer step with momentum and weight decay.
//
// For a matrix G, X_0 the one of G and G^T with no more rows than columns (p <= q),
// divided by ||G||_F + eps, and for every step with its coefficients (a, b, c)
//     A = X X^T,   B = b A + c A A,   X <- a X + B X,
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the
// singular vectors as they are. A step is 2 p^2 q + p^3 multiply-adds when the
// symmetry of A and of A A is used, against p q values read and written: beyond
// sizes of a few hundred it is bound by the tensor cores.
//
// Numbers. The products take fp16 operands and sum in fp32. fp16 rather than bf16:
// both run at one rate, every matrix here is bounded (|x| <= ||X||_2 <= about 1.3 under
// the usual coefficients), so the exponent's range is not needed, and the three more
// bits are: rounding X puts noise into its small singular directions, which the first
// steps multiply by a each (1.2e-2 off the exact result in the 2-norm with bf16, 3e-3
// with fp16, sizes 128 to 2048). The rest of that noise goes by keeping X as the sum of
// two fp16 values, X = hi + lo, for the term a X of the first two steps (1e-3); the
// products take hi alone, since their error is filtered by B, which vanishes on the
// small directions. From the third step on the term is folded into B (B + a I), and X is
// hi alone. X is held times 2^10 and A and B times 2^8 (powers of two: exact), which
// keeps their small values out of fp16's subnormal range and leaves a factor of 40 and
// more below its largest value.
//
// The norm. Squares are summed in three classes of magnitude, each scaled to stay in
// range, so that no finite matrix overflows or underflows it.
//
// Layout in the workspace: X as [p, q] with rows padded to 64 values, A and B as [p, p]
// likewise. The transposition of a tall matrix is done where it is read (cast_kernel) and
// where the result is written (the last product's epilogue), so the products exist in
// one orientation only.
#include "tbe_internal.cuh"
#include "tensor_core.cuh"

#include <cmath>
#include <cudaTypedefs.h>

namespace cbtbe {
namespace {

constexpr float kScaleX = 1024.f;  // X is stored times this,
constexpr float kScaleA = 256.f;   // A and B times this
constexpr int kTwoTerm = 2;        // steps whose term a X takes hi + lo
constexpr int kMaxSteps = 64;

// ---------------------------------------------------------------- norm and momentum

// x^2 summed by magnitude: |x| >= 2^40 times 2^-160, |x| < 2^-40 times 2^160, the rest
// as it is, with what its additions and squares round off kept beside it: the norm then is
// the same whatever the order of its sum (for a transposed or strided matrix, too). A NaN
// goes with the rest.
struct SquareSum {
    float mid = 0.f, rest = 0.f, big = 0.f, small = 0.f;
    __device__ __forceinline__ void add_mid(float x) {  // the exact error of a sum of two floats
        const float t = mid + x, y = t - mid;
        rest += (mid - (t - y)) + (x - y);
        mid = t;
    }
    __device__ __forceinline__ void add(float x) {
        const float m = fabsf(x);
        if (m >= 0x1p40f) {
            const float y = x * 0x1p-80f;
            big = fmaf(y, y, big);
        } else if (m < 0x1p-40f) {
            const float y = x * 0x1p80f;
            small = fmaf(y, y, small);
        } else {
            const float p = x * x;
            rest += fmaf(x, x, -p);
            add_mid(p);
        }
    }
    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N]) {  // the usual magnitudes without a branch for each
        bool usual = true;
#pragma unroll
        for (int k = 0; k < N; ++k) usual &= x[k] == 0.f || (fabsf(x[k]) >= 0x1p-40f && fabsf(x[k]) < 0x1p40f);
        if (usual) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float p = x[k] * x[k];
                rest += fmaf(x[k], x[k], -p);
                add_mid(p);
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) add(x[k]);
        }
    }
    __device__ __forceinline__ void add(const SquareSum& o) {
        add_mid(o.mid);
        rest += o.rest;
        big += o.big;
        small += o.small;
    }
    __device__ __forceinline__ void add_lanes() {  // lane 0 gets the warp's sum
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) {
            SquareSum o;
            o.mid = __shfl_down_sync(kFull, mid, off);
            o.rest = __shfl_down_sync(kFull, rest, off);
            o.big = __shfl_down_sync(kFull, big, off);
            o.small = __shfl_down_sync(kFull, small, off);
            add(o);
        }
    }
};

struct MatrixIn {
    const void* g;         // the gradient, of dtype
    float* momentum;       // or null: the update is g itself
    int64_t g_batch, g_row, m_batch, m_row;  // strides in values
    int32_t dtype;
    int32_t rows, cols;
    float beta;
    int32_t nesterov;
};

__device__ __forceinline__ float load_value(const void* p, int64_t i, int dtype) {
    if (dtype == CB_F32) return static_cast<const float*>(p)[i];
    const uint16_t h = static_cast<const uint16_t*>(p)[i];
    if (dtype == CB_BF16) return __uint_as_float(static_cast<uint32_t>(h) << 16);
    __half x;
    memcpy(&x, &h, 2);
    return __half2float(x);
}
__device__ __forceinline__ void store_value(void* p, int64_t i, float v, int dtype) {
    if (dtype == CB_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == CB_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
template <int DT>
__device__ __forceinline__ void store_values4(void* p, int64_t i, const float (&v)[4]) {
    if constexpr (DT == CB_F32) {
        *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        uint2 w;
        if constexpr (DT == CB_BF16) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
            memcpy(&w.x, &a, 4);
            memcpy(&w.y, &b, 4);
        } else {
            const __half2 a = __floats2half2_rn(v[0], v[1]), b = __floats2half2_rn(v[2], v[3]);
            memcpy(&w.x, &a, 4);
            memcpy(&w.y, &b, 4);
        }
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = w;
    }
}

// V consecutive values (V = 1, or 4 or 8 with the alignment of 16 bytes or of all of them).
template <int V>
__device__ __forceinline__ void load_values(const void* p, int64_t i, int dtype, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = load_value(p, i, dtype);
    } else if constexpr (V == 8) {
        if (dtype == CB_F32) {
            const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
            const float4 x = q[0], y = q[1];
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
            v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        } else {
            const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
            if (dtype == CB_BF16) unpack<CB_BF16>(x, v);
            else unpack<CB_F16>(x, v);
        }
    } else if (dtype == CB_F32) {
        const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
        const uint32_t w[2] = {x.x, x.y};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (dtype == CB_BF16) {
                v[2 * k] = __uint_as_float(w[k] << 16);
                v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            } else {
                __half2 h;
                memcpy(&h, &w[k], 4);
                const float2 f = __half22float2(h);
                v[2 * k] = f.x;
                v[2 * k + 1] = f.y;
            }
        }
    }
}

__host__ __device__ __forceinline__ float mix_momentum(float m, float g, float beta) { return fmaf(beta, m, g); }
// m <- beta m + g, and the update from it.
__device__ __forceinline__ float update_value(const MatrixIn& in, float g, float& m) {
    m = mix_momentum(m, g, in.beta);
    return in.nesterov ? mix_momentum(m, g, in.beta) : m;
}

constexpr int kNormThreads = 512;
constexpr int kNormBlocks = 304;  // most blocks (and partial sums) per matrix

// m <- beta m + g in place, and a block's part of the squares of the update u
// (g; m; or g + beta m). Blocks (x of a matrix, matrix).
template <int V>
__global__ void __launch_bounds__(kNormThreads) muon_norm_kernel(MatrixIn in, SquareSum* __restrict__ partial) {
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
    }
}

// kScaleX / (norm + eps) as a product of two floats, so that neither a huge nor a tiny
// norm takes it out of range; in fp64 only where fp32's range asks for it.
__device__ __forceinline__ float2 inverse_norm(const SquareSum& t, float eps) {
    const float mid = t.mid + t.rest;
    if (t.big == 0.f && mid >= 0x1p-60f)  // the small class is below fp32's precision then
        return make_float2(1.f, kScaleX / (sqrtf(mid) + eps));
    const double norm = sqrt(static_cast<double>(mid) + static_cast<double>(t.big) * 0x1p160 +
                             static_cast<double>(t.small) * 0x1p-160) + static_cast<double>(eps);
    // A matrix of zeros with eps = 0 stays zeros.
    const double inv = norm == 0.0 ? 0.0 : static_cast<double>(kScaleX) / norm;
    int e = 0;
    const double mant = frexp(inv, &e);
    const int half = e / 2;
    return make_float2(static_cast<float>(ldexp(1.0, half)), static_cast<float>(ldexp(mant, e - half)));
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
// A block takes a 64 x 64 tile of u, a thread four times 4 consecutive values of it (V = 4: in
// one load each) and of X, one row of tiles after another: blocks (column tile, first row tile,
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
    const int c = (threadIdx.x & 15) * 4, rq = threadIdx.x >> 4;
    float2 f = make_float2(0.f, 0.f);
    for (int r0 = blockIdx.y * kCastTile; r0 < in.rows; r0 += gridDim.y * kCastTile) {
        float v[4][4], m[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t row = r0 + rq + 16 * k;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k][e] = m[k][e] = 0.f;
            if (row >= in.rows) continue;
            if constexpr (V == 4) {
                if (c0 + c < in.cols) {
                    load_values<4>(g, row * in.g_row + c0 + c, in.dtype, v[k]);
                    if (mom) load_values<4>(mom, row * in.m_row + c0 + c, CB_F32, m[k]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c0 + c + e < in.cols) {
                        v[k][e] = load_value(g, row * in.g_row + c0 + c + e, in.dtype);
                        if (mom) m[k][e] = mom[row * in.m_row + c0 + c + e];
                    }
            }
        }
        if (mom) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[k][e] = in.nesterov ? mix_momentum(m[k][e], v[k][e], in.beta) : m[k][e];
        }
        if (r0 == static_cast<int>(blockIdx.y) * kCastTile)  // behind the first tile's loads
            f = inverse_norm(partial + static_cast<int64_t>(b) * kNormBlocks, norm_blocks, eps);
        auto put = [&](int64_t at, const float (&x)[4]) {
            uint32_t h[2], l[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const __half2 top = __floats2half2_rn(x[2 * e], x[2 * e + 1]);
                const float2 back = __half22float2(top);
                const __half2 rest = __floats2half2_rn(x[2 * e] - back.x, x[2 * e + 1] - back.y);
                memcpy(&h[e], &top, 4);
                memcpy(&l[e], &rest, 4);
            }
            *reinterpret_cast<uint2*>(hi + at) = make_uint2(h[0], h[1]);
            *reinterpret_cast<uint2*>(lo + at) = make_uint2(l[0], l[1]);
        };
        const int64_t base = b * x_batch;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = r0 + rq + 16 * k;
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = (v[k][e] * f.x) * f.y;
                if constexpr (TRANSPOSED) tile[rq + 16 * k][c + e] = x[e];
            }
            if (!TRANSPOSED && row < in.rows) put(base + static_cast<int64_t>(row) * ld + c0 + c, x);
        }
        if constexpr (TRANSPOSED) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int col = c0 + rq + 16 * k;  // value (row, col) of u is X[col, row]
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = tile[c + e][rq + 16 * k];
                if (col < in.cols) put(base + static_cast<int64_t>(col) * ld + r0 + c, x);
            }
            __syncthreads();
        }
    }
}

// ---------------------------------------------------------------- products

enum Product {
    kGram,    // A = X X^T                          (symmetric)
    kPoly,    // B = b A + c A A (+ a I)            (symmetric)
    kUpdate,  // X' = (a X +) B X
    kResult   // the same, into the caller's matrix
};
template <Product WHAT> constexpr bool kSymmetric = WHAT == kGram || WHAT == kPoly;

constexpr int kTileM = 128, kTileK = 64;
constexpr int kEpilogueWarps = 8;  // two for each quarter of TMEM's lanes, every other 32 columns each
constexpr int kProductThreads = (kEpilogueWarps + 2) * 32;  // + a copying warp, + a multiplying warp
constexpr uint32_t kBoxBytes = 64 * 64 * 2;                 // 64 rows of 64 fp16
template <int BN> constexpr int kStages = BN == 128 ? 6 : 8;
constexpr int kPartsMost = 4;

// Parts of K in which A = X X^T is summed, the parts' sums then added in order: as many blocks
// can share a tile (muon_split_kernel), and a result is the same whether they do or one block
// takes the parts in turn, so that a matrix gives the same bits alone and in a stack. Two or
// four, of a dozen steps of 64 at least, where a matrix is of few tiles.
int gram_parts(int64_t p, int64_t k) {
    const int64_t ksteps = (k + 63) / 64;
    return p > 512 || ksteps < 24 ? 1 : (ksteps < 48 ? 2 : 4);
}
// Sums of a tile in TMEM: two of its width, or of every part's.
template <int BN, Product WHAT> constexpr int kSumColumns = WHAT == kGram && BN == 64 ? kPartsMost * BN : BN;
template <int BN> constexpr uint32_t kStageBytes = (kTileM + BN) * kTileK * 2;

struct ProductArgs {
    int32_t m, n, k;          // C [m, n], K
    int32_t batch;
    int32_t row_tiles, col_tiles;
    int32_t width;            // columns of a tile
    int32_t parts;            // kGram: parts of K summed apart (gram_parts)
    int64_t tiles;            // per matrix
    float a, b, c;            // the step's coefficients (a = 0: no term a X, or a I)
    const __half* term_hi;    // kPoly: A; kUpdate, kResult: X
    const __half* term_lo;    // or null
    int64_t term_batch;
    int32_t term_ld;
    __half* out_hi;
    __half* out_lo;           // or null
    int64_t out_batch;
    int32_t out_ld;
    // kResult
    void* user;               // the caller's output, or weights
    int64_t user_batch, user_row;
    int32_t user_dtype;
    int32_t transposed;       // value (i, j) of C is value (j, i) of the caller's
    int32_t user_vector;      // its rows can be taken 4 values at a time
    int32_t weights;          // W <- keep W - rate O, instead of O
    float keep, rate;
    int* error;
};

struct Tile {
    int32_t b, i, j;
};

// Column tiles of `width` of row tile i (of `height`) that reach the lower triangle.
__host__ __device__ __forceinline__ int lower_tiles(int i, int height, int width, int col_tiles) {
    const int need = ((i + 1) * height + width - 1) / width;
    return need < col_tiles ? need : col_tiles;
}

template <int HEIGHT, Product WHAT>
__device__ __forceinline__ Tile tile_at(const ProductArgs& P, int64_t t) {
    Tile T;
    T.b = static_cast<int>(t / P.tiles);
    int r = static_cast<int>(t - T.b * P.tiles);
    if constexpr (kSymmetric<WHAT>) {
        T.i = 0;
        while (true) {
            const int c = lower_tiles(T.i, HEIGHT, P.width, P.col_tiles);
            if (r < c) break;
            r -= c;
            ++T.i;
        }
        T.j = r;
    } else {
        // Eight row tiles at a time, so that concurrent tiles share operands in L2.
        constexpr int G = 8;
        const int group = r / (G * P.col_tiles), first = group * G;
        const int rows = P.row_tiles - first < G ? P.row_tiles - first : G;
        r -= group * G * P.col_tiles;
        T.i = first + r % rows;
        T.j = r / rows;
    }
    return T;
}

__device__ __forceinline__ void unpack_halves(const uint4* p, float (&v)[32]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float f[8];
        unpack<CB_F16>(p[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * k + e] = f[e];
    }
}
__device__ __forceinline__ void store_halves(__half* p, const float (&v)[32]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __half2 h = __floats2half2_rn(v[8 * k + 2 * e], v[8 * k + 2 * e + 1]);
            memcpy(&w[e], &h, 4);
        }
        reinterpret_cast<uint4*>(p)[k] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// 16 columns of a warp's 32 rows into the caller's matrix, through shared memory so that
// lanes run along the caller's rows, 4 values each: loads (of weights) first, then stores.
constexpr int kStageFloats = 32 * 20;  // rows of 16 (or, transposed, 32) values padded to 20 (36)
template <int DT>
__device__ __forceinline__ void finish_result(const ProductArgs& P, int batch, int row, int col, const float* v,
                                              float* stage, int lane) {
    char* user = static_cast<char*>(P.user) + batch * P.user_batch * dtype_bytes(DT);
    __syncwarp();
    if (P.transposed) {
#pragma unroll
        for (int k = 0; k < 16; ++k) stage[k * 36 + lane] = v[k];
    } else {
#pragma unroll
        for (int k = 0; k < 16; k += 4)
            *reinterpret_cast<float4*>(stage + lane * 20 + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    }
    __syncwarp();
    const int row0 = P.transposed ? col : row - lane, col0 = P.transposed ? row - lane : col;
    const int rows = P.transposed ? P.n : P.m, cols = P.transposed ? P.m : P.n;  // of the caller's matrix
    const int wide = P.transposed ? 8 : 4, pitch = P.transposed ? 36 : 20;       // lanes per row
    const int c = lane % wide * 4, r = lane / wide, step = 32 / wide;
    const int64_t at = static_cast<int64_t>(row0 + r) * P.user_row + col0 + c, down = step * P.user_row;
    float w[4][4] = {};
    if (P.weights) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (row0 + r + k * step >= rows) break;
            if (P.user_vector) {
                if (col0 + c < cols) load_values<4>(user, at + k * down, DT, w[k]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col0 + c + e < cols) w[k][e] = load_value(user, at + k * down + e, DT);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (row0 + r + k * step >= rows) break;
        const float4 s = *reinterpret_cast<const float4*>(stage + (r + k * step) * pitch + c);
        float x[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] *= 1.f / kScaleX;
            if (P.weights) x[e] = fmaf(-P.rate, x[e], P.keep * w[k][e]);
        }
        if (P.user_vector) {
            if (col0 + c < cols) store_values4<DT>(user, at + k * down, x);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col0 + c + e < cols) store_value(user, at + k * down + e, x[e], DT);
        }
    }
}

// What the result at a lane's 32 columns has added to it: loaded a turn ahead of its use.
struct Term {
    uint4 hi[4], lo[4];
};
template <Product WHAT>
__device__ __forceinline__ void load_term(const ProductArgs& P, int batch, int row, int col, Term& t) {
    if (row >= P.m || col >= P.n || WHAT == kGram || (WHAT != kPoly && P.a == 0.f)) return;
    const int64_t at = batch * P.term_batch + static_cast<int64_t>(row) * P.term_ld + col;
    const uint4* hi = reinterpret_cast<const uint4*>(P.term_hi + at);
#pragma unroll
    for (int k = 0; k < 4; ++k) t.hi[k] = hi[k];
    if (WHAT != kPoly && P.term_lo) {
        const uint4* lo = reinterpret_cast<const uint4*>(P.term_lo + at);
#pragma unroll
        for (int k = 0; k < 4; ++k) t.lo[k] = lo[k];
    }
}

// 32 columns [col, col + 32) of row `row` of a tile's result: `v` holds the products' sums.
template <Product WHAT>
__device__ __forceinline__ void finish(const ProductArgs& P, int batch, int row, int col, float (&v)[32],
                                       const Term& term, float* stage, int lane) {
    const bool live = row < P.m;
    if constexpr (WHAT == kGram) {
        constexpr float s = kScaleA / (kScaleX * kScaleX);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= s;
    } else if constexpr (WHAT == kPoly) {
        float t[32];
        unpack_halves(term.hi, t);
        const float c = P.c / kScaleA, diagonal = P.a * kScaleA;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            v[k] = fmaf(c, v[k], P.b * t[k]);
            if (row == col + k) v[k] += diagonal;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= 1.f / kScaleA;
        if (P.a != 0.f) {
            float t[32];
            if (P.term_lo) {
                unpack_halves(term.lo, t);
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] = fmaf(P.a, t[k], v[k]);
            }
            unpack_halves(term.hi, t);
#pragma unroll
            for (int k = 0; k < 32; ++k) v[k] = fmaf(P.a, t[k], v[k]);
        }
    }
    if constexpr (kSymmetric<WHAT>) {
        __half* out = P.out_hi + batch * P.out_batch;
        const int block = col / kTileM, row_block = row / kTileM;
        if (live && block <= row_block) store_halves(out + static_cast<int64_t>(row) * P.out_ld + col, v);
        if (live && block < row_block) {  // whole blocks of columns below the diagonal: all within the matrix
#pragma unroll
            for (int k = 0; k < 32; ++k) out[static_cast<int64_t>(col + k) * P.out_ld + row] = __float2half_rn(v[k]);
        }
    } else if constexpr (WHAT == kUpdate) {
        if (live) {
            const int64_t at = batch * P.out_batch + static_cast<int64_t>(row) * P.out_ld + col;
            store_halves(P.out_hi + at, v);
            if (P.out_lo) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] -= __half2float(__float2half_rn(v[k]));
                store_halves(P.out_lo + at, v);
            }
        }
    } else {
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            if (P.user_dtype == CB_F32) finish_result<CB_F32>(P, batch, row, col + h, v + h, stage, lane);
            else if (P.user_dtype == CB_BF16) finish_result<CB_BF16>(P, batch, row, col + h, v + h, stage, lane);
            else finish_result<CB_F16>(P, batch, row, col + h, v + h, stage, lane);
        }
    }
}

// The epilogue of a tile: a warp's rows row0 .. row0 + 31, every other 32 columns. Those that no
// row of C has, or that the other triangle gives, are skipped.
template <Product WHAT>
__device__ __forceinline__ void finish_tile(const ProductArgs& P, int batch, int row0, int col0, int width, uint32_t tmem,
                                            uint32_t ready, uint32_t parity, float* stage, int warp, int lane, bool& ok,
                                            int parts = 1) {
    const int row = row0 + lane;
    auto skip = [&](int c) { return c >= width || col0 + c >= P.n || (kSymmetric<WHAT> && (col0 + c) / kTileM > row0 / kTileM); };
    int c = warp / 4 * 32;
    Term next{};
    if (!skip(c)) load_term<WHAT>(P, batch, row, col0 + c, next);
    ok = __all_sync(kFull, tc::barrier_wait(ready, parity));
    if (!ok) return;
    tc::fence_after();
    for (; !skip(c); c += 64) {
        const Term term = next;
        float v[32];
        const uint32_t at = tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16) + c;
        tc::tmem_load32(at, v);
        if constexpr (WHAT == kGram) {
            for (int k = 1; k < parts; ++k) {
                float more[32];
                tc::tmem_load32(at + k * width, more);
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] += more[i];
            }
        }
        if (!skip(c + 64)) load_term<WHAT>(P, batch, row, col0 + c + 64, next);
        finish<WHAT>(P, batch, row, col0 + c, v, term, stage, lane);
    }
    tc::fence_before();
    __syncwarp();
}

// C = A B in tiles of 128 x BN, tile after tile by each block. Operand A is K-major; B is
// K-major for the symmetric products (A's own rows), and X as it lies (MN-major) for B X.
// One warp copies tiles of 64 of K into a ring of stages, one issues the products into
// one of two accumulators in TMEM, four take the other through the epilogue.
template <int BN, Product WHAT>
__global__ void __launch_bounds__(kProductThreads, 1)
muon_product_kernel(const __grid_constant__ CUtensorMap left, const __grid_constant__ CUtensorMap right,
                    const ProductArgs P) {
    constexpr int S = kStages<BN>;
    constexpr int kSums = kSumColumns<BN, WHAT>;
    constexpr uint32_t kColumns = 2 * kSums;
    extern __shared__ unsigned char dynamic[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[S], empty[S], ready[2], drained[2];
    __shared__ uint32_t tmem_at;
    __shared__ __align__(16) float stage[WHAT == kResult ? kEpilogueWarps * kStageFloats : 4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::barrier_init(tc::smem_addr(full + s), 1);
            tc::barrier_init(tc::smem_addr(empty + s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            tc::barrier_init(tc::smem_addr(ready + s), 1);
            tc::barrier_init(tc::smem_addr(drained + s), kEpilogueWarps);
        }
        tc::barrier_init_fence();
        tc::tma_prefetch(&left);
        tc::tma_prefetch(&right);
    }
    if (warp == kEpilogueWarps) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), kColumns);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int64_t total = P.tiles * P.batch;
    const int ksteps = (P.k + kTileK - 1) / kTileK;
    const int per = kSums > BN ? (ksteps + P.parts - 1) / P.parts : ksteps;  // of a part
    bool ok = true;

    if (warp == kEpilogueWarps) {
        if (lane == 0) {  // copies
            int s = 0;
            uint32_t phase = 0;
            for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
                const Tile T = tile_at<kTileM, WHAT>(P, t);
                for (int k = 0; k < ksteps; ++k) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                    const uint32_t bar = tc::smem_addr(full + s);
                    uint32_t at = tc::smem_addr(ring) + s * kStageBytes<BN>;
                    tc::barrier_expect(bar, kStageBytes<BN>);
#pragma unroll
                    for (int x = 0; x < kTileM / 64; ++x, at += kBoxBytes)
                        tc::tma_load(at, &left, bar, k * kTileK, T.i * kTileM + x * 64, T.b);
#pragma unroll
                    for (int x = 0; x < BN / 64; ++x, at += kBoxBytes) {
                        if constexpr (kSymmetric<WHAT>) tc::tma_load(at, &right, bar, k * kTileK, T.j * BN + x * 64, T.b);
                        else tc::tma_load(at, &right, bar, T.j * BN + x * 64, k * kTileK, T.b);
                    }
                    if (++s == S) s = 0, phase ^= 1;
                }
            }
            // Copies in flight land before the block's shared memory goes away: those of
            // stages that were never multiplied, after a wait that ran out.
            if (!ok)
                for (int x = 0; x < S; ++x) {
                    if (--s < 0) s = S - 1, phase ^= 1;
                    if (!tc::barrier_wait(tc::smem_addr(full + s), phase)) break;
                }
        }
    } else if (warp == kEpilogueWarps + 1) {
        if (lane == 0) {  // products
            constexpr uint32_t shape = tc::mma_shape(kTileM, BN, !kSymmetric<WHAT>);
            int s = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(drained + acc), acc_phase ^ 1))) break;
                tc::fence_after();
                uint32_t sums = tmem + acc * kSums;
                int within = 0;  // steps done of a part
                for (int k = 0; k < ksteps; ++k) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                    tc::fence_after();
                    if (kSums > BN && within == per) within = 0, sums += BN;
                    const uint32_t at = tc::smem_addr(ring) + s * kStageBytes<BN>, bt = at + kTileM * kTileK * 2;
#pragma unroll
                    for (int x = 0; x < kTileK / 16; ++x) {
                        const uint64_t da = tc::operand_k_major(at + x * 32);
                        const uint64_t db = kSymmetric<WHAT> ? tc::operand_k_major(bt + x * 32)
                                                            : tc::operand_mn_major(bt + x * 2048, kBoxBytes);
                        tc::mma_f16<1>(sums, da, db, shape, within > 0 || x > 0);
                    }
                    ++within;
                    tc::mma_commit<1>(tc::smem_addr(empty + s));
                    if (++s == S) s = 0, phase ^= 1;
                }
                tc::mma_commit<1>(tc::smem_addr(ready + acc));
                if (++acc == 2) acc = 0, acc_phase ^= 1;
            }
        }
    } else {  // epilogue
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
            const Tile T = tile_at<kTileM, WHAT>(P, t);
            finish_tile<WHAT>(P, T.b, T.i * kTileM + warp % 4 * 32, T.j * BN, BN, tmem + acc * kSums,
                              tc::smem_addr(ready + acc), acc_phase, stage + (WHAT == kResult ? warp * kStageFloats : 0), warp,
                              lane, ok, kSums > BN ? (ksteps + per - 1) / per : 1);
            if (!ok) break;
            if (lane == 0) tc::barrier_arrive(tc::smem_addr(drained + acc));
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
    }
    if (!ok && lane == 0) set_error(P.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == kEpilogueWarps) tc::tmem_free<1>(tmem, kColumns);
}

// The same in tiles of 256 x P.width by pairs of blocks on two SMs: each block copies and
// keeps 128 rows of A and half of the columns of B, one thread of the first block issues the
// products of both, and each block has 128 rows of the sums in its TMEM. A 128 x 128 tile
// reads and writes 256 bytes of shared memory a clock at the tensor cores' rate, twice what
// an SM has; a pair's 256 x 256 tile 128 bytes. P.width is a multiple of 32 (a block's
// half of the columns, of 16; 128 are copied) so that a few rounds of tiles can be made to
// fill the GPU. Operands that are K-major come in boxes of 128 rows, fewer copies than of 64.
constexpr int kPairM = 256, kPairWidth = 256, kPairStages = 6;
constexpr uint32_t kPairStageBytes = (128 + kPairWidth / 2) * kTileK * 2;

template <Product WHAT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1)
muon_pair_kernel(const __grid_constant__ CUtensorMap left, const __grid_constant__ CUtensorMap right,
                 const ProductArgs P) {
    constexpr int S = kPairStages;
    constexpr uint32_t kColumns = 2 * kPairWidth;
    extern __shared__ unsigned char dynamic[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    // full, drained: those of the first block count for both; empty, ready: each block's own.
    __shared__ uint64_t full[S], empty[S], ready[2], drained[2];
    __shared__ uint32_t tmem_at;
    __shared__ __align__(16) float stage[WHAT == kResult ? kEpilogueWarps * kStageFloats : 4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(tc::cluster_rank());
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::barrier_init(tc::smem_addr(full + s), 1);
            tc::barrier_init(tc::smem_addr(empty + s), 1);
        }
        for (int s = 0; s < 2; ++s) {
            tc::barrier_init(tc::smem_addr(ready + s), 1);
            tc::barrier_init(tc::smem_addr(drained + s), 2 * kEpilogueWarps);
        }
        tc::barrier_init_fence();
        tc::tma_prefetch(&left);
        tc::tma_prefetch(&right);
    }
    if (warp == kEpilogueWarps) tc::tmem_alloc<2>(tc::smem_addr(&tmem_at), kColumns);
    tc::fence_before();
    tc::cluster_sync();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int64_t total = P.tiles * P.batch;
    const int64_t first = blockIdx.x / 2, step = gridDim.x / 2;
    const int ksteps = (P.k + kTileK - 1) / kTileK, half = P.width / 2;
    bool ok = true;

    if (warp == kEpilogueWarps) {
        if (lane == 0) {  // copies
            int s = 0;
            uint32_t phase = 0;
            for (int64_t t = first; t < total && ok; t += step) {
                const Tile T = tile_at<kPairM, WHAT>(P, t);
                const int row = T.i * kPairM + rank * 128, col = T.j * P.width + rank * half;
                for (int k = 0; k < ksteps; ++k) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                    const uint32_t bar = tc::in_first_block(tc::smem_addr(full + s));
                    uint32_t at = tc::smem_addr(ring) + s * kPairStageBytes;
                    if (rank == 0) tc::barrier_expect(tc::smem_addr(full + s), 2 * kPairStageBytes);
                    tc::tma_load_pair(at, &left, bar, k * kTileK, row, T.b);
                    at += 2 * kBoxBytes;
                    if constexpr (kSymmetric<WHAT>) {
                        tc::tma_load_pair(at, &right, bar, k * kTileK, col, T.b);
                    } else {
                        tc::tma_load_pair(at, &right, bar, col, k * kTileK, T.b);
                        tc::tma_load_pair(at + kBoxBytes, &right, bar, col + 64, k * kTileK, T.b);
                    }
                    if (++s == S) s = 0, phase ^= 1;
                }
            }
            if (!ok && rank == 0)  // copies in flight land before the blocks' shared memory goes away
                for (int x = 0; x < S; ++x) {
                    if (--s < 0) s = S - 1, phase ^= 1;
                    if (!tc::barrier_wait(tc::smem_addr(full + s), phase)) break;
                }
        }
    } else if (warp == kEpilogueWarps + 1) {
        if (lane == 0 && rank == 0) {  // products of both blocks
            const uint32_t shape = tc::mma_shape(kPairM, P.width, !kSymmetric<WHAT>);
            int s = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            for (int64_t t = first; t < total && ok; t += step) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(drained + acc), acc_phase ^ 1))) break;
                tc::fence_after();
                for (int k = 0; k < ksteps; ++k) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                    tc::fence_after();
                    const uint32_t at = tc::smem_addr(ring) + s * kPairStageBytes, bt = at + 2 * kBoxBytes;
#pragma unroll
                    for (int x = 0; x < kTileK / 16; ++x) {
                        const uint64_t da = tc::operand_k_major(at + x * 32);
                        const uint64_t db = kSymmetric<WHAT> ? tc::operand_k_major(bt + x * 32)
                                                             : tc::operand_mn_major(bt + x * 2048, kBoxBytes);
                        tc::mma_f16<2>(tmem + acc * kPairWidth, da, db, shape, k > 0 || x > 0);
                    }
                    tc::mma_commit<2>(tc::smem_addr(empty + s));
                    if (++s == S) s = 0, phase ^= 1;
                }
                tc::mma_commit<2>(tc::smem_addr(ready + acc));
                if (++acc == 2) acc = 0, acc_phase ^= 1;
            }
        }
    } else {  // epilogue
        int acc = 0;
        uint32_t acc_phase = 0;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile T = tile_at<kPairM, WHAT>(P, t);
            finish_tile<WHAT>(P, T.b, T.i * kPairM + rank * 128 + warp % 4 * 32, T.j * P.width, P.width,
                              tmem + acc * kPairWidth, tc::smem_addr(ready + acc), acc_phase,
                              stage + (WHAT == kResult ? warp * kStageFloats : 0), warp, lane, ok);
            if (!ok) break;
            if (lane == 0) tc::barrier_arrive_cluster(tc::in_first_block(tc::smem_addr(drained + acc)));
            if (++acc == 2) acc = 0, acc_phase ^= 1;
        }
    }
    if (!ok && lane == 0) set_error(P.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    tc::cluster_sync();  // neither block ends while the other may signal its barriers
    tc::fence_after();
    if (warp == kEpilogueWarps) tc::tmem_free<2>(tmem, kColumns);
}

// A = X X^T of few tiles and a long K: a cluster of P.parts blocks takes a tile of 128 x 64, a
// part of K each, and every block adds up a share of the tile's rows over all of them, in
// order, from their shared memory.

__global__ void __launch_bounds__(kProductThreads, 1)
muon_split_kernel(const __grid_constant__ CUtensorMap rows, const ProductArgs P) {
    constexpr int BN = 64, S = kStages<BN>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    float* sums = reinterpret_cast<float*>(ring);  // [128][64], once the products are done
    __shared__ uint64_t full[S], empty[S], ready;
    __shared__ uint32_t tmem_at;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            tc::barrier_init(tc::smem_addr(full + s), 1);
            tc::barrier_init(tc::smem_addr(empty + s), 1);
        }
        tc::barrier_init(tc::smem_addr(&ready), 1);
        tc::barrier_init_fence();
        tc::tma_prefetch(&rows);
    }
    if (warp == kEpilogueWarps) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), BN);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int rank = static_cast<int>(tc::cluster_rank());
    const Tile T = tile_at<kTileM, kGram>(P, blockIdx.x / P.parts);
    const int all = (P.k + kTileK - 1) / kTileK, per = (all + P.parts - 1) / P.parts;
    const int first = rank * per, count = max(0, min(per, all - first));
    bool ok = true;

    if (warp == kEpilogueWarps) {
        if (lane == 0) {  // copies
            int k = 0;
            for (; k < count; ++k) {
                const int s = k % S;
                if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), (k / S & 1) ^ 1))) break;
                const uint32_t bar = tc::smem_addr(full + s);
                const uint32_t at = tc::smem_addr(ring) + s * kStageBytes<BN>;
                const int x = (first + k) * kTileK;
                tc::barrier_expect(bar, kStageBytes<BN>);
                tc::tma_load(at, &rows, bar, x, T.i * kTileM, T.b);
                tc::tma_load(at + kBoxBytes, &rows, bar, x, T.i * kTileM + 64, T.b);
                tc::tma_load(at + 2 * kBoxBytes, &rows, bar, x, T.j * BN, T.b);
            }
            if (!ok)  // copies in flight land before the block's shared memory goes away
                for (int x = max(0, k - S); x < k; ++x)
                    if (!tc::barrier_wait(tc::smem_addr(full + x % S), x / S & 1)) break;
        }
    } else if (warp == kEpilogueWarps + 1) {
        if (lane == 0) {  // products
            constexpr uint32_t shape = tc::mma_shape(kTileM, BN, false);
            for (int k = 0; k < count && ok; ++k) {
                const int s = k % S;
                if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), k / S & 1))) break;
                tc::fence_after();
                const uint32_t at = tc::smem_addr(ring) + s * kStageBytes<BN>, bt = at + 2 * kBoxBytes;
#pragma unroll
                for (int x = 0; x < kTileK / 16; ++x)
                    tc::mma_f16<1>(tmem, tc::operand_k_major(at + x * 32), tc::operand_k_major(bt + x * 32), shape,
                                   k > 0 || x > 0);
                tc::mma_commit<1>(tc::smem_addr(empty + s));
            }
            if (ok && count > 0) tc::mma_commit<1>(tc::smem_addr(&ready));
        }
    } else {
        const int row = warp % 4 * 32 + lane, c = warp / 4 * 32;
        float v[32] = {};
        if (count > 0) {
            ok = __all_sync(kFull, tc::barrier_wait(tc::smem_addr(&ready), 0));
            tc::fence_after();
            tc::tmem_load32(tmem + (static_cast<uint32_t>(warp % 4 * 32) << 16) + c, v);
        }
        // After a wait that ran out copies may still be on their way into the ring: the sums
        // then stay unwritten (the result is reported as incomplete).
        if (ok) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)  // 16-byte pieces of a row, swizzled over the banks
                *reinterpret_cast<float4*>(sums + row * BN + (((c + k) / 4 ^ (row & 15)) << 2)) =
                    make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        }
    }
    if (!ok && lane == 0) set_error(P.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    tc::cluster_sync();
    if (warp < kEpilogueWarps) {
        const int share = kTileM / P.parts, columns = BN / 4;
        constexpr float scale = kScaleA / (kScaleX * kScaleX);
        __half* out = P.out_hi + T.b * P.out_batch;
        for (int i = threadIdx.x; i < share * columns; i += kEpilogueWarps * 32) {
            const int r = rank * share + i % share, c4 = i / share;  // lanes along the rows
            const uint32_t at = tc::smem_addr(sums + r * BN + ((c4 ^ (r & 15)) << 2));
            float4 part[kPartsMost];
#pragma unroll
            for (int k = 0; k < kPartsMost; ++k)
                part[k] = k < P.parts ? tc::load_cluster(tc::in_block(at, k)) : make_float4(0.f, 0.f, 0.f, 0.f);
            float4 t = part[0];
#pragma unroll
            for (int k = 1; k < kPartsMost; ++k) {
                t.x += part[k].x;
                t.y += part[k].y;
                t.z += part[k].z;
                t.w += part[k].w;
            }
            const int row = T.i * kTileM + r, col = T.j * BN + c4 * 4, block = col / kTileM;
            if (row >= P.m || col >= P.n || block > T.i) continue;
            const __half2 h0 = __floats2half2_rn(t.x * scale, t.y * scale), h1 = __floats2half2_rn(t.z * scale, t.w * scale);
            uint2 w;
            memcpy(&w.x, &h0, 4);
            memcpy(&w.y, &h1, 4);
            *reinterpret_cast<uint2*>(out + static_cast<int64_t>(row) * P.out_ld + col) = w;  // rows are padded to 64
            if (block < T.i) {
                const __half h[4] = {__low2half(h0), __high2half(h0), __low2half(h1), __high2half(h1)};
#pragma unroll
                for (int e = 0; e < 4; ++e) out[static_cast<int64_t>(col + e) * P.out_ld + row] = h[e];
            }
        }
    }
    tc::cluster_sync();  // no block ends while others read its sums
    tc::fence_after();
    if (warp == kEpilogueWarps) tc::tmem_free<1>(tmem, BN);
}

// ---------------------------------------------------------------- small matrices in one launch

// Up to 128 x 3 K: all steps of a matrix in one kernel, by a cluster of blocks that each keep
// up to 384 columns of X in shared memory (fp16, for the products) and in TMEM (fp32, a X as
// the sums that B X is added to). The Gram matrix of the blocks' columns is added up
// across the cluster, in a fixed order, a share of its rows in each block; A A and B are
// taken by every block for itself. What is left of a step is a chain of three products
// of half a microsecond and their epilogues, in which a thread of TN / 128 has 32 columns of
// its row at a time: 512 threads a block (128 x 256, five steps: 34 us, 42 with 256), or 256 of
// two blocks per SM where narrow matrices would otherwise queue (300 of 128 x 128: 34 us, 47).
constexpr int kSmallRows = 128, kSmallCols = 384, kSmallCluster = 8;
constexpr uint32_t kSlab = 128 * 128;  // bytes of 128 rows of 64 values

struct SmallArgs {
    int32_t p, q, cols;      // X [p, q], columns per block (a multiple of 64)
    int32_t transposed, blocks, steps;
    float eps;
    float coefficients[3 * kMaxSteps];
    void* user;
    int64_t user_batch, user_row;
    int32_t user_dtype, user_vector, in_vector;
    int32_t weights;
    float keep, rate;
    int* error;
};

// 16 bytes (8 values from column c of 64) of a row of a slab, swizzled as TMA would.
__device__ __forceinline__ uint32_t slab_at(int row, int c) { return row * 128 + ((c / 8 ^ (row & 7)) << 4); }
__device__ __forceinline__ void store_slab32(unsigned char* slab, int row, int c, const float (&v)[32]) {
#pragma unroll
    for (int k = 0; k < 32; k += 8) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __half2 h = __floats2half2_rn(v[k + 2 * e], v[k + 2 * e + 1]);
            memcpy(&w[e], &h, 4);
        }
        *reinterpret_cast<uint4*>(slab + slab_at(row, c + k)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <bool CLUSTER, int NT>
__global__ void __launch_bounds__(NT) muon_small_kernel(const MatrixIn in, const __grid_constant__ SmallArgs P) {
    extern __shared__ unsigned char dynamic[];
    unsigned char* X = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    unsigned char* A = X + P.cols / 64 * kSlab;  // A, then B
    float* sums = reinterpret_cast<float*>(A + 2 * kSlab);  // CLUSTER: this block's part of A, fp32 [128][128]
    __shared__ uint64_t done;
    __shared__ uint32_t tmem_at;
    __shared__ float2 factor;
    __shared__ __align__(16) float squares[NT / 32 + 1][4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CLUSTER ? static_cast<int>(tc::cluster_rank()) : 0;
    const int b = blockIdx.x / P.blocks;
    const uint32_t columns = P.cols <= 128 ? 256 : 512;
    if (threadIdx.x == 0) {
        tc::barrier_init(tc::smem_addr(&done), 1);
        tc::barrier_init_fence();
    }
    if (warp == 0) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), columns);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
    const uint32_t sum_x = tmem_at, sum_a = tmem_at + columns - 128;
    begin_kernel();

    // The update: a thread has row `row` of X, and 32 of every NT / 4 of the block's columns.
    const int row = warp % 4 * 32 + lane, first = warp / 4 * 32, col0 = rank * P.cols;
    const char* g = static_cast<const char*>(in.g) + b * in.g_batch * dtype_bytes(in.dtype);
    float* mom = in.momentum ? in.momentum + b * in.m_batch : nullptr;
    SquareSum squared;
    for (int c = first; c < P.cols; c += NT / 4) {
        float v[32], m[32];
#pragma unroll
        for (int k = 0; k < 32; k += 4) {
            float x[4] = {}, y[4] = {};
            const int col = col0 + c + k;
            if (row < P.p) {
                if (!P.transposed && P.in_vector) {
                    if (col < P.q) {
                        load_values<4>(g, row * in.g_row + col, in.dtype, x);
                        if (mom) load_values<4>(mom, row * in.m_row + col, CB_F32, y);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (col + e < P.q) {
                            const int64_t r = P.transposed ? col + e : row, i = P.transposed ? row : col + e;
                            x[e] = load_value(g, r * in.g_row + i, in.dtype);
                            if (mom) y[e] = mom[r * in.m_row + i];
                        }
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k + e] = x[e], m[k + e] = y[e];
        }
        if (mom) {
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                v[k] = update_value(in, v[k], m[k]);
                const int col = col0 + c + k;
                if (row < P.p && col < P.q)
                    mom[P.transposed ? static_cast<int64_t>(col) * in.m_row + row : row * in.m_row + col] = m[k];
            }
        }
        squared.add(v);
        tc::tmem_store32(sum_x + lanes + c, v);
    }
    auto put = [](float (&to)[4], const SquareSum& s) { to[0] = s.mid, to[1] = s.rest, to[2] = s.big, to[3] = s.small; };
    auto get = [](const float4& f) {
        SquareSum s;
        s.mid = f.x, s.rest = f.y, s.big = f.z, s.small = f.w;
        return s;
    };
    squared.add_lanes();
    if (lane == 0) put(squares[warp], squared);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NT / 32; ++w) squared.add(get(*reinterpret_cast<const float4*>(squares[w])));
        put(squares[NT / 32], squared);
    }
    if constexpr (CLUSTER) tc::cluster_sync();
    if (threadIdx.x == 0) {
        if constexpr (CLUSTER) {
            const uint32_t at = tc::smem_addr(squares[NT / 32]);
            squared = get(tc::load_cluster(tc::in_block(at, 0)));
            for (int r = 1; r < P.blocks; ++r) squared.add(get(tc::load_cluster(tc::in_block(at, r))));
        }
        factor = inverse_norm(squared, P.eps);
    }
    __syncthreads();
    const float2 f = factor;
    for (int c = first; c < P.cols; c += NT / 4) {
        float v[32];
        tc::tmem_load32(sum_x + lanes + c, v);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = (v[k] * f.x) * f.y;
        store_slab32(X + c / 64 * kSlab, row, c % 64, v);
        const float a = P.coefficients[0] * kScaleA;
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] *= a;
        tc::tmem_store32(sum_x + lanes + c, v);
    }

    // A wait that ran out is reported, and the rest is then computed without waiting: the
    // cluster's blocks stay in step.
    bool ok = true;
    uint32_t phase = 0;
    auto handed_over = [&] {  // what all threads stored, to the tensor core
        tc::fence_to_tensor_core();
        tc::fence_before();
        __syncthreads();
    };
    auto products_done = [&] {
        ok = ok && tc::barrier_wait(tc::smem_addr(&done), phase);
        phase ^= 1;
        tc::fence_after();
    };
    const uint32_t x_at = tc::smem_addr(X), a_at = tc::smem_addr(A);
    for (int step = 0; step < P.steps; ++step) {
        const float a = P.coefficients[3 * step], bb = P.coefficients[3 * step + 1], cc = P.coefficients[3 * step + 2];
        const bool two_term = step < kTwoTerm;
        handed_over();
        if (threadIdx.x == 0) {  // A = X X^T
            tc::fence_after();
            constexpr uint32_t shape = tc::mma_shape(128, 128, false);
            for (int x = 0; x < P.cols / 16; ++x) {
                const uint64_t d = tc::operand_k_major(x_at + x / 4 * kSlab + x % 4 * 32);
                tc::mma_f16<1>(sum_a, d, d, shape, x > 0);
            }
            tc::mma_commit<1>(tc::smem_addr(&done));
        }
        products_done();
        constexpr float scale = kScaleA / (kScaleX * kScaleX);
        for (int c = first; c < 128; c += NT / 4) {
            float v[32];
            tc::tmem_load32(sum_a + lanes + c, v);
            if constexpr (CLUSTER) {  // 16-byte pieces of a row, swizzled over the banks
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                    *reinterpret_cast<float4*>(sums + row * 128 + (((c + k) / 4 ^ lane) << 2)) =
                        make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
            } else {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] *= scale;
                store_slab32(A + c / 64 * kSlab, row, c % 64, v);
            }
        }
        if constexpr (CLUSTER) {
            tc::cluster_sync();
            const int share = 128 / P.blocks;  // rows that this block adds up, for all
            for (int i = threadIdx.x; i < share * 32; i += NT) {
                const int r = rank * share + i / 32, c4 = i % 32;
                const uint32_t at = tc::smem_addr(sums + r * 128 + ((c4 ^ (r & 31)) << 2));
                float4 part[kSmallCluster];
#pragma unroll
                for (int k = 0; k < kSmallCluster; ++k)
                    part[k] = k < P.blocks ? tc::load_cluster(tc::in_block(at, k)) : make_float4(0.f, 0.f, 0.f, 0.f);
                float4 t = part[0];
#pragma unroll
                for (int k = 1; k < kSmallCluster; ++k) {
                    t.x += part[k].x;
                    t.y += part[k].y;
                    t.z += part[k].z;
                    t.w += part[k].w;
                }
                const __half2 h0 = __floats2half2_rn(t.x * scale, t.y * scale), h1 = __floats2half2_rn(t.z * scale, t.w * scale);
                uint2 w;
                memcpy(&w.x, &h0, 4);
                memcpy(&w.y, &h1, 4);
                const uint32_t to = a_at + c4 / 16 * kSlab + slab_at(r, c4 % 16 * 4) + c4 % 2 * 8;
                for (int k = 0; k < P.blocks; ++k) tc::store_cluster(tc::in_block(to, k), w);
            }
            tc::fence_to_tensor_core();
            tc::cluster_sync();
        }
        handed_over();
        if (threadIdx.x == 0) {  // A A
            tc::fence_after();
            constexpr uint32_t shape = tc::mma_shape(128, 128, false);
            for (int x = 0; x < 8; ++x) {
                const uint64_t d = tc::operand_k_major(a_at + x / 4 * kSlab + x % 4 * 32);
                tc::mma_f16<1>(sum_a, d, d, shape, x > 0);
            }
            tc::mma_commit<1>(tc::smem_addr(&done));
        }
        products_done();
        for (int c = first; c < 128; c += NT / 4) {  // B in the place of A
            float v[32];
            tc::tmem_load32(sum_a + lanes + c, v);
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
                float t[8];
                unpack<CB_F16>(*reinterpret_cast<const uint4*>(A + c / 64 * kSlab + slab_at(row, c % 64 + k)), t);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[k + e] = fmaf(cc / kScaleA, v[k + e], bb * t[e]);
                    if (!two_term && row == c + k + e) v[k + e] += a * kScaleA;
                }
            }
            store_slab32(A + c / 64 * kSlab, row, c % 64, v);
        }
        handed_over();
        if (threadIdx.x == 0) {  // X <- (a X +) B X
            tc::fence_after();
            for (int c = 0; c < P.cols; c += 256) {  // as many columns as one product takes
                const uint32_t shape = tc::mma_shape(128, P.cols - c < 256 ? P.cols - c : 256, true);
                for (int x = 0; x < 8; ++x)
                    tc::mma_f16<1>(sum_x + c, tc::operand_k_major(a_at + x / 4 * kSlab + x % 4 * 32),
                                   tc::operand_mn_major(x_at + c / 64 * kSlab + x * 2048, kSlab), shape, two_term || x > 0);
            }
            tc::mma_commit<1>(tc::smem_addr(&done));
        }
        products_done();
        const bool final = step + 1 == P.steps;
        for (int c = first; c < P.cols; c += NT / 4) {
            float v[32];
            tc::tmem_load32(sum_x + lanes + c, v);
            if (!final) {
#pragma unroll
                for (int k = 0; k < 32; ++k) v[k] *= 1.f / kScaleA;
                store_slab32(X + c / 64 * kSlab, row, c % 64, v);
                if (step + 1 < kTwoTerm) {
                    const float next = P.coefficients[3 * step + 3] * kScaleA;
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] *= next;
                    tc::tmem_store32(sum_x + lanes + c, v);
                }
            } else if (row < P.p) {
                char* user = static_cast<char*>(P.user) + b * P.user_batch * dtype_bytes(P.user_dtype);
                const bool vector = P.user_vector && !P.transposed;
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                    const int col = col0 + c + k;
                    float w[4] = {}, o[4];
                    auto at = [&](int e) {
                        return P.transposed ? static_cast<int64_t>(col + e) * P.user_row + row : row * P.user_row + col + e;
                    };
                    if (P.weights) {
                        if (vector) {
                            if (col < P.q) load_values<4>(user, at(0), P.user_dtype, w);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (col + e < P.q) w[e] = load_value(user, at(e), P.user_dtype);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[e] = v[k + e] * (1.f / (kScaleA * kScaleX));
                        if (P.weights) o[e] = fmaf(-P.rate, o[e], P.keep * w[e]);
                    }
                    if (vector) {
                        if (col < P.q) {
                            if (P.user_dtype == CB_F32) store_values4<CB_F32>(user, at(0), o);
                            else if (P.user_dtype == CB_BF16) store_values4<CB_BF16>(user, at(0), o);
                            else store_values4<CB_F16>(user, at(0), o);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < P.q) store_value(user, at(e), o[e], P.user_dtype);
                    }
                }
            }
        }
    }
    if (!ok && lane == 0) set_error(P.error, CB_ERR_TIMEOUT);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == 0) tc::tmem_free<1>(tmem_at, columns);
}

// ---------------------------------------------------------------- host

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) !=
                cudaSuccess || q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            fn = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    return encode;
}

// [batch][rows][cols] of fp16 with rows of `ld` values, in boxes of 64 values of box_rows rows;
// values past a row or past the rows read as zeros.
bool tensor_map(CUtensorMap* map, const void* data, int64_t cols, int64_t rows, int64_t batch, int64_t ld,
                uint32_t box_rows) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                                static_cast<cuuint64_t>(batch)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * rows * 2};
    const cuuint32_t box[3] = {64, box_rows, 1};
    const cuuint32_t step[3] = {1, 1, 1};
    return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(data), dims, strides, box,
                                step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Blocks per matrix of muon_small_kernel (a power of two), 0 where it does not apply.
int small_blocks(int64_t p, int64_t q) {
    if (p > kSmallRows || q > kSmallCols * kSmallCluster) return 0;
    int blocks = 1;
    while (blocks * kSmallCols < q) blocks *= 2;
    return blocks;
}
struct Workspace {
    int64_t p, q, ldx, lda;
    size_t hi[2], lo[2], gram, poly, partial, error, bytes;
};
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
    w.error = take(4);
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

template <Product WHAT>
int64_t tiles_of(int32_t m, int32_t n, int height, int width) {
    const int row_tiles = (m + height - 1) / height, col_tiles = (n + width - 1) / width;
    if (!kSymmetric<WHAT>) return static_cast<int64_t>(row_tiles) * col_tiles;
    int64_t t = 0;
    for (int i = 0; i < row_tiles; ++i) t += lower_tiles(i, height, width, col_tiles);
    return t;
}
template <Product WHAT>
void set_tiles(ProductArgs& P, int height, int width) {
    P.row_tiles = (P.m + height - 1) / height;
    P.col_tiles = (P.n + width - 1) / width;
    P.width = width;
    P.tiles = tiles_of<WHAT>(P.m, P.n, height, width);
}
template <class KernelT>
bool shared_memory(KernelT kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) == cudaSuccess;
}

// As launch(), by clusters of `cluster` blocks.
template <class... Params, class... Args>
bool launch_clusters(void (*kernel)(Params...), int cluster, int64_t grid, int block, size_t smem, cudaStream_t s,
                     const Args&... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...) == cudaSuccess;
}
bool launch_split(const CUtensorMap& rows, ProductArgs P, cudaStream_t s) {
    set_tiles<kGram>(P, kTileM, 64);
    constexpr size_t smem = kStages<64> * kStageBytes<64> + 1024;
    static const bool ready = shared_memory(muon_split_kernel, smem);
    return ready && launch_clusters(muon_split_kernel, P.parts, P.tiles * P.batch * P.parts, kProductThreads, smem, s, rows, P);
}

template <int BN, Product WHAT>
bool launch_product(const CUtensorMap& left, const CUtensorMap& right, ProductArgs P, int sms, cudaStream_t s) {
    set_tiles<WHAT>(P, kTileM, BN);
    constexpr size_t smem = kStages<BN> * kStageBytes<BN> + 1024;
    static const bool ready = shared_memory(muon_product_kernel<BN, WHAT>, smem);
    if (!ready) return false;
    launch(muon_product_kernel<BN, WHAT>, dim3(static_cast<unsigned>(min64(P.tiles * P.batch, sms))),
           dim3(kProductThreads), smem, s, left, right, P);
    return true;
}
template <Product WHAT>
bool launch_pairs(const CUtensorMap& left, const CUtensorMap& right, ProductArgs P, int width, int sms, cudaStream_t s) {
    set_tiles<WHAT>(P, kPairM, width);
    constexpr size_t smem = kPairStages * kPairStageBytes + 1024;
    static const bool ready = shared_memory(muon_pair_kernel<WHAT>, smem);
    if (!ready) return false;
    launch(muon_pair_kernel<WHAT>, dim3(static_cast<unsigned>(2 * min64(P.tiles * P.batch, sms / 2))),
           dim3(kProductThreads), smem, s, left, right, P);
    return true;
}

// A matrix of the workspace as an operand, by the boxes that a kernel copies.
struct Operand {
    CUtensorMap box64, box128;
    bool set(const void* data, int64_t cols, int64_t rows, int64_t batch, int64_t ld) {
        return tensor_map(&box64, data, cols, rows, batch, ld, 64) && tensor_map(&box128, data, cols, rows, batch, ld, 128);
    }
};

// The tiles with the least time, in clocks: rounds of tiles over the GPU, each the steps of 64
// of K that it takes, and what a kernel takes besides. Fitted to all three products at sizes
// of 200 to 4096, each with tiles of one kind forced, in clocks a step: 590 (128 x 64), 630 (128
// x 128), 654 to 692 (256 x 160 to 256 by a pair; about 700 at any width where B is MN-major; the
// tensor cores need 320 to 512 of them: shared memory and the way there bound it). Whole calls
// with the kind chosen, and with the best single kind: 1024 x 1024 138 us (64 wide), 4 x 1024 x
// 1024 201 us (128; 223 by pairs, 279 at 64), 2048 x 2048 283 us, 4096 x 4096 1060 us (pairs;
// 1661 at 128, 2860 at 64).
template <Product WHAT>
bool launch_best(const Operand& left, const Operand& right, const ProductArgs& P, int sms, cudaStream_t s) {
    const int64_t ksteps = (P.k + kTileK - 1) / kTileK;
    auto time = [&](int height, int width, int at_once, int64_t step, int64_t fixed) {
        return (tiles_of<WHAT>(P.m, P.n, height, width) * P.batch + at_once - 1) / at_once * ksteps * step + fixed;
    };
    int64_t best = time(kTileM, 64, sms, 590, 7000);
    if constexpr (WHAT == kGram) {
        if (P.parts > 1) {
            const int64_t blocks = tiles_of<kGram>(P.m, P.n, kTileM, 64) * P.batch * P.parts;
            const int64_t split = (blocks + sms - 1) / sms * ((ksteps + P.parts - 1) / P.parts * 590 + 11000);
            return split < best ? launch_split(left.box64, P, s) : launch_product<64, WHAT>(left.box64, right.box64, P, sms, s);
        }
    }
    int width = 64;
    const int64_t t128 = time(kTileM, 128, sms, 630, 8900);
    if (t128 < best) best = t128, width = 128;
    bool pair = false;
    for (int w = 160; w <= kPairWidth; w += 32) {
        const int64_t t = kSymmetric<WHAT> ? time(kPairM, w, sms / 2, 590 + 2 * w / 5, 6000 + 30 * w)
                                           : time(kPairM, w, sms / 2, 700, 13700);
        if (t < best || (pair && t == best)) best = t, width = w, pair = true;
    }
    if (pair) return launch_pairs<WHAT>(left.box128, kSymmetric<WHAT> ? right.box128 : right.box64, P, width, sms, s);
    if (width == 128) return launch_product<128, WHAT>(left.box64, right.box64, P, sms, s);
    return launch_product<64, WHAT>(left.box64, right.box64, P, sms, s);
}

template <bool CLUSTER, int NT>
bool launch_small(const MatrixIn& in, const SmallArgs& P, int32_t batch, cudaStream_t s) {
    const size_t most = (kSmallCols / 64 + 2) * kSlab + (CLUSTER ? 128 * 128 * 4 : 0) + 1024;
    static const bool ready = shared_memory(muon_small_kernel<CLUSTER, NT>, most);
    if (!ready) return false;
    const size_t smem = (P.cols / 64 + 2) * kSlab + (CLUSTER ? 128 * 128 * 4 : 0) + 1024;
    return launch_clusters(muon_small_kernel<CLUSTER, NT>, P.blocks, static_cast<int64_t>(batch) * P.blocks, NT, smem, s,
                           in, P);
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
    if (batch < 0 || in.rows < 0 || in.cols < 0 || batch > 65535 || in.rows > (1 << 20) || in.cols > (1 << 20))
        return CB_ERR_INVALID_ARG;
    if (steps < 1 || steps > kMaxSteps || !coefficients || !(eps >= 0.f) || !valid_dtype(in.dtype) ||
        !valid_dtype(out.dtype))
        return CB_ERR_INVALID_ARG;
    for (int k = 0; k < 3 * steps; ++k)
        if (!std::isfinite(coefficients[k])) return CB_ERR_INVALID_ARG;
    if (batch == 0 || in.rows == 0 || in.cols == 0) return CB_OK;
    const int64_t matrix = static_cast<int64_t>(in.rows) * in.cols;
    if (!in.g || !out.data || in.g_row < in.cols || out.row_stride < in.cols ||
        (batch > 1 && (in.g_batch < 0 || out.batch_stride < matrix)) || matrix > (int64_t(1) << 38) / batch)
        return CB_ERR_INVALID_ARG;
    if (in.momentum && (in.m_row < in.cols || (batch > 1 && in.m_batch < matrix))) return CB_ERR_INVALID_ARG;
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
    const Workspace w = layout(batch, in.rows, in.cols);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < static_cast<int64_t>(w.bytes)) return CB_ERR_CAPACITY;
    char* base = static_cast<char*>(workspace);
    if (!error) error = reinterpret_cast<int*>(base + w.error);  // any value: read by nobody
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
        if (!current_sms(&sms)) return CB_ERR_CUDA;
        const bool sent = blocks > 1                       ? launch_small<true, 512>(in, P, batch, s)
                          : P.cols <= 128 && batch > sms ? launch_small<false, 256>(in, P, batch, s)
                                                           : launch_small<false, 512>(in, P, batch, s);
        return cudaGetLastError() == cudaSuccess && sent ? CB_OK : CB_ERR_CUDA;
    }
    int sms = 0;
    if (!current_sms(&sms) || !tensor_map_encoder()) return CB_ERR_CUDA;
    __half* hi[2] = {reinterpret_cast<__half*>(base + w.hi[0]), reinterpret_cast<__half*>(base + w.hi[1])};
    __half* lo[2] = {reinterpret_cast<__half*>(base + w.lo[0]), reinterpret_cast<__half*>(base + w.lo[1])};
    __half* gram = reinterpret_cast<__half*>(base + w.gram);
    __half* poly = reinterpret_cast<__half*>(base + w.poly);
    SquareSum* partial = reinterpret_cast<SquareSum*>(base + w.partial);

    Operand op_x[2], op_gram, op_poly;
    if (!op_x[0].set(hi[0], w.q, w.p, batch, w.ldx) || !op_x[1].set(hi[1], w.q, w.p, batch, w.ldx) ||
        !op_gram.set(gram, w.p, w.p, batch, w.lda) || !op_poly.set(poly, w.p, w.p, batch, w.lda))
        return CB_ERR_CUDA;

    // 8192 values a block, on up to 2 blocks per SM in all.
    const int norm_blocks = static_cast<int>(
        max64(1, min64(min64(kNormBlocks, 2 * sms / batch), (matrix + 8 * 1024 - 1) / (8 * 1024))));
    const dim3 norm_grid(norm_blocks, batch);
    if (wide) launch(muon_norm_kernel<8>, norm_grid, dim3(kNormThreads), 0, s, in, partial);
    else if (vector) launch(muon_norm_kernel<4>, norm_grid, dim3(kNormThreads), 0, s, in, partial);
    else launch(muon_norm_kernel<1>, norm_grid, dim3(kNormThreads), 0, s, in, partial);
    const int cast_cols = (in.cols + kCastTile - 1) / kCastTile, cast_rows = (in.rows + kCastTile - 1) / kCastTile;
    const dim3 cast_grid(cast_cols,
                         static_cast<unsigned>(max64(1, min64(cast_rows, 8 * sms / (static_cast<int64_t>(cast_cols) * batch)))),
                         batch);
    const int64_t x_batch = w.p * w.ldx, a_batch = w.p * w.lda;
    const int ldx = static_cast<int>(w.ldx), lda = static_cast<int>(w.lda);
    auto cast = tall ? (vector ? muon_cast_kernel<true, 4> : muon_cast_kernel<true, 1>)
                     : (vector ? muon_cast_kernel<false, 4> : muon_cast_kernel<false, 1>);
    launch(cast, cast_grid, dim3(256), 0, s, in, static_cast<const SquareSum*>(partial), norm_blocks, eps, hi[0], lo[0], ldx,
           x_batch);

    bool sent = true;
    for (int k = 0; k < steps; ++k) {
        const int now = k & 1, next = now ^ 1;
        const float a = coefficients[3 * k], b = coefficients[3 * k + 1], c = coefficients[3 * k + 2];
        const bool two_term = k < kTwoTerm;
        ProductArgs P{};
        P.batch = batch;
        P.error = error;
        P.m = P.n = static_cast<int32_t>(w.p);
        P.k = static_cast<int32_t>(w.q);
        P.parts = gram_parts(w.p, w.q);
        P.out_hi = gram;
        P.out_batch = a_batch;
        P.out_ld = lda;
        sent &= launch_best<kGram>(op_x[now], op_x[now], P, sms, s);
        P.k = P.m;
        P.a = two_term ? 0.f : a;
        P.b = b;
        P.c = c;
        P.term_hi = gram;
        P.term_batch = a_batch;
        P.term_ld = lda;
        P.out_hi = poly;
        sent &= launch_best<kPoly>(op_gram, op_gram, P, sms, s);
        P.n = static_cast<int32_t>(w.q);
        P.a = two_term ? a : 0.f;
        P.term_hi = hi[now];
        P.term_lo = two_term ? lo[now] : nullptr;
        P.term_batch = x_batch;
        P.term_ld = ldx;
        P.out_hi = hi[next];
        P.out_lo = k + 1 < kTwoTerm ? lo[next] : nullptr;
        P.out_batch = x_batch;
        P.out_ld = ldx;
        if (k + 1 < steps) {
            sent &= launch_best<kUpdate>(op_poly, op_x[now], P, sms, s);
        } else {
            P.user = out.data;
            P.user_batch = out.batch_stride;
            P.user_row = out.row_stride;
            P.user_dtype = out.dtype;
            P.transposed = tall;
            P.user_vector = user_vector;
            P.weights = out.weights;
            P.keep = out.keep;
            P.rate = out.rate;
            sent &= launch_best<kResult>(op_poly, op_x[now], P, sms, s);
        }
    }
    return cudaGetLastError() == cudaSuccess && sent ? CB_OK : CB_ERR_CUDA;
}

}  // namespace
}  // namespace cbtbe

extern "C" int64_t cb_muon_workspace_bytes(int32_t batch, int32_t rows, int32_t cols) {
    if (batch <= 0 || rows <= 0 || cols <= 0) return 0;
    return static_cast<int64_t>(cbtbe::layout(batch, rows, cols).bytes);
}

extern "C" cb_status cb_muon_orthogonalise(const void* g, cb_dtype g_dtype, int32_t batch, int32_t rows, int32_t cols,
                                           int64_t g_batch_stride, int64_t g_row_stride, float eps,
                                           const float* coefficients, int32_t steps, void* out, cb_dtype out_dtype,
                                           int64_t out_batch_stride, int64_t out_row_stride, void* workspace,
                                           int64_t workspace_bytes, int* error, cudaStream_t stream) {
    using namespace cbtbe;
    MatrixIn in{};
    in.g = g;
    in.g_batch = g_batch_stride;
    in.g_row = g_row_stride;
    in.dtype = g_dtype;
    in.rows = rows;
    in.cols = cols;
    const Result r{out, out_dtype, out_batch_stride, out_row_stride, false, 0.f, 0.f};
    return orthogonalise(in, batch, eps, coefficients, steps, r, workspace, workspace_bytes, error, stream);
}

extern "C" cb_status cb_muon_step(void* weights, cb_dtype w_dtype, int64_t w_batch_stride, int64_t w_row_stride,
                                  const void* g, cb_dtype g_dtype, int64_t g_batch_stride, int64_t g_row_stride,
                                  float* momentum, int64_t m_batch_stride, int64_t m_row_stride, int32_t batch,
                                  int32_t rows, int32_t cols, float lr, float weight_decay, float beta, int nesterov,
                                  float eps, const float* coefficients, int32_t steps, float update_scale,
                                  void* workspace, int64_t workspace_bytes, int* error, cudaStream_t stream) {
    using namespace cbtbe;
    if (!(lr == lr) || !(weight_decay == weight_decay) || !(beta >= 0.f) || !(update_scale == update_scale))
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
    in.rows = rows;
    in.cols = cols;
    in.beta = beta;
    in.nesterov = nesterov;
    const Result r{weights, w_dtype, w_batch_stride, w_row_stride, true,
                   static_cast<float>(1.0 - static_cast<double>(lr) * weight_decay),
                   static_cast<float>(static_cast<double>(lr) * update_scale)};
    return orthogonalise(in, batch, eps, coefficients, steps, r, workspace, workspace_bytes, error, stream);
}
