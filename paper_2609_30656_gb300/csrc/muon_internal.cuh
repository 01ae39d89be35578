// muon_internal.cuh -- what the kernels for orthogonalised updates share: the scales, the norm's
// sums, values of any type, and the launchers of the products (muon_products.cu) and of small
// matrices (muon_small.cu) for muon.cu.
#pragma once

#include <atomic>
#include <cmath>
#include <cudaTypedefs.h>

#include "tbe_internal.cuh"
#include "tensor_core.cuh"

namespace cbtbe {
namespace muon {

constexpr float kScaleX = 1024.f;  // X is stored times this,
constexpr float kScaleA = 256.f;   // A and B times this
constexpr int kMaxSteps = 64;

// What is added to the diagonal of B before it is rounded, and taken off a: the largest power of
// two not above -(b + c), so that on directions of singular value 1, where B is b + c, and on those that
// are still small, where it is 0, little is left to round (fp16's spacing halves below a power of
// two). 0 where b + c >= 0; 16 at most, which leaves B its range.
inline float diagonal_shift(float b, float c) {
    return b + c < 0.f ? std::fmin(std::ldexp(1.f, std::ilogb(-(b + c))), 16.f) : 0.f;
}

// ---------------------------------------------------------------- norm and momentum

// x^2 summed by magnitude: |x| >= 2^40 times 2^-160, |x| < 2^-40 times 2^160, the rest
// as it is, with what its additions and squares round off kept beside it: the norm of
// values in this middle range then is the same whatever the order of its sum (for a transposed or
// strided matrix, too); the outer classes are plain sums. A NaN goes with the rest.
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

// kScaleX / (norm + eps) as a product of two floats, so that neither a huge nor a tiny
// norm takes it out of range; in fp64 only where fp32's range asks for it.
__device__ __forceinline__ float2 inverse_norm(const SquareSum& t, float eps) {
    const float mid = t.mid + t.rest;
    // Up to 2^38 values below 2^-40 are 2^-42 of the sum: nothing beside 2^-16 in fp32.
    if (t.big == 0.f && (t.small == 0.f || mid >= 0x1p-16f) && mid >= 0x1p-60f)
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

// ---------------------------------------------------------------- products

enum Product {
    kGram,    // A = X X^T                          (symmetric)
    kPoly,    // B = b A + c A A + shift I          (symmetric)
    kUpdate,  // X' = (a - shift) hi + a lo + B hi
    kResult   // the same, into the caller's matrix
};
template <Product WHAT> constexpr bool kSymmetric = WHAT == kGram || WHAT == kPoly;

constexpr int kPartsMost = 4;

// Parts of K in which A = X X^T is summed, the parts' sums then added in order: as many blocks
// can share a tile (muon_split_kernel), and a result is the same whether they do or one block
// takes the parts in turn, so that a matrix gives the same bits alone and in a stack. Two or
// four, of a dozen steps of 64 at least, where a matrix is of few tiles.
inline int gram_parts(int64_t p, int64_t k) {
    const int64_t ksteps = (k + 63) / 64;
    return p > 512 || ksteps < 24 ? 1 : (ksteps < 48 ? 2 : 4);
}

struct ProductArgs {
    int32_t m, n, k;          // C [m, n], K
    int32_t batch;
    int32_t row_tiles, col_tiles;
    int32_t width;            // columns of a tile
    int32_t parts;            // kGram: parts of K summed apart (gram_parts)
    int64_t tiles;            // per matrix
    float a, b, c, shift;     // the step's coefficients, diagonal_shift(b, c)
    const __half* term_hi;    // kPoly: A; kUpdate, kResult: X
    const __half* term_lo;    // kUpdate, kResult
    int64_t term_batch;
    int32_t term_ld;
    __half* out_hi;
    __half* out_lo;           // kUpdate
    int64_t out_batch;
    int32_t out_ld;
    // kResult
    void* user;               // the caller's output, or weights
    int64_t user_batch, user_row;
    int32_t user_dtype;
    int32_t transposed;       // value (i, j) of C is value (j, i) of the caller's
    int32_t user_vector;      // its rows can be taken 4, or 8 (of 16 bits), values at a time; or 0
    int32_t user_sectors;     // it is not transposed and its rows are whole pieces of 32 bytes
    int32_t weights;          // W <- keep W - rate O, instead of O
    float keep, rate;
    int* error;               // the caller's, or null
    int* fault;               // this call's own: not 0 once a wait ran out; the last product then writes nothing
};

// A matrix of the workspace as an operand, by the boxes that a kernel copies.
struct Operand {
    CUtensorMap box64, box128;  // of 64 and 128 rows of 64 values
    bool set(const void* data, int64_t cols, int64_t rows, int64_t batch, int64_t ld);
};
bool tensor_maps_work();  // the driver's encoder can be reached
// C = left right, finished as `what` says, by the tiles with the least time.
bool launch_product(Product what, const Operand& left, const Operand& right, const ProductArgs& P, int sms,
                    cudaStream_t s);

// ---------------------------------------------------------------- small matrices

constexpr int kSmallRows = 128, kSmallCols = 384, kSmallCluster = 8;

struct SmallArgs {
    int32_t p, q, cols;      // X [p, q], columns per block (a multiple of 64)
    int32_t transposed, blocks, steps;
    float eps;
    float coefficients[3 * kMaxSteps], shift[kMaxSteps];
    void* user;
    int64_t user_batch, user_row;
    int32_t user_dtype, user_vector, in_vector;
    int32_t weights;
    float keep, rate;
    int* error;              // or null
};

// Blocks per matrix of muon_small_kernel (a power of two), 0 where it does not apply.
inline int small_blocks(int64_t p, int64_t q) {
    if (p > kSmallRows || q > kSmallCols * kSmallCluster) return 0;
    int blocks = 1;
    while (blocks * kSmallCols < q) blocks *= 2;
    return blocks;
}
// All steps of every matrix; P.blocks from small_blocks.
bool launch_small(const MatrixIn& in, const SmallArgs& P, int32_t batch, int sms, cudaStream_t s);

// ---------------------------------------------------------------- launches

// Lets a kernel have `bytes` of dynamic shared memory, once for each device that it runs on.
template <class KernelT>
inline bool shared_memory(KernelT kernel, size_t bytes, std::atomic<uint64_t>& devices) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const uint64_t bit = 1ull << (dev & 63);
    if (devices.load(std::memory_order_acquire) & bit) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)) != cudaSuccess)
        return false;
    devices.fetch_or(bit, std::memory_order_release);
    return true;
}

// As launch(), by clusters of `cluster` blocks.
template <class... Params, class... Args>
inline bool launch_clusters(void (*kernel)(Params...), int cluster, int64_t grid, int block, size_t smem, cudaStream_t s,
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

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

}  // namespace muon
}  // namespace cbtbe
