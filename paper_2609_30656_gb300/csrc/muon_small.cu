// muon_small.cu -- Newton-Schulz steps of matrices that one block, or a cluster of a few, holds.
#include "muon_internal.cuh"

namespace cbtbe {
namespace muon {
namespace {

// Up to 128 x 3 K: all steps of a matrix in one kernel, by a cluster of blocks that each keep
// up to 384 columns of X in shared memory (fp16, for the products) and in TMEM (fp32, the term
// that B X is added to). The Gram matrix of the blocks' columns is added up
// across the cluster, in a fixed order, a share of its rows in each block; A A and B are
// taken by every block for itself. What is left of a step is a chain of three products
// of half a microsecond and their epilogues, in which a thread takes 32 columns of its row at a
// time: 512 threads a block (128 x 256, five steps: 34 us, 42 with 256), or 256 of
// two blocks per SM where narrow matrices would otherwise queue (300 of 128 x 128: 34 us, 47).
constexpr uint32_t kSlab = 128 * 128;  // bytes of 128 rows of 64 values

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
    __shared__ int failed;  // a wait ran out, here or (after a step's sums are exchanged) in the cluster
    __shared__ __align__(16) float squares[NT / 32 + 1][4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CLUSTER ? static_cast<int>(tc::cluster_rank()) : 0;
    const int b = blockIdx.x / P.blocks;
    const uint32_t columns = P.cols <= 128 ? 256 : 512;
    if (threadIdx.x == 0) {
        failed = 0;
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
    // What step `step` adds B hi to: (a - shift) hi + a lo = a X - shift hi, times kScaleA.
    auto to_term = [&](float (&v)[32], int step) {
        const float a = P.coefficients[3 * step] * kScaleA, shift = P.shift[step] * kScaleA;
#pragma unroll
        for (int k = 0; k < 32; k += 2) {  // two conversions at once, the same as those stored
            const float2 hi = __half22float2(__floats2half2_rn(v[k], v[k + 1]));
            v[k] = fmaf(a, v[k], -shift * hi.x);
            v[k + 1] = fmaf(a, v[k + 1], -shift * hi.y);
        }
    };
    for (int c = first; c < P.cols; c += NT / 4) {
        float v[32];
        tc::tmem_load32(sum_x + lanes + c, v);
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = (v[k] * f.x) * f.y;
        store_slab32(X + c / 64 * kSlab, row, c % 64, v);
        to_term(v, 0);
        tc::tmem_store32(sum_x + lanes + c, v);
    }

    // After a wait that ran out a thread waits no more and issues no products, but goes through the rest
    // with the others, so that the cluster's blocks stay in step; nothing is written at the end.
    bool ok = true;
    uint32_t phase = 0;
    auto handed_over = [&] {  // what all threads stored, to the tensor core
        tc::fence_to_tensor_core();
        tc::fence_before();
        __syncthreads();
    };
    auto products_done = [&] {
        if (ok && !tc::barrier_wait(tc::smem_addr(&done), phase)) {
            ok = false;
            failed = 1;
        }
        phase ^= 1;
        tc::fence_after();
    };
    const uint32_t x_at = tc::smem_addr(X), a_at = tc::smem_addr(A);
    for (int step = 0; step < P.steps; ++step) {
        const float bb = P.coefficients[3 * step + 1], cc = P.coefficients[3 * step + 2];
        const float diagonal = P.shift[step] * kScaleA;
        handed_over();
        if (threadIdx.x == 0 && ok) {  // A = X X^T
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
            if (threadIdx.x == 0)
                for (int k = 0; k < P.blocks; ++k)
                    if (tc::load_cluster_int(tc::in_block(tc::smem_addr(&failed), k)) != 0) failed = 1;
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
        if (threadIdx.x == 0 && ok) {  // A A
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
                    if (row == c + k + e) v[k + e] += diagonal;
                }
            }
            store_slab32(A + c / 64 * kSlab, row, c % 64, v);
        }
        handed_over();
        if (threadIdx.x == 0 && ok) {  // X <- (a - shift) hi + a lo + B hi
            tc::fence_after();
            for (int c = 0; c < P.cols; c += 256) {  // as many columns as one product takes
                const uint32_t shape = tc::mma_shape(128, P.cols - c < 256 ? P.cols - c : 256, true);
                for (int x = 0; x < 8; ++x)
                    tc::mma_f16<1>(sum_x + c, tc::operand_k_major(a_at + x / 4 * kSlab + x % 4 * 32),
                                   tc::operand_mn_major(x_at + c / 64 * kSlab + x * 2048, kSlab), shape, true);
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
                to_term(v, step + 1);
                tc::tmem_store32(sum_x + lanes + c, v);
            } else if (row < P.p && ok && !failed) {
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
    if (!ok && P.error) set_error(P.error, CB_ERR_TIMEOUT);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == 0) tc::tmem_free<1>(tmem_at, columns);
}

template <bool CLUSTER, int NT>
bool launch_blocks(const MatrixIn& in, const SmallArgs& P, int32_t batch, cudaStream_t s) {
    const size_t most = (kSmallCols / 64 + 2) * kSlab + (CLUSTER ? 128 * 128 * 4 : 0) + 1024;
    static std::atomic<uint64_t> devices{0};
    if (!shared_memory(muon_small_kernel<CLUSTER, NT>, most, devices)) return false;
    const size_t smem = (P.cols / 64 + 2) * kSlab + (CLUSTER ? 128 * 128 * 4 : 0) + 1024;
    return launch_clusters(muon_small_kernel<CLUSTER, NT>, P.blocks, static_cast<int64_t>(batch) * P.blocks, NT, smem, s,
                           in, P);
}

}  // namespace

bool launch_small(const MatrixIn& in, const SmallArgs& P, int32_t batch, int sms, cudaStream_t s) {
    if (P.blocks > 1) return launch_blocks<true, 512>(in, P, batch, s);
    if (P.cols <= 128 && batch > sms) return launch_blocks<false, 256>(in, P, batch, s);
    return launch_blocks<false, 512>(in, P, batch, s);
}

}  // namespace muon
}  // namespace cbtbe
