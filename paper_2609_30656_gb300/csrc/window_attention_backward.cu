// window_attention_backward.cu -- the backward pass of windowed attention by the tensor cores.
//
//   delta_t = do_t . o_t;  P = exp(S - lse),  dP = dO V^T,  dS = P (dP - delta)
//   dQ = scale dS K;  dK = scale dS^T Q;  dV = P^T dO
//
// Two kernels, one over tiles of queries (S, dP and dQ: three products a block of 128 x 128), one over tiles of keys
// (S^T, dP^T, dV and dK: four). One kernel would do with five, but dQ is then added up by many blocks: in fp32
// in memory, in an order that changes its bits. Sums stay in TMEM, heads that share keys are summed by one block.
//
// P and dS are operands in the rows' type. fp16 has five bits for exponents: P goes times 2^12, and dS times the
// power of two that brings the largest gradient to 16 .. 32, so that small gradients (and loss scales) keep
// their digits; a value that grows past fp16 all the same makes its row not finite, and such rows are computed
// again key by key in fp32 (as are those that met an infinity or a NaN behind a mask).
#include "window_attention_tc.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "muon_internal.cuh"

namespace cbtbe {
namespace attention {
namespace {

constexpr int kWorkWarps = 8, kCopyWarp = 8, kMultiplyWarp = 9, kStatWarp = 10, kThreads = 384;
constexpr int kMoreRegisters = 208, kFewerRegisters = 72;  // 256 x 208 + 128 x 72 of 384 x 168

template <bool BF16> constexpr float kPShift = BF16 ? 0.f : 12.f;
template <bool BF16>
__device__ __forceinline__ float slope_scale(const Shape& S) {
    if constexpr (BF16) return 1.f;
    const uint32_t bits = *S.largest;
    return bits == 0 ? 1.f : exp2f(static_cast<float>(4 - ilogbf(__uint_as_float(bits))));
}

// delta, and the largest |grad_out|: 16 bytes a lane, D / 8 lanes a row.
template <int D, bool BF16>
__global__ void __launch_bounds__(256) attention_delta_kernel(const Backward B) {
    constexpr int DT = BF16 ? CB_BF16 : CB_F16, kLanes = D / 8, kRowsAtOnce = 32 / kLanes;
    begin_kernel();
    const Shape& S = B.S;
    const int lane = threadIdx.x & 31, c = lane % kLanes * 8;
    const int64_t rows = S.tokens * S.heads;
    float largest = 0.f;
    for (int64_t i = warp_id_global() * kRowsAtOnce + lane / kLanes; i - lane / kLanes < rows; i += warps_in_grid() * kRowsAtOnce) {
        float a[8] = {}, b[8] = {}, sum = 0.f;
        const int64_t t = i / S.heads;
        const int h = static_cast<int>(i - t * S.heads);
        if (i < rows && c < S.dim) {
            widen<DT, 8>(load_piece<DT, 8>(static_cast<const uint16_t*>(B.go.data) + t * B.go.token + h * B.go.head + c), a);
            widen<DT, 8>(load_piece<DT, 8>(static_cast<const uint16_t*>(B.out.data) + t * B.out.token + h * B.out.head + c), b);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            sum = fmaf(a[k], b[k], sum);
            if constexpr (!BF16) largest = fabsf(a[k]) < INFINITY ? fmaxf(largest, fabsf(a[k])) : largest;
        }
#pragma unroll
        for (int off = kLanes / 2; off >= 1; off >>= 1) sum += __shfl_xor_sync(kFull, sum, off);
        if (i < rows && lane % kLanes == 0) B.delta[h * S.tokens + t] = sum;
    }
    if constexpr (!BF16) {
        const uint32_t most = __reduce_max_sync(kFull, __float_as_uint(largest));
        if (lane == 0 && most) atomicMax(S.largest, most);
    }
}

template <bool BF16, int D>
__device__ __forceinline__ void put_row(const float (&v)[kLaneValues], unsigned char* tile, int r) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int c = (threadIdx.x & 31) + 32 * i;
        *reinterpret_cast<uint16_t*>(tile + tile_byte(r, c / 8) + c % 8 * 2) =
            static_cast<uint16_t>(narrow<BF16 ? CB_BF16 : CB_F16>(v[i]));
    }
}
template <bool BF16, int D>
__device__ __noinline__ void dq_again(const Backward& B, int64_t t, int h, unsigned char* tile, int r) {
    float dq[kLaneValues];
    row_dq<BF16 ? CB_BF16 : CB_F16>(B, t, h, dq);
    put_row<BF16, D>(dq, tile, r);
}
template <bool BF16, int D>
__device__ __noinline__ void dkv_again(const Backward& B, int64_t j, int kv, bool keys, unsigned char* tile, int r) {
    float dk[kLaneValues], dv[kLaneValues];
    row_dkv<BF16 ? CB_BF16 : CB_F16>(B, j, kv, dk, dv);
    if (keys) put_row<BF16, D>(dk, tile, r);
    else put_row<BF16, D>(dv, tile, r);
}

// A row of sums from TMEM, times `by`, into its tile in shared memory; whether all are finite.
template <int D, bool BF16>
__device__ __forceinline__ bool finish_row(uint32_t at, float by, bool real, unsigned char* tile, int row) {
    bool finite = true;
#pragma unroll
    for (int d = 0; d < D; d += 32) {
        float o[32];
        tc::tmem_load32(at + d, o);
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
            uint32_t w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float lo = real ? o[k + 2 * u] * by : 0.f, hi = real ? o[k + 2 * u + 1] * by : 0.f;
                finite &= fabsf(lo) < INFINITY && fabsf(hi) < INFINITY;
                w[u] = pack2<BF16>(lo, hi);
            }
            *reinterpret_cast<uint4*>(tile + tile_byte(row, (d + k) / 8)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    return finite;
}
template <int D>
__device__ __forceinline__ void zero_row(unsigned char* tile, int row) {
#pragma unroll
    for (int d = 0; d < D; d += 8) *reinterpret_cast<uint4*>(tile + tile_byte(row, d / 8)) = make_uint4(0, 0, 0, 0);
}

// ---------------------------------------------------------------- dQ

constexpr int kQueryStages = 3;
template <int D> constexpr size_t kQueryShared = 1024 + (4 + kQueryStages) * kRowsBytes<D>;

// As the forward, two tiles of queries a block. A tile's S, dP and dS take turns in the same columns of TMEM (P stays in
// the row's thread meanwhile), so that two tiles fit with their dQ: one's products run beside the other's exponentials.
template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attention_dq_kernel(const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km,
                    const __grid_constant__ CUtensorMap vm, const __grid_constant__ CUtensorMap gm,
                    const __grid_constant__ CUtensorMap dqm, const __grid_constant__ Backward B, const bool pair_heads) {
    constexpr int S = kQueryStages;
    constexpr uint32_t kRows = kRowsBytes<D>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* queries = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    unsigned char* ring = queries + 4 * kRows;  // Q and dO of tile 0, of tile 1
    __shared__ uint64_t q_full, full[S], empty[S], scores[2], taken[2], grads[2], slopes[2], done;
    __shared__ uint32_t tmem_at;
    __shared__ SightParts parts[2];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const Work W = work_of(B.S, blockIdx.x, pair_heads);

    if (threadIdx.x == 0) {
        tc::barrier_init(tc::smem_addr(&q_full), 1);
        for (int i = 0; i < 2; ++i) {
            tc::barrier_init(tc::smem_addr(scores + i), 1);
            tc::barrier_init(tc::smem_addr(taken + i), 4);
            tc::barrier_init(tc::smem_addr(grads + i), 1);
            tc::barrier_init(tc::smem_addr(slopes + i), 4);
        }
        for (int i = 0; i < S; ++i) {
            tc::barrier_init(tc::smem_addr(full + i), 1);
            tc::barrier_init(tc::smem_addr(empty + i), 1);
        }
        tc::barrier_init(tc::smem_addr(&done), 1);
        tc::barrier_init_fence();
        for (const CUtensorMap* m : {&qm, &km, &vm, &gm, &dqm}) tc::tma_prefetch(m);
    }
    if (warp == kMultiplyWarp) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), 512);
    begin_kernel();
    const int mine = warp >> 2 & 1, row = threadIdx.x & 127;  // of the work warps
    const int64_t t = W.token[mine] + row;
    Row r{0, 0, false};
    if (warp < kWorkWarps) {
        r = row_of(B.S, t);
        note_row(parts[mine], r, static_cast<int>(t), warp & 3, lane);
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    const Blocks blocks(sight_of(parts[0], B.S.sinks), sight_of(parts[1], B.S.sinks));
    bool ok = true;

    if (warp >= kWorkWarps) {
        registers_down<kFewerRegisters>();
        if (warp == kCopyWarp && tc::elect()) {
            if (blocks.count > 0) {
                tc::barrier_expect(tc::smem_addr(&q_full), 4 * kRows);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    load_tile<D>(tc::smem_addr(queries) + 2 * i * kRows, &qm, tc::smem_addr(&q_full), W.head[i], W.token[i]);
                    load_tile<D>(tc::smem_addr(queries) + (2 * i + 1) * kRows, &gm, tc::smem_addr(&q_full), W.head[i], W.token[i]);
                }
            }
            int s = 0, issued = 0;
            uint32_t phase = 0;
            for (int i = 0; i < 2 * blocks.count; ++i) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                const uint32_t bar = tc::smem_addr(full + s);
                tc::barrier_expect(bar, kRows);
                load_tile<D>(tc::smem_addr(ring) + s * kRows, i & 1 ? &vm : &km, bar, W.kv, blocks.at(i >> 1).at);
                ++issued;
                if (++s == S) s = 0, phase ^= 1;
            }
            if (!ok)  // copies in flight land before the block's shared memory goes away
                for (int i = max(0, issued - S); i < issued; ++i)
                    if (!tc::barrier_wait(tc::smem_addr(full + i % S), i / S & 1)) break;
        }
        if (warp == kMultiplyWarp) {
            constexpr uint32_t shape_s = mma_shape<BF16>(kTile, kTile, false), shape_q = mma_shape<BF16>(kTile, D, true);
            const bool one = tc::elect();
            const uint32_t q0 = tc::smem_addr(queries), k0 = tc::smem_addr(ring);
            int s = 0;
            uint32_t phase = 0, taken_phase[2] = {0, 0}, slopes_phase[2] = {0, 0};
            bool begun[2] = {false, false};
            auto next = [&] { if (++s == S) s = 0, phase ^= 1; };
            auto multiply = [&](int x, uint32_t left, uint32_t stage, uint64_t* bar) {  // Q_x K^T or dO_x V^T
                if (!one) return;
                const uint64_t a = tc::operand_k_major(q0 + left * kRows), b = tc::operand_k_major(k0 + stage * kRows);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = k / 4 * kBoxBytes + k % 4 * 32;
                    tc::mma_f16<1>(tmem + x * 128, tc::advance(a, off), tc::advance(b, off), shape_s, k > 0);
                }
                tc::mma_commit<1>(tc::smem_addr(bar + x));
            };
            uint32_t k_stage = 0;
            if (blocks.count > 0) {
                ok = tc::barrier_wait(tc::smem_addr(&q_full), 0) && tc::barrier_wait(tc::smem_addr(full), 0);
                tc::fence_after();
                if (ok) {
                    const Blocks::Block b = blocks.at(0);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (b.use[x]) multiply(x, 2 * x, 0, scores);
                    next();
                }
            }
            for (int i = 0; i < blocks.count && ok; ++i) {
                const Blocks::Block b = blocks.at(i), c = blocks.at(i + 1);
                const bool more = i + 1 < blocks.count;
                const uint32_t v_stage = s;
                if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                next();
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!b.use[x]) continue;
                    if (!(ok = tc::barrier_wait(tc::smem_addr(taken + x), taken_phase[x]))) break;
                    taken_phase[x] ^= 1;
                    tc::fence_after();
                    multiply(x, 2 * x + 1, v_stage, grads);
                }
                if (!ok) break;
                if (one) tc::mma_commit<1>(tc::smem_addr(empty + v_stage));
                const uint32_t next_k = s;
                if (more) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                    next();
                }
                const uint64_t keys = tc::operand_mn_major(k0 + k_stage * kRows, kBoxBytes);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (b.use[x]) {
                        if (!(ok = tc::barrier_wait(tc::smem_addr(slopes + x), slopes_phase[x]))) break;
                        slopes_phase[x] ^= 1;
                        tc::fence_after();
                        if (one)
#pragma unroll
                            for (int k = 0; k < kTile / 16; ++k)
                                mma_tmem(tmem + 256 + x * D, tmem + x * 128 + k * 8, tc::advance(keys, k * 2048), shape_q, begun[x] || k > 0);
                        begun[x] = true;
                    }
                    if (more && c.use[x]) multiply(x, 2 * x, next_k, scores);
                }
                if (!ok) break;
                if (one) {
                    tc::mma_commit<1>(tc::smem_addr(empty + k_stage));
                    if (!more) tc::mma_commit<1>(tc::smem_addr(&done));
                }
                k_stage = next_k;
            }
        }
    } else {
        registers_up<kMoreRegisters>();
        const float c = B.S.scale * kLog2e, f = slope_scale<BF16>(B.S);
        float lse = 0.f, delta = 0.f;
        if (r.real) {
            lse = -B.lse[W.head[mine] * B.S.tokens + t] * kLog2e;
            delta = -B.delta[W.head[mine] * B.S.tokens + t] * f;
        }
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + mine * 128 + lanes, q_at = tmem + 256 + mine * D + lanes;
        const TwoRanges sees{r.first, r.real ? static_cast<int>(t) + 1 : 0, r.start,
                             r.real ? static_cast<int>(min64(static_cast<int64_t>(r.start) + B.S.sinks, r.first)) : 0};
        const float2 c2 = make_float2(c, c), lse2 = make_float2(lse, lse), f2 = make_float2(f, f), delta2 = make_float2(delta, delta);
        uint32_t phase = 0;
        bool any = false;
        for (int i = 0; i < blocks.count; ++i) {
            const Blocks::Block b = blocks.at(i);
            if (!b.use[mine]) continue;
            any = true;
            if (!(ok = tc::barrier_wait(tc::smem_addr(scores + mine), phase))) break;
            tc::fence_after();
            const bool whole = __all_sync(kFull, b.from[mine] <= b.at && b.to[mine] >= b.at + kTile && sees.all(b.at, kTile));
            uint32_t bits[4];
#pragma unroll
            for (int w = 0; w < 4; ++w)
                bits[w] = whole ? ~0u : sees.bits(b.at + w * 32) & range_bits(b.from[mine], b.to[mine], b.at + w * 32);
            uint32_t p[2][64];
            tmem_load64(s_at, p[0]);
            tmem_load64(s_at + 64, p[1]);
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::barrier_arrive(tc::smem_addr(taken + mine));
#pragma unroll
            for (int k = 0; k < 128; k += 2) {
                uint32_t &lo = p[k / 64][k % 64], &hi = p[k / 64][k % 64 + 1];
                const float2 x = fma2(make_float2(__uint_as_float(lo), __uint_as_float(hi)), c2, lse2);
                lo = __float_as_uint(exp2_fast(x.x));
                hi = __float_as_uint(exp2_fast(x.y));
            }
            if (!(ok = tc::barrier_wait(tc::smem_addr(grads + mine), phase))) break;
            phase ^= 1;
            tc::fence_after();
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t d[64], packed[32];
                tmem_load64(s_at + w * 64, d);
#pragma unroll
                for (int k = 0; k < 64; k += 2) {
                    float2 x = fma2(make_float2(__uint_as_float(d[k]), __uint_as_float(d[k + 1])), f2, delta2);
                    x = mul2(x, make_float2(__uint_as_float(p[w][k]), __uint_as_float(p[w][k + 1])));
                    if (!whole) {
                        x.x = bits[w * 2 + k / 32] >> k % 32 & 1 ? x.x : 0.f;
                        x.y = bits[w * 2 + k / 32] >> (k % 32 + 1) & 1 ? x.y : 0.f;
                    }
                    packed[k / 2] = pack2<BF16>(x.x, x.y);
                }
                tmem_store32_begin(s_at + w * 32, packed);
            }
            tmem_store_wait();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::barrier_arrive(tc::smem_addr(slopes + mine));
        }
        if (ok && any) ok = tc::barrier_wait(tc::smem_addr(&done), 0);
        if (ok && blocks.count > 0) ok = tc::barrier_wait(tc::smem_addr(&q_full), 0);
        tc::fence_after();
        unsigned char* tile = queries + 2 * mine * kRows;
        if (ok) {
            bool finite = true;
            if (any) finite = finish_row<D, BF16>(q_at, B.S.scale / f, r.real, tile, row);
            else zero_row<D>(tile, row);
            for (uint32_t left = __ballot_sync(kFull, !finite); left; left &= left - 1) {
                const int other = (row & ~31) + __ffs(left) - 1;
                __syncwarp();
                dq_again<BF16, D>(B, W.token[mine] + other, W.head[mine], tile, other);
            }
            fence_to_tma();
        }
        named_barrier(1 + mine, 128);
        if (ok && row == 0 && W.token[mine] < B.S.tokens) {
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
                tma_store(&dqm, tc::smem_addr(tile) + x * kBoxBytes, x * 64, W.head[mine], W.token[mine]);
            tma_store_done();
        }
    }
    if (!ok && B.S.error) set_error(B.S.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == kMultiplyWarp) tc::tmem_free<1>(tmem, 512);
}

// ---------------------------------------------------------------- dK and dV

constexpr int kKeyStages = 4, kStatStages = 4;
template <int D> constexpr size_t kKeyShared = 1024 + (2 + kKeyStages) * kRowsBytes<D>;

// A block has 128 keys of a head and takes the queries that see one of them, 128 at a time, for every head that
// shares the keys. S^T and dP^T have a key a lane, so that P^T and dS^T are operands from TMEM as they are; a warp takes
// half of the queries of its 32 keys. The products of a block follow one another as their operands
// come: S, dP | dV, S' (while dS is worked out) | dK, dP' (while P' is).
template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attention_dkv_kernel(const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km,
                     const __grid_constant__ CUtensorMap vm, const __grid_constant__ CUtensorMap gm,
                     const __grid_constant__ CUtensorMap dkm, const __grid_constant__ CUtensorMap dvm,
                     const __grid_constant__ Backward B) {
    constexpr int S = kKeyStages;
    constexpr uint32_t kRows = kRowsBytes<D>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* keys = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    unsigned char* ring = keys + 2 * kRows;  // K, V
    __shared__ uint64_t kv_full, full[S], empty[S], scores, weights, grads, slopes, done, stat_full[kStatStages], stat_empty[kStatStages];
    __shared__ uint32_t tmem_at;
    __shared__ int last_of[4];
    __shared__ __align__(16) float stats[kStatStages][2][kTile];  // -lse log2 e (+ shift) and -delta (times the slopes' scale)
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int tile_index = static_cast<int>(blockIdx.x / static_cast<unsigned>(B.S.kv_heads));
    const int kv = static_cast<int>(blockIdx.x - static_cast<unsigned>(tile_index) * B.S.kv_heads), first = tile_index * kTile;

    if (threadIdx.x == 0) {
        for (uint64_t* b : {&kv_full, &scores, &grads, &done}) tc::barrier_init(tc::smem_addr(b), 1);
        for (uint64_t* b : {&weights, &slopes}) tc::barrier_init(tc::smem_addr(b), kWorkWarps);
        for (int i = 0; i < S; ++i) {
            tc::barrier_init(tc::smem_addr(full + i), 1);
            tc::barrier_init(tc::smem_addr(empty + i), 1);
        }
        for (int i = 0; i < kStatStages; ++i) {
            tc::barrier_init(tc::smem_addr(stat_full + i), 1);
            tc::barrier_init(tc::smem_addr(stat_empty + i), kWorkWarps);
        }
        tc::barrier_init_fence();
        for (const CUtensorMap* m : {&qm, &km, &vm, &gm, &dkm, &dvm}) tc::tma_prefetch(m);
    }
    if (warp == kMultiplyWarp) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), 512);
    begin_kernel();
    const int row = threadIdx.x & 127, half = warp >> 2 & 1;
    const int64_t j = first + row;
    int last = 0;  // behind the last token that sees key j
    bool real = false;
    if (warp < kWorkWarps && j < B.S.tokens && B.S.end[j] > j) {
        real = true;
        last = static_cast<int>(j - B.S.start[j] < B.S.sinks ? B.S.end[j] : min64(B.S.end[j], j + B.S.window));
    }
    if (warp < 4) {
        const int most = __reduce_max_sync(kFull, last);
        if (lane == 0) last_of[warp] = most;
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    const int until = max(max(last_of[0], last_of[1]), max(last_of[2], last_of[3]));
    const int blocks = tiles_of(max(until - first, 0));  // of queries, for each head
    const int64_t count = static_cast<int64_t>(blocks) * B.S.group;
    const int head0 = kv * B.S.group;
    bool ok = true;

    if (warp >= kWorkWarps) {
        registers_down<kFewerRegisters>();
        if (warp == kCopyWarp && tc::elect()) {
            if (count > 0) {
                tc::barrier_expect(tc::smem_addr(&kv_full), 2 * kRows);
                load_tile<D>(tc::smem_addr(keys), &km, tc::smem_addr(&kv_full), kv, first);
                load_tile<D>(tc::smem_addr(keys) + kRows, &vm, tc::smem_addr(&kv_full), kv, first);
            }
            int s = 0, h = 0, i = 0;
            uint32_t phase = 0;
            int64_t issued = 0;
            for (int64_t n = 0; n < 2 * count; ++n) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                const uint32_t bar = tc::smem_addr(full + s);
                tc::barrier_expect(bar, kRows);
                load_tile<D>(tc::smem_addr(ring) + s * kRows, n & 1 ? &gm : &qm, bar, head0 + h, first + i * kTile);
                ++issued;
                if (++s == S) s = 0, phase ^= 1;
                if (n & 1)
                    if (++i == blocks) i = 0, ++h;
            }
            if (!ok)
                for (int64_t n = max64(0, issued - S); n < issued; ++n)
                    if (!tc::barrier_wait(tc::smem_addr(full + n % S), n / S & 1)) break;
        }
        if (warp == kStatWarp) {
            const float f = slope_scale<BF16>(B.S) * exp2f(-kPShift<BF16>);
            int s = 0, h = 0, i = 0;
            uint32_t phase = 0;
            for (int64_t n = 0; n < count; ++n) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(stat_empty + s), phase ^ 1))) break;
#pragma unroll
                for (int k = 0; k < kTile / 32; ++k) {
                    const int64_t t = first + static_cast<int64_t>(i) * kTile + k * 32 + lane;
                    const int64_t at = (head0 + h) * B.S.tokens + t;
                    stats[s][0][k * 32 + lane] = t < B.S.tokens ? kPShift<BF16> - B.lse[at] * kLog2e : 0.f;
                    stats[s][1][k * 32 + lane] = t < B.S.tokens ? -B.delta[at] * f : 0.f;
                }
                __syncwarp();
                if (lane == 0) tc::barrier_arrive(tc::smem_addr(stat_full + s));
                if (++s == kStatStages) s = 0, phase ^= 1;
                if (++i == blocks) i = 0, ++h;
            }
        }
        if (warp == kMultiplyWarp && count > 0) {
            constexpr uint32_t shape_s = mma_shape<BF16>(kTile, kTile, false), shape_d = mma_shape<BF16>(kTile, D, true);
            const bool one = tc::elect();
            const uint32_t k0 = tc::smem_addr(keys), q0 = tc::smem_addr(ring);
            auto multiply = [&](uint32_t left, int stage, uint32_t to, uint64_t* bar) {  // K Q^T or V dO^T
                if (!one) return;
                const uint64_t a = tc::operand_k_major(k0 + left * kRows), b = tc::operand_k_major(q0 + stage * kRows);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t off = k / 4 * kBoxBytes + k % 4 * 32;
                    tc::mma_f16<1>(tmem + to, tc::advance(a, off), tc::advance(b, off), shape_s, k > 0);
                }
                tc::mma_commit<1>(tc::smem_addr(bar));
            };
            auto accumulate = [&](uint32_t from, int stage, uint32_t to, bool add) {  // P^T dO or dS^T Q
                if (!one) return;
                const uint64_t b = tc::operand_mn_major(q0 + stage * kRows, kBoxBytes);
#pragma unroll
                for (int k = 0; k < kTile / 16; ++k)  // half of the queries in columns 0 .. 31, half in 64 .. 95
                    mma_tmem(tmem + to, tmem + from + k / 4 * 64 + k % 4 * 8, tc::advance(b, k * 2048), shape_d, add || k > 0);
            };
            auto wait = [&](uint64_t* bar, int64_t n) { return tc::barrier_wait(tc::smem_addr(bar), static_cast<uint32_t>(n & 1)); };
            // The tile of turn m in the ring (Q of block n: m = 2 n, dO: 2 n + 1).
            auto wait_full = [&](int64_t m) { return tc::barrier_wait(tc::smem_addr(full + m % S), static_cast<uint32_t>(m / S & 1)); };
            ok = tc::barrier_wait(tc::smem_addr(&kv_full), 0) && wait_full(0) && wait_full(1);
            tc::fence_after();
            if (ok) {
                multiply(0, 0, 0, &scores);
                multiply(1, 1, 128, &grads);
            }
            for (int64_t n = 0; n < count && ok; ++n) {
                const int q = static_cast<int>(2 * n % S), g = q + 1, q_next = static_cast<int>((2 * n + 2) % S);
                const bool more = n + 1 < count;
                if (!(ok = wait(&weights, n))) break;
                tc::fence_after();
                accumulate(0, g, 256, n > 0);
                if (more) {
                    if (!(ok = wait_full(2 * n + 2))) break;
                    multiply(0, q_next, 0, &scores);
                }
                if (!(ok = wait(&slopes, n))) break;
                tc::fence_after();
                accumulate(128, q, 256 + D, n > 0);
                if (one) {
                    tc::mma_commit<1>(tc::smem_addr(empty + q));
                    tc::mma_commit<1>(tc::smem_addr(empty + g));
                }
                if (more) {
                    if (!(ok = wait_full(2 * n + 3))) break;
                    multiply(1, q_next + 1, 128, &grads);
                } else if (one) {
                    tc::mma_commit<1>(tc::smem_addr(&done));
                }
            }
        }
    } else {
        registers_up<kMoreRegisters>();
        const float c = B.S.scale * kLog2e, f = slope_scale<BF16>(B.S) * exp2f(-kPShift<BF16>);
        const float2 c2 = make_float2(c, c), f2 = make_float2(f, f);
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + lanes + half * 64, g_at = s_at + 128;
        const TwoRanges seen{static_cast<int>(j), last, 0, 0};
        int s = 0, i = 0;
        uint32_t stat_phase = 0;
        for (int64_t n = 0; n < count; ++n) {
            const uint32_t phase = static_cast<uint32_t>(n & 1);
            const int at = first + i * kTile + half * 64;
            if (++i == blocks) i = 0;
            const bool whole = __all_sync(kFull, seen.all(at, 64));
            const uint32_t bits[2] = {seen.bits(at), seen.bits(at + 32)};
            if (!(ok = tc::barrier_wait(tc::smem_addr(stat_full + s), stat_phase))) break;
            if (!(ok = tc::barrier_wait(tc::smem_addr(&scores), phase))) break;
            tc::fence_after();
            uint32_t p[64], packed[32];
            tmem_load64(s_at, p);
            const float4* lse = reinterpret_cast<const float4*>(stats[s][0] + half * 64);
            const float4* delta = reinterpret_cast<const float4*>(stats[s][1] + half * 64);
#pragma unroll
            for (int k = 0; k < 64; k += 4) {
                const float4 l = lse[k / 4];
                float2 x = fma2(make_float2(__uint_as_float(p[k]), __uint_as_float(p[k + 1])), c2, make_float2(l.x, l.y));
                float2 y = fma2(make_float2(__uint_as_float(p[k + 2]), __uint_as_float(p[k + 3])), c2, make_float2(l.z, l.w));
                x.x = exp2_fast(x.x);
                x.y = exp2_fast(x.y);
                y.x = exp2_fast(y.x);
                y.y = exp2_fast(y.y);
                if (!whole) {
                    x.x = bits[k / 32] >> k % 32 & 1 ? x.x : 0.f;
                    x.y = bits[k / 32] >> (k % 32 + 1) & 1 ? x.y : 0.f;
                    y.x = bits[k / 32] >> (k % 32 + 2) & 1 ? y.x : 0.f;
                    y.y = bits[k / 32] >> (k % 32 + 3) & 1 ? y.y : 0.f;
                }
                packed[k / 2] = pack2<BF16>(x.x, x.y);
                packed[k / 2 + 1] = pack2<BF16>(y.x, y.y);
                p[k] = __float_as_uint(x.x);
                p[k + 1] = __float_as_uint(x.y);
                p[k + 2] = __float_as_uint(y.x);
                p[k + 3] = __float_as_uint(y.y);
            }
            tmem_store32_begin(s_at, packed);
            tmem_store_wait();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::barrier_arrive(tc::smem_addr(&weights));
            if (!(ok = tc::barrier_wait(tc::smem_addr(&grads), phase))) break;
            tc::fence_after();
            uint32_t d[64];
            tmem_load64(g_at, d);
#pragma unroll
            for (int k = 0; k < 64; k += 4) {
                const float4 l = delta[k / 4];
                float2 x = fma2(make_float2(__uint_as_float(d[k]), __uint_as_float(d[k + 1])), f2, make_float2(l.x, l.y));
                float2 y = fma2(make_float2(__uint_as_float(d[k + 2]), __uint_as_float(d[k + 3])), f2, make_float2(l.z, l.w));
                x = mul2(x, make_float2(__uint_as_float(p[k]), __uint_as_float(p[k + 1])));
                y = mul2(y, make_float2(__uint_as_float(p[k + 2]), __uint_as_float(p[k + 3])));
                if (!whole) {
                    x.x = bits[k / 32] >> k % 32 & 1 ? x.x : 0.f;
                    x.y = bits[k / 32] >> (k % 32 + 1) & 1 ? x.y : 0.f;
                    y.x = bits[k / 32] >> (k % 32 + 2) & 1 ? y.x : 0.f;
                    y.y = bits[k / 32] >> (k % 32 + 3) & 1 ? y.y : 0.f;
                }
                packed[k / 2] = pack2<BF16>(x.x, x.y);
                packed[k / 2 + 1] = pack2<BF16>(y.x, y.y);
            }
            tmem_store32_begin(g_at, packed);
            tmem_store_wait();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) {
                tc::barrier_arrive(tc::smem_addr(&slopes));
                tc::barrier_arrive(tc::smem_addr(stat_empty + s));
            }
            if (++s == kStatStages) s = 0, stat_phase ^= 1;
        }
        // The first four warps finish dV, the others dK, in the place of V and K.
        if (ok && count > 0) ok = tc::barrier_wait(tc::smem_addr(&done), 0);
        tc::fence_after();
        unsigned char* tile = keys + (half ? 0 : kRows);
        if (ok) {
            bool finite = true;
            const float by = half ? B.S.scale / slope_scale<BF16>(B.S) : exp2f(-kPShift<BF16>);
            if (count > 0) finite = finish_row<D, BF16>(tmem + lanes + 256 + half * D, by, real, tile, row);
            else zero_row<D>(tile, row);
            for (uint32_t left = __ballot_sync(kFull, !finite); left; left &= left - 1) {
                const int other = (row & ~31) + __ffs(left) - 1;
                __syncwarp();
                dkv_again<BF16, D>(B, first + other, kv, half, tile, other);
            }
            fence_to_tma();
        }
        named_barrier(1 + half, 128);
        if (ok && row == 0) {
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
                tma_store(half ? &dkm : &dvm, tc::smem_addr(tile) + x * kBoxBytes, x * 64, kv, first);
            tma_store_done();
        }
    }
    if (!ok && B.S.error) set_error(B.S.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == kMultiplyWarp) tc::tmem_free<1>(tmem, 512);
}

template <int D, bool BF16>
bool launch_typed(const Backward& B, cudaStream_t s) {
    const Shape& S = B.S;
    CUtensorMap qm, km, vm, gm, dqm, dkm, dvm;
    if (!tile_map(&qm, B.q, S.tokens, S.heads, S.dim, S.dtype) || !tile_map(&km, B.k, S.tokens, S.kv_heads, S.dim, S.dtype) ||
        !tile_map(&vm, B.v, S.tokens, S.kv_heads, S.dim, S.dtype) || !tile_map(&gm, B.go, S.tokens, S.heads, S.dim, S.dtype) ||
        !tile_map(&dqm, B.dq, S.tokens, S.heads, S.dim, S.dtype) || !tile_map(&dkm, B.dk, S.tokens, S.kv_heads, S.dim, S.dtype) ||
        !tile_map(&dvm, B.dv, S.tokens, S.kv_heads, S.dim, S.dtype))
        return false;
    static std::atomic<uint64_t> dq_devices{0}, dkv_devices{0};
    if (!muon::shared_memory(attention_dq_kernel<D, BF16>, kQueryShared<D>, dq_devices) ||
        !muon::shared_memory(attention_dkv_kernel<D, BF16>, kKeyShared<D>, dkv_devices))
        return false;
    const int64_t key_tiles = (S.tokens + kTile - 1) / kTile * S.kv_heads, items = work_items(S);
    if (items > INT32_MAX || key_tiles > INT32_MAX) return false;
    launch(attention_delta_kernel<D, BF16>, dim3(warp_grid((S.tokens * S.heads * D / 8 + 31) / 32, 152 * 32)), dim3(256), 0, s, B);
    launch(attention_dkv_kernel<D, BF16>, dim3(static_cast<unsigned>(key_tiles)), dim3(kThreads), kKeyShared<D>, s, qm, km, vm, gm,
           dkm, dvm, B);
    launch(attention_dq_kernel<D, BF16>, dim3(static_cast<unsigned>(items)), dim3(kThreads), kQueryShared<D>, s, qm, km, vm, gm, dqm,
           B, pairs_heads(S));
    return true;
}

}  // namespace

bool launch_backward(const Backward& B, cudaStream_t s) {
    if (B.S.dtype == CB_BF16) return B.S.dim <= 64 ? launch_typed<64, true>(B, s) : launch_typed<128, true>(B, s);
    return B.S.dim <= 64 ? launch_typed<64, false>(B, s) : launch_typed<128, false>(B, s);
}

}  // namespace attention
}  // namespace cbtbe
