// window_attention_forward.cu -- windowed attention over packed sessions by the tensor cores.
//
// A block takes two tiles of 128 queries that read the same key and value heads (the same tokens of two heads
// that share them, else 256 tokens of one head) through their keys, 128 at a time, with one pass
// softmax: S = Q K^T into TMEM, P = exp(S - m) back into TMEM over it, O += P V from there. One warp copies, one
// issues the products, four for each tile have a row a thread (no shuffles: a lane reads its row of S from TMEM).
// While one tile's warps are at their exponentials, the other's products run. O stays in TMEM; it is scaled
// down only where a row's maximum has risen by more than 2^8 (the sums have room for that), by the row's own thread.
#include "window_attention_tc.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "muon_internal.cuh"

namespace cbtbe {
namespace attention {
namespace {

constexpr int kSoftmaxWarps = 8, kCopyWarp = 8, kMultiplyWarp = 9, kThreads = 384;  // two warps are idle
template <int D> constexpr int kStages = D == 64 ? 8 : 4;
template <int D> constexpr size_t kShared = 1024 + (2 + kStages<D>) * kRowsBytes<D>;
// Of the 168 registers that a thread is launched with, the copying warps give some to the softmax warps, whose
// threads hold a row of 128 scores: 256 x 208 + 128 x 72 of the block's 384 x 168.
constexpr int kMoreRegisters = 208, kFewerRegisters = 72;
constexpr float kRise = 8.f;  // how far, in powers of two, exponents may lie above the maximum they began with

template <bool BF16, int D>
__device__ __noinline__ void output_again(const Forward& F, int64_t t, int h, unsigned char* tile, int r) {
    float o[kLaneValues], lse;
    row_output<BF16 ? CB_BF16 : CB_F16>(F, t, h, o, lse);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int c = (threadIdx.x & 31) + 32 * i;
        *reinterpret_cast<uint16_t*>(tile + tile_byte(r, c / 8) + c % 8 * 2) =
            static_cast<uint16_t>(narrow<BF16 ? CB_BF16 : CB_F16>(o[i]));
    }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attention_forward_kernel(const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km,
                         const __grid_constant__ CUtensorMap vm, const __grid_constant__ CUtensorMap om,
                         const __grid_constant__ Forward F, const bool pair_heads) {
    constexpr int S = kStages<D>;
    constexpr uint32_t kRows = kRowsBytes<D>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* queries = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    unsigned char* ring = queries + 2 * kRows;
    __shared__ uint64_t q_full[2], full[S], empty[S], scores[2], weights[2], done;
    __shared__ uint32_t tmem_at;
    __shared__ SightParts parts[2];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const Work W = work_of(F.S, blockIdx.x, pair_heads);

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            tc::barrier_init(tc::smem_addr(q_full + i), 1);
            tc::barrier_init(tc::smem_addr(scores + i), 1);
            tc::barrier_init(tc::smem_addr(weights + i), 4);
        }
        for (int i = 0; i < S; ++i) {
            tc::barrier_init(tc::smem_addr(full + i), 1);
            tc::barrier_init(tc::smem_addr(empty + i), 1);
        }
        tc::barrier_init(tc::smem_addr(&done), 1);
        tc::barrier_init_fence();
        tc::tma_prefetch(&qm);
        tc::tma_prefetch(&km);
        tc::tma_prefetch(&vm);
        tc::tma_prefetch(&om);
    }
    if (warp == kMultiplyWarp) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), 512);
    begin_kernel();
    const int mine = warp >> 2 & 1, row = threadIdx.x & 127;  // of the softmax warps
    const int64_t t = W.token[mine] + row;
    Row r{0, 0, false};
    if (warp < kSoftmaxWarps) {
        r = row_of(F.S, t);
        note_row(parts[mine], r, static_cast<int>(t), warp & 3, lane);
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    const Blocks blocks(sight_of(parts[0], F.S.sinks), sight_of(parts[1], F.S.sinks));
    bool ok = true;

    if (warp >= kSoftmaxWarps) {
        registers_down<kFewerRegisters>();
        if (warp == kCopyWarp && tc::elect()) {
            if (blocks.count > 0) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    tc::barrier_expect(tc::smem_addr(q_full + i), kRows);
                    load_tile<D>(tc::smem_addr(queries) + i * kRows, &qm, tc::smem_addr(q_full + i), W.head[i], W.token[i]);
                }
            }
            int s = 0;
            uint32_t phase = 0;
            int issued = 0;
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
        constexpr uint32_t shape_s = mma_shape<BF16>(kTile, kTile, false), shape_o = mma_shape<BF16>(kTile, D, true);
        const bool one = tc::elect();
        const uint32_t q0 = tc::smem_addr(queries), k0 = tc::smem_addr(ring);
        int s = 0;  // stage of the next copy
        uint32_t phase = 0;
        uint32_t weights_phase[2] = {0, 0};
        bool begun[2] = {false, false};
        auto next = [&] { if (++s == S) s = 0, phase ^= 1; };
        auto multiply_scores = [&](int x, uint32_t stage) {  // S_x = Q_x K^T
            if (!one) return;
            const uint64_t a = tc::operand_k_major(q0 + x * kRows), b = tc::operand_k_major(k0 + stage * kRows);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = k / 4 * kBoxBytes + k % 4 * 32;
                tc::mma_f16<1>(tmem + x * 128, tc::advance(a, off), tc::advance(b, off), shape_s, k > 0);
            }
            tc::mma_commit<1>(tc::smem_addr(scores + x));
        };
        if (blocks.count > 0) {
            ok = tc::barrier_wait(tc::smem_addr(q_full), 0) && tc::barrier_wait(tc::smem_addr(q_full + 1), 0) &&
                 tc::barrier_wait(tc::smem_addr(full), 0);
            tc::fence_after();
            if (ok) {
                const Blocks::Block b = blocks.at(0);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (b.use[x]) multiply_scores(x, 0);
                if (one) tc::mma_commit<1>(tc::smem_addr(empty));
                next();
            }
        }
        for (int i = 0; i < blocks.count && ok; ++i) {
            const Blocks::Block b = blocks.at(i);
            const bool more = i + 1 < blocks.count;
            const Blocks::Block c = blocks.at(i + 1);
            const uint32_t v_stage = s;
            if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
            next();
            const uint32_t k_stage = s;
            if (more) {
                if (!(ok = tc::barrier_wait(tc::smem_addr(full + s), phase))) break;
                next();
            }
            const uint64_t v = tc::operand_mn_major(k0 + v_stage * kRows, kBoxBytes);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (b.use[x]) {
                    if (!(ok = tc::barrier_wait(tc::smem_addr(weights + x), weights_phase[x]))) break;
                    weights_phase[x] ^= 1;
                    tc::fence_after();
                    if (one)
#pragma unroll
                        for (int k = 0; k < kTile / 16; ++k)
                            mma_tmem(tmem + 256 + x * D, tmem + x * 128 + k * 8, tc::advance(v, k * 2048), shape_o, begun[x] || k > 0);
                    begun[x] = true;
                }
                if (more && c.use[x]) multiply_scores(x, k_stage);
            }
            if (!ok) break;
            if (one) {
                tc::mma_commit<1>(tc::smem_addr(empty + v_stage));
                if (more) tc::mma_commit<1>(tc::smem_addr(empty + k_stage));
                else tc::mma_commit<1>(tc::smem_addr(&done));
            }
        }
        }
    } else {
        registers_up<kMoreRegisters>();
        // exponentials: x = s c - m c in powers of two, c > 0 (the sign of the scale goes to s)
        const float c = fmaxf(fabsf(F.S.scale) * kLog2e, 1e-30f);
        const uint32_t flip = F.S.scale < 0.f ? 0x80000000u : 0u;
        // fp16 holds P times 2^6: its small values keep their digits, and P <= 2^8.
        constexpr float kShift = BF16 ? 0.f : 6.f;
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + mine * 128 + lanes, o_at = tmem + 256 + mine * D + lanes;
        const TwoRanges sees{r.first, r.real ? static_cast<int>(t) + 1 : 0, r.start,
                             r.real ? static_cast<int>(min64(static_cast<int64_t>(r.start) + F.S.sinks, r.first)) : 0};
        float most = -INFINITY;  // of the raw scores, that the exponents are taken against
        float2 sums = make_float2(0.f, 0.f);
        uint32_t phase = 0;
        bool any = false;
        for (int i = 0; i < blocks.count; ++i) {
            const Blocks::Block b = blocks.at(i);
            if (!b.use[mine]) continue;
            if (!(ok = tc::barrier_wait(tc::smem_addr(scores + mine), phase))) break;
            phase ^= 1;
            tc::fence_after();
            uint32_t v[2][64];
            tmem_load64(s_at, v[0]);
            tmem_load64(s_at + 64, v[1]);
            if (flip)
#pragma unroll
                for (int k = 0; k < 128; ++k) v[k / 64][k % 64] ^= flip;
            const bool whole = b.from[mine] <= b.at && b.to[mine] >= b.at + kTile && sees.all(b.at, kTile);
            if (!__all_sync(kFull, whole)) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t bits = sees.bits(b.at + w * 32) & range_bits(b.from[mine], b.to[mine], b.at + w * 32);
#pragma unroll
                    for (int k = 0; k < 32; ++k)
                        if (!(bits >> k & 1)) v[w / 2][w % 2 * 32 + k] = 0xff800000u;
                }
            }
            float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < 128; k += 4)
#pragma unroll
                for (int u = 0; u < 4; ++u) top[u] = fmaxf(top[u], __uint_as_float(v[k / 64][k % 64 + u]));
            const float highest = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            if (__any_sync(kFull, (highest - most) * c > kRise)) {  // false for two infinities
                const float raised = fmaxf(most, highest);
                const float keep = raised == most ? 1.f : exp2_fast((most - raised) * c);
                most = raised;
                sums = make_float2(sums.x * keep, sums.y * keep);
                if (any) {
#pragma unroll
                    for (int d = 0; d < D; d += 32) {
                        float o[32];
                        tc::tmem_load32(o_at + d, o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] *= keep;
                        tc::tmem_store32(o_at + d, o);
                    }
                }
            }
            any = true;
            const float base = most == -INFINITY ? 0.f : kShift - most * c;
            const float2 c2 = make_float2(c, c), base2 = make_float2(base, base);
            float2 more = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                uint32_t p[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    float2 x = fma2(make_float2(__uint_as_float(v[w][2 * k]), __uint_as_float(v[w][2 * k + 1])), c2, base2);
                    x.x = exp2_fast(x.x);
                    x.y = exp2_fast(x.y);
                    if (k & 1) more = add2(more, x);
                    else sums = add2(sums, x);
                    p[k] = pack2<BF16>(x.x, x.y);
                }
                tmem_store32_begin(s_at + w * 32, p);
            }
            sums = add2(sums, more);
            tmem_store_wait();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::barrier_arrive(tc::smem_addr(weights + mine));
        }
        // The last products are done with Q, whose place the output takes; a tile without keys waits for its copy.
        if (ok && any) ok = tc::barrier_wait(tc::smem_addr(&done), 0);
        if (ok && blocks.count > 0) ok = tc::barrier_wait(tc::smem_addr(q_full + mine), 0);
        tc::fence_after();
        unsigned char* tile = queries + mine * kRows;
        if (ok) {
            const float sum = sums.x + sums.y;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;  // a NaN stays one
            bool again = false;
#pragma unroll
            for (int d = 0; d < D; d += 32) {
                float o[32];
                if (any) tc::tmem_load32(o_at + d, o);
#pragma unroll
                for (int k = 0; k < 32; k += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float lo = r.real && any ? o[k + 2 * u] * inv : 0.f, hi = r.real && any ? o[k + 2 * u + 1] * inv : 0.f;
                        again |= !(fabsf(lo) < INFINITY) || !(fabsf(hi) < INFINITY);
                        w[u] = pack2<BF16>(lo, hi);
                    }
                    *reinterpret_cast<uint4*>(tile + tile_byte(row, (d + k) / 8)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            for (uint32_t left = __ballot_sync(kFull, again); left; left &= left - 1) {
                const int other = (row & ~31) + __ffs(left) - 1;
                __syncwarp();
                output_again<BF16, D>(F, W.token[mine] + other, W.head[mine], tile, other);
            }
            if (F.lse && t < F.S.tokens)
                F.lse[W.head[mine] * F.S.tokens + t] = r.real ? ((most == -INFINITY ? 0.f : most * c) + __log2f(sum) - kShift) * kLn2 : -INFINITY;
            tc::fence_to_tensor_core();
        }
        named_barrier(1 + mine, 128);
        if (ok && row == 0 && W.token[mine] < F.S.tokens) {
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
                tma_store(&om, tc::smem_addr(tile) + x * kBoxBytes, x * 64, W.head[mine], W.token[mine]);
            tma_store_done();
        }
    }
    if (!ok && F.S.error) set_error(F.S.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == kMultiplyWarp) tc::tmem_free<1>(tmem, 512);
}

template <int D, bool BF16>
bool launch_typed(const Forward& F, cudaStream_t s) {
    CUtensorMap qm, km, vm, om;
    const Shape& S = F.S;
    if (!tile_map(&qm, F.q, S.tokens, S.heads, S.dim, S.dtype) || !tile_map(&km, F.k, S.tokens, S.kv_heads, S.dim, S.dtype) ||
        !tile_map(&vm, F.v, S.tokens, S.kv_heads, S.dim, S.dtype) || !tile_map(&om, F.out, S.tokens, S.heads, S.dim, S.dtype))
        return false;
    static std::atomic<uint64_t> devices{0};
    if (!muon::shared_memory(attention_forward_kernel<D, BF16>, kShared<D>, devices)) return false;
    const bool pair_heads = pairs_heads(S);
    const int64_t grid = work_items(S);
    if (grid > INT32_MAX) return false;
    launch(attention_forward_kernel<D, BF16>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), kShared<D>, s, qm, km, vm, om, F,
           pair_heads);
    return true;
}

}  // namespace

bool launch_forward(const Forward& F, cudaStream_t s) {
    if (F.S.dtype == CB_BF16) return F.S.dim <= 64 ? launch_typed<64, true>(F, s) : launch_typed<128, true>(F, s);
    return F.S.dim <= 64 ? launch_typed<64, false>(F, s) : launch_typed<128, false>(F, s);
}

}  // namespace attention
}  // namespace cbtbe
