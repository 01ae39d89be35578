// window_attention_backward.cu -- the backward pass of windowed attention by the tensor cores.
//
//   delta_t = do_t . o_t;  P = exp(S - lse),  dP = dO V^T,  dS = P (dP - delta)
//   dQ = scale dS K;  dK = scale dS^T Q;  dV = P^T dO
//
// Two kernels, one over tiles of queries (S, dP and dQ: three products a block of 128 x 128), one over tiles of keys
// (S^T, dP^T, dV and dK: four). One kernel would do with five, but dQ is then added up by many blocks: in fp32
// in memory, in an order that changes its bits. Sums stay in TMEM, heads that share keys are summed by one block.
//
// 65536 tokens in sessions of 8192, 16 heads of 128 over 4, window 2048, bf16: 2460 us; delta 92 (the copy rate), over keys 1240
// (1.69 PFLOP/s of its four products, masked values too: 87 % of a library product's rate), over queries 942 (1.6), parts 24.
// Seven products for five: the floor of five is 1243 us. (Key by key: 785 ms; a block for each tile: 3000 us.)
//
// P and dS are operands in the rows' type: dS's rounding adds to dQ and dK about what the rounding of the results does (off by
// 2.5e-3 of their norm against 1.7e-3 in bf16, 3.2e-4 against 2.1e-4 in fp16; a second product for what it cuts off would be a
// third of dQ's time more). fp16 has five bits for exponents: P goes times 2^12, and dS times a power of two of the row's own,
// which its thread takes out of the sums again. It brings the largest |grad_out| that the row's sums hold to 16 .. 32: of the
// token itself for dQ, of the tokens that see the key for dK. So small gradients (and loss scales) keep their digits, whatever
// those of other sessions or of tokens out of sight are (with one factor for all, dQ of a session 2^-20 below another's was off by
// ten times its bound). A value that grows past fp16 all the same makes its row not finite, and such rows are computed
// again in fp32 by a kernel behind these (as are those that met an infinity or a NaN behind a mask).
#include "window_attention_tc.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "muon_internal.cuh"

namespace cbtbe {
namespace attention {
namespace {

constexpr int kWorkWarps = 8, kCopyWarp = 8, kMultiplyWarp = 9, kAheadWarp = 10, kThreads = 384;
constexpr int kStoreWarp = 11;  // over queries
constexpr int kStatWarp = 11;   // over keys
// Registers of the threads that work and of the others, of 384 x 168 at launch: what leaves either fewest spills (with
// shared memory taken, little of L1 is left, and a spilled register costs hundreds of clocks).
constexpr int kQueryMore = 208, kQueryFewer = 88, kKeyMore = 208, kKeyFewer = 88;

template <bool BF16> constexpr float kPShift = BF16 ? 0.f : 12.f;
// The power of two that brings values of this exponent (a byte of Backward::largest) to 16 .. 32.
__device__ __forceinline__ float slope_scale(uint32_t exponent) {
    return exponent ? __uint_as_float((127 + 4 + 127 - exponent) << 23) : 1.f;
}

// Behind the last token that sees key j, 0 for a token of no session.
__device__ __forceinline__ int seen_until(const Shape& S, int64_t j) {
    if (j >= S.tokens || S.end[j] <= j) return 0;
    return static_cast<int>(j - S.start[j] < S.sinks ? S.end[j] : min64(S.end[j], j + S.window));
}
// A tile of keys whose queries go far beyond their windows (a session's first keys are seen to its end) is
// taken in parts of so many blocks of queries, whose sums are joined by attention_parts_kernel: as many as a window
// reaches, and enough to pay for the sums' way through memory. That is 16 times the heads that share the keys where there are
// many tiles to fill the GPU with; with few the longest decides, and 16 altogether are enough. One session of 23100
// tokens: 1077 us in one piece, 149 in parts; 33 sessions of 27 to 2379 tokens x 8 heads over 2: 242 with the larger parts,
// 215 with the smaller.
// (part_blocks, on the host, decides it for a call: few tiles are fewer than 8 an SM.)
__device__ __forceinline__ int parts_of(int per, int blocks) {
    return blocks <= 2 * per ? 0 : (blocks + per - 1) / per;
}

constexpr int kDeltaThreads = 256;
// Which part of which tile has each place: the tiles in order, as far as there is room (so that the same tiles are
// taken in parts every time: their sums are added in another order than a whole tile's). By a block.
__device__ __forceinline__ void order_parts(const Backward& B) {
    __shared__ int of_warp[kDeltaThreads / 32];
    const Order& O = B.order;
    const int tiles = tiles_of(static_cast<int>(B.S.tokens)), warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    int before = 0;
    for (int first = 0; first < tiles; first += kDeltaThreads) {
        const int tile = first + static_cast<int>(threadIdx.x);
        const int parts = tile < tiles ? __ldcg(O.split + tile) : 0;
        int up_to = parts;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int other = __shfl_up_sync(kFull, up_to, off);
            if (lane >= off) up_to += other;
        }
        __syncthreads();
        if (lane == 31) of_warp[warp] = up_to;
        __syncthreads();
        int all = 0, place = before + up_to - parts;
        for (int w = 0; w < kDeltaThreads / 32; ++w) {
            if (w < warp) place += of_warp[w];
            all += of_warp[w];
        }
        if (parts && place + parts <= O.room) {
            for (int p = 0; p < parts; ++p) O.list[place + p] = make_int2(tile, p);
        } else if (parts) {  // in one piece; places that are left stay empty
            for (int p = place; p < O.room; ++p) O.list[p] = make_int2(-1, 0);
            O.split[tile] = 0;
        }
        before = min(before + all, 1 << 29);
    }
    if (threadIdx.x == 0) *O.parts = before;
}

// delta, and each row's largest |grad_out|: 16 bytes a lane, D / 8 lanes a row.
template <int D, bool BF16>
__global__ void __launch_bounds__(kDeltaThreads) attention_delta_kernel(const Backward B) {
    constexpr int DT = BF16 ? CB_BF16 : CB_F16, kLanes = D / 8, kRowsAtOnce = 32 / kLanes;
    begin_kernel();
    const Shape& S = B.S;
    const int lane = threadIdx.x & 31, c = lane % kLanes * 8;
    const int64_t rows = S.tokens * S.heads;
    for (int64_t i = warp_id_global() * kRowsAtOnce + lane / kLanes; i - lane / kLanes < rows; i += warps_in_grid() * kRowsAtOnce) {
        float a[8] = {}, b[8] = {}, sum = 0.f, largest = 0.f;
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
        if constexpr (!BF16) {
#pragma unroll
            for (int off = kLanes / 2; off >= 1; off >>= 1) largest = fmaxf(largest, __shfl_xor_sync(kFull, largest, off));
            if (i < rows && lane % kLanes == 0)
                B.largest[h * B.padded + t] = static_cast<uint8_t>(__float_as_uint(largest) >> 23);
        }
    }
    // In how many parts each tile of keys is to be taken, where some may be.
    const int tiles = B.order.room ? tiles_of(static_cast<int>(S.tokens)) : 0;
    for (int64_t w = warp_id_global(); w < tiles; w += warps_in_grid()) {
        const int from = static_cast<int>(w) * kTile;
        int until = 0;
#pragma unroll
        for (int k = 0; k < kTile / 32; ++k) until = max(until, seen_until(S, from + k * 32 + lane));
        until = __reduce_max_sync(kFull, until);
        if (lane == 0) B.order.split[w] = parts_of(B.order.part, tiles_of(max(until - from, 0)));
    }
    if (tiles == 0) return;
    __shared__ bool last;  // of the blocks: every tile's number of parts is there
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(B.order.done, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    order_parts(B);
}

// A row of sums from TMEM, times `by`, into its tile in shared memory; whether all are finite.
template <int D, bool BF16>
__device__ __forceinline__ bool finish_row(uint32_t at, float by, bool real, unsigned char* tile, int row) {
    const float2 by2 = make_float2(by, by), zero2 = make_float2(0.f, 0.f);
    float2 check = zero2;  // stays 0 while all is finite
#pragma unroll 1
    for (int d = 0; d < D; d += 32) {
        float o[32];
        tc::tmem_load32(at + d, o);
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
            uint32_t w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float2 x = real ? mul2(make_float2(o[k + 2 * u], o[k + 2 * u + 1]), by2) : zero2;
                check = fma2(x, zero2, check);
                w[u] = pack2<BF16>(x.x, x.y);
            }
            *reinterpret_cast<uint4*>(tile + tile_byte(row, (d + k) / 8)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    return check.x + check.y == 0.f;
}
template <int D>
__device__ __forceinline__ void zero_row(unsigned char* tile, int row) {
#pragma unroll
    for (int d = 0; d < D; d += 8) *reinterpret_cast<uint4*>(tile + tile_byte(row, d / 8)) = make_uint4(0, 0, 0, 0);
}

// ---------------------------------------------------------------- dQ

constexpr int kKeyBuffers = 2;  // of keys; one of values
template <int D> constexpr size_t kQueryShared = 1024 + (4 + kKeyBuffers + 1) * kRowsBytes<D>;

// As the forward, two tiles of queries a block, which stays and takes its share of the work. A tile's S, dP and dS take turns in
// the same columns of TMEM (P stays in the row's thread meanwhile), so that two tiles fit with their dQ: one's products run
// beside the other's exponentials. Keys are needed at both ends of a block (S, dQ), values in between (dP): two
// places for keys and one for values let both come a block ahead.
template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attention_dq_kernel(const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km,
                    const __grid_constant__ CUtensorMap vm, const __grid_constant__ CUtensorMap gm,
                    const __grid_constant__ CUtensorMap dqm, const __grid_constant__ Backward B, const bool pair_heads,
                    const int items) {
    constexpr uint32_t kRows = kRowsBytes<D>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* queries = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    unsigned char* grads_out = queries + 2 * kRows;  // dO, and dQ in its place
    unsigned char* keys = queries + 4 * kRows;
    unsigned char* values = keys + kKeyBuffers * kRows;
    __shared__ uint64_t q_full, q_empty, g_full[2], stored[2], k_full[2], k_empty[2], k_landed[2], v_full, v_empty, v_landed;
    __shared__ uint64_t scores[2], taken[2], grads[2], slopes[2][2], sums[2], staged[2], item_full[2], item_empty[2];
    __shared__ uint32_t tmem_at;
    __shared__ Item info[2];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (uint64_t* b : {&q_full, &q_empty, &v_full, &v_empty, &v_landed}) tc::barrier_init(tc::smem_addr(b), 1);
        for (int i = 0; i < 2; ++i) {
            for (uint64_t* b : {g_full, stored, k_full, k_empty, k_landed, scores, grads, sums, item_full})
                tc::barrier_init(tc::smem_addr(b + i), 1);
            for (uint64_t* b : {taken, slopes[0], slopes[1], staged}) tc::barrier_init(tc::smem_addr(b + i), 4);
            tc::barrier_init(tc::smem_addr(item_empty + i), kWorkWarps + 3);
        }
        tc::barrier_init_fence();
        for (const CUtensorMap* m : {&qm, &km, &vm, &gm, &dqm}) tc::tma_prefetch(m);
    }
    if (warp == kMultiplyWarp) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), 512);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int first = static_cast<int>(blockIdx.x), stride = static_cast<int>(gridDim.x);
    const int rounds = (items - first + stride - 1) / stride;
    bool ok = true;
    // One thread waits, or a whole warp.
    auto wait = [&](uint64_t* bar, uint32_t parity) { return ok = tc::barrier_wait(tc::smem_addr(bar), parity & 1); };
    auto meet = [&](uint64_t* bar, uint32_t parity) { return ok = warp_wait(bar, parity); };
    // The n-th item, for one thread; it is done with it at item_done.
    auto item_of = [&](int n) -> const Item& {
        wait(item_full + (n & 1), n >> 1);
        return info[n & 1];
    };
    auto item_done = [&](int n) { tc::barrier_arrive(tc::smem_addr(item_empty + (n & 1))); };

    if (warp >= kWorkWarps) {
        registers_down<kQueryFewer>();
        if (warp == kAheadWarp) {
            for (int n = 0; n < rounds; ++n) {
                const Work W = work_of(B.S, first + n * stride, pair_heads);
                if (!(ok = warp_wait(item_empty + (n & 1), (n >> 1) ^ 1))) break;
                Item& it = info[n & 1];
                if (lane == 0) it.W = W;
                look_ahead(B.S, it, 0, W.token[0], lane);
                look_ahead(B.S, it, 1, W.token[1], lane);
                warp_arrive(item_full + (n & 1));
            }
        } else if (warp == kStoreWarp) {
            uint32_t k_turns = 0, v_turns = 0;
            int begun = 0;  // blocks before the item's
            for (int n = 0; n < rounds && ok; ++n) {
                if (!meet(item_full + (n & 1), n >> 1)) break;
                const Work W = info[n & 1].W;
                const Blocks blocks(info[n & 1].sight[0], info[n & 1].sight[1]);
                warp_arrive(item_empty + (n & 1));
                auto clear = [&](int i, int count) {
                    const uint32_t b = static_cast<uint32_t>(begun + i) & 1;
                    return ok = clear_landed<D>(k_landed, k_full, b, k_turns, keys + b * kRows, count, lane) &&
                                clear_landed<D>(&v_landed, &v_full, 0, v_turns, values, count, lane);
                };
                if (!blocks.to_clear(0, blocks.count, clear)) break;
                begun += blocks.count;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!meet(staged + x, n)) break;
                    if (lane == 0) {
                        if (W.token[x] < B.S.tokens)
#pragma unroll
                            for (int d = 0; d < D / 64; ++d)
                                tma_store(&dqm, tc::smem_addr(grads_out) + x * kRows + d * kBoxBytes, d * 64, W.head[x], W.token[x]);
                        tma_store_done();
                    }
                    warp_arrive(stored + x);
                }
            }
        } else if (warp == kCopyWarp && tc::elect()) {
            int i_all = 0, n = 0, loaded_q = 0, loaded_g[2] = {0, 0}, loaded_k = 0, loaded_v = 0;
            int cleared_k[2] = {0, 0}, cleared_v = 0;  // tiles that land to be cleared
            bool last_k[2] = {false, false}, last_v = false;  // whether the last was one
            for (; n < rounds && ok; ++n) {
                const Item& it = item_of(n);
                if (!ok) break;
                const Work W = it.W;
                const Blocks blocks(it.sight[0], it.sight[1]);
                item_done(n);
                if (!wait(&q_empty, n ^ 1)) break;
                tc::barrier_expect(tc::smem_addr(&q_full), 2 * kRows);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    load_tile<D>(tc::smem_addr(queries) + x * kRows, &qm, tc::smem_addr(&q_full), W.head[x], W.token[x]);
                ++loaded_q;
                auto load_keys = [&](int i) {
                    const int b = (i_all + i) & 1;
                    if (!wait(k_empty + b, ((i_all + i) >> 1) ^ 1)) return;
                    const bool clear = blocks.counted(i) < kTile;
                    const uint32_t bar = tc::smem_addr((clear ? k_landed : k_full) + b);
                    tc::barrier_expect(bar, kRows);
                    load_tile<D>(tc::smem_addr(keys) + b * kRows, &km, bar, W.kv, blocks.at(i).at);
                    ++loaded_k;
                    cleared_k[b] += last_k[b] = clear;
                };
                if (blocks.count > 0) load_keys(0);
#pragma unroll
                for (int x = 0; x < 2 && ok; ++x) {  // the dQ before has left its place
                    if (!wait(stored + x, n ^ 1)) break;
                    tc::barrier_expect(tc::smem_addr(g_full + x), kRows);
                    load_tile<D>(tc::smem_addr(grads_out) + x * kRows, &gm, tc::smem_addr(g_full + x), W.head[x], W.token[x]);
                    ++loaded_g[x];
                }
                for (int i = 0; i < blocks.count && ok; ++i) {
                    if (!wait(&v_empty, (i_all + i) ^ 1)) break;
                    const bool clear = blocks.counted(i) < kTile;
                    const uint32_t bar = tc::smem_addr(clear ? &v_landed : &v_full);
                    tc::barrier_expect(bar, kRows);
                    load_tile<D>(tc::smem_addr(values), &vm, bar, W.kv, blocks.at(i).at);
                    ++loaded_v;
                    cleared_v += last_v = clear;
                    if (i + 1 < blocks.count) load_keys(i + 1);
                }
                i_all += blocks.count;
            }
            if (!ok) {  // copies in flight land before the block's shared memory goes away
                auto land = [&](uint64_t* bar, int parity) { tc::barrier_wait(tc::smem_addr(bar), parity & 1); };
                if (loaded_q) land(&q_full, loaded_q - 1);
                for (int x = 0; x < 2; ++x)
                    if (loaded_g[x]) land(g_full + x, loaded_g[x] - 1);
                if (loaded_v) last_v ? land(&v_landed, cleared_v - 1) : land(&v_full, loaded_v - 1);
                for (int k = max(0, loaded_k - 2); k < loaded_k; ++k)
                    last_k[k & 1] ? land(k_landed + (k & 1), cleared_k[k & 1] - 1) : land(k_full + (k & 1), k >> 1);
            }
        } else if (warp == kMultiplyWarp) {
            const bool one = tc::elect();
            constexpr uint32_t shape_s = mma_shape<BF16>(kTile, kTile, false), shape_q = mma_shape<BF16>(kTile, D, true);
            const uint64_t q0 = tc::operand_k_major(tc::smem_addr(queries)), g0 = tc::operand_k_major(tc::smem_addr(grads_out));
            const uint64_t k0 = tc::operand_k_major(tc::smem_addr(keys)), v0 = tc::operand_k_major(tc::smem_addr(values));
            const uint64_t turned0 = tc::operand_mn_major(tc::smem_addr(keys), kBoxBytes);
            int i_all = 0;
            uint32_t taken_turn[2] = {0, 0}, slopes_turn[2] = {0, 0};
            auto commit = [&](uint64_t* bar) {
                if (one) tc::mma_commit<1>(tc::smem_addr(bar));
                __syncwarp();
            };
            auto multiply = [&](int x, uint64_t a, uint64_t b, uint64_t* bar) {  // Q_x K^T or dO_x V^T
                a = tc::advance(a, x * kRows);
                if (one) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = k / 4 * kBoxBytes + k % 4 * 32;
                        tc::mma_f16<1>(tmem + x * 128, tc::advance(a, off), tc::advance(b, off), shape_s, k > 0);
                    }
                    tc::mma_commit<1>(tc::smem_addr(bar + x));
                }
                __syncwarp();
            };
            auto multiply_grads = [&](int x) {  // dP_x, once S_x has been read from its columns
                if (!meet(taken + x, taken_turn[x])) return false;
                taken_turn[x] ^= 1;
                tc::fence_after();
                multiply(x, g0, v0, grads);
                return true;
            };
            auto add_keys = [&](int x, int buffer, bool add) {  // dQ_x += dS_x K
                const uint64_t b = tc::advance(turned0, buffer * kRows);
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // half of the keys, then the other half
                    if (!meet(slopes[x] + h, slopes_turn[x])) return false;
                    tc::fence_after();
                    if (one)
#pragma unroll
                        for (int k = 4 * h; k < 4 * h + 4; ++k)
                            mma_tmem(tmem + 256 + x * D, tmem + x * 128 + k * 8, tc::advance(b, k * 2048), shape_q, add || k > 0);
                    __syncwarp();
                }
                slopes_turn[x] ^= 1;
                return true;
            };
            // In turns dQ of one tile, dP of the other, S of the first: each finds its operands ready while the one
            // before runs.
            for (int n = 0; n < rounds && ok; ++n) {
                if (!meet(item_full + (n & 1), n >> 1)) break;
                const Item& it = info[n & 1];
                const Blocks blocks(it.sight[0], it.sight[1]);
                warp_arrive(item_empty + (n & 1));
                if (!meet(&q_full, n)) break;
                bool begun[2] = {false, false}, use[2] = {false, false};
                if (blocks.count > 0) {
                    if (!meet(k_full + (i_all & 1), i_all >> 1)) break;
                    tc::fence_after();
                    const uint64_t key = tc::advance(k0, (i_all & 1) * kRows);
                    const Blocks::Block b = blocks.at(0);
                    use[0] = b.use[0];
                    use[1] = b.use[1];
                    if (use[0]) multiply(0, q0, key, scores);
                    if (!meet(g_full, n) || !meet(g_full + 1, n) || !meet(&v_full, i_all)) break;
                    if (use[0] && !multiply_grads(0)) break;
                    if (use[1]) multiply(1, q0, key, scores);
                } else if (!meet(g_full, n) || !meet(g_full + 1, n)) {
                    break;  // no phase is skipped: a later wait could take it for its own
                }
                if (blocks.count <= 1) commit(&q_empty);
                for (int i = 0; i < blocks.count; ++i, ++i_all) {
                    const bool more = i + 1 < blocks.count;
                    const Blocks::Block c = blocks.at(i + 1);
                    const int here = i_all & 1, there = here ^ 1;
                    const bool next0 = more && c.use[0], next1 = more && c.use[1];
                    if (use[0] && !add_keys(0, here, begun[0])) break;
                    begun[0] |= use[0];
                    if (use[1] && !multiply_grads(1)) break;
                    commit(&v_empty);
                    if (!more) commit(sums);
                    if (more && !meet(k_full + there, (i_all + 1) >> 1)) break;
                    const uint64_t key = tc::advance(k0, there * kRows);
                    if (next0) multiply(0, q0, key, scores);
                    if (use[1] && !add_keys(1, here, begun[1])) break;
                    begun[1] |= use[1];
                    commit(k_empty + here);
                    if (more) {
                        if (!meet(&v_full, i_all + 1)) break;
                        if (next0 && !multiply_grads(0)) break;
                        if (next1) multiply(1, q0, key, scores);
                        if (i + 2 == blocks.count) commit(&q_empty);  // the last scores
                    } else {
                        commit(sums + 1);
                    }
                    use[0] = next0;
                    use[1] = next1;
                }
            }
        }
    } else {
        registers_up<kQueryMore>();
        const int mine = warp >> 2, row = threadIdx.x & 127;
        const float c = B.S.scale * kLog2e;
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + mine * 128 + lanes, q_at = tmem + 256 + mine * D + lanes;
        const float2 c2 = make_float2(c, c);
        uint32_t phase = 0, sums_phase = 0;
        for (int n = 0; n < rounds; ++n) {
            if (!(ok = warp_wait(item_full + (n & 1), n >> 1))) break;
            const Item& it = info[n & 1];
            const int t = it.W.token[mine] + row, head = it.W.head[mine];
            const Row r = row_in(B.S, it, mine, row);
            float lse = 0.f, delta = 0.f, f = 1.f;
            if (r.real) {
                if constexpr (!BF16) f = slope_scale(B.largest[head * B.padded + t]);
                lse = -B.lse[head * B.S.tokens + t] * kLog2e;
                delta = -B.delta[head * B.S.tokens + t] * f;
            }
            const float2 lse2 = make_float2(lse, lse), delta2 = make_float2(delta, delta), f2 = make_float2(f, f);
            // What all of the warp's rows see whole.
            const int whole0 = __reduce_max_sync(kFull, r.real ? r.first : INT32_MAX);
            const int whole1 = __reduce_min_sync(kFull, r.real ? t + 1 : 0);
            const Sight& own = it.sight[mine];
            const Blocks blocks(it.sight[0], it.sight[1]);
            const int sink_blocks = tiles_of(own.s1 - own.s0), main0 = blocks.base + max(own.lo - blocks.base, 0) / kTile * kTile;
            const int count = sink_blocks + tiles_of(max(own.hi - main0, 0)), all_count = blocks.count;
            for (int i = 0; i < count; ++i) {
                const int at = i < sink_blocks ? own.s0 + i * kTile : main0 + (i - sink_blocks) * kTile;
                const bool whole = i >= sink_blocks && at >= whole0 && at + kTile <= whole1;
                if (!(ok = warp_wait(scores + mine, phase))) break;
                tc::fence_after();
                uint32_t p[2][64];
                tmem_load64(s_at, p[0]);
                tmem_load64(s_at + 64, p[1]);
                tc::fence_before();
                warp_arrive(taken + mine);
#pragma unroll
                for (int k = 0; k < 128; k += 2) {
                    uint32_t &lo = p[k / 64][k % 64], &hi = p[k / 64][k % 64 + 1];
                    const float2 x = fma2(make_float2(__uint_as_float(lo), __uint_as_float(hi)), c2, lse2);
                    lo = __float_as_uint(exp2_fast(x.x));
                    hi = __float_as_uint(exp2_fast(x.y));
                }
                if (!whole) {
                    const int from = i < sink_blocks ? own.s0 : own.lo, to = i < sink_blocks ? own.s1 : own.hi;
                    const TwoRanges sees{r.first, r.real ? t + 1 : 0, r.start,
                                         r.real ? static_cast<int>(min64(static_cast<int64_t>(r.start) + B.S.sinks, r.first)) : 0};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t bits = sees.bits(at + w * 32) & range_bits(from, to, at + w * 32);
                        if (__all_sync(kFull, bits == ~0u)) continue;
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (!(bits >> k & 1)) p[w / 2][w % 2 * 32 + k] = 0u;
                    }
                }
                if (!(ok = warp_wait(grads + mine, phase))) break;
                phase ^= 1;
                tc::fence_after();
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float d[32];
                    uint32_t packed[16];
                    tc::tmem_load32(s_at + w * 32, d);
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        const float2 x = fma2(make_float2(d[k], d[k + 1]), f2, delta2);
                        const uint32_t* weight = p[w / 2] + w % 2 * 32 + k;
                        const float2 y = mul2(x, make_float2(__uint_as_float(weight[0]), __uint_as_float(weight[1])));
                        packed[k / 2] = pack2<BF16>(y.x, y.y);
                    }
                    tmem_store16_begin(s_at + w * 16, packed);
                    if (w % 2 == 0) continue;
                    tmem_store_wait();
                    tc::fence_before();
                    warp_arrive(slopes[mine] + w / 2);
                }
            }
            if (!ok) break;
            if (all_count > 0) {
                if (!(ok = warp_wait(sums + mine, sums_phase))) break;
                sums_phase ^= 1;
            }
            if (!(ok = warp_wait(g_full + mine, n))) break;  // its place is dQ's now
            tc::fence_after();
            unsigned char* tile = grads_out + mine * kRows;
            bool finite = true;
            if (count > 0) finite = finish_row<D, BF16>(q_at, B.S.scale / f, r.real, tile, row);
            else zero_row<D>(tile, row);
            note_again(B.again, __ballot_sync(kFull, !finite), t & ~31, head, kDq);
            fence_to_tma();
            tc::fence_before();
            warp_arrive(staged + mine);
            warp_arrive(item_empty + (n & 1));
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

// A tile of keys and the queries that see one of them.
struct KeyItem {
    int first, kv;    // token, head
    int from, blocks; // of 128 queries, from token `from` on, for each head that shares the keys; -1: no more items
    int until;        // behind the last token that sees one of the keys
    int place;        // -1, or the part's in the list
    int last[kTile];  // behind the last token that sees the key, 0 for one of no session
    float slope[kTile];  // fp16: what the key's dS goes times
};

// The largest of neighbours among 128 bytes, at level k of 2^k of them from each on (as far as there are some); so of any
// interval in two readings. A warp builds it, four bytes a lane.
struct Largest {
    uint32_t level[8][kTile / 4];
    __device__ __forceinline__ void build(uint32_t four, int lane) {
        __syncwarp();
        level[0][lane] = four;
#pragma unroll
        for (int k = 0; k < 7; ++k) {
            const int words = max(1, (1 << k) / 4);
            uint32_t next = __shfl_down_sync(kFull, four, words);
            if (lane + words > 31) next = 0u;
            if (k < 2) next = __funnelshift_r(four, next, 8 << k);
            four = __vmaxu4(four, next);
            level[k + 1][lane] = four;
        }
        __syncwarp();
    }
    __device__ __forceinline__ uint32_t of(int from, int to) const {  // from < to
        const int k = 31 - __clz(to - from);
        const uint8_t* bytes = reinterpret_cast<const uint8_t*>(level[k]);
        return max(static_cast<uint32_t>(bytes[from]), static_cast<uint32_t>(bytes[to - (1 << k)]));
    }
};
// The exponent of the largest |grad_out| among the tokens of an item that see the key, in all heads that share it: of
// keys first + lane + 32 k, which tokens up to last[k] see. By the warp that looks ahead. Where all keys that go on see whole tiles
// these are read 512 bytes at a time, several on their way (a tile at a time one session of 4096 tokens x 8 heads over 1
// waited 30 us for the first of these, of 390), the tiles that some see in part by the table.
__device__ __forceinline__ void largest_seen(const Backward& B, Largest& table, int first, int kv, int from, int blocks,
                                             const int (&last)[kTile / 32], int lane, uint32_t (&largest)[kTile / 32]) {
    const uint8_t* bytes = B.largest + static_cast<int64_t>(kv) * B.S.group * B.padded;
    const int end = from + blocks * kTile;
#pragma unroll
    for (uint32_t& x : largest) x = 0u;
    for (int at = from; at < end;) {
        int least = end;  // what all keys that go on from here see
#pragma unroll
        for (int k = 0; k < kTile / 32; ++k) least = last[k] > at ? min(least, last[k]) : least;
        least = __reduce_min_sync(kFull, least);
        const int whole = at == first ? 0 : (least - at) / kTile * kTile;
        if (whole > 0) {
            uint32_t most = 0u;
            for (int begin = 0; begin < whole; begin += 2048)
#pragma unroll 4
                for (int h = 0; h < B.S.group; ++h) {
                    uint4 v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int place = begin + u * 512 + lane * 16;
                        v[u] = make_uint4(0u, 0u, 0u, 0u);
                        if (place < whole) v[u] = *reinterpret_cast<const uint4*>(bytes + h * B.padded + at + place);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        most = __vmaxu4(__vmaxu4(most, __vmaxu4(v[u].x, v[u].y)), __vmaxu4(v[u].z, v[u].w));
                }
            const uint32_t two = __vmaxu2(most & 0xff00ff, most >> 8 & 0xff00ff);
            most = __reduce_max_sync(kFull, max(two & 0xffff, two >> 16));
#pragma unroll
            for (int k = 0; k < kTile / 32; ++k)
                if (last[k] > at) largest[k] = max(largest[k], most);
            at += whole;
            continue;
        }
        uint32_t four = 0u;
#pragma unroll 4
        for (int h = 0; h < B.S.group; ++h)
            four = __vmaxu4(four, *reinterpret_cast<const uint32_t*>(bytes + h * B.padded + at + 4 * lane));
        table.build(four, lane);
#pragma unroll
        for (int k = 0; k < kTile / 32; ++k) {
            const int lo = max(first + k * 32 + lane - at, 0), hi = min(last[k] - at, kTile);
            if (lo < hi) largest[k] = max(largest[k], table.of(lo, hi));
        }
        at += kTile;
    }
}

// A block has 128 keys of a head and takes the queries that see one of them, 128 at a time, for every head that
// shares the keys. S^T and dP^T have a key a lane, so that P^T and dS^T are operands from TMEM as they are; a warp takes
// half of the queries of its 32 keys. The products of a block follow one another as their operands
// come: S, dP | dV, S' (while dS is worked out) | dK, dP' (while P' is). Blocks stay and take the next tile
// from a counter, those with the most queries first: a session's first keys are seen to its end.
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
    unsigned char* ring = keys + 2 * kRows;  // K and V, and dK and dV in their place
    __shared__ uint64_t kv_full, stored, staged[2], full[S], empty[S], landed[S], scores, weights, grads, slopes, done;
    __shared__ uint64_t stat_full[kStatStages], stat_empty[kStatStages], item_full[2], item_empty[2];
    __shared__ uint32_t tmem_at;
    __shared__ KeyItem info[2];
    __shared__ __align__(16) float stats[kStatStages][2][kTile];  // -lse log2 e (+ shift) and -delta
    __shared__ Largest table;
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (uint64_t* b : {&kv_full, &stored, &scores, &grads, &done}) tc::barrier_init(tc::smem_addr(b), 1);
        for (uint64_t* b : {&weights, &slopes}) tc::barrier_init(tc::smem_addr(b), kWorkWarps);
        for (int i = 0; i < S; ++i) {
            tc::barrier_init(tc::smem_addr(full + i), 1);
            tc::barrier_init(tc::smem_addr(empty + i), 1);
            tc::barrier_init(tc::smem_addr(landed + i), 1);
        }
        for (int i = 0; i < kStatStages; ++i) {
            tc::barrier_init(tc::smem_addr(stat_full + i), 1);
            tc::barrier_init(tc::smem_addr(stat_empty + i), kWorkWarps);
        }
        for (int i = 0; i < 2; ++i) {
            tc::barrier_init(tc::smem_addr(staged + i), 4);
            tc::barrier_init(tc::smem_addr(item_full + i), 1);
            tc::barrier_init(tc::smem_addr(item_empty + i), kWorkWarps + 4);
        }
        tc::barrier_init_fence();
        for (const CUtensorMap* m : {&qm, &km, &vm, &gm, &dkm, &dvm}) tc::tma_prefetch(m);
    }
    if (warp == kMultiplyWarp) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), 512);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    bool ok = true;
    // One thread waits, or a whole warp.
    auto wait = [&](uint64_t* bar, uint32_t parity) { return ok = tc::barrier_wait(tc::smem_addr(bar), parity & 1); };
    auto meet = [&](uint64_t* bar, uint32_t parity) { return ok = warp_wait(bar, parity); };

    if (warp >= kWorkWarps) {
        registers_down<kKeyFewer>();
        if (warp == kAheadWarp) {  // the next item, and the results of the one before
            const int kv_heads = B.S.kv_heads, tiles = tiles_of(static_cast<int>(B.S.tokens));
            const int64_t listed = B.order.room ? static_cast<int64_t>(min(*B.order.parts, B.order.room)) * kv_heads : 0;
            const int64_t all = listed + static_cast<int64_t>(tiles) * kv_heads;
            auto store = [&](int n) {  // of the n-th item
                const int first = info[n & 1].first, kv = info[n & 1].kv;
                if (!(ok = warp_wait(staged, n) && warp_wait(staged + 1, n))) return;
                if (lane == 0 && info[n & 1].place < 0) {
#pragma unroll
                    for (int x = 0; x < D / 64; ++x) {
                        tma_store(&dkm, tc::smem_addr(keys) + x * kBoxBytes, x * 64, kv, first);
                        tma_store(&dvm, tc::smem_addr(keys) + kRows + x * kBoxBytes, x * 64, kv, first);
                    }
                    tma_store_done();
                }
                __syncwarp();
                warp_arrive(&stored);
                warp_arrive(item_empty + (n & 1));
            };
            for (int n = 0;; ++n) {
                int first = 0, kv = 0, until = 0, part = 0, place = -1, last[kTile / 32];
                bool some = false;
                while (!some) {
                    unsigned w = 0;
                    if (lane == 0) w = atomicAdd(B.order.next, 1u);
                    w = __shfl_sync(kFull, w, 0);
                    if (w >= all) break;
                    const int64_t index = w < listed ? w : w - listed;
                    int tile = static_cast<int>(index / kv_heads);
                    kv = static_cast<int>(index % kv_heads);
                    place = -1;
                    if (w < listed) {
                        place = tile;
                        const int2 entry = B.order.list[place];
                        tile = entry.x;
                        part = entry.y;
                        some = tile >= 0;
                    } else {
                        some = !B.order.room || B.order.split[tile] == 0;
                    }
                    if (!some) continue;
                    first = tile * kTile;
                    until = 0;
#pragma unroll
                    for (int k = 0; k < kTile / 32; ++k) {
                        last[k] = seen_until(B.S, first + k * 32 + lane);
                        until = max(until, last[k]);
                    }
                    until = __reduce_max_sync(kFull, until);
                }
                const int blocks = tiles_of(max(until - first, 0)), per = B.order.part;
                const int from = place < 0 ? first : first + part * per * kTile;
                const int count = !some ? -1 : (place < 0 ? blocks : max(min(per, blocks - part * per), 0));
                uint32_t largest[kTile / 32];
                if constexpr (!BF16) largest_seen(B, table, first, kv, from, count, last, lane, largest);
                // The place of the item before the last one: its results are stored first.
                if (n >= 2) {
                    store(n - 2);
                    if (!ok) break;
                }
                if (!(ok = warp_wait(item_empty + (n & 1), (n >> 1) ^ 1))) break;
                KeyItem& it = info[n & 1];
                if (lane == 0) {
                    it.first = first;
                    it.kv = kv;
                    it.place = place;
                    it.from = from;
                    it.blocks = count;
                    it.until = until;
                }
                if (some)
#pragma unroll
                    for (int k = 0; k < kTile / 32; ++k) {
                        it.last[k * 32 + lane] = last[k];
                        if constexpr (!BF16) it.slope[k * 32 + lane] = slope_scale(largest[k]);
                    }
                warp_arrive(item_full + (n & 1));
                if (!some) {
                    if (n >= 1) store(n - 1);
                    break;
                }
            }
        } else if (warp == kCopyWarp && tc::elect()) {
            int s = 0, n = 0;
            uint32_t phase = 0, used = 0, cleared = 0, turns = 0;  // stages: in use; whose copies land to be cleared, their phases
            for (;; ++n) {
                if (!wait(item_full + (n & 1), n >> 1)) break;
                const KeyItem& it = info[n & 1];
                const int first = it.first, from = it.from, kv = it.kv, blocks = it.blocks, until = it.until;
                tc::barrier_arrive(tc::smem_addr(item_empty + (n & 1)));
                if (blocks < 0) break;
                int64_t m = 0;
                auto load = [&] {  // the next tile of the ring
                    if (!wait(empty + s, phase ^ 1)) return false;
                    const int b = static_cast<int>(m >> 1), h = b / blocks, i = b - h * blocks;
                    const bool clear = until - from - i * kTile < kTile;
                    const uint32_t bar = tc::smem_addr((clear ? landed : full) + s);
                    used |= 1u << s;
                    cleared = (cleared & ~(1u << s)) | (clear ? 1u << s : 0u);
                    turns ^= clear ? 1u << s : 0u;
                    tc::barrier_expect(bar, kRows);
                    load_tile<D>(tc::smem_addr(ring) + s * kRows, m & 1 ? &gm : &qm, bar, kv * B.S.group + h, from + i * kTile);
                    ++m;
                    if (++s == S) s = 0, phase ^= 1;
                    return true;
                };
                const int64_t all = 2 * static_cast<int64_t>(blocks) * B.S.group;
                // The first queries come while the results before leave the keys' place.
                while (m < 2 && m < all && load()) {}
                if (!ok || !wait(&stored, n ^ 1)) break;
                tc::barrier_expect(tc::smem_addr(&kv_full), 2 * kRows);
                load_tile<D>(tc::smem_addr(keys), &km, tc::smem_addr(&kv_full), kv, first);
                load_tile<D>(tc::smem_addr(keys) + kRows, &vm, tc::smem_addr(&kv_full), kv, first);
                while (m < all && load()) {}
                if (!ok) {
                    tc::barrier_wait(tc::smem_addr(&kv_full), n & 1);
                    break;
                }
            }
            if (!ok)  // copies in flight land before the block's shared memory goes away
                for (int i = 0; i < S; ++i)  // of the stages, those from s on are a round behind
                    if (used >> i & 1)
                        cleared >> i & 1 ? tc::barrier_wait(tc::smem_addr(landed + i), turns >> i & 1 ^ 1)
                                         : tc::barrier_wait(tc::smem_addr(full + i), phase ^ (i >= s));
        } else if (warp == kStatWarp) {
            int s = 0;
            uint32_t phase = 0, turns = 0, turn = 0;
            for (int n = 0; ok; ++n) {
                if (!(ok = warp_wait(item_full + (n & 1), n >> 1))) break;
                const int from = info[n & 1].from, kv = info[n & 1].kv, blocks = info[n & 1].blocks, until = info[n & 1].until;
                warp_arrive(item_empty + (n & 1));
                if (blocks < 0) break;
                for (int h = 0; h < B.S.group && ok; ++h) {
                    const int64_t row = static_cast<int64_t>(kv * B.S.group + h) * B.S.tokens;
                    for (int i = 0; i < blocks; ++i, ++turn) {
                        if (!(ok = warp_wait(stat_empty + s, phase ^ 1))) break;
#pragma unroll
                        for (int k = 0; k < kTile / 32; ++k) {
                            const int64_t t = from + static_cast<int64_t>(i) * kTile + k * 32 + lane;
                            stats[s][0][k * 32 + lane] = t < until ? kPShift<BF16> - B.lse[row + t] * kLog2e : 0.f;
                            stats[s][1][k * 32 + lane] = t < until ? -B.delta[row + t] : 0.f;
                        }
                        warp_arrive(stat_full + s);
                        if (++s == kStatStages) s = 0, phase ^= 1;
                        const int seeing = until - from - i * kTile;  // tokens of the block that see a key
                        if (seeing >= kTile) continue;
                        for (uint32_t m = 2 * turn; m < 2 * turn + 2 && ok; ++m)  // their queries, their gradients
                            ok = clear_landed<D>(landed, full, m % S, turns, ring + m % S * kRows, seeing, lane);
                        if (!ok) break;
                    }
                }
            }
        } else if (warp == kMultiplyWarp) {
            const bool one = tc::elect();
            constexpr uint32_t shape_s = mma_shape<BF16>(kTile, kTile, false), shape_d = mma_shape<BF16>(kTile, D, true);
            const uint64_t k0 = tc::operand_k_major(tc::smem_addr(keys)), q0 = tc::operand_k_major(tc::smem_addr(ring));
            const uint64_t turned0 = tc::operand_mn_major(tc::smem_addr(ring), kBoxBytes);
            auto commit = [&](uint64_t* bar) {
                if (one) tc::mma_commit<1>(tc::smem_addr(bar));
                __syncwarp();
            };
            auto multiply = [&](uint32_t left, int stage, uint32_t to, uint64_t* bar) {  // K Q^T or V dO^T
                const uint64_t a = tc::advance(k0, left * kRows), b = tc::advance(q0, stage * kRows);
                if (one) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = k / 4 * kBoxBytes + k % 4 * 32;
                        tc::mma_f16<1>(tmem + to, tc::advance(a, off), tc::advance(b, off), shape_s, k > 0);
                    }
                    tc::mma_commit<1>(tc::smem_addr(bar));
                }
                __syncwarp();
            };
            auto accumulate = [&](uint32_t from, int stage, uint32_t to, bool add) {  // P^T dO or dS^T Q
                const uint64_t b = tc::advance(turned0, stage * kRows);
                if (one)
#pragma unroll
                    for (int k = 0; k < kTile / 16; ++k)  // half of the queries in columns 0 .. 31, half in 64 .. 95
                        mma_tmem(tmem + to, tmem + from + k / 4 * 64 + k % 4 * 8, tc::advance(b, k * 2048), shape_d, add || k > 0);
                __syncwarp();
            };
            uint32_t turn = 0;  // blocks before: block `turn` has its Q in the ring's tile 2 turn, dO in 2 turn + 1
            auto tile_here = [&](uint32_t m) { return meet(full + m % S, m / S); };
            for (int n = 0; ok; ++n) {
                if (!meet(item_full + (n & 1), n >> 1)) break;
                const int blocks = info[n & 1].blocks;
                warp_arrive(item_empty + (n & 1));
                if (blocks < 0) break;
                const int64_t count = static_cast<int64_t>(blocks) * B.S.group;
                if (!meet(&kv_full, n)) break;
                if (count == 0) continue;
                if (!tile_here(2 * turn)) break;
                tc::fence_after();
                multiply(0, 2 * turn % S, 0, &scores);
                if (!tile_here(2 * turn + 1)) break;
                multiply(1, 2 * turn % S + 1, 128, &grads);
                for (int64_t i = 0; i < count; ++i, ++turn) {
                    const int q = static_cast<int>(2 * turn % S), g = q + 1, q_next = static_cast<int>((2 * turn + 2) % S);
                    const bool more = i + 1 < count;
                    if (!meet(&weights, turn)) break;
                    tc::fence_after();
                    accumulate(0, g, 256, i > 0);
                    commit(empty + g);
                    if (more) {
                        if (!tile_here(2 * turn + 2)) break;
                        multiply(0, q_next, 0, &scores);
                    }
                    if (!meet(&slopes, turn)) break;
                    tc::fence_after();
                    accumulate(128, q, 256 + D, i > 0);
                    commit(empty + q);
                    if (more) {
                        if (!tile_here(2 * turn + 3)) break;
                        multiply(1, q_next + 1, 128, &grads);
                    } else {
                        commit(&done);
                    }
                }
            }
        }
    } else {
        registers_up<kKeyMore>();
        const int row = threadIdx.x & 127, half = warp >> 2;
        const float c = B.S.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + lanes + half * 64, g_at = s_at + 128;
        int s = 0;
        uint32_t stat_phase = 0, turn = 0, items_with_blocks = 0;
        for (int n = 0;; ++n) {
            if (!(ok = warp_wait(item_full + (n & 1), n >> 1))) break;
            const KeyItem& it = info[n & 1];
            const int first = it.first, from = it.from, kv = it.kv, blocks = it.blocks, place = it.place;
            const int last = blocks < 0 ? 0 : it.last[row];
            const float scale_s = BF16 || blocks < 0 ? 1.f : it.slope[row], f = scale_s * exp2f(-kPShift<BF16>);
            const float2 f2 = make_float2(f, f);
            warp_arrive(item_empty + (n & 1));
            if (blocks < 0) break;
            const TwoRanges seen{first + row, last, 0, 0};
            // Queries that see all of the warp's keys.
            const int whole0 = first + (row | 31), whole1 = __reduce_min_sync(kFull, last);
            const int64_t count = static_cast<int64_t>(blocks) * B.S.group;
            int i = 0;
            for (int64_t b = 0; b < count; ++b, ++turn) {
                const int at = from + i * kTile + half * 64;
                if (++i == blocks) i = 0;
                if (!(ok = warp_wait(stat_full + s, stat_phase))) break;
                if (!(ok = warp_wait(&scores, turn))) break;
                tc::fence_after();
                uint32_t p[64], packed[32];
                tmem_load64(s_at, p);
                const float4* lse = reinterpret_cast<const float4*>(stats[s][0] + half * 64);
                const float4* delta = reinterpret_cast<const float4*>(stats[s][1] + half * 64);
#pragma unroll
                for (int k = 0; k < 64; k += 4) {
                    const float4 l = lse[k / 4];
                    const float2 s0 = make_float2(__uint_as_float(p[k]), __uint_as_float(p[k + 1]));
                    const float2 s1 = make_float2(__uint_as_float(p[k + 2]), __uint_as_float(p[k + 3]));
                    const float2 x = fma2(s0, c2, make_float2(l.x, l.y)), y = fma2(s1, c2, make_float2(l.z, l.w));
                    p[k] = __float_as_uint(exp2_fast(x.x));
                    p[k + 1] = __float_as_uint(exp2_fast(x.y));
                    p[k + 2] = __float_as_uint(exp2_fast(y.x));
                    p[k + 3] = __float_as_uint(exp2_fast(y.y));
                }
                if (at < whole0 || at + 64 > whole1) {
                    const uint32_t bits[2] = {seen.bits(at), seen.bits(at + 32)};
#pragma unroll
                    for (int k = 0; k < 64; ++k)
                        if (!(bits[k / 32] >> k % 32 & 1)) p[k] = 0u;
                }
#pragma unroll
                for (int k = 0; k < 64; k += 2) packed[k / 2] = pack2<BF16>(__uint_as_float(p[k]), __uint_as_float(p[k + 1]));
                tmem_store32_begin(s_at, packed);
                tmem_store_wait();
                tc::fence_before();
                warp_arrive(&weights);
                if (!(ok = warp_wait(&grads, turn))) break;
                tc::fence_after();
                uint32_t d[64];
                tmem_load64(g_at, d);
#pragma unroll
                for (int k = 0; k < 64; k += 4) {
                    const float4 l = delta[k / 4];
                    float2 x = add2(make_float2(__uint_as_float(d[k]), __uint_as_float(d[k + 1])), make_float2(l.x, l.y));
                    float2 y = add2(make_float2(__uint_as_float(d[k + 2]), __uint_as_float(d[k + 3])), make_float2(l.z, l.w));
                    if constexpr (!BF16) {
                        x = mul2(x, f2);
                        y = mul2(y, f2);
                    }
                    x = mul2(x, make_float2(__uint_as_float(p[k]), __uint_as_float(p[k + 1])));
                    y = mul2(y, make_float2(__uint_as_float(p[k + 2]), __uint_as_float(p[k + 3])));
                    packed[k / 2] = pack2<BF16>(x.x, x.y);
                    packed[k / 2 + 1] = pack2<BF16>(y.x, y.y);
                }
                tmem_store32_begin(g_at, packed);
                tmem_store_wait();
                tc::fence_before();
                warp_arrive(&slopes);
                warp_arrive(stat_empty + s);
                if (++s == kStatStages) s = 0, stat_phase ^= 1;
            }
            if (!ok) break;
            // The first four warps finish dV, the others dK, in the place of V and K.
            if (count > 0) {
                if (!(ok = warp_wait(&done, items_with_blocks))) break;
                ++items_with_blocks;
            }
            if (!(ok = warp_wait(&kv_full, n))) break;
            tc::fence_after();
            unsigned char* tile = keys + (half ? 0 : kRows);
            if (place >= 0) {  // sums in fp32, of dK without its scale of dS, joined by another kernel
                const float by = half ? 1.f / scale_s : 1.f;
                float* to = B.order.sums + ((static_cast<int64_t>(place) * B.S.kv_heads + kv) * 2 + half) * kTile * D + row * D;
#pragma unroll 1
                for (int d = 0; d < D; d += 32) {
                    float o[32] = {};
                    if (count > 0) tc::tmem_load32(tmem + lanes + 256 + half * D + d, o);
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<float4*>(to + d + k) = make_float4(o[k] * by, o[k + 1] * by, o[k + 2] * by, o[k + 3] * by);
                }
                tc::fence_before();
                warp_arrive(staged + half);
                continue;
            }
            bool finite = true;
            const float by = half ? B.S.scale / scale_s : exp2f(-kPShift<BF16>);
            if (count > 0) finite = finish_row<D, BF16>(tmem + lanes + 256 + half * D, by, last > 0, tile, row);
            else zero_row<D>(tile, row);
            note_again(B.again, __ballot_sync(kFull, !finite), first + (row & ~31), kv, half ? kDk : kDv);
            fence_to_tma();
            tc::fence_before();
            warp_arrive(staged + half);
        }
    }
    if (!ok && B.S.error) set_error(B.S.error, CB_ERR_TIMEOUT);
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    if (warp == kMultiplyWarp) tc::tmem_free<1>(tmem, 512);
}

// The sums of a tile's parts, in order: a block for 32 rows of a tile and head, a warp for four of them, as many parts on their
// way at once (33 sessions of 27 to 2379 tokens x 8 heads of 72 over 2: 22 us; of 128 rows a block 53).
template <int D, bool BF16>
__global__ void __launch_bounds__(256) attention_parts_kernel(const Backward B) {
    constexpr int DT = BF16 ? CB_BF16 : CB_F16, N = D / 32, kRowsAtOnce = 32, kGroups = kTile / kRowsAtOnce;
    __shared__ uint32_t again;  // of the block's rows
    if (threadIdx.x == 0) again = 0u;
    begin_kernel();
    const int listed = min(*B.order.parts, B.order.room), lane = threadIdx.x & 31;
    const float by[2] = {exp2f(-kPShift<BF16>), B.S.scale};
    for (int64_t w = blockIdx.x; w < static_cast<int64_t>(listed) * B.S.kv_heads * kGroups; w += gridDim.x) {
        const int64_t head = w / kGroups;
        const int place = static_cast<int>(head / B.S.kv_heads), kv = static_cast<int>(head % B.S.kv_heads);
        const int2 entry = B.order.list[place];
        if (entry.x < 0 || entry.y != 0) continue;
        const int parts = B.order.split[entry.x], first = static_cast<int>(w % kGroups) * kRowsAtOnce;  // of the tile's rows
        __syncthreads();
        for (int row = first + static_cast<int>(threadIdx.x) / 32; row < first + kRowsAtOnce; row += 8) {
            const int64_t j = static_cast<int64_t>(entry.x) * kTile + row;
            if (j >= B.S.tokens) break;
            const bool real = B.S.end[j] > j;
            float v[2][kLaneValues] = {};
            bool finite = true;
#pragma unroll 4
            for (int p = 0; p < (real ? parts : 0); ++p)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t at = ((static_cast<int64_t>(place) + p) * B.S.kv_heads + kv) * 2 + h;
                    const float* from = B.order.sums + at * kTile * D + row * D;
#pragma unroll
                    for (int i = 0; i < N; ++i) v[h][i] += __ldcg(from + lane + 32 * i);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    v[h][i] *= by[h];
                    finite &= fabsf(v[h][i]) < INFINITY || lane + 32 * i >= B.S.dim;
                }
            if (!__all_sync(kFull, finite) && lane == 0) atomicOr(&again, 1u << (row - first));
            store_row<DT>(B.dv, j, kv, B.S.dim, v[0]);
            store_row<DT>(B.dk, j, kv, B.S.dim, v[1]);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            note_again(B.again, again, static_cast<int64_t>(entry.x) * kTile + first, kv, kDkAndDv);
            again = 0u;
        }
    }
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
    if (items > INT32_MAX / 2 || key_tiles > INT32_MAX / 4) return false;
    launch(attention_delta_kernel<D, BF16>, dim3(warp_grid((S.tokens * S.heads * D / 8 + 31) / 32, 8 * sm_count())),
           dim3(kDeltaThreads), 0, s, B);
    launch(attention_dkv_kernel<D, BF16>, dim3(static_cast<unsigned>(std::min<int64_t>(key_tiles, sm_count()))), dim3(kThreads),
           kKeyShared<D>, s, qm, km, vm, gm, dkm, dvm, B);
    const int64_t joined = std::min<int64_t>(static_cast<int64_t>(B.order.room) * S.kv_heads * 4, 8 * sm_count());
    if (joined > 0) launch(attention_parts_kernel<D, BF16>, dim3(static_cast<unsigned>(joined)), dim3(256), 0, s, B);
    launch(attention_dq_kernel<D, BF16>, dim3(static_cast<unsigned>(std::min<int64_t>(items, sm_count()))), dim3(kThreads),
           kQueryShared<D>, s, qm, km, vm, gm, dqm, B, pairs_heads(S), static_cast<int>(items));
    launch_again(B, s);
    return true;
}

}  // namespace

int32_t part_blocks(int64_t tokens, int32_t heads, int32_t kv_heads, int64_t window) {
    const int64_t tiles = (tokens + kTile - 1) / kTile, group = std::max(1, heads / kv_heads);
    const int64_t least = tiles * kv_heads < 8 * sm_count() ? (16 + group - 1) / group : 16;
    return static_cast<int32_t>(std::max(least, std::min(window, int64_t{1} << 30) / kTile + 2));
}
int64_t parts_room(int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim, int64_t window, int64_t sinks) {
    const int64_t tiles = (tokens + kTile - 1) / kTile;
    const int64_t per = part_blocks(tokens, heads, kv_heads, window);
    if (sinks == 0 || dim > 128 || tiles <= 2 * per) return 0;
    // A session's first keys lie in at most so many tiles, each seen by its blocks, two per - 1 of them or more a part.
    const int64_t most = (std::min(sinks, tokens) / kTile + 2) * ((tiles + per - 1) / per * 2);
    const int64_t bytes = static_cast<int64_t>(kv_heads) * 2 * kTile * (dim <= 64 ? 64 : 128) * 4;
    return std::min(most, std::max<int64_t>((int64_t{256} << 20) / bytes, 1));
}
int64_t parts_bytes(int64_t room, int32_t kv_heads, int32_t dim) {
    return room * kv_heads * 2 * kTile * (dim <= 64 ? 64 : 128) * 4;
}

bool launch_backward(const Backward& B, cudaStream_t s) {
    if (B.S.dtype == CB_BF16) return B.S.dim <= 64 ? launch_typed<64, true>(B, s) : launch_typed<128, true>(B, s);
    return B.S.dim <= 64 ? launch_typed<64, false>(B, s) : launch_typed<128, false>(B, s);
}

}  // namespace attention
}  // namespace cbtbe
