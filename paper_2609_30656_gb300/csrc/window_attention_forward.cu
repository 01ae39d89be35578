// window_attention_forward.cu -- windowed attention over packed sessions by the tensor cores.
//
// A block takes two tiles of 128 queries that read the same key and value heads (the same tokens of two heads
// that share them, else 256 tokens of one head) through their keys, 128 at a time, with one pass
// softmax: S = Q K^T into TMEM, P = exp(S - m) back into TMEM over it, O += P V from there. One warp copies, one
// issues the products, four for each tile have a row a thread (no shuffles: a lane reads its row of S from TMEM).
// O stays in TMEM. The products of the two tiles take turns, so that while one's warps are at their exponentials the other's
// run (with a warp to issue for each tile both fell into step, and the tensor cores waited for both).
//
// m need not be the maximum, only near enough for P's type: a row keeps the m of its first keys until the maximum has
// risen too far (2^8 for fp16, 2^60 for bf16); then the row's own thread scales its sums down. P goes to the tensor
// cores a half at a time, while the next is worked out.
//
// Blocks stay, one an SM, and take their share of the work: while a pair of tiles is finished, the queries and first keys of
// the next are on their way, by a warp that looks ahead at what they see, one that copies, and one that stores (and clears the
// values that no row sees).
//
// 65536 tokens in sessions of 8192, 16 heads of 128 over 4, window 2048, bf16: 740 us, 1.30 PFLOP/s (67 % of a library
// product's rate; a key by key kernel took 247 ms). What bounds it: the products wait for the exponentials of a tile and
// these for the products; Q, K and V are read from shared memory at 77 % of what it gives while products run. One block for
// each pair of tiles took 879 us, one warp to issue for each tile 241 against 207 us at 16384 tokens, O written to global
// memory by its threads 3900 clocks a tile. Small heads are bound by the exponentials (16 a clock and SM): 16384 tokens x 8
// heads of 64, window 512: 49 us where heads share keys in fours and 51 where none does. Sessions of 60 tokens (30000 tokens x
// 4 heads of 32, window 50) take 32 us: 3 blocks of keys a pair of tiles, whose latencies nothing hides.
#include "window_attention_tc.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

#include "muon_internal.cuh"

namespace cbtbe {
namespace attention {
namespace {

constexpr int kSoftmaxWarps = 8, kCopyWarp = 8, kMultiplyWarp = 9, kAheadWarp = 10, kStoreWarp = 11, kThreads = 384;
template <int D> constexpr int kStages = D == 64 ? 4 : 2;  // of the values of a block and the keys of the next
template <int D> constexpr size_t kShared = 1024 + (3 + 2 * kStages<D>) * kRowsBytes<D>;  // queries, those, output
// Of the 168 registers that a thread is launched with, the other warps give some to the softmax warps, whose
// threads hold a row of 128 scores: 256 x 216 + 128 x 72 of the block's 384 x 168.
constexpr int kMoreRegisters = 216, kFewerRegisters = 72;
// How far, in powers of two, weights may lie above 1. A bf16 has fp32's range, and n of them their sums'; fp16 holds
// weights times 2^6, so that small ones keep their digits, up to 2^14.
constexpr int kParts = 2;  // in which P goes to the tensor cores
template <bool BF16> constexpr float kRise = BF16 ? 60.f : 8.f;
template <bool BF16> constexpr float kShift = BF16 ? 0.f : 6.f;

// Weights 2^(s c + base) of 32 scores, packed, and their sums.
template <bool BF16, int FROM>
__device__ __forceinline__ void weigh(const uint32_t (&v)[64], float c, float base, uint32_t (&p)[16], float2& sum0, float2& sum1) {
    const float2 c2 = make_float2(c, c), base2 = make_float2(base, base);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        float2 x = fma2(make_float2(__uint_as_float(v[FROM + 2 * k]), __uint_as_float(v[FROM + 2 * k + 1])), c2, base2);
        x.x = exp2_fast(x.x);
        x.y = exp2_fast(x.y);
        if (k & 1) sum1 = add2(sum1, x);
        else sum0 = add2(sum0, x);
        p[k] = pack2<BF16>(x.x, x.y);
    }
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attention_forward_kernel(const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km,
                         const __grid_constant__ CUtensorMap vm, const __grid_constant__ CUtensorMap om,
                         const __grid_constant__ Forward F, const bool pair_heads, const int items) {
    constexpr int S = kStages<D>;
    constexpr uint32_t kRows = kRowsBytes<D>;
    extern __shared__ unsigned char dynamic[];
    unsigned char* queries = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    unsigned char* ring = queries + 2 * kRows;
    unsigned char* output = ring + 2 * S * kRows;  // of one tile after the other
    __shared__ uint64_t q_full, q_empty, full[S], empty[S], landed[S], scores[2], part[2][kParts], sums[2], staged[2], stored[2];
    __shared__ uint64_t item_full[2], item_empty[2];
    __shared__ uint32_t tmem_at;
    __shared__ Item info[2];
    const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        tc::barrier_init(tc::smem_addr(&q_full), 1);
        tc::barrier_init(tc::smem_addr(&q_empty), 1);
        for (int i = 0; i < 2; ++i) {
            tc::barrier_init(tc::smem_addr(scores + i), 1);
            for (int k = 0; k < kParts; ++k) tc::barrier_init(tc::smem_addr(part[i] + k), 4);
            tc::barrier_init(tc::smem_addr(sums + i), 1);
            tc::barrier_init(tc::smem_addr(staged + i), 4);
            tc::barrier_init(tc::smem_addr(stored + i), 1);
            tc::barrier_init(tc::smem_addr(item_full + i), 1);
            tc::barrier_init(tc::smem_addr(item_empty + i), kSoftmaxWarps + 3);
        }
        for (int i = 0; i < S; ++i) {
            tc::barrier_init(tc::smem_addr(full + i), 1);
            tc::barrier_init(tc::smem_addr(empty + i), 1);
            tc::barrier_init(tc::smem_addr(landed + i), 1);
        }
        tc::barrier_init_fence();
        for (const CUtensorMap* m : {&qm, &km, &vm, &om}) tc::tma_prefetch(m);
    }
    if (warp == kMultiplyWarp) tc::tmem_alloc<1>(tc::smem_addr(&tmem_at), 512);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = tmem_at;
    begin_kernel();
    const int first = static_cast<int>(blockIdx.x), stride = static_cast<int>(gridDim.x);
    bool ok = true;
    // The n-th item, for one thread; it is done with it at item_done.
    auto item_of = [&](int n) -> const Item& {
        ok = tc::barrier_wait(tc::smem_addr(item_full + (n & 1)), n >> 1 & 1);
        return info[n & 1];
    };
    auto item_done = [&](int n) { tc::barrier_arrive(tc::smem_addr(item_empty + (n & 1))); };
    const int rounds = (items - first + stride - 1) / stride;

    if (warp >= kSoftmaxWarps) {
        registers_down<kFewerRegisters>();
        if (warp == kAheadWarp) {
            for (int n = 0; n < rounds; ++n) {
                const Work W = work_of(F.S, first + n * stride, pair_heads);
                if (!(ok = warp_wait(item_empty + (n & 1), (n >> 1) ^ 1))) break;
                Item& it = info[n & 1];
                if (lane == 0) it.W = W;
                look_ahead(F.S, it, 0, W.token[0], lane);
                look_ahead(F.S, it, 1, W.token[1], lane);
                warp_arrive(item_full + (n & 1));
            }
        } else if (warp == kStoreWarp) {
            uint32_t turns = 0;
            int begun = 0;  // stages before the item's
            for (int n = 0; n < rounds && ok; ++n) {
                if (!(ok = warp_wait(item_full + (n & 1), n >> 1))) break;
                const Work W = info[n & 1].W;
                const Blocks blocks(info[n & 1].sight[0], info[n & 1].sight[1]);
                warp_arrive(item_empty + (n & 1));
                auto clear = [&](int i, int keys) {  // of the values of block i, which come in the stage behind the first keys'
                    const uint32_t s = static_cast<uint32_t>(begun + 1 + i) % S;
                    return ok = clear_landed<D>(landed, full, s, turns, ring + s * 2 * kRows, keys, lane);
                };
                if (!blocks.to_clear(0, blocks.count, clear)) break;
                begun += blocks.count ? blocks.count + 1 : 0;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!(ok = warp_wait(staged + x, n))) break;
                    if (lane == 0) {
                        if (W.token[x] < F.S.tokens)
#pragma unroll
                            for (int d = 0; d < D / 64; ++d)
                                tma_store(&om, tc::smem_addr(output) + d * kBoxBytes, d * 64, W.head[x], W.token[x]);
                        tma_store_done();
                    }
                    warp_arrive(stored + x);
                }
            }
        } else if (warp == kCopyWarp && tc::elect()) {
            int s = 0;
            uint32_t phase = 0, used = 0, cleared = 0, turns = 0;  // stages: in use; whose copies land to be cleared, their phases
            int queries_issued = 0;
            for (int n = 0; n < rounds && ok; ++n) {
                const Item& it = item_of(n);
                if (!ok) break;
                const Work W = it.W;
                const Blocks blocks(it.sight[0], it.sight[1]);
                item_done(n);
                if (!(ok = tc::barrier_wait(tc::smem_addr(&q_empty), (n & 1) ^ 1))) break;
                tc::barrier_expect(tc::smem_addr(&q_full), 2 * kRows);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    load_tile<D>(tc::smem_addr(queries) + x * kRows, &qm, tc::smem_addr(&q_full), W.head[x], W.token[x]);
                ++queries_issued;
                // The first keys come alone, then values and the next block's keys together, in a stage.
                for (int i = -1; i < blocks.count; ++i) {
                    if (i < 0 && blocks.count == 0) continue;
                    if (!(ok = tc::barrier_wait(tc::smem_addr(empty + s), phase ^ 1))) break;
                    const bool clear = i >= 0 && blocks.counted(i) < kTile, keys = i + 1 < blocks.count;
                    const uint32_t bar = tc::smem_addr((clear ? landed : full) + s), at = tc::smem_addr(ring) + s * 2 * kRows;
                    used |= 1u << s;
                    cleared = (cleared & ~(1u << s)) | (clear ? 1u << s : 0u);
                    turns ^= clear ? 1u << s : 0u;
                    tc::barrier_expect(bar, i >= 0 && keys ? 2 * kRows : kRows);
                    if (i >= 0) load_tile<D>(at, &vm, bar, W.kv, blocks.at(i).at);
                    if (keys) load_tile<D>(at + kRows, &km, bar, W.kv, blocks.at(i + 1).at);
                    if (++s == S) s = 0, phase ^= 1;
                }
            }
            if (!ok) {  // copies in flight land before the block's shared memory goes away
                for (int i = 0; i < S; ++i)  // of the stages, those from s on are a round behind
                    if (used >> i & 1)
                        cleared >> i & 1 ? tc::barrier_wait(tc::smem_addr(landed + i), turns >> i & 1 ^ 1)
                                         : tc::barrier_wait(tc::smem_addr(full + i), phase ^ (i >= s));
                if (queries_issued) tc::barrier_wait(tc::smem_addr(&q_full), (queries_issued - 1) & 1);
            }
        } else if (warp == kMultiplyWarp) {
            const bool one = tc::elect();
            constexpr uint32_t shape_s = mma_shape<BF16>(kTile, kTile, false), shape_o = mma_shape<BF16>(kTile, D, true);
            const uint64_t q0 = tc::operand_k_major(tc::smem_addr(queries));
            const uint64_t k0 = tc::operand_k_major(tc::smem_addr(ring) + kRows);
            const uint64_t v0 = tc::operand_mn_major(tc::smem_addr(ring), kBoxBytes);
            int s = 0;  // stage of the next copies
            uint32_t phase = 0, p_phase[2] = {0, 0};
            auto commit = [&](uint64_t* bar) {
                if (one) tc::mma_commit<1>(tc::smem_addr(bar));
                __syncwarp();
            };
            auto multiply_scores = [&](int x, uint32_t stage) {  // S_x = Q_x K^T
                const uint64_t a = tc::advance(q0, x * kRows), b = tc::advance(k0, stage * 2 * kRows);
                if (one) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = k / 4 * kBoxBytes + k % 4 * 32;
                        tc::mma_f16<1>(tmem + x * 128, tc::advance(a, off), tc::advance(b, off), shape_s, k > 0);
                    }
                    tc::mma_commit<1>(tc::smem_addr(scores + x));
                }
                __syncwarp();
            };
            for (int n = 0; n < rounds && ok; ++n) {
                if (!(ok = warp_wait(item_full + (n & 1), n >> 1))) break;
                const Item& it = info[n & 1];
                const Blocks blocks(it.sight[0], it.sight[1]);
                warp_arrive(item_empty + (n & 1));
                if (!(ok = warp_wait(&q_full, n))) break;
                bool begun[2] = {false, false}, use[2] = {false, false};
                if (blocks.count > 0) {
                    if (!(ok = warp_wait(full + s, phase))) break;
                    tc::fence_after();
                    const Blocks::Block b = blocks.at(0);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        use[x] = b.use[x];
                        if (use[x]) multiply_scores(x, s);
                    }
                    commit(empty + s);
                    if (++s == S) s = 0, phase ^= 1;
                    if (!(ok = warp_wait(full + s, phase))) break;
                }
                if (blocks.count <= 1) commit(&q_empty);
                // Only a few products are queued: what can be found out ahead is, while there are some.
                bool next0 = blocks.count > 1 && blocks.at(1).use[0], next1 = blocks.count > 1 && blocks.at(1).use[1];
                for (int i = 0; i < blocks.count; ++i) {
                    const bool more = i + 1 < blocks.count;
                    const int stage = s;
                    const uint64_t v = tc::advance(v0, stage * 2 * kRows);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (use[x]) {
#pragma unroll
                            for (int h = 0; h < kParts; ++h) {
                                if (!(ok = warp_wait(part[x] + h, p_phase[x]))) break;
                                tc::fence_after();
                                if (one)
#pragma unroll
                                    for (int k = 8 / kParts * h; k < 8 / kParts * (h + 1); ++k)
                                        mma_tmem(tmem + 256 + x * D, tmem + x * 128 + k * 8, tc::advance(v, k * 2048), shape_o,
                                                 begun[x] || k > 0);
                                __syncwarp();
                            }
                            if (!ok) break;
                            p_phase[x] ^= 1;
                            begun[x] = true;
                        }
                        use[x] = x ? next1 : next0;
                        if (use[x]) multiply_scores(x, stage);
                        if (!more) commit(sums + x);
                        if (x == 0) {
                            if (++s == S) s = 0, phase ^= 1;
                            if (more && !(ok = warp_wait(full + s, phase))) break;
                            next0 = i + 2 < blocks.count;
                        }
                    }
                    if (!ok) break;
                    commit(empty + stage);
                    if (i + 2 == blocks.count) commit(&q_empty);  // the last scores
                    if (next0) {
                        const Blocks::Block b = blocks.at(i + 2);
                        next0 = b.use[0];
                        next1 = b.use[1];
                    } else {
                        next1 = false;
                    }
                }
            }
        }
    } else {
        registers_up<kMoreRegisters>();
        const int mine = warp >> 2, row = threadIdx.x & 127;
        // exponentials: x = s c - m c in powers of two, c > 0 (the sign of the scale goes to s)
        const float c = fmaxf(fabsf(F.S.scale) * kLog2e, 1e-30f);
        const uint32_t flip = F.S.scale < 0.f ? 0x80000000u : 0u;
        const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + mine * 128 + lanes, o_at = tmem + 256 + mine * D + lanes;
        uint32_t phase = 0, sums_phase = 0;
        for (int n = 0; n < rounds; ++n) {
            if (!(ok = warp_wait(item_full + (n & 1), n >> 1))) break;
            const Item& it = info[n & 1];
            const int t = it.W.token[mine] + row, head = it.W.head[mine];
            const Row r = row_in(F.S, it, mine, row);
            // What all of the warp's rows see whole.
            const int whole0 = __reduce_max_sync(kFull, r.real ? r.first : INT32_MAX);
            const int whole1 = __reduce_min_sync(kFull, r.real ? t + 1 : 0);
            const Sight& own = it.sight[mine];
            // This tile's own blocks: its session's first tokens, and the common row of blocks from the first that it sees on.
            const int base = Blocks(it.sight[0], it.sight[1]).base;
            const int sink_blocks = tiles_of(own.s1 - own.s0), main0 = base + max(own.lo - base, 0) / kTile * kTile;
            const int count = sink_blocks + tiles_of(max(own.hi - main0, 0));
            const int it_blocks = Blocks(it.sight[0], it.sight[1]).count;
            float most = -INFINITY;  // what the exponents are taken against, a raw score
            float2 sum0 = make_float2(0.f, 0.f), sum1 = make_float2(0.f, 0.f);
            for (int i = 0; i < count; ++i) {
                const int at = i < sink_blocks ? own.s0 + i * kTile : main0 + (i - sink_blocks) * kTile;
                if (!(ok = warp_wait(scores + mine, phase))) break;
                phase ^= 1;
                tc::fence_after();
                uint32_t v[2][64], p[16];
                tmem_load64(s_at, v[0]);
                tmem_load64(s_at + 64, v[1]);
                if (flip)
#pragma unroll
                    for (int k = 0; k < 128; ++k) v[k / 64][k % 64] ^= flip;
                if (i < sink_blocks || at < whole0 || at + kTile > whole1) {
                    const int from = i < sink_blocks ? own.s0 : own.lo, to = i < sink_blocks ? own.s1 : own.hi;
                    const TwoRanges sees{r.first, r.real ? t + 1 : 0, r.start,
                                         r.real ? static_cast<int>(min64(static_cast<int64_t>(r.start) + F.S.sinks, r.first)) : 0};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t bits = sees.bits(at + w * 32) & range_bits(from, to, at + w * 32);
                        if (__all_sync(kFull, bits == ~0u)) continue;
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (!(bits >> k & 1)) v[w / 2][w % 2 * 32 + k] = 0xff800000u;
                    }
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 128; k += 8)
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const uint32_t* two = v[k / 64] + k % 64 + 2 * u;
                        top[u] = max3(top[u], __uint_as_float(two[0]), __uint_as_float(two[1]));
                    }
                const float highest = max3(fmaxf(top[0], top[1]), top[2], top[3]);
                if (__any_sync(kFull, (highest - most) * c > kRise<BF16>)) {  // false for two infinities
                    const float raised = fmaxf(most, highest);
                    const float keep = raised == most ? 1.f : exp2_fast((most - raised) * c);
                    most = raised;
                    sum0 = make_float2(sum0.x * keep, sum0.y * keep);
                    sum1 = make_float2(sum1.x * keep, sum1.y * keep);
                    if (i > 0)
#pragma unroll 1
                        for (int d = 0; d < D; d += 8) scale8(o_at + d, keep);
                }
                const float less = most == -INFINITY ? 0.f : kShift<BF16> - most * c;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    if (w == 0) weigh<BF16, 0>(v[0], c, less, p, sum0, sum1);
                    if (w == 1) weigh<BF16, 32>(v[0], c, less, p, sum0, sum1);
                    if (w == 2) weigh<BF16, 0>(v[1], c, less, p, sum0, sum1);
                    if (w == 3) weigh<BF16, 32>(v[1], c, less, p, sum0, sum1);
                    tmem_store16_begin(s_at + w * 16, p);
                    if ((w + 1) % (4 / kParts)) continue;
                    tmem_store_wait();
                    tc::fence_before();
                    warp_arrive(part[mine] + (w + 1) / (4 / kParts) - 1);
                }
            }
            if (ok && it_blocks > 0) {
                ok = warp_wait(sums + mine, sums_phase);
                sums_phase ^= 1;
            }
            tc::fence_after();
            // The tiles take turns in the output's place, once the store before has read it. (Each waits for every phase of
            // a barrier of its own: a wait that skips phases takes the one two before for its own, where items without a
            // key follow one another.)
            if (!ok || !(ok = warp_wait(stored + (mine ^ 1), mine ? n : n ^ 1))) break;
            const float2 both = add2(sum0, sum1);
            const float sum = both.x + both.y;
            const float inv = 1.f / sum;  // rows that see nothing do not use it
            const float2 inv2 = make_float2(inv, inv), zero2 = make_float2(0.f, 0.f);
            float2 check = zero2;  // stays 0 while all is finite
#pragma unroll 1
            for (int d = 0; d < D; d += 32) {
                float o[32];
                if (count > 0) tc::tmem_load32(o_at + d, o);
#pragma unroll
                for (int k = 0; k < 32; k += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float2 x = count > 0 && r.real ? mul2(make_float2(o[k + 2 * u], o[k + 2 * u + 1]), inv2) : zero2;
                        check = fma2(x, zero2, check);
                        w[u] = pack2<BF16>(x.x, x.y);
                    }
                    *reinterpret_cast<uint4*>(output + tile_byte(row, (d + k) / 8)) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            note_again(F.again, __ballot_sync(kFull, !(check.x + check.y == 0.f)), t & ~31, head, kOut);
            fence_to_tma();
            tc::fence_before();
            warp_arrive(staged + mine);
            warp_arrive(item_empty + (n & 1));
            if (F.lse && t < F.S.tokens) {
                const float against = most == -INFINITY ? 0.f : most * c;
                F.lse[head * F.S.tokens + t] = r.real ? (against + __log2f(sum) - kShift<BF16>) * kLn2 : -INFINITY;
            }
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
    const int64_t items = work_items(S);
    if (items > INT32_MAX / 2) return false;
    launch(attention_forward_kernel<D, BF16>, dim3(static_cast<unsigned>(std::min<int64_t>(items, sm_count()))), dim3(kThreads),
           kShared<D>, s, qm, km, vm, om, F, pair_heads, static_cast<int>(items));
    launch_again(F, s);
    return true;
}

}  // namespace

bool launch_forward(const Forward& F, cudaStream_t s) {
    if (F.S.dtype == CB_BF16) return F.S.dim <= 64 ? launch_typed<64, true>(F, s) : launch_typed<128, true>(F, s);
    return F.S.dim <= 64 ? launch_typed<64, false>(F, s) : launch_typed<128, false>(F, s);
}

}  // namespace attention
}  // namespace cbtbe
