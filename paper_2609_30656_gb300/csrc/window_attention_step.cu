// window_attention_step.cu -- windowed attention of one new token for each session over a cache of keys
// and values (include/cb_tbe.h).
#include "muon_internal.cuh"
#include "spans.h"
#include "window_attention.cuh"

#include <algorithm>
#include <atomic>
#include <cmath>

namespace cbtbe {
namespace attention {
namespace {

constexpr int kWarps = 8;

struct Step {
    const void *q, *k, *v;
    void* out;
    int64_t q_seq, q_head, k_seq, k_token, k_head, v_seq, v_token, v_head, out_seq, out_head;  // strides in values
    int64_t sequences, capacity, window;
    int32_t heads, kv_heads, group, dim, sinks, dtype;
    float scale;
    const void* lengths;
    int32_t lengths32;
    int* error;  // or null
};

// Tokens of session b in its cache; one that does not fit sets the error word and counts as none.
__device__ __forceinline__ int64_t length_of(const Step& A, int64_t b) {
    const int64_t n = load_index(A.lengths, b, A.lengths32);
    if (n >= 0 && n <= A.capacity) return n;
    if (A.error && threadIdx.x == 0) set_error(A.error, CB_ERR_INDEX_OOB);
    return 0;
}

// The caches of session b.
__device__ __forceinline__ const void* k_of(const Step& A, int64_t b) {
    return static_cast<const char*>(A.k) + b * A.k_seq * (A.dtype == CB_F32 ? 4 : 2);
}
__device__ __forceinline__ const void* v_of(const Step& A, int64_t b) {
    return static_cast<const char*>(A.v) + b * A.v_seq * (A.dtype == CB_F32 ? 4 : 2);
}

// A block for a head of a session; its warps take every eighth key and join what they have.
template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_step_rowwise_kernel(const Step A) {
    __shared__ float most_of[kWarps], sum_of[kWarps], o_of[kWarps][kMaxDim];
    begin_kernel();
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    for (int64_t w = blockIdx.x; w < A.sequences * A.heads; w += gridDim.x) {
        const int64_t b = w / A.heads;
        const int h = static_cast<int>(w - b * A.heads), kv = h / A.group;
        const int64_t n = length_of(A, b), first = max64(0, n - A.window), sinks = min64(A.sinks, first);
        float q[kLaneValues], o[kLaneValues] = {}, k[kLaneValues], v[kLaneValues];
        float most = -INFINITY, sum = 0.f;
        load_row<DT>({A.q, A.q_seq, A.q_head}, b, h, A.dim, q);
        for (int64_t i = warp; i < sinks + (n - first); i += kWarps) {
            const int64_t j = i < sinks ? i : first + (i - sinks);
            load_row<DT>({k_of(A, b), A.k_token, A.k_head}, j, kv, A.dim, k);
            load_row<DT>({v_of(A, b), A.v_token, A.v_head}, j, kv, A.dim, v);
            float s = 0.f;
#pragma unroll
            for (int x = 0; x < kLaneValues; ++x) s = fmaf(q[x], k[x], s);
            s = warp_sum(s) * (A.scale * kLog2e);
            const float top = fmaxf(most, s), keep = most == top ? 1.f : exp2f(most - top);
            const float p = s == -INFINITY ? 0.f : exp2f(s - top);
            sum = fmaf(sum, keep, p);
#pragma unroll
            for (int x = 0; x < kLaneValues; ++x) o[x] = fmaf(o[x], keep, p * v[x]);
            most = top;
        }
        if (lane == 0) {
            most_of[warp] = most;
            sum_of[warp] = sum;
        }
#pragma unroll
        for (int x = 0; x < kLaneValues; ++x) o_of[warp][lane + 32 * x] = o[x];
        __syncthreads();
        float top = -INFINITY, total = 0.f, value = 0.f;
        for (int x = 0; x < kWarps; ++x) top = fmaxf(top, most_of[x]);
        for (int x = 0; x < kWarps; ++x) {
            if (sum_of[x] == 0.f) continue;  // no key
            const float f = exp2f(most_of[x] - top);
            total = fmaf(sum_of[x], f, total);
            value = fmaf(o_of[x][threadIdx.x], f, value);
        }
        if (static_cast<int>(threadIdx.x) < A.dim) {
            const float r = n > 0 ? value / total : 0.f;
            const int64_t at = b * A.out_seq + h * A.out_head + threadIdx.x;
            if constexpr (DT == CB_F32) static_cast<float*>(A.out)[at] = r;
            else static_cast<uint16_t*>(A.out)[at] = static_cast<uint16_t>(narrow<DT>(r));
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- 16-bit rows in whole 16-byte pieces

// The keys and values of a session are read once, by the 16 heads at most that share them: bytes bound it, and what
// counts is how many are on their way. A block of four warps has a part of the keys of one head of keys; each warp
// copies its own tiles of 16 keys and values ahead (cp.async, three tiles of 8 KB) and waits for no other.
// Scores and sums are small products (mma.sync, 16 x 8 x 16, the queries of the sharing heads as rows): on the
// CUDA cores 16 bytes of keys would cost 16 multiplications for every head. The warps' sums are joined at the block's end, the
// parts' by a second kernel, both in order. 256 sessions of 4100 keys of 4 heads of 128, bf16, 16 query heads: 2.15 GB in
// 329 us, 6.5 TB/s, 96 % of the copy rate; rows that go key by key instead (256 x 2048 keys of 64): 1280 us in fp32 and 1528
// for 63 halves, against 105 us for 64 halves.
constexpr int kStepWarps = 4, kStepKeys = 16, kStepStages = 3, kStepHeads = 16;
template <int D> constexpr int kStepRow = D * 2;  // bytes
template <int D> constexpr int kStepTile = 2 * kStepKeys * kStepRow<D>;
template <int D> constexpr size_t kStepShared = static_cast<size_t>(kStepWarps) * kStepStages * kStepTile<D>;

struct Parts {
    int32_t parts, head_blocks;
    float* sums;  // [sequences][heads][parts][dim + 2]: sums of values, the maximum, the sum of weights; null for one part
};

template <bool BF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t r;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {  // zeros where not `in`
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void load_matrices(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void load_matrices_turned(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
template <bool BF16>
__device__ __forceinline__ void multiply(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
                     "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
                     "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kStepWarps * 32, 2)
attention_step_kernel(const Step A, const Parts P) {
    constexpr int kPieces = D / 8, kPerLane = kStepKeys * kPieces / 32;
    constexpr float kShift = BF16 ? 0.f : 8.f;  // fp16 holds weights times 2^8: small ones keep their digits
    extern __shared__ __align__(128) unsigned char tiles[];
    begin_kernel();
    const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
    // Parts of one session and head are neighbours, then heads that read the same lines of the cache.
    int64_t w = blockIdx.x;
    const int part = static_cast<int>(w % P.parts);
    w /= P.parts;
    const int head_block = static_cast<int>(w % P.head_blocks);
    w /= P.head_blocks;
    const int kv = static_cast<int>(w % A.kv_heads);
    const int64_t b = w / A.kv_heads;
    const int head0 = kv * A.group + head_block * kStepHeads, heads = min(A.group - head_block * kStepHeads, kStepHeads);
    const int n = static_cast<int>(length_of(A, b)), first = static_cast<int>(max64(0, n - A.window));
    const int sinks = min(A.sinks, first), seen = sinks + (n - first);
    // This part's share of the keys in sight, in whole tiles; and this warp's tiles of it.
    const int tiles_all = (seen + kStepKeys - 1) / kStepKeys, share = (tiles_all + P.parts - 1) / P.parts;
    const int tile0 = min(part * share, tiles_all), tile1 = min(tile0 + share, tiles_all);
    const char* keys = static_cast<const char*>(k_of(A, b)) + kv * A.k_head * 2;
    const char* values = static_cast<const char*>(v_of(A, b)) + kv * A.v_head * 2;
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(tiles)) + warp * kStepStages * kStepTile<D>;
    // 16 bytes c of row r: 8 neighbouring rows at one c are in 8 different places of 128 bytes.
    auto place = [&](int r, int c) { return static_cast<uint32_t>(r * kStepRow<D> + ((c ^ (r & 7)) << 4)); };
    auto copy = [&](int tile, int stage) {
        if (tile < tile1) {
            const uint32_t to = mine + stage * kStepTile<D>;
#pragma unroll
            for (int x = 0; x < kPerLane; ++x) {
                const int at = x * 32 + lane, r = at / kPieces, c = at % kPieces;
                const int i = tile * kStepKeys + r;
                const int64_t pos = i < sinks ? i : first + (i - sinks);
                const bool in = i < seen && c * 8 < A.dim;
                copy16(to + place(r, c), in ? keys + (pos * A.k_token + c * 8) * 2 : keys, in);
                copy16(to + kStepTile<D> / 2 + place(r, c), in ? values + (pos * A.v_token + c * 8) * 2 : values, in);
            }
        }
        copies_begun();
    };
#pragma unroll
    for (int s = 0; s < kStepStages - 1; ++s) copy(tile0 + warp + s * kStepWarps, s);

    // The queries: rows lane / 4 and lane / 4 + 8 of 16, columns (lane % 4) * 2 and 8 on, of every 16.
    uint32_t q[D / 16][4];
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int r = lane / 4 + (x & 1) * 8, c = k * 16 + (x >> 1) * 8 + lane % 4 * 2;
            q[k][x] = 0u;
            if (r < heads && c < A.dim) {
                const uint16_t* p = static_cast<const uint16_t*>(A.q) + b * A.q_seq +
                                    static_cast<int64_t>(head0 + r) * A.q_head + c;
                q[k][x] = static_cast<uint32_t>(p[0]) | static_cast<uint32_t>(p[1]) << 16;
            }
        }
    const float c = fmaxf(fabsf(A.scale) * kLog2e, 1e-30f), sign = A.scale < 0.f ? -1.f : 1.f;
    float o[D / 8][4] = {}, most[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
    int stage = 0;
    for (int tile = tile0 + warp; tile < tile1; tile += kStepWarps) {
        copies_done<kStepStages - 2>();
        __syncwarp();
        const uint32_t at = mine + stage * kStepTile<D>;
        float s[2][4] = {};
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            uint32_t m[4];  // keys 0 .. 7 by values 0 .. 7 and 8 .. 15 of these 16, keys 8 .. 15 alike
            load_matrices(at + place((lane & 7) + (lane >> 4) * 8, k * 2 + (lane >> 3 & 1)), m);
            multiply<BF16>(s[0], q[k], m[0], m[1]);
            multiply<BF16>(s[1], q[k], m[2], m[3]);
        }
        const int left = seen - tile * kStepKeys;  // keys of the tile
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[x][i] = x * 8 + lane % 4 * 2 + (i & 1) < left ? s[x][i] * sign : -INFINITY;
                top[i >> 1] = fmaxf(top[i >> 1], s[x][i]);
            }
        float keep[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(kFull, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(kFull, top[i], 2));
            top[i] = fmaxf(top[i], most[i]);
            keep[i] = top[i] == most[i] ? 1.f : exp2f((most[i] - top[i]) * c);
            most[i] = top[i];
            sum[i] *= keep[i];
        }
        if (__any_sync(kFull, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
            for (int d = 0; d < D / 8; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[d][i] *= keep[i >> 1];
        }
        const float base[2] = {kShift - (top[0] == -INFINITY ? 0.f : top[0] * c),
                               kShift - (top[1] == -INFINITY ? 0.f : top[1] * c)};
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[x][i] = exp2f(fmaf(s[x][i], c, base[i >> 1]));
                sum[i >> 1] += s[x][i];
            }
        const uint32_t p[4] = {pack<BF16>(s[0][0], s[0][1]), pack<BF16>(s[0][2], s[0][3]), pack<BF16>(s[1][0], s[1][1]),
                               pack<BF16>(s[1][2], s[1][3])};
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            uint32_t m[4];  // values 0 .. 7 of these 16 by keys 0 .. 7 and 8 .. 15, values 8 .. 15 alike
            load_matrices_turned(at + kStepTile<D> / 2 + place((lane & 7) + (lane >> 3 & 1) * 8, d * 2 + (lane >> 4)), m);
            multiply<BF16>(o[2 * d], p, m[0], m[1]);
            multiply<BF16>(o[2 * d + 1], p, m[2], m[3]);
        }
        __syncwarp();
        copy(tile + (kStepStages - 1) * kStepWarps, stage == 0 ? kStepStages - 1 : stage - 1);
        if (++stage == kStepStages) stage = 0;
    }
    copies_done<0>();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(kFull, sum[i], 1);
        sum[i] += __shfl_xor_sync(kFull, sum[i], 2);
    }
    // The warps' sums, joined in order.
    constexpr int kJoin = D + 4;  // floats of a head
    static_assert(kStepWarps * kStepHeads * kJoin * 4 <= kStepShared<D>, "");
    float* joined = reinterpret_cast<float*>(tiles);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float* to = joined + (warp * kStepHeads + lane / 4 + i * 8) * kJoin;
#pragma unroll
        for (int d = 0; d < D / 8; ++d) {
            to[d * 8 + lane % 4 * 2] = o[d][2 * i];
            to[d * 8 + lane % 4 * 2 + 1] = o[d][2 * i + 1];
        }
        if (lane % 4 == 0) {
            to[D] = most[i];
            to[D + 1] = sum[i];
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < heads * D; x += kStepWarps * 32) {
        const int h = x / D, d = x % D;
        if (d >= A.dim) continue;
        float top = -INFINITY, total = 0.f, value = 0.f;
        for (int y = 0; y < kStepWarps; ++y) top = fmaxf(top, joined[(y * kStepHeads + h) * kJoin + D]);
        for (int y = 0; y < kStepWarps; ++y) {
            const float* from = joined + (y * kStepHeads + h) * kJoin;
            if (from[D + 1] == 0.f) continue;  // no key
            const float f = from[D] == top ? 1.f : exp2f((from[D] - top) * c);
            total = fmaf(from[D + 1], f, total);
            value = fmaf(from[d], f, value);
        }
        const int64_t row = b * A.heads + head0 + h;
        if (P.sums) {
            float* to = P.sums + (row * P.parts + part) * (A.dim + 2);
            to[d] = value;
            if (d == 0) {
                to[A.dim] = top;
                to[A.dim + 1] = total;
            }
        } else {
            const float r = n > 0 ? value / total : 0.f;
            static_cast<uint16_t*>(A.out)[b * A.out_seq + static_cast<int64_t>(head0 + h) * A.out_head + d] =
                static_cast<uint16_t>(narrow<BF16 ? CB_BF16 : CB_F16>(r));
        }
    }
}

// The parts' sums of a head of a session, joined by a block: what each part counts for first, then their values, a thread
// for a value and, of many parts, every eighth of them (one thread for all of 256 parts waited for one after the
// other: 180 of 200 us for one session of 65536 tokens). All sums in one order.
constexpr int kMostParts = 2048, kJoinColumns = 128, kJoinGroups = 8;
inline int join_threads(int parts) { return parts < 2 * kJoinGroups ? kJoinColumns : kJoinColumns * kJoinGroups; }
template <bool BF16>
__global__ void __launch_bounds__(kJoinColumns * kJoinGroups) attention_step_join_kernel(const Step A, const Parts P) {
    __shared__ float counts[kMostParts], values[kJoinGroups][kJoinColumns], of_warp[2][kJoinColumns * kJoinGroups / 32];
    begin_kernel();
    const float c = fmaxf(fabsf(A.scale) * kLog2e, 1e-30f);
    const int64_t row = blockIdx.x, b = row / A.heads;
    const int h = static_cast<int>(row - b * A.heads), threads = static_cast<int>(blockDim.x), t = static_cast<int>(threadIdx.x);
    const int stride = A.dim + 2;
    const float* from = P.sums + row * P.parts * stride;
    float top = -INFINITY, total = 0.f, value = 0.f;
    for (int y = t; y < P.parts; y += threads) top = fmaxf(top, __ldcg(from + static_cast<int64_t>(y) * stride + A.dim));
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, off));
    if (t % 32 == 0) of_warp[0][t / 32] = top;
    __syncthreads();
    for (int w = 0; w < threads / 32; ++w) top = fmaxf(top, of_warp[0][w]);
    for (int y = t; y < P.parts; y += threads) {
        const float* at = from + static_cast<int64_t>(y) * stride + A.dim;
        const float most = __ldcg(at), sum = __ldcg(at + 1), f = most == top ? 1.f : exp2f((most - top) * c);
        counts[y] = sum == 0.f ? -1.f : f;  // no key
        if (sum != 0.f) total = fmaf(sum, f, total);
    }
    total = warp_sum(total);
    if (t % 32 == 0) of_warp[1][t / 32] = total;
    __syncthreads();
    const int d = t % kJoinColumns, group = t / kJoinColumns, groups = threads / kJoinColumns;
    if (d < A.dim) {
#pragma unroll 4
        for (int y = group; y < P.parts; y += groups) {
            const float x = __ldcg(from + static_cast<int64_t>(y) * stride + d), f = counts[y];
            value = f < 0.f ? value : fmaf(x, f, value);
        }
    }
    values[group][d] = value;
    __syncthreads();
    if (t >= A.dim || t >= kJoinColumns) return;
    total = value = 0.f;
    for (int w = 0; w < threads / 32; ++w) total += of_warp[1][w];
    for (int g = 0; g < groups; ++g) value += values[g][d];
    const float r = length_of(A, b) > 0 ? value / total : 0.f;
    static_cast<uint16_t*>(A.out)[b * A.out_seq + static_cast<int64_t>(h) * A.out_head + d] =
        static_cast<uint16_t>(narrow<BF16 ? CB_BF16 : CB_F16>(r));
}

// Parts of the keys of a session: so many that the blocks make four rounds of the GPU's two blocks an SM, none of
// fewer than 256 keys. With more, a block's beginning and end and the joining weigh more, with fewer the last round idles more
// of the GPU (of 12, 6, 4 and 3 rounds: 256 sessions of 4100 keys 360, 329, 329 and 331 us; 16 of 65536 338, 332, 315 and
// 355; 4 of 65536 134, 109, 102 and 97; 64 of 1 to 16384 185, 167, 163 and 162).
int parts_of(int64_t sequences, int32_t kv_heads, int32_t group, int64_t capacity, int64_t window, int64_t sinks) {
    const int64_t blocks = sequences * kv_heads * ((group + kStepHeads - 1) / kStepHeads);
    const int64_t seen = std::min(capacity, window > capacity ? capacity : window + std::min(sinks, capacity));
    const int64_t wanted = (static_cast<int64_t>(sm_count()) * 2 * 4 + blocks - 1) / blocks;
    return static_cast<int>(std::max<int64_t>(1, std::min({wanted, seen / 256, int64_t{kMostParts}})));
}

template <int D, bool BF16>
bool launch_step(const Step& A, const Parts& P, cudaStream_t s) {
    static std::atomic<uint64_t> devices{0};
    if (!muon::shared_memory(attention_step_kernel<D, BF16>, kStepShared<D>, devices)) return false;
    const int64_t grid = A.sequences * A.kv_heads * P.head_blocks * P.parts;
    if (grid > INT32_MAX || A.sequences * A.heads > INT32_MAX) return false;
    launch(attention_step_kernel<D, BF16>, dim3(static_cast<unsigned>(grid)), dim3(kStepWarps * 32), kStepShared<D>, s, A, P);
    if (P.sums)
        launch(attention_step_join_kernel<BF16>, dim3(static_cast<unsigned>(A.sequences * A.heads)),
               dim3(join_threads(P.parts)), 0, s, A, P);
    return true;
}

bool type_ok(int t) { return t == CB_F32 || t == CB_F16 || t == CB_BF16; }
constexpr int64_t kMost = int64_t{1} << 40;
bool stride_ok(int64_t s) { return s >= 0 && s <= kMost; }
bool sizes_ok(int64_t sequences, int64_t capacity, int32_t heads, int32_t kv_heads, int32_t dim, int64_t window, int64_t sinks) {
    return sequences >= 0 && sequences < (int64_t{1} << 31) && capacity >= 0 && capacity < (int64_t{1} << 31) - 1024 &&
           heads >= 1 && heads <= 65535 && kv_heads >= 1 && heads % kv_heads == 0 && dim >= 1 &&
           dim <= kMaxDim && window >= 1 && sinks >= 0;
}

}  // namespace
}  // namespace attention
}  // namespace cbtbe

extern "C" int64_t cb_attention_step_workspace_bytes(int64_t sequences, int32_t heads, int32_t kv_heads, int32_t dim,
                                                     int64_t capacity, int64_t window, int64_t sinks) {
    using namespace cbtbe::attention;
    if (!sizes_ok(sequences, capacity, heads, kv_heads, dim, window, sinks) || sequences == 0) return 0;
    const int parts = parts_of(sequences, kv_heads, heads / kv_heads, capacity, window, sinks);
    return parts > 1 ? sequences * heads * parts * (dim + 2) * 4 : 0;
}

extern "C" cb_status cb_attention_step(const void* q, const void* k_cache, const void* v_cache, cb_dtype dtype,
                                       int64_t sequences, int64_t capacity, int32_t heads, int32_t kv_heads, int32_t dim,
                                       int64_t q_sequence_stride, int64_t q_head_stride, int64_t k_sequence_stride,
                                       int64_t k_token_stride, int64_t k_head_stride, int64_t v_sequence_stride,
                                       int64_t v_token_stride, int64_t v_head_stride, const void* lengths,
                                       cb_index_dtype idx_dtype, int64_t window, int64_t sinks, float scale, void* out,
                                       int64_t out_sequence_stride, int64_t out_head_stride, void* workspace,
                                       int64_t workspace_bytes, int* error, cudaStream_t stream) {
    using namespace cbtbe::attention;
    if (!type_ok(dtype) || !sizes_ok(sequences, capacity, heads, kv_heads, dim, window, sinks) || !(scale == scale) ||
        (idx_dtype != CB_I32 && idx_dtype != CB_I64) || reinterpret_cast<uintptr_t>(error) % 4)
        return CB_ERR_INVALID_ARG;
    for (const int64_t s : {q_sequence_stride, q_head_stride, k_sequence_stride, k_token_stride, k_head_stride,
                            v_sequence_stride, v_token_stride, v_head_stride, out_sequence_stride, out_head_stride})
        if (!stride_ok(s)) return CB_ERR_INVALID_ARG;
    if (!cbtbe::rows_apart(sequences, out_sequence_stride, heads, out_head_stride, dim)) return CB_ERR_INVALID_ARG;
    if (sequences == 0) return CB_OK;
    const uintptr_t mask = dtype == CB_F32 ? 3 : 1;
    if (!q || !out || !lengths || (capacity > 0 && (!k_cache || !v_cache)) || (reinterpret_cast<uintptr_t>(q) & mask) ||
        (reinterpret_cast<uintptr_t>(k_cache) & mask) || (reinterpret_cast<uintptr_t>(v_cache) & mask) ||
        (reinterpret_cast<uintptr_t>(out) & mask) ||
        reinterpret_cast<uintptr_t>(lengths) % (idx_dtype == CB_I32 ? 4 : 8))
        return CB_ERR_INVALID_ARG;
    const int64_t need = cb_attention_step_workspace_bytes(sequences, heads, kv_heads, dim, capacity, window, sinks);
    if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < need)) return CB_ERR_CAPACITY;
    auto span = [&](const void* p, int64_t sequence, int64_t token, int64_t head, int64_t tokens, int32_t n) {
        const int64_t size = mask + 1;
        return cbtbe::Span(p, dim * size).by(sequences, sequence * size).by(tokens, token * size).by(n, head * size);
    };
    if (cbtbe::overlap({span(out, out_sequence_stride, 0, out_head_stride, 1, heads), {workspace, need}, {error, 4}},
                       {span(q, q_sequence_stride, 0, q_head_stride, 1, heads),
                        span(k_cache, k_sequence_stride, k_token_stride, k_head_stride, capacity, kv_heads),
                        span(v_cache, v_sequence_stride, v_token_stride, v_head_stride, capacity, kv_heads),
                        {lengths, sequences * (idx_dtype == CB_I32 ? 4 : 8)}}))
        return CB_ERR_INVALID_ARG;
    Step A{};
    A.q = q;
    A.k = k_cache;
    A.v = v_cache;
    A.out = out;
    A.q_seq = q_sequence_stride;
    A.q_head = q_head_stride;
    A.k_seq = k_sequence_stride;
    A.k_token = k_token_stride;
    A.k_head = k_head_stride;
    A.v_seq = v_sequence_stride;
    A.v_token = v_token_stride;
    A.v_head = v_head_stride;
    A.out_seq = out_sequence_stride;
    A.out_head = out_head_stride;
    A.sequences = sequences;
    A.capacity = capacity;
    A.window = std::min<int64_t>(window, int64_t{1} << 31);
    A.heads = heads;
    A.kv_heads = kv_heads;
    A.group = heads / kv_heads;
    A.dim = dim;
    A.sinks = static_cast<int32_t>(std::min<int64_t>(sinks, (int64_t{1} << 31) - 1));
    A.dtype = dtype;
    A.scale = scale;
    A.lengths = lengths;
    A.lengths32 = idx_dtype == CB_I32;
    A.error = error;
    bool fast = dtype != CB_F32 && dim % 8 == 0 && dim <= 128;
    for (const int64_t x : {k_sequence_stride, k_token_stride, k_head_stride, v_sequence_stride, v_token_stride, v_head_stride})
        fast = fast && x % 8 == 0;
    fast = fast && reinterpret_cast<uintptr_t>(k_cache) % 16 == 0 && reinterpret_cast<uintptr_t>(v_cache) % 16 == 0;
    if (fast) {
        Parts P{};
        P.parts = parts_of(sequences, kv_heads, A.group, capacity, window, sinks);
        P.head_blocks = (A.group + kStepHeads - 1) / kStepHeads;
        P.sums = P.parts > 1 ? static_cast<float*>(workspace) : nullptr;
        bool ok;
        if (dtype == CB_BF16) ok = dim <= 64 ? launch_step<64, true>(A, P, stream) : launch_step<128, true>(A, P, stream);
        else ok = dim <= 64 ? launch_step<64, false>(A, P, stream) : launch_step<128, false>(A, P, stream);
        return cudaGetLastError() == cudaSuccess && ok ? CB_OK : CB_ERR_CUDA;
    }
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(sequences * heads, 1 << 20)));
    if (dtype == CB_F32) cbtbe::launch(attention_step_rowwise_kernel<CB_F32>, grid, dim3(kWarps * 32), 0, stream, A);
    else if (dtype == CB_F16) cbtbe::launch(attention_step_rowwise_kernel<CB_F16>, grid, dim3(kWarps * 32), 0, stream, A);
    else cbtbe::launch(attention_step_rowwise_kernel<CB_BF16>, grid, dim3(kWarps * 32), 0, stream, A);
    return cudaGetLastError() == cudaSuccess ? CB_OK : CB_ERR_CUDA;
}
