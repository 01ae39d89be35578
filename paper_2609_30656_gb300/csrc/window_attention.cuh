// window_attention.cuh -- what the kernels of windowed attention over packed sessions share.
//
//   token t of a session [s, e) sees token j, s <= j <= t, where t - j < window or j - s < sinks
//   S_tj = scale q_t . k_j,  lse_t = log sum_j exp S_tj,  P = exp(S - lse),  o_t = sum_j P_tj v_j
//   dv_j = sum_t P_tj do_t,  dP_tj = do_t . v_j,  delta_t = do_t . o_t,  dS = P (dP - delta)
//   dq_t = scale sum_j dS_tj k_j,  dk_j = scale sum_t dS_tj q_t
//
// A tile of 128 tokens of the packed batch may hold many sessions: which token a row may see is a matter of
// where its session begins, which one small kernel looks up for every token first (2 to 3 us).
//
// fp16 and bf16 rows of a multiple of 8 and at most 128 values go through the tensor cores, all others key by key in fp32: 16384
// tokens x 8 heads of 64 over 2 heads of keys, window 512, 4 first tokens: 49 us forward and 155 backward against 7250 and
// 23100 in fp32 (63 halves: 7900 and 24700). Nothing between them: the rows of such models are halves.
#pragma once

#include "token_rows.cuh"

namespace cbtbe {
namespace attention {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Heads {  // head h of token t at t * token + h * head values
    const void* data;
    int64_t token, head;
};

struct Shape {
    int64_t tokens, sequences, window;
    int32_t heads, kv_heads, group, dim, sinks, dtype;
    float scale;
    const void* offsets;
    int32_t offsets32;
    int32_t* start;  // [tokens] where the token's session begins, and
    int32_t* end;    // [tokens] ends; both t for a token t of no session
    uint32_t* words;  // [kWords] in the workspace, 0 before the tensor-core kernels; or null
    int* error;      // or null
};
constexpr int kWords = 4, kOrderParts = 0, kOrderNext = 1, kOrderDone = 2, kAgainCount = 3;

// Sum over a warp, in every lane.
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(kFull, v, off);
    return v;
}

// Rows whose result is not finite, noted by the tensor-core kernels for those that follow them (window_attention_again.cu):
// the first of 32 tokens, the head (of keys for dK and dV), which of the 32, which result.
struct Again {
    uint32_t* count;  // notes: 0 before
    int4* list;
};
enum Result { kOut = 0, kDq = 0, kDk = 1, kDv = 2, kDkAndDv = 3 };

struct Forward {
    Shape S;
    Heads q, k, v, out;
    float* lse;  // [heads, tokens], or null
    Again again;
};
// How the tiles of keys are taken: those in parts first, then the others. (Results do not depend on who takes what.)
struct Order {
    int32_t* parts;       // how many parts there are,
    uint32_t* next;       // the next item to take: 0 before,
    uint32_t* done;       // blocks that have counted their tiles' parts: 0 before,
    int32_t room;         // parts there is room for; 0: no tile is taken in parts
    int32_t part;         // blocks of queries of a part
    int2* list;           // [room] tile (-1: none) and which of its parts
    int32_t* split;       // [tiles of 128 tokens] parts of each, 0 for one taken whole
    float* sums;          // [room][kv_heads][2][128][64 or 128] dV and dK of each
};
struct Backward {
    Shape S;
    Heads go, q, k, v, out, dq, dk, dv;
    const float* lse;
    float* delta;  // [heads, tokens]
    uint8_t* largest;  // fp16: [heads, padded] the exponent (as of its fp32) of each row's largest finite |grad_out|, 0: all zeros
    int64_t padded;    // tokens in whole tiles
    Order order;
    Again again;
};

// ---------------------------------------------------------------- a row at a time

// Rows of any type and length up to 256, by a warp that goes key by key, in fp32. A row whose sums have all become NaNs
// is done: what follows cannot change it.
constexpr int kMaxDim = 256, kLaneValues = kMaxDim / 32;

// A row of up to 256 values, value lane + 32 i in v[i].
template <int DT>
__device__ __forceinline__ void load_row(const Heads& h, int64_t token, int head, int dim, float (&v)[kLaneValues]) {
    const int64_t at = token * h.token + head * h.head;
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) {
        const int c = (threadIdx.x & 31) + 32 * i;
        v[i] = 0.f;
        if (c < dim) {
            if constexpr (DT == CB_F32) v[i] = static_cast<const float*>(h.data)[at + c];
            else v[i] = widen<DT>(static_cast<const uint16_t*>(h.data)[at + c]);
        }
    }
}
template <int DT>
__device__ __forceinline__ void store_row(const Heads& h, int64_t token, int head, int dim, const float (&v)[kLaneValues]) {
    const int64_t at = token * h.token + head * h.head;
    void* data = const_cast<void*>(h.data);
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) {
        const int c = (threadIdx.x & 31) + 32 * i;
        if (c >= dim) continue;
        if constexpr (DT == CB_F32) static_cast<float*>(data)[at + c] = v[i];
        else static_cast<uint16_t*>(data)[at + c] = static_cast<uint16_t>(narrow<DT>(v[i]));
    }
}
__device__ __forceinline__ float dot(const float (&a)[kLaneValues], const float (&b)[kLaneValues]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) s = fmaf(a[i], b[i], s);
    return warp_sum(s);
}
__device__ __forceinline__ void add_scaled(float (&a)[kLaneValues], float f, const float (&b)[kLaneValues]) {
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) a[i] = fmaf(f, b[i], a[i]);
}

// What token t sees: n tokens, the first `sinks` from `start` on, the others from `first` on. None for one of no session.
struct Seen {
    int64_t start, sinks, first, n;
    __device__ __forceinline__ int64_t at(int64_t i) const { return i < sinks ? start + i : first + (i - sinks); }
};
__device__ __forceinline__ Seen seen_by(const Shape& S, int64_t t) {
    if (S.end[t] <= t) return {t, 0, t, 0};
    Seen a;
    a.start = S.start[t];
    a.first = max64(a.start, t - S.window + 1);
    a.sinks = min64(S.sinks, a.first - a.start);
    a.n = a.sinks + t + 1 - a.first;
    return a;
}
// Behind the last token that sees key j, j for a token of no session.
__device__ __forceinline__ int64_t seen_to(const Shape& S, int64_t j) {
    const int64_t end = S.end[j];
    return end <= j ? j : (j - S.start[j] < S.sinks ? end : min64(end, j + S.window));
}

// Head h of token t: its output, and its lse.
template <int DT>
__device__ __forceinline__ void row_output(const Forward& F, int64_t t, int h, float (&o)[kLaneValues], float& lse) {
    const Shape& S = F.S;
    const int kv = h / S.group;
    float q[kLaneValues], k[kLaneValues], v[kLaneValues];
    float most = -INFINITY, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) o[i] = 0.f;
    lse = -INFINITY;
    const Seen a = seen_by(S, t);
    if (a.n == 0) return;
    load_row<DT>(F.q, t, h, S.dim, q);
    for (int64_t i = 0; i < a.n; ++i) {
        const int64_t j = a.at(i);
        load_row<DT>(F.k, j, kv, S.dim, k);
        load_row<DT>(F.v, j, kv, S.dim, v);
        const float s = dot(q, k) * (S.scale * kLog2e);
        const float top = fmaxf(most, s), keep = most == top ? 1.f : exp2f(most - top);
        const float p = s == -INFINITY ? 0.f : exp2f(s - top);
        sum = fmaf(sum, keep, p);
#pragma unroll
        for (int x = 0; x < kLaneValues; ++x) o[x] = fmaf(o[x], keep, p * v[x]);
        most = top;
        if (sum != sum) break;
    }
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) o[i] /= sum;
    lse = (most + log2f(sum)) * kLn2;
}
template <int DT>
__device__ __forceinline__ void row_dq(const Backward& B, int64_t t, int h, float (&dq)[kLaneValues]) {
    const Shape& S = B.S;
    const int kv = h / S.group;
    float q[kLaneValues], go[kLaneValues], k[kLaneValues], v[kLaneValues];
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) dq[i] = 0.f;
    const Seen a = seen_by(S, t);
    if (a.n == 0) return;
    load_row<DT>(B.q, t, h, S.dim, q);
    load_row<DT>(B.go, t, h, S.dim, go);
    const float lse = B.lse[h * S.tokens + t], delta = B.delta[h * S.tokens + t];
    for (int64_t i = 0; i < a.n; ++i) {
        const int64_t j = a.at(i);
        load_row<DT>(B.k, j, kv, S.dim, k);
        load_row<DT>(B.v, j, kv, S.dim, v);
        const float slope = exp2f((dot(q, k) * S.scale - lse) * kLog2e) * (dot(go, v) - delta) * S.scale;
        add_scaled(dq, slope, k);
        if (slope != slope) break;
    }
}
// Head kv of key j, over the heads that share it and the tokens that see it.
template <int DT>
__device__ __forceinline__ void row_dkv(const Backward& B, int64_t j, int kv, float (&dk)[kLaneValues], float (&dv)[kLaneValues]) {
    const Shape& S = B.S;
    float q[kLaneValues], go[kLaneValues], k[kLaneValues], v[kLaneValues];
#pragma unroll
    for (int i = 0; i < kLaneValues; ++i) dk[i] = dv[i] = 0.f;
    const int64_t last = seen_to(S, j);
    if (last == j) return;
    load_row<DT>(B.k, j, kv, S.dim, k);
    load_row<DT>(B.v, j, kv, S.dim, v);
    for (int h = kv * S.group; h < (kv + 1) * S.group; ++h)
        for (int64_t t = j; t < last; ++t) {
            load_row<DT>(B.q, t, h, S.dim, q);
            load_row<DT>(B.go, t, h, S.dim, go);
            const float p = exp2f((dot(q, k) * S.scale - B.lse[h * S.tokens + t]) * kLog2e);
            add_scaled(dv, p, go);
            add_scaled(dk, p * (dot(go, v) - B.delta[h * S.tokens + t]) * S.scale, q);
            if (p != p) return;
        }
}

// For the 32 tokens from `token` on, by lane 0 of a warp.
__device__ __forceinline__ void note_again(const Again& A, uint32_t rows, int64_t token, int head, Result which) {
    if (rows && (threadIdx.x & 31) == 0)
        A.list[atomicAdd(A.count, 1u)] = make_int4(static_cast<int>(token), head, static_cast<int>(rows), which);
}

inline size_t rows_bytes(int64_t tokens) { return static_cast<size_t>((tokens * 4 + 255) / 256 * 256); }

// The tensor-core kernels (window_attention_forward.cu, window_attention_backward.cu); they want fp16 or
// bf16, rows of a multiple of 8 and at most 128 values, addresses and strides in multiples of 16 bytes.
bool tensor_core_rows(const Shape& S, const Heads& h, int heads);
int sm_count();  // of the current device
int32_t part_blocks(int64_t tokens, int32_t heads, int32_t kv_heads, int64_t window);
int64_t parts_room(int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim, int64_t window, int64_t sinks);
int64_t parts_bytes(int64_t room, int32_t kv_heads, int32_t dim);
bool launch_forward(const Forward& F, cudaStream_t s);
bool launch_backward(const Backward& B, cudaStream_t s);
void launch_again(const Forward& F, cudaStream_t s);  // behind them
void launch_again(const Backward& B, cudaStream_t s);

}  // namespace attention
}  // namespace cbtbe
