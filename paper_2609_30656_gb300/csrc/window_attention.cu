// window_attention.cu -- windowed attention over packed sessions (include/cb_tbe.h): where each
// token's session begins, the kernels for rows that the tensor cores' do not take (fp32, lengths that are no
// multiple of 8 or over 128, unaligned), and the entry points.
#include "spans.h"
#include "window_attention_tc.cuh"

#include <algorithm>
#include <cmath>
#include <cudaTypedefs.h>

namespace cbtbe {
namespace attention {
namespace {

constexpr int kWarps = 8;

// The session of each token, by a search over the offsets. Offsets that decrease or leave [0, tokens]
// set the error word; what is stored stays within the tokens all the same.
__global__ void __launch_bounds__(256) attention_rows_kernel(const Shape S) {
    begin_kernel();
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    for (int64_t t = first; t < S.tokens; t += step) {
        int64_t lo = 0, hi = S.sequences + 1;  // the first offset above t
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (load_index(S.offsets, mid, S.offsets32) <= t) lo = mid + 1;
            else hi = mid;
        }
        int64_t s = t, e = t;
        if (lo > 0 && lo <= S.sequences) {
            s = max64(0, min64(load_index(S.offsets, lo - 1, S.offsets32), t));
            e = max64(t + 1, min64(load_index(S.offsets, lo, S.offsets32), S.tokens));
        }
        S.start[t] = static_cast<int32_t>(s);
        S.end[t] = static_cast<int32_t>(e);
    }
    if (S.words && first < kWords) S.words[first] = 0u;
    if (!S.error) return;
    for (int64_t i = first; i <= S.sequences; i += step) {
        const int64_t here = load_index(S.offsets, i, S.offsets32);
        const int64_t before = i ? load_index(S.offsets, i - 1, S.offsets32) : 0;
        if (here < before || here < 0 || here > S.tokens) set_error(S.error, CB_ERR_BAD_OFFSETS);
    }
}

// A warp for a head of a token, key after key.
template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_rowwise_kernel(const Forward F) {
    begin_kernel();
    const Shape& S = F.S;
    for (int64_t w = warp_id_global(); w < S.tokens * S.heads; w += warps_in_grid()) {
        const int64_t t = w / S.heads;
        const int h = static_cast<int>(w - t * S.heads);
        float o[kLaneValues], lse;
        row_output<DT>(F, t, h, o, lse);
        store_row<DT>(F.out, t, h, S.dim, o);
        if (F.lse && (threadIdx.x & 31) == 0) F.lse[h * S.tokens + t] = lse;
    }
}

// delta_t = do_t . o_t for a head of a token.
template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_delta_rowwise_kernel(const Backward B) {
    begin_kernel();
    const Shape& S = B.S;
    for (int64_t w = warp_id_global(); w < S.tokens * S.heads; w += warps_in_grid()) {
        const int64_t t = w / S.heads;
        const int h = static_cast<int>(w - t * S.heads);
        float a[kLaneValues], b[kLaneValues];
        load_row<DT>(B.go, t, h, S.dim, a);
        load_row<DT>(B.out, t, h, S.dim, b);
        const float d = dot(a, b);
        if ((threadIdx.x & 31) == 0) B.delta[h * S.tokens + t] = d;
    }
}

template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_dq_rowwise_kernel(const Backward B) {
    begin_kernel();
    const Shape& S = B.S;
    for (int64_t w = warp_id_global(); w < S.tokens * S.heads; w += warps_in_grid()) {
        const int64_t t = w / S.heads;
        const int h = static_cast<int>(w - t * S.heads);
        float dq[kLaneValues];
        row_dq<DT>(B, t, h, dq);
        store_row<DT>(B.dq, t, h, S.dim, dq);
    }
}

// A warp for a head of a key, over the heads that share it and the tokens that see it.
template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_dkv_rowwise_kernel(const Backward B) {
    begin_kernel();
    const Shape& S = B.S;
    for (int64_t w = warp_id_global(); w < S.tokens * S.kv_heads; w += warps_in_grid()) {
        const int64_t j = w / S.kv_heads;
        const int kv = static_cast<int>(w - j * S.kv_heads);
        float dk[kLaneValues], dv[kLaneValues];
        row_dkv<DT>(B, j, kv, dk, dv);
        store_row<DT>(B.dk, j, kv, S.dim, dk);
        store_row<DT>(B.dv, j, kv, S.dim, dv);
    }
}

template <int DT>
void launch_forward_rowwise(const Forward& F, cudaStream_t s) {
    launch(attention_rowwise_kernel<DT>, dim3(warp_grid(F.S.tokens * F.S.heads, 1 << 20)), dim3(kWarps * 32), 0, s, F);
}
template <int DT>
void launch_backward_rowwise(const Backward& B, cudaStream_t s) {
    const dim3 rows(warp_grid(B.S.tokens * B.S.heads, 1 << 20)), keys(warp_grid(B.S.tokens * B.S.kv_heads, 1 << 20));
    launch(attention_delta_rowwise_kernel<DT>, rows, dim3(kWarps * 32), 0, s, B);
    launch(attention_dq_rowwise_kernel<DT>, rows, dim3(kWarps * 32), 0, s, B);
    launch(attention_dkv_rowwise_kernel<DT>, keys, dim3(kWarps * 32), 0, s, B);
}

bool type_ok(int t) { return t == CB_F32 || t == CB_F16 || t == CB_BF16; }
constexpr int64_t kMostTmaStride = int64_t{1} << 38;  // values: 2^40 bytes are refused
constexpr int64_t kMostTokens = (int64_t{1} << 31) - 1024, kMostStride = int64_t{1} << 40;

bool heads_ok(const Shape& S, const Heads& h, int heads, bool written) {
    const int size = S.dtype == CB_F32 ? 4 : 2;
    if (!h.data || reinterpret_cast<uintptr_t>(h.data) % size || h.token < 0 || h.head < 0 || h.token > kMostStride ||
        h.head > kMostStride)
        return false;
    return !written || rows_apart(S.tokens, h.token, heads, h.head, S.dim);
}
// The memory of a tensor. Blocks read what others have written by then, so results lie apart from what is read.
Span span(const Shape& S, const Heads& h, int heads) {
    const int64_t size = S.dtype == CB_F32 ? 4 : 2;
    return Span(h.data, S.dim * size).by(S.tokens, h.token * size).by(heads, h.head * size);
}
Span offsets_span(const Shape& S) { return Span(S.offsets, (S.sequences + 1) * (S.offsets32 ? 4 : 8)); }
cb_status sizes_ok(const Shape& S) {
    if (!type_ok(S.dtype) || S.tokens < 0 || S.tokens > kMostTokens || S.sequences < 0 || S.sequences > kMostTokens ||
        S.heads < 1 || S.kv_heads < 1 || S.heads > 65535 || S.heads % S.kv_heads || S.dim < 1 || S.dim > kMaxDim ||
        S.window < 1 || S.sinks < 0 || !(S.scale == S.scale) || !S.offsets ||
        reinterpret_cast<uintptr_t>(S.offsets) % (S.offsets32 ? 4 : 8) || reinterpret_cast<uintptr_t>(S.error) % 4)
        return CB_ERR_INVALID_ARG;
    return CB_OK;
}
Shape shape(int dtype, int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim, const void* offsets, int idx,
            int64_t sequences, int64_t window, int64_t sinks, float scale, int* error) {
    Shape S{};
    S.tokens = tokens;
    S.sequences = sequences;
    S.window = std::min<int64_t>(window, kMostTokens);
    S.heads = heads;
    S.kv_heads = kv_heads;
    S.group = kv_heads > 0 ? heads / kv_heads : 0;
    S.dim = dim;
    S.sinks = sinks < 0 ? -1 : static_cast<int32_t>(std::min<int64_t>(sinks, kMostTokens));
    S.dtype = dtype;
    S.scale = scale;
    S.offsets = idx == CB_I32 || idx == CB_I64 ? offsets : nullptr;
    S.offsets32 = idx == CB_I32;
    S.error = error;
    return S;
}
// The workspace: bytes before each part of it, and all.
struct Layout {
    size_t words, again, delta, largest, list, split, sums, bytes;
    int64_t room;
};
Layout layout(int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim, int64_t window, int64_t sinks, bool backward) {
    const int64_t tiles = tiles_of(static_cast<int>(tokens));
    // 32 rows of a tile and head are noted at most once for each result.
    const int64_t notes = dim % 8 || dim > 128 ? 0 : tiles * (4 * heads + (backward ? 8 * kv_heads : 0));
    Layout L{};
    L.words = 2 * rows_bytes(tokens);
    L.again = L.words + 256;
    L.delta = L.again + rows_bytes(4 * notes);
    L.bytes = L.delta;
    if (!backward) return L;
    L.room = parts_room(tokens, heads, kv_heads, dim, window, sinks);
    L.largest = L.delta + rows_bytes(tokens * heads);
    L.list = L.largest + rows_bytes(tiles * heads * (kTile / 4));
    L.split = L.list + rows_bytes(2 * L.room);
    L.sums = L.split + (L.room ? rows_bytes(tiles) : 0);
    L.bytes = L.sums + static_cast<size_t>(parts_bytes(L.room, kv_heads, dim));
    return L;
}
bool workspace_ok(const void* w, int64_t bytes, int64_t need) {
    return w && reinterpret_cast<uintptr_t>(w) % 256 == 0 && bytes >= need;
}
void set_rows(Shape& S, Again& again, void* workspace, const Layout& L, cudaStream_t s) {
    char* base = static_cast<char*>(workspace);
    S.start = reinterpret_cast<int32_t*>(base);
    S.end = reinterpret_cast<int32_t*>(base + rows_bytes(S.tokens));
    S.words = reinterpret_cast<uint32_t*>(base + L.words);
    again = {S.words + kAgainCount, reinterpret_cast<int4*>(base + L.again)};
    const int64_t n = std::max(S.tokens, S.sequences + 1);
    launch(attention_rows_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((n + 255) / 256, 1 << 16))), dim3(256), 0, s, S);
}

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static PFN_cuTensorMapEncodeTiled_v12000 encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            fn = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    return encode;
}

}  // namespace

int sm_count() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 152;
    return sms;
}

// [tokens][heads][dim] in boxes of 64 values of 128 tokens of one head; what is outside reads as zeros.
bool tile_map(CUtensorMap* map, const Heads& h, int64_t tokens, int32_t heads, int32_t dim, int32_t dtype) {
    if (!tensor_map_encoder()) return false;
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(heads > 1 ? h.head : dim) * 2,
                                   static_cast<cuuint64_t>(tokens > 1 ? h.token : dim) * 2};
    const cuuint32_t box[3] = {64, 1, kTile};
    const cuuint32_t step[3] = {1, 1, 1};
    return tensor_map_encoder()(map, dtype == CB_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                                const_cast<void*>(h.data), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows that TMA can copy: 16-byte addresses and strides, no two rows in one place.
bool tensor_core_rows(const Shape& S, const Heads& h, int heads) {
    return S.dtype != CB_F32 && S.dim % 8 == 0 && S.dim <= 128 && reinterpret_cast<uintptr_t>(h.data) % 16 == 0 &&
           (S.tokens <= 1 || (h.token % 8 == 0 && h.token >= S.dim && h.token < kMostTmaStride)) &&
           (heads <= 1 || (h.head % 8 == 0 && h.head >= S.dim && h.head < kMostTmaStride));
}

}  // namespace attention
}  // namespace cbtbe

extern "C" int64_t cb_attention_workspace_bytes(int64_t tokens, int32_t heads, int32_t kv_heads, int32_t dim, int64_t window,
                                                int64_t sinks, int backward) {
    using namespace cbtbe::attention;
    if (tokens <= 0 || tokens > kMostTokens || heads < 1 || heads > 65535 || kv_heads < 1 || dim < 1 || dim > kMaxDim ||
        window < 1 || sinks < 0)
        return 0;
    return static_cast<int64_t>(layout(tokens, heads, kv_heads, dim, window, sinks, backward != 0).bytes);
}

extern "C" cb_status cb_attention_forward(const void* q, const void* k, const void* v, cb_dtype dtype, int64_t tokens,
                                          int32_t heads, int32_t kv_heads, int32_t dim, int64_t q_token_stride,
                                          int64_t q_head_stride, int64_t k_token_stride, int64_t k_head_stride,
                                          int64_t v_token_stride, int64_t v_head_stride, const void* offsets,
                                          cb_index_dtype idx_dtype, int64_t sequences, int64_t window, int64_t sinks,
                                          float scale, void* out, int64_t out_token_stride, int64_t out_head_stride, float* lse,
                                          void* workspace, int64_t workspace_bytes, int* error, cudaStream_t stream) {
    using namespace cbtbe::attention;
    Forward F{};
    F.S = shape(dtype, tokens, heads, kv_heads, dim, offsets, idx_dtype, sequences, window, sinks, scale, error);
    if (sizes_ok(F.S) != CB_OK) return CB_ERR_INVALID_ARG;
    if (tokens == 0) return CB_OK;
    F.q = {q, q_token_stride, q_head_stride};
    F.k = {k, k_token_stride, k_head_stride};
    F.v = {v, v_token_stride, v_head_stride};
    F.out = {out, out_token_stride, out_head_stride};
    F.lse = lse;
    if (!heads_ok(F.S, F.q, heads, false) || !heads_ok(F.S, F.k, kv_heads, false) || !heads_ok(F.S, F.v, kv_heads, false) ||
        !heads_ok(F.S, F.out, heads, true) || reinterpret_cast<uintptr_t>(lse) % 4)
        return CB_ERR_INVALID_ARG;
    const int64_t need = cb_attention_workspace_bytes(tokens, heads, kv_heads, dim, window, sinks, 0);
    if (!workspace_ok(workspace, workspace_bytes, need)) return CB_ERR_CAPACITY;
    if (cbtbe::overlap({span(F.S, F.out, heads), {lse, 4 * tokens * heads}, {workspace, need}, {error, 4}},
                       {span(F.S, F.q, heads), span(F.S, F.k, kv_heads), span(F.S, F.v, kv_heads), offsets_span(F.S)}))
        return CB_ERR_INVALID_ARG;
    set_rows(F.S, F.again, workspace, layout(tokens, heads, kv_heads, dim, window, sinks, false), stream);
    bool ok = true;
    if (tensor_core_rows(F.S, F.q, heads) && tensor_core_rows(F.S, F.k, kv_heads) && tensor_core_rows(F.S, F.v, kv_heads) &&
        tensor_core_rows(F.S, F.out, heads))
        ok = launch_forward(F, stream);
    else if (dtype == CB_F32) launch_forward_rowwise<CB_F32>(F, stream);
    else if (dtype == CB_F16) launch_forward_rowwise<CB_F16>(F, stream);
    else launch_forward_rowwise<CB_BF16>(F, stream);
    return cudaGetLastError() == cudaSuccess && ok ? CB_OK : CB_ERR_CUDA;
}

extern "C" cb_status cb_attention_backward(const void* grad_out, const void* q, const void* k, const void* v, const void* out,
                                           const float* lse, cb_dtype dtype, int64_t tokens, int32_t heads, int32_t kv_heads,
                                           int32_t dim, int64_t go_token_stride, int64_t go_head_stride, int64_t q_token_stride,
                                           int64_t q_head_stride, int64_t k_token_stride, int64_t k_head_stride,
                                           int64_t v_token_stride, int64_t v_head_stride, int64_t out_token_stride,
                                           int64_t out_head_stride, const void* offsets, cb_index_dtype idx_dtype,
                                           int64_t sequences, int64_t window, int64_t sinks, float scale, void* grad_q,
                                           void* grad_k, void* grad_v, int64_t dq_token_stride, int64_t dq_head_stride,
                                           int64_t dk_token_stride, int64_t dk_head_stride, int64_t dv_token_stride,
                                           int64_t dv_head_stride, void* workspace, int64_t workspace_bytes, int* error,
                                           cudaStream_t stream) {
    using namespace cbtbe::attention;
    Backward B{};
    B.S = shape(dtype, tokens, heads, kv_heads, dim, offsets, idx_dtype, sequences, window, sinks, scale, error);
    if (sizes_ok(B.S) != CB_OK) return CB_ERR_INVALID_ARG;
    if (tokens == 0) return CB_OK;
    B.go = {grad_out, go_token_stride, go_head_stride};
    B.q = {q, q_token_stride, q_head_stride};
    B.k = {k, k_token_stride, k_head_stride};
    B.v = {v, v_token_stride, v_head_stride};
    B.out = {out, out_token_stride, out_head_stride};
    B.dq = {grad_q, dq_token_stride, dq_head_stride};
    B.dk = {grad_k, dk_token_stride, dk_head_stride};
    B.dv = {grad_v, dv_token_stride, dv_head_stride};
    B.lse = lse;
    if (!heads_ok(B.S, B.go, heads, false) || !heads_ok(B.S, B.q, heads, false) || !heads_ok(B.S, B.k, kv_heads, false) ||
        !heads_ok(B.S, B.v, kv_heads, false) || !heads_ok(B.S, B.out, heads, false) || !heads_ok(B.S, B.dq, heads, true) ||
        !heads_ok(B.S, B.dk, kv_heads, true) || !heads_ok(B.S, B.dv, kv_heads, true) || !lse ||
        reinterpret_cast<uintptr_t>(lse) % 4)
        return CB_ERR_INVALID_ARG;
    const int64_t need = cb_attention_workspace_bytes(tokens, heads, kv_heads, dim, window, sinks, 1);
    if (!workspace_ok(workspace, workspace_bytes, need)) return CB_ERR_CAPACITY;
    if (cbtbe::overlap({span(B.S, B.dq, heads), span(B.S, B.dk, kv_heads), span(B.S, B.dv, kv_heads), {workspace, need}, {error, 4}},
                       {span(B.S, B.go, heads), span(B.S, B.q, heads), span(B.S, B.k, kv_heads), span(B.S, B.v, kv_heads),
                        span(B.S, B.out, heads), {lse, 4 * tokens * heads}, offsets_span(B.S)}))
        return CB_ERR_INVALID_ARG;
    const Layout L = layout(tokens, heads, kv_heads, dim, window, sinks, true);
    char* base = static_cast<char*>(workspace);
    B.delta = reinterpret_cast<float*>(base + L.delta);
    B.largest = reinterpret_cast<uint8_t*>(base + L.largest);
    B.padded = static_cast<int64_t>(tiles_of(static_cast<int>(tokens))) * kTile;
    set_rows(B.S, B.again, workspace, L, stream);
    B.order = {reinterpret_cast<int32_t*>(B.S.words + kOrderParts), B.S.words + kOrderNext, B.S.words + kOrderDone,
               static_cast<int32_t>(L.room), part_blocks(tokens, heads, kv_heads, window), reinterpret_cast<int2*>(base + L.list),
               reinterpret_cast<int32_t*>(base + L.split), reinterpret_cast<float*>(base + L.sums)};
    bool ok = true;
    bool fast = true;
    for (const Heads* x : {&B.go, &B.q, &B.out, &B.dq}) fast = fast && tensor_core_rows(B.S, *x, heads);
    for (const Heads* x : {&B.k, &B.v, &B.dk, &B.dv}) fast = fast && tensor_core_rows(B.S, *x, kv_heads);
    if (fast) ok = launch_backward(B, stream);
    else if (dtype == CB_F32) launch_backward_rowwise<CB_F32>(B, stream);
    else if (dtype == CB_F16) launch_backward_rowwise<CB_F16>(B, stream);
    else launch_backward_rowwise<CB_BF16>(B, stream);
    return cudaGetLastError() == cudaSuccess && ok ? CB_OK : CB_ERR_CUDA;
}
