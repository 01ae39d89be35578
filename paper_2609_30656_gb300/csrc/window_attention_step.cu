// window_attention_step.cu -- windowed attention of one new token for each session over a cache of keys
// and values (include/cb_tbe.h).
#include "window_attention.cuh"

#include <algorithm>
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
            const float top = fmaxf(most, s), keep = most == top ? 1.f : exp2f(most - top), p = exp2f(s - top);
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

bool type_ok(int t) { return t == CB_F32 || t == CB_F16 || t == CB_BF16; }
constexpr int64_t kMost = int64_t{1} << 40;
bool stride_ok(int64_t s) { return s >= 0 && s <= kMost; }

}  // namespace
}  // namespace attention
}  // namespace cbtbe

extern "C" int64_t cb_attention_step_workspace_bytes(int64_t sequences, int32_t heads, int32_t kv_heads, int32_t dim,
                                                     int64_t capacity, int64_t window, int64_t sinks) {
    return 0;
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
    if (!type_ok(dtype) || sequences < 0 || sequences >= (int64_t{1} << 31) || capacity < 0 || capacity >= (int64_t{1} << 31) ||
        heads < 1 || heads > 65535 || kv_heads < 1 || heads % kv_heads || dim < 1 || dim > kMaxDim || window < 1 || sinks < 0 ||
        !(scale == scale) || (idx_dtype != CB_I32 && idx_dtype != CB_I64) || reinterpret_cast<uintptr_t>(error) % 4)
        return CB_ERR_INVALID_ARG;
    for (const int64_t s : {q_sequence_stride, q_head_stride, k_sequence_stride, k_token_stride, k_head_stride,
                            v_sequence_stride, v_token_stride, v_head_stride, out_sequence_stride, out_head_stride})
        if (!stride_ok(s)) return CB_ERR_INVALID_ARG;
    if (!cbtbe::rows_apart(sequences, out_sequence_stride, heads, out_head_stride, dim)) return CB_ERR_INVALID_ARG;
    if (sequences == 0) return CB_OK;
    const uintptr_t mask = dtype == CB_F32 ? 3 : 1;
    if (!q || !out || !lengths || (capacity > 0 && (!k_cache || !v_cache)) || (reinterpret_cast<uintptr_t>(q) & mask) ||
        (reinterpret_cast<uintptr_t>(k_cache) & mask) || (reinterpret_cast<uintptr_t>(v_cache) & mask) ||
        (reinterpret_cast<uintptr_t>(out) & mask) || reinterpret_cast<uintptr_t>(lengths) % (idx_dtype == CB_I32 ? 4 : 8))
        return CB_ERR_INVALID_ARG;
    const int64_t need = cb_attention_step_workspace_bytes(sequences, heads, kv_heads, dim, capacity, window, sinks);
    if (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 || workspace_bytes < need)) return CB_ERR_CAPACITY;
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
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(sequences * heads, 1 << 20)));
    if (dtype == CB_F32) cbtbe::launch(attention_step_rowwise_kernel<CB_F32>, grid, dim3(kWarps * 32), 0, stream, A);
    else if (dtype == CB_F16) cbtbe::launch(attention_step_rowwise_kernel<CB_F16>, grid, dim3(kWarps * 32), 0, stream, A);
    else cbtbe::launch(attention_step_rowwise_kernel<CB_BF16>, grid, dim3(kWarps * 32), 0, stream, A);
    return cudaGetLastError() == cudaSuccess ? CB_OK : CB_ERR_CUDA;
}
