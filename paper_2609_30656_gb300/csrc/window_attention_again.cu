// window_attention_again.cu -- rows of windowed attention whose result the tensor-core kernels found not finite
// (include/cb_tbe.h), computed again key by key in fp32.
//
// A block for a row, its warps every eighth key, joined in order: the same bits every time. The notes of a warp are 32
// neighbouring rows, which go to as many blocks. Nothing else waits for these rows: within the tensor-core kernels they kept the
// other warps of a block waiting, whose waits have a limit, so that a long session's would have ended them early. Where
// nothing is noted a call takes 1 to 2 us more.
#include "window_attention.cuh"

namespace cbtbe {
namespace attention {
namespace {

constexpr int kWarps = 8, kMostDim = 128;  // of rows that the tensor cores take

struct Sums {  // of the block's warps
    float value[2][kWarps][kMostDim], most[kWarps], sum[kWarps];
    int stop;
};

// The n-th row noted: its token and head; which result, or -1 for none.
__device__ __forceinline__ int row_noted(const Again& A, int64_t n, uint32_t count, int64_t& token, int& head) {
    const int4 note = A.list[n % count];
    const int bit = static_cast<int>(n / count);
    token = note.x + bit;
    head = note.y;
    return static_cast<uint32_t>(note.z) >> bit & 1 ? note.w : -1;
}
__device__ __forceinline__ void put(float (&to)[kMostDim], const float (&v)[kLaneValues]) {
#pragma unroll
    for (int i = 0; i < kMostDim / 32; ++i) to[(threadIdx.x & 31) + 32 * i] = v[i];
}
template <int DT>
__device__ __forceinline__ void store_value(const Heads& h, int64_t token, int head, float v) {
    static_cast<uint16_t*>(const_cast<void*>(h.data))[token * h.token + head * h.head + threadIdx.x] =
        static_cast<uint16_t>(narrow<DT>(v));
}
__device__ __forceinline__ float joined(const float (&value)[kWarps][kMostDim]) {
    float sum = 0.f;
    for (int w = 0; w < kWarps; ++w) sum += value[w][threadIdx.x];
    return sum;
}

template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_output_again_kernel(const Forward F) {
    __shared__ Sums shared;
    begin_kernel();
    const uint32_t count = *F.again.count;
    const int warp = threadIdx.x / 32;
    for (int64_t n = blockIdx.x; n < int64_t{32} * count; n += gridDim.x) {
        int64_t t;
        int h;
        if (row_noted(F.again, n, count, t, h) < 0) continue;
        if (threadIdx.x == 0) shared.stop = 0;
        __syncthreads();
        float o[kLaneValues], most, sum;
        row_output<DT>(F, t, h, warp, kWarps, o, most, sum, &shared.stop);
        put(shared.value[0][warp], o);
        shared.most[warp] = most;
        shared.sum[warp] = sum;
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < F.S.dim) {
            float top = -INFINITY, total = 0.f, value = 0.f;
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, shared.most[w]);
            for (int w = 0; w < kWarps; ++w) {
                const float f = shared.most[w] == top ? 1.f : exp2f(shared.most[w] - top);  // 0 where the warp had no key
                total = fmaf(shared.sum[w], f, total);
                value = fmaf(shared.value[0][w][threadIdx.x], f, value);
            }
            store_value<DT>(F.out, t, h, value / total);
        }
        __syncthreads();
    }
}

template <int DT>
__global__ void __launch_bounds__(kWarps * 32) attention_gradients_again_kernel(const Backward B) {
    __shared__ Sums shared;
    begin_kernel();
    const uint32_t count = *B.again.count;
    const int warp = threadIdx.x / 32;
    for (int64_t n = blockIdx.x; n < int64_t{32} * count; n += gridDim.x) {
        int64_t t;
        int h;
        const int which = row_noted(B.again, n, count, t, h);
        if (which < 0) continue;
        if (threadIdx.x == 0) shared.stop = 0;
        __syncthreads();
        float a[kLaneValues], b[kLaneValues];  // dQ or dK, and dV
        if (which == kDq) row_dq<DT>(B, t, h, warp, kWarps, a, &shared.stop);
        else if (which == kDk) row_dkv<DT, true, false>(B, t, h, warp, kWarps, a, b, &shared.stop);
        else if (which == kDv) row_dkv<DT, false, true>(B, t, h, warp, kWarps, a, b, &shared.stop);
        else row_dkv<DT, true, true>(B, t, h, warp, kWarps, a, b, &shared.stop);
        if (which != kDv) put(shared.value[0][warp], a);
        if (which == kDv || which == kDkAndDv) put(shared.value[1][warp], b);
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < B.S.dim) {
            if (which != kDv) store_value<DT>(which == kDq ? B.dq : B.dk, t, h, joined(shared.value[0]));
            if (which == kDv || which == kDkAndDv) store_value<DT>(B.dv, t, h, joined(shared.value[1]));
        }
        __syncthreads();
    }
}

dim3 grid() { return dim3(static_cast<unsigned>(3 * sm_count())); }

}  // namespace

void launch_again(const Forward& F, cudaStream_t s) {
    launch(F.S.dtype == CB_BF16 ? attention_output_again_kernel<CB_BF16> : attention_output_again_kernel<CB_F16>, grid(),
           dim3(kWarps * 32), 0, s, F);
}
void launch_again(const Backward& B, cudaStream_t s) {
    launch(B.S.dtype == CB_BF16 ? attention_gradients_again_kernel<CB_BF16> : attention_gradients_again_kernel<CB_F16>, grid(),
           dim3(kWarps * 32), 0, s, B);
}

}  // namespace attention
}  // namespace cbtbe
