// window_attention_again.cu -- rows of windowed attention whose result the tensor-core kernels found not finite
// (include/cb_tbe.h), computed again in fp32.
//
// Their tiles multiply what a row does not see by zeros, which infinities and NaNs behind the mask survive; rows that do see some
// come here too. A block takes a row, its warps its keys (of dK and dV the tokens that see it) four at a time, joined in one
// order: the same bits every time. A note is 32 neighbouring rows, which go to as many blocks. Nothing else waits
// for these rows: within the tensor-core kernels they kept the other warps of a block waiting, whose waits have a limit,
// so that a long session's ended them early. Latency bounds it, hence four at once. Where nothing is noted a call takes as long as
// without it (its launch overlaps).
#include "window_attention.cuh"

namespace cbtbe {
namespace attention {
namespace {

constexpr int kWarps = 8, kAtOnce = 4, kStep = kWarps * kAtOnce;
constexpr int kMostDim = 128, kValues = kMostDim / 32;  // of rows that the tensor cores take; of a lane

struct Sums {  // of the block's warps
    float value[2][kWarps][kMostDim], most[kWarps], sum[kWarps];
    int stop;  // a warp's sums have all become NaNs, and so have the row's, whatever the others find
};

// The n-th row noted: its token and head; which result, or -1 for none.
__device__ __forceinline__ int row_noted(const Again& A, int64_t n, uint32_t count, int64_t& token, int& head) {
    const int4 note = A.list[n % count];
    const int bit = static_cast<int>(n / count);
    token = note.x + bit;
    head = note.y;
    return static_cast<uint32_t>(note.z) >> bit & 1 ? note.w : -1;
}

template <int DT>
__device__ __forceinline__ void load(const Heads& h, int64_t token, int head, int dim, float (&v)[kValues]) {
    const uint16_t* row = static_cast<const uint16_t*>(h.data) + token * h.token + head * h.head;
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
        const int c = (threadIdx.x & 31) + 32 * i;
        v[i] = c < dim ? widen<DT>(row[c]) : 0.f;
    }
}
template <int DT>
__device__ __forceinline__ void store_value(const Heads& h, int64_t token, int head, float v) {
    static_cast<uint16_t*>(const_cast<void*>(h.data))[token * h.token + head * h.head + threadIdx.x] =
        static_cast<uint16_t>(narrow<DT>(v));
}
// Products of a row with four others.
__device__ __forceinline__ void dots(const float (&a)[kValues], const float (&b)[kAtOnce][kValues], float (&s)[kAtOnce]) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
        s[u] = 0.f;
#pragma unroll
        for (int i = 0; i < kValues; ++i) s[u] = fmaf(a[i], b[u][i], s[u]);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) s[u] = warp_sum(s[u]);
}
__device__ __forceinline__ void add(float (&a)[kValues], float f, const float (&b)[kValues]) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) a[i] = fmaf(f, b[i], a[i]);
}
__device__ __forceinline__ void put(float (&to)[kMostDim], const float (&v)[kValues]) {
#pragma unroll
    for (int i = 0; i < kValues; ++i) to[(threadIdx.x & 31) + 32 * i] = v[i];
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
    const Shape& S = F.S;
    const uint32_t count = *F.again.count;
    const int warp = threadIdx.x / 32;
    volatile int* stop = &shared.stop;
    for (int64_t n = blockIdx.x; n < int64_t{32} * count; n += gridDim.x) {
        int64_t t;
        int h;
        if (row_noted(F.again, n, count, t, h) < 0) continue;
        if (threadIdx.x == 0) shared.stop = 0;
        __syncthreads();
        const Seen a = seen_by(S, t);
        const int kv = h / S.group;
        float q[kValues], o[kValues] = {}, most = -INFINITY, sum = 0.f;
        load<DT>(F.q, t, h, S.dim, q);
        for (int64_t i = warp * kAtOnce; i < a.n && !*stop; i += kStep) {
            float k[kAtOnce][kValues], v[kAtOnce][kValues], s[kAtOnce];
            const int some = static_cast<int>(min64(a.n - i, kAtOnce));
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int64_t j = a.at(u < some ? i + u : i);
                load<DT>(F.k, j, kv, S.dim, k[u]);
                load<DT>(F.v, j, kv, S.dim, v[u]);
            }
            dots(q, k, s);
            float top = most;
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                s[u] *= S.scale * kLog2e;
                top = fmaxf(top, s[u]);  // the first again where there are fewer
            }
            const float keep = most == top ? 1.f : exp2f(most - top);
            sum *= keep;
#pragma unroll
            for (int x = 0; x < kValues; ++x) o[x] *= keep;
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (u >= some) continue;
                const float p = s[u] == -INFINITY ? 0.f : exp2f(s[u] - top);
                sum += p;
                add(o, p, v[u]);
            }
            most = top;
            if (sum != sum) *stop = 1;
        }
        put(shared.value[0][warp], o);
        shared.most[warp] = most;
        shared.sum[warp] = sum;
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < S.dim) {
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
__device__ __forceinline__ void dq_again(const Backward& B, int64_t t, int h, int warp, float (&dq)[kValues], volatile int* stop) {
    const Shape& S = B.S;
    const Seen a = seen_by(S, t);
    const int kv = h / S.group;
    float q[kValues], go[kValues];
    load<DT>(B.q, t, h, S.dim, q);
    load<DT>(B.go, t, h, S.dim, go);
    const float lse = B.lse[h * S.tokens + t], delta = B.delta[h * S.tokens + t];
    for (int64_t i = warp * kAtOnce; i < a.n && !*stop; i += kStep) {
        float k[kAtOnce][kValues], v[kAtOnce][kValues], s[kAtOnce], d[kAtOnce];
        const int some = static_cast<int>(min64(a.n - i, kAtOnce));
        bool nan = false;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t j = a.at(u < some ? i + u : i);
            load<DT>(B.k, j, kv, S.dim, k[u]);
            load<DT>(B.v, j, kv, S.dim, v[u]);
        }
        dots(q, k, s);
        dots(go, v, d);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (u >= some) continue;
            const float slope = exp2f((s[u] * S.scale - lse) * kLog2e) * (d[u] - delta) * S.scale;
            add(dq, slope, k[u]);
            nan = nan || slope != slope;
        }
        if (nan) *stop = 1;
    }
}

// dK, dV or both of head kv of key j, over the heads that share it and the tokens that see it.
template <int DT, bool KEYS, bool VALUES>
__device__ __forceinline__ void dkv_again(const Backward& B, int64_t j, int kv, int warp, float (&dk)[kValues],
                                          float (&dv)[kValues], volatile int* stop) {
    const Shape& S = B.S;
    const int64_t seeing = seen_to(S, j) - j, all = seeing * S.group;  // of a head; of all that share it, one after the other
    float k[kValues], v[kValues];
    load<DT>(B.k, j, kv, S.dim, k);
    load<DT>(B.v, j, kv, S.dim, v);
    for (int64_t i = warp * kAtOnce; i < all && !*stop; i += kStep) {
        float q[kAtOnce][kValues], go[kAtOnce][kValues], s[kAtOnce], d[kAtOnce], lse[kAtOnce], delta[kAtOnce];
        const int some = static_cast<int>(min64(all - i, kAtOnce));
        const int64_t head = i / seeing;
        bool nan = false;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            int h = kv * S.group + static_cast<int>(head);
            int64_t t = j + (i - head * seeing) + (u < some ? u : 0);
            for (; t >= j + seeing; t -= seeing) ++h;
            load<DT>(B.q, t, h, S.dim, q[u]);
            load<DT>(B.go, t, h, S.dim, go[u]);
            lse[u] = B.lse[h * S.tokens + t];
            delta[u] = B.delta[h * S.tokens + t];
        }
        dots(k, q, s);
        if constexpr (KEYS) dots(v, go, d);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (u >= some) continue;
            const float p = exp2f((s[u] * S.scale - lse[u]) * kLog2e);
            float slope = p;
            if constexpr (VALUES) add(dv, p, go[u]);
            if constexpr (KEYS) {
                slope = p * (d[u] - delta[u]) * S.scale;
                add(dk, slope, q[u]);
            }
            nan = nan || (VALUES ? p != p : slope != slope);
        }
        if (nan) *stop = 1;
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
        const bool values = which == kDv || which == kDkAndDv;
        if (threadIdx.x == 0) shared.stop = 0;
        __syncthreads();
        float a[kValues] = {}, b[kValues] = {};  // dQ or dK, and dV
        if (which == kDq) dq_again<DT>(B, t, h, warp, a, &shared.stop);
        else if (which == kDk) dkv_again<DT, true, false>(B, t, h, warp, a, b, &shared.stop);
        else if (which == kDv) dkv_again<DT, false, true>(B, t, h, warp, a, b, &shared.stop);
        else dkv_again<DT, true, true>(B, t, h, warp, a, b, &shared.stop);
        put(shared.value[0][warp], a);
        put(shared.value[1][warp], b);
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < B.S.dim) {
            if (which != kDv) store_value<DT>(which == kDq ? B.dq : B.dk, t, h, joined(shared.value[0]));
            if (values) store_value<DT>(B.dv, t, h, joined(shared.value[1]));
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
