// wait_probe.cu -- a bounded wait on a barrier that nothing arrives on, and the last product of
// an orthogonalised update after an earlier one has reported such a wait, for test_wait_limits_gpu.py.
#include "muon_internal.cuh"

namespace {

// No copies and no products are in flight: the wait can only be answered by the arrival below.
__global__ void wait_kernel(int arrive, uint32_t polls, int* complete, int* error) {
    __shared__ uint64_t bar;
    using namespace cbtbe;
    const uint32_t at = tc::smem_addr(&bar);
    if (threadIdx.x == 0) {
        tc::barrier_init(at, 1);
        tc::barrier_init_fence();
    }
    __syncthreads();
    if (threadIdx.x == 0 && arrive) tc::barrier_arrive(at);
    const bool ok = __all_sync(kFull, tc::barrier_wait(at, 0, polls));
    if (threadIdx.x == 0) *complete = ok;
    if (!ok && threadIdx.x == 0) set_error(error, CB_ERR_TIMEOUT);
}

}  // namespace

extern "C" int probe_wait(int arrive, uint32_t polls, int* complete, int* error, cudaStream_t s) {
    wait_kernel<<<1, 32, 0, s>>>(arrive, polls, complete, error);
    return cudaGetLastError() == cudaSuccess ? 0 : 1;
}

// weights <- keep weights - rate ((poly hi / 2^8 + (a - shift) hi + a lo) / 2^10), unless *fault.
extern "C" int probe_result(const __half* poly, const __half* hi, const __half* lo, float* weights, int* fault, int batch,
                            int p, int q, int lda, int ldx, float a, float shift, float keep, float rate, cudaStream_t s) {
    using namespace cbtbe::muon;
    Operand left, right;
    if (!tensor_maps_work() || !left.set(poly, p, p, batch, lda) || !right.set(hi, q, p, batch, ldx)) return 1;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 1;
    ProductArgs P{};
    P.batch = batch;
    P.m = P.k = p;
    P.n = q;
    P.a = a;
    P.shift = shift;
    P.term_hi = hi;
    P.term_lo = lo;
    P.term_batch = static_cast<int64_t>(p) * ldx;
    P.term_ld = ldx;
    P.user = weights;
    P.user_batch = static_cast<int64_t>(p) * q;
    P.user_row = q;
    P.user_dtype = CB_F32;
    P.weights = 1;
    P.keep = keep;
    P.rate = rate;
    P.fault = fault;
    return launch_product(kResult, left, right, P, sms, s) && cudaGetLastError() == cudaSuccess ? 0 : 1;
}
