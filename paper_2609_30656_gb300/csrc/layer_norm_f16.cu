// layer_norm_f16.cu -- layer normalisation of rows read in f16.
#include "layer_norm.cuh"

namespace cbtbe {
namespace norm {

void launch_f16(const Args& A, const Shape& S, bool back, cudaStream_t s) {
    if (A.out_dtype == CB_F32) back ? launch_typed<CB_F16, CB_F32, true>(A, S, s) : launch_typed<CB_F16, CB_F32, false>(A, S, s);
    if (A.out_dtype == CB_F16) back ? launch_typed<CB_F16, CB_F16, true>(A, S, s) : launch_typed<CB_F16, CB_F16, false>(A, S, s);
}

}  // namespace norm
}  // namespace cbtbe
