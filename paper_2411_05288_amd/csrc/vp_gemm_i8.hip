// The output layer's logits from 8-bit integers: the fast kernel (vp_gemm_bf16_fast.h) with integer products, whose operands of 16
// bytes hold 16 integers in place of 8 numbers; data movement, tiles and tile order are the same.
#include "vp_gemm_bf16_fast.h"

namespace vp {

hipError_t launch_gemm_i8(const GemmI8Group& g, hipStream_t st) {
    ProfScope prof(K_GEMM_I8, st);
    return launch_fast_t<true, true, Epi::LogitsI8>(g, st);
}

}  // namespace vp
