// The one-pass backward kernel of the norms around a block for bf16, by the types of the gradients that come in and leave.
#include "vp_block_norm.h"

namespace vp {

hipError_t launch_bwd_one_pass_bf16(const BlockNormGrad& p, vp_dtype dH_dt, vp_dtype grad_dt, const ColumnSums& s, hipStream_t st) {
    if (dH_dt == VP_F32)
        return grad_dt == VP_F32 ? launch_bwd_one_pass<u16, float, float>(p, s, st) : launch_bwd_one_pass<u16, float, u16>(p, s, st);
    return grad_dt == VP_F32 ? launch_bwd_one_pass<u16, u16, float>(p, s, st) : launch_bwd_one_pass<u16, u16, u16>(p, s, st);
}

}  // namespace vp
