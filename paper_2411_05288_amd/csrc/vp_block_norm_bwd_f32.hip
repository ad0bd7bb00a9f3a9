// The one-pass backward kernel of the norms around a block for fp32.
#include "vp_block_norm.h"

namespace vp {

hipError_t launch_bwd_one_pass_f32(const BlockNormGrad& p, const ColumnSums& s, hipStream_t st) {
    return launch_bwd_one_pass<float, float, float>(p, s, st);
}

}  // namespace vp
