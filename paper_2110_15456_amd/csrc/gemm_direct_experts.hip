// gemm_direct_experts.hip -- the few-output products of experts (gemm_direct.h,
// SEG), groups of 16, every operand format.
#include "gemm_direct.h"

namespace fastbfp {

FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_INSTANTIATE, 1, 1)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_INSTANTIATE, 1, 2)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_INSTANTIATE, 2, 1)
FASTBFP_DIRECT_EXPERTS_ALL(FASTBFP_DIRECT_EXPERTS_INSTANTIATE, 2, 2)

}  // namespace fastbfp
