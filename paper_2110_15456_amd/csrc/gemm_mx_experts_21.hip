// gemm_mx_experts_21.hip -- the products of experts (gemm_mx.h, SEG) with 2 chunk
// plane(s) of A and 1 of B, groups of 16, every plane-0 format of either operand.
#include "gemm_mx.h"

namespace fastbfp {

FASTBFP_MX_EXPERTS_ALL(FASTBFP_MX_EXPERTS_INSTANTIATE, 2, 1)

}  // namespace fastbfp
