// gated_gemm_relu.hip -- gated_gemm.hpp with activation relu.
#define FBL_ACT 1
#include "gated_gemm.hpp"
