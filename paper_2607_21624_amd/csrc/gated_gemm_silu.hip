// gated_gemm_silu.hip -- gated_gemm.hpp with activation silu.
#define FBL_ACT 4
#include "gated_gemm.hpp"
