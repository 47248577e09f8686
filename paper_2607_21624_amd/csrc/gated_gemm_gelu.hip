// gated_gemm_gelu.hip -- gated_gemm.hpp with activation gelu.
#define FBL_ACT 2
#include "gated_gemm.hpp"
