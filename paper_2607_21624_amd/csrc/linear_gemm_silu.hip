// linear_gemm_silu.hip -- linear_gemm.hpp with activation silu.
#define FBL_ACT 4
#include "linear_gemm.hpp"
