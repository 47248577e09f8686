// linear_gemm_gelu.hip -- linear_gemm.hpp with activation gelu.
#define FBL_ACT 2
#include "linear_gemm.hpp"
