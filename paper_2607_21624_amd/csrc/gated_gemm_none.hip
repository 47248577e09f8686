// gated_gemm_none.hip -- gated_gemm.hpp with activation none.
#define FBL_ACT 0
#include "gated_gemm.hpp"
