// linear_gemm_none.hip -- linear_gemm.hpp with activation none.
#define FBL_ACT 0
#include "linear_gemm.hpp"
