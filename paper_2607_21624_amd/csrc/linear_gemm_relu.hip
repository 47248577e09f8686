// linear_gemm_relu.hip -- linear_gemm.hpp with activation relu.
#define FBL_ACT 1
#include "linear_gemm.hpp"
