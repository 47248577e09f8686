// linear_gemm_gelu_tanh.hip -- linear_gemm.hpp with activation gelu_tanh.
#define FBL_ACT 3
#include "linear_gemm.hpp"
