// gated_gemm_gelu_tanh.hip -- gated_gemm.hpp with activation gelu_tanh.
#define FBL_ACT 3
#include "gated_gemm.hpp"
