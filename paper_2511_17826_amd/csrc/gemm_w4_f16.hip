// The kernels of gemm_w4.hip for fp16, in a translation unit of their own.
#define TBIK_W4_F16_UNIT
#define TBIK_W4_F16 true
#include "gemm_w4.hip"
