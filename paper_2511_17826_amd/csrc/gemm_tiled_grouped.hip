// The kernels of gemm_tiled.hip for products grouped by expert, in a translation unit of their own.
#define TBIK_GROUPED_UNIT
#include "gemm_tiled.hip"
