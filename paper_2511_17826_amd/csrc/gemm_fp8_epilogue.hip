// The 8-bit tiled kernels of gemm_fp8.hip with an epilogue, in a translation unit of their own (see there).
#define TBIK_EPILOGUE_UNIT 8
#include "gemm_fp8.hip"
