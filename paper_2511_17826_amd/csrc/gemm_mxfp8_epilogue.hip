// The MXFP8 tiled kernels of gemm_fp8.hip with an epilogue, in a translation unit of their own (see there).
#define TBIK_EPILOGUE_UNIT 88
#include "gemm_fp8.hip"
