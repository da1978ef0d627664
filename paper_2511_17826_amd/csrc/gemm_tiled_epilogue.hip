// The kernels of gemm_tiled.hip with an epilogue, in a translation unit of their own: they take as long to compile as all others.
#define TBIK_EPILOGUE_UNIT
#include "gemm_tiled.hip"
