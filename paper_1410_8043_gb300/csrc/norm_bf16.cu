// Layer norm of bf16 rows.
#include "norm.cuh"

template cudaError_t esspt::launch_norm<__nv_bfloat16>(Norm&, bool, int, int, unsigned*, cudaStream_t);
