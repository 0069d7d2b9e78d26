// Layer norm of f16 rows.
#include "norm.cuh"

template cudaError_t esspt::launch_norm<__half>(Norm&, bool, int, int, unsigned*, cudaStream_t);
