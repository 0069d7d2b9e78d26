// Layer norm of f32 rows.
#include "norm.cuh"

template cudaError_t esspt::launch_norm<float>(Norm&, bool, int, int, unsigned*, cudaStream_t);
