// Products of a few rows with a matrix of 4-bit weights: kernels for f16 rows.
#include "w4_thin.cuh"

cudaError_t strassen::thin::launch_f16(const Ptrs &p, int group, bool zeros, int sm_count, cudaStream_t stream) { return launch_type<XF16>(p, group, zeros, sm_count, stream); }
