#include "decode_attention.cuh"

namespace strassen {
namespace decode {

cudaError_t launch_f16(const Args &p, int dp, int nt, int sm_count, cudaStream_t stream)
{
    if (dp == 64) return nt == 1 ? launch<F16, 64, 1>(p, sm_count, stream) : launch<F16, 64, 2>(p, sm_count, stream);
    return nt == 1 ? launch<F16, 128, 1>(p, sm_count, stream) : launch<F16, 128, 2>(p, sm_count, stream);
}

}  // namespace decode
}  // namespace strassen
