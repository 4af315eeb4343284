#include "decode_attention.cuh"

namespace strassen {
namespace decode {

cudaError_t launch_f16(const Args &p, int dp, int nt, int sm_count, cudaStream_t stream)
{
    if (dp == 64) return nt == 1 ? launch<F16, 64, 1>(p, sm_count, stream) : launch<F16, 64, 2>(p, sm_count, stream);
    return nt == 1 ? launch<F16, 128, 1>(p, sm_count, stream) : launch<F16, 128, 2>(p, sm_count, stream);
}

int ranks_f16(const AttentionArgs &a, int dp, int nt, int64_t heads, int sm_count)
{
    if (dp == 64) return nt == 1 ? ranks_for<F16, 64, 1>(a, heads, sm_count) : ranks_for<F16, 64, 2>(a, heads, sm_count);
    return nt == 1 ? ranks_for<F16, 128, 1>(a, heads, sm_count) : ranks_for<F16, 128, 2>(a, heads, sm_count);
}

}  // namespace decode
}  // namespace strassen
