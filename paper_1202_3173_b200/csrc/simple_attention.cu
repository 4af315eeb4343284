// Attention over a paged cache: a warp for each head of each new token, a row of the cache after the other.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "attention.h"
#include "llm.h"

namespace strassen {

namespace {

__device__ __forceinline__ float value(const uint8_t *row, int i, int type)
{
    if (type == STRASSEN_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(row)[i]);
    if (type == STRASSEN_F16) return __half2float(reinterpret_cast<const __half *>(row)[i]);
    return float(reinterpret_cast<const __nv_fp8_e4m3 *>(row)[i]);
}

__global__ void __launch_bounds__(128) attention_kernel(const AttentionArgs p)
{
    after_work_before();
    const int64_t t = blockIdx.x;
    const int h = blockIdx.y * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31, d = p.cache.d;
    if (h >= p.heads) return;
    int b = int(t);
    if (p.seq.offsets) {
        b = -1;
        for (int i = 0; i < p.seq.batch; ++i) {
            const NewTokens n = new_tokens(p.seq, i);
            if (t >= n.first && t < n.end) b = i;
        }
        if (b < 0) return;
    }
    const NewTokens n = new_tokens(p.seq, b);
    const int64_t position = n.length - (n.end - t), most = int64_t(p.seq.width) << p.cache.page_shift;
    const int64_t end = position + 1 < most ? position + 1 : most, lo = p.window ? position + 1 - p.window : 0;
    const int kvh = h / (p.heads / p.cache.kv_heads);
    const uint8_t *q = static_cast<const uint8_t *>(p.q.p) + 2 * (t * p.q.row + h * p.q.head);
    // what 256 rows give is added up apart: a long sequence's many small weights would be lost one by one beside a large one
    float x[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f, big_o[4] = {0.f, 0.f, 0.f, 0.f}, big_l = 0.f;
    for (int i = 0; i < 4; ++i) x[i] = lane + 32 * i < d ? value(q, lane + 32 * i, p.type) * p.scale : 0.f;
    for (int64_t j = lo > 0 ? lo : 0; j < end; ++j) {
        if (j % 256 == 0) {
            big_l += l;
            l = 0.f;
            for (int i = 0; i < 4; ++i) {
                big_o[i] += o[i];
                o[i] = 0.f;
            }
        }
        const int page = page_of(p.cache, p.seq, b, j);
        const int64_t slot = j & ((1 << p.cache.page_shift) - 1);
        const int64_t at = page * p.cache.page_stride + kvh * p.cache.head_stride + slot * p.cache.row_stride;
        float ks = 1.f, vs = 1.f;
        if (page >= 0 && p.cache.type == STRASSEN_E4M3) {
            const int64_t scale = ((int64_t(page) * p.cache.kv_heads + kvh) << p.cache.page_shift) + slot;
            ks = p.cache.k_scale[scale];
            vs = p.cache.v_scale[scale];
        }
        float s = 0.f;
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < d && page >= 0) s += x[i] * value(p.cache.k + at, lane + 32 * i, p.cache.type);
        for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(~0u, s, i);
        s *= ks;
        const float next = fmaxf(m, s), back = m == next ? 1.f : expf(m - next), w = expf(s - next);
        l = l * back + w;
        big_l *= back;
        for (int i = 0; i < 4; ++i) big_o[i] *= back;
        for (int i = 0; i < 4; ++i) o[i] = o[i] * back + (lane + 32 * i < d && page >= 0 ? w * vs * value(p.cache.v + at, lane + 32 * i, p.cache.type) : 0.f);
        m = next;
    }
    uint16_t *out = static_cast<uint16_t *>(p.out) + t * p.out_row + h * p.out_head;
    for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < d) {
            const float y = l + big_l == 0.f ? 0.f : (o[i] + big_o[i]) / (l + big_l);
            out[lane + 32 * i] = p.type == STRASSEN_BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
        }
}

}  // namespace

cudaError_t launch_simple(const AttentionArgs &a, cudaStream_t stream)
{
    return launch_after(attention_kernel, dim3(unsigned(a.seq.tokens), unsigned((a.heads + 3) / 4)), dim3(128), 0, stream, dim3(1, 1), a);
}

}  // namespace strassen
