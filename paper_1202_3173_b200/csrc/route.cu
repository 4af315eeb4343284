// Routing of tokens to experts.
//
//   score_e = softmax(l)_e  or  1 / (1 + exp(-l_e));   key_e = score_e + bias_e   (softmax without a bias: l_e, whose order is the same)
//   groups of experts / groups neighbours: a group's rating is its largest key (softmax) or the sum of its two largest (sigmoid); only
//   the experts of the top_groups best groups stay;  ids: the `top` largest keys, in order;  weight = score [/ sum of the chosen scores] * factor
//
// Ties go to the lowest index, of groups and of experts.  Logits of -inf and NaN, and keys of -inf and NaN, are experts that are left out:
// they take no part in the softmax and are never chosen; where too few are left, ids end in -1 with weight 0.  Chosen scores that are all 0 (sigmoids
// of large negative numbers) stay 0 when they are renormalised.
//
// One warp a token, expert i * 32 + lane in register i.  Keys become unsigned numbers of the same order, so that the warp's largest is one
// reduction instruction and the lowest index among equals another.  A few kilobytes a token: bound by launch and latency
// (16384 tokens, 64 experts of which 8: 9.4 us, 3.1 MB; one token: the launch).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "llm.h"
#include "strassen_b200.h"

namespace strassen {

namespace {

constexpr int WARPS = 4;

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__half v) { return __half2float(v); }
__device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }

// An unsigned number of the same order, 0 for what is left out (-inf, NaN).  -0 and 0 are equal.
__device__ __forceinline__ uint32_t ordered(float v)
{
    if (!(v > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

template <class T, int V> __global__ void __launch_bounds__(WARPS * 32) route_kernel(const RouteArgs p)
{
    extern __shared__ float keys_of[];           // groups only: the keys of each warp's token
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t token = int64_t(blockIdx.x) * WARPS + warp;
    after_work_before();
    if (token >= p.tokens) return;
    const T *logits = static_cast<const T *>(p.logits) + token * p.ld;
    float score[V], key[V];
    bool out[V];
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = i * 32 + lane;
        const float l = e < p.experts ? value(logits[e]) : -INFINITY;
        out[i] = !(l > -INFINITY);
        key[i] = l;
        if (!out[i]) mx = fmaxf(mx, l);
    }
    if (p.softmax) {
        mx = warp_max(mx);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            score[i] = out[i] ? 0.f : key[i] == mx ? 1.f : expf(key[i] - mx);
            sum += score[i];
        }
        sum = warp_sum(sum);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            score[i] /= sum;
            if (p.bias) key[i] = score[i] + (out[i] ? 0.f : p.bias[i * 32 + lane]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            score[i] = out[i] ? 0.f : 1.f / (1.f + expf(-key[i]));
            key[i] = score[i] + (p.bias && !out[i] ? p.bias[i * 32 + lane] : 0.f);
        }
    }
    uint32_t order[V];
#pragma unroll
    for (int i = 0; i < V; ++i) order[i] = out[i] ? 0u : ordered(key[i]);

    if (p.groups > 1) {
        float *const keys = keys_of + warp * p.experts;
        const int size = p.experts / p.groups;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i * 32 + lane < p.experts) keys[i * 32 + lane] = order[i] ? key[i] : -INFINITY;
        __syncwarp();
        float first = -INFINITY, second = -INFINITY;
        if (lane < p.groups) {
            int j = lane % size;                 // lanes start at different places: their banks differ
            for (int n = 0; n < size; ++n) {
                const float v = keys[lane * size + j];
                second = fmaxf(second, fminf(first, v));
                first = fmaxf(first, v);
                if (++j == size) j = 0;
            }
        }
        // a group with a single expert left counts that one
        uint32_t rating = ordered(p.softmax || second == -INFINITY ? first : first + second);
        uint32_t chosen = 0;
        for (int n = 0; n < p.top_groups; ++n) {
            const uint32_t best = __reduce_max_sync(~0u, rating);
            if (best == 0) break;
            const int g = __ffs(__ballot_sync(~0u, rating == best)) - 1;
            chosen |= 1u << g;
            if (lane == g) rating = 0;
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (!(chosen >> ((size == 1 ? lane : __umulhi(uint32_t(i * 32 + lane), p.size_magic)) & 31) & 1)) order[i] = 0;
    }

    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) best = order[i] > best ? order[i] : best;
    int id = -1;                                 // lane j: the j-th
    float weight = 0.f;
    for (int j = 0; j < p.top; ++j) {
        const uint32_t most = __reduce_max_sync(~0u, best);
        if (most == 0) break;
        uint32_t mine = 0xffffffffu;
        float s = 0.f;
        if (best == most) {
#pragma unroll
            for (int i = V - 1; i >= 0; --i)
                if (order[i] == most) {
                    mine = i * 32 + lane;
                    s = score[i];
                }
        }
        const uint32_t e = __reduce_min_sync(~0u, mine);
        s = __shfl_sync(~0u, s, int(e & 31));
        if (lane == j) {
            id = int(e);
            weight = s;
        }
        if (mine == e) {
            best = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (i * 32 + lane == int(e)) order[i] = 0;
                best = order[i] > best ? order[i] : best;
            }
        }
    }
    if (p.renormalize) {
        const float sum = warp_sum(weight);
        weight = id >= 0 && sum > 0.f ? weight / sum : 0.f;
    }
    if (lane < p.top) {
        p.ids[token * p.top + lane] = id;
        p.weights[token * p.top + lane] = id >= 0 ? weight * p.factor : 0.f;         // 0 whatever the factor, an infinity too
    }
}

template <class T, int V> cudaError_t launch_as(const RouteArgs &p, cudaStream_t stream)
{
    const size_t bytes = p.groups > 1 ? size_t(WARPS) * p.experts * sizeof(float) : 0;
    return launch_after(route_kernel<T, V>, dim3(unsigned((p.tokens + WARPS - 1) / WARPS)), dim3(WARPS * 32), bytes, stream, dim3(1, 1), p);
}

template <class T> cudaError_t launch_type(const RouteArgs &p, cudaStream_t stream)
{
    if (p.experts <= 32) return launch_as<T, 1>(p, stream);
    if (p.experts <= 64) return launch_as<T, 2>(p, stream);
    if (p.experts <= 128) return launch_as<T, 4>(p, stream);
    if (p.experts <= 256) return launch_as<T, 8>(p, stream);
    if (p.experts <= 512) return launch_as<T, 16>(p, stream);
    return launch_as<T, 32>(p, stream);
}

}  // namespace

cudaError_t launch_route(RouteArgs p, cudaStream_t stream)
{
    const uint32_t size = uint32_t(p.experts / p.groups);
    p.size_magic = size == 1 ? 0 : uint32_t((uint64_t(1) << 32) / size + 1);       // e / size = high half of e * magic for e < 1024
    if (p.type == STRASSEN_BF16) return launch_type<__nv_bfloat16>(p, stream);
    if (p.type == STRASSEN_F16) return launch_type<__half>(p, stream);
    return launch_type<float>(p, stream);
}

}  // namespace strassen
