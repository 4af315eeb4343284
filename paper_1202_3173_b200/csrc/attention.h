// Attention operators: what the host entry points (attention_api.cu) and the kernels share.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "strassen_b200.h"

namespace strassen {

constexpr int kMostHeadSize = 128, kMostHeads = 1024, kLeastPage = 8, kMostPage = 1024;

// The cache as kernels see it; strides in bytes.
struct CacheArgs {
    int type, kv_heads, d, page_shift;       // rows of d values; 1 << page_shift rows of a head in a page
    int64_t pages;
    uint8_t *k, *v;
    int64_t page_stride, head_stride, row_stride;
    float *k_scale, *v_scale;                // e4m3: one for each row, (page * kv_heads + head) << page_shift | slot
};

// Whether the cache's rows are one after another, head after head and page after page.  The stride of a dimension of one is nobody's.
inline bool rows_in_a_row(const CacheArgs &c)
{
    const int64_t of_head = c.row_stride << c.page_shift;
    return (c.kv_heads == 1 || c.head_stride == of_head) && (c.pages == 1 || c.page_stride == of_head * c.kv_heads);
}

// Where the sequences are.  offsets NULL: one new token each.
struct SequenceArgs {
    int batch, width;                        // entries of a row of the table
    const int *table;
    int64_t ld_table;
    const int *lengths, *offsets;
    int64_t tokens;                          // rows of q
};

struct Heads {
    const void *p;
    int64_t row, head;                       // elements between rows, between the heads of a row
};

struct AppendArgs {
    CacheArgs cache;
    SequenceArgs seq;
    int type, heads;                         // heads 0: there is no q
    Heads q, k, v;
    void *out;
    int64_t out_row, out_head;
    const float *frequencies;
    int rotary, interleaved;
    bool wide;                               // all rows start at multiples of 16 bytes
};

struct AttentionArgs {
    CacheArgs cache;
    SequenceArgs seq;
    int type, heads;
    Heads q;
    void *out;
    int64_t out_row, out_head;
    float scale;
    int window;                              // 0: none
    void *workspace;
};

cudaError_t launch_append(const AppendArgs &a, int sm_count, cudaStream_t stream);
int64_t decode_workspace(const AttentionArgs &a, int sm_count);
cudaError_t launch_decode(const AttentionArgs &a, int sm_count, cudaStream_t stream);
bool prompt_takes(const AttentionArgs &a, int sm_count);          // there are not too many tokens and heads
int64_t prompt_workspace(const AttentionArgs &a, int sm_count);
cudaError_t prompt_gave_up(int *flag);        // reads and clears the flag of prompt_attention.cu
cudaError_t launch_prompt(const AttentionArgs &a, int sm_count, cudaStream_t stream);

// How the attention of one token is cut up, from the sizes alone.
namespace decode {
constexpr int MOST_RANKS = 16;                        // CTAs of a cluster

// Steps of a sequence at most, by the table's width.
inline int64_t steps_of(const AttentionArgs &a, int step)
{
    const int64_t rows = int64_t(a.seq.width) << a.cache.page_shift, seen = a.window && a.window < rows ? a.window : rows;
    return seen > 0 ? (seen + step - 1) / step : 1;
}

// CTAs of an item's cluster; 0: even runs and the join kernel.  most: 16, or 8 where the device holds no larger cluster.
//
// Few short items, as the table's width has it: each has a cluster, of as many CTAs as there is room for and steps to do, and there is no second kernel and no plan
// to make (32 heads over 8 of 128, bf16: 1000 rows 6.8 us instead of 10.2, 4000 10.1 instead of 17.5, 8000 14.1 for 18.4; 8 sequences of 1000 10.3 for 13.1).  Clusters of 16 only
// where they all have SMs to themselves (two sequences of 1000: 7.5 in eights, 12.0 in sixteens).  Longer ones take turns that are uneven where lengths are, and up to 8
// steps of a CTA, 16 where eights fill the GPU, that costs less than the rest spares (4 sequences of 8000: 24.9 for 30.6; 16 of 4000, not taken: 40.9 for 38.2).
// Many short items are better off in runs (64 sequences of 240: 21 us, 25 with a CTA each; of 57: 9.6, 19).
// What has clusters without a window has them with one: no more steps, and no fewer CTAs than those.
inline int ranks_of(const AttentionArgs &a, int step, int64_t heads, int sm_count, int most)
{
    const int64_t steps = steps_of(a, step), items = heads * a.seq.batch;
    int64_t ranks = most >= 16 && 16 * items <= sm_count ? 16 : 8;
    while (ranks > 1 && (ranks >= 2 * steps || ranks * items > 2 * sm_count)) ranks /= 2;
    return ranks * items <= 2 * sm_count && steps <= (ranks == 8 && ranks * items >= sm_count ? 16 : 8) * ranks ? int(ranks) : 0;
}
}  // namespace decode

#ifdef __CUDACC__
// Allows Kernel its dynamic shared memory, and clusters of up to 16 CTAs where it has such, on the current device, the first time it is launched there: asked each time, a launch takes a microsecond longer.
template <auto Kernel> cudaError_t allow_shared(int bytes, bool large_clusters = false)
{
    static std::atomic<uint64_t> done{0};            // a bit for each device; entry points refuse more than 64
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (done.load(std::memory_order_acquire) >> dev & 1)) return e;
    e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && large_clusters) e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) done.fetch_or(uint64_t(1) << dev, std::memory_order_release);
    return e;
}

// The new tokens of sequence b: rows first .. end - 1 of q, whatever offsets hold; the last one is at position lengths[b] - 1.
struct NewTokens {
    int64_t first, end;
    int length;
};
__device__ __forceinline__ NewTokens new_tokens(const SequenceArgs &s, int b)
{
    NewTokens n;
    n.length = s.lengths[b];
    n.first = b;
    n.end = b + 1;
    if (s.offsets) {
        const int64_t first = s.offsets[b], end = s.offsets[b + 1];
        n.first = first < 0 ? 0 : first < s.tokens ? first : s.tokens;
        n.end = end < n.first ? n.first : end < s.tokens ? end : s.tokens;
    }
    return n;
}
// The page of row j of sequence b, -1 if there is none.
__device__ __forceinline__ int page_of(const CacheArgs &c, const SequenceArgs &s, int b, int64_t j)
{
    const int64_t at = j >> c.page_shift;
    if (at >= s.width) return -1;
    const int page = s.table[b * s.ld_table + at];
    return uint32_t(page) < uint64_t(c.pages) ? page : -1;
}
#endif

}  // namespace strassen
