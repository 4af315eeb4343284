// Attention of one new token a sequence: arguments of the kernels in decode_attention.cuh.
#include "decode_attention.cuh"

namespace strassen {

namespace {

struct Shape {
    int dp, nt, blocks;
};

Shape shape_of(const AttentionArgs &a)
{
    const int group = a.heads / a.cache.kv_heads;
    Shape s;
    s.dp = a.cache.d <= 64 ? 64 : 128;
    s.nt = group <= 8 ? 1 : 2;
    s.blocks = (group + 8 * s.nt - 1) / (8 * s.nt);
    return s;
}

}  // namespace

int64_t decode_workspace(const AttentionArgs &a, int sm_count)
{
    const Shape s = shape_of(a);
    const auto ranks = a.cache.type == STRASSEN_BF16 ? decode::ranks_bf16 : a.cache.type == STRASSEN_F16 ? decode::ranks_f16 : decode::ranks_e4m3;
    if (ranks(a, s.dp, s.nt, a.cache.kv_heads * int64_t(s.blocks), sm_count) > 0) return 0;
    // two parts and a note for each run
    return 2 * sm_count * (2 * int64_t(decode::part_floats(s.dp, s.nt)) * 4 + int64_t(sizeof(decode::Meta)));
}

cudaError_t launch_decode(const AttentionArgs &a, int sm_count, cudaStream_t stream)
{
    const Shape s = shape_of(a);
    decode::Args p;
    p.a = a;
    if (a.cache.pages == 0) p.a.seq.width = 0;       // rows that are not there read as zeros, whose mean is what a token that sees nothing gets
    p.items = a.cache.kv_heads * s.blocks;
    p.blocks = s.blocks;
    p.group = a.heads / a.cache.kv_heads;
    p.wide = reinterpret_cast<uintptr_t>(a.q.p) % 16 == 0 && a.q.row % 8 == 0 && a.q.head % 8 == 0;
    p.meta = static_cast<decode::Meta *>(a.workspace);
    p.parts = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + 2 * sm_count * sizeof(decode::Meta));
    if (a.cache.type == STRASSEN_BF16) return decode::launch_bf16(p, s.dp, s.nt, sm_count, stream);
    if (a.cache.type == STRASSEN_F16) return decode::launch_f16(p, s.dp, s.nt, sm_count, stream);
    return decode::launch_e4m3(p, s.dp, s.nt, sm_count, stream);
}

}  // namespace strassen
