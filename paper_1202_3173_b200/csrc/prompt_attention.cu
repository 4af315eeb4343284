// Attention of many new tokens a sequence over a paged cache, on the fifth-generation tensor cores.
//
// A row of a tile is a head of a token: the heads that share a key head and as many tokens as make up to 128 rows, so few tokens fill a tile as long as there
// are many heads.  A CTA has two tiles (Q0, Q1) of neighbouring tokens and goes along the cache 128 rows (K, V) at a time:
//     S (128 x 128, 32 bits, tensor memory) = Q K^T;   P = 2^(c S - M), rounded to 16 bits, tensor memory;   O (128 x head_size, tensor memory) += P V
// with a running maximum M and the rows' sums in registers.  12 warps:
//   * warps 0-3 and 4-7: the softmax of tile 0 and 1, a thread a row.  O is scaled down only when a row's maximum has grown by more than 2^8: until
//     then M stays as it is, which the division at the end makes good (weights are at most 2^8, in f16 2^14: RAISE);
//   * warp 8 brings Q, K and V by tensor-map copies, a page or a part of it a box, and a ring of tiles;
//   * one lane of warp 9 issues the products.  S has one place in tensor memory, which both tiles use in turn: its columns are read into registers at once, so
//     that the next S is formed while the weights of this one are;
//   * warp 11 clears the rows of V that no row of the CTA sees (a page's slots behind the sequence may hold NaN, and 0 * NaN is NaN);
//   * warp 10 finds out what there is to do, ahead of the others.
// The CTAs stay and take blocks of tokens, those that see most first, in every other round in the opposite order, which evens out what they cost.
// Where there are few blocks and many rows in the cache, the rows are cut into parts, whose sums the join kernel adds in order (64 tokens of 32
// heads over 8 behind 16000: 40 us).
//
// What a token does not see has no effect on it.  Scores are replaced, but a weight of 0 times a value that is no number is none either.  So where a tile holds rows that some of the
// CTA's tokens see and some do not, warp 11 looks for such values of V, puts zeros in their place and raises a flag; then the tokens that do see them
// add them at the end, from memory.
//
// Over a cache in 8 bits the products are in f16, in which its values are exact.  Warps 12 to 15 then turn each tile of K and V, which a smaller ring brings, into 16 bits, and clear V, and queries in bf16 are brought into f16's range by a power of two a row.  Scores are multiplied by the key rows' scales, weights by the value rows', and
// M is the largest of score + log2(value scale), so that scaled weights keep within f16's range.  That is a multiplication by the key row's scale, an fma for the maximum and a
// multiplication by the value row's scale a score more than in 16 bits, and warps that turn tiles beside them: 2.3 times the instructions, 868 us for 8192 tokens of 32 heads over 8 of 128
// where 16 bits take 407 (0.63 PFLOP/s; tensor cores busy for 25 % of the time).
//
// A weight is rounded to 16 bits for its product, whose operands have one type: off by half a step of it, so a result by as much of the sum of weight times |value|, which is
// what rounding the result to that type costs where values have one sign.
//
// Bound, for head_size 128, by power: 16384 tokens of 32 heads over 8 run on and on in 1.78 ms, 1.24 PFLOP/s, at 1.46 GHz, where cuBLAS keeps up 1.38; the tensor cores are busy for 2048
// of 2830 clocks of a pair of tiles.  In short runs, at up to 1.9 GHz, they take 1.55 ms, 1.42 PFLOP/s, and 8192 tokens 407 us, 1.35.  For smaller heads by the softmax (8192 tokens of 64
// heads over 8 of 64 values: 673 us, 0.82 PFLOP/s; on and on 718): 128 exponentials of a thread take the special-function units 1050 clocks, with all around it 1250 for one warp of a
// scheduler and 2150 for two (timed alone), 2820 here, where a warp also waits for S (260), reads it (130), finds its largest (410), waits for the product before (200) and writes P
// (190 clocks a tile) while the other's exponentials take the issue slots.  What was tried: P over S, and S formed behind P V (the first form): 462 us at 8192 tokens of 32 heads
// over 8 of 128, then 407; a quarter of the exponentials by a polynomial of degree 4 446, for heads of 64 of degree 3 744 instead of 685, an eighth 687; two threads a row: 570; warps
// of exponentials in turns: 448 instead of 436; two places for S at head_size 64: the same; S in halves, the second one's largest found between the first one's exponentials: 436 instead of
// 406, for heads of 64 759 instead of 690; one vote a tile on the waits' outcome in place of three: 705 instead of 679.
//
// Every wait has a limit, after which the CTA gives up, frees its tensor memory and raises a flag (wait_for).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "attention.h"
#include "llm.h"
#include "tensor_cores.cuh"

namespace strassen {
namespace prompt {
namespace {

using namespace tc;

constexpr int TILE = 128;                            // rows of Q and of K and V
constexpr int SOFTMAX_WARPS = 8, LOAD_WARP = 8, MMA_WARP = 9, PLAN_WARP = 10, CLEAR_WARP = 11;
// Columns of tensor memory: S, which both tiles of Q use in turn; P and O of each.
constexpr int S_AT = 0, P_AT = TILE, P_WIDTH = TILE / 2, O_AT = 2 * TILE;
constexpr int MOST_BOXES = TILE / kLeastPage;
// What the cache holds.
enum { BF16 = 0, F16 = 1, EIGHT = 2 };
constexpr int RAW = 3, SCALES = 3;                   // stages of tiles in 8 bits, and of their rows' scales
constexpr int PLANS = 4, BLOCK = TILE * 128;         // bytes of a block of 64 values of 128 rows
constexpr int64_t kWaitLimit = int64_t(1) << 36;     // clocks of a wait for others to be through with a block: 2^24 tiles of the longest sequence take as long
constexpr int ONE_TILE = 48;                         // tiles of K and V up to which a CTA may have one tile of Q
constexpr int LEAST_TILES = 2;                       // tiles of K and V in a part (200 tokens of 8 heads over 2 behind 1000: 14.8 us; of 4: 18.7)

// Set by a CTA that gave up on a wait; read and cleared by strassen_device_status.
__device__ int g_gave_up;

struct Args {
    AttentionArgs a;
    int heads, blocks;       // heads of a key head in a tile, and how many such blocks of heads a key head has
    int group;               // heads of a key head
    int tokens;              // of a tile
    int block;               // of a block: of one tile or of two
    int box;                 // rows of K and V in a copy
    int wide;                // bytes that out's rows start at multiples of, and are long: 32, 16 or 0 (less)
    int parts;               // of a block's rows of the cache
    int most;                // blocks at most
    float *sums;             // parts > 1: part_floats() for each part of each block
};

// A part: what it is of, M, the sum of weights, and O in fours of columns, of the rows of both tiles.
constexpr int HEADER = 4;
__host__ __device__ constexpr int64_t part_floats(int d) { return HEADER + 2 * TILE * int64_t(2 + d); }

// What there is to do for one block of tokens and heads.
struct Plan {
    int done;                // 1: nothing more
    int b, kv, head0, heads; // heads that there are from head0 on, up to Args::heads
    int row0, count;         // first row of q; tokens, of both tiles
    int position;            // of the first token
    int last;                // last row of the cache that can be seen
    int from[2], to[2];      // tiles of K and V for each tile of Q; none: from == to
    int sees_from, sees_to;  // rows that some token sees ..
    int all_from, all_to;    // .. and that all see
    int slot;                // where its sums go
    int bad;                 // a value of V was no number where not all see it
    __device__ __forceinline__ int first() const { return from[0] == to[0] ? from[1] : from[1] == to[1] || from[0] < from[1] ? from[0] : from[1]; }
    __device__ __forceinline__ int end() const { return to[0] > to[1] ? to[0] : to[1]; }
    // whether tile j of V holds rows that some token does not see
    __device__ __forceinline__ bool ragged(int j) const { return j * TILE < all_from || j * TILE + TILE - 1 > all_to; }
};

template <int KIND, int DP> struct Shape {
    // warps that clear V, in 8 bits four of a warpgroup of their own that turn tiles; all warps' registers
    static constexpr int CLEARERS = KIND == EIGHT ? 4 : 1, THREADS = KIND == EIGHT ? 32 * 16 : 32 * 12, SOFTMAX_REGISTERS = KIND == EIGHT ? 184 : 216, OTHER_REGISTERS = 72;
    static constexpr int BLOCKS = DP / 64, BYTES = BLOCKS * BLOCK;         // of a tile
    static constexpr int STAGES = DP == 128 ? (KIND == EIGHT ? 3 : 5) : (KIND == EIGHT ? 6 : 8);
    // in 8 bits: tiles as they are in the cache; scales of a tile's rows of K and of V, as they are and as the softmax wants them
    static constexpr int RAW_BYTES = DP * TILE, RAW_AT = (2 + STAGES) * BYTES, RAW_SCALES_AT = RAW_AT + RAW * RAW_BYTES, SCALES_AT = RAW_SCALES_AT + RAW * 2 * TILE * 4;
    static constexpr int SMEM = (KIND == EIGHT ? SCALES_AT + SCALES * 3 * TILE * 4 : RAW_AT) + 1024;
    static_assert(SMEM + 1024 <= 227 * 1024, "shared memory");
};

struct Shared {
    uint64_t full[8], empty[8], q_full, q_empty, s_full[2], s_free, p_ready[2], o_done[2], o_free[2], cleared[8], plan_full[PLANS], plan_empty[PLANS], plan_cleared[PLANS];
    uint64_t raw_full[RAW], raw_empty[RAW], scales_full[SCALES], scales_empty[SCALES], q_ready;
    Plan plan[PLANS];
    uint32_t tmem;
    int dead;
};

// Waits until phase `parity` of the barrier is over.  False: the limit was reached; the caller leaves its loop, and the results of the call are not valid.  It is a
// number of tries, 2^20 of up to two microseconds each, which the hardware may end sooner: two seconds at most, and for what is a few tiles away.  One loop of three instructions: what a wait costs beyond the time waited comes between products (with the
// clock read on the way, 8192 tokens took 432 us instead of 407).
__device__ __forceinline__ bool wait_for(uint64_t *b, uint32_t parity, Shared *sh)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p, q;\n .reg .u32 n;\n mov.u32 n, 0;\nAGAIN:\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 2000;\n @p bra DONE;\n add.u32 n, n, 1;\n setp.lt.u32 q, n, 1048576;\n @q bra AGAIN;\nDONE:\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(smem_addr(b)), "r"(parity)
                 : "memory");
    if (ok) return true;
    *reinterpret_cast<volatile int *>(&sh->dead) = 1;
    g_gave_up = 1;
    return false;
}
// The same where the others may have a whole block to do, until one of them gives up: for plans (plan_full, plan_empty), and for the clearing of a block's last tile of V
// (plan_cleared), which a tile of Q without rows of the cache waits for from the block's start.  All other waits are for a few tiles: the rings' stages.
__device__ __forceinline__ bool wait_for_block(uint64_t *b, uint32_t parity, Shared *sh)
{
    if (bar_try(b, parity)) return true;
    for (const int64_t start = clock64(); clock64() - start < kWaitLimit;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (bar_try(b, parity)) return true;
        if (*reinterpret_cast<volatile int *>(&sh->dead)) return false;
    }
    *reinterpret_cast<volatile int *>(&sh->dead) = 1;
    g_gave_up = 1;
    return false;
}

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool BF> __device__ __forceinline__ uint32_t two_16_bits(float lo, float hi)
{
    uint32_t d;
    if (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float log2_of(float x)
{
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two e4m3 as two f16, exactly.
__device__ __forceinline__ uint32_t two_of_e4m3(uint32_t v)
{
    uint32_t d;
    asm("{\n .reg .b16 h;\n cvt.u16.u32 h, %1;\n cvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(d) : "r"(v));
    return d;
}
// (a b + c) for two pairs at once
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n fma.rn.f32x2 z, x, y, z;\n mov.b64 {%0, %1}, z;\n}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

__device__ __forceinline__ float largest(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float largest(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// The blocks of tokens in the order in which they are taken, as a whole warp sees them.
//
// Of up to 31 sequences, a lane one: offsets and lengths are read once, since each look at memory is half a microsecond that nothing else is done in, and
// blocks are in order of what they cost, the dearest first, so that the CTAs, which take them in turn, end together (7 prompts of up to 2049
// tokens, head_size 80: 245 us at the time, 274 in the sequences' order and with rows of no token masked).  How many blocks of a sequence cost c tiles or more needs no counting, so the n-th is found by halving.
//
// Of more sequences: the last first.  Sequence b's blocks begin with number offsets[b] / block + b, enough for its own, and found without adding up the ones before.
struct Order {
    const Args &p;
    const SequenceArgs &s;
    const bool few;
    int my_begin, my_count, my_length, my_blocks, all;
    __device__ __forceinline__ int cut(int o) const { return o < 0 ? 0 : o < s.tokens ? o : int(s.tokens); }
    __device__ __forceinline__ explicit Order(const Args &of) : p(of), s(of.a.seq), few(of.a.seq.batch < 32), my_begin(0), my_count(0), my_length(0), my_blocks(0)
    {
        const int lane = threadIdx.x & 31;
        if (!few) {
            all = cut(s.offsets[s.batch]) / p.block + s.batch;
            return;
        }
        if (lane <= s.batch) my_begin = cut(s.offsets[lane]);
        if (lane < s.batch) my_length = s.lengths[lane];
        const int stop = __shfl_down_sync(~0u, my_begin, 1);
        if (lane < s.batch && stop > my_begin) my_count = stop - my_begin;
        my_blocks = (my_count + p.block - 1) / p.block;
        // no more than there are places for, whatever offsets hold
        all = min(__reduce_add_sync(~0u, my_blocks), int(s.tokens / p.block) + s.batch);
    }
    // Blocks of the lane's sequence whose last token sees c tiles or more before its own, with a window as many as it leaves.  They are the last ones.
    __device__ __forceinline__ int dear(int c) const
    {
        if (c <= 0) return my_blocks;                // those of tokens that see nothing among them
        const int64_t row = int64_t(c) * TILE, start = int64_t(my_length) - my_count;
        if (my_count == 0 || start + my_count - 1 < row || (p.a.window && row > int64_t(p.a.window) + p.block)) return 0;
        // here 0 <= row < length, so that 32 bits do: a division of 64 takes longer than the rest
        const uint32_t before = row > start ? uint32_t(row - start) / uint32_t(p.block) : 0;
        return my_blocks - (before < uint32_t(my_blocks) ? int(before) : my_blocks - 1);
    }
    // Number n: its sequence and first token there.  False: there is none (of many sequences some numbers are of no block).
    __device__ __forceinline__ bool find(int n, int &b, int &first, int &begin, int &count, int &length) const
    {
        const int lane = threadIdx.x & 31;
        if (few) {
            // the largest c that more than n blocks cost
            int lo = 0, hi = __reduce_max_sync(~0u, my_count > 0 && my_length > 0 ? my_length / TILE + 1 : 1);
            while (hi - lo > 1) {
                const int c = lo + (hi - lo) / 2;
                if (__reduce_add_sync(~0u, dear(c)) > n) lo = c;
                else hi = c;
            }
            const int upto = dear(lo), above = dear(lo + 1), mine = upto - above, left = n - __reduce_add_sync(~0u, above);
            int before = mine;
            for (int i = 1; i < 32; i <<= 1) {
                const int other = __shfl_up_sync(~0u, before, i);
                if (lane >= i) before += other;
            }
            before -= mine;
            const unsigned found = __ballot_sync(~0u, left >= before && left < before + mine);
            if (!found) return false;
            b = __ffs(found) - 1;
            first = __shfl_sync(~0u, my_blocks - upto + left - before, b) * p.block;
            begin = __shfl_sync(~0u, my_begin, b);
            count = __shfl_sync(~0u, my_count, b);
            length = __shfl_sync(~0u, my_length, b);
            return true;
        }
        const int id = all - 1 - n;
        b = 0;
        for (int left = s.batch; left > 1;) {
            const int step = (left + 31) / 32;
            const bool below = lane * step < left && cut(s.offsets[b + lane * step]) / p.block + b + lane * step <= id;
            const int k = __popc(__ballot_sync(~0u, below));
            const int at = (k > 0 ? k - 1 : 0) * step;
            b += at;
            left = left - at < step ? left - at : step;
        }
        begin = cut(s.offsets[b]);
        count = cut(s.offsets[b + 1]) - begin;
        length = s.lengths[b];
        first = (id - (begin / p.block + b)) * p.block;
        return first >= 0 && first < count;
    }
};
__device__ __forceinline__ int all_plans(const Args &p, const Order &order) { return order.all * p.a.cache.kv_heads * p.blocks * p.parts; }

// What number n is; false if it has no tokens.  The whole warp takes part.
__device__ __forceinline__ bool plan_of(const Args &p, const Order &order, int n, Plan &to)
{
    const AttentionArgs &a = p.a;
    const int block = p.block, items = a.cache.kv_heads * p.blocks, whole = n / p.parts, part = n - whole * p.parts, item = whole % items;
    int lo, at, begin, n_tokens, length;
    if (!order.find(whole / items, lo, at, begin, n_tokens, length)) return false;
    to.slot = n;
    to.done = 0;
    to.b = lo;
    to.kv = item / p.blocks;
    to.head0 = to.kv * p.group + item % p.blocks * p.heads;
    to.heads = min(p.heads, (to.kv + 1) * p.group - to.head0);
    to.row0 = begin + at;
    to.count = n_tokens - at < block ? n_tokens - at : block;
    const int64_t position = int64_t(length) - n_tokens + at, most = int64_t(a.seq.width) << a.cache.page_shift;
    to.position = int(position > -(1 << 30) ? position : -(1 << 30));        // far below zero or just below is the same for up to 2^30 tokens' first ones
    to.last = length <= 0 ? -1 : int((length < most ? length : most) - 1);
    const auto low = [&](int64_t position) { return a.window && position >= a.window ? int(position - a.window + 1) : 0; };
    to.sees_from = to.all_from = 0;
    to.sees_to = to.all_to = -1;
    for (int x = 0; x < 2; ++x) {
        const int first = x * p.tokens, end = min((x + 1) * p.tokens, to.count);
        to.from[x] = to.to[x] = 0;
        if (first >= end) continue;
        const int64_t p0 = int64_t(to.position) + first, p1 = int64_t(to.position) + end - 1;
        const int from = low(p0), last = int(p1 < to.last ? p1 : to.last);
        if (last < from) continue;
        to.from[x] = from / TILE;
        to.to[x] = last / TILE + 1;
    }
    // of the whole block
    const int64_t p0 = to.position, p1 = p0 + to.count - 1;
    to.sees_from = low(p0);
    to.sees_to = int(p1 < to.last ? p1 : to.last);
    to.all_from = low(p1);
    to.all_to = int(p0 < to.last ? p0 : to.last);
    to.bad = 0;
    if (p.parts > 1) {
        const int first = to.first(), chunk = (to.end() - first + p.parts - 1) / p.parts, lowest = first + part * chunk;
        for (int x = 0; x < 2; ++x) {
            to.from[x] = max(to.from[x], lowest);
            to.to[x] = min(to.to[x], lowest + chunk);
            if (to.from[x] >= to.to[x]) to.from[x] = to.to[x] = 0;
        }
    }
    return true;
}

// LINEAR: the cache's rows are one after another, head after head and page after page; k_map and v_map have two dimensions, else four.
template <int KIND, int DP, bool LINEAR> __global__ void __launch_bounds__(Shape<KIND, DP>::THREADS, 1)
    prompt_kernel(const Args p, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using S = Shape<KIND, DP>;
    constexpr bool BF = KIND == BF16;
    constexpr int STAGES = S::STAGES;
    constexpr float RAISE = BF ? 0.f : 6.f, SLACK = 8.f;
    extern __shared__ uint8_t raw[];
    __shared__ Shared sh;
    uint8_t *const q_at = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023), *const ring = q_at + 2 * S::BYTES;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const AttentionArgs &a = p.a;
    const auto wait = [&](uint64_t *b, uint32_t parity) { return wait_for(b, parity, &sh); };
    const auto warp_wait_block = [&](uint64_t *b, uint32_t parity) { return bool(__all_sync(~0u, wait_for_block(b, parity, &sh))); };
    const auto warp_wait = [&](uint64_t *b, uint32_t parity) { return bool(__all_sync(~0u, wait_for(b, parity, &sh))); };

    if (warp == LOAD_WARP && elected()) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(&sh.full[i], S::CLEARERS);              // in 16 bits of the copies
            bar_init(&sh.empty[i], KIND == EIGHT ? 1 : 2);   // the products, and the warp that clears
            bar_init(&sh.cleared[i], 1);
        }
        bar_init(&sh.q_full, 1);
        bar_init(&sh.q_empty, 1);
        for (int x = 0; x < 2; ++x) {
            bar_init(&sh.s_full[x], 1);
            bar_init(&sh.p_ready[x], 4);
            bar_init(&sh.o_done[x], 1);
            bar_init(&sh.o_free[x], 4);
        }
        bar_init(&sh.s_free, 4);
        if (KIND == EIGHT) {
            for (int i = 0; i < RAW; ++i) {
                bar_init(&sh.raw_full[i], 1 + 32);           // the tile, and each lane's scales
                bar_init(&sh.raw_empty[i], S::CLEARERS);
            }
            for (int i = 0; i < SCALES; ++i) {
                bar_init(&sh.scales_full[i], S::CLEARERS);
                bar_init(&sh.scales_empty[i], SOFTMAX_WARPS);
            }
            bar_init(&sh.q_ready, SOFTMAX_WARPS);
        }
        for (int i = 0; i < PLANS; ++i) {
            bar_init(&sh.plan_full[i], 1);
            bar_init(&sh.plan_empty[i], SOFTMAX_WARPS + 2 + S::CLEARERS);
            bar_init(&sh.plan_cleared[i], S::CLEARERS);
        }
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    // tensor memory is taken when the work before is done: none is held while waiting for a kernel that may want it
    after_work_before();
    if (warp == MMA_WARP) alloc(&sh.tmem);
    __syncwarp();
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t tmem = sh.tmem;
    uint8_t *const raw_tiles = q_at + S::RAW_AT;
    float *const raw_scales = reinterpret_cast<float *>(q_at + S::RAW_SCALES_AT), *const scales = reinterpret_cast<float *>(q_at + S::SCALES_AT);
    // the plan of this role's next block; false: it is over
    int seen = 0;
    const auto take = [&]() -> const Plan * {
        if (!warp_wait_block(&sh.plan_full[seen % PLANS], (seen / PLANS) & 1)) return nullptr;
        const Plan *const plan = &sh.plan[seen % PLANS];
        return plan->done ? nullptr : plan;
    };
    const auto give_back = [&] {
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.plan_empty[seen % PLANS]);
        ++seen;
    };

    if (warp < SOFTMAX_WARPS) {
        // ---- softmax of tile x, a thread a row ---------------------------------------------------------------------------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::SOFTMAX_REGISTERS));
        const int x = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + (uint32_t((warp & 3) * 32) << 16), s_at = lanes + S_AT, p_at = lanes + P_AT + x * P_WIDTH, o_at = lanes + O_AT + x * DP;
        const bool negative = a.scale < 0.f;
        const float c = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1.17549435e-38f);        // not 0: -inf stays what it is
        const int token = r / p.heads, head = r - token * p.heads;
        uint32_t tiles = 0;                          // of this tile so far: phases of s_full and o_done
        uint32_t blocks = 0, scaled = 0;             // in 8 bits: blocks, and tiles of K and V, so far
        bool alive = true;
        while (alive) {
            const Plan *const plan = take();
            if (!plan) break;
            const int at = x * p.tokens + token;     // of the block's tokens
            const bool mine = token < p.tokens && at < plan->count && head < plan->heads;
            const int64_t position = int64_t(plan->position) + at;
            // rows of the cache that this row sees; one of no token: all, since its results go nowhere and where scores have to be replaced takes longer
            const int high = !mine ? 0x7fffffff : int(position < plan->last ? position : plan->last), low = mine && a.window && position >= a.window ? int(position - a.window + 1) : 0;
            const int first = plan->from[x], end = plan->to[x];
            float m = -INFINITY, l = 0.f, factor = c;        // factor: of scores
            if (KIND == EIGHT && plan->first() < plan->end()) {
                // this row of Q in f16
                if (!(alive = warp_wait(&sh.q_full, blocks & 1))) break;
                ++blocks;
                if (a.type == STRASSEN_BF16 && plan->count > x * p.tokens) {
                    uint8_t *const row = q_at + x * S::BYTES + r * 128;
                    float most = 0.f;
#pragma unroll 4
                    for (int i = 0; i < S::BLOCKS * 8; ++i) {
                        const uint4 u = *reinterpret_cast<const uint4 *>(row + (i >> 3) * BLOCK + (i & 7) * 16);
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(__uint_as_float(w[e] << 16)), fabsf(__uint_as_float(w[e] & 0xffff0000u))));
                    }
                    // the power of two that brings the largest to 1 .. 2; queries that are 0 or no numbers are left alone
                    const uint32_t e = __float_as_uint(most) >> 23;
                    const bool turn = e > 1 && e < 253;
                    const float down = turn ? __uint_as_float((254 - e) << 23) : 1.f;
                    factor = fmaxf(c * (turn ? __uint_as_float(e << 23) : 1.f), 1.17549435e-38f);
#pragma unroll 4
                    for (int i = 0; i < S::BLOCKS * 8; ++i) {
                        uint4 *const at = reinterpret_cast<uint4 *>(row + (i >> 3) * BLOCK + (i & 7) * 16);
                        uint32_t w[4] = {at->x, at->y, at->z, at->w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = two_16_bits<false>(__uint_as_float(w[e] << 16) * down, __uint_as_float(w[e] & 0xffff0000u) * down);
                        *at = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.q_ready);
            }
            for (int j = KIND == EIGHT ? plan->first() : first; j < (KIND == EIGHT ? plan->end() : end); ++j) {
                const float *const k_scale = scales + scaled % SCALES * 3 * TILE, *const v_scale = k_scale + TILE, *const v_log2 = v_scale + TILE;
                if (KIND == EIGHT) {
                    if (!(alive = warp_wait(&sh.scales_full[scaled % SCALES], (scaled / SCALES) & 1))) break;
                    if (j < first || j >= end) {
                        __syncwarp();
                        if (lane == 0) bar_arrive(&sh.scales_empty[scaled % SCALES]);
                        ++scaled;
                        continue;
                    }
                }
                if (!(alive = warp_wait(&sh.s_full[x], tiles & 1))) break;
                after_sync();
                float s[TILE];
#pragma unroll
                for (int i = 0; i < 4; ++i) load32(s + 32 * i, s_at + 32 * i);
                wait_loads();
                before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.s_free);
                if (negative) {
#pragma unroll
                    for (int i = 0; i < TILE; ++i) s[i] = -s[i];
                }
                if (KIND == EIGHT) {
#pragma unroll
                    for (int i = 0; i < TILE; i += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(k_scale + i);
                        const float2 lo = mul2(make_float2(s[i], s[i + 1]), make_float2(f.x, f.y)), hi = mul2(make_float2(s[i + 2], s[i + 3]), make_float2(f.z, f.w));
                        s[i] = lo.x, s[i + 1] = lo.y, s[i + 2] = hi.x, s[i + 3] = hi.y;
                    }
                }
                const int to = high - j * TILE, from = low - j * TILE;
                const bool cut = __any_sync(~0u, to < TILE - 1 || from > 0);
                if (cut) {
#pragma unroll
                    for (int i = 0; i < TILE; ++i) s[i] = i <= to && i >= from ? s[i] : -INFINITY;
                }
                float here;
                if (KIND == EIGHT) {
                    float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < TILE; i += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(v_log2 + i);
                        const float2 lo = fma2(make_float2(s[i], s[i + 1]), make_float2(factor, factor), make_float2(f.x, f.y)),
                                     hi = fma2(make_float2(s[i + 2], s[i + 3]), make_float2(factor, factor), make_float2(f.z, f.w));
                        most[0] = largest(most[0], lo.x, lo.y);
                        most[1] = largest(most[1], hi.x, hi.y);
                    }
                    here = largest(most[0], most[1]);
                } else {
                    float most[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                    for (int i = 4; i + 8 <= TILE; i += 8) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) most[e] = largest(most[e], s[i + 2 * e], s[i + 2 * e + 1]);
                    }
                    here = largest(largest(most[0], most[1], most[2]), most[3], largest(largest(s[TILE - 4], s[TILE - 3]), s[TILE - 2], s[TILE - 1])) * factor;
                }
                float back = 1.f;
                bool grows = false;
                if (j == first) {
                    m = here;
                } else if (__any_sync(~0u, mine && !(here <= m + SLACK))) {
                    // a score that is no number makes m, and with it the whole row, none
                    const float next = largest(m, here);
                    back = m == next ? 1.f : exp2_of(m - next);
                    m = next;
                    l *= back;
                    grows = true;
                }
                // nothing but -inf so far: weights of 0; an infinite score: no numbers
                const float off = m == -INFINITY ? 0.f : RAISE - m + (m - m);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                uint32_t w[TILE / 2];
#pragma unroll
                for (int e = 0; e < TILE / 2; ++e) {
                    float2 v = fma2(make_float2(s[2 * e], s[2 * e + 1]), make_float2(factor, factor), make_float2(off, off));
                    v.x = exp2_of(v.x);
                    v.y = exp2_of(v.y);
                    sum[e & 1] = add2(sum[e & 1], v);
                    if (KIND == EIGHT) v = mul2(v, *reinterpret_cast<const float2 *>(v_scale + 2 * e));
                    w[e] = two_16_bits<BF>(v.x, v.y);
                }
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                if (KIND == EIGHT) {
                    __syncwarp();
                    if (lane == 0) bar_arrive(&sh.scales_empty[scaled % SCALES]);
                    ++scaled;
                }
                // the product with the weights before is done: their place is free, and O at rest
                if (j > first && !(alive = warp_wait(&sh.o_done[x], (tiles - 1) & 1))) break;
                if (grows) {
                    after_sync();
#pragma unroll 1
                    for (int i = 0; i < a.cache.d; i += 16) {
                        float o[16];
                        load16(o, o_at + i);
                        wait_loads();
                        uint32_t u[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(o[e] * back);
                        store16(o_at + i, u);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) store16(p_at + 16 * i, w + 16 * i);
                ++tiles;
                wait_stores();
                before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.p_ready[x]);
            }
            if (!alive) break;
            // the whole block for the warps of a tile that has no rows of the cache
            if (!(alive = warp_wait_block(&sh.plan_cleared[seen % PLANS], (seen / PLANS) & 1))) break;
            const bool bad = plan->bad != 0, any = first < end;
            if (any) {
                if (!(alive = warp_wait(&sh.o_done[x], (tiles - 1) & 1))) break;
                after_sync();
            }
            // a part leaves its sums as they are
            const float inv = p.parts > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
            float *const sums = p.sums + plan->slot * part_floats(a.cache.d) + HEADER + x * TILE + r;
            if (p.parts > 1) {
                sums[0] = m;
                sums[2 * TILE] = l;
            }
            uint16_t *const out = static_cast<uint16_t *>(a.out) + int64_t(plan->row0 + at) * a.out_row + (plan->head0 + head) * a.out_head;
#pragma unroll 1
            for (int i = 0; i < a.cache.d; i += 32) {
                float o[32];
                if (any) {
                    load32(o, o_at + i);
                    wait_loads();
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = any ? o[e] * inv : 0.f;
                if (bad && mine) {
                    // values of V that are no numbers, in rows that not all tokens of the block see: this one's
                    for (int part = 0; part < 2; ++part) {
                        // of the tiles that this part of the block has: an infinity of another part's, added to sums that weigh 0 in the end, would be NaN
                        const int begin = max(part == 0 ? low : max(low, max(plan->all_to + 1, plan->all_from)), first * TILE), stop = min(part == 0 ? min(high + 1, plan->all_from) : high + 1, end * TILE);
                        for (int j = begin; j < stop; ++j) {
                            const int page = page_of(a.cache, a.seq, plan->b, j);
                            if (page < 0) continue;
                            const int slot = j & ((1 << a.cache.page_shift) - 1);
                            const uint8_t *const bytes = a.cache.v + page * a.cache.page_stride + plan->kv * a.cache.head_stride + slot * a.cache.row_stride;
                            if (KIND == EIGHT) {
                                const float f = a.cache.v_scale[((int64_t(page) * a.cache.kv_heads + plan->kv) << a.cache.page_shift) + slot];
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (i + e < a.cache.d) {
                                        const float v = f * float(reinterpret_cast<const __nv_fp8_e4m3 *>(bytes)[i + e]);
                                        if (!(v - v == 0.f)) o[e] += v;
                                    }
                                continue;
                            }
                            const uint16_t *const row = reinterpret_cast<const uint16_t *>(bytes);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (i + e < a.cache.d) {
                                    const float v = BF ? __uint_as_float(uint32_t(row[i + e]) << 16) : __half2float(__ushort_as_half(row[i + e]));
                                    if (!(v - v == 0.f)) o[e] += v;
                                }
                        }
                    }
                }
                if (p.parts > 1) {
                    if (any && mine) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (i + 4 * e < a.cache.d) *reinterpret_cast<float4 *>(sums - (x * TILE + r) + 4 * TILE + ((i / 4 + e) * 2 * TILE + x * TILE + r) * 4) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                    }
                } else if (mine) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = BF || (KIND == EIGHT && a.type == STRASSEN_BF16) ? two_16_bits<true>(o[2 * e], o[2 * e + 1]) : two_16_bits<false>(o[2 * e], o[2 * e + 1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (i + 8 * e >= a.cache.d) break;
                        if (p.wide == 32) {
                            // whole sectors: 16 values at a time
                            if (e % 2 == 0)
                                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + i + 8 * e), "r"(w[4 * e]), "r"(w[4 * e + 1]), "r"(w[4 * e + 2]), "r"(w[4 * e + 3]),
                                             "r"(w[4 * e + 4]), "r"(w[4 * e + 5]), "r"(w[4 * e + 6]), "r"(w[4 * e + 7])
                                             : "memory");
                        } else if (p.wide) {
                            *reinterpret_cast<uint4 *>(out + i + 8 * e) = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                        } else {
#pragma unroll
                            for (int k = 0; k < 8; ++k) out[i + 8 * e + k] = uint16_t(w[4 * e + k / 2] >> (16 * (k & 1)));
                        }
                    }
                }
            }
            if (any) {
                before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.o_free[x]);
            }
            give_back();
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::OTHER_REGISTERS));
        if (warp == PLAN_WARP) {
            // ---- what there is to do ---------------------------------------------------------------------------------------
            const Order order(p);
            const int all = all_plans(p, order);
            int round = 0, from = 0;                 // from: this round's first
            for (int n = 0;; ++n) {
                Plan plan;
                bool some = false;
                for (; !some && from < all; from += int(gridDim.x), ++round) {
                    const int at = from + int(round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
                    if (at >= all) continue;
                    some = plan_of(p, order, at, plan);
                    // for the join kernel
                    if (p.parts > 1 && lane == 0)
                        *reinterpret_cast<int4 *>(p.sums + at * part_floats(a.cache.d)) = make_int4(some ? plan.count : 0, plan.row0, plan.head0, plan.heads);
                }
                if (n >= PLANS && !warp_wait_block(&sh.plan_empty[n % PLANS], (n / PLANS - 1) & 1)) break;
                if (lane == 0) {
                    if (!some) plan.done = 1;
                    sh.plan[n % PLANS] = plan;
                    bar_arrive(&sh.plan_full[n % PLANS]);
                }
                __syncwarp();
                if (!some) break;
            }
        } else if (warp == LOAD_WARP) {
            // ---- copies ------------------------------------------------------------------------------------------------------
            const uint32_t q_to = smem_addr(q_at), ring_to = smem_addr(ring);
            const int boxes = TILE / p.box;
            int tiles = 0, blocks = 0;
            bool alive = true;
            // the box that lane i brings of tile j: its page, or one past the last, which reads as zeros
            const auto page_at = [&](const Plan &plan, int j) {
                const int64_t row = int64_t(j) * TILE + lane * p.box;
                int page = -1;
                if (lane < boxes && row <= plan.last) page = page_of(a.cache, a.seq, plan.b, row);
                return page < 0 ? int(a.cache.pages) : page;
            };
            while (alive) {
                const Plan *const taken = take();
                if (!taken) break;
                const Plan &plan = *taken;
                const int first = plan.first(), end = plan.end();
                if (first < end) {
                    int page = page_at(plan, first);
                    if (blocks > 0 && !(alive = warp_wait(&sh.q_empty, (blocks - 1) & 1))) break;
                    ++blocks;
                    if (elected()) {
                        const int used = plan.count > p.tokens ? 2 : 1;
                        bar_expect(&sh.q_full, uint32_t(used * S::BLOCKS * p.heads * p.tokens * 128));
                        for (int x = 0; x < used; ++x)
                            for (int i = 0; i < S::BLOCKS; ++i) box3(q_to + x * S::BYTES + i * BLOCK, &q_map, 64 * i, plan.head0, plan.row0 + x * p.tokens, &sh.q_full);
                    }
                    __syncwarp();
                    // K of tile j + 1 before V of tile j
                    int pages = page;
                    for (int j = first - 1; j < end && alive; ++j) {
                        const int before = pages;        // of tile j
                        pages = page;
                        if (j + 2 < end) page = page_at(plan, j + 2);
                        for (int which = j + 1 < end ? 0 : 1; which < (j < first ? 1 : 2); ++which, ++tiles) {
                            // in 8 bits into the ring of those
                            constexpr int RING = KIND == EIGHT ? RAW : STAGES;
                            uint64_t *const full = KIND == EIGHT ? sh.raw_full : sh.full, *const empty = KIND == EIGHT ? sh.raw_empty : sh.empty;
                            const int stage = tiles % RING;
                            if (tiles >= RING && !(alive = warp_wait(&empty[stage], (tiles / RING - 1) & 1))) break;
                            // the pages' numbers first, then all boxes in one go: one at a time, pages of 16 rows kept the tensor cores waiting
                            int number[MOST_BOXES];
                            const int mine = which ? before : pages, row = (which ? j : j + 1) * TILE;
#pragma unroll
                            for (int i = 0; i < MOST_BOXES; ++i) number[i] = __shfl_sync(~0u, mine, i);
                            if (elected()) {
                                const CUtensorMap *const map = which ? &v_map : &k_map;
                                const uint32_t to = KIND == EIGHT ? smem_addr(raw_tiles) + stage * S::RAW_BYTES : ring_to + stage * S::BYTES;
                                bar_expect(&full[stage], KIND == EIGHT ? S::RAW_BYTES : S::BYTES);
#pragma unroll
                                for (int i = 0; i < MOST_BOXES; ++i) {
                                    if (i >= boxes) break;
                                    const int slot = (row + i * p.box) & ((1 << a.cache.page_shift) - 1), at = ((number[i] * a.cache.kv_heads + plan.kv) << a.cache.page_shift) + slot;
#pragma unroll
                                    for (int k = 0; k < (KIND == EIGHT ? 1 : S::BLOCKS); ++k) {
                                        const uint32_t there = KIND == EIGHT ? to + i * p.box * DP : to + k * BLOCK + i * p.box * 128;
                                        // the fewer numbers say where a box is, the sooner it is issued
                                        if (LINEAR) box2(there, map, 64 * k, at, &full[stage]);
                                        else box4(there, map, 64 * k, slot, plan.kv, number[i], &full[stage]);
                                    }
                                }
                            }
                            __syncwarp();
                            if (KIND == EIGHT) {
                                // with a tile of K the scales of its rows and of V's
                                if (which == 0) {
#pragma unroll
                                    for (int i = 0; i < TILE / 32; ++i) {
                                        const int r = lane + 32 * i, number = __shfl_sync(~0u, mine, r / p.box), slot = (row + r) & ((1 << a.cache.page_shift) - 1);
                                        const bool there = number < a.cache.pages;
                                        const int64_t at = there ? ((int64_t(number) * a.cache.kv_heads + plan.kv) << a.cache.page_shift) + slot : 0;
                                        const uint32_t to = smem_addr(raw_scales) + (stage * 2 * TILE + r) * 4;
                                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(a.cache.k_scale + at), "r"(there ? 4 : 0) : "memory");
                                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + TILE * 4), "l"(a.cache.v_scale + at), "r"(there ? 4 : 0) : "memory");
                                    }
                                }
                                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(&full[stage])) : "memory");
                            }
                        }
                    }
                }
                if (alive) give_back();
            }
            // what has been brought is used up, and the arrivals that say so are here, before the CTA is left
            if (KIND == EIGHT) {
                for (int n = tiles > RAW ? tiles - RAW : 0; n < tiles && alive; ++n) alive = warp_wait(&sh.raw_empty[n % RAW], (n / RAW) & 1);
            }
            for (int n = tiles > STAGES ? tiles - STAGES : 0; n < tiles && alive; ++n) alive = warp_wait(&sh.empty[n % STAGES], (n / STAGES) & 1);
            if (alive && blocks > 0) alive = warp_wait(&sh.q_empty, (blocks - 1) & 1);
            if (!alive)
                for (int i = 0; i < 10000; ++i) __nanosleep(100);        // after giving up: the copies under way end before the CTA does
        } else if (warp == MMA_WARP) {
            // ---- products: one lane does it all, since what it does between them is time in which the tensor cores may run dry ---------
            if (elected()) {
                constexpr uint32_t format = BF ? 1 : 0;
                constexpr uint32_t both = (1u << 4) | (format << 7) | (format << 10) | (uint32_t(TILE >> 4) << 24);
                constexpr uint32_t s_desc = both | (uint32_t(TILE >> 3) << 17);
                const uint32_t o_desc = both | (1u << 16) | (uint32_t((a.cache.d + 15) / 16 * 2) << 17);
                const uint64_t q_from = rows_operand(smem_addr(q_at)), k_from = rows_operand(smem_addr(ring)), v_from = columns_operand(smem_addr(ring), BLOCK);
                const int steps = (a.cache.d + 15) / 16;
                // A place in the ring: K of tile first, K of first + 1, V of first, K of first + 2, V of first + 1, .. V of end - 1
                struct Place {
                    int stage;
                    uint32_t phase;
                    __device__ __forceinline__ void skip(int n)
                    {
                        stage += n;
                        if (stage >= STAGES) {
                            stage -= STAGES;
                            phase ^= 1;
                        }
                    }
                } k_place = {0, 0}, v_place;
                uint32_t blocks = 0, scores = 0, ready[2] = {0, 0}, outputs[2] = {0, 0};
                bool alive = true;
                while (alive) {
                    if (!(alive = wait_for_block(&sh.plan_full[seen % PLANS], (seen / PLANS) & 1, &sh))) break;
                    const Plan &plan = sh.plan[seen % PLANS];
                    if (plan.done) break;
                    const int from0 = plan.from[0], to0 = plan.to[0], from1 = plan.from[1], to1 = plan.to[1], first = plan.first(), end = plan.end(), all_from = plan.all_from, all_to = plan.all_to;
                    bar_arrive(&sh.plan_empty[seen % PLANS]);
                    ++seen;
                    if (first >= end) continue;
                    const auto active = [&](int x, int j) { return x ? j >= from1 && j < to1 : j >= from0 && j < to0; };
                    if (!(alive = wait(KIND == EIGHT ? &sh.q_ready : &sh.q_full, blocks & 1))) break;
                    ++blocks;
                    v_place = k_place;
                    v_place.skip(end - first > 1 ? 2 : 1);
                    // S of tile kj for one tile of Q and then the other, as long as there are tiles
                    int kj = first, kx = active(0, first) ? 0 : 1;
                    bool k_here = false;
                    const auto next_scores = [&] {
                        if (kj >= end) return true;
                        if (!k_here && !wait(&sh.full[k_place.stage], k_place.phase)) return false;
                        if (scores > 0 && !wait(&sh.s_free, (scores - 1) & 1)) return false;
                        ++scores;
                        after_sync();
                        const uint64_t kd = k_from + uint32_t(k_place.stage * (S::BYTES / 16)), qd = q_from + uint32_t(kx * (S::BYTES / 16));
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            if (k >= steps) break;
                            const int at = (k / 4) * (BLOCK / 16) + (k % 4) * 2;
                            mma_ss(tmem + S_AT, qd + at, kd + at, s_desc, k > 0);
                        }
                        commit(&sh.s_full[kx]);
                        k_here = kx == 0 && active(1, kj);
                        if (k_here) {
                            kx = 1;
                        } else {
                            commit(&sh.empty[k_place.stage]);
                            k_place.skip(kj == first ? 1 : 2);
                            ++kj;
                            kx = kj < end && active(0, kj) ? 0 : 1;
                            if (kj == end) commit(&sh.q_empty);
                        }
                        return true;
                    };
                    // S is three ahead of P V: it can be formed when the one before has been read, which is when the weights of the one before that are done.
                    // It comes in the middle of P V, whose first half fills the time until then, and whose second half nothing waits for.  Where there is one
                    // tile of Q alone, two ahead: the weights of the next S but one would wait for this P V.
                    const int ahead = from0 < to0 && from1 < to1 ? 3 : 2;
                    for (int n = 0; n < ahead && alive; ++n) alive = next_scores();
                    for (int j = first; j < end && alive; ++j) {
                        const uint64_t vd = v_from + uint32_t(v_place.stage * (S::BYTES / 16));
                        bool v_here = false;
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            if (!active(x, j)) continue;
                            if (!v_here) {
                                if (!(alive = wait(&sh.full[v_place.stage], v_place.phase))) break;
                                if (KIND != EIGHT && (j * TILE < all_from || j * TILE + TILE - 1 > all_to) && !(alive = wait(&sh.cleared[v_place.stage], v_place.phase))) break;
                                v_here = true;
                            }
                            const bool begins = j == (x ? from1 : from0);
                            if (begins && outputs[x] > 0 && !(alive = wait(&sh.o_free[x], (outputs[x] - 1) & 1))) break;
                            if (begins) ++outputs[x];
                            if (!(alive = wait(&sh.p_ready[x], ready[x] & 1))) break;
                            ++ready[x];
                            after_sync();
                            const auto values = [&](int k) { mma_ts(tmem + O_AT + x * DP, tmem + P_AT + x * P_WIDTH + k * 8, vd + k * (16 * 128 / 16), o_desc, !begins || k > 0); };
#pragma unroll
                            for (int k = 0; k < TILE / 32; ++k) values(k);
                            if (!(alive = next_scores())) break;
#pragma unroll
                            for (int k = TILE / 32; k < TILE / 16; ++k) values(k);
                            commit(&sh.o_done[x]);
                        }
                        if (!alive) break;
                        commit(&sh.empty[v_place.stage]);
                        if (j + 1 < end) v_place.skip(j + 2 < end ? 2 : 1);
                    }
                    k_place = v_place;
                    k_place.skip(1);
                }
            }
            __syncwarp();
        } else if (warp == (KIND == EIGHT ? 12 + (warp & 3) : CLEAR_WARP)) {
            // ---- rows of V that not all tokens see -------------------------------------------------------------------------------
            int tiles = 0;
            uint32_t scaled = 0;                     // in 8 bits: tiles whose scales have been handed on
            bool alive = true;
            while (alive) {
                const Plan *const taken = take();
                if (!taken) break;
                const Plan &plan = *taken;
                const int first = plan.first(), end = plan.end();
                bool bad = false;
                for (int n = 0; n < 2 * (end - first) && alive; ++n, ++tiles) {
                    const int stage = tiles % STAGES, last = 2 * (end - first) - 1, j = n == last ? end - 1 : first + n / 2 - 1;
                    if (KIND == EIGHT) {
                        const bool is_v = n == last || (n > 0 && n % 2 == 0);
                        const int raw_stage = tiles % RAW;
                        if (!(alive = warp_wait(&sh.raw_full[raw_stage], (tiles / RAW) & 1))) break;
                        if (!is_v) {
                            // of K: its rows' scales, and those of V of the same tile; what no token sees weighs nothing, whatever its scale
                            const int k_tile = n == 0 ? first : first + (n + 1) / 2;
                            const uint32_t slot = scaled % SCALES;
                            const int quarter = warp & 3;
                            if (scaled >= SCALES && !(alive = warp_wait(&sh.scales_empty[slot], (scaled / SCALES - 1) & 1))) break;
                            {
                                const int r = lane + 32 * quarter, number = k_tile * TILE + r;
                                const float *const from = raw_scales + raw_stage * 2 * TILE + r;
                                float v = from[TILE];
                                if (number < plan.sees_from || number > plan.sees_to) v = 0.f;
                                if ((number < plan.all_from || number > plan.all_to) && !(v - v == 0.f)) {
                                    v = 0.f;
                                    bad = true;
                                }
                                float *const to = scales + slot * 3 * TILE + r;
                                to[0] = from[0];
                                to[TILE] = v;
                                to[2 * TILE] = log2_of(fmaxf(fabsf(v), kMinRowScale));
                            }
                            __syncwarp();
                            if (lane == 0) bar_arrive(&sh.scales_full[slot]);
                            ++scaled;
                        }
                        if (tiles >= STAGES && !(alive = warp_wait(&sh.empty[stage], (tiles / STAGES - 1) & 1))) break;
                        // 16 values a lane: two chunks of a swizzled row, the second one first in the second block, so that lanes of both fall into different banks
                        constexpr int PER_ROW = DP / 16;
#pragma unroll 4
                        for (int i = lane + (warp & 3) * (TILE / 4 * PER_ROW); i < ((warp & 3) + 1) * (TILE / 4 * PER_ROW); i += 32) {
                            const int r = i / PER_ROW, c = i % PER_ROW, number = j * TILE + r;
                            const uint4 u = *reinterpret_cast<const uint4 *>(raw_tiles + raw_stage * S::RAW_BYTES + i * 16);
                            uint32_t w[4] = {u.x, u.y, u.z, u.w}, h[8];
                            if (is_v && (number < plan.all_from || number > plan.all_to)) {
                                const bool none = number < plan.sees_from || number > plan.sees_to;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    // NaN: all bits but the sign's
                                    const uint32_t nan = __vcmpeq4(w[e] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                                    bad |= !none && nan != 0;
                                    w[e] = none ? 0 : w[e] & ~nan;
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                h[2 * e] = two_of_e4m3(w[e]);
                                h[2 * e + 1] = two_of_e4m3(w[e] >> 16);
                            }
                            uint8_t *const row = ring + stage * S::BYTES + c / 4 * BLOCK + r * 128;
                            const int chunk = c % 4 * 2, swap = c / 4;
                            const uint4 lo = make_uint4(h[0], h[1], h[2], h[3]), hi = make_uint4(h[4], h[5], h[6], h[7]);
                            *reinterpret_cast<uint4 *>(row + 16 * ((chunk + swap) ^ (r & 7))) = swap ? hi : lo;
                            *reinterpret_cast<uint4 *>(row + 16 * ((chunk + 1 - swap) ^ (r & 7))) = swap ? lo : hi;
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            bar_arrive(&sh.full[stage]);
                            bar_arrive(&sh.raw_empty[raw_stage]);
                        }
                        continue;
                    }
                    if (!(alive = warp_wait(&sh.full[stage], (tiles / STAGES) & 1))) break;
                    if ((n == last || (n > 0 && n % 2 == 0)) && plan.ragged(j)) {          // of V: the others are of K
                        // a lane has one 16-byte chunk of every fourth row
                        const int base = j * TILE;
                        const int zeros_to = min(max(plan.sees_from - base, 0), TILE), zeros_from = min(max(plan.sees_to + 1 - base, 0), TILE);        // rows that none sees
                        const int from = min(max(plan.all_from - base, 0), TILE), to = min(max(plan.all_to + 1 - base, from), TILE);            // rows that all see
#pragma unroll 1
                        for (int k = 0; k < S::BLOCKS; ++k) {
                            uint4 *const v = reinterpret_cast<uint4 *>(ring + stage * S::BYTES + k * BLOCK) + (lane & 7);
                            const int first = lane >> 3;
                            for (int r = first; r < zeros_to; r += 4) v[r * 8] = make_uint4(0, 0, 0, 0);
                            for (int r = first + ((zeros_from - first + 3) & ~3); r < TILE; r += 4) v[r * 8] = make_uint4(0, 0, 0, 0);
                            // before the rows that all see, and after
                            for (int part = 0; part < 2; ++part) {
                                const int begin = part ? max(to, zeros_to) : zeros_to, stop = part ? zeros_from : min(from, zeros_from);
                                // exponents of all ones: one more in their last place carries into the sign's
                                constexpr uint32_t ones = BF ? 0x7f807f80u : 0x7c007c00u, one = BF ? 0x00800080u : 0x04000400u, signs = 0x80008000u;
                                constexpr int AT_ONCE = 8;
                                for (int r0 = begin + first; r0 < stop; r0 += 4 * AT_ONCE) {
                                    uint4 u[AT_ONCE];
#pragma unroll
                                    for (int n = 0; n < AT_ONCE; ++n) u[n] = r0 + 4 * n < stop ? v[(r0 + 4 * n) * 8] : make_uint4(0, 0, 0, 0);
                                    uint32_t found = 0;
#pragma unroll
                                    for (int n = 0; n < AT_ONCE; ++n)
                                        found |= ((u[n].x & ones) + one) | ((u[n].y & ones) + one) | ((u[n].z & ones) + one) | ((u[n].w & ones) + one);
                                    if (found & signs) {
                                        bad = true;
#pragma unroll 1
                                        for (int r = r0; r < min(stop, r0 + 4 * AT_ONCE); r += 4) {
                                            uint32_t *const word = reinterpret_cast<uint32_t *>(v + r * 8);
                                            for (int k = 0; k < 4; ++k)
                                                for (int h = 0; h < 32; h += 16)
                                                    if ((word[k] >> h & ones >> 16) == ones >> 16) word[k] &= ~(0xffffu << h);
                                        }
                                    }
                                }
                            }
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    if (lane == 0) {
                        bar_arrive(&sh.cleared[stage]);
                        bar_arrive(&sh.empty[stage]);
                    }
                }
                if (!alive) break;
                bad = __any_sync(~0u, bad);
                if (lane == 0) {
                    if (bad) sh.plan[seen % PLANS].bad = 1;
                    bar_arrive(&sh.plan_cleared[seen % PLANS]);
                }
                give_back();
            }
        }
    }
    __syncwarp();
    before_sync();
    __syncthreads();
    after_sync();
    if (warp == MMA_WARP) dealloc(tmem);
}

// The parts of block blockIdx.x, added up in order: a CTA has 32 rows of 16 columns; lane r a row, and warp w the parts w, w + 8, ..
constexpr int JOIN_WARPS = 8, JOIN_COLUMNS = 16;
template <bool BF> __global__ void __launch_bounds__(32 * JOIN_WARPS) join_kernel(const Args p)
{
    __shared__ float sh[JOIN_WARPS][2 + JOIN_COLUMNS][32];
    after_work_before();
    const AttentionArgs &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = 32 * blockIdx.z + lane, x = row / TILE, r = row % TILE, token = r / p.heads, head = r - token * p.heads,
              at = x * p.tokens + token, first = JOIN_COLUMNS * blockIdx.y;
    if (int(blockIdx.x) * p.parts >= all_plans(p, Order(p))) return;
    const float *const header = p.sums + int64_t(blockIdx.x) * p.parts * part_floats(a.cache.d), *const first_part = header + HEADER;
    const int4 of = *reinterpret_cast<const int4 *>(header);             // tokens, row, head, heads
    // (of a CTA that gave up there may be no header)
    const bool mine = token < p.tokens && at < of.x && head < of.w && of.y >= 0 && int64_t(of.y) + at < a.seq.tokens && of.z >= 0 && of.z < a.heads - head;
    if (!__syncthreads_or(mine)) return;
    float m = -INFINITY, l = 0.f, o[JOIN_COLUMNS];
#pragma unroll
    for (int e = 0; e < JOIN_COLUMNS; ++e) o[e] = 0.f;
    if (mine) {
#pragma unroll 4
        for (int k = warp; k < p.parts; k += JOIN_WARPS) {
            const float *const part = first_part + k * part_floats(a.cache.d);
            const float here = part[row], sum = part[2 * TILE + row];
            float4 v[JOIN_COLUMNS / 4];
#pragma unroll
            for (int e = 0; e < JOIN_COLUMNS / 4; ++e)
                v[e] = first + 4 * e < a.cache.d ? reinterpret_cast<const float4 *>(part + 4 * TILE)[(first / 4 + e) * 2 * TILE + row] : make_float4(0.f, 0.f, 0.f, 0.f);
            if (here == -INFINITY) continue;         // it has seen nothing, and may not have written its O
            const float next = largest(m, here), back = m == next ? 1.f : exp2_of(m - next), w = here == next ? 1.f : exp2_of(here - next);
            m = next;
            l = l * back + w * sum;
#pragma unroll
            for (int e = 0; e < JOIN_COLUMNS / 4; ++e) {
                o[4 * e] = o[4 * e] * back + w * v[e].x;
                o[4 * e + 1] = o[4 * e + 1] * back + w * v[e].y;
                o[4 * e + 2] = o[4 * e + 2] * back + w * v[e].z;
                o[4 * e + 3] = o[4 * e + 3] * back + w * v[e].w;
            }
        }
    }
    sh[warp][0][lane] = m;
    sh[warp][1][lane] = l;
#pragma unroll
    for (int e = 0; e < JOIN_COLUMNS; ++e) sh[warp][2 + e][lane] = o[e];
    __syncthreads();
    // warp w has columns 2 w and 2 w + 1 of every row
    if (!mine || first + 2 * warp >= a.cache.d) return;
    float most = -INFINITY, sum = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) most = largest(most, sh[w][0][lane]);
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) {
        const float here = sh[w][0][lane], f = here == most ? 1.f : exp2_of(here - most);
        if (here == -INFINITY) continue;
        sum += f * sh[w][1][lane];
        y0 += f * sh[w][2 + 2 * warp][lane];
        y1 += f * sh[w][3 + 2 * warp][lane];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t *const out = static_cast<uint16_t *>(a.out) + int64_t(of.y + at) * a.out_row + (of.z + head) * a.out_head + first + 2 * warp;
    const uint32_t both = two_16_bits<BF>(y0 * inv, y1 * inv);
    if (p.wide) {
        *reinterpret_cast<uint32_t *>(out) = both;
    } else {
        out[0] = uint16_t(both);
        out[1] = uint16_t(both >> 16);
    }
}

// How the work is cut up, from the sizes alone: lengths and offsets are the device's.
struct Cut {
    int blocks, heads, tokens, block, parts;
    int64_t most;            // blocks of tokens and heads, at most
};
Cut cut_of(const AttentionArgs &a, int sm_count)
{
    Cut c;
    const int group = a.heads / a.cache.kv_heads;
    c.blocks = (group + TILE - 1) / TILE;
    c.heads = (group + c.blocks - 1) / c.blocks;
    c.tokens = TILE / c.heads;
    const auto blocks = [&](int of) { return (a.seq.tokens / of + a.seq.batch) * a.cache.kv_heads * c.blocks; };
    // tiles of the longest sequence that the table has room for
    const int64_t rows = int64_t(a.seq.width) << a.cache.page_shift, seen = a.window ? int64_t(a.window) + 2 * c.tokens + TILE : rows, tiles = ((seen < rows ? seen : rows) + TILE - 1) / TILE;
    // One tile of Q a CTA as long as there are SMs enough: its softmax does not share the schedulers (512 tokens of 32 heads over 8: 15.1 us, 17.0 with two; behind 1000: 25.4, 44.2).
    // Behind many rows two, and more parts: half as many bytes out of the second cache, which bounds that (200 tokens behind 16000: 72.6 us, 96.4 with one; 8 x 37 of
    // 32 heads over 2 behind up to 15724: 69.8, 92.5; the other way round 512 behind 4000: 62.1, 54.3).
    c.block = blocks(c.tokens) <= sm_count && tiles <= ONE_TILE ? c.tokens : 2 * c.tokens;
    c.most = blocks(c.block);
    // Parts: the fewest rounds of the shortest pieces, where a piece takes some 4 tiles' time more and the join as long once.  Rounds that are not full cost most where
    // blocks are few and long: 24 sequences of up to 406 tokens behind 6763, 2 heads of 64: 53.9 us, 102.0 in one part; 32 of 21 behind 7569, 32 over 4: 95.6, 146.4.
    c.parts = 1;
    // Of the numbers of parts with as many rounds the largest is looked at, made smaller as far as pieces stay as they are.
    const auto over = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
    if (c.most > 0 && c.most < 2 * sm_count) {
        int64_t best = over(c.most, sm_count) * (tiles + 4);
        const int64_t limit = tiles / LEAST_TILES < sm_count ? tiles / LEAST_TILES : sm_count;
        for (int64_t rounds = 1; rounds <= 16; ++rounds) {
            const int64_t most = rounds * sm_count / c.most;
            if ((most < limit ? most : limit) < 2) continue;
            const int64_t piece = over(tiles, most < limit ? most : limit), parts = over(tiles, piece), cost = over(c.most * parts, sm_count) * (piece + 4) + 4;
            if (cost < best) {
                best = cost;
                c.parts = int(parts);
            }
            if (most >= limit) break;
        }
    }
    return c;
}

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);

// The driver's function that fills a tensor map, looked up once.
EncodeTiled encode_tiled()
{
    static std::atomic<EncodeTiled> found{nullptr};
    EncodeTiled f = found.load(std::memory_order_acquire);
    if (!f) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        f = reinterpret_cast<EncodeTiled>(p);
        found.store(f, std::memory_order_release);
    }
    return f;
}

// strides in bytes, of all dimensions but the first
bool encode(CUtensorMap *map, const void *at, int dims, const cuuint64_t *sizes, const cuuint64_t *strides, const cuuint32_t *box, bool bytes = false)
{
    const EncodeTiled f = encode_tiled();
    const cuuint32_t steps[4] = {1, 1, 1, 1};
    return f && f(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, cuuint32_t(dims), const_cast<void *>(at), sizes, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  bytes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND, int DP, bool LINEAR> cudaError_t launch_as(const Args &p, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, int ctas, cudaStream_t stream)
{
    using S = Shape<KIND, DP>;
    const auto kernel = prompt_kernel<KIND, DP, LINEAR>;
    // The warps' shares of registers come out of what the block has from the start.
    static const bool enough = [&] {
        cudaFuncAttributes attr;
        return cudaFuncGetAttributes(&attr, kernel) == cudaSuccess && attr.numRegs * S::THREADS >= 32 * SOFTMAX_WARPS * S::SOFTMAX_REGISTERS + (S::THREADS - 32 * SOFTMAX_WARPS) * S::OTHER_REGISTERS;
    }();
    if (!enough) return cudaErrorInvalidConfiguration;
    const cudaError_t e = allow_shared<prompt_kernel<KIND, DP, LINEAR>>(S::SMEM);
    if (e != cudaSuccess) return e;
    const cudaError_t launched = launch_after(kernel, dim3(unsigned(ctas)), dim3(S::THREADS), S::SMEM, stream, dim3(1, 1), p, q, k, v);
    if (launched != cudaSuccess || p.parts == 1) return launched;
    const auto join = p.a.type == STRASSEN_BF16 ? join_kernel<true> : join_kernel<false>;
    return launch_after(join, dim3(unsigned(p.most), unsigned((p.a.cache.d + JOIN_COLUMNS - 1) / JOIN_COLUMNS), unsigned((p.block > p.tokens ? 2 : 1) * TILE / 32)), dim3(32 * JOIN_WARPS), 0, stream, dim3(1, 1), p);
}
template <int KIND, int DP> cudaError_t launch(const Args &p, bool linear, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, int ctas, cudaStream_t stream)
{
    return linear ? launch_as<KIND, DP, true>(p, q, k, v, ctas, stream) : launch_as<KIND, DP, false>(p, q, k, v, ctas, stream);
}

}  // namespace
}  // namespace prompt

cudaError_t prompt_gave_up(int *flag)
{
    const int zero = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(flag, prompt::g_gave_up, sizeof(int));
    return e != cudaSuccess || !*flag ? e : cudaMemcpyToSymbol(prompt::g_gave_up, &zero, sizeof(int));
}

bool prompt_takes(const AttentionArgs &a, int sm_count)
{
    const prompt::Cut c = prompt::cut_of(a, sm_count);
    return c.most * c.parts <= 0x7fffffff - sm_count;
}

int64_t prompt_workspace(const AttentionArgs &a, int sm_count)
{
    const prompt::Cut c = prompt::cut_of(a, sm_count);
    return c.parts > 1 ? c.most * c.parts * prompt::part_floats(a.cache.d) * 4 : 0;
}

cudaError_t launch_prompt(const AttentionArgs &given, int sm_count, cudaStream_t stream)
{
    prompt::Args p;
    p.a = given;
    AttentionArgs &a = p.a;
    const prompt::Cut c = prompt::cut_of(a, sm_count);
    p.group = a.heads / a.cache.kv_heads;
    p.blocks = c.blocks;
    p.heads = c.heads;
    p.tokens = c.tokens;
    p.block = c.block;
    p.parts = c.parts;
    p.most = int(c.most);
    p.sums = static_cast<float *>(a.workspace);
    const int page = 1 << a.cache.page_shift;
    p.box = page < prompt::TILE ? page : prompt::TILE;
    const uintptr_t places = reinterpret_cast<uintptr_t>(a.out) | uintptr_t(a.out_row * 2) | uintptr_t(a.out_head * 2);
    p.wide = (places | uintptr_t(a.cache.d * 2)) % 32 == 0 ? 32 : places % 16 == 0 ? 16 : 0;
    bool linear = false;
    CUtensorMap q, k, v;
    {
        const cuuint64_t sizes[3] = {cuuint64_t(a.cache.d), cuuint64_t(a.heads), cuuint64_t(a.seq.tokens)};
        const cuuint64_t strides[2] = {cuuint64_t(a.q.head ? a.q.head : a.cache.d) * 2, cuuint64_t(a.q.row ? a.q.row : a.cache.d) * 2};
        const cuuint32_t box[3] = {64, cuuint32_t(p.heads), cuuint32_t(p.tokens)};
        if (!prompt::encode(&q, a.q.p, 3, sizes, strides, box)) return cudaErrorInvalidValue;
    }
    if (a.cache.pages > 0) {
        const cuuint64_t sizes[4] = {cuuint64_t(a.cache.d), cuuint64_t(page), cuuint64_t(a.cache.kv_heads), cuuint64_t(a.cache.pages)};
        const cuuint64_t strides[3] = {cuuint64_t(a.cache.row_stride), cuuint64_t(a.cache.head_stride), cuuint64_t(a.cache.page_stride)};
        const bool eight = a.cache.type == STRASSEN_E4M3;             // whole rows, not swizzled
        const cuuint32_t box[4] = {cuuint32_t(eight && a.cache.d > 64 ? 128 : 64), cuuint32_t(p.box), 1, 1};
        // 7 prompts of up to 2049 tokens, head_size 80, pages of 16 rows: 207 us instead of 246; of 64: 192 instead of 195; 8000 tokens of 8 heads over one of
        // 128, pages of 16: 121 instead of 144
        const int64_t rows = int64_t(page) * a.cache.kv_heads;
        linear = rows_in_a_row(a.cache) && (a.cache.pages + 1) * rows <= 0x7fffffff;
        const cuuint64_t linear_sizes[2] = {cuuint64_t(a.cache.d), cuuint64_t(rows * a.cache.pages)};
        const auto map = [&](CUtensorMap *to, const void *at) { return linear ? prompt::encode(to, at, 2, linear_sizes, strides, box, eight) : prompt::encode(to, at, 4, sizes, strides, box, eight); };
        if (!map(&k, a.cache.k) || !map(&v, a.cache.v)) return cudaErrorInvalidValue;
    } else {
        // rows that are not there read as zeros, whose mean is what a token that sees nothing gets
        a.seq.width = 0;
        k = v = q;
    }
    const int64_t all = c.most * c.parts;
    const int ctas = int(all < sm_count ? all : sm_count);
    const bool narrow = a.cache.d <= 64;
    if (a.cache.type == STRASSEN_BF16) return narrow ? prompt::launch<prompt::BF16, 64>(p, linear, q, k, v, ctas, stream) : prompt::launch<prompt::BF16, 128>(p, linear, q, k, v, ctas, stream);
    if (a.cache.type == STRASSEN_F16) return narrow ? prompt::launch<prompt::F16, 64>(p, linear, q, k, v, ctas, stream) : prompt::launch<prompt::F16, 128>(p, linear, q, k, v, ctas, stream);
    return narrow ? prompt::launch<prompt::EIGHT, 64>(p, linear, q, k, v, ctas, stream) : prompt::launch<prompt::EIGHT, 128>(p, linear, q, k, v, ctas, stream);
}

}  // namespace strassen
