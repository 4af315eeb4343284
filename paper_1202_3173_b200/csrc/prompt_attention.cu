// Attention of many new tokens a sequence over a paged cache, on the fifth-generation tensor cores.
//
// A row of a tile is a head of a token: the heads that share a key head and as many tokens as make up to 128 rows, so few tokens fill a tile as long as there
// are many heads.  A CTA has two tiles (Q0, Q1) of neighbouring tokens and goes along the cache 128 rows (K, V) at a time:
//     S (128 x 128, 32 bits, tensor memory) = Q K^T;   P = 2^(c S - M), rounded to 16 bits, over S;   O (128 x head_size, tensor memory) += P V
// with a running maximum M and the rows' sums in registers.  12 warps:
//   * warps 0-3 and 4-7: the softmax of tile 0 and 1, a thread a row.  O is scaled down only when a row's maximum has grown by more than 2^8: until
//     then M stays as it is, which the division at the end makes good (weights are at most 2^8, in f16 2^14: RAISE).  No barrier is needed
//     for that: S of the next rows is issued behind P V of these, so when S has arrived O is at rest;
//   * warp 8 brings Q, K and V by tensor-map copies, a page or a part of it a box, and a ring of tiles;
//   * one lane of warp 9 issues the products.  While one tile's rows are in the softmax, the other's products run;
//   * warp 10 clears the rows of V that no row of the CTA sees (a page's slots behind the sequence may hold NaN, and 0 * NaN is NaN);
//   * warp 11 finds out what there is to do, ahead of the others.
// The CTAs stay and take blocks of tokens, the last ones, which see most, first; in every other round in the opposite order, which evens out what they cost.
//
// What a token does not see has no effect on it.  Scores are replaced, but a weight of 0 times a value that is no number is none either.  So where a tile holds rows that some of the
// CTA's tokens see and some do not, warp 10 looks for such values of V, puts zeros in their place and raises a flag; then the tokens that do see them
// add them at the end, from memory.
//
// Bound by the tensor cores and the special-function units alike: a tile of 128 x 128 scores of head_size 128 takes 1024 clocks of each (8192
// operations and 16 exponentials a clock).
//
// Every wait has a limit, after which the CTA gives up, frees its tensor memory and raises a flag (wait_for).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "attention.h"
#include "llm.h"
#include "tensor_cores.cuh"

namespace strassen {
namespace prompt {
namespace {

using namespace tc;

constexpr int TILE = 128;                            // rows of Q and of K and V
constexpr int LOAD_WARP = 8, MMA_WARP = 9, CLEAR_WARP = 10, PLAN_WARP = 11, THREADS = 32 * 12;
constexpr int PLANS = 4, BLOCK = TILE * 128;         // bytes of a block of 64 values of 128 rows
constexpr int64_t kWaitLimit = int64_t(1) << 31;     // clocks of a wait, about a second

// Set by a CTA that gave up on a wait; read and cleared by strassen_device_status.
__device__ int g_gave_up;

struct Args {
    AttentionArgs a;
    int heads, blocks;       // heads of a key head in a tile, and how many such blocks of heads a key head has
    int group;               // heads of a key head
    int tokens;              // of a tile
    int box;                 // rows of K and V in a copy
    bool wide;               // out's rows start at multiples of 16 bytes
};

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
    int bad;                 // a value of V was no number where not all see it
    __device__ __forceinline__ int first() const { return from[0] == to[0] ? from[1] : from[1] == to[1] || from[0] < from[1] ? from[0] : from[1]; }
    __device__ __forceinline__ int end() const { return to[0] > to[1] ? to[0] : to[1]; }
    // whether tile j of V holds rows that some token does not see
    __device__ __forceinline__ bool ragged(int j) const { return j * TILE < all_from || j * TILE + TILE - 1 > all_to; }
};

template <int DP> struct Shape {
    static constexpr int BLOCKS = DP / 64, BYTES = BLOCKS * BLOCK;         // of a tile
    static constexpr int STAGES = DP == 128 ? 5 : 8, SMEM = (2 + STAGES) * BYTES + 1024;
};

struct Shared {
    uint64_t full[8], empty[8], q_full, q_empty, s_full[2], p_ready[2], o_full[2], o_free[2], cleared[8], plan_full[PLANS], plan_empty[PLANS], plan_cleared[PLANS];
    Plan plan[PLANS];
    uint32_t tmem;
    int dead;
};

// Waits until phase `parity` of the barrier is over.  False: the limit was reached, here or elsewhere in the CTA; the caller leaves its loop, and the results of
// the call are not valid.
__device__ __forceinline__ bool wait_for(uint64_t *b, uint32_t parity, Shared *sh)
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
// (a b + c) for two pairs at once
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n .reg .b64 x, y, z;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n fma.rn.f32x2 z, x, y, z;\n mov.b64 {%0, %1}, z;\n}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}" : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// The next block of tokens of this CTA that has any; `round` counts them.  The whole warp takes part.
__device__ __forceinline__ bool next_plan(const Args &p, int &round, Plan &to)
{
    const AttentionArgs &a = p.a;
    const int lane = threadIdx.x & 31, block = 2 * p.tokens, items = a.cache.kv_heads * p.blocks;
    const auto offset = [&](int b) {
        const int64_t o = a.seq.offsets[b];
        return o < 0 ? 0 : o < a.seq.tokens ? o : a.seq.tokens;
    };
    // blocks are numbered so that sequence b's begin with offsets[b] / block + b: enough for its own, and found without adding up the ones before
    const int64_t all = (offset(a.seq.batch) / block + a.seq.batch) * items;
    for (;; ++round) {
        const int64_t n = int64_t(round) * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        if (int64_t(round) * gridDim.x >= all) return false;
        if (n >= all) continue;
        const int64_t id = all / items - 1 - n / items;
        const int item = int(n % items);
        int lo = 0;
        for (int left = a.seq.batch; left > 1;) {
            const int step = (left + 31) / 32;
            const bool below = lane * step < left && offset(lo + lane * step) / block + lo + lane * step <= id;
            const int k = __popc(__ballot_sync(~0u, below));
            const int at = (k > 0 ? k - 1 : 0) * step;
            lo += at;
            left = left - at < step ? left - at : step;
        }
        const NewTokens s = new_tokens(a.seq, lo);
        const int64_t at = (id - (offset(lo) / block + lo)) * block, n_tokens = s.end - s.first;
        if (at < 0 || at >= n_tokens) continue;
        to.done = 0;
        to.b = lo;
        to.kv = item / p.blocks;
        to.head0 = to.kv * p.group + item % p.blocks * p.heads;
        to.heads = min(p.heads, (to.kv + 1) * p.group - to.head0);
        to.row0 = int(s.first + at);
        to.count = int(n_tokens - at < block ? n_tokens - at : block);
        const int64_t position = s.length - n_tokens + at, most = int64_t(a.seq.width) << a.cache.page_shift;
        to.position = int(position > -(1 << 30) ? position : -(1 << 30));        // far below zero or just below is the same for up to 2^30 tokens' first ones
        to.last = s.length <= 0 ? -1 : int((s.length < most ? s.length : most) - 1);
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
        return true;
    }
}

template <bool BF, int DP> __global__ void __launch_bounds__(THREADS, 1)
    prompt_kernel(const Args p, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using S = Shape<DP>;
    constexpr int STAGES = S::STAGES;
    constexpr float RAISE = BF ? 0.f : 6.f, SLACK = 8.f;
    extern __shared__ uint8_t raw[];
    __shared__ Shared sh;
    uint8_t *const q_at = raw + ((1024 - (smem_addr(raw) & 1023)) & 1023), *const ring = q_at + 2 * S::BYTES;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const AttentionArgs &a = p.a;
    const auto wait = [&](uint64_t *b, uint32_t parity) { return wait_for(b, parity, &sh); };
    const auto warp_wait = [&](uint64_t *b, uint32_t parity) { return bool(__all_sync(~0u, wait_for(b, parity, &sh))); };

    if (warp == LOAD_WARP && elected()) {
        for (int i = 0; i < STAGES; ++i) {
            bar_init(&sh.full[i], 1);
            bar_init(&sh.empty[i], 2);               // the products, and the warp that clears
            bar_init(&sh.cleared[i], 1);
        }
        bar_init(&sh.q_full, 1);
        bar_init(&sh.q_empty, 1);
        for (int x = 0; x < 2; ++x) {
            bar_init(&sh.s_full[x], 1);
            bar_init(&sh.p_ready[x], 4);
            bar_init(&sh.o_full[x], 1);
            bar_init(&sh.o_free[x], 4);
        }
        for (int i = 0; i < PLANS; ++i) {
            bar_init(&sh.plan_full[i], 1);
            bar_init(&sh.plan_empty[i], 11);         // 8 warps of softmax, the three others
            bar_init(&sh.plan_cleared[i], 1);
        }
        sh.dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    if (warp == MMA_WARP) alloc(&sh.tmem);
    __syncwarp();
    before_sync();
    __syncthreads();
    after_sync();
    after_work_before();
    const uint32_t tmem = sh.tmem;
    // the plan of this role's next block; false: it is over
    int seen = 0;
    const auto take = [&](Plan &plan) {
        if (!warp_wait(&sh.plan_full[seen % PLANS], (seen / PLANS) & 1)) return false;
        plan = sh.plan[seen % PLANS];
        return !plan.done;
    };
    const auto give_back = [&] {
        __syncwarp();
        if (lane == 0) bar_arrive(&sh.plan_empty[seen % PLANS]);
        ++seen;
    };

    if (warp < 8) {
        // ---- softmax of tile x ------------------------------------------------------------------------------------------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int x = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = uint32_t((warp & 3) * 32) << 16, s_at = tmem + lanes + x * TILE, o_at = tmem + lanes + 2 * TILE + x * DP;
        const bool negative = a.scale < 0.f;
        const float c = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1.17549435e-38f);        // not 0: -inf stays what it is
        const int token = r / p.heads, head = r - token * p.heads;
        uint32_t tiles = 0, outputs = 0;             // of this tile so far: phases of s_full and o_full
        bool alive = true;
        Plan plan;
        while (alive && take(plan)) {
            const int at = x * p.tokens + token;     // of the block's tokens
            const bool mine = token < p.tokens && at < plan.count && head < plan.heads;
            const int64_t position = int64_t(plan.position) + at;
            // rows of the cache that this row sees
            const int high = !mine ? -1 : int(position < plan.last ? position : plan.last), low = a.window && position >= a.window ? int(position - a.window + 1) : 0;
            float m = -INFINITY, l = 0.f;
            for (int j = plan.from[x]; j < plan.to[x]; ++j) {
                if (!(alive = warp_wait(&sh.s_full[x], tiles & 1))) break;
                ++tiles;
                after_sync();
                float s[TILE];
#pragma unroll
                for (int i = 0; i < 4; ++i) load32(s + 32 * i, s_at + 32 * i);
                wait_loads();
                if (negative) {
#pragma unroll
                    for (int i = 0; i < TILE; ++i) s[i] = -s[i];
                }
                const int to = high - j * TILE, from = low - j * TILE;
                if (__any_sync(~0u, to < TILE - 1 || from > 0)) {
#pragma unroll
                    for (int i = 0; i < TILE; ++i) s[i] = i <= to && i >= from ? s[i] : -INFINITY;
                }
                float most[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int i = 4; i < TILE; i += 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) most[e] = fmaxf(most[e], s[i + e]);
                }
                const float here = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * c;
                if (j == plan.from[x]) {
                    m = here;
                } else if (__any_sync(~0u, here > m + SLACK)) {
                    const float next = fmaxf(m, here), back = m == next ? 1.f : exp2_of(m - next);
                    m = next;
                    l *= back;
#pragma unroll 1
                    for (int i = 0; i < DP; i += 32) {
                        float o[32];
                        load32(o, o_at + i);
                        wait_loads();
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(o[e] * back);
                        store16(o_at + i, w);
                        store16(o_at + i + 16, w + 16);
                    }
                }
                // nothing but -inf so far: weights of 0
                const float off = m == -INFINITY ? 0.f : RAISE - m;
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float2 v = fma2(make_float2(s[32 * i + 2 * e], s[32 * i + 2 * e + 1]), make_float2(c, c), make_float2(off, off));
                        v.x = exp2_of(v.x);
                        v.y = exp2_of(v.y);
                        sum[e & 1] = add2(sum[e & 1], v);
                        w[e] = two_16_bits<BF>(v.x, v.y);
                    }
                    store16(s_at + 16 * i, w);
                }
                l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                wait_stores();
                before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&sh.p_ready[x]);
            }
            if (!alive) break;
            const bool any = plan.from[x] < plan.to[x];
            if (!(alive = warp_wait(&sh.plan_cleared[seen % PLANS], (seen / PLANS) & 1))) break;
            const bool bad = sh.plan[seen % PLANS].bad != 0;
            if (any) {
                if (!(alive = warp_wait(&sh.o_full[x], outputs & 1))) break;
                ++outputs;
                after_sync();
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            uint16_t *const out = static_cast<uint16_t *>(a.out) + int64_t(plan.row0 + at) * a.out_row + (plan.head0 + head) * a.out_head;
#pragma unroll 1
            for (int i = 0; i < DP; i += 32) {
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
                        const int first = part == 0 ? low : max(low, max(plan.all_to + 1, plan.all_from)), end = part == 0 ? min(high + 1, plan.all_from) : high + 1;
                        for (int j = first; j < end; ++j) {
                            const int page = page_of(a.cache, a.seq, plan.b, j);
                            if (page < 0) continue;
                            const uint16_t *const row = reinterpret_cast<const uint16_t *>(a.cache.v + page * a.cache.page_stride + plan.kv * a.cache.head_stride +
                                                                                           (j & ((1 << a.cache.page_shift) - 1)) * a.cache.row_stride);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (i + e < a.cache.d) {
                                    const float v = BF ? __uint_as_float(uint32_t(row[i + e]) << 16) : __half2float(__ushort_as_half(row[i + e]));
                                    if (!(v - v == 0.f)) o[e] += v;
                                }
                        }
                    }
                }
                if (mine) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = two_16_bits<BF>(o[2 * e], o[2 * e + 1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (i + 8 * e >= a.cache.d) break;
                        if (p.wide) {
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
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == PLAN_WARP) {
            // ---- what there is to do ---------------------------------------------------------------------------------------
            int round = 0;
            for (int n = 0;; ++n) {
                Plan plan;
                const bool some = next_plan(p, round, plan);
                ++round;
                if (n >= PLANS && !warp_wait(&sh.plan_empty[n % PLANS], (n / PLANS - 1) & 1)) break;
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
            Plan plan;
            // the box that lane i brings of tile j: its page, or one past the last, which reads as zeros
            const auto page_at = [&](int j) {
                const int64_t row = int64_t(j) * TILE + lane * p.box;
                int page = -1;
                if (lane < boxes && row <= plan.last) page = page_of(a.cache, a.seq, plan.b, row);
                return page < 0 ? int(a.cache.pages) : page;
            };
            while (alive && take(plan)) {
                const int first = plan.first(), end = plan.end();
                if (first < end) {
                    int page = page_at(first);
                    if (blocks > 0 && !(alive = warp_wait(&sh.q_empty, (blocks - 1) & 1))) break;
                    ++blocks;
                    if (elected()) {
                        const int used = plan.count > p.tokens ? 2 : 1;
                        bar_expect(&sh.q_full, uint32_t(used * S::BLOCKS * p.heads * p.tokens * 128));
                        for (int x = 0; x < used; ++x)
                            for (int i = 0; i < S::BLOCKS; ++i) box3(q_to + x * S::BYTES + i * BLOCK, &q_map, 64 * i, plan.head0, plan.row0 + x * p.tokens, &sh.q_full);
                    }
                    __syncwarp();
                    for (int j = first; j < end && alive; ++j) {
                        const int pages = page;
                        if (j + 1 < end) page = page_at(j + 1);
                        for (int which = 0; which < 2; ++which, ++tiles) {
                            const int stage = tiles % STAGES;
                            if (tiles >= STAGES && !(alive = warp_wait(&sh.empty[stage], (tiles / STAGES - 1) & 1))) break;
                            if (elected()) bar_expect(&sh.full[stage], S::BYTES);
                            __syncwarp();
                            for (int i = 0; i < boxes; ++i) {
                                const int number = __shfl_sync(~0u, pages, i), slot = (j * TILE + i * p.box) & ((1 << a.cache.page_shift) - 1);
                                if (elected()) {
#pragma unroll
                                    for (int k = 0; k < S::BLOCKS; ++k)
                                        box4(ring_to + stage * S::BYTES + k * BLOCK + i * p.box * 128, which ? &v_map : &k_map, 64 * k, slot, plan.kv, number, &sh.full[stage]);
                                }
                                __syncwarp();
                            }
                        }
                    }
                }
                if (alive) give_back();
            }
            // what has been brought is used up, and the arrivals that say so are here, before the CTA is left
            for (int n = tiles > STAGES ? tiles - STAGES : 0; n < tiles && alive; ++n) alive = warp_wait(&sh.empty[n % STAGES], (n / STAGES) & 1);
            if (alive && blocks > 0) alive = warp_wait(&sh.q_empty, (blocks - 1) & 1);
            if (!alive)
                for (int i = 0; i < 10000; ++i) __nanosleep(100);        // after giving up: the copies under way end before the CTA does
        } else if (warp == MMA_WARP) {
            // ---- products ----------------------------------------------------------------------------------------------------
            constexpr uint32_t format = BF ? 1 : 0;
            constexpr uint32_t both = (1u << 4) | (format << 7) | (format << 10) | (uint32_t(TILE >> 4) << 24);
            constexpr uint32_t s_desc = both | (uint32_t(TILE >> 3) << 17), o_desc = both | (1u << 16) | (uint32_t(DP >> 3) << 17);
            const uint32_t ring_from = smem_addr(ring), q_from = smem_addr(q_at);
            int tiles = 0, blocks = 0;
            uint32_t ready[2] = {0, 0}, outputs[2] = {0, 0};
            bool alive = true;
            Plan plan;
            // S of tile x and K in `stage`
            const auto scores = [&](int x, int stage) {
                if (elected()) {
                    const uint64_t qd = rows_operand(q_from + x * S::BYTES), kd = rows_operand(ring_from + stage * S::BYTES);
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k) {
                        const int at = (k / 4) * (BLOCK / 16) + (k % 4) * 2;
                        mma_ss(tmem + x * TILE, qd + at, kd + at, s_desc, k > 0);
                    }
                    commit(&sh.s_full[x]);
                }
                __syncwarp();
            };
            while (alive && take(plan)) {
                const int first = plan.first(), end = plan.end();
                if (first < end) {
                    const auto active = [&](int x, int j) { return j >= plan.from[x] && j < plan.to[x]; };
                    if (!(alive = warp_wait(&sh.q_full, blocks & 1))) break;
                    ++blocks;
                    if (!(alive = warp_wait(&sh.full[tiles % STAGES], (tiles / STAGES) & 1))) break;
                    after_sync();
                    for (int x = 0; x < 2; ++x)
                        if (active(x, first)) scores(x, tiles % STAGES);
                    if (elected()) {
                        commit(&sh.empty[tiles % STAGES]);
                        if (first + 1 == end) commit(&sh.q_empty);
                    }
                    __syncwarp();
                    ++tiles;
                    for (int j = first; j < end && alive; ++j) {
                        const int v_stage = tiles % STAGES, k_stage = (tiles + 1) % STAGES;
                        if (!(alive = warp_wait(&sh.full[v_stage], (tiles / STAGES) & 1))) break;
                        if (plan.ragged(j) && !(alive = warp_wait(&sh.cleared[v_stage], (tiles / STAGES) & 1))) break;
                        const bool more = j + 1 < end;
                        bool k_here = false;
                        for (int x = 0; x < 2 && alive; ++x) {
                            if (active(x, j)) {
                                if (j == plan.from[x] && outputs[x] > 0 && !(alive = warp_wait(&sh.o_free[x], (outputs[x] - 1) & 1))) break;
                                if (!(alive = warp_wait(&sh.p_ready[x], ready[x] & 1))) break;
                                ++ready[x];
                                after_sync();
                                if (elected()) {
                                    const uint64_t vd = columns_operand(ring_from + v_stage * S::BYTES, BLOCK);
#pragma unroll
                                    for (int k = 0; k < TILE / 16; ++k) mma_ts(tmem + 2 * TILE + x * DP, tmem + x * TILE + k * 8, vd + k * (16 * 128 / 16), o_desc, j > plan.from[x] || k > 0);
                                    if (j + 1 == plan.to[x]) commit(&sh.o_full[x]);
                                }
                                __syncwarp();
                                if (j + 1 == plan.to[x]) ++outputs[x];
                            }
                            if (more && active(x, j + 1)) {
                                if (!k_here && !(alive = warp_wait(&sh.full[k_stage], ((tiles + 1) / STAGES) & 1))) break;
                                k_here = true;
                                after_sync();
                                scores(x, k_stage);
                            }
                        }
                        if (!alive) break;
                        if (elected()) {
                            commit(&sh.empty[v_stage]);
                            if (more) commit(&sh.empty[k_stage]);
                            if (j + 2 == end) commit(&sh.q_empty);
                        }
                        __syncwarp();
                        tiles += more ? 2 : 1;
                    }
                }
                if (alive) give_back();
            }
        } else {
            // ---- rows of V that not all tokens see -------------------------------------------------------------------------------
            int tiles = 0;
            bool alive = true;
            Plan plan;
            while (alive && take(plan)) {
                const int first = plan.first(), end = plan.end();
                bool bad = false;
                for (int n = 0; n < 2 * (end - first) && alive; ++n, ++tiles) {
                    const int stage = tiles % STAGES, j = first + n / 2;
                    if (!(alive = warp_wait(&sh.full[stage], (tiles / STAGES) & 1))) break;
                    if ((n & 1) && plan.ragged(j)) {
                        uint8_t *const v = ring + stage * S::BYTES;
#pragma unroll 1
                        for (int i = lane; i < S::BLOCKS * TILE * 8; i += 32) {
                            const int row = (i >> 3) & (TILE - 1), number = j * TILE + row;
                            uint4 *const at = reinterpret_cast<uint4 *>(v) + i;
                            if (number >= plan.all_from && number <= plan.all_to) continue;
                            if (number < plan.sees_from || number > plan.sees_to) {
                                *at = make_uint4(0, 0, 0, 0);
                                continue;
                            }
                            // exponents of all ones
                            constexpr uint32_t ones = BF ? 0x7f807f80u : 0x7c007c00u;
                            uint4 u = *at;
                            uint32_t *const w = reinterpret_cast<uint32_t *>(&u);
                            bool here = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t e = __vcmpeq2(w[k] & ones, ones);
                                here |= e != 0;
                                w[k] &= ~e;
                            }
                            if (here) {
                                *at = u;
                                bad = true;
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
bool encode(CUtensorMap *map, const void *at, int dims, const cuuint64_t *sizes, const cuuint64_t *strides, const cuuint32_t *box)
{
    const EncodeTiled f = encode_tiled();
    const cuuint32_t steps[4] = {1, 1, 1, 1};
    return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, cuuint32_t(dims), const_cast<void *>(at), sizes, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF, int DP> cudaError_t launch(const Args &p, const CUtensorMap &q, const CUtensorMap &k, const CUtensorMap &v, int ctas, cudaStream_t stream)
{
    const auto kernel = prompt_kernel<BF, DP>;
    // The warps' shares of registers come out of what the block has from the start: 256 threads of 216 and 128 of 72.
    static const bool enough = [&] {
        cudaFuncAttributes attr;
        return cudaFuncGetAttributes(&attr, kernel) == cudaSuccess && attr.numRegs * THREADS >= 256 * 216 + 128 * 72;
    }();
    if (!enough) return cudaErrorInvalidConfiguration;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<DP>::SMEM);
    if (e != cudaSuccess) return e;
    return launch_after(kernel, dim3(unsigned(ctas)), dim3(THREADS), Shape<DP>::SMEM, stream, dim3(1, 1), p, q, k, v);
}

}  // namespace
}  // namespace prompt

cudaError_t prompt_gave_up(int *flag)
{
    const int zero = 0;
    const cudaError_t e = cudaMemcpyFromSymbol(flag, prompt::g_gave_up, sizeof(int));
    return e != cudaSuccess || !*flag ? e : cudaMemcpyToSymbol(prompt::g_gave_up, &zero, sizeof(int));
}

int64_t prompt_workspace(const AttentionArgs &, int) { return 0; }

cudaError_t launch_prompt(const AttentionArgs &given, int sm_count, cudaStream_t stream)
{
    if (given.cache.type == STRASSEN_E4M3) return launch_simple(given, stream);
    prompt::Args p;
    p.a = given;
    AttentionArgs &a = p.a;
    p.group = a.heads / a.cache.kv_heads;
    p.blocks = (p.group + prompt::TILE - 1) / prompt::TILE;
    p.heads = (p.group + p.blocks - 1) / p.blocks;
    p.tokens = prompt::TILE / p.heads;
    const int page = 1 << a.cache.page_shift;
    p.box = page < prompt::TILE ? page : prompt::TILE;
    p.wide = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && a.out_row % 8 == 0 && a.out_head % 8 == 0;
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
        const cuuint32_t box[4] = {64, cuuint32_t(p.box), 1, 1};
        if (!prompt::encode(&k, a.cache.k, 4, sizes, strides, box) || !prompt::encode(&v, a.cache.v, 4, sizes, strides, box)) return cudaErrorInvalidValue;
    } else {
        // rows that are not there read as zeros, whose mean is what a token that sees nothing gets
        a.seq.width = 0;
        k = v = q;
    }
    const int64_t items = (a.seq.tokens / (2 * p.tokens) + a.seq.batch) * a.cache.kv_heads * p.blocks;
    const int ctas = int(items < sm_count ? items : sm_count);
    if (a.type == STRASSEN_BF16) return a.cache.d <= 64 ? prompt::launch<true, 64>(p, q, k, v, ctas, stream) : prompt::launch<true, 128>(p, q, k, v, ctas, stream);
    return a.cache.d <= 64 ? prompt::launch<false, 64>(p, q, k, v, ctas, stream) : prompt::launch<false, 128>(p, q, k, v, ctas, stream);
}

}  // namespace strassen
