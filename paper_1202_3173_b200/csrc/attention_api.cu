// Host entry points of the attention operators (declared in include/strassen_b200.h): argument checking and launches.
// Nothing here allocates device memory, waits for the device or keeps anything of a call for the next one.
#include "strassen_b200.h"

#include <string>

#include "attention.h"
#include "entry.h"

using namespace strassen;
using namespace strassen::entry;

namespace {

bool wide_strides(uintptr_t at, int64_t row, int64_t head, int size) { return at % 16 == 0 && row * size % 16 == 0 && head * size % 16 == 0; }

// The memory of rows of heads as a byte range.
Range heads_of(const void *p, int64_t rows, int64_t row, int64_t heads, int64_t head, int d, int size)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return {lo, lo + (p && rows > 0 && heads > 0 ? uintptr_t((rows - 1) * row + (heads - 1) * head + d) * uintptr_t(size) : 0)};
}

int check_heads(const char *name, const void *p, int64_t rows, int64_t row, int64_t heads, int64_t head, int d)
{
    if (!p) return fail(STRASSEN_INVALID_ARG, std::string(name) + " must be non-NULL");
    if ((rows > 1 && (row < d || row > kMaxLd)) || (heads > 1 && (head < d || head > kMaxLd)))
        return fail(STRASSEN_INVALID_ARG, std::string("strides of ") + name + " must be at least head_size");
    if (misaligned(p, 2)) return fail(STRASSEN_MISALIGNED, std::string(name) + " must be aligned to its elements");
    return STRASSEN_OK;
}

int check_cache(const strassen_paged_cache *c, CacheArgs *to)
{
    if (!c) return fail(STRASSEN_INVALID_ARG, "the cache must be non-NULL");
    if (c->type != STRASSEN_BF16 && c->type != STRASSEN_F16 && c->type != STRASSEN_E4M3)
        return fail(STRASSEN_INVALID_ARG, "the cache's type must be STRASSEN_BF16, STRASSEN_F16 or STRASSEN_E4M3");
    const int t = type_size(c->type), d = c->head_size;
    if (d < 16 / t || d > kMostHeadSize || d * t % 16 != 0)
        return fail(STRASSEN_INVALID_ARG, "head_size must be a multiple of 8 (e4m3: 16) up to 128");
    if (c->kv_heads < 1 || c->kv_heads > kMostHeads) return fail(STRASSEN_INVALID_ARG, "kv_heads must be 1 .. 1024");
    if (c->page_size < kLeastPage || c->page_size > kMostPage || (c->page_size & (c->page_size - 1)))
        return fail(STRASSEN_INVALID_ARG, "page_size must be a power of two, 8 .. 1024");
    if (c->pages < 0 || c->pages > 0x7fffffff) return fail(STRASSEN_INVALID_ARG, "pages must be 0 .. 2^31 - 1");
    if (c->pages > 0 && (!c->k || !c->v)) return fail(STRASSEN_INVALID_ARG, "k and v of the cache must be non-NULL");
    const int64_t strides[] = {c->pages > 1 ? c->page_stride : d, c->kv_heads > 1 ? c->head_stride : d, c->row_stride};
    for (const int64_t s : strides) {
        if (s < d || s > kMaxLd) return fail(STRASSEN_INVALID_ARG, "strides of the cache must be at least head_size");
        if (s * t % 16 != 0) return fail(STRASSEN_MISALIGNED, "strides of the cache must be multiples of 16 bytes");
    }
    if (misaligned(c->k, 16) || misaligned(c->v, 16)) return fail(STRASSEN_MISALIGNED, "k and v of the cache must be 16-byte aligned");
    const bool scales = c->type == STRASSEN_E4M3;
    if (c->pages > 0 && (!c->k_scale != !scales || !c->v_scale != !scales)) return fail(STRASSEN_INVALID_ARG, "k_scale and v_scale must be given if, and only if, the cache is STRASSEN_E4M3");
    if (misaligned(c->k_scale, 4) || misaligned(c->v_scale, 4)) return fail(STRASSEN_MISALIGNED, "scales must be aligned to their elements");
    int shift = 0;
    while (1 << shift < c->page_size) ++shift;
    *to = {c->type, c->kv_heads, d, shift, c->pages, static_cast<uint8_t *>(c->k), static_cast<uint8_t *>(c->v), strides[0] * t, strides[1] * t, strides[2] * t, c->k_scale, c->v_scale};
    return STRASSEN_OK;
}

Range cache_range(const CacheArgs &c, const uint8_t *p)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    if (c.pages == 0) return {lo, lo};
    return {lo, lo + uintptr_t((c.pages - 1) * c.page_stride + (c.kv_heads - 1) * c.head_stride + ((int64_t(1) << c.page_shift) - 1) * c.row_stride + c.d * type_size(c.type))};
}

// n numbers of 32 bits one after another.
Range packed(const void *p, int64_t n)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return p && n > 0 ? Range{lo, lo + uintptr_t(n) * 4} : Range{0, 0};
}
Range scale_range(const CacheArgs &c, const float *p) { return packed(p, (c.pages * c.kv_heads) << c.page_shift); }

// Whether `r` lies over the scales, the table, the lengths or the offsets, all of which are read while results are written.
bool over_what_is_read(const Range &r, const CacheArgs &c, const SequenceArgs &s)
{
    return overlap(r, scale_range(c, c.k_scale)) || overlap(r, scale_range(c, c.v_scale)) || overlap(r, packed(s.table, s.batch > 0 && s.width > 0 ? (s.batch - 1) * s.ld_table + s.width : 0)) ||
           overlap(r, packed(s.lengths, s.batch)) || overlap(r, packed(s.offsets, s.batch + int64_t(1)));
}

// Rows of heads as the kernels see them.
struct RowsOfHeads {
    const void *p;
    int64_t rows, row, heads, head;
    Range range(int d) const { return heads_of(p, rows, row, heads, head, d, 2); }
};
bool same(const RowsOfHeads &a, const RowsOfHeads &b) { return a.p == b.p && a.row == b.row && a.head == b.head; }
// Whether an element is in both.  Rows of views of one wider tensor are the same distance apart and lie between one another: there it is found out exactly; else ranges of memory are compared.
bool share(const RowsOfHeads &a, const RowsOfHeads &b, int d)
{
    if (!a.p || !b.p || !overlap(a.range(d), b.range(d))) return false;
    if (a.row != b.row) return true;
    const int64_t apart = (int64_t(reinterpret_cast<uintptr_t>(b.p)) - int64_t(reinterpret_cast<uintptr_t>(a.p))) / 2, row = a.row, as_long = (a.heads - 1) * a.head + d, bs_long = (b.heads - 1) * b.head + d;
    if (row > 0 && as_long <= row && bs_long <= row) {
        const int64_t behind = (apart % row + row) % row;        // from the begin of a row of a to the next one of b
        if (behind >= as_long && behind + bs_long <= row) return false;
    }
    // A head of a row of b begins `off` behind one of the same row of a: whether they, or those of rows n apart, have an element in common.
    const auto meet = [&](int64_t off) {
        off = off < 0 ? -off : off;
        if (off < d) return true;
        const int64_t n = off < row || row == 0 ? 0 : off / row, left = off - n * row;
        return (left < d && n < a.rows) || (row > 0 && row - left < d && n + 1 < a.rows);
    };
    if (a.head == b.head) {
        for (int64_t i = 1 - a.heads; i < b.heads; ++i)
            if (meet(apart + i * a.head)) return true;
        return false;
    }
    for (int64_t i = 0; i < a.heads; ++i)
        for (int64_t j = 0; j < b.heads; ++j)
            if (meet(apart + j * b.head - i * a.head)) return true;
    return false;
}

int check_sequences(int64_t batch, const int *table, int64_t ld_table, int64_t width, const int *lengths, const int *offsets, int64_t tokens, SequenceArgs *to)
{
    if (batch < 0 || batch > kMaxExtent || width < 0 || width > kMaxExtent || tokens < 0 || tokens > kMaxExtent)
        return fail(STRASSEN_INVALID_ARG, "batch, width and tokens must be 0 .. 2^30");
    if (!offsets && tokens != batch) return fail(STRASSEN_INVALID_ARG, "without offsets there is one token for each sequence");
    if (batch > 0 && (!lengths || (width > 0 && !table))) return fail(STRASSEN_INVALID_ARG, "table and lengths must be non-NULL");
    if (batch > 1 && (ld_table < width || ld_table > kMaxLd)) return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    if (misaligned(table, 4) || misaligned(lengths, 4) || misaligned(offsets, 4)) return fail(STRASSEN_MISALIGNED, "table, lengths and offsets must be aligned to their elements");
    *to = {int(batch), int(width), table, ld_table, lengths, offsets, tokens};
    return STRASSEN_OK;
}

int check_types(int type, const CacheArgs &c)
{
    if (type != STRASSEN_BF16 && type != STRASSEN_F16) return fail(STRASSEN_INVALID_ARG, "the type of q must be STRASSEN_BF16 or STRASSEN_F16");
    if (c.type != STRASSEN_E4M3 && c.type != type) return fail(STRASSEN_INVALID_ARG, "a cache in 16 bits must have the type of q");
    return STRASSEN_OK;
}

// What the two attention entries check alike.
int check_attention(const strassen_paged_cache *cache, int64_t batch, const int *table, int64_t ld_table, int64_t width, const int *lengths, const int *offsets, int64_t tokens,
                    int type, int64_t heads, const void *q, int64_t q_row, int64_t q_head, void *out, int64_t out_row, int64_t out_head, float scale, int64_t window,
                    void *workspace, AttentionArgs *to)
{
    CacheArgs c;
    SequenceArgs s;
    int rc = check_cache(cache, &c);
    if (rc == STRASSEN_OK) rc = check_sequences(batch, table, ld_table, width, lengths, offsets, tokens, &s);
    if (rc == STRASSEN_OK) rc = check_types(type, c);
    if (rc != STRASSEN_OK) return rc;
    if (heads < 1 || heads > kMostHeads || heads % c.kv_heads != 0) return fail(STRASSEN_INVALID_ARG, "heads must be a multiple of kv_heads, 1 .. 1024");
    if (!(scale - scale == 0.f)) return fail(STRASSEN_INVALID_ARG, "scale must be a finite number");
    if (window < 0) return fail(STRASSEN_INVALID_ARG, "window must not be negative");
    if (tokens > 0) {
        rc = check_heads("q", q, tokens, q_row, heads, q_head, c.d);
        if (rc == STRASSEN_OK) rc = check_heads("out", out, tokens, out_row, heads, out_head, c.d);
        if (rc != STRASSEN_OK) return rc;
        const Range o = heads_of(out, tokens, out_row, heads, out_head, c.d, 2);
        if (overlap(o, heads_of(q, tokens, q_row, heads, q_head, c.d, 2)) || overlap(o, cache_range(c, c.k)) || overlap(o, cache_range(c, c.v)) || over_what_is_read(o, c, s))
            return fail(STRASSEN_ALIAS, "out overlaps another argument");
    }
    *to = {c, s, type, int(heads), {q, tokens > 1 ? q_row : 0, heads > 1 ? q_head : 0}, out, tokens > 1 ? out_row : 0, heads > 1 ? out_head : 0, scale,
           window > 0x7fffffff ? 0x7fffffff : int(window), workspace};
    return STRASSEN_OK;
}

int check_workspace(const AttentionArgs &a, int64_t need, size_t given, const char *which)
{
    if (need == 0) return STRASSEN_OK;
    if (!a.workspace || given < size_t(need)) return fail(STRASSEN_WORKSPACE_TOO_SMALL, "a workspace of " + std::to_string(need) + " bytes is needed (" + which + ")");
    if (misaligned(a.workspace, 256)) return fail(STRASSEN_MISALIGNED, "workspace must be 256-byte aligned");
    const uintptr_t lo = reinterpret_cast<uintptr_t>(a.workspace);
    const Range ws = {lo, lo + uintptr_t(need)};
    if (overlap(ws, heads_of(a.out, a.seq.tokens, a.out_row, a.heads, a.out_head, a.cache.d, 2)) ||
        overlap(ws, heads_of(a.q.p, a.seq.tokens, a.q.row, a.heads, a.q.head, a.cache.d, 2)) || overlap(ws, cache_range(a.cache, a.cache.k)) || overlap(ws, cache_range(a.cache, a.cache.v)) ||
        over_what_is_read(ws, a.cache, a.seq))
        return fail(STRASSEN_ALIAS, "workspace overlaps another argument");
    return STRASSEN_OK;
}

// Sizes alone, for the workspace queries.
bool sizes_only(const strassen_paged_cache *cache, int64_t batch, int64_t heads, int64_t width, int64_t tokens, int64_t window, AttentionArgs *to)
{
    CacheArgs c = {};
    if (check_cache(cache, &c) != STRASSEN_OK || batch < 0 || batch > kMaxExtent || width < 0 || width > kMaxExtent || tokens < 0 || tokens > kMaxExtent || window < 0 ||
        heads < 1 || heads > kMostHeads || heads % c.kv_heads != 0)
        return false;
    *to = {};
    to->cache = c;
    to->seq.batch = int(batch);
    to->seq.width = int(width);
    to->seq.tokens = tokens;
    to->heads = int(heads);
    to->window = window > 0x7fffffff ? 0x7fffffff : int(window);
    return true;
}

}  // namespace

extern "C" int strassen_rotate_append(const strassen_paged_cache *cache, int64_t batch, const int *table, int64_t ld_table, int64_t width, const int *lengths,
                                      const int *offsets, int64_t tokens, int type, int64_t heads, const void *q, int64_t q_row, int64_t q_head, const void *k,
                                      int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head, void *out, int64_t out_row, int64_t out_head,
                                      const float *frequencies, int rotary, int interleaved, void *stream)
{
    set_last_error("");
    AppendArgs a = {};
    int rc = check_cache(cache, &a.cache);
    if (rc == STRASSEN_OK) rc = check_sequences(batch, table, ld_table, width, lengths, offsets, tokens, &a.seq);
    if (rc == STRASSEN_OK) rc = check_types(type, a.cache);
    if (rc != STRASSEN_OK) return rc;
    const int d = a.cache.d, kv = a.cache.kv_heads;
    if (heads < 0 || heads > kMostHeads) return fail(STRASSEN_INVALID_ARG, "heads must be 0 .. 1024");
    if (rotary < 0 || rotary > d || rotary % 2 != 0) return fail(STRASSEN_INVALID_ARG, "rotary must be even, 0 .. head_size");
    if (!frequencies != (rotary == 0)) return fail(STRASSEN_INVALID_ARG, "frequencies must be given if, and only if, rotary is not 0");
    if (misaligned(frequencies, 4)) return fail(STRASSEN_MISALIGNED, "frequencies must be aligned to their elements");
    if (heads == 0 && (q || out)) return fail(STRASSEN_INVALID_ARG, "q and out must be NULL for 0 heads");
    if (batch == 0 || tokens == 0) return STRASSEN_OK;
    if (heads > 0) {
        rc = check_heads("q", q, tokens, q_row, heads, q_head, d);
        if (rc == STRASSEN_OK) rc = check_heads("out", out, tokens, out_row, heads, out_head, d);
    }
    if (rc == STRASSEN_OK) rc = check_heads("k", k, tokens, k_row, kv, k_head, d);
    if (rc == STRASSEN_OK) rc = check_heads("v", v, tokens, v_row, kv, v_head, d);
    if (rc != STRASSEN_OK) return rc;
    a.type = type;
    a.heads = int(heads);
    const int64_t many = tokens > 1, many_heads = heads > 1, many_kv = kv > 1;
    a.q = {q, many * q_row, many_heads * q_head};
    a.k = {k, many * k_row, many_kv * k_head};
    a.v = {v, many * v_row, many_kv * v_head};
    a.out = out;
    a.out_row = many * out_row;
    a.out_head = many_heads * out_head;
    a.frequencies = frequencies;
    a.rotary = rotary;
    a.interleaved = interleaved != 0;
    a.wide = wide_strides(reinterpret_cast<uintptr_t>(k), a.k.row, a.k.head, 2) && wide_strides(reinterpret_cast<uintptr_t>(v), a.v.row, a.v.head, 2) &&
             wide_strides(reinterpret_cast<uintptr_t>(q), a.q.row, a.q.head, 2) && wide_strides(reinterpret_cast<uintptr_t>(out), a.out_row, a.out_head, 2);
    const CacheArgs &c = a.cache;
    const RowsOfHeads o = {out, tokens, a.out_row, heads, a.out_head}, qs = {q, tokens, a.q.row, heads, a.q.head}, ks = {k, tokens, a.k.row, kv, a.k.head}, vs = {v, tokens, a.v.row, kv, a.v.head};
    const Range turns = packed(frequencies, rotary / 2);
    for (const Range &f : {cache_range(c, c.k), cache_range(c, c.v), scale_range(c, c.k_scale), scale_range(c, c.v_scale)})
        for (const Range &r : {qs.range(d), ks.range(d), vs.range(d), o.range(d), turns, packed(a.seq.table, width > 0 ? (batch - 1) * ld_table + width : 0), packed(lengths, batch), packed(offsets, batch + 1)})
            if (overlap(f, r)) return fail(STRASSEN_ALIAS, "the cache overlaps another argument");
    if (c.pages > 0 && (c.k == c.v || overlap(scale_range(c, c.k_scale), scale_range(c, c.v_scale)))) return fail(STRASSEN_ALIAS, "keys and values of the cache are in the same place");
    if (overlap(o.range(d), turns) || over_what_is_read(o.range(d), c, a.seq)) return fail(STRASSEN_ALIAS, "out overlaps another argument");
    if (!same(o, qs) && share(o, qs, d)) return fail(STRASSEN_ALIAS, "out overlaps q; it may be q itself, with its strides");
    if (share(o, ks, d) || share(o, vs, d)) return fail(STRASSEN_ALIAS, "out overlaps k or v");
    int sms = 0;
    if ((rc = current_device(&sms)) != STRASSEN_OK) return rc;
    const cudaError_t e = launch_append(a, sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" int strassen_decode_attention(const strassen_paged_cache *cache, int64_t batch, const int *table, int64_t ld_table, int64_t width, const int *lengths,
                                         int type, int64_t heads, const void *q, int64_t q_row, int64_t q_head, void *out, int64_t out_row, int64_t out_head,
                                         float scale, int64_t window, void *workspace, size_t workspace_bytes, void *stream)
{
    set_last_error("");
    AttentionArgs a;
    int rc = check_attention(cache, batch, table, ld_table, width, lengths, nullptr, batch, type, heads, q, q_row, q_head, out, out_row, out_head, scale, window, workspace, &a);
    if (rc != STRASSEN_OK || batch == 0) return rc;
    int sms = 0;
    if ((rc = current_device(&sms)) != STRASSEN_OK) return rc;
    if ((rc = check_workspace(a, decode_workspace(a, sms), workspace_bytes, "strassen_decode_attention_workspace_bytes")) != STRASSEN_OK) return rc;
    const cudaError_t e = launch_decode(a, sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" size_t strassen_decode_attention_workspace_bytes(const strassen_paged_cache *cache, int64_t batch, int64_t heads, int64_t width)
{
    AttentionArgs a;
    int sms = 0;
    if (!sizes_only(cache, batch, heads, width, batch, 0, &a) || current_device(&sms) != STRASSEN_OK) return 0;
    return size_t(decode_workspace(a, sms));
}

extern "C" int strassen_prompt_attention(const strassen_paged_cache *cache, int64_t batch, const int *table, int64_t ld_table, int64_t width, const int *lengths,
                                         const int *offsets, int64_t tokens, int type, int64_t heads, const void *q, int64_t q_row, int64_t q_head, void *out,
                                         int64_t out_row, int64_t out_head, float scale, int64_t window, void *workspace, size_t workspace_bytes, void *stream)
{
    set_last_error("");
    AttentionArgs a;
    int rc = check_attention(cache, batch, table, ld_table, width, lengths, offsets, tokens, type, heads, q, q_row, q_head, out, out_row, out_head, scale, window, workspace, &a);
    if (rc != STRASSEN_OK) return rc;
    if (batch > 0 && !offsets) return fail(STRASSEN_INVALID_ARG, "offsets must be non-NULL");
    if (batch == 0 || tokens == 0) return STRASSEN_OK;
    if (!wide_strides(reinterpret_cast<uintptr_t>(q), a.q.row, a.q.head, 2)) return fail(STRASSEN_MISALIGNED, "q must be 16-byte aligned, with strides that are multiples of 16 bytes");
    int sms = 0;
    if ((rc = current_device(&sms)) != STRASSEN_OK) return rc;
    if (!prompt_takes(a, sms)) return fail(STRASSEN_INVALID_ARG, "too many tokens and heads for one call");
    if ((rc = check_workspace(a, prompt_workspace(a, sms), workspace_bytes, "strassen_prompt_attention_workspace_bytes")) != STRASSEN_OK) return rc;
    const cudaError_t e = launch_prompt(a, sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" size_t strassen_prompt_attention_workspace_bytes(const strassen_paged_cache *cache, int64_t batch, int64_t heads, int64_t width, int64_t tokens, int64_t window)
{
    AttentionArgs a;
    int sms = 0;
    if (!sizes_only(cache, batch, heads, width, tokens, window, &a) || current_device(&sms) != STRASSEN_OK) return 0;
    return size_t(prompt_workspace(a, sms));
}
