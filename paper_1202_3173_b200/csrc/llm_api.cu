// Host entry points of the feed-forward operators (declared in include/strassen_b200.h): argument checking and launches.
// Nothing here allocates device memory, waits for the device or keeps anything of a call for the next one.
#include "strassen_b200.h"

#include <new>
#include <string>

#include "attention.h"
#include "entry.h"
#include "llm.h"

using namespace strassen;
using namespace strassen::entry;

struct strassen_w4 {
    W4Layout lay;
    uint8_t *packed = nullptr;
};

namespace {

// What the two row operators check alike.
int check_rows(const RowArgs &a, const char *first, const char *second)
{
    if (a.m < 0 || a.k < 1 || a.m > kMaxExtent || a.k > kMaxExtent) return fail(STRASSEN_INVALID_ARG, "rows must be 0 .. 2^30 and their length 1 .. 2^30");
    if (a.type != STRASSEN_BF16 && a.type != STRASSEN_F16 && a.type != STRASSEN_F32)
        return fail(STRASSEN_INVALID_ARG, "the input type must be STRASSEN_BF16, STRASSEN_F16 or STRASSEN_F32");
    if (a.m == 0) return STRASSEN_OK;
    const int t = type_size(a.type);
    if (!a.a || !a.q || !a.scale) return fail(STRASSEN_INVALID_ARG, std::string(first) + ", q and scale must be non-NULL");
    if (a.m > 1 && (a.lda < a.k || a.ldq < a.k || (a.b && a.ldb < a.k) || a.lda > kMaxLd || a.ldb > kMaxLd || a.ldq > kMaxLd))
        return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    if (misaligned(a.a, t) || misaligned(a.b, t) || misaligned(a.scale, 4))
        return fail(STRASSEN_MISALIGNED, std::string(first) + ", " + second + " and scale must be aligned to their elements");
    const Range q = rows_of(a.q, a.m, a.k, a.ldq, 1), s = rows_of(a.scale, 1, a.m, a.m, 4), x = rows_of(a.a, a.m, a.k, a.lda, t),
                b = rows_of(a.b, a.b ? a.m : 0, a.k, a.ldb, t);
    if (overlap(q, x) || overlap(q, b) || overlap(s, x) || overlap(s, b) || overlap(q, s))
        return fail(STRASSEN_ALIAS, "q and scale must not overlap the inputs or each other");
    return STRASSEN_OK;
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

}  // namespace

extern "C" int strassen_rms_norm_quant(int64_t m, int64_t k, int type, const void *x, int64_t ldx, const void *residual, int64_t ldr,
                                       const void *weight, float eps, void *sum, int64_t lds, void *q, int64_t ldq, float *scale, void *stream)
{
    set_last_error("");
    const RowArgs a = {m, k, type, x, residual, ldx, ldr, weight, eps, sum, lds, static_cast<uint8_t *>(q), ldq, scale};
    int rc = check_rows(a, "x", "residual");
    if (rc != STRASSEN_OK) return rc;
    if (!(eps >= 0.f)) return fail(STRASSEN_INVALID_ARG, "eps must not be negative");
    if (m == 0) return STRASSEN_OK;
    const int t = type_size(type);
    if (!weight) return fail(STRASSEN_INVALID_ARG, "weight must be non-NULL");
    if (!residual != !sum) return fail(STRASSEN_INVALID_ARG, "residual and sum go together: both or neither");
    if (misaligned(weight, t) || misaligned(sum, t)) return fail(STRASSEN_MISALIGNED, "weight and sum must be aligned to their elements");
    if (sum && m > 1 && (lds < k || lds > kMaxLd)) return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    const Range w = rows_of(weight, 1, k, k, t), h = rows_of(sum, sum ? m : 0, k, lds, t), qr = rows_of(q, m, k, ldq, 1), sr = rows_of(scale, 1, m, m, 4);
    if (overlap(w, qr) || overlap(w, sr) || overlap(w, h) || overlap(h, qr) || overlap(h, sr))
        return fail(STRASSEN_ALIAS, "the outputs must not overlap weight or each other");
    if ((overlap(h, rows_of(x, m, k, ldx, t)) && !same_rows(sum, lds, x, ldx, m)) ||
        (overlap(h, rows_of(residual, residual ? m : 0, k, ldr, t)) && !same_rows(sum, lds, residual, ldr, m)))
        return fail(STRASSEN_ALIAS, "sum may take the place of x or of residual, but not overlap them otherwise");
    int sms = 0;
    if ((rc = current_device(&sms)) != STRASSEN_OK) return rc;
    const cudaError_t e = launch_rms_norm_quant(a, sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" int strassen_silu_mul_quant(int64_t m, int64_t k, int type, const void *gate, int64_t ldg, const void *up, int64_t ldu, void *q,
                                       int64_t ldq, float *scale, void *stream)
{
    set_last_error("");
    const RowArgs a = {m, k, type, gate, up, ldg, ldu, nullptr, 0.f, nullptr, 0, static_cast<uint8_t *>(q), ldq, scale};
    int rc = check_rows(a, "gate", "up");
    if (rc != STRASSEN_OK) return rc;
    if (m == 0) return STRASSEN_OK;
    if (!up) return fail(STRASSEN_INVALID_ARG, "up must be non-NULL");
    int sms = 0;
    if ((rc = current_device(&sms)) != STRASSEN_OK) return rc;
    const cudaError_t e = launch_silu_mul_quant(a, sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" int strassen_route_experts(int64_t tokens, int64_t experts, int type, const void *logits, int64_t ld, const float *bias, int score, int groups,
                                      int top_groups, int top, int renormalize, float factor, int *ids, float *weights, void *stream)
{
    set_last_error("");
    if (tokens < 0 || tokens > kMaxExtent) return fail(STRASSEN_INVALID_ARG, "tokens must be 0 .. 2^30");
    if (experts < 1 || experts > kMostExperts) return fail(STRASSEN_INVALID_ARG, "experts must be 1 .. 1024");
    if (type != STRASSEN_BF16 && type != STRASSEN_F16 && type != STRASSEN_F32)
        return fail(STRASSEN_INVALID_ARG, "the logits' type must be STRASSEN_BF16, STRASSEN_F16 or STRASSEN_F32");
    if (score != STRASSEN_SOFTMAX && score != STRASSEN_SIGMOID) return fail(STRASSEN_INVALID_ARG, "the score must be STRASSEN_SOFTMAX or STRASSEN_SIGMOID");
    if (groups < 1 || groups > kMostGroups || experts % groups != 0 || top_groups < 1 || top_groups > groups)
        return fail(STRASSEN_INVALID_ARG, "groups must be 1 .. 32, divide the experts, and top_groups 1 .. groups");
    if (top < 1 || top > kMostTop || top > experts / groups * top_groups)
        return fail(STRASSEN_INVALID_ARG, "top must be 1 .. 32 and no more than the experts of top_groups groups");
    if (!(factor == factor)) return fail(STRASSEN_INVALID_ARG, "factor must be a number");
    if (tokens == 0) return STRASSEN_OK;
    if (!logits || !ids || !weights) return fail(STRASSEN_INVALID_ARG, "logits, ids and weights must be non-NULL");
    if (tokens > 1 && (ld < experts || ld > kMaxLd)) return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    const int t = type_size(type);
    if (misaligned(logits, t) || misaligned(bias, 4) || misaligned(ids, 4) || misaligned(weights, 4))
        return fail(STRASSEN_MISALIGNED, "logits, bias, ids and weights must be aligned to their elements");
    const Range l = rows_of(logits, tokens, experts, ld, t), b = rows_of(bias, bias ? 1 : 0, experts, experts, 4), i = rows_of(ids, tokens, top, top, 4),
                w = rows_of(weights, tokens, top, top, 4);
    if (overlap(i, l) || overlap(i, b) || overlap(w, l) || overlap(w, b) || overlap(i, w)) return fail(STRASSEN_ALIAS, "ids and weights must not overlap the inputs or each other");
    int sms = 0, rc = current_device(&sms);
    if (rc != STRASSEN_OK) return rc;
    const RouteArgs a = {tokens, int(experts), type, logits, ld, bias, score == STRASSEN_SOFTMAX, groups, top_groups, top, renormalize != 0, factor, ids, weights, 0};
    const cudaError_t e = launch_route(a, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" strassen_w4 *strassen_w4_create(int64_t n, int64_t k, int group, int scale_type, int has_zeros)
{
    return strassen_w4_create_experts(1, n, k, group, scale_type, has_zeros);
}

extern "C" strassen_w4 *strassen_w4_create_experts(int64_t experts, int64_t n, int64_t k, int group, int scale_type, int has_zeros)
{
    set_last_error("");
    if (n < 1 || k < 1 || n > kMaxExtent || k > kMaxExtent) {
        fail(STRASSEN_INVALID_ARG, "n and k must be 1 .. 2^30");
        return nullptr;
    }
    if (experts < 1 || experts > kMostExperts) {
        fail(STRASSEN_INVALID_ARG, "experts must be 1 .. 1024");
        return nullptr;
    }
    if (group != 32 && group != 64 && group != 128) {
        fail(STRASSEN_INVALID_ARG, "the group must be 32, 64 or 128");
        return nullptr;
    }
    if (scale_type != STRASSEN_BF16 && scale_type != STRASSEN_F16) {
        fail(STRASSEN_INVALID_ARG, "scales must be STRASSEN_BF16 or STRASSEN_F16");
        return nullptr;
    }
    W4Layout l;
    l.n = n;
    l.k = k;
    l.experts = experts;
    l.group = group;
    l.scale_type = scale_type;
    l.has_zeros = has_zeros != 0;
    l.row_tiles = round_up(n, kW4Rows) / kW4Rows;
    l.depth_tiles = round_up(k, kW4Depth) / kW4Depth;
    const int64_t tiles = experts * l.row_tiles * l.depth_tiles;
    if (tiles > 0x7fffffff) {
        fail(STRASSEN_INVALID_ARG, "the matrices are too large (2^31 tiles of 128 x 128)");
        return nullptr;
    }
    l.tile_bytes = kW4NibbleBytes + kW4Depth / group * kW4Rows * (l.has_zeros ? 3 : 2);
    l.exponent_off = size_t(round_up(tiles * l.tile_bytes, 256));
    l.bytes = l.exponent_off + size_t(experts * l.row_tiles) * kW4Rows * 4;
    strassen_w4 *w = new (std::nothrow) strassen_w4;
    if (!w) {
        fail(STRASSEN_OUT_OF_MEMORY, "out of host memory");
        return nullptr;
    }
    w->lay = l;
    return w;
}

extern "C" void strassen_w4_destroy(strassen_w4 *w) { delete w; }

extern "C" size_t strassen_w4_bytes(const strassen_w4 *w) { return w ? w->lay.bytes : 0; }

extern "C" int strassen_w4_pack(strassen_w4 *w, const uint8_t *q, int64_t ldq, const void *scales, int64_t lds, const uint8_t *zeros, int64_t ldz,
                                void *packed, void *stream)
{
    set_last_error("");
    if (!w || !q || !scales || !packed) return fail(STRASSEN_INVALID_ARG, "the matrix, q, scales and packed must be non-NULL");
    const W4Layout &l = w->lay;
    if (!zeros != !l.has_zeros) return fail(STRASSEN_INVALID_ARG, "zero points must be given if, and only if, the matrix was created with them");
    const int64_t half = (l.k + 1) / 2, groups = (l.k + l.group - 1) / l.group;
    const int64_t rows = l.experts * l.n;
    if (rows > 1 && (ldq < half || lds < groups || (zeros && ldz < groups) || ldq > kMaxLd || lds > kMaxLd || ldz > kMaxLd))
        return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    if (misaligned(scales, 2)) return fail(STRASSEN_MISALIGNED, "scales must be 2-byte aligned");
    if (misaligned(packed, 256)) return fail(STRASSEN_MISALIGNED, "packed must be 256-byte aligned");
    const Range out = {reinterpret_cast<uintptr_t>(packed), reinterpret_cast<uintptr_t>(packed) + l.bytes};
    if (overlap(out, rows_of(q, rows, half, ldq, 1)) || overlap(out, rows_of(scales, rows, groups, lds, 2)) ||
        overlap(out, rows_of(zeros, zeros ? rows : 0, groups, ldz, 1)))
        return fail(STRASSEN_ALIAS, "packed overlaps an input");
    int sms = 0, rc = current_device(&sms);
    if (rc != STRASSEN_OK) return rc;
    const W4PackArgs a = {l, q, ldq, scales, lds, zeros, ldz, static_cast<uint8_t *>(packed)};
    const cudaError_t e = launch_w4_pack(a, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_fail(e, "kernel launch");
    w->packed = a.packed;
    return STRASSEN_OK;
}

extern "C" size_t strassen_w4_workspace_bytes(const strassen_w4 *w, int64_t m, int type, const void *x, int64_t ldx)
{
    if (!w || m <= kThinRows || m > kMaxExtent) return 0;
    W4Args a = {};
    a.lay = w->lay;
    a.m = m;
    a.type = type;
    a.x = x;
    a.ldx = ldx;
    return size_t(w4_tiles_workspace(a));
}

extern "C" int strassen_w4_matmul(const strassen_w4 *w, int64_t m, int type, const void *x, int64_t ldx, const float *x_scale, int out_type,
                                  void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    set_last_error("");
    if (!w) return fail(STRASSEN_INVALID_ARG, "the matrix must be non-NULL");
    if (!w->packed) return fail(STRASSEN_INVALID_ARG, "the matrix has not been laid out (strassen_w4_pack)");
    const W4Layout &l = w->lay;
    if (l.experts != 1) return fail(STRASSEN_INVALID_ARG, "several matrices: strassen_w4_experts multiplies by those that ids name");
    if (m < 0 || m > kMaxExtent) return fail(STRASSEN_INVALID_ARG, "m must be 0 .. 2^30");
    if (type != STRASSEN_BF16 && type != STRASSEN_F16 && type != STRASSEN_E4M3)
        return fail(STRASSEN_INVALID_ARG, "the type of x must be STRASSEN_BF16, STRASSEN_F16 or STRASSEN_E4M3");
    if (out_type != STRASSEN_BF16 && out_type != STRASSEN_F16) return fail(STRASSEN_INVALID_ARG, "the output type must be STRASSEN_BF16 or STRASSEN_F16");
    if (m == 0) return STRASSEN_OK;
    if (!x || !out) return fail(STRASSEN_INVALID_ARG, "x and out must be non-NULL");
    if (m > 1 && (ldx < l.k || ldo < l.n || ldx > kMaxLd || ldo > kMaxLd))
        return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    const int t = type_size(type);
    if (misaligned(x, t) || misaligned(x_scale, 4) || misaligned(out, 2)) return fail(STRASSEN_MISALIGNED, "x, x_scale and out must be aligned to their elements");
    const Range o = rows_of(out, m, l.n, ldo, 2);
    const Range inputs[] = {rows_of(x, m, l.k, ldx, t), rows_of(x_scale, x_scale ? 1 : 0, m, m, 4),
                            {reinterpret_cast<uintptr_t>(w->packed), reinterpret_cast<uintptr_t>(w->packed) + l.bytes}};
    for (const Range &r : inputs)
        if (overlap(o, r)) return fail(STRASSEN_ALIAS, "out overlaps an input");
    int sms = 0, rc = current_device(&sms);
    if (rc != STRASSEN_OK) return rc;
    const W4Args a = {l, w->packed, m, type, x, ldx, x_scale, out_type, out, ldo, workspace, nullptr, 0, false, nullptr};
    const int64_t need = m > kThinRows ? w4_tiles_workspace(a) : 0;
    if (need > 0) {
        if (!workspace || workspace_bytes < size_t(need))
            return fail(STRASSEN_WORKSPACE_TOO_SMALL, "these rows need a workspace of " + std::to_string(need) + " bytes (strassen_w4_workspace_bytes)");
        if (misaligned(workspace, 256)) return fail(STRASSEN_MISALIGNED, "workspace must be 256-byte aligned");
        const Range ws = {reinterpret_cast<uintptr_t>(workspace), reinterpret_cast<uintptr_t>(workspace) + uintptr_t(need)};
        if (overlap(ws, o)) return fail(STRASSEN_ALIAS, "workspace overlaps another argument");
        for (const Range &r : inputs)
            if (overlap(ws, r)) return fail(STRASSEN_ALIAS, "workspace overlaps another argument");
    }
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = m <= kThinRows ? launch_w4_thin(a, sms, st) : launch_w4_tiles(a, sms, st);
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" size_t strassen_w4_experts_workspace_bytes(const strassen_w4 *w, int64_t tokens, int64_t top, int weighted)
{
    if (!w || tokens < 0 || top < 1 || top > kMostTop || tokens * top <= kThinIds || tokens > kMaxExtent / kMostTop) return 0;
    W4Args a = {};
    a.lay = w->lay;
    a.m = tokens;
    a.top = top;
    static const float some = 0.f;
    a.weights = weighted ? &some : nullptr;
    return size_t(w4_experts_workspace(a));
}

extern "C" int strassen_w4_experts(const strassen_w4 *w, int64_t tokens, int64_t top, const int *ids, int type, const void *x, int64_t ldx, int each,
                                   const float *x_scale, const float *weights, int out_type, void *out, int64_t ldo, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    set_last_error("");
    if (!w) return fail(STRASSEN_INVALID_ARG, "the matrices must be non-NULL");
    if (!w->packed) return fail(STRASSEN_INVALID_ARG, "the matrices have not been laid out (strassen_w4_pack)");
    const W4Layout &l = w->lay;
    if (tokens < 0 || tokens > kMaxExtent / kMostTop) return fail(STRASSEN_INVALID_ARG, "tokens must be 0 .. 2^25");
    if (top < 1 || top > kMostTop) return fail(STRASSEN_INVALID_ARG, "top must be 1 .. 32");
    if (type != STRASSEN_BF16 && type != STRASSEN_F16 && type != STRASSEN_E4M3)
        return fail(STRASSEN_INVALID_ARG, "the type of x must be STRASSEN_BF16, STRASSEN_F16 or STRASSEN_E4M3");
    if (out_type != STRASSEN_BF16 && out_type != STRASSEN_F16) return fail(STRASSEN_INVALID_ARG, "the output type must be STRASSEN_BF16 or STRASSEN_F16");
    if (tokens == 0) return STRASSEN_OK;
    if (!ids || !x || !out) return fail(STRASSEN_INVALID_ARG, "ids, x and out must be non-NULL");
    const int64_t pairs = tokens * top, x_rows = each ? pairs : tokens, out_rows = weights ? tokens : pairs;
    if ((x_rows > 1 && (ldx < l.k || ldx > kMaxLd)) || (out_rows > 1 && (ldo < l.n || ldo > kMaxLd)))
        return fail(STRASSEN_INVALID_ARG, "leading dimensions must be at least the rows' length");
    const int t = type_size(type);
    if (misaligned(x, t) || misaligned(x_scale, 4) || misaligned(out, 2) || misaligned(ids, 4) || misaligned(weights, 4))
        return fail(STRASSEN_MISALIGNED, "ids, x, x_scale, weights and out must be aligned to their elements");
    const Range inputs[] = {rows_of(x, x_rows, l.k, ldx, t), rows_of(x_scale, x_scale ? 1 : 0, x_rows, x_rows, 4), rows_of(ids, 1, pairs, pairs, 4),
                            rows_of(weights, weights ? 1 : 0, pairs, pairs, 4), {reinterpret_cast<uintptr_t>(w->packed), reinterpret_cast<uintptr_t>(w->packed) + l.bytes}};
    const Range o = rows_of(out, out_rows, l.n, ldo, 2);
    for (const Range &r : inputs)
        if (overlap(o, r)) return fail(STRASSEN_ALIAS, "out overlaps an input");
    int sms = 0, rc = current_device(&sms);
    if (rc != STRASSEN_OK) return rc;
    const W4Args a = {l, w->packed, tokens, type, x, ldx, x_scale, out_type, out, ldo, workspace, ids, top, each != 0, weights};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (pairs <= kThinIds) {
        e = launch_w4_thin(a, sms, st);
    } else {
        const size_t need = size_t(w4_experts_workspace(a));
        if (!workspace || workspace_bytes < need)
            return fail(STRASSEN_WORKSPACE_TOO_SMALL, "these rows need a workspace of " + std::to_string(need) + " bytes (strassen_w4_experts_workspace_bytes)");
        if (misaligned(workspace, 256)) return fail(STRASSEN_MISALIGNED, "workspace must be 256-byte aligned");
        const Range ws = {reinterpret_cast<uintptr_t>(workspace), reinterpret_cast<uintptr_t>(workspace) + need};
        if (overlap(ws, o)) return fail(STRASSEN_ALIAS, "workspace overlaps another argument");
        for (const Range &r : inputs)
            if (overlap(ws, r)) return fail(STRASSEN_ALIAS, "workspace overlaps another argument");
        e = launch_w4_experts_tiles(a, sms, st);
    }
    return e == cudaSuccess ? STRASSEN_OK : cuda_fail(e, "kernel launch");
}

extern "C" int strassen_device_status(void)
{
    set_last_error("");
    int sms = 0, rc = current_device(&sms);
    if (rc != STRASSEN_OK) return rc;
    cudaError_t e = cudaDeviceSynchronize();
    int tiles = 0, rows = 0, prompts = 0;
    if (e == cudaSuccess) e = read_gave_up(&tiles);
    if (e == cudaSuccess) e = rows8_gave_up(&rows);
    if (e == cudaSuccess) e = prompt_gave_up(&prompts);
    if (e != cudaSuccess) return cuda_fail(e, "reading the device's status");
    if (tiles || rows || prompts) return fail(STRASSEN_CUDA_ERROR, "a kernel gave up waiting for its own copies or tensor instructions; its results are not valid");
    return STRASSEN_OK;
}
