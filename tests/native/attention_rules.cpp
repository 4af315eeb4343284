// Host-side check of the rules by which the attention operators choose their kernels, built with AddressSanitizer and UBSan by tests/test_attention_rules_host.py.
// Prints "ok <checks>" or the first violation.
#include <cstdio>
#include <cstdlib>

#include "attention.h"

using namespace strassen;

static long long g_checks = 0;
#define CHECK(x)                                                   \
    do {                                                           \
        ++g_checks;                                                \
        if (!(x)) {                                                \
            printf("FAIL line %d: %s\n", __LINE__, #x);            \
            exit(1);                                               \
        }                                                          \
    } while (0)

// A cache as the entry points hand it on: the strides of dimensions of one are head_size.
static CacheArgs cache(int64_t pages, int kv, int page_shift, int d, int size, int64_t row)
{
    CacheArgs c = {};
    c.kv_heads = kv;
    c.d = d;
    c.page_shift = page_shift;
    c.pages = pages;
    c.row_stride = row * size;
    c.head_stride = (kv > 1 ? row << page_shift : d) * size;
    c.page_stride = (pages > 1 ? (row << page_shift) * kv : d) * size;
    return c;
}

static void rows()
{
    for (int64_t pages : {1, 2, 1000})
        for (int kv : {1, 2, 8})
            for (int shift = 3; shift <= 10; ++shift)
                for (int d : {64, 80, 128})
                    for (int64_t row : {int64_t(d), int64_t(d) + 16}) {
                        CacheArgs c = cache(pages, kv, shift, d, 2, row);
                        CHECK(rows_in_a_row(c));
                        CacheArgs other = c;
                        other.head_stride += 32;
                        CHECK(rows_in_a_row(other) == (kv == 1));
                        other = c;
                        other.page_stride += 32;
                        CHECK(rows_in_a_row(other) == (pages == 1));
                        // rows before heads
                        other = c;
                        other.row_stride = c.row_stride * kv;
                        other.head_stride = c.row_stride;
                        CHECK(rows_in_a_row(other) == (kv == 1));
                    }
}

// Clusters of one token's attention: within what the GPU holds, no larger than the device allows, steps enough for each, and what has them without a window, when the size of
// the workspace is asked for, has them with any.
static void clusters()
{
    using namespace decode;
    long long sixteens = 0, eights = 0, none = 0;
    for (int sms : {1, 20, 132, 148})
        for (int most : {8, 16})
            for (int step : {64, 128, 256})
                for (int batch : {1, 2, 3, 7, 18, 19, 37, 148, 297, 100000})
                    for (int heads : {1, 2, 3, 8, 64, 1024})
                        for (int width : {0, 1, 2, 7, 16, 33, 60, 63, 64, 65, 128, 250, 1000, 1 << 20}) {
                            AttentionArgs a = {};
                            a.seq.batch = batch;
                            a.seq.width = width;
                            a.cache.page_shift = 6;
                            const int r = ranks_of(a, step, heads, sms, most);
                            const int64_t steps = steps_of(a, step), items = int64_t(heads) * batch;
                            CHECK(r == 0 || (r <= most && (r & (r - 1)) == 0 && r * items <= 2 * sms && r < 2 * steps && steps <= 16 * r));
                            CHECK(r < 16 || 16 * items <= sms);
                            (r == 16 ? sixteens : r == 8 ? eights : none) += 1;
                            for (int window : {1, 63, 64, 65, 500, 1000, 4000, 1 << 20, 0x7fffffff}) {
                                a.window = window;
                                CHECK(r == 0 || ranks_of(a, step, heads, sms, most) > 0);
                            }
                        }
    CHECK(sixteens > 0 && eights > 0 && none > 0);
    // few short sequences on a device that holds no cluster of 16: eights, or where these have too many steps even runs
    AttentionArgs a = {};
    a.seq.batch = 1;
    a.seq.width = 16;
    a.cache.page_shift = 6;
    CHECK(ranks_of(a, 64, 8, 148, 16) == 16 && ranks_of(a, 64, 8, 148, 8) == 8);
    a.seq.width = 100;
    CHECK(ranks_of(a, 64, 8, 148, 16) == 16 && ranks_of(a, 64, 8, 148, 8) == 0);
}

int main()
{
    rows();
    clusters();
    printf("ok %lld\n", g_checks);
    return 0;
}
