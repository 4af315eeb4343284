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

int main()
{
    rows();
    printf("ok %lld\n", g_checks);
    return 0;
}
