/* Walks the host side of the paged calls - argument checks, extents of rows and pages, the plan of the attention, its workspace
 * query - as host_paths.c does that of the other entry points: no call below gets as far as a launch. */
#include <stdint.h>
#include <stdio.h>

#include "fedrag.h"

static int failures = 0;
#define EXPECT(call, want)                                                                          \
    do {                                                                                            \
        const int got_ = (int)(call);                                                               \
        if (got_ != (int)(want)) {                                                                  \
            printf("line %d: %s -> %d, expected %d\n", __LINE__, #call, got_, (int)(want));         \
            ++failures;                                                                             \
        }                                                                                           \
    } while (0)

#define P(n) ((void*)(uintptr_t)((uint64_t)(n) << 44)) /* fake device pointers, far apart */
#define PI(n) ((int32_t*)P(n))
#define PL(n) ((int64_t*)P(n))
#define PF(n) ((float*)P(n))

static uint64_t rng_state = 0x9E3779B97F4A7C15ull;
static uint64_t rnd64(void) { /* splitmix64 */
    uint64_t z = (rng_state += 0x9E3779B97F4A7C15ull);
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
static int64_t upto(int64_t n) { return (int64_t)(rnd64() % ((uint64_t)n + 1)); }
/* 0 .. most, evenly over the logarithm, the ends among them */
static int64_t some(int64_t most) {
    int bits = 0;
    if (rnd64() % 16 == 0) return most;
    while (bits < 62 && ((int64_t)1 << bits) <= most) ++bits;
    const int64_t x = (int64_t)(rnd64() >> 1) & (((int64_t)1 << upto(bits)) - 1);
    return x < most ? x : most;
}

int main(void) {
    const int32_t pages[] = {16, 32, 64, 128, 256};
    const int64_t most = INT32_MAX, huge = INT64_MAX;

    /* ---- the map */
    EXPECT(fedrag_paged_map(2, 40, 16, 4, NULL, PI(2), PI(3), 9, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_NULL);
    EXPECT(fedrag_paged_map(2, huge, 16, 4, PI(1), PI(2), PI(3), 9, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_SHAPE);
    EXPECT(fedrag_paged_map(2, 40, 16, huge, PI(1), PI(2), PI(3), 9, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_SHAPE);
    EXPECT(fedrag_paged_map(2, 40, 16, 4, PI(1), PI(2), PI(3), INT64_MIN, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_SHAPE);
    EXPECT(fedrag_paged_map(INT32_MAX, 40, 16, 4, PI(1), PI(2), PI(3), 9, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_SHAPE);
    EXPECT(fedrag_paged_map(INT32_MIN, 40, 16, 4, PI(1), PI(2), PI(3), 9, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_SHAPE);
    /* a table of 2^64 bytes, and one of 2^61, which the other arrays lie in */
    EXPECT(fedrag_paged_map(INT32_MAX - 255, most, 256, most, PI(1), PI(2), PI(3), most, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL),
           FEDRAG_ERR_SHAPE);
    EXPECT(fedrag_paged_map(INT32_MAX - 255, most, 256, 1 << 28, PI(1), PI(2), PI(3), most, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL),
           FEDRAG_ERR_ALIAS);
    EXPECT(fedrag_paged_map(2, 40, INT32_MIN, 4, PI(1), PI(2), PI(3), 9, PI(4), PI(5), PI(6), PI(7), PL(8), PI(9), PI(10), PI(11), NULL), FEDRAG_ERR_UNSUPPORTED);

    /* ---- numbers at their ends */
    {
        const fedrag_shape s = {2, 8, 2, 128, FEDRAG_BF16}, wide = {INT32_MAX, INT32_MAX, INT32_MAX, 128, FEDRAG_F32}, one = {1, INT32_MAX, 1, 128, FEDRAG_F32};
        fedrag_rows q = {P(1), 128, 1024};
        fedrag_paged_cache c = {P(2), P(3), 10, 0, 16};
        const int64_t ends[] = {INT64_MIN, -1, huge, huge - 15, (int64_t)1 << 62, (int64_t)1 << 61};
        for (int i = 0; i < 6; ++i) {
            fedrag_rows bad = {P(1), ends[i], 1024}, bad2 = {P(1), 128, ends[i]};
            fedrag_paged_cache cs = {P(2), P(3), 10, ends[i], 16}, cn = {P(2), P(3), ends[i], 0, 16};
            EXPECT(fedrag_paged_attn(&s, 40, &bad, &c, PI(4), 4, PI(5), PI(6), 8, 1, 0.1f, PF(7), PF(8), P(9), 1u << 30, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_attn(&s, 40, &bad2, &c, PI(4), 4, PI(5), PI(6), 8, 1, 0.1f, PF(7), PF(8), P(9), 1u << 30, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_attn(&s, 40, &q, &cs, PI(4), 4, PI(5), PI(6), 8, 1, 0.1f, PF(7), PF(8), P(9), 1u << 30, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_attn(&s, 40, &q, &cn, PI(4), 4, PI(5), PI(6), 8, 1, 0.1f, PF(7), PF(8), P(9), 1u << 30, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_write(&s, 40, &bad, &q, PL(4), &c, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_write(&s, 40, &q, &bad2, PL(4), &c, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_write(&s, 40, &q, &q, PL(4), &cs, NULL), FEDRAG_ERR_SHAPE);
            EXPECT(fedrag_paged_write(&s, ends[i], &q, &q, PL(4), &c, NULL), FEDRAG_ERR_SHAPE);
            if (ends[i] >= 0) EXPECT(fedrag_paged_attn_workspace_bytes(&s, 40, 4, 16, ends[i]) > 0, 0); /* an expectation has no bound */
            else EXPECT(fedrag_paged_attn_workspace_bytes(&s, 40, 4, 16, ends[i]), 0);
            EXPECT(fedrag_paged_attn_workspace_bytes(&s, ends[i], 4, 16, 8), 0);
            EXPECT(fedrag_paged_attn_workspace_bytes(&s, 40, ends[i], 16, 8), 0);
        }
        fedrag_rows far = {P(1), (int64_t)1 << 55, 0};
        fedrag_paged_cache all = {P(2), P(3), INT32_MAX, 0, 256};
        EXPECT(fedrag_paged_attn(&wide, most, &far, &all, PI(4), 4, PI(5), PI(6), 8, 1, 0.1f, PF(7), PF(8), P(9), 1u << 30, NULL), FEDRAG_ERR_SHAPE);
        EXPECT(fedrag_paged_attn(&one, most, &far, &c, PI(4), 4, PI(5), PI(6), 8, 1, 0.1f, PF(7), PF(8), P(9), 1u << 30, NULL), FEDRAG_ERR_SHAPE);
        EXPECT(fedrag_paged_write(&wide, most, &far, &far, PL(4), &all, NULL), FEDRAG_ERR_SHAPE);
        EXPECT(fedrag_paged_attn_workspace_bytes(&wide, most, 4, 16, 0), 0);
        EXPECT(fedrag_paged_attn_workspace_bytes(&one, most, 4, 16, 0), 0);
    }

    /* ---- any sizes: scratch missing, or nothing needed and an output over an input; V's pages over K's */
    for (int i = 0; i < 200000; ++i) {
        const int32_t Hkv = (int32_t)some(i % 2 ? 64 : INT32_MAX - 1) + 1, G = (int32_t)some(INT32_MAX / Hkv - 1) + 1;
        const fedrag_shape s = {(int32_t)some(INT32_MAX), Hkv * G, Hkv, i % 3 ? 128 : 64, (int32_t)upto(2)};
        const int32_t page = pages[upto(4)];
        const int64_t T = some(most), columns = some(most), max_q = some(i % 5 ? 4096 : huge - 1);
        const size_t need = fedrag_paged_attn_workspace_bytes(&s, T, columns, page, max_q);
        if (need > (size_t)69 << 20) ++failures, printf("%d rows: %zu bytes\n", (int)T, need);
        fedrag_rows rows = {P(1), some((int64_t)1 << 40) / 8 * 8, some((int64_t)1 << 40) / 8 * 8};
        fedrag_paged_cache cache = {P(2), P(2), some(most), 0, page};
        const fedrag_status st = fedrag_paged_attn(&s, T, &rows, &cache, PI(2), columns, PI(2), PI(2), max_q, i & 1, 0.1f, PF(2), PF(2), NULL, 0, NULL);
        const int nothing = T == 0 || s.batch == 0;
        if (st == FEDRAG_OK ? !nothing : need > 0 && st != FEDRAG_ERR_WORKSPACE && st != FEDRAG_ERR_SHAPE && st != FEDRAG_ERR_ALIAS)
            ++failures, printf("attention of %d rows: status %d, %zu bytes\n", (int)T, (int)st, need);
        const fedrag_status w = fedrag_paged_write(&s, T, &rows, &rows, PL(2), &cache, NULL);
        if (w == FEDRAG_OK ? T != 0 && cache.n_pages != 0 : w != FEDRAG_ERR_SHAPE && w != FEDRAG_ERR_ALIAS)
            ++failures, printf("rows into pages, %d: status %d\n", (int)T, (int)w);
        const fedrag_status m = fedrag_paged_map(s.batch, T, page, columns, PI(1), PI(1), PI(1), some(most), PI(1), PI(1), PI(1), PI(1), PL(1), PI(1),
                                                 PI(1), PI(1), NULL);
        if (m != FEDRAG_ERR_SHAPE && m != FEDRAG_ERR_ALIAS) ++failures, printf("map of %d rows: status %d\n", (int)T, (int)m);
        if (failures > 20) break;
    }
    if (failures) {
        printf("%d failures\n", failures);
        return 1;
    }
    printf("paged host paths ok\n");
    return 0;
}
