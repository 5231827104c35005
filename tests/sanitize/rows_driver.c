/* Host sanitizer run of the row-table operators' argument validation (rows_api.cpp
 * with host-only launcher stubs): bad arguments return their documented status, leave
 * a message and launch nothing; good ones reach their launcher.  Device pointers are
 * fake addresses that are never dereferenced.  Exit status 0 = all checks passed. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "hs_merge.h"

extern int hs_stub_launches;
static int fails = 0;
#define CHECK(c)                                                                            \
    do {                                                                                    \
        if (!(c)) {                                                                         \
            fprintf(stderr, "check failed at line %d: %s (last error: %s)\n", __LINE__, #c, \
                    hs_last_error());                                                       \
            ++fails;                                                                        \
        }                                                                                   \
    } while (0)
#define REJECT(call, s)                                                                     \
    do {                                                                                    \
        int before = hs_stub_launches;                                                      \
        CHECK((call) == (s));                                                               \
        CHECK(hs_last_error()[0] != 0 && hs_stub_launches == before);                       \
    } while (0)
#define ACCEPT(call)                                                                        \
    do {                                                                                    \
        int before = hs_stub_launches;                                                      \
        CHECK((call) == HS_OK);                                                             \
        CHECK(hs_last_error()[0] == 0 && hs_stub_launches == before + 1);                   \
    } while (0)
#define P(x) ((void *)(uintptr_t)(x))
static const uintptr_t A = 0x10000000, B = 1ull << 44, C = 2ull << 44, D = 3ull << 44;

int main(void) {
    /* the largest table there may be: sizes stay within 64 bits */
    hs_row_table t = {P(A), P(B), INT32_MAX, 16384, HS_FP4_E2M1, HS_BF16, 32};
    ACCEPT(hs_embed(&t, P(C), 0, (int64_t)1 << 30, 2.0f, -1, P(D), HS_F32, NULL));
    ACCEPT(hs_score_packed(&t, P(C), HS_F32, 1, P(D), HS_F32, INT32_MAX, NULL));
    REJECT(hs_score_packed(&t, P(C), HS_F32, 1 << 20, P(A), HS_F32, (int64_t)1 << 40, NULL),
           HS_ERR_INVALID_ARG);
    t.dtype = HS_F32;
    ACCEPT(hs_embed(&t, P(D), 1, 3, 2.0f, INT64_MIN, P(1ull << 55), HS_BF16, NULL));
    REJECT(hs_score_packed(&t, P(C), HS_F32, 1, P(D), HS_F32, INT32_MAX, NULL),
           HS_ERR_UNSUPPORTED);
    t.dtype = -1;
    REJECT(hs_embed(&t, P(C), 0, 1, 2.0f, -1, P(D), HS_F32, NULL), HS_ERR_UNSUPPORTED);
    REJECT(hs_embed(NULL, P(C), 0, 1, 2.0f, -1, P(D), HS_F32, NULL), HS_ERR_INVALID_ARG);
    t.dtype = HS_BF16;
    REJECT(hs_embed(&t, P(C), 0, 1, NAN, -1, P(D), HS_F32, NULL), HS_ERR_INVALID_ARG);
    REJECT(hs_embed(&t, P(C), 0, INT64_MAX, 1.0f, -1, P(D), HS_F32, NULL), HS_ERR_INVALID_ARG);

    ACCEPT(hs_pack_rows(P(A), HS_F32, 1000, 256, 64, HS_F32, P(B), P(C), NULL));
    REJECT(hs_pack_rows(P(A), HS_F32, 1000, 256, 96, HS_F32, P(B), P(C), NULL),
           HS_ERR_UNSUPPORTED);
    REJECT(hs_pack_rows(P(A), HS_F32, INT64_MIN, 256, 64, HS_F32, P(B), P(C), NULL),
           HS_ERR_INVALID_ARG);

    size_t need = 0;
    CHECK(hs_embed_grad_bytes(5000, 300, 72, &need) == HS_OK && need > 0);
    REJECT(hs_embed_grad_bytes(5000, 300, INT64_MAX, &need), HS_ERR_INVALID_ARG);
    ACCEPT(hs_embed_grad(P(A), HS_BF16, P(B), 1, 5000, 300, 72, 1.0f, 0, 1, P(C), HS_BF16, P(D),
                         need, NULL));
    REJECT(hs_embed_grad(P(A), HS_BF16, P(B), 1, 5000, 300, 72, 1.0f, 0, 1, P(C), HS_BF16, P(D),
                         need - 1, NULL), HS_ERR_WORKSPACE);
    REJECT(hs_embed_grad(P(A), HS_BF16, P(B), 1, 5000, 300, 72, 1.0f, 0, 1, P(A), HS_BF16, P(D),
                         need, NULL), HS_ERR_INVALID_ARG);

    hs_adjust a;
    memset(&a, 0, sizeof(a));
    a.allow = (const uint32_t *)P(B);
    ACCEPT(hs_adjust_scores(&a, P(A), 4000, P(A), 4000, HS_BF16, 7, 3999, NULL));
    ACCEPT(hs_adjust_scores(&a, P(A), 4000, P(C), 3999, HS_BF16, 7, 3999, NULL));
    REJECT(hs_adjust_scores(&a, P(A), 4000, P(A), 4001, HS_BF16, 7, 3999, NULL),
           HS_ERR_INVALID_ARG);
    REJECT(hs_adjust_scores(&a, P(A), INT64_MAX, P(C), 3999, HS_BF16, 7, 3999, NULL),
           HS_ERR_INVALID_ARG);
    a.allow_stride = INT64_MAX;
    REJECT(hs_adjust_scores(&a, P(A), 4000, P(C), 4000, HS_BF16, 7, 3999, NULL),
           HS_ERR_INVALID_ARG);

    CHECK(hs_topk_rows_bytes(7, 3999, 64, &need) == HS_OK && need > 0);
    ACCEPT(hs_topk_rows(P(A), HS_F32, 4000, 7, 3999, 64, P(B), P(C), P(D), need, NULL));
    REJECT(hs_topk_rows(P(A), HS_F32, 4000, 7, 3999, INT32_MIN, P(B), P(C), P(D), need, NULL),
           HS_ERR_INVALID_ARG);
    REJECT(hs_topk_rows(P(A), HS_F32, 4000, 7, 3999, 64, P(B), P(C), P(D), need - 1, NULL),
           HS_ERR_WORKSPACE);
    if (fails) {
        fprintf(stderr, "%d checks failed\n", fails);
        return 1;
    }
    printf("all checks passed\n");
    return 0;
}
