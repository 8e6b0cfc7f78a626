/*
 * The host-side code of the dense operators (f3s_cross.h, f3s_cache.h) under
 * AddressSanitizer and UndefinedBehaviorSanitizer, on a machine without a GPU
 * (built and run by tests/test_sanitize_dense.py): the division of ragged
 * batches up to the point where the plan wants device memory, the sizes of
 * workspaces over the whole int32 range, and the argument checks.  Any memory
 * error, leak in the library or undefined behaviour aborts the run.  Prints "ok"
 * on success.
 */
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "f3s_cache.h"
#include "f3s_cross.h"

#define CHECK(c)                                                           \
    do {                                                                   \
        if (!(c)) {                                                        \
            fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); \
            return 1;                                                      \
        }                                                                  \
    } while (0)

static uint32_t state = 1;
static int32_t draw(int32_t below)
{
    state = state * 1664525u + 1013904223u;
    return (int32_t)((state >> 8) % (uint32_t)below);
}

int main(void)
{
    /* plans: ragged, padded, empty and long, in exactly sized arrays */
    for (int round = 0; round < 200; ++round) {
        const int32_t n = draw(9), kv = 1 + draw(4), g = 1 + draw(5), d = 32 * (1 + draw(8));
        const size_t ptr = (size_t)(n + 1) * 4, len = (size_t)n * 4;
        int32_t *qp = malloc(ptr), *kp = malloc(ptr), *ql = malloc(len + !len),
                *kl = malloc(len + !len);
        CHECK(qp && kp && ql && kl);
        qp[0] = kp[0] = 0;
        const int32_t most = round % 3 ? 300 : 200000;
        for (int32_t b = 0; b < n; ++b) {
            const int32_t q = draw(4) ? draw(most) : 0, k = draw(4) ? draw(most) : 0;
            qp[b + 1] = qp[b] + q;
            kp[b + 1] = kp[b] + k;
            ql[b] = draw(q + 1);
            kl[b] = draw(k + 1);
        }
        const int padded = draw(2);
        CHECK(f3s_cross_plan(qp, kp, padded ? ql : NULL, padded ? kl : NULL, n, kv * g, kv, d) ==
              NULL);
        CHECK(f3s_last_error() == F3S_ERR_HIP);
        free(qp);
        free(kp);
        free(ql);
        free(kl);
    }
    const int32_t far[] = {0, INT_MAX};
    CHECK(f3s_cross_plan(far, far, NULL, NULL, 1, 65535, 65535, 32) == NULL);
    CHECK(f3s_last_error() == F3S_ERR_TOO_LARGE);
    CHECK(f3s_cross_plan(far, far, NULL, NULL, INT_MIN, 1, 1, 32) == NULL);
    f3s_cross_destroy(NULL);
    CHECK(f3s_cross_forward_workspace_bytes(NULL) == 0);
    CHECK(f3s_cross_forward(NULL, NULL, NULL, NULL, F3S_DTYPE_F16, NULL, NULL, 1.f, NULL, 0,
                            NULL) == F3S_ERR_INVALID_VALUE);
    CHECK(f3s_cross_backward(NULL, NULL, NULL, NULL, F3S_DTYPE_F16, NULL, NULL, NULL, NULL, NULL,
                             NULL, 1.f, NULL, 0, NULL) == F3S_ERR_INVALID_VALUE);

    /* workspaces: every size of int32 */
    const int32_t sizes[] = {INT_MIN, -1, 0, 1, 2, 17, 4096, 1 << 20, 1 << 28, INT_MAX - 1,
                             INT_MAX};
    const int n = sizeof sizes / sizeof *sizes;
    char *mem = (char *)0x100000;
    for (int page = 16; page <= 256; page *= 4)
        for (int kv = 0; kv < n; ++kv) {
            f3s_cache_t c = {mem, mem, (uint8_t *)mem, (uint8_t *)mem, 1, sizes[kv], page, 128};
            for (int a = 0; a < n; ++a)
                for (int b = 0; b < n; ++b)
                    for (int e = 0; e < n; ++e)
                        for (int f = 0; f < n; ++f) {
                            const int64_t heads = (int64_t)sizes[kv] * 4;
                            const int32_t h = heads > INT_MAX ? sizes[kv] : (int32_t)heads;
                            const size_t bytes = f3s_cache_attend_workspace_bytes(
                                &c, sizes[a], sizes[b], sizes[e], h, sizes[f]);
                            CHECK(bytes < (size_t)1 << 60);
                        }
        }

    /* checks: each call ends at one, or for want of a device */
    for (int round = 0; round < 20000; ++round) {
        f3s_cache_t c = {mem + 16 * draw(2), mem, (uint8_t *)mem, (uint8_t *)mem + draw(2),
                         draw(5) ? 1 + draw(9) : sizes[draw(n)],
                         draw(5) ? 1 + draw(4) : sizes[draw(n)],
                         draw(5) ? 16 << draw(5) : sizes[draw(n)],
                         draw(5) ? 32 * (1 + draw(8)) : sizes[draw(n)]};
        char *far_mem = (char *)((uintptr_t)1 << 40);
        const int32_t pages = draw(3) ? draw(9) : sizes[draw(n)];
        const int32_t seqs = draw(3) ? draw(9) : sizes[draw(n)];
        const int32_t tokens = draw(3) ? draw(9) : sizes[draw(n)];
        const int32_t heads = draw(3) ? 4 * (1 + draw(8)) : sizes[draw(n)];
        const int32_t prefix = draw(3) ? draw(900) : sizes[draw(n)];
        const f3s_dtype_t t = (f3s_dtype_t)draw(4);
        const int32_t *lens = (const int32_t *)(far_mem - 4096);
        f3s_status_t st = f3s_cache_write(&c, far_mem, far_mem, t, lens, pages, lens, seqs,
                                          tokens, NULL);
        CHECK(st >= F3S_OK && st <= F3S_ERR_TOO_LARGE);
        st = f3s_cache_read(&c, far_mem, NULL, t, lens, pages, lens, seqs, tokens, NULL);
        CHECK(st >= F3S_OK && st <= F3S_ERR_TOO_LARGE);
        st = f3s_cache_attend(&c, far_mem, t, far_mem + ((size_t)1 << 44),
                              (float *)(far_mem + ((size_t)1 << 45)), lens, pages, lens, seqs,
                              tokens, heads, lens, prefix, draw(9) ? 0.5f : INFINITY,
                              far_mem + ((size_t)1 << 43), SIZE_MAX >> 1, NULL);
        CHECK(st >= F3S_OK && st <= F3S_ERR_TOO_LARGE);
    }
    printf("ok\n");
    return 0;
}
