/* Plans, divisions, workspace sizes and checks of random sizes: without a GPU every call
   ends before device work, and plans where they would be copied to one.  Prints "ok". */
#include <stdio.h>
#include <stdlib.h>

#include "f3s_cache.h"
#include "f3s_pages.h"
#include "f3s_window.h"

/* addresses that are never read, far from one another */
static char *at(int k) { return (char *)((size_t)1 << 46) + ((size_t)k << 40); }

static int any(int n) { return rand() % n; }

static void plans(void)
{
    int n = any(6), g = 1 + any(5), kv = 1 + any(3), d = 32 * (1 + any(8));
    int32_t *q = malloc((n + 1) * sizeof *q), *k = malloc((n + 1) * sizeof *k);
    int32_t *ql = malloc((n + 1) * sizeof *ql), *kl = malloc((n + 1) * sizeof *kl);
    q[0] = k[0] = 0;
    for (int b = 0; b < n; ++b) {
        q[b + 1] = q[b] + any(3000);
        k[b + 1] = k[b] + any(3000);
        ql[b] = any(q[b + 1] - q[b] + 1);
        kl[b] = any(k[b + 1] - k[b] + 1);
    }
    int window = any(7) ? any(4000) : 2147483647, sinks = any(3) ? any(300) : 0;
    f3s_window_plan_t p = f3s_window_plan(q, k, any(2) ? ql : NULL, any(2) ? kl : NULL, n, kv * g,
                                          kv, d, window, sinks);
    if (p) {
        f3s_window_forward_workspace_bytes(p);
        f3s_window_backward_workspace_bytes(p);
        f3s_window_destroy(p);
    }
    free(q);
    free(k);
    free(ql);
    free(kl);
}

static void calls(void)
{
    int kv = 1 + any(3), heads = kv * (1 + any(5)), d = 32 * (1 + any(8));
    f3s_cache_t c = {at(1), at(2), (uint8_t *)at(3), (uint8_t *)at(4), 1 + any(100), kv,
                     16 << any(5), d};
    int pages = any(5000), n_seqs = any(300), n = any(300), window = any(9000), sinks = any(300);
    int prefix = any(2) * any(5000);
    size_t w = f3s_cache_attend_window_workspace_bytes(&c, pages, n_seqs, n, heads, window, sinks);
    f3s_cache_attend_window(&c, at(5), F3S_DTYPE_F16, at(6), (float *)at(7), (int32_t *)at(8),
                            pages, (int32_t *)at(9), n_seqs, n, heads, window, sinks, 0.1f,
                            at(10), w, 0);
    w = f3s_cache_attend_tree_workspace_bytes(&c, pages, n_seqs, n, heads, prefix);
    f3s_cache_attend_tree(&c, at(5), F3S_DTYPE_BF16, at(6), (float *)at(7), (int32_t *)at(8),
                          pages, (int32_t *)at(9), n_seqs, n, heads, (int32_t *)at(11),
                          prefix ? (int32_t *)at(12) : NULL, prefix, 0.1f, at(10), w, 0);
    f3s_cache_keep(&c, (int32_t *)at(8), pages, (int32_t *)at(9), n_seqs, n, (int32_t *)at(11), n,
                   (int32_t *)at(12), 0);
    n_seqs *= 20;
    w = f3s_pages_assign_workspace_bytes(n_seqs, pages, n);
    f3s_pages_assign((int32_t *)at(1), (int32_t *)at(2), 1 + any(1000), (int32_t *)at(8), pages,
                     (int32_t *)at(9), (int32_t *)at(10), (int32_t *)at(11), (int64_t *)at(12),
                     n_seqs, n, 16 << any(5), at(13), w, 0);
}

int main(void)
{
    for (int turn = 0; turn < 400; ++turn) {
        plans();
        calls();
    }
    printf("ok\n");
    return 0;
}
