/* Host-only check of which workspaces the attention calls over pages take, with the stand-ins of launch_check.c: those of other calls of the same sequences and nodes do if they hold one part of the
 * rows, two with groups or where more selected pages may be seen than a list holds; nothing less. */
#define main others_main
#include "launch_check.c"
#undef main

static void expect_status(int status, int want, const char *what, const dream_attn_desc *d, int n, int page, long long keys, int seen, size_t bytes)
{
    if (status != want) {
        printf("%s: D %d, heads %d/%d, batch %d, %d nodes, pages of %d, %lld keys, hint %d, %zu bytes: status %d, not %d (%s)\n", what, d->head_dim, d->n_q_heads, d->n_kv_heads, d->batch, n, page, keys, seen,
               bytes, status, want, status ? dream_last_error() : "");
        bad++;
    }
}

int main(void)
{
    static const int shapes[][5] = {{64, 8, 8, 1, 1}, {128, 32, 8, 1, 60}, {128, 32, 8, 12, 33}, {256, 16, 8, 3, 200}, {128, 8, 1, 40, 1}};      /* D, Hq, Hkv, batch, nodes */
    static const struct { int page; long long keys; } caches[] = {{64, 300}, {64, 5000}, {16, 5000}, {64, 70000}, {16, 131060}, {16, 8000000}};
    static const int hints[] = {0, 1, 19, 900};
    void *const p = (void *)0x10000;         /* never dereferenced: nothing runs */
    int i, j, k, h;
    (void)others_main;
    OK(dream_init());
    initialised = 1;
    for (i = 0; i < 5; i++)
        for (j = 0; j < 6; j++)
            for (k = 0; k < 2; k++) {        /* bf16, float32 */
                const int n = shapes[i][4], page = caches[j].page;
                const long long keys = caches[j].keys;
                const dream_attn_desc d = {shapes[i][3], shapes[i][1], shapes[i][2], shapes[i][0], k ? DREAM_F32 : DREAM_BF16, 0.0f, 0};
                const dream_page_desc pages = {page, 5000, (int)(keys / page) + 2};
                const size_t part = (size_t)d.batch * d.n_q_heads * n * (d.head_dim + 2) * 4;
                size_t parts;
                if (keys < n)
                    continue;
                for (parts = 1; parts <= 5; parts++) {
                    const size_t bytes = parts * part < 256 ? 256 : parts * part;
                    expect_status(dream_paged_verify_attn(&d, &pages, p, p, p, p, p, n, p, NULL, 0, NULL, NULL, 0, keys, p, NULL, p, bytes, NULL), 0, "paged", &d, n, page, keys, 0, bytes);
                    expect_status(dream_paged_verify_attn(&d, &pages, p, p, p, p, p, n, p, NULL, 1, p, p, keys / 2, keys, p, NULL, p, bytes, NULL), bytes < 2 * part ? DREAM_ERR_WORKSPACE : 0, "groups", &d, n,
                                  page, keys, 0, bytes);
                    for (h = 0; h < 4; h++) {
                        long long seen = (keys + page - 1) / page;
                        if (hints[h] && (long long)hints[h] * n < seen)
                            seen = (long long)hints[h] * n;
                        seen += n / page + 2;
                        expect_status(dream_sparse_verify_attn(&d, &pages, p, p, p, p, p, p, n, p, NULL, keys, hints[h], p, NULL, p, bytes, NULL),
                                      seen > (n > 64 ? 512 : 1024) && bytes < 2 * part ? DREAM_ERR_WORKSPACE : 0, "selected", &d, n, page, keys, hints[h], bytes);
                    }
                }
                for (h = 0; h < 4; h++) {    /* what is asked for is taken, and is in proportion */
                    const size_t bytes = dream_sparse_verify_attn_workspace(&d, &pages, n, keys, hints[h]);
                    expect_status(dream_sparse_verify_attn(&d, &pages, p, p, p, p, p, p, n, p, NULL, keys, hints[h], p, NULL, p, bytes, NULL), 0, "asked for", &d, n, page, keys, hints[h], bytes);
                    if (bytes > 48 * part + 256) {
                        printf("%d nodes, %lld keys in pages of %d, hint %d: %zu bytes, %zu parts\n", n, keys, page, hints[h], bytes, bytes / part);
                        bad++;
                    }
                }
            }
    printf("bad: %d; launches: %ld\n", bad, launches);
    return bad > 0;
}
