/* Host-only check of what the calls for caches in pages ask HIP for, with the stand-ins of launch_check.c: no limit raised after dream_init, no launch beyond its kernel's limit of
 * LDS or with an empty or oversized grid, every kernel with a raised limit launched by some call. */
#define main others_main
#include "launch_check.c"
#undef main
#include "dream_tuning.h"

static void paged_sweep(void)
{
    static const int layouts[][3] = {{1, 1, 64}, {32, 32, 64}, {4, 2, 64}, {32, 32, 128}, {32, 8, 128}, {28, 4, 128}, {64, 1, 128}, {16, 8, 256}, {4, 4, 256}, {64, 1, 256}};
    static const int batches[] = {1, 3, 8, 40, 300}, trees[] = {1, 7, 33, 60, 64, 65, 129, 256}, lengths[] = {1, 100, 770, 4100, 17000, 140000};
    void *const p = (void *)0x10000;         /* never dereferenced: nothing runs */
    void *const far[] = {(void *)(1ull << 44), (void *)(2ull << 44), (void *)(3ull << 44), (void *)(4ull << 44), (void *)(5ull << 44)};
    void *pools[300];
    const size_t all = (size_t)1 << 44;
    int i, j, t, k, n, w, page;
    for (i = 0; i < 300; i++)
        pools[i] = p;
    for (i = 0; i < (int)(sizeof layouts / sizeof *layouts); i++)
        for (j = 0; j < (int)(sizeof batches / sizeof *batches); j++)
            for (n = 0; n < 2; n++)
                for (page = 16; page <= 256; page *= 4) {
                    const dream_attn_desc desc = {batches[j], layouts[i][0], layouts[i][1], layouts[i][2], n ? DREAM_F32 : DREAM_BF16, 0.0f, 0};
                    const dream_page_desc pages = {page, 1000, 200000 / page};
                    OK(dream_paged_commit(&desc, &pages, p, pools, 300, p, 60, p, 7, p, NULL, NULL));
                    for (k = 0; k < (int)(sizeof lengths / sizeof *lengths); k++) {
                        if ((long long)desc.batch * lengths[k] <= 1 << 20)
                            OK(dream_paged_append(&desc, &pages, p, far[0], far[1], far[2], lengths[k], p, NULL, NULL, NULL, NULL, NULL, p, 64, n, 0.0f, far[0], far[3], far[4], NULL));
                        OK(dream_page_bounds(&desc, &pages, p, p, NULL, p, lengths[k], p, NULL));
                        for (t = 0; t < (int)(sizeof trees / sizeof *trees); t++) {
                            const int keys = lengths[k] + trees[t];
                            OK(dream_page_select(&desc, &pages, p, p, p, p, trees[t], 1, 2, 16, keys, p, p, all, NULL));
                            OK(dream_paged_verify_attn(&desc, &pages, p, p, p, p, p, trees[t], p, NULL, 0, NULL, NULL, 0, keys, p, NULL, p, all, NULL));
                            OK(dream_paged_verify_attn(&desc, &pages, p, p, p, p, p, trees[t], p, NULL, 1 + desc.batch / 3, p, p, lengths[k], keys, p, p, p, all, NULL));
                            OK(dream_sparse_verify_attn(&desc, &pages, p, p, p, p, p, p, trees[t], p, NULL, keys, 0, p, NULL, p, all, NULL));
                            OK(dream_sparse_verify_attn(&desc, &pages, p, p, p, p, p, p, trees[t], NULL, p, keys, 19, p, NULL, p, all, NULL));
                        }
                    }
                }
    for (w = 4; w <= 8; w += 4)              /* every shape, also where no size above takes it */
        for (n = 1; n <= 2; n++)
            for (i = 0; i < (int)(sizeof layouts / sizeof *layouts); i++)
                for (t = 0; t < (int)(sizeof trees / sizeof *trees); t++) {
                    const dream_attn_desc desc = {3, layouts[i][0], layouts[i][1], layouts[i][2], DREAM_BF16, 0.0f, 0};
                    const dream_page_desc pages = {16, 1000, 12500};
                    dream_set_tile_waves(w);
                    dream_set_q_tiles(n);
                    OK(dream_paged_verify_attn(&desc, &pages, p, p, p, p, p, trees[t], p, NULL, 2, p, p, 100, 1000, p, NULL, p, all, NULL));
                    OK(dream_sparse_verify_attn(&desc, &pages, p, p, p, p, p, p, trees[t], p, NULL, 150000, 0, p, NULL, p, all, NULL));
                    OK(dream_sparse_verify_attn(&desc, &pages, p, p, p, p, p, p, trees[t], p, NULL, 1000, 5, p, NULL, p, all, NULL));
                }
    dream_set_tile_waves(0);
    dream_set_q_tiles(0);
}

int main(void)
{
    int i, seen, n = 0, never = 0;
    (void)others_main;
    for (device = 0; device < 2; device++) {
        initialised = 0;
        OK(dream_init());
        initialised = 1;
        seen = n_funcs;                      /* those with a raised limit, of all calls */
        for (i = 0; i < seen; i++)
            launched[i] = 0;
        paged_sweep();
        for (i = n = 0; i < n_funcs; i++)
            n += launched[i] > 0;
        for (i = never = 0; i < n_funcs; i++)
            never += launched[i] > 0 && limits[device][i] > 65536;
        printf("device %d: %d kernels launched, %d with a raised limit; raised after dream_init: %d; bad: %d; launches: %ld\n", device, n, never, late, bad, launches);
        if (late || bad)
            return 1;
    }
    return 0;
}
