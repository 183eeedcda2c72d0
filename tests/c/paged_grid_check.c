/* Host-only check that no call over pages asks HIP for a grid of 2^32 threads or more along an axis, at the sizes dream.h allows: such calls are refused.  With the stand-ins of launch_check.c. */
#define main others_main
#define hipLaunchKernel others_launch
#include "launch_check.c"
#undef hipLaunchKernel
#undef main
#include "dream_tuning.h"

static unsigned long long widest;
int hipLaunchKernel(const void *f, grid3 grid, grid3 block, void **args, size_t lds, void *stream)
{
    const unsigned long long x = (unsigned long long)grid.x * block.x;
    if (x > widest)
        widest = x;
    if (x >> 32 || grid.x >> 31) {
        printf("grid %u x %u x %u of %u threads\n", grid.x, grid.y, grid.z, block.x);
        bad++;
    }
    return others_launch(f, grid, block, args, lds, stream);
}

int main(void)
{
    static const int batches[] = {1, 16, 100, 4096, 16384, 65535}, heads[][2] = {{1, 1}, {16, 16}, {16, 8}, {16, 1}, {64, 64}, {256, 2}, {4096, 4096}, {4096, 1}}, trees[] = {1, 5, 33, 64, 65, 255, 256}, dims[] = {64, 128, 256};
    void *const p = (void *)0x10000;         /* never dereferenced: nothing runs */
    const size_t all = (size_t)1 << 62;
    int i, j, t, k, n, f, refused = 0;
    (void)others_main;
    OK(dream_init());
    initialised = 1;
    for (f = 0; f < 2; f++)                  /* the call's own splits; as many as can be forced */
        for (i = 0; i < 6; i++)
            for (j = 0; j < 8; j++)
                for (t = 0; t < 7; t++)
                    for (k = 0; k < 3; k++)
                        for (n = 0; n < 2; n++) {
                            const dream_attn_desc d = {batches[i], heads[j][0], heads[j][1], dims[k], n ? DREAM_F32 : DREAM_BF16, 0.0f, 0};
                            const dream_page_desc pages = {64, 1000, 2000};
                            const long long rows = (long long)batches[i] * heads[j][0] * trees[t];
                            int status[3], m;
                            if ((long long)batches[i] * heads[j][0] > 1 << 20)
                                continue;
                            dream_set_kv_splits(f ? 64 : 0);
                            status[0] = dream_paged_verify_attn(&d, &pages, p, p, p, p, p, trees[t], p, NULL, 0, NULL, NULL, 0, 3000, p, NULL, p, all, NULL);
                            status[1] = dream_paged_verify_attn(&d, &pages, p, p, p, p, p, trees[t], p, NULL, (batches[i] + 2) / 3, p, p, 2000, 3000, p, NULL, p, all, NULL);
                            status[2] = dream_sparse_verify_attn(&d, &pages, p, p, p, p, p, p, trees[t], p, NULL, 3000, 5, p, NULL, p, all, NULL);
                            for (m = 0; m < 3; m++) {
                                refused += status[m] == DREAM_ERR_UNSUPPORTED;
                                if (status[m] && (status[m] != DREAM_ERR_UNSUPPORTED || (rows <= 1 << 23 && !f))) {
                                    printf("call %d: batch %d, heads %d/%d, %d nodes, D %d, f32 %d: status %d, %s\n", m, batches[i], heads[j][0], heads[j][1], trees[t], dims[k], n, status[m], dream_last_error());
                                    bad++;
                                }
                            }
                        }
    dream_set_kv_splits(0);
    printf("bad: %d; refused: %d; the widest launch: %llu threads; launches: %ld\n", bad, refused, widest, launches);
    return bad > 0 || !refused;
}
