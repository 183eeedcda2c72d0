/* Which kernels dream_window_verify_attn and dream_mx_verify_attn launch, and how: this program defines the HIP functions through which libdream registers and launches its kernels, so that
 * nothing reaches a device.  Reads calls from stdin, one a line: mx dtype batch q_heads kv_heads head_dim n_tree max_kv_len window n_sink q_tiles waves splits; answers each with the
 * status, and per launch the kernel's name, its grid, threads and the words that say which workgroup does what. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include "dream.h"
#include "dream_tuning.h"

typedef struct { unsigned x, y, z; } grid3;

enum { MAX_FUNCS = 1024 };
static struct { const void *stub; const char *name; } known[MAX_FUNCS];
static int n_known;

void __hipRegisterFunction(void **modules, const void *stub, char *device, const char *name, unsigned limit, void *tid, void *bid, void *block, void *grid, int *size)
{
    (void)modules; (void)device; (void)limit; (void)tid; (void)bid; (void)block; (void)grid; (void)size;
    if (n_known == MAX_FUNCS)
        exit(3);
    known[n_known].stub = stub;
    known[n_known++].name = name;
}
int hipGetDevice(int *current) { *current = 0; return 0; }
int hipGetLastError(void) { return 0; }
static struct { grid3 grid, block; size_t lds; void *stream; } config;
int __hipPushCallConfiguration(grid3 grid, grid3 block, size_t lds, void *stream)
{
    config.grid = grid;
    config.block = block;
    config.lds = lds;
    config.stream = stream;
    return 0;
}
int __hipPopCallConfiguration(grid3 *grid, grid3 *block, size_t *lds, void **stream)
{
    *grid = config.grid;
    *block = config.block;
    *lds = config.lds;
    *stream = config.stream;
    return 0;
}
int hipLaunchKernel(const void *f, grid3 grid, grid3 block, void **args, size_t lds, void *stream)
{
    const char *name = "?";
    (void)lds; (void)stream;
    for (int i = 0; i < n_known; i++)
        if (known[i].stub == f)
            name = known[i].name;
    printf(" %s %u %u %u %u", name, grid.x, grid.y, grid.z, block.x * block.y * block.z);
    /* k, v, k_scales, v_scales, prefix_len, s_max, heads_splits, heads_magic, tree_units, ... of the two kernels that take the keys in tiles */
    if (block.x == 256 || block.x == 512) {
        int tiled = 0;
        for (const char *p = name; *p; p++)
            tiled |= (p[0] == 'w' && p[1] == 'i' && p[7] == 'a' && p[8] == 't') || (p[0] == 'w' && p[1] == 'i' && p[7] == 's');
        printf(" %u %u %u", tiled ? *(uint32_t *)args[6] : 0, tiled ? *(uint32_t *)args[7] : 0, tiled ? *(uint32_t *)args[8] : 0);
    }
    return 0;
}

int main(void)
{
    int mx, dtype, b, hq, hkv, d, t, window, sink, tiles, waves, splits;
    long long keys;
    void *const p = (void *)0x10000;         /* never dereferenced: nothing runs */
    while (scanf("%d %d %d %d %d %d %d %lld %d %d %d %d %d", &mx, &dtype, &b, &hq, &hkv, &d, &t, &keys, &window, &sink, &tiles, &waves, &splits) == 13) {
        const dream_attn_desc desc = {b, hq, hkv, d, dtype, 0.0f, keys};
        dream_set_q_tiles(tiles);
        dream_set_tile_waves(waves);
        dream_set_kv_splits(splits);
        const size_t bytes = mx ? dream_mx_verify_attn_workspace(&desc, t, keys, window, sink) : dream_window_verify_attn_workspace(&desc, t, keys, window, sink);
        const int status = mx ? dream_mx_verify_attn(&desc, p, p, p, p, p, p, t, p, NULL, window, sink, keys, p, NULL, p, bytes, NULL)
                              : dream_window_verify_attn(&desc, p, p, p, p, t, p, NULL, window, sink, keys, p, NULL, p, bytes, NULL);
        printf(" %d\n", status);
    }
    return 0;
}
