// The address maps of csrc/window_maps.h for the host: what tests/test_window_maps.py checks.
#include "window_maps.h"

using namespace dream;

// one load: tensor (0 K, 1 V, 2 K's scales, 3 V's), lane or thread, half, piece, bytes from the descriptor's base as the kernels add them up (32 bits), width, the row and the channel it is used for (-1: see channel_of)
struct Load {
    int64_t tensor, lane, half, piece, at, width, row, channel;
};

template <int D, bool MX>
static int of_wave(uint32_t tile, Load *out)
{
    using L = WaveLoads<D, MX>;
    int n = 0;
    for (int lane = 0; lane < 64; lane++) {
        const int c = lane & 15, g = lane >> 4;
        const uint32_t k = L::k(c, g) + tile * (TILE * L::ROW), ks = L::k_scale(c, g) + tile * (TILE * L::SCALES);
        const uint32_t v = L::v(lane) + tile * (TILE * L::ROW), vs = L::v_scale(lane) + tile * (TILE * L::SCALES);
        for (int half = 0; half < 2; half++)
            for (int i = 0; i < L::K_PIECES; i++) {
                out[n++] = {0, lane, half, i, k + L::k_further(half, i), L::K_WIDTH, half * 16 + c, -1};
                if (MX)
                    out[n++] = {2, lane, half, i, ks + L::k_scale_further(half, i), 1, half * 16 + c, -1};
            }
        for (int i = 0; i < L::V_PIECES; i++) {
            out[n++] = {1, lane, 0, i, v + L::v_further(i), 16, L::v_row(lane, i), L::v_column(lane) * L::V_VALUES};
            if (MX)
                out[n++] = {3, lane, 0, i, vs + L::v_scale_further(i), 1, L::v_row(lane, i), L::v_column(lane) * L::V_VALUES};
        }
    }
    return n;
}

template <int D, bool MX>
static int of_group(uint32_t tile, Load *out)
{
    using L = GroupLoads<D, MX>;
    int n = 0;
    for (int tid = 0; tid < L::THREADS; tid++)
        for (int v = 0; v < 2; v++) {
            if (L::HALVES && L::takes_v(tid) != (v == 1))
                continue;
            const int t = L::thread(tid);
            const uint32_t at = L::at(t) + tile * (TILE * L::ROW), scale = L::scale(t) + tile * (TILE * L::SCALES);
            for (int i = 0; i < L::PIECES; i++) {
                out[n++] = {v, tid, 0, i, at + L::further(i), L::WIDTH, L::row(t, i), L::channel(t, i)};
                if (MX)
                    out[n++] = {2 + v, tid, 0, i, scale + L::scale_further(i), 1, L::row(t, i), L::channel(t, i)};
            }
        }
    return n;
}

struct Call {
    int window, n_sink, n_tree;
};

extern "C" {
int wave_loads(int D, int mx, uint32_t tile, Load *out)
{
    return D == 64    ? (mx ? of_wave<64, true>(tile, out) : of_wave<64, false>(tile, out))
           : D == 128 ? (mx ? of_wave<128, true>(tile, out) : of_wave<128, false>(tile, out))
                      : (mx ? of_wave<256, true>(tile, out) : of_wave<256, false>(tile, out));
}
int group_loads(int D, int mx, uint32_t tile, Load *out)
{
    return D == 64    ? of_group<64, false>(tile, out)
           : D == 128 ? (mx ? of_group<128, true>(tile, out) : of_group<128, false>(tile, out))
                      : (mx ? of_group<256, true>(tile, out) : of_group<256, false>(tile, out));
}
int wave_channel(int D, int mx, int ks, int g)
{
    return D == 64 ? (mx ? channel_of<64, true>(ks, g) : channel_of<64, false>(ks, g))
           : D == 128 ? (mx ? channel_of<128, true>(ks, g) : channel_of<128, false>(ks, g)) : (mx ? channel_of<256, true>(ks, g) : channel_of<256, false>(ks, g));
}
int bytes_of_row(int D, int mx) { return row_bytes(D, mx); }
int bytes_of_scales(int D) { return scale_bytes(D); }
int64_t most_rows() { return MAX_ROWS; }
int live_prefix(int given, uint32_t s_max, int n_tree) { return prefix_rows(given, s_max, n_tree); }
uint32_t behind(uint32_t rows) { return tile_behind(rows); }
uint32_t early(uint32_t wave, uint32_t s_max) { return early_tile(wave, s_max); }
// the list of tiles; returns how many
int tile_list(int window, int n_sink, int n_tree, int P, int32_t *out, int room)
{
    const Tiles t = tiles_of(Call{window, n_sink, n_tree}, P);
    for (int i = 0; i < t.count && i < room; i++)
        out[i] = t.at(i);
    return t.count;
}
// the tile asked for in the place of the t-th of the list, by a workgroup with this split (as in the kernels)
uint32_t asked_for(int window, int n_sink, int n_tree, int P, uint32_t split, uint32_t lg_splits, int t)
{
    const Tiles tiles = tiles_of(Call{window, n_sink, n_tree}, P);
    return t < split_end(tiles.count, split, tiles_per_split(tiles.count, lg_splits)) ? (uint32_t)tiles.at(t) : tile_behind(P + n_tree);
}
void share(int count, uint32_t split, uint32_t lg_splits, int32_t *out)
{
    const int per = tiles_per_split(count, lg_splits);
    out[0] = split * per;
    out[1] = split_end(count, split, per);
}
}
