// Which bytes of a cache the kernels of attn_window.hip ask for: plain integer arithmetic, also compiled for the host by the test of these maps.
//
// A kernel reads a head's rows through descriptors (base: the head's first row; size: live rows times bytes of a row), whose loads return zeros where they lie behind the size.  Offsets are
// 32 bits: a tile's first byte plus a lane's own.  A load is 16, 8 or 1 bytes of one row, at a multiple of its width, and rows are multiples of that, so that it lies either within a live row or wholly behind the
// size; the last tile that is ever asked for ends below 2^32 (MAX_ROWS).
#pragma once
#include <cstdint>
#include "dream.h"

namespace dream {

constexpr uint32_t TILE = 32;                                      // keys of a tile
constexpr int64_t MAX_ROWS = DREAM_MAX_WINDOW_ROWS;                // of a head: up to 512 bytes each
constexpr int row_bytes(int D, bool mx) { return mx ? D / 2 : D * 2; }
constexpr int scale_bytes(int D) { return D / DREAM_MX_GROUP; }    // of a row

constexpr int least(int a, int b) { return a < b ? a : b; }
constexpr int most(int a, int b) { return a > b ? a : b; }

// The prefix rows of a sequence, never past the cache, whatever the array holds.
constexpr int prefix_rows(int given, uint32_t s_max, int n_tree) { return least(most(given, 0), (int)s_max - n_tree); }

// The first tile that lies wholly behind `rows` rows.
template <class Rows>
constexpr uint32_t tile_behind(Rows rows) { return (rows + 31) / 32; }
// What a wave asks for before the number of live rows is known, under a descriptor of the whole cache.
constexpr uint32_t early_tile(uint32_t wave, uint32_t s_max) { return wave < tile_behind(s_max) ? wave : tile_behind(s_max); }

// The key tiles of a sequence, in the order they are taken: those of the sinks, then those from the root's window on.
struct Tiles {
    int sinks, first, count;
    constexpr int at(int i) const { return i < sinks ? i : i - sinks + first; }
};
template <class Args>      // window, n_sink, n_tree
constexpr Tiles tiles_of(const Args &a, int P)
{
    Tiles t = {};
    const int start = a.window ? most(0, P - a.window + 1) : 0;
    t.sinks = a.window ? (least(a.n_sink, start) + 31) / 32 : 0;
    t.first = most(start / 32, t.sinks);
    t.count = t.sinks + (P + a.n_tree + 31) / 32 - t.first;
    return t;
}
// A split's part of the list: tiles of a split; behind its last.  (In the place of a tile behind that the kernels ask for the one behind the live rows.)
constexpr int tiles_per_split(int count, uint32_t lg_splits) { return lg_splits == 0 ? count : (uint32_t)(count + (1u << lg_splits) - 1) >> lg_splits; }
constexpr int split_end(int count, uint32_t split, int per) { return least(count, (int)(split * per) + per); }

// window_attn_kernel: bytes from the tile's first on.  K: lane (c, g) = (lane % 16, lane / 16) takes key c of either half, piece after piece (of 4 bits at head_dim 64 8 bytes, else 16).
template <int D, bool MX>
struct WaveLoads {
    static constexpr int ROW = row_bytes(D, MX), SCALES = scale_bytes(D);
    static constexpr int K_WIDTH = MX && D == 64 ? 8 : 16, K_PIECES = MX ? (D == 256 ? 2 : 1) : D / 32;      // of a lane and a half
    static constexpr int V_PER_ROW = ROW / 16, V_PIECES = 32 * V_PER_ROW / 64;                               // of a lane
    static constexpr uint32_t k(int c, int g) { return c * ROW + g * K_WIDTH; }
    static constexpr uint32_t k_further(int half, int piece) { return half * 16 * ROW + piece * 64; }
    static constexpr uint32_t k_scale(int c, int g) { return c * SCALES + (D == 64 ? g >> 1 : g); }
    static constexpr uint32_t k_scale_further(int half, int piece) { return half * 16 * SCALES + piece * 4; }
    // V in the order of memory; of 4 bits a piece is what has one scale
    static constexpr uint32_t v(int lane) { return lane * 16; }
    static constexpr uint32_t v_further(int piece) { return piece * 1024; }
    static constexpr uint32_t v_scale(int lane) { return lane; }
    static constexpr uint32_t v_scale_further(int piece) { return piece * 64; }
    static constexpr int v_row(int lane, int piece) { return lane / V_PER_ROW + piece * (64 / V_PER_ROW); }
    static constexpr int V_VALUES = MX ? 32 : 8;                                                             // of a piece
    static constexpr int v_column(int lane) { return lane % V_PER_ROW; }                                     // pieces in front of it
};
// First of the 8 channels of k-step ks that lane group g holds: of a 4-bit row consecutive runs of what it loads at once.
template <int D, bool MX>
constexpr int channel_of(int ks, int g)
{
    return !MX ? ks * 32 + g * 8 : D == 64 ? g * 16 + ks * 8 : (ks >> 2) * 128 + g * 32 + (ks & 3) * 8;
}

// window_shared_kernel: the threads take K's pieces, and V's, in the order of memory; where a tile has half as many as there are threads, one half of them takes K and the other V.
template <int D, bool MX>
struct GroupLoads {
    static constexpr int THREADS = 512;
    static constexpr int ROW = row_bytes(D, MX), SCALES = scale_bytes(D);
    static constexpr int PIECE = MX ? D / 8 : 8, WIDTH = MX ? PIECE / 2 : 16;                // values, bytes
    static constexpr int PER_ROW = D / PIECE;
    static constexpr bool HALVES = 32 * PER_ROW < THREADS;
    static constexpr int PIECES = HALVES ? 1 : 32 * PER_ROW / THREADS;                       // of a thread, of K and of V
    static_assert(HALVES ? 64 * PER_ROW == THREADS : 32 * PER_ROW % THREADS == 0, "pieces");
    static constexpr int thread(int tid) { return HALVES ? tid % (THREADS / 2) : tid; }      // among those that take the same tensor
    static constexpr bool takes_v(int tid) { return HALVES && tid >= THREADS / 2; }          // (where not HALVES, every thread takes both)
    static constexpr uint32_t at(int thread) { return thread * WIDTH; }
    static constexpr uint32_t further(int piece) { return piece * THREADS * WIDTH; }
    static constexpr uint32_t scale(int thread) { return thread * PIECE / DREAM_MX_GROUP; }
    static constexpr uint32_t scale_further(int piece) { return piece * THREADS * PIECE / DREAM_MX_GROUP; }
    static constexpr int row(int thread, int piece) { return (thread + piece * THREADS) / PER_ROW; }
    static constexpr int channel(int thread, int piece) { return (thread + piece * THREADS) % PER_ROW * PIECE; }
};

}  // namespace dream
