// Tree-masked attention that may see a window of positions and the first tokens only (dream_window_verify_attn), and the same over caches held in 4 bits (dream_mx_verify_attn).
//
// out_i = sum_j softmax_j(scale q_i k_j) v_j over the keys j that node i sees (Eq. 1 under the draft-tree mask of Section 3.1): with a window w, keys of the prefix less than w
// positions back from the node's own (prefix length plus depth), the first n_sink keys, and of the tree's nodes those that its mask names and the window reaches.  Keys that no node sees
// are not read: the range is cut into tiles of 32 keys, first those of the sinks, then those from the root's window on.
//
// A workgroup serves QT tiles of 16 query rows of one KV head (the rows that share it are numbered through all heads of its group) and one share of the key tiles; its NW waves take the tiles
// in turn, each for all of the rows, and never meet until the end.  One pass over the keys with a running maximum and sum (raised only when a score exceeds the reference by 8 octaves):
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16 with the keys as A operand.  The order of the channels is free as long as both operands agree, so a lane takes what it can load at
//                 once: of a 4-bit row 16 bytes, the 32 channels of one scale, which go from memory through v_cvt_scalef32_pk_bf16_fp4 (exact: code times power of two) straight into the operand.
//   O^T += V^T P^T   the scores' registers, as bf16, are the B operand; V needs turning, so a wave writes its rows (as bf16) to LDS that is its own and reads them transposed.
// A row of 4 bits is turned into bf16 once for all QT tiles of a wave.  (The matrix instruction that takes 4-bit operands beside 8-bit ones, with the queries as two parts, drops what lies 2^13
// below its largest product; the scores would be off by more than the rounding of bf16 rows allows.)
//
// What bounds it: a wave issues a vector instruction every 6 clocks alone and every 3.5 to 5.5 beside a second one, a scalar one every 10; a step over 32 keys is some 200 to 340 of them
// (head_dim 128, one query tile: 1500 clocks), and before the first lie the arguments, the prefix length, the tree and the first tile from memory, 4200 clocks.  Where many waves share a SIMD
// that is issue (of a SIMD's time 89 % at B 32, 74 % at B 8); a lone wave waits, step after step, for its own chain of conversions, products, maximum and LDS.  Measured, one call of a
// graph (medians; a few percent from one run to the next), against 5.2 TB/s for a large copy and 1390 TFLOP/s for a large matrix product:
//   4-bit   B 1, 32 heads of 128, 60 nodes, 704 keys     7.6 us    (read and written: 4.3 MB, 0.8 us; a kernel that does nothing 1.6 us; issue 44 %: 128 workgroups, six steps a wave)
//           B 8, 32 heads on 8, 128, 60 nodes, 1283     19.6 us    (8.1 GFLOP, 5.8 us)
//           B 32, 32 heads of 64, 60 nodes, 1600        46 to 49 us    (131 MB, 25 us; 26 GFLOP, 19 us)
//           B 4, 32 heads on 8, 128, 1 node, 32700      30.4 us    (122 MB, 24 us)
//   16-bit  B 4, 16 heads on 8, 256, 33 nodes, window 1024 of 1283    22.9 us    (36 MB, 7.0 us; the states of 8 splits are 17 MB, written and then read: 6.7 us)
//           B 1, 32 heads of 128, 1 node, window 1020 and 4 first tokens    10.9 us    (17 MB, 3.3 us; two launches)
#include <cfloat>
#include <type_traits>
#include "common.h"
#include "quick_div.h"
#include "window_maps.h"

using namespace dream;

namespace {

constexpr int GROUP = DREAM_MX_GROUP;
constexpr float SLACK = 8.0f;      // octaves by which a score may exceed its row's reference
constexpr int MAX_SPLITS = 64;
constexpr uint32_t UNITS_Y = 32768;   // units of a grid's second dimension, by eights

struct WindowArgs {
    const void *q, *k, *v;           // k, v: codes where the cache is held in 4 bits
    const uint8_t *k_scales, *v_scales;
    const int32_t *prefix_len, *parent;
    const uint64_t *tree_mask;
    void *out;
    float *lse;
    float *part, *part_ml;           // split states: O [slot][D]; reference and sum [slot][2]
    int64_t s_max;
    int32_t n_q_heads, n_kv_heads, group, n_tree, mask_words, window, n_sink;
    int32_t n_rg, n_splits, n_units; // row groups of a KV head; key splits; B * Hkv * n_splits
    uint32_t tree_magic, heads_magic; // for quick_div by n_tree, by n_kv_heads
    float scale, scale_log2;
};

// A value that every lane of a wave wants and this launch does not write, by the scalar unit: a vector load would be waited for before anything that follows it.
__device__ __forceinline__ int scalar_load(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }

// Bits of the 32 keys from j0 on that lie in [from, to).
__device__ __forceinline__ uint32_t key_bits(int j0, int from, int to)
{
    const int lo = max(from - j0, 0), hi = min(to - j0, 32);
    if (lo >= hi)
        return 0u;
    return (0xffffffffu >> (32 - (hi - lo))) << lo;
}

// Which tree nodes the rows see (bit a % 64 of word a / 64) and how deep they are; in LDS.
struct Tree {
    uint64_t *mask;
    int32_t *depth;
    int32_t deepest;
};

// Takes what the window leaves out of the masks of nodes [first, T), every `step`-th; only where the window may end inside the tree.
__device__ __forceinline__ void cut_masks(const Tree &t, const WindowArgs &a, int P, int first, int step)
{
    const int W = a.mask_words;
    for (int i = first; i < a.n_tree; i += step)
        for (int w = 0; w < W; w++) {
            uint64_t m = t.mask[i * W + w], keep = m;
            while (m) {
                const int bit = __builtin_ctzll(m), n = w * 64 + bit;
                m &= m - 1;
                if (t.depth[i] - t.depth[n] >= a.window && P + t.depth[n] >= a.n_sink)
                    keep &= ~(1ull << bit);
            }
            t.mask[i * W + w] = keep;
        }
}

// Trees of up to 64 nodes: every wave has its own in registers, lane l node l's mask and depth, and meets nobody.  `parent`: of this lane's node (-1: none).  The paths are joined by halves:
// a node's mask holds its path up to `up`, and takes in what `up` has found; log2 of the depth rounds.
struct SmallTree {
    uint64_t mask;
    int depth, deepest;
};
__device__ __forceinline__ SmallTree small_tree(const WindowArgs &a, bool windowed, int b, int T, int parent, int lane)
{
    SmallTree t = {1ull << lane, 0, 0};
    int up = parent;
    while (__any(up >= 0)) {
        const int from = max(up, 0);
        const uint64_t more = (uint64_t)(uint32_t)__shfl((int)(t.mask >> 32), from) << 32 | (uint32_t)__shfl((int)t.mask, from);
        const int next = __shfl(up, from);
        t.mask |= up >= 0 ? more : 0ull;
        up = up >= 0 ? next : -1;
    }
    if (windowed) {
        t.depth = __popcll(t.mask) - 1;
        t.deepest = (int)wave_max((float)t.depth);
    }
    if (a.tree_mask) {
        t.mask = lane < T ? a.tree_mask[(int64_t)b * T + lane] : 0ull;
        if (T < 64)
            t.mask &= (1ull << T) - 1;
    }
    return t;
}
// Takes what the window leaves out of the masks; only where it may end inside the tree.  `depths`: 64 words of LDS.
__device__ __forceinline__ void cut_small_masks(SmallTree &t, const WindowArgs &a, int P, int32_t *depths, int lane)
{
    depths[lane] = t.depth;
    wave_lds_fence();
    uint64_t m = t.mask;
    while (m) {
        const int bit = __builtin_ctzll(m), depth = depths[bit];
        m &= m - 1;
        if (t.depth - depth >= a.window && P + depth >= a.n_sink)
            t.mask &= ~(1ull << bit);
    }
}

// Any tree, by all threads of the workgroup; ends with a barrier.  `parent` (n_tree of them) and `deepest` are LDS.
__device__ __forceinline__ void build_tree(Tree &t, const WindowArgs &a, int b, int P, int32_t *parent, int32_t *deepest, int tid, int threads)
{
    const int T = a.n_tree, W = a.mask_words;
    const bool walk = !a.tree_mask || a.window;
    if (walk) {
        for (int i = tid; i < T; i += threads) {
            const int p = a.parent[(int64_t)b * T + i];
            parent[i] = p < i ? p : -1;        // a walk up the tree always ends
        }
        if (tid == 0)
            *deepest = 0;
        __syncthreads();
    }
    for (int i = tid; i < T; i += threads) {
        for (int w = 0; w < W; w++) {
            uint64_t m = 0;
            if (a.tree_mask) {
                m = a.tree_mask[((int64_t)b * T + i) * W + w];
                if (T - w * 64 < 64)
                    m &= (1ull << (T - w * 64)) - 1;
            } else if (i >> 6 == w) {
                m = 1ull << (i & 63);
            }
            t.mask[i * W + w] = m;
        }
        if (walk) {
            int depth = 0;
            for (int p = parent[i]; p >= 0; p = parent[p]) {
                depth++;
                if (!a.tree_mask)
                    t.mask[i * W + (p >> 6)] |= 1ull << (p & 63);
            }
            t.depth[i] = depth;
            if (a.window)
                atomicMax(deepest, depth);
        }
    }
    __syncthreads();
    t.deepest = a.window ? *deepest : 0;
    if (a.window && a.window < T) {
        cut_masks(t, a, P, tid, threads);
        __syncthreads();
    }
}

// The keys of the prefix from j0 on that a node of this depth sees.  lo: where the root's window starts.
__device__ __forceinline__ uint32_t visible_prefix(const WindowArgs &a, int depth, int lo, int P, int j0)
{
    return a.window ? key_bits(j0, lo + depth, P) | key_bits(j0, 0, min(a.n_sink, P)) : key_bits(j0, 0, P);
}
// And of the tree, as its mask has them: one word, or those of a large tree in LDS.
__device__ __forceinline__ uint32_t visible_nodes(uint64_t mask, int P, int j0)
{
    const int rel = j0 - P;
    return rel <= -32 || rel >= 64 ? 0u : rel <= 0 ? (uint32_t)(mask << -rel) : (uint32_t)(mask >> rel);
}
__device__ __forceinline__ uint32_t visible_keys(const Tree &t, const WindowArgs &a, int node, int lo, int P, int j0)
{
    uint32_t bits = visible_prefix(a, a.window ? t.depth[node] : 0, lo, P, j0);
    const int rel = j0 - P, W = a.mask_words;
    if (rel > -32 && rel < a.n_tree) {
        const uint64_t *m = t.mask + node * W;
        if (rel <= 0) {
            bits |= (uint32_t)(m[0] << -rel);
        } else {
            const int w = rel >> 6, s = rel & 63;
            uint64_t x = m[w] >> s;
            if (s && w + 1 < W)
                x |= m[w + 1] << (64 - s);
            bits |= (uint32_t)x;
        }
    }
    return bits;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8 from_codes(uint32_t codes, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The largest of eight scores; NaN where one is (v_maximum3_f32, which needs no quieting of its inputs).
__device__ __forceinline__ float largest(f32x4 a, f32x4 b)
{
    auto of = [](float x, float y) { return __builtin_elementwise_maximum(x, y); };
    return of(of(of(of(of(of(of(a[0], a[1]), a[2]), a[3]), b[0]), b[1]), b[2]), b[3]);
}
// not 0 where one of the two bf16 values is not finite
__device__ __forceinline__ uint32_t strange_halves(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ u32x4 without_strange(u32x4 x)
{
#pragma unroll
    for (int e = 0; e < 4; e++)
        x[e] &= ((x[e] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((x[e] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
    return x;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// `bytes` from `base` on (the same in all lanes) as a buffer: loads behind its end return zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint8_t *base, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// What a wave has of one tile, as it came from memory.
template <int D, bool MX>
struct Raw;
template <int D>
struct Raw<D, true> {
    static constexpr int KP = WaveLoads<D, true>::K_PIECES, VP = WaveLoads<D, true>::V_PIECES;
    uint32_t k[2][D / 32];
    uint8_t ks[2][KP];
    u32x4 v[VP];
    uint8_t vs[VP];
};
template <int D>
struct Raw<D, false> {
    u32x4 k[2][D / 32];
    u32x4 v[D / 16];
};

// The state of a query tile: O^T (a lane owns query row c = lane % 16 and channels 16 dt + 4 (lane / 16) + r), the reference of its scores in octaves and the lane's share of the sum.
template <int QT, int NDT>
struct RowState {
    f32x4 o[QT][NDT];
    float m[QT], l[QT];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            m[qt] = -INFINITY;
            l[qt] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)
                o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
};

// Online softmax of a tile of 32 keys: a lane owns query row c and keys 4 g + r of both halves.  `vis` (of this lane's eight keys: bits 0 to 3 and 16 to 19) counts where the tile is not `whole`.
// The scores are left as they are, and what the two kinds of tile do apart stands apart: values that either way may have written are copied on both.
// Probabilities are rounded to bf16, half a step of 2^-8 each, as the matrix instruction takes them; sums stay float32.
template <bool WHOLE, int QT, int NDT>
__device__ __forceinline__ void softmax_tile(f32x4 (&s)[2][QT], RowState<QT, NDT> &st, const uint32_t (&vis)[QT], float scale_log2, bf16x8 (&pf)[QT])
{
    auto seen = [&](int qt, int e) { return (vis[qt] >> ((e >> 2) * 16 + (e & 3)) & 1u) != 0u; };
    float top[QT];
    if constexpr (WHOLE) {
#pragma unroll
        for (int qt = 0; qt < QT; qt++)
            top[qt] = largest(s[0][qt], s[1][qt]) * scale_log2;
    } else {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                s[e >> 2][qt][e & 3] = seen(qt, e) ? s[e >> 2][qt][e & 3] * scale_log2 : -INFINITY;
            top[qt] = largest(s[0][qt], s[1][qt]);
        }
    }
    bool raise = false;
#pragma unroll
    for (int qt = 0; qt < QT; qt++)
        raise = raise || top[qt] > st.m[qt] + SLACK;
    if (__any(raise)) {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            float x = fmaxf(top[qt], __shfl_xor(top[qt], 16));
            x = fmaxf(x, __shfl_xor(x, 32));
            if (x > st.m[qt] + SLACK) {
                const float f = __builtin_amdgcn_exp2f(st.m[qt] - x);       // 0 where nothing was seen before
                st.m[qt] = x;
                st.l[qt] *= f;
#pragma unroll
                for (int dt = 0; dt < NDT; dt++)
                    st.o[qt][dt] *= f;
            }
        }
    }
    float sum[QT];
    if constexpr (WHOLE) {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const float ref = fmaxf(st.m[qt], -FLT_MAX);      // where all scores so far are -inf, their weight is 0 and not exp(-inf + inf)
            sum[qt] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][qt][e & 3], scale_log2, -ref));
                sum[qt] += p;
                pf[qt][e] = (__bf16)p;
            }
        }
    } else {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const float ref = st.m[qt] == -INFINITY ? 0.0f : st.m[qt];
            sum[qt] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float p = __builtin_amdgcn_exp2f(s[e >> 2][qt][e & 3] - ref);
                sum[qt] += p;
                pf[qt][e] = (__bf16)p;
            }
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; qt++)
        st.l[qt] += sum[qt];
}

// V^T for channels 16 dt .. +15 of a 32-key tile [32][VSTR] in LDS, as the A operand whose keys are in the order in which a lane holds its probabilities.
template <int VSTR>
__device__ __forceinline__ bf16x8 read_turned(const uint16_t *tile, int dt, int c, int g)
{
    const uint16_t *at = tile + (g * 4 + (c >> 2)) * VSTR + (c & 3) * 4 + dt * 16;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 16 * VSTR));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// O^T += V^T P^T
template <int QT, int NDT, int VSTR>
__device__ __forceinline__ void add_values(const uint16_t *tile, const bf16x8 (&pf)[QT], RowState<QT, NDT> &st, int c, int g)
{
#pragma unroll
    for (int dt = 0; dt < NDT; dt++) {
        const bf16x8 vf = read_turned<VSTR>(tile, dt, c, g);
#pragma unroll
        for (int qt = 0; qt < QT; qt++)
            st.o[qt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qt], st.o[qt][dt], 0, 0, 0);
    }
}

// Of a tile [32][VSTR] that holds ones in the places of values that are not finite: how many of them the keys in `vis` have, per channel; what counts any is NaN.
template <int QT, int NDT, int VSTR>
__device__ __forceinline__ void mark_strange(const uint16_t *tile, int qt, uint32_t vis, RowState<QT, NDT> &st, int c, int g)
{
    bf16x8 seen;
#pragma unroll
    for (int e = 0; e < 8; e++)
        seen[e] = (__bf16)(float)(vis >> ((e >> 2) * 16 + (e & 3)) & 1u);
#pragma unroll
    for (int dt = 0; dt < NDT; dt++) {
        const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(read_turned<VSTR>(tile, dt, c, g), seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; r++)
            st.o[qt][dt][r] = n[r] > 0.0f ? __builtin_nanf("") : st.o[qt][dt][r];
    }
}
// ones in the places of values that are not finite
__device__ __forceinline__ u32x4 strange_places(u32x4 x)
{
#pragma unroll
    for (int e = 0; e < 4; e++)
        x[e] = ((x[e] & 0x7f80u) == 0x7f80u ? 0x3f80u : 0u) | ((x[e] & 0x7f800000u) == 0x7f800000u ? 0x3f800000u : 0u);
    return x;
}

// Workgroup ids that are congruent mod 8 run on one XCD.  Row groups of one unit (a stream's share of the keys) meet in one XCD's L2, or, where there are so few units that XCDs would stay
// without, in that of 2, 4 or 8.
struct Place {
    uint32_t unit, rg;
};
__device__ __forceinline__ Place place_of(uint32_t heads_splits)
{
    const uint32_t lg = heads_splits >> 24, part = (blockIdx.z * UNITS_Y + blockIdx.y) * 8 + (blockIdx.x & 7);
    return {part >> lg, (blockIdx.x >> 3) << lg | (part & ((1u << lg) - 1))};
}

template <int D, int QT, int NW, bool MX>
struct WindowGeom {
    static constexpr int VSTR = D + 16;                          // V row stride in LDS (values): four consecutive rows land 8 banks apart
    static constexpr int TILE = 32 * VSTR * 2, STATE = QT * 16 * D * 4;
    static constexpr int AREA = TILE > STATE ? TILE : STATE;     // bytes of a wave's LDS: its V tile, at the end its O
    // waves of a SIMD that the registers have to leave room for: O, the queries, the scores and the tiles as they come from memory
    static constexpr int WAVES = MX ? (D == 64 ? (QT == 1 ? 4 : QT == 2 ? 3 : 2) : D == 128 ? (QT == 1 ? 3 : 2) : 2) : D == 64 ? (QT == 1 ? 4 : 3) : D == 128 ? 2 : 1;
};

// Key tiles shared out over NW waves: few rows read the same keys, so what counts is that many waves have a tile each on its way.  Each wave asks for its next tile as soon as a tile's
// registers are free (two, three or four tiles ahead brought nothing: code that is unrolled for them costs what waiting less wins; lines touched two steps ahead, into the L2, neither).
// What stands ahead of a launch's first loads comes as plain arguments, the 14 dwords that are in scalar registers when a wave starts.
template <int D, int QT, int NW, bool MX>
__global__ __launch_bounds__(64 * NW, (WindowGeom<D, QT, NW, MX>::WAVES)) void window_attn_kernel(const uint8_t *k, const uint8_t *v, const uint8_t *k_scales, const uint8_t *v_scales,
                                                                                                const int32_t *prefix_len, uint32_t s_max, uint32_t heads_splits, uint32_t heads_magic,
                                                                                                uint32_t tree_units, WindowArgs a)
{
    using G = WindowGeom<D, QT, NW, MX>;
    constexpr int NKS = D / 32, NDT = D / 16, VSTR = G::VSTR;
    using Loads = WaveLoads<D, MX>;
    constexpr int ROWB = Loads::ROW, SCB = Loads::SCALES;        // bytes of a row, and of its scales
    __shared__ __attribute__((aligned(16))) uint8_t s_area[NW][G::AREA];
    __shared__ uint64_t s_mask[DREAM_MAX_TREE * 4];              // of more than 64 nodes
    __shared__ int32_t s_depth[DREAM_MAX_TREE], s_parent[DREAM_MAX_TREE], s_deepest;
    __shared__ float s_ml[NW][QT][2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const Place place = place_of(heads_splits);
    const uint32_t unit = place.unit, rg = place.rg, n_heads = heads_splits & 0xffff, lg_splits = heads_splits >> 16 & 0xff, n_splits = 1u << lg_splits;
    const int T = tree_units & 0x1ff;
    const bool windowed = tree_units & 0x200;
    if (unit >= tree_units >> 10)
        return;
    const uint32_t stream = unit >> lg_splits, split = unit & (n_splits - 1);
    const uint32_t b = quick_div(stream, heads_magic), kvh = stream - b * n_heads;
    const int prefix = scalar_load(prefix_len + b);
    const int64_t head_row = (int64_t)stream * s_max;
    k += head_row * ROWB;
    v += head_row * ROWB;
    k_scales += head_row * SCB;
    v_scales += head_row * SCB;

    // The pieces of a tile that this lane loads: K's as the matrix instruction has them, V's in the order of memory.  Every call has as many loads, so that what waits for one tile never
    // waits for another: behind the last live row, and for a tile that is not this workgroup's, they return zeros and go nowhere (the descriptors' bounds).  One descriptor a tensor
    // for the whole range: a scalar instruction costs a wave as long as ten vector lanes' work (a wave's scalar instructions issue every 10 clocks, its vector ones every 6).
    constexpr int VPL = Loads::V_PIECES;
    const int vrow = Loads::v_row(lane, 0), vcol = Loads::v_column(lane);
    struct Range {
        __amdgpu_buffer_rsrc_t k, v, ks, vs;
    };
    auto range_of = [&](uint32_t rows) __attribute__((always_inline)) {
        Range r;
        r.k = buffer_of(k, rows * ROWB);
        r.v = buffer_of(v, rows * ROWB);
        if (MX) {
            r.ks = buffer_of(k_scales, rows * SCB);
            r.vs = buffer_of(v_scales, rows * SCB);
        }
        return r;
    };
    const uint32_t k_at = Loads::k(c, g), ks_at = Loads::k_scale(c, g);
    auto request_k = [&](Raw<D, MX> &r, const Range &from, uint32_t tile) __attribute__((always_inline)) {
        const uint32_t at = k_at + tile * (TILE * ROWB);
#pragma unroll
        for (int hh = 0; hh < 2; hh++) {
            if constexpr (!MX) {
#pragma unroll
                for (int ks = 0; ks < NKS; ks++)
                    r.k[hh][ks] = __builtin_amdgcn_raw_buffer_load_b128(from.k, at + Loads::k_further(hh, ks), 0, 0);
            } else if constexpr (D == 64) {
                const auto x = __builtin_amdgcn_raw_buffer_load_b64(from.k, at + Loads::k_further(hh, 0), 0, 0);
                r.k[hh][0] = x[0];
                r.k[hh][1] = x[1];
            } else {
#pragma unroll
                for (int i = 0; i < Loads::K_PIECES; i++) {
                    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from.k, at + Loads::k_further(hh, i), 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        r.k[hh][i * 4 + e] = x[e];
                }
            }
        }
        if constexpr (MX) {
            const uint32_t sat = ks_at + tile * (TILE * SCB);
#pragma unroll
            for (int hh = 0; hh < 2; hh++)
#pragma unroll
                for (int i = 0; i < Raw<D, MX>::KP; i++)
                    r.ks[hh][i] = __builtin_amdgcn_raw_buffer_load_b8(from.ks, sat + Loads::k_scale_further(hh, i), 0, 0);
        }
    };
    auto request_v = [&](Raw<D, MX> &r, const Range &from, uint32_t tile) __attribute__((always_inline)) {
        const uint32_t at = Loads::v(lane) + tile * (TILE * ROWB);
#pragma unroll
        for (int i = 0; i < VPL; i++)
            r.v[i] = __builtin_amdgcn_raw_buffer_load_b128(from.v, at + Loads::v_further(i), 0, 0);
        if constexpr (MX) {
            const uint32_t sat = Loads::v_scale(lane) + tile * (TILE * SCB);
#pragma unroll
            for (int i = 0; i < VPL; i++)
                r.vs[i] = __builtin_amdgcn_raw_buffer_load_b8(from.vs, sat + Loads::v_scale_further(i), 0, 0);
        }
    };

    // What a wave waits for one after the other is most of a short call: the arguments, the prefix length, the tree, the queries, the first tile.  So all are requested as soon as their
    // addresses are known, and the tree, which needs the parents only, is built meanwhile.
    const bool walk = T <= 64 && (!a.tree_mask || windowed);
    // (requested together, not where each is used: every trip to memory that is waited for here is 600 clocks)
    asm volatile("" ::"s"(prefix), "s"(a.q), "s"(a.tree_magic), "s"(a.group), "s"(a.n_q_heads), "s"(a.scale_log2));
    int parent = 0;
    if (walk)
        parent = a.parent[(int64_t)b * T + min(lane, T - 1)];
    Raw<D, MX> raw;
    const bool early = n_splits == 1 && !windowed;               // the first tile is known without the prefix length
    if (early) {
        const Range all = range_of(s_max);
        const uint32_t tile = early_tile(wave, s_max);
        request_k(raw, all, tile);
        request_v(raw, all, tile);
    }
    int P, t0, t1;
    Tiles tiles;
    Range live;
    uint32_t no_tile;                                            // behind the live rows
    auto tile_of = [&](int t) __attribute__((always_inline)) { return t < t1 ? (uint32_t)tiles.at(t) : no_tile; };
    auto find_tiles = [&]() __attribute__((always_inline)) {
        P = prefix_rows(prefix, s_max, T);
        tiles = tiles_of(a, P);
        const int per = tiles_per_split(tiles.count, lg_splits);
        t0 = split * per + wave;
        t1 = split_end(tiles.count, split, per);
        live = range_of(P + T);
        no_tile = tile_behind(P + T);
    };
    if (!early) {
        find_tiles();
        const uint32_t tile = tile_of(t0);
        request_k(raw, live, tile);
        request_v(raw, live, tile);
    }

    // the queries of this workgroup's rows: row f of a KV head is node f % T of its head f / T
    const uint32_t rows = T * a.group;
    if (rg * QT * 16 >= rows)
        return;
    bf16x8 qf[QT][NKS];
    int node[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        uint32_t f = (rg * QT + qt) * 16 + c;
        f = f < rows ? f : 0;
        const uint32_t head = quick_div(f, a.tree_magic);
        node[qt] = f - head * T;
        const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (((int64_t)b * T + node[qt]) * a.n_q_heads + kvh * a.group + head) * D;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
            qf[qt][ks] = *reinterpret_cast<const bf16x8 *>(qp + channel_of<D, MX>(ks, g));
    }
    SmallTree small = {0, 0, 0};
    if (T <= 64)
        small = small_tree(a, windowed, b, T, walk && lane < T && parent < lane ? parent : -1, lane);      // (a path up the tree always ends)
    if (early)
        find_tiles();
    Tree tree = {s_mask, s_depth, small.deepest};
    if (T > 64)
        build_tree(tree, a, b, P, s_parent, &s_deepest, tid, 64 * NW);
    else if (windowed && a.window < T)
        cut_small_masks(small, a, P, reinterpret_cast<int32_t *>(s_area[wave]), lane);
    uint64_t mask[QT];
    int depth[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        mask[qt] = (uint64_t)(uint32_t)__shfl((int)(small.mask >> 32), node[qt]) << 32 | (uint32_t)__shfl((int)small.mask, node[qt]);
        depth[qt] = windowed ? __shfl(small.depth, node[qt]) : 0;
    }
    const int lo_min = windowed ? P - a.window + 1 : 0, lo_max = windowed ? lo_min + tree.deepest : 0;      // windows' starts, root and deepest node
    // tiles [w0, w1) of the list are seen whole by every row (a negative scale goes the general way)
    const int w0 = max(tiles.sinks, tiles.sinks + (lo_max + 31) / 32 - tiles.first), w1 = a.scale_log2 >= 0.0f ? tiles.sinks + P / 32 - tiles.first : 0;

    RowState<QT, NDT> st;
    st.clear();
    uint16_t *area = reinterpret_cast<uint16_t *>(s_area[wave]);
    // (the queries are waited for here: in the loop it would be for every load since)
#pragma unroll
    for (int qt = 0; qt < QT; qt++)
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
            asm volatile("" : "+v"(qf[qt][ks]));
    auto visible = [&](int qt, int j0) __attribute__((always_inline)) {
        return T <= 64 ? visible_prefix(a, depth[qt], lo_min, P, j0) | visible_nodes(mask[qt], P, j0) : visible_keys(tree, a, node[qt], lo_min, P, j0);
    };
    bool poisoned = false;
    // One tile, the t-th of the list; `raw` then receives the wave's next.
    auto step = [&](auto seen, int t) __attribute__((always_inline)) {
        constexpr bool whole = decltype(seen)::value;
        const uint32_t next = tile_of(t + NW);
        // ---- S^T = K Q^T
        f32x4 s[2][QT];
#pragma unroll
        for (int hh = 0; hh < 2; hh++)
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                s[hh][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) {
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
                bf16x8 kf;
                if constexpr (MX)
                    kf = from_codes(raw.k[hh][ks], scale_value(raw.ks[hh][D == 256 ? ks >> 2 : 0]));
                else
                    kf = __builtin_bit_cast(bf16x8, raw.k[hh][ks]);
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    s[hh][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[qt][ks], s[hh][qt], 0, 0, 0);
            }
        }
        request_k(raw, live, next);

        // ---- V to LDS, as bf16.  Where not every row sees every key, zeros stand for what is not finite (0 * NaN is no zero); what that does to the rows that see it comes behind the loop
        if constexpr (MX) {
            const uint32_t last = whole ? 255u : 252u;
#pragma unroll
            for (int i = 0; i < VPL; i++) {
                uint16_t *to = area + (vrow + Loads::v_row(0, i)) * VSTR + vcol * Loads::V_VALUES;
                const uint32_t byte = raw.vs[i];
                poisoned = poisoned || byte > last;
                const float scale = scale_value(byte > last ? 0u : byte);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    *reinterpret_cast<bf16x8 *>(to + e * 8) = from_codes(raw.v[i][e], scale);
            }
        } else {
            if (!whole) {
                uint32_t found = 0;
#pragma unroll
                for (int i = 0; i < VPL; i++) {
                    found |= (strange_halves(raw.v[i][0]) | strange_halves(raw.v[i][1])) | (strange_halves(raw.v[i][2]) | strange_halves(raw.v[i][3]));
                    raw.v[i] = without_strange(raw.v[i]);
                }
                poisoned = poisoned || found != 0u;
            }
#pragma unroll
            for (int i = 0; i < VPL; i++)
                *reinterpret_cast<u32x4 *>(area + (vrow + Loads::v_row(0, i)) * VSTR + vcol * Loads::V_VALUES) = raw.v[i];
        }
        request_v(raw, live, next);

        uint32_t vis[QT] = {};
        if (!whole) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                vis[qt] = visible(qt, tiles.at(t) * 32) >> (g * 4);
        }
        bf16x8 pf[QT];
        softmax_tile<whole>(s, st, vis, a.scale_log2, pf);
        wave_lds_fence();
        add_values<QT, NDT, VSTR>(area, pf, st, c, g);
        wave_lds_fence();
    };
    // Tiles that every row sees whole in straight code of their own: one step is some 200 instructions that a wave issues one by one, and flags and branches were a quarter of them.
    const int w2 = min(w1, t1);
    for (int t = t0; t < t1; t += NW) {
        for (; t >= w0 && t < w2; t += NW)
            step(std::true_type(), t);
        if (t < t1)
            step(std::false_type(), t);
    }

    if (__any(poisoned)) {
        // Tiles that some row does not see all of, again: ones in the places of values that are not finite, and ones for the keys a row sees, count them, and what counts
        // any is NaN.
#pragma unroll 1
        for (int t = t0; t < t1; t += NW) {
            if (t >= w0 && t < w1)
                continue;
            const int j0 = tiles.at(t) * 32;
#pragma unroll 1
            for (int p = lane; p < 32 * D / 8; p += 64) {
                const int row = p / (D / 8), piece = p % (D / 8), j = j0 + row;
                const bool none = j >= P + T || (j < lo_min && j >= a.n_sink);
                const int64_t at = none ? j0 : j;
                u32x4 x;
                if constexpr (MX)
                    x = __builtin_bit_cast(u32x4, from_codes(*reinterpret_cast<const uint32_t *>(v + at * ROWB + piece * 4), scale_value(v_scales[at * SCB + piece / 4])));
                else
                    x = *reinterpret_cast<const u32x4 *>(v + at * ROWB + piece * 16);
                *reinterpret_cast<u32x4 *>(area + row * VSTR + piece * 8) = none ? u32x4{0u, 0u, 0u, 0u} : strange_places(x);
            }
            wave_lds_fence();
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                mark_strange<QT, NDT, VSTR>(area, qt, visible(qt, j0) >> (g * 4), st, c, g);
            wave_lds_fence();
        }
    }

    // ---- the waves' states meet in LDS, in wave order
    f32x4 *mine = reinterpret_cast<f32x4 *>(s_area[wave]);
    wave_lds_fence();
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        float l = st.l[qt];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            s_ml[wave][qt][0][c] = st.m[qt];
            s_ml[wave][qt][1][c] = l;
        }
#pragma unroll
        for (int dt = 0; dt < NDT; dt++)
            mine[(qt * NDT + dt) * 64 + lane] = st.o[qt][dt];
    }
    __syncthreads();
    // a thread takes 8 channels of a row at a time, 16 rows side by side
#pragma unroll
    for (int i = 0; i < (QT * 2 * D + 64 * NW - 1) / (64 * NW); i++) {
        const int item = i * 64 * NW + tid;
        if (QT * 2 * D % (64 * NW) && item >= QT * 2 * D)
            break;
        const int qt = item / (2 * D), ch = item / 16 % (D / 8);
        const uint32_t f = (rg * QT + qt) * 16 + c;
        float mt = -INFINITY, lt = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; w++)
            mt = fmaxf(mt, s_ml[w][qt][0][c]);
        const float ref = mt == -INFINITY ? 0.0f : mt;
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
        const int from = qt * NDT * 64 + (ch >> 1) * 64 + (ch & 1) * 32 + c;
#pragma unroll
        for (int w = 0; w < NW; w++) {
            const float wgt = __builtin_amdgcn_exp2f(s_ml[w][qt][0][c] - ref);
            const f32x4 *src = reinterpret_cast<const f32x4 *>(s_area[w]);
            lt += s_ml[w][qt][1][c] * wgt;
            x += src[from] * wgt;
            y += src[from + 16] * wgt;
        }
        if (f >= rows)
            continue;
        if (n_splits > 1) {
            const int64_t slot = (((int64_t)unit * a.n_rg + rg) * QT + qt) * 16 + c;
            f32x4 *dst = reinterpret_cast<f32x4 *>(a.part + slot * D + ch * 8);
            dst[0] = x;
            dst[1] = y;
            if (ch == 0) {
                a.part_ml[slot * 2] = mt;
                a.part_ml[slot * 2 + 1] = lt;
            }
        } else {
            const float inv = lt != 0.0f ? 1.0f / lt : 0.0f;
            bf16x8 r;
#pragma unroll
            for (int e = 0; e < 4; e++) {
                r[e] = (__bf16)(x[e] * inv);
                r[4 + e] = (__bf16)(y[e] * inv);
            }
            const uint32_t head = quick_div(f, a.tree_magic), n = f - head * T, hq = kvh * a.group + head;
            *reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(a.out) + (((int64_t)b * T + n) * a.n_q_heads + hq) * D + ch * 8) = r;
            if (a.lse && ch == 0)
                a.lse[((int64_t)b * a.n_q_heads + hq) * T + n] = lt != 0.0f ? (mt + log2f(lt)) * 0.6931471805599453f : -INFINITY;
        }
    }
}

// All rows of a KV head in one workgroup, or as many as its eight waves hold.  What a CU can pull, 64 KB in flight, bounds a kernel whose workgroups for 16 rows each read the same keys, and so
// does what it takes to turn 4 bits into 16: here a tile of 32 keys is read once, lies in LDS as bf16 and serves every wave's QT query tiles.  Two stages: while the waves work on one, the next
// tile goes from registers to the other, and the two after that are on their way (one: 24.2 us, two: 22.6 to 22.9, at B 4, 16 heads on 8 of 256, 33 nodes, 1024 keys); one barrier a tile.  The keys are shared out over workgroups (splits), whose states window_merge_kernel joins.
template <int D, int QT, bool MX>
struct SharedGeom {
    static constexpr int NW = 8, THREADS = GroupLoads<D, MX>::THREADS;
    static constexpr int KSTR = D + 8, VSTR = D + 16;            // row strides in LDS (values): 16-byte reads of K rows and transposing ones of V meet in no bank
    static constexpr int STAGE = 32 * (KSTR + VSTR);             // values
};

template <int D, int QT, bool MX>
__global__ __launch_bounds__(512, 2) void window_shared_kernel(const uint8_t *k, const uint8_t *v, const uint8_t *k_scales, const uint8_t *v_scales, const int32_t *prefix_len,
                                                               uint32_t s_max, uint32_t heads_splits, uint32_t heads_magic, uint32_t tree_units, WindowArgs a)
{
    using G = SharedGeom<D, QT, MX>;
    using Loads = GroupLoads<D, MX>;
    constexpr int NKS = D / 32, NDT = D / 16, KSTR = G::KSTR, VSTR = G::VSTR;
    constexpr int ROWB = Loads::ROW, SCB = Loads::SCALES, N = Loads::PIECES;
    constexpr bool HALVES = Loads::HALVES;
    __shared__ __attribute__((aligned(16))) uint16_t s_stage[2][G::STAGE];
    __shared__ uint64_t s_mask[DREAM_MAX_TREE * 4];
    __shared__ int32_t s_depth[DREAM_MAX_TREE], s_parent[DREAM_MAX_TREE], s_deepest, s_strange[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const Place place = place_of(heads_splits);
    const uint32_t unit = place.unit, rg = place.rg, n_heads = heads_splits & 0xffff, lg_splits = heads_splits >> 16 & 0xff, n_splits = 1u << lg_splits;
    if (unit >= tree_units >> 10)
        return;
    const uint32_t stream = unit >> lg_splits, split = unit & (n_splits - 1);
    const uint32_t b = quick_div(stream, heads_magic), kvh = stream - b * n_heads;
    const int T = tree_units & 0x1ff;
    const bool windowed = tree_units & 0x200;
    const int64_t head_row = (int64_t)stream * s_max;
    k += head_row * ROWB;
    v += head_row * ROWB;
    k_scales += head_row * SCB;
    v_scales += head_row * SCB;
    if (tid < 2)
        s_strange[tid] = -1;

    const int prefix = scalar_load(prefix_len + b);
    const bool walk = T <= 64 && (!a.tree_mask || windowed);
    asm volatile("" ::"s"(prefix), "s"(a.q), "s"(a.tree_magic), "s"(a.group), "s"(a.n_q_heads), "s"(a.scale_log2));      // (requested together: see window_attn_kernel)
    int parent = 0;
    if (walk)
        parent = a.parent[(int64_t)b * T + min(lane, T - 1)];
    const int P = prefix_rows(prefix, s_max, T);
    const Tiles tiles = tiles_of(a, P);
    const int per = tiles_per_split(tiles.count, lg_splits);
    const int t0 = split * per, t1 = split_end(tiles.count, split, per);

    // a thread's pieces of a tile; loads of rows that are not there return zeros (see window_attn_kernel)
    const bool second = Loads::takes_v(tid);
    const int ptid = Loads::thread(tid);
    constexpr int BYTES = Loads::WIDTH;
    struct Part {
        u32x4 x[N];
        uint8_t scale[N];
    };
    struct Pieces {
        Part part[HALVES ? 1 : 2];
    } even, odd;                                                 // of the tiles at even and at odd distances from t0
    // (a wave's threads all take K or all take V)
    const bool wave_second = HALVES && wave >= G::NW / 2;
    const auto first_rows = buffer_of(wave_second ? v : k, (P + T) * ROWB), second_rows = buffer_of(v, (P + T) * ROWB);
    const auto first_scales = buffer_of(wave_second ? v_scales : k_scales, (P + T) * SCB), second_scales = buffer_of(v_scales, (P + T) * SCB);
    const uint32_t no_tile = tile_behind(P + T);
    auto request = [&](Pieces &of, int t) __attribute__((always_inline)) {
        const uint32_t tile = t < t1 ? (uint32_t)tiles.at(t) : no_tile;
        const uint32_t at = Loads::at(ptid) + tile * (TILE * ROWB), scale_at = Loads::scale(ptid) + tile * (TILE * SCB);
#pragma unroll
        for (int half = 0; half < (HALVES ? 1 : 2); half++) {
#pragma unroll
            for (int i = 0; i < N; i++) {
                const auto rows_at = half ? second_rows : first_rows;
                if constexpr (BYTES == 16) {
                    of.part[half].x[i] = __builtin_amdgcn_raw_buffer_load_b128(rows_at, at + Loads::further(i), 0, 0);
                } else if constexpr (BYTES == 8) {
                    const auto y = __builtin_amdgcn_raw_buffer_load_b64(rows_at, at + Loads::further(i), 0, 0);
                    of.part[half].x[i][0] = y[0];
                    of.part[half].x[i][1] = y[1];
                } else {
                    of.part[half].x[i][0] = __builtin_amdgcn_raw_buffer_load_b32(rows_at, at + Loads::further(i), 0, 0);
                }
                if constexpr (MX)
                    of.part[half].scale[i] = __builtin_amdgcn_raw_buffer_load_b8(half ? second_scales : first_scales, scale_at + Loads::scale_further(i), 0, 0);
            }
        }
    };
    // tiles [w0, w1) are seen whole by every row; lo_min: where the root's window starts
    int w0 = 0, w1 = 0, lo_min = 0;
    auto deliver = [&](const Pieces &of, int t) __attribute__((always_inline)) {
        uint16_t *stage = s_stage[(t - t0) & 1];
        const bool whole = t >= w0 && t < w1;
        bool strange = false;
#pragma unroll
        for (int half = 0; half < (HALVES ? 1 : 2); half++) {
            const bool of_v = HALVES ? second : half == 1;
            uint16_t *tile = stage + (of_v ? 32 * KSTR : 0);
#pragma unroll
            for (int i = 0; i < N; i++) {
                uint16_t *to = tile + Loads::row(ptid, i) * (of_v ? VSTR : KSTR) + Loads::channel(ptid, i);
#pragma unroll
                for (int e = 0; e < Loads::PIECE / 8; e++) {
                    u32x4 x;
                    if constexpr (MX)
                        x = __builtin_bit_cast(u32x4, from_codes(of.part[half].x[i][e], scale_value(of.part[half].scale[i])));
                    else
                        x = of.part[half].x[i];
                    if (of_v && !whole) {        // (0 * NaN is no zero: see window_attn_kernel)
                        strange = strange || ((strange_halves(x[0]) | strange_halves(x[1])) | (strange_halves(x[2]) | strange_halves(x[3]))) != 0u;
                        x = without_strange(x);
                    }
                    *reinterpret_cast<u32x4 *>(to + e * 8) = x;
                }
            }
        }
        if (!whole && __any(strange) && lane == 0)
            s_strange[(t - t0) & 1] = t;
    };

    request(even, t0);
    request(odd, t0 + 1);
    const uint32_t rows = T * a.group;
    if (rg * G::NW * QT * 16 >= rows)
        return;
    bf16x8 qf[QT][NKS];
    int node[QT];
    const bool idle = ((rg * G::NW + wave) * QT) * 16 >= rows;   // (a wave without rows only brings keys)
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        uint32_t f = ((rg * G::NW + wave) * QT + qt) * 16 + c;
        f = f < rows ? f : 0;
        const uint32_t head = quick_div(f, a.tree_magic);
        node[qt] = f - head * T;
        const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (((int64_t)b * T + node[qt]) * a.n_q_heads + kvh * a.group + head) * D;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
            qf[qt][ks] = *reinterpret_cast<const bf16x8 *>(qp + ks * 32 + g * 8);
    }
    SmallTree small = {0, 0, 0};
    Tree tree = {s_mask, s_depth, 0};
    if (T <= 64) {
        small = small_tree(a, windowed, b, T, walk && lane < T && parent < lane ? parent : -1, lane);      // (a path up the tree always ends)
        tree.deepest = small.deepest;
        if (windowed && a.window < T)
            cut_small_masks(small, a, P, reinterpret_cast<int32_t *>(s_stage[1]) + wave * 64, lane);
        __syncthreads();                                         // (s_strange, and s_stage[1] again)
    } else {
        build_tree(tree, a, b, P, s_parent, &s_deepest, tid, G::THREADS);
    }
    uint64_t mask[QT];
    int depth[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        mask[qt] = (uint64_t)(uint32_t)__shfl((int)(small.mask >> 32), node[qt]) << 32 | (uint32_t)__shfl((int)small.mask, node[qt]);
        depth[qt] = windowed ? __shfl(small.depth, node[qt]) : 0;
    }
    if (windowed)
        lo_min = P - a.window + 1;
    w0 = max(tiles.sinks, tiles.sinks + ((windowed ? lo_min + tree.deepest : 0) + 31) / 32 - tiles.first);
    w1 = a.scale_log2 >= 0.0f ? tiles.sinks + P / 32 - tiles.first : 0;
    RowState<QT, NDT> st;
    st.clear();
    if (t0 < t1)
        deliver(even, t0);
    request(even, t0 + 2);
#pragma unroll
    for (int qt = 0; qt < QT; qt++)
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
            asm volatile("" : "+v"(qf[qt][ks]));
    __syncthreads();
    auto visible = [&](int qt, int j0) __attribute__((always_inline)) {
        return T <= 64 ? visible_prefix(a, depth[qt], lo_min, P, j0) | visible_nodes(mask[qt], P, j0) : visible_keys(tree, a, node[qt], lo_min, P, j0);
    };
    bool poisoned = false;
    auto step = [&](Pieces &next, int t) __attribute__((always_inline)) {
        const uint16_t *stage = s_stage[(t - t0) & 1];
        if (t + 1 < t1)
            deliver(next, t + 1);
        request(next, t + 3);
        const bool whole = t >= w0 && t < w1;
        const int j0 = tiles.at(t) * 32;
        poisoned = poisoned || (!whole && s_strange[(t - t0) & 1] == t);
        if (!idle) {
            f32x4 s[2][QT];
#pragma unroll
            for (int hh = 0; hh < 2; hh++)
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    s[hh][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < NKS; ks++)
#pragma unroll
                for (int hh = 0; hh < 2; hh++) {
                    const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(stage + (16 * hh + c) * KSTR + ks * 32 + g * 8);
#pragma unroll
                    for (int qt = 0; qt < QT; qt++)
                        s[hh][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[qt][ks], s[hh][qt], 0, 0, 0);
                }
            uint32_t vis[QT] = {};
            if (!whole) {
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    vis[qt] = visible(qt, j0) >> (g * 4);
            }
            bf16x8 pf[QT];
            if (whole)
                softmax_tile<true>(s, st, vis, a.scale_log2, pf);
            else
                softmax_tile<false>(s, st, vis, a.scale_log2, pf);
            add_values<QT, NDT, VSTR>(stage + 32 * KSTR, pf, st, c, g);
        }
        __syncthreads();
    };
    // (no way out between two steps: the loads in flight at the loop's head have to be the same on every way there)
    int t = t0;
    for (; t + 1 < t1; t += 2) {
        step(odd, t);
        step(even, t + 1);
    }
    if (t < t1)
        step(odd, t);
    if (poisoned) {      // (the same for all waves) see window_attn_kernel
        uint16_t *tile = s_stage[0];
#pragma unroll 1
        for (int t = t0; t < t1; t++) {
            if (t >= w0 && t < w1)
                continue;
            const int j0 = tiles.at(t) * 32;
#pragma unroll 1
            for (int p = tid; p < 32 * D / 8; p += G::THREADS) {
                const int row = p / (D / 8), piece = p % (D / 8), j = j0 + row;
                const bool none = j >= P + T || (j < lo_min && j >= a.n_sink);
                const int64_t at = none ? j0 : j;
                u32x4 x;
                if constexpr (MX)
                    x = __builtin_bit_cast(u32x4, from_codes(*reinterpret_cast<const uint32_t *>(v + at * ROWB + piece * 4), scale_value(v_scales[at * SCB + piece / 4])));
                else
                    x = *reinterpret_cast<const u32x4 *>(v + at * ROWB + piece * 16);
                *reinterpret_cast<u32x4 *>(tile + row * VSTR + piece * 8) = none ? u32x4{0u, 0u, 0u, 0u} : strange_places(x);
            }
            __syncthreads();
            if (!idle) {
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    mark_strange<QT, NDT, VSTR>(tile, qt, visible(qt, j0) >> (g * 4), st, c, g);
            }
            __syncthreads();
        }
    }
    if (idle)
        return;
    // ---- a lane has 4 adjacent channels of a row in every 16
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        float l = st.l[qt];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const uint32_t f = ((rg * G::NW + wave) * QT + qt) * 16 + c;
        if (f >= rows)
            continue;
        if (n_splits > 1) {
            const int64_t slot = ((((int64_t)unit * a.n_rg + rg) * G::NW + wave) * QT + qt) * 16 + c;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)
                *reinterpret_cast<f32x4 *>(a.part + slot * D + dt * 16 + g * 4) = st.o[qt][dt];
            if (g == 0) {
                a.part_ml[slot * 2] = st.m[qt];
                a.part_ml[slot * 2 + 1] = l;
            }
        } else {
            const float inv = l != 0.0f ? 1.0f / l : 0.0f;
            const uint32_t head = quick_div(f, a.tree_magic), n = f - head * T, hq = kvh * a.group + head;
            uint16_t *to = static_cast<uint16_t *>(a.out) + (((int64_t)b * T + n) * a.n_q_heads + hq) * D + g * 4;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++) {
                bf16x4 r;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    r[e] = (__bf16)(st.o[qt][dt][e] * inv);
                *reinterpret_cast<bf16x4 *>(to + dt * 16) = r;
            }
            if (a.lse && g == 0)
                a.lse[((int64_t)b * a.n_q_heads + hq) * T + n] = l != 0.0f ? (st.m[qt] + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
    }
}

// The states of a row's key splits, in their order.  D / 4 lanes a row.  What other XCDs wrote comes from memory: 2.2 to 5 us with the launch.  (A row's splits over several waves that meet in
// LDS took longer: 5.6 instead of 4.7 us for 1056 rows of 256 with 8 splits, 2.6 instead of 2.2 for 32 rows of 128.)
template <int D>
__global__ __launch_bounds__(256) void window_merge_kernel(WindowArgs a, int rows_per_unit)
{
    constexpr int LPR = D / 4;
    const int rows = a.n_tree * a.group, n = a.n_splits;
    const uint32_t stream = blockIdx.z * UNITS_Y + blockIdx.y, f = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int lane = threadIdx.x % LPR;
    if (stream * n >= (uint32_t)a.n_units || f >= (uint32_t)rows)
        return;
    const int64_t slot = (int64_t)stream * n * rows_per_unit + f;
    // eight splits' loads at a time (behind the last: the first again, weighted with nothing)
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += 8) {
        float mm[8], ll[8];
        f32x4 oo[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const int64_t i = slot + (int64_t)(s0 + j < n ? s0 + j : 0) * rows_per_unit;
            mm[j] = a.part_ml[i * 2];
            ll[j] = a.part_ml[i * 2 + 1];
            oo[j] = *reinterpret_cast<const f32x4 *>(a.part + i * D + lane * 4);
        }
        float top = m;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            mm[j] = s0 + j < n ? mm[j] : -INFINITY;
            top = fmaxf(top, mm[j]);
        }
        const float ref = top == -INFINITY ? 0.0f : top, old = __builtin_amdgcn_exp2f(m - ref);
        l *= old;
        o *= old;
        m = top;
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (s0 + j < n) {
                const float w = __builtin_amdgcn_exp2f(mm[j] - ref);
                l += w * ll[j];
                o += oo[j] * w;
            }
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    const uint32_t b = quick_div(stream, a.heads_magic), head = quick_div(f, a.tree_magic), node = f - head * a.n_tree, hq = (stream - b * a.n_kv_heads) * a.group + head;
    bf16x4 r;
#pragma unroll
    for (int e = 0; e < 4; e++)
        r[e] = (__bf16)(o[e] * inv);
    *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.out) + (((int64_t)b * a.n_tree + node) * a.n_q_heads + hq) * D + lane * 4) = r;
    if (a.lse && lane == 0)
        a.lse[((int64_t)b * a.n_q_heads + hq) * a.n_tree + node] = l != 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// float32 queries and rows (the small configuration): one workgroup of 4 waves per (node, head, sequence), D / 4 lanes a key, each with 4 channels; every wave keeps a state
// of its own keys and they meet in LDS.  Only keys that the node's window reaches are read, but every node reads its own: there for its precision and for small shapes, not for long ones.
// 4 heads on 2 of 64, 21 nodes, 121 keys: 5.3 us (4-bit 5.4; the launch and one round of loads).  32 heads of 128, 60 nodes, 764 keys: 80 us (4-bit 82), where the 25 MB read once would take 5;
// one token with a window of 1024: 44 us, 32 workgroups.
template <int D, bool MX>
__global__ __launch_bounds__(256) void window_f32_kernel(WindowArgs a)
{
    constexpr int LPK = D / 4, KPW = 64 / LPK, U = 4, PASS = 4 * KPW * U;
    __shared__ uint64_t s_mask[DREAM_MAX_TREE * 4];
    __shared__ int32_t s_depth[DREAM_MAX_TREE], s_parent[DREAM_MAX_TREE], s_deepest;
    __shared__ __attribute__((aligned(16))) float s_o[4][D];
    __shared__ float s_m[4], s_l[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane % LPK;
    const int node = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, T = a.n_tree;
    const int P = (int)min((int64_t)max(a.prefix_len[b], 0), a.s_max - T);
    const int64_t head_row = ((int64_t)b * a.n_kv_heads + hq / a.group) * a.s_max;
    const f32x4 q = reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.q) + (((int64_t)b * T + node) * a.n_q_heads + hq) * D)[col];
    Tree tree = {s_mask, s_depth, 0};
    build_tree(tree, a, b, P, s_parent, &s_deepest, tid, 256);
    const int lo = a.window ? max(0, P - a.window + 1 + tree.depth[node]) : 0, start = min(lo, P);
    const int sinks = a.window ? min(a.n_sink, start) : 0, count = sinks + P + T - start;
    auto value = [&](const void *x, const uint8_t *scales, int64_t row) {
        if constexpr (MX) {
            const uint32_t codes = *reinterpret_cast<const uint16_t *>(static_cast<const uint8_t *>(x) + row * (D / 2) + col * 2);
            const float scale = scale_value(scales[row * (D / GROUP) + col / 8]);
            const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
            return f32x4{p[0], p[1], r[0], r[1]};
        } else {
            return reinterpret_cast<const f32x4 *>(static_cast<const float *>(x) + row * D)[col];
        }
    };
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < count; i0 += PASS) {
        f32x4 kr[U], vr[U];
        bool see[U];
        float sc[U], top = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int i = i0 + (u * 4 + wave) * KPW + lane / LPK;
            const int ii = min(i, count - 1), j = ii < sinks ? ii : ii - sinks + start, rel = j - P;
            see[u] = i < count && (rel < 0 || (tree.mask[node * a.mask_words + (rel >> 6)] >> (rel & 63) & 1ull));
            kr[u] = value(a.k, a.k_scales, head_row + j);
            vr[u] = value(a.v, a.v_scales, head_row + j);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            float dot = (q[0] * kr[u][0] + q[1] * kr[u][1]) + (q[2] * kr[u][2] + q[3] * kr[u][3]);
#pragma unroll
            for (int d = 1; d < LPK; d *= 2)
                dot += __shfl_xor(dot, d);
            sc[u] = see[u] ? dot * a.scale : -INFINITY;
            top = fmaxf(top, sc[u]);
        }
#pragma unroll
        for (int d = LPK; d < 64; d *= 2)
            top = fmaxf(top, __shfl_xor(top, d));
        const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.0f : mn, f = expf(m - ref);
        l *= f;
        o *= f;
        m = mn;
#pragma unroll
        for (int u = 0; u < U; u++) {
            const float p = expf(sc[u] - ref);
            l += p;
            if (see[u])                           // (what a row does not see is not touched: 0 * NaN is no zero)
                o += vr[u] * p;
        }
    }
#pragma unroll
    for (int d = LPK; d < 64; d *= 2) {
        l += __shfl_xor(l, d);
#pragma unroll
        for (int e = 0; e < 4; e++)
            o[e] += __shfl_xor(o[e], d);
    }
    if (lane < LPK)
        reinterpret_cast<f32x4 *>(s_o[wave])[col] = o;
    if (lane == 0) {
        s_m[wave] = m;
        s_l[wave] = l;
    }
    __syncthreads();
    if (tid < D) {
        const float mt = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), ref = mt == -INFINITY ? 0.0f : mt;
        float lt = 0.0f, r = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float f = expf(s_m[w] - ref);
            lt += s_l[w] * f;
            r += s_o[w][tid] * f;
        }
        static_cast<float *>(a.out)[(((int64_t)b * T + node) * a.n_q_heads + hq) * D + tid] = lt != 0.0f ? r / lt : 0.0f;
        if (a.lse && tid == 0)
            a.lse[((int64_t)b * a.n_q_heads + hq) * T + node] = lt != 0.0f ? mt + logf(lt) : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
struct WindowPlan {
    bool shared;                   // window_shared_kernel
    int qt, nw, n_rg, n_splits;
    int64_t n_units, slots;        // (stream, split) pairs; rows of parts of O
    size_t off_ml;
};

// Which kernel a call takes, and into how many parts its keys are split, is what is estimated to take the shortest.  Where one workgroup is on a CU a wave's steps cost what one takes to come
// through; where many are, what the CU can issue; whichever is more:
//     us = base + per_group * groups + steps * max(latency, issue * groups)  [+ many_nodes]  [+ 2.3 + 0.11 * splits + 1e-6 * head_dim * rows of parts, for the join]
// with groups the workgroups (of four waves) a CU gets, steps those of a wave.  The constants are those with which the choice is best over measured times of every kernel with every split from
// 1 to 64 in powers of two, over 7 head layouts x batches of 1, 4, 16, 64 x trees of 1, 16, 60, 250 x 40 to 40000 keys, 528 shapes of 4-bit and 515 of 16-bit caches: 0.8 % and 0.6 % behind
// the fastest in the geometric mean, 5 % and 3 % at the 95th percentile, 34 % at most.  These are the data that it was fitted to, without a window; over 144 shapes each with windows of 500 to 4096
// keys, measured afterwards, 1.7 % and 1.3 %, 9 % and 7 %, 17 % at most.  What the forms are worth without one (4-bit, 16-bit): the fastest would take 4 % and 30 % longer without the shared kernel, 5 % and 1.5 % without several query tiles to a wave, 33 % and 57 % without splits, and
// 1 % without the eight-wave form over 4-bit caches; over 16-bit ones that brought 0.2 % and is left out, as is the shared kernel over 4-bit caches at head_dim 64 (0.1 %).
struct Steps {
    float base, per_group, latency, latency_tile, issue, issue_tile, many_nodes;      // window_attn_kernel; .._tile: for each query tile of a wave
    float s_base, s_per_group, s_latency, s_issue, s_many_nodes;                      // window_shared_kernel
};

constexpr Steps STEPS[2][3] = {{{3.9f, 0.66f, 0.48f, 0.11f, 0.65f, 0.00f, 3.1f, 1.1f, 4.3f, 0.72f, 0.82f, 4.8f},
                                {2.6f, 0.63f, 0.35f, 0.33f, 1.3f, 0.42f, 0.0f, 1.3f, 3.7f, 0.62f, 0.71f, 7.1f},
                                {0.54f, 5.1f, 0.35f, 0.20f, 2.3f, 0.59f, 2.9f, 0.03f, 8.7f, 1.4f, 1.4f, 2.2f}},
                               {{2.7f, 0.56f, 0.37f, 0.11f, 0.093f, 0.099f, 2.1f, 0.f, 0.f, 0.f, 0.f, 0.f},
                                {3.3f, 2.1f, 0.24f, 0.25f, 0.15f, 0.22f, 1.6f, 2.4f, 3.0f, 0.012f, 1.0f, 4.2f},
                                {5.1f, 0.87f, 1.1f, 0.097f, 0.85f, 0.14f, 2.4f, 3.0f, 4.2f, 0.51f, 1.1f, 3.5f}}};

// query tiles a wave of window_attn_kernel may have, and those of window_shared_kernel's (0: there is none)
constexpr int most_tiles(int D, bool mx) { return D == 64 ? (mx ? 4 : 2) : D == 128 && mx ? 2 : 1; }
constexpr int shared_tiles(int D, bool mx) { return D == 64 ? (mx ? 0 : 2) : 1; }

struct Choice {
    bool shared;
    int qt, nw;
};

// All a call may take, the overrides obeyed.  each(choice, groups of rows, most splits)
template <class F>
void every_choice(const dream_attn_desc *d, bool mx, int tiles, int64_t steps, F each)
{
    const int most = most_tiles(d->head_dim, mx), in_shared = shared_tiles(d->head_dim, mx);
    const int waves = tile_waves_override(), asked = q_tiles_override(), forced = asked <= 0 ? 0 : asked < 2 || most < 2 ? 1 : asked < 4 || most < 4 ? 2 : 4;
    const int64_t streams = (int64_t)d->batch * d->n_kv_heads;
    auto offer = [&](const Choice &c) {
        const int64_t groups = ceil_div(tiles, c.qt * (c.shared ? c.nw : 1));
        int64_t splits = (c.shared ? 512 : 2048) / (streams * groups);       // parts beyond these only cost the join
        splits = splits > steps ? steps : splits;
        each(c, (int)groups, (int)(splits < 1 ? 1 : splits > MAX_SPLITS ? MAX_SPLITS : splits));
    };
    const bool eight = waves == 8, four = waves == 4;
    for (int qt = 1; qt <= most; qt *= 2) {
        if (forced ? qt != forced : qt > 1 && qt / 2 >= tiles)
            continue;
        const bool has_eight = mx && qt == 1;
        if (!eight || (forced && !has_eight))
            offer({false, qt, 4});
        if (has_eight && !four && !(eight && !forced && in_shared))
            offer({false, qt, 8});
    }
    if (in_shared && !four && !forced && (eight || tiles > 2))       // (fewer tiles leave most of its waves idle: never measured, never taken)
        offer({true, in_shared, 8});
}

void shape_of(const dream_attn_desc *d, int n_tree, int64_t max_kv_len, int window, int n_sink, int *tiles, int64_t *steps)
{
    int64_t keys = max_kv_len;
    if (window && (int64_t)window + n_tree + n_sink + 64 < keys)
        keys = (int64_t)window + n_tree + n_sink + 64;
    *tiles = ceil_div((int64_t)d->n_q_heads / d->n_kv_heads * n_tree, 16);
    *steps = ceil_div(keys, 32);
}

// a power of two, like what the choice takes (a shift divides by it), and units below 2^22 (the launch's arguments)
int forced_splits(int64_t streams)
{
    int n = kv_splits_override() > MAX_SPLITS ? MAX_SPLITS : kv_splits_override();
    while (n > 1 && ((n & (n - 1)) || streams * n >= 1 << 22))
        n--;
    return n < 0 ? 0 : n;
}

int64_t slots_of(const dream_attn_desc *d, const Choice &c, int groups, int splits)
{
    return (int64_t)d->batch * d->n_kv_heads * splits * groups * (c.shared ? c.nw : 1) * c.qt * 16;
}

size_t bytes_of(const dream_attn_desc *d, int64_t slots, int splits)
{
    if (splits == 1 || d->dtype != DREAM_BF16)
        return DREAM_WORKSPACE_MIN_BYTES;
    return align_up((size_t)slots * d->head_dim * 4, 256) + align_up((size_t)slots * 8, 256);
}

void make_plan(const dream_attn_desc *d, bool mx, int n_tree, int64_t max_kv_len, int window, int n_sink, WindowPlan *p)
{
    int tiles;
    int64_t steps;
    shape_of(d, n_tree, max_kv_len, window, n_sink, &tiles, &steps);
    const int64_t streams = (int64_t)d->batch * d->n_kv_heads;
    const Steps &s = STEPS[mx][d->head_dim == 64 ? 0 : d->head_dim == 128 ? 1 : 2];
    float least = INFINITY;
    *p = {};
    every_choice(d, mx, tiles, steps, [&](const Choice &c, int groups, int most) {
        const int forced = forced_splits(streams);
        for (int splits = forced ? forced : 1; splits <= (forced ? forced : most); splits *= 2) {
            const int64_t slots = slots_of(d, c, groups, splits);
            const float load = (float)((streams * groups * splits + 255) / 256) * (c.shared ? 1.0f : c.nw * 0.25f);
            const float n = (float)((steps + splits - 1) / splits);
            float us;
            if (c.shared)
                us = s.s_base + s.s_per_group * load + n * fmaxf(s.s_latency, s.s_issue * load) + (n_tree > 64 ? s.s_many_nodes : 0.0f);
            else
                us = s.base + s.per_group * load + (n_tree > 64 ? s.many_nodes : 0.0f) +
                     (float)(((int64_t)n + c.nw - 1) / c.nw) * fmaxf(s.latency + s.latency_tile * c.qt, (s.issue + s.issue_tile * c.qt) * load);
            if (splits > 1)
                us += 2.3f + 0.11f * splits + 1e-6f * d->head_dim * slots;
            if (us < least) {
                least = us;
                p->shared = c.shared;
                p->qt = c.qt; p->nw = c.nw; p->n_rg = groups; p->n_splits = splits;
                p->slots = slots;
            }
        }
    });
    p->n_units = streams * p->n_splits;
    p->off_ml = align_up((size_t)p->slots * d->head_dim * 4, 256);
}

template <int D, bool MX>
auto kernel_of(const WindowPlan &p)
{
    constexpr int MOST = most_tiles(D, MX), TWO = MOST < 2 ? MOST : 2, SHARED = shared_tiles(D, MX);
    if constexpr (SHARED > 0)
        if (p.shared)
            return &window_shared_kernel<D, SHARED, MX>;
    if constexpr (MX)
        if (p.nw == 8)
            return &window_attn_kernel<D, 1, 8, MX>;
    return p.qt == 1 ? &window_attn_kernel<D, 1, 4, MX> : p.qt == 2 ? &window_attn_kernel<D, TWO, 4, MX> : &window_attn_kernel<D, MOST, 4, MX>;
}

template <int D, bool MX>
int launch(WindowArgs &a, const WindowPlan &p, hipStream_t st)
{
    auto *kernel = kernel_of<D, MX>(p);
    // the fewest XCDs to a unit with which the busiest one has at most a fifth more than its share (2 KV heads, 125 row groups each: 104 us on two XCDs, 36 on eight)
    int lg = 0;
    while (lg < 3 && 2 << lg <= p.n_rg && 5 * 8 * (((p.n_units << lg) + 7) / 8) > 6 * (p.n_units << lg))
        lg++;
    const int64_t eights = ((p.n_units << lg) + 7) / 8;
    const dim3 grid(8 * ((p.n_rg + (1 << lg) - 1) >> lg), (unsigned)(eights < UNITS_Y ? eights : UNITS_Y), (unsigned)((eights + UNITS_Y - 1) / UNITS_Y));
    hipLaunchKernelGGL(kernel, grid, dim3(p.shared ? 512 : 64 * p.nw), 0, st, static_cast<const uint8_t *>(a.k), static_cast<const uint8_t *>(a.v), a.k_scales, a.v_scales, a.prefix_len,
                       (uint32_t)a.s_max, (uint32_t)a.n_kv_heads | (uint32_t)__builtin_ctz(p.n_splits) << 16 | (uint32_t)lg << 24, magic_of(a.n_kv_heads),
                       (uint32_t)a.n_tree | (a.window ? 0x200u : 0u) | (uint32_t)p.n_units << 10, a);
    if (int rc = check_launch("window_attn_kernel"))
        return rc;
    if (p.n_splits == 1)
        return DREAM_OK;
    const int64_t streams = p.n_units / p.n_splits, rows = (int64_t)a.n_tree * a.group, at_once = 1024 / D;
    const dim3 merge((unsigned)((rows + at_once - 1) / at_once), (unsigned)(streams < UNITS_Y ? streams : UNITS_Y), (unsigned)((streams + UNITS_Y - 1) / UNITS_Y));
    hipLaunchKernelGGL(window_merge_kernel<D>, merge, dim3(256), 0, st, a, p.n_rg * (p.shared ? 8 : 1) * p.qt * 16);
    return check_launch("window_merge_kernel");
}

int check_desc(const dream_attn_desc *d, const char *who)
{
    if (!d)
        return fail(DREAM_ERR_INVALID_ARG, "%s: desc is NULL", who);
    if (d->batch < 1 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->s_max < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: batch, head counts and s_max must be positive", who);
    if (d->n_q_heads % d->n_kv_heads)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_q_heads %d is not a multiple of n_kv_heads %d", who, d->n_q_heads, d->n_kv_heads);
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: head_dim %d not in {64,128,256}", who, d->head_dim);
    if (d->dtype != DREAM_F32 && d->dtype != DREAM_BF16)
        return fail(DREAM_ERR_INVALID_ARG, "%s: unknown dtype %d", who, d->dtype);
    if (d->batch > 65535 || d->n_q_heads > 4096 || (int64_t)d->batch * d->n_q_heads > (1 << 20) || d->s_max > MAX_ROWS)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: batch is limited to 65535, n_q_heads to 4096, their product to 2^20, s_max to %lld", who, (long long)MAX_ROWS);
    return DREAM_OK;
}

size_t workspace_for(const dream_attn_desc *d, bool mx, int n_tree, int64_t max_kv_len, int window, int n_sink)
{
    if (!d || d->batch < 1 || d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads || d->head_dim < 1 || n_tree < 1 || max_kv_len < 1 ||
        window < 0 || n_sink < 0)
        return DREAM_WORKSPACE_MIN_BYTES;
    // what the most splits of any choice need, so that it never falls as max_kv_len rises
    int tiles;
    int64_t steps;
    shape_of(d, n_tree, max_kv_len, window, n_sink, &tiles, &steps);
    size_t total = DREAM_WORKSPACE_MIN_BYTES;
    every_choice(d, mx, tiles, steps, [&](const Choice &c, int groups, int most) {
        const int forced = forced_splits((int64_t)d->batch * d->n_kv_heads), splits = forced ? forced : most;
        const size_t bytes = bytes_of(d, slots_of(d, c, groups, splits), splits);
        total = bytes > total ? bytes : total;
    });
    return total;
}

int run(const char *who, const dream_attn_desc *d, bool mx, WindowArgs &a, int64_t max_kv_len, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = check_desc(d, who))
        return rc;
    if (!a.q || !a.k || !a.v || !a.prefix_len || !a.out || (mx && (!a.k_scales || !a.v_scales)))
        return fail(DREAM_ERR_INVALID_ARG, "%s: q, the caches, prefix_len and out must not be NULL", who);
    if (!a.parent && (!a.tree_mask || a.window))
        return fail(DREAM_ERR_INVALID_ARG, "%s: parent is NULL: without a tree_mask it says what a node sees, with a window how deep it is", who);
    if (a.n_tree < 1 || a.n_tree > DREAM_MAX_TREE)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: n_tree %d outside [1, %d]", who, a.n_tree, DREAM_MAX_TREE);
    if (a.window < 0 || a.n_sink < 0 || a.window > (1 << 30) || a.n_sink > (1 << 30))
        return fail(DREAM_ERR_INVALID_ARG, "%s: window %d and n_sink %d must be in [0, 2^30]", who, a.window, a.n_sink);
    if (max_kv_len < a.n_tree || max_kv_len > d->s_max)
        return fail(DREAM_ERR_INVALID_ARG, "%s: max_kv_len %lld outside [n_tree, s_max]", who, (long long)max_kv_len);
    if ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.out)) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: q, the caches and out must be 16-byte aligned", who);
    if (mx && ((reinterpret_cast<uintptr_t>(a.k_scales) | reinterpret_cast<uintptr_t>(a.v_scales)) & 7))
        return fail(DREAM_ERR_INVALID_ARG, "%s: scales must be 8-byte aligned", who);
    WindowPlan p;
    make_plan(d, mx, a.n_tree, max_kv_len, a.window, a.n_sink, &p);
    const size_t needed = workspace_for(d, mx, a.n_tree, max_kv_len, a.window, a.n_sink);
    if (!ws || ws_bytes < needed || (reinterpret_cast<uintptr_t>(ws) & 15))
        return fail(DREAM_ERR_WORKSPACE, "%s: 16-byte aligned workspace of %zu bytes, %zu needed", who, ws_bytes, needed);
    a.part = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(ws) + p.off_ml);
    a.s_max = d->s_max;
    a.n_q_heads = d->n_q_heads; a.n_kv_heads = d->n_kv_heads; a.group = d->n_q_heads / d->n_kv_heads;
    a.mask_words = ceil_div(a.n_tree, 64);
    a.tree_magic = magic_of(a.n_tree);
    a.heads_magic = magic_of(a.n_kv_heads);
    a.n_rg = p.n_rg; a.n_splits = p.n_splits; a.n_units = (int32_t)p.n_units;
    a.scale = d->scale != 0.0f ? d->scale : 1.0f / sqrtf((float)d->head_dim);
    a.scale_log2 = a.scale * 1.4426950408889634f;
    hipStream_t st = as_stream(stream);
    if (d->dtype == DREAM_F32) {
        const dim3 grid(a.n_tree, d->n_q_heads, d->batch);
        auto *kernel = d->head_dim == 64 ? (mx ? &window_f32_kernel<64, true> : &window_f32_kernel<64, false>)
                       : d->head_dim == 128 ? (mx ? &window_f32_kernel<128, true> : &window_f32_kernel<128, false>)
                                            : (mx ? &window_f32_kernel<256, true> : &window_f32_kernel<256, false>);
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a);
        return check_launch("window_f32_kernel");
    }
    if (mx)
        return d->head_dim == 64 ? launch<64, true>(a, p, st) : d->head_dim == 128 ? launch<128, true>(a, p, st) : launch<256, true>(a, p, st);
    return d->head_dim == 64 ? launch<64, false>(a, p, st) : d->head_dim == 128 ? launch<128, false>(a, p, st) : launch<256, false>(a, p, st);
}

}  // namespace

extern "C" {

size_t dream_window_verify_attn_workspace(const dream_attn_desc *desc, int32_t n_tree, int64_t max_kv_len, int32_t window, int32_t n_sink)
{
    return workspace_for(desc, false, n_tree, max_kv_len, window, n_sink);
}

size_t dream_mx_verify_attn_workspace(const dream_attn_desc *desc, int32_t n_tree, int64_t max_kv_len, int32_t window, int32_t n_sink)
{
    return workspace_for(desc, true, n_tree, max_kv_len, window, n_sink);
}

int dream_window_verify_attn(const dream_attn_desc *desc, const void *q, const void *k_cache, const void *v_cache, const int32_t *prefix_len,
                             int32_t n_tree, const int32_t *parent, const uint64_t *tree_mask, int32_t window, int32_t n_sink,
                             int64_t max_kv_len, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    WindowArgs a = {};
    a.q = q; a.k = k_cache; a.v = v_cache;
    a.prefix_len = prefix_len; a.parent = parent; a.tree_mask = tree_mask; a.out = out; a.lse = lse;
    a.n_tree = n_tree; a.window = window; a.n_sink = n_sink;
    return run("dream_window_verify_attn", desc, false, a, max_kv_len, workspace, workspace_bytes, stream);
}

int dream_mx_verify_attn(const dream_attn_desc *desc, const void *q, const void *k_codes, const void *k_scales, const void *v_codes,
                         const void *v_scales, const int32_t *prefix_len, int32_t n_tree, const int32_t *parent, const uint64_t *tree_mask,
                         int32_t window, int32_t n_sink, int64_t max_kv_len, void *out, float *lse, void *workspace, size_t workspace_bytes,
                         void *stream)
{
    WindowArgs a = {};
    a.q = q; a.k = k_codes; a.v = v_codes; a.k_scales = static_cast<const uint8_t *>(k_scales); a.v_scales = static_cast<const uint8_t *>(v_scales);
    a.prefix_len = prefix_len; a.parent = parent; a.tree_mask = tree_mask; a.out = out; a.lse = lse;
    a.n_tree = n_tree; a.window = window; a.n_sink = n_sink;
    return run("dream_mx_verify_attn", desc, true, a, max_kv_len, workspace, workspace_bytes, stream);
}

}  // extern "C"
