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
// A row of 4 bits is turned into bf16 once for all QT tiles of a wave.
#include <type_traits>
#include "common.h"

using namespace dream;

namespace {

constexpr int GROUP = DREAM_MX_GROUP;
constexpr float SLACK = 8.0f;      // octaves by which a score may exceed its row's reference
constexpr int MAX_SPLITS = 64;

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
    float scale, scale_log2;
};

// Bits of the 32 keys from j0 on that lie in [from, to).
__device__ __forceinline__ uint32_t key_bits(int j0, int from, int to)
{
    const int lo = max(from - j0, 0), hi = min(to - j0, 32);
    if (lo >= hi)
        return 0u;
    return (0xffffffffu >> (32 - (hi - lo))) << lo;
}

// Which tree nodes the rows see, and where their windows start; in LDS.
struct TreeLds {
    uint64_t mask[DREAM_MAX_TREE * (DREAM_MAX_TREE / 64)];
    int32_t parent[DREAM_MAX_TREE], depth[DREAM_MAX_TREE];
    int32_t deepest;
};

// All threads of the workgroup; ends with a barrier.
__device__ __forceinline__ void build_tree(TreeLds &t, const WindowArgs &a, int b, int P, int tid, int threads)
{
    const int T = a.n_tree, W = a.mask_words;
    const bool walk = !a.tree_mask || a.window;
    if (walk) {
        for (int i = tid; i < T; i += threads) {
            const int p = a.parent[(int64_t)b * T + i];
            t.parent[i] = p < i ? p : -1;      // a walk up the tree always ends
        }
        if (tid == 0)
            t.deepest = 0;
        __syncthreads();
    }
    for (int i = tid; i < T; i += threads) {
        int depth = 0;
        uint64_t m0 = 0;
        for (int w = 0; w < W; w++) {
            uint64_t m = 0;
            if (a.tree_mask) {
                m = a.tree_mask[((int64_t)b * T + i) * W + w];
                if (T - w * 64 < 64)
                    m &= (1ull << (T - w * 64)) - 1;
            } else if (i >> 6 == w) {
                m = 1ull << (i & 63);
            }
            if (W == 1)
                m0 = m;
            else
                t.mask[i * W + w] = m;
        }
        if (walk) {
            for (int p = t.parent[i]; p >= 0; p = t.parent[p]) {
                depth++;
                if (!a.tree_mask) {
                    if (W == 1)
                        m0 |= 1ull << p;
                    else
                        t.mask[i * W + (p >> 6)] |= 1ull << (p & 63);
                }
            }
            t.depth[i] = depth;
            if (a.window)
                atomicMax(&t.deepest, depth);
        }
        if (W == 1)
            t.mask[i] = m0;
    }
    __syncthreads();
    if (a.window && a.window < T) {            // the window may end inside the tree
        for (int i = tid; i < T; i += threads)
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
        __syncthreads();
    }
}

// The keys from j0 on that node i sees, whose window starts at lo.
__device__ __forceinline__ uint32_t visible_keys(const TreeLds &t, const WindowArgs &a, int node, int lo, int P, int j0)
{
    uint32_t bits = key_bits(j0, lo, P);
    if (a.window)
        bits |= key_bits(j0, 0, min(a.n_sink, P));
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

// The key tiles of a sequence, in the order they are taken: those of the sinks, then those from the root's window on.
struct Tiles {
    int sinks, first, count;
    __device__ __forceinline__ int at(int i) const { return i < sinks ? i : i - sinks + first; }
};
__device__ __forceinline__ Tiles tiles_of(const WindowArgs &a, int P)
{
    Tiles t;
    const int start = a.window ? max(0, P - a.window + 1) : 0;
    t.sinks = a.window ? (min(a.n_sink, start) + 31) / 32 : 0;
    t.first = max(start / 32, t.sinks);
    t.count = t.sinks + (P + a.n_tree + 31) / 32 - t.first;
    return t;
}

__device__ __forceinline__ bf16x8 from_codes(uint32_t codes, float scale)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// What a wave has of one tile, as it came from memory.
template <int D, bool MX>
struct Raw;
template <int D>
struct Raw<D, true> {
    static constexpr int KS = D == 256 ? 2 : 1, VP = D / 64;     // scales of a lane's K; 16-byte pieces of its V
    uint32_t k[2][D / 32];
    uint8_t ks[2][KS];
    u32x4 v[VP];
    uint8_t vs[VP];
};
template <int D>
struct Raw<D, false> {
    u32x4 k[2][D / 32];
    u32x4 v[D / 16];
};

template <int D, int QT, int NW, bool MX>
struct WindowGeom {
    static constexpr int VSTR = D + 16;                          // V row stride in LDS (values)
    static constexpr int AREA = 32 * VSTR * 2;                   // bytes of a wave's V tile; also holds 16 rows' O at the end
    static_assert(AREA >= 16 * D * 4, "the states of a query tile meet in the V areas");
};

template <int D, int QT, int NW, bool MX>
__global__ __launch_bounds__(64 * NW) void window_attn_kernel(WindowArgs a)
{
    using G = WindowGeom<D, QT, NW, MX>;
    constexpr int NKS = D / 32, NDT = D / 16, VSTR = G::VSTR;
    constexpr int ROWB = MX ? D / 2 : D * 2;                     // bytes of a row
    __shared__ __attribute__((aligned(16))) uint8_t s_area[NW][G::AREA];
    __shared__ TreeLds s_tree;
    __shared__ float s_ml[NW][QT][16][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    // row groups of one share of the keys get ids that are congruent mod 8, so that they meet in one XCD's L2
    const int unit = (int)(blockIdx.x / (8 * a.n_rg)) * 8 + (blockIdx.x & 7), rg = (blockIdx.x >> 3) % a.n_rg;
    if (unit >= a.n_units)
        return;
    const int split = unit % a.n_splits, stream = unit / a.n_splits, kvh = stream % a.n_kv_heads, b = stream / a.n_kv_heads;
    const int T = a.n_tree, rows = T * a.group;
    const int P = (int)min((int64_t)max(a.prefix_len[b], 0), a.s_max - T);   // never past the cache, whatever the array holds
    const Tiles tiles = tiles_of(a, P);
    const int per = (tiles.count + a.n_splits - 1) / a.n_splits;
    const int t0 = split * per + wave, t1 = min(tiles.count, split * per + per);
    const int64_t head_row = (int64_t)stream * a.s_max;
    const uint8_t *kb = static_cast<const uint8_t *>(a.k) + head_row * ROWB, *vb = static_cast<const uint8_t *>(a.v) + head_row * ROWB;
    const uint8_t *ksb = MX ? a.k_scales + head_row * (D / GROUP) : nullptr, *vsb = MX ? a.v_scales + head_row * (D / GROUP) : nullptr;

    auto request = [&](Raw<D, MX> &r, int j0) {
        const int last = (int)min((int64_t)31, a.s_max - 1 - j0);          // of a tile's rows inside the cache
        const uint8_t *kt = kb + (int64_t)j0 * ROWB, *vt = vb + (int64_t)j0 * ROWB;
        if constexpr (MX) {
            const uint8_t *kst = ksb + (int64_t)j0 * (D / GROUP), *vst = vsb + (int64_t)j0 * (D / GROUP);
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
                const int row = min(16 * hh + c, last);
                if constexpr (D == 64) {
                    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(kt + row * ROWB + g * 8);
                    r.k[hh][0] = x[0];
                    r.k[hh][1] = x[1];
                    r.ks[hh][0] = kst[row * 2 + (g >> 1)];
                } else {
#pragma unroll
                    for (int i = 0; i < D / 128; i++) {
                        const u32x4 x = *reinterpret_cast<const u32x4 *>(kt + row * ROWB + i * 64 + g * 16);
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            r.k[hh][i * 4 + e] = x[e];
                        r.ks[hh][i] = kst[row * (D / GROUP) + i * 4 + g];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < D / 64; i++) {
                const int p = lane + 64 * i, row = min(p / (D / GROUP), last), grp = p % (D / GROUP);
                r.v[i] = *reinterpret_cast<const u32x4 *>(vt + row * ROWB + grp * 16);
                r.vs[i] = vst[row * (D / GROUP) + grp];
            }
        } else {
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
                const int row = min(16 * hh + c, last);
#pragma unroll
                for (int ks = 0; ks < NKS; ks++)
                    r.k[hh][ks] = *reinterpret_cast<const u32x4 *>(kt + row * ROWB + ks * 64 + g * 16);
            }
#pragma unroll
            for (int i = 0; i < D / 16; i++) {
                const int p = lane + 64 * i, row = min(p / (D / 8), last);
                r.v[i] = *reinterpret_cast<const u32x4 *>(vt + row * ROWB + p % (D / 8) * 16);
            }
        }
    };

    Raw<D, MX> next;
    if (t0 < t1)
        request(next, tiles.at(t0) * 32);

    // the queries of this workgroup's rows, as the B operand; the channels in the order of the keys' pieces
    bf16x8 qf[QT][NKS];
    int node[QT], head[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        int f = (rg * QT + qt) * 16 + c;
        f = f < rows ? f : 0;
        head[qt] = kvh * a.group + f / T;
        node[qt] = f % T;
        const uint16_t *qp = static_cast<const uint16_t *>(a.q) + (((int64_t)b * T + node[qt]) * a.n_q_heads + head[qt]) * D;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++) {
            const int ch = !MX ? ks * 32 + g * 8 : D == 64 ? g * 16 + ks * 8 : (ks >> 2) * 128 + g * 32 + (ks & 3) * 8;
            qf[qt][ks] = *reinterpret_cast<const bf16x8 *>(qp + ch);
        }
    }
    build_tree(s_tree, a, b, P, tid, 64 * NW);
    const int lo_min = a.window ? P - a.window + 1 : 0, lo_max = a.window ? lo_min + s_tree.deepest : 0;      // windows' starts, root and deepest node

    f32x4 o[QT][NDT];
    float m[QT], l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        m[qt] = -INFINITY;
        l[qt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < NDT; dt++)
            o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    uint16_t *area = reinterpret_cast<uint16_t *>(s_area[wave]);
    const uint16_t *turned = area + (g * 4 + (c >> 2)) * VSTR + (c & 3) * 4;      // what this lane reads transposed
    auto read_v = [&](int dt) {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(turned + dt * 16));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(turned + dt * 16 + 16 * VSTR));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    for (int t = t0; t < t1; t += NW) {
        const Raw<D, MX> raw = next;
        const int j0 = tiles.at(t) * 32;
        if (t + NW < t1)
            request(next, tiles.at(t + NW) * 32);
        // every row sees every key of this tile, as it does but at the ends (a negative scale goes the general way)
        const bool whole = j0 + 32 <= P && (j0 >= lo_max || j0 + 32 <= a.n_sink) && a.scale_log2 >= 0.0f;

        // ---- S^T = K Q^T
        f32x4 s[2][QT];
#pragma unroll
        for (int hh = 0; hh < 2; hh++) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                s[hh][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < NKS; ks++) {
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

        // ---- V to LDS, as bf16.  Where not every row sees every key: rows that nobody may read are zeros, and so is, for now, what is not finite (0 * NaN is no zero)
        bool odd = false;
        auto dead = [&](int row) {
            const int j = j0 + row;
            return j >= P + T || (j < lo_min && j >= a.n_sink);
        };
        if constexpr (MX) {
#pragma unroll
            for (int i = 0; i < D / 64; i++) {
                const int p = lane + 64 * i, row = p / (D / GROUP), grp = p % (D / GROUP);
                uint32_t byte = raw.vs[i];
                if (!whole) {
                    byte = dead(row) ? 0u : byte;
                    odd = odd || byte > 252u;
                    byte = byte > 252u ? 0u : byte;
                }
                const float scale = scale_value(byte);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    *reinterpret_cast<bf16x8 *>(area + row * VSTR + grp * 32 + e * 8) = from_codes(raw.v[i][e], scale);
            }
        } else {
#pragma unroll
            for (int i = 0; i < D / 16; i++) {
                const int p = lane + 64 * i, row = p / (D / 8);
                u32x4 x = raw.v[i];
                if (!whole) {
                    const bool none = dead(row);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const bool lo = (x[e] & 0x7f80u) == 0x7f80u, hi = (x[e] & 0x7f800000u) == 0x7f800000u;
                        odd = odd || (!none && (lo || hi));
                        x[e] = none ? 0u : x[e] & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
                    }
                }
                *reinterpret_cast<u32x4 *>(area + row * VSTR + p % (D / 8) * 8) = x;
            }
        }

        // ---- online softmax; a lane owns query row c and keys g * 4 + r of both halves
        uint32_t vis[QT];
        float top[QT];
        float mult = a.scale_log2;
        if (whole) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                float x = s[0][qt][0];
#pragma unroll
                for (int e = 1; e < 8; e++)
                    x = fmaxf(x, s[e >> 2][qt][e & 3]);
                top[qt] = x * a.scale_log2;
                vis[qt] = 0xffffffffu;
            }
        } else {
            mult = 1.0f;
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                const int lo = a.window ? lo_min + s_tree.depth[node[qt]] : 0;
                vis[qt] = visible_keys(s_tree, a, node[qt], lo, P, j0) >> (g * 4);
                float x = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float y = vis[qt] >> ((e >> 2) * 16 + (e & 3)) & 1u ? s[e >> 2][qt][e & 3] * a.scale_log2 : -INFINITY;
                    s[e >> 2][qt][e & 3] = y;
                    x = fmaxf(x, y);
                }
                top[qt] = x;
            }
        }
        bool raise = false;
#pragma unroll
        for (int qt = 0; qt < QT; qt++)
            raise = raise || top[qt] > m[qt] + SLACK;
        if (__any(raise)) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                float x = fmaxf(top[qt], __shfl_xor(top[qt], 16));
                x = fmaxf(x, __shfl_xor(x, 32));
                if (x > m[qt] + SLACK) {
                    const float f = __builtin_amdgcn_exp2f(m[qt] - x);       // 0 where nothing was seen before
                    m[qt] = x;
                    l[qt] *= f;
#pragma unroll
                    for (int dt = 0; dt < NDT; dt++)
                        o[qt][dt] *= f;
                }
            }
        }
        bf16x8 pf[QT];
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const float neg = m[qt] == -INFINITY ? 0.0f : -m[qt];
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][qt][e & 3], mult, neg));
                sum += p;
                pf[qt][e] = (__bf16)p;       // (probabilities of a tile are rounded to bf16, half a step of 2^-8 each, as the matrix instruction takes them; sums stay float32)
            }
            l[qt] += sum;
        }

        // ---- O^T += V^T P^T
        wave_lds_fence();
#pragma unroll
        for (int dt = 0; dt < NDT; dt++) {
            const bf16x8 vf = read_v(dt);
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                o[qt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qt], o[qt][dt], 0, 0, 0);
        }
        wave_lds_fence();
        if (!whole && __any(odd)) {
            // Values that are not finite, in a tile that some row does not see all of: ones in their places and ones for the keys a row sees count them, and what
            // counts any is NaN.
#pragma unroll 1
            for (int i = 0; i < (MX ? D / 64 : D / 16); i++) {
                const int p = lane + 64 * i, row = p / (MX ? D / GROUP : D / 8);
                const int64_t at = min((int64_t)j0 + row, a.s_max - 1);
                if constexpr (MX) {
                    const int grp = p % (D / GROUP);
                    const bool bad = !dead(row) && vsb[at * (D / GROUP) + grp] > 252;
                    const u32x4 x = u32x4{1u, 1u, 1u, 1u} * (bad ? 0x3f803f80u : 0u);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        *reinterpret_cast<u32x4 *>(area + row * VSTR + grp * 32 + e * 8) = x;
                } else {
                    u32x4 x = *reinterpret_cast<const u32x4 *>(vb + at * ROWB + p % (D / 8) * 16);
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        x[e] = dead(row) ? 0u : ((x[e] & 0x7f80u) == 0x7f80u ? 0x3f80u : 0u) | ((x[e] & 0x7f800000u) == 0x7f800000u ? 0x3f800000u : 0u);
                    *reinterpret_cast<u32x4 *>(area + row * VSTR + p % (D / 8) * 8) = x;
                }
            }
            wave_lds_fence();
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    pf[qt][e] = (__bf16)(float)(vis[qt] >> ((e >> 2) * 16 + (e & 3)) & 1u);
#pragma unroll
            for (int dt = 0; dt < NDT; dt++) {
                const bf16x8 vf = read_v(dt);
#pragma unroll
                for (int qt = 0; qt < QT; qt++) {
                    const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qt], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; r++)
                        o[qt][dt][r] = n[r] > 0.0f ? __builtin_nanf("") : o[qt][dt][r];
                }
            }
            wave_lds_fence();
        }
    }

    // ---- the waves' states meet, one query tile after the other, in wave order
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        l[qt] += __shfl_xor(l[qt], 16);
        l[qt] += __shfl_xor(l[qt], 32);
        if (g == 0) {
            s_ml[wave][qt][c][0] = m[qt];
            s_ml[wave][qt][c][1] = l[qt];
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        __syncthreads();
        float mt = -INFINITY, lt = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; w++)
            mt = fmaxf(mt, s_ml[w][qt][c][0]);
        const float ref = mt == -INFINITY ? 0.0f : mt;
#pragma unroll
        for (int w = 0; w < NW; w++)
            lt += s_ml[w][qt][c][1] * __builtin_amdgcn_exp2f(s_ml[w][qt][c][0] - ref);
        const float f = __builtin_amdgcn_exp2f(m[qt] - ref);
        f32x4 *mine = reinterpret_cast<f32x4 *>(s_area[wave]);
#pragma unroll
        for (int dt = 0; dt < NDT; dt++)
            mine[dt * 64 + lane] = o[qt][dt] * f;
        __syncthreads();
        // a thread takes 8 channels of row c
        const int fr = (rg * QT + qt) * 16 + c;
        for (int k = tid >> 4; k < D / 8; k += 4 * NW) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
            const int from = (k >> 1) * 64 + (k & 1) * 32 + c;
#pragma unroll
            for (int w = 0; w < NW; w++) {
                const f32x4 *src = reinterpret_cast<const f32x4 *>(s_area[w]);
                x += src[from];
                y += src[from + 16];
            }
            if (fr < rows) {
                if (a.n_splits > 1) {
                    const int64_t slot = (((int64_t)unit * a.n_rg + rg) * QT + qt) * 16 + c;
                    f32x4 *dst = reinterpret_cast<f32x4 *>(a.part + slot * D + k * 8);
                    dst[0] = x;
                    dst[1] = y;
                    if (k == 0) {
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
                    const int hq = kvh * a.group + fr / T, n = fr % T;
                    *reinterpret_cast<bf16x8 *>(static_cast<uint16_t *>(a.out) + (((int64_t)b * T + n) * a.n_q_heads + hq) * D + k * 8) = r;
                    if (a.lse && k == 0)
                        a.lse[((int64_t)b * a.n_q_heads + hq) * T + n] = lt != 0.0f ? (mt + log2f(lt)) * 0.6931471805599453f : -INFINITY;
                }
            }
        }
    }
}

// The states of a row's key splits, in their order.  D / 4 lanes a row.
template <int D>
__global__ __launch_bounds__(256) void window_merge_kernel(WindowArgs a, int rows_per_unit)
{
    constexpr int LPR = D / 4;
    const int rows = a.n_tree * a.group, n = a.n_splits;
    const int64_t at = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int lane = threadIdx.x % LPR;
    const int64_t stream = at / rows;
    const int f = (int)(at - stream * rows);
    if (stream * n >= a.n_units)
        return;
    const int64_t slot = stream * n * rows_per_unit + f;
    float m = -INFINITY;
    for (int s = 0; s < n; s++)
        m = fmaxf(m, a.part_ml[(slot + (int64_t)s * rows_per_unit) * 2]);
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < n; s++) {
        const int64_t i = slot + (int64_t)s * rows_per_unit;
        const float w = __builtin_amdgcn_exp2f(a.part_ml[i * 2] - ref);
        l += w * a.part_ml[i * 2 + 1];
        o += *reinterpret_cast<const f32x4 *>(a.part + i * D + lane * 4) * w;
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    const int kvh = (int)(stream % a.n_kv_heads), hq = kvh * a.group + f / a.n_tree, node = f % a.n_tree;
    const int64_t b = stream / a.n_kv_heads;
    bf16x4 r;
#pragma unroll
    for (int e = 0; e < 4; e++)
        r[e] = (__bf16)(o[e] * inv);
    *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(a.out) + ((b * a.n_tree + node) * a.n_q_heads + hq) * D + lane * 4) = r;
    if (a.lse && lane == 0)
        a.lse[(b * a.n_q_heads + hq) * a.n_tree + node] = l != 0.0f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// float32 queries and rows (the small configuration): one workgroup of 4 waves per (node, head, sequence), D / 4 lanes a key, each with 4 channels; every wave keeps a state
// of its own keys and they meet in LDS.  Only keys that the node's window reaches are read.
template <int D, bool MX>
__global__ __launch_bounds__(256) void window_f32_kernel(WindowArgs a)
{
    constexpr int LPK = D / 4, KPW = 64 / LPK, U = 4, PASS = 4 * KPW * U;
    __shared__ TreeLds s_tree;
    __shared__ __attribute__((aligned(16))) float s_o[4][D];
    __shared__ float s_m[4], s_l[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane % LPK;
    const int node = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, T = a.n_tree;
    const int P = (int)min((int64_t)max(a.prefix_len[b], 0), a.s_max - T);
    const int64_t head_row = ((int64_t)b * a.n_kv_heads + hq / a.group) * a.s_max;
    const f32x4 q = reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.q) + (((int64_t)b * T + node) * a.n_q_heads + hq) * D)[col];
    build_tree(s_tree, a, b, P, tid, 256);
    const int lo = a.window ? max(0, P - a.window + 1 + s_tree.depth[node]) : 0, start = min(lo, P);
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
            see[u] = i < count && (rel < 0 || (s_tree.mask[node * a.mask_words + (rel >> 6)] >> (rel & 63) & 1ull));
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
    int qt, nw, n_rg, n_splits;
    int64_t n_units, slots;
    size_t off_ml, total;
};

void make_plan(const dream_attn_desc *d, int n_tree, int64_t max_kv_len, int window, int n_sink, WindowPlan *p)
{
    const int64_t streams = (int64_t)d->batch * d->n_kv_heads;
    const int tiles = ceil_div((int64_t)d->n_q_heads / d->n_kv_heads * n_tree, 16);
    int64_t keys = max_kv_len;
    if (window && (int64_t)window + n_tree + n_sink + 64 < keys)
        keys = (int64_t)window + n_tree + n_sink + 64;
    const int64_t steps = ceil_div(keys, 32);
    const int most = d->head_dim == 256 ? 2 : 4;
    p->nw = 4;
    p->qt = 1;
    while (p->qt < most && p->qt < tiles)
        p->qt *= 2;
    while (p->qt > 1 && streams * ceil_div(tiles, p->qt) < 256)
        p->qt /= 2;
    p->n_rg = ceil_div(tiles, p->qt);
    const int64_t wgs = streams * p->n_rg;
    int64_t splits = wgs >= 256 ? 1 : 512 / wgs;
    if (splits > steps / (2 * p->nw))
        splits = steps / (2 * p->nw);
    p->n_splits = (int)(splits < 1 ? 1 : splits > MAX_SPLITS ? MAX_SPLITS : splits);
    p->n_units = streams * p->n_splits;
    p->slots = p->n_units * p->n_rg * p->qt * 16;
    p->off_ml = 0;
    p->total = DREAM_WORKSPACE_MIN_BYTES;
    if (p->n_splits > 1 && d->dtype == DREAM_BF16) {
        p->off_ml = align_up((size_t)p->slots * d->head_dim * 4, 256);
        p->total = p->off_ml + align_up((size_t)p->slots * 8, 256);
    }
}

template <int D, bool MX>
int launch(const WindowArgs &a, const WindowPlan &p, hipStream_t st)
{
    constexpr int MOST = D == 256 ? 2 : 4;
    auto *kernel = p.qt == 1 ? &window_attn_kernel<D, 1, 4, MX> : p.qt == 2 ? &window_attn_kernel<D, 2, 4, MX> : &window_attn_kernel<D, MOST, 4, MX>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((p.n_units + 7) / 8 * 8 * p.n_rg)), dim3(64 * p.nw), 0, st, a);
    if (int rc = check_launch("window_attn_kernel"))
        return rc;
    if (p.n_splits == 1)
        return DREAM_OK;
    const int64_t rows = p.n_units / p.n_splits * a.n_tree * a.group;
    hipLaunchKernelGGL(window_merge_kernel<D>, dim3((unsigned)((rows + 1024 / D - 1) / (1024 / D))), dim3(256), 0, st, a, p.n_rg * p.qt * 16);
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
    if (d->batch > 65535 || d->n_q_heads > 65535 || (int64_t)d->batch * d->n_q_heads > (1 << 20) || d->s_max > (1 << 30))
        return fail(DREAM_ERR_UNSUPPORTED, "%s: batch and n_q_heads are limited to 65535, their product to 2^20, s_max to 2^30", who);
    return DREAM_OK;
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
    make_plan(d, a.n_tree, max_kv_len, a.window, a.n_sink, &p);
    if (!ws || ws_bytes < p.total || (reinterpret_cast<uintptr_t>(ws) & 15))
        return fail(DREAM_ERR_WORKSPACE, "%s: 16-byte aligned workspace of %zu bytes, %zu needed", who, ws_bytes, p.total);
    a.part = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float *>(static_cast<char *>(ws) + p.off_ml);
    a.s_max = d->s_max;
    a.n_q_heads = d->n_q_heads; a.n_kv_heads = d->n_kv_heads; a.group = d->n_q_heads / d->n_kv_heads;
    a.mask_words = ceil_div(a.n_tree, 64);
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

size_t workspace_for(const dream_attn_desc *d, int n_tree, int64_t max_kv_len, int window, int n_sink)
{
    if (!d || d->batch < 1 || d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads || d->head_dim < 1 || n_tree < 1 || max_kv_len < 1 ||
        window < 0 || n_sink < 0)
        return DREAM_WORKSPACE_MIN_BYTES;
    WindowPlan p;
    make_plan(d, n_tree, max_kv_len, window, n_sink, &p);
    return p.total;
}

}  // namespace

extern "C" {

size_t dream_window_verify_attn_workspace(const dream_attn_desc *desc, int32_t n_tree, int64_t max_kv_len, int32_t window, int32_t n_sink)
{
    return workspace_for(desc, n_tree, max_kv_len, window, n_sink);
}

size_t dream_mx_verify_attn_workspace(const dream_attn_desc *desc, int32_t n_tree, int64_t max_kv_len, int32_t window, int32_t n_sink)
{
    return workspace_for(desc, n_tree, max_kv_len, window, n_sink);
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
