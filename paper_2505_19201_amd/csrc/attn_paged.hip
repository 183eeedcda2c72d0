// Tree-masked attention over caches held in pages (dream_paged_verify_attn), with a prefix that sequences share read once for all of them, and over pages that were selected for each node
// (dream_sparse_verify_attn).
//
// out_i = sum_j softmax_j(scale q_i k_j) v_j over the keys j that node i sees (Eq. 1 under the draft-tree mask of Section 3.1).  One pass over the keys with a running maximum and sum; a softmax
// over two sets of keys joins from (maximum, sum, weighted rows) of each, so the shared positions and a sequence's own are two sets: of the first, the rows of all sequences of a group
// that share a KV head are one long list of query rows over the first sequence's pages; of the second, every sequence has its own.  Each set is cut further where there are too few workgroups, and
// the parts are joined by a second kernel.
//
// A workgroup has QT tiles of 16 query rows in each of its waves, and a list of pages in LDS (physical page; for selected pages also where it stands in the sequence and which nodes see it), which it
// takes tile by tile straight to LDS (the pages' addresses are scalars, 16 rows never leave a page).  S^T = K Q^T and O^T += V^T P^T by v_mfma_f32_16x16x32_bf16: a lane owns a query row, its
// scores are the second product's operand as they come.  Two forms: WR = 1, few rows: the waves share the keys out and have stages of their own, so they meet only at the end; WR > 1, many rows: the
// waves share the tiles and have rows of their own, one barrier a tile.
//
// What rows that nobody sees hold does not matter: V's are overwritten with zeros in LDS.  A value that is not finite in a row that some nodes see and others do not would poison the others through
// 0 * inf; instead of looking at every value, a workgroup looks at its sums at the end, and where one is not finite it takes its rows again, one by one over the keys they see (attend_rows_singly,
// which is also the whole of the float32 form).
#include <float.h>
#include <type_traits>
#include "lds_tiles.h"
#include "paged.h"

using namespace dream;

namespace {

constexpr float SLACK = 8.0f;             // octaves a score may exceed its row's reference by before that is raised
constexpr int DENSE_LIST = 512;           // pages a workgroup's list holds where all are taken

struct PagedAttnArgs {
    const unsigned char *q, *k, *v;
    const int32_t *table, *prefix_len, *parent, *group_start, *shared_len;
    const uint64_t *tree_mask, *nodes;
    void *out;
    float *lse, *part_o;
    float2 *part_ml;
    int64_t all_rows;                     // rows of a slot of part_o
    int32_t batch, n_tree, words, hq, hkv, group, rows;      // rows: query rows of a sequence and KV head
    int32_t lg_page, n_pages, max_pages, n_groups;
    int32_t shared, splits, slot, n_slots, shared_slots, streams, row_groups, list_size;      // of this launch: are these the shared positions; its slots
    float scale_log2;
};

// What a workgroup does.
struct Unit {
    int b, kvh, split, row0, n_rows;      // the sequence whose pages are read; rows are numbered through the sequences from b on
    int lo, hi, P;                        // positions [lo, hi), of which those from P on are the tree's
};

__device__ __forceinline__ int clamped_prefix(const PagedAttnArgs &a, int p) { return min(max(p, 0), (a.max_pages << a.lg_page) - a.n_tree); }

// The group that sequence b is in: its first sequence, and how many positions it shares; no group: b and 0.
__device__ __forceinline__ void group_of(const PagedAttnArgs &a, int b, int lane, int &first, int &shared)
{
    first = b;
    shared = -1;
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
        const int g = min(g0 + lane, a.n_groups - 1);
        const int s = a.group_start[g], e = a.group_start[g + 1], n = a.shared_len[g];
        const uint64_t mine = __ballot(s <= b && b < e);
        if (mine) {
            const int l = __builtin_ctzll(mine);
            first = min(max(__builtin_amdgcn_readlane(s, l), 0), b);
            shared = min(max(__builtin_amdgcn_readlane(n, l), 0), a.max_pages << a.lg_page);
            return;
        }
    }
}

// The group whose query rows the t-th tile of `cap` rows of all groups has.  first, n (sequences), shared, row0; n = 0: there is no such tile.
__device__ __forceinline__ void group_of_tile(const PagedAttnArgs &a, int t, int cap, int lane, int &first, int &n, int &shared, int &row0)
{
    n = 0;
    first = shared = row0 = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
        const int g = g0 + lane;
        int s = 0, e = 0, len = 0;
        if (g < a.n_groups) {
            s = min(max(a.group_start[g], 0), a.batch);
            e = min(max(a.group_start[g + 1], s), a.batch);
            len = a.shared_len[g];
        }
        const int tiles = (int)(((int64_t)(e - s) * a.rows + cap - 1) / cap);
        int sum = tiles;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(sum, d);
            sum += lane >= d ? x : 0;
        }
        const uint64_t behind = __ballot(t < sum);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            first = __builtin_amdgcn_readlane(s, l);
            n = __builtin_amdgcn_readlane(e, l) - first;
            shared = min(max(__builtin_amdgcn_readlane(len, l), 0), a.max_pages << a.lg_page);
            row0 = (t - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(tiles, l))) * cap;
            return;
        }
        t -= __builtin_amdgcn_readlane(sum, 63);
    }
}

// Workgroup ids that are congruent mod 8 run on one XCD: row groups that read the same keys meet in one L2.
__device__ __forceinline__ bool unit_of(const PagedAttnArgs &a, int cap, int lane, Unit &u)
{
    const uint32_t at = blockIdx.x >> 3, rg = at % (uint32_t)a.row_groups, stream = at / (uint32_t)a.row_groups * 8 + (blockIdx.x & 7);
    if (stream >= (uint32_t)a.streams)
        return false;
    u.split = stream % (uint32_t)a.splits;
    const uint32_t head = stream / (uint32_t)a.splits;
    u.kvh = head % (uint32_t)a.hkv;
    if (a.shared) {
        int n, shared;
        group_of_tile(a, rg, cap, lane, u.b, n, shared, u.row0);
        u.n_rows = n * a.rows;
        u.lo = 0;
        u.hi = u.P = shared;
        return n > 0;
    }
    u.b = head / (uint32_t)a.hkv;
    u.row0 = rg * cap;
    u.n_rows = a.rows;
    u.P = clamped_prefix(a, uniform_load(a.prefix_len + u.b));
    u.hi = u.P + a.n_tree;
    u.lo = 0;
    if (a.n_groups) {
        int first, shared;
        group_of(a, u.b, lane, first, shared);
        u.lo = min(max(shared, 0), u.P);
    }
    return true;
}

// ---- the list of pages -----------------------------------------------------------------------------------------------
constexpr uint32_t TREE_PAGE = 1u << 31;      // of an entry of s_logical: the tree's rows in it are meant

// Batch after batch of the pages that this split takes.  Positions along the list: x counts rows of its pages from `base` on; tiles of KEYS rows start at multiples of KEYS.
template <int KEYS, int THREADS, bool SPARSE>
struct PageList {
    static constexpr int TILE = KEYS, SCAN = 4 * THREADS;      // SCAN: pages looked at in a batch, where they are selected
    int32_t *phys;
    uint32_t *logical;
    uint64_t *word;
    int32_t *counts;
    int n, base, first;             // entries; x of the first one; its place in the sequence (dense)
    int tile, tile_end;             // of the batch
    int next_page, end_page, all_first, all_end, rank, scanned;

    __device__ __forceinline__ void start(const PagedAttnArgs &a, const Unit &u, unsigned char *smem)
    {
        phys = reinterpret_cast<int32_t *>(smem);
        logical = reinterpret_cast<uint32_t *>(smem + 4 * a.list_size);
        word = reinterpret_cast<uint64_t *>(smem + 8 * a.list_size);
        counts = reinterpret_cast<int32_t *>(smem + 8 * a.list_size + (SPARSE ? 8 * a.words * a.list_size : 0));
        rewind(a, u);
    }
    __device__ __forceinline__ void rewind(const PagedAttnArgs &a, const Unit &u)
    {
        if constexpr (SPARSE) {
            rank = scanned = 0;
        } else {
            const int t0 = u.lo / KEYS, t1 = u.hi > u.lo ? (u.hi + KEYS - 1) / KEYS : t0;
            const int per = (t1 - t0 + a.splits - 1) / a.splits;
            all_first = min(t0 + u.split * per, t1);
            all_end = min(all_first + per, t1);
            next_page = (all_first * KEYS) >> a.lg_page;
            end_page = all_end > all_first ? min((int)(((int64_t)all_end * KEYS + (1 << a.lg_page) - 1) >> a.lg_page), a.max_pages) : next_page;
        }
    }
    // The next batch, by all threads; false: there is none.  Starts and ends with a barrier.
    __device__ __forceinline__ bool next(const PagedAttnArgs &a, const Unit &u, int tid)
    {
        const int32_t *table = a.table + (int64_t)u.b * a.max_pages;
        if constexpr (!SPARSE) {
            if (next_page >= end_page)
                return false;
            __syncthreads();
            n = min(end_page - next_page, a.list_size);
            for (int i = tid; i < n; i += THREADS)
                phys[i] = min(max(table[next_page + i], 0), a.n_pages - 1);
            first = next_page;
            base = first << a.lg_page;
            tile = max(all_first, base / KEYS);
            next_page += n;
            tile_end = next_page >= end_page ? all_end : min(all_end, (next_page << a.lg_page) / KEYS);
            __syncthreads();
            return true;
        } else {
            const int in_prefix = (u.P + (1 << a.lg_page) - 1) >> a.lg_page, tree_page = u.P >> a.lg_page;
            const int total = in_prefix + ((u.hi - 1) >> a.lg_page) - tree_page + 1;
            if (scanned >= total)
                return false;
            __syncthreads();
            const int lane = tid & 63, wave = tid >> 6;
            const uint64_t *nodes = a.nodes + ((int64_t)u.b * a.hkv + u.kvh) * a.max_pages * a.words;
            const uint64_t last = a.n_tree & 63 ? (1ull << (a.n_tree & 63)) - 1 : ~0ull;
            int taken = 0;
            uint32_t mine = 0;
            const int v0 = scanned + tid * 4;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                bool in = v0 + i >= in_prefix && v0 + i < total;
                if (v0 + i < in_prefix)
                    for (int w = 0; w < a.words; w++)
                        in = in || (nodes[(int64_t)(v0 + i) * a.words + w] & (w == a.words - 1 ? last : ~0ull)) != 0ull;
                mine |= (uint32_t)in << i;
                taken += in;
            }
            int sum = taken;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int x = __shfl_up(sum, d);
                sum += lane >= d ? x : 0;
            }
            if (lane == 63)
                counts[wave] = sum;
            __syncthreads();
            int before = rank, all = 0;
#pragma unroll
            for (int w = 0; w < THREADS / 64; w++) {
                const int x = counts[w];
                before += w < wave ? x : 0;
                all += x;
            }
            auto upto = [&](int r) { return r > u.split ? (r - u.split + a.splits - 1) / a.splits : 0; };      // this split's among the first r
            const int skipped = upto(rank);
            int r = before + sum - taken;
            for (int i = 0; i < 4; i++) {
                if (!(mine >> i & 1))
                    continue;
                if (r % a.splits == u.split) {
                    const int at = upto(r) - skipped, v = v0 + i;
                    const int page = v < in_prefix ? v : tree_page + v - in_prefix;
                    phys[at] = min(max(table[page], 0), a.n_pages - 1);
                    logical[at] = (uint32_t)page | (v < in_prefix ? 0u : TREE_PAGE);
                    for (int w = 0; w < a.words; w++)
                        word[at * a.words + w] = v < in_prefix ? nodes[(int64_t)v * a.words + w] : 0ull;
                }
                r++;
            }
            rank = __builtin_amdgcn_readfirstlane(rank + all);
            n = __builtin_amdgcn_readfirstlane(upto(rank) - skipped);
            scanned += SCAN;
            base = first = 0;
            tile = 0;
            tile_end = ((n << a.lg_page) + KEYS - 1) / KEYS;
            __syncthreads();
            return true;
        }
    }
    static size_t bytes(int list_size, int words) { return (size_t)list_size * (8 + (SPARSE ? 8 * words : 0)) + 64; }
};

// Where 16 rows of the list stand (all of it the same in every lane).
struct Chunk {
    int entry, at;                  // of the list; row in the page
    int pos;                        // position of the first row
    bool live, tree, prefix;        // the list has it; the rows that are meant: the tree's, the prefix's
};
template <bool SPARSE, class List>
__device__ __forceinline__ Chunk chunk_at(const PagedAttnArgs &a, const List &list, int x)
{
    Chunk c;
    x -= list.base;
    const int e = x >> a.lg_page;
    c.live = e < list.n;
    c.entry = min(e, list.n - 1);
    c.at = x & ((1 << a.lg_page) - 1);
    if constexpr (SPARSE) {
        const uint32_t l = __builtin_amdgcn_readfirstlane((int)list.logical[c.entry]);
        c.tree = l >> 31;
        c.prefix = !c.tree;
        c.pos = (int)((l & ~TREE_PAGE) << a.lg_page) + c.at;
    } else {
        c.tree = c.prefix = true;
        c.pos = ((list.first + e) << a.lg_page) + c.at;
    }
    return c;
}

// ---- rows ------------------------------------------------------------------------------------------------------------
struct Row {
    int b, r;                       // its sequence and number there
    int node, head;
};
__device__ __forceinline__ Row row_at(const PagedAttnArgs &a, const Unit &u, int j)
{
    Row w;
    w.b = u.b;
    w.r = j;
    if (a.shared) {
        const int s = (uint32_t)j / (uint32_t)a.rows;
        w.b += s;
        w.r = j - s * a.rows;
    }
    w.node = (uint32_t)w.r / (uint32_t)a.group;
    w.head = u.kvh * a.group + w.r - w.node * a.group;
    return w;
}
__device__ __forceinline__ int64_t row_of_q(const PagedAttnArgs &a, const Row &w) { return ((int64_t)w.b * a.n_tree + w.node) * a.hq + w.head; }
__device__ __forceinline__ int64_t row_of_part(const PagedAttnArgs &a, const Unit &u, const Row &w) { return (int64_t)(a.slot + u.split) * a.all_rows + ((int64_t)w.b * a.hkv + u.kvh) * a.rows + w.r; }
// Prefix positions below this are the row's
__device__ __forceinline__ int row_limit(const PagedAttnArgs &a, const Unit &u, const Row &w) { return a.shared ? min(u.hi, clamped_prefix(a, a.prefix_len[w.b])) : u.P; }

__device__ __forceinline__ void put_ml(const PagedAttnArgs &a, const Unit &u, const Row &w, float m, float l)
{
    if (a.n_slots > 1)
        a.part_ml[row_of_part(a, u, w)] = make_float2(m, l);
    else if (a.lse)
        a.lse[((int64_t)w.b * a.hq + w.head) * a.n_tree + w.node] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// Which nodes of the tree each of the workgroup's rows sees, `words` words a row; by all threads, ends with a barrier.  parents: n_tree words of LDS.
__device__ __forceinline__ void build_masks(const PagedAttnArgs &a, const Unit &u, uint64_t *masks, int32_t *parents, int cap, int tid, int threads)
{
    if (!a.tree_mask) {
        for (int i = tid; i < a.n_tree; i += threads)
            parents[i] = a.parent[(int64_t)u.b * a.n_tree + i];
        __syncthreads();
    }
    const uint64_t last = a.n_tree & 63 ? (1ull << (a.n_tree & 63)) - 1 : ~0ull;
    for (int j = tid; j < min(cap, u.n_rows - u.row0); j += threads) {
        const int node = (uint32_t)(u.row0 + j) / (uint32_t)a.group;
        if (a.tree_mask) {
            for (int w = 0; w < a.words; w++)
                masks[j * a.words + w] = a.tree_mask[((int64_t)u.b * a.n_tree + node) * a.words + w] & (w == a.words - 1 ? last : ~0ull);
            continue;
        }
        for (int w = 0; w < a.words; w++)
            masks[j * a.words + w] = 0ull;
        for (int p = node;;) {
            masks[j * a.words + (p >> 6)] |= 1ull << (p & 63);
            const int up = parents[p];
            if (up < 0 || up >= p)      // (a parent that does not precede its node is none)
                break;
            p = up;
        }
    }
    __syncthreads();
}
// Of the nodes n0 .. n0 + 3 (n0 may be negative) those that a row's mask has, as four bits
__device__ __forceinline__ uint32_t four_nodes(const PagedAttnArgs &a, const uint64_t *mask, int n0)
{
    if (n0 <= -4 || n0 >= a.n_tree)
        return 0u;
    if (n0 < 0)
        return (uint32_t)(mask[0] << -n0) & 15u;
    const int w = n0 >> 6, s = n0 & 63;
    uint64_t x = mask[w] >> s;
    if (s > 60 && w + 1 < a.words)
        x |= mask[w + 1] << (64 - s);
    return (uint32_t)x & 15u;
}

// ---- row by row ------------------------------------------------------------------------------------------------------
// The workgroup's rows, one to a wave at a time: a lane takes a key's whole product, then D / 64 channels of the weighted sum.  Only rows that the node sees are read.
// s_q: D floats for each wave.
template <class T, int D, int THREADS, bool SPARSE, class List>
__device__ void attend_rows_singly(const PagedAttnArgs &a, const Unit &u, List &list, const uint64_t *masks, float *s_q, int cap)
{
    constexpr int NW = THREADS / 64, CH = D / 64, N = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int count = min(cap, u.n_rows - u.row0), ps_mask = (1 << a.lg_page) - 1;
    float *q = s_q + wave * D;
    for (int j0 = 0; j0 < count; j0 += NW) {
        const bool mine = j0 + wave < count;
        const int j = min(j0 + wave, count - 1);
        const Row w = row_at(a, u, u.row0 + j);
        const int limit = row_limit(a, u, w);
        for (int i = lane; i < D; i += 64) {
            const T *p = reinterpret_cast<const T *>(a.q) + row_of_q(a, w) * D + i;
            if constexpr (std::is_same_v<T, float>)
                q[i] = *p;
            else
                q[i] = bf16_bits_to_float(*p);
        }
        float m = -INFINITY, l = 0.0f, o[CH];
#pragma unroll
        for (int i = 0; i < CH; i++)
            o[i] = 0.0f;
        list.rewind(a, u);
        while (list.next(a, u, tid)) {
            const int end = min(SPARSE ? list.n << a.lg_page : list.base + (list.n << a.lg_page), list.tile_end * List::TILE);
            for (int x0 = list.tile * List::TILE; x0 < end; x0 += 64) {
                const int x = x0 + lane - list.base, e = min(x >> a.lg_page, list.n - 1), at = x & ps_mask;
                int pos;
                bool sees = x0 + lane < end;
                const uint32_t entry = SPARSE ? list.logical[e] : 0u;
                pos = (SPARSE ? (int)((entry & ~TREE_PAGE) << a.lg_page) : (list.first + e) << a.lg_page) + at;
                const bool in_prefix = pos >= u.lo && pos < limit && (!SPARSE || (!(entry >> 31) && (list.word[e * a.words + (w.node >> 6)] >> (w.node & 63) & 1)));
                const int node = pos - u.P;
                const bool in_tree = !a.shared && node >= 0 && node < a.n_tree && (!SPARSE || entry >> 31) && (masks[j * a.words + (node >> 6)] >> (node & 63) & 1);
                sees = sees && (in_prefix || in_tree);
                float s = -INFINITY;
                const int64_t row = ((((int64_t)list.phys[e] * a.hkv + u.kvh) << a.lg_page) + at) * D;
                if (sees) {
                    const T *k = reinterpret_cast<const T *>(a.k) + row;
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
                    for (int i = 0; i < D; i += N) {
                        const u32x4 raw = *reinterpret_cast<const u32x4 *>(k + i);
#pragma unroll
                        for (int d = 0; d < 4; d++) {
                            if constexpr (std::is_same_v<T, float>) {
                                sum[d] = __builtin_fmaf(__uint_as_float(raw[d]), q[i + d], sum[d]);
                            } else {
                                sum[d] = __builtin_fmaf(__uint_as_float(raw[d] << 16), q[i + 2 * d], sum[d]);
                                sum[d] = __builtin_fmaf(__uint_as_float(raw[d] & 0xffff0000u), q[i + 2 * d + 1], sum[d]);
                            }
                        }
                    }
                    s = ((sum[0] + sum[1]) + (sum[2] + sum[3])) * a.scale_log2;
                }
                const float top = fmaxf(m, wave_max(s));
                const float f = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top), ref = fmaxf(top, -FLT_MAX);
                m = top;
                const float p = sees ? __builtin_amdgcn_exp2f(s - ref) : 0.0f;
                l = l * f + p;
#pragma unroll
                for (int i = 0; i < CH; i++)
                    o[i] *= f;
                for (uint64_t left = __ballot(sees); left; left &= left - 1) {
                    const int key = __builtin_ctzll(left);
                    const float pk = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), key));
                    const int64_t of = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(row >> 32), key) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)row, key));
                    const T *v = reinterpret_cast<const T *>(a.v) + of + lane * CH;
#pragma unroll
                    for (int i = 0; i < CH; i++) {
                        if constexpr (std::is_same_v<T, float>)
                            o[i] = __builtin_fmaf(pk, v[i], o[i]);
                        else
                            o[i] = __builtin_fmaf(pk, bf16_bits_to_float(v[i]), o[i]);
                    }
                }
            }
        }
        l = wave_sum(l);
        if (!mine)
            continue;
        if (lane == 0)
            put_ml(a, u, w, m, l);
#pragma unroll
        for (int i = 0; i < CH; i++) {
            const float x = a.n_slots > 1 ? o[i] : l == 0.0f ? 0.0f : o[i] / l;
            if (a.n_slots > 1)
                a.part_o[row_of_part(a, u, w) * D + lane * CH + i] = x;
            else if constexpr (std::is_same_v<T, float>)
                static_cast<float *>(a.out)[row_of_q(a, w) * D + lane * CH + i] = x;
            else
                static_cast<uint16_t *>(a.out)[row_of_q(a, w) * D + lane * CH + i] = __builtin_bit_cast(uint16_t, (__bf16)x);
        }
    }
}

// float32: there for its precision and for small shapes.
constexpr int SINGLE_ROWS = 4;
template <int D, bool SPARSE>
__global__ __launch_bounds__(256) void paged_f32_kernel(PagedAttnArgs a)
{
    using List = PageList<64, 256, SPARSE>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float *s_q = reinterpret_cast<float *>(smem);
    uint64_t *masks = reinterpret_cast<uint64_t *>(smem + 4 * D * 4);
    int32_t *parents = reinterpret_cast<int32_t *>(masks + SINGLE_ROWS * a.words);
    Unit u;
    if (!unit_of(a, SINGLE_ROWS, threadIdx.x & 63, u))
        return;
    if (!a.shared)
        build_masks(a, u, masks, parents, SINGLE_ROWS, threadIdx.x, 256);
    List list;
    list.start(a, u, smem + 4 * D * 4 + SINGLE_ROWS * a.words * 8 + DREAM_MAX_TREE * 4);
    attend_rows_singly<float, D, 256, SPARSE>(a, u, list, masks, s_q, SINGLE_ROWS);
}

// ---- bf16 ------------------------------------------------------------------------------------------------------------
template <int D, int QT, int WR, int WK>
struct PagedGeom {
    static constexpr int NW = WR * WK, THREADS = 64 * NW, CAP = 16 * QT * WR;
    static constexpr int ROW = 2 * D, KEYS = WR == 1 || D == 256 ? 32 : 64, TILE = KEYS * ROW, STAGE = 2 * TILE;
    static constexpr int NS = WR == 1 ? 2 : 3;
    static constexpr int LOADS = TILE / 1024 / WR;                          // of a wave, a tile and K or V
    static constexpr int STAGES = WK * NS * STAGE;
    static constexpr int JOIN = WR == 1 ? WK * 16 * QT * (D + 4) * 4 : 0;   // the waves' sums meet here
    static constexpr int MASKS = STAGES > JOIN ? STAGES : JOIN;
    static_assert(LOADS * 1024 * WR == TILE, "loads");
    static int masks(int words) { return CAP * words * 8; }
    static int small(int words) { return masks(words) + DREAM_MAX_TREE * 4 + NW * 8 + WK * 16 * QT * 8; }      // masks, parents, flags, (m, l) of the waves
};

template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ float largest(f32x4 a) { return fmaxf(fmaxf(fmaxf(a[0], a[1]), a[2]), a[3]); }

template <int D, int QT, int WR, int WK, bool SPARSE>
__global__ __launch_bounds__(64 * WR * WK) void paged_attn_kernel(PagedAttnArgs a)
{
    using G = PagedGeom<D, QT, WR, WK>;
    constexpr int ROW = G::ROW, KEYS = G::KEYS, NKS = D / 32, NDT = D / 16, LPR = ROW / 16, RPI = 1024 / ROW, NS = G::NS;
    using List = PageList<KEYS, G::THREADS, SPARSE>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave % WR, wk = wave / WR;
    const int c = lane & 15, g = lane >> 4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    uint64_t *masks = reinterpret_cast<uint64_t *>(smem + G::MASKS);
    int32_t *parents = reinterpret_cast<int32_t *>(smem + G::MASKS + G::CAP * a.words * 8);
    int32_t *flags = parents + DREAM_MAX_TREE;
    float2 *s_ml = reinterpret_cast<float2 *>(flags + 2 * G::NW);
    unsigned char *list_at = reinterpret_cast<unsigned char *>(s_ml + WK * 16 * QT);

    Unit u;
    if (!unit_of(a, G::CAP, lane, u))
        return;
    List list;
    list.start(a, u, list_at);

    // ---- query fragments: lane (c, g) has row c's channels 8 g .. of every 32
    bf16x8 qf[QT][NKS];
    int limit[QT], node[QT];
    int whole = 0x7fffffff;                       // prefix positions below it are everyone's
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        const Row w = row_at(a, u, min(u.row0 + (wr * QT + qt) * 16 + c, u.n_rows - 1));
        const unsigned char *q = a.q + row_of_q(a, w) * ROW + g * 16;
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
            qf[qt][ks] = *reinterpret_cast<const bf16x8 *>(q + ks * 64);
        limit[qt] = row_limit(a, u, w);
        node[qt] = w.node;
        whole = min(whole, limit[qt]);
    }
    if (a.shared) {
#pragma unroll
        for (int s = 1; s < 16; s *= 2)
            whole = min(whole, __shfl_xor(whole, s));
        whole = __builtin_amdgcn_readfirstlane(whole);
    } else {
        whole = u.P;
        build_masks(a, u, masks, parents, G::CAP, tid, G::THREADS);
    }

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
    const int foff = fragment_k<ROW>(c, g), voff = fragment_v<ROW>(c, g);
    const int krow = lane / LPR, kl = piece_k<ROW>(lane), vl = piece_v<ROW>(lane);
    const float scale_log2 = a.scale_log2;

    auto stage_at = [&](int i) { return (wk * NS + i % NS) * G::STAGE; };
    // The wave's share of tile t: 16-row pieces that its load instructions lie in, each within a page
    auto issue = [&](int t, int at) {
#pragma unroll
        for (int i = 0; i < G::LOADS; i++) {
            const int j = wr * G::LOADS + i;
            const Chunk ch = chunk_at<SPARSE>(a, list, t * KEYS + (j * RPI & ~15));
            const int page = __builtin_amdgcn_readfirstlane(list.phys[ch.entry]);
            const int64_t from = ((((int64_t)page * a.hkv + u.kvh) << a.lg_page) + ch.at + (j * RPI & 15)) * ROW;
            lds_load16(a.k + from, (uint32_t)(krow * ROW + (kl ^ swizzle_k<ROW>(j))), lds0 + at + j * 1024);
            lds_load16(a.v + from, (uint32_t)(krow * ROW + (vl ^ swizzle_v<ROW>(j))), lds0 + at + G::TILE + j * 1024);
        }
    };
    auto plain = [&](const Chunk &ch) { return ch.live && ch.prefix && ch.pos >= u.lo && ch.pos + 16 <= whole; };      // all its rows are everyone's (or everyone's whose page it is)
    // Zeros over the values of rows that are nobody's, by the wave that loaded them
    auto clear_dead = [&](int t, int at) {
        bool any = false;
#pragma unroll
        for (int i = 0; i < G::LOADS; i++) {
            const int j = wr * G::LOADS + i;
            const Chunk ch = chunk_at<SPARSE>(a, list, t * KEYS + (j * RPI & ~15));
            if (plain(ch))
                continue;
            const int pos = ch.pos + (j * RPI & 15) + krow;
            const bool seen = ch.live && ((ch.prefix && pos >= u.lo && pos < u.P) || (ch.tree && pos >= u.P && pos < u.hi));
            if (!seen)
                *reinterpret_cast<u32x4 *>(smem + at + G::TILE + j * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
            any = true;
        }
        if (any)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };

    // 32 keys from row `sub` * 32 of the tile at `at` on
    auto compute = [&](int t, int at, int sub) {
        Chunk ch[2];
        bool straight = true;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            ch[h] = chunk_at<SPARSE>(a, list, t * KEYS + sub * 32 + h * 16);
            straight = straight && plain(ch[h]);
        }
        bool in[2][QT];                           // selected pages: is the lane's node one of theirs
        if constexpr (SPARSE) {
            bool any = !straight;
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int qt = 0; qt < QT; qt++) {
                    in[h][qt] = list.word[ch[h].entry * a.words + (node[qt] >> 6)] >> (node[qt] & 63) & 1;
                    any = any || in[h][qt];
                }
            if (!__any(any))
                return;
        }
        const unsigned char *kt = smem + at + sub * 32 * ROW, *vt = smem + at + G::TILE + sub * 32 * ROW;
        f32x4 s[2][QT];
        {
            bf16x8 kf[NKS][2];
#pragma unroll
            for (int ks = 0; ks < NKS; ks++)
#pragma unroll
                for (int h = 0; h < 2; h++)
                    kf[ks][h] = *reinterpret_cast<const bf16x8 *>(kt + h * 16 * ROW + at_key_step(foff, ks));
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    s[h][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < NKS; ks++)
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int qt = 0; qt < QT; qt++)
                        s[h][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks][h], qf[qt][ks], s[h][qt], 0, 0, 0);
        }
        // ---- online softmax: a lane owns query row c and keys 4 g + r of both halves
        float top[QT];
        straight = straight && scale_log2 >= 0.0f;
        if (straight) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                if constexpr (SPARSE) {
                    const float x = in[0][qt] ? largest(s[0][qt]) : -INFINITY, y = in[1][qt] ? largest(s[1][qt]) : -INFINITY;
                    top[qt] = fmaxf(x, y) * scale_log2;
                } else {
                    top[qt] = fmaxf(largest(s[0][qt]), largest(s[1][qt])) * scale_log2;
                }
            }
        } else {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                top[qt] = -INFINITY;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int pos = ch[h].pos + 4 * g;
                    uint32_t vis = 0u;
                    if (ch[h].live && ch[h].prefix && (!SPARSE || in[h][qt])) {
#pragma unroll
                        for (int r = 0; r < 4; r++)
                            vis |= (uint32_t)(pos + r >= u.lo && pos + r < limit[qt]) << r;
                    }
                    if (ch[h].live && ch[h].tree && !a.shared)
                        vis |= four_nodes(a, masks + ((wr * QT + qt) * 16 + c) * a.words, pos - u.P);
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        s[h][qt][r] = vis >> r & 1u ? s[h][qt][r] * scale_log2 : -INFINITY;
                        top[qt] = fmaxf(top[qt], s[h][qt][r]);
                    }
                }
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
            const float ref = fmaxf(m[qt], -FLT_MAX);      // where all scores so far are -inf, their weight is 0 and not exp(-inf + inf)
            float sum = 0.0f;
            if (straight) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const float mult = SPARSE && !in[h][qt] ? 0.0f : scale_log2, less = SPARSE && !in[h][qt] ? -INFINITY : -ref;
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][qt][r], mult, less));
                        sum += p;
                        pf[qt][h * 4 + r] = (__bf16)p;      // rounded as the matrix instruction takes it, half a step of 2^-8; the sum stays float32
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const float p = __builtin_amdgcn_exp2f(s[e >> 2][qt][e & 3] - ref);
                    sum += p;
                    pf[qt][e] = (__bf16)p;
                }
            }
            l[qt] += sum;
        }
        // ---- O^T += V^T P^T
#pragma unroll
        for (int dt = 0; dt < NDT; dt++) {
            const unsigned char *vp = vt + at_column_tile(voff, dt);
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)vp);
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(vp + 16 * ROW));
            const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                o[qt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[qt], o[qt][dt], 0, 0, 0);
        }
    };

    while (list.next(a, u, tid)) {
        const int first = list.tile + wk, steps = max(0, (list.tile_end - first + WK - 1) / WK);
        constexpr int AHEAD = WR == 1 ? NS : NS - 1;
#pragma unroll
        for (int i = 0; i < AHEAD; i++)
            if (i < steps)
                issue(first + i * WK, stage_at(i));
        for (int i = 0; i < steps; i++) {
            const int t = first + i * WK, at = stage_at(i);
            if (i + AHEAD <= steps)
                wait_loads<(AHEAD - 1) * 2 * G::LOADS>();
            else
                wait_loads<0>();
            clear_dead(t, at);
            if constexpr (WR > 1) {
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // the tile is there, and all have done with the stage that is loaded next
                if (i + AHEAD < steps)
                    issue(t + AHEAD * WK, stage_at(i + AHEAD));
            }
#pragma unroll
            for (int sub = 0; sub < KEYS / 32; sub++)
                compute(t, at, sub);
            if constexpr (WR == 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (i + AHEAD < steps)
                    issue(t + AHEAD * WK, at);
            }
        }
    }

    // ---- the end: sums that are not finite have the rows taken again
    float strange = 0.0f;
#pragma unroll
    for (int qt = 0; qt < QT; qt++) {
        l[qt] += __shfl_xor(l[qt], 16);
        l[qt] += __shfl_xor(l[qt], 32);
        strange = __builtin_fmaf(l[qt], 0.0f, strange);
#pragma unroll
        for (int dt = 0; dt < NDT; dt++)
#pragma unroll
            for (int r = 0; r < 4; r++)
                strange = __builtin_fmaf(o[qt][dt][r], 0.0f, strange);
    }
    const bool mine = __any(strange != 0.0f);      // (0 * inf and 0 * NaN are NaN)
    if (lane == 0)
        flags[wave] = mine;
    if constexpr (WR == 1) {
        if (g == 0)
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                s_ml[wk * 16 * QT + qt * 16 + c] = make_float2(m[qt], l[qt]);
    }
    __syncthreads();
    int again = 0;
#pragma unroll
    for (int w = 0; w < G::NW; w++)
        again |= flags[w];
    if (again) {
        attend_rows_singly<uint16_t, D, G::THREADS, SPARSE>(a, u, list, masks, reinterpret_cast<float *>(smem), G::CAP);
        return;
    }
    if constexpr (WR == 1) {
        constexpr int STR = D + 4;
        float *join = reinterpret_cast<float *>(smem);
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            float most = -INFINITY;
#pragma unroll
            for (int w = 0; w < WK; w++)
                most = fmaxf(most, s_ml[w * 16 * QT + qt * 16 + c].x);
            const float f = m[qt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m[qt] - most);
            float *row = join + ((wk * QT + qt) * 16 + c) * STR + 4 * g;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)
                *reinterpret_cast<f32x4 *>(row + dt * 16) = o[qt][dt] * f;
        }
        __syncthreads();
        const int count = min(G::CAP, u.n_rows - u.row0);
        for (int i = tid; i < count * (D / 4); i += G::THREADS) {
            const int j = i / (D / 4), ch = i % (D / 4);
            const Row w = row_at(a, u, u.row0 + j);
            float most = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int x = 0; x < WK; x++)
                most = fmaxf(most, s_ml[x * 16 * QT + j].x);
            f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < WK; x++) {
                const float2 ml = s_ml[x * 16 * QT + j];
                sum += ml.x == -INFINITY ? 0.0f : ml.y * __builtin_amdgcn_exp2f(ml.x - most);
                all += *reinterpret_cast<const f32x4 *>(join + (x * 16 * QT + j) * STR + ch * 4);
            }
            if (ch == 0)
                put_ml(a, u, w, most, sum);
            if (a.n_slots > 1) {
                *reinterpret_cast<f32x4 *>(a.part_o + row_of_part(a, u, w) * D + ch * 4) = all;
            } else {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row_of_q(a, w) * D + ch * 4) = make_uint2(pack_bf16(all[0] * inv, all[1] * inv), pack_bf16(all[2] * inv, all[3] * inv));
            }
        }
    } else {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const int j = u.row0 + (wr * QT + qt) * 16 + c;
            if (j >= u.n_rows)
                continue;
            const Row w = row_at(a, u, j);
            if (g == 0)
                put_ml(a, u, w, m[qt], l[qt]);
            if (a.n_slots > 1) {
                float *row = a.part_o + row_of_part(a, u, w) * D + 4 * g;
#pragma unroll
                for (int dt = 0; dt < NDT; dt++)
                    *reinterpret_cast<f32x4 *>(row + dt * 16) = o[qt][dt];
            } else {
                const float inv = l[qt] == 0.0f ? 0.0f : 1.0f / l[qt];
                uint16_t *row = static_cast<uint16_t *>(a.out) + row_of_q(a, w) * D + 4 * g;
#pragma unroll
                for (int dt = 0; dt < NDT; dt++)
                    *reinterpret_cast<uint2 *>(row + dt * 16) = make_uint2(pack_bf16(o[qt][dt][0] * inv, o[qt][dt][1] * inv), pack_bf16(o[qt][dt][2] * inv, o[qt][dt][3] * inv));
            }
        }
    }
}

// ---- the parts of a row, in their order: D / 4 lanes a row -----------------------------------------------------------
template <class T, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnArgs a)
{
    constexpr int LANES = D / 4;
    const int64_t id = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int ch = threadIdx.x % LANES;
    if (id >= a.all_rows)
        return;
    const uint32_t head = (uint32_t)(id / a.rows);
    Row w;
    w.r = (int)(id - (int64_t)head * a.rows);
    w.b = head / (uint32_t)a.hkv;
    w.node = (uint32_t)w.r / (uint32_t)a.group;
    w.head = (head - w.b * a.hkv) * a.group + w.r - w.node * a.group;
    int first_slot = 0;
    if (a.shared_slots) {                 // a sequence outside every group has no shared parts
        bool in = false;
        for (int g = 0; g < a.n_groups && !in; g++)
            in = a.group_start[g] <= w.b && w.b < a.group_start[g + 1];
        first_slot = in ? 0 : a.shared_slots;
    }
    float most = -INFINITY, sum = 0.0f;
    for (int s = first_slot; s < a.n_slots; s++)
        most = fmaxf(most, a.part_ml[s * a.all_rows + id].x);
    f32x4 all = {0.f, 0.f, 0.f, 0.f};
    for (int s = first_slot; s < a.n_slots; s++) {
        const float2 ml = a.part_ml[s * a.all_rows + id];
        const f32x4 x = *reinterpret_cast<const f32x4 *>(a.part_o + (s * a.all_rows + id) * D + ch * 4);
        if (ml.y != 0.0f) {               // (NaN: not 0)
            const float f = __builtin_amdgcn_exp2f(fmaxf(ml.x, -FLT_MAX) - fmaxf(most, -FLT_MAX));
            sum = __builtin_fmaf(ml.y, f, sum);
            all += x * f;
        }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (ch == 0 && a.lse)
        a.lse[((int64_t)w.b * a.hq + w.head) * a.n_tree + w.node] = sum == 0.0f ? -INFINITY : (most + __log2f(sum)) * 0.6931471805599453f;
    const int64_t at = row_of_q(a, w) * D + ch * 4;
    if constexpr (std::is_same_v<T, float>)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.out) + at) = all * inv;
    else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16(all[0] * inv, all[1] * inv), pack_bf16(all[2] * inv, all[3] * inv));
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
struct Shape {                            // of a launch's workgroups: query tiles of a wave, waves for rows, waves for keys; qt = 0: float32
    int qt, wr, wk;
    int cap() const { return qt ? 16 * qt * wr : SINGLE_ROWS; }
    int keys(int D) const { return wr == 1 || D == 256 ? 32 : 64; }
    int threads() const { return qt ? 64 * wr * wk : 256; }
};
struct Launch {
    Shape shape;
    int splits, row_groups, streams;
};
struct PagedPlan {
    Launch shared, own;
    int n_slots;
    int64_t all_rows;
    size_t bytes;
};

Shape shape_for(int D, bool f32, int64_t rows)
{
    if (f32)
        return {0, 1, 4};
    const int wk = D == 256 ? 2 : 4;
    if (rows <= 16)
        return {1, 1, wk};
    if (rows <= 32)
        return {2, 1, wk};
    if (D == 256)
        return {1, 8, 1};
    if (rows <= 64)
        return {4, 1, wk};
    return rows <= 128 ? Shape{2, 4, 1} : Shape{2, 8, 1};
}

int splits_for(const Shape &s, int D, int64_t units, int64_t keys)
{
    const int64_t tiles = (keys + s.keys(D) - 1) / s.keys(D), least = s.wk > 1 ? 2 * s.wk : 4;
    if (const int forced = kv_splits_override())
        return forced < 64 ? forced : 64;
    int64_t n = 256 / (units > 0 ? units : 1);
    if (n > tiles / least)
        n = tiles / least;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

PagedPlan plan_for(const dream_attn_desc *d, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv, int32_t n_groups, int64_t max_shared, int64_t seen_pages)
{
    PagedPlan p = {};
    const int64_t capacity = paged_rows(pages), rows = (int64_t)n_tree * (d->n_q_heads / d->n_kv_heads);
    max_kv = max_kv < 1 ? 1 : max_kv > capacity ? capacity : max_kv;
    max_shared = max_shared < 1 ? 1 : max_shared > max_kv ? max_kv : max_shared;
    const bool f32 = d->dtype == DREAM_F32;
    p.own.shape = shape_for(d->head_dim, f32, rows);
    p.own.row_groups = ceil_div(rows, p.own.shape.cap());
    const int64_t heads = (int64_t)d->batch * d->n_kv_heads;
    int64_t own_keys = n_groups ? max_kv - max_shared + 1 : max_kv;
    if (seen_pages > 0 && seen_pages * pages->page_size + n_tree < own_keys)
        own_keys = seen_pages * pages->page_size + n_tree;
    p.own.splits = splits_for(p.own.shape, d->head_dim, heads * p.own.row_groups, own_keys);
    p.own.streams = (int)(heads * p.own.splits);
    p.n_slots = p.own.splits;
    p.all_rows = heads * rows;
    if (n_groups) {
        p.shared.shape = shape_for(d->head_dim, f32, d->batch * rows / n_groups);
        p.shared.row_groups = (int)(d->batch * rows / p.shared.shape.cap() + n_groups);
        p.shared.splits = splits_for(p.shared.shape, d->head_dim, (int64_t)d->n_kv_heads * (p.shared.row_groups - n_groups + 1), max_shared);
        p.shared.streams = d->n_kv_heads * p.shared.splits;
        p.n_slots += p.shared.splits;
    }
    p.bytes = p.n_slots > 1 ? (size_t)p.n_slots * p.all_rows * (d->head_dim + 2) * 4 : 0;
    return p;
}

template <int D, int QT, int WR, int WK, bool SPARSE>
int launch_bf16(PagedAttnArgs &a, int blocks, hipStream_t st)
{
    using G = PagedGeom<D, QT, WR, WK>;
    static std::atomic<uint64_t> done{0};
    using List = PageList<G::KEYS, G::THREADS, SPARSE>;
    a.list_size = SPARSE ? List::SCAN / a.splits + 2 : DENSE_LIST;
    const size_t lds = (size_t)G::MASKS + G::small(a.words) + List::bytes(a.list_size, a.words);
    auto *kernel = &paged_attn_kernel<D, QT, WR, WK, SPARSE>;
    if (int rc = raise_lds_limit(done, reinterpret_cast<const void *>(kernel), 160 * 1024, "paged attention"))
        return rc;
    if (lds > 160 * 1024)
        return fail(DREAM_ERR_UNSUPPORTED, "paged attention: %zu bytes of LDS", lds);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(G::THREADS), lds, st, a);
    return check_launch("paged_attn_kernel");
}

template <int D, bool SPARSE>
int launch_part(PagedAttnArgs &a, const Launch &l, hipStream_t st)
{
    a.splits = l.splits;
    a.streams = l.streams;
    a.row_groups = l.row_groups;
    const int blocks = ceil_div(l.streams, 8) * 8 * l.row_groups;
    const Shape s = l.shape;
    if (s.qt == 0) {
        using List = PageList<64, 256, SPARSE>;
        a.list_size = SPARSE ? List::SCAN / a.splits + 2 : DENSE_LIST;
        const size_t lds = 16 * D + SINGLE_ROWS * a.words * 8 + DREAM_MAX_TREE * 4 + List::bytes(a.list_size, a.words);
        hipLaunchKernelGGL((paged_f32_kernel<D, SPARSE>), dim3(blocks), dim3(256), lds, st, a);
        return check_launch("paged_f32_kernel");
    }
    constexpr int WK = D == 256 ? 2 : 4;
    if (s.wr == 1 && s.qt == 1)
        return launch_bf16<D, 1, 1, WK, SPARSE>(a, blocks, st);
    if (s.wr == 1 && s.qt == 2)
        return launch_bf16<D, 2, 1, WK, SPARSE>(a, blocks, st);
    if constexpr (D == 256) {
        return launch_bf16<D, 1, 8, 1, SPARSE>(a, blocks, st);
    } else {
        if (s.wr == 1)
            return launch_bf16<D, 4, 1, WK, SPARSE>(a, blocks, st);
        return s.wr == 4 ? launch_bf16<D, 2, 4, 1, SPARSE>(a, blocks, st) : launch_bf16<D, 2, 8, 1, SPARSE>(a, blocks, st);
    }
}

template <int D, bool SPARSE>
int launch_all(PagedAttnArgs &a, const PagedPlan &p, bool f32, hipStream_t st)
{
    a.n_slots = p.n_slots;
    a.all_rows = p.all_rows;
    a.shared_slots = a.n_groups ? p.shared.splits : 0;
    if (!SPARSE && a.n_groups) {
        a.shared = 1;
        a.slot = 0;
        if (int rc = launch_part<D, false>(a, p.shared, st))
            return rc;
    }
    a.shared = 0;
    a.slot = a.shared_slots;
    if (int rc = launch_part<D, SPARSE>(a, p.own, st))
        return rc;
    if (p.n_slots == 1)
        return DREAM_OK;
    const int blocks = ceil_div(p.all_rows, 256 / (D / 4));
    if (f32)
        hipLaunchKernelGGL((paged_join_kernel<float, D>), dim3(blocks), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((paged_join_kernel<uint16_t, D>), dim3(blocks), dim3(256), 0, st, a);
    return check_launch("paged_join_kernel");
}

int check_attn(const char *who, const dream_attn_desc *d, const dream_page_desc *pages, int32_t n_tree, int32_t n_groups)
{
    if (int rc = check_pages(who, d, pages))
        return rc;
    if (n_tree < 1 || n_tree > DREAM_MAX_TREE || n_tree > paged_rows(pages))
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_tree %d outside [1, min(%d, max_pages * page_size)]", who, n_tree, DREAM_MAX_TREE);
    if ((int64_t)d->batch * d->n_q_heads > (1 << 20))
        return fail(DREAM_ERR_UNSUPPORTED, "%s: batch * n_q_heads exceeds 2^20", who);
    if (n_groups < 0 || n_groups > d->batch)
        return fail(DREAM_ERR_INVALID_ARG, "%s: %d groups of %d sequences", who, n_groups, d->batch);
    return DREAM_OK;
}

int run(const char *who, const dream_attn_desc *d, const dream_page_desc *pages, PagedAttnArgs &a, const PagedPlan &p, void *ws, size_t ws_bytes, void *stream)
{
    if (!a.q || !a.k || !a.v || !a.table || !a.prefix_len || (!a.parent && !a.tree_mask) || !a.out || !ws)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.out) | reinterpret_cast<uintptr_t>(ws)) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: a tensor is not 16-byte aligned", who);
    if (ws_bytes < p.bytes)
        return fail(DREAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, p.bytes);
    a.part_o = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float2 *>(a.part_o + (size_t)p.n_slots * p.all_rows * d->head_dim);
    a.batch = d->batch; a.hq = d->n_q_heads; a.hkv = d->n_kv_heads; a.group = a.hq / a.hkv; a.rows = a.n_tree * a.group; a.words = (a.n_tree + 63) / 64;
    a.lg_page = log2_of(pages->page_size); a.n_pages = pages->n_pages; a.max_pages = pages->max_pages;
    const float scale = d->scale != 0.0f ? d->scale : 1.0f / sqrtf((float)d->head_dim);
    a.scale_log2 = scale * 1.4426950408889634f;
    const bool f32 = d->dtype == DREAM_F32;
    hipStream_t st = as_stream(stream);
    if (a.nodes)
        return d->head_dim == 64 ? launch_all<64, true>(a, p, f32, st) : d->head_dim == 128 ? launch_all<128, true>(a, p, f32, st) : launch_all<256, true>(a, p, f32, st);
    return d->head_dim == 64 ? launch_all<64, false>(a, p, f32, st) : d->head_dim == 128 ? launch_all<128, false>(a, p, f32, st) : launch_all<256, false>(a, p, f32, st);
}

}  // namespace

extern "C" {

size_t dream_paged_verify_attn_workspace(const dream_attn_desc *desc, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len, int32_t n_groups, int64_t max_shared_len)
{
    if (check_attn("dream_paged_verify_attn_workspace", desc, pages, n_tree, n_groups))
        return DREAM_WORKSPACE_MIN_BYTES;
    const size_t n = plan_for(desc, pages, n_tree, max_kv_len, n_groups, max_shared_len, 0).bytes;
    return n < DREAM_WORKSPACE_MIN_BYTES ? DREAM_WORKSPACE_MIN_BYTES : n;
}

int dream_paged_verify_attn(const dream_attn_desc *desc, const dream_page_desc *pages, const void *q, const void *k_pages, const void *v_pages, const int32_t *page_table,
                            const int32_t *prefix_len, int32_t n_tree, const int32_t *parent, const uint64_t *tree_mask, int32_t n_groups, const int32_t *group_start,
                            const int32_t *shared_len, int64_t max_shared_len, int64_t max_kv_len, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "dream_paged_verify_attn";
    if (int rc = check_attn(who, desc, pages, n_tree, n_groups))
        return rc;
    if (n_groups && (!group_start || !shared_len))
        return fail(DREAM_ERR_INVALID_ARG, "%s: groups without group_start or shared_len", who);
    PagedAttnArgs a = {};
    a.q = static_cast<const unsigned char *>(q); a.k = static_cast<const unsigned char *>(k_pages); a.v = static_cast<const unsigned char *>(v_pages);
    a.table = page_table; a.prefix_len = prefix_len; a.n_tree = n_tree; a.parent = parent; a.tree_mask = tree_mask; a.n_groups = n_groups; a.group_start = group_start;
    a.shared_len = shared_len; a.out = out; a.lse = lse;
    return run(who, desc, pages, a, plan_for(desc, pages, n_tree, max_kv_len, n_groups, max_shared_len, 0), workspace, workspace_bytes, stream);
}

size_t dream_sparse_verify_attn_workspace(const dream_attn_desc *desc, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len, int32_t max_pages_seen)
{
    if (check_attn("dream_sparse_verify_attn_workspace", desc, pages, n_tree, 0))
        return DREAM_WORKSPACE_MIN_BYTES;
    const size_t n = plan_for(desc, pages, n_tree, max_kv_len, 0, 0, max_pages_seen).bytes;
    return n < DREAM_WORKSPACE_MIN_BYTES ? DREAM_WORKSPACE_MIN_BYTES : n;
}

int dream_sparse_verify_attn(const dream_attn_desc *desc, const dream_page_desc *pages, const void *q, const void *k_pages, const void *v_pages, const int32_t *page_table,
                             const uint64_t *page_nodes, const int32_t *prefix_len, int32_t n_tree, const int32_t *parent, const uint64_t *tree_mask, int64_t max_kv_len,
                             int32_t max_pages_seen, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "dream_sparse_verify_attn";
    if (int rc = check_attn(who, desc, pages, n_tree, 0))
        return rc;
    if (!page_nodes)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    PagedAttnArgs a = {};
    a.q = static_cast<const unsigned char *>(q); a.k = static_cast<const unsigned char *>(k_pages); a.v = static_cast<const unsigned char *>(v_pages);
    a.table = page_table; a.nodes = page_nodes; a.prefix_len = prefix_len; a.n_tree = n_tree; a.parent = parent; a.tree_mask = tree_mask; a.out = out; a.lse = lse;
    return run(who, desc, pages, a, plan_for(desc, pages, n_tree, max_kv_len, 0, 0, max_pages_seen), workspace, workspace_bytes, stream);
}

}  // extern "C"
