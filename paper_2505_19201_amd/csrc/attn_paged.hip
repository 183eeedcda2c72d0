// Tree-masked attention over caches held in pages (dream_paged_verify_attn), with a prefix that sequences share read once for all of them, and over pages that were selected for each node
// (dream_sparse_verify_attn).
//
// out_i = sum_j softmax_j(scale q_i k_j) v_j over the keys j that node i sees (Eq. 1 under the draft-tree mask of Section 3.1).  One pass over the keys with a running maximum and sum; a softmax
// over two sets of keys joins from (maximum, sum, weighted rows) of each, so the shared positions and a sequence's own are two sets: of the first, the rows of all sequences of a group
// that share a KV head are one long list of query rows over the first sequence's pages; of the second, every sequence has its own.  Each set is cut further where there are too few workgroups, and
// the parts are joined by a second kernel.
//
// A workgroup has QT tiles of 16 query rows in each of its waves, and takes keys and values tile by tile straight to LDS: 16 rows never leave a page, so that a tile's addresses are scalars, of which
// every lane holds those of one of the next 64 tiles.  (Selected pages stand in a list in LDS: the physical page, its place in the sequence, the nodes that see it.)  S^T = K Q^T and O^T += V^T P^T
// by v_mfma_f32_16x16x32_bf16: a lane owns a query row, its scores are the second product's operand as they come.  Two forms: paged_keys_kernel, few rows: the waves share the keys out and have stages
// of their own, so they meet only at the end; paged_rows_kernel, many rows: the waves share the tiles and have rows of their own, one barrier a tile.
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

// One of a launch's two kinds of workgroups: those of the shared positions, and those of what is a sequence's own.
struct Part {
    int32_t blocks, streams, row_groups, splits, slot;      // workgroups; units of a sequence or all groups, KV head and split; workgroups of a unit; its first slot
    uint32_t row_groups_magic, splits_magic;                // for divide()
};
struct PagedAttnArgs {
    const unsigned char *q, *k, *v;
    const int32_t *table, *prefix_len, *parent, *group_start, *shared_len;
    const uint64_t *tree_mask, *nodes;
    void *out;
    float *lse, *part_o;
    float2 *part_ml;
    int64_t all_rows;                     // rows of a slot of part_o
    int32_t batch, n_tree, words, hq, hkv, group, rows;      // rows: query rows of a sequence and KV head
    int32_t lg_page, n_pages, max_pages, n_groups, n_slots, shared_slots, list_size;
    float scale_log2;
    uint32_t hkv_magic, group_magic, rows_magic;
    Part shared, own;
};
// What stands ahead of a workgroup's first loads, as plain arguments of the kernels: those are in scalar registers when a wave starts, the structure is a trip to memory away.  Of the own part.
#define PLAIN const int32_t *table, const int32_t *prefix_len, int32_t max_pages, int32_t hkv, uint32_t hkv_magic, int32_t shared_blocks, int32_t row_groups, uint32_t row_groups_magic, int32_t splits, \
              uint32_t splits_magic, int32_t streams, int32_t lg_and_early

constexpr int PLAIN_BYTES = 2 * 8 + 10 * 4;      // of them, the structure lies behind
static_assert(PLAIN_BYTES % alignof(PagedAttnArgs) == 0);
// The structure once more, for what is at a kernel's end: what is used there alone is loaded there, instead of being held (and, where pages are listed, spilled) from the start on
__device__ __forceinline__ const PagedAttnArgs &args_again()
{
    typedef const __attribute__((address_space(4))) char *Arguments;
    Arguments p = (Arguments)__builtin_amdgcn_kernarg_segment_ptr() + PLAIN_BYTES;
    asm volatile("" : "+s"(p));
    return *(const PagedAttnArgs *)p;
}

// x / d by a multiplication, magic = (2^32 - 1) / d
__device__ __forceinline__ uint32_t divide(uint32_t x, uint32_t d, uint32_t magic)
{
    const uint32_t q = __umulhi(x, magic);
    return x - q * d >= d ? q + 1 : q;
}

// The same value, from which the compiler forms nothing ahead of the loop it stands in: the addresses of a step are a few instructions, and all of them kept are more registers than there are.
__device__ __forceinline__ int here(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ int here_scalar(int x)
{
    x = __builtin_amdgcn_readfirstlane(x);
    asm volatile("" : "+s"(x));
    return x;
}

// What a workgroup does.
struct Unit {
    bool shared, alone;                                 // alone: outside every group, where there are some
    int b, kvh, split, splits, slot, row0, n_rows;      // the sequence whose pages are read; its slot; rows are numbered through the sequences from b on
    uint32_t splits_magic;
    int lo, hi, P;                                      // positions [lo, hi), of which those from P on are the tree's
};

__device__ __forceinline__ int clamped_prefix(const PagedAttnArgs &a, int p) { return min(max(p, 0), (a.max_pages << a.lg_page) - a.n_tree); }

// How many positions sequence b shares; -1 outside every group.
__device__ __forceinline__ int shared_by(const PagedAttnArgs &a, int b, int lane)
{
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
        const int g = min(g0 + lane, a.n_groups - 1);
        const int s = a.group_start[g], e = a.group_start[g + 1], n = a.shared_len[g];
        const uint64_t mine = __ballot(s <= b && b < e);
        if (mine)
            return min(max(__builtin_amdgcn_readlane(n, __builtin_ctzll(mine)), 0), a.max_pages << a.lg_page);
    }
    return -1;
}

// The group whose query rows the t-th tile of `cap` rows of all groups has: its first sequence, sequences, shared positions, and the tile's first row; n = 0: there is no such tile.
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

// Workgroup ids that are congruent mod 8 run on one XCD: row groups that read the same keys meet in one L2.  What needs no load; false: there is no such unit.
__device__ __forceinline__ bool unit_at(const PagedAttnArgs &a, int hkv, uint32_t hkv_magic, uint32_t shared_blocks, uint32_t row_groups, uint32_t row_groups_magic, uint32_t splits,
                                        uint32_t splits_magic, uint32_t streams, int cap, Unit &u, int &rg)
{
    uint32_t block = blockIdx.x;
    u.shared = block < shared_blocks;
    if (u.shared) {
        row_groups = a.shared.row_groups;
        row_groups_magic = a.shared.row_groups_magic;
        splits = a.shared.splits;
        splits_magic = a.shared.splits_magic;
        streams = a.shared.streams;
    } else {
        block -= shared_blocks;
    }
    const uint32_t at = block >> 3, slot = divide(at, row_groups, row_groups_magic), stream = slot * 8 + (block & 7);
    rg = at - slot * row_groups;
    const uint32_t head = divide(stream, splits, splits_magic), b = divide(head, hkv, hkv_magic);      // (shared: b is 0)
    u.splits = splits;
    u.splits_magic = splits_magic;
    u.split = stream - head * splits;
    u.kvh = head - b * hkv;
    u.b = b;
    u.row0 = rg * cap;
    u.lo = 0;
    u.alone = false;
    return stream < streams;
}
#define UNIT_AT(args, cap) unit_at(args, hkv, hkv_magic, shared_blocks, row_groups, row_groups_magic, splits, splits_magic, streams, cap, u, rg)
// And what does: the prefix length (asked for by the caller), the groups
__device__ __forceinline__ bool unit_of(const PagedAttnArgs &a, int cap, int lane, int rg, int prefix, Unit &u)
{
    u.slot = (u.shared ? a.shared.slot : a.own.slot) + u.split;
    u.n_rows = a.rows;
    if (u.shared) {
        int n, shared;
        group_of_tile(a, rg, cap, lane, u.b, n, shared, u.row0);
        u.n_rows = n * a.rows;
        u.hi = u.P = shared;
        return n > 0;
    }
    u.P = clamped_prefix(a, prefix);
    u.hi = u.P + a.n_tree;
    if (a.n_groups) {
        const int shared = shared_by(a, u.b, lane);
        u.alone = shared < 0;
        u.lo = min(max(shared, 0), u.P);
    }
    return true;
}

// ---- selected pages --------------------------------------------------------------------------------------------------
constexpr int SPARSE_LIST = 1024;              // entries of a list (trees of up to 64 nodes; others half of that)
constexpr uint32_t TREE_PAGE = 1u << 31;      // of an entry of `logical`: the tree's rows in it are meant, otherwise the prefix's

// The pages of a sequence that some node of the workgroup's rows sees, and those of the tree: of them, by their rank, every splits-th, in LDS, `list_size` of them from the `skip`-th of these on.  Rows of the list are numbered through its pages.
template <int THREADS>
struct PageList {
    static constexpr int EACH = THREADS == 512 ? 2 : 4, SCAN = EACH * THREADS;      // pages looked at at a time: by a thread; by all
    int32_t *phys;
    uint32_t *logical;
    uint64_t *word;
    int n, all;                     // entries; this split's pages
    int32_t id[EACH + 1];           // of a thread's pages, one in front of them first; which nodes see them (trees of one word)
    uint64_t seen[EACH];

    // Of the thread's pages from `first` on: needs no length, so the first are asked for with it
    __device__ __forceinline__ void ask(const PagedAttnArgs &a, const Unit &u, int first)
    {
        const int32_t *table = a.table + (int64_t)u.b * a.max_pages;
        const uint64_t *nodes = a.nodes + ((int64_t)u.b * a.hkv + u.kvh) * a.max_pages * a.words;
#pragma unroll
        for (int i = 0; i <= EACH; i++)
            id[i] = table[min(max(first + i - 1, 0), a.max_pages - 1)];
        if (a.words == 1)
#pragma unroll
            for (int i = 0; i < EACH; i++)
                seen[i] = nodes[min(first + i, a.max_pages - 1)];
    }
    // By all threads, each of which has asked for its first pages; starts and ends with a barrier.
    __device__ __forceinline__ void build(const PagedAttnArgs &a, const Unit &u, int cap, int tid, unsigned char *smem, int skip)
    {
        phys = reinterpret_cast<int32_t *>(smem);
        logical = reinterpret_cast<uint32_t *>(smem + 4 * a.list_size);
        word = reinterpret_cast<uint64_t *>(smem + 8 * a.list_size);
        int32_t *counts = reinterpret_cast<int32_t *>(smem + (8 + 8 * a.words) * a.list_size);
        const int in_prefix = (u.P + (1 << a.lg_page) - 1) >> a.lg_page, tree_page = u.P >> a.lg_page;
        const int total = in_prefix + ((u.hi - 1) >> a.lg_page) - tree_page + 1;
        const int lane = tid & 63, wave = tid >> 6;
        const uint64_t *nodes = a.nodes + ((int64_t)u.b * a.hkv + u.kvh) * a.max_pages * a.words;
        const int node0 = (uint32_t)u.row0 / (uint32_t)a.group, node1 = (uint32_t)(min(u.row0 + cap, u.n_rows) - 1) / (uint32_t)a.group;
        auto ours = [&](int w) {      // of word w
            const int lo = max(node0 - 64 * w, 0), hi = min(node1 - 64 * w, 63);
            return lo > hi ? 0ull : ~0ull >> (63 - hi) & ~0ull << lo;
        };
        auto upto = [&](int r) { return r > u.split ? (int)divide(r - u.split + u.splits - 1, u.splits, u.splits_magic) : 0; };      // this split's among the first r
        int rank = 0;
        for (int scanned = 0; scanned < total; scanned += SCAN) {
            __syncthreads();
            int taken = 0;
            uint32_t mine = 0;
            const int v0 = scanned + tid * EACH;
            if (scanned)
                ask(a, u, v0);
#pragma unroll
            for (int i = 0; i < EACH; i++) {
                bool in = v0 + i >= in_prefix && v0 + i < total;
                if (a.words == 1)
                    in = in || (v0 + i < in_prefix && (seen[i] & ours(0)) != 0ull);
                else if (v0 + i < in_prefix)
                    for (int w = 0; w < a.words; w++)
                        in = in || (nodes[(int64_t)(v0 + i) * a.words + w] & ours(w)) != 0ull;
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
            int r = rank + sum - taken;
#pragma unroll
            for (int w = 0; w < THREADS / 64; w++) {
                const int x = counts[w];
                r += w < wave ? x : 0;
                rank += x;
            }
#pragma unroll
            for (int i = 0; i < EACH; i++) {
                const int at = upto(r) - skip;
                if ((mine >> i & 1) && at * u.splits + skip * u.splits + u.split == r && at >= 0 && at < a.list_size) {
                    const int v = v0 + i;
                    const bool prefix = v < in_prefix, in_front = !prefix && tree_page < in_prefix;      // (the tree begins in the prefix's last page)
                    phys[at] = min(max(in_front ? id[i] : id[i + 1], 0), a.n_pages - 1);
                    logical[at] = (uint32_t)(prefix ? v : tree_page + v - in_prefix) | (prefix ? 0u : TREE_PAGE);
                    if (a.words == 1)
                        word[at] = prefix ? seen[i] : 0ull;
                    else
                        for (int w = 0; w < a.words; w++)
                            word[at * a.words + w] = prefix ? nodes[(int64_t)v * a.words + w] : 0ull;
                }
                r += mine >> i & 1;
            }
        }
        all = __builtin_amdgcn_readfirstlane(upto(rank));
        n = min(max(all - skip, 0), a.list_size);
        __syncthreads();
    }
    static size_t bytes(int list_size, int words) { return (size_t)list_size * (8 + 8 * words) + 64; }
};

// Where 16 rows stand that are taken together (the same in every lane).
struct Chunk {
    int entry;                      // of the list
    int pos;                        // position of the first row
    bool live, tree, prefix;        // there are such rows; those that are meant: the tree's, the prefix's
};
// Row x of a list
template <class List>
__device__ __forceinline__ Chunk listed_chunk(const PagedAttnArgs &a, const List &list, int x)
{
    Chunk c;
    const int e = x >> a.lg_page;
    c.live = e < list.n;
    c.entry = min(e, list.n - 1);
    const uint32_t l = __builtin_amdgcn_readfirstlane((int)list.logical[c.entry]);
    c.tree = l >> 31;
    c.prefix = !c.tree;
    c.pos = (int)((l & ~TREE_PAGE) << a.lg_page) + (x & ((1 << a.lg_page) - 1));
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
    if (u.shared) {
        const int s = divide(j, a.rows, a.rows_magic);
        w.b += s;
        w.r = j - s * a.rows;
    }
    w.node = divide(w.r, a.group, a.group_magic);
    w.head = u.kvh * a.group + w.r - w.node * a.group;
    return w;
}
__device__ __forceinline__ int64_t row_of_q(const PagedAttnArgs &a, const Row &w) { return ((int64_t)w.b * a.n_tree + w.node) * a.hq + w.head; }
__device__ __forceinline__ int64_t row_of_part(const PagedAttnArgs &a, const Unit &u, const Row &w) { return (int64_t)u.slot * a.all_rows + ((int64_t)w.b * a.hkv + u.kvh) * a.rows + w.r; }
// Prefix positions below this are the row's
__device__ __forceinline__ int row_limit(const PagedAttnArgs &a, const Unit &u, const Row &w) { return u.shared ? min(u.hi, clamped_prefix(a, a.prefix_len[w.b])) : u.P; }

// part: in its part's slot, not as the row's own
__device__ __forceinline__ void put_ml(const PagedAttnArgs &a, const Unit &u, const Row &w, float m, float l, bool part)
{
    if (part)
        a.part_ml[row_of_part(a, u, w)] = make_float2(m, l);
    else if (a.lse)
        a.lse[((int64_t)w.b * a.hq + w.head) * a.n_tree + w.node] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * 0.6931471805599453f;
}
// A row's reference and sum so far, and what those and the sums of its channels are to be multiplied with, where a list is not the first of its workgroup: what the lists in front of it gave stands in the
// part's slot.  By all lanes of the row; what one of them writes there afterwards comes after all have read it (they are lanes of one wave).
struct Earlier {
    float old, now;                     // factors of what the slot holds, and of this list's
    __device__ __forceinline__ void join(const PagedAttnArgs &a, const Unit &u, const Row &w, float &m, float &l)
    {
        const float2 ml = a.part_ml[row_of_part(a, u, w)];
        const float top = fmaxf(ml.x, m);
        old = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);
        now = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        l = __builtin_fmaf(ml.y, old, l * now);
        m = top;
    }
};
// The rows of a sequence outside every group have empty shared parts
__device__ __forceinline__ void no_shared_parts(const PagedAttnArgs &a, const Unit &u, int cap, int tid, int threads)
{
    if (u.split == 0)
        for (int j = u.row0 + tid; j < min(u.row0 + cap, u.n_rows); j += threads)
            for (int s = 0; s < a.shared_slots; s++)
                a.part_ml[(int64_t)s * a.all_rows + ((int64_t)u.b * a.hkv + u.kvh) * a.rows + j] = make_float2(-INFINITY, 0.0f);
}
__device__ __forceinline__ uint32_t pack_bf16(float x, float y)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
}

// Which nodes of the tree each of the workgroup's rows sees, `words` words a row in LDS; by all threads, ends with a barrier.  parents: n_tree words of LDS.
__device__ __forceinline__ void build_masks(const PagedAttnArgs &a, const Unit &u, uint64_t *masks, int32_t *parents, int cap, int tid, int threads)
{
    if (!a.tree_mask) {
        for (int i = tid; i < a.n_tree; i += threads)
            parents[i] = a.parent[(int64_t)u.b * a.n_tree + i];
        __syncthreads();
    }
    const uint64_t last = a.n_tree & 63 ? (1ull << (a.n_tree & 63)) - 1 : ~0ull;
    for (int j = tid; j < cap; j += threads) {
        if (u.row0 + j >= u.n_rows) {      // (no such row: it sees no node, so that its sums stay finite)
            for (int w = 0; w < a.words; w++)
                masks[j * a.words + w] = 0ull;
            continue;
        }
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
// Trees of up to 64 nodes: lane l gets node l's mask.  parent: of this lane's node.  The paths are joined by halves: a node's mask holds its path in front of `up`, and takes in what `up` has found.
__device__ __forceinline__ uint64_t small_tree(int lane, int n_tree, int parent)
{
    uint32_t lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
    int up = lane < n_tree && parent < lane ? parent : -1;      // (a parent that does not precede its node is none)
    while (__any(up >= 0)) {
        const int from = max(up, 0);
        const uint32_t l = __shfl(lo, from), h = __shfl(hi, from);
        const int next = __shfl(up, from);
        if (up >= 0) {
            lo |= l;
            hi |= h;
            up = next;
        }
    }
    return (uint64_t)hi << 32 | lo;
}
// Of the nodes n0 .. n0 + 3 (n0 may be negative) those that a row's mask has, as four bits: the mask of a small tree, or that in LDS
__device__ __forceinline__ uint32_t four_nodes(const PagedAttnArgs &a, uint64_t small, const uint64_t *mask, int n0)
{
    if (n0 <= -4 || n0 >= a.n_tree)
        return 0u;
    if (a.words > 1) {
        if (n0 < 0)
            return (uint32_t)(mask[0] << -n0) & 15u;
        const int w = n0 >> 6, s = n0 & 63;
        uint64_t x = mask[w] >> s;
        if (s > 60 && w + 1 < a.words)
            x |= mask[w + 1] << (64 - s);
        return (uint32_t)x & 15u;
    }
    return (uint32_t)(n0 < 0 ? small << -n0 : small >> n0) & 15u;
}

// ---- row by row ------------------------------------------------------------------------------------------------------
// The sum over groups of N lanes (8 to 64), in all of them: neighbours, pairs, halves of a row of sixteen turned round, rows
template <int CTRL>
__device__ __forceinline__ float from_lane(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true)); }
template <int N>
__device__ __forceinline__ float lanes_sum(float x)
{
    x += from_lane<0xb1>(x);              // quad_perm [1, 0, 3, 2]
    x += from_lane<0x4e>(x);              // quad_perm [2, 3, 0, 1]
    x += from_lane<0x141>(x);             // row_half_mirror
    if constexpr (N > 8)
        x += from_lane<0x140>(x);         // row_mirror
    if constexpr (N > 16)
        x += __shfl_xor(x, 16);
    if constexpr (N > 32)
        x += __shfl_xor(x, 32);
    return x;
}
// LDS of attend_rows_singly: masks, parents, the list
int single_bytes(int cap, int words) { return cap * words * 8 + DREAM_MAX_TREE * 4; }

// The workgroup's rows, one to a wave at a time.  64 keys: each lane looks one up, then 16 bytes of a row are a lane's, so that a wave reads several whole rows at a time; keys and values are asked for
// together.  What the node does not see has no weight, whatever it holds.  Where the keys are shared out, a workgroup has every splits-th run of `run` keys from the tile of `tile` keys on that holds
// the first.  (A lane with a key's whole product, and values key by key: 60 nodes x 764 keys x 32 heads of 128 in
// float32 146 us, so 78; 21 nodes x 121 keys x 4 heads of 64 13.0 and 8.0.  A step of 64 keys takes 1.7 us at 64, 4 at 128.)
template <class T, int D, int THREADS, bool SPARSE>
__device__ __forceinline__ void attend_rows_singly(const PagedAttnArgs &a, const Unit &u, int cap, int tile, int run, unsigned char *smem)
{
    constexpr int NW = THREADS / 64, N = 16 / sizeof(T), LANES = D / N, G = 64 / LANES;      // values of a lane; lanes of a row; rows that a wave reads at a time
    constexpr int MOST = std::is_same_v<T, float> ? 16 : 4, BATCH = MOST < LANES ? MOST : LANES;
    const int tid = here(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), piece = lane % LANES, in_group = lane / LANES;
    const int count = min(cap, u.n_rows - u.row0), ps_mask = (1 << a.lg_page) - 1;
    uint64_t *masks = reinterpret_cast<uint64_t *>(smem);
    int32_t *parents = reinterpret_cast<int32_t *>(masks + cap * a.words);
    PageList<THREADS> list;
    const int32_t *table = a.table + (int64_t)u.b * a.max_pages;
    auto value = [](const u32x4 &raw, int i) {
        if constexpr (std::is_same_v<T, float>)
            return __uint_as_float(raw[i]);
        else
            return __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
    };
    if (!u.shared)
        build_masks(a, u, masks, parents, cap, tid, THREADS);
    for (int j0 = 0; j0 < count; j0 += NW) {
        const bool mine = j0 + wave < count;
        const int j = min(j0 + wave, count - 1);
        const Row w = row_at(a, u, u.row0 + j);
        const int limit = row_limit(a, u, w);
        const u32x4 q = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const T *>(a.q) + row_of_q(a, w) * D + piece * N);
        float m = -INFINITY, l = 0.0f, o[N];      // (the lanes of a row hold the same)
#pragma unroll
        for (int i = 0; i < N; i++)
            o[i] = 0.0f;
        // 64 keys: this lane's row of the page and where it stands; `kind`: which of them are meant (1: the prefix's, 2: the tree's)
        auto keys = [&](bool there, int page, int pos, int kind, const uint64_t *word) {
            const int node = pos - u.P;
            const bool in_prefix = (kind & 1) && pos >= u.lo && pos < limit && (!SPARSE || (word[w.node >> 6] >> (w.node & 63) & 1));
            const bool in_tree = (kind & 2) && !u.shared && node >= 0 && node < a.n_tree && (masks[j * a.words + (node >> 6)] >> (node & 63) & 1);
            const uint64_t seen = __ballot(there && (in_prefix || in_tree));
            const uint32_t row = (((uint32_t)page * a.hkv + u.kvh) << a.lg_page) + (pos & ps_mask);      // (of the pool; 2^32 of the shortest rows are 512 GB)
#pragma unroll 1
            for (int k0 = 0; k0 < 64; k0 += BATCH * G) {
                if (!(seen >> k0 & (BATCH * G == 64 ? ~0ull : (1ull << (BATCH * G & 63)) - 1)))
                    continue;
                u32x4 k[BATCH], v[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; i++) {
                    const int key = k0 + i * G + in_group;
                    const int64_t of = (int64_t)(uint32_t)__shfl((int)row, key) * D + piece * N;
                    k[i] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const T *>(a.k) + of);
                    v[i] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const T *>(a.v) + of);
                }
                if constexpr (BATCH * G < 64)
                    __builtin_amdgcn_sched_barrier(0);      // all are asked for before the first is looked at: 900 keys of 128 float32 94 -> 63 us; of 64, where they are all 64 keys, 30 -> 33
                float s[BATCH], top = m;
#pragma unroll
                for (int i = 0; i < BATCH; i++) {
                    float x = 0.0f;
#pragma unroll
                    for (int e = 0; e < N; e++)
                        x = __builtin_fmaf(value(k[i], e), value(q, e), x);
                    x = lanes_sum<LANES>(x);
                    s[i] = seen >> (k0 + i * G + in_group) & 1 ? x * a.scale_log2 : -INFINITY;
                    top = fmaxf(top, s[i]);
                }
#pragma unroll
                for (int d = LANES; d < 64; d *= 2)
                    top = fmaxf(top, __shfl_xor(top, d));
                const float f = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top), ref = fmaxf(top, -FLT_MAX);
                m = top;
                l *= f;
#pragma unroll
                for (int e = 0; e < N; e++)
                    o[e] *= f;
#pragma unroll
                for (int i = 0; i < BATCH; i++) {
                    const float p = seen >> (k0 + i * G + in_group) & 1 ? __builtin_amdgcn_exp2f(s[i] - ref) : 0.0f;
                    l += p;
#pragma unroll
                    for (int e = 0; e < N; e++)      // (a key of weight 0 through a score of -inf adds nothing, whatever its values)
                        o[e] = s[i] == -INFINITY ? o[e] : __builtin_fmaf(p, value(v[i], e), o[e]);
                }
            }
        };
        if constexpr (SPARSE) {
            int skip = 0;
            do {
                list.ask(a, u, tid * list.EACH);
                list.build(a, u, cap, tid, reinterpret_cast<unsigned char *>(parents + DREAM_MAX_TREE), skip);
                for (int x0 = 0; x0 < list.n << a.lg_page; x0 += 64) {
                    const int e = min((x0 + lane) >> a.lg_page, list.n - 1);
                    const uint32_t entry = list.logical[e];
                    keys(x0 + lane < list.n << a.lg_page, list.phys[e], (int)((entry & ~TREE_PAGE) << a.lg_page) + ((x0 + lane) & ps_mask), entry >> 31 ? 2 : 1, list.word + e * a.words);
                }
                skip += a.list_size;
            } while (skip < list.all);
        } else {
            // the pages of the keys that come next are asked for ahead of these
            auto page_of = [&](int x0) { return table[min(x0 + lane, u.hi - 1) >> a.lg_page]; };
            int start = u.lo / tile * tile + u.split * run, x0 = start, page = start < u.hi ? page_of(x0) : 0;
            while (start < u.hi) {
                const int end = min(start + run, u.hi), now = x0, id = page;
                x0 += 64;
                if (x0 >= end) {
                    start += u.splits * run;
                    x0 = start;
                }
                if (start < u.hi)
                    page = page_of(x0);
                keys(now + lane < end, min(max(id, 0), a.n_pages - 1), now + lane, 3, nullptr);
            }
        }
#pragma unroll
        for (int d = LANES; d < 64; d *= 2) {
            l += __shfl_xor(l, d);
#pragma unroll
            for (int e = 0; e < N; e++)
                o[e] += __shfl_xor(o[e], d);
        }
        if (!mine || in_group)
            continue;
        if (lane == 0)
            put_ml(a, u, w, m, l, a.n_slots > 1);
        if (a.n_slots > 1 || std::is_same_v<T, float>) {
            float *to = (a.n_slots > 1 ? a.part_o + row_of_part(a, u, w) * D : static_cast<float *>(a.out) + row_of_q(a, w) * D) + piece * N;
            const float divisor = a.n_slots > 1 ? 1.0f : l;
#pragma unroll
            for (int e = 0; e < N; e += 4)
                *reinterpret_cast<f32x4 *>(to + e) = l == 0.0f ? f32x4{0.f, 0.f, 0.f, 0.f} : f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]} / divisor;
        } else {
            u32x4 row = {0u, 0u, 0u, 0u};
            if (l != 0.0f)
#pragma unroll
                for (int e = 0; e < N; e += 2)
                    row[e / 2] = pack_bf16(o[e] / l, o[e + 1] / l);
            *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(a.out) + row_of_q(a, w) * D + piece * N) = row;
        }
    }
}

// float32: there for its precision and for small shapes.
constexpr int SINGLE_ROWS = 4, SINGLE_RUN = 64;
template <int D, bool SPARSE>
__global__ __launch_bounds__(256) void paged_f32_kernel(PLAIN, PagedAttnArgs a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    Unit u;
    int rg;
    if (!UNIT_AT(a, SINGLE_ROWS))
        return;
    const int prefix = u.shared ? 0 : uniform_load(prefix_len + u.b);
    if (!unit_of(a, SINGLE_ROWS, threadIdx.x & 63, rg, prefix, u))
        return;
    if (u.alone)
        no_shared_parts(a, u, SINGLE_ROWS, threadIdx.x, 256);
    attend_rows_singly<float, D, 256, SPARSE>(a, u, SINGLE_ROWS, SINGLE_RUN, SINGLE_RUN, smem);
}

// ---- bf16 ------------------------------------------------------------------------------------------------------------
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ float largest(f32x4 a) { return fmaxf(fmaxf(fmaxf(a[0], a[1]), a[2]), a[3]); }

// The query rows of a wave, QT tiles of 16, and their sums.  Lane (c, g) = (lane % 16, lane / 16) has of row c: of the queries the channels 8 g .. of every 32; of O^T the channels
// 16 dt + 4 g + r; and scores of the keys 4 g + r of every 16.  A step takes NC chunks of 16 keys.
//
// A weight goes into the second product as PIECES bf16 numbers, its value rounded and what that leaves: with two of them what is lost is 2^-16 of it, with one 2^-8, as much as the row's own rounding
// (against 64 bits rows are off by 0.0017 and by 0.0023 of their size, root mean square).  Two where that costs little: bf16 weights in one part and in two, us a layer,
//   keys, 128: one sequence, 60 nodes x 764 keys 12.2 and 12.4; 8 sequences, one node x 16 100 keys 86.1 and 86.1
//   rows, 256: 16 sequences, one node x 8011 shared keys 31.2 and 31.7; selected pages, 4 x 33 nodes 66.9 and 70.0 (attention 44 of them); 16 x 60 nodes x 2000 keys 72.8 and 78.0
//   rows, 128: 64 rows a workgroup, 8 x 60 nodes x 1343 keys 30.8 and 35.5, selected pages 88.0 and 95.7; 128 rows, 8 x 60 nodes x 4096 shared keys 60.8 and 90.3 (the registers do not hold both)
//   rows, 64: 32 x 33 nodes x 1600 shared keys 45.3 and 53.5; so one in the rows kernel below 256
template <int D, int QT, int NC, bool SPARSE, int PIECES>
struct QueryRows {
    static constexpr int ROW = 2 * D, NKS = D / 32, NDT = D / 16;
    typedef bf16x8 Weights[PIECES][NC / 2][QT];
    bf16x8 qf[QT][NKS];
    f32x4 o[QT][NDT];
    float m[QT], l[QT];
    int limit[QT], node[QT];
    uint64_t small[QT];                           // what a row sees of a tree of up to 64 nodes
    const uint64_t *large;                        // of a larger one: in LDS, row c's of tile 0
    int whole;                                    // prefix positions below it are everyone's

    __device__ __forceinline__ void load(const PagedAttnArgs &a, const Unit &u, int first, int c, int g)
    {
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const Row w = row_at(a, u, min(first + qt * 16 + c, u.n_rows - 1));
            const unsigned char *q = a.q + row_of_q(a, w) * ROW + g * 16;
#pragma unroll
            for (int ks = 0; ks < NKS; ks++)
                qf[qt][ks] = *reinterpret_cast<const bf16x8 *>(q + ks * 64);
            node[qt] = w.node;
            limit[qt] = u.shared ? a.prefix_len[w.b] : 0;
            m[qt] = -INFINITY;
            l[qt] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < NDT; dt++)
                o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // parent: of the lane's node of a small tree; tid, threads, masks, parents: for a large one
    __device__ __forceinline__ void see(const PagedAttnArgs &a, const Unit &u, int first, int cap, int parent, int c, int tid, int threads, uint64_t *masks, int32_t *parents, int in_group)
    {
        whole = u.P;
        if (u.shared) {
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                limit[qt] = min(u.hi, clamped_prefix(a, limit[qt]));
                whole = min(whole, limit[qt]);
                small[qt] = 0ull;
            }
#pragma unroll
            for (int s = 1; s < 16; s *= 2)
                whole = min(whole, __shfl_xor(whole, s));
            whole = __builtin_amdgcn_readfirstlane(whole);
            return;
        }
        const uint64_t tree = a.words > 1 || a.tree_mask ? 0ull : small_tree(tid & 63, a.n_tree, parent);
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            limit[qt] = u.P;
            small[qt] = 0ull;
            if (a.words > 1)
                continue;
            if (a.tree_mask)
                small[qt] = a.tree_mask[(int64_t)u.b * a.n_tree + node[qt]] & (a.n_tree & 63 ? (1ull << (a.n_tree & 63)) - 1 : ~0ull);
            else
                small[qt] = (uint64_t)(uint32_t)__shfl((int)(tree >> 32), node[qt]) << 32 | (uint32_t)__shfl((int)tree, node[qt]);
            if (first + qt * 16 + c >= u.n_rows)
                small[qt] = 0ull;
        }
        if (a.words > 1) {
            build_masks(a, u, masks, parents, cap, tid, threads);
            large = masks + (in_group + c) * a.words;
        }
    }

    // S^T = K Q^T of chunks h0 and h0 + 1
    __device__ __forceinline__ void scores(const unsigned char *kt, int foff, int h0, f32x4 (&s)[NC][QT]) const
    {
        bf16x8 kf[NKS][2];
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
#pragma unroll
            for (int h = 0; h < 2; h++)
                kf[ks][h] = *reinterpret_cast<const bf16x8 *>(kt + (h0 + h) * 16 * ROW + at_key_step(foff, ks));
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                s[h0 + h][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < NKS; ks++)
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    s[h0 + h][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks][h], qf[qt][ks], s[h0 + h][qt], 0, 0, 0);
    }
    // All rows of the chunk are everyone's (or everyone's whose page it is)
    __device__ __forceinline__ bool plain(const Unit &u, const Chunk &c) const { return c.live && c.prefix && c.pos >= u.lo && c.pos + 16 <= whole; }

    // Of a step that is not everyone's: scores as multiples of an octave, -inf for what a row does not see.  Bit h * QT + qt of `in`: does the row see chunk h's page (selected pages).
    __device__ __forceinline__ void mask(const PagedAttnArgs &a, const Unit &u, const Chunk (&ch)[NC], uint32_t in, int g, f32x4 (&s)[NC][QT]) const
    {
#pragma unroll
        for (int qt = 0; qt < QT; qt++)
#pragma unroll
            for (int h = 0; h < NC; h++) {
                const int pos = ch[h].pos + 4 * g;
                uint32_t vis = 0u;
                if (ch[h].live && ch[h].prefix && (!SPARSE || (in >> (h * QT + qt) & 1u))) {
#pragma unroll
                    for (int r = 0; r < 4; r++)
                        vis |= (uint32_t)(pos + r >= u.lo && pos + r < limit[qt]) << r;
                }
                if (ch[h].live && ch[h].tree && !u.shared)
                    vis |= four_nodes(a, small[qt], large + qt * 16 * a.words, pos - u.P);
#pragma unroll
                for (int r = 0; r < 4; r++)
                    s[h][qt][r] = vis >> r & 1u ? s[h][qt][r] * a.scale_log2 : -INFINITY;
            }
    }
    // Online softmax of a step, first half: the references where its scores (times `scaled` octaves) exceed them.  (What masked steps and others do apart is mask() alone: values that may have come
    // by two ways would be held twice.)
    __device__ __forceinline__ void raise(float scaled, uint32_t in, const f32x4 (&s)[NC][QT])
    {
        float top[QT];
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            top[qt] = -INFINITY;
#pragma unroll
            for (int h = 0; h < NC; h++) {
                const float x = largest(s[h][qt]);
                top[qt] = fmaxf(top[qt], SPARSE && !(in >> (h * QT + qt) & 1u) ? -INFINITY : x);
            }
            top[qt] *= scaled;
        }
        bool above = false;
#pragma unroll
        for (int qt = 0; qt < QT; qt++)
            above = above || top[qt] > m[qt] + SLACK;
        if (__any(above)) {      // (no branch of its own for a lane, for the same reason)
#pragma unroll
            for (int qt = 0; qt < QT; qt++) {
                float x = fmaxf(top[qt], __shfl_xor(top[qt], 16));
                x = fmaxf(x, __shfl_xor(x, 32));
                const bool up = x > m[qt] + SLACK;
                const float f = up ? __builtin_amdgcn_exp2f(m[qt] - x) : 1.0f;       // 0 where nothing was seen before
                m[qt] = up ? x : m[qt];
                l[qt] *= f;
#pragma unroll
                for (int dt = 0; dt < NDT; dt++)
                    o[qt][dt] *= f;
            }
        }
    }
    // Second half: the weights of slice i (query tile i % QT, chunk i / QT), and their sum
    __device__ __forceinline__ void weigh(float scaled, uint32_t in, int i, const f32x4 (&s)[NC][QT], Weights &pf)
    {
        const int qt = i % QT, h = i / QT;
        const float ref = fmaxf(m[qt], -FLT_MAX);      // where all scores so far are -inf, their weight is 0 and not exp(-inf + inf)
        const bool out = SPARSE && !(in >> (h * QT + qt) & 1u);
        const float mult = out ? 0.0f : scaled, less = out ? -INFINITY : -ref;
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; r++) {
            p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[h][qt][r], mult, less));
            pf[0][h / 2][qt][h % 2 * 4 + r] = (__bf16)p[r];      // (the sum stays float32, of the weights as they were)
            if constexpr (PIECES > 1)
                pf[1][h / 2][qt][h % 2 * 4 + r] = (__bf16)(p[r] - (float)(__bf16)p[r]);
        }
        l[qt] += (p[0] + p[1]) + (p[2] + p[3]);
    }
    static constexpr int SLICES = NC * QT, STEPS = NC / 2 * NKS;
    // The scores of the next step, and meanwhile this one's weights: every STEPS-th part of the products (two chunks, 32 channels) is followed by its part of the weights, and its keys are asked
    // for two parts ahead.  (Left to itself the compiler asks for them when it needs them: 1621 clocks for a tile of 64 keys and 32 rows of 128; 512 of matrix products.)
    __device__ __forceinline__ void scores_and_weights(const unsigned char *kt, int foff, f32x4 (&next)[NC][QT], float scaled, uint32_t in, const f32x4 (&s)[NC][QT], Weights &pf)
    {
        constexpr int AHEAD = STEPS < 2 ? STEPS : 2;
        bf16x8 kf[AHEAD + 1][2];
        auto ask = [&](int i) {
#pragma unroll
            for (int h = 0; h < 2; h++)
                kf[i % (AHEAD + 1)][h] = *reinterpret_cast<const bf16x8 *>(kt + (i / NKS * 2 + h) * 16 * ROW + at_key_step(foff, i % NKS));
        };
#pragma unroll
        for (int i = 0; i < AHEAD; i++)
            ask(i);
#pragma unroll
        for (int h = 0; h < NC; h++)
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                next[h][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < STEPS; i++) {
            if (i + AHEAD < STEPS)
                ask(i + AHEAD);
#pragma unroll
            for (int j = i * SLICES / STEPS; j < (i + 1) * SLICES / STEPS; j++)
                weigh(scaled, in, j, s, pf);
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    next[i / NKS * 2 + h][qt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i % (AHEAD + 1)][h], qf[qt][i % NKS], next[i / NKS * 2 + h][qt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // O^T += V^T P^T; values are asked for two parts (16 channels of 32 keys) ahead of their products
    __device__ __forceinline__ void add_values(const unsigned char *vt, int voff, const Weights &pf)
    {
        constexpr int PARTS = NC / 2 * NDT, AHEAD = 4;
        bf16x8 vf[AHEAD + 1];
        auto ask = [&](int i) {
            const unsigned char *vp = vt + i / NDT * 32 * ROW + at_column_tile(voff, i % NDT);
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)vp);
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(vp + 16 * ROW));
            vf[i % (AHEAD + 1)] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        };
#pragma unroll
        for (int i = 0; i < AHEAD; i++)
            ask(i);
#pragma unroll
        for (int i = 0; i < PARTS; i++) {
            if (i + AHEAD < PARTS)
                ask(i + AHEAD);
#pragma unroll
            for (int part = 0; part < PIECES; part++)
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    o[qt][i % NDT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i % (AHEAD + 1)], pf[part][i / NDT][qt], o[qt][i % NDT], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // The rows' sums over all four g; true where one is not finite
    __device__ __forceinline__ bool finish()
    {
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
        return __any(strange != 0.0f);      // (0 * inf and 0 * NaN are NaN)
    }
    // Chunks of a list from row x on: which of their pages the rows see, and are they everyone's (whose page it is); false where no row sees any
    template <class List>
    __device__ __forceinline__ bool seen_by(const PagedAttnArgs &a, const Unit &u, const List &list, int x, bool &straight, uint32_t &in) const
    {
        auto look = [&](int h, uint32_t &bits) {
            const Chunk c = listed_chunk(a, list, x + h * 16);
            bits = 0u;
            if (a.words == 1) {
                const uint64_t word = list.word[c.entry];
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    bits |= (uint32_t)(word >> node[qt] & 1) << qt;
            } else {
#pragma unroll
                for (int qt = 0; qt < QT; qt++)
                    bits |= (uint32_t)(list.word[c.entry * a.words + (node[qt] >> 6)] >> (node[qt] & 63) & 1) << qt;
            }
            return c;
        };
        uint32_t bits;
        if (16 * NC <= 1 << a.lg_page) {          // one page
            Chunk c = look(0, bits);
            straight = plain(u, c);
            c.pos += 16 * (NC - 1);
            straight = straight && plain(u, c);
            in = bits * (QT == 1 ? (1u << NC) - 1 : NC == 2 ? 5u : 0x55u);
        } else {
            straight = true;
            in = 0u;
#pragma unroll
            for (int h = 0; h < NC; h++) {
                const Chunk c = look(h, bits);
                straight = straight && plain(u, c);
                in |= bits << (h * QT);
            }
        }
        return !straight || __any(in != 0u);
    }
};

// Byte offset of a lane's row, held as two registers and read by another lane's number
struct Offset {
    uint32_t lo, hi;
    __device__ __forceinline__ void set(const PagedAttnArgs &a, int kvh, int page, int row, int row_bytes)
    {
        page = min(max(page, 0), a.n_pages - 1);
        const uint64_t x = (((uint64_t)((uint64_t)(uint32_t)page * (uint32_t)a.hkv + (uint32_t)kvh) << a.lg_page) + (uint32_t)(row & ((1 << a.lg_page) - 1))) * (uint32_t)row_bytes;
        lo = (uint32_t)x;
        hi = (uint32_t)(x >> 32);
    }
    __device__ __forceinline__ int64_t of(int lane) const { return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)lo, lane)); }
};
// N pieces of 1024 bytes, one behind the other in memory and in LDS; lane_at(j): of the lane's 16 bytes in piece j
template <int N, class F>
__device__ __forceinline__ void lds_load_run(const void *from, F lane_at, uint32_t to)
{
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"   // m0 is reserved; naming it as clobbered is right all the same
    if constexpr (N >= 4) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\ts_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %5\n\t"
                     "s_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %5\n\ts_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %5" ::"s"(to),
                     "v"(lane_at(0)), "v"(lane_at(1) + 1024u), "v"(lane_at(2) + 2 * 1024u), "v"(lane_at(3) + 3 * 1024u), "s"(from)
                     : "memory", "m0", "scc");
        lds_load_run<N - 4>(static_cast<const char *>(from) + 4096, [&](int j) { return lane_at(j + 4); }, to + 4096);
    } else if constexpr (N >= 2) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\ts_add_u32 m0, m0, 1024\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" ::"s"(to), "v"(lane_at(0)),
                     "v"(lane_at(1) + 1024u), "s"(from)
                     : "memory", "m0", "scc");
        lds_load_run<N - 2>(static_cast<const char *>(from) + 2048, [&](int j) { return lane_at(j + 2); }, to + 2048);
    } else if constexpr (N == 1) {
        lds_load16(from, lane_at(0), to);
    }
#pragma clang diagnostic pop
}

template <int D, int QT, int NW>
struct KeysGeom {
    static constexpr int THREADS = 64 * NW, CAP = 16 * QT, ROW = 2 * D, TILE = 32 * ROW, LOADS = TILE / 1024;
    static constexpr int MAIN = NW * 2 * TILE;
    static_assert(CAP * D * 4 <= 2 * TILE, "a wave's sums fit its stage");
    static int bytes(int words) { return MAIN + NW * CAP * 8 + NW * 8 + (words > 1 ? CAP * words * 8 + DREAM_MAX_TREE * 4 : 0); }
};

// Few rows: the waves take the key tiles in turn, each for all of the rows, and never meet until the end.  A wave asks for its next keys as soon as a tile's scores are there, and for its next
// values as soon as they are added up.  What bounds it: memory where caches are long (8 sequences of up to 16 100 rows, 8 KV heads of 128, one node: 439 MB in 84 us, 5.2 TB/s); where they are short, what a CU
// pulls (75 to 87 KB a us) and the trips to memory ahead of the first scores and behind the last (one sequence, 60 nodes, 764 rows, 32 KV heads of 128: 12.4 us, of which a wave is in its tiles for 5).
template <int D, int QT, int NW, bool SPARSE>
__global__ __launch_bounds__(64 * NW) void paged_keys_kernel(PLAIN, PagedAttnArgs first)
{
    using G = KeysGeom<D, QT, NW>;
    constexpr int ROW = G::ROW, LPR = ROW / 16, RPI = 1024 / ROW, HALF = G::LOADS / 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid0 = threadIdx.x, lane0 = tid0 & 63, wave = __builtin_amdgcn_readfirstlane(tid0 >> 6);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    float2 *s_ml = reinterpret_cast<float2 *>(smem + G::MAIN);
    int32_t *flags = reinterpret_cast<int32_t *>(s_ml + NW * G::CAP);
    uint64_t *masks = reinterpret_cast<uint64_t *>(flags + 2 * NW);
    int32_t *parents = reinterpret_cast<int32_t *>(masks + G::CAP * first.words);

    Unit u;
    int rg;
    if (!UNIT_AT(first, G::CAP))
        return;
    // what needs no load is asked for first: of an own part the pages of the wave's tiles, the prefix length, the tree, the queries
    const int prefix = u.shared ? 0 : uniform_load(prefix_len + u.b);
    const int stride = u.splits * NW, mine = u.split * NW + wave;
    const bool early = !SPARSE && lg_and_early >> 8;       // no groups: the first tile is the first, whatever else the call holds
    const int lg_page = lg_and_early & 255;
    int page[2] = {0, 0};
    auto ask_pages = [&](int first) {      // of tiles first + lane * stride
#pragma unroll
        for (int h = 0; h < 2; h++)
            page[h] = table[(int64_t)u.b * max_pages + min(((first + lane0 * stride) * 2 + h) >> (lg_page - 4), max_pages - 1)];
    };
    PageList<G::THREADS> list;
    if constexpr (SPARSE)
        list.ask(first, u, tid0 * list.EACH);
    if (early)
        ask_pages(mine);
    int parent = -1;
    if (!u.shared && first.words == 1 && !first.tree_mask)
        parent = first.parent[(int64_t)u.b * first.n_tree + min(lane0, first.n_tree - 1)];
    if (!unit_of(first, G::CAP, lane0, rg, prefix, u))
        return;
    if (u.alone)
        no_shared_parts(first, u, G::CAP, tid0, G::THREADS);
    // Selected pages: list by list.  (One, but where more pages are seen than were expected: what the lists in front gave waits in the part's slot, and joins.)
    for (int skip = 0;;) {
        const int tid = SPARSE ? here(tid0) : tid0, lane = tid & 63, c = lane & 15, g = lane >> 4;      // (nothing but this is kept from list to list)
        if constexpr (SPARSE)
            list.build(args_again(), u, G::CAP, tid, reinterpret_cast<unsigned char *>(masks + (first.words > 1 ? G::CAP * first.words + DREAM_MAX_TREE / 2 : 0)), skip);
        const PagedAttnArgs &a = SPARSE ? args_again() : first;
        QueryRows<D, QT, 2, SPARSE, 2> rows;
        rows.load(a, u, u.row0, c, g);
        const int tile0 = u.lo / 32;
        if (!SPARSE && !early)
            ask_pages(tile0 + mine);

        const int foff = fragment_k<ROW>(c, g), voff = fragment_v<ROW>(c, g);
        const int krow = lane / LPR, k_lane = krow * ROW + piece_k<ROW>(lane), v_lane = krow * ROW + piece_v<ROW>(lane);
        const int stage = wave * 2 * G::TILE;
        auto chunk = [&](int i, int h) -> Chunk {
            if constexpr (SPARSE) {
                return listed_chunk(a, list, (wave + i * NW) * 32 + h * 16);
            } else {
                const int pos = (tile0 + mine + i * stride) * 32 + h * 16;
                return Chunk{0, pos, pos < u.hi, true, true};
            }
        };
        Offset offset[2];                             // of the chunks of the lane's tile (of the list's: in units of a run of 64 as well)
        auto locate = [&](int i) {                    // tiles i .. i + 63
#pragma unroll
            for (int h = 0; h < 2; h++) {
                if constexpr (SPARSE) {
                    const int x = (wave + (i + lane) * NW) * 32 + h * 16;
                    offset[h].set(a, u.kvh, list.phys[min(x >> lg_page, list.n - 1)], x, ROW);
                } else {
                    offset[h].set(a, u.kvh, page[h], (tile0 + mine + (i + lane) * stride) * 32 + h * 16, ROW);
                }
            }
        };
        auto place = [&](int i, int h) { return offset[h].of(i & 63); };
        auto ask_k = [&](int i) {
            if ((i & 63) == 0) {
                if (!SPARSE && i)
                    ask_pages(tile0 + mine + i * stride);
                locate(i);
            }
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int at = here(k_lane);
                lds_load_run<HALF>(a.k + place(i, h), [&](int j) { return (uint32_t)(at ^ swizzle_k<ROW>(h * HALF + j)); }, here_scalar(lds0 + stage) + h * HALF * 1024);
            }
        };
        auto ask_v = [&](int i) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const int at = here(v_lane);
                lds_load_run<HALF>(a.v + place(i, h), [&](int j) { return (uint32_t)(at ^ swizzle_v<ROW>(h * HALF + j)); }, here_scalar(lds0 + stage) + G::TILE + h * HALF * 1024);
            }
        };
        // Zeros over the values of rows that are nobody's
        auto clear_dead = [&](const Chunk (&ch)[2]) {
            const int vat = here_scalar(stage + G::TILE);
#pragma unroll
            for (int h = 0; h < 2; h++) {
                if (rows.plain(u, ch[h]))
                    continue;
#pragma unroll 1
                for (int j = 0; j < HALF; j++) {
                    const int pos = ch[h].pos + j * RPI + krow;
                    if (!(ch[h].live && ((ch[h].prefix && pos >= u.lo && pos < u.P) || (ch[h].tree && pos >= u.P && pos < u.hi))))
                        *reinterpret_cast<u32x4 *>(smem + vat + (h * HALF + j) * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
                }
            }
            wait_lds();
        };
        auto take = [&](int steps) {
            for (int i = 0; i < steps; i++) {
                Chunk ch[2];
                bool straight;
                uint32_t in = 0u;
                if constexpr (SPARSE) {
                    rows.seen_by(a, u, list, (wave + i * NW) * 32, straight, in);
                } else {
                    const int pos = (tile0 + mine + i * stride) * 32;
                    straight = pos >= u.lo && pos + 32 <= rows.whole;
                }
                if (!straight || a.scale_log2 < 0.0f) {
                    ch[0] = chunk(i, 0);
                    ch[1] = chunk(i, 1);
                }
                f32x4 s[2][QT];
                typename decltype(rows)::Weights pf;
                wait_loads<G::LOADS>();
                rows.scores(smem + stage, here(foff), 0, s);
                wait_lds();
                if (i + 1 < steps)
                    ask_k(i + 1);
                const bool masked = !straight || a.scale_log2 < 0.0f;      // (the largest score of a negative scale is the smallest product)
                if (masked)
                    rows.mask(a, u, ch, in, g, s);
                const float scaled = masked ? 1.0f : a.scale_log2;
                in = masked ? ~0u : in;
                rows.raise(scaled, in, s);
#pragma unroll
                for (int j = 0; j < rows.SLICES; j++)
                    rows.weigh(scaled, in, j, s, pf);
                if (i + 1 < steps)
                    wait_loads<G::LOADS>();
                else
                    wait_loads<0>();
                if (!straight)
                    clear_dead(ch);
                rows.add_values(smem + stage + G::TILE, here(voff), pf);
                wait_lds();
                if (i + 1 < steps)
                    ask_v(i + 1);
            }
        };
        const int steps = SPARSE ? (((list.n << a.lg_page) + 31) / 32 - wave + NW - 1) / NW : u.hi > u.lo ? ((u.hi + 31) / 32 - tile0 - mine + stride - 1) / stride : 0;
        if (steps > 0) {
            ask_k(0);
            ask_v(0);
        }
        rows.see(a, u, u.row0, G::CAP, parent, c, tid, G::THREADS, masks, parents, 0);
        take(steps);

        // ---- the waves' sums meet, each wave's in its own stage: 16-byte piece i of row r at i ^ (r mod 16)
        const bool strange = rows.finish();
        if (lane == 0)
            flags[wave] = strange;
        if (g == 0)
#pragma unroll
            for (int qt = 0; qt < QT; qt++)
                s_ml[wave * G::CAP + qt * 16 + c] = make_float2(rows.m[qt], rows.l[qt]);
#pragma unroll
        for (int qt = 0; qt < QT; qt++)
#pragma unroll
            for (int dt = 0; dt < D / 16; dt++)
                *reinterpret_cast<f32x4 *>(smem + stage + (qt * 16 + c) * (4 * D) + ((dt * 4 + g) ^ c) * 16) = rows.o[qt][dt];
        __syncthreads();
        const PagedAttnArgs &z = args_again();
        int again = 0;
#pragma unroll
        for (int w = 0; w < NW; w++)
            again |= flags[w];
        if (again)
            break;
        const int count = min(G::CAP, u.n_rows - u.row0);
        const bool more = SPARSE && skip + z.list_size < list.all;
        for (int i = tid; i < count * (D / 4); i += G::THREADS) {
            const int j = i / (D / 4), ch = i % (D / 4);
            const Row w = row_at(z, u, u.row0 + j);
            float2 ml[NW];
            float most = -INFINITY, sum = 0.0f;
            f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < NW; x++) {
                ml[x] = s_ml[x * G::CAP + j];
                most = fmaxf(most, ml[x].x);
            }
#pragma unroll
            for (int x = 0; x < NW; x++) {
                const float f = ml[x].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[x].x - most);
                sum = __builtin_fmaf(ml[x].y, f, sum);
                all += *reinterpret_cast<const f32x4 *>(smem + x * 2 * G::TILE + j * (4 * D) + (ch ^ (j & 15)) * 16) * f;
            }
            float *slot = z.part_o + row_of_part(z, u, w) * D + ch * 4;
            if (SPARSE && skip) {
                Earlier earlier;
                earlier.join(z, u, w, most, sum);
                all = *reinterpret_cast<const f32x4 *>(slot) * earlier.old + all * earlier.now;
            }
            const bool part = z.n_slots > 1 || (SPARSE && more);
            if (ch == 0)
                put_ml(z, u, w, most, sum, part);
            if (part) {
                *reinterpret_cast<f32x4 *>(slot) = all;
            } else {
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(z.out) + row_of_q(z, w) * D + ch * 4) = make_uint2(pack_bf16(all[0] * inv, all[1] * inv), pack_bf16(all[2] * inv, all[3] * inv));
            }
        }
        if (!more)
            return;
        skip += z.list_size;
        list.ask(args_again(), u, tid * list.EACH);
    }
    // a sum is not finite: all of the keys again, row by row
    __syncthreads();
    attend_rows_singly<uint16_t, D, G::THREADS, SPARSE>(args_again(), u, G::CAP, 32, 32 * NW, smem);
}

template <int D, int QT, int WR, int NS>
struct RowsGeom {
    static constexpr int THREADS = 64 * WR, CAP = 16 * QT * WR, ROW = 2 * D, KEYS = D == 256 ? 32 : 64, TILE = KEYS * ROW, STAGE = 2 * TILE;
    static constexpr int LOADS = TILE / 1024 / WR;                          // of a wave, a tile and K or V: rows of one chunk
    static constexpr int MAIN = NS * STAGE;
    static_assert(LOADS * 1024 * WR == TILE && KEYS / WR <= 16, "loads");
    static int bytes(int words) { return MAIN + WR * 8 + (words > 1 ? CAP * words * 8 + DREAM_MAX_TREE * 4 : 0); }
};

// Many rows: the waves share the tiles and have rows of their own; one barrier a tile, NS - 1 tiles on their way.  What bounds it: issue.  A tile of 64 keys against a wave's 32 rows of 128 is 1024
// clocks of matrix products and 3200 to 3700 of a lone wave's time (scores and exponentials 1450 to 1680, weighted sums 770 to 880, asking 380 to 470, references 330, the barrier 110), 2400 of each of two
// on a SIMD; 580 TFLOP/s over the call below.  (8 sequences of 60 nodes with 4096 shared rows of 8 KV heads of 128, 32 query heads: 59 us, and 7 for the join.)  At head_dim 64 a wave of 16 rows is held to 128
// registers, four waves a SIMD: 33 nodes of 32 sequences in groups 44.5 -> 40.2 us.
template <int D, int QT, int WR, int NS, bool SPARSE>
__global__ __launch_bounds__(64 * WR, D == 64 && QT == 1 && !SPARSE ? 4 : 2) void paged_rows_kernel(PLAIN, PagedAttnArgs first)
{
    using G = RowsGeom<D, QT, WR, NS>;
    constexpr int ROW = G::ROW, KEYS = G::KEYS, NC = KEYS / 16, LPR = ROW / 16, RPI = 1024 / ROW;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid0 = threadIdx.x, lane0 = tid0 & 63, wave = __builtin_amdgcn_readfirstlane(tid0 >> 6);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    int32_t *flags = reinterpret_cast<int32_t *>(smem + G::MAIN);
    uint64_t *masks = reinterpret_cast<uint64_t *>(flags + 2 * WR);
    int32_t *parents = reinterpret_cast<int32_t *>(masks + G::CAP * first.words);

    Unit u;
    int rg;
    if (!UNIT_AT(first, G::CAP))
        return;
    const int prefix = u.shared ? 0 : uniform_load(prefix_len + u.b);
    const int own_rows = wave * (KEYS / WR), own_chunk = own_rows & ~15;      // of a tile: the rows that this wave asks for, and the chunk that they lie in
    const bool early = !SPARSE && lg_and_early >> 8;       // no groups: the first tile is the first, whatever else the call holds
    const int lg_page = lg_and_early & 255;
    int page = 0;
    auto ask_pages = [&](int first) { page = table[(int64_t)u.b * max_pages + min(((first + lane0 * u.splits) * KEYS + own_chunk) >> lg_page, max_pages - 1)]; };      // of tiles first + lane * splits
    PageList<G::THREADS> list;
    if constexpr (SPARSE)
        list.ask(first, u, tid0 * list.EACH);
    if (early)
        ask_pages(u.split);
    int parent = -1;
    if (!u.shared && first.words == 1 && !first.tree_mask)
        parent = first.parent[(int64_t)u.b * first.n_tree + min(lane0, first.n_tree - 1)];
    if (!unit_of(first, G::CAP, lane0, rg, prefix, u))
        return;
    if (u.alone)
        no_shared_parts(first, u, G::CAP, tid0, G::THREADS);
    // Selected pages: list by list
    for (int skip = 0;;) {
        const int tid = SPARSE ? here(tid0) : tid0, lane = tid & 63, c = lane & 15, g = lane >> 4;      // (nothing but this is kept from list to list)
        if constexpr (SPARSE)
            list.build(args_again(), u, G::CAP, tid, reinterpret_cast<unsigned char *>(masks + (first.words > 1 ? G::CAP * first.words + DREAM_MAX_TREE / 2 : 0)), skip);
        const PagedAttnArgs &a = SPARSE ? args_again() : first;
        QueryRows<D, QT, NC, SPARSE, D == 256 ? 2 : 1> rows;
        const int first_row = u.row0 + wave * QT * 16;
        rows.load(a, u, first_row, c, g);
        const int tile0 = u.lo / KEYS + u.split;
        if (!SPARSE && !early)
            ask_pages(tile0);

        const int foff = fragment_k<ROW>(c, g), voff = fragment_v<ROW>(c, g);
        const int krow = lane / LPR, k_lane = krow * ROW + piece_k<ROW>(lane), v_lane = krow * ROW + piece_v<ROW>(lane);
        auto chunk = [&](int i, int at) -> Chunk {
            if constexpr (SPARSE) {
                return listed_chunk(a, list, i * KEYS + at);
            } else {
                const int pos = (tile0 + i * u.splits) * KEYS + at;
                return Chunk{0, pos, pos < u.hi, true, true};
            }
        };
        Offset offset;                                         // of the wave's rows of the lane's tile
        auto locate = [&](int i) {                             // tiles i .. i + 63
            if constexpr (SPARSE) {
                const int x = (i + lane) * KEYS + own_rows;
                offset.set(a, u.kvh, list.phys[min(x >> lg_page, list.n - 1)], x, ROW);
            } else {
                offset.set(a, u.kvh, page, (tile0 + (i + lane) * u.splits) * KEYS + own_rows, ROW);
            }
        };
        auto ask_tile = [&](const unsigned char *from, int lane_at, bool values, int stage) {
            lds_load_run<G::LOADS>(from, [&](int j) { return (uint32_t)(lane_at ^ (values ? swizzle_v<ROW>(wave * G::LOADS + j) : swizzle_k<ROW>(wave * G::LOADS + j))); },
                                   lds0 + (values ? NS + stage : stage) * G::TILE + wave * G::LOADS * 1024);
        };
        auto after = [](int stage) { return stage == NS - 1 ? 0 : stage + 1; };
        // Zeros over the values of rows that are nobody's, by the wave that loaded them
        auto clear_dead = [&](int i, int stage) {
            const Chunk ch = chunk(i, own_chunk);
            if (rows.plain(u, ch))
                return;
#pragma unroll
            for (int j = 0; j < G::LOADS; j++) {
                const int pos = ch.pos + (own_rows & 15) + j * RPI + krow;
                if (!(ch.live && ((ch.prefix && pos >= u.lo && pos < u.P) || (ch.tree && pos >= u.P && pos < u.hi))))
                    *reinterpret_cast<u32x4 *>(smem + (NS + stage) * G::TILE + (wave * G::LOADS + j) * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
            }
        };
        const int steps = SPARSE ? ((list.n << a.lg_page) + KEYS - 1) / KEYS : u.hi > u.lo ? max(0, ((u.hi + KEYS - 1) / KEYS - tile0 + u.splits - 1) / u.splits) : 0;

        // What is known of a tile: scores and how they are to be read; have: some of the wave's rows see it
        struct Tile {
            f32x4 s[NC][QT];
            float scaled;
            uint32_t in;
            bool have, masked;
        };
        auto look = [&](int i, Tile &t) {
            bool straight;
            if constexpr (SPARSE) {
                t.have = rows.seen_by(a, u, list, i * KEYS, straight, t.in);
            } else {
                const int pos = (tile0 + i * u.splits) * KEYS;
                straight = pos >= u.lo && pos + KEYS <= rows.whole;
                t.have = true;
                t.in = 0u;
            }
            t.masked = !straight || a.scale_log2 < 0.0f;      // (the largest score of a negative scale is the smallest product)
            t.scaled = t.masked ? 1.0f : a.scale_log2;
        };
        typename decltype(rows)::Weights pf;
        // Scores that have come: what nobody sees is left out, the references are raised
        auto settle = [&](int i, Tile &t) {
            if (t.masked) {
                Chunk ch[NC];
#pragma unroll
                for (int h = 0; h < NC; h++)
                    ch[h] = chunk(i, h * 16);
                rows.mask(a, u, ch, t.in, g, t.s);
                t.in = ~0u;
            }
            rows.raise(t.scaled, t.in, t.s);
        };
        auto add_values = [&](int stage) { rows.add_values(smem + (NS + stage) * G::TILE, here(voff), pf); };
        // Interval i: the keys of tile i + 1 and the values of tile i are there; those that NS - 1 intervals later need are asked for
        int64_t next_v = 0;             // where the values lie that are asked for next
        int k_stage = 0, v_stage = 0, k_ask = 0, v_ask = 0;
        auto ask = [&](int i) {         // what interval i needs
            ask_tile(a.v + next_v, v_lane, true, v_ask);
            if ((i + 1 & 63) == 0 && i + 1 < steps) {
                if (!SPARSE)
                    ask_pages(tile0 + (i + 1) * u.splits);
                locate(i + 1);
            }
            next_v = offset.of(min(i + 1, steps - 1) & 63);      // (behind the last tile that one again: such keys are never used)
            ask_tile(a.k + next_v, k_lane, false, k_ask);
            k_ask = after(k_ask);
            v_ask = after(v_ask);
        };
        if (steps > 0) {
            locate(0);
            next_v = offset.of(0);
            ask_tile(a.k + next_v, k_lane, false, 0);
            k_ask = after(0);
#pragma unroll
            for (int i = 0; i < NS - 1; i++)
                if (i < steps)
                    ask(i);
        }
        rows.see(a, u, first_row, G::CAP, parent, c, tid, G::THREADS, masks, parents, wave * QT * 16);
        if (steps > 0) {
            if (steps >= NS - 1)
                wait_loads<(NS - 1) * 2 * G::LOADS>();
            else
                wait_loads<0>();
            asm volatile("s_barrier" ::: "memory");
            Tile even, odd;
            {
                look(0, even);
                if (even.have) {
#pragma unroll
                    for (int h = 0; h < NC; h += 2)
                        rows.scores(smem, here(foff), h, even.s);
                    settle(0, even);
                }
            }
            // Interval i: the weights of tile i while the matrix cores are at the scores of tile i + 1, then the values of tile i, then what the new scores change
            auto interval = [&](int i, Tile &t, Tile &n) {
                if (i + NS - 2 < steps)
                    wait_loads<(NS - 2) * 2 * G::LOADS>();
                else
                    wait_loads<0>();
                if (t.masked)
                    clear_dead(i, v_stage);
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // the tiles are there, and all have done with the stages that are loaded next
                if (i + NS - 1 < steps)
                    ask(i + NS - 1);
                k_stage = after(k_stage);
                const unsigned char *kt = smem + k_stage * G::TILE;
                n.have = false;
                if (i + 1 < steps)
                    look(i + 1, n);
                if (t.have && n.have) {
                    rows.scores_and_weights(kt, here(foff), n.s, t.scaled, t.in, t.s, pf);
                } else if (t.have) {
#pragma unroll
                    for (int j = 0; j < rows.SLICES; j++)
                        rows.weigh(t.scaled, t.in, j, t.s, pf);
                } else if (n.have) {
#pragma unroll
                    for (int h = 0; h < NC; h += 2)
                        rows.scores(kt, here(foff), h, n.s);
                }
                if (t.have)
                    add_values(v_stage);
                if (n.have)
                    settle(i + 1, n);
                v_stage = after(v_stage);
            };
            for (int i = 0; i < steps; i += 2) {
                interval(i, even, odd);
                if (i + 1 < steps)
                    interval(i + 1, odd, even);
            }
        }

        const bool strange = rows.finish();
        if (lane == 0)
            flags[wave] = strange;
        __syncthreads();
        const PagedAttnArgs &z = args_again();
        int again = 0;
#pragma unroll
        for (int w = 0; w < WR; w++)
            again |= flags[w];
        if (again)
            break;
        const bool more = SPARSE && skip + z.list_size < list.all, part = z.n_slots > 1 || more;
#pragma unroll
        for (int qt = 0; qt < QT; qt++) {
            const int j = first_row + qt * 16 + c;
            if (j >= u.n_rows)
                continue;
            const Row w = row_at(z, u, j);
            float *slot = z.part_o + row_of_part(z, u, w) * D + 4 * g;
            if (SPARSE && skip) {
                Earlier earlier;
                earlier.join(z, u, w, rows.m[qt], rows.l[qt]);
#pragma unroll
                for (int dt = 0; dt < D / 16; dt++)
                    rows.o[qt][dt] = *reinterpret_cast<const f32x4 *>(slot + dt * 16) * earlier.old + rows.o[qt][dt] * earlier.now;
            }
            if (g == 0)
                put_ml(z, u, w, rows.m[qt], rows.l[qt], part);
            if (part) {
#pragma unroll
                for (int dt = 0; dt < D / 16; dt++)
                    *reinterpret_cast<f32x4 *>(slot + dt * 16) = rows.o[qt][dt];
            } else {
                const float inv = rows.l[qt] == 0.0f ? 0.0f : 1.0f / rows.l[qt];
                uint16_t *row = static_cast<uint16_t *>(z.out) + row_of_q(z, w) * D + 4 * g;
#pragma unroll
                for (int dt = 0; dt < D / 16; dt++)
                    *reinterpret_cast<uint2 *>(row + dt * 16) =
                        make_uint2(pack_bf16(rows.o[qt][dt][0] * inv, rows.o[qt][dt][1] * inv), pack_bf16(rows.o[qt][dt][2] * inv, rows.o[qt][dt][3] * inv));
            }
        }
        if (!more)
            return;
        skip += z.list_size;
        list.ask(args_again(), u, tid * list.EACH);
    }
    // a sum is not finite: all of the keys again, row by row
    __syncthreads();
    attend_rows_singly<uint16_t, D, G::THREADS, SPARSE>(args_again(), u, G::CAP, KEYS, KEYS, smem);
}

// ---- the parts of a row, in their order: D / 4 lanes a row, AT parts at a time ------------------------------------------
template <class T, int D, int AT>
__global__ __launch_bounds__(256) void paged_join_kernel(const float *part_o, const float2 *part_ml, void *out, float *lse, uint32_t all_rows, int n_slots, uint32_t rows, uint32_t rows_magic, uint32_t hkv,
                                                         uint32_t hkv_magic, uint32_t group, uint32_t group_magic, int hq, int n_tree)
{
    constexpr int LANES = D / 4;
    const uint32_t id = blockIdx.x * (blockDim.x / LANES) + threadIdx.x / LANES;
    const int ch = threadIdx.x % LANES;
    if (id >= all_rows)
        return;
    float most = -FLT_MAX, sum = 0.0f;
    f32x4 all = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n_slots; s0 += AT) {
        float2 ml[AT];
        f32x4 x[AT];
#pragma unroll
        for (int i = 0; i < AT; i++) {
            const int64_t row = (int64_t)min(s0 + i, n_slots - 1) * all_rows + id;
            ml[i] = part_ml[row];
            x[i] = *reinterpret_cast<const f32x4 *>(part_o + row * D + ch * 4);
        }
        float top = most;
#pragma unroll
        for (int i = 0; i < AT; i++)
            top = fmaxf(top, ml[i].x);
        const float raised = __builtin_amdgcn_exp2f(most - top);
        sum *= raised;
        all *= raised;
        most = top;
#pragma unroll
        for (int i = 0; i < AT; i++)
            if (s0 + i < n_slots && ml[i].y != 0.0f) {      // (NaN: not 0.  A part without keys holds anything)
                const float f = __builtin_amdgcn_exp2f(fmaxf(ml[i].x, -FLT_MAX) - most);
                sum = __builtin_fmaf(ml[i].y, f, sum);
                all += x[i] * f;
            }
    }
    const uint32_t head = divide(id, rows, rows_magic), b = divide(head, hkv, hkv_magic), r = id - head * rows, node = divide(r, group, group_magic);
    const int q_head = (int)((head - b * hkv) * group + r - node * group);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (ch == 0 && lse)
        lse[((int64_t)b * hq + q_head) * n_tree + node] = sum == 0.0f ? -INFINITY : (most + __log2f(sum)) * 0.6931471805599453f;
    const int64_t at = (((int64_t)b * n_tree + node) * hq + q_head) * D + ch * 4;
    if constexpr (std::is_same_v<T, float>)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + at) = all * inv;
    else
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(pack_bf16(all[0] * inv, all[1] * inv), pack_bf16(all[2] * inv, all[3] * inv));
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
enum Form { SINGLY, KEYS, ROWS };
struct Shape {                            // of a launch's workgroups
    Form form;
    int qt, waves;                        // query tiles of a wave
    int threads() const { return 64 * waves; }
    int cap() const { return form == SINGLY ? SINGLE_ROWS : form == KEYS ? 16 * qt : 16 * qt * waves; }
    int keys(int D) const { return form == SINGLY ? SINGLE_RUN : form == KEYS ? 32 * waves : D == 256 ? 32 : 64; }      // that a step of a workgroup takes
    bool operator==(const Shape &o) const { return form == o.form && qt == o.qt && waves == o.waves; }
};
struct Segment {
    Shape shape;
    Part part;
};
struct PagedPlan {
    Segment shared, own;
    int n_slots, shared_slots, list_size;
    int64_t all_rows, threads;            // threads: of the largest launch
    size_t bytes;
};

// The shapes there are, and what they are estimated to take: where a CU has `groups` workgroups,
//     us = base + per_group * (groups - 1) + steps * max(latency, issue * groups, kilobytes of a step / (FILL * min(row groups, 2)))  [+ the join]
// as long as memory does not take longer (the sixth root of both sixth powers).  FILL: what a CU pulls that nobody asks for beside it.  The constants are those with which the choice is best over
// measured times of every shape with every number of splits below (7 head layouts x batches of 1, 4, 16, 48 x trees of 1 to 120 nodes x 100 to 12000 keys, 558 problems, 9785 times): 1.5 % behind the
// fastest in the geometric mean, 8 % at the 95th percentile, 39 % at most, on the data that they were fitted to.  What a shape is worth over these problems (mean and most that the fastest would take
// longer without it): 16 rows 3.1 % and 24 %, 32 rows 0.5 % and 17 %, 64 rows 2.9 % and 54 %, 128 rows 0.9 % and 25 %, 128 rows of 256 on eight waves 0.1 % and 5 %; eight waves at
// smaller head_dim (0.2 %) and four query tiles a wave are left out.
// Two parts by the same constants, and calls over selected pages, measured afterwards: 27 problems with groups, every shape and split of both parts: 5.5 % behind the fastest in the geometric mean, 34 % at most
// (12 % but for two problems of two KV heads of 256); 17 of selected pages: 2.2 % and 10 %.
struct Kind {
    Shape shape;
    float base, per_group, latency, issue;
};
constexpr int KINDS = 4;
constexpr Kind KIND[3][KINDS] = {{{{KEYS, 1, 8}, 5.63f, 1.64f, 0.834f, 0.770f}, {{KEYS, 2, 8}, 7.12f, 5.07f, 1.049f, 1.075f}, {{ROWS, 1, 4}, 5.79f, 1.48f, 0.772f, 0.359f}, {{ROWS, 2, 4}, 7.58f, 2.26f, 0.954f, 0.670f}},
                                 {{{KEYS, 1, 8}, 6.22f, 5.03f, 1.312f, 1.563f}, {{KEYS, 2, 8}, 8.59f, 7.55f, 1.522f, 1.801f}, {{ROWS, 1, 4}, 6.64f, 2.69f, 0.996f, 0.657f}, {{ROWS, 2, 4}, 8.76f, 2.77f, 1.322f, 1.017f}},
                                 {{{KEYS, 1, 4}, 8.17f, 7.01f, 1.692f, 1.832f}, {{KEYS, 1, 4}, 8.17f, 7.01f, 1.692f, 1.832f}, {{ROWS, 1, 4}, 7.43f, 3.07f, 0.934f, 0.622f}, {{ROWS, 1, 8}, 9.52f, 6.35f, 1.137f, 1.137f}}};
constexpr int kinds_of(int D) { return D == 64 ? 0 : D == 128 ? 1 : 2; }
constexpr float FILL = 87.2f, MEMORY = 4.90e6f, JOIN = 2.18f, JOIN_SPLIT = 0.106f, JOIN_BYTE = 1.27e-6f;      // KB / us; bytes / us; us, us a split, us a value
constexpr int SPLITS[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48}, MOST_SPLITS = 128;      // of a part; of both, where they are forced

uint32_t magic_for(uint32_t d) { return 0xffffffffu / d; }

// What a part is: KV heads (of all sequences), query rows of each, keys; `groups`: lists of rows that end in a workgroup of their own (0: one a head); bytes of keys and values; the nodes that see
// keys of their own (0: none)
struct Problem {
    int64_t heads, rows, keys, groups;
    float bytes;
    int nodes_of, all_keys;               // query rows a node (selected pages: a workgroup with more nodes sees more pages)
};
int64_t row_groups_of(const Problem &p, const Shape &s) { return p.groups ? p.rows / s.cap() + p.groups : (p.rows + s.cap() - 1) / s.cap(); }

// A part in workgroups of one shape: workgroups of a split, steps of a unit, what a step cannot be shorter than
struct Load {
    float units, steps, step, joined;     // joined: us that its splits' join takes for each
    int64_t most_splits;
};
Load load_of(int D, const Problem &p, const Kind &k)
{
    const Shape &s = k.shape;
    const int64_t groups = row_groups_of(p, s), units = p.heads * (p.groups ? p.rows / s.cap() + 1 : groups);
    float keys = (float)p.keys;
    if (p.nodes_of) {                     // nodes that ask alike see more pages together: two 1.26 to 1.42 times as many as one, 60 2.3 to 3.9 (2^0.33 to 2^0.51, 60^0.2 to 60^0.33)
        const float nodes = (float)(p.rows < s.cap() ? p.rows : s.cap()) / (float)p.nodes_of;
        keys *= nodes > 1.0f ? powf(nodes, 0.4f) : 1.0f;
        keys = keys < (float)p.all_keys ? keys : (float)p.all_keys;
    }
    const int64_t steps = (int64_t)(keys / (float)s.keys(D)) + 1;
    const float fill = (float)(s.keys(D) * D) * 4e-3f / (FILL * (groups > 1 ? 2.0f : 1.0f));
    return {(float)units, (float)steps, k.latency > fill ? k.latency : fill, JOIN_SPLIT + JOIN_BYTE * (float)p.heads * (float)p.rows * (float)D, steps};
}
float sixth_roots_power(float us, float memory)
{
    us *= 1e-3f;                          // (in ms: the longest calls take seconds, and 3e38 is not far from the sixth power of their microseconds)
    memory *= 1e-3f;
    us *= us * us;
    memory *= memory * memory;
    return us * us + memory * memory;
}
// What a launch takes with so many splits of a part, and of a second one beside it, to the sixth power; `joined`: the part's rows have others, in a launch of their own
float launch_time(const Kind &k, const Load &x, int splits, bool joined, const Load *y, int y_splits, float memory)
{
    const float x_steps = (float)(((int)x.steps + splits - 1) / splits), y_steps = y ? (float)(((int)y->steps + y_splits - 1) / y_splits) : 0.0f;
    const float units = x.units * splits + (y ? y->units * y_splits : 0.0f), per_cu = (float)(((int64_t)units + 255) / 256);
    // (one part: a CU's busiest workgroups are as long as any other)
    const float work = y ? k.issue * (x.units * splits * x_steps + y->units * y_splits * y_steps) / 256.0f : k.issue * per_cu * x_steps;
    const float chain = y && y_steps * y->step > x_steps * x.step ? y_steps * y->step : x_steps * x.step;
    float us = k.base + k.per_group * (per_cu - 1.0f) + (chain > work ? chain : work);
    us += y ? x.joined * splits + y->joined * y_splits : joined ? x.joined * splits : splits > 1 ? JOIN + x.joined * splits : 0.0f;
    return sixth_roots_power(us, memory);
}

// The best of the shapes and splits, `most` at most, for a part, or for two parts in one launch, by launch_time
float choose(int D, bool f32, const Problem &p, bool joined, int most, Segment &out, const Problem *p2 = nullptr, Segment *out2 = nullptr)
{
    const int tiles = q_tiles_override(), waves = tile_waves_override(), forced = kv_splits_override();
    const float memory = (p.bytes + (p2 ? p2->bytes : 0.0f)) / MEMORY + 5.0f;
    float best = INFINITY;
    out = Segment{};
    if (p2)
        *out2 = Segment{};
    auto consider = [&](const Kind &k) {
        const Load x = load_of(D, p, k), y = p2 ? load_of(D, *p2, k) : Load{};
        for (int m : SPLITS) {
            if (p2 && !forced && (m > 4 || (m > 1 && (m > y.most_splits || m >= most))))
                break;
            const int room = !p2 ? most : forced ? most / 2 : most - m;      // (1 at least)
            for (int n : SPLITS) {
                if (n > 1 && (forced || n > x.most_splits || n > room))
                    break;
                const int splits = !forced ? n : forced < room ? forced : room;
                const float us = launch_time(k, x, splits, joined, p2 ? &y : nullptr, forced ? splits : m, memory);
                if (us < best || !out.part.splits) {      // (the first, whatever it takes)
                    best = us;
                    out.shape = k.shape;
                    out.part.splits = splits;
                    if (p2) {
                        out2->shape = k.shape;
                        out2->part.splits = forced ? splits : m;
                    }
                }
            }
            if (!p2 || forced)
                break;
        }
    };
    if (f32) {
        consider({{SINGLY, 0, 4}, 6.0f, 3.0f, 6.0f, 3.0f});
    } else {
        for (int i = 0; i < KINDS; i++) {
            const Kind &k = KIND[kinds_of(D)][i];
            const bool of_form = !waves || (waves == 8) == (k.shape.form == ROWS), last = i == (waves == 4 ? 1 : KINDS - 1);
            if (of_form && (!tiles || k.shape.qt == tiles || (last && tiles > k.shape.qt)))
                consider(k);
        }
        if (!out.part.splits)
            consider(KIND[kinds_of(D)][0]);
    }
    out.part.row_groups = (int)row_groups_of(p, out.shape);
    if (p2)
        out2->part.row_groups = (int)row_groups_of(*p2, out2->shape);
    return 1e3f * powf(best, 1.0f / 6.0f);
}

// Pages that a workgroup's rows may see, those of the tree included: what its lists, of all splits together, have to hold
int64_t listed_pages(const dream_page_desc *pages, int32_t n_tree, int64_t max_kv, int64_t seen_pages)
{
    int64_t most = (max_kv + pages->page_size - 1) / pages->page_size;
    if (seen_pages > 0 && seen_pages * n_tree < most)
        most = seen_pages * n_tree;
    return most + n_tree / pages->page_size + 2;
}

// Entries of a list, for so many pages: whole tiles of all waves (16 entries, 256 rows), and not so few that calls in which more pages are seen than was said take many lists (64 are 1 KB, and change no
// number of workgroups on a CU).
int list_size_of(int64_t pages, int32_t n_tree)
{
    const int64_t most = n_tree > 64 ? SPARSE_LIST / 2 : SPARSE_LIST, size = pages < 64 ? 64 : (pages + 15) / 16 * 16;
    return (int)(size < most ? size : most);
}

// most_slots: parts that there is room for, 2 at least where there are groups
PagedPlan plan_for(const dream_attn_desc *d, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv, int32_t n_groups, int64_t max_shared, bool sparse, int64_t seen_pages, int most_slots = MOST_SPLITS)
{
    PagedPlan p = {};
    const int D = d->head_dim;
    const bool f32 = d->dtype == DREAM_F32;
    const int64_t capacity = paged_rows(pages), group = d->n_q_heads / d->n_kv_heads, rows = n_tree * group, heads = (int64_t)d->batch * d->n_kv_heads, row_bytes = D * (f32 ? 8 : 4);
    max_kv = max_kv < 1 ? 1 : max_kv > capacity ? capacity : max_kv;
    max_shared = max_shared < 1 ? 1 : max_shared > max_kv ? max_kv : max_shared;
    auto finish = [&](Segment &s, int64_t n_heads, int least) {
        s.part.splits = s.part.splits > least ? s.part.splits : least;
        s.part.streams = (int)(n_heads * s.part.splits);
        const int64_t blocks = (int64_t)ceil_div(s.part.streams, 8) * 8 * s.part.row_groups, threads = blocks * s.shape.threads();
        s.part.blocks = (int)blocks;      // (where it does not fit, `threads` is refused)
        const bool together = p.n_slots && p.shared.shape == s.shape;      // (one launch for the shared and the own part)
        p.threads = together ? p.threads + threads : p.threads > threads ? p.threads : threads;
        s.part.row_groups_magic = magic_for(s.part.row_groups);
        s.part.splits_magic = magic_for(s.part.splits);
        s.part.slot = p.n_slots;
        p.n_slots += s.part.splits;
    };
    int64_t own_keys = n_groups ? max_kv - max_shared + 1 : max_kv;
    const bool some = sparse && seen_pages > 0 && seen_pages * pages->page_size + n_tree < own_keys;
    const int64_t all_keys = own_keys, listed = listed_pages(pages, n_tree, max_kv, seen_pages);
    own_keys = some ? seen_pages * pages->page_size + n_tree : own_keys;
    const Problem own = {heads, rows, own_keys, 0, (float)heads * (float)own_keys * (float)row_bytes, some ? (int)group : 0, (int)all_keys};
    if (n_groups) {
        const Problem shared = {d->n_kv_heads, d->batch * rows, max_shared, n_groups, (float)n_groups * (float)d->n_kv_heads * (float)max_shared * (float)row_bytes, 0, 0};
        Segment together, beside;
        const float one = choose(D, f32, shared, true, most_slots, together, &own, &beside);
        float two = choose(D, f32, shared, true, most_slots - 1, p.shared);
        two += choose(D, f32, own, true, most_slots - p.shared.part.splits, p.own);
        if (one <= two) {
            p.shared = together;
            p.own = beside;
        }
        finish(p.shared, d->n_kv_heads, 1);
        p.shared_slots = p.n_slots;
    } else {
        choose(D, f32, own, false, most_slots, p.own);
    }
    finish(p.own, heads, sparse && listed > (n_tree > 64 ? SPARSE_LIST / 2 : SPARSE_LIST) ? 2 : 1);      // (pages that no list holds: two workgroups at least, each list by list)
    p.list_size = sparse ? list_size_of(ceil_div(listed, p.own.part.splits), n_tree) : 0;
    p.all_rows = heads * rows;
    const bool several = sparse && !f32 && (int64_t)p.list_size * p.own.part.splits <= pages->max_pages;      // a workgroup may need several lists, and a slot for what they give (the page that the prefix ends in may be listed for the tree as well)
    if (p.n_slots > 1 && p.threads < p.all_rows * (D / 4))
        p.threads = p.all_rows * (D / 4);
    p.bytes = p.n_slots > 1 || several ? (size_t)p.n_slots * p.all_rows * (D + 2) * 4 : 0;
    return p;
}

// One kernel: of the bytes of LDS that it may take, and its launch
template <class F>
int launch_kernel(F *kernel, const PagedAttnArgs &a, int threads, size_t lds, const char *name, hipStream_t st)
{
    if (lds > 160 * 1024)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: %zu bytes of LDS", name, lds);
    hipLaunchKernelGGL(kernel, dim3(a.shared.blocks + a.own.blocks), dim3(threads), lds, st, a.table, a.prefix_len, a.max_pages, a.hkv, a.hkv_magic, a.shared.blocks, a.own.row_groups,
                       a.own.row_groups_magic, a.own.splits, a.own.splits_magic, a.own.streams, a.lg_page | (a.n_groups ? 0 : 256), a);
    return check_launch(name);
}
template <int THREADS, bool SPARSE>
size_t list_bytes(const PagedAttnArgs &a)
{
    return SPARSE ? PageList<THREADS>::bytes(a.list_size, a.words) : 0;
}
template <int D, int QT, int NW, bool SPARSE>
int launch_keys(PagedAttnArgs &a, hipStream_t st, bool set_up)
{
    using G = KeysGeom<D, QT, NW>;
    static std::atomic<uint64_t> done{0};
    auto *kernel = &paged_keys_kernel<D, QT, NW, SPARSE>;
    int rc = raise_lds_limit(done, reinterpret_cast<const void *>(kernel), 160 * 1024, "paged attention");
    if (rc || set_up)
        return rc;
    const size_t list = list_bytes<G::THREADS, SPARSE>(a), main = G::bytes(a.words) + list, again = single_bytes(G::CAP, a.words) + list;
    return launch_kernel(kernel, a, G::THREADS, main > again ? main : again, "paged_keys_kernel", st);
}
template <int D, int QT, int WR, int NS, bool SPARSE>
int launch_rows(PagedAttnArgs &a, hipStream_t st, bool set_up)
{
    using G = RowsGeom<D, QT, WR, NS>;
    static std::atomic<uint64_t> done{0};
    auto *kernel = &paged_rows_kernel<D, QT, WR, NS, SPARSE>;
    int rc = raise_lds_limit(done, reinterpret_cast<const void *>(kernel), 160 * 1024, "paged attention");
    if (rc || set_up)
        return rc;
    const size_t list = list_bytes<G::THREADS, SPARSE>(a), main = G::bytes(a.words) + list, again = single_bytes(G::CAP, a.words) + list;
    return launch_kernel(kernel, a, G::THREADS, main > again ? main : again, "paged_rows_kernel", st);
}

template <int D, bool SPARSE>
int launch_shape(PagedAttnArgs &a, const Shape &s, hipStream_t st, bool set_up = false)
{
    if (s.form == SINGLY) {
        const size_t list = list_bytes<256, SPARSE>(a);
        return launch_kernel(&paged_f32_kernel<D, SPARSE>, a, 256, single_bytes(SINGLE_ROWS, a.words) + list, "paged_f32_kernel", st);
    }
    if (s.form == ROWS) {
        if constexpr (D == 256)
            return s.waves == 8 ? launch_rows<D, 1, 8, 3, SPARSE>(a, st, set_up) : launch_rows<D, 1, 4, 2, SPARSE>(a, st, set_up);
        else
            return s.qt == 2 ? launch_rows<D, 2, 4, 2, SPARSE>(a, st, set_up) : launch_rows<D, 1, 4, 2, SPARSE>(a, st, set_up);
    }
    if constexpr (D == 256) {
        return launch_keys<D, 1, 4, SPARSE>(a, st, set_up);
    } else {
        return s.qt == 2 ? launch_keys<D, 2, 8, SPARSE>(a, st, set_up) : launch_keys<D, 1, 8, SPARSE>(a, st, set_up);
    }
}

template <int D, bool SPARSE>
int launch_all(PagedAttnArgs &a, const PagedPlan &p, bool f32, hipStream_t st)
{
    a.n_slots = p.n_slots;
    a.shared_slots = p.shared_slots;
    a.list_size = p.list_size;
    a.all_rows = p.all_rows;
    a.shared = p.shared.part;
    a.own = p.own.part;
    if (!SPARSE && a.n_groups && !(p.shared.shape == p.own.shape)) {      // two kernels
        a.own.blocks = 0;
        if (int rc = launch_shape<D, false>(a, p.shared.shape, st))
            return rc;
        a.shared.blocks = 0;
        a.own = p.own.part;
    }
    if (int rc = launch_shape<D, SPARSE>(a, p.own.shape, st))
        return rc;
    if (p.n_slots == 1)
        return DREAM_OK;
    auto join = [&](auto kernel) {
        const int threads = p.all_rows * (D / 4) <= 64 * 1024 ? 64 : 256;      // few rows over all CUs (256 rows of 256, 33 parts: 7.2 -> 6.5 us; fewer parts: no difference)
        hipLaunchKernelGGL(kernel, dim3(ceil_div(p.all_rows, threads / (D / 4))), dim3(threads), 0, st, a.part_o, a.part_ml, a.out, a.lse, (uint32_t)p.all_rows, p.n_slots, a.rows, a.rows_magic, a.hkv,
                           a.hkv_magic, a.group, a.group_magic, a.hq, a.n_tree);
    };
    if (f32)
        join(p.n_slots <= 2 ? &paged_join_kernel<float, D, 2> : p.n_slots <= 4 ? &paged_join_kernel<float, D, 4> : &paged_join_kernel<float, D, 8>);
    else
        join(p.n_slots <= 2 ? &paged_join_kernel<uint16_t, D, 2> : p.n_slots <= 4 ? &paged_join_kernel<uint16_t, D, 4> : &paged_join_kernel<uint16_t, D, 8>);
    return check_launch("paged_join_kernel");
}
template <int D, bool SPARSE>
int set_up()
{
    PagedAttnArgs a = {};
    for (const Kind &k : KIND[kinds_of(D)])
        if (int rc = launch_shape<D, SPARSE>(a, k.shape, nullptr, true))
            return rc;
    return DREAM_OK;
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

// Plan: from how many parts there is room for
template <class Plan>
int run(const char *who, const dream_attn_desc *d, const dream_page_desc *pages, PagedAttnArgs &a, Plan plan, void *ws, size_t ws_bytes, void *stream)
{
    if (!a.q || !a.k || !a.v || !a.table || !a.prefix_len || (!a.parent && !a.tree_mask) || !a.out || !ws)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if ((reinterpret_cast<uintptr_t>(a.q) | reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v) | reinterpret_cast<uintptr_t>(a.out) | reinterpret_cast<uintptr_t>(ws)) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: a tensor is not 16-byte aligned", who);
    PagedPlan p = plan(MOST_SPLITS);
    if (ws_bytes < p.bytes) {                 // one that another call's size was asked for: fewer parts
        const size_t needed = p.bytes, room = ws_bytes / (p.bytes / p.n_slots);
        if (room > 1)
            p = plan((int)room);
        else if (!a.n_groups)
            p = plan(1);
        if (ws_bytes < p.bytes)
            return fail(DREAM_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, needed);
    }
    if (p.threads >= (1ll << 32) - 1024)      // (the join's last workgroup may be whole)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: a launch of %lld threads, 2^32 or more", who, (long long)p.threads);
    a.part_o = static_cast<float *>(ws);
    a.part_ml = reinterpret_cast<float2 *>(a.part_o + (size_t)p.n_slots * p.all_rows * d->head_dim);
    a.batch = d->batch; a.hq = d->n_q_heads; a.hkv = d->n_kv_heads; a.group = a.hq / a.hkv; a.rows = a.n_tree * a.group; a.words = (a.n_tree + 63) / 64;
    a.lg_page = log2_of(pages->page_size); a.n_pages = pages->n_pages; a.max_pages = pages->max_pages;
    a.hkv_magic = magic_for(a.hkv); a.group_magic = magic_for(a.group); a.rows_magic = magic_for(a.rows);
    const float scale = d->scale != 0.0f ? d->scale : 1.0f / sqrtf((float)d->head_dim);
    a.scale_log2 = scale * 1.4426950408889634f;
    const bool f32 = d->dtype == DREAM_F32;
    hipStream_t st = as_stream(stream);
    if (a.nodes)
        return d->head_dim == 64 ? launch_all<64, true>(a, p, f32, st) : d->head_dim == 128 ? launch_all<128, true>(a, p, f32, st) : launch_all<256, true>(a, p, f32, st);
    return d->head_dim == 64 ? launch_all<64, false>(a, p, f32, st) : d->head_dim == 128 ? launch_all<128, false>(a, p, f32, st) : launch_all<256, false>(a, p, f32, st);
}

}  // namespace

int dream::paged_attn_init()
{
    for (int rc : {set_up<64, false>(), set_up<64, true>(), set_up<128, false>(), set_up<128, true>(), set_up<256, false>(), set_up<256, true>()})
        if (rc)
            return rc;
    return DREAM_OK;
}

extern "C" {

size_t dream_paged_verify_attn_workspace(const dream_attn_desc *desc, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len, int32_t n_groups, int64_t max_shared_len)
{
    if (check_attn("dream_paged_verify_attn_workspace", desc, pages, n_tree, n_groups))
        return DREAM_WORKSPACE_MIN_BYTES;
    const size_t n = plan_for(desc, pages, n_tree, max_kv_len, n_groups, max_shared_len, false, 0).bytes;
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
    auto plan = [&](int slots) { return plan_for(desc, pages, n_tree, max_kv_len, n_groups, max_shared_len, false, 0, slots); };
    return run(who, desc, pages, a, plan, workspace, workspace_bytes, stream);
}

size_t dream_sparse_verify_attn_workspace(const dream_attn_desc *desc, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len, int32_t max_pages_seen)
{
    if (check_attn("dream_sparse_verify_attn_workspace", desc, pages, n_tree, 0))
        return DREAM_WORKSPACE_MIN_BYTES;
    const size_t n = plan_for(desc, pages, n_tree, max_kv_len, 0, 0, true, max_pages_seen).bytes;
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
    auto plan = [&](int slots) { return plan_for(desc, pages, n_tree, max_kv_len, 0, 0, true, max_pages_seen, slots); };
    return run(who, desc, pages, a, plan, workspace, workspace_bytes, stream);
}

}  // extern "C"
