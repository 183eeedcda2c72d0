// dream_page_select: which pages of its prefix each node sees, by an upper bound of its scores there.
//
// With a page's largest value U_d and smallest W_d in every channel, q . k <= sum_d max(q_d, 0) U_d + min(q_d, 0) W_d for each of its keys; summed over the query heads of a KV head that is one
// number for a node, a KV head and a page.  Queries and bounds are held as whole numbers up to 127 times a power of two (queries to nearest, bounds rounded outwards, so that they stay bounds).
// Two reasons: the sums are whole numbers, so no order of adding them changes which page comes first, and the matrix instruction takes 8-bit numbers at four times the rate.  What is lost is a
// step of 2^-7 of the largest value, of numbers that only rank pages.
//
// Two launches.  score_kernel: S^T = pages x nodes by v_mfma_i32_16x16x64_i8, the parts c+ against U and c- against W one behind the other.  The heads' numbers add up before the product (it is linear in
// them): the sum, at most 64 * 127, goes in as two numbers, 64 hi + lo.  choose_kernel: a wave per node finds the n_best-th score by halving the range of the scores, taken as whole numbers
// in their order, until as many lie above as are wanted; where equal scores straddle the border the lower pages win.
#include <type_traits>
#include "paged.h"

using namespace dream;

namespace {

constexpr int NODES = 64;            // of a workgroup: the bits of a word
constexpr int PAGES = 64;            // of a workgroup of score_kernel: 16 for each wave
constexpr int RANGE = 2048;          // pages whose words choose_kernel holds at a time

struct SelectArgs {
    const void *q, *bounds;
    const int32_t *table, *prefix_len;
    uint32_t *keys;                  // [B, Hkv, n_tree, stride]
    uint64_t *page_nodes;
    int32_t n_tree, hq, hkv, group, lg_page, n_pages, max_pages, max_prefix, stride, n_first, n_last, n_best;
};

__device__ __forceinline__ int pages_of(const SelectArgs &a, int b)
{
    const int P = min(max(uniform_load(a.prefix_len + b), 0), a.max_prefix);
    return (P + (1 << a.lg_page) - 1) >> a.lg_page;
}

// The least e in [-100, 122] with top <= 127 * 2^e; top >= 0
__device__ __forceinline__ int least_exponent(float top) { return min(max((int)((__float_as_uint(top) + 0x1ffffu) >> 23) - 133, -100), 122); }

template <class T>
struct Sixteen {                     // values of a row
    float v[16];
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (std::is_same_v<T, float>) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(p + i * 4);
#pragma unroll
                for (int e = 0; e < 4; e++)
                    v[i * 4 + e] = x[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(p + i * 8);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    v[i * 8 + e * 2] = __uint_as_float(x[e] << 16);
                    v[i * 8 + e * 2 + 1] = __uint_as_float(x[e] & 0xffff0000u);
                }
            }
        }
    }
    __device__ __forceinline__ float top() const
    {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i++)
            t = __builtin_elementwise_maximum(t, __builtin_fabsf(v[i]));      // (a NaN stays)
        return t;
    }
};

__device__ __forceinline__ int byte_of(int x, int at) { return (x & 255) << (8 * at); }

template <class T, int UP>
__device__ __forceinline__ i32x4 bound_codes(const Sixteen<T> &x, float scale)
{
    i32x4 r = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const float y = x.v[i] * scale;
        r[i >> 2] |= byte_of((int)(UP ? ceilf(y) : floorf(y)), i & 3);
    }
    return r;
}

// A workgroup: 64 pages against 64 nodes of a sequence and KV head.
template <class T, int D>
__global__ __launch_bounds__(256) void score_kernel(SelectArgs a)
{
    constexpr int KS = D / 64, NSTR = 4 * D + 16;         // bytes of a node in LDS: positive hi, lo, negative hi, lo
    __shared__ __attribute__((aligned(16))) unsigned char s_q[NODES * NSTR];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int groups = (a.n_tree + NODES - 1) / NODES;
    const int b = blockIdx.z, kvh = blockIdx.y / groups, node0 = (blockIdx.y - kvh * groups) * NODES, n_nodes = min(NODES, a.n_tree - node0);
    const int n = pages_of(a, b), page0 = blockIdx.x * PAGES;
    // (only pages in between are ranked)
    if (page0 >= n - a.n_last || page0 + PAGES <= a.n_first)
        return;
    // the pages' bounds are on their way while the queries become whole numbers
    const int mine = min(page0 + wave * 16 + c, n - 1);
    const int id = min(max(a.table[(int64_t)b * a.max_pages + mine], 0), a.n_pages - 1);
    const T *bound = static_cast<const T *>(a.bounds) + ((int64_t)id * a.hkv + kvh) * 2 * D;
    Sixteen<T> u[KS], w[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
        u[ks].load(bound + ks * 64 + g * 16);
        w[ks].load(bound + D + ks * 64 + g * 16);
    }
    // ---- queries: D / 16 lanes a node
    constexpr int LANES = D / 16;
    for (int at = tid / LANES; at < (n_nodes + 15) / 16 * 16; at += 256 / LANES) {
        const int node = min(at, n_nodes - 1), part = tid % LANES;
        const T *q = static_cast<const T *>(a.q) + (((int64_t)b * a.n_tree + node0 + node) * a.hq + (int64_t)kvh * a.group) * D + part * 16;
        float top = 0.0f;
        for (int h = 0; h < a.group; h++) {
            Sixteen<T> x;
            x.load(q + (int64_t)h * D);
            top = fmaxf(top, x.top());
        }
#pragma unroll
        for (int s = 1; s < LANES; s *= 2)
            top = fmaxf(top, __shfl_xor(top, s));
        const float scale = __uint_as_float((uint32_t)(127 - least_exponent(top)) << 23);
        int pos[16], neg[16];
#pragma unroll
        for (int i = 0; i < 16; i++)
            pos[i] = neg[i] = 0;
        for (int h = 0; h < a.group; h++) {
            Sixteen<T> x;
            x.load(q + (int64_t)h * D);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int v = (int)rintf(x.v[i] * scale);
                pos[i] += max(v, 0);
                neg[i] += max(-v, 0);
            }
        }
        i32x4 d[4] = {};
#pragma unroll
        for (int i = 0; i < 16; i++) {
            d[0][i >> 2] |= byte_of(pos[i] >> 6, i & 3);
            d[1][i >> 2] |= byte_of(pos[i] & 63, i & 3);
            d[2][i >> 2] |= byte_of(neg[i] >> 6, i & 3);
            d[3][i >> 2] |= byte_of(neg[i] & 63, i & 3);
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
            *reinterpret_cast<i32x4 *>(s_q + at * NSTR + i * D + part * 16) = d[i];
    }
    // ---- this wave's sixteen pages
    float top = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ks++)
        top = __builtin_elementwise_maximum(top, __builtin_elementwise_maximum(u[ks].top(), w[ks].top()));
    top = __builtin_elementwise_maximum(top, __shfl_xor(top, 16));
    top = __builtin_elementwise_maximum(top, __shfl_xor(top, 32));
    const int e = top <= 3.4028234e38f ? least_exponent(top) : 1000;
    const float scale = __uint_as_float((uint32_t)(127 - min(e, 122)) << 23);
    i32x4 up[KS], down[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ks++) {
        up[ks] = bound_codes<T, 1>(u[ks], scale);
        down[ks] = bound_codes<T, 0>(w[ks], scale);
    }
    int exponent[4];
#pragma unroll
    for (int r = 0; r < 4; r++)
        exponent[r] = __shfl(e, 4 * g + r);
    __syncthreads();
    const int first = page0 + wave * 16 + 4 * g;
    for (int nt = 0; nt * 16 < n_nodes; nt++) {
        const unsigned char *row = s_q + (nt * 16 + c) * NSTR + g * 16;
        i32x4 hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0}, nhi = {0, 0, 0, 0}, nlo = {0, 0, 0, 0};
#pragma unroll
        for (int ks = 0; ks < KS; ks++) {
            auto part = [&](int i) { return *reinterpret_cast<const i32x4 *>(row + i * D + ks * 64); };
            hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[ks], part(0), hi, 0, 0, 0);
            lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(up[ks], part(1), lo, 0, 0, 0);
            nhi = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[ks], part(2), nhi, 0, 0, 0);
            nlo = __builtin_amdgcn_mfma_i32_16x16x64_i8(down[ks], part(3), nlo, 0, 0, 0);
        }
        const int node = nt * 16 + c;
        u32x4 key;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const float s = ldexpf((float)((hi[r] - nhi[r]) * 64 + (lo[r] - nlo[r])), exponent[r]);
            const uint32_t bits = __float_as_uint(exponent[r] > 122 ? INFINITY : s);
            key[r] = bits >> 31 ? ~bits : bits | 0x80000000u;      // in the scores' order
        }
        if (node < n_nodes)
            *reinterpret_cast<u32x4 *>(a.keys + (((int64_t)b * a.hkv + kvh) * a.n_tree + node0 + node) * a.stride + first) = key;
    }
}

// A workgroup per 64 nodes of a sequence and KV head, a wave per node.  VALUES: scores a lane holds (0: they are read again every time).
template <int VALUES>
__global__ __launch_bounds__(1024) void choose_kernel(SelectArgs a)
{
    __shared__ uint64_t s_words[RANGE];
    __shared__ uint32_t s_border[NODES], s_ties[NODES];      // scores above the border are in, and of those at it the pages below s_ties
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int b = blockIdx.z, kvh = blockIdx.y, node0 = blockIdx.x * NODES, n_nodes = min(NODES, a.n_tree - node0);
    const int n = pages_of(a, b), lo = min(a.n_first, n), hi = max(n - a.n_last, lo), between = hi - lo;
    const int words = (a.n_tree + 63) / 64;
    auto scores = [&](int node) { return a.keys + (((int64_t)b * a.hkv + kvh) * a.n_tree + node0 + node) * a.stride; };
    if (a.n_best > 0 && a.n_best < between) {
        for (int node = wave; node < n_nodes; node += waves) {
            const uint32_t *key = scores(node) + lo;
            uint32_t held[VALUES ? VALUES : 1];
            uint32_t most = 0u, least = ~0u;
            if constexpr (VALUES > 0) {
#pragma unroll
                for (int i = 0; i < VALUES; i++) {
                    const int at = i * 64 + lane;
                    held[i] = key[min(at, between - 1)];
                }
#pragma unroll
                for (int i = 0; i < VALUES; i++) {
                    most = max(most, held[i]);
                    least = min(least, held[i]);
                    held[i] = i * 64 + lane < between ? held[i] : 0u;      // (no score is 0: that would be a NaN's)
                }
            } else {
                for (int at = lane; at < between; at += 64) {
                    most = max(most, key[at]);
                    least = min(least, key[at]);
                }
            }
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                most = max(most, (uint32_t)__shfl_xor((int)most, s));
                least = min(least, (uint32_t)__shfl_xor((int)least, s));
            }
            auto count = [&](uint32_t from) {      // scores at or above it
                int sum = 0;
                if constexpr (VALUES > 0) {
#pragma unroll
                    for (int i = 0; i < VALUES; i++)
                        sum += __popcll(__ballot(held[i] >= from));
                } else {
                    for (int at = 0; at < between; at += 64)
                        sum += __popcll(__ballot(at + lane < between && key[min(at + lane, between - 1)] >= from));
                }
                return sum;
            };
            // count(from) >= n_best > count(above), above - from shrinking to 1
            uint32_t from = __builtin_amdgcn_readfirstlane((int)least), above = (uint32_t)__builtin_amdgcn_readfirstlane((int)most) + 1u;
            int have = between;
            while (have != a.n_best && above - from > 1u) {
                const uint32_t middle = from + (above - from) / 2u;
                const int k = count(middle);
                if (k >= a.n_best) {
                    from = middle;
                    have = k;
                } else {
                    above = middle;
                }
            }
            uint32_t ties = ~0u;
            if (have != a.n_best) {      // the equal scores at the border: the lower pages
                int room = a.n_best - count(from + 1u);
                for (int at = 0; at < between; at += 64) {
                    const uint64_t equal = __ballot(at + lane < between && key[min(at + lane, between - 1)] == from);
                    const int k = __popcll(equal);
                    if (k >= room) {      // the page behind the last one taken
                        const bool last = equal >> lane & 1 && __popcll(equal & ((2ull << lane) - 1)) == room;
                        ties = (uint32_t)(lo + at + __builtin_ctzll(__ballot(last)) + 1);
                        break;
                    }
                    room -= k;
                }
            }
            if (lane == 0) {
                s_border[node] = from;
                s_ties[node] = ties;
            }
        }
    }
    const uint64_t all = n_nodes == 64 ? ~0ull : (1ull << n_nodes) - 1;
    for (int page0 = 0; page0 < a.max_pages; page0 += RANGE) {
        const int pages = min(RANGE, a.max_pages - page0);
        __syncthreads();      // (the borders are there; the range before is written)
        for (int i = tid; i < pages; i += blockDim.x) {
            const int page = page0 + i;
            s_words[i] = page < n && (page < lo || page >= hi || a.n_best >= between) ? all : 0ull;
        }
        __syncthreads();
        if (a.n_best > 0 && a.n_best < between) {
            const int first = max(lo, page0), last = min(hi, page0 + pages);
            for (int node = wave; node < n_nodes; node += waves) {
                const uint32_t *key = scores(node);
                const uint32_t border = s_border[node], ties = s_ties[node];
                for (int page = first + lane; page < last; page += 64) {
                    const uint32_t x = key[page];
                    if (x > border || (x == border && (uint32_t)page < ties))
                        atomicOr(reinterpret_cast<unsigned long long *>(s_words + page - page0), 1ull << node);
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < pages; i += blockDim.x)
            a.page_nodes[(((int64_t)b * a.hkv + kvh) * a.max_pages + page0 + i) * words + blockIdx.x] = s_words[i];
    }
}

int select_stride(const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len)
{
    const int64_t rows = paged_rows(pages), live = (max_kv_len < rows ? max_kv_len : rows) - n_tree;
    return (int)align_up((size_t)ceil_div(live > 0 ? live : 1, pages->page_size), PAGES);
}

int check_select(const char *who, const dream_attn_desc *desc, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len)
{
    if (int rc = check_pages(who, desc, pages))
        return rc;
    if (n_tree < 1 || n_tree > DREAM_MAX_TREE || n_tree > paged_rows(pages))
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_tree %d outside [1, min(%d, max_pages * page_size)]", who, n_tree, DREAM_MAX_TREE);
    if (max_kv_len < n_tree)
        return fail(DREAM_ERR_INVALID_ARG, "%s: max_kv_len %lld is less than n_tree", who, (long long)max_kv_len);
    if (desc->n_q_heads / desc->n_kv_heads > 64)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: more than 64 query heads on a KV head", who);
    return DREAM_OK;
}

template <class T>
int launch_select(const SelectArgs &a, int D, int B, hipStream_t st)
{
    const int groups = ceil_div(a.n_tree, NODES);
    if (a.n_best > 0) {
        auto *score = D == 64 ? &score_kernel<T, 64> : D == 128 ? &score_kernel<T, 128> : &score_kernel<T, 256>;
        hipLaunchKernelGGL(score, dim3(a.stride / PAGES, a.hkv * groups, B), dim3(256), 0, st, a);
        if (int rc = check_launch("score_kernel"))
            return rc;
    }
    auto *choose = a.stride <= 256 ? &choose_kernel<4> : a.stride <= 2048 ? &choose_kernel<32> : &choose_kernel<0>;
    const int waves = a.n_tree >= 16 ? 16 : a.n_tree;
    hipLaunchKernelGGL(choose, dim3(groups, a.hkv, B), dim3(waves < 4 ? 256 : waves * 64), 0, st, a);
    return check_launch("choose_kernel");
}

}  // namespace

extern "C" {

size_t dream_page_select_workspace(const dream_attn_desc *desc, const dream_page_desc *pages, int32_t n_tree, int64_t max_kv_len)
{
    if (check_select("dream_page_select_workspace", desc, pages, n_tree, max_kv_len))
        return DREAM_WORKSPACE_MIN_BYTES;
    return (size_t)desc->batch * desc->n_kv_heads * n_tree * select_stride(pages, n_tree, max_kv_len) * 4 + DREAM_WORKSPACE_MIN_BYTES;
}

int dream_page_select(const dream_attn_desc *desc, const dream_page_desc *pages, const int32_t *page_table, const void *q, const void *bounds, const int32_t *prefix_len,
                      int32_t n_tree, int32_t n_first, int32_t n_last, int32_t n_best, int64_t max_kv_len, uint64_t *page_nodes, void *workspace, size_t workspace_bytes,
                      void *stream)
{
    const char *who = "dream_page_select";
    if (int rc = check_select(who, desc, pages, n_tree, max_kv_len))
        return rc;
    if (!page_table || !q || !bounds || !prefix_len || !page_nodes || !workspace)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_first < 0 || n_last < 0 || n_best < 0)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_first, n_last and n_best must not be negative", who);
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(bounds) | reinterpret_cast<uintptr_t>(workspace)) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: a tensor is not 16-byte aligned", who);
    if (workspace_bytes < dream_page_select_workspace(desc, pages, n_tree, max_kv_len))
        return fail(DREAM_ERR_WORKSPACE, "%s: workspace of %zu bytes is too small", who, workspace_bytes);
    SelectArgs a = {};
    const int64_t rows = paged_rows(pages), bound = max_kv_len < rows ? max_kv_len : rows;
    a.q = q; a.bounds = bounds; a.table = page_table; a.prefix_len = prefix_len; a.keys = static_cast<uint32_t *>(workspace); a.page_nodes = page_nodes;
    a.n_tree = n_tree; a.hq = desc->n_q_heads; a.hkv = desc->n_kv_heads; a.group = a.hq / a.hkv; a.lg_page = log2_of(pages->page_size); a.n_pages = pages->n_pages;
    a.max_pages = pages->max_pages; a.max_prefix = (int)(bound - n_tree); a.stride = select_stride(pages, n_tree, max_kv_len);
    a.n_first = n_first; a.n_last = n_last; a.n_best = n_best;
    const int groups = ceil_div(n_tree, NODES);
    if ((int64_t)a.hkv * groups > 65535)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: %d KV heads of %d nodes", who, a.hkv, n_tree);
    return desc->dtype == DREAM_F32 ? launch_select<float>(a, desc->head_dim, desc->batch, as_stream(stream)) : launch_select<uint16_t>(a, desc->head_dim, desc->batch, as_stream(stream));
}

}  // extern "C"
