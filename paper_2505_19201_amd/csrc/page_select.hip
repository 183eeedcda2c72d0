// dream_page_select: which pages of its prefix each node sees, by a bound of what its queries, as they are rounded here, score there.
//
// With a page's largest value U_d and smallest W_d in every channel, q . k <= sum_d max(q_d, 0) U_d + min(q_d, 0) W_d for each of its keys; summed over the query heads of a KV head that is one
// number for a node, a KV head and a page.  Queries and bounds are held as whole numbers up to 127 times a power of two (queries to nearest, bounds rounded outwards: the score bounds the products of the rounded queries).
// Two reasons: the sums are whole numbers, so no order of adding them changes which page comes first, and the matrix instruction takes 8-bit numbers at four times the rate.  What is lost is a
// step of 2^-7 of the largest value, of numbers that only rank pages.
//
// Two launches.  score_kernel: S^T = pages x nodes by v_mfma_i32_16x16x64_i8, the parts c+ against U and c- against W one behind the other.  The heads' numbers add up before the product (it is linear in
// them): the sum, at most 64 * 127, goes in as two numbers, 64 hi + lo.  choose_kernel: a wave per node finds the n_best-th score by halving the range of the scores, taken as whole numbers
// in their order, until as many lie above as are wanted; where equal scores straddle the border the lower pages win.  (Sixteen waves where there is one node and many pages.)
// What bounds them: trips to memory and, in the second, some twenty halvings one behind the other (8 sequences of 60 nodes, 250 pages of 64 rows, 8 KV heads of 128: 8.5 and 6.1 us; one node, 2047
// pages: 5.8 and 8.4; 4 sequences of 33 nodes, 376 pages, 8 KV heads of 256: 8.5 and 6.7).
#include <float.h>
#include <type_traits>
#include "paged.h"

using namespace dream;

namespace {

constexpr int NODES = 64;            // of a workgroup: the bits of a word
constexpr int PAGES = 64;            // of a workgroup of score_kernel: 16 for each wave
constexpr int RANGE = 2048;          // pages whose bits choose_kernel holds at a time where no lane holds their scores

struct SelectArgs {
    const void *q, *bounds;
    const int32_t *table, *prefix_len;
    uint32_t *keys;                  // [B, Hkv, n_tree, stride]
    uint64_t *page_nodes;
    int32_t n_tree, hq, hkv, group, lg_page, n_pages, max_pages, max_prefix, stride, n_first, n_last, n_best;
};

__device__ __forceinline__ int pages_of(const int32_t *prefix_len, int b, int max_prefix, int lg_page)
{
    const int P = min(max(uniform_load(prefix_len + b), 0), max_prefix);
    return (P + (1 << lg_page) - 1) >> lg_page;
}

// The least e in [-100, 122] with top <= 127 * 2^e; top >= 0
__device__ __forceinline__ int least_exponent(float top) { return min(max((int)((__float_as_uint(top) + 0x1ffffu) >> 23) - 133, -100), 122); }

// Sixteen values of a row as they stand in memory
template <class T>
struct Sixteen {
    static constexpr int N = sizeof(T);
    u32x4 raw[N];
    __device__ __forceinline__ void load(const T *p)
    {
#pragma unroll
        for (int i = 0; i < N; i++)
            raw[i] = reinterpret_cast<const u32x4 *>(p)[i];
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (std::is_same_v<T, float>)
            return __uint_as_float(raw[i >> 2][i & 3]);
        else
            return __uint_as_float(i & 1 ? raw[i >> 3][i >> 1 & 3] & 0xffff0000u : raw[i >> 3][i >> 1 & 3] << 16);
    }
    __device__ __forceinline__ float top() const
    {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; i++)
            t = __builtin_elementwise_maximum(t, __builtin_fabsf((*this)[i]));      // (a NaN stays)
        return t;
    }
};

// Lowest bytes of four numbers, in order
__device__ __forceinline__ uint32_t bytes_of(int a, int b, int c, int d)
{
    return __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u) | __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x04000c0cu);
}

template <class T, int UP>
__device__ __forceinline__ i32x4 bound_codes(const Sixteen<T> &x, float scale)
{
    i32x4 r;
    // (a product that is less than any float is still not 0: rounded outwards it is a whole step)
    auto code = [&](int i) {
        const float v = x[i], p = v * scale;
        return (int)(UP ? ceilf(v > 0.0f ? fmaxf(p, FLT_MIN) : p) : floorf(v < 0.0f ? fminf(p, -FLT_MIN) : p));
    };
#pragma unroll
    for (int i = 0; i < 4; i++)
        r[i] = (int)bytes_of(code(4 * i), code(4 * i + 1), code(4 * i + 2), code(4 * i + 3));
    return r;
}

// (Plain arguments: they are in registers when a wave starts.)
//
// A workgroup: 64 pages against 64 nodes of a sequence and KV head; waves 16 pages x 64 channels each.  Latency bounds it (a workgroup reads some 60 KB and multiplies for 300 clocks): everything
// that is read is asked for at the start, queries before they are needed twice over, bounds of pages before it is known whether they are live.
template <class T, int D>
__global__ __launch_bounds__(4 * D) void score_kernel(const int32_t *table, const T *queries, const T *bounds, const int32_t *prefix_len, int n_tree, int hq, int hkv, int group, int max_pages, int n_pages, int max_prefix,
                                                      int lg_page, int n_first, int n_last, int stride, uint32_t *keys)
{
    constexpr int KS = D / 64, NSTR = 4 * D + 16;         // bytes of a node in LDS: positive hi, lo, negative hi, lo
    constexpr int SSTR = PAGES + 17;                      // (a step of 17 banks from node to node)
    constexpr int HEADS = std::is_same_v<T, float> ? 2 : 4;      // that a lane holds at a time
    __shared__ __attribute__((aligned(16))) unsigned char s_q[NODES * NSTR];
    __shared__ int s_sum[NODES * SSTR], s_exponent[PAGES];
    __shared__ float s_top[KS][PAGES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4, pt = wave & 3, ks = wave >> 2;
    const int groups = (n_tree + NODES - 1) / NODES;
    const int b = blockIdx.z, kvh = blockIdx.y / groups, node0 = (blockIdx.y - kvh * groups) * NODES, n_nodes = min(NODES, n_tree - node0), page0 = blockIdx.x * PAGES;
    const int entry = table[(int64_t)b * max_pages + min(page0 + pt * 16 + c, max_pages - 1)];
    // ---- queries: D / 16 lanes a node
    constexpr int LANES = D / 16;
    const int at = tid / LANES, part = tid % LANES;
    const bool quantises = at < (n_nodes + 15) / 16 * 16;
    const T *q = queries + (((int64_t)b * n_tree + node0 + min(at, n_nodes - 1)) * hq + (int64_t)kvh * group) * D + part * 16;
    Sixteen<T> x[HEADS];
    auto heads_from = [&](int h) {                // (heads behind the last: the last again)
#pragma unroll
        for (int i = 0; i < HEADS; i++)
            x[i].load(q + (int64_t)min(h + i, group - 1) * D);
    };
    if (quantises)
        heads_from(0);
    // ---- bounds of this wave's sixteen pages
    const T *bound = bounds + ((int64_t)min(max(entry, 0), n_pages - 1) * hkv + kvh) * 2 * D + ks * 64 + g * 16;
    Sixteen<T> u, w;
    u.load(bound);
    w.load(bound + D);
    const int n = pages_of(prefix_len, b, max_prefix, lg_page);
    if (page0 >= n - n_last || page0 + PAGES <= n_first)      // (only pages in between are ranked)
        return;
    for (int i = tid; i < NODES * SSTR; i += 4 * D)
        s_sum[i] = 0;
    if (quantises) {
        float top = 0.0f;
        for (int h = 0;;) {
#pragma unroll
            for (int i = 0; i < HEADS; i++)
                top = fmaxf(top, x[i].top());
            h += HEADS;
            if (h >= group)
                break;
            heads_from(h);
        }
#pragma unroll
        for (int s = 1; s < LANES; s *= 2)
            top = fmaxf(top, __shfl_xor(top, s));
        const float scale = __uint_as_float((uint32_t)(127 - least_exponent(top)) << 23);
        float sum[16], size[16];                  // of the heads' whole numbers: at most 64 * 127, exact
#pragma unroll
        for (int i = 0; i < 16; i++)
            sum[i] = size[i] = 0.0f;
        for (int h = 0; h < group; h += HEADS) {
            if (group > HEADS)
                heads_from(h);
#pragma unroll
            for (int j = 0; j < HEADS; j++)
                if (h + j < group) {
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const float v = rintf(x[j][i] * scale);
                        sum[i] += v;
                        size[i] += __builtin_fabsf(v);
                    }
                }
        }
        // Two at a time as 16-bit halves: bits 6 to 13 are the quotient by 64, with its sign
        i32x4 d[4];
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint32_t two[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    auto part_of = [&](int j) { return (uint32_t)(int)((k ? sum[j] - size[j] : sum[j] + size[j]) * 0.5f); };
                    two[e] = __builtin_amdgcn_perm(part_of(4 * i + 2 * e + 1), part_of(4 * i + 2 * e), 0x05040100u);
                }
                d[2 * k][i] = (int)__builtin_amdgcn_perm(two[1] >> 6, two[0] >> 6, 0x06040200u);
                d[2 * k + 1][i] = (int)(__builtin_amdgcn_perm(two[1], two[0], 0x06040200u) & 0x3f3f3f3fu);
            }
#pragma unroll
        for (int i = 0; i < 4; i++)
            *reinterpret_cast<i32x4 *>(s_q + at * NSTR + i * D + part * 16) = d[i];
    }
    float top = __builtin_elementwise_maximum(u.top(), w.top());
    top = __builtin_elementwise_maximum(top, __shfl_xor(top, 16));
    top = __builtin_elementwise_maximum(top, __shfl_xor(top, 32));
    if (g == 0)
        s_top[ks][pt * 16 + c] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KS; i++)
        top = __builtin_elementwise_maximum(top, s_top[i][pt * 16 + c]);
    const int e = top <= 3.4028234e38f ? least_exponent(top) : 1000;
    const float scale = __uint_as_float((uint32_t)(127 - min(e, 122)) << 23);
    if (ks == 0 && g == 0)
        s_exponent[pt * 16 + c] = e;
    const i32x4 up = bound_codes<T, 1>(u, scale), down = bound_codes<T, 0>(w, scale);
    for (int nt = 0; nt * 16 < n_nodes; nt++) {
        const unsigned char *row = s_q + (nt * 16 + c) * NSTR + ks * 64 + g * 16;
        auto codes = [&](int i) { return *reinterpret_cast<const i32x4 *>(row + i * D); };
        i32x4 hi = {0, 0, 0, 0}, lo = {0, 0, 0, 0};
        hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(up, codes(0), hi, 0, 0, 0);
        lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(up, codes(1), lo, 0, 0, 0);
        hi = __builtin_amdgcn_mfma_i32_16x16x64_i8(down, codes(2), hi, 0, 0, 0);
        lo = __builtin_amdgcn_mfma_i32_16x16x64_i8(down, codes(3), lo, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; r++)
            atomicAdd(&s_sum[(nt * 16 + c) * SSTR + pt * 16 + 4 * g + r], hi[r] * 64 + lo[r]);      // (whole numbers: any order)
    }
    __syncthreads();
    for (int node = tid / 16; node < n_nodes; node += D / 4) {
        const int page = tid % 16 * 4;
        u32x4 key;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int exponent = s_exponent[page + r];
            const float s = ldexpf((float)s_sum[node * SSTR + page + r], exponent);
            const uint32_t bits = __float_as_uint(exponent > 122 ? INFINITY : s);
            key[r] = bits >> 31 ? ~bits : bits | 0x80000000u;      // in the scores' order
        }
        *reinterpret_cast<u32x4 *>(keys + (((int64_t)b * hkv + kvh) * n_tree + node0 + node) * stride + page0 + page) = key;
    }
}

// TEAM waves to a node (one, or all of the workgroup: its barriers are among those); VALUES: scores that a lane holds (0: they are read again every time; TEAM is 1 then).  The nodes' choices meet in LDS as one bit a page and leave it as
// their part of every page's word.
template <int VALUES, int TEAM>
__global__ __launch_bounds__(TEAM == 1 ? 512 : 1024) void choose_kernel(const uint32_t *keys, const int32_t *prefix_len, uint64_t *page_nodes, int n_tree, int hkv, int stride, int max_pages, int max_prefix, int lg_page,
                                                                         int n_first, int n_last, int n_best)
{
    static_assert(TEAM == 1 || TEAM == 16);
    constexpr int WAVES = TEAM == 1 ? 8 : 16, HERE = WAVES / TEAM, HELD = VALUES ? VALUES * TEAM * 64 : RANGE;      // nodes of a workgroup; pages that it holds at a time
    __shared__ uint64_t s_bits[HERE][HELD / 64];
    __shared__ uint32_t s_team[2][WAVES][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), member = wave % TEAM, at = wave / TEAM;
    const int b = blockIdx.z, kvh = blockIdx.y, node0 = blockIdx.x * HERE, node = min(node0 + at, n_tree - 1);
    const uint32_t *scores = keys + (((int64_t)b * hkv + kvh) * n_tree + node) * stride;
    // scores are asked for before it is known how many there are (the array has as many as a lane asks for, of pages that may be none)
    uint32_t held[VALUES ? VALUES : 1];
    if constexpr (VALUES > 0) {
#pragma unroll
        for (int i = 0; i < VALUES; i++)
            held[i] = n_best > 0 ? scores[min((i * TEAM + member) * 64 + lane, stride - 1)] : 0u;
    }
    const int n = pages_of(prefix_len, b, max_prefix, lg_page), lo = min(n_first, n), hi = max(n - n_last, lo), between = hi - lo;
    const bool ranked = n_best > 0 && n_best < between;
    uint32_t border = 0u, ties = ~0u;             // scores above the border are in, and of those at it the pages below `ties`
    if (ranked) {
        uint32_t most = 0u, least = ~0u;
        if constexpr (VALUES > 0) {
#pragma unroll
            for (int i = 0; i < VALUES; i++) {
                const int page = (i * TEAM + member) * 64 + lane;
                const bool in = page >= lo && page < hi;
                most = in ? max(most, held[i]) : most;
                least = in ? min(least, held[i]) : least;
                held[i] = in ? held[i] : 0u;      // (no score is 0: that would be a NaN's)
            }
        } else {
            for (int page = lo + lane; page < hi; page += 64) {
                most = max(most, scores[page]);
                least = min(least, scores[page]);
            }
        }
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            most = max(most, (uint32_t)__shfl_xor((int)most, s));
            least = min(least, (uint32_t)__shfl_xor((int)least, s));
        }
        int turn = 0;
        if constexpr (TEAM > 1) {
            if (lane == 0) {
                s_team[1][wave][0] = most;
                s_team[1][wave][1] = least;
            }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < TEAM; w++) {
                most = max(most, s_team[1][at * TEAM + w][0]);
                least = min(least, s_team[1][at * TEAM + w][1]);
            }
        }
        auto count = [&](uint32_t from) {         // scores at or above it; by all of the team, as often
            int sum = 0;
            if constexpr (VALUES > 0) {
#pragma unroll
                for (int i = 0; i < VALUES; i++)
                    sum += __popcll(__ballot(held[i] >= from));
            } else {
                for (int page = lo; page < hi; page += 64)
                    sum += __popcll(__ballot(page + lane < hi && scores[min(page + lane, hi - 1)] >= from));
            }
            if constexpr (TEAM > 1) {
                if (lane == 0)
                    s_team[0][wave][turn] = sum;
                __syncthreads();
                sum = 0;
#pragma unroll
                for (int w = 0; w < TEAM; w++)
                    sum += s_team[0][at * TEAM + w][turn];
                sum = __builtin_amdgcn_readfirstlane(sum);
                turn ^= 1;
            }
            return sum;
        };
        // count(from) >= n_best > count(above), above - from shrinking to 1
        uint32_t from = __builtin_amdgcn_readfirstlane((int)least), above = (uint32_t)__builtin_amdgcn_readfirstlane((int)most) + 1u;
        int have = between, over = 0;
        while (have != n_best && above - from > 1u) {
            const uint32_t middle = from + (above - from) / 2u;
            const int k = count(middle);
            if (k >= n_best) {
                from = middle;
                have = k;
            } else {
                above = middle;
                over = k;
            }
        }
        border = from;
        if (have != n_best) {                   // the equal scores at the border (`over` are above it): the lower pages
            int room = n_best - over;
            if constexpr (TEAM == 1) {
                for (int page = lo & ~63; page < hi; page += 64) {
                    const uint64_t equal = __ballot(page + lane >= lo && page + lane < hi && scores[min(max(page + lane, lo), hi - 1)] == from);
                    const int k = __popcll(equal);
                    if (k >= room) {              // the page behind the last one taken
                        const bool last = equal >> lane & 1 && __popcll(equal & ((2ull << lane) - 1)) == room;
                        ties = (uint32_t)(page + __builtin_ctzll(__ballot(last)) + 1);
                        break;
                    }
                    room -= k;
                }
            } else {
                // by halving again: the least page with `room` equal ones below it
                uint32_t low = 0u, high = (uint32_t)hi;
                while (high - low > 1u) {
                    const uint32_t middle = low + (high - low) / 2u;
                    int sum = 0;
#pragma unroll
                    for (int i = 0; i < (VALUES ? VALUES : 1); i++)
                        sum += __popcll(__ballot(held[i] == from && (uint32_t)((i * TEAM + member) * 64 + lane) < middle));
                    if (lane == 0)
                        s_team[0][wave][turn] = sum;
                    __syncthreads();
                    sum = 0;
#pragma unroll
                    for (int w = 0; w < TEAM; w++)
                        sum += s_team[0][at * TEAM + w][turn];
                    turn ^= 1;
                    if (__builtin_amdgcn_readfirstlane(sum) >= room)
                        high = middle;
                    else
                        low = middle;
                }
                ties = high;
            }
        }
    }
    auto takes = [&](int page, uint32_t score) {
        return page < n && (page < lo || page >= hi || (n_best > 0 && (!ranked || score > border || (score == border && (uint32_t)page < ties))));
    };
    const int words = (n_tree + 63) / 64, rest = n_tree - node0;      // nodes from this workgroup's first on
    const bool there = node0 + at < n_tree;
    uint64_t *out = page_nodes + ((int64_t)b * hkv + kvh) * max_pages * words + node0 / 64;
    const int live = min(n, max_pages);
    for (int page0 = 0; page0 < live; page0 += HELD) {      // (pages that lanes hold are all there are)
        __syncthreads();                          // (the range before is written)
        if constexpr (VALUES > 0) {
#pragma unroll
            for (int i = 0; i < VALUES; i++) {
                const int page = (i * TEAM + member) * 64 + lane;
                const uint64_t bits = there ? __ballot(takes(page, held[i])) : 0ull;
                if (lane == 0)
                    s_bits[at][i * TEAM + member] = bits;
            }
        } else {
            for (int i = 0; i < HELD / 64; i++) {
                const int page = page0 + i * 64 + lane;
                const uint64_t bits = there ? __ballot(takes(page, scores[min(page, stride - 1)])) : 0ull;
                if (lane == 0)
                    s_bits[at][i] = bits;
            }
        }
        __syncthreads();
        for (int i = tid; i < min(HELD, live - page0); i += 64 * WAVES) {
            uint32_t mine = 0u;
#pragma unroll
            for (int w = 0; w < HERE; w++)
                mine |= (uint32_t)(s_bits[w][i >> 6] >> (i & 63) & 1) << w;
            uint64_t *word = out + (int64_t)(page0 + i) * words;
            const int first = node0 & 63;         // of the word's bits; the last workgroup of a word writes what is left of it
            if (first == 0 && rest <= HERE)
                *word = mine;
            else if (HERE > 1) {
                uint8_t *parts = reinterpret_cast<uint8_t *>(word);
                parts[first / 8] = (uint8_t)mine;
                if (rest <= HERE)
                    for (int k = first / 8 + 1; k < 8; k++)
                        parts[k] = 0;
            }
        }
    }
    if ((node0 & 63) == 0)                        // words of pages that there are not
        for (int page = live + tid; page < max_pages; page += 64 * WAVES)
            out[(int64_t)page * words] = 0ull;
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
        hipLaunchKernelGGL(score, dim3(a.stride / PAGES, a.hkv * groups, B), dim3(4 * D), 0, st, a.table, static_cast<const T *>(a.q), static_cast<const T *>(a.bounds), a.prefix_len, a.n_tree, a.hq,
                           a.hkv, a.group, a.max_pages, a.n_pages, a.max_prefix, a.lg_page, a.n_first, a.n_last, a.stride, a.keys);
        if (int rc = check_launch("score_kernel"))
            return rc;
    }
    auto choose = [&](auto kernel, int nodes, int threads) {      // nodes of a workgroup
        hipLaunchKernelGGL(kernel, dim3(ceil_div(a.n_tree, nodes), a.hkv, B), dim3(threads), 0, st, a.keys, a.prefix_len, a.page_nodes, a.n_tree, a.hkv, a.stride, a.max_pages, a.max_prefix, a.lg_page, a.n_first,
                           a.n_last, a.n_best);
    };
    // One token, many pages: all of a workgroup's waves rank them together.  (With the scores, sixteen waves and one, us: 500 pages 12.0 and 10.3, 1000 13.0 and 13.6, 2000 14.4 and 21.0; of eight
    // sequences 16.5 and 13.3, 21.7 and 21.5, 30.6 and 36.9.)
    if (a.n_tree == 1 && a.stride > 1024 && a.stride <= 8192)
        choose(a.stride <= 2048 ? &choose_kernel<2, 16> : &choose_kernel<8, 16>, 1, 1024);
    else
        choose(a.stride <= 128    ? &choose_kernel<2, 1>
               : a.stride <= 256  ? &choose_kernel<4, 1>
               : a.stride <= 512  ? &choose_kernel<8, 1>
               : a.stride <= 1024 ? &choose_kernel<16, 1>
               : a.stride <= 2048 ? &choose_kernel<32, 1>
                                  : &choose_kernel<0, 1>,
               8, 512);
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
