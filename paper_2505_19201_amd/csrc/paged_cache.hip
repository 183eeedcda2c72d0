// Rows of caches held in pages: dream_paged_append, dream_paged_commit, dream_page_bounds.  (The attention over them: attn_paged.hip, page_select.hip.)
//
// Append.  A pair (x, y) of a row at position p becomes amplitude * (x cos a - y sin a, x sin a + y cos a), a = p * inv_freq[i], as in rotary.hip: the angle formed and reduced to a part of a
// turn in 64 bits, the turn in float32, rounded once to the row's type.  Queries turn into a dense tensor, keys turn and values go as they are into the pages: one launch, each row read
// once and written once.
// Commit.  The accepted path's rows move up, in all layers' pools by one launch: everything a workgroup moves is in registers before it writes any of it.  (40 pools of 8 heads of 128: 3.7 us, four
// trips to memory.)
// Bounds.  The largest and smallest value of each channel of a page: a page and head is one contiguous run of page_size * D values.  (A prompt's 39 MB in 10.2 us, 3.8 TB/s; a round's pages in 3.5.)
#include <float.h>
#include <type_traits>
#include "paged.h"
#include "quick_div.h"

namespace dream {

int check_pages(const char *who, const dream_attn_desc *desc, const dream_page_desc *pages)
{
    if (!desc || !pages)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL descriptor", who);
    if (desc->dtype != DREAM_F32 && desc->dtype != DREAM_BF16)
        return fail(DREAM_ERR_INVALID_ARG, "%s: unknown dtype %d", who, desc->dtype);
    if (desc->head_dim != 64 && desc->head_dim != 128 && desc->head_dim != 256)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: head_dim %d is not 64, 128 or 256", who, desc->head_dim);
    if (desc->batch < 1 || desc->batch > 65535)
        return fail(DREAM_ERR_INVALID_ARG, "%s: batch %d outside [1, 65535]", who, desc->batch);
    if (desc->n_kv_heads < 1 || desc->n_q_heads < 1 || desc->n_q_heads > 4096 || desc->n_q_heads % desc->n_kv_heads)
        return fail(DREAM_ERR_INVALID_ARG, "%s: %d query heads on %d KV heads", who, desc->n_q_heads, desc->n_kv_heads);
    const int32_t ps = pages->page_size;
    if (ps < MIN_PAGE || ps > MAX_PAGE || (ps & (ps - 1)))
        return fail(DREAM_ERR_UNSUPPORTED, "%s: page_size %d is not 16, 32, 64, 128 or 256", who, ps);
    if (pages->n_pages < 1 || pages->max_pages < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_pages and max_pages must be positive", who);
    if (paged_rows(pages) > DREAM_MAX_WINDOW_ROWS)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: max_pages * page_size exceeds %d", who, DREAM_MAX_WINDOW_ROWS);
    return DREAM_OK;
}

}  // namespace dream

using namespace dream;

namespace {

// ---- append ----------------------------------------------------------------------------------------------------------
constexpr int BATCH = 4;           // pieces a thread has in flight

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out, *k_pages, *v_pages;
    const int32_t *table, *row_base, *row_index, *n_live, *pos, *pos_base, *parent;
    const float *inv_freq;
    int32_t n_rows, hq, hkv, head_dim, rot, lg_page, n_pages, max_pages;
    int32_t pieces;                // of a head that may turn; of a value's head 16 bytes each
    int32_t end_q, end_k, end_v;   // of a row's pieces: queries, keys, values
    uint32_t rows_magic, pieces_magic, vpieces_magic;      // for quick_div; 0: divide
    float amplitude;
};

// N neighbouring values as they stand in memory: 16 bytes as words (as an array of values they would be kept in memory, not in registers), or one or two values
template <class T, int N>
struct Piece {
    static constexpr bool WIDE = sizeof(T) * N == 16, NARROW_TYPE = sizeof(T) == 2;
    using Raw = std::conditional_t<WIDE, u32x4, T[N]>;
    Raw raw;
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (WIDE) {
            raw = *reinterpret_cast<const u32x4 *>(p);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                raw[i] = p[i];
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (WIDE) {
            *reinterpret_cast<u32x4 *>(p) = raw;
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                p[i] = raw[i];
        }
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (!NARROW_TYPE)
            return WIDE ? __uint_as_float(raw[i]) : raw[i];
        else if constexpr (WIDE)
            return __uint_as_float(i & 1 ? raw[i / 2] & 0xffff0000u : raw[i / 2] << 16);
        else
            return bf16_bits_to_float(raw[i]);
    }
    // Values i and i + 1 (i alone, if it is the only one), each rounded once to the type
    __device__ __forceinline__ void set(int i, float x, float y)
    {
        if constexpr (!NARROW_TYPE && WIDE) {
            raw[i] = __float_as_uint(x);
            raw[i + 1] = __float_as_uint(y);
        } else if constexpr (!NARROW_TYPE) {
            raw[i] = x;
            if constexpr (N > 1)
                raw[i + 1] = y;
        } else if constexpr (WIDE) {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            raw[i / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
        } else {
            raw[i] = __builtin_bit_cast(uint16_t, (__bf16)x);
            if constexpr (N > 1)
                raw[i + 1] = __builtin_bit_cast(uint16_t, (__bf16)y);
        }
    }
};

// The value of something that is the same in every lane
template <class V>
__device__ __forceinline__ V here(V v)
{
    asm volatile("" : "+s"(v));
    return v;
}

// One workgroup per row, or where there are few rows several: a row's angles are formed once and lie in LDS while its first pieces are on their way.  A thread takes pieces of a head, N values each
// (in the half layout with the N values rot / 2 further on).  What the first loads need are
// plain arguments, in registers when a wave starts, and what a piece chooses from is chosen by value (of
// variables the compiler chooses an address instead, in a copy of theirs in memory: 312 bytes a thread).  PAIRED: the pairs are neighbours (2i, 2i + 1); else (i, i + rot / 2).
template <class T, bool PAIRED, int N>
__global__ __launch_bounds__(256) void append_kernel(const int32_t *row_base, const int32_t *table, const int32_t *pos_base, const T *q, const T *k, const T *v, int n_rows, uint32_t rows_magic, int max_pages, int lg_page,
                                                                int hq, int hkv, uint32_t pieces_magic, uint32_t vpieces_magic, T *q_out, T *k_pages, T *v_pages, AppendArgs a)
{
    constexpr int NV = 16 / sizeof(T);               // values of a piece that does not turn
    __shared__ float2 s_turn[128];
    const int tid = threadIdx.x;
    const int b = rows_magic ? quick_div(blockIdx.x, rows_magic) : blockIdx.x / n_rows, r = blockIdx.x - b * n_rows;
    const int D = a.head_dim, rot = a.rot, half = rot / 2, pieces = a.pieces;
    const int turned = rot ? (PAIRED ? rot : half) / N : 0;     // pieces of a head that turn; the others are copied
    const int stride = gridDim.y * 256;
    const bool walk = rot && a.parent && !a.pos;
    // all that the position and the place need is requested before anything is waited for
    int32_t par[DREAM_MAX_TREE / 64];                 // every wave holds the tree, lane l nodes l, 64 + l, ...
#pragma unroll
    for (int i = 0; i < DREAM_MAX_TREE / 64; i++) {
        const int node = i * 64 + (tid & 63);
        par[i] = walk && node < n_rows ? a.parent[(int64_t)b * n_rows + node] : -1;
    }
    const int live = a.n_live ? uniform_load(a.n_live + b) : n_rows;
    const int base = uniform_load(row_base + b), start = !rot ? 0 : a.pos ? uniform_load(a.pos + blockIdx.x) : pos_base ? uniform_load(pos_base + b) : base;
    const int64_t row = (int64_t)base + (a.row_index ? uniform_load(a.row_index + blockIdx.x) : r);
    const float freq = rot ? a.inv_freq[tid < half ? tid : 0] : 0.0f;
    if (r >= live)
        return;
    const int page = row >= 0 && row >> lg_page < max_pages ? uniform_load(table + (int64_t)b * max_pages + (row >> lg_page)) : -1;
    Piece<T, N> x[BATCH], y[BATCH];
    Piece<T, NV> w[BATCH];
    auto source = [&](int idx, bool &value, int &h, int &it) {      // of piece idx: its tensor's row of heads, its head and its place there
        value = idx >= a.end_k;
        const T *src = idx < a.end_q ? here(q) : value ? here(v) : here(k);
        const int at = idx - (idx < a.end_q ? 0 : value ? here(a.end_k) : here(a.end_q)), per = value ? D / NV : pieces;
        const uint32_t magic = value ? here(vpieces_magic) : here(pieces_magic);
        h = magic ? quick_div(at, magic) : at / per;
        it = at - h * per;
        return src + ((int64_t)blockIdx.x * (idx < a.end_q ? here(hq) : here(hkv)) + h) * D;
    };
    auto channel = [&](int it) { return PAIRED || it < turned ? it * N : it * N + half; };
    // all of a thread's pieces are on their way before the position is known; BATCH of them are all there are (launch_append)
    const int first = blockIdx.y * 256;
#pragma unroll
    for (int u = 0; u < BATCH; u++) {
        const int idx = first + u * stride + tid;
        if (idx < a.end_v) {
            bool value;
            int h, it;
            const T *src = source(idx, value, h, it);
            if constexpr (N == NV) {              // a value's piece is one that does not turn
                x[u].load(src + (value ? it * N : channel(it)));
            } else if (value) {
                w[u].load(src + it * NV);
            } else {
                x[u].load(src + channel(it));
            }
            if (!PAIRED && !value && it < turned)
                y[u].load(src + channel(it) + half);
        }
    }
    int64_t pos = start;
    if (walk) {
        int p = r;
        for (int step = 0;; step++) {
            int32_t up = par[0];
#pragma unroll
            for (int i = 1; i < DREAM_MAX_TREE / 64; i++)
                up = p >> 6 == i ? par[i] : up;
            up = __builtin_amdgcn_readlane(up, p & 63);
            if (up < 0 || up >= p) {                  // (a parent behind its node is none: a walk up the tree always ends)
                pos += step;
                break;
            }
            p = up;
        }
    } else if (!a.pos) {
        pos += r;
    }
    if (tid < half) {
        const double turns = (double)pos * (double)freq * 0.15915494309189533577;
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        s_turn[tid] = make_float2(c * a.amplitude, s * a.amplitude);
    }
    __syncthreads();
    const bool kept = page >= 0 && page < a.n_pages;
    const int64_t in_pool = (((int64_t)(kept ? page : 0) * hkv << lg_page) + (row & ((1 << lg_page) - 1))) * D;      // of head 0
#pragma unroll
    for (int u = 0; u < BATCH; u++) {
        const int idx = first + u * stride + tid;
        if (idx >= a.end_v || (idx >= a.end_q && !kept))
            continue;
        bool value;
        int h, it;
        source(idx, value, h, it);
        T *dst = idx < a.end_q ? here(q_out) + ((int64_t)blockIdx.x * here(hq) + h) * D
                               : (value ? here(v_pages) : here(k_pages)) + in_pool + ((int64_t)h << lg_page) * D;
        if (N != NV && value) {
            w[u].store(dst + it * NV);
            continue;
        }
        if (!value && it < turned) {
            if constexpr (PAIRED) {
#pragma unroll
                for (int i = 0; i < N; i += 2) {
                    const float2 t = s_turn[it * (N / 2) + i / 2];
                    const float p = x[u][i], q = x[u][i + 1];
                    x[u].set(i, p * t.x - q * t.y, p * t.y + q * t.x);
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; i += 2) {
                    constexpr int SECOND = N > 1;
                    const float2 t0 = s_turn[it * N + i], t1 = s_turn[it * N + i + SECOND];
                    const float p0 = x[u][i], q0 = y[u][i], p1 = x[u][i + SECOND], q1 = y[u][i + SECOND];
                    x[u].set(i, p0 * t0.x - q0 * t0.y, p1 * t1.x - q1 * t1.y);
                    y[u].set(i, p0 * t0.y + q0 * t0.x, p1 * t1.y + q1 * t1.x);
                }
                y[u].store(dst + channel(it) + half);
            }
        }
        x[u].store(dst + (value ? it * N : channel(it)));
    }
}

template <class T>
int launch_append(const AppendArgs &a, bool paired, bool wide, int64_t rows, hipStream_t st)
{
    constexpr int N = 16 / sizeof(T);
    auto *kernel = paired ? (wide ? &append_kernel<T, true, N> : &append_kernel<T, true, 2>) : wide ? &append_kernel<T, false, N> : &append_kernel<T, false, 1>;
    // workgroups of a row: at least so many that a thread has all of its pieces in flight, parts * 256 * BATCH >= end_v, which append_kernel relies on (685 rows of 96 float32 heads of 128 18.2 -> 15.4 us)
    const int64_t most = (a.end_v + 255) / 256, least = (a.end_v + 256 * BATCH - 1) / (256 * BATCH), parts = 1024 / rows > least ? 1024 / rows : least;
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows, (unsigned)(parts < 1 ? 1 : parts < most ? parts : most)), dim3(256), 0, st, a.row_base, a.table,
                       a.pos_base, static_cast<const T *>(a.q), static_cast<const T *>(a.k), static_cast<const T *>(a.v), a.n_rows, a.rows_magic, a.max_pages, a.lg_page, a.hq, a.hkv, a.pieces_magic,
                       a.vpieces_magic, static_cast<T *>(a.q_out), static_cast<T *>(a.k_pages), static_cast<T *>(a.v_pages), a);
    return check_launch("append_kernel");
}

// ---- commit ----------------------------------------------------------------------------------------------------------
constexpr int POOLS_PER_LAUNCH = 128;
constexpr int CHUNKS_PER_THREAD = 16;   // 256 threads x 16 chunks x 16 bytes = 64 KB of rows per workgroup

struct PagedCommitArgs {
    const int32_t *table, *accept_len, *path, *prefix_len;
    int32_t *prefix_len_out;
    int32_t hkv, heads_per_wg, path_stride, n_tree, cpr, lg_page, n_pages, max_pages, first_pool;
    void *pool[POOLS_PER_LAUNCH];
};

// Where node `node`'s row of head h starts, in 16-byte chunks; -1 outside the pool
__device__ __forceinline__ int64_t tree_chunk(const PagedCommitArgs &a, int b, int P, int node, int h)
{
    const int row = P + node, page = a.table[(int64_t)b * a.max_pages + (row >> a.lg_page)];
    if (page < 0 || page >= a.n_pages)
        return -1;
    return ((((int64_t)page * a.hkv + h) << a.lg_page) + (row & ((1 << a.lg_page) - 1))) * a.cpr;
}

template <int N>
__device__ __forceinline__ void move_paged(const PagedCommitArgs &a, u32x4 *pool, int b, int P, int h0, int total, int per_head)
{
    const int tid = threadIdx.x;
    u32x4 r[N];
    int64_t to[N];
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int idx = min(tid + i * 256, total - 1);
        const int hl = idx / per_head, rest = idx - hl * per_head;
        const int j = rest / a.cpr, c = rest - j * a.cpr;
        const int node = min(max(a.path[(int64_t)b * a.path_stride + j], 0), a.n_tree - 1);
        const int64_t from = tree_chunk(a, b, P, node, h0 + hl);
        to[i] = tree_chunk(a, b, P, j, h0 + hl);
        to[i] = from < 0 || to[i] < 0 ? -1 : to[i] + c;
        r[i] = pool[max(from, (int64_t)0) + c];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();   // every source chunk of these heads is in a register
#pragma unroll
    for (int i = 0; i < N; i++)
        if (tid + i * 256 < total && to[i] >= 0)
            pool[to[i]] = r[i];
}

__global__ __launch_bounds__(256) void paged_commit_kernel(PagedCommitArgs a)
{
    const int b = blockIdx.y;
    const int prefix = uniform_load(a.prefix_len + b), accepted = uniform_load(a.accept_len + b);
    const int h0 = blockIdx.x * a.heads_per_wg, n_heads = min(a.heads_per_wg, a.hkv - h0);
    const int P = min(max(prefix, 0), (a.max_pages << a.lg_page) - a.n_tree);
    // device metadata is trusted, but stay inside the tree rows whatever it holds
    const int n = min(max(accepted, 0), min(a.path_stride, a.n_tree) - 1);
    if (blockIdx.x == 0 && blockIdx.z == 0 && a.first_pool == 0 && threadIdx.x == 0 && a.prefix_len_out)
        a.prefix_len_out[b] = P + n + 1;
    const int per_head = (n + 1) * a.cpr, total = n_heads * per_head;
    u32x4 *pool = static_cast<u32x4 *>(a.pool[blockIdx.z]);
    if (total <= 256)
        move_paged<1>(a, pool, b, P, h0, total, per_head);
    else if (total <= 512)
        move_paged<2>(a, pool, b, P, h0, total, per_head);
    else if (total <= 1024)
        move_paged<4>(a, pool, b, P, h0, total, per_head);
    else
        move_paged<CHUNKS_PER_THREAD>(a, pool, b, P, h0, total, per_head);
}

// ---- bounds ----------------------------------------------------------------------------------------------------------
struct BoundsArgs {
    const void *k;
    void *bounds;
    const int32_t *table, *from_len, *to_len;
    int32_t hkv, lg_page, n_pages, max_pages, slots;
};

// A page of a sequence's run and head: TEAM waves, 4 (a workgroup) or, where that is at most 8 KB, or 16 of many, 1.  A thread has 16 bytes of a row, the rows of a page are shared out over 64 TEAM / (row / 16) threads;
// those of a wave meet by exchange, the waves in LDS.  (Plain arguments: they are in registers when a wave starts.)  Four waves and one, us: 126
// pages of 32 heads of 64, 4 KB 13.5 and 6.5, 66 of 8 KB 9.4 and 6.0; 256 of 8 heads of 128, 16 KB 8.3 and 7.1; 128 of 8 heads of 256, 16 KB 4.95 both; one of 8 heads, 8 KB 4.2 and 4.1, 16 KB 4.1 and 4.8.
template <class T, int D, int TEAM>
__global__ __launch_bounds__(256) void bounds_kernel(const int32_t *table, const int32_t *from_len, const int32_t *to_len, const T *k, int lg_page, int max_pages, int n_pages, int hkv, int slots, T *bounds)
{
    constexpr int N = 16 / sizeof(T), PER_ROW = D / N, ROWS = 64 * TEAM / PER_ROW;
    __shared__ __attribute__((aligned(16))) float s_ends[TEAM == 4 ? 4 : 1][2][D];      // of a wave's rows: largest and smallest
    const int wave = threadIdx.x >> 6, tid = TEAM == 4 ? threadIdx.x : threadIdx.x & 63, c = tid % PER_ROW, r0 = tid / PER_ROW;
    const int b = blockIdx.z, h = TEAM == 4 ? blockIdx.y : blockIdx.y * 4 + wave;
    const int ps = 1 << lg_page, rows = max_pages << lg_page;
    const int from = from_len ? min(max(uniform_load(from_len + b), 0), rows) : 0, to = min(uniform_load(to_len + b), rows);
    if (to <= from || h >= hkv)
        return;
    for (int i = (from >> lg_page) + blockIdx.x; (i << lg_page) < to; i += slots) {
        const int page = uniform_load(table + (int64_t)b * max_pages + i);
        if (page < 0 || page >= n_pages)
            continue;
        const int live = min(ps, to - (i << lg_page));
        const T *src = k + (((int64_t)page * hkv + h) << lg_page) * D + c * N;
        float most[N], least[N];
#pragma unroll
        for (int e = 0; e < N; e++)
            most[e] = -INFINITY, least[e] = INFINITY;
#pragma unroll 4
        for (int r = r0; r < live; r += ROWS) {
            Piece<T, N> x;
            x.load(src + (int64_t)r * D);
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float v = x[e];
                const bool finite = fabsf(v) <= FLT_MAX;
                most[e] = fmaxf(most[e], finite ? v : INFINITY);
                least[e] = fminf(least[e], finite ? v : -INFINITY);
            }
        }
#pragma unroll
        for (int d = PER_ROW; d < 64; d *= 2)
#pragma unroll
            for (int e = 0; e < N; e++) {
                most[e] = fmaxf(most[e], __shfl_xor(most[e], d));
                least[e] = fminf(least[e], __shfl_xor(least[e], d));
            }
        if constexpr (TEAM == 4) {
            if ((tid & 63) < PER_ROW)
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    *reinterpret_cast<f32x4 *>(&s_ends[wave][0][c * N + e]) = f32x4{most[e], most[e + 1], most[e + 2], most[e + 3]};
                    *reinterpret_cast<f32x4 *>(&s_ends[wave][1][c * N + e]) = f32x4{least[e], least[e + 1], least[e + 2], least[e + 3]};
                }
            __syncthreads();
        }
        if (tid < PER_ROW) {
            Piece<T, N> up, down;
#pragma unroll
            for (int e = 0; e < N; e++) {
                if constexpr (TEAM == 4) {
                    most[e] = s_ends[0][0][tid * N + e], least[e] = s_ends[0][1][tid * N + e];
#pragma unroll
                    for (int w = 1; w < 4; w++) {
                        most[e] = fmaxf(most[e], s_ends[w][0][tid * N + e]);
                        least[e] = fminf(least[e], s_ends[w][1][tid * N + e]);
                    }
                }
                const bool finite = most[e] <= FLT_MAX && least[e] >= -FLT_MAX;
                most[e] = finite ? most[e] : INFINITY;
                least[e] = finite ? least[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                up.set(e, most[e], most[e + 1]);
                down.set(e, least[e], least[e + 1]);
            }
            T *dst = bounds + ((int64_t)page * hkv + h) * 2 * D + tid * N;
            up.store(dst);
            down.store(dst + D);
        }
        if constexpr (TEAM == 4)
            __syncthreads();
    }
}

template <class T>
int launch_bounds(const BoundsArgs &a, int D, int B, hipStream_t st)
{
    const int64_t bytes = (int64_t)D * sizeof(T) << a.lg_page, units = (int64_t)a.slots * a.hkv * B;
    const bool small = bytes <= 8192 || (bytes <= 16384 && units >= 2048);
    auto *kernel = D == 64    ? (small ? &bounds_kernel<T, 64, 1> : &bounds_kernel<T, 64, 4>)
                   : D == 128 ? (small ? &bounds_kernel<T, 128, 1> : &bounds_kernel<T, 128, 4>)
                              : (small ? &bounds_kernel<T, 256, 1> : &bounds_kernel<T, 256, 4>);
    hipLaunchKernelGGL(kernel, dim3(a.slots, small ? (a.hkv + 3) / 4 : a.hkv, B), dim3(256), 0, st, a.table, a.from_len, a.to_len, static_cast<const T *>(a.k), a.lg_page, a.max_pages, a.n_pages, a.hkv, a.slots,
                       static_cast<T *>(a.bounds));
    return check_launch("bounds_kernel");
}

}  // namespace

extern "C" {

int dream_paged_append(const dream_attn_desc *desc, const dream_page_desc *pages, const int32_t *page_table, const void *q, const void *k, const void *v, int32_t n_rows,
                       const int32_t *row_base, const int32_t *row_index, const int32_t *n_live, const int32_t *pos, const int32_t *pos_base, const int32_t *parent,
                       const float *inv_freq, int32_t rot_dim, int32_t interleaved, float amplitude, void *q_out, void *k_pages, void *v_pages, void *stream)
{
    const char *who = "dream_paged_append";
    if (int rc = check_pages(who, desc, pages))
        return rc;
    if (!page_table || !k || !v || !row_base || !k_pages || !v_pages || !q != !q_out)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_rows < 1 || (int64_t)desc->batch * n_rows > (1 << 20))
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_rows must be positive, batch * n_rows at most 2^20", who);
    const int D = desc->head_dim, size = desc->dtype == DREAM_F32 ? 4 : 2, n = 16 / size;
    if (inv_freq && (rot_dim < 2 || rot_dim % 2 || rot_dim > D))
        return fail(DREAM_ERR_INVALID_ARG, "%s: rot_dim %d is not an even number up to head_dim", who, rot_dim);
    if (inv_freq && !pos && parent && n_rows > DREAM_MAX_TREE)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: %d rows of a tree exceed %d", who, n_rows, DREAM_MAX_TREE);
    for (const void *p : {q, k, v, (const void *)q_out, (const void *)k_pages, (const void *)v_pages})
        if (reinterpret_cast<uintptr_t>(p) & 15)
            return fail(DREAM_ERR_INVALID_ARG, "%s: a tensor is not 16-byte aligned", who);
    // a launch's workgroups come in any order: what one writes none may read, but its own rows in place
    const int64_t rows = (int64_t)desc->batch * n_rows, head = rows * D * size, pool = (int64_t)pages->n_pages * desc->n_kv_heads * pages->page_size * D * size;
    const struct { const void *p; int64_t bytes; const char *name; bool out; } mem[] = {
        {q_out, desc->n_q_heads * head, "q_out", true}, {k_pages, pool, "k_pages", true}, {v_pages, pool, "v_pages", true},
        {q, desc->n_q_heads * head, "q", false}, {k, desc->n_kv_heads * head, "k", false}, {v, desc->n_kv_heads * head, "v", false}};
    for (int i = 0; i < 3; i++)
        for (int j = i + 1; j < 6; j++) {
            const uintptr_t x = reinterpret_cast<uintptr_t>(mem[i].p), y = reinterpret_cast<uintptr_t>(mem[j].p);
            if (x && y && !(i == 0 && j == 3 && x == y) && x < y + mem[j].bytes && y < x + mem[i].bytes)
                return fail(DREAM_ERR_INVALID_ARG, "%s: %s overlaps %s", who, mem[i].name, mem[j].name);
        }
    AppendArgs a = {};
    const int rot = inv_freq ? rot_dim : 0, half = rot / 2;
    const bool paired = interleaved != 0 && rot, wide = (paired ? rot : half) % n == 0;
    const int step = wide ? n : paired ? 2 : 1;
    a.pieces = paired ? D / step : half / step + (D - rot) / step;
    a.end_q = q ? desc->n_q_heads * a.pieces : 0;
    a.end_k = a.end_q + desc->n_kv_heads * a.pieces;
    a.end_v = a.end_k + desc->n_kv_heads * (D / n);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_pages = k_pages; a.v_pages = v_pages;
    a.table = page_table; a.row_base = row_base; a.row_index = row_index; a.n_live = n_live; a.pos = pos; a.pos_base = pos_base; a.parent = parent; a.inv_freq = inv_freq;
    a.n_rows = n_rows; a.hq = desc->n_q_heads; a.hkv = desc->n_kv_heads; a.head_dim = D; a.rot = rot;
    a.lg_page = log2_of(pages->page_size); a.n_pages = pages->n_pages; a.max_pages = pages->max_pages;
    a.amplitude = amplitude != 0.0f ? amplitude : 1.0f;
    a.rows_magic = rows * n_rows < 1ll << 32 ? magic_of(n_rows) : 0;
    a.pieces_magic = (int64_t)a.end_v * a.pieces < 1ll << 32 ? magic_of(a.pieces) : 0;
    a.vpieces_magic = magic_of(D / n);
    return desc->dtype == DREAM_F32 ? launch_append<float>(a, paired, wide, rows, as_stream(stream)) : launch_append<uint16_t>(a, paired, wide, rows, as_stream(stream));
}

int dream_paged_commit(const dream_attn_desc *desc, const dream_page_desc *pages, const int32_t *page_table, void *const *pools_host, int32_t n_pools,
                       const int32_t *prefix_len, int32_t n_tree, const int32_t *accept_path, int32_t path_stride, const int32_t *accept_len, int32_t *prefix_len_out,
                       void *stream)
{
    const char *who = "dream_paged_commit";
    if (int rc = check_pages(who, desc, pages))
        return rc;
    if (!page_table || !pools_host || !prefix_len || !accept_path || !accept_len)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_pools < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_pools %d < 1", who, n_pools);
    if (n_tree < 1 || n_tree > DREAM_MAX_TREE_ACCEPT || n_tree > paged_rows(pages))
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_tree %d outside [1, min(%d, max_pages * page_size)]", who, n_tree, DREAM_MAX_TREE_ACCEPT);
    if (path_stride < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: path_stride %d < 1", who, path_stride);
    if (prefix_len_out == prefix_len || prefix_len_out == accept_len)
        return fail(DREAM_ERR_INVALID_ARG, "%s: prefix_len_out must not alias prefix_len or accept_len", who);
    const int cpr = desc->head_dim * (desc->dtype == DREAM_F32 ? 4 : 2) / 16;
    const int64_t max_rows = path_stride < n_tree ? path_stride : n_tree;
    if (max_rows * cpr > 256 * CHUNKS_PER_THREAD)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: up to %lld rows of %d bytes exceed the 64 KB a workgroup moves", who, (long long)max_rows, cpr * 16);
    for (int32_t i = 0; i < n_pools; i++) {
        if (!pools_host[i] || (reinterpret_cast<uintptr_t>(pools_host[i]) & 15))
            return fail(DREAM_ERR_INVALID_ARG, "%s: pool %d is NULL or not 16-byte aligned", who, i);
    }
    PagedCommitArgs a = {};
    a.table = page_table; a.accept_len = accept_len; a.path = accept_path; a.prefix_len = prefix_len; a.prefix_len_out = prefix_len_out;
    a.hkv = desc->n_kv_heads; a.path_stride = path_stride; a.n_tree = n_tree; a.cpr = cpr; a.lg_page = log2_of(pages->page_size); a.n_pages = pages->n_pages;
    a.max_pages = pages->max_pages;
    // heads per workgroup: as many as the registers of a workgroup hold, while about a thousand workgroups remain
    const int64_t fit = (256 * CHUNKS_PER_THREAD) / (max_rows * cpr);
    const int64_t spare = ((int64_t)a.hkv * desc->batch * (n_pools < POOLS_PER_LAUNCH ? n_pools : POOLS_PER_LAUNCH)) / 1024;
    int64_t hpw = fit < spare ? fit : spare;
    hpw = hpw > a.hkv ? a.hkv : hpw < 1 ? 1 : hpw;
    a.heads_per_wg = (int)hpw;
    for (int32_t first = 0; first < n_pools; first += POOLS_PER_LAUNCH) {
        const int m = n_pools - first < POOLS_PER_LAUNCH ? n_pools - first : POOLS_PER_LAUNCH;
        for (int i = 0; i < POOLS_PER_LAUNCH; i++)
            a.pool[i] = i < m ? pools_host[first + i] : nullptr;
        a.first_pool = first;
        hipLaunchKernelGGL(paged_commit_kernel, dim3(ceil_div(a.hkv, hpw), desc->batch, m), dim3(256), 0, as_stream(stream), a);
        if (int rc = check_launch("paged_commit_kernel"))
            return rc;
    }
    return DREAM_OK;
}

int dream_page_bounds(const dream_attn_desc *desc, const dream_page_desc *pages, const int32_t *page_table, const void *k_pages, const int32_t *from_len, const int32_t *to_len,
                      int64_t max_new, void *bounds, void *stream)
{
    const char *who = "dream_page_bounds";
    if (int rc = check_pages(who, desc, pages))
        return rc;
    if (!page_table || !k_pages || !to_len || !bounds)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (max_new < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: max_new must be positive", who);
    if ((reinterpret_cast<uintptr_t>(k_pages) | reinterpret_cast<uintptr_t>(bounds)) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: a tensor is not 16-byte aligned", who);
    BoundsArgs a = {};
    a.k = k_pages; a.bounds = bounds; a.table = page_table; a.from_len = from_len; a.to_len = to_len;
    a.hkv = desc->n_kv_heads; a.lg_page = log2_of(pages->page_size); a.n_pages = pages->n_pages; a.max_pages = pages->max_pages;
    const int64_t slots = (max_new < paged_rows(pages) ? max_new - 1 : paged_rows(pages)) / pages->page_size + 2;      // pages that so many rows may touch
    a.slots = (int)(slots < pages->max_pages ? slots : pages->max_pages);
    return desc->dtype == DREAM_F32 ? launch_bounds<float>(a, desc->head_dim, desc->batch, as_stream(stream)) : launch_bounds<uint16_t>(a, desc->head_dim, desc->batch, as_stream(stream));
}

}  // extern "C"
