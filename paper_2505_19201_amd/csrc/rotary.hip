// dream_rotary_rows: rotary positions for the rows a step adds.  Section 3.1's maps (dream_project_rows) leave queries and keys without positions; models that
// turn them do it between the maps and the attention calls, with a drafted node standing at its prefix plus its depth in the tree.
//
// A pair (x, y) of a row at position p becomes amplitude * (x cos a - y sin a, x sin a + y cos a), a = p * inv_freq[i].  The angle is formed and reduced to a part of a turn in 64
// bits: in 32 its rounding alone would be p * 2^-25, a hundredth of a radian at position 400 000.  The turn itself is float32, rounded once to the row's type.
//
// One workgroup per row, or where there are few rows several: the angles of a row are the same for all its heads, so they are formed once, by rot_dim / 2 threads, and lie in LDS; the
// row's first pieces are requested ahead of that, and every wave holds the tree in registers.  A thread then takes 16 bytes of a head (in the half layout with the 16 bytes rot_dim / 2 further
// on), whatever job the head belongs to: one launch serves the queries and the keys.  Sizes that 16-byte pieces do not divide, and unaligned tensors, go pair by pair.
// Roofline: HBM for prompts (rows read and written once): 210 MB in 40 to 41 us, 5.2 TB/s, what a large copy reaches.  For a tree the launch and the chain parents, angles, rows: 60 rows of
// 64 heads of 128 in 3.7 us (with one workgroup a row 4.3; a kernel that does nothing 1.6), 0.4 us of them the walk up the tree.
#include <type_traits>
#include "common.h"
#include "quick_div.h"

using namespace dream;

namespace {

constexpr int MAX_DIM = 512;       // head_dim
constexpr int BATCH = 4;           // pieces a thread has in flight

struct RotaryJob {
    const void *x;
    void *out;
    const int32_t *row_base, *row_index;
    int32_t n_heads;
    int32_t end;                   // of the job's pieces among a row's
};
struct RotaryArgs {
    RotaryJob job[DREAM_MAX_ROTARY_JOBS];
    const int32_t *pos, *pos_base, *parent;
    const float *inv_freq;
    int64_t s_max;
    int32_t n_rows, head_dim, rot, pieces;   // pieces of a head
    uint32_t rows_magic, pieces_magic;       // for quick_div; 0: divide
    float amplitude;
};

// 16 bytes, or what a pair needs: N values of type T
template <class T, int N>
struct Piece {
    T v[N];
};

template <class T>
__device__ __forceinline__ float widen(T v)
{
    if constexpr (std::is_same_v<T, float>)
        return v;
    else
        return bf16_bits_to_float(v);
}
template <class T>
__device__ __forceinline__ T narrow(float v)
{
    if constexpr (std::is_same_v<T, float>)
        return v;
    else
        return __builtin_bit_cast(uint16_t, (__bf16)v);
}

template <class T, int N>
__device__ __forceinline__ Piece<T, N> load_piece(const T *p)
{
    if constexpr (sizeof(T) * N == 16) {
        return __builtin_bit_cast(Piece<T, N>, *reinterpret_cast<const u32x4 *>(p));
    } else {
        Piece<T, N> r;
#pragma unroll
        for (int i = 0; i < N; i++)
            r.v[i] = p[i];
        return r;
    }
}
template <class T, int N>
__device__ __forceinline__ void store_piece(T *p, const Piece<T, N> &r)
{
    if constexpr (sizeof(T) * N == 16) {
        *reinterpret_cast<u32x4 *>(p) = __builtin_bit_cast(u32x4, r);
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
            p[i] = r.v[i];
    }
}

// PAIRED: the pairs are neighbours (2i, 2i + 1); else (i, i + rot / 2).  N values a piece.
template <class T, bool PAIRED, int N>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a)
{
    __shared__ float2 s_turn[MAX_DIM / 2];
    const int tid = threadIdx.x;
    const int b = a.rows_magic ? quick_div(blockIdx.x, a.rows_magic) : blockIdx.x / a.n_rows, r = blockIdx.x - b * a.n_rows;
    const int D = a.head_dim, rot = a.rot, half = rot / 2, pieces = a.pieces;
    const int turned = (PAIRED ? rot : half) / N;     // pieces of a head that turn; the others are copied
    const int total = a.job[DREAM_MAX_ROTARY_JOBS - 1].end;
    const int stride = gridDim.y * 256;
    Piece<T, N> x[BATCH], y[BATCH];
    T *dst[BATCH];
    int at[BATCH];                                    // piece of its head
    auto request = [&](int first) {
#pragma unroll
        for (int u = 0; u < BATCH; u++) {
            const int idx = first + u * stride + tid;
            dst[u] = nullptr;
            at[u] = 0;
            if (idx < total) {
                int j = 0, start = 0;
#pragma unroll
                for (int i = 0; i + 1 < DREAM_MAX_ROTARY_JOBS; i++)
                    if (idx >= a.job[i].end) {
                        j = i + 1;
                        start = a.job[i].end;
                    }
                const T *src = nullptr;
                T *out = nullptr;
                const int32_t *base = nullptr, *index = nullptr;
                int heads = 1;
#pragma unroll
                for (int i = 0; i < DREAM_MAX_ROTARY_JOBS; i++)      // (no indexed read of the arguments)
                    if (j == i) {
                        src = static_cast<const T *>(a.job[i].x);
                        out = static_cast<T *>(a.job[i].out);
                        base = a.job[i].row_base;
                        index = a.job[i].row_index;
                        heads = a.job[i].n_heads;
                    }
                const int h = a.pieces_magic ? quick_div(idx - start, a.pieces_magic) : (idx - start) / pieces, it = idx - start - h * pieces;
                const int c = PAIRED || it < turned ? it * N : it * N + half;     // first channel
                const int64_t dense = ((int64_t)blockIdx.x * heads + h) * D;
                int64_t to = dense;
                bool kept = true;
                if (base) {
                    const int64_t row = (int64_t)base[b] + (index ? index[(int64_t)b * a.n_rows + r] : r);
                    kept = row >= 0 && row < a.s_max;
                    to = (((int64_t)b * heads + h) * a.s_max + row) * D;
                }
                x[u] = load_piece<T, N>(src + dense + c);
                if (!PAIRED && it < turned)
                    y[u] = load_piece<T, N>(src + dense + c + half);
                at[u] = it;
                dst[u] = kept ? out + to + c : nullptr;
            }
        }
    };
    // all that the position needs is requested before anything is waited for
    const bool walk = a.parent && !a.pos;
    int32_t par[DREAM_MAX_TREE / 64];                 // every wave holds the tree, lane l nodes l, 64 + l, ...
#pragma unroll
    for (int i = 0; i < DREAM_MAX_TREE / 64; i++) {
        const int node = i * 64 + (tid & 63);
        par[i] = walk && node < a.n_rows ? a.parent[(int64_t)b * a.n_rows + node] : -1;
    }
    const int32_t start = a.pos ? a.pos[blockIdx.x] : a.pos_base[b];
    const float freq = a.inv_freq[tid < half ? tid : 0];
    request(blockIdx.y * 256);
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
    for (int first = blockIdx.y * 256; first < total; first += stride * BATCH) {
        if (first >= stride)
            request(first);
#pragma unroll
        for (int u = 0; u < BATCH; u++) {
            if (!dst[u])
                continue;
            if (at[u] < turned) {
                if constexpr (PAIRED) {
#pragma unroll
                    for (int i = 0; i < N; i += 2) {
                        const float2 t = s_turn[at[u] * (N / 2) + i / 2];
                        const float p = widen(x[u].v[i]), q = widen(x[u].v[i + 1]);
                        x[u].v[i] = narrow<T>(p * t.x - q * t.y);
                        x[u].v[i + 1] = narrow<T>(p * t.y + q * t.x);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        const float2 t = s_turn[at[u] * N + i];
                        const float p = widen(x[u].v[i]), q = widen(y[u].v[i]);
                        x[u].v[i] = narrow<T>(p * t.x - q * t.y);
                        y[u].v[i] = narrow<T>(p * t.y + q * t.x);
                    }
                    store_piece(dst[u] + half, y[u]);
                }
            }
            store_piece(dst[u], x[u]);
        }
    }
}

template <class T>
int launch(const RotaryArgs &a, bool paired, bool wide, int64_t rows, hipStream_t st)
{
    constexpr int N = 16 / sizeof(T);
    auto *kernel = paired ? (wide ? &rotary_kernel<T, true, N> : &rotary_kernel<T, true, 2>) : wide ? &rotary_kernel<T, false, N> : &rotary_kernel<T, false, 1>;
    const int64_t parts = 1024 / rows, most = (a.job[DREAM_MAX_ROTARY_JOBS - 1].end + 255) / 256;
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows, (unsigned)(parts < 1 ? 1 : parts < most ? parts : most)), dim3(256), 0, st, a);
    return check_launch("rotary_kernel");
}

}  // namespace

extern "C" {

int dream_rotary_rows(const dream_attn_desc *desc, const dream_rotary_job *jobs, int32_t n_jobs, int32_t n_rows, const int32_t *pos,
                      const int32_t *pos_base, const int32_t *parent, const float *inv_freq, int32_t rot_dim, int32_t interleaved,
                      float amplitude, void *stream)
{
    const char *who = "dream_rotary_rows";
    if (!desc || !jobs || !inv_freq)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_jobs < 1 || n_jobs > DREAM_MAX_ROTARY_JOBS)
        return fail(DREAM_ERR_INVALID_ARG, "%s: %d jobs outside [1, %d]", who, n_jobs, DREAM_MAX_ROTARY_JOBS);
    if (desc->dtype != DREAM_F32 && desc->dtype != DREAM_BF16)
        return fail(DREAM_ERR_INVALID_ARG, "%s: unknown dtype %d", who, desc->dtype);
    if (desc->batch < 1 || n_rows < 1 || (int64_t)desc->batch * n_rows > (1 << 20))
        return fail(DREAM_ERR_INVALID_ARG, "%s: batch and n_rows must be positive, batch * n_rows at most 2^20", who);
    if (desc->head_dim < 2 || desc->head_dim % 2 || desc->head_dim > MAX_DIM)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: head_dim %d is not an even number up to %d", who, desc->head_dim, MAX_DIM);
    if (rot_dim < 2 || rot_dim % 2 || rot_dim > desc->head_dim)
        return fail(DREAM_ERR_INVALID_ARG, "%s: rot_dim %d is not an even number up to head_dim", who, rot_dim);
    if (!pos && !pos_base)
        return fail(DREAM_ERR_INVALID_ARG, "%s: neither positions nor their base given", who);
    if (!pos && parent && n_rows > DREAM_MAX_TREE)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: %d rows of a tree exceed %d", who, n_rows, DREAM_MAX_TREE);
    RotaryArgs a = {};
    const int size = desc->dtype == DREAM_F32 ? 4 : 2, n = 16 / size, half = rot_dim / 2;
    bool wide = desc->head_dim % n == 0 && (interleaved ? rot_dim : half) % n == 0;
    for (int j = 0; j < n_jobs; j++) {
        const dream_rotary_job &jb = jobs[j];
        if (!jb.x || !jb.out)
            return fail(DREAM_ERR_INVALID_ARG, "%s: NULL tensor in job %d", who, j);
        if (jb.n_heads < 1 || jb.n_heads > 65535)
            return fail(DREAM_ERR_INVALID_ARG, "%s: n_heads of job %d outside [1, 65535]", who, j);
        if (jb.row_base && desc->s_max < 1)
            return fail(DREAM_ERR_INVALID_ARG, "%s: cache output needs s_max", who);
        if (!jb.row_base && jb.row_index)
            return fail(DREAM_ERR_INVALID_ARG, "%s: row_index without row_base in job %d", who, j);
        if ((reinterpret_cast<uintptr_t>(jb.x) | reinterpret_cast<uintptr_t>(jb.out)) & (size - 1))
            return fail(DREAM_ERR_INVALID_ARG, "%s: a tensor of job %d is not aligned to its values", who, j);
        if (jb.row_base && jb.x == jb.out)
            return fail(DREAM_ERR_INVALID_ARG, "%s: job %d writes a cache over its own rows", who, j);
        wide = wide && !((reinterpret_cast<uintptr_t>(jb.x) | reinterpret_cast<uintptr_t>(jb.out)) & 15);
    }
    // a launch's workgroups come in any order: what one writes none may read, but its own rows in place
    const int64_t values = (int64_t)desc->batch * n_rows * desc->head_dim * size;
    auto overlap = [&](const void *p, const dream_rotary_job &of_p, const void *q, const dream_rotary_job &of_q) {
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(p), b0 = reinterpret_cast<uintptr_t>(q);
        return a0 < b0 + of_q.n_heads * values && b0 < a0 + of_p.n_heads * values;
    };
    for (int j = 0; j < n_jobs; j++)
        for (int i = 0; i < n_jobs && !jobs[j].row_base; i++)
            if ((!(i == j && jobs[j].x == jobs[j].out) && overlap(jobs[j].out, jobs[j], jobs[i].x, jobs[i])) ||
                (i < j && !jobs[i].row_base && overlap(jobs[j].out, jobs[j], jobs[i].out, jobs[i])))
                return fail(DREAM_ERR_INVALID_ARG, "%s: out of job %d overlaps a tensor of job %d", who, j, i);
    const int step = wide ? n : interleaved ? 2 : 1;
    a.pieces = interleaved ? desc->head_dim / step : half / step + (desc->head_dim - rot_dim) / step;
    int64_t end = 0;
    for (int j = 0; j < DREAM_MAX_ROTARY_JOBS; j++) {
        if (j < n_jobs) {
            a.job[j].x = jobs[j].x; a.job[j].out = jobs[j].out;
            a.job[j].row_base = jobs[j].row_base; a.job[j].row_index = jobs[j].row_index;
            a.job[j].n_heads = jobs[j].n_heads;
            end += (int64_t)jobs[j].n_heads * a.pieces;
        }
        a.job[j].end = (int32_t)end;
    }
    a.pos = pos; a.pos_base = pos_base; a.parent = parent; a.inv_freq = inv_freq;
    a.s_max = desc->s_max; a.n_rows = n_rows; a.head_dim = desc->head_dim; a.rot = rot_dim;
    a.amplitude = amplitude != 0.0f ? amplitude : 1.0f;
    const int64_t rows = (int64_t)desc->batch * n_rows;
    a.rows_magic = rows * n_rows < 1ll << 32 ? magic_of(n_rows) : 0;
    a.pieces_magic = end * a.pieces < 1ll << 32 ? magic_of(a.pieces) : 0;
    return desc->dtype == DREAM_F32 ? launch<float>(a, interleaved != 0, wide, rows, as_stream(stream))
                                    : launch<uint16_t>(a, interleaved != 0, wide, rows, as_stream(stream));
}

}  // extern "C"
