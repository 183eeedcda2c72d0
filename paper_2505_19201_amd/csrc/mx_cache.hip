// Key/value caches held in 4 bits: dream_mx_append, dream_mx_read, dream_mx_commit.
//
// A row of a head is D codes of 4 bits (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) and D / 32 scales, powers of two held as their exponent plus 127.
// These are the types that gfx950's conversions take, so a value costs half an instruction to read, and a code times its scale is a bfloat16 without rounding.
// The scale s of 32 values is the smallest power of two with max|x| <= 7 s.  Beyond 6 s the largest code is off by at most s, which is what rounding to it or to 4 may be off by
// as well; a smaller s would clip, the next one halves the resolution of everything.  Zeros and values far below 2^-125 keep the smallest scale, 2^-125, so that
// every value a cache stands for is a normal number.  A group with a value that is not finite has scale 255 and stands for NaN.
//
// All three calls only move bytes.  Append: a lane takes 16 bytes of a row; the lanes that share a scale are neighbours (4 for bf16, 8 for float32) and find their
// maximum by moves between registers.  A workgroup takes consecutive rows of one head, whose codes and scales are consecutive in the cache.
// Roofline: HBM, 531 MB in 101 us (5.2 TB/s, what a large copy reaches); for the rows of a tree the launch: 33 rows of 4 heads of 256 in 2.2 us, a kernel that does nothing 1.6.
#include <type_traits>
#include "common.h"

using namespace dream;

namespace {

constexpr int GROUP = DREAM_MX_GROUP;
constexpr int MAX_CACHES = 64;      // a launch

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// exponent byte of the scale of a group whose largest magnitude has these bits
__device__ __forceinline__ uint32_t scale_of(uint32_t top)
{
    const int e = (int)((top + 0x1fffffu) >> 23) - 2;      // mantissas above 1.75 take the next exponent
    return top >= 0x7f800000u ? 255u : (uint32_t)min(max(e, 2), 252);
}

template <int CTRL>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}

struct AppendArgs {
    const void *rows[2];
    uint8_t *codes[2], *scales[2];
    const int32_t *row_base, *row_index;
    int64_t s_max;
    int32_t n_rows, n_heads;
};

// N values of 16 bytes a lane; grid: (pieces of the rows of a head, head, sequence * 2 + K or V)
template <class T, int D>
__global__ __launch_bounds__(256) void mx_append_kernel(AppendArgs a)
{
    constexpr int N = 16 / sizeof(T), PER_ROW = D / N;
    const int which = blockIdx.z & 1, b = blockIdx.z >> 1, h = blockIdx.y;
    const int idx = blockIdx.x * 256 + threadIdx.x, total = a.n_rows * PER_ROW;
    const int r = min(idx / PER_ROW, a.n_rows - 1), piece = idx % PER_ROW;
    const T *rows = static_cast<const T *>(which ? a.rows[1] : a.rows[0]);
    const u32x4 raw = *reinterpret_cast<const u32x4 *>(rows + (((int64_t)b * a.n_rows + r) * a.n_heads + h) * D + piece * N);
    const int64_t to = (int64_t)a.row_base[b] + (a.row_index ? a.row_index[(int64_t)b * a.n_rows + r] : r);
    uint32_t top = 0u;
    if constexpr (N == 8) {
#pragma unroll
        for (int i = 0; i < 4; i++)
            top = max(top, max(raw[i] & 0x7fff0000u, (raw[i] << 16) & 0x7fffffffu));
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            top = max(top, raw[i] & 0x7fffffffu);
    }
    top = lanes_max<0xb1>(top);           // lanes 1 apart, 2 apart (quad_perm), and for float32 the other quad of 8 (row_half_mirror)
    top = lanes_max<0x4e>(top);
    if constexpr (N == 4)
        top = lanes_max<0x141>(top);
    const uint32_t e = scale_of(top);
    const float scale = __uint_as_float(e << 23);
    uint32_t codes = 0u;
    if constexpr (N == 8) {
        const uint32_t w[4] = {raw[0], raw[1], raw[2], raw[3]};      // (a bit_cast of a vector's element takes its first)
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w[0]), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w[1]), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w[2]), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, w[3]), scale, 3);
    } else {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(raw[0]), __uint_as_float(raw[1]), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __uint_as_float(raw[2]), __uint_as_float(raw[3]), scale, 1);
    }
    if (idx >= total || to < 0 || to >= a.s_max)
        return;
    const int64_t row = ((int64_t)b * a.n_heads + h) * a.s_max + to;
    uint8_t *out = (which ? a.codes[1] : a.codes[0]) + row * (D / 2) + piece * (N / 2);
    if constexpr (N == 8)
        *reinterpret_cast<uint32_t *>(out) = codes;
    else
        *reinterpret_cast<uint16_t *>(out) = (uint16_t)codes;
    if (piece % (GROUP / N) == 0)
        (which ? a.scales[1] : a.scales[0])[row * (D / GROUP) + piece / (GROUP / N)] = (uint8_t)e;
}

struct ReadArgs {
    const uint8_t *codes[MAX_CACHES], *scales[MAX_CACHES];
    const int32_t *row_base;
    void *out;
    int64_t s_max;
    int32_t n_rows, n_heads, batch;
};

// grid: (pieces of the rows of a head, head, cache * batch + sequence)
template <class T, int D>
__global__ __launch_bounds__(256) void mx_read_kernel(ReadArgs a)
{
    constexpr int N = 16 / sizeof(T), PER_ROW = D / N;
    const int b = blockIdx.z % a.batch, ci = blockIdx.z / a.batch, h = blockIdx.y;
    const int idx = blockIdx.x * 256 + threadIdx.x;
    if (idx >= a.n_rows * PER_ROW)
        return;
    const int r = idx / PER_ROW, piece = idx % PER_ROW;
    const int64_t from = (a.row_base ? a.row_base[b] : 0) + (int64_t)r;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (from >= 0 && from < a.s_max) {
        const int64_t row = ((int64_t)b * a.n_heads + h) * a.s_max + from;
        const uint8_t *codes = a.codes[ci] + row * (D / 2) + piece * (N / 2);
        const float scale = __uint_as_float((uint32_t)a.scales[ci][row * (D / GROUP) + piece / (GROUP / N)] << 23);
        if constexpr (N == 8) {
            const uint32_t c = *reinterpret_cast<const uint32_t *>(codes);
            v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
            v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
            v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
            v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
        } else {
            const uint32_t c = *reinterpret_cast<const uint16_t *>(codes);
            const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
            v = u32x4{__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(hi[0]), __float_as_uint(hi[1])};
        }
    }
    const int64_t row = (((int64_t)ci * a.batch + b) * a.n_heads + h) * a.n_rows + r;
    reinterpret_cast<u32x4 *>(a.out)[row * PER_ROW + piece] = v;
}

// dream_mx_commit: the codes and scales of the accepted path's rows become the next rows of the prefix, in place.  A head of a sequence in a cache is moved by one wave, or, where the longest
// path has more pieces than four for each of its lanes, by a workgroup: what is to move, a few hundred bytes to a few KB, is in registers before anything is written.  A row is D / 32 pieces of
// 16 bytes of codes and one piece of D / 32 bytes of scales.  (16 caches of 8 sequences of 32 heads of 64, paths of up to 7 rows: 4.8 us, with a workgroup a head 17.9.)
// Bound by trips to memory, one after the other: the arguments, the lengths, the path, the rows; a path of four rows is 12 pieces of 16 bytes, so four of five lanes have none.  The bytes, about
// 1 MB each way, would take 0.4 us.  It runs once a round behind all layers' attention, 0.2 us a layer, which is why it was left so.
constexpr int WAVE_MOVES = 4, GROUP_MOVES = 8;            // pieces a lane holds

struct CommitArgs {
    uint8_t *codes[MAX_CACHES], *scales[MAX_CACHES];
    const int32_t *prefix_len, *path, *accept_len;
    int32_t *prefix_len_out;
    int64_t s_max;
    int32_t n_heads, n_tree, path_stride, first_cache;
};

// LANES: 64 or 256 to a head
template <int D, int LANES>
__global__ __launch_bounds__(256) void mx_commit_kernel(CommitArgs a)
{
    constexpr int MOVES = LANES == 64 ? WAVE_MOVES : GROUP_MOVES;
    constexpr int CPR = D / GROUP, PPR = CPR + 1;
    using Scales = std::conditional_t<D == 64, uint16_t, std::conditional_t<D == 128, uint32_t, uint64_t>>;
    const int h = blockIdx.x * (256 / LANES) + threadIdx.x / LANES, b = blockIdx.y, ci = blockIdx.z, tid = threadIdx.x % LANES;
    if (h >= a.n_heads)
        return;
    const int32_t *path = a.path + (int64_t)b * a.path_stride;
    const int P = (int)min((int64_t)max(a.prefix_len[b], 0), a.s_max - a.n_tree);
    const int n = min(max(a.accept_len[b], 0), min(a.path_stride, a.n_tree) - 1);
    if (h == 0 && ci == 0 && a.first_cache == 0 && tid == 0 && a.prefix_len_out)
        a.prefix_len_out[b] = P + n + 1;
    const int total = (n + 1) * PPR;
    const int64_t tree = ((int64_t)b * a.n_heads + h) * a.s_max + P;
    u32x4 *codes = reinterpret_cast<u32x4 *>(a.codes[ci]) + tree * CPR;
    Scales *scales = reinterpret_cast<Scales *>(a.scales[ci]) + tree;
    u32x4 v[MOVES];
    Scales s[MOVES];
#pragma unroll
    for (int i = 0; i < MOVES; i++) {
        const int idx = tid + i * LANES;
        if (idx < total) {
            const int j = idx / PPR, c = idx % PPR;
            const int node = min(max(path[j], 0), a.n_tree - 1);
            if (c < CPR)
                v[i] = codes[(int64_t)node * CPR + c];
            else
                s[i] = scales[node];
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (LANES > 64)
        __syncthreads();   // every source of this head is in a register
#pragma unroll
    for (int i = 0; i < MOVES; i++) {
        const int idx = tid + i * LANES;
        if (idx < total) {
            const int j = idx / PPR, c = idx % PPR;
            if (c < CPR)
                codes[(int64_t)j * CPR + c] = v[i];
            else
                scales[j] = s[i];
        }
    }
}

int check_cache(const char *who, const dream_attn_desc *d)
{
    if (!d)
        return fail(DREAM_ERR_INVALID_ARG, "%s: desc is NULL", who);
    if (d->batch < 1 || d->n_kv_heads < 1 || d->s_max < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: batch, n_kv_heads and s_max must be positive", who);
    if (d->dtype != DREAM_F32 && d->dtype != DREAM_BF16)
        return fail(DREAM_ERR_INVALID_ARG, "%s: unknown dtype %d", who, d->dtype);
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: head_dim %d not in {64,128,256}", who, d->head_dim);
    if (d->batch > DREAM_MAX_MX_BATCH || d->n_kv_heads > 65535)      // (append's grid has K and V of a sequence in one dimension)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: batch is limited to %d, n_kv_heads to 65535", who, DREAM_MAX_MX_BATCH);
    return DREAM_OK;
}

bool unaligned(const void *codes, const void *scales)
{
    return (reinterpret_cast<uintptr_t>(codes) & 15) || (reinterpret_cast<uintptr_t>(scales) & 7);
}

template <class T>
auto append_kernel(int d) { return d == 64 ? &mx_append_kernel<T, 64> : d == 128 ? &mx_append_kernel<T, 128> : &mx_append_kernel<T, 256>; }
template <int LANES>
auto commit_kernel(int d) { return d == 64 ? &mx_commit_kernel<64, LANES> : d == 128 ? &mx_commit_kernel<128, LANES> : &mx_commit_kernel<256, LANES>; }
template <class T>
auto read_kernel(int d) { return d == 64 ? &mx_read_kernel<T, 64> : d == 128 ? &mx_read_kernel<T, 128> : &mx_read_kernel<T, 256>; }

}  // namespace

extern "C" {

int dream_mx_append(const dream_attn_desc *desc, const void *k_rows, const void *v_rows, int32_t n_rows, const int32_t *row_base,
                    const int32_t *row_index, void *k_codes, void *k_scales, void *v_codes, void *v_scales, void *stream)
{
    const char *who = "dream_mx_append";
    if (int rc = check_cache(who, desc))
        return rc;
    if (!k_rows || !v_rows || !row_base || !k_codes || !k_scales || !v_codes || !v_scales)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_rows < 1 || (int64_t)desc->batch * n_rows > (1 << 20))
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_rows must be positive, batch * n_rows at most 2^20", who);
    if ((reinterpret_cast<uintptr_t>(k_rows) | reinterpret_cast<uintptr_t>(v_rows)) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned", who);
    if (unaligned(k_codes, k_scales) || unaligned(v_codes, v_scales))
        return fail(DREAM_ERR_INVALID_ARG, "%s: codes must be 16-byte aligned, scales 8-byte aligned", who);
    AppendArgs a = {};
    a.rows[0] = k_rows; a.rows[1] = v_rows;
    a.codes[0] = static_cast<uint8_t *>(k_codes); a.codes[1] = static_cast<uint8_t *>(v_codes);
    a.scales[0] = static_cast<uint8_t *>(k_scales); a.scales[1] = static_cast<uint8_t *>(v_scales);
    a.row_base = row_base; a.row_index = row_index;
    a.s_max = desc->s_max; a.n_rows = n_rows; a.n_heads = desc->n_kv_heads;
    const int per_row = desc->head_dim * (desc->dtype == DREAM_F32 ? 4 : 2) / 16;
    const dim3 grid(ceil_div((int64_t)n_rows * per_row, 256), desc->n_kv_heads, desc->batch * 2);
    hipLaunchKernelGGL(desc->dtype == DREAM_F32 ? append_kernel<float>(desc->head_dim) : append_kernel<uint16_t>(desc->head_dim), grid, dim3(256), 0,
                       as_stream(stream), a);
    return check_launch("mx_append_kernel");
}

int dream_mx_read(const dream_attn_desc *desc, void *const *codes_host, void *const *scales_host, int32_t n_caches,
                  const int32_t *row_base, int32_t n_rows, void *out, void *stream)
{
    const char *who = "dream_mx_read";
    if (int rc = check_cache(who, desc))
        return rc;
    if (!codes_host || !scales_host || !out)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_caches < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_caches %d < 1", who, n_caches);
    if (n_rows < 1 || n_rows > desc->s_max || n_rows > (1 << 24))
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_rows %d outside [1, min(s_max, 2^24)]", who, n_rows);
    if (reinterpret_cast<uintptr_t>(out) & 15)
        return fail(DREAM_ERR_INVALID_ARG, "%s: out must be 16-byte aligned", who);
    for (int32_t i = 0; i < n_caches; i++) {
        if (!codes_host[i] || !scales_host[i])
            return fail(DREAM_ERR_INVALID_ARG, "%s: cache %d is NULL", who, i);
        if (unaligned(codes_host[i], scales_host[i]))
            return fail(DREAM_ERR_INVALID_ARG, "%s: cache %d: codes must be 16-byte aligned, scales 8-byte aligned", who, i);
    }
    const int size = desc->dtype == DREAM_F32 ? 4 : 2, per_row = desc->head_dim * size / 16;
    int step = 65535 / desc->batch;      // (a grid's extent)
    step = step < MAX_CACHES ? step : MAX_CACHES;
    for (int32_t first = 0; first < n_caches; first += step) {
        const int m = n_caches - first < step ? n_caches - first : step;
        ReadArgs a = {};
        for (int i = 0; i < m; i++) {
            a.codes[i] = static_cast<const uint8_t *>(codes_host[first + i]);
            a.scales[i] = static_cast<const uint8_t *>(scales_host[first + i]);
        }
        a.row_base = row_base; a.s_max = desc->s_max; a.n_rows = n_rows; a.n_heads = desc->n_kv_heads; a.batch = desc->batch;
        a.out = static_cast<char *>(out) + (int64_t)first * desc->batch * desc->n_kv_heads * n_rows * desc->head_dim * size;
        const dim3 grid(ceil_div((int64_t)n_rows * per_row, 256), desc->n_kv_heads, desc->batch * m);
        hipLaunchKernelGGL(desc->dtype == DREAM_F32 ? read_kernel<float>(desc->head_dim) : read_kernel<uint16_t>(desc->head_dim), grid, dim3(256), 0,
                           as_stream(stream), a);
        if (int rc = check_launch("mx_read_kernel"))
            return rc;
    }
    return DREAM_OK;
}

int dream_mx_commit(const dream_attn_desc *desc, void *const *codes_host, void *const *scales_host, int32_t n_caches,
                    const int32_t *prefix_len, int32_t n_tree, const int32_t *accept_path, int32_t path_stride,
                    const int32_t *accept_len, int32_t *prefix_len_out, void *stream)
{
    const char *who = "dream_mx_commit";
    if (int rc = check_cache(who, desc))
        return rc;
    if (!codes_host || !scales_host || !prefix_len || !accept_path || !accept_len)
        return fail(DREAM_ERR_INVALID_ARG, "%s: NULL argument", who);
    if (n_caches < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_caches %d < 1", who, n_caches);
    if (n_tree < 1 || n_tree > DREAM_MAX_TREE_ACCEPT || n_tree > desc->s_max)
        return fail(DREAM_ERR_INVALID_ARG, "%s: n_tree %d outside [1, min(%d, s_max)]", who, n_tree, DREAM_MAX_TREE_ACCEPT);
    if (path_stride < 1)
        return fail(DREAM_ERR_INVALID_ARG, "%s: path_stride %d < 1", who, path_stride);
    if (prefix_len_out == prefix_len)
        return fail(DREAM_ERR_INVALID_ARG, "%s: prefix_len_out must not alias prefix_len", who);
    const int64_t max_rows = path_stride < n_tree ? path_stride : n_tree;
    const int64_t pieces = max_rows * (desc->head_dim / GROUP + 1);
    if (pieces > 256 * GROUP_MOVES)
        return fail(DREAM_ERR_UNSUPPORTED, "%s: a path of %lld rows is longer than a workgroup moves", who, (long long)max_rows);
    for (int32_t i = 0; i < n_caches; i++) {
        if (!codes_host[i] || !scales_host[i])
            return fail(DREAM_ERR_INVALID_ARG, "%s: cache %d is NULL", who, i);
        if (unaligned(codes_host[i], scales_host[i]))
            return fail(DREAM_ERR_INVALID_ARG, "%s: cache %d: codes must be 16-byte aligned, scales 8-byte aligned", who, i);
    }
    for (int32_t first = 0; first < n_caches; first += MAX_CACHES) {
        const int m = n_caches - first < MAX_CACHES ? n_caches - first : MAX_CACHES;
        CommitArgs a = {};
        for (int i = 0; i < m; i++) {
            a.codes[i] = static_cast<uint8_t *>(codes_host[first + i]);
            a.scales[i] = static_cast<uint8_t *>(scales_host[first + i]);
        }
        a.prefix_len = prefix_len; a.path = accept_path; a.accept_len = accept_len; a.prefix_len_out = prefix_len_out;
        a.s_max = desc->s_max; a.n_heads = desc->n_kv_heads; a.n_tree = n_tree; a.path_stride = path_stride; a.first_cache = first;
        const bool wave = pieces <= 64 * WAVE_MOVES;
        auto *kernel = wave ? commit_kernel<64>(desc->head_dim) : commit_kernel<256>(desc->head_dim);
        hipLaunchKernelGGL(kernel, dim3(wave ? (desc->n_kv_heads + 3) / 4 : desc->n_kv_heads, desc->batch, m), dim3(256), 0, as_stream(stream), a);
        if (int rc = check_launch("mx_commit_kernel"))
            return rc;
    }
    return DREAM_OK;
}

}  // extern "C"
