// dq8: rows of new keys and values into a paged cache, with the norms and the rotation of queries and keys on the way
// (dq8_cache_append of include/dq8_cache.h).  Built with the flags of dq8.hip: no contraction of products and sums.
//
// A row is `dim` elements of one token and head, held by LPR neighbouring lanes, eight elements each (dim <= 8 LPR), so a
// wavefront works on 64 / LPR rows at a time and the row's sum of squares and maximum are reductions over LPR lanes.  The partner
// of an element that is turned half a rotation away lies in another lane: it is loaded from memory once more (the same cache
// lines, a few instructions earlier) instead of passed between lanes.
#include <hip/hip_runtime.h>

#include "dq8_cache_check.hpp"
#include "dq8_device.hpp"
#include "dq8_kernels_small.hpp"

namespace {

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out;
    size_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs;  // elements from token to token and head to head
    const int64_t *slots, *positions;
    const float *rotation, *q_weight, *k_weight;
    uint8_t *codes;
    float *scales;
    uint64_t n_positions, n_slots;
    double eps;
    uint32_t tokens, heads, kv_heads, dim, half, interleaved, page_shift;
    uint32_t kv_groups;  // workgroups that work on keys and values, the rest on queries
};

template <typename T>
struct Eight {
    typedef T type __attribute__((ext_vector_type(8)));
};

// Eight elements from an address that is a multiple of the element's size.
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8])
{
    typedef typename Eight<T>::type V __attribute__((aligned(sizeof(T))));
    const V v = *reinterpret_cast<const V *>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&y)[8])
{
    typedef typename Eight<T>::type V __attribute__((aligned(sizeof(T))));
    V v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)y[e];
    *reinterpret_cast<V *>(p) = v;
}

template <int LPR>
__device__ __forceinline__ float row_sum(float v)
{
#pragma unroll
    for (int m = 1; m < LPR; m *= 2) v += __shfl_xor(v, m);
    return v;
}

template <int LPR>
__device__ __forceinline__ double row_sum(double v)
{
#pragma unroll
    for (int m = 1; m < LPR; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// This lane's eight elements i0 .. i0 + 7 of a row, normed and turned, in F (double for keys, float for queries).  `row` and `turn`
// are valid addresses for every lane; lanes whose elements lie behind the row (i0 >= dim) take part in the sums with zeros.
template <typename F, int LPR, typename T>
__device__ __forceinline__ void normed_and_turned(const AppendArgs &a, const T *row, const float *weight, const float *turn, uint32_t i0,
                                                  F (&y)[8])
{
    const bool in = i0 < a.dim;
    float x[8] = {};
    if (in) load8(row + i0, x);
    F r = 1;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[e];
    if (weight) {
        F sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += y[e] * y[e];
        r = F(1) / sqrt(row_sum<LPR>(sum) / F(a.dim) + F(a.eps));
        if (in) {
            float w[8];
            load8(weight + i0, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = y[e] * r * F(w[e]);
        }
    }
    const uint32_t half = a.half;
    if (!turn || i0 >= 2 * half) return;
    if (!a.interleaved && half % 8 == 0) {  // all eight on one side, and so their partners
        const bool low = i0 < half;
        const uint32_t j0 = low ? i0 + half : i0 - half, p0 = low ? i0 : j0;
        float other[8], c[8], s[8], w[8] = {1, 1, 1, 1, 1, 1, 1, 1};
        load8(row + j0, other);
        load8(turn + p0, c);
        load8(turn + half + p0, s);
        if (weight) load8(weight + j0, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const F o = weight ? F(other[e]) * r * F(w[e]) : F(other[e]);
            y[e] = low ? y[e] * F(c[e]) - o * F(s[e]) : y[e] * F(c[e]) + o * F(s[e]);
        }
    } else if (a.interleaved) {  // pairs inside the lane
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const uint32_t p = (i0 + e) / 2;
            if (p < half) {
                const F c = turn[p], s = turn[half + p], u = y[e], v = y[e + 1];
                y[e] = u * c - v * s;
                y[e + 1] = v * c + u * s;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t i = i0 + e;
            if (i < 2 * half) {
                const bool low = i < half;
                const uint32_t j = low ? i + half : i - half, p = low ? i : j;
                const F o = weight ? F((float)row[j]) * r * F(weight[j]) : F((float)row[j]);
                const F c = turn[p], s = turn[half + p];
                y[e] = low ? y[e] * c - o * s : y[e] * c + o * s;
            }
        }
    }
}

// The angles of token t; false where its position has none.  Without a rotation: no angles, true.
__device__ __forceinline__ bool angles(const AppendArgs &a, uint32_t t, const float **turn)
{
    *turn = nullptr;
    if (!a.rotation) return true;
    const uint64_t p = (uint64_t)a.positions[t];
    const bool ok = p < a.n_positions;
    *turn = a.rotation + (ok ? p : 0) * 2 * a.half;
    return ok;
}

// Workgroups 0 .. kv_groups - 1 walk the rows of keys, then those of values; the others walk the rows of queries.
template <int LPR, typename T>
__global__ __launch_bounds__(kWg) void k_cache_append(const uint32_t *__restrict__ tab, AppendArgs a)
{
    extern __shared__ uint32_t lds[];
    constexpr uint32_t kRows = kWave / LPR;  // of a wavefront
    const uint32_t lane = threadIdx.x & 63, i0 = (lane % LPR) * 8, sub = lane / LPR;
    if (blockIdx.x >= a.kv_groups) {
        const uint32_t rows = a.tokens * a.heads, step = (gridDim.x - a.kv_groups) * kWavesPerWg * kRows;
        for (uint32_t at = ((blockIdx.x - a.kv_groups) * kWavesPerWg + wave_in_wg()) * kRows; at < rows; at += step) {
            const uint32_t row = at + sub < rows ? at + sub : rows - 1;  // lanes behind the last row work on it and store nothing
            const uint32_t t = row / a.heads, h = row % a.heads;
            const float *turn;
            const bool ok = angles(a, t, &turn);
            float y[8];
            normed_and_turned<float, LPR>(a, static_cast<const T *>(a.q) + t * a.q_ts + h * a.q_hs, a.q_weight, turn, i0, y);
            if (!ok) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __builtin_nanf("");
            }
            if (at + sub < rows && i0 < a.dim) store8(static_cast<T *>(a.q_out) + t * a.o_ts + h * a.o_hs + i0, y);
        }
        return;
    }
    const Search sr = load_bucket_table<kWg>(tab, lds);
    __syncthreads();
    const uint32_t rows = a.tokens * a.kv_heads, steps = (rows + kRows - 1) / kRows;  // of keys, and as many of values
    for (uint32_t at = blockIdx.x * kWavesPerWg + wave_in_wg(); at < 2 * steps; at += a.kv_groups * kWavesPerWg) {
        const bool values = at >= steps;
        const uint32_t first = (values ? at - steps : at) * kRows + sub;
        const uint32_t row = first < rows ? first : rows - 1;
        const uint32_t t = row / a.kv_heads, h = row % a.kv_heads;
        const float *turn;
        const bool ok = angles(a, t, &turn);
        float y[8] = {};
        if (values) {
            if (i0 < a.dim) load8(static_cast<const T *>(a.v) + t * a.v_ts + h * a.v_hs + i0, y);
        } else {
            // binary64: whatever order its sums are taken in, the row that is compressed is the same binary32 values
            double d[8];
            normed_and_turned<double, LPR>(a, static_cast<const T *>(a.k) + t * a.k_ts + h * a.k_hs, a.k_weight, turn, i0, d);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = i0 < a.dim ? (float)d[e] : 0.0f;
        }
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = m > abs_bits(y[e]) ? m : abs_bits(y[e]);
        m = group_max_u32<LPR>(m);
        const bool finite = m < 0x7F800000u;  // a row with an infinity or NaN stands for NaN
        const float scale = finite ? u2f(m) : __builtin_nanf(""), d = finite && m ? u2f(m) : 1.0f;
        const v4f z = {0, 0, 0, 0}, lo = finite ? v4f{y[0], y[1], y[2], y[3]} : z, hi = finite ? v4f{y[4], y[5], y[6], y[7]} : z;
        const uint2 word = {encode_quad_own_scale(sr, lo, d), encode_quad_own_scale(sr, hi, d)};
        const uint64_t slot = (uint64_t)a.slots[t];
        if (ok && slot < a.n_slots && first < rows) {
            // row of the cache: ((part * pages + page) * kv_heads + h) * page_size + place
            const uint64_t page = (slot >> a.page_shift) + (values ? a.n_slots >> a.page_shift : 0);
            const uint64_t to = (((page * a.kv_heads + h) << a.page_shift) + (slot & ((1u << a.page_shift) - 1)));
            if (i0 < a.dim) *reinterpret_cast<uint2 *>(a.codes + to * a.dim + i0) = word;
            if (i0 == 0) a.scales[to] = scale;
        }
    }
}

}  // namespace

using dq8::extent;
using dq8::failed;
using dq8::meet;
using dq8::sane;

extern "C" int dq8_cache_append(int kind, const dq8_cache *cache, const dq8_append *in, void *hip_stream)
{
    static const char who[] = "dq8_cache_append";
    int rc = dq8::check_cache(who, kind, cache);
    if (rc) return rc;
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_append &a = *in;
    if (a.type < DQ8_FLOAT32 || a.type > DQ8_FLOAT16) return failed(DQ8_ERR_ARG, "%s: unknown type %d", who, a.type);
    if (a.heads < 0 || a.heads > 65535) return failed(DQ8_ERR_ARG, "%s: %d query heads", who, a.heads);
    if (a.tokens == 0) return DQ8_OK;
    if (!a.k || !a.v || !a.slots || (a.heads > 0 && (!a.q || !a.q_out)) || (a.rotation && !a.positions))
        return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if (a.tokens >= dq8::kCacheLimit || a.tokens * (size_t)(a.heads > cache->kv_heads ? a.heads : cache->kv_heads) >= dq8::kCacheLimit / 2)
        return failed(DQ8_ERR_ARG, "%s: too many tokens", who);
    if (a.heads == 0 && a.q_weight) return failed(DQ8_ERR_ARG, "%s: a norm of queries without queries", who);
    if (a.rotation && (a.half < 1 || 2 * a.half > cache->dim || a.n_positions < 1 || a.n_positions >= dq8::kCacheLimit))
        return failed(DQ8_ERR_ARG, "%s: a rotation of %d pairs in heads of %d elements at %zu positions", who, a.half, cache->dim, a.n_positions);
    if ((a.q_weight || a.k_weight) && !(a.eps >= 0.0 && a.eps <= 1e30)) return failed(DQ8_ERR_ARG, "%s: eps must be finite and not negative", who);
    for (size_t s : {a.q_token_stride, a.q_head_stride, a.k_token_stride, a.k_head_stride, a.v_token_stride, a.v_head_stride,
                     a.q_out_token_stride, a.q_out_head_stride})
        if (!sane(s)) return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
    const size_t size = a.type == DQ8_FLOAT32 ? 4 : 2;
    if ((((uintptr_t)a.k | (uintptr_t)a.v | (a.heads ? (uintptr_t)a.q | (uintptr_t)a.q_out : 0)) & (size - 1)) != 0 ||
        (((uintptr_t)a.rotation | (uintptr_t)a.q_weight | (uintptr_t)a.k_weight) & 3) != 0 || (((uintptr_t)a.slots | (uintptr_t)a.positions) & 7) != 0)
        return failed(DQ8_ERR_ARG, "%s: an array does not start at a multiple of its element's size", who);
    // what is written: the cache and q_out; what is read: everything else
    const size_t rows = dq8::cache_rows(cache);
    const int dim = cache->dim, kv = cache->kv_heads;
    const size_t n_out = extent(a.tokens, a.q_out_token_stride, a.heads, a.q_out_head_stride, dim, size);
    const bool in_place = a.q_out == a.q && a.q_out_token_stride == a.q_token_stride && a.q_out_head_stride == a.q_head_stride;
    const struct {
        const void *p;
        size_t n;
    } read[] = {{in_place ? nullptr : a.q, in_place ? 0 : extent(a.tokens, a.q_token_stride, a.heads, a.q_head_stride, dim, size)},
                {in_place ? nullptr : a.k, extent(a.tokens, a.k_token_stride, kv, a.k_head_stride, dim, size)},
                {in_place ? nullptr : a.v, extent(a.tokens, a.v_token_stride, kv, a.v_head_stride, dim, size)},
                {a.slots, a.tokens * 8},
                {a.positions, a.positions ? a.tokens * 8 : 0},
                {a.rotation, a.rotation ? a.n_positions * 2 * (size_t)a.half * 4 : 0},
                {a.q_weight, a.q_weight ? (size_t)dim * 4 : 0},
                {a.k_weight, a.k_weight ? (size_t)dim * 4 : 0}};
    bool bad = meet(a.q_out, n_out, cache->codes, rows * dim) || meet(a.q_out, n_out, cache->scales, rows * 4) ||
               meet(cache->codes, rows * dim, cache->scales, rows * 4);
    for (const auto &r : read) {
        if (r.p == nullptr) continue;
        bad = bad || meet(r.p, r.n, cache->codes, rows * dim) || meet(r.p, r.n, cache->scales, rows * 4) || meet(r.p, r.n, a.q_out, n_out);
    }
    if (bad) return failed(DQ8_ERR_ARG, "%s: an output overlaps another array", who);
    dq8::DeviceTables dev;
    rc = dq8::device_tables(kind, &dev);
    if (rc) return rc;
    AppendArgs k;
    k.q = a.q, k.k = a.k, k.v = a.v, k.q_out = a.q_out;
    k.q_ts = a.q_token_stride, k.q_hs = a.q_head_stride, k.k_ts = a.k_token_stride, k.k_hs = a.k_head_stride;
    k.v_ts = a.v_token_stride, k.v_hs = a.v_head_stride, k.o_ts = a.q_out_token_stride, k.o_hs = a.q_out_head_stride;
    k.slots = a.slots, k.positions = a.positions, k.rotation = a.rotation, k.q_weight = a.q_weight, k.k_weight = a.k_weight;
    k.codes = cache->codes, k.scales = cache->scales;
    k.n_positions = a.n_positions, k.n_slots = cache->pages * (size_t)cache->page_size, k.eps = a.eps;
    k.tokens = (uint32_t)a.tokens, k.heads = (uint32_t)a.heads, k.kv_heads = (uint32_t)kv, k.dim = (uint32_t)dim;
    k.half = a.rotation ? (uint32_t)a.half : 0, k.interleaved = a.interleaved != 0;
    k.page_shift = (uint32_t)__builtin_ctz((unsigned)cache->page_size);
    const int lpr = dim <= 64 ? 8 : dim <= 128 ? 16 : 32;
    const size_t per = kWavesPerWg * (kWave / lpr);  // rows of a workgroup
    const size_t most = (size_t)dev.cus * 4;
    size_t kv_groups = (2 * a.tokens * kv + per - 1) / per, q_groups = (a.tokens * a.heads + per - 1) / per;
    if (kv_groups > most) kv_groups = most;
    if (q_groups > most) q_groups = most;
    k.kv_groups = (uint32_t)kv_groups;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define DQ8_APPEND(LPR, T) \
    hipLaunchKernelGGL((k_cache_append<LPR, T>), dim3((unsigned)(kv_groups + q_groups)), dim3(kWg), dev.search_words * sizeof(uint32_t), stream, dev.tab, k)
#define DQ8_APPEND_T(T)       \
    switch (lpr) {            \
    case 8: DQ8_APPEND(8, T); break;   \
    case 16: DQ8_APPEND(16, T); break; \
    default: DQ8_APPEND(32, T); break; \
    }
    switch (a.type) {
    case DQ8_FLOAT32: DQ8_APPEND_T(float) break;
    case DQ8_BFLOAT16: DQ8_APPEND_T(__bf16) break;
    default: DQ8_APPEND_T(_Float16) break;
    }
#undef DQ8_APPEND_T
#undef DQ8_APPEND
    return dq8::after_launch_of("k_cache_append", stream);
}
