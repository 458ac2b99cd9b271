// dq8: rows of new keys and values into a paged cache, with the norms and the rotation of queries and keys on the way
// (dq8_cache_append of include/dq8_cache.h).  Built with the flags of dq8.hip: no contraction of products and sums.
//
// A row is `dim` elements of one token and head, held by LPR neighbouring lanes, eight elements each (dim <= 8 LPR), so a
// wavefront works on 64 / LPR rows at a time and the row's sum of squares and maximum are reductions over LPR lanes.  What a
// wavefront is given is an item: item_steps times so many heads of one token, queries, keys or values.  A lane has the same places of
// every head, so that the angles and weights, four times the bytes of a row of 16-bit elements, are loaded once per item.  The steps
// are a loop and not written out: the calls of a decoding step run through this code once, and what they wait for then is the code
// itself (2077 tokens of 12 heads in binary32: 20 us with four steps written out, 13 with the loop).
//
// What bounds it: the vector unit for many rows, busy for 87 % of 54 us at 8191 tokens with 32 + 8 + 8 heads of 128, norms and a rotation (185
// MB, 3.4 TB/s; 35 us at the rates of a large copy; without norms 43 us).  Few tokens take a launch and a chain of loads, 4 to 5 us.
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
    uint32_t item_steps; // of 64 / LPR heads
    uint32_t any_at;     // word of LDS from which on pairs that lie anywhere are exchanged
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

// The value of another lane; lane4: four times its number.
__device__ __forceinline__ float from_lane(float v, int lane4) { return u2f((uint32_t)__builtin_amdgcn_ds_bpermute(lane4, (int)f2u(v))); }

__device__ __forceinline__ double from_lane(double v, int lane4)
{
    int w[2];
    __builtin_memcpy(w, &v, 8);
    w[0] = __builtin_amdgcn_ds_bpermute(lane4, w[0]);
    w[1] = __builtin_amdgcn_ds_bpermute(lane4, w[1]);
    __builtin_memcpy(&v, w, 8);
    return v;
}

// How the elements of a pair lie to each other: the same places of two lanes, two places of a lane, or (kAnywhere) neither.
enum Turn { kNoTurn, kLanes, kInside, kAnywhere };

// What a lane needs of an item beside its rows: cosines and sines of its eight elements' pairs and their weights.
struct Places {
    float c[8], s[8], w[8];
    Turn turn;
    bool normed, low;
    int partner4;  // kLanes: four times the number of the lane with the pairs' other elements
};

// `turning`: the token's row of the table, null without a rotation.
__device__ __forceinline__ Places places_of(const AppendArgs &a, const float *weight, const float *turning, uint32_t i0, uint32_t lane)
{
    Places p = {};
    p.normed = weight != nullptr;
    const bool in = i0 < a.dim;
    if (weight && in) load8(weight + i0, p.w);
    const uint32_t half = a.half;
    p.turn = !turning ? kNoTurn : a.interleaved ? half % 4 == 0 ? kInside : kAnywhere : half % 8 == 0 ? kLanes : kAnywhere;
    p.low = i0 < half;
    if (p.turn == kLanes) {  // (elements behind the rotation: times one, minus zero times something finite or not at all)
        const bool turned = i0 < 2 * half;
        p.partner4 = 4 * (int)(turned ? p.low ? lane + half / 8 : lane - half / 8 : lane);
        const uint32_t p0 = p.low ? i0 : turned ? i0 - half : 0;
        load8(turning + p0, p.c);
        load8(turning + half + p0, p.s);
    } else if (p.turn == kInside && i0 < 2 * half) {
        typedef v4f V __attribute__((aligned(4)));
        const v4f c = *reinterpret_cast<const V *>(turning + i0 / 2), s = *reinterpret_cast<const V *>(turning + half + i0 / 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) p.c[e] = c[e], p.s[e] = s[e];
    }
    return p;
}

// This lane's eight elements of a row (x), normed and turned, in F (double for keys, float for queries).  Lanes whose elements lie behind
// the row have zeros and take part in the sums.  `any`: LDS of this wavefront for pairs that lie anywhere, null where none do.
template <typename F, int LPR, bool ANY>
__device__ __forceinline__ void normed_and_turned(const AppendArgs &a, const Places &p, const float (&x)[8], const float *turning, uint32_t i0,
                                                  uint32_t lane, double *any, F (&y)[8])
{
    const bool in = i0 < a.dim;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[e];
    if (p.normed) {
        F sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += y[e] * y[e];
        sum = row_sum<LPR>(sum);
        F r = F(1) / sqrt(sum / F(a.dim) + F(a.eps));
        if constexpr (sizeof(F) == 4) {  // squares that binary32 does not hold, or holds with few bits where eps does not hide them
            const bool large = sum > 0x1p120f;
            if (large || (sum < 0x1p-100f && a.eps < 0x1p-33)) {  // (the same for all lanes of a row)
                const float by = large ? 0x1p-80f : 0x1p80f;
                sum = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += (y[e] * by) * (y[e] * by);
                r = by / sqrt(row_sum<LPR>(sum) / F(a.dim) + (float)(a.eps * (double)by * (double)by));
            }
        }
        if (in)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = y[e] * r * F(p.w[e]);
    }
    const bool turned = i0 < 2 * a.half;
    if (p.turn == kLanes) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const F o = from_lane(y[e], p.partner4), t = o * F(p.s[e]);
            if (turned) y[e] = y[e] * F(p.c[e]) + (p.low ? -t : t);
        }
    } else if (p.turn == kInside) {
        if (turned)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const F c = p.c[e / 2], s = p.s[e / 2], u = y[e], v = y[e + 1];
                y[e] = u * c - v * s;
                y[e + 1] = v * c + u * s;
            }
    }
    if constexpr (ANY) {
        if (p.turn == kNoTurn) return;
        F *const row = reinterpret_cast<F *>(any) + (lane / LPR) * (8 * LPR);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < 8; ++e) row[i0 + e] = y[e];
        __builtin_amdgcn_wave_barrier();
        const uint32_t half = a.half;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t i = i0 + e;
            if (i < 2 * half) {
                const bool low = a.interleaved ? i % 2 == 0 : i < half;
                const uint32_t j = a.interleaved ? i ^ 1 : low ? i + half : i - half, q = a.interleaved ? i / 2 : low ? i : j;
                const F t = row[j] * F(turning[half + q]);
                y[e] = y[e] * F(turning[q]) + (low ? -t : t);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The angles of token t; false where its position has none.  Without a rotation: no angles, true.
__device__ __forceinline__ bool angles(const AppendArgs &a, uint32_t t, const float **turning)
{
    *turning = nullptr;
    if (!a.rotation) return true;
    const uint64_t p = (uint64_t)a.positions[t];
    const bool ok = p < a.n_positions;
    *turning = a.rotation + (ok ? p : 0) * 2 * a.half;
    return ok;
}

// kv_groups of the workgroups, spread evenly over all, walk the items of keys, then those of values (the vector unit bounds these); the
// others walk those of queries (the memory does).
// ANY: pairs lie anywhere (kernels of their own: the addresses that such pairs need cost the others registers).
template <int LPR, bool ANY, typename T>
__global__ __launch_bounds__(kWg, ANY ? 4 : 5) void k_cache_append(const uint32_t *__restrict__ tab, AppendArgs a)
{
    extern __shared__ uint32_t lds[];
    constexpr uint32_t kRows = kWave / LPR;  // heads at a time
    const uint32_t item_heads = kRows * a.item_steps;
    const uint32_t lane = threadIdx.x & 63, i0 = (lane % LPR) * 8, sub = lane / LPR;
    typedef typename Eight<T>::type Raw;
    typedef Raw RawAny __attribute__((aligned(sizeof(T))));
    double *const any = reinterpret_cast<double *>(lds + a.any_at) + wave_in_wg() * (kWave * 8);
    // this lane's elements of a head
    auto request = [&](const T *token, size_t stride, uint32_t h, uint32_t heads) {
        Raw raw = {};
        if (h < heads && i0 < a.dim) raw = *reinterpret_cast<const RawAny *>(token + h * stride + i0);
        return raw;
    };
    const uint32_t kv_before = blockIdx.x * a.kv_groups / gridDim.x, kv_upto = (blockIdx.x + 1) * a.kv_groups / gridDim.x;
    if (kv_before == kv_upto) {
        const uint32_t per = (a.heads + item_heads - 1) / item_heads, items = a.tokens * per, step = (gridDim.x - a.kv_groups) * kWavesPerWg;
        for (uint32_t at = (blockIdx.x - kv_before) * kWavesPerWg + wave_in_wg(); at < items; at += step) {
            const uint32_t t = at / per, h0 = (at - t * per) * item_heads, end = h0 + item_heads < a.heads ? h0 + item_heads : a.heads;
            const T *const from = static_cast<const T *>(a.q) + t * a.q_ts;
            T *const to = static_cast<T *>(a.q_out) + t * a.o_ts;
            Raw next = request(from, a.q_hs, h0 + sub, end);
            const float *turning;
            const bool ok = angles(a, t, &turning);
            const Places p = places_of(a, a.q_weight, turning, i0, lane);
#pragma unroll 1
            for (uint32_t h1 = h0; h1 < end; h1 += kRows) {
                const uint32_t h = h1 + sub;
                float x[8], y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = (float)next[e];
                next = request(from, a.q_hs, h + kRows, end);
                normed_and_turned<float, LPR, ANY>(a, p, x, turning, i0, lane, any, y);
                if (!ok) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = __builtin_nanf("");
                }
                if (h < a.heads && i0 < a.dim) store8(to + h * a.o_hs + i0, y);
            }
        }
        return;
    }
    const Search sr = load_bucket_table<kWg>(tab, lds);
    __syncthreads();
    const uint32_t per = (a.kv_heads + item_heads - 1) / item_heads, items = a.tokens * per;  // of keys, and as many of values
    for (uint32_t at = kv_before * kWavesPerWg + wave_in_wg(); at < 2 * items; at += a.kv_groups * kWavesPerWg) {
        const bool values = at >= items;
        const uint32_t item = values ? at - items : at, t = item / per, h0 = (item - t * per) * item_heads, end = h0 + item_heads < a.kv_heads ? h0 + item_heads : a.kv_heads;
        const T *const from = values ? static_cast<const T *>(a.v) + t * a.v_ts : static_cast<const T *>(a.k) + t * a.k_ts;
        const size_t stride = values ? a.v_hs : a.k_hs;
        Raw next = request(from, stride, h0 + sub, end);
        const float *turning;
        const bool ok = angles(a, t, &turning);
        const uint64_t slot = (uint64_t)a.slots[t];
        if (!(ok && slot < a.n_slots)) continue;  // (uniform)
        if (values) turning = nullptr;
        const float *const weight = values ? nullptr : a.k_weight;
        Places p = places_of(a, weight, turning, i0, lane);
        // row of the cache: ((part * pages + page) * kv_heads + h) * page_size + place
        const uint64_t page = (slot >> a.page_shift) + (values ? a.n_slots >> a.page_shift : 0), place = slot & ((1u << a.page_shift) - 1);
#pragma unroll 1
        for (uint32_t h1 = h0; h1 < end; h1 += kRows) {
            const uint32_t h = h1 + sub;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (float)next[e];
            next = request(from, stride, h + kRows, end);
            if (p.normed || p.turn != kNoTurn) {
                // (made to look new: the 24 of them in binary64, kept for the loop, would be 48 registers)
#pragma unroll
                for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(p.c[e]), "+v"(p.s[e]), "+v"(p.w[e]));
                // binary64: whatever order its sums are taken in, the row that is compressed is the same binary32 values
                double d[8];
                normed_and_turned<double, LPR, ANY>(a, p, y, turning, i0, lane, any, d);
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
            if (h < a.kv_heads) {
                const uint64_t to = ((page * a.kv_heads + h) << a.page_shift) + place;
                if (i0 < a.dim) *reinterpret_cast<uint2 *>(a.codes + to * a.dim + i0) = word;
                if (i0 == 0) a.scales[to] = scale;
            }
        }
    }
}

}  // namespace

using dq8::apart;
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
    const size_t kv_heads = (size_t)cache->kv_heads, heads = (size_t)a.heads;
    for (size_t s : {a.q_token_stride, a.k_token_stride, a.v_token_stride, a.q_out_token_stride})
        if (!sane(s, a.tokens)) return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
    if (!sane(a.q_head_stride, heads) || !sane(a.q_out_head_stride, heads) || !sane(a.k_head_stride, kv_heads) || !sane(a.v_head_stride, kv_heads))
        return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
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
                {a.k, extent(a.tokens, a.k_token_stride, kv, a.k_head_stride, dim, size)},
                {a.v, extent(a.tokens, a.v_token_stride, kv, a.v_head_stride, dim, size)},
                {a.slots, a.tokens * 8},
                {a.positions, a.positions ? a.tokens * 8 : 0},
                {a.rotation, a.rotation ? a.n_positions * 2 * (size_t)a.half * 4 : 0},
                {a.q_weight, a.q_weight ? (size_t)dim * 4 : 0},
                {a.k_weight, a.k_weight ? (size_t)dim * 4 : 0}};
    bool bad = meet(a.q_out, n_out, cache->codes, rows * dim) || meet(a.q_out, n_out, cache->scales, rows * 4) ||
               meet(cache->codes, rows * dim, cache->scales, rows * 4);
    // keys or values and queries in place that are parts of the same tokens: they lie side by side in each
    auto beside = [&](const void *p, size_t token_stride, size_t head_stride) {
        const intptr_t stride = (intptr_t)(a.q_out_token_stride * size);
        if (!in_place || token_stride != a.q_out_token_stride || stride == 0) return false;
        const intptr_t from = ((intptr_t)p - (intptr_t)a.q_out) % stride, at = from < 0 ? from + stride : from;
        return at >= (intptr_t)extent(1, 0, a.heads, a.q_out_head_stride, dim, size) && at + (intptr_t)extent(1, 0, kv, head_stride, dim, size) <= stride;
    };
    for (const auto &r : read) {
        if (r.p == nullptr) continue;
        const bool side = (r.p == a.k && beside(a.k, a.k_token_stride, a.k_head_stride)) || (r.p == a.v && beside(a.v, a.v_token_stride, a.v_head_stride));
        bad = bad || meet(r.p, r.n, cache->codes, rows * dim) || meet(r.p, r.n, cache->scales, rows * 4) || (!side && meet(r.p, r.n, a.q_out, n_out));
    }
    bad = bad || !apart(a.tokens, a.q_out_token_stride, a.heads, a.q_out_head_stride, dim);
    if (bad) return failed(DQ8_ERR_ARG, "%s: an output overlaps another array or itself", who);
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
    // Items of four times the heads that a wavefront has at once where there are many, of one time where every wavefront counts (32 + 8 + 8 heads
    // of 128 in 16 bits, us with one | four: 64 tokens 4.5 | 5.6, 256 5.5 | 5.9, 512 7.9 | 6.7, 2048 19 | 13, 8192 59 | 42).
    const size_t at_once = (size_t)(kWave / lpr);
    auto items = [&](size_t steps) { return a.tokens * ((heads + at_once * steps - 1) / (at_once * steps) + 2 * ((kv + at_once * steps - 1) / (at_once * steps))); };
    k.item_steps = items(4) >= (size_t)dev.cus * 8 ? 4 : 1;
    const size_t per = at_once * k.item_steps, most = (size_t)dev.cus * 5;  // that are resident (four: 47 us, five 43, eight 43 at 8192)
    const size_t kv_items = 2 * a.tokens * ((kv + per - 1) / per), q_items = a.tokens * ((heads + per - 1) / per);
    size_t kv_groups = (kv_items + kWavesPerWg - 1) / kWavesPerWg, q_groups = (q_items + kWavesPerWg - 1) / kWavesPerWg;
    if (kv_groups + q_groups > most) {
        const size_t share = most * kv_items / (kv_items + q_items);
        kv_groups = share < 1 ? 1 : kv_groups < share ? kv_groups : share;
        if (q_groups > most - kv_groups) q_groups = most - kv_groups;
    }
    k.kv_groups = (uint32_t)kv_groups;
    k.any_at = dev.search_words;  // (whole quads)
    const bool anywhere = a.rotation && a.half % (a.interleaved ? 4 : 8) != 0;
    const size_t lds = dev.search_words * sizeof(uint32_t) + (anywhere ? kWg * 8 * sizeof(double) : 0);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define DQ8_APPEND(LPR, T)                                                                                                                  \
    if (anywhere)                                                                                                                           \
        hipLaunchKernelGGL((k_cache_append<LPR, true, T>), dim3((unsigned)(kv_groups + q_groups)), dim3(kWg), lds, stream, dev.tab, k);     \
    else                                                                                                                                    \
        hipLaunchKernelGGL((k_cache_append<LPR, false, T>), dim3((unsigned)(kv_groups + q_groups)), dim3(kWg), lds, stream, dev.tab, k)
#define DQ8_APPEND_T(T)                \
    switch (lpr) {                     \
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
