// dq8: attention of new tokens over a paged cache of 8-bit keys and values (dq8_cache_attention of include/dq8_cache.h).
//
// Mathematics.  For a query row q and the cached tokens j that it sees, with weights p_j = exp2(t_j - m), t_j = log2(e) softmax_scale q . k_j
// and m the largest t_j so far:  out = sum p_j v_j / sum p_j.  Both sums and m are carried through one pass over the tokens; when m grows they
// are multiplied by exp2(m_old - m_new).  k_j = ks_j cb[kc_j] and v_j = vs_j cb[vc_j] (one scale per row), so the scales leave the
// products: t_j = (sum_d q_d cb[kc_jd]) ks_j c, and vs_j joins the weight p_j.
//
// Matrix instructions (16x16x32, binary16 in, binary32 sums).  All queries that share a cached head are rows of one product, so a code
// is looked up once for all of them.  Transposed products keep everything in the lanes where it is needed next: S^T = K Q^T has a query
// per column, lane % 16, and four tokens in a lane's registers; out^T = V^T P^T wants P^T with a query per column and eight tokens
// per lane.  Which token stands at which place of that sum is free as long as V^T has the same, so two S^T tiles of 16 tokens are
// P^T as they are, and no weight ever leaves its lane.  In the same way the order of the elements d in q . k is that in which 16-byte
// loads deliver a row's codes, and the order of the output's elements that in which a lane's load delivers a value row's.
//
// Codes become binary16 through the table in LDS that dq8_decode uses, one copy per lane (dq8_device.hpp).  Its entries are
// cb[c] * 32 * 1280 (linear: * 256 * 127): the magnitudes above a tenth of the maximum are whole numbers of 1/1280 there, at most 1920,
// so that binary16's 11 bits hold them exactly; smaller ones are rounded once, and the smallest but zero is above 2^-12, none subnormal.
// (With entries cb[c] 2^15, all rounded, binary16 outputs were off by 4.9e-4 of their size, 2.1e-4 of it their own rounding.)  A query
// row is scaled by a power of two to a largest element of 2^14 .. 2^15, weights times value scales by a power of two to at most
// 2^15 (kWeightTop), which the accumulators are followed by when a larger scale appears.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "dq8_cache_check.hpp"
#include "dq8_device.hpp"

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;          // tokens that a wavefront takes at a time
constexpr int kAttendWaves = 4;    // of a workgroup
constexpr int kAttendWg = kAttendWaves * kWave;
constexpr int kQueryTop = 14;      // a query row's largest element is in [2^14, 2^15) in binary16
constexpr int kWeightTop = 14;     // the largest value scale so far is in [2^14, 2^15) where it multiplies a weight
constexpr int kLeastExp = -90;     // of scales and queries that are still brought to those ranges
constexpr float kNothing = -FLT_MAX;  // the running maximum before anything was seen

struct AttendArgs {
    const void *q;
    void *out;
    size_t q_ts, q_hs, o_ts, o_hs;
    const uint8_t *k_codes, *v_codes;
    const float *k_scales, *v_scales;
    const int32_t *pages, *lens, *starts;
    uint32_t tokens, batch, each, heads, kv_heads, group, dim, n_pages, max_pages, page_shift;
    int32_t window;
    float entry;   // table entries are cb[c] * entry
    float factor;  // log2(e) * softmax_scale / entry
    // workspace (null: no job is split)
    int4 *records;  // per workgroup: the job that begins there and is finished by others: sequence, job, parts
    float2 *sums;   // per part: maximum and sum of weights of each query row
    v4 *parts;      // per part: weighted values, one float4 per lane and block (see Blocks)
};

// A sequence's part of the work.
struct Seq {
    uint32_t first, n;     // its new tokens in q
    int32_t len;           // cached tokens
    uint32_t lo_tile, tiles;  // tiles of kTile tokens that its queries see: lo_tile .. lo_tile + tiles - 1, one at least
    uint32_t q_tiles;      // groups of `rows` query rows per cached head; a job is one of them with one head
};

__device__ __forceinline__ Seq sequence(const AttendArgs &a, uint32_t b, uint32_t rows)
{
    Seq s;
    uint32_t end;
    if (a.starts) {
        const int32_t s0 = a.starts[b], s1 = a.starts[b + 1];
        s.first = s0 < 0 ? 0 : (uint32_t)s0 < a.tokens ? (uint32_t)s0 : a.tokens;
        end = s1 < 0 ? 0 : (uint32_t)s1 < a.tokens ? (uint32_t)s1 : a.tokens;
        if (end < s.first) end = s.first;
    } else {
        s.first = b * a.each;
        end = s.first + a.each;
    }
    s.n = end - s.first;
    const int32_t most = (int32_t)(a.max_pages << a.page_shift), len = a.lens[b];
    s.len = len < 0 ? 0 : len < most ? len : most;
    int32_t lo = a.window > 0 ? s.len - (int32_t)s.n + 1 - a.window : 0;
    if (lo < 0) lo = 0;
    s.lo_tile = (uint32_t)lo / kTile;
    const uint32_t hi = ((uint32_t)s.len + kTile - 1) / kTile;
    s.tiles = hi > s.lo_tile ? hi - s.lo_tile : 1;
    s.q_tiles = (s.n * a.group + rows - 1) / rows;
    return s;
}

__device__ __forceinline__ uint64_t work_of(const AttendArgs &a, const Seq &s) { return (uint64_t)s.q_tiles * a.kv_heads * s.tiles; }

__device__ __forceinline__ uint64_t wave_scan(uint64_t v, uint32_t lane)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint64_t o = __shfl_up(v, d);
        if (lane >= (uint32_t)d) v += o;
    }
    return v;
}

// The tiles of all jobs, in the order of sequences, query groups, heads, tokens, are one line that is cut into equal parts, one per
// workgroup: whatever the lengths of the sequences, everybody reads as much.  `at`: where this workgroup's part begins.
struct Share {
    uint64_t total, begin, end;
    uint32_t groups;  // workgroups that have a part
    uint32_t b;       // sequence and place in its work of the first tile
    uint64_t place;
};

__device__ __forceinline__ Share share_of(const AttendArgs &a, uint32_t rows, uint64_t *lds)
{
    // lds: kAttendWaves + 3 words
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share s;
    uint64_t total = 0, mine = 0;
    for (uint32_t b = threadIdx.x; b < a.batch; b += kAttendWg) mine += work_of(a, sequence(a, b, rows));
    const uint64_t sum = wave_scan(mine, lane);
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    for (int w = 0; w < kAttendWaves; ++w) total += lds[w];
    s.total = total;
    // at least a tile for every wavefront of a workgroup
    const uint64_t most = (total + kAttendWaves - 1) / kAttendWaves;
    s.groups = (uint32_t)(gridDim.x < most ? gridDim.x : most);
    s.b = 0;
    s.place = 0;
    if (blockIdx.x >= s.groups) {
        s.begin = s.end = 0;
        return s;
    }
    s.begin = total * blockIdx.x / s.groups;
    s.end = total * (blockIdx.x + 1) / s.groups;
    // the sequence that holds `begin`
    uint64_t before = 0;
    for (uint32_t b0 = 0; b0 < a.batch; b0 += kAttendWg) {
        __syncthreads();
        const uint32_t b = b0 + threadIdx.x;
        const uint64_t w = b < a.batch ? work_of(a, sequence(a, b, rows)) : 0;
        const uint64_t upto = wave_scan(w, lane);
        if (lane == 63) lds[wave] = upto;
        __syncthreads();
        uint64_t base = before;
        for (uint32_t v = 0; v < wave; ++v) base += lds[v];
        if (s.begin >= base + upto - w && s.begin < base + upto) {
            lds[kAttendWaves + 1] = b;
            lds[kAttendWaves + 2] = s.begin - (base + upto - w);
        }
        for (int v = 0; v < kAttendWaves; ++v) before += lds[v];
        if (s.begin < before) break;
    }
    __syncthreads();
    s.b = (uint32_t)lds[kAttendWaves + 1];
    s.place = lds[kAttendWaves + 2];
    return s;
}

// Table with entries in binary16, in both halves of a word; see place_lut.
__device__ __forceinline__ void place_half_table(const uint32_t *tab, float entry, uint32_t *lds)
{
    const _Float16 h = (_Float16)(u2f(tab[kCbOff + (threadIdx.x & 255)]) * entry);
    uint16_t u;
    __builtin_memcpy(&u, &h, 2);
    place_lut<kAttendWg>(u2f(u | ((uint32_t)u << 16)), reinterpret_cast<float *>(lds));
}

template <int J>
__device__ __forceinline__ _Float16 half_at(const uint32_t *lut, uint32_t w, uint32_t lane4)
{
    const uint32_t addr = __builtin_amdgcn_perm(w, lane4, 0x0C0C0400u + (J << 8));
    return *reinterpret_cast<const _Float16 *>(reinterpret_cast<const char *>(lut) + addr);
}

// Eight codes, lowest byte first.
__device__ __forceinline__ v8h eight(const uint32_t *lut, uint32_t lo, uint32_t hi, uint32_t lane4)
{
    return v8h{half_at<0>(lut, lo, lane4), half_at<1>(lut, lo, lane4), half_at<2>(lut, lo, lane4), half_at<3>(lut, lo, lane4),
               half_at<0>(lut, hi, lane4), half_at<1>(lut, hi, lane4), half_at<2>(lut, hi, lane4), half_at<3>(lut, hi, lane4)};
}

__device__ __forceinline__ float max_over_groups(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

__device__ __forceinline__ float sum_over_groups(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// Exponent e with 2^e <= v < 2^(e + 1), at least kLeastExp; v is not negative (0, infinities and NaN give some value in range).
__device__ __forceinline__ int exponent(float v)
{
    const int e = (int)(f2u(v) >> 23) - 127;
    return e < kLeastExp ? kLeastExp : e > 127 ? 127 : e;
}

template <int N>
struct Bytes;
template <>
struct Bytes<4> {
    typedef uint32_t type __attribute__((aligned(4)));
};
template <>
struct Bytes<8> {
    typedef uint32_t type __attribute__((ext_vector_type(2), aligned(8)));
};
template <>
struct Bytes<16> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(16)));
};

// What a wavefront loads of a tile: lane l holds of keys the rows l % 16 of both halves of 16 tokens, 16 bytes of every 64, and
// of values the bytes CPL (l % 16) .. of the eight tokens whose weights it will hold.
template <int DP>
struct TileData {
    static constexpr int kLoads = DP / 64, CPL = DP / 16;
    u4 k[2][kLoads];
    typename Bytes<CPL>::type v[8];
    v4 ks[2], vs[2];
    uint32_t valid;  // bit h: half h lies on a page of the cache
};

template <int DP>
__device__ __forceinline__ void fetch(const AttendArgs &a, const int32_t *table, uint32_t head, uint32_t tile, uint32_t lane, TileData<DP> &d)
{
    constexpr int CPL = DP / 16;
    const uint32_t m = lane & 15, g = lane >> 4;
    d.valid = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t token = tile * kTile + h * 16;
        uint32_t index = token >> a.page_shift;
        index = index < a.max_pages ? index : a.max_pages - 1;  // behind the last page: not seen by anybody
        const uint32_t page = (uint32_t)__builtin_amdgcn_readfirstlane(table[index]);
        const bool ok = page < a.n_pages;
        d.valid |= ok ? 1u << h : 0;
        const uint64_t row = ((((uint64_t)(ok ? page : 0) * a.kv_heads + head) << a.page_shift) + (token & ((1u << a.page_shift) - 1)));
        const uint8_t *kc = a.k_codes + (row + m) * a.dim, *vc = a.v_codes + (row + 4 * g) * a.dim;
#pragma unroll
        for (int c = 0; c < TileData<DP>::kLoads; ++c) {
            const uint32_t at = 64 * c + 16 * g;
            d.k[h][c] = *reinterpret_cast<const u4 *>(kc + (at < a.dim ? at : 0));
        }
        const uint32_t at = m * CPL < a.dim ? m * CPL : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) d.v[4 * h + i] = *reinterpret_cast<const typename Bytes<CPL>::type *>(vc + (size_t)i * a.dim + at);
        d.ks[h] = *reinterpret_cast<const v4 *>(a.k_scales + row + 4 * g);
        d.vs[h] = *reinterpret_cast<const v4 *>(a.v_scales + row + 4 * g);
    }
}

template <int N>
__device__ __forceinline__ uint32_t word_of(const typename Bytes<N>::type &v, int i)
{
    if constexpr (N == 4)
        return v;
    else
        return v[i];
}

// Weighted values (as sums of table entries) over the sum of weights; zeros where there was none.
__device__ __forceinline__ v4 mean_of(const AttendArgs &a, v4 sum, float weights)
{
    return weights == 0.0f ? v4{0, 0, 0, 0} : sum * (1.0f / (weights * a.entry));
}

// Where a query row's output goes: lane's column, block (tile j of 16 elements, group nt of 16 rows).
template <typename T, int DP>
__device__ __forceinline__ void store_block(const AttendArgs &a, const Seq &s, uint32_t head, uint32_t row, uint32_t j, v4 value, uint32_t lane)
{
    constexpr int CPL = DP / 16;
    if (row >= s.n * a.group) return;
    T *to = static_cast<T *>(a.out) + (s.first + row / a.group) * a.o_ts + (head * a.group + row % a.group) * a.o_hs;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t d = CPL * (4 * (lane >> 4) + i) + j;
        if (d < a.dim) to[d] = (T)value[i];
    }
}

// One job's tiles t0 .. t1 - 1: query rows q_tile * 16 NT .. of a sequence against a cached head.  part: where the sums go if the job is
// not finished here (-1: it is, and the output is stored).
template <int DP, int NT, typename T>
__device__ void attend(const AttendArgs &a, const Seq &s, uint32_t b, uint32_t q_tile, uint32_t head, uint32_t t0, uint32_t t1, int64_t part,
                       const uint32_t *lut, float *area)
{
    constexpr int CPL = DP / 16, KS = DP / 32;
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, lane4 = lane * 4, wave = wave_in_wg();
    const int32_t *table = a.pages + (size_t)b * a.max_pages;
    v8h q[NT][KS];
    float scale[NT], top[NT], sum[NT];
    int32_t pos[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const uint32_t row = (q_tile * NT + nt) * 16 + n;
        const bool in = row < s.n * a.group;
        const uint32_t token = in ? row / a.group : 0, qh = in ? row % a.group : 0;
        pos[nt] = in ? s.len - (int32_t)s.n + (int32_t)token : -1;
        const T *src = static_cast<const T *>(a.q) + (s.first + token) * a.q_ts + (head * a.group + qh) * a.q_hs;
        float x[KS][8], most = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const uint32_t d = 16 * (g + 4 * (k / 2)) + 8 * (k % 2);
            typedef T V __attribute__((ext_vector_type(8)));
            typedef V VA __attribute__((aligned(sizeof(T))));
            const bool there = in && d < a.dim;
            V v = {};
            if (there) v = *reinterpret_cast<const VA *>(src + d);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[k][e] = (float)v[e];
                most = fmaxf(most, fabsf(x[k][e]));
            }
        }
        const int e = exponent(max_over_groups(most));
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[nt][k][i] = (_Float16)__builtin_amdgcn_ldexpf(x[k][i], kQueryTop - e);
        scale[nt] = __builtin_amdgcn_ldexpf(a.factor, e - kQueryTop);
        top[nt] = kNothing;
        sum[nt] = 0.0f;
    }
    v4 acc[NT][CPL];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < CPL; ++j) acc[nt][j] = v4{0, 0, 0, 0};
    int vexp = kLeastExp;  // exponent of the largest value scale so far
    const int32_t p_first = s.len - (int32_t)s.n;  // position of the sequence's first query, the least of any row here

    auto work = [&](uint32_t tile, const TileData<DP> &d) {
        const int32_t t = (int32_t)(tile * kTile);
        // whether some row does not see some token of the tile (a window's lower end: rows up to the last position)
        const bool masked = t + kTile - 1 > p_first || (a.window > 0 && t <= s.len - 1 - a.window) || d.valid != 3;
        v4 st[NT][2];
        v4 ks[2] = {d.ks[0], d.ks[1]}, vs[2] = {d.vs[0], d.vs[1]};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) st[nt][h] = v4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const v8h f = eight(lut, d.k[h][k / 2][2 * (k % 2)], d.k[h][k / 2][2 * (k % 2) + 1], lane4);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) st[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q[nt][k], st[nt][h], 0, 0, 0);
            }
        }
        if (masked) {  // scales of tokens that nobody here sees do not count
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t + 16 * h + 4 * (int32_t)g + i >= s.len || !(d.valid >> h & 1)) vs[h][i] = 0.0f;
        }
        float most = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, vs[h][i]);
        const int e = __builtin_amdgcn_readfirstlane(exponent(max_over_groups(most)));
        if (e > vexp) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < CPL; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nt][j][i] = __builtin_amdgcn_ldexpf(acc[nt][j][i], vexp - e);
            vexp = e;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) vs[h][i] = __builtin_amdgcn_ldexpf(vs[h][i], kWeightTop - vexp);
        v8h p[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float high = kNothing;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = st[nt][h][i] * (ks[h][i] * scale[nt]);
                    if (masked) {
                        const int32_t token = t + 16 * h + 4 * (int32_t)g + i;
                        const bool seen = token <= pos[nt] && (a.window <= 0 || token > pos[nt] - a.window) && (d.valid >> h & 1);
                        v = seen ? v : -__builtin_inff();
                    }
                    st[nt][h][i] = v;
                    high = fmaxf(high, v);
                }
            if (__builtin_amdgcn_ballot_w64(high > top[nt]) != 0) {
                const float now = fmaxf(top[nt], max_over_groups(high)), less = __builtin_amdgcn_exp2f(top[nt] - now);
                sum[nt] *= less;
#pragma unroll
                for (int j = 0; j < CPL; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nt][j][i] *= less;
                top[nt] = now;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(st[nt][h][i] - top[nt]);
                    sum[nt] += w;
                    // a hidden token's scale may be anything, and its weight is zero
                    p[nt][4 * h + i] = (_Float16)(masked && !(st[nt][h][i] > -__builtin_inff() || st[nt][h][i] != st[nt][h][i]) ? 0.0f : w * vs[h][i]);
                }
        }
#pragma unroll
        for (int j = 0; j < CPL; ++j) {
            // byte j of the eight tokens' words
            v8h f;
            const uint32_t sel = 0x0C0C0400u + ((j & 3) << 8);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f[i] = *reinterpret_cast<const _Float16 *>(reinterpret_cast<const char *>(lut) +
                                                           __builtin_amdgcn_perm(word_of<CPL>(d.v[i], j / 4), lane4, sel));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, p[nt], acc[nt][j], 0, 0, 0);
        }
    };

    uint32_t tile = s.lo_tile + t0 + wave;
    const uint32_t end = s.lo_tile + t1;
    if (tile < end) {
        TileData<DP> x, y;
        fetch<DP>(a, table, head, tile, lane, x);
        for (;;) {
            uint32_t next = tile + kAttendWaves;
            fetch<DP>(a, table, head, next < end ? next : tile, lane, y);
            work(tile, x);
            if (next >= end) break;
            tile = next;
            next = tile + kAttendWaves;
            fetch<DP>(a, table, head, next < end ? next : tile, lane, x);
            work(tile, y);
            if (next >= end) break;
            tile = next;
        }
    }

    // The four wavefronts' sums become one: maxima and sums of weights first, then the weighted values, four blocks of 16 x 16 at a time,
    // of which every wavefront adds one.
    float2 *ml = reinterpret_cast<float2 *>(area);
    __syncthreads();  // (the area may still be read for the job before)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        sum[nt] = sum_over_groups(sum[nt]);
        if (g == 0) ml[(wave * NT + nt) * 16 + n] = float2{top[nt], sum[nt]};
    }
    __syncthreads();
    float all[NT], whole[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        all[nt] = kNothing;
        whole[nt] = 0.0f;
        for (int w = 0; w < kAttendWaves; ++w) all[nt] = fmaxf(all[nt], ml[(w * NT + nt) * 16 + n].x);
        for (int w = 0; w < kAttendWaves; ++w) {
            const float2 o = ml[(w * NT + nt) * 16 + n];
            whole[nt] += o.y * __builtin_amdgcn_exp2f(o.x - all[nt]);
        }
        const float mine = __builtin_amdgcn_exp2f(top[nt] - all[nt]);
#pragma unroll
        for (int j = 0; j < CPL; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[nt][j][i] = __builtin_amdgcn_ldexpf(acc[nt][j][i] * mine, vexp - kWeightTop);
    }
    if (part >= 0 && wave == 0 && g == 0)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) a.sums[(size_t)part * NT * 16 + nt * 16 + n] = float2{all[nt], whole[nt]};
    v4 *blocks = reinterpret_cast<v4 *>(area);
#pragma unroll
    for (int c = 0; c < CPL * NT; c += 4) {  // block c + u: group (c + u) % NT, tile (c + u) / NT
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) blocks[(u * kAttendWaves + wave) * kWave + lane] = acc[(c + u) % NT][(c + u) / NT];
        __syncthreads();
        v4 v = {0, 0, 0, 0};
        for (int w = 0; w < kAttendWaves; ++w) v += blocks[(wave * kAttendWaves + w) * kWave + lane];
        const uint32_t at = c + wave, nt = at % NT, j = at / NT;
        if (part >= 0) {
            a.parts[((size_t)part * CPL * NT + at) * kWave + lane] = v;
        } else {
            float l = 0.0f;
#pragma unroll
            for (int i = 0; i < NT; ++i) l = i == (int)nt ? whole[i] : l;
            store_block<T, DP>(a, s, head, (q_tile * NT + nt) * 16 + n, j, mean_of(a, v, l), lane);
        }
    }
}

template <int DP, int NT, typename T>
__global__ __launch_bounds__(kAttendWg) void k_cache_attend(const uint32_t *__restrict__ tab, AttendArgs a)
{
    __shared__ __align__(256) uint32_t lds[256 * kLutCopies + 4096];
    float *area = reinterpret_cast<float *>(lds + 256 * kLutCopies);
    place_half_table(tab, a.entry, lds);
    const Share share = share_of(a, 16 * NT, reinterpret_cast<uint64_t *>(area));
    __syncthreads();
    uint32_t b = (uint32_t)__builtin_amdgcn_readfirstlane(share.b);
    uint64_t place = share.place, at = share.begin;
    int4 record = {0, 0, 0, 0};
    while (at < share.end && b < a.batch) {
        const Seq s = sequence(a, b, 16 * NT);
        const uint64_t work = work_of(a, s);
        if (place >= work) {  // the next sequence
            ++b;
            place = 0;
            continue;
        }
        const uint32_t job = (uint32_t)(place / s.tiles);
        uint32_t t0 = (uint32_t)(place % s.tiles), t1 = s.tiles;
        const uint64_t left = share.end - at;
        int64_t part = -1;
        if (a.parts) {
            if (left < t1 - t0) t1 = t0 + (uint32_t)left;
            if (t0 > 0 || t1 < s.tiles) part = 2 * (int64_t)blockIdx.x + (t0 == 0);
            if (t0 == 0 && t1 < s.tiles) {  // finished by the workgroups whose parts reach the job's end
                const uint64_t end = at + s.tiles;
                record = int4{(int)b, (int)job, (int)((end * share.groups + share.total - 1) / share.total - blockIdx.x), 0};
            }
            attend<DP, NT, T>(a, s, b, job / a.kv_heads, job % a.kv_heads, t0, t1, part, lds, area);
        } else if (t0 == 0) {  // whole jobs: those that begin in this part
            attend<DP, NT, T>(a, s, b, job / a.kv_heads, job % a.kv_heads, t0, t1, -1, lds, area);
        }
        place += t1 - t0;
        at += t1 - t0;
    }
    if (a.parts && threadIdx.x == 0) a.records[blockIdx.x] = record;
}

// A job that several workgroups worked on: workgroup w of this launch joins the parts of the job that began in workgroup w of the
// other.
template <int DP, int NT, typename T>
__global__ __launch_bounds__(kAttendWg) void k_cache_join(AttendArgs a)
{
    constexpr int CPL = DP / 16;
    const int4 record = a.records[blockIdx.x];
    if (record.z == 0) return;
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, wave = wave_in_wg();
    const Seq s = sequence(a, (uint32_t)record.x, 16 * NT);
    const uint32_t head = (uint32_t)record.y % a.kv_heads, q_tile = (uint32_t)record.y / a.kv_heads;
    auto part_of = [&](int i) { return 2 * ((size_t)blockIdx.x + i) + (i == 0); };
    for (uint32_t at = wave; at < CPL * NT; at += kAttendWaves) {
        const uint32_t nt = at % NT, j = at / NT;
        float top = kNothing, l = 0.0f;
        for (int i = 0; i < record.z; ++i) top = fmaxf(top, a.sums[part_of(i) * NT * 16 + nt * 16 + n].x);
        v4 v = {0, 0, 0, 0};
        for (int i = 0; i < record.z; ++i) {
            const float2 o = a.sums[part_of(i) * NT * 16 + nt * 16 + n];
            const float f = __builtin_amdgcn_exp2f(o.x - top);
            l += o.y * f;
            v += a.parts[(part_of(i) * CPL * NT + at) * kWave + lane] * f;
        }
        store_block<T, DP>(a, s, head, (q_tile * NT + nt) * 16 + n, j, mean_of(a, v, l), lane);
    }
}

// What a call launches.
struct Shape {
    int dp, nt;        // padded head length, groups of 16 query rows
    unsigned groups;   // workgroups
};

Shape shape_of(const dq8_cache *c, const dq8_attention &a, int cus)
{
    Shape s;
    s.dp = c->dim <= 64 ? 64 : c->dim <= 128 ? 128 : 256;
    const size_t group = (size_t)(a.heads / c->kv_heads);
    size_t new_tokens = a.starts ? (a.max_new ? a.max_new : a.tokens) : a.tokens / a.batch;
    if (new_tokens > a.tokens) new_tokens = a.tokens;
    const size_t rows = new_tokens * group;
    s.nt = rows <= 16 ? 1 : rows <= 32 || s.dp == 256 ? 2 : 4;
    // as many as are resident; no more than the work can give a tile per wavefront
    const size_t per = 16 * (size_t)s.nt;
    const size_t jobs = (a.tokens * group / per + a.batch) * (size_t)c->kv_heads;
    const size_t tiles = (a.max_pages * (size_t)c->page_size + kTile - 1) / kTile;
    const size_t most = jobs > dq8::kCacheLimit / tiles ? dq8::kCacheLimit : jobs * tiles;
    size_t groups = (size_t)cus * 2;
    const size_t useful = (most + kAttendWaves - 1) / kAttendWaves;
    if (groups > useful) groups = useful;
    s.groups = (unsigned)groups;
    return s;
}

size_t record_bytes(const Shape &s) { return (s.groups * sizeof(int4) + 255) / 256 * 256; }
size_t sums_bytes(const Shape &s) { return (size_t)s.groups * 2 * s.nt * 16 * sizeof(float2); }
size_t parts_bytes(const Shape &s) { return (size_t)s.groups * 2 * (s.dp / 16) * s.nt * kWave * sizeof(v4); }

// What does not look at the arrays of the call.  0 tokens or sequences pass: such a call launches nothing.
int check_shape(const char *who, int kind, const dq8_cache *cache, const dq8_attention *in)
{
    using dq8::failed;
    const int rc = dq8::check_cache(who, kind, cache);
    if (rc) return rc;
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_attention &a = *in;
    if (a.type != DQ8_BFLOAT16 && a.type != DQ8_FLOAT16) return failed(DQ8_ERR_ARG, "%s: type %d is neither bfloat16 nor float16", who, a.type);
    if (a.heads < 1 || a.heads > 65535 || a.heads % cache->kv_heads != 0)
        return failed(DQ8_ERR_ARG, "%s: %d query heads are no multiple of %d cached heads", who, a.heads, cache->kv_heads);
    if (a.batch >= dq8::kCacheLimit || a.tokens >= dq8::kCacheLimit || a.tokens * (size_t)a.heads >= dq8::kCacheLimit)
        return failed(DQ8_ERR_ARG, "%s: too many tokens or sequences", who);
    if (!a.starts && (a.batch ? a.tokens % a.batch : a.tokens) != 0)
        return failed(DQ8_ERR_ARG, "%s: %zu tokens are not as many for each of %zu sequences", who, a.tokens, a.batch);
    if (a.tokens == 0 || a.batch == 0) return DQ8_OK;
    if (a.max_pages < 1 || a.max_pages >= dq8::kCacheLimit / (size_t)cache->page_size || a.batch > ((size_t)1 << 40) / a.max_pages)
        return failed(DQ8_ERR_ARG, "%s: %zu pages per sequence", who, a.max_pages);
    if (a.window < 0) return failed(DQ8_ERR_ARG, "%s: window %d", who, a.window);
    if (!(a.softmax_scale >= -FLT_MAX && a.softmax_scale <= FLT_MAX)) return failed(DQ8_ERR_ARG, "%s: softmax_scale is not finite", who);
    for (size_t s : {a.q_token_stride, a.q_head_stride, a.out_token_stride, a.out_head_stride})
        if (!dq8::sane(s)) return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
    return DQ8_OK;
}

int check_arrays(const char *who, const dq8_cache *cache, const dq8_attention &a, const void *workspace, size_t workspace_bytes)
{
    using dq8::failed;
    using dq8::meet;
    if (!a.q || !a.out || !a.pages || !a.lens) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if ((((uintptr_t)a.q | (uintptr_t)a.out) & 1) != 0 || (((uintptr_t)a.pages | (uintptr_t)a.lens | (uintptr_t)a.starts) & 3) != 0 ||
        ((uintptr_t)workspace & 15) != 0)
        return failed(DQ8_ERR_ARG, "%s: an array does not start at a multiple of its element's size (workspace: 16 bytes)", who);
    const size_t n_out = dq8::extent(a.tokens, a.out_token_stride, a.heads, a.out_head_stride, cache->dim, 2);
    const struct {
        const void *p;
        size_t n;
    } read[] = {{a.q, dq8::extent(a.tokens, a.q_token_stride, a.heads, a.q_head_stride, cache->dim, 2)},
                {cache->codes, dq8::cache_rows(cache) * cache->dim},
                {cache->scales, dq8::cache_rows(cache) * 4},
                {a.pages, a.batch * a.max_pages * 4},
                {a.lens, a.batch * 4},
                {a.starts, a.starts ? (a.batch + 1) * 4 : 0}};
    bool bad = workspace && meet(a.out, n_out, workspace, workspace_bytes);
    for (const auto &r : read) bad = bad || meet(a.out, n_out, r.p, r.n) || (workspace && meet(workspace, workspace_bytes, r.p, r.n));
    if (bad) return failed(DQ8_ERR_ARG, "%s: out or workspace overlaps another array", who);
    return DQ8_OK;
}

template <int DP, int NT>
int launch(int type, const uint32_t *tab, const AttendArgs &k, unsigned groups, hipStream_t stream)
{
#define DQ8_ATTEND(T)                                                                                                      \
    hipLaunchKernelGGL((k_cache_attend<DP, NT, T>), dim3(groups), dim3(kAttendWg), 0, stream, tab, k);                    \
    int rc = dq8::after_launch_of("k_cache_attend", stream);                                                              \
    if (rc || !k.parts) return rc;                                                                                        \
    hipLaunchKernelGGL((k_cache_join<DP, NT, T>), dim3(groups), dim3(kAttendWg), 0, stream, k);                            \
    return dq8::after_launch_of("k_cache_join", stream);
    if (type == DQ8_BFLOAT16) {
        DQ8_ATTEND(__bf16)
    } else {
        DQ8_ATTEND(_Float16)
    }
#undef DQ8_ATTEND
}

}  // namespace

extern "C" {

size_t dq8_cache_attention_workspace_bytes(const dq8_cache *cache, const dq8_attention *a)
{
    static const char who[] = "dq8_cache_attention_workspace_bytes";
    if (check_shape(who, 0, cache, a) || a->tokens == 0 || a->batch == 0) return 0;
    dq8::DeviceTables dev;
    if (dq8::device_tables(0, &dev)) return 0;
    const Shape s = shape_of(cache, *a, dev.cus);
    return record_bytes(s) + sums_bytes(s) + parts_bytes(s);
}

int dq8_cache_attention(int kind, const dq8_cache *cache, const dq8_attention *in, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    static const char who[] = "dq8_cache_attention";
    int rc = check_shape(who, kind, cache, in);
    if (rc) return rc;
    const dq8_attention &a = *in;
    if (a.tokens == 0 || a.batch == 0) return DQ8_OK;
    rc = check_arrays(who, cache, a, workspace, workspace_bytes);
    if (rc) return rc;
    dq8::DeviceTables dev;
    rc = dq8::device_tables(kind, &dev);
    if (rc) return rc;
    const Shape s = shape_of(cache, a, dev.cus);
    AttendArgs k;
    k.q = a.q, k.out = a.out, k.q_ts = a.q_token_stride, k.q_hs = a.q_head_stride, k.o_ts = a.out_token_stride, k.o_hs = a.out_head_stride;
    const size_t half = dq8::cache_rows(cache) / 2;
    k.k_codes = cache->codes, k.v_codes = cache->codes + half * cache->dim;
    k.k_scales = cache->scales, k.v_scales = cache->scales + half;
    k.pages = a.pages, k.lens = a.lens, k.starts = a.starts;
    k.tokens = (uint32_t)a.tokens, k.batch = (uint32_t)a.batch, k.each = a.starts ? 0 : (uint32_t)(a.tokens / a.batch);
    k.heads = (uint32_t)a.heads, k.kv_heads = (uint32_t)cache->kv_heads, k.group = k.heads / k.kv_heads, k.dim = (uint32_t)cache->dim;
    k.n_pages = (uint32_t)cache->pages, k.max_pages = (uint32_t)a.max_pages;
    k.page_shift = (uint32_t)__builtin_ctz((unsigned)cache->page_size);
    k.window = a.window;
    k.entry = kind == DQ8_LINEAR ? 127.0f * 256.0f : 1280.0f * 32.0f;
    k.factor = a.softmax_scale * 1.44269504088896340736f / k.entry;
    k.records = nullptr, k.sums = nullptr, k.parts = nullptr;
    if (workspace && workspace_bytes >= record_bytes(s) + sums_bytes(s) + parts_bytes(s)) {
        char *w = static_cast<char *>(workspace);
        k.records = reinterpret_cast<int4 *>(w);
        k.sums = reinterpret_cast<float2 *>(w + record_bytes(s));
        k.parts = reinterpret_cast<v4 *>(w + record_bytes(s) + sums_bytes(s));
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define DQ8_ATTEND_SHAPE(DP, NT) \
    if (s.dp == DP && s.nt == NT) return launch<DP, NT>(a.type, dev.tab, k, s.groups, stream);
    DQ8_ATTEND_SHAPE(64, 1)
    DQ8_ATTEND_SHAPE(64, 2)
    DQ8_ATTEND_SHAPE(64, 4)
    DQ8_ATTEND_SHAPE(128, 1)
    DQ8_ATTEND_SHAPE(128, 2)
    DQ8_ATTEND_SHAPE(128, 4)
    DQ8_ATTEND_SHAPE(256, 1)
    DQ8_ATTEND_SHAPE(256, 2)
#undef DQ8_ATTEND_SHAPE
    return dq8::failed(DQ8_ERR_ARG, "%s: no kernel", who);
}

}  // extern "C"
