// dq8 kernels: attention over a paged cache of 8-bit keys and values, few query rows per cached head.
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
// row is scaled by a power of two to a largest element of 2^14 .. 2^15.
//
// m need not be the largest score.  What becomes binary16 is a weight times a value scale, and every row has its own m, which brings the
// largest of these products that the row has met to 2^kProductTop; it moves, and the sums with it, when one passes 2^kProductLimit.
// So a product is rounded once to 11 bits, below 2^-22 of the row's largest to a multiple of 2^-32 of that, and what a row does not see,
// or only others see, changes nothing of it.  (One exponent for all value scales that a wavefront had met, seen or not, took as many
// instructions, but outputs of rows that saw only scales 2^-30 times as large vanished.)  Where one number does not do for weights and
// products, there are two: Row.
//
// What bounds it: memory, less well used than by a copy.  64 sequences of up to 4096, 8 heads of 128: 292 MB in 60 us (4.9 TB/s) and 5 us of
// join; two of up to 131072: 391 MB in 75 us (5.2 TB/s) and 7 us; loads alone in the same order reach 6.7.  A wavefront holds two tiles, one
// in flight; LDS, a look-up per code and its 16-bit half, is busy for 57 % of the time, the vector unit 39 %, the matrix units 7 %.
// Short calls (one sequence of 1337: 10 us) wait for the instructions themselves, the table and three loads that need each other.
#pragma once
#include <cfloat>

#include "dq8_device.hpp"

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;          // tokens that a wavefront takes at a time
constexpr int kAttendWaves = 8;    // of a workgroup: they share one table
constexpr int kAttendWg = kAttendWaves * kWave;
constexpr int kQueryTop = 14;      // a query row's largest element is in [2^14, 2^15) in binary16
constexpr float kProductTop = 8.0f, kProductLimit = 15.0f;  // powers of two: of a row's largest weight times value scale, and of any
constexpr float kApart = 60.0f, kWeightLimit = 68.0f;        // of a row's largest weight, from one, and of any
constexpr float kDeep = 56.0f;     // how far products are lifted beyond that (a weight times that is below 2^124)
constexpr int kLeastExp = -90;     // of queries that are still brought to that range

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
    uint32_t *n_records;
    int4 *records;  // of a job: sequence, number in it, the part it begins with, parts (0: it has none, one wavefront did all of it)
    float2 *sums;   // per part and query row: sum_of_part
    float *parts;   // per part: its output [rows][DP], in binary32 as large as the values themselves (their weighted sum may not fit)
    uint32_t rows;  // query rows of a part: as many as a job has at most
    uint32_t in_a_row;  // whether a job's parts lie one after the other, from the number in its record on
    uint32_t by_wave;   // whether the records are those of the job that a wavefront begins and leaves to others, if any, else of all jobs
};

// A sequence's part of the work.
struct Seq {
    bool falls;            // it would end before its beginning
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
        s.falls = end < s.first;
        if (s.falls) end = s.first;
    } else {
        s.falls = false;
        s.first = b * a.each;
        end = s.first + a.each;
    }
    s.n = end - s.first;
    const int32_t most = (int32_t)(a.max_pages << a.page_shift), len = a.lens[b];
    s.len = len < 0 ? 0 : len < most ? len : most;
    int32_t lo = a.window > 0 && s.len > (int32_t)s.n ? s.len - (int32_t)s.n + 1 - a.window : 0;
    if (lo < 0) lo = 0;
    s.lo_tile = (uint32_t)lo / kTile;
    const uint32_t hi = ((uint32_t)s.len + kTile - 1) / kTile;
    s.tiles = hi > s.lo_tile ? hi - s.lo_tile : 1;
    s.q_tiles = (s.n * a.group + rows - 1) / rows;
    return s;
}

// Sequences that the calling lane adds up: a run of them, run * lane on.  tally(sequence) of a run is summed, and where the boundaries
// descend anywhere, all sums are zero: such sequences lie over each other, and the host's bounds of the number of jobs, which
// records and grids are made for, come from tokens that belong to one sequence each.
template <typename F>
__device__ __forceinline__ uint64_t run_sum(const AttendArgs &a, uint32_t rows, uint32_t lane, uint32_t run, F tally)
{
    uint64_t mine = 0;
    bool falls = false;
    for (uint32_t i = 0; i < run; ++i) {
        const uint32_t b = lane * run + i;
        if (b >= a.batch) break;
        const Seq s = sequence(a, b, rows);
        falls |= s.falls;
        mine += tally(s);
    }
    return __builtin_amdgcn_ballot_w64(falls) ? 0 : mine;
}

// Tiles and, in the upper half, jobs of a sequence.
__device__ __forceinline__ uint64_t work_of(const AttendArgs &a, const Seq &s)
{
    const uint32_t jobs = s.q_tiles * a.kv_heads;
    return (uint64_t)jobs << 32 | jobs * s.tiles;
}

__device__ __forceinline__ uint64_t wave_scan(uint64_t v, uint32_t lane)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint64_t o = __shfl_up(v, d);
        if (lane >= (uint32_t)d) v += o;
    }
    return v;
}

__device__ __forceinline__ uint64_t lane_of(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// The tiles of all jobs, in the order of sequences, query groups, heads, tokens, are one line that is cut into parts that differ by
// a tile at most, one per wavefront: whatever the lengths of the sequences, everybody reads as much.  (The host refuses work of
// 2^31 tiles.)  Every wavefront finds its part by itself: a lane adds up a run of sequences, the runs are scanned, and then the
// sequences of the run that holds the beginning.
struct Share {
    uint32_t waves;        // wavefronts that have a part
    uint32_t per, more;    // tiles of a part; the first `more` parts have one more
    uint32_t begin, end;   // this wavefront's
    uint32_t b, place;     // sequence that holds `begin`, and the place in its work
    uint32_t before, jobs; // jobs of the sequences before it, and of all

    // Wavefronts whose parts lie before or reach over place e > 0.
    __device__ uint32_t upto(uint32_t e) const
    {
        const uint32_t longer = more * (per + 1);
        return e <= longer ? (e + per) / (per + 1) : more + (e - longer + per - 1) / per;
    }
};

__device__ __forceinline__ Share share_of(const AttendArgs &a, uint32_t rows, uint32_t w)
{
    const uint32_t lane = threadIdx.x & 63, run = (a.batch + kWave - 1) / kWave;
    const uint64_t mine = run_sum(a, rows, lane, run, [&](const Seq &s) { return work_of(a, s); });
    const uint64_t upto = wave_scan(mine, lane), all = lane_of(upto, 63);
    const uint32_t total = (uint32_t)all;
    Share s;
    s.jobs = (uint32_t)(all >> 32);
    s.waves = gridDim.x * kAttendWaves < total ? gridDim.x * kAttendWaves : total;
    s.per = s.waves ? total / s.waves : 0;
    s.more = total - s.per * s.waves;
    s.b = s.place = s.begin = s.end = s.before = 0;
    if (w >= s.waves) return s;
    s.begin = w * s.per + (w < s.more ? w : s.more);
    s.end = s.begin + s.per + (w < s.more);
    const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64((uint32_t)upto > s.begin));
    uint64_t before = lane_of(upto - mine, owner);
    s.b = (uint32_t)owner * run;
    for (uint32_t i = 0; run > 1 && i < run; i += kWave) {
        const uint32_t b = (uint32_t)owner * run + i + lane;
        const uint64_t work = i + lane < run && b < a.batch ? work_of(a, sequence(a, b, rows)) : 0, sum = wave_scan(work, lane);
        const uint64_t past = __builtin_amdgcn_ballot_w64((uint32_t)(before + sum) > s.begin);
        if (past) {
            const int l = __builtin_ctzll(past);
            s.b = (uint32_t)owner * run + i + (uint32_t)l;
            before += lane_of(sum - work, l);
            break;
        }
        before += lane_of(sum, 63);
    }
    s.b = uniform(s.b);
    s.place = uniform(s.begin - (uint32_t)before);
    s.before = uniform((uint32_t)(before >> 32));
    return s;
}

// Table with entries in binary16, in both halves of a word; see place_lut.
__device__ __forceinline__ void place_half_table(float value, float entry, uint32_t *lds)
{
    const _Float16 h = (_Float16)(value * entry);
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

// Byte J of each of eight words.
template <int J>
__device__ __forceinline__ v8h eighth(const uint32_t *lut, const uint32_t (&w)[8], uint32_t lane4)
{
    return v8h{half_at<J>(lut, w[0], lane4), half_at<J>(lut, w[1], lane4), half_at<J>(lut, w[2], lane4), half_at<J>(lut, w[3], lane4),
               half_at<J>(lut, w[4], lane4), half_at<J>(lut, w[5], lane4), half_at<J>(lut, w[6], lane4), half_at<J>(lut, w[7], lane4)};
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

// A query row's references: weights are exp2(score - shift), their products with value scales are taken as exp2(score - shift + lift) times
// the scale.  The lift is zero, and the shift alone brings the products into range, unless scales lie beyond 2^-kApart .. 2^kApart or
// scores beyond 2^20: a number near these is too coarse for that, so that the shift is then a score itself.
struct Row {
    float shift, lift, sum;  // sum: of the weights

    __device__ __forceinline__ void clear()
    {
        shift = -FLT_MAX;
        lift = sum = 0.0f;
    }

    // high: the largest score of what comes next (-infinity: nothing is seen), large: the log2 of its largest product of
    // exp2(score - high) and scale (-infinity: none).  Returns the factor of the products that were added up.
    __device__ __forceinline__ float raise(float high, float large)
    {
        if (!(high > -__builtin_inff())) return 1.0f;
        // relative to high: the shift as it was, the reference of the products as it was and as it is to be
        const float s0 = shift - high, p0 = s0 - lift, p = fmaxf(p0, large - kProductTop);
        const bool fine = fabsf(high) < 0x1p20f;
        const float near = fine ? fmaxf(fminf(p, kApart), -kApart) : 0.0f;
        if (near <= s0) {  // the shift stays
            const float was = lift;
            lift = fminf(lift, s0 + kProductTop - large);
            return __builtin_amdgcn_exp2f(lift - was);
        }
        shift = high + near;
        const float s = shift - high;  // (rounded as the shift is)
        lift = fine && near == p ? 0.0f : fminf(s - p, kDeep);
        sum *= __builtin_amdgcn_exp2f(s0 - s);
        return __builtin_amdgcn_exp2f(p0 - (s - lift));
    }
};

// A part's sum of weights as a number near one and the log2 of what it is to be multiplied with: references of parts may lie further
// apart than binary32 reaches.  (Those that are too coarse to be moved are scores: the sum is no less than one.)
__device__ __forceinline__ float2 sum_of_part(float shift, float sum)
{
    const int e = fabsf(shift) < 0x1p20f ? __builtin_amdgcn_frexp_expf(sum) : 0;
    return float2{shift + (float)e, __builtin_amdgcn_ldexpf(sum, -e)};
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

template <int N>
__device__ __forceinline__ uint32_t word_of(const typename Bytes<N>::type &v, int i)
{
    if constexpr (N == 4)
        return v;
    else
        return v[i];
}

// A load from a uniform address plus a lane's 32-bit byte offset.  The offset is made to look new each time, or its extension to 64 bits is
// kept for the whole loop and added to the base by the vector unit: two registers and an instruction per load.
// ONCE: nobody reads it again in this call; it need not stay in the caches.
template <typename T, bool ONCE = false>
__device__ __forceinline__ T load_at(const void *uniform_base, uint32_t byte)
{
    asm volatile("" : "+v"(byte));
    const DQ8_GLOBAL T *p = (const DQ8_GLOBAL T *)(uniform_global(static_cast<const char *>(uniform_base)) + byte);
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    return *p;
}

// The page numbers of 64 tiles from `first` on, in the lanes, so that a tile's addresses wait for no load.
struct Pages {
    const int32_t *table;
    uint32_t page[2];  // lane l: of both halves of tile l of the 64

    __device__ void load(const AttendArgs &a, uint32_t first, uint32_t lane)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t token = (first + lane) * kTile + h * 16, index = token >> a.page_shift;
            page[h] = (uint32_t)table[index < a.max_pages ? index : a.max_pages - 1];  // behind the last page: not seen by anybody
        }
    }
};

// Where a wavefront is in its tiles: the one that is loaded next.
struct Walk {
    uint32_t tile, end, i;  // i: its lane in Pages
    __device__ bool done() const { return tile >= end; }
    __device__ void step(const AttendArgs &a, Pages &p, uint32_t lane)
    {
        ++tile;
        if (++i == kWave && tile < end) {
            p.load(a, tile, lane);
            i = 0;
        }
    }
};

// What a wavefront loads of a tile: lane l holds of keys the rows l % 16 of both halves of 16 tokens, 16 bytes of every 64, and
// of values the bytes CPL (l % 16) .. of the eight tokens whose weights it will hold, with the scales of the tokens of its scores.
template <int DP>
struct TileData {
    static constexpr int KL = DP / 64, CPL = DP / 16;
    u4 k[2][KL];
    typename Bytes<CPL>::type v[8];
    v4 ks[2], vs[2];
    bool valid[2];  // whether the half's page is one of the cache
};

template <int DP, bool ONCE>
__device__ __forceinline__ void fetch(const AttendArgs &a, const Pages &p, uint32_t head, uint32_t lane, const Walk &w, TileData<DP> &d)
{
    constexpr uint32_t CPL = DP / 16;
    const uint32_t n = lane & 15, g = lane >> 4;
    const bool behind = w.done();
    const uint32_t tile = behind ? w.tile - 1 : w.tile, i = behind ? w.i - 1 : w.i;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)p.page[h], (int)i), token = tile * kTile + h * 16;
        d.valid[h] = page < a.n_pages;
        const uint64_t row = (((uint64_t)(d.valid[h] ? page : 0) * a.kv_heads + head) << a.page_shift) + (token & ((1u << a.page_shift) - 1));
        const uint8_t *kc = a.k_codes + row * a.dim, *vc = a.v_codes + row * a.dim;
#pragma unroll
        for (int c = 0; c < TileData<DP>::KL; ++c) d.k[h][c] = load_at<u4, ONCE>(kc, behind ? 0 : n * a.dim + (64 * c + 16 * g < a.dim ? 64 * c + 16 * g : 0));
        d.ks[h] = load_at<v4, ONCE>(a.k_scales + row, 16 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r) d.v[4 * h + r] = load_at<typename Bytes<CPL>::type, ONCE>(vc, behind ? 0 : (4 * g + r) * a.dim + (n * CPL < a.dim ? n * CPL : 0));
        d.vs[h] = load_at<v4, ONCE>(a.v_scales + row, 16 * g);
    }
}

// One job's tiles t0 .. t1 - 1: query rows q_tile * 16 NT .. of a sequence against a cached head.  part: where the sums go if the job is
// not finished here (-1: it is, and the output is stored).
//
template <int DP, int NT>
constexpr bool kQueryInLds = DP * NT > 128;

// With one group of 16 rows there is one job per sequence and cached head, and a tile is read once: past the caches (64 sequences of
// 4096 at most: 73 us through them, 66 past; two of 131072: 87 and 84).  With more rows two jobs may read it (180 MB, 20 rows of each
// of 16: 46 us and 50), and rows of 64 bytes are half a line that two loads share (75 MB: 26.8 and 28.3).
template <int DP, int NT>
constexpr bool kOnce = DP == 128 && NT == 1;

template <int DP, int NT, typename T>
__device__ __forceinline__ void attend(const AttendArgs &a, const Seq &s, uint32_t b, uint32_t q_tile, uint32_t head, uint32_t t0, uint32_t t1, int32_t part,
                       const uint32_t *lut, v8h *query)
{
    constexpr int CPL = DP / 16, KS = DP / 32;
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, lane4 = lane * 4;
    const uint32_t tile = s.lo_tile + t0, end = s.lo_tile + t1;
    Pages pages;
    pages.table = a.pages + (size_t)b * a.max_pages;
    pages.load(a, tile, lane);

    // The query rows as operands of the products, in registers or, where these are needed for the sums, in LDS: the lane's eight elements of
    // step k of group nt.
    v8h q[kQueryInLds<DP, NT> ? 1 : NT][KS];
    float scale[NT];
    Row ref[NT];
    bool far = false;  // whether some row has a lift
    int32_t pos[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const uint32_t row = (q_tile * NT + nt) * 16 + n;
        const bool in = row < s.n * a.group;
        const uint32_t token = in ? row / a.group : 0, qh = in ? row - token * a.group : 0;
        const T *src = static_cast<const T *>(a.q) + (s.first + token) * a.q_ts + (head * a.group + qh) * a.q_hs;
        typedef T V __attribute__((ext_vector_type(8)));
        typedef V VA __attribute__((aligned(sizeof(T))));
        V x[KS];
        float most = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const uint32_t d = 16 * (g + 4 * (k / 2)) + 8 * (k % 2);
            x[k] = V{};
            if (in && d < a.dim) x[k] = *reinterpret_cast<const VA *>(src + d);
        }
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)x[k][e]));
        const int e = exponent(max_over_groups(most));
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            v8h h;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (_Float16)__builtin_amdgcn_ldexpf((float)x[k][i], kQueryTop - e);
            if constexpr (kQueryInLds<DP, NT>)
                query[(nt * KS + k) * kWave + lane] = h;
            else
                q[nt][k] = h;
        }
        pos[nt] = in ? s.len - (int32_t)s.n + (int32_t)token : -1;
        scale[nt] = __builtin_amdgcn_ldexpf(a.factor, e - kQueryTop);
        ref[nt].clear();
    }
    v4 acc[NT][CPL];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < CPL; ++j) acc[nt][j] = v4{0, 0, 0, 0};
    const int32_t p_first = s.len - (int32_t)s.n;  // position of the sequence's first query, the least of any row here

    auto work = [&](uint32_t tile, const TileData<DP> &d) {
        v4 st[NT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) st[nt][h] = v4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if (k % 2 == 0) __builtin_amdgcn_sched_barrier(0);
                const v8h f = eight(lut, d.k[h][k / 2][2 * (k % 2)], d.k[h][k / 2][2 * (k % 2) + 1], lane4);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) st[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, kQueryInLds<DP, NT> ? query[(nt * KS + k) * kWave + lane] : q[kQueryInLds<DP, NT> ? 0 : nt][k], st[nt][h], 0, 0, 0);
            }
        }
        const int32_t t = (int32_t)(tile * kTile);
        // whether some row does not see some token of the tile (a window's lower end: rows up to the last position)
        const bool masked = t + kTile - 1 > p_first || (a.window > 0 && t <= s.len - 1 - a.window) || !d.valid[0] || !d.valid[1];
        v8h p[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float x[2][4], c[2][4], y[2][4], w[2][4], z[2][4];  // scores x c, value scales, weights, products
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[h][r] = st[nt][h][r];
                    c[h][r] = d.ks[h][r] * scale[nt];
                    y[h][r] = d.vs[h][r];
                }
            if (masked) {  // hidden tokens: weight zero, whatever their scales are
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int32_t token = t + 16 * h + 4 * (int32_t)g + r;
                        if (!(token <= pos[nt] && (a.window <= 0 || token > pos[nt] - a.window) && d.valid[h])) {
                            x[h][r] = -__builtin_inff();
                            c[h][r] = 1.0f;
                            y[h][r] = 0.0f;
                        }
                    }
            }
            Row &row = ref[nt];
            float added;
            auto weigh = [&]() {  // whether one leaves its range
                float large = 0.0f;
                added = 0.0f;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        w[h][r] = __builtin_amdgcn_exp2f(x[h][r] * c[h][r] - row.shift);
                        z[h][r] = w[h][r] * y[h][r];
                        added += w[h][r];
                    }
                if (far) {
                    const float rest = __builtin_amdgcn_exp2f(row.lift);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r) z[h][r] = w[h][r] * rest * y[h][r];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) large = fmaxf(large, fabsf(z[h][r]));
                return added > 0x1p68f || large > 0x1p15f;
            };
            if (__builtin_amdgcn_ballot_w64(weigh()) != 0) {
                float high = -__builtin_inff(), large = -__builtin_inff();
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) high = fmaxf(high, x[h][r] * c[h][r]);
                high = max_over_groups(high);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) large = fmaxf(large, x[h][r] * c[h][r] - high + __builtin_amdgcn_logf(fabsf(y[h][r])));
                const float less = row.raise(high, max_over_groups(large));
#pragma unroll
                for (int j = 0; j < CPL; ++j) acc[nt][j] *= less;
                far = far || __builtin_amdgcn_ballot_w64(row.lift != 0.0f) != 0;
                weigh();
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r) p[nt][4 * h + r] = (_Float16)z[h][r];
            row.sum += added;
        }
#pragma unroll
        for (int j4 = 0; j4 < CPL / 4; ++j4) {
            uint32_t word[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) word[r] = word_of<CPL>(d.v[r], j4);
            __builtin_amdgcn_sched_barrier(0);
            const v8h f0 = eighth<0>(lut, word, lane4), f1 = eighth<1>(lut, word, lane4);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                acc[nt][4 * j4] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f0, p[nt], acc[nt][4 * j4], 0, 0, 0);
                acc[nt][4 * j4 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f1, p[nt], acc[nt][4 * j4 + 1], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            const v8h f2 = eighth<2>(lut, word, lane4), f3 = eighth<3>(lut, word, lane4);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                acc[nt][4 * j4 + 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f2, p[nt], acc[nt][4 * j4 + 2], 0, 0, 0);
                acc[nt][4 * j4 + 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f3, p[nt], acc[nt][4 * j4 + 3], 0, 0, 0);
            }
        }
    };

    // The next tile's loads are in flight while a wavefront works on the present one.  They are issued without a condition (a
    // branch around them makes the waits for older loads wait for all); behind the last tile all lanes load its first row.
    Walk walk{tile, end, 0};
    TileData<DP> x, y;
    fetch<DP, kOnce<DP, NT>>(a, pages, head, lane, walk, x);
    for (;;) {
        const uint32_t one = walk.tile;
        walk.step(a, pages, lane);
        fetch<DP, kOnce<DP, NT>>(a, pages, head, lane, walk, y);
        work(one, x);
        if (walk.done()) break;
        const uint32_t two = walk.tile;
        walk.step(a, pages, lane);
        fetch<DP, kOnce<DP, NT>>(a, pages, head, lane, walk, x);
        work(two, y);
        if (walk.done()) break;
    }

    // A lane has elements 16 x (4 g + i) / 16 .. of its row: CPL neighbours for each i.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const float sum = sum_over_groups(ref[nt].sum);
        const uint32_t local = nt * 16 + n, row = q_tile * NT * 16 + local;
        const float r = sum == 0.0f ? 0.0f : 1.0f / (sum * a.entry), down = __builtin_amdgcn_exp2f(-ref[nt].lift);
        if (row >= s.n * a.group) continue;
        if (part >= 0) {
            const size_t at = (size_t)part * a.rows + local;
            if (g == 0) a.sums[at] = sum_of_part(ref[nt].shift, sum);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CPL; j += 4)
                    *reinterpret_cast<v4 *>(a.parts + at * DP + CPL * (4 * g + i) + j) =
                        v4{acc[nt][j][i], acc[nt][j + 1][i], acc[nt][j + 2][i], acc[nt][j + 3][i]} * r * down;
        } else {
            const uint32_t token = row / a.group;
            T *to = static_cast<T *>(a.out) + (s.first + token) * a.o_ts + (head * a.group + row - token * a.group) * a.o_hs;
            typedef T V __attribute__((ext_vector_type(4)));
            typedef V VA __attribute__((aligned(sizeof(T))));
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < CPL; j += 4) {
                    const uint32_t d = CPL * (4 * g + i) + j;
                    const v4 m = v4{acc[nt][j][i], acc[nt][j + 1][i], acc[nt][j + 2][i], acc[nt][j + 3][i]} * r * down;
                    if (d < a.dim) *reinterpret_cast<VA *>(to + d) = V{(T)m.x, (T)m.y, (T)m.z, (T)m.w};
                }
        }
    }
}

template <int DP, int NT, typename T>
__global__ __launch_bounds__(kAttendWg, 2) void k_cache_attend(const uint32_t *__restrict__ tab, AttendArgs a)
{
    __shared__ __align__(256) uint32_t lds[256 * kLutCopies];
    __shared__ v8h queries[kQueryInLds<DP, NT> ? kAttendWaves * NT * (DP / 32) * kWave : 1];
    const uint32_t wave = wave_in_wg(), w = blockIdx.x * kAttendWaves + wave;
    v8h *const query = queries + (kQueryInLds<DP, NT> ? wave * NT * (DP / 32) * kWave : 0);
    place_half_table(request_lut(tab), a.entry, lds);
    const Share share = share_of(a, 16 * NT, w);
    __syncthreads();
    const bool first = (threadIdx.x & 63) == 0;
    if (a.parts && w == 0 && first) *a.n_records = a.by_wave ? gridDim.x * kAttendWaves : share.jobs;
    bool recorded = false;
    uint32_t b = share.b, place = share.place, at = share.begin, before = share.before;
    while (at < share.end && b < a.batch) {
        const Seq s = sequence(a, b, 16 * NT);
        const uint64_t work = work_of(a, s);
        if (place >= (uint32_t)work) {  // the next sequence
            before += (uint32_t)(work >> 32);
            ++b;
            place = 0;
            continue;
        }
        const uint32_t job = uniform(place / s.tiles), t0 = uniform(place - job * s.tiles);
        uint32_t t1 = s.tiles;
        int32_t part = -1;
        if (a.parts) {
            const uint32_t left = share.end - at;
            if (left < t1 - t0) t1 = t0 + left;
            if (t0 > 0 || t1 < s.tiles) part = 2 * (int32_t)w + (t0 == 0);
            if (t0 == 0 && (!a.by_wave || t1 < s.tiles)) {  // where it does not end here: the wavefronts whose parts reach its end
                recorded = true;
                if (first) a.records[a.by_wave ? w : before + job] = int4{(int)b, (int)job, (int)w, t1 < s.tiles ? (int)(share.upto(at + s.tiles) - w) : 0};
            }
        }
        // without a workspace, whole jobs: those that begin in this part
        if (a.parts || t0 == 0) attend<DP, NT, T>(a, s, b, job / a.kv_heads, job % a.kv_heads, t0, t1, part, lds, query);
        place += t1 - t0;
        at += t1 - t0;
    }
    if (a.parts && a.by_wave && !recorded && first) a.records[w] = int4{0, 0, 0, 0};
}

// The jobs that several wavefronts worked on, one per workgroup in x, SLICE of its rows in y.  A part lies far away (another die's
// cache wrote it), so that what counts is how many loads are in flight and how few wait for each other: a thread has four elements of
// a row, groups of threads take every so manieth part, the first of them before anything is known of the sums, and the groups' sums are
// added in LDS.
constexpr int kJoinParts = 256, kJoinAhead = 4;

template <int DP, uint32_t ROWS, int SLICE, int WG, typename T>
__global__ __launch_bounds__(WG) void k_cache_join(AttendArgs a)
{
    constexpr uint32_t QUADS = DP / 4, CELLS = SLICE * QUADS, GROUPS = WG / CELLS;
    static_assert(WG % CELLS == 0 && WG >= SLICE * kWave, "whole groups, a wavefront per row");
    __shared__ float factor[kJoinParts * SLICE];  // of a part and row: its share of the sum of weights
    __shared__ float largest[SLICE], weights[SLICE];
    __shared__ v4 sums[WG];
    const uint32_t records = *a.n_records;
    const int4 record = a.records[blockIdx.x];  // (there is room for as many as the grid has)
    if (blockIdx.x >= records) return;
    const uint32_t w = (uint32_t)record.z, parts = (uint32_t)record.w;
    if (parts == 0) return;
    auto part_of = [&](uint32_t i) { return a.in_a_row ? (size_t)w + i : 2 * ((size_t)w + i) + (i == 0); };
    const Seq s = sequence(a, (uint32_t)record.x, ROWS);
    const uint32_t head = (uint32_t)record.y % a.kv_heads, q_tile = (uint32_t)record.y / a.kv_heads;
    const uint32_t left = s.n * a.group - q_tile * ROWS, rows = left < ROWS ? left : ROWS;  // of this job
    const uint32_t first = blockIdx.y * SLICE;
    if (first >= rows) return;
    const uint32_t group = threadIdx.x / CELLS, cell = threadIdx.x % CELLS, row = cell / QUADS, d = 4 * (cell % QUADS);
    const bool mine = first + row < rows;
    const float *p = a.parts + (size_t)(mine ? first + row : first) * DP + d;
    v4 ahead[kJoinAhead];
#pragma unroll
    for (uint32_t k = 0; k < kJoinAhead; ++k) {
        const uint32_t i = group + k * GROUPS;
        ahead[k] = *reinterpret_cast<const v4 *>(p + part_of(i < parts ? i : 0) * a.rows * DP);
    }
    if (threadIdx.x < SLICE * kWave) {  // a wavefront looks at a row's parts
        const uint32_t row = first + (threadIdx.x >> 6);
        float top = -FLT_MAX, l = 0.0f;
        if (row < rows)
            for (uint32_t i = threadIdx.x & 63; i < parts; i += kWave) {
                const float2 o = a.sums[part_of(i) * a.rows + row];
                const float now = fmaxf(top, o.x);
                l = l * __builtin_amdgcn_exp2f(top - now) + o.y * __builtin_amdgcn_exp2f(o.x - now);
                top = now;
            }
        float all = top;
#pragma unroll
        for (int m = 1; m < kWave; m *= 2) all = fmaxf(all, __shfl_xor(all, m));
        l *= __builtin_amdgcn_exp2f(top - all);
#pragma unroll
        for (int m = 1; m < kWave; m *= 2) l += __shfl_xor(l, m);
        if ((threadIdx.x & 63) == 0) {
            largest[threadIdx.x >> 6] = all;
            weights[threadIdx.x >> 6] = l;
        }
    }
    v4 v = {0, 0, 0, 0};
    for (uint32_t i0 = 0; i0 < parts; i0 += kJoinParts) {
        const uint32_t some = parts - i0 < kJoinParts ? parts - i0 : kJoinParts;
        __syncthreads();
        for (uint32_t x = threadIdx.x; x < some * SLICE; x += WG)
            if (first + x % SLICE < rows) {
                const float2 o = a.sums[part_of(i0 + x / SLICE) * a.rows + first + x % SLICE];
                const float all = weights[x % SLICE];
                factor[x] = all == 0.0f ? 0.0f : o.y * __builtin_amdgcn_exp2f(o.x - largest[x % SLICE]) / all;
            }
        __syncthreads();
        if (mine) {
            uint32_t i = group;
            if (i0 == 0) {
#pragma unroll
                for (uint32_t k = 0; k < kJoinAhead; ++k, i += GROUPS)
                    if (i < some) v += ahead[k] * factor[i * SLICE + row];
            }
#pragma unroll 4
            for (; i < some; i += GROUPS) v += *reinterpret_cast<const v4 *>(p + part_of(i0 + i) * a.rows * DP) * factor[i * SLICE + row];
        }
    }
    if (GROUPS > 1) {
        sums[threadIdx.x] = v;
        __syncthreads();
    }
    if (group == 0 && mine && d < a.dim) {
#pragma unroll 8
        for (uint32_t o = 1; o < GROUPS; ++o) v += sums[o * CELLS + cell];
        const uint32_t at = q_tile * ROWS + first + row, token = at / a.group;
        typedef T V __attribute__((ext_vector_type(4)));
        typedef V VA __attribute__((aligned(sizeof(T))));
        T *to = static_cast<T *>(a.out) + (s.first + token) * a.o_ts + (head * a.group + at - token * a.group) * a.o_hs;
        *reinterpret_cast<VA *>(to + d) = V{(T)v.x, (T)v.y, (T)v.z, (T)v.w};
    }
}

}  // namespace
