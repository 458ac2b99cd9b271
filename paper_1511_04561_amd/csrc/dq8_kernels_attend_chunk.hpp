// dq8 kernels: attention over a paged cache of 8-bit keys and values, many query rows per cached head (prompts and their chunks).
//
// The mathematics is that of dq8_kernels_attend.hpp; here the matrix instructions and the vector unit bound the time, not the
// memory.  A workgroup of eight wavefronts has 256 query rows of one cached head, 32 per wavefront.  A tile of tokens is
// looked up once for all of them: every wavefront turns its eighth of the tile's codes into binary16 and leaves it in LDS in the order
// in which the lanes of a matrix instruction take it (16 bytes per lane, so that neither side has bank conflicts), one tile ahead of
// the one that is multiplied.  Products are 32x32x16: S^T = K Q^T with a query per column, lane % 32, sixteen tokens in a lane's
// registers; these are P^T as operand of out^T = V^T P^T, where the order of a lane's eight tokens is that of its registers.
// The scales of a tile's tokens go through LDS as factors of scores and weights, brought into range by one wavefront.
#pragma once
#include "dq8_kernels_attend.hpp"

namespace {

typedef float v16 __attribute__((ext_vector_type(16)));

constexpr int kChunkWaves = 8, kChunkWg = kChunkWaves * kWave;

// The job of number idx, counted over sequences: sequence b and the number in it.  Every wavefront by itself; idx < their number.
struct Place {
    uint32_t b, job, jobs;  // jobs: how many there are
};

__device__ __forceinline__ Place place_of(const AttendArgs &a, uint32_t rows, uint32_t idx)
{
    const uint32_t lane = threadIdx.x & 63, run = (a.batch + kWave - 1) / kWave;
    uint64_t mine = 0;
    for (uint32_t i = 0; i < run; ++i) {
        const uint32_t b = lane * run + i;
        if (b < a.batch) mine += sequence(a, b, rows).q_tiles * a.kv_heads;
    }
    const uint64_t upto = wave_scan(mine, lane);
    Place p;
    p.jobs = (uint32_t)lane_of(upto, 63);
    p.b = p.job = 0;
    if (idx >= p.jobs) return p;
    const int owner = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > idx));
    uint64_t before = lane_of(upto - mine, owner);
    p.b = (uint32_t)owner * run;
    for (uint32_t i = 0; run > 1 && i < run; i += kWave) {
        const uint32_t b = (uint32_t)owner * run + i + lane;
        const uint64_t work = i + lane < run && b < a.batch ? sequence(a, b, rows).q_tiles * a.kv_heads : 0, sum = wave_scan(work, lane);
        const uint64_t past = __builtin_amdgcn_ballot_w64(before + sum > idx);
        if (past) {
            const int l = __builtin_ctzll(past);
            p.b = (uint32_t)owner * run + i + (uint32_t)l;
            before += lane_of(sum - work, l);
            break;
        }
        before += lane_of(sum, 63);
    }
    p.b = uniform(p.b);
    p.job = uniform(idx - (uint32_t)before);
    return p;
}

// DP: padded head length; TH: halves of 32 tokens of a tile.
template <int DP, int TH>
struct ChunkShape {
    static constexpr int kRows = 32 * kChunkWaves, kTokens = TH * 32;
    static constexpr int KS = DP / 16;             // steps of 16 elements of a score
    static constexpr int JT = DP / 32;             // groups of 32 elements of an output row
    static constexpr int US = TH * 2;              // steps of 16 tokens of an output
    static constexpr int kKeyFrags = TH * KS, kValueFrags = US * JT;
    // Two operands are prepared from one load of 16 bytes per lane (keys) or eight words (values).  A wavefront has one pair of each or,
    // where there are only four of them, one of either.
    static constexpr int kPairs = kKeyFrags / 2;
    static constexpr bool kApart = kPairs < kChunkWaves;
    static constexpr int kBuffer = (kKeyFrags + kValueFrags) * 1024;  // bytes of a tile
    static_assert(kKeyFrags == kValueFrags && (kApart ? 2 * kPairs == kChunkWaves : kPairs == kChunkWaves), "as much work for every wavefront");
    static_assert(kTokens <= kWave, "a lane for every token's scales");
};

// One tile's scales in LDS: factors of scores and of weights, which tokens are there, and the exponent that the latter were brought to.
template <int TOKENS>
struct ChunkScales {
    float key[TOKENS], value[TOKENS];
    uint64_t there;
    int32_t exponent, pad;
};

template <int DP, int TH, typename T>
__global__ __launch_bounds__(kChunkWg, 2) void k_cache_attend_chunk(const uint32_t *__restrict__ tab, AttendArgs a, uint32_t splits)
{
    typedef ChunkShape<DP, TH> S;
    constexpr int KS = S::KS, JT = S::JT, US = S::US, TOKENS = S::kTokens;
    __shared__ __align__(256) uint32_t lut[256 * kLutCopies];
    __shared__ __align__(16) uint8_t tiles[2 * S::kBuffer];
    __shared__ __align__(16) ChunkScales<TOKENS> scales[2];
    const uint32_t lane = threadIdx.x & 63, wave = wave_in_wg(), n = lane & 31, hh = lane >> 5, lane4 = lane * 4;
    // the last query rows of a sequence see most: they begin first
    const Place place = place_of(a, S::kRows, blockIdx.x / splits);
    if (a.parts && blockIdx.x == 0 && threadIdx.x == 0) *a.jobs = place.jobs;
    if (blockIdx.x / splits >= place.jobs) return;
    {
        const _Float16 h = (_Float16)(u2f(tab[kCbOff + (threadIdx.x & 255)]) * a.entry);
        uint16_t u;
        __builtin_memcpy(&u, &h, 2);
        place_lut<kChunkWg>(u2f(u | ((uint32_t)u << 16)), reinterpret_cast<float *>(lut));
    }
    const Seq s = sequence(a, place.b, S::kRows);
    const uint32_t q_tile = s.q_tiles - 1 - place.job / a.kv_heads, head = place.job % a.kv_heads, split = blockIdx.x % splits;
    const uint32_t total_rows = s.n * a.group, row0 = q_tile * S::kRows;
    const int32_t p0 = s.len - (int32_t)s.n;  // position of the sequence's first query
    // tokens that some row of the workgroup sees: from .. upto - 1
    const uint32_t last_row = row0 + S::kRows < total_rows ? row0 + S::kRows - 1 : total_rows - 1;
    const int32_t upto = p0 + (int32_t)(last_row / a.group) + 1, lowest = a.window > 0 ? p0 + (int32_t)(row0 / a.group) - a.window + 1 : 0;
    const uint32_t first_tile = lowest > 0 ? (uint32_t)lowest / TOKENS : 0, end_tile = upto > 0 ? ((uint32_t)upto + TOKENS - 1) / TOKENS : 0;
    const uint32_t count = end_tile > first_tile ? end_tile - first_tile : 0;
    const uint32_t t_begin = first_tile + (uint32_t)((uint64_t)count * split / splits), t_end = first_tile + (uint32_t)((uint64_t)count * (split + 1) / splits);

    // the wavefront's 32 query rows as operands, scaled by a power of two each: eight elements of step k, see fetch for their order
    v8h q[KS];
    const uint32_t w_first = row0 + wave * 32, row = w_first + n;
    const bool in = row < total_rows;
    const uint32_t row_token = in ? row / a.group : 0, row_head = head * a.group + (in ? row - row_token * a.group : 0);
    const int32_t pos = in ? p0 + (int32_t)row_token : -1;
    float up, top = kNothing, sum = 0.0f;  // up: the power of two that a row's scores are multiplied by; top: the reference of its weights
    {
        const T *src = static_cast<const T *>(a.q) + (s.first + row_token) * a.q_ts + row_head * a.q_hs;
        typedef T V __attribute__((ext_vector_type(8)));
        typedef V VA __attribute__((aligned(sizeof(T))));
        V x[KS];
        float most = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const uint32_t d = 32 * (k / 2) + 16 * hh + 8 * (k % 2);
            x[k] = V{};
            if (in && d < a.dim) x[k] = *reinterpret_cast<const VA *>(src + d);
        }
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf((float)x[k][e]));
        const int e = exponent(fmaxf(most, __shfl_xor(most, 32)));
        const float sign = a.factor < 0.0f ? -1.0f : 1.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[k][i] = (_Float16)(__builtin_amdgcn_ldexpf((float)x[k][i], kQueryTop - e) * sign);
        up = __builtin_amdgcn_ldexpf(1.0f, e - kQueryTop);
    }
    v16 acc[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] = 0.0f;
    int vexp = kLeastExp;
    // positions of the wavefront's first and last row (-1: it has none)
    const int32_t p_first = w_first < total_rows ? p0 + (int32_t)(w_first / a.group) : -1;
    const int32_t p_last = w_first < total_rows ? p0 + (int32_t)((w_first + 31 < total_rows ? w_first + 31 : total_rows - 1) / a.group) : -1;

    // ---- the tile's way into LDS.  Keys: a lane takes 16 bytes of one of 32 tokens, which are its eight elements of two steps.  Values: a
    // lane takes a word of each of the eight tokens of its half of step u, two bytes of which are elements of its two groups.
    const int32_t *table = a.pages + (size_t)place.b * a.max_pages;
    auto page_at = [&](uint32_t token) {
        const uint32_t index = token >> a.page_shift;
        return (uint32_t)table[index < a.max_pages ? index : a.max_pages - 1];
    };
    auto row_of = [&](uint32_t page, uint32_t token) {
        return (((uint64_t)(page < a.n_pages ? page : 0) * a.kv_heads + head) << a.page_shift) + (token & ((1u << a.page_shift) - 1));
    };
    const bool has_keys = !S::kApart || wave < (uint32_t)S::kPairs, has_values = !S::kApart || !has_keys;
    const uint32_t kp = wave % S::kPairs, k_half = kp / JT, k_pair = kp % JT;       // this wavefront's pair of key operands
    const uint32_t vp = wave % S::kPairs, u = vp % US, two = vp / US;               // and of value operands
    const uint32_t v_select = 0x0C0C0400u + ((two & 1) << 9);                       // its first byte of a word
    u4 kc = {0, 0, 0, 0};
    uint32_t vc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    uint32_t k_page = 0, v_page = 0, s_page = 0;  // of the tile that is loaded next
    float ks = 0.0f, vs = 0.0f;
    bool s_there = false;
    int32_t staged = kLeastExp;  // (wavefront 0) exponent of the largest value scale so far
    auto fetch_pages = [&](uint32_t tile) {
        if (has_keys) k_page = page_at(tile * TOKENS + k_half * 32 + n);
        if (has_values) v_page = page_at(tile * TOKENS + u * 16);
        if (wave == 0) s_page = page_at(tile * TOKENS + lane % TOKENS);
    };
    auto fetch = [&](uint32_t tile) {
        if (has_keys) {
            const uint32_t d = 32 * k_pair + 16 * hh;
            kc = *reinterpret_cast<const u4 *>(a.k_codes + row_of(k_page, tile * TOKENS + k_half * 32 + n) * a.dim + (d < a.dim ? d : 0));
        }
        if (has_values) {
            const uint32_t d = JT * n + 4 * (two / 2);
            const uint8_t *v = a.v_codes + row_of(v_page, tile * TOKENS + u * 16 + 4 * hh) * a.dim + (d < a.dim ? d : 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint8_t *at = v + (i % 4 + 8 * (i / 4)) * a.dim;
                vc[i] = JT == 2 ? *reinterpret_cast<const uint16_t *>(at) : *reinterpret_cast<const uint32_t *>(at);
            }
        }
        if (wave == 0) {
            const uint64_t at = row_of(s_page, tile * TOKENS + lane % TOKENS);
            ks = a.k_scales[at];
            vs = a.v_scales[at];
            s_there = (int32_t)(tile * TOKENS + lane % TOKENS) < s.len && s_page < a.n_pages;
        }
    };
    const float factor = fabsf(a.factor);
    auto eighth_of = [&](uint32_t select) {
        v8h f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = *reinterpret_cast<const _Float16 *>(reinterpret_cast<const char *>(lut) + __builtin_amdgcn_perm(vc[i], lane4, select));
        return f;
    };
    auto put = [&](uint32_t buffer) {
        v8h *const to = reinterpret_cast<v8h *>(tiles + buffer * S::kBuffer) + lane;
        if (has_keys) {
            v8h *const f = to + (k_half * KS + 2 * k_pair) * kWave;
            f[0] = eight(lut, kc.x, kc.y, lane4);
            f[kWave] = eight(lut, kc.z, kc.w, lane4);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (has_values) {
            v8h *const f = to + (S::kKeyFrags + u * JT + 2 * two) * kWave;
            f[0] = eighth_of(v_select);
            f[kWave] = eighth_of(v_select + 0x100u);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (wave == 0) {
            const float y = s_there ? vs : 0.0f;
            float most = y;
#pragma unroll
            for (int m = 1; m < TOKENS; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
            const int e = (int)uniform((uint32_t)exponent(fmaxf(most, 0.0f)));
            staged = e > staged ? e : staged;
            ChunkScales<TOKENS> &sc = scales[buffer];
            if (lane < TOKENS) {
                sc.key[lane] = ks * factor;
                sc.value[lane] = y * __builtin_amdgcn_ldexpf(1.0f, kWeightTop - staged);
            }
            const uint64_t all = __builtin_amdgcn_ballot_w64(s_there);
            if (lane == 0) {
                sc.there = all;
                sc.exponent = staged;
            }
        }
    };

    auto multiply = [&](uint32_t tile, uint32_t buffer) {
        const v8h *const keys = reinterpret_cast<const v8h *>(tiles + buffer * S::kBuffer) + lane, *const values = keys + S::kKeyFrags * kWave;
        const ChunkScales<TOKENS> &sc = scales[buffer];
        const int32_t t = (int32_t)(tile * TOKENS);
        v16 st[TH];
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) st[h][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int h = 0; h < TH; ++h) st[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(keys[(h * KS + k) * kWave], q[k], st[h], 0, 0, 0);
        const int e = sc.exponent;
        if (e > vexp) {
            const float less = __builtin_amdgcn_ldexpf(1.0f, vexp - e);
#pragma unroll
            for (int j = 0; j < JT; ++j) acc[j] *= less;
            vexp = e;
        }
        // scores times their keys' scales; those that a row does not see become -infinity
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const v4 f = *reinterpret_cast<const v4 *>(sc.key + 32 * h + 8 * i4 + 4 * hh);
#pragma unroll
                for (int i = 0; i < 4; ++i) st[h][4 * i4 + i] *= f[i];
            }
        const uint64_t there = sc.there;
        const bool masked = t + TOKENS - 1 > p_first || (a.window > 0 && t <= p_last - a.window) || there != ~0ull;  // (32 tokens: both halves of the wavefront say the same)
        if (masked) {
#pragma unroll
            for (int h = 0; h < TH; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int32_t at = 32 * h + 8 * (i / 4) + 4 * (int32_t)hh + i % 4, token = t + at;
                    const bool seen = (token <= pos) & ((a.window <= 0) | (token > pos - a.window)) & (int)(there >> at & 1);
                    st[h][i] = seen ? st[h][i] : -__builtin_inff();
                }
        }
        float high = kNothing;
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) high = fmaxf(high, st[h][i]);
        // `top` need not be the largest score, only near it: weights up to 2^kSlack fit
        if (__builtin_amdgcn_ballot_w64(high * up > top + kSlack) != 0) {
            const float now = fmaxf(top, fmaxf(high, __shfl_xor(high, 32)) * up), less = __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= less;
#pragma unroll
            for (int j = 0; j < JT; ++j) acc[j] *= less;
        }
        v8h p[US];
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const v4 f = *reinterpret_cast<const v4 *>(sc.value + 32 * h + 8 * i4 + 4 * hh);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // (up is a power of two: the product is exact, and what is subtracted from it is such a product)
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(st[h][4 * i4 + i], up, -top));
                    sum += w;
                    p[2 * h + i4 / 2][4 * (i4 % 2) + i] = (_Float16)(w * f[i]);
                }
            }
        if (masked)  // a hidden token's scale may be anything
#pragma unroll
            for (int h = 0; h < TH; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (st[h][i] == -__builtin_inff()) p[2 * h + i / 8][i % 8] = (_Float16)0.0f;
#pragma unroll
        for (int x = 0; x < US; ++x)
#pragma unroll
            for (int j = 0; j < JT; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values[(x * JT + j) * kWave], p[x], acc[j], 0, 0, 0);
    };

    __syncthreads();  // the table
    if (t_begin < t_end) {
        // behind the last tile the last is loaded again
        const uint32_t last = t_end - 1;
        auto limited = [&](uint32_t tile) { return tile < t_end ? tile : last; };
        fetch_pages(t_begin);
        fetch(t_begin);
        fetch_pages(limited(t_begin + 1));
        put(0);
        fetch(limited(t_begin + 1));
        fetch_pages(limited(t_begin + 2));
        __syncthreads();
        for (uint32_t tile = t_begin, buffer = 0;; ++tile, buffer ^= 1) {
            const bool seen = (int32_t)(tile * TOKENS) <= p_last && (a.window <= 0 || (int32_t)(tile * TOKENS + TOKENS) > p_first - a.window + 1);
            if (tile < last) {
                // the next tile's codes are here: into the other buffer; then the loads of the tile after it and of the page
                // numbers of the one after that
                put(buffer ^ 1);
                fetch(limited(tile + 2));
                fetch_pages(limited(tile + 3));
            }
            if (seen) multiply(tile, buffer);
            if (tile == last) break;
            __syncthreads();
        }
    }

    const size_t part = (size_t)(blockIdx.x / splits) * splits + split;
    if (a.parts && splits > 1 && split == 0 && threadIdx.x == 0)
        a.records[blockIdx.x / splits] = int4{(int)place.b, (int)(q_tile * a.kv_heads + head), (int)part, (int)splits};
    const float size = __builtin_amdgcn_ldexpf(1.0f, vexp - kWeightTop);
    sum += __shfl_xor(sum, 32);
    if (!in) return;
    constexpr int W = JT < 4 ? JT : 4;
    if (splits > 1) {
        const size_t at = part * a.rows + wave * 32 + n;
        if (hh == 0) a.sums[at] = float2{top, sum};
        typedef float V __attribute__((ext_vector_type(W)));
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int j = 0; j < JT; j += W) {
                V v;
#pragma unroll
                for (int x = 0; x < W; ++x) v[x] = acc[j + x][i] * size;
                *reinterpret_cast<V *>(a.parts + at * DP + JT * (8 * (i / 4) + 4 * hh + i % 4) + j) = v;
            }
        return;
    }
    T *to = static_cast<T *>(a.out) + (s.first + row_token) * a.o_ts + row_head * a.o_hs;
    const float r = sum == 0.0f ? 0.0f : size / (sum * a.entry);
    typedef T V __attribute__((ext_vector_type(W)));
    typedef V VA __attribute__((aligned(sizeof(T))));
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int j = 0; j < JT; j += W) {
            const uint32_t d = JT * (8 * (i / 4) + 4 * hh + i % 4) + j;
            V v;
#pragma unroll
            for (int x = 0; x < W; ++x) v[x] = (T)(acc[j + x][i] * r);
            if (d < a.dim) *reinterpret_cast<VA *>(to + d) = v;
        }
}

}  // namespace
