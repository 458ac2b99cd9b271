// dq8 kernels: attention over a paged cache of 8-bit keys and values, many query rows per cached head (prompts and their chunks).
//
// The mathematics is that of dq8_kernels_attend.hpp; here the matrix instructions and the vector unit bound the time, not the
// memory.  A workgroup of eight wavefronts has 256 query rows of one cached head, 32 per wavefront.  A tile of tokens is
// looked up once for all of them: every wavefront turns its eighth of the tile's codes into binary16 and leaves it in LDS in the order
// in which the lanes of a matrix instruction take it (16 bytes per lane, so that neither side has bank conflicts), one tile ahead of
// the one that is multiplied.  Products are 32x32x16: S^T = K Q^T with a query per column, lane % 32, sixteen tokens in a lane's
// registers; these are P^T as operand of out^T = V^T P^T, where the order of a lane's eight tokens is that of its registers.
// The scales of a tile's tokens go through LDS as factors of scores and weights.  Whether a row's products of weights and value scales stay
// in range is asked of its largest weight and the tile's largest scale; where they may not, its reference is moved by these two too, which
// say too much by 2^kEven at most, or else by all of its products.
//
// What bounds it (2048 new tokens after 8192, 32 heads on 8 of 128: 309 GFLOP in 440 to 500 us by the card's clocks, 0.62 to 0.70
// PFLOP/s; a large matrix product of the library reaches 1.20): a tile's scores, weights and sums are one chain, and two wavefronts
// per SIMD, all that the registers allow, do not cover it.  Counters (a dispatch of 511 us): the matrix units are busy for 30 % of the time,
// the vector unit 43 %, LDS 49 %, and wavefronts wait for half of theirs.  Half of the wavefronts go half a tile late, so that one's
// products meet another's weights (562 -> 520 us in the profiler's clocks); 64 rows per wavefront and four of them: many more spills;
// without LDS, each wavefront looking up its own tiles: 3260 us.  Of the 256 registers the heads of 128 spill 28: a tile with hidden tokens
// reads 13 of them back, the others are for the branch that moves references.  Heads of 256 spill 84, some in every tile.
#pragma once
#include "dq8_kernels_attend.hpp"

namespace {

typedef float v16 __attribute__((ext_vector_type(16)));

constexpr int kGroupVector = 0x2, kGroupMatrix = 0x8, kGroupRead = 0x100;  // instructions, for the scheduler
constexpr int kChunkWaves = 8, kChunkWg = kChunkWaves * kWave;

// The job of number idx, counted over sequences: sequence b and the number in it.  Every wavefront by itself; idx < their number.
struct Place {
    uint32_t b, job, jobs;  // jobs: how many there are
};

__device__ __forceinline__ Place place_of(const AttendArgs &a, uint32_t rows, uint32_t idx)
{
    const uint32_t lane = threadIdx.x & 63, run = (a.batch + kWave - 1) / kWave;
    const uint64_t mine = run_sum(a, rows, lane, run, [&](const Seq &s) { return (uint64_t)s.q_tiles * a.kv_heads; });
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
    static constexpr int kKeyBytes = kKeyFrags * 1024, kValueBytes = kValueFrags * 1024;  // of a tile
    static_assert(kKeyFrags == kValueFrags && (kApart ? 2 * kPairs == kChunkWaves : kPairs == kChunkWaves), "as much work for every wavefront");
    static_assert(kTokens <= kWave, "a lane for every token's scales");
};

constexpr int kEven = 3;
// Scales are staged times powers of two.  Value scales: beside those near 2^128 weights down to 2^-22 of the largest stay normal numbers.
// Key scales: their products with those of 256 elements of a query and a code (2^39) stay in binary32, whatever the softmax's factor.
constexpr float kStaged = 14.0f;
constexpr int kKeyStaged = 40;

// One tile's scales in LDS: factors of scores and of weights, which tokens are there, the log2 of the largest of the latter
// and whether some are less than 2^-kEven of it.
// A token whose value scale is not finite has weight factor 0 and a score that is NaN.
template <int TOKENS>
struct ChunkScales {
    float key[TOKENS], value[TOKENS];
    uint64_t there;
    float most;
    uint32_t uneven;
};

template <int DP, int TH, typename T>
__global__ __launch_bounds__(kChunkWg, 2) void k_cache_attend_chunk(const uint32_t *__restrict__ tab, AttendArgs a, uint32_t splits)
{
    typedef ChunkShape<DP, TH> S;
    constexpr int KS = S::KS, JT = S::JT, US = S::US, TOKENS = S::kTokens;
    __shared__ __align__(256) uint32_t lut[256 * kLutCopies];
    __shared__ __align__(16) uint8_t key_tiles[2 * S::kKeyBytes], value_tiles[3 * S::kValueBytes];
    __shared__ __align__(16) ChunkScales<TOKENS> scales[3];
    __shared__ float ups[kChunkWg];  // a thread's `up` as it is without a lift
    __shared__ Row lifted[kChunkWg];  // and its row where rows have lifts
    const uint32_t lane = threadIdx.x & 63, wave = wave_in_wg(), n = lane & 31, hh = lane >> 5, lane4 = lane * 4;
    // the last query rows of a sequence see most: they begin first
    const Place place = place_of(a, S::kRows, blockIdx.x / splits);
    if (a.parts && blockIdx.x == 0 && threadIdx.x == 0) *a.n_records = place.jobs;
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
    const int32_t upto = p0 + (int32_t)(last_row / a.group) + 1, first_pos = p0 + (int32_t)(row0 / a.group);
    const int32_t lowest = a.window > 0 && first_pos > 0 ? first_pos - a.window + 1 : 0;  // (queries before position 0 see nothing)
    const uint32_t first_tile = lowest > 0 ? (uint32_t)lowest / TOKENS : 0, end_tile = upto > 0 ? ((uint32_t)upto + TOKENS - 1) / TOKENS : 0;
    const uint32_t count = end_tile > first_tile ? end_tile - first_tile : 0;
    const uint32_t t_begin = first_tile + (uint32_t)((uint64_t)count * split / splits), t_end = first_tile + (uint32_t)((uint64_t)count * (split + 1) / splits);

    // the wavefront's 32 query rows as operands, scaled by a power of two each: eight elements of step k, see fetch for their order
    v8h q[KS];
    const uint32_t w_first = row0 + wave * 32, row = w_first + n;
    const bool in = row < total_rows;
    const uint32_t row_token = in ? row / a.group : 0, row_head = head * a.group + (in ? row - row_token * a.group : 0);
    const int32_t pos = in ? p0 + (int32_t)row_token : -1;
    // Weights are exp2(products of a row times up - from).  up: a power of two, exact, so that a largest score and its reference are the
    // same number.  far: whether some row of the wavefront has a lift, or had; the scores are then replaced by those minus the shift plus
    // the lift, and shift, lift and sum are in LDS, where they take no registers.
    float up, from = -FLT_MAX, sum = 0.0f;
    bool far = false;
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
        // (neither zero nor infinite: times the -infinity of what is not seen, or a score of zero, it would be NaN)
        up = fminf(fmaxf(__builtin_amdgcn_ldexpf(1.0f, __builtin_amdgcn_frexp_expf(a.factor) + e - kQueryTop + kKeyStaged), 0x1p-149f), 0x1p127f);
        ups[threadIdx.x] = up;
    }
    v16 acc[JT];
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[j][i] = 0.0f;
    // positions of the wavefront's first and last row (-1: it has none)
    const int32_t p_first = w_first < total_rows ? p0 + (int32_t)(w_first / a.group) : -1;
    const int32_t p_last = w_first < total_rows ? p0 + (int32_t)((w_first + 31 < total_rows ? w_first + 31 : total_rows - 1) / a.group) : -1;

    // ---- the tile's way into LDS.  Keys: a lane takes 16 bytes of one of 32 tokens, which are its eight elements of two steps.  Values: a
    // lane takes a word of each of the eight tokens of its half of step u, two bytes of which are elements of its two groups.
    // The page numbers of 64 groups of 16 tokens are in the lanes, those of the next 64 too.
    constexpr uint32_t GROUPS = TOKENS / 16, BLOCK = kWave / GROUPS;  // groups of a tile; tiles of 64 groups
    const int32_t *table = a.pages + (size_t)place.b * a.max_pages;
    auto pages_from = [&](uint32_t tile) {
        const uint32_t index = (tile * TOKENS + lane * 16) >> a.page_shift;
        return (uint32_t)table[index < a.max_pages ? index : a.max_pages - 1];
    };
    uint32_t pages_now = pages_from(t_begin), pages_then = pages_from(t_begin + BLOCK), in_block = 0;
    const bool has_keys = !S::kApart || wave < (uint32_t)S::kPairs, has_values = !S::kApart || !has_keys;
    const uint32_t kp = wave % S::kPairs, k_half = kp / JT, k_pair = kp % JT;       // this wavefront's pair of key operands
    const uint32_t vp = wave % S::kPairs, u = vp % US, two = vp / US;               // and of value operands
    const uint32_t v_select = 0x0C0C0400u + ((two & 1) << 9);                       // its first byte of a word
    const uint32_t in_page = (1u << a.page_shift) - 1, page_rows = a.kv_heads << a.page_shift, page_bytes = page_rows * a.dim;
    const uint32_t head_row = head << a.page_shift;
    const uint32_t dim = a.dim;
    const uint32_t k_d = 32 * k_pair + 16 * hh, k_at = head_row * dim + (k_d < dim ? k_d : 0);
    const uint32_t v_d = JT * n + 4 * (two / 2), v_at = 4 * hh * dim + (v_d < dim ? v_d : 0);
    u4 kc = {0, 0, 0, 0};
    uint32_t vc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    float ks = 0.0f, vs = 0.0f;
    bool s_there = false;
    auto inside = [&](uint32_t page) { return page < a.n_pages ? page : 0; };
    // the loads of a tile; tiles in order
    auto fetch = [&](uint32_t tile) {
        if (in_block == BLOCK) {
            in_block = 0;
            pages_now = pages_then;
            pages_then = pages_from(tile + BLOCK);
        }
        const int first = (int)(in_block * GROUPS);
        ++in_block;
        if (has_keys) {
            const uint32_t p0 = (uint32_t)__builtin_amdgcn_readlane((int)pages_now, first + 2 * (int)k_half), p1 = (uint32_t)__builtin_amdgcn_readlane((int)pages_now, first + 2 * (int)k_half + 1);
            const uint32_t page = n < 16 ? inside(p0) : inside(p1), token = tile * TOKENS + k_half * 32 + n;
            kc = *reinterpret_cast<const u4 *>(a.k_codes + (uint64_t)page * page_bytes + (k_at + (token & in_page) * dim));
        }
        if (has_values) {
            const uint32_t page = inside((uint32_t)__builtin_amdgcn_readlane((int)pages_now, first + (int)u));
            const uint8_t *v = a.v_codes + (uint64_t)page * page_bytes + (head_row + ((tile * TOKENS + u * 16) & in_page)) * dim;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint8_t *at = v + (i % 4 + 8 * (i / 4)) * dim;
                vc[i] = JT == 2 ? load_at<uint16_t>(at, v_at) : load_at<uint32_t>(at, v_at);
            }
        }
        if (wave == 0) {
            const uint32_t page = (uint32_t)__shfl((int)pages_now, first + (int)(lane % TOKENS) / 16), token = tile * TOKENS + lane % TOKENS;
            const uint64_t at = (uint64_t)inside(page) * page_rows + head_row + (token & in_page);
            ks = a.k_scales[at];
            vs = a.v_scales[at];
            s_there = (int32_t)token < s.len && page < a.n_pages;
        }
    };
    const float factor = __builtin_amdgcn_ldexpf(__builtin_amdgcn_frexp_mantf(fabsf(a.factor)), -kKeyStaged);  // (its exponent is in `up`)
    auto eighth_of = [&](uint32_t select) {
        v8h f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = *reinterpret_cast<const _Float16 *>(reinterpret_cast<const char *>(lut) + __builtin_amdgcn_perm(vc[i], lane4, select));
        return f;
    };
    auto put = [&](uint32_t buffer2, uint32_t buffer3) {
        if (has_keys) {
            v8h *const f = reinterpret_cast<v8h *>(key_tiles + buffer2 * S::kKeyBytes) + (k_half * KS + 2 * k_pair) * kWave + lane;
            f[0] = eight(lut, kc.x, kc.y, lane4);
            f[kWave] = eight(lut, kc.z, kc.w, lane4);
        }
        if (has_values) {
            v8h *const f = reinterpret_cast<v8h *>(value_tiles + buffer3 * S::kValueBytes) + (u * JT + 2 * two) * kWave + lane;
            f[0] = eighth_of(v_select);
            f[kWave] = eighth_of(v_select + 0x100u);
        }
    };
    auto put_scales = [&](uint32_t buffer3) {
        if (wave != 0) return;
        const bool finite = fabsf(vs) <= FLT_MAX;  // (if not, the score becomes NaN for whoever sees it)
        const float y = s_there && finite ? vs * 0x1p-14f : 0.0f;
        float most = fabsf(y);
#pragma unroll
        for (int m = 1; m < TOKENS; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
        ChunkScales<TOKENS> &sc = scales[buffer3];
        if (lane < TOKENS) {
            sc.key[lane] = finite ? ks * factor : __builtin_nanf("");
            sc.value[lane] = y;
        }
        const uint64_t all = __builtin_amdgcn_ballot_w64(s_there);
        const uint64_t low = __builtin_amdgcn_ballot_w64(s_there && fabsf(y) * (float)(1 << kEven) < most);
        if (lane == 0) {
            sc.there = all;
            sc.most = __builtin_amdgcn_logf(most);
            sc.uneven = low != 0;
        }
    };

    v16 st[TH];
    auto score = [&](uint32_t buffer2) {
        const v8h *const keys = reinterpret_cast<const v8h *>(key_tiles + buffer2 * S::kKeyBytes) + lane;
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) st[h][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int h = 0; h < TH; ++h) st[h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(keys[(h * KS + k) * kWave], q[k], st[h], 0, 0, 0);
    };
    const int32_t hidden_upto = a.window > 0 && in ? pos - a.window : INT32_MIN;
    auto add = [&](uint32_t tile, uint32_t buffer3) {
        const v8h *const values = reinterpret_cast<const v8h *>(value_tiles + buffer3 * S::kValueBytes) + lane;
        const ChunkScales<TOKENS> &sc = scales[buffer3];
        const int32_t t = (int32_t)(tile * TOKENS);
        const uint64_t there = sc.there;  // (32 tokens: both halves of the wavefront say the same)
        const float most = sc.most;
        // scores times their keys' scales; those that a row does not see become -infinity
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const v4 f = *reinterpret_cast<const v4 *>(sc.key + 32 * h + 8 * i4 + 4 * hh);
#pragma unroll
                for (int i = 0; i < 4; ++i) st[h][4 * i4 + i] *= f[i];
            }
        const bool masked = t + TOKENS - 1 > p_first || (a.window > 0 && t <= p_last - a.window) || there != ~0ull;
        if (masked) {
#pragma unroll
            for (int h = 0; h < TH; ++h)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int32_t token = t + 32 * h + 8 * (i / 4) + 4 * (int32_t)hh + i % 4;
                    st[h][i] = ((token <= pos) & (token > hidden_upto)) ? st[h][i] : -__builtin_inff();
                }
            if (there != ~0ull)
#pragma unroll
                for (int h = 0; h < TH; ++h)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!(there >> (32 * h + 8 * (i / 4) + 4 * hh + i % 4) & 1)) st[h][i] = -__builtin_inff();
        }
        float high = -__builtin_inff();
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i) high = fmaxf(high, st[h][i]);
        if (far || __builtin_amdgcn_ballot_w64(high * up > from + kWeightLimit || high * up + most > from + kProductLimit) != 0) {
            const float by = ups[threadIdx.x];
            Row ref = {from, 0.0f, sum};
            if (far) ref = lifted[threadIdx.x];
            high = fmaxf(high, __shfl_xor(high, 32)) * by;
            float large = most;
            if (sc.uneven) {
                large = -__builtin_inff();
#pragma unroll
                for (int h = 0; h < TH; ++h)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const v4 f = *reinterpret_cast<const v4 *>(sc.value + 32 * h + 8 * i4 + 4 * hh);
#pragma unroll
                        for (int i = 0; i < 4; ++i) large = fmaxf(large, __builtin_fmaf(st[h][4 * i4 + i], by, -high) + __builtin_amdgcn_logf(fabsf(f[i])));
                    }
                large = fmaxf(large, __shfl_xor(large, 32));
            }
            const float less = ref.raise(high, large);
#pragma unroll
            for (int j = 0; j < JT; ++j) acc[j] *= less;
            from = ref.shift;
            far = far || __builtin_amdgcn_ballot_w64(ref.lift != 0.0f) != 0;
            if (far) {
#pragma unroll
                for (int h = 0; h < TH; ++h)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float t = __builtin_fmaf(st[h][i], by, -ref.shift);
                        ref.sum += __builtin_amdgcn_exp2f(t);
                        st[h][i] = t + ref.lift;
                    }
                lifted[threadIdx.x] = ref;
                up = 1.0f;
                from = 0.0f;
            }
            sum = ref.sum;
        }
        v8h p[US];
#pragma unroll
        for (int h = 0; h < TH; ++h)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                const v4 f = *reinterpret_cast<const v4 *>(sc.value + 32 * h + 8 * i4 + 4 * hh);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(st[h][4 * i4 + i], up, -from));
                    sum += w;
                    p[2 * h + i4 / 2][4 * (i4 % 2) + i] = (_Float16)(w * f[i]);
                }
            }
#pragma unroll
        for (int x = 0; x < US; ++x)
#pragma unroll
            for (int j = 0; j < JT; ++j) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values[(x * JT + j) * kWave], p[x], acc[j], 0, 0, 0);
        // the products of the first half of the tokens between the weights of the second
        if constexpr (TH == 2) {
            __builtin_amdgcn_sched_group_barrier(kGroupVector, 72, 0);
#pragma unroll
            for (int i = 0; i < US * JT / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(kGroupMatrix, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kGroupVector, 144 / (US * JT), 0);
            }
        }
    };

    __syncthreads();  // the table
    if (t_begin < t_end) {
        // Half of the wavefronts, one of each SIMD's two, take the weights and sums of a tile together with the next tile's scores: while one
        // of the two uses the vector unit, the other has products to do.  A barrier per tile, two buffers of keys and three of values.
        const bool late = wave >= kChunkWaves / 2;
        const int32_t low = a.window > 0 && p_first > 0 ? p_first - a.window + 1 : 0, least = low > 0 ? low : 0;  // of the tokens that its rows see
        auto seen = [&](uint32_t tile) {
            const int32_t t = (int32_t)(tile * TOKENS);
            return t <= p_last && t > least - TOKENS;
        };
        fetch(t_begin);
        put(0, 0);
        put_scales(0);
        if (t_begin + 1 < t_end) fetch(t_begin + 1);
        __syncthreads();
        uint32_t two_of = 0, three_of = 0;  // buffers of the present tile
        for (uint32_t tile = t_begin; tile < t_end; ++tile) {
            const uint32_t before = three_of == 0 ? 2 : three_of - 1, behind = three_of == 2 ? 0 : three_of + 1;
            if (late && tile > t_begin && seen(tile - 1)) add(tile - 1, before);
            // (behind the last tile that one again, for nobody; the scores of a tile that no row sees, for nobody)
            put(two_of ^ 1, behind);
            score(two_of);
            if constexpr (!S::kApart) {  // products, look-ups and what they need in turn
#pragma unroll
                for (int i = 0; i < S::kKeyFrags; ++i) {
                    __builtin_amdgcn_sched_group_barrier(kGroupRead, 3, 0);
                    __builtin_amdgcn_sched_group_barrier(kGroupMatrix, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kGroupVector, 4, 0);
                }
            }
            put_scales(behind);
            if (tile + 2 < t_end) fetch(tile + 2);
            if (!late && seen(tile)) add(tile, three_of);
            __syncthreads();
            two_of ^= 1;
            three_of = behind;
        }
        if (late && seen(t_end - 1)) add(t_end - 1, three_of == 0 ? 2 : three_of - 1);
    }

    const size_t part = (size_t)(blockIdx.x / splits) * splits + split;
    if (a.parts && splits > 1 && split == 0 && threadIdx.x == 0)
        a.records[blockIdx.x / splits] = int4{(int)place.b, (int)(q_tile * a.kv_heads + head), (int)part, (int)splits};
    Row ref = {from, 0.0f, sum};
    if (far) ref = lifted[threadIdx.x];
    sum = ref.sum;
    sum += __shfl_xor(sum, 32);
    const float r = sum == 0.0f ? 0.0f : 1.0f / (sum * a.entry), down = __builtin_amdgcn_exp2f(kStaged - ref.lift);
    if (!in) return;
    constexpr int W = JT < 4 ? JT : 4;
    if (splits > 1) {
        const size_t at = part * a.rows + wave * 32 + n;
        if (hh == 0) a.sums[at] = sum_of_part(ref.shift, sum);
        typedef float V __attribute__((ext_vector_type(W)));
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int j = 0; j < JT; j += W) {
                V v;
#pragma unroll
                for (int x = 0; x < W; ++x) v[x] = acc[j + x][i] * r * down;
                *reinterpret_cast<V *>(a.parts + at * DP + JT * (8 * (i / 4) + 4 * hh + i % 4) + j) = v;
            }
        return;
    }
    T *to = static_cast<T *>(a.out) + (s.first + row_token) * a.o_ts + row_head * a.o_hs;
    typedef T V __attribute__((ext_vector_type(W)));
    typedef V VA __attribute__((aligned(sizeof(T))));
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int j = 0; j < JT; j += W) {
            const uint32_t d = JT * (8 * (i / 4) + 4 * hh + i % 4) + j;
            V v;
#pragma unroll
            for (int x = 0; x < W; ++x) v[x] = (T)(acc[j + x][i] * r * down);
            if (d < a.dim) *reinterpret_cast<VA *>(to + d) = v;
        }
}

}  // namespace
