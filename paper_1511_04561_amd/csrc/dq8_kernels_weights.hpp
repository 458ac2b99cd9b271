// dq8 kernels: weights in 4 bits and their products with a few rows of activations.
//
// Format.  A code is a 4-bit floating-point number (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6); gfx950 turns two of
// them into two binary16 or bfloat16 numbers in one instruction.  A tile of 16 rows and 128 columns is 1 KiB in the order in which
// the lanes of a wavefront load it: lane 16 g + n holds of row n the words s = 0 .. 3, and word s the columns 32 s + 8 g .. + 7.  So
// word s of all lanes is the operand of one 16x16x32 matrix instruction, and the 32 columns of that share a scale.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef _Float16 w8h __attribute__((ext_vector_type(8)));
typedef __bf16 w8b __attribute__((ext_vector_type(8)));
typedef _Float16 w2h __attribute__((ext_vector_type(2)));
typedef __bf16 w2b __attribute__((ext_vector_type(2)));
typedef float w4f __attribute__((ext_vector_type(4)));
typedef uint32_t w4u __attribute__((ext_vector_type(4)));

constexpr int kTileRows = 16, kTileCols = 128, kTileBytes = 1024, kPieces = 64;
constexpr float kScaleTop = 170.0f * 0x1p118f;  // the largest bfloat16 number whose sixfold is finite

__device__ __forceinline__ float bf16_value(uint32_t bits16) { return __uint_as_float(bits16 << 16); }

// ---------------------------------------------------------------- compression and expansion

typedef uint16_t w2s __attribute__((ext_vector_type(2)));

// The last elements of a row, fewer than eight, from column k on, zeros behind them: all loads at once (with a branch around each, one would wait for the other).
template <typename T>
__device__ __forceinline__ w4u last_eight(const T *row, size_t k, size_t cols)
{
    static_assert(sizeof(T) == 2, "bfloat16 or binary16");
    const uint16_t *bits = reinterpret_cast<const uint16_t *>(row);
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = bits[k + e < cols ? k + e : cols - 1];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < cols ? v[e] : 0;
    return w4u{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
}

// 16 bytes without their first `halves` times two, zeros behind them.
__device__ __forceinline__ w4u moved_down(w4u v, size_t halves)
{
    uint64_t lo = (uint64_t)v.y << 32 | v.x, hi = (uint64_t)v.w << 32 | v.z;
    const uint32_t bits = 16 * (uint32_t)(halves & 3);
    if (halves & 4) lo = hi, hi = 0;
    lo = lo >> bits | hi << 1 << (63 - bits), hi >>= bits;
    if (halves >= 8) lo = hi = 0;
    return w4u{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// The scale of a group whose largest absolute value has these bits as binary32: the nearest bfloat16 number to a sixth of it.
__device__ __forceinline__ float scale_of(uint32_t most)
{
    const uint32_t bits = __float_as_uint(__uint_as_float(most) / 6.0f);
    const float s = bf16_value((bits + 0x7FFFu + ((bits >> 16) & 1)) >> 16);
    return s < kScaleTop ? s : kScaleTop;
}

__device__ __forceinline__ uint32_t most_of_row(uint32_t most)
{
#pragma unroll
    for (int d = 16; d <= 32; d *= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)most, d);
        most = o > most ? o : most;
    }
    return most;
}

// A lane's eight elements of a run, and how they become codes.  binary32: the nearest of eight magnitudes, the smaller of two as near, by comparisons with the
// borders between them times the scale.  These products have 3 + 8 bits: they are exact, and the comparison is one of real numbers.
template <typename T>
struct Eight {
    float x[8];

    __device__ __forceinline__ void take(const w4u *row, uint32_t piece, uint32_t n)
    {
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
            const w4u v = row[(2 * piece + h) ^ n];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * h + e] = __uint_as_float(v[e]);
        }
    }

    // The bits of the largest absolute value: infinities and NaN are above all others.
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = __float_as_uint(x[e]) & 0x7FFFFFFFu;
            m = b > m ? b : m;
        }
        return m;
    }

    __device__ __forceinline__ uint32_t codes(float s) const
    {
        const float b0 = 0.25f * s, b1 = 0.75f * s, b2 = 1.25f * s, b3 = 1.75f * s, b4 = 2.5f * s, b5 = 3.5f * s, b6 = 5.0f * s;
        uint32_t v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = fabsf(x[e]);
            const bool c2 = a > b3, c1 = a > (c2 ? b5 : b1), c0 = a > (c2 ? (c1 ? b6 : b4) : (c1 ? b2 : b0));
            v |= ((__float_as_uint(x[e]) >> 31) * 8 + (uint32_t)c2 * 4 + (uint32_t)c1 * 2 + (uint32_t)c0) << (4 * e);
        }
        return v;
    }
};

// 16 bits: the conversion to 4 bits rounds the quotient x / s to the nearest, and to even where it lies between two.  A border times the scale and x have 11
// bits at most, so that x, where it is not on a border, is at least 2^-11 of itself away from it: quotients that are all made smaller by 2^-13 (their
// own rounding is below 2^-22) lie on the same side of every border as the true ones, and those on a border below it.  The scale's exponent goes into the
// conversion and one over the rest into a product, so that no reciprocal leaves binary32.
template <typename T>
struct Eight16 {
    w4u raw;

    __device__ __forceinline__ void take(const w4u *row, uint32_t piece, uint32_t n) { raw = row[piece ^ n]; }

    __device__ __forceinline__ float at(int e) const
    {
        const uint32_t w = raw[e / 2];
        if constexpr (__is_same(T, __bf16)) {
            return __uint_as_float(e % 2 ? w & 0xFFFF0000u : w << 16);
        } else {
            const uint16_t u = (uint16_t)(e % 2 ? w >> 16 : w);
            T h;
            __builtin_memcpy(&h, &u, 2);
            return (float)h;
        }
    }

    __device__ __forceinline__ uint32_t most() const
    {
        w2s m = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = raw[i] & 0x7FFF7FFFu;
            w2s h;
            __builtin_memcpy(&h, &u, 4);
            m = __builtin_elementwise_max(m, h);
        }
        const uint16_t u = m.x > m.y ? m.x : m.y;
        T h;
        __builtin_memcpy(&h, &u, 2);
        return __float_as_uint((float)h);
    }

    __device__ __forceinline__ uint32_t codes(float s) const
    {
        const uint32_t e = __float_as_uint(s) & 0x7F800000u, power = e ? e : 0x00800000u;  // 2^exponent, of the smallest normal number at least
        const float two = __uint_as_float(power), part = __builtin_amdgcn_ldexpf(s, 127 - (int)(power >> 23)), f = (1.0f - 0x1p-13f) / part;
        uint32_t v = 0;
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, at(0) * f, at(1) * f, two, 0);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, at(2) * f, at(3) * f, two, 1);
        v = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, at(4) * f, at(5) * f, two, 2);
        return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(v, at(6) * f, at(7) * f, two, 3);
    }
};
template <>
struct Eight<__bf16> : Eight16<__bf16> {};
template <>
struct Eight<_Float16> : Eight16<_Float16> {};

// A wavefront per tile: lane 16 g + n has of row n the four runs of eight columns that its piece holds.  The tile comes in by way of LDS (the wavefront's own; 16 bytes
// change places by the row, so that neither side meets bank conflicts): 256 or 512 bytes of a row lie side by side in a load.
// 14336 x 4096 bfloat16, groups of 32: 150 MB in 25.5 us (memory; 26 with loads of 64 bytes of each of sixteen rows, and 48 where these start between two words; 49
// with the bisection of binary32, which is bound by the vector unit).
template <typename T, int GROUP>
__global__ __launch_bounds__(256) void k_weights_encode(const T *__restrict__ w, size_t stride, size_t rows, size_t cols, uint32_t col_tiles, size_t tiles,
                                                        uint8_t *__restrict__ codes, uint16_t *__restrict__ scales)
{
    constexpr int PER = kTileCols / GROUP, RUNS = 4 / PER;  // groups of a row in a tile; runs of a group
    constexpr uint32_t EACH = 16 / sizeof(T), UNITS = kTileCols / EACH, LOADS = kTileRows * UNITS / 64;
    __shared__ w4u lds[4][kTileRows * UNITS];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const size_t tile = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    w4u *mine = lds[threadIdx.x >> 6];
    const size_t rt = tile / col_tiles, ct = tile - rt * col_tiles;
    const T *from = w + rt * kTileRows * stride + ct * kTileCols;
    const uint32_t tall = rows - rt * kTileRows < kTileRows ? (uint32_t)(rows - rt * kTileRows) : kTileRows;
    const uint32_t wide = cols - ct * kTileCols < kTileCols ? (uint32_t)(cols - ct * kTileCols) : kTileCols;
    auto place = [&](uint32_t at, w4u v) { mine[at / UNITS * UNITS + (at % UNITS ^ at / UNITS)] = v; };
    if (tall == kTileRows && wide == kTileCols) {  // (all its loads at once)
        typedef w4u WA __attribute__((aligned(2)));
        w4u unit[LOADS];
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t at = i * 64 + lane;
            unit[i] = *reinterpret_cast<const WA *>(from + at / UNITS * stride + at % UNITS * EACH);
        }
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) place(i * 64 + lane, unit[i]);
    } else if (wide >= EACH) {  // (of a ragged end the row's last 16 bytes, moved down, so that these too go out together)
        typedef w4u WA __attribute__((aligned(2)));
        w4u unit[LOADS];
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t at = i * 64 + lane, m = at / UNITS, k = at % UNITS * EACH;
            unit[i] = *reinterpret_cast<const WA *>(from + (m < tall ? m : tall - 1) * stride + (k + EACH <= wide ? k : wide - EACH));
        }
#pragma unroll
        for (uint32_t i = 0; i < LOADS; ++i) {
            const uint32_t at = i * 64 + lane, k = at % UNITS * EACH;
            if (wide % EACH != 0 && k + EACH > wide) unit[i] = moved_down(unit[i], (k + EACH - wide) * (sizeof(T) / 2));
            place(at, at / UNITS < tall && k < wide ? unit[i] : w4u{0, 0, 0, 0});
        }
    } else {
        for (uint32_t at = lane; at < kTileRows * UNITS; at += 64) place(at, w4u{0, 0, 0, 0});
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < tall)
            for (uint32_t k = 0; k < wide; ++k) reinterpret_cast<T *>(mine + lane * UNITS + lane)[k] = from[lane * stride + k];  // (the first 16 bytes of row `lane` are there)
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    Eight<T> x[4];
#pragma unroll
    for (uint32_t s = 0; s < 4; ++s) x[s].take(mine + n * UNITS, 4 * s + g, n);
    w4u word;
    uint32_t scale[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        uint32_t most = 0;
#pragma unroll
        for (int s = p * RUNS; s < (p + 1) * RUNS; ++s) {
            const uint32_t m = x[s].most();
            most = m > most ? m : most;
        }
        most = most_of_row(most);
        const bool bad = most >= 0x7F800000u;
        const float s = scale_of(most);
        scale[p] = bad ? 0x7FC0u : __float_as_uint(s) >> 16;
        const uint32_t keep = bad ? 0u : s == 0.0f ? 0x88888888u : 0xFFFFFFFFu;
#pragma unroll
        for (int r = p * RUNS; r < (p + 1) * RUNS; ++r) word[r] = x[r].codes(s == 0.0f ? 1.0f : s) & keep;
    }
    reinterpret_cast<w4u *>(codes + tile * kTileBytes)[lane] = word;
    if (g == 0) {
        uint16_t *to = scales + (tile * kTileRows + n) * PER;
        if constexpr (PER == 4)
            *reinterpret_cast<uint2 *>(to) = uint2{scale[0] | scale[1] << 16, scale[2] | scale[3] << 16};
        else if constexpr (PER == 2)
            *reinterpret_cast<uint32_t *>(to) = scale[0] | scale[1] << 16;
        else
            *to = (uint16_t)scale[0];
    }
}

// Two values of a word's byte B, times 2^0.
template <int B>
__device__ __forceinline__ void two_values(uint32_t word, float &a, float &b)
{
    const w2h v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, 1.0f, B);
    a = (float)v.x;
    b = (float)v.y;
}

// The reverse, bound by its writes: 24.5 us.  The values go out by way of LDS (a wavefront's own; 16 bytes change places by the row, so that neither side meets bank
// conflicts), so that 256 or 512 bytes of a row lie side by side in a store: rows that start anywhere cost 29 us (14336 x 4104 bfloat16), stores of 64 bytes of each of
// sixteen rows 47, and 28 where they start at multiples of 64 bytes.
template <typename T, int GROUP>
__global__ __launch_bounds__(256) void k_weights_decode(const uint8_t *__restrict__ codes, const uint16_t *__restrict__ scales, size_t rows, size_t cols,
                                                        uint32_t col_tiles, size_t tiles, T *__restrict__ w, size_t stride)
{
    constexpr int PER = kTileCols / GROUP, RUNS = 4 / PER;
    constexpr uint32_t EACH = 16 / sizeof(T), UNITS = kTileCols / EACH;  // values of 16 bytes, and such of a row
    typedef T V __attribute__((ext_vector_type(EACH)));
    typedef V VA __attribute__((aligned(sizeof(T))));
    __shared__ V lds[4][kTileRows * UNITS];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const size_t tile = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    V *mine = lds[threadIdx.x >> 6];
    const size_t rt = tile / col_tiles, ct = tile - rt * col_tiles;
    const w4u word = *reinterpret_cast<const w4u *>(codes + tile * kTileBytes + lane * 16);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float s = bf16_value(scales[(tile * kTileRows + n) * PER + r / RUNS]);
        float x[8];
        two_values<0>(word[r], x[0], x[1]);
        two_values<1>(word[r], x[2], x[3]);
        two_values<2>(word[r], x[4], x[5]);
        two_values<3>(word[r], x[6], x[7]);
#pragma unroll
        for (uint32_t h = 0; h < 8 / EACH; ++h) {
            V v;
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e) v[e] = (T)(x[h * EACH + e] * s);
            mine[n * UNITS + (((4 * r + g) * (8 / EACH) + h) ^ n)] = v;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (uint32_t i = 0; i < kTileRows * UNITS / 64; ++i) {
        const uint32_t at = i * 64 + lane, m = at / UNITS, u = at % UNITS;
        const size_t row = rt * kTileRows + m, k = ct * kTileCols + u * EACH;
        if (row >= rows || k >= cols) continue;
        const V v = mine[m * UNITS + (u ^ m)];
        T *to = w + row * stride + k;
        if (k + EACH <= cols) {
            *reinterpret_cast<VA *>(to) = v;
        } else {
#pragma unroll
            for (uint32_t e = 0; e < EACH; ++e)
                if (k + e < cols) to[e] = v[e];
        }
    }
}

// ---------------------------------------------------------------- products

struct ProductArgs {
    const uint8_t *codes;
    const uint16_t *scales;
    const void *x;
    void *out;
    const float *bias;
    size_t x_stride, out_stride;
    uint32_t tokens, rows, cols, row_tiles, col_tiles;
    int wide;  // whether the results are binary32
};

// What depends on the type of the activations.  Weights enter the products at 1 / kLift of their value, so that a group's sum of 128 products
// leaves binary32 for no activation that binary32's exponents hold; the result is lifted at the end.  (Binary16 needs none of that.)
template <typename T>
struct Operand;
template <>
struct Operand<_Float16> {
    typedef w8h type;
    static constexpr float kLift = 1.0f;
    static __device__ __forceinline__ type weights(uint32_t v)
    {
        const w2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 1);
        const w2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(v, 1.0f, 3);
        return type{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    }
    static __device__ __forceinline__ w4f product(type a, type b, w4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Operand<__bf16> {
    typedef w8b type;
    static constexpr float kLift = 0x1p10f;
    static __device__ __forceinline__ type weights(uint32_t v)
    {
        const w2b a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 0x1p-10f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 0x1p-10f, 1);
        const w2b c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 0x1p-10f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, 0x1p-10f, 3);
        return type{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
    }
    static __device__ __forceinline__ w4f product(type a, type b, w4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// The scales of a weight row in a tile: PER neighbours.
template <int PER>
struct ScaleWord;
template <>
struct ScaleWord<1> {
    typedef uint16_t type;
};
template <>
struct ScaleWord<2> {
    typedef uint32_t type;
};
template <>
struct ScaleWord<4> {
    typedef uint32_t type __attribute__((ext_vector_type(2)));
};

template <int PER>
__device__ __forceinline__ float scale_at(typename ScaleWord<PER>::type v, int p)
{
    if constexpr (PER == 1) {
        return bf16_value(v);
    } else {
        uint32_t w;
        if constexpr (PER == 2)
            w = v;
        else
            w = v[p / 2];
        return __uint_as_float(p % 2 ? w & 0xFFFF0000u : w << 16);
    }
}

// What a wavefront loads of R row tiles that lie `apart` tiles from each other.
template <int GROUP, int R>
struct TileWords {
    static constexpr int PER = kTileCols / GROUP;
    typedef typename ScaleWord<PER>::type Scale;
    w4u word[R];
    Scale scale[R];
};

// Where a wavefront's R row tiles begin; behind the last one they are the last one again.
template <int GROUP, int R>
struct TileSource {
    static constexpr int PER = kTileCols / GROUP;
    const uint8_t *codes[R];
    const uint16_t *scales[R];

    __device__ __forceinline__ TileSource(const ProductArgs &a, uint32_t row_tile)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const size_t tile = (size_t)(row_tile + r < a.row_tiles ? row_tile + r : a.row_tiles - 1) * a.col_tiles;
            codes[r] = a.codes + tile * kTileBytes;
            scales[r] = a.scales + tile * kTileRows * PER;
        }
    }

    // Weights are read once: past the caches.
    __device__ __forceinline__ void fetch(uint32_t col_tile, uint32_t lane, TileWords<GROUP, R> &t) const
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            t.word[r] = __builtin_nontemporal_load(reinterpret_cast<const w4u *>(codes[r] + (size_t)col_tile * kTileBytes) + lane);
            t.scale[r] = reinterpret_cast<const typename ScaleWord<PER>::type *>(scales[r] + (size_t)col_tile * kTileRows * PER)[lane & 15];
        }
    }
};

// A tile's products: the lane's 16 bytes of its row of activations in LDS for each of the four steps are at x + step[.], TOKENS_APART bytes
// from one token tile to the next.  Products have tokens as rows and weight rows as columns, so that a lane's sums share the scale of its weight
// row.  A lane has four of the 16 tokens of a token tile; with Q = 2 or 1 every token is there 2 or 4 times, and only one of them is scaled
// and added up (16 multiply-adds of a tile with groups of 32 become 4: a third of the vector instructions).
template <typename T, int GROUP, int MT, int Q, int R, int TOKENS_APART>
__device__ __forceinline__ void add_tile(const char *x, const uint32_t (&step)[4], const TileWords<GROUP, R> &t, float (&sum)[MT][R][Q])
{
    constexpr int PER = kTileCols / GROUP, RUNS = 4 / PER;
    typedef Operand<T> Op;
    typedef typename Op::type V;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        V v[MT][RUNS];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int k = 0; k < RUNS; ++k) v[m][k] = *reinterpret_cast<const V *>(x + m * TOKENS_APART + step[p * RUNS + k]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            w4f d[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) d[m] = w4f{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < RUNS; ++k) {
                const V w = Op::weights(t.word[r][p * RUNS + k]);
#pragma unroll
                for (int m = 0; m < MT; ++m) d[m] = Op::product(v[m][k], w, d[m]);
            }
            const float f = scale_at<PER>(t.scale[r], p);
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < Q; ++q) sum[m][r][q] = __builtin_fmaf(d[m][q * (4 / Q)], f, sum[m][r][q]);
        }
    }
}

template <typename T>
__device__ __forceinline__ void store_result(const ProductArgs &a, uint32_t token, uint32_t row, float v)
{
    v *= Operand<T>::kLift;
    if (a.bias) v += a.bias[row];
    const size_t at = token * a.out_stride + row;
    if (a.wide)
        static_cast<float *>(a.out)[at] = v;
    else
        static_cast<T *>(a.out)[at] = (T)v;
}

// A wavefront's results, MT 16 tokens from `first` on and R row tiles, by way of `space` (MT 16 times 64 bytes of LDS that nobody else uses), so that a lane stores
// 16 bytes of a token and not single results of 64 (500 x 22235 results of 128 columns: 18.5 us, without 23.6; 500 x 8192 of 4096 columns 40.4, without 42.2).
template <typename T, typename O, int MT, int R>
__device__ __forceinline__ void store_rows(const ProductArgs &a, char *space, uint32_t lane, uint32_t first, uint32_t row_tile, const float (&sum)[MT][R][4])
{
    typedef w4u WA __attribute__((aligned(2)));
    constexpr int TILES = R * 16 * sizeof(O) < 64 ? R : 64 / (16 * sizeof(O));  // row tiles at a time
    constexpr uint32_t ROWS = TILES * 16, PIECES = ROWS * sizeof(O) / 16, EACH = 16 / sizeof(O);
    const uint32_t n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int r0 = 0; r0 < R; r0 += TILES) {
#pragma unroll
        for (int r = r0; r < r0 + TILES; ++r) {
            const uint32_t row = (row_tile + r) * kTileRows + n;
            const float more = a.bias && row < a.rows ? a.bias[row] : 0.0f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v = sum[m][r][q] * Operand<T>::kLift;
                    if (a.bias) v += more;
                    reinterpret_cast<O *>(space)[(m * 16 + g * 4 + q) * ROWS + (r - r0) * 16 + n] = (O)v;
                }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (uint32_t i = 0; i < MT * 16 * PIECES / 64; ++i) {
            const uint32_t at = i * 64 + lane, token = first + at / PIECES, row = (row_tile + r0) * kTileRows + at % PIECES * EACH;
            if (token >= a.tokens || row >= a.rows) continue;
            O *to = static_cast<O *>(a.out) + token * a.out_stride + row;
            if (row + EACH <= a.rows) {
                *reinterpret_cast<WA *>(to) = reinterpret_cast<const w4u *>(space)[at];
            } else {
                for (uint32_t e = 0; row + e < a.rows; ++e) to[e] = reinterpret_cast<const O *>(space)[at * EACH + e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Sums of KW wavefronts that have the same rows, added up in LDS in their order and handed to `store` (token tile, row tile, sum of the lane, value).
template <int MT, int R, int Q, int KW, typename F>
__device__ __forceinline__ void join_sums(float *parts, uint32_t wave, uint32_t lane, const float (&sum)[MT][R][Q], F store)
{
    constexpr int CELLS = MT * R * Q;
    if constexpr (KW == 1) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int q = 0; q < Q; ++q) store(m, r, q, sum[m][r][q]);
    } else {
        __syncthreads();
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int q = 0; q < Q; ++q) parts[(wave * CELLS + (m * R + r) * Q + q) * 64 + lane] = sum[m][r][q];
        __syncthreads();
        const uint32_t kw = wave % KW;
        for (uint32_t cell = kw; cell < CELLS; cell += KW) {
            const float *p = parts + ((wave - kw) * CELLS + cell) * 64 + lane;
            float v = *p;
#pragma unroll
            for (int o = 1; o < KW; ++o) v += p[o * CELLS * 64];
            store(cell / Q / R, cell / Q % R, cell % Q, v);
        }
    }
}

// Eight activations of a row from column k on, zeros behind the last one.  Where rows are staged whole, with few of them ragged (28672 x 8192, one token: 19.0 us,
// with eight_of_rest 19.8):
template <typename T>
__device__ __forceinline__ w4u eight_columns(const T *row, size_t k, uint32_t cols)
{
    typedef w4u WA __attribute__((aligned(2)));
    if (k + 8 <= cols) return *reinterpret_cast<const WA *>(row + k);
    if (k >= cols) return w4u{0, 0, 0, 0};
    return last_eight(row, k, cols);
}

// In the last chunk: of a ragged end the row's last eight, moved down, so that a thread's loads need no branch and go out together (17 tokens, 1000 x 777: 6.9 us;
// with a branch around each 7.5).
template <typename T>
__device__ __forceinline__ w4u eight_of_rest(const T *row, size_t k, uint32_t cols)
{
    typedef w4u WA __attribute__((aligned(2)));
    if (cols < 8) return k < cols ? last_eight(row, k, cols) : w4u{0, 0, 0, 0};
    const size_t from = k + 8 <= cols ? k : cols - 8, past = k - from;
    return moved_down(*reinterpret_cast<const WA *>(row + from), past);
}

constexpr uint32_t kRowPad = 16;  // bytes between the rows of activations in LDS, so that 16 rows' pieces lie in different banks

// Up to 4 Q tokens whose rows fit LDS: staged once, and no wavefront waits for another until the end.  A workgroup has a row tile, its
// wavefronts every KW-th column tile of it, D of them in flight.
// 28672 x 8192 weights, group 128, one token: 19.4 us, 6.2 TB/s, what loads alone reach; 4096 x 4096, group 32: 3.3 us in a graph (kernel start and end, three
// round trips to memory).  With activations staged in chunks, as below, 21.5 and 4.0.  With more tokens every workgroup stages more than its weights.
template <typename T, int GROUP, int Q, int KW, int D>
__global__ __launch_bounds__(KW * 64, 4) void k_weights_product_few(ProductArgs a)
{
    constexpr uint32_t WG = KW * 64;
    extern __shared__ __align__(16) char lds[];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t stride = a.col_tiles * 2 * kTileCols + kRowPad;
    const TileSource<GROUP, 1> source(a, blockIdx.x);
    auto inside = [&](uint32_t ct) { return ct < a.col_tiles ? ct : a.col_tiles - 1; };
    TileWords<GROUP, 1> t[D];
    const uint32_t per = a.col_tiles * (kTileCols / 8), pieces = a.tokens * per;
    auto load = [&](uint32_t i) { return eight_columns(static_cast<const T *>(a.x) + (i / per) * a.x_stride, (size_t)(i % per) * 8, a.cols); };
    auto place = [&](uint32_t i, w4u v) { *reinterpret_cast<w4u *>(lds + i / per * stride + i % per * 16) = v; };
    uint32_t i = threadIdx.x;
    w4u one = {0, 0, 0, 0};
    if (i < pieces) one = load(i);
#pragma unroll
    for (int d = 0; d < D; ++d) source.fetch(inside(wave + d * KW), lane, t[d]);
    if (i < pieces) place(i, one);
    for (i += WG; i < pieces; i += WG) place(i, load(i));
    float sum[1][1][Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) sum[0][0][q] = 0.0f;
    uint32_t token = n / (4 / Q);
    token = token < a.tokens ? token : a.tokens - 1;
    const char *x = lds + token * stride + g * 16;
    const uint32_t step[4] = {0, 64, 128, 192};
    __syncthreads();
    for (uint32_t ct = wave; ct < a.col_tiles; ct += D * KW) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const uint32_t now = ct + d * KW;
            if (now < a.col_tiles) add_tile<T, GROUP, 1, Q, 1, 0>(x + now * 2 * kTileCols, step, t[d], sum);
            source.fetch(inside(now + D * KW), lane, t[d]);  // (without a condition: a branch around loads makes the waits for others wait for all)
        }
    }
    join_sums<1, 1, Q, KW>(reinterpret_cast<float *>(lds), wave, lane, sum, [&](uint32_t, uint32_t, uint32_t q, float v) {
        const uint32_t to = blockIdx.x * kTileRows + n, m = g * Q + q;
        if (to < a.rows && m < a.tokens) store_result<T>(a, m, to, v);
    });
}

// Any number of tokens, 4 Q MT of them in a workgroup (grid y), RW R row tiles (from LEAST R on, by the launch); the column tiles are cut into chunks of KW, a wavefront has one tile of a chunk
// of R row tiles.  A chunk of the activations is staged in LDS for all wavefronts, one ahead of its use, and D more chunks of activations and
// weights are on their way to registers: both by the same distance, for loads are waited for in the order of their issue.  What a
// compute unit gets from L2 is about 25 bytes a cycle, of HBM's weights 12: with few row tiles in a workgroup, activations cost more than weights.
// With `parts` (workspace) the chunks are divided over the workgroups of grid z as well, and k_weights_join adds up their sums.
// 50021 x 4096, 13 tokens: 22 us of 16.5 that its bytes take (weights' loads alone 18.8); 4096 x 14336, 20 tokens over four splits: 10.5 us
// (chunks one after the other: a barrier, LDS, four dependent matrix instructions) and 3 of the join; 8192 x 4096, 500 tokens: 40.4 us, 830 TFLOP/s (matrix and
// vector instructions of two wavefronts a SIMD in turn; 32 us without loads).
struct SplitArgs {
    float *parts;  // [splits][tokens][rows]
    uint32_t splits;
    uint32_t each = 0, more = 0;  // whole chunks of a split, one more in the first `more`
};

template <typename T, int GROUP, int MT, int Q, int R, int RW, int KW, int D, int OCC, int LEAST = RW>
__global__ __launch_bounds__(RW * KW * 64, OCC) void k_weights_product(ProductArgs a, SplitArgs split)
{
    constexpr uint32_t TOKENS = 4 * Q * MT, COLS = KW * kTileCols, STRIDE = 2 * COLS;
    constexpr uint32_t PIECES = TOKENS * STRIDE / 16, FEWEST = LEAST * KW * 64, MINE = (PIECES + FEWEST - 1) / FEWEST;
    const uint32_t WG = LEAST == RW ? RW * KW * 64 : blockDim.x, rw = LEAST == RW ? RW : WG / (KW * 64);
    constexpr uint32_t STAGED = 2 * TOKENS * STRIDE, JOINED = KW > 1 ? RW * KW * MT * R * Q * 256 : 0;
    __shared__ __align__(16) char lds[STAGED > JOINED ? STAGED : JOINED];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t kw = wave % KW, row_tile = (blockIdx.x * rw + wave / KW) * R, first = blockIdx.y * TOKENS;
    // this workgroup's whole chunks; the last one has the columns behind them too
    const uint32_t whole = a.cols / COLS, z = blockIdx.z, c0 = z * split.each + (z < split.more ? z : split.more), c1 = c0 + split.each + (z < split.more ? 1 : 0);
    const bool rest = whole * COLS < a.cols && blockIdx.z == split.splits - 1;
    const TileSource<GROUP, R> source(a, row_tile);
    float sum[MT][R][Q];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[m][r][q] = 0.0f;
    // Of a row's pieces in LDS every 16 change places by the row: rows lie 256 bytes or a multiple apart, and the 16 lanes that are served together are of all the
    // rows of a token tile, some with one g and the others with the next, so that each finds banks of its own (with rows 16 bytes further apart instead 38 to 46 % of the LDS
    // cycles were conflicts; 64 tokens, 28672 x 8192 49 -> 46.5 us, 512 tokens, 8192 x 8192 81 -> 78).
    auto turn = [](uint32_t row) { return row * (4 / Q) & 15; };
    // a thread's pieces of a chunk: 16 bytes of a token (behind the last one: of the last one again; nobody looks at its results)
    const T *from[MINE];
    uint32_t to[MINE];
#pragma unroll
    for (uint32_t i = 0; i < MINE; ++i) {
        const uint32_t at = threadIdx.x + i * WG, m = at / (STRIDE / 16) % TOKENS, c = at % (STRIDE / 16), token = first + m < a.tokens ? first + m : a.tokens - 1;
        from[i] = static_cast<const T *>(a.x) + token * a.x_stride + c * 8;
        to[i] = m * STRIDE + (c ^ turn(m)) * 16;
    }
    struct Pieces {
        w4u v[MINE];
    };
    auto fetch_x = [&](uint32_t chunk, Pieces &p) {
        typedef w4u WA __attribute__((aligned(2)));
#pragma unroll
        for (uint32_t i = 0; i < MINE; ++i) p.v[i] = *reinterpret_cast<const WA *>(from[i] + (size_t)chunk * COLS);
    };
    auto place_x = [&](uint32_t buffer, const Pieces &p) {
#pragma unroll
        for (uint32_t i = 0; i < MINE; ++i)
            if ((LEAST == RW && PIECES % FEWEST == 0) || threadIdx.x + i * WG < PIECES) *reinterpret_cast<w4u *>(lds + buffer * TOKENS * STRIDE + to[i]) = p.v[i];
    };
    uint32_t step[4];
#pragma unroll
    for (uint32_t s = 0; s < 4; ++s) step[s] = n / (4 / Q) * STRIDE + kw * 2 * kTileCols + ((4 * s + g) ^ turn(n / (4 / Q))) * 16;
    auto work = [&](const TileWords<GROUP, R> &t, uint32_t buffer) { add_tile<T, GROUP, MT, Q, R, 4 * Q * STRIDE>(lds + buffer * TOKENS * STRIDE, step, t, sum); };

    TileWords<GROUP, R> t_rest = {};
    Pieces x_rest = {};
    if (rest) {
        if (whole * KW + kw < a.col_tiles) source.fetch(whole * KW + kw, lane, t_rest);
#pragma unroll
        for (uint32_t i = 0; i < MINE; ++i) {
            const uint32_t c = (threadIdx.x + i * WG) % (STRIDE / 16) * 8;
            x_rest.v[i] = eight_of_rest(from[i] - c, (size_t)whole * COLS + c, a.cols);
        }
    }
    if (c1 > c0) {
        auto inside = [&](uint32_t c) { return c < c1 ? c : c1 - 1; };
        TileWords<GROUP, R> t[D];
        Pieces p[D];
#pragma unroll
        for (int d = 0; d < D; ++d) {
            fetch_x(inside(c0 + d), p[d]);
            source.fetch(inside(c0 + d) * KW + kw, lane, t[d]);
        }
        place_x(0, p[0]);
        fetch_x(inside(c0 + D), p[0]);
        static_assert(D % 2 == 0, "the two buffers in turn");
        for (uint32_t c = c0; c < c1; c += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                __syncthreads();  // chunk c + d is there, and nobody reads the one before any more
                place_x((d & 1) ^ 1, p[(d + 1) % D]);
                fetch_x(inside(c + d + 1 + D), p[(d + 1) % D]);
                if (c + d < c1) work(t[d], d & 1);
                source.fetch(inside(c + d + D) * KW + kw, lane, t[d]);
            }
        }
    }
    if (rest) {
        __syncthreads();
        place_x(0, x_rest);
        __syncthreads();
        if (whole * KW + kw < a.col_tiles) work(t_rest, 0);
    }
    if constexpr (KW == 1 && MT == 4) {
        static_assert(Q == 4 && RW * MT * 16 * 64 <= sizeof(lds), "LDS of a wavefront's results");
        __syncthreads();
        char *space = lds + wave * (MT * 16 * 64);
        if (a.wide)
            store_rows<T, float, MT, R>(a, space, lane, first, row_tile, sum);
        else
            store_rows<T, T, MT, R>(a, space, lane, first, row_tile, sum);
        return;
    }
    join_sums<MT, R, Q, KW>(reinterpret_cast<float *>(lds), wave, lane, sum, [&](uint32_t m, uint32_t r, uint32_t q, float v) {
        const uint32_t token = first + m * (4 * Q) + g * Q + q, row = (row_tile + r) * kTileRows + n;
        if (row >= a.rows || token >= a.tokens) return;
        if (split.splits > 1)
            split.parts[((size_t)blockIdx.z * a.tokens + token) * a.rows + row] = v;
        else
            store_result<T>(a, token, row, v);
    });
}

// The sums of the workgroups that share a chunk range, in their order.
template <typename T>
__global__ __launch_bounds__(256) void k_weights_join(ProductArgs a, SplitArgs split)
{
    const uint32_t row = blockIdx.x * 256 + threadIdx.x, token = blockIdx.y;
    if (row >= a.rows) return;
    const float *p = split.parts + (size_t)token * a.rows + row;
    float v = *p;
#pragma unroll 4
    for (uint32_t z = 1; z < split.splits; ++z) v += p[(size_t)z * a.tokens * a.rows];
    store_result<T>(a, token, row, v);
}

}  // namespace
