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

// The nearest of eight magnitudes, the smaller of two as near, by comparisons with the borders between them times the scale.  These
// products have 3 + 8 bits: they are exact, and the comparison is one of real numbers.
struct Borders {
    float b[7];
    __device__ __forceinline__ explicit Borders(float s) : b{0.25f * s, 0.75f * s, 1.25f * s, 1.75f * s, 2.5f * s, 3.5f * s, 5.0f * s} {}
    __device__ __forceinline__ uint32_t code(float a) const
    {
        const bool c2 = a > b[3];
        const bool c1 = a > (c2 ? b[5] : b[1]);
        const bool c0 = a > (c2 ? (c1 ? b[6] : b[4]) : (c1 ? b[2] : b[0]));
        return (uint32_t)c2 * 4 + (uint32_t)c1 * 2 + (uint32_t)c0;
    }
};

// Eight elements of a row from column k on, zeros behind the last one.
template <typename T>
__device__ __forceinline__ void eight_of(const T *row, size_t k, size_t cols, float (&x)[8])
{
    typedef T V __attribute__((ext_vector_type(8)));
    typedef V VA __attribute__((aligned(sizeof(T))));
    if (k + 8 <= cols) {
        const V v = *reinterpret_cast<const VA *>(row + k);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e < cols ? (float)row[k + e] : 0.0f;
    }
}

// A wavefront per tile: lane 16 g + n has of row n the four runs of eight columns that its piece holds.
template <typename T, int GROUP>
__global__ __launch_bounds__(256) void k_weights_encode(const T *__restrict__ w, size_t stride, size_t rows, size_t cols, uint32_t col_tiles, size_t tiles,
                                                        uint8_t *__restrict__ codes, uint16_t *__restrict__ scales)
{
    constexpr int PER = kTileCols / GROUP, RUNS = 4 / PER;  // groups of a row in a tile; runs of a group
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const size_t tile = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const size_t rt = tile / col_tiles, ct = tile - rt * col_tiles, row = rt * kTileRows + n;
    float x[4][8];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        if (row < rows)
            eight_of(w + row * stride, ct * kTileCols + 32 * s + 8 * g, cols, x[s]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) x[s][e] = 0.0f;
    }
    uint32_t word[4], scale[PER];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        uint32_t most = 0;  // of the absolute values' bits: infinities and NaN are above all others
#pragma unroll
        for (int s = p * RUNS; s < (p + 1) * RUNS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = __float_as_uint(x[s][e]) & 0x7FFFFFFFu;
                most = b > most ? b : most;
            }
#pragma unroll
        for (int d = 16; d <= 32; d *= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)most, d);
            most = o > most ? o : most;
        }
        const bool bad = most >= 0x7F800000u;
        const float q = __uint_as_float(most) / 6.0f;
        const uint32_t bits = __float_as_uint(q);
        float s = bf16_value((bits + 0x7FFFu + ((bits >> 16) & 1)) >> 16);
        s = s < kScaleTop ? s : kScaleTop;
        scale[p] = bad ? 0x7FC0u : __float_as_uint(s) >> 16;
        const bool none = bad || s == 0.0f;
        const Borders borders(s);
#pragma unroll
        for (int r = p * RUNS; r < (p + 1) * RUNS; ++r) {
            uint32_t v = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) v |= (none ? 0u : borders.code(fabsf(x[r][e]))) << (4 * e) | (bad ? 0u : __float_as_uint(x[r][e]) >> 31) << (4 * e + 3);
            word[r] = v;
        }
    }
    *reinterpret_cast<w4u *>(codes + tile * kTileBytes + lane * 16) = w4u{word[0], word[1], word[2], word[3]};
    if (g == 0) {
#pragma unroll
        for (int p = 0; p < PER; ++p) scales[(tile * kTileRows + n) * PER + p] = (uint16_t)scale[p];
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

template <typename T, int GROUP>
__global__ __launch_bounds__(256) void k_weights_decode(const uint8_t *__restrict__ codes, const uint16_t *__restrict__ scales, size_t rows, size_t cols,
                                                        uint32_t col_tiles, size_t tiles, T *__restrict__ w, size_t stride)
{
    constexpr int PER = kTileCols / GROUP, RUNS = 4 / PER;
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const size_t tile = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (tile >= tiles) return;
    const size_t rt = tile / col_tiles, ct = tile - rt * col_tiles, row = rt * kTileRows + n;
    const w4u word = *reinterpret_cast<const w4u *>(codes + tile * kTileBytes + lane * 16);
    if (row >= rows) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float s = bf16_value(scales[(tile * kTileRows + n) * PER + r / RUNS]);
        float x[8];
        two_values<0>(word[r], x[0], x[1]);
        two_values<1>(word[r], x[2], x[3]);
        two_values<2>(word[r], x[4], x[5]);
        two_values<3>(word[r], x[6], x[7]);
        typedef T V __attribute__((ext_vector_type(8)));
        typedef V VA __attribute__((aligned(sizeof(T))));
        V v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (T)(x[e] * s);
        const size_t k = ct * kTileCols + 32 * r + 8 * g;
        T *to = w + row * stride + k;
        if (k + 8 <= cols) {
            *reinterpret_cast<VA *>(to) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
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

// A workgroup has R row tiles and 16 MT tokens; its wavefronts take every WAVES-th column tile and add up their sums in LDS at the end.
// The products have tokens as rows and weight rows as columns, so that a lane's four sums share the scale of its weight row.
template <typename T, int GROUP, int MT, int R, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_weights_product(ProductArgs a)
{
    constexpr int PER = kTileCols / GROUP, RUNS = 4 / PER;
    typedef Operand<T> Op;
    typedef typename Op::type V;
    typedef V VA __attribute__((aligned(sizeof(T))));
    __shared__ w4f parts[WAVES][MT * R][64];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = threadIdx.x >> 6;
    const uint32_t rt = blockIdx.x * R, first = blockIdx.y * 16 * MT;
    w4f sum[MT][R];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) sum[m][r] = w4f{0, 0, 0, 0};
    const T *row[MT];
    bool in[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const uint32_t token = first + 16 * m + n;
        in[m] = token < a.tokens;
        row[m] = static_cast<const T *>(a.x) + (in[m] ? token : 0) * a.x_stride;
    }
    for (uint32_t ct = wave; ct < a.col_tiles; ct += WAVES) {
        w4u word[R];
        uint32_t scale[R][PER];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const size_t tile = (size_t)(rt + r < a.row_tiles ? rt + r : rt) * a.col_tiles + ct;
            word[r] = *reinterpret_cast<const w4u *>(a.codes + tile * kTileBytes + lane * 16);
#pragma unroll
            for (int p = 0; p < PER; ++p) scale[r][p] = a.scales[(tile * kTileRows + n) * PER + p];
        }
        V x[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint32_t k = ct * kTileCols + 32 * s + 8 * g;
                x[m][s] = V{};
                if (in[m]) {
                    if (k + 8 <= a.cols) {
                        x[m][s] = *reinterpret_cast<const VA *>(row[m] + k);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (k + e < a.cols) x[m][s][e] = row[m][k + e];
                    }
                }
            }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                w4f d[MT];
#pragma unroll
                for (int m = 0; m < MT; ++m) d[m] = w4f{0, 0, 0, 0};
#pragma unroll
                for (int s = p * RUNS; s < (p + 1) * RUNS; ++s) {
                    const V v = Op::weights(word[r][s]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) d[m] = Op::product(x[m][s], v, d[m]);
                }
                const float f = bf16_value(scale[r][p]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[m][r][i] = __builtin_fmaf(d[m][i], f, sum[m][r][i]);
            }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) parts[wave][m * R + r][lane] = sum[m][r];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < MT * R * 64; i += WAVES * 64) {
        const uint32_t cell = i >> 6, m = cell / R, r = cell % R;
        w4f v = parts[0][cell][lane];
#pragma unroll
        for (int o = 1; o < WAVES; ++o) v += parts[o][cell][lane];
        v *= Op::kLift;
        const uint32_t to = (rt + r) * kTileRows + n;
        if (to >= a.rows) continue;
        if (a.bias) v += a.bias[to];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t token = first + 16 * m + 4 * g + e;
            if (token >= a.tokens) break;
            const size_t at = token * a.out_stride + to;
            if (a.wide)
                static_cast<float *>(a.out)[at] = v[e];
            else
                static_cast<T *>(a.out)[at] = (T)v[e];
        }
    }
}

}  // namespace
