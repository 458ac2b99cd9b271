// dq8: weights in 4 bits (include/dq8_weights.h): checks of arguments and launches.  The kernels are in dq8_kernels_weights.hpp.
// Built with the flags of dq8.hip.
#include "dq8_weights.h"

#include "dq8_cache_check.hpp"
#include "dq8_kernels_weights.hpp"

namespace {

using dq8::failed;

// Grids of 256 lanes a row tile, or a tile in four, count their lanes in 32 bits.
constexpr size_t kRowLimit = ((size_t)1 << 28) - 16, kTileLimit = (size_t)1 << 25;

size_t size_of(int type) { return type == DQ8_FLOAT32 ? 4 : 2; }

struct Tiles {
    size_t rows, cols, all;
};

Tiles tiles_of(const dq8_weights &w)
{
    Tiles t;
    t.rows = (w.rows + kTileRows - 1) / kTileRows, t.cols = (w.cols + kTileCols - 1) / kTileCols;
    t.all = t.rows * t.cols;
    return t;
}

size_t code_bytes(const dq8_weights &w) { return tiles_of(w).all * kTileBytes; }
size_t scale_bytes(const dq8_weights &w) { return tiles_of(w).all * kTileRows * (kTileCols / (size_t)w.group) * 2; }

// 0 rows or columns pass: such weights have no tiles.
int check_weights(const char *who, const dq8_weights *w)
{
    if (!w) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if (w->group != 32 && w->group != 64 && w->group != 128) return failed(DQ8_ERR_ARG, "%s: group %d is not 32, 64 or 128", who, w->group);
    if (w->rows > kRowLimit || w->cols >= dq8::kCacheLimit || tiles_of(*w).all >= kTileLimit)
        return failed(DQ8_ERR_ARG, "%s: %zu x %zu weights are too many", who, w->rows, w->cols);
    if (w->rows == 0 || w->cols == 0) return DQ8_OK;
    if (!w->codes || !w->scales) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if (((uintptr_t)w->codes & 15) != 0 || ((uintptr_t)w->scales & 7) != 0)
        return failed(DQ8_ERR_ARG, "%s: codes must start at a multiple of 16 bytes, scales of 8", who);
    if (dq8::meet(w->codes, code_bytes(*w), w->scales, scale_bytes(*w))) return failed(DQ8_ERR_ARG, "%s: codes and scales overlap", who);
    return DQ8_OK;
}

// A matrix of `type` beside the weights.
int check_matrix(const char *who, const char *what, const dq8_weights &w, int type, const void *p, size_t rows, size_t cols, size_t stride, bool written)
{
    if (!p) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if (((uintptr_t)p & (size_of(type) - 1)) != 0) return failed(DQ8_ERR_ARG, "%s: %s does not start at a multiple of its element's size", who, what);
    if (!dq8::sane(stride, rows)) return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
    const size_t bytes = dq8::extent(rows, stride, 1, 0, 0, size_of(type)) + cols * size_of(type);
    if (written && rows > 1 && stride < cols) return failed(DQ8_ERR_ARG, "%s: rows of %s overlap", who, what);
    if (dq8::meet(p, bytes, w.codes, code_bytes(w)) || dq8::meet(p, bytes, w.scales, scale_bytes(w)))
        return failed(DQ8_ERR_ARG, "%s: %s overlaps codes or scales", who, what);
    return DQ8_OK;
}

bool known(int type) { return type == DQ8_FLOAT32 || type == DQ8_BFLOAT16 || type == DQ8_FLOAT16; }

template <typename T, int GROUP>
int encode(const void *w, size_t stride, const dq8_weights &o, hipStream_t stream)
{
    const Tiles t = tiles_of(o);
    hipLaunchKernelGGL((k_weights_encode<T, GROUP>), dim3((unsigned)((t.all + 3) / 4)), dim3(256), 0, stream, static_cast<const T *>(w), stride, o.rows, o.cols,
                       (uint32_t)t.cols, t.all, o.codes, static_cast<uint16_t *>(o.scales));
    return dq8::after_launch_of("k_weights_encode", stream);
}

template <typename T, int GROUP>
int decode(const dq8_weights &o, void *w, size_t stride, hipStream_t stream)
{
    const Tiles t = tiles_of(o);
    hipLaunchKernelGGL((k_weights_decode<T, GROUP>), dim3((unsigned)((t.all + 3) / 4)), dim3(256), 0, stream, o.codes, static_cast<const uint16_t *>(o.scales), o.rows,
                       o.cols, (uint32_t)t.cols, t.all, static_cast<T *>(w), stride);
    return dq8::after_launch_of("k_weights_decode", stream);
}

template <typename T>
int encode(const void *w, size_t stride, const dq8_weights &o, hipStream_t stream)
{
    return o.group == 32 ? encode<T, 32>(w, stride, o, stream) : o.group == 64 ? encode<T, 64>(w, stride, o, stream) : encode<T, 128>(w, stride, o, stream);
}

template <typename T>
int decode(const dq8_weights &o, void *w, size_t stride, hipStream_t stream)
{
    return o.group == 32 ? decode<T, 32>(o, w, stride, stream) : o.group == 64 ? decode<T, 64>(o, w, stride, stream) : decode<T, 128>(o, w, stride, stream);
}

// What a product launches.  The number behind a name: row tiles of a workgroup; with 7 and 13 the most.
enum Form {
    kFew16, kFew8, kFew4,          // one token or two, whole rows of activations staged; 16, 8, 4 wavefronts along the columns
    kToken4x1, kToken4x2, kToken4x3, kToken4x2Short, kToken4x7, kToken4x13,  // in chunks: up to 4 tokens; 8, 4, 4, 2, 2, 1 wavefronts along the columns
    kToken8x1, kToken8x2, kToken8x3, kToken8x4, kToken8x7, kToken8x13,       // up to 8; 8, 4, 4, 2, 2, 1
    kToken16x1, kToken16x2, kToken16x3, kToken16x4, kToken16x7, kToken16x13,  // up to 16; 8, 4, 4, 2, 2, 1
    kToken32x2, kToken32x4, kToken32x4Deep, kToken32x8, kToken32x13,  // 32 a workgroup; 4, 2, 2 (with more loads ahead), 1, 1
    kToken64x4, kToken64x8, kToken64x16, kToken64x32              // 64 a workgroup; 2, 1, 1, 1
};

struct Shape {
    Form form;
    unsigned row_tiles;  // of a workgroup
    unsigned columns;    // of a chunk
    unsigned splits;     // workgroups along the columns, where there is workspace for their sums
};

constexpr size_t kFewBytes = 65536;  // of LDS, for whole rows; half of it where workgroups share a compute unit

// With few row tiles wavefronts share one, or compute units stay idle; with many a workgroup has several, for it reads its tokens' activations once for all
// of them.  us, groups of 32, bfloat16 (in parentheses with other forms):
//   1 token, 4096 x 8192 kFew16 5.7 (kFew8 6.2), 8192 x 4096 kFew8 5.4 (kFew16 5.9), 28672 x 8192 kFew4 21.6 (kFew8 22.5, in chunks 22.7), 14336 x 14336 20.5 (21.3),
//   4096 x 28672 kFew16 12.8 (14.6); in chunks 8192 x 28672 21.4 (kFew8 23.3), 20000 x 28672 59 (kFew4 62); 2 tokens, 4096 x 4096 kFew16 4.3 (in chunks 4.5), in
//   chunks 28672 x 8192 24.7 (kFew4 27.8), 8192 x 14336 12.3 (kFew8 14.3);
//   4 tokens, 4096 x 8192 kToken4x1 6.8 (kToken4x2 8.2), 8192 x 8192 kToken4x2 9.0 (10.1, kToken4x2Short 10.7, whole rows staged 9.9), 28672 x 8192
//   kToken4x7 26.4 (kToken4x2Short 27.7), 50016 x 4096 kToken4x13 22.5 (23.4);
//   8 tokens, 4096 x 4096 kToken8x1 5.1 (kToken8x2 6.1), 28672 x 8192 kToken8x7 26.5 (kToken8x4 28), 50016 x 4096 kToken8x13 22.9 (26.8);
//   13 tokens, 4096 x 4096 kToken16x1 6.4 (kToken16x2 6.5), 8192 x 8192 kToken16x2 10.4 (kToken16x4 14), 14336 x 4096 kToken16x4 10.2 (kToken16x7 with 7 row tiles 11.8),
//   20480 x 4096 kToken16x7 with 5 13.0 (kToken16x4 16.2), 32000 x 4096 with 4 15.7 (8 16.6), 50021 x 4096 kToken16x13 23.7 (workgroups of 8 row tiles 26.1);
//   32 tokens, 8192 x 4096 kToken32x2 9.9 (kToken32x4 11.8), 16384 x 4096 kToken32x4Deep 13.1 (kToken32x8 22), 14336 x 8192 20.2 (kToken32x4 21.0), 50016 x 4096
//   kToken32x13 28.3 (kToken32x8 32, kToken32x4Deep 42), 128256 x 4096 kToken32x8 67.5 (kToken32x13 73);
//   64 tokens, 4096 x 4096 kToken32x2 9.3 (kToken32x4 11.5, kToken64x4 16.8), 8192 x 8192 kToken32x4 19.8 (kToken32x2 26.6, kToken64x4 28.7): two workgroups that
//   read the same weights cost less than one whose chunks take twice as long; 96 tokens, 6144 x 8192 kToken64x4 28.8 (kToken32x4 29.4), 2048 columns 10.8 (11.1).
// A workgroup of 7 or 13 row tiles at most gets as many as make all of a turn alike: some compute units with two and others with one cost what they idle.  (So do three
// row tiles where there are up to three for each compute unit: 7 tokens, 9944 x 23552 kToken8x3 27.7 (kToken8x4 33, kToken8x2 35), 13 tokens 30.3 (38.6, 42), 4 tokens
// 27.1 (kToken4x2Short 33.7); 7 tokens, 11008 x 4096 7.9 (8.5).)
// Where kToken32x2 leaves half the compute units idle, columns from 6144 on are divided, and from 12288 on for kToken32x4: 32 tokens, 4096 x 8192 over two splits
// 11.7 (one 13.3; kToken32x4 over four 11.4), 4096 x 4096 9.3 (8.6); 2048 x 8192 over four 9.7 (two 10.8, one 12.8); 4096 x 14336 kToken32x4 over four 15.3 (kToken32x2
// over two 16.0), 2048 x 28672 over eight 15.6 (over four 16.4).  Of 9 to 16 tokens those from 12288 on, for kToken16x4: 4096 x 14336 over four 13.6 (kToken16x1 14.5),
// 8192 x 14336 over two 17.2 (kToken16x2 19.7), 1024 x 28672 over eight 12.4 (kToken16x1 23.3); 4096 x 8192 10.5 (kToken16x1 9.9).
// From there on what counts is how often the compute units take a workgroup: with 2048 columns kToken64x8 takes 12.5 us a turn and 4.5 once, kToken64x16 24.5 a
// turn, kToken64x32 43 (groups of 128: 12, 21, 39), and the form whose turns cost least runs: 500 tokens, 8192 rows one turn of kToken64x16 27.6 (two of kToken64x8
// 28.3, half a one of kToken64x32 42); 700 tokens, 8192 rows kToken64x8 38.7 (kToken64x16 48.5, kToken64x32 42.5); 300, 14336 kToken64x8 37.9 (45.9, 42.1); 200, 28672
// kToken64x32 43.7 (49.8, 49.3); 1500, 8192 kToken64x16 72.5 (73, kToken64x32 83); 2048, 28672 kToken64x32 306 (380, 347); 1024, 28672 x 8192 551 (kToken64x16 597).
// split: whether there is workspace for divided columns.
Shape shape_of(const dq8_weights &w, size_t tokens, int cus_, bool split)
{
    const size_t cus = (size_t)cus_, rows = tiles_of(w).rows, blocks = (tokens + 63) / 64, blocks32 = (tokens + 31) / 32;
    const size_t pairs = (rows + 1) / 2 * blocks32, fours = (rows + 3) / 4 * blocks32;
    const bool divide = split && (tokens > 16 ? pairs <= cus / 2 && w.cols >= 6144 : tokens > 8 && fours <= cus / 2 && w.cols >= 12288);
    auto turns = [&](size_t tiles) { return ((rows + tiles - 1) / tiles * blocks + cus - 1) / cus; };
    // row tiles of a workgroup, so that all workgroups of a turn have as many: at most `most` of them
    auto even = [&](size_t most) {
        const size_t turn = cus * ((rows + most * cus - 1) / (most * cus));
        return (unsigned)((rows + turn - 1) / turn);
    };
    Shape s;
    const size_t whole = tokens * (tiles_of(w).cols * 2 * kTileCols + kRowPad);
    if (rows <= cus ? tokens <= 2 && whole <= kFewBytes : tokens == 1 && whole <= kFewBytes / 2)
        s = rows <= cus ? Shape{kFew16, 1, 0, 1} : rows <= 4 * cus ? Shape{kFew8, 1, 0, 1} : Shape{kFew4, 1, 0, 1};
    else if (tokens <= 4)
        s = rows <= cus       ? Shape{kToken4x1, 1, 1024, 1}
            : rows <= 2 * cus ? Shape{kToken4x2, 2, 512, 1}
            : rows <= 3 * cus ? Shape{kToken4x3, 3, 512, 1}
            : rows <= 4 * cus ? Shape{kToken4x2Short, 2, 256, 1}
            : rows <= 8 * cus ? Shape{kToken4x7, even(7), 256, 1}
                              : Shape{kToken4x13, even(13), 128, 1};
    else if (tokens <= 8)
        s = rows <= cus       ? Shape{kToken8x1, 1, 1024, 1}
            : rows <= 2 * cus ? Shape{kToken8x2, 2, 512, 1}
            : rows <= 3 * cus ? Shape{kToken8x3, 3, 512, 1}
            : rows <= 4 * cus ? Shape{kToken8x4, 4, 256, 1}
            : rows <= 8 * cus ? Shape{kToken8x7, even(7), 256, 1}
                              : Shape{kToken8x13, even(13), 128, 1};
    else if (tokens <= 16)
        s = divide            ? Shape{kToken16x4, 4, 256, 1}
            : rows <= cus     ? Shape{kToken16x1, 1, 1024, 1}
            : rows <= 2 * cus ? Shape{kToken16x2, 2, 512, 1}
            : rows <= 3 * cus ? Shape{kToken16x3, 3, 512, 1}
            : rows <= 4 * cus ? Shape{kToken16x4, 4, 256, 1}
            : rows <= 8 * cus ? Shape{kToken16x7, even(7), 256, 1}
                              : Shape{kToken16x13, even(13), 128, 1};
    else if (pairs <= cus)
        s = divide && w.cols >= 12288 ? Shape{kToken32x4, 4, 256, 1} : Shape{kToken32x2, 2, 512, 1};
    else if (tokens <= 32)
        s = rows <= 4 * cus                      ? Shape{kToken32x4Deep, 4, 256, 1}
            : rows <= 8 * cus || rows > 13 * cus ? Shape{kToken32x8, 8, 128, 1}
                                                 : Shape{kToken32x13, even(13), 128, 1};
    else if (fours <= cus)
        s = Shape{kToken32x4, 4, 256, 1};
    else if ((rows + 3) / 4 * blocks <= cus)
        s = Shape{kToken64x4, 4, 256, 1};
    else {
        const size_t t8 = 25 * turns(8) + 9, t16 = 49 * turns(16), t32 = 85 * turns(32);
        s = t32 <= t16 && t32 <= t8 ? Shape{kToken64x32, 32, 128, 1} : t16 <= t8 ? Shape{kToken64x16, 16, 128, 1} : Shape{kToken64x8, 8, 128, 1};
    }
    if (divide) {
        const size_t idle = cus / ((rows + s.row_tiles - 1) / s.row_tiles * blocks32), most = w.cols / 1024;
        s.splits = (unsigned)(idle < most ? idle : most);
    }
    return s;
}

size_t workspace_of(const dq8_weights &w, size_t tokens, const Shape &s) { return s.splits > 1 ? s.splits * tokens * w.rows * sizeof(float) : 0; }

template <typename T, int GROUP, int Q, int KW, int D>
int few(const ProductArgs &k, hipStream_t stream)
{
    const size_t x = k.tokens * ((size_t)k.col_tiles * 2 * kTileCols + kRowPad), sums = KW * Q * 256;
    hipLaunchKernelGGL((k_weights_product_few<T, GROUP, Q, KW, D>), dim3(k.row_tiles), dim3(KW * 64), x > sums ? x : sums, stream, k);
    return dq8::after_launch_of("k_weights_product_few", stream);
}

template <typename T, int GROUP, int MT, int Q, int R, int RW, int KW, int D, int OCC, int LEAST = RW>
int chunks(const ProductArgs &k, uint32_t row_tiles, const SplitArgs &split, hipStream_t stream)
{
    constexpr uint32_t TOKENS = 4 * Q * MT;
    hipLaunchKernelGGL((k_weights_product<T, GROUP, MT, Q, R, RW, KW, D, OCC, LEAST>),
                       dim3((k.row_tiles + row_tiles - 1) / row_tiles, (k.tokens + TOKENS - 1) / TOKENS, split.splits), dim3(row_tiles / R * KW * 64), 0, stream, k, split);
    const int rc = dq8::after_launch_of("k_weights_product", stream);
    if (rc || split.splits == 1) return rc;
    hipLaunchKernelGGL(k_weights_join<T>, dim3((k.rows + 255) / 256, k.tokens), dim3(256), 0, stream, k, split);
    return dq8::after_launch_of("k_weights_join", stream);
}

template <typename T, int GROUP>
int product(const ProductArgs &k, const Shape &s, const SplitArgs &split, hipStream_t stream)
{
    const uint32_t n = s.row_tiles;
    switch (s.form) {
    case kFew16: return few<T, GROUP, 1, 16, 2>(k, stream);
    case kFew8: return few<T, GROUP, 1, 8, 2>(k, stream);
    case kFew4: return few<T, GROUP, 1, 4, 4>(k, stream);
    case kToken4x1: return chunks<T, GROUP, 1, 1, 1, 1, 8, 2, 4>(k, n, split, stream);
    case kToken4x2: return chunks<T, GROUP, 1, 1, 1, 2, 4, 4, 4>(k, n, split, stream);
    case kToken4x3: return chunks<T, GROUP, 1, 1, 1, 3, 4, 2, 4>(k, n, split, stream);
    case kToken4x2Short: return chunks<T, GROUP, 1, 1, 1, 2, 2, 4, 4>(k, n, split, stream);
    case kToken4x7: return chunks<T, GROUP, 1, 1, 1, 7, 2, 2, 4, 4>(k, n, split, stream);
    case kToken4x13: return chunks<T, GROUP, 1, 1, 1, 13, 1, 2, 4, 7>(k, n, split, stream);
    case kToken8x1: return chunks<T, GROUP, 1, 2, 1, 1, 8, 2, 4>(k, n, split, stream);
    case kToken8x2: return chunks<T, GROUP, 1, 2, 1, 2, 4, 4, 4>(k, n, split, stream);
    case kToken8x3: return chunks<T, GROUP, 1, 2, 1, 3, 4, 2, 4>(k, n, split, stream);
    case kToken8x4: return chunks<T, GROUP, 1, 2, 1, 4, 2, 4, 4>(k, n, split, stream);
    case kToken8x7: return chunks<T, GROUP, 1, 2, 1, 7, 2, 2, 4, 4>(k, n, split, stream);
    case kToken8x13: return chunks<T, GROUP, 1, 2, 1, 13, 1, 2, 4, 7>(k, n, split, stream);
    case kToken16x1: return chunks<T, GROUP, 1, 4, 1, 1, 8, 2, 4>(k, n, split, stream);
    case kToken16x2: return chunks<T, GROUP, 1, 4, 1, 2, 4, 2, 4>(k, n, split, stream);
    case kToken16x3: return chunks<T, GROUP, 1, 4, 1, 3, 4, 2, 4>(k, n, split, stream);
    case kToken16x4: return chunks<T, GROUP, 1, 4, 1, 4, 2, 4, 5>(k, n, split, stream);
    case kToken16x7: return chunks<T, GROUP, 1, 4, 1, 7, 2, 2, 4, 4>(k, n, split, stream);
    case kToken16x13: return chunks<T, GROUP, 1, 4, 1, 13, 1, 2, 4, 7>(k, n, split, stream);
    case kToken32x2: return chunks<T, GROUP, 2, 4, 1, 2, 4, 2, 4>(k, n, split, stream);
    case kToken32x4: return chunks<T, GROUP, 2, 4, 1, 4, 2, 2, 4>(k, n, split, stream);
    case kToken32x4Deep: return chunks<T, GROUP, 2, 4, 1, 4, 2, 4, 2>(k, n, split, stream);
    case kToken32x8: return chunks<T, GROUP, 2, 4, 1, 8, 1, 4, 2>(k, n, split, stream);
    case kToken32x13: return chunks<T, GROUP, 2, 4, 1, 13, 1, 2, 4, 8>(k, n, split, stream);
    case kToken64x4: return chunks<T, GROUP, 4, 4, 1, 4, 2, 2, 2>(k, n, split, stream);
    case kToken64x8: return chunks<T, GROUP, 4, 4, 1, 8, 1, 2, 2>(k, n, split, stream);
    case kToken64x16: return chunks<T, GROUP, 4, 4, 2, 8, 1, 2, 1>(k, n, split, stream);
    case kToken64x32: return chunks<T, GROUP, 4, 4, 4, 8, 1, 2, 1>(k, n, split, stream);
    }
    return DQ8_OK;
}

template <typename T>
int product(int group, const ProductArgs &k, const Shape &s, const SplitArgs &split, hipStream_t stream)
{
    return group == 32 ? product<T, 32>(k, s, split, stream) : group == 64 ? product<T, 64>(k, s, split, stream) : product<T, 128>(k, s, split, stream);
}

// What looks at sizes and types.  No tokens or rows pass: such a call launches nothing.
int check_product(const char *who, const dq8_weights *w, const dq8_product *in)
{
    const int rc = check_weights(who, w);
    if (rc) return rc;
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_product &p = *in;
    if (p.type != DQ8_BFLOAT16 && p.type != DQ8_FLOAT16) return failed(DQ8_ERR_ARG, "%s: type %d is neither bfloat16 nor float16", who, p.type);
    if (p.out_type != p.type && p.out_type != DQ8_FLOAT32) return failed(DQ8_ERR_ARG, "%s: out_type %d is neither type nor float32", who, p.out_type);
    if (p.tokens > DQ8_WEIGHTS_MAX_TOKENS) return failed(DQ8_ERR_ARG, "%s: %zu tokens", who, p.tokens);
    if (w->rows && p.tokens && w->cols == 0) return failed(DQ8_ERR_ARG, "%s: weights without columns", who);
    return DQ8_OK;
}

}  // namespace

extern "C" {

int dq8_weights_encode(int type, const void *w, size_t row_stride, const dq8_weights *out, void *hip_stream)
{
    static const char who[] = "dq8_weights_encode";
    if (!known(type)) return failed(DQ8_ERR_ARG, "%s: unknown type %d", who, type);
    int rc = check_weights(who, out);
    if (rc || out->rows == 0 || out->cols == 0) return rc;
    rc = check_matrix(who, "w", *out, type, w, out->rows, out->cols, row_stride, false);
    if (rc) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (type == DQ8_FLOAT32) return encode<float>(w, row_stride, *out, stream);
    return type == DQ8_BFLOAT16 ? encode<__bf16>(w, row_stride, *out, stream) : encode<_Float16>(w, row_stride, *out, stream);
}

int dq8_weights_decode(const dq8_weights *in, int type, void *w, size_t row_stride, void *hip_stream)
{
    static const char who[] = "dq8_weights_decode";
    if (!known(type)) return failed(DQ8_ERR_ARG, "%s: unknown type %d", who, type);
    int rc = check_weights(who, in);
    if (rc || in->rows == 0 || in->cols == 0) return rc;
    rc = check_matrix(who, "w", *in, type, w, in->rows, in->cols, row_stride, true);
    if (rc) return rc;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (type == DQ8_FLOAT32) return decode<float>(*in, w, row_stride, stream);
    return type == DQ8_BFLOAT16 ? decode<__bf16>(*in, w, row_stride, stream) : decode<_Float16>(*in, w, row_stride, stream);
}

size_t dq8_weights_product_workspace_bytes(const dq8_weights *w, const dq8_product *p)
{
    if (check_product("dq8_weights_product_workspace_bytes", w, p) || w->rows == 0 || p->tokens <= 8) return 0;
    dq8::DeviceTables dev;
    if (dq8::device_tables(0, &dev)) return 0;
    return workspace_of(*w, p->tokens, shape_of(*w, p->tokens, dev.cus, true));
}

int dq8_weights_product(const dq8_weights *w, const dq8_product *in, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    static const char who[] = "dq8_weights_product";
    int rc = check_product(who, w, in);
    if (rc) return rc;
    const dq8_product &p = *in;
    if (w->rows == 0 || p.tokens == 0) return DQ8_OK;
    rc = check_matrix(who, "x", *w, p.type, p.x, p.tokens, w->cols, p.x_stride, false);
    if (!rc) rc = check_matrix(who, "out", *w, p.out_type, p.out, p.tokens, w->rows, p.out_stride, true);
    if (rc) return rc;
    if (((uintptr_t)p.bias & 3) != 0 || ((uintptr_t)workspace & 15) != 0)
        return failed(DQ8_ERR_ARG, "%s: bias does not start at a multiple of 4 bytes or workspace of 16", who);
    const size_t n_out = ((p.tokens - 1) * p.out_stride + w->rows) * size_of(p.out_type), n_x = ((p.tokens - 1) * p.x_stride + w->cols) * 2;
    const size_t n_bias = p.bias ? w->rows * 4 : 0, n_work = workspace ? workspace_bytes : 0;
    using dq8::meet;
    if (meet(p.out, n_out, p.x, n_x) || meet(p.out, n_out, p.bias, n_bias) || meet(p.out, n_out, workspace, n_work) || meet(workspace, n_work, p.x, n_x) ||
        meet(workspace, n_work, p.bias, n_bias) || meet(workspace, n_work, w->codes, code_bytes(*w)) || meet(workspace, n_work, w->scales, scale_bytes(*w)))
        return failed(DQ8_ERR_ARG, "%s: out or workspace overlaps another array", who);
    dq8::DeviceTables dev;
    rc = dq8::device_tables(0, &dev);
    if (rc) return rc;
    const Tiles t = tiles_of(*w);
    ProductArgs k;
    k.codes = w->codes, k.scales = static_cast<const uint16_t *>(w->scales), k.x = p.x, k.out = p.out, k.bias = p.bias;
    k.x_stride = p.x_stride, k.out_stride = p.out_stride;
    k.tokens = (uint32_t)p.tokens, k.rows = (uint32_t)w->rows, k.cols = (uint32_t)w->cols, k.row_tiles = (uint32_t)t.rows, k.col_tiles = (uint32_t)t.cols;
    k.wide = p.out_type == DQ8_FLOAT32;
    Shape s = shape_of(*w, p.tokens, dev.cus, workspace != nullptr);
    if (workspace_bytes < workspace_of(*w, p.tokens, s)) s = shape_of(*w, p.tokens, dev.cus, false);
    SplitArgs split;
    split.parts = s.splits > 1 ? static_cast<float *>(workspace) : nullptr, split.splits = s.splits;
    if (s.columns) split.each = (uint32_t)(w->cols / s.columns / s.splits), split.more = (uint32_t)(w->cols / s.columns % s.splits);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return p.type == DQ8_BFLOAT16 ? product<__bf16>(w->group, k, s, split, stream) : product<_Float16>(w->group, k, s, split, stream);
}

}  // extern "C"
