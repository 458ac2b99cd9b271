// dq8: weights in 4 bits (include/dq8_weights.h): checks of arguments and launches.  The kernels are in dq8_kernels_weights.hpp.
// Built with the flags of dq8.hip.
#include "dq8_weights.h"

#include "dq8_cache_check.hpp"
#include "dq8_kernels_weights.hpp"

namespace {

using dq8::failed;

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
    if (w->rows >= dq8::kCacheLimit || w->cols >= dq8::kCacheLimit || tiles_of(*w).all >= dq8::kCacheLimit)
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

template <typename T, int GROUP, int MT, int R>
int product(const ProductArgs &k, hipStream_t stream)
{
    constexpr int WAVES = 8;
    hipLaunchKernelGGL((k_weights_product<T, GROUP, MT, R, WAVES>), dim3((k.row_tiles + R - 1) / R, (k.tokens + 16 * MT - 1) / (16 * MT)), dim3(WAVES * 64), 0, stream, k);
    return dq8::after_launch_of("k_weights_product", stream);
}

template <typename T, int GROUP>
int product(const ProductArgs &k, hipStream_t stream)
{
    if (k.tokens <= 16) return product<T, GROUP, 1, 1>(k, stream);
    if (k.tokens <= 32) return product<T, GROUP, 2, 1>(k, stream);
    return product<T, GROUP, 4, 2>(k, stream);
}

template <typename T>
int product(int group, const ProductArgs &k, hipStream_t stream)
{
    return group == 32 ? product<T, 32>(k, stream) : group == 64 ? product<T, 64>(k, stream) : product<T, 128>(k, stream);
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

int dq8_weights_product(const dq8_weights *w, const dq8_product *in, void *hip_stream)
{
    static const char who[] = "dq8_weights_product";
    int rc = check_weights(who, w);
    if (rc) return rc;
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_product &p = *in;
    if (p.type != DQ8_BFLOAT16 && p.type != DQ8_FLOAT16) return failed(DQ8_ERR_ARG, "%s: type %d is neither bfloat16 nor float16", who, p.type);
    if (p.out_type != p.type && p.out_type != DQ8_FLOAT32) return failed(DQ8_ERR_ARG, "%s: out_type %d is neither type nor float32", who, p.out_type);
    if (p.tokens > DQ8_WEIGHTS_MAX_TOKENS) return failed(DQ8_ERR_ARG, "%s: %zu tokens", who, p.tokens);
    if (w->rows == 0 || p.tokens == 0) return DQ8_OK;
    if (w->cols == 0) return failed(DQ8_ERR_ARG, "%s: weights without columns", who);
    rc = check_matrix(who, "x", *w, p.type, p.x, p.tokens, w->cols, p.x_stride, false);
    if (!rc) rc = check_matrix(who, "out", *w, p.out_type, p.out, p.tokens, w->rows, p.out_stride, true);
    if (rc) return rc;
    if (((uintptr_t)p.bias & 3) != 0) return failed(DQ8_ERR_ARG, "%s: bias does not start at a multiple of 4 bytes", who);
    const size_t n_out = ((p.tokens - 1) * p.out_stride + w->rows) * size_of(p.out_type), n_x = ((p.tokens - 1) * p.x_stride + w->cols) * 2;
    if (dq8::meet(p.out, n_out, p.x, n_x) || (p.bias && dq8::meet(p.out, n_out, p.bias, w->rows * 4))) return failed(DQ8_ERR_ARG, "%s: out overlaps x or bias", who);
    const Tiles t = tiles_of(*w);
    ProductArgs k;
    k.codes = w->codes, k.scales = static_cast<const uint16_t *>(w->scales), k.x = p.x, k.out = p.out, k.bias = p.bias;
    k.x_stride = p.x_stride, k.out_stride = p.out_stride;
    k.tokens = (uint32_t)p.tokens, k.rows = (uint32_t)w->rows, k.cols = (uint32_t)w->cols, k.row_tiles = (uint32_t)t.rows, k.col_tiles = (uint32_t)t.cols;
    k.wide = p.out_type == DQ8_FLOAT32;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return p.type == DQ8_BFLOAT16 ? product<__bf16>(w->group, k, stream) : product<_Float16>(w->group, k, stream);
}

}  // extern "C"
