// Argument checks that the calls for a cache of keys and values share (host code).
#pragma once
#include <cstddef>
#include <cstdint>

#include "dq8_cache.h"
#include "dq8_launch.hpp"

namespace dq8 {

constexpr size_t kCacheLimit = (size_t)1 << 31;  // of counts that kernels hold in 32 bits

inline int check_cache(const char *who, int kind, const dq8_cache *c)
{
    if (kind < 0 || kind > DQ8_MANTISSA) return failed(DQ8_ERR_KIND, "unknown data type %d", kind);
    if (!c || !c->codes || !c->scales) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if ((((uintptr_t)c->codes | (uintptr_t)c->scales) & 15) != 0)
        return failed(DQ8_ERR_ARG, "%s: codes and scales must start at a multiple of 16 bytes", who);
    if (c->dim < 16 || c->dim > DQ8_CACHE_MAX_DIM || c->dim % 16 != 0)
        return failed(DQ8_ERR_ARG, "%s: dim %d is not a multiple of 16 up to %d", who, c->dim, DQ8_CACHE_MAX_DIM);
    if (c->page_size < 16 || c->page_size > DQ8_CACHE_MAX_PAGE || (c->page_size & (c->page_size - 1)) != 0)
        return failed(DQ8_ERR_ARG, "%s: page_size %d is not a power of two from 16 to %d", who, c->page_size, DQ8_CACHE_MAX_PAGE);
    if (c->kv_heads < 1 || c->kv_heads > 65535) return failed(DQ8_ERR_ARG, "%s: %d cached heads", who, c->kv_heads);
    if (c->pages < 1 || c->pages >= kCacheLimit / (size_t)c->page_size || c->pages * (size_t)c->page_size >= ((size_t)1 << 50) / ((size_t)c->kv_heads * (size_t)c->dim))
        return failed(DQ8_ERR_ARG, "%s: %zu pages of %d", who, c->pages, c->page_size);
    if ((size_t)c->kv_heads * (size_t)c->page_size * (size_t)c->dim >= kCacheLimit) return failed(DQ8_ERR_ARG, "%s: a page of more than 2 GiB", who);
    return DQ8_OK;
}

// Bytes of the cache's two arrays.
inline size_t cache_rows(const dq8_cache *c) { return 2 * c->pages * (size_t)c->kv_heads * (size_t)c->page_size; }

// Bytes from the first to behind the last element of an array of rows.
inline size_t extent(size_t tokens, size_t token_stride, int heads, size_t head_stride, int dim, size_t size)
{
    return tokens == 0 || heads == 0 ? 0 : ((tokens - 1) * token_stride + (size_t)(heads - 1) * head_stride + (size_t)dim) * size;
}

// Strides of `count` tokens or heads over less than 2^56 elements, so that extents in bytes stay far inside 64 bits.
inline bool sane(size_t stride, size_t count) { return stride < (size_t)1 << 40 && (count < 2 || stride < ((size_t)1 << 56) / (count - 1)); }

// Whether no two rows of an array that is written overlap: all heads of a token lie before the next token's, or the other way round.
inline bool apart(size_t tokens, size_t token_stride, int heads, size_t head_stride, int dim)
{
    if (tokens == 0 || heads == 0) return true;
    const size_t t = tokens - 1, h = (size_t)heads - 1, d = (size_t)dim;
    return ((h == 0 || head_stride >= d) && (t == 0 || token_stride >= h * head_stride + d)) ||
           ((t == 0 || token_stride >= d) && (h == 0 || head_stride >= t * token_stride + d));
}

inline bool meet(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return na != 0 && nb != 0 && a0 < b0 + nb && b0 < a0 + na;
}

}  // namespace dq8
