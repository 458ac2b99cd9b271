/*
 * dq8 -- a paged cache of keys and values in the 8-bit types of dq8.h, and the attention that reads it.
 *
 * The rows of a transformer's keys and values are activations that are kept for as long as their sequence lives, and a decoding
 * step reads all of them.  Here a row (one token, one head, `dim` values) is one scale block of the codec: dim codes and one fp32
 * maximum.  dq8_cache_append compresses the rows of new tokens into the places that their slots name, with the norms and the rotation
 * that a model applies to keys and queries between its projection and its attention in the same pass; dq8_cache_attention reads
 * codes and scales and expands them in registers, so that a step moves one byte per cached element.
 *
 * Conventions (streams, device pointers, tables, error codes, DQ8_DEBUG, threads) are those of dq8.h.  The structs are HOST memory, read
 * before the call returns; the pointers in them are DEVICE pointers.  What the host cannot see -- slots, positions, page numbers,
 * lengths -- is checked by the kernels as described below; nothing outside the given arrays is read or written.
 */
#ifndef DQ8_CACHE_H
#define DQ8_CACHE_H

#include "dq8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of keys, values, queries and outputs. */
enum {
    DQ8_FLOAT32 = 0, /* dq8_cache_append only */
    DQ8_BFLOAT16 = 1,
    DQ8_FLOAT16 = 2
};

#define DQ8_CACHE_MAX_DIM 256
#define DQ8_CACHE_MAX_PAGE 1024

/*
 * The cache.  codes: [2][pages][kv_heads][page_size][dim] bytes, keys before values; scales: [2][pages][kv_heads][page_size] floats; both
 * at a multiple of 16 bytes.  dim: a multiple of 16 up to DQ8_CACHE_MAX_DIM; page_size: a power of two from 16 to
 * DQ8_CACHE_MAX_PAGE; kv_heads * page_size * dim below 2^31, pages * page_size too.  Slot s is place s % page_size of page s / page_size.  The row of token slot s and head h stands for
 * dq8_decode of its codes with its scale.
 */
typedef struct {
    uint8_t *codes;
    float *scales;
    size_t pages;
    int kv_heads, page_size, dim;
} dq8_cache;

/*
 * New tokens: k and v [tokens][kv_heads][dim], q [tokens][heads][dim], of one type; token t and head h of an array start
 * t * token_stride + h * head_stride elements after its pointer (parts of a fused projection's output, say), the elements of a
 * row lie side by side, and a pointer is a multiple of its element's size.
 * slots: the slot of every token; a token whose slot lies outside the cache is padding: nothing of it is stored.  A slot is
 * named at most once in a call (the rows of a slot named twice hold parts of either).
 * With q_weight / k_weight (dim floats), rows of q / k are normed: x_i / sqrt(mean of x^2 + eps) * weight_i.
 * With rotation ([n_positions][2][half] floats: cosines, then sines), pairs (a, b) of the first 2 * half elements become
 * (a cos - b sin, b cos + a sin) of the row positions[t]: elements (i, half + i), or (2 i, 2 i + 1) with `interleaved`.  A token whose
 * position lies outside the table is not stored, and its queries become NaN.
 * Keys: evaluated in binary64 from the given values, rounded once to binary32, then compressed as dq8_encode does with one scale
 * for the row.  (The order of the sum of squares shows in the last bits of binary64 only: codes and scales do not depend on it
 * but for a value that lies that close to a rounding border.)  Values: compressed as they are.  A row of keys or values that
 * holds an infinity or NaN gets scale NaN and stands for NaN.
 * Queries: evaluated in binary32, rounded once to their type into q_out; q may be NULL with heads == 0.  q_out may be q with its
 * strides (k and v may then be parts of the same tokens' rows); otherwise it must overlap no other array.  Its own rows must not overlap:
 * all heads of a token lie before the next token's, or all tokens of a head before the next head's.
 */
typedef struct {
    int type; /* DQ8_FLOAT32, DQ8_BFLOAT16 or DQ8_FLOAT16: of q, k, v and q_out */
    size_t tokens;
    int heads;
    const void *q, *k, *v;
    void *q_out;
    size_t q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride, q_out_token_stride, q_out_head_stride;
    const int64_t *slots;
    const int64_t *positions; /* NULL without rotation */
    const float *rotation;    /* NULL: no rotation */
    size_t n_positions;
    int half, interleaved;
    const float *q_weight, *k_weight; /* NULL: not normed */
    double eps;
} dq8_append;

int dq8_cache_append(int kind, const dq8_cache *cache, const dq8_append *a, void *hip_stream);

/*
 * Attention of new tokens over the cache.  q and out: [tokens][heads][dim], `type` DQ8_BFLOAT16 or DQ8_FLOAT16, strides as above (of out as of q_out); heads is a
 * multiple of kv_heads, and query head h reads cached head h / (heads / kv_heads).
 * batch sequences; the new tokens of sequence b are starts[b] .. starts[b + 1] of q (starts: batch + 1 ascending integers), or with starts ==
 * NULL tokens / batch each, which must divide.  lens[b]: tokens of the sequence in the cache, its new ones among them (append
 * first): the new tokens are the last ones.  pages: [batch][max_pages], row b the page numbers of the sequence in order.
 * The query at position p sees the cached tokens 0 .. p of its sequence, with window > 0 only the last `window` of them; its output is
 * the mean of their values weighted with exp(softmax_scale * q . key).  A query that sees nothing (lens[b] smaller than the number
 * of new tokens) gets zeros.  Tokens of q behind the last sequence keep their place in `out` as it was.  Lengths beyond
 * max_pages * page_size count as that, negative ones as 0; tokens on pages outside the cache are not seen; starts outside
 * 0 .. tokens count as the nearer end, and where they descend anywhere nothing is written.  Places of the cache that no query sees may hold anything, NaN included.
 * Products and sums are held in binary32; a code's value, a query and a weight times its value's scale are rounded to binary16 (11 bits)
 * where the matrix instructions take them: one rounding each, as large as that of a binary16 output.  Each query's products of
 * weight and scale are brought into range by the largest that it sees itself: one that is less than 2^-19 of that is off by at most 2^-30 of it
 * instead, and nothing that the query does not see counts.  (Where the largest is made of a value scale below 1e-28 or above 1e35, bits are
 * lost sooner.)
 * Results do not depend on anything but the arguments (workspace size and max_new among them).
 * max_new: the largest number of new tokens of a sequence, as far as the host knows (0: unknown); it chooses between kernels that are
 * right for any number.
 * workspace: dq8_cache_attention_workspace_bytes bytes at a multiple of 16, whose contents are of no meaning before and after; calls that
 * may run at the same time must not share it.  Without (NULL, or too few bytes) one wavefront or workgroup reads the whole of a
 * sequence's head: slow where there are few sequences.  The call that asks for its size has the tokens, batch, max_pages, heads, type
 * and max_new of the call that uses it, and starts if that has starts.
 * Work that 32 bits do not count (query rows in groups of 16 to 256, times cached heads, times max_pages * page_size / 32: 2^31) is refused.
 */
typedef struct {
    int type;
    size_t tokens;
    int heads;
    const void *q;
    void *out;
    size_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    size_t batch, max_pages;
    const int32_t *pages, *lens, *starts;
    size_t max_new;
    int window;
    float softmax_scale;
} dq8_attention;

/* (Looks at sizes, type, window and whether starts is NULL; the pointers may be anything.  0 after an error.) */
size_t dq8_cache_attention_workspace_bytes(const dq8_cache *cache, const dq8_attention *a);
int dq8_cache_attention(int kind, const dq8_cache *cache, const dq8_attention *a, void *workspace, size_t workspace_bytes,
                        void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DQ8_CACHE_H */
