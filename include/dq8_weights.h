/*
 * dq8 -- weights of linear layers in 4 bits, and their products with the activations of a few tokens.
 *
 * A decoding step reads every weight once for a handful of tokens: what it costs is the bytes of the weights.  Here `group` neighbours of
 * a row share one scale, as a row of the cache does (dq8_cache.h), and an element has four bits: a sign, two bits of exponent and one of mantissa.
 *
 * Conventions (streams, device pointers, error codes, DQ8_DEBUG, threads) are those of dq8.h.  The structs are HOST memory, read before the
 * call returns; the pointers in them are DEVICE pointers.  Types: DQ8_FLOAT32, DQ8_BFLOAT16, DQ8_FLOAT16 of dq8_cache.h.  For serving: the
 * calls have no gradient.
 */
#ifndef DQ8_WEIGHTS_H
#define DQ8_WEIGHTS_H

#include "dq8_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DQ8_WEIGHTS_MAX_TOKENS (1 << 20)

/*
 * Compressed weights of a matrix [rows][cols].  group: 32, 64 or 128.
 * Value: magnitude m of a code, 0, 0.5, 1, 1.5, 2, 3, 4, 6 for its three lower bits 0 .. 7, negative where its fourth bit is set, times the
 * scale of its group (exactly: a product has ten bits).
 * Layout: tiles of 16 rows and 128 columns, [row tiles][column tiles], the last ones filled up with zeros.  codes: 1024 bytes of a tile, at a
 * multiple of 16 bytes; piece 16 g + n of its 64 pieces of 16 bytes is of row n, and word s of its four words holds the columns 32 s + 8 g ..
 * + 7, four bits each from the lowest on.  scales: bfloat16 [row tiles][column tiles][16 rows][128 / group], at a multiple of 8 bytes.
 * (A wavefront's 64 loads of 16 bytes are one tile, and each of the four words one operand of a matrix instruction whose products share a scale.)
 * rows up to 2^28 - 16, cols below 2^31, ceil(rows / 16) * ceil(cols / 128) tiles below 2^25.
 */
typedef struct {
    uint8_t *codes;
    void *scales;
    size_t rows, cols;
    int group;
} dq8_weights;

/*
 * w: [rows][cols] of `type`, row r starts r * row_stride elements after its pointer, which is a multiple of its element's size.
 * Scale of a group: the bfloat16 number nearest to max |w| / 6 (evaluated in binary32), at most 170 * 2^118, whose sixfold is still
 * finite.  Code: the magnitude whose product with the scale is nearest to |w| in real arithmetic, the smaller of two as near; the sign of w.  With
 * scale zero the codes are zeros that keep the sign.  A group that holds an infinity or NaN gets scale NaN and stands for NaN.
 */
int dq8_weights_encode(int type, const void *w, size_t row_stride, const dq8_weights *out, void *hip_stream);

/* The values, rounded once to `type` (not at all for DQ8_FLOAT32).  Rows of w must not overlap. */
int dq8_weights_decode(const dq8_weights *in, int type, void *w, size_t row_stride, void *hip_stream);

/*
 * out[m][n] = sum over k of x[m][k] * value[n][k], plus bias[n] where bias is not NULL, for `tokens` rows m of x (up to
 * DQ8_WEIGHTS_MAX_TOKENS; none, or weights without rows, is no error, weights without columns are).
 * x: [tokens][cols] of `type` DQ8_BFLOAT16 or DQ8_FLOAT16; out: [tokens][rows] of out_type, `type` or DQ8_FLOAT32; strides of rows in
 * elements; pointers are multiples of their element's size.  out must overlap no other array, its rows not each other.
 * Products are exact, sums are held in binary32 (of 32 .. 128 products in the matrix instructions, then times the group's scale; of bfloat16 activations
 * at 2^-10 of their size, so that no sum of a group leaves binary32, and results below 2^-115 have fewer bits), the result is rounded once.  Their order depends on rows, cols, tokens and group and on whether there is a workspace: equal calls give equal bits.  An
 * infinity or NaN in a row of x makes that row of out what it makes the sum; other rows do not depend on it.
 * workspace: dq8_weights_product_workspace_bytes bytes at a multiple of 16 (0: none is used, as for up to 8 tokens), whose contents are of no meaning before
 * and after; calls that may run at the same time must not share it.  Without (NULL, or too few bytes) a workgroup has all columns of its rows:
 * slower where there are few rows.
 */
typedef struct {
    int type, out_type;
    size_t tokens;
    const void *x;
    size_t x_stride;
    void *out;
    size_t out_stride;
    const float *bias;
} dq8_product;

/* (Looks at sizes and types; the pointers of p may be anything.  0 after an error.) */
size_t dq8_weights_product_workspace_bytes(const dq8_weights *w, const dq8_product *p);
int dq8_weights_product(const dq8_weights *w, const dq8_product *p, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DQ8_WEIGHTS_H */
