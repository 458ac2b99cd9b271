/*
 * dq8 -- what a decoding step needs around its cache (dq8_cache.h): where its tokens go, and which of its drafted tokens stay.
 *
 * dq8_cache_plan makes the slots and positions of dq8_cache_append and the page tables, lengths and starts of dq8_cache_attention from the
 * lengths of the requests; dq8_draft_verify judges drafted tokens by the target model's probabilities, and the number of those it
 * rejects is what the next plan takes back.  A sequence that the plan refuses has no tokens in the step, and the drop that it was refused with is
 * still to come: dq8_draft_verify takes the plan's `granted` and `drop` and hands that drop on.  Neither waits for the host, and both can be
 * captured into a graph.
 *
 * Conventions (streams, device pointers, error codes, DQ8_DEBUG, threads) are those of dq8.h.  The structs are HOST memory, read before the
 * call returns; the pointers in them are DEVICE pointers; fields that a caller does not use are 0.  What the host cannot see is checked by the kernels as described below; nothing
 * outside the given arrays is read or written.
 */
#ifndef DQ8_SERVE_H
#define DQ8_SERVE_H

#include "dq8_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DQ8_PLAN_MAX_BATCH 4096

/*
 * Sequence b has lens[b] cached tokens (negative counts as 0, more than max_pages * page_size as that) on the first ceil(lens[b] / page_size)
 * pages of row b of `pages` [batch][max_pages].  drop[b] of them are taken back from its end (drop NULL or negative: none, more than it
 * has: all), then new_tokens[b] are added (negative: none).  Pages that it no longer needs go onto the stack of free pages, those it needs
 * more are taken from the stack's top; a page that it keeps stays where it is.
 * free_pages [free_capacity]: the stack, n_free[0] entries of it valid.  All pages given back in a call are put on it first, in the order of
 * the sequences and of the pages in a sequence (what finds no room any more is lost), then pages are taken from its end in the same order.
 * A sequence is granted all that it asks for or refused: where it would have more than max_pages pages, where its new tokens would end
 * behind `tokens`, or where the stack does not hold the pages that it and the sequences before it take.  (A refused sequence takes none, but
 * counts among those before the next: after one that found too few pages none that needs any gets them.)  For a refused sequence nothing
 * changes, its drop included, which a later plan has to be given again.
 * Written: starts[batch + 1], the sums of new tokens before each sequence, refused ones counted (at most `tokens`); granted[b]: new tokens
 * granted, -1 where refused; lens_out[b]: the length after the step; n_free_out[0]; and for tokens i = 0 .. `tokens` - 1 of the step, packed in the
 * order of the sequences, positions[i], the place in its sequence, and slots[i] = page * page_size + place in the page; both are -1 for tokens of
 * refused sequences and behind the last one (dq8_cache_append stores nothing for such tokens, and their queries and outputs mean nothing).  pages and
 * free_pages change in place; entries that nobody needs stay as they were.
 * lens_out may be lens and n_free_out may be n_free: the state then moves on in place.  All other arrays must be apart from each other.
 * page_size: a power of two from 16 to DQ8_CACHE_MAX_PAGE; batch from 1 to DQ8_PLAN_MAX_BATCH; batch * max_pages, max_pages * page_size, tokens and
 * free_capacity below 2^31.
 */
typedef struct {
    size_t batch, max_pages, tokens, free_capacity;
    int page_size;
    const int32_t *lens, *new_tokens, *drop;
    int32_t *pages, *free_pages;
    const int32_t *n_free;
    int64_t *slots, *positions;
    int32_t *starts, *lens_out, *granted, *n_free_out;
} dq8_plan;

int dq8_cache_plan(const dq8_plan *p, void *hip_stream);

/*
 * Rows starts[b] .. starts[b + 1] - 1 of a step belong to sequence b (starts NULL: tokens / batch each, which must divide): its last accepted token and then
 * its drafted ones; ids[i] is the token that was fed in row i.  target [tokens][vocab]: the target model's probabilities behind each row,
 * so that row i judges the drafted token of row i + 1; draft: the probabilities which that token was drawn from, in row i too (NULL: the
 * draft is sure of it, 1 for the token and 0 for all others).  Both of `type`, strides of rows in elements.  Probabilities need not add up to
 * one; what is no positive number (negative, NaN, infinite) counts as 0, and so does a drafted token outside 0 .. vocab - 1, which is refused.
 * A drafted token d of row i + 1 is accepted while uniform[i] * draft[i][d] < target[i][d] (exactly; NaN: not).  Behind the accepted ones one
 * token is drawn: where a draft was refused with weights max(target - draft, 0) of its row i, or with the target's if these are all 0; where
 * none was with the target's of the last row.  It is the first t whose weights 0 .. t add up to more than sample[b] times the sum of all, or the last with
 * a weight where none does (sample[b] of 1 and more; NaN and negative count as 0).  Differences and sums in binary64.
 * Written: out, for each row of a sequence: the accepted tokens, the drawn one, then -1 (the drawn one is -1 too if all its weights are 0); accepted[b]: how
 * many drafts were accepted, -1 for a sequence without rows; rejected[b]: how many were not.  Rows of no sequence, before the first and behind the last,
 * stay as they were, or are -1 where `fill` is not 0.  (Without sequences nothing is written.)
 * batch up to 65535, tokens below 2^31, vocab from 1 to below 2^31 - 4096.
 * starts outside 0 .. tokens count as the nearer end; they must not descend (a sequence whose do has no rows, and rows that two claim hold
 * tokens of either, with `fill` perhaps -1).
 * granted [batch] (NULL: nobody was refused) and drop [batch] (NULL: 0 for all): those of the plan that gave the rows their places.  The rows of a sequence with granted[b]
 * negative hold no tokens, whatever is in them: out is -1 there, accepted[b] is -1, and rejected[b] is what the plan did not take back, drop[b] (negative:
 * 0).  So `rejected` is the next plan's drop for every sequence.  rejected may be drop; without granted, drop is not read.
 * workspace: dq8_draft_verify_workspace_bytes bytes at a multiple of 16, whose contents are of no meaning before and after; calls that
 * may run at the same time must not share it.  Without (NULL, or too few bytes) one workgroup reads a sequence's whole row.  Results do not depend on it.
 */
typedef struct {
    int type;
    size_t tokens, batch, vocab;
    const void *target, *draft;
    size_t target_stride, draft_stride;
    const int64_t *ids;
    const float *uniform, *sample;
    const int32_t *starts;
    int64_t *out;
    int32_t *accepted, *rejected;
    const int32_t *granted, *drop;
    int fill;
} dq8_verify;

/* (Looks at sizes; the pointers may be anything.  0 after an error, or where none is of use.) */
size_t dq8_draft_verify_workspace_bytes(const dq8_verify *v);
int dq8_draft_verify(const dq8_verify *v, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* DQ8_SERVE_H */
