/*
 * lorann_evict.h - C ABI for keeping the states of a sequence within a budget: which keys later tokens attended to, and moving the states of those to other pages.
 *
 *   lorann_attend_weights   adds up the weight that causal attention gives each key, over a sequence's newest tokens and the query heads of each head
 *   lorann_states_evict     keeps of every sequence and head the newest keys and those with the largest sums, in order, on other pages
 *
 * Both are offered over the 8-bit store (lorann_states.h) and the 4-bit one (lorann_states4.h: ..4_..).  Conventions, limits and errors are those of lorann_states.h.
 */
#ifndef LORANN_EVICT_H
#define LORANN_EVICT_H

#include "lorann_states.h"
#include "lorann_states4.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * lorann_attend_weights - sums[s][h][j] = before[s][h][j] + sum over the queries i of sequence s and the query heads g of head h of
 *   softmax_j(scale <q_ig, k_j>)  over the keys j <= lengths[s] - T_s + i,  the weights of lorann_attend_chunk with the same arguments (0 for a key that a query does not see)
 *   qs        as for lorann_attend_chunk; `out` and its distances are not used
 *   before    [sequences][heads][width * page_size] float, or NULL for zeros; may be `sums` itself
 *   sums      the same shape: every element is written, those of keys that no query sees with what was there before
 * A query without a key adds nothing, nor does one whose logits are all -infinity (the query holds an infinity, all keys that it sees have the other sign there).  A query with a logit that
 * is NaN or +infinity (a key's states hold a NaN, the query a NaN or another infinity) makes the sums of all keys NaN that it sees.  Products are exact, their sums and everything after them float.  Two runs give the same bits.
 *   workspace      lorann_attend_weights_workspace() bytes of device memory, 16-byte aligned; calls that may overlap need one each
 */
int lorann_attend_weights(const lorann_states *st, const lorann_questions *qs, const int32_t *tables, int32_t width, const int32_t *lengths,
                          const float *before, float *sums, void *workspace, int64_t workspace_bytes, void *hip_stream);
int lorann_attend4_weights(const lorann_states4 *st, const lorann_questions *qs, const int32_t *tables, int32_t width, const int32_t *lengths,
                           const float *before, float *sums, void *workspace, int64_t workspace_bytes, void *hip_stream);
/* Bytes of workspace for these sizes; a negative value is an error code.  Host arithmetic only: pointers in the structures are not looked at (but q_start: NULL or not). */
int64_t lorann_attend_weights_workspace(const lorann_states *st, const lorann_questions *qs, int32_t width);
int64_t lorann_attend4_weights_workspace(const lorann_states4 *st, const lorann_questions *qs, int32_t width);

/*
 * lorann_states_evict - of the keys 0 .. lengths[s] - 1 of each sequence s, for each head apart: if there are more than `budget`, those among the last `recent` keys are kept and, of the
 * others, those with the largest sums until `budget` are kept (equal sums: the earlier key first; a NaN counts as less than every number); otherwise all are.  The r-th kept
 * key, in the order that they had, becomes key r of the destination: its codes, factors and steps are copied as they are.
 *   tables, width, lengths   [sequences][width], [sequences]: as in lorann_attend_chunk; keys of an entry outside [0, pages) are not there (they are neither kept nor counted)
 *   sums          [sequences][heads][width * page_size] float, as lorann_attend_weights leaves them
 *   recent        0 .. budget
 *   to_tables     [sequences][to_width] int32: pages of the destination, to_width * page_size >= budget; tokens of an entry outside [0, pages) are not written.  No page that
 *                 is written to may be one that the call reads, and none may stand twice; pages that several sequences read are fine.
 *   kept          [sequences][heads][budget] int32: numbers of the kept keys in order, -1 behind the last
 *   kept_lengths  [sequences] int32: how many were kept (the same for each head)
 *   kept_sums     [sequences][heads][to_width * page_size] float, or NULL: sums of the kept keys, 0 behind the last; not an array that the call reads
 *   workspace     lorann_evict_workspace() bytes of device memory, 16-byte aligned (NULL if that is 0); calls that may overlap need one each
 * What stands on the destination's pages behind the last kept token stays as it was.
 */
int lorann_states_evict(const lorann_states *st, const int32_t *tables, int32_t width, const int32_t *lengths, int64_t sequences, const float *sums, int32_t budget, int32_t recent,
                        const int32_t *to_tables, int32_t to_width, int32_t *kept, int32_t *kept_lengths, float *kept_sums, void *workspace, int64_t workspace_bytes, void *hip_stream);
int lorann_states4_evict(const lorann_states4 *st, const int32_t *tables, int32_t width, const int32_t *lengths, int64_t sequences, const float *sums, int32_t budget, int32_t recent,
                         const int32_t *to_tables, int32_t to_width, int32_t *kept, int32_t *kept_lengths, float *kept_sums, void *workspace, int64_t workspace_bytes, void *hip_stream);
/* Bytes of workspace of lorann_states_evict and lorann_states4_evict for a store of so many heads and tables of so many tokens (width * page_size); a negative value is an error code. */
int64_t lorann_evict_workspace(int32_t heads, int64_t table_tokens, int64_t sequences);

#ifdef __cplusplus
}
#endif
#endif /* LORANN_EVICT_H */
