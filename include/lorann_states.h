/*
 * lorann_states.h - C ABI of the state store beside the index: keys and values of tokens in 8 bits, in pages, and the attention that reads
 * them.  What a search returns are ids of corpus rows; a model that answers with them reads the states (keys and values) that an encoder
 * made of the passages behind the ids, and keeps those of its own tokens.  Both live in one store:
 *
 *   lorann_states_write      quantises the states of new tokens into their slots
 *   lorann_states_read       reads tokens back as values
 *   lorann_attend_chunk      causal attention of every sequence's newest tokens over the sequence's own pages (one token or many)
 *   lorann_attend_passages   attention over the states of the passages found for each sequence: takes the ids as lorann_search leaves them
 *
 * Conventions shared by the entry points
 *   - Every pointer inside the structures and every array argument is device memory of the current HIP device (host memory and that of another
 *     GPU are refused); the structures themselves are host memory.  The library keeps no caller pointer and no state between calls: the store's memory and the workspace are the caller's.
 *   - Work is enqueued on `hip_stream` (a hipStream_t; NULL: the null stream) and the call returns.  Nothing is allocated, copied to the host
 *     or waited for, so a call can be captured into a HIP graph.  Calls that write and read the same slots are ordered by the caller
 *     (one stream, or events).
 *   - There are no gradients: the store holds rounded codes, and nothing here keeps what a backward pass would need.
 *   - Return value: LORANN_OK or a negative error code of lorann.h, with the message in lorann_last_error(); on error nothing is enqueued.
 *   - Page numbers, slots, ids, lengths and offsets in device memory are checked on the device against the sizes that the call names: what
 *     lies outside is left out, as stated at each, and never read or written through.
 */
#ifndef LORANN_STATES_H
#define LORANN_STATES_H

#include "lorann.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of what is written, read, asked and answered. */
enum { LORANN_F32 = 0, LORANN_F16 = 1, LORANN_BF16 = 2 };

/* Limits of this implementation. */
#define LORANN_MIN_PAGE 16        /* tokens per page: a power of two from here ... */
#define LORANN_MAX_PAGE 256       /* ... to here */
#define LORANN_MAX_DIM 128        /* values per head: a multiple of 32 up to this */
#define LORANN_MAX_HEADS 1024     /* heads of the store; query heads likewise */
#define LORANN_MAX_FOUND 4096     /* passages per sequence */

/*
 * The store: `pages` pages of `page_size` tokens, `heads` heads of `dim` values.  Token t of page p is slot p * page_size + t.
 * Each row x of `dim` values (one token and head, keys and values apart) is held as x ~= step * code with step = max|x| / 127 and
 * code = 127 x / max|x| rounded to the nearest integer, ties to even: absmax quantization as the index's factors have it (Sec. 3.3).  A row with
 * max|x| < 2^-100 is held as zeros with step 0; a row that holds a NaN or an infinity as codes 0 with a NaN step, and reads back as NaN.
 *   k_codes   [pages][heads][page_size][dim] int8, 16-byte aligned
 *   v_codes   [pages][heads][dim][page_size] int8, 16-byte aligned: a page's values are transposed, since the second product of the
 *             attention contracts over the tokens
 *   k_scales, v_scales  [pages][heads][page_size] float: the steps (a step of 0 stands beside codes of 0)
 */
typedef struct lorann_states {
    int8_t *k_codes, *v_codes;
    float *k_scales, *v_scales;
    int64_t pages;
    int32_t heads, page_size, dim;
} lorann_states;

/*
 * lorann_states_write - quantise the keys and values of `tokens` tokens into their slots.
 *   k, v                     rows of `dim` consecutive values of type `type` (LORANN_F32 / F16 / BF16), aligned to their type;
 *   k_token, k_head, ...     distances in elements between tokens and between heads (any sign), so that slices of a fused projection or another order of the
 *                            axes are taken as they are
 *   slots                    [tokens] int64: slot of each token; outside [0, pages * page_size): the token is left out.  Two tokens of one
 *                            call with the same slot leave either one's states, or parts of both.
 */
int lorann_states_write(const lorann_states *st, const void *k, const void *v, int32_t type, int64_t tokens,
                        int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, const int64_t *slots, void *hip_stream);

/*
 * lorann_states_read - the values step * code of `tokens` tokens, formed in float and rounded once to `type`.
 *   slots  as above, in any order, with repetitions; a token whose slot is outside the store reads as zeros
 *   k, v   are written with the same meaning of the distances; rows must not overlap.  Either may be NULL (not read).
 */
int lorann_states_read(const lorann_states *st, const int64_t *slots, int64_t tokens, void *k, void *v, int32_t type,
                       int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void *hip_stream);

/*
 * The queries of an attention: `tokens` tokens of `sequences` sequences, `heads` heads each - a multiple of the store's heads: query head g
 * reads head g / (heads / store heads), so heads next to each other share keys and values.
 *   q, out       rows of the store's `dim` consecutive values, type LORANN_F16 or LORANN_BF16, with distances in elements; out must not overlap q
 *   q_start      [sequences + 1] int32, non-decreasing, within [0, tokens]: sequence s owns tokens q_start[s] .. q_start[s + 1] - 1 (none is
 *                legal).  Rows of tokens that belong to no sequence are not written.  NULL: every sequence owns tokens / sequences tokens (which must
 *                divide evenly).
 *   scale        factor of the products, finite (usually dim^-1/2)
 */
typedef struct lorann_questions {
    const void *q;
    void *out;
    int32_t type, heads;
    int64_t tokens, sequences;
    int64_t q_token, q_head, out_token, out_head;
    const int32_t *q_start;
    float scale;
} lorann_questions;

/*
 * lorann_attend_chunk - every sequence's newest tokens attend to the sequence's tokens up to and including themselves:
 *   out_i = sum_j softmax_j(scale <q_i, k_j>) v_j  over the keys j <= lengths[s] - T_s + i  of sequence s, T_s its number of queries, i = 0 .. T_s - 1.
 * The new tokens' own states have been written into the store before (lorann_states_write on the same stream).
 *   tables    [sequences][width] int32: page numbers of each sequence; key j is token j % page_size of page tables[s][j / page_size].
 *             Entries beyond a sequence's length are not used.  The keys of an entry outside [0, pages) are left out.
 *   lengths   [sequences] int32: tokens of the sequence in the store, the new ones included; taken within [0, width * page_size]
 * A query without a key (length 0, or more queries than tokens) answers with zeros.  A key whose states hold a NaN makes the answers of
 * those queries NaN that see it, and no others.  Products of 8-bit codes and 16-bit queries are exact, their sums float, as are the softmax statistics
 * and sums; the weights of the second product are rounded to 11 bits (those below 2^-23 of the largest to a multiple of 2^-33 of it), the answer once to its type.
 *   workspace      lorann_attend_workspace() bytes of device memory, 16-byte aligned (NULL if that is 0); calls that may overlap need one each
 */
int lorann_attend_chunk(const lorann_states *st, const lorann_questions *qs, const int32_t *tables, int32_t width, const int32_t *lengths,
                        void *workspace, int64_t workspace_bytes, void *hip_stream);

/*
 * lorann_attend_passages - the queries of sequence s attend to all tokens of the passages ids[s][0 .. found - 1]:
 *   out_i = sum_{r, j} softmax_{r, j}(scale <q_i, k_{id_r, j}> + score_weight * scores[s][r]) v_{id_r, j}
 *   ids       [sequences][found] int64: passage numbers, as lorann_search returns them for a corpus whose row ids are passage numbers; a number
 *             outside [0, passages) (the search's -1 among them) is left out, a number that stands twice counts twice
 *   scores    [sequences][found] float, or NULL (no term).  With the search's distances and a negative score_weight a nearer passage weighs
 *             more: only the terms' differences from the largest count, so they may be large.  A passage whose term is -inf is left out.
 *   tables    [passages][width] int32, lengths [passages] int32: pages and tokens of each passage, with the meaning above
 * No passages, or none with tokens: the answer is zeros.
 */
int lorann_attend_passages(const lorann_states *st, const lorann_questions *qs, const int64_t *ids, int32_t found, const float *scores,
                           float score_weight, const int32_t *tables, int32_t width, const int32_t *lengths, int64_t passages,
                           void *workspace, int64_t workspace_bytes, void *hip_stream);

/* Bytes of workspace that the two attentions need for these sizes: found = 0 for lorann_attend_chunk.  0 is possible; a negative value is an
 * error code.  Host arithmetic only: pointers in the structures are not looked at. */
int64_t lorann_attend_workspace(const lorann_states *st, const lorann_questions *qs, int32_t found, int32_t width);

#ifdef __cplusplus
}
#endif
#endif /* LORANN_STATES_H */
