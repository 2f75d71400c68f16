/*
 * lorann_states4.h - C ABI of the state store in 4 bits: what lorann_states.h offers, over a store that takes dim / 2 + 8 bytes for a row instead of dim + 4.
 *
 *   lorann_states4_write      quantises the states of new tokens into their slots
 *   lorann_states4_read       reads tokens back as values
 *   lorann_attend4_chunk      causal attention of every sequence's newest tokens over the sequence's own pages (one token or many)
 *   lorann_attend4_passages   attention over the states of the passages found for each sequence
 *
 * Conventions, element types, limits, arguments and errors are those of lorann_states.h; what differs is stated here.
 */
#ifndef LORANN_STATES4_H
#define LORANN_STATES4_H

#include "lorann_states.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The store: `pages` pages of `page_size` tokens, `heads` heads of `dim` values (a multiple of 32).  Token t of page p is slot p * page_size + t.
 * Each row x of `dim` values (one token and head, keys and values apart) is held as x ~= step * r_g * code, g the group of 32 values that a value is in:
 *   step   max|x| / 6, a float
 *   r_g    the smallest number (1 + m / 8) 2^e, m = 0 .. 7, from 2^-13 to 1, with r_g max|x| >= the group's largest magnitude; held in a byte: bits 7 .. 14 of the number in binary16
 *   code   a sign (bit 3: that of the value) and one of the magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6 (bits 0 .. 2: 0 .. 7), nearest to 6 x / (r_g max|x|), halfway to the even code
 * A row with max|x| < 2^-100 is held as codes 0 with step 0; a row that holds a NaN or an infinity as codes 0 with a NaN step, and reads back as NaN; both with the smallest factors.
 *   k_codes    [pages][heads][page_size][dim / 2] bytes, 16-byte aligned: components 2 i (low four bits) and 2 i + 1 in byte i
 *   v_codes    [pages][heads][dim / 2][page_size] bytes, 16-byte aligned: transposed inside a page, components 32 g + n (low four bits) and 32 g + 16 + n in row 16 g + n
 *   k_factors, v_factors  [pages][heads][page_size][4] bytes, 4-byte aligned: byte g is that of values 32 g .. 32 g + 31; bytes beyond dim / 32 are written as 0 and not used
 *   k_scales, v_scales    [pages][heads][page_size] float: the steps
 * Bit 7 of a factor's byte is 0 and not looked at; what slots that were never written hold does not matter, as long as no length covers them.
 * A token's codes share no byte with another's: tokens of one call, or of calls on several streams, may be written in any order.
 */
typedef struct lorann_states4 {
    uint8_t *k_codes, *v_codes, *k_factors, *v_factors;
    float *k_scales, *v_scales;
    int64_t pages;
    int32_t heads, page_size, dim;
} lorann_states4;

/* As lorann_states_write. */
int lorann_states4_write(const lorann_states4 *st, const void *k, const void *v, int32_t type, int64_t tokens,
                         int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, const int64_t *slots, void *hip_stream);

/* As lorann_states_read: the values step * r_g * code, r_g * code exact, their product with the step formed in float and rounded once to `type`. */
int lorann_states4_read(const lorann_states4 *st, const int64_t *slots, int64_t tokens, void *k, void *v, int32_t type,
                        int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void *hip_stream);

/* As lorann_attend_chunk and lorann_attend_passages.  Products of 16-bit queries with r_g * code are exact, as those with 8-bit codes are; everything after them is the same. */
int lorann_attend4_chunk(const lorann_states4 *st, const lorann_questions *qs, const int32_t *tables, int32_t width, const int32_t *lengths,
                         void *workspace, int64_t workspace_bytes, void *hip_stream);
int lorann_attend4_passages(const lorann_states4 *st, const lorann_questions *qs, const int64_t *ids, int32_t found, const float *scores,
                            float score_weight, const int32_t *tables, int32_t width, const int32_t *lengths, int64_t passages,
                            void *workspace, int64_t workspace_bytes, void *hip_stream);

/* As lorann_attend_workspace. */
int64_t lorann_attend4_workspace(const lorann_states4 *st, const lorann_questions *qs, int32_t found, int32_t width);

#ifdef __cplusplus
}
#endif
#endif /* LORANN_STATES4_H */
