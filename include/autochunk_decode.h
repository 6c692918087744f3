/*
 * Decoding behind the same library: the operators that a causal decoder runs for each new token (or few) once its prompt is
 * in a cache: linear layers with 4-bit weights, the append of rotated keys and values to a paged 8-bit cache, and the
 * attention that reads this cache.  The conventions are those of autochunk_rt.h: "dev" pointers are the caller's device
 * memory, `stream` is a hipStream_t, nothing is allocated, kept or synchronised, dtypes are AC_BF16 and AC_F32, a call
 * returns AC_OK or a negative ac_status with its text in ac_last_error().
 */
#ifndef AUTOCHUNK_DECODE_H
#define AUTOCHUNK_DECODE_H

#include <stdint.h>

#include "autochunk_rt.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * out[m, n] = act(sum_k x[m, k] * (code[n, k] - zero[n, k / group]) * scale[n, k / group] + bias[n]) + residual[m, n].
 * w holds the codes 0..15, two to a byte: byte i of row n holds column 2 i in its low four bits and column 2 i + 1 in its high
 * ones; rows start `ldw` bytes apart, a multiple of 16 that is at least (k + 1) / 2; a row is read in pieces of 16 bytes, codes past column k are not used.
 * scale (and zero, NULL = 8 everywhere) [n, ceil(k / group)], rows lds (ldz) elements apart, of type `dtype` as x, bias (may be
 * NULL), residual (may be NULL, may be out) and out.  group: 32, 64 or a multiple of 128.  Sums are fp32,
 * and no weight is rounded; in products of many bf16 rows zeros that are no whole numbers take longer.  The products of a row of x that holds an infinity or a NaN are
 * infinities or NaN, where an infinity is due also NaN, and every activation leaves NaN as it is; other rows do not see them.  The sums
 * over a group of |x|, twice that with zeros up to 16, and of |x (code - zero)| / 16 have to be within fp32's range.
 * m is at most 16 * 65535, n 2^26, else AC_ERR_UNSUPPORTED, k and group 2^30.  w on a 16-byte boundary, else AC_ERR_ALIGN.  Rows of x on 16-byte boundaries (ldx a multiple of 8 in bf16, of 4 in fp32) are read
 * faster than others.
 */
int ac_op_linear_w4(const void* x, int64_t ldx, const void* w, int64_t ldw, const void* scale, int64_t lds, const void* zero,
                    int64_t ldz, int64_t group, const void* bias, const void* residual, int64_t ldr, void* out, int64_t ldo,
                    int64_t m, int64_t n, int64_t k, int activation, int dtype, void* stream);

/*
 * Keys and values of one layer in 8 bits, in pages of `page` tokens (a multiple of 16).  A block is a run of 16 tokens of one head,
 * aligned to 16 in its sequence; it has one scale for its keys and one for its values, and a code stands for
 * (e4m3 value) * (its block's scale).  e4m3: sign, 4 bits of exponent, 3 of mantissa, largest number 448, no infinities.
 *   k        [pages][heads][page][head_dim]             codes, pages stride_page bytes apart
 *   v        [pages][heads][page / 16][head_dim][16]    codes, the 16 tokens of a block side by side, pages stride_page bytes apart
 *   k_scale, v_scale  [pages][heads][page / 16]         fp32, pages stride_scale floats apart
 * Scales of blocks that hold tokens are powers of two, as the append leaves them: the attention may apply a scale by its exponent alone.
 * head_dim 32, 64, 96, 128, 192 or 256, else AC_ERR_UNSUPPORTED; k, v and stride_page in multiples of 16 bytes, else AC_ERR_ALIGN.
 */
typedef struct ac_kv_cache {
  void* k; void* v;                 /* dev */
  float* k_scale; float* v_scale;   /* dev */
  int64_t pages, stride_page, stride_scale;
  int32_t page, heads, head_dim;
} ac_kv_cache;

/*
 * The rows of one call and where their sequences' tokens lie.  Sequence b has the rows row_begin[b] .. row_begin[b + 1] - 1 of
 * the call's matrices (possibly none; rows past the matrices' n_rows do not exist), which are the last of its length[b] tokens; token t lies in page
 * page_table[b * ld_page_table + t / page], at place t mod page.  Places past ld_page_table pages do not exist; a page number outside
 * [0, pages) names no memory: what would be stored there is dropped, what would be read there counts as masked.  So do rows that a length
 * shorter than the sequence's rows would put in front of token 0.  max_rows and max_length: the most rows and tokens of one
 * sequence as far as the host knows, by which launches are sized; sequences that exceed them are still computed, more slowly.
 * There may be no sequences, no rows, no places (ld_page_table 0) and no pages in the cache; pointers to what is not there may be NULL.
 * At most 65535 sequences, 2^30 rows (times heads, in the attention) and 2^30 places of a sequence, else AC_ERR_UNSUPPORTED.
 */
typedef struct ac_cache_rows {
  const int32_t* row_begin;         /* dev, [batch + 1] */
  const int32_t* length;            /* dev, [batch] */
  const int32_t* page_table;        /* dev, [batch][ld_page_table] */
  int64_t ld_page_table, batch, max_rows, max_length;
} ac_cache_rows;

/*
 * Rotation by position: pair i of a head (0 <= i < pairs) is turned by the angle whose cosine and sine stand in row p of two fp32
 * tables: (a, b) -> (a cos - b sin, a sin + b cos).  The pair's elements are i and i + pairs of the head, or, interleaved, 2 i and 2 i + 1; elements
 * from 2 * pairs on stay as they are.  p is positions[axis * ld_positions + row], where the first section[0] pairs belong to
 * axis 0, the next section[1] to axis 1 and so on (time, height and width of an image or a video; text has one axis), or, with
 * positions = NULL, the row's place in its sequence; it is brought into [0, table_rows).
 */
typedef struct ac_rotary {
  const float* cos; const float* sin;   /* dev, [table_rows][ld_table], ld_table >= pairs; at most 2^30 elements */
  int64_t table_rows, ld_table;
  const int32_t* positions;             /* dev, [axes][ld_positions], or NULL */
  int64_t ld_positions;
  int32_t pairs, interleaved, axes;     /* pairs a multiple of 4, axes 1..4 */
  int32_t section[4];                   /* sum over the axes = pairs */
} ac_rotary;

/*
 * Rotates the rows' keys (and queries) and stores keys and values in the cache.  k, v: [n_rows][cache->heads * head_dim], rows ldk, ldv apart;
 * q (may be NULL): [n_rows][heads * head_dim], its rotated rows go to q_out, which may be q.  rotary may be NULL (positions are in the rows already).
 * A block that gets rows takes as its scale the least power of two s >= 2^-100 with |x| <= 448 s for all its finite new elements, or the scale that it has if it holds older
 * tokens and that one is larger; elements are stored as the nearest e4m3 number (ties to even) of x / s, infinities and NaN as NaN.  Where older tokens' scale
 * grows, their codes are rewritten as the nearest of code * (old scale / s), which is exact for all but the smallest numbers.  Tokens of a block
 * behind the sequence's last stay as they are.  Two sequences must not append into the same block.
 * All rows and q_out's on 8-byte (bf16) / 16-byte (fp32) boundaries, tables (if there are pairs) on 16-byte ones, ld_table a multiple of 4, else AC_ERR_ALIGN.
 */
int ac_op_cache_append(const void* q, int64_t ldq, void* q_out, int64_t ldqo, int heads, const void* k, int64_t ldk, const void* v,
                       int64_t ldv, int64_t n_rows, const ac_kv_cache* cache, const ac_cache_rows* rows, const ac_rotary* rotary,
                       int dtype, void* stream);

/*
 * out[r, h] = softmax(scale * q[r, h] . k) v over the tokens that row r sees: all of its sequence's, or with causal != 0 those up to its own place.
 * Query head h reads head h / (heads / cache->heads) of the cache (heads a multiple of cache->heads).  A row that sees nothing (length 0)
 * comes out as zeros; tokens that a row does not see do not reach it, whatever their codes.  Scores, maxima and sums are fp32.  Probabilities are fp32 with fp32 rows; with bf16
 * rows they meet the values with 16 bits, and with 8 where many rows go through tiles for prompts.  q, out: [n_rows][heads * head_dim], rows on
 * 16-byte boundaries, else AC_ERR_ALIGN.  Few rows over many tokens are split over the tokens, and the parts joined by a second kernel:
 * workspace (dev, 16-byte aligned) holds them, ac_cache_attention_workspace_bytes() large (0: none needed), else AC_ERR_WORKSPACE.
 * Results do not depend on what else runs, but on the split: on max_rows, max_length, batch and n_rows.
 */
int ac_op_cache_attention(const void* q, int64_t ldq, void* out, int64_t ldo, int64_t n_rows, int heads, const ac_kv_cache* cache,
                          const ac_cache_rows* rows, int causal, float scale, void* workspace, uint64_t workspace_bytes, int dtype,
                          void* stream);
uint64_t ac_cache_attention_workspace_bytes(int64_t n_rows, int heads, const ac_kv_cache* cache, const ac_cache_rows* rows, int causal,
                                            int dtype);

#ifdef __cplusplus
}
#endif
#endif /* AUTOCHUNK_DECODE_H */
