/*
 * eas_language.h -- operators of the language model that the Encode stage feeds (sm_100a).
 *
 * The paper co-locates the Encode stage with the prefill (and decode) workers of its language model (Section 3.4: the
 * encoder gets a share of the SMs, the neighbour the rest).  These are the attention operators of those
 * neighbours: causal attention of packed prompts, an 8-bit paged key/value cache that prompts and single tokens are written
 * to, the attention of single tokens and of several new tokens a sequence over it, and rotary positions, alone and on the way into the cache.  They follow the conventions of eas_encoder.h: caller-owned memory, an
 * eas_status and eas_last_error(), work enqueued on `stream`, at most `sm_budget` SMs (0 = all), the same bytes for any
 * sm_budget.  All pointers are on the device that is current at the call.
 *
 * Data types: queries, keys, values and outputs are bf16 or fp16 (one type a call).  A row is one token; the heads of a token
 * lie side by side, head_dim elements each; `ld` is the distance of two tokens in elements (a multiple of 8), so that
 * the thirds of a packed projection can be passed as they are.  head_dim is 64 or 128; n_heads is a multiple of n_kv_heads,
 * and query head h reads key/value head h / (n_heads / n_kv_heads).  Row pointers are 16-byte aligned.
 */
#ifndef EAS_LANGUAGE_H_
#define EAS_LANGUAGE_H_

#include "eas_encoder.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { EAS_DTYPE_BF16 = 0, EAS_DTYPE_FP16 = 1 };

/* ---- causal attention of packed prompts ----
 * Sequence s has queries cu_q[s] .. cu_q[s+1] - 1 and keys cu_k[s] .. cu_k[s+1] - 1; its queries are the LAST tokens among its
 * keys: query i sees keys 0 .. i + (keys - queries).  (cu_k = cu_q: whole prompts.  More keys than queries: a chunk of a
 * prompt behind a prefix.  Fewer: the first queries see nothing; their output rows are 0.)
 *   out = softmax(scale * q k^T) v,  fp32 inside; probabilities are rounded to the data type before they meet v.
 * A row reads nothing it does not see: Inf or NaN in keys and values behind it, or in other sequences, does not reach it.  What it does see counts
 * as in the formula: a key that scores -Inf has weight 0, a score of Inf or NaN, or -Inf alone, makes the row NaN, and an infinite value its element
 * (NaN with one of the other sign, with NaN, or where its key has weight 0).  Rows with such elements are looked at a second time, slowly. */
typedef struct {
  const void* q;       /* device [cu_q[n_seqs], n_heads * head_dim], distance ld_q */
  const void* k;       /* device [cu_k[n_seqs], n_kv_heads * head_dim], distance ld_k */
  const void* v;       /* the same, distance ld_v */
  void* out;           /* device, as q, distance ld_out, overlaps none of them; rows behind cu_q[n_seqs] and in front of cu_q[0] are left alone */
  int64_t ld_q, ld_k, ld_v, ld_out;
  int32_t dtype;       /* EAS_DTYPE_* */
  int32_t n_heads, n_kv_heads, head_dim; /* at most 128 query heads per key/value head */
  float scale;         /* > 0, finite; 1 / sqrt(head_dim) as a rule */
  int32_t n_seqs;      /* >= 0 */
  const int32_t* cu_q; /* host [n_seqs + 1], from >= 0, not decreasing */
  const int32_t* cu_k; /* host [n_seqs + 1], likewise */
} eas_prompt_inputs;

/* Device scratch of a call on the current device, for these shapes: 0 for most (and on bad arguments).  A call whose query tiles are too few
 * for the device's SMs although its key ranges are long cuts the key ranges and joins the parts; a sequence's last bits then depend on
 * what else is in the call. */
size_t eas_prompt_attention_workspace_bytes(const eas_prompt_inputs* in);

/* workspace: device, 256-byte aligned, of that size (NULL where it is 0); its contents do not matter, and nothing of it is used by a later
 * call, but calls that may run at the same time need one each.  status_dev: device uint32 (caller zeroes it) that the kernel raises to 1 when a
 * bounded wait expires.
 * Errors (nothing launched): INVALID_ARG, UNSUPPORTED (head_dim, dtype, heads per key/value head, more than 2^24 units of query rows), WORKSPACE, ARCH, CUDA. */
eas_status eas_prompt_attention(const eas_prompt_inputs* in, void* workspace, size_t workspace_bytes, int32_t sm_budget, void* stream,
                                uint32_t* status_dev);

/* ---- 8-bit key/value cache ----
 * Keys and values are signed 8-bit numbers in blocks of block_size tokens, with one scale for each block and head (keys and
 * values apart): value = number * scale.  A sequence's token t lies in block block_table[s][t / block_size] at place
 * t % block_size; any number of sequences may read a block, but only one may write it. */
typedef struct {
  int8_t* k;           /* device [n_blocks][n_kv_heads][block_size][head_dim], 16-byte aligned */
  int8_t* v;
  float* k_scale;      /* device [n_blocks][n_kv_heads], >= 0 */
  float* v_scale;
  int32_t n_blocks, block_size; /* block_size 16, 32, 64 or 128 */
  int32_t n_kv_heads, head_dim;
} eas_cache_desc;

typedef struct eas_cache eas_cache; /* opaque: the description and its tensor maps; allocates and owns no device memory */
eas_status eas_cache_create(const eas_cache_desc* desc, eas_cache** out);
void eas_cache_destroy(eas_cache* cache);

/* Which tokens of which sequences a call is about; all arrays on the device, read when the call's work runs, so that a captured
 * call can be replayed for other lengths.  What points outside the cache (a block number outside 0 .. n_blocks - 1, a place
 * behind max_blocks * block_size, a negative start) is skipped and raises the status word to EAS_DEVICE_CACHE_RANGE. */
typedef struct {
  int32_t n_seqs;             /* >= 0 */
  const int32_t* block_table; /* [n_seqs][max_blocks], distance ld_table */
  int32_t max_blocks;
  int64_t ld_table;
  const int32_t* cu_seqlens;  /* store, load: [n_seqs + 1] rows of each sequence in k and v, not decreasing */
  const int32_t* start;       /* store, load: [n_seqs] the place of each sequence's first row, >= 0 */
  const int32_t* seq_lens;    /* attention: [n_seqs] tokens to attend to */
} eas_cache_seqs;
enum { EAS_DEVICE_CACHE_RANGE = 3 }; /* value of the status word, beside 1 (a bounded wait expired) */

/* Writes rows cu_seqlens[s] .. cu_seqlens[s+1] - 1 of k and v to places start[s], start[s] + 1, ... of sequence s.
 *   scale = max(largest magnitude of the block's new values / 127, scale of the tokens that are in the block already, 2^-100)
 *   number = nearest integer to value / scale, ties to even
 * "In the block already" are the tokens at places below start[s] of the same block; where the scale grows their numbers are
 * rounded again (number * old scale / scale).  Places behind the last one written keep whatever they hold.  A value that is
 * not finite makes the scale of its block and head NaN, and with it all that is read from there, until the block is written from its first place again.
 * n_rows: rows of k and v that exist (a bound on cu_seqlens).  Deterministic: no atomics. */
eas_status eas_cache_store(const eas_cache* cache, const eas_cache_seqs* seqs, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                           int32_t n_rows, int32_t dtype, int32_t sm_budget, void* stream, uint32_t* status_dev);

/* The opposite direction: the values of the same places, rounded to dtype, into rows of k and v.  Rows that are not named
 * (or whose block is out of range) are left as they were. */
eas_status eas_cache_load(const eas_cache* cache, const eas_cache_seqs* seqs, void* k, int64_t ld_k, void* v, int64_t ld_v,
                          int32_t n_rows, int32_t dtype, int32_t sm_budget, void* stream, uint32_t* status_dev);

/* out[s] = softmax(scale * q[s] k^T) v over places 0 .. seq_lens[s] - 1 of sequence s: one token per sequence.  A sequence
 * of length 0 (or less) gets 0, a query with Inf or NaN in it NaN.  Inside, the query is fp16 times a power of two (elements below 2^-24 of its
 * largest are lost) and the weights are rounded to fp16, 2^-32 of the largest at the finest; sums are fp32.  workspace: device scratch of eas_cache_attention_workspace_bytes() (0 on bad arguments), 256-byte
 * aligned; its contents do not matter and nothing of it is used by a later call, but calls that may run at the same time need one each. */
size_t eas_cache_attention_workspace_bytes(const eas_cache* cache, int32_t n_seqs, int32_t n_heads);
eas_status eas_cache_attention(const eas_cache* cache, const eas_cache_seqs* seqs, const void* q, int64_t ld_q, void* out, int64_t ld_out,
                               int32_t n_heads, int32_t dtype, float scale, void* workspace, size_t workspace_bytes,
                               int32_t sm_budget, void* stream, uint32_t* status_dev);

/* ---- attention of several new tokens a sequence over the cache ----
 * Rows cu_seqlens[s] .. cu_seqlens[s+1] - 1 of q are the LAST tokens among places 0 .. seq_lens[s] - 1 of sequence s (their keys and values stored before): the
 * next chunk of a prompt, a draft to be verified, single tokens between them.  Row i of n sees places 0 .. i + seq_lens[s] - n; a row that sees nothing (a sequence
 * shorter than its chunk, or of length 0 or less) gets 0, and rows that cu_seqlens does not name are left alone.  out = softmax(scale * q k^T) v with the types and
 * the precision of eas_cache_attention; it overlaps no input.  Of `seqs` it takes cu_seqlens and seq_lens; they are read when the call's work runs.
 * Which kernels run is decided by n_seqs, n_rows, max_new, the heads and max_blocks: the same inputs give the same bits for any sm_budget and in every replay, but
 * with another max_new, another width of the table or other sequences beside it a sequence's last bits may differ.
 * n_rows: rows of q that exist (a bound on cu_seqlens).  max_new: the most new tokens that a sequence has: a sequence with more is not computed and raises the
 * status word to EAS_DEVICE_CACHE_RANGE.  Any bound is right (n_rows, if nothing is known); the kernels are chosen by it, so the exact number is the fastest.
 * workspace: device scratch of eas_cache_chunk_workspace_bytes() (0 on bad arguments), 256-byte aligned; its contents do not matter and nothing of it is used
 * by a later call, but calls that may run at the same time need one each.
 * Limits (UNSUPPORTED): 128 query heads a key/value head, 2^30 places a sequence (max_blocks * block_size), n_rows * n_heads below 2^31. */
size_t eas_cache_chunk_workspace_bytes(const eas_cache* cache, int32_t n_seqs, int32_t n_rows, int32_t max_new, int32_t n_heads);
eas_status eas_cache_chunk_attention(const eas_cache* cache, const eas_cache_seqs* seqs, const void* q, int64_t ld_q, void* out, int64_t ld_out,
                                     int32_t n_rows, int32_t max_new, int32_t n_heads, int32_t dtype, float scale, void* workspace, size_t workspace_bytes,
                                     int32_t sm_budget, void* stream, uint32_t* status_dev);

/* ---- rotary positions with several axes ----
 * The first rotary_dim dimensions of a head are pairs; pair i turns by angle = position * inv_freq[i], the token's position along axis[i]:
 *   a' = scale (a cos angle - b sin angle),  b' = scale (b cos angle + a sin angle);  the other dimensions stay as they are.
 * One axis for text; time, height and width for the embeddings of images and clips.  Angles are exact to 2^-32 turns for every 32-bit position; the arithmetic is fp32. */
enum { EAS_ROTARY_HALVES = 0,      /* pair i: dimensions i and i + rotary_dim / 2 */
       EAS_ROTARY_NEIGHBOURS = 1   /* dimensions 2 i and 2 i + 1 */ };
typedef struct {
  int32_t head_dim;       /* 64 or 128 */
  int32_t rotary_dim;     /* a multiple of 16, at most head_dim */
  int32_t pairing;        /* EAS_ROTARY_* */
  int32_t n_axes;         /* 1 .. 4 */
  const double* inv_freq; /* host [rotary_dim / 2], radians a position, finite */
  const int32_t* axis;    /* host [rotary_dim / 2], 0 .. n_axes - 1 (NULL: all 0) */
  float scale;            /* > 0, finite; 1 as a rule */
} eas_rotary_desc;

typedef struct eas_rotary eas_rotary; /* opaque: the frequencies; host memory only, good for any device */
eas_status eas_rotary_create(const eas_rotary_desc* desc, eas_rotary** out);
void eas_rotary_destroy(eas_rotary* rotary);

typedef struct {
  const void* q;          /* device [n_rows, n_heads * head_dim], distance ld_q; NULL with n_heads 0 */
  const void* k;          /* device [n_rows, n_kv_heads * head_dim], distance ld_k; NULL with n_kv_heads 0 */
  void* out_q;            /* as q, as k: the same address and distance (in place), or memory that overlaps no input */
  void* out_k;
  int64_t ld_q, ld_k, ld_out_q, ld_out_k;
  const int32_t* positions; /* device [n_axes][n_rows], distance ld_positions (0: one row for all axes) */
  int64_t ld_positions;
  int32_t n_rows, n_heads, n_kv_heads, dtype;
  int32_t inverse;        /* 1: by -angle, which takes the rotation back; times scale, the gradient's way through it */
} eas_rotary_inputs;

/* out = rotated q and k, rounded once to the data type.  Errors (nothing launched): INVALID_ARG, UNSUPPORTED, ARCH, CUDA. */
eas_status eas_rotary_apply(const eas_rotary* rotary, const eas_rotary_inputs* in, int32_t sm_budget, void* stream);

/* eas_cache_store of the rotated keys and the values, and the rotated queries to out_q (n_heads 0: none), in one launch.  The keys are rotated in fp32 and
 * rounded once, to their number in the cache.  in: k [n_rows, n_kv_heads of the cache], out_k NULL, inverse 0; positions NULL: a token's place in its sequence,
 * along every axis.  Queries of rows that cu_seqlens does not name are left alone; those whose key has no place in the cache are written all the same. */
eas_status eas_cache_append(const eas_cache* cache, const eas_cache_seqs* seqs, const eas_rotary* rotary, const eas_rotary_inputs* in, const void* v, int64_t ld_v,
                            int32_t sm_budget, void* stream, uint32_t* status_dev);

#ifdef __cplusplus
}
#endif
#endif /* EAS_LANGUAGE_H_ */
