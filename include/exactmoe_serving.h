/*
 * exactmoe_serving.h -- decoding of many sequences at once around the W4A16
 * routed-expert layer: a paged key-value cache, the append of new keys and
 * values with the rotary positions on the way, the attention of one new token
 * per row over that cache, and what stands between the logits and the next
 * token (penalties for repeated tokens, biases, grammar masks).
 *
 * The paper decodes with a KV cache and SDPA attention (Sec. 4.1-4.2) and
 * says no more about either; these calls are the batched form of the synthetic
 * decoder's own steps (exactmoe_decoder.h), whose emoe_decoder_forward_paged
 * makes them.  Conventions of exactmoe.h apply (status codes, caller-owned
 * buffers, asynchrony on `stream`, which belongs to the current device).  No
 * call allocates or synchronizes, so each may be captured into a HIP graph.
 */
#ifndef EXACTMOE_SERVING_H
#define EXACTMOE_SERVING_H

#include "exactmoe_decoder.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  E4M3 is the OCP 8-bit float (largest value 448, no infinity). */
enum emoe_dtype { EMOE_F32 = 0, EMOE_BF16 = 1, EMOE_F16 = 2, EMOE_E4M3 = 3 };

/* ---------------------------------------------------------------- the paged cache */
/* Keys and values of many sequences in pages of `page_size` positions, taken
 * from one pool.  Element (page, slot, head, dim) of k_pages and of v_pages is
 * at page * page_stride + slot * slot_stride + head * head_stride + dim
 * (elements).  Pages are the outermost axis; slots and heads may come in
 * either order, and gaps are allowed.  A page table row lists the pages of one
 * sequence: position p lies in slot p % page_size of page
 * table[p / page_size].  Sequences may share pages.
 * Entries outside [0, n_pages) mean "no page": nothing is appended there and
 * the attention leaves those positions out, so pages behind a sliding window
 * can be given back.
 * E4M3 caches hold x / scale with one scale per key head; k_scale and v_scale
 * are device f32 [n_kv_heads], both NULL for scales of 1 and for 16-bit caches. */
typedef struct emoe_paged_kv {
  void* k_pages;
  void* v_pages;
  const float* k_scale;
  const float* v_scale;
  int64_t page_stride, slot_stride, head_stride;
  int32_t dtype;       /* EMOE_BF16, EMOE_F16 or EMOE_E4M3 */
  int32_t n_pages;
  int32_t page_size;   /* a power of two, 8 .. 1024 */
  int32_t n_kv_heads;
  int32_t head_dim;    /* 64, 128 or 256 */
} emoe_paged_kv;

/* EMOE_OK if the cache is one that these calls take: 16-byte aligned pages and
 * strides, a page within 2^30 bytes, axes that do not overlap. */
int32_t emoe_check_paged_kv(const emoe_paged_kv* kv);

/* ---------------------------------------------------------------- append */
/* For token t at position p = positions[t] of sequence s = seqs[t]:
 *   the first rotary_dim dimensions of every head of q and k are turned by the
 *   angles p * inv_freq[i] (fp64, as are their sine and cosine), in pairs
 *   (i, i + rotary_dim/2), or (2i, 2i+1) when interleaved; the others stay;
 *   q_out[t] = the turned q, rounded once;
 *   the turned k and v go to the cache at position p of sequence s, rounded
 *   once to its type (E4M3: x / scale, saturated at +-448, NaN kept).
 * Tokens with s outside [0, n_seqs) or p < 0 are padding: nothing of theirs is
 * written.  Tokens whose position has no page, or lies past the table, get
 * their q_out and append nothing.  No two tokens of a call may have the same
 * position of the same sequence, nor may their pages be shared: that slot
 * would hold a mix of both. */
typedef struct emoe_paged_append_args {
  const void* q;              /* device [tokens][n_heads][head_dim], or NULL for none */
  const void* k;              /* device [tokens][n_kv_heads][head_dim] */
  const void* v;
  void* q_out;                /* device [tokens][n_heads][head_dim]; may be q itself */
  const int32_t* positions;   /* device [tokens] */
  const int32_t* seqs;        /* device [tokens], or NULL: token t is of sequence t */
  const int32_t* page_table;  /* device [n_seqs][table_width] */
  const double* inv_freq;     /* device [rotary_dim / 2]; |p * inv_freq| below 2^31 */
  int64_t q_stride, k_stride, v_stride, q_out_stride; /* between tokens, elements, multiples of 8 */
  int64_t table_stride;       /* between the table's rows, elements */
  int32_t dtype;              /* of q, k, v and q_out: EMOE_BF16 or EMOE_F16; a 16-bit cache has the same */
  int32_t tokens;             /* >= 0 */
  int32_t n_heads;            /* of q, 1 .. 2^20; without a q not read */
  int32_t n_seqs, table_width;
  int32_t rotary_dim;         /* a multiple of 16, 0 (no rotation) .. head_dim */
  int32_t interleaved;        /* 0 or 1 */
} emoe_paged_append_args;

int32_t emoe_paged_append(const emoe_paged_kv* kv, const emoe_paged_append_args* args,
                          hipStream_t stream);

/* ---------------------------------------------------------------- attention */
/* For row r (sequence s = seqs[r], n = lengths[r] keys) and query head h, with
 * key head g = h / (n_heads / n_kv_heads):
 *   keys j in [max(0, n - window), n) (window 0: all) that have a page;
 *   z_j = scale * k_scale[g] * (q . k_j),  w = softmax(z),
 *   out[r][h] = v_scale[g] * sum_j w_j v_j, rounded once;
 *   lse[r][h] = log sum_j exp(z_j).
 * Products of 16-bit values are summed in fp32, the softmax is fp32, its
 * weights enter the second product as two 16-bit halves: to 2^-16 of each, over
 * fp16 pages down to 2^-64 of the largest (an infinity among the values that a
 * row sees makes its dimension infinite or NaN, and so may the sums of values
 * above 2^88).  A row without keys
 * (n <= 0, s outside [0, n_seqs), no page) has out = 0 and lse = -inf.  n is
 * cut to max_keys and to the table.  What lies in slots without a key (never
 * written, NaN) has no effect.  The last token's own key is one of the n:
 * append first, then attend with n = position + 1.  Several rows may be of one
 * sequence (a prompt's tokens, each with its own n).  Sums are joined in an
 * order that the lengths alone decide, so equal calls give equal bits. */
typedef struct emoe_paged_attention_args {
  const void* q;              /* device [rows][n_heads][head_dim] */
  void* out;                  /* device [rows][n_heads][head_dim] */
  float* lse;                 /* device [rows][n_heads], or NULL */
  const int32_t* lengths;     /* device [rows] */
  const int32_t* seqs;        /* device [rows], or NULL: row r is of sequence r */
  const int32_t* page_table;  /* device [n_seqs][table_width] */
  int64_t q_stride, out_stride; /* between rows, elements, multiples of 8 */
  int64_t table_stride;
  float scale;                /* of the scores, e.g. 1 / sqrt(head_dim); within +-2e38 */
  int32_t dtype;              /* of q and out: EMOE_BF16 or EMOE_F16; a 16-bit cache has the same */
  int32_t rows;               /* >= 0 */
  int32_t n_heads;            /* a multiple of n_kv_heads, at most 2^20 */
  int32_t n_seqs, table_width;
  int32_t max_keys;           /* bound of lengths[], 0 .. 2^30: how finely the call is split */
  int32_t window;             /* >= 0 */
} emoe_paged_attention_args;

/* Workspace of the attention.  Its first EMOE_SERVING_TICKET_BYTES count
 * finished workgroups: zero them once, before the workspace's first call; every
 * call leaves them zero.  The rest needs no initial value.  One workspace may
 * serve attention calls of any sizes, captured or not, as long as no two of them
 * overlap in time, and no other use. */
#define EMOE_SERVING_TICKET_BYTES 131072
size_t emoe_paged_attention_workspace_bytes(const emoe_paged_kv* kv, int32_t rows, int32_t n_heads,
                                            int32_t max_keys);

int32_t emoe_paged_attention(const emoe_paged_kv* kv, const emoe_paged_attention_args* args,
                             void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------- logits */
/* For row b and token id v, in fp32, one rounding after each operation, in this
 * order (a NULL array leaves its step out):
 *   x = logits[b][v];
 *   v in history[b]:               x = x > 0 ? x / repetition[b] : x * repetition[b];
 *   c = times v was generated:     x = x - frequency[b] * c;  c > 0: x = x - presence[b];
 *   v in bias_ids[b]:              x = x + its bias_values (an id listed twice: the later one);
 *   bit v of the row's mask is 0:  x = -inf;
 *   out[b][v] = x, rounded to its type;
 *   next_token[b] = the smallest v whose x (before that rounding) is the
 *   largest of the row; NaN is never chosen; -1 when nothing exceeds -inf.
 * history[b] holds history_lengths[b] ids, the first prompt_lengths[b] of them
 * the prompt's and the others generated; ids outside [0, vocab) are skipped,
 * lengths are cut to the arrays' widths. */
typedef struct emoe_logits_args {
  const void* logits;              /* device [rows][vocab] */
  void* out;                       /* device [rows][vocab]; may be logits itself */
  int32_t* next_token;             /* device [rows], or NULL */
  const int32_t* history;          /* device [rows][history_width], or NULL */
  const int32_t* history_lengths;  /* device [rows], or NULL: history_width each */
  const int32_t* prompt_lengths;   /* device [rows], or NULL: 0 each */
  const float* repetition;         /* device [rows], or NULL */
  const float* presence;
  const float* frequency;
  const int32_t* bias_ids;         /* device [rows][bias_width], or NULL */
  const float* bias_values;        /* device [rows][bias_width] */
  const int32_t* bias_counts;      /* device [rows], or NULL: bias_width each */
  const uint32_t* mask;            /* device [n_masks][>= ceil(vocab/32)] bits, 1 = allowed, or NULL */
  const int32_t* mask_rows;        /* device [rows], the mask of each row, outside [0, n_masks): none;
                                      or NULL: row b has mask b (n_masks >= rows) */
  int64_t logits_stride, out_stride, history_stride, bias_stride, mask_stride; /* elements */
  int32_t dtype;                   /* of logits and out: EMOE_F32, EMOE_BF16 or EMOE_F16 */
  int32_t rows, vocab;             /* >= 0, >= 1 */
  int32_t history_width, bias_width, n_masks;  /* bias_width below 2^23 */
} emoe_logits_args;

/* Workspace (needed with next_token only): what the workgroups of a row hand
 * over to each other.  Zero it once, before its first call; every call leaves it
 * zero.  Over one that was not zeroed calls end, but their tokens are undefined,
 * and so are those of later calls until it is.  It may serve calls of any sizes, captured or not, as long as no two of
 * them overlap in time, and no other use. */
size_t emoe_process_logits_workspace_bytes(int32_t rows, int32_t vocab);

int32_t emoe_process_logits(const emoe_logits_args* args, void* workspace, size_t workspace_bytes,
                            hipStream_t stream);

/* ---------------------------------------------------------------- the decoder over a paged cache */
/* Tokens of many sequences in one call of the synthetic decoder: prompts,
 * parts of prompts and decode steps, mixed as the caller likes. */
typedef struct emoe_decoder_batch {
  const int32_t* tokens;      /* device [n_tokens], ids outside [0, V) are clamped */
  const int32_t* positions;   /* device [n_tokens] */
  const int32_t* seqs;        /* device [n_tokens], or NULL: token t is of sequence t */
  const int32_t* page_table;  /* device [n_seqs][table_width], for every layer */
  const int32_t* out_rows;    /* device [n_out]: tokens whose logits are wanted (clamped to the call's
                                 tokens), or NULL: all (n_out = n_tokens) */
  int64_t table_stride;
  int32_t n_tokens, n_seqs, table_width;
  int32_t n_out;              /* 1 .. n_tokens */
  int32_t max_keys;           /* bound of positions[] + 1, 0 .. 2^30 */
} emoe_decoder_batch;

/* Workspace of emoe_decoder_forward_paged; needs no initial value, since the
 * call clears what has to be zero. */
size_t emoe_decoder_paged_workspace_bytes(const emoe_decoder_dims* dims, int32_t n_tokens,
                                          int32_t n_out, int32_t max_keys);

/* As emoe_decoder_forward, with emoe_paged_append and emoe_paged_attention per
 * layer in place of the contiguous cache, and emoe_process_logits at the end.
 *   kv: host array of n_layers caches with n_heads key heads of head_dim, bf16
 *       or e4m3; pages are written at the tokens' positions, and the positions
 *       before them that a token attends to must hold earlier tokens';
 *   logits: device f32 [n_out][V], after processing;
 *   process: penalties, biases and masks of the n_out rows (the arrays and
 *       their widths and strides; the other fields are not read), or NULL;
 *   next_token: device int32 [n_out], or NULL.
 * A token with seqs[t] outside [0, n_seqs) or a negative position is padding:
 * it appends nothing and attends to nothing; its logits mean nothing.
 * Captured into a graph as emoe_moe_forward is: with fully resident experts,
 * and up to 4 tokens per call (more take rocBLAS, whose calls choose memory). */
int32_t emoe_decoder_forward_paged(emoe_decoder* dec, const emoe_paged_kv* kv,
                                   const emoe_decoder_batch* batch, float* logits,
                                   const emoe_logits_args* process, int32_t* next_token,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream,
                                   emoe_stats* stats);

#ifdef __cplusplus
}
#endif
#endif /* EXACTMOE_SERVING_H */
