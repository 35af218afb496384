/*
 * exactmoe_drafts.h -- several drafted tokens of a sequence checked in one step,
 * over the paged caches of exactmoe_serving.h.  A drafter proposes a tree of
 * tokens behind each sequence; the model sees all of them in one call, and those
 * that it would have chosen itself stay:
 *   emoe_paged_append_axes     stores the nodes' keys and values, node i at cache
 *                              position n + i with the angle of position n + depth;
 *   emoe_paged_tree_attention  attends from every node to the sequence and to the
 *                              node's own ancestors;
 *   emoe_process_logits        chooses the token that follows each node;
 *   emoe_accept_drafts         walks down the tree as long as the drafts agree;
 *   emoe_paged_compact         moves the accepted nodes' keys and values to the
 *                              positions that they then have, in all layers.
 * emoe_paged_fork begins sequences where others stand (beams, several answers to
 * one prompt).  Conventions of exactmoe_serving.h apply: no call allocates or
 * synchronizes, so each may be captured into a HIP graph.  emoe_decoder_forward_paged
 * takes no trees: the append and the attention here are for a program that calls its
 * layers itself.
 *
 * A tree of T nodes (0 .. 64) is given by what its nodes see: bit j of tree[i] is
 * set if node i sees node j, as a rule its ancestors and itself.  The depth of
 * node i is the number of nodes before it (j < i) that it sees, its parent the
 * last of those.  Where `tree` is NULL every node sees those before it and itself
 * (a chain of drafts, a part of a prompt).  The rows of a call's trees stand
 * behind each other: tree g has rows starts[g] .. starts[g + 1] - 1 of the call's
 * (starts NULL: max_nodes rows each), of which the first max_nodes count.  Rows
 * of no tree are not read, and what belongs to them is left as it was.
 */
#ifndef EXACTMOE_DRAFTS_H
#define EXACTMOE_DRAFTS_H

#include "exactmoe_serving.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EMOE_MAX_NODES 64

/* ---------------------------------------------------------------- append */
/* As emoe_paged_append, which see, but for the angles: pair i turns by
 *   angles[t][axes[i]] * inv_freq[i]  (fp64; below 2^31 in magnitude)
 * in place of positions[t] * inv_freq[i]; positions[t] says where the token lies in
 * its sequence, and nothing else.  With one axis the angles are those of drafted
 * nodes (n + depth); images and videos have an axis each for time, height and
 * width, and axes[] deals the pairs out among them.  Angles may be negative; a
 * pair whose axis lies outside [0, n_axes) does not turn. */
typedef struct emoe_paged_axes {
  const int32_t* angles;  /* device [tokens][n_axes] */
  const int32_t* axes;    /* device [rotary_dim / 2], or NULL: axis 0 each */
  int64_t angle_stride;   /* between tokens, elements */
  int32_t n_axes;         /* >= 1 */
} emoe_paged_axes;

int32_t emoe_paged_append_axes(const emoe_paged_kv* kv, const emoe_paged_append_args* args,
                               const emoe_paged_axes* axes, hipStream_t stream);

/* ---------------------------------------------------------------- attention */
/* For tree g (sequence s = seqs[g], n = lengths[g] keys before the tree, T nodes
 * at the cache positions n .. n + T - 1), node i of it and query head h, with key
 * head c = h / (n_heads / n_kv_heads):
 *   node i stands at p_i = n + its depth, the sequence's key j at p_j = j;
 *   it sees the keys j < n and the nodes of its mask, of both those that have a
 *   page and, with a window, p_j > p_i - window;
 *   x_j = scale * k_scale[c] * (q . k_j),  x_j = cap * tanh(x_j / cap) if cap > 0,
 *   z_j = x_j - slopes[h] * |p_i - p_j|,   w = softmax(z),
 *   out = v_scale[c] * sum_j w_j v_j, rounded once;  lse = log sum_j exp(z_j).
 * A node that sees nothing has out = 0 and lse = -inf; so has every node of a
 * sequence outside [0, n_seqs) or of a negative length.  Keys from position
 * max_keys on, or past the table, are not seen.  What a node does not see has no
 * effect on it, whatever it holds (NaN, infinities, nothing ever written).
 * Precision as in emoe_paged_attention (of an infinite value that a node sees, its
 * own dimension of the output is infinite or NaN).  Sums are joined in an order that the
 * lengths and numbers of nodes alone decide, so equal calls give equal bits. */
typedef struct emoe_paged_tree_args {
  const void* q;              /* device [rows][n_heads][head_dim] */
  void* out;                  /* device [rows][n_heads][head_dim] */
  float* lse;                 /* device [rows][n_heads], or NULL */
  const int32_t* lengths;     /* device [trees] */
  const int32_t* starts;      /* device [trees + 1], or NULL: tree g has rows g * max_nodes .. */
  const int32_t* seqs;        /* device [trees], or NULL: tree g is of sequence g */
  const uint64_t* tree;       /* device [rows], or NULL: chains */
  const float* slopes;        /* device [n_heads], or NULL: 0 */
  const int32_t* page_table;  /* device [n_seqs][table_width] */
  int64_t q_stride, out_stride; /* between rows, elements, multiples of 8 */
  int64_t table_stride;
  float scale;                /* of the scores, e.g. 1 / sqrt(head_dim); within +-2e38 */
  float cap;                  /* 0: none; else 2^-60 .. 2^60 */
  int32_t dtype;              /* of q and out: EMOE_BF16 or EMOE_F16; a 16-bit cache has the same */
  int32_t rows, trees;        /* >= 0 */
  int32_t n_heads;            /* a multiple of n_kv_heads, at most 2^20; those of a key head times
                                 max_nodes at most 2^20 */
  int32_t n_seqs, table_width;
  int32_t max_keys;           /* bound of lengths[] and nodes together, 0 .. 2^30 */
  int32_t max_nodes;          /* bound of a tree's nodes, 1 .. 64; the call is laid out for trees of
                                 so many, so that a bound far above them costs time */
  int32_t window;             /* >= 0; 0: none */
} emoe_paged_tree_args;

/* Workspace of the tree attention; needs no initial value.  One workspace may
 * serve calls of any sizes, captured or not, as long as no two of them overlap in
 * time. */
size_t emoe_paged_tree_attention_workspace_bytes(const emoe_paged_kv* kv, int32_t trees,
                                                 int32_t n_heads, int32_t max_keys,
                                                 int32_t max_nodes);

int32_t emoe_paged_tree_attention(const emoe_paged_kv* kv, const emoe_paged_tree_args* args,
                                  void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------- acceptance */
/* For tree g, from node 0 on: the next node is the first child c of the present
 * one (node c's parent is the present one) whose token is the one chosen after the
 * present one, tokens[c] == chosen[present]; negative choices (no token was
 * allowed) agree with none.  Node 0, the token that the last step gave, counts as
 * accepted.
 *   accepted[g] = m, the nodes on that way (0 for a tree without nodes);
 *   path[g][i] = the i-th of them, new_tokens[g][i] = the token chosen after it, for
 *   i < m (m tokens that the model itself gives), both -1 for m <= i < max_nodes;
 *   new_lengths[g] = lengths[g] + m. */
typedef struct emoe_accept_args {
  const int32_t* tokens;   /* device [rows], the drafted token of each node */
  const int32_t* chosen;   /* device [rows], the model's choice after each node */
  const uint64_t* tree;    /* device [rows], or NULL: chains */
  const int32_t* starts;   /* device [trees + 1], or NULL */
  const int32_t* lengths;  /* device [trees], or NULL with new_lengths NULL */
  int32_t* path;           /* device [trees][max_nodes] */
  int32_t* accepted;       /* device [trees] */
  int32_t* new_tokens;     /* device [trees][max_nodes], or NULL */
  int32_t* new_lengths;    /* device [trees], or NULL; may be lengths itself */
  int64_t path_stride, new_tokens_stride; /* between trees, elements */
  int32_t rows, trees, max_nodes;
} emoe_accept_args;

int32_t emoe_accept_drafts(const emoe_accept_args* args, hipStream_t stream);

/* ---------------------------------------------------------------- moves in the caches */
/* Both calls act on n_layers caches (a host array) of the same type, sizes and
 * strides, whose page tables are one and the same; what is stored in them, keys and
 * values of all layers, lies in places of its own. */

/* For tree g of sequence s = seqs[g] and every i < accepted[g] with path[g][i] > i:
 * position lengths[g] + i of s takes the key and the value that position
 * lengths[g] + path[g][i] held before the call.  (lengths[] are those before the
 * acceptance; path and accepted as emoe_accept_drafts gives them, accepted cut to
 * [0, max_nodes].  What path holds need not ascend.)  Trees of a sequence outside
 * [0, n_seqs) or of a negative length are skipped, and so are moves from or to a
 * position without a page.  The positions that a tree's moves write or read belong
 * to that tree alone: no sequence comes twice, and no other one shares their
 * pages. */
typedef struct emoe_compact_args {
  const int32_t* lengths;     /* device [trees] */
  const int32_t* path;        /* device [trees][max_nodes] */
  const int32_t* accepted;    /* device [trees] */
  const int32_t* seqs;        /* device [trees], or NULL: tree g is of sequence g */
  const int32_t* page_table;  /* device [n_seqs][table_width] */
  int64_t path_stride, table_stride;
  int32_t trees, max_nodes, n_seqs, table_width;
} emoe_compact_args;

int32_t emoe_paged_compact(const emoe_paged_kv* kv, int32_t n_layers, const emoe_compact_args* args,
                           hipStream_t stream);

/* Row f of new_table becomes a sequence that goes on where the first n = lengths[f]
 * positions of sequence p = parents[f] of page_table end:
 *   its first n / page_size entries are the parent's (the pages are shared);
 *   if a part of a page is left (n % page_size > 0), the next entry is fresh[f], and
 *   the parent's keys and values of that part are copied there in all layers; the
 *   rest of that page is left as it was.  A fresh[f] outside [0, n_pages) (or fresh
 *   NULL) has the child go on in the parent's own page, as one of a parent's
 *   children may.  A parent's page that is missing stays missing;
 *   all further entries are -1.
 * n is cut to the table.  A parent outside [0, n_seqs) or a negative length leaves
 * a row of -1.  new_table may not overlap page_table, from the first row's start to the
 * last one's end: rows of one between rows of the other are refused too.  No fresh page
 * comes twice, nor may it hold anything of a parent's. */
typedef struct emoe_fork_args {
  const int32_t* page_table;  /* device [n_seqs][table_width] */
  const int32_t* parents;     /* device [forks] */
  const int32_t* lengths;     /* device [forks] */
  const int32_t* fresh;       /* device [forks], or NULL */
  int32_t* new_table;         /* device [forks][table_width] */
  int64_t table_stride, new_table_stride;
  int32_t forks, n_seqs, table_width;
} emoe_fork_args;

int32_t emoe_paged_fork(const emoe_paged_kv* kv, int32_t n_layers, const emoe_fork_args* args,
                        hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* EXACTMOE_DRAFTS_H */
