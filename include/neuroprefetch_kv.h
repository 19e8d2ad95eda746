/*
 * neuroprefetch_kv.h -- C ABI of the attention side of a layer: a paged
 * key-value cache and the attention that reads it, next to the MLP calls of
 * neuroprefetch.h (whose conventions on errors, streams, memory and alignment
 * hold here too).
 *
 * The method keeps attention resident and dense while the MLP is sparse
 * (Sec. 3.1: "sparse suffix layers: resident attention and sparse MLP").  One
 * layer of one step is np_kv_append -> np_attn_decode (or np_attn_prompt) ->
 * output projection -> np_sparse_mlp / np_dense_mlp, after one np_kv_extend
 * per step:
 *
 *   np_kv_extend    room for the step's new tokens in every sequence: pages
 *                   from the free ones; a shared last page is copied first
 *   np_kv_append    rotary positions on the new queries and keys; keys and
 *                   values into their pages (np_kv_append_norm: a norm of each
 *                   query and key head before that)
 *   np_attn_decode  attention of one new token per sequence
 *                   (np_attn_decode_shared: of sequences that share a prefix)
 *   np_attn_prompt  causal attention of many new tokens per sequence, packed
 *   np_kv_read      tokens' keys and values back out of their pages
 *
 * and between steps np_kv_fork (a sequence that shares a prefix of another),
 * np_kv_free (a finished sequence) and np_kv_compact (the pages in use moved
 * to the low end of the pool).
 *
 * The cache (np_kv_shape)
 * -----------------------
 *  L = layers, Hq = heads, Hkv = kv_heads (query head i reads key-value head
 *  i / (Hq / Hkv)), D = head_dim, P = page_size (tokens a page holds),
 *  N = n_pages, S = max_seqs, M = seq_pages (pages a sequence can have),
 *  w = dtype of queries, keys, values and outputs, plus NP_KV_E4M3 for a cache
 *  of 8-bit elements.
 *  Requirements: L >= 1; Hkv divides Hq <= 1024; D a multiple of 8, 8..256;
 *  P one of 16, 32, 64, 128, 256; 1 <= N <= 2^20; 1 <= S <= 4096; M >= 1 and
 *  M * P <= 2^30; with NP_KV_E4M3, D a multiple of 16.  Any violation is
 *  NP_ERR_INVALID_ARG.
 *
 *  pool [L][N][2][Hkv][P][D] of type w, device: page p of layer l holds the
 *  keys ([0]) and the values ([1]) of P consecutive positions of a sequence,
 *  head by head.  The pool and one layer of it may be larger than 4 GiB.
 *  With NP_KV_E4M3 the pool is bytes [L][N][2][Hkv][P D + P]: of each head, P
 *  rows of D elements (OCP e4m3: 4 exponent and 3 mantissa bits, 448 the
 *  largest, no infinities), then a byte b for each row, whose elements x stand
 *  for x 2^(b - 127).  What is appended is first rounded to w, as for a plain
 *  cache; a row whose largest finite magnitude is m then takes the least b >= 1
 *  with m <= 448 2^(b - 127), and each value the nearest element, the even one
 *  of two as near, except that the elements stop at 240 where 256 2^(b - 127)
 *  is past the largest number of w.  A value that is not finite becomes NaN.  An
 *  element is off by at most 2^-4 of its value, or 2^(b - 137) where that is
 *  more (and by 1/16 of w's largest number, next to it).  All calls here take
 *  such a cache; in place of w's values the attention calls see what the
 *  elements stand for, which w holds exactly.
 *  np_kv_state, device int32: page_table [S][M] (page of positions
 *  [j P, (j+1) P) of sequence s, or -1), kv_len [S] (tokens reserved), refs
 *  [N] (how many sequences hold a page; 0: free).  np_kv_append and the
 *  attention calls read page_table alone, so a caller may also keep it by
 *  other means than the calls here.
 *
 * A batch (np_kv_batch)
 * ---------------------
 *  The new tokens of n_seq sequences, packed: row b brings tokens
 *  cu_tokens[b] .. cu_tokens[b+1]-1 of the token arrays (cu_tokens NULL: one
 *  token each) for sequence seqs[b] (seqs NULL: sequence b).  Its i-th token
 *  has position pos0[b] + i and sees the keys of its own sequence at positions
 *  max(0, pos - window + 1) .. pos (window 0: 0 .. pos), its own among them.
 *  pos0[b] < 0: the row is not served in this call: nothing is appended for
 *  it, and its attention outputs are zero.
 */
#ifndef NEUROPREFETCH_KV_H
#define NEUROPREFETCH_KV_H

#include "neuroprefetch.h"

#ifdef __cplusplus
extern "C" {
#endif

/* np_kv_shape.dtype: w, or w | NP_KV_E4M3 */
#define NP_KV_E4M3 0x100

typedef struct np_kv_shape {
  int32_t layers;    /* L */
  int32_t heads;     /* Hq */
  int32_t kv_heads;  /* Hkv */
  int32_t head_dim;  /* D */
  int32_t page_size; /* P */
  int32_t n_pages;   /* N */
  int32_t max_seqs;  /* S */
  int32_t seq_pages; /* M */
  int32_t dtype;     /* np_dtype, | NP_KV_E4M3 for 8-bit elements */
} np_kv_shape;

typedef struct np_kv_state {
  int32_t* page_table; /* [S][M] */
  int32_t* kv_len;     /* [S] */
  int32_t* refs;       /* [N] */
} np_kv_state;

/* n_seq, n_tokens (rows of the token arrays), max_tokens (no row brings
 * more) and max_len (no position of the batch reaches it) are host values;
 * max_len bounds the keys a call covers and max_tokens only picks kernels.
 * Work is split by them: the closer they are, the better it is spread.
 * The arrays are device int32, 4-byte aligned; each may change between calls
 * without the host knowing.  Device-side checks: a sequence outside [0, S), a
 * cu_tokens that descends or leaves [0, n_tokens], and a position at or past
 * max_len or M P set NP_DEVERR_STATE, and the row is not served (one whose
 * cu_tokens are bad has no tokens; a token that several others then claim is
 * appended for the first of them, and its outputs are those of any); a page
 * outside [0, N) where a token sees keys sets NP_DEVERR_NOT_RESIDENT (its keys
 * count as not visible).  Outputs of tokens that no row has are not written.  At
 * most 2^24 tokens and 2^30 query heads in all. */
typedef struct np_kv_batch {
  int32_t n_seq;
  int32_t n_tokens;
  int32_t max_tokens;
  int32_t max_len;
  const int32_t* seqs;      /* [n_seq] or NULL */
  const int32_t* cu_tokens; /* [n_seq + 1] or NULL (then n_tokens == n_seq) */
  const int32_t* pos0;      /* [n_seq] */
} np_kv_batch;

/* A layer's new queries, keys and values (device, type w): token t's head i
 * starts at q + t * q_stride + i * D (strides in elements, multiples of 8 for
 * 16-bit types and 4 for fp32, so views of one fused projection can be
 * given).  q_out receives the rotated queries (it may be q itself, with the
 * same stride; no other overlap).  Of a batch without tokens (here and in the
 * attention calls) the arrays may be NULL; such a call enqueues nothing. */
typedef struct np_kv_rows {
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  int64_t q_stride;
  int64_t k_stride;
  int64_t v_stride;
  int64_t q_out_stride;
} np_kv_rows;

/* Rotary positions: cos and sin, device fp32 [max_pos][dim / 2], 16-byte
 * aligned; the first dim elements of each query and key head are turned in
 * pairs (i, i + dim/2), or (2i, 2i + 1) when interleaved != 0:
 *     a' = a cos - b sin,  b' = b cos + a sin    (fp32, rounded once to w).
 * dim: a multiple of 16, 16..D.  A token at or past max_pos sets
 * NP_DEVERR_STATE and is not appended. */
typedef struct np_rotary {
  const float* cos;
  const float* sin;
  int32_t dim;
  int32_t max_pos;
  int32_t interleaved;
} np_rotary;

/* Norms of the query and key heads: q_weight and k_weight, device, type w, [D],
 * 16-byte aligned, each NULL for ones; a head x becomes
 *     x_d weight_d / sqrt(mean of x_d^2 over the head + eps)    (fp32).
 * eps: finite, >= 0.  (A head of zeros stays zero, also when eps is 0; one with a
 * NaN becomes NaN.) */
typedef struct np_qk_norm {
  const void* q_weight;
  const void* k_weight;
  float eps;
} np_qk_norm;

/* Rows of a batch that share a prefix (np_attn_decode_shared): lead and prefix,
 * device int32 [n_seq], 4-byte aligned.  lead[b] is the first row of row b's
 * group: the rows of a group lie next to each other and all name the first of
 * them, which names itself.  Sequence seqs[b] then has the same keys and values
 * at positions 0 .. prefix[lead[b]] - 1 as sequence seqs[lead[b]] (as np_kv_fork
 * makes them: the same pages, and copies of a partly filled last one); those of
 * the latter are read.  prefix of other rows is not read; of a prefix past max_len the
 * positions below it count.  max_prefix: a host value that no group's prefix exceeds.  A lead outside [0, b], one that does not
 * name itself, whose rows do not lie next to each other, whose sequence is outside
 * [0, S), or whose prefix is outside [0, max_prefix] sets NP_DEVERR_STATE, and the
 * row is computed by itself, from its own pages, as in np_attn_decode. */
typedef struct np_kv_shared {
  int32_t max_prefix;
  const int32_t* lead;
  const int32_t* prefix;
} np_kv_shared;

/* Validates a shape (the requirements above).  Host only. */
np_status np_kv_shape_check(const np_kv_shape* shape);

/* Bytes of device workspace ("dev_ws") the calls below need: one workspace
 * per stream of calls, zeroed or given to np_kv_reset (of any shape) before
 * its first use.  It starts with the sticky error word that np_device_error
 * reads.  Caches of several shapes may take turns on one workspace of at least
 * the largest size any of them needs; the error word is then theirs together.
 * The calls of neuroprefetch.h need a workspace of their own.  Host only. */
np_status np_kv_workspace_size(const np_kv_shape* shape, size_t* dev_ws_bytes);

/* An empty cache: page_table -1, kv_len 0, refs 0, error word cleared.  The
 * pool is not touched. */
np_status np_kv_reset(const np_kv_shape* shape, const np_kv_state* state, void* dev_ws,
                      hipStream_t stream);

/* Room for n_new[b] more tokens (n_new NULL: one each; device int32 [n_seq])
 * in sequences seqs[b] (device int32 [n_seq]; NULL: b), all in one step:
 *  - pos0[b] (device int32 [n_seq], out) is the length before the call, the
 *    position of the first new token; kv_len grows by n_new[b].
 *  - Row by row and in order of position, each place that needs a page takes
 *    the lowest free page id left.
 *  - A partly filled last page that other sequences hold too is replaced by a
 *    new page, which gets a copy of the sequence's kv_len % P tokens of every
 *    layer; when all its holders are rows of this call, the first of them
 *    keeps it.
 * With fewer free pages than needed nothing changes at all: every pos0 is -1
 * (so the step's appends and attention serve no row) and NP_DEVERR_OVERFLOW
 * is set.  A sequence that would outgrow M P tokens is left out with the same
 * bit, one outside [0, S), named twice (its later rows), with a negative
 * n_new or an inconsistent table with NP_DEVERR_STATE; their pos0 is -1.
 * Two kernels on `stream`. */
np_status np_kv_extend(const np_kv_shape* shape, const np_kv_state* state, void* pool,
                       int32_t n_seq, const int32_t* seqs, const int32_t* n_new, int32_t* pos0,
                       void* dev_ws, hipStream_t stream);

/* For each pair (src[i], dst[i]) (device int32 [n]): empty sequence dst[i]
 * becomes the first lens[i] tokens of sequence src[i] (lens NULL: all of it)
 * by holding the same pages; nothing is copied (np_kv_extend copies a shared
 * page before it is written).  Every pair reads the state before the call.
 * src or dst outside [0, S), dst not empty or named by an earlier pair, and
 * lens outside [0, length] set NP_DEVERR_STATE and the pair is left out.  One
 * kernel. */
np_status np_kv_fork(const np_kv_shape* shape, const np_kv_state* state, int32_t n,
                     const int32_t* src, const int32_t* dst, const int32_t* lens, void* dev_ws,
                     hipStream_t stream);

/* Empties sequences seqs[i] (device int32 [n]; NULL: i): each of their pages
 * loses a holder, and is free when it has none.  An empty sequence stays as
 * it is, a sequence named twice is emptied once; one outside [0, S) sets
 * NP_DEVERR_STATE.  One kernel. */
np_status np_kv_free(const np_kv_shape* shape, const np_kv_state* state, int32_t n,
                     const int32_t* seqs, void* dev_ws, hipStream_t stream);

/* Moves the pages in use to the low end of the pool: with U pages in use, the
 * i-th of them at or past U (ascending) moves to the i-th free page below U,
 * in every layer; page_table and refs follow.  n_moved (device int32, may be
 * NULL) receives the number of moved pages.  Two kernels. */
np_status np_kv_compact(const np_kv_shape* shape, const np_kv_state* state, void* pool,
                        int32_t* n_moved, void* dev_ws, hipStream_t stream);

/* Rotary positions (rotary NULL: none) on the batch's queries and keys of one
 * layer; queries to rows->q_out, keys and values into their pages.  Tokens of
 * a row that is not served write nothing.  One kernel. */
np_status np_kv_append(const np_kv_shape* shape, int32_t layer, const np_kv_batch* batch,
                       const int32_t* page_table, const np_kv_rows* rows,
                       const np_rotary* rotary, void* pool, void* dev_ws, hipStream_t stream);

/* The same behind a norm of each query and key head (norm NULL: none), all in
 * 32 bits up to the one rounding to w (keys of 8-bit caches in 64, rounded to 32 before
 * it).  q_out, strides and what is not served as above.  One kernel. */
np_status np_kv_append_norm(const np_kv_shape* shape, int32_t layer, const np_kv_batch* batch,
                            const int32_t* page_table, const np_kv_rows* rows,
                            const np_qk_norm* norm, const np_rotary* rotary, void* pool,
                            void* dev_ws, hipStream_t stream);

/* The batch's tokens read back from one layer: token t's keys of head i to k_out
 * + t * k_stride + i * D, its values to v_out + t * v_stride + i * D (device, type
 * w, strides in elements as in np_kv_rows; either may be NULL).  Zeros for tokens
 * of a row that is not served, and, with NP_DEVERR_NOT_RESIDENT, where the table
 * names no page; a token that no row has is not written.  One kernel. */
np_status np_kv_read(const np_kv_shape* shape, int32_t layer, const np_kv_batch* batch,
                     const int32_t* page_table, const void* pool, void* k_out, int64_t k_stride,
                     void* v_out, int64_t v_stride, void* dev_ws, hipStream_t stream);

/* Attention of the batch's tokens over the cache of one layer:
 *     out = sum_j softmax_j(scale q.k_j) v_j   over the keys the token sees,
 * zero where it sees none.  q and out: device, type w, head i of token t at
 * t * stride + i * D (strides in elements as in np_kv_rows); out may be q
 * with the same stride.  scale: finite.  window >= 0.  Sums, softmax
 * statistics and accumulators are fp32; for 16-bit types the probabilities
 * are rounded to w before they meet the values, as the matrix cores take
 * them.  A NaN or +infinity among a token's scores makes its outputs of that
 * head NaN; one whose scores are all -infinity gets zeros, as if it saw
 * nothing.  Memory at positions outside the keys a row's tokens see together may
 * hold anything, NaN and infinities included; a value that is not finite at a
 * position that some token of the row sees may also reach those of its tokens
 * that do not see it (there it is multiplied by a weight of zero).
 * np_attn_decode: one token per row (cu_tokens must be NULL).  np_attn_prompt:
 * any number of tokens per row, the keys and values of the new tokens already
 * appended.  One kernel each: where the keys of a row are split over
 * workgroups, the last of them to finish joins the parts, in a fixed order.
 * Both give the same bits from run to run. */
np_status np_attn_decode(const np_kv_shape* shape, int32_t layer, const np_kv_batch* batch,
                         const int32_t* page_table, const void* q, int64_t q_stride,
                         const void* pool, float scale, int32_t window, void* out,
                         int64_t out_stride, void* dev_ws, hipStream_t stream);
np_status np_attn_prompt(const np_kv_shape* shape, int32_t layer, const np_kv_batch* batch,
                         const int32_t* page_table, const void* q, int64_t q_stride,
                         const void* pool, float scale, int32_t window, void* out,
                         int64_t out_stride, void* dev_ws, hipStream_t stream);

/* np_attn_decode for rows that share prefixes: the same outputs (up to the
 * rounding of sums in another order; the same bits from run to run), but the
 * keys and values of a group's prefix are read once for its rows together, each
 * row's other keys after that.  Two kernels, the second to join the parts.  Where
 * little can be gained (max_prefix, window and batch bound what sharing saves: up to
 * some 30 MB of keys and values it is not worth the second kernel, nor for many short
 * rows of 8-bit elements), and for batches
 * of more than 32768 query heads in all, or more than 128 query heads per key-value
 * head (16 in fp32), it is np_attn_decode, leads and prefixes then unread.  A value of
 * a group's prefix that is not finite, at a position that some row of the group sees,
 * may also reach rows of the group that do not see it (their window has passed it, or
 * they end before it); rows of other groups it does not. */
np_status np_attn_decode_shared(const np_kv_shape* shape, int32_t layer, const np_kv_batch* batch,
                                const np_kv_shared* shared, const int32_t* page_table,
                                const void* q, int64_t q_stride, const void* pool, float scale,
                                int32_t window, void* out, int64_t out_stride, void* dev_ws,
                                hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* NEUROPREFETCH_KV_H */
