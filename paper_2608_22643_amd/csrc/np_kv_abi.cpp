// np_kv_abi.cpp -- host side of the cache and attention calls: argument
// validation, workspace sizing and dispatch.  Validation runs before anything
// is enqueued.
#include <cmath>

#include "np_kv.hpp"

namespace np {

static bool aligned4(const void* p) { return p && ((uintptr_t)p & 3u) == 0; }
static bool aligned4_or_null(const void* p) { return ((uintptr_t)p & 3u) == 0; }

static np_status check_kv_shape(const np_kv_shape* s) {
  if (!s) return fail(NP_ERR_INVALID_ARG, "kv shape is NULL");
  if (s->dtype < NP_F32 || s->dtype > NP_BF16)
    return fail(NP_ERR_INVALID_ARG, "dtype %d is not an np_dtype", s->dtype);
  if (s->layers < 1) return fail(NP_ERR_INVALID_ARG, "layers %d < 1", s->layers);
  if (s->heads < 1 || s->heads > 1024 || s->kv_heads < 1 || s->heads % s->kv_heads)
    return fail(NP_ERR_INVALID_ARG, "heads %d (at most 1024) and kv_heads %d: kv_heads must divide heads",
                s->heads, s->kv_heads);
  if (s->head_dim < 8 || s->head_dim > 256 || s->head_dim % 8)
    return fail(NP_ERR_INVALID_ARG, "head_dim %d is not a multiple of 8 in [8, 256]", s->head_dim);
  const int P = s->page_size;
  if (P < 16 || P > 256 || (P & (P - 1)))
    return fail(NP_ERR_INVALID_ARG, "page_size %d is not one of 16, 32, 64, 128, 256", P);
  if (s->n_pages < 1 || s->n_pages > (1 << 20))
    return fail(NP_ERR_INVALID_ARG, "n_pages %d outside [1, 2^20]", s->n_pages);
  if (s->max_seqs < 1 || s->max_seqs > KV_MAX_SEQS)
    return fail(NP_ERR_INVALID_ARG, "max_seqs %d outside [1, %d]", s->max_seqs, KV_MAX_SEQS);
  if (s->seq_pages < 1 || (int64_t)s->seq_pages * P > ((int64_t)1 << 30))
    return fail(NP_ERR_INVALID_ARG, "seq_pages %d: positions outside [1, 2^30]", s->seq_pages);
  return NP_OK;
}

static np_status check_kv_state(const char* fn, const np_kv_state* st) {
  if (!st || !aligned16(st->page_table) || !aligned16(st->kv_len) || !aligned16(st->refs))
    return fail(NP_ERR_INVALID_ARG, "%s: state arrays must be non-NULL and 16-byte aligned", fn);
  return NP_OK;
}

static np_status check_batch(const char* fn, const np_kv_shape* s, int32_t layer,
                             const np_kv_batch* b) {
  if (layer < 0 || layer >= s->layers)
    return fail(NP_ERR_INVALID_ARG, "%s: layer %d outside [0, %d)", fn, layer, s->layers);
  if (!b) return fail(NP_ERR_INVALID_ARG, "%s: batch is NULL", fn);
  if (b->n_seq < 0 || b->n_seq > s->max_seqs)
    return fail(NP_ERR_INVALID_ARG, "%s: n_seq %d outside [0, max_seqs]", fn, b->n_seq);
  if (b->n_tokens < 0 || b->n_tokens > (1 << 24))
    return fail(NP_ERR_INVALID_ARG, "%s: n_tokens %d outside [0, 2^24]", fn, b->n_tokens);
  if ((int64_t)b->n_tokens * s->heads > ((int64_t)1 << 30))
    return fail(NP_ERR_UNSUPPORTED, "%s: %d tokens of %d heads: more than 2^30 query heads", fn,
                b->n_tokens, s->heads);
  if (!b->cu_tokens && b->n_tokens != b->n_seq)
    return fail(NP_ERR_INVALID_ARG, "%s: %d tokens for %d rows of one token", fn, b->n_tokens,
                b->n_seq);
  if (b->max_tokens < 0 || b->max_len < 0)
    return fail(NP_ERR_INVALID_ARG, "%s: negative max_tokens or max_len", fn);
  if (b->n_seq > 0 && (!aligned4(b->pos0) || !aligned4_or_null(b->seqs) ||
                       !aligned4_or_null(b->cu_tokens)))
    return fail(NP_ERR_INVALID_ARG, "%s: batch arrays must be 4-byte aligned and pos0 non-NULL", fn);
  return NP_OK;
}

// token rows of `heads` heads: stride in elements.  An array of no tokens may
// be anywhere.
static np_status check_rows(const char* fn, const char* what, const np_kv_shape* s, const void* p,
                            int64_t stride, int heads, int n_tokens) {
  if (n_tokens > 0 && !aligned16(p))
    return fail(NP_ERR_INVALID_ARG, "%s: %s must be non-NULL and 16-byte aligned", fn, what);
  if (stride < (int64_t)heads * s->head_dim || stride % vec_elems(s->dtype) ||
      stride > ((int64_t)1 << 31))
    return fail(NP_ERR_INVALID_ARG,
                "%s: %s stride %lld: a multiple of %d elements, at least a token's %d", fn, what,
                (long long)stride, vec_elems(s->dtype), heads * s->head_dim);
  return NP_OK;
}

static np_status attn_common(const char* fn, const np_kv_shape* s, int32_t layer,
                             const np_kv_batch* b, const int32_t* table, const void* q,
                             int64_t q_stride, const void* pool, float scale, int32_t window,
                             void* out, int64_t out_stride, void* ws, hipStream_t stream) {
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_batch(fn, s, layer, b);
  if (st == NP_OK) st = check_rows(fn, "q", s, q, q_stride, s->heads, b->n_tokens);
  if (st == NP_OK) st = check_rows(fn, "out", s, out, out_stride, s->heads, b->n_tokens);
  if (st != NP_OK) return st;
  if (!std::isfinite(scale)) return fail(NP_ERR_INVALID_ARG, "%s: scale is not finite", fn);
  if (window < 0) return fail(NP_ERR_INVALID_ARG, "%s: window %d < 0", fn, window);
  if (!aligned16(table) || !aligned16(pool) || !aligned16(ws))
    return fail(NP_ERR_INVALID_ARG, "%s: pointers must be non-NULL and 16-byte aligned", fn);
  if (out == q && b->n_tokens > 0 && out_stride != q_stride)
    return fail(NP_ERR_INVALID_ARG, "%s: in place, but out_stride differs from q_stride", fn);
  if (b->n_seq == 0 || b->n_tokens == 0) return NP_OK;
  hipError_t e = launch_attn(*s, layer, *b, table, q, q_stride, pool, scale, window, out,
                             out_stride, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, fn);
}

}  // namespace np

using namespace np;

extern "C" {

np_status np_kv_shape_check(const np_kv_shape* s) { return check_kv_shape(s); }

np_status np_kv_workspace_size(const np_kv_shape* s, size_t* bytes) {
  np_status st = check_kv_shape(s);
  if (st != NP_OK) return st;
  if (!bytes) return fail(NP_ERR_INVALID_ARG, "dev_ws_bytes is NULL");
  *bytes = kv_ws_layout(*s, nullptr, nullptr);
  return NP_OK;
}

np_status np_kv_reset(const np_kv_shape* s, const np_kv_state* state, void* ws,
                      hipStream_t stream) {
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_kv_state("np_kv_reset", state);
  if (st != NP_OK) return st;
  if (!aligned16(ws))
    return fail(NP_ERR_INVALID_ARG, "np_kv_reset: dev_ws must be non-NULL and 16-byte aligned");
  hipError_t e = launch_kv_reset(*s, *state, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, "np_kv_reset launch");
}

np_status np_kv_extend(const np_kv_shape* s, const np_kv_state* state, void* pool, int32_t n_seq,
                       const int32_t* seqs, const int32_t* n_new, int32_t* pos0, void* ws,
                       hipStream_t stream) {
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_kv_state("np_kv_extend", state);
  if (st != NP_OK) return st;
  if (n_seq < 0 || n_seq > s->max_seqs)
    return fail(NP_ERR_INVALID_ARG, "np_kv_extend: n_seq %d outside [0, max_seqs]", n_seq);
  if (!aligned16(pool) || !aligned16(ws) ||
      (n_seq > 0 && (!aligned4(pos0) || !aligned4_or_null(seqs) || !aligned4_or_null(n_new))))
    return fail(NP_ERR_INVALID_ARG, "np_kv_extend: pointers must be non-NULL and aligned");
  if (n_seq == 0) return NP_OK;
  hipError_t e = launch_kv_extend(*s, *state, pool, n_seq, seqs, n_new, pos0, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, "np_kv_extend launch");
}

np_status np_kv_fork(const np_kv_shape* s, const np_kv_state* state, int32_t n, const int32_t* src,
                     const int32_t* dst, const int32_t* lens, void* ws, hipStream_t stream) {
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_kv_state("np_kv_fork", state);
  if (st != NP_OK) return st;
  if (n < 0 || n > s->max_seqs)
    return fail(NP_ERR_INVALID_ARG, "np_kv_fork: n %d outside [0, max_seqs]", n);
  if (!aligned16(ws) ||
      (n > 0 && (!aligned4(src) || !aligned4(dst) || !aligned4_or_null(lens))))
    return fail(NP_ERR_INVALID_ARG, "np_kv_fork: pointers must be non-NULL and aligned");
  if (n == 0) return NP_OK;
  hipError_t e = launch_kv_fork(*s, *state, n, src, dst, lens, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, "np_kv_fork launch");
}

np_status np_kv_free(const np_kv_shape* s, const np_kv_state* state, int32_t n,
                     const int32_t* seqs, void* ws, hipStream_t stream) {
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_kv_state("np_kv_free", state);
  if (st != NP_OK) return st;
  if (n < 0 || n > s->max_seqs)
    return fail(NP_ERR_INVALID_ARG, "np_kv_free: n %d outside [0, max_seqs]", n);
  if (!aligned16(ws) || !aligned4_or_null(seqs))
    return fail(NP_ERR_INVALID_ARG, "np_kv_free: pointers must be non-NULL and aligned");
  if (n == 0) return NP_OK;
  hipError_t e = launch_kv_free(*s, *state, n, seqs, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, "np_kv_free launch");
}

np_status np_kv_compact(const np_kv_shape* s, const np_kv_state* state, void* pool,
                        int32_t* n_moved, void* ws, hipStream_t stream) {
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_kv_state("np_kv_compact", state);
  if (st != NP_OK) return st;
  if (!aligned16(pool) || !aligned16(ws) || !aligned4_or_null(n_moved))
    return fail(NP_ERR_INVALID_ARG, "np_kv_compact: pointers must be non-NULL and aligned");
  hipError_t e = launch_kv_compact(*s, *state, pool, n_moved, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, "np_kv_compact launch");
}

np_status np_kv_append(const np_kv_shape* s, int32_t layer, const np_kv_batch* b,
                       const int32_t* table, const np_kv_rows* r, const np_rotary* rot, void* pool,
                       void* ws, hipStream_t stream) {
  const char* fn = "np_kv_append";
  np_status st = check_kv_shape(s);
  if (st == NP_OK) st = check_batch(fn, s, layer, b);
  if (st != NP_OK) return st;
  if (!r) return fail(NP_ERR_INVALID_ARG, "%s: rows is NULL", fn);
  const int n = b->n_tokens;
  if ((st = check_rows(fn, "q", s, r->q, r->q_stride, s->heads, n)) != NP_OK ||
      (st = check_rows(fn, "k", s, r->k, r->k_stride, s->kv_heads, n)) != NP_OK ||
      (st = check_rows(fn, "v", s, r->v, r->v_stride, s->kv_heads, n)) != NP_OK ||
      (st = check_rows(fn, "q_out", s, r->q_out, r->q_out_stride, s->heads, n)) != NP_OK)
    return st;
  if (r->q_out == r->q && n > 0 && r->q_out_stride != r->q_stride)
    return fail(NP_ERR_INVALID_ARG, "%s: in place, but q_out_stride differs from q_stride", fn);
  if (rot) {
    if (rot->dim < 16 || rot->dim % 16 || rot->dim > s->head_dim)
      return fail(NP_ERR_INVALID_ARG, "%s: rotary dim %d is not a multiple of 16 in [16, %d]", fn,
                  rot->dim, s->head_dim);
    if (rot->max_pos < 1) return fail(NP_ERR_INVALID_ARG, "%s: max_pos %d < 1", fn, rot->max_pos);
    if (!aligned16(rot->cos) || !aligned16(rot->sin))
      return fail(NP_ERR_INVALID_ARG, "%s: cos and sin must be non-NULL and 16-byte aligned", fn);
  }
  if (!aligned16(table) || !aligned16(pool) || !aligned16(ws))
    return fail(NP_ERR_INVALID_ARG, "%s: pointers must be non-NULL and 16-byte aligned", fn);
  if (b->n_seq == 0 || b->n_tokens == 0) return NP_OK;
  hipError_t e = launch_kv_append(*s, layer, *b, table, *r, rot, pool, ws, stream);
  return e == hipSuccess ? NP_OK : hip_fail(e, "np_kv_append launch");
}

np_status np_attn_decode(const np_kv_shape* s, int32_t layer, const np_kv_batch* b,
                         const int32_t* table, const void* q, int64_t q_stride, const void* pool,
                         float scale, int32_t window, void* out, int64_t out_stride, void* ws,
                         hipStream_t stream) {
  if (b && b->cu_tokens)
    return fail(NP_ERR_INVALID_ARG,
                "np_attn_decode: one token per row, cu_tokens must be NULL (np_attn_prompt)");
  return attn_common("np_attn_decode", s, layer, b, table, q, q_stride, pool, scale, window, out,
                     out_stride, ws, stream);
}

np_status np_attn_prompt(const np_kv_shape* s, int32_t layer, const np_kv_batch* b,
                         const int32_t* table, const void* q, int64_t q_stride, const void* pool,
                         float scale, int32_t window, void* out, int64_t out_stride, void* ws,
                         hipStream_t stream) {
  return attn_common("np_attn_prompt", s, layer, b, table, q, q_stride, pool, scale, window, out,
                     out_stride, ws, stream);
}

}  // extern "C"
