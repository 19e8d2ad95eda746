// np_kv.hpp -- definitions shared by the paged key-value cache, the attention
// kernels and their host side: workspace layout, launch arguments, the batch
// as the kernels read it.
#pragma once

#include "neuroprefetch_kv.h"
#include "np_device.hpp"

namespace np {

// ---------------------------------------------------------------------------
// Workspace of the cache and attention calls.
//   [0, 4096)      control block: the error word (as in every workspace) and
//                  +512 the number of entries of the copy list
//   page scratch   int32 [N] each: free pages, copy sources, copy targets,
//                  copied tokens, page renaming, two marks per page; int32
//                  [S] each: first place and split flag of a row
//   zeros          KV_ZEROS bytes that stay 0: what stands in for a page that a
//                  table does not name (eight rows of 256 fp32)
//   counts         int32 [KV_MAX_BLOCKS]: arrivals of a split row block's
//                  workgroups, 0 between calls
//   partials       of split attention rows: fp32 [KV_PART_ROWS][DP] outputs,
//                  then fp32 [KV_PART_ROWS][2] (maximum, sum)
// ---------------------------------------------------------------------------
constexpr size_t WS_KV_COPIES = 512;
constexpr int KV_PART_ROWS = 65536;
constexpr size_t KV_ZEROS = 8192;
constexpr int KV_MAX_BLOCKS = 8192;
constexpr int KV_MAX_SEQS = 4096;

inline int kv_dpad(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct KvScratch {
  int32_t *free_ids, *src, *dst, *rows, *remap, *mark, *cnt, *off, *split;
  char* zeros;
  int32_t* count;
  float *part, *ml;
};
inline size_t kv_ws_layout(const np_kv_shape& s, char* ws, KvScratch* k) {
  size_t at = WS_CTRL_BYTES;
  auto take = [&](size_t n) {
    char* p = ws + at;
    at = align256(at + n);
    return p;
  };
  KvScratch t;
  for (int32_t** p : {&t.free_ids, &t.src, &t.dst, &t.rows, &t.remap, &t.mark, &t.cnt})
    *p = (int32_t*)take((size_t)s.n_pages * 4);
  for (int32_t** p : {&t.off, &t.split}) *p = (int32_t*)take((size_t)(s.max_seqs + 1) * 4);
  t.zeros = take(KV_ZEROS);
  t.count = (int32_t*)take(KV_MAX_BLOCKS * 4);
  t.part = (float*)take((size_t)KV_PART_ROWS * kv_dpad(s.head_dim) * 4);
  t.ml = (float*)take((size_t)KV_PART_ROWS * 2 * 4);
  if (k) *k = t;
  return at;
}

// bytes of one page of one layer
inline size_t kv_page_bytes(const np_kv_shape& s) {
  return (size_t)2 * s.kv_heads * s.page_size * s.head_dim * dtype_size(s.dtype);
}

// ---------------------------------------------------------------------------
// The batch in a kernel
// ---------------------------------------------------------------------------
struct KvBatch {
  const int32_t* seqs;
  const int32_t* cu;
  const int32_t* pos0;
  int n_seq, n_tokens;
  int S;
  int lim;  // positions below min(max_len, M P)
};

struct KvRow {
  int begin, n;  // tokens [begin, begin + n) of the token arrays
  int p0;        // position of the first, or -1: not served
  int seq;       // 0 <= seq < S
};

// Row b of the batch (0 <= b < n_seq); err: where to put NP_DEVERR_* bits, or
// nullptr.  What it returns is in range whatever the arrays hold.
__device__ inline KvRow kv_row(const KvBatch& a, int b, int32_t* err) {
  KvRow r;
  int bad = 0;
  r.begin = b;
  r.n = 1;
  if (a.cu) {
    const int lo = a.cu[b], hi = a.cu[b + 1];
    if (lo < 0 || hi < lo || hi > a.n_tokens) {
      bad = 1;
      r.begin = r.n = 0;
    } else {
      r.begin = lo;
      r.n = hi - lo;
    }
  }
  r.seq = a.seqs ? a.seqs[b] : b;
  if (r.seq < 0 || r.seq >= a.S) {
    bad = 1;
    r.seq = 0;
    r.p0 = -1;
  } else {
    r.p0 = a.pos0[b];
  }
  if (r.p0 < 0) r.p0 = -1;
  if (r.p0 >= 0 && r.n > a.lim - min(r.p0, a.lim)) {
    bad = 1;
    r.p0 = -1;
  }
  if (bad && err) atomicOr(err, NP_DEVERR_STATE);
  return r;
}

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
hipError_t launch_kv_reset(const np_kv_shape& s, const np_kv_state& st, void* ws,
                           hipStream_t stream);
hipError_t launch_kv_extend(const np_kv_shape& s, const np_kv_state& st, void* pool, int n,
                            const int32_t* seqs, const int32_t* n_new, int32_t* pos0, void* ws,
                            hipStream_t stream);
hipError_t launch_kv_fork(const np_kv_shape& s, const np_kv_state& st, int n, const int32_t* src,
                          const int32_t* dst, const int32_t* lens, void* ws, hipStream_t stream);
hipError_t launch_kv_free(const np_kv_shape& s, const np_kv_state& st, int n, const int32_t* seqs,
                          void* ws, hipStream_t stream);
hipError_t launch_kv_compact(const np_kv_shape& s, const np_kv_state& st, void* pool,
                             int32_t* n_moved, void* ws, hipStream_t stream);
hipError_t launch_kv_append(const np_kv_shape& s, int layer, const np_kv_batch& b,
                            const int32_t* table, const np_kv_rows& r, const np_rotary* rot,
                            void* pool, void* ws, hipStream_t stream);
hipError_t launch_attn(const np_kv_shape& s, int layer, const np_kv_batch& b,
                       const int32_t* table, const void* q, int64_t q_stride, const void* pool,
                       float scale, int window, void* out, int64_t out_stride, void* ws,
                       hipStream_t stream);

}  // namespace np
