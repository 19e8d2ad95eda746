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
//   zeros          KV_ZEROS bytes that stay 0: what stands in for a page that a
//                  table does not name (eight rows of 256 fp32)
//   counts         int32 [KV_MAX_BLOCKS]: arrivals of a split block's
//                  workgroups, 0 between calls
//   page scratch   int32 [N] each: free pages, copy sources, copy targets,
//                  copied tokens, page renaming, two marks per page; int32
//                  [S] each: first place and split flag of a row
//   partials       of split attention rows: fp32 [KV_PART_ROWS][DP] outputs,
//                  then fp32 [KV_PART_ROWS][2] (maximum, sum); as many rows as
//                  two tiles of 128 on every compute unit, split in two
//   shared plan    of np_attn_decode_shared: int32 [KV_SHARED_HEADS] twice (the
//                  workgroups of a part), [S] (a row's lead)
// Zeros and counts have to last from call to call, so they come before
// everything whose size depends on the shape: one workspace serves caches of
// several shapes in turn.
// ---------------------------------------------------------------------------
constexpr size_t WS_KV_COPIES = 512;
constexpr int KV_PART_ROWS = 131072;
constexpr size_t KV_ZEROS = 8192;
constexpr int KV_MAX_BLOCKS = 8192;
constexpr int KV_MAX_SEQS = 4096;
constexpr int KV_SHARED_HEADS = 32768;  // most query heads of a batch that np_attn_decode_shared splits

inline int kv_dpad(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

struct KvScratch {
  int32_t *free_ids, *src, *dst, *rows, *remap, *mark, *cnt, *off, *split;
  char* zeros;
  int32_t* count;
  float *part, *ml;
  int32_t *shared_p, *shared_s, *shared_lead;
};
inline size_t kv_ws_layout(const np_kv_shape& s, char* ws, KvScratch* k) {
  size_t at = WS_CTRL_BYTES;
  auto take = [&](size_t n) {
    char* p = ws + at;
    at = align256(at + n);
    return p;
  };
  KvScratch t;
  t.zeros = take(KV_ZEROS);
  t.count = (int32_t*)take(KV_MAX_BLOCKS * 4);
  for (int32_t** p : {&t.free_ids, &t.src, &t.dst, &t.rows, &t.remap, &t.mark, &t.cnt})
    *p = (int32_t*)take((size_t)s.n_pages * 4);
  for (int32_t** p : {&t.off, &t.split}) *p = (int32_t*)take((size_t)(s.max_seqs + 1) * 4);
  t.part = (float*)take((size_t)KV_PART_ROWS * kv_dpad(s.head_dim) * 4);
  t.ml = (float*)take((size_t)KV_PART_ROWS * 2 * 4);
  t.shared_p = (int32_t*)take(KV_SHARED_HEADS * 4);
  t.shared_s = (int32_t*)take(KV_SHARED_HEADS * 4);
  t.shared_lead = (int32_t*)take((size_t)s.max_seqs * 4);
  if (k) *k = t;
  return at;
}

// The type of the heads, and whether the cache holds 8-bit elements.
inline int kv_dtype(const np_kv_shape& s) { return s.dtype & ~NP_KV_E4M3; }
inline bool kv_e4m3(const np_kv_shape& s) { return s.dtype & NP_KV_E4M3; }
// bytes of a row of the cache, of its scale, and of one page of one layer
inline int kv_row_bytes(const np_kv_shape& s) {
  return s.head_dim * (kv_e4m3(s) ? 1 : dtype_size(s.dtype));
}
inline int kv_scale_bytes(const np_kv_shape& s) { return kv_e4m3(s) ? 1 : 0; }
inline size_t kv_page_bytes(const np_kv_shape& s) {
  return (size_t)2 * s.kv_heads * s.page_size * (kv_row_bytes(s) + kv_scale_bytes(s));
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

// A uniform address read through the scalar cache: the result is uniform too,
// and the load is counted apart from vector loads in flight.
typedef const __attribute__((address_space(4))) int32_t* scalar_i32_t;
__device__ inline int32_t load_scalar(const int32_t* p, int64_t i) {
  return ((scalar_i32_t)(uintptr_t)p)[i];
}

struct KvRawRow {
  int lo, hi, seq, p0;
};

// Row b of the batch as it stands in memory (0 <= b < n_seq, uniform).
__device__ inline KvRawRow kv_row_load(const KvBatch& a, int b) {
  KvRawRow r;
  r.p0 = load_scalar(a.pos0, b);
  r.seq = a.seqs ? load_scalar(a.seqs, b) : b;
  r.lo = a.cu ? load_scalar(a.cu, b) : b;
  r.hi = a.cu ? load_scalar(a.cu, b + 1) : b + 1;
  return r;
}

// The same within its ranges whatever the arrays hold; err: where to put
// NP_DEVERR_* bits, or nullptr.
__device__ inline KvRow kv_row_check(const KvBatch& a, const KvRawRow& w, int32_t* err) {
  KvRow r = {w.lo, w.hi - w.lo, w.p0, w.seq};
  bool bad = false;
  if (w.lo < 0 || w.hi < w.lo || w.hi > a.n_tokens) {
    bad = true;
    r.begin = r.n = 0;
  }
  if (r.seq < 0 || r.seq >= a.S) {
    bad = true;
    r.seq = 0;
    r.p0 = -1;
  }
  if (r.p0 < 0) r.p0 = -1;
  if (r.p0 >= 0 && r.n > a.lim - min(r.p0, a.lim)) {
    bad = true;
    r.p0 = -1;
  }
  if (bad && err) atomicOr(err, NP_DEVERR_STATE);
  return r;
}

__device__ inline KvRow kv_row(const KvBatch& a, int b, int32_t* err) {
  return kv_row_check(a, kv_row_load(a, b), err);
}

// 2^(b - 127) of a row's scale byte (1 .. 254)
__device__ inline float scale_of_byte(uint32_t b) { return __uint_as_float(b << 23); }

// Two elements (the low or the high half of a dword of four) times a scale that
// is a power of two, as a dword of 16-bit values, or as two fp32.
typedef float f32x2_t __attribute__((ext_vector_type(2)));
template <class T>
__device__ inline uint32_t element_pair(uint32_t e, float scale, bool high) {
  if constexpr (T::dtype == NP_F16) {
    const half2_t x = high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(e, scale, true)
                           : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(e, scale, false);
    return __builtin_bit_cast(uint32_t, x);
  } else {
    const bf162_t x = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(e, scale, true)
                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(e, scale, false);
    return __builtin_bit_cast(uint32_t, x);
  }
}
__device__ inline f32x2_t element_pair_f32(uint32_t e, float scale, bool high) {
  return high ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(e, scale, true)
              : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(e, scale, false);
}

// A grid of at least `blocks` workgroups of up to 256 threads, numbered by
// grid_block().  A launch may have fewer than 2^32 threads along an axis; the
// calls allow 2^24 tokens and 2^26 row blocks.
constexpr int GRID_X = 23;  // log2 of the workgroups along x when there are several along y
inline dim3 block_grid(int64_t blocks) {
  const int64_t x = blocks < (1 << GRID_X) ? blocks : 1 << GRID_X;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}
__device__ inline int grid_block() { return (int)(blockIdx.y << GRID_X | blockIdx.x); }

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
                            const int32_t* table, const np_kv_rows& r, const np_qk_norm* norm,
                            const np_rotary* rot, void* pool, void* ws, hipStream_t stream);
hipError_t launch_kv_read(const np_kv_shape& s, int layer, const np_kv_batch& b,
                          const int32_t* table, const void* pool, void* k, int64_t k_stride,
                          void* v, int64_t v_stride, void* ws, hipStream_t stream);
hipError_t launch_attn(const np_kv_shape& s, int layer, const np_kv_batch& b,
                       const int32_t* table, const void* q, int64_t q_stride, const void* pool,
                       float scale, int window, void* out, int64_t out_stride, void* ws,
                       hipStream_t stream);
hipError_t launch_attn_shared(const np_kv_shape& s, int layer, const np_kv_batch& b,
                              const np_kv_shared& sh, const int32_t* table, const void* q,
                              int64_t q_stride, const void* pool, float scale, int window,
                              void* out, int64_t out_stride, void* ws, hipStream_t stream);

}  // namespace np
