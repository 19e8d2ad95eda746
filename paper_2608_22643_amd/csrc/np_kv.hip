// np_kv.hip -- the paged key-value cache: reserving, sharing, freeing and
// compacting pages on the device, and the append of a step's keys and values
// with rotary positions.
//
// The page planners are one workgroup each: they handle a few thousand
// integers in a chain of dependent steps (lengths -> tables -> reference
// counts -> free pages), so latency bounds them and the host never has to
// wait for a count.  A split over workgroups would add a trip past the L2
// (microseconds) between any two of those steps.  Measured: 16 sequences of
// up to 2001 tokens in pages of 64: extend 7.4 us, fork 2.8, free 2.4; the
// plan of a compaction of 48 sequences 5.6.  The page bytes they decide about
// are moved by a second kernel over the whole card, which reads how many pages
// there are from the device, as np_stage_gather does with its lists.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "np_kv.hpp"

namespace np {

namespace {

constexpr int PT = 1024;  // threads of a planner

__device__ inline void raise(int32_t* err, int bits) { atomicOr(err, bits); }

// A value that other threads of the workgroup changed with atomics since it
// was last read: past the vector cache.
__device__ inline int32_t fresh(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }

__global__ void kv_reset_kernel(np_kv_state st, size_t table, int S, int N, int32_t* err,
                                uint32_t* zeros, int32_t* count) {
  const size_t i0 = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  const size_t step = (size_t)gridDim.x * blockDim.x;
  if (i0 == 0) *err = 0;
  for (size_t i = i0; i < KV_ZEROS / 4; i += step) zeros[i] = 0;
  for (size_t i = i0; i < KV_MAX_BLOCKS; i += step) count[i] = 0;
  for (size_t i = i0; i < table; i += step) st.page_table[i] = -1;
  for (size_t i = i0; i < (size_t)N; i += step) st.refs[i] = 0;
  for (size_t i = i0; i < (size_t)S; i += step) st.kv_len[i] = 0;
}

// The first index at which each sequence is named: owner[s] = min i.
// owner: LDS [S].  seqs nullptr: identity.
__device__ inline void name_owners(int32_t* owner, int S, const int32_t* seqs, int n) {
  for (int s = threadIdx.x; s < S; s += PT) owner[s] = INT_MAX;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += PT) {
    const int s = seqs ? seqs[i] : i;
    if (s >= 0 && s < S) atomicMin(&owner[s], i);
  }
  __syncthreads();
}

// Collects pages by a test of their reference count, ascending, 16 a thread
// at a time: put(k, page) for the k-th.  Stops once `want` are found; returns
// how many it saw (all of them when want is INT_MAX).
template <class Test, class Put>
__device__ inline int collect_pages(const int32_t* refs, int lo, int hi, int want, uint32_t* lds,
                                    Test test, Put put) {
  int found = 0;
  for (int base = lo & ~15; base < hi && found < want; base += PT * 16) {
    const int p0 = base + (int)threadIdx.x * 16;
    uint32_t bits = 0;
    if (p0 < hi) {
      int v[16];
      if (p0 + 16 <= hi) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int4 x = *(const int4*)(refs + p0 + 4 * j);
          v[4 * j] = x.x;
          v[4 * j + 1] = x.y;
          v[4 * j + 2] = x.z;
          v[4 * j + 3] = x.w;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = p0 + j < hi ? refs[p0 + j] : 0;
      }
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (p0 + j >= lo && p0 + j < hi && test(v[j])) bits |= 1u << j;
    }
    uint32_t total;
    int k = found + (int)block_excl_scan<PT>(__popc(bits), lds, &total);
    while (bits) {
      const int j = __ffs(bits) - 1;
      bits &= bits - 1;
      put(k++, p0 + j);
    }
    found += (int)total;
  }
  return found;
}

// np_kv_extend.  LDS: owner [S], off [n + 1].
struct ExtendArgs {
  np_kv_state st;
  KvScratch k;
  const int32_t *seqs, *n_new;
  int32_t *pos0, *err, *n_copies;
  int n, S, N, M, P;
};

__global__ __launch_bounds__(PT) void kv_extend_kernel(ExtendArgs a) {
  extern __shared__ int32_t lds[];
  __shared__ uint32_t scan[PT / WAVE];
  __shared__ int s_shared;  // some row's last page is
  int32_t* owner = lds;
  int32_t* off = lds + a.S;
  const int tid = threadIdx.x;
  if (tid == 0) s_shared = 0;
  name_owners(owner, a.S, a.seqs, a.n);
  // k.split[i]: -1 left out, 0 nothing to copy, else 1 + the last page, partly
  // filled and held by others too; its marks are cleared by all who will set
  // them (every writer writes the same value)
  for (int i = tid; i < a.n; i += PT) {
    const int s = a.seqs ? a.seqs[i] : i;
    const int nn = a.n_new ? a.n_new[i] : 1;
    int split = 0;
    if (s < 0 || s >= a.S || owner[s] != i || nn < 0) {
      raise(a.err, NP_DEVERR_STATE);
      split = -1;
    } else {
      const int len = a.st.kv_len[s];
      if (len < 0 || len > a.M * a.P) {
        raise(a.err, NP_DEVERR_STATE);
        split = -1;
      } else if (nn > a.M * a.P - len) {
        raise(a.err, NP_DEVERR_OVERFLOW);
        split = -1;
      } else if (len % a.P && nn > 0) {
        const int pg = a.st.page_table[(size_t)s * a.M + len / a.P];
        if (pg < 0 || pg >= a.N || a.st.refs[pg] < 1) {
          raise(a.err, NP_DEVERR_STATE);
          split = -1;
        } else if (a.st.refs[pg] > 1) {
          __hip_atomic_store(&a.k.mark[pg], INT_MAX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          __hip_atomic_store(&a.k.cnt[pg], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          split = pg + 1;
          s_shared = 1;
        }
      }
    }
    a.k.split[i] = split;
  }
  __syncthreads();
  if (s_shared) {
    for (int i = tid; i < a.n; i += PT) {
      const int split = a.k.split[i];
      if (split <= 0) continue;
      atomicMin(&a.k.mark[split - 1], i);
      atomicAdd(&a.k.cnt[split - 1], 1);
    }
    __syncthreads();
  }
  // how many pages each row needs, and where its pages start in the list
  int total = 0, copies = 0;
  for (int base = 0; base < a.n; base += PT) {
    const int i = base + tid;
    int need = 0, split = i < a.n ? a.k.split[i] : -1;
    if (split >= 0) {
      const int s = a.seqs ? a.seqs[i] : i;
      const int len = a.st.kv_len[s], nn = a.n_new ? a.n_new[i] : 1;
      // past N the call is refused whatever the rest needs: sums stay in range
      need = min(div_up(len + nn, a.P) - div_up(len, a.P), a.N + 1);
      if (split > 0) {
        // when all its holders are rows of this call, the first keeps it
        const int pg = split - 1;
        if (a.st.refs[pg] == fresh(&a.k.cnt[pg]) && fresh(&a.k.mark[pg]) == i) split = 0;
        else ++need;
        a.k.split[i] = split;
      }
    }
    uint32_t t;
    const int at = total + (int)block_excl_scan<PT>((uint32_t)need, scan, &t);
    // at most N pages can be given out; a sum past that is refused below, so
    // it is enough that it stays past it
    total = (int)min((int64_t)total + (int64_t)t, (int64_t)INT_MAX / 2);
    if (i < a.n) off[i] = at;
    const int c = copies + (int)block_excl_scan<PT>(split > 0 ? 1u : 0u, scan, &t);
    copies += (int)t;
    if (split > 0) a.k.off[i] = c;
  }
  if (tid == 0) off[a.n] = total;
  __syncthreads();
  int got = 0;
  if (total > 0 && total <= a.N)
    got = collect_pages(
        a.st.refs, 0, a.N, total, scan, [](int r) { return r <= 0; },
        [&](int k, int page) {
          if (k < total) a.k.free_ids[k] = page;
        });
  __syncthreads();
  if (got < total) {  // not enough: nothing changes
    for (int i = tid; i < a.n; i += PT) a.pos0[i] = -1;
    if (tid == 0) {
      *a.n_copies = 0;
      raise(a.err, NP_DEVERR_OVERFLOW);
    }
    return;
  }
  for (int j = tid; j < total; j += PT) {
    int lo = 0, hi = a.n;  // the last row with off <= j
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (off[mid] <= j) lo = mid;
      else hi = mid;
    }
    const int s = a.seqs ? a.seqs[lo] : lo;
    const int len = a.st.kv_len[s], split = a.k.split[lo];
    const int page = a.k.free_ids[j];
    const int first = div_up(len, a.P) - (split > 0 ? 1 : 0);
    const int place = first + j - off[lo];
    a.st.page_table[(size_t)s * a.M + place] = page;
    a.st.refs[page] = 1;
    if (split > 0 && place == len / a.P) {
      const int c = a.k.off[lo];
      a.k.src[c] = split - 1;
      a.k.dst[c] = page;
      a.k.rows[c] = len % a.P;
      atomicSub(&a.st.refs[split - 1], 1);
    }
  }
  __syncthreads();
  for (int i = tid; i < a.n; i += PT) {
    if (a.k.split[i] < 0) {
      a.pos0[i] = -1;
      continue;
    }
    const int s = a.seqs ? a.seqs[i] : i;
    const int len = a.st.kv_len[s];
    a.pos0[i] = len;
    a.st.kv_len[s] = len + (a.n_new ? a.n_new[i] : 1);
  }
  if (tid == 0) *a.n_copies = copies;
}

// np_kv_fork.  LDS: owner [S], the length each pair shares [n].
__global__ __launch_bounds__(PT) void kv_fork_kernel(np_kv_state st, const int32_t* src,
                                                     const int32_t* dst, const int32_t* lens,
                                                     int n, int S, int N, int M, int P,
                                                     int32_t* err) {
  extern __shared__ int32_t lds[];
  int32_t* owner = lds;
  int32_t* share = lds + S;
  name_owners(owner, S, dst, n);
  for (int i = threadIdx.x; i < n; i += PT) {
    const int a = src[i], b = dst[i];
    int len = -1;
    if (a >= 0 && a < S && b >= 0 && b < S && owner[b] == i && st.kv_len[b] == 0) {
      const int have = st.kv_len[a];
      const int want = lens ? lens[i] : have;
      if (have >= 0 && have <= M * P && want >= 0 && want <= have) len = want;
    }
    if (len < 0) raise(err, NP_DEVERR_STATE);
    share[i] = len;
  }
  __syncthreads();
  // a wave per pair, its lanes over the pages
  for (int i = threadIdx.x / WAVE; i < n; i += PT / WAVE) {
    const int len = share[i];
    if (len <= 0) continue;
    const int a = src[i], b = dst[i];
    for (int j = threadIdx.x % WAVE; j < div_up(len, P); j += WAVE) {
      const int page = st.page_table[(size_t)a * M + j];
      st.page_table[(size_t)b * M + j] = page;
      if (page >= 0 && page < N) atomicAdd(&st.refs[page], 1);
      else raise(err, NP_DEVERR_STATE);
    }
    if (threadIdx.x % WAVE == 0) st.kv_len[b] = len;
  }
}

// np_kv_free.  LDS: owner [S].
__global__ __launch_bounds__(PT) void kv_free_kernel(np_kv_state st, const int32_t* seqs, int n,
                                                     int S, int N, int M, int P, int32_t* err) {
  extern __shared__ int32_t lds[];
  int32_t* owner = lds;
  name_owners(owner, S, seqs, n);
  for (int i = threadIdx.x / WAVE; i < n; i += PT / WAVE) {
    const int s = seqs ? seqs[i] : i;
    if (s < 0 || s >= S) {
      if (threadIdx.x % WAVE == 0) raise(err, NP_DEVERR_STATE);
      continue;
    }
    if (owner[s] != i) continue;
    int len = st.kv_len[s];
    if (len < 0 || len > M * P) {
      if (threadIdx.x % WAVE == 0) raise(err, NP_DEVERR_STATE);
      len = len < 0 ? 0 : M * P;
    }
    for (int j = threadIdx.x % WAVE; j < div_up(len, P); j += WAVE) {
      int32_t* e = st.page_table + (size_t)s * M + j;
      const int page = *e;
      *e = -1;
      if (page < 0 || page >= N || atomicSub(&st.refs[page], 1) < 1) {
        raise(err, NP_DEVERR_STATE);
        if (page >= 0 && page < N) atomicAdd(&st.refs[page], 1);
      }
    }
    if (threadIdx.x % WAVE == 0) st.kv_len[s] = 0;
  }
}

// np_kv_compact: which page goes where.
__global__ __launch_bounds__(PT) void kv_compact_kernel(np_kv_state st, KvScratch k, int N, int P,
                                                        int32_t* n_copies, int32_t* n_moved) {
  __shared__ uint32_t scan[PT / WAVE];
  const int used = collect_pages(
      st.refs, 0, N, INT_MAX, scan, [](int r) { return r > 0; }, [](int, int) {});
  const int holes = collect_pages(
      st.refs, 0, used, INT_MAX, scan, [](int r) { return r <= 0; },
      [&](int i, int page) { k.dst[i] = page; });
  for (int p = used + (int)threadIdx.x; p < N; p += PT) k.remap[p] = -1;
  __syncthreads();
  collect_pages(
      st.refs, used, N, holes, scan, [](int r) { return r > 0; },
      [&](int i, int page) { k.src[i] = page; });
  __syncthreads();
  for (int i = threadIdx.x; i < holes; i += PT) {
    const int from = k.src[i], to = k.dst[i];
    k.remap[from] = to;
    k.rows[i] = P;
    st.refs[to] = st.refs[from];
    st.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    // U for the table's renaming: pages below it stay
    k.off[0] = used;
    *n_copies = holes;
    if (n_moved) *n_moved = holes;
  }
}

// The copy list's pages, in every layer.  A wave copies the first rows[i]
// tokens of one (layer, key or value, head) block of a page: at most P D w
// contiguous bytes, 16 per lane, 8 loads in flight.  table (np_kv_compact):
// its entries follow the moved pages.  Bound by memory: 247 MB read and
// written in 46.7 us (5.3 TB/s; a large copy reaches 4.96); 17.5 MB in 4.8 us.
struct CopyArgs {
  KvScratch k;
  const int32_t* n_copies;
  int32_t* err;
  char* pool;
  size_t layer_bytes, page_bytes;
  int blocks;       // 2 Hkv: blocks of a page of one layer
  int block_bytes;  // P D w, and the scales' P
  int row_bytes;    // D w
  int scales_at;    // 8-bit elements: where a block's scales begin; 0: it has none
  int layers;
  int32_t* table;  // nullptr: no renaming
  size_t entries;
  int N;
};

constexpr int COPY_T = 256, COPY_UNROLL = 8;

__global__ __launch_bounds__(COPY_T) void kv_copy_kernel(CopyArgs a) {
  const int n = *a.n_copies;
  if (a.table) {
    const int used = a.k.off[0];
    for (size_t i = (size_t)blockIdx.x * COPY_T + threadIdx.x; i < a.entries;
         i += (size_t)gridDim.x * COPY_T) {
      const int page = a.table[i];
      if (page < used) continue;
      const int to = page < a.N ? a.k.remap[page] : -1;
      if (to >= 0) a.table[i] = to;
      else raise(a.err, NP_DEVERR_STATE);  // a table that names a free page
    }
  }
  const int lane = threadIdx.x % WAVE;
  const int64_t items = (int64_t)n * a.layers * a.blocks;
  const int64_t waves = (int64_t)gridDim.x * (COPY_T / WAVE);
  for (int64_t it = (int64_t)blockIdx.x * (COPY_T / WAVE) + threadIdx.x / WAVE; it < items;
       it += waves) {
    const int blk = (int)(it % a.blocks);
    const int64_t rest = it / a.blocks;
    const int layer = (int)(rest % a.layers);
    const int c = (int)(rest / a.layers);
    const size_t at = (size_t)layer * a.layer_bytes + (size_t)blk * a.block_bytes;
    const char* src = a.pool + at + (size_t)a.k.src[c] * a.page_bytes;
    char* dst = a.pool + at + (size_t)a.k.dst[c] * a.page_bytes;
    const int bytes = a.k.rows[c] * a.row_bytes;
    if (a.scales_at)
      for (int o = lane; o < a.k.rows[c]; o += WAVE) dst[a.scales_at + o] = src[a.scales_at + o];
    for (int o = lane * 16; o < bytes; o += WAVE * 16 * COPY_UNROLL) {
      uint4 v[COPY_UNROLL];
#pragma unroll
      for (int u = 0; u < COPY_UNROLL; ++u)
        if (o + u * WAVE * 16 < bytes) v[u] = load_nt((const uint4*)(src + o + u * WAVE * 16));
#pragma unroll
      for (int u = 0; u < COPY_UNROLL; ++u)
        if (o + u * WAVE * 16 < bytes) store_nt((uint4*)(dst + o + u * WAVE * 16), v[u]);
    }
  }
}

// ---------------------------------------------------------------------------
// np_kv_append
// ---------------------------------------------------------------------------
struct AppendArgs {
  KvBatch b;
  const int32_t* table;
  const char *q, *k, *v;
  char* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // bytes
  const float *cos, *sin;
  char* pool;  // of the layer
  size_t page_bytes;
  int Hq, Hkv, D, P, M, N;
  int R, max_pos;
  int32_t* err;
  // norms and 8-bit elements (kv_append_heads_kernel)
  bool norm;
  const char *wq, *wk;  // nullptr: ones
  float eps, inv_dim;  // 1 / D
  double inv_dim64;
  int lanes;           // log2 of the lanes that share a head
  int sets;            // that a token's heads come in
  bool split;          // a workgroup for each four of them
  int top;    // the scale byte at which 256 2^(b - 127) leaves the type
};

template <class T>
__device__ inline uint4 pack_row(const float* f) {
  if constexpr (T::V == 4) {
    return make_uint4(T::from_f32(f[0]), T::from_f32(f[1]), T::from_f32(f[2]), T::from_f32(f[3]));
  } else {
    uint4 o;
    o.x = T::from_f32(f[0]) | T::from_f32(f[1]) << 16;
    o.y = T::from_f32(f[2]) | T::from_f32(f[3]) << 16;
    o.z = T::from_f32(f[4]) | T::from_f32(f[5]) << 16;
    o.w = T::from_f32(f[6]) | T::from_f32(f[7]) << 16;
    return o;
  }
}

constexpr int APP_T = 256;

// The place of token t in the cache.  Every thread of a workgroup takes part.
// error: nullptr where another workgroup of the token reports.
struct TokenAt {
  enum { NOBODYS, UNSERVED, NO_PAGE, HERE } what;
  int pos, page;
};
__device__ inline TokenAt find_token(const KvBatch& b, const int32_t* table, int M, int N, int P,
                                     int t, int32_t* error) {
  // the token's row, as the attention calls have it: the one whose tokens
  // include it, bad rows (reported with token 0) having none
  int row = t;
  if (b.cu) {
    if (t == 0 && error)
      for (int i = threadIdx.x; i < b.n_seq; i += APP_T) {
        const int lo = b.cu[i], hi = b.cu[i + 1];
        if (lo < 0 || hi < lo || hi > b.n_tokens) raise(error, NP_DEVERR_STATE);
      }
    row = -1;
    const int lane = threadIdx.x % WAVE;
    for (int base = 0; base < b.n_seq; base += WAVE) {
      const int i = min(base + lane, b.n_seq - 1);
      const int lo = b.cu[i], hi = b.cu[i + 1];
      const uint64_t hit = __ballot((lo >= 0) & (lo <= t) & (t < hi) & (hi <= b.n_tokens));
      if (hit) {
        row = min(base + __ffsll((unsigned long long)hit) - 1, b.n_seq - 1);
        break;
      }
    }
    if (row < 0) return {TokenAt::NOBODYS, -1, -1};
  }
  row = __builtin_amdgcn_readfirstlane(row);
  int32_t* err = threadIdx.x == 0 ? error : nullptr;
  const KvRow r = kv_row(b, row, err);
  if (t < r.begin || t >= r.begin + r.n) return {TokenAt::NOBODYS, -1, -1};
  if (r.p0 < 0) return {TokenAt::UNSERVED, -1, -1};
  const int pos = r.p0 + (t - r.begin);
  const int page = table[(size_t)r.seq * M + pos / P];
  if (page < 0 || page >= N) {
    if (err) raise(err, NP_DEVERR_NOT_RESIDENT);
    return {TokenAt::NO_PAGE, pos, -1};
  }
  return {TokenAt::HERE, pos, page};
}

// A workgroup per token.  A unit is 16 bytes of a head, or for the split pairs
// (i, i + R/2) the two pieces of 16 bytes that turn into each other; a thread
// takes units tid, tid + 256, ...  Everything is read once and written once,
// so memory bounds it: four bf16 prompts of 9,800 tokens in all, 64 + 8 + 8
// heads of 128, 483 MB in 90 us (5.4 TB/s; a large copy reaches 4.96).  With
// few tokens the latency of position -> page -> heads does, in line as the code
// has them (only the stores of keys and values need the page): 4.2 us for 8
// tokens, about 2 of them an empty launch.
template <class T, bool INTER>
__global__ __launch_bounds__(APP_T) void kv_append_kernel(AppendArgs a) {
  constexpr int V = T::V;
  constexpr int W = 16 / V;
  const int t = grid_block();
  if (t >= a.b.n_tokens) return;
  const TokenAt at = find_token(a.b, a.table, a.M, a.N, a.P, t, a.err);
  if (at.what != TokenAt::HERE) return;
  const int pos = at.pos, page = at.page;
  if (a.R && pos >= a.max_pos) {
    if (threadIdx.x == 0) raise(a.err, NP_DEVERR_STATE);
    return;
  }
  const char* q = a.q + t * a.q_stride;
  const char* k = a.k + t * a.k_stride;
  const char* v = a.v + t * a.v_stride;
  char* q_out = a.q_out + t * a.q_out_stride;
  // keys of head h at kp + h P D w; values Hkv P D w further
  const size_t head = (size_t)a.P * a.D * W;
  char* kp = a.pool + (size_t)page * a.page_bytes + (size_t)(pos % a.P) * a.D * W;
  char* vp = kp + (size_t)a.Hkv * head;
  const float* cs = a.cos + (size_t)pos * (a.R / 2);
  const float* sn = a.sin + (size_t)pos * (a.R / 2);

  const int chunks = a.D / V;                       // 16-byte pieces of a head
  const int half = INTER ? 0 : a.R / 2 / V;         // pieces that have a partner
  const int units = chunks - half;                  // units of a query or key head
  const int turned = (a.Hq + a.Hkv) * units, all = turned + a.Hkv * chunks;
  for (int u = threadIdx.x; u < all; u += APP_T) {
    if (u >= turned) {
      const int h = (u - turned) / chunks, c = (u - turned) % chunks;
      *(uint4*)(vp + h * head + c * 16) = *(const uint4*)(v + ((size_t)h * a.D * W + c * 16));
      continue;
    }
    int h = u / units;
    const int c = u % units;
    const char* src;
    char* dst;
    if (h < a.Hq) {
      src = q + (size_t)h * a.D * W;
      dst = q_out + (size_t)h * a.D * W;
    } else {
      h -= a.Hq;
      src = k + (size_t)h * a.D * W;
      dst = kp + h * head;
    }
    if constexpr (INTER) {
      const uint4 x = *(const uint4*)(src + c * 16);
      if (c * V >= a.R) {
        *(uint4*)(dst + c * 16) = x;
        continue;
      }
      float f[V], o[V];
      T::unpack(x, f);
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float co = cs[(c * V + e) / 2], si = sn[(c * V + e) / 2];
        o[e] = f[e] * co - f[e + 1] * si;
        o[e + 1] = f[e + 1] * co + f[e] * si;
      }
      *(uint4*)(dst + c * 16) = pack_row<T>(o);
    } else {
      if (c >= half) {  // past the rotary part: pieces 2 half, 2 half + 1, ...
        *(uint4*)(dst + (c + half) * 16) = *(const uint4*)(src + (c + half) * 16);
        continue;
      }
      const uint4 xa = *(const uint4*)(src + c * 16), xb = *(const uint4*)(src + (c + half) * 16);
      float fa[V], fb[V], oa[V], ob[V];
      T::unpack(xa, fa);
      T::unpack(xb, fb);
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const float4 co = *(const float4*)(cs + c * V + e), si = *(const float4*)(sn + c * V + e);
        const float* cp = &co.x;
        const float* sp = &si.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          oa[e + j] = fa[e + j] * cp[j] - fb[e + j] * sp[j];
          ob[e + j] = fb[e + j] * cp[j] + fa[e + j] * sp[j];
        }
      }
      *(uint4*)(dst + c * 16) = pack_row<T>(oa);
      *(uint4*)(dst + (c + half) * 16) = pack_row<T>(ob);
    }
  }
}

// A reduction over 2^lanes neighbouring lanes, all of which get the result:
// within 16 by moves between lanes' registers, past them by swapped rows.
template <class Op>
__device__ inline float reduce_lanes(float v, int lanes, Op op) {
  auto dpp = [&](auto ctrl) {
    const int x = __float_as_int(v);
    return op(v, __int_as_float(__builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xF, 0xF,
                                                            false)));
  };
  if (lanes > 0) v = dpp(std::integral_constant<int, 0xB1>{});   // lane ^ 1
  if (lanes > 1) v = dpp(std::integral_constant<int, 0x4E>{});   // lane ^ 2
  if (lanes > 2) v = dpp(std::integral_constant<int, 0x141>{});  // 7 - lane, within eight
  if (lanes > 3) v = dpp(std::integral_constant<int, 0x140>{});  // 15 - lane, within sixteen
  if (lanes > 4) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = op(__uint_as_float(x[0]), __uint_as_float(x[1]));
  }
  if (lanes > 5) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = op(__uint_as_float(x[0]), __uint_as_float(x[1]));
  }
  return v;
}

// The sum of 64-bit values in the same way, the two halves of each moved apart.
__device__ inline double sum_lanes(double v, int lanes) {
  auto from = [](uint32_t lo, uint32_t hi) {
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  auto dpp = [&](auto ctrl) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const int lo = (int)u, hi = (int)(u >> 32);
    constexpr int C = decltype(ctrl)::value;
    return v + from(__builtin_amdgcn_update_dpp(lo, lo, C, 0xF, 0xF, false),
                    __builtin_amdgcn_update_dpp(hi, hi, C, 0xF, 0xF, false));
  };
  if (lanes > 0) v = dpp(std::integral_constant<int, 0xB1>{});
  if (lanes > 1) v = dpp(std::integral_constant<int, 0x4E>{});
  if (lanes > 2) v = dpp(std::integral_constant<int, 0x141>{});
  if (lanes > 3) v = dpp(std::integral_constant<int, 0x140>{});
  for (int off = 16; off < 1 << lanes; off *= 2) v += __shfl_xor(v, off, WAVE);
  return v;
}

// 1 / sqrt(x), x > 0: the instruction's estimate and two steps of r (3 - x r^2) / 2
// (infinity gives 0).
__device__ inline double rsqrt64(double x) {
  double r = __builtin_amdgcn_rsq(x);
  if (r == 0.0) return r;
#pragma unroll
  for (int i = 0; i < 2; ++i) r = r * __builtin_fma(-0.5 * x * r, r, 1.5);
  return r;
}

__device__ inline bool finite_f32(float v) {
  return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
}

// The scale byte of a row with largest finite magnitude m: the least b >= 1
// with m <= 448 2^(b - 127); 448 is 1.75 2^8.
__device__ inline int scale_byte(float m) {
  const uint32_t u = __float_as_uint(m);
  return max(1, (int)(u >> 23) - 8 + ((u & 0x007FFFFFu) > 0x00600000u ? 1 : 0));
}

// V values as elements under scale byte b, rounded to the nearest (ties to
// even); what is not finite becomes NaN.
template <int V>
__device__ inline void to_elements(const float* f, int b, int top, uint32_t* out) {
  const float inv = scale_of_byte(254 - b), most = b >= top ? 240.f : 448.f;
  float y[V];
#pragma unroll
  for (int e = 0; e < V; ++e)
    y[e] = finite_f32(f[e]) ? fminf(fmaxf(f[e] * inv, -most), most) : __uint_as_float(0x7FC00000u);
#pragma unroll
  for (int e = 0; e < V; e += 4) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(y[e], y[e + 1], 0, false);
    out[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[e + 2], y[e + 3], x, true);
  }
}

// The same of 16 bytes of w that are finite, under a scale that needs no limit:
// the conversion divides by the scale and rounds once.
template <class T>
__device__ inline void to_elements_fast(uint4 x, float scale, uint32_t* out) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  s16x2 r = {0, 0};
  if constexpr (T::V == 4) {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[0]), __uint_as_float(w[1]),
                                                 scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[2]), __uint_as_float(w[3]),
                                                 scale, true);
    out[0] = __builtin_bit_cast(uint32_t, r);
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if constexpr (T::dtype == NP_F16) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, as_h2(w[2 * e]), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, as_h2(w[2 * e + 1]), scale, true);
      } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, as_b2(w[2 * e]), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, as_b2(w[2 * e + 1]), scale, true);
      }
      out[e] = __builtin_bit_cast(uint32_t, r);
    }
  }
}

// The largest magnitude in 16 bytes of w, as the bits of a w without its sign
// (whose order is that of the magnitudes; infinities and NaN are past them all).
template <class T>
__device__ inline uint32_t largest_bits(uint4 x, uint32_t m) {
  if constexpr (T::V == 4) {
    const uint32_t s = 0x7FFFFFFFu;
    return max(max(max(x.x & s, x.y & s), max(x.z & s, x.w & s)), m);
  } else {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    auto mag = [](uint32_t u) { return __builtin_bit_cast(u16x2, u & 0x7FFF7FFFu); };
    const u16x2 y = __builtin_elementwise_max(__builtin_elementwise_max(mag(x.x), mag(x.y)),
                                              __builtin_elementwise_max(mag(x.z), mag(x.w)));
    return max(max((uint32_t)y.x, (uint32_t)y.y), m);
  }
}

// fp32 to w, 16 bytes of it
template <class T>
__device__ inline uint4 round_row(const float* f) {
  if constexpr (T::V == 4) {
    return pack_row<T>(f);
  } else {
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x2_t v = {f[2 * e], f[2 * e + 1]};
      if constexpr (T::dtype == NP_F16)
        u[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
      else
        u[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf162_t));
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
}

// np_kv_append_norm, and any append of 8-bit elements.  A head is shared by
// 2^lanes neighbouring lanes, so that its sum of squares and its largest magnitude
// are reductions between lanes' registers.  A lane has NP pieces of 16 bytes: one
// (rotary pairs that are neighbours, or none), or the two that turn into each
// other (pairs i, i + R/2; behind the rotary part one; with one piece a lane, and
// the partner's fetched from its lane, 124 us where this took 117).  A set is as
// many heads of a token as a wave holds, all queries, all keys or all values, so
// that what a wave does with them, and their addresses, are the same for its
// lanes.  The heads are asked for before the token's place is looked up, and a
// set's before the one before it is worked on: their addresses need only the
// token's number.
//
// Bound by memory: 11,649 bf16 tokens, 64 + 8 + 8 heads of 128, normed, 483 MB in
// 97 us (5.0 TB/s; a large copy reaches 5.1).  A few tokens take 4.0 to 4.8 us, a
// chain of latencies.
template <class T, int NP, bool E8>
__global__ __launch_bounds__(APP_T) void kv_append_heads_kernel(AppendArgs a) {
  constexpr int V = T::V;
  constexpr int W = 16 / V;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
  const int lane = threadIdx.x % WAVE;
  const int id = grid_block();
  int t = id, set = wave, sets = a.sets;
  bool report = true;
  if (a.split) {  // a workgroup for every four sets
    const int groups = (a.sets + APP_T / WAVE - 1) / (APP_T / WAVE);
    t = id / groups;
    set += (id - t * groups) * (APP_T / WAVE);
    report = id == t * groups;
    sets = min(sets, set + 1);
  }
  if (t >= a.b.n_tokens) return;
  const int chunks = a.D / V;
  const int half = NP == 2 ? a.R / 2 / V : 0;  // pieces that have a partner
  const int u = lane & ((1 << a.lanes) - 1), hl = lane >> a.lanes;
  const int per = 6 - a.lanes;  // log2 of a set's heads
  const bool pair = NP == 2 && u < half;
  const int c0 = pair ? u : u + half, c1 = u + half;  // this lane's pieces, c1 only of pairs
  const int sq = (a.Hq + (1 << per) - 1) >> per, sk = (a.Hkv + (1 << per) - 1) >> per;

  struct Heads {
    int kind, h;  // 0, 1, 2: queries, keys, values; this lane's head
    bool live;
    uint4 x[NP], w[NP];  // it, and its norm's weights
  };
  auto load = [&](int set) {
    Heads d;
    d.kind = set < sq ? 0 : set < sq + sk ? 1 : 2;
    d.h = ((set - (d.kind == 0 ? 0 : d.kind == 1 ? sq : sq + sk)) << per) + hl;
    d.live = d.h < (d.kind ? a.Hkv : a.Hq) && u < chunks - half;
#pragma unroll
    for (int p = 0; p < NP; ++p) d.x[p] = d.w[p] = make_uint4(0, 0, 0, 0);
    auto from = [&](const char* heads, const char* g) {
      if (!d.live) return;
      const char* src = heads + d.h * a.D * W;
      d.x[0] = *(const uint4*)(src + c0 * 16);
      if (pair) d.x[NP - 1] = *(const uint4*)(src + c1 * 16);
      if (g) {
        d.w[0] = *(const uint4*)(g + c0 * 16);
        if (pair) d.w[NP - 1] = *(const uint4*)(g + c1 * 16);
      }
    };
    if (d.kind == 0) from(a.q + t * a.q_stride, a.wq);
    else if (d.kind == 1) from(a.k + t * a.k_stride, a.wk);
    else from(a.v + t * a.v_stride, nullptr);
    return d;
  };
  Heads next;
  if (set < sets) next = load(set);
  const TokenAt at = find_token(a.b, a.table, a.M, a.N, a.P, t, report ? a.err : nullptr);
  if (at.what != TokenAt::HERE) return;
  if (a.R && at.pos >= a.max_pos) {
    if (threadIdx.x == 0 && report) raise(a.err, NP_DEVERR_STATE);
    return;
  }
  // this lane's angles, the same in every set
  constexpr int NA = NP == 1 ? V / 2 : V;
  float cs[NA], sn[NA];
  const bool turns = a.R && (NP == 2 ? pair : c0 * V < a.R);
  if (turns) {
    const size_t first = (size_t)at.pos * (a.R / 2) + c0 * NA;
#pragma unroll
    for (int e = 0; e < NA; e += 2) {
      *(float2*)&cs[e] = *(const float2*)(a.cos + first + e);
      *(float2*)&sn[e] = *(const float2*)(a.sin + first + e);
    }
  }
  char* const page = a.pool + (size_t)at.page * a.page_bytes;
  const int slot = at.pos % a.P;
  const int head_bytes = a.P * (E8 ? a.D + 1 : a.D * W);  // of a page

  auto add = [](float x, float y) { return x + y; };
  auto most = [](float x, float y) { return fmaxf(x, y); };
  for (; set < sets; set += APP_T / WAVE) {
    Heads d = next;
    if (set + APP_T / WAVE < sets) next = load(set + APP_T / WAVE);
    // Two elements are a sixteenth of their value apart, so that an error of 32 bits
    // next to the border between them would grow to that: keys that become elements
    // are normed and turned in 64 bits (in 32, about 20 of 16.8 million fell to the
    // other side, in 64 none).  That costs a sixth: 38 us against 32 for 4106
    // tokens of 32 fp16 heads over 32 of 128.
    bool done = false;
    if constexpr (E8) {
      if (d.kind == 1 && (a.norm || a.R)) {
        float f[NP * V], w[NP * V];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          T::unpack(d.x[p], f + p * V);
          T::unpack(d.w[p], w + p * V);
        }
        double r = 1.0;
        if (a.norm) {
          double ss = 0.0;
#pragma unroll
          for (int e = 0; e < NP * V; ++e) ss = __builtin_fma((double)f[e], (double)f[e], ss);
          const double mean = sum_lanes(ss, a.lanes) * a.inv_dim64 + (double)a.eps;
          r = mean == 0.0 ? 0.0 : rsqrt64(mean);  // of a NaN, NaN
        }
        const bool weighed = a.norm && a.wk;
        auto value = [&](int e) {
          const double v = (double)f[e] * r;
          return weighed ? v * (double)w[e] : v;
        };
#pragma unroll
        for (int e = 0; e < NP * V / 2; ++e) {  // pairs
          const int i = NP == 1 ? 2 * e : e, j = NP == 1 ? 2 * e + 1 : e + V;
          double x = value(i), y = value(j);
          if (turns) {
            const double c = cs[e], n = sn[e], x0 = x;
            x = x0 * c - y * n;
            y = y * c + x0 * n;
          }
          f[i] = (float)x;
          f[j] = (float)y;
        }
        if (a.norm || turns)
#pragma unroll
          for (int p = 0; p < NP; ++p) d.x[p] = round_row<T>(f + p * V);
        done = true;
      }
    }
    if (!done && d.kind < 2 && (a.norm || a.R)) {
      float f[NP * V];
#pragma unroll
      for (int p = 0; p < NP; ++p) T::unpack(d.x[p], f + p * V);
      if (a.norm) {
        // the mean square in fp32; where the sum would leave fp32's range, that of
        // the head divided by a power of two next to its largest magnitude (or to
        // eps's root), which every lane of a head finds alike
        float ss = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p) ss = T::dot(d.x[p], d.x[p], ss);
        ss = reduce_lanes(ss, a.lanes, add);
        const float mean = ss * a.inv_dim + a.eps;
        float r = mean == 0.f ? 0.f : __builtin_amdgcn_rsqf(mean);  // of a NaN, NaN
        const bool far = !(ss < 1e36f) || mean < 1e-27f;
        if (__any(d.live && far)) {
          float m = 0.f;
#pragma unroll
          for (int e = 0; e < NP * V; ++e) m = finite_f32(f[e]) ? fmaxf(m, fabsf(f[e])) : m;
          m = fmaxf(reduce_lanes(m, a.lanes, most), sqrtf(a.eps));
          const int ex = min(max((int)(__float_as_uint(m) >> 23), 2), 252);
          const float scale = scale_of_byte(254 - ex);
          float s2 = 0.f;
#pragma unroll
          for (int e = 0; e < NP * V; ++e) s2 = __builtin_fmaf(f[e] * scale, f[e] * scale, s2);
          s2 = reduce_lanes(s2, a.lanes, add);
          if (far && m > 0.f) {
            r = __builtin_amdgcn_rsqf(s2 * a.inv_dim + a.eps * scale * scale);
#pragma unroll
            for (int e = 0; e < NP * V; ++e) f[e] *= scale;
          }
        }
#pragma unroll
        for (int e = 0; e < NP * V; ++e) f[e] *= r;
        if (d.kind == 0 ? a.wq : a.wk) {
          float w[V];
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            T::unpack(d.w[p], w);
#pragma unroll
            for (int e = 0; e < V; ++e) f[p * V + e] *= w[e];
          }
        }
      }
      if (turns)
#pragma unroll
        for (int e = 0; e < NA; ++e) {
          const int i = NP == 1 ? 2 * e : e, j = NP == 1 ? 2 * e + 1 : e + V;
          const float x = f[i], y = f[j];
          f[i] = x * cs[e] - y * sn[e];
          f[j] = y * cs[e] + x * sn[e];
        }
      if (a.norm || turns)  // the rounding to w
#pragma unroll
        for (int p = 0; p < NP; ++p) d.x[p] = round_row<T>(f + p * V);
    }
    if (d.kind == 0 || !E8) {
      char* dst = d.kind == 0
                      ? a.q_out + t * a.q_out_stride
                      : page + (d.kind == 1 ? 0 : (size_t)a.Hkv * head_bytes) + slot * a.D * W;
      if (d.live) {
        dst += (size_t)d.h * (d.kind == 0 ? a.D * W : head_bytes);
        *(uint4*)(dst + c0 * 16) = d.x[0];
        if (pair) *(uint4*)(dst + c1 * 16) = d.x[NP - 1];
      }
      continue;
    }
    if constexpr (E8) {
      uint32_t bits = 0;
#pragma unroll
      for (int p = 0; p < NP; ++p) bits = largest_bits<T>(d.x[p], bits);
      float m;
      if constexpr (V == 4) m = __uint_as_float(bits);
      else m = T::lo(bits);
      m = reduce_lanes(m, a.lanes, [](float x, float y) {  // NaN and infinity stay so
        return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y)));
      });
      int b = scale_byte(m);
      uint32_t el[NP][V / 4];
      if (__any(d.live && (!finite_f32(m) || b >= a.top))) {
        float f[NP * V];
#pragma unroll
        for (int p = 0; p < NP; ++p) T::unpack(d.x[p], f + p * V);
        m = 0.f;
#pragma unroll
        for (int e = 0; e < NP * V; ++e) m = finite_f32(f[e]) ? fmaxf(m, fabsf(f[e])) : m;
        b = scale_byte(reduce_lanes(m, a.lanes, most));
#pragma unroll
        for (int p = 0; p < NP; ++p) to_elements<V>(f + p * V, b, a.top, el[p]);
      } else {
#pragma unroll
        for (int p = 0; p < NP; ++p) to_elements_fast<T>(d.x[p], scale_of_byte(b), el[p]);
      }
      if (d.live) {
        char* dst = page + (d.kind == 1 ? 0 : (size_t)a.Hkv * head_bytes) +
                    (size_t)d.h * head_bytes;
        auto put = [&](int c, const uint32_t* e) {
          char* p = dst + slot * a.D + c * V;
          if constexpr (V == 8) *(uint2*)p = make_uint2(e[0], e[1]);
          else *(uint32_t*)p = e[0];
        };
        put(c0, el[0]);
        if (pair) put(c1, el[NP - 1]);
        if (u == 0) dst[a.P * a.D + slot] = (char)b;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// np_kv_read: pieces of 16 bytes of a token's keys and values, NB of them a
// thread, all asked for before the first is stored.  Bound by memory, mostly of what
// is written: 4,106 tokens of 32 heads of 128 from 8-bit elements to fp16, 101 MB in
// 21.5 us (4.7 TB/s); a few tokens 3.2 us.
// ---------------------------------------------------------------------------
struct ReadArgs {
  KvBatch b;
  const int32_t* table;
  const char* pool;  // of the layer
  char *k, *v;
  int64_t k_stride, v_stride;  // bytes
  size_t page_bytes;
  int Hkv, D, P, M, N, parts;  // parts: workgroups of a token
  int32_t* err;
};

template <class T, bool E8, int NB>
__global__ __launch_bounds__(APP_T) void kv_read_kernel(ReadArgs a) {
  constexpr int V = T::V, W = 16 / V;
  const int id = grid_block();
  int t = id, part = 0;
  if (a.parts > 1) {
    t = id / a.parts;
    part = id - t * a.parts;
  }
  if (t >= a.b.n_tokens) return;
  const TokenAt at = find_token(a.b, a.table, a.M, a.N, a.P, t, part ? nullptr : a.err);
  if (at.what == TokenAt::NOBODYS) return;
  const int chunks = a.D / V, n = a.Hkv * chunks;
  const int slot = at.pos % a.P, head_bytes = a.P * (E8 ? a.D + 1 : a.D * W);
  const char* page = a.pool + (size_t)at.page * a.page_bytes;
  char* const k_out = a.k ? a.k + t * a.k_stride : nullptr;
  char* const v_out = a.v ? a.v + t * a.v_stride : nullptr;
  char* out[NB];
  uint4 x[NB];
  float s[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    int c = (part * NB + i) * APP_T + (int)threadIdx.x;
    const bool value = c >= n;
    if (value) c -= n;
    out[i] = value ? v_out : k_out;
    if (c >= n) out[i] = nullptr;
    x[i] = make_uint4(0, 0, 0, 0);
    s[i] = 1.f;
    if (!out[i]) continue;
    out[i] += c * 16;
    if (at.what != TokenAt::HERE) continue;
    const int h = c / chunks;
    c -= h * chunks;
    const char* head = page + (size_t)((value ? a.Hkv : 0) + h) * head_bytes;
    if constexpr (!E8) {
      x[i] = *(const uint4*)(head + (slot * a.D + c * V) * W);
    } else {
      s[i] = scale_of_byte((uint8_t)head[a.P * a.D + slot]);
      if constexpr (V == 8) {
        const uint2 e = *(const uint2*)(head + slot * a.D + c * V);
        x[i].x = e.x;
        x[i].y = e.y;
      } else {
        x[i].x = *(const uint32_t*)(head + slot * a.D + c * V);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    if (!out[i]) continue;
    uint4 y = x[i];
    if constexpr (E8 && V == 8)
      y = make_uint4(element_pair<T>(x[i].x, s[i], false), element_pair<T>(x[i].x, s[i], true),
                     element_pair<T>(x[i].y, s[i], false), element_pair<T>(x[i].y, s[i], true));
    if constexpr (E8 && V == 4) {
      const f32x2_t lo = element_pair_f32(x[i].x, s[i], false);
      const f32x2_t hi = element_pair_f32(x[i].x, s[i], true);
      y = make_uint4(__float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x),
                     __float_as_uint(hi.y));
    }
    *(uint4*)out[i] = y;
  }
}

}  // namespace

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
hipError_t launch_kv_reset(const np_kv_shape& s, const np_kv_state& st, void* ws,
                           hipStream_t stream) {
  const size_t table = (size_t)s.max_seqs * s.seq_pages;
  const size_t most = std::max({table, (size_t)s.n_pages, (size_t)s.max_seqs});
  const unsigned grid = (unsigned)std::min<size_t>((most + 255) / 256, 2048);
  KvScratch k;
  kv_ws_layout(s, (char*)ws, &k);
  hipLaunchKernelGGL(kv_reset_kernel, dim3(grid), dim3(256), 0, stream, st, table, s.max_seqs,
                     s.n_pages, (int32_t*)((char*)ws + WS_ERR), (uint32_t*)k.zeros, k.count);
  return hipGetLastError();
}

static hipError_t launch_copies(const np_kv_shape& s, const KvScratch& k, void* pool, void* ws,
                                int32_t* table, int64_t most, hipStream_t stream) {
  CopyArgs a;
  a.k = k;
  a.n_copies = (const int32_t*)((char*)ws + WS_KV_COPIES);
  a.err = (int32_t*)((char*)ws + WS_ERR);
  a.pool = (char*)pool;
  a.page_bytes = kv_page_bytes(s);
  a.layer_bytes = a.page_bytes * s.n_pages;
  a.blocks = 2 * s.kv_heads;
  a.row_bytes = kv_row_bytes(s);
  a.block_bytes = s.page_size * (a.row_bytes + kv_scale_bytes(s));
  a.scales_at = kv_e4m3(s) ? s.page_size * a.row_bytes : 0;
  a.layers = s.layers;
  a.table = table;
  a.entries = (size_t)s.max_seqs * s.seq_pages;
  a.N = s.n_pages;
  int64_t work = (most * s.layers * a.blocks + COPY_T / WAVE - 1) / (COPY_T / WAVE);
  if (table) work = std::max<int64_t>(work, ((int64_t)a.entries + COPY_T - 1) / COPY_T);
  const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(work, 2048));
  hipLaunchKernelGGL(kv_copy_kernel, dim3(grid), dim3(COPY_T), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_kv_extend(const np_kv_shape& s, const np_kv_state& st, void* pool, int n,
                            const int32_t* seqs, const int32_t* n_new, int32_t* pos0, void* ws,
                            hipStream_t stream) {
  ExtendArgs a;
  kv_ws_layout(s, (char*)ws, &a.k);
  a.st = st;
  a.seqs = seqs;
  a.n_new = n_new;
  a.pos0 = pos0;
  a.err = (int32_t*)((char*)ws + WS_ERR);
  a.n_copies = (int32_t*)((char*)ws + WS_KV_COPIES);
  a.n = n;
  a.S = s.max_seqs;
  a.N = s.n_pages;
  a.M = s.seq_pages;
  a.P = s.page_size;
  hipLaunchKernelGGL(kv_extend_kernel, dim3(1), dim3(PT), (size_t)(s.max_seqs + n + 1) * 4, stream,
                     a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_copies(s, a.k, pool, ws, nullptr, n, stream);
}

hipError_t launch_kv_fork(const np_kv_shape& s, const np_kv_state& st, int n, const int32_t* src,
                          const int32_t* dst, const int32_t* lens, void* ws, hipStream_t stream) {
  hipLaunchKernelGGL(kv_fork_kernel, dim3(1), dim3(PT), (size_t)(s.max_seqs + n) * 4, stream, st,
                     src, dst, lens, n, s.max_seqs, s.n_pages, s.seq_pages, s.page_size,
                     (int32_t*)((char*)ws + WS_ERR));
  return hipGetLastError();
}

hipError_t launch_kv_free(const np_kv_shape& s, const np_kv_state& st, int n, const int32_t* seqs,
                          void* ws, hipStream_t stream) {
  hipLaunchKernelGGL(kv_free_kernel, dim3(1), dim3(PT), (size_t)s.max_seqs * 4, stream, st, seqs, n,
                     s.max_seqs, s.n_pages, s.seq_pages, s.page_size,
                     (int32_t*)((char*)ws + WS_ERR));
  return hipGetLastError();
}

hipError_t launch_kv_compact(const np_kv_shape& s, const np_kv_state& st, void* pool,
                             int32_t* n_moved, void* ws, hipStream_t stream) {
  KvScratch k;
  kv_ws_layout(s, (char*)ws, &k);
  hipLaunchKernelGGL(kv_compact_kernel, dim3(1), dim3(PT), 0, stream, st, k, s.n_pages,
                     s.page_size, (int32_t*)((char*)ws + WS_KV_COPIES), n_moved);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_copies(s, k, pool, ws, st.page_table, s.n_pages / 2, stream);
}

hipError_t launch_kv_append(const np_kv_shape& s, int layer, const np_kv_batch& b,
                            const int32_t* table, const np_kv_rows& r, const np_qk_norm* norm,
                            const np_rotary* rot, void* pool, void* ws, hipStream_t stream) {
  const int dtype = kv_dtype(s);
  const int64_t w = dtype_size(dtype);
  AppendArgs a;
  a.b = {b.seqs, b.cu_tokens, b.pos0, b.n_seq, b.n_tokens, s.max_seqs,
         (int)std::min<int64_t>(b.max_len, (int64_t)s.seq_pages * s.page_size)};
  a.table = table;
  a.q = (const char*)r.q;
  a.k = (const char*)r.k;
  a.v = (const char*)r.v;
  a.q_out = (char*)r.q_out;
  a.q_stride = r.q_stride * w;
  a.k_stride = r.k_stride * w;
  a.v_stride = r.v_stride * w;
  a.q_out_stride = r.q_out_stride * w;
  a.cos = rot ? rot->cos : nullptr;
  a.sin = rot ? rot->sin : nullptr;
  a.R = rot ? rot->dim : 0;
  a.max_pos = rot ? rot->max_pos : 0;
  a.page_bytes = kv_page_bytes(s);
  a.pool = (char*)pool + (size_t)layer * s.n_pages * a.page_bytes;
  a.Hq = s.heads;
  a.Hkv = s.kv_heads;
  a.D = s.head_dim;
  a.P = s.page_size;
  a.M = s.seq_pages;
  a.N = s.n_pages;
  a.err = (int32_t*)((char*)ws + WS_ERR);
  const bool inter = rot && rot->interleaved, e8 = kv_e4m3(s);
  const bool heads = norm || e8;
  a.norm = norm;
  a.wq = norm ? (const char*)norm->q_weight : nullptr;
  a.wk = norm ? (const char*)norm->k_weight : nullptr;
  a.eps = norm ? norm->eps : 0.f;
  a.inv_dim = 1.f / (float)a.D;
  a.inv_dim64 = 1.0 / a.D;
  a.top = dtype == NP_F16 ? 127 + 8 : 127 + 120;
  const bool pairs = a.R && !inter;
  const int v = vec_elems(dtype), units = a.D / v - (pairs ? a.R / 2 / v : 0);
  a.lanes = 0;
  while (1 << a.lanes < units) ++a.lanes;
  const int per = WAVE >> a.lanes;
  a.sets = (s.heads + per - 1) / per + 2 * ((s.kv_heads + per - 1) / per);
  const int groups = (a.sets + APP_T / WAVE - 1) / (APP_T / WAVE);
  // Few tokens: a workgroup for every four of a token's sets, while all of them are on the
  // card at once (us, whole tokens / split: 17 tokens of 56 heads 6.7 / 4.6, 4097 tokens of 96
  // heads 31.6 / 64).
  a.split = (int64_t)b.n_tokens * groups <= 2048;
  auto go = [&](auto kernel, int64_t blocks) {
    hipLaunchKernelGGL(kernel, block_grid(blocks), dim3(APP_T), 0, stream, a);
  };
  auto of = [&](auto t) {
    using T = decltype(t);
    const int64_t n = b.n_tokens, wgs = a.split ? n * groups : n;
    if (!heads) inter ? go(kv_append_kernel<T, true>, n) : go(kv_append_kernel<T, false>, n);
    else if (e8) pairs ? go(kv_append_heads_kernel<T, 2, true>, wgs)
                       : go(kv_append_heads_kernel<T, 1, true>, wgs);
    else pairs ? go(kv_append_heads_kernel<T, 2, false>, wgs)
               : go(kv_append_heads_kernel<T, 1, false>, wgs);
  };
  if (dtype == NP_F32) of(TF32{});
  else if (dtype == NP_F16) of(TF16{});
  else of(TBF16{});
  return hipGetLastError();
}

hipError_t launch_kv_read(const np_kv_shape& s, int layer, const np_kv_batch& b,
                          const int32_t* table, const void* pool, void* k, int64_t k_stride,
                          void* v, int64_t v_stride, void* ws, hipStream_t stream) {
  const int dtype = kv_dtype(s);
  const int64_t w = dtype_size(dtype);
  ReadArgs a;
  a.b = {b.seqs, b.cu_tokens, b.pos0, b.n_seq, b.n_tokens, s.max_seqs,
         (int)std::min<int64_t>(b.max_len, (int64_t)s.seq_pages * s.page_size)};
  a.table = table;
  a.page_bytes = kv_page_bytes(s);
  a.pool = (const char*)pool + (size_t)layer * s.n_pages * a.page_bytes;
  a.k = (char*)k;
  a.v = (char*)v;
  a.k_stride = k_stride * w;
  a.v_stride = v_stride * w;
  a.Hkv = s.kv_heads;
  a.D = s.head_dim;
  a.P = s.page_size;
  a.M = s.seq_pages;
  a.N = s.n_pages;
  const int pieces = 2 * s.kv_heads * (s.head_dim / vec_elems(dtype));
  // many pieces: four a thread, which find their token once (28.9 -> 21.5 us for the above);
  // with few of them the workgroups count for more
  const bool many = pieces > 2 * APP_T && (int64_t)b.n_tokens * pieces > 2048 * APP_T;
  a.parts = (pieces + APP_T * (many ? 4 : 1) - 1) / (APP_T * (many ? 4 : 1));
  a.err = (int32_t*)((char*)ws + WS_ERR);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, block_grid((int64_t)b.n_tokens * a.parts), dim3(APP_T), 0, stream,
                       a);
  };
  auto of = [&](auto t) {
    using T = decltype(t);
    if (kv_e4m3(s)) many ? go(kv_read_kernel<T, true, 4>) : go(kv_read_kernel<T, true, 1>);
    else many ? go(kv_read_kernel<T, false, 4>) : go(kv_read_kernel<T, false, 1>);
  };
  if (dtype == NP_F32) of(TF32{});
  else if (dtype == NP_F16) of(TF16{});
  else of(TBF16{});
  return hipGetLastError();
}

}  // namespace np
