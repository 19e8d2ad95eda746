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
  int block_bytes;  // P D w
  int row_bytes;    // D w
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
  // the token's row, as the attention calls have it: the one whose tokens
  // include it, bad rows (reported with token 0) having none
  int row = t;
  if (a.b.cu) {
    if (t == 0)
      for (int i = threadIdx.x; i < a.b.n_seq; i += APP_T) {
        const int lo = a.b.cu[i], hi = a.b.cu[i + 1];
        if (lo < 0 || hi < lo || hi > a.b.n_tokens) raise(a.err, NP_DEVERR_STATE);
      }
    row = -1;
    const int lane = threadIdx.x % WAVE;
    for (int base = 0; base < a.b.n_seq; base += WAVE) {
      const int i = min(base + lane, a.b.n_seq - 1);
      const int lo = a.b.cu[i], hi = a.b.cu[i + 1];
      const uint64_t hit = __ballot((lo >= 0) & (lo <= t) & (t < hi) & (hi <= a.b.n_tokens));
      if (hit) {
        row = min(base + __ffsll((unsigned long long)hit) - 1, a.b.n_seq - 1);
        break;
      }
    }
    if (row < 0) return;  // nobody's token
  }
  row = __builtin_amdgcn_readfirstlane(row);
  int32_t* err = threadIdx.x == 0 ? a.err : nullptr;
  const KvRow r = kv_row(a.b, row, err);
  if (r.p0 < 0 || t < r.begin || t >= r.begin + r.n) return;
  const int pos = r.p0 + (t - r.begin);
  const int page = a.table[(size_t)r.seq * a.M + pos / a.P];
  if (page < 0 || page >= a.N) {
    if (err) raise(err, NP_DEVERR_NOT_RESIDENT);
    return;
  }
  if (a.R && pos >= a.max_pos) {
    if (err) raise(err, NP_DEVERR_STATE);
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
  a.row_bytes = s.head_dim * dtype_size(s.dtype);
  a.block_bytes = s.page_size * a.row_bytes;
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
                            const int32_t* table, const np_kv_rows& r, const np_rotary* rot,
                            void* pool, void* ws, hipStream_t stream) {
  const int64_t w = dtype_size(s.dtype);
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
  const bool inter = rot && rot->interleaved;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, block_grid(b.n_tokens), dim3(APP_T), 0, stream, a);
  };
  if (s.dtype == NP_F32) {
    if (inter) go(kv_append_kernel<TF32, true>);
    else go(kv_append_kernel<TF32, false>);
  } else if (s.dtype == NP_F16) {
    if (inter) go(kv_append_kernel<TF16, true>);
    else go(kv_append_kernel<TF16, false>);
  } else {
    if (inter) go(kv_append_kernel<TBF16, true>);
    else go(kv_append_kernel<TBF16, false>);
  }
  return hipGetLastError();
}

}  // namespace np
