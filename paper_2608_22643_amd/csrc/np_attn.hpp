// np_attn.hpp -- attention over the paged key-value cache: the kernels and the
// rules that choose among them, for plain caches (np_attn.hip), caches of 8-bit
// elements (np_attn8.hip) and shared prefixes (np_attn_shared.hip).
//
// For a query at position p with visible keys j (p - window < j <= p):
//     o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),   s_j = scale q.k_j,
// m the maximum of the s_j seen so far: one pass over keys and values with a
// running maximum and sum; when the maximum rises, sums and outputs are
// scaled by exp(m_old - m_new).  exp is taken as 2^(s log2 e), log2 e folded
// into the scale.
//
// All query heads of a key-value head share its keys, so a row of the kernels
// is a (token, head of the group) pair and a block of rows reads each key and
// value once.
#pragma once

#include <algorithm>
#include <type_traits>

#include "np_kv.hpp"

namespace np {

struct AttnArgs {
  KvBatch b;
  const int32_t* table;
  const char* q;
  char* out;
  int64_t q_stride, out_stride;  // bytes per token
  const char* pool;              // of the layer
  size_t page_bytes;
  int Hkv, G, D, M, N;
  int pshift;  // log2 P
  float scale;  // times log2 e
  int window;
  int tiles;  // row blocks (of one key-value head) the grid covers
  int chunk;  // keys per split, a multiple of GROUP (EVEN: groups a share has at least)
  int splits;
  float *part, *ml;
  const char* zeros;  // KV_ZEROS bytes
  int* count;         // arrivals of a block's splits, 0 between calls
  int prow;  // rows of a block that have partials: min(16, G) with one token a row
  int32_t* err;
};

// The arguments that every attention call has in common.
AttnArgs attn_args(const np_kv_shape& s, int layer, const np_kv_batch& b, const int32_t* table,
                   const void* q, int64_t q_stride, const void* pool, float scale, int window,
                   void* out, int64_t out_stride, void* ws);
// keys: the most a block of rows can see
hipError_t launch_attn_e4m3(int dtype, AttnArgs& a, int64_t keys, int max_tokens,
                            hipStream_t stream);

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

// a value that every lane of the wave has alike, for the scalar registers
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// A block of RB consecutive rows (token-major, then head of the group) of one
// batch row.
struct Tile {
  KvRow row;
  int rho0, nrow;      // rows [rho0, rho0 + nrow) of the batch row's n * G
  int minpos, maxpos;  // of their tokens; maxpos < 0: they see nothing
};

// Where block `tile` of the batch is: block *pblk of row *prow; false past the
// last one.  Every lane of the wave takes part and gets the same result.  err:
// where this workgroup reports what is wrong with its row, or nullptr; the one
// with tile 0 reports every row of a bad cu_tokens (a row without tokens has no
// block).
template <int RB>
__device__ inline bool find_block(const KvBatch& b, int G, int tile, int32_t* err, int* prow,
                                  int* pblk) {
  int row, blk;
  if (!b.cu) {
    const int per = (G + RB - 1) / RB;
    row = tile / per;
    blk = tile - row * per;
    if (row >= b.n_seq) return false;
  } else {
    const int lane = threadIdx.x % WAVE;
    if (err && tile == 0 && threadIdx.x < WAVE)
      for (int i = lane; i < b.n_seq; i += WAVE)
        if (b.cu[i] < 0 || b.cu[i + 1] < b.cu[i] || b.cu[i + 1] > b.n_tokens)
          atomicOr(err, NP_DEVERR_STATE);
    // blocks of the rows before: a running count, 64 rows at a time
    int before = 0;
    row = -1;
    for (int base = 0; base < b.n_seq; base += WAVE) {
      int n = 0;
      if (base + lane < b.n_seq) {
        const int lo = b.cu[base + lane], hi = b.cu[base + lane + 1];
        if (lo >= 0 && hi >= lo && hi <= b.n_tokens)
          n = (int)(((int64_t)(hi - lo) * G + RB - 1) / RB);
      }
      const int incl = (int)wave_incl_scan((uint32_t)n);
      const uint64_t hit = __ballot(before + incl > tile);
      if (hit) {
        const int l = __ffsll((unsigned long long)hit) - 1;
        row = base + l;
        blk = tile - before - (__shfl(incl, l, WAVE) - __shfl(n, l, WAVE));
        break;
      }
      before += __shfl(incl, WAVE - 1, WAVE);
    }
    if (row < 0 || blk < 0) return false;  // blk: a cu_tokens that counts tokens twice
  }
  *prow = uniform(row);
  *pblk = uniform(blk);
  return true;
}

// The same with the blocks in another order: those that reach furthest first,
// so that the longest do not start last.  With up to 64 rows, one a lane: block
// blk of a row has level (its first key, in blocks) + blk, every row has at most
// one block of a level, and block number `rank` is found by counting those above
// a level.  More rows leave the order as it is (there are blocks enough to fill
// in behind the longest).
template <int RB>
__device__ inline bool find_block_longest(const KvBatch& b, int G, int rank, int tiles,
                                          int32_t* err, int* prow, int* pblk) {
  if (!b.cu || b.n_seq > WAVE) return find_block<RB>(b, G, tiles - 1 - rank, err, prow, pblk);
  const int lane = threadIdx.x % WAVE;
  int n = 0, lo = 0;
  if (lane < b.n_seq) {
    const KvRawRow w = {b.cu[lane], b.cu[lane + 1], 0, b.pos0[lane]};
    if (w.lo < 0 || w.hi < w.lo || w.hi > b.n_tokens) {
      if (err && rank == 0 && threadIdx.x < WAVE) atomicOr(err, NP_DEVERR_STATE);
    } else {
      n = (int)(((int64_t)(w.hi - w.lo) * G + RB - 1) / RB);
      // rows past level 2^30 (2^37 query heads from their start) share that level
      lo = (int)min((int64_t)min(max(w.p0, 0), b.lim) * G / RB, (int64_t)1 << 30);
    }
  }
  auto above = [&](int x) {  // blocks of level x or more
    const int c = min(n, max(0, lo + n - max(x, lo)));
    return __builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)c), WAVE - 1);
  };
  if (above(0) <= rank) return false;
  int x0 = 0, x1 = (int)wave_max(n ? (uint32_t)(lo + n) : 0u);  // above(x0) > rank >= above(x1)
  while (x1 - x0 > 1) {
    const int x = x0 + (x1 - x0) / 2;
    if (above(x) > rank) x0 = x;
    else x1 = x;
  }
  // the rank - above(x1)-th row that has a block of level x0
  const uint32_t has = n > 0 && lo <= x0 && x0 < lo + n;
  const int nth = (int)wave_incl_scan(has) - 1, want = rank - above(x1);  // every lane takes part
  const uint64_t hit = __ballot(has && nth == want);
  const int l = __ffsll((unsigned long long)hit) - 1;
  if (l < 0) return false;
  *prow = l;
  *pblk = x0 - __builtin_amdgcn_readlane(lo, l);
  return true;
}

template <int RB>
__device__ inline bool make_tile(const KvRow& row, int G, int blk, Tile* t) {
  t->row = row;
  t->rho0 = blk * RB;
  t->nrow = min(RB, row.n * G - t->rho0);
  if (t->nrow <= 0) return false;
  t->minpos = row.p0 + t->rho0 / G;
  t->maxpos = row.p0 + (t->rho0 + t->nrow - 1) / G;
  if (row.p0 < 0) t->minpos = t->maxpos = -1;
  return true;
}

// The first key that any row of the block sees.
__device__ inline int first_key(const Tile& t, int window) {
  return window && t.maxpos >= 0 ? max(0, t.minpos - window + 1) : 0;
}

// Two fp32 to a dword of 16-bit values (round to nearest even).
template <class T>
__device__ inline uint32_t pack2(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 v = {a, b};
  if constexpr (T::dtype == NP_F16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, half2_t));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf162_t));
}

// 16 bytes of global memory (an address the compiler cannot trace to an
// argument would become a flat load, which waits for LDS too)
typedef const __attribute__((address_space(1))) u32x4_t* global16_t;
__device__ inline u32x4_t load_global16(const char* p) { return *(global16_t)(uintptr_t)p; }
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(1))) u32x2_t* global8_t;
__device__ inline u32x2_t load_global8(const char* p) { return *(global8_t)(uintptr_t)p; }

typedef const __attribute__((address_space(1))) uint32_t* global4_t;
__device__ inline uint32_t load_global4(const char* p) { return *(global4_t)(uintptr_t)p; }
typedef const __attribute__((address_space(1))) uint8_t* global1_t;
__device__ inline uint32_t load_global1(const char* p) { return *(global1_t)(uintptr_t)p; }

// The part-th V of the elements in x, as 16 bytes of w (V of them).
template <class T>
__device__ inline u32x4_t elements16(u32x4_t x, int part, float scale) {
  u32x4_t y;
  if constexpr (T::V == 8) {
    const uint32_t a = x[2 * part], b = x[2 * part + 1];
    y.x = element_pair<T>(a, scale, false);
    y.y = element_pair<T>(a, scale, true);
    y.z = element_pair<T>(b, scale, false);
    y.w = element_pair<T>(b, scale, true);
  } else {
    const f32x2_t lo = element_pair_f32(x[part], scale, false);
    const f32x2_t hi = element_pair_f32(x[part], scale, true);
    y.x = __float_as_uint(lo.x);
    y.y = __float_as_uint(lo.y);
    y.z = __float_as_uint(hi.x);
    y.w = __float_as_uint(hi.y);
  }
  return y;
}

__device__ inline float max_groups(float v) {  // over lanes l, l ^ 16, l ^ 32, l ^ 48
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float sum_groups(float v) {
  v = swap16_add(v, v);
  return swap32_add(v, v);
}

// ---------------------------------------------------------------------------
// Row blocks: 16 rows against a range of keys, the keys dealt to the four
// waves in steps of KS.  Nothing of K or V passes through LDS:
//  * S^T = K Q^T on 16 x 16 tiles.  Which key an A-operand row stands for is
//    free, so the rows are dealt such that the accumulator of a lane (query
//    l % 16, four rows of each tile) holds, over the step's tiles, the very
//    keys the lane supplies as B operand of O^T = V^T P^T: probabilities go
//    from accumulator to operand inside the lane.
//  * V is loaded row by row as it lies, 16 lanes over a row, and transposed
//    in registers with byte permutes; column 16 NV s + NV c + j of V is row c
//    of output tile (s, j), so a lane ends up with NV consecutive outputs.
// Each lane owns one query (l % 16): maximum, sum and rescaling need no
// exchange beyond the maximum over the four lanes of a query.
// Bound by the K and V bytes: one bf16 row of 131072 keys, 8 key-value heads of
// 128, 537 MB in 95 us (5.65 TB/s; a plain stream of that length reaches 5.6 to
// 6.1); 64 fp16 rows of 1 to 8192 keys, 326 MB in 69 us (4.7 TB/s).  Short calls
// are bound by the chain table -> keys -> scores -> values -> join: 8.9 us for
// 777 keys and 32 heads.  fp32 prompts run here too: 4096 tokens of 16 heads over
// 4 at 81, 74 and 93 TFLOP/s for heads of 64, 128 and 256 (an 8192^3 fp32 library
// product reaches 149 to 154).  8-bit elements become w on their way to the matrix
// cores: one row of 131071 keys, 8 key-value heads of 128, 270 MB in 47 to 56 us (4.8 to 5.7
// TB/s, from card to card); 777 keys and 32 heads 8.8 us.
// ---------------------------------------------------------------------------
constexpr int RB = 16;
constexpr int NWAVE = 4;
constexpr int ROWS_T = NWAVE * WAVE;
constexpr int MAX_SPLITS = 128;
constexpr int GROUP = 128;  // keys a workgroup takes at once: a step or two of each wave

template <class T, int DP, bool E8>
struct RowsCfg {
  static constexpr int V = T::V;
  static constexpr int W = 16 / V;               // bytes of an element
  static constexpr int KS = V == 8 ? 32 : 16;    // keys of a step
  static constexpr int KT = KS / 16;             // 16-key tiles of a step
  static constexpr int KD = DP / (4 * V);        // MFMA steps over the head
  static constexpr int KP = E8 ? DP / 64 : KD;   // K loads of a row
  static constexpr int NS = KD / KP;             // MFMA steps of a load
  static constexpr int NV = V == 4 ? 4 : DP == 64 ? 4 : 8;  // V elements of a load
  static constexpr int VS = DP / (16 * NV);      // V loads of a row
  static constexpr int VR = KS / 4;              // V rows of a lane
  static constexpr int OP = DP + 4;              // LDS row of outputs, padded
  // the first of the V elements that lanes of group g hold in MFMA step s: which
  // they are is free as long as queries and keys agree, and 16 8-bit elements
  // that lie together make a load
  __device__ static inline int kdim(int s, int g) {
    return E8 ? 64 * (s / NS) + 16 * g + V * (s % NS) : 4 * V * s + V * g;
  }
};

// FULL: D == DP; otherwise the key pieces past D are zeroed (a piece inside D is
// read in their place), and the output columns past D are not stored.
// E8: 8-bit elements, turned into w on the way to the matrix cores.
//
// One stretch of keys: the rows of a block against keys [k0, k1) of its [kbeg,
// kend), K's head h, this lane's query at qp (position qpos), the pages of the
// sequence with page table trow.  minpos and maxpos bound the rows' positions.
// Each of NW waves takes every NW-th step, and has its own maximum m, sum l and
// outputs o afterwards; missing: a key had no page.
// CUT: the rows may see keys before kbeg or from kend on, which other stretches have.
// QT: blocks of 16 rows at once, each with its own queries and results; the keys
// and values are loaded, and turned into operands, for all of them together.
template <class T, int DP, bool FULL, bool E8, bool CUT, int QT, int NW = NWAVE,
          class C = RowsCfg<T, DP, E8>>
__device__ __forceinline__ void rows_keys(int tid, const AttnArgs& a, const int32_t* trow, int h,
                                          int minpos, int maxpos, int kbeg, int kend, int k0, int k1,
                                          const char* const (&qp)[QT], const int (&qpos)[QT],
                                          f32x4 (&o)[QT][C::VS][C::NV], float (&m)[QT],
                                          float (&l)[QT], bool& missing) {
  constexpr int V = C::V, W = C::W, KS = C::KS, KT = C::KT, KD = C::KD, KP = C::KP, NS = C::NS,
                NV = C::NV, VS = C::VS, VR = C::VR;
  const int lane = tid % WAVE;
  const int wave = NW == 1 ? 0 : uniform(tid / WAVE);
  const int r = lane & 15, g = lane >> 4;
  const int klast = max(kend - 1, 0);
  // the keys that this lane's query counts
  int klast_seen[QT], kfirst_seen[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    klast_seen[x] = CUT ? min(qpos[x], kend - 1) : qpos[x];
    kfirst_seen[x] = max(a.window ? qpos[x] - a.window + 1 : 0, CUT ? kbeg : 0);
  }
  // page ids through the scalar cache.  A step of 32 keys has two pages when
  // P is 16.
  struct Pages {
    int a, b;
  };
  auto pages_of = [&](int base) {
    Pages p;
    p.a = load_scalar(trow, max(kbeg, min(base, klast)) >> a.pshift);
    p.b = KS == 32 ? load_scalar(trow, max(kbeg, min(base + 16, klast)) >> a.pshift) : p.a;
    return p;
  };
  int base = k0 + wave * KS;
  Pages pg = {0, 0};
  if (base < k1) pg = pages_of(base);
  // this lane's query (B operand): column r
  uint4 qf[QT][KD];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
#pragma unroll
    for (int s = 0; s < KD; ++s) {
      const int d = C::kdim(s, g);
      qf[x][s] = FULL || d < a.D ? *(const uint4*)(qp[x] + d * W) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int s = 0; s < VS; ++s)
#pragma unroll
      for (int j = 0; j < NV; ++j) o[x][s][j] = (f32x4)(0.f);
    m[x] = -INFINITY;
    l[x] = 0.f;
  }

  const int P1 = (1 << a.pshift) - 1;
  constexpr int EW = E8 ? 1 : W;  // bytes of an element of the cache
  const int rowb = a.D * EW;
  const size_t headb = ((size_t)rowb + (E8 ? 1 : 0)) << a.pshift;
  const char* kpool = a.pool + h * headb;
  const size_t vofs = a.Hkv * headb;
  const int scales = rowb << a.pshift;  // E8: from a head's elements to its scales

  // keys of a lane: A-operand row r of tile kt is key kk + 4 kt (16-bit) or r
  const int kk = V == 8 ? 8 * (r >> 2) + (r & 3) : r;
  const int vk = VR * g;  // first value row of the lane
  // byte offsets of the lane's pieces in a row
  int kd[KP], vd[VS];
#pragma unroll
  for (int p = 0; p < KP; ++p) {
    const int d = C::kdim(p * NS, g);
    kd[p] = (FULL || d < a.D ? d : 0) * EW;
  }
#pragma unroll
  for (int s = 0; s < VS; ++s) {
    const int d = 16 * NV * s + NV * r;
    vd[s] = (FULL || d < a.D ? d : 0) * EW;
  }

  constexpr int VB = NV * EW;  // bytes of a V load
  u32x4_t kf[KT][KP];
  u32x4_t vf[VR][VS];  // VB bytes of each are used
  uint32_t ks[KT], vs[(VR + 3) / 4];  // E8: scale bytes of this lane's keys and value rows
  int ok = 0, next_ok = 0;  // which 16-key halves of a step have a page
  missing = false;          // a bad table entry among the keys
  const char *vptr, *vsp;
  uint32_t vrow[VR];

  // Addresses of a step.  A half without a page (a bad table entry) is read
  // from zeros and masked.  Value rows outside [kbeg, kend) repeat the first or
  // the last one inside: they get no weight, but memory there may hold
  // anything, and 0 * NaN would reach the output.
  auto load_k = [&](int base, Pages p) {
    const bool ha = (uint32_t)p.a < (uint32_t)a.N, hb = (uint32_t)p.b < (uint32_t)a.N;
    next_ok = (ha ? 1 : 0) | (hb ? 2 : 0);
    const bool hk = V == 8 && r >= 8 ? hb : ha, hv = V == 8 && g >= 2 ? hb : ha;
    const int pk = V == 8 && r >= 8 ? p.b : p.a, pv = V == 8 && g >= 2 ? p.b : p.a;
    const char* kptr = kpool + (int64_t)pk * (int64_t)a.page_bytes + ((base + kk) & P1) * rowb;
    vptr = kpool + vofs + (int64_t)pv * (int64_t)a.page_bytes;
    if constexpr (E8) {
      // scores of keys that are masked may be anything, so their scale may too
      const char* sp = kpool + (int64_t)pk * (int64_t)a.page_bytes + scales + ((base + kk) & P1);
      if (!hk) sp = a.zeros;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) ks[kt] = load_global1(sp + 4 * kt);
      vsp = hv ? vptr + scales + ((base + vk) & P1) : a.zeros;
    }
    if (!hk) kptr = a.zeros;
    if (!hv) vptr = a.zeros;
    if (base >= kbeg && base + KS <= kend) {
#pragma unroll
      for (int e = 0; e < VR; ++e) vrow[e] = hv ? (((base + vk) & P1) + e) * rowb : 0;
    } else {
#pragma unroll
      for (int e = 0; e < VR; ++e)
        vrow[e] = hv ? (max(kbeg, min(base + vk + e, klast)) & P1) * rowb : 0;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int s = 0; s < KP; ++s) kf[kt][s] = load_global16(kptr + 4 * kt * rowb + kd[s]);
  };
  auto load_v = [&]() {
#pragma unroll
    for (int e = 0; e < VR; ++e)
#pragma unroll
      for (int s = 0; s < VS; ++s) {
        const char* p = vptr + vrow[e] + vd[s];
        if constexpr (VB == 16) {
          vf[e][s] = load_global16(p);
        } else if constexpr (VB == 8) {
          const u32x2_t x = load_global8(p);
          vf[e][s].x = x.x;
          vf[e][s].y = x.y;
        } else {
          vf[e][s].x = load_global4(p);
        }
      }
    if constexpr (E8) {
      if constexpr (VR == 8) {
        const u32x2_t x = load_global8(vsp);
        vs[0] = x.x;
        vs[1] = x.y;
      } else {
        vs[0] = load_global4(vsp);
      }
    }
  };

  // One step.  LAST: no step of this wave follows.  Its values are asked for
  // while its keys are on their way, the next step's keys as soon as this
  // one's are used, so that loads are in flight during all of the arithmetic.
  auto step = [&](auto last) {
    constexpr bool LAST = decltype(last)::value;
    const int next = base + NW * KS;
    load_v();
    __builtin_amdgcn_sched_barrier(0);
    const bool full = ok == 3 && base + KS - 1 <= minpos &&
                      (a.window == 0 || base > maxpos - a.window) &&
                      (!CUT || (base >= kbeg && base + KS <= kend));
    f32x4 sc[QT][KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
      for (int x = 0; x < QT; ++x) sc[x][kt] = (f32x4)(0.f);
#pragma unroll
      for (int s = 0; s < KD; ++s) {
        u32x4_t k;
        if constexpr (E8) k = elements16<T>(kf[kt][s / NS], s % NS, scale_of_byte(ks[kt]));
        else k = kf[kt][s];
        if (!FULL && C::kdim(s, g) >= a.D) k = (u32x4_t)(0u);
#pragma unroll
        for (int x = 0; x < QT; ++x) sc[x][kt] = mfma_step<T>(as_uint4(k), qf[x][s], sc[x][kt]);
      }
    }
    if constexpr (!LAST) {
      // kept behind the products: earlier, the new keys would need registers
      // of their own
      __builtin_amdgcn_sched_barrier(0);
      load_k(next, pg);
      pg = pages_of(next + NW * KS);
    }
    const bool has = (ok >> (KS == 32 && g >= 2 ? 1 : 0)) & 1;
    uint4 pb[QT];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      // scores of key base + vk + 4 kt + i
      float p[4 * KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[4 * kt + i] = sc[x][kt][i] * a.scale;
      if (!full) {
#pragma unroll
        for (int i = 0; i < 4 * KT; ++i) {
          const int key = base + vk + i;
          if (!has || key > klast_seen[x] || key < kfirst_seen[x]) p[i] = -INFINITY;
        }
      }
      float mx = p[0];
#pragma unroll
      for (int i = 1; i < 4 * KT; ++i) mx = fmaxf(mx, p[i]);
      mx = max_groups(mx);
      if (__any(mx > m[x])) {
        const float mn = fmaxf(m[x], mx);
        const float alpha = m[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[x] - mn);
        m[x] = mn;
        l[x] *= alpha;
#pragma unroll
        for (int s = 0; s < VS; ++s)
#pragma unroll
          for (int j = 0; j < NV; ++j) o[x][s][j] *= alpha;
      }
      const float mu = m[x] == -INFINITY ? 0.f : m[x];  // nothing visible yet: 2^(-inf) = 0
#pragma unroll
      for (int i = 0; i < 4 * KT; ++i) {
        p[i] = __builtin_amdgcn_exp2f(p[i] - mu);
        l[x] += p[i];
      }
      if constexpr (V == 8) {
        // rounded to the type of V, as the matrix cores take it; the sum l
        // keeps the unrounded values
        pb[x].x = pack2<T>(p[0], p[1]);
        pb[x].y = pack2<T>(p[2], p[3]);
        pb[x].z = pack2<T>(p[4], p[5]);
        pb[x].w = pack2<T>(p[6], p[7]);
      } else {
        pb[x] = make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]),
                           __float_as_uint(p[3]));
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    float f[VR];
    if constexpr (E8) {
      // the rows' scales; of a row that repeats another one, and has no weight,
      // any that is finite
      const bool inside = base >= kbeg && base + KS <= kend;
#pragma unroll
      for (int e = 0; e < VR; ++e) {
        uint32_t b = vs[e / 4] >> (8 * (e % 4)) & 0xFFu;
        if (!inside) b = base + vk + e < kbeg || base + vk + e > klast ? 127u : b;
        f[e] = scale_of_byte(b);
      }
    }
#pragma unroll
    for (int s = 0; s < VS; ++s) {
      uint32_t w[VR];  // 16-bit types: elements j & ~1 and j | 1 of each row
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        uint4 av;
        if constexpr (V == 8) {
          if (j % 2 == 0)
#pragma unroll
            for (int e = 0; e < VR; ++e) {
              if constexpr (E8) w[e] = element_pair<T>(vf[e][s][j / 4], f[e], j % 4 == 2);
              else w[e] = vf[e][s][j / 2];
            }
          const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;  // high or low halves
          av.x = __builtin_amdgcn_perm(w[1], w[0], sel);
          av.y = __builtin_amdgcn_perm(w[3], w[2], sel);
          av.z = __builtin_amdgcn_perm(w[5], w[4], sel);
          av.w = __builtin_amdgcn_perm(w[7], w[6], sel);
        } else if constexpr (E8) {
#pragma unroll
          for (int e = 0; e < VR; ++e)
            w[e] = __float_as_uint(element_pair_f32(vf[e][s].x, f[e], j >= 2)[j & 1]);
          av = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
          av = make_uint4(vf[0][s][j], vf[1][s][j], vf[2][s][j], vf[3][s][j]);
        }
#pragma unroll
        for (int x = 0; x < QT; ++x) o[x][s][j] = mfma_step<T>(av, pb[x], o[x][s][j]);
      }
    }
    if constexpr (!LAST) {
      ok = next_ok;
      missing |= ok != 3;
      base = next;
    }
  };

  if (base < k1) {
    load_k(base, pg);
    ok = next_ok;
    missing |= ok != 3;
    pg = pages_of(base + NW * KS);
    if (base + NW * KS < k1) {
      do step(std::false_type{});
      while (base + NW * KS < k1);
    }
    step(std::true_type{});
  }
}

// The four waves' results of rows_keys on their way through LDS: stored, and,
// behind a barrier, four columns of a row joined (M, L: the row's maximum, sum).
template <class C>
__device__ __forceinline__ void rows_meet(const f32x4 (&o)[C::VS][C::NV], float m, float l,
                                          float (&s_o)[NWAVE][RB][C::OP], float (&s_m)[NWAVE][RB],
                                          float (&s_l)[NWAVE][RB]) {
  constexpr int NV = C::NV;
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int r = lane & 15, g = lane >> 4;
  l = sum_groups(l);
  if (g == 0) {
    s_m[wave][r] = m;
    s_l[wave][r] = l;
  }
#pragma unroll
  for (int s = 0; s < C::VS; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NV; j += 4)
        *(float4*)&s_o[wave][r][16 * NV * s + NV * (4 * g + i) + j] =
            make_float4(o[s][j][i], o[s][j + 1][i], o[s][j + 2][i], o[s][j + 3][i]);
}

template <class C>
__device__ __forceinline__ float4 rows_met(const float (&s_o)[NWAVE][RB][C::OP],
                                           const float (&s_m)[NWAVE][RB],
                                           const float (&s_l)[NWAVE][RB], int qr, int d, float& M,
                                           float& L) {
  M = -INFINITY;
#pragma unroll
  for (int w = 0; w < NWAVE; ++w) M = fmaxf(M, s_m[w][qr]);
  float4 sum = make_float4(0, 0, 0, 0);
  L = 0.f;
#pragma unroll
  for (int w = 0; w < NWAVE; ++w) {
    const float mw = s_m[w][qr], lw = s_l[w][qr];
    // without a maximum the sum is 0, or NaN when every score was
    const float f = mw == -INFINITY ? lw : __builtin_amdgcn_exp2f(mw - M);
    const float4 x = *(const float4*)&s_o[w][qr][d];
    L += f * lw;
    sum.x += f * x.x;
    sum.y += f * x.y;
    sum.z += f * x.z;
    sum.w += f * x.w;
  }
  return sum;
}

// EVEN: one token a row, the keys of all rows dealt evenly to the workgroups;
// otherwise a workgroup per (block, head, split).
// Workgroups a compute unit: 8-bit elements in flight take half the registers (64
// rows of 47,000 keys in all, 8 key-value heads of 256: 62 us with one, 44 with two).
template <class T, int DP, bool FULL, bool EVEN, bool E8>
__global__ __launch_bounds__(ROWS_T, DP < 256 ? (E8 ? 3 : 2) : E8 ? 2 : 1) void attn_rows_kernel(
    AttnArgs a) {
  using C = RowsCfg<T, DP, E8>;
  constexpr int V = C::V, W = C::W, KS = C::KS, NV = C::NV, VS = C::VS;
  __shared__ float s_o[NWAVE][RB][C::OP];
  __shared__ float s_m[NWAVE][RB], s_l[NWAVE][RB];

  const int lane = threadIdx.x % WAVE;
  const int wave = uniform((int)threadIdx.x / WAVE);
  const int r = lane & 15;

  // One segment: block `blk` of head h of a batch row against keys [k0, k1) of
  // its [kal, kend).  With parts > 1 other workgroups have the block's other
  // keys: the outputs go to partial row block `slot`, and the last of the parts
  // to arrive at *count joins them, part c being row block slot0 for c = 0 and
  // slotc + c * dslot after it.
  auto segment = [&](Tile t, int h, int kbeg, int kend, int k0, int k1, int parts, uint32_t slot,
                     uint32_t slot0, uint32_t slotc, uint32_t dslot, int* count) {
  for (int* p : {&t.row.begin, &t.row.n, &t.row.p0, &t.row.seq, &t.rho0, &t.nrow, &t.minpos,
                 &t.maxpos, &h, &kbeg, &kend, &k0, &k1, &parts})
    *p = uniform(*p);  // they are; the compiler loses sight of it in the loop below
  const int rr = min(r, t.nrow - 1);
  const int tok = (t.rho0 + rr) / a.G, head = h * a.G + (t.rho0 + rr) % a.G;
  const int qpos = t.row.p0 + tok;
  f32x4 o[1][VS][NV];
  float m[1], l[1];
  bool missing;
  const char* const qp[1] = {a.q + (int64_t)(t.row.begin + tok) * a.q_stride +
                             (int64_t)head * a.D * W};
  const int qps[1] = {qpos};
  rows_keys<T, DP, FULL, E8, false, 1>(threadIdx.x, a, a.table + (int64_t)t.row.seq * a.M, h,
                                       t.minpos, t.maxpos, kbeg, kend, k0, k1, qp, qps, o, m, l,
                                       missing);
  if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);

  // the four waves' results meet in LDS
  rows_meet<C>(o[0], m[0], l[0], s_o, s_m, s_l);
  __syncthreads();
  auto store_out = [&](int qr, int d, float4 sum, float L) {
    const float inv = 1.f / L;
    const bool none = L == 0.f;  // a row that sees nothing is zero
    const float f[4] = {none ? 0.f : sum.x * inv, none ? 0.f : sum.y * inv,
                        none ? 0.f : sum.z * inv, none ? 0.f : sum.w * inv};
    const int rho = t.rho0 + qr;
    char* op = a.out + (int64_t)(t.row.begin + rho / a.G) * a.out_stride +
               ((int64_t)(h * a.G + rho % a.G) * a.D + d) * W;
    if constexpr (V == 8)
      *(uint2*)op = make_uint2(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]));
    else
      *(float4*)op = make_float4(f[0], f[1], f[2], f[3]);
  };
  constexpr int TD = DP / 4;
  const __amdgpu_buffer_rsrc_t prs = make_rsrc(a.part, (uint32_t)KV_PART_ROWS * DP * 4);
  for (int u = threadIdx.x; u < t.nrow * TD; u += ROWS_T) {
    const int qr = u / TD, d = u % TD * 4;
    float M, L;
    const float4 sum = rows_met<C>(s_o, s_m, s_l, qr, d, M, L);
    if (parts > 1) {
      const uint32_t row = slot * a.prow + qr;
      buf_store16_agent(prs, (row * DP + d) * 4, sum);
      if (d == 0)
        __hip_atomic_store((uint64_t*)a.ml + row,
                           (uint64_t)__float_as_uint(L) << 32 | __float_as_uint(M),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else if (d < a.D) {
      store_out(qr, d, sum, L);
    }
  }
  if (parts <= 1) return;

  // The last workgroup of a block to arrive joins its parts: the stores
  // above go to the level that all XCDs share, and are complete before the
  // count rises.  The order of the sums is that of the parts, whoever joins.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  int* const s_last = (int*)&s_l[0][0];
  if (threadIdx.x == 0) {
    const int old = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *s_last = old == parts - 1;
    if (old == parts - 1)  // for the next call
      __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!*s_last) return;
  // the weight of each part, a wave per row
  auto part_row = [&](int c) { return (c ? slotc + c * dslot : slot0) * a.prow; };
  float* const s_w = &s_o[0][0][0];  // [nrow][MAX_SPLITS]
  static_assert(sizeof(s_o) >= RB * MAX_SPLITS * 4 + ROWS_T * 16, "weights and sums fit");
  for (int qr = wave; qr < t.nrow; qr += NWAVE) {
    float mx[MAX_SPLITS / WAVE], ls[MAX_SPLITS / WAVE];
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < MAX_SPLITS / WAVE; ++i) {
      const int c = lane + i * WAVE;
      uint64_t v = __float_as_uint(-INFINITY);
      if (c < parts)
        v = __hip_atomic_load((uint64_t*)a.ml + part_row(c) + qr, __ATOMIC_RELAXED,
                              __HIP_MEMORY_SCOPE_AGENT);
      mx[i] = __uint_as_float((uint32_t)v);
      ls[i] = __uint_as_float((uint32_t)(v >> 32));
      M = fmaxf(M, mx[i]);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, WAVE));
    float L = 0.f;
#pragma unroll
    for (int i = 0; i < MAX_SPLITS / WAVE; ++i) {
      const float f = mx[i] == -INFINITY ? ls[i] : __builtin_amdgcn_exp2f(mx[i] - M);
      L += f * ls[i];
      s_w[qr * MAX_SPLITS + lane + i * WAVE] = f;
    }
    L = wave_sum(L);
    if (lane == 0) s_m[0][qr] = L;
  }
  __syncthreads();
  // 16-byte pieces of the rows over the threads; with fewer pieces than
  // threads, several threads share a piece's parts
  const int units = t.nrow * TD;
  const int sub = units >= ROWS_T ? 1 : ROWS_T / units;
  float4* const s_sum = (float4*)(s_w + RB * MAX_SPLITS);
  for (int u0 = 0; u0 < units; u0 += ROWS_T) {
    const int u = u0 + (sub > 1 ? (int)threadIdx.x % units : (int)threadIdx.x);
    const int part = sub > 1 ? (int)threadIdx.x / units : 0;
    const int qr = u / TD, d = u % TD * 4;
    float4 sum = make_float4(0, 0, 0, 0);
    if (u < units && part < sub) {
      // a round trip past the L2 takes microseconds: many loads in flight
      auto add_parts = [&](auto batch) {
        constexpr int NB = decltype(batch)::value;
        for (int c0 = part; c0 < parts; c0 += NB * sub) {
          float4 v[NB];
#pragma unroll
          for (int i = 0; i < NB; ++i) {
            const int c = c0 + i * sub;
            v[i] = buf_load16_agent(prs, c < parts ? ((part_row(c) + qr) * DP + d) * 4 : BUF_OOB);
          }
#pragma unroll
          for (int i = 0; i < NB; ++i) {
            const float w = s_w[qr * MAX_SPLITS + min(c0 + i * sub, MAX_SPLITS - 1)];
            sum.x += w * v[i].x;
            sum.y += w * v[i].y;
            sum.z += w * v[i].z;
            sum.w += w * v[i].w;
          }
        }
      };
      if (parts > 4 * sub) add_parts(std::integral_constant<int, 16>{});
      else add_parts(std::integral_constant<int, 4>{});
    }
    if (sub > 1) {
      s_sum[threadIdx.x] = sum;
      __syncthreads();
      if (part) continue;
      for (int i = 1; i < sub; ++i) {
        const float4 v = s_sum[threadIdx.x + i * units];
        sum.x += v.x;
        sum.y += v.y;
        sum.z += v.z;
        sum.w += v.w;
      }
    }
    if (u < units && d < a.D) store_out(qr, d, sum, s_m[0][qr]);
  }
  };

  if constexpr (!EVEN) {
    const int id = grid_block();  // past the last block: a split there is none of
    const int h = id % a.Hkv, tile = id / a.Hkv % a.tiles, split = id / a.Hkv / a.tiles;
    int32_t* const err = split == 0 && h == 0 ? a.err : nullptr;
    int row, blk;
    Tile t;
    if (!find_block<RB>(a.b, a.G, tile, err, &row, &blk) ||
        !make_tile<RB>(kv_row(a.b, row, threadIdx.x == 0 ? err : nullptr), a.G, blk, &t))
      return;
    const int kbeg = first_key(t, a.window), kend = t.maxpos + 1;
    const int kal = kbeg / KS * KS;
    const int ns = min(a.splits, max(1, (kend - kal + a.chunk - 1) / a.chunk));
    if (split >= ns) return;
    const int k0 = kal + split * a.chunk;
    const uint32_t block = tile * a.Hkv + h, slot0 = block * a.splits;
    segment(t, h, kbeg, kend, k0, split + 1 < ns ? k0 + a.chunk : kend, ns, slot0 + split, slot0,
            slot0, 1, a.count + block);
  } else {
    // One token a row.  The keys of all blocks, in groups of GROUP, lie one
    // block after the other on a line, and every workgroup has an equal stretch
    // of it, whatever the lengths of the rows: row by row nb = (blocks of 16
    // heads) * Hkv blocks of the row's groups each.
    const int per = (a.G + RB - 1) / RB, nb = per * a.Hkv;
    auto groups_of = [&](int p0) {  // a row that sees nothing has one, for its zeros
      const int first = a.window && p0 >= 0 ? max(0, p0 - a.window + 1) / KS * KS : 0;
      return max(1, (p0 + 1 - first + GROUP - 1) / GROUP);
    };
    // rows i0 .. i0 + 63 of the batch, one a lane
    KvRow lr;
    int i0 = 0;
    auto load_rows = [&](int first) {
      i0 = first;
      const int i = min(first + lane, a.b.n_seq - 1);
      const KvRawRow w = {i, i + 1, a.b.seqs ? a.b.seqs[i] : i, a.b.pos0[i]};
      lr = kv_row_check(a.b, w, blockIdx.x == 0 && threadIdx.x < WAVE ? a.err : nullptr);
      return first + lane < a.b.n_seq ? groups_of(lr.p0) : 0;
    };
    auto row_at = [&](int i) {
      if (i >= i0 + WAVE) load_rows(i);
      KvRow k;
      k.begin = i;
      k.n = 1;
      k.p0 = __builtin_amdgcn_readlane(lr.p0, i - i0);
      k.seq = __builtin_amdgcn_readlane(lr.seq, i - i0);
      return k;
    };
    int n = 0, sum = 0;
    for (int i = (a.b.n_seq - 1) / WAVE * WAVE; i >= 0; i -= WAVE) {
      n = load_rows(i);
      sum += n;
    }
    sum = __builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)sum), WAVE - 1);
    const int total = uniform(sum * nb);
    // no block may have more than MAX_SPLITS parts: a.chunk groups at least
    const int share = max(a.chunk, (total + (int)gridDim.x - 1) / (int)gridDim.x);
    // workgroups go round the eight XCDs; each XCD gets one stretch in a piece
    const int wg = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    int at = wg * share;
    const int end = min(total, at + share);
    if (at >= end) return;
    // the row, block and group of the first key of the stretch
    int row = 0, before = 0;  // groups of the rows before
    for (const int want = at / nb;; n = load_rows(i0 + WAVE)) {
      const int incl = (int)wave_incl_scan((uint32_t)n);
      const uint64_t hit = __ballot(before + incl > want);
      if (hit) {
        const int l = __ffsll((unsigned long long)hit) - 1;
        row = i0 + l;
        before += __builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(n, l);
        break;
      }
      before += __builtin_amdgcn_readlane(incl, WAVE - 1);
    }
    row = uniform(row);
    before = uniform(before);
    KvRow kr = row_at(row);
    int groups = uniform(groups_of(kr.p0));
    int j = (at - before * nb) / groups;
    int start = before * nb + j * groups;  // of the block on the line
    while (true) {
      Tile t;
      make_tile<RB>(kr, a.G, j / a.Hkv, &t);
      const int kbeg = first_key(t, a.window), kend = t.maxpos + 1;
      const int kal = kbeg / KS * KS;
      const int stop = min(end, start + groups);
      const int w0 = start / share, w1 = (start + groups - 1) / share;
      // a workgroup has at most two blocks that it shares: the one its stretch
      // begins in, or the one it ends in
      const uint32_t slot0 = 2 * w0 + (w0 * share < start ? 1 : 0);
      segment(t, j % a.Hkv, kbeg, kend, kal + (at - start) * GROUP,
              min(kend, kal + (stop - start) * GROUP), w1 - w0 + 1,
              wg == w0 ? slot0 : 2 * wg, slot0, 2 * w0, 2, a.count + w0);
      at = stop;
      if (at >= end) return;
      start += groups;
      if (++j == nb) {
        j = 0;
        kr = row_at(++row);
        groups = uniform(groups_of(kr.p0));
      }
      __syncthreads();  // LDS is free again
    }
  }
}

// One token a row, a wave for all keys of a block: no exchange between waves, and
// as many blocks under way as the card holds waves.  A lane has its query's
// outputs, NV of them together, so they leave from the registers.
template <class T, int DP, bool FULL, bool E8>
__global__ __launch_bounds__(ROWS_T, DP < 256 ? (E8 ? 3 : 2) : E8 ? 2 : 1) void attn_waves_kernel(
    AttnArgs a) {
  using C = RowsCfg<T, DP, E8>;
  constexpr int V = C::V, W = C::W, NV = C::NV;
  const int lane = threadIdx.x % WAVE, r = lane & 15, g = lane >> 4;
  const int id = uniform(grid_block() * NWAVE + (int)threadIdx.x / WAVE);
  const int per = (a.G + RB - 1) / RB, nb = per * a.Hkv;
  const int row = id / nb, j = id % nb, h = j % a.Hkv;
  if (row >= a.b.n_seq) return;
  Tile t;
  make_tile<RB>(kv_row(a.b, row, j == 0 && lane == 0 ? a.err : nullptr), a.G, j / a.Hkv, &t);
  for (int* p : {&t.row.begin, &t.row.p0, &t.row.seq, &t.minpos, &t.maxpos}) *p = uniform(*p);
  const int kbeg = first_key(t, a.window), kend = t.maxpos + 1;
  const int head = h * a.G + t.rho0 + min(r, t.nrow - 1);
  const char* const qp[1] = {a.q + (int64_t)t.row.begin * a.q_stride + (int64_t)head * a.D * W};
  const int qpos[1] = {t.row.p0};
  f32x4 o[1][C::VS][NV];
  float m[1], l[1];
  bool missing;
  rows_keys<T, DP, FULL, E8, false, 1, 1>(threadIdx.x, a, a.table + (int64_t)t.row.seq * a.M, h,
                                          t.minpos, t.maxpos, kbeg, kend, kbeg / C::KS * C::KS,
                                          kend, qp, qpos, o, m, l, missing);
  if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
  const float sum = sum_groups(l[0]), inv = 1.f / sum;
  const bool none = sum == 0.f;  // a row that sees nothing is zero
  if (r >= t.nrow) return;
  char* op = a.out + (int64_t)t.row.begin * a.out_stride + (int64_t)head * a.D * W;
#pragma unroll
  for (int s = 0; s < C::VS; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 16 * NV * s + NV * (4 * g + i);
      if (d >= a.D) continue;
      float f[NV];
#pragma unroll
      for (int x = 0; x < NV; ++x) f[x] = none ? 0.f : o[0][s][x][i] * inv;
#pragma unroll
      for (int x = 0; x < NV; x += 4)
        if constexpr (V == 8)
          *(uint2*)(op + (d + x) * W) = make_uint2(pack2<T>(f[x], f[x + 1]),
                                                   pack2<T>(f[x + 2], f[x + 3]));
        else
          *(float4*)(op + (d + x) * W) = make_float4(f[x], f[x + 1], f[x + 2], f[x + 3]);
    }
}

// ---------------------------------------------------------------------------
// Tiles: 128 rows against all their keys, for many 16-bit query rows.  Four
// waves of 32 rows share K and V in steps of KB keys through LDS (double
// buffered: the next step's rows are on their way from memory to registers
// while this one is computed).  S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16
// tiles, as in the row blocks: a lane owns query l % 32, its accumulator rows
// 8 a + 4 h + b (h = l / 32) are keys, and the key slots of the second product
// are numbered such that its P operand is the lane's own scores.  V comes out
// of LDS transposed (ds_read_tr: four keys of one column per lane).
//
// 128 rows, so that a step's products (32 cycles a wave and matrix instruction)
// cover the loads of the next; 64 keys, so that two workgroups fit a compute unit
// and one's softmax runs beside the other's products.  No single part bounds it:
// without the LDS reads of V 16384 bf16 tokens with 64 heads of 128 take 6% less,
// without exponentials 5%, without loads 12%; the matrix cores are busy 44% of the
// time, LDS 33%, with no bank conflicts.  Those take 4.5 to 5.0 ms, 880 to
// 980 TFLOP/s (an 8192^3 library product reaches 1140 to 1400, from card to card);
// 2048 fp16 tokens and 32 heads 62 to 65 us (530 to 550 TFLOP/s; a library product
// of as many operations 52 to 57 us).
// 8-bit elements become w between registers and LDS; the second product reads as
// before, at the same rates from heads of 80 on (8192 bf16 tokens of 64 heads over 8 of 128:
// 1.12 ms, 984 TFLOP/s; 4096 of 32 over 8 of 64: 119 us, of 16-bit elements 98).  Two stores
// a row meet in half of the banks; in an order of theirs that does not it takes as long.
// Measured and dropped: one workgroup of eight waves in two groups half a step
// apart, 4.68 to 5.05 ms; the next step's score products dealt between this step's
// exponentials, 4.56 ms (16384 tokens) and 119 against 106 us (packed prompts).
//
// LDS rows are permuted in 16-byte pieces so that neither the row reads of K
// (32 rows, one piece) nor the transposed reads of V (8 rows, four pieces)
// meet in a bank.
// ---------------------------------------------------------------------------
constexpr int TB = 128;
constexpr int TILE_T = 256;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T>
__device__ inline f32x16 mfma32(uint4 a, uint4 b, f32x16 c) {
  if constexpr (T::dtype == NP_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int DP, bool E8>
struct TileCfg {
  static constexpr int KB = DP == 256 ? 32 : 64;    // keys of a step
  static constexpr int KT = KB / 32;                // 32-key tiles of a step
  static constexpr int DT = DP / 32;                // output tiles
  static constexpr int CPR = DP / 8;                // 16-byte pieces of an LDS row
  static constexpr int PL = E8 ? 2 : 1;             // pieces that a 16-byte load becomes
  static constexpr int LPR = CPR / PL;              // loads of a row
  static constexpr int NL = KB * LPR / TILE_T;      // loads of a thread
  static constexpr int RSTEP = TILE_T / LPR;        // rows between them
  static constexpr int WROWS = WAVE / LPR;          // rows of a wave's load
  static constexpr int ROW = CPR * 16;              // bytes of an LDS row
  // piece c of a row lies at piece c ^ kx (K) or c ^ vx (V)
  __device__ static inline int kx(int row) { return DP == 64 ? row >> 1 & 7 : row & 15; }
  __device__ static inline int vx(int row) {
    return DP == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3);
  }
};

// FULL: D == DP; otherwise the pieces past D stay zero in LDS.
// E8: 8-bit elements, turned into w on their way to LDS.
//
// One stretch of keys [kbeg, kend) of the sequence with page table trow, K's head
// h, against a tile's rows: this lane's query at qp has position qpos, those of its
// wave lie in [wmin, wmax].  Afterwards a lane has its query's maximum m, half of
// its sum l (the other half is lane ^ 32's) and its outputs o; missing: a key had no
// page.
// CUT: the rows may see keys from kend on, which other stretches have.
template <class T, int DP, bool FULL, bool E8, bool CUT, class C = TileCfg<DP, E8>>
__device__ __forceinline__ void tile_keys(int tid, const AttnArgs& a, const int32_t* trow, int h,
                                          int kbeg, int kend, int wmin, int wmax, const char* qp,
                                          int qpos, char* s_k, char* s_v, f32x16 (&o)[C::DT],
                                          float& m, float& l, bool& missing) {
  constexpr int KB = C::KB, NL = C::NL, RSTEP = C::RSTEP, KT = C::KT, KD = DP / 16, DT = C::DT;
  const int lane = tid % WAVE;
  const int wave = uniform(tid / WAVE);
  const int r = lane & 31, h2 = lane >> 5;
  // a negative scale turns into negated queries, so that the largest q.k has
  // the largest score
  const uint32_t flip = a.scale < 0 ? 0x80008000u : 0u;
  const float scale = fmaxf(fabsf(a.scale), 1.17549435e-38f);  // not 0: -inf * 0
  uint4 qf[KD];
#pragma unroll
  for (int s = 0; s < KD; ++s) {
    const int d = 16 * s + 8 * h2;
    qf[s] = d < a.D ? *(const uint4*)(qp + d * 2) : make_uint4(0, 0, 0, 0);
    qf[s].x ^= flip;
    qf[s].y ^= flip;
    qf[s].z ^= flip;
    qf[s].w ^= flip;
  }

#pragma unroll
  for (int j = 0; j < DT; ++j) o[j] = (f32x16)(0.f);
  m = -INFINITY;
  l = 0.f;

  // Loads: 16 bytes lc of rows lr, lr + RSTEP, ...  A wave's rows of one load lie
  // in 16 consecutive keys, so in one page: page ids and row blocks are scalar,
  // and a lane adds an offset that stays the same.  Rows outside the tile's
  // keys repeat its first or last one: they get no weight, but have to be
  // finite.
  const int lc = tid % C::LPR, lr = tid / C::LPR;
  const bool lon = FULL || lc * 8 * C::PL < a.D;
  const int P1 = (1 << a.pshift) - 1;
  const int rowb = a.D * (E8 ? 1 : 2);  // of the cache
  const size_t headb = ((size_t)rowb + (E8 ? 1 : 0)) << a.pshift;
  const size_t vofs = a.Hkv * headb;
  const char* hpool = a.pool + h * headb;
  u32x4_t sk[NL] = {}, sv[NL] = {};
  uint32_t ks[NL], vs[NL];  // E8: the rows' scale bytes
  constexpr int NB = KB / 16;  // blocks of 16 keys in a step: each in one page
  // the block of the step that this wave's load i is in
  auto block_of = [&](int i) { return (RSTEP * i + C::WROWS * wave) / 16; };
  uint32_t lofs[NL], sofs[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int row = lr + RSTEP * i - 16 * block_of(i);
    lofs[i] = row * rowb + lc * 16;
    sofs[i] = (rowb << a.pshift) + row;  // scales follow a head's elements
  }
  int ids[NB];
  // a table that names no page for some key of the step: its keys are looked up
  // again and masked one by one
  bool bad = false, next_bad = false;
  missing = false;
  auto load_pages = [&](int base) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
      ids[b] = load_scalar(trow, max(kbeg, min(base + 16 * b, kend - 1)) >> a.pshift);
  };
  auto load_rows = [&](int base) {
    int page[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i)
      if constexpr (4 * C::WROWS <= 16)  // the four waves' rows
        page[i] = ids[RSTEP * i / 16];
      else if constexpr (4 * C::WROWS == 32)
        page[i] = wave >> 1 ? ids[2 * i + 1] : ids[2 * i];
      else
        page[i] = wave >> 1 ? (wave & 1 ? ids[4 * i + 3] : ids[4 * i + 2])
                            : (wave & 1 ? ids[4 * i + 1] : ids[4 * i]);
    const char* p[NL];
    uint32_t o[NL], so[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      p[i] = hpool + (int64_t)page[i] * (int64_t)a.page_bytes;
      const int slot = (base + 16 * block_of(i)) & P1;
      o[i] = lofs[i] + slot * rowb;
      so[i] = sofs[i] + slot;
    }
    if (base < kbeg || base + KB > kend) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int slot = max(kbeg, min(base + lr + i * RSTEP, kend - 1)) & P1;
        o[i] = slot * rowb + lc * 16;
        so[i] = (rowb << a.pshift) + slot;
      }
    }
    const char* pv[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) pv[i] = p[i] + vofs;
    next_bad = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) next_bad |= (uint32_t)ids[b] >= (uint32_t)a.N;
    if (next_bad)
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (page[i] < 0 || page[i] >= a.N) {  // masked below, but has to be finite
          p[i] = pv[i] = a.zeros;
          o[i] = lc * 16;
          so[i] = 0;
        }
    if (lon) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        if constexpr (E8) {
          ks[i] = load_global1(p[i] + so[i]);
          vs[i] = load_global1(pv[i] + so[i]);
        }
        sk[i] = load_global16(p[i] + o[i]);
        sv[i] = load_global16(pv[i] + o[i]);
      }
    }
  };
  auto store_rows = [&](int buf) {
    if (lon) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = lr + i * RSTEP, at = (buf * KB + row) * C::ROW;
        if constexpr (E8) {
          const float fk = scale_of_byte(ks[i]), fv = scale_of_byte(vs[i]);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int c = 2 * lc + x;
            *(u32x4_t*)(s_k + at + (c ^ C::kx(row)) * 16) = elements16<T>(sk[i], x, fk);
            *(u32x4_t*)(s_v + at + (c ^ C::vx(row)) * 16) = elements16<T>(sv[i], x, fv);
          }
        } else {
          *(u32x4_t*)(s_k + at + (lc ^ C::kx(row)) * 16) = sk[i];
          *(u32x4_t*)(s_v + at + (lc ^ C::vx(row)) * 16) = sv[i];
        }
      }
    }
  };
  if constexpr (!FULL) {
    if (!lon)
#pragma unroll
      for (int i = 0; i < 2 * NL; ++i) {
        const int row = lr + i * RSTEP;
#pragma unroll
        for (int x = 0; x < C::PL; ++x) {
          const int c = C::PL * lc + x;
          *(u32x4_t*)(s_k + row * C::ROW + (c ^ C::kx(row)) * 16) = (u32x4_t)(0u);
          *(u32x4_t*)(s_v + row * C::ROW + (c ^ C::vx(row)) * 16) = (u32x4_t)(0u);
        }
      }
  }

  // the keys that this lane's query counts
  const int klast_seen = CUT ? min(qpos, kend - 1) : qpos;
  const int kfirst_seen = a.window ? qpos - a.window + 1 : 0;

  // LDS addresses of a lane.  K: piece 2 s + h2 of row r (+ 32 kt); V: four
  // columns of rows vr and vr + 8 (+ 16 mm), column 32 j + vc.  The pieces' xor
  // with s or j can be taken on the whole address, since rows are aligned.
  const int vr = 4 * h2 + (lane >> 2 & 3), vc = 16 * (lane >> 4 & 1) + 4 * (lane & 3);
  const uint32_t ka = r * C::ROW + (h2 ^ C::kx(r)) * 16;
  const uint32_t va = vr * C::ROW + ((vc >> 3) ^ C::vx(vr)) * 16 + (vc & 4) * 2;
  const uint32_t vb = (vr + 8) * C::ROW + ((vc >> 3) ^ C::vx(vr + 8)) * 16 + (vc & 4) * 2;

  const int k0 = kbeg / KB * KB;
  if (kend > 0) {
    load_pages(k0);
    __builtin_amdgcn_sched_barrier(0);  // all ids before the first is waited for
    load_rows(k0);
    load_pages(k0 + KB);
    store_rows(0);
  }
  __syncthreads();
  int buf = 0;
  if (CUT && wmax < 0) {  // a wave without rows: its share of the loads
    for (int base = k0; base < kend; base += KB, buf ^= 1) {
      if (base + KB < kend) {
        load_rows(base + KB);
        load_pages(base + 2 * KB);
        store_rows(buf ^ 1);
      }
      __syncthreads();
    }
    return;
  }
  for (int base = k0; base < kend; base += KB, buf ^= 1) {
    const bool more = base + KB < kend;
    bad = next_bad;
    missing |= bad;
    if (more) {
      load_rows(base + KB);
      load_pages(base + 2 * KB);
    }
    // CUT: all steps count; a step left out would cost moves of the outputs
    // between registers in every other one
    if (CUT || (base <= wmax && (a.window == 0 || base + KB - 1 > wmin - a.window))) {
      const bool full = !bad && base + KB - 1 <= wmin &&
                        (a.window == 0 || base > wmax - a.window) && (!CUT || base + KB <= kend);
      const uint32_t bo = buf * KB * C::ROW;
      f32x16 sc[KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) sc[kt] = (f32x16)(0.f);
#pragma unroll
      for (int s = 0; s < KD; ++s)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const u32x4_t k = *(const u32x4_t*)(s_k + ((ka + bo) ^ (32 * s)) + 32 * kt * C::ROW);
          sc[kt] = mfma32<T>(as_uint4(k), qf[s], sc[kt]);
        }
      if (!full) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = base + 32 * kt + 8 * (i / 4) + 4 * h2 + i % 4;
            if (key > klast_seen || key < kfirst_seen) sc[kt][i] = -INFINITY;
          }
        if (bad) {
          uint32_t hide = 0;  // bit 16 kt + i
#pragma unroll 1
          for (int x = 0; x < 16 * KT; ++x) {
            const int key = base + x / 16 * 32 + 8 * (x % 16 / 4) + 4 * h2 + x % 4;
            const int p = trow[min(key, kend - 1) >> a.pshift];
            if (p < 0 || p >= a.N) hide |= 1u << x;
          }
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (hide >> (16 * kt + i) & 1) sc[kt][i] = -INFINITY;
        }
      }
      float mx = sc[0][0];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[kt][i]);
      {
        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx),
                                                        false, false);
        mx = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * scale;
      }
      // m follows the maximum only when it falls 8 behind (in powers of two):
      // probabilities then reach 2^8 at most, and the outputs are rarely scaled
      if (__any(mx > m + 8.f)) {
        const float mn = fmaxf(m, mx);
        const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[j] *= alpha;
      }
      const float mu = m == -INFINITY ? 0.f : m;
      uint4 pf[2 * KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][i], scale, -mu));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kt][i + 1], scale, -mu));
          l += p0 + p1;
          u[i / 2] = pack2<T>(p0, p1);  // rounded to w, as the matrix cores take it
        }
        pf[2 * kt] = make_uint4(u[0], u[1], u[2], u[3]);
        pf[2 * kt + 1] = make_uint4(u[4], u[5], u[6], u[7]);
      }
      // V^T: rows 32 j + l % 32, keys 16 mm + 4 h + {0..3} and 8 further
#pragma unroll
      for (int mm = 0; mm < 2 * KT; ++mm)
#pragma unroll
        for (int j = 0; j < DT; ++j) {
          typedef __attribute__((address_space(3))) s16x4 lds4;
          const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4*)(s_v + ((va + bo) ^ (64 * j)) + 16 * mm * C::ROW));
          const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4*)(s_v + ((vb + bo) ^ (64 * j)) + 16 * mm * C::ROW));
          const uint2 xu = __builtin_bit_cast(uint2, x), yu = __builtin_bit_cast(uint2, y);
          o[j] = mfma32<T>(make_uint4(xu.x, xu.y, yu.x, yu.y), pf[mm], o[j]);
        }
    }
    if (more) store_rows(buf ^ 1);
    __syncthreads();
  }
}

template <class T, int DP, bool FULL, bool E8>
__global__ __launch_bounds__(TILE_T, DP == 256 ? 1 : 2) void attn_tile_kernel(AttnArgs a) {
  using C = TileCfg<DP, E8>;
  constexpr int KB = C::KB, DT = C::DT;
  __shared__ __attribute__((aligned(1024))) char s_k[2 * KB * C::ROW];
  __shared__ __attribute__((aligned(1024))) char s_v[2 * KB * C::ROW];

  const int tid = threadIdx.x, lane = tid % WAVE;
  const int wave = uniform(tid / WAVE);
  const int r = lane & 31, h2 = lane >> 5;
  const int h = blockIdx.x % a.Hkv, rank = blockIdx.x / a.Hkv % a.tiles;
  const int split = blockIdx.x / a.Hkv / a.tiles;
  Tile t;
  int32_t* const err = split == 0 && h == 0 ? a.err : nullptr;
  int row, blk;
  if (!find_block_longest<TB>(a.b, a.G, rank, a.tiles, err, &row, &blk) ||
      !make_tile<TB>(kv_row(a.b, row, tid == 0 ? err : nullptr), a.G, blk, &t))
    return;

  // the tile's keys, in steps, and this part of them
  const int tbeg = first_key(t, a.window), tend = t.maxpos + 1;
  const int step0 = tbeg / KB, steps = (tend + KB - 1) / KB - step0;
  const int parts = max(1, min(a.splits, (steps + a.chunk - 1) / a.chunk));
  if (split >= parts) return;
  const int kbeg = max(tbeg, (step0 + steps * split / parts) * KB);
  const int kend = min(tend, (step0 + steps * (split + 1) / parts) * KB);
  const int rowb = a.D * 2;

  // this wave's rows and this lane's query
  const int w0 = min(wave * 32, t.nrow - 1), w1 = min(wave * 32 + 31, t.nrow - 1);
  const int wmin = t.row.p0 < 0 ? -1 : t.row.p0 + (t.rho0 + w0) / a.G;
  const int wmax = t.row.p0 < 0 ? -1 : t.row.p0 + (t.rho0 + w1) / a.G;
  const int rho = t.rho0 + min(wave * 32 + r, t.nrow - 1);
  const int tok = rho / a.G, head = h * a.G + rho % a.G;
  const int qpos = t.row.p0 < 0 ? -1 : t.row.p0 + tok;
  const char* qp = a.q + (int64_t)(t.row.begin + tok) * a.q_stride + (int64_t)head * rowb;
  f32x16 o[DT];
  float m, l;
  bool missing;
  tile_keys<T, DP, FULL, E8, false>(tid, a, a.table + (size_t)t.row.seq * a.M, h, kbeg, kend, wmin,
                                    wmax, qp, qpos, s_k, s_v, o, m, l, missing);
  if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);

  l = swap32_add(l, l);
  if (parts > 1) {
    // as in the row blocks: the parts to the level that all XCDs share, the last
    // to arrive adds them up in their order.  A thread's outputs are its own in
    // every part, so they go out as they lie in the registers.
    const __amdgpu_buffer_rsrc_t prs = make_rsrc(a.part, (uint32_t)KV_PART_ROWS * DP * 4);
    constexpr int NO = 4 * DT;  // 16-byte pieces of a thread
    const uint32_t block = (uint32_t)rank * a.Hkv + h, slot0 = block * a.splits;
    auto at = [&](int c, int i) { return (((slot0 + c) * NO + i) * TILE_T + tid) * 16; };
    uint64_t* const ml = (uint64_t*)a.ml + (size_t)slot0 * TB + wave * 32 + r;
    const bool live = wave * 32 < t.nrow;  // a wave past the tile's rows has nothing to join
    if (live)
#pragma unroll
      for (int i = 0; i < NO; ++i)
        buf_store16_agent(prs, at(split, i),
                          make_float4(o[i / 4][i % 4 * 4], o[i / 4][i % 4 * 4 + 1],
                                      o[i / 4][i % 4 * 4 + 2], o[i / 4][i % 4 * 4 + 3]));
    if (live && h2 == 0)
      __hip_atomic_store(ml + split * TB, (uint64_t)__float_as_uint(l) << 32 | __float_as_uint(m),
                         __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int* const s_last = (int*)s_k;
    if (tid == 0) {
      int* const count = a.count + block;
      const int old = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      *s_last = old == parts - 1;
      if (old == parts - 1)  // for the next call
        __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!*s_last || !live) return;
    // a round trip past the L2 takes about a microsecond: several loads at once
    auto stats = [&](int c) {
      return __hip_atomic_load(ml + min(c, parts - 1) * TB, __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    };
    float M = -INFINITY;
    for (int c = 0; c < parts; c += 8) {
      uint64_t v[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] = stats(c + x);
#pragma unroll
      for (int x = 0; x < 8; ++x) M = fmaxf(M, __uint_as_float((uint32_t)v[x]));
    }
    l = 0.f;
#pragma unroll
    for (int j = 0; j < DT; ++j) o[j] = (f32x16)(0.f);
    for (int c = 0; c < parts; c += 2) {
      const uint64_t st[2] = {stats(c), stats(c + 1)};
      float4 v[2][NO];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < NO; ++i)
          v[x][i] = buf_load16_agent(prs, c + x < parts ? at(c + x, i) : BUF_OOB);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float mc = __uint_as_float((uint32_t)st[x]);
        const float lc = c + x < parts ? __uint_as_float((uint32_t)(st[x] >> 32)) : 0.f;
        // without a maximum the sum is 0, or NaN when every score was
        const float f = mc == -INFINITY ? lc : __builtin_amdgcn_exp2f(mc - M);
        l += f * lc;
#pragma unroll
        for (int i = 0; i < NO; ++i) {
          o[i / 4][i % 4 * 4] += f * v[x][i].x;
          o[i / 4][i % 4 * 4 + 1] += f * v[x][i].y;
          o[i / 4][i % 4 * 4 + 2] += f * v[x][i].z;
          o[i / 4][i % 4 * 4 + 3] += f * v[x][i].w;
        }
      }
    }
  }
  if (wave * 32 + r >= t.nrow) return;
  const bool none = l == 0.f;  // a row that sees nothing is zero
  const float inv = 1.f / l;
  char* op = a.out + (int64_t)(t.row.begin + tok) * a.out_stride + (int64_t)head * rowb;
#pragma unroll
  for (int j = 0; j < DT; ++j)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = 32 * j + 2 * i + 4 * h2;
      if (d >= a.D) continue;
      *(uint2*)(op + d * 2) =
          none ? make_uint2(0, 0)
               : make_uint2(pack2<T>(o[j][i] * inv, o[j][i + 1] * inv),
                            pack2<T>(o[j][i + 2] * inv, o[j][i + 3] * inv));
    }
}

// The keys of a tile are split while the tiles do not give every compute unit two
// workgroups (64 tokens of 32 heads over 8 behind 32000 others: 774 us unsplit, 75
// split; 256 tokens behind 2000: 63 and 30), but into 32 parts at most and 256 keys
// at least: the join costs about 0.6 us a part (8 tokens of 64 heads over 8 behind
// 32000: 48 in 32 parts, 54 in 64; 256 tokens of 32 over 8 behind 2000: 30 with
// 256 keys a part, 35 with 512).
template <class T, int DP, bool E8>
hipError_t launch_tile(AttnArgs a, hipStream_t stream) {
  constexpr int KB = TileCfg<DP, E8>::KB;
  a.tiles = (int)((int64_t)a.b.n_tokens * a.G / TB) + a.b.n_seq;
  const int64_t blocks = (int64_t)a.tiles * a.Hkv;
  int64_t keys = a.b.lim;  // the most a tile can see
  if (a.window > 0) keys = std::min<int64_t>(keys, (int64_t)a.window + TB + KB);
  int64_t splits = std::min({(512 + blocks - 1) / blocks, keys / 256, (int64_t)32,
                             (int64_t)KV_PART_ROWS / (TB * blocks)});
  if (splits < 1 || blocks > KV_MAX_BLOCKS) splits = 1;
  a.splits = (int)splits;
  a.chunk = (int)(((keys + KB - 1) / KB + splits - 1) / splits);
  const dim3 grid((unsigned)(blocks * splits));
  if (a.D == DP)
    hipLaunchKernelGGL((attn_tile_kernel<T, DP, true, E8>), grid, dim3(TILE_T), 0, stream, a);
  else
    hipLaunchKernelGGL((attn_tile_kernel<T, DP, false, E8>), grid, dim3(TILE_T), 0, stream, a);
  return hipGetLastError();
}

// Whether even shares deal more than 768 blocks of up to 256 keys better than a wave for
// each block does.  The card has 1024 such blocks at once, a workgroup of four on every
// compute unit; units that get one more take up to twice as long over long blocks, while
// the shares stay even.  Us, even shares / a wave each, 32 heads over 32, rows of 1 to `keys`
// keys, by the number of blocks:
//                       1024         1088         1280         1536         1792         2176
//   fp32 128, 256  39.9 / 39.6  42.6 / 63.2  51.5 / 65.2  59.6 / 66.2  62.9 / 69.0  73.8 / 89.4
//        128, 128  20.6 / 18.1  28.4 / 30.1  30.2 / 34.6  30.9 / 34.7  40.0 / 35.8  48.7 / 40.6
//         64, 256  24.6 / 21.4  24.8 / 29.3  31.5 / 33.2  35.5 / 34.9  37.7 / 36.3  42.7 / 47.4
//         64, 128  13.4 / 11.2  17.4 / 15.4  17.8 / 16.8  18.0 / 17.0  23.0 / 18.0  28.1 / 20.5
//        256, 256  79.8 / 70.5  82.9 / 83.1   103 / 101    117 / 105    122 / 119    144 / 128
//   fp16 128, 256  24.2 / 20.2  25.9 / 30.5  31.6 / 31.6  35.5 / 32.7  37.6 / 34.8  43.3 / 42.1
//        128, 128  12.4 / 10.0  15.4 / 13.3  16.1 / 15.1  16.6 / 15.1  20.7 / 16.6  25.9 / 19.1
//   fp32 and 8-bit elements:
//        128, 256  34.8 / 28.9  34.4 / 43.3  35.8 / 46.5  42.7 / 46.7  43.1 / 47.2  52.3 / 54.7
//        128, 128  22.0 / 16.8  21.9 / 22.7  22.1 / 25.6  22.3 / 25.5  33.4 / 25.8  33.8 / 26.0
// Rows that all have 256 keys: fp32 of 256, 1088 blocks, 112 / 138.  16-bit heads over 8-bit
// elements of up to 128 take 0.34 to 1.09 of the even shares' time throughout.
template <class T, int DP, bool E8>
bool shares_better(int D, int64_t blocks, int64_t keys) {
  const int64_t rounds = (blocks + 1023) / 1024, bytes = keys * D * (16 / T::V);
  auto filled_below = [&](int percent) { return blocks * 100 < rounds * 1024 * percent; };
  if (E8) return T::V == 4 && keys > 64 && rounds == 2 && filled_below(80);
  if (DP == 256) return bytes > 192 * 1024 && rounds == 2 && filled_below(65);
  if (T::V == 8) return bytes > 48 * 1024 && rounds == 2 && filled_below(65);
  return (bytes > 48 * 1024 && rounds == 2 && filled_below(80)) ||
         (keys > 192 && D == DP && (rounds == 2 || rounds == 3) && filled_below(90));
}

// keys: the most a block can see.  Four ways to deal the keys of `blocks`
// blocks to workgroups (us, fp16 or bf16, D 128, before -> with the rule):
//  - Every 128 keys to a workgroup of its own while all of them fit on the card
//    at once (three to a compute unit): one row of 777 keys and 32 heads 9.3
//    with 256 keys each, 8.9 with 128.
//  - More keys, one row: as many workgroups as compute units, since a long
//    stream from few places is the fastest (131072 keys, 8 key-value heads: 95
//    with 256 workgroups, 99 with 512, 105 with 768).
//  - More keys, several rows, whose lengths the host does not know: an even
//    share of all keys to each of 512 workgroups (64 rows of 1 to 8192 keys:
//    70, against 80 with the best fixed split of each row, most of whose
//    workgroups find nothing to do).  8-bit elements leave registers for three
//    workgroups a compute unit up to heads of 128: 768 of them (64 rows of 47,000
//    keys in all, 8 key-value heads, 97 MB: 27.1, with 512 30.4).
//  - Many blocks of few keys: each would cost its workgroup the whole chain from
//    table to join for a step or two of its waves; up to 256 keys a wave has a
//    block to itself, and all of them are under way at once.  Us, even shares / a
//    wave each, rows of 1 to 64, 256 and 512 keys: 8-bit elements, 32 rows of 32
//    heads over 32 11.1 / 6.1, 19.7 / 12.9, 22.2 / 21.3, 160 rows 30.8 / 13.5, 53.6 /
//    36.5, 96.6 / 72.4; fp16 36.4 / 18.9, 87.8 / 75.0, 152 / 145; fp32 of 64 and 8-bit
//    elements 34.3 / 17.2, 71 / 47, 109 / 95; but with 512 blocks, 64 rows of 32 over
//    8, of 256 keys 12.6 / 11.6, 13.3 / 13.8, 14.6 / 19.6.  But see shares_better.
// Prompts (rows of more tokens) have many blocks; they are split while those do
// not give every compute unit two workgroups (64 tokens of 32 heads over 8 behind
// 2000 others: 29 with one a compute unit, 23 with two), or one if they are few
// (up to 64: 8 tokens behind 32000 others 38 and 47), in pieces of at least 256
// keys (a join costs about 3 us: 250 fp32 keys 10.2 in two pieces, 7.4 in one).
template <class T, int DP, bool E8>
hipError_t launch_rows(AttnArgs a, int64_t keys, int max_tokens, hipStream_t stream) {
  const int64_t blocks = (int64_t)a.tiles * a.Hkv;
  const int64_t groups = (keys + GROUP - 1) / GROUP;
  a.prow = a.b.cu ? RB : std::min(a.G, RB);
  const bool ones = !a.b.cu || max_tokens <= 1;
  const bool small = ones && groups * blocks <= 768;
  // the line of groups is counted in 32 bits
  const bool even = !a.b.cu && !small && a.b.n_seq > 1 && groups * blocks < ((int64_t)1 << 30);
  dim3 grid;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(ROWS_T), 0, stream, a);
    return hipGetLastError();
  };
  if (!a.b.cu && !small && blocks > 768 && keys <= 256 &&
      !shares_better<T, DP, E8>(a.D, blocks, keys)) {
    grid = block_grid((blocks + NWAVE - 1) / NWAVE);
    if (a.D == DP) return go(attn_waves_kernel<T, DP, true, E8>);
    return go(attn_waves_kernel<T, DP, false, E8>);
  }
  if (even) {
    a.chunk = (int)((groups + MAX_SPLITS - 3) / (MAX_SPLITS - 2));
    grid.x = E8 && DP <= 128 ? 768 : 512;
  } else {
    const int64_t least = ones ? GROUP : 256;
    int64_t splits = small                  ? groups
                     : ones || blocks <= 64 ? (256 + blocks - 1) / blocks
                                            : 512 / blocks;
    splits = std::min({splits, (keys + least - 1) / least, (int64_t)MAX_SPLITS,
                       (int64_t)KV_PART_ROWS / (blocks * a.prow)});
    if (splits < 1 || blocks > KV_MAX_BLOCKS) splits = 1;
    a.chunk = (int)(((keys + splits - 1) / splits + GROUP - 1) / GROUP * GROUP);
    a.splits = (int)((keys + a.chunk - 1) / a.chunk);
    grid = block_grid(blocks * a.splits);
  }
  if (even) {
    if (a.D == DP) return go(attn_rows_kernel<T, DP, true, true, E8>);
    return go(attn_rows_kernel<T, DP, false, true, E8>);
  }
  if (a.D == DP) return go(attn_rows_kernel<T, DP, true, false, E8>);
  return go(attn_rows_kernel<T, DP, false, false, E8>);
}

// Tiles reach three to four times the rate of row blocks, but a step of theirs
// takes 1.2 to 1.6 us however few there are, and a tile with few rows is mostly
// empty.  Us in row blocks / in tiles (bf16, D 128, heads over key-value heads; in
// brackets the most pairs of query and key the host can tell):
//   32 over 8,  512 tokens                 18.6 / 17.5   (8.4e6)
//    4 over 4, 1000 tokens                 19.1 / 20.4   (4.0e6)
//   32 over 8,  128 tokens behind 2000     24.3 / 26.3   (8.7e6)
//   32 over 8,  256 tokens behind 2000     46.0 / 30.4   (18e6)
//    4 over 4,   64 tokens behind 32000    35.2 / 45.9   (8.2e6)
//   64 over 8,    8 tokens behind 32000    90.8 / 48.8   (16e6)
//   64 over 8,  128 tokens behind 32000     552 / 166    (263e6)
//   32 over 32,   8 tokens behind 32000    89.9 / 100.5; 17: 107.8 / 100.6
template <class T, bool E8>
hipError_t launch_attn_t(AttnArgs& a, int64_t keys, int max_tokens, hipStream_t stream) {
  if constexpr (T::V == 8) {
    const int64_t most = (int64_t)a.b.n_tokens * a.G * a.Hkv * keys;  // pairs of query and key
    if (a.b.cu && max_tokens > 1 && (int64_t)max_tokens * a.G >= 32 && most > 10000000) {
      if (a.D <= 64) return launch_tile<T, 64, E8>(a, stream);
      if (a.D <= 128) return launch_tile<T, 128, E8>(a, stream);
      return launch_tile<T, 256, E8>(a, stream);
    }
  }
  if (a.D <= 64) return launch_rows<T, 64, E8>(a, keys, max_tokens, stream);
  if (a.D <= 128) return launch_rows<T, 128, E8>(a, keys, max_tokens, stream);
  return launch_rows<T, 256, E8>(a, keys, max_tokens, stream);
}

}  // namespace

}  // namespace np
