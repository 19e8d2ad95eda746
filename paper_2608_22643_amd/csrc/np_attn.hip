// np_attn.hip -- attention over the paged key-value cache.
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
#include <algorithm>

#include "np_kv.hpp"

namespace np {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

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
  int chunk;  // keys per split, a multiple of 128
  int splits;
  float *part, *ml;
  int32_t* err;
};

// A block of RB consecutive rows (token-major, then head of the group) of one
// batch row.
struct Tile {
  KvRow row;
  int rho0, nrow;      // rows [rho0, rho0 + nrow) of the batch row's n * G
  int minpos, maxpos;  // of their tokens; maxpos < 0: they see nothing
};

// Block `tile` of the batch; false past the last one.  Every lane of the wave
// takes part and gets the same result.  err: where this workgroup reports what
// is wrong with its row, or nullptr; the one with tile 0 reports every row of a
// bad cu_tokens (a row without tokens has no block).
template <int RB>
__device__ inline bool find_tile(const KvBatch& b, int G, int tile, int32_t* err, Tile* t) {
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
        if (lo >= 0 && hi >= lo && hi <= b.n_tokens) n = (int)(((int64_t)(hi - lo) * G + RB - 1) / RB);
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
  row = __builtin_amdgcn_readfirstlane(row);
  blk = __builtin_amdgcn_readfirstlane(blk);
  const KvRow r = kv_row(b, row, threadIdx.x == 0 ? err : nullptr);
  t->row.begin = __builtin_amdgcn_readfirstlane(r.begin);  // the same in every lane
  t->row.n = __builtin_amdgcn_readfirstlane(r.n);
  t->row.p0 = __builtin_amdgcn_readfirstlane(r.p0);
  t->row.seq = __builtin_amdgcn_readfirstlane(r.seq);
  t->rho0 = blk * RB;
  t->nrow = min(RB, t->row.n * G - t->rho0);
  if (t->nrow <= 0) return false;
  t->minpos = t->row.p0 + t->rho0 / G;
  t->maxpos = t->row.p0 + (t->rho0 + t->nrow - 1) / G;
  if (t->row.p0 < 0) t->minpos = t->maxpos = -1;
  return true;
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
// Bound by the K and V bytes (decode) or, in fp32, by the matrix cores.
// ---------------------------------------------------------------------------
constexpr int RB = 16;
constexpr int NWAVE = 4;
constexpr int ROWS_T = NWAVE * WAVE;

template <class T, int DP>
struct RowsCfg {
  static constexpr int V = T::V;
  static constexpr int W = 16 / V;               // bytes of an element
  static constexpr int KS = V == 8 ? 32 : 16;    // keys of a step
  static constexpr int KT = KS / 16;             // 16-key tiles of a step
  static constexpr int KD = DP / (4 * V);        // MFMA steps over the head
  static constexpr int NV = V == 4 ? 4 : DP == 64 ? 4 : 8;  // V elements of a load
  static constexpr int VS = DP / (16 * NV);      // V loads of a row
  static constexpr int VR = KS / 4;              // V rows of a lane
  static constexpr int OP = DP + 4;              // LDS row of outputs, padded
};

template <class T, int DP>
__global__ __launch_bounds__(ROWS_T, DP == 256 ? 1 : 2) void attn_rows_kernel(AttnArgs a) {
  using C = RowsCfg<T, DP>;
  constexpr int V = C::V, W = C::W, KS = C::KS, KT = C::KT, KD = C::KD, NV = C::NV, VS = C::VS,
                VR = C::VR;
  __shared__ float s_o[NWAVE][RB][C::OP];
  __shared__ float s_m[NWAVE][RB], s_l[NWAVE][RB];

  const int lane = threadIdx.x % WAVE;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / WAVE);
  const int r = lane & 15, g = lane >> 4;
  const int id = blockIdx.x;
  const int h = id % a.Hkv, tile = id / a.Hkv % a.tiles, split = id / a.Hkv / a.tiles;
  Tile t;
  if (!find_tile<RB>(a.b, a.G, tile, split == 0 && h == 0 ? a.err : nullptr, &t))
    return;

  const int kbeg = a.window && t.maxpos >= 0 ? max(0, t.minpos - a.window + 1) : 0;
  const int kend = t.maxpos + 1;
  const int kal = kbeg / KS * KS;
  const int ns = min(a.splits, max(1, (kend - kal + a.chunk - 1) / a.chunk));
  if (split >= ns) return;
  const int k0 = kal + split * a.chunk;
  const int k1 = split + 1 < ns ? k0 + a.chunk : kend;

  // this lane's query (B operand): column r, d = 4 V s + V g
  const int rr = min(r, t.nrow - 1);
  const int tok = (t.rho0 + rr) / a.G, head = h * a.G + (t.rho0 + rr) % a.G;
  const int qpos = t.row.p0 + tok;
  uint4 qf[KD];
  {
    const char* qp = a.q + (int64_t)(t.row.begin + tok) * a.q_stride + (int64_t)head * a.D * W;
#pragma unroll
    for (int s = 0; s < KD; ++s) {
      const int d = 4 * V * s + V * g;
      qf[s] = d < a.D ? *(const uint4*)(qp + d * W) : make_uint4(0, 0, 0, 0);
    }
  }

  f32x4 o[VS][NV];
#pragma unroll
  for (int s = 0; s < VS; ++s)
#pragma unroll
    for (int j = 0; j < NV; ++j) o[s][j] = (f32x4)(0.f);
  float m = -INFINITY, l = 0.f;

  const int P1 = (1 << a.pshift) - 1;
  const size_t hb = (size_t)h << a.pshift;  // rows before head h in a page's keys
  const size_t vb = (size_t)a.Hkv << a.pshift;
  const int32_t* trow = a.table + (size_t)t.row.seq * a.M;
  const int rowb = a.D * W;

  // keys of a lane: A-operand row r of tile kt is key kk + 4 kt (16-bit) or r
  const int kk = V == 8 ? 8 * (r >> 2) + (r & 3) : r;
  const int vk = VR * g;  // first value row of the lane

  uint4 kf[KT][KD];
  uint32_t vf[VR][VS][NV * W / 4];
  int okbits = 0;  // which 16-key halves of the loaded step have a page

  // page of key `key` (uniform), or -1: beyond the keys of this block (no
  // error) or a bad table entry
  auto page_of = [&](int key) -> int {
    if (key >= kend) return -1;
    const int p = trow[key >> a.pshift];
    if (p < 0 || p >= a.N) {
      if (threadIdx.x % WAVE == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
      return -1;
    }
    return p;
  };
  const char *kptr, *vptr;
  auto locate = [&](int base) {
    const int pa = page_of(base);
    int pb = pa;
    if constexpr (KS == 32) {
      if (a.pshift == 4) pb = page_of(base + 16);
    }
    okbits = (pa >= 0 ? 1 : 0) | (pb >= 0 ? 2 : 0);
    // a missing half is read from page 0 and masked
    const int pk = max(0, V == 8 && r >= 8 ? pb : pa), pv = max(0, V == 8 && g >= 2 ? pb : pa);
    kptr = a.pool + (size_t)pk * a.page_bytes + (hb + ((base + kk) & P1)) * rowb;
    vptr = a.pool + (size_t)pv * a.page_bytes + (vb + hb + ((base + vk) & P1)) * rowb;
  };
  auto load_k = [&]() {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int s = 0; s < KD; ++s) {
        const int d = 4 * V * s + V * g;
        kf[kt][s] = d < a.D ? *(const uint4*)(kptr + 4 * kt * rowb + d * W) : make_uint4(0, 0, 0, 0);
      }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int e = 0; e < VR; ++e)
#pragma unroll
      for (int s = 0; s < VS; ++s) {
        const int d = 16 * NV * s + NV * r;
        if constexpr (NV * W == 16) {
          const uint4 x = d < a.D ? *(const uint4*)(vptr + e * rowb + d * W) : make_uint4(0, 0, 0, 0);
          vf[e][s][0] = x.x;
          vf[e][s][1] = x.y;
          vf[e][s][2] = x.z;
          vf[e][s][3] = x.w;
        } else {
          const uint2 x = d < a.D ? *(const uint2*)(vptr + e * rowb + d * W) : make_uint2(0, 0);
          vf[e][s][0] = x.x;
          vf[e][s][1] = x.y;
        }
      }
  };

  int base = k0 + wave * KS;
  if (base < k1) {
    locate(base);
    load_k();
    load_v();
  }
  for (; base < k1; base += NWAVE * KS) {
    const int ok = okbits;
    const bool full = ok == 3 && base + KS - 1 <= t.minpos &&
                      (a.window == 0 || base > t.maxpos - a.window);
    const bool more = base + NWAVE * KS < k1;
    f32x4 sc[KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      sc[kt] = (f32x4)(0.f);
#pragma unroll
      for (int s = 0; s < KD; ++s) sc[kt] = mfma_step<T>(kf[kt][s], qf[s], sc[kt]);
    }
    if (more) {
      locate(base + NWAVE * KS);
      load_k();
    }
    // scores of key base + vk + 4 kt + i
    float p[4 * KT];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * kt + i] = sc[kt][i] * a.scale;
        if (!full) {
          const int key = base + vk + 4 * kt + i;
          const bool has = (ok >> (KS == 32 && g >= 2 ? 1 : 0)) & 1;
          if (!has || key > qpos || (a.window && key <= qpos - a.window)) p[4 * kt + i] = -INFINITY;
        }
      }
    float mx = p[0];
#pragma unroll
    for (int i = 1; i < 4 * KT; ++i) mx = fmaxf(mx, p[i]);
    mx = max_groups(mx);
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx);
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int s = 0; s < VS; ++s)
#pragma unroll
        for (int j = 0; j < NV; ++j) o[s][j] *= alpha;
    }
    const float mu = m == -INFINITY ? 0.f : m;  // nothing visible yet: 2^(-inf) = 0
#pragma unroll
    for (int i = 0; i < 4 * KT; ++i) {
      p[i] = __builtin_amdgcn_exp2f(p[i] - mu);
      l += p[i];
    }
    uint4 pb;
    if constexpr (V == 8) {
      // rounded to the type of V, as the matrix cores take it; the sum l
      // keeps the unrounded values
      pb.x = pack2<T>(p[0], p[1]);
      pb.y = pack2<T>(p[2], p[3]);
      pb.z = pack2<T>(p[4], p[5]);
      pb.w = pack2<T>(p[6], p[7]);
    } else {
      pb = make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]),
                      __float_as_uint(p[3]));
    }
    if (!full) {
      // values no row of the block sees must not meet the products: memory
      // past a sequence's end may hold anything (0 * NaN)
      const bool has = (ok >> (KS == 32 && g >= 2 ? 1 : 0)) & 1;
#pragma unroll
      for (int e = 0; e < VR; ++e) {
        const int key = base + vk + e;
        if (!has || key < kbeg || key >= kend) {
#pragma unroll
          for (int s = 0; s < VS; ++s)
#pragma unroll
            for (int x = 0; x < NV * W / 4; ++x) vf[e][s][x] = 0;
        }
      }
    }
#pragma unroll
    for (int s = 0; s < VS; ++s)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        uint4 av;
        if constexpr (V == 8) {
          constexpr uint32_t LO = 0x05040100u, HI = 0x07060302u;
          const uint32_t sel = j & 1 ? HI : LO;
          av.x = __builtin_amdgcn_perm(vf[1][s][j / 2], vf[0][s][j / 2], sel);
          av.y = __builtin_amdgcn_perm(vf[3][s][j / 2], vf[2][s][j / 2], sel);
          av.z = __builtin_amdgcn_perm(vf[5][s][j / 2], vf[4][s][j / 2], sel);
          av.w = __builtin_amdgcn_perm(vf[7][s][j / 2], vf[6][s][j / 2], sel);
        } else {
          av = make_uint4(vf[0][s][j], vf[1][s][j], vf[2][s][j], vf[3][s][j]);
        }
        o[s][j] = mfma_step<T>(av, pb, o[s][j]);
      }
    if (more) load_v();
  }

  // the four waves' results meet in LDS
  l = sum_groups(l);
  if (g == 0) {
    s_m[wave][r] = m;
    s_l[wave][r] = l;
  }
#pragma unroll
  for (int s = 0; s < VS; ++s)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NV; j += 4)
        *(float4*)&s_o[wave][r][16 * NV * s + NV * (4 * g + i) + j] =
            make_float4(o[s][j][i], o[s][j + 1][i], o[s][j + 2][i], o[s][j + 3][i]);
  __syncthreads();
  const size_t slot = ((size_t)tile * a.Hkv + h) * a.splits + split;
  for (int u = threadIdx.x; u < t.nrow * (DP / 4); u += ROWS_T) {
    const int qr = u / (DP / 4), d = u % (DP / 4) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NWAVE; ++w) M = fmaxf(M, s_m[w][qr]);
    float4 sum = make_float4(0, 0, 0, 0);
    float L = 0.f;
#pragma unroll
    for (int w = 0; w < NWAVE; ++w) {
      const float mw = s_m[w][qr];
      const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - M);
      const float4 x = *(const float4*)&s_o[w][qr][d];
      L += f * s_l[w][qr];
      sum.x += f * x.x;
      sum.y += f * x.y;
      sum.z += f * x.z;
      sum.w += f * x.w;
    }
    if (ns > 1) {
      *(float4*)(a.part + (slot * RB + qr) * DP + d) = sum;
      if (d == 0) {
        a.ml[(slot * RB + qr) * 2] = M;
        a.ml[(slot * RB + qr) * 2 + 1] = L;
      }
    } else if (d < a.D) {
      const float inv = M == -INFINITY ? 0.f : 1.f / L;  // a row that sees nothing is zero
      const int rho = t.rho0 + qr;
      char* op = a.out + (int64_t)(t.row.begin + rho / a.G) * a.out_stride +
                 ((int64_t)(h * a.G + rho % a.G) * a.D + d) * W;
      const float f[4] = {M == -INFINITY ? 0.f : sum.x * inv, M == -INFINITY ? 0.f : sum.y * inv,
                          M == -INFINITY ? 0.f : sum.z * inv, M == -INFINITY ? 0.f : sum.w * inv};
      if constexpr (V == 8)
        *(uint2*)op = make_uint2(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]));
      else
        *(float4*)op = make_float4(f[0], f[1], f[2], f[3]);
    }
  }
}

// Joins the splits of a row: a workgroup per (row of a block, block and
// head), DP / 4 threads over the row, the splits dealt to its other threads.
template <class T, int DP>
__global__ __launch_bounds__(ROWS_T) void attn_join_kernel(AttnArgs a) {
  constexpr int W = 16 / T::V, KS = RowsCfg<T, DP>::KS;
  constexpr int TD = DP / 4, SUB = ROWS_T / TD;
  __shared__ float4 s_o[SUB][TD];
  __shared__ float s_l[SUB];
  const int h = blockIdx.x % a.Hkv, tile = blockIdx.x / a.Hkv, qr = blockIdx.y;
  Tile t;
  if (!find_tile<RB>(a.b, a.G, tile, nullptr, &t) || qr >= t.nrow) return;
  const int kbeg = a.window && t.maxpos >= 0 ? max(0, t.minpos - a.window + 1) : 0;
  const int kal = kbeg / KS * KS;
  const int ns = min(a.splits, max(1, (t.maxpos + 1 - kal + a.chunk - 1) / a.chunk));
  if (ns <= 1) return;  // written by the row kernel
  const size_t slot = ((size_t)tile * a.Hkv + h) * a.splits;
  const int x = threadIdx.x % TD, sub = threadIdx.x / TD;
  float M = -INFINITY;
  for (int c = 0; c < ns; ++c) M = fmaxf(M, a.ml[((slot + c) * RB + qr) * 2]);
  float4 sum = make_float4(0, 0, 0, 0);
  float L = 0.f;
  for (int c = sub; c < ns; c += SUB) {
    const float* ml = a.ml + ((slot + c) * RB + qr) * 2;
    const float f = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - M);
    const float4 v = *(const float4*)(a.part + ((slot + c) * RB + qr) * DP + x * 4);
    L += f * ml[1];
    sum.x += f * v.x;
    sum.y += f * v.y;
    sum.z += f * v.z;
    sum.w += f * v.w;
  }
  s_o[sub][x] = sum;
  if (x == 0) s_l[sub] = L;
  __syncthreads();
  if (sub || x * 4 >= a.D) return;
  for (int i = 1; i < SUB; ++i) {
    const float4 v = s_o[i][x];
    sum.x += v.x;
    sum.y += v.y;
    sum.z += v.z;
    sum.w += v.w;
    L += s_l[i];
  }
  const bool none = M == -INFINITY;
  const float inv = 1.f / L;
  const float f[4] = {none ? 0.f : sum.x * inv, none ? 0.f : sum.y * inv,
                      none ? 0.f : sum.z * inv, none ? 0.f : sum.w * inv};
  const int rho = t.rho0 + qr;
  char* op = a.out + (int64_t)(t.row.begin + rho / a.G) * a.out_stride +
             ((int64_t)(h * a.G + rho % a.G) * a.D + x * 4) * W;
  if constexpr (T::V == 8)
    *(uint2*)op = make_uint2(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]));
  else
    *(float4*)op = make_float4(f[0], f[1], f[2], f[3]);
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

template <int DP>
struct TileCfg {
  static constexpr int KB = DP == 256 ? 32 : 64;    // keys of a step
  static constexpr int CPR = DP / 8;                // 16-byte pieces of a row
  static constexpr int NL = KB * CPR / TILE_T;      // pieces a thread loads
  static constexpr int RSTEP = TILE_T / CPR;        // rows between them
  // piece permutations of K and V rows
  __device__ static inline int kperm(int row, int c) {
    return c ^ (DP == 64 ? row >> 1 & 7 : row & 15);
  }
  __device__ static inline int vperm(int row, int c) {
    return c ^ (DP == 64 ? (row >> 1 & 1) << 2 | (row >> 2 & 3) : (row & 3) << 2 | (row >> 2 & 3));
  }
};

// FULL: D == DP; otherwise the pieces past D stay zero in LDS.
template <class T, int DP, bool FULL>
__global__ __launch_bounds__(TILE_T, DP == 256 ? 1 : 2) void attn_tile_kernel(AttnArgs a) {
  using C = TileCfg<DP>;
  constexpr int KB = C::KB, CPR = C::CPR, NL = C::NL, RSTEP = C::RSTEP;
  constexpr int KT = KB / 32, KD = DP / 16, DT = DP / 32;
  __shared__ u32x4_t s_k[2][KB * CPR];
  __shared__ u32x4_t s_v[2][KB * CPR];

  const int tid = threadIdx.x, lane = tid % WAVE;
  const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int r = lane & 31, h2 = lane >> 5;
  const int h = blockIdx.x % a.Hkv;
  const int tile = a.tiles - 1 - (int)blockIdx.x / a.Hkv;  // the longest of a prompt first
  Tile t;
  if (!find_tile<TB>(a.b, a.G, tile, h == 0 ? a.err : nullptr, &t)) return;

  const int kbeg = a.window && t.maxpos >= 0 ? max(0, t.minpos - a.window + 1) : 0;
  const int kend = t.maxpos + 1;
  const int rowb = a.D * 2;

  // this wave's rows and this lane's query
  const int w0 = min(wave * 32, t.nrow - 1), w1 = min(wave * 32 + 31, t.nrow - 1);
  const int wmin = t.row.p0 < 0 ? -1 : t.row.p0 + (t.rho0 + w0) / a.G;
  const int wmax = t.row.p0 < 0 ? -1 : t.row.p0 + (t.rho0 + w1) / a.G;
  const int rho = t.rho0 + min(wave * 32 + r, t.nrow - 1);
  const int tok = rho / a.G, head = h * a.G + rho % a.G;
  const int qpos = t.row.p0 < 0 ? -1 : t.row.p0 + tok;
  const char* qp = a.q + (int64_t)(t.row.begin + tok) * a.q_stride + (int64_t)head * rowb;
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

  f32x16 o[DT];
#pragma unroll
  for (int j = 0; j < DT; ++j) o[j] = (f32x16)(0.f);
  float m = -INFINITY, l = 0.f;

  // loads: piece lc of rows lr, lr + RSTEP, ...  Rows outside the tile's keys
  // repeat its first or last one: they get no weight, but have to be finite.
  const int lc = tid % CPR, lr = tid / CPR;
  const bool lon = FULL || lc * 8 < a.D;
  const int P1 = (1 << a.pshift) - 1;
  const size_t hrow = (size_t)h << a.pshift;
  const size_t vofs = ((size_t)a.Hkv << a.pshift) * rowb;
  const char* hpool = a.pool + hrow * rowb + lc * 16;
  const int32_t* trow = a.table + (size_t)t.row.seq * a.M;
  // a table that names no page somewhere in the tile's keys: those keys are
  // looked up again and masked one by one
  int any_bad = 0;
  for (int j = (kbeg >> a.pshift) + tid; j <= (kend - 1) >> a.pshift; j += TILE_T)
    any_bad |= trow[j] < 0 || trow[j] >= a.N;
  const bool bad = __builtin_amdgcn_readfirstlane(__syncthreads_or(any_bad)) != 0;
  if (bad && tid == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
  u32x4_t sk[NL] = {}, sv[NL] = {};
  auto key_of = [&](int base, int i) { return max(kbeg, min(base + lr + i * RSTEP, kend - 1)); };
  int page[NL];
  auto load_pages = [&](int base) {
#pragma unroll
    for (int i = 0; i < NL; ++i) page[i] = trow[key_of(base, i) >> a.pshift];
  };
  auto load_rows = [&](int base) {
    const char* p[NL];
    int64_t vo[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      p[i] = hpool + (int64_t)page[i] * (int64_t)a.page_bytes + (key_of(base, i) & P1) * rowb;
      vo[i] = vofs;
    }
    if (bad)
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (page[i] < 0 || page[i] >= a.N) {  // masked below: any finite row will do
          p[i] = a.q + (int64_t)t.row.begin * a.q_stride + lc * 16;
          vo[i] = 0;
        }
    if (lon) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        sk[i] = load_global16(p[i]);
        sv[i] = load_global16(p[i] + vo[i]);
      }
    }
  };
  auto store_rows = [&](int buf) {
    if (lon) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = lr + i * RSTEP;
        s_k[buf][row * CPR + C::kperm(row, lc)] = sk[i];
        s_v[buf][row * CPR + C::vperm(row, lc)] = sv[i];
      }
    }
  };
  if constexpr (!FULL) {
    if (!lon)
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = lr + i * RSTEP;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          s_k[x][row * CPR + C::kperm(row, lc)] = (u32x4_t)(0u);
          s_v[x][row * CPR + C::vperm(row, lc)] = (u32x4_t)(0u);
        }
      }
  }

  const int k0 = kbeg / KB * KB;
  if (kend > 0) load_pages(k0);
  if (kend > 0) {
    load_rows(k0);
    load_pages(k0 + KB);
    store_rows(0);
  }
  __syncthreads();
  int buf = 0;
  for (int base = k0; base < kend; base += KB, buf ^= 1) {
    const bool more = base + KB < kend;
    if (more) {
      load_rows(base + KB);
      load_pages(base + 2 * KB);
    }
    if (base <= wmax && (a.window == 0 || base + KB - 1 > wmin - a.window)) {
      const bool full = !bad && base + KB - 1 <= wmin && (a.window == 0 || base > wmax - a.window);
      f32x16 sc[KT];
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        sc[kt] = (f32x16)(0.f);
        const int row = 32 * kt + r;
#pragma unroll
        for (int s = 0; s < KD; ++s)
          sc[kt] = mfma32<T>(as_uint4(s_k[buf][row * CPR + C::kperm(row, 2 * s + h2)]), qf[s], sc[kt]);
      }
      if (!full) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = base + 32 * kt + 8 * (i / 4) + 4 * h2 + i % 4;
            if (key > qpos || (a.window && key <= qpos - a.window)) sc[kt][i] = -INFINITY;
          }
        if (bad)
          for (int kt = 0; kt < KT; ++kt)
            for (int i = 0; i < 16; ++i) {
              const int key = base + 32 * kt + 8 * (i / 4) + 4 * h2 + i % 4;
              const int p = trow[min(key, kend - 1) >> a.pshift];
              if (p < 0 || p >= a.N) sc[kt][i] = -INFINITY;
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
      if (__any(mx > m)) {
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
      const int vr = 4 * h2 + (lane >> 2 & 3), vc = 16 * (lane >> 4 & 1) + 4 * (lane & 3);
#pragma unroll
      for (int mm = 0; mm < 2 * KT; ++mm)
#pragma unroll
        for (int j = 0; j < DT; ++j) {
          const int ra = 16 * mm + vr, rb = ra + 8, d = 32 * j + vc;
          typedef __attribute__((address_space(3))) s16x4 lds4;
          const char* vb = (const char*)s_v[buf];
          const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4*)(vb + (ra * CPR + C::vperm(ra, d / 8)) * 16 + (d & 4) * 2));
          const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds4*)(vb + (rb * CPR + C::vperm(rb, d / 8)) * 16 + (d & 4) * 2));
          const uint2 xu = __builtin_bit_cast(uint2, x), yu = __builtin_bit_cast(uint2, y);
          o[j] = mfma32<T>(make_uint4(xu.x, xu.y, yu.x, yu.y), pf[mm], o[j]);
        }
    }
    if (more) store_rows(buf ^ 1);
    __syncthreads();
  }

  l = swap32_add(l, l);
  if (wave * 32 + r >= t.nrow) return;
  const bool none = m == -INFINITY;  // a row that sees nothing is zero
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

template <class T, int DP>
hipError_t launch_tile(AttnArgs a, hipStream_t stream) {
  a.tiles = a.b.cu ? (int)((int64_t)a.b.n_tokens * a.G / TB) + a.b.n_seq
                   : a.b.n_seq * ((a.G + TB - 1) / TB);
  const dim3 grid((unsigned)((int64_t)a.tiles * a.Hkv));
  if (a.D == DP)
    hipLaunchKernelGGL((attn_tile_kernel<T, DP, true>), grid, dim3(TILE_T), 0, stream, a);
  else
    hipLaunchKernelGGL((attn_tile_kernel<T, DP, false>), grid, dim3(TILE_T), 0, stream, a);
  return hipGetLastError();
}

template <class T, int DP>
hipError_t launch_rows(AttnArgs a, int64_t keys, hipStream_t stream) {
  // enough workgroups to fill the card, at least 128 keys (one step of each
  // wave) in each
  const int64_t blocks = (int64_t)a.tiles * a.Hkv;
  int64_t splits = std::min<int64_t>((1024 + blocks - 1) / blocks, KV_SLOTS / std::max<int64_t>(blocks, 1));
  splits = std::max<int64_t>(1, std::min(splits, (keys + 127) / 128));
  a.chunk = (int)(((keys + splits - 1) / splits + 127) / 128 * 128);
  a.splits = (int)((keys + a.chunk - 1) / a.chunk);
  if (a.splits < 1) a.splits = 1;
  hipLaunchKernelGGL((attn_rows_kernel<T, DP>), dim3((unsigned)(blocks * a.splits)), dim3(ROWS_T), 0,
                     stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const unsigned rows = a.b.cu ? RB : std::min(a.G, RB);
  hipLaunchKernelGGL((attn_join_kernel<T, DP>), dim3((unsigned)blocks, rows), dim3(ROWS_T), 0, stream,
                     a);
  return hipGetLastError();
}

template <class T>
hipError_t launch_attn_t(AttnArgs& a, int64_t keys, int max_tokens, hipStream_t stream) {
  if constexpr (T::V == 8) {
    if (a.b.cu && (int64_t)max_tokens * a.G > 64) {
      if (a.D <= 64) return launch_tile<T, 64>(a, stream);
      if (a.D <= 128) return launch_tile<T, 128>(a, stream);
      return launch_tile<T, 256>(a, stream);
    }
  }
  if (a.D <= 64) return launch_rows<T, 64>(a, keys, stream);
  if (a.D <= 128) return launch_rows<T, 128>(a, keys, stream);
  return launch_rows<T, 256>(a, keys, stream);
}

}  // namespace

hipError_t launch_attn(const np_kv_shape& s, int layer, const np_kv_batch& b,
                       const int32_t* table, const void* q, int64_t q_stride, const void* pool,
                       float scale, int window, void* out, int64_t out_stride, void* ws,
                       hipStream_t stream) {
  const int64_t w = dtype_size(s.dtype);
  AttnArgs a;
  KvScratch k;
  kv_ws_layout(s, (char*)ws, &k);
  a.b = {b.seqs, b.cu_tokens, b.pos0, b.n_seq, b.n_tokens, s.max_seqs,
         (int)std::min<int64_t>(b.max_len, (int64_t)s.seq_pages * s.page_size)};
  a.table = table;
  a.q = (const char*)q;
  a.out = (char*)out;
  a.q_stride = q_stride * w;
  a.out_stride = out_stride * w;
  a.page_bytes = kv_page_bytes(s);
  a.pool = (const char*)pool + (size_t)layer * s.n_pages * a.page_bytes;
  a.Hkv = s.kv_heads;
  a.G = s.heads / s.kv_heads;
  a.D = s.head_dim;
  a.M = s.seq_pages;
  a.N = s.n_pages;
  a.pshift = __builtin_ctz((unsigned)s.page_size);
  a.scale = scale * LOG2E;
  a.window = window;
  a.part = k.part;
  a.ml = k.ml;
  a.err = (int32_t*)((char*)ws + WS_ERR);
  // row blocks: at most one partly filled per row of the batch
  a.tiles = b.cu_tokens ? (int)((int64_t)b.n_tokens * a.G / RB) + b.n_seq
                        : b.n_seq * ((a.G + RB - 1) / RB);
  // keys a block can see
  int64_t keys = a.b.lim;
  if (window > 0) keys = std::min<int64_t>(keys, (int64_t)window + RB + 32);
  keys = std::max<int64_t>(keys, 1);
  if (s.dtype == NP_F32) return launch_attn_t<TF32>(a, keys, b.max_tokens, stream);
  if (s.dtype == NP_F16) return launch_attn_t<TF16>(a, keys, b.max_tokens, stream);
  return launch_attn_t<TBF16>(a, keys, b.max_tokens, stream);
}

}  // namespace np
