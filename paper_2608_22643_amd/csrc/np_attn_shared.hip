// np_attn_shared.hip -- np_attn_decode_shared: decode of sequences that share
// prefixes.
//
// The softmax over a row's keys is joined from any parts of them: with (m_i,
// l_i, o_i) the maximum, sum and weighted values of part i,
//     out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i,   M = max_i m_i.
// So a group's prefix is one part of all its rows, and the query heads of those
// rows are rows of one tile against it: a key or value is read once for up to
// 128 of them.  Each row's own keys are row blocks as in np_attn_decode.
//
// One kernel computes the parts, a second joins them.  The parts' keys lie on
// a line (the tiles' first), weighed by what they cost, and every workgroup
// has an equal stretch of it, whatever the lengths, which only the device
// knows.  A block (a tile or a row block, of one key-value head) that the cuts
// leave in several workgroups has its first part's results in rows of its own
// (one for every query head of the batch, for prefix and own keys each), and
// every further one in the rows of the workgroup whose stretch it begins.
#include "np_attn.hpp"

namespace np {

namespace {

struct SharedArgs {
  AttnArgs a;
  const int32_t *lead, *prefix;
  int max_prefix;
  int Hq, n;
  int least;  // weight of a stretch at least
  int32_t *info_p, *info_s, *row_lead;
};

constexpr int SH_WG = 512;     // workgroups at most
constexpr int FAR = 1 << 30;    // past all positions
constexpr int OWN_WEIGHT = 4;  // of 128 keys of a row: the line counts 32 keys
static_assert(2 * KV_SHARED_HEADS + SH_WG * TB <= KV_PART_ROWS, "rows of all parts fit");

// What a block of shared keys is for type T: 128 rows against steps through LDS,
// or 16 rows against 128 keys in registers (fp32).
template <class T, int DP, bool E8>
struct SharedCfg {
  static constexpr bool TILE = T::V == 8;
  static constexpr int ROWS = TILE ? TB : RB;
  static constexpr int KEYS = TILE ? TileCfg<DP, E8>::KB : GROUP;
  static constexpr int WEIGHT = KEYS / 32;
};

__device__ inline int div_up_pos(int a, int b) { return a > 0 ? (a + b - 1) / b : 0; }

// A row of the batch (cu_tokens NULL) as every lane may ask for it.
__device__ inline KvRow lane_row(const KvBatch& b, int i, int32_t* err) {
  return kv_row_check(b, {i, i + 1, b.seqs ? b.seqs[i] : i, b.pos0[i]}, err);
}

// Rows i0 .. i0 + 63, one a lane.
struct SharedRow {
  KvRow row;
  int lead;    // the first row of its group, or -1: by itself
  int prefix;  // positions it has in common with it
  int seq;     // the lead's sequence
  int run;     // the first of the neighbouring rows that name the same lead
};
__device__ inline SharedRow shared_row(const SharedArgs& x, int i0, int run_before, int32_t* err) {
  const int lane = threadIdx.x % WAVE, n = x.n;
  const int i = min(i0 + lane, n - 1);
  SharedRow s;
  const int L = x.lead[i], before = x.lead[max(i - 1, 0)], after = x.lead[min(i + 1, n - 1)];
  s.row = lane_row(x.a.b, i, err);
  const uint64_t cuts = __ballot(i == 0 || before != L) & (~0ull >> (WAVE - 1 - lane));
  s.run = cuts ? i0 + 63 - __clzll((long long)cuts) : run_before;
  bool ok = L >= 0 && L <= i && s.run <= L;
  const int at = ok ? L : 0;
  s.prefix = x.prefix[at];
  s.seq = x.a.b.seqs ? x.a.b.seqs[at] : at;
  ok = ok && s.prefix >= 0 && s.prefix <= x.max_prefix && s.seq >= 0 && s.seq < x.a.b.S;
  if (!ok && err && i0 + lane < n) atomicOr(err, NP_DEVERR_STATE);
  const bool alone = L == i && (i + 1 >= n || after != L);
  s.lead = ok && !alone && s.prefix > 0 ? L : -1;
  if (s.lead < 0) s.prefix = s.seq = 0;
  return s;
}

// Keys of a row beside its group's: the first, and groups of 128 of them (a row
// that sees nothing has one, for its zeros).
template <int KS>
__device__ inline int own_first(int p0, int prefix, int window) {
  return max(min(prefix, p0 + 1), window && p0 >= 0 ? max(0, p0 - window + 1) : 0);
}
template <int KS>
__device__ inline int own_groups(int p0, int prefix, int window) {
  const int first = own_first<KS>(p0, prefix, window) / KS * KS;
  return max(1, div_up_pos(p0 + 1 - first, GROUP));
}

// The thread's number, anew for each part: what the parts derive from it would
// otherwise be kept for all of them at once, past the registers there are.
__device__ inline int own_tid() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

__device__ inline int lane_max(int v) { return (int)wave_max((uint32_t)(v + 1)) - 1; }  // v >= -1

template <class T, int DP, bool FULL, bool E8>
__global__ __launch_bounds__(ROWS_T, DP == 256 ? 1 : 2) void attn_shared_kernel(SharedArgs x) {
  using P = SharedCfg<T, DP, E8>;
  using C = RowsCfg<T, DP, E8>;
  using TC = TileCfg<DP, E8>;
  constexpr int W = C::W, KS = C::KS;
  struct RowsLds {
    float o[NWAVE][RB][C::OP];
    float m[NWAVE][RB], l[NWAVE][RB];
  };
  constexpr int TILE_LDS = P::TILE ? 4 * TC::KB * TC::ROW : 0;
  constexpr int LDS = TILE_LDS > (int)sizeof(RowsLds) ? TILE_LDS : (int)sizeof(RowsLds);
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  // of the rows i0 .. i0 + 63 (each wave finds the same): what would stand in the
  // way of the tiles' registers
  __shared__ struct {
    int steps[WAVE], up_at[WAVE], lead[WAVE], prefix[WAVE], lead_seq[WAVE];
    int us[WAVE], us_at[WAVE], p0[WAVE], seq[WAVE];
  } rows;
  RowsLds& rl = *(RowsLds*)lds;

  const AttnArgs& a = x.a;
  const int lane = threadIdx.x % WAVE;
  const int wave = uniform((int)threadIdx.x / WAVE);
  const int n = x.n, RT = P::ROWS / a.G;       // rows of the batch in a tile
  const int per = (a.G + RB - 1) / RB, nb = per * a.Hkv;
  int32_t* const err = blockIdx.x == 0 && threadIdx.x < WAVE ? a.err : nullptr;

  // A lane's row, its units on the line (up: steps of its tile, all heads; us:
  // groups of its own keys), and theirs up to it.
  SharedRow sr;
  int steps, up, us, up_at, us_at;
  auto load = [&](int first, int run_before, int32_t* e) {
    sr = shared_row(x, first, run_before, e);
    const bool here = first + lane < n;
    steps = sr.lead >= 0 && here && (first + lane - sr.lead) % RT == 0
                ? div_up_pos(sr.prefix, P::KEYS)
                : 0;
    up = steps * a.Hkv;
    us = here ? own_groups<KS>(sr.row.p0, sr.prefix, a.window) * nb : 0;
    up_at = (int)wave_incl_scan((uint32_t)up);
    us_at = (int)wave_incl_scan((uint32_t)us);
  };
  auto last = [&](int v) { return __builtin_amdgcn_readlane(v, WAVE - 1); };
  int tp = 0, ts = 0, run = 0;
  for (int i = 0; i < n; i += WAVE) {
    load(i, run, err);
    run = last(sr.run);
    tp += last(up_at);
    ts += last(us_at);
    if (err && i + lane < n) x.row_lead[i + lane] = sr.lead;
  }
  tp = uniform(tp);
  ts = uniform(ts);
  const int total = tp * P::WEIGHT + ts * OWN_WEIGHT;
  const int share = max(x.least, (total + (int)gridDim.x - 1) / (int)gridDim.x);
  // workgroups go round the eight XCDs; each XCD gets one stretch in a piece
  const int wg = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  if ((int64_t)wg * share >= total) return;
  const int beg = wg * share, end = min(total, beg + share);
  const int s0 = min(tp, div_up_pos(beg, P::WEIGHT)), s1 = min(tp, div_up_pos(end, P::WEIGHT));
  const int g0 = div_up_pos(beg - tp * P::WEIGHT, OWN_WEIGHT);
  const int g1 = min(ts, div_up_pos(end - tp * P::WEIGHT, OWN_WEIGHT));

  // where the row of query head hq of batch row b goes, for the first part of
  // its block and for a further one
  auto part_of = [&](bool first, int base, int b, int hq, int local) {
    return first ? base + b * x.Hq + hq : 2 * n * x.Hq + wg * P::ROWS + local;
  };
  auto put = [&](int row, int d, float4 v) { *(float4*)(a.part + (size_t)row * DP + d) = v; };

  // steps [c0, c1) of a tile's: rows b0 .. of group L against its prefix
  auto shared_part = [&](int b0, int L, int p, int seq, int h, int c0, int c1, bool first) {
    const int tid = own_tid(), lane = tid % WAVE;
    // its rows, and the positions they span
    int cnt = 0;
    for (int i = 0; i < RT && cnt == i; i += WAVE) {
      const int b = b0 + i + lane;
      const uint64_t out = ~__ballot(i + lane < RT && b < n && x.lead[min(b, n - 1)] == L);
      cnt = i + (out ? __ffsll((unsigned long long)out) - 1 : WAVE);
    }
    int tmax = -1, tmin = FAR;
    for (int i = 0; i < cnt; i += WAVE) {
      const int p0 = i + lane < cnt ? lane_row(a.b, b0 + i + lane, nullptr).p0 : -1;
      tmax = max(tmax, p0);
      if (p0 >= 0) tmin = min(tmin, p0);
    }
    tmax = uniform(lane_max(tmax));
    tmin = uniform(tmax < 0 ? 0 : FAR - lane_max(FAR - tmin));
    cnt = uniform(cnt);
    const int kbeg0 = a.window && tmax >= 0 ? max(0, tmin - a.window + 1) : 0;
    const int kend0 = min(p, tmax + 1);
    int kbeg = max(kbeg0, c0 * P::KEYS), kend = min(kend0, c1 * P::KEYS);
    const int32_t* trow = a.table + (int64_t)seq * a.M;
    // this lane's query
    const int r = P::TILE ? wave * 32 + (lane & 31) : lane & 15;
    const int rho = min(r, cnt * a.G - 1), b = b0 + rho / a.G, hq = h * a.G + rho % a.G;
    const int p0 = lane_row(a.b, b, nullptr).p0;
    const int qpos = p0 < 0 ? tmax : p0;  // of a row that is not served: nothing is made of it
    const char* qp = a.q + (int64_t)b * a.q_stride + (int64_t)hq * a.D * W;
    bool missing = false;
    if constexpr (P::TILE) {
      if (kbeg >= kend) kbeg = kend = 0;
      f32x16 o[TC::DT];
      float m, l;
      // a wave without rows has nothing to compute, but its share of the loads
      tile_keys<T, DP, FULL, E8, true>(tid, a, trow, h, kbeg, kend, tmin,
                                       wave * 32 < cnt * a.G ? tmax : -1, qp, qpos, lds,
                                       lds + TILE_LDS / 2, o, m, l, missing);
      l = swap32_add(l, l);
      if (r < cnt * a.G) {
        const int h2 = lane >> 5;
        const int row = part_of(first, 0, b, hq, r);
#pragma unroll
        for (int j = 0; j < TC::DT; ++j)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            put(row, 32 * j + 2 * i + 4 * h2,
                make_float4(o[j][i], o[j][i + 1], o[j][i + 2], o[j][i + 3]));
        if (h2 == 0) *(float2*)(a.ml + (size_t)row * 2) = make_float2(m, l);
      }
    } else {
      const int kal = kbeg / KS * KS;
      if (kbeg >= kend) kbeg = kend = 0;
      f32x4 o[C::VS][C::NV];
      float m, l;
      rows_keys<T, DP, FULL, E8, true>(tid, a, trow, h, tmin, tmax, kbeg, kend, kend ? kal : 0, kend, qp, qpos,
                                 o, m, l, missing);
      rows_meet<C>(o, m, l, rl.o, rl.m, rl.l);
      __syncthreads();
      for (int u = threadIdx.x; u < cnt * a.G * (DP / 4); u += ROWS_T) {
        const int q = u / (DP / 4), d = u % (DP / 4) * 4;
        float M, L2;
        const float4 sum = rows_met<C>(rl.o, rl.m, rl.l, q, d, M, L2);
        const int row = part_of(first, 0, b0 + q / a.G, h * a.G + q % a.G, q);
        put(row, d, sum);
        if (d == 0) *(float2*)(a.ml + (size_t)row * 2) = make_float2(M, L2);
      }
      __syncthreads();  // LDS is free again
    }
    if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
  };

  // groups [c0, c1) of block j of a row's own keys
  auto own_part = [&](int b, int p0, int seq, int prefix, int j, int c0, int c1, bool first) {
    const int tid = own_tid(), lane = tid % WAVE;
    const int h = j % a.Hkv, q0 = j / a.Hkv * RB, rows = min(RB, a.G - q0);
    const int kbeg = own_first<KS>(p0, prefix, a.window), kend = p0 + 1;
    const int k0 = kbeg / KS * KS + c0 * GROUP;
    const int k1 = kbeg < kend ? min(kend, kbeg / KS * KS + c1 * GROUP) : k0;  // none: no step
    const int hq = h * a.G + q0 + min(lane & 15, rows - 1);
    f32x4 o[C::VS][C::NV];
    float m, l;
    bool missing;
    rows_keys<T, DP, FULL, E8, true>(tid, a, a.table + (int64_t)seq * a.M, h, p0, p0, kbeg, kend, k0, k1,
                               a.q + (int64_t)b * a.q_stride + (int64_t)hq * a.D * W, p0, o, m, l,
                               missing);
    if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
    rows_meet<C>(o, m, l, rl.o, rl.m, rl.l);
    __syncthreads();
    for (int u = threadIdx.x; u < rows * (DP / 4); u += ROWS_T) {
      const int q = u / (DP / 4), d = u % (DP / 4) * 4;
      float M, L;
      const float4 sum = rows_met<C>(rl.o, rl.m, rl.l, q, d, M, L);
      const int row = part_of(first, n * x.Hq, b, h * a.G + q0 + q, q);
      put(row, d, sum);
      if (d == 0) *(float2*)(a.ml + (size_t)row * 2) = make_float2(M, L);
    }
    __syncthreads();  // LDS is free again
  };

  int pb = 0, sb = 0;  // units of the chunks before
  run = 0;
  for (int i0 = 0; i0 < n && (pb < s1 || sb < g1); i0 += WAVE) {
    if (n > WAVE) {
      load(i0, run, nullptr);
      run = last(sr.run);
      __syncthreads();
    }
    if (wave == 0) {
      rows.steps[lane] = steps;
      rows.up_at[lane] = pb + up_at - up;
      rows.lead[lane] = sr.lead;
      rows.prefix[lane] = sr.prefix;
      rows.lead_seq[lane] = sr.seq;
      rows.us[lane] = us;
      rows.us_at[lane] = sb + us_at - us;
      rows.p0[lane] = sr.row.p0;
      rows.seq[lane] = sr.row.seq;
    }
    uint64_t tiles = __ballot(up > 0 && pb + up_at > s0 && pb + up_at - up < s1);
    uint64_t own = __ballot(us > 0 && sb + us_at > g0 && sb + us_at - us < g1);
    pb += last(up_at);
    sb += last(us_at);
    __syncthreads();
    while (tiles) {
      const int l = __ffsll((unsigned long long)tiles) - 1;
      tiles &= tiles - 1;
      const int st = uniform(rows.steps[l]), at = uniform(rows.up_at[l]);
      for (int h = max(0, s0 - at) / st; h < a.Hkv; ++h) {
        const int x0 = at + h * st, c0 = max(s0, x0), c1 = min(s1, x0 + st);
        if (c0 >= c1) break;
        if (c0 == x0 && threadIdx.x == 0)
          x.info_p[(i0 + l) * a.Hkv + h] = wg | (x0 + st - 1) * P::WEIGHT / share << 16;
        shared_part(i0 + l, uniform(rows.lead[l]), uniform(rows.prefix[l]),
                    uniform(rows.lead_seq[l]), h, c0 - x0, c1 - x0, c0 == x0);
      }
    }
    while (own) {
      const int l = __ffsll((unsigned long long)own) - 1;
      own &= own - 1;
      const int gr = uniform(rows.us[l]) / nb, at = uniform(rows.us_at[l]);
      for (int j = max(0, g0 - at) / gr; j < nb; ++j) {
        const int x0 = at + j * gr, c0 = max(g0, x0), c1 = min(g1, x0 + gr);
        if (c0 >= c1) break;
        if (c0 == x0 && threadIdx.x == 0)
          x.info_s[(i0 + l) * nb + j] =
              wg | (tp * P::WEIGHT + (x0 + gr - 1) * OWN_WEIGHT) / share << 16;
        own_part(i0 + l, uniform(rows.p0[l]), uniform(rows.seq[l]), uniform(rows.prefix[l]), j,
                 c0 - x0, c1 - x0, c0 == x0);
      }
    }
  }
}

// A wave per query head: its parts joined, in their order.
template <class T, int DP, int ROWS>
__global__ __launch_bounds__(ROWS_T) void attn_shared_join_kernel(SharedArgs x) {
  constexpr int TD = DP / 4, SUB = WAVE / TD, W = 16 / T::V;
  const AttnArgs& a = x.a;
  const int lane = threadIdx.x % WAVE;
  const int id = uniform((int)(blockIdx.x * (ROWS_T / WAVE) + threadIdx.x / WAVE));
  if (id >= x.n * x.Hq) return;
  const int b = id / x.Hq, hq = id % x.Hq, h = hq / a.G, g = hq % a.G;
  const int per = (a.G + RB - 1) / RB, nb = per * a.Hkv, RT = ROWS / a.G;
  const int L = load_scalar(x.row_lead, b);
  const int is = load_scalar(x.info_s, b * nb + g / RB * a.Hkv + h);
  const int b0 = L < 0 ? b : L + (b - L) / RT * RT;
  const int ip = L < 0 ? 0 : load_scalar(x.info_p, b0 * a.Hkv + h);
  const KvRow row = kv_row(a.b, b, nullptr);
  const int np = L < 0 ? 0 : (ip >> 16) - (ip & 0xFFFF) + 1;
  const int ns = (is >> 16) - (is & 0xFFFF) + 1;
  const int extra = 2 * x.n * x.Hq;
  auto part_row = [&](int c) {
    if (c < np) return c ? extra + ((ip & 0xFFFF) + c) * ROWS + (b - b0) * a.G + g : id;
    c -= np;
    return c ? extra + ((is & 0xFFFF) + c) * ROWS + g % RB : x.n * x.Hq + id;
  };
  const int parts = np + ns;
  float M = -INFINITY;
  for (int c = lane; c < parts; c += WAVE) M = fmaxf(M, a.ml[(size_t)part_row(c) * 2]);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, WAVE));
  const int sub = lane / TD, d = lane % TD * 4;
  float l = 0.f;
  float4 sum = make_float4(0, 0, 0, 0);
  constexpr int NB = 8;
  for (int c0 = sub; c0 < parts; c0 += NB * SUB) {
    float4 v[NB];
    float2 ml[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int r = part_row(min(c0 + i * SUB, parts - 1));
      v[i] = *(const float4*)(a.part + (size_t)r * DP + d);
      ml[i] = *(const float2*)(a.ml + (size_t)r * 2);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      // without a maximum the sum is 0, or NaN when every score was
      float f = ml[i].x == -INFINITY ? ml[i].y : __builtin_amdgcn_exp2f(ml[i].x - M);
      if (c0 + i * SUB >= parts) continue;
      l += f * ml[i].y;
      sum.x += f * v[i].x;
      sum.y += f * v[i].y;
      sum.z += f * v[i].z;
      sum.w += f * v[i].w;
    }
  }
#pragma unroll
  for (int off = TD; off < WAVE; off *= 2) {
    l += __shfl_xor(l, off, WAVE);
    sum.x += __shfl_xor(sum.x, off, WAVE);
    sum.y += __shfl_xor(sum.y, off, WAVE);
    sum.z += __shfl_xor(sum.z, off, WAVE);
    sum.w += __shfl_xor(sum.w, off, WAVE);
  }
  if (sub || d >= a.D) return;
  const float inv = 1.f / l;
  const bool none = l == 0.f || row.p0 < 0;  // a row that sees nothing is zero
  const float f[4] = {none ? 0.f : sum.x * inv, none ? 0.f : sum.y * inv, none ? 0.f : sum.z * inv,
                      none ? 0.f : sum.w * inv};
  char* op = a.out + (int64_t)b * a.out_stride + ((int64_t)hq * a.D + d) * W;
  if constexpr (T::V == 8)
    *(uint2*)op = make_uint2(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3]));
  else
    *(float4*)op = make_float4(f[0], f[1], f[2], f[3]);
}

template <class T, int DP, bool E8>
hipError_t launch_shared(const SharedArgs& x, hipStream_t stream) {
  using P = SharedCfg<T, DP, E8>;
  const dim3 grid(DP == 256 ? SH_WG / 2 : SH_WG), block(ROWS_T);
  if (x.a.D == DP)
    hipLaunchKernelGGL((attn_shared_kernel<T, DP, true, E8>), grid, block, 0, stream, x);
  else
    hipLaunchKernelGGL((attn_shared_kernel<T, DP, false, E8>), grid, block, 0, stream, x);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned waves = (unsigned)(x.n * x.Hq);
  hipLaunchKernelGGL((attn_shared_join_kernel<T, DP, P::ROWS>),
                     dim3((waves + ROWS_T / WAVE - 1) / (ROWS_T / WAVE)), block, 0, stream, x);
  return hipGetLastError();
}

template <class T, bool E8>
hipError_t launch_shared_t(const SharedArgs& x, hipStream_t stream) {
  if (x.a.D <= 64) return launch_shared<T, 64, E8>(x, stream);
  if (x.a.D <= 128) return launch_shared<T, 128, E8>(x, stream);
  return launch_shared<T, 256, E8>(x, stream);
}

}  // namespace

hipError_t launch_attn_shared(const np_kv_shape& s, int layer, const np_kv_batch& b,
                              const np_kv_shared& sh, const int32_t* table, const void* q,
                              int64_t q_stride, const void* pool, float scale, int window,
                              void* out, int64_t out_stride, void* ws, hipStream_t stream) {
  const int dtype = kv_dtype(s), G = s.heads / s.kv_heads;
  const int64_t n = b.n_seq, heads = n * s.heads;
  SharedArgs x;
  x.a = attn_args(s, layer, b, table, q, q_stride, pool, scale, window, out, out_stride, ws);
  // the line's length: at most a tile a row, and every row's own keys
  const int64_t line = n * s.kv_heads * ((int64_t)sh.max_prefix / 32 + 8) +
                       heads * ((int64_t)x.a.b.lim / 32 + 8);
  if (sh.max_prefix == 0 || n < 2 || heads > KV_SHARED_HEADS || G > (dtype == NP_F32 ? RB : TB) ||
      line >= ((int64_t)1 << 30))
    return launch_attn(s, layer, b, table, q, q_stride, pool, scale, window, out, out_stride, ws,
                       stream);
  KvScratch k;
  kv_ws_layout(s, (char*)ws, &k);
  x.lead = sh.lead;
  x.prefix = sh.prefix;
  x.max_prefix = sh.max_prefix;
  x.Hq = s.heads;
  x.n = (int)n;
  x.least = 8;
  x.info_p = k.shared_p;
  x.info_s = k.shared_s;
  x.row_lead = k.shared_lead;
  if (kv_e4m3(s)) {
    if (dtype == NP_F32) return launch_shared_t<TF32, true>(x, stream);
    if (dtype == NP_F16) return launch_shared_t<TF16, true>(x, stream);
    return launch_shared_t<TBF16, true>(x, stream);
  }
  if (dtype == NP_F32) return launch_shared_t<TF32, false>(x, stream);
  if (dtype == NP_F16) return launch_shared_t<TF16, false>(x, stream);
  return launch_shared_t<TBF16, false>(x, stream);
}

}  // namespace np
