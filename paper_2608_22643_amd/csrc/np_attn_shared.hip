// np_attn_shared.hip -- np_attn_decode_shared: decode of sequences that share
// prefixes.
//
// The softmax over a row's keys is joined from any parts of them: with (m_i,
// l_i, o_i) the maximum, sum and weighted values of part i,
//     out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i,   M = max_i m_i.
// So a group's prefix is one part of all its rows, and the query heads of those
// rows are rows of one tile against it: a key or value is read once for up to
// 128 of them.  Small groups, all of fp32, and each row's own keys are row blocks
// as in np_attn_decode: 16 query heads against keys in registers.
//
// What it costs beside the keys: the groups' search (2 us), a first step (5 to 7) and
// the join (4 to 9).  32 fp16 rows of 32 heads over 8 of 128 in four groups behind up to 3000
// keys take 22 us (np_attn_decode 35, of which the reads are 6.5): latencies in line.  48 bf16 rows
// of 64 heads over 8 behind 32768 keys of 8-bit elements take 80 to 91 us (np_attn_decode 430,
// the products alone 37 at the rate of a large one): 27 steps of a tile in each workgroup at
// 2.2 to 2.9 us, and 33 MB of parts written and read.
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

// A block on the line: `units` (steps of a tile, or groups of a row's own keys)
// of weight W behind a stretch of weight FIX for its beginning and end.  Unit u
// lies at FIX + u W of its block, and belongs to the workgroup whose stretch has
// that place.
struct Cost {
  int fix, w;
  __device__ int block(int units) const { return fix + units * w; }
  // the first unit at or past place x of a block
  __device__ int unit(int x) const { return x > fix ? (x - fix + w - 1) / w : 0; }
  __device__ int place(int unit) const { return fix + unit * w; }
};

constexpr int SH_WG = 512;  // workgroups at most

struct SharedArgs {
  AttnArgs a;
  const int32_t *lead, *prefix;
  int max_prefix;
  int Hq, n;
  int least;  // weight of a stretch at least
  int small;  // most query heads per key-value head of a group that has row blocks
  int alone;  // groups of a row's own keys, at most, that a wave takes by itself
  Cost tile, own, few;
  int32_t *info_p, *info_s, *row_lead;
  __device__ Cost cost(bool is_tile) const {
    return {is_tile ? tile.fix : own.fix, is_tile ? tile.w : own.w};
  }
  // of a row's own keys
  __device__ Cost cost_own(int groups) const {
    return {groups <= alone ? few.fix : own.fix, groups <= alone ? few.w : own.w};
  }
};

constexpr int FAR = 1 << 30;  // past all positions
static_assert(2 * KV_SHARED_HEADS + SH_WG * TB <= KV_PART_ROWS, "rows of all parts fit");

__device__ inline int div_up_pos(int a, int b) { return a > 0 ? (a + b - 1) / b : 0; }

// A row of the batch (cu_tokens NULL) as every lane may ask for it.
__device__ inline KvRow lane_row(const KvBatch& b, int i, int32_t* err) {
  return kv_row_check(b, {i, i + 1, b.seqs ? b.seqs[i] : i, b.pos0[i]}, err);
}

// The thread's number, anew for each part: what the parts derive from it would
// otherwise be kept for all of them at once, past the registers there are.
__device__ inline int own_tid() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid;
}

// What a group's shared keys are computed in: row blocks, two of them side by side
// (the keys loaded once for both), or tiles.  Two side by side pay where the keys are
// bound by memory and not by one unit's latency (us, one block after the other / side
// by side: 8 rows of 32 heads over 8 behind 2048 keys 16.0 / 19.3, behind 8192 25.5 / 24.4,
// behind 32768 53 / 41; 32 rows of 32 over 32 behind 8192 59 / 43), and never in fp32, which
// the products bound (32 rows of 4 over 4: 15.0 / 19.2, 20.5 / 22.4, 34 / 34).
enum { BLOCK, TWO_BLOCKS, TILE };
constexpr int SIDE_BY_SIDE = 65536;  // keys of all heads from which on
__device__ inline int kind_rows(int kind) {
  return kind == TILE ? TB : kind == TWO_BLOCKS ? 2 * RB : RB;
}

// Rows i0 .. i0 + 63, one a lane.
struct SharedRow {
  KvRow row;
  int lead;    // the first row of its group, or -1: by itself
  int prefix;  // positions below max_len it has in common with it
  int seq;     // the lead's sequence
  int run;     // the first of the neighbouring rows that name the same lead
  int name;    // the lead that the row names
  int kind;    // what the group's shared keys are computed in
};
template <bool TILES>
__device__ inline SharedRow shared_row(const SharedArgs& x, int i0, int run_before, int32_t* err) {
  const int lane = own_tid() % WAVE, n = x.n;
  const int i = min(i0 + lane, n - 1);
  SharedRow s;
  const int L = x.lead[i], before = x.lead[max(i - 1, 0)], after = x.lead[min(i + 1, n - 1)];
  s.name = L;
  s.row = lane_row(x.a.b, i, err);
  const uint64_t cuts = __ballot(i == 0 || before != L) & (~0ull >> (WAVE - 1 - lane));
  s.run = cuts ? i0 + 63 - __clzll((long long)cuts) : run_before;
  bool ok = L >= 0 && L <= i && s.run <= L;
  const int at = ok ? L : 0;
  const int prefix = x.prefix[at];
  // positions past max_len and the table are seen by no row, and sums with a prefix that
  // has them would leave 32 bits
  s.prefix = min(prefix, x.a.b.lim);
  s.seq = x.a.b.seqs ? x.a.b.seqs[at] : at;
  // whether the group has more rows than `small` (the same answer for all of them)
  const int past = at + x.small / x.a.G;
  s.kind = BLOCK;
  if (TILES && past < n && x.lead[past] == at) s.kind = TILE;
  else if (TILES && (int64_t)s.prefix * x.a.Hkv >= SIDE_BY_SIDE) s.kind = TWO_BLOCKS;
  ok = ok && prefix >= 0 && prefix <= x.max_prefix && s.seq >= 0 && s.seq < x.a.b.S;
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

__device__ inline int lane_max(int v) { return (int)wave_max((uint32_t)(v + 1)) - 1; }  // v >= -1

// With a window, a bound from below on the first shared key that a served row sees of
// those that a block of this lane's row can have: of its group, and at most TB / G of them.
// The lanes have the rows first .. first + 63.
__device__ inline int block_first(const SharedArgs& x, const SharedRow& s, int first) {
  const int lane = own_tid() % WAVE;  // (the lanes' addresses would be kept, too)
  int low = s.row.p0 < 0 ? FAR : s.row.p0;
#pragma unroll
  for (int off = 1; off < WAVE; off *= 2) {
    const int from = min(lane + off, WAVE - 1) * 4;  // the last lane's own rows are in all of them
    const int v = __builtin_amdgcn_ds_bpermute(from, low);
    if (__builtin_amdgcn_ds_bpermute(from, s.name) == s.name) low = min(low, v);
  }
  if (first + WAVE < x.n) {  // a group that goes on behind the lanes
    const int name = load_scalar(x.lead, first + WAVE);
    int behind = FAR;
    for (int i = first + WAVE; i < min(x.n, first + WAVE + TB / x.a.G - 1); i += WAVE) {
      const int b = min(i + lane, x.n - 1), p0 = lane_row(x.a.b, b, nullptr).p0;
      if (x.lead[b] == name && p0 >= 0) behind = min(behind, p0);
    }
    behind = FAR - lane_max(FAR - behind);
    if (s.name == name) low = min(low, behind);
  }
  return max(0, low - x.a.window + 1);
}

template <class T, int DP, bool FULL, bool E8>
__global__ __launch_bounds__(ROWS_T, DP == 256 ? 1 : 2) void attn_shared_kernel(SharedArgs x) {
  constexpr bool TILES = T::V == 8;
  using C = RowsCfg<T, DP, E8>;
  using TC = TileCfg<DP, E8>;
  constexpr int W = C::W, KS = C::KS;
  struct RowsLds {
    float o[NWAVE][RB][C::OP];
    float m[NWAVE][RB], l[NWAVE][RB];
  };
  constexpr int TILE_LDS = TILES ? 4 * TC::KB * TC::ROW : 0;
  constexpr int LDS = TILE_LDS > (int)sizeof(RowsLds) ? TILE_LDS : (int)sizeof(RowsLds);
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  // of the rows i0 .. i0 + 63 (each wave finds the same): what would stand in the
  // way of the tiles' registers
  __shared__ struct {
    int steps[WAVE], skip[WAVE], up_at[WAVE], lead[WAVE], name[WAVE], prefix[WAVE], lead_seq[WAVE];
    int kind[WAVE], groups[WAVE], us_at[WAVE], p0[WAVE], seq[WAVE];
  } rows;
  RowsLds& rl = *(RowsLds*)lds;

  const AttnArgs& a = x.a;
  const int lane = threadIdx.x % WAVE;
  const int wave = uniform((int)threadIdx.x / WAVE);
  const int n = x.n;
  const int per = (a.G + RB - 1) / RB, nb = per * a.Hkv;
  int32_t* const err = blockIdx.x == 0 && threadIdx.x < WAVE ? a.err : nullptr;

  // A lane's row, its blocks' weight on the line (up: its tile of all heads, us:
  // its own keys), and the weights up to it; steps: units of the shared keys, behind
  // `skip` of them that no row sees.
  SharedRow sr;
  int steps, skip, groups, up, us, up_at, us_at;
  auto load = [&](int first, int run_before, int32_t* e) {
    const int lane = own_tid() % WAVE;
    sr = shared_row<TILES>(x, first, run_before, e);
    const bool here = first + lane < n;
    steps = sr.lead >= 0 && here && (first + lane - sr.lead) % (kind_rows(sr.kind) / a.G) == 0
                ? div_up_pos(sr.prefix, sr.kind == TILE ? TC::KB : GROUP)
                : 0;
    // shared keys before the windows of all its rows cost nothing (one unit stays, for the
    // join, where all are)
    skip = 0;
    if (a.window) {
      const int units = block_first(x, sr, first) / (sr.kind == TILE ? TC::KB : GROUP);
      skip = max(0, min(units, steps - 1));
      steps -= skip;
    }
    groups = own_groups<KS>(sr.row.p0, sr.prefix, a.window);
    up = steps ? x.cost(sr.kind == TILE).block(steps) * a.Hkv : 0;
    us = here ? x.cost_own(groups).block(groups) * nb : 0;
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
    if (err && i + lane < n) x.row_lead[i + lane] = sr.lead < 0 ? -1 : sr.lead * 4 + sr.kind;
  }
  tp = uniform(tp);
  const int total = tp + uniform(ts);
  const int share = max(x.least, (total + (int)gridDim.x - 1) / (int)gridDim.x);
  // workgroups go round the eight XCDs; each XCD gets one stretch in a piece
  const int wg = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
  if ((int64_t)wg * share >= total) return;
  const int beg = wg * share, end = min(total, beg + share);

  // where the row of query head hq of batch row b goes, for the first part of
  // its block and for a further one
  auto part_of = [&](bool first, int base, int b, int hq, int local) {
    return first ? base + b * x.Hq + hq : 2 * n * x.Hq + wg * TB + local;
  };
  auto put = [&](int row, int d, float4 v) { *(float4*)(a.part + (size_t)row * DP + d) = v; };

  int i0 = 0;
  auto row_p0 = [&](int b) {
    return b < i0 + WAVE ? rows.p0[b - i0] : lane_row(a.b, b, nullptr).p0;
  };

  // Units [c0, c1) of block j of row i0 + at: of its group's shared keys
  // (shared), or of its own keys.
  auto part = [&](bool shared, int at, int j, int c0, int c1) __attribute__((always_inline)) {
    const int tid = own_tid(), lane = tid % WAVE;
    const int b0 = i0 + at, p = uniform(rows.prefix[at]);
    // a row block: query heads rho0 .. rho0 + nrow - 1 of head h of the rows from
    // b0 on, whose positions lie in [minpos, maxpos], against [k0, k1) of the keys
    // [kbeg, kend) that count
    int rho0 = 0, nrow, seq, h, minpos, maxpos, kbeg, kend, k0, k1;
    if (shared) {
      const int kind = uniform(rows.kind[at]);
      const bool tile = kind == TILE;
      const int RT = kind_rows(kind) / a.G, L = uniform(rows.lead[at]);
      seq = uniform(rows.lead_seq[at]);
      h = j;
      // its rows (up to RT of one group), and the positions they span
      int cnt = 0;
      for (int i = 0; i < RT && cnt == i; i += WAVE) {
        const int b = min(b0 + i + lane, n - 1);
        const int name = b < i0 + WAVE ? rows.name[b - i0] : x.lead[b];
        const uint64_t out = ~__ballot(i + lane < RT && b0 + i + lane < n && name == L);
        cnt = i + (out ? __ffsll((unsigned long long)out) - 1 : WAVE);
      }
      maxpos = -1;
      minpos = FAR;
      for (int i = 0; i < cnt; i += WAVE) {
        const int p0 = i + lane < cnt ? row_p0(b0 + i + lane) : -1;
        maxpos = max(maxpos, p0);
        if (p0 >= 0) minpos = min(minpos, p0);
      }
      maxpos = uniform(lane_max(maxpos));
      minpos = uniform(maxpos < 0 ? 0 : FAR - lane_max(FAR - minpos));
      nrow = uniform(cnt) * a.G;
      const int keys = tile ? TC::KB : GROUP;
      const int skip = uniform(rows.skip[at]);
      kbeg = max(a.window && maxpos >= 0 ? minpos - a.window + 1 : 0, (skip + c0) * keys);
      kend = min(min(p, maxpos + 1), (skip + c1) * keys);
      if (kbeg >= kend) kbeg = kend = 0;
      if constexpr (TILES) {
        if (tile) {
          // this lane's query; of a row that is not served nothing is made, and any
          // position will do
          const int wave = uniform(tid / WAVE), r = wave * 32 + (lane & 31);
          const int rho = min(r, nrow - 1), b = b0 + rho / a.G, hq = h * a.G + rho % a.G;
          const int p0 = row_p0(b);
          const char* qp = a.q + (int64_t)b * a.q_stride + (int64_t)hq * a.D * W;
          f32x16 o[TC::DT];
          float m, l;
          bool missing;
          tile_keys<T, DP, FULL, E8, true>(tid, a, a.table + (int64_t)seq * a.M, h, kbeg, kend,
                                           minpos, wave * 32 < nrow ? maxpos : -1, qp,
                                           p0 < 0 ? maxpos : p0, lds, lds + TILE_LDS / 2, o, m, l,
                                           missing);
          if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
          l = swap32_add(l, l);
          if (r < nrow) {
            const int h2 = lane >> 5;
            const int row = part_of(c0 == 0, 0, b, hq, r);
#pragma unroll
            for (int j = 0; j < TC::DT; ++j)
#pragma unroll
              for (int i = 0; i < 16; i += 4)
                put(row, 32 * j + 2 * i + 4 * h2,
                    make_float4(o[j][i], o[j][i + 1], o[j][i + 2], o[j][i + 3]));
            if (h2 == 0) *(float2*)(a.ml + (size_t)row * 2) = make_float2(m, l);
          }
          return;
        }
      }
      k0 = kbeg / KS * KS;
      k1 = kend;
    } else {
      h = j % a.Hkv;
      rho0 = j / a.Hkv * RB;
      nrow = min(RB, a.G - rho0);
      seq = uniform(rows.seq[at]);
      minpos = maxpos = uniform(rows.p0[at]);
      kbeg = own_first<KS>(maxpos, p, a.window);
      kend = maxpos + 1;
      k0 = kbeg / KS * KS + c0 * GROUP;
      k1 = kbeg < kend ? min(kend, kbeg / KS * KS + c1 * GROUP) : k0;  // none: no step
    }
    auto rows_part = [&](auto blocks) __attribute__((always_inline)) {
      constexpr int QT = decltype(blocks)::value;
      const char* qp[QT];
      int qpos[QT];
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        const int rho = rho0 + min(RB * i + (lane & 15), nrow - 1);
        const int b = b0 + rho / a.G, hq = h * a.G + rho % a.G, p0 = row_p0(b);
        qp[i] = a.q + (int64_t)b * a.q_stride + (int64_t)hq * a.D * W;
        qpos[i] = p0 < 0 ? maxpos : p0;
      }
      f32x4 o[QT][C::VS][C::NV];
      float m[QT], l[QT];
      bool missing;
      rows_keys<T, DP, FULL, E8, true, QT>(tid, a, a.table + (int64_t)seq * a.M, h, minpos, maxpos,
                                           kbeg, kend, k0, k1, qp, qpos, o, m, l, missing);
      if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
#pragma unroll
      for (int i = 0; i < QT; ++i) {
        rows_meet<C>(o[i], m[i], l[i], rl.o, rl.m, rl.l);
        __syncthreads();
        for (int u = tid; u < min(RB, nrow - RB * i) * (DP / 4); u += ROWS_T) {
          const int q = u / (DP / 4), d = u % (DP / 4) * 4, rho = rho0 + RB * i + q;
          float M, L;
          const float4 sum = rows_met<C>(rl.o, rl.m, rl.l, q, d, M, L);
          const int row = part_of(c0 == 0, shared ? 0 : n * x.Hq, b0 + rho / a.G,
                                  h * a.G + rho % a.G, RB * i + q);
          put(row, d, sum);
          if (d == 0) *(float2*)(a.ml + (size_t)row * 2) = make_float2(M, L);
        }
        __syncthreads();  // LDS is free again
      }
    };
    if (TILES && nrow > RB) rows_part(std::integral_constant<int, TILES ? 2 : 1>{});
    else rows_part(std::integral_constant<int, 1>{});
  };

  // All of block j of row i0 + at's own keys, by this wave: no exchange with others.
  auto wave_part = [&](int at, int j) __attribute__((always_inline)) {
    const int lane = own_tid() % WAVE;
    const int b = i0 + at, h = j % a.Hkv, rho0 = j / a.Hkv * RB, nrow = min(RB, a.G - rho0);
    const int pos = uniform(rows.p0[at]), seq = uniform(rows.seq[at]);
    const int kbeg = own_first<KS>(pos, uniform(rows.prefix[at]), a.window), kend = pos + 1;
    const int k0 = kbeg / KS * KS, hq = h * a.G + rho0 + min(lane & 15, nrow - 1);
    const char* const qp[1] = {a.q + (int64_t)b * a.q_stride + (int64_t)hq * a.D * W};
    const int qpos[1] = {pos};
    f32x4 o[1][C::VS][C::NV];
    float m[1], l[1];
    bool missing;
    rows_keys<T, DP, FULL, E8, true, 1, 1>(lane, a, a.table + (int64_t)seq * a.M, h, pos, pos, kbeg,
                                           kend, k0, kbeg < kend ? kend : k0, qp, qpos, o, m, l,
                                           missing);
    if (missing && lane == 0) atomicOr(a.err, NP_DEVERR_NOT_RESIDENT);
    l[0] = sum_groups(l[0]);
    if (lane == 0) x.info_s[b * nb + j] = wg | wg << 16;
    if ((lane & 15) >= nrow) return;
    const int g = lane >> 4, row = part_of(true, n * x.Hq, b, hq, 0);
#pragma unroll
    for (int s = 0; s < C::VS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int y = 0; y < C::NV; y += 4)
          put(row, 16 * C::NV * s + C::NV * (4 * g + i) + y,
              make_float4(o[0][s][y][i], o[0][s][y + 1][i], o[0][s][y + 2][i], o[0][s][y + 3][i]));
    if (g == 0) *(float2*)(a.ml + (size_t)row * 2) = make_float2(m[0], l[0]);
  };

  int pb = 0, sb = tp;  // weights before the chunk
  run = 0;
  for (; i0 < n && (pb < min(tp, end) || sb < end); i0 += WAVE) {
    if (n > WAVE) {
      load(i0, run, nullptr);
      run = last(sr.run);
      __syncthreads();
    }
    if (wave == 0) {
      rows.steps[lane] = steps;
      rows.skip[lane] = skip;
      rows.up_at[lane] = pb + up_at - up;
      rows.lead[lane] = sr.lead;
      rows.name[lane] = sr.name;
      rows.prefix[lane] = sr.prefix;
      rows.lead_seq[lane] = sr.seq;
      rows.kind[lane] = sr.kind;
      rows.groups[lane] = groups;
      rows.us_at[lane] = sb + us_at - us;
      rows.p0[lane] = sr.row.p0;
      rows.seq[lane] = sr.row.seq;
    }
    const uint64_t with_tiles = __ballot(up > 0 && pb + up_at > beg && pb + up_at - up < end);
    const uint64_t with_own = __ballot(us > 0 && sb + us_at > beg && sb + us_at - us < end);
    pb += last(up_at);
    sb += last(us_at);
    __syncthreads();
    for (int kind = 0; kind < 2; ++kind) {
      const bool shared = kind == 0;
      uint64_t hit = shared ? with_tiles : with_own;
      while (hit) {
        const int at = __ffsll((unsigned long long)hit) - 1;
        hit &= hit - 1;
        // this row's blocks that have units in the stretch
        const int units = uniform(shared ? rows.steps[at] : rows.groups[at]);
        const Cost c = shared ? x.cost(uniform(rows.kind[at]) == TILE) : x.cost_own(units);
        const int start = uniform(shared ? rows.up_at[at] : rows.us_at[at]);
        const int count = shared ? a.Hkv : nb, len = c.block(units);
        int32_t* const info = shared ? x.info_p : x.info_s;
        for (int j = max(0, beg - start) / len; j < count; ++j) {
          const int x0 = start + j * len;
          if (x0 >= end) break;
          const int c0 = min(units, c.unit(beg - x0)), c1 = min(units, c.unit(end - x0));
          if (c0 >= c1) continue;
          if (!shared && units <= x.alone && c0 == 0 && c1 == units) {
            // this block and the next ones that are here as a whole, a wave each
            int many = 1;
            while (many < NWAVE && j + many < count &&
                   x0 + many * len + c.place(units - 1) < end)
              ++many;
            if (wave < many) wave_part(at, j + wave);
            j += many - 1;
            continue;
          }
          if (c0 == 0 && threadIdx.x == 0)
            info[(i0 + at) * count + j] = wg | (x0 + c.place(units - 1)) / share << 16;
          part(shared, at, j, c0, c1);
        }
      }
    }
  }
}

// A wave per query head: its parts joined, in their order.
template <class T, int DP>
__global__ __launch_bounds__(ROWS_T) void attn_shared_join_kernel(SharedArgs x) {
  constexpr int TD = DP / 4, SUB = WAVE / TD, W = 16 / T::V;
  const AttnArgs& a = x.a;
  const int lane = threadIdx.x % WAVE;
  const int id = uniform((int)(blockIdx.x * (ROWS_T / WAVE) + threadIdx.x / WAVE));
  if (id >= x.n * x.Hq) return;
  const int b = id / x.Hq, hq = id % x.Hq, h = hq / a.G, g = hq % a.G;
  const int per = (a.G + RB - 1) / RB, nb = per * a.Hkv;
  const int named = load_scalar(x.row_lead, b), L = named >> 2;
  const int RT = kind_rows(named & 3) / a.G;
  const int is = load_scalar(x.info_s, b * nb + g / RB * a.Hkv + h);
  const int b0 = L < 0 ? b : L + (b - L) / RT * RT;
  const int ip = L < 0 ? 0 : load_scalar(x.info_p, b0 * a.Hkv + h);
  const KvRow row = kv_row(a.b, b, nullptr);
  const int np = L < 0 ? 0 : (ip >> 16) - (ip & 0xFFFF) + 1;
  const int ns = (is >> 16) - (is & 0xFFFF) + 1;
  const int extra = 2 * x.n * x.Hq;
  auto part_row = [&](int c) {
    if (c < np) return c ? extra + ((ip & 0xFFFF) + c) * TB + (b - b0) * a.G + g : id;
    c -= np;
    return c ? extra + ((is & 0xFFFF) + c) * TB + g % RB : x.n * x.Hq + id;
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
  const dim3 grid(DP == 256 ? SH_WG / 2 : SH_WG), block(ROWS_T);
  if (x.a.D == DP)
    hipLaunchKernelGGL((attn_shared_kernel<T, DP, true, E8>), grid, block, 0, stream, x);
  else
    hipLaunchKernelGGL((attn_shared_kernel<T, DP, false, E8>), grid, block, 0, stream, x);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned waves = (unsigned)(x.n * x.Hq);
  hipLaunchKernelGGL((attn_shared_join_kernel<T, DP>),
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
  auto apart = [&] {
    return launch_attn(s, layer, b, table, q, q_stride, pool, scale, window, out, out_stride, ws,
                       stream);
  };
  if (heads > KV_SHARED_HEADS || G > (dtype == NP_F32 ? RB : TB)) return apart();
  // The line counts 32 keys of a tile's rows: a row block's 128 keys cost as much as
  // a tile's 128 (its rows are fewer, but so are the keys in flight), and a tile's
  // beginning and end as much as four to eight of its steps.  Us with tiles' beginning
  // and step at 8, 2 / 0, 2 / 0, 4 / 32, 2: 32 rows of 32 heads over 8 in four groups
  // behind up to 3000 keys 22.2 / 27.7 / 23.2 / 24.1, 48 rows of 64 over 8 behind 32768 in
  // 8-bit elements 79.7 / 87.6 / 104.9 / 86.1.
  x.tile = {8, s.head_dim > 128 ? 1 : 2};
  x.own = {0, 4};
  // More blocks of own keys than workgroups, which would have them one after the other:
  // up to 256 keys in a wave each, four of them in the time of two of the others.  Us, all
  // waves on a block / a wave a block (weight 1): 90 fp16 rows of 40 heads over 40 in three
  // groups behind up to 1500 keys, 1 to 60 of their own 51.5 / 39.6 (41.7), of 32 over 32
  // behind 300 36.3 / 29.9 (28.0), of 40 over 8 behind 1500 31.3 / 28.2 (27.4); 20 of 32 over
  // 32 of 256 behind 1000, 1 to 250 of their own 38.6 / 28.8 (36.5); but with 256 blocks, 32
  // rows of 32 over 8 behind 3000, 1 to 300 of their own 22.3 / 24.6 (26.1).
  x.few = {0, 2};
  x.alone = heads / G * ((G + RB - 1) / RB) > SH_WG ? 2 : 0;
  x.least = 4;
  x.small = dtype == NP_F32 ? 0 : 32;
  // the line's length: at most a block of shared keys a row, and every row's own
  const int64_t longest = std::min<int64_t>(sh.max_prefix, x.a.b.lim);
  const int64_t line =
      n * s.kv_heads * ((longest / 32 + 1) * x.tile.w + x.tile.fix + x.own.fix) +
      heads * (((int64_t)x.a.b.lim / GROUP + 2) * x.own.w + x.own.fix);
  // What sharing saves is at most the bytes of the prefix, or of a window of it, for all
  // rows but one; the join, and the search for the groups, cost 4 us and 0.1 a row, about
  // what 32 MB and 1 MB a row take to read.  Us apart / shared (bf16, 32 heads over 8 of 128; the
  // bytes in brackets): 2 rows behind 2048 keys 11 / 15 (8 MB), behind 8192 22 / 20 (34
  // MB); 8 rows behind 512 9 / 15 (15 MB), behind 2048 18 / 16 (59 MB); 32 rows behind
  // 512 18 / 20 (65 MB), behind 2048 33 / 23 (260 MB); what the groups really save only the
  // device knows: 32 rows behind 2048 as four groups 35 / 26, as pairs 44 / 35, alone 48 / 51;
  // of 64 over 8 behind 4096 in 8-bit elements 39 / 29, 41 / 45, 48 / 52.  With a window half as much again (48
  // rows of 64 over 8 behind 32768, windows of 600, 1000 and 4096 keys: 21.5 / 26.8, 28.8 /
  // 28.3, 102 / 37; 8 of 32 over 8 of 256, 1000 and 4096: 19.8 / 24.6, 53 / 39; where keys
  // that no row sees stood on the line too, 256 to 4096 took 64 to 69 us of the first).
  const int64_t seen = window > 0 ? std::min(sh.max_prefix, window) : sh.max_prefix;
  const int64_t saved = (n - 1) * seen * s.kv_heads * 2 * kv_row_bytes(s);
  // Rows of up to 256 keys of 8-bit elements, many blocks: np_attn_decode has a wave for each
  // (36 rows of 40 heads over 40, 192 keys shared, 17.3 / 20.1; 160 of 32 over 32 34.2 / 37.5
  // to 41.3; plain fp16 25.0 / 21.9, 50.0 / 47.9).
  const bool brief = kv_e4m3(s) && x.a.b.lim <= 256 && (int64_t)x.a.tiles * s.kv_heads > 768;
  const int64_t asked = (32 + n) * (window > 0 ? 1500000 : 1000000);
  if (saved < asked || brief || line >= ((int64_t)1 << 30)) return apart();
  KvScratch k;
  kv_ws_layout(s, (char*)ws, &k);
  x.lead = sh.lead;
  x.prefix = sh.prefix;
  x.max_prefix = sh.max_prefix;
  x.Hq = s.heads;
  x.n = (int)n;
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
