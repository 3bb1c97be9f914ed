// Attention over the 4-bit cache for few query rows: a token step of a serving
// loop, where the cache is read once and nothing is computed twice.
//
// For a tile of 16 query rows (the rows of a request's tokens for the query
// heads that share a key head) and 32 tokens u at a time:
//   S^T = K Q^T     two v_mfma_f32_16x16x32 per 32 channels, keys as operand A
//   m' = max(m, S), P = 2^(S - m'), l' = l 2^(m - m') + sum P
//   O^T = O^T 2^(m - m') + V^T P^T     one per 16 channels, values as operand A
// Both products have the query row as their column, which is the lane: the
// softmax's statistics stay one register each, and S^T comes out as the operand
// P^T goes in.  A lane holds 8 tokens of one row: tokens are given to the two
// halves of S so that its 8 are the 8 consecutive ones whose values it loads.
//
// Codes are widened by v_cvt_scalef32_pk, scale applied, two a instruction;
// values come as channels by token and are transposed two by two with v_perm.
//
// Bound: HBM, then latency; a step of 32 tokens is 32 (D + 2 S) bytes against some
// 200 vector instructions and D / 8 matrix instructions of one wave.  Measured, 128
// channels: 16 requests of up to 4096 tokens, 32 heads, 36.5 us, 160 MB at 4.4 TB/s
// (the loads alone 31.6, without any of the arithmetic); 64 requests of up to
// 2000, 8 heads, 21.3 us, 79 MB at 3.7; one request of 131072 tokens, 8 heads, 31 us
// and 5 for the join of 64 splits, 142 MB at 4.6; one of 93 tokens 5.2 us.  More
// waves, deeper requests or more occupancy gain nothing.
#include "attn_tile.h"

namespace {

using spl::AttnArgs;
using spl::Bf16;
using spl::F16;
using spl::f32x4;
using spl::u32x2;
using spl::u32x4;

constexpr int kRows = spl::kFewRows;
constexpr int kStep = 32;
constexpr int kWaves = 4;
constexpr int kGroupsPerCu = 2;
constexpr int kMaxSplits = 64;
constexpr int kMinChunk = 16;
constexpr int kWideSteps = 64;
constexpr int kShortSteps = 20;

template <int D>
struct Geom {
  static constexpr int G = D / 32;                               // groups
  static constexpr int S = G <= 2 ? 2 : (G <= 4 ? 4 : 8);        // scale bytes
  static constexpr int U = D == 64 ? 4 : (D == 256 ? 16 : 8);    // channels of a unit: those of one lane
  static constexpr int kUnits = D / U;                           // 16, or 12 (the other lanes idle)
  static constexpr int VD = U;                                   // dwords of a unit's 8 tokens
};

// A wave's raw data of one step.
template <int D>
struct Raw {
  uint32_t k[2][Geom<D>::G];
  uint32_t ks[2][(Geom<D>::S + 3) / 4];
  uint32_t v[Geom<D>::VD];
  uint32_t vs[2];
};

// Page numbers of the step's two halves of 16 tokens; -1: none there.  What the
// table holds past the request's pages may be anything: tokens are masked by the
// length.
struct Where {
  int32_t page[2];
};

__device__ __forceinline__ Where where(const AttnArgs& a, const int32_t* table, int32_t t0, int shift) {
  Where w;
  const int32_t last = (int32_t)a.width - 1;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int32_t at = (t0 + 16 * h) >> shift, p = spl::uniform_load(table + (at < last ? at : last));
    w.page[h] = p >= 0 && p < a.cache.pages ? p : -1;
  }
  return w;
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t* d, const uint8_t* p) {
  // pieces of 16 bytes, then of 8 and 4; p is aligned to the piece (to 4 bytes for N == 3)
  if constexpr (N == 3) {
    typedef uint32_t w3 __attribute__((ext_vector_type(3), aligned(4)));
    const w3 v = *reinterpret_cast<const w3*>(p);
    d[0] = v[0], d[1] = v[1], d[2] = v[2];
  } else if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * i);
      d[i] = v[0], d[i + 1] = v[1], d[i + 2] = v[2], d[i + 3] = v[3];
    }
  } else if constexpr (N == 2) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    d[0] = v[0], d[1] = v[1];
  } else {
    d[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// The tokens of a step that lane / 16 = j holds, i = 0 .. 7 in the order of the
// matrix instruction's depth.  They are chosen so that each load instruction of
// a wave covers whole lines: 16 bytes a lane, 1 KB in a row.
template <int D>
__device__ __forceinline__ int token_of(int j, int i) {
  constexpr int U = Geom<D>::U;
  if (U == 4) return 8 * j + i;
  if (U == 8) return (i & 3) + 4 * j + 16 * (i >> 2);
  return (i & 1) + 2 * j + 8 * (i >> 1);
}

// Where a lane's data lie in a region, for half a step at the region's start:
// the key of the half's row m = lane % 16 (token_of(m / 4, m % 4), and 16
// further in the second half), of every group the 8 channels j = lane / 16; the
// values of unit m.  With 64 channels the halves' rows lie 8 j apart instead,
// so that a lane's 8 values are one piece of 16 bytes, and a step is loaded as
// one.
struct LaneOff {
  uint32_t k, ks, v, vs;
};
template <int D>
__device__ __forceinline__ LaneOff lane_off(int page, int lane) {
  using Gm = Geom<D>;
  const int m = lane & 15, j = lane >> 4, u = m < Gm::kUnits ? m : Gm::kUnits - 1;
  LaneOff o;
  const int b = token_of<D>(m >> 2, m & 3) & (page - 1);
  o.k = b * (D / 2) + 4 * Gm::G * j;
  o.ks = page * D + b * Gm::S;
  o.v = page * (D / 2);
  o.vs = page * (D + Gm::S) + u * Gm::U / 32 * 8;
  if (Gm::U == 4) {
    const int b8 = ((8 * j) & (page - 1)) >> 3;
    o.v += (b8 * Gm::kUnits + u) * 16;
    o.vs += b8 * Gm::S * 8;
  } else if (Gm::U == 8) {
    o.v += ((j >> 1) * Gm::kUnits + u) * 32 + (j & 1) * 16;
    o.vs += (j >> 1) * Gm::S * 8 + (j & 1) * 4;
  } else {
    o.v += u * 64 + j * 16;
    o.vs += 2 * j;
  }
  return o;
}

template <int D>
__device__ __forceinline__ void load_scales(uint32_t* d, const uint8_t* p) {
  if constexpr (Geom<D>::S == 2) d[0] = *reinterpret_cast<const uint16_t*>(p);
  else load_words<Geom<D>::S / 4>(d, p);
}

// The step at t0 (a multiple of 32).  A page that does not exist reads page 0
// instead (its tokens are masked).
template <int D>
__device__ __forceinline__ void load_step(Raw<D>& r, const AttnArgs& a, int head, int32_t t0, const Where& w,
                                          const LaneOff& o, int lane) {
  using Gm = Geom<D>;
  const int page = a.cache.page, bytes = page * (D + 2 * Gm::S);
  const uint8_t* base = static_cast<const uint8_t*>(a.cache.data);
  const auto region = [&](int32_t p) {
    return base + ((int64_t)(p < 0 ? 0 : p) * a.cache.heads + head) * (int64_t)bytes;
  };
  if constexpr (Gm::U == 4) {
    const int off = t0 & (page - 1);
    const uint8_t *c = region(w.page[0]) + off * (D / 2), *s = region(w.page[0]) + off * Gm::S, *cv = c, *sv = s;
    if (page == 16) {                            // the second half is in another page
      const uint8_t* r1 = region(w.page[1]);
      cv = lane >= 32 ? r1 : c, sv = lane >= 32 ? r1 : s;
      if (lane & 8) c = s = r1;
    }
    load_words<Gm::G>(r.k[0], c + o.k);
    load_words<Gm::G>(r.k[1], c + (o.k + 2 * D));
    load_scales<D>(r.ks[0], s + o.ks);
    load_scales<D>(r.ks[1], s + (o.ks + 4 * Gm::S));
    load_words<Gm::VD>(r.v, cv + o.v);
    load_words<2>(r.vs, sv + o.vs);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int off = (t0 + 16 * h) & (page - 1);
      const uint8_t *c = region(w.page[h]) + off * (D / 2), *s = region(w.page[h]) + off * Gm::S;
      load_words<Gm::G>(r.k[h], c + o.k);
      load_scales<D>(r.ks[h], s + o.ks);
      if constexpr (Gm::U == 8) {
        load_words<4>(r.v + 4 * h, c + o.v);
        load_words<1>(r.vs + h, s + o.vs);
      } else {
        load_words<4>(r.v + 8 * h, c + o.v);
        load_words<4>(r.v + 8 * h + 4, c + (o.v + 1024));
        r.vs[h] = *reinterpret_cast<const uint16_t*>(s + o.vs) |
                  ((uint32_t)*reinterpret_cast<const uint16_t*>(s + (o.vs + 8 * Gm::S)) << 16);
      }
    }
  }
}

// S^T of the step: s[r][i] is token token_of(j, i) against the lane's query row
// of tile r.
template <class T, int D, int R>
__device__ __forceinline__ void scores(const Raw<D>& r, const u32x4 (&q)[R][Geom<D>::G], float (&s)[R][8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 acc[R];
#pragma unroll
    for (int t = 0; t < R; ++t) acc[t] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int g = 0; g < Geom<D>::G; ++g) {
      const u32x4 k = spl::cvt8<T>(r.k[h][g], spl::scale_of(r.ks[h][g / 4], g % 4));
#pragma unroll
      for (int t = 0; t < R; ++t) acc[t] = spl::mfma16(T{}, k, q[t][g], acc[t]);
    }
#pragma unroll
    for (int t = 0; t < R; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][4 * h + i] = acc[t][i];
  }
}

// The values' operand for channels U u + 2 c and U u + 2 c + 1: their pairs by
// token, transposed.
template <class T, int D>
__device__ __forceinline__ void value_pair(const Raw<D>& r, int c, u32x4& even, u32x4& odd) {
  constexpr int U = Geom<D>::U;
  uint32_t pr[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float scale = spl::scale_of(r.vs[i / 4], i % 4);
    if constexpr (U == 4) {                      // a token's 4 channels are half a dword
      pr[i] = spl::cvt_pair(T{}, r.v[i / 2], scale, 2 * (i % 2) + c);
    } else {
      pr[i] = spl::cvt_pair(T{}, r.v[i * (U / 8) + c / 4], scale, c % 4);
    }
  }
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    even[w] = __builtin_amdgcn_perm(pr[2 * w + 1], pr[2 * w], 0x05040100u);
    odd[w] = __builtin_amdgcn_perm(pr[2 * w + 1], pr[2 * w], 0x07060302u);
  }
}

// The state of a tile's softmax: per lane the row's m, with mc = c m - lift; l
// (four times the same) the sum of the weights 2^(c s - mc) as they meet the
// values: rounded to 16 bits, which the matrix instruction multiplies, so that what
// a rounding adds to a weight it adds to the sum too; o[n] channels U (4 j + i) + n of the row.  l is a row of ones among the
// values: a matrix instruction adds it up.  m is a maximum of the scores so far,
// but moves only when one passes it by the slack of reference_of.
template <int D>
struct State {
  float m, mc;
  f32x4 l;
  f32x4 o[Geom<D>::U];
};

template <int R>
struct RowView {
  int32_t pos[R], first[R];                      // what the lane's rows see: [first, pos]
  int32_t low, high;                             // the least and the most of the tile's
  int32_t window;
};

template <class T, int D, int R>
__device__ __forceinline__ void step(State<D> (&st)[R], Raw<D>& r, const u32x4 (&q)[R][Geom<D>::G],
                                     const RowView<R>& v, int32_t t0, const Where& w, int32_t len, float c, int lane) {
  using Gm = Geom<D>;
  const int j = lane >> 4;
  const bool whole = w.page[0] >= 0 && w.page[1] >= 0 && t0 + kStep - 1 <= v.low && t0 + kStep <= len &&
                     (v.window == 0 || t0 > v.high - v.window);
  float s[R][8];
  scores<T, D, R>(r, q, s);
  uint32_t poison[R] = {};                       // groups of 32 channels in which the row sees a NaN (rare)
  if (!whole) {
    uint32_t seen[R] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = token_of<D>(j, i);
      const int32_t t = t0 + at;
      const bool here = ((at < 16 ? w.page[0] : w.page[1]) >= 0) & (t < len);
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const bool see = here & (t <= v.pos[k]) & (t >= v.first[k]);
        seen[k] |= see ? 1u << i : 0u;
        s[k][i] = see ? s[k][i] : -INFINITY;
      }
    }
    // values that some row does not see must not reach it as 0 * NaN: take what
    // is not finite out of the product and put NaNs where it is seen
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (((r.vs[i / 4] >> (8 * (i % 4))) & 0xffu) > spl::max_scale(T{})) bad |= 1u << i;
    if (__ballot(bad != 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (bad >> i & 1) r.vs[i / 4] = (r.vs[i / 4] & ~(0xffu << (8 * (i % 4)))) | (127u << (8 * (i % 4)));
      for (int g = 0; g < Gm::G; ++g) {
        const int from = (lane & 48) + g * 32 / Gm::U;           // a lane of the same tokens that holds group g
        const uint32_t b = __shfl(bad, from);
#pragma unroll
        for (int k = 0; k < R; ++k)
          if (b & seen[k]) poison[k] |= 1u << g;
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        poison[k] |= __shfl_xor(poison[k], 16);
        poison[k] |= __shfl_xor(poison[k], 32);
      }
    }
  }
  constexpr spl::Reference ref = spl::reference_of(T{});
  constexpr uint32_t kOne = T::code == SPL_F16 ? 0x3c003c00u : 0x3f803f80u;
  u32x4 pf[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const float* x = s[k];
    const float top =
        fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    if (__ballot(top * c > st[k].mc + (ref.lift + ref.slack))) {
      const float m = fmaxf(st[k].m, spl::quad_max(top));
      const float mc = m == -INFINITY ? -INFINITY : m * c - ref.lift;
      const float alpha = m == -INFINITY ? 1.0f : spl::exp2_fast(st[k].mc - mc);
      st[k].l *= alpha;
#pragma unroll
      for (int n = 0; n < Gm::U; ++n) st[k].o[n] *= alpha;
      st[k].m = m;
      st[k].mc = mc;
    }
    const float base = st[k].m == -INFINITY ? 0.0f : -st[k].mc;
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = spl::exp2_fast(__builtin_fmaf(x[i], c, base));
#pragma unroll
    for (int i = 0; i < 4; ++i) pf[k][i] = spl::pack2(T{}, p[2 * i], p[2 * i + 1]);
    st[k].l = spl::mfma16(T{}, u32x4{kOne, kOne, kOne, kOne}, pf[k], st[k].l);
  }
#pragma unroll
  for (int n = 0; n < Gm::U; n += 2) {
    u32x4 even, odd;
    value_pair<T, D>(r, n / 2, even, odd);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      st[k].o[n] = spl::mfma16(T{}, even, pf[k], st[k].o[n]);
      st[k].o[n + 1] = spl::mfma16(T{}, odd, pf[k], st[k].o[n + 1]);
    }
  }
#pragma unroll
  for (int k = 0; k < R; ++k)
    if (poison[k]) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (poison[k] >> (Gm::U * (4 * j + i) / 32) & 1)
#pragma unroll
          for (int n = 0; n < Gm::U; ++n) st[k].o[n][i] = NAN;
    }
}

// The request that place `at` of the launch serves when the workgroups of
// `round` requests go to the chip's CUs in each round: the longest first, every
// other round backwards, so that what a CU gets in two rounds is alike.
// Requests up to 64: each lane ranks one (lengths past kMostRanked are alike).
constexpr int32_t kMostRanked = (1 << 26) - 1;
__device__ __forceinline__ int32_t ranked_request(const AttnArgs& a, int at, int round) {
  const int lane = spl::lane_id(), n = (int)a.requests;
  int32_t len = lane < n ? a.lens[lane] : 0;
  len = len < 0 ? 0 : (len > kMostRanked ? kMostRanked : len);
  const uint32_t key = lane < n ? (uint32_t)len << 6 | (63 - lane) : 0;      // all different
  int rank = 0;
  for (int from = 0; from < n; from += 16)
#pragma unroll
    for (int i = 0; i < 16; ++i) rank += (uint32_t)__builtin_amdgcn_readlane((int)key, from + i) > key ? 1 : 0;
  const int first = at / round * round, size = n - first < round ? n - first : round;
  const int want = at / round & 1 ? 2 * first + size - 1 - at : at;
  const uint64_t who = __ballot(lane < n && rank == want);
  return who ? __builtin_ctzll(who) : -1;
}

// What the waves of a workgroup pass to each other at the end.
template <int D>
struct Shared {
  float o[2][Geom<D>::U * 4][64];
  float m[kWaves][kRows], l[kWaves][kRows];
};

// One workgroup's work: R tiles of 16 rows of a request from row0 on, a key
// head, one of the splits of their tokens.  The four waves take every fourth
// step and are joined through LDS.  early: r0 holds the first step already.
template <class T, int D, int R>
__device__ __forceinline__ void rows_of_tile(const AttnArgs& a, Shared<D>& lds, int group, int head, int split,
                                             int splits, int chunk, int32_t req, const spl::Rows& rows, int32_t row0,
                                             bool early, Raw<D>& r0, Where& w0, const LaneOff& off, int lane,
                                             int wave) {
  using Gm = Geom<D>;
  const int32_t all = rows.count * group;
  const int n = all - row0 < R * kRows ? all - row0 : R * kRows;
  const int m16 = lane & 15, j = lane >> 4;
  const int32_t* table = a.table + req * a.width;
  const int shift = __builtin_ctz((unsigned)a.cache.page);
  const spl::Span ts = spl::tile_span(rows, row0, row0 + n, group, a.window, kStep, splits, chunk);
  const int32_t s0 = ts.s0, from = split * ts.share;
  const int32_t to = from + ts.share < ts.steps ? from + ts.share : ts.steps;
  const bool only = ts.steps <= ts.share;        // the tile is one split's
  if (split > 0 && from >= ts.steps) return;
  RowView<R> view;
  view.low = ts.low;
  view.high = ts.high;
  view.window = a.window;
  // the scores' factor is taken positive: its sign goes to q, and 0 makes all scores 0
  float c = fabsf(a.scale) * spl::kLog2e;
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, keep = c > 0.0f ? 0xffffffffu : 0u;
  c = c > 0.0f ? c : 1.0f;
  u32x4 q[R][Gm::G];
  State<D> st[R];
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const int at = 16 * k + m16;
    const int32_t row = row0 + (at < n ? at : n - 1), tok = row / group;
    view.pos[k] = at < n ? rows.pos + tok : -1;
    view.first[k] = a.window > 0 ? view.pos[k] - a.window + 1 : 0;
    const uint16_t* x = static_cast<const uint16_t*>(a.q.data) + (rows.first + tok) * a.q.token_stride +
                        (int64_t)(head * group + (row - tok * group)) * a.q.head_stride;
#pragma unroll
    for (int g = 0; g < Gm::G; ++g) q[k][g] = *reinterpret_cast<const u32x4*>(x + 32 * g + 8 * j);
#pragma unroll
    for (int g = 0; g < Gm::G; ++g) q[k][g] = (q[k][g] ^ flip) & keep;
    st[k].m = st[k].mc = -INFINITY;
    st[k].l = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < Gm::U; ++i) st[k].o[i] = f32x4{0, 0, 0, 0};
  }

  int32_t i = from + wave;
  if (i < to) {
    // the next step's data are requested before this one's are used (two steps ahead gained nothing)
    const auto fetch = [&](Raw<D>& r, Where& w, int32_t k) {
      k = k < to ? k : i;
      w = where(a, table, (s0 + k) * kStep, shift);
      load_step<D>(r, a, head, (s0 + k) * kStep, w, off, lane);
    };
    Raw<D> r1;
    Where w1;
    if (!early) fetch(r0, w0, i);
    const auto turn = [&](Raw<D>& now, Where& wn, Raw<D>& ahead, Where& wa) {
      fetch(ahead, wa, i + kWaves);
      step<T, D, R>(st, now, q, view, (s0 + i) * kStep, wn, rows.len, c, lane);
      i += kWaves;
    };
    while (true) {
      turn(r0, w0, r1, w1);
      if (i >= to) break;
      turn(r1, w1, r0, w0);
      if (i >= to) break;
    }
  }

  const spl::Parts part = spl::parts_of(a, D, splits);
#pragma unroll
  for (int k = 0; k < R; ++k) {
    State<D>& x = st[k];
    // join the waves
    if (lane < kRows) lds.m[wave][lane] = x.mc, lds.l[wave][lane] = x.l[0];
    __syncthreads();
    float top = lds.m[0][m16];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, lds.m[w][m16]);
    const auto weight = [&](float m) { return m == -INFINITY ? 0.0f : spl::exp2_fast(m - top); };
    float total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += lds.l[w][m16] * weight(lds.m[w][m16]);
    const float mine = weight(x.mc);
#pragma unroll
    for (int i = 0; i < Gm::U; ++i) x.o[i] *= mine;
    const auto give = [&](int buf) {
#pragma unroll
      for (int i = 0; i < Gm::U; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds.o[buf][4 * i + e][lane] = x.o[i][e];
    };
    const auto take = [&](int buf) {
#pragma unroll
      for (int i = 0; i < Gm::U; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x.o[i][e] += lds.o[buf][4 * i + e][lane];
    };
    if (wave >= 2) give(wave - 2);
    __syncthreads();
    if (wave < 2) take(wave);
    __syncthreads();
    if (wave == 1) give(0);
    __syncthreads();
    const int32_t at_row = 16 * k + m16;
    if (wave == 0) take(0);
    if (wave == 0 && at_row < n) {
      const int32_t row = row0 + at_row, tok = row / group;
      const int64_t out_row = (rows.first + tok) * a.q.heads + head * group + (row - tok * group);
      if (splits > 1 && split == 0 && j == 1) part.counts[out_row] = only ? 1 : (ts.steps + ts.share - 1) / ts.share;
      if (!only) {
        const int64_t at = out_row * splits + split;
        if (j == 0) part.stats[2 * at] = top, part.stats[2 * at + 1] = total;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ch = Gm::U * (4 * j + e);
          if (ch >= D) break;
#pragma unroll
          for (int i = 0; i < Gm::U; i += 4)
            *reinterpret_cast<f32x4*>(part.sums + at * D + ch + i) =
                f32x4{x.o[i][e], x.o[i + 1][e], x.o[i + 2][e], x.o[i + 3][e]};
        }
      } else {
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;   // no key: 0 (a NaN stays one)
        uint16_t* out = static_cast<uint16_t*>(a.out) + out_row * D;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int ch = Gm::U * (4 * j + e);
          if (ch >= D) break;
#pragma unroll
          for (int i = 0; i < Gm::U; i += 4) {
            u32x2 v;
            v[0] = spl::pack2(T{}, x.o[i][e] * inv, x.o[i + 1][e] * inv);
            v[1] = spl::pack2(T{}, x.o[i + 2][e] * inv, x.o[i + 3][e] * inv);
            *reinterpret_cast<u32x2*>(out + ch + i) = v;
          }
        }
        if (a.lse && j == 0)
          a.lse[out_row] = total == 0.0f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
      }
    }
    if (k + 1 < R) __syncthreads();
  }
}

// R: tiles of 16 rows that a workgroup takes where the request has them; O: waves
// a SIMD.
template <class T, int D, int R, int O>
__global__ __launch_bounds__(kWaves * 64, O) void k_attn_rows(
    AttnArgs a, int group, int direct, int all_splits, int chunk, int snake, int most) {
  const int splits = R == 1 ? all_splits : 1;    // enough workgroups: not split
  __shared__ Shared<D> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // heads fastest: consecutive workgroups go to different XCDs, so each has a
  // share of every request, however their lengths differ
  const int place = blockIdx.x / a.cache.heads, head = blockIdx.x - place * a.cache.heads, split = blockIdx.y;
  spl::Tile tile{place, 0, {0, 0, 0, 0}};
  if (!direct) tile = spl::find_tile(a, group, R * kRows, 0, place);
  else if (snake > 0) tile.request = ranked_request(a, place, snake);
  const int32_t req = tile.request;
  if (req < 0) return;
  const LaneOff off = lane_off<D>(a.cache.page, lane);
  // where the first step is known without the lengths, its data are requested before they are
  Raw<D> r0;
  Where w0;
  const bool early = R == 1 && direct && splits == 1 && a.window == 0;
  if (early) {
    w0 = where(a, a.table + req * a.width, wave * kStep, __builtin_ctz((unsigned)a.cache.page));
    load_step<D>(r0, a, head, wave * kStep, w0, off, lane);
  }
  const spl::Rows rows = direct ? spl::wave_rows_of(a, req) : tile.rows;
  const int32_t row0 = tile.index * (R * kRows), all = rows.count * group;
  if (row0 >= all || all > most) return;         // more rows than most: another kernel's
  if (R > 1 && all - row0 > kRows)
    rows_of_tile<T, D, R>(a, lds, group, head, split, splits, chunk, req, rows, row0, early, r0, w0, off, lane, wave);
  else
    rows_of_tile<T, D, 1>(a, lds, group, head, split, splits, chunk, req, rows, row0, early, r0, w0, off, lane, wave);
}

// The splits of a row joined (by the last of its workgroups instead, with a fence
// that writes the L2 back in each, 131072 tokens take 53 us and not 37; by a wave a
// row 39): W waves a row that share the splits, D / 64 channels a lane.  per > 0: the
// rows are the first `per` of a request and key head; a request of more than `most`
// is another kernel's, one of more than `per` has its first ones joined.  A lane
// knows the statistics of one split.
// Loads go out in two rounds: the counts and statistics, then all sums.
constexpr int kJoinWaves = 8;                    // of a workgroup
constexpr int kJoinDeep = kMaxSplits / kJoinWaves;               // splits of a wave
template <class T, int D, int W>
__global__ __launch_bounds__(kJoinWaves * 64) void k_attn_join(AttnArgs a, int splits, int group, int per, int joins,
                                                            int most) {
  constexpr int C = D == 256 ? 4 : 2;                            // channels of a lane; D 64 and 96 leave lanes idle
  typedef float vec __attribute__((ext_vector_type(C)));
  const int lane = threadIdx.x & 63, in = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = in & (W - 1);
  const spl::Parts p = spl::parts_of(a, D, splits);
  const int32_t join = (int32_t)blockIdx.x * (kJoinWaves / W) + in / W;
  if (join >= joins) return;                     // W 1: no wave waits for another
  int64_t row = join;
  if (per > 0) {
    const int32_t place = join / per, at = join - place * per;
    const int32_t req = place / a.cache.heads, head = place - req * a.cache.heads;
    const spl::Rows rows = spl::wave_rows_of(a, req);
    if (at >= rows.count * group || rows.count * group > most) return;
    const int32_t tok = at / group;
    row = (rows.first + tok) * a.q.heads + head * group + (at - tok * group);
  } else {
    const int32_t t = join / a.q.heads;          // tokens * heads < 2^31
    if (t < spl::uniform_load(a.row_start) || t >= spl::uniform_load(a.row_start + a.requests)) return;  // no request's
  }
  int n = __builtin_amdgcn_readfirstlane(p.counts[row]);
  const float* st = p.stats + 2 * (row * splits + (lane < splits ? lane : 0));
  float m = st[0], l = st[1];
  if (n <= 1) return;                            // written by its one split
  n = n < splits ? n : splits;
  m = lane < n ? m : -INFINITY;
  l = lane < n ? l : 0.0f;
  const int ch = lane * C;
  const float* part = p.sums + row * splits * D + (ch < D ? ch : 0);
  vec x[kJoinDeep];
#pragma unroll
  for (int i = 0; i < kJoinDeep; ++i) {
    const int s = wave + i * W;
    if (i * W < n) x[i] = *reinterpret_cast<const vec*>(part + (int64_t)(s < n ? s : 0) * D);
  }
  float top = m;
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float w = m == -INFINITY && l == 0.0f ? 0.0f : spl::exp2_fast(m - top);          // saw no key: 0
  float total = l * w;
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
  vec o = 0;
#pragma unroll
  for (int i = 0; i < kJoinDeep; ++i) {
    const int s = wave + i * W;
    if (s < n) {
      const float ws = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), s));
      o += ws * x[i];                            // a weight of 0 too: 0 times a NaN of the split is the row's NaN
    }
  }
  if constexpr (W > 1) {
    __shared__ vec o_s[W - 1][64];
    if (wave > 0) o_s[wave - 1][lane] = o;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) o += o_s[k][lane];
  }
  o *= total == 0.0f ? 0.0f : 1.0f / total;
  if (ch < D) {
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + row * D + ch);
#pragma unroll
    for (int k = 0; k < C; k += 2) out[k / 2] = spl::pack2(T{}, o[k], o[k + 1]);
  }
  if (a.lse && lane == 0) a.lse[row] = total == 0.0f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

// k_attn_prefill takes over where its tiles give every CU a workgroup.  us of
// k_attn_rows / k_attn_prefill, bf16, 128 channels, one request: 512 tokens of 32
// heads 13.5 / 17.9, the last 512 of 8192 100 / 150; 1024 tokens of 32 heads 32.1 /
// 28.7, of 16 heads 18.7 / 26.5; 2048 of 32 80 / 56.  With 256 channels its
// registers do not hold a step (1024 tokens of 16 heads 51.6 / 85.4).
// Splits: twice as many workgroups as CUs are enough (16 requests of up to 4096
// tokens, 32 heads: 512 workgroups 37.0 us, 1024 with the join 40.2; 64 requests of
// up to 2000, 8 heads: 21.6 and 31.4), and a wave wants four steps.
// 256 channels hold a step in the registers of one wave a SIMD, and one workgroup a
// CU is enough then (us with two / one, 16 heads: 24 requests of up to 1200 tokens
// 34.7 / 29.8, of 2000 43.7 / 39.9; 8 of 8000, 8 heads, 38.5 / 33.5).  Tiles of
// prompts, whose keys come from the L2, and many short requests gain more from a
// second wave than its spills cost (one / two: 1112 tokens of 32 heads over 16 114 /
// 95; 24 requests of up to 300 tokens 18.9 / 15.7, of 600 23.0 / 21.4, of 1200 29.8 /
// 35.7, of 4000 58 / 78).
// Two tiles a workgroup, which halve the widening, where enough are left and
// their tokens many.  us with one / two, bf16, 32 heads over 8, 128 channels, the
// last 512 tokens of 1024: 22.5 / 21.8, of 2048 37.1 / 32.6, of 8192 130 / 100;
// 64 channels of 2048 25.8 / 23.1; a 512-token prompt 14.8 / 15.8; 24 requests
// under a window of 1024, 64 channels, 26.2 / 28.6; the last 256 tokens of 4096,
// half the workgroups, 39.9 / 49.3.  They spill 16 registers at 128 channels and 6 at
// 96 (68 and 28 bytes of scratch a lane), and gain that much over it.
spl::AttnPlan plan_of(const AttnArgs& a) {
  const int64_t cus = spl::device_cus();
  spl::AttnPlan p{};
  p.group = a.q.heads / a.cache.heads;
  const int64_t rows = a.tokens * (int64_t)p.group;
  p.direct = a.max_new > 0 && a.max_new * p.group <= kRows;
  if (!p.direct && a.cache.head_dim < 256 && rows * a.cache.heads >= spl::kPrefillRows * cus) {
    const int64_t most = rows / spl::kPrefillRows + a.requests;
    p.prefill_tiles = most < rows ? most : rows;
    if (a.requests == 1) p.prefill_tiles = (rows + spl::kPrefillRows - 1) / spl::kPrefillRows;
    p.direct = 1;                                // what is left
  }
  int64_t len = a.width * (int64_t)a.cache.page;
  if (a.max_len > 0 && a.max_len < len) len = a.max_len;
  if (a.window > 0) {
    const int64_t seen = a.window + (a.max_new > 0 && a.max_new < kRows ? a.max_new : kRows);
    len = len < seen ? len : seen;
  }
  const int64_t steps = (len + kStep - 1) / kStep;
  const auto tiles = [&](int size) {
    const int64_t most = rows / size + a.requests;
    return most < rows ? most : rows;
  };
  p.wide = !p.direct && a.cache.head_dim < 256 && steps >= kWideSteps &&
           tiles(2 * kRows) * a.cache.heads >= kGroupsPerCu * cus;
  p.tiles = p.direct ? a.requests : tiles(p.wide ? 2 * kRows : kRows);
  if (p.prefill_tiles > 0 && a.requests == 1) p.tiles = rows > kRows ? 0 : 1;
  // split the tokens into chunks while the launch has fewer workgroups than the chip takes
  const int64_t groups = p.tiles * a.cache.heads;
  const int64_t full = (p.direct && a.cache.head_dim == 256 ? 1 : kGroupsPerCu) * cus;
  int64_t s = groups > 0 ? (full + groups - 1) / groups : 1;
  s = s < 1 ? 1 : (s > kMaxSplits ? kMaxSplits : s);
  int64_t chunk = (steps + s - 1) / s;
  chunk = chunk < kMinChunk ? kMinChunk : chunk;
  chunk = (chunk + kWaves - 1) / kWaves * kWaves;
  p.chunk = (int)chunk;
  p.splits = p.tiles > 0 ? (int)((steps + chunk - 1) / chunk) : 1;
  // no fewer than any smaller number of steps is split into
  const int64_t chunks = (steps + kMinChunk - 1) / kMinChunk;
  p.most_splits = p.tiles > 0 ? (int)(s < chunks ? s : chunks) : 1;
  p.two = a.cache.head_dim == 256 && (!p.direct || (groups > cus && steps <= kShortSteps));
  // several requests of unknown lengths, and more workgroups than CUs; ranking
  // them takes as long as they are many.  us in their order / ranked, bf16, 128
  // channels, 64 requests of 8 heads of up to 200, 400, 800, 1600, 8000 tokens 7.9 /
  // 8.5, 10.1 / 10.4, 13.2 / 12.7, 18.8 / 17.8, 72.8 / 67.2; 16 of 32 heads of up to
  // 200, 800, 1600 7.5 / 7.5, 13.7 / 11.5, 20.0 / 16.6
  const int64_t round = cus / a.cache.heads;
  const bool ranked = p.direct && a.requests <= 64 && 4 * steps >= a.requests && round >= 1 && a.requests > round;
  p.snake = ranked ? (int)round : 0;
  return p;
}

template <class T, int D>
hipError_t run(const AttnArgs& a, const spl::AttnPlan& p, hipStream_t s) {
  const int most = p.prefill_tiles > 0 ? kRows : INT32_MAX;      // rows of a request that are not another kernel's
  if (p.tiles > 0) {
    const dim3 grid((unsigned)(p.tiles * a.cache.heads), (unsigned)p.splits);
    const auto go = [&](auto kernel) {
      kernel<<<grid, kWaves * 64, 0, s>>>(a, p.group, p.direct, p.splits, p.chunk, p.snake, most);
    };
    if constexpr (D == 256) {
      if (p.two) go(k_attn_rows<T, D, 1, 2>);
      else go(k_attn_rows<T, D, 1, 1>);
    } else {
      if (p.wide) go(k_attn_rows<T, D, 2, 2>);
      else go(k_attn_rows<T, D, 1, 3>);
    }
  }
  if (p.prefill_tiles > 0) {
    const hipError_t e = spl::launch_attn_prefill(a, p, s);
    if (e != hipSuccess) return e;
  }
  if (p.splits > 1) {
    // of a direct launch only requests of one tile are split
    const int64_t one = a.max_new * p.group;
    const int per = !p.direct ? 0 : (p.prefill_tiles > 0 || one > kRows ? kRows : (int)one);
    const int64_t joins = per ? a.requests * a.cache.heads * per : a.tokens * a.q.heads;
    // few splits: a wave a row (2 splits of 5484 rows 22 us with eight, 5.7 with one)
    if (p.splits <= kJoinDeep)
      k_attn_join<T, D, 1><<<dim3((unsigned)((joins + kJoinWaves - 1) / kJoinWaves)), kJoinWaves * 64, 0, s>>>(
          a, p.splits, p.group, per, (int)joins, most);
    else
      k_attn_join<T, D, kJoinWaves><<<dim3((unsigned)joins), kJoinWaves * 64, 0, s>>>(a, p.splits, p.group, per,
                                                                                     (int)joins, most);
  }
  return hipGetLastError();
}

template <class T>
hipError_t run_dim(const AttnArgs& a, const spl::AttnPlan& p, hipStream_t s) {
  switch (a.cache.head_dim) {
    case 64: return run<T, 64>(a, p, s);
    case 96: return run<T, 96>(a, p, s);
    case 128: return run<T, 128>(a, p, s);
    default: return run<T, 256>(a, p, s);
  }
}

}  // namespace

namespace spl {

int64_t attn_workspace_bytes(const AttnArgs& a) {
  const AttnPlan p = plan_of(a);
  if (p.most_splits <= 1) return 0;
  return a.tokens * a.q.heads * ((int64_t)p.most_splits * (a.cache.head_dim + 2) + 1) * 4;
}

// The joins are fewer: of at most 16 rows each of the tiles that are split.
bool attn_fits(const AttnArgs& a) {
  const AttnPlan p = plan_of(a);
  return p.tiles * a.cache.heads <= kMaxThreads / (kWaves * 64) &&
         p.prefill_tiles * a.cache.heads <= kMaxThreads / kPrefillThreads;
}

hipError_t launch_attn(const AttnArgs& a, hipStream_t s) {
  const AttnPlan p = plan_of(a);
  return a.cache.dtype == SPL_F16 ? run_dim<F16>(a, p, s) : run_dim<Bf16>(a, p, s);
}

}  // namespace spl
