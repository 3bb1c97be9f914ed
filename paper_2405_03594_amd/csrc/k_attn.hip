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
// Bound: HBM; a step of 32 tokens is 32 (D + 2 S) bytes against some 200 vector
// instructions and D / 8 matrix instructions of one wave.
#include "attn_tile.h"

namespace {

using spl::AttnArgs;
using spl::Bf16;
using spl::F16;
using spl::f32x4;
using spl::u32x2;
using spl::u32x4;

constexpr int kRows = 16;
constexpr int kStep = 32;
constexpr int kWaves = 4;

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

struct Where {
  int64_t page[2];                               // of the step's two halves; -1: none
};

template <int D>
__device__ __forceinline__ Where where(const AttnArgs& a, const int32_t* table, int32_t t0, int32_t len, int shift) {
  Where w;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int32_t t = t0 + 16 * h;
    const int64_t p = t < len ? table[t >> shift] : -1;
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

// The lane's data of the step at t0: the key of token 8 (m / 4) + m % 4 and of
// the one four further (m = lane % 16), of every group the 8 channels j = lane
// / 16; the values of tokens 8 j .. 8 j + 7, unit lane % 16.  A page that does
// not exist reads page 0 instead (its tokens are masked).
template <int D>
__device__ __forceinline__ void load_step(Raw<D>& r, const AttnArgs& a, int head, int32_t t0, const Where& w,
                                          int lane) {
  using Gm = Geom<D>;
  const int page = a.cache.page, bytes = page * (D + 2 * Gm::S);
  const int m = lane & 15, j = lane >> 4;
  const uint8_t* base = static_cast<const uint8_t*>(a.cache.data);
  const auto region = [&](int64_t p) { return base + ((p < 0 ? 0 : p) * a.cache.heads + head) * (int64_t)bytes; };
  const uint8_t* r0 = region(w.page[0]);
  const uint8_t* r1 = region(w.page[1]);
  const int off = (t0 & (page - 1));
  {
    const uint8_t* rk = m < 8 ? r0 : r1;
    const int b = ((off + 8 * (m >> 2)) & (page - 1)) + (m & 3);
    const uint8_t* p = rk + b * (D / 2) + 4 * Gm::G * j;
    const uint8_t* s = rk + page * D + b * Gm::S;
    load_words<Gm::G>(r.k[0], p);
    load_words<Gm::G>(r.k[1], p + 4 * (D / 2));
    if constexpr (Gm::S == 2) {
      r.ks[0][0] = *reinterpret_cast<const uint16_t*>(s);
      r.ks[1][0] = *reinterpret_cast<const uint16_t*>(s + 4 * Gm::S);
    } else {
      load_words<Gm::S / 4>(r.ks[0], s);
      load_words<Gm::S / 4>(r.ks[1], s + 4 * Gm::S);
    }
  }
  {
    const uint8_t* rv = j < 2 ? r0 : r1;
    const int b8 = ((off + 8 * j) & (page - 1)) >> 3, u = m < Gm::kUnits ? m : Gm::kUnits - 1;
    load_words<Gm::VD>(r.v, rv + page * (D / 2) + (b8 * Gm::kUnits + u) * (4 * Gm::U));
    load_words<2>(r.vs, rv + page * (D + Gm::S) + (b8 * Gm::S + u * Gm::U / 32) * 8);
  }
}

// S^T of the step: s[i] is token 8 j + i against the lane's query row.
template <class T, int D>
__device__ __forceinline__ void scores(const Raw<D>& r, const u32x4* q, float* s) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int g = 0; g < Geom<D>::G; ++g)
      acc = spl::mfma16(T{}, spl::cvt8<T>(r.k[h][g], spl::scale_of(r.ks[h][g / 4], g % 4)), q[g], acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[4 * h + i] = acc[i];
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

// The state of a tile's softmax: per lane the row's maximum (times log2 e) and
// the sum over the lane's tokens; o[n] channels U (4 j + i) + n of the row.
template <int D>
struct State {
  float m, l;
  f32x4 o[Geom<D>::U];
};

struct RowView {
  int32_t pos;                                   // of the lane's row; -1: sees nothing
  int32_t low, high;                             // the least and the most of the tile's
  int32_t window;
};

template <class T, int D>
__device__ __forceinline__ void step(State<D>& st, Raw<D>& r, const u32x4* q, const RowView& v, int32_t t0,
                                     const Where& w, int32_t len, float c, int lane) {
  using Gm = Geom<D>;
  const int j = lane >> 4;
  const bool whole = w.page[0] >= 0 && w.page[1] >= 0 && t0 + kStep - 1 <= v.low && t0 + kStep <= len &&
                     (v.window == 0 || t0 > v.high - v.window);
  float s[8];
  scores<T, D>(r, q, s);
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] *= c;
  uint32_t poison = 0;                           // groups of 32 channels in which the row sees a NaN (rare)
  if (!whole) {
    const bool held = (j < 2 ? w.page[0] : w.page[1]) >= 0;
    const int32_t t = t0 + 8 * j;
    uint32_t seen = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool see = held && t + i < len && t + i <= v.pos && (v.window == 0 || t + i > v.pos - v.window);
      seen |= see ? 1u << i : 0u;
      s[i] = see ? s[i] : -INFINITY;
    }
    // values that some row does not see must not reach it as 0 * NaN: take the
    // NaNs out of the product and put them where they are seen
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (((r.vs[i / 4] >> (8 * (i % 4))) & 0xffu) == 255u) bad |= 1u << i;
    if (__ballot(bad != 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (bad >> i & 1) r.vs[i / 4] = (r.vs[i / 4] & ~(0xffu << (8 * (i % 4)))) | (127u << (8 * (i % 4)));
      for (int g = 0; g < Gm::G; ++g) {
        const int from = (lane & 48) + g * 32 / Gm::U;           // a lane of this block of tokens that holds group g
        const uint32_t b = __shfl(bad, from);
        if (b & seen) poison |= 1u << g;
      }
      poison |= __shfl_xor(poison, 16);
      poison |= __shfl_xor(poison, 32);
    }
  }
  float top = s[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = fmaxf(top, s[i]);
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  const float m = fmaxf(st.m, top);
  if (__ballot(m != st.m)) {
    const float alpha = m == -INFINITY ? 1.0f : spl::exp2_fast(st.m - m);
    st.l *= alpha;
#pragma unroll
    for (int n = 0; n < Gm::U; ++n) st.o[n] *= alpha;
    st.m = m;
  }
  const float base = m == -INFINITY ? 0.0f : m;
  float p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = spl::exp2_fast(s[i] - base);
    st.l += p[i];
  }
  u32x4 pf;
#pragma unroll
  for (int i = 0; i < 4; ++i) pf[i] = spl::pack2(T{}, p[2 * i], p[2 * i + 1]);
#pragma unroll
  for (int n = 0; n < Gm::U; n += 2) {
    u32x4 even, odd;
    value_pair<T, D>(r, n / 2, even, odd);
    st.o[n] = spl::mfma16(T{}, even, pf, st.o[n]);
    st.o[n + 1] = spl::mfma16(T{}, odd, pf, st.o[n + 1]);
  }
  if (poison) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (poison >> (Gm::U * (4 * j + i) / 32) & 1)
#pragma unroll
        for (int n = 0; n < Gm::U; ++n) st.o[n][i] = NAN;
  }
}

// One workgroup: a tile of rows, a key head, one of the splits of its tokens.
// The four waves take every fourth step and are joined through LDS.
template <class T, int D>
__global__ __launch_bounds__(kWaves * 64) void k_attn_rows(AttnArgs a, int group, int direct, int splits) {
  using Gm = Geom<D>;
  __shared__ float o_s[2][Gm::U * 4][64];
  __shared__ float m_s[kWaves][kRows], l_s[kWaves][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.y, split = blockIdx.z;
  spl::Tile tile{(int64_t)blockIdx.x, 0};
  if (!direct) tile = spl::find_tile(a, group, kRows, blockIdx.x);
  const int64_t req = __builtin_amdgcn_readfirstlane((int)tile.request);
  if (req < 0) return;
  const spl::Rows rows = spl::rows_of(a, req);
  const int64_t row0 = tile.index * kRows, all = (int64_t)rows.count * group;
  if (row0 >= all) return;
  const int n = (int)(all - row0 < kRows ? all - row0 : kRows);            // rows of this tile
  const int m16 = lane & 15, j = lane >> 4;
  const int32_t first_pos = rows.len - rows.count;
  const int64_t row = row0 + (m16 < n ? m16 : n - 1);
  const int32_t tok = (int32_t)(row / group);
  const int64_t t_row = rows.first + tok, h_row = head * group + (row - (int64_t)tok * group);
  RowView view;
  view.pos = m16 < n ? first_pos + tok : -1;
  view.low = first_pos + (int32_t)(row0 / group);
  view.high = first_pos + (int32_t)((row0 + n - 1) / group);
  view.window = a.window;
  // the steps that any row of the tile sees, and this split's share of them
  const int32_t end = view.high + 1 < rows.len ? view.high + 1 : rows.len;
  const int32_t begin = a.window > 0 && view.low - a.window + 1 > 0 ? view.low - a.window + 1 : 0;
  const int32_t s0 = begin / kStep, steps = end > begin ? (end + kStep - 1) / kStep - s0 : 0;
  const int32_t share = (steps + splits - 1) / splits;
  const int32_t from = split * share, to = from + share < steps ? from + share : steps;
  const int32_t* table = a.table + req * a.width;
  const int shift = __builtin_ctz((unsigned)a.cache.page);

  u32x4 q[Gm::G];
  {
    const uint16_t* at = static_cast<const uint16_t*>(a.q.data) + t_row * a.q.token_stride + h_row * a.q.head_stride;
#pragma unroll
    for (int g = 0; g < Gm::G; ++g) q[g] = *reinterpret_cast<const u32x4*>(at + 32 * g + 8 * j);
  }
  State<D> st;
  st.m = -INFINITY;
  st.l = 0;
#pragma unroll
  for (int i = 0; i < Gm::U; ++i) st.o[i] = f32x4{0, 0, 0, 0};
  const float c = a.scale * spl::kLog2e;

  int32_t i = from + wave;
  if (i < to) {
    Raw<D> cur;
    Where w = where<D>(a, table, (s0 + i) * kStep, rows.len, shift);
    load_step<D>(cur, a, head, (s0 + i) * kStep, w, lane);
    for (; i < to; i += kWaves) {
      const int32_t next = i + kWaves < to ? i + kWaves : i;
      const Where wn = where<D>(a, table, (s0 + next) * kStep, rows.len, shift);
      Raw<D> ahead;
      load_step<D>(ahead, a, head, (s0 + next) * kStep, wn, lane);
      step<T, D>(st, cur, q, view, (s0 + i) * kStep, w, rows.len, c, lane);
      cur = ahead;
      w = wn;
    }
  }

  // join the waves
  st.l += __shfl_xor(st.l, 16);
  st.l += __shfl_xor(st.l, 32);
  if (lane < kRows) m_s[wave][lane] = st.m, l_s[wave][lane] = st.l;
  __syncthreads();
  float top = m_s[0][m16];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, m_s[w][m16]);
  const auto weight = [&](float m) { return m == -INFINITY ? 0.0f : spl::exp2_fast(m - top); };
  float total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) total += l_s[w][m16] * weight(m_s[w][m16]);
  const float mine = weight(st.m);
#pragma unroll
  for (int k = 0; k < Gm::U; ++k) st.o[k] *= mine;
  const auto give = [&](int buf) {
#pragma unroll
    for (int k = 0; k < Gm::U; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) o_s[buf][4 * k + e][lane] = st.o[k][e];
  };
  const auto take = [&](int buf) {
#pragma unroll
    for (int k = 0; k < Gm::U; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) st.o[k][e] += o_s[buf][4 * k + e][lane];
  };
  if (wave >= 2) give(wave - 2);
  __syncthreads();
  if (wave < 2) take(wave);
  __syncthreads();
  if (wave == 1) give(0);
  __syncthreads();
  if (wave != 0) return;
  take(0);
  if (m16 >= n) return;

  const int64_t out_row = t_row * a.q.heads + h_row;
  if (splits > 1) {
    float* part = static_cast<float*>(a.workspace);
    const int64_t all_rows = a.tokens * a.q.heads;
    const int64_t at = out_row * splits + split;
    float* stats = part + all_rows * splits * D;
    if (j == 0) stats[2 * at] = top, stats[2 * at + 1] = total;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ch = Gm::U * (4 * j + e);
      if (ch >= D) break;
#pragma unroll
      for (int k = 0; k < Gm::U; k += 4)
        *reinterpret_cast<f32x4*>(part + at * D + ch + k) =
            f32x4{st.o[k][e], st.o[k + 1][e], st.o[k + 2][e], st.o[k + 3][e]};
    }
    return;
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;         // no key: 0 (a NaN stays one)
  uint16_t* out = static_cast<uint16_t*>(a.out) + out_row * D;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int ch = Gm::U * (4 * j + e);
    if (ch >= D) break;
#pragma unroll
    for (int k = 0; k < Gm::U; k += 4) {
      u32x2 v;
      v[0] = spl::pack2(T{}, st.o[k][e] * inv, st.o[k + 1][e] * inv);
      v[1] = spl::pack2(T{}, st.o[k + 2][e] * inv, st.o[k + 3][e] * inv);
      *reinterpret_cast<u32x2*>(out + ch + k) = v;
    }
  }
  if (a.lse && j == 0) a.lse[out_row] = total == 0.0f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

// The splits of a row joined: one wave a row, D / 64 channels a lane.
template <class T, int D>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, int splits) {
  constexpr int C = D == 256 ? 4 : 2;                            // channels of a lane; D 64 and 96 leave lanes idle
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), rows = a.tokens * a.q.heads;
  if (row >= rows) return;
  // rows that no request owns have no partial results
  const int64_t t = row / a.q.heads;
  const int64_t t0 = a.row_start[0], t1 = a.row_start[a.requests];
  if (t < t0 || t >= t1) return;
  const float* part = static_cast<const float*>(a.workspace);
  const float* stats = part + rows * splits * D + 2 * row * splits;
  float top = -INFINITY;
  for (int s = lane; s < splits; s += 64) top = fmaxf(top, stats[2 * s]);
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  float total = 0, o[C];
#pragma unroll
  for (int k = 0; k < C; ++k) o[k] = 0;
  const int ch = lane * C;
  for (int s = 0; s < splits; ++s) {
    const float m = stats[2 * s], l = stats[2 * s + 1];
    if (m == -INFINITY && l == 0.0f) continue;                   // saw no key
    const float w = spl::exp2_fast(m - top);
    total += l * w;
    if (ch < D) {
#pragma unroll
      for (int k = 0; k < C; ++k) o[k] += w * part[(row * splits + s) * D + ch + k];
    }
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  if (ch < D) {
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + row * D + ch);
#pragma unroll
    for (int k = 0; k < C; k += 2) out[k / 2] = spl::pack2(T{}, o[k] * inv, o[k + 1] * inv);
  }
  if (a.lse && lane == 0) a.lse[row] = total == 0.0f ? -INFINITY : (top + log2f(total)) * 0.6931471805599453f;
}

struct Plan {
  int64_t tiles;
  int group, direct, splits;
};

Plan plan_of(const AttnArgs& a) {
  Plan p;
  p.group = a.q.heads / a.cache.heads;
  p.direct = a.max_new > 0 && a.max_new * p.group <= kRows;
  const int64_t most = a.tokens * (int64_t)p.group / kRows + a.requests;
  p.tiles = p.direct ? a.requests : (most < a.tokens * p.group ? most : a.tokens * p.group);
  // split the tokens while the launch has fewer workgroups than the chip takes
  int64_t len = a.width * (int64_t)a.cache.page;
  if (a.max_len > 0 && a.max_len < len) len = a.max_len;
  if (a.window > 0) {
    const int64_t seen = a.window + (a.max_new > 0 && a.max_new < kRows ? a.max_new : kRows);
    len = len < seen ? len : seen;
  }
  const int64_t groups = p.tiles * a.cache.heads, want = 4 * (int64_t)spl::device_cus();
  const int64_t steps = (len + kStep - 1) / kStep;
  int64_t s = (want + groups - 1) / groups;
  const int64_t most_s = (steps + 2 * kWaves - 1) / (2 * kWaves);
  s = s < most_s ? s : most_s;
  s = s < 1 ? 1 : (s > 256 ? 256 : s);
  p.splits = (int)s;
  return p;
}

template <class T, int D>
hipError_t run(const AttnArgs& a, const Plan& p, hipStream_t s) {
  const dim3 grid((unsigned)p.tiles, (unsigned)a.cache.heads, (unsigned)p.splits);
  k_attn_rows<T, D><<<grid, kWaves * 64, 0, s>>>(a, p.group, p.direct, p.splits);
  if (p.splits > 1) {
    const int64_t rows = a.tokens * a.q.heads;
    k_attn_join<T, D><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, s>>>(a, p.splits);
  }
  return hipGetLastError();
}

template <class T>
hipError_t run_dim(const AttnArgs& a, const Plan& p, hipStream_t s) {
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
  const Plan p = plan_of(a);
  if (p.splits == 1) return 0;
  return a.tokens * a.q.heads * (int64_t)p.splits * (a.cache.head_dim + 2) * 4;
}

hipError_t launch_attn(const AttnArgs& a, hipStream_t s) {
  const Plan p = plan_of(a);
  return a.cache.dtype == SPL_F16 ? run_dim<F16>(a, p, s) : run_dim<Bf16>(a, p, s);
}

}  // namespace spl
