// Attention over the 4-bit cache for many query rows: prompts and their chunks.
//
// A workgroup takes 128 rows that share a key head and walks the tokens they
// see, kTok at a time.  Its eight waves widen the step's keys and values once,
// into LDS, as operands of v_mfma_f32_32x32x16; then each takes 32 of the rows
// and half of the tokens:
//   S^T = K Q^T, P = 2^(S - m), O^T += V^T P^T
// with the row as the column of both products, which is the lane (lane % 32):
// statistics stay one register each and S^T comes out as P^T goes in.  Slot s of
// S^T holds token p(s), p exchanging bits 2 and 3, so that a lane's 8 weights of
// a depth of 16 are 8 consecutive tokens, the ones whose values the cache stores
// together.  The two halves are joined through LDS at the end: tiles see very
// different numbers of tokens, and the longest should not take twice as long.
//
// Steps are pipelined: while one is multiplied out of one half of LDS, the next
// is widened into the other and the one after is on its way into registers; one
// barrier a step.  Pieces of 16 bytes in LDS are exchanged among neighbours so
// that both sides touch all banks.
//
// Bound: neither unit alone.  A step of 128 channels asks 0.85 us of the matrix
// unit, 1.1 of the vector unit and 1.0 of LDS, and takes 2.3 on each CU; fewer
// additions, operands read six ahead and other orders of the products change it by
// 1%; without widening, exponentials or operand reads (8192 tokens) it would take
// 0.88, 0.92, 0.87 of the time, without all three 0.71, at the rate of the library's
// large product.  Measured, bf16, 32 heads of 128 channels: 1024 tokens 27.2 us,
// 2048 55.3 us (622 TFLOP/s; 10 us are the launch's start, 4 each workgroup's start
// and end), 4096 176 (780), 8192 632 (870, the library 1247); of 64 channels 2048
// 35 us, 8192 392.
#include "attn_tile.h"

namespace {

using spl::AttnArgs;
using spl::Bf16;
using spl::F16;
using spl::f32x16;
using spl::f32x4;
using spl::u32x2;
using spl::u32x4;

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
static_assert(kThreads == spl::kPrefillThreads, "the launch's bound counts them");
constexpr int kRows = spl::kPrefillRows;         // of a workgroup

template <int D>
struct Geom {
  static constexpr int G = D / 32;                               // groups, and tiles of 32 channels
  static constexpr int S = G <= 2 ? 2 : 4;                       // scale bytes
  static constexpr int U = D == 64 ? 4 : 8;                      // channels of a unit of values
  static constexpr int kTok = 128;                               // tokens of a step
  static constexpr int kDeep = D / 16;                           // depths of 16 channels
  static constexpr int kKeyBytes = kTok * D * 2, kBytes = 2 * kKeyBytes;
};

// What a thread carries of the next step: one token's key, 8 channels j of every
// group; 4 channels of 8 tokens (block) of the values: part of a unit.  A wave's
// keys are 16 tokens, its values 32: their pages are scalars.
template <int D>
struct Raw {
  uint32_t k[Geom<D>::G];
  uint32_t ks;
  uint32_t v[8];
  uint32_t vs[2];
  bool held;                                     // the keys' page exists
};

// The fixed part of a thread: where its data lie in a region for a step at the
// region's start, and where they go in LDS.
struct Job {
  uint32_t key_at, key_scale_at, value_at, value_scale_at;
  uint32_t key_to, value_to[4];
  int key_unit, value_unit;                      // first of its wave's 16 tokens
  int part;                                      // half of the unit of values: 0 or 1
  int key_flag, value_flag;                      // -1: sets none
  bool key, value;
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t* d, const uint8_t* p) {
  if constexpr (N == 3) {
    typedef uint32_t w3 __attribute__((ext_vector_type(3), aligned(4)));
    const w3 x = *reinterpret_cast<const w3*>(p);
    d[0] = x[0], d[1] = x[1], d[2] = x[2];
  } else if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(p + 4 * i);
      d[i] = x[0], d[i + 1] = x[1], d[i + 2] = x[2], d[i + 3] = x[3];
    }
  } else if constexpr (N == 2) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    d[0] = x[0], d[1] = x[1];
  } else {
    d[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Page numbers of a wave's keys and of both halves of its values; -1: none.  What
// the table holds past the request's pages may be anything: its tokens are past
// every row.
struct Pages {
  int32_t k, v[2];
};
__device__ __forceinline__ Pages pages_at(const AttnArgs& a, const int32_t* table, const Job& job, int32_t t0,
                                          int shift) {
  const int32_t last = (int32_t)a.width - 1;
  const auto page = [&](int32_t t) {
    const int32_t at = t >> shift, p = spl::uniform_load(table + (at < last ? at : last));
    return p >= 0 && p < a.cache.pages ? p : -1;
  };
  return {page(t0 + job.key_unit), {page(t0 + job.value_unit), page(t0 + job.value_unit + 16)}};
}

// A page that does not exist reads page 0 instead (its tokens are masked).
template <int D>
__device__ __forceinline__ void load_raw(Raw<D>& r, const AttnArgs& a, int head, const Job& job, int32_t t0,
                                         const Pages& pg, int lane) {
  using Gm = Geom<D>;
  const int page = a.cache.page, bytes = page * (D + 2 * Gm::S);
  const uint8_t* base = static_cast<const uint8_t*>(a.cache.data);
  const auto region = [&](int32_t p) {
    return base + ((int64_t)(p < 0 ? 0 : p) * a.cache.heads + head) * (int64_t)bytes;
  };
  r.held = pg.k >= 0;
  if (job.key) {
    const uint8_t* at = region(pg.k);
    const int off = (t0 + job.key_unit) & (page - 1);
    load_words<Gm::G>(r.k, at + off * (D / 2) + job.key_at);
    const uint8_t* s = at + off * Gm::S + job.key_scale_at;
    if constexpr (Gm::S == 2) r.ks = *reinterpret_cast<const uint16_t*>(s);
    else load_words<1>(&r.ks, s);
  }
  if (job.value) {
    const int off0 = (t0 + job.value_unit) & (page - 1), off1 = (t0 + job.value_unit + 16) & (page - 1);
    const uint8_t *r0 = region(pg.v[0]), *r1 = region(pg.v[1]);
    const uint8_t* c = (lane < 32 ? r0 + off0 * (D / 2) : r1 + off1 * (D / 2)) + job.value_at;
    const uint8_t* s = (lane < 32 ? r0 + off0 * Gm::S : r1 + off1 * Gm::S) + job.value_scale_at;
    load_words<Gm::U>(r.v, c);                   // 8 tokens of 2 bytes, or of 4, half of each used
    load_words<2>(r.vs, s);
  }
}

// Where a piece of 16 bytes lies in LDS.  Keys: depth (8 channels of the two
// halves of the wave) of a tile of 32 slots; values: 32 channels by 16 tokens.
template <int D>
__device__ __forceinline__ int key_piece(int tile, int deep, int half, int slot) {
  return ((tile * Geom<D>::kDeep + deep) * 64 + half * 32 + (slot ^ ((2 * (deep & 1) + half) << 2))) * 16;
}
template <int D>
__device__ __forceinline__ int value_piece(int tile, int deep, int half, int channel) {
  const int at = half * 32 + channel;
  return Geom<D>::kKeyBytes +
         ((tile * (Geom<D>::kTok / 16) + deep) * 64 + (at ^ ((at >> 4 & 1) | (tile & 3) << 1))) * 16;
}

// Flags of half a step: a byte for each (block, group) with a bit for every
// token whose values are not finite (they go in as numbers), then one for each
// 16 tokens without a page.
constexpr int kFlags = 64, kPageFlags = 32;

template <int D>
__device__ __forceinline__ Job job_of(int page, int tid) {
  using Gm = Geom<D>;
  constexpr int kHalf = Gm::kTok / 2;
  Job job;
  const int token = tid >> 2, j = tid & 3;
  job.key = token < Gm::kTok;
  job.key_unit = __builtin_amdgcn_readfirstlane(job.key ? token & ~15 : 0);
  job.key_at = (token & 15) * (D / 2) + 4 * Gm::G * j;
  job.key_scale_at = page * D + (token & 15) * Gm::S;
  const int t = token & 31, slot = (t & 19) | (t >> 2 & 1) << 3 | (t >> 3 & 1) << 2;
  job.key_to = key_piece<D>(token >> 5, j >> 1, j & 1, slot);
  job.key_flag = job.key && j == 0 && (token & 15) == 0 ? token / kHalf * kFlags + kPageFlags + token % kHalf / 16 : -1;

  const int block = (tid >> 4) & (Gm::kTok / 8 - 1), unit = (tid & 15) < D / Gm::U ? tid & 15 : 0;
  job.part = __builtin_amdgcn_readfirstlane(tid / (2 * Gm::kTok));
  job.value = job.part < Gm::U / 4 && (tid & 15) < D / Gm::U;
  job.value_unit = __builtin_amdgcn_readfirstlane((block & ~3) * 8);
  job.value_at = page * (D / 2) + (block & 1) * (4 * D) + unit * (4 * Gm::U);
  job.value_scale_at = page * (D + Gm::S) + ((block & 1) * Gm::S + unit * Gm::U / 32) * 8;
  const int channel = unit * Gm::U + 4 * job.part;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    job.value_to[c] = value_piece<D>(channel >> 5, block >> 1, block & 1, (channel & 31) + c);
  job.value_flag = job.value && (channel & 31) == 0
                       ? block / (kHalf / 8) * kFlags + block % (kHalf / 8) * Gm::G + (channel >> 5)
                       : -1;
  return job;
}

// A thread's data widened into LDS.
template <class T, int D, int kPart>
__device__ __forceinline__ void widen_values(uint8_t* lds, const Raw<D>& r, const Job& job) {
  using Gm = Geom<D>;
  u32x4 x[4];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t pr[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float scale = spl::scale_of(r.vs[i / 4], i % 4);
      if constexpr (Gm::U == 4) pr[i] = spl::cvt_pair(T{}, r.v[i / 2], scale, 2 * (i % 2) + c);
      else pr[i] = spl::cvt_pair(T{}, r.v[i], scale, 2 * kPart + c);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x[2 * c][w] = __builtin_amdgcn_perm(pr[2 * w + 1], pr[2 * w], 0x05040100u);
      x[2 * c + 1][w] = __builtin_amdgcn_perm(pr[2 * w + 1], pr[2 * w], 0x07060302u);
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) *reinterpret_cast<u32x4*>(lds + job.value_to[c]) = x[c];
}
template <class T, int D>
__device__ __forceinline__ void widen(uint8_t* lds, uint8_t* flags, Raw<D>& r, const Job& job) {
  using Gm = Geom<D>;
  if (job.key) {
    uint8_t* to = lds + job.key_to;
#pragma unroll
    for (int g = 0; g < Gm::G; ++g)              // a group is two depths
      *reinterpret_cast<u32x4*>(to + g * 2048) = spl::cvt8<T>(r.k[g], spl::scale_of(r.ks, g));
    if (job.key_flag >= 0) flags[job.key_flag] = r.held ? 0 : 1;
  }
  if (job.value) {
    // bytes above the type's largest scale, four at a time: their low 7 bits pass the limit's
    constexpr uint32_t kAdd = (255u - spl::max_scale(T{})) * 0x01010101u;
    uint32_t bad = (((r.vs[0] & 0x7f7f7f7fu) + kAdd) & r.vs[0] & 0x80808080u) >> 7 |
                   (((r.vs[1] & 0x7f7f7f7fu) + kAdd) & r.vs[1] & 0x80808080u) >> 3;
    if (bad) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t all = (bad >> (4 * h) & 0x01010101u) * 255u;
        r.vs[h] = (r.vs[h] & ~all) | (0x7f7f7f7fu & all);
      }
      // one bit a token: byte i of the first word is bit i, of the second bit 4 + i
      bad |= bad >> 7;
      bad |= bad >> 14;
    }
    if (job.value_flag >= 0) flags[job.value_flag] = (uint8_t)bad;
    if (Gm::U == 4 || job.part == 0) widen_values<T, D, 0>(lds, r, job);
    else widen_values<T, D, 1>(lds, r, job);
  }
}

// Per lane the row's m with mc = c m - lift (reference_of), the sum of the lane's
// weights 2^(c s - mc), and the row's products with the values.  The weights are
// rounded to 16 bits for those products alone, which 16-bit matrix instructions do;
// the sum is of the exact ones, which are at hand in a register (rounded ones, added
// by a product with ones, took no less time).
template <int D>
struct State {
  float m, mc, l;
  f32x16 o[Geom<D>::G];
};

__device__ __forceinline__ float pair_max(float x) {             // over the two halves of the wave
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// A wave's rows against its part (th) of a step in LDS, whose first token is t0.
// first, last: what the lane's row sees; low: the least last of the wave's rows;
// high: their most position.
template <class T, int D>
__device__ __forceinline__ void multiply(State<D>& st, const uint8_t* lds, const uint8_t* flags, const u32x4* q,
                                         int th, int32_t t0, int32_t first, int32_t last, int32_t low, int32_t high,
                                         int32_t window, float c, int lane) {
  using Gm = Geom<D>;
  constexpr int kHalf = Gm::kTok / 2, kTiles = kHalf / 32;
  const int half = lane >> 5, col = lane & 31;
  const uint64_t flagged = __ballot(flags[lane] != 0);
  const auto piece = [](const uint8_t* base, int at) { return *reinterpret_cast<const u32x4*>(base + at); };
  // pieces of even and of odd depths of the keys share their exchange
  const uint8_t* kp[2] = {lds + key_piece<D>(th * kTiles, 0, half, col), lds + key_piece<D>(th * kTiles, 1, half, col)};
  f32x16 s[kTiles];
  __builtin_amdgcn_s_setprio(1);                 // the matrix unit before the other wave's vector work
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    s[t] = f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < Gm::kDeep; ++d)
      s[t] = spl::mfma32(T{}, piece(kp[d & 1], (t * Gm::kDeep + (d & ~1)) * 1024), q[d], s[t]);
  }
  __builtin_amdgcn_s_setprio(0);
  if (t0 + kHalf - 1 > low || (window > 0 && t0 <= high - window) || flagged >> kPageFlags) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int at = 32 * t + 16 * (i >> 3) + 8 * half + (i & 7);
        const bool see = t0 + at <= last && t0 + at >= first &&
                         !(flagged >> (kPageFlags + 2 * t + (i >> 3)) & 1);
        s[t][i] = see ? s[t][i] : -INFINITY;
      }
  }
  float top = s[0][0];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[t][i]);
  constexpr spl::Reference ref = spl::reference_of(T{});
  if (__ballot(top * c > st.mc + (ref.lift + ref.slack))) {
    const float m = fmaxf(st.m, pair_max(top)), mc = m == -INFINITY ? -INFINITY : m * c - ref.lift;
    const float alpha = m == -INFINITY ? 1.0f : spl::exp2_fast(st.mc - mc);
    st.l *= alpha;
#pragma unroll
    for (int g = 0; g < Gm::G; ++g) st.o[g] *= alpha;
    st.m = m;
    st.mc = mc;
  }
  const float base = st.m == -INFINITY ? 0.0f : -st.mc;
  u32x4 p[2 * kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float x = spl::exp2_fast(__builtin_fmaf(s[t][i], c, base));
      const float y = spl::exp2_fast(__builtin_fmaf(s[t][i + 1], c, base));
      st.l += x + y;
      p[2 * t + (i >> 3)][(i & 7) >> 1] = spl::pack2(T{}, x, y);
    }
  const uint8_t* vp[Gm::G];
#pragma unroll
  for (int g = 0; g < Gm::G; ++g) vp[g] = lds + value_piece<D>(g, th * 2 * kTiles, half, col);
#pragma unroll
  for (int d = 0; d < 2 * kTiles; ++d)
#pragma unroll
    for (int g = 0; g < Gm::G; ++g)
      st.o[g] = spl::mfma32(T{}, piece(vp[g], d * 1024), p[d], st.o[g]);
  if ((uint32_t)flagged) {                       // values that are not finite reach the rows that see them
    for (int f = 0; f < kHalf / 8 * Gm::G; ++f) {
      if (!(flagged >> f & 1)) continue;
      const int block = f / Gm::G, g = f - block * Gm::G;
      bool hit = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int32_t t = t0 + 8 * block + i;
        hit |= (flags[f] >> i & 1) && t <= last && t >= first &&
               !(flagged >> (kPageFlags + (block >> 1)) & 1);
      }
#pragma unroll
      for (int k = 0; k < Gm::G; ++k)
        if (hit && k == g) st.o[k] = st.o[k] * NAN;
    }
  }
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void k_attn_prefill(AttnArgs a, int group, int tiles) {
  using Gm = Geom<D>;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][Gm::kBytes];
  __shared__ uint8_t flags[2][2 * kFlags];
  __shared__ float stats_s[4][2][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int place = blockIdx.x / a.cache.heads, head = blockIdx.x - place * a.cache.heads;
  const Job job = job_of<D>(a.cache.page, tid);
  const int shift = __builtin_ctz((unsigned)a.cache.page);
  Raw<D> raw, ahead;
  const auto start = [&](const int32_t* table, int32_t t0, int32_t t1) {
    const Pages p0 = pages_at(a, table, job, t0, shift), p1 = pages_at(a, table, job, t1, shift);
    load_raw<D>(raw, a, head, job, t0, p0, lane);
    load_raw<D>(ahead, a, head, job, t1, p1, lane);
  };
  // where the first steps are known without the lengths, their data are requested before they are
  const bool early = a.requests == 1 && a.window == 0;
  if (early) start(a.table, 0, Gm::kTok);
  // the tiles that see the most first
  const spl::Tile tile = a.requests == 1 ? spl::Tile{0, tiles - 1 - place, spl::wave_rows_of(a, 0)}
                                         : spl::find_tile(a, group, kRows, spl::kFewRows, tiles - 1 - place);
  const int32_t req = tile.request;
  if (req < 0) return;
  const spl::Rows rows = tile.rows;
  const int32_t row0 = tile.index * kRows, all = rows.count * group;
  if (row0 >= all) return;
  const int32_t end_row = all - row0 < kRows ? all : row0 + kRows;
  const spl::Span span = spl::tile_span(rows, row0, end_row, group, a.window, Gm::kTok, 1, 0);
  const int32_t steps = span.steps;

  // the wave's rows
  const int col = lane & 31, half = lane >> 5;
  const int th = wave >> 2;                      // its half of the tokens
  const int32_t wave0 = row0 + 32 * (wave & 3);
  const bool some = wave0 < end_row;             // the wave has rows
  const int32_t row = wave0 + col < end_row ? wave0 + col : end_row - 1, tok = row / group;
  const int64_t t_row = rows.first + tok, h_row = head * group + (row - tok * group);
  const int32_t pos = wave0 + col < end_row ? rows.pos + tok : -1, end = rows.len - 1;
  const int32_t first = a.window > 0 ? pos - a.window + 1 : 0, last = pos < end ? pos : end;
  const int32_t low = rows.pos + wave0 / group, least = low < end ? low : end;
  const int32_t high = rows.pos + ((wave0 + 32 < end_row ? wave0 + 32 : end_row) - 1) / group;
  float c = fabsf(a.scale) * spl::kLog2e;
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, keep = c > 0.0f ? 0xffffffffu : 0u;
  c = c > 0.0f ? c : 1.0f;
  State<D> st;
  st.m = st.mc = -INFINITY;
  st.l = 0;
#pragma unroll
  for (int g = 0; g < Gm::G; ++g) st.o[g] = f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};

  u32x4 q[Gm::kDeep];
  const auto load_q = [&] {
    const uint16_t* at = static_cast<const uint16_t*>(a.q.data) + t_row * a.q.token_stride + h_row * a.q.head_stride;
#pragma unroll
    for (int d = 0; d < Gm::kDeep; ++d)
      q[d] = (*reinterpret_cast<const u32x4*>(at + 16 * d + 8 * half) ^ flip) & keep;
  };
  if (steps > 0) {
    if (tid < 4 * kFlags) (&flags[0][0])[tid] = 0;               // also the bytes that no thread writes
    const int32_t* table = a.table + req * a.width;
    const auto at = [&](int32_t i) { return (span.s0 + (i < steps ? i : steps - 1)) * Gm::kTok; };
    if (!early) start(table, at(0), at(1));
    Pages pg = pages_at(a, table, job, at(2), shift);
    load_q();
    __syncthreads();
    widen<T, D>(lds[0], flags[0], raw, job);
    raw = ahead;
    __syncthreads();
    for (int32_t i = 0; i < steps; ++i) {
      const int now = i & 1;
      // the two waves of a SIMD widen at different times, so that one has vector
      // work while the other's matrix instructions run
      const bool more = i + 1 < steps;
      const auto prepare = [&] {
        widen<T, D>(lds[now ^ 1], flags[now ^ 1], raw, job);
        load_raw<D>(raw, a, head, job, at(i + 2), pg, lane);
        pg = pages_at(a, table, job, at(i + 3), shift);
      };
      if (more && th == 0) prepare();
      const int32_t t0 = at(i) + th * (Gm::kTok / 2);
      if (some && t0 <= high && (a.window == 0 || t0 + Gm::kTok / 2 - 1 > low - a.window))
        multiply<T, D>(st, lds[now], flags[now] + th * kFlags, q, th, t0, first, last, least, high, a.window, c, lane);
      if (more && th == 1) prepare();
      __syncthreads();
    }
  }
  // join the halves: the second's state goes through LDS, [rows][value][lane]
  float total = pair_sum(st.l);
  float* joint = reinterpret_cast<float*>(&lds[0][0]) + (wave & 3) * (16 * Gm::G * 64);
  if (th == 1) {
    stats_s[wave & 3][0][lane] = st.mc, stats_s[wave & 3][1][lane] = total;
#pragma unroll
    for (int g = 0; g < Gm::G; ++g)
#pragma unroll
      for (int e = 0; e < 16; ++e) joint[(16 * g + e) * 64 + lane] = st.o[g][e];
  }
  __syncthreads();
  if (th == 1 || !(wave0 + col < end_row)) return;
  {
    const float other = stats_s[wave & 3][0][lane], top = fmaxf(st.mc, other);
    const float mine = st.mc == -INFINITY ? 0.0f : spl::exp2_fast(st.mc - top);
    const float its = other == -INFINITY ? 0.0f : spl::exp2_fast(other - top);
    total = total * mine + stats_s[wave & 3][1][lane] * its;
    st.mc = top;
#pragma unroll
    for (int g = 0; g < Gm::G; ++g)
#pragma unroll
      for (int e = 0; e < 16; ++e) st.o[g][e] = st.o[g][e] * mine + joint[(16 * g + e) * 64 + lane] * its;
  }
  const int64_t out_row = t_row * a.q.heads + h_row;
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;         // no key: 0 (a NaN stays one)
  uint16_t* out = static_cast<uint16_t*>(a.out) + out_row * D;
#pragma unroll
  for (int g = 0; g < Gm::G; ++g)
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
      u32x2 v;
      v[0] = spl::pack2(T{}, st.o[g][e] * inv, st.o[g][e + 1] * inv);
      v[1] = spl::pack2(T{}, st.o[g][e + 2] * inv, st.o[g][e + 3] * inv);
      *reinterpret_cast<u32x2*>(out + 32 * g + 2 * e + 4 * half) = v;
    }
  if (a.lse && half == 0) a.lse[out_row] = total == 0.0f ? -INFINITY : (st.mc + log2f(total)) * 0.6931471805599453f;
}

template <class T, int D>
hipError_t run(const AttnArgs& a, const spl::AttnPlan& p, hipStream_t s) {
  const dim3 grid((unsigned)(p.prefill_tiles * a.cache.heads));
  k_attn_prefill<T, D><<<grid, kThreads, 0, s>>>(a, p.group, (int)p.prefill_tiles);
  return hipGetLastError();
}

template <class T>
hipError_t run_dim(const AttnArgs& a, const spl::AttnPlan& p, hipStream_t s) {
  switch (a.cache.head_dim) {
    case 64: return run<T, 64>(a, p, s);
    case 96: return run<T, 96>(a, p, s);
    default: return run<T, 128>(a, p, s);
  }
}

}  // namespace

namespace spl {

hipError_t launch_attn_prefill(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
  return a.cache.dtype == SPL_F16 ? run_dim<F16>(a, p, s) : run_dim<Bf16>(a, p, s);
}

}  // namespace spl
