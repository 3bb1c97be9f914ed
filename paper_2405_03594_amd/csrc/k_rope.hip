// Norms of query and key heads with the rotation by position in the same pass,
// storing keys and values in the 4-bit cache, and the gradients.
//
// A head's D channels are read by LPH = 8, 16 or 32 lanes (D / 8 rounded up to
// a power of two), eight channels (16 bytes) a lane, so that a wave holds
// 64 / LPH heads and everything stays in registers: one read and one write of
// each element.  A wave takes several slots of heads of one token, so the
// angles and norm weights of its channels are loaded once for all of them.
//
// The mean of squares adds neighbours in pairs (channels 2i and 2i + 1, then
// pairs of pairs, ...), by lane exchanges whose sums do not depend on the side:
// together with products and sums that are rounded one by one this makes every
// bit of a key, and so its 4-bit codes, a function of the key alone.
//
// Bound: HBM at large sizes (2 + 2 bytes an element forward, 4 + 2 backward),
// the launch at small ones.  Measured, bf16, 2048 tokens of 128 channels: 32 + 32
// heads forward 17.8 us (67 MB at 3.8 TB/s; copies make 5.2 at 142 to 160 MB, 4.8 at
// 4 GiB), the gradient
// 23.6 (101 MB at 4.3) and 4 for the weights' sums; 32 + 8 heads stored in the
// cache 15.0, read back 4.9.  16 tokens of 32 + 32 heads stored 4.6, read back 2.8.
// What is left over a copy is the arithmetic of waves that all start together.
// Nontemporal stores: 15.1 forward, but a reader after it loses more.
#include "spl_attn.h"

#pragma clang fp contract(off)

namespace {

using spl::Bf16;
using spl::F16;
using spl::u32x2;
using spl::u32x4;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

template <int C>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), C, 0xf, 0xf, true));
}

// Sum over the LPH lanes of a head, added in pairs of neighbours.  Past the
// quad a mirrored lane stands for the exchanged one: its group has the same sum.
template <int LPH>
__device__ __forceinline__ float head_sum(float x) {
  x += dpp<0xB1>(x);                            // lane ^ 1
  x += dpp<0x4E>(x);                            // lane ^ 2
  x += dpp<0x141>(x);                           // half row mirrored: the other quad
  if (LPH >= 16) x += dpp<0x140>(x);            // row mirrored: the other half row
  if (LPH >= 32) x += __shfl_xor(x, 16);
  return x;
}

__device__ __forceinline__ float pair_tree(const float* p) {
  return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
}

template <class T>
__device__ __forceinline__ void widen(const u32x4& v, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = T::to_f32(v[i] & 0xffffu);
    x[2 * i + 1] = T::to_f32(v[i] >> 16);
  }
}
// Round to nearest even: bf16 two an instruction (v_cvt_pk_bf16_f32).
template <class T>
__device__ __forceinline__ u32x4 narrow(const float* x) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (T::code == SPL_BF16) {
      const bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
      v[i] = __builtin_bit_cast(uint32_t, p);
    } else {
      v[i] = (uint32_t)T::from_f32(x[2 * i]) | ((uint32_t)T::from_f32(x[2 * i + 1]) << 16);
    }
  }
  return v;
}

// The rotation's part of a lane: for each of its channels the cosine and the
// signed sine, and the lane that holds the other channel of each pair (halves).
template <bool kInter>
struct Turn {
  float c[8], s[8];
  int partner;
  bool on;                                      // the lane's channels are rotated
};

template <int LPH, bool kInter, bool kWhole>
__device__ __forceinline__ Turn<kInter> load_turn(const float* rope, int64_t rows, int64_t pos, int rot, int chunk,
                                                  int lane) {
  Turn<kInter> t;
  const int half = kWhole ? LPH / 2 : rot >> 4; // chunks of one half of the rotated channels
  t.on = kWhole || chunk < 2 * half;
  t.partner = lane;
  const bool known = pos >= 0 && pos < rows;
  if (!t.on) return t;
  const float* row = rope + (known ? pos : 0) * rot;
  if (kInter) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c = known ? row[8 * chunk + 2 * i] : NAN, s = known ? row[8 * chunk + 2 * i + 1] : NAN;
      t.c[2 * i] = t.c[2 * i + 1] = c;
      t.s[2 * i] = -s;
      t.s[2 * i + 1] = s;
    }
  } else {
    const bool low = chunk < half;
    t.partner = low ? lane + half : lane - half;
    const float* at = row + 16 * (low ? chunk : chunk - half);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = known ? at[2 * i] : NAN, s = known ? at[2 * i + 1] : NAN;
      t.c[i] = c;
      t.s[i] = low ? -s : s;
    }
  }
  return t;
}

// x turned by the angle (kBack: by its negative): x c + other s, each product
// and the sum rounded.  Every lane of the wave takes part.
template <int LPH, bool kInter, bool kWhole, bool kBack>
__device__ __forceinline__ void turn(const Turn<kInter>& t, float* x) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (kInter) y[i] = x[i ^ 1];
    else if (kWhole && LPH == 16) y[i] = dpp<0x128>(x[i]);      // the other half row: a rotation by 8 lanes
    else y[i] = __shfl(x[i], t.partner);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float p = y[i] * t.s[i], z = kBack ? x[i] * t.c[i] - p : x[i] * t.c[i] + p;
    x[i] = kWhole || t.on ? z : x[i];
  }
}

// 1 / rms of the heads of N payloads a lane.  The root and the division are
// some thirty instructions: each lane of a group of N does them for one of its
// heads, and the others take the result from it.
template <class T, int LPH, int N>
__device__ __forceinline__ void inverse_rms(const u32x4* x, float inv_dim, float eps, bool zero, int lane, float* r) {
  float ms[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float f[8];
    widen<T>(x[i], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = f[e] * f[e];
    ms[i] = head_sum<LPH>(zero ? 0.0f : pair_tree(f)) * inv_dim;
  }
  float mine = ms[0];
#pragma unroll
  for (int i = 1; i < N; ++i) mine = (lane & (N - 1)) == i ? ms[i] : mine;
  mine = 1.0f / sqrtf(mine + eps);
  if (N == 1) r[0] = mine;
  if (N == 2) r[0] = dpp<0xA0>(mine), r[1] = dpp<0xF5>(mine);                // the even, the odd lane of each pair
  if (N == 4) r[0] = dpp<0x00>(mine), r[1] = dpp<0x55>(mine), r[2] = dpp<0xAA>(mine), r[3] = dpp<0xFF>(mine);
}

// ---- the 4-bit cache

// Scale byte and eight 4-bit codes of a lane's channels; the four lanes of a
// quad hold one group of 32.  A group that holds an infinity or a NaN gets
// scale 255, which reads back as NaN.
template <class T>
__device__ __forceinline__ uint32_t encode8(const u32x4& bits, uint32_t* code) {
  constexpr uint32_t kInf = T::code == SPL_F16 ? 0x7c00u : 0x7f80u;
  constexpr int kLow = T::code == SPL_F16 ? 104 : 2, kHigh = T::code == SPL_F16 ? 140 : 252;
  uint32_t top = 0;                             // magnitudes are ordered as their bits
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = bits[i] & 0x7fffu, hi = (bits[i] >> 16) & 0x7fffu;
    top = top > lo ? top : lo;
    top = top > hi ? top : hi;
  }
  uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true);
  top = top > o ? top : o;
  o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, true);
  top = top > o ? top : o;
  // amax = f 2^x with 1 <= f < 2: the least e with amax <= 7 * 2^e is x - 2, or x - 1 for f > 1.75
  const uint32_t u = __float_as_uint(T::to_f32(top));
  int byte = (int)(u >> 23) - 2 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  byte = byte < kLow ? kLow : (byte > kHigh ? kHigh : byte);
  const float scale = __uint_as_float((uint32_t)byte << 23);
  float x[8];
  widen<T>(bits, x);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
  *code = c;
  return top >= kInf ? 255u : (uint32_t)byte;
}

// Where a lane's eight channels (chunk c of the head) of token b go.
__device__ __forceinline__ void store_codes(uint8_t* region, const spl::PageGeom& g, bool value, int b, int c,
                                            uint32_t code, uint32_t scale) {
  if (!value) {
    const int grp = c >> 2, j = c & 3;
    *reinterpret_cast<uint32_t*>(region + b * (g.dim >> 1) + (j * g.groups + grp) * 4) = code;
    if (j == 0) region[g.page * g.dim + b * g.scale_bytes + grp] = (uint8_t)scale;
    return;
  }
  uint8_t* at = region + g.page * (g.dim >> 1);
  if (g.unit == 8) {
    *reinterpret_cast<uint32_t*>(at + ((b >> 3) * (g.dim >> 3) + c) * 32 + (b & 7) * 4) = code;
  } else if (g.unit == 16) {
    *reinterpret_cast<uint32_t*>(at + ((b >> 3) * 16 + (c >> 1)) * 64 + (b & 7) * 8 + (c & 1) * 4) = code;
  } else {
    uint16_t* p = reinterpret_cast<uint16_t*>(at + ((b >> 3) * 16 + 2 * c) * 16 + (b & 7) * 2);
    p[0] = (uint16_t)code;
    p[8] = (uint16_t)(code >> 16);
  }
  if ((c & 3) == 0)
    region[g.page * (g.dim + g.scale_bytes) + ((b >> 3) * g.scale_bytes + (c >> 2)) * 8 + (b & 7)] = (uint8_t)scale;
}

// Where a task's heads are: a token's first tasks are q's, then k's, then (with
// a cache) v's, each of kIter slots of 64 / LPH heads.  Flat, for few heads: the
// call's first tasks are q's, and their slots run on from token to token.
struct Task {
  int token;
  bool is_q, is_v;
  int first;                                    // head, flat: row of (token, head)
};
template <bool kFlat>
__device__ __forceinline__ Task task_of(int task, int q_tasks, int k_tasks, int all_tasks, int heads) {
  const int t = kFlat ? 0 : task / all_tasks, part = task - t * all_tasks;
  Task k;
  k.token = t;
  k.is_q = part < q_tasks;
  k.is_v = part >= q_tasks + k_tasks;
  k.first = (k.is_q ? part : (k.is_v ? part - q_tasks - k_tasks : part - q_tasks)) * heads;
  return k;
}
// The token and head of a slot; one past the last repeats it (in: it does not).
struct Slot {
  int64_t token;
  int head;
  bool in;
};
template <bool kFlat>
__device__ __forceinline__ Slot slot_of(int token, int at, int heads, int64_t tokens) {
  const int last = (kFlat ? (int)tokens * heads : heads) - 1, x = at < last ? at : last;
  if (!kFlat) return {token, x, at <= last};
  const int t = x / heads;
  return {t, x - t * heads, at <= last};
}

// A wave takes tasks in a fixed stride, the next one's heads requested before
// this one's are used.
template <class T, int LPH, bool kInter, int kIter, bool kWhole, bool kFlat>
__global__ __launch_bounds__(kThreads) void k_norm_rope(spl::NormRopeArgs a, int q_tasks, int k_tasks, int all_tasks,
                                                        float inv_dim) {
  constexpr int kSlots = 64 / LPH;
  const int lane = threadIdx.x & 63, chunk = lane & (LPH - 1);
  const bool live = kWhole || 8 * chunk < a.dim;
  const int at = live ? 8 * chunk : 0;
  const int tasks = kFlat ? all_tasks : (int)a.tokens * all_tasks, stride = gridDim.x * kWaves;        // < 2^31
  u32x4 x[kIter], ahead[kIter];
  const auto fetch = [&](int task) {
    const Task k = task_of<kFlat>(task, q_tasks, k_tasks, all_tasks, kIter * kSlots);
    const spl_heads& src = k.is_q ? a.q : (k.is_v ? a.v : a.k);
    const uint16_t* in = static_cast<const uint16_t*>(src.data) + at;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const Slot s = slot_of<kFlat>(k.token, k.first + lane / LPH + i * kSlots, src.heads, a.tokens);
      ahead[i] = *reinterpret_cast<const u32x4*>(in + s.token * src.token_stride + s.head * src.head_stride);
    }
  };
  const auto turn_of = [&](int64_t t) {
    return load_turn<LPH, kInter, kWhole>(a.rope, a.rope_rows, kWhole || a.rot ? a.positions[t] : 0, a.rot, chunk, lane);
  };
  int task = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + (threadIdx.x >> 6)));
  if (task < tasks) fetch(task);
  for (; task < tasks; task += stride) {
    const Task k = task_of<kFlat>(task, q_tasks, k_tasks, all_tasks, kIter * kSlots);
    const int heads = k.is_q ? a.q.heads : a.k.heads, mine = k.first + lane / LPH;
    const bool full = kWhole && k.first + kIter * kSlots <= (kFlat ? (int)a.tokens * heads : heads);
#pragma unroll
    for (int i = 0; i < kIter; ++i) x[i] = ahead[i];
    if (tasks - task > stride) fetch(task + stride);
    const bool store = !k.is_q && a.cache.data;
    const int64_t slot = !kFlat && store ? a.slots[k.token] : -1;
    const uint16_t* w16 = static_cast<const uint16_t*>(k.is_q ? a.wq : a.wk);
    if (!k.is_v) {
      float w[8], r[kIter];
      if (w16) widen<T>(*reinterpret_cast<const u32x4*>(w16 + at), w);
      Turn<kInter> tr;
      if (!kFlat) tr = turn_of(k.token);
      uint16_t* out = static_cast<uint16_t*>(k.is_q ? a.q_out : a.k_out);
      if (out) out += at;
      if (w16) inverse_rms<T, LPH, kIter>(x, inv_dim, a.eps, !live, lane, r);
#pragma unroll
      for (int i = 0; i < kIter; ++i) {
        const Slot s = slot_of<kFlat>(k.token, mine + i * kSlots, heads, a.tokens);
        if (kFlat) tr = turn_of(s.token);
        float f[8];
        widen<T>(x[i], f);
        if (w16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = f[e] * r[i] * w[e];
        }
        if (kWhole || a.rot) turn<LPH, kInter, kWhole, false>(tr, f);
        x[i] = narrow<T>(f);
        if (out && (full || (live && s.in)))
          *reinterpret_cast<u32x4*>(out + (s.token * heads + s.head) * a.dim) = x[i];
      }
    }
    if (!store) continue;
    const int shift = __builtin_ctz((unsigned)a.cache.page);
    const spl::PageGeom g = spl::page_geom(a.dim, a.cache.page);
    if (!kFlat && (slot < 0 || (slot >> shift) >= a.cache.pages)) continue;
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      uint32_t code;
      const uint32_t scale = encode8<T>(x[i], &code);
      const Slot s = slot_of<kFlat>(k.token, mine + i * kSlots, heads, a.tokens);
      const int64_t to = kFlat ? a.slots[s.token] : slot;
      if (!(live && s.in) || (kFlat && (to < 0 || (to >> shift) >= a.cache.pages))) continue;
      uint8_t* page = static_cast<uint8_t*>(a.cache.data) + (to >> shift) * (int64_t)a.cache.heads * g.bytes;
      store_codes(page + (int64_t)s.head * g.bytes, g, k.is_v, (int)(to & (a.cache.page - 1)), chunk, code, scale);
    }
  }
}

// The cache's values of given slots: eight channels of one key and value a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void k_cache_read(spl_kv_cache c, const int32_t* slots, int64_t tokens,
                                                         uint16_t* k, uint16_t* v) {
  const spl::PageGeom g = spl::page_geom(c.head_dim, c.page);
  const int chunks = g.dim >> 3, shift = __builtin_ctz((unsigned)c.page);
  const int64_t n = tokens * c.heads * chunks;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const int64_t th = i / chunks, t = th / c.heads;
  const int ch = (int)(i - th * chunks), h = (int)(th - t * c.heads);
  const int64_t slot = slots[t];
  u32x4 ko = {0, 0, 0, 0}, vo = {0, 0, 0, 0};
  if (slot >= 0 && (slot >> shift) < c.pages) {
    const int b = (int)(slot & (c.page - 1));
    const uint8_t* r = static_cast<const uint8_t*>(c.data) + ((slot >> shift) * c.heads + h) * (int64_t)g.bytes;
    const int grp = ch >> 2;
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(r + b * (g.dim >> 1) + ((ch & 3) * g.groups + grp) * 4);
    const uint32_t ks = r[g.page * g.dim + b * g.scale_bytes + grp];
    const uint8_t* at = r + g.page * (g.dim >> 1);
    uint32_t vc;
    if (g.unit == 8) {
      vc = *reinterpret_cast<const uint32_t*>(at + ((b >> 3) * (g.dim >> 3) + ch) * 32 + (b & 7) * 4);
    } else if (g.unit == 16) {
      vc = *reinterpret_cast<const uint32_t*>(at + ((b >> 3) * 16 + (ch >> 1)) * 64 + (b & 7) * 8 + (ch & 1) * 4);
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(at + ((b >> 3) * 16 + 2 * ch) * 16 + (b & 7) * 2);
      vc = (uint32_t)p[0] | ((uint32_t)p[8] << 16);
    }
    const uint32_t vs = r[g.page * (g.dim + g.scale_bytes) + ((b >> 3) * g.scale_bytes + grp) * 8 + (b & 7)];
    const float fk = __uint_as_float(ks << 23), fv = __uint_as_float(vs << 23);
#define SPL_READ2(i)                                                                                       \
  if (T::code == SPL_F16) {                                                                                \
    ko[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(kc, fk, i));             \
    vo[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(vc, fv, i));             \
  } else {                                                                                                 \
    ko[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kc, fk, i));            \
    vo[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc, fv, i));            \
  }
    SPL_READ2(0) SPL_READ2(1) SPL_READ2(2) SPL_READ2(3)
#undef SPL_READ2
  }
  if (k) *reinterpret_cast<u32x4*>(k + th * g.dim + 8 * ch) = ko;
  if (v) *reinterpret_cast<u32x4*>(v + th * g.dim + 8 * ch) = vo;
}

// ---- gradients
//
// With xh = x r, r = 1 / rms(x), y = turn(xh w) and g = turn back(dy):
//   dw = sum over tokens and heads of g xh,   dx = r (g w - xh mean(g w xh)).
// A workgroup walks tokens in a fixed stride, its lanes keeping the same
// channels, so dw's terms stay in registers; its sums go to one row of
// `partial`, which k_norm_rope_dw adds up in order: the result does not change
// from run to run.
template <class T, int LPH, bool kInter, int kIter, bool kWhole, bool kFlat>
__global__ __launch_bounds__(kThreads) void k_norm_rope_grad(spl::NormRopeGradArgs a, int q_groups, int groups,
                                                             float inv_dim) {
  constexpr int kSlots = 64 / LPH;
  __shared__ float sum_s[kWaves][LPH * 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunk = lane & (LPH - 1);
  const bool is_q = (int)blockIdx.x < q_groups, live = kWhole || 8 * chunk < a.dim;
  const int group = is_q ? blockIdx.x : blockIdx.x - q_groups, count = is_q ? q_groups : groups - q_groups;
  const spl_heads& src = is_q ? a.q : a.k;
  const spl_heads& grad = is_q ? a.dq : a.dk;
  const int at = live ? 8 * chunk : 0;
  uint16_t* out = static_cast<uint16_t*>(is_q ? a.dq_out : a.dk_out) + at;
  const uint16_t* in = static_cast<const uint16_t*>(src.data) + at;
  const uint16_t* up = static_cast<const uint16_t*>(grad.data) + at;
  const uint16_t* w16 = static_cast<const uint16_t*>(is_q ? a.wq : a.wk);
  float w[8], dw[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[e] = 0.0f, w[e] = 1.0f;
  if (w16) widen<T>(*reinterpret_cast<const u32x4*>(w16 + at), w);
  // tasks of one token; flat: slots run on from token to token
  const int rows = kFlat ? (int)a.tokens * src.heads : src.heads, per = (rows + kIter * kSlots - 1) / (kIter * kSlots);
  const int64_t tasks = kFlat ? per : a.tokens * per;           // < 2^31
  const auto turn_of = [&](int64_t t) {
    return load_turn<LPH, kInter, kWhole>(a.rope, a.rope_rows, kWhole || a.rot ? a.positions[t] : 0, a.rot, chunk, lane);
  };
  for (int64_t task = (int64_t)group * kWaves + wave; task < tasks; task += (int64_t)count * kWaves) {
    const int task32 = __builtin_amdgcn_readfirstlane((int)task), t32 = kFlat ? 0 : task32 / per;
    const int first = (task32 - t32 * per) * kIter * kSlots, mine = first + lane / LPH;
    const bool full = kWhole && first + kIter * kSlots <= rows;
    u32x4 x[kIter], g[kIter];
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const Slot s = slot_of<kFlat>(t32, mine + i * kSlots, src.heads, a.tokens);
      g[i] = *reinterpret_cast<const u32x4*>(up + s.token * grad.token_stride + s.head * grad.head_stride);
      if (w16) x[i] = *reinterpret_cast<const u32x4*>(in + s.token * src.token_stride + s.head * src.head_stride);
    }
    Turn<kInter> tr;
    if (!kFlat) tr = turn_of(t32);
    float r[kIter];
    if (w16) inverse_rms<T, LPH, kIter>(x, inv_dim, a.eps, !live, lane, r);
#pragma unroll
    for (int i = 0; i < kIter; ++i) {
      const Slot s = slot_of<kFlat>(t32, mine + i * kSlots, src.heads, a.tokens);
      const bool counts = full || (live && s.in);               // a repeated head adds nothing to dw
      if (kFlat) tr = turn_of(s.token);
      float f[8], d[8];
      widen<T>(g[i], d);
      if (kWhole || a.rot) turn<LPH, kInter, kWhole, true>(tr, d);
      if (w16) {
        widen<T>(x[i], f);
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          f[e] *= r[i];
          dw[e] = __builtin_fmaf(full || counts ? d[e] : 0.0f, f[e], dw[e]);
          d[e] *= w[e];
          p[e] = d[e] * f[e];
        }
        const float m = head_sum<LPH>(live ? pair_tree(p) : 0.0f) * -inv_dim;
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = r[i] * __builtin_fmaf(f[e], m, d[e]);
      }
      if (counts) *reinterpret_cast<u32x4*>(out + (s.token * src.heads + s.head) * a.dim) = narrow<T>(d);
    }
  }
  if (!w16) return;                                             // the same for the whole workgroup
#pragma unroll
  for (int e = 0; e < 8; ++e)
    for (int o = LPH; o < 64; o <<= 1) dw[e] += __shfl_xor(dw[e], o);
  if (lane < LPH) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sum_s[wave][8 * chunk + e] = dw[e];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < a.dim; c += kThreads) {
    float s = 0.0f;
    for (int v = 0; v < kWaves; ++v) s += sum_s[v][c];
    a.partial[(int64_t)blockIdx.x * a.dim + c] = s;
  }
}

// dw[c] = the sum of a column of `partial`: 32 columns a workgroup, its 32 row
// groups added in order.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void k_norm_rope_dw(const float* partial, int q_groups, int groups, int dim,
                                                              float* dwq, float* dwk) {
  constexpr int kRowGroups = kSumThreads / 32;
  __shared__ float sum_s[kRowGroups][32];
  const bool is_q = blockIdx.y == 0;
  float* dw = is_q ? dwq : dwk;
  if (!dw) return;
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
  const int r0 = is_q ? 0 : q_groups, r1 = is_q ? q_groups : groups;
  float s = 0.0f;
  if (c < dim) {
#pragma unroll 8
    for (int r = r0 + row; r < r1; r += kRowGroups) s += partial[(int64_t)r * dim + c];
  }
  sum_s[row][threadIdx.x & 31] = s;
  __syncthreads();
  if (row == 0 && c < dim) {
    float total = 0.0f;
#pragma unroll
    for (int r = 0; r < kRowGroups; ++r) total += sum_s[r][threadIdx.x & 31];
    dw[c] = total;
  }
}

// Slots of a wave: four, but two where four would leave the chip without enough
// waves to hide the loads (forward and backward of 397 tokens of 24 + 8 heads of
// 96 channels: 14.5 us with four, 12.1 with two; 2048 of 32 + 32 of 128: 44.5 and
// 51.7).
constexpr int kFewWaves = 16;                   // a CU
int slots_of(int64_t tokens, int64_t heads, int lph) {
  return tokens * heads * lph >= (int64_t)kFewWaves * spl::device_cus() * 64 * 4 ? 4 : 2;
}
int lanes_of(int dim) { return dim <= 64 ? 8 : (dim <= 128 ? 16 : 32); }

// Few heads: where those of a token fill less than half of its slots, the slots
// run on over the tokens (two of a wave, with angles of their own).  us in a
// token's slots / flat: 4 + 1 heads of 4096 tokens stored 15.6 / 11.8, 1 + 1 of
// 87186 212 / 42; 6 + 1 of 64 channels, 7960 tokens, forward and backward 33.4 / 21.8.
constexpr int kFlatSlots = 2;
int wave_slots(int64_t tokens, int32_t q_heads, int32_t k_heads, int lph, bool cache, bool* flat) {
  const int64_t all = q_heads + (cache ? 2 : 1) * (int64_t)k_heads;
  const int iter = slots_of(tokens, all, lph), per = iter * (64 / lph);
  const auto filled = [&](int64_t h) { return (h + per - 1) / per * per; };
  *flat = 2 * all < filled(q_heads) + (cache ? 2 : 1) * filled(k_heads);
  return *flat ? kFlatSlots : iter;
}
int64_t tasks_of(int64_t tokens, int64_t heads, int per, bool flat) {
  return flat ? (tokens * heads + per - 1) / per : tokens * ((heads + per - 1) / per);
}

// Workgroups of the gradient for q and for k: shared out by heads, at most as
// many as the chip holds (134 registers; 2048 tokens of 32 + 32 heads of 128
// channels: three a CU 23.8 us, four 27.1).
void grad_groups(int64_t tokens, int32_t q_heads, int32_t k_heads, int32_t dim, int* q, int* k) {
  const int lph = lanes_of(dim);
  bool flat;
  const int per = wave_slots(tokens, q_heads, k_heads, lph, false, &flat) * (64 / lph);
  const int64_t most = 3 * (int64_t)spl::device_cus();
  const auto groups = [&](int64_t h) { return (tasks_of(tokens, h, per, flat) + kWaves - 1) / kWaves; };
  const int64_t gq = groups(q_heads), gk = groups(k_heads);
  int64_t nq = gq, nk = gk;
  if (gq + gk > most) {
    nq = most * gq / (gq + gk);
    nq = nq < 1 ? 1 : nq;
    nk = most - nq < 1 ? 1 : most - nq;
  }
  *q = (int)nq;
  *k = (int)nk;
}

// The instance for a head's lanes, the pairs, the slots, and whether all of its
// lanes hold rotated channels (then nothing is masked).
#define SPL_PICK(kernel, lph, inter, iter, whole, ...)                                                   \
  do {                                                                                                   \
    if ((lph) == 8) SPL_PICK_I(kernel, 8, inter, iter, whole, __VA_ARGS__);                              \
    else if ((lph) == 16) SPL_PICK_I(kernel, 16, inter, iter, whole, __VA_ARGS__);                       \
    else SPL_PICK_I(kernel, 32, inter, iter, whole, __VA_ARGS__);                                        \
  } while (0)
#define SPL_PICK_I(kernel, L, inter, iter, whole, ...)                                                   \
  do {                                                                                                   \
    if (inter) SPL_PICK_N(kernel, L, true, iter, whole, __VA_ARGS__);                                    \
    else SPL_PICK_N(kernel, L, false, iter, whole, __VA_ARGS__);                                         \
  } while (0)
#define SPL_PICK_N(kernel, L, I, iter, whole, ...)                                                       \
  do {                                                                                                   \
    if (flat) SPL_PICK_W(kernel, L, I, kFlatSlots, true, whole, __VA_ARGS__);                            \
    else if ((iter) == 4) SPL_PICK_W(kernel, L, I, 4, false, whole, __VA_ARGS__);                        \
    else SPL_PICK_W(kernel, L, I, 2, false, whole, __VA_ARGS__);                                         \
  } while (0)
#define SPL_PICK_W(kernel, L, I, N, F, whole, ...)                                                       \
  do {                                                                                                   \
    if (whole) kernel<T, L, I, N, true, F> __VA_ARGS__;                                                  \
    else kernel<T, L, I, N, false, F> __VA_ARGS__;                                                       \
  } while (0)

template <class T>
hipError_t norm_rope(const spl::NormRopeArgs& a, hipStream_t s) {
  const int lph = lanes_of(a.dim);
  bool flat;
  const int iter = wave_slots(a.tokens, a.q.heads, a.k.heads, lph, a.cache.data != nullptr, &flat);
  const int64_t tokens = flat ? a.tokens : 1;    // that the tasks are counted over
  const int per = iter * (64 / lph);
  const int qw = (int)tasks_of(tokens, a.q.heads, per, flat), kw = (int)tasks_of(tokens, a.k.heads, per, flat);
  const int all = qw + kw + (a.cache.data ? kw : 0);
  // as many waves as the chip holds (85 to 128 registers): 2048 tokens of 32 + 32
  // heads of 128 channels 18.2 us with a wave a task, 17.5 so; 2 or 3 workgroups a
  // CU 20.2, 18.3
  const int64_t need = ((flat ? 1 : a.tokens) * all + kWaves - 1) / kWaves, most = 4 * (int64_t)spl::device_cus();
  const dim3 grid((unsigned)(need < most ? need : most));
  const float inv = (float)(1.0 / a.dim);
  SPL_PICK(k_norm_rope, lph, a.interleaved, iter, a.rot == 8 * lph,
           <<<grid, kThreads, 0, s>>>(a, qw, kw, all, inv));
  return hipGetLastError();
}

template <class T>
hipError_t norm_rope_grad(const spl::NormRopeGradArgs& a, hipStream_t s) {
  int nq, nk;
  grad_groups(a.tokens, a.q.heads, a.k.heads, a.dim, &nq, &nk);
  const int lph = lanes_of(a.dim);
  bool flat;
  const int iter = wave_slots(a.tokens, a.q.heads, a.k.heads, lph, false, &flat);
  const float inv = (float)(1.0 / a.dim);
  SPL_PICK(k_norm_rope_grad, lph, a.interleaved, iter, a.rot == 8 * lph,
           <<<nq + nk, kThreads, 0, s>>>(a, nq, nq + nk, inv));
  if (a.dwq || a.dwk)
    k_norm_rope_dw<<<dim3((unsigned)((a.dim + 31) / 32), 2), kSumThreads, 0, s>>>(a.partial, nq, nq + nk, a.dim,
                                                                                a.dwq, a.dwk);
  return hipGetLastError();
}

}  // namespace

namespace spl {

hipError_t launch_norm_rope(const NormRopeArgs& a, int32_t dtype, hipStream_t s) {
  return dtype == SPL_F16 ? norm_rope<F16>(a, s) : norm_rope<Bf16>(a, s);
}

hipError_t launch_cache_read(const spl_kv_cache& c, const int32_t* slots, int64_t tokens, void* k, void* v,
                             hipStream_t s) {
  const int64_t n = cache_read_threads(c, tokens);
  const dim3 grid((unsigned)((n + kThreads - 1) / kThreads));
  if (c.dtype == SPL_F16)
    k_cache_read<F16><<<grid, kThreads, 0, s>>>(c, slots, tokens, (uint16_t*)k, (uint16_t*)v);
  else
    k_cache_read<Bf16><<<grid, kThreads, 0, s>>>(c, slots, tokens, (uint16_t*)k, (uint16_t*)v);
  return hipGetLastError();
}

int64_t norm_rope_grad_bytes(int64_t tokens, int32_t q_heads, int32_t k_heads, int32_t dim) {
  int nq, nk;
  grad_groups(tokens, q_heads, k_heads, dim, &nq, &nk);
  return (int64_t)(nq + nk) * dim * 4;
}

hipError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int32_t dtype, hipStream_t s) {
  return dtype == SPL_F16 ? norm_rope_grad<F16>(a, s) : norm_rope_grad<Bf16>(a, s);
}

}  // namespace spl
