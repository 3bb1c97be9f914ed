// Device code shared by the attention kernels: operands out of the 4-bit
// cache, the requests' rows in tiles, the masks.
#pragma once

#include "spl_attn.h"

namespace spl {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t cvt_pair(Bf16, uint32_t code, float scale, int sel) {
  switch (sel) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3));
  }
}
__device__ __forceinline__ uint32_t cvt_pair(F16, uint32_t code, float scale, int sel) {
  switch (sel) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, scale, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, scale, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, scale, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(code, scale, 3));
  }
}
// The eight values of a dword of codes under scale byte `b` of the word `s`
// (the conversion reads the scale's exponent alone: what the shift leaves in
// the sign and the fraction has no effect).
template <class T>
__device__ __forceinline__ u32x4 cvt8(uint32_t code, float scale) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = cvt_pair(T{}, code, scale, i);
  return v;
}
__device__ __forceinline__ float scale_of(uint32_t s, int b) {
  return __uint_as_float(b == 0 ? s << 23 : b == 1 ? s << 15 : b == 2 ? s << 7 : s >> 1);
}

// The largest scale byte whose values the type holds.
__device__ constexpr uint32_t max_scale(Bf16) { return 252; }
__device__ constexpr uint32_t max_scale(F16) { return 140; }

__device__ __forceinline__ f32x4 mfma16(Bf16, const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ f32x4 mfma16(F16, const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                0);
}

__device__ __forceinline__ f32x16 mfma32(Bf16, const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ f32x16 mfma32(F16, const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                0);
}

// How the softmax's weights 2^(c s - reference) are kept in the type: they are at
// most 2^lift when the reference is set, to a maximum of the scores, and it moves
// only when they would pass 2^(lift + slack).  bf16 has fp32's range, so its
// weights keep 8 bits at any size.  fp16 ends at 2^16 and loses bits below 2^-14:
// lifted, a weight is whole down to 2^-24 of the largest.
struct Reference {
  float lift, slack;
};
__device__ constexpr Reference reference_of(Bf16) { return {0.0f, 8.0f}; }
__device__ constexpr Reference reference_of(F16) { return {10.0f, 5.0f}; }

// Two floats rounded to nearest even, the first in the low half.
__device__ __forceinline__ uint32_t pack2(Bf16, float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint32_t pack2(F16, float a, float b) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A wave-uniform load through the scalar cache (the memory is not written by
// the kernel).
__device__ __forceinline__ int32_t uniform_load(const int32_t* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>((uintptr_t)p);
}

// Maximum over the four lanes that share lane % 16.
__device__ __forceinline__ float quad_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t v = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Row indexes of a request, clamped to the call's rows, its length, clamped to the
// table's, and its first row's position, which follows from both as they are given:
// a request may have more rows than the call, and more tokens than pages.
struct Rows {
  int64_t first;
  int32_t count, len, pos;
};
__device__ __forceinline__ Rows rows_of(const AttnArgs& a, int64_t r) {
  const int64_t t = a.tokens;
  int64_t s = a.row_start[r], e = a.row_start[r + 1];    // lane by lane: requests may differ
  const int64_t most = a.width * (int64_t)a.cache.page;
  int64_t len = a.lens[r];
  len = len < 0 ? 0 : len;
  s = s < 0 ? 0 : (s > t ? t : s);
  const int32_t pos = (int32_t)(len - e + s);
  e = e < s ? s : (e > t ? t : e);
  return {s, (int32_t)(e - s), (int32_t)(len > most ? most : len), pos};
}

// The same for a request that is the wave's: scalar loads, all at once.
__device__ __forceinline__ Rows wave_rows_of(const AttnArgs& a, int32_t r) {
  const int32_t t = (int32_t)a.tokens, most = (int32_t)(a.width * a.cache.page);          // < 2^31
  int32_t s = uniform_load(a.row_start + r), e = uniform_load(a.row_start + r + 1), len = uniform_load(a.lens + r);
  len = len < 0 ? 0 : len;
  s = s < 0 ? 0 : (s > t ? t : s);
  const int32_t pos = (int32_t)((uint32_t)len - (uint32_t)e + (uint32_t)s);
  e = e < s ? s : (e > t ? t : e);
  return {s, e - s, len > most ? most : len, pos};
}

// Inclusive sum over the lanes of a wave: within rows of 16, then a row's or two
// rows' last lane added to what follows.
__device__ __forceinline__ int32_t lane_sums(int32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The request that owns tile `tile` when each of more than `few` rows (rows *
// group) has ceil(rows * group / size) tiles, the tile's number in it and its
// rows; request -1 past the last.  Every lane of the wave calls it with the same
// tile; the launch's tiles are fewer than 2^31.
struct Tile {
  int32_t request, index;
  Rows rows;
};
__device__ __forceinline__ Tile find_tile(const AttnArgs& a, int group, int size, int few, int32_t tile) {
  const int lane = lane_id();
  const int32_t requests = (int32_t)a.requests;
  for (int32_t base = 0; base < requests; base += 64) {
    const Rows r = rows_of(a, base + lane < requests ? base + lane : requests - 1);
    int32_t n = base + lane < requests ? r.count * group : 0;
    n = n > few ? (n - 1) / size + 1 : 0;
    const int32_t sum = lane_sums(n);
    const uint64_t past = __ballot(sum > tile);
    if (past) {
      const int k = __builtin_ctzll(past);
      const int32_t index = tile - __builtin_amdgcn_readlane(sum - n, k);
      // requests that overlap may pass 2^31 tiles in all: none of theirs then
      if ((uint32_t)index >= (uint32_t)__builtin_amdgcn_readlane(n, k)) break;
      return {base + k, index,
              {__builtin_amdgcn_readlane((int32_t)r.first, k), __builtin_amdgcn_readlane(r.count, k),
               __builtin_amdgcn_readlane(r.len, k), __builtin_amdgcn_readlane(r.pos, k)}};
    }
    tile -= __builtin_amdgcn_readlane(sum, 63);
  }
  return {-1, 0, {0, 0, 0, 0}};
}

// The steps of `unit` tokens that any of the rows [row0, end_row) of a request
// sees, and a split's share of them: chunk of them, more where the splits would
// not reach the end.
struct Span {
  int32_t low, high;                             // positions of the first and the last row
  int32_t s0, steps, share;
};
__device__ __forceinline__ Span tile_span(const Rows& rows, int32_t row0, int32_t end_row, int group, int32_t window,
                                          int unit, int splits, int chunk) {
  Span t;
  t.low = rows.pos + row0 / group;
  t.high = rows.pos + (end_row - 1) / group;
  const int32_t end = t.high + 1 < rows.len ? t.high + 1 : rows.len;
  const int32_t begin = window > 0 && t.low - window + 1 > 0 ? t.low - window + 1 : 0;
  t.s0 = begin / unit;
  t.steps = end > begin ? (end + unit - 1) / unit - t.s0 : 0;
  const int32_t least = (t.steps + splits - 1) / splits;
  t.share = chunk > least ? chunk : least;
  return t;
}

// The workspace of split calls: per row and split the sums and (reference times
// log2 e, weight), per row the splits that hold any of it.
struct Parts {
  float* sums;
  float* stats;
  int32_t* counts;
};
__device__ __forceinline__ Parts parts_of(const AttnArgs& a, int dim, int splits) {
  const int64_t n = a.tokens * a.q.heads * splits;
  float* w = static_cast<float*>(a.workspace);
  return {w, w + n * dim, reinterpret_cast<int32_t*>(w + n * (dim + 2))};
}

}  // namespace spl
