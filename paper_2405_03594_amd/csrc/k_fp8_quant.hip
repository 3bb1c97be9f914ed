// Quantization to 8-bit floats with a power-of-two scale for each block of 128
// (the format stands in spl.h), for gfx950.
//
// A workgroup of 256 threads takes 128 x 128 entries of X: thread (rg, cg) has rows
// 8 rg .. 8 rg + 7 and columns 8 cg .. 8 cg + 7 in registers, so a row's 128
// entries are 16 neighbouring lanes (their largest magnitude by four lane
// moves) and a column's are 8 registers, 4 lanes and 4 waves.  Both results come
// from one read.  Rows leave as 8 bytes a lane, 128 to a row; the transpose's codes
// are converted two rows at a time, so that a thread's 8 rows of a column are 8
// bytes, and go through LDS (their place in a row of 128 bytes turned by the
// column) to leave as 16 bytes a lane.
#include <type_traits>

#include "spl_fp8.h"

namespace spl {
namespace {

struct F32In {};
template <class T>
__device__ __forceinline__ float widen(const void* p, int64_t at) {
  if constexpr (std::is_same<T, F32In>::value)
    return static_cast<const float*>(p)[at];
  else
    return T::to_f32(static_cast<const uint16_t*>(p)[at]);
}

// 8 neighbours from an address of 16 bytes' alignment.
template <class T>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&v)[8]) {
  if constexpr (std::is_same<T, F32In>::value) {
    const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
    const f32x4 a = q[0], b = q[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[2 * j] = T::to_f32(a[j] & 0xffffu), v[2 * j + 1] = T::to_f32(a[j] >> 16);
  }
}

__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Of fp32 (a training step's masters; 64 registers of entries): 4096 x 4096 in 128 x 128 blocks, both results, 16.5 us (6.1
// TB/s), a scale a row 19.2 (5.2); 11008 x 4096 47.8 and 50.7.
template <class T, bool kRows, bool kCols, int kBlock>
__global__ void __launch_bounds__(256) k_fp8_quantize(const Fp8QuantArgs a, const int wide) {
  static_assert(std::is_same<T, F32In>::value, "16-bit types: below");
  __shared__ __align__(16) uint8_t tile[kCols ? 128 * 128 : 16];
  __shared__ uint32_t most[4][128];
  const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4, wave = tid >> 6;
  // my tile: rows [r0, rend) of X, which are block tb of a column of the transpose
  int r0 = blockIdx.y * 128, rend = (int)a.rows;
  const int tb = blockIdx.y;
  if (a.starts) {
    const Segment s = find_tile(a.starts, a.groups, (int)a.rows, 128, tb);
    if (s.group < 0) return;
    r0 = s.row, rend = s.end;
  }
  const int c0 = blockIdx.x * 128, z = blockIdx.z;
  const int64_t base = (int64_t)z * a.rows * a.row_stride;
  float v[8][8];
  const int c = c0 + 8 * cg;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 8 * rg + i;
    const int64_t at = base + (int64_t)r * a.row_stride + c;
    if (r < rend && wide && c + 8 <= a.cols) {
      load8<T>(a.X, at, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
      if (r < rend && c < a.cols) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < a.cols) v[i][j] = widen<T>(a.X, at + j);
      }
    }
  }

  uint32_t whole = 0;
  if constexpr (kBlock == 128) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) whole = umax(whole, mag(v[i][j]));
    whole = row16_max(whole);
    if (cg == 0) most[0][rg] = whole;
    __syncthreads();
    whole = row16_max(most[0][cg]);
    whole = fp8_scale_byte(whole);
  }

  if constexpr (kRows) {
    uint8_t* codes = const_cast<uint8_t*>(a.out.codes) + z * a.out.code_stride;
    uint8_t* scales = const_cast<uint8_t*>(a.out.scales) + z * a.out.scale_stride;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + 8 * rg + i;
      uint32_t byte = whole;
      if constexpr (kBlock == 1) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = umax(m, mag(v[i][j]));
        byte = fp8_scale_byte(row16_max(m));
      }
      const float f = fp8_inverse(byte);
      u32x2 q = {fp8_four(v[i][0] * f, v[i][1] * f, v[i][2] * f, v[i][3] * f),
                 fp8_four(v[i][4] * f, v[i][5] * f, v[i][6] * f, v[i][7] * f)};
      if (byte == 255) q = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
      if (r < rend) {
        *reinterpret_cast<u32x2*>(codes + (int64_t)r * a.out.pitch + c) = q;
        if (kBlock == 1 && cg == 0) scales[(int64_t)r * a.out.spitch + blockIdx.x] = (uint8_t)byte;
      }
    }
    if (kBlock == 128 && tid == 0) scales[(int64_t)tb * a.out.spitch + blockIdx.x] = (uint8_t)whole;
  }

  if constexpr (kCols) {
    uint8_t* codes = const_cast<uint8_t*>(a.out_t.codes) + z * a.out_t.code_stride;
    uint8_t* scales = const_cast<uint8_t*>(a.out_t.scales) + z * a.out_t.scale_stride;
    uint32_t byte[8];
    if constexpr (kBlock == 1) {
      uint32_t m[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m[j] = umax(m[j], mag(v[i][j]));
        m[j] = umax(m[j], (uint32_t)__shfl_xor((int)m[j], 16));
        m[j] = umax(m[j], (uint32_t)__shfl_xor((int)m[j], 32));
      }
      if ((rg & 3) == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) most[wave][8 * cg + j] = m[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = 8 * cg + j;
        byte[j] = fp8_scale_byte(umax(umax(most[0][k], most[1][k]), umax(most[2][k], most[3][k])));
        if (rg == 0 && c + j < a.cols) scales[(int64_t)(c + j) * a.out_t.spitch + tb] = (uint8_t)byte[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) byte[j] = whole;
      if (tid == 0) scales[(int64_t)blockIdx.x * a.out_t.spitch + tb] = (uint8_t)whole;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float f = fp8_inverse(byte[j]);
      u32x2 q = {fp8_four(v[0][j] * f, v[1][j] * f, v[2][j] * f, v[3][j] * f),
                 fp8_four(v[4][j] * f, v[5][j] * f, v[6][j] * f, v[7][j] * f)};
      if (byte[j] == 255) q = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
      *reinterpret_cast<u32x2*>(tile + (8 * cg + j) * 128 + 8 * (rg ^ cg)) = q;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = 32 * q + (tid >> 3), u = 2 * (tid & 7);
      const u32x2 lo = *reinterpret_cast<const u32x2*>(tile + k * 128 + 8 * (u ^ (k >> 3)));
      const u32x2 hi = *reinterpret_cast<const u32x2*>(tile + k * 128 + 8 * ((u + 1) ^ (k >> 3)));
      if (c0 + k < a.cols)
        *reinterpret_cast<u32x4*>(codes + (int64_t)(c0 + k) * a.out_t.pitch + (int64_t)tb * 128 + 8 * u) =
            u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
}

// The same for 16-bit types, which stay two to a register (32 of them instead of 64, and a conversion takes two values with
// their scale): 2048 x 11008 of bf16, both results, 22.5 -> 17.6 us (5.1 TB/s), its transpose
// alone 17.7 -> 13.4; 4096 x 4096 in blocks of 128 x 128 11.9 (5.6 TB/s).
template <class T, bool kRows, bool kCols, int kBlock>
__global__ void __launch_bounds__(256) k_fp8_quantize16(const Fp8QuantArgs a, const int wide) {
  __shared__ __align__(16) uint8_t tile[kCols ? 128 * 128 : 16];
  __shared__ uint32_t most[4][64];
  const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4, wave = tid >> 6;
  int r0 = blockIdx.y * 128, rend = (int)a.rows;
  const int tb = blockIdx.y;
  if (a.starts) {
    const Segment s = find_tile(a.starts, a.groups, (int)a.rows, 128, tb);
    if (s.group < 0) return;
    r0 = s.row, rend = s.end;
  }
  const int c0 = blockIdx.x * 128, z = blockIdx.z, c = c0 + 8 * cg;
  const uint16_t* x = static_cast<const uint16_t*>(a.X) + (int64_t)z * a.rows * a.row_stride;
  u32x4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 8 * rg + i;
    const uint16_t* row = x + (int64_t)r * a.row_stride + c;
    if (r < rend && wide && c + 8 <= a.cols) {
      v[i] = *reinterpret_cast<const u32x4*>(row);
    } else {
      v[i] = u32x4{0u, 0u, 0u, 0u};
      if (r < rend && c < a.cols) {                  // (lanes past the columns do not wait for single loads)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t lo = c + 2 * j < a.cols ? row[2 * j] : 0u, hi = c + 2 * j + 1 < a.cols ? row[2 * j + 1] : 0u;
          v[i][j] = lo | (hi << 16);
        }
      }
    }
  }
  const auto byte_of = [](uint32_t m) { return fp8_scale_byte(__float_as_uint(T::to_f32(m))); };

  uint32_t whole = 0;
  if constexpr (kBlock == 128) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) whole = max16(whole, mag16(v[i][j]));
    whole = row16_max(umax(whole & 0xffffu, whole >> 16));
    if (cg == 0) most[0][rg] = whole;
    __syncthreads();
    whole = byte_of(row16_max(most[0][cg]));
  }

  if constexpr (kRows) {
    uint8_t* codes = const_cast<uint8_t*>(a.out.codes) + z * a.out.code_stride;
    uint8_t* scales = const_cast<uint8_t*>(a.out.scales) + z * a.out.scale_stride;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + 8 * rg + i;
      uint32_t byte = whole;
      if constexpr (kBlock == 1) {
        const uint32_t m = max16(max16(mag16(v[i][0]), mag16(v[i][1])), max16(mag16(v[i][2]), mag16(v[i][3])));
        byte = byte_of(row16_max(umax(m & 0xffffu, m >> 16)));
      }
      const float f = fp8_scale(byte);
      u32x2 q = {fp8_code4<T>(v[i][0], v[i][1], f), fp8_code4<T>(v[i][2], v[i][3], f)};
      if (byte == 255) q = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
      if (r < rend) {
        *reinterpret_cast<u32x2*>(codes + (int64_t)r * a.out.pitch + c) = q;
        if (kBlock == 1 && cg == 0) scales[(int64_t)r * a.out.spitch + blockIdx.x] = (uint8_t)byte;
      }
    }
    if (kBlock == 128 && tid == 0) scales[(int64_t)tb * a.out.spitch + blockIdx.x] = (uint8_t)whole;
  }

  if constexpr (kCols) {
    uint8_t* codes = const_cast<uint8_t*>(a.out_t.codes) + z * a.out_t.code_stride;
    uint8_t* scales = const_cast<uint8_t*>(a.out_t.scales) + z * a.out_t.scale_stride;
    uint32_t pair[4];                                // two columns' largest magnitudes, then their bytes
    if constexpr (kBlock == 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pair[j] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) pair[j] = max16(pair[j], mag16(v[i][j]));
        pair[j] = max16(pair[j], (uint32_t)__shfl_xor((int)pair[j], 16));
        pair[j] = max16(pair[j], (uint32_t)__shfl_xor((int)pair[j], 32));
      }
      if ((rg & 3) == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) most[wave][4 * cg + j] = pair[j];
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = 4 * cg + j;
        const uint32_t m = max16(max16(most[0][k], most[1][k]), max16(most[2][k], most[3][k]));
        pair[j] = byte_of(m & 0xffffu) | (byte_of(m >> 16) << 16);
        if (rg == 0) {
          if (c + 2 * j < a.cols) scales[(int64_t)(c + 2 * j) * a.out_t.spitch + tb] = (uint8_t)pair[j];
          if (c + 2 * j + 1 < a.cols) scales[(int64_t)(c + 2 * j + 1) * a.out_t.spitch + tb] = (uint8_t)(pair[j] >> 16);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) pair[j] = whole | (whole << 16);
      if (tid == 0) scales[(int64_t)blockIdx.x * a.out_t.spitch + tb] = (uint8_t)whole;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t byte = j & 1 ? pair[j >> 1] >> 16 : pair[j >> 1] & 0xffffu;
      const float f = fp8_scale(byte);
      const uint32_t pick = j & 1 ? 0x07060302u : 0x05040100u;       // column j of two rows
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(v[2 * i + 1][j >> 1], v[2 * i][j >> 1], pick);
      u32x2 q = {fp8_code4<T>(w[0], w[1], f), fp8_code4<T>(w[2], w[3], f)};
      if (byte == 255) q = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
      *reinterpret_cast<u32x2*>(tile + (8 * cg + j) * 128 + 8 * (rg ^ cg)) = q;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = 32 * q + (tid >> 3), u = 2 * (tid & 7);
      const u32x2 lo = *reinterpret_cast<const u32x2*>(tile + k * 128 + 8 * (u ^ (k >> 3)));
      const u32x2 hi = *reinterpret_cast<const u32x2*>(tile + k * 128 + 8 * ((u + 1) ^ (k >> 3)));
      if (c0 + k < a.cols)
        *reinterpret_cast<u32x4*>(codes + (int64_t)(c0 + k) * a.out_t.pitch + (int64_t)tb * 128 + 8 * u) =
            u32x4{lo.x, lo.y, hi.x, hi.y};
    }
  }
}

// Rows only, a scale a row: 16 rows of 128 entries a workgroup, a piece a thread (us, so / by a workgroup of 128
// rows: 1 x 4096 2.4 / 4.1, 2048 x 11008 12.2 / 14.2; 5.5 TB/s).
template <class T>
__global__ void __launch_bounds__(256) k_fp8_quantize_rows(const Fp8QuantArgs a, const int wide) {
  const int cg = threadIdx.x & 15, c = blockIdx.x * 128 + 8 * cg;
  const int r = blockIdx.y * 16 + (threadIdx.x >> 4);
  const int64_t z = blockIdx.z, at = (z * a.rows + r) * a.row_stride + c;
  float v[8];
  if (r < a.rows && wide && c + 8 <= a.cols) {
    load8<T>(a.X, at, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (r < a.rows && c < a.cols) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < a.cols) v[j] = widen<T>(a.X, at + j);
    }
  }
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = umax(m, mag(v[j]));
  const uint32_t byte = fp8_scale_byte(row16_max(m));
  const float f = fp8_inverse(byte);
  u32x2 q = {fp8_four(v[0] * f, v[1] * f, v[2] * f, v[3] * f), fp8_four(v[4] * f, v[5] * f, v[6] * f, v[7] * f)};
  if (byte == 255) q = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
  if (r >= a.rows) return;
  *reinterpret_cast<u32x2*>(const_cast<uint8_t*>(a.out.codes) + z * a.out.code_stride + (int64_t)r * a.out.pitch + c) = q;
  if (cg == 0)
    const_cast<uint8_t*>(a.out.scales)[z * a.out.scale_stride + (int64_t)r * a.out.spitch + blockIdx.x] = (uint8_t)byte;
}

template <class T>
hipError_t quantize(const Fp8QuantArgs& a, hipStream_t s) {
  const int64_t tiles = a.starts ? most_tiles(a.rows, a.groups, 128) : (a.rows + 127) / 128;
  if (tiles < 1) return hipSuccess;
  if (tiles > 65535) return hipErrorNotSupported;
  const dim3 grid((unsigned)((a.cols + 127) / 128), (unsigned)tiles, (unsigned)a.count);
  constexpr int E = std::is_same<T, F32In>::value ? 4 : 2;
  const int wide = (reinterpret_cast<uintptr_t>(a.X) & 15) == 0 && a.row_stride * E % 16 == 0;
  const bool r = a.out.codes, c = a.out_t.codes, big = (r ? a.out : a.out_t).shift == 7;
  if (r && !c && !big && !a.starts && (a.rows + 15) / 16 <= 65535) {   // (what a grid's second axis holds)
    const dim3 few((unsigned)((a.cols + 127) / 128), (unsigned)((a.rows + 15) / 16), (unsigned)a.count);
    hipLaunchKernelGGL(k_fp8_quantize_rows<T>, few, dim3(256), 0, s, a, wide);
    return hipGetLastError();
  }
#define SPL_Q(R, C, B)                                                                    \
  if constexpr (E == 4)                                                                   \
    hipLaunchKernelGGL((k_fp8_quantize<T, R, C, B>), grid, dim3(256), 0, s, a, wide);     \
  else                                                                                    \
    hipLaunchKernelGGL((k_fp8_quantize16<T, R, C, B>), grid, dim3(256), 0, s, a, wide)
  if (r && c && big) {
    SPL_Q(true, true, 128);
  } else if (r && c) {
    SPL_Q(true, true, 1);
  } else if (r && big) {
    SPL_Q(true, false, 128);
  } else if (r) {
    SPL_Q(true, false, 1);                           // rows of groups, or more than the kernel above is launched for
  } else if (big) {
    SPL_Q(false, true, 128);
  } else {
    SPL_Q(false, true, 1);
  }
#undef SPL_Q
  return hipGetLastError();
}

// out = code * 2^e, one rounding: a thread an entry's group of 8, stored one by one (rows of any length): 11008 x 4096 to bf16
// 56 us, 2.4 TB/s.
template <class T>
__global__ void __launch_bounds__(256) k_fp8_dequantize(const Fp8View m, int64_t cols, int64_t first, int64_t groups, void* out) {
  const int64_t i = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= groups) return;
  const int64_t per = (cols + 7) / 8, row = i / per, c = 8 * (i - row * per);
  const int64_t z = row / m.rows, r = row - z * m.rows;
  const u32x2 q = *reinterpret_cast<const u32x2*>(m.codes + z * m.code_stride + r * m.pitch + c);
  const uint32_t byte = m.scales[z * m.scale_stride + (r >> m.shift) * m.spitch + c / 128];
  const float f = byte == 255 ? __uint_as_float(0x7fc00000u) : (byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23));
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (c + j >= cols) break;
    const uint32_t w = j < 4 ? q.x : q.y;
    const float v = __builtin_amdgcn_cvt_f32_fp8((int)(w >> (8 * (j & 3))), 0) * f;
    const int64_t at = row * cols + c + j;
    if constexpr (std::is_same<T, F32In>::value)
      static_cast<float*>(out)[at] = v;
    else
      static_cast<uint16_t*>(out)[at] = T::from_f32(v);
  }
}

// Zeros into the rows of y [rows][row bytes, a multiple of 2] before the first group and behind the last: where starts do not
// fall, those in between all have a group; where they do, into every row.  Two runs of 16-bit words, 8 of them a thread
// at a time; where every row has a group (the usual call) a workgroup reads starts and leaves: 2 us between other launches.
__global__ void __launch_bounds__(256) k_fp8_clear_rest(const int32_t* starts, const int groups, const int rows, uint16_t* y,
                                                        const int64_t width) {
  int falls = 0;
  for (int g = threadIdx.x; g < groups; g += 256) falls |= starts[g] > starts[g + 1];
  falls = __syncthreads_or(falls);
  const auto bound = [&](int v) { return (int64_t)(v < 0 ? 0 : (v > rows ? rows : v)); };
  const int64_t all = rows * width, head = falls ? all : bound(starts[0]) * width, tail = falls ? all : bound(starts[groups]) * width;
  const auto clear = [&](int64_t from, int64_t to) {   // words [from, to)
    const int64_t each = (int64_t)gridDim.x * 256 * 8;
    for (int64_t i = from / 8 * 8 + 8 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < to; i += each) {
      if (i >= from && i + 8 <= to) {
        *reinterpret_cast<u32x4*>(y + i) = u32x4{0u, 0u, 0u, 0u};
      } else {
        for (int64_t k = i < from ? from : i; k < i + 8 && k < to; ++k) y[k] = 0;
      }
    }
  };
  clear(0, head);
  clear(tail, all);
}

}  // namespace

hipError_t launch_fp8_clear_rest(const int32_t* starts, int32_t groups, int64_t rows, int64_t width, void* y, hipStream_t s) {
  const int64_t blocks = (rows * width + 2047) / 2048, most = 2 * device_cus();
  hipLaunchKernelGGL(k_fp8_clear_rest, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, starts, (int)groups,
                     (int)rows, static_cast<uint16_t*>(y), width);
  return hipGetLastError();
}

hipError_t launch_fp8_quantize(const Fp8QuantArgs& a, int32_t dtype, hipStream_t s) {
  if (dtype == SPL_F32) return quantize<F32In>(a, s);
  return dtype == SPL_BF16 ? quantize<Bf16>(a, s) : quantize<F16>(a, s);
}

hipError_t launch_fp8_dequantize(const Fp8View& m, int64_t cols, int64_t count, int32_t dtype, void* out, hipStream_t s) {
  const int64_t groups = count * m.rows * ((cols + 7) / 8), most = ((int64_t)1 << 24) - 1;   // workgroups of a launch
  for (int64_t first = 0; first < groups; first += 256 * most) {
    const int64_t blocks = (groups - first + 255) / 256;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (dtype == SPL_F32)
      hipLaunchKernelGGL(k_fp8_dequantize<F32In>, grid, dim3(256), 0, s, m, cols, first, groups, out);
    else if (dtype == SPL_BF16)
      hipLaunchKernelGGL(k_fp8_dequantize<Bf16>, grid, dim3(256), 0, s, m, cols, first, groups, out);
    else
      hipLaunchKernelGGL(k_fp8_dequantize<F16>, grid, dim3(256), 0, s, m, cols, first, groups, out);
  }
  return hipGetLastError();
}

}  // namespace spl
