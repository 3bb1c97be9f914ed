// Products of 8-bit floats for few rows, for gfx950: a workgroup streams 16 rows
// of W past up to 64 rows of X.
//
// Its waves share the sum, a run of blocks each: a wave loads 16 rows x 128
// columns of W straight into the operand of one scaled matrix instruction (two
// requests of 16 bytes a lane, 64 neighbouring bytes of a row by 4 lanes), and
// one for each 16 rows of X.  Partial sums are added in LDS, in the waves' order.
// Rows of X may also come in 16 bits: a lane then has 32 of a block's 128
// entries, the largest magnitude is found by two lane moves, and the codes are
// those of k_fp8_quantize.
#include <type_traits>

#include "fp8_tile.h"

namespace spl {
namespace {

constexpr int kWaves = 8;

// 16 entries of a row in 16 bits from column c on, zeros past the last.
template <class T>
__device__ __forceinline__ void load16(const uint16_t* row, int c, int cols, bool wide, float (&v)[16]) {
  if (wide && c + 16 <= cols) {
    const u32x4 p = *reinterpret_cast<const u32x4*>(row + c), q = *reinterpret_cast<const u32x4*>(row + c + 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = T::to_f32(p[j] & 0xffffu), v[2 * j + 1] = T::to_f32(p[j] >> 16);
      v[8 + 2 * j] = T::to_f32(q[j] & 0xffffu), v[9 + 2 * j] = T::to_f32(q[j] >> 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = c + j < cols ? T::to_f32(row[c + j]) : 0.f;
  }
}

struct Codes {};                                // X is quantized already

template <class T, int MT, bool kExact>
__global__ void __launch_bounds__(64 * kWaves) k_fp8_stream(const Fp8GemmArgs a, const int wide) {
  constexpr bool kCodes = std::is_same<T, Codes>::value;
  __shared__ f32x4 sums[kWaves][MT][64];
  const Fp8Part p = fp8_part(a, 16 * MT, blockIdx.y, blockIdx.z);
  if (p.none) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int fr = lane & 15, fg = lane >> 4;
  const int64_t n0 = 16 * (int64_t)blockIdx.x;
  const int64_t wr = n0 + fr < a.N ? n0 + fr : a.N - 1;             // rows past the last repeat it and are not stored
  const uint8_t* wp = a.w.codes + p.w_codes + wr * a.w.pitch + 16 * fg;
  const uint8_t* ws = a.w.scales + p.w_scales + (wr >> a.w.shift) * a.w.spitch;
  const uint8_t* xp[MT];
  const uint8_t* xs[MT];
  const uint16_t* xh[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    int64_t m = p.m0 + 16 * j + fr;
    m = m < p.mend ? m : p.mend - 1;
    xp[j] = a.x.codes + m * a.x.pitch + 16 * fg;
    xs[j] = a.x.scales + (m >> a.x.shift) * a.x.spitch;
    xh[j] = static_cast<const uint16_t*>(a.x16) + m * a.x16_stride;
  }
  const int per = (p.k1 - p.k0 + kWaves - 1) / kWaves;
  const int b0 = p.k0 + wave * per, b1 = b0 + per < p.k1 ? b0 + per : p.k1;
  f32x4 acc[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int b = b0; b < b1; ++b) {
    const u32x4 a0 = *reinterpret_cast<const u32x4*>(wp + 128 * (int64_t)b);
    const u32x4 a1 = *reinterpret_cast<const u32x4*>(wp + 128 * (int64_t)b + 64);
    const uint32_t sa = ws[b];
    Wide8 aw;
    if constexpr (kExact) aw = fp8_widen32(a0, a1, sa);
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      u32x4 x0, x1;
      uint32_t sb;
      if constexpr (kCodes) {
        x0 = *reinterpret_cast<const u32x4*>(xp[j] + 128 * (int64_t)b);
        x1 = *reinterpret_cast<const u32x4*>(xp[j] + 128 * (int64_t)b + 64);
        sb = xs[j][b];
      } else {
        float u[16], v[16];
        load16<T>(xh[j], 128 * b + 16 * fg, a.cols, wide, u);
        load16<T>(xh[j], 128 * b + 64 + 16 * fg, a.cols, wide, v);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          m = umax(m, umax(__float_as_uint(u[i]) & 0x7fffffffu, __float_as_uint(v[i]) & 0x7fffffffu));
        m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
        m = umax(m, (uint32_t)__shfl_xor((int)m, 32));
        sb = fp8_scale_byte(m);
        const float f = fp8_inverse(sb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x0[i] = fp8_four(u[4 * i] * f, u[4 * i + 1] * f, u[4 * i + 2] * f, u[4 * i + 3] * f);
          x1[i] = fp8_four(v[4 * i] * f, v[4 * i + 1] * f, v[4 * i + 2] * f, v[4 * i + 3] * f);
        }
        if (sb == 255) x0 = x1 = u32x4{0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
      }
      if constexpr (kExact)
        acc[j] = fp8_mfma_wide(aw, fp8_widen32(x0, x1, sb), acc[j]);
      else
        acc[j] = fp8_mfma(a0, a1, x0, x1, acc[j], sa, sb);
    }
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) sums[wave][j][lane] = acc[j];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < (MT + kWaves - 1) / kWaves; ++q) {
    const int j = wave + kWaves * q;
    if (j >= MT) break;
    f32x4 v = sums[0][j][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][j][lane];
    const int64_t m = p.m0 + 16 * j + fr;
    if (m < p.mend) fp8_store4(a, m, n0 + 4 * fg, v, p.y);
  }
}

template <class T, bool kExact>
hipError_t stream(const Fp8GemmArgs& a, int wide, hipStream_t s) {
  const int mt = a.M <= 16 ? 1 : (a.M <= 32 ? 2 : 4);
  const int64_t tiles = fp8_row_tiles(a, 16 * mt);
  if (tiles > 65535) return hipErrorNotSupported;
  const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)tiles, a.mode == kFp8Sum ? (unsigned)a.groups : 1u);
  if (mt == 1)
    hipLaunchKernelGGL((k_fp8_stream<T, 1, kExact>), grid, dim3(64 * kWaves), 0, s, a, wide);
  else if (mt == 2)
    hipLaunchKernelGGL((k_fp8_stream<T, 2, kExact>), grid, dim3(64 * kWaves), 0, s, a, wide);
  else
    hipLaunchKernelGGL((k_fp8_stream<T, 4, kExact>), grid, dim3(64 * kWaves), 0, s, a, wide);
  return hipGetLastError();
}
template <class T>
hipError_t by_type(const Fp8GemmArgs& a, int wide, hipStream_t s) {
  return a.dtype == SPL_F32 ? stream<T, true>(a, wide, s) : stream<T, false>(a, wide, s);
}

}  // namespace

hipError_t launch_fp8_stream(const Fp8GemmArgs& a, hipStream_t s) {
  if (!a.x16) return by_type<Codes>(a, 0, s);
  const int wide = (reinterpret_cast<uintptr_t>(a.x16) & 15) == 0 && a.x16_stride % 8 == 0;
  return a.x16_dtype == SPL_BF16 ? by_type<Bf16>(a, wide, s) : by_type<F16>(a, wide, s);
}

}  // namespace spl
