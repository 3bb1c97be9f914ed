// Products of 8-bit floats for few rows, for gfx950: a workgroup streams 16 NR rows
// of W past up to 16 MT rows of X.
//
// Its four or eight waves share the sum, a run of blocks each: a wave loads 16 rows x 128
// columns of W straight into the operand of one scaled matrix instruction (two
// requests of 16 bytes a lane, 64 neighbouring bytes of a row by 4 lanes), and
// of X likewise; what several blocks need is requested together, before the first
// of them is multiplied, so that a wave of a 4096-column sum waits for memory
// once.  Partial sums are added in LDS, in the waves' order.
// Rows of X may also come in 16 bits: a lane then has 32 of a block's 128
// entries, the largest magnitude is found by two lane moves, and the codes are
// those of k_fp8_quantize.
//
// Bound by W's bytes where they are many (11008 x 4096 by one row 12.7 us with codes, 3.5 TB/s; 8192 x 8192 by one of bf16 17.7
// with the launch that quantizes it, 3.8 TB/s), by the launch and two trips to memory where they are few (1111 x 1000 3.9).
#include <type_traits>

#include "fp8_tile.h"

namespace spl {
namespace {

struct Codes {};                                // X is quantized already

// A lane's part of a block of X: 32 codes (a quarter's pieces fg and fg + 4), or as many values of 16 bits.
template <class T>
struct Part {
  u32x4 q[std::is_same<T, Codes>::value ? 2 : 4];
};

// 16 entries of a row in 16 bits from column c on, zeros past the last.
__device__ __forceinline__ void load16(const uint16_t* row, int c, int cols, bool wide, u32x4& p, u32x4& q) {
  if (wide && c + 16 <= cols) {
    p = *reinterpret_cast<const u32x4*>(row + c), q = *reinterpret_cast<const u32x4*>(row + c + 8);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t lo = c + 2 * j < cols ? row[c + 2 * j] : 0u, hi = c + 2 * j + 1 < cols ? row[c + 2 * j + 1] : 0u;
      (j < 4 ? p : q)[j & 3] = lo | (hi << 16);
    }
  }
}

// The block's scale byte, and the lane's codes.
template <class T>
__device__ __forceinline__ uint32_t quantize(const Part<T>& v, u32x4& x0, u32x4& x1) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max16(m, mag16(v.q[i][j]));
  m = umax(m & 0xffffu, m >> 16);
  m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
  m = umax(m, (uint32_t)__shfl_xor((int)m, 32));
  const uint32_t byte = fp8_scale_byte(__float_as_uint(T::to_f32(m)));
  const float scale = fp8_scale(byte);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    x0[2 * j] = fp8_code4<T>(v.q[j][0], v.q[j][1], scale), x0[2 * j + 1] = fp8_code4<T>(v.q[j][2], v.q[j][3], scale);
    x1[2 * j] = fp8_code4<T>(v.q[2 + j][0], v.q[2 + j][1], scale), x1[2 * j + 1] = fp8_code4<T>(v.q[2 + j][2], v.q[2 + j][3], scale);
  }
  if (byte == 255) x0 = x1 = u32x4{0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
  return byte;
}

// U: blocks requested together, of kWaves waves.  kEach: waves that a SIMD's registers are to hold.
template <class T, int MT, int NR, int U, int kWaves, int kEach, bool kExact>
__global__ void __launch_bounds__(64 * kWaves, kEach) k_fp8_stream(const Fp8GemmArgs a, const int wide) {
  constexpr bool kCodes = std::is_same<T, Codes>::value;
  __shared__ f32x4 sums[kWaves][NR * MT][64];
  const Fp8Part p = fp8_part(a, 16 * MT, a.first_tile + (int)blockIdx.y, blockIdx.z);
  if (p.none) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int fr = lane & 15, fg = lane >> 4;
  const int64_t n0 = 16 * NR * (int64_t)blockIdx.x;
  const uint8_t* wp[NR];
  const uint8_t* ws[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    int64_t wr = n0 + 16 * i + fr;
    wr = wr < a.N ? wr : a.N - 1;                // rows past the last repeat it and are not stored
    wp[i] = a.w.codes + p.w_codes + wr * a.w.pitch + 16 * fg;
    ws[i] = a.w.scales + p.w_scales + (wr >> a.w.shift) * a.w.spitch;
  }
  const uint8_t* xp[MT];
  const uint8_t* xs[MT];
  const uint16_t* xh[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    int64_t m = p.m0 + 16 * j + fr;
    m = m < p.mend ? m : p.mend - 1;
    if constexpr (kCodes) {
      xp[j] = a.x.codes + m * a.x.pitch + 16 * fg;
      xs[j] = a.x.scales + (m >> a.x.shift) * a.x.spitch;
    } else {
      xh[j] = static_cast<const uint16_t*>(a.x16) + m * a.x16_stride;
    }
  }
  // Places before k0 and from k1 on take a block of the wave's again, with codes of zero for X: a NaN in it is in the sum anyway.
  static_assert(U == 4 || U == 2, "a word's blocks");
  const Fp8Run run = fp8_run(p.k0, p.k1, wave, kWaves);
  const int b0 = run.b0, b1 = run.b1, first = run.first;
  const auto block = [&](int b) { return b < first ? first : (b < b1 ? b : b1 - 1); };
  f32x4 acc[NR][MT];
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int b = b0; b < b1 && first < b1; b += U) {
    // X first: it is near, and in 16 bits it is quantized while W is on its way
    Part<T> x[U][MT];
    Part<Codes> w[U][NR];
    uint32_t sw[NR], sx[MT];
    const int word = b & ~3;                     // (a place past the word is not of the sum)
    if constexpr (kCodes) {
#pragma unroll
      for (int j = 0; j < MT; ++j) sx[j] = *reinterpret_cast<const uint32_t*>(xs[j] + word);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = block(b + u);
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        if constexpr (kCodes) {
          x[u][j].q[0] = *reinterpret_cast<const u32x4*>(xp[j] + 128 * (int64_t)at);
          x[u][j].q[1] = *reinterpret_cast<const u32x4*>(xp[j] + 128 * (int64_t)at + 64);
        } else {
          load16(xh[j], 128 * at + 16 * fg, a.cols, wide, x[u][j].q[0], x[u][j].q[1]);
          load16(xh[j], 128 * at + 64 + 16 * fg, a.cols, wide, x[u][j].q[2], x[u][j].q[3]);
        }
      }
    }
    if constexpr (!kCodes) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NR; ++i) sw[i] = *reinterpret_cast<const uint32_t*>(ws[i] + word);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = block(b + u);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        w[u][i].q[0] = *reinterpret_cast<const u32x4*>(wp[i] + 128 * (int64_t)at);
        w[u][i].q[1] = *reinterpret_cast<const u32x4*>(wp[i] + 128 * (int64_t)at + 64);
      }
    }
    if constexpr (!kCodes) __builtin_amdgcn_sched_barrier(0);
    u32x4 x0[U][MT], x1[U][MT];
    uint32_t sb[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t live = b + u >= p.k0 && b + u < b1 ? ~0u : 0u;   // (a branch here would take the requests along)
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        if constexpr (kCodes)
          x0[u][j] = x[u][j].q[0], x1[u][j] = x[u][j].q[1], sb[u][j] = fp8_scale_at(sx[j], b + u);
        else
          sb[u][j] = quantize<T>(x[u][j], x0[u][j], x1[u][j]);
        x0[u][j] &= live, x1[u][j] &= live, sb[u][j] &= live;
      }
    }
    if constexpr (!kCodes) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t live = b + u >= p.k0 && b + u < b1 ? ~0u : 0u;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const uint32_t sa = fp8_scale_at(sw[i], b + u) & live;      // the matrix instruction takes the low byte
        if constexpr (kExact) {
          const Wide8 v = fp8_widen32(w[u][i].q[0], w[u][i].q[1], sa & 255u);
#pragma unroll
          for (int j = 0; j < MT; ++j)
            acc[i][j] = fp8_mfma_wide(v, fp8_widen32(x0[u][j], x1[u][j], sb[u][j] & 255u), acc[i][j]);
        } else {
#pragma unroll
          for (int j = 0; j < MT; ++j)
            acc[i][j] = fp8_mfma(w[u][i].q[0], w[u][i].q[1], x0[u][j], x1[u][j], acc[i][j], sa, sb[u][j]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) sums[wave][i * MT + j][lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int q = 0; q < (NR * MT + kWaves - 1) / kWaves; ++q) {
    const int f = wave + kWaves * q, i = f / MT, j = f % MT;
    if (f >= NR * MT) break;
    f32x4 v = sums[0][f][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][f][lane];
    const int64_t m = p.m0 + 16 * j + fr;
    if (m < p.mend) fp8_store4(a, m, n0 + 16 * i + 4 * fg, v, p.y);
  }
}

template <class T, int MT, int NR, int U, int W, int E>
hipError_t launch(const Fp8GemmArgs& a, int wide, hipStream_t s) {
  const int64_t tiles = fp8_row_tiles(a, 16 * MT);
  Fp8GemmArgs part = a;
  for (int64_t first = 0; first < tiles; first += 65535) {          // what a grid's second axis holds
    const dim3 grid((unsigned)((a.N + 16 * NR - 1) / (16 * NR)), (unsigned)(tiles - first < 65535 ? tiles - first : 65535),
                    a.mode == kFp8Sum ? (unsigned)a.groups : 1u);
    part.first_tile = (int32_t)first;
    if (a.dtype == SPL_F32)
      hipLaunchKernelGGL((k_fp8_stream<T, MT, NR, U, W, E, true>), grid, dim3(64 * W), 0, s, part, wide);
    else
      hipLaunchKernelGGL((k_fp8_stream<T, MT, NR, U, W, E, false>), grid, dim3(64 * W), 0, s, part, wide);
  }
  return hipGetLastError();
}
template <class T, int MT, int NR, int U, int E>
hipError_t by_sum(const Fp8GemmArgs& a, bool eight, int wide, hipStream_t s) {
  return eight ? launch<T, MT, NR, U, 8, E>(a, wide, s) : launch<T, MT, NR, U, 4, E>(a, wide, s);
}
template <class T>
hipError_t rows16(const Fp8GemmArgs& a, int32_t kernel, bool eight, hipStream_t s) {
  const int wide = (reinterpret_cast<uintptr_t>(a.x16) & 15) == 0 && a.x16_stride % 8 == 0;
  if (kernel == kRows32) return by_sum<T, 2, 1, 2, 4>(a, eight, wide, s);
  if (kernel == kRows16x32) return by_sum<T, 1, 2, 2, 5>(a, eight, wide, s);
  return by_sum<T, 1, 1, 2, 6>(a, eight, wide, s);
}

}  // namespace

// Four waves for up to 16 blocks of 128 columns, which would leave eight of them two or fewer each (us, 4 / 8 waves:
// 5632 x 2048 6.0 / 8.2, 1111 x 1000 3.9 / 5.0, 4096 x 4096 7.6 / 6.5, 4096 x 11008 16.3 / 13.0).
// Rows in 16 bits are quantized by each workgroup anew, which is most of its arithmetic: two blocks of 16 rows of W a
// workgroup where that leaves each CU one, of long sums four, which then end more evenly (us, two / one: 1 x 4096 x 4096, 128
// workgroups of two, 8.8 / 7.8; 16 x 8192 x 2048, 256 of them, 7.9 / 9.1; 1 x 11008 x 2048 9.2 / 9.7; 1 x 32000 x 1000 10.9 /
// 12.7; 1 x 11008 x 4096 15.8 / 14.7; of experts, 16 rows of 8 x 1024 x 1024, 256 of them, 5.0 / 5.6, 32 rows of 8 x 5632 x 2048
// 19.0 / 21.8, 64 rows of 32 x 2048 x 1024 11.2 / 13.9, 24 rows of 8 x 4096 x 4096 23.6 / 26.8).
int32_t fp8_stream_kernel(const Fp8GemmArgs& a) {
  const int32_t eight = a.blocks <= 16 ? 0 : kEightWaves;
  const double each = fp8_rows_each(a);
  if (!a.x16) return eight + (each <= 16 ? kStream16 : (each <= 32 ? kStream32 : kStream32x32));
  const int64_t wgs = (a.N + 31) / 32 * (a.mode == kFp8Rows ? (a.M < a.groups ? a.M : a.groups) : 1);
  return eight + (each > 16 ? kRows32 : (wgs >= (a.blocks <= 16 ? 1 : 4) * device_cus() ? kRows16x32 : kRows16));
}

hipError_t launch_fp8_stream(const Fp8GemmArgs& a, int32_t kernel, hipStream_t s) {
  const bool eight = kernel >= kEightWaves;
  kernel -= eight ? kEightWaves : 0;
  if (a.x16) return a.x16_dtype == SPL_BF16 ? rows16<Bf16>(a, kernel, eight, s) : rows16<F16>(a, kernel, eight, s);
  if (kernel == kStream16) return by_sum<Codes, 1, 1, 4, 6>(a, eight, 0, s);
  if (kernel == kStream32) return by_sum<Codes, 2, 1, 4, 4>(a, eight, 0, s);
  return by_sum<Codes, 2, 2, 4, 2>(a, eight, 0, s);
}

}  // namespace spl
