// Shared by the kernels of the 8-bit float linears and of the optimizer step
// (not part of the ABI): the format's geometry, its conversions, and what the
// launchers take.
#pragma once

#include "spl_common.h"

namespace spl {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// A matrix of the format as kernels take it (one of `count`: the strides lead to the others).
struct Fp8View {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t rows;
  int64_t code_stride, scale_stride;            // bytes from one matrix to the next
  int32_t pitch, spitch;                        // bytes of a row of codes, of a row of scales
  int32_t shift;                                // rows per scale: 1 << shift
};
inline __host__ __device__ int64_t fp8_pitch(int64_t cols) { return (cols + 127) / 128 * 128; }
inline __host__ __device__ int64_t fp8_spitch(int64_t cols) { return (fp8_pitch(cols) / 128 + 3) / 4 * 4; }
inline int64_t fp8_scale_rows(int64_t rows, int32_t block) { return (rows + block - 1) / block; }
inline Fp8View fp8_view(const spl_fp8_matrix& m) {
  Fp8View v;
  v.codes = static_cast<const uint8_t*>(m.codes);
  v.scales = static_cast<const uint8_t*>(m.scales);
  v.rows = m.rows;
  v.pitch = (int32_t)fp8_pitch(m.cols);
  v.spitch = (int32_t)fp8_spitch(m.cols);
  v.shift = m.block == 128 ? 7 : 0;
  v.code_stride = m.rows * v.pitch;
  v.scale_stride = fp8_scale_rows(m.rows, m.block) * v.spitch;
  return v;
}

// The scale byte of a block whose largest magnitude has these bits: e + 127
// of the least e >= -127 with amax <= 448 2^e (448 = 1.75 2^8, so the fraction
// decides whether the exponent 8 below amax's is enough); 255 for infinity or NaN.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t amax) {
  const int e = (int)(amax >> 23);
  const int b = e - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e == 255 ? 255u : (uint32_t)(b > 0 ? b : 0);
}
// 2^(127 - byte), the inverse of the scale (bytes up to 247 occur).
__device__ __forceinline__ float fp8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// Two values of at most 448 to codes, in the low or high half of `old`.
template <bool kHigh>
__device__ __forceinline__ uint32_t fp8_pair(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, kHigh);
}
__device__ __forceinline__ uint32_t fp8_four(float a, float b, float c, float d) {
  return fp8_pair<true>(c, d, fp8_pair<false>(a, b, 0u));
}

// Two values of 16 bits in a word: the larger magnitudes of two words; four values, divided by the scale of a byte (bytes up
// to 247 occur), to codes.  Exact powers of two, so the codes are those of the fp32 way.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ uint32_t mag16(uint32_t a) { return a & 0x7fff7fffu; }
__device__ __forceinline__ float fp8_scale(uint32_t byte) { return byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23); }
template <class T>
__device__ __forceinline__ uint32_t fp8_code4(uint32_t a, uint32_t b, float scale) {
  s16x2 z = {0, 0};
  if constexpr (T::code == SPL_BF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(z, __builtin_bit_cast(bf16x2, a), scale, false);
    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(z, __builtin_bit_cast(bf16x2, b), scale, true);
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(z, __builtin_bit_cast(f16x2, a), scale, false);
    z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(z, __builtin_bit_cast(f16x2, b), scale, true);
  }
  return __builtin_bit_cast(uint32_t, z);
}

// The largest of a value over the 16 lanes of a row (unsigned compares: magnitudes' bits).
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t row16_max(uint32_t x) {
  x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));   // row_ror:1
  x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));   // row_ror:2
  x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));   // row_ror:4
  x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));   // row_ror:8
  return x;
}

// Groups of rows, starts[0 .. groups], of which group g's tiles of `size` rows
// are counted after those of the groups before it.  A wave asks together; the
// answer is the same in its lanes.
struct Segment {
  int group;                                    // -1: none
  int row;                                      // the first row of tile t
  int end;                                      // the group's end
  int tile;                                     // tiles before the group
};
__device__ __forceinline__ void segment_rows(const int32_t* starts, int64_t g, int rows, int& a, int& b) {
  a = starts[g], b = starts[g + 1];
  a = a < 0 ? 0 : (a > rows ? rows : a);
  b = b < a ? a : (b > rows ? rows : b);
}
// The group that tile t belongs to.
__device__ __forceinline__ Segment find_tile(const int32_t* starts, int groups, int rows, int size, int t) {
  const int lane = (int)lane_id();
  uint32_t before = 0;
  for (int base = 0; base < groups; base += 64) {
    int a = 0, b = 0;
    if (base + lane < groups) segment_rows(starts, base + lane, rows, a, b);
    const uint32_t mine = (uint32_t)(b - a + size - 1) / (uint32_t)size;
    const uint32_t incl = wave_inclusive_scan(mine) + before;
    const uint64_t past = __ballot(incl > (uint32_t)t);
    if (past) {
      const int l = __builtin_ctzll(past);
      Segment s;
      s.group = base + l;
      s.tile = __builtin_amdgcn_readlane((int)(incl - mine), l);
      s.row = __builtin_amdgcn_readlane(a, l) + (t - s.tile) * size;
      s.end = __builtin_amdgcn_readlane(b, l);
      return s;
    }
    before = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
  }
  return Segment{-1, 0, 0, 0};
}
// Where group g begins among the tiles, in `tile`; its rows [row, end).
__device__ __forceinline__ Segment find_group(const int32_t* starts, int g, int rows, int size) {
  const int lane = (int)lane_id();
  uint32_t before = 0;
  for (int base = 0; base < g; base += 64) {
    int a = 0, b = 0;
    if (base + lane < g) segment_rows(starts, base + lane, rows, a, b);
    before += (uint32_t)__builtin_amdgcn_readlane(
        (int)wave_inclusive_scan((uint32_t)(b - a + size - 1) / (uint32_t)size), 63);
  }
  Segment s;
  s.group = g, s.tile = (int)before;
  segment_rows(starts, g, rows, s.row, s.end);
  return s;
}
// Tiles that `groups` groups of `rows` rows in all have at most.
inline int64_t most_tiles(int64_t rows, int64_t groups, int64_t size) {
  return (rows + (size - 1) * (rows < groups ? rows : groups)) / size;
}

struct Fp8QuantArgs {
  const void* X;
  int64_t row_stride;
  int64_t rows, cols, count;
  const int32_t* starts;                        // NULL: none
  int32_t groups;
  Fp8View out, out_t;                           // codes NULL: not wanted
};
hipError_t launch_fp8_quantize(const Fp8QuantArgs& a, int32_t dtype, hipStream_t s);
// Zeros into the rows of y [rows][width] (16-bit words, 16-byte aligned) that no group has; in all where starts fall.
hipError_t launch_fp8_clear_rest(const int32_t* starts, int32_t groups, int64_t rows, int64_t width, void* y, hipStream_t s);
hipError_t launch_fp8_dequantize(const Fp8View& m, int64_t cols, int64_t count, int32_t dtype, void* out, hipStream_t s);

// How the products' rows are grouped.
enum { kFp8Plain = 0, kFp8Rows = 1, kFp8Sum = 2 };   // not; X's rows, a matrix each; the sum's columns, a result each
struct Fp8GemmArgs {
  Fp8View w, x;                                 // N and M rows
  void* y;
  int64_t M, N;
  int32_t blocks;                               // of 128 columns: the whole sum's, or (kFp8Sum) the most there can be
  int32_t dtype;                                // of y
  int32_t mode;
  int32_t splits;                               // of the sum (set by the launcher)
  int32_t first_tile;                           // of rows, of this launch (set by the launcher)
  const int32_t* starts;
  int32_t groups;
  int32_t tokens;                               // kFp8Sum: the rows that starts counts
  const void* x16;                              // rows to be quantized by the kernel itself, or NULL
  int64_t x16_stride;
  int32_t x16_dtype;
  int32_t cols;                                 // of x16
  void* partial;                                // fp8_partial_bytes, or NULL where that is 0
};
hipError_t launch_fp8_gemm(const Fp8GemmArgs& a, hipStream_t s);
// The kernel that it launches, by the numbers of spl_linear_fp8_kernel.
enum {
  kStream16 = 1, kStream32 = 2, kStream32x32 = 3, kRows16 = 4, kRows16x32 = 5, kRows32 = 6, kEightWaves = 8,
  kTile64 = 16, kTile128 = 17, kTileMiddle = 18, kTileLarge = 19, kTileMixed = 20, kTileWide = 21, kTileSplit = 22
};
int32_t fp8_kernel(const Fp8GemmArgs& a);
// Scratch of a plain product of codes whose sum is split over workgroups: fp32 [splits][M][N]; 0: it is not.  The same for
// every type of y.
int64_t fp8_partial_bytes(int64_t M, int64_t N, int32_t blocks);
// Whether the kernel for few rows quantizes rows of 16 bits itself, which every workgroup of 16 or 32 rows of W does anew,
// or a launch before it does.  us in a graph, weights from memory, fused / two launches (a call of its own costs the host 7.8 /
// 12.3 us, which is why what is near is fused).  A matrix: by one row 4096 x 4096 7.8 / 8.9, 8192 x 2048 7.4 / 8.3, 11008 x 4096
// 14.7 / 13.9 (13.5 / 13.7 with weights in the cache), 9000 x 6000 19.8 / 18.2, 8192 x 8192 19.2 / 17.6, 32000 x 4096 33 / 29; by
// 16 rows 8192 x 2048 7.7 / 9.9, 4096 x 4096 9.7 / 10.0, 1024 x 8192 14.2 / 13.1, 11008 x 4096 20.6 / 19.5; 512 x 11008
// 17.5 / 15.0; by 24 1111 x 1000 6.3 / 7.6, 2048 x 2048 8.0 / 7.5, 1024 x 4096 11.2 / 10.1, 4096 x 4096 12.4 / 11.3; by 32 1111 x
// 1000 6.5 / 8.0, 4096 x 2048 8.9 / 8.5, 4096 x 4096 14.3 / 12.1.
// Experts, (rows) experts x N x cols: (64) 8 x 4096 x 1024 9.9 / 10.9, (600) 64 x 1024 x 1024 18.1 / 21.3, (160) 16 x 2048 x 2048
// 19.3 / 21.9, (64) 8 x 5632 x 2048 23.8 / 24.6 and (85) 27.1 / 22.8, (600) 64 x 1408 x 2048 42.7 / 41.0; of longer sums (64) 16 x
// 1024 x 4096 19.3 / 19.1 and (128) 24.0 / 20.8, (24) 4 x 4096 x 4096 18.0 / 17.4, (40) 8 x 1024 x 8192 22.0 / 19.9.
// Where cols are no multiple of 8, rows one after another are not aligned, and entries are loaded one by one: 1 x 1111 x 1001 6.8 /
// 6.5, 8 x 8192 x 1004 8.8 / 9.0, 1 x 4096 x 2100 13.3 / 7.6, 8 x 4096 x 4100 32.8 / 10.3; (6) 8 x 2048 x 1003 8.9 / 9.8 and (32)
// 13.3 / 10.4, (32) 8 x 5632 x 2050 53 / 24.
inline bool fp8_fused(int64_t M, int64_t N, int64_t cols, int64_t experts) {
  const bool whole = cols % 8 == 0;
  if (!whole && cols > 1024) return false;
  if (experts > 1) {                            // up to so many rows each, where groups are one and a half times the mean
    const int64_t most = !whole ? 3 : (cols > 2048 ? 6 : (N * cols <= ((int64_t)1 << 26) / experts ? 16 : 12));
    return 3 * M <= 2 * most * experts;
  }
  return M <= 32 && M * cols <= (int64_t)1 << 16 && N * cols <= (int64_t)3 << 24 && M * N * cols <= (int64_t)1 << 28;
}

struct AdamwHyper {
  double lr, beta1, beta2, eps;
  int64_t step;
  const int32_t* step_on_device;
  const float* grad_scale;
  uint32_t seed;
};
int64_t adamw_plan_chunks(const spl_adamw_tensor* t, int64_t count);
int64_t adamw_plan_bytes(const spl_adamw_tensor* t, int64_t count);
void adamw_plan_write(const spl_adamw_tensor* t, int64_t count, const spl_adamw_types& types, void* host);
hipError_t launch_adamw(const void* plan, int64_t chunks, const spl_adamw_types& types, const AdamwHyper& h,
                        hipStream_t s);

}  // namespace spl
