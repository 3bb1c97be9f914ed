// Products of 8-bit floats for many rows, for gfx950.
//
// A workgroup of WN x WM waves computes 16 FN WN columns of 16 FM WM rows of X, a wave 16 FN x 16 FM of them.  The sum
// advances a block of 128 columns a stage, which is one scaled matrix instruction for every 16 x 16 outputs.  Both
// operands go from memory straight into LDS, a ring of R stage buffers of 128-byte rows whose 16-byte piece c sits at
// c ^ (row % 8); the rows' scale bytes likewise, four stages a word.  A wave has its FM fragments of X in registers and takes
// those of W two at a time, the next two on their way; behind the last product of a fragment of X the next stage's is read
// in its place.  The one barrier of a stage stands before its last two fragments of W: the buffer has been read by then and
// is refilled, and the next stage's has been waited for (counted, so that later requests stay on their way).
//
// Bound by the matrix instructions and, beside them, by LDS and by what a round starts and ends with: 8192 x 8192 x 8192 437
// to 448 us (2.45 to 2.5 PFLOP/s), 2048 x 11008 x 4096 99 to 103, 2048 x 4096 x 4096 37, fp32 results 4096 x 4096 x 2048 67.
#include <math.h>

#include <type_traits>

#include "fp8_tile.h"

namespace spl {
namespace {

constexpr uint32_t kOob = 0x80000000u;

__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t src, unsigned char* dst, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, voff, soff, 0, 0);
}
// At most N of this wave's vector-memory requests remain, and no LDS read.
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | ((N >> 4) << 14));
}
__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct alignas(32) Codes32 {
  u32x4 lo, hi;
};

// The same instruction with its sums in accumulator registers, which the compiler does not keep there by itself when
// they are all of them (it moves and spills).  What it cannot know of this text is kept by hand: two wait states after
// a vector instruction that may have written an operand (s_nop 1), none between instructions on other sums, and
// settle() before the sums are read.
__device__ __forceinline__ void mfma_acc(const i32x8& a, const i32x8& b, f32x4& c, uint32_t sa, uint32_t sb) {
  asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
               : "+a"(c)
               : "v"(a), "v"(b), "v"(sa), "v"(sb));
}
template <int FN, int FM>
__device__ __forceinline__ void settle(f32x4 (&acc)[FN][FM]) {
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" : "+a"(acc[0][0]));
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) asm volatile("" : "+a"(acc[i][j]));
}

constexpr int tile_waves(int FN, int FM) { return FN * FM > 32 ? 1 : 2; }   // a SIMD's waves that the registers are held to

// Tile w of tn x tm (columns from nbase on).  T: of the results; kExact: summed by bf16 instructions.
template <class T, bool kExact, int FN, int FM, int WN, int WM, int R>
__device__ __forceinline__ void tile_body(const Fp8GemmArgs& a, int w, int tn, int tm, int64_t nbase) {
  constexpr int NW = WN * WM, BN = 16 * FN * WN, BM = 16 * FM * WM;
  constexpr int PW = BN / 8 / NW, PX = BM / 8 / NW;   // requests of 8 rows a wave and stage
  constexpr int SZ = (BN + BM) * 128, RQ = PW + PX;
  static_assert(BN % (8 * NW) == 0 && BM % (8 * NW) == 0, "whole requests");
  extern __shared__ __align__(16) unsigned char dsm[];
  // the XCDs (blockIdx % 8) take contiguous runs of tiles, four row tiles to a column of column tiles
  int bn, bm;
  {
    const int total = tm * tn;
    const int q = total / 8, r = total % 8, x = w % 8, i = w / 8;
    const int t = x * q + (x < r ? x : r) + i;
    const int gsz = 4 * tn, grp = t / gsz, h = tm - grp * 4 < 4 ? tm - grp * 4 : 4, in = t - grp * gsz;
    bm = grp * 4 + in % h;
    bn = in / h;
  }
  const Fp8Part p = fp8_part(a, BM, a.first_tile + bm, blockIdx.z);
  if (p.none) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wn = wave % WN, wm = wave / WN, fr = lane & 15, fg = lane >> 4;
  const int64_t n0 = nbase + (int64_t)bn * BN;
  const int Nr = (int)(a.N - n0 < BN ? a.N - n0 : BN), Mr = p.mend - p.m0 < BM ? p.mend - p.m0 : BM;
  const int nst = p.k1 - p.k0;

  const unsigned char* wbase = a.w.codes + p.w_codes + n0 * a.w.pitch;
  const unsigned char* xbase = a.x.codes + (int64_t)p.m0 * a.x.pitch;
  uint32_t woff[PW], xoff[PX];
  const uint32_t piece = 16u * (uint32_t)((lane & 7) ^ (lane >> 3));
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int row = 8 * (PW * wave + i) + (lane >> 3);
    woff[i] = row < Nr ? (uint32_t)row * (uint32_t)a.w.pitch + piece : kOob;
  }
#pragma unroll
  for (int i = 0; i < PX; ++i) {
    const int row = 8 * (PX * wave + i) + (lane >> 3);
    xoff[i] = row < Mr ? (uint32_t)row * (uint32_t)a.x.pitch + piece : kOob;
  }
  // Request i of a stage, into stage buffer `buf`; stages past the last read through empty descriptors: zeros.
  auto request_codes = [&](int i, int st, int buf) {
    const bool w = i < PW;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<unsigned char*>(w ? wbase : xbase), (short)0, st < nst ? (w ? Nr * a.w.pitch : Mr * a.x.pitch) : 0, 0x00020000);
    const int at = 128 * (p.k0 + st);
    if (w)
      dma16(r, dsm + buf * SZ + (PW * wave + i) * 1024, woff[i], at);
    else
      dma16(r, dsm + buf * SZ + BN * 128 + (PX * wave + i - PW) * 1024, xoff[i - PW], at);
  };
  // The rows' scale bytes, four stages a word, in a ring of four words a row behind the stage buffers: 64 rows a request.
  constexpr int SW = (BN + BM) / 64, SQ = (SW + NW - 1) / NW;
  static_assert(BM % 64 == 0 && BN % 64 == 0, "whole requests");
  const auto scale_request = [&](int i) { return NW * i + wave < SW ? NW * i + wave : SW - 1; };   // the last one again
  const uint8_t* wsc = a.w.scales + p.w_scales + (n0 >> a.w.shift) * a.w.spitch;
  const uint8_t* xsc = a.x.scales + ((int64_t)p.m0 >> a.x.shift) * a.x.spitch;
  uint32_t soff[SQ];
#pragma unroll
  for (int i = 0; i < SQ; ++i) {
    const int q = scale_request(i), row = 64 * (q < BN / 64 ? q : q - BN / 64) + lane;
    if (q < BN / 64)
      soff[i] = row < Nr ? (uint32_t)(row >> a.w.shift) * (uint32_t)a.w.spitch : kOob;
    else
      soff[i] = row < Mr ? (uint32_t)(((p.m0 + row) >> a.x.shift) - (p.m0 >> a.x.shift)) * (uint32_t)a.x.spitch : kOob;
  }
  const int lead = p.k0 & 3;                         // stages from a word's begin to mine
  auto request_scales = [&](int i, int st) {         // the word of stage st, which four stages request (the same bytes)
    const int word = (lead + st) >> 2, at = (p.k0 - lead) + 4 * word;
    const int q = scale_request(i);
    const bool w = q < BN / 64;
    const int rows = w ? ((Nr - 1) >> a.w.shift) + 1 : ((p.m0 + Mr - 1) >> a.x.shift) - (p.m0 >> a.x.shift) + 1;
    const int bytes = at < a.w.spitch ? rows * (w ? a.w.spitch : a.x.spitch) : 0;   // words past a row: zeros
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(w ? wsc : xsc), (short)0, bytes, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(dsm + R * SZ + (word & 3) * (BN + BM) * 4 + 256 * q), 4, soff[i], at, 0, 0);
  };
  constexpr int G = RQ + SQ;                         // a stage's requests
  auto request = [&](int i, int st, int buf) {
    if (i < SQ)
      request_scales(i, st);
    else
      request_codes(i - SQ, st, buf);
  };
  // My rows' scales, of W's fragments, then of X's: the word as it is read, then shifted so that the stage's byte is the
  // low one (the matrix instruction looks at no other).
  uint32_t sc[FN + FM];
  const uint32_t wscale = lds_off(dsm) + R * SZ + 4 * (16 * FN * wn + fr);
  const uint32_t xscale = lds_off(dsm) + R * SZ + 4 * (BN + 16 * FM * wm + fr);
  auto scale_place = [&](int st) { return (uint32_t)((((lead + st) >> 2) & 3) * (BN + BM) * 4); };
  auto read_scale = [&](int i, uint32_t place) {
    sc[i] = i < FN ? lds_load4(wscale + place + 64 * i) : lds_load4(xscale + place + 64 * (i - FN));
  };

  // a row's pieces fg and fg + 4 in a stage buffer
  const uint32_t turn = 16 * (uint32_t)(fg ^ (fr & 7));
  const uint32_t arow = lds_off(dsm) + 128 * (16 * FN * wn + fr), brow = lds_off(dsm) + BN * 128 + 128 * (16 * FM * wm + fr);
  Codes32 A[2][2], B[FM];
  auto read_a = [&](Codes32 (&d)[2], int step, uint32_t off) {
    const uint32_t lo = arow + turn + off, hi = arow + (turn ^ 64u) + off;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      d[i].lo = lds_load16(lo + 2048 * (2 * step + i));
      d[i].hi = lds_load16(hi + 2048 * (2 * step + i));
    }
  };
  auto read_b = [&](int j, uint32_t off) {
    B[j].lo = lds_load16(brow + turn + off + 2048 * j);
    B[j].hi = lds_load16(brow + (turn ^ 64u) + off + 2048 * j);
  };
  f32x4 acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  Wide8 aw[kExact ? 2 : 1], bw[kExact ? FM : 1];
  // the stage's scales of two fragments of W, of a fragment of X (and, for fp32 results, their values)
  auto ready_a = [&](const Codes32 (&w)[2], int step, int shift) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sc[2 * step + i] >>= shift;
      if constexpr (kExact) aw[i] = fp8_widen32(w[i].lo, w[i].hi, sc[2 * step + i] & 255u);
    }
  };
  auto ready_b = [&](int j, int shift) {
    sc[FN + j] >>= shift;
    if constexpr (kExact) bw[j] = fp8_widen32(B[j].lo, B[j].hi, sc[FN + j] & 255u);
  };
  // two fragments of W by fragment j of X
  auto multiply = [&](const Codes32 (&w)[2], int step, int j) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x4& c = acc[2 * step + i][j];
      if constexpr (kExact)
        c = fp8_mfma_wide(aw[i], bw[j], c);
      else if constexpr (FN * FM > 32)
        mfma_acc(__builtin_bit_cast(i32x8, w[i]), __builtin_bit_cast(i32x8, B[j]), c, sc[2 * step + i], sc[FN + j]);
      else
        c = fp8_mfma(w[i].lo, w[i].hi, B[j].lo, B[j].hi, c, sc[2 * step + i], sc[FN + j]);
    }
  };

  // Stage st + R - 1's requests: the first half behind the barrier of stage st - 1, which frees their buffer, the second
  // in the first step of stage st.  At the barrier of stage st those up to stage st + 1 have to be there.
  constexpr int H = G / 2;
  static_assert(R >= 2 && R <= 7 && (R - 2) * G + H < 64, "counted waits; a ring of four words of four stages");
  if (nst > 0) {
#pragma unroll
    for (int i = 0; i < (R - 1) * G + H; ++i) request(i % G, i / G, i / G);
    wait_vm<(R - 2) * G + H>();
    tile_barrier();
#pragma unroll
    for (int i = 0; i < FN + FM; ++i) read_scale(i, scale_place(0));
    read_a(A[0], 0, 0);
#pragma unroll
    for (int j = 0; j < FM; ++j) read_b(j, 0);
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 0) | (3 << 14));   // else the loop would wait here for its own later reads
    int buf = 0;
#pragma unroll 1
    for (int st = 0; st < nst; ++st) {
      const uint32_t here = (uint32_t)(buf * SZ);
      const int shift = 8 * ((lead + st) & 3);
      const int after = buf + 1 == R ? 0 : buf + 1, last = buf == 0 ? R - 1 : buf - 1;
#pragma unroll
      for (int step = 0; step < FN / 2 - 1; ++step) {
        __builtin_amdgcn_sched_barrier(0);
        ready_a(A[step & 1], step, shift);
#pragma unroll
        for (int j = 0; j < FM; ++j) {
          if (step == 0) ready_b(j, shift);
          multiply(A[step & 1], step, j);
          if (j == 0) {                              // behind the first product, which has waited long enough
            __builtin_amdgcn_sched_barrier(0);
            read_a(A[(step + 1) & 1], step + 1, here);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (step == 0) {
#pragma unroll
            for (int i = H + (G - H) * j / FM; i < H + (G - H) * (j + 1) / FM; ++i) request(i, st + R - 1, last);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      wait_vm<(R - 2) * G>();                        // and for my reads of this buffer
      tile_barrier();
      const uint32_t place = scale_place(st + 1);
      ready_a(A[1], FN / 2 - 1, shift);
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        multiply(A[1], FN / 2 - 1, j);
        if (j == 0) {
          __builtin_amdgcn_sched_barrier(0);
          read_a(A[0], 0, (uint32_t)(after * SZ));
#pragma unroll
          for (int i = 0; i < FN - 2; ++i) read_scale(i, place);
          __builtin_amdgcn_sched_barrier(0);
        }
        read_b(j, (uint32_t)(after * SZ));
        read_scale(FN + j, place);
        if (j == FM - 1) read_scale(FN - 2, place), read_scale(FN - 1, place);
#pragma unroll
        for (int i = H * j / FM; i < H * (j + 1) / FM; ++i) request(i, st + R, buf);
      }
      __builtin_amdgcn_sched_barrier(0);
      buf = after;
    }
    if constexpr (FN * FM > 32) settle(acc);
    wait_vm<0>();                                    // no request outlives the workgroup's LDS
  }

  // Results: 16 rows of the wave's at a time through LDS, so that a row's leave as 16-byte pieces.  A lane has columns
  // 4 fg .. 4 fg + 3 of each fragment, row fr; piece c of a row sits at c ^ row.
  constexpr int E = T::code == SPL_F32 ? 4 : 2, CH = 16 * FN * E / 16;   // bytes of a result, pieces of a row
  tile_barrier();                                    // the other waves have read their last stage
  unsigned char* out = dsm + wave * (2 * 16 * CH * 16);
  const int64_t nw = n0 + 16 * FN * wn;
#pragma unroll
  for (int j = 0; j < FM; ++j) {
    unsigned char* half = out + (j & 1) * (16 * CH * 16);
#pragma unroll
    for (int i = 0; i < FN; ++i) {
      const f32x4 v = acc[i][j];
      if constexpr (E == 4) {
        *reinterpret_cast<f32x4*>(half + fr * (CH * 16) + 16 * ((4 * i + fg) ^ (fr & (CH - 1)))) = v;
      } else {
        *reinterpret_cast<u32x2*>(half + fr * (CH * 16) + 16 * ((2 * i + (fg >> 1)) ^ (fr & (CH - 1))) + 8 * (fg & 1)) =
            u32x2{fp8_pack2<T>(v[0], v[1]), fp8_pack2<T>(v[2], v[3])};
      }
    }
    wave_lds_sync();
    const int m = 16 * (FM * wm + j);
    unsigned char* y = static_cast<unsigned char*>(a.y) + (p.y + (p.m0 + m) * a.N + nw) * E;
#pragma unroll
    for (int q = 0; q < 16 * CH / 64; ++q) {
      const int e = 64 * q + lane, row = e / CH, c = e % CH;
      const unsigned char* from = half + row * (CH * 16) + 16 * (c ^ (row & (CH - 1)));
      unsigned char* to = y + (int64_t)row * a.N * E + 16 * c;
      const int have = m + row < Mr ? (int)(a.N - nw < 16 * FN ? a.N - nw : 16 * FN) - c * (16 / E) : 0;
      if (have >= 16 / E) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(from);
        __builtin_memcpy(to, &v, 16);                // (rows of any length: their starts have E bytes' alignment)
      } else {
#pragma unroll 1
        for (int k = 0; k < have; ++k) __builtin_memcpy(to + E * k, from + E * k, E);
      }
    }
  }
}

template <class T, bool kExact, int FN, int FM, int WN, int WM, int R>
__global__ void __launch_bounds__(64 * WN * WM, tile_waves(FN, FM)) k_fp8_tile(const Fp8GemmArgs a, const int tn,
                                                                               const int tm) {
  tile_body<T, kExact, FN, FM, WN, WM, R>(a, (int)blockIdx.x, tn, tm, 0);
}

// `big` tiles of 256 x 256, which fill the chip whole times, then the rest of the columns in tiles of 256 x 128.
template <class T>
__global__ void __launch_bounds__(256, 1) k_fp8_mixed(const Fp8GemmArgs a, const int tnb, const int tmb, const int tn,
                                                      const int tm) {
  const int big = tnb * tmb, w = (int)blockIdx.x;
  if (w < big)
    tile_body<T, false, 8, 8, 2, 2, 2>(a, w, tnb, tmb, 0);
  else
    tile_body<T, false, 8, 4, 2, 2, 2>(a, w - big, tn, tm, (int64_t)tnb * 256);
}

constexpr int tile_lds(int BN, int BM, int R) { return R * (BN + BM) * 128 + 4 * (BN + BM) * 4; }
constexpr int64_t kMostTiles = (int64_t)1 << 22;        // of a launch; more rows' take further ones

template <class T, bool kExact, int FN, int FM, int WN, int WM, int R>
hipError_t launch_tile(const Fp8GemmArgs& a, hipStream_t s) {
  constexpr int BN = 16 * FN * WN, BM = 16 * FM * WM, LDS = tile_lds(BN, BM, R);
  static PerDeviceFlag done;
  auto* kernel = k_fp8_tile<T, kExact, FN, FM, WN, WM, R>;
  const hipError_t e = allow_lds_once(done, kernel, LDS);
  if (e != hipSuccess) return e;
  const int64_t tn = (a.N + BN - 1) / BN, all = fp8_row_tiles(a, BM);   // (N < 2^28: tn is half of kMostTiles at most)
  Fp8GemmArgs part = a;
  for (int64_t first = 0; first < all; first += kMostTiles / tn) {
    const int64_t tm = all - first < kMostTiles / tn ? all - first : kMostTiles / tn;
    const dim3 grid((unsigned)(tn * tm), 1u, a.mode == kFp8Sum ? (unsigned)a.groups : (unsigned)a.splits);
    part.first_tile = (int32_t)first;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * WN * WM), LDS, s, part, (int)tn, (int)tm);
  }
  return hipGetLastError();
}

template <class T>
hipError_t launch_mixed(const Fp8GemmArgs& a, int64_t tnb, hipStream_t s) {
  constexpr int LDS = tile_lds(256, 256, 2);
  static PerDeviceFlag done;
  const hipError_t e = allow_lds_once(done, k_fp8_mixed<T>, LDS);
  if (e != hipSuccess) return e;
  const int64_t tmb = fp8_row_tiles(a, 256), tm = fp8_row_tiles(a, 128), tn = (a.N + 255) / 256 - tnb;
  hipLaunchKernelGGL(k_fp8_mixed<T>, dim3((unsigned)(tnb * tmb + tn * tm)), dim3(256), LDS, s, a, (int)tnb, (int)tmb,
                     (int)tn, (int)tm);
  return hipGetLastError();
}

// How long a call takes, in us, in tiles of one kind: rounds of the chip, each a fixed part and one for each stage, which
// differs where a CU has one workgroup only.  Fitted to launches of 128 to 8192 rows (us; 256 x 256 tiles / 256 x 128 of eight
// waves and three stage buffers / 128 x 128, four stage buffers / 128 x 64): 8192 x 8192 x 8192 437 / 538 / 652 / 714, 2048 x
// 11008 x 4096 107 / - / 126 / 132 (256 x 256, then 256 x 128 of four waves: 99), 2048 x 4096 x 4096 50 / 36.3 / 42.5 / 45.6, 1000 x
// 4096 x 4096 50 / 30 / 23.3 / 25.4, 512 x 4096 x 4096 48 / 29 / 20.7 / 16.1, 4096 rows of 16 experts x 5632 x 2048 104 / 102 / 122 /
// 116; fp32 results, 128 x 256 / 128 x 128 / 128 x 64: 4096 x 4096 x 2048 67 / 69 / 82, 1024 x 1024 x 2048 27 / 20.5 / 15.0.
struct Cost {
  double fixed, full, alone;                         // a stage: with every place taken, with at most one workgroup a CU
  int places;                                        // workgroups of a CU
  double rounds(double tiles, double stages, int cus) const {
    const double room = (double)cus * places, whole = floor(tiles / room), rest = tiles - whole * room;
    return whole * (fixed + full * stages) + (rest <= 0 ? 0 : fixed + (rest <= cus ? alone : full) * stages);
  }
};
constexpr Cost kLarge{12, 1.45, 1.45, 1}, kMiddle{8, 0.88, 0.88, 1}, kRest{9, 0.85, 0.85, 1}, kDeep{6.5, 0.53, 0.53, 1},
    kNarrow{5, 0.6, 0.32, 2};
constexpr Cost kLarge32{8, 1.6, 1.6, 1}, kSmall32{6, 1.75, 0.85, 2}, kNarrow32{5, 1.15, 0.6, 2};

// Tiles and stages of the call, as far as the host can tell: groups are taken as equal, each with half a tile to spare.
double about_tiles(const Fp8GemmArgs& a, int BN, int BM) {
  const double tn = (double)((a.N + BN - 1) / BN);
  if (a.mode != kFp8Rows) return tn * (double)((a.M + BM - 1) / BM) * (a.mode == kFp8Sum ? a.groups : 1);
  const double groups = (double)(a.M < a.groups ? a.M : a.groups);
  return tn * groups * ((double)a.M / groups / BM + 0.5);
}
double about_stages(const Fp8GemmArgs& a) {
  return a.mode == kFp8Sum ? (double)a.tokens / a.groups / 128 + 0.5 : (double)a.blocks;
}

// Workgroups that share a tile's sum, joined by a second launch (3 us and the partial sums): as many as are worth
// it where the tiles of 128 x 64 leave CUs without work.
int splits_of(int64_t M, int64_t N, int32_t blocks) {
  if (M <= 32) return 1;
  const int cus = device_cus();
  const double tiles = (double)((N + 127) / 128) * (double)((M + 63) / 64);
  double best = kNarrow.rounds(tiles, blocks, cus);
  int splits = 1;
  for (int n = 2; n <= 16 && blocks / n >= 4; ++n) {
    const double join = 3 + (double)M * N * 4 * (n + 1) / 4e6;
    const double t = kNarrow.rounds(tiles * n, (double)((blocks + n - 1) / n), cus) + join;
    if (t < 0.9 * best) best = t, splits = n;
  }
  return splits;
}

// The kind of tile; with kTileMixed, `columns` of 256 x 256 tiles.
int32_t tile_kernel(const Fp8GemmArgs& a, int64_t& columns) {
  const int cus = device_cus();
  const double st = about_stages(a), t64 = about_tiles(a, 128, 64), t128 = about_tiles(a, 128, 128);
  if (a.dtype == SPL_F32) {
    const double large = kLarge32.rounds(about_tiles(a, 128, 256), st, cus), small = kSmall32.rounds(t128, st, cus),
                 narrow = kNarrow32.rounds(t64, st, cus);
    if (narrow <= small && narrow <= large) return kTile64;
    return small <= large ? kTile128 : kTileWide;
  }
  const double t256 = about_tiles(a, 256, 256);
  const double large = kLarge.rounds(t256, st, cus), middle = kMiddle.rounds(about_tiles(a, 256, 128), st, cus),
               deep = kDeep.rounds(t128, st, cus), narrow = kNarrow.rounds(t64, st, cus);
  double best = large < middle ? large : middle;
  best = deep < best ? deep : best;
  best = narrow < best ? narrow : best;
  if (a.mode == kFp8Plain && t256 > cus) {             // whole rounds of large tiles, the rest of the columns in middle ones
    const int64_t tm = (a.M + 255) / 256, tn = (a.N + 255) / 256;
    const int64_t tnb = (int64_t)(t256 / cus) * cus / tm;
    const double mixed = kLarge.rounds((double)(tnb * tm), st, cus) +
                         kRest.rounds((double)(tn - tnb) * (double)((a.M + 127) / 128), st, cus);
    if (tnb > 0 && tnb < tn && mixed < best && 2 * tn * tm < kMostTiles) {   // (in one launch)
      columns = tnb;
      return kTileMixed;
    }
  }
  if (best == narrow) return kTile64;
  if (best == deep) return kTile128;
  return best == middle ? kTileMiddle : kTileLarge;
}

template <class T>
hipError_t launch_kind(const Fp8GemmArgs& a, int32_t kind, int64_t columns, hipStream_t s) {
  if constexpr (T::code == SPL_F32) {
    if (kind == kTile64) return launch_tile<T, true, 4, 2, 2, 2, 3>(a, s);
    return kind == kTile128 ? launch_tile<T, true, 4, 4, 2, 2, 2>(a, s) : launch_tile<T, true, 4, 4, 2, 4, 3>(a, s);
  } else {
    if (kind == kTileMixed) return launch_mixed<T>(a, columns, s);
    if (kind == kTile64) return launch_tile<T, false, 4, 2, 2, 2, 3>(a, s);
    if (kind == kTile128) return launch_tile<T, false, 4, 4, 2, 2, 4>(a, s);
    return kind == kTileMiddle ? launch_tile<T, false, 4, 4, 4, 2, 3>(a, s) : launch_tile<T, false, 8, 8, 2, 2, 2>(a, s);
  }
}

// Whether the streaming kernel is the one: up to 32 rows of a matrix; up to 64 where tiles of 128 x 64 would take longer
// (us, streaming / tiles whose sums are not split, 64 rows: 4096 x 4096 11.1 / 16.3, 11008 x 4096 31.1 / 15.8); of groups by
// the sum's length, as tiles end with a round whatever it is (us, streaming / tiles, (rows) experts x N x cols: (16) 8 x 4096 x 1024
// and (64) 32 x 2048 x 1024 11.1 / 8.1 and 16.9 / 14.3, (100) 16 x 4096 x 1408 21.5 / 23.5, (32, 48, 64, 85) 8 x 5632 x 2048 17.6,
// 21.8, 22.8, 25.5 / 20.3, 21.9, 22.1, 20.2, (100) 16 x 2048 x 2048 13.8 / 17.0, (600) 64 x 1408 x 2048 41.5 / 37.9, (160)
// 16 x 1024 x 4096 20.1 / 20.4, (40) 4 x 4096 x 4096 20.6 / 21.0, (80) 8 x 1024 x 8192 23.3 / 36.0).
bool streams(const Fp8GemmArgs& a) {
  const double each = fp8_rows_each(a);
  if (a.mode == kFp8Rows) return a.blocks > 8 && each <= (a.blocks > 16 ? 16 : 10);
  if (each <= 32) return true;
  if (each > 64 || a.mode != kFp8Plain || splits_of(a.M, a.N, a.blocks) > 1) return false;
  const double cus = device_cus(), wgs = (double)((a.N + 31) / 32) * 2 / cus;
  const Cost& narrow = a.dtype == SPL_F32 ? kNarrow32 : kNarrow;
  return 4 + (wgs > 1 ? wgs : 1) * a.blocks * 0.27 < narrow.rounds(about_tiles(a, 128, 64), a.blocks, (int)cus);
}

// The sum of the splits, in their order: 4 results a thread.
template <class T>
__global__ void __launch_bounds__(256) k_fp8_join(const float* partial, int splits, int64_t n, void* y) {
  const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
  if (i >= n) return;
  if (i + 4 <= n && (n & 3) == 0) {
    f32x4 v = *reinterpret_cast<const f32x4*>(partial + i);
    for (int s = 1; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(partial + s * n + i);
    if constexpr (T::code == SPL_F32)
      *reinterpret_cast<f32x4*>(static_cast<float*>(y) + i) = v;
    else
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(y) + i) = u32x2{fp8_pack2<T>(v[0], v[1]), fp8_pack2<T>(v[2], v[3])};
  } else {
    for (int k = 0; k < 4 && i + k < n; ++k) {
      float v = partial[i + k];
      for (int s = 1; s < splits; ++s) v += partial[s * n + i + k];
      if constexpr (T::code == SPL_F32)
        static_cast<float*>(y)[i + k] = v;
      else
        static_cast<uint16_t*>(y)[i + k] = T::from_f32(v);
    }
  }
}

}  // namespace

int64_t fp8_partial_bytes(int64_t M, int64_t N, int32_t blocks) {
  const int splits = splits_of(M, N, blocks);
  return splits > 1 ? 4 * M * N * splits : 0;
}

static int32_t kernel_of(const Fp8GemmArgs& a, int64_t& columns) {
  if (a.x16 || streams(a)) return fp8_stream_kernel(a);
  return a.mode == kFp8Plain && a.partial ? (int32_t)kTileSplit : tile_kernel(a, columns);
}
int32_t fp8_kernel(const Fp8GemmArgs& a) {
  int64_t columns;
  return kernel_of(a, columns);
}

hipError_t launch_fp8_gemm(const Fp8GemmArgs& given, hipStream_t s) {
  Fp8GemmArgs a = given;
  a.splits = 1;
  int64_t columns = 0;
  const int32_t kind = kernel_of(a, columns);
  if (kind < kTile64) return launch_fp8_stream(a, kind, s);
  if (kind == kTileSplit) {
    a.splits = splits_of(a.M, a.N, a.blocks);
    a.y = a.partial;
    hipError_t e = a.dtype == SPL_F32 ? launch_tile<F32Out, true, 4, 2, 2, 2, 3>(a, s) : launch_tile<F32Out, false, 4, 2, 2, 2, 3>(a, s);
    if (e != hipSuccess) return e;
    const int64_t n = a.M * a.N;
    const dim3 grid((unsigned)((n + 1023) / 1024));
    const float* from = static_cast<const float*>(a.partial);
    if (a.dtype == SPL_F32)
      hipLaunchKernelGGL(k_fp8_join<F32Out>, grid, dim3(256), 0, s, from, a.splits, n, given.y);
    else if (a.dtype == SPL_BF16)
      hipLaunchKernelGGL(k_fp8_join<Bf16>, grid, dim3(256), 0, s, from, a.splits, n, given.y);
    else
      hipLaunchKernelGGL(k_fp8_join<F16>, grid, dim3(256), 0, s, from, a.splits, n, given.y);
    return hipGetLastError();
  }
  if (a.dtype == SPL_F32) return launch_kind<F32Out>(a, kind, columns, s);
  return a.dtype == SPL_BF16 ? launch_kind<Bf16>(a, kind, columns, s) : launch_kind<F16>(a, kind, columns, s);
}

}  // namespace spl
