// Products of 8-bit floats for many rows, for gfx950.
//
// A workgroup of WN x WM waves computes 16 FN WN columns of 16 FM WM rows of X, a wave 16 FN x 16 FM of them.  The sum
// advances a block of 128 columns a stage, which is one scaled matrix instruction for every 16 x 16 outputs.  Both
// operands go from memory straight into LDS, two stage buffers of 128-byte rows whose 16-byte piece c sits at c ^ (row
// % 8).  A wave's outputs are four quadrants, and its operands four halves in registers, A0, A1 (of W) and B0, B1 (of
// X); a stage multiplies A0 Bx, A0 By, A1 By, A1 Bx with x and y changing places every stage, so that each half is
// read from LDS, one a quadrant, into the registers that the quadrant before has left: By, A1, then A0 and By of the
// next stage.  The one barrier of a stage stands before its third quadrant: the buffer has been read by then and is
// refilled with the stage after the next, and the next stage's has been waited for.
#include <type_traits>

#include "fp8_tile.h"

namespace spl {
namespace {

constexpr uint32_t kOob = 0x80000000u;

__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t src, unsigned char* dst, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (__attribute__((address_space(3))) void*)dst, 16, voff, soff, 0, 0);
}
__device__ __forceinline__ void wait_vm0() { __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8)); }
__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

struct alignas(32) Codes32 {
  u32x4 lo, hi;
};

__device__ __forceinline__ uint32_t lds_load1(uint32_t addr) {
  return *reinterpret_cast<const __attribute__((address_space(3))) uint8_t*>((uintptr_t)addr);
}

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

// T: of the results; fp32 ones are summed by bf16 instructions.
template <class T, int FN, int FM, int WN, int WM>
__global__ void __launch_bounds__(64 * WN * WM, tile_waves(FN, FM)) k_fp8_tile(const Fp8GemmArgs a, const int tn,
                                                                               const int tm) {
  constexpr bool kExact = T::code == SPL_F32;
  constexpr int NW = WN * WM, BN = 16 * FN * WN, BM = 16 * FM * WM;
  constexpr int PW = BN / 8 / NW, PX = BM / 8 / NW;   // requests of 8 rows a wave and stage
  constexpr int SZ = (BN + BM) * 128, RQ = PW + PX;
  static_assert(BN % (8 * NW) == 0 && BM % (8 * NW) == 0, "whole requests");
  extern __shared__ __align__(16) unsigned char dsm[];
  // the XCDs (blockIdx % 8) take contiguous runs of tiles, four row tiles to a column of column tiles
  int bn, bm;
  {
    const int total = tm * tn, w = (int)blockIdx.x;
    const int q = total / 8, r = total % 8, x = w % 8, i = w / 8;
    const int t = x * q + (x < r ? x : r) + i;
    const int gsz = 4 * tn, grp = t / gsz, h = tm - grp * 4 < 4 ? tm - grp * 4 : 4, in = t - grp * gsz;
    bm = grp * 4 + in % h;
    bn = in / h;
  }
  const Fp8Part p = fp8_part(a, BM, bm, blockIdx.z);
  if (p.none) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wn = wave % WN, wm = wave / WN, fr = lane & 15, fg = lane >> 4;
  const int64_t n0 = (int64_t)bn * BN;
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
  // Request i of a stage; stages past the last read through empty descriptors: zeros.
  auto request = [&](int i, int st, int buf) {
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
  constexpr int SQ = (BN + BM) / 64 / NW;
  static_assert((BN + BM) % (64 * NW) == 0 && BN % 64 == 0, "whole requests");
  const uint8_t* wsc = a.w.scales + p.w_scales + (n0 >> a.w.shift) * a.w.spitch;
  const uint8_t* xsc = a.x.scales + ((int64_t)p.m0 >> a.x.shift) * a.x.spitch;
  uint32_t soff[SQ];
#pragma unroll
  for (int i = 0; i < SQ; ++i) {
    const int q = NW * i + wave, row = 64 * (q < BN / 64 ? q : q - BN / 64) + lane;
    if (q < BN / 64)
      soff[i] = row < Nr ? (uint32_t)(row >> a.w.shift) * (uint32_t)a.w.spitch : kOob;
    else
      soff[i] = row < Mr ? (uint32_t)(((p.m0 + row) >> a.x.shift) - (p.m0 >> a.x.shift)) * (uint32_t)a.x.spitch : kOob;
  }
  const int kal = p.k0 & ~3;
  auto request_scales = [&](int word) {              // the word'th from the one that k0 is in
    const int at = kal + 4 * word;
#pragma unroll
    for (int i = 0; i < SQ; ++i) {
      const int q = NW * i + wave;
      const bool w = q < BN / 64;
      const int rows = w ? ((Nr - 1) >> a.w.shift) + 1 : ((p.m0 + Mr - 1) >> a.x.shift) - (p.m0 >> a.x.shift) + 1;
      const int bytes = at < a.w.spitch ? rows * (w ? a.w.spitch : a.x.spitch) : 0;   // words past a row: zeros
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(w ? wsc : xsc), (short)0, bytes, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          r, (__attribute__((address_space(3))) void*)(dsm + 2 * SZ + (word & 3) * (BN + BM) * 4 + 256 * q), 4, soff[i], at, 0, 0);
    }
  };
  const uint32_t sbase = lds_off(dsm) + 2 * SZ + 4 * fr;
  uint32_t sc[FN + FM], coming[FN + FM];              // the scale bytes of this stage, of the next one
  auto read_scales = [&](int st) {
    const int b = (p.k0 & 3) + st;
    const uint32_t at = sbase + (uint32_t)(((b >> 2) & 3) * (BN + BM) * 4 + (b & 3));
#pragma unroll
    for (int i = 0; i < FN + FM; ++i)
      coming[i] = lds_load1(at + 4 * (i < FN ? 16 * (FN * wn + i) : BN + 16 * (FM * wm + i - FN)));
  };

  // a row's pieces fg and fg + 4, in the first stage buffer and in the second
  const uint32_t turn = 16 * (uint32_t)(fg ^ (fr & 7));
  const uint32_t arow = lds_off(dsm) + 128 * (16 * FN * wn + fr), brow = lds_off(dsm) + BN * 128 + 128 * (16 * FM * wm + fr);
  const uint32_t al[2] = {arow + turn, arow + turn + SZ}, ah[2] = {arow + (turn ^ 64u), arow + (turn ^ 64u) + SZ};
  const uint32_t bl[2] = {brow + turn, brow + turn + SZ}, bh[2] = {brow + (turn ^ 64u), brow + (turn ^ 64u) + SZ};
  Codes32 A[2][2], B[FM];
  auto read_a = [&](Codes32 (&d)[2], int step, int buf) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      d[i].lo = lds_load16(al[buf] + 2048 * (2 * step + i));
      d[i].hi = lds_load16(ah[buf] + 2048 * (2 * step + i));
    }
  };
  auto read_b = [&](int j, int buf) {
    B[j].lo = lds_load16(bl[buf] + 2048 * j);
    B[j].hi = lds_load16(bh[buf] + 2048 * j);
  };
  f32x4 acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  Wide8 aw[kExact ? 2 : 1], bw[kExact ? FM : 1];
  auto widen_a = [&](const Codes32 (&w)[2], int step) {
    if constexpr (kExact) {
#pragma unroll
      for (int i = 0; i < 2; ++i) aw[i] = fp8_widen32(w[i].lo, w[i].hi, sc[2 * step + i]);
    }
  };
  auto widen_b = [&]() {
    if constexpr (kExact) {
#pragma unroll
      for (int j = 0; j < FM; ++j) bw[j] = fp8_widen32(B[j].lo, B[j].hi, sc[FN + j]);
    }
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

  if (nst > 0) {
#pragma unroll
    for (int i = 0; i < RQ + RQ / 2; ++i) request(i % RQ, i / RQ, i / RQ);
    request_scales(0);
    request_scales(1);
    wait_vm0();
    tile_barrier();
    read_scales(0);
    read_a(A[0], 0, 0);
#pragma unroll
    for (int j = 0; j < FM; ++j) read_b(j, 0);
    auto stage = [&](int st, auto x) {
      constexpr int buf = decltype(x)::value;
      const uint32_t mask = st < nst ? 255u : 0u;    // the stage past the last has codes of zero, and 0 as its scale
#pragma unroll
      for (int i = 0; i < FN + FM; ++i) sc[i] = coming[i] & mask;
      widen_b();
#pragma unroll
      for (int step = 0; step < FN / 2 - 1; ++step) {
        __builtin_amdgcn_sched_barrier(0);
        read_a(A[(step + 1) & 1], step + 1, buf);
        if (step == FN / 2 - 2) read_scales(st + 1);
        __builtin_amdgcn_sched_barrier(0);
        widen_a(A[step & 1], step);
#pragma unroll
        for (int j = 0; j < FM; ++j) {
          multiply(A[step & 1], step, j);
          if (step == 0) {                           // the second half of stage st + 1's
#pragma unroll
            for (int i = RQ * (FM + j) / (2 * FM); i < RQ * (FM + j + 1) / (2 * FM); ++i) request(i, st + 1, 1 - buf);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_waitcnt(0);                 // my reads of this buffer, my requests for the next
      tile_barrier();
      if (buf == 0) request_scales(st / 4 + 2);      // (twice the same: a branch here would cost more)
      read_a(A[0], 0, 1 - buf);
      __builtin_amdgcn_sched_barrier(0);
      widen_a(A[1], FN / 2 - 1);
#pragma unroll
      for (int j = 0; j < FM; ++j) {
        multiply(A[1], FN / 2 - 1, j);
        read_b(j, 1 - buf);
#pragma unroll
        for (int i = RQ * j / (2 * FM); i < RQ * (j + 1) / (2 * FM); ++i) request(i, st + 2, buf);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    for (int st = 0; st < nst; st += 2) {            // the stage past an odd number's last multiplies zeros
      stage(st, std::integral_constant<int, 0>{});
      stage(st + 1, std::integral_constant<int, 1>{});
    }
    if constexpr (FN * FM > 32) settle(acc);
    wait_vm0();                                      // no request outlives the workgroup's LDS
  }

  // Results: 16 rows of the wave's at a time through LDS, so that a row's leave as 16-byte pieces.  A lane has columns
  // 4 fg .. 4 fg + 3 of each fragment, row fr; piece c of a row sits at c ^ row.
  constexpr int E = kExact ? 4 : 2, CH = 16 * FN * E / 16;   // bytes of a result, pieces of a row
  tile_barrier();                                    // the other waves have read their last stage
  unsigned char* out = dsm + wave * (2 * 16 * CH * 16);
  const int64_t nw = n0 + 16 * FN * wn;
  const bool whole = nw + 16 * FN <= a.N && (a.N * E) % 16 == 0;
#pragma unroll
  for (int j = 0; j < FM; ++j) {
    unsigned char* half = out + (j & 1) * (16 * CH * 16);
#pragma unroll
    for (int i = 0; i < FN; ++i) {
      const f32x4 v = acc[i][j];
      if constexpr (kExact) {
        *reinterpret_cast<f32x4*>(half + fr * (CH * 16) + 16 * ((4 * i + fg) ^ (fr & (CH - 1)))) = v;
      } else {
        *reinterpret_cast<u32x2*>(half + fr * (CH * 16) + 16 * ((2 * i + (fg >> 1)) ^ (fr & (CH - 1))) + 8 * (fg & 1)) =
            u32x2{fp8_pack2<T>(v[0], v[1]), fp8_pack2<T>(v[2], v[3])};
      }
    }
    wave_lds_sync();
#pragma unroll
    for (int q = 0; q < 16 * CH / 64; ++q) {
      const int e = 64 * q + lane, row = e / CH, c = e % CH;
      const u32x4 v = *reinterpret_cast<const u32x4*>(half + row * (CH * 16) + 16 * (c ^ (row & (CH - 1))));
      const int m = 16 * (FM * wm + j) + row;
      if (m >= Mr) continue;
      const int64_t n = nw + c * (16 / E), at = p.y + (p.m0 + m) * a.N + n;
      unsigned char* y = static_cast<unsigned char*>(a.y) + at * E;
      if (whole) {
        *reinterpret_cast<u32x4*>(y) = v;
      } else {
#pragma unroll
        for (int k = 0; k < 16 / E; ++k) {
          if (n + k >= a.N) break;
          if constexpr (kExact)
            reinterpret_cast<uint32_t*>(y)[k] = v[k];
          else
            reinterpret_cast<uint16_t*>(y)[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
        }
      }
    }
  }
}

template <class T, int FN, int FM, int WN, int WM>
hipError_t launch_tile(const Fp8GemmArgs& a, hipStream_t s) {
  constexpr int BN = 16 * FN * WN, BM = 16 * FM * WM, LDS = 2 * (BN + BM) * 128 + 4 * (BN + BM) * 4;
  static PerDeviceFlag done;
  auto* kernel = k_fp8_tile<T, FN, FM, WN, WM>;
  const hipError_t e = allow_lds_once(done, kernel, LDS);
  if (e != hipSuccess) return e;
  const int64_t tn = (a.N + BN - 1) / BN, tm = fp8_row_tiles(a, BM);
  if (tn * tm >= (int64_t)1 << 22) return hipErrorNotSupported;
  const dim3 grid((unsigned)(tn * tm), 1u, a.mode == kFp8Sum ? (unsigned)a.groups : 1u);
  hipLaunchKernelGGL(kernel, grid, dim3(64 * WN * WM), LDS, s, a, (int)tn, (int)tm);
  return hipGetLastError();
}

template <class T>
hipError_t by_size(const Fp8GemmArgs& a, hipStream_t s) {
  if constexpr (T::code != SPL_F32) {
    const int64_t big = ((a.N + 255) / 256) * fp8_row_tiles(a, 256) * (a.mode == kFp8Sum ? a.groups : 1);
    if (big >= 128) return launch_tile<T, 8, 8, 2, 2>(a, s);
  }
  return launch_tile<T, 4, 4, 2, 2>(a, s);
}

}  // namespace

hipError_t launch_fp8_gemm(const Fp8GemmArgs& a, hipStream_t s) {
  if (a.x16 || a.M <= 64) return launch_fp8_stream(a, s);
  if (a.dtype == SPL_F32) return by_size<F32Out>(a, s);
  return a.dtype == SPL_BF16 ? by_size<Bf16>(a, s) : by_size<F16>(a, s);
}

}  // namespace spl
