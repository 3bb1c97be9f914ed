// AdamW over many tensors in one launch, for gfx950 (the formulas stand in spl.h).
//
// A plan lists the tensors and cuts them into chunks of 2048 or 8192 elements, one
// a workgroup; a thread has 8 neighbouring elements at a time, so that 8-bit
// states' blocks of 128 are 16 neighbouring lanes and their scales come from
// four lane moves.  Everything is read and written once, which bounds it: 60.8 million elements, fp32 p, bf16
// gradient and copy, 340 us (5.0 TB/s); 8-bit states 218 (4.5; 208 with the root that is not rounded to nearest, so there
// the arithmetic counts too).  16 small tensors 4.4 us.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "spl_fp8.h"

// Every product and sum is rounded by itself, as the formula in spl.h has it: by default a product that is added is fused
// with the sum, the compiler's choice which, and the update would differ between compilers.  (The intrinsics named after
// roundings to nearest do not keep products and sums apart here, and the one of the root is the approximate instruction.)
#pragma clang fp contract(off)

namespace spl {
namespace {

constexpr int kThreads = 256, kEach = 8;
// Elements of a chunk: a workgroup's one turn where all tensors together do not fill the chip anyway, else four of them.
constexpr int64_t kTurn = kThreads * kEach, kFew = 2048 * kTurn;

// A chunk with its tensor's addresses, so that a workgroup's data is two trips to memory away.
struct Chunk {
  void* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* ms;
  uint8_t* vs;
  void* copy;
  int64_t begin;
  double decay;
  int32_t size;
  int32_t tensor;
  int32_t wide;                                 // every array is aligned for 16-byte (8-bit codes: 8-byte) accesses
  int32_t pad_[3];
};
int64_t chunk_size(const spl_adamw_tensor* t, int64_t count) {
  int64_t n = 0;
  for (int64_t i = 0; i < count; ++i) n += t[i].n;
  return n <= kFew ? kTurn : 4 * kTurn;
}

struct F32P {};
template <class T>
__device__ __forceinline__ float get(const void* p, int64_t i) {
  if constexpr (std::is_same<T, F32P>::value)
    return static_cast<const float*>(p)[i];
  else
    return T::to_f32(static_cast<const uint16_t*>(p)[i]);
}
template <class T>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
  if constexpr (std::is_same<T, F32P>::value)
    static_cast<float*>(p)[i] = v;
  else
    static_cast<uint16_t*>(p)[i] = T::from_f32(v);
}
// `have` (1 to 8) of 8 neighbours; wide: all 8 of them, aligned.
template <class T>
__device__ __forceinline__ void get8(const void* p, int64_t i, int have, bool wide, float (&v)[8]) {
  if (wide) {
    if constexpr (std::is_same<T, F32P>::value) {
      const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
      const f32x4 a = q[0], b = q[1];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
    } else {
      const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[2 * j] = T::to_f32(a[j] & 0xffffu), v[2 * j + 1] = T::to_f32(a[j] >> 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < have ? get<T>(p, i + j) : 0.f;
  }
}
template <class T>
__device__ __forceinline__ void put8(void* p, int64_t i, int have, bool wide, const float (&v)[8]) {
  if (wide) {
    if constexpr (std::is_same<T, F32P>::value) {
      f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
      q[0] = f32x4{v[0], v[1], v[2], v[3]};
      q[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      u32x4 a;
#pragma unroll
      for (int j = 0; j < 4; ++j) a[j] = (uint32_t)T::from_f32(v[2 * j]) | ((uint32_t)T::from_f32(v[2 * j + 1]) << 16);
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i) = a;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < have) put<T>(p, i + j, v[j]);
  }
}

// A hash of 32 bits: shifts and odd multipliers (2^32 over the golden ratio, over the root of 3).
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x9E3779B1u;
  x = (x ^ (x >> 15)) * 0x93CD3A2Du;
  return x ^ (x >> 16);
}

// x^t by squaring, in 64 bits.
__device__ __forceinline__ double power(double x, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1) {
    if (t & 1) r *= x;
    x *= x;
  }
  return r;
}

// |x| <= 448 to one of the two codes' values next to it: past the smallest
// normal one, 2^-6, by adding the random bits below the code's last fraction
// bit; below it in steps of 2^-9.
// keep: what is not 0 does not become 0.
__device__ __forceinline__ float stochastic(float x, uint32_t rnd, bool keep) {
  const float a = fabsf(x);
  float r = __uint_as_float((__float_as_uint(a) + rnd) & 0xfff00000u);
  if (a < 0x1p-6f) r = floorf(a * 512.f + (float)rnd * 0x1p-20f) * 0x1p-9f;
  if (keep && r < 0x1p-9f) r = 0x1p-9f;
  return copysignf(r, x);
}

// 8 values of a lane to codes at c[i], the block's scale to s[i / 128]; every lane of the wave takes part.
__device__ __forceinline__ void encode8(float (&x)[8], const uint32_t (&rnd)[8], bool keep, uint8_t* c, uint8_t* s,
                                        int64_t i, bool mine) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = umax(m, __float_as_uint(x[j]) & 0x7fffffffu);
  const uint32_t byte = fp8_scale_byte(row16_max(m));
  const float f = fp8_inverse(byte);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = stochastic(x[j] * f, rnd[j], keep && x[j] > 0.f);
  u32x2 q = {fp8_four(x[0], x[1], x[2], x[3]), fp8_four(x[4], x[5], x[6], x[7])};
  if (byte == 255) q = u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
  if (!mine) return;
  *reinterpret_cast<u32x2*>(c + i) = q;
  if ((i & 127) == 0) s[i >> 7] = (uint8_t)byte;
}
__device__ __forceinline__ void decode8(const uint8_t* c, const uint8_t* s, int64_t i, bool mine, float (&x)[8]) {
  const u32x2 q = mine ? *reinterpret_cast<const u32x2*>(c + i) : u32x2{0u, 0u};
  const uint32_t byte = mine ? s[i >> 7] : 0u;
  const float f = byte == 255 ? __uint_as_float(0x7fc00000u) : (byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23));
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 0) * f, x[1] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 1) * f;
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 2) * f, x[3] = __builtin_amdgcn_cvt_f32_fp8((int)q.x, 3) * f;
  x[4] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 0) * f, x[5] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 1) * f;
  x[6] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 2) * f, x[7] = __builtin_amdgcn_cvt_f32_fp8((int)q.y, 3) * f;
}

template <class P, class G, bool k8>
__global__ void __launch_bounds__(kThreads) k_adamw(const Chunk* chunks, const AdamwHyper h, const int copy) {
  const float gs = h.grad_scale ? *h.grad_scale : 1.f;
  const Chunk t = chunks[blockIdx.x];
  int64_t step = h.step_on_device ? *h.step_on_device : h.step;
  step = step < 1 ? 1 : step;
  const float keep = (float)(1.0 - h.lr * t.decay), rate = (float)(h.lr / (1.0 - power(h.beta1, step)));
  const float root = (float)(1.0 / sqrt(1.0 - power(h.beta2, step)));
  const float b1 = (float)h.beta1, c1 = (float)(1.0 - h.beta1), b2 = (float)h.beta2, c2 = (float)(1.0 - h.beta2);
  const float eps = (float)h.eps;
  uint32_t key = 0;
  if constexpr (k8) key = mix(mix(h.seed ^ ((uint32_t)step * 0x6A09E667u)) + (uint32_t)t.tensor);
  const int64_t begin = t.begin, end = isfinite(gs) ? begin + t.size : begin;   // a scale that is not finite: nothing is updated
  // whole waves go through the loop together: 8-bit blocks ask their neighbours
  for (int64_t at = begin; at < end; at += kThreads * kEach) {
    const int64_t i = at + kEach * (int64_t)threadIdx.x;
    const int have = (int)(end - i < 8 ? end - i : 8);
    const bool mine = have > 0, wide = t.wide && have == 8;
    float p[8], g[8], m[8], v[8], r[8];
    get8<P>(t.p, i, have, wide, p);
    get8<G>(t.g, i, have, wide, g);
    if constexpr (k8) {
      decode8(static_cast<const uint8_t*>(t.m), t.ms, i, mine, m);
      decode8(static_cast<const uint8_t*>(t.v), t.vs, i, mine, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= have) m[j] = v[j] = 0.f;
        v[j] = v[j] * v[j];
      }
    } else {
      get8<F32P>(t.m, i, have, wide, m);
      get8<F32P>(t.v, i, have, wide, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = g[j] * gs;
      m[j] = m[j] * b1 + d * c1;
      v[j] = v[j] * b2 + d * d * c2;
      r[j] = sqrtf(v[j]);                            // (to nearest, as the quotient: hipcc's default for both)
      p[j] = p[j] * keep - rate * (m[j] / (r[j] * root + eps));
    }
    if (mine) {
      put8<P>(t.p, i, have, wide, p);
      if (copy == SPL_BF16) put8<Bf16>(t.copy, i, have, wide, p);
      if (copy == SPL_F16) put8<F16>(t.copy, i, have, wide, p);
    }
    if constexpr (k8) {
      uint32_t ra[8], rb[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t x = mix((uint32_t)(i + j) + key);
        ra[j] = x >> 12, rb[j] = mix(x + 1u) >> 12;
      }
      encode8(m, ra, false, static_cast<uint8_t*>(t.m), t.ms, i, mine);
      encode8(r, rb, true, static_cast<uint8_t*>(t.v), t.vs, i, mine);
    } else if (mine) {
      put8<F32P>(t.m, i, have, wide, m);
      put8<F32P>(t.v, i, have, wide, v);
    }
  }
}

template <class P, class G>
hipError_t launch(const void* plan, int64_t chunks, const spl_adamw_types& ty, const AdamwHyper& h, hipStream_t s) {
  const Chunk* c = static_cast<const Chunk*>(plan);
  if (ty.state_bits == 8)
    hipLaunchKernelGGL((k_adamw<P, G, true>), dim3((unsigned)chunks), dim3(kThreads), 0, s, c, h, ty.copy_dtype);
  else
    hipLaunchKernelGGL((k_adamw<P, G, false>), dim3((unsigned)chunks), dim3(kThreads), 0, s, c, h, ty.copy_dtype);
  return hipGetLastError();
}
template <class P>
hipError_t by_grad(const void* plan, int64_t chunks, const spl_adamw_types& ty, const AdamwHyper& h, hipStream_t s) {
  if (ty.grad_dtype == SPL_F32) return launch<P, F32P>(plan, chunks, ty, h, s);
  return ty.grad_dtype == SPL_BF16 ? launch<P, Bf16>(plan, chunks, ty, h, s) : launch<P, F16>(plan, chunks, ty, h, s);
}

}  // namespace

int64_t adamw_plan_chunks(const spl_adamw_tensor* t, int64_t count) {
  const int64_t size = chunk_size(t, count);
  int64_t c = 0;
  for (int64_t i = 0; i < count; ++i) c += (t[i].n + size - 1) / size;
  return c;
}
int64_t adamw_plan_bytes(const spl_adamw_tensor* t, int64_t count) {
  return adamw_plan_chunks(t, count) * (int64_t)sizeof(Chunk);
}

static_assert(sizeof(Chunk) % 16 == 0, "alignment");
void adamw_plan_write(const spl_adamw_tensor* t, int64_t count, const spl_adamw_types& ty, void* host) {
  const int64_t size = chunk_size(t, count);
  memset(host, 0, (size_t)adamw_plan_bytes(t, count));
  Chunk* c = static_cast<Chunk*>(host);
  for (int64_t i = 0; i < count; ++i) {
    const spl_adamw_tensor& x = t[i];
    uintptr_t all = reinterpret_cast<uintptr_t>(x.param) | reinterpret_cast<uintptr_t>(x.grad);
    if (ty.state_bits == 32) all |= reinterpret_cast<uintptr_t>(x.m) | reinterpret_cast<uintptr_t>(x.v);
    if (ty.copy_dtype) all |= reinterpret_cast<uintptr_t>(x.copy);
    for (int64_t k = 0; k < x.n; k += size)
      *c++ = Chunk{x.param, x.grad, x.m, x.v, x.m_scales, x.v_scales, x.copy, k, x.decay,
                   (int32_t)(x.n - k < size ? x.n - k : size), (int32_t)i, (all & 15) == 0, {0, 0, 0}};
  }
}

hipError_t launch_adamw(const void* plan, int64_t chunks, const spl_adamw_types& ty, const AdamwHyper& h,
                        hipStream_t s) {
  if (ty.param_dtype == SPL_F32) return by_grad<F32P>(plan, chunks, ty, h, s);
  return ty.param_dtype == SPL_BF16 ? by_grad<Bf16>(plan, chunks, ty, h, s) : by_grad<F16>(plan, chunks, ty, h, s);
}

}  // namespace spl
