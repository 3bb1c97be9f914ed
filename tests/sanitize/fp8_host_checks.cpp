// Sanitizer driver for the host side of the 8-bit float linears and of the optimizer step (test infrastructure).  Every
// entry point with arguments that its checks must reject before any HIP call, and every size function at its limits, built
// with -fsanitize=address,undefined on the host: an overflow in the arithmetic of sizes aborts the run.  Nothing here
// reaches a launch.  Prints "ok <checks>" and exits 0, or names the first failed check.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <limits>
#include <vector>

#include "spl.h"

// The one launch of another file that these entry points make.
namespace spl {
hipError_t launch_zero_fill(void*, int64_t, hipStream_t) {
  fprintf(stderr, "a launch\n");
  abort();
}
}  // namespace spl

static int checks = 0, failed = 0;
static void expect(bool ok, const char* what, int line) {
  ++checks;
  if (!ok && !failed) fprintf(stderr, "FAIL line %d: %s\n", line, what);
  failed += ok ? 0 : 1;
}
#define EXPECT(c) expect((c), #c, __LINE__)
#define REJECTS(call) expect((call) != SPL_OK, #call, __LINE__)

static const int64_t kBig = std::numeric_limits<int64_t>::max(), kMin = std::numeric_limits<int64_t>::min();
static void* at(uintptr_t a) { return reinterpret_cast<void*>(a); }

static spl_fp8_matrix matrix(int64_t rows, int64_t cols, int64_t count, int32_t block, uintptr_t where) {
  spl_fp8_matrix m{};
  m.codes = at(where), m.scales = at(where + ((uintptr_t)1 << 44)), m.rows = rows, m.cols = cols, m.count = count, m.block = block;
  m.codes_bytes = m.scales_bytes = kBig;
  return m;
}

int main() {
  const int64_t dims[] = {kMin, -1, 0, 1, 127, 128, 129, 4096, 65535, 65536, 1ll << 22, (1ll << 22) + 1, (1ll << 28) - 1, 1ll << 28,
                          (1ll << 31) - 1, 1ll << 31, 1ll << 40, kBig};
  const int32_t types[] = {-1, 0, SPL_F16, SPL_BF16, SPL_I8, SPL_I4, SPL_F32, 99};

  // sizes: -1, or what the format takes, below 2^42 bytes
  for (int64_t r : dims)
    for (int64_t c : dims) {
      const int64_t g = spl_fp8_grouped_cols(r, c);
      EXPECT(g == -1 || (g >= 128 && g % 128 == 0 && g >= r && g <= 1ll << 22));
      for (int64_t n : dims) {
        const int64_t b = spl_fp8_codes_bytes(r, c, n);
        EXPECT(b == -1 || (b > 0 && b <= 1ll << 42 && b % 128 == 0));
        for (int32_t block : {0, 1, 64, 128}) {
          const int64_t s = spl_fp8_scales_bytes(r, c, n, block);
          EXPECT(s == -1 || (s > 0 && s <= 1ll << 42 && b > 0 && (block == 1 || block == 128)));
        }
        const int64_t w = spl_linear_fp8_workspace_bytes(r, c, n), x = spl_linear_fp8_rows_workspace_bytes(r, c, n);
        EXPECT((w == -1 || (w >= 0 && w % 256 == 0)) && (x == -1 || (x >= 0 && x % 256 == 0)));
        EXPECT(w == -1 || r >= 1);
        for (int64_t e : dims) {
          const int64_t y = spl_linear_fp8_grouped_rows_workspace_bytes(r, c, n, e), z = spl_linear_fp8_grad_workspace_bytes(r, c, n, e);
          EXPECT((y == -1 || (y >= 0 && y % 256 == 0)) && (z == -1 || (z >= 0 && z % 256 == 0)));
          for (int32_t form : {-1, 0, 1, 2, 3})
            for (int32_t t : {0, (int)SPL_BF16, (int)SPL_F32}) {
              const int32_t k = spl_linear_fp8_kernel(form, r, c, n, e, t, SPL_BF16);
              EXPECT(k == -1 || (k >= 1 && k <= 22 && r > 0 && c > 0 && (n > 0 || (n == 0 && form == 2))));   // (no tokens: gradients of zeros)
            }
        }
      }
    }

  // matrices of every size against calls that have something else wrong: no answer but a refusal
  void *Y = at((uintptr_t)1 << 46), *ws = at((uintptr_t)1 << 47), *X = at((uintptr_t)3 << 46);
  const int32_t* starts = static_cast<const int32_t*>(at(0x1000));
  for (int64_t r : dims)
    for (int64_t c : dims)
      for (int64_t n : dims) {
        const spl_fp8_matrix m = matrix(r, c, n, 1, (uintptr_t)1 << 43), w = matrix(c, r, n, 128, (uintptr_t)1 << 45);
        spl_fp8_matrix small = m;
        small.codes_bytes = 127;
        REJECTS(spl_linear_fp8(&m, &small, SPL_BF16, Y, ws, nullptr));
        REJECTS(spl_linear_fp8(&m, &m, SPL_BF16, m.codes, ws, nullptr));      // the result in the codes
        REJECTS(spl_linear_fp8(&m, &w, SPL_I8, Y, ws, nullptr));
        REJECTS(spl_linear_fp8(&m, &w, SPL_F32, at(((uintptr_t)1 << 46) + 8), ws, nullptr));
        REJECTS(spl_linear_fp8_grouped(&m, &w, nullptr, SPL_BF16, Y, nullptr));
        REJECTS(spl_linear_fp8_grouped_weight_grad(&m, &m, starts, n, r, SPL_F32, at(8), nullptr));
        REJECTS(spl_linear_fp8_grouped_weight_grad(&m, &m, nullptr, n, r, SPL_F32, Y, nullptr));
        REJECTS(spl_dequantize_fp8(&m, SPL_F32, m.codes, nullptr));
        REJECTS(spl_dequantize_fp8(&m, SPL_I4, Y, nullptr));
        for (int64_t v : dims) {
          if (v > 0) REJECTS(spl_linear_fp8_rows(X, SPL_BF16, v, r, &m, SPL_BF16, m.codes, ws, nullptr));
          if (v > 0) REJECTS(spl_linear_fp8_grouped_rows(X, SPL_BF16, v, r, &m, starts, SPL_BF16, at(8), ws, nullptr));
          REJECTS(spl_linear_fp8_grouped_rows(X, SPL_BF16, v, r, &m, nullptr, SPL_BF16, Y, ws, nullptr));
          if (v != 0) REJECTS(spl_linear_fp8_grad(X, r, X, c, SPL_BF16, v, &m, starts, SPL_F32, m.codes, Y, ws, nullptr));
          REJECTS(spl_linear_fp8_grad(X, r, X, c, SPL_F32, v, &m, starts, SPL_F32, Y, nullptr, ws, nullptr));
          REJECTS(spl_linear_fp8_grad(X, r, X, c, SPL_BF16, v, &m, starts, SPL_F32, nullptr, nullptr, ws, nullptr));
          if (r != 0) REJECTS(spl_quantize_fp8(m.codes, SPL_BF16, r, c, v, n, nullptr, 0, &m, nullptr, nullptr));
          if (r != 0) REJECTS(spl_quantize_fp8(X, SPL_BF16, r, c, v, n, starts, v, &small, &w, nullptr));
        }
      }
  for (int32_t t : types) REJECTS(spl_quantize_fp8(X, t, 1, 1, 1, 1, nullptr, 0, nullptr, nullptr, nullptr));

  // plans
  std::vector<spl_adamw_tensor> list;
  for (int64_t n : dims)
    for (int32_t pd : types)
      for (int32_t bits : {0, 8, 32}) {
        spl_adamw_tensor t{};
        t.param = at(0x100000), t.grad = at((uintptr_t)1 << 42), t.m = at((uintptr_t)1 << 43), t.v = at((uintptr_t)1 << 44);
        t.m_scales = static_cast<uint8_t*>(at((uintptr_t)1 << 45)), t.v_scales = static_cast<uint8_t*>(at((uintptr_t)1 << 46));
        t.n = n;
        const spl_adamw_types ty{pd, SPL_BF16, 0, bits};
        for (int64_t count : {int64_t(-1), int64_t(0), int64_t(1), int64_t(2)}) {
          const spl_adamw_tensor two[2] = {t, t};
          const int64_t b = spl_adamw_plan_bytes(two, count, &ty), k = spl_adamw_plan_chunks(two, count, &ty);
          EXPECT((b == -1) == (k == -1) && (k == -1 || (k >= 0 && k < 1 << 24 && b % 16 == 0)));
          if (b > 0 && count == 2) {
            std::vector<unsigned char> host((size_t)(b < 1 << 20 ? b : 16) + 8);
            if (b < 1 << 20) REJECTS(spl_adamw_plan(two, 2, &ty, host.data() + (8 - (uintptr_t)host.data() % 8) % 8));   // both at one place
          }
          if (b == -1) REJECTS(spl_adamw_plan(two, count, &ty, &list));
        }
      }
  // a real plan, in the bytes that it asks for
  {
    const spl_adamw_types ty{SPL_F32, SPL_BF16, SPL_BF16, 8};
    uintptr_t next = 0x100000;
    for (int64_t n : {1, 127, 128, 129, 0, 8193, 5000000}) {
      spl_adamw_tensor t{};
      const auto take = [&](int64_t bytes) {
        void* p = at(next);
        next += (uintptr_t)(bytes + 255) / 256 * 256;
        return p;
      };
      t.n = n, t.decay = 0.1, t.param = take(4 * n), t.grad = take(2 * n), t.m = take(n + 128), t.v = take(n + 128), t.copy = take(2 * n);
      t.m_scales = static_cast<uint8_t*>(take(n / 128 + 1)), t.v_scales = static_cast<uint8_t*>(take(n / 128 + 1));
      list.push_back(t);
      const int64_t b = spl_adamw_plan_bytes(list.data(), (int64_t)list.size(), &ty);
      EXPECT(b > 0);
      std::vector<uint64_t> host((size_t)b / 8);
      EXPECT(spl_adamw_plan(list.data(), (int64_t)list.size(), &ty, host.data()) == SPL_OK);
    }
    for (double bad : {(double)NAN, (double)INFINITY, -1.0}) {
      REJECTS(spl_adamw_step(at(16), 1, &ty, 1e-3, bad, 0.9, 1e-8, 1, nullptr, nullptr, 0, nullptr));
      REJECTS(spl_adamw_step(at(16), 1, &ty, 1e-3, 0.9, bad, 1e-8, 1, nullptr, nullptr, 0, nullptr));
      REJECTS(spl_adamw_step(at(16), 1, &ty, 1e-3, 0.9, 0.9, bad, 1, nullptr, nullptr, 0, nullptr));
    }
    for (int64_t v : dims) {
      if (v < 1 || v >= 1ll << 31) REJECTS(spl_adamw_step(at(16), 1, &ty, 1e-3, 0.9, 0.9, 1e-8, v, nullptr, nullptr, 0, nullptr));
      if (v < 0 || v >= 1 << 24) REJECTS(spl_adamw_step(at(16), v, &ty, 1e-3, 0.9, 0.9, 1e-8, 1, nullptr, nullptr, 0, nullptr));
      if (v > 0) REJECTS(spl_adamw_step(at(8), 1, &ty, 1e-3, 0.9, 0.9, 1e-8, 1, nullptr, nullptr, 0, nullptr));
    }
  }
  if (failed) return fprintf(stderr, "%d of %d failed\n", failed, checks), 1;
  printf("ok %d\n", checks);
  return 0;
}
