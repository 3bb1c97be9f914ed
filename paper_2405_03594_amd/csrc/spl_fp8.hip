// extern "C" entry points of the 8-bit float linears and of the optimizer step:
// argument checks on the host, then launches on the caller's stream.
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>
#include <vector>

#include "spl.h"
#include "spl_fp8.h"

namespace {

using spl::Fp8GemmArgs;

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxCols = (int64_t)1 << 22;
constexpr int64_t kMaxBytes = (int64_t)1 << 42;
constexpr int64_t kMaxCount = 65535;
constexpr int64_t kMaxN = (int64_t)1 << 28;             // rows of W: 2^32 threads of the streaming kernels

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool given(const void* p, uintptr_t a) { return p && aligned(p, a); }
bool half_type(int32_t d) { return d == SPL_F16 || d == SPL_BF16; }
bool float_type(int32_t d) { return half_type(d) || d == SPL_F32; }
int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

spl_status launched(hipError_t e) {
  if (e == hipSuccess) return SPL_OK;
  return e == hipErrorNotSupported ? SPL_ERR_UNSUPPORTED : SPL_ERR_DEVICE;
}

bool sizes_ok(int64_t rows, int64_t cols, int64_t count) {
  return rows >= 1 && rows < kMaxRows && cols >= 1 && cols <= kMaxCols && count >= 1 && count <= kMaxCount &&
         rows <= kMaxBytes / spl::fp8_pitch(cols) / count;
}
spl_status check_matrix(const spl_fp8_matrix* m) {
  if (!m || (m->block != 1 && m->block != 128) || !sizes_ok(m->rows, m->cols, m->count) || !given(m->codes, 16) ||
      !given(m->scales, 4))
    return SPL_ERR_INVALID_ARG;
  if (m->codes_bytes < spl_fp8_codes_bytes(m->rows, m->cols, m->count) ||
      m->scales_bytes < spl_fp8_scales_bytes(m->rows, m->cols, m->count, m->block))
    return SPL_ERR_INVALID_ARG;
  return SPL_OK;
}

// Whether a result, fully in [p, p + bytes), is apart from other memory of the call: workgroups write it while others read.
bool apart(const void* p, int64_t bytes, const void* q, int64_t more) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return !p || !q || a + (uintptr_t)bytes <= b || b + (uintptr_t)more <= a;
}
bool apart(const void* p, int64_t bytes, const spl_fp8_matrix& m) {
  return apart(p, bytes, m.codes, spl_fp8_codes_bytes(m.rows, m.cols, m.count)) &&
         apart(p, bytes, m.scales, spl_fp8_scales_bytes(m.rows, m.cols, m.count, m.block));
}
bool apart(const spl_fp8_matrix& out, const void* q, int64_t more) { return apart(q, more, out); }
bool apart(const spl_fp8_matrix& a, const spl_fp8_matrix& b) {
  return apart(a.codes, spl_fp8_codes_bytes(a.rows, a.cols, a.count), b) &&
         apart(a.scales, spl_fp8_scales_bytes(a.rows, a.cols, a.count, a.block), b);
}
int64_t type_bytes(int32_t d) { return d == SPL_F32 ? 4 : 2; }
int64_t rows_bytes(int64_t rows, int64_t stride, int64_t cols, int32_t d) { return ((rows - 1) * stride + cols) * type_bytes(d); }

int64_t codes_workspace(int64_t M, int64_t N, int64_t cols) {
  return align256(spl::fp8_partial_bytes(M, N, (int32_t)(spl::fp8_pitch(cols) / 128)));
}
int64_t rows_workspace(int64_t M, int64_t N, int64_t cols, int64_t experts) {
  if (spl::fp8_fused(M, N, cols, experts)) return 0;
  return align256(M * spl::fp8_pitch(cols)) + align256(M * spl::fp8_spitch(cols)) +
         (experts == 1 ? codes_workspace(M, N, cols) : 0);
}
bool product_ok(int64_t M, int64_t N, int64_t cols, int64_t experts) {
  return M >= 0 && M < kMaxRows && (M == 0 || sizes_ok(M, cols, 1)) && sizes_ok(N, cols, experts) &&
         (M == 0 || N <= kMaxBytes / M);
}

// What the products of rows in 16 bits share: fused, or codes in the workspace first.
spl_status rows_product(const void* X, int32_t x_dtype, int64_t M, int64_t row_stride, const spl_fp8_matrix* W,
                        const int32_t* starts, int32_t dtype, void* Y, void* workspace, hipStream_t stream) {
  spl_status st = check_matrix(W);
  if (st != SPL_OK) return st;
  if (!half_type(x_dtype) || !float_type(dtype)) return SPL_ERR_UNSUPPORTED;
  if (!product_ok(M, W->rows, W->cols, W->count) || (!starts && W->count != 1)) return SPL_ERR_INVALID_ARG;
  if (M == 0) return SPL_OK;
  if (row_stride < W->cols || row_stride > kMaxBytes / M || !given(X, 2) || !given(Y, 16) || !aligned(starts, 4))
    return SPL_ERR_INVALID_ARG;
  const int64_t need = rows_workspace(M, W->rows, W->cols, W->count);
  if (need > 0 && !given(workspace, 256)) return SPL_ERR_INVALID_ARG;
  const int64_t bytes = M * W->rows * type_bytes(dtype);
  if (!apart(Y, bytes, *W) || !apart(Y, bytes, X, rows_bytes(M, row_stride, W->cols, x_dtype)) ||
      !apart(Y, bytes, workspace, need))
    return SPL_ERR_INVALID_ARG;
  if (M > kMaxCols || W->rows >= kMaxN) return SPL_ERR_UNSUPPORTED;
  (void)hipGetLastError();
  Fp8GemmArgs a{};
  a.w = spl::fp8_view(*W);
  a.M = M, a.N = W->rows, a.blocks = a.w.pitch / 128, a.dtype = dtype, a.y = Y, a.cols = (int32_t)W->cols;
  a.starts = starts, a.groups = (int32_t)W->count, a.mode = starts ? spl::kFp8Rows : spl::kFp8Plain;
  if (need == 0) {
    a.x16 = X, a.x16_stride = row_stride, a.x16_dtype = x_dtype;
    return launched(spl::launch_fp8_gemm(a, stream));
  }
  uint8_t* base = static_cast<uint8_t*>(workspace);
  spl_fp8_matrix q{};
  q.codes = base, q.scales = base + align256(M * a.w.pitch), q.rows = M, q.cols = W->cols, q.count = 1, q.block = 1;
  spl::Fp8QuantArgs z{};
  z.X = X, z.row_stride = row_stride, z.rows = M, z.cols = W->cols, z.count = 1, z.out = spl::fp8_view(q);
  const hipError_t e = spl::launch_fp8_quantize(z, x_dtype, stream);
  if (e != hipSuccess) return launched(e);
  a.x = z.out;
  const int64_t codes = align256(M * a.w.pitch) + align256(M * a.w.spitch);
  if (!starts && need > codes) a.partial = base + codes;
  return launched(spl::launch_fp8_gemm(a, stream));
}

}  // namespace

extern "C" {

int64_t spl_fp8_codes_bytes(int64_t rows, int64_t cols, int64_t count) {
  return sizes_ok(rows, cols, count) ? count * rows * spl::fp8_pitch(cols) : -1;
}
int64_t spl_fp8_scales_bytes(int64_t rows, int64_t cols, int64_t count, int32_t block) {
  if (!sizes_ok(rows, cols, count) || (block != 1 && block != 128)) return -1;
  return count * spl::fp8_scale_rows(rows, block) * spl::fp8_spitch(cols);
}
int64_t spl_fp8_grouped_cols(int64_t rows, int64_t groups) {
  if (rows < 0 || rows > kMaxCols || groups < 1 || groups > kMaxCount) return -1;
  const int64_t c = 128 * spl::most_tiles(rows, groups, 128);
  return c < 128 ? 128 : (c <= kMaxCols ? c : -1);
}

spl_status spl_quantize_fp8(const void* X, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, int64_t count,
                            const int32_t* starts, int64_t groups, const spl_fp8_matrix* out,
                            const spl_fp8_matrix* out_t, hipStream_t stream) {
  if (!float_type(dtype)) return SPL_ERR_UNSUPPORTED;
  if (rows < 0 || rows >= kMaxRows || cols < 1 || cols >= kMaxRows || count < 1 || count > kMaxCount || (!out && !out_t))
    return SPL_ERR_INVALID_ARG;
  if (rows > kMaxCols || cols > kMaxCols) return SPL_ERR_UNSUPPORTED;
  if (starts && (count != 1 || groups < 1 || groups > kMaxCount || !aligned(starts, 4))) return SPL_ERR_INVALID_ARG;
  if (rows == 0) return SPL_OK;
  if (row_stride < cols || row_stride > kMaxBytes / rows / count || !given(X, dtype == SPL_F32 ? 4 : 2))
    return SPL_ERR_INVALID_ARG;
  spl::Fp8QuantArgs a{};
  const int64_t bytes = rows_bytes(count * rows, row_stride, cols, dtype);
  if (out) {
    const spl_status st = check_matrix(out);
    if (st != SPL_OK) return st;
    if (out->rows != rows || out->cols != cols || out->count != count || (starts && out->block != 1))
      return SPL_ERR_INVALID_ARG;
    if (!apart(*out, X, bytes)) return SPL_ERR_INVALID_ARG;
    a.out = spl::fp8_view(*out);
  }
  if (out_t) {
    const spl_status st = check_matrix(out_t);
    if (st != SPL_OK) return st;
    const int64_t want = starts ? spl_fp8_grouped_cols(rows, groups) : rows;
    if (out_t->rows != cols || out_t->count != count || want < 0 || (starts ? out_t->cols < want : out_t->cols != want) ||
        (starts && out_t->block != 1) || (out && out->block != out_t->block))
      return SPL_ERR_INVALID_ARG;
    if (!apart(*out_t, X, bytes) || (out && !apart(*out, *out_t))) return SPL_ERR_INVALID_ARG;
    a.out_t = spl::fp8_view(*out_t);
  }
  a.X = X, a.row_stride = row_stride, a.rows = rows, a.cols = cols, a.count = count, a.starts = starts;
  a.groups = (int32_t)(starts ? groups : 0);
  (void)hipGetLastError();
  return launched(spl::launch_fp8_quantize(a, dtype, stream));
}

spl_status spl_dequantize_fp8(const spl_fp8_matrix* A, int32_t dtype, void* out, hipStream_t stream) {
  const spl_status st = check_matrix(A);
  if (st != SPL_OK) return st;
  if (!float_type(dtype)) return SPL_ERR_UNSUPPORTED;
  if (!given(out, 16) || !apart(out, A->count * A->rows * A->cols * type_bytes(dtype), *A)) return SPL_ERR_INVALID_ARG;
  (void)hipGetLastError();
  return launched(spl::launch_fp8_dequantize(spl::fp8_view(*A), A->cols, A->count, dtype, out, stream));
}

int64_t spl_linear_fp8_workspace_bytes(int64_t M, int64_t N, int64_t cols) {
  return M >= 1 && product_ok(M, N, cols, 1) ? codes_workspace(M, N, cols) : -1;
}
spl_status spl_linear_fp8(const spl_fp8_matrix* X, const spl_fp8_matrix* W, int32_t dtype, void* Y, void* workspace,
                          hipStream_t stream) {
  spl_status st = check_matrix(X);
  if (st == SPL_OK) st = check_matrix(W);
  if (st != SPL_OK) return st;
  if (!float_type(dtype)) return SPL_ERR_UNSUPPORTED;
  if (X->cols != W->cols || X->count != 1 || W->count != 1 || !product_ok(X->rows, W->rows, W->cols, 1) || !given(Y, 16))
    return SPL_ERR_INVALID_ARG;
  const int64_t bytes = X->rows * W->rows * type_bytes(dtype);
  if (!apart(Y, bytes, *X) || !apart(Y, bytes, *W)) return SPL_ERR_INVALID_ARG;
  if (W->rows >= kMaxN) return SPL_ERR_UNSUPPORTED;
  Fp8GemmArgs a{};
  a.x = spl::fp8_view(*X), a.w = spl::fp8_view(*W);
  a.M = X->rows, a.N = W->rows, a.blocks = a.w.pitch / 128, a.dtype = dtype, a.y = Y, a.mode = spl::kFp8Plain;
  const int64_t partial = spl::fp8_partial_bytes(a.M, a.N, a.blocks);
  if (partial > 0) {
    if (!given(workspace, 256) || !apart(Y, bytes, workspace, partial)) return SPL_ERR_INVALID_ARG;
    a.partial = workspace;
  }
  (void)hipGetLastError();
  return launched(spl::launch_fp8_gemm(a, stream));
}

int64_t spl_linear_fp8_rows_workspace_bytes(int64_t M, int64_t N, int64_t cols) {
  return product_ok(M, N, cols, 1) ? (M == 0 ? 0 : rows_workspace(M, N, cols, 1)) : -1;
}
spl_status spl_linear_fp8_rows(const void* X, int32_t x_dtype, int64_t M, int64_t row_stride, const spl_fp8_matrix* W,
                               int32_t dtype, void* Y, void* workspace, hipStream_t stream) {
  return rows_product(X, x_dtype, M, row_stride, W, nullptr, dtype, Y, workspace, stream);
}

spl_status spl_linear_fp8_grouped(const spl_fp8_matrix* X, const spl_fp8_matrix* W, const int32_t* starts,
                                  int32_t dtype, void* Y, hipStream_t stream) {
  spl_status st = check_matrix(X);
  if (st == SPL_OK) st = check_matrix(W);
  if (st != SPL_OK) return st;
  if (!float_type(dtype)) return SPL_ERR_UNSUPPORTED;
  if (X->cols != W->cols || X->count != 1 || !product_ok(X->rows, W->rows, W->cols, W->count) || !given(Y, 16) ||
      !given(starts, 4))
    return SPL_ERR_INVALID_ARG;
  const int64_t bytes = X->rows * W->rows * type_bytes(dtype);
  if (!apart(Y, bytes, *X) || !apart(Y, bytes, *W)) return SPL_ERR_INVALID_ARG;
  if (X->rows > kMaxCols || W->rows >= kMaxN) return SPL_ERR_UNSUPPORTED;
  Fp8GemmArgs a{};
  a.x = spl::fp8_view(*X), a.w = spl::fp8_view(*W);
  a.M = X->rows, a.N = W->rows, a.blocks = a.w.pitch / 128, a.dtype = dtype, a.y = Y;
  a.mode = spl::kFp8Rows, a.starts = starts, a.groups = (int32_t)W->count;
  (void)hipGetLastError();
  return launched(spl::launch_fp8_gemm(a, stream));
}

int64_t spl_linear_fp8_grouped_rows_workspace_bytes(int64_t M, int64_t N, int64_t cols, int64_t experts) {
  return product_ok(M, N, cols, experts) ? (M == 0 ? 0 : rows_workspace(M, N, cols, experts)) : -1;
}
spl_status spl_linear_fp8_grouped_rows(const void* X, int32_t x_dtype, int64_t M, int64_t row_stride,
                                       const spl_fp8_matrix* W, const int32_t* starts, int32_t dtype, void* Y,
                                       void* workspace, hipStream_t stream) {
  if (!starts) return SPL_ERR_INVALID_ARG;
  return rows_product(X, x_dtype, M, row_stride, W, starts, dtype, Y, workspace, stream);
}

spl_status spl_linear_fp8_grouped_weight_grad(const spl_fp8_matrix* dYt, const spl_fp8_matrix* Xt,
                                              const int32_t* starts, int64_t experts, int64_t tokens, int32_t dtype,
                                              void* dW, hipStream_t stream) {
  spl_status st = check_matrix(dYt);
  if (st == SPL_OK) st = check_matrix(Xt);
  if (st != SPL_OK) return st;
  if (!float_type(dtype)) return SPL_ERR_UNSUPPORTED;
  const int64_t want = spl_fp8_grouped_cols(tokens, experts);
  if (want < 0 || dYt->cols != Xt->cols || dYt->cols < want || dYt->count != 1 || Xt->count != 1 || !given(starts, 4) ||
      !given(dW, 16) || Xt->rows > kMaxBytes / dYt->rows / experts)
    return SPL_ERR_INVALID_ARG;
  const int64_t bytes = experts * dYt->rows * Xt->rows * type_bytes(dtype);
  if (!apart(dW, bytes, *dYt) || !apart(dW, bytes, *Xt)) return SPL_ERR_INVALID_ARG;
  if (Xt->rows >= kMaxN) return SPL_ERR_UNSUPPORTED;
  Fp8GemmArgs a{};
  a.x = spl::fp8_view(*dYt), a.w = spl::fp8_view(*Xt);
  a.M = dYt->rows, a.N = Xt->rows, a.blocks = a.w.pitch / 128, a.dtype = dtype, a.y = dW;
  a.mode = spl::kFp8Sum, a.starts = starts, a.groups = (int32_t)experts, a.tokens = (int32_t)tokens;
  (void)hipGetLastError();
  return launched(spl::launch_fp8_gemm(a, stream));
}

// The workspace of both gradients: dY's codes, its transpose's, those of X's transpose, the split sums of either product.
struct GradSpace {
  int64_t tokens;                                       // columns of the transposes
  int64_t q, q_scales, qt, qt_scales, xt, xt_scales, partial, bytes;   // offsets
};
static bool grad_space(int64_t M, int64_t N, int64_t K, int64_t experts, GradSpace* g) {
  if (M < 1 || M > kMaxCols || N < 1 || N > kMaxCols || K < 1 || K > kMaxCols || experts < 0 || experts > kMaxCount)
    return false;
  g->tokens = experts ? spl_fp8_grouped_cols(M, experts) : M;
  if (g->tokens < 0 || !sizes_ok(M, N, 1) || !sizes_ok(K, N, experts ? experts : 1) || !sizes_ok(N, g->tokens, 1) ||
      !sizes_ok(K, g->tokens, 1))
    return false;
  int64_t at = 0;
  const auto take = [&](int64_t n) {
    const int64_t here = at;
    at += align256(n);
    return here;
  };
  g->q = take(M * spl::fp8_pitch(N)), g->q_scales = take(M * spl::fp8_spitch(N));
  g->qt = take(N * spl::fp8_pitch(g->tokens)), g->qt_scales = take(N * spl::fp8_spitch(g->tokens));
  g->xt = take(K * spl::fp8_pitch(g->tokens)), g->xt_scales = take(K * spl::fp8_spitch(g->tokens));
  int64_t most = 0;
  if (!experts) {
    const int64_t x = codes_workspace(M, K, N), w = codes_workspace(N, K, M);
    most = x > w ? x : w;
  }
  g->partial = take(most);
  g->bytes = at;
  return true;
}

int64_t spl_linear_fp8_grad_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t experts) {
  GradSpace g;
  if (M == 0) return N >= 1 && N <= kMaxCols && K >= 1 && K <= kMaxCols && experts >= 0 && experts <= kMaxCount ? 0 : -1;
  return grad_space(M, N, K, experts, &g) ? g.bytes : -1;
}
spl_status spl_linear_fp8_grad(const void* dY, int64_t dy_stride, const void* X, int64_t x_stride, int32_t dtype,
                               int64_t M, const spl_fp8_matrix* Wt, const int32_t* starts, int32_t grad_dtype,
                               void* dX, void* dW, void* workspace, hipStream_t stream) {
  const spl_status st = check_matrix(Wt);
  if (st != SPL_OK) return st;
  if (!half_type(dtype) || !float_type(grad_dtype)) return SPL_ERR_UNSUPPORTED;
  const int64_t N = Wt->cols, K = Wt->rows, experts = starts ? Wt->count : 0;
  if (M < 0 || (!starts && Wt->count != 1) || !aligned(starts, 4) || !aligned(dX, 16) || !aligned(dW, 16) || (!dX && !dW) ||
      N > kMaxBytes / K / Wt->count)
    return SPL_ERR_INVALID_ARG;
  (void)hipGetLastError();
  if (M == 0) {
    if (!dW) return SPL_OK;
    return launched(spl::launch_zero_fill(dW, Wt->count * N * K * (grad_dtype == SPL_F32 ? 2 : 1), stream));
  }
  GradSpace g;
  if (!grad_space(M, N, K, experts, &g)) return SPL_ERR_UNSUPPORTED;
  if (!given(dY, 2) || !given(X, 2) || dy_stride < N || x_stride < K || dy_stride > kMaxBytes / M ||
      x_stride > kMaxBytes / M || !given(workspace, 256))
    return SPL_ERR_INVALID_ARG;
  const int64_t dx_bytes = M * K * 2, dw_bytes = Wt->count * N * K * type_bytes(grad_dtype);
  if (!apart(dX, dx_bytes, *Wt) || !apart(dW, dw_bytes, *Wt) || !apart(dX, dx_bytes, dW, dw_bytes) ||
      !apart(dX, dx_bytes, workspace, g.bytes) || !apart(dW, dw_bytes, workspace, g.bytes))
    return SPL_ERR_INVALID_ARG;                         // (dY and X have been read when these are written)
  uint8_t* base = static_cast<uint8_t*>(workspace);
  const auto view = [&](int64_t codes, int64_t scales, int64_t rows, int64_t cols) {
    spl_fp8_matrix m{};
    m.codes = base + codes, m.scales = base + scales, m.rows = rows, m.cols = cols, m.count = 1, m.block = 1;
    return spl::fp8_view(m);
  };
  const spl::Fp8View q = view(g.q, g.q_scales, M, N), qt = view(g.qt, g.qt_scales, N, g.tokens),
                     xt = view(g.xt, g.xt_scales, K, g.tokens);
  spl::Fp8QuantArgs z{};
  z.X = dY, z.row_stride = dy_stride, z.rows = M, z.cols = N, z.count = 1, z.starts = starts, z.groups = (int32_t)experts;
  if (dX) z.out = q;
  if (dW) z.out_t = qt;
  hipError_t e = spl::launch_fp8_quantize(z, dtype, stream);
  if (e == hipSuccess && dW) {
    z.X = X, z.row_stride = x_stride, z.cols = K, z.out = spl::Fp8View{}, z.out_t = xt;
    e = spl::launch_fp8_quantize(z, dtype, stream);
  }
  void* partial = base + g.partial;
  if (e == hipSuccess && dX && starts)                  // before the product, which then writes the rows of experts
    e = spl::launch_fp8_clear_rest(starts, (int32_t)experts, M, K, dX, stream);
  if (e == hipSuccess && dX) {
    Fp8GemmArgs a{};
    a.x = q, a.w = spl::fp8_view(*Wt), a.M = M, a.N = K, a.blocks = a.w.pitch / 128, a.dtype = dtype, a.y = dX;
    a.mode = starts ? spl::kFp8Rows : spl::kFp8Plain, a.starts = starts, a.groups = (int32_t)experts;
    if (!starts && spl::fp8_partial_bytes(M, K, a.blocks) > 0) a.partial = partial;
    e = spl::launch_fp8_gemm(a, stream);
  }
  if (e == hipSuccess && dW) {
    Fp8GemmArgs a{};
    a.x = qt, a.w = xt, a.M = N, a.N = K, a.blocks = a.w.pitch / 128, a.dtype = grad_dtype, a.y = dW;
    a.mode = starts ? spl::kFp8Sum : spl::kFp8Plain, a.starts = starts, a.groups = (int32_t)experts;
    a.tokens = (int32_t)M;
    if (!starts && spl::fp8_partial_bytes(N, K, a.blocks) > 0) a.partial = partial;
    e = spl::launch_fp8_gemm(a, stream);
  }
  return launched(e);
}

int32_t spl_linear_fp8_kernel(int32_t form, int64_t M, int64_t N, int64_t cols, int64_t groups, int32_t x_dtype,
                              int32_t dtype) {
  if (form < 0 || form > 2 || M < 1 || !float_type(dtype) || (x_dtype != 0 && (!half_type(x_dtype) || form == 2))) return -1;
  Fp8GemmArgs a{};
  a.M = M, a.N = N, a.dtype = dtype;
  if (form == 2) {
    const int64_t want = spl_fp8_grouped_cols(cols, groups);
    if (want < 0 || !sizes_ok(M, want, 1) || !sizes_ok(N, want, 1) || N >= kMaxN || N > kMaxBytes / M / groups) return -1;
    a.blocks = (int32_t)(want / 128), a.mode = spl::kFp8Sum, a.groups = (int32_t)groups, a.tokens = (int32_t)cols;
    return spl::fp8_kernel(a);
  }
  const int64_t experts = form == 1 ? groups : 1;
  if (!product_ok(M, N, cols, experts) || N >= kMaxN || ((form == 1 || x_dtype) && M > kMaxCols)) return -1;
  a.blocks = (int32_t)(spl::fp8_pitch(cols) / 128), a.mode = form == 1 ? spl::kFp8Rows : spl::kFp8Plain;
  a.groups = (int32_t)experts;
  if (x_dtype && spl::fp8_fused(M, N, cols, experts)) a.x16 = &a;      // (looked at, not read)
  if (form == 0 && !a.x16 && spl::fp8_partial_bytes(M, N, a.blocks) > 0) a.partial = &a;
  return spl::fp8_kernel(a);
}

static bool adamw_types(const spl_adamw_types* ty) {
  return ty && float_type(ty->param_dtype) && float_type(ty->grad_dtype) &&
         (ty->copy_dtype == 0 || half_type(ty->copy_dtype)) && (ty->state_bits == 32 || ty->state_bits == 8);
}
static bool adamw_tensors(const spl_adamw_tensor* t, int64_t count, const spl_adamw_types* ty) {
  if (!adamw_types(ty) || count < 0 || count >= kMaxRows || (count > 0 && !t)) return false;
  const int64_t pb = ty->param_dtype == SPL_F32 ? 4 : 2, gb = ty->grad_dtype == SPL_F32 ? 4 : 2;
  const bool eight = ty->state_bits == 8;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (t[i].n < 0 || t[i].n >= (int64_t)1 << 40 || !isfinite(t[i].decay)) return false;
    if ((total += t[i].n) >= (int64_t)1 << 40) return false;
    if (t[i].n == 0) continue;
    if (!given(t[i].param, pb) || !given(t[i].grad, gb) || !given(t[i].m, eight ? 16 : 4) ||
        !given(t[i].v, eight ? 16 : 4) || (eight && (!t[i].m_scales || !t[i].v_scales)) ||
        (ty->copy_dtype != 0 && !given(t[i].copy, 2)))
      return false;
  }
  return spl::adamw_plan_chunks(t, count) < (int64_t)1 << 24;       // workgroups of one launch
}

int64_t spl_adamw_plan_chunks(const spl_adamw_tensor* tensors, int64_t count, const spl_adamw_types* types) {
  return adamw_tensors(tensors, count, types) ? spl::adamw_plan_chunks(tensors, count) : -1;
}
int64_t spl_adamw_plan_bytes(const spl_adamw_tensor* tensors, int64_t count, const spl_adamw_types* types) {
  return adamw_tensors(tensors, count, types) ? spl::adamw_plan_bytes(tensors, count) : -1;
}
// Whether an array that a step writes shares memory with another one (gradients,
// which are read, may be shared among themselves).
static bool adamw_overlap(const spl_adamw_tensor* t, int64_t count, const spl_adamw_types& ty) {
  struct Span {
    uintptr_t at, end;
    bool read;
  };
  std::vector<Span> spans;
  spans.reserve((size_t)count * 7);
  const auto add = [&](const void* p, int64_t bytes, bool read) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    spans.push_back(Span{at, at + (uintptr_t)bytes, read});
  };
  const int64_t pb = ty.param_dtype == SPL_F32 ? 4 : 2, gb = ty.grad_dtype == SPL_F32 ? 4 : 2;
  for (int64_t i = 0; i < count; ++i) {
    const int64_t n = t[i].n, blocks = (n + 127) / 128;
    if (n == 0) continue;
    add(t[i].param, n * pb, false), add(t[i].grad, n * gb, true);
    if (ty.copy_dtype) add(t[i].copy, n * 2, false);
    const int64_t state = ty.state_bits == 8 ? 128 * blocks : 4 * n;
    add(t[i].m, state, false), add(t[i].v, state, false);
    if (ty.state_bits == 8) add(t[i].m_scales, blocks, false), add(t[i].v_scales, blocks, false);
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t any = 0, written = 0;                          // where the spans so far end
  for (const Span& s : spans) {
    if (s.at < (s.read ? written : any)) return true;
    any = std::max(any, s.end);
    if (!s.read) written = std::max(written, s.end);
  }
  return false;
}
spl_status spl_adamw_plan(const spl_adamw_tensor* tensors, int64_t count, const spl_adamw_types* types,
                          void* host_plan) {
  if (!adamw_tensors(tensors, count, types) || (count > 0 && !given(host_plan, 8))) return SPL_ERR_INVALID_ARG;
  try {
    if (adamw_overlap(tensors, count, *types)) return SPL_ERR_INVALID_ARG;
  } catch (const std::bad_alloc&) {
    return SPL_ERR_OVERFLOW;
  }
  if (count > 0) spl::adamw_plan_write(tensors, count, *types, host_plan);
  return SPL_OK;
}

spl_status spl_adamw_step(const void* plan, int64_t chunks, const spl_adamw_types* types, double lr, double beta1,
                          double beta2, double eps, int64_t step, const int32_t* step_on_device,
                          const float* grad_scale, uint32_t seed, hipStream_t stream) {
  if (!adamw_types(types) || chunks < 0 || chunks >= (int64_t)1 << 24 || !isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) ||
      !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !isfinite(eps) || (!step_on_device && (step < 1 || step >= kMaxRows)) ||
      !aligned(step_on_device, 4) || !aligned(grad_scale, 4))
    return SPL_ERR_INVALID_ARG;
  if (chunks == 0) return SPL_OK;
  if (!given(plan, 16)) return SPL_ERR_INVALID_ARG;
  spl::AdamwHyper h{};
  h.lr = lr, h.beta1 = beta1, h.beta2 = beta2, h.eps = eps, h.step = step, h.step_on_device = step_on_device;
  h.grad_scale = grad_scale, h.seed = seed;
  (void)hipGetLastError();
  return launched(spl::launch_adamw(plan, chunks, *types, h, stream));
}

}  // extern "C"
