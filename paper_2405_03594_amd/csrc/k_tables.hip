// Block tables and slots of a batch's new tokens (spl_block_tables).
//
// Everything follows from two exclusive prefix sums over the requests: of the
// new tokens (row_start) and of the pages they need beyond those held.  Each
// workgroup computes both sums for itself, 1024 requests at a time, keeps that
// chunk's sums in LDS, and then serves the rows of its own window of tokens and
// its share of the new pages by binary search in LDS.  So one launch does it
// all, with nothing exchanged between workgroups: a token in a new page takes
// the page from the free list, as the workgroup that writes the table does.
// Bound: the latency of a chunk (two loads, a scan over four waves, ten LDS
// steps of the search); the bytes are a few hundred KB at most.  Measured: 3
// requests of a token each 4.8 us, 512 requests of 16384 tokens 7.9.
#include "spl_common.h"

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 4;                       // requests of one thread in a chunk
constexpr int kChunk = kThreads * kPer;

struct TablesArgs {
  const int32_t* cached;
  const int32_t* fresh;
  int32_t* table;
  const int32_t* free_pages;
  const int32_t* free_head;
  int32_t* row_start;
  int32_t* lens;
  int32_t* positions;
  int32_t* slots;
  int32_t* state;
  int64_t width;
  int64_t free_count;
  int64_t tokens;
  int64_t window;                             // tokens of a workgroup
  int32_t requests;
  int32_t shift;                              // log2 of the page
};

// Index of the last of a[0..n) that is <= x, for ascending a with a[0] <= x.
__device__ __forceinline__ int last_le(const int64_t* a, int n, int64_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int64_t wave_scan(int64_t x, int lane) {
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

__global__ __launch_bounds__(kThreads) void k_block_tables(TablesArgs a) {
  __shared__ int64_t row_s[kChunk + 1], page_s[kChunk + 1];     // sums before each request of the chunk
  __shared__ int32_t cached_s[kChunk], have_s[kChunk];
  __shared__ int64_t wave_s[3][kThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t page = (int64_t)1 << a.shift;
  const int64_t w0 = (int64_t)blockIdx.x * a.window;
  const int64_t w1 = w0 + a.window < a.tokens ? w0 + a.window : a.tokens;
  int64_t head = *a.free_head;
  head = head < 0 ? 0 : (head > a.free_count ? a.free_count : head);
  int64_t rows_before = 0, pages_before = head, missing = 0;

  for (int32_t base = 0; base < a.requests; base += kChunk) {
    const int count = a.requests - base < kChunk ? a.requests - base : kChunk;
    int64_t n[kPer], need[kPer], rows = 0, pages = 0;
    int32_t c[kPer], have[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = tid * kPer + i;
      const bool in = k < count;
      const int32_t ci = in ? a.cached[base + k] : 0, ni = in ? a.fresh[base + k] : 0;
      c[i] = ci < 0 ? 0 : ci;
      n[i] = ni < 0 ? 0 : ni;
      const int64_t len = c[i] + n[i];
      const int64_t h = (c[i] + page - 1) >> a.shift, w = (len + page - 1) >> a.shift;
      have[i] = (int32_t)(h < a.width ? h : a.width);
      need[i] = (w < a.width ? w : a.width) - have[i];
      rows += n[i];
      pages += need[i];
      if (in && blockIdx.x == 0) a.lens[base + k] = (int32_t)(len < INT32_MAX ? len : INT32_MAX);
    }
    // sums over the workgroup
    const int64_t rs = wave_scan(rows, lane), ps = wave_scan(pages, lane);
    __syncthreads();                                            // the previous chunk's readers are done
    if (lane == 63) wave_s[0][wave] = rs, wave_s[1][wave] = ps;
    __syncthreads();
    int64_t row = rows_before + rs - rows, pg = pages_before + ps - pages;
    for (int w = 0; w < wave; ++w) row += wave_s[0][w], pg += wave_s[1][w];
    int64_t row_end = rows_before, page_end = pages_before;
    for (int w = 0; w < kThreads / 64; ++w) row_end += wave_s[0][w], page_end += wave_s[1][w];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = tid * kPer + i;
      if (k < count) {
        row_s[k] = row, page_s[k] = pg, cached_s[k] = c[i], have_s[k] = have[i];
        if (blockIdx.x == 0) {
          a.row_start[base + k] = (int32_t)(row < INT32_MAX ? row : INT32_MAX);
          // of the tokens that have a row (the others are missing as such): those in the
          // page begun before, in new pages handed out, and the rest
          const int64_t in_rows = a.tokens - row, m = in_rows < 0 ? 0 : (in_rows < n[i] ? in_rows : n[i]);
          const int64_t room = m > 0 ? (int64_t)have[i] * page - c[i] : 0;
          int64_t got = 0;
          if (room > 0 && a.table[(base + k) * a.width + have[i] - 1] >= 0) got += room < m ? room : m;
          int64_t given = a.free_count - pg;
          given = given < 0 ? 0 : (given < need[i] ? given : need[i]);
          const int64_t rest = m - (room > 0 ? room : 0);
          if (rest > 0 && c[i] <= (int64_t)have[i] * page) got += rest < given * page ? rest : given * page;
          missing += m - got;
        }
      }
      row += n[i];
      pg += need[i];
    }
    if (tid == 0) row_s[count] = row_end, page_s[count] = page_end;
    __syncthreads();

    // the new pages of this chunk, over all workgroups
    for (int64_t p = page_s[0] + (int64_t)blockIdx.x * kThreads + tid; p < page_end;
         p += (int64_t)gridDim.x * kThreads) {
      const int k = last_le(page_s, count, p);
      a.table[(base + k) * a.width + have_s[k] + (p - page_s[k])] = p < a.free_count ? a.free_pages[p] : -1;
    }
    // the tokens of this chunk in this workgroup's window
    const int64_t t0 = w0 > row_s[0] ? w0 : row_s[0], t1 = w1 < row_end ? w1 : row_end;
    for (int64_t t = t0 + tid; t < t1; t += kThreads) {
      const int k = last_le(row_s, count, t);
      const int64_t pos = cached_s[k] + (t - row_s[k]), j = pos >> a.shift;
      int64_t entry = -1;
      if (j < have_s[k]) {
        entry = a.table[(base + k) * a.width + j];
      } else {
        const int64_t p = page_s[k] + (j - have_s[k]);
        if (j < a.width && p < a.free_count) entry = a.free_pages[p];
      }
      const int64_t slot = entry < 0 ? -1 : (entry << a.shift) + (pos & (page - 1));
      a.positions[t] = (int32_t)(pos < INT32_MAX ? pos : INT32_MAX);
      a.slots[t] = slot > INT32_MAX ? -1 : (int32_t)slot;
    }
    rows_before = row_end;
    pages_before = page_end;
  }
  // rows past the last request's
  for (int64_t t = (w0 > rows_before ? w0 : rows_before) + tid; t < w1; t += kThreads) {
    a.positions[t] = 0;
    a.slots[t] = -1;
  }
  if (blockIdx.x != 0) return;
  const int64_t ms = wave_scan(missing, lane);
  if (lane == 63) wave_s[2][wave] = ms;
  __syncthreads();
  if (tid == 0) {
    int64_t m = rows_before > a.tokens ? rows_before - a.tokens : 0;
    for (int w = 0; w < kThreads / 64; ++w) m += wave_s[2][w];
    a.row_start[a.requests] = (int32_t)(rows_before < INT32_MAX ? rows_before : INT32_MAX);
    a.state[0] = (int32_t)(pages_before < a.free_count ? pages_before : a.free_count);
    a.state[1] = (int32_t)(m < INT32_MAX ? m : INT32_MAX);
  }
}

}  // namespace

namespace spl {

hipError_t launch_block_tables(const int32_t* cached, const int32_t* fresh, int64_t requests, int64_t tokens,
                               int32_t page, int32_t* table, int64_t width, const int32_t* free_pages,
                               int64_t free_count, const int32_t* free_head, int32_t* row_start, int32_t* lens,
                               int32_t* positions, int32_t* slots, int32_t* state, hipStream_t s) {
  // one row per thread, up to two workgroups a CU
  const int64_t most = 2 * (int64_t)device_cus();
  int64_t groups = (tokens + kThreads - 1) / kThreads;
  groups = groups < 1 ? 1 : (groups > most ? most : groups);
  const int64_t window = ((tokens + groups - 1) / groups + kThreads - 1) / kThreads * kThreads;
  TablesArgs a{cached, fresh,     table,     free_pages, free_head, row_start, lens,              positions,
               slots,  state,     width,     free_count, tokens,    window,    (int32_t)requests, __builtin_ctz((unsigned)page)};
  k_block_tables<<<dim3((unsigned)groups), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace spl
