// Shared by the kernels of the attention half of a layer (not part of the
// ABI): the 4-bit cache's page layout and what the launchers take.
#pragma once

#include "spl_common.h"

namespace spl {

// Geometry of one head's region of a page (the layout stands in spl.h).
struct PageGeom {
  int32_t dim;                                  // D
  int32_t page;                                 // tokens
  int32_t groups;                               // D / 32
  int32_t scale_bytes;                          // of a token: groups rounded up to a power of two
  int32_t unit;                                 // channels of V stored together
  int32_t bytes;                                // of the region
};
inline __host__ __device__ PageGeom page_geom(int32_t dim, int32_t page) {
  PageGeom g;
  g.dim = dim;
  g.page = page;
  g.groups = dim / 32;
  g.scale_bytes = g.groups <= 2 ? 2 : (g.groups <= 4 ? 4 : 8);
  g.unit = dim == 64 ? 4 : (dim == 256 ? 16 : 8);
  g.bytes = page * (dim + 2 * g.scale_bytes);
  return g;
}

// Threads that a launch can have in x.
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;

struct NormRopeArgs {
  spl_heads q, k, v;                            // v only with a cache
  void* q_out;
  void* k_out;                                  // may be NULL with a cache
  const void* wq;
  const void* wk;                               // NULL: no norm
  const int32_t* positions;
  const float* rope;
  int64_t rope_rows;
  const int32_t* slots;
  spl_kv_cache cache;                           // data NULL: none
  int64_t tokens;
  int32_t dim;
  int32_t rot;
  int32_t interleaved;
  float eps;
};
hipError_t launch_norm_rope(const NormRopeArgs& a, int32_t dtype, hipStream_t s);
inline int64_t cache_read_threads(const spl_kv_cache& c, int64_t tokens) { return tokens * c.heads * (c.head_dim / 8); }
hipError_t launch_cache_read(const spl_kv_cache& c, const int32_t* slots, int64_t tokens, void* k, void* v,
                             hipStream_t s);

struct NormRopeGradArgs {
  spl_heads dq, dk, q, k;
  void* dq_out;
  void* dk_out;
  const void* wq;
  const void* wk;
  float* dwq;
  float* dwk;
  const int32_t* positions;
  const float* rope;
  int64_t rope_rows;
  int64_t tokens;
  int32_t dim;
  int32_t rot;
  int32_t interleaved;
  float eps;
  float* partial;                               // norm_rope_grad_bytes
};
int64_t norm_rope_grad_bytes(int64_t tokens, int32_t q_heads, int32_t k_heads, int32_t dim);
hipError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int32_t dtype, hipStream_t s);

hipError_t launch_block_tables(const int32_t* cached, const int32_t* fresh, int64_t requests, int64_t tokens,
                               int32_t page, int32_t* table, int64_t width, const int32_t* free_pages,
                               int64_t free_count, const int32_t* free_head, int32_t* row_start, int32_t* lens,
                               int32_t* positions, int32_t* slots, int32_t* state, hipStream_t s);

struct AttnArgs {
  spl_heads q;
  spl_kv_cache cache;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* row_start;
  void* out;
  float* lse;                                   // may be NULL
  int64_t width;
  int64_t tokens;
  int64_t requests;
  int64_t max_new;                              // 0: not known
  int64_t max_len;                              // 0: not known
  float scale;
  int32_t window;                               // 0: none
  void* workspace;
};
// How a call is launched: k_attn_rows for all requests (prefill_tiles 0), or
// k_attn_prefill for those of more than kFewRows rows and k_attn_rows for the
// others, a tile each (tiles 0: there are none).
constexpr int kFewRows = 16;                    // of a tile of k_attn_rows
constexpr int kPrefillRows = 128;               // of a tile of k_attn_prefill
constexpr int kPrefillThreads = 512;            // of a workgroup of it
struct AttnPlan {
  int64_t tiles, prefill_tiles;
  int group;                                    // query heads of a key head
  int direct;                                   // a tile is a request
  int wide;                                     // tiles of twice the rows
  int two;                                      // 256 channels: two waves a SIMD, not one
  int splits, chunk;                            // of the tokens in k_attn_rows; chunk in its steps
  int most_splits;                              // of this call under any window: the workspace's
  int snake;                                    // requests of a round of the chip, 0: in their order
};
hipError_t launch_attn_prefill(const AttnArgs& a, const AttnPlan& p, hipStream_t s);
int64_t attn_workspace_bytes(const AttnArgs& a);                // the window does not count
bool attn_fits(const AttnArgs& a);                              // into launches; the window does not count
hipError_t launch_attn(const AttnArgs& a, hipStream_t s);

}  // namespace spl
