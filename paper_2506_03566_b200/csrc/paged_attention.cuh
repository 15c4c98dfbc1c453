// Tree-masked attention over pages: what the two kernels and their host side share.
#pragma once
#include "paged.cuh"

struct PagedAttnArgs {
  PageGeo g;
  int layer, batch, rows, Hq, G;
  const void* q;
  long long ld_q;                      // elements between consecutive rows
  const int32_t *prefix_len, *n_rows;
  const uint64_t* mask;
  int mask_words;
  float scale;
  void* out;
  void* ws;
  int32_t* status;
};

// SIMT kernel: every type, head dimension and page size
size_t paged_attn_simt_workspace(int batch, int rows, int Hq, int Hkv, int d);
void launch_paged_attn_simt(Launcher& L, const PagedAttnArgs& a, const void* pool, int dtype);

// tcgen05 kernel: bf16, head dimension 64 or 128, pages of 16 .. 256 slots (powers of two), at most 128 query heads per KV head,
// scale > 0
bool paged_attn_tc_supported(const poss_page_pool& p, int G, float scale);
size_t paged_attn_tc_workspace(const poss_page_pool& p, int batch, int rows, int Hq, int max_pages);
void launch_paged_attn_tc(Launcher& L, const PagedAttnArgs& a, const void* pool, const poss_page_pool& p);

// visibility of 32 consecutive slots from `key0` on: every slot below `prefix`, slot prefix + t iff bit t of
// (lo, hi) is set.  The mask has already been cut to the rows that exist, so slots behind them come out unseen.
__host__ __device__ __forceinline__ uint32_t paged_visible32(int key0, int prefix, uint64_t lo, uint64_t hi) {
  const int t0 = key0 - prefix;
  if (t0 <= -32) return 0xffffffffu;
  if (t0 < 0) return ((uint32_t)lo << (-t0)) | ((1u << (-t0)) - 1u);
  if (t0 >= 128) return 0u;
  if (t0 >= 64) return (uint32_t)(hi >> (t0 - 64));
  return (uint32_t)(lo >> t0) | (t0 > 32 ? (uint32_t)(hi << (64 - t0)) : 0u);
}
// a row's ancestor bits, cut to the n rows that exist
__device__ __forceinline__ void paged_row_mask(const uint64_t* mask, size_t row, int words, int n, uint64_t* lo,
                                               uint64_t* hi) {
  *lo = mask[row * words];
  *hi = words > 1 ? mask[row * words + 1] : 0ull;
  if (n < 64) { *lo &= (1ull << n) - 1; *hi = 0; }
  else if (n < 128) *hi &= (1ull << (n - 64)) - 1;
}
