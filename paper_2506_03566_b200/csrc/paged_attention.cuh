// Tree-masked attention over pages: what the two kernels and their host side share.
#pragma once
#include "paged.cuh"
#include <cuda.h>

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
  float2* ml;                          // NULL, or [batch][rows][Hq]: what a query row leaves for the slots' weights
};
// A query row's reference maximum (scores times scale times log2 e) and the inverse of its sum; a row that sees nothing weighs nothing.
__device__ __forceinline__ float2 paged_ml(float m, float l) {
  return l == 0.f ? make_float2(INFINITY, 0.f) : make_float2(m == -INFINITY ? 0.f : m, 1.f / l);
}

// SIMT kernel: every type, head dimension and page size
size_t paged_attn_simt_workspace(int batch, int rows, int Hq, int Hkv, int d);
// scores: NULL, or where the rows leave theirs (times scale times log2 e, -inf where a slot is not seen) for the slots' weights,
// [batch][Hkv][rows * G][paged_simt_scores_ld]
long long paged_simt_scores_ld(int max_pages, int page);
void launch_paged_attn_simt(Launcher& L, const PagedAttnArgs& a, const void* pool, int dtype, float* scores = nullptr);

// tcgen05 kernel: bf16, head dimension 64 or 128, pages of 16 .. 256 slots (powers of two), at most 128 query heads per KV head,
// scale > 0
bool paged_attn_tc_supported(const poss_page_pool& p, int G, float scale);
size_t paged_attn_tc_workspace(const poss_page_pool& p, int batch, int rows, int Hq, int max_pages);
// mass (with room for scores): the slots' weights too, for calls of so few lines (rows x heads of a group) that paged_attn_tc_scores, the
// bytes of that room, is not 0
struct PagedMassArgs;
size_t paged_attn_tc_scores(const poss_page_pool& p, int batch, int rows, int Hq, int max_pages);
void launch_paged_attn_tc(Launcher& L, const PagedAttnArgs& a, const void* pool, const poss_page_pool& p,
                          const PagedMassArgs* mass = nullptr);

// Tensor maps of the tcgen05 kernels.  The layer as a matrix of slots: rows (page, keys / values, head, slot), head_dim columns, a box of
// `slots` rows times 64 columns; rows_total is the first row behind it.  The queries: columns, heads of a group, groups (KV heads), tree
// rows, sequences, a box of `tree_rows` tree rows of one KV head times 64 columns; rows behind the call's last one arrive as zeros.
bool paged_take_lost_load();             // whether this launch is to lose a load (poss_debug_paged_lose_load); counts it
bool paged_kv_map(CUtensorMap* map, const PagedAttnArgs& a, const void* layer, int slots);
bool paged_q_map(CUtensorMap* map, const PagedAttnArgs& a, int tree_rows);

// The weight that every slot draws, from the queries and the rows' maxima and sums (a.ml)
struct PagedMassArgs {
  PagedAttnArgs a;
  float* mass;                         // the layer's: [batch][Hkv][mass_slots]
  long long mass_slots;
  const float* weights;                // NULL, or [batch][rows]
  float scale_log2;
  // NULL, or scratch for the scores [batch][Hkv][rows * G][ld]: of the tcgen05 attention ld whole tiles of 64 slots (paged_attn_tc_scores bytes),
  // of the SIMT attention paged_simt_scores_ld, and batch * rows * Hq * ld * 4 bytes
  float* scores;
};
// tcgen05 kernel: the shapes of the attention's
void launch_paged_mass_tc(Launcher& L, const PagedMassArgs& s, const void* pool);
// from the scores that the SIMT attention has left
void launch_paged_mass_scores(Launcher& L, const PagedMassArgs& s);
// SIMT kernel: every type and shape
void launch_paged_mass_simt(Launcher& L, const PagedMassArgs& s, const void* pool, int dtype);

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
