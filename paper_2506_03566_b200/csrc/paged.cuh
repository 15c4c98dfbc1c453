// Paged caches: the geometry and the bounds rules that every kernel of the paged calls shares.
#pragma once
#include "poss_internal.cuh"
#include "../../include/poss_paged.h"

// What a kernel needs to find a slot.  Offsets inside a pool pass 32 bits early (a 32-layer cache of 131072 slots holds
// 2^33 elements), so they are formed in 64 bits; slot numbers and table places fit 31 (checked on the host).
struct PageGeo {
  int n_layers, n_pages, Hkv, page, d;
  const int32_t* tables;   // [sequences][max_pages]
  int max_pages;
};

// The page of table place `i` of a sequence, or -1 where the table has none: places behind the table, negative
// entries and entries past the pool are never followed.
__host__ __device__ __forceinline__ int page_at(const int32_t* table, int max_pages, int n_pages, int i) {
  if (i < 0 || i >= max_pages) return -1;
  const int p = table[i];
  return p >= 0 && p < n_pages ? p : -1;
}
// element offset of (layer, page, keys 0 / values 1, head) inside the pool: the first slot's first element
__host__ __device__ __forceinline__ size_t page_offset(const PageGeo& g, int layer, int page, int kv, int head) {
  return ((((size_t)layer * g.n_pages + page) * 2 + kv) * g.Hkv + head) * ((size_t)g.page * g.d);
}

// A sequence's lengths as the kernels use them.  Out of range (negative, more rows than the call has, more slots than
// its table has places): no rows, no slots, `bad` set.
struct SeqLen {
  int prefix, rows;
  bool bad;
};
__host__ __device__ __forceinline__ SeqLen seq_len_of(int prefix, int rows, int max_rows, long long slots) {
  SeqLen s;
  s.bad = prefix < 0 || rows < 0 || rows > max_rows || (long long)prefix + rows > slots;
  s.prefix = s.bad ? 0 : prefix;
  s.rows = s.bad ? 0 : rows;
  return s;
}

__device__ __forceinline__ void raise_status(int32_t* status, int code) {
  if (status) atomicMax(status, code);
}

// 2^x, 2^-22 relative
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// two fp32 operations per instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 w, x, y;\n\t"
      "mov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

inline int page_pool_check(const poss_page_pool* p) {
  if (!p || p->n_layers < 1 || p->n_pages < 1 || p->n_kv_heads < 1 || p->page_slots < 1) return POSS_E_INVALID;
  if (p->dtype != POSS_FP32 && p->dtype != POSS_BF16) return POSS_E_INVALID;
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return POSS_E_SHAPE;
  if (p->page_slots > POSS_MAX_PAGE_SLOTS || p->n_kv_heads > 1024) return POSS_E_CAPACITY;
  // rows of one layer (page, keys / values, head, slot) are counted in 31 bits
  if ((long long)p->n_pages * 2 * p->n_kv_heads * p->page_slots >= (1ll << 31)) return POSS_E_CAPACITY;
  return POSS_OK;
}
// a table of max_pages places and a batch that the kernels' index arithmetic covers
inline int page_table_check(const poss_page_pool* p, int max_pages, int batch) {
  if (max_pages < 1 || batch < 1) return POSS_E_INVALID;
  if (batch > POSS_MAX_PAGED_BATCH) return POSS_E_CAPACITY;
  if ((long long)max_pages * p->page_slots >= (1ll << 30)) return POSS_E_CAPACITY;
  return POSS_OK;
}
inline PageGeo page_geo(const poss_page_pool* p, const int32_t* tables, int max_pages) {
  PageGeo g;
  g.n_layers = p->n_layers; g.n_pages = p->n_pages; g.Hkv = p->n_kv_heads; g.page = p->page_slots; g.d = p->head_dim;
  g.tables = tables; g.max_pages = max_pages;
  return g;
}
// do two arrays of na and nb bytes share some (a missing one shares none)
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && x < y + nb && y < x + na;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// SMs of the current device (148 when it cannot be asked: a grid size, nothing else depends on it)
int current_sm_count();
