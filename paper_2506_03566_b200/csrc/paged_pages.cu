// Pages of a cache: writing new rows, committing accepted paths, remapping sequences.
//
// All of it is data movement.  A row of one (layer, keys / values, head) is d contiguous elements (64 to 512 bytes) and
// moves in 16-byte pieces; consecutive slots of a page are contiguous, so what a page copy moves is one run per head.
#include "paged.cuh"

POSS_TRACE_REGISTER()

int current_sm_count() {
  static int known[PerDeviceFlags::MAX_DEVICES];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= PerDeviceFlags::MAX_DEVICES) return 148;
  if (!known[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 148;
    known[dev] = n;
  }
  return known[dev];
}

namespace {

// ------------------------------------------------------------------ append
// One warp per new row: it reads the row's keys and values (n_kv_heads x d elements each, contiguous) and writes one
// run of d elements per head; eight pieces of 16 bytes per lane are on their way at a time.  For a tree or a token the time is
// three trips to memory (lengths, table, data): 2 to 3 us of a captured graph.
template <int ES>
__global__ void __launch_bounds__(256) k_pages_append(PageGeo g, int layer, char* pool, int batch, int rows,
                                                      const char* k, const char* v, long long ld_bytes,
                                                      const int32_t* prefix_len, const int32_t* n_rows,
                                                      int32_t* status) {
  pdl_enter(POSS_K_PAGES_APPEND);
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (item >= (long long)batch * rows) return;
  const int b = (int)(item / rows), r = (int)(item - (long long)b * rows);
  const SeqLen s = seq_len_of(prefix_len[b], n_rows ? n_rows[b] : rows, rows, (long long)g.max_pages * g.page);
  if (s.bad && r == 0 && lane == 0) raise_status(status, POSS_E_INVALID);
  if (r >= s.rows) return;
  const int slot = s.prefix + r, place = slot / g.page, off = slot - place * g.page;
  const int p = page_at(g.tables + (size_t)b * g.max_pages, g.max_pages, g.n_pages, place);
  if (p < 0) {
    if (lane == 0) raise_status(status, POSS_E_INVALID);
    return;
  }
  const int per_head = g.d * ES / 16, n = g.Hkv * per_head;         // 16-byte pieces per head / per row
  const size_t head_bytes = (size_t)g.page * g.d * ES;
  char* const dk = pool + (page_offset(g, layer, p, 0, 0) + (size_t)off * g.d) * ES;
  char* const dv = dk + (size_t)g.Hkv * head_bytes;
  const char* const sk = k + (size_t)item * ld_bytes;
  const char* const sv = v + (size_t)item * ld_bytes;
  for (int i0 = lane; i0 < n; i0 += 128) {
    uint4 a[4], c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + 32 * j;
      if (i < n) {
        a[j] = *reinterpret_cast<const uint4*>(sk + (size_t)i * 16);
        c[j] = *reinterpret_cast<const uint4*>(sv + (size_t)i * 16);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + 32 * j;
      if (i < n) {
        const int h = i / per_head;
        const size_t o = h * head_bytes + (size_t)(i - h * per_head) * 16;
        *reinterpret_cast<uint4*>(dk + o) = a[j];
        *reinterpret_cast<uint4*>(dv + o) = c[j];
      }
    }
  }
}

// ------------------------------------------------------------------ compact
// One block per (layer, keys / values, sequence).  A path is increasing, so path[k] >= k: a target slot may be a later
// step's source, and every source of a head is read before the head's first target is written.
// What bounds it: the chain lengths and path -> table -> rows -> their new places.  16 sequences over 32 layers, 17 MB to and
// fro at the most: 7.3 us (the bytes alone 2.6); one sequence over 2 layers: 2.2 us, most of it the launch.
template <int ES>
__global__ void __launch_bounds__(256) k_pages_compact(PageGeo g, char* pool, const int32_t* prefix_len,
                                                       const int32_t* path, const int32_t* n_accepted,
                                                       int32_t* out_len, int32_t* status) {
  __shared__ int s_src[POSS_MAX_DEPTH], s_dst[POSS_MAX_DEPTH];      // page * page_slots + slot inside it
  pdl_enter(POSS_K_PAGES_COMPACT);
  const int b = blockIdx.y, layer = blockIdx.x >> 1, kv = blockIdx.x & 1, t = threadIdx.x;
  const int prefix = prefix_len[b], a = n_accepted[b];
  const int32_t* pb = path + (size_t)b * (POSS_MAX_DEPTH + 1);
  const int from = t < POSS_MAX_DEPTH ? pb[t + 1] : 0, before = t && t < POSS_MAX_DEPTH ? pb[t] : 0;   // (one trip with the lengths)
  const long long slots = (long long)g.max_pages * g.page;
  bool ok = prefix >= 0 && a >= 0 && a <= POSS_MAX_DEPTH && (long long)prefix + a < slots;
  if (ok && t < a) {
    ok = from > before && (long long)prefix + from < slots;
    if (ok) {
      const int32_t* table = g.tables + (size_t)b * g.max_pages;
      const int ss = prefix + from, ds = prefix + t + 1;
      const int sp = page_at(table, g.max_pages, g.n_pages, ss / g.page);
      const int dp = page_at(table, g.max_pages, g.n_pages, ds / g.page);
      ok = sp >= 0 && dp >= 0;
      s_src[t] = sp * g.page + ss % g.page;
      s_dst[t] = dp * g.page + ds % g.page;
    }
  }
  ok = __syncthreads_and(ok);
  if (blockIdx.x == 0 && t == 0) {
    out_len[b] = ok ? prefix + a + 1 : prefix;
    if (!ok) raise_status(status, POSS_E_INVALID);
  }
  if (!ok || a == 0) return;
  const int per_row = g.d * ES / 16, per_head = a * per_row;
  const int heads = per_head < 1024 ? 1024 / per_head : 1;          // heads whose rows fit four pieces per thread
  for (int h0 = 0; h0 < g.Hkv; h0 += heads) {
    const int n = (g.Hkv - h0 < heads ? g.Hkv - h0 : heads) * per_head;
    uint4 x[4];
    char* to[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = t + 256 * j;
      to[j] = nullptr;
      if (i < n) {
        const int h = i / per_head, rem = i - h * per_head, row = rem / per_row, piece = rem - row * per_row;
        const int src = s_src[row], dst = s_dst[row];
        if (src != dst) {
          const int sp = src / g.page, dp = dst / g.page;
          x[j] = *reinterpret_cast<const uint4*>(
              pool + (page_offset(g, layer, sp, kv, h0 + h) + (size_t)(src - sp * g.page) * g.d) * ES + piece * 16);
          to[j] = pool + (page_offset(g, layer, dp, kv, h0 + h) + (size_t)(dst - dp * g.page) * g.d) * ES + piece * 16;
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (to[j]) *reinterpret_cast<uint4*>(to[j]) = x[j];
  }
}

// ------------------------------------------------------------------ remap: the tables
// One block decides everything; the pool is touched by the copy kernel behind it.
//   1  refs minus the old holders plus the new ones; per page the number of new sequences that will write it and the
//      last of them in order (integer adds and maxima: any order gives the same)
//   2  a writer keeps its page iff all holders left are writers and it is the last (the others have taken fresh pages
//      by its turn); every other needed place of the write region is fresh.  Fresh places per sequence -> prefix sum
//   3  pages without a holder, in order, up to the number needed -> the fresh places, in order
// A page is free after the call iff step 1 leaves it without holders: where every holder is a writer the last stays.
// One block and not more: the steps depend on one another over the whole pool, and a grid's barrier costs more than the
// few thousand counts do.  64 sequences of up to 8 pages: 9.6 us beside the copies' 20 to 36; 4 of 44 pages: 5.5 beside 1.5, a chain of trips to
// memory and barriers.
constexpr int REMAP_THREADS = 1024;

struct RemapArgs {
  PageGeo g;
  int32_t* out_tables;
  int n_before, n_after;
  const int32_t *seq_len, *refs, *parents, *room;
  int32_t *out_refs, *out_len, *out_free, *status;
  int32_t *writers, *last;     // [n_pages]
  int32_t* free_list;          // [n_pages]
  int32_t* copies;             // [n_after][3]: source page, target page, slots (0: none)
  int fresh;                   // outputs that hold nothing yet: tables and lengths are emptied where it does not fit
};

struct RemapSeq { int parent, kept, room, needed; };
__device__ __forceinline__ RemapSeq remap_seq(const RemapArgs& a, int i, bool* bad) {
  RemapSeq s;
  s.parent = a.parents ? a.parents[i] : i;
  s.room = a.room ? a.room[i] : 0;
  s.kept = 0;
  *bad = s.parent >= a.n_before || s.room < 0;
  if (!*bad && s.parent >= 0) {
    s.kept = a.seq_len[s.parent];
    if (s.kept < 0) *bad = true;
  }
  const long long slots = (long long)a.g.max_pages * a.g.page;
  if (!*bad && (long long)s.kept + s.room > slots) *bad = true;
  if (*bad) { s.parent = -1; s.kept = 0; s.room = 0; }
  s.needed = (s.kept + s.room + a.g.page - 1) / a.g.page;
  return s;
}
// the page that place `at` of a new sequence takes over from its parent, -1 where there is none
__device__ __forceinline__ int remap_taken(const RemapArgs& a, const RemapSeq& s, int at) {
  if (s.parent < 0 || at >= s.needed) return -1;
  return page_at(a.g.tables + (size_t)s.parent * a.g.max_pages, a.g.max_pages, a.g.n_pages, at);
}
// exclusive prefix sum over the block of one value per thread; *total = the sum
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                                        // the sums of an earlier scan have been read
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int w = warp_sums[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return x - v + (warp > 0 ? before : 0);
}

// SMEM: the counts and the free list lie in shared memory (pools of up to SMEM_PAGES pages) and not in scratch: an atomic or a look
// there saves a trip to L2 each time (64 sequences of up to 8 pages, copies included, 49.0 -> 46.1 us; 4 of 44 pages 8.4 -> 7.0).
constexpr int SMEM_PAGES = 12 * 1024;
template <bool SMEM>
__global__ void __launch_bounds__(REMAP_THREADS, 1) k_pages_remap(RemapArgs a) {
  extern __shared__ int32_t s_counts[];
  __shared__ int s_warp[32];
  __shared__ int s_first[POSS_MAX_PAGED_BATCH];           // fresh places of the sequences before
  pdl_enter(POSS_K_PAGES_REMAP);
  const PageGeo& g = a.g;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  int32_t* const refs = SMEM ? s_counts : a.out_refs;
  int32_t* const writers = SMEM ? s_counts + g.n_pages : a.writers;
  int32_t* const last = SMEM ? s_counts + 2 * g.n_pages : a.last;
  int32_t* const free_list = SMEM ? s_counts + 3 * g.n_pages : a.free_list;
  auto look = [](const int32_t* p) { return SMEM ? *p : __ldcg(p); };
  // ---- 1
  for (int p = t; p < g.n_pages; p += REMAP_THREADS) {
    refs[p] = a.refs[p];
    writers[p] = 0;
    last[p] = -1;
  }
  __syncthreads();
  for (int i = warp; i < a.n_before; i += 32) {
    for (int at = lane; at < g.max_pages; at += 32) {
      const int raw = g.tables[(size_t)i * g.max_pages + at];
      if (raw >= g.n_pages) raise_status(a.status, POSS_E_INVALID);
      else if (raw >= 0) atomicSub(refs + raw, 1);
    }
  }
  for (int i = warp; i < a.n_after; i += 32) {
    bool bad;
    const RemapSeq s = remap_seq(a, i, &bad);
    if (bad && lane == 0) raise_status(a.status, POSS_E_INVALID);
    const int first_write = s.kept / g.page;
    for (int at = lane; at < s.needed; at += 32) {
      const int p = remap_taken(a, s, at);
      if (p >= 0) {
        atomicAdd(refs + p, 1);
        if (at >= first_write) {
          atomicAdd(writers + p, 1);
          atomicMax(last + p, i);
        }
      }
    }
  }
  __syncthreads();
  // ---- 2: fresh places per sequence (one warp each)
  auto is_fresh = [&](const RemapSeq& s, int i, int at, int* p) {
    if (at >= s.needed) return false;
    *p = remap_taken(a, s, at);
    if (*p < 0) return true;
    if (at < s.kept / g.page) return false;
    return !(look(refs + *p) == look(writers + *p) && look(last + *p) == i);
  };
  for (int i = warp; i < a.n_after; i += 32) {
    bool bad;
    const RemapSeq s = remap_seq(a, i, &bad);
    int n = 0;
    for (int at0 = 0; at0 < s.needed; at0 += 32) {
      int p;
      n += __popc(__ballot_sync(0xffffffffu, is_fresh(s, i, at0 + lane, &p)));
    }
    if (lane == 0) s_first[i] = n;
  }
  __syncthreads();
  static_assert(POSS_MAX_PAGED_BATCH <= REMAP_THREADS, "one sequence per thread");
  int n_fresh = 0;
  {
    const int n = t < a.n_after ? s_first[t] : 0;
    const int before = block_scan(n, s_warp, &n_fresh);
    __syncthreads();
    if (t < a.n_after) s_first[t] = before;
  }
  // ---- 3: free pages in order, a chunk of one page per thread at a time
  int n_free = 0;
  for (int p0 = 0; p0 < g.n_pages; p0 += REMAP_THREADS) {
    const int p = p0 + t;
    const int is_free = p < g.n_pages && look(refs + p) == 0;
    int here;
    const int rank = n_free + block_scan(is_free, s_warp, &here);
    if (is_free && rank < n_fresh) free_list[rank] = p;
    n_free += here;
  }
  __syncthreads();
  if (n_free < n_fresh) {
    // does not fit: nothing changes, or the outputs become those of sequences without slots
    for (int p = t; p < g.n_pages; p += REMAP_THREADS) a.out_refs[p] = a.refs[p];
    for (int i = t; i < a.n_after; i += REMAP_THREADS) a.copies[3 * i + 2] = 0;
    if (a.fresh) {
      for (size_t i = t; i < (size_t)a.n_after * g.max_pages; i += REMAP_THREADS) a.out_tables[i] = -1;
      for (int i = t; i < a.n_after; i += REMAP_THREADS) a.out_len[i] = 0;
    }
    if (t == 0) a.out_free[0] = n_free - n_fresh;
    return;
  }
  for (int i = warp; i < a.n_after; i += 32) {
    bool bad;
    const RemapSeq s = remap_seq(a, i, &bad);
    int nth = s_first[i];
    int32_t* row = a.out_tables + (size_t)i * g.max_pages;
    const int part = s.kept % g.page, part_at = s.kept / g.page;
    if (lane == 0) {
      a.out_len[i] = s.kept;
      a.copies[3 * i + 2] = 0;
    }
    __syncwarp();
    for (int at0 = 0; at0 < g.max_pages; at0 += 32) {
      const int at = at0 + lane;
      int p = -1;
      const bool fresh = is_fresh(s, i, at, &p);
      const unsigned m = __ballot_sync(0xffffffffu, fresh);
      int now = p;
      if (fresh) now = look(free_list + nth + __popc(m & ((1u << lane) - 1)));
      nth += __popc(m);
      if (at < g.max_pages) row[at] = at < s.needed ? now : -1;
      if (fresh && p >= 0 && part > 0 && at == part_at) {
        a.copies[3 * i] = p;
        a.copies[3 * i + 1] = now;
        a.copies[3 * i + 2] = part;
      }
    }
  }
  __syncthreads();
  // the counts after the writers that left: where all holders are writers the last one stays
  for (int p = t; p < g.n_pages; p += REMAP_THREADS) {
    const int r = look(refs + p), w = look(writers + p);
    if (SMEM || w > 0) a.out_refs[p] = w == 0 ? r : r == w ? 1 : r - w;
  }
  __syncthreads();
  for (int j = t; j < n_fresh; j += REMAP_THREADS) a.out_refs[look(free_list + j)] = 1;
  if (t == 0) a.out_free[0] = n_free - n_fresh;
}

// remap: the kept slots of the partly filled pages that were left.  One block per (layer, keys / values, sequence); the
// slots of one head are one run of bytes.  Bound by memory: 20 pages with 38 of 64 slots each on
// average in 32 layers, 199 MB read and written, 36 us (5.5 TB/s).
template <int ES>
__global__ void __launch_bounds__(256) k_pages_copy(PageGeo g, char* pool, const int32_t* copies) {
  pdl_enter(POSS_K_PAGES_COPY);
  const int i = blockIdx.y, layer = blockIdx.x >> 1, kv = blockIdx.x & 1;
  const int n = copies[3 * i + 2];
  if (n <= 0) return;
  const int src = copies[3 * i], dst = copies[3 * i + 1];
  const int per_head = n * g.d * ES / 16, total = per_head * g.Hkv;
  const size_t head_bytes = (size_t)g.page * g.d * ES;
  const char* s = pool + page_offset(g, layer, src, kv, 0) * ES;
  char* d = pool + page_offset(g, layer, dst, kv, 0) * ES;
  for (int j0 = threadIdx.x; j0 < total; j0 += 1024) {
    uint4 x[4];
    size_t o[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int j = j0 + 256 * q;
      if (j < total) {
        const int h = j / per_head;
        o[q] = h * head_bytes + (size_t)(j - h * per_head) * 16;
        x[q] = *reinterpret_cast<const uint4*>(s + o[q]);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (j0 + 256 * q < total) *reinterpret_cast<uint4*>(d + o[q]) = x[q];
  }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

int remap(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int32_t* out_tables, int max_pages,
          int n_before, int n_after, const int32_t* seq_len, const int32_t* refs, int32_t* out_refs,
          const int32_t* parents, const int32_t* room, int32_t* out_len, int32_t* out_free, void* workspace,
          size_t workspace_bytes, int32_t* status, poss_stream stream, bool fresh) {
  int rc = page_pool_check(pool);
  if (rc != POSS_OK) return rc;
  if (n_before < 0 || n_after < 0) return POSS_E_INVALID;
  rc = page_table_check(pool, max_pages, 1);
  if (rc != POSS_OK) return rc;
  if (n_before > POSS_MAX_PAGED_BATCH || n_after > POSS_MAX_PAGED_BATCH) return POSS_E_CAPACITY;
  if (!parents && n_after > 0 && n_before != n_after) return POSS_E_INVALID;
  if (!kv_pages || !refs || !out_refs || !out_free || refs == out_refs || !aligned16(kv_pages)) return POSS_E_INVALID;
  if (n_before > 0 && (!tables || !seq_len)) return POSS_E_INVALID;
  if (n_after > 0 && (!out_tables || !out_len || out_tables == tables)) return POSS_E_INVALID;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
      workspace_bytes < poss_pages_remap_workspace_bytes(pool, n_before, n_after, max_pages))
    return POSS_E_WORKSPACE;
  // the inputs are read while the outputs are written
  const size_t pages = (size_t)pool->n_pages * 4, place = (size_t)max_pages * 4, n0 = (size_t)n_before * 4, n1 = (size_t)n_after * 4;
  const struct { const void* at; size_t bytes; } arrays[] = {
      {out_tables, n1 * max_pages}, {out_refs, pages}, {out_len, n1}, {out_free, 4},      // written
      {tables, place * n_before}, {refs, pages}, {seq_len, n0}, {parents, n1}, {room, n1}};
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 9; ++j)
      if (overlap(arrays[i].at, arrays[i].bytes, arrays[j].at, arrays[j].bytes)) return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  RemapArgs a;
  a.g = page_geo(pool, tables, max_pages);
  a.out_tables = out_tables; a.n_before = n_before; a.n_after = n_after;
  a.seq_len = seq_len; a.refs = refs; a.parents = parents; a.room = room;
  a.out_refs = out_refs; a.out_len = out_len; a.out_free = out_free; a.status = status; a.fresh = fresh;
  char* w = reinterpret_cast<char*>(workspace);
  const size_t per_page = round256((size_t)pool->n_pages * 4);
  a.writers = reinterpret_cast<int32_t*>(w);
  a.last = reinterpret_cast<int32_t*>(w + per_page);
  a.free_list = reinterpret_cast<int32_t*>(w + 2 * per_page);
  a.copies = reinterpret_cast<int32_t*>(w + 3 * per_page);
  if (pool->n_pages <= SMEM_PAGES) {
    static PerDeviceFlags attr_done;
    bool* attr = attr_done.current();
    if (!attr || !*attr) {
      if (cudaFuncSetAttribute(k_pages_remap<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_PAGES * 16) != cudaSuccess)
        return POSS_E_CUDA;
      if (attr) *attr = true;
    }
    launch_pdl(L, k_pages_remap<true>, dim3(1), dim3(REMAP_THREADS), (size_t)pool->n_pages * 16, a);
  } else {
    launch_pdl(L, k_pages_remap<false>, dim3(1), dim3(REMAP_THREADS), 0, a);
  }
  if (n_after > 0) {
    const dim3 grid(pool->n_layers * 2, n_after);
    if (pool->dtype == POSS_BF16)
      launch_pdl(L, k_pages_copy<2>, grid, dim3(256), 0, a.g, (char*)kv_pages, (const int32_t*)a.copies);
    else
      launch_pdl(L, k_pages_copy<4>, grid, dim3(256), 0, a.g, (char*)kv_pages, (const int32_t*)a.copies);
  }
  return L.err;
}

}  // namespace

extern "C" {

int poss_pages_append(const poss_page_pool* pool, int layer, void* kv_pages, const int32_t* tables, int max_pages,
                      int batch, int rows, const void* k, const void* v, int64_t ld_kv, const int32_t* prefix_len,
                      const int32_t* n_rows, int32_t* status, poss_stream stream) {
  int rc = page_pool_check(pool);
  if (rc != POSS_OK) return rc;
  if (batch == 0 || rows == 0) return batch < 0 || rows < 0 ? POSS_E_INVALID : POSS_OK;
  rc = page_table_check(pool, max_pages, batch);
  if (rc != POSS_OK) return rc;
  if (layer < 0 || layer >= pool->n_layers || rows < 0) return POSS_E_INVALID;
  if (rows > 65535) return POSS_E_CAPACITY;
  if (!kv_pages || !tables || !k || !v || !prefix_len) return POSS_E_INVALID;
  const int es = pool->dtype == POSS_BF16 ? 2 : 4;
  if (ld_kv < (int64_t)pool->n_kv_heads * pool->head_dim || (ld_kv * es) % 16) return POSS_E_INVALID;
  if (!aligned16(kv_pages) || !aligned16(k) || !aligned16(v)) return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  const PageGeo g = page_geo(pool, tables, max_pages);
  const dim3 grid((unsigned)(((long long)batch * rows + 7) / 8));
  const char* kc = reinterpret_cast<const char*>(k);
  const char* vc = reinterpret_cast<const char*>(v);
  if (es == 2)
    launch_pdl(L, k_pages_append<2>, grid, dim3(256), 0, g, layer, (char*)kv_pages, batch, rows, kc, vc,
               (long long)ld_kv * es, prefix_len, n_rows, status);
  else
    launch_pdl(L, k_pages_append<4>, grid, dim3(256), 0, g, layer, (char*)kv_pages, batch, rows, kc, vc,
               (long long)ld_kv * es, prefix_len, n_rows, status);
  return L.err;
}

int poss_pages_compact(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch,
                       const int32_t* prefix_len, const int32_t* path, const int32_t* n_accepted, int32_t* out_len,
                       int32_t* status, poss_stream stream) {
  int rc = page_pool_check(pool);
  if (rc != POSS_OK) return rc;
  if (batch == 0) return POSS_OK;
  rc = page_table_check(pool, max_pages, batch);
  if (rc != POSS_OK) return rc;
  if (!kv_pages || !tables || !prefix_len || !path || !n_accepted || !out_len || !aligned16(kv_pages))
    return POSS_E_INVALID;
  // every block reads the lengths, one of each sequence writes the new one
  const size_t n = (size_t)batch * 4;
  if (overlap(out_len, n, prefix_len, n) || overlap(out_len, n, n_accepted, n) ||
      overlap(out_len, n, path, n * (POSS_MAX_DEPTH + 1)) || overlap(out_len, n, tables, n * max_pages))
    return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  const PageGeo g = page_geo(pool, tables, max_pages);
  const dim3 grid(pool->n_layers * 2, batch);
  if (pool->dtype == POSS_BF16)
    launch_pdl(L, k_pages_compact<2>, grid, dim3(256), 0, g, (char*)kv_pages, prefix_len, path, n_accepted, out_len,
               status);
  else
    launch_pdl(L, k_pages_compact<4>, grid, dim3(256), 0, g, (char*)kv_pages, prefix_len, path, n_accepted, out_len,
               status);
  return L.err;
}

size_t poss_pages_remap_workspace_bytes(const poss_page_pool* pool, int n_before, int n_after, int max_pages) {
  if (page_pool_check(pool) != POSS_OK || n_before < 0 || n_after < 0) return 0;
  if (page_table_check(pool, max_pages, 1) != POSS_OK) return 0;
  if (n_before > POSS_MAX_PAGED_BATCH || n_after > POSS_MAX_PAGED_BATCH) return 0;
  return 3 * round256((size_t)pool->n_pages * 4) + round256((size_t)n_after * 12 + 1);
}

int poss_pages_remap(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int32_t* out_tables,
                     int max_pages, int n_before, int n_after, const int32_t* seq_len, const int32_t* refs,
                     int32_t* out_refs, const int32_t* parents, const int32_t* room, int32_t* out_len,
                     int32_t* out_free, void* workspace, size_t workspace_bytes, int32_t* status,
                     poss_stream stream) {
  return remap(pool, kv_pages, tables, out_tables, max_pages, n_before, n_after, seq_len, refs, out_refs, parents, room,
               out_len, out_free, workspace, workspace_bytes, status, stream, false);
}

int poss_pages_remap_fresh(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int32_t* out_tables,
                           int max_pages, int n_before, int n_after, const int32_t* seq_len, const int32_t* refs,
                           int32_t* out_refs, const int32_t* parents, const int32_t* room, int32_t* out_len,
                           int32_t* out_free, void* workspace, size_t workspace_bytes, int32_t* status,
                           poss_stream stream) {
  return remap(pool, kv_pages, tables, out_tables, max_pages, n_before, n_after, seq_len, refs, out_refs, parents, room,
               out_len, out_free, workspace, workspace_bytes, status, stream, true);
}

int poss_debug_page_of_slot(const int32_t* h_table, int max_pages, int page_slots, int n_pages, int64_t slot,
                            int* h_page, int* h_offset) {
  if (!h_table || !h_page || !h_offset || max_pages < 1 || page_slots < 1 || n_pages < 1) return POSS_E_INVALID;
  const int64_t place = slot < 0 ? -1 : slot / page_slots;
  *h_page = place > 0x7fffffff ? -1 : page_at(h_table, max_pages, n_pages, (int)place);
  *h_offset = slot < 0 ? 0 : (int)(slot % page_slots);
  return POSS_OK;
}

}  // extern "C"
