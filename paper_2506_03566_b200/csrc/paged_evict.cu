// Eviction from paged caches by accumulated attention weight.
//
// Of a sequence's n slots keep[b] stay, for every layer and KV head its own: the first `first`, the last `recent`, and of those between
// the ones with the greatest weight, ties to the lower slot.  They move to slots 0 .. keep - 1 in their order, weights with them.
//
//   choose  a block per (sequence, layer, KV head).  Weights become whole numbers that order alike; a block has 8192 in registers (16 rows
//           of 512 slots), more are read again in each round.  Three rounds over 11, 11 and 10 of the numbers' bits count how many
//           share each value of those bits and narrow the last one that stays down to its value T and to how many slots equal to T
//           stay (the lowest ones).  Ballots and one sum over rows and warps then number the slots that stay.
//   move    a block per (sequence, layer, KV head, keys / values) brings the rows forward, some dozen at a time.  A row's new place is
//           never behind its old one and rows go in order, so a step may write as soon as all of its own rows are in registers: what
//           it overwrites is gone or has been read.  The next step's places are looked up while a step's rows are on their way.  Where
//           blocks are few, several share a row, each with columns of its own.
// What bounds it, four sequences of up to 8191 slots cut to 2048 in eight layers of 8 heads, 546 MB: memory in the move, 84 us of 106 (6.4 TB/s);
// trips and barriers in the choice.  Three sequences of up to 700 slots in two layers: 10.6 us, some 6 of them the choice.
#include "paged.cuh"

POSS_TRACE_REGISTER()

namespace {

constexpr int CHOOSE_THREADS = 512, CHOOSE_WARPS = 16;
constexpr int PER = 16;                      // slots per thread and chunk
constexpr int CHUNK = CHOOSE_THREADS * PER;
constexpr int BINS = 2048;

struct EvictArgs {
  PageGeo g;
  int batch, first, recent;
  const float* mass;
  float* out_mass;
  long long mass_slots;                      // weights per (layer, sequence, head)
  const int32_t *seq_len, *keep;
  int32_t *out_len, *status;
  int32_t* src;                              // [layers][batch][heads][slots]: the slot that moves to each place
  int32_t* hole;                             // [layers][batch][heads]: the first place that changes; out_len where none does
};

// a weight as a number that orders alike; -0 is 0, NaN below all
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
// exclusive prefix sum over the block; *total = the sum.  sums: one int per warp, free for use behind the barrier before the call
__device__ __forceinline__ int scan(int v, int* sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  const int w = lane < CHOOSE_WARPS ? sums[lane] : 0;
  *total = __reduce_add_sync(0xffffffffu, w);
  return x - v + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
}

// refs: NULL, or the holders of every page.  (Not among EvictArgs, 8 bytes of which more cost both kernels together 1.5 us of 106.)
__global__ void __launch_bounds__(CHOOSE_THREADS) k_evict_choose(EvictArgs a, const int32_t* refs) {
  static_assert(PER * CHOOSE_WARPS <= CHOOSE_THREADS && CHOOSE_WARPS * 32 == CHOOSE_THREADS, "a count per row and warp");
  __shared__ int s_bins[BINS], s_sums[4][CHOOSE_WARPS], s_bin, s_left, s_count, s_hole;
  __shared__ int s_sure[PER * CHOOSE_WARPS], s_tie[PER * CHOOSE_WARPS];
  pdl_enter(POSS_K_EVICT_CHOOSE);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int head = blockIdx.x % a.g.Hkv, lb = blockIdx.x / a.g.Hkv, b = lb % a.batch;
  const int n = a.seq_len[b], keep = a.keep[b];
  const long long slots = (long long)a.g.max_pages * a.g.page;
  bool ok = n >= 0 && n <= slots && keep >= 0 && (n <= keep || (long long)a.first + a.recent <= keep);
  const size_t row = (size_t)lb * a.g.Hkv + head;
  const float* x = a.mass + row * a.mass_slots;
  float* out = a.out_mass + row * a.mass_slots;
  float w[PER];                                           // the thread's slots of a chunk, one of each row
  auto slot = [&](int chunk, int p) { return chunk * CHUNK + p * CHOOSE_THREADS + t; };
  auto rows_of = [&](int chunk) { return min(PER, (n - chunk * CHUNK + CHOOSE_THREADS - 1) / CHOOSE_THREADS); };
  auto load = [&](int chunk) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int i = slot(chunk, p);
      w[p] = i < n ? x[i] : 0.f;
    }
  };
  const bool cuts = ok && n > keep;
  const int chunks = cuts ? (n + CHUNK - 1) / CHUNK : 0;
  if (chunks == 1) load(0);
  // (the pages are looked at while the weights are on their way)
  const int32_t* table = a.g.tables + (size_t)b * a.g.max_pages;
  if (cuts)
    for (int i = t; i < (n + a.g.page - 1) / a.g.page; i += CHOOSE_THREADS) ok &= page_at(table, a.g.max_pages, a.g.n_pages, i) >= 0;
  // a page that others hold is read alone: no place from `first` on lies in it.  (The same for all layers and heads: so is the new length.)
  if (refs && cuts && keep > a.first)
    for (int i = a.first / a.g.page + t; i * (long long)a.g.page < keep; i += CHOOSE_THREADS) {
      const int p = page_at(table, a.g.max_pages, a.g.n_pages, i);
      ok &= p >= 0 && refs[p] <= 1;
    }
  for (int i = t; i < BINS; i += CHOOSE_THREADS) s_bins[i] = 0;
  if (t == 0) s_hole = keep;
  ok = __syncthreads_and(ok);
  const int stays = !ok || n <= keep ? n : keep;
  if (blockIdx.x == (unsigned)(b * a.g.Hkv) && t == 0) {  // (the first layer's first head)
    a.out_len[b] = stays;
    if (!ok) raise_status(a.status, POSS_E_INVALID);
  }
  if (!ok || n <= keep) {
    if (t == 0) a.hole[row] = stays;
    if (ok && out != x)
      for (int i = t; i < n; i += CHOOSE_THREADS) out[i] = x[i];
    return;
  }
  // ---- the last weight that stays, of slots [lo, hi)
  const int lo = a.first, hi = n - a.recent;
  int left = keep - a.first - a.recent;                   // how many of them stay
  uint32_t fixed = 0, mask = 0;                           // the bits of it that are known
  int equal = 0;                                          // slots that equal it and stay
  if (left > 0) {
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bins = round == 2 ? 1024 : 2048;
      if (round > 0) {
        for (int i = t; i < bins; i += CHOOSE_THREADS) s_bins[i] = 0;
        __syncthreads();
      }
#pragma unroll 1
      for (int c = 0; c < chunks; ++c) {
        if (chunks > 1) load(c);
        const int n_rows = rows_of(c);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
          if (p >= n_rows) break;
          const int i = slot(c, p);
          const uint32_t u = order_of(w[p]);
          if (i >= lo && i < hi && (u & mask) == fixed) atomicAdd(&s_bins[(u >> shift) & (bins - 1)], 1);
        }
      }
      __syncthreads();
      // from the greatest value down: the bin that the left-th falls into
      const int per = bins / CHOOSE_THREADS;              // 4 or 2 bins per thread, greatest first
      int mine = 0, total;
      for (int i = 0; i < per; ++i) mine += s_bins[bins - 1 - (t * per + i)];
      int before = scan(mine, s_sums[round], &total);
      if (before < left && left <= before + mine) {
        for (int i = 0; i < per; ++i) {
          const int bin = bins - 1 - (t * per + i), c = s_bins[bin];
          if (left <= before + c) { s_bin = bin; s_left = left - before; s_count = c; break; }
          before += c;
        }
      }
      __syncthreads();
      fixed |= (uint32_t)s_bin << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      left = s_left;
      if (s_count == left && fixed) {                     // the whole bin stays: T is the number below it (no weight has 0 alone above it)
        --fixed;
        left = 0;
        break;
      }
      // (the next round's counts begin behind a barrier, and with them the writes of s_bin, s_left and s_count)
    }
    equal = left;
  } else {
    fixed = 0xffffffffu;                                  // (above every weight)
  }
  // ---- the slots that stay, in order: their places.  (In place a weight's new place is never behind its old one, and a chunk's weights are
  // in registers before the chunk's barrier.)
  int32_t* src = a.src + row * slots;
  int at = 0, ties = 0, hole = keep;                      // places given so far, ties met so far
#pragma unroll 1
  for (int c = 0; c < chunks; ++c) {
    if (chunks > 1) load(c);
    const int n_rows = rows_of(c);
    uint32_t sure, tie;
    auto look = [&](int p) {
      const int i = slot(c, p);
      const bool inner = i >= lo && i < hi;
      const uint32_t u = order_of(w[p]);
      sure = __ballot_sync(0xffffffffu, i < n && (!inner || u > fixed));
      tie = __ballot_sync(0xffffffffu, inner && u == fixed);
    };
    __syncthreads();                                      // the last use of the counts is over
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      if (p >= n_rows) break;
      look(p);
      if (lane == 0) { s_sure[p * CHOOSE_WARPS + warp] = __popc(sure); s_tie[p * CHOOSE_WARPS + warp] = __popc(tie); }
    }
    __syncthreads();
    // counts before each row's warp: in place
    const bool has = t < n_rows * CHOOSE_WARPS;
    int all_sure, all_ties;
    const int vs = scan(has ? s_sure[t] : 0, s_sums[0], &all_sure), vt = scan(has ? s_tie[t] : 0, s_sums[3], &all_ties);
    if (has) { s_sure[t] = vs; s_tie[t] = vt; }
    __syncthreads();
    const uint32_t below = (1u << lane) - 1;
    auto kept_of = [&](int ties_before) { return min(ties_before, equal); };   // of the first ties_before ties
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      if (p >= n_rows) break;
      look(p);                                            // (once more: 32 words of bits would not fit the registers)
      const int tb = ties + s_tie[p * CHOOSE_WARPS + warp] + __popc(tie & below);
      const bool on = (sure >> lane & 1u) || ((tie >> lane & 1u) && tb < equal);
      const int place = at + s_sure[p * CHOOSE_WARPS + warp] + __popc(sure & below) + kept_of(tb) - kept_of(ties), i = slot(c, p);
      if (on) {
        src[place] = i;
        out[place] = w[p];
        if (place != i) hole = min(hole, place);
      }
    }
    at += all_sure + kept_of(ties + all_ties) - kept_of(ties);
    ties += all_ties;
  }
  hole = __reduce_min_sync(0xffffffffu, hole);
  if (lane == 0) atomicMin(&s_hole, hole);
  __syncthreads();
  if (t == 0) a.hole[row] = s_hole;
}

// Block: (sequence, layer, head), keys / values, and one of `parts` parts of the columns.  A step: four pieces of 16 bytes per thread.
// Places are looked up a step ahead; AHEAD (few blocks): the slots that they are of two steps ahead, so that a step waits for one trip to memory
// and not two, for registers that many blocks need better (four sequences of 8191 slots in eight layers 106 us, 115 so; two sequences of 4653
// in seven layers of 2 heads 40, 29 so).  A step's targets are read behind its barrier, while others may be a step further: they have a third
// buffer.
template <int ES, int THREADS, bool AHEAD>
__global__ void __launch_bounds__(THREADS) k_evict_move(EvictArgs a, char* pool, int log_parts) {
  constexpr int PIECES = 4, ROWS = PIECES / 2;            // pieces, and rows at the most, of a thread (two pieces per row at the least)
  __shared__ long long s_src[2][THREADS * ROWS], s_dst[3][THREADS * ROWS];
  pdl_enter(POSS_K_EVICT_MOVE);
  const int t = threadIdx.x, part = blockIdx.x & ((1 << log_parts) - 1), kv = blockIdx.x >> log_parts & 1;
  const int row = blockIdx.x >> log_parts >> 1, head = row % a.g.Hkv, lb = row / a.g.Hkv, b = lb % a.batch, layer = lb / a.batch;
  const int keep = a.out_len[b], hole = a.hole[row];
  if (hole >= keep) return;
  const long long slots = (long long)a.g.max_pages * a.g.page;
  const int32_t* src = a.src + (size_t)row * slots;
  const int32_t* table = a.g.tables + (size_t)b * a.g.max_pages;
  const int per_row = a.g.d * ES / 16 >> log_parts, rows = THREADS * PIECES / per_row;   // (a power of two)
  const int shift = __ffs(per_row) - 1;
  pool += part * per_row * 16;
  auto where = [&](int slot) {
    const int place = slot / a.g.page;                    // (every page of the sequence was seen to be there)
    const int p = page_at(table, a.g.max_pages, a.g.n_pages, place);
    return (long long)(page_offset(a.g, layer, p < 0 ? 0 : p, kv, head) + (size_t)(slot - place * a.g.page) * a.g.d) * ES;
  };
  int from[ROWS];
  auto fetch = [&](int r0) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int r = t + i * THREADS;
      from[i] = r < min(rows, keep - r0) ? src[r0 + r] : 0;
    }
  };
  auto look_up = [&](int r0, int buf, int to) {
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int r = t + i * THREADS;
        if (r < min(rows, keep - r0)) {
          s_src[buf][r] = where(from[i]);
          s_dst[to][r] = where(r0 + r);
        }
      }
      fetch(r0 + rows);
    } else {
      for (int r = t; r < min(rows, keep - r0); r += THREADS) {
        s_src[buf][r] = where(src[r0 + r]);
        s_dst[to][r] = where(r0 + r);
      }
    }
  };
  int buf = 0, to = 0;
  if (AHEAD) fetch(hole);
  look_up(hole, 0, 0);
  __syncthreads();
#pragma unroll 1
  for (int r0 = hole; r0 < keep; r0 += rows) {
    const int n = min(rows, keep - r0), next_to = to == 2 ? 0 : to + 1;
    uint4 x[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const int i = t + j * THREADS, r = i >> shift;
      if (r < n) x[j] = *reinterpret_cast<const uint4*>(pool + s_src[buf][r] + (i - (r << shift)) * 16);
    }
    if (r0 + rows < keep) look_up(r0 + rows, buf ^ 1, next_to);
    __syncthreads();                                      // the step's rows are in registers, the next one's places known
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const int i = t + j * THREADS, r = i >> shift;
      if (r < n) *reinterpret_cast<uint4*>(pool + s_dst[to][r] + (i - (r << shift)) * 16) = x[j];
    }
    buf ^= 1;
    to = next_to;
  }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// both entries; refs NULL: the caller answers for it that nobody else holds the pages
int evict(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch, const int32_t* refs, const float* mass,
          float* out_mass, int64_t mass_slots, const int32_t* seq_len, const int32_t* keep, int first, int recent, int32_t* out_len,
          void* workspace, size_t workspace_bytes, int32_t* status, poss_stream stream) {
  int rc = page_pool_check(pool);
  if (rc != POSS_OK) return rc;
  if (batch < 0 || first < 0 || recent < 0) return POSS_E_INVALID;
  if (batch == 0) return POSS_OK;
  rc = page_table_check(pool, max_pages, batch);
  if (rc != POSS_OK) return rc;
  const size_t need = poss_pages_evict_workspace_bytes(pool, batch, max_pages);
  if (!need) return POSS_E_CAPACITY;
  if (!kv_pages || !tables || !mass || !out_mass || !seq_len || !keep || !out_len || !aligned16(kv_pages)) return POSS_E_INVALID;
  if (mass_slots < (int64_t)max_pages * pool->page_slots) return POSS_E_INVALID;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need) return POSS_E_WORKSPACE;
  const size_t rows = (size_t)pool->n_layers * batch * pool->n_kv_heads;
  if (out_mass != mass && overlap(out_mass, rows * mass_slots * 4, mass, rows * mass_slots * 4)) return POSS_E_INVALID;
  const size_t nb = (size_t)batch * 4;
  if (overlap(out_len, nb, seq_len, nb) || overlap(out_len, nb, keep, nb) || overlap(out_len, nb, tables, nb * max_pages) ||
      overlap(out_len, nb, mass, rows * mass_slots * 4) || overlap(out_len, nb, out_mass, rows * mass_slots * 4) ||
      overlap(out_len, nb, refs, (size_t)pool->n_pages * 4) || overlap(out_mass, rows * mass_slots * 4, refs, (size_t)pool->n_pages * 4))
    return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  EvictArgs a;
  a.g = page_geo(pool, tables, max_pages);
  a.batch = batch; a.first = first; a.recent = recent;
  a.mass = mass; a.out_mass = out_mass; a.mass_slots = mass_slots;
  a.seq_len = seq_len; a.keep = keep; a.out_len = out_len; a.status = status;
  a.hole = reinterpret_cast<int32_t*>(workspace);
  a.src = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(workspace) + round256(rows * 4));
  launch_pdl(L, k_evict_choose, dim3((unsigned)rows), dim3(CHOOSE_THREADS), 0, a, refs);
  if (L.err != POSS_OK) return L.err;
  // columns are shared out while that leaves two pieces or more to each and the device has room, and blocks are larger where there are few and
  // a table has room for some steps: fewer steps, one behind the other (one sequence of 8191 slots, 8 heads, 7000 stay: 44 -> 41 us; three of
  // 700 slots 10.7, with large blocks 11.0)
  int log_parts = 0;
  const int es = pool->dtype == POSS_BF16 ? 2 : 4, pieces = pool->head_dim * es / 16;
  const size_t sms = current_sm_count();
  const bool steps = (int64_t)max_pages * pool->page_slots > 2048;
  while (log_parts < (steps ? 3 : 2) && pieces >> (log_parts + 1) >= 2 && (rows << (log_parts + 2)) <= 4 * sms) ++log_parts;
  const size_t blocks = rows << (1 + log_parts);
  auto move = [&](auto kernel, int threads) {
    launch_pdl(L, kernel, dim3((unsigned)blocks), dim3(threads), 0, a, reinterpret_cast<char*>(kv_pages), log_parts);
  };
  if (blocks <= 2 * sms && steps) es == 2 ? move(k_evict_move<2, 512, true>, 512) : move(k_evict_move<4, 512, true>, 512);
  else es == 2 ? move(k_evict_move<2, 256, false>, 256) : move(k_evict_move<4, 256, false>, 256);
  return L.err;
}

}  // namespace

extern "C" {

size_t poss_pages_evict_workspace_bytes(const poss_page_pool* pool, int batch, int max_pages) {
  if (page_pool_check(pool) != POSS_OK || page_table_check(pool, max_pages, batch) != POSS_OK) return 0;
  const size_t rows = (size_t)pool->n_layers * batch * pool->n_kv_heads;
  if (rows >= (1ull << 30)) return 0;
  return round256(rows * 4) + round256(rows * (size_t)max_pages * pool->page_slots * 4);
}

int poss_pages_evict(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch, const float* mass,
                     float* out_mass, int64_t mass_slots, const int32_t* seq_len, const int32_t* keep, int first, int recent,
                     int32_t* out_len, void* workspace, size_t workspace_bytes, int32_t* status, poss_stream stream) {
  return evict(pool, kv_pages, tables, max_pages, batch, nullptr, mass, out_mass, mass_slots, seq_len, keep, first, recent, out_len,
               workspace, workspace_bytes, status, stream);
}

int poss_pages_evict_refs(const poss_page_pool* pool, void* kv_pages, const int32_t* tables, int max_pages, int batch,
                          const int32_t* refs, const float* mass, float* out_mass, int64_t mass_slots, const int32_t* seq_len,
                          const int32_t* keep, int first, int recent, int32_t* out_len, void* workspace, size_t workspace_bytes,
                          int32_t* status, poss_stream stream) {
  return evict(pool, kv_pages, tables, max_pages, batch, refs, mass, out_mass, mass_slots, seq_len, keep, first, recent, out_len, workspace,
               workspace_bytes, status, stream);
}

}  // extern "C"
