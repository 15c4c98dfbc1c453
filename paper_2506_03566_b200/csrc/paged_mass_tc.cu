// The weight that every slot draws, on the 5th-generation tensor cores (bf16, head dimension 64 or 128).
//
// Scores are formed with the keys as rows and the query lines (tree row, head) as columns: S^T = K Q^T, 128 slots times up to 256 lines.
// A slot is then a lane of TMEM, its thread takes its own lane's scores, adds w / l 2^(scale s - m) up over the columns and writes one
// number: no sum crosses threads.  A column's constants (-m, w / l) come from shared memory, the same address for all lanes.
//
// A unit of work is 128 slots of one (sequence, KV head); the units of the whole batch are cut into one contiguous range per CTA, one CTA
// per SM.  More than 256 lines take a pass each over the CTA's slots; the later ones add to what the first has written.
//   warps 0-3 / 4-7  weights of even / odd tiles (each has a score buffer of its own)
//   warp 8           keys, through a ring of stages (one box per page and 64 columns), and a pass's queries
//   warp 9           products, one lane
// What bounds it: the exponentials where lines are many (128 x 244 of them per tile, 16 per cycle: 1952 cycles), the read of the keys
// where they are few.
//
// Every wait is bounded; on expiry the CTA raises POSS_E_TIMEOUT, runs through its (bounded) walk without meaning, waits (bounded) for
// its copies in flight, frees its TMEM and returns.
#include "paged_attention.cuh"
#include "tc_ptx.cuh"
#include <string.h>

POSS_TRACE_REGISTER()

namespace {

using namespace tcptx;

constexpr int KT = 128;                 // slots per tile
constexpr int MAX_LINES = 256;          // query lines per pass
constexpr int N_SUMS = 256;             // threads that form weights
constexpr int N_THREADS = N_SUMS + 64;
constexpr int WARP_KEYS = 8, WARP_MMA = 9;
constexpr int K_BLOCK = KT * 128;       // bytes of 128 slots x 64 bf16
constexpr int Q_BLOCK = MAX_LINES * 128;
constexpr int MAX_STAGES = 6;
constexpr uint32_t TMEM_COLS = 512;     // two buffers of 256 columns

template <int HD> struct Shape {
  static constexpr int CB = HD / 64;
  static constexpr int TILE = CB * K_BLOCK, Q_BYTES = CB * Q_BLOCK;
  static constexpr int NK = HD == 128 ? 4 : 6;
  static constexpr int K_OFF = Q_BYTES, CTL_OFF = K_OFF + NK * TILE;
};

struct Work {
  int prefix, rows, total, tiles;
  uint32_t units;                       // (a batch's units fit 31 bits: checked on the host)
};
struct Args {
  PagedMassArgs s;
  int pass_rows;                        // tree rows per pass
  int rows_total;                       // rows of the pool's layer: the first coordinate behind it
  int page_shift;
};
__device__ __forceinline__ Work work_of(const PagedAttnArgs& a, int b) {
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows, (long long)a.g.max_pages * a.g.page);
  Work w;
  w.prefix = n.prefix; w.rows = n.rows;
  w.total = n.prefix + n.rows;
  w.tiles = n.rows ? (w.total + KT - 1) / KT : 0;
  w.units = (uint32_t)a.g.Hkv * w.tiles;
  return w;
}
// Barriers are waited for by parity; no role can be two phases ahead of another on one: keys by the ring, scores by s_empty, queries by
// q_empty, which follows the pass's last product.
struct Ctl {
  uint64_t k_full[MAX_STAGES], k_empty[MAX_STAGES], q_full, q_empty, s_full[2], s_empty[2], drain;
  uint32_t tmem;
  int abort;
  uint32_t u, u_end, offset;            // the CTA's range; its first unit inside its first sequence
  int seq;
  // by pass, in turn: two columns' (-m, -m, w / l, w / l), and every column's ancestor bits
  float4 col[2][MAX_LINES / 2];
  ulonglong2 mask[2][MAX_LINES];
};

// a CTA's passes in order; every role walks them by itself
struct Pass {
  int b, head, tile0, n, group;         // n tiles from tile0 on, the group-th `pass_rows` rows
  Work w;
};
struct Walk {
  uint32_t u, u_end, offset;
  int b, group, groups, left;
  __device__ __forceinline__ void start(const Ctl& c, const PagedAttnArgs& a, Pass* p) {
    u = c.u; u_end = c.u_end; offset = c.offset; b = c.seq;
    group = groups = 0;
    if (u < u_end) p->w = work_of(a, b);
  }
  __device__ __forceinline__ bool next(const Args& k, Pass* p) {
    const PagedAttnArgs& a = k.s.a;
    if (group + 1 < groups) {
      p->group = ++group;
      return true;
    }
    if (u >= u_end) return false;
    while (offset >= p->w.units) {
      offset -= p->w.units;
      if (++b >= a.batch) return false;                     // (not reached: the range lies inside the batch's units)
      p->w = work_of(a, b);
    }
    p->b = b;
    p->head = (int)(offset / (uint32_t)p->w.tiles);
    p->tile0 = (int)(offset - (uint32_t)p->head * p->w.tiles);
    p->n = min(p->w.tiles - p->tile0, (int)(u_end - u));
    u += p->n;
    offset += p->n;
    p->group = group = 0;
    groups = (p->w.rows + k.pass_rows - 1) / k.pass_rows;
    return true;
  }
};

// adds w / l 2^(scale s - m) of 32 columns
__device__ __forceinline__ void add32(const uint32_t* s, const float4* col, float2 scale, float2& s0, float2& s1) {
#pragma unroll
  for (int x = 0; x < 32; x += 4) {
    const float4 a = col[x / 2], b = col[x / 2 + 1];
    const float2 u = fma2(make_float2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), scale, make_float2(a.x, a.y));
    const float2 v = fma2(make_float2(__uint_as_float(s[x + 2]), __uint_as_float(s[x + 3])), scale, make_float2(b.x, b.y));
    s0 = fma2(make_float2(ex2(u.x), ex2(u.y)), make_float2(a.z, a.w), s0);
    s1 = fma2(make_float2(ex2(v.x), ex2(v.y)), make_float2(b.z, b.w), s1);
  }
}

template <int HD>
__global__ void __launch_bounds__(N_THREADS, 1) k_slot_mass_tc(const __grid_constant__ CUtensorMap map,
                                                               const __grid_constant__ CUtensorMap map_q, const Args k) {
  using Z = Shape<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Ctl& c = *reinterpret_cast<Ctl*>(smem + Z::CTL_OFF);
  const uint32_t base = smem_u32(smem);
  const PagedAttnArgs& a = k.s.a;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  auto bar = [&](uint64_t& x) { return smem_u32(&x); };

  if (warp == WARP_MMA) {
    if (lane == 0) {
      c.abort = base & 1023u ? 1 : 0;                     // (tiles start on 1024 bytes)
      for (int i = 0; i < MAX_STAGES; ++i) {
        mbar_init(bar(c.k_full[i]), 1);
        mbar_init(bar(c.k_empty[i]), 1);
      }
      mbar_init(bar(c.q_full), 1);
      mbar_init(bar(c.q_empty), 1);
      mbar_init(bar(c.drain), 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(bar(c.s_full[i]), 1);
        mbar_init(bar(c.s_empty[i]), N_SUMS / 2);
      }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      prefetch_tensormap(&map);
      prefetch_tensormap(&map_q);
    }
    __syncwarp();
    tmem_alloc(smem_u32(&c.tmem), TMEM_COLS);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  volatile int* abort_flag = &c.abort;
  const uint32_t tm = __shfl_sync(0xffffffffu, c.tmem, 0);
  // The successor may start only now that this CTA holds its TMEM columns: one that took columns on this SM first would
  // keep them until this grid has finished.
  pdl_begin();
  pdl_sync(POSS_K_SLOT_MASS);

  if (warp == 0) {
    // the batch's units, the CTA's range of them, and the sequence that its first one lies in
    uint32_t t = 0;
    for (int x = lane; x < a.batch; x += 32) t += work_of(a, x).units;
    t = __reduce_add_sync(0xffffffffu, t);
    const uint32_t u0 = (uint32_t)((uint64_t)t * blockIdx.x / gridDim.x), u1 = (uint32_t)((uint64_t)t * (blockIdx.x + 1) / gridDim.x);
    if (lane == 0) { c.u = u0; c.u_end = u1; c.seq = 0; c.offset = 0; }
    __syncwarp();
    if (u0 < u1) {
      uint32_t at = u0;
      for (int b0 = 0; b0 < a.batch; b0 += 32) {
        const uint32_t own = b0 + lane < a.batch ? work_of(a, b0 + lane).units : 0;
        uint32_t x = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        const unsigned here = __ballot_sync(0xffffffffu, at < x);
        if (here) {
          const int first = __ffs(here) - 1;
          if (lane == first) { c.seq = b0 + first; c.offset = at - (x - own); }
          break;
        }
        at -= __shfl_sync(0xffffffffu, x, 31);
      }
    }
  }
  __syncthreads();

  Pass p;
  Walk walk;
  walk.start(c, a, &p);
  bool ok = __all_sync(0xffffffffu, *abort_flag == 0);
  int done = 0;                                           // tiles of the passes before
  int issued = 0, queries = 0;                            // copies: tiles and passes' queries under way or here
  uint32_t elected = 0;
  if (warp == WARP_MMA) elected = elect_one();
  auto wait = [&](uint64_t& b, int phase) {
    if (ok) ok = mbar_wait(bar(b), (uint32_t)(phase & 1), abort_flag);
  };

  for (int pass = 0; walk.next(k, &p); ++pass) {
    const int r0 = p.group * k.pass_rows, lines = min(k.pass_rows, p.w.rows - r0) * a.G;
    const int32_t* const table = a.g.tables + (size_t)p.b * a.g.max_pages;
    if (warp < N_SUMS / 32) {
      // -------------------------------------------------------------- weights, one thread per slot
      const int wg = warp >> 2, par = pass & 1;
      {
        // the pass's columns: a thread each
        const int col = threadIdx.x, r = r0 + col / a.G;
        float2 ml = make_float2(INFINITY, 0.f);
        float w = 0.f;
        uint64_t lo = 0, hi = 0;
        if (col < lines) {
          const size_t row = (size_t)p.b * a.rows + r;
          ml = a.ml[row * a.Hq + p.head * a.G + col % a.G];
          w = k.s.weights ? k.s.weights[row] : 1.f;
          paged_row_mask(a.mask, row, a.mask_words, p.w.rows, &lo, &hi);
        }
        float* f = reinterpret_cast<float*>(&c.col[par][col >> 1]) + (col & 1);
        f[0] = -ml.x;
        f[2] = w * ml.y;
        c.mask[par][col] = make_ulonglong2(lo, hi);
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const float2 scale = make_float2(k.s.scale_log2, k.s.scale_log2);
      const float4* const cols = c.col[par];
      float* const mass = k.s.mass + ((size_t)p.b * a.g.Hkv + p.head) * k.s.mass_slots;
      const uint32_t t_s = tm + ((uint32_t)((warp & 3) * 32) << 16) + wg * MAX_LINES;
#pragma unroll 1
      for (int t = (done + wg) & 1; t < p.n; t += 2) {
        const int key0 = (p.tile0 + t) * KT, key = key0 + (warp & 3) * 32 + lane;
        const int use = (done + t) >> 1;
        const bool there = key < p.w.total && page_at(table, a.g.max_pages, a.g.n_pages, key >> k.page_shift) >= 0;
        const bool add = key < p.w.prefix || p.group > 0;
        const float old = key < p.w.total && add ? mass[key] : 0.f;
        wait(c.s_full[wg], use);
        tc_fence_after();
        float2 s0 = make_float2(0.f, 0.f), s1 = s0;
        if (key0 + KT <= p.w.prefix) {                    // every line sees every slot
          int x = 0;
#pragma unroll 1
          for (; x + 32 <= lines; x += 32) {
            uint32_t s[32];
            tmem_ld32(t_s + x, s);
            tmem_wait_ld();
            tie32(s);
            add32(s, cols + x / 2, scale, s0, s1);
          }
#pragma unroll 1
          for (; x < lines; x += 16) {
            float s[16];
            tmem_ld16(t_s + x, s);
#pragma unroll
            for (int y = 0; y < 16; y += 2) {
              const float4 f = cols[(x + y) / 2];
              // (columns behind the last line hold anything)
              if (x + y < lines) s0.x = fmaf(ex2(fmaf(s[y], scale.x, f.x)), f.z, s0.x);
              if (x + y + 1 < lines) s0.y = fmaf(ex2(fmaf(s[y + 1], scale.x, f.y)), f.w, s0.y);
            }
          }
        } else {
          const int j = key - p.w.prefix;                 // place among the call's rows
#pragma unroll 1
          for (int x = 0; x < lines; x += 16) {
            float s[16];
            tmem_ld16(t_s + x, s);
#pragma unroll
            for (int y = 0; y < 16; ++y) {
              const float4 f = cols[(x + y) / 2];
              const ulonglong2 m = c.mask[par][x + y];
              const bool sees = j < 0 || ((j < 64 ? m.x >> j : m.y >> (j - 64)) & 1u);
              if (x + y < lines && sees) s0.x = fmaf(ex2(fmaf(s[y], scale.x, y & 1 ? f.y : f.x)), y & 1 ? f.w : f.z, s0.x);
            }
          }
        }
        tc_fence_before();
        mbar_arrive(bar(c.s_empty[wg]));
        if (key < p.w.total && ok) mass[key] = old + (there ? (s0.x + s0.y) + (s1.x + s1.y) : 0.f);
      }
    } else if (warp == WARP_KEYS) {
      // -------------------------------------------------------------- keys, a lane per page of a tile; the pass's queries
      const int page = a.g.page, per_tile = page < KT ? KT / page : 1;
      auto fetch = [&](int tile) {
        const int key0 = tile * KT + lane * page;
        return lane < per_tile && key0 < p.w.total ? page_at(table, a.g.max_pages, a.g.n_pages, key0 >> k.page_shift) : -1;
      };
      int next = fetch(p.tile0);
      const int with = min(p.n, Z::NK - 1) - 1;           // the queries follow this tile: the first ones need not wait for their place
#pragma unroll 1
      for (int t = 0; ok && t < p.n; ++t) {
        const int at_page = next;
        if (t + 1 < p.n) next = fetch(p.tile0 + t + 1);
        const int st = issued % Z::NK;
        if (issued >= Z::NK) wait(c.k_empty[st], issued / Z::NK - 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(bar(c.k_full[st]), Z::TILE);
        __syncwarp();
        if (lane < per_tile) {
          const int in_page = page > KT ? (p.tile0 + t) * KT & (page - 1) : 0;
          const int row = at_page >= 0 ? (at_page * 2 * a.g.Hkv + p.head) * page + in_page : k.rows_total;
#pragma unroll
          for (int cb = 0; cb < Z::CB; ++cb)
            tma_load(base + Z::K_OFF + st * Z::TILE + cb * K_BLOCK + lane * page * 128, &map, bar(c.k_full[st]), cb * 64, row);
        }
        __syncwarp();
        ++issued;
        if (t == with) {
          if (pass > 0) wait(c.q_empty, pass - 1);
          ok = __all_sync(0xffffffffu, ok);
          if (ok && lane == 0) {
            mbar_expect_tx(bar(c.q_full), k.pass_rows * a.G * HD * 2);
#pragma unroll
            for (int cb = 0; cb < Z::CB; ++cb) tma_load_5d(base + cb * Q_BLOCK, &map_q, bar(c.q_full), cb * 64, p.head, r0, p.b);
          }
          queries += ok;
          __syncwarp();
        }
      }
    } else if (elected) {
      // -------------------------------------------------------------- products
      const uint32_t idesc = instr_desc_bf16(KT, (lines + 15) & ~15);
      const uint64_t q_desc = smem_desc_sw128(base);
      wait(c.q_full, pass);
#pragma unroll 1
      for (int t = 0; ok && t < p.n; ++t) {
        const int n = done + t, st = n % Z::NK, buf = n & 1;
        wait(c.k_full[st], n / Z::NK);
        if (n >= 2) wait(c.s_empty[buf], (n >> 1) - 1);
        if (!ok) break;
        tc_fence_after();
        const uint64_t k_desc = smem_desc_sw128(base + Z::K_OFF + st * Z::TILE);
#pragma unroll
        for (int cb = 0; cb < Z::CB; ++cb)
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            umma_bf16(tm + buf * MAX_LINES, k_desc + cb * (K_BLOCK >> 4) + 2 * kk, q_desc + cb * (Q_BLOCK >> 4) + 2 * kk, idesc,
                      (cb | kk) ? 1u : 0u);
        umma_commit(bar(c.s_full[buf]));
        umma_commit(bar(c.k_empty[st]));
        if (t == p.n - 1) umma_commit(bar(c.q_empty));
      }
    }
    __syncwarp();
    done += p.n;
  }

  if (*abort_flag) {
    // copies and products under way must end before the CTA's shared memory and TMEM go away
    const uint64_t t0 = global_ns();
    auto drained = [&](uint64_t& b, int phase) {
      while (!mbar_try_wait(bar(b), (uint32_t)(phase & 1)) && global_ns() - t0 < WAIT_LIMIT_NS / 2) __nanosleep(64);
    };
    if (warp == WARP_KEYS) {
      if (queries > 0) drained(c.q_full, queries - 1);
      for (int i = issued > Z::NK ? issued - Z::NK : 0; i < issued; ++i) drained(c.k_full[i % Z::NK], i / Z::NK);
    } else if (elected) {
      umma_commit(bar(c.drain));
      drained(c.drain, 0);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == WARP_MMA) tmem_dealloc(tm, TMEM_COLS);
  if (threadIdx.x == 0 && *abort_flag) raise_status(a.status, POSS_E_TIMEOUT);
}

template <int HD> void launch(Launcher& L, const Args& k, const CUtensorMap& map, const CUtensorMap& map_q, long long units) {
  using Z = Shape<HD>;
  const size_t smem = Z::CTL_OFF + sizeof(Ctl);
  static PerDeviceFlags attr_done;
  bool* attr = attr_done.current();
  if (!attr || !*attr) {
    if (cudaFuncSetAttribute(k_slot_mass_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
      L.err = POSS_E_CUDA;
      return;
    }
    if (attr) *attr = true;
  }
  const int sms = current_sm_count();
  launch_pdl(L, k_slot_mass_tc<HD>, dim3(units < sms ? (int)units : sms), dim3(N_THREADS), smem, map, map_q, k);
}

}  // namespace

void launch_paged_mass_tc(Launcher& L, const PagedMassArgs& s, const void* pool) {
  const PagedAttnArgs& a = s.a;
  // (units are fewer than the attention's, which are below 2^31)
  const long long units = (long long)a.batch * a.g.Hkv * (((long long)a.g.max_pages * a.g.page + KT - 1) / KT);
  Args k;
  memset(&k, 0, sizeof(k));
  k.s = s;
  k.pass_rows = MAX_LINES / a.G < a.rows ? MAX_LINES / a.G : a.rows;
  k.rows_total = a.g.n_pages * 2 * a.g.Hkv * a.g.page;
  while (1 << k.page_shift < a.g.page) ++k.page_shift;
  const bf16* layer = reinterpret_cast<const bf16*>(pool) + page_offset(a.g, a.layer, 0, 0, 0);
  CUtensorMap map, map_q;
  if (!paged_kv_map(&map, a, layer, a.g.page < KT ? a.g.page : KT) || !paged_q_map(&map_q, a, k.pass_rows)) {
    L.err = POSS_E_CUDA;
    return;
  }
  if (a.g.d == 128) launch<128>(L, k, map, map_q, units);
  else launch<64>(L, k, map, map_q, units);
}
