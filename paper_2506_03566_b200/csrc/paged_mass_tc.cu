// The weight that every slot draws, on the 5th-generation tensor cores (bf16, head dimension 64 or 128).
//
// Scores are formed with the keys as rows and the query lines (tree row, head) as columns: S^T = K Q^T, 128 slots times up to 256 lines.
// A slot is then a lane of TMEM, its thread takes its own lane's scores, adds w / l 2^(scale s - m) up over the columns and writes one
// number: no sum crosses threads.  A column's constants (-m, w / l) come from shared memory, the same address for all lanes.
//
// A tile is 128 slots of one (sequence, KV head).  The tiles of the whole batch, weighed by their lines, are cut into one contiguous range
// per CTA, one CTA per SM (16 trees of 12 to 61 rows, cut by tiles alone: 106 us).  More than 256 lines take a pass each over the CTA's
// slots; the later ones add to what the first has written.
//   warps 0-15  weights: four groups of four warps, each every fourth 16 of a tile's columns; they leave their sums in shared memory, and
//               a tile later one group, in turn, adds the four and writes the tile's weights.  Groups wait for one another only where a
//               score buffer is to be filled again (meeting once per tile cost 0.3 us each of 1.6), and the next tile's product runs
//               meanwhile into the other buffer.
//   warp 16     keys, through a ring of stages (one box per page and 64 columns), and a pass's queries
//   warp 17     products, one lane
// What bounds it: nothing alone.  16 trees of 12 to 61 rows of 4 heads over 4096 to 8191 slots take 77 us, of which the exponentials (8 cycles
// per tile and line: 128 lanes at 16 a cycle and SM) would need 28 and the keys 31; by the counters the exponentials' pipe is busy 38 % of the
// time, the schedulers issue 1.9 instructions of 4 a cycle, and warps mostly wait for fixed latencies, loads of TMEM and shared memory.  Clocks
// read in one warp show 10 to 17 cycles per line in the powers and sums and some 500 per tile in waits and hand-overs; a least-squares fit
// over all CTAs gives 1394 per tile and 7.2 per line, fewer than the exponentials alone take: it splits the two wrongly, though their sum is
// right for trees of these sizes, which is what the cut of the work goes by.  Measured and not better there: 8 warps, each all columns of every second tile, 94 us; two groups per tile and parity, each half of the columns, 81 to 88;
// four buffers of 128 columns, 87; a quarter of the 2^x as a polynomial on the multiply-add pipe, 82; 32 columns at a time in two steps, 89
// (registers).  Reads of TMEM were measured at 413 bytes a cycle and SM and are no bound.  (Calls of few lines take the weights from the
// attention's own scores instead: paged_attention_tc.cu.)
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
constexpr int GROUPS = 4;               // of 128 threads that form weights, one per slot of the tile
constexpr int N_SUMS = GROUPS * KT;
constexpr int N_THREADS = N_SUMS + 64;
constexpr int WARP_KEYS = 16, WARP_MMA = 17;
constexpr int K_BLOCK = KT * 128;       // bytes of 128 slots x 64 bf16
constexpr int Q_BLOCK = MAX_LINES * 128;
constexpr int MAX_STAGES = 6;
constexpr uint32_t TMEM_COLS = 512;     // two buffers of 256 columns

// What a tile costs beside its lines, in lines: 1394 cycles and 7.2 for each line, the fit over the times of all CTAs for 16 trees of 12 to 61
// rows.
constexpr uint32_t TILE_WEIGHT = 192;

template <int HD> struct Shape {
  static constexpr int CB = HD / 64;
  static constexpr int TILE = CB * K_BLOCK, Q_BYTES = CB * Q_BLOCK;
  static constexpr int NK = HD == 128 ? 4 : 6;
  static constexpr int K_OFF = Q_BYTES, CTL_OFF = K_OFF + NK * TILE;
};

struct Work {
  int prefix, rows, total, tiles;
  uint32_t n_tiles;                     // of all heads (a batch's fit 31 bits: checked on the host)
  uint32_t weight;                      // of one tile
};
struct Args {
  PagedMassArgs s;
  int pass_rows;                        // tree rows per pass
  int rows_total;                       // rows of the pool's layer: the first coordinate behind it
  int page_shift;
  int inject_lost_load;
};
__device__ __forceinline__ Work work_of(const PagedAttnArgs& a, int b) {
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows, (long long)a.g.max_pages * a.g.page);
  Work w;
  w.prefix = n.prefix; w.rows = n.rows;
  w.total = n.prefix + n.rows;
  w.tiles = n.rows ? (w.total + KT - 1) / KT : 0;
  w.n_tiles = (uint32_t)a.g.Hkv * w.tiles;
  w.weight = TILE_WEIGHT + (uint32_t)(n.rows * a.G);
  return w;
}
// Barriers are waited for by parity; no role can be two phases ahead of another on one: keys by the ring, scores by s_empty, queries by
// q_empty, which follows the pass's last product.  Sums have four places: a group writes a tile's once its scores are there, so that all
// groups have left the tile before the last; the group that adds up the tile four before did so ahead of that one.
constexpr int PLACES = 4;
struct Ctl {
  uint64_t k_full[MAX_STAGES], k_empty[MAX_STAGES], q_full, q_empty, s_full[2], s_empty[2], sums[PLACES], drain;
  uint32_t tmem;
  int abort;
  uint32_t n_tiles, offset;             // tiles of the CTA's range; the first one's place inside its sequence
  int seq;
  // by pass, in turn: two columns' (-m, -m, w / l, w / l), and by slot of the call's rows the columns that see it
  float4 col[2][MAX_LINES / 2];
  uint32_t sees[2][POSS_MAX_ROWS][MAX_LINES / 32];
  float part[PLACES][GROUPS][KT];       // the groups' sums
};

// a CTA's passes in order; every role walks them by itself
struct Pass {
  int b, head, tile0, n, group;         // n tiles from tile0 on, the group-th `pass_rows` rows
  Work w;
};
struct Walk {
  uint32_t left, offset;                // tiles still to come; the next one's place inside sequence b
  int b, group, groups;
  __device__ __forceinline__ void start(const Ctl& c, const PagedAttnArgs& a, Pass* p) {
    left = c.n_tiles; offset = c.offset; b = c.seq;
    group = groups = 0;
    if (left) p->w = work_of(a, b);
  }
  __device__ __forceinline__ bool next(const Args& k, Pass* p) {
    const PagedAttnArgs& a = k.s.a;
    if (group + 1 < groups) {
      p->group = ++group;
      return true;
    }
    if (left == 0) return false;
    while (offset >= p->w.n_tiles) {
      offset -= p->w.n_tiles;
      if (++b >= a.batch) return false;                     // (not reached: the range lies inside the batch's tiles)
      p->w = work_of(a, b);
    }
    p->b = b;
    p->head = (int)(offset / (uint32_t)p->w.tiles);
    p->tile0 = (int)(offset - (uint32_t)p->head * p->w.tiles);
    p->n = min(p->w.tiles - p->tile0, (int)left);
    left -= p->n;
    offset += p->n;
    p->group = group = 0;
    groups = (p->w.rows + k.pass_rows - 1) / k.pass_rows;
    return true;
  }
};

__device__ __forceinline__ void tmem_ld16_async(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                 "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
// orders the use of registers behind the wait for the loads that fill them
__device__ __forceinline__ void tie16(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]),
                 "+r"(r[i + 6]), "+r"(r[i + 7]));
}
// adds w / l 2^(scale s - m) of 16 columns
__device__ __forceinline__ void add16(const uint32_t* s, const float4* col, float2 scale, float2& s0, float2& s1) {
#pragma unroll
  for (int x = 0; x < 16; x += 4) {
    const float4 a = col[x / 2], b = col[x / 2 + 1];
    const float2 u = fma2(make_float2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), scale, make_float2(a.x, a.y));
    const float2 v = fma2(make_float2(__uint_as_float(s[x + 2]), __uint_as_float(s[x + 3])), scale, make_float2(b.x, b.y));
    s0 = fma2(make_float2(ex2(u.x), ex2(u.y)), make_float2(a.z, a.w), s0);
    s1 = fma2(make_float2(ex2(v.x), ex2(v.y)), make_float2(b.z, b.w), s1);
  }
}
// the same of the columns whose bit is set; what the others hold is of no account
__device__ __forceinline__ void add16_of(uint32_t bits, const uint32_t* s, const float4* col, float2 scale, float2& s0, float2& s1) {
#pragma unroll
  for (int x = 0; x < 16; x += 2) {
    const float4 a = col[x / 2];
    const float2 u = fma2(make_float2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), scale, make_float2(a.x, a.y));
    const float p = ex2(u.x) * a.z, q = ex2(u.y) * a.w;
    s0 = add2(s0, make_float2((bits >> x) & 1u ? p : 0.f, (bits >> x) & 2u ? q : 0.f));
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
        mbar_init(bar(c.s_empty[i]), N_SUMS / 32);
      }
      for (int i = 0; i < PLACES; ++i) mbar_init(bar(c.sums[i]), N_SUMS / 32);
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
    // The batch's weight is cut evenly; a tile belongs to the CTA whose share its first gram lies in.  Tiles before a place, counted over
    // the sequences, give the CTA's first tile and the one behind its last.
    uint64_t w = 0;
    for (int x = lane; x < a.batch; x += 32) {
      const Work own = work_of(a, x);
      w += (uint64_t)own.n_tiles * own.weight;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
    const uint64_t each = w / gridDim.x, more = w - each * gridDim.x;
    uint64_t begin = blockIdx.x * each + min((uint64_t)blockIdx.x, more);
    uint64_t end = begin + each + (blockIdx.x < more);
    if (lane == 0) { c.n_tiles = 0; c.seq = 0; c.offset = 0; }
    __syncwarp();
    uint32_t mine = 0, place = 0;
    int seq = -1;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
      Work own;
      own.n_tiles = 0; own.weight = 1;
      if (b0 + lane < a.batch) own = work_of(a, b0 + lane);
      const uint64_t weight = (uint64_t)own.n_tiles * own.weight;
      uint64_t x = weight;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      const uint64_t before = x - weight;
      // the sequence's tiles whose first gram lies in [begin, end)
      auto first_from = [&](uint64_t at) {
        if (at <= before) return 0u;
        const uint64_t n = (at - before + own.weight - 1) / own.weight;
        return n < own.n_tiles ? (uint32_t)n : own.n_tiles;
      };
      const uint32_t t0 = first_from(begin), t1 = first_from(end), n = t1 - t0;
      const unsigned here = __ballot_sync(0xffffffffu, n > 0);
      if (here && seq < 0) {
        seq = b0 + __ffs(here) - 1;
        place = __shfl_sync(0xffffffffu, t0, __ffs(here) - 1);
      }
      mine += __reduce_add_sync(0xffffffffu, n);
      const uint64_t all = __shfl_sync(0xffffffffu, x, 31);
      begin = begin > all ? begin - all : 0;
      end = end > all ? end - all : 0;
      if (end == 0) break;
    }
    if (lane == 0 && mine) { c.n_tiles = mine; c.seq = seq; c.offset = place; }
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
      // -------------------------------------------------------------- weights, a thread per slot and quarter of the columns
      const int group = warp >> 2, par = pass & 1, row = (warp & 3) * 32 + lane;
      if (threadIdx.x < MAX_LINES) {
        // the pass's columns: a thread each
        const int col = threadIdx.x, r = r0 + col / a.G;
        float2 ml = make_float2(INFINITY, 0.f);
        float w = 0.f;
        uint64_t lo = 0, hi = 0;
        if (col < lines) {
          const size_t at = (size_t)p.b * a.rows + r;
          ml = a.ml[at * a.Hq + p.head * a.G + col % a.G];
          w = k.s.weights ? k.s.weights[at] : 1.f;
          paged_row_mask(a.mask, at, a.mask_words, p.w.rows, &lo, &hi);
        }
        float* f = reinterpret_cast<float*>(&c.col[par][col >> 1]) + (col & 1);
        f[0] = -ml.x;
        f[2] = w * ml.y;
        // the ancestor bits of 32 columns, turned: a slot's word has a bit for each
        if ((p.tile0 + p.n) * KT > p.w.prefix)
#pragma unroll 1
          for (int j0 = 0; j0 < p.w.rows; j0 += 32) {
            const uint32_t bits = (uint32_t)((j0 < 64 ? lo : hi) >> (j0 & 32));
            uint32_t word = 0;
#pragma unroll 8
            for (int j = 0; j < 32; ++j) {
              const uint32_t x = __ballot_sync(0xffffffffu, (bits >> j) & 1u);
              if (lane == j) word = x;
            }
            c.sees[par][j0 + lane][col >> 5] = word;
          }
      }
      asm volatile("bar.sync 1, 512;" ::: "memory");
      const float2 scale = make_float2(k.s.scale_log2, k.s.scale_log2);
      const float4* const cols = c.col[par];
      float* const mass = k.s.mass + ((size_t)p.b * a.g.Hkv + p.head) * k.s.mass_slots;
      // what the slot held, and its page: asked for four tiles ahead, for the tiles that the group writes
      int mine = (group - done) & (GROUPS - 1);
      float old = 0.f;
      int entry = -1;
      auto ask = [&](int t) {
        const int key = (p.tile0 + t) * KT + row;
        old = 0.f;
        entry = -1;
        if (t < p.n && key < p.w.total) {
          entry = table[key >> k.page_shift];             // (looked at when it is needed: a look would wait for it)
          if (key < p.w.prefix || p.group > 0) old = mass[key];
        }
      };
      auto add_up = [&] {
        const int n = done + mine, key = (p.tile0 + mine) * KT + row;
        wait(c.sums[n % PLACES], n / PLACES);
        float sum = c.part[n % PLACES][0][row];
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) sum += c.part[n % PLACES][i][row];
        if (key < p.w.total && ok) mass[key] = old + (entry >= 0 && entry < a.g.n_pages ? sum : 0.f);
        mine += GROUPS;
        ask(mine);
      };
      static_assert(PLACES == GROUPS, "a group writes the tiles of one place");
      ask(mine);
#pragma unroll 1
      for (int t = 0; t < p.n; ++t) {
        const int n = done + t, buf = n & 1, key0 = (p.tile0 + t) * KT;
        const uint32_t t_s = tm + ((uint32_t)((warp & 3) * 32) << 16) + buf * MAX_LINES;
        wait(c.s_full[buf], n >> 1);
        tc_fence_after();
        float2 s0 = make_float2(0.f, 0.f), s1 = s0;
        // the columns that see the slot; all of them see a committed one
        const int j = key0 + row - p.w.prefix;
        const bool partly = key0 + KT > p.w.prefix;
        const uint32_t* const sees = c.sees[par][j < 0 || j >= p.w.rows ? 0 : j];
        // the group's columns: 16 of every 64.  (The next ones are on their way while these are worked on.)
        auto add = [&](int x, uint32_t* r) {
          const float4* const f = cols + x / 2;
          if (partly || x + 16 > lines) {                 // (columns behind the last line hold anything)
            uint32_t bits = 0xffffu >> (x + 16 > lines ? x + 16 - lines : 0);
            if (j >= 0) bits &= j < p.w.rows ? sees[x >> 5] >> (x & 16) : 0u;
            add16_of(bits, r, f, scale, s0, s1);
          } else {
            add16(r, f, scale, s0, s1);
          }
        };
        uint32_t r[2][16];
        int x = group * 16;
        if (x < lines) tmem_ld16_async(t_s + x, r[0]);
#pragma unroll 1
        while (x < lines) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            if (x < lines) {
              tmem_wait_ld();
              tie16(r[y]);
              if (x + 64 < lines) tmem_ld16_async(t_s + x + 64, r[y ^ 1]);
              add(x, r[y]);
              x += 64;
            }
          }
        }
        tc_fence_before();
        c.part[n % PLACES][group][row] = (s0.x + s0.y) + (s1.x + s1.y);
        __syncwarp();
        if (lane == 0) {                                  // (an arrival of every thread would take 0.5 us)
          mbar_arrive(bar(c.s_empty[buf]));
          mbar_arrive(bar(c.sums[n % PLACES]));
        }
        if (mine < t) add_up();                           // a tile behind: the others' sums are there
      }
      if (mine < p.n) add_up();
    } else if (warp == WARP_KEYS) {
      // -------------------------------------------------------------- keys, a lane per page of a tile; the pass's queries
      // (a table's entries are fetched 32 at a time, one batch of tiles ahead: one by one a tile would take a trip to memory)
      const int page = a.g.page, per_tile = page < KT ? KT / page : 1, batch = 32 / per_tile;
      auto fetch = [&](int t) {
        const int key0 = (p.tile0 + t + lane / per_tile) * KT + lane % per_tile * page;
        return key0 < p.w.total ? page_at(table, a.g.max_pages, a.g.n_pages, key0 >> k.page_shift) : -1;
      };
      int pages = -1, next = fetch(0);
      const int with = min(p.n, Z::NK - 1) - 1;           // the queries follow this tile: the first ones need not wait for their place
#pragma unroll 1
      for (int t = 0; ok && t < p.n; ++t) {
        const int in_batch = t & (batch - 1);
        if (in_batch == 0) {
          pages = next;
          if (t + batch < p.n) next = fetch(t + batch);
        }
        const int at_page = __shfl_sync(0xffffffffu, pages, (in_batch * per_tile + lane) & 31);
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
            for (int cb = k.inject_lost_load ? Z::CB : 0; cb < Z::CB; ++cb) tma_load_5d(base + cb * Q_BLOCK, &map_q, bar(c.q_full), cb * 64, p.head, r0, p.b);
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

template <int HD> void launch(Launcher& L, const Args& k, const CUtensorMap& map, const CUtensorMap& map_q, long long tiles) {
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
  launch_pdl(L, k_slot_mass_tc<HD>, dim3(tiles < sms ? (int)tiles : sms), dim3(N_THREADS), smem, map, map_q, k);
}

}  // namespace

void launch_paged_mass_tc(Launcher& L, const PagedMassArgs& s, const void* pool) {
  const PagedAttnArgs& a = s.a;
  // (fewer than the attention's units, which are below 2^31)
  const long long tiles = (long long)a.batch * a.g.Hkv * (((long long)a.g.max_pages * a.g.page + KT - 1) / KT);
  Args k;
  memset(&k, 0, sizeof(k));
  k.s = s;
  k.pass_rows = MAX_LINES / a.G < a.rows ? MAX_LINES / a.G : a.rows;
  k.rows_total = a.g.n_pages * 2 * a.g.Hkv * a.g.page;
  while (1 << k.page_shift < a.g.page) ++k.page_shift;
  k.inject_lost_load = paged_take_lost_load();
  const bf16* layer = reinterpret_cast<const bf16*>(pool) + page_offset(a.g, a.layer, 0, 0, 0);
  CUtensorMap map, map_q;
  if (!paged_kv_map(&map, a, layer, a.g.page < KT ? a.g.page : KT) || !paged_q_map(&map_q, a, k.pass_rows)) {
    L.err = POSS_E_CUDA;
    return;
  }
  if (a.g.d == 128) launch<128>(L, k, map, map_q, tiles);
  else launch<64>(L, k, map, map_q, tiles);
}
