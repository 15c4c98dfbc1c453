// Tree-masked attention over pages on the 5th-generation tensor cores (bf16, head dimension 64 or 128).
//
// The G = Hq / Hkv query heads of a KV head and a sequence's tree rows form one matrix of query rows (row * G + head), cut
// into items of up to 256: (sequence, KV head, 256 query rows).  A unit of work is one item's product with 128 keys; the
// units of the whole batch, in order of sequence, head, item and key, are cut into one contiguous range per CTA, one CTA
// per SM, so that every SM streams the same number of keys however long the sequences are.  The part of an item that
// falls into one CTA is a segment: one pass over its keys with the running maximum and sum of a softmax.  A segment that is
// the whole item writes the output, any other leaves fp32 partials that a second kernel merges in key order.
//
// Inside a CTA two "slots" of 128 query rows share the key tiles:
//   * items with more than 128 query rows: slot = half of the rows, both use every tile (each key is read once);
//   * smaller items: both slots hold the same rows and take the even / the odd tiles; they are merged at the end.
// Warps 0-3 / 4-7 do the softmax of slot 0 / 1 (one thread per query row), one thread of warp 8 issues the products,
// warp 9 the copies:
//   * copies: TMA, one box per page and 64 columns, keys and values of a tile in turn through a ring of stages.  A page that
//     is missing or behind the last slot is read from behind the pool: zeros;
//   * S = Q K^T (fp32, TMEM); the softmax thread reads its row of S once (128 registers), masks it where the tile reaches the
//     tree, takes the maximum, writes P = 2^(s - m) as bf16 over S in TMEM; O += P V with P as the TMEM operand;
//   * the reference maximum m moves only when a row's maximum has grown by more than 2^8 (P stays below 2^8, which bf16
//     and the fp32 sums hold as well as 1): then the thread scales its row of O in TMEM.  Otherwise O is never touched;
//   * while one slot's softmax runs, the other slot's products do.
//
// Unseen slots.  A score is replaced by -inf, so what a key holds is of no account.  A value is multiplied by an exact zero,
// which is not enough for infinities and NaN: in tiles that reach behind the committed slots the values behind the last slot
// are set to zero, and infinities and NaN of tree slots too, in shared memory; the rows that do see such a slot get them
// added at the end.
//
// The probabilities are rounded to bf16 (half a step, 2^-8): the second product's error stays near that of the output's
// own rounding.  Sums, maxima and accumulators are fp32.
//
// What bounds it: with one token per sequence the read of keys and values; with 61 rows of 4 heads the products and the
// exponentials come near to it.  DRAM traffic is the keys and values once.
//
// Every wait is bounded; on expiry the CTA raises POSS_E_TIMEOUT, runs through its (bounded) walk without meaning, waits
// (bounded) for its copies in flight, frees its TMEM and returns.
#include "paged_attention.cuh"
#include "tc_ptx.cuh"
#include <atomic>
#include <string.h>

POSS_TRACE_REGISTER()

namespace {

using namespace tcptx;

constexpr int KT = 128;                 // keys per tile
constexpr int QR = 128;                 // query rows per slot
constexpr int ITEM_ROWS = 2 * QR;
constexpr int N_SOFTMAX = 256;
constexpr int N_THREADS = N_SOFTMAX + 64;
constexpr int WARP_MMA = 8, WARP_TMA = 9;
constexpr int BLOCK = QR * 128;         // bytes of 128 rows x 64 bf16
constexpr int MAX_STAGES = 8;
constexpr float RESCALE_LOG2 = 8.f;
constexpr uint32_t TMEM_COLS = 512;

template <int HD> struct Shape {
  static constexpr int CB = HD / 64;                      // 64-column blocks
  static constexpr int TILE = CB * BLOCK;                 // bytes of a key, value or query tile
  static constexpr int STAGES = HD == 128 ? 5 : 8;
  static constexpr int Q_OFF = 0, KV_OFF = 2 * TILE, CTL_OFF = KV_OFF + STAGES * TILE;
};

struct Ctl {
  uint64_t kv_full[MAX_STAGES], kv_empty[MAX_STAGES], q_full, s_full[2], p_full[2], pv_done[2], o_free, drain;
  uint32_t tmem;
  int abort;
  int missing[2];                       // by parity of the segment: a page that the segment needs is not there
  unsigned long long nonfinite[2][2];   // by parity: tree slots whose values hold infinities or NaN
  long long total;                      // units of the batch
  long long offset0;                    // the CTA's first unit inside its first sequence
  int seq0, grid;                       // that sequence; CTAs that share the units
  float2 ml[2][QR];                     // a slot's maximum and sum, for the merge of two slots with the same rows
};
static_assert(sizeof(Ctl) <= 3072, "the control block lies behind the tiles");

struct TcArgs {
  PagedAttnArgs a;
  float scale_log2;                     // |scale| log2 e
  uint32_t q_flip;                      // sign bits of two bf16 where the scale is negative
  int row_cap;                          // query rows that a partial has room for
  int rows_total;                       // rows of the pool's layer: the first coordinate behind it
  int inject_lost_load;
  uint32_t smem_bytes;
  const bf16* layer;                    // the layer's first element
};

// ---- the units of a sequence
struct SeqWork {
  int prefix, rows, total, tiles, nq, groups;   // groups: items per KV head
  long long units;
  bool bad;
};
__device__ __forceinline__ SeqWork seq_work(const PagedAttnArgs& a, int b) {
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows,
                              (long long)a.g.max_pages * a.g.page);
  SeqWork s;
  s.bad = n.bad; s.prefix = n.prefix; s.rows = n.rows;
  s.total = n.prefix + n.rows;
  s.tiles = (s.total + KT - 1) / KT;
  s.nq = n.rows * a.G;
  s.groups = (s.nq + ITEM_ROWS - 1) / ITEM_ROWS;
  s.units = (long long)s.groups * a.g.Hkv * s.tiles;      // no rows: no groups
  return s;
}
// One warp: units of all sequences, and of those before sequence `upto`.
__device__ __forceinline__ void count_units(const PagedAttnArgs& a, int upto, long long* total, long long* before) {
  const int lane = threadIdx.x & 31;
  long long t = 0, f = 0;
  for (int b = lane; b < a.batch; b += 32) {
    const long long u = seq_work(a, b).units;
    t += u;
    if (b < upto) f += u;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    t += __shfl_xor_sync(0xffffffffu, t, o);
    f += __shfl_xor_sync(0xffffffffu, f, o);
  }
  *total = t;
  *before = f;
}
// CTAs that share `total` units
__device__ __forceinline__ int unit_grid(long long total, int ctas) {
  return total < ctas ? (total < 1 ? 1 : (int)total) : ctas;
}
__device__ __forceinline__ long long range_begin(long long c, long long total, int grid) { return c * total / grid; }
__device__ __forceinline__ int cta_of_unit(long long u, long long total, int grid) {
  return (int)(((u + 1) * grid + total - 1) / total - 1);   // the largest c with range_begin(c) <= u
}

struct Segment {
  int b, head, group, tile0, n;         // n tiles from tile0 on
  SeqWork s;
};
// A CTA's segments in order; every role walks them by itself.
struct Walk {
  long long u, u_end, offset;
  int b;
  __device__ __forceinline__ void start(const Ctl& c) {
    u = blockIdx.x < c.grid ? range_begin(blockIdx.x, c.total, c.grid) : c.total;
    u_end = blockIdx.x < c.grid ? range_begin(blockIdx.x + 1, c.total, c.grid) : c.total;
    b = c.seq0;
    offset = c.offset0;
  }
  __device__ __forceinline__ bool next(const PagedAttnArgs& a, Segment* g) {
    if (u >= u_end) return false;
    g->s = seq_work(a, b);
    while (offset >= g->s.units) {
      offset -= g->s.units;
      if (++b >= a.batch) return false;                   // (not reached: the range lies inside the batch's units)
      g->s = seq_work(a, b);
    }
    g->b = b;
    const long long item = offset / g->s.tiles;
    g->tile0 = (int)(offset - item * g->s.tiles);
    g->head = (int)(item / g->s.groups);
    g->group = (int)(item - (long long)g->head * g->s.groups);
    const long long left = u_end - u;
    g->n = g->s.tiles - g->tile0;
    if (g->n > left) g->n = (int)left;
    u += g->n;
    offset += g->n;
    return true;
  }
};
// two slots of different rows (true) or of the same rows and alternating tiles
__device__ __forceinline__ bool two_halves(const Segment& g) { return g.s.nq - g.group * ITEM_ROWS > QR; }

// ---- PTX
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
               "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
                 "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
                 "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
                 "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {"
               "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {"
               "%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
               "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                 "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                 "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// orders the use of registers behind the wait for the loads that fill them
__device__ __forceinline__ void tie32(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]),
                 "+r"(r[i + 6]), "+r"(r[i + 7]));
}
// A from TMEM, B from shared memory
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// MN-major operand, 128-byte swizzle: 64 columns are one 128-byte line, consecutive keys consecutive lines, 8-line groups
// 1024 bytes apart, the next 64 columns one BLOCK further
__device__ __forceinline__ uint64_t smem_desc_values(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(BLOCK >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= 1ull << 46;
  d |= 2ull << 61;
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool nonfinite2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite2(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
  return w;
}

// where a CTA leaves the partials of its first (which 0) and of its last (1) segment: [HD/4][row_cap][4] outputs, then
// [row_cap] pairs (maximum, sum)
__device__ __forceinline__ float* partial_of(const TcArgs& k, int hd, int cta, int which) {
  return reinterpret_cast<float*>(k.a.ws) + ((size_t)cta * 2 + which) * ((size_t)k.row_cap * (hd + 2));
}

// ---------------------------------------------------------------------------------------------------- the kernel
template <int HD>
__global__ void __launch_bounds__(N_THREADS, 1) k_paged_attn_tc(const __grid_constant__ CUtensorMap map, const TcArgs k) {
  using Z = Shape<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Ctl& c = *reinterpret_cast<Ctl*>(smem + Z::CTL_OFF);
  const uint32_t base = smem_u32(smem);
  const PagedAttnArgs& a = k.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](uint64_t& x) { return smem_u32(&x); };

  if (warp == WARP_MMA) {
    if (lane == 0) {
      // (tiles start on 1024 bytes and fit: checked on the host, and here)
      c.abort = (base & 1023u) || Z::CTL_OFF + sizeof(Ctl) > k.smem_bytes ? 1 : 0;
      c.missing[0] = c.missing[1] = 0;
      for (int i = 0; i < 2; ++i) c.nonfinite[i][0] = c.nonfinite[i][1] = 0;
      for (int i = 0; i < Z::STAGES; ++i) {
        mbar_init(bar(c.kv_full[i]), 1);
        mbar_init(bar(c.kv_empty[i]), 1);
      }
      mbar_init(bar(c.q_full), N_SOFTMAX);
      mbar_init(bar(c.o_free), N_SOFTMAX);
      mbar_init(bar(c.drain), 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(bar(c.s_full[i]), 1);
        mbar_init(bar(c.p_full[i]), QR);
        mbar_init(bar(c.pv_done[i]), 1);
      }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      prefetch_tensormap(&map);
    }
    __syncwarp();
    tmem_alloc(smem_u32(&c.tmem), TMEM_COLS);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  volatile int* abort_flag = &c.abort;
  const uint32_t tm = c.tmem;
  // The successor may start only now that this CTA holds its TMEM columns: one that took columns on this SM first would
  // keep them until this grid has finished.
  pdl_begin();
  pdl_sync(POSS_K_PAGED_ATTN);

  if (warp == 0) {
    // the batch's units, and the sequence that the CTA's first one lies in
    long long total, none;
    count_units(a, 0, &total, &none);
    const int grid = unit_grid(total, (int)gridDim.x);
    if ((int)blockIdx.x < grid && total > 0) {
      long long at = range_begin(blockIdx.x, total, grid);
      for (int b0 = 0; b0 < a.batch; b0 += 32) {
        const long long u = b0 + lane < a.batch ? seq_work(a, b0 + lane).units : 0;
        long long x = u;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const long long y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        const unsigned here = __ballot_sync(0xffffffffu, at < x);
        if (here) {
          const int first = __ffs(here) - 1;
          if (lane == first) {
            c.seq0 = b0 + first;
            c.offset0 = at - (x - u);
          }
          break;
        }
        at -= __shfl_sync(0xffffffffu, x, 31);
      }
    }
    if (lane == 0) {
      c.total = total;
      c.grid = total > 0 ? grid : 0;
    }
    if (blockIdx.x == 0)
      for (int b = lane; b < a.batch; b += 32)
        if (seq_work(a, b).bad) raise_status(a.status, POSS_E_INVALID);
  }
  __syncthreads();

  Walk walk;
  walk.start(c);
  Segment g;

  if (warp == WARP_TMA) {
    // ---------------------------------------------------------------- copies
    const int page = a.g.page, per_tile = page < KT ? KT / page : 1;
    const uint64_t policy = policy_evict_normal();
    int idx = 0;                                          // tiles loaded so far, keys and values counted apart
    bool ok = __all_sync(0xffffffffu, *abort_flag == 0);
    while (ok && walk.next(a, &g)) {
      const int32_t* table = a.g.tables + (size_t)g.b * a.g.max_pages;
      // the lane's page of a tile (lanes below per_tile), fetched one tile ahead
      auto fetch = [&](int tile) {
        const int key0 = tile * KT + lane * page;
        int p = -1;
        if (lane < per_tile && key0 < g.s.total) {
          p = page_at(table, a.g.max_pages, a.g.n_pages, key0 / page);
          if (p < 0) raise_status(a.status, POSS_E_INVALID);
        }
        return p;
      };
      int p_next = fetch(g.tile0);
      for (int t = 0; ok && t < g.n; ++t) {
        const int p = p_next;
        if (t + 1 < g.n) p_next = fetch(g.tile0 + t + 1);
        const int in_page = page > KT ? (g.tile0 + t) * KT % page : 0;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++idx) {
          const int st = idx % Z::STAGES, turn = idx / Z::STAGES;
          if (turn > 0) ok = mbar_wait(bar(c.kv_empty[st]), (uint32_t)((turn - 1) & 1), abort_flag);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const uint32_t full = bar(c.kv_full[st]), dst = base + Z::KV_OFF + st * Z::TILE;
          if (lane == 0) mbar_expect_tx(full, Z::TILE);
          __syncwarp();
          if (lane < per_tile && !(k.inject_lost_load && kv)) {
            const int row = p >= 0 ? ((p * 2 + kv) * a.g.Hkv + g.head) * page + in_page : k.rows_total;
#pragma unroll
            for (int cb = 0; cb < Z::CB; ++cb)
              tma_load_2d(dst + cb * BLOCK + lane * page * 128, &map, full, cb * 64, row, policy);
          }
          __syncwarp();
        }
      }
    }
    if (*abort_flag) {
      // the copies under way must land before the CTA's shared memory goes away
      const uint64_t t0 = global_ns();
      for (int i = idx > Z::STAGES ? idx - Z::STAGES : 0; i < idx; ++i)
        while (!mbar_try_wait(bar(c.kv_full[i % Z::STAGES]), (uint32_t)((i / Z::STAGES) & 1)) &&
               global_ns() - t0 < WAIT_LIMIT_NS / 2)
          __nanosleep(64);
    }
  } else if (warp == WARP_MMA) {
    // ---------------------------------------------------------------- products
    if (lane == 0) {
      const uint32_t idesc_s = instr_desc_bf16(QR, KT);
      const uint32_t idesc_o = instr_desc_bf16(QR, HD) | (1u << 16);     // the values are MN-major
      int tiles_before = 0, seg = 0;
      int n_pv[2] = {0, 0};                               // second products issued per slot
      bool ok = *abort_flag == 0;
      auto wait = [&](uint64_t& b, int phase) { ok = ok && mbar_wait(bar(b), (uint32_t)(phase & 1), abort_flag); };
      for (; ok && walk.next(a, &g); ++seg) {
        const bool halves = two_halves(g);
        const int steps = halves ? 2 * g.n : g.n;
        auto tile_of = [&](int x) { return halves ? x >> 1 : x; };
        auto issue_s = [&](int x) {
          const int slot = x & 1, i = 2 * (tiles_before + tile_of(x)), st = i % Z::STAGES;
          if (!halves || !(x & 1)) wait(c.kv_full[st], i / Z::STAGES);
          if (!ok) return;
          tc_fence_after();
          const uint32_t d = tm + slot * KT, kb = base + Z::KV_OFF + st * Z::TILE, qb = base + Z::Q_OFF + slot * Z::TILE;
#pragma unroll
          for (int cb = 0; cb < Z::CB; ++cb) {
            const uint64_t ad = smem_desc_sw128(qb + cb * BLOCK), bd = smem_desc_sw128(kb + cb * BLOCK);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)                // 16 bf16 = 32 bytes = 2 address units
              umma_bf16(d, ad + (uint64_t)(2 * kk), bd + (uint64_t)(2 * kk), idesc_s, (cb | kk) ? 1u : 0u);
          }
          umma_commit(bar(c.s_full[slot]));
          if (!halves || (x & 1)) umma_commit(bar(c.kv_empty[st]));
        };
        wait(c.q_full, seg);
        // P of a slot lies over its S: the last segment's second products must have read theirs
        for (int s = 0; s < 2; ++s)
          if (n_pv[s] > 0) wait(c.pv_done[s], n_pv[s] - 1);
        issue_s(0);
        if (steps > 1) issue_s(1);
        for (int x = 0; ok && x < steps; ++x) {
          const int slot = x & 1, t = tile_of(x), i = 2 * (tiles_before + t) + 1, st = i % Z::STAGES;
          wait(c.p_full[slot], n_pv[slot]);
          if (x == 0 && seg > 0) wait(c.o_free, seg - 1);
          if (!halves || !(x & 1)) wait(c.kv_full[st], i / Z::STAGES);
          if (!ok) break;
          tc_fence_after();
          const int keys = g.s.total - (g.tile0 + t) * KT, n16 = keys >= KT ? KT / 16 : (keys + 15) / 16;
          const uint32_t d = tm + 2 * KT + slot * HD, p = tm + slot * KT, vb = base + Z::KV_OFF + st * Z::TILE;
          for (int ks = 0; ks < n16; ++ks)
            umma_bf16_ts(d, p + ks * 8, smem_desc_values(vb + ks * 2048), idesc_o, (x >= 2 || ks > 0) ? 1u : 0u);
          umma_commit(bar(c.pv_done[slot]));
          if (!halves || (x & 1)) umma_commit(bar(c.kv_empty[st]));
          ++n_pv[slot];
          if (x + 2 < steps) {
            wait(c.pv_done[slot], n_pv[slot] - 1);        // P has been read: S may take its place
            issue_s(x + 2);
          }
        }
        tiles_before += g.n;
      }
      if (*abort_flag) {
        // the products under way must end before the CTA's TMEM and shared memory go away
        const uint64_t t0 = global_ns();
        umma_commit(bar(c.drain));
        while (!mbar_try_wait(bar(c.drain), 0) && global_ns() - t0 < WAIT_LIMIT_NS / 2) __nanosleep(64);
      }
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- softmax, one thread per query row
    const int wg = warp >> 2, row = (warp & 3) * 32 + lane, tid = threadIdx.x;
    const uint32_t t_lane = tm + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t t_s = t_lane + wg * KT, t_o = t_lane + 2 * KT + wg * HD;
    int tiles_before = 0, n_s = 0, n_other = 0;           // steps of this slot / of the other one so far
    bool ok = true;
    auto wait = [&](uint64_t& b, int phase) { ok = ok && mbar_wait(bar(b), (uint32_t)(phase & 1), abort_flag); };
    for (int seg = 0; walk.next(a, &g); ++seg) {
      const bool halves = two_halves(g);
      const int par = seg & 1;
      softmax_sync();                                     // both slots have left the segment before
      if (tid == 0) {
        c.missing[par ^ 1] = 0;
        c.nonfinite[par ^ 1][0] = c.nonfinite[par ^ 1][1] = 0;
      }
      const int32_t* table = a.g.tables + (size_t)g.b * a.g.max_pages;
      {
        const int end = min((g.tile0 + g.n) * KT, g.s.total);
        for (int i = g.tile0 * KT / a.g.page + tid; i * a.g.page < end; i += N_SOFTMAX)
          if (page_at(table, a.g.max_pages, a.g.n_pages, i) < 0) c.missing[par] = 1;
      }
      // ---- the slot's queries into shared memory: 128 rows, 16-byte pieces swizzled by row
      const int q0 = g.group * ITEM_ROWS + (halves ? wg * QR : 0);
      {
        constexpr int PIECES = HD / 8, ROWS_AT_ONCE = 128 / PIECES;
        const int piece = (tid & 127) % PIECES, r0 = (tid & 127) / PIECES;
        const char* q = reinterpret_cast<const char*>(a.q);
        uint4 v[QR / ROWS_AT_ONCE];
#pragma unroll
        for (int j = 0; j < QR / ROWS_AT_ONCE; ++j) {
          const int qi = q0 + r0 + j * ROWS_AT_ONCE;
          v[j] = make_uint4(0, 0, 0, 0);
          if (qi < g.s.nq) {
            const int r = qi / a.G;
            v[j] = *reinterpret_cast<const uint4*>(
                q + (((size_t)g.b * a.rows + r) * a.ld_q + (size_t)(g.head * a.G + qi - r * a.G) * HD + piece * 8) * 2);
            v[j].x ^= k.q_flip; v[j].y ^= k.q_flip; v[j].z ^= k.q_flip; v[j].w ^= k.q_flip;
          }
        }
        uint8_t* dst = smem + Z::Q_OFF + wg * Z::TILE + (piece >> 3) * BLOCK;
#pragma unroll
        for (int j = 0; j < QR / ROWS_AT_ONCE; ++j) {
          const int r = r0 + j * ROWS_AT_ONCE;
          *reinterpret_cast<uint4*>(dst + r * 128 + (((piece & 7) ^ (r & 7)) << 4)) = v[j];
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(bar(c.q_full));
      softmax_sync();
      const bool missing = *(volatile int*)&c.missing[par] != 0;

      const int qi = q0 + row;
      const bool valid = qi < g.s.nq, live = q0 + (row & ~31) < g.s.nq;   // live: some row of the warp exists
      const int r = valid ? qi / a.G : 0;
      uint64_t lo = 0, hi = 0;
      if (valid) paged_row_mask(a.mask, (size_t)g.b * a.rows + r, a.mask_words, g.s.rows, &lo, &hi);
      float m = -INFINITY, l = 0.f;                       // reference maximum (scores times scale_log2), sum
      const int steps = halves ? g.n : (g.n - wg + 1) >> 1;
      for (int i = 0; i < steps; ++i, ++n_s) {
        const int t = halves ? i : 2 * i + wg, key0 = (g.tile0 + t) * KT;
        const bool partly = key0 + KT > g.s.prefix;       // the tile reaches the tree
        wait(c.s_full[wg], n_s);
        tc_fence_after();
        if (partly && (!halves || wg == 0)) {
          // values behind the last slot, and infinities and NaN of tree slots, become zeros; one thread per key
          const int iv = 2 * (tiles_before + t) + 1, st = iv % Z::STAGES;
          wait(c.kv_full[st], iv / Z::STAGES);
          const int key = key0 + row, n16 = min(KT, (g.s.total - key0 + 15) & ~15);
          if (ok && row < n16 && key >= g.s.prefix) {
            uint8_t* v = smem + Z::KV_OFF + st * Z::TILE + row * 128;
            bool found = false;
#pragma unroll
            for (int j = 0; j < HD / 8; ++j) {
              uint4* p = reinterpret_cast<uint4*>(v + (j >> 3) * BLOCK + (((j & 7) ^ (row & 7)) << 4));
              if (key >= g.s.total) {
                *p = make_uint4(0, 0, 0, 0);
              } else {
                uint4 x = *p;
                if (nonfinite2(x.x) || nonfinite2(x.y) || nonfinite2(x.z) || nonfinite2(x.w)) {
                  found = true;
                  *p = make_uint4(finite2(x.x), finite2(x.y), finite2(x.z), finite2(x.w));
                }
              }
            }
            const int j = key - g.s.prefix;
            if (found) atomicOr(&c.nonfinite[par][j >> 6], 1ull << (j & 63));
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (live) {
          uint32_t s[KT];
#pragma unroll
          for (int j = 0; j < KT; j += 32) tmem_ld32(t_s + j, s + j);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < KT; j += 32) tie32(s + j);
          if (partly || missing) {
#pragma unroll
            for (int j = 0; j < KT; j += 32) {
              uint32_t vis = paged_visible32(key0 + j, g.s.prefix, lo, hi);
              if (missing) {
#pragma unroll 1
                for (int x = 0; x < 32; x += 16)          // a page holds 16 slots or a multiple
                  if (page_at(table, a.g.max_pages, a.g.n_pages, (key0 + j + x) / a.g.page) < 0) vis &= ~(0xffffu << x);
              }
#pragma unroll
              for (int x = 0; x < 32; ++x)
                if (!((vis >> x) & 1u)) s[j + x] = 0xff800000u;
            }
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < KT; ++j) m4[j & 3] = fmaxf(m4[j & 3], __uint_as_float(s[j]));
          const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * k.scale_log2;
          if (i == 0) {
            m = mx;
          } else if (__any_sync(0xffffffffu, mx > m + RESCALE_LOG2)) {
            // (the scores' completion was committed behind that of the slot's last second product)
            const float now = mx > m + RESCALE_LOG2 ? mx : m;
            const float f = now == m ? 1.f : (m == -INFINITY ? 0.f : ex2(m - now));
            m = now;
            l *= f;
#pragma unroll 1
            for (int j = 0; j < HD; j += 32) {
              uint32_t o[32];
              tmem_ld32(t_o + j, o);
              tmem_wait_ld();
              tie32(o);
#pragma unroll
              for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
              tmem_st32(t_o + j, o);
            }
          }
          const float off = m == -INFINITY ? 0.f : m;     // nothing seen so far: 2^(-inf) = 0
          float l4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < KT; j += 32) {
            uint32_t p[16];
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
              const float p0 = ex2(fmaf(__uint_as_float(s[j + x]), k.scale_log2, -off));
              const float p1 = ex2(fmaf(__uint_as_float(s[j + x + 1]), k.scale_log2, -off));
              l4[x & 3] += p0;
              l4[(x & 3) + 1] += p1;
              p[x >> 1] = pack_bf16(p0, p1);
            }
            tmem_st16(t_s + (j >> 1), p);
          }
          l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
          tmem_wait_st();
        }
        tc_fence_before();
        mbar_arrive(bar(c.p_full[wg]));
      }

      // ---- the segment's output: final where it is the whole item, else partials
      const int other = halves ? g.n : (g.n - (wg ^ 1) + 1) >> 1;
      n_other += other;
      if (steps > 0) wait(c.pv_done[wg], n_s - 1);
      float c0 = 1.f, c1 = 0.f;                           // weights of slot 0's and slot 1's outputs (same rows)
      if (!halves) {
        c.ml[wg][row] = make_float2(m, l);
        if (other > 0) wait(c.pv_done[wg ^ 1], n_other - 1);
        softmax_sync();
        const float2 x0 = c.ml[0][row], x1 = c.ml[1][row];
        m = fmaxf(x0.x, x1.x);
        // a slot that has seen nothing has sum 0 and is left out; one whose scores were all NaN has not
        c0 = x0.x == -INFINITY ? (x0.y == 0.f ? 0.f : 1.f) : ex2(x0.x - m);
        c1 = x1.x == -INFINITY ? (x1.y == 0.f ? 0.f : 1.f) : ex2(x1.x - m);
        l = x0.y * c0 + x1.y * c1;
      }
      tc_fence_after();
      if (live) {
        const bool whole = g.tile0 == 0 && g.n == g.s.tiles;
        const int rr = halves ? wg * QR + row : row;      // row inside the item
        const float inv = l == 0.f ? 0.f : 1.f / l;       // a row that sees nothing: zeros
        uint64_t nf_lo = c.nonfinite[par][0] & lo, nf_hi = c.nonfinite[par][1] & hi;
        float* part = nullptr;
        if (!whole) {
          const bool first = g.tile0 > 0 || range_begin(blockIdx.x, c.total, c.grid) == walk.u - g.n;
          part = partial_of(k, HD, blockIdx.x, first ? 0 : 1);
          if (valid && (halves || wg == 0))
            __stcg(reinterpret_cast<float2*>(part + (size_t)k.row_cap * HD) + rr, make_float2(m, l));
        }
        bf16* const out = reinterpret_cast<bf16*>(a.out) +
                          (((size_t)g.b * a.rows + r) * a.Hq + g.head * a.G + (qi - r * a.G)) * HD;
        const int col0 = halves ? 0 : wg * (HD / 2), cols = halves ? HD : HD / 2;
#pragma unroll 1
        for (int j = col0; j < col0 + cols; j += 32) {
          uint32_t o[32];
          if (halves) {
            tmem_ld32(t_o + j, o);
            tmem_wait_ld();
            tie32(o);
          } else {
            uint32_t o1[32];
            tmem_ld32(t_lane + 2 * KT + j, o);
            tmem_ld32(t_lane + 2 * KT + HD + j, o1);
            tmem_wait_ld();
            tie32(o);
            tie32(o1);
#pragma unroll
            for (int x = 0; x < 32; ++x) {                // (a slot left out: its accumulator may never have been written)
              const float y0 = c0 == 0.f ? 0.f : __uint_as_float(o[x]) * c0;
              const float y1 = c1 == 0.f ? 0.f : __uint_as_float(o1[x]) * c1;
              o[x] = __float_as_uint(y0 + y1);
            }
          }
          if (nf_lo | nf_hi) {
            // tree slots with infinities or NaN that this row sees: they were zeros in the product
#pragma unroll 1
            for (int w = 0; w < 2; ++w) {
              for (uint64_t bits = w ? nf_hi : nf_lo; bits; bits &= bits - 1) {
                const int slot = g.s.prefix + w * 64 + __ffsll((long long)bits) - 1;
                const int p = page_at(table, a.g.max_pages, a.g.n_pages, slot / a.g.page);
                if (p < 0) continue;
                const bf16* v = k.layer + page_offset(a.g, 0, p, 1, g.head) + (size_t)(slot % a.g.page) * HD + j;
#pragma unroll
                for (int x = 0; x < 32; ++x) {
                  const float y = to_f(v[x]);
                  if (!(fabsf(y) < INFINITY)) o[x] = __float_as_uint(__uint_as_float(o[x]) + y);
                }
              }
            }
          }
          if (valid) {
            if (whole) {
#pragma unroll
              for (int x = 0; x < 32; x += 8) {
                uint32_t w[4];
#pragma unroll
                for (int y = 0; y < 4; ++y)
                  w[y] = pack_bf16(__uint_as_float(o[x + 2 * y]) * inv, __uint_as_float(o[x + 2 * y + 1]) * inv);
                *reinterpret_cast<uint4*>(out + j + x) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            } else {
#pragma unroll
              for (int x = 0; x < 32; x += 4)
                __stcg(reinterpret_cast<uint4*>(part) + (size_t)((j + x) >> 2) * k.row_cap + rr,
                       make_uint4(o[x], o[x + 1], o[x + 2], o[x + 3]));
            }
          }
        }
      }
      tc_fence_before();
      mbar_arrive(bar(c.o_free));                         // the accumulators may take the next segment
      tiles_before += g.n;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == WARP_MMA) tmem_dealloc(tm, TMEM_COLS);
  if (threadIdx.x == 0 && *abort_flag) raise_status(a.status, POSS_E_TIMEOUT);
}

// ---------------------------------------------------------------------------------------------------- merge
// A block: 32 query rows of one item, eight threads per row.  The item's segments lie in consecutive CTAs, in key order.
template <int HD>
__global__ void __launch_bounds__(256) k_paged_attn_tc_merge(const TcArgs k, int ctas, int max_groups) {
  constexpr int NV = HD / 32;                             // float4 per thread
  __shared__ long long s_total, s_before;
  pdl_enter(POSS_K_PAGED_ATTN_COMBINE);
  const PagedAttnArgs& a = k.a;
  const int b = blockIdx.z, head = blockIdx.y / max_groups, group = blockIdx.y - head * max_groups;
  const SeqWork s = seq_work(a, b);
  if (group >= s.groups || group * ITEM_ROWS + (int)blockIdx.x * 32 >= s.nq) return;
  if (threadIdx.x < 32) {
    long long total, before;
    count_units(a, b, &total, &before);
    if (threadIdx.x == 0) { s_total = total; s_before = before; }
  }
  __syncthreads();
  const int grid = unit_grid(s_total, ctas);
  const long long u0 = s_before + ((long long)head * s.groups + group) * s.tiles;
  const int first = cta_of_unit(u0, s_total, grid), last = cta_of_unit(u0 + s.tiles - 1, s_total, grid);
  if (first == last) return;                              // written by its CTA
  const int rr = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, qi = group * ITEM_ROWS + rr;
  if (qi >= s.nq) return;
  // the first CTA's segment is its last one unless its range starts with the item; every later one's is its first
  auto part_of = [&](int cta) {
    return partial_of(k, HD, cta, cta == first && range_begin(first, s_total, grid) < u0 ? 1 : 0);
  };
  auto ml_of = [&](int cta) {
    return __ldcg(reinterpret_cast<const float2*>(part_of(cta) + (size_t)k.row_cap * HD) + rr);
  };
  float m = -INFINITY;
  for (int i = first; i <= last; ++i) m = fmaxf(m, ml_of(i).x);
  float l = 0.f;
  float4 o[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) o[v] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int i = first; i <= last; ++i) {
    const float2 x = ml_of(i);
    const float4* p = reinterpret_cast<const float4*>(part_of(i));
    float4 y[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) y[v] = __ldcg(p + (size_t)(slice * NV + v) * k.row_cap + rr);
    if (x.x == -INFINITY && x.y == 0.f) continue;         // has seen nothing
    const float c = x.x == -INFINITY ? 1.f : ex2(x.x - m);
    l = fmaf(x.y, c, l);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      o[v].x = fmaf(y[v].x, c, o[v].x); o[v].y = fmaf(y[v].y, c, o[v].y);
      o[v].z = fmaf(y[v].z, c, o[v].z); o[v].w = fmaf(y[v].w, c, o[v].w);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int r = qi / a.G;
  bf16* out = reinterpret_cast<bf16*>(a.out) +
              (((size_t)b * a.rows + r) * a.Hq + head * a.G + (qi - r * a.G)) * HD + slice * (HD / 8);
#pragma unroll
  for (int v = 0; v < NV; ++v)
    *reinterpret_cast<uint2*>(out + 4 * v) =
        make_uint2(pack_bf16(o[v].x * inv, o[v].y * inv), pack_bf16(o[v].z * inv, o[v].w * inv));
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

std::atomic<int> g_lost_loads{0};

int row_cap_of(int rows, int G) {
  const int nq = rows * G;
  return nq >= ITEM_ROWS ? ITEM_ROWS : (nq + 31) / 32 * 32;
}

template <int HD>
void launch(Launcher& L, const TcArgs& k0, const CUtensorMap& map, int max_pages) {
  using Z = Shape<HD>;
  TcArgs k = k0;
  const PagedAttnArgs& a = k.a;
  const size_t smem = Z::CTL_OFF + 3072;
  k.smem_bytes = (uint32_t)smem;
  static PerDeviceFlags attr_done;
  bool* attr = attr_done.current();
  if (!attr || !*attr) {
    if (cudaFuncSetAttribute(k_paged_attn_tc<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
      L.err = POSS_E_CUDA;
      return;
    }
    if (attr) *attr = true;
  }
  // one CTA per SM, as many as the fullest tables can give a unit
  const long long tiles = ((long long)max_pages * a.g.page + KT - 1) / KT;
  const int groups = (a.rows * a.G + ITEM_ROWS - 1) / ITEM_ROWS;
  const long long units = (long long)a.batch * a.g.Hkv * groups * tiles;
  const int sms = current_sm_count();
  const int ctas = units < sms ? (int)units : sms;
  launch_pdl(L, k_paged_attn_tc<HD>, dim3(ctas), dim3(N_THREADS), smem, map, k);
  if (tiles > 1 && L.err == POSS_OK)                      // (an item of one tile is never cut)
    launch_pdl(L, k_paged_attn_tc_merge<HD>, dim3(k.row_cap / 32, a.g.Hkv * groups, a.batch), dim3(256), 0, k, ctas,
               groups);
}

}  // namespace

bool paged_attn_tc_supported(const poss_page_pool& p, float scale) {
  if (p.dtype != POSS_BF16 || (p.head_dim != 64 && p.head_dim != 128)) return false;
  if (scale == 0.f) return false;                         // -inf * 0: the SIMT kernel masks after scaling
  const int s = p.page_slots;
  return s == 16 || s == 32 || s == 64 || s == 128 || s == 256;
}

size_t paged_attn_tc_workspace(const poss_page_pool& p, int batch, int rows, int Hq, int max_pages) {
  // two partials per CTA (its first and its last segment); the grid is at most the SM count
  (void)batch; (void)max_pages;
  return (size_t)current_sm_count() * 2 * row_cap_of(rows, Hq / p.n_kv_heads) * (p.head_dim + 2) * 4;
}

void launch_paged_attn_tc(Launcher& L, const PagedAttnArgs& a, const void* pool, const poss_page_pool& p) {
  EncodeTiledFn encode = encode_fn();
  if (!encode) { L.err = POSS_E_CUDA; return; }
  TcArgs k;
  memset(&k, 0, sizeof(k));
  k.a = a;
  k.layer = reinterpret_cast<const bf16*>(pool) + page_offset(a.g, a.layer, 0, 0, 0);
  k.scale_log2 = fabsf(a.scale) * 1.4426950408889634f;
  k.q_flip = a.scale < 0.f ? 0x80008000u : 0u;
  k.row_cap = row_cap_of(a.rows, a.G);
  k.rows_total = a.g.n_pages * 2 * a.g.Hkv * a.g.page;
  int lost = g_lost_loads.load();
  while (lost > 0 && !g_lost_loads.compare_exchange_weak(lost, lost - 1)) {}
  k.inject_lost_load = lost > 0;
  // The layer as a matrix of slots: rows (page, keys / values, head, slot), head_dim columns.  A box is a page's slots of
  // one head (at most one tile of keys) times 64 columns.
  CUtensorMap map;
  cuuint64_t gdim[2] = {(cuuint64_t)a.g.d, (cuuint64_t)k.rows_total};
  cuuint64_t gstr[1] = {(cuuint64_t)a.g.d * 2};
  cuuint32_t box[2] = {64, (cuuint32_t)(a.g.page < KT ? a.g.page : KT)};
  cuuint32_t estr[2] = {1, 1};
  if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<bf16*>(k.layer), gdim, gstr, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
    L.err = POSS_E_CUDA;
    return;
  }
  if (a.g.d == 128) launch<128>(L, k, map, a.g.max_pages);
  else launch<64>(L, k, map, a.g.max_pages);
}

extern "C" int poss_debug_paged_lose_load(int launches) {
  if (launches < 0) return POSS_E_INVALID;
  g_lost_loads.store(launches);
  return POSS_OK;
}
