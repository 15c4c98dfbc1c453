// Tree-masked attention over pages on the 5th-generation tensor cores (bf16, head dimension 64 or 128).
//
// The G = Hq / Hkv query heads of a KV head and a sequence's tree rows form one matrix of query rows (row * G + head), cut
// into items of up to 256: (sequence, KV head, two slots of floor(128 / G) tree rows).  A unit of work is one item's product
// with 64 keys; the units of the whole batch, in order of sequence, head, item and key, are cut into one contiguous range per
// CTA, one CTA per SM, so that every SM streams the same number of key tiles however long the sequences are.  The part of an item that
// falls into one CTA is a segment: one pass over its keys with the running maximum and sum of a softmax.  A segment that is
// the whole item writes the output, any other leaves fp32 partials that a second kernel merges in key order.  Where items are
// short the ranges end at items instead (Plan).
//
// Inside a CTA two "slots" of 128 query rows share the key tiles:
//   * items with rows for both slots: each has its own, both use every tile (each key is read once);
//   * smaller items: both slots hold the same rows and take the even / the odd tiles; they are merged at the end.
// Warps 0-3 / 4-7 do the softmax of slot 0 / 1 (one thread per query row), warps 8 and 11 issue the copies of keys and of
// values, one lane each of warps 9 and 10 the products of slot 0 and 1:
//   * copies: TMA, one box per page and 64 columns, through a ring of stages each for keys and values.  A page that is missing
//     or behind the last slot is read from behind the pool: zeros.  The next segment's queries come the same way while the
//     last one ends;
//   * S = Q K^T (fp32, TMEM); the softmax thread masks its row of S in place where the tile reaches the tree, takes its
//     maximum, writes P = 2^(s - m) over S in TMEM as the sum of two bf16; O += P V with P as the TMEM operand, two products
//     per 16 keys;
//   * the reference maximum m moves only when a row's maximum has grown by more than 2^8 (P stays below 2^8, which two bf16
//     and the fp32 sums hold as well as 1): then the thread scales its row of O in TMEM.  Otherwise O is never touched;
//   * a slot's scores have two buffers: while its softmax works on one tile, the products of the tile before and of the tile
//     behind run.
//
// Unseen slots.  A score is replaced by -inf, so what a key holds is of no account.  A value is multiplied by an exact zero,
// which is not enough for infinities and NaN: in tiles that reach behind the committed slots the values behind the last slot
// are set to zero, and infinities and NaN of tree slots too, in shared memory; the rows that do see such a slot get them
// added at the end.
//
// A probability is cut to bf16 and what that leaves over rounded to bf16, 2^-15 of it in all; the kernel of the contiguous caches
// splits it as well.  With one bf16 (2^-8) the output's error is 1.4 times that of its own rounding and up to 3.3 times the bound
// that holds there; 16 trees of 1 to 61 rows over up to 8191 slots would take 126 us for 148 in a graph.  Sums, maxima and
// accumulators are fp32.
//
// What bounds it.  One token per sequence: the read of keys and values, once (16 sequences of up to 16384 slots, 834 MB: 146 us
// with pages of 64, 5.7 TB/s; 169 us with pages of 16, whose boxes are 2 KB; in a loop the power limit lowers the clock).  61 rows
// of 4 heads over the same slots: 298 us, 684 TFLOP/s of scores and one output product; a step of 64 keys and two slots takes 1.7
// us, of which the products alone need some 1800 cycles (M128 N64 K16 50 cycles, M128 N128 K16 64, two of these per 16 keys) and the
// exponentials 1024.  The rest is latency between the roles: barriers, commits and operand registers of a slot's product lane, loads,
// maxima and barriers of its softmax, and both slots come to run in step, so that neither fills the other's gaps.  With
// probabilities in one bf16, where the same took 246 us, these were measured and not better: 16 softmax warps of half a row each,
// 251 us; a lane for each kind of product in place of each slot, 257 us; three product lanes, 252 us; a late start of slot 1,
// 247 us.  Short sequences: 17 us for 1 row over 1024 slots, 6 us of it before the first scores (lengths, pages, the first copies),
// the rest two or three steps, partials and the merge's launch.
//
// Every CTA gets the same number of units, but a unit of an item with rows for both slots takes twice the work of one whose slots
// take the tiles in turn: with 16 trees of 1 to 61 rows the fullest CTA has 1.33 to 1.37 times the mean, with one of 81 rows 1.42.
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

constexpr int KT = 64;                  // keys per tile
constexpr int QR = 128;                 // query rows per slot
constexpr int N_SOFTMAX = 256;
constexpr int N_THREADS = N_SOFTMAX + 128;
constexpr int WARP_KEYS = 8, WARP_MMA = 9, WARP_VALUES = 11;   // WARP_MMA + slot issues the slot's products
constexpr int MAX_CTAS = 160;           // segments of one item that the merge can hold; a device's SMs otherwise
constexpr int GONE_RING = 32;           // tiles whose "a page is missing" is remembered: more than the copies run ahead
constexpr int BLOCK = QR * 128;         // bytes of 128 query rows x 64 bf16
constexpr int KV_BLOCK = KT * 128;      // bytes of a tile's 64 keys x 64 bf16
constexpr int MAX_STAGES = 8;
constexpr float RESCALE_LOG2 = 8.f;
constexpr uint32_t TMEM_COLS = 512;
constexpr int S_COLS = 2 * KT;          // a slot's scores: two buffers, in turn (P lies over its scores)
constexpr int P_COLS = KT / 2;          // a tile's probabilities as bf16; what they leave over lies behind them

template <int HD> struct Shape {
  static constexpr int CB = HD / 64;                      // 64-column blocks
  static constexpr int Q_TILE = CB * BLOCK, TILE = CB * KV_BLOCK;   // bytes of a slot's queries, of a tile's keys or values
  // Keys and values have a ring of stages each: a stage that both copy warps used in turn would let one of them, half a
  // turn ahead, take the other's phase for its own.  Values stay until the second product, keys until the first.
  static constexpr int NK = HD == 128 ? 4 : 8, NV = HD == 128 ? 6 : 8;
  static_assert(NK % 2 == 0 && NV % 2 == 0, "a slot that takes every other tile keeps to its own stages");
  static constexpr int Q_OFF = 0, K_OFF = 2 * Q_TILE, V_OFF = K_OFF + NK * TILE, CTL_OFF = V_OFF + NV * TILE;
};

struct TcArgs {
  PagedAttnArgs a;
  float scale_log2;                     // scale times log2 e, positive
  int slot_rows;                        // tree rows per slot: floor(128 / G); a slot's lines are (tree row, head)
  int row_cap;                          // query rows that a partial has room for
  int rows_total;                       // rows of the pool's layer: the first coordinate behind it
  int inject_lost_load;
  uint32_t smem_bytes;
  const bf16* layer;                    // the layer's first element
  // SCORES: few rows leave their scores for the slots' weights, -inf where they do not see a slot: [batch][Hkv][rows * G][scores_ld]
  float* scores;
  long long scores_ld;
  float* mass;                          // the layer's weights, see PagedMassArgs
  long long mass_slots;
  const float* row_weights;
  int merge_blocks;                     // blocks of the merge; those behind them add up weights
  struct PlanOut* plan;                 // what the merge needs to know, left by the first CTA
};

// ---- the units of a sequence
struct SeqWork {
  int prefix, rows, total, tiles, groups;       // groups: items per KV head
  uint32_t units;                       // (a batch's units fit 31 bits: checked on the host)
  bool bad;
};
__device__ __forceinline__ SeqWork seq_work(const TcArgs& k, int b) {
  const PagedAttnArgs& a = k.a;
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows,
                              (long long)a.g.max_pages * a.g.page);
  SeqWork s;
  s.bad = n.bad; s.prefix = n.prefix; s.rows = n.rows;
  s.total = n.prefix + n.rows;
  s.tiles = (s.total + KT - 1) / KT;
  s.groups = (n.rows + 2 * k.slot_rows - 1) / (2 * k.slot_rows);
  s.units = (uint32_t)s.groups * a.g.Hkv * s.tiles;       // no rows: no groups
  return s;
}
// Barriers are waited for by parity, so no role may be able to fall, or run, two phases behind another on one barrier:
//   s_full / p_full / pv_done [slot][step & 1]: S of step y + 2 is issued behind the second product of step y, which waits for
//     P of step y -- a softmax that has seen S of step y knows that the products of step y - 2 are complete;
//   kv_full / kv_empty [keys, values][stage]: filled in order by one warp, but copies land in any order.  A slot that uses every
//     tile sees every phase; one that uses every other tile must meet the same stages again and no others, so that it has seen
//     a stage's last phase itself: the rings have even lengths.  (At a segment's start all earlier phases are over: q_full
//     follows q_empty, which follows all of the last segment's first products, and o_free all of its second ones.)
//   q_full, q_empty, o_free: one phase per segment.  A slot without steps in a segment waits for no o_free there, but a slot
//     with steps gives q_empty up only behind its wait for the o_free before: whoever has seen q_full of segment s + 1 knows
//     that o_free of segment s - 1 is complete.
// ml has no second copy: a slot writes its own for a segment only when the other one has read it for the segment before.  A slot with
// steps has waited for second products, which follow that segment's o_free; one without steps waits for o_free itself.
//   clean, in turn: one phase per tile that slot 0 puts right for both slots.  A segment has at most three; slot 0 can be past those
//     of one segment and two of the next (its second products there wait for o_free of this one) while slot 1 waits for this one's
//     first, five ahead: with six barriers none is a phase ahead of a wait.
constexpr int N_CLEAN = 6;
struct Ctl {
  uint64_t clean[N_CLEAN];
  uint64_t kv_full[2][MAX_STAGES], kv_empty[2][MAX_STAGES], q_full, q_empty, s_full[2][2], p_full[2][2], pv_done[2][2], o_free, drain[2];
  uint32_t tmem;
  int abort;
  uint8_t gone[GONE_RING];              // by tile: a page of it is missing
  unsigned long long nonfinite[2][N_SOFTMAX / 32][2];   // by parity and warp: tree slots whose values hold infinities or NaN
  uint32_t total, offset0, skipped;     // units of the batch; the CTA's first unit inside its first sequence; units of its
                                        // range that another CTA takes
  int seq0, grid, whole;                // that sequence; see Plan
  SeqWork work0;                        // its work
  float2 ml[2][QR];                     // a slot's maximum and sum, for the merge of two slots with the same rows
};
constexpr int CTL_BYTES = 3 * 1024;
static_assert(sizeof(Ctl) <= CTL_BYTES, "the control block lies behind the tiles");

// CTAs that share `total` units (MIN_UNITS each at least), and the cut: the first total % grid of them take one unit more.
// Two units and not one: partials and their merge cost more than a second step where few rows meet more keys than the CTAs
// can take one unit each of (1 row over 1024 slots: 17.4 against 18.2 us; over 400 it would be 13.3 for 15.2, the others are alike).
constexpr uint32_t MIN_UNITS = 2;
__device__ __forceinline__ int unit_grid(uint32_t total, uint32_t ctas) {
  const uint32_t n = (total + MIN_UNITS - 1) / MIN_UNITS;
  return (int)(n < ctas ? n : ctas);
}
struct Cut {
  uint32_t each, more;
  __device__ __forceinline__ Cut(uint32_t total, uint32_t grid) { each = total / grid; more = total - each * grid; }
  __device__ __forceinline__ uint32_t begin(uint32_t c) const { return c * each + (c < more ? c : more); }
  __device__ __forceinline__ int cta_of(uint32_t u) const {
    const uint32_t longer = more * (each + 1);            // units of the CTAs with one more
    return u < longer ? u / (each + 1) : more + (u - longer) / each;
  }
};
// One warp: the units of all sequences, and how they are cut.  For up to 32 sequences every lane keeps its own one's work in *mine.
struct Plan {
  uint32_t total;
  int grid;                             // CTAs that share them
  bool whole;                           // items are not cut: a CTA takes those that begin in its range
};
struct PlanOut {
  uint32_t total;
  int grid, whole, unused;
  uint32_t before[POSS_MAX_PAGED_BATCH];   // units of the sequences before
};
__device__ __forceinline__ uint32_t inclusive_scan(uint32_t x) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if ((int)(threadIdx.x & 31) >= o) x += y;
  }
  return x;
}
// Cutting costs the partials' way through L2 and the merge, the more the more rows there are: units that whole items may make the
// longest range longer.  Measured cut / whole: 61 rows of 4 heads over 100 slots (2 and 3 units) 19.5 / 15.6 us, 7 ragged trees of 25
// rows over up to 300 slots (2 and 6) 13.5 / 11.2, 16 x 61 rows over up to 500 (8 and 9) 41.8 / 39.3; 4 x 61 rows over up to 1000 (4 and 17)
// 25.9 / 34.1, 1 row over 1024 17.2 / 22.7, over 400 (2 and 6) 14.9 / 14.2.
__device__ __forceinline__ uint32_t whole_extra(int row_cap) { return 2 + row_cap / 32; }
__device__ __forceinline__ Plan make_plan(const TcArgs& k, uint32_t ctas, SeqWork* mine) {
  const int lane = threadIdx.x & 31;
  uint32_t t = 0, longest = 0, shortest = 0xffffffffu;
  mine->units = 0;
  for (int x = lane; x < k.a.batch; x += 32) {
    const SeqWork s = seq_work(k, x);
    if (x < 32) *mine = s;
    t += s.units;
    if (s.units) {
      longest = max(longest, (uint32_t)s.tiles);
      shortest = min(shortest, (uint32_t)s.tiles);
    }
  }
  Plan p;
  p.total = __reduce_add_sync(0xffffffffu, t);
  longest = __reduce_max_sync(0xffffffffu, longest);
  shortest = __reduce_min_sync(0xffffffffu, shortest);
  p.grid = unit_grid(p.total, ctas);
  p.whole = false;
  if (p.total) {
    // the longest range if items stay whole: a share and the rest of an item; known better where all are equal
    const uint32_t share = (p.total + p.grid - 1) / p.grid;
    const uint32_t worst = longest == shortest ? (share + longest - 1) / longest * longest : share + longest - 1;
    p.whole = worst <= share + whole_extra(k.row_cap);
  }
  return p;
}

struct Segment {
  int b, head, group, tile0, n;         // n tiles from tile0 on
  SeqWork s;
};
// A CTA's segments in order; every role walks them by itself.
struct Walk {
  uint32_t u, u_end, offset;
  int b, whole;
  __device__ __forceinline__ void start(const Ctl& c, Segment* g) {
    u = u_end = 0;
    if ((int)blockIdx.x < c.grid) {
      const Cut cut(c.total, c.grid);
      u = cut.begin(blockIdx.x) + c.skipped;
      u_end = cut.begin(blockIdx.x + 1);
    }
    b = c.seq0;
    offset = c.offset0;
    whole = c.whole;
    g->s = c.work0;
  }
  __device__ __forceinline__ bool next(const TcArgs& k, Segment* g) {
    if (u >= u_end) return false;                           // (g still holds its sequence's work)
    while (offset >= g->s.units) {
      offset -= g->s.units;
      if (++b >= k.a.batch) return false;                   // (not reached: the range lies inside the batch's units)
      g->s = seq_work(k, b);
    }
    g->b = b;
    const uint32_t item = offset / (uint32_t)g->s.tiles;
    g->tile0 = (int)(offset - item * g->s.tiles);
    g->head = (int)item;
    g->group = 0;
    if (g->s.groups > 1) {
      g->head = (int)(item / (uint32_t)g->s.groups);
      g->group = (int)item - g->head * g->s.groups;
    }
    g->n = g->s.tiles - g->tile0;
    if (!whole) g->n = min(g->n, (int)(u_end - u));
    u += g->n;
    offset += g->n;
    return true;
  }
};
// two slots of different rows (true) or of the same rows and alternating tiles
__device__ __forceinline__ bool two_halves(const TcArgs& k, const Segment& g) {
  return g.s.rows - g.group * 2 * k.slot_rows > k.slot_rows;
}

// ---- PTX
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
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t pack64(uint32_t lo, uint32_t hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
  return d;
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
// 1024 bytes apart, the next 64 columns one KV_BLOCK further
__device__ __forceinline__ uint64_t smem_desc_values(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(KV_BLOCK >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= 1ull << 46;
  d |= 2ull << 61;
  return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float max32(const uint32_t* s, float m) {
  float a = __uint_as_float(s[0]), b = __uint_as_float(s[1]);
#pragma unroll
  for (int x = 2; x < 30; x += 4) {
    a = max3(a, __uint_as_float(s[x]), __uint_as_float(s[x + 1]));
    b = max3(b, __uint_as_float(s[x + 2]), __uint_as_float(s[x + 3]));
  }
  a = max3(a, __uint_as_float(s[30]), __uint_as_float(s[31]));
  return max3(a, b, m);
}
// p = 2^(s * scale + off) for 32 scores as bf16, and what that leaves over in `rest`; their sum goes to l0, l1.  (A part of the 2^x as a polynomial on the
// multiply-add pipe was measured too, with one bf16 each: it loses, 261 against 249 us for 16 trees of 61 rows over 16383 slots.)
__device__ __forceinline__ void exp32(const uint32_t* s, float2 scale, float2 off, uint32_t* p, uint32_t* rest, float2& l0, float2& l1) {
#pragma unroll
  for (int x = 0; x < 32; x += 2) {
    const float2 a = fma2(make_float2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), scale, off);
    const float2 e = make_float2(ex2(a.x), ex2(a.y));
    if (x & 2) l1 = add2(l1, e);
    else l0 = add2(l0, e);
    // cut, not rounded, and a little short, so that the rest of what is above 0 is too: an infinite value that is seen would
    // otherwise meet a rest of 0 or below and come out as NaN
    const float2 t = fma2(e, make_float2(1.f - 0x1p-20f, 1.f - 0x1p-20f), make_float2(0.f, 0.f));
    const uint32_t tx = __float_as_uint(t.x), ty = __float_as_uint(t.y);
    p[x >> 1] = __byte_perm(tx, ty, 0x7632);
    const float2 d = add2(e, make_float2(__uint_as_float((tx & 0xffff0000u) ^ 0x80000000u), __uint_as_float((ty & 0xffff0000u) ^ 0x80000000u)));
    rest[x >> 1] = pack_bf16(d.x, d.y);                 // (d is exact)
  }
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
// Every role walks the CTA's segments by itself, in one loop that they share: code that a launch runs once costs its
// instruction fetches (about 25 cycles per instruction that no warp of the SM has run yet), so there is one copy of it.
template <int HD, bool SCORES>
__global__ void __launch_bounds__(N_THREADS, 1) k_paged_attn_tc(const __grid_constant__ CUtensorMap map,
                                                                 const __grid_constant__ CUtensorMap map_q,
                                                                 const TcArgs k) {
  using Z = Shape<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Ctl& c = *reinterpret_cast<Ctl*>(smem + Z::CTL_OFF);
  const uint32_t base = smem_u32(smem);
  const PagedAttnArgs& a = k.a;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  auto bar = [&](uint64_t& x) { return smem_u32(&x); };

  if (warp == WARP_MMA) {
    if (lane == 0) {
      // (tiles start on 1024 bytes and fit: checked on the host, and here)
      c.abort = (base & 1023u) || Z::CTL_OFF + sizeof(Ctl) > k.smem_bytes ? 1 : 0;
      for (int i = 0; i < 2 * MAX_STAGES; ++i) {
        mbar_init(bar(c.kv_full[i / MAX_STAGES][i % MAX_STAGES]), 1);
        mbar_init(bar(c.kv_empty[i / MAX_STAGES][i % MAX_STAGES]), 2);
      }
      mbar_init(bar(c.q_full), 1);
      mbar_init(bar(c.q_empty), 2);
      mbar_init(bar(c.o_free), N_SOFTMAX);
      for (int i = 0; i < N_CLEAN; ++i) mbar_init(bar(c.clean[i]), QR);
      for (int i = 0; i < 2; ++i) {
        mbar_init(bar(c.drain[i]), 1);
        for (int j = 0; j < 2; ++j) {
          mbar_init(bar(c.s_full[i][j]), 1);
          mbar_init(bar(c.p_full[i][j]), QR);
          mbar_init(bar(c.pv_done[i][j]), 1);
        }
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
  pdl_sync(POSS_K_PAGED_ATTN);

  if (warp == 0) {
    // the batch's units, and the sequence that the CTA's first one lies in
    SeqWork own;
    const Plan plan = make_plan(k, gridDim.x, &own);
    if ((int)blockIdx.x < plan.grid) {
      uint32_t at = Cut(plan.total, plan.grid).begin(blockIdx.x);
      for (int b0 = 0; b0 < a.batch; b0 += 32) {
        if (b0 > 0) {
          own.units = 0;
          if (b0 + lane < a.batch) own = seq_work(k, b0 + lane);
        }
        const uint32_t x = inclusive_scan(own.units);
        const unsigned here = __ballot_sync(0xffffffffu, at < x);
        if (here) {
          const int first = __ffs(here) - 1;
          if (lane == first) {
            const uint32_t off = at - (x - own.units), into = plan.whole ? off % (uint32_t)own.tiles : 0u;
            c.seq0 = b0 + first;
            c.work0 = own;
            c.skipped = into ? (uint32_t)own.tiles - into : 0u;   // the item that began before
            c.offset0 = off + c.skipped;
          }
          break;
        }
        at -= __shfl_sync(0xffffffffu, x, 31);
      }
    }
    if (lane == 0) {
      c.total = plan.total;
      c.grid = plan.grid;
      c.whole = plan.whole;
      if (blockIdx.x == 0) { k.plan->total = plan.total; k.plan->grid = plan.grid; k.plan->whole = plan.whole; }
    }
  }
  __syncthreads();

  Segment g;
  Walk walk;
  walk.start(c, &g);
  const uint32_t u_first = walk.u;
  // what a role carries from segment to segment
  bool ok = __all_sync(0xffffffffu, *abort_flag == 0);
  int tiles_before = 0;                                   // tiles of the segments before
  int n_own = 0, n_partly = 0;                            // softmax and products: steps of the slot; copies: tiles
  int n_queries = 0;                                      // copies: segments whose queries are on their way or here
  // copies: stage and phase of the next keys or values
  uint32_t c_ph = 0, elected = 0;
  int c_st = 0;
  if (warp == WARP_MMA || warp == WARP_MMA + 1) elected = elect_one();
  constexpr uint32_t ROW16 = 2;                           // 16 bf16 = 32 bytes, in 16-byte address units
  constexpr uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(KT >> 3) << 17) | ((uint32_t)(QR >> 4) << 24);
  constexpr uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(HD >> 3) << 17) |
                               ((uint32_t)(QR >> 4) << 24) | (1u << 16);       // the values are MN-major
  const uint64_t q_desc = smem_desc_sw128(base + Z::Q_OFF), k_desc = smem_desc_sw128(base + Z::K_OFF),
                 v_desc = smem_desc_values(base + Z::V_OFF);
  auto wait = [&](uint64_t& b, int phase) {
    if (ok) ok = mbar_wait(bar(b), (uint32_t)(phase & 1), abort_flag);
  };

  for (int seg = 0; walk.next(k, &g); ++seg) {
    const bool halves = two_halves(k, g);
    const int par = seg & 1;
    const int32_t* const table = a.g.tables + (size_t)g.b * a.g.max_pages;

    if (warp < N_SOFTMAX / 32) {
      // -------------------------------------------------------------- softmax, one thread per query row
      const int wg = warp >> 2, row = (warp & 3) * 32 + lane;
      const uint32_t t_lane = tm + ((uint32_t)((warp & 3) * 32) << 16);
      const uint32_t t_s = t_lane + wg * S_COLS, t_o = t_lane + 2 * S_COLS + wg * HD;
      // the thread's line of the slot: tree row and head
      const int r0 = (2 * g.group + (halves ? wg : 0)) * k.slot_rows, in_slot = row / a.G, head = row - in_slot * a.G;
      const bool valid = in_slot < k.slot_rows && r0 + in_slot < g.s.rows;
      const bool live = __any_sync(0xffffffffu, valid);   // some line of the warp exists
      const int r = valid ? r0 + in_slot : 0;
      uint64_t lo = 0, hi = 0;
      if (valid) paged_row_mask(a.mask, (size_t)g.b * a.rows + r, a.mask_words, g.s.rows, &lo, &hi);
      if (lane == 0) c.nonfinite[par][warp][0] = c.nonfinite[par][warp][1] = 0;
      __syncwarp();
      float m = -INFINITY, l = 0.f;                       // reference maximum (scores times scale_log2), sum
      const int steps = halves ? g.n : (g.n - wg + 1) >> 1;   // the slot's tiles: all, or every other one
      const float2 sc = make_float2(k.scale_log2, k.scale_log2);
#pragma unroll 1
      for (int i = 0; i < steps; ++i, ++n_own) {
        const int t = halves ? i : 2 * i + wg, key0 = (g.tile0 + t) * KT;
        const bool partly = key0 + KT > g.s.prefix;       // the tile reaches the tree
        if (partly && (!halves || wg == 0)) {
          // values behind the last slot, and infinities and NaN of tree slots, become zeros; two threads per key
          // (once the scores are there, the slot's last values but one have been used: the stage is in this tile's turn)
          const int st = (tiles_before + t) % Z::NV;
          wait(c.s_full[wg][n_own & 1], n_own >> 1);
          wait(c.kv_full[1][st], (tiles_before + t) / Z::NV);
          const int kr = row % KT, key = key0 + kr, n16 = min(KT, (g.s.total - key0 + 15) & ~15);
          if (ok && kr < n16 && key >= g.s.prefix) {
            constexpr int N = HD / 16;                    // pieces of 16 bytes per thread
            uint8_t* v = smem + Z::V_OFF + st * Z::TILE + kr * 128;
            auto piece = [&](int x) {
              const int i = (row / KT) * N + x;
              return reinterpret_cast<uint4*>(v + (i >> 3) * KV_BLOCK + (((i & 7) ^ (kr & 7)) << 4));
            };
            if (key >= g.s.total) {
#pragma unroll
              for (int x = 0; x < N; ++x) *piece(x) = make_uint4(0, 0, 0, 0);
            } else {
              uint4 x[N];
              bool found = false;
#pragma unroll
              for (int i = 0; i < N; ++i) x[i] = *piece(i);
#pragma unroll
              for (int i = 0; i < N; ++i) found |= nonfinite2(x[i].x) | nonfinite2(x[i].y) | nonfinite2(x[i].z) | nonfinite2(x[i].w);
              if (found) {
#pragma unroll 1
                for (int i = 0; i < N; ++i) {
                  const uint4 y = *piece(i);
                  *piece(i) = make_uint4(finite2(y.x), finite2(y.y), finite2(y.z), finite2(y.w));
                }
                const int j = key - g.s.prefix;
                atomicOr(&c.nonfinite[par][warp][j >> 6], 1ull << (j & 63));
              }
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (partly && halves) {
          // slot 1's product reads what slot 0's warps have put right
          uint64_t& b = c.clean[n_partly % N_CLEAN];
          if (wg == 0) mbar_arrive(bar(b));
          else wait(b, n_partly / N_CLEAN);
          ++n_partly;
        }
        const int buf = n_own & 1;
        wait(c.s_full[wg][buf], n_own >> 1);
        tc_fence_after();
        const bool missing = *(volatile uint8_t*)&c.gone[(tiles_before + t) % GONE_RING] != 0;   // (written before the keys' copies)
        if (live) {
          uint32_t sa[32], sb[32], p[32], rest[32];
          tmem_ld32(t_s + buf * KT, sa);
          tmem_ld32(t_s + buf * KT + 32, sb);
          tmem_wait_ld();
          tie32(sa);
          tie32(sb);
          if (partly || missing) {
            uint32_t va = paged_visible32(key0, g.s.prefix, lo, hi), vb = paged_visible32(key0 + 32, g.s.prefix, lo, hi);
            if (missing) {
#pragma unroll 1
              for (int x = 0; x < 32; x += 16) {        // a page holds 16 slots or a multiple
                if (page_at(table, a.g.max_pages, a.g.n_pages, (key0 + x) / a.g.page) < 0) va &= ~(0xffffu << x);
                if (page_at(table, a.g.max_pages, a.g.n_pages, (key0 + 32 + x) / a.g.page) < 0) vb &= ~(0xffffu << x);
              }
            }
#pragma unroll
            for (int x = 0; x < 32; ++x) {
              if (!((va >> x) & 1u)) sa[x] = 0xff800000u;
              if (!((vb >> x) & 1u)) sb[x] = 0xff800000u;
            }
          }
          if constexpr (SCORES) {                       // (an item of one slot: its line is the thread's row)
            if (valid) {
              uint4* const to = reinterpret_cast<uint4*>(k.scores + (((size_t)g.b * a.g.Hkv + g.head) * (a.rows * a.G) + row) * k.scores_ld + key0);
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                to[x] = make_uint4(sa[4 * x], sa[4 * x + 1], sa[4 * x + 2], sa[4 * x + 3]);
                to[8 + x] = make_uint4(sb[4 * x], sb[4 * x + 1], sb[4 * x + 2], sb[4 * x + 3]);
              }
            }
          }
          const float mx = max32(sb, max32(sa, -INFINITY)) * k.scale_log2;
          if (i == 0) {
            m = mx;
          } else if (__any_sync(0xffffffffu, mx > m + RESCALE_LOG2)) {
            wait(c.pv_done[wg][buf ^ 1], (n_own - 1) >> 1);   // O is at rest until this step's P is there
            tc_fence_after();
            const float now = mx > m + RESCALE_LOG2 ? mx : m;
            const float f = now == m ? 1.f : (m == -INFINITY ? 0.f : ex2(m - now));
            m = now;
            l *= f;
#pragma unroll 1
            for (int j = 0; j < HD; j += 16) {
              uint32_t o[16];
              tmem_ld16(t_o + j, reinterpret_cast<float*>(o));
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
              tmem_st16(t_o + j, o);
            }
          }
          const float off = m == -INFINITY ? 0.f : -m;  // nothing seen so far: 2^(-inf) = 0
          const float2 of = make_float2(off, off);
          float2 l0 = make_float2(0.f, 0.f), l1 = l0;
          exp32(sa, sc, of, p, rest, l0, l1);
          exp32(sb, sc, of, p + 16, rest + 16, l0, l1);
          tmem_st32(t_s + buf * KT, p);                 // (over the scores)
          tmem_st32(t_s + buf * KT + P_COLS, rest);
          l += (l0.x + l0.y) + (l1.x + l1.y);
          tmem_wait_st();
        }
        tc_fence_before();
        mbar_arrive(bar(c.p_full[wg][buf]));
      }
      // ---- the segment's output: final where it is the whole item, else partials
      if (steps > 0) wait(c.pv_done[wg][(n_own - 1) & 1], (n_own - 1) >> 1);
      float c0 = 1.f, c1 = 0.f;                           // weights of slot 0's and slot 1's outputs (same rows)
      if (!halves) {
        if (steps == 0 && seg > 0) wait(c.o_free, seg - 1);   // (slot 0's next outputs wait for it as well: no time is lost)
        c.ml[wg][row] = make_float2(m, l);
        tc_fence_before();
        softmax_sync();                                   // both slots' outputs are complete
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
        uint64_t nf_lo = 0, nf_hi = 0;
#pragma unroll
        for (int w = 0; w < N_SOFTMAX / 32; ++w) {
          nf_lo |= c.nonfinite[par][w][0];
          nf_hi |= c.nonfinite[par][w][1];
        }
        nf_lo &= lo;
        nf_hi &= hi;
        float* part = nullptr;
        if (!whole) {
          // the CTA's first segment, or its last
          part = partial_of(k, HD, blockIdx.x, g.tile0 > 0 || u_first == walk.u - g.n ? 0 : 1);
          if (valid && (halves || wg == 0))
            __stcg(reinterpret_cast<float2*>(part + (size_t)k.row_cap * HD) + rr, make_float2(m, l));
        } else if (a.ml && valid && (halves || wg == 0)) {
          a.ml[((size_t)g.b * a.rows + r) * a.Hq + g.head * a.G + head] = paged_ml(m, l);
        }
        bf16* const out = reinterpret_cast<bf16*>(a.out) +
                          (((size_t)g.b * a.rows + r) * a.Hq + g.head * a.G + head) * HD;
        const int col0 = halves ? 0 : wg * (HD / 2), cols = halves ? HD : HD / 2;
        // (16 columns at a time: the code is met for the first time here, and less of it comes sooner)
#pragma unroll 1
        for (int j = col0; j < col0 + cols; j += 16) {
          uint32_t o[16];
          if (halves) {
            tmem_ld16(t_o + j, reinterpret_cast<float*>(o));
          } else {
            uint32_t o1[16];
            tmem_ld16(t_lane + 2 * S_COLS + j, reinterpret_cast<float*>(o));
            tmem_ld16(t_lane + 2 * S_COLS + HD + j, reinterpret_cast<float*>(o1));
#pragma unroll
            for (int x = 0; x < 16; ++x) {                // (a slot left out: its accumulator may never have been written)
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
                for (int x = 0; x < 16; ++x) {
                  const float y = to_f(v[x]);
                  if (!(fabsf(y) < INFINITY)) o[x] = __float_as_uint(__uint_as_float(o[x]) + y);
                }
              }
            }
          }
          if (valid) {
            if (whole) {
#pragma unroll
              for (int x = 0; x < 16; x += 8) {
                uint32_t w[4];
#pragma unroll
                for (int y = 0; y < 4; ++y)
                  w[y] = pack_bf16(__uint_as_float(o[x + 2 * y]) * inv, __uint_as_float(o[x + 2 * y + 1]) * inv);
                *reinterpret_cast<uint4*>(out + j + x) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            } else {
              uint4* dst = reinterpret_cast<uint4*>(part) + (size_t)(j >> 2) * k.row_cap + rr;
#pragma unroll
              for (int x = 0; x < 16; x += 4, dst += k.row_cap) __stcg(dst, make_uint4(o[x], o[x + 1], o[x + 2], o[x + 3]));
            }
          }
        }
      }
      tc_fence_before();
      mbar_arrive(bar(c.o_free));                         // the accumulators may take the next segment
    } else if (warp == WARP_KEYS || warp == WARP_VALUES) {
      // -------------------------------------------------------------- keys (and queries), values: a warp each, since a page's
      // box is one lane's instruction and small pages make many of them
      const int kv = warp == WARP_VALUES, n_stages = kv ? Z::NV : Z::NK;
      const int page = a.g.page, per_tile = page < KT ? KT / page : 1;
      // the lane's page of a tile (lanes below per_tile), fetched one tile ahead
      auto fetch = [&](int tile) {
        const int key0 = tile * KT + lane * page;
        return lane < per_tile && key0 < g.s.total ? page_at(table, a.g.max_pages, a.g.n_pages, key0 / page) : -1;
      };
      int p_next = fetch(g.tile0);
      // the queries: (tree row, head) lines of both slots (of the same rows twice where they share them)
      auto load_queries = [&] {
        if (seg > 0) wait(c.q_empty, seg - 1);            // the last segment's first products have read theirs
        ok = __all_sync(0xffffffffu, ok);
        if (ok && lane == 0) {
          mbar_expect_tx(bar(c.q_full), 2 * k.slot_rows * a.G * HD * 2);
#pragma unroll 1
          for (int i = 0; i < 2 * Z::CB; ++i) {
            const int slot = i & 1, cb = i >> 1;
            tma_load_5d(base + Z::Q_OFF + slot * Z::Q_TILE + cb * BLOCK, &map_q, bar(c.q_full), cb * 64, g.head,
                        (2 * g.group + (halves ? slot : 0)) * k.slot_rows, g.b);
          }
        }
        n_queries += ok;
        __syncwarp();
      };
#pragma unroll 1
      for (int t = 0; ok && t < g.n; ++t) {
        const int p = p_next;
        if (t + 1 < g.n) p_next = fetch(g.tile0 + t + 1);
        const int in_page = page > KT ? (g.tile0 + t) * KT % page : 0;
        if (!kv) {
          const bool gone = __any_sync(0xffffffffu, p < 0 && lane < per_tile && (g.tile0 + t) * KT + lane * page < g.s.total);
          if (lane == 0) {
            c.gone[(tiles_before + t) % GONE_RING] = gone;
            if (gone) raise_status(a.status, POSS_E_INVALID);
          }
        }
        if (n_own >= n_stages) wait(c.kv_empty[kv][c_st], c_ph ^ 1);   // (a stage's first use waits for nobody)
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t full = bar(c.kv_full[kv][c_st]);
        const uint32_t dst = base + (kv ? Z::V_OFF : Z::K_OFF) + c_st * Z::TILE + lane * page * 128;
        if (lane == 0) mbar_expect_tx(full, Z::TILE);
        __syncwarp();
        if (lane < per_tile && !(k.inject_lost_load && kv)) {
          const int at = p >= 0 ? ((p * 2 + kv) * a.g.Hkv + g.head) * page + in_page : k.rows_total;
#pragma unroll
          for (int cb = 0; cb < Z::CB; ++cb) tma_load(dst + cb * KV_BLOCK, &map, full, cb * 64, at);
        }
        __syncwarp();
        ++n_own;
        if (++c_st == n_stages) { c_st = 0; c_ph ^= 1; }
        // (behind the first tile: keys need not wait for the last segment to give its queries' place up)
        if (ok && t == 0 && !kv) load_queries();
      }
    } else {
      // -------------------------------------------------------------- products
      const uint32_t slot = warp - WARP_MMA;
      const int steps = halves ? g.n : (g.n - (int)slot + 1) >> 1;
      // One lane walks and issues.  The tensor core needs 630 cycles for a step's products of one slot; what the lane does between
      // them leaves it idle unless the other slot's products fill the gap.
      if (elected && ok) {
        const uint32_t bars = base + Z::CTL_OFF;
        auto at = [&](const void* b) { return bars + (uint32_t)(reinterpret_cast<const char*>(b) - reinterpret_cast<const char*>(&c)); };
        auto pass = [&](uint32_t b, uint32_t phase) { ok = mbar_wait(b, phase, abort_flag); };
        const uint32_t b_s = at(&c.s_full[0][0]) + slot * 16, b_p = at(&c.p_full[0][0]) + slot * 16, b_o = at(&c.pv_done[0][0]) + slot * 16;
        const uint32_t b_kf = at(&c.kv_full[0][0]), b_vf = at(&c.kv_full[1][0]), b_ke = at(&c.kv_empty[0][0]), b_ve = at(&c.kv_empty[1][0]);
        const uint32_t d_s = tm + slot * S_COLS, d_o = tm + 2 * S_COLS + slot * HD;
        // (only a descriptor's lower word moves)
        const uint32_t q_lo = (uint32_t)q_desc + slot * (Z::Q_TILE >> 4), k_lo = (uint32_t)k_desc, v_lo = (uint32_t)v_desc;
        const uint32_t qk_hi = (uint32_t)(q_desc >> 32), v_hi = (uint32_t)(v_desc >> 32);
        const uint32_t stride = halves ? 8 : 16;
        // the slot's next keys and values: their stage's place among the barriers (8 times the stage), and phase
        const int skip = halves ? 0 : (int)slot, t0 = tiles_before + skip;
        uint32_t k_at = t0 % Z::NK * 8, k_ph = (t0 / Z::NK) & 1, v_at = t0 % Z::NV * 8, v_ph = (t0 / Z::NV) & 1;
        int keys = g.s.total - (g.tile0 + skip) * KT;     // keys from the step's first one on
        auto advance = [&](uint32_t& x, uint32_t& ph, uint32_t n) {
          x += stride;
          if (x >= n * 8) { x -= n * 8; ph ^= 1; }
        };
        // a stage is free after two arrivals: one of each slot, or both of the one slot that uses the tile
        auto release = [&](uint32_t b) {
          umma_commit(b);
          if (!halves) umma_commit(b);
        };
        pass(at(&c.q_full), par);
        if (steps == 0) mbar_arrive(at(&c.q_empty));
        // S = Q K^T of the slot's next tile, keys that have landed
        auto scores = [&](uint32_t d, uint32_t bar_s) {
          const uint32_t kd = k_lo + k_at * (Z::TILE >> 7);
#pragma unroll
          for (int cb = 0; cb < Z::CB; ++cb)
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              umma_bf16(d, pack64(q_lo + cb * (BLOCK >> 4) + ROW16 * kk, qk_hi), pack64(kd + cb * (KV_BLOCK >> 4) + ROW16 * kk, qk_hi),
                        idesc_s, (cb | kk) ? 1u : 0u);
          umma_commit(bar_s);
          release(b_ke + k_at);
          advance(k_at, k_ph, Z::NK);
        };
        // ---- the first two tiles' scores
#pragma unroll 1
        for (int y = 0; y < 2 && y < steps && ok; ++y) {
          pass(b_kf + k_at, k_ph);
          tc_fence_after();
          const uint32_t buf = (n_own + y) & 1;
          if (ok) scores(d_s + buf * KT, b_s + buf * 8);
        }
        if (seg > 0 && steps > 0) pass(at(&c.o_free), par ^ 1);
        if (steps > 0 && steps <= 2) umma_commit(at(&c.q_empty));   // (see Ctl; with more steps, behind the last first product)
        // ---- O += P V of step y, then S = Q K^T of step y + 2 over the P that was read: one thread's products run in order.
        // The slot's softmax works on step y + 1 meanwhile.  (Phases run on over the segments: n_own steps before this one.)
#pragma unroll 1
        for (int y = 0; ok && y < steps; ++y) {
          const uint32_t n = n_own + y, buf = n & 1, d = d_s + buf * KT;
          const bool more = y + 2 < steps;
          // the three barriers are asked one behind the other: an answer takes 80 cycles
          const uint32_t v_here = mbar_try_wait(b_vf + v_at, v_ph), k_here = more ? mbar_try_wait(b_kf + k_at, k_ph) : 1u,
                         p_here = mbar_try_wait(b_p + buf * 8, (n >> 1) & 1);
          if (!v_here) pass(b_vf + v_at, v_ph);
          if (!p_here && ok) pass(b_p + buf * 8, (n >> 1) & 1);
          if (!ok) break;
          tc_fence_after();
          const uint32_t v = v_lo + v_at * (Z::TILE >> 7), acc = y > 0;
          if (keys >= KT) {
            umma_bf16_ts(d_o, d, pack64(v, v_hi), idesc_o, acc);
            umma_bf16_ts(d_o, d + P_COLS, pack64(v, v_hi), idesc_o, 1u);
#pragma unroll
            for (int ks = 1; ks < KT / 16; ++ks) {        // 16 keys = 2048 bytes further each
              umma_bf16_ts(d_o, d + ks * 8, pack64(v + ks * 128, v_hi), idesc_o, 1u);
              umma_bf16_ts(d_o, d + P_COLS + ks * 8, pack64(v + ks * 128, v_hi), idesc_o, 1u);
            }
          } else {
#pragma unroll 1
            for (int ks = 0; ks * 16 < keys; ++ks) {
              umma_bf16_ts(d_o, d + ks * 8, pack64(v + ks * 128, v_hi), idesc_o, ks ? 1u : acc);
              umma_bf16_ts(d_o, d + P_COLS + ks * 8, pack64(v + ks * 128, v_hi), idesc_o, 1u);
            }
          }
          umma_commit(b_o + buf * 8);
          release(b_ve + v_at);
          advance(v_at, v_ph, Z::NV);
          keys -= (int)stride * (KT / 8);
          if (more) {
            if (!k_here) {
              pass(b_kf + k_at, k_ph);
              if (!ok) break;
              tc_fence_after();
            }
            scores(d, b_s + buf * 8);
            if (y + 3 == steps) umma_commit(at(&c.q_empty));
          }
        }
      }
      n_own += steps;
      __syncwarp();
    }
    tiles_before += g.n;
  }

  if (*abort_flag) {
    // copies and products under way must end before the CTA's shared memory and TMEM go away
    const uint64_t t0 = global_ns();
    if (warp == WARP_KEYS || warp == WARP_VALUES) {
      const int kv = warp == WARP_VALUES, n = kv ? Z::NV : Z::NK;
      while (n_queries > 0 && !mbar_try_wait(bar(c.q_full), (uint32_t)((n_queries - 1) & 1)) && global_ns() - t0 < WAIT_LIMIT_NS / 2)
        __nanosleep(64);
      for (int i = n_own > n ? n_own - n : 0; i < n_own; ++i)
        while (!mbar_try_wait(bar(c.kv_full[kv][i % n]), (uint32_t)((i / n) & 1)) && global_ns() - t0 < WAIT_LIMIT_NS / 2)
          __nanosleep(64);
    } else if (elected) {
      umma_commit(bar(c.drain[warp - WARP_MMA]));
      while (!mbar_try_wait(bar(c.drain[warp - WARP_MMA]), 0) && global_ns() - t0 < WAIT_LIMIT_NS / 2) __nanosleep(64);
    }
  }
  if (blockIdx.x == 0 && warp == WARP_KEYS) {
    uint32_t before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 32) {
      const int b = b0 + lane;
      uint32_t u = 0;
      if (b < a.batch) {
        const SeqWork s = seq_work(k, b);
        if (s.bad) raise_status(a.status, POSS_E_INVALID);
        u = s.units;
      }
      const uint32_t x = inclusive_scan(u);
      if (b < a.batch) k.plan->before[b] = before + x - u;
      before += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == WARP_MMA) tmem_dealloc(tm, TMEM_COLS);
  if (threadIdx.x == 0 && *abort_flag) raise_status(a.status, POSS_E_TIMEOUT);
}

// ---------------------------------------------------------------------------------------------------- merge
// A block: 32 query rows of one item, eight threads per row.  The item's segments lie in consecutive CTAs, in key order.
// SCORES: the slots' weights, from the scores that the attention has left.  A block is dealt 1024 slots of an item at a time; own: a thread's
// line's maximum and the inverse of its sum, for the first threads.  Where the blocks of merge and weights are few they share a launch (1 token
// over 1024 slots 18.2 us, with a launch more 21.6; 16 tokens 31.8 and 33.8) and the lines' sums come from the parts once more; else the
// weights are a launch of their own, whose blocks need a third of the merge's registers (16 tokens over up to 8191 slots 101 us, in one launch
// 106).
struct Lines { float2 ml[32]; };             // by line: maximum, and the inverse of the sum times the row's weight
__device__ __forceinline__ void add_weights(const TcArgs& k, const SeqWork& s, int b, int head, float2 own, int first_key, int step, Lines& sh) {
  const PagedAttnArgs& a = k.a;
  const int t = threadIdx.x, lines = s.rows * a.G;
  if (t < 32) {
    if (k.row_weights && t < lines) own.y *= k.row_weights[(size_t)b * a.rows + t / a.G];
    sh.ml[t] = own;
  }
  __syncthreads();
  const float* const scores = k.scores + ((size_t)b * a.g.Hkv + head) * (a.rows * a.G) * k.scores_ld;
  float* const mass = k.mass + ((size_t)b * a.g.Hkv + head) * k.mass_slots;
  for (int key = first_key + 4 * t; key < s.total; key += step) {
    float old[4], sum[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      old[x] = key + x < s.prefix ? mass[key + x] : 0.f;
      sum[x] = 0.f;
    }
#pragma unroll 4
    for (int i = 0; i < lines; ++i) {
      const float4 y = __ldcg(reinterpret_cast<const float4*>(scores + i * k.scores_ld + key));
      const float2 c = sh.ml[i];
      const float v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float p = ex2(fmaf(v[x], k.scale_log2, -c.x)) * c.y;
        sum[x] += v[x] == -INFINITY ? 0.f : p;            // (unseen: nothing, even where the row's sum is NaN)
      }
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (key + x < s.total) mass[key + x] = old[x] + sum[x];
  }
}
__global__ void __launch_bounds__(256) k_paged_attn_weights(const TcArgs k) {
  __shared__ Lines sh;
  pdl_enter(POSS_K_SLOT_MASS);
  const int b = blockIdx.z, head = blockIdx.y, t = threadIdx.x;
  const SeqWork s = seq_work(k, b);
  if (!s.rows) return;
  float2 own = make_float2(INFINITY, 0.f);
  if (t < s.rows * k.a.G) own = __ldcg(k.a.ml + ((size_t)b * k.a.rows + t / k.a.G) * k.a.Hq + head * k.a.G + t % k.a.G);
  add_weights(k, s, b, head, own, blockIdx.x * 1024, gridDim.x * 1024, sh);
}
// in the merge's launch: the line's maximum and sum from the segments' (by thread, for those below the number of lines)
template <int HD>
__device__ __forceinline__ float2 line_of(const TcArgs& k, const SeqWork& s, int b, int head, uint32_t total, uint32_t before, int whole,
                                          int cut_grid, float2 (*s_ml)[32]) {
  const PagedAttnArgs& a = k.a;
  const int t = threadIdx.x, lines = s.rows * a.G;
  int first = 0, last = 0, which = 0;
  if (!whole) {
    const Cut cut(total, cut_grid);
    const uint32_t u0 = before + (uint32_t)head * s.tiles;
    first = cut.cta_of(u0);
    last = cut.cta_of(u0 + s.tiles - 1);
    which = cut.begin(first) < u0 ? 1 : 0;
  }
  if (first == last) return t < lines ? __ldcg(a.ml + ((size_t)b * a.rows + t / a.G) * a.Hq + head * a.G + t % a.G) : make_float2(INFINITY, 0.f);
  for (int i = t >> 5; i <= last - first; i += 8)
    if ((t & 31) < lines)
      s_ml[i][t & 31] = __ldcg(reinterpret_cast<const float2*>(partial_of(k, HD, first + i, i == 0 ? which : 0) + (size_t)k.row_cap * HD) + (t & 31));
  __syncthreads();
  if (t >= lines) return make_float2(INFINITY, 0.f);
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i <= last - first; ++i) m = fmaxf(m, s_ml[i][t].x);
  for (int i = 0; i <= last - first; ++i) {               // (as the merge does)
    const float2 x = s_ml[i][t];
    const float c = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : ex2(x.x - m);
    if (c != 0.f) l = fmaf(x.y, c, l);
  }
  return paged_ml(m, l);
}
template <int HD, bool SCORES>
__global__ void __launch_bounds__(256) k_paged_attn_tc_merge(const TcArgs k, int max_groups) {
  constexpr int NV = HD / 32;                             // float4 per thread
  __shared__ float2 s_ml[MAX_CTAS][32];
  pdl_enter(POSS_K_PAGED_ATTN_COMBINE);
  const PagedAttnArgs& a = k.a;
  const int b = blockIdx.z, head = blockIdx.y / max_groups, group = blockIdx.y - head * max_groups;
  const PlanOut* const plan = k.plan;
  const uint32_t total = __ldcg(&plan->total), before = __ldcg(&plan->before[b]);
  const int whole = __ldcg(&plan->whole), cut_grid = __ldcg(&plan->grid);
  const SeqWork s = seq_work(k, b);
  if constexpr (SCORES) {
    if ((int)blockIdx.x >= k.merge_blocks) {
      __shared__ Lines sh;
      if (s.rows)
        add_weights(k, s, b, head, line_of<HD>(k, s, b, head, total, before, whole, cut_grid, s_ml), (blockIdx.x - k.merge_blocks) * 1024,
                    (gridDim.x - k.merge_blocks) * 1024, sh);
      return;
    }
  }
  if (whole || group >= s.groups) return;                 // (whole: nothing was cut)
  // line rr of the item: slot, tree row and head
  const int rr = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5, line = rr % QR;
  const int in_slot = line / a.G, r = (2 * group + rr / QR) * k.slot_rows + in_slot, qh = line - in_slot * a.G;
  const Cut cut(total, cut_grid);
  const uint32_t u0 = before + ((uint32_t)head * s.groups + group) * s.tiles;
  const int first = cut.cta_of(u0), last = cut.cta_of(u0 + s.tiles - 1);
  if (first == last) return;                              // written by its CTA
  // the first CTA's segment is its last one unless its range starts with the item; every later one's is its first
  const int which = cut.begin(first) < u0 ? 1 : 0;
  auto part_of = [&](int cta) { return partial_of(k, HD, cta, cta == first ? which : 0); };
  const bool valid = in_slot < k.slot_rows && r < s.rows;
  // the segments' maxima and sums, eight segments at a time
  if (valid)
    for (int i = slice; i <= last - first; i += 8)
      s_ml[i][rr & 31] = __ldcg(reinterpret_cast<const float2*>(part_of(first + i) + (size_t)k.row_cap * HD) + rr);
  __syncthreads();
  if (!valid) return;
  const int n = last - first + 1;
  float l = 0.f;
  float4 o[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) o[v] = make_float4(0.f, 0.f, 0.f, 0.f);
  // Four segments' outputs are in flight at a time, the first four beside the maxima: two trips to memory in all for up to four.
  auto load = [&](int i, float4* y) {
    const float4* p = reinterpret_cast<const float4*>(part_of(first + (i < n ? i : n - 1)));
#pragma unroll
    for (int v = 0; v < NV; ++v) y[v] = __ldcg(p + (size_t)(slice * NV + v) * k.row_cap + rr);
  };
  float4 y[4][NV];
#pragma unroll
  for (int i = 0; i < 4; ++i) load(i, y[i]);
  float m = -INFINITY;
  for (int i = 0; i < n; ++i) m = fmaxf(m, s_ml[i][rr & 31].x);
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i0 + i < n) {
        const float2 x = s_ml[i0 + i][rr & 31];
        // a segment that has seen nothing is left out (sum 0); one whose scores were all NaN is not
        const float c = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : ex2(x.x - m);
        if (c != 0.f) {                                   // (NaN too)
          l = fmaf(x.y, c, l);
#pragma unroll
          for (int v = 0; v < NV; ++v) {
            o[v].x = fmaf(y[i][v].x, c, o[v].x); o[v].y = fmaf(y[i][v].y, c, o[v].y);
            o[v].z = fmaf(y[i][v].z, c, o[v].z); o[v].w = fmaf(y[i][v].w, c, o[v].w);
          }
        }
      }
      if (i0 + 4 + i < n) load(i0 + 4 + i, y[i]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16* out = reinterpret_cast<bf16*>(a.out) + (((size_t)b * a.rows + r) * a.Hq + head * a.G + qh) * HD + slice * (HD / 8);
#pragma unroll
  for (int v = 0; v < NV; ++v)
    *reinterpret_cast<uint2*>(out + 4 * v) =
        make_uint2(pack_bf16(o[v].x * inv, o[v].y * inv), pack_bf16(o[v].z * inv, o[v].w * inv));
  if (!SCORES && a.ml && slice == 0) a.ml[((size_t)b * a.rows + r) * a.Hq + head * a.G + qh] = paged_ml(m, l);
}

std::atomic<int> g_spared_loads{0}, g_lost_loads{0};   // launches that go on before, and those that lose a load

constexpr size_t PLAN_BYTES = (sizeof(PlanOut) + 255) / 256 * 256;
// lines of an item that can hold query rows: one slot's, or both
int row_cap_of(int rows, int G) { return rows > QR / G ? 2 * QR : (rows * G + 31) / 32 * 32; }

template <int HD, bool SCORES>
void launch(Launcher& L, const TcArgs& k0, const CUtensorMap& map, const CUtensorMap& map_q, long long units, long long tiles, int groups) {
  using Z = Shape<HD>;
  TcArgs k = k0;
  const PagedAttnArgs& a = k.a;
  const size_t smem = Z::CTL_OFF + CTL_BYTES;
  k.smem_bytes = (uint32_t)smem;
  static PerDeviceFlags attr_done;
  bool* attr = attr_done.current();
  if (!attr || !*attr) {
    if (cudaFuncSetAttribute(k_paged_attn_tc<HD, SCORES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
      L.err = POSS_E_CUDA;
      return;
    }
    if (attr) *attr = true;
  }
  // one CTA per SM, as many as the fullest tables can give a unit
  const int sms = current_sm_count();
  int ctas = units < sms ? (int)units : sms;
  if (ctas > MAX_CTAS) ctas = MAX_CTAS;
  k.merge_blocks = tiles > 1 ? k.row_cap / 32 : 0;        // (an item of one tile is never cut)
  launch_pdl(L, k_paged_attn_tc<HD, SCORES>, dim3(ctas), dim3(N_THREADS), smem, map, map_q, k);
  // weights: some sixteen blocks per SM in all, each with 1024 slots at least
  const long long items = (long long)a.batch * a.g.Hkv, most = (tiles * KT + 1023) / 1024, n = (16 * sms + items - 1) / items;
  const int weights = SCORES ? (int)(n < most ? n : most) : 0;
  const bool together = (k.merge_blocks + weights) * items <= 4 * sms;   // (two waves of blocks, two per SM)
  const int blocks = k.merge_blocks + (together ? weights : 0);
  if (blocks && L.err == POSS_OK) {
    const dim3 grid(blocks, a.g.Hkv * groups, a.batch);
    if (SCORES && together) launch_pdl(L, k_paged_attn_tc_merge<HD, true>, grid, dim3(256), 0, k, groups);
    else launch_pdl(L, k_paged_attn_tc_merge<HD, false>, grid, dim3(256), 0, k, groups);
  }
  if (weights && !together && L.err == POSS_OK) launch_pdl(L, k_paged_attn_weights, dim3(weights, a.g.Hkv, a.batch), dim3(256), 0, k);
}

}  // namespace

namespace {
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
}  // namespace

bool paged_take_lost_load() {
  auto take = [](std::atomic<int>& left) {
    int n = left.load();
    while (n > 0 && !left.compare_exchange_weak(n, n - 1)) {}
    return n > 0;
  };
  return !take(g_spared_loads) && take(g_lost_loads);
}
bool paged_kv_map(CUtensorMap* map, const PagedAttnArgs& a, const void* layer, int slots) {
  const EncodeTiledFn encode = encode_fn();
  const cuuint64_t dim[2] = {(cuuint64_t)a.g.d, (cuuint64_t)a.g.n_pages * 2 * a.g.Hkv * a.g.page};
  const cuuint64_t str[1] = {(cuuint64_t)a.g.d * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)slots}, one[2] = {1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(layer), dim, str, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool paged_q_map(CUtensorMap* map, const PagedAttnArgs& a, int tree_rows) {
  const EncodeTiledFn encode = encode_fn();
  const cuuint64_t row = (cuuint64_t)a.ld_q * 2;
  const cuuint64_t dim[5] = {(cuuint64_t)a.g.d, (cuuint64_t)a.G, (cuuint64_t)a.g.Hkv, (cuuint64_t)a.rows, (cuuint64_t)a.batch};
  const cuuint64_t str[4] = {(cuuint64_t)a.g.d * 2, (cuuint64_t)a.G * a.g.d * 2, row, row * a.rows};
  const cuuint32_t box[5] = {64, (cuuint32_t)a.G, 1, (cuuint32_t)tree_rows, 1}, one[5] = {1, 1, 1, 1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(a.q), dim, str, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool paged_attn_tc_supported(const poss_page_pool& p, int G, float scale) {
  if (G > QR) return false;
  if (p.dtype != POSS_BF16 || (p.head_dim != 64 && p.head_dim != 128)) return false;
  if (!(scale > 0.f)) return false;                       // maxima are taken before scaling
  const int s = p.page_slots;
  return s == 16 || s == 32 || s == 64 || s == 128 || s == 256;
}

// Scores go through memory (4 bytes to and fro per line and slot) where that is no more than reading the keys again (2 bytes per element) to
// form them anew.  16 trees of 4 heads over up to 8191 slots, attention and weights: 1 row 101 us (keys again: 144), 4 rows 114 (150), 8 rows
// 140 (147), 9 rows, just above, 148; 64 single tokens over up to 8000: 306 (413).
size_t paged_attn_tc_scores(const poss_page_pool& p, int batch, int rows, int Hq, int max_pages) {
  const int lines = rows * (Hq / p.n_kv_heads);
  if (lines > p.head_dim / 4) return 0;
  const size_t ld = ((size_t)max_pages * p.page_slots + KT - 1) / KT * KT;
  return (size_t)batch * p.n_kv_heads * lines * ld * 4;
}

size_t paged_attn_tc_workspace(const poss_page_pool& p, int batch, int rows, int Hq, int max_pages) {
  // the plan; two partials per CTA (its first and its last segment); the grid is at most the SM count
  (void)batch; (void)max_pages;
  const int sms = current_sm_count();
  return PLAN_BYTES + (size_t)(sms < MAX_CTAS ? sms : MAX_CTAS) * 2 * row_cap_of(rows, Hq / p.n_kv_heads) * (p.head_dim + 2) * 4;
}

void launch_paged_attn_tc(Launcher& L, const PagedAttnArgs& a, const void* pool, const poss_page_pool& p, const PagedMassArgs* mass) {
  const long long tiles = ((long long)a.g.max_pages * a.g.page + KT - 1) / KT;
  const int groups = (a.rows + 2 * (QR / a.G) - 1) / (2 * (QR / a.G));
  const long long units = (long long)a.batch * a.g.Hkv * groups * tiles;
  if (units >= (1ll << 31)) { L.err = POSS_E_CAPACITY; return; }
  TcArgs k;
  memset(&k, 0, sizeof(k));
  k.a = a;
  k.plan = reinterpret_cast<PlanOut*>(a.ws);
  k.a.ws = reinterpret_cast<char*>(a.ws) + PLAN_BYTES;
  k.layer = reinterpret_cast<const bf16*>(pool) + page_offset(a.g, a.layer, 0, 0, 0);
  k.scale_log2 = a.scale * 1.4426950408889634f;
  k.slot_rows = QR / a.G;
  k.row_cap = row_cap_of(a.rows, a.G);
  k.rows_total = a.g.n_pages * 2 * a.g.Hkv * a.g.page;
  k.inject_lost_load = paged_take_lost_load();
  CUtensorMap map, map_q;
  if (!paged_kv_map(&map, a, k.layer, a.g.page < KT ? a.g.page : KT) || !paged_q_map(&map_q, a, k.slot_rows)) {
    L.err = POSS_E_CUDA;
    return;
  }
  if (!mass) {
    if (a.g.d == 128) launch<128, false>(L, k, map, map_q, units, tiles, groups);
    else launch<64, false>(L, k, map, map_q, units, tiles, groups);
    return;
  }
  k.scores = mass->scores;
  k.scores_ld = tiles * KT;
  k.mass = mass->mass;
  k.mass_slots = mass->mass_slots;
  k.row_weights = mass->weights;
  if (a.g.d == 128) launch<128, true>(L, k, map, map_q, units, tiles, groups);
  else launch<64, true>(L, k, map, map_q, units, tiles, groups);
}

extern "C" int poss_debug_paged_lose_load(int launches) { return poss_debug_paged_lose_load_after(0, launches); }

extern "C" int poss_debug_paged_lose_load_after(int spared, int launches) {
  if (spared < 0 || launches < 0) return POSS_E_INVALID;
  g_lost_loads.store(0);                                  // (a launch meanwhile loses nothing)
  g_spared_loads.store(spared);
  g_lost_loads.store(launches);
  return POSS_OK;
}
