// Log-probabilities of given tokens, with each row's entropy and best tokens, over a vocabulary.
//
//   p = softmax(x / T);  log p(token);  H = -sum p log p;  the K best tokens with log p
//
// One pass over the logits and one launch: a row belongs to a cluster of 1 to 8 CTAs, each of which streams 8192 logits per step, 32 per
// thread.  A thread keeps s = sum 2^t and w = sum t 2^t, t = x log2(e) / T - base, with a whole number as its base (the product is exact
// inside the multiply-add, the difference rounded once); at the end
//   log sum e^(x / T) = ln 2 (base + log2 s),  H = ln 2 (log2 s - w / s).
// Nothing is looked at while all goes well: a logit far above the base, a banned one (-inf: 0 times its t is NaN), NaN and logits beyond
// 2^20 show in a step's sums, which are then formed anew, or with care in a pass of their own.  That saves the clamps and the extremes.
// Logits below -2^20, such as a mask of the type's lowest value, are left out where others make up the sum.
//
// The K best.  The first step's bound is the K-th best of 32 maxima of disjoint parts of the CTA: K logits are at or above it.  What reaches
// the bound is listed; behind steps 4, 16, ... and the last the list is cut to its K best, the last of which is the next bound (only
// greater ones can follow: places rise from step to step).  Listing costs nothing but where a thread's maximum of eight reaches the bound.
// A step that is mostly masked (most parts' maxima equal the bound) lists what is above the mask, is cut at once, and leaves the bound to the
// next step if that was fewer than K.  A list that overflows (ever rising logits), or whose K best are no better than a mask, makes the CTA
// read its part again, a slower way: warps keep their K best in order, one per lane.  Entries are 64-bit numbers that order as (value, token)
// do, so that an entry's place is the count of those above it; the cluster's first CTA joins the others' lists and sums.
// w / s and log2 s are at most some 20 (a thread's base is its first step's maximum, until a step passes it by some 17): as fp32 quotient and sum
// that leaves an entropy off by 2e-6 at the worst, besides what the terms' own roundings make.
// Given tokens with rows of their own (a tree's) are looked for by every row's first CTA, rows x n_tokens reads: 2048 tokens of 2048 rows 4 us,
// 32768 tokens 85.
// What bounds it: 2048 rows over 128256 bf16 tokens, 525 MB, take 93 to 95 us without best tokens (5.5 TB/s), 110 with one and 134 with 10 (with
// a quarter of the tokens banned in one piece 143 and 179, with all but 0.1 % 150 and 183, with 70 % strewn 169 and 188), where a CTA's few
// barriers and a warp's looks at reached bounds cost more than the maxima.  Nothing is full by the counters: with the best one DRAM 55 %, the
// exponentials' pipe 60 %, 2.4 instructions of 4 a cycle; the last of 4.6 waves of CTAs is two thirds full.  1024 rows over as many fp32 tokens,
// the same bytes: 80 us (6.5 TB/s), 85 with one, 93 with 10.  One row over 128256 fp32 tokens with 10 best ones 9.2 us: launch, two steps, a
// cut and the cluster's join.
#include "paged.cuh"
#include <atomic>
#include <cooperative_groups.h>
#include <float.h>

POSS_TRACE_REGISTER()

namespace {

namespace cg = cooperative_groups;

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int PER = 32;                      // logits of a thread and step
constexpr int STEP = THREADS * PER;
constexpr int KMAX = POSS_MAX_TOPK;
constexpr int MAX_CLUSTER = 8;               // (log_cs 0 to 3)
constexpr int PARTS = 32;                    // of eight threads each: their maxima give the first bound
constexpr int LIST = 512;                    // entries that may wait for the next cut
constexpr int AT_ONCE = 8;                   // logits of a thread on their way in the slower ways

struct Args {
  const void* logits;
  long long ld;
  int rows, V, K, n_tokens;
  float c;                   // log2(e) / T
  double inv_t;
  const int32_t *tokens, *token_rows;
  float *out_logp, *out_lse, *out_entropy;
  int32_t* out_top;
  float* out_top_logp;
};

__device__ __forceinline__ float max_nan(float a, float b, float c) {   // NaN if one of them is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// (value, index): greater value first, then lower index
__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }
// the same as a number (0: none): greater is earlier.  -0 is 0.
__device__ __forceinline__ unsigned long long key_of(float v, int i) {
  const uint32_t b = __float_as_uint(v + 0.f), o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (unsigned long long)o << 32 | (0xffffffffu - (uint32_t)i);
}
__device__ __forceinline__ float value_of(unsigned long long key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int token_of(unsigned long long key) { return (int)(0xffffffffu - (uint32_t)key); }
// the next value above a finite one or -inf
__device__ __forceinline__ float above(float v) {
  const int b = __float_as_int(v);
  return v == 0.f ? __int_as_float(1) : __int_as_float(v > 0.f ? b + 1 : b - 1);
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(uint4 w, float* x) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
};
template <> struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(uint4 w, float* x) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
};

__device__ __forceinline__ float max8(const float* x) {
  return max_nan(max_nan(max_nan(x[0], x[1], x[2]), x[3], x[4]), max_nan(x[5], x[6], x[7]), x[7]);
}

// Sums of any number of threads against a base in units of log2.  (s 0: nothing yet)
struct Sums { double base; float s, w; };
__device__ __forceinline__ Sums moved(Sums a, double base) {             // to a base that is not below it
  if (a.s != 0.f) {
    const float d = (float)fmax(a.base - base, -200.0), f = ex2(d);      // (2^-200 is 0, and 0 times a finite number)
    a.w = f * fmaf(a.s, d, a.w);
    a.s *= f;
  }
  a.base = base;
  return a;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b) {
  if (b.s == 0.f) return a;
  if (a.s == 0.f) return b;
  const double base = fmax(a.base, b.base);
  a = moved(a, base);
  b = moved(b, base);
  a.s += b.s;
  a.w += b.w;
  return a;
}
// the same with a base that fp32 holds
struct Sums32 { float base, s, w; };
__device__ __forceinline__ Sums32 joined(Sums32 a, Sums32 b) {
  if (b.s == 0.f) return a;
  if (a.s == 0.f) return b;
  const float base = fmaxf(a.base, b.base), da = fmaxf(a.base - base, -200.f), db = fmaxf(b.base - base, -200.f), fa = ex2(da), fb = ex2(db);
  return {base, fmaf(a.s, fa, b.s * fb), fmaf(fmaf(a.s, da, a.w), fa, fmaf(b.s, db, b.w) * fb)};
}
__device__ __forceinline__ Sums32 shfl_xor(Sums32 a, int o) {
  return {__shfl_xor_sync(0xffffffffu, a.base, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.w, o)};
}
__device__ __forceinline__ Sums shfl_xor(Sums a, int o) {
  return {__shfl_xor_sync(0xffffffffu, a.base, o), __shfl_xor_sync(0xffffffffu, a.s, o), __shfl_xor_sync(0xffffffffu, a.w, o)};
}
// A thread's sums while it streams
constexpr float SMALL = 0x1p20f;                          // bases below this: whole numbers that fp32 holds exactly
struct Stream {
  float base, s, w;
  bool rare;                                              // something that only `careful` can sum up
  // CLAMPED: with banned logits or some beyond all measure, whose power is 0 and t -inf
  template <bool CLAMPED> __device__ __forceinline__ bool plain(const float* x, float c) {
    const float2 cc = make_float2(c, c), off = make_float2(-base, -base), zero = make_float2(0.f, 0.f);
    float2 s0 = zero, s1 = zero, w0 = zero, w1 = zero;
#pragma unroll
    for (int j = 0; j < PER; j += 4) {
      float2 u = fma2(make_float2(x[j], x[j + 1]), cc, off), v = fma2(make_float2(x[j + 2], x[j + 3]), cc, off);
      if (CLAMPED) {
        u = make_float2(fmaxf(u.x, -200.f), fmaxf(u.y, -200.f));
        v = make_float2(fmaxf(v.x, -200.f), fmaxf(v.y, -200.f));
      }
      const float2 eu = make_float2(ex2(u.x), ex2(u.y)), ev = make_float2(ex2(v.x), ex2(v.y));
      s0 = add2(s0, eu);
      s1 = add2(s1, ev);
      w0 = fma2(eu, u, w0);
      w1 = fma2(ev, v, w1);
    }
    const float gs = (s0.x + s0.y) + (s1.x + s1.y), gw = (w0.x + w0.y) + (w1.x + w1.y);
    if (!(gs + fabsf(gw) < 0x1p21f)) return false;        // (NaN, or a logit some 17 above the base in units of log2)
    s += gs;
    w += gw;
    return true;
  }
  __device__ __forceinline__ void add(const float* x, float c, bool first) {
    if (first) {
      const float top = rintf(max_of(x) * c);
      if (fabsf(top) < SMALL) base = top;
    }
    if (plain<false>(x, c)) return;
    const float m = max_of(x), top = rintf(m * c);
    if (m == -INFINITY) return;                           // (banned all)
    if (top <= -SMALL) {                                  // nothing beside a logit that is not as low; else the base tells of it
      if (s == 0.f) base = -FLT_MAX;
      return;
    }
    if (!(top < SMALL)) { rare = true; return; }
    if (!(base >= top)) {
      if (s != 0.f) {
        const float d = fmaxf(base - top, -200.f), f = ex2(d);
        w = f * fmaf(s, d, w);
        s *= f;
      }
      base = top;
    }
    plain<true>(x, c);
  }
  static __device__ __forceinline__ float max_of(const float* x) {       // NaN if one of them is
    return max_nan(max_nan(max8(x), max8(x + 8), max8(x + 16)), max8(x + 24), max8(x + 24));
  }
};
// A thread's sums of elements [e0, e1) of a row, every THREADS-th from its own on, whatever they are: differences to a reference come
// first (one that overflows is -inf; those that count are near the reference, where they lose nothing).
template <typename T> __device__ __noinline__ Sums careful(const T* row, int e0, int e1, float c) {
  float ref = -INFINITY, s = 0.f, w = 0.f;
  for (int i = e0 + (int)threadIdx.x; i < e1; i += THREADS * AT_ONCE) {
    float xs[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) xs[u] = i + u * THREADS < e1 ? to_f(row[i + u * THREADS]) : -INFINITY;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const float x = xs[u];
      if (!(fabsf(x) < INFINITY)) continue;
      float t = (x - ref) * c;
      if (!(t <= 4.f)) {
        const float d = fmaxf((ref - x) * c, -200.f), f = s == 0.f ? 0.f : ex2(d);
        w = s == 0.f ? 0.f : f * fmaf(s, d, w);
        s *= f;
        ref = x;
        t = 0.f;
      }
      t = fmaxf(t, -200.f);
      const float e = ex2(t);
      s += e;
      w = fmaf(e, t, w);
    }
  }
  return {s == 0.f ? 0.0 : (double)ref * (double)c, s, w};
}

struct Shared {
  Sums32 sums[WARPS];
  Sums careful_sums[WARPS];
  unsigned long long list[LIST];
  int n;
  float part_max[PARTS];
  volatile float warp_bound[WARPS];          // the slower way: each warp's K-th best so far
  // what the cluster's first CTA is given
  Sums part[MAX_CLUSTER];
  unsigned long long best[MAX_CLUSTER * KMAX];
  double ref, ln_s;                          // the row's result: ln of the sum of e^((x - ref) / T)
  int any;
};

// The whole block: cuts a list of n entries (none twice; behind a barrier) to its K best, in order; 0 behind the last.  *reset = K on the way.
__device__ __forceinline__ void cut(unsigned long long* list, int n, int K, int* reset) {
  const int t = threadIdx.x;
  unsigned long long key[LIST / THREADS];
  int r[LIST / THREADS], valid = 0;
#pragma unroll
  for (int i = 0; i < LIST / THREADS; ++i) {
    const int at = t + i * THREADS;
    key[i] = at < n ? list[at] : 0ull;
    r[i] = K;
    if (key[i]) {
      r[i] = 0;
#pragma unroll 8
      for (int o = 0; o < n; ++o) r[i] += list[o] > key[i];
    }
  }
#pragma unroll
  for (int i = 0; i < LIST / THREADS; ++i)
    if (i == 0 || n > i * THREADS) valid += __syncthreads_count(key[i] != 0ull);
  if (t < K && t >= valid) list[t] = 0ull;
  if (t == 0) *reset = K;
#pragma unroll
  for (int i = 0; i < LIST / THREADS; ++i)
    if (r[i] < K) list[r[i]] = key[i];
  __syncthreads();
}
// The slower way: the K best of elements [e0, e1) to sh.list.  Every warp keeps its K best in order, one per lane, and takes in what is above
// the K-th and at or above any other warp's K-th (which proves that K of the CTA's are no worse).
template <typename T> __device__ __noinline__ void best_slowly(const T* row, int e0, int e1, int K, Shared* sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) sh->warp_bound[warp] = -INFINITY;
  __syncthreads();
  float lv = -INFINITY;                      // the lane's entry of the warp's list
  int li = 0x7fffffff;
  auto bound = [&] {
    float others = lane < WARPS ? sh->warp_bound[lane] : -INFINITY;
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) others = fmaxf(others, __shfl_xor_sync(0xffffffffu, others, o));
    const float own = __shfl_sync(0xffffffffu, lv, K - 1);
    return fmaxf(above(own), __shfl_sync(0xffffffffu, others, 0));   // (places rise)
  };
#pragma unroll 1
  for (int j0 = e0 + warp * 32; j0 < e1; j0 += THREADS * AT_ONCE) {
    float xs[AT_ONCE], m = -INFINITY;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) xs[u] = j0 + u * THREADS + lane < e1 ? to_f(row[j0 + u * THREADS + lane]) : -INFINITY;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (!(fabsf(xs[u]) < INFINITY)) xs[u] = -INFINITY;
      m = fmaxf(m, xs[u]);
    }
    if (!__any_sync(0xffffffffu, m >= bound())) continue;
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const float x = xs[u];
      unsigned who = __ballot_sync(0xffffffffu, x >= bound());
      if (!who) continue;
      while (who) {
        const int src = __ffs(who) - 1;
        who &= who - 1;
        const float v = __shfl_sync(0xffffffffu, x, src);
        const int vi = j0 + u * THREADS + src, pos = __popc(__ballot_sync(0xffffffffu, before(lv, li, v, vi)));
        const float uv = __shfl_up_sync(0xffffffffu, lv, 1);
        const int ui = __shfl_up_sync(0xffffffffu, li, 1);
        if (lane == pos) { lv = v; li = vi; }
        else if (lane > pos) { lv = uv; li = ui; }
      }
      const float now = __shfl_sync(0xffffffffu, lv, K - 1);
      if (lane == 0) sh->warp_bound[warp] = now;
    }
  }
  if (lane < K) sh->list[warp * K + lane] = lv > -INFINITY ? key_of(lv, li) : 0ull;
  __syncthreads();
  cut(sh->list, WARPS * K, K, &sh->n);
}

template <typename T>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 ? 3 : 4) k_token_logprobs(Args a, int log_cs) {
  constexpr int N = Vec<T>::N, PIECES = PER / N;
  constexpr bool AHEAD = sizeof(T) == 2;
  __shared__ Shared sh;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, K = a.K;
  const int row = blockIdx.x >> log_cs, cs = 1 << log_cs, rank = blockIdx.x & (cs - 1);
  if (t == 0) sh.n = 0;
  // (the cluster's first CTA must have begun before the others write to it)
  if (cs > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  __syncthreads();
  pdl_enter(POSS_K_TOKEN_LOGPROBS);
  const T* const base = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld;
  // the row: single logits up to a 16-byte boundary, pieces of 16 bytes that the CTAs share, single logits
  const int head = min(a.V, (int)((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / (int)sizeof(T));
  const int pieces = (a.V - head) / N, tail = a.V - head - pieces * N;
  const int p0 = (int)((long long)pieces * rank >> log_cs), p1 = (int)((long long)pieces * (rank + 1) >> log_cs);
  const int n_head = rank == 0 ? head : 0, n_tail = rank == cs - 1 ? tail : 0;
  const int steps = (p1 - p0 + THREADS * PIECES - 1) / (THREADS * PIECES), all_steps = steps + (n_head + n_tail > 0);
  const uint4* const body = reinterpret_cast<const uint4*>(base + head);

  Stream sum = {NAN, 0.f, 0.f, false};
  float lo = -FLT_MAX;                       // what may be among the best: at or above it
  constexpr int FIRST_CUT = 4;
  int next_cut = FIRST_CUT, span = 3 * FIRST_CUT;         // steps between that cut and the one behind it
  bool overflow = false;
  int bound_at = 0;                          // the step whose maxima give a bound
  float skipped = -INFINITY;                 // what equals it or is less may not be listed
  const int full = (p1 - p0) / (THREADS * PIECES);        // steps without a gap
  auto fetch = [&](int it, uint4* w) {
    const uint4* const from = body + p0 + it * (THREADS * PIECES) + t;
    if (it < full) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) w[i] = __ldcs(from + i * THREADS);
    } else {
      const uint32_t none = N == 8 ? 0xff80ff80u : 0xff800000u;          // -inf
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        w[i] = p0 + it * (THREADS * PIECES) + t + i * THREADS < p1 ? __ldcs(from + i * THREADS) : make_uint4(none, none, none, none);
    }
  };
  // bf16: the next step's logits are on their way while a step is worked on (16 registers, and three CTAs per SM instead of four: 2048 rows
  // over 128256 with the best one 118 -> 109 us); twice as many registers for fp32 cost more than they give (one row 8.9 -> 10.2 us)
  uint4 ahead[PIECES];
  if (AHEAD) fetch(0, ahead);
#pragma unroll 1
  for (int it = 0; it < all_steps; ++it) {
    // the step's logits; the step behind the last: single ones
    const int at = p0 + it * (THREADS * PIECES) + t;
    float x[PER];
    if (it < steps) {
      if (!AHEAD) fetch(it, ahead);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) Vec<T>::get(ahead[i], x + i * N);
      if (AHEAD) fetch(it + 1, ahead);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) x[i] = -INFINITY;
      if (t < n_head) x[0] = to_f(base[t]);
      if (t < n_tail) x[1] = to_f(base[a.V - n_tail + t]);
    }
    sum.add(x, a.c, it == 0);
    if (K > 0) {
      float q[PER / 8], m;
      auto maxima = [&] {
#pragma unroll
        for (int j = 0; j < PER / 8; ++j) q[j] = max8(x + 8 * j);
        m = max_nan(max_nan(q[0], q[1], q[2]), q[3], q[3]);
      };
      static_assert(PER == 32, "four eights");
      maxima();
      if (!(m < INFINITY)) {
#pragma unroll
        for (int j = 0; j < PER; ++j) x[j] = fabsf(x[j]) < INFINITY ? x[j] : -INFINITY;
        maxima();
      }
      if (it == bound_at) {
        float mp = m;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) mp = fmaxf(mp, __shfl_xor_sync(0xffffffffu, mp, o));
        if ((lane & 7) == 0) sh.part_max[t >> 3] = mp;
        __syncthreads();
        // the K-th best of them
        static_assert(PARTS == 32 && THREADS == 8 * PARTS && KMAX <= PARTS, "one per lane");
        const float own = sh.part_max[lane];
        int r = 0;
#pragma unroll
        for (int o = 0; o < PARTS; ++o) r += before(sh.part_max[o], o, own, lane);
        const unsigned who = __ballot_sync(0xffffffffu, r == K - 1);
        const float b = __shfl_sync(0xffffffffu, own, __ffs(who) - 1);
        lo = fmaxf(lo, b);
        // Most parts have nothing better: a mask, whatever its value.  (2048 rows over 128256 bf16 tokens, 10 best of the 0.1 % above the type's
        // lowest value, 516 -> 183 us; rows without a mask 131 -> 134)
        if (__popc(__ballot_sync(0xffffffffu, own == b)) > PARTS - KMAX) {
          if (b > -INFINITY) { lo = fmaxf(lo, above(b)); skipped = fmaxf(skipped, b); }
          next_cut = it + 1;
          span = 1;
        }
      } else if (it == steps && span != 3 * FIRST_CUT) {  // after a cut: single ones lie before or behind the others, an equal one may be earlier
        const unsigned long long last = sh.list[K - 1];   // (not written since the last cut)
        if (last) lo = value_of(last);
      }
      if (m >= lo) {
#pragma unroll
        for (int g = 0; g < PER / 8; ++g) {
          if (q[g] >= lo) {
#pragma unroll
            for (int j = 8 * g; j < 8 * g + 8; ++j)
              if (x[j] >= lo) {
                const int i = it < steps ? head + (at + (j / N) * THREADS) * N + j % N : j == 0 ? t : a.V - n_tail + t;
                const int to = atomicAdd(&sh.n, 1);
                if (to < LIST) sh.list[to] = key_of(x[j], i);
              }
          }
        }
      }
      if (it + 1 == next_cut || it + 1 == all_steps) {
        __syncthreads();
        const int n = sh.n;
        overflow |= n > LIST;                             // (the same for all; the list is of no use from here on)
        next_cut = it + 1 + span;
        span = bound_at == it ? span : 4 * span;
        if (overflow) {
          lo = INFINITY;                                  // (nothing more is listed)
        } else {
          cut(sh.list, n, K, &sh.n);
          const unsigned long long last = sh.list[K - 1];
          if (last) lo = above(value_of(last));
          else bound_at = it + 1;                         // (as good as all banned so far)
        }
      }
    }
  }
  // ---- the CTA's sums and list, the slower ways
  const int e0 = rank == 0 ? 0 : head + p0 * N, e1 = rank == cs - 1 ? a.V : head + p1 * N;
  bool rare = __syncthreads_or(sum.rare);
  if (skipped > -INFINITY && !overflow) {                 // (the same for all, the list in order)
    const unsigned long long last = sh.list[K - 1];
    overflow = !(last && value_of(last) > skipped);
  }
  if (overflow) best_slowly(base, e0, e1, K, &sh);
  Sums all;                                               // of the CTA, then of the row: warp 0 has them
  if (!rare) {
    Sums32 x = {sum.base, sum.s, sum.w};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = joined(x, shfl_xor(x, o));
    if (lane == 0) sh.sums[warp] = x;
    __syncthreads();
    x = sh.sums[lane & (WARPS - 1)];
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) x = joined(x, shfl_xor(x, o));
    all = {x.s == 0.f ? 0.0 : (double)x.base, x.s, x.w};
    // low ones were left out: right where the sum is of others (what is missing is 2^-255 of it)
    if (!(x.s != 0.f && x.base >= 256.f - SMALL)) rare = __syncthreads_or(x.s != 0.f || sum.base == -FLT_MAX);
  }
  if (rare) {
    all = careful(base, e0, e1, a.c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) all = joined(all, shfl_xor(all, o));
    if (lane == 0) sh.careful_sums[warp] = all;
    __syncthreads();
    all = sh.careful_sums[lane & (WARPS - 1)];
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) all = joined(all, shfl_xor(all, o));
  }
  unsigned long long best = t < K && all_steps > 0 ? sh.list[t] : 0ull;
  if (cs > 1) {
    // every CTA hands its results to the first
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    cg::cluster_group cluster = cg::this_cluster();
    if (t == 0) *cluster.map_shared_rank(&sh.part[rank], 0) = all;
    if (t < K) *cluster.map_shared_rank(&sh.best[rank * K + t], 0) = best;
    cluster.sync();
    if (rank != 0) return;
    if (warp == 0) {
      all = lane < cs ? sh.part[lane] : Sums{0.0, 0.f, 0.f};
#pragma unroll
      for (int o = MAX_CLUSTER / 2; o > 0; o >>= 1) all = joined(all, shfl_xor(all, o));
    }
    if (K > 0) {
      cut(sh.best, cs * K, K, &sh.n);
      if (t < K) best = sh.best[t];
    }
  }
  // ---- the row's results.  A row without a finite logit: s = 0, every log-probability -inf, entropy 0.
  if (t == 0) {
    const bool any = all.s > 0.f;
    const double ln_s = any ? log((double)all.s) : 0.0;
    // the base as a logit: with it the factor's rounding touches differences alone
    const double ref = all.base / (double)a.c;            // (the careful way's is a logit times c: exact)
    sh.any = any;
    sh.ln_s = ln_s;
    sh.ref = ref;
    if (a.out_lse) a.out_lse[row] = any ? (float)(ref * a.inv_t + ln_s) : -INFINITY;
    if (a.out_entropy) a.out_entropy[row] = any ? fmaxf((float)(ln_s - (double)(all.w / all.s) * 0.69314718055994530942), 0.f) : 0.f;
  }
  __syncthreads();
  const bool any = sh.any;
  const double ref = sh.ref, ln_s = sh.ln_s;
  auto logp = [&](float x) {                              // (a best one's own power may come out a rounding above 1)
    if (!any || !(fabsf(x) < INFINITY)) return -INFINITY;
    return fminf((float)(((double)x - ref) * a.inv_t - ln_s), 0.f);
  };
  if (t < K) {
    a.out_top[(size_t)row * K + t] = best ? token_of(best) : -1;
    a.out_top_logp[(size_t)row * K + t] = best ? logp(value_of(best)) : -INFINITY;
  }
  // ---- the given tokens of this row; what belongs to no row is the first row's
  auto token = [&](int i) {
    const int at = a.tokens[i];
    a.out_logp[i] = at < 0 ? 0.f : at < a.V ? logp(to_f(base[at])) : -INFINITY;
  };
  if (!a.token_rows) {
    if (t == 0 && row < a.n_tokens) token(row);
  } else {
    for (int i = t; i < a.n_tokens; i += THREADS) {
      const int of = a.token_rows[i];
      if (of == row) token(i);
      else if (row == 0 && (of < 0 || of >= a.rows)) a.out_logp[i] = of < 0 || a.tokens[i] < 0 ? 0.f : -INFINITY;
    }
  }
}

// How many clusters of 2^log_cs CTAs the device holds at once (a cluster's SMs are neighbours, so that fewer fit than their CTAs would)
template <typename T> int clusters_at_once(int log_cs) {
  static std::atomic<int> known[PerDeviceFlags::MAX_DEVICES][4];           // one more than the answer
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= PerDeviceFlags::MAX_DEVICES) return 0;
  int n = known[dev][log_cs].load(std::memory_order_relaxed);
  if (!n) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 1 << log_cs; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1 << log_cs);
    cfg.blockDim = dim3(THREADS);
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int most = 0;
    if (cudaOccupancyMaxActiveClusters(&most, k_token_logprobs<T>, &cfg) != cudaSuccess) return 0;
    known[dev][log_cs].store(n = most + 1, std::memory_order_relaxed);
  }
  return n - 1;
}
// CTAs per row: one step each at the least, and no more than are resident at once.  61 rows over 32000 bf16 tokens with the 10 best: 10.9, 9.8,
// 9.2 and 10.9 us with 1, 2, 4 and 8; one row over 128256 fp32 tokens 19.8, 15.0, 10.7, 8.8; 48 rows over 71943 bf16 tokens with the best one
// 10.7 with 8, 54 rows 14.5 (with 4 11.8).
template <typename T> int log_cluster_of(int rows, int vocab) {
  int log_cs = 0;
  while (1 << log_cs < MAX_CLUSTER && (long long)vocab > (long long)STEP << log_cs && rows <= clusters_at_once<T>(log_cs + 1)) ++log_cs;
  return log_cs;
}

}  // namespace

extern "C" int poss_token_logprobs(const void* logits, int64_t ld, int dtype, int rows, int vocab, float temperature,
                                   const int32_t* tokens, const int32_t* token_rows, int n_tokens, float* out_logp,
                                   float* out_lse, float* out_entropy, int topk, int32_t* out_top_tokens, float* out_top_logp,
                                   poss_stream stream) {
  if (dtype != POSS_FP32 && dtype != POSS_BF16) return POSS_E_INVALID;
  if (rows < 0 || vocab < 1 || n_tokens < 0 || topk < 0 || ld < vocab) return POSS_E_INVALID;
  if (!(temperature > 0.f) || !(temperature < INFINITY)) return POSS_E_INVALID;
  if (rows == 0) return n_tokens ? POSS_E_INVALID : POSS_OK;
  if (topk > POSS_MAX_TOPK || vocab > (1 << 28) || rows > (1 << 24) || n_tokens > (1 << 24)) return POSS_E_CAPACITY;
  const double c = 1.4426950408889634 / (double)temperature;
  if (!(c < 3e38) || !((float)c > 0.f)) return POSS_E_INVALID;
  if (!logits || (n_tokens && (!tokens || !out_logp)) || (topk && (!out_top_tokens || !out_top_logp))) return POSS_E_INVALID;
  if (!token_rows && n_tokens > rows) return POSS_E_INVALID;
  const int es = dtype == POSS_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es) return POSS_E_INVALID;
  // one row's results may be written while another's logits are read
  const size_t n_in = ((size_t)(rows - 1) * ld + vocab) * es, list = (size_t)rows * topk * 4;
  const struct { const void* p; size_t n; } out[5] = {{out_logp, n_tokens ? (size_t)n_tokens * 4 : 0}, {out_lse, (size_t)rows * 4},
                                                      {out_entropy, (size_t)rows * 4}, {out_top_tokens, list}, {out_top_logp, list}};
  for (int i = 0; i < 5; ++i) {
    if (overlap(out[i].p, out[i].n, logits, n_in) || overlap(out[i].p, out[i].n, tokens, (size_t)n_tokens * 4) ||
        overlap(out[i].p, out[i].n, token_rows, (size_t)n_tokens * 4))
      return POSS_E_INVALID;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return POSS_E_INVALID;
  }
  Args a;
  a.logits = logits; a.ld = ld; a.rows = rows; a.V = vocab; a.K = topk; a.n_tokens = n_tokens;
  a.c = (float)c; a.inv_t = 1.0 / (double)temperature;
  a.tokens = tokens; a.token_rows = token_rows;
  a.out_logp = out_logp; a.out_lse = out_lse; a.out_entropy = out_entropy;
  a.out_top = out_top_tokens; a.out_top_logp = out_top_logp;
  const int log_cs = dtype == POSS_BF16 ? log_cluster_of<bf16>(rows, vocab) : log_cluster_of<float>(rows, vocab), cs = 1 << log_cs;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cs; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)rows * cs);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cfg.attrs = at;
  cfg.numAttrs = cs > 1 ? 2 : 1;
  const cudaError_t e = dtype == POSS_BF16 ? cudaLaunchKernelEx(&cfg, k_token_logprobs<bf16>, a, log_cs)
                                           : cudaLaunchKernelEx(&cfg, k_token_logprobs<float>, a, log_cs);
  return e == cudaSuccess ? POSS_OK : POSS_E_CUDA;
}
