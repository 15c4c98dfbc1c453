// Selection step of a beam search over beams x vocabulary.
//
// One pass over the logits: a block streams a chunk of one beam's row into registers and leaves the chunk's maximum, its
// sum of exponentials and its K best (value, token); a second kernel forms each beam's log-sum-exp from the chunks and
// picks the K best of the group's beams x chunks x K candidates by score[beam] + (logit - lse), in 64 bits.  What bounds
// the first kernel is the read of the logits; the rest of its work per logit is kept to a few instructions:
//   a lower bound of the chunk's K-th best value comes for free with the maxima -- the least of K (8 or 16) maxima of
//   disjoint parts of the chunk has K values at or above it -- so only the values at or above that bound (a few dozen
//   of 8192 for logits in no order) are ever compared with one another.
// Measured (fp32, in a captured graph): 32 groups of 8 beams over 128256 tokens, 131 MB, 43 us: 31 the first kernel (4.2 TB/s; the
// registers of a chunk allow 4 blocks per SM, whose reductions and compares leave the memory idle a third of the time), 12 the
// second, a chain of trips to memory and barriers in 32 blocks.  (A finished beam's logits are not read: with 13 % of them 114 MB,
// 28 and 12 us.)  4 beams over 32000 tokens: 10.4 us, 4.2 and 6.2.  The chunks stay at 8192 there too: with 2048 it took 8.4 for
// 10.0, but 8 beams over 128256 12.2 for 9.8, since the second kernel's lists grow.
#include "paged.cuh"
#include <float.h>

POSS_TRACE_REGISTER()

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int CHUNK = 8192;                  // logits per block
constexpr int PER = CHUNK / THREADS;         // logits per thread
constexpr int MAX_CAND = 512;                // candidates of a chunk that are ranked against one another
constexpr int KMAX = POSS_MAX_TOPK;

struct BeamArgs {
  int batch, K, V, n_chunks, eos;
  const float* scores;
  const int32_t* finished;
  float *cmax, *csum;        // [batch * K][n_chunks]
  float* cval;               // [batch * K][n_chunks][K], best first; entries behind the chunk's last value: token -1
  int32_t* ctok;
  int32_t *out_tokens, *out_parents, *out_finished;
  float* out_scores;
};

__device__ __forceinline__ float finite_or_banned(float x) { return fabsf(x) < INFINITY ? x : -INFINITY; }
__device__ __forceinline__ float max_nan(float a, float b, float c) {   // NaN if one of them is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// (value, index): greater value first, then lower index
__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// 4 fp32 or 8 bf16 logits of 16 bytes
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

// Place in its chunk of a thread's j-th logit.  A whole chunk is read in pieces of 16 bytes; one that the row does not fill in
// single logits, dealt to all threads: parts of the block that get none would leave the selection without a bound (4 beams over
// 1000 bf16 tokens 16.5 us, in pieces, against 8.5).  So are all chunks where
// rows start between 16-byte boundaries (32 groups of 8 beams over 128255 tokens: fp32 44 us and bf16 45, over 128256 42 and 38).
template <typename T> __device__ __forceinline__ int place(bool filled, int j) {
  constexpr int N = Vec<T>::N;
  return filled ? ((j / N) * THREADS + (int)threadIdx.x) * N + j % N : j * THREADS + (int)threadIdx.x;
}
// the thread's logits of a chunk; places outside the row count as banned
template <typename T>
__device__ __forceinline__ void load_chunk(const T* base, int V, int first, bool filled, float (&x)[PER]) {
  constexpr int N = Vec<T>::N;
  if (filled) {
#pragma unroll
    for (int j = 0; j < PER / N; ++j)
      Vec<T>::get(__ldcs(reinterpret_cast<const uint4*>(base + first + (j * THREADS + (int)threadIdx.x) * N)), x + j * N);
  } else {
    const int at = first + (int)threadIdx.x;
    const T* const p = base + at;                         // (place<T>(false, j) = j * THREADS + threadIdx.x)
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      x[j] = -INFINITY;
      if ((unsigned)(at + j * THREADS) < (unsigned)V) x[j] = to_f(p[j * THREADS]);
    }
  }
}

// Block (chunk, row).
template <typename T>
__global__ void __launch_bounds__(THREADS, 4) k_beam_lists(BeamArgs a, const T* logits) {
  __shared__ float s_max[16], s_sum[WARPS];
  __shared__ int s_count;
  __shared__ float s_val[MAX_CAND];
  __shared__ int s_tok[MAX_CAND];
  pdl_enter(POSS_K_BEAM_LISTS);
  const int row = blockIdx.y, t = threadIdx.x, lane = t & 31, warp = t >> 5, K = a.K;
  const float score = a.scores[row];
  if (!(fabsf(score) < INFINITY) || (a.finished && a.finished[row])) return;   // (the second kernel skips it too)
  // Which logits a thread takes goes by their place in the row alone, and not by where the row starts: beams that are alike
  // have the same sums to the last bit and tie.
  const T* const base = logits + (size_t)row * a.V;
  const int chunk = blockIdx.x, first = chunk * CHUNK;
  float x[PER];
  const bool filled = first + CHUNK <= a.V && a.V % Vec<T>::N == 0;
  load_chunk<T>(base, a.V, first, filled, x);
  // Maxima of fours and of the thread.  (-inf needs no care, +inf and NaN are rare: they show in the maximum.)
  float q[PER / 4], m = -INFINITY;
  auto maxima = [&] {
#pragma unroll
    for (int j = 0; j < PER / 4; ++j) q[j] = max_nan(max_nan(x[4 * j], x[4 * j + 1], x[4 * j + 2]), x[4 * j + 3], x[4 * j + 3]);
    m = max_nan(max_nan(q[0], q[1], q[2]), max_nan(q[3], q[4], q[5]), max_nan(q[6], q[7], q[7]));
  };
  static_assert(PER == 32, "eight fours");
  maxima();
  if (!(m < INFINITY)) {
#pragma unroll
    for (int j = 0; j < PER; ++j) x[j] = finite_or_banned(x[j]);
    maxima();
  }
  // maxima of the 16 half warps
  float mh = m;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) mh = fmaxf(mh, __shfl_xor_sync(0xffffffffu, mh, o));
  if ((lane & 15) == 0) s_max[t >> 4] = mh;
  if (t == 0) s_count = 0;
  __syncthreads();
  float mx = -INFINITY, bound = INFINITY;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    const float lo = s_max[2 * w], hi = s_max[2 * w + 1];
    mx = fmaxf(mx, fmaxf(lo, hi));
    bound = fminf(bound, K <= WARPS ? fmaxf(lo, hi) : fminf(lo, hi));
  }
  bound = fmaxf(bound, -FLT_MAX);                       // banned logits never reach it
  // candidates: values at or above the bound
  if (m >= bound) {
#pragma unroll
    for (int j4 = 0; j4 < PER; j4 += 4) {
      if (q[j4 / 4] >= bound) {
#pragma unroll
        for (int j = j4; j < j4 + 4; ++j) {
          if (x[j] >= bound) {
            const int at = atomicAdd(&s_count, 1);
            if (at < MAX_CAND) {
              s_val[at] = x[j];
              s_tok[at] = first + place<T>(filled, j);
            }
          }
        }
      }
    }
  }
  // Sum of exponentials below the chunk's maximum (an all-banned chunk: maximum -inf, sum 0).  The differences come first: the
  // maximum's own term is 1 exactly, so that no log-probability is above 0, and logits of any finite size (masks of -1e10, the type's
  // lowest value) are safe; those that count are near the maximum, where differences lose nothing, and one that overflows is -inf,
  // whose power is 0.  (2^(x log2 e - maximum log2 e) would be one operation less, but what the rounded second product leaves over
  // grows with it: from 2^31 on its power leaves fp32.)
  float sum = 0.f;
  if (mx > -INFINITY) {
    const float2 L2E = make_float2(1.4426950408889634f, 1.4426950408889634f), off = make_float2(-mx, -mx);
    float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
    for (int j = 0; j < PER; j += 4) {
      const float2 u = fma2(add2(make_float2(x[j], x[j + 1]), off), L2E, make_float2(0.f, 0.f));
      const float2 v = fma2(add2(make_float2(x[j + 2], x[j + 3]), off), L2E, make_float2(0.f, 0.f));
      s0 = add2(s0, make_float2(ex2(u.x), ex2(u.y)));   // 2^-22 relative
      s1 = add2(s1, make_float2(ex2(v.x), ex2(v.y)));
    }
    sum = (s0.x + s0.y) + (s1.x + s1.y);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  const size_t list = (size_t)row * a.n_chunks + chunk;
  float* val = a.cval + list * K;
  int32_t* tok = a.ctok + list * K;
  if (t == THREADS - 1) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += s_sum[w];
    a.cmax[list] = mx;
    a.csum[list] = s;
  }
  const int n = s_count;
  if (n <= MAX_CAND) {
    // the candidate with r others before it is the (r + 1)-th best (the order in which they were stored is of no
    // account: (value, token) pairs are all different)
    for (int c = t; c < n; c += THREADS) {
      const float v = s_val[c];
      const int i = s_tok[c];
      int r = 0;
#pragma unroll 4
      for (int o = 0; o < n; ++o) r += before(s_val[o], s_tok[o], v, i);
      if (r < K) { val[r] = v; tok[r] = i; }
    }
    for (int r = n + t; r < K; r += THREADS) tok[r] = -1;
  } else {
    // Too many at or above the bound (equal logits by the hundred, or a part of the chunk banned): K rounds, each
    // taking the best value behind the last one taken.
    float lv = INFINITY;
    int li = -1;
    for (int r = 0; r < K; ++r) {
      float bv = -INFINITY;
      int bi = 0x7fffffff, f = filled;
      asm volatile("" : "+r"(f));                         // (the places are worked out in each round, not kept for all)
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const int i = first + place<T>(f != 0, j);
        if (x[j] > -INFINITY && before(lv, li, x[j], i) && before(x[j], i, bv, bi)) { bv = x[j]; bi = i; }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, bv, o);
        const int i = __shfl_xor_sync(0xffffffffu, bi, o);
        if (before(v, i, bv, bi)) { bv = v; bi = i; }
      }
      __syncthreads();
      if (lane == 0) { s_val[warp] = bv; s_tok[warp] = bi; }
      __syncthreads();
      for (int w = 0; w < WARPS; ++w)
        if (before(s_val[w], s_tok[w], bv, bi)) { bv = s_val[w]; bi = s_tok[w]; }
      if (t == 0) { val[r] = bv; tok[r] = bi; }         // (more than MAX_CAND >= K values: there is always one)
      lv = bv; li = bi;
    }
  }
}

// (score, flat index beam * V + token), index -1: none
struct Cand { double s; int beam, tok; };
__device__ __forceinline__ bool better(const Cand& a, const Cand& b) {
  if (a.beam < 0) return false;
  if (b.beam < 0) return true;
  return a.s > b.s || (a.s == b.s && (a.beam < b.beam || (a.beam == b.beam && a.tok < b.tok)));
}
__device__ __forceinline__ Cand shfl_xor(const Cand& c, int o) {
  Cand r;
  r.s = __shfl_xor_sync(0xffffffffu, c.s, o);
  r.beam = __shfl_xor_sync(0xffffffffu, c.beam, o);
  r.tok = __shfl_xor_sync(0xffffffffu, c.tok, o);
  return r;
}
__device__ __forceinline__ Cand warp_best(Cand c) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Cand d = shfl_xor(c, o);
    if (better(d, c)) c = d;
  }
  return c;
}

// One block per group.  The chunks' lists are sorted, so a list whose head is worse than K other heads has nothing to give:
//   1  the heads are dealt to 8 (or 16) parts of the block; the least of the parts' best heads is a bound that K heads reach
//   2  the entries that reach it, from the front of each list (a few times K)
//   3  an entry with r better ones is the (r + 1)-th of the group
constexpr int MAX_ENTRIES = 1024;
constexpr int PRE = 4;                       // entries fetched ahead
__global__ void __launch_bounds__(THREADS) k_beam_merge(BeamArgs a) {
  __shared__ double s_lse[KMAX], s_score[KMAX];
  __shared__ int s_kind[KMAX];                            // 0: no continuation, 1: open, 2: finished
  __shared__ Cand s_head[16];
  __shared__ int s_n;
  __shared__ Cand s_entry[MAX_ENTRIES];
  __shared__ int s_pre_tok[PRE][THREADS];
  __shared__ float s_pre_val[PRE][THREADS];
  pdl_enter(POSS_K_BEAM_MERGE);
  const int g = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5, K = a.K;
  Cand none;
  none.s = 0.0; none.beam = -1; none.tok = -1;
  // Lists are dealt to the parts in turn: thread t takes lists l0, l0 + THREADS, ...  The first entries of its first list are on
  // their way while the sums are worked on: a group of few chunks is a chain of trips to memory and little else.
  const int lists = K * a.n_chunks, parts = K <= WARPS ? WARPS : 2 * WARPS;
  const int part = t / (THREADS / parts), l0 = (t % (THREADS / parts)) * parts + part;
  {
    int tok[PRE];
    float val[PRE];
#pragma unroll
    for (int i = 0; i < PRE; ++i) {
      const bool there = l0 < lists && i < K;
      const size_t at = ((size_t)g * lists + (there ? l0 : 0)) * K + (there ? i : 0);
      tok[i] = there ? a.ctok[at] : -1;
      val[i] = there ? a.cval[at] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < PRE; ++i) { s_pre_tok[i][t] = tok[i]; s_pre_val[i][t] = val[i]; }
  }
  for (int b = warp; b < K; b += WARPS) {
    const int row = g * K + b;
    const size_t c0 = (size_t)row * a.n_chunks;
    // (a beam without lists: whatever lies there is not used)
    const float score = a.scores[row], own_max = lane < a.n_chunks ? a.cmax[c0 + lane] : -INFINITY,
                own_sum = lane < a.n_chunks ? a.csum[c0 + lane] : 0.f;
    const bool alive = fabsf(score) < INFINITY, done = a.finished && a.finished[row];
    double lse = 0.0;
    if (alive && !done) {
      float mx = own_max;
      for (int c = lane + 32; c < a.n_chunks; c += 32) mx = fmaxf(mx, a.cmax[c0 + c]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      double s = own_max > -INFINITY ? (double)own_sum * exp((double)own_max - (double)mx) : 0.0;
      for (int c = lane + 32; c < a.n_chunks; c += 32) {
        const float m = a.cmax[c0 + c];
        if (m > -INFINITY) s += (double)a.csum[c0 + c] * exp((double)m - (double)mx);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      lse = (double)mx + log(s);
    }
    if (lane == 0) {
      s_lse[b] = lse;
      s_score[b] = (double)score;
      // (an open beam whose tokens are all banned has no finite sum)
      s_kind[b] = !alive ? 0 : done ? 2 : fabs(lse) < (double)INFINITY ? 1 : 0;
    }
  }
  if (t == 0) s_n = 0;
  __syncthreads();
  // entry i of list l (beam l / n_chunks); a finished beam has one, in its first list
  auto make = [&](int l, int i, int tok, float val) {
    Cand e = none;
    const int b = l / a.n_chunks;
    if (s_kind[b] == 1) {
      if (tok >= 0) {
        e.beam = b;
        e.tok = tok;
        e.s = s_score[b] + ((double)val - s_lse[b]);
      }
    } else if (s_kind[b] == 2 && l == b * a.n_chunks && i == 0) {
      e.beam = b;
      e.tok = a.eos;
      e.s = s_score[b];
    }
    return e;
  };
  auto entry = [&](int l, int i) {
    const size_t at = ((size_t)g * lists + l) * K + i;
    return make(l, i, a.ctok[at], a.cval[at]);            // (a beam without lists: whatever lies there is not looked at)
  };
  // ---- 1
  Cand head = l0 < lists ? make(l0, 0, s_pre_tok[0][t], s_pre_val[0][t]) : none;
  for (int l = l0 + THREADS; l < lists; l += THREADS) {
    const Cand e = entry(l, 0);
    if (better(e, head)) head = e;
  }
  for (int o = 1; o < THREADS / parts; o <<= 1) {
    const Cand d = shfl_xor(head, o);
    if (better(d, head)) head = d;
  }
  if (t % (THREADS / parts) == 0) s_head[part] = head;
  __syncthreads();
  Cand bound = s_head[lane & (parts - 1)];                // (a part without heads: no bound)
  for (int o = 1; o < parts; o <<= 1) {
    const Cand d = shfl_xor(bound, o);
    if (better(bound, d)) bound = d;
  }
  // ---- 2
  auto take = [&](const Cand& e) {
    if (e.beam < 0 || better(bound, e)) return false;     // (the list's next ones are worse)
    const int at = atomicAdd(&s_n, 1);                    // (the order of the entries is of no account: no two are equal)
    if (at < MAX_ENTRIES) s_entry[at] = e;
    return true;
  };
  if (l0 < lists) {
#pragma unroll 1
    for (int i = 0; i < K; ++i) {
      const size_t at = ((size_t)g * lists + l0) * K + i;
      if (!take(make(l0, i, i < PRE ? s_pre_tok[i][t] : a.ctok[at], i < PRE ? s_pre_val[i][t] : a.cval[at]))) break;
    }
  }
#pragma unroll 1
  for (int l = l0 + THREADS; l < lists; l += THREADS)
#pragma unroll 1
    for (int i = 0; i < K && take(entry(l, i)); ++i) {}
  __syncthreads();
  const int n = s_n;
  auto write = [&](int r, const Cand& e) {
    const int o = g * K + r;
    a.out_tokens[o] = e.beam < 0 ? -1 : e.tok;
    a.out_parents[o] = e.beam < 0 ? -1 : g * K + e.beam;
    a.out_scores[o] = e.beam < 0 ? -INFINITY : (float)e.s;
    a.out_finished[o] = e.beam < 0 || s_kind[e.beam] == 2 || e.tok == a.eos;
  };
  if (n <= MAX_ENTRIES) {
    // ---- 3
    // (a warp per entry, its lanes over the others: with a thread per entry the few dozen comparisons of 64 bits, one behind the
    // other, took 4 us of a call's 13)
    for (int c = warp; c < n; c += WARPS) {
      const Cand e = s_entry[c];
      int r = 0;
      for (int o = lane; o < n; o += 32) r += better(s_entry[o], e);
      r = __reduce_add_sync(0xffffffffu, r);
      if (lane == 0 && r < K) write(r, e);
    }
    for (int r = n + t; r < K; r += THREADS) write(r, none);
    return;
  }
  // Too many (a vocabulary of hundreds of chunks with equal logits): K rounds, each taking the best behind the last taken.
  Cand last = none;
  for (int r = 0; r < K; ++r) {
    Cand best = none;
    for (int l = t; l < lists; l += THREADS) {
      for (int i = 0; i < K; ++i) {
        const Cand e = entry(l, i);
        if (e.beam < 0) break;
        if (last.beam < 0 || better(last, e)) {
          if (better(e, best)) best = e;
          break;                                          // (the list's next ones are worse)
        }
      }
    }
    best = warp_best(best);
    __syncthreads();
    if (lane == 0) s_head[warp] = best;
    __syncthreads();
    for (int w = 0; w < WARPS; ++w)
      if (better(s_head[w], best)) best = s_head[w];
    if (t == 0) write(r, best);
    last = best;                                          // (more than MAX_ENTRIES >= K entries: there is always one)
  }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
int chunks_of(int vocab) { return (vocab + CHUNK - 1) / CHUNK; }

}  // namespace

extern "C" {

size_t poss_beam_select_workspace_bytes(int batch, int beams, int vocab) {
  if (batch < 1 || beams < 1 || vocab < 1 || beams > POSS_MAX_TOPK) return 0;
  if ((long long)batch * beams > 65535 || vocab > (1 << 28)) return 0;
  const size_t lists = (size_t)batch * beams * chunks_of(vocab);
  return 2 * round256(lists * 4) + 2 * round256(lists * beams * 4);
}

int poss_beam_select(const void* logits, int dtype, int batch, int beams, int vocab, const float* scores,
                     const int32_t* finished, int eos, int32_t* out_tokens, int32_t* out_parents, float* out_scores,
                     int32_t* out_finished, void* workspace, size_t workspace_bytes, poss_stream stream) {
  if (dtype != POSS_FP32 && dtype != POSS_BF16) return POSS_E_INVALID;
  if (batch < 0 || beams < 1 || vocab < 1 || eos >= vocab || (finished && eos < 0)) return POSS_E_INVALID;
  if (batch == 0) return POSS_OK;
  if (beams > POSS_MAX_TOPK || (long long)batch * beams > 65535 || vocab > (1 << 28)) return POSS_E_CAPACITY;
  if (!logits || !scores || !out_tokens || !out_parents || !out_scores || !out_finished) return POSS_E_INVALID;
  if (reinterpret_cast<uintptr_t>(logits) & 15) return POSS_E_INVALID;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
      workspace_bytes < poss_beam_select_workspace_bytes(batch, beams, vocab))
    return POSS_E_WORKSPACE;
  // in place or apart: a group's scores are read before they are written, another group's may not have been
  const size_t n = (size_t)batch * beams * 4;
  auto crossed = [&](const void* o, const void* in, bool in_place) { return overlap(o, n, in, n) && !(in_place && o == in); };
  const void* const outs[4] = {out_tokens, out_parents, out_scores, out_finished};
  for (int i = 0; i < 4; ++i) {
    if (crossed(outs[i], scores, i == 2) || crossed(outs[i], finished, i == 3)) return POSS_E_INVALID;
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], n, outs[j], n)) return POSS_E_INVALID;
  }
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  BeamArgs a;
  a.batch = batch; a.K = beams; a.V = vocab; a.n_chunks = chunks_of(vocab); a.eos = eos;
  a.scores = scores; a.finished = finished;
  const size_t lists = (size_t)batch * beams * a.n_chunks;
  char* w = reinterpret_cast<char*>(workspace);
  a.cmax = reinterpret_cast<float*>(w); w += round256(lists * 4);
  a.csum = reinterpret_cast<float*>(w); w += round256(lists * 4);
  a.cval = reinterpret_cast<float*>(w); w += round256(lists * beams * 4);
  a.ctok = reinterpret_cast<int32_t*>(w);
  a.out_tokens = out_tokens; a.out_parents = out_parents; a.out_finished = out_finished; a.out_scores = out_scores;
  const dim3 grid(a.n_chunks, batch * beams);
  if (dtype == POSS_BF16)
    launch_pdl(L, k_beam_lists<bf16>, grid, dim3(THREADS), 0, a, reinterpret_cast<const bf16*>(logits));
  else
    launch_pdl(L, k_beam_lists<float>, grid, dim3(THREADS), 0, a, reinterpret_cast<const float*>(logits));
  launch_pdl(L, k_beam_merge, dim3(batch), dim3(THREADS), 0, a);
  return L.err;
}

}  // extern "C"
