// Log-probabilities of given tokens, with each row's entropy and best tokens, over a vocabulary.
//
//   p = softmax(x / T);  log p(token);  H = -sum p log p;  the K best tokens with log p
//
// One pass over the logits and one launch: a row belongs to a cluster of 1 to 8 CTAs, a warp of which streams 1024 logits at a time.
// A thread keeps s = sum 2^t and w = sum t 2^t, t = (x - ref) log2(e) / T, against a reference of its own that moves only when a
// logit lies far above it; at the end
//   log sum e^(x / T) = ref / T + ln s,  H = ln 2 (log2 s - w / s).
// The K best: a warp keeps its K best in order, one per lane, and takes in what is above the K-th and at or above the K-th of any other
// warp of the CTA (a warp with K values there proves that nothing below can be among the best).  The first logits' bound is the K-th
// best of the lanes' maxima.  Warps', then CTAs' lists are joined by counting, for each entry, those before it.
// What bounds it: the read of the logits; for few rows the latency of a cluster's trips (part of the row, lists, lists of the others).
#include "paged.cuh"
#include <cooperative_groups.h>
#include <float.h>

POSS_TRACE_REGISTER()

namespace {

namespace cg = cooperative_groups;

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int PER = 32;                      // logits of a thread and step
constexpr int STEP = THREADS * PER;
constexpr int KMAX = POSS_MAX_TOPK;
constexpr int MAX_CLUSTER = 8;
constexpr float MOVE_LOG2 = 16.f;            // how far t may rise above the reference: sums stay far below fp32's range

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
__device__ __forceinline__ float min3(float a, float b, float c) {
  float d;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// (value, index): greater value first, then lower index
__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }
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

// sums against a reference (ref -inf: nothing yet, s = w = 0)
struct Sums { float ref, s, w; };
__device__ __forceinline__ Sums moved(Sums a, float ref, float c) {      // to a reference that is not below it
  if (a.s == 0.f) { a.ref = ref; return a; }
  const float d = fmaxf((a.ref - ref) * c, -200.f), f = ex2(d);          // (2^-200 is 0, and 0 times a finite number)
  a.w = f * fmaf(a.s, d, a.w);
  a.s *= f;
  a.ref = ref;
  return a;
}
__device__ __forceinline__ Sums joined(Sums a, Sums b, float c) {
  const float ref = fmaxf(a.ref, b.ref);
  a = moved(a, ref, c);
  b = moved(b, ref, c);
  a.s += b.s;
  a.w += b.w;
  return a;
}

struct Shared {
  volatile float bound[WARPS];               // each warp's K-th best so far
  Sums sums[WARPS];
  float val[WARPS * KMAX];                   // the warps' lists, then the CTAs'
  int tok[WARPS * KMAX];
  // what the cluster's first CTA collects
  Sums part;
  float best_val[KMAX];
  int best_tok[KMAX];
};

// entries (val, tok) [0, n), token -1: none; the K best, in order, to out
__device__ __forceinline__ void best_of(const float* val, const int* tok, int n, int K, float* out_val, int* out_tok) {
  const int t = threadIdx.x;
  if (t < K) out_tok[t] = -1;
  __syncthreads();
  if (t < n && tok[t] >= 0) {
    const float v = val[t];
    const int i = tok[t];
    int r = 0;
#pragma unroll 8
    for (int o = 0; o < n; ++o) r += tok[o] >= 0 && before(val[o], tok[o], v, i);
    if (r < K) { out_val[r] = v; out_tok[r] = i; }
  }
  __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 4) k_token_logprobs(Args a, int cs) {
  constexpr int N = Vec<T>::N, PIECES = PER / N;
  __shared__ Shared sh;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, K = a.K;
  const int row = blockIdx.x / cs, rank = blockIdx.x - row * cs;
  if (lane == 0) sh.bound[warp] = -INFINITY;
  __syncthreads();
  pdl_enter(POSS_K_TOKEN_LOGPROBS);
  const T* const base = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld;
  // the row: single logits up to a 16-byte boundary, pieces of 16 bytes that the CTAs share, single logits
  const int head = min(a.V, (int)((16 - (reinterpret_cast<uintptr_t>(base) & 15)) & 15) / (int)sizeof(T));
  const int pieces = (a.V - head) / N, tail = a.V - head - pieces * N;
  const int p0 = (int)((long long)pieces * rank / cs), p1 = (int)((long long)pieces * (rank + 1) / cs);
  const int n_head = rank == 0 ? head : 0, n_tail = rank == cs - 1 ? tail : 0;
  const int steps = (p1 - p0 + THREADS * PIECES - 1) / (THREADS * PIECES), more = n_head + n_tail > 0;
  const uint4* const body = reinterpret_cast<const uint4*>(base + head);

  Sums sum = {-INFINITY, 0.f, 0.f};
  float lv = -INFINITY;                      // the lane's entry of the warp's list
  int li = 0x7fffffff;
  const float2 c2 = make_float2(a.c, a.c);
#pragma unroll 1
  for (int it = 0; it < steps + more; ++it) {
    const bool single = it == steps;
    const int at = p0 + it * (THREADS * PIECES) + t;
    float x[PER];
    if (!single) {
      uint4 w[PIECES];
      const uint32_t none = N == 8 ? 0xff80ff80u : 0xff800000u;          // -inf
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
        w[i] = at + i * THREADS < p1 ? __ldcs(body + at + i * THREADS) : make_uint4(none, none, none, none);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) Vec<T>::get(w[i], x + i * N);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) x[i] = -INFINITY;
      if (t < n_head) x[0] = to_f(base[t]);
      if (t < n_tail) x[1] = to_f(base[a.V - n_tail + t]);
    }
    // maxima of fours; the thread's maximum and minimum.  (NaN and +inf show in the maximum.)
    float q[PER / 4], m, least;
    auto extremes = [&] {
#pragma unroll
      for (int j = 0; j < PER / 4; ++j) q[j] = max_nan(max_nan(x[4 * j], x[4 * j + 1], x[4 * j + 2]), x[4 * j + 3], x[4 * j + 3]);
      m = max_nan(max_nan(q[0], q[1], q[2]), max_nan(q[3], q[4], q[5]), max_nan(q[6], q[7], q[7]));
      least = x[0];
#pragma unroll
      for (int j = 1; j < PER - 1; j += 2) least = min3(least, x[j], x[j + 1]);
      least = fminf(least, x[PER - 1]);
    };
    extremes();
    if (!(m < INFINITY)) {
#pragma unroll
      for (int j = 0; j < PER; ++j) x[j] = fabsf(x[j]) < INFINITY ? x[j] : -INFINITY;
      extremes();
    }
    if (m > -INFINITY) {
      if (!((m - sum.ref) * a.c <= MOVE_LOG2)) sum = moved(sum, m, a.c);
      const float2 off = make_float2(-sum.ref, -sum.ref), zero = make_float2(0.f, 0.f);
      float2 s0 = zero, s1 = zero, w0 = zero, w1 = zero;
      // (differences first: logits of any finite size are safe, and those that count are near the reference)
      if ((least - sum.ref) * a.c > -1e30f) {
#pragma unroll
        for (int j = 0; j < PER; j += 4) {
          const float2 u = fma2(add2(make_float2(x[j], x[j + 1]), off), c2, zero), v = fma2(add2(make_float2(x[j + 2], x[j + 3]), off), c2, zero);
          const float2 eu = make_float2(ex2(u.x), ex2(u.y)), ev = make_float2(ex2(v.x), ex2(v.y));
          s0 = add2(s0, eu);
          s1 = add2(s1, ev);
          w0 = fma2(eu, u, w0);
          w1 = fma2(ev, v, w1);
        }
      } else {                                            // banned logits, or some beyond all measure: their power is 0
#pragma unroll
        for (int j = 0; j < PER; j += 2) {
          const float2 u = make_float2(fmaxf((x[j] - sum.ref) * a.c, -200.f), fmaxf((x[j + 1] - sum.ref) * a.c, -200.f));
          const float2 e = make_float2(ex2(u.x), ex2(u.y));
          s0 = add2(s0, e);
          w0 = fma2(e, u, w0);
        }
      }
      sum.s += (s0.x + s0.y) + (s1.x + s1.y);
      sum.w += (w0.x + w0.y) + (w1.x + w1.y);
    }
    if (K > 0) {
      // what may be among the best: at or above `lo`
      float own = __shfl_sync(0xffffffffu, lv, K - 1);
      float others = -INFINITY;
      if (lane < WARPS) others = sh.bound[lane];
#pragma unroll
      for (int o = WARPS / 2; o > 0; o >>= 1) others = fmaxf(others, __shfl_xor_sync(0xffffffffu, others, o));
      others = __shfl_sync(0xffffffffu, others, 0);
      // (places rise from step to step: a later one has to be greater, but for the single logits)
      float lo = fmaxf(single ? fmaxf(own, -FLT_MAX) : above(own), others);
      if (__any_sync(0xffffffffu, m >= lo)) {
        if (own == -INFINITY) {
          // the K-th best of the lanes' maxima
          int r = 0;
#pragma unroll 4
          for (int o = 0; o < 32; ++o) r += before(__shfl_sync(0xffffffffu, m, o), o, m, lane);
          const unsigned who = __ballot_sync(0xffffffffu, r == K - 1);
          lo = fmaxf(lo, __shfl_sync(0xffffffffu, m, __ffs(who) - 1));
        }
#pragma unroll
        for (int j4 = 0; j4 < PER / 4; ++j4) {
          if (!__any_sync(0xffffffffu, q[j4] >= lo)) continue;
#pragma unroll
          for (int j = 4 * j4; j < 4 * j4 + 4; ++j) {
            unsigned who = __ballot_sync(0xffffffffu, x[j] >= lo);
            const int i = single ? (j == 0 ? t : a.V - n_tail + t) : head + (at + (j / N) * THREADS) * N + j % N;
            while (who) {
              const int from = __ffs(who) - 1;
              who &= who - 1;
              const float v = __shfl_sync(0xffffffffu, x[j], from);
              const int vi = __shfl_sync(0xffffffffu, i, from);
              const int pos = __popc(__ballot_sync(0xffffffffu, before(lv, li, v, vi)));
              const float uv = __shfl_up_sync(0xffffffffu, lv, 1);
              const int ui = __shfl_up_sync(0xffffffffu, li, 1);
              if (lane == pos) { lv = v; li = vi; }
              else if (lane > pos) { lv = uv; li = ui; }
            }
          }
        }
        const float now = __shfl_sync(0xffffffffu, lv, K - 1);
        if (lane == 0) sh.bound[warp] = now;
      }
    }
  }
  // ---- the CTA's sums and list
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b;
    b.ref = __shfl_xor_sync(0xffffffffu, sum.ref, o);
    b.s = __shfl_xor_sync(0xffffffffu, sum.s, o);
    b.w = __shfl_xor_sync(0xffffffffu, sum.w, o);
    sum = joined(sum, b, a.c);
  }
  if (lane == 0) sh.sums[warp] = sum;
  if (lane < K) {
    sh.val[warp * K + lane] = lv;
    sh.tok[warp * K + lane] = lv > -INFINITY ? li : -1;
  }
  __syncthreads();
  sum = sh.sums[0];
#pragma unroll
  for (int w = 1; w < WARPS; ++w) sum = joined(sum, sh.sums[w], a.c);
  if (K > 0) best_of(sh.val, sh.tok, WARPS * K, K, sh.best_val, sh.best_tok);
  if (cs > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    if (t == 0) sh.part = sum;
    cluster.sync();
    if (rank == 0) {
      for (int i = 1; i < cs; ++i) sum = joined(sum, *cluster.map_shared_rank(&sh.part, i), a.c);
      if (t < cs * K) {
        const int from = t / K, e = t - from * K;
        sh.val[t] = *cluster.map_shared_rank(&sh.best_val[e], from);
        sh.tok[t] = *cluster.map_shared_rank(&sh.best_tok[e], from);
      }
    }
    cluster.sync();                                       // (the others stay until they have been read)
    if (rank != 0) return;
    if (K > 0) best_of(sh.val, sh.tok, cs * K, K, sh.best_val, sh.best_tok);
  }
  // ---- the row's results.  A row without a finite logit: s = 0, every log-probability -inf, entropy 0.
  const bool any = sum.s > 0.f;
  const double ln_s = any ? log((double)sum.s) : 0.0;
  auto logp = [&](float x) {                              // (a best one's own power may come out a rounding above 1)
    if (!any || !(fabsf(x) < INFINITY)) return -INFINITY;
    return fminf((float)(((double)x - (double)sum.ref) * a.inv_t - ln_s), 0.f);
  };
  if (t == 0) {
    if (a.out_lse) a.out_lse[row] = any ? (float)((double)sum.ref * a.inv_t + ln_s) : -INFINITY;
    if (a.out_entropy) a.out_entropy[row] = any ? fmaxf((float)(ln_s - (double)sum.w / (double)sum.s * 0.69314718055994530942), 0.f) : 0.f;
  }
  if (t < K) {
    const int i = sh.best_tok[t];
    a.out_top[(size_t)row * K + t] = i;
    a.out_top_logp[(size_t)row * K + t] = i >= 0 ? logp(sh.best_val[t]) : -INFINITY;
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
      else if (row == 0 && (of < 0 || of >= a.rows)) a.out_logp[i] = of < 0 ? 0.f : -INFINITY;
    }
  }
}

// CTAs per row: enough to fill the device where rows are few, at least a step's logits each
int cluster_of(int rows, int vocab) {
  int cs = 1;
  while (cs < MAX_CLUSTER && (long long)rows * cs * 2 <= 4 * 148 && (long long)vocab >= (long long)STEP * cs * 2) cs *= 2;
  return cs;
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
  const int cs = cluster_of(rows, vocab);
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
  const cudaError_t e = dtype == POSS_BF16 ? cudaLaunchKernelEx(&cfg, k_token_logprobs<bf16>, a, cs)
                                           : cudaLaunchKernelEx(&cfg, k_token_logprobs<float>, a, cs);
  return e == cudaSuccess ? POSS_OK : POSS_E_CUDA;
}
