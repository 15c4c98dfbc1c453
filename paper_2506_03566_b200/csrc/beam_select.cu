// Selection step of a beam search over beams x vocabulary.
//
// One pass over the logits: a block streams a chunk of one beam's row into registers and leaves the chunk's maximum, its
// sum of exponentials and its K best (value, token); a second kernel forms each beam's log-sum-exp from the chunks and
// picks the K best of the group's beams x chunks x K candidates by score[beam] + (logit - lse), in 64 bits.  What bounds
// the first kernel is the read of the logits; the rest of its work per logit is kept to a few instructions:
//   a lower bound of the chunk's K-th best value comes for free with the maxima -- the least of K (8 or 16) maxima of
//   disjoint parts of the chunk has K values at or above it -- so only the values at or above that bound (a few dozen
//   of 8192 for logits in no order) are ever compared with one another.
#include "poss_internal.cuh"
#include "../../include/poss_paged.h"

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

template <typename T>
__global__ void __launch_bounds__(THREADS) k_beam_lists(BeamArgs a, const T* logits) {
  constexpr int N = Vec<T>::N, NV = PER / N;              // values per load, loads per thread
  __shared__ float s_max[16], s_sum[WARPS];
  __shared__ int s_count;
  __shared__ float s_val[MAX_CAND];
  __shared__ int s_tok[MAX_CAND];
  pdl_enter(POSS_K_BEAM_LISTS);
  const int row = blockIdx.y, chunk = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5, K = a.K;
  const float score = a.scores[row];
  if (!(fabsf(score) < INFINITY) || (a.finished && a.finished[row])) return;   // (the second kernel skips it too)
  // Chunks start on the 16-byte boundary at or below the row's first logit: every load but those at the row's two ends
  // is whole and aligned.
  const T* const base = logits + (size_t)row * a.V;
  const int shift = (int)((reinterpret_cast<uintptr_t>(base) & 15) / sizeof(T));
  float x[PER];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i0 = chunk * CHUNK + (j * THREADS + t) * N - shift;              // first token of this load
    if (i0 >= 0 && i0 + N <= a.V) {
      Vec<T>::get(__ldcs(reinterpret_cast<const uint4*>(base + i0)), x + j * N);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[j * N + e] = i0 + e >= 0 && i0 + e < a.V ? to_f(base[i0 + e]) : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    x[j] = finite_or_banned(x[j]);
    m = fmaxf(m, x[j]);
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
  // sum of exponentials below the chunk's maximum (an all-banned chunk: maximum -inf, sum 0)
  float sum = 0.f;
  if (mx > -INFINITY) {
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < PER; ++j) s4[j & 3] += expf(x[j] - mx);
    sum = (s4[0] + s4[1]) + (s4[2] + s4[3]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  // candidates: values at or above the bound (banned ones never)
  if (m >= bound && m > -INFINITY) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (x[j] >= bound && x[j] > -INFINITY) {
        const int at = atomicAdd(&s_count, 1);
        if (at < MAX_CAND) {
          s_val[at] = x[j];
          s_tok[at] = chunk * CHUNK + ((j / N) * THREADS + t) * N - shift + j % N;
        }
      }
    }
  }
  __syncthreads();
  const size_t list = (size_t)row * a.n_chunks + chunk;
  float* val = a.cval + list * K;
  int32_t* tok = a.ctok + list * K;
  if (t == 0) {
    float s = 0.f;
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
      for (int o = 0; o < n; ++o) r += before(s_val[o], s_tok[o], v, i);
      if (r < K) { val[r] = v; tok[r] = i; }
    }
    for (int r = n + t; r < K; r += THREADS) tok[r] = -1;
    return;
  }
  // Too many at or above the bound (equal logits by the hundred, or a part of the chunk banned): K rounds, each
  // taking the best value behind the last one taken.
  float lv = INFINITY;
  int li = -1;
  for (int r = 0; r < K; ++r) {
    float bv = -INFINITY;
    int bi = 0x7fffffff;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int i = chunk * CHUNK + ((j / N) * THREADS + t) * N - shift + j % N;
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
    if (t == 0) { val[r] = bv; tok[r] = bi; }             // (more than MAX_CAND >= K values: there is always one)
    lv = bv; li = bi;
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

// One block per group.  The chunks' lists are sorted: a warp takes lists in turn, and its K best come out of K rounds
// over the lanes' heads; the first warp does the same with the warps' results.
__global__ void __launch_bounds__(THREADS) k_beam_merge(BeamArgs a) {
  __shared__ double s_lse[KMAX];
  __shared__ int s_kind[KMAX];                            // 0: no continuation, 1: open, 2: finished
  __shared__ Cand s_best[WARPS][KMAX];
  pdl_enter(POSS_K_BEAM_MERGE);
  const int g = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5, K = a.K;
  for (int b = warp; b < K; b += WARPS) {
    const int row = g * K + b;
    const bool alive = fabsf(a.scores[row]) < INFINITY, done = a.finished && a.finished[row];
    double lse = 0.0;
    if (alive && !done) {
      float mx = -INFINITY;
      for (int c = lane; c < a.n_chunks; c += 32) mx = fmaxf(mx, a.cmax[(size_t)row * a.n_chunks + c]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      double s = 0.0;
      for (int c = lane; c < a.n_chunks; c += 32) {
        const float m = a.cmax[(size_t)row * a.n_chunks + c];
        if (m > -INFINITY) s += (double)a.csum[(size_t)row * a.n_chunks + c] * exp((double)m - (double)mx);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      lse = (double)mx + log(s);
    }
    if (lane == 0) {
      s_lse[b] = lse;
      s_kind[b] = !alive ? 0 : done ? 2 : 1;
    }
  }
  __syncthreads();
  // entry e of the group: beam e / (n_chunks * K), then chunk, then place in the chunk's list
  const int per_beam = a.n_chunks * K, total = K * per_beam;
  auto entry = [&](int e) {
    Cand c;
    c.s = 0.0; c.tok = -1;
    c.beam = e / per_beam;
    const int i = e - c.beam * per_beam, row = g * K + c.beam;
    const int kind = s_kind[c.beam];
    if (kind == 1) {
      c.tok = a.ctok[(size_t)row * per_beam + i];
      c.s = (double)a.scores[row] + ((double)a.cval[(size_t)row * per_beam + i] - s_lse[c.beam]);
      if (c.tok < 0) c.beam = -1;
    } else if (kind == 2 && i == 0) {
      c.tok = a.eos;
      c.s = (double)a.scores[row];
    } else {
      c.beam = -1;
    }
    return c;
  };
  Cand last;                                              // the warp's last one taken; beam -1: none yet
  last.beam = -1; last.s = 0.0; last.tok = -1;
  for (int r = 0; r < K; ++r) {
    Cand best;
    best.beam = -1; best.s = 0.0; best.tok = -1;
    for (int e = t; e < total; e += THREADS) {
      const Cand c = entry(e);
      if ((last.beam < 0 || better(last, c)) && better(c, best)) best = c;
    }
    best = warp_best(best);
    if (lane == 0) s_best[warp][r] = best;
    if (best.beam < 0) {                                  // nothing left in this warp's share
      for (int q = r + 1; q < K; ++q)
        if (lane == 0) s_best[warp][q] = best;
      break;
    }
    last = best;
  }
  __syncthreads();
  if (warp > 0) return;
  // lane w < WARPS walks warp w's list
  int head = 0;
  for (int r = 0; r < K; ++r) {
    Cand c;
    c.beam = -1; c.s = 0.0; c.tok = -1;
    if (lane < WARPS && head < K) c = s_best[lane][head];
    const Cand best = warp_best(c);
    if (c.beam >= 0 && c.beam == best.beam && c.tok == best.tok) ++head;
    if (lane == 0) {
      const int o = g * K + r;
      if (best.beam < 0) {
        a.out_tokens[o] = -1; a.out_parents[o] = -1; a.out_scores[o] = -INFINITY; a.out_finished[o] = 1;
      } else {
        a.out_tokens[o] = best.tok;
        a.out_parents[o] = g * K + best.beam;
        a.out_scores[o] = (float)best.s;
        a.out_finished[o] = s_kind[best.beam] == 2 || best.tok == a.eos;
      }
    }
  }
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
// one chunk more than the row fills: the row's first logit may lie behind a 16-byte boundary
int chunks_of(int vocab) { return (vocab + 7 + CHUNK - 1) / CHUNK; }

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
