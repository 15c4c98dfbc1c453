// The attention weight that every slot of a paged cache draws, added up over rows and calls.
//
//   mass[head][s] (+)= sum over rows r, query heads h of the KV head: w_r 2^(scale s(r, h, s) - m(r, h)) / l(r, h)
//
// with the reference maximum m and the sum l that the attention of the same call leaves behind (paged_attention.cu).  A committed slot
// is added to, a slot of the call's own rows is set: it has no weight from before.  A slot belongs to one thread, which adds its terms
// in one order: no atomics, equal calls give equal bits.
#include "paged_attention.cuh"

POSS_TRACE_REGISTER()

namespace {

constexpr int QB = 32, KB = 32;

template <typename T> __device__ __forceinline__ float4 load4(const T* p);
template <> __device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <> __device__ __forceinline__ float4 load4<bf16>(const bf16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const float2 lo = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w.x));
  const float2 hi = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w.y));
  return make_float4(lo.x, lo.y, hi.x, hi.y);
}

// SIMT kernel, every type and shape, where scores were not kept (a scale of 0 or below on a shape of the tensor cores, a table with room for
// too many slots): a block owns 32 slots of one (sequence, KV head), keeps their keys in shared memory and walks the
// query rows (row * G + head) 32 at a time; a thread forms 2 rows x 4 slots of the scores, a thread per slot adds the rows' weights up.
// Bound by fp32 multiply-adds and the shared-memory reads that feed them.
template <typename T, int D>
__global__ void __launch_bounds__(128) k_slot_mass(PagedMassArgs s, const T* pool) {
  constexpr int LD = D + 4;                               // rows of 8 consecutive keys fall into different banks
  __shared__ __align__(16) float sq[QB][LD], sk[KB][LD];
  __shared__ float sp[QB][KB + 1], s_m[QB], s_w[QB];
  __shared__ unsigned s_seen[QB];
  __shared__ long long s_at[KB];                          // element offset of a slot's key, -1: none
  pdl_enter(POSS_K_SLOT_MASS);
  const PagedAttnArgs& a = s.a;
  const int b = blockIdx.z, kvh = blockIdx.y, key0 = blockIdx.x * KB;
  const int t = threadIdx.x, ty = t >> 3, tx = t & 7;
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows, (long long)a.g.max_pages * a.g.page);
  const int total = n.prefix + n.rows, nq = n.rows * a.G;
  if (key0 >= total || nq == 0) return;                   // (without rows nothing is added)
  if (t < KB) {
    const int key = key0 + t;
    long long at = -1;
    if (key < total) {
      const int p = page_at(a.g.tables + (size_t)b * a.g.max_pages, a.g.max_pages, a.g.n_pages, key / a.g.page);
      if (p >= 0) at = (long long)(page_offset(a.g, a.layer, p, 0, kvh) + (size_t)(key % a.g.page) * D);
    }
    s_at[t] = at;
  }
  __syncthreads();
  for (int e = t; e < KB * (D / 4); e += 128) {
    const int row = e / (D / 4), c = (e - row * (D / 4)) * 4;
    *reinterpret_cast<float4*>(&sk[row][c]) = s_at[row] >= 0 ? load4<T>(pool + s_at[row] + c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const uint32_t have = __ballot_sync(0xffffffffu, s_at[t & 31] >= 0);
  const T* q = reinterpret_cast<const T*>(a.q);
  float sum = 0.f;                                        // thread t < 32: of slot key0 + t
  for (int q0 = 0; q0 < nq; q0 += QB) {
    __syncthreads();                                      // the last rows have been read
    for (int e = t; e < QB * (D / 4); e += 128) {
      const int row = e / (D / 4), c = (e - row * (D / 4)) * 4, qi = q0 + row;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (qi < nq) {
        const int r = qi / a.G;
        v = load4<T>(q + ((size_t)b * a.rows + r) * a.ld_q + (size_t)(kvh * a.G + qi - r * a.G) * D + c);
      }
      *reinterpret_cast<float4*>(&sq[row][c]) = v;
    }
    if (t < QB) {
      const int qi = q0 + t;
      float2 ml = make_float2(INFINITY, 0.f);
      float w = 0.f;
      uint32_t seen = 0;
      if (qi < nq) {
        const int r = qi / a.G;
        const size_t row = (size_t)b * a.rows + r;
        ml = a.ml[row * a.Hq + kvh * a.G + qi - r * a.G];
        w = s.weights ? s.weights[row] : 1.f;
        uint64_t lo, hi;
        paged_row_mask(a.mask, row, a.mask_words, n.rows, &lo, &hi);
        seen = paged_visible32(key0, n.prefix, lo, hi) & have;
      }
      s_m[t] = ml.x;
      s_w[t] = w * ml.y;
      s_seen[t] = seen;
    }
    __syncthreads();
    float x[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 8
    for (int c = 0; c < D; c += 4) {
      float4 qv[2], kv[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) qv[i] = *reinterpret_cast<const float4*>(&sq[2 * ty + i][c]);
#pragma unroll
      for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(&sk[tx + 8 * j][c]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[i][j] = fmaf(qv[i].x, kv[j].x, x[i][j]);
          x[i][j] = fmaf(qv[i].y, kv[j].y, x[i][j]);
          x[i][j] = fmaf(qv[i].z, kv[j].z, x[i][j]);
          x[i][j] = fmaf(qv[i].w, kv[j].w, x[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int row = 2 * ty + i;
        const bool on = (s_seen[row] >> (tx + 8 * j)) & 1u;
        sp[row][tx + 8 * j] = on ? exp2f(fmaf(x[i][j], s.scale_log2, -s_m[row])) * s_w[row] : 0.f;
      }
    __syncthreads();
    if (t < KB) {
#pragma unroll 8
      for (int row = 0; row < QB; ++row) sum += sp[row][t];
    }
  }
  if (t < KB && key0 + t < total) {
    float* m = s.mass + ((size_t)b * a.g.Hkv + kvh) * s.mass_slots + key0 + t;
    *m = key0 + t < n.prefix ? *m + sum : sum;
  }
}

// From the scores that the attention has left: a block owns 32 slots of one (sequence, KV head), a warp takes every eighth line, a lane a slot;
// the warps' sums meet in shared memory.  Bound by the read of the scores, and for few rows by a chain of trips.
constexpr int WARPS = 8;
__global__ void __launch_bounds__(32 * WARPS) k_slot_mass_scores(PagedMassArgs s, long long ld) {
  __shared__ float part[WARPS][32];
  pdl_enter(POSS_K_SLOT_MASS);
  const PagedAttnArgs& a = s.a;
  const int b = blockIdx.z, kvh = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows, (long long)a.g.max_pages * a.g.page);
  const int total = n.prefix + n.rows, lines = n.rows * a.G;
  if (lines == 0) return;                                 // (without rows nothing is added)
  const float* const scores = s.scores + ((size_t)b * a.g.Hkv + kvh) * a.rows * a.G * ld;
  float* const mass = s.mass + ((size_t)b * a.g.Hkv + kvh) * s.mass_slots;
  for (int key0 = blockIdx.x * 32; key0 < total; key0 += gridDim.x * 32) {
    const int key = key0 + lane;                          // (scores have room for whole tiles of 32 slots)
    const float old = warp == 0 && key < n.prefix ? mass[key] : 0.f;
    float sum = 0.f;
#pragma unroll 4
    for (int i = warp; i < lines; i += WARPS) {
      const size_t row = (size_t)b * a.rows + i / a.G;
      const float2 ml = a.ml[row * a.Hq + kvh * a.G + i % a.G];
      const float w = s.weights ? s.weights[row] * ml.y : ml.y, x = __ldcg(scores + i * ld + key);
      sum += x == -INFINITY ? 0.f : exp2f(x - ml.x) * w;  // (unseen: nothing, even where the row's sum is NaN)
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && key < total) {
#pragma unroll
      for (int i = 1; i < WARPS; ++i) sum += part[i][lane];
      mass[key] = old + sum;
    }
    __syncthreads();
  }
}

template <typename T, int D> void launch_simt(Launcher& L, const PagedMassArgs& s, const void* pool) {
  const long long slots = (long long)s.a.g.max_pages * s.a.g.page;
  launch_pdl(L, k_slot_mass<T, D>, dim3((unsigned)((slots + KB - 1) / KB), s.a.g.Hkv, s.a.batch), dim3(128), 0, s,
             reinterpret_cast<const T*>(pool));
}

}  // namespace

void launch_paged_mass_scores(Launcher& L, const PagedMassArgs& s) {
  // some sixteen blocks per SM in all, each with 32 slots at least
  const long long items = (long long)s.a.batch * s.a.g.Hkv, ld = paged_simt_scores_ld(s.a.g.max_pages, s.a.g.page);
  const long long n = (16 * current_sm_count() + items - 1) / items, most = ld / 32;
  launch_pdl(L, k_slot_mass_scores, dim3((unsigned)(n < most ? n : most), s.a.g.Hkv, s.a.batch), dim3(32 * WARPS), 0, s, ld);
}

void launch_paged_mass_simt(Launcher& L, const PagedMassArgs& s, const void* pool, int dtype) {
  const bool h = dtype == POSS_BF16;
  switch (s.a.g.d) {
    case 32: h ? launch_simt<bf16, 32>(L, s, pool) : launch_simt<float, 32>(L, s, pool); break;
    case 64: h ? launch_simt<bf16, 64>(L, s, pool) : launch_simt<float, 64>(L, s, pool); break;
    default: h ? launch_simt<bf16, 128>(L, s, pool) : launch_simt<float, 128>(L, s, pool); break;
  }
}
