// Tree-masked attention over pages: the SIMT kernel (fp32 check mode, and the bf16 shapes that the tensor-core kernel
// does not take) and the C entry.
//
// The G = Hq / Hkv query heads of a KV head and the tree rows form one matrix of query rows (query row = row * G + head).
// A block owns 32 query rows of one (sequence, KV head) and every ns-th part of its keys, walks them 32 at a time and
// keeps a running maximum, sum and output in registers (one pass over the keys).  Four query rows of a warp share
// every key and value that it reads from shared memory; a thread holds 2 rows x 4 keys of the scores and 2 rows x d/8
// columns of the output.  With ns > 1 the parts are left in scratch and a second kernel merges them in key order.
// What bounds it: fp32 multiply-adds and the shared-memory reads that feed them for trees over long contexts (16 trees of 61
// rows over up to 8191 slots in bf16: 4.6 ms, the tensor-core kernel 0.15), the trips to memory of a 32-key step and of the merge for
// short ones (3 trees of 15 rows over up to 517 slots, fp32: 12.3 us).
#include "paged_attention.cuh"
#include <math.h>

POSS_TRACE_REGISTER()

namespace {

constexpr int QB = 32, KB = 32;

struct SimtArgs {
  PagedAttnArgs a;
  int q_tiles, ns;
  float scale_log2;
  float* part;      // [batch][Hkv][q_tiles][ns][QB][d + 2]: maximum, sum, outputs
};

template <typename T> __device__ __forceinline__ float4 load4(const T* p);
template <> __device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <> __device__ __forceinline__ float4 load4<bf16>(const bf16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  const float2 lo = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w.x));
  const float2 hi = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w.y));
  return make_float4(lo.x, lo.y, hi.x, hi.y);
}
template <typename T> __device__ __forceinline__ void store4(T* p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
template <> __device__ __forceinline__ void store4<bf16>(bf16* p, float4 v) {
  __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}

template <typename T, int D>
__global__ void __launch_bounds__(128) k_paged_attn(SimtArgs s, const T* pool) {
  constexpr int LD = D + 4;                               // rows of 8 consecutive keys fall into different banks
  constexpr int NV = D / 32;                              // float4 columns of the output per thread
  __shared__ __align__(16) float sq[QB][LD], skv[KB][LD];
  __shared__ float sp[QB][KB + 1];
  __shared__ long long s_at[KB];                          // element offset of a key's row in the pool, -1: none
  pdl_enter(POSS_K_PAGED_ATTN);
  const PagedAttnArgs& a = s.a;
  const int split = blockIdx.x, b = blockIdx.z, kvh = blockIdx.y / s.q_tiles, qt = blockIdx.y - kvh * s.q_tiles;
  const int t = threadIdx.x, ty = t >> 3, tx = t & 7;
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows,
                              (long long)a.g.max_pages * a.g.page);
  if (n.bad && t == 0) raise_status(a.status, POSS_E_INVALID);
  const int nq = n.rows * a.G;
  if (qt * QB >= nq) return;
  const int total = n.prefix + n.rows, tiles = (total + KB - 1) / KB;
  const int tile0 = (int)((long long)split * tiles / s.ns), tile1 = (int)((long long)(split + 1) * tiles / s.ns);
  const int32_t* table = a.g.tables + (size_t)b * a.g.max_pages;

  const T* q = reinterpret_cast<const T*>(a.q);
  for (int i = t; i < QB * (D / 4); i += 128) {
    const int row = i / (D / 4), c = (i - row * (D / 4)) * 4, qi = qt * QB + row;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (qi < nq) {
      const int r = qi / a.G;
      v = load4<T>(q + ((size_t)b * a.rows + r) * a.ld_q + (size_t)(kvh * a.G + qi - r * a.G) * D + c);
    }
    *reinterpret_cast<float4*>(&sq[row][c]) = v;
  }
  uint64_t lo[2] = {0, 0}, hi[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int qi = qt * QB + 2 * ty + i;
    if (qi < nq) paged_row_mask(a.mask, (size_t)b * a.rows + qi / a.G, a.mask_words, n.rows, &lo[i], &hi[i]);
  }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float4 o[2][NV];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int v = 0; v < NV; ++v) o[i][v] = make_float4(0.f, 0.f, 0.f, 0.f);

  // where a key's row lies: thread `t`'s key of a tile, asked for one tile ahead
  auto find = [&](int tile) {
    const int key = tile * KB + t;
    long long at = -1;
    if (t < KB && tile < tile1 && key < total) {
      const int p = page_at(table, a.g.max_pages, a.g.n_pages, key / a.g.page);
      if (p >= 0) at = (long long)(page_offset(a.g, a.layer, p, 0, kvh) + (size_t)(key % a.g.page) * D);
      else raise_status(a.status, POSS_E_INVALID);
    }
    return at;
  };
  constexpr int PER = KB * (D / 4) / 128;                 // pieces of four of a tile's keys, or values, per thread
  const size_t to_values = (size_t)a.g.Hkv * a.g.page * D;
  long long next_at = find(tile0);
  for (int tile = tile0; tile < tile1; ++tile) {
    const int key0 = tile * KB;
    __syncthreads();                                      // the last tile's values and probabilities have been read
    if (t < KB) s_at[t] = next_at;
    __syncthreads();
    next_at = find(tile + 1);
    // keys and values are on their way together; the values wait in registers for the keys' place
    float4 keys[PER], values[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = t + 128 * i, row = e / (D / 4), c = (e - row * (D / 4)) * 4;
      const long long at = s_at[row];
      keys[i] = values[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (at >= 0) {
        keys[i] = load4<T>(pool + at + c);
        values[i] = load4<T>(pool + at + to_values + c);
      }
    }
    auto store_rows = [&](const float4* v) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int e = t + 128 * i, row = e / (D / 4), c = (e - row * (D / 4)) * 4;
        *reinterpret_cast<float4*>(&skv[row][c]) = v[i];
      }
    };
    store_rows(keys);
    const bool partly = key0 + KB > n.prefix;             // some row may not see some key
    const uint32_t have = __ballot_sync(0xffffffffu, s_at[t & 31] >= 0);
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
      for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(&skv[tx + 8 * j][c]);
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
    uint32_t seen_any[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t seen = partly ? paged_visible32(key0, n.prefix, lo[i], hi[i]) & have : have;
      seen_any[i] = seen;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = (seen >> (tx + 8 * j)) & 1u ? x[i][j] * s.scale_log2 : -INFINITY;
        mx = fmaxf(mx, x[i][j]);
      }
#pragma unroll
      for (int d = 4; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
      const float mn = fmaxf(m[i], mx);
      const float off = mn == -INFINITY ? 0.f : mn;       // nothing seen so far: every 2^x below is 2^-inf = 0
      const float c = m[i] == mn ? 1.f : exp2f(m[i] - off);
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool on = (seen >> (tx + 8 * j)) & 1u;
        const float p = on ? exp2f(x[i][j] - off) : 0.f;
        sum += p;
        sp[2 * ty + i][tx + 8 * j] = p;
      }
#pragma unroll
      for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      l[i] = l[i] * c + sum;
      m[i] = mn;
#pragma unroll
      for (int v = 0; v < NV; ++v) { o[i][v].x *= c; o[i][v].y *= c; o[i][v].z *= c; o[i][v].w *= c; }
    }
    __syncthreads();                                      // the keys have been read
    store_rows(values);
    __syncthreads();
    // an unseen value takes no part, whatever it holds: 0 x inf would
    auto add = [&](int j, bool on0, bool on1) {
      const float p0 = sp[2 * ty][j], p1 = sp[2 * ty + 1][j];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const float4 w = *reinterpret_cast<const float4*>(&skv[j][tx * 4 + 32 * v]);
        if (on0) {
          o[0][v].x = fmaf(p0, w.x, o[0][v].x); o[0][v].y = fmaf(p0, w.y, o[0][v].y);
          o[0][v].z = fmaf(p0, w.z, o[0][v].z); o[0][v].w = fmaf(p0, w.w, o[0][v].w);
        }
        if (on1) {
          o[1][v].x = fmaf(p1, w.x, o[1][v].x); o[1][v].y = fmaf(p1, w.y, o[1][v].y);
          o[1][v].z = fmaf(p1, w.z, o[1][v].z); o[1][v].w = fmaf(p1, w.w, o[1][v].w);
        }
      }
    };
    if (__all_sync(0xffffffffu, (seen_any[0] & seen_any[1]) == 0xffffffffu)) {
#pragma unroll 8
      for (int j = 0; j < KB; ++j) add(j, true, true);
    } else {
#pragma unroll 1
      for (int j = 0; j < KB; ++j) add(j, (seen_any[0] >> j) & 1u, (seen_any[1] >> j) & 1u);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int qi = qt * QB + 2 * ty + i;
    if (qi >= nq) continue;
    if (s.ns == 1) {
      const int r = qi / a.G;
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];   // a row that sees nothing: zeros
      T* dst = reinterpret_cast<T*>(a.out) + (((size_t)b * a.rows + r) * a.Hq + kvh * a.G + qi - r * a.G) * D;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        store4<T>(dst + tx * 4 + 32 * v, make_float4(o[i][v].x * inv, o[i][v].y * inv, o[i][v].z * inv, o[i][v].w * inv));
    } else {
      float* dst = s.part + ((((size_t)b * gridDim.y + blockIdx.y) * s.ns + split) * QB + 2 * ty + i) * (D + 2);
      if (tx == 0) { dst[0] = m[i]; dst[1] = l[i]; }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float* p = dst + 2 + tx * 4 + 32 * v;
        p[0] = o[i][v].x; p[1] = o[i][v].y; p[2] = o[i][v].z; p[3] = o[i][v].w;
      }
    }
  }
}

constexpr int MAX_SPLITS = 64;
// merges the ns parts of a query row: one warp per query row, a lane per part's weight, then the outputs in key order
template <typename T, int D>
__global__ void __launch_bounds__(128) k_paged_attn_merge(SimtArgs s) {
  pdl_enter(POSS_K_PAGED_ATTN_COMBINE);
  const PagedAttnArgs& a = s.a;
  const int b = blockIdx.z, kvh = blockIdx.y / s.q_tiles, qt = blockIdx.y - kvh * s.q_tiles;
  const int lane = threadIdx.x & 31, row = blockIdx.x * 4 + (threadIdx.x >> 5), qi = qt * QB + row;
  const SeqLen n = seq_len_of(a.prefix_len[b], a.n_rows ? a.n_rows[b] : a.rows, a.rows,
                              (long long)a.g.max_pages * a.g.page);
  if (qi >= n.rows * a.G) return;
  const size_t step = (size_t)QB * (D + 2);
  const float* p = s.part + (((size_t)b * gridDim.y + blockIdx.y) * s.ns * QB + row) * (D + 2);
  // Lane i has the maximum and the sum of parts i and 32 + i, and their weights; a part that has seen nothing is left out (its sum is
  // zero; one whose scores were all NaN is not).
  static_assert(MAX_SPLITS == 64, "two parts per lane");
  float m[2], w[2], mx = -INFINITY, l = 0.f;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int i = lane + 32 * x;
    m[x] = i < s.ns ? p[i * step] : -INFINITY;
    w[x] = i < s.ns ? p[i * step + 1] : 0.f;
    mx = fmaxf(mx, m[x]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  const float off = mx == -INFINITY ? 0.f : mx;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const bool nothing = m[x] == -INFINITY && w[x] == 0.f;
    const float c = nothing ? 0.f : m[x] == -INFINITY ? 1.f : exp2f(m[x] - off);
    l = nothing ? l : fmaf(w[x], c, l);
    w[x] = nothing ? -1.f : c;                            // (a weight that no part has)
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  float o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = 0.f;
  // eight parts' outputs are on their way at a time
  for (int i0 = 0; i0 < s.ns; i0 += 8) {
    float y[8][D / 32];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* part = p + (i0 + i < s.ns ? i0 + i : i0) * step + 2 + lane;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) y[i][e] = part[32 * e];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = __shfl_sync(0xffffffffu, i0 < 32 ? w[0] : w[1], (i0 + i) & 31);
      if (i0 + i < s.ns && c >= 0.f) {
#pragma unroll
        for (int e = 0; e < D / 32; ++e) o[e] = fmaf(y[i][e], c, o[e]);
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int r = qi / a.G;
  T* dst = reinterpret_cast<T*>(a.out) + (((size_t)b * a.rows + r) * a.Hq + kvh * a.G + qi - r * a.G) * D;
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dst[lane + 32 * e] = from_f<T>(o[e] * inv);
}

// Parts per (sequence, KV head, query tile): enough blocks for four per SM of a 148-SM device, at least one 32-key tile
// each where the table is full.  Scratch: SIMT_BLOCKS blocks and more make one part each, which goes straight to the output;
// with fewer, blocks * ns < SIMT_BLOCKS + blocks.
constexpr int SIMT_BLOCKS = 592;
int simt_splits(long long blocks, long long slots) {
  long long ns = (SIMT_BLOCKS + blocks - 1) / blocks;
  const long long tiles = (slots + KB - 1) / KB;
  if (ns > tiles) ns = tiles;
  if (ns > MAX_SPLITS) ns = MAX_SPLITS;
  return ns < 1 ? 1 : (int)ns;
}

template <typename T, int D>
void launch_simt(Launcher& L, const SimtArgs& s, const void* pool) {
  const PagedAttnArgs& a = s.a;
  launch_pdl(L, k_paged_attn<T, D>, dim3(s.ns, a.g.Hkv * s.q_tiles, a.batch), dim3(128), 0, s,
             reinterpret_cast<const T*>(pool));
  if (s.ns > 1)
    launch_pdl(L, k_paged_attn_merge<T, D>, dim3(QB / 4, a.g.Hkv * s.q_tiles, a.batch), dim3(128), 0, s);
}

}  // namespace

size_t paged_attn_simt_workspace(int batch, int rows, int Hq, int Hkv, int d) {
  const long long blocks = (long long)batch * Hkv * (((long long)rows * (Hq / Hkv) + QB - 1) / QB);
  return (size_t)(SIMT_BLOCKS + (blocks < SIMT_BLOCKS ? blocks : SIMT_BLOCKS - 1)) * QB * (d + 2) * 4;
}

void launch_paged_attn_simt(Launcher& L, const PagedAttnArgs& a, const void* pool, int dtype) {
  SimtArgs s;
  s.a = a;
  s.q_tiles = (a.rows * a.G + QB - 1) / QB;
  s.ns = simt_splits((long long)a.batch * a.g.Hkv * s.q_tiles, (long long)a.g.max_pages * a.g.page);
  s.scale_log2 = a.scale * 1.4426950408889634f;
  s.part = reinterpret_cast<float*>(a.ws);
  const bool h = dtype == POSS_BF16;
  switch (a.g.d) {
    case 32: h ? launch_simt<bf16, 32>(L, s, pool) : launch_simt<float, 32>(L, s, pool); break;
    case 64: h ? launch_simt<bf16, 64>(L, s, pool) : launch_simt<float, 64>(L, s, pool); break;
    default: h ? launch_simt<bf16, 128>(L, s, pool) : launch_simt<float, 128>(L, s, pool); break;
  }
}

extern "C" {

size_t poss_paged_attention_workspace_bytes(const poss_page_pool* pool, int batch, int rows, int n_q_heads,
                                            int max_pages) {
  if (page_pool_check(pool) != POSS_OK || page_table_check(pool, max_pages, batch) != POSS_OK) return 0;
  if (rows < 1 || rows > POSS_MAX_ROWS || n_q_heads < 1 || n_q_heads % pool->n_kv_heads) return 0;
  size_t n = paged_attn_simt_workspace(batch, rows, n_q_heads, pool->n_kv_heads, pool->head_dim);
  if (paged_attn_tc_supported(*pool, n_q_heads / pool->n_kv_heads, 1.f)) {
    const size_t m = paged_attn_tc_workspace(*pool, batch, rows, n_q_heads, max_pages);
    if (m > n) n = m;
  }
  return (n + 255) / 256 * 256;
}

int poss_paged_tree_attention(const poss_page_pool* pool, int layer, const void* kv_pages, const int32_t* tables,
                              int max_pages, int batch, int rows, int n_q_heads, const void* q, int64_t ld_q,
                              const int32_t* prefix_len, const int32_t* n_rows, const uint64_t* anc_mask, float scale,
                              void* out, void* workspace, size_t workspace_bytes, int32_t* status,
                              poss_stream stream) {
  int rc = page_pool_check(pool);
  if (rc != POSS_OK) return rc;
  if (batch < 0 || rows < 0 || n_q_heads < 1 || layer < 0 || layer >= pool->n_layers) return POSS_E_INVALID;
  if (n_q_heads % pool->n_kv_heads) return POSS_E_SHAPE;
  if (!isfinite(scale)) return POSS_E_INVALID;
  if (batch == 0 || rows == 0) return POSS_OK;
  rc = page_table_check(pool, max_pages, batch);
  if (rc != POSS_OK) return rc;
  if (rows > POSS_MAX_ROWS) return POSS_E_CAPACITY;
  // a launch's grid: query tiles of 32 rows times KV heads
  if (pool->n_kv_heads * (((long long)rows * (n_q_heads / pool->n_kv_heads) + 31) / 32) > 65535) return POSS_E_CAPACITY;
  if (!kv_pages || !tables || !q || !prefix_len || !anc_mask || !out) return POSS_E_INVALID;
  const int es = pool->dtype == POSS_BF16 ? 2 : 4;
  if (ld_q < (int64_t)n_q_heads * pool->head_dim || (ld_q * es) % 16) return POSS_E_INVALID;
  if (!aligned16(kv_pages) || !aligned16(q) || !aligned16(out)) return POSS_E_INVALID;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) ||
      workspace_bytes < poss_paged_attention_workspace_bytes(pool, batch, rows, n_q_heads, max_pages))
    return POSS_E_WORKSPACE;
  // one block's queries may be read while another's rows are written
  const size_t row = (size_t)n_q_heads * pool->head_dim * es, n = (size_t)batch * rows;
  if (overlap(out, n * row, q, (n - 1) * ld_q * es + row)) return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  PagedAttnArgs a;
  a.g = page_geo(pool, tables, max_pages);
  a.layer = layer; a.batch = batch; a.rows = rows; a.Hq = n_q_heads; a.G = n_q_heads / pool->n_kv_heads;
  a.q = q; a.ld_q = ld_q; a.prefix_len = prefix_len; a.n_rows = n_rows; a.mask = anc_mask;
  a.mask_words = (rows + 63) / 64; a.scale = scale; a.out = out; a.ws = workspace; a.status = status;
  if (paged_attn_tc_supported(*pool, a.G, scale)) launch_paged_attn_tc(L, a, kv_pages, *pool);
  else launch_paged_attn_simt(L, a, kv_pages, pool->dtype);
  return L.err;
}

}  // extern "C"
