// Rotary positions: pairs of a head's elements turned by position times the pair's frequency, on rows that stay where they are
// (poss_rotary) and on rows that go into pages (poss_pages_append_rotary, queries in the same launch).
//
//   (u, v) -> (u cos a - v sin a, v cos a + u sin a) * magnitude,  a = position * frequency of the pair
//
// The angle of a far position is where 32 bits would fail (at position 10^6 an fp32 product is off by 0.06 radians): position and
// frequency are multiplied in 64 bits as turns, the whole turns are taken off (the fused multiply-add leaves the fraction exactly), and
// only the fraction goes on in 32 bits.  What is left is the rounding of the frequency in turns, 2^-52 of the angle.
//
// One block per row: all threads stream the row's heads, two pieces of 16 bytes at a time; while the first are on their way a thread per
// pair leaves cosine and sine in shared memory.  With halves as pairs the two pieces are partners, so a row may be turned in place.
// What bounds it: memory for prompts of wide rows (8192 rows of 48 heads of 128 in bf16, 201 MB: 37.8 us, 5.3 TB/s; in fp32, 403 MB: 65 us, 6.2
// TB/s); a chain of trips (lengths and position, table, data) for a token: 3.1 us.  Narrow rows leave most of a block's threads without a
// task and are bound by the blocks' chains: 32768 rows of 12 heads of 64, 101 MB, take 50 us, 131072 rows of 10 heads of 32, 168 MB, 166.
#include "paged.cuh"
#include <math.h>

POSS_TRACE_REGISTER()

namespace {

constexpr int THREADS = 128;
constexpr int MAX_HALF = POSS_MAX_ROTARY_DIM / 2;

// What is turned, and how
struct Turn {
  const double* freq;        // radians per position, [half]
  int half;                  // pairs
  int interleaved;           // pairs are neighbours; else element i and half + i
  float magnitude;
};
// The heads of a row in global memory: those that turn from two places (queries and keys), then those that do not (values).  Sources are
// contiguous, targets dst_step bytes apart per head.
struct Group {
  const char* src;
  char* dst;
  size_t dst_step;
  int n;
};
struct Row { Group g[3]; };

__device__ __forceinline__ void angles(const Turn& turn, int position, float2* cs) {
  for (int i = threadIdx.x; i < turn.half; i += THREADS) {
    const double t = turn.freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
    const double p = (double)position;
    const float fraction = (float)fma(p, t, -rint(p * t));
    float s, c;
    sincospif(2.f * fraction, &s, &c);
    cs[i] = make_float2(c * turn.magnitude, s * turn.magnitude);
  }
}
__device__ __forceinline__ float2 turned(float u, float v, float2 cs) {
  return make_float2(u * cs.x - v * cs.y, v * cs.x + u * cs.y);
}

template <typename T> struct Piece;          // 16 bytes as fp32 values
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(uint4 w, float* x) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Piece<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(uint4 w, float* x) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};

// The row's heads, two pieces of 16 bytes per task, BATCH tasks per thread at a time: the first ones' loads go out before the angles are
// worked out.  Pieces a and b of a head: with halves as pairs a and its partner while there are pairs; behind them, and with neighbours as
// pairs from the start, consecutive ones.
// BATCH 3 hides a row's latency and takes 104 registers; with BATCH 1 twelve blocks fit an SM, which hide it in one another.  One token of 48
// heads 3.1 us (with BATCH 1 3.5), 976 rows 5.6 (9.0), 8192 rows 51 (37.8).
template <typename T, int BATCH>
__device__ __forceinline__ void stream_row(const Row& row, const Turn& turn, int position, int d, float2* cs) {
  constexpr int N = Piece<T>::N;
  const int pieces = d / N, steps = (pieces + 1) / 2, paired = turn.interleaved ? 0 : turn.half / N;
  const int turning = row.g[0].n + row.g[1].n, tasks = (turning + row.g[2].n) * steps;
  for (int i0 = threadIdx.x;; i0 += BATCH * THREADS) {
    uint4 x[BATCH][2];
    uint4* to[BATCH];
    int a[BATCH], b[BATCH];                               // b < 0: a head's last, odd piece; a < 0: nothing
    bool turns[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const int i = i0 + k * THREADS;
      a[k] = b[k] = -1;
      turns[k] = false;
      if (i < tasks) {
        int head = i / steps;
        const int j = i - head * steps;
        turns[k] = head < turning;
        const bool first = head < row.g[0].n;
        head -= first ? 0 : turns[k] ? row.g[0].n : turning;
        const bool pair = turns[k] && j < paired;
        a[k] = pair ? j : 2 * j;
        b[k] = pair ? j + paired : 2 * j + 1 < pieces ? 2 * j + 1 : -1;
        const uint4* from = reinterpret_cast<const uint4*>(first ? row.g[0].src : turns[k] ? row.g[1].src : row.g[2].src) + (size_t)head * pieces;
        to[k] = reinterpret_cast<uint4*>((first ? row.g[0].dst : turns[k] ? row.g[1].dst : row.g[2].dst) +
                                         head * (first ? row.g[0].dst_step : turns[k] ? row.g[1].dst_step : row.g[2].dst_step));
        x[k][0] = from[a[k]];
        if (b[k] >= 0) x[k][1] = from[b[k]];
      }
    }
    if (i0 == (int)threadIdx.x) {                         // (every thread comes here once)
      angles(turn, position, cs);
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      if (a[k] < 0) continue;
      if (turns[k]) {
        float u[N], v[N];
        Piece<T>::get(x[k][0], u);
        Piece<T>::get(x[k][1], v);
        if (turn.interleaved) {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const int pa = (a[k] * N + e) / 2, pb = pa + N / 2;
            if (pa < turn.half) { const float2 y = turned(u[e], u[e + 1], cs[pa]); u[e] = y.x; u[e + 1] = y.y; }
            if (pb < turn.half) { const float2 y = turned(v[e], v[e + 1], cs[pb]); v[e] = y.x; v[e + 1] = y.y; }
          }
        } else if (a[k] < paired) {
          // (two pairs' angles per access: a warp's lanes lie 64 bytes apart in bf16, four to a bank)
          const float4* const c = reinterpret_cast<const float4*>(cs + a[k] * N);
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const float4 f = c[e / 2];
            const float2 y = turned(u[e], v[e], make_float2(f.x, f.y)), z = turned(u[e + 1], v[e + 1], make_float2(f.z, f.w));
            u[e] = y.x; v[e] = y.y;
            u[e + 1] = z.x; v[e + 1] = z.y;
          }
        }
        x[k][0] = Piece<T>::put(u);
        x[k][1] = Piece<T>::put(v);
      }
      to[k][a[k]] = x[k][0];
      if (b[k] >= 0) to[k][b[k]] = x[k][1];
    }
    if (i0 - (int)threadIdx.x + BATCH * THREADS >= tasks) break;         // (the same for all)
  }
}
// halves as pairs whose partners do not lie whole pieces apart: one pair, or one element that stays, per thread
template <typename T>
__device__ __forceinline__ void stream_elements(const Row& row, const Turn& turn, int position, int d, float2* cs) {
  angles(turn, position, cs);
  __syncthreads();
  for (int g = 0; g < 3; ++g) {
    const int half = g < 2 ? turn.half : 0, steps = d - half;
    for (int i = threadIdx.x; i < row.g[g].n * steps; i += THREADS) {
      const int head = i / steps, j = i - head * steps;
      const T* src = reinterpret_cast<const T*>(row.g[g].src) + (size_t)head * d;
      T* dst = reinterpret_cast<T*>(row.g[g].dst + head * row.g[g].dst_step);
      if (j < half) {
        const float2 y = turned(to_f(src[j]), to_f(src[j + half]), cs[j]);
        dst[j] = from_f<T>(y.x);
        dst[j + half] = from_f<T>(y.y);
      } else {
        dst[j + half] = src[j + half];
      }
    }
  }
}
template <typename T, int BATCH>
__device__ __forceinline__ void turn_row(const Row& row, const Turn& turn, int position, int d, float2* cs) {
  if (turn.interleaved || turn.half % Piece<T>::N == 0) stream_row<T, BATCH>(row, turn, position, d, cs);
  else stream_elements<T>(row, turn, position, d, cs);
}

template <typename T, int BATCH>
__global__ void __launch_bounds__(THREADS, BATCH == 1 ? 12 : 1) k_rotary(Turn turn, int heads, int d, const char* x, long long ld, char* out,
                                                    long long ld_out, const int32_t* positions) {
  __shared__ __align__(16) float2 cs[MAX_HALF];
  pdl_enter(POSS_K_ROTARY);
  const size_t row = blockIdx.x;
  const Row r = {{{x + row * ld, out + row * ld_out, (size_t)d * sizeof(T), heads}, {nullptr, nullptr, 0, 0}, {nullptr, nullptr, 0, 0}}};
  turn_row<T, BATCH>(r, turn, positions[row], d, cs);
}

struct AppendArgs {
  PageGeo g;
  int layer, rows, Hq;
  char* pool;
  const char *k, *v, *q;
  char* out_q;
  long long ld_kv, ld_q, ld_out_q;           // bytes
  const int32_t *prefix_len, *n_rows, *positions;
  int32_t* status;
};
template <typename T, int BATCH>
__global__ void __launch_bounds__(THREADS, BATCH == 1 ? 12 : 1) k_append_rotary(AppendArgs a, Turn turn) {
  __shared__ __align__(16) float2 cs[MAX_HALF];
  pdl_enter(POSS_K_APPEND_ROTARY);
  const size_t row = blockIdx.x;
  const int b = blockIdx.x / a.rows, r = blockIdx.x - b * a.rows;
  const int prefix = a.prefix_len[b], own = a.n_rows ? a.n_rows[b] : a.rows;
  int position = a.positions ? a.positions[row] : 0;   // (one trip with the lengths)
  const SeqLen s = seq_len_of(prefix, own, a.rows, (long long)a.g.max_pages * a.g.page);
  if (s.bad && r == 0 && threadIdx.x == 0) raise_status(a.status, POSS_E_INVALID);
  if (r >= s.rows) return;
  const int slot = s.prefix + r, place = slot / a.g.page;
  if (!a.positions) position = slot;
  const int p = page_at(a.g.tables + (size_t)b * a.g.max_pages, a.g.max_pages, a.g.n_pages, place);
  if (p < 0 && threadIdx.x == 0) raise_status(a.status, POSS_E_INVALID);
  const size_t head_bytes = (size_t)a.g.page * a.g.d * sizeof(T);
  char* const dk = a.pool + (page_offset(a.g, a.layer, p < 0 ? 0 : p, 0, 0) + (size_t)(slot - place * a.g.page) * a.g.d) * sizeof(T);
  const int kv = p < 0 ? 0 : a.g.Hkv;                     // (without a page the queries alone)
  const Row t = {{{a.q + row * a.ld_q, a.out_q + row * a.ld_out_q, (size_t)a.g.d * sizeof(T), a.Hq},
                  {a.k + row * a.ld_kv, dk, head_bytes, kv},
                  {a.v + row * a.ld_kv, dk + a.g.Hkv * head_bytes, head_bytes, kv}}};
  turn_row<T, BATCH>(t, turn, position, a.g.d, cs);
}

// (by 976 and 8192 rows of 48 heads)
bool many_rows(int64_t n) { return n > 10 * current_sm_count(); }

int turn_check(int head_dim, int rot_dim, float magnitude, const double* freq) {
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim || !isfinite(magnitude) || !freq) return POSS_E_INVALID;
  return rot_dim > POSS_MAX_ROTARY_DIM ? POSS_E_CAPACITY : POSS_OK;
}
// rows of `bytes` bytes, ld apart, n of them: does the target touch a source that it is not, row for row
bool crossed(const void* out, int64_t ld_out, const void* in, int64_t ld_in, size_t bytes, int64_t n) {
  if (out == in && ld_out == ld_in) return false;
  return overlap(out, (size_t)(n - 1) * ld_out + bytes, in, (size_t)(n - 1) * ld_in + bytes);
}
// n rows of a_bytes and n of b_bytes, both ld >= either bytes apart: do two of them, of any places, share a byte
bool rows_meet(const void* a, size_t a_bytes, const void* b, size_t b_bytes, int64_t ld, int64_t n) {
  const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)), near = -apart / ld;
  for (int64_t m = near - 1; m <= near + 1; ++m)          // (row i of a and row i - m of b)
    if (m > -n && m < n && m * ld + apart < (int64_t)b_bytes && -(m * ld + apart) < (int64_t)a_bytes) return true;
  return false;
}

}  // namespace

extern "C" {

int poss_rotary_frequencies(double* h_freq, int rot_dim, double theta, int scaling, double factor, double low, double high,
                            double original_len) {
  if (!h_freq || rot_dim < 2 || rot_dim % 2 || !(theta > 1.0) || !isfinite(theta)) return POSS_E_INVALID;
  if (rot_dim > POSS_MAX_ROTARY_DIM) return POSS_E_CAPACITY;
  if (scaling < POSS_ROTARY_PLAIN || scaling > POSS_ROTARY_RAMP) return POSS_E_INVALID;
  if (scaling != POSS_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return POSS_E_INVALID;
  const bool parts = scaling == POSS_ROTARY_BANDS || scaling == POSS_ROTARY_RAMP;
  if (parts && (!(low > 0.0) || !(high > low) || !isfinite(high) || !(original_len > 0.0) || !isfinite(original_len)))
    return POSS_E_INVALID;
  if (scaling == POSS_ROTARY_BASE) {
    if (rot_dim < 4) return POSS_E_INVALID;
    theta *= pow(factor, (double)rot_dim / (rot_dim - 2));
  }
  const double two_pi = 6.283185307179586477, half = rot_dim / 2;
  // the pair that makes `turns` turns over the original context
  auto pair_of = [&](double turns) { return half * log(original_len / (turns * two_pi)) / log(theta); };
  double first = 0.0, last = 0.0;
  if (scaling == POSS_ROTARY_RAMP) {
    first = fmax(floor(pair_of(high)), 0.0);
    last = fmin(ceil(pair_of(low)), (double)rot_dim - 1.0);
    if (last <= first) last = first + 0.001;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = pow(theta, -(double)i / half);
    double kept = 1.0;                                    // share of the frequency that is not divided
    if (scaling == POSS_ROTARY_LINEAR) kept = 0.0;
    if (scaling == POSS_ROTARY_BANDS) kept = (original_len * f / two_pi - low) / (high - low);
    if (scaling == POSS_ROTARY_RAMP) kept = 1.0 - (i - first) / (last - first);
    kept = fmin(fmax(kept, 0.0), 1.0);
    h_freq[i] = kept * f + (1.0 - kept) * (f / factor);
    if (scaling == POSS_ROTARY_BASE || scaling == POSS_ROTARY_PLAIN) h_freq[i] = f;
  }
  return POSS_OK;
}

int poss_rotary(const void* x, int64_t ld_x, void* out, int64_t ld_out, int dtype, int64_t n, int heads, int head_dim,
                const int32_t* positions, const double* freq, int rot_dim, int interleaved, float magnitude, poss_stream stream) {
  if (dtype != POSS_FP32 && dtype != POSS_BF16) return POSS_E_INVALID;
  if (n < 0 || heads < 1 || head_dim < 2) return POSS_E_INVALID;
  const int es = dtype == POSS_BF16 ? 2 : 4;
  if (head_dim * (int64_t)es % 16) return POSS_E_SHAPE;
  int rc = turn_check(head_dim, rot_dim, magnitude, freq);
  if (rc != POSS_OK) return rc;
  if (n == 0) return POSS_OK;
  if (n >= (1ll << 31) || head_dim > (1 << 16) || (int64_t)heads * head_dim >= (1ll << 28)) return POSS_E_CAPACITY;
  if (!x || !out || !positions || !aligned16(x) || !aligned16(out)) return POSS_E_INVALID;
  const int64_t row = (int64_t)heads * head_dim;
  if (ld_x < row || ld_out < row || (ld_x * es) % 16 || (ld_out * es) % 16) return POSS_E_INVALID;
  if (crossed(out, ld_out * es, x, ld_x * es, row * es, n)) return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  const Turn turn = {freq, rot_dim / 2, interleaved != 0, magnitude};
  const bool many = many_rows(n);
  launch_pdl(L, dtype == POSS_BF16 ? (many ? k_rotary<bf16, 1> : k_rotary<bf16, 3>) : many ? k_rotary<float, 1> : k_rotary<float, 3>, dim3((unsigned)n), dim3(THREADS), 0, turn, heads, head_dim,
             reinterpret_cast<const char*>(x), ld_x * es, reinterpret_cast<char*>(out), ld_out * es, positions);
  return L.err;
}

int poss_pages_append_rotary(const poss_page_pool* pool, int layer, void* kv_pages, const int32_t* tables, int max_pages, int batch,
                             int rows, const void* k, const void* v, int64_t ld_kv, int n_q_heads, const void* q, int64_t ld_q,
                             void* out_q, int64_t ld_out_q, const int32_t* prefix_len, const int32_t* n_rows,
                             const int32_t* positions, const double* freq, int rot_dim, int interleaved, float magnitude,
                             int32_t* status, poss_stream stream) {
  int rc = page_pool_check(pool);
  if (rc != POSS_OK) return rc;
  if (batch < 0 || rows < 0 || n_q_heads < 0 || layer < 0 || layer >= pool->n_layers) return POSS_E_INVALID;
  rc = turn_check(pool->head_dim, rot_dim, magnitude, freq);
  if (rc != POSS_OK) return rc;
  if (batch == 0 || rows == 0) return POSS_OK;
  rc = page_table_check(pool, max_pages, batch);
  if (rc != POSS_OK) return rc;
  if (rows > 65535 || n_q_heads > (1 << 16)) return POSS_E_CAPACITY;
  if (!kv_pages || !tables || !k || !v || !prefix_len) return POSS_E_INVALID;
  const int64_t es = pool->dtype == POSS_BF16 ? 2 : 4, d = pool->head_dim;
  if (ld_kv < pool->n_kv_heads * d || (ld_kv * es) % 16) return POSS_E_INVALID;
  if (!aligned16(kv_pages) || !aligned16(k) || !aligned16(v)) return POSS_E_INVALID;
  if (n_q_heads) {
    if (!q || !out_q || !aligned16(q) || !aligned16(out_q)) return POSS_E_INVALID;
    const int64_t row = n_q_heads * d, n = (int64_t)batch * rows;
    if (ld_q < row || ld_out_q < row || (ld_q * es) % 16 || (ld_out_q * es) % 16) return POSS_E_INVALID;
    if (crossed(out_q, ld_out_q * es, q, ld_q * es, row * es, n)) return POSS_E_INVALID;
    // (in place the three may be parts of one projection, whose rows lie between one another: its columns must not meet then)
    const size_t kv_row = pool->n_kv_heads * d * es, kv_bytes = (size_t)(n - 1) * ld_kv * es + kv_row;
    for (const void* in : {k, v})
      if (out_q == q && ld_q == ld_kv ? rows_meet(out_q, row * es, in, kv_row, ld_kv * es, n)
                                      : overlap(out_q, ((n - 1) * ld_out_q + row) * es, in, kv_bytes))
        return POSS_E_INVALID;
  }
  // one row's slots may be written while another's elements are read
  const size_t rows_before = (size_t)batch * rows - 1, pool_bytes = (size_t)pool->n_layers * pool->n_pages * 2 * pool->n_kv_heads * pool->page_slots * d * es;
  const size_t kv_span = (rows_before * ld_kv + pool->n_kv_heads * d) * es, q_span = (rows_before * ld_q + n_q_heads * d) * es;
  if (overlap(kv_pages, pool_bytes, k, kv_span) || overlap(kv_pages, pool_bytes, v, kv_span)) return POSS_E_INVALID;
  if (n_q_heads && (overlap(kv_pages, pool_bytes, q, q_span) ||
                    overlap(kv_pages, pool_bytes, out_q, (rows_before * ld_out_q + n_q_heads * d) * es)))
    return POSS_E_INVALID;
  int64_t launches = 0;
  Launcher L{reinterpret_cast<cudaStream_t>(stream), &launches, POSS_OK};
  AppendArgs a;
  a.g = page_geo(pool, tables, max_pages);
  a.layer = layer; a.rows = rows; a.Hq = n_q_heads;
  a.pool = reinterpret_cast<char*>(kv_pages);
  a.k = reinterpret_cast<const char*>(k); a.v = reinterpret_cast<const char*>(v); a.q = reinterpret_cast<const char*>(q);
  a.out_q = reinterpret_cast<char*>(out_q);
  a.ld_kv = ld_kv * es; a.ld_q = ld_q * es; a.ld_out_q = ld_out_q * es;
  a.prefix_len = prefix_len; a.n_rows = n_rows; a.positions = positions; a.status = status;
  const Turn turn = {freq, rot_dim / 2, interleaved != 0, magnitude};
  const bool many = many_rows((int64_t)batch * rows);
  launch_pdl(L, pool->dtype == POSS_BF16 ? (many ? k_append_rotary<bf16, 1> : k_append_rotary<bf16, 3>)
                                         : many ? k_append_rotary<float, 1> : k_append_rotary<float, 3>, dim3((unsigned)(batch * rows)),
             dim3(THREADS), 0, a, turn);
  return L.err;
}

}  // extern "C"
