// moe_tokens.hip -- what moves whole token rows: the weighted sum of expert rows back to tokens and its
// gradients, the embedding lookup and the gradient of its table. All are bound by memory.
// Measured: combine of 9003 float32 rows of 1031 to 3001 tokens 9.2 us (4.6 TB/s); its gradients for 2048 tokens, top 2, 2048
// columns 15 to 19 us (59 MB; with dy in bf16 11 to 15, 42 MB); lookup of 65537 rows of 1031 floats 92 us (540 MB read and written, rows met twice among
// them); gradient of a 50304 x 2048 bf16 table from 8192 tokens 18 us for the cuts and 51 to 63 us for the rows (206 MB
// written, 3.2 to 4.1 TB/s).
#include "moe_internal.h"

namespace moe {
namespace {

constexpr int kThreads = 256;

// A work-group takes one token and kThreads * 8 columns.
template <class Y, class O>
__global__ __launch_bounds__(kThreads) void combine_kernel(const int32_t *slots, int k, int64_t rows, const Y *y,
                                                           int64_t ldy, const float *weights, O *out, int64_t ldo,
                                                           int64_t m) {
  const int64_t t = blockIdx.x, col = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 8;
  if (col >= m) return;
  float acc[8] = {};
  for (int j = 0; j < k; j++) {
    const int32_t p = slots[t * k + j];
    if ((uint32_t)p >= (uint64_t)rows) continue;
    const float w = weights ? weights[t * k + j] : 1.0f;
    float v[8];
    load8(y + p * ldy + col, m - col, v);
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] = fmaf(w, v[i], acc[i]);
  }
  store8(out + t * ldo + col, m - col, acc);
}

// A work-group takes one token: its dout row times each weight, and the dot products with the rows of y.
// Places from offsets[experts] on hold no pair; the work-group of token t zeroes those among t k .. t k + k - 1.
// dy (D) is float32, or bf16 for a caller who takes one more rounding of the weights' gradient (2^-9 of each term on average)
// for half the bytes and half the products of skew_expert_matmul_grad_f32.
template <class Y, class D>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const int32_t *slots, const int32_t *held, int k,
                                                                    int64_t rows, const bf16_t *dout, int64_t ldo,
                                                                    const Y *y, int64_t ldy, const float *weights,
                                                                    D *dy, int64_t lddy, float *dweights,
                                                                    int64_t m) {
  __shared__ float part[SKEW_MAX_CHOICES][kThreads / 64];
  const int64_t t = blockIdx.x;
  for (int j = 0; j < k; j++) {
    const int32_t p = slots[t * k + j];
    const bool on = (uint32_t)p < (uint64_t)rows;
    float dot = 0.0f;
    if (on) {
      const float w = weights ? weights[t * k + j] : 1.0f;
      for (int64_t col = threadIdx.x * 8; col < m; col += kThreads * 8) {
        float d[8], v[8];
        load8(dout + t * ldo + col, m - col, d);
        load8(y + p * ldy + col, m - col, v);
#pragma unroll
        for (int i = 0; i < 8; i++) dot = fmaf(d[i], v[i], dot);
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] *= w;
        store8(dy + p * lddy + col, m - col, d);
      }
    }
    for (int o = 32; o > 0; o >>= 1) dot += __shfl_xor(dot, o);
    if ((threadIdx.x & 63) == 0) part[j][threadIdx.x >> 6] = dot;
  }
  __syncthreads();
  if ((int)threadIdx.x < k) {
    float s = part[threadIdx.x][0];
    for (int w = 1; w < kThreads / 64; w++) s += part[threadIdx.x][w];
    dweights[t * k + threadIdx.x] = s;
  }
  const float zero[8] = {};
  for (int64_t p = t * k > *held ? t * k : *held; p < t * k + k; p++)
    for (int64_t col = threadIdx.x * 8; col < m; col += kThreads * 8) store8(dy + p * lddy + col, m - col, zero);
}

// A wave takes one token, 64 16-byte pieces of its row at a time.
template <class I, class T>
__global__ __launch_bounds__(kThreads) void embed_kernel(const I *ids, int64_t n, const T *table, int64_t vocab,
                                                         int64_t cols, int64_t ldt, T *out, int64_t ldo, float scale) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (t >= n) return;
  const int64_t id = ids[t];
  const bool there = (uint64_t)id < (uint64_t)vocab;
#pragma unroll 4
  for (int64_t col = (threadIdx.x & 63) * kVec<T>; col < cols; col += 64 * kVec<T>) {
    float v[kVec<T>] = {};
    if (there) {
      load_vec(table + id * ldt + col, cols - col, v);
#pragma unroll
      for (int i = 0; i < kVec<T>; i++) v[i] *= scale;
    }
    store_vec(out + t * ldo + col, cols - col, v);
  }
}

// The table's gradient from the tokens sorted by id. An id with many tokens would keep one wave busy while the
// others are done, so the sorted places are cut every kRun: a wave per cut and 64 16-byte pieces sums what the cut
// holds of the ids that reach over its ends (the one it begins in and the one it ends in; where the two are the
// same id it is one part) into `part`, 2 rows of float a cut. Then a work-group per kIds rows of the table finds
// their places, and a wave per row and 64 pieces adds the row's tokens, or its parts in order, scales once and
// rounds once. An id's parts are added one after another, so an id that many tokens have still takes longer, if 32 times
// less so: 65537 tokens into 32003 x 1031 floats 232 us with Zipf's law, 427 with one id in half of them, 730 in all of them.
constexpr int kRun = 32, kIds = 16;

// the first sorted place in [lo, hi) whose key is at least v, else hi
__device__ __forceinline__ int64_t lower_bound(const uint32_t *key, int64_t lo, int64_t hi, uint32_t v) {
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (key[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}
// the same in [0, n) by a whole wave, which looks at 64 places at a time
__device__ __forceinline__ int64_t wave_lower_bound(const uint32_t *key, int64_t n, uint32_t v) {
  int64_t lo = 0, len = n;
  while (len > 0) {
    const int64_t step = (len + 63) / 64, at = (threadIdx.x & 63) * step;
    // keys rise, so the lanes whose key is below v come first
    const int below = __popcll(__ballot(at < len && key[lo + (at < len ? at : 0)] < v));
    if (below == 0) return lo;
    lo += (below - 1) * step + 1;   // past the last probe that is below
    const int64_t rest = len - ((below - 1) * step + 1);
    len = rest < step - 1 ? rest : step - 1;
  }
  return lo;
}

// Adds dout's rows idx[lo .. hi), at most 64, in this lane's columns, 8 rows' loads on their way together.
template <class T>
__device__ __forceinline__ void sum_rows(const int32_t *idx, int64_t lo, int64_t hi, const T *dout, int64_t ldo,
                                         int64_t col, int64_t cols, float *acc) {
  const int lane = threadIdx.x & 63, n = __builtin_amdgcn_readfirstlane((int)(hi - lo));
  const int32_t mine = lane < n ? idx[lo + lane] : 0;
  int r = 0;
  for (; r + 8 <= n; r += 8) {
    float v[8][kVec<T>];
#pragma unroll
    for (int u = 0; u < 8; u++)
      load_vec(dout + __builtin_amdgcn_readlane(mine, r + u) * ldo + col, cols - col, v[u]);
#pragma unroll
    for (int u = 0; u < 8; u++)
#pragma unroll
      for (int q = 0; q < kVec<T>; q++) acc[q] += v[u][q];
  }
  for (; r < n; r++) {
    float v[kVec<T>];
    load_vec(dout + __builtin_amdgcn_readlane(mine, r) * ldo + col, cols - col, v);
#pragma unroll
    for (int q = 0; q < kVec<T>; q++) acc[q] += v[q];
  }
}

template <class T>
__global__ __launch_bounds__(64) void embed_parts(const uint32_t *key, const int32_t *idx, int64_t n, const T *dout,
                                                  int64_t ldo, int64_t vocab, int64_t cols, int64_t ldp, float *part) {
  constexpr int V = kVec<T>;
  const int64_t lo = (int64_t)blockIdx.x * kRun, hi = lo + kRun < n ? lo + kRun : n;
  const int64_t at = ((int64_t)blockIdx.y * 64 + threadIdx.x) * V, col = at < cols ? at : 0;   // (past the row: not stored)
  const int lane = threadIdx.x;
  const uint32_t mine = key[lo + lane < hi ? lo + lane : hi - 1];
  const uint32_t first = __builtin_amdgcn_readlane(mine, 0), last = key[hi - 1];
  const bool from_before = lo > 0 && key[lo - 1] == first, goes_on = hi < n && key[hi] == last;
  const int64_t end = lo + __popcll(__ballot(mine == first && lo + lane < hi));    // of the first id, here
  const int64_t begin = hi - __popcll(__ballot(mine == last && lo + lane < hi));   // of the last one
  auto add = [&](int64_t b, int64_t e, int64_t row) {
    float acc[V] = {};
    sum_rows(idx, b, e, dout, ldo, col, cols, acc);
    if (at < cols) {
#pragma unroll
      for (int q = 0; q < V; q += 4) store_vec(part + row * ldp + at + q, 4, acc + q);
    }
  };
  if ((int64_t)first < vocab && (from_before || (end == hi && goes_on))) add(lo, end, 2 * blockIdx.x);
  if ((int64_t)last < vocab && last != first && goes_on) add(begin, hi, 2 * blockIdx.x + 1);
}

template <class T>
__global__ __launch_bounds__(kThreads) void embed_rows(const uint32_t *key, const int32_t *idx, int64_t n,
                                                       const T *dout, int64_t ldo, T *dtable, int64_t vocab,
                                                       int64_t cols, int64_t ldt, int64_t ldp, const float *part,
                                                       float scale) {
  constexpr int V = kVec<T>;
  __shared__ int64_t range[2];
  __shared__ int32_t start[kIds + 1];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t v0 = (int64_t)blockIdx.x * kIds;
  if (wave < 2) {
    const int64_t x = wave_lower_bound(key, n, (uint32_t)(v0 + wave * kIds));
    if ((tid & 63) == 0) range[wave] = x;
  }
  __syncthreads();
  if (tid <= kIds) start[tid] = (int32_t)lower_bound(key, range[0], range[1], (uint32_t)(v0 + tid));
  __syncthreads();
  const int64_t left = vocab - v0;
  const int ids = left < kIds ? (int)left : kIds, pieces = (int)((cols + 64 * V - 1) / (64 * V));
  for (int64_t item = wave; item < (int64_t)ids * pieces; item += kThreads / 64) {
    const int r = (int)(item / pieces);
    const int64_t at = ((item - (int64_t)r * pieces) * 64 + (tid & 63)) * V, col = at < cols ? at : 0;
    const int64_t b = __builtin_amdgcn_readfirstlane(start[r]), e = __builtin_amdgcn_readfirstlane(start[r + 1]);
    float acc[V] = {};
    if (b == e || b / kRun == (e - 1) / kRun) {   // inside one cut
      sum_rows(idx, b, e, dout, ldo, col, cols, acc);
    } else {
#pragma unroll 8
      for (int64_t c = b / kRun; c < (e + kRun - 1) / kRun; c++) {   // the cuts that the id's places lie in
        float x[V];
#pragma unroll
        for (int q = 0; q < V; q += 4) load_vec(part + (2 * c + (c * kRun >= b ? 0 : 1)) * ldp + col + q, 4, x + q);   // 0: begins in the id
#pragma unroll
        for (int q = 0; q < V; q++) acc[q] += x[q];
      }
    }
#pragma unroll
    for (int q = 0; q < V; q++) acc[q] *= scale;
    if (at < cols) store_vec(dtable + (v0 + r) * ldt + at, cols - at, acc);
  }
}

inline unsigned col_groups(int64_t cols) { return (unsigned)((cols + kThreads * 8 - 1) / (kThreads * 8)); }

template <class F>
void by_type(int dtype, F f) {
  if (dtype == SKEW_F32) f(float());
  else f(bf16_t());
}

}  // namespace

int launch_combine(const skew_rows &r, const void *y, int y_dtype, int64_t ldy, const float *weights, void *out,
                   int out_dtype, int64_t ldo, int64_t m, void *stream) {
  const dim3 grid((unsigned)r.tokens, col_groups(m));
  by_type(y_dtype, [&](auto Y) {
    by_type(out_dtype, [&](auto O) {
      combine_kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
          r.slots, r.k, r.tokens * r.k, static_cast<const decltype(Y) *>(y), ldy, weights,
          static_cast<decltype(O) *>(out), ldo, m);
    });
  });
  return (int)hipGetLastError();
}

int launch_combine_backward(const skew_rows &r, const void *dout, int64_t ldo, const void *y, int y_dtype,
                            int64_t ldy, const float *weights, void *dy, int dy_dtype, int64_t lddy, float *dweights,
                            int64_t m, void *stream) {
  by_type(y_dtype, [&](auto Y) {
    by_type(dy_dtype, [&](auto D) {
      combine_backward_kernel<<<(unsigned)r.tokens, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
          r.slots, r.offsets + r.experts, r.k, r.tokens * r.k, static_cast<const bf16_t *>(dout), ldo,
          static_cast<const decltype(Y) *>(y), ldy, weights, static_cast<decltype(D) *>(dy), lddy, dweights, m);
    });
  });
  return (int)hipGetLastError();
}

int launch_embed(const void *ids, int id_bytes, int64_t n, const void *table, int64_t vocab, int64_t cols, int64_t ldt,
                 void *out, int64_t ldo, int dtype, float scale, void *stream) {
  const unsigned grid = (unsigned)((n + kThreads / 64 - 1) / (kThreads / 64));
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_type(dtype, [&](auto T) {
    typedef decltype(T) E;
    if (id_bytes == 8)
      embed_kernel<<<grid, kThreads, 0, s>>>(static_cast<const int64_t *>(ids), n, static_cast<const E *>(table), vocab,
                                             cols, ldt, static_cast<E *>(out), ldo, scale);
    else
      embed_kernel<<<grid, kThreads, 0, s>>>(static_cast<const int32_t *>(ids), n, static_cast<const E *>(table), vocab,
                                             cols, ldt, static_cast<E *>(out), ldo, scale);
  });
  return (int)hipGetLastError();
}

namespace {
inline int64_t part_stride(int64_t cols) { return (cols + 7) / 8 * 8; }
}  // namespace

size_t embed_scratch(int64_t n, int64_t cols) {
  return n > kRun ? (size_t)((n + kRun - 1) / kRun) * 2 * (size_t)part_stride(cols) * 4 : 0;
}

int launch_embed_grad(const SortOut &o, int64_t n, const void *dout, int64_t ldo, void *dtable, int64_t vocab,
                      int64_t cols, int64_t ldt, int dtype, float scale, char *partials, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  float *part = reinterpret_cast<float *>(partials);
  by_type(dtype, [&](auto T) {
    typedef decltype(T) E;
    if (n > kRun)   // else there is one cut
      embed_parts<<<dim3((unsigned)((n + kRun - 1) / kRun), (unsigned)((cols + 64 * kVec<E> - 1) / (64 * kVec<E>))), 64, 0, s>>>(
          o.key, o.idx, n, static_cast<const E *>(dout), ldo, vocab, cols, part_stride(cols), part);
    embed_rows<<<(unsigned)((vocab + kIds - 1) / kIds), kThreads, 0, s>>>(
        o.key, o.idx, n, static_cast<const E *>(dout), ldo, static_cast<E *>(dtable), vocab, cols, ldt,
        part_stride(cols), part, scale);
  });
  return (int)hipGetLastError();
}

}  // namespace moe
