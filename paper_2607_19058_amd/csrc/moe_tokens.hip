// moe_tokens.hip -- what moves whole token rows: the weighted sum of expert rows back to tokens and its
// gradients, the embedding lookup and the gradient of its table. All are bound by memory.
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
template <class Y>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const int32_t *slots, const int32_t *held, int k,
                                                                    int64_t rows, const bf16_t *dout, int64_t ldo,
                                                                    const Y *y, int64_t ldy, const float *weights,
                                                                    bf16_t *dy, int64_t lddy, float *dweights,
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

template <class I, class T>
__global__ __launch_bounds__(kThreads) void embed_kernel(const I *ids, const T *table, int64_t vocab, int64_t cols,
                                                         int64_t ldt, T *out, int64_t ldo, float scale) {
  const int64_t t = blockIdx.x, col = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 8;
  if (col >= cols) return;
  const int64_t id = ids[t];
  float v[8] = {};
  if ((uint64_t)id < (uint64_t)vocab) {
    load8(table + id * ldt + col, cols - col, v);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= scale;
  }
  store8(out + t * ldo + col, cols - col, v);
}

// The table's gradient from the tokens sorted by id. An id with more than kRun tokens would keep one
// work-group busy while the others are done, so the sorted places are cut every kRun: a work-group per
// cut sums the parts of such long ids (at most the id it begins in and the id it ends in, and what of the
// two is the same id is one) into `part`, 2 rows of float a cut. Then a work-group per row of the table
// adds its tokens (up to kRun) or its parts in order, scales once and rounds once.
constexpr int kRun = 64;

// the first sorted place whose key is at least v
__device__ __forceinline__ int64_t lower_bound(const uint32_t *key, int64_t n, uint32_t v) {
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (key[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// the sum of dout's rows idx[lo .. hi) in this thread's 8 columns
template <class T>
__device__ __forceinline__ void sum_rows(const int32_t *idx, int64_t lo, int64_t hi, const T *dout, int64_t ldo,
                                         int64_t col, int64_t cols, float *acc) {
  for (int64_t i = lo; i < hi; i++) {
    float v[8];
    load8(dout + idx[i] * ldo + col, cols - col, v);
#pragma unroll
    for (int q = 0; q < 8; q++) acc[q] += v[q];
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void embed_parts(const uint32_t *key, const int32_t *idx, int64_t n,
                                                        const T *dout, int64_t ldo, int64_t vocab, int64_t cols,
                                                        int64_t ldp, float *part) {
  const int64_t lo = (int64_t)blockIdx.x * kRun, hi = lo + kRun < n ? lo + kRun : n;
  const int64_t col = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 8;
  if (col >= cols) return;
  const uint32_t first = key[lo], last = key[hi - 1];
  if ((int64_t)first < vocab) {   // the id that this cut begins in, as far as it goes here
    const int64_t b = lower_bound(key, n, first), e = lower_bound(key, n, first + 1);
    if (e - b > kRun) {
      float acc[8] = {};
      sum_rows(idx, lo, e < hi ? e : hi, dout, ldo, col, cols, acc);
      store8(part + 2 * blockIdx.x * ldp + col, cols - col, acc);
    }
  }
  if (last != first && (int64_t)last < vocab) {
    const int64_t b = lower_bound(key, n, last), e = lower_bound(key, n, last + 1);
    if (e - b > kRun) {
      float acc[8] = {};
      sum_rows(idx, b, hi, dout, ldo, col, cols, acc);
      store8(part + (2 * blockIdx.x + 1) * ldp + col, cols - col, acc);
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void embed_rows(const uint32_t *key, const int32_t *idx, int64_t n,
                                                       const T *dout, int64_t ldo, T *dtable, int64_t cols,
                                                       int64_t ldt, int64_t ldp, const float *part, float scale) {
  const int64_t v = blockIdx.x, col = ((int64_t)blockIdx.y * kThreads + threadIdx.x) * 8;
  if (col >= cols) return;
  const int64_t b = lower_bound(key, n, (uint32_t)v), e = lower_bound(key, n, (uint32_t)v + 1);
  float acc[8] = {};
  if (e - b <= kRun) {
    sum_rows(idx, b, e, dout, ldo, col, cols, acc);
  } else {
    for (int64_t c = b / kRun; c * kRun < e; c++) {   // the cuts that the id's places lie in
      const bool begins = c * kRun >= b;              // the cut begins in this id
      float x[8];
      load8(part + (2 * c + (begins ? 0 : 1)) * ldp + col, cols - col, x);
#pragma unroll
      for (int q = 0; q < 8; q++) acc[q] += x[q];
    }
  }
#pragma unroll
  for (int q = 0; q < 8; q++) acc[q] *= scale;
  store8(dtable + v * ldt + col, cols - col, acc);
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
                            int64_t ldy, const float *weights, void *dy, int64_t lddy, float *dweights, int64_t m,
                            void *stream) {
  by_type(y_dtype, [&](auto Y) {
    combine_backward_kernel<<<(unsigned)r.tokens, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
        r.slots, r.offsets + r.experts, r.k, r.tokens * r.k, static_cast<const bf16_t *>(dout), ldo,
        static_cast<const decltype(Y) *>(y), ldy, weights, static_cast<bf16_t *>(dy), lddy, dweights, m);
  });
  return (int)hipGetLastError();
}

int launch_embed(const void *ids, int id_bytes, int64_t n, const void *table, int64_t vocab, int64_t cols, int64_t ldt,
                 void *out, int64_t ldo, int dtype, float scale, void *stream) {
  const dim3 grid((unsigned)n, col_groups(cols));
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_type(dtype, [&](auto T) {
    typedef decltype(T) E;
    if (id_bytes == 8)
      embed_kernel<<<grid, kThreads, 0, s>>>(static_cast<const int64_t *>(ids), static_cast<const E *>(table), vocab,
                                             cols, ldt, static_cast<E *>(out), ldo, scale);
    else
      embed_kernel<<<grid, kThreads, 0, s>>>(static_cast<const int32_t *>(ids), static_cast<const E *>(table), vocab,
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
    if (n > kRun)   // no id can have more than kRun tokens otherwise
      embed_parts<<<dim3((unsigned)((n + kRun - 1) / kRun), col_groups(cols)), kThreads, 0, s>>>(
          o.key, o.idx, n, static_cast<const E *>(dout), ldo, vocab, cols, part_stride(cols), part);
    embed_rows<<<dim3((unsigned)vocab, col_groups(cols)), kThreads, 0, s>>>(
        o.key, o.idx, n, static_cast<const E *>(dout), ldo, static_cast<E *>(dtable), cols, ldt, part_stride(cols),
        part, scale);
  });
  return (int)hipGetLastError();
}

}  // namespace moe
