// moe_internal.h -- device helpers and launchers shared by the mixture-of-experts kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include "../../include/skew_moe.h"

namespace moe {

// How the operands of a product lie: a (rows of the result) and b (its columns), contiguous in the contraction or along the result.
//   kForward   a in the contraction, b along the result
//   kBackward  both in the contraction
//   kWeights   both along the result; the contraction is an expert's places, and a's rows are looked up
//   kOuter     both along the result; the contraction is the rows of both, from Tile::first on
enum { kForward = 0, kBackward = 1, kWeights = 2, kOuter = 3 };

constexpr int kMaxDigit = 9;             // radix digits of the sort: up to 512 bins

// Number of bits that hold 0 .. x.
inline int bits_for(uint64_t x) {
  int b = 0;
  while (b < 64 && (x >> b) != 0) b++;
  return b < 1 ? 1 : b;
}
// bf16 rows whose byte offsets stay below 2^31, with a row to spare
// (a single row may have any stride, whose products pass 2^63)
constexpr bool short_rows(int64_t rows, int64_t ld) { return ld <= 0x7FFFFFFF / (2 * (rows + 1)); }
// Length of the round that begins at `base` of `total` in rounds of at most `most`. (base + most may pass 2^31.)
constexpr int round_length(int base, int total, int most) { return total - base > most ? most : total - base; }
inline size_t pad256(size_t x) { return (x + 255) / 256 * 256; }

// How n keys of 0 .. keys (`keys` itself: none) are sorted, and where its scratch lies.
struct SortPlan {
  int64_t n = 0;
  uint32_t keys = 0;
  int passes = 0, digit = 0;     // radix passes of `digit` bits
  bool one = false;              // one work-group
  int steps = 1;                 // items of a thread in the larger sort
  int64_t nb = 0;                // its work-groups
  size_t off_key[2] = {0, 0}, off_idx[2] = {0, 0}, off_hist = 0, off_total = 0, bytes = 0;
};
SortPlan sort_plan(int64_t n, int64_t keys);

// Sorts: sorted keys and indices to `key` / `idx` (device pointers into the scratch, set by the call).
// With offsets/rows/slots (expert order) those are written too, and key/idx may stay unset.
struct SortOut {
  const uint32_t *key = nullptr;
  const int32_t *idx = nullptr;
  int32_t *offsets = nullptr, *rows = nullptr, *slots = nullptr;
};
int launch_sort(const SortPlan &p, const void *ids, int id_bytes, char *ws, SortOut *out, void *stream);

int launch_route(const skew_route_desc &d, const void *logits, const float *bias, float *weights, int32_t *chosen,
                 void *stream);
int launch_route_backward(const skew_route_desc &d, const void *logits, const int32_t *chosen, const float *dweights,
                          void *dlogits, void *stream);

int launch_combine(const skew_rows &r, const void *y, int y_dtype, int64_t ldy, const float *weights, void *out,
                   int out_dtype, int64_t ldo, int64_t m, void *stream);
int launch_combine_backward(const skew_rows &r, const void *dout, int64_t ldo, const void *y, int y_dtype,
                            int64_t ldy, const float *weights, void *dy, int dy_dtype, int64_t lddy, float *dweights,
                            int64_t m, void *stream);

size_t embed_scratch(int64_t n, int64_t cols);   // partial sums of skew_embed_grad
int launch_embed(const void *ids, int id_bytes, int64_t n, const void *table, int64_t vocab, int64_t cols, int64_t ldt,
                 void *out, int64_t ldo, int dtype, float scale, void *stream);
int launch_embed_grad(const SortOut &s, int64_t n, const void *dout, int64_t ldo, void *dtable, int64_t vocab,
                      int64_t cols, int64_t ldt, int dtype, float scale, char *partials, void *stream);

size_t product_scratch(const skew_rows &r, const skew_product_desc &p);
int launch_product(const skew_rows &r, const skew_product_desc &p, char *ws, void *stream);
int launch_product_grad(const skew_rows &r, const skew_product_desc &p, void *stream);
size_t product_grad_f32_scratch(const skew_rows &r, const skew_product_desc &p);
int launch_product_grad_f32(const skew_rows &r, const skew_product_desc &p, char *ws, void *stream);

}  // namespace moe

#ifdef __HIPCC__
#include <hip/hip_runtime.h>

namespace moe {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
// 16 bytes at any element position (the hardware takes unaligned 16-byte accesses)
typedef unsigned u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

struct bf16_t {
  uint16_t v;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x.v << 16); }
// two floats -> two bf16, round to nearest even, packed low|high
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t *p, float v) { p->v = (uint16_t)pack2(v, 0.0f); }

// 8 neighbouring values; n < 8: only the first n are read, the rest are 0
__device__ __forceinline__ void load8(const bf16_t *p, int64_t n, float *o) {
  if (n >= 8) {
    const u32x4 u = *reinterpret_cast<const u32x4_a2 *>(p);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      o[2 * i] = __uint_as_float(u[i] << 16);
      o[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = i < n ? to_f32(p[i]) : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float *p, int64_t n, float *o) {
  if (n >= 8) {
    const f32x4 a = *reinterpret_cast<const f32x4_a4 *>(p), b = *reinterpret_cast<const f32x4_a4 *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      o[i] = a[i];
      o[4 + i] = b[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = i < n ? p[i] : 0.0f;
  }
}
__device__ __forceinline__ void store8(bf16_t *p, int64_t n, const float *v) {
  if (n >= 8) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; i++) u[i] = pack2(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<u32x4_a2 *>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) put(p + i, v[i]);
  }
}
__device__ __forceinline__ void store8(float *p, int64_t n, const float *v) {
  if (n >= 8) {
    const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    *reinterpret_cast<f32x4_a4 *>(p) = a;
    *reinterpret_cast<f32x4_a4 *>(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) p[i] = v[i];
  }
}

// 8 values at p, of which the first n exist (n <= 0: none)
__device__ __forceinline__ u32x4 load_chunk(const bf16_t *p, int64_t n) {
  u32x4 u = {0, 0, 0, 0};
  if (n >= 8) {
    u = *reinterpret_cast<const u32x4_a2 *>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 7; i++)
      if (i < n) u[i >> 1] |= (uint32_t)p[i].v << (16 * (i & 1));
  }
  return u;
}

// One 16-byte access: kVec neighbouring values; n < kVec: only the first n exist.
template <class T>
constexpr int kVec = 16 / sizeof(T);
__device__ __forceinline__ void load_vec(const bf16_t *p, int64_t n, float *o) { load8(p, n, o); }
__device__ __forceinline__ void store_vec(bf16_t *p, int64_t n, const float *v) { store8(p, n, v); }
__device__ __forceinline__ void load_vec(const float *p, int64_t n, float *o) {
  if (n >= 4) {
    const f32x4 a = *reinterpret_cast<const f32x4_a4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = a[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = i < n ? p[i] : 0.0f;
  }
}
__device__ __forceinline__ void store_vec(float *p, int64_t n, const float *v) {
  if (n >= 4) {
    *reinterpret_cast<f32x4_a4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) p[i] = v[i];
  }
}

// Rows cut into `per` chunks of 8 values (per < 2^31 - 2^16), chunks of all rows in order, `tile` of them a work-group, given to
// its threads in turn.
struct Place {
  int64_t row, col;
  bool there;
};
struct Chunks {
  int64_t row0, rows;
  uint32_t first, per;
  __device__ __forceinline__ Chunks(int64_t rows_, int64_t per_, int tile) : rows(rows_), per((uint32_t)per_) {
    const int64_t at = (int64_t)blockIdx.x * tile;
    row0 = at / per;
    first = (uint32_t)(at - row0 * per);
  }
  // chunk i of this thread
  __device__ __forceinline__ Place at(int i) const {
    const uint32_t t = first + threadIdx.x + i * blockDim.x, r = t / per;
    return {row0 + r, (int64_t)(t - r * per) * 8, row0 + r < rows};
  }
};

}  // namespace moe
#endif
