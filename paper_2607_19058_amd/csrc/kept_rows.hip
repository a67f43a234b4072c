// kept_rows.hip -- rows kept in 8 bits, and the activation between an expert's products, which keeps its inputs.
//
// A lane takes 8 neighbours of a row, 4 lanes a block of 32: one 16-byte access of bf16, 8 bytes of codes, and the block's largest
// magnitude by two exchanges inside the four lanes. A scale is a power of two, so that a code times it is a bf16 number
// and the scale comes from the exponent without a rounding.
//
// All of it is bound by memory; the activations' exponentials and divisions (some 60 instructions a value at most, of 250 that a SIMD
// has time for) hide behind it. 16384 x 8192 bf16: to 8 bits 94 us, back 67 us (together 5.2 TB/s); gated activation with its checkpoints 245 us and its
// gradient from them 259, 510 us a pass (4.7 TB/s, a copy reaches 4.9); 9003 x 2765 float32 without a gate 54 and 67 us (4.6 TB/s).
#include "moe_internal.h"
#include "kept_internal.h"

namespace moe {
namespace {

constexpr int kThreads = 256, kUnroll = 2;   // chunks of a thread
constexpr int kTile = kThreads * kUnroll;    // chunks of a work-group

template <int kPerm>   // the value of another of four neighbouring lanes
__device__ __forceinline__ uint32_t quad(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kPerm, 0xF, 0xF, true);
}

// 8 values to their codes (two words) and their block's byte. Every lane of the four takes part.
__device__ __forceinline__ uint32_t keep(const float *v, uint2 *codes) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
    top = m < 0x7F800000u && m > top ? m : top;
  }
  uint32_t o = quad<0xB1>(top);
  top = o > top ? o : top;
  o = quad<0x4E>(top);
  top = o > top ? o : top;
  // the largest is m 2^(top >> 23 - 127) with 1 <= m < 2; 127.5 = 1.9921875 2^6 (mantissa 0x7F0000);
  // scales from 2^-126 to 2^121
  const int b0 = (int)(top >> 23) - ((top & 0x7FFFFFu) > 0x7F0000u ? 5 : 6), b = b0 < 1 ? 1 : b0 > 248 ? 248 : b0;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const bool finite = (__float_as_uint(v[i]) & 0x7F800000u) != 0x7F800000u;
    float q = __builtin_rintf(__builtin_ldexpf(v[i], 127 - b));
    q = q > 127.0f ? 127.0f : q < -127.0f ? -127.0f : q;
    const int code = finite ? (int)q : -128;
    w[i >> 2] |= ((uint32_t)code & 0xFFu) << (8 * (i & 3));
  }
  *codes = make_uint2(w[0], w[1]);
  return (uint32_t)b;
}

__device__ __forceinline__ void restore(uint2 codes, uint32_t b, float *v) {
  const float s = __uint_as_float(b << 23);
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const int code = (int)((i < 4 ? codes.x : codes.y) << (24 - 8 * (i & 3))) >> 24;
    v[i] = code == -128 ? __uint_as_float(0x7FC00000u) : (float)code * s;
  }
}

// Chunks of a row in whole blocks.
__host__ __device__ inline int64_t chunks_of(int64_t cols) { return (cols + 31) / 32 * 4; }

// The place of a chunk's codes and of its block's byte.
__device__ __forceinline__ void put_kept(const Chunks &c, const Place &p, uint2 codes, uint32_t b, int8_t *at, uint8_t *scales) {
  const int64_t chunk = p.row * c.per + p.col / 8;
  *reinterpret_cast<uint2 *>(at + chunk * 8) = codes;
  if ((chunk & 3) == 0) scales[chunk >> 2] = (uint8_t)b;
}
struct KeptChunk {
  uint2 codes;
  uint32_t b;
};
__device__ __forceinline__ KeptChunk get_kept(const Chunks &c, const Place &p, const int8_t *at, const uint8_t *scales) {
  const int64_t chunk = p.row * c.per + p.col / 8;
  return {*reinterpret_cast<const uint2 *>(at + chunk * 8), scales[chunk >> 2]};
}

template <class T>
__global__ __launch_bounds__(kThreads) void keep_kernel(const T *x, int64_t rows, int64_t cols, int64_t ldx, int8_t *codes,
                                                        uint8_t *scales) {
  const Chunks c(rows, chunks_of(cols), kTile);
  float v[kUnroll][8];
  Place p[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    p[i] = c.at(i);
    load8(x + p[i].row * ldx + p[i].col, p[i].there ? cols - p[i].col : 0, v[i]);
  }
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    uint2 w;
    const uint32_t b = keep(v[i], &w);
    if (p[i].there) put_kept(c, p[i], w, b, codes, scales);
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void restore_kernel(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                                                           T *x, int64_t ldx) {
  const Chunks c(rows, chunks_of(cols), kTile);
  Place p[kUnroll];
  KeptChunk k[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    p[i] = c.at(i);
    if (p[i].there) k[i] = get_kept(c, p[i], codes, scales);
  }
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    if (!p[i].there || p[i].col >= cols) continue;
    float v[8];
    restore(k[i].codes, k[i].b, v);
    store8(x + p[i].row * ldx + p[i].col, cols - p[i].col, v);
  }
}

__global__ __launch_bounds__(kThreads) void restore_places_kernel(const int8_t *codes, const uint8_t *scales, int64_t cols, bf16_t *x,
                                                                  int64_t ldx, const int32_t *rows, int64_t places, int32_t k) {
  const Chunks c(places, chunks_of(cols), kTile);
  Place p[kUnroll];
  KeptChunk v[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    p[i] = c.at(i);
    const int32_t pair = p[i].there ? rows[p[i].row] : -1;
    p[i].there = pair >= 0;
    if (p[i].there) v[i] = get_kept(c, {pair / k, p[i].col, true}, codes, scales);
  }
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    if (!p[i].there) continue;
    float o[8];
    restore(v[i].codes, v[i].b, o);
    store8(x + p[i].row * ldx + p[i].col, 8, o);
  }
}

__global__ __launch_bounds__(kThreads) void copy_rows_kernel(const bf16_t *x, int64_t rows, int64_t cols, int64_t ldx, bf16_t *y, int64_t ldy) {
  const Chunks c(rows, ldy / 8, kTile);
  Place p[kUnroll];
  u32x4 v[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    p[i] = c.at(i);
    v[i] = load_chunk(x + p[i].row * ldx + p[i].col, p[i].there ? cols - p[i].col : 0);
  }
#pragma unroll
  for (int i = 0; i < kUnroll; i++)
    if (p[i].there) *reinterpret_cast<u32x4 *>(y + p[i].row * ldy + p[i].col) = v[i];
}

// f(g) and f'(g). s = 1 / (1 + exp(-y)) and 1 - s from exp(-|y|), so that neither cancels.
template <int KIND>
__device__ __forceinline__ void act(float g, float *f, float *df) {
  if (KIND == SKEW_ACT_RELU) {
    *f = g <= 0.0f ? 0.0f : g;
    *df = g <= 0.0f ? 0.0f : g > 0.0f ? 1.0f : g;   // (NaN stays one)
    return;
  }
  constexpr float k2 = 1.5957691216057308f;   // 2 sqrt(2 / pi)
  const float g2 = g * g;
  const float y = KIND == SKEW_ACT_SILU ? g : k2 * __builtin_fmaf(0.044715f * g2, g, g);
  const float e = expf(-fabsf(y)), r = 1.0f / (1.0f + e), er = e * r;
  const float s = y < 0.0f ? er : r, s1 = y < 0.0f ? r : er;
  *f = s == 0.0f ? 0.0f : g * s;
  const float both = KIND == SKEW_ACT_SILU ? s1 : s1 * (k2 * __builtin_fmaf(3.0f * 0.044715f, g2, 1.0f));
  *df = s == 0.0f || s1 == 0.0f ? s : __builtin_fmaf(*f, both, s);   // (0 times an infinite g^2)
}

template <class T, class O, int KIND>
__global__ __launch_bounds__(kThreads) void act_kernel(skew_act_desc d) {
  const Chunks c(d.rows, chunks_of(d.cols), kTile);
  float g[kUnroll][8], u[kUnroll][8];
  Place p[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    p[i] = c.at(i);
    const int64_t n = p[i].there ? d.cols - p[i].col : 0;
    load8(static_cast<const T *>(d.g) + p[i].row * d.ldg + p[i].col, n, g[i]);
    if (d.u) load8(static_cast<const T *>(d.u) + p[i].row * d.ldu + p[i].col, n, u[i]);
  }
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    if (d.codes_g) {
      uint2 w;
      const uint32_t b = keep(g[i], &w);
      if (p[i].there) put_kept(c, p[i], w, b, d.codes_g, d.scales_g);
    }
    if (d.codes_u) {
      uint2 w;
      const uint32_t b = keep(u[i], &w);
      if (p[i].there) put_kept(c, p[i], w, b, d.codes_u, d.scales_u);
    }
    if (!p[i].there || p[i].col >= d.cols) continue;
    float a[8], df;
#pragma unroll
    for (int j = 0; j < 8; j++) {
      act<KIND>(g[i][j], &a[j], &df);
      if (d.u) a[j] *= u[i][j];
    }
    store8(static_cast<O *>(d.a) + p[i].row * d.lda + p[i].col, d.cols - p[i].col, a);
  }
}

template <class T, class O, int KIND>
__global__ __launch_bounds__(kThreads) void act_backward_kernel(skew_act_desc d) {
  const Chunks c(d.rows, chunks_of(d.cols), kTile);
  float da[kUnroll][8];
  Place p[kUnroll];
  KeptChunk kg[kUnroll], ku[kUnroll];
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    p[i] = c.at(i);
    load8(static_cast<const T *>(d.da) + p[i].row * d.ldda + p[i].col, p[i].there ? d.cols - p[i].col : 0, da[i]);
    if (p[i].there) {
      kg[i] = get_kept(c, p[i], d.codes_g, d.scales_g);
      if (d.codes_u) ku[i] = get_kept(c, p[i], d.codes_u, d.scales_u);
    }
  }
#pragma unroll
  for (int i = 0; i < kUnroll; i++) {
    const int64_t n = d.cols - p[i].col;
    if (!p[i].there || n <= 0) continue;
    float g[8], u[8], a[8], dg[8], du[8];
    restore(kg[i].codes, kg[i].b, g);
    if (d.codes_u) restore(ku[i].codes, ku[i].b, u);
#pragma unroll
    for (int j = 0; j < 8; j++) {
      float f, df;
      act<KIND>(g[j], &f, &df);
      a[j] = d.codes_u ? f * u[j] : f;
      dg[j] = (d.codes_u ? da[i][j] * u[j] : da[i][j]) * df;
      du[j] = da[i][j] * f;
    }
    if (d.a) store8(static_cast<O *>(d.a) + p[i].row * d.lda + p[i].col, n, a);
    store8(static_cast<O *>(d.dg) + p[i].row * d.lddg + p[i].col, n, dg);
    if (d.codes_u) store8(static_cast<O *>(d.du) + p[i].row * d.lddu + p[i].col, n, du);
  }
}

int64_t groups(int64_t rows, int64_t cols) {
  return (rows * chunks_of(cols) + kTile - 1) / kTile;
}

// calls f with null pointers of the element types of in and out
template <class F>
void with_types(int in, int out, F f) {
  const bf16_t *b = nullptr;
  const float *s = nullptr;
  if (in == SKEW_BF16) out == SKEW_BF16 ? f(b, b) : f(b, s);
  else out == SKEW_BF16 ? f(s, b) : f(s, s);
}
template <class P>
struct Pointee;
template <class T>
struct Pointee<const T *> {
  typedef T type;
};

template <bool BACK>
int launch(const skew_act_desc &d, void *stream) {
  const dim3 grid((unsigned)groups(d.rows, d.cols));
  hipStream_t s = static_cast<hipStream_t>(stream);
  with_types(d.in_dtype, d.out_dtype, [&](auto in, auto out) {
    typedef typename Pointee<decltype(in)>::type T;
    typedef typename Pointee<decltype(out)>::type O;
    auto go = [&](auto kind) {
      if (BACK) act_backward_kernel<T, O, decltype(kind)::value><<<grid, kThreads, 0, s>>>(d);
      else act_kernel<T, O, decltype(kind)::value><<<grid, kThreads, 0, s>>>(d);
    };
    if (d.kind == SKEW_ACT_RELU) go(std::integral_constant<int, SKEW_ACT_RELU>());
    else if (d.kind == SKEW_ACT_SILU) go(std::integral_constant<int, SKEW_ACT_SILU>());
    else go(std::integral_constant<int, SKEW_ACT_GELU_TANH>());
  });
  return (int)hipGetLastError();
}

}  // namespace

int launch_keep8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t *codes, uint8_t *scales, void *stream) {
  const dim3 grid((unsigned)groups(rows, cols));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == SKEW_BF16) keep_kernel<<<grid, kThreads, 0, s>>>(static_cast<const bf16_t *>(x), rows, cols, ldx, codes, scales);
  else keep_kernel<<<grid, kThreads, 0, s>>>(static_cast<const float *>(x), rows, cols, ldx, codes, scales);
  return (int)hipGetLastError();
}

int launch_restore8(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, void *x, int dtype, int64_t ldx,
                    void *stream) {
  const dim3 grid((unsigned)groups(rows, cols));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == SKEW_BF16) restore_kernel<<<grid, kThreads, 0, s>>>(codes, scales, rows, cols, static_cast<bf16_t *>(x), ldx);
  else restore_kernel<<<grid, kThreads, 0, s>>>(codes, scales, rows, cols, static_cast<float *>(x), ldx);
  return (int)hipGetLastError();
}

int launch_restore_places(const skew_rows &r, const int8_t *codes, const uint8_t *scales, int64_t cols, void *x, int64_t ldx, void *stream) {
  const int64_t places = r.tokens * r.k;
  restore_places_kernel<<<(unsigned)groups(places, cols), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
      codes, scales, cols, static_cast<bf16_t *>(x), ldx, r.rows, places, r.k);
  return (int)hipGetLastError();
}

int launch_copy_rows(const void *x, int64_t rows, int64_t cols, int64_t ldx, void *y, int64_t ldy, void *stream) {
  copy_rows_kernel<<<(unsigned)((rows * (ldy / 8) + kTile - 1) / kTile), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
      static_cast<const bf16_t *>(x), rows, cols, ldx, static_cast<bf16_t *>(y), ldy);
  return (int)hipGetLastError();
}

int launch_act(const skew_act_desc &d, void *stream) { return launch<false>(d, stream); }
int launch_act_backward(const skew_act_desc &d, void *stream) { return launch<true>(d, stream); }

}  // namespace moe
