// head_loss.hip -- the head's loss: the order of its products, and the small kernels around them.
//
//   forward   logits' tiles -> a pair (largest, sum) for each row and run of columns -> loss and lse
//   backward  x and, piece by piece of the vocabulary, w to float16 beside powers of two; logits' tiles again -> G of the piece
//             (float16) -> dx += G w^T, the piece of dw = x^T G
//
// G is rounded before the products that it enters. In bf16 that would be an error of the size of the results' own rounding; in float16,
// which the matrix cores take at the same rate, it is an eighth. That needs float16 x and w: w is converted piece by
// piece (a pass of its bytes, twice read and once written), x once. For few tokens, see BackwardPlan. Words that float16 has no room for beside
// the tokens' factors get their part of dw from a second pass (head_rare.hip).
//
// What bounds them (benchmark's head, 2048 x 50304): one token's loss, w's bytes (206 MB in 32 us from the Infinity Cache, 35 from memory); 8192
// tokens, the matrix cores at the power limit (clocks of 1.75 to 2.0 of 2.4 GHz): forward 1.35 to 1.40 ms and the logits again 1.58 to 1.62 (1.2
// and 1.06 PFLOP/s; the library's plain product, with the logits written, 1.55 ms), dx 1.34 to 1.42 (the library 1.22), dw 1.24 to 1.27 (the
// library 1.68), rare words' launches 0.04.
#include <algorithm>

#include "head_plan.h"

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostGroups = 1 << 24;   // of a launch

__device__ __forceinline__ int64_t id_at(const void *ids, int bytes, int64_t i) {
  return bytes == 8 ? static_cast<const int64_t *>(ids)[i] : static_cast<const int32_t *>(ids)[i];
}
__device__ __forceinline__ bool is_token(const skew_head_desc &h, int64_t t) {
  const int64_t y = id_at(h.targets, h.target_bytes, t);
  return y >= 0 && y < h.vocab;
}
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
  return m < 0x7F800000u ? m : 0u;
}

__global__ __launch_bounds__(kThreads) void zero_kernel(uint32_t *p, int n) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i < n) p[i] = 0;
}

__global__ __launch_bounds__(kThreads) void fill_zero_kernel(bf16_t *p, int64_t rows, int64_t cols, int64_t ld) {
  const Chunks c(rows, (cols + 7) / 8, kThreads);
  const Place at = c.at(0);
  const float v[8] = {};
  if (at.there) store8(p + at.row * ld + at.col, cols - at.col, v);
}

// loss and lse of a row from its pairs: W waves a row.
struct Pair {
  float m, s;   // s 2^m
};
__device__ __forceinline__ Pair joined(Pair a, Pair b) {
  const float top = fmaxf(a.m, b.m), base = top == -INFINITY ? 0.0f : top;   // (a run past the end has -inf and 0)
  return {top, a.s * __builtin_amdgcn_exp2f(a.m - base) + b.s * __builtin_amdgcn_exp2f(b.m - base)};
}
template <int W>
__global__ __launch_bounds__(kThreads) void loss_kernel(skew_head_desc h, float c, const HeadPair *part, int64_t ld, int parts,
                                                        const float *target_sum, float *loss, float *lse) {
  constexpr int kRowsHere = kThreads / 64 / W;
  __shared__ Pair held[kThreads / 64];
  const int wave = threadIdx.x >> 6, in = threadIdx.x % (64 * W);
  const int64_t t = (int64_t)blockIdx.x * kRowsHere + wave / W;
  Pair p = {-INFINITY, 0.0f};
  if (t < h.tokens) {
#pragma unroll 4
    for (int i = in; i < parts; i += 64 * W) {
      const HeadPair q = part[t * ld + i];
      p = joined(p, {q.top, q.sum});
    }
  }
  for (int o = 32; o > 0; o >>= 1) p = joined(p, {__shfl_xor(p.m, o), __shfl_xor(p.s, o)});
  if (W > 1) {
    if ((threadIdx.x & 63) == 0) held[wave] = p;
    __syncthreads();
    p = held[wave / W * W];
#pragma unroll
    for (int i = 1; i < W; i++) p = joined(p, held[wave / W * W + i]);
  }
  if (in == 0 && t < h.tokens) {
    const bool token = is_token(h, t);
    const double all = ((double)p.m + log2((double)p.s)) * ((double)h.scale / (double)c);
    lse[t] = token ? (float)all : 0.0f;
    loss[t] = token ? (float)(all - (double)h.scale * (double)target_sum[t]) : 0.0f;
  }
}
int launch_loss(const skew_head_desc &h, float c, const HeadPair *part, int64_t ld, int parts, const float *target_sum, float *loss, float *lse,
                hipStream_t s) {
  if (h.tokens <= 64) loss_kernel<4><<<(unsigned)h.tokens, kThreads, 0, s>>>(h, c, part, ld, parts, target_sum, loss, lse);
  else loss_kernel<1><<<(unsigned)((h.tokens + 3) / 4), kThreads, 0, s>>>(h, c, part, ld, parts, target_sum, loss, lse);
  return (int)hipGetLastError();
}

// The factors of G's rows.
__device__ __forceinline__ void factors(const skew_head_desc &h, const float *dloss, const float *dlse, int64_t t, float *both, float *one) {
  *one = h.scale * dloss[t];
  *both = dlse ? h.scale * (dloss[t] + dlse[t]) : *one;
}
struct Factors {
  const float *lse, *dloss, *dlse;
  uint32_t *top;    // bits of the largest; NULL: G is split
  HeadRow *row;
  int32_t *exponent;   // of each row of G
  float c;
};
// the larger of a token's, as bits
__device__ __forceinline__ uint32_t factor_bits(const skew_head_desc &h, const Factors &f, int64_t t) {
  float both, one;
  factors(h, f.dloss, f.dlse, t, &both, &one);
  return max(finite_bits(both), finite_bits(one));
}

// The largest m of a work-group's threads, in every one of them.
__device__ __forceinline__ uint32_t largest(uint32_t m) {
  __shared__ uint32_t held[kThreads / 64];
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if ((threadIdx.x & 63) == 0) held[threadIdx.x >> 6] = m;
  __syncthreads();
  return max(max(held[0], held[1]), max(held[2], held[3]));
}

// Largest magnitudes, as bits, of the columns of `rows` x cols values: top has to be zero before. A work-group takes 256 columns of
// 8 `each` rows, a thread 8 columns of every eighth row. With `masked` rows that are no token are left out, and the work-groups past
// those of x find the largest of G's factors.
struct Tops {
  const bf16_t *x;
  int64_t ld, rows, cols;
  uint32_t *top;
  int32_t each, masked;
  int64_t groups;
};
__global__ __launch_bounds__(kThreads) void top_kernel(Tops p, skew_head_desc h, Factors f) {
  if (blockIdx.x >= p.groups) {
    uint32_t m = 0;
    const int64_t step = (int64_t)(gridDim.x - p.groups) * kThreads;
    for (int64_t t = (blockIdx.x - p.groups) * kThreads + threadIdx.x; t < h.tokens; t += step)
      if (is_token(h, t)) m = max(m, factor_bits(h, f, t));
    m = largest(m);
    if (threadIdx.x == 0 && m) atomicMax(f.top, m);
    return;
  }
  __shared__ uint32_t held[kThreads][9];
  const int64_t strips = (p.cols + 255) / 256, strip = blockIdx.x % strips, row0 = blockIdx.x / strips * (8 * p.each);
  const int64_t col = strip * 256 + (threadIdx.x & 31) * 8;
  uint32_t m[8] = {};
#pragma unroll 4
  for (int i = 0; i < p.each; i++) {
    const int64_t row = row0 + i * 8 + (threadIdx.x >> 5);
    if (row >= p.rows || col >= p.cols) continue;
    const bool token = !p.masked || is_token(h, row);
    float v[8];
    load8(p.x + row * p.ld + col, p.cols - col, v);   // (whether it is a token's or not: the loads go together)
#pragma unroll
    for (int q = 0; q < 8; q++) m[q] = max(m[q], token ? finite_bits(v[q]) : 0u);
  }
#pragma unroll
  for (int q = 0; q < 8; q++) held[threadIdx.x][q] = m[q];
  __syncthreads();
  const int c = threadIdx.x;   // a thread a column
  uint32_t all = 0;
  for (int i = 0; i < 8; i++) all = max(all, held[i * 32 + c / 8][c % 8]);
  if (strip * 256 + c < p.cols && all) atomicMax(p.top + strip * 256 + c, all);   // (an old value looked up first: 37 -> 66 us for 103 M values)
}

// 8 bf16 values to float16 times 2^-(e + more)
__device__ __forceinline__ u32x4 to_half8(u32x4 v, const int *e, int more) {
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float a = __builtin_ldexpf(__uint_as_float(v[i] << 16), -e[2 * i] - more);
    const float b = __builtin_ldexpf(__uint_as_float(v[i] & 0xFFFF0000u), -e[2 * i + 1] - more);
    u[i] = __builtin_bit_cast(uint16_t, (_Float16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)b) << 16;
  }
  return u;
}

// Values to whole rows of whole chunks (rows8 x cols8, zeros past rows and cols): float16 beside their columns' powers of two (half),
// and as they are (copy). A thread takes one chunk of columns, whose powers it loads once, of kPadRows rows. With `masked` rows that
// are no token are zeros, and the work-groups past those of x make the rows' HeadRow.
struct Padded {
  const bf16_t *x;
  int64_t ld, rows, cols, rows8, cols8, ldto;
  uint16_t *half;
  bf16_t *copy, *again;   // (two copies)
  const uint32_t *top;
  int masked;
  int64_t groups;
};
constexpr int kPadRows = 8;
__host__ __device__ inline int64_t pad_wide(int64_t cols8) { return cols8 / 8 < kThreads ? cols8 / 8 : kThreads; }   // chunks side by side
__global__ __launch_bounds__(kThreads) void pad_kernel(Padded p, skew_head_desc h, Factors f) {
  if (blockIdx.x >= p.groups) {
    const int64_t t = (blockIdx.x - p.groups) * kThreads + threadIdx.x;
    if (t >= h.tokens) return;
    HeadRow r = {0.0f, 0.0f, 0.0f, -1};
    int e = 0;
    if (is_token(h, t)) {
      factors(h, f.dloss, f.dlse, t, &r.both, &r.one);
      e = f.top ? factor_exponent(factor_bits(h, f, t)) : 0;
      r.both = __builtin_ldexpf(r.both, -e);
      r.one = __builtin_ldexpf(r.one, -e);
      r.l2 = (float)((double)f.lse[t] * ((double)f.c / (double)h.scale));
      r.target = (int32_t)id_at(h.targets, h.target_bytes, t);
    }
    f.row[t] = r;
    if (f.exponent) f.exponent[t] = e;
    return;
  }
  const uint32_t wide = (uint32_t)pad_wide(p.cols8), side = kThreads / wide, at = threadIdx.x / wide;
  const int64_t strips = (p.cols8 / 8 + kThreads - 1) / kThreads, strip = blockIdx.x % strips;
  const int64_t col = (strip * kThreads + threadIdx.x - at * wide) * 8, row0 = blockIdx.x / strips * (side * kPadRows) + at;
  if (at >= side || col >= p.cols8) return;
  u32x4 v[kPadRows];
  bool token[kPadRows];
#pragma unroll
  for (int i = 0; i < kPadRows; i++) {
    const int64_t row = row0 + (int64_t)i * side;
    v[i] = load_chunk(p.x + row * p.ld + col, row < p.rows ? p.cols - col : 0);
    token[i] = !p.masked || (row < p.rows && is_token(h, row));
  }
#pragma unroll
  for (int i = 0; i < kPadRows; i++)
    if (!token[i]) v[i] = u32x4{0, 0, 0, 0};
  int e[8], less[kPadRows];   // of the columns; how much less than the largest row of G a token's row is
#pragma unroll
  for (int q = 0; q < 8; q++) e[q] = p.half && col + q < p.cols ? half_exponent(p.top[col + q]) : 0;
#pragma unroll
  for (int i = 0; i < kPadRows; i++) {
    less[i] = 0;
    if (p.half && p.masked && token[i]) less[i] = factor_exponent(*f.top) - factor_exponent(factor_bits(h, f, row0 + (int64_t)i * side));
  }
#pragma unroll
  for (int i = 0; i < kPadRows; i++) {
    const int64_t row = row0 + (int64_t)i * side, to = row * p.ldto + col;
    if (row >= p.rows8) break;
    if (p.half) *reinterpret_cast<u32x4 *>(p.half + to) = to_half8(v[i], e, less[i]);
    if (p.copy) *reinterpret_cast<u32x4 *>(p.copy + to) = v[i];
    if (p.again) *reinterpret_cast<u32x4 *>(p.again + to) = v[i];
  }
}
// The same beside the rows' powers of two, whose largest magnitudes it finds: a work-group a row.
__global__ __launch_bounds__(kThreads) void pad_rows_kernel(Padded p, uint32_t *top) {
  const int64_t row = blockIdx.x;
  const bf16_t *x = p.x + row * p.ld;
  const int64_t cols = row < p.rows ? p.cols : 0;
  uint32_t m = 0;
#pragma unroll 4
  for (int64_t col = threadIdx.x * 8; col < cols; col += kThreads * 8) {
    float v[8];
    load8(x + col, cols - col, v);
#pragma unroll
    for (int q = 0; q < 8; q++) m = max(m, finite_bits(v[q]));
  }
  m = largest(m);
  if (threadIdx.x == 0) top[row] = m;
  int e[8];
#pragma unroll
  for (int q = 0; q < 8; q++) e[q] = half_exponent(m);
#pragma unroll 4
  for (int64_t col = threadIdx.x * 8; col < p.cols8; col += kThreads * 8) {
    const u32x4 v = load_chunk(x + col, cols - col);
    *reinterpret_cast<u32x4 *>(p.half + row * p.ldto + col) = to_half8(v, e, 0);
    if (p.copy) *reinterpret_cast<u32x4 *>(p.copy + row * p.ldto + col) = v;
  }
}

// f: also the rows of G (p.x are the tokens' rows)
int launch_pad(Padded p, const skew_head_desc &h, const Factors *f, hipStream_t s) {
  const int64_t strips = (p.cols8 / 8 + kThreads - 1) / kThreads, side = kThreads / pad_wide(p.cols8) * kPadRows;
  p.groups = strips * ((p.rows8 + side - 1) / side);
  const int64_t grid = p.groups + (f ? (h.tokens + kThreads - 1) / kThreads : 0);
  if (grid > kMostGroups) return (int)hipErrorInvalidConfiguration;
  pad_kernel<<<(unsigned)grid, kThreads, 0, s>>>(p, h, f ? *f : Factors{});
  return (int)hipGetLastError();
}
// the piece of w at v0, padded
Padded piece_of(const skew_head_desc &h, const HeadPlan &p, int64_t v0, uint16_t *half, bf16_t *copy, const uint32_t *top) {
  const int64_t cols = piece_cols(h, p, v0), cols8 = up(cols, 8);
  const bf16_t *w = reinterpret_cast<const bf16_t *>(words(h, v0));
  if (tied(h)) return {w, h.ldw, cols, h.d, cols8, p.d8, p.ldd, half, copy, nullptr, top, 0, 0};
  return {w, h.ldw, h.d, cols, p.d8, cols8, lines(cols), half, copy, nullptr, top, 0, 0};
}
// f: also the largest of G's factors
int launch_tops(const bf16_t *x, int64_t ld, int64_t rows, int64_t cols, uint32_t *top, const skew_head_desc &h, const Factors *f,
                hipStream_t s) {
  const int64_t strips = (cols + 255) / 256;
  const int each = strips * ((rows + 127) / 128) >= 512 ? 16 : 4;   // rows of a thread
  Tops p = {x, ld, rows, cols, top, each, f != nullptr, strips * ((rows + 8 * each - 1) / (8 * each))};
  const int64_t more = f ? std::min((h.tokens + kThreads - 1) / kThreads, (int64_t)64) : 0;
  if (p.groups + more > kMostGroups) return (int)hipErrorInvalidConfiguration;
  top_kernel<<<(unsigned)(p.groups + more), kThreads, 0, s>>>(p, h, f ? *f : Factors{});
  return (int)hipGetLastError();
}

// x w as they are
HeadProduct whole_of(const skew_head_desc &h) { return {h.x, h.w, h.ldx, h.ldw, h.tokens, h.vocab, h.d, 0, h.vocab}; }

float log2_scale(const skew_head_desc &h) { return (float)((double)h.scale * 1.4426950408889634); }

}  // namespace

size_t head_forward_scratch(const skew_head_desc &h) { return forward_plan(h).bytes; }
size_t head_backward_scratch(const skew_head_desc &h) { return backward_plan(h).bytes; }

int launch_fill_zero(void *dw, int64_t rows, int64_t cols, int64_t ld, void *stream) {
  const int64_t per = (cols + 7) / 8, most = (kMostGroups - 1) * kThreads / per;   // rows of a launch (a row has 2^21 chunks at most)
  for (int64_t row = 0; row < rows; row += most) {
    const int64_t n = std::min(most, rows - row);
    fill_zero_kernel<<<(unsigned)((n * per + kThreads - 1) / kThreads), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
        static_cast<bf16_t *>(dw) + row * ld, n, cols, ld);
    const int e = (int)hipGetLastError();
    if (e != (int)hipSuccess) return e;
  }
  return (int)hipSuccess;
}

#define TRY(call)                             \
  do {                                        \
    const int e_ = (call);                    \
    if (e_ != (int)hipSuccess) return e_;     \
  } while (0)

int launch_head_loss(const skew_head_desc &h, float *loss, float *lse, char *ws, void *stream) {
  const ForwardPlan f = forward_plan(h);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const float c = log2_scale(h);
  HeadPair *part = reinterpret_cast<HeadPair *>(ws + f.part);
  float *sum = reinterpret_cast<float *>(ws + f.sum);
  bf16_t *x_copy = reinterpret_cast<bf16_t *>(ws + f.x), *w_copy = reinterpret_cast<bf16_t *>(ws + f.w);
  if (f.few) {
    TRY(launch_head_few(whole_of(h), {c, h.targets, h.target_bytes, h.vocab, 0, part, f.part_ld, 0, sum}, stream));
    return launch_loss(h, c, part, f.part_ld, (int)f.part_ld, sum, loss, lse, s);
  }
  for (int64_t t0 = 0; t0 < h.tokens; t0 += f.run) {
    skew_head_desc r = h;   // this run's rows
    r.tokens = std::min(f.run, h.tokens - t0);
    r.x = static_cast<const bf16_t *>(h.x) + t0 * h.ldx;
    r.targets = static_cast<const char *>(h.targets) + t0 * h.target_bytes;
    if (!f.x_as_is)
      TRY(launch_pad({static_cast<const bf16_t *>(r.x), h.ldx, r.tokens, h.d, r.tokens, f.d8, f.ldd, nullptr, x_copy, nullptr, nullptr, 0, 0}, r, nullptr, s));
    int64_t at = 0;
    for (int64_t v0 = 0; v0 < h.vocab; v0 += f.piece) {
      if (!f.w_as_is) TRY(launch_pad(piece_of(h, f, v0, nullptr, w_copy, nullptr), r, nullptr, s));
      const HeadProduct p = logits_of(h, f, f.x_as_is ? r.x : x_copy, f.x_as_is ? h.ldx : f.ldd, r.tokens, v0, f.w_as_is ? nullptr : w_copy);
      TRY(launch_head_forward(mode_of(h), p, {c, r.targets, h.target_bytes, h.vocab, v0, part, f.part_ld, at, sum}, stream));
      at += head_parts(mode_of(h), p);
    }
    TRY(launch_loss(r, c, part, f.part_ld, (int)at, sum, loss + t0, lse + t0, s));
  }
  return (int)hipSuccess;
}

int launch_head_loss_backward(const skew_head_desc &h, const float *lse, const float *dloss, const float *dlse, void *dx, int dx_dtype,
                              int64_t lddx, void *dw, int64_t lddw, char *ws, void *stream) {
  const BackwardPlan b = backward_plan(h);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const float c = log2_scale(h);
  uint32_t *coef = reinterpret_cast<uint32_t *>(ws + b.tops), *x_top = coef + 1, *w_top = x_top + b.d8, *word_top = w_top + b.d8;
  HeadRow *row = reinterpret_cast<HeadRow *>(ws + b.row);
  uint16_t *x16 = reinterpret_cast<uint16_t *>(ws + b.x16), *w16 = reinterpret_cast<uint16_t *>(ws + b.w16),
           *g = reinterpret_cast<uint16_t *>(ws + b.g);
  bf16_t *x_copy = b.x_as_is ? nullptr : reinterpret_cast<bf16_t *>(ws + b.x), *w_copy = b.w_as_is ? nullptr : reinterpret_cast<bf16_t *>(ws + b.w);
  float *dx_sum = reinterpret_cast<float *>(ws + b.dx);
  const bf16_t *x = static_cast<const bf16_t *>(h.x);
  int32_t *exponent = reinterpret_cast<int32_t *>(ws + b.exponent);
  const Factors factors = {lse, dloss, dlse, b.split ? nullptr : coef, row, b.split ? nullptr : exponent, c};
  if (b.split) {
    bf16_t *copy = reinterpret_cast<bf16_t *>(x16);
    TRY(launch_pad({x, h.ldx, h.tokens, h.d, h.tokens, b.d8, b.ldd, nullptr, copy, copy + h.tokens * b.ldd, nullptr, 1, 0}, h, &factors, s));
  } else {
    zero_kernel<<<(unsigned)((b.top_count + kThreads - 1) / kThreads), kThreads, 0, s>>>(coef, (int)b.top_count);
    TRY((int)hipGetLastError());
    TRY(launch_tops(x, h.ldx, h.tokens, h.d, x_top, h, &factors, s));
    TRY(launch_pad({x, h.ldx, h.tokens, h.d, h.tokens, b.d8, b.ldd, x16, x_copy, nullptr, x_top, 1, 0}, h, &factors, s));
  }
  for (int64_t v0 = 0; v0 < h.vocab; v0 += b.piece) {
    const Padded p = piece_of(h, b, v0, b.split ? nullptr : w16, w_copy, w_top);
    const bool first = v0 == 0, last = v0 + b.piece >= h.vocab;
    if (b.split) {
      if (!b.w_as_is) TRY(launch_pad(p, h, nullptr, s));
    } else if (tied(h)) {
      if (!first) {
        zero_kernel<<<(unsigned)((b.d8 + kThreads - 1) / kThreads), kThreads, 0, s>>>(w_top, (int)b.d8);
        TRY((int)hipGetLastError());
      }
      TRY(launch_tops(p.x, p.ld, p.rows, p.cols, w_top, h, nullptr, s));
      TRY(launch_pad(p, h, nullptr, s));
    } else {
      pad_rows_kernel<<<(unsigned)p.rows8, kThreads, 0, s>>>(p, w_top);
      TRY((int)hipGetLastError());
    }
    const void *w = b.split ? static_cast<const void *>(w_copy) : w16;
    TRY(launch_head_grad(mode_of(h), logits_of(h, b, b.x_as_is ? h.x : x_copy, b.x_as_is ? h.ldx : b.ldd, h.tokens, v0, w_copy),
                         {c, row, h.vocab, v0, g, b.ldg, word_top}, b.split, stream));
    HeadResult to_dx = {last ? dx : dx_sum, last ? lddx : b.d8, last ? dx_dtype : SKEW_F32, first ? nullptr : dx_sum, b.d8};
    HeadResult to_dw = {static_cast<bf16_t *>(dw) + (tied(h) ? v0 * lddw : v0), lddw, SKEW_BF16, nullptr, 0};
    to_dx.split = to_dw.split = to_dx.fold = b.split;
    to_dx.token = row;
    if (!b.split) {
      to_dx.top = w_top;
      to_dx.row_exponent = exponent;
      to_dw.top = x_top;
      to_dw.by_row = !tied(h);
      to_dw.coef = coef;
    }
    TRY(launch_head_result(dx_mode(h), dx_of(h, b, g, w, v0), to_dx, ws + b.rest, stream));
    TRY(launch_head_result(kOuter, dw_of(h, b, x16, g, v0), to_dw, ws + b.rest, stream));
    if (!b.split)   // (the float16 words and G are no longer read)
      TRY(launch_head_rare({b.x_as_is ? h.x : x_copy, x16, b.x_as_is ? h.ldx : b.ldd, b.ldd, h.tokens, h.d, b.d8, words(h, v0), h.ldw,
                            piece_cols(h, b, v0), tied(h), c, row, word_top + v0, x_top, coef, v0, reinterpret_cast<int32_t *>(ws + b.list), w16,
                            tied(h) ? b.ldd : lines(b.piece), g, b.ldg, to_dw.y, lddw}, stream));
  }
  return (int)hipSuccess;
}

}  // namespace moe
