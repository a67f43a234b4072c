// head_products.hip -- the gradients of the head's rows and weights: products of float16 operands on the matrix cores, or of bf16 ones, of which
// G is the sum of two. With float16 tiles of 256 x 256 the compiler spills 15 to 18 registers, outside the main loop. Bound by the matrix cores: 8192 rows' gradient from 25152 words, width 2048, 672 to 707 us (1.19 to 1.26 PFLOP/s,
// cores busy 54%; words in rows 655 to 664, 59%); 24576 words' gradient from 8192 rows 580 to 597 us (1.38 to 1.42, 69%).
#include "head_plan.h"
#include "product_tiles.h"

namespace moe {
namespace {

template <bool HALF>
struct ResultOp {
  static constexpr bool kHalf = HALF;
  HeadResult r;
  int64_t rows, cols;
  int32_t parts;
  template <int MODE, int BM, int BN>
  __device__ __forceinline__ bool take(const ProductArgs &a, Tile *t) const {
    uint32_t tr, tc, part;
    t->expert = 0;
    t->first = 0;
    t->r1 = MODE == kOuter ? a.n : a.places;
    t->c1 = MODE == kBackward ? a.n : a.m;
    t->K = (int)(MODE == kOuter ? a.places : MODE == kBackward ? a.m : a.n);
    if (!plain_tile((uint32_t)a.row_tiles, ((uint32_t)t->c1 + BN - 1) / BN, (uint32_t)parts, &tr, &tc, &part)) return false;
    t->part = (int)part;
    t->r0 = (int64_t)tr * BM;
    t->c0 = (int64_t)tc * BN;
    return true;
  }
  template <int MODE, int FM, int FN>
  __device__ __forceinline__ void finish(const ProductArgs &a, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN],
                                         char *room) const {
    const int lane = threadIdx.x & 63;
    const int64_t row_w = t.r0 + wr, col_w = t.c0 + wc, row0 = row_w + (lane & 15), col0 = col_w + (lane >> 4) * 4;
    if (a.part) {   // the sums themselves, for join_kernel
      float *y = static_cast<float *>(a.y) + (int64_t)t.part * rows * a.ldy + row0 * a.ldy + col0;
#pragma unroll
      for (int i = 0; i < FM; i++) {
        if (row0 + i * 16 >= rows) break;
#pragma unroll
        for (int j = 0; j < FN; j++)
          if (col0 + j * 16 < cols) *reinterpret_cast<f32x4 *>(y + i * 16 * a.ldy + j * 16) = acc[i][j];   // (ldy: whole fours)
      }
      return;
    }
    const int all = !HALF || r.row_exponent ? 0 : factor_exponent(*r.coef);
    auto power = [&](int64_t at, int64_t end) { return HALF && at < end ? half_exponent(r.top[at]) + all : 0; };
    int ec[FN][4];
    if (!r.by_row) {
#pragma unroll
      for (int j = 0; j < FN; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) ec[j][q] = power(col0 + j * 16 + q, cols);
    }
    const bool f32 = r.y_dtype == SKEW_F32;
#pragma unroll
    for (int i = 0; i < FM; i++) {
      const int64_t row = row0 + i * 16;
      const int er = (r.by_row ? power(row, rows) : 0) + (HALF && r.row_exponent && row < rows ? r.row_exponent[row] : 0);
      const bool none = r.token && row < rows && r.token[row].target < 0;
#pragma unroll
      for (int j = 0; j < FN; j++) {
        const int64_t n = row < rows ? cols - col0 - j * 16 : 0;
        f32x4 v;
#pragma unroll
        for (int q = 0; q < 4; q++) {
          v[q] = HALF ? __builtin_ldexpf(acc[i][j][q], r.by_row ? er : er + ec[j][q]) : acc[i][j][q];
          if (none) v[q] = 0.0f;
        }
        if (r.prev && n > 0) {   // (rows of whole fours)
          v += *reinterpret_cast<const f32x4 *>(r.prev + row * r.ldprev + col0 + j * 16);
        }
        if (!f32) {
          put_room<FN>(room, i, j, make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])));
        } else {
          float *y = static_cast<float *>(r.y) + row * r.ldy + col0 + j * 16;
          if (n >= 4) {
            *reinterpret_cast<f32x4_a4 *>(y) = v;
          } else {
#pragma unroll
            for (int q = 0; q < 3; q++)
              if (q < n) y[q] = v[q];
          }
        }
      }
    }
    if (!f32) store_room<FM, FN, false>(room, static_cast<uint16_t *>(r.y) + row_w * r.ldy + col_w, r.ldy, rows - row_w, cols - col_w);
  }
};

template <bool HALF, int MODE, int FM, int FN, int NS, int KS>
__global__ __launch_bounds__(256, per_unit(FM, FN, KS)) void result_kernel(ProductArgs a, ResultOp<HALF> op) {
  tile_body<MODE, FM, FN, NS, KS>(a, op);
}

// Sums the parts of a shared contraction, in order, and finishes them as ResultOp does.
__global__ __launch_bounds__(256) void join_kernel(HeadResult r, int64_t rows, int64_t cols, const float *part, int parts, int64_t ld) {
  const Chunks c(rows, (cols + 7) / 8, 256);
  const Place p = c.at(0);
  if (!p.there) return;
  float v[8] = {};
#pragma unroll 4
  for (int i = 0; i < parts; i++) {
    const f32x4 *y = reinterpret_cast<const f32x4 *>(part + ((int64_t)i * rows + p.row) * ld + p.col);
    const f32x4 lo = y[0], hi = y[1];
#pragma unroll
    for (int q = 0; q < 4; q++) {
      v[q] += lo[q];
      v[4 + q] += hi[q];
    }
  }
  const int64_t n = cols - p.col;
  const bool none = r.token && r.token[p.row].target < 0;
  const int of_g = r.split ? 0 : r.row_exponent ? r.row_exponent[p.row] : factor_exponent(*r.coef);
#pragma unroll
  for (int q = 0; q < 8; q++) {
    if (none) v[q] = 0.0f;
    if (q < n && !r.split) v[q] = __builtin_ldexpf(v[q], of_g + half_exponent(r.top[r.by_row ? p.row : p.col + q]));
    if (r.prev && q < n) v[q] += r.prev[p.row * r.ldprev + p.col + q];
  }
  if (r.y_dtype == SKEW_F32) store8(static_cast<float *>(r.y) + p.row * r.ldy + p.col, n, v);
  else store8(static_cast<bf16_t *>(r.y) + p.row * r.ldy + p.col, n, v);
}

constexpr int64_t kMostGroups = 1 << 24;

// The part of a product from (row, col) on, and of its result.
HeadProduct part_of(int mode, const HeadProduct &p, int64_t row, int64_t col, int64_t rows, int64_t cols) {
  HeadProduct q = p;
  q.a = static_cast<const bf16_t *>(p.a) + (mode == kOuter ? row : row * p.lda);
  q.b = static_cast<const bf16_t *>(p.b) + (mode == kBackward ? col * p.ldb : col);
  q.rows = rows;
  q.cols = cols;
  q.pad_rows = row + rows == p.rows ? p.pad_rows - row : rows;
  q.pad_cols = col + cols == p.cols ? p.pad_cols - col : cols;
  return q;
}
HeadResult result_of(const HeadResult &r, int64_t row, int64_t col) {
  HeadResult q = r;
  q.y = static_cast<char *>(r.y) + (row * r.ldy + col) * (r.y_dtype == SKEW_F32 ? 4 : 2);
  if (r.prev) q.prev = r.prev + row * r.ldprev + col;
  if (r.top) q.top = r.top + (r.by_row ? row : col);
  if (r.row_exponent) q.row_exponent = r.row_exponent + row;
  if (r.token) q.token = r.token + row;
  return q;
}
template <bool HALF, int MODE, int FM, int FN, int NS, int KS>
int launch_one(const HeadProduct &p, const HeadResult &r, ResultChoice c, char *ws, void *stream) {
  ProductArgs a = {};
  a.x = static_cast<const bf16_t *>(p.a);   // (float16 bits)
  a.w = static_cast<const bf16_t *>(p.b);
  a.ldx = p.lda;
  a.ldw = p.ldb;
  a.k = 1;
  a.experts = 1;
  a.places = MODE == kOuter ? p.K : p.rows;
  a.n = MODE == kOuter ? p.pad_rows : MODE == kBackward ? p.pad_cols : p.K;
  a.m = MODE == kBackward ? p.K : p.pad_cols;
  a.row_tiles = (p.rows + 32 * FM - 1) / (32 * FM);
  const int64_t cols = (p.pad_cols + 32 * FN - 1) / (32 * FN);
  int parts = 1;
  const bool joined = c.parts > 1 || r.fold;
  if (joined) {
    a.part = (int32_t)(((p.K + c.parts - 1) / c.parts + 63) / 64 * 64);
    parts = (int)((p.K + a.part - 1) / a.part);
    a.y = ws;
    a.ldy = part_ld(p.cols);
  }
  const int64_t grid = plain_grid(a.row_tiles * cols * parts);
  if (grid > kMostGroups) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = static_cast<hipStream_t>(stream);
  result_kernel<HALF, MODE, FM, FN, NS, KS><<<(unsigned)grid, 256, 0, s>>>(a, ResultOp<HALF>{r, p.rows, p.cols, parts});
  const int e = (int)hipGetLastError();
  if (e != (int)hipSuccess || !joined) return e;
  const int64_t rows = r.fold ? p.rows / 2 : p.rows;   // (a part's second half is as if it were a part)
  join_kernel<<<(unsigned)((rows * (part_ld(p.cols) / 8) + 255) / 256), 256, 0, s>>>(r, rows, p.cols, reinterpret_cast<float *>(ws), r.fold ? 2 * parts : parts,
                                                                                     a.ldy);
  return (int)hipGetLastError();
}
template <bool HALF, int MODE>
int launch_choice(const HeadProduct &p, const HeadResult &r, ResultChoice c, char *ws, void *stream) {
  constexpr int S = MODE == kBackward ? 2 : 1;
  if (c.tile == 0) return launch_one<HALF, MODE, 8, 8, 4 / S, S>(p, r, c, ws, stream);
  if (c.tile == 1) return launch_one<HALF, MODE, 4, 8, 3, 1>(p, r, c, ws, stream);
  return launch_one<HALF, MODE, 2, 4, 4 / S, S>(p, r, c, ws, stream);
}
template <bool HALF, int MODE>
int launch_mode(const HeadProduct &p, const HeadResult &r, char *ws, void *stream) {
  const ResultPlan s = plan_result(MODE, p, r.fold);
  if (s.rest.parts == 0) return launch_choice<HALF, MODE>(p, r, s.main, ws, stream);
  const int e = launch_choice<HALF, MODE>(part_of(MODE, p, 0, 0, s.rows, s.cols), r, s.main, ws, stream);
  if (e != (int)hipSuccess) return e;
  const int64_t row = s.rows < p.rows ? s.rows : 0, col = s.rows < p.rows ? 0 : s.cols;
  return launch_choice<HALF, MODE>(part_of(MODE, p, row, col, p.rows - row, p.cols - col), result_of(r, row, col), s.rest, ws, stream);
}
}  // namespace

int launch_head_result(int mode, const HeadProduct &p, const HeadResult &r, char *ws, void *stream) {
  if (r.split) {
    if (mode == kOuter) return launch_mode<false, kOuter>(p, r, ws, stream);
    return mode == kBackward ? launch_mode<false, kBackward>(p, r, ws, stream) : launch_mode<false, kForward>(p, r, ws, stream);
  }
  if (mode == kOuter) return launch_mode<true, kOuter>(p, r, ws, stream);
  return mode == kBackward ? launch_mode<true, kBackward>(p, r, ws, stream) : launch_mode<true, kForward>(p, r, ws, stream);
}

}  // namespace moe
