// head_logits.hip -- the head's logits on the matrix cores, taken from the sums' registers: their softmax sums, and
// their gradient. No logit reaches memory.
//
// A lane of a finished tile holds rows lane % 16 of FM blocks and 4 FN of each row's columns. Forward it finds their largest, adds up powers of
// two relative to it, and joins four lanes; a wave writes one pair for each row. Backward a logit becomes its gradient in
// place, which leaves through LDS as float16. Per logit that is some 32 cycles of a SIMD (16 of them the exponential's), 8200 for a tile of
// 256 x 256, beside its 64 K / 32 matrix instructions of 16. 8192 rows, 50304 words of width 2048: forward 1.35 to 1.39 ms
// (matrix cores busy 59% at 2.0 GHz, 12% of the lines missing in L2), with words in rows 1.48; the gradient 1.58 to 1.62 (49%), of which each
// word's largest entry is 1.5%. 1024 rows: 195 us. One row: 32 us for w's 206 MB.
#include "head_plan.h"
#include "product_tiles.h"

namespace moe {
namespace {

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }   // (1 ulp; 0 below 2^-126)

// The tile of a product without experts.
template <int MODE, int BM, int BN>
__device__ __forceinline__ bool take_plain(const ProductArgs &a, Tile *t) {
  uint32_t tr, tc, part;
  t->expert = 0;
  t->first = 0;
  t->part = 0;
  t->r1 = a.places;
  t->c1 = MODE == kBackward ? a.n : a.m;
  t->K = (int)(MODE == kBackward ? a.m : a.n);
  if (!plain_tile((uint32_t)a.row_tiles, ((uint32_t)t->c1 + BN - 1) / BN, 1, &tr, &tc, &part)) return false;
  t->r0 = (int64_t)tr * BM;
  t->c0 = (int64_t)tc * BN;
  return true;
}

// The element of a lane's 4 FN values that is column `at` of the wave's columns, if the lane has it.
template <int FN>
__device__ __forceinline__ bool pick(const f32x4 (&acc)[FN], int at, float *v) {
  const bool mine = at >= 0 && at < 16 * FN && ((at >> 2) & 3) == (int)((threadIdx.x & 63) >> 4);
  if (__ballot(mine) == 0) return false;
#pragma unroll
  for (int j = 0; j < FN; j++)
#pragma unroll
    for (int q = 0; q < 4; q++)
      if ((at >> 4) == j && (at & 3) == q) *v = acc[j][q];
  return mine;
}

struct ForwardOp {
  static constexpr bool kHalf = false;
  HeadForward f;
  template <int MODE, int BM, int BN>
  __device__ __forceinline__ bool take(const ProductArgs &a, Tile *t) const {
    return take_plain<MODE, BM, BN>(a, t);
  }
  template <int MODE, int FM, int FN>
  __device__ __forceinline__ void finish(const ProductArgs &a, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN], char *) const {
    const int lane = threadIdx.x & 63;
    const int64_t col_w = t.c0 + wc, row_w = t.r0 + wr + (lane & 15);
    const int64_t left = f.vocab - f.col0 - col_w;   // columns of the vocabulary from the wave's first on
    const bool whole = left >= 16 * FN;
    const int mine = (int)(left < 16 * FN ? left : 16 * FN) - (lane >> 4) * 4;
#pragma unroll
    for (int i = 0; i < FM; i++) {
      const int64_t row = row_w + i * 16;
      f32x4 v[FN];
#pragma unroll
      for (int j = 0; j < FN; j++) {
        v[j] = acc[i][j];
        if (!whole) {
#pragma unroll
          for (int q = 0; q < 4; q++)
            if (j * 16 + q >= mine) v[j][q] = -INFINITY;
        }
      }
      int64_t y = -1;
      if (row < t.r1) y = f.target_bytes == 8 ? static_cast<const int64_t *>(f.targets)[row] : static_cast<const int32_t *>(f.targets)[row];
      const int64_t at = y - f.col0 - col_w;
      float z;
      if (pick<FN>(v, y >= 0 && y < f.vocab && at >= 0 && at < 16 * FN ? (int)at : -1, &z)) f.target_sum[row] = z;
      float m = v[0][0];
#pragma unroll
      for (int j = 0; j < FN; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) m = fmaxf(m, v[j][q]);
      m *= f.c;
      const float base = m == -INFINITY ? 0.0f : m;   // (columns past the end alone)
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < FN; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) s += exp2_(__builtin_fmaf(v[j][q], f.c, -base));
      const float m16 = fmaxf(m, __shfl_xor(m, 16)), top = fmaxf(m16, __shfl_xor(m16, 32));
      s *= exp2_(m - (top == -INFINITY ? 0.0f : top));
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      if (lane < 16 && row < t.r1) f.part[row * f.part_ld + f.part_at + col_w / (16 * FN)] = HeadPair{top, s};
    }
  }
};

// The largest of 16 lanes' bits, in each of them.
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, true));   // the lanes 8, 4, 2, 1 further on
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xF, 0xF, true));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xF, 0xF, true));
}
// The largest of each column of a wave joins `to`, which is at the wave's first column: `left` columns there. Of the 4 FN columns that
// 16 lanes share, lane i takes i and (FN = 8) 16 + i.
template <int FN>
__device__ __forceinline__ void put_tops(const float (&top)[FN][4], uint32_t *to, int64_t left) {
  const int lane = threadIdx.x & 63;
  uint32_t mine[FN / 4] = {};
#pragma unroll
  for (int s = 0; s < 4 * FN; s++) {
    const uint32_t m = row_max(__float_as_uint(top[s >> 2][s & 3]));
    if ((lane & 15) == (s & 15)) mine[s >> 4] = m;
  }
#pragma unroll
  for (int i = 0; i < FN / 4; i++) {
    const int col = (i * 4 + ((lane & 15) >> 2)) * 16 + (lane >> 4) * 4 + (lane & 3);
    if (mine[i] && col < left) atomicMax(to + col, mine[i]);
  }
}

// SPLIT: the gradient is the sum of two bf16 numbers, its upper half, cut off, and the rest, which is exact before its own rounding.
template <bool SPLIT>
struct GradOp {
  static constexpr bool kHalf = false;
  HeadGrad g;
  template <int MODE, int BM, int BN>
  __device__ __forceinline__ bool take(const ProductArgs &a, Tile *t) const {
    return take_plain<MODE, BM, BN>(a, t);
  }
  // 16 bits of a value: float16; SPLIT: part 0 or 1 of it
  template <int PART>
  static __device__ __forceinline__ uint32_t bits(float x) {
    if (!SPLIT) return __builtin_bit_cast(uint16_t, (_Float16)x);
    const uint32_t u = __float_as_uint(x);
    if (PART == 0) return u >> 16;
    const bool finite = (u & 0x7F800000u) != 0x7F800000u;
    return finite ? pack2(x - __uint_as_float(u & 0xFFFF0000u), 0.0f) & 0xFFFFu : u >> 16;
  }
  template <int MODE, int FM, int FN>
  __device__ __forceinline__ void finish(const ProductArgs &a, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN],
                                         char *room) const {
    const int lane = threadIdx.x & 63;
    const int64_t col_w = t.c0 + wc, row_w = t.r0 + wr;
    const int64_t left = g.vocab - g.col0 - col_w;
    const bool whole = left >= 16 * FN;
    const int mine = (int)(left < 16 * FN ? left : 16 * FN) - (lane >> 4) * 4;
    auto part = [&](auto PART) {
      typedef uint16_t __attribute__((may_alias)) u16;
      float top[FN][4] = {};   // of the lane's columns, over its rows
#pragma unroll
      for (int i = 0; i < FM; i++) {
        const int64_t row = row_w + i * 16 + (lane & 15);
        HeadRow r = {0.0f, 0.0f, 0.0f, -1};
        if (row < t.r1) r = g.row[row];
        const bool token = r.target >= 0;
#pragma unroll
        for (int j = 0; j < FN; j++) {
          uint32_t h[4];
#pragma unroll
          for (int q = 0; q < 4; q++) {
            float v = r.both * exp2_(__builtin_fmaf(acc[i][j][q], g.c, -r.l2));
            if (!whole && j * 16 + q >= mine) v = 0.0f;
            v = token ? v : 0.0f;   // (a row that is no token may hold NaN)
            h[q] = bits<PART>(v);
            if (!SPLIT) top[j][q] = fmaxf(top[j][q], fabsf(v));
          }
          put_room<FN>(room, i, j, make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16));
        }
        const int64_t at = r.target - g.col0 - col_w;
        const int k = token && at >= 0 && at < 16 * FN ? (int)at : -1;
        float z;
        if (pick<FN>(acc[i], k, &z)) {   // both p - one, where p is near 1: (both - one) p + one (p - 1)
          const float d = __builtin_fmaf(z, g.c, -r.l2);
          const float v = __builtin_fmaf(r.both - r.one, exp2_(d), r.one * expm1f(d * 0.6931471805599453f));
          const int row16 = i * 16 + (lane & 15);
          *reinterpret_cast<u16 *>(room + row16 * (FN * 32) + ((k >> 3) ^ (row16 & 7)) * 16 + (k & 7) * 2) = (uint16_t)bits<PART>(v);
          if (!SPLIT) atomicMax(g.word_top + r.target, __float_as_uint(v) & 0x7FFFFFFFu);
        }
      }
      if (!SPLIT) put_tops<FN>(top, g.word_top + g.col0 + col_w, left);
      store_room<FM, FN, true>(room, g.g + (row_w + PART * t.r1) * g.ldg + col_w, g.ldg, t.r1 - row_w, t.c1 - col_w);
    };
    part(std::integral_constant<int, 0>());
    if constexpr (SPLIT) {
      __builtin_amdgcn_wave_barrier();   // the room is written again (the values are computed twice: registers for all of them would be more)
      part(std::integral_constant<int, 1>());
    }
  }
};

template <int MODE, int FM, int FN, int NS, int KS, class Op>
__global__ __launch_bounds__(256, per_unit(FM, FN, KS)) void logits_kernel(ProductArgs a, Op op) {
  tile_body<MODE, FM, FN, NS, KS>(a, op);
}

constexpr int64_t kMostGroups = 1 << 24;

// The columns of a product from `at` on, `cols` of them (at: a multiple of every tile's).
HeadProduct columns(int mode, const HeadProduct &p, int64_t at, int64_t cols) {
  HeadProduct q = p;
  q.b = static_cast<const bf16_t *>(p.b) + (mode == kBackward ? at * p.ldb : at);
  q.cols = cols;
  q.pad_cols = at + cols == p.cols ? p.pad_cols - at : cols;
  return q;
}

ProductArgs args_of(const HeadProduct &p, int mode, int tile) {
  ProductArgs a = {};
  a.x = static_cast<const bf16_t *>(p.a);
  a.w = static_cast<const bf16_t *>(p.b);
  a.ldx = p.lda;
  a.ldw = p.ldb;
  a.places = p.rows;
  a.n = mode == kBackward ? p.pad_cols : p.K;
  a.m = mode == kBackward ? p.K : p.pad_cols;
  a.k = 1;
  a.experts = 1;
  a.row_tiles = (p.rows + head_tile(mode == kBackward, tile).rows - 1) / head_tile(mode == kBackward, tile).rows;
  return a;
}

template <class Op, int MODE, int FM, int FN, int NS, int KS>
int launch_one(const HeadProduct &p, const Op &op, int tile, void *stream) {
  const ProductArgs a = args_of(p, MODE, tile);
  const int64_t grid = plain_grid(a.row_tiles * ((p.pad_cols + 32 * FN - 1) / (32 * FN)));
  if (grid > kMostGroups) return (int)hipErrorInvalidConfiguration;
  logits_kernel<MODE, FM, FN, NS, KS, Op><<<(unsigned)grid, 256, 0, static_cast<hipStream_t>(stream)>>>(a, op);
  return (int)hipGetLastError();
}
template <class Op, int MODE>
int launch_tiles(const HeadProduct &p, const Op &op, int tile, void *stream) {
  constexpr int S = MODE == kBackward ? 2 : 1;
  switch (tile) {
    case 0: return launch_one<Op, MODE, 8, 8, 4 / S, S>(p, op, tile, stream);
    case 1: return launch_one<Op, MODE, 4, 8, 3, 1>(p, op, tile, stream);
    case 2: return launch_one<Op, MODE, 2, 8, 4 / S, S>(p, op, tile, stream);
    default: return launch_one<Op, MODE, 2, 4, 4 / S, S>(p, op, tile, stream);
  }
}
ForwardOp shifted(const ForwardOp &op, int mode, const LogitsChoice &c) {
  ForwardOp o = op;
  o.f.col0 += c.first;
  o.f.part_at += head_runs(mode, c.tile, c.first);
  return o;
}
template <bool SPLIT>
GradOp<SPLIT> shifted(const GradOp<SPLIT> &op, int, const LogitsChoice &c) {
  GradOp<SPLIT> o = op;
  o.g.col0 += c.first;
  o.g.g += c.first;
  return o;
}
template <class Op, int MODE>
int launch_mode(const HeadProduct &p, const Op &op, void *stream) {
  const LogitsChoice c = choose_logits(MODE, p);
  if (c.first == p.cols) return launch_tiles<Op, MODE>(p, op, c.tile, stream);
  const int e = launch_tiles<Op, MODE>(columns(MODE, p, 0, c.first), op, c.tile, stream);
  if (e != (int)hipSuccess) return e;
  return launch_tiles<Op, MODE>(columns(MODE, p, c.first, p.cols - c.first), shifted(op, MODE, c), c.rest, stream);
}

}  // namespace

int launch_head_forward(int mode, const HeadProduct &p, const HeadForward &f, void *stream) {
  const ForwardOp op = {f};
  return mode == kBackward ? launch_mode<ForwardOp, kBackward>(p, op, stream) : launch_mode<ForwardOp, kForward>(p, op, stream);
}
int launch_head_grad(int mode, const HeadProduct &p, const HeadGrad &g, bool split, void *stream) {
  if (split) {
    const GradOp<true> op = {g};
    return mode == kBackward ? launch_mode<GradOp<true>, kBackward>(p, op, stream) : launch_mode<GradOp<true>, kForward>(p, op, stream);
  }
  const GradOp<false> op = {g};
  return mode == kBackward ? launch_mode<GradOp<false>, kBackward>(p, op, stream) : launch_mode<GradOp<false>, kForward>(p, op, stream);
}

}  // namespace moe
