// moe_product.hip -- the experts' matrix products on the matrix cores.
//
//   forward   y[p] = s_p a_p W[e]        contraction over n: a's rows are contiguous in it, W's columns are not
//   backward  y[p] = s_p a_p W[e]^T      contraction over m: contiguous in both
//   weights   dW[e] = sum_p a_p^T d_p    contraction over an expert's places: contiguous in neither
//
// A work-group computes one tile of one expert's result. Operand tiles go through LDS in the order they
// have in memory; a lane of the matrix instruction needs 8 neighbours along the contraction, which are
// one 16-byte LDS read where memory is contiguous in it, and two transposing LDS reads (4 rows by 16 columns
// to 4 neighbours per lane) where it is not. 16-byte chunks are placed in LDS with their index xor-ed with bits of
// their row, so that the lanes of one LDS access fall into different banks.
// The matrix instruction is called with W's side first: a lane then holds 4 neighbouring columns of
// one result row, which it stores together.
#include "moe_internal.h"

namespace moe {
namespace {

enum { kForward = 0, kBackward = 1, kWeights = 2 };

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct ProductArgs {
  const bf16_t *x;
  const bf16_t *w;     // the weights; kWeights: d
  void *y;             // kWeights: dW
  const float *scale;
  const int32_t *offsets, *rows;
  int64_t ldx, ldw, slice, ldy;   // kWeights: ldw is d's row stride, ldy and slice are dW's
  int64_t n, m, places;           // n x m weights
  int32_t k, experts, gather, f32;
  int64_t row_tiles;              // forward, backward: tiles of rows in the grid
};

constexpr int kBK = 64;   // contraction length of a stage

// ---- LDS tiles ------------------------------------------------------------------------------
// Contiguous in the contraction: rows of kBK values, 8 chunks of 8.
__device__ __forceinline__ int chunk_k(int row, int c) { return row * 8 + (c ^ (row & 7)); }
// Contiguous along the result: kBK rows of W values (W / 8 chunks). A transposing read takes two
// neighbouring chunks of 4 rows in each of 4 lane groups, which are 8 rows apart.
template <int W>
__device__ __forceinline__ int chunk_t(int row, int c) {
  const int f = W >= 128 ? (row & 3) | ((row >> 1) & 4) : ((row >> 1) & 1) | ((row >> 2) & 2);
  return row * (W / 8) + (c ^ (f << 1));
}

// 8 neighbours along the contraction (k .. k + 7 with k = 32 step + 8 (lane / 16)) of row `r0 + lane % 16`
__device__ __forceinline__ bf16x8 frag_k(const u32x4 *tile, int r0, int step) {
  const int lane = threadIdx.x & 63, row = r0 + (lane & 15);
  return __builtin_bit_cast(bf16x8, tile[chunk_k(row, step * 4 + (lane >> 4))]);
}
template <int W>
__device__ __forceinline__ bf16x8 frag_t(const u32x4 *tile, int c0, int step) {
  const int lane = threadIdx.x & 63, i = lane & 15;
  const int row = step * 32 + (lane >> 4) * 8 + (i >> 2);
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const char *base = reinterpret_cast<const char *>(tile);
  const int chunk = c0 / 8 + ((i & 3) >> 1), half = (i & 1) * 8;
  s16x4 *a = reinterpret_cast<s16x4 *>(const_cast<char *>(base) + chunk_t<W>(row, chunk) * 16 + half);
  s16x4 *b = reinterpret_cast<s16x4 *>(const_cast<char *>(base) + chunk_t<W>(row + 4, chunk) * 16 + half);
  struct {
    s16x4 lo, hi;
  } v;
  v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)a);
  v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)b);
  return __builtin_bit_cast(bf16x8, v);
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

// The expert whose rows hold row tile `tile` (tiles of BM places, experts in order, then the places that
// hold no pair as a last one), and the tile's first place and end. Every wave of the work-group finds it for itself.
template <int BM>
__device__ __forceinline__ bool find_tile(const ProductArgs &a, int64_t tile, int *expert, int64_t *lo, int64_t *hi) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int e0 = 0; e0 <= a.experts; e0 += 64) {
    const int e = e0 + lane;
    int64_t b = 0, c = 0;
    if (e <= a.experts) {
      b = a.offsets[e];
      c = (e < a.experts ? (int64_t)a.offsets[e + 1] : a.places) - b;
    }
    const int mine = (int)((c + BM - 1) / BM);
    int incl = mine;
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(incl, o);
      if (lane >= o) incl += u;
    }
    const int all = __shfl(incl, 63);
    if (tile < before + all) {
      const uint64_t reached = __ballot(before + incl > tile);
      const int at = (int)__builtin_ctzll(reached);
      const int first = __shfl(incl - mine, at);
      const int64_t bb = __shfl((int)b, at), cc = __shfl((int)c, at);
      *expert = e0 + at;
      *lo = bb + (tile - before - first) * BM;
      *hi = bb + cc;
      return true;
    }
    before += all;
  }
  return false;
}

// ---- the kernel -----------------------------------------------------------------------------
template <int MODE, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM *WN * 64) void product_kernel(ProductArgs a) {
  constexpr int kThreads = WM * WN * 64;
  constexpr int kA = BM * kBK / 8, kB = BN * kBK / 8;   // chunks of a stage
  constexpr int kPA = kA / kThreads, kPB = kB / kThreads;
  constexpr int FM = BM / WM / 16, FN = BN / WN / 16;   // 16 x 16 results of a wave
  static_assert(kA % kThreads == 0 && kB % kThreads == 0, "whole chunks per thread");
  __shared__ u32x4 ta[kA], tb[kB];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wr = (wave / WN) * (BM / WM), wc = (wave % WN) * (BN / WN);

  // what this work-group computes: rows [r0, r1) and columns [c0, c1) of the result, contraction length K
  int expert;
  int64_t r0, r1, c0, c1, K, first = 0;
  if (MODE == kWeights) {
    const int64_t tn = (a.n + BM - 1) / BM, tm = (a.m + BN - 1) / BN;
    int64_t b = blockIdx.x;
    c0 = b % tm * BN;
    b /= tm;
    r0 = b % tn * BM;
    expert = (int)(b / tn);
    r1 = a.n;
    c1 = a.m;
    first = a.offsets[expert];
    K = a.offsets[expert + 1] - first;
  } else {
    const int64_t cols = MODE == kForward ? a.m : a.n, tc = (cols + BN - 1) / BN;
    if (!find_tile<BM>(a, blockIdx.x / tc, &expert, &r0, &r1)) return;
    c0 = blockIdx.x % tc * BN;
    c1 = cols;
    K = expert < a.experts ? (MODE == kForward ? a.n : a.m) : 0;   // the places without a pair: zeros
  }

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // row of x at place p
  auto source = [&](int64_t p) -> int64_t { return a.gather ? a.rows[p] / a.k : p; };
  const bf16_t *w = MODE == kWeights ? a.w : a.w + (int64_t)(K ? expert : 0) * a.slice;
  u32x4 ga[kPA], gb[kPB];
  auto load = [&](int64_t k0) {
#pragma unroll
    for (int i = 0; i < kPA; i++) {
      const int q = tid + i * kThreads;
      if (MODE == kWeights) {
        const int64_t k = k0 + q / (BM / 8), c = r0 + q % (BM / 8) * 8;
        ga[i] = k < K ? load_chunk(a.x + source(first + k) * a.ldx + c, a.n - c) : u32x4{0, 0, 0, 0};
      } else {
        const int64_t p = r0 + q / 8, k = k0 + q % 8 * 8;
        ga[i] = p < r1 ? load_chunk(a.x + source(p) * a.ldx + k, K - k) : u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll
    for (int i = 0; i < kPB; i++) {
      const int q = tid + i * kThreads;
      if (MODE == kBackward) {
        const int64_t c = c0 + q / 8, k = k0 + q % 8 * 8;
        gb[i] = c < c1 ? load_chunk(w + c * a.ldw + k, K - k) : u32x4{0, 0, 0, 0};
      } else {
        const int64_t k = k0 + q / (BN / 8), c = c0 + q % (BN / 8) * 8;
        const int64_t row = MODE == kWeights ? first + k : k;
        gb[i] = k < K ? load_chunk(w + row * a.ldw + c, c1 - c) : u32x4{0, 0, 0, 0};
      }
    }
  };
  if (K > 0) load(0);
  for (int64_t k0 = 0; k0 < K; k0 += kBK) {
#pragma unroll
    for (int i = 0; i < kPA; i++) {
      const int q = tid + i * kThreads;
      ta[MODE == kWeights ? chunk_t<BM>(q / (BM / 8), q % (BM / 8)) : chunk_k(q / 8, q % 8)] = ga[i];
    }
#pragma unroll
    for (int i = 0; i < kPB; i++) {
      const int q = tid + i * kThreads;
      tb[MODE == kBackward ? chunk_k(q / 8, q % 8) : chunk_t<BN>(q / (BN / 8), q % (BN / 8))] = gb[i];
    }
    __syncthreads();
    if (k0 + kBK < K) load(k0 + kBK);
#pragma unroll
    for (int step = 0; step < kBK / 32; step++) {
      bf16x8 fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; i++)
        fa[i] = MODE == kWeights ? frag_t<BM>(ta, wr + i * 16, step) : frag_k(ta, wr + i * 16, step);
#pragma unroll
      for (int j = 0; j < FN; j++)
        fb[j] = MODE == kBackward ? frag_k(tb, wc + j * 16, step) : frag_t<BN>(tb, wc + j * 16, step);
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  }

  // lane: result row wr + 16 i + lane % 16, columns wc + 16 j + 4 (lane / 16) .. + 3
#pragma unroll
  for (int i = 0; i < FM; i++) {
    const int64_t row = r0 + wr + i * 16 + (lane & 15);
    if (row >= r1) continue;
    const float s = MODE != kWeights && a.scale && expert < a.experts ? a.scale[a.rows[row]] : 1.0f;
    const int64_t at = MODE == kWeights ? (int64_t)expert * a.slice + row * a.ldy : row * a.ldy;
#pragma unroll
    for (int j = 0; j < FN; j++) {
      const int64_t col = c0 + wc + j * 16 + (lane >> 4) * 4;
#pragma unroll
      for (int q = 0; q < 4; q++)
        if (col + q < c1) {
          if (a.f32) static_cast<float *>(a.y)[at + col + q] = s * acc[i][j][q];
          else put(static_cast<bf16_t *>(a.y) + at + col + q, s * acc[i][j][q]);
        }
    }
  }
}

template <int MODE, int BM, int BN, int WM, int WN>
int launch(ProductArgs a, void *stream) {
  int64_t grid;
  if (MODE == kWeights) {
    grid = a.experts * ((a.n + BM - 1) / BM) * ((a.m + BN - 1) / BN);
  } else {
    const int64_t cols = MODE == kForward ? a.m : a.n;
    // an expert (and the places without a pair) ends in at most one tile that is not full
    a.row_tiles = a.places / BM + a.experts + 1 < a.places ? a.places / BM + a.experts + 1 : a.places;
    grid = a.row_tiles * ((cols + BN - 1) / BN);
  }
  if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidConfiguration;
  product_kernel<MODE, BM, BN, WM, WN><<<(unsigned)grid, WM * WN * 64, 0, static_cast<hipStream_t>(stream)>>>(a);
  return (int)hipGetLastError();
}

ProductArgs args_of(const skew_rows &r, const skew_product_desc &p) {
  ProductArgs a = {};
  a.x = static_cast<const bf16_t *>(p.x);
  a.w = static_cast<const bf16_t *>(p.w);
  a.y = p.y;
  a.scale = p.scale;
  a.offsets = r.offsets;
  a.rows = r.rows;
  a.ldx = p.ldx;
  a.ldw = p.ldw;
  a.slice = p.slice;
  a.ldy = p.ldy;
  a.n = p.n;
  a.m = p.m;
  a.places = r.tokens * r.k;
  a.k = r.k;
  a.experts = r.experts;
  a.gather = (p.flags & SKEW_GATHER) != 0;
  a.f32 = p.out_dtype == SKEW_F32;
  return a;
}

}  // namespace

size_t product_scratch(const skew_rows &, const skew_product_desc &) { return 0; }

int launch_product(const skew_rows &r, const skew_product_desc &p, char *, void *stream) {
  const ProductArgs a = args_of(r, p);
  return p.flags & SKEW_TRANSPOSE ? launch<kBackward, 64, 64, 2, 2>(a, stream) : launch<kForward, 64, 64, 2, 2>(a, stream);
}

int launch_product_grad(const skew_rows &r, const skew_product_desc &p, void *stream) {
  ProductArgs a = args_of(r, p);
  a.w = static_cast<const bf16_t *>(p.y);
  a.y = const_cast<void *>(p.w);
  a.ldw = p.ldy;
  a.ldy = p.ldw;
  a.f32 = 0;
  return launch<kWeights, 64, 64, 2, 2>(a, stream);
}

}  // namespace moe
