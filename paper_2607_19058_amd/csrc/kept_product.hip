// kept_product.hip -- the experts' weights' gradient from rows kept in 8 bits.
//
// What bounds it: up to some 300 rows an expert the bytes of dW (32 experts of 2048 x 8192 with 32 rows each: 1.07 GB in 227 us, 4.7 TB/s, the
// restored rows' pass among it); beyond, the matrix cores, which are busy for 39% of the time with 512 rows each (654 to 677 us, 0.81 to 0.84 PFLOP/s):
// sixteen stages a tile, and the stores of all tiles of a round together.
//
// The values are restored into the workspace in the order of the places (with SKEW_GATHER a token's row once for each of its experts), so
// that an expert's rows of both operands are plain rows: no list of rows is looked up in the main loop, and rows of x begin
// at 16-byte positions. Rows of d that do not are copied too.
#include "kept_internal.h"
#include "product_tiles.h"

namespace moe {
namespace {

constexpr int64_t kMostGroups = 1 << 24;

// A result's tile of an expert; n and m are the results' ends, a.n and a.m those of the (padded) operands.
template <bool CHUNKS>
struct GradOp {
  static constexpr bool kHalf = false;
  int64_t n, m;
  template <int MODE, int BM, int BN>
  __device__ __forceinline__ bool take(const ProductArgs &a, Tile *t) const {
    uint32_t tr, tc, part;
    const uint32_t down = ((uint32_t)a.n + BM - 1) / BM;
    if (!plain_tile<true>(a.experts * down, ((uint32_t)a.m + BN - 1) / BN, 1, &tr, &tc, &part)) return false;
    t->expert = __builtin_amdgcn_readfirstlane(tr / down);
    t->part = 0;
    t->r0 = (int64_t)(tr - t->expert * down) * BM;
    t->r1 = a.n;
    t->c0 = (int64_t)tc * BN;
    t->c1 = a.m;
    t->first = a.offsets[t->expert];
    t->K = __builtin_amdgcn_readfirstlane(a.offsets[t->expert + 1] - (int)t->first);
    return true;
  }
  template <int MODE, int FM, int FN>
  __device__ __forceinline__ void finish(const ProductArgs &a, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN], char *room) const {
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
      for (int j = 0; j < FN; j++) {
        const f32x4 v = acc[i][j];
        put_room<FN>(room, i, j, make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])));
      }
    const int64_t row = t.r0 + wr, col = t.c0 + wc;
    store_room<FM, FN, CHUNKS>(room, static_cast<uint16_t *>(a.y) + (int64_t)t.expert * a.slice + row * a.ldy + col, a.ldy, n - row, m - col);
  }
};

template <int FM, int FN, int NS, class Op>
__global__ __launch_bounds__(256, per_unit(FM, FN, 1)) void grad_kernel(ProductArgs a, Op op) {
  tile_body<kOuter, FM, FN, NS, 1>(a, op);
}

template <int FM, int FN, int NS, bool CHUNKS>
int launch_tiles(const ProductArgs &a, int64_t n, int64_t m, hipStream_t s) {
  const int64_t grid = plain_grid(a.experts * ((a.n + 32 * FM - 1) / (32 * FM)) * ((a.m + 32 * FN - 1) / (32 * FN)));
  if (grid > kMostGroups) return (int)hipErrorInvalidConfiguration;
  grad_kernel<FM, FN, NS><<<(unsigned)grid, 256, 0, s>>>(a, GradOp<CHUNKS>{n, m});
  return (int)hipGetLastError();
}
template <bool CHUNKS>
int launch(const ProductArgs &a, int64_t n, int64_t m, hipStream_t s) {
  switch (kept_tile(a.places, a.experts, n, m)) {
    case 0: return launch_tiles<8, 8, 4, CHUNKS>(a, n, m, s);
    case 1: return launch_tiles<4, 8, 3, CHUNKS>(a, n, m, s);
    default: return launch_tiles<2, 4, 4, CHUNKS>(a, n, m, s);
  }
}

}  // namespace

int launch_grad_rows(const skew_rows &r, const skew_product_desc &p, const void *x, int64_t ldx, const void *d, int64_t ldd, void *stream) {
  ProductArgs a = {};
  a.x = static_cast<const bf16_t *>(x);
  a.w = static_cast<const bf16_t *>(d);
  a.y = const_cast<void *>(p.w);
  a.offsets = r.offsets;
  a.ldx = ldx;
  a.ldw = ldd;
  a.slice = p.slice;
  a.ldy = p.ldw;
  a.n = (p.n + 7) / 8 * 8;
  a.m = (p.m + 7) / 8 * 8;
  a.places = r.tokens * r.k;
  a.k = r.k;
  a.experts = r.experts;
  const bool chunks = ((uintptr_t)a.y & 15) == 0 && a.ldy % 8 == 0 && a.slice % 8 == 0 && p.m % 8 == 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return chunks ? launch<true>(a, p.n, p.m, s) : launch<false>(a, p.n, p.m, s);
}

}  // namespace moe
