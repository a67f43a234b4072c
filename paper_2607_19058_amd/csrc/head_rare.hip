// head_rare.hip -- the weights' gradient of words that are rare for every token, whose entries of G float16 cannot hold beside the tokens'
// factors (see rare_top): listed in order, their words gathered, their G computed again and kept beside a power of two of each word's own,
// and their part of dw written again.
//
// How many there are is known on the device alone: the grids are fixed and their work-groups go on until no tile is left. Where there are
// none the four launches end at once, after 5 to 10 us for the list and 4.5 us each (and the words' largest entries cost the logits' kernel 1.5%).
// Backward calls of 8192 tokens, 50304 words of width 2048 (untied | tied, ms), of 768 tokens (us), by the share of words that are rare:
//   none 4.45 | 4.52, 740 | 754;  1 in 200 4.69 | 4.75, 818 | 808;  1 in 20 4.94 | 4.82, 954 | 824;  all 13.1 | 11.2, 2319 | 1739
#include "head_internal.h"
#include "product_tiles.h"

namespace moe {
namespace {

constexpr int kThreads = 256, kLister = 1024, kGather = 512, kUnits = 256;
constexpr int kFM = 2, kFN = 4, kBM = 32 * kFM, kBN = 32 * kFN;   // tiles of 64 x 128: few words fill few of them

__device__ __forceinline__ int64_t up8(int64_t x) { return (x + 7) / 8 * 8; }

// One work-group; a wave looks at a run of words, 64 at a time. Bits of magnitudes are ordered as the magnitudes are. (0: no entry at all)
__global__ __launch_bounds__(kLister) void list_kernel(HeadRare r, uint32_t below) {
  constexpr int kWaves = kLister / 64;
  __shared__ int32_t held[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t each = (r.words + kLister - 1) / kLister * 64, first = wave * each, end = first + each < r.words ? first + each : r.words;
  constexpr int kAtOnce = 8;
  uint32_t t[kAtOnce];
  auto load = [&](int64_t i) {
#pragma unroll
    for (int k = 0; k < kAtOnce; k++) t[k] = i + k * 64 + lane < end ? r.word_top[i + k * 64 + lane] : 0u;
  };
  auto rare = [&](int k) { return t[k] != 0 && t[k] < below; };
  int32_t mine = 0;
  for (int64_t i = first; i < end; i += 64 * kAtOnce) {
    load(i);
#pragma unroll
    for (int k = 0; k < kAtOnce; k++) mine += __popcll(__ballot(rare(k)));
  }
  if (lane == 0) held[wave] = mine;
  __syncthreads();
  int32_t at = 0, all = 0;
  for (int i = 0; i < kWaves; i++) {
    if (i < wave) at += held[i];
    all += held[i];
  }
  if (threadIdx.x == 0) r.list[0] = all;
  if (mine == 0) return;
  for (int64_t i = first; i < end; i += 64 * kAtOnce) {
    load(i);
#pragma unroll
    for (int k = 0; k < kAtOnce; k++) {
      const uint64_t set = __ballot(rare(k));
      if (rare(k)) r.list[1 + at + __popcll(set & ((1ull << lane) - 1))] = (int32_t)(i + k * 64 + lane);
      at += __popcll(set);
    }
  }
}

// The words themselves; zeros past d.
__global__ __launch_bounds__(kThreads) void gather_kernel(HeadRare r) {
  const int64_t n = r.list[0], step = (int64_t)gridDim.x * kThreads;
  const bf16_t *w = static_cast<const bf16_t *>(r.w);
  bf16_t *copy = static_cast<bf16_t *>(r.copy);
  if (r.tied) {
    const int64_t per = r.d8 / 8;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n * per; i += step) {
      const int64_t j = i / per, col = (i - j * per) * 8;
      *reinterpret_cast<u32x4 *>(copy + j * r.ldcopy + col) = load_chunk(w + r.list[1 + j] * r.ldw + col, r.d - col);
    }
  } else {
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n * r.d8; i += step) {
      const int64_t k = i / n, j = i - k * n;
      copy[k * r.ldcopy + j] = k < r.d ? w[k * r.ldw + r.list[1 + j]] : bf16_t{0};
    }
  }
}

// Tile `at` of a result of `across` columns of tiles.
struct RareTile {
  HeadRare r;
  int64_t at, across;
  int32_t n;   // rare words
  __device__ __forceinline__ void place(Tile *t, int64_t rows, int64_t cols, int64_t K) const {
    t->expert = 0;
    t->part = 0;
    t->first = 0;
    t->K = (int)K;
    t->r0 = at / across * kBM;
    t->c0 = at % across * kBN;
    t->r1 = rows;
    t->c1 = cols;
  }
};

struct RareGradOp : RareTile {
  static constexpr bool kHalf = false;
  template <int MODE, int BM, int BN>
  __device__ __forceinline__ bool take(const ProductArgs &, Tile *t) const {
    place(t, r.tokens, up8(n), r.d8);
    return true;
  }
  // where a word is in the list; -1: nowhere
  __device__ __forceinline__ int32_t find(int64_t word) const {
    int32_t lo = 0, hi = n;
    while (lo < hi) {
      const int32_t mid = lo + (hi - lo) / 2;
      if (r.list[1 + mid] < word) lo = mid + 1;
      else hi = mid;
    }
    return lo < n && r.list[1 + lo] == word ? lo : -1;
  }
  template <int MODE, int FM, int FN>
  __device__ __forceinline__ void finish(const ProductArgs &, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN], char *room) const {
    const int lane = threadIdx.x & 63;
    const int64_t row_w = t.r0 + wr, col_w = t.c0 + wc, col0 = col_w + (lane >> 4) * 4;
    int e[FN][4];
#pragma unroll
    for (int j = 0; j < FN; j++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int64_t col = col0 + j * 16 + q;
        e[j][q] = col < n ? half_exponent(r.word_top[r.list[1 + col]]) : 0;
      }
#pragma unroll
    for (int i = 0; i < FM; i++) {
      const int64_t row = row_w + i * 16 + (lane & 15);
      HeadRow h = {0.0f, 0.0f, 0.0f, -1};
      if (row < t.r1) h = r.row[row];
      const bool token = h.target >= 0;
      const int32_t y = token ? find(h.target - r.word0) : -1;
#pragma unroll
      for (int j = 0; j < FN; j++) {
        uint32_t bits[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int64_t col = col0 + j * 16 + q;
          const float d = __builtin_fmaf(acc[i][j][q], r.c, -h.l2), p = __builtin_amdgcn_exp2f(d);
          float v = h.both * p;
          if (col == y) v = __builtin_fmaf(h.both - h.one, p, h.one * expm1f(d * 0.6931471805599453f));   // as in head_logits.hip
          if (!token || col >= n) v = 0.0f;
          bits[q] = __builtin_bit_cast(uint16_t, (_Float16)__builtin_ldexpf(v, -e[j][q]));
        }
        put_room<FN>(room, i, j, make_uint2(bits[0] | bits[1] << 16, bits[2] | bits[3] << 16));
      }
    }
    store_room<FM, FN, true>(room, r.g + row_w * r.ldg + col_w, r.ldg, t.r1 - row_w, t.c1 - col_w);
  }
};

template <int MODE, int NS, int KS>
__global__ __launch_bounds__(kThreads, per_unit(kFM, kFN, KS)) void rare_grad_kernel(ProductArgs a, HeadRare r) {
  const int32_t n = __builtin_amdgcn_readfirstlane(r.list[0]);
  const int64_t across = (n + kBN - 1) / kBN, total = (r.tokens + kBM - 1) / kBM * across;
  for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
    tile_body<MODE, kFM, kFN, NS, KS>(a, RareGradOp{{r, at, across, n}});
    __syncthreads();   // the room is stages again
  }
}

struct RareResultOp : RareTile {
  static constexpr bool kHalf = true;
  template <int MODE, int BM, int BN>
  __device__ __forceinline__ bool take(const ProductArgs &, Tile *t) const {
    place(t, r.tied ? up8(n) : r.d8, r.tied ? r.d8 : up8(n), r.tokens);
    return true;
  }
  template <int MODE, int FM, int FN>
  __device__ __forceinline__ void finish(const ProductArgs &, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN], char *) const {
    const int lane = threadIdx.x & 63;
    const int64_t row0 = t.r0 + wr + (lane & 15), col0 = t.c0 + wc + (lane >> 4) * 4;
    const int all = factor_exponent(*r.coef);
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
      for (int j = 0; j < FN; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int64_t row = row0 + i * 16, col = col0 + j * 16 + q, at = r.tied ? row : col, k = r.tied ? col : row;
          if (at >= n || k >= r.d) continue;
          const int64_t word = r.list[1 + at];
          const int e = half_exponent(r.x_top[k]) + all + half_exponent(r.word_top[word]);
          put(static_cast<bf16_t *>(r.dw) + (r.tied ? word * r.lddw + k : k * r.lddw + word), __builtin_ldexpf(acc[i][j][q], e));
        }
  }
};

__global__ __launch_bounds__(kThreads, per_unit(kFM, kFN, 1)) void rare_result_kernel(ProductArgs a, HeadRare r) {
  const int32_t n = __builtin_amdgcn_readfirstlane(r.list[0]);
  if (n == 0) return;
  const int64_t rows = r.tied ? n : r.d8, cols = r.tied ? r.d8 : n, across = (cols + kBN - 1) / kBN, total = (rows + kBM - 1) / kBM * across;
  for (int64_t at = blockIdx.x; at < total; at += gridDim.x) {
    tile_body<kOuter, kFM, kFN, 4, 1>(a, RareResultOp{{r, at, across, n}});
    __syncthreads();
  }
}

ProductArgs args_of(const void *x, int64_t ldx, const void *w, int64_t ldw) {
  ProductArgs a = {};
  a.x = static_cast<const bf16_t *>(x);
  a.w = static_cast<const bf16_t *>(w);
  a.ldx = ldx;
  a.ldw = ldw;
  a.k = 1;
  return a;
}

}  // namespace

int launch_head_rare(const HeadRare &r, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid(kUnits * per_unit(kFM, kFN, 1));
  list_kernel<<<1, kLister, 0, s>>>(r, __builtin_bit_cast(uint32_t, rare_top(r.tokens)));
  gather_kernel<<<kGather, kThreads, 0, s>>>(r);
  const ProductArgs logits = args_of(r.x, r.ldx, r.copy, r.ldcopy);
  if (r.tied) rare_grad_kernel<kBackward, 2, 2><<<grid, kThreads, 0, s>>>(logits, r);
  else rare_grad_kernel<kForward, 4, 1><<<grid, kThreads, 0, s>>>(logits, r);
  const ProductArgs result = r.tied ? args_of(r.g, r.ldg, r.x16, r.ldx16) : args_of(r.x16, r.ldx16, r.g, r.ldg);
  rare_result_kernel<<<grid, kThreads, 0, s>>>(result, r);
  return (int)hipGetLastError();
}

}  // namespace moe
