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
//
// What bounds them: with some 300 rows an expert or fewer, the bytes of W (or of dW); with more, the matrix cores.
// Kernel times: 1024 tokens, top 2 of 128 experts of 2048 x 8192, forward: 673 us, W at 6.0 TB/s (a copy: 4.9, reads alone: 7.1). 8
// experts of 4096 x 11008 with 2048 rows each, forward: 1306 to 1452 us, 1.02 to 1.13 PFLOP/s (the library's product of that size:
// 1.25). 32 experts of 8192 x 2048 with 128 uneven rows each: backward 328 to 350 us; weights 386 to 410 us from bf16 rows (2.7 TB/s of
// dW), 497 to 528 us and 17 us for the split from float32 rows. 512 uneven rows of 2048 x 8192 each: forward 725, backward 696, weights
// 700 us (0.79 PFLOP/s), from float32 rows 1253.
#include <type_traits>

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
  int32_t direct;                 // 16-byte rows in both operands (and in a bf16 result), lengths that are multiples of 8
  int32_t wide;                   // 4 neighbouring results can be stored together
  int64_t row_tiles;              // forward, backward: tiles of rows in the grid
  int32_t in_patches;             // how tiles are given out (patch_tile)
  int32_t part;                   // forward, backward: contraction length of a work-group (a multiple of its stages)
};

constexpr int kBK = 32;   // contraction length of a step: one matrix instruction's

// ---- LDS tiles ------------------------------------------------------------------------------
// Contiguous in the contraction: rows of KS steps of kBK values, 4 KS chunks of 8. A 16-byte read takes two
// cycles of 16 lanes each: rows 0-3 and 12-15 at one chunk with rows 4-11 at the next one, and the other way about.
// KS = 1: 4 rows are as long as the banks; with the rows' groups of 4 xor-ed by 0, 2, 3, 1 the lanes fall into different banks
// (with 0, 1, 2, 3 a third of the reads' cycles were conflicts). KS = 2: 2 rows are, and the row does it.
template <int KS>
__device__ __forceinline__ int swizzle_k(int row) {
  return KS == 1 ? (((row >> 2) ^ (row >> 3)) & 1) << 1 | ((row >> 3) & 1) : row & 7;
}
// Contiguous along the result: kBK rows of W values (W / 8 chunks). A transposing read takes two
// neighbouring chunks of 4 rows in each of 4 lane groups, which are 8 rows apart.
template <int W>
__device__ __forceinline__ int swizzle_t(int row) {
  return (W >= 128 ? (row & 3) | ((row >> 1) & 4) : ((row >> 1) & 1) | ((row >> 2) & 2)) << 1;
}

__device__ __forceinline__ uint32_t lds_offset(const void *p) {
  typedef __attribute__((address_space(3))) const void lds;
  return (uint32_t)(uintptr_t)(lds *)p;
}
template <class V>
__device__ __forceinline__ const __attribute__((address_space(3))) V *lds_at(uint32_t byte) {
  return (const __attribute__((address_space(3))) V *)(uintptr_t)byte;
}

// A wave's fragments: 8 neighbours along the contraction (8 (lane / 16) .. + 7) of each of 16 result rows (lane % 16).
// get(buf, i): rows r0 + 16 i .. of the buffer `buf` bytes on. Contiguous in the contraction: fragments are a
// constant apart, as the xor takes bits of the row below 16.
template <int KS>
struct FragK {
  uint32_t at[KS];
  __device__ __forceinline__ FragK(const u32x4 *tile, int r0) {
    const int lane = threadIdx.x & 63, row = lane & 15;
#pragma unroll
    for (int k = 0; k < KS; k++)
      at[k] = lds_offset(tile) + (r0 + row) * (64 * KS) + ((k * 4 + (lane >> 4)) ^ swizzle_k<KS>(row)) * 16;
  }
  __device__ __forceinline__ bf16x8 get(int step, int i) const {
    return __builtin_bit_cast(bf16x8, *lds_at<u32x4>(at[step] + i * 1024 * KS));
  }
  __device__ __forceinline__ void move(int32_t bytes) {
#pragma unroll
    for (int k = 0; k < KS; k++) at[k] += bytes;
  }
};
// Contiguous along the result: fragments are 16 columns apart, which the xor mixes with the row.
template <int B, int F>
struct FragT {
  uint32_t at[F];
  __device__ __forceinline__ FragT(const u32x4 *tile, int c0) {
    const int lane = threadIdx.x & 63, i = lane & 15;
    const int row = (lane >> 4) * 8 + (i >> 2), chunk = c0 / 8 + ((i & 3) >> 1);
#pragma unroll
    for (int f = 0; f < F; f++)
      at[f] = lds_offset(tile) + row * (B * 2) + ((chunk + 2 * f) ^ swizzle_t<B>(row)) * 16 + (i & 1) * 8;
  }
  __device__ __forceinline__ bf16x8 get(int step, int f) const {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    struct {
      s16x4 lo, hi;   // rows row .. + 3 and, with the same xor, row + 4 .. + 7
    } v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at[f] + step * kBK * B * 2));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at[f] + (step * kBK + 4) * B * 2));
    return __builtin_bit_cast(bf16x8, v);
  }
  __device__ __forceinline__ void move(int32_t bytes) {
#pragma unroll
    for (int f = 0; f < F; f++) at[f] += bytes;
  }
};

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

// 4 neighbouring results at element `at`, of which the first n exist
__device__ __forceinline__ void store4(const ProductArgs &a, int64_t at, int64_t n, f32x4 v) {
  if (a.f32) {
    float *y = static_cast<float *>(a.y) + at;
    if (a.wide && n >= 4) {
      *reinterpret_cast<f32x4 *>(y) = v;
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++)
        if (q < n) y[q] = v[q];
    }
  } else {
    bf16_t *y = static_cast<bf16_t *>(a.y) + at;
    if (a.wide && n >= 4) {
      *reinterpret_cast<uint2 *>(y) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++)
        if (q < n) put(y + q, v[q]);
    }
  }
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
      const int bb = __shfl((int)b, at), cc = __shfl((int)c, at);
      *expert = e0 + at;
      *lo = bb + (tile - before - first) * BM;
      *hi = (int64_t)bb + cc;
      return true;
    }
    before += all;
  }
  return false;
}

// 16 bytes a lane from global memory (a scalar base and the lane's byte offset) to LDS: lane i of the wave to byte
// `to` + 16 i of LDS (`to` the same in every lane).
// Written out because the compiler, which cannot tell the stage buffers apart, would wait for these loads
// before every LDS read. It does not count them either: every use of the data comes after vm_wait() and a barrier.
// m0 is a reserved register, about which naming it warns; the compiler sets it anew for each use of its own after it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(const char *base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(__builtin_amdgcn_readfirstlane(to)),
               "v"(offset), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop
// waits until at most N of this wave's loads are on their way
template <int N>
__device__ __forceinline__ void vm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void *p) { return __builtin_amdgcn_readfirstlane(lds_offset(p)); }

// a value that is the same in every lane, as a scalar
__device__ __forceinline__ int64_t scalar(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ const char *scalar(const char *p) {
  return reinterpret_cast<const char *>(scalar((int64_t)(uintptr_t)p));
}

// Which tile a work-group takes. Work-groups go to the 8 dies in turn (id % 8), and each die has its own L2, so
// patches of kPatchR x kPatchC tiles (one for each of a die's 32 compute units) go to the dies in turn: a
// patch's tiles share their operands' rows and columns in one L2. patch_tile: false where the patch passes the edge.
// Fewer patches than kMinPatches would leave dies idle: then single tiles go to the dies in turn.
constexpr int kDies = 8, kPatchR = 4, kPatchC = 8, kMinPatches = 4 * kDies;
inline int64_t patches(int64_t rows, int64_t cols) {
  return ((rows + kPatchR - 1) / kPatchR) * ((cols + kPatchC - 1) / kPatchC);
}
inline int64_t patch_grid(int64_t rows, int64_t cols, bool in_patches) {
  return in_patches ? (patches(rows, cols) + kDies - 1) / kDies * kDies * (kPatchR * kPatchC) : rows * cols;
}
__device__ __forceinline__ bool patch_tile(bool in_patches, uint32_t rows, uint32_t cols, uint32_t *row, uint32_t *col) {
  if (!in_patches) {
    *row = blockIdx.x / cols;
    *col = blockIdx.x - *row * cols;
    return true;
  }
  const uint32_t i = blockIdx.x / kDies, in = i % (kPatchR * kPatchC);
  const uint32_t patch = i / (kPatchR * kPatchC) * kDies + blockIdx.x % kDies, pc = (cols + kPatchC - 1) / kPatchC;
  const uint32_t pr = patch / pc;
  *row = pr * kPatchR + in % kPatchR;
  *col = (patch - pr * pc) * kPatchC + in / kPatchR;
  return *row < rows && *col < cols;
}

// acc += the product of two fragments (result rows along the second). IN_A: the sums stay in the accumulation
// registers, which the compiler, left to itself, copies to others and back when they are 256 of a lane's 512.
// It does not know the written-out instruction's latency: the sums go through mfma_done() before they are read.
template <bool IN_A>
__device__ __forceinline__ void mfma(f32x4 &acc, bf16x8 b, bf16x8 a) {
  if (IN_A) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
  else acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, acc, 0, 0, 0);
}
template <int FM, int FN>
__device__ __forceinline__ void mfma_done(f32x4 (&acc)[FM][FN]) {
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) asm volatile("" : "+a"(acc[i][j]));   // what reads them depends on this, which stays behind the wait
}

// What a tiled work-group computes: rows [r0, r1) and columns [c0, c1) of the result of one expert, contraction length K;
// kWeights: places first .. first + K - 1.
struct Tile {
  int expert, K;
  int64_t r0, r1, c0, c1, first;
};
template <int MODE, int BM, int BN>
__device__ __forceinline__ bool take_tile(const ProductArgs &a, Tile *t) {
  uint32_t tr, tc;   // (the grid has fewer than 2^31 tiles)
  t->first = 0;
  t->c1 = MODE == kBackward ? a.n : a.m;
  const uint32_t cols = ((uint32_t)t->c1 + BN - 1) / BN;
  if (MODE == kWeights) {
    const uint32_t tn = ((uint32_t)a.n + BM - 1) / BM;
    if (!patch_tile(a.in_patches, a.experts * tn, cols, &tr, &tc)) return false;
    t->expert = __builtin_amdgcn_readfirstlane(tr / tn);
    t->r0 = (int64_t)(tr - t->expert * tn) * BM;
    t->r1 = a.n;
    t->first = a.offsets[t->expert];
    t->K = __builtin_amdgcn_readfirstlane(a.offsets[t->expert + 1] - (int)t->first);
  } else {
    if (!patch_tile(a.in_patches, (uint32_t)a.row_tiles, cols, &tr, &tc) || !find_tile<BM>(a, tr, &t->expert, &t->r0, &t->r1))
      return false;
    t->expert = __builtin_amdgcn_readfirstlane(t->expert);   // the same in every lane, but found in a loop over lanes
    t->r0 = scalar(t->r0);
    t->r1 = scalar(t->r1);
    t->K = t->expert < a.experts ? (int)(MODE == kForward ? a.n : a.m) : 0;   // the places without a pair: zeros
  }
  t->c0 = (int64_t)tc * BN;
  return true;
}

// Stores a wave's FM x FN blocks of 16 x 16 results from row wr and column wc of the tile. A lane holds row
// lane % 16 of each block and its columns 4 (lane / 16) .. + 3.
// bf16 results go through `room` (FM FN 512 bytes of LDS of this wave's own), so that a row's 32 FN bytes leave
// together: 8-byte stores of 16 rows at once reached 3.1 TB/s on a gradient that is all output.
template <int MODE, int FM, int FN, bool CHUNKS>
__device__ __forceinline__ void store_tile(const ProductArgs &a, const Tile &t, int wr, int wc, const f32x4 (&acc)[FM][FN],
                                           char *room) {
  const int lane = threadIdx.x & 63;
  const int64_t row0 = t.r0 + wr + (lane & 15), col0 = t.c0 + wc + (lane >> 4) * 4;
  float s[FM];
#pragma unroll
  for (int i = 0; i < FM; i++) s[i] = 1.0f;
  if (MODE != kWeights && a.scale && t.expert < a.experts) {
#pragma unroll
    for (int i = 0; i < FM; i++)
      if (row0 + i * 16 < t.r1) s[i] = a.scale[a.rows[row0 + i * 16]];
  }
  if (MODE == kWeights || !a.f32) {
    constexpr int kChunks = 2 * FN;   // of a row, placed with their index xor-ed with the row
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
      for (int j = 0; j < FN; j++) {
        const int row = i * 16 + (lane & 15), c = 2 * j + (lane >> 5);
        const f32x4 v = s[i] * acc[i][j];
        *reinterpret_cast<uint2 *>(room + row * (kChunks * 16) + (c ^ (row & 7)) * 16 + (lane >> 4 & 1) * 8) =
            make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int kRows = 64 / kChunks;   // rows of one store
    const int c = lane % kChunks, row_in = lane / kChunks;
    const int64_t col = t.c0 + wc + c * 8, left = t.r1 - (t.r0 + wr);
    const int rows = left < 16 * FM ? (int)left : 16 * FM, n = (int)(t.c1 - col < 8 ? t.c1 - col : 8);   // of the wave's; of the lane's 8 columns
    bf16_t *y = static_cast<bf16_t *>(a.y) + (MODE == kWeights ? (int64_t)t.expert * a.slice : 0) +
                (t.r0 + wr + row_in) * a.ldy + col;
    const int64_t step = kRows * a.ldy;
    auto read = [&](int i) {
      const int row = i * kRows + row_in;
      return *reinterpret_cast<const u32x4 *>(room + row * (kChunks * 16) + (c ^ (row & 7)) * 16);
    };
    if (CHUNKS) {   // not a case of the loop below: its reads wait for each other, and its code is in the registers' way
#pragma unroll
      for (int i = 0; i < 16 * FM / kRows; i++, y += step) {
        const u32x4 v = read(i);
        if (i * kRows + row_in < rows && n > 0) *reinterpret_cast<u32x4 *>(y) = v;
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 16 * FM / kRows; i++, y += step) {
      const u32x4 v = read(i);
      if (i * kRows + row_in >= rows || n <= 0) continue;
      if (n == 8) {
        *reinterpret_cast<u32x4_a2 *>(y) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 7; e++)
          if (e < n) y[e].v = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
      }
    }
    return;
  }
  float *y = static_cast<float *>(a.y) + row0 * a.ldy + col0;   // (dW is bf16)
#pragma unroll
  for (int i = 0; i < FM; i++) {
    if (row0 + i * 16 >= t.r1) break;
#pragma unroll
    for (int j = 0; j < FN; j++) {
      const f32x4 v = s[i] * acc[i][j];
      float *at = y + i * 16 * a.ldy + j * 16;
      const int64_t n = t.c1 - col0 - j * 16;
      if (n >= 4) {
        *reinterpret_cast<f32x4_a4 *>(at) = v;
      } else {
#pragma unroll
        for (int q = 0; q < 3; q++)
          if (q < n) at[q] = v[q];
      }
    }
  }
}

// ---- tiles whose chunks go from memory to LDS without registers ---------------------------------
// For rows at 16-byte positions and lengths that are multiples of 8, so that a chunk is inside its row or outside.
// Tiles of 32 FM x 32 FN results, 4 waves, each FM x FN matrix instructions a stage; NS LDS buffers of a stage.
// A stage is KS steps. While a wave multiplies one step from registers it reads the next one from LDS into other registers
// and sends for a stage further on, one load or fragment after every few matrix instructions. A load's address is a
// scalar, which moves from stage to stage, plus a lane's 32-bit offset, which stays.
// Rows and columns past the edge of the result repeat the last one inside and are not stored; past the end of the
// contraction both operands are zero, so nothing there meets a NaN.
constexpr int kList = 1024;   // places whose rows kWeights looks up at once

template <int MODE, int FM, int FN, int NS, int KS>
__global__ __launch_bounds__(256, FM * FN * KS >= 64 ? 1 : FM * FN == 8 ? 3 : 2) void tile_kernel(ProductArgs a) {
  constexpr int BM = 32 * FM, BN = 32 * FN, BK = KS * kBK, kThreads = 256;
  constexpr int kCA = BM * BK / 8, kCB = BN * BK / 8, kPA = kCA / kThreads, kPB = kCB / kThreads;   // chunks of a stage
  constexpr int kBytesA = kCA * 16, kBytesB = kCB * 16, kLoads = kPA + kPB;
  constexpr bool kInA = FM * FN == 64;
  constexpr int kAhead = KS == 1 ? NS - 1 : NS;   // a stage of two steps is sent for when its buffer's second step was read
  static_assert(FM * FN * 512 * 4 <= NS * (kBytesA + kBytesB), "room for the results");
  static_assert(kPA * kThreads == kCA && kPB * kThreads == kCB, "whole chunks per thread");
  __shared__ u32x4 lds[NS * (kCA + kCB) + (MODE == kWeights ? kList / 4 : 0)];
  u32x4 *const ta = lds, *const tb = lds + NS * kCA;
  uint32_t *const list = reinterpret_cast<uint32_t *>(tb + NS * kCB);   // byte offsets of x's rows
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = (wave >> 1) * (BM / 2), wc = (wave & 1) * (BN / 2);
  Tile t;
  if (!take_tile<MODE, BM, BN>(a, &t)) return;
  int K = t.K;

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // Slot i of this thread is chunk q = tid + i kThreads of a stage's tile in LDS. A tile that is contiguous in the
  // contraction holds result row q / (4 KS) and chunk (q % (4 KS)) ^ swizzle there; one that is not holds contraction row
  // q / (tile width / 8) likewise. ka, kb: the slot's contraction index in its stage; oa, ob: its byte offset from xa, xb, where
  // the next stage that is sent for begins (kWeights: oa without the row of x).
  const char *xa = reinterpret_cast<const char *>(a.x), *xb = reinterpret_cast<const char *>(a.w);
  int64_t step_a = 0, step_b;
  if (MODE == kWeights) {
    xb += 2 * t.first * a.ldw;
  } else {
    xb += 2 * (int64_t)(K ? t.expert : 0) * a.slice;
    if (!a.gather) xa += 2 * t.r0 * a.ldx;
    step_a = 2 * BK;
  }
  step_b = MODE == kBackward ? 2 * BK : 2 * BK * a.ldw;
  if (MODE != kWeights && a.part) {   // this work-group's part of a contraction that several share
    const int k0 = (int)blockIdx.y * a.part;
    K = K - k0 < a.part ? (K > k0 ? K - k0 : 0) : a.part;
    if (K > 0) {
      xa += k0 / BK * step_a;
      xb += k0 / BK * step_b;
    }
  }
  if (MODE == kBackward) xb += 2 * t.c0 * a.ldw;
  xa = scalar(xa);
  xb = scalar(xb);
  step_b = scalar(step_b);
  uint32_t oa[kPA], ob[kPB];
  int ka[kPA], kb[kPB];
#pragma unroll
  for (int i = 0; i < kPA; i++) {
    const int q = tid + i * kThreads;
    if (MODE == kWeights) {
      const int row = q / (BM / 8), c = (q % (BM / 8)) ^ swizzle_t<BM>(row);
      ka[i] = row;
      oa[i] = (uint32_t)(2 * (t.r0 + c * 8 < t.r1 ? t.r0 + c * 8 : t.r1 - 8));
    } else {
      const int row = q / (4 * KS), c = (q % (4 * KS)) ^ swizzle_k<KS>(row);
      const int r = t.r0 + row < t.r1 ? row : (int)(t.r1 - 1 - t.r0);
      ka[i] = c * 8;
      oa[i] = (uint32_t)((K > 0 && a.gather ? (int64_t)(a.rows[t.r0 + r] / a.k) : r) * a.ldx + c * 8) * 2;
    }
  }
#pragma unroll
  for (int i = 0; i < kPB; i++) {
    const int q = tid + i * kThreads;
    if (MODE == kBackward) {
      const int row = q / (4 * KS), c = (q % (4 * KS)) ^ swizzle_k<KS>(row);
      kb[i] = c * 8;
      ob[i] = (uint32_t)((t.c0 + row < t.c1 ? row : t.c1 - 1 - t.c0) * a.ldw + c * 8) * 2;
    } else {
      const int row = q / (BN / 8), c = (q % (BN / 8)) ^ swizzle_t<BN>(row);
      kb[i] = row;
      ob[i] = (uint32_t)(row * a.ldw + (t.c0 + c * 8 < t.c1 ? t.c0 + c * 8 : t.c1 - 8)) * 2;
    }
  }
  // W's rows in the contraction are a power of two apart in most models, so that tiles at the same place of their rows ask the
  // same memory channels: the tiles of a row of tiles begin at different stages and go round.
  int turn = -1, sent_at = 0;
  if (MODE == kBackward && K % BK == 0 && K > 0) {
    turn = K / BK;
    sent_at = __builtin_amdgcn_readfirstlane((int)((t.c0 / BN * 3 + t.expert) % turn));
    xa += sent_at * step_a;
    xb += sent_at * step_b;
  }
  const uint32_t la = lds_address(ta + wave * 64), lb = lds_address(tb + wave * 64);

  int reading = 0, sending = 0;   // buffers of the stages that are read, and sent for, next
  int base = 0, end = K;   // the contraction [base, end) of this round (kWeights: the places in the list)
  uint32_t row_next[kPA];   // kWeights: the rows of x of the next stage that is sent for
  auto look_up = [&](int stage) {
    if (MODE == kWeights) {
#pragma unroll
      for (int i = 0; i < kPA; i++) row_next[i] = list[(stage * BK + ka[i]) & (kList - 1)];
    }
  };
  // load i of a stage: the slots of a, then those of b
  auto send = [&](int i) {
    if (i < kPA) load_lds(xa, oa[i < kPA ? i : 0] + (MODE == kWeights ? row_next[i < kPA ? i : 0] : 0),
                          la + sending * kBytesA + i * kThreads * 16);
    else load_lds(xb, ob[i < kPA ? 0 : i - kPA], lb + sending * kBytesB + (i - kPA) * kThreads * 16);
  };
  auto sent_all = [&]() {
    xa += step_a;
    xb += step_b;
    sending = sending + 1 == NS ? 0 : sending + 1;
    if (MODE == kBackward && ++sent_at == turn) {   // round the end of the contraction
      xa -= turn * step_a;
      xb -= turn * step_b;
      sent_at = 0;
    }
  };
  // the same for any stage, also one that the contraction ends in
  auto send_stage = [&](int stage) {
    const int left = end - base - stage * BK;
    look_up(stage);
    if (left >= BK) {
#pragma unroll
      for (int i = 0; i < kLoads; i++) send(i);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; i++) {
        const bool is_a = i < kPA;
        const int sl = is_a ? i : i - kPA;
        if ((is_a ? ka[is_a ? sl : 0] : kb[is_a ? 0 : sl]) < left) send(i);
        else if (is_a) ta[sending * kCA + tid + sl * kThreads] = u32x4{0, 0, 0, 0};
        else tb[sending * kCB + tid + sl * kThreads] = u32x4{0, 0, 0, 0};
      }
    }
    sent_all();
  };

  // this lane's fragments, in the buffer of the stage that is read next
  FragK<KS> ra_k(ta, wr), rb_k(tb, wc);
  FragT<BM, FM> ra_t(ta, wr);
  FragT<BN, FN> rb_t(tb, wc);
  bf16x8 fa[2][FM], fb[2][FN];
  auto read_a = [&](int k, int i, bf16x8 *d) { d[i] = MODE == kWeights ? ra_t.get(k, i) : ra_k.get(k, i); };
  auto read_b = [&](int k, int i, bf16x8 *d) { d[i] = MODE == kBackward ? rb_k.get(k, i) : rb_t.get(k, i); };
  auto advance = [&]() {
    const bool wrap = reading + 1 == NS;
    const int32_t by_a = wrap ? -(NS - 1) * kBytesA : kBytesA, by_b = wrap ? -(NS - 1) * kBytesB : kBytesB;
    if (MODE == kWeights) ra_t.move(by_a);
    else ra_k.move(by_a);
    if (MODE == kBackward) rb_k.move(by_b);
    else rb_t.move(by_b);
    reading = wrap ? 0 : reading + 1;
  };
  // multiply fragments X; NEXT: read step k of the stage that is read next into the others; MORE: send for a
  // stage. The loads come first.
  auto step = [&](auto X, auto NEXT, auto MORE, int k) {
    constexpr int x = X, y = 1 - x, kDo = (MORE ? kLoads : 0) + (NEXT ? FM + FN : 0);
    auto due = [](int m) { return m >= FM * FN - 2 ? kDo : m * kDo / (FM * FN - 2); };   // how many come before instruction m
#pragma unroll
    for (int m = 0; m < FM * FN; m++) {
      mfma<kInA>(acc[m / FN][m % FN], fb[x][m % FN], fa[x][m / FN]);
#pragma unroll
      for (int d = due(m); d < due(m + 1); d++) {
        const int r = d - (MORE ? kLoads : 0);
        if (r < 0) send(d);
        else if (r < FM) read_a(k, r, fa[y]);
        else read_b(k, r - FM, fb[y]);
      }
    }
    if (MORE) sent_all();
    if (NEXT && k == KS - 1) advance();
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  const std::true_type yes;
  const std::false_type no;

  for (; base < K; base = end) {
    if (MODE == kWeights) {
      end = base + round_length(base, K, kList);
      __syncthreads();   // the list of the round before is no longer read
      for (int i = tid; i < end - base; i += kThreads) {
        const int64_t p = t.first + base + i;
        list[i] = (uint32_t)((a.gather ? (int64_t)(a.rows[p] / a.k) : p) * a.ldx * 2);
      }
      __syncthreads();
    }
    const int S = (end - base + BK - 1) / BK;
    for (int i = 0; i < kAhead && i < S; i++) send_stage(i);
    // of the stages that were sent for, all but `n` have arrived in every wave
    auto meet = [&](bool whole, auto n) {
      if (whole) vm_wait<n * kLoads>();
      else vm_wait<0>();   // the last stage may have sent for less than kLoads loads
      __syncthreads();
    };
    const std::integral_constant<int, kAhead - 1> one;    // one stage is there
    const std::integral_constant<int, kAhead - 2> two;
    meet(S > kAhead, one);
#pragma unroll
    for (int i = 0; i < FM; i++) read_a(0, i, fa[0]);
#pragma unroll
    for (int i = 0; i < FN; i++) read_b(0, i, fb[0]);
    if (KS == 1) advance();
    int s = 0;
    if constexpr (KS == 1) {
      // Before stage s: stage s + 1 is there, and the buffer of stage s + kAhead is no longer read.
      look_up(kAhead);
      for (; s + kAhead + 2 < S; s += 2) {    // sends for stages s + kAhead and s + kAhead + 1, which are whole
        meet(true, two);
        step(even, yes, yes, 0);
        look_up(s + kAhead + 1);
        meet(true, two);
        step(odd, yes, yes, 0);
        look_up(s + kAhead + 2);
      }
      for (; s + 1 < S; s += 2) {
        meet(s + kAhead < S, two);
        if (s + kAhead < S) send_stage(s + kAhead);
        step(even, yes, no, 0);
        meet(s + kAhead + 1 < S, two);
        if (s + kAhead + 1 < S) send_stage(s + kAhead + 1);
        step(odd, yes, no, 0);   // at the end of an even number of stages this reads what is not used
      }
      if (s < S) step(even, no, no, 0);
    } else {
      // Between a stage's steps: stage s + 1 is there, and the buffer of stage s, the one of s + kAhead, is no longer read.
      auto first_step = [&]() {
        step(even, yes, no, 1);
      };
      for (; s + kAhead + 1 < S; s++) {   // sends for stage s + kAhead, which is whole
        first_step();
        meet(true, two);
        step(odd, yes, yes, 0);
      }
      for (; s < S; s++) {
        first_step();
        meet(s + kAhead < S, two);
        if (s + kAhead < S) send_stage(s + kAhead);
        step(odd, yes, no, 0);   // of the last stage: reads what is not used
      }
    }
    if (kInA) mfma_done(acc);   // here, not after the loop: where a contraction may be empty, the sums are copied on the loop's way out
    // the next round, if any, starts in the buffer that is sent for next
    while (reading != sending) advance();
    __syncthreads();   // the buffers are no longer read
  }
  if (MODE != kWeights && a.part) a.y = static_cast<float *>(a.y) + (int64_t)blockIdx.y * a.places * a.ldy;
  store_tile<MODE, FM, FN, true>(a, t, wr, wc, acc, reinterpret_cast<char *>(lds) + wave * (FM * FN * 512));
}

// ---- tiles of any shape ---------------------------------------------------------------------
// The same tiles through registers: the next stage's chunks are loaded from any position while a stage is multiplied. Where
// the result is at least a tile wide, its last tile is moved back inside (its results are computed twice, from the same
// numbers in the same order), so that all chunks but those at the end of the contraction are whole; else, and
// there, chunks are loaded element by element. At 2-byte positions that are no 4-byte ones a 16-byte load takes four
// times as long (from L2 9.5 TB/s, else 35). 16 experts of 2765 x 1031 with 563 rows each, forward: 133 us, 0.39 PFLOP/s;
// with 2760 x 1032, through tile_kernel: 97 us. Calls: forward 145, backward 154, weights 146 us; 2760 x 1032: 113, 143, 116.
// The 4 x 8 tiles are short of registers: the compiler spills 6 vector ones forward and 15 in the weights' kernel, outside
// the main loops.
template <int MODE, int FM, int FN, int kSets>
__global__ __launch_bounds__(256, 2) void any_kernel(ProductArgs a) {
  constexpr int BM = 32 * FM, BN = 32 * FN, kThreads = 256;
  constexpr int kCA = BM * kBK / 8, kCB = BN * kBK / 8, kPA = kCA / kThreads, kPB = kCB / kThreads;
  static_assert(kPA * kThreads == kCA && kPB * kThreads == kCB, "whole chunks per thread");
  constexpr int kRoom = FM * FN * 128;   // chunks of the tile's bf16 results
  __shared__ u32x4 lds[kRoom > 2 * kCA + 2 * kCB ? kRoom : 2 * kCA + 2 * kCB];
  u32x4 *const ta = lds, *const tb = lds + 2 * kCA;
  __shared__ int32_t list[MODE == kWeights ? kList : 1];   // x's rows
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = (wave >> 1) * (BM / 2), wc = (wave & 1) * (BN / 2);
  Tile t;
  if (!take_tile<MODE, BM, BN>(a, &t)) return;
  if (t.c0 + BN > t.c1 && t.c1 >= BN) t.c0 = t.c1 - BN;
  if (MODE == kWeights && t.r0 + BM > t.r1 && t.r1 >= BM) t.r0 = t.r1 - BM;
  int K = t.K, k_first = 0;   // this work-group's part of the contraction
  if (MODE != kWeights && a.part) {
    k_first = (int)blockIdx.y * a.part;
    K = K - k_first < a.part ? (K > k_first ? K - k_first : 0) : a.part;
  }
  const bool inside = t.c0 + BN <= t.c1 && (MODE != kWeights || t.r0 + BM <= t.r1);

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // slots as in tile_kernel; na, nb: how many of the chunk's values are in the row
  const bf16_t *w = MODE == kWeights ? a.w + t.first * a.ldw : a.w + (int64_t)(K ? t.expert : 0) * a.slice;
  const bf16_t *pa[kPA], *pb[kPB];
  int ka[kPA], kb[kPB], na[kPA], nb[kPB];
  auto clip = [](int64_t x) { return (int)(x < 0 ? 0 : x > 8 ? 8 : x); };
#pragma unroll
  for (int i = 0; i < kPA; i++) {
    const int q = tid + i * kThreads;
    if (MODE == kWeights) {
      const int row = q / (BM / 8), c = (q % (BM / 8)) ^ swizzle_t<BM>(row);
      ka[i] = row;
      na[i] = clip(t.r1 - (t.r0 + c * 8));
      pa[i] = a.x + t.r0 + c * 8;
    } else {
      const int row = q / 4, c = (q % 4) ^ swizzle_k<1>(row);
      const int64_t p = t.r0 + row < t.r1 ? t.r0 + row : t.r1 - 1;
      ka[i] = c * 8;
      na[i] = 8;
      pa[i] = a.x + (K > 0 && a.gather ? (int64_t)(a.rows[p] / a.k) : p) * a.ldx + k_first + c * 8;
    }
  }
#pragma unroll
  for (int i = 0; i < kPB; i++) {
    const int q = tid + i * kThreads;
    if (MODE == kBackward) {
      const int row = q / 4, c = (q % 4) ^ swizzle_k<1>(row);
      kb[i] = c * 8;
      nb[i] = 8;
      pb[i] = w + (t.c0 + row < t.c1 ? t.c0 + row : t.c1 - 1) * a.ldw + k_first + c * 8;
    } else {
      const int row = q / (BN / 8), c = (q % (BN / 8)) ^ swizzle_t<BN>(row);
      kb[i] = row;
      nb[i] = clip(t.c1 - (t.c0 + c * 8));
      pb[i] = w + (int64_t)(k_first + row) * a.ldw + t.c0 + c * 8;
    }
  }
  // kSets stages are on their way into registers, set by set
  u32x4 ga[kSets][kPA], gb[kSets][kPB];
  // Unsigned, as stages past the end of 2^31 - 1 places begin beyond it.
  uint32_t base = 0, end = 0;   // kWeights: the places in the list
  auto load = [&](auto SET, auto WHOLE, uint32_t k0) {
    const int64_t ob = MODE == kBackward ? k0 : k0 * a.ldw;
#pragma unroll
    for (int i = 0; i < kPA; i++) {
      const int left = (int)(end - k0) - ka[i];   // contraction values from this chunk on
      const bf16_t *p = pa[i] + (MODE != kWeights ? k0 : WHOLE || left > 0 ? list[k0 - base + ka[i]] * a.ldx : 0);
      if (WHOLE) ga[SET][i] = *reinterpret_cast<const u32x4_a2 *>(p);
      else ga[SET][i] = left > 0 ? load_chunk(p, MODE == kWeights ? na[i] : left) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < kPB; i++) {
      const int left = (int)(end - k0) - kb[i];
      if (WHOLE) gb[SET][i] = *reinterpret_cast<const u32x4_a2 *>(pb[i] + ob);
      else gb[SET][i] = left > 0 ? load_chunk(pb[i] + ob, MODE == kBackward ? left : nb[i]) : u32x4{0, 0, 0, 0};
    }
  };
  auto put_stage = [&](auto SET, int buf) {
#pragma unroll
    for (int i = 0; i < kPA; i++) ta[buf * kCA + tid + i * kThreads] = ga[SET][i];
#pragma unroll
    for (int i = 0; i < kPB; i++) tb[buf * kCB + tid + i * kThreads] = gb[SET][i];
  };
  FragK<1> ra_k(ta, wr), rb_k(tb, wc);
  FragT<BM, FM> ra_t(ta, wr);
  FragT<BN, FN> rb_t(tb, wc);
  int buf = 0;   // the buffer of the stage that is multiplied
  // one stage: the next one goes from SET to the other buffer, and the stage at `ahead` is sent for into SET
  auto stage = [&](auto SET, auto WHOLE, uint32_t ahead) {
    __syncthreads();
    put_stage(SET, buf ^ 1);
    load(SET, WHOLE, ahead);
    bf16x8 fa[FM], fb[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) fa[i] = MODE == kWeights ? ra_t.get(0, i) : ra_k.get(0, i);
#pragma unroll
    for (int i = 0; i < FN; i++) fb[i] = MODE == kBackward ? rb_k.get(0, i) : rb_t.get(0, i);
    const int32_t by_a = buf ? -kCA * 16 : kCA * 16, by_b = buf ? -kCB * 16 : kCB * 16;   // to the other buffer
    if (MODE == kWeights) ra_t.move(by_a);
    else ra_k.move(by_a);
    if (MODE == kBackward) rb_k.move(by_b);
    else rb_t.move(by_b);
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
      for (int j = 0; j < FN; j++)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    buf ^= 1;
  };
  const std::integral_constant<int, 0> set0;
  const std::integral_constant<int, 1> set1;
  const std::integral_constant<int, kSets - 1> last_set;
  const std::true_type whole;
  const std::false_type any;
  for (; base < (uint32_t)K; base = end) {   // kWeights: rounds of the places in the list
    end = MODE == kWeights ? base + round_length((int)base, K, kList) : K;
    if (MODE == kWeights) {
      __syncthreads();
      for (uint32_t i = tid; i < end - base; i += kThreads)
        list[i] = a.gather ? a.rows[t.first + base + i] / a.k : (int32_t)(t.first + base + i);
      __syncthreads();
    }
    load(set0, any, base);
    load(set1, any, base + kBK);
    if (kSets == 3) load(last_set, any, base + 2 * kBK);
    put_stage(set0, buf);
    load(set0, any, base + kSets * kBK);
    // a round of kSets stages; each sends for the stage kSets + 1 further on
    auto round = [&](auto WHOLE, uint32_t k0) {
      stage(set1, WHOLE, k0 + (kSets + 1) * kBK);
      if (WHOLE || k0 + kBK < end) {
        if (kSets == 3) stage(last_set, WHOLE, k0 + (kSets + 2) * kBK);
        else stage(set0, WHOLE, k0 + (kSets + 2) * kBK);
      }
      if (kSets == 3 && (WHOLE || k0 + 2 * kBK < end)) stage(set0, WHOLE, k0 + (kSets + 3) * kBK);
    };
    uint32_t k0 = base;
    if (inside)
      for (; k0 + (2 * kSets + 1) * kBK <= end; k0 += kSets * kBK) round(whole, k0);
    for (; k0 < end; k0 += kSets * kBK) round(any, k0);
  }
  if (MODE != kWeights && a.part) a.y = static_cast<float *>(a.y) + (int64_t)blockIdx.y * a.places * a.ldy;
  __syncthreads();   // the buffers are no longer read
  store_tile<MODE, FM, FN, false>(a, t, wr, wc, acc, reinterpret_cast<char *>(lds) + wave * (FM * FN * 512));
}

__host__ __device__ inline int64_t part_stride(int64_t cols) { return (cols + 3) / 4 * 4; }
// (about 3 us, a launch, for one token's 2 x 8192 results in 4 parts)
// Sums the parts of a contraction that several work-groups shared, in order: y[p] = s_p sum of part[i][p].
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a, const float *part, int parts, int64_t cols, int held_at) {
  const int64_t p = blockIdx.x, col = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  if (col >= cols) return;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < parts; i++) acc += *reinterpret_cast<const f32x4 *>(part + ((int64_t)i * a.places + p) * part_stride(cols) + col);
  if (a.scale && p < a.offsets[held_at]) acc *= a.scale[a.rows[p]];
  store4(a, p * a.ldy + col, cols - col, acc);
}

// d (float32) for the weights' gradient: a row of d becomes two of bf16, d = high + low up to 2^-16 of a value (high is
// d's upper half, cut off; low, the rest, is exact before its own rounding). An expert's rows of high come before those of
// low, so with the rows of x named twice the product of twice as many places is the gradient.
//   offsets2[e] = 2 offsets[e];  place q of the 2 held: row rows2[q] of x and row q of d2.
// Infinities and NaN are in both. 16 KB in and out a place of 2048 columns: bound by memory; 4096 places 17 us (67 MB).
__global__ __launch_bounds__(256) void split_kernel(ProductArgs a, const float *d, int64_t ldd, int32_t *offsets2,
                                                    int32_t *rows2, bf16_t *d2, int64_t ld2) {
  const int tid = threadIdx.x;
  if (blockIdx.x == 0)
    for (int e = tid; e <= a.experts; e += 256) offsets2[e] = 2 * a.offsets[e];
  const int32_t held = a.offsets[a.experts];
  for (int64_t p = blockIdx.x; p < held; p += gridDim.x) {
    int e = 0, end = a.experts;   // the last expert that begins at p or before holds it
    while (end - e > 1) {
      const int mid = (e + end) >> 1;
      if (a.offsets[mid] <= p) e = mid;
      else end = mid;
    }
    const int64_t high = a.offsets[e] + p, low = a.offsets[e + 1] + p;
    if (tid == 0) rows2[high] = rows2[low] = a.gather ? a.rows[p] / a.k : (int32_t)p;
    for (int64_t col = tid * 8; col < a.m; col += 256 * 8) {
      float v[8], h[8], l[8];
      load8(d + p * ldd + col, a.m - col, v);
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const bool finite = (__float_as_uint(v[i]) & 0x7F800000u) != 0x7F800000u;
        h[i] = finite ? __uint_as_float(__float_as_uint(v[i]) & 0xFFFF0000u) : v[i];
        l[i] = finite ? v[i] - h[i] : v[i];
        if (l[i] == 0.0f) l[i] = h[i] * 0x1p-24f;   // not 0 unless d is: an infinity of x times it would be NaN
      }
      store8(d2 + high * ld2 + col, a.m - col, h);
      store8(d2 + low * ld2 + col, a.m - col, l);
    }
  }
}

// The grid of a tiled kernel.
template <int MODE>
int64_t tiles(ProductArgs &a, int64_t bm, int64_t bn) {
  // an expert (and the places without a pair) ends in at most one tile that is not full
  a.row_tiles = a.places / bm + a.experts + 1 < a.places ? a.places / bm + a.experts + 1 : a.places;
  const int64_t rows = MODE == kWeights ? a.experts * ((a.n + bm - 1) / bm) : a.row_tiles;
  const int64_t cols = ((MODE == kBackward ? a.n : a.m) + bn - 1) / bn;
  a.in_patches = patches(rows, cols) >= kMinPatches;
  return patch_grid(rows, cols, a.in_patches);
}

// Which kernel, by the rows an expert has on average and so that there are tiles for the chip. Times (us) on 32
// experts of 2048 x 8192 with even rows, for tiles of 64 x 256, 128 x 256 and 256 x 256 (forward, backward), weights of the
// last two:
//   rows an expert   forward            backward           weights
//    32              199  189  259      196  204  263      242  281
//   128              258  199  257      251  225  266      339  402
//   256              418  326  291      407  367  290      523  515
//   512              752  594  515      728  671  516      737  709
// With 256 x 256 the rows of an expert that do not fill a tile cost more. Forward, 32 experts, even rows of 256, 300, 340, 380: 128 x 256
// 352, 413, 427, 445, 256 x 256 302, 479, 474, 471; uneven ones of the same mean: 402, 418, 456, 490 and 434, 481, 510, 538. So below 384
// it pays for rows that fill its tiles alone (and for the 380 of 8 experts of 4096 x 11008: 394, 317). Backward and for weights the two
// are mostly within 6% of each other there, either way.
// any_kernel takes its 128 x 256 tiles from half as many on: 16 experts of 1031 x 5001, 125 rows each, forward 73 us (64 x 128: 70),
// 8 of 2765 x 4101, 312 rows, 154 (184), 64 of 1031 x 2051, 94 rows, 142 (134); with uneven rows 76 (82), 138 (174), 170 (137).
// The rule looks at the mean of the rows, which the host knows; with uneven ones it can be off by the likes of the last figure.
// Where even tiles of 64 x 128 are few, several work-groups share a contraction and join_kernel adds their parts.
struct Choice {
  int fm, fn, parts;
};
template <int MODE>
Choice choose(const ProductArgs &a) {
  const int64_t rows = a.places / a.experts, cols = MODE == kBackward ? a.n : a.m, K = MODE == kForward ? a.n : a.m;
  auto count = [&](int64_t bm, int64_t bn) {   // tiles, if the rows fill theirs
    return (MODE == kWeights ? a.experts * ((a.n + bm - 1) / bm) : (a.places + bm - 1) / bm) * ((cols + bn - 1) / bn);
  };
  constexpr int64_t kEnough = 512;   // two for each compute unit
  if (rows >= (MODE == kForward ? 384 : 256) && count(256, 256) >= kEnough) return {8, 8, 1};
  if ((rows >= 64 || MODE == kWeights) && count(128, 256) >= (a.direct ? kEnough : kEnough / 2)) return {4, 8, 1};
  if (MODE == kWeights) return {2, 4, 1};
  const int64_t part_full = a.places / 64 + a.experts;   // row tiles with those that are not full
  const int64_t row_tiles = part_full < a.places ? part_full : a.places;
  if (row_tiles * ((cols + 255) / 256) >= kEnough) return {2, 8, 1};
  // (below 2048 the join, 3 us, costs about what the shorter contractions save: contractions of 1024, one | shared, in us: one token's
  // 2 x 8192 results 10.7 | 10.4, 2 x 1024 8.8 | 7.7, 64 tokens' 128 x 1024 9.3 | 10.2; of 512 6.8 | 7.8; of 1536 14.1 | 14.6, 11.5 | 8.2,
  // 11.6 | 11.4)
  int64_t parts = K < 2048 ? 1 : kEnough / (row_tiles * ((cols + 127) / 128));
  if (parts > K / 256) parts = K / 256;
  return {2, 4, parts > 1 ? (int)parts : 1};
}

template <int MODE, int FM, int FN, int NS, int KS>
int launch_tile(ProductArgs a, int parts, void *stream) {
  const int64_t grid = tiles<MODE>(a, 32 * FM, 32 * FN);
  if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidConfiguration;
  tile_kernel<MODE, FM, FN, NS, KS><<<dim3((unsigned)grid, parts), 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  return (int)hipGetLastError();
}
template <int MODE, int FM, int FN, int kSets>
int launch_any(ProductArgs a, int parts, void *stream) {
  const int64_t grid = tiles<MODE>(a, 32 * FM, 32 * FN);
  if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidConfiguration;
  any_kernel<MODE, FM, FN, kSets><<<dim3((unsigned)grid, parts), 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  return (int)hipGetLastError();
}

// Stages of two steps where W's rows run along the contraction: whole 128-byte lines of them.
template <int MODE>
int launch_mode(const ProductArgs &a, char *ws, void *stream) {
  constexpr int kSteps = MODE == kBackward ? 2 : 1;
  const Choice c = choose<MODE>(a);
  if (a.direct && c.fm == 8) return launch_tile<MODE, 8, 8, 4 / kSteps, kSteps>(a, 1, stream);
  if (a.direct && c.fm == 4) return launch_tile<MODE, 4, 8, 3, kSteps>(a, 1, stream);
  if (c.fm >= 4) return launch_any<MODE, 4, 8, 2>(a, 1, stream);
  if constexpr (MODE != kWeights) {
    if (a.direct && c.fn == 8) return launch_tile<MODE, 2, 8, 4 / kSteps, kSteps>(a, 1, stream);
    if (c.parts > 1) {
      const int64_t cols = MODE == kBackward ? a.n : a.m, K = MODE == kForward ? a.n : a.m;
      ProductArgs b = a;
      b.part = (int32_t)(((K + c.parts - 1) / c.parts + 63) / 64 * 64);
      b.y = ws;
      b.scale = nullptr;
      b.ldy = part_stride(cols);
      b.f32 = b.wide = 1;
      const int parts = (int)((K + b.part - 1) / b.part);
      const int e = a.direct ? launch_tile<MODE, 2, 4, 4 / kSteps, kSteps>(b, parts, stream) : launch_any<MODE, 2, 4, 3>(b, parts, stream);
      if (e != (int)hipSuccess) return e;
      join_kernel<<<dim3((unsigned)a.places, (unsigned)((cols + 1023) / 1024)), 256, 0, static_cast<hipStream_t>(stream)>>>(
          a, reinterpret_cast<const float *>(ws), parts, cols, a.experts);
      return (int)hipGetLastError();
    }
  }
  return a.direct ? launch_tile<MODE, 2, 4, 4 / kSteps, kSteps>(a, 1, stream) : launch_any<MODE, 2, 4, 3>(a, 1, stream);
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

// The direct loads' offsets of lanes have 32 bits. Where a call names rows of x all over (gathered ones, and every place of the
// weights' gradient) they have to lie within 2^31 bytes; beyond, any_kernel takes it. 8 experts of 8192 x 2048 on either side of that
// line (131000 and 131100 rows): gathered forward 3565 and 4055 us, forward 3247 and 3395 (the same kernel), gradient 3259 and 4553.
constexpr int64_t kMaxTile = 256;   // result rows, or contraction rows, that a lane's offset spans
bool chunks(const void *p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

}  // namespace

ProductArgs product_args(const skew_rows &r, const skew_product_desc &p) {
  ProductArgs a = args_of(r, p);
  a.direct = chunks(a.x, a.ldx) && chunks(a.w, a.ldw) && a.slice % 8 == 0 && a.n % 8 == 0 && a.m % 8 == 0 &&
             short_rows(a.gather ? r.tokens : kMaxTile, a.ldx) && short_rows(kMaxTile, a.ldw);
  a.wide = ((uintptr_t)a.y & 15) == 0 && a.ldy % 4 == 0;
  if (!a.f32) a.direct = a.direct && a.wide && a.ldy % 8 == 0;
  return a;
}

size_t product_scratch(const skew_rows &r, const skew_product_desc &p) {
  if (r.tokens == 0) return 0;
  const ProductArgs a = product_args(r, p);
  const bool back = (p.flags & SKEW_TRANSPOSE) != 0;
  const int parts = back ? choose<kBackward>(a).parts : choose<kForward>(a).parts;   // whatever the alignment
  return parts > 1 ? (size_t)parts * (size_t)a.places * (size_t)part_stride(back ? a.n : a.m) * 4 : 0;
}

int launch_product(const skew_rows &r, const skew_product_desc &p, char *ws, void *stream) {
  const ProductArgs a = product_args(r, p);
  return p.flags & SKEW_TRANSPOSE ? launch_mode<kBackward>(a, ws, stream) : launch_mode<kForward>(a, ws, stream);
}

namespace {
// x_rows: the rows of x that places name
int product_grad(const skew_rows &r, const skew_product_desc &p, int64_t x_rows, void *stream) {
  ProductArgs a = args_of(r, p);
  a.w = static_cast<const bf16_t *>(p.y);
  a.y = const_cast<void *>(p.w);
  a.ldw = p.ldy;
  a.ldy = p.ldw;
  a.f32 = 0;
  a.direct = chunks(a.x, a.ldx) && chunks(a.w, a.ldw) && a.n % 8 == 0 && a.m % 8 == 0 &&
             short_rows(x_rows, a.ldx) && short_rows(kMaxTile, a.ldw);
  a.wide = ((uintptr_t)a.y & 15) == 0 && a.ldy % 4 == 0 && a.slice % 4 == 0;
  a.direct = a.direct && a.wide && a.ldy % 8 == 0 && a.slice % 8 == 0;
  return launch_mode<kWeights>(a, nullptr, stream);
}

// scratch of skew_expert_matmul_grad_f32: offsets2, rows2, d2
struct SplitPlan {
  size_t off_rows, off_d, bytes;
  int64_t ld;
};
SplitPlan split_plan(const skew_rows &r, const skew_product_desc &p) {
  const size_t places = (size_t)(r.tokens * r.k);
  SplitPlan s;
  s.ld = (p.m + 7) / 8 * 8;
  s.off_rows = pad256(((size_t)r.experts + 1) * 4);
  s.off_d = s.off_rows + pad256(2 * places * 4);
  s.bytes = s.off_d + 2 * places * (size_t)s.ld * 2;
  return s;
}
}  // namespace

int launch_product_grad(const skew_rows &r, const skew_product_desc &p, void *stream) {
  return product_grad(r, p, p.flags & SKEW_GATHER ? r.tokens : r.tokens * r.k, stream);
}

size_t product_grad_f32_scratch(const skew_rows &r, const skew_product_desc &p) {
  return r.tokens == 0 ? 0 : split_plan(r, p).bytes;
}

int launch_product_grad_f32(const skew_rows &r, const skew_product_desc &p, char *ws, void *stream) {
  const SplitPlan s = split_plan(r, p);
  const int64_t places = r.tokens * r.k;
  int32_t *offsets2 = reinterpret_cast<int32_t *>(ws), *rows2 = reinterpret_cast<int32_t *>(ws + s.off_rows);
  bf16_t *d2 = reinterpret_cast<bf16_t *>(ws + s.off_d);
  constexpr int64_t kMostGroups = 1 << 16;
  split_kernel<<<(unsigned)(places < kMostGroups ? places : kMostGroups), 256, 0, static_cast<hipStream_t>(stream)>>>(
      args_of(r, p), static_cast<const float *>(p.y), p.ldy, offsets2, rows2, d2, s.ld);
  const int e = (int)hipGetLastError();
  if (e != (int)hipSuccess) return e;
  const skew_rows twice = {offsets2, rows2, nullptr, 2 * places, 1, r.experts};   // pairs of one choice: their own tokens
  skew_product_desc q = p;
  q.y = d2;
  q.ldy = s.ld;
  q.flags = SKEW_GATHER;
  return product_grad(twice, q, p.flags & SKEW_GATHER ? r.tokens : places, stream);
}

}  // namespace moe
