// product_tiles.h -- tiles of matrix products on the matrix cores: operands from memory to LDS to fragments, and the main loop.
//
// A work-group computes one tile of a result. Operand tiles go through LDS in the order they have in memory; a lane of the
// matrix instruction needs 8 neighbours along the contraction, which are one 16-byte LDS read where memory is contiguous in it, and
// two transposing LDS reads (4 rows by 16 columns to 4 neighbours per lane) where it is not. 16-byte chunks are placed in LDS with
// their index xor-ed with bits of their row, so that the lanes of one LDS access fall into different banks.
// The matrix instruction is called with the second operand's side first: a lane then holds 4 neighbouring columns of
// one result row, which it stores together.
#pragma once

#include <type_traits>

#include "moe_internal.h"

namespace moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
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

// The same for a product without experts, whose contraction may be shared by `parts` work-groups. Tiles are counted in strips
// of kPatchC columns, row by row in a strip, part by part; of every 256 of them, a round of the chip, each die takes 32
// neighbours (4 rows of a strip), and of the last ones an eighth. No place of a round stays empty, however the result is shaped.
// The 256 tiles of 8192 rows' gradient (2048 columns, contraction 25152): 713 us with columns to the dies in turn, 52% of the lines missing
// in their L2s.
constexpr int kRound = kDies * kPatchR * kPatchC;
__host__ __device__ inline int64_t plain_grid(int64_t total) { return total / kRound * kRound + (total % kRound + kDies - 1) / kDies * kDies; }
// BANDS: bands of kPatchR rows, column by column, instead of strips: for results that are most of the bytes, whose rows the dies then write
// side by side (32 experts' weights' gradient of 2048 x 8192: 684 us, in strips 839).
template <bool BANDS = false>
__device__ __forceinline__ bool plain_tile(uint32_t rows, uint32_t cols, uint32_t parts, uint32_t *row, uint32_t *col, uint32_t *part) {
  const uint32_t total = rows * cols * parts, whole = total / kRound * kRound;   // (below 2^31)
  const uint32_t die = blockIdx.x % kDies, i = blockIdx.x / kDies;
  uint32_t at;
  if (blockIdx.x < whole) {
    at = i / (kRound / kDies) * kRound + die * (kRound / kDies) + i % (kRound / kDies);
  } else {
    const uint32_t share = (total - whole + kDies - 1) / kDies;
    at = whole + die * share + (i - whole / kDies);
    if (at >= total) return false;
  }
  *part = at / (rows * cols);
  at -= *part * (rows * cols);
  const uint32_t along = BANDS ? cols : rows, across = BANDS ? rows : cols;
  constexpr uint32_t kWide = BANDS ? kPatchR : kPatchC;
  const uint32_t strip = at / (along * kWide), width = across - strip * kWide < kWide ? across - strip * kWide : kWide;
  at -= strip * along * kWide;
  const uint32_t a = at / width, b = strip * kWide + at - a * width;
  *row = BANDS ? b : a;
  *col = BANDS ? a : b;
  return true;
}

// acc += the product of two fragments (result rows along the second). IN_A: the sums stay in the accumulation
// registers, which the compiler, left to itself, copies to others and back when they are 256 of a lane's 512.
// It does not know the written-out instruction's latency: the sums go through mfma_done() before they are read.
// HALF: of float16 values (with their subnormal ones) instead of bf16 ones.
template <bool IN_A, bool HALF>
__device__ __forceinline__ void mfma(f32x4 &acc, bf16x8 b, bf16x8 a) {
  if (HALF) {
    if (IN_A) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
    else acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), acc, 0, 0, 0);
  } else {
    if (IN_A) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
    else acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, acc, 0, 0, 0);
  }
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
// kWeights: places first .. first + K - 1. part: this work-group's of a contraction that several share (ProductArgs::part long each).
struct Tile {
  int expert, K, part;
  int64_t r0, r1, c0, c1, first;
};
// 16-bit results of a wave (FM x FN blocks of 16 x 16; a lane holds row lane % 16 of each and its columns 4 (lane / 16) .. + 3) go
// through `room` (FM FN 512 bytes of LDS of this wave's own), so that a row's 32 FN bytes leave together: 8-byte stores of
// 16 rows at once reached 3.1 TB/s on a gradient that is all output. Chunks of 8 are placed with their index xor-ed with the row.
template <int FN>
__device__ __forceinline__ void put_room(char *room, int i, int j, uint2 v) {
  constexpr int kChunks = 2 * FN;   // of a row
  const int lane = threadIdx.x & 63, row = i * 16 + (lane & 15), c = 2 * j + (lane >> 5);
  *reinterpret_cast<uint2 *>(room + row * (kChunks * 16) + (c ^ (row & 7)) * 16 + (lane >> 4 & 1) * 8) = v;
}
// Stores them: y is the wave's first result, which has `rows` rows and `cols` columns left (of a row's, whole chunks with CHUNKS).
template <int FM, int FN, bool CHUNKS>
__device__ __forceinline__ void store_room(const char *room, uint16_t *y, int64_t ldy, int64_t rows_left, int64_t cols_left) {
  constexpr int kChunks = 2 * FN, kRows = 64 / kChunks;   // rows of one store
  const int lane = threadIdx.x & 63, c = lane % kChunks, row_in = lane / kChunks;
  __builtin_amdgcn_wave_barrier();
  const int64_t left = cols_left - c * 8;
  const int rows = rows_left < 16 * FM ? (int)rows_left : 16 * FM, n = (int)(left < 8 ? left : 8);   // of the wave's; of the lane's 8 columns
  y += row_in * ldy + c * 8;
  const int64_t step = kRows * ldy;
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
        if (e < n) y[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
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

// Op: op.take() names the tile (false: none), op.finish() takes its sums, with the LDS of the stages as room of a wave's own.
// Work-groups of a compute unit that its registers are meant for:
constexpr int per_unit(int FM, int FN, int KS) { return FM * FN * KS >= 64 ? 1 : FM * FN == 8 ? 3 : 2; }

template <int MODE, int FM, int FN, int NS, int KS, class Op>
__device__ __forceinline__ void tile_body(ProductArgs a, const Op &op) {
  constexpr bool kTurnA = MODE == kWeights || MODE == kOuter, kTurnB = MODE != kBackward;   // along the result
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
  if (!op.template take<MODE, BM, BN>(a, &t)) return;
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
  } else if (MODE == kOuter) {
    xa += 2 * t.first * a.ldx;
    xb += 2 * t.first * a.ldw;
    step_a = 2 * BK * a.ldx;
  } else {
    xb += 2 * (int64_t)(K ? t.expert : 0) * a.slice;
    if (!a.gather) xa += 2 * t.r0 * a.ldx;
    step_a = 2 * BK;
  }
  step_b = kTurnB ? 2 * BK * a.ldw : 2 * BK;
  if (MODE != kWeights && a.part) {   // this work-group's part of a contraction that several share
    const int k0 = t.part * a.part;
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
    } else if (MODE == kOuter) {
      const int row = q / (BM / 8), c = (q % (BM / 8)) ^ swizzle_t<BM>(row);
      ka[i] = row;
      oa[i] = (uint32_t)(row * a.ldx + (t.r0 + c * 8 < t.r1 ? t.r0 + c * 8 : t.r1 - 8)) * 2;
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
  auto read_a = [&](int k, int i, bf16x8 *d) { d[i] = kTurnA ? ra_t.get(k, i) : ra_k.get(k, i); };
  auto read_b = [&](int k, int i, bf16x8 *d) { d[i] = kTurnB ? rb_t.get(k, i) : rb_k.get(k, i); };
  auto advance = [&]() {
    const bool wrap = reading + 1 == NS;
    const int32_t by_a = wrap ? -(NS - 1) * kBytesA : kBytesA, by_b = wrap ? -(NS - 1) * kBytesB : kBytesB;
    if (kTurnA) ra_t.move(by_a);
    else ra_k.move(by_a);
    if (kTurnB) rb_t.move(by_b);
    else rb_k.move(by_b);
    reading = wrap ? 0 : reading + 1;
  };
  // multiply fragments X; NEXT: read step k of the stage that is read next into the others; MORE: send for a
  // stage. The loads come first.
  auto step = [&](auto X, auto NEXT, auto MORE, int k) {
    constexpr int x = X, y = 1 - x, kDo = (MORE ? kLoads : 0) + (NEXT ? FM + FN : 0);
    auto due = [](int m) { return m >= FM * FN - 2 ? kDo : m * kDo / (FM * FN - 2); };   // how many come before instruction m
#pragma unroll
    for (int m = 0; m < FM * FN; m++) {
      mfma<kInA, Op::kHalf>(acc[m / FN][m % FN], fb[x][m % FN], fa[x][m / FN]);
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
  op.template finish<MODE, FM, FN>(a, t, wr, wc, acc, reinterpret_cast<char *>(lds) + wave * (FM * FN * 512));
}

}  // namespace
}  // namespace moe
