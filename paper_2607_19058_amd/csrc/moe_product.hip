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
#include <stdlib.h>

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
  int32_t direct;                 // 16-byte rows in both operands and lengths that are multiples of 8
  int32_t wide;                   // 4 neighbouring results can be stored together
  int64_t row_tiles;              // forward, backward: tiles of rows in the grid
};

constexpr int kBK = 32;   // contraction length of a stage: one matrix instruction's

// ---- LDS tiles ------------------------------------------------------------------------------
// Contiguous in the contraction: rows of kBK values, 4 chunks of 8, so 4 rows are as long as the banks. A 16-byte
// read takes two cycles of 16 lanes each: rows 0-3 and 12-15 at one chunk with rows 4-11 at the next one, and the other way
// about. With the rows' groups of 4 xor-ed by 0, 2, 3, 1 these fall into different banks (0, 1, 2, 3: a third of the reads' cycles
// were conflicts).
__device__ __forceinline__ int swizzle_k(int row) { return (((row >> 2) ^ (row >> 3)) & 1) << 1 | ((row >> 3) & 1); }
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
template <int B>
struct FragK {
  uint32_t at;
  __device__ __forceinline__ FragK(const u32x4 *tile, int r0) {
    const int lane = threadIdx.x & 63, row = lane & 15;
    at = lds_offset(tile) + (r0 + row) * 64 + ((lane >> 4) ^ swizzle_k(row)) * 16;
  }
  __device__ __forceinline__ bf16x8 get(uint32_t buf, int i) const {
    return __builtin_bit_cast(bf16x8, *lds_at<u32x4>(at + buf + i * 1024));
  }
  __device__ __forceinline__ void move(int32_t bytes) { at += bytes; }
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
  __device__ __forceinline__ bf16x8 get(uint32_t buf, int f) const {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    struct {
      s16x4 lo, hi;   // rows row .. + 3 and, with the same xor, row + 4 .. + 7
    } v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at[f] + buf));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at[f] + buf + 4 * B * 2));
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
__device__ __forceinline__ void load_lds(const char *base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
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
// patch's tiles share their operands' rows and columns in one L2. Returns false where the patch passes the edge.
constexpr int kDies = 8, kPatchR = 4, kPatchC = 8;
__host__ __device__ inline int64_t patch_grid(int64_t rows, int64_t cols) {
  const int64_t p = ((rows + kPatchR - 1) / kPatchR) * ((cols + kPatchC - 1) / kPatchC);
  return (p + kDies - 1) / kDies * kDies * (kPatchR * kPatchC);
}
__device__ __forceinline__ bool patch_tile(int64_t rows, int64_t cols, int64_t *row, int64_t *col) {
  const uint32_t i = blockIdx.x / kDies, in = i % (kPatchR * kPatchC);
  const uint32_t patch = i / (kPatchR * kPatchC) * kDies + blockIdx.x % kDies, pc = (uint32_t)((cols + kPatchC - 1) / kPatchC);
  *row = (int64_t)(patch / pc) * kPatchR + in % kPatchR;
  *col = (int64_t)(patch % pc) * kPatchC + in / kPatchR;
  return *row < rows && *col < cols;
}

// acc += the product of two fragments (result rows along the second). IN_A: the sums stay in the accumulation
// registers, which the compiler, left to itself, copies to others and back when they are 256 of a lane's 512.
// It does not know the written-out instruction's latency: mfma_done() comes before the sums are read.
template <bool IN_A>
__device__ __forceinline__ void mfma(f32x4 &acc, bf16x8 b, bf16x8 a) {
  if (IN_A) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
  else acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, acc, 0, 0, 0);
}
__device__ __forceinline__ void mfma_done() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// What a tiled work-group computes: rows [r0, r1) and columns [c0, c1) of the result of one expert, contraction length K;
// kWeights: places first .. first + K - 1.
struct Tile {
  int expert, K;
  int64_t r0, r1, c0, c1, first;
};
template <int MODE, int B>
__device__ __forceinline__ bool take_tile(const ProductArgs &a, Tile *t) {
  int64_t tr, tc;
  t->first = 0;
  if (MODE == kWeights) {
    const int64_t tn = (a.n + B - 1) / B, tm = (a.m + B - 1) / B;
    if (!patch_tile(a.experts * tn, tm, &tr, &tc)) return false;
    t->expert = (int)(tr / tn);
    t->r0 = tr % tn * B;
    t->r1 = a.n;
    t->c1 = a.m;
    t->first = a.offsets[t->expert];
    t->K = __builtin_amdgcn_readfirstlane(a.offsets[t->expert + 1] - (int)t->first);
  } else {
    t->c1 = MODE == kForward ? a.m : a.n;
    if (!patch_tile(a.row_tiles, (t->c1 + B - 1) / B, &tr, &tc) || !find_tile<B>(a, tr, &t->expert, &t->r0, &t->r1)) return false;
    t->expert = __builtin_amdgcn_readfirstlane(t->expert);   // the same in every lane, but found in a loop over lanes
    t->r0 = scalar(t->r0);
    t->r1 = scalar(t->r1);
    t->K = t->expert < a.experts ? (int)(MODE == kForward ? a.n : a.m) : 0;   // the places without a pair: zeros
  }
  t->c0 = tc * B;
  return true;
}

// Stores a wave's F x F blocks of 16 x 16 results from row wr and column wc of the tile. A lane holds row
// lane % 16 of each block and its columns 4 (lane / 16) .. + 3.
template <int MODE, int F>
__device__ __forceinline__ void store_tile(const ProductArgs &a, const Tile &t, int wr, int wc, const f32x4 (&acc)[F][F]) {
  const int lane = threadIdx.x & 63;
  const int64_t row0 = t.r0 + wr + (lane & 15), col0 = t.c0 + wc + (lane >> 4) * 4;
  float s[F];
#pragma unroll
  for (int i = 0; i < F; i++) s[i] = 1.0f;
  if (MODE != kWeights && a.scale && t.expert < a.experts) {
#pragma unroll
    for (int i = 0; i < F; i++)
      if (row0 + i * 16 < t.r1) s[i] = a.scale[a.rows[row0 + i * 16]];
  }
  const int64_t at = (MODE == kWeights ? (int64_t)t.expert * a.slice : 0) + row0 * a.ldy + col0;
  if (a.wide && t.c0 + 32 * F <= t.c1) {   // every column exists
#pragma unroll
    for (int i = 0; i < F; i++) {
      if (row0 + i * 16 >= t.r1) break;
      if (a.f32) {
        float *y = static_cast<float *>(a.y) + at + i * 16 * a.ldy;
#pragma unroll
        for (int j = 0; j < F; j++) *reinterpret_cast<f32x4 *>(y + j * 16) = s[i] * acc[i][j];
      } else {
        bf16_t *y = static_cast<bf16_t *>(a.y) + at + i * 16 * a.ldy;
#pragma unroll
        for (int j = 0; j < F; j++) {
          const f32x4 v = s[i] * acc[i][j];
          *reinterpret_cast<uint2 *>(y + j * 16) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < F; i++) {
    if (row0 + i * 16 >= t.r1) break;
#pragma unroll
    for (int j = 0; j < F; j++) store4(a, at + i * 16 * a.ldy + j * 16, t.c1 - col0 - j * 16, s[i] * acc[i][j]);
  }
}

// ---- tiles whose chunks go from memory to LDS without registers ---------------------------------
// For rows at 16-byte positions and lengths that are multiples of 8, so that a chunk is inside its row or outside.
// Tiles of 32 F x 32 F results, 4 waves, each F x F matrix instructions a stage; kStages LDS buffers of a stage.
// While a wave multiplies stage s from registers it reads stage s + 1 from LDS into other registers and sends for
// stage s + kAhead, in F steps of one load, one fragment of each side and F matrix instructions. A load's address
// is a scalar, which moves from stage to stage, plus a lane's 32-bit offset, which stays.
// Rows and columns past the edge of the result repeat the last one inside and are not stored; past the end of the
// contraction both operands are zero, so nothing there meets a NaN.
constexpr int kList = 2048;   // places whose rows kWeights looks up at once

template <int MODE, int F>
__global__ __launch_bounds__(256, F == 8 ? 1 : 2) void tile_kernel(ProductArgs a) {
  constexpr int B = 32 * F, kThreads = 256;
  constexpr int kC = B * kBK / 8, kP = kC / kThreads;   // chunks of a stage's tile, and of a thread in it
  constexpr int kBytes = kC * 16;
  static_assert(2 * kP == F, "one load a step");
  // LDS buffers of a stage: all that fit at F = 8 (160 KiB, and kWeights' list), 64 KiB at F = 4 for two work-groups
  constexpr int kStages = F == 8 && MODE != kWeights ? 5 : 4, kAhead = kStages - 1;
  __shared__ u32x4 lds[2 * kStages * kC + (MODE == kWeights ? kList / 4 : 0)];
  u32x4 *const ta = lds, *const tb = lds + kStages * kC;
  uint32_t *const list = reinterpret_cast<uint32_t *>(tb + kStages * kC);   // byte offsets of x's rows
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = (wave >> 1) * (B / 2), wc = (wave & 1) * (B / 2);
  Tile t;
  if (!take_tile<MODE, B>(a, &t)) return;
  const int K = t.K;

  f32x4 acc[F][F];
#pragma unroll
  for (int i = 0; i < F; i++)
#pragma unroll
    for (int j = 0; j < F; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // Slot i of this thread is chunk q = tid + i kThreads of a stage's tile in LDS. A tile that is contiguous in the
  // contraction holds result row q / 4 and chunk (q % 4) ^ swizzle there; one that is not holds contraction row
  // q / (B / 8) likewise. ka, kb: the slot's contraction index in its stage; oa, ob: its byte offset from xa, xb, where
  // the next stage that is sent for begins (kWeights: oa without the row of x).
  const char *xa = reinterpret_cast<const char *>(a.x), *xb = reinterpret_cast<const char *>(a.w);
  int64_t step_a = 0, step_b;
  if (MODE == kWeights) {
    xb += 2 * t.first * a.ldw;
  } else {
    xb += 2 * (int64_t)(K ? t.expert : 0) * a.slice;
    if (!a.gather) xa += 2 * t.r0 * a.ldx;
    step_a = 2 * kBK;
  }
  step_b = MODE == kBackward ? 2 * kBK : 2 * kBK * a.ldw;
  if (MODE == kBackward) xb += 2 * t.c0 * a.ldw;
  xa = scalar(xa);
  xb = scalar(xb);
  step_b = scalar(step_b);
  uint32_t oa[kP], ob[kP];
  int ka[kP], kb[kP];
#pragma unroll
  for (int i = 0; i < kP; i++) {
    const int q = tid + i * kThreads;
    if (MODE == kWeights) {
      const int row = q / (B / 8), c = (q % (B / 8)) ^ swizzle_t<B>(row);
      ka[i] = row;
      oa[i] = (uint32_t)(2 * (t.r0 + c * 8 < t.r1 ? t.r0 + c * 8 : t.r1 - 8));
    } else {
      const int row = q / 4, c = (q % 4) ^ swizzle_k(row);
      const int r = t.r0 + row < t.r1 ? row : (int)(t.r1 - 1 - t.r0);
      ka[i] = c * 8;
      oa[i] = (uint32_t)((K > 0 && a.gather ? (int64_t)(a.rows[t.r0 + r] / a.k) : r) * a.ldx + c * 8) * 2;
    }
    if (MODE == kBackward) {
      const int row = q / 4, c = (q % 4) ^ swizzle_k(row);
      kb[i] = c * 8;
      ob[i] = (uint32_t)((t.c0 + row < t.c1 ? row : t.c1 - 1 - t.c0) * a.ldw + c * 8) * 2;
    } else {
      const int row = q / (B / 8), c = (q % (B / 8)) ^ swizzle_t<B>(row);
      kb[i] = row;
      ob[i] = (uint32_t)(row * a.ldw + (t.c0 + c * 8 < t.c1 ? t.c0 + c * 8 : t.c1 - 8)) * 2;
    }
  }
  const uint32_t la = lds_address(ta + wave * 64), lb = lds_address(tb + wave * 64);

  int reading = 0, sending = 0;   // buffers of the stages that are read, and sent for, next
  int base = 0, end = K;   // the contraction [base, end) of this round (kWeights: the places in the list)
  uint32_t row_next[kP];   // kWeights: the rows of x of the next stage that is sent for
  auto look_up = [&](int stage) {
    if (MODE == kWeights) {
#pragma unroll
      for (int i = 0; i < kP; i++) row_next[i] = list[(stage * kBK + ka[i]) & (kList - 1)];
    }
  };
  // load i of a stage: the slots of a, then those of b
  auto send = [&](int i, uint32_t buf) {
    if (i < kP) load_lds(xa, oa[i] + (MODE == kWeights ? row_next[i] : 0), la + buf + i * kThreads * 16);
    else load_lds(xb, ob[i - kP], lb + buf + (i - kP) * kThreads * 16);
  };
  auto sent_all = [&]() {
    xa += step_a;
    xb += step_b;
    sending = sending + 1 == kStages ? 0 : sending + 1;
  };
  // the same for any stage, also one that the contraction ends in
  auto send_stage = [&](int stage) {
    const uint32_t buf = sending * kBytes;
    const int left = end - base - stage * kBK;
    look_up(stage);
    if (left >= kBK) {
#pragma unroll
      for (int i = 0; i < F; i++) send(i, buf);
    } else {
#pragma unroll
      for (int i = 0; i < F; i++) {
        const bool is_a = i < kP;
        const int sl = is_a ? i : i - kP;
        if ((is_a ? ka[sl] : kb[sl]) < left) send(i, buf);
        else (is_a ? ta : tb)[sending * kC + tid + sl * kThreads] = u32x4{0, 0, 0, 0};
      }
    }
    sent_all();
  };

  // this lane's fragments, in the buffer of the stage that is read next
  FragK<B> ra_k(ta, wr), rb_k(tb, wc);
  FragT<B, F> ra_t(ta, wr), rb_t(tb, wc);
  auto move = [&](int32_t bytes) {
    if (MODE == kWeights) ra_t.move(bytes);
    else ra_k.move(bytes);
    if (MODE == kBackward) rb_k.move(bytes);
    else rb_t.move(bytes);
  };
  bf16x8 fa[2][F], fb[2][F];
  auto read_a = [&](int i, bf16x8 *d) { d[i] = MODE == kWeights ? ra_t.get(0, i) : ra_k.get(0, i); };
  auto read_b = [&](int i, bf16x8 *d) { d[i] = MODE == kBackward ? rb_k.get(0, i) : rb_t.get(0, i); };
  auto after = [&](int buf) { return buf + 1 == kStages ? 0 : buf + 1; };
  auto advance = [&]() {
    move(reading + 1 == kStages ? -(kStages - 1) * kBytes : kBytes);
    reading = after(reading);
  };
  // multiply fragments X; NEXT: read the next stage into the others; MORE: send for a stage
  auto stage = [&](auto X, auto NEXT, auto MORE) {
    constexpr int x = X, y = 1 - x;
#pragma unroll
    for (int i = 0; i < F; i++) {
#pragma unroll
      for (int j = 0; j < F; j++) {
        mfma<F == 8>(acc[i][j], fb[x][j], fa[x][i]);
        if (MORE && j == 0) send(i, sending * kBytes);
        if (NEXT && j == F / 4) read_a(i, fa[y]);
        if (NEXT && j == F / 2) read_b(i, fb[y]);
      }
    }
    if (MORE) sent_all();
    if (NEXT) advance();
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  const std::true_type yes;
  const std::false_type no;

  for (; base < K; base = end) {
    if (MODE == kWeights) {
      end = base + kList < K ? base + kList : K;
      __syncthreads();   // the list of the round before is no longer read
      for (int i = tid; i < end - base; i += kThreads) {
        const int64_t p = t.first + base + i;
        list[i] = (uint32_t)((a.gather ? (int64_t)(a.rows[p] / a.k) : p) * a.ldx * 2);
      }
      __syncthreads();
    }
    const int S = (end - base + kBK - 1) / kBK;
    for (int i = 0; i < kAhead && i < S; i++) send_stage(i);
    // of the stages that were sent for, all but `n` have arrived in every wave
    auto meet = [&](bool whole, auto n) {
      if (whole) vm_wait<n * F>();
      else vm_wait<0>();   // the last stage may have sent for less than F loads
      __syncthreads();
    };
    const std::integral_constant<int, kAhead - 1> one;    // one stage is there
    const std::integral_constant<int, kAhead - 2> two;
    meet(S > kAhead, one);
#pragma unroll
    for (int i = 0; i < F; i++) {
      read_a(i, fa[0]);
      read_b(i, fb[0]);
    }
    advance();
    // Before stage s: stage s + 1 is there, and the buffer of stage s + kAhead is no longer read.
    int s = 0;
    look_up(kAhead);
    for (; s + kAhead + 2 < S; s += 2) {    // sends for stages s + kAhead and s + kAhead + 1, which are whole
      meet(true, two);
      stage(even, yes, yes);
      look_up(s + kAhead + 1);
      meet(true, two);
      stage(odd, yes, yes);
      look_up(s + kAhead + 2);
    }
    for (; s + 1 < S; s += 2) {
      meet(s + kAhead < S, two);
      if (s + kAhead < S) send_stage(s + kAhead);
      stage(even, yes, no);
      meet(s + kAhead + 1 < S, two);
      if (s + kAhead + 1 < S) send_stage(s + kAhead + 1);
      stage(odd, yes, no);   // at the end of an even number of stages this reads what is not used
    }
    if (s < S) stage(even, no, no);
    // the next round, if any, starts in the buffer that is sent for next
    while (reading != sending) advance();
    __syncthreads();   // the buffers are no longer read
  }
  if (F == 8) mfma_done();
  store_tile<MODE, F>(a, t, wr, wc, acc);
}

// ---- tiles of any shape ---------------------------------------------------------------------
// The same tiles through registers: chunks are loaded from any position, at the ends of rows element by element,
// while the stage before is multiplied.
template <int MODE, int F>
__global__ __launch_bounds__(256, 2) void any_kernel(ProductArgs a) {
  constexpr int B = 32 * F, kThreads = 256;
  constexpr int kC = B * kBK / 8, kP = kC / kThreads, kBytes = kC * 16;
  __shared__ u32x4 ta[2 * kC], tb[2 * kC];
  const int tid = threadIdx.x, wave = tid >> 6;
  const int wr = (wave >> 1) * (B / 2), wc = (wave & 1) * (B / 2);
  Tile t;
  if (!take_tile<MODE, B>(a, &t)) return;
  const int K = t.K;

  f32x4 acc[F][F];
#pragma unroll
  for (int i = 0; i < F; i++)
#pragma unroll
    for (int j = 0; j < F; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // slots as in tile_kernel; na, nb: how many of the chunk's values are in the row
  const bf16_t *w = MODE == kWeights ? a.w + t.first * a.ldw : a.w + (int64_t)(K ? t.expert : 0) * a.slice;
  const bf16_t *pa[kP], *pb[kP];
  int ka[kP], kb[kP], na[kP], nb[kP];
  auto clip = [](int64_t x) { return (int)(x < 0 ? 0 : x > 8 ? 8 : x); };
#pragma unroll
  for (int i = 0; i < kP; i++) {
    const int q = tid + i * kThreads;
    if (MODE == kWeights) {
      const int row = q / (B / 8), c = (q % (B / 8)) ^ swizzle_t<B>(row);
      ka[i] = row;
      na[i] = clip(t.r1 - (t.r0 + c * 8));
      pa[i] = a.x + t.r0 + c * 8;
    } else {
      const int row = q / 4, c = (q % 4) ^ swizzle_k(row);
      const int64_t p = t.r0 + row < t.r1 ? t.r0 + row : t.r1 - 1;
      ka[i] = c * 8;
      na[i] = 8;
      pa[i] = a.x + (K > 0 && a.gather ? (int64_t)(a.rows[p] / a.k) : p) * a.ldx + c * 8;
    }
    if (MODE == kBackward) {
      const int row = q / 4, c = (q % 4) ^ swizzle_k(row);
      kb[i] = c * 8;
      nb[i] = 8;
      pb[i] = w + (t.c0 + row < t.c1 ? t.c0 + row : t.c1 - 1) * a.ldw + c * 8;
    } else {
      const int row = q / (B / 8), c = (q % (B / 8)) ^ swizzle_t<B>(row);
      kb[i] = row;
      nb[i] = clip(t.c1 - (t.c0 + c * 8));
      pb[i] = w + row * a.ldw + t.c0 + c * 8;
    }
  }
  const int64_t step_b = MODE == kBackward ? kBK : kBK * a.ldw;
  u32x4 ga[kP], gb[kP];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kP; i++) {
      const int la = K - k0 - ka[i], lb = K - k0 - kb[i];   // contraction values from this chunk on
      const bf16_t *p = pa[i];
      if (MODE == kWeights && la > 0) {
        const int64_t place = t.first + k0 + ka[i];
        p += (a.gather ? (int64_t)(a.rows[place] / a.k) : place) * a.ldx;
      }
      ga[i] = la > 0 ? load_chunk(p, MODE == kWeights ? na[i] : la) : u32x4{0, 0, 0, 0};
      gb[i] = lb > 0 ? load_chunk(pb[i], MODE == kBackward ? lb : nb[i]) : u32x4{0, 0, 0, 0};
      if (MODE != kWeights) pa[i] += kBK;
      pb[i] += step_b;
    }
  };
  auto put_stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kP; i++) {
      ta[buf * kC + tid + i * kThreads] = ga[i];
      tb[buf * kC + tid + i * kThreads] = gb[i];
    }
  };
  const FragK<B> ra_k(ta, wr), rb_k(tb, wc);
  const FragT<B, F> ra_t(ta, wr), rb_t(tb, wc);
  if (K > 0) {
    load(0);
    put_stage(0);
  }
  int buf = 0;
  for (int k0 = 0; k0 < K; k0 += kBK) {
    __syncthreads();
    const bool more = k0 + kBK < K;
    if (more) load(k0 + kBK);
    bf16x8 fa[F], fb[F];
#pragma unroll
    for (int i = 0; i < F; i++) {
      fa[i] = MODE == kWeights ? ra_t.get(buf * kBytes, i) : ra_k.get(buf * kBytes, i);
      fb[i] = MODE == kBackward ? rb_k.get(buf * kBytes, i) : rb_t.get(buf * kBytes, i);
    }
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
      for (int j = 0; j < F; j++)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    buf ^= 1;
    if (more) put_stage(buf);
  }
  store_tile<MODE, F>(a, t, wr, wc, acc);
}

template <int MODE, int F, bool DIRECT>
int launch(ProductArgs a, void *stream) {
  constexpr int B = 32 * F;
  int64_t grid;
  if (MODE == kWeights) {
    grid = patch_grid(a.experts * ((a.n + B - 1) / B), (a.m + B - 1) / B);
  } else {
    const int64_t cols = MODE == kForward ? a.m : a.n;
    // an expert (and the places without a pair) ends in at most one tile that is not full
    a.row_tiles = a.places / B + a.experts + 1 < a.places ? a.places / B + a.experts + 1 : a.places;
    grid = patch_grid(a.row_tiles, (cols + B - 1) / B);
  }
  if (grid > 0x7FFFFFFF) return (int)hipErrorInvalidConfiguration;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if constexpr (DIRECT) tile_kernel<MODE, F><<<(unsigned)grid, 256, 0, s>>>(a);
  else any_kernel<MODE, F><<<(unsigned)grid, 256, 0, s>>>(a);
  return (int)hipGetLastError();
}

template <int MODE>
int launch_mode(const ProductArgs &a, void *stream) {
  if (!a.direct) return launch<MODE, 4, false>(a, stream);
  return getenv("MOE_F4") ? launch<MODE, 4, true>(a, stream) : launch<MODE, 8, true>(a, stream);
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

constexpr int64_t kMaxTile = 256;   // result rows, or contraction rows, that a lane's offset spans
// rows whose byte offsets are 32-bit numbers, with a row to spare
bool short_rows(int64_t rows, int64_t ld) { return (rows + 1) * ld * 2 < (int64_t)1 << 32; }
bool chunks(const void *p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

}  // namespace

size_t product_scratch(const skew_rows &, const skew_product_desc &) { return 0; }

int launch_product(const skew_rows &r, const skew_product_desc &p, char *, void *stream) {
  ProductArgs a = args_of(r, p);
  a.direct = chunks(a.x, a.ldx) && chunks(a.w, a.ldw) && a.slice % 8 == 0 && a.n % 8 == 0 && a.m % 8 == 0 &&
             short_rows(a.gather ? r.tokens : kMaxTile, a.ldx) && short_rows(kMaxTile, a.ldw);
  a.wide = ((uintptr_t)a.y & 15) == 0 && a.ldy % 4 == 0;
  return p.flags & SKEW_TRANSPOSE ? launch_mode<kBackward>(a, stream) : launch_mode<kForward>(a, stream);
}

int launch_product_grad(const skew_rows &r, const skew_product_desc &p, void *stream) {
  ProductArgs a = args_of(r, p);
  a.w = static_cast<const bf16_t *>(p.y);
  a.y = const_cast<void *>(p.w);
  a.ldw = p.ldy;
  a.ldy = p.ldw;
  a.f32 = 0;
  a.direct = chunks(a.x, a.ldx) && chunks(a.w, a.ldw) && a.n % 8 == 0 && a.m % 8 == 0 &&
             short_rows(a.gather ? r.tokens : a.places, a.ldx) && short_rows(kMaxTile, a.ldw);
  a.wide = ((uintptr_t)a.y & 15) == 0 && a.ldy % 4 == 0 && a.slice % 4 == 0;
  return launch_mode<kWeights>(a, stream);
}

}  // namespace moe
