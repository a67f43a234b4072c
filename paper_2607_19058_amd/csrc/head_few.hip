// head_few.hip -- the head's logits of a few rows, and their softmax sums: w is read once, straight into fragments.
//
// Up to 64 rows the products are nothing beside w's bytes, so w goes from memory to registers without LDS, and a wave has 16 to 32 loads
// on their way. Fragments of the matrix instruction hold 8 neighbours along the contraction:
//   w [K x V]   a lane loads 8 columns of 8 rows and turns the 8 x 8 block in its registers (4 byte permutes a load). Its 8 fragments
//               are 8 products, of which number f has columns 8 j + f. The 8 waves of a work-group share the contraction.
//   w [V x K]   a lane loads 32 bytes of a row, two fragments; the order of the contraction is the same for x.
// Rows, columns and the contraction may end anywhere, and rows may begin anywhere.
#include "head_internal.h"
#include "product_tiles.h"

namespace moe {
namespace {

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }   // (1 ulp; 0 below 2^-126)
__device__ __forceinline__ float or_zero(float m) { return m == -INFINITY ? 0.0f : m; }

struct Few {
  const bf16_t *x, *w;
  int64_t ldx, ldw, rows, cols, K;
};

__device__ __forceinline__ int64_t target_of(const HeadForward &f, int64_t row) {
  return f.target_bytes == 8 ? static_cast<const int64_t *>(f.targets)[row] : static_cast<const int32_t *>(f.targets)[row];
}
// x[row][k .. k + 7], zeros past its ends
__device__ __forceinline__ bf16x8 x_part(const Few &p, int64_t row, int64_t k) {
  return __builtin_bit_cast(bf16x8, load_chunk(p.x + row * p.ldx + k, row < p.rows ? p.K - k : 0));
}

constexpr int kWaves = 8;   // that share a contraction
template <int TM>
__global__ __launch_bounds__(64 * kWaves) void few_kernel(Few p, HeadForward f) {
  __shared__ float held[kWaves][16][132];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j = lane & 15, group = lane >> 4;
  const int64_t col = ((int64_t)blockIdx.x * 16 + j) * 8, left = p.cols - col;
  f32x4 acc[TM][8] = {};
  const int64_t steps = (p.K + 31) / 32;
  u32x4 w[2][8];
  auto load = [&](int64_t step, u32x4 *to) {
    const int64_t k = step * 32 + group * 8;
    const bf16_t *at = p.w + k * p.ldw + col;
    if (k + 8 <= p.K && left >= 8) {
#pragma unroll
      for (int r = 0; r < 8; r++) to[r] = *reinterpret_cast<const u32x4_a2 *>(at + r * p.ldw);
    } else {
#pragma unroll
      for (int r = 0; r < 8; r++) to[r] = load_chunk(at + r * p.ldw, k + r < p.K ? left : 0);
    }
  };
  auto multiply = [&](int64_t step, const u32x4 *v) {
    bf16x8 a[TM];
#pragma unroll
    for (int t = 0; t < TM; t++) a[t] = x_part(p, t * 16 + j, step * 32 + group * 8);
#pragma unroll
    for (int c = 0; c < 8; c++) {
      u32x4 b;
#pragma unroll
      for (int i = 0; i < 4; i++) b[i] = __builtin_amdgcn_perm(v[2 * i + 1][c / 2], v[2 * i][c / 2], c % 2 ? 0x07060302 : 0x05040100);
#pragma unroll
      for (int t = 0; t < TM; t++)
        acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), a[t], acc[t][c], 0, 0, 0);
    }
  };
  int64_t s = wave;
  if (s < steps) load(s, w[0]);
  for (; s < steps; s += 2 * kWaves) {
    if (s + kWaves < steps) load(s + kWaves, w[1]);
    multiply(s, w[0]);
    if (s + 2 * kWaves < steps) load(s + 2 * kWaves, w[0]);
    if (s + kWaves < steps) multiply(s + kWaves, w[1]);
  }
#pragma unroll
  for (int t = 0; t < TM; t++) {
    if (t) __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; c++)
#pragma unroll
      for (int q = 0; q < 4; q++) held[wave][j][8 * (4 * group + q) + c] = acc[t][c][q];
    __syncthreads();
    // 32 threads a row, 4 columns each; the waves' parts in order
    const int row16 = tid >> 5;
    const int64_t row = t * 16 + row16, first = (int64_t)blockIdx.x * 128 + (tid & 31) * 4;
    float z[4] = {}, m = -INFINITY, sum = 0.0f;
    const int64_t y = row < p.rows ? target_of(f, row) : -1;
#pragma unroll
    for (int q = 0; q < 4; q++) {
#pragma unroll
      for (int i = 0; i < kWaves; i++) z[q] += held[i][row16][(tid & 31) * 4 + q];
      if (y == first + q && y < p.cols) f.target_sum[row] = z[q];
      z[q] = first + q < p.cols ? z[q] : -INFINITY;
      m = fmaxf(m, z[q]);
    }
    m *= f.c;
#pragma unroll
    for (int q = 0; q < 4; q++) sum += exp2_(__builtin_fmaf(z[q], f.c, -or_zero(m)));
    float top = m;
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    sum *= exp2_(m - or_zero(top));
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((tid & 31) == 0 && row < p.rows) f.part[row * f.part_ld + blockIdx.x] = make_float2(top, sum);
  }
}

constexpr int kAhead = 4;   // 128-byte pieces of 16 rows that are on their way
template <int TM>
__global__ __launch_bounds__(256) void few_tied_kernel(Few p, HeadForward f) {
  __shared__ float2 held[4][TM * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, j = lane & 15, group = lane >> 4;
  const int64_t word0 = ((int64_t)blockIdx.x * 4 + wave) * 16;
  const bf16_t *at = p.w + (word0 + j < p.cols ? word0 + j : p.cols - 1) * p.ldw;
  f32x4 acc[TM] = {};
  u32x4 w[kAhead][2];
  auto load = [&](int64_t k0, u32x4 *to) {
    const int64_t k = k0 + group * 16;
    if (k + 16 <= p.K) {
      to[0] = *reinterpret_cast<const u32x4_a2 *>(at + k);
      to[1] = *reinterpret_cast<const u32x4_a2 *>(at + k + 8);
    } else {
      to[0] = load_chunk(at + k, p.K - k);
      to[1] = load_chunk(at + k + 8, p.K - k - 8);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; i++) load(i * 64, w[i]);
  for (int64_t k0 = 0; k0 < p.K; k0 += kAhead * 64) {
#pragma unroll
    for (int i = 0; i < kAhead; i++) {
      const int64_t k = k0 + i * 64;
#pragma unroll
      for (int h = 0; h < 2; h++)
#pragma unroll
        for (int t = 0; t < TM; t++)
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[i][h]), x_part(p, t * 16 + j, k + group * 16 + h * 8),
                                                           acc[t], 0, 0, 0);
      load(k + kAhead * 64, w[i]);
    }
  }
#pragma unroll
  for (int t = 0; t < TM; t++) {   // lane: row 16 t + j, words word0 + 4 group .. + 3
    const int64_t row = t * 16 + j, first = word0 + 4 * group;
    const int64_t y = row < p.rows ? target_of(f, row) : -1;
    float z[4], m = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; q++) {
      if (y == first + q && y < p.cols) f.target_sum[row] = acc[t][q];
      z[q] = first + q < p.cols ? acc[t][q] : -INFINITY;
      m = fmaxf(m, z[q]);
    }
    m *= f.c;
#pragma unroll
    for (int q = 0; q < 4; q++) sum += exp2_(__builtin_fmaf(z[q], f.c, -or_zero(m)));
    float top = fmaxf(m, __shfl_xor(m, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    sum *= exp2_(m - or_zero(top));
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (group == 0) held[wave][t * 16 + j] = make_float2(top, sum);
  }
  __syncthreads();
  if (tid < TM * 16 && tid < p.rows) {
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) top = fmaxf(top, held[i][tid].x);
#pragma unroll
    for (int i = 0; i < 4; i++) sum += held[i][tid].y * exp2_(held[i][tid].x - or_zero(top));
    f.part[tid * f.part_ld + blockIdx.x] = make_float2(top, sum);
  }
}

}  // namespace

int64_t head_few_parts(int mode, const HeadProduct &p) { return mode == kBackward ? (p.cols + 63) / 64 : (p.cols + 127) / 128; }

int launch_head_few(int mode, const HeadProduct &p, const HeadForward &f, void *stream) {
  const Few q = {static_cast<const bf16_t *>(p.a), static_cast<const bf16_t *>(p.b), p.lda, p.ldb, p.rows, p.cols, p.K};
  const unsigned grid = (unsigned)head_few_parts(mode, p);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (mode == kBackward) {
    if (p.rows <= 16) few_tied_kernel<1><<<grid, 256, 0, s>>>(q, f);
    else if (p.rows <= 32) few_tied_kernel<2><<<grid, 256, 0, s>>>(q, f);
    else few_tied_kernel<4><<<grid, 256, 0, s>>>(q, f);
  } else {
    if (p.rows <= 16) few_kernel<1><<<grid, 64 * kWaves, 0, s>>>(q, f);
    else if (p.rows <= 32) few_kernel<2><<<grid, 64 * kWaves, 0, s>>>(q, f);
    else few_kernel<4><<<grid, 64 * kWaves, 0, s>>>(q, f);
  }
  return (int)hipGetLastError();
}

}  // namespace moe
