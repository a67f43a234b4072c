// head_few.hip -- the head's logits of a few rows where w's rows begin anywhere, and their softmax sums: w is read once, straight into
// fragments of the matrix instruction.
//
// The tiles of head_logits.hip need rows at 16-byte positions. To copy w for them costs more than the product of a few rows, which is
// nothing beside w's bytes. A lane loads 8 columns of 8 rows and turns the 8 x 8 block in its registers (4 byte permutes a load), as a
// fragment holds 8 neighbours along the contraction. Its 8 fragments are 8 products, of which number f has columns 8 j + f. The 8 waves of a
// work-group share the contraction. Rows, columns and the contraction may end anywhere.
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
// Registers for two work-groups on a compute unit. 50257 words of width 2048: 72 us, 2.9 TB/s (16-byte loads at odd 2-byte positions); at 16-byte
// positions 39 us.
__global__ __launch_bounds__(64 * kWaves, 4) void few_kernel(Few p, HeadForward f) {
  __shared__ float held[kWaves][16][132];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, group = lane >> 4;
  const int64_t col = ((int64_t)blockIdx.x * 16 + j) * 8, left = p.cols - col;
  f32x4 acc[8] = {};
  const int64_t steps = (p.K + 31) / 32;
  // a row's place: a scalar that moves from step to step, and the lane's 32-bit offset, which stays (24 rows and a row's columns lie within
  // 2^31 bytes)
  const uint32_t offset = (uint32_t)((group * 8 * p.ldw + col) * 2);
  const char *base = scalar(reinterpret_cast<const char *>(p.w));
  const int64_t row_bytes = scalar(p.ldw * 2);
  u32x4 w[2][8];
  auto load = [&](int64_t s, u32x4 *to) {
    const int64_t k = s * 32 + group * 8;
    const char *at = base + s * 32 * row_bytes;
    if (k + 8 <= p.K && left >= 8) {
#pragma unroll
      for (int r = 0; r < 8; r++) to[r] = *reinterpret_cast<const u32x4_a2 *>(at + r * row_bytes + offset);
    } else {
#pragma unroll
      for (int r = 0; r < 8; r++)
        to[r] = load_chunk(reinterpret_cast<const bf16_t *>(at + r * row_bytes + offset), k + r < p.K ? left : 0);
    }
  };
  auto multiply = [&](int64_t s, const u32x4 *v) {
    const bf16x8 x = x_part(p, j, s * 32 + group * 8);
#pragma unroll
    for (int c = 0; c < 8; c++) {
      u32x4 b;
#pragma unroll
      for (int i = 0; i < 4; i++) b[i] = __builtin_amdgcn_perm(v[2 * i + 1][c / 2], v[2 * i][c / 2], c % 2 ? 0x07060302 : 0x05040100);
      acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), x, acc[c], 0, 0, 0);
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
  for (int c = 0; c < 8; c++)
#pragma unroll
    for (int q = 0; q < 4; q++) held[wave][j][8 * (4 * group + q) + c] = acc[c][q];
  __syncthreads();
  // 32 threads a row, 4 columns each; the waves' parts in order
  const int row = tid >> 5;
  const int64_t first = (int64_t)blockIdx.x * 128 + (tid & 31) * 4;
  float z[4] = {}, m = -INFINITY, sum = 0.0f;
  const int64_t y = row < p.rows ? target_of(f, row) : -1;
#pragma unroll
  for (int q = 0; q < 4; q++) {
#pragma unroll
    for (int i = 0; i < kWaves; i++) z[q] += held[i][row][(tid & 31) * 4 + q];
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
  if ((tid & 31) == 0 && row < p.rows) f.part[row * f.part_ld + blockIdx.x] = HeadPair{top, sum};
}

}  // namespace

int launch_head_few(const HeadProduct &p, const HeadForward &f, void *stream) {
  const Few q = {static_cast<const bf16_t *>(p.a), static_cast<const bf16_t *>(p.b), p.lda, p.ldb, p.rows, p.cols, p.K};
  few_kernel<<<(unsigned)head_few_parts(p.cols), 64 * kWaves, 0, static_cast<hipStream_t>(stream)>>>(q, f);
  return (int)hipGetLastError();
}

}  // namespace moe
