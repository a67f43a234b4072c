// moe_order.hip -- stable radix sort of small keys: places by expert, tokens by id.
//
// A pass sorts by one digit of up to 9 bits. Within a wave, the lanes that hold the same digit are
// found by one ballot per digit bit; a lane's rank is the number of such lanes before it plus the
// wave's running count of the digit in LDS. Ranks of waves and work-groups are joined by exclusive
// sums, so equal keys keep their order and no atomic decides a place.
//   up to 16384 items: one work-group of 16 waves, all passes in LDS (a key and an index share 32 bits)
//   more: per pass a histogram per work-group of 4096 items, the sums over the groups, and the scatter
#include "moe_internal.h"

namespace moe {

SortPlan sort_plan(int64_t n, int64_t keys) {
  SortPlan p;
  p.n = n;
  p.keys = (uint32_t)keys;
  const int bits = bits_for((uint64_t)keys);
  p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  p.digit = (bits + p.passes - 1) / p.passes;
  p.small = n <= kSmallSort && bits <= 18;   // 14 bits of index and 18 of key share a word
  p.nb = (n + kSortBlock - 1) / kSortBlock;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += pad256(bytes);
    return o;
  };
  for (int i = 0; i < 2; i++) {
    p.off_key[i] = take((size_t)n * 4);
    p.off_idx[i] = take((size_t)n * 4);
  }
  if (!p.small) {
    p.off_hist = take((size_t)p.nb << (p.digit + 2));
    p.off_total = take((size_t)4 << p.digit);
  }
  p.bytes = at;
  return p;
}

namespace {

__device__ __forceinline__ uint32_t key_of(const void *ids, int id_bytes, int64_t i, uint32_t keys) {
  const int64_t v = id_bytes == 8 ? static_cast<const int64_t *>(ids)[i] : static_cast<const int32_t *>(ids)[i];
  return v < 0 || v >= (int64_t)keys ? keys : (uint32_t)v;
}

// The lanes of the wave whose digit is this lane's, among the lanes of `live`.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, uint64_t live) {
  uint64_t m = live;
  for (int b = 0; b < bits; b++) {
    const uint64_t one = __ballot((d >> b) & 1);
    m &= (d >> b) & 1 ? one : ~one;
  }
  return m;
}

// This lane's rank among the wave's items of digit d so far; cnt: the wave's counts in LDS.
__device__ __forceinline__ uint32_t wave_rank(uint32_t d, int bits, bool on, volatile uint32_t *cnt) {
  const uint64_t m = same_digit(d, bits, __ballot(on));
  const uint64_t before = m & ((1ull << (threadIdx.x & 63)) - 1);
  uint32_t old = 0;
  if (on) old = cnt[d];
  __builtin_amdgcn_wave_barrier();
  if (on && before == 0) cnt[d] = old + (uint32_t)__popcll(m);
  __builtin_amdgcn_wave_barrier();
  return old + (uint32_t)__popcll(before);
}

// Exclusive sum over the work-group's threads (a multiple of 64); tmp: one word per wave.
__device__ uint32_t block_exclusive(uint32_t v, uint32_t *tmp) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  uint32_t s = v;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(s, o);
    if (lane >= o) s += u;
  }
  if (lane == 63) tmp[w] = s;
  __syncthreads();
  uint32_t base = 0;
  for (int i = 0; i < nw; i++)
    if (i < w) base += tmp[i];
  __syncthreads();
  return base + s - v;
}

// One work-group sorts everything. Item words: key << 14 | index.
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64, kPerThread = kSmallSort / kSmallThreads;

__global__ __launch_bounds__(kSmallThreads) void sort_small(const void *ids, int id_bytes, int n, uint32_t keys,
                                                            int passes, int digit, uint32_t *key, int32_t *idx,
                                                            int32_t *offsets, int32_t *rows, int32_t *slots) {
  __shared__ uint32_t item[kSmallSort];
  __shared__ uint32_t cnt[kSmallWaves << kMaxDigit];
  __shared__ uint32_t first[1 << kMaxDigit];
  __shared__ uint32_t tmp[kSmallWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, bins = 1 << digit;
  // wave w takes items [w * per, (w + 1) * per), 64 at a time
  const int steps = (n + kSmallThreads - 1) / kSmallThreads, per = steps * 64;
  uint32_t it[kPerThread], rank[kPerThread];
#pragma unroll
  for (int s = 0; s < kPerThread; s++) {
    const int i = w * per + s * 64 + lane;
    it[s] = s < steps && i < n ? key_of(ids, id_bytes, i, keys) << 14 | (uint32_t)i : 0;
  }
  for (int pass = 0; pass < passes; pass++) {
    const int shift = 14 + pass * digit;
    for (int i = tid; i < kSmallWaves * bins; i += kSmallThreads) cnt[i] = 0;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kPerThread; s++)
      if (s < steps)
        rank[s] = wave_rank((it[s] >> shift) & (bins - 1), digit, w * per + s * 64 + lane < n, cnt + w * bins);
    __syncthreads();
    uint32_t total = 0;
    if (tid < bins)
      for (int v = 0; v < kSmallWaves; v++) {
        const uint32_t c = cnt[v * bins + tid];
        cnt[v * bins + tid] = total;
        total += c;
      }
    const uint32_t base = block_exclusive(total, tmp);
    if (tid < bins) first[tid] = base;
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kPerThread; s++)
      if (s < steps && w * per + s * 64 + lane < n) {
        const uint32_t d = (it[s] >> shift) & (bins - 1);
        item[first[d] + cnt[w * bins + d] + rank[s]] = it[s];
      }
    __syncthreads();
    if (pass + 1 < passes) {
#pragma unroll
      for (int s = 0; s < kPerThread; s++) {
        const int i = w * per + s * 64 + lane;
        if (s < steps && i < n) it[s] = item[i];
      }
    }
  }
  for (int i = tid; i < n; i += kSmallThreads) {
    const uint32_t v = item[i], k = v >> 14;
    const int32_t j = (int32_t)(v & (kSmallSort - 1));
    if (rows) {
      rows[i] = k < keys ? j : -1;
      slots[j] = k < keys ? i : -1;
    } else {
      key[i] = k;
      idx[i] = j;
    }
  }
  // offsets[e]: the number of keys below e, by halving
  if (offsets)
    for (uint32_t e = tid; e <= keys; e += kSmallThreads) {
      int lo = 0, hi = n;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((item[mid] >> 14) < e) lo = mid + 1;
        else hi = mid;
      }
      offsets[e] = lo;
    }
}

constexpr int kSortThreads = 256, kSortWaves = kSortThreads / 64, kSortSteps = kSortBlock / kSortThreads;

// item i of this thread: waves take runs of kSortBlock / 4 items, 64 at a time
__device__ __forceinline__ int64_t sort_item(int s) {
  return (int64_t)blockIdx.x * kSortBlock + (threadIdx.x >> 6) * (kSortSteps * 64) + s * 64 + (threadIdx.x & 63);
}

// hist[digit][group]: how many of the group's items have the digit
__global__ __launch_bounds__(kSortThreads) void sort_count(const void *ids, int id_bytes, const uint32_t *key_in,
                                                           int64_t n, uint32_t keys, int shift, int digit,
                                                           uint32_t *hist, int64_t nb) {
  __shared__ uint32_t cnt[1 << kMaxDigit];
  const int bins = 1 << digit;
  for (int i = threadIdx.x; i < bins; i += kSortThreads) cnt[i] = 0;
  __syncthreads();
  for (int s = 0; s < kSortSteps; s++) {
    const int64_t i = sort_item(s);
    if (i < n) {
      const uint32_t k = key_in ? key_in[i] : key_of(ids, id_bytes, i, keys);
      atomicAdd(&cnt[(k >> shift) & (bins - 1)], 1u);   // integer counts: their order does not show
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kSortThreads) hist[(int64_t)i * nb + blockIdx.x] = cnt[i];
}

// One work-group per digit: its counts become their exclusive sums, its total goes to total[digit]
__global__ __launch_bounds__(256) void sort_sums(uint32_t *hist, int64_t nb, uint32_t *total) {
  __shared__ uint32_t tmp[4];
  __shared__ uint32_t carry;
  uint32_t *h = hist + (int64_t)blockIdx.x * nb;
  uint32_t run = 0;
  for (int64_t b = 0; b < nb; b += 256) {
    const int64_t i = b + threadIdx.x;
    const uint32_t v = i < nb ? h[i] : 0;
    const uint32_t ex = block_exclusive(v, tmp);
    if (i < nb) h[i] = run + ex;
    if (threadIdx.x == 255) carry = ex + v;
    __syncthreads();
    run += carry;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[blockIdx.x] = run;
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter(const void *ids, int id_bytes, const uint32_t *key_in,
                                                             const int32_t *idx_in, int64_t n, uint32_t keys,
                                                             int shift, int digit, const uint32_t *hist, int64_t nb,
                                                             const uint32_t *total, uint32_t *key_out,
                                                             int32_t *idx_out, int32_t *rows, int32_t *slots) {
  __shared__ uint32_t cnt[kSortWaves << kMaxDigit];
  __shared__ uint32_t first[1 << kMaxDigit];
  __shared__ uint32_t tmp[kSortWaves];
  const int tid = threadIdx.x, w = tid >> 6, bins = 1 << digit;
  for (int i = tid; i < kSortWaves * bins; i += kSortThreads) cnt[i] = 0;
  // the first place of each digit: two digits a thread
  const uint32_t t0 = 2 * tid < bins ? total[2 * tid] : 0, t1 = 2 * tid + 1 < bins ? total[2 * tid + 1] : 0;
  const uint32_t ex = block_exclusive(t0 + t1, tmp);
  if (2 * tid < bins) first[2 * tid] = ex + hist[(int64_t)(2 * tid) * nb + blockIdx.x];
  if (2 * tid + 1 < bins) first[2 * tid + 1] = ex + t0 + hist[(int64_t)(2 * tid + 1) * nb + blockIdx.x];
  __syncthreads();
  uint32_t key[kSortSteps], rank[kSortSteps];
#pragma unroll
  for (int s = 0; s < kSortSteps; s++) {
    const int64_t i = sort_item(s);
    key[s] = i < n ? (key_in ? key_in[i] : key_of(ids, id_bytes, i, keys)) : 0;
    rank[s] = wave_rank((key[s] >> shift) & (bins - 1), digit, i < n, cnt + w * bins);
  }
  __syncthreads();
  for (int d = tid; d < bins; d += kSortThreads) {
    uint32_t run = first[d];
    for (int v = 0; v < kSortWaves; v++) {
      const uint32_t c = cnt[v * bins + d];
      cnt[v * bins + d] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < kSortSteps; s++) {
    const int64_t i = sort_item(s);
    if (i < n) {
      const uint32_t at = cnt[w * bins + ((key[s] >> shift) & (bins - 1))] + rank[s];
      const int32_t j = idx_in ? idx_in[i] : (int32_t)i;
      key_out[at] = key[s];
      if (rows) {
        rows[at] = key[s] < keys ? j : -1;
        slots[j] = key[s] < keys ? (int32_t)at : -1;
      } else {
        idx_out[at] = j;
      }
    }
  }
}

// offsets[e]: the number of sorted keys below e
__global__ __launch_bounds__(256) void sort_offsets(const uint32_t *key, int64_t n, uint32_t keys, int32_t *offsets) {
  const uint32_t e = blockIdx.x * 256 + threadIdx.x;
  if (e > keys) return;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (key[mid] < e) lo = mid + 1;
    else hi = mid;
  }
  offsets[e] = (int32_t)lo;
}

}  // namespace

int launch_sort(const SortPlan &p, const void *ids, int id_bytes, char *ws, SortOut *out, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  auto key = [&](int i) { return reinterpret_cast<uint32_t *>(ws + p.off_key[i]); };
  auto idx = [&](int i) { return reinterpret_cast<int32_t *>(ws + p.off_idx[i]); };
  if (p.small) {
    sort_small<<<1, kSmallThreads, 0, s>>>(ids, id_bytes, (int)p.n, p.keys, p.passes, p.digit, key(0), idx(0),
                                           out->offsets, out->rows, out->slots);
    out->key = key(0);
    out->idx = idx(0);
    return (int)hipGetLastError();
  }
  uint32_t *hist = reinterpret_cast<uint32_t *>(ws + p.off_hist), *total = reinterpret_cast<uint32_t *>(ws + p.off_total);
  const uint32_t *key_in = nullptr;
  const int32_t *idx_in = nullptr;
  for (int pass = 0; pass < p.passes; pass++) {
    const bool last = pass + 1 == p.passes;
    const int to = pass & 1, shift = pass * p.digit;
    sort_count<<<(unsigned)p.nb, kSortThreads, 0, s>>>(ids, id_bytes, key_in, p.n, p.keys, shift, p.digit, hist, p.nb);
    sort_sums<<<1u << p.digit, 256, 0, s>>>(hist, p.nb, total);
    sort_scatter<<<(unsigned)p.nb, kSortThreads, 0, s>>>(ids, id_bytes, key_in, idx_in, p.n, p.keys, shift, p.digit,
                                                         hist, p.nb, total, key(to), idx(to),
                                                         last ? out->rows : nullptr, last ? out->slots : nullptr);
    key_in = key(to);
    idx_in = idx(to);
  }
  if (out->offsets) sort_offsets<<<(p.keys + 256) / 256, 256, 0, s>>>(key_in, p.n, p.keys, out->offsets);
  out->key = key_in;
  out->idx = idx_in;
  return (int)hipGetLastError();
}

}  // namespace moe
