// moe_route.hip -- tokens choose experts: scores, groups, top-k, weights; and the logits' gradient.
//
// L lanes hold a token's logits, V neighbouring ones each (lane i: experts i V .. i V + V - 1), so a
// reduction over the experts is V - 1 register steps and log2(L) lane steps, and the lowest lane that
// holds a value holds its lowest index. 16 lanes a token (up to 256 experts) keep the lane steps inside a
// row of 16, where they are one instruction each; 64 lanes hold up to 1024 experts.
// The chosen experts go to a few words of LDS; from there lane j of the token computes weight j.
// The vector instructions bound it where tokens are many: 40001 tokens of 192 experts, 6 chosen from 3 of 6 groups, 30 us
// (its bytes are 4; 6 us of it are the scores' exponentials and divisions in full), gradient 10 us; 8192 tokens, top 2 of 128, 4 us
// each way.
#include "moe_internal.h"

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxGroups = SKEW_MAX_GROUPS;
constexpr float kClosed = -INFINITY;

// value of the lane that is N lanes on within its row of 16
template <int N>
__device__ __forceinline__ float ror(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xF, 0xF, false));
}
template <int L, class F>
__device__ __forceinline__ float all_reduce(float x, F f) {
  x = f(x, ror<8>(x));
  x = f(x, ror<4>(x));
  x = f(x, ror<2>(x));
  x = f(x, ror<1>(x));
  if (L == 64) {
    x = f(x, __shfl_xor(x, 16));
    x = f(x, __shfl_xor(x, 32));
  }
  return x;
}
template <int L>
__device__ __forceinline__ float max_over(float x) {
  return all_reduce<L>(x, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ __forceinline__ float sum_over(float x) {
  return all_reduce<L>(x, [](float a, float b) { return a + b; });
}

// the two highest of two pairs (a1 >= a2, b1 >= b2)
__device__ __forceinline__ void top2(float &a1, float &a2, float b1, float b2) {
  const float lo = fminf(a1, b1);
  a1 = fmaxf(a1, b1);
  a2 = fmaxf(lo, fmaxf(a2, b2));
}
template <int L>
__device__ __forceinline__ void top2_over(float &a1, float &a2) {
  top2(a1, a2, ror<8>(a1), ror<8>(a2));
  top2(a1, a2, ror<4>(a1), ror<4>(a2));
  top2(a1, a2, ror<2>(a1), ror<2>(a2));
  top2(a1, a2, ror<1>(a1), ror<1>(a2));
  if (L == 64) {
    top2(a1, a2, __shfl_xor(a1, 16), __shfl_xor(a2, 16));
    top2(a1, a2, __shfl_xor(a1, 32), __shfl_xor(a2, 32));
  }
}

template <int V, class T>
__device__ __forceinline__ void load_row(const T *p, int n, float *o) {
  if (V >= 8) {
#pragma unroll
    for (int v = 0; v < V; v += 8) load8(p + v, n - v, o + v);
  } else {
#pragma unroll
    for (int v = 0; v < V; v++) o[v] = v < n ? to_f32(p[v]) : 0.0f;
  }
}

__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }
// The sigmoids of a token's chosen logits (-inf: none) up to a common factor, for weights that are renormalised: with
// u = min(l, 0), sigmoid(l) = exp(u) / (1 + exp(-|l|)), and exp(u - max u) does not underflow for all of them.
template <int L>
__device__ __forceinline__ float shifted_sigmoid(float l) {
  const float u = fminf(l, 0.0f), m = max_over<L>(u);   // (a NaN is in the divisor)
  return l == kClosed ? 0.0f : expf(u - m) / (1.0f + expf(-fabsf(l)));
}

template <int L, int V, class T>
__global__ __launch_bounds__(kThreads) void route_kernel(skew_route_desc d, const T *logits, const float *bias,
                                                         float *weights, int32_t *chosen) {
  constexpr int kTokens = kThreads / L;
  __shared__ float gval[kTokens][kMaxGroups];
  __shared__ int32_t pick_e[kTokens][SKEW_MAX_CHOICES];
  const int lane = threadIdx.x % L, slot = threadIdx.x / L;
  const int64_t t = (int64_t)blockIdx.x * kTokens + slot;
  const bool on = t < d.tokens;
  const int e0 = lane * V, n = on ? d.experts - e0 : 0;   // this lane's experts: the first n of its V
  float l[V], c[V];
  load_row<V>(logits + (on ? t * d.ld + (n > 0 ? e0 : 0) : 0), n, l);
#pragma unroll
  for (int v = 0; v < V; v++)
    if (v >= n) l[v] = kClosed;

  float mx = 0.0f, sum = 0.0f;
  const bool whole = d.score == SKEW_SCORE_SOFTMAX && (bias != nullptr || !d.renormalize);
  if (whole) {
    mx = l[0];
#pragma unroll
    for (int v = 1; v < V; v++) mx = fmaxf(mx, l[v]);
    mx = max_over<L>(mx);
    mx = mx == kClosed ? 0.0f : mx;   // no open expert: every exp is 0
#pragma unroll
    for (int v = 0; v < V; v++) {
      c[v] = expf(l[v] - mx);
      sum += c[v];
    }
    sum = sum_over<L>(sum);
  }
  if (bias != nullptr) {
    float add[V];
    load_row<V>(bias + (n > 0 ? e0 : 0), n, add);
    // A NaN or an infinity makes the sum NaN: its own value stays NaN, which is the highest, and the others have their bias.
    const float r = sum != sum ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int v = 0; v < V; v++) {
      const float x = (d.score == SKEW_SCORE_SOFTMAX ? c[v] * r : sigmoid(l[v])) + add[v];
      c[v] = l[v] == kClosed ? kClosed : x;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; v++) c[v] = l[v];
  }
#pragma unroll
  for (int v = 0; v < V; v++) c[v] = c[v] != c[v] ? INFINITY : c[v];

  if (d.top_groups < d.groups) {
    const int per = d.experts / d.groups;
    const bool whole_lanes = per % V == 0;   // a lane's experts are of one group
    const int own = e0 / per;
    float a1 = kClosed, a2 = kClosed;
    if (whole_lanes) {
#pragma unroll
      for (int v = 0; v < V; v++) top2(a1, a2, c[v], kClosed);
    }
    auto value = [&](float v1, float v2) { return d.group_sum == 2 && v2 != kClosed ? v1 + v2 : v1; };
    const int lanes = per / V;
    if (whole_lanes && (lanes & (lanes - 1)) == 0) {   // all groups at once: each is 1, 2, 4 .. lanes
      for (int o = 1; o < lanes; o <<= 1) top2(a1, a2, __shfl_xor(a1, o), __shfl_xor(a2, o));
      if (lane % lanes == 0 && own < d.groups) gval[slot][own] = value(a1, a2);
    } else {
      for (int g = 0; g < d.groups; g++) {
        float b1 = kClosed, b2 = kClosed;
        if (whole_lanes) {
          b1 = own == g ? a1 : kClosed;
          b2 = own == g ? a2 : kClosed;
        } else {
#pragma unroll
          for (int v = 0; v < V; v++) top2(b1, b2, (unsigned)(e0 + v - g * per) < (unsigned)per ? c[v] : kClosed, kClosed);
        }
        top2_over<L>(b1, b2);
        if (lane == 0) gval[slot][g] = value(b1, b2);
      }
    }
    __syncthreads();
    // a group is kept if fewer than top_groups are before it
    uint64_t kept = 0;
    for (int g0 = 0; g0 < d.groups; g0 += L) {
      const int g = g0 + lane;
      bool keep = false;
      if (g < d.groups) {
        const float mine = gval[slot][g];
        int before = 0;
        for (int h = 0; h < d.groups; h++) {
          const float x = gval[slot][h];
          before += x > mine || (x == mine && h < g);
        }
        keep = before < d.top_groups;
      }
      uint64_t b = __ballot(keep);
      if (L < 64) b = (b >> (threadIdx.x & 63 & ~(L - 1))) & ((1ull << (L & 63)) - 1);
      kept |= b << g0;
    }
    int g = own, left = per - (e0 - own * per);   // experts until the next group
#pragma unroll
    for (int v = 0; v < V; v++) {
      if (v < n && !((kept >> g) & 1)) c[v] = kClosed;
      if (--left == 0) {
        left = per;
        g++;
      }
    }
  }

  for (int j = 0; j < d.k; j++) {
    float head = c[0];
#pragma unroll
    for (int v = 1; v < V; v++) head = fmaxf(head, c[v]);
    const float m = max_over<L>(head);
    uint64_t b = __ballot(head == m && m != kClosed);
    if (L < 64) b = (b >> (threadIdx.x & 63 & ~(L - 1))) & ((1ull << (L & 63)) - 1);
    const int win = b != 0 ? (int)__builtin_ctzll(b) : -1;
    bool open = lane == win;   // this lane holds it: the first of its values that equals m
    int at = 0;
#pragma unroll
    for (int v = 0; v < V; v++) {
      const bool hit = open && c[v] == m;
      at = hit ? v : at;
      c[v] = hit ? kClosed : c[v];
      open = open && !hit;
    }
    if (lane == win || (win < 0 && lane == 0)) pick_e[slot][j] = win < 0 ? -1 : e0 + at;
  }
  __syncthreads();
  if (!on) return;
  const bool has = lane < d.k;
  const int e = has ? pick_e[slot][lane] : -1;
  const float x = e >= 0 ? to_f32(logits[t * d.ld + e]) : kClosed;
  float s;
  if (d.score == SKEW_SCORE_SOFTMAX) {
    if (d.renormalize) {   // the softmax over the chosen logits
      mx = max_over<L>(x);
      sum = 1.0f;
    }
    s = e >= 0 ? expf(x - mx) / sum : 0.0f;
  } else {
    s = d.renormalize ? shifted_sigmoid<L>(x) : e >= 0 ? sigmoid(x) : 0.0f;
  }
  if (d.renormalize) {
    const float total = sum_over<L>(s);
    s = e < 0 ? 0.0f : s / total;   // (a NaN in the total is not a weight of the places left over)
  }
  if (has) {
    weights[t * d.k + lane] = d.scale * s;
    chosen[t * d.k + lane] = e;
  }
}

template <int L, int V, class T>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(skew_route_desc d, const T *logits,
                                                                  const int32_t *chosen, const float *dweights,
                                                                  T *dlogits) {
  constexpr int kTokens = kThreads / L;
  const int lane = threadIdx.x % L, slot = threadIdx.x / L;
  const int64_t t = (int64_t)blockIdx.x * kTokens + slot;
  const bool on = t < d.tokens;
  const T *row = logits + (on ? t * d.ld : 0);
  const bool has = on && lane < d.k;
  int e = has ? chosen[t * d.k + lane] : -1;
  if ((unsigned)e >= (unsigned)d.experts) e = -1;
  const float x = e >= 0 ? to_f32(row[e]) : kClosed;
  const float dw = e >= 0 ? d.scale * dweights[t * d.k + lane] : 0.0f;
  const int e0 = lane * V, n = on ? d.experts - e0 : 0;
  float o[V];
#pragma unroll
  for (int v = 0; v < V; v++) o[v] = 0.0f;
  float g;   // the gradient of this lane's chosen logit (without renormalisation: the part on the chosen alone)
  if (d.score == SKEW_SCORE_SOFTMAX) {
    float mx, sum, s;
    if (d.renormalize) {
      mx = max_over<L>(x);
      s = e >= 0 ? expf(x - mx) : 0.0f;
      sum = sum_over<L>(s);
    } else {
      float l[V];
      load_row<V>(row + (n > 0 ? e0 : 0), n, l);
      mx = kClosed;
#pragma unroll
      for (int v = 0; v < V; v++) mx = fmaxf(mx, v < n ? l[v] : kClosed);
      mx = max_over<L>(mx);
      mx = mx == kClosed ? 0.0f : mx;
      sum = 0.0f;
#pragma unroll
      for (int v = 0; v < V; v++) {
        o[v] = v < n ? expf(l[v] - mx) : 0.0f;
        sum += o[v];
      }
      sum = sum_over<L>(sum);
      s = e >= 0 ? expf(x - mx) : 0.0f;
    }
    s = sum == 0.0f ? 0.0f : s / sum;
    const float mean = sum_over<L>(dw * s);   // sum of ds_i s_i over the chosen
    g = s * (dw - mean);
    if (!d.renormalize) {
      const float f = sum == 0.0f ? 0.0f : mean / sum;
#pragma unroll
      for (int v = 0; v < V; v++) o[v] = -o[v] * f;
    }
  } else {
    const float rest = e >= 0 ? sigmoid(-x) : 0.0f;   // 1 - s without its cancellation
    if (d.renormalize) {
      const float s = shifted_sigmoid<L>(x);
      const float total = sum_over<L>(s);
      const float w = total == 0.0f ? 0.0f : s / total;
      const float mean = sum_over<L>(dw * w);
      g = w * rest * (dw - mean);
    } else {
      g = e >= 0 ? dw * sigmoid(x) * rest : 0.0f;
    }
  }
  for (int j = 0; j < d.k; j++) {
    const int src = (threadIdx.x & 63 & ~(L - 1)) + j;
    const int ej = __shfl(e, src);
    const float gj = __shfl(g, src);
#pragma unroll
    for (int v = 0; v < V; v++)
      if (ej == e0 + v) o[v] = gj;
  }
  T *out = dlogits + (on ? t * d.experts : 0) + e0;
  if (n <= 0) return;
  if (V >= 8) {
#pragma unroll
    for (int v = 0; v < V; v += 8) store8(out + v, n - v, o + v);
  } else {
#pragma unroll
    for (int v = 0; v < V; v++)
      if (v < n) put(out + v, o[v]);
  }
}

template <class F>
void by_experts(int experts, F f) {
  auto c = [](auto x) { return x; };
  using std::integral_constant;
  if (experts <= 16) f(c(integral_constant<int, 16>()), c(integral_constant<int, 1>()));
  else if (experts <= 64) f(c(integral_constant<int, 16>()), c(integral_constant<int, 4>()));
  else if (experts <= 128) f(c(integral_constant<int, 16>()), c(integral_constant<int, 8>()));
  else if (experts <= 256) f(c(integral_constant<int, 16>()), c(integral_constant<int, 16>()));
  else if (experts <= 512) f(c(integral_constant<int, 64>()), c(integral_constant<int, 8>()));
  else f(c(integral_constant<int, 64>()), c(integral_constant<int, 16>()));
}

}  // namespace

int launch_route(const skew_route_desc &d, const void *logits, const float *bias, float *weights, int32_t *chosen,
                 void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_experts(d.experts, [&](auto L, auto V) {
    const unsigned grid = (unsigned)((d.tokens + kThreads / L - 1) / (kThreads / L));
    if (d.dtype == SKEW_F32)
      route_kernel<L, V, float><<<grid, kThreads, 0, s>>>(d, static_cast<const float *>(logits), bias, weights, chosen);
    else
      route_kernel<L, V, bf16_t><<<grid, kThreads, 0, s>>>(d, static_cast<const bf16_t *>(logits), bias, weights, chosen);
  });
  return (int)hipGetLastError();
}

int launch_route_backward(const skew_route_desc &d, const void *logits, const int32_t *chosen, const float *dweights,
                          void *dlogits, void *stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  by_experts(d.experts, [&](auto L, auto V) {
    const unsigned grid = (unsigned)((d.tokens + kThreads / L - 1) / (kThreads / L));
    if (d.dtype == SKEW_F32)
      route_backward_kernel<L, V, float><<<grid, kThreads, 0, s>>>(d, static_cast<const float *>(logits), chosen,
                                                                   dweights, static_cast<float *>(dlogits));
    else
      route_backward_kernel<L, V, bf16_t><<<grid, kThreads, 0, s>>>(d, static_cast<const bf16_t *>(logits), chosen,
                                                                    dweights, static_cast<bf16_t *>(dlogits));
  });
  return (int)hipGetLastError();
}

}  // namespace moe
