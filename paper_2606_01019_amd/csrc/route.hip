// Routing of rows to experts (gfx950): scores, the choice among groups and
// experts, and the weights of the chosen.
//
// With l the logits of a row: s = softmax(l) or sigmoid(l) per expert,
// c = s + bias; a group counts the sum of its two best c; the top_groups best
// groups stay, and among their experts the k best c are chosen, in descending
// order, the lower index on ties.  Weights are s (not c) of the chosen, over
// their sum if renorm, times scale.  An expert with a logit of -inf or NaN (or
// such a c) is masked: it is never chosen and no group counts it; places
// without an expert get id -1 and weight 0.
//
// Scores are computed in 64 bits: a choice between two experts whose scores
// differ by less than a 32-bit rounding is the same however the exponentials
// are evaluated, and the 64-bit work of 256 experts is a few hundred cycles.
//
// One wave per row, the row's experts dealt over the lanes (expert i * 64 +
// lane), everything in registers; rows are independent, so the launch is
// bound by the latency of one row (a load, the score, k rounds of a wave-wide
// maximum) until there are several thousand.
#include "common.h"
#include "moe.h"
#include "kernels.h"

namespace hvd {

constexpr int kRouteRows = 4;  // rows (waves) per workgroup

// Exchanges within a wave in the vector ALU (data-parallel permutes): an LDS
// shuffle costs a round trip per step, and a row is k wave-wide maxima.
template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Every lane gets f over all 64 lanes' values: neighbours, pairs of two (quad
// permutes), of four and eight (mirrors), then across the four rows of 16.
template <class F>
__device__ __forceinline__ double wave_all_d(double v, F f) {
  v = f(v, dpp_d<0xB1>(v));
  v = f(v, dpp_d<0x4E>(v));
  v = f(v, dpp_d<0x141>(v));
  v = f(v, dpp_d<0x140>(v));
  uint64_t u = __builtin_bit_cast(uint64_t, v);
  const auto l16 = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false);
  const auto h16 = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  v = f(__builtin_bit_cast(double, (uint64_t)h16[0] << 32 | l16[0]), __builtin_bit_cast(double, (uint64_t)h16[1] << 32 | l16[1]));
  u = __builtin_bit_cast(uint64_t, v);
  const auto l32 = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false);
  const auto h32 = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
  return f(__builtin_bit_cast(double, (uint64_t)h32[0] << 32 | l32[0]), __builtin_bit_cast(double, (uint64_t)h32[1] << 32 | l32[1]));
}
__device__ __forceinline__ double wave_max_d(double v) {
  return wave_all_d(v, [](double a, double b) { return a > b ? a : b; });
}
__device__ __forceinline__ double wave_sum_d(double v) {
  return wave_all_d(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double shfl_xor_d(double v, int o) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __shfl_xor((uint32_t)u, o), hi = __shfl_xor((uint32_t)(u >> 32), o);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double read_lane_d(double v, int lane) {  // lane: wave-uniform
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, lane), hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float load_logit(const void* p, int64_t i, int dtype) {
  if (dtype == ET_F32) return ((const float*)p)[i];
  const uint16_t b = ((const uint16_t*)p)[i];
  return dtype == ET_BF16 ? bf2f(b) : h2f(b);
}

// P: experts per lane
template <int P>
__global__ __launch_bounds__(64 * kRouteRows) void route_rows(RouteArgs a) {
  constexpr double kNone = -__builtin_inf();
  __shared__ double sc[kRouteRows][P * 64];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.x * kRouteRows + wv;
  if (row >= a.rows) return;
  float l[P];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = i * 64 + lane;
    float v = e < a.E ? load_logit(a.logits, row * a.stride + e, a.dtype) : -INFINITY;
    v = v > -INFINITY ? fminf(v, 3.402823466e38f) : -INFINITY;  // NaN counts as masked
    l[i] = v;
    m = fmaxf(m, v);
  }
  m = (float)wave_max_d((double)m);  // (exact both ways)
  double s[P], c[P];
  if (a.sigmoid) {
#pragma unroll
    for (int i = 0; i < P; ++i) s[i] = 1.0 / (1.0 + exp(-(double)l[i]));
  } else {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      s[i] = l[i] > -INFINITY ? exp((double)l[i] - (double)m) : 0.0;
      sum += s[i];
    }
    sum = wave_sum_d(sum);
#pragma unroll
    for (int i = 0; i < P; ++i) s[i] = s[i] / sum;
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = i * 64 + lane;
    c[i] = l[i] > -INFINITY ? s[i] + (a.bias ? (double)a.bias[e] : 0.0) : kNone;
    if (!(c[i] > kNone)) c[i] = kNone;
  }

  if (a.G > 1) {
    // L = 64 / (next power of two of G) lanes per group find its two best
    const int S = a.E / a.G;
    int L = 64;
    while (64 / L < a.G) L >>= 1;
    const int g = lane / L, j = lane & (L - 1);
#pragma unroll
    for (int i = 0; i < P; ++i) sc[wv][i * 64 + lane] = c[i];
    __builtin_amdgcn_wave_barrier();  // (one wave's LDS accesses execute in order)
    double b1 = kNone, b2 = kNone;
    if (g < a.G)
      for (int q = j; q < S; q += L) {
        const double v = sc[wv][g * S + q];
        if (v > b1) {
          b2 = b1;
          b1 = v;
        } else if (v > b2) {
          b2 = v;
        }
      }
    for (int o = 1; o < L; o <<= 1) {
      const double o1 = shfl_xor_d(b1, o), o2 = shfl_xor_d(b2, o);
      b2 = o1 > b1 ? (b1 > o2 ? b1 : o2) : (o1 > b2 ? o1 : b2);
      b1 = o1 > b1 ? o1 : b1;
    }
    const double score = b2 > kNone ? b1 + b2 : b1;  // one unmasked expert counts alone
    int rank = 0;
    for (int q = 0; q < a.G; ++q) {
      const double other = read_lane_d(score, q * L);
      rank += (other > score || (other == score && q < g)) ? 1 : 0;
    }
    const uint64_t keep = __builtin_amdgcn_ballot_w64(g < a.G && rank < a.top_groups);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int e = i * 64 + lane;
      if (e < a.E && !(keep >> (e / S * L) & 1)) c[i] = kNone;
    }
  }

  // k rounds: the wave's best value, then the lowest expert that has it
  int my_id = -1;
  double my_s = 0.0, total = 0.0;
  for (int r = 0; r < a.k; ++r) {
    double best = c[0];
#pragma unroll
    for (int i = 1; i < P; ++i) best = c[i] > best ? c[i] : best;
    best = wave_max_d(best);
    if (!(best > kNone)) break;  // no expert is left
    bool found = false;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t has = __builtin_amdgcn_ballot_w64(c[i] == best);
      if (!found && has) {  // (wave-uniform)
        found = true;
        const int src = __builtin_ctzll(has);
        const double ws = read_lane_d(s[i], src);
        total += ws;
        if (lane == r) {
          my_id = i * 64 + src;
          my_s = ws;
        }
        if (lane == src) c[i] = kNone;
      }
    }
  }
  if (lane < a.k) {
    if (a.renorm) my_s = total > 0.0 ? my_s / total : 0.0;
    a.ids[(size_t)row * a.k + lane] = my_id;
    a.weights[(size_t)row * a.k + lane] = (float)(my_s * (double)a.scale);
  }
}

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  const dim3 grid((a.rows + kRouteRows - 1) / kRouteRows), block(64 * kRouteRows);
  if (a.E <= 64) hvd_launch(route_rows<1>, grid, block, 0, s, a);
  else if (a.E <= 128) hvd_launch(route_rows<2>, grid, block, 0, s, a);
  else if (a.E <= 256) hvd_launch(route_rows<4>, grid, block, 0, s, a);
  else hvd_launch(route_rows<8>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace hvd
