// Norms before and after a block, fused with its gate and residual scale
// (gfx950).  For each row, with rms(v) = v / sqrt(mean(v^2) + eps):
//
//   v  = rms(y) * post_gain        (y itself without a post_gain)
//   x' = x + scale * gate * v      (x itself without a y)
//   h  = rms(x') * gain
//
// x' and h come from the same 32-bit values (h does not see x' rounded to its
// type); each output is rounded once.  Memory bound: every element is read
// once and held in registers through both norms, a row per wave up to 1024
// columns and a row per 4-wave workgroup above, 8 columns per lane and step, and
// the columns left over one to a lane: 5.3 TB/s with 16383 rows of 4096 bf16
// columns and a gate per element (a copy: 4.9), 4.35 at 4099 columns, whose rows
// start at any even address (with the three columns past 4096 as an octet of
// their own: 3.65).  Not kept there: as many waves as the row needs (184 -> 195
// us); octets shifted to aligned addresses (175 us, but 4096 columns 125 -> 168:
// more instructions per element, of which these rows have few to spare).
#include "common.h"
#include "kernels.h"
#include "moe.h"

#include <algorithm>

namespace hvd {

// Eight elements at any address their type allows: the types say so, as
// global memory needs no more.
typedef uint16_t u16x8_a2 __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4_e __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float elem(const void* p, int64_t i, int type) {
  if (type == ET_F32) return ((const float*)p)[i];
  const uint16_t b = ((const uint16_t*)p)[i];
  return type == ET_BF16 ? bf2f(b) : h2f(b);
}
// Round to nearest even, NaN kept (f2bf takes finite values only).
__device__ __forceinline__ uint16_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

__device__ __forceinline__ void load8(const void* p, int64_t i, int type, float (&v)[8]) {
  if (type == ET_F32) {
    const f32x4_e a = *(const f32x4_e*)((const float*)p + i), b = *(const f32x4_e*)((const float*)p + i + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  } else {
    const u16x8_a2 a = *(const u16x8_a2*)((const uint16_t*)p + i);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = type == ET_BF16 ? bf2f(a[j]) : h2f(a[j]);
  }
}
__device__ __forceinline__ void store8(void* p, int64_t i, int type, const float (&v)[8]) {
  if (type == ET_F32) {
    float* d = (float*)p + i;
    *(f32x4_e*)d = f32x4_e{v[0], v[1], v[2], v[3]};
    *(f32x4_e*)(d + 4) = f32x4_e{v[4], v[5], v[6], v[7]};
  } else {
    u16x8_a2 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = type == ET_BF16 ? bf16_bits(v[j]) : f2h(v[j]);
    *(u16x8_a2*)((uint16_t*)p + i) = o;
  }
}
__device__ __forceinline__ void store1(void* p, int64_t i, int type, float v) {
  if (type == ET_F32) ((float*)p)[i] = v;
  else ((uint16_t*)p)[i] = type == ET_BF16 ? bf16_bits(v) : f2h(v);
}

// Sum over the LANES threads of a row (64: a wave; 256: the workgroup), in a
// fixed order.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (LANES > 64) {
    __syncthreads();  // the previous sum has been read
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) v += red[w];
  }
  return v;
}

// LANES threads per row, NCH steps of LANES * 8 columns up to column `octets`;
// the columns left over, at most LANES, go one to a lane (a last octet read
// element by element held every row up, as did a whole step for a few columns).
// FRAG: h goes out as the verify path's GEMM operand.
template <int LANES, int NCH, bool FRAG>
__global__ __launch_bounds__(256) void block_norm_rows(BlockNormArgs a, int octets) {
  __shared__ float red[4];
  const int t = threadIdx.x & (LANES - 1);
  const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (row >= a.rows) return;  // whole waves (LANES 64) or none (LANES 256)
  const int64_t R = row;
  float x[NCH][8], v[NCH][8];
  const int ce = octets + t;  // this lane's single column
  const bool one = !FRAG && ce < a.D;
  float xe = 0.f, ve = 0.f;
  if (one) {
    xe = elem(a.x, R * a.x_stride + ce, a.x_type);
    if (a.y) ve = elem(a.y, R * a.y_stride + ce, a.y_type);
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LANES + t) * 8;
    if (c < octets) load8(a.x, R * a.x_stride + c, a.x_type, x[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
  }
  if (a.y) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * LANES + t) * 8;
      if (c < octets) load8(a.y, R * a.y_stride + c, a.y_type, v[i]);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
    float f = a.scale;
    if (a.gate && a.gate_col == 0) f *= elem(a.gate, R * a.gate_row, a.gate_type);
    if (a.post_gain) {
      float q = ve * ve;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) q += v[i][j] * v[i][j];
      f *= rsqrtf(row_sum<LANES>(q, red) / (float)a.D + a.eps);
      if (one) ve *= a.post_gain[ce];
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (i * LANES + t) * 8;
        float g[8];
        if (c < octets) {
          load8(a.post_gain, c, ET_F32, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
      }
    }
    if (a.gate && a.gate_col != 0) {
      if (one) ve *= elem(a.gate, R * a.gate_row + ce, a.gate_type);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (i * LANES + t) * 8;
        float g[8];
        if (c < octets) {
          load8(a.gate, R * a.gate_row + c, a.gate_type, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] += f * v[i][j];
    if (one) xe += f * ve;
  }
  float q = xe * xe;
  if (one && a.x_out) store1(a.x_out, R * a.x_out_stride + ce, a.x_type, xe);
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LANES + t) * 8;
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sq += x[i][j] * x[i][j];
    q += sq;
    if (c < octets && a.x_out) store8(a.x_out, R * a.x_out_stride + c, a.x_type, x[i]);
    if constexpr (FRAG) {
      const float other = __shfl_xor(sq, 1);  // (D is a multiple of 16 here)
      if (c < octets) {
        float g[8], o[8];
        load8(a.gain, c, ET_F32, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = x[i][j] * g[j];
        uint4 hi, lo;
        split8(o, hi, lo);
        const size_t off = afrag_off(row, c, a.MTtot);
        *(uint4*)(a.Nhi + off) = hi;
        *(uint4*)(a.Nlo + off) = lo;
        if ((t & 1) == 0) a.ss_out[(size_t)row * (a.D >> 4) + (c >> 4)] = sq + other;
      }
    }
  }
  if constexpr (!FRAG) {
    if (!a.h) return;
    const float ir = rsqrtf(row_sum<LANES>(q, red) / (float)a.D + a.eps);
    if (one) store1(a.h, R * a.h_stride + ce, a.h_type, xe * ir * a.gain[ce]);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * LANES + t) * 8;
      if (c >= octets) continue;
      float g[8];
      load8(a.gain, c, ET_F32, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= x[i][j] * ir;
      store8(a.h, R * a.h_stride + c, a.h_type, g);
    }
  }
}

template <int LANES, int NCH, bool FRAG>
static void launch_n(const BlockNormArgs& a, hipStream_t s) {
  const int octets = std::min(NCH * LANES * 8, a.D & ~7);
  hvd_launch((block_norm_rows<LANES, NCH, FRAG>), dim3(LANES == 64 ? (a.rows + 3) / 4 : a.rows), dim3(256), 0, s, a, octets);
}
// One column per lane past the last step, unless FRAG (whole 64-column blocks).
template <bool FRAG>
static void launch_bn(const BlockNormArgs& a, hipStream_t s) {
  constexpr int X1 = FRAG ? 0 : 64, X4 = FRAG ? 0 : 256;
  if (a.D <= 512 + X1) launch_n<64, 1, FRAG>(a, s);
  else if (a.D <= 1024 + X1) launch_n<64, 2, FRAG>(a, s);
  else if (a.D <= 2048 + X4) launch_n<256, 1, FRAG>(a, s);
  else if (a.D <= 4096 + X4) launch_n<256, 2, FRAG>(a, s);
  else if (a.D <= 6144 + X4) launch_n<256, 3, FRAG>(a, s);
  else if (a.D <= 8192 + X4) launch_n<256, 4, FRAG>(a, s);
  else launch_n<256, 8, FRAG>(a, s);
}

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  if (a.Nhi) launch_bn<true>(a, s);
  else launch_bn<false>(a, s);
  return hipGetLastError();
}

}  // namespace hvd
