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
// columns and a row per 4-wave workgroup above, 8 columns per lane and step:
// 5.4 TB/s with 16383 rows of 4096 bf16 columns and a gate per element (a copy:
// 4.9), 3.7 at 4099 columns, whose rows start at any even address.  Not kept: as
// many waves as the row needs (4099 columns 184 -> 195 us); octets shifted to
// aligned addresses (175 us, but 4096 columns 125 -> 168: more instructions
// per element, of which these rows have few to spare).
#include "common.h"
#include "kernels.h"
#include "moe.h"

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

// n (1..8) elements from i on; the others are 0
__device__ __forceinline__ void load8(const void* p, int64_t i, int type, int n, float (&v)[8]) {
  if (n == 8) {
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
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? elem(p, i + j, type) : 0.f;
  }
}
__device__ __forceinline__ void store8(void* p, int64_t i, int type, int n, const float (&v)[8]) {
  if (type == ET_F32) {
    float* d = (float*)p + i;
    if (n == 8) {
      *(f32x4_e*)d = f32x4_e{v[0], v[1], v[2], v[3]};
      *(f32x4_e*)(d + 4) = f32x4_e{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) d[j] = v[j];
    }
  } else {
    uint16_t* d = (uint16_t*)p + i;
    u16x8_a2 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = type == ET_BF16 ? bf16_bits(v[j]) : f2h(v[j]);
    if (n == 8) {
      *(u16x8_a2*)d = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) d[j] = o[j];
    }
  }
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

// LANES threads per row, NCH steps of LANES * 8 columns.  FRAG: h goes out as
// the verify path's GEMM operand.
template <int LANES, int NCH, bool FRAG>
__global__ __launch_bounds__(256) void block_norm_rows(BlockNormArgs a) {
  __shared__ float red[4];
  const int t = threadIdx.x & (LANES - 1);
  const int row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (row >= a.rows) return;  // whole waves (LANES 64) or none (LANES 256)
  const int64_t R = row;
  float x[NCH][8], v[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LANES + t) * 8, n = min(8, a.D - c);
    if (n > 0) load8(a.x, R * a.x_stride + c, a.x_type, n, x[i]);
    else
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
  }
  if (a.y) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * LANES + t) * 8, n = min(8, a.D - c);
      if (n > 0) load8(a.y, R * a.y_stride + c, a.y_type, n, v[i]);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
    float f = a.scale;
    if (a.gate && a.gate_col == 0) f *= elem(a.gate, R * a.gate_row, a.gate_type);
    if (a.post_gain) {
      float q = 0.f;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) q += v[i][j] * v[i][j];
      f *= rsqrtf(row_sum<LANES>(q, red) / (float)a.D + a.eps);
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (i * LANES + t) * 8, n = min(8, a.D - c);
        float g[8];
        if (n > 0) {
          load8(a.post_gain, c, ET_F32, n, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
      }
    }
    if (a.gate && a.gate_col != 0) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int c = (i * LANES + t) * 8, n = min(8, a.D - c);
        float g[8];
        if (n > 0) {
          load8(a.gate, R * a.gate_row + c, a.gate_type, n, g);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] += f * v[i][j];
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * LANES + t) * 8, n = min(8, a.D - c);
    float sq = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sq += x[i][j] * x[i][j];
    q += sq;
    if (n > 0 && a.x_out) store8(a.x_out, R * a.x_out_stride + c, a.x_type, n, x[i]);
    if constexpr (FRAG) {
      const float other = __shfl_xor(sq, 1);  // (D is a multiple of 16 here)
      if (n > 0) {
        float g[8], o[8];
        load8(a.gain, c, ET_F32, n, g);
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
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * LANES + t) * 8, n = min(8, a.D - c);
      if (n <= 0) continue;
      float g[8];
      load8(a.gain, c, ET_F32, n, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= x[i][j] * ir;
      store8(a.h, R * a.h_stride + c, a.h_type, n, g);
    }
  }
}

template <bool FRAG>
static void launch_bn(const BlockNormArgs& a, hipStream_t s) {
  const dim3 block(256), wide(a.rows), narrow((a.rows + 3) / 4);
  if (a.D <= 512) hvd_launch((block_norm_rows<64, 1, FRAG>), narrow, block, 0, s, a);
  else if (a.D <= 1024) hvd_launch((block_norm_rows<64, 2, FRAG>), narrow, block, 0, s, a);
  else if (a.D <= 2048) hvd_launch((block_norm_rows<256, 1, FRAG>), wide, block, 0, s, a);
  else if (a.D <= 4096) hvd_launch((block_norm_rows<256, 2, FRAG>), wide, block, 0, s, a);
  else if (a.D <= 6144) hvd_launch((block_norm_rows<256, 3, FRAG>), wide, block, 0, s, a);
  else if (a.D <= 8192) hvd_launch((block_norm_rows<256, 4, FRAG>), wide, block, 0, s, a);
  else hvd_launch((block_norm_rows<256, 8, FRAG>), wide, block, 0, s, a);
}

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  if (a.Nhi) launch_bn<true>(a, s);
  else launch_bn<false>(a, s);
  return hipGetLastError();
}

}  // namespace hvd
