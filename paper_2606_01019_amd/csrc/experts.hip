// The products of the experts a router chose (gfx950):
//
//   out[t] = sum_j w[t][j] Wd[e] (silu(Wg[e] x[t]) * (Wu[e] x[t])),  e = ids[t][j]
//
// A slot is one (t, j); ids outside [0, E) are empty slots.  The slots are put
// in expert order (ascending within an expert, so the order is fixed), the
// gate/up product runs over each expert's rows in that order, the down product
// over its result, and each row's k expert outputs are summed in 32 bits in
// the order of its slots.  The same expert twice in a row counts twice.
//
// Types: fp16 or bf16 weights with activations of the same type, or fp16
// weights with 32-bit activations as the fp16 hi + lo pair (two MFMAs per
// tile, about 22 bits).  The activation silu(gate) * up is rounded to that
// form, which is what the matrix instructions take; everything that is summed
// is 32-bit.
#include "common.h"
#include "kernels.h"
#include "moe.h"

namespace hvd {

// ---------------------------------------------------------------- weights

// dst fragment (expert, strip s, K step kt), lane l, half j = src row's element
// 32 kt + 8 (l/16) + j, with row 16 s + l%16 of the matrix (gate and up rows in
// alternating strips), at ((s/4 * KT + kt) * 4 + s%4) * 512 of the expert.
template <bool TO_F16>
__global__ void pack_experts(const uint16_t* __restrict__ gate, const uint16_t* __restrict__ up,
                             uint16_t* __restrict__ dst, int n, int rows, int cols) {
  const int KT = cols >> 5, strips = (up ? 2 * rows : rows) >> 4;
  const size_t per = (size_t)strips * KT * 64, total = per * n;
  for (size_t t = (size_t)blockIdx.x * blockDim.x + threadIdx.x; t < total; t += (size_t)gridDim.x * blockDim.x) {
    const size_t e = t / per, u = t - e * per;
    const int l = (int)(u & 63);
    const size_t frag = u >> 6;
    const int kt = (int)((frag >> 2) % KT), s = (int)((frag >> 2) / KT) * 4 + (int)(frag & 3);
    const uint16_t* src = up ? (s & 1 ? up : gate) : gate;
    const int row = (up ? s >> 1 : s) * 16 + (l & 15);
    uint4 v = *(const uint4*)(src + (e * rows + row) * (size_t)cols + kt * 32 + (l >> 4) * 8);
    if constexpr (TO_F16) {
      uint32_t* w = (uint32_t*)&v;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = pack_h2(bf2f((uint16_t)(w[j] & 0xFFFFu)), bf2f((uint16_t)(w[j] >> 16)));
    }
    *(uint4*)(dst + t * 8) = v;
  }
}

hipError_t launch_pack_experts(const uint16_t* gate, const uint16_t* up, uint16_t* dst, int n, int rows, int cols,
                               bool to_f16, hipStream_t s) {
  const size_t total = (size_t)n * (up ? 2 : 1) * rows * (cols / 8);
  const dim3 grid((unsigned)std::min<size_t>((total + 255) / 256, 65535 * 8));
  if (to_f16) hvd_launch(pack_experts<true>, grid, dim3(256), 0, s, gate, up, dst, n, rows, cols);
  else hvd_launch(pack_experts<false>, grid, dim3(256), 0, s, gate, up, dst, n, rows, cols);
  return hipGetLastError();
}

// ---------------------------------------------------------------- types

// BF: bf16 operands; HL: fp16 with activations as the hi + lo pair.
template <bool BF>
__device__ __forceinline__ f32x4 mfma16(const u32x4& a, const u32x4& b, f32x4 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return mfma_f16(a, b, c);
}
template <bool BF>
__device__ __forceinline__ uint16_t to16(float v) {
  if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)v);
  else return f2h(v);
}
// (exp through the hardware exp2: 1 + exp(-v) is good to a few 2^-24; v below -88 gives v / inf = -0)
__device__ __forceinline__ float silu(float v) { return v / (1.f + __expf(-v)); }

// ---------------------------------------------------------------- slots in expert order

// Workgroup e lists the slots of expert e: a count of the slots of lower
// experts places its list, so no workgroup waits for another.  Each thread
// takes a contiguous run of slots, and a prefix sum over the threads keeps the
// list ascending.
__global__ __launch_bounds__(256) void experts_sort(ExpertsArgs a) {
  __shared__ int s_lt[4], s_eq[4];
  const int e = blockIdx.x, n = a.T * a.k, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int run = (n + 255) / 256, i0 = min(n, tid * run), i1 = min(n, i0 + run);
  int lt = 0, eq = 0;
  for (int i = i0; i < i1; ++i) {
    const int id = a.ids[i];
    lt += id >= 0 && id < e;
    eq += id == e;
    if (e == 0 && (unsigned)id >= (unsigned)a.w.E) a.pos[i] = -1;
  }
  int inc = eq;  // inclusive prefix within the wave
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(inc, o);
    if (lane >= o) inc += v;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) lt += __shfl_xor(lt, o);
  if (lane == 63) s_eq[wv] = inc;
  if (lane == 0) s_lt[wv] = lt;
  __syncthreads();
  const int base = s_lt[0] + s_lt[1] + s_lt[2] + s_lt[3];
  int p = base + inc - eq;
  for (int w = 0; w < wv; ++w) p += s_eq[w];
  for (int i = i0; i < i1; ++i)
    if (a.ids[i] == e) {
      a.perm[p] = i;
      a.pos[i] = p;
      ++p;
    }
  if (tid == 0) {
    a.off[e] = base;
    a.cnt[e] = s_eq[0] + s_eq[1] + s_eq[2] + s_eq[3];
  }
}

// ---------------------------------------------------------------- row tiles

// Row tile `tile` of BM rows over all experts' lists, found by every wave for
// itself: lane l sums the tiles of 8 experts.
struct RowTile {
  int e, row0, rows;  // expert, first place, rows (0: no such tile)
};
template <int BM>
__device__ __forceinline__ RowTile find_tile(const ExpertsArgs& a, int tile) {
  const int lane = threadIdx.x & 63;
  int nt[8], sum = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = lane * 8 + i;
    nt[i] = e < a.w.E ? (a.cnt[e] + BM - 1) / BM : 0;
    sum += nt[i];
  }
  int inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(inc, o);
    if (lane >= o) inc += v;
  }
  int before = inc - sum, e = -1, r = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (tile >= before && tile < before + nt[i]) {
      e = lane * 8 + i;
      r = tile - before;
    }
    before += nt[i];
  }
  const uint64_t hit = __builtin_amdgcn_ballot_w64(e >= 0);
  if (!hit) return {0, 0, 0};
  const int src = __builtin_ctzll(hit);
  e = __builtin_amdgcn_readlane(e, src);
  r = __builtin_amdgcn_readlane(r, src);
  return {e, a.off[e] + r * BM, min(BM, a.cnt[e] - r * BM)};
}

// ---------------------------------------------------------------- products

// 16 rows x 256 columns per workgroup, 64 columns per wave, operands straight
// from global memory.  GU: rows of x gathered through perm, silu(gate) * up
// out; else rows of that, the expert's output out.
template <bool GU, bool BF, bool HL>
__global__ __launch_bounds__(256) void experts_gemm(ExpertsArgs a) {
  const RowTile rt = find_tile<16>(a, blockIdx.x);
  if (rt.rows == 0) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int D = a.w.D, F = a.w.F;
  const int K = GU ? D : F, N = GU ? 2 * F : D, KT = K / 32;
  const int cb = blockIdx.y * 4 + wv;  // 64-column block
  if (cb * 64 >= N) return;
  const int p = rt.row0 + min(lane & 15, rt.rows - 1);
  const uint16_t *ah, *al = nullptr;
  if constexpr (GU) {
    const int t = a.perm[p] / a.k;
    if constexpr (HL) {
      ah = a.xhi + (size_t)t * D;
      al = a.xlo + (size_t)t * D;
    } else {
      ah = (const uint16_t*)a.x + t * a.x_stride;
    }
  } else {
    ah = a.hhi + (size_t)p * F;
    if constexpr (HL) al = a.hlo + (size_t)p * F;
  }
  const int kc = (lane >> 4) * 8;
  const u32x4* w = (const u32x4*)(GU ? a.w.gu : a.w.dn) + ((size_t)rt.e * (N / 64) + cb) * KT * 256 + lane;
  f32x4 acc[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) acc[s] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kt = 0; kt < KT; ++kt) {
    const u32x4 h = *(const u32x4*)(ah + kt * 32 + kc);
    u32x4 l = h;
    if constexpr (HL) l = *(const u32x4*)(al + kt * 32 + kc);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 b = w[(size_t)kt * 256 + s * 64];
      acc[s] = mfma16<BF>(h, b, acc[s]);
      if constexpr (HL) acc[s] = mfma16<BF>(l, b, acc[s]);
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int m = 4 * (lane >> 4) + r;
    if (m >= rt.rows) continue;
    const size_t row = rt.row0 + m;
    if constexpr (GU) {
#pragma unroll
      for (int s = 0; s < 4; s += 2) {
        const float v = silu(acc[s][r]) * acc[s + 1][r];
        const size_t at = row * F + cb * 32 + s * 8 + (lane & 15);
        if constexpr (HL) split_f16(v, a.hhi[at], a.hlo[at]);
        else a.hhi[at] = to16<BF>(v);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) a.y[row * D + cb * 64 + s * 16 + (lane & 15)] = acc[s][r];
    }
  }
}

// The activations' fp16 pair, 8 elements per thread.
__global__ __launch_bounds__(256) void experts_split(ExpertsArgs a) {
  const int D = a.w.D, per = D / 8;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.T * per) return;
  const int t = i / per, c = (i - t * per) * 8;
  const float4* p = (const float4*)((const float*)a.x + t * a.x_stride + c);
  const float4 u = p[0], q = p[1];
  const float v[8] = {u.x, u.y, u.z, u.w, q.x, q.y, q.z, q.w};
  uint4 hi, lo;
  split8(v, hi, lo);
  *(uint4*)(a.xhi + (size_t)t * D + c) = hi;
  *(uint4*)(a.xlo + (size_t)t * D + c) = lo;
}

// out[t] = sum_j w[t][j] y[pos[t][j]], 4 columns per thread.
__global__ __launch_bounds__(256) void experts_combine(ExpertsArgs a) {
  const int D = a.w.D, c = (blockIdx.y * 256 + threadIdx.x) * 4, t = blockIdx.x;
  if (c >= D) return;
  float4 v{0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < a.k; ++j) {
    const int p = a.pos[t * a.k + j];
    if (p < 0) continue;
    const float w = a.weights[t * a.k + j];
    const float4 y = *(const float4*)(a.y + (size_t)p * D + c);
    v.x += w * y.x;
    v.y += w * y.y;
    v.z += w * y.z;
    v.w += w * y.w;
  }
  const int64_t at = t * a.out_stride + c;
  if (a.x_type == ET_F32) {
    *(float4*)((float*)a.out + at) = v;
  } else {
    uint32_t o[2];
    if (a.x_type == ET_BF16) {
      o[0] = to16<true>(v.x) | (uint32_t)to16<true>(v.y) << 16;
      o[1] = to16<true>(v.z) | (uint32_t)to16<true>(v.w) << 16;
    } else {
      o[0] = pack_h2(v.x, v.y);
      o[1] = pack_h2(v.z, v.w);
    }
    *(uint2*)((uint16_t*)a.out + at) = uint2{o[0], o[1]};
  }
}

// ---------------------------------------------------------------- the call

size_t experts_carve(ExpertsArgs& a, void* base) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? (char*)base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  const size_t n = (size_t)a.T * a.k, D = a.w.D, F = a.w.F;
  const bool pair = a.x_type == ET_F32;
  a.perm = (int32_t*)take(n * 4);
  a.pos = (int32_t*)take(n * 4);
  a.cnt = (int32_t*)take((size_t)a.w.E * 4);
  a.off = (int32_t*)take((size_t)a.w.E * 4);
  a.hhi = (uint16_t*)take(n * F * 2);
  a.hlo = pair ? (uint16_t*)take(n * F * 2) : nullptr;
  a.xhi = pair ? (uint16_t*)take((size_t)a.T * D * 2) : nullptr;
  a.xlo = pair ? (uint16_t*)take((size_t)a.T * D * 2) : nullptr;
  a.y = (float*)take(n * D * 4);
  return off;
}

template <bool BF, bool HL>
static void launch_products(const ExpertsArgs& a, hipStream_t s) {
  const int n = a.T * a.k, tiles = n / 16 + std::min(n, a.w.E);  // at most: whole tiles, and a ragged one per expert
  hvd_launch((experts_gemm<true, BF, HL>), dim3(tiles, (2 * a.w.F / 64 + 3) / 4), dim3(256), 0, s, a);
  hvd_launch((experts_gemm<false, BF, HL>), dim3(tiles, (a.w.D / 64 + 3) / 4), dim3(256), 0, s, a);
}

hipError_t launch_experts(const ExpertsArgs& a, hipStream_t s) {
  hvd_launch(experts_sort, dim3(a.w.E), dim3(256), 0, s, a);
  if (a.x_type == ET_F32) {
    hvd_launch(experts_split, dim3((a.T * (a.w.D / 8) + 255) / 256), dim3(256), 0, s, a);
    launch_products<false, true>(a, s);
  } else if (a.w.wtype == ET_BF16) {
    launch_products<true, false>(a, s);
  } else {
    launch_products<false, false>(a, s);
  }
  hvd_launch(experts_combine, dim3(a.T, (a.w.D / 4 + 255) / 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hvd
