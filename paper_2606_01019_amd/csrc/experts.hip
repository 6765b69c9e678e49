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
//
// 32-bit values have a larger range than the pair, so each row of x, and of
// silu(gate) * up each row (of 32 columns in the few-row form), is scaled by
// the power of two that brings its largest magnitude to [2^14, 2^15): the pair
// keeps 22 bits of values down to 2^-17 of the largest, and 2^-39 of the
// largest below.  The scale is undone on 32-bit sums.  (silu * up is about
// quadratic in x: unscaled, x of size 1e-2 left 11 bits of it, 1e-4 none, and 100
// overflowed.)
#include "common.h"
#include "kernels.h"
#include "moe.h"

#include <type_traits>

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
// (exp through the hardware exp2: its relative error is a few 2^-24 and |v| 2^-24 more
// from the exponent's rounding, which counts where exp(-v) does, below 0; v below -88 gives v / inf = -0)
__device__ __forceinline__ float silu(float v) { return v / (1.f + __expf(-v)); }

// ---------------------------------------------------------------- scaled pairs

// The power of two of values up to m in magnitude, as a biased exponent b in
// [1, 240]: v * pow2_down(b) is below 2^15, pow2_up(b) undoes it.
__device__ __forceinline__ int scale_exp(float m) { return max((int)(__float_as_uint(m) >> 23) - 14, 1); }
__device__ __forceinline__ float pow2_up(int b) { return __uint_as_float((uint32_t)b << 23); }
__device__ __forceinline__ float pow2_down(int b) { return __uint_as_float((uint32_t)(254 - b) << 23); }
// Infinities and NaN do not count: they stay what they are under any scale.
__device__ __forceinline__ float max_finite(float m, float v) {
  const float a = fabsf(v);
  return a <= 3.402823466e38f ? fmaxf(m, a) : m;
}
// The max over the 16 lanes of a row, by data-parallel permutes.
__device__ __forceinline__ float row16_max(float v) {
  auto dpp = [](float x, auto ctrl) __attribute__((always_inline)) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
  };
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0xB1>{}));
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x4E>{}));
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x141>{}));
  return fmaxf(v, dpp(v, std::integral_constant<int, 0x140>{}));
}

// ---------------------------------------------------------------- slots in expert order

// Workgroup e lists the slots of expert e: a count of the slots of lower
// experts places its list, so no workgroup waits for another.  Each thread
// takes a contiguous run of slots, and a prefix sum over the threads keeps the
// list ascending.
typedef int32_t i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));  // (ids may lie at any 4-byte aligned address)
__global__ __launch_bounds__(256) void experts_sort(ExpertsArgs a) {
  __shared__ int s_lt[4], s_eq[4];
  const int e = blockIdx.x, n = a.T * a.k, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int run = ((n + 255) / 256 + 3) & ~3, i0 = min(n, tid * run), i1 = min(n, i0 + run);
  int lt = 0, eq = 0;
  auto scan = [&](auto&& f) __attribute__((always_inline)) {  // f(slot, id) over the run, four ids a load
    int i = i0;
#pragma unroll 4
    for (; i + 4 <= i1; i += 4) {
      const i32x4_a4 v = *(const i32x4_a4*)(a.ids + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) f(i + j, v[j]);
    }
    for (; i < i1; ++i) f(i, a.ids[i]);
  };
  scan([&](int i, int id) {
    lt += id >= 0 && id < e;
    eq += id == e;
    if (e == 0 && (unsigned)id >= (unsigned)a.w.E) a.pos[i] = -1;
  });
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
  if (eq)
    scan([&](int i, int id) {
      if (id == e) {
        a.perm[p] = i;
        a.pos[i] = p;
        ++p;
      }
    });
  if (e == 0) a.arrived[tid] = 0u;  // (before the products that count on it)
  if (tid == 0) {
    a.off[e] = base;
    a.cnt[e] = s_eq[0] + s_eq[1] + s_eq[2] + s_eq[3];
  }
}

// ---------------------------------------------------------------- row tiles

// The row tile and column block of a workgroup, found by every wave for itself
// from the experts' slot counts: lane l sums the tiles of 8 experts.  Tiles are
// numbered expert by expert, within one by column block, then row tile, and
// each XCD takes a run of them: an expert's row tiles of one column block are
// neighbours there and share its weights in that XCD's L2.
//
// SPLIT (one workgroup per CU): the tiles past the last whole round of CUs
// would leave most of them idle for as long as a tile takes; their K range is
// dealt to as many workgroups as fit one round, kMaxSplits at most.
constexpr int kTileCUs = 256, kMaxSplits = 4;
struct Tile {
  int e, row0, rows, cb;  // expert, first place, rows (0: no such tile), column block
  int kb, ke;             // K steps (kb even)
  int left, split, splits;  // tile shared by several workgroups: its number, this part, the parts
};
template <int BM, bool SPLIT>
__device__ __forceinline__ Tile find_tile(const ExpertsArgs& a, int CB, int KT) {
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
  const int total = __builtin_amdgcn_readlane(inc, 63) * CB;
  const int id = blockIdx.x;
  Tile t{0, 0, 0, 0, 0, KT, -1, 0, 1};
  const int rest = SPLIT ? total % kTileCUs : 0, whole = total - rest;
  const int splits = rest ? min(min(kTileCUs / rest, kMaxSplits), max(1, KT / 16)) : 1;
  const int run = splits > 1 ? whole : total;  // tiles in one piece
  int at;
  if (id < run) {
    // XCD x (= id % 8 under the round-robin dispatch) takes the x-th run of positions
    const int x = id & 7, q = run >> 3;
    at = x * q + min(x, run & 7) + (id >> 3);
  } else {
    const int u = id - run;
    if (u >= (total - run) * splits) return t;
    t.left = __builtin_amdgcn_readfirstlane(u / splits);
    t.split = u - t.left * splits;
    t.splits = splits;
    t.kb = __builtin_amdgcn_readfirstlane(t.split * KT / splits) & ~1;
    t.ke = t.split + 1 == splits ? KT : __builtin_amdgcn_readfirstlane((t.split + 1) * KT / splits) & ~1;
    at = run + t.left;
  }
  int before = (inc - sum) * CB, e = -1, r = 0, nte = 1;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (at >= before && at < before + nt[i] * CB) {
      e = lane * 8 + i;
      r = at - before;
      nte = nt[i];
    }
    before += nt[i] * CB;
  }
  const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(e >= 0));
  e = __builtin_amdgcn_readlane(e, src);
  r = __builtin_amdgcn_readlane(r, src);
  nte = __builtin_amdgcn_readlane(nte, src);
  const int cb = r / nte, tile = r - cb * nte;
  t.e = e;
  t.row0 = a.off[e] + tile * BM;
  t.rows = min(BM, a.cnt[e] - tile * BM);
  t.cb = cb;
  return t;
}

// ---------------------------------------------------------------- products, many rows

// The grouped product on MFMA 32x32x16: a workgroup of WY x WX waves owns
// BM = 32 WM WY places of one expert's list and BN = 32 WN WX columns.  The
// operands are copied straight into rings of LDS slots (global_load_lds) well
// ahead of the MFMAs: weights, 1 KB fragments of 16 columns, in 32-wide K steps;
// rows in slabs of 64, every second step.  The rows are gathered there from
// wherever they are, so no gathered copy of x exists; a copy instruction takes
// 8 rows of 128 bytes, whole cache lines (16 rows of 64 bytes come from L2 at 37
// bytes per ns and CU, lines at 126), and the 16-byte pieces of a line are
// permuted by the row's low bits so that reading 32 rows of one piece spreads
// over the LDS banks.  Weights fresh from memory come at 28 bytes per ns and CU,
// the whole chip's 7.3 TB/s: what bounds these products until an expert has
// hundreds of rows.
// Places past the list repeat its last one and are not stored; a tile belongs
// to one expert.
// GU: rows of x, silu(gate) * up out (OP: as a pair); else rows of that
// product, the expert's output out.  AP: the row operand is a pair; GU's is then
// scaled (xs), and its product goes out in 32 bits, to be scaled by whole rows.
template <int WY_, int WX_, int WM_, int WN_>
struct TileShape {
  static constexpr int WY = WY_, WX = WX_, WM = WM_, WN = WN_, NW = WY * WX;
  static constexpr int BM = 32 * WM * WY, BN = 32 * WN * WX;
  static constexpr int LDS = NW == 8 ? 160 * 1024 : 80 * 1024;  // one or two workgroups per CU
  static constexpr bool SPLIT = NW == 8;                          // tiles past the last whole round are shared
};

using T64 = TileShape<1, 4, 2, 2>;   // 64 x 256, 4 waves: two workgroups per CU
using T128 = TileShape<2, 4, 2, 2>;  // 128 x 256, 8 waves: one workgroup per CU

typedef float f32x16 __attribute__((ext_vector_type(16)));
template <bool BF>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, const u32x4& b, f32x16 c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Eight values as 16-bit elements, and what they leave over (the pair's lo part).
template <bool BF>
__device__ __forceinline__ void to16x8(const float (&v)[8], uint4& hi) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = to16<BF>(v[2 * i]) | (uint32_t)to16<BF>(v[2 * i + 1]) << 16;
  hi = uint4{h[0], h[1], h[2], h[3]};
}
template <bool BF>
__device__ __forceinline__ float from16(uint16_t b) {
  if constexpr (BF) return bf2f(b);
  else return h2f(b);
}
// What hi leaves over of v: nothing of an infinity, which would make NaN of it.
template <bool BF>
__device__ __forceinline__ uint16_t lo16(float v, uint16_t hi) {
  const float h = from16<BF>(hi);
  return to16<BF>(fabsf(h) == INFINITY ? 0.f : v - h);
}
template <bool BF>
__device__ __forceinline__ void pair8(const float (&v)[8], uint4& hi, uint4& lo) {
  to16x8<BF>(v, hi);
  const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w};
  uint32_t l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    l[i] = lo16<BF>(v[2 * i], (uint16_t)(h[i] & 0xFFFFu)) | (uint32_t)lo16<BF>(v[2 * i + 1], (uint16_t)(h[i] >> 16)) << 16;
  lo = uint4{l[0], l[1], l[2], l[3]};
}

// f(constant of value i), i clamped to [0, N)
template <int N, class F>
__device__ __forceinline__ void with_constant(int i, F&& f) {
  if constexpr (N == 1) {
    f(std::integral_constant<int, 0>{});
  } else {
    if (i >= N - 1) f(std::integral_constant<int, N - 1>{});
    else with_constant<N - 1>(i, f);
  }
}

constexpr int kRegionStride = 72;  // floats per row of a wave's epilogue region: rows 4 apart land 32 banks apart
constexpr int kRegionBytes = 32 * kRegionStride * 4;

// Copies that may still be in flight when iteration i waits (before its own):
// every iteration t copies a K step of weights (SW - 1 steps ahead, cw copies),
// an even one a slab before it (PA slabs ahead, ca copies).  The wait covers
// the weights of step i + 1 and, where i is odd, the slab of step i + 1.
constexpr int in_flight(bool odd, int SW, int PA, int cw, int ca) {
  auto issued = [&](int t) { return cw + ((odd ? t + 1 : t) % 2 == 0 ? ca : 0); };  // at iteration i + t
  int w = 0;
  for (int t = 3 - SW; t <= -1; ++t) w += issued(t);
  if (!odd) return w;
  int a = cw;  // the weights of the slab's own iteration follow it
  for (int t = 2 - 2 * PA; t <= -1; ++t) a += issued(t);
  return a < w ? a : w;
}

template <class S, bool GU, bool BF, bool AP, bool OP>
__global__ __launch_bounds__(64 * S::NW, 2) void experts_tiled(ExpertsArgs a, int CB) {
  constexpr int NW = S::NW, WM = S::WM, WN = S::WN, BM = S::BM, BN = S::BN;
  constexpr int NP = AP ? 2 : 1;                           // parts of the row operand
  constexpr int WF = BN / 16, WPW = WF / NW;               // weight fragments of a step; per wave
  constexpr int RPW = BM / 8 / NW;                         // row copies (8 rows) per wave, part and slab
  constexpr int SLAB = NP * BM * 128, STEP = WF * 1024;    // bytes
  constexpr int PA = 3 * SLAB + 4 * STEP <= S::LDS ? 2 : 1, SA = PA + 1;  // slabs ahead; slots
  constexpr int SW0 = (S::LDS - SA * SLAB) / STEP, SW = SW0 > 6 ? 6 : SW0;
  static_assert(WF % NW == 0 && BM % (8 * NW) == 0 && SW >= 3, "every wave copies alike");
  __shared__ u32x4 sbuf[(SA * SLAB + SW * STEP) / 16];
  static_assert(NW * kRegionBytes + 16 <= (int)sizeof(sbuf), "the epilogue's regions and a word fit the rings");
  u32x4* const sw = sbuf + SA * SLAB / 16;

  constexpr bool SPLIT = GU && S::SPLIT;  // (the down product's K range is too short)
  const int D = a.w.D, F = a.w.F;
  const int K = GU ? D : F, N = GU ? 2 * F : D, KT = K / 32;
  const Tile tl = find_tile<BM, SPLIT>(a, CB, KT);
  if (tl.rows == 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wy = wave / S::WX, wx = wave % S::WX;

  const char *asrc[NP][RPW], *wsrc[WPW];
#pragma unroll
  for (int q = 0; q < RPW; ++q) {
    const int p = tl.row0 + min((q * NW + wave) * 8 + (lane >> 3), tl.rows - 1);
    const int piece = ((lane & 7) ^ (lane >> 3)) * 8;
    const int t = GU ? a.perm[p] / a.k : 0;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const uint16_t* row;
      if constexpr (GU && AP) row = (n ? a.xlo : a.xhi) + (size_t)t * D;
      else if constexpr (GU) row = (const uint16_t*)a.x + t * a.x_stride;
      else row = (n ? a.hlo : a.hhi) + (size_t)p * F;
      asrc[n][q] = (const char*)(row + piece);
    }
  }
#pragma unroll
  for (int q = 0; q < WPW; ++q) {
    const int st = min(tl.cb * WF + q * NW + wave, N / 16 - 1);  // strips past the matrix: any valid one
    wsrc[q] = (const char*)((GU ? a.w.gu : a.w.dn) + (((size_t)tl.e * (N / 64) + (st >> 2)) * KT * 4 + (st & 3)) * 512 + lane * 8);
  }

  f32x16 acc[WM][WN];
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int j = 0; j < WN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // 32 columns of one 16-wide K sub-step s: lane l takes column l%32, K 16s + 8(l/32)..+8
  const int fl = (lane & 15) + 16 * (lane >> 5), fo = (lane >> 4) & 1;
  const int live = (tl.rows - wy * 32 * WM + 31) / 32;  // row blocks of this wave that hold rows
  // Iteration i multiplies the first half of step i while its second half is
  // read; then it waits until step i+1 has landed, refills the slots of step
  // i-1 (and slab i/2-1), and multiplies the second half while the first half of
  // step i+1 is read.  L of the wave's WM row blocks hold rows of the list: the
  // others are neither read nor multiplied (a wave without any only copies).
  // Likewise the wave makes G of its RPW row copies.
  auto k_loop = [&](auto blocks, auto copies) __attribute__((always_inline)) {
    constexpr int L = decltype(blocks)::value, G = decltype(copies)::value, CA = NP * G;
    const int m0 = tl.kb / 2, m1 = (tl.ke - 1) / 2;
    // (steps and slabs past the range re-copy the last one: the counts stay constant)
    auto issue_w = [&](int slot, int kt) __attribute__((always_inline)) {
      kt = min(kt, tl.ke - 1);
#pragma unroll
      for (int q = 0; q < WPW; ++q)
        __builtin_amdgcn_global_load_lds((const void*)(wsrc[q] + (size_t)kt * 4096),
                                         (lds_void*)(sw + (slot * WF + q * NW + wave) * 64), 16, 0, 0);
    };
    auto issue_a = [&](int slot, int m) __attribute__((always_inline)) {
      m = min(m, m1);
#pragma unroll
      for (int n = 0; n < NP; ++n)
#pragma unroll
        for (int q = 0; q < G; ++q)
          __builtin_amdgcn_global_load_lds((const void*)(asrc[n][q] + (size_t)m * 128),
                                           (lds_void*)(sbuf + (slot * SLAB + n * BM * 128 + (q * NW + wave) * 1024) / 16), 16, 0, 0);
    };
    struct Ops {
      u32x4 ah[L ? L : 1], al[AP && L ? L : 1], bw[WN];
    };
    // sub-step s (0..3) of slab slot as_, of which weight slot ws holds s % 2
    auto read_ops = [&](int as_, int ws, int s, Ops& o) __attribute__((always_inline)) {
      if constexpr (L > 0) {
        const int piece = (s * 2 + (lane >> 5)) ^ (lane & 7);
        const u32x4* ap = sbuf + as_ * (SLAB / 16) + (wy * WM * 32 + (lane & 31)) * 8 + piece;
#pragma unroll
        for (int i = 0; i < L; ++i) {
          o.ah[i] = ap[i * 256];
          if constexpr (AP) o.al[i] = ap[BM * 8 + i * 256];
        }
        const u32x4* wp = sw + (ws * WF + wx * 2 * WN + fo) * 64 + fl + 32 * (s & 1);
#pragma unroll
        for (int j = 0; j < WN; ++j) o.bw[j] = wp[j * 128];
      }
    };
    auto mfma_ops = [&](const Ops& o, auto&& between) __attribute__((always_inline)) {
      if constexpr (L > 0) acc[0][0] = mfma32<BF>(o.ah[0], o.bw[0], acc[0][0]);
      __builtin_amdgcn_sched_barrier(0);
      between();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) {
          if (i != 0 || j != 0) acc[i][j] = mfma32<BF>(o.ah[i], o.bw[j], acc[i][j]);
          if constexpr (AP) acc[i][j] = mfma32<BF>(o.al[i], o.bw[j], acc[i][j]);
        }
      __builtin_amdgcn_sched_barrier(0);
    };
    Ops o0, o1;
    // what iterations before the first would have copied, in their order
    constexpr int T0 = 2 * PA > SW - 1 ? 2 * PA : SW - 1;
#pragma unroll
    for (int t = -T0; t < 0; ++t) {
      if (t % 2 == 0 && t / 2 + PA >= 0) issue_a(t / 2 + PA, m0 + t / 2 + PA);
      if (t + SW - 1 >= 0) issue_w(t + SW - 1, tl.kb + t + SW - 1);
    }
    vm_wait<in_flight(true, SW, PA, WPW, CA)>();
    block_barrier();
    read_ops(0, 0, 0, o0);
    int ws = 0, as_ = 0;  // slots of step i and of its slab
    auto iteration = [&](auto parity, int i) __attribute__((always_inline)) {
      constexpr int ODD = decltype(parity)::value;
      const int wn = ws + 1 == SW ? 0 : ws + 1, wprev = ws == 0 ? SW - 1 : ws - 1;
      const int an = ODD ? (as_ + 1 == SA ? 0 : as_ + 1) : as_, aprev = as_ == 0 ? SA - 1 : as_ - 1;
      mfma_ops(o0, [&]() { read_ops(as_, ws, 2 * ODD + 1, o1); });
      vm_wait<in_flight(ODD, SW, PA, WPW, CA)>();
      block_barrier();
      if constexpr (!ODD) issue_a(aprev, i / 2 + PA);
      issue_w(wprev, i + SW - 1);
      mfma_ops(o1, [&]() { read_ops(an, wn, ODD ? 0 : 2, o0); });
      ws = wn;
      as_ = an;
    };
    int i = tl.kb;  // (even)
    for (; i + 2 <= tl.ke; i += 2) {
      iteration(std::integral_constant<int, 0>{}, i);
      iteration(std::integral_constant<int, 1>{}, i + 1);
    }
    if (i < tl.ke) iteration(std::integral_constant<int, 0>{}, i);
  };
  auto with_blocks = [&](auto copies) __attribute__((always_inline)) {
    with_constant<WM + 1>(live, [&](auto blocks) __attribute__((always_inline)) { k_loop(blocks, copies); });
  };
  if (RPW > 1 && tl.rows <= BM / 2) with_blocks(std::integral_constant<int, RPW / 2>{});
  else with_blocks(std::integral_constant<int, RPW>{});
  float row_up[WM][2];  // what undoes the scale of the rows this lane stores
  if constexpr (GU && AP)
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int it = 0; it < 2; ++it)
        row_up[i][it] = a.xs[a.perm[tl.row0 + min(wy * 32 * WM + 32 * i + (lane >> 2) + 16 * it, tl.rows - 1)] / a.k];
  vm_wait<0>();  // no copy may land after the ring is reused or released
  __syncthreads();

  if constexpr (SPLIT) {
    if (tl.splits > 1) {
      // A shared tile: each part goes out in lane-native order with device-scope
      // stores and is counted; the last to arrive sums the parts in K order
      // (the same order whoever is last) and goes on as if it had them all.
      constexpr int WAVE_BYTES = WM * WN * 64 * 64;  // 16 floats per lane and 32 x 32 block
      const uint32_t mine = ((uint32_t)(tl.left * tl.splits) * NW + wave) * WAVE_BYTES + lane * 16;
#pragma unroll
      for (int i = 0; i < WM; ++i)
        if (i < live)
#pragma unroll
          for (int j = 0; j < WN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
              st_f4_dev(a.part, mine + (uint32_t)tl.split * NW * WAVE_BYTES + ((i * WN + j) * 4 + g) * 1024,
                        float4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]});
      vm_wait<0>();  // this wave's stores are done
      // (in the ring: a second LDS variable makes the compiler wait for every
      // copy in flight before each LDS read of the K loop)
      int& last_part = *(int*)&sbuf[sizeof(sbuf) / 16 - 1];
      __syncthreads();
      if (threadIdx.x == 0) last_part = atomicAdd(a.arrived + tl.left, 1u) == (uint32_t)tl.splits - 1u;
      __syncthreads();
      if (!last_part) return;  // (the epilogue's regions lie below it)
#pragma unroll
      for (int i = 0; i < WM; ++i)
        if (i < live)
#pragma unroll
          for (int j = 0; j < WN; ++j) {
            float4 v[kMaxSplits][4];  // all parts of the block on their way at once
#pragma unroll
            for (int q = 0; q < kMaxSplits; ++q)
#pragma unroll
              for (int g = 0; g < 4; ++g)
                v[q][g] = ld_f4_dev(a.part, mine + (uint32_t)(q < tl.splits ? q : 0) * NW * WAVE_BYTES + ((i * WN + j) * 4 + g) * 1024);
#pragma unroll
            for (int q = 0; q < kMaxSplits; ++q)
              if (q < tl.splits) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                  const float o[4] = {v[q][g].x, v[q][g].y, v[q][g].z, v[q][g].w};
#pragma unroll
                  for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = q ? acc[i][j][4 * g + e] + o[e] : o[e];
                }
              }
          }
    }
  }

  // Blocks of 32 rows x 64 columns through the wave's LDS region, so that the
  // stores are 16 bytes of one row per lane (MFMA 32x32: element r of lane l is
  // row 8 (r/4) + 4 (l/32) + r%4, column l%32).
  float* lds = (float*)sbuf + wave * (kRegionBytes / 4);
#pragma unroll
  for (int i = 0; i < WM; ++i) {
#pragma unroll
    for (int j = 0; j < WN; j += 2) {
      const int col0 = tl.cb * BN + wx * 32 * WN + 32 * j, row0 = wy * 32 * WM + 32 * i;
      if (col0 >= N || row0 >= tl.rows) continue;  // (wave-uniform)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float* p = lds + (8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * kRegionStride + (lane & 31);
        p[0] = acc[i][j][r];
        p[32] = acc[i][j + 1][r];
      }
      __builtin_amdgcn_wave_barrier();  // (one wave's LDS accesses execute in order)
      auto oct = [&](int row, int c, float (&v)[8]) __attribute__((always_inline)) {
        const float4 x = *(const float4*)(lds + row * kRegionStride + c), y = *(const float4*)(lds + row * kRegionStride + c + 4);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
      };
      if constexpr (GU) {
        // a 32-column tile is one (gate strip, up strip) pair
        const int o = lane & 3, c = 32 * (o >> 1) + 8 * (o & 1);
#pragma unroll
        for (int it = 0; it < 2; ++it) {
          const int row = (lane >> 2) + 16 * it;
          float g[8], u[8];
          oct(row, c, g);
          oct(row, c + 16, u);
          if constexpr (AP)
#pragma unroll
            for (int n = 0; n < 8; ++n) {
              g[n] *= row_up[i][it];
              u[n] *= row_up[i][it];
            }
#pragma unroll
          for (int n = 0; n < 8; ++n) g[n] = silu(g[n]) * u[n];
          if (row0 + row < tl.rows) {
            const size_t at = (size_t)(tl.row0 + row0 + row) * F + (col0 >> 1) + o * 8;
            if constexpr (AP) {
              *(float4*)(a.y + at) = float4{g[0], g[1], g[2], g[3]};
              *(float4*)(a.y + at + 4) = float4{g[4], g[5], g[6], g[7]};
            } else {
              uint4 hi, lo;
              if constexpr (OP) {
                pair8<BF>(g, hi, lo);
                *(uint4*)(a.hlo + at) = lo;
              } else {
                to16x8<BF>(g, hi);
              }
              *(uint4*)(a.hhi + at) = hi;
            }
          }
        }
      } else {
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          const int row = (lane >> 3) + 8 * it;
          if (row0 + row < tl.rows) {
            const float* p = lds + row * kRegionStride + (lane & 7) * 8;
            float* y = a.y + (size_t)(tl.row0 + row0 + row) * D + col0 + (lane & 7) * 8;
            *(float4*)y = *(const float4*)p;
            *(float4*)(y + 4) = *(const float4*)(p + 4);
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// ---------------------------------------------------------------- products, few rows

// Up to 16 MT rows: every product streams the chosen experts' weights once,
// straight into registers, and all rows ride along (the MFMA work of rows that
// did not choose an expert is free while the launch waits for weights).  The
// workgroups find the distinct experts of the call themselves, in ascending
// order, so nothing runs before them: two launches in all.
constexpr int kFewSlots = 256;   // slots (T * k) of the few-row form
constexpr int kFewWaves = 8;

// The distinct experts among n slots, ascending.
struct Distinct {
  uint32_t bits[kMaxExperts / 32];
  int count;
  int16_t list[kFewSlots];
};
// This thread's slot's expert (-1: none); the list is ready after a barrier.
__device__ __forceinline__ int find_distinct(const ExpertsArgs& a, int n, Distinct& d) {
  const int tid = threadIdx.x;
  int mine = tid < n ? a.ids[tid] : -1;
  if ((unsigned)mine >= (unsigned)a.w.E) mine = -1;
  if (tid < kMaxExperts / 32) d.bits[tid] = 0u;
  __syncthreads();
  if (mine >= 0) atomicOr(&d.bits[mine >> 5], 1u << (mine & 31));
  __syncthreads();
  // thread e (one per possible expert): its rank among the chosen
  int below = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kMaxExperts / 32; ++w) {
    const uint32_t b = d.bits[w];
    below += w < (tid >> 5) ? __popc(b) : w == (tid >> 5) ? __popc(b & ((1u << (tid & 31)) - 1u)) : 0;
    all += __popc(b);
  }
  if (d.bits[tid >> 5] >> (tid & 31) & 1u) d.list[below] = (int16_t)tid;
  if (tid == 0) d.count = all;
  return mine;
}

// The same for a single row, by every wave for itself and without LDS or a
// barrier: lane d holds the d-th slot's expert and weight in ascending order of
// experts; an id that comes twice stays two entries.  8 of 64 experts of
// 4096 x 1024: gate/up 22.9 -> 22.7 us, down 15.5 -> 14.1.
struct RowChoice {
  int id;
  float w;
  int count;  // valid slots, wave-uniform
  __device__ __forceinline__ RowChoice() : id(-1), w(0.f), count(0) {}
  __device__ __forceinline__ explicit RowChoice(const ExpertsArgs& a) {
    const int lane = threadIdx.x & 63;
    const int e = lane < a.k ? a.ids[lane] : -1;
    const float ew = lane < a.k ? a.weights[lane] : 0.f;
    const bool ok = (unsigned)e < (unsigned)a.w.E;
    const int key = ok ? e : 0x7fffffff;
    int rank = 0;
    for (int i = 0; i < a.k; ++i) {
      const int o = __builtin_amdgcn_readlane(key, i);
      rank += o < key || (o == key && i < lane) ? 1 : 0;
    }
    if (lane >= a.k) rank = lane;
    id = __builtin_amdgcn_ds_permute(rank * 4, e);
    w = __int_as_float(__builtin_amdgcn_ds_permute(rank * 4, __float_as_int(ew)));
    count = __popcll(__builtin_amdgcn_ballot_w64(ok));
  }
  __device__ __forceinline__ int expert(int d) const { return __builtin_amdgcn_readlane(id, d); }
  __device__ __forceinline__ float weight(int d) const { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), d)); }
};

// Gate/up: workgroup (column block, y) streams NS strips of the y-th distinct
// expert; its 8 waves deal the K steps among themselves, so that the workgroup
// reads one contiguous window, and sum in LDS.  h of expert y, row t goes to
// row y * 16 MT + t, as a pair.
// XF: x is 32-bit and multiplied as the scaled pair.  A launch before this one
// makes it, except for ONE, a single row: a workgroup reads that once ahead for its
// scale, while the first weights are on their way.  (With more rows x is up to half
// as many bytes as the weights to a workgroup: all of them reading 9 rows ahead, top 8 of 64
// experts of 4096 x 1024, took this kernel from 94 to 113 us.)  The 32 columns of h
// that a workgroup makes are one K step of the down product; their scale goes to hx
// by (expert, step, row).
template <int MT, int NS, bool BF, bool XF, bool ONE>
__global__ __launch_bounds__(64 * kFewWaves, MT == 1 ? 4 : 2) void experts_gu_few(ExpertsArgs a) {
  constexpr int U = XF ? 3 : 4;  // K steps in flight
  constexpr int XQ = XF ? 2 : 1;  // 16-byte loads per lane and row tile
  __shared__ float red[kFewWaves][MT][NS][256];
  int e;
  if constexpr (ONE) {
    const RowChoice rc(a);
    if ((int)blockIdx.y >= rc.count) return;
    e = rc.expert(blockIdx.y);
  } else {
    __shared__ Distinct ds;
    find_distinct(a, a.T * a.k, ds);
    __syncthreads();
    if ((int)blockIdx.y >= ds.count) return;
    e = ds.list[blockIdx.y];
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int D = a.w.D, F = a.w.F, KT = D / 32;
  const int nsteps = wave < KT ? (KT - wave + kFewWaves - 1) / kFewWaves : 0;
  const u32x4* wp[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int st = blockIdx.x * NS + s;
    wp[s] = (const u32x4*)a.w.gu + ((size_t)e * (2 * F / 64) + (st >> 2)) * KT * 256 + (st & 3) * 64 + lane;
  }
  const char* xp[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int t = min(m * 16 + (lane & 15), a.T - 1);
    if constexpr (XF && !ONE) xp[m] = (const char*)(a.xhi + (size_t)t * D * 2 + (lane >> 4) * 8);
    else xp[m] = (const char*)a.x + (t * a.x_stride + (lane >> 4) * 8) * (XF ? 4 : 2);
  }
  constexpr int xq = XF && !ONE ? 64 : 16;  // from a lane's first 16 bytes of a step to its second
  f32x4 acc[MT][NS];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int s = 0; s < NS; ++s) acc[m][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  float x_down = 1.f, x_up[MT];  // a single row's scale; what undoes the scales of the rows this thread finishes
  if constexpr (XF && !ONE)
#pragma unroll
    for (int m = 0; m < MT; ++m) x_up[m] = a.xs[min(m * 16 + (int)(threadIdx.x >> 4 & 15), a.T - 1)];
  u32x4 qw[U][NS], qx[U][MT][XQ];
  auto load_w = [&](int u, int j) __attribute__((always_inline)) {
    const int kt = wave + j * kFewWaves;
#pragma unroll
    for (int s = 0; s < NS; ++s) qw[u][s] = __builtin_nontemporal_load(wp[s] + (size_t)kt * 256);
  };
  auto load_x = [&](int u, int j) __attribute__((always_inline)) {
    const int kt = wave + j * kFewWaves;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < XQ; ++q) qx[u][m][q] = *(const u32x4*)(xp[m] + (size_t)kt * (XF ? 128 : 64) + q * xq);
  };
  auto load = [&](int u, int j) __attribute__((always_inline)) {
    load_w(u, j);
    load_x(u, j);
  };
  auto consume = [&](int u) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if constexpr (XF) {
        u32x4 h, l;
        if constexpr (ONE) {
          // (scaling the next steps' values early would hold them twice, and spill)
          __builtin_amdgcn_sched_barrier(0);
          float v[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = __uint_as_float(qx[u][m][0][i]) * x_down;
            v[4 + i] = __uint_as_float(qx[u][m][1][i]) * x_down;
          }
          uint4 hi, lo;
          pair8<false>(v, hi, lo);
          h = u32x4{hi.x, hi.y, hi.z, hi.w};
          l = u32x4{lo.x, lo.y, lo.z, lo.w};
        } else {
          h = qx[u][m][0];
          l = qx[u][m][1];
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          acc[m][s] = mfma16<BF>(h, qw[u][s], acc[m][s]);
          acc[m][s] = mfma16<BF>(l, qw[u][s], acc[m][s]);
        }
      } else {
#pragma unroll
        for (int s = 0; s < NS; ++s) acc[m][s] = mfma16<BF>(qx[u][m][0], qw[u][s], acc[m][s]);
      }
    }
  };
  if constexpr (XF && ONE) {
    if (nsteps >= U)
#pragma unroll
      for (int u = 0; u < U; ++u) load_w(u, u);
    __builtin_amdgcn_sched_barrier(0);
    __shared__ float s_max[kFewWaves];
    const float* p = (const float*)a.x;
    float mx = 0.f;
    for (int c = threadIdx.x * 4; c < D; c += 64 * kFewWaves * 4) {
      const f32x4 v = *(const f32x4*)(p + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = max_finite(mx, v[i]);
    }
    mx = rows_max(row16_max(mx));
    if (lane == 0) s_max[wave] = mx;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) mx = fmaxf(mx, s_max[w]);
    const int b = scale_exp(mx);
    x_down = pow2_down(b);
    x_up[0] = pow2_up(b);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (nsteps >= U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (!(XF && ONE)) load_w(u, u);
      load_x(u, u);
    }
    int j = 0;
    for (; j + 2 * U <= nsteps; j += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        consume(u);
        load(u, j + u + U);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      consume(u);
      if (j + u + U < nsteps) load(u, j + u + U);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j + u + U < nsteps) consume(u);
  } else {
    for (int j = 0; j < nsteps; ++j) {
      load(0, j);
      consume(0);
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int s = 0; s < NS; ++s) *(f32x4*)&red[wave][m][s][lane * 4] = acc[m][s];
  __syncthreads();
  // element (row, col) of a 16 x 16 tile is at [16 (row/4) + col] * 4 + row%4
  if constexpr (XF) {
    // 16 lanes per row and (gate strip, up strip) pair; the row's scale is both pairs'
    static_assert(NS == 4, "a workgroup makes one K step of the down product");
    __shared__ float s_top[MT][2][16];
    const int c = threadIdx.x & 15, row = threadIdx.x >> 4 & 15, sp = threadIdx.x >> 8;
    const int at = ((row >> 2) * 16 + c) * 4 + (row & 3);
    float v[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float g = 0.f, u = 0.f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        g += red[w][m][2 * sp][at];
        u += red[w][m][2 * sp + 1][at];
      }
      v[m] = silu(g * x_up[m]) * (u * x_up[m]);
      const float top = row16_max(max_finite(0.f, v[m]));
      if (c == 0) s_top[m][sp][row] = top;
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int t = m * 16 + row, b = scale_exp(fmaxf(s_top[m][0][row], s_top[m][1][row]));
      if (t < a.T) {
        const float h = v[m] * pow2_down(b);
        const uint16_t hi = f2h(h);
        const size_t o = ((size_t)blockIdx.y * (16 * MT) + t) * F + (blockIdx.x * 2 + sp) * 16 + c;
        a.hhi[o] = hi;
        a.hlo[o] = lo16<false>(h, hi);
        if (c == 0 && sp == 0) a.hx[((size_t)blockIdx.y * gridDim.x + blockIdx.x) * (16 * MT) + t] = (uint8_t)b;
      }
    }
    return;
  }
  for (int i = threadIdx.x; i < MT * (NS / 2) * 256; i += 64 * kFewWaves) {
    const int c = i & 15, row = i >> 4 & 15, sp = (i >> 8) % (NS / 2), m = (i >> 8) / (NS / 2);
    const int at = ((row >> 2) * 16 + c) * 4 + (row & 3);
    float g = 0.f, u = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      g += red[w][m][2 * sp][at];
      u += red[w][m][2 * sp + 1][at];
    }
    const int t = m * 16 + row;
    if (t < a.T) {
      const float v = silu(g) * u;
      const uint16_t hi = to16<BF>(v);
      const size_t o = ((size_t)blockIdx.y * (16 * MT) + t) * F + (blockIdx.x * (NS / 2) + sp) * 16 + c;
      a.hhi[o] = hi;
      a.hlo[o] = lo16<BF>(v, hi);
    }
  }
}

// Down: a workgroup owns NS strips of d_model and runs over all distinct
// experts, the K steps of each dealt to its 8 waves; after an expert, each
// row's products are weighted and added to its total (rows that did not choose
// the expert add nothing, whatever is in them).  So the workgroups all stream
// alike, however the rows chose, the sums over k need no further pass, and a
// row's result does not depend on the other rows of the call (alone, a row that
// has an id twice adds the two products, not the weights: a rounding apart).
// XF: h is scaled by (row, K step): each step's products are scaled back into the
// expert's sum.
template <int MT, int NS, bool BF, bool XF, bool ONE>
__global__ __launch_bounds__(64 * kFewWaves, 2) void experts_down_few(ExpertsArgs a) {
  constexpr int U = MT == 1 ? 8 : 4;
  __shared__ Distinct ds;
  __shared__ float wmap[kFewSlots][16 * MT];  // weight of (expert, row)
  __shared__ uint32_t vmask[kFewSlots];       // rows that chose the expert
  __shared__ int16_t s_rank[kFewSlots];       // place of each slot's expert among the distinct ones
  __shared__ float s_w[kFewSlots];
  __shared__ float red[kFewWaves][MT][NS][256];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int T = a.T, k = a.k, D = a.w.D, F = a.w.F, KT = F / 32;
  const RowChoice rc = [&] {
    if constexpr (ONE) return RowChoice(a);
    else return RowChoice();
  }();
  int nd;
  if constexpr (ONE) {
    nd = rc.count;
  } else {
    // each slot's weight comes in with its id; one thread per row then adds a
    // row's up, in order, while the first weights are on their way
    const float my_w = tid < T * k ? a.weights[tid] : 0.f;
    if (tid < kFewSlots) {
      vmask[tid] = 0u;
#pragma unroll
      for (int r = 0; r < 16 * MT; r += 4) *(float4*)&wmap[tid][r] = float4{0.f, 0.f, 0.f, 0.f};
    }
    const int mine = find_distinct(a, T * k, ds);
    if (tid < T * k) {
      int r = -1;
      if (mine >= 0) {
        r = __popc(ds.bits[mine >> 5] & ((1u << (mine & 31)) - 1u));
        for (int w = 0; w < (mine >> 5); ++w) r += __popc(ds.bits[w]);
        atomicOr(&vmask[r], 1u << (tid / k));
      }
      s_rank[tid] = (int16_t)r;
      s_w[tid] = my_w;
    }
    __syncthreads();
    nd = ds.count;
  }
  auto weigh = [&]() __attribute__((always_inline)) {
    if constexpr (ONE) return;
    if (tid < T)
      for (int j = 0; j < k; ++j) {
        const int r = s_rank[tid * k + j];
        if (r >= 0) wmap[r][tid] += s_w[tid * k + j];
      }
    __syncthreads();
  };

  f32x4 tot[MT][NS], acc[MT][NS];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int s = 0; s < NS; ++s) tot[m][s] = acc[m][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int spw = wave < KT ? (KT - wave + kFewWaves - 1) / kFewWaves : 0;  // steps per expert
  const int total = spw * nd;
  if (total > 0) {
    u32x4 qw[U][NS], qh[U][MT], ql[U][MT];
    uint32_t qe[U][MT];  // XF: the scales of this lane's four output rows, a byte each
    // the loader's place: expert ld, step li of it
    int ld = 0, li = 0;
    const u32x4* wp;
    uint32_t hoff[MT];  // halves; rows that did not choose the expert read its first row that did
    const uint8_t* xe;
    auto enter = [&]() __attribute__((always_inline)) {
      const int e = ONE ? rc.expert(ld) : __builtin_amdgcn_readfirstlane(ds.list[ld]);
      const uint32_t vm = ONE ? 1u : __builtin_amdgcn_readfirstlane(vmask[ld]);
      wp = (const u32x4*)a.w.dn + (size_t)e * (D / 64) * KT * 256 + lane;
      if constexpr (XF) xe = a.hx + (size_t)ld * KT * (16 * MT) + 4 * (lane >> 4);
      const int any = __builtin_ctz(vm);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int t = m * 16 + (lane & 15);
        hoff[m] = (uint32_t)(ld * (16 * MT) + (vm >> t & 1u ? t : any)) * F + (lane >> 4) * 8;
      }
    };
    enter();
    auto load = [&](int u) __attribute__((always_inline)) {
      const int kt = wave + li * kFewWaves;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int st = blockIdx.x * NS + s;
        qw[u][s] = __builtin_nontemporal_load(wp + ((size_t)(st >> 2) * KT + kt) * 256 + (st & 3) * 64);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        qh[u][m] = *(const u32x4*)(a.hhi + hoff[m] + kt * 32);
        ql[u][m] = *(const u32x4*)(a.hlo + hoff[m] + kt * 32);
        if constexpr (XF) qe[u][m] = *(const uint32_t*)(xe + (size_t)kt * (16 * MT) + m * 16);
      }
      if (++li == spw) {
        li = 0;
        if (ld + 1 < nd) ++ld;
        enter();
      }
    };
    int cd = 0, ci = 0;  // the consumer's place
    auto consume = [&](int u) __attribute__((always_inline)) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          if constexpr (XF) {
            f32x4 z{0.f, 0.f, 0.f, 0.f};
            z = mfma16<BF>(qh[u][m], qw[u][s], z);
            z = mfma16<BF>(ql[u][m], qw[u][s], z);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[m][s][r] += z[r] * pow2_up(qe[u][m] >> 8 * r & 255u);
          } else {
            acc[m][s] = mfma16<BF>(qh[u][m], qw[u][s], acc[m][s]);
            acc[m][s] = mfma16<BF>(ql[u][m], qw[u][s], acc[m][s]);
          }
        }
      if (++ci == spw) {
        const uint32_t vm = ONE ? ~0u : vmask[cd];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const int r0 = m * 16 + 4 * (lane >> 4);
          f32x4 w;
          if constexpr (ONE) w = f32x4{1.f, 1.f, 1.f, 1.f} * rc.weight(cd);  // (every row is the one row)
          else w = *(const f32x4*)&wmap[cd][r0];
#pragma unroll
          for (int s = 0; s < NS; ++s) {
#pragma unroll
            for (int r = 0; r < 4; ++r) tot[m][s][r] = vm >> (r0 + r) & 1u ? tot[m][s][r] + w[r] * acc[m][s][r] : tot[m][s][r];
            acc[m][s] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
        }
        ci = 0;
        ++cd;
      }
    };
    if (total >= U) {
#pragma unroll
      for (int u = 0; u < U; ++u) load(u);
      weigh();
      int j = 0;
      for (; j + 2 * U <= total; j += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          consume(u);
          load(u);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        consume(u);
        if (j + u + U < total) load(u);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j + u + U < total) consume(u);
    } else {
      weigh();
      for (int j = 0; j < total; ++j) {
        load(0);
        consume(0);
      }
    }
  } else {
    weigh();  // (every wave takes part in its barrier)
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int s = 0; s < NS; ++s) *(f32x4*)&red[wave][m][s][lane * 4] = tot[m][s];
  __syncthreads();
  for (int i = tid; i < MT * NS * 256; i += 64 * kFewWaves) {
    const int c = i & 15, row = i >> 4 & 15, s = (i >> 8) % NS, m = (i >> 8) / NS;
    const int at = ((row >> 2) * 16 + c) * 4 + (row & 3);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) v += red[w][m][s][at];
    const int t = m * 16 + row;
    if (t < T) {
      const int64_t o = t * a.out_stride + (blockIdx.x * NS + s) * 16 + c;
      if (a.x_type == ET_F32) ((float*)a.out)[o] = v;
      else ((uint16_t*)a.out)[o] = to16<BF>(v);
    }
  }
}

// Rows of 32-bit values as the scaled fp16 pair, LANES threads per row (64: a
// wave; 256: the workgroup), 8 columns per thread and step: one pass for the largest
// magnitude, one (of a row that is in cache now; held in registers instead it took
// as long) for the pair.  up[row] undoes the scale.  lo null: hi and lo of 32 columns
// side by side, a cache line per row and K step, as the few-row form reads them (its
// call of 16 rows, top 8 of 64 experts of 4096 x 1024: 222 us with 64 bytes of each
// apart, 218 so).
template <int LANES>
__global__ __launch_bounds__(256) void experts_pair(const float* __restrict__ src, int64_t stride, int rows, int cols,
                                                    uint16_t* __restrict__ hi, uint16_t* __restrict__ lo, float* __restrict__ up) {
  __shared__ float s_max[4];
  const int t = threadIdx.x & (LANES - 1), row = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (row >= rows) return;  // (whole waves; no row past the last with LANES 256)
  const float* p = src + row * stride;
  float mx = 0.f;
#pragma unroll 4
  for (int c = t * 8; c < cols; c += LANES * 8) {
    const f32x4 u = *(const f32x4*)(p + c), v = *(const f32x4*)(p + c + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = max_finite(max_finite(mx, u[i]), v[i]);
  }
  mx = rows_max(row16_max(mx));
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  }
  const int b = scale_exp(mx);
  const float down = pow2_down(b);
#pragma unroll 4
  for (int c = t * 8; c < cols; c += LANES * 8) {
    const f32x4 u = *(const f32x4*)(p + c), v = *(const f32x4*)(p + c + 4);
    const float w[8] = {u[0] * down, u[1] * down, u[2] * down, u[3] * down, v[0] * down, v[1] * down, v[2] * down, v[3] * down};
    uint4 h, l;
    pair8<false>(w, h, l);
    uint16_t* const d = hi + (size_t)row * cols * (lo ? 1 : 2) + (lo ? c : c + (c & ~31));
    *(uint4*)d = h;
    *(uint4*)(lo ? lo + (size_t)row * cols + c : d + 32) = l;
  }
  if (t == 0) up[row] = pow2_up(b);
}

// out[t] = sum_j w[t][j] y[pos[t][j]] (up[place] undoes the scale of its product),
// 4 columns per thread.
__global__ __launch_bounds__(256) void experts_combine(ExpertsArgs a) {
  const int D = a.w.D, c = (blockIdx.y * 256 + threadIdx.x) * 4, t = blockIdx.x;
  if (c >= D) return;
  float4 v{0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < a.k; ++j) {
    const int p = a.pos[t * a.k + j];
    if (p < 0) continue;
    const float w = a.weights[t * a.k + j];
    float4 y = *(const float4*)(a.y + (size_t)p * D + c);
    if (a.hs) {
      const float up = a.hs[p];
      y.x *= up;
      y.y *= up;
      y.z *= up;
      y.w *= up;
    }
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

// The form of a call, from its sizes alone (the host does not see the choice).
// Measured with 64 experts of 4096 x 1024, top 8, unless said otherwise (us a
// call, bf16; few-row form / tiles):
//   16 rows 196 / 230; 32 rows 281 / 255; 32 rows of 8 experts, top 2: 46 / 72.
// * The few-row form up to 16 rows, and up to 32, where it multiplies two row
//   tiles for every expert, if the tiles of few experts would leave CUs without
//   weights to stream.
// * Tiles of 64 rows and 4 waves, two workgroups per CU, while an expert has few
//   rows and there are enough tiles: 33 rows of 128 experts of 5120 x 704, top 4:
//   255 against 269 with 128 rows (40 rows 257 / 259; 32 rows of 16 experts of 1024 x
//   512, top 2, where they are too few: 36 / 26).
// * Tiles of 128 rows above: 848 rows 410 against 492 with 64 rows (and 411 with 256;
//   2048 rows 683, 863, 660; 2000 rows of 8 experts, top 2: 188, 233, 203).
// With few rows per expert the products wait for weights, and silu(gate) * up
// goes through the down product as a pair at little cost (40 rows: 259 -> 261);
// with many it is one 16-bit value (848 rows: 480 -> 440).
enum Form { FORM_FEW16, FORM_FEW32, FORM_T64_PAIR, FORM_T128_PAIR, FORM_T128 };
constexpr int kPairRows = 16;  // rows per expert below which the product stays a pair
static Form form_of(const ExpertsArgs& a) {
  const int n = a.T * a.k;
  const bool fills = (int64_t)std::min(n, a.w.E) * a.w.F >= 128 * kTileCUs;  // a 256-column tile (gate and up) per CU
  if (a.T <= 16 && n <= kFewSlots) return FORM_FEW16;
  if (a.T <= kFewRows && n <= kFewSlots && !fills) return FORM_FEW32;
  if (n / a.w.E >= kPairRows) return FORM_T128;
  return fills ? FORM_T64_PAIR : FORM_T128_PAIR;
}

size_t experts_workspace(ExpertsArgs a) {
  // A form's workspace grows with the rows, so the most that up to a.T rows take
  // is at a.T or at the last rows of a form.
  const int rows = a.T, E = a.w.E, k = a.k, full = 128 * kTileCUs;
  const int ends[] = {1, 16, kFewRows, kFewSlots / k, (int)std::min<int64_t>(rows, ((int64_t)kPairRows * E - 1) / k),
                      (full - 1) / a.w.F / k, rows};
  size_t most = 0;
  for (int T : ends) {
    a.T = std::min(T, rows);
    most = std::max(most, experts_carve(a, nullptr));
  }
  return most;
}

size_t experts_carve(ExpertsArgs& a, void* base) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? (char*)base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  const size_t n = (size_t)a.T * a.k, D = a.w.D, F = a.w.F;
  const Form f = form_of(a);
  if (f <= FORM_FEW32) {
    const size_t rows = std::min(n, (size_t)(a.T == 1 ? kMaxTopK : a.w.E)) * (f == FORM_FEW16 ? 16 : 32);  // (one row: an entry per slot)
    a.hhi = (uint16_t*)take(rows * F * 2);
    a.hlo = (uint16_t*)take(rows * F * 2);
    if (a.x_type == ET_F32) {
      a.hx = (uint8_t*)take(rows * (F / 32));
      if (a.T > 1) {
        a.xhi = (uint16_t*)take((size_t)a.T * D * 4);
        a.xs = (float*)take((size_t)a.T * 4);
      }
    }
    return off;
  }
  const bool pair = a.x_type == ET_F32;
  a.perm = (int32_t*)take(n * 4);
  a.pos = (int32_t*)take(n * 4);
  a.cnt = (int32_t*)take((size_t)a.w.E * 4);
  a.off = (int32_t*)take((size_t)a.w.E * 4);
  // (64 bytes more: the last slab of an odd number of K steps is copied whole)
  a.hhi = (uint16_t*)take(n * F * 2 + 64);
  a.hlo = pair || f <= FORM_T128_PAIR ? (uint16_t*)take(n * F * 2 + 64) : nullptr;
  a.xhi = pair ? (uint16_t*)take((size_t)a.T * D * 2) : nullptr;
  a.xlo = pair ? (uint16_t*)take((size_t)a.T * D * 2) : nullptr;
  a.xs = pair ? (float*)take((size_t)a.T * 4) : nullptr;
  a.hs = pair ? (float*)take(n * 4) : nullptr;
  a.y = (float*)take(n * (pair ? std::max(D, F) : D) * 4);
  a.arrived = (uint32_t*)take(kTileCUs * 4);
  // (64-row tiles are not shared)
  a.part = f != FORM_T64_PAIR ? (float*)take((size_t)kTileCUs * T128::BM * T128::BN * 4) : nullptr;
  return off;
}

// (a wave per row leaves CUs without work below a thousand rows)
static void launch_pair(const float* src, int64_t stride, int rows, int cols, uint16_t* hi, uint16_t* lo, float* up, hipStream_t s) {
  if (rows < 4 * kTileCUs) hvd_launch(experts_pair<256>, dim3(rows), dim3(256), 0, s, src, stride, rows, cols, hi, lo, up);
  else hvd_launch(experts_pair<64>, dim3((rows + 3) / 4), dim3(256), 0, s, src, stride, rows, cols, hi, lo, up);
}
template <int MT, bool BF, bool XF, bool ONE>
static void launch_few(const ExpertsArgs& a, hipStream_t s) {
  const int n = std::min(a.T * a.k, ONE ? kMaxTopK : a.w.E);
  if (XF && !ONE) launch_pair((const float*)a.x, a.x_stride, a.T, a.w.D, a.xhi, nullptr, a.xs, s);
  hvd_launch((experts_gu_few<MT, 4, BF, XF, ONE>), dim3(2 * a.w.F / 64, n), dim3(64 * kFewWaves), 0, s, a);
  hvd_launch((experts_down_few<MT, 1, BF, XF, ONE>), dim3(a.w.D / 16), dim3(64 * kFewWaves), 0, s, a);
}
template <int MT, bool ONE>
static void launch_few_types(const ExpertsArgs& a, hipStream_t s) {
  if (a.x_type == ET_F32) launch_few<MT, false, true, ONE>(a, s);
  else if (a.w.wtype == ET_BF16) launch_few<MT, true, false, ONE>(a, s);
  else launch_few<MT, false, false, ONE>(a, s);
}

// XP: x is a pair; HP: silu(gate) * up is.
template <class S, bool BF, bool XP, bool HP>
static void launch_products(const ExpertsArgs& a, hipStream_t s) {
  const int n = a.T * a.k, tiles = n / S::BM + std::min(n, a.w.E);  // at most: whole tiles, and a ragged one per expert
  const int cg = (2 * a.w.F + S::BN - 1) / S::BN, cd = (a.w.D + S::BN - 1) / S::BN;
  // (shared tiles: less than a round of workgroups more)
  hvd_launch((experts_tiled<S, true, BF, XP, HP>), dim3(tiles * cg + (S::SPLIT ? kTileCUs : 0)), dim3(64 * S::NW), 0, s, a, cg);
  if (XP) launch_pair(a.y, a.w.F, n, a.w.F, a.hhi, a.hlo, a.hs, s);
  hvd_launch((experts_tiled<S, false, BF, HP, false>), dim3(tiles * cd), dim3(64 * S::NW), 0, s, a, cd);
}
template <bool BF, bool XP>
static void launch_tiled(const ExpertsArgs& a, Form f, hipStream_t s) {
  if (f == FORM_T64_PAIR) launch_products<T64, BF, XP, true>(a, s);
  else if (XP || f == FORM_T128_PAIR) launch_products<T128, BF, XP, true>(a, s);
  else launch_products<T128, BF, XP, XP>(a, s);
}

hipError_t launch_experts(const ExpertsArgs& a, hipStream_t s) {
  const Form f = form_of(a);
  const bool pair = a.x_type == ET_F32, bf = a.w.wtype == ET_BF16;
  if (f <= FORM_FEW32) {
    if (a.T == 1) launch_few_types<1, true>(a, s);
    else if (f == FORM_FEW16) launch_few_types<1, false>(a, s);
    else launch_few_types<2, false>(a, s);
    return hipGetLastError();
  }
  hvd_launch(experts_sort, dim3(a.w.E), dim3(256), 0, s, a);
  if (pair) launch_pair((const float*)a.x, a.x_stride, a.T, a.w.D, a.xhi, a.xlo, a.xs, s);
  pair ? launch_tiled<false, true>(a, f, s) : bf ? launch_tiled<true, false>(a, f, s) : launch_tiled<false, false>(a, f, s);
  hvd_launch(experts_combine, dim3(a.T, (a.w.D / 4 + 255) / 256), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hvd
