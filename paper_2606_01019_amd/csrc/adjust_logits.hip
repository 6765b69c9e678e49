// Penalties for repeated tokens, biases and masks on the logits of a step's
// rows, and the best token of each (gfx950).
//
// For a row of sequence s and a token v, with n the times v was generated (in
// the history from prompt_lengths[s] on, and on the row's own path through this
// step: the rows of its sequence up to itself, or those of its tree mask) and
// "seen" where n > 0 or v lies anywhere in the history:
//
//   x' = seen ? (x > 0 ? x / repetition : x * repetition) : x
//   x' = x' - frequency * n;  x' = x' - presence * [n > 0];  x' = x' + bias(v)
//   x' = allowed(v) ? x' : -inf
//
// each step a 32-bit operation of its own, in that order, rounded to the
// logits' type once at the end; the best token is the lowest one that has the
// largest 32-bit x'.
//
// A workgroup takes a part of the vocabulary and a run of rows.  The part's
// counts live in LDS, a word per token: bits 0-19 the count n, 20-30 the entry
// of the bias list + 1 (the later entry wins), 31 "in the history's prompt".
// A sequence's history is counted once for its rows of the run (integer
// atomics: no order matters), a row's path is added and taken away.
#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace hvd {
namespace {

#pragma clang fp contract(off)

constexpr int kThreads = 256;
constexpr uint32_t kPrompt = 1u << 31;
constexpr uint32_t kCount = (1u << 20) - 1;

typedef uint16_t u16x8_a2 __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4_e __attribute__((ext_vector_type(4), aligned(4)));

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
__device__ __forceinline__ float load1(const void* p, int64_t i, int type) {
  if (type == ET_F32) return ((const float*)p)[i];
  const uint16_t b = ((const uint16_t*)p)[i];
  return type == ET_BF16 ? bf2f(b) : h2f(b);
}
__device__ __forceinline__ uint16_t half_bits(float v, int type) {
  return type == ET_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)v) : f2h(v);
}
__device__ __forceinline__ void store8(void* p, int64_t i, int type, const float (&v)[8]) {
  if (type == ET_F32) {
    float* d = (float*)p + i;
    *(f32x4_e*)d = f32x4_e{v[0], v[1], v[2], v[3]};
    *(f32x4_e*)(d + 4) = f32x4_e{v[4], v[5], v[6], v[7]};
  } else {
    u16x8_a2 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = half_bits(v[j], type);
    *(u16x8_a2*)((uint16_t*)p + i) = o;
  }
}
__device__ __forceinline__ void store1(void* p, int64_t i, int type, float v) {
  if (type == ET_F32) ((float*)p)[i] = v;
  else ((uint16_t*)p)[i] = half_bits(v, type);
}

// Larger for a larger value, then for a lower token; 0 for a value that is
// never chosen (-inf, NaN).  Both zeros count as equal.
__device__ __forceinline__ uint64_t rank_of(float v, int token) {
  if (!(v > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(v + 0.f);
  const uint32_t o = u >> 31 ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (0xffffffffu - (uint32_t)token);
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t w = (uint64_t)(uint32_t)__shfl_xor((uint32_t)(v >> 32), o) << 32 | (uint32_t)__shfl_xor((uint32_t)v, o);
    v = w > v ? w : v;
  }
  return v;
}

struct Penalty {
  float repetition, frequency, presence;
  const float* bias;
  bool rep, freq, pres;
};

__device__ __forceinline__ float adjusted(float x, uint32_t w, const Penalty& p) {
  const uint32_t n = w & kCount;
  if (p.rep && (w & (kPrompt | kCount))) x = x > 0.f ? x / p.repetition : x * p.repetition;
  if (n) {
    if (p.freq) x = x - p.frequency * (float)n;
    if (p.pres) x = x - p.presence;
  }
  const uint32_t e = w >> 20 & 2047;
  if (e) x = x + p.bias[e - 1];
  return x;
}

__global__ __launch_bounds__(kThreads) void adjust_rows(AdjustArgs a, int seg, int segs, int run) {
  extern __shared__ __attribute__((aligned(16))) uint32_t word[];
  __shared__ uint64_t red[2][kThreads / 64];  // by turns: a row is read while the next one is written
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % segs;
  const int v0 = part * seg, nv = min(seg, a.V - v0);
  const int r0 = blockIdx.x / segs * run, r1 = min(r0 + run, a.b.T);
  const bool counts = a.repetition || a.frequency || a.presence;
  const bool words = counts || a.n_bias > 0;
  auto bump = [&](int token, uint32_t by) __attribute__((always_inline)) {
    const int d = token - v0;
    if ((unsigned)d < (unsigned)nv) atomicAdd(&word[d], by);
  };
  int held = -1;  // the sequence whose words are in LDS
  int b = 0, e = 0;
  Penalty p{};
  for (int row = r0; row < r1; ++row) {
    const int s = seq_of_row(a.b, row);
    const bool live = s < a.b.S;
    uint64_t mask = 0;
    if (live) {
      seq_rows(a.b, s, b, e);
      if (counts && a.b.tree) mask = a.b.tree[row];
      if (s != held) {
        if (words) {
          __syncthreads();
          for (int i = tid; i < nv; i += kThreads) word[i] = 0;
          __syncthreads();
        }
        if (counts && a.history) {
          const int n = min(max(a.history_lengths[s], 0), a.max_history);
          const int prompt = a.prompt_lengths ? a.prompt_lengths[s] : 0;
          const int32_t* h = a.history + s * a.history_stride;
          for (int i = tid; i < n; i += kThreads) {
            const int d = h[i] - v0;
            if ((unsigned)d < (unsigned)nv) {
              if (i < prompt) atomicOr(&word[d], kPrompt);
              else atomicAdd(&word[d], 1u);
            }
          }
        }
        if (counts && a.tokens && !a.b.tree)
          for (int i = b + tid; i < row; i += kThreads) bump(a.tokens[i], 1u);
        for (int i = tid; i < a.n_bias; i += kThreads) {
          const int d = a.bias_ids[s * a.bias_ids_stride + i] - v0;
          if ((unsigned)d < (unsigned)nv) {
            uint32_t old = word[d];
            while ((old >> 20 & 2047) < (uint32_t)(i + 1)) {
              const uint32_t was = atomicCAS(&word[d], old, (old & ~(2047u << 20)) | (uint32_t)(i + 1) << 20);
              if (was == old) break;
              old = was;
            }
          }
        }
        held = s;
        p.rep = a.repetition != nullptr;
        p.freq = a.frequency != nullptr;
        p.pres = a.presence != nullptr;
        p.repetition = p.rep ? a.repetition[s] : 1.f;
        p.frequency = p.freq ? a.frequency[s] : 0.f;
        p.presence = p.pres ? a.presence[s] : 0.f;
        p.bias = a.bias + s * a.bias_stride;
      }
      if (counts && a.tokens) {
        if (!a.b.tree) {
          if (tid == 0) bump(a.tokens[row], 1u);
        } else if (tid < 64 && (mask >> tid & 1) && b + tid < e) {
          bump(a.tokens[b + tid], 1u);
        }
      }
      if (words) __syncthreads();
    }
    const int64_t in = row * a.logits_stride + v0, to = row * a.out_stride + v0;
    const int32_t* ok = live && a.allowed ? a.allowed + row * a.allowed_stride : nullptr;
    uint64_t best = 0;
    for (int c = tid * 8; c < nv; c += kThreads * 8) {
      const int v = v0 + c;
      const uint32_t bits = ok ? (uint32_t)ok[v >> 5] >> (v & 31) : 0xffu;
      if (c + 8 <= nv) {
        float x[8];
        load8(a.logits, in + c, a.type, x);
        if (live && words) {
          const uint4 wa = *(const uint4*)&word[c], wb = *(const uint4*)&word[c + 4];
          const uint32_t w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (w[j]) x[j] = adjusted(x[j], w[j], p);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!(bits >> j & 1)) x[j] = -INFINITY;
        if (a.out) store8(a.out, to + c, a.type, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint64_t k = rank_of(x[j], v + j);
          best = k > best ? k : best;
        }
      } else {
        for (int j = 0; c + j < nv; ++j) {
          float x = load1(a.logits, in + c + j, a.type);
          if (live && words && word[c + j]) x = adjusted(x, word[c + j], p);
          if (!(bits >> j & 1)) x = -INFINITY;
          if (a.out) store1(a.out, to + c + j, a.type, x);
          const uint64_t k = rank_of(x, v + j);
          best = k > best ? k : best;
        }
      }
    }
    if (a.best) {
      best = wave_max_u64(best);
      if (lane == 0) red[row & 1][wave] = best;
    }
    __syncthreads();
    if (a.best && tid == 0) {
      for (int w = 1; w < kThreads / 64; ++w) best = red[row & 1][w] > best ? red[row & 1][w] : best;
      a.part[(int64_t)row * segs + part] = live ? best : 0;
    }
    // a tree's next row starts without this one's path
    if (live && counts && a.tokens && a.b.tree && tid < 64 && (mask >> tid & 1) && b + tid < e) bump(a.tokens[b + tid], ~0u);
  }
}

__global__ __launch_bounds__(kThreads) void best_of_parts(const uint64_t* part, int segs, int rows, int32_t* best) {
  const int row = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= rows) return;
  uint64_t v = 0;
  for (int i = lane; i < segs; i += 64) {
    const uint64_t w = part[(int64_t)row * segs + i];
    v = w > v ? w : v;
  }
  v = wave_max_u64(v);
  if (lane == 0) best[row] = v ? (int32_t)(0xffffffffu - (uint32_t)v) : -1;
}

// The vocabulary's parts and the rows of a workgroup.
struct Plan {
  int seg, segs, run;
};
Plan plan_of(const AdjustArgs& a) {
  const int seg = a.b.T <= 8 ? 2048 : 8192;
  const int segs = (a.V + seg - 1) / seg;
  const int run = std::min(16, std::max(1, (int)((int64_t)a.b.T * segs / 2048)));
  return Plan{seg, segs, run};
}

}  // namespace

size_t adjust_workspace(const AdjustArgs& a) { return (size_t)a.b.T * plan_of(a).segs * sizeof(uint64_t); }

hipError_t launch_adjust_logits(const AdjustArgs& a, hipStream_t s) {
  const Plan p = plan_of(a);
  const int groups = (a.b.T + p.run - 1) / p.run;
  const bool words = a.repetition || a.frequency || a.presence || a.n_bias > 0;
  hvd_launch(adjust_rows, dim3((unsigned)(groups * p.segs)), dim3(kThreads), words ? p.seg * 4 : 0, s, a, p.seg, p.segs, p.run);
  if (a.best)
    hvd_launch(best_of_parts, dim3((a.b.T + 3) / 4), dim3(kThreads), 0, s, (const uint64_t*)a.part, p.segs, a.b.T, a.best);
  return hipGetLastError();
}

}  // namespace hvd
