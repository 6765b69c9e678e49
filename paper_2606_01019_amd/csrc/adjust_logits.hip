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
// atomics: no order matters); from row to row the words follow the path.
//
// Bound by memory for many rows: a row's logits of the part are on their way to
// registers before the words are ready, and only touched tokens cost more than
// a copy.  905 rows of 128256 32-bit logits, everything given: 233 us, 4.0 TB/s
// (a large copy: 4.7 to 4.8); one row, 16 to 17 us, bound by the call itself (kernels: 8).
#include "common.h"
#include "kernels.h"
#include "rows.h"

#include <algorithm>

namespace hvd {
namespace {

#pragma clang fp contract(off)

constexpr int kThreads = 256;
constexpr uint32_t kPrompt = 1u << 31;
constexpr uint32_t kCount = (1u << 20) - 1;

typedef uint16_t u16x8_a2 __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4_e __attribute__((ext_vector_type(4), aligned(4)));

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

// Larger for a larger value, then for a lower token; 0 for a value that is never
// chosen (-inf, NaN).  Both zeros count as equal.
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
template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float wave_max_f(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  v = fmaxf(v, dpp_f<0x140>(v));
  return rows_max(v);
}

__device__ __forceinline__ int wave_min_i(int v) {
  v = min(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false));
  v = min(v, __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false));
  v = min(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false));
  v = min(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false));
  const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = min((int)a[0], (int)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return min((int)b[0], (int)b[1]);
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

// Eight logits of one row.
template <int TYPE>
struct Octet {
  f32x4_e a, b;
  __device__ __forceinline__ void load(const void* p, int64_t at) {
    a = *(const f32x4_e*)((const float*)p + at);
    b = *(const f32x4_e*)((const float*)p + at + 4);
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  }
};
template <int TYPE>
struct HalfOctet {
  u16x8_a2 a;
  __device__ __forceinline__ void load(const void* p, int64_t at) { a = *(const u16x8_a2*)((const uint16_t*)p + at); }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = TYPE == ET_BF16 ? bf2f(a[j]) : h2f(a[j]);
  }
};
template <>
struct Octet<ET_F16> : HalfOctet<ET_F16> {};
template <>
struct Octet<ET_BF16> : HalfOctet<ET_BF16> {};

// The words of a sequence's history: 16 tokens per thread at once.
__device__ __forceinline__ void count_history(const AdjustArgs& a, int s, int v0, int nv, uint32_t* word) {
  typedef int32_t i32x4_e __attribute__((ext_vector_type(4), aligned(4)));
  const int n = min(max(a.history_lengths[s], 0), a.max_history);
  const int prompt = a.prompt_lengths ? a.prompt_lengths[s] : 0;
  const int32_t* h = a.history + s * a.history_stride;
  constexpr int U = 4;
  for (int i0 = threadIdx.x * 4; i0 < n; i0 += kThreads * 4 * U) {
    i32x4_e t[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kThreads * 4;
      t[u] = i32x4_e{-1, -1, -1, -1};
      if (i + 4 <= n) {
        t[u] = *(const i32x4_e*)(h + i);
      } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (i + j < n) t[u][j] = h[i + j];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = t[u][j] - v0;
        if (t[u][j] >= 0 && (unsigned)d < (unsigned)nv) {
          if (i0 + u * kThreads * 4 + j < prompt) atomicOr(&word[d], kPrompt);
          else atomicAdd(&word[d], 1u);
        }
      }
  }
}

// CH octets of logits per thread: a part has 2048 CH tokens, octet i of thread t
// starts at token (i * 256 + t) * 8 of it; the vocabulary's last tokens, where
// they are no octet, go one to a thread.
template <int CH, int TYPE>
__global__ __launch_bounds__(kThreads, 4) void adjust_rows(AdjustArgs a, int segs, int run) {
  extern __shared__ __attribute__((aligned(16))) uint32_t word[];
  __shared__ float2 red[2][kThreads / 64];  // by turns: a row is read while the next one is written
  constexpr int SEG = CH * kThreads * 8;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = blockIdx.x % segs;
  const int v0 = part * SEG, nv = min(SEG, a.V - v0), nv8 = nv & ~7;
  const int r0 = blockIdx.x / segs * run, r1 = min(r0 + run, a.b.T);
  const bool counts = a.repetition || a.frequency || a.presence;
  const bool words = counts || a.n_bias > 0, path = counts && a.tokens;
  const auto clear = [&]() __attribute__((always_inline)) {
    for (int i = tid * 4; i < SEG; i += kThreads * 4) *(uint4*)&word[i] = uint4{0, 0, 0, 0};
  };
  const auto bump = [&](int token, uint32_t by) __attribute__((always_inline)) {
    const int d = token - v0;
    if ((unsigned)d < (unsigned)nv) atomicAdd(&word[d], by);
  };
  if (words) clear();
  bool live = false;
  int b = 0, e = 0;        // rows of the sequence whose words are in LDS
  uint64_t on_path = 0;    // its rows that are counted in them (tree)
  int my_token = -1;       // of row b + tid (tree)
  Penalty p{};
  for (int row = r0; row < r1; ++row) {
    // (octets past the part's end are not used: any other in their place)
    Octet<TYPE> raw[CH];
    uint32_t bits[CH];  // of the mask
    const auto load = [&]() __attribute__((always_inline)) {
      if (nv8 > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const int c = min((i * kThreads + tid) * 8, nv8 - 8);
          raw[i].load(a.logits, row * a.logits_stride + v0 + c);
          bits[i] = a.allowed ? (uint32_t)a.allowed[row * a.allowed_stride + ((v0 + c) >> 5)] >> (c & 31) : ~0u;
        }
      }
    };
    const uint64_t mask = path && a.b.tree ? (uint64_t)a.b.tree[row] : 0;
    const int own = path && !a.b.tree ? a.tokens[row] : -1;
    // on their way while the words are made, where registers allow it
    constexpr bool kEarly = CH * (TYPE == ET_F32 ? 2 : 1) <= 4;
    if (kEarly) load();
    if (row == r0 || (live && row >= e)) {
      const int s = seq_of_row(a.b, row);
      live = s < a.b.S;
      if (live) {
        seq_rows(a.b, s, b, e);
        if (words) {
          if (row != r0) clear();  // (every wave has read them: the barrier at a row's end)
          __syncthreads();
        }
        if (counts && a.history) count_history(a, s, v0, nv, word);
        if (path) {
          on_path = 0;
          if (a.b.tree) my_token = tid < 64 && b + tid < e ? a.tokens[b + tid] : -1;
          else
            for (int i = b + tid; i < row; i += kThreads) bump(a.tokens[i], 1u);
        }
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
        p.rep = a.repetition != nullptr;
        p.freq = a.frequency != nullptr;
        p.pres = a.presence != nullptr;
        p.repetition = p.rep ? a.repetition[s] : 1.f;
        p.frequency = p.freq ? a.frequency[s] : 0.f;
        p.presence = p.pres ? a.presence[s] : 0.f;
        p.bias = a.bias + s * a.bias_stride;
      }
    }
    if (!kEarly) load();
    if (live) {
      if (path) {
        if (a.b.tree) {  // from the last row's path to this one's
          const uint64_t change = mask ^ on_path;
          if (tid < 64 && (change >> lane & 1)) bump(my_token, mask >> lane & 1 ? 1u : ~0u);
          on_path = mask;
        } else if (tid == 0) {
          bump(own, 1u);
        }
      }
      if (words) __syncthreads();
    }
    const int64_t to = row * a.out_stride + v0;
    const int32_t* ok = live && a.allowed ? a.allowed + row * a.allowed_stride : nullptr;
    float top = -INFINITY;  // the thread's largest and its first place: 8 i + j, 8 CH for the single token
    int place = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      __builtin_amdgcn_sched_barrier(0);  // one octet at a time: registers
      const int c = (i * kThreads + tid) * 8;
      if (c >= nv8) break;
      float x[8];
      raw[i].values(x);
      if (live && words) {
        const uint4 wa = *(const uint4*)&word[c], wb = *(const uint4*)&word[c + 4];
        const uint32_t w[8] = {wa.x, wa.y, wa.z, wa.w, wb.x, wb.y, wb.z, wb.w};
        uint32_t touched = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) touched |= w[j] ? 1u << j : 0;
        while (touched) {  // few are: one at a time
          const int j = __builtin_ctz(touched);
          touched &= touched - 1;
          float v = x[0];
#pragma unroll
          for (int q = 1; q < 8; ++q) v = j == q ? x[q] : v;
          v = adjusted(v, word[c + j], p);
#pragma unroll
          for (int q = 0; q < 8; ++q) x[q] = j == q ? v : x[q];
        }
      }
      if (ok) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = bits[i] >> j & 1 ? x[j] : -INFINITY;
      }
      if (a.out) store8(a.out, to + c, TYPE, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool more = x[j] > top;
        top = more ? x[j] : top;
        place = more ? 8 * i + j : place;
      }
    }
    if (nv8 + tid < nv) {
      const int c = nv8 + tid;
      float x = load1(a.logits, row * a.logits_stride + v0 + c, TYPE);
      if (live && words && word[c]) x = adjusted(x, word[c], p);
      if (ok && !((uint32_t)ok[(v0 + c) >> 5] >> (c & 31) & 1)) x = -INFINITY;
      if (a.out) store1(a.out, to + c, TYPE, x);
      if (x > top) {
        top = x;
        place = 8 * CH;
      }
    }
    if (a.best) {
      const int token = v0 + (place == 8 * CH ? nv8 + tid : ((place >> 3) * kThreads + tid) * 8 + (place & 7));
      const float most = wave_max_f(top);
      const int lowest = wave_min_i(top == most ? token : 0x7fffffff);
      if (lane == 0) red[row & 1][wave] = float2{most, __int_as_float(lowest)};
    }
    __syncthreads();
    if (a.best && tid == 0) {
      uint64_t k = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 64; ++w) {
        const uint64_t r = rank_of(red[row & 1][w].x, __float_as_int(red[row & 1][w].y));
        k = r > k ? r : k;
      }
      a.part[(int64_t)row * segs + part] = live ? k : 0;
    }
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

// The vocabulary's parts and the rows of a workgroup.  Small parts while the rows do not
// fill the card: up to 8 rows of 128256 logits 7.7 to 9.5 us of kernels, with large ones 9.9
// to 12.2; every part reads the whole history, so that 33 rows with 4096 tokens take 18.3
// in place of 15.7 (between them, 9 to 16 rows would still gain 2).  Runs of rows share
// a count: one for every 4096 workgroups there would be takes 905 rows in 233 us, one for
// every 2048 254 and every 8192 275.
struct Plan {
  bool small;  // parts of 2048 tokens
  int segs, run;
};
Plan plan_of(const AdjustArgs& a) {
  const bool small = a.b.T <= 8;
  const int seg = small ? 2048 : 8192;
  const int segs = (a.V + seg - 1) / seg;
  const int run = std::min(16, std::max(1, (int)((int64_t)a.b.T * segs / 4096)));
  return Plan{small, segs, run};
}

template <int CH, int TYPE>
void launch_type(const AdjustArgs& a, const Plan& p, hipStream_t s) {
  const bool words = a.repetition || a.frequency || a.presence || a.n_bias > 0;
  const int groups = (a.b.T + p.run - 1) / p.run;
  hvd_launch((adjust_rows<CH, TYPE>), dim3((unsigned)(groups * p.segs)), dim3(kThreads), words ? CH * kThreads * 8 * 4 : 0, s, a,
             p.segs, p.run);
}
template <int CH>
void launch_ch(const AdjustArgs& a, const Plan& p, hipStream_t s) {
  if (a.type == ET_F32) launch_type<CH, ET_F32>(a, p, s);
  else if (a.type == ET_F16) launch_type<CH, ET_F16>(a, p, s);
  else launch_type<CH, ET_BF16>(a, p, s);
}

}  // namespace

size_t adjust_workspace(const AdjustArgs& a) { return (size_t)a.b.T * plan_of(a).segs * sizeof(uint64_t); }

hipError_t launch_adjust_logits(const AdjustArgs& a, hipStream_t s) {
  const Plan p = plan_of(a);
  if (p.small) launch_ch<1>(a, p, s);
  else launch_ch<4>(a, p, s);
  if (a.best)
    hvd_launch(best_of_parts, dim3((a.b.T + 3) / 4), dim3(kThreads), 0, s, (const uint64_t*)a.part, p.segs, a.b.T, a.best);
  return hipGetLastError();
}

}  // namespace hvd
