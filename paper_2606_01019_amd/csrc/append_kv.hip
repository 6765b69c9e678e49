// Keys and values of a step's rows into a paged cache, keys (and queries)
// rotated on the way (gfx950).
//
// Row i of a sequence with n rows and a length of len keys (these included) is
// key ctx + i, ctx = len - n: token (ctx + i) % page of the cache page
// pages[(ctx + i) / page].  With the angle t = position * freqs[j] a pair (a, b)
// becomes (a cos t - b sin t, b cos t + a sin t); pairs are (j, j + rot / 2) or
// neighbours.  The angle is taken in 64 bits and reduced to a fraction of a turn
// there: off by the product's three roundings, 5e-7 radians at position 2^31 and less
// before it.  Its cosine and sine, and the rotation, are 32-bit, and each output is
// rounded once to the cache's type.
//
// Bound by memory for many rows and by latency for few.  A workgroup takes 4 rows
// (parts of one row where there are fewer than 1024): its threads compute each row's
// cosines and sines once for all heads, into LDS, and then go over the rows' octets
// of columns.  16437 rows of 20 heads of 80: 27 to 30 us, 3.5 to 3.9 TB/s; 878 rows of 48 heads of
// 128 from 32 bits 9.7 us.
#include "common.h"
#include "kernels.h"
#include "rows.h"

namespace hvd {
namespace {

constexpr int kThreads = 256;

template <int V>
struct Vec {
  typedef uint16_t half_ty __attribute__((ext_vector_type(V), aligned(2)));
  typedef uint16_t half_al __attribute__((ext_vector_type(V), aligned(2 * V)));
  typedef float float_ty __attribute__((ext_vector_type(V), aligned(4)));
};
template <>
struct Vec<1> {
  typedef uint16_t half_ty;
  typedef uint16_t half_al;
  typedef float float_ty;
};

template <int V>
__device__ __forceinline__ float at(const typename Vec<V>::float_ty& v, int j) {
  if constexpr (V == 1) return v;
  else return v[j];
}

template <int V>
__device__ __forceinline__ void load_v(const void* p, int64_t i, int type, float (&v)[V]) {
  if (type == ET_F32) {
    const auto a = *(const typename Vec<V>::float_ty*)((const float*)p + i);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = at<V>(a, j);
  } else {
    const auto a = *(const typename Vec<V>::half_ty*)((const uint16_t*)p + i);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      uint16_t b;
      if constexpr (V == 1) b = a;
      else b = a[j];
      v[j] = type == ET_BF16 ? bf2f(b) : h2f(b);
    }
  }
}
template <int V>
__device__ __forceinline__ void store_v(uint16_t* p, bool bf16, const float (&v)[V]) {
  typename Vec<V>::half_al o;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint16_t b = bf16 ? __builtin_bit_cast(uint16_t, (__bf16)v[j]) : f2h(v[j]);
    if constexpr (V == 1) o = b;
    else o[j] = b;
  }
  *(typename Vec<V>::half_al*)p = o;
}

// V columns per thread and step; ROWS rows per workgroup.
template <int V, int ROWS>
__global__ __launch_bounds__(kThreads) void append_rows(AppendArgs a, int parts) {
  __shared__ float2 turn[ROWS][kMaxRowDim / 2];
  __shared__ int s_page[ROWS], s_slot[ROWS], s_pos[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = blockIdx.x / parts, part = blockIdx.x - group * parts;
  const int row0 = group * ROWS;
  for (int r = wave; r < ROWS; r += kThreads / 64) {
    const int row = row0 + r;
    int page = -1, slot = 0, pos = 0;
    if (row < a.b.T) {
      const int s = seq_of_row(a.b, row);
      if (s < a.b.S) {
        int b, e;
        seq_rows(a.b, s, b, e);
        const int ctx = a.b.lengths[s] - (e - b);
        const int key = ctx + row - b;
        pos = a.positions ? a.positions[row]
                          : a.b.tree ? ctx + __builtin_popcountll(a.b.tree[row]) - 1 : key;
        const int pi = key >> a.page_shift;
        if (key >= 0 && pi < a.b.P) {
          page = a.b.pages[s * a.b.pages_stride + pi];
          if ((unsigned)page >= (unsigned)a.n_pages) page = -1;
        }
        if (page < 0) page = -2;  // no place in the cache; the query is rotated all the same
        slot = key & ((1 << a.page_shift) - 1);
      }
    }
    if (lane == 0) {
      s_page[r] = page;
      s_slot[r] = slot;
      s_pos[r] = pos;
    }
  }
  __syncthreads();
  const int half = a.rot >> 1;
  for (int i = tid; i < ROWS * half; i += kThreads) {
    const int r = i / half, j = i - r * half;
    double t = (double)s_pos[r] * a.freqs[j] * 0.15915494309189533577;  // turns
    t -= rint(t);
    const float x = 2.f * (float)t;
    turn[r][j] = float2{cospif(x), sinpif(x)};
  }
  __syncthreads();
  const int per_head = a.D / V;
  const int heads = 2 * a.H + (a.xq ? a.Hq : 0);
  const int units = heads * per_head;
  for (int u = part * kThreads + tid; u < ROWS * units; u += parts * kThreads) {
    const int r = u / units, w = u - r * units;
    int h = w / per_head;
    const int c = (w - h * per_head) * V;
    const int64_t row = row0 + r;
    if (row >= a.b.T) break;
    const int page = s_page[r];
    // heads in the order key, value, query
    const int what = h < a.H ? 0 : h < 2 * a.H ? 1 : 2;
    if (page < 0 && what < 2) continue;
    h -= what * a.H;
    const void* src = what == 0 ? a.xk : what == 1 ? a.xv : a.xq;
    const int64_t off = what == 0 ? row * a.k_row + h * a.k_head
                        : what == 1 ? row * a.v_row + h * a.v_head : row * a.q_row + h * a.q_head;
    float x[V];
    if (page == -1) {  // a query behind the last sequence
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = 0.f;
    } else {
      load_v<V>(src, off + c, a.in_type, x);
      if (what != 1 && c < a.rot) {
        if (a.interleaved) {
          if constexpr (V > 1) {
#pragma unroll
            for (int j = 0; j < V; j += 2) {
              const float2 t = turn[r][(c + j) >> 1];
              const float p = x[j] * t.x - x[j + 1] * t.y;
              x[j + 1] = x[j + 1] * t.x + x[j] * t.y;
              x[j] = p;
            }
          }
        } else {
          const bool low = c < half;
          float y[V];
          load_v<V>(src, off + (low ? c + half : c - half), a.in_type, y);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float2 t = turn[r][(low ? c : c - half) + j];
            x[j] = low ? x[j] * t.x - y[j] * t.y : x[j] * t.x + y[j] * t.y;
          }
        }
      }
    }
    uint16_t* dst;
    if (what == 2) {
      dst = (uint16_t*)a.q_out + (row * a.Hq + h) * a.D + c;
    } else {
      const CacheView& cv = what == 0 ? a.k : a.v;
      dst = (uint16_t*)cv.p + page * cv.page + h * cv.head + (int64_t)s_slot[r] * cv.tok + c;
    }
    store_v<V>(dst, a.cache_type == ET_BF16, x);
  }
}

template <int V>
void launch_v(const AppendArgs& a, hipStream_t s) {
  const int units = (2 * a.H + (a.xq ? a.Hq : 0)) * (a.D / V);
  constexpr int ROWS = 4;
  if (a.b.T >= 1024) {
    hvd_launch((append_rows<V, ROWS>), dim3((a.b.T + ROWS - 1) / ROWS), dim3(kThreads), 0, s, a, 1);
  } else {
    const int parts = (units + kThreads - 1) / kThreads;
    hvd_launch((append_rows<V, 1>), dim3(a.b.T * parts), dim3(kThreads), 0, s, a, parts);
  }
}

}  // namespace

hipError_t launch_append_kv(const AppendArgs& a, hipStream_t s) {
  // whole vectors of columns on either side of every pair
  const int u = a.interleaved ? a.rot : a.rot / 2;
  if (u % 8 == 0) launch_v<8>(a, s);
  else if (u % 4 == 0) launch_v<4>(a, s);
  else if (u % 2 == 0) launch_v<2>(a, s);
  else launch_v<1>(a, s);
  return hipGetLastError();
}

}  // namespace hvd
