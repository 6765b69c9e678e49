// Operators on the rows of several sequences (append_kv.hip, attend.hip,
// adjust_logits.hip): kernel arguments, launchers, and the device code that
// finds a row's sequence.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "moe.h"

namespace hvd {

constexpr int kMaxSeqs = 4096;         // sequences of one batch
constexpr int kMaxStepRows = 1 << 20;  // rows of one call
constexpr int kMaxRowHeads = 256;      // heads of one tensor
constexpr int kMaxRowDim = 256;        // head dimension
constexpr int kMaxKeys = 1 << 29;      // keys that a sequence's pages may hold
constexpr int64_t kMaxTokStride = 1 << 26;
constexpr int kMaxVocab = 1 << 24;
constexpr int kMaxAdjustRows = 1 << 16;  // rows of one call of adjust_logits
constexpr int kMaxHistory = (1 << 20) - 1 - kMaxAdjustRows;  // a count has 20 bits
constexpr int kMaxBias = 2046;         // biased ids of one sequence

// The rows of a step (hvd_row_batch).  Row r of sequence s has starts[s] <= r <
// starts[s + 1]; everything read from here is bounded before it is used.
struct RowBatch {
  const int32_t* starts;   // [S + 1]
  const int32_t* lengths;  // [S]
  const int32_t* pages;    // [S][P], pages_stride apart
  const int64_t* tree;     // nullable [T]
  int64_t pages_stride;
  int S, T, P;
};
// One of the two halves of a paged cache: element strides of page, head, token.
struct CacheView {
  void* p;
  int64_t page, head, tok;
};

struct AppendArgs {
  RowBatch b;
  CacheView k, v;
  int n_pages, page_shift, H, Hq, D;
  int in_type, cache_type;
  const void *xk, *xv, *xq;  // xq nullable
  int64_t k_row, k_head, v_row, v_head, q_row, q_head;
  void* q_out;  // [T][Hq][D], of the cache's type
  const double* freqs;  // nullable [rot / 2]
  const int32_t* positions;  // nullable [T]
  int rot, interleaved;
};
hipError_t launch_append_kv(const AppendArgs& a, hipStream_t s);

struct AttendArgs {
  RowBatch b;
  CacheView k, v;
  int n_pages, page_shift, H, Hq, D;
  int type;
  const void* q;
  int64_t q_row, q_head;
  void* out;
  int64_t out_row, out_head;
  const float* slopes;   // nullable [Hq]
  const int32_t* first;  // nullable [T]
  const int32_t* prefix; // nullable [S]
  float scale, cap;
  int window;  // 0: none
  float* part;  // partial results, or null: no row's keys are split
};
size_t attend_workspace(const AttendArgs& a);
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);

struct AdjustArgs {
  RowBatch b;
  const void* logits;
  int64_t logits_stride;
  void* out;  // nullable
  int64_t out_stride;
  int type, V;
  int32_t* best;  // nullable [T]
  const int32_t* tokens;  // nullable [T]
  const int32_t* history;  // nullable [S][max_history]
  int64_t history_stride;
  int max_history;
  const int32_t *history_lengths, *prompt_lengths;
  const float *repetition, *frequency, *presence;  // nullable [S]
  const int32_t* bias_ids;  // nullable [S][n_bias]
  const float* bias;
  int64_t bias_ids_stride, bias_stride;
  int n_bias;
  const int32_t* allowed;  // nullable [T][(V + 31) / 32]
  int64_t allowed_stride;
  uint64_t* part;  // best of each part of a row
};
size_t adjust_workspace(const AdjustArgs& a);
hipError_t launch_adjust_logits(const AdjustArgs& a, hipStream_t s);

#ifdef __HIPCC__

// Inclusive sum over the lanes of a wave, in the vector ALU (row shifts, then
// the last lane of a row of 16, then of 32, handed on).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// First row and end of sequence s, within the rows there are (s = S: the rows
// behind the last sequence).
__device__ __forceinline__ void seq_rows(const RowBatch& b, int s, int& a, int& e) {
  a = min(max(b.starts[s], 0), b.T);
  e = s < b.S ? min(max(b.starts[s + 1], a), b.T) : b.T;
}

// The sequence of a row, S if it lies behind the last one: how many sequences
// end at or before it, 64 at a time.  The whole wave calls it with one row.
__device__ __forceinline__ int seq_of_row(const RowBatch& b, int row) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  for (int s = 0; s < b.S; s += 64) {
    const int i = s + lane;
    const uint64_t ended = __builtin_amdgcn_ballot_w64(i < b.S && b.starts[min(i + 1, b.S)] <= row);
    n += __builtin_popcountll(ended);
    if (ended != ~0ull) break;
  }
  return n;
}

#endif

}  // namespace hvd
