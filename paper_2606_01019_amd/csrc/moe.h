// Kernel argument blocks and host-side launchers of an expert layer's
// operators (route.hip, block_norm.hip, experts.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/hvd.h"

namespace hvd {

// Element types of the operators' buffers (HVD_F16, HVD_BF16, HVD_F32).
enum ElemType { ET_F16 = 0, ET_BF16 = 1, ET_F32 = 2 };
inline size_t elem_bytes(int t) { return t == ET_F32 ? 4 : 2; }

constexpr int kMaxExperts = 512;
constexpr int kMaxTopK = 16;
constexpr int kMaxGroups = 64;
constexpr int kMaxNormDim = 16384;
constexpr int kMaxOpRows = 1 << 23;         // rows of one routing or norm call
constexpr int kFewRows = 32;               // most rows of the experts' few-row form
constexpr int kMaxExpertRows = 1 << 18;  // rows of one call of the experts

struct RouteArgs {
  const void* logits;  // [rows][E], `stride` elements apart
  int64_t stride;
  int dtype;
  int rows, E, k;
  int sigmoid, G, top_groups, renorm;
  float scale;
  const float* bias;  // nullable [E]
  int32_t* ids;       // [rows][k]
  float* weights;     // [rows][k]
};
hipError_t launch_route(const RouteArgs& a, hipStream_t s);
// Checks of hvd_route's config, and its arguments as the launcher takes them (operators.cpp).
hvd_status check_route_config(const hvd_route_config* c);
RouteArgs route_args(const hvd_route_config& c, int rows, const void* logits, int dtype, int64_t stride,
                     const float* bias, int32_t* ids, float* weights);

// v = y (normalised, times post_gain, where post_gain is given) times gate;
// x_out = x + scale * v; h = x_out normalised, times gain.
struct BlockNormArgs {
  const void* x;
  int64_t x_stride;
  int x_type;
  const void* y;  // nullable
  int64_t y_stride;
  int y_type;
  const void* gate;  // nullable; strides in elements, 0 = broadcast
  int64_t gate_row, gate_col;
  int gate_type;
  const float* post_gain;  // nullable [D]
  const float* gain;       // nullable [D] (null: no h)
  float scale, eps;
  void* x_out;  // nullable; type of x
  int64_t x_out_stride;
  void* h;  // nullable
  int64_t h_stride;
  int h_type;
  // the verify path's form of h (then h is null): x_out * gain as fp16 hi + lo
  // operand fragments of MTtot row tiles and the sums of squares per 16 columns
  uint16_t *Nhi, *Nlo;
  float* ss_out;
  int MTtot;
  int rows, D;
};
hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s);

// Packed expert weights: the 16 x 32 operand fragments of pack_weight, expert
// after expert.  Gate and up rows alternate in strips of 16, so that a
// 32-column tile holds matching gate and up columns.
struct ExpertsW {
  const uint16_t* gu;  // [E][2F/64][D/32][4][512]
  const uint16_t* dn;  // [E][D/64][F/32][4][512]
  int E, D, F;
  int wtype;  // ET_F16 or ET_BF16
};

struct ExpertsArgs {
  ExpertsW w;
  const void* x;     // [T][D], x_stride elements apart
  int64_t x_stride;
  int x_type;        // the weights' type, or ET_F32 with fp16 weights (activations as an fp16 hi + lo pair)
  int T, k;
  const int32_t* ids;    // [T][k]
  const float* weights;  // [T][k]
  void* out;             // [T][D] of x's type
  int64_t out_stride;
  // workspace
  int32_t* perm;     // [T*k] slots in expert order, ascending within an expert
  int32_t* pos;      // [T*k] place of a slot in perm, -1 = an empty slot
  int32_t* cnt;      // [E] slots of each expert
  int32_t* off;      // [E] first place of each expert
  uint16_t *hhi, *hlo;  // silu(gate) * up, [places][F]
  uint16_t *xhi, *xlo;  // the activations' pair (ET_F32), [T][D]; few rows: xhi alone, [T][D/32][hi, lo][32]
  float *xs, *hs;       // ET_F32: what undoes the scales of x's rows [T] and the places' products [T*k]
  uint8_t* hx;          // ET_F32, few rows: the scales of hhi and hlo as biased exponents [places][F/32][rows]
  float* y;          // [T*k][D] expert outputs by place (ET_F32: before that, the places' products [T*k][F])
  uint32_t* arrived;  // parts of each shared tile that are done (cleared by every call)
  float* part;        // shared tiles' partial sums
};
// Bytes of the workspace of a call with up to a.T rows.
size_t experts_workspace(ExpertsArgs a);
// Bytes of the workspace of a call of exactly a.T rows, and its layout over `base`.
size_t experts_carve(ExpertsArgs& a, void* base);
hipError_t launch_experts(const ExpertsArgs& a, hipStream_t s);
// Packs the weights of n experts: src row-major [n][rows][cols] on the device,
// 16-bit; to_f16 converts bf16 values to fp16.  up == nullptr: the down
// projection (gate = wd, rows = D, cols = F).
hipError_t launch_pack_experts(const uint16_t* gate, const uint16_t* up, uint16_t* dst, int n, int rows, int cols,
                               bool to_f16, hipStream_t s);

}  // namespace hvd
