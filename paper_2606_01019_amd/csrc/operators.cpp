// C ABI of an expert layer's operators: argument checks, then the launchers of
// route.hip, experts.hip and block_norm.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "../../include/hvd.h"
#include "error.h"
#include "moe.h"

using namespace hvd;

namespace hvd {

hvd_status check_route_config(const hvd_route_config* c) {
  if (!c) return set_err(HVD_ERR_ARG, "null config");
  if (c->n_experts < 1 || c->n_experts > kMaxExperts) return set_err(HVD_ERR_ARG, "n_experts must be in [1, 512]");
  if (c->top_k < 1 || c->top_k > kMaxTopK) return set_err(HVD_ERR_ARG, "top_k must be in [1, 16]");
  if (c->score != HVD_SCORE_SOFTMAX && c->score != HVD_SCORE_SIGMOID) return set_err(HVD_ERR_ARG, "unknown score");
  if (c->n_groups < 1 || c->n_groups > kMaxGroups || c->n_experts % c->n_groups)
    return set_err(HVD_ERR_ARG, "n_groups must be in [1, 64] and divide n_experts");
  if (c->top_groups < 1 || c->top_groups > c->n_groups) return set_err(HVD_ERR_ARG, "top_groups must be in [1, n_groups]");
  if (c->top_k > c->n_experts / c->n_groups * c->top_groups)
    return set_err(HVD_ERR_ARG, "top_k must fit the experts of top_groups groups");
  if (!std::isfinite(c->scale)) return set_err(HVD_ERR_ARG, "scale must be finite");
  return HVD_OK;
}

RouteArgs route_args(const hvd_route_config& c, int rows, const void* logits, int dtype, int64_t stride,
                     const float* bias, int32_t* ids, float* weights) {
  return RouteArgs{logits, stride, dtype, rows, c.n_experts, c.top_k, c.score == HVD_SCORE_SIGMOID, c.n_groups,
                   c.top_groups, c.renorm != 0, c.scale, bias, ids, weights};
}

}  // namespace hvd

struct hvd_experts_s {
  hvd_experts_config cfg;
  ExpertsW w;
  void* base = nullptr;
  bool owned = false;
};

namespace {

bool float_type(int t) { return t == HVD_F16 || t == HVD_BF16 || t == HVD_F32; }

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

hvd_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return HVD_OK;
  return set_err(HVD_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

hvd_status check_experts_config(const hvd_experts_config* c) {
  if (!c) return set_err(HVD_ERR_ARG, "null config");
  if (c->n_experts < 1 || c->n_experts > kMaxExperts) return set_err(HVD_ERR_ARG, "n_experts must be in [1, 512]");
  if (c->d_model < 64 || c->d_model % 64 || c->d_model > (1 << 17)) return set_err(HVD_ERR_ARG, "d_model must be a positive multiple of 64, at most 131072");
  if (c->ffn_dim < 32 || c->ffn_dim % 32 || c->ffn_dim > (1 << 17)) return set_err(HVD_ERR_ARG, "ffn_dim must be a positive multiple of 32, at most 131072");
  if (c->dtype != HVD_F16 && c->dtype != HVD_BF16) return set_err(HVD_ERR_ARG, "experts' dtype must be HVD_F16 or HVD_BF16");
  return HVD_OK;
}

size_t matrix_bytes(const hvd_experts_config& c) { return (size_t)c.n_experts * c.d_model * c.ffn_dim * 2; }

hvd_status check_forward(hvd_experts e, int rows, int top_k, int x_dtype) {
  if (!e) return set_err(HVD_ERR_ARG, "null experts");
  if (rows < 0 || rows > kMaxExpertRows) return set_err(HVD_ERR_ARG, "rows must be in [0, 262144]");
  if (top_k < 1 || top_k > kMaxTopK) return set_err(HVD_ERR_ARG, "top_k must be in [1, 16]");
  if (x_dtype != e->cfg.dtype && !(x_dtype == HVD_F32 && e->cfg.dtype == HVD_F16))
    return set_err(HVD_ERR_ARG, "x must have the weights' type, or HVD_F32 with HVD_F16 weights");
  return HVD_OK;
}

}  // namespace

extern "C" hvd_status hvd_route(const hvd_route_config* cfg, int32_t rows, const void* logits, int32_t logits_dtype,
                                int64_t logits_stride, const float* bias, int32_t* ids, float* weights, void* stream) {
  if (hvd_status st = check_route_config(cfg); st != HVD_OK) return st;
  if (rows < 0 || rows > kMaxOpRows) return set_err(HVD_ERR_ARG, "rows must be in [0, 8388608]");
  if (!float_type(logits_dtype)) return set_err(HVD_ERR_ARG, "unknown logits dtype");
  if (rows == 0) return HVD_OK;
  if (!logits || !ids || !weights) return set_err(HVD_ERR_ARG, "null logits, ids or weights");
  if (logits_stride < cfg->n_experts && rows > 1) return set_err(HVD_ERR_ARG, "logits rows overlap");
  if (!aligned(logits, elem_bytes(logits_dtype)) || !aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4))
    return set_err(HVD_ERR_ARG, "a buffer is not aligned to its elements");
  return launched(launch_route(route_args(*cfg, rows, logits, logits_dtype, logits_stride, bias, ids, weights),
                               (hipStream_t)stream), "route");
}

extern "C" size_t hvd_experts_bytes(const hvd_experts_config* cfg) {
  return check_experts_config(cfg) == HVD_OK ? 3 * matrix_bytes(*cfg) : 0;
}

extern "C" hvd_status hvd_experts_load(const hvd_experts_config* cfg, const void* gate, const void* up, const void* down,
                                       void* dev_buf, size_t dev_bytes, void* stream, hvd_experts* out) {
  if (hvd_status st = check_experts_config(cfg); st != HVD_OK) return st;
  if (!gate || !up || !down || !out) return set_err(HVD_ERR_ARG, "null weights or out");
  if (!aligned(gate, 16) || !aligned(up, 16) || !aligned(down, 16) || !aligned(dev_buf, 16))
    return set_err(HVD_ERR_ARG, "weights and dev_buf must be 16-byte aligned");
  const size_t m = matrix_bytes(*cfg);
  if (dev_buf && dev_bytes < 3 * m) return set_err(HVD_ERR_ARG, "dev_buf smaller than hvd_experts_bytes");
  auto* e = new (std::nothrow) hvd_experts_s();
  if (!e) return set_err(HVD_ERR_OOM, "out of host memory");
  e->cfg = *cfg;
  e->base = dev_buf;
  if (!dev_buf) {
    if (hipMalloc(&e->base, 3 * m) != hipSuccess) {
      (void)hipGetLastError();
      delete e;
      return set_err(HVD_ERR_OOM, "hipMalloc of the experts' weights failed");
    }
    e->owned = true;
  }
  uint16_t* p = (uint16_t*)e->base;
  e->w = ExpertsW{p, p + m, cfg->n_experts, cfg->d_model, cfg->ffn_dim, cfg->dtype};
  hipStream_t s = (hipStream_t)stream;
  hipError_t err = launch_pack_experts((const uint16_t*)gate, (const uint16_t*)up, p, cfg->n_experts, cfg->ffn_dim,
                                       cfg->d_model, false, s);
  if (err == hipSuccess)
    err = launch_pack_experts((const uint16_t*)down, nullptr, p + m, cfg->n_experts, cfg->d_model, cfg->ffn_dim, false, s);
  if (err != hipSuccess) {
    hvd_experts_free(e);
    return launched(err, "packing the experts' weights");
  }
  *out = e;
  return HVD_OK;
}

extern "C" void hvd_experts_free(hvd_experts e) {
  if (!e) return;
  if (e->owned) (void)hipFree(e->base);
  delete e;
}

extern "C" size_t hvd_experts_workspace(hvd_experts e, int32_t rows, int32_t top_k, int32_t x_dtype) {
  if (check_forward(e, rows, top_k, x_dtype) != HVD_OK) return 0;
  ExpertsArgs a{};
  a.w = e->w;
  a.T = rows;
  a.k = top_k;
  a.x_type = x_dtype;
  return std::max<size_t>(experts_workspace(a), 256);  // (0 is a refusal)
}

extern "C" hvd_status hvd_experts_forward(hvd_experts e, int32_t rows, int32_t top_k, const void* x, int32_t x_dtype,
                                          int64_t x_stride, const int32_t* ids, const float* weights, void* out,
                                          int64_t out_stride, void* work, size_t work_bytes, void* stream) {
  if (hvd_status st = check_forward(e, rows, top_k, x_dtype); st != HVD_OK) return st;
  if (rows == 0) return HVD_OK;
  if (!x || !ids || !weights || !out || !work) return set_err(HVD_ERR_ARG, "null x, ids, weights, out or work");
  const size_t es = elem_bytes(x_dtype);
  if (!aligned(x, 16) || !aligned(out, 16) || !aligned(work, 16) || !aligned(ids, 4) || !aligned(weights, 4) ||
      x_stride * (int64_t)es % 16 || out_stride * (int64_t)es % 16)
    return set_err(HVD_ERR_ARG, "x, out, work and their rows must be 16-byte aligned");
  if (rows > 1 && (x_stride < e->cfg.d_model || out_stride < e->cfg.d_model))
    return set_err(HVD_ERR_ARG, "rows of x or out overlap");
  ExpertsArgs a{};
  a.w = e->w;
  a.x = x;
  a.x_stride = x_stride;
  a.x_type = x_dtype;
  a.T = rows;
  a.k = top_k;
  a.ids = ids;
  a.weights = weights;
  a.out = out;
  a.out_stride = out_stride;
  if (experts_carve(a, work) > work_bytes) return set_err(HVD_ERR_ARG, "work smaller than hvd_experts_workspace");
  return launched(launch_experts(a, (hipStream_t)stream), "experts");
}

extern "C" hvd_status hvd_block_norm(const hvd_block_norm_args* g, int32_t rows, int32_t dim, void* stream) {
  if (!g) return set_err(HVD_ERR_ARG, "null arguments");
  if (rows < 0 || rows > kMaxOpRows) return set_err(HVD_ERR_ARG, "rows must be in [0, 8388608]");
  if (dim < 1 || dim > kMaxNormDim) return set_err(HVD_ERR_ARG, "dim must be in [1, 16384]");
  if (rows == 0) return HVD_OK;
  if (!g->x || (!g->x_out && !g->h)) return set_err(HVD_ERR_ARG, "null x, or neither x_out nor h");
  if ((g->h != nullptr) != (g->gain != nullptr)) return set_err(HVD_ERR_ARG, "h and gain go together");
  if (!g->y && (g->gate || g->post_gain)) return set_err(HVD_ERR_ARG, "gate and post_gain belong to a y");
  if (!(g->eps >= 0.f)) return set_err(HVD_ERR_ARG, "eps must be >= 0");
  struct {
    const void* p;
    int64_t stride;
    int type;
  } bufs[] = {{g->x, g->x_stride, g->x_dtype}, {g->x_out, g->x_out_stride, g->x_dtype}, {g->y, g->y_stride, g->y_dtype},
              {g->h, g->h_stride, g->h_dtype}};
  for (const auto& b : bufs) {
    if (!b.p) continue;
    if (!float_type(b.type)) return set_err(HVD_ERR_ARG, "unknown dtype");
    if (!aligned(b.p, elem_bytes(b.type))) return set_err(HVD_ERR_ARG, "a buffer is not aligned to its elements");
    if (rows > 1 && b.stride < dim) return set_err(HVD_ERR_ARG, "rows overlap");
  }
  if (g->x_out == g->x && g->x_out_stride != g->x_stride && rows > 1)
    return set_err(HVD_ERR_ARG, "x_out in place of x needs x's stride");
  if (g->gate) {
    if (!float_type(g->gate_dtype) || !aligned(g->gate, elem_bytes(g->gate_dtype))) return set_err(HVD_ERR_ARG, "bad gate type or alignment");
    if ((g->gate_col_stride != 0 && g->gate_col_stride != 1) || g->gate_row_stride < 0)
      return set_err(HVD_ERR_ARG, "the gate's column stride must be 0 or 1, its row stride >= 0");
  }
  if (!aligned(g->gain, 4) || !aligned(g->post_gain, 4)) return set_err(HVD_ERR_ARG, "gains must be 4-byte aligned");
  BlockNormArgs a{};
  a.x = g->x;
  a.x_stride = g->x_stride;
  a.x_type = g->x_dtype;
  a.y = g->y;
  a.y_stride = g->y_stride;
  a.y_type = g->y_dtype;
  a.gate = g->gate;
  a.gate_row = g->gate_row_stride;
  a.gate_col = g->gate_col_stride;
  a.gate_type = g->gate_dtype;
  a.post_gain = g->post_gain;
  a.gain = g->gain;
  a.scale = g->scale;
  a.eps = g->eps;
  a.x_out = g->x_out;
  a.x_out_stride = g->x_out_stride;
  a.h = g->h;
  a.h_stride = g->h_stride;
  a.h_type = g->h_dtype;
  a.rows = rows;
  a.D = dim;
  return launched(launch_block_norm(a, (hipStream_t)stream), "block norm");
}
