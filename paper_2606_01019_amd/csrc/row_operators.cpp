// C ABI of the operators on a step's rows: argument checks, then the launchers
// of append_kv.hip, attend.hip and adjust_logits.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <cmath>
#include <string>
#include <utility>

#include "../../include/hvd.h"
#include "error.h"
#include "rows.h"

using namespace hvd;

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool float_type(int t) { return t == HVD_F16 || t == HVD_BF16 || t == HVD_F32; }

hvd_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return HVD_OK;
  return set_err(HVD_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

hvd_status check_batch(const hvd_row_batch* b, int rows, int most, bool keys, RowBatch& out) {
  if (!b) return set_err(HVD_ERR_ARG, "null batch");
  if (rows < 0 || rows > most) return set_err(HVD_ERR_ARG, "rows must be in [0, " + std::to_string(most) + "]");
  if (b->n_seqs < 0 || b->n_seqs > kMaxSeqs) return set_err(HVD_ERR_ARG, "n_seqs must be in [0, 4096]");
  if (!b->starts) return set_err(HVD_ERR_ARG, "null starts");
  if (!aligned(b->starts, 4) || !aligned(b->tree, 8)) return set_err(HVD_ERR_ARG, "starts or tree is not aligned to its elements");
  if (keys) {
    if (b->max_pages < 0 || b->max_pages > kMaxKeys) return set_err(HVD_ERR_ARG, "bad max_pages");
    if (b->n_seqs > 0 && (!b->lengths || (!b->pages && b->max_pages > 0))) return set_err(HVD_ERR_ARG, "null lengths or pages");
    if (b->n_seqs > 1 && b->pages_stride < b->max_pages) return set_err(HVD_ERR_ARG, "pages of two sequences overlap");
    if (!aligned(b->lengths, 4) || !aligned(b->pages, 4)) return set_err(HVD_ERR_ARG, "lengths or pages is not aligned to its elements");
  }
  out = RowBatch{b->starts, b->lengths, b->pages, b->tree, b->pages_stride, b->n_seqs, rows, keys ? b->max_pages : 0};
  return HVD_OK;
}

// Dimensions of a tensor beside its contiguous one: (stride, size).
using Dims = std::array<std::pair<int64_t, int64_t>, 3>;

// Whether runs of `width` elements at these strides are apart from one another.
bool apart(Dims d, int64_t width) {
  std::sort(d.begin(), d.end());
  int64_t extent = width;
  for (const auto& [stride, n] : d) {
    if (n <= 1) continue;
    if (stride < extent || stride > ((int64_t)1 << 46) / n) return false;
    extent += stride * (n - 1);
  }
  return true;
}
// The same for pages, heads and tokens of one half of the cache.
bool apart(int64_t page, int64_t head, int64_t tok, const hvd_paged_kv& c) {
  return apart({{{page, c.n_pages}, {head, c.n_heads}, {tok, c.page_size}}}, c.head_dim);
}

// A dimension of two tensors.
struct Dim2 {
  int64_t a, b, n;
};
// Whether runs of `width` elements at the places of d[0 .. left) have an element in
// common, b's `delta` elements from a's; those of a are apart, the longest stride
// first.  Strides that differ where the extents meet count as a place in common.
bool meet(const Dim2* d, int left, __int128 delta, int64_t width) {
  __int128 ea = width, eb = width;
  for (int i = 0; i < left; ++i) {
    ea += (__int128)d[i].a * (d[i].n - 1);
    eb += (__int128)d[i].b * (d[i].n - 1);
  }
  if (delta >= ea || delta <= -eb) return false;
  if (left == 0 || d->a != d->b) return true;
  // what is left once the places in this dimension are i apart; few i come near
  const __int128 last = (__int128)d->a * (d->n - 1), ia = ea - last, ib = eb - last;
  for (__int128 i = -(d->n - 1), near = (delta - ia) / d->a - 1; (i = std::max(i, near)) <= d->n - 1; ++i) {
    if (delta - i * d->a <= -ib) return false;
    if (meet(d + 1, left - 1, delta - i * d->a, width)) return true;
  }
  return false;
}
// Whether two tensors of the same sizes have a place in common; a's are apart.
bool meet(const void* pa, const Dims& a, const void* pb, const Dims& b, int64_t width, int64_t elem) {
  Dim2 d[3];
  int n = 0;
  for (int i = 0; i < 3; ++i)
    if (a[i].second > 1) d[n++] = Dim2{a[i].first, b[i].first, a[i].second};
  std::sort(d, d + n, [](const Dim2& x, const Dim2& y) { return x.a > y.a; });
  return meet(d, n, ((int64_t)(uintptr_t)pb - (int64_t)(uintptr_t)pa) / elem, width);
}
// The same places, element by element.
bool in_place(const void* pa, const Dims& a, const void* pb, const Dims& b) {
  bool same = pa == pb;
  for (int i = 0; i < 3; ++i) same = same && (a[i].second <= 1 || a[i].first == b[i].first);
  return same;
}

hvd_status check_kv(const hvd_paged_kv* c, const hvd_row_batch* b, CacheView& k, CacheView& v, int& shift) {
  if (!c) return set_err(HVD_ERR_ARG, "null cache");
  if (c->dtype != HVD_F16 && c->dtype != HVD_BF16) return set_err(HVD_ERR_ARG, "the cache's dtype must be HVD_F16 or HVD_BF16");
  if (c->n_pages < 0) return set_err(HVD_ERR_ARG, "n_pages must not be negative");
  if (c->n_heads < 1 || c->n_heads > kMaxRowHeads) return set_err(HVD_ERR_ARG, "n_heads must be in [1, 256]");
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
    return set_err(HVD_ERR_ARG, "page_size must be a power of two from 16 to 1024");
  if (c->head_dim < 8 || c->head_dim > kMaxRowDim || c->head_dim % 8)
    return set_err(HVD_ERR_ARG, "head_dim must be a multiple of 8 from 8 to 256");
  if ((int64_t)b->max_pages * c->page_size > kMaxKeys) return set_err(HVD_ERR_ARG, "max_pages * page_size must be at most 2^29");
  if (c->n_pages > 0 && (!c->k || !c->v)) return set_err(HVD_ERR_ARG, "null k or v cache");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return set_err(HVD_ERR_ARG, "the cache must be 16-byte aligned");
  for (int64_t s : {c->k_page_stride, c->k_head_stride, c->k_token_stride, c->v_page_stride, c->v_head_stride, c->v_token_stride})
    if (s < 0 || s % 8) return set_err(HVD_ERR_ARG, "the cache's strides must be multiples of 8");
  if (c->k_token_stride > kMaxTokStride || c->v_token_stride > kMaxTokStride)
    return set_err(HVD_ERR_ARG, "the cache's token strides must be at most 2^26");
  if (!apart(c->k_page_stride, c->k_head_stride, c->k_token_stride, *c) || !apart(c->v_page_stride, c->v_head_stride, c->v_token_stride, *c))
    return set_err(HVD_ERR_ARG, "places of the cache overlap");
  k = CacheView{c->k, c->k_page_stride, c->k_head_stride, c->k_token_stride};
  v = CacheView{c->v, c->v_page_stride, c->v_head_stride, c->v_token_stride};
  shift = __builtin_ctz(c->page_size);
  return HVD_OK;
}

hvd_status check_attend(const hvd_row_batch* b, const hvd_paged_kv* c, int q_heads, int rows, AttendArgs& a) {
  if (hvd_status st = check_batch(b, rows, kMaxStepRows, true, a.b); st != HVD_OK) return st;
  if (hvd_status st = check_kv(c, b, a.k, a.v, a.page_shift); st != HVD_OK) return st;
  if (q_heads < 1 || q_heads > kMaxRowHeads || q_heads % c->n_heads)
    return set_err(HVD_ERR_ARG, "q_heads must be a multiple of n_heads, at most 256");
  a.n_pages = c->n_pages;
  a.H = c->n_heads;
  a.Hq = q_heads;
  a.D = c->head_dim;
  a.type = c->dtype;
  return HVD_OK;
}

hvd_status check_adjust(const hvd_row_batch* b, const hvd_adjust_args* g, int rows, AdjustArgs& a) {
  if (hvd_status st = check_batch(b, rows, kMaxAdjustRows, false, a.b); st != HVD_OK) return st;
  if (!g) return set_err(HVD_ERR_ARG, "null arguments");
  if (g->vocab < 1 || g->vocab > kMaxVocab) return set_err(HVD_ERR_ARG, "vocab must be in [1, 16777216]");
  if (!float_type(g->dtype)) return set_err(HVD_ERR_ARG, "unknown dtype");
  a.V = g->vocab;
  a.type = g->dtype;
  return HVD_OK;
}

}  // namespace

extern "C" hvd_status hvd_append_kv(const hvd_row_batch* batch, const hvd_paged_kv* kv, const hvd_append_args* g, int32_t rows,
                                    void* stream) {
  AppendArgs a{};
  if (hvd_status st = check_batch(batch, rows, kMaxStepRows, true, a.b); st != HVD_OK) return st;
  if (hvd_status st = check_kv(kv, batch, a.k, a.v, a.page_shift); st != HVD_OK) return st;
  if (!g) return set_err(HVD_ERR_ARG, "null arguments");
  if (!float_type(g->dtype)) return set_err(HVD_ERR_ARG, "unknown dtype");
  if (g->rot < 0 || g->rot > kv->head_dim || g->rot % 2) return set_err(HVD_ERR_ARG, "rot must be even, in [0, head_dim]");
  if (g->rot > 0 && !g->freqs) return set_err(HVD_ERR_ARG, "null freqs");
  if ((g->q != nullptr) != (g->q_out != nullptr) && rows > 0) return set_err(HVD_ERR_ARG, "q and q_out go together");
  if (g->q && (g->q_heads < 1 || g->q_heads > kMaxRowHeads)) return set_err(HVD_ERR_ARG, "q_heads must be in [1, 256]");
  if (rows == 0) return HVD_OK;
  if (!g->k || !g->v) return set_err(HVD_ERR_ARG, "null k or v");
  const size_t es = elem_bytes(g->dtype);
  if (!aligned(g->k, es) || !aligned(g->v, es) || !aligned(g->q, es) || !aligned(g->freqs, 8) || !aligned(g->positions, 4))
    return set_err(HVD_ERR_ARG, "a buffer is not aligned to its elements");
  if (!aligned(g->q_out, 16)) return set_err(HVD_ERR_ARG, "q_out must be 16-byte aligned");
  for (int64_t s : {g->k_row_stride, g->k_head_stride, g->v_row_stride, g->v_head_stride, g->q_row_stride, g->q_head_stride})
    if (s < 0) return set_err(HVD_ERR_ARG, "strides must not be negative");
  const auto places = [&](const CacheView& c) { return Dims{{{c.page, kv->n_pages}, {c.head, kv->n_heads}, {c.tok, kv->page_size}}}; };
  if (kv->n_pages > 0 && meet(kv->k, places(a.k), kv->v, places(a.v), kv->head_dim, 2))
    return set_err(HVD_ERR_ARG, "keys and values share memory");
  a.n_pages = kv->n_pages;
  a.H = kv->n_heads;
  a.Hq = g->q ? g->q_heads : 0;
  a.D = kv->head_dim;
  a.in_type = g->dtype;
  a.cache_type = kv->dtype;
  a.xk = g->k;
  a.k_row = g->k_row_stride;
  a.k_head = g->k_head_stride;
  a.xv = g->v;
  a.v_row = g->v_row_stride;
  a.v_head = g->v_head_stride;
  a.xq = g->q;
  a.q_row = g->q_row_stride;
  a.q_head = g->q_head_stride;
  a.q_out = g->q_out;
  a.freqs = g->freqs;
  a.positions = g->positions;
  a.rot = g->rot;
  a.interleaved = g->interleaved != 0;
  return launched(launch_append_kv(a, (hipStream_t)stream), "append");
}

extern "C" size_t hvd_attend_workspace(const hvd_row_batch* batch, const hvd_paged_kv* kv, int32_t q_heads, int32_t rows) {
  AttendArgs a{};
  if (check_attend(batch, kv, q_heads, rows, a) != HVD_OK) return 0;
  return std::max<size_t>(rows ? attend_workspace(a) : 0, 16);  // (0 is a refusal)
}

extern "C" hvd_status hvd_attend(const hvd_row_batch* batch, const hvd_paged_kv* kv, const hvd_attend_args* g, int32_t rows,
                                 void* work, size_t work_bytes, void* stream) {
  AttendArgs a{};
  if (!g) return set_err(HVD_ERR_ARG, "null arguments");
  if (hvd_status st = check_attend(batch, kv, g->q_heads, rows, a); st != HVD_OK) return st;
  // (its factor to base-2 exponents has to be finite too)
  if (!(std::fabs(g->scale) <= 0x1p127f)) return set_err(HVD_ERR_ARG, "scale must be in [-2^127, 2^127]");
  if (!(g->cap >= 0.f) || !std::isfinite(g->cap)) return set_err(HVD_ERR_ARG, "cap must be finite and >= 0");
  if (g->window < 0) return set_err(HVD_ERR_ARG, "window must be >= 0");
  if (rows == 0) return HVD_OK;
  if (!g->q || !g->out) return set_err(HVD_ERR_ARG, "null q or out");
  if (!aligned(g->q, 16) || !aligned(g->out, 16)) return set_err(HVD_ERR_ARG, "q and out must be 16-byte aligned");
  for (int64_t s : {g->q_row_stride, g->q_head_stride, g->out_row_stride, g->out_head_stride})
    if (s < 0 || s % 8) return set_err(HVD_ERR_ARG, "strides of q and out must be multiples of 8");
  const Dims to = {{{g->out_row_stride, rows}, {g->out_head_stride, g->q_heads}, {0, 1}}};
  if (!apart(to, kv->head_dim))
    return set_err(HVD_ERR_ARG, "rows or heads of out overlap");
  const Dims from = {{{g->q_row_stride, rows}, {g->q_head_stride, g->q_heads}, {0, 1}}};
  if (!in_place(g->out, to, g->q, from) && meet(g->out, to, g->q, from, kv->head_dim, 2))
    return set_err(HVD_ERR_ARG, "out shares memory with q otherwise than in its place");
  if (!aligned(g->slopes, 4) || !aligned(g->first, 4) || !aligned(g->prefix, 4))
    return set_err(HVD_ERR_ARG, "a buffer is not aligned to its elements");
  a.q = g->q;
  a.q_row = g->q_row_stride;
  a.q_head = g->q_head_stride;
  a.out = g->out;
  a.out_row = g->out_row_stride;
  a.out_head = g->out_head_stride;
  a.slopes = g->slopes;
  a.first = g->first;
  a.prefix = g->prefix;
  a.scale = g->scale;
  a.cap = g->cap;
  a.window = g->window;
  if (const size_t need = attend_workspace(a)) {
    if (!work || !aligned(work, 16)) return set_err(HVD_ERR_ARG, "work must be 16-byte aligned and not null");
    if (work_bytes < need) return set_err(HVD_ERR_ARG, "work smaller than hvd_attend_workspace");
    a.part = (float*)work;
  }
  return launched(launch_attend(a, (hipStream_t)stream), "attend");
}

extern "C" size_t hvd_adjust_workspace(const hvd_row_batch* batch, const hvd_adjust_args* g, int32_t rows) {
  AdjustArgs a{};
  if (check_adjust(batch, g, rows, a) != HVD_OK) return 0;
  return std::max<size_t>(rows ? adjust_workspace(a) : 0, 16);
}

extern "C" hvd_status hvd_adjust_logits(const hvd_row_batch* batch, const hvd_adjust_args* g, int32_t rows, void* work,
                                        size_t work_bytes, void* stream) {
  AdjustArgs a{};
  if (hvd_status st = check_adjust(batch, g, rows, a); st != HVD_OK) return st;
  if (g->max_history < 0 || g->max_history > kMaxHistory) return set_err(HVD_ERR_ARG, "max_history must be in [0, 983039]");
  if (g->n_bias < 0 || g->n_bias > kMaxBias) return set_err(HVD_ERR_ARG, "n_bias must be in [0, 2046]");
  const int S = a.b.S;
  if (g->history && S > 0 && !g->history_lengths) return set_err(HVD_ERR_ARG, "history needs history_lengths");
  if (g->history && S > 1 && g->history_stride < g->max_history) return set_err(HVD_ERR_ARG, "histories overlap");
  if ((g->bias_ids != nullptr) != (g->bias != nullptr)) return set_err(HVD_ERR_ARG, "bias_ids and bias go together");
  if (g->bias && S > 1 && (g->bias_ids_stride < g->n_bias || g->bias_stride < g->n_bias))
    return set_err(HVD_ERR_ARG, "biases of two sequences overlap");
  if (g->allowed && g->allowed_stride != 0 && g->allowed_stride < (g->vocab + 31) / 32 && rows > 1)
    return set_err(HVD_ERR_ARG, "masks of two rows overlap");
  if (rows == 0) return HVD_OK;
  if (!g->logits || (!g->out && !g->best)) return set_err(HVD_ERR_ARG, "null logits, or neither out nor best");
  const size_t es = elem_bytes(g->dtype);
  for (const void* p : {(const void*)g->best, (const void*)g->tokens, (const void*)g->history, (const void*)g->history_lengths,
                        (const void*)g->prompt_lengths, (const void*)g->repetition, (const void*)g->frequency,
                        (const void*)g->presence, (const void*)g->bias_ids, (const void*)g->bias, (const void*)g->allowed})
    if (!aligned(p, 4)) return set_err(HVD_ERR_ARG, "a buffer is not aligned to its elements");
  if (!aligned(g->logits, es) || !aligned(g->out, es)) return set_err(HVD_ERR_ARG, "logits or out is not aligned to its elements");
  if (rows > 1 && (g->logits_stride < g->vocab || (g->out && g->out_stride < g->vocab)))
    return set_err(HVD_ERR_ARG, "rows overlap");
  const Dims to = {{{g->out_stride, rows}, {0, 1}, {0, 1}}}, from = {{{g->logits_stride, rows}, {0, 1}, {0, 1}}};
  if (g->out && !in_place(g->out, to, g->logits, from) && meet(g->out, to, g->logits, from, g->vocab, (int64_t)es))
    return set_err(HVD_ERR_ARG, "out shares memory with logits otherwise than in their place");
  a.logits = g->logits;
  a.logits_stride = g->logits_stride;
  a.out = g->out;
  a.out_stride = g->out_stride;
  a.best = g->best;
  a.tokens = g->tokens;
  a.history = g->max_history > 0 ? g->history : nullptr;
  a.history_stride = g->history_stride;
  a.max_history = g->max_history;
  a.history_lengths = g->history_lengths;
  a.prompt_lengths = g->prompt_lengths;
  a.repetition = g->repetition;
  a.frequency = g->frequency;
  a.presence = g->presence;
  a.bias_ids = g->bias_ids;
  a.bias = g->bias;
  a.bias_ids_stride = g->bias_ids_stride;
  a.bias_stride = g->bias_stride;
  a.n_bias = g->bias ? g->n_bias : 0;
  a.allowed = g->allowed;
  a.allowed_stride = g->allowed_stride;
  if (a.best) {
    if (!work || !aligned(work, 16)) return set_err(HVD_ERR_ARG, "work must be 16-byte aligned and not null");
    if (work_bytes < adjust_workspace(a)) return set_err(HVD_ERR_ARG, "work smaller than hvd_adjust_workspace");
    a.part = (uint64_t*)work;
  }
  return launched(launch_adjust_logits(a, (hipStream_t)stream), "adjust logits");
}
