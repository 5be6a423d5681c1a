// C ABI of the operators around the decoder where it learns and answers:
// argument checks (all before anything is enqueued), workspace layouts, and the
// launches.  Lengths and the optimizer's tensors travel in the kernels' arguments,
// so no call copies anything to the device and a captured call keeps them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/svl.h"
#include "learn_ops.h"
#include "lm_loss.h"
#include "svl_internal.h"

namespace svl {
namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round256(int64_t x) { return (x + 255) & ~int64_t(255); }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

svl_status err(svl_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
svl_status err(svl_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return set_error(st, buf);
}

svl_status hip_status(hipError_t e, const char* where) {
  if (e == hipSuccess) return SVL_OK;
  return err(SVL_E_HIP, "%s: %s", where, hipGetErrorString(e));
}

template <class F>
hipError_t timed_launch(int cls, hipStream_t st, const F& f) {
  return timed_call(cls, st, [](const void* p) { return (*static_cast<const F*>(p))(); }, &f);
}

// ------------------------------------------------------------------ checks
bool known_type(int32_t t) { return t == SVL_TYPE_F32 || t == SVL_TYPE_BF16 || t == SVL_TYPE_F16; }

constexpr int64_t MAX_ROWS = (1 << 24) - 1;

svl_status check_row_count(int32_t rows) {
  if (rows < 0 || rows > MAX_ROWS) return err(SVL_E_SHAPE, "rows = %d outside [0, 2^24)", rows);
  return SVL_OK;
}

svl_status check_pointer(const void* p, const char* what, uintptr_t align = 16) {
  if (!p) return err(SVL_E_NULL, "%s is NULL", what);
  if (!aligned(p, align)) return err(SVL_E_ALIGN, "%s not %d-byte aligned", what, (int)align);
  return SVL_OK;
}

// Rows of `width` values, `ld` apart.
svl_status check_array(const void* p, int64_t ld, int64_t width, const char* what, int64_t most = 1 << 23) {
  const svl_status s = check_pointer(p, what);
  if (s != SVL_OK) return s;
  if (ld < width || ld % 8 || ld > most)
    return err(SVL_E_SHAPE, "row stride %lld of %s: at least %lld, at most %lld and a multiple of 8", (long long)ld,
               what, (long long)width, (long long)most);
  return SVL_OK;
}

svl_status check_optional(const void* p, int64_t ld, int64_t width, const char* what, int64_t most = 1 << 23) {
  return p ? check_array(p, ld, width, what, most) : SVL_OK;
}

svl_status check_flag(int32_t v, const char* what) {
  return v == 0 || v == 1 ? SVL_OK : err(SVL_E_VALUE, "%s must be 0 or 1, not %d", what, v);
}

svl_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return SVL_OK;
  const svl_status s = check_pointer(ws, "workspace");
  if (s != SVL_OK) return s;
  if (have < need) return err(SVL_E_WORKSPACE, "workspace %zu bytes < %zu needed", have, need);
  return SVL_OK;
}

// Regions of a workspace, each from a multiple of 256 bytes on.
struct Layout {
  char* base;
  int64_t at = 0;
  template <class T>
  T* take(int64_t n) {
    T* p = reinterpret_cast<T*>(base + at);
    at += round256(n * (int64_t)sizeof(T));
    return p;
  }
};

#define SVL_TRY(call)                        \
  do {                                       \
    const svl_status svl_try_ = (call);      \
    if (svl_try_ != SVL_OK) return svl_try_; \
  } while (0)

// ------------------------------------------------------------------ embedding
svl_status check_embedding(const svl_embedding* e) {
  if (!e) return err(SVL_E_NULL, "embedding description is NULL");
  if (e->width <= 0 || e->width % 8 || e->width > 65536)
    return err(SVL_E_SHAPE, "width = %d must be a multiple of 8 in [8, 65536]", e->width);
  if (e->vocab <= 0 || e->vocab > MAX_ROWS) return err(SVL_E_SHAPE, "vocab = %d outside [1, 2^24)", e->vocab);
  if (!known_type(e->table_type) || !known_type(e->row_type))
    return err(SVL_E_DTYPE, "unknown type (table %d, rows %d)", e->table_type, e->row_type);
  if (!std::isfinite(e->scale)) return err(SVL_E_VALUE, "scale must be finite");
  return SVL_OK;
}

EmbedArgs embed_args(const svl_embedding& e, int32_t rows, const int32_t* tokens) {
  EmbedArgs a{};
  a.tokens = tokens;
  a.rows = rows;
  a.width = e.width;
  a.vocab = e.vocab;
  a.table_type = e.table_type;
  a.row_type = e.row_type;
  a.scale = e.scale;
  return a;
}

// A run of this many rows is summed in one go; with more rows there are pieces.
constexpr int32_t EMBED_PIECES_FROM = 256;

int64_t embed_layout(const svl_embedding& e, int32_t rows, char* base, SortArgs* s, EmbedArgs* a) {
  Layout l{base};
  s->rows = rows;
  s->vocab = e.vocab;
  s->passes = 0;
  for (uint32_t v = (uint32_t)e.vocab; v; v >>= 8) ++s->passes;
  s->units = (int32_t)cdiv(rows, SORT_UNIT);
  for (int i = 0; i < 2; ++i) {
    s->key[i] = l.take<uint32_t>(rows);
    s->at[i] = l.take<uint32_t>(rows);
  }
  a->run = l.take<int32_t>((int64_t)e.vocab + 1);
  if (rows > SORT_ALONE) s->count = l.take<uint32_t>(256 * (int64_t)s->units);
  if (rows > EMBED_PIECES_FROM) a->sum32 = l.take<float>((int64_t)(rows / 32) * e.width);
  if (rows >= 1024) a->sum1024 = l.take<float>((int64_t)(rows / 1024) * e.width);
  a->key = s->key[(s->passes - 1) & 1];
  a->at = s->at[(s->passes - 1) & 1];
  return l.at;
}

// ------------------------------------------------------------------ norm
svl_status check_norm(const svl_norm* n) {
  if (!n) return err(SVL_E_NULL, "norm description is NULL");
  if (n->width <= 0 || n->width % 8 || n->width > SVL_NORM_MAX_WIDTH)
    return err(SVL_E_SHAPE, "width = %d must be a multiple of 8 in [8, %d]", n->width, SVL_NORM_MAX_WIDTH);
  if (n->kind != SVL_NORM_RMS && n->kind != SVL_NORM_LAYER) return err(SVL_E_VALUE, "unknown norm kind %d", n->kind);
  if (!known_type(n->x_type) || !known_type(n->y_type) || !known_type(n->gain_type))
    return err(SVL_E_DTYPE, "unknown type (x %d, y %d, gain %d)", n->x_type, n->y_type, n->gain_type);
  if (!(n->eps >= 0.f) || !std::isfinite(n->eps)) return err(SVL_E_VALUE, "eps must be finite and >= 0");
  return SVL_OK;
}

RowNormArgs norm_args(const svl_norm& n, int32_t rows, const void* x, int64_t ldx, const void* gain) {
  RowNormArgs a{};
  a.x = x;
  a.ldx = ldx;
  a.gain = gain;
  a.rows = rows;
  a.width = n.width;
  a.x_type = n.x_type;
  a.y_type = n.y_type;
  a.gain_type = n.gain_type;
  a.layer = n.kind == SVL_NORM_LAYER;
  a.eps = n.eps;
  return a;
}

int64_t norm_bytes(const svl_norm& n, int32_t rows) {
  return round256((int64_t)std::min(std::max(rows, 1), NORM_PIECES) * 2 * n.width * 4);
}

// ------------------------------------------------------------------ language-model loss
constexpr int64_t LM_MAX_LD = 1 << 21;    // a tile's rows span less than 2 GiB

svl_status check_head(const svl_lm_head* h) {
  if (!h) return err(SVL_E_NULL, "head description is NULL");
  if (h->d_model <= 0 || h->d_model % 64 || h->d_model > 65536)
    return err(SVL_E_SHAPE, "d_model = %d must be a multiple of 64 in [64, 65536]", h->d_model);
  if (h->vocab <= 0 || h->vocab > (1 << 20)) return err(SVL_E_SHAPE, "vocab = %d outside [1, 2^20]", h->vocab);
  if (h->compute != SVL_COMPUTE_F16 && h->compute != SVL_COMPUTE_BF16)
    return err(SVL_E_DTYPE, "unknown compute type %d", h->compute);
  return SVL_OK;
}

// Rows of a pass: as many as 1 GiB of exponentials hold, at least 1024.  A pass more costs the
// float32 sums of the head's gradient once in and out (32000 x 4096: 1 GB, beside 6 TFLOP of
// 8192 rows).
int32_t lm_chunk(int32_t rows, int64_t vp) {
  const int64_t fit = std::max<int64_t>(1024, ((int64_t)1 << 29) / vp / LM_TILE * LM_TILE);
  return (int32_t)std::min<int64_t>(fit, cdiv(std::max(rows, 1), LM_TILE) * LM_TILE);
}

int64_t lm_layout(const svl_lm_head& h, int32_t rows, bool want_x, bool want_w, char* base, LmArgs* a) {
  Layout l{base};
  a->rows = rows;
  a->d = h.d_model;
  a->vocab = h.vocab;
  a->vp = (int32_t)(cdiv(h.vocab, LM_TILE) * LM_TILE);
  a->chunk = lm_chunk(rows, a->vp);
  a->head = l.take<LmHead>(1);
  a->row_of = l.take<int32_t>(rows);
  a->label = l.take<int32_t>(rows);
  a->weight = l.take<float>(rows);
  a->xc = l.take<uint16_t>(cdiv(rows, LM_ROWS) * LM_ROWS * h.d_model);
  a->label_logit = l.take<float>(a->chunk);
  a->total = l.take<float2>(a->chunk);
  const int64_t across = a->vp / LM_TILE;
  a->slab = rows <= LM_FEW || across * (a->chunk / LM_TILE) <= LM_SMALL ? 64 : LM_SLAB;
  // room for the small slabs of fewer rows too, so that a workspace serves any call of at most its rows
  const int64_t small = std::min<int64_t>(a->chunk, LM_TILE * std::max<int64_t>(1, LM_SMALL / across));
  a->stats = l.take<float2>(std::max((int64_t)a->chunk * (a->vp / a->slab), small * (a->vp / 64)));
  if (want_x || want_w) {
    a->e = l.take<uint16_t>((int64_t)a->chunk * a->vp);
    a->parts = l.take<float>(std::max(want_x ? lm_parts(*a, LM_GRAD_X) : 0, want_w ? lm_parts(*a, LM_GRAD_W) : 0) *
                             LM_TILE * LM_TILE);
  }
  if (want_w && a->chunk < rows) a->sum_w = l.take<float>((int64_t)h.vocab * h.d_model);
  return l.at;
}

// ------------------------------------------------------------------ optimizer
svl_status check_adamw(const svl_adamw* a) {
  if (!a) return err(SVL_E_NULL, "optimizer description is NULL");
  if (!std::isfinite(a->lr)) return err(SVL_E_VALUE, "lr must be finite");
  if (!(a->beta1 >= 0. && a->beta1 < 1.) || !(a->beta2 >= 0. && a->beta2 < 1.))
    return err(SVL_E_VALUE, "betas must be in [0, 1)");
  if (!(a->eps >= 0.) || !std::isfinite(a->eps)) return err(SVL_E_VALUE, "eps must be finite and >= 0");
  if (!(a->weight_decay >= 0.) || !std::isfinite(a->weight_decay))
    return err(SVL_E_VALUE, "weight_decay must be finite and >= 0");
  if (a->state_bits != 32 && a->state_bits != 8) return err(SVL_E_DTYPE, "state_bits must be 32 or 8, not %d", a->state_bits);
  return SVL_OK;
}

svl_status check_tensor(const svl_adamw_tensor& t, int32_t i, int32_t bits) {
  if (t.n < 0 || t.n > ((int64_t)1 << 40)) return err(SVL_E_SHAPE, "tensor %d has n = %lld", i, (long long)t.n);
  if (!known_type(t.param_type) || !known_type(t.grad_type))
    return err(SVL_E_DTYPE, "tensor %d: unknown type (param %d, grad %d)", i, t.param_type, t.grad_type);
  if (t.n == 0) return SVL_OK;
  const struct { const void* p; const char* what; } all[] = {
      {t.param, "param"}, {t.grad, "grad"}, {t.m, "m"}, {t.v, "v"}};
  for (const auto& x : all) {
    if (!x.p) return err(SVL_E_NULL, "%s of tensor %d is NULL", x.what, i);
    if (!aligned(x.p, 16)) return err(SVL_E_ALIGN, "%s of tensor %d not 16-byte aligned", x.what, i);
  }
  if (!aligned(t.master, 16)) return err(SVL_E_ALIGN, "master of tensor %d not 16-byte aligned", i);
  if (bits == 8) {
    if (!t.m_scale || !t.v_scale) return err(SVL_E_NULL, "a scale of tensor %d is NULL", i);
    if (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))
      return err(SVL_E_ALIGN, "a scale of tensor %d not 4-byte aligned", i);
  }
  return SVL_OK;
}

}  // namespace
}  // namespace svl

using namespace svl;

extern "C" {

svl_status svl_embed(const svl_embedding* emb, int32_t rows, const int32_t* tokens, const void* table,
                     int64_t ld_table, void* out, int64_t ld_out, void* stream) {
  SVL_TRY(check_embedding(emb));
  SVL_TRY(check_row_count(rows));
  if (rows == 0) return SVL_OK;
  SVL_TRY(check_pointer(tokens, "tokens", 4));
  SVL_TRY(check_array(table, ld_table, emb->width, "table"));
  SVL_TRY(check_array(out, ld_out, emb->width, "out"));
  EmbedArgs a = embed_args(*emb, rows, tokens);
  a.table = table; a.ldt = ld_table;
  a.out = out; a.ldr = ld_out;
  const hipStream_t st = (hipStream_t)stream;
  return hip_status(timed_launch(K_GATHER, st, [&] { return launch_embed(a, st); }), "embedding");
}

size_t svl_embed_workspace_bytes(const svl_embedding* emb, int32_t rows) {
  if (check_embedding(emb) != SVL_OK || check_row_count(rows) != SVL_OK) return 0;
  SortArgs s{};
  EmbedArgs a{};
  return (size_t)std::max<int64_t>(256, embed_layout(*emb, rows, nullptr, &s, &a));
}

svl_status svl_embed_backward(const svl_embedding* emb, int32_t rows, const int32_t* tokens,
                              const void* grad_rows, int64_t ld_grad_rows, void* grad_table,
                              int64_t ld_grad_table, int32_t accumulate, void* ws, size_t ws_bytes,
                              void* stream) {
  SVL_TRY(check_embedding(emb));
  SVL_TRY(check_row_count(rows));
  SVL_TRY(check_flag(accumulate, "accumulate"));
  SVL_TRY(check_array(grad_table, ld_grad_table, emb->width, "grad_table"));
  if (rows == 0 && accumulate) return SVL_OK;
  if (rows > 0) {
    SVL_TRY(check_pointer(tokens, "tokens", 4));
    SVL_TRY(check_array(grad_rows, ld_grad_rows, emb->width, "grad_rows"));
  }
  SVL_TRY(check_workspace(ws, ws_bytes, svl_embed_workspace_bytes(emb, rows)));
  EmbedArgs a = embed_args(*emb, rows, tokens);
  SortArgs s{};
  embed_layout(*emb, rows, static_cast<char*>(ws), &s, &a);
  s.tokens = tokens;
  a.grad_rows = grad_rows; a.ldr = ld_grad_rows;
  a.out = grad_table; a.ldt = ld_grad_table;
  a.accumulate = accumulate != 0;
  const hipStream_t st = (hipStream_t)stream;
  return hip_status(timed_launch(K_GATHER, st, [&] {
    if (rows > 0) {
      const hipError_t e = launch_sort_tokens(s, st);
      if (e != hipSuccess) return e;
    }
    return launch_embed_backward(a, st);
  }), "embedding gradient");
}

svl_status svl_norm_forward(const svl_norm* norm, int32_t rows, const void* x, int64_t ld_x, const void* gain,
                            const void* bias, void* y, int64_t ld_y, float* stats, void* stream) {
  SVL_TRY(check_norm(norm));
  SVL_TRY(check_row_count(rows));
  if (rows == 0) return SVL_OK;
  SVL_TRY(check_array(x, ld_x, norm->width, "x"));
  SVL_TRY(check_array(y, ld_y, norm->width, "y"));
  if (!aligned(gain, 16) || !aligned(bias, 16)) return err(SVL_E_ALIGN, "gain or bias not 16-byte aligned");
  if (!aligned(stats, 8)) return err(SVL_E_ALIGN, "stats not 8-byte aligned");
  if (x == y && (norm->x_type != norm->y_type || ld_x != ld_y))
    return err(SVL_E_VALUE, "y may be x only with its type and stride");
  RowNormArgs a = norm_args(*norm, rows, x, ld_x, gain);
  a.bias = bias;
  a.y = y; a.ldy = ld_y;
  a.stats = stats;
  const hipStream_t st = (hipStream_t)stream;
  return hip_status(timed_launch(K_NORM, st, [&] { return launch_row_norm(a, st); }), "row norm");
}

size_t svl_norm_workspace_bytes(const svl_norm* norm, int32_t rows) {
  if (check_norm(norm) != SVL_OK || check_row_count(rows) != SVL_OK) return 0;
  return (size_t)norm_bytes(*norm, rows);
}

svl_status svl_norm_backward(const svl_norm* norm, int32_t rows, const void* x, int64_t ld_x, const void* gain,
                             const float* stats, const void* grad_y, int64_t ld_grad_y, void* grad_x,
                             int64_t ld_grad_x, float* grad_gain, float* grad_bias, int32_t accumulate, void* ws,
                             size_t ws_bytes, void* stream) {
  SVL_TRY(check_norm(norm));
  SVL_TRY(check_row_count(rows));
  SVL_TRY(check_flag(accumulate, "accumulate"));
  if (!aligned(grad_gain, 16) || !aligned(grad_bias, 16))
    return err(SVL_E_ALIGN, "grad_gain or grad_bias not 16-byte aligned");
  const bool weights = grad_gain || grad_bias;
  if (rows > 0) {
    SVL_TRY(check_array(x, ld_x, norm->width, "x"));
    SVL_TRY(check_array(grad_y, ld_grad_y, norm->width, "grad_y"));
    SVL_TRY(check_optional(grad_x, ld_grad_x, norm->width, "grad_x"));
    SVL_TRY(check_pointer(stats, "stats", 8));
    if (!aligned(gain, 16)) return err(SVL_E_ALIGN, "gain not 16-byte aligned");
    if (grad_x && grad_x == grad_y && (norm->x_type != norm->y_type || ld_grad_x != ld_grad_y))
      return err(SVL_E_VALUE, "grad_x may be grad_y only with its type and stride");
    if (weights) SVL_TRY(check_workspace(ws, ws_bytes, (size_t)norm_bytes(*norm, rows)));
  }
  if ((!grad_x || rows == 0) && !weights) return SVL_OK;
  RowNormArgs a = norm_args(*norm, rows, x, ld_x, gain);
  a.stats = const_cast<float*>(stats);
  a.grad_y = grad_y; a.ldgy = ld_grad_y;
  a.grad_x = grad_x; a.ldgx = ld_grad_x;
  a.want_gain = grad_gain != nullptr;
  a.want_bias = grad_bias != nullptr;
  a.partial = static_cast<float*>(ws);
  const hipStream_t st = (hipStream_t)stream;
  return hip_status(timed_launch(K_NORM, st, [&] {
    hipError_t e = rows > 0 ? launch_row_norm_backward(a, st) : hipSuccess;
    if (e == hipSuccess && weights)
      e = launch_norm_join(a.partial, norm_pieces(rows, norm->width), norm->width, grad_gain ? grad_gain : grad_bias,
                           grad_gain ? grad_bias : nullptr, accumulate != 0, st);
    return e;
  }), "row norm gradient");
}

size_t svl_lm_loss_workspace_bytes(const svl_lm_head* head, int32_t rows, int32_t want_grad_x,
                                   int32_t want_grad_w) {
  if (check_head(head) != SVL_OK || check_row_count(rows) != SVL_OK) return 0;
  if (check_flag(want_grad_x, "want_grad_x") != SVL_OK || check_flag(want_grad_w, "want_grad_w") != SVL_OK) return 0;
  LmArgs a{};
  return (size_t)lm_layout(*head, rows, want_grad_x != 0, want_grad_w != 0, nullptr, &a);
}

svl_status svl_lm_loss(const svl_lm_head* head, int32_t rows, const void* x, int64_t ld_x, const void* w,
                       int64_t ld_w, const int32_t* labels, const float* row_weight, float* loss, float* lse,
                       void* grad_x, int64_t ld_grad_x, void* grad_w, int64_t ld_grad_w, int32_t accumulate,
                       void* ws, size_t ws_bytes, void* stream) {
  SVL_TRY(check_head(head));
  SVL_TRY(check_row_count(rows));
  SVL_TRY(check_flag(accumulate, "accumulate"));
  SVL_TRY(check_optional(grad_w, ld_grad_w, head->d_model, "grad_w", LM_MAX_LD));
  if (rows > 0) {
    SVL_TRY(check_array(x, ld_x, head->d_model, "x", LM_MAX_LD));
    SVL_TRY(check_array(w, ld_w, head->d_model, "w", LM_MAX_LD));
    SVL_TRY(check_pointer(labels, "labels", 4));
    if (!aligned(row_weight, 4)) return err(SVL_E_ALIGN, "row_weight not 4-byte aligned");
    SVL_TRY(check_pointer(loss, "loss", 4));
    if (!aligned(lse, 4)) return err(SVL_E_ALIGN, "lse not 4-byte aligned");
    SVL_TRY(check_optional(grad_x, ld_grad_x, head->d_model, "grad_x", LM_MAX_LD));
    SVL_TRY(check_workspace(ws, ws_bytes, svl_lm_loss_workspace_bytes(head, rows, grad_x != nullptr, grad_w != nullptr)));
  }
  LmArgs a{};
  lm_layout(*head, rows, grad_x != nullptr, grad_w != nullptr, static_cast<char*>(ws), &a);
  a.x = static_cast<const uint16_t*>(x); a.ldx = ld_x;
  a.w = static_cast<const uint16_t*>(w); a.ldw = ld_w;
  a.labels = labels;
  a.row_weight = row_weight;
  a.loss = loss;
  a.lse = lse;
  a.grad_x = static_cast<uint16_t*>(grad_x); a.ldgx = ld_grad_x;
  a.grad_w = static_cast<uint16_t*>(grad_w); a.ldgw = ld_grad_w;
  a.accumulate = accumulate != 0;
  const hipStream_t st = (hipStream_t)stream;
  const bool f16 = head->compute == SVL_COMPUTE_F16;
  return hip_status(timed_launch(K_CTRL, st, [&] {
    if (rows == 0) return grad_w && !accumulate ? launch_lm_zero_w(a, st) : hipSuccess;
    hipError_t e = launch_lm_rows(a, st);
    for (a.chunk0 = 0; e == hipSuccess && a.chunk0 < rows; a.chunk0 += a.chunk) {
      a.first = a.chunk0 == 0;
      a.last = a.chunk0 + a.chunk >= rows;
      if (e == hipSuccess) e = launch_lm_product(a, LM_LOGITS, f16, st);
      if (e == hipSuccess) e = launch_lm_stats(a, st);
      if (e == hipSuccess && a.e) e = launch_lm_softmax(a, f16, st);
      if (e == hipSuccess && grad_x) e = launch_lm_product(a, LM_GRAD_X, f16, st);
      if (e == hipSuccess && f16 && grad_x && grad_w && row_weight) e = launch_lm_weigh(a, st);
      if (e == hipSuccess && grad_w) e = launch_lm_product(a, LM_GRAD_W, f16, st);
    }
    return e;
  }), "language-model loss");
}

svl_status svl_adamw_step(const svl_adamw* adam, int32_t n_tensors, const svl_adamw_tensor* tensors, int64_t step,
                          uint32_t seed, float grad_scale, const svl_adamw_dev* dev, void* stream) {
  SVL_TRY(check_adamw(adam));
  if (n_tensors < 0) return err(SVL_E_SHAPE, "n_tensors = %d is negative", n_tensors);
  if (n_tensors > 0 && !tensors) return err(SVL_E_NULL, "tensors is NULL");
  if (!dev && step < 1) return err(SVL_E_VALUE, "step = %lld must be at least 1", (long long)step);
  if (!dev && !std::isfinite(grad_scale)) return err(SVL_E_VALUE, "grad_scale must be finite");
  if (!aligned(dev, 4)) return err(SVL_E_ALIGN, "dev not 4-byte aligned");
  for (int32_t i = 0; i < n_tensors; ++i) SVL_TRY(check_tensor(tensors[i], i, adam->state_bits));
  AdamwArgs a{};
  a.beta1 = (float)adam->beta1;
  a.beta2 = (float)adam->beta2;
  a.rest1 = (float)(1.0 - adam->beta1);
  a.rest2 = (float)(1.0 - adam->beta2);
  a.eps = (float)adam->eps;
  a.decay = (float)adam->weight_decay;
  a.dev = dev;
  a.now = svl_adamw_dev{(float)adam->lr, (float)(1.0 - std::pow(adam->beta1, (double)step)),
                        (float)(1.0 - std::pow(adam->beta2, (double)step)), grad_scale, seed};
  // a launch's threads stay under 2^32
  constexpr int64_t MOST = 1 << 23;
  const hipStream_t st = (hipStream_t)stream;
  return hip_status(timed_launch(K_CTRL, st, [&] {
    int64_t done = 0;                      // items of tensor i that earlier launches took
    for (int32_t i = 0; i < n_tensors;) {
      if (tensors[i].n == 0) {
        ++i;
        continue;
      }
      // tensor numbers of a launch are consecutive: an empty one ends it
      a.number0 = i;
      a.first_item = done;
      a.count = 0;
      int64_t items = 0;
      while (i < n_tensors && a.count < ADAMW_TENSORS && items < MOST && tensors[i].n > 0) {
        const svl_adamw_tensor& t = tensors[i];
        const int64_t left = cdiv(t.n, ADAMW_ITEM) - done, take = std::min(left, MOST - items);
        a.t[a.count++] = AdamwTensor{t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.n, (int32_t)items,
                                     (int16_t)t.param_type, (int16_t)t.grad_type};
        items += take;
        if (take < left) {
          done += take;
          break;
        }
        done = 0;
        ++i;
      }
      const hipError_t e = launch_adamw(a, adam->state_bits == 8, (int32_t)items, st);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }), "optimizer step");
}

svl_status svl_adamw_read_state(int32_t second, int64_t n, const void* codes, const float* scales, float* out,
                                void* stream) {
  SVL_TRY(check_flag(second, "second"));
  if (n < 0 || n > ((int64_t)1 << 40)) return err(SVL_E_SHAPE, "n = %lld out of range", (long long)n);
  if (n == 0) return SVL_OK;
  SVL_TRY(check_pointer(codes, "codes"));
  SVL_TRY(check_pointer(scales, "scales", 4));
  SVL_TRY(check_pointer(out, "out"));
  const hipStream_t st = (hipStream_t)stream;
  return hip_status(timed_launch(K_CTRL, st, [&] {
    return launch_adamw_read(second != 0, n, static_cast<const uint8_t*>(codes), scales, out, st);
  }), "optimizer state");
}

}  // extern "C"
