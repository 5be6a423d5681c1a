// C ABI of the windowed attention and of the 4-bit K / V cache: argument checks
// (all before anything is enqueued), how the work is cut, and the launches.
// Segments go to the kernels by value, so no call copies anything to the device
// and a captured call keeps the lengths it was made with.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "../../include/svl.h"
#include "attn_ops.h"
#include "svl_internal.h"

namespace svl {
namespace {

bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
int64_t round256(int64_t x) { return (x + 255) & ~int64_t(255); }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
svl_status check_attention(const svl_attention* t) {
  if (!t) return err(SVL_E_NULL, "attention description is NULL");
  if (t->n_heads <= 0 || t->n_kv_heads <= 0 || t->n_heads % t->n_kv_heads)
    return err(SVL_E_SHAPE, "n_heads = %d must be a positive multiple of n_kv_heads = %d", t->n_heads,
               t->n_kv_heads);
  if (t->head_dim != 64 && t->head_dim != 128)
    return err(SVL_E_SHAPE, "head_dim must be 64 or 128, not %d", t->head_dim);
  if ((int64_t)t->n_heads * t->head_dim > 65536)
    return err(SVL_E_SHAPE, "n_heads * head_dim above 65536");
  if (t->compute != SVL_COMPUTE_F16 && t->compute != SVL_COMPUTE_BF16)
    return err(SVL_E_DTYPE, "unknown compute type %d", t->compute);
  if (t->window < 0 || t->sinks < 0)
    return err(SVL_E_VALUE, "window = %d and sinks = %d must not be negative", t->window, t->sinks);
  if (!(t->scale > 0.f) || !std::isfinite(t->scale))
    return err(SVL_E_VALUE, "scale must be finite and > 0");
  return SVL_OK;
}

// cu: [batch + 1] row offsets, not decreasing, from 0 or more.
svl_status check_rows(int32_t batch, const int32_t* cu, const char* what) {
  if (batch <= 0) return err(SVL_E_SHAPE, "batch must be positive");
  if (!cu) return err(SVL_E_NULL, "%s is NULL", what);
  if (cu[0] < 0) return err(SVL_E_VALUE, "%s[0] = %d is negative", what, cu[0]);
  for (int32_t b = 0; b < batch; ++b)
    if (cu[b + 1] < cu[b])
      return err(SVL_E_VALUE, "%s decreases at %d (%d after %d)", what, b + 1, cu[b + 1], cu[b]);
  return SVL_OK;
}

// A row array of 16-bit values: rows at least `width` apart.  `rows` = 0: may be NULL.
svl_status check_array(const void* p, int64_t ld, int64_t width, int64_t rows, const char* what) {
  if (rows <= 0) return SVL_OK;
  if (!p) return err(SVL_E_NULL, "%s is NULL", what);
  if (!is_aligned16(p)) return err(SVL_E_ALIGN, "%s not 16-byte aligned", what);
  if (ld < width || ld % 8 || ld > (1 << 23))
    return err(SVL_E_SHAPE, "row stride %lld of %s: at least %lld, at most 2^23 and a multiple of 8",
               (long long)ld, what, (long long)width);
  return SVL_OK;
}

svl_status check_cache(int32_t batch, const int32_t* cu, const int32_t* pos, const void* cache,
                       int32_t max_len) {
  svl_status s = check_rows(batch, cu, "cu_rows");
  if (s != SVL_OK) return s;
  if (!pos) return err(SVL_E_NULL, "pos is NULL");
  if (!cache) return err(SVL_E_NULL, "cache is NULL");
  if (!is_aligned16(cache)) return err(SVL_E_ALIGN, "cache not 16-byte aligned");
  if (max_len <= 0 || max_len > SVL_KV4_MAX_LEN)
    return err(SVL_E_SHAPE, "max_len = %d outside [1, %d]", max_len, SVL_KV4_MAX_LEN);
  for (int32_t b = 0; b < batch; ++b) {
    const int64_t rows = (int64_t)cu[b + 1] - cu[b];
    if (pos[b] < 0 || pos[b] + rows > max_len)
      return err(SVL_E_VALUE, "sample %d: %lld rows from position %d do not fit max_len = %d", b,
                 (long long)rows, pos[b], max_len);
  }
  return SVL_OK;
}

// Queries are the last rows of their sample's keys.
svl_status check_packed(int32_t batch, const int32_t* cu_q, const int32_t* cu_k) {
  svl_status s = check_rows(batch, cu_q, "cu_q");
  if (s != SVL_OK) return s;
  if ((s = check_rows(batch, cu_k, "cu_k")) != SVL_OK) return s;
  if (cu_q[batch] > (1 << 30) || cu_k[batch] > (1 << 30)) return err(SVL_E_SHAPE, "too many packed rows");
  for (int32_t b = 0; b < batch; ++b)
    if (cu_q[b + 1] - cu_q[b] > cu_k[b + 1] - cu_k[b])
      return err(SVL_E_VALUE, "sample %d has %d queries for %d keys", b, cu_q[b + 1] - cu_q[b],
                 cu_k[b + 1] - cu_k[b]);
  return SVL_OK;
}

// ------------------------------------------------------------------ segments
struct CacheRows {
  const int32_t* cu;
  const int32_t* pos;
  int32_t n_kv_heads;
};
CacheSeg cache_seg(const void* ctx, int32_t b) {
  const CacheRows& r = *static_cast<const CacheRows*>(ctx);
  CacheSeg s{};
  s.row0 = r.cu[b];
  s.rows = r.cu[b + 1] - r.cu[b];
  s.pos0 = r.pos[b];
  s.sample = b;
  s.kv_cnt = r.n_kv_heads;
  return s;
}

struct PackedRows {
  const int32_t* cu_q;
  const int32_t* cu_k;
  int32_t n_heads;
};
WinSeg win_seg(const void* ctx, int32_t b) {
  const PackedRows& r = *static_cast<const PackedRows*>(ctx);
  WinSeg s{};
  s.q0 = r.cu_q[b];
  s.nq = r.cu_q[b + 1] - r.cu_q[b];
  s.k0 = r.cu_k[b];
  s.nk = r.cu_k[b + 1] - r.cu_k[b];
  s.h_cnt = r.n_heads;
  return s;
}

Kv4Args kv4_args(const svl_attention& t, void* cache, int32_t max_len) {
  Kv4Args a{};
  a.n_kv_heads = t.n_kv_heads;
  a.rep = t.n_heads / t.n_kv_heads;
  a.cache = static_cast<uint8_t*>(cache);
  a.tiles = cdiv(max_len, KV4_TILE);
  a.scale = t.scale;
  a.window = window_of(t.window);
  a.sinks = t.sinks;
  return a;
}

// Launches `f` for the segments, their tiles as work items.
template <class F>
hipError_t tile_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n, const F& f) {
  for (int32_t i = 0; i < n;) {
    a.nsegs = 0;
    int64_t items = 0;
    for (; i < n && a.nsegs < SEGS_PER_LAUNCH; ++i) {
      CacheSeg s = get(ctx, i);
      if (s.rows <= 0 || s.kv_cnt <= 0) continue;
      const int64_t tiles = (s.pos0 + (int64_t)s.rows - 1) / KV4_TILE - s.pos0 / KV4_TILE + 1;
      if (items + tiles * s.kv_cnt > INT32_MAX / 2 && a.nsegs > 0) break;
      s.item0 = (int32_t)items;
      items += tiles * s.kv_cnt;
      a.seg[a.nsegs++] = s;
    }
    if (items > INT32_MAX / 2) return hipErrorInvalidValue;
    a.nitems = (int32_t)items;
    if (a.nsegs == 0) continue;
    const hipError_t e = f();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Units (of KV4_UNIT positions) that a segment's rows see, at most.
int64_t seg_units(const Kv4Args& a, const CacheSeg& s) {
  const int64_t p1 = (int64_t)s.pos0 + s.rows - 1;
  const int64_t start = a.window > 0 ? std::max<int64_t>(0, (int64_t)s.pos0 - a.window + 1) : 0;
  const int64_t uw = start / KV4_UNIT;
  const int64_t us = std::min(cdiv(std::min<int64_t>(a.sinks, start), KV4_UNIT), uw);
  return us + p1 / KV4_UNIT + 1 - uw;
}

// Key / value gradient of the windowed attention: how its work is cut.  Two items a
// compute unit (rows of 4096 and 3001 in a window of 1024, 32 on 8 heads, with the
// join: 256 items 727 us, 512 460, 640 444, 768 475), and no piece of fewer than 8
// list entries (rows of 640 and 577, 32 heads: from 4 on cut, with the join 76 us,
// from 8 on not, 42).
constexpr int64_t kDkvTarget = 512, kDkvMin = 8;   // work items of a launch; list entries of a piece

// Fills a.seg with the next samples from b on; returns the next sample.  dkv: the
// work items of the key / value gradient, otherwise those of the query gradient.
int32_t bwd_segments(WinBwdArgs& a, int32_t batch, const int32_t* cu_q, const int32_t* cu_k, int32_t b,
                     bool dkv, int64_t* blocks) {
  const int64_t rep = a.n_heads / a.n_kv_heads, KV = a.n_kv_heads;
  a.nsegs = 0;
  a.nitems = 0;
  *blocks = 0;
  int64_t sum = 0;
  int64_t w_sink[SEGS_PER_LAUNCH], w_other[SEGS_PER_LAUNCH];
  for (; b < batch && a.nsegs < SEGS_PER_LAUNCH; ++b) {
    WinBwdSeg s{};
    s.q0 = cu_q[b];
    s.nq = cu_q[b + 1] - cu_q[b];
    s.k0 = cu_k[b];
    s.nk = cu_k[b + 1] - cu_k[b];
    if (dkv ? s.nk <= 0 : s.nq <= 0) continue;
    const int64_t nkt = cdiv(s.nk, WIN_DK), all = rep * cdiv(s.nq, WIN_DQ);
    s.nst = a.window > 0 ? (int32_t)std::min<int64_t>(cdiv(std::min(a.sinks, s.nk), WIN_DK), nkt) : 0;
    w_sink[a.nsegs] = all;
    // a later row sees fewer tiles after it: half of them on average without a window
    w_other[a.nsegs] = a.window > 0 ? std::min(all, rep * cdiv((int64_t)a.window + WIN_DK, WIN_DQ))
                                    : std::max<int64_t>(1, all - all * (s.nq - 1) / (2 * (int64_t)s.nk));
    sum += KV * (s.nst * w_sink[a.nsegs] + (nkt - s.nst) * w_other[a.nsegs]);
    a.seg[a.nsegs++] = s;
  }
  int64_t items = 0;
  const int64_t per = std::max(kDkvMin, cdiv(sum, kDkvTarget));
  for (int32_t i = 0; i < a.nsegs; ++i) {
    WinBwdSeg& s = a.seg[i];
    s.item0 = (int32_t)items;
    if (dkv) {
      const int64_t nkt = cdiv(s.nk, WIN_DK);
      s.ps = (int32_t)std::max<int64_t>(1, (w_sink[i] + per / 2) / per);
      s.po = (int32_t)std::max<int64_t>(1, (w_other[i] + per / 2) / per);
      const int64_t n_sink = KV * s.nst * s.ps, n_other = KV * (nkt - s.nst) * s.po;
      s.part0 = (int32_t)*blocks;
      if (s.ps > 1) *blocks += n_sink;
      s.part1 = (int32_t)*blocks;
      if (s.po > 1) *blocks += n_other;
      items += n_sink + n_other;
    } else {
      items += cdiv(s.nq, 128) * a.n_heads;
    }
  }
  a.nitems = items > INT32_MAX ? -1 : (int32_t)items;
  return b;
}

// delta and exponents of the query rows, then the partial blocks.
int64_t bwd_rows_bytes(const svl_attention& t, int64_t rows) { return round256(rows * t.n_heads * 4); }

}  // namespace

hipError_t kv4_append_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n, int32_t head_dim,
                               bool f16, hipStream_t st) {
  return tile_segments(a, get, ctx, n, [&] {
    return timed_launch(K_KV_APPEND, st, [&] { return launch_kv4_append(a, head_dim, f16, st); });
  });
}

hipError_t kv4_read_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n, int32_t head_dim,
                             bool f16, hipStream_t st) {
  return tile_segments(a, get, ctx, n, [&] {
    return timed_launch(K_KV_APPEND, st, [&] { return launch_kv4_read(a, head_dim, f16, st); });
  });
}

// A piece has at least 1 / KV4_TARGET_ITEMS of the launch's units, so the pieces
// of segments that are cut are at most twice KV4_TARGET_ITEMS.
size_t kv4_partial_bytes(int32_t head_dim) {
  return (size_t)(2 * KV4_TARGET_ITEMS * kv4_partial_floats(head_dim) * 4);
}

hipError_t kv4_attention_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n,
                                  int32_t head_dim, bool f16, hipStream_t st) {
  for (int32_t i = 0; i < n;) {
    a.nsegs = 0;
    int64_t columns = 0;
    for (; i < n && a.nsegs < SEGS_PER_LAUNCH; ++i) {
      const CacheSeg s = get(ctx, i);
      if (s.rows <= 0 || s.kv_cnt <= 0) continue;
      columns = std::max(columns, (int64_t)s.rows * a.rep);
      a.seg[a.nsegs++] = s;
    }
    if (a.nsegs == 0) continue;
    int64_t units = 0;
    for (int32_t k = 0; k < a.nsegs; ++k)
      units += cdiv((int64_t)a.seg[k].rows * a.rep, KV4_COLS) * a.seg[k].kv_cnt * seg_units(a, a.seg[k]);
    const int64_t per = std::max<int64_t>(KV4_MIN_UNITS, cdiv(units, KV4_TARGET_ITEMS));
    int64_t items = 0, parts = 0, cut = 0;
    for (int32_t k = 0; k < a.nsegs; ++k) {
      CacheSeg& s = a.seg[k];
      const int64_t blocks = cdiv((int64_t)s.rows * a.rep, KV4_COLS) * s.kv_cnt;
      // (a cut pays for its join from two pieces' worth of work on)
      const int64_t u = seg_units(a, s);
      s.nsplit = u < 2 * per ? 1 : (int32_t)cdiv(u, per);
      s.item0 = (int32_t)items;
      s.part0 = (int32_t)parts;
      s.join0 = (int32_t)cut;
      items += blocks * s.nsplit;
      if (s.nsplit > 1) {
        parts += blocks * s.nsplit;
        cut += blocks;
      }
      if (items > INT32_MAX / 64) return hipErrorInvalidValue;
    }
    a.nitems = (int32_t)items;
    hipError_t e = timed_launch(K_ATTN, st, [&] { return launch_kv4_attention(a, head_dim, f16, st); });
    if (e != hipSuccess) return e;
    if (cut > 0) {
      const int32_t most = (int32_t)std::min<int64_t>(columns, KV4_COLS);
      e = timed_launch(K_ATTN, st, [&] { return launch_kv4_join(a, head_dim, f16, (int32_t)cut, most, st); });
      if (e != hipSuccess) return e;
    }
  }
  return hipSuccess;
}

hipError_t window_segments(WinArgs& a, WinSegOf get, const void* ctx, int32_t n, int32_t head_dim,
                           bool f16, hipStream_t st) {
  for (int32_t i = 0; i < n;) {
    a.nsegs = 0;
    int64_t items = 0;
    for (; i < n && a.nsegs < SEGS_PER_LAUNCH; ++i) {
      const WinSeg s = get(ctx, i);
      if (s.nq <= 0 || s.h_cnt <= 0) continue;
      items += cdiv(s.nq, 128) * s.h_cnt;
      a.seg[a.nsegs++] = s;
    }
    if (a.nsegs == 0) continue;
    // two workgroups fit a CU: with fewer of 128 rows, 64 rows each (640 rows of 32
    // heads in a window of 256: 19 us against 25, causal rows of 640 and 577 25.5
    // against 28; up to 3008 rows of 28 heads on 4 264 against 219)
    const int32_t bq = items < 512 ? 64 : 128;
    items = 0;
    for (int32_t k = 0; k < a.nsegs; ++k) {
      if (items > INT32_MAX) return hipErrorInvalidValue;
      a.seg[k].item0 = (int32_t)items;
      items += cdiv(a.seg[k].nq, bq) * a.seg[k].h_cnt;
    }
    if (items > INT32_MAX) return hipErrorInvalidValue;
    a.nitems = (int32_t)items;
    const hipError_t e =
        timed_launch(K_ATTN, st, [&] { return launch_window_attention(a, head_dim, f16, bq, st); });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace svl

using namespace svl;

extern "C" {

size_t svl_kv4_cache_bytes(const svl_attention* att, int32_t batch, int32_t max_len) {
  if (check_attention(att) != SVL_OK) return 0;
  if (batch <= 0 || max_len <= 0 || max_len > SVL_KV4_MAX_LEN) {
    err(SVL_E_SHAPE, "batch = %d or max_len = %d out of range", batch, max_len);
    return 0;
  }
  return (size_t)batch * att->n_kv_heads * cdiv(max_len, KV4_TILE) * kv4_tile_bytes(att->head_dim);
}

svl_status svl_kv4_append(const svl_attention* att, int32_t batch, const int32_t* cu_rows,
                          const int32_t* pos, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                          void* cache, int32_t max_len, void* stream) {
  svl_status s = check_attention(att);
  if (s != SVL_OK) return s;
  if ((s = check_cache(batch, cu_rows, pos, cache, max_len)) != SVL_OK) return s;
  const int64_t width = (int64_t)att->n_kv_heads * att->head_dim, rows = (int64_t)cu_rows[batch] - cu_rows[0];
  if ((s = check_array(k, ld_k, width, rows, "k")) != SVL_OK) return s;
  if ((s = check_array(v, ld_v, width, rows, "v")) != SVL_OK) return s;
  Kv4Args a = kv4_args(*att, cache, max_len);
  a.k = k; a.ldk = ld_k;
  a.v = v; a.ldv = ld_v;
  const CacheRows r{cu_rows, pos, att->n_kv_heads};
  return hip_status(kv4_append_segments(a, cache_seg, &r, batch, att->head_dim,
                                        att->compute == SVL_COMPUTE_F16, (hipStream_t)stream), "4-bit append");
}

svl_status svl_kv4_read(const svl_attention* att, int32_t batch, const int32_t* cu_rows,
                        const int32_t* pos, const void* cache, int32_t max_len, void* k, int64_t ld_k,
                        void* v, int64_t ld_v, void* stream) {
  svl_status s = check_attention(att);
  if (s != SVL_OK) return s;
  if ((s = check_cache(batch, cu_rows, pos, cache, max_len)) != SVL_OK) return s;
  const int64_t width = (int64_t)att->n_kv_heads * att->head_dim, rows = (int64_t)cu_rows[batch] - cu_rows[0];
  if ((s = check_array(k, ld_k, width, rows, "k")) != SVL_OK) return s;
  if ((s = check_array(v, ld_v, width, rows, "v")) != SVL_OK) return s;
  Kv4Args a = kv4_args(*att, const_cast<void*>(cache), max_len);
  a.k_out = k; a.ldk = ld_k;
  a.v_out = v; a.ldv = ld_v;
  const CacheRows r{cu_rows, pos, att->n_kv_heads};
  return hip_status(kv4_read_segments(a, cache_seg, &r, batch, att->head_dim,
                                      att->compute == SVL_COMPUTE_F16, (hipStream_t)stream), "4-bit read");
}

size_t svl_kv4_workspace_bytes(const svl_attention* att) {
  if (check_attention(att) != SVL_OK) return 0;
  return kv4_partial_bytes(att->head_dim);
}

svl_status svl_kv4_attention(const svl_attention* att, int32_t batch, const int32_t* cu_rows,
                             const int32_t* pos, const void* q, int64_t ld_q, const void* cache,
                             int32_t max_len, void* out, int64_t ld_out, void* ws, size_t ws_bytes,
                             void* stream) {
  svl_status s = check_attention(att);
  if (s != SVL_OK) return s;
  if ((s = check_cache(batch, cu_rows, pos, cache, max_len)) != SVL_OK) return s;
  const int64_t width = (int64_t)att->n_heads * att->head_dim, rows = (int64_t)cu_rows[batch] - cu_rows[0];
  if ((s = check_array(q, ld_q, width, rows, "q")) != SVL_OK) return s;
  if ((s = check_array(out, ld_out, width, rows, "out")) != SVL_OK) return s;
  if (!ws) return err(SVL_E_NULL, "workspace is NULL");
  if (!is_aligned16(ws)) return err(SVL_E_ALIGN, "workspace not 16-byte aligned");
  if (ws_bytes < kv4_partial_bytes(att->head_dim))
    return err(SVL_E_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, kv4_partial_bytes(att->head_dim));
  Kv4Args a = kv4_args(*att, const_cast<void*>(cache), max_len);
  a.q = q; a.ldq = ld_q;
  a.out = out; a.ldo = ld_out;
  a.partial = static_cast<float*>(ws);
  const CacheRows r{cu_rows, pos, att->n_kv_heads};
  return hip_status(kv4_attention_segments(a, cache_seg, &r, batch, att->head_dim,
                                           att->compute == SVL_COMPUTE_F16, (hipStream_t)stream),
                    "attention over the 4-bit cache");
}

svl_status svl_window_attention(const svl_attention* att, int32_t batch, const int32_t* cu_q,
                                const int32_t* cu_k, const void* q, int64_t ld_q, const void* k,
                                int64_t ld_k, const void* v, int64_t ld_v, const uint8_t* key_mask,
                                void* out, int64_t ld_out, float* lse, void* stream) {
  svl_status s = check_attention(att);
  if (s != SVL_OK) return s;
  if (!cu_k) cu_k = cu_q;
  if ((s = check_packed(batch, cu_q, cu_k)) != SVL_OK) return s;
  const int64_t qw = (int64_t)att->n_heads * att->head_dim, kw = (int64_t)att->n_kv_heads * att->head_dim;
  const int64_t rows = (int64_t)cu_q[batch] - cu_q[0];
  if ((s = check_array(q, ld_q, qw, rows, "q")) != SVL_OK) return s;
  if ((s = check_array(k, ld_k, kw, rows, "k")) != SVL_OK) return s;
  if ((s = check_array(v, ld_v, kw, rows, "v")) != SVL_OK) return s;
  if ((s = check_array(out, ld_out, qw, rows, "out")) != SVL_OK) return s;
  WinArgs a{};
  a.n_heads = att->n_heads;
  a.n_kv_heads = att->n_kv_heads;
  a.q = q; a.ldq = ld_q;
  a.k = k; a.ldk = ld_k;
  a.v = v; a.ldv = ld_v;
  a.out = out; a.ldo = ld_out;
  a.lse = lse;
  a.key_mask = key_mask;
  a.scale = att->scale;
  a.window = window_of(att->window);
  a.sinks = att->sinks;
  const PackedRows r{cu_q, cu_k, att->n_heads};
  return hip_status(window_segments(a, win_seg, &r, batch, att->head_dim,
                                    att->compute == SVL_COMPUTE_F16, (hipStream_t)stream), "windowed attention");
}

size_t svl_window_workspace_bytes(const svl_attention* att, int32_t batch, const int32_t* cu_q,
                                  const int32_t* cu_k) {
  if (check_attention(att) != SVL_OK) return 0;
  if (!cu_k) cu_k = cu_q;
  if (check_packed(batch, cu_q, cu_k) != SVL_OK) return 0;
  WinBwdArgs a{};
  a.n_heads = att->n_heads;
  a.n_kv_heads = att->n_kv_heads;
  a.window = window_of(att->window);
  a.sinks = att->sinks;
  int64_t most = 0;
  for (int32_t b = 0; b < batch;) {
    int64_t blocks;
    b = bwd_segments(a, batch, cu_q, cu_k, b, true, &blocks);
    most = std::max(most, blocks);
  }
  return (size_t)(2 * bwd_rows_bytes(*att, cu_q[batch]) + most * 2 * WIN_DK * att->head_dim * 4 + 256);
}

svl_status svl_window_attention_backward(const svl_attention* att, int32_t batch, const int32_t* cu_q,
                                         const int32_t* cu_k, const void* q, int64_t ld_q,
                                         const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                                         const uint8_t* key_mask, const void* out, int64_t ld_out,
                                         const float* lse, const void* grad_out, int64_t ld_grad_out,
                                         void* grad_q, int64_t ld_grad_q, void* grad_k, int64_t ld_grad_k,
                                         void* grad_v, int64_t ld_grad_v, void* ws, size_t ws_bytes,
                                         void* stream) {
  svl_status s = check_attention(att);
  if (s != SVL_OK) return s;
  if (!cu_k) cu_k = cu_q;
  if ((s = check_packed(batch, cu_q, cu_k)) != SVL_OK) return s;
  const int64_t qw = (int64_t)att->n_heads * att->head_dim, kw = (int64_t)att->n_kv_heads * att->head_dim;
  const int64_t rows = (int64_t)cu_q[batch] - cu_q[0], keys = (int64_t)cu_k[batch] - cu_k[0];
  if ((s = check_array(q, ld_q, qw, rows, "q")) != SVL_OK) return s;
  if ((s = check_array(k, ld_k, kw, keys, "k")) != SVL_OK) return s;
  if ((s = check_array(v, ld_v, kw, keys, "v")) != SVL_OK) return s;
  if ((s = check_array(out, ld_out, qw, rows, "out")) != SVL_OK) return s;
  if ((s = check_array(grad_out, ld_grad_out, qw, rows, "grad_out")) != SVL_OK) return s;
  if ((s = check_array(grad_q, ld_grad_q, qw, rows, "grad_q")) != SVL_OK) return s;
  if ((s = check_array(grad_k, ld_grad_k, kw, keys, "grad_k")) != SVL_OK) return s;
  if ((s = check_array(grad_v, ld_grad_v, kw, keys, "grad_v")) != SVL_OK) return s;
  if (rows > 0 && !lse) return err(SVL_E_NULL, "lse is NULL");
  if (!ws) return err(SVL_E_NULL, "workspace is NULL");
  if (!is_aligned16(ws)) return err(SVL_E_ALIGN, "workspace not 16-byte aligned");
  const size_t need = svl_window_workspace_bytes(att, batch, cu_q, cu_k);
  if (ws_bytes < need) return err(SVL_E_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
  WinBwdArgs a{};
  a.n_heads = att->n_heads;
  a.n_kv_heads = att->n_kv_heads;
  a.q = q; a.ldq = ld_q;
  a.k = k; a.ldk = ld_k;
  a.v = v; a.ldv = ld_v;
  a.out = out; a.ldo = ld_out;
  a.grad = grad_out; a.ldg = ld_grad_out;
  a.dq = grad_q; a.lddq = ld_grad_q;
  a.dk = grad_k; a.lddk = ld_grad_k;
  a.dv = grad_v; a.lddv = ld_grad_v;
  a.lse = lse;
  a.key_mask = key_mask;
  uint8_t* w = static_cast<uint8_t*>(ws);
  const int64_t rb = bwd_rows_bytes(*att, cu_q[batch]);
  a.delta = reinterpret_cast<float*>(w);
  a.expo = reinterpret_cast<int32_t*>(w + rb);
  a.partial = reinterpret_cast<float*>(w + 2 * rb);
  a.scale = att->scale;
  a.window = window_of(att->window);
  a.sinks = att->sinks;
  const bool f16 = att->compute == SVL_COMPUTE_F16;
  const hipStream_t st = (hipStream_t)stream;
  const int32_t d = att->head_dim;
  for (int pass = 0; pass < 2; ++pass) {
    for (int32_t b = 0; b < batch;) {
      int64_t blocks;
      b = bwd_segments(a, batch, cu_q, cu_k, b, pass == 1, &blocks);
      if (a.nitems < 0) return err(SVL_E_SHAPE, "too many rows for one launch");
      if (a.nsegs == 0) continue;
      hipError_t e = timed_launch(K_ATTN, st, [&] {
        return pass ? launch_window_dkv(a, d, f16, st) : launch_window_dq(a, d, f16, st);
      });
      if (e == hipSuccess && blocks > 0)
        e = timed_launch(K_ATTN, st, [&] { return launch_window_dkv_join(a, d, f16, st); });
      if (e != hipSuccess) return hip_status(e, "windowed attention backward");
    }
  }
  return SVL_OK;
}

}  // extern "C"
