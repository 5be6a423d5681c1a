// The 4-bit K / V cache: rows quantised as they are written, read back, and
// attended to.
//
// A group of 64 dims of one head's row stands for lo + s c: lo its smallest
// value, s = (largest - smallest) / 15 rounded towards zero to the rows' type
// (so no value leaves the group's range), c = round((x - lo) / s), ties to
// even, within 0..15.  A group with an inf or NaN gets s = lo = NaN.
#include "attn_ops.h"
#include "device_util.h"

namespace svl {
namespace {

__device__ __forceinline__ int find_seg(const Kv4Args& a, int item) {
  int lo = 0, hi = a.nsegs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seg[mid].item0 <= item) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <int D>
struct Tile {
  static constexpr int G = D / KV4_GROUP;
  static constexpr int CODES = KV4_TILE * D / 2;      // bytes of the K (or V) codes
  static constexpr int PARAMS = KV4_TILE * G * 4;     // bytes of the K (or V) pairs
  static constexpr int BYTES = 2 * CODES + 2 * PARAMS;
  static constexpr int KW = D / 32;                   // K words of a lane (row, 8-dim quarter)
  static constexpr int VW = 2 * G;                    // V words of a lane (quad, 4 dims of each group)
};

template <int D>
__device__ __forceinline__ uint8_t* tile_ptr(const Kv4Args& a, int sample, int kvh, int64_t tile) {
  return a.cache + (((int64_t)sample * a.n_kv_heads + kvh) * a.tiles + tile) * Tile<D>::BYTES;
}

// The largest 16-bit value that is not above q >= 0.
template <bool F16>
__device__ __forceinline__ uint32_t round_down_bits(double q) {
  uint32_t b = f32_to_act_bits<F16>((float)q);
  if ((double)act_bits_to_f32<F16>(b) > q) return b - 1;
  if ((double)act_bits_to_f32<F16>(b + 1) <= q) return b + 1;
  return b;
}

constexpr int NT = 256;   // append and read: four waves, each the K or the V half of a tile

// One wave quantises the K or V half of a tile: lane = (row, quarter of its
// dims).  Bound by memory: 2 d bytes in and d / 2 + d / 16 out per row.  The
// codes are decided in float32 except within 2e-5 of a border between two
// codes (float32's own error is below 5e-6 there), where float64 decides.
template <int D, bool F16>
__global__ __launch_bounds__(NT) void kv4_append_kernel(Kv4Args a) {
  typedef Tile<D> T;
  constexpr int EL = D / 4, LG = KV4_GROUP / EL;   // dims of a lane, lanes of a group
  __shared__ __attribute__((aligned(16))) uint8_t s_code[NT / 64][KV4_TILE][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int item = blockIdx.x * (NT / 128) + (wave >> 1);
  const bool is_v = wave & 1;
  if (item >= a.nitems) return;
  const CacheSeg& sg = a.seg[find_seg(a, item)];
  const int local = item - sg.item0;
  const int slot = local % sg.kv_cnt;
  const int tile = sg.pos0 / KV4_TILE + local / sg.kv_cnt;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const int first = max(sg.pos0 - tile * KV4_TILE, 0);                       // rows of the tile
  const int last = min(sg.pos0 + sg.rows - tile * KV4_TILE, KV4_TILE);       // [first, last)
  const int r = lane >> 2, qd = lane & 3;
  const bool on = r >= first && r < last;
  uint32_t w[EL / 2];
  if (on) {
    const int64_t row = (int64_t)sg.row0 + (tile * KV4_TILE + r - sg.pos0);
    const uint16_t* src = static_cast<const uint16_t*>(is_v ? a.v : a.k) +
                          row * (is_v ? a.ldv : a.ldk) + kvh * D + qd * EL;
#pragma unroll
    for (int i = 0; i < EL / 8; ++i) {
      const uint4 x = reinterpret_cast<const uint4*>(src)[i];
      w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EL / 2; ++i) w[i] = 0;
  }
  float lo = __builtin_inff(), hi = -__builtin_inff();
  uint32_t top = 0;   // largest magnitude, as bits: tells inf and NaN
#pragma unroll
  for (int i = 0; i < EL / 2; ++i) {
    const float x0 = act_bits_to_f32<F16>(w[i] & 0xffffu), x1 = act_bits_to_f32<F16>(w[i] >> 16);
    lo = fminf(lo, fminf(x0, x1));
    hi = fmaxf(hi, fmaxf(x0, x1));
    top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
  }
#pragma unroll
  for (int o = 1; o < LG; o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o, 64));
    hi = fmaxf(hi, __shfl_xor(hi, o, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  }
  const bool bad = top >= (F16 ? 0x7c00u : 0x7f80u);
  const uint32_t sb = bad ? (F16 ? 0x7e00u : 0x7fc0u) : round_down_bits<F16>(((double)hi - lo) / 15.0);
  const uint32_t lb = bad ? (F16 ? 0x7e00u : 0x7fc0u) : f32_to_act_bits<F16>(lo);
  const float s = act_bits_to_f32<F16>(sb);
  const bool flat = bad || sb == 0;
  const float inv = 1.0f / s;
  auto code = [&](float x) -> uint32_t {
    const float t = (x - lo) * inv;
    float c = rintf(t);
    if (!(fabsf(t - c) < 0.49998f)) c = (float)rint(((double)x - lo) / s);
    return flat ? 0u : (uint32_t)fminf(fmaxf(c, 0.f), 15.f);
  };
  uint8_t* tp = tile_ptr<D>(a, sg.sample, kvh, tile);
  if (on && qd % LG == 0) {
    uint32_t* par = reinterpret_cast<uint32_t*>(tp + 2 * T::CODES + (is_v ? T::PARAMS : 0));
    par[((r >> 2) * T::G + qd / LG) * 4 + (r & 3)] = sb | (lb << 16);
  }
  if (!is_v) {
    // word j of the lane holds the dims of row word (qd EL / 8 + j)
    if (!on) return;
#pragma unroll
    for (int j = 0; j < EL / 8; ++j) {
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        word |= code(act_bits_to_f32<F16>(w[4 * j + i] & 0xffffu)) << (8 * i);
        word |= code(act_bits_to_f32<F16>(w[4 * j + i] >> 16)) << (8 * i + 4);
      }
      const int row_word = qd * (EL / 8) + j;
      const int place = (row_word & 3) * T::KW + (row_word >> 2);
      reinterpret_cast<uint32_t*>(tp)[r * (D / 8) + place] = word;
    }
    return;
  }
  // V words hold two dims of four positions: exchange through LDS, and keep the
  // nibbles of positions outside this call
#pragma unroll
  for (int i = 0; i < EL / 4; ++i) {
    const uint32_t c4 = code(act_bits_to_f32<F16>(w[2 * i] & 0xffffu)) |
                        code(act_bits_to_f32<F16>(w[2 * i] >> 16)) << 8 |
                        code(act_bits_to_f32<F16>(w[2 * i + 1] & 0xffffu)) << 16 |
                        code(act_bits_to_f32<F16>(w[2 * i + 1] >> 16)) << 24;
    *reinterpret_cast<uint32_t*>(&s_code[wave][r][qd * EL + 4 * i]) = c4;
  }
  wave_lds_handoff();
  uint32_t* vw = reinterpret_cast<uint32_t*>(tp + T::CODES);
#pragma unroll
  for (int i = 0; i < KV4_TILE * D / 8 / 64; ++i) {
    const int f = lane + 64 * i, j = f % T::VW, L = f / T::VW % 16, quad = f / T::VW / 16;
    const int dim = KV4_GROUP * (j >> 1) + 4 * L + 2 * (j & 1);
    uint32_t word = 0, mine = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t two = *reinterpret_cast<const uint16_t*>(&s_code[wave][4 * quad + p][dim]);
      const int sh = 4 * (p >> 1) + 16 * (p & 1);    // dim 0; dim 1 eight bits above
      word |= ((two & 15u) | (two >> 8) << 8) << sh;
      const int pos = 4 * quad + p;
      if (pos >= first && pos < last) mine |= 0x0f0fu << sh;
    }
    if (mine == 0) continue;
    if (mine != 0xffffffffu) word = (word & mine) | (vw[f] & ~mine);
    vw[f] = word;
  }
}

// One wave reads back the K or V half of a tile: lane = (row, quarter).  Bound
// by memory, as the append.
template <int D, bool F16>
__global__ __launch_bounds__(NT) void kv4_read_kernel(Kv4Args a) {
  typedef Tile<D> T;
  constexpr int EL = D / 4, LG = KV4_GROUP / EL;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int item = blockIdx.x * (NT / 128) + (wave >> 1);
  const bool is_v = wave & 1;
  if (item >= a.nitems) return;
  const CacheSeg& sg = a.seg[find_seg(a, item)];
  const int local = item - sg.item0;
  const int slot = local % sg.kv_cnt;
  const int tile = sg.pos0 / KV4_TILE + local / sg.kv_cnt;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const int r = lane >> 2, qd = lane & 3;
  const int pos = tile * KV4_TILE + r;
  if (pos < sg.pos0 || pos >= sg.pos0 + sg.rows) return;
  const uint8_t* tp = tile_ptr<D>(a, sg.sample, kvh, tile);
  const uint32_t pr = reinterpret_cast<const uint32_t*>(
      tp + 2 * T::CODES + (is_v ? T::PARAMS : 0))[((r >> 2) * T::G + qd / LG) * 4 + (r & 3)];
  const float s = act_bits_to_f32<F16>(pr & 0xffffu), lo = act_bits_to_f32<F16>(pr >> 16);
  auto value = [&](uint32_t c) { return fmaf(s, (float)c, lo); };
  uint32_t w[EL / 2];
  if (!is_v) {
    const uint32_t* kw = reinterpret_cast<const uint32_t*>(tp) + r * (D / 8);
#pragma unroll
    for (int j = 0; j < EL / 8; ++j) {
      const int row_word = qd * (EL / 8) + j;
      const uint32_t x = kw[(row_word & 3) * T::KW + (row_word >> 2)];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[4 * j + i] = pack_act2<F16>(value((x >> (8 * i)) & 15u), value((x >> (8 * i + 4)) & 15u));
    }
  } else {
    const uint32_t* vw = reinterpret_cast<const uint32_t*>(tp + T::CODES);
    const int sh = 4 * ((r >> 1) & 1) + 16 * (r & 1);
#pragma unroll
    for (int i = 0; i < EL / 4; ++i) {
      const int dim = qd * EL + 4 * i, g = dim / KV4_GROUP, L = dim % KV4_GROUP / 4;
      const uint2 x = *reinterpret_cast<const uint2*>(vw + ((r >> 2) * 16 + L) * T::VW + 2 * g);
      w[2 * i] = pack_act2<F16>(value((x.x >> sh) & 15u), value((x.x >> (sh + 8)) & 15u));
      w[2 * i + 1] = pack_act2<F16>(value((x.y >> sh) & 15u), value((x.y >> (sh + 8)) & 15u));
    }
  }
  uint16_t* dst = static_cast<uint16_t*>(is_v ? a.v_out : a.k_out) +
                  ((int64_t)sg.row0 + pos - sg.pos0) * (is_v ? a.ldv : a.ldk) + kvh * D + qd * EL;
#pragma unroll
  for (int i = 0; i < EL / 8; ++i)
    reinterpret_cast<uint4*>(dst)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// ---------------------------------------------------------------- attention
// One workgroup: up to 16 NCB columns (query row, head of the K/V head's
// group) of one K/V head, over one piece of the visible positions; four waves
// take 32 positions (a unit) in turn, each with a running maximum and sum, and
// are joined at the end.
//
// The products run on the codes themselves.  A nibble in the low ten bits of a
// half word is an fp16 subnormal, c 2^-24 (or c 2^-20 four bits higher), and the
// matrix cores keep subnormals, so one AND makes an operand pair of two codes.
// Scores: S^T = C Q^T per group of 64 dims, C the K codes (positions x dims), Q
// the query scaled by a power of two into fp16 (exact to 2^-35 of its largest
// value), then s S + lo sum(q) per position and group, in float32.
// Values: O^T = V^T P'^T per group with P' = p s, rounded to fp16 once, plus
// sum(p lo) in float32.  So neither K nor V is rounded to 16 bits on the way.
// The lanes' positions and dims are laid out so that an accumulator of the
// first product is an operand of the second.
constexpr int AT = 256, AW = AT / 64;
constexpr int UNIT = KV4_UNIT;

// Where a work item's positions lie: units [0, us) of the sinks, then from uw on.
struct Units {
  int us, uw, n;
};
__device__ __forceinline__ Units units_of(int p_lo, int p_hi, int window, int sinks) {
  const int start = window > 0 ? max(0, p_lo - window + 1) : 0;
  Units u;
  u.uw = start / UNIT;
  u.us = min((min(sinks, start) + UNIT - 1) / UNIT, u.uw);
  u.n = u.us + p_hi / UNIT + 1 - u.uw;
  return u;
}

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

template <int N> struct Words;
template <> struct Words<4> { typedef uint4 type; };
template <> struct Words<2> { typedef uint2 type; };

template <int D, bool F16, int NCB>
__global__ __launch_bounds__(AT) void kv4_attn_kernel(Kv4Args a) {
  typedef Tile<D> T;
  constexpr int G = T::G, NS = D / 32;
  typedef typename Words<T::KW>::type KWords;
  typedef typename Words<T::VW>::type VWords;
  __shared__ float s_o[AW][16][D + 4];
  __shared__ float s_m[AW][16], s_l[AW][16];
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const CacheSeg& sg = a.seg[find_seg(a, item)];
  const int rep = a.rep, cols = sg.rows * rep, ncb = (cols + 16 * NCB - 1) / (16 * NCB);
  const int local = item - sg.item0, split = local % sg.nsplit, block = local / sg.nsplit;
  const int cb = block % ncb, slot = block / ncb;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int gq = lane >> 4, lq = lane & 15;
  const int c0 = cb * 16 * NCB;
  const int p_lo = sg.pos0 + c0 / rep, p_hi = sg.pos0 + (min(c0 + 16 * NCB, cols) - 1) / rep;
  const Units un = units_of(p_lo, p_hi, a.window, a.sinks);
  const int u0 = (int)((int64_t)un.n * split / sg.nsplit);
  const int u1 = (int)((int64_t)un.n * (split + 1) / sg.nsplit);

  // query fragments; a pair of codes is (dim i, dim i + 4) of a word, the pairs
  // 1 and 3 carry a factor 16
  const float sl2 = a.scale * 1.4426950408889634f;   // scores in log2 units
  uint4 qf[NCB][NS];
  float qs[NCB][G], fl[NCB];
  int pq[NCB];                                       // the column's position
#pragma unroll
  for (int n = 0; n < NCB; ++n) {
    const int c = c0 + 16 * n + lq;
    const bool on = c < cols;
    const int i = on ? c / rep : 0, h = kvh * rep + (on ? c % rep : 0);
    pq[n] = on ? sg.pos0 + i : -1;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((int64_t)sg.row0 + i) * a.ldq +
                         (int64_t)h * D + 8 * gq;
    float x[NS][8];
    float top = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) qs[n][g] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const uint4 v = on ? *reinterpret_cast<const uint4*>(qp + 32 * s) : make_uint4(0, 0, 0, 0);
      const uint32_t wv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[s][2 * e] = act_bits_to_f32<F16>(wv[e] & 0xffffu);
        x[s][2 * e + 1] = act_bits_to_f32<F16>(wv[e] >> 16);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        qs[n][s / 2] += x[s][e];
        top = fmaxf(top, fabsf(x[s][e]));
      }
    }
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
      top = fmaxf(top, __shfl_xor(top, o, 64));
#pragma unroll
      for (int g = 0; g < G; ++g) qs[n][g] += __shfl_xor(qs[n][g], o, 64);
    }
    // 2^k brings the largest magnitude into [2^14, 2^15)
    const int k = top > 0.f ? max(-100, min(100, 141 - (int)(__float_as_uint(top) >> 23))) : 0;
    const float up = pow2f(k);
    fl[n] = ldexpf(sl2, 24 - k);
#pragma unroll
    for (int g = 0; g < G; ++g) qs[n][g] *= pow2f(k - 24);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const float* y = x[s];
      const float up4 = up * 0.0625f;
      qf[n][s] = make_uint4(pack_act2<true>(y[0] * up, y[4] * up), pack_act2<true>(y[1] * up4, y[5] * up4),
                            pack_act2<true>(y[2] * up, y[6] * up), pack_act2<true>(y[3] * up4, y[7] * up4));
    }
  }

  float m[NCB], l[NCB], ol[NCB][G];
  floatx4 o[NCB][G][4];
#pragma unroll
  for (int n = 0; n < NCB; ++n) {
    m[n] = -__builtin_inff();
    l[n] = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      ol[n][g] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[n][g][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // P' = p s 2^ve: fp16 scales fit with a fixed factor; bf16 ones follow the
  // largest scale seen
  int ve = F16 ? 2 : 126;

  const uint8_t* head = tile_ptr<D>(a, sg.sample, kvh, 0);
  const int64_t last_tile = a.tiles - 1;
  for (int u = u0 + wave; u < u1; u += AW) {
    const int unit = u < un.us ? u : un.uw + (u - un.us);
    const int kv0 = unit * UNIT;
    KWords kw[2];
    VWords vw[2];
    uint4 kp[2][G], vp[2][G];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // the second tile of the last unit may lie past the cache: any tile will do
      const uint8_t* tp = head + min((int64_t)2 * unit + t, last_tile) * T::BYTES;
      kw[t] = reinterpret_cast<const KWords*>(tp)[lq * 4 + gq];
      vw[t] = reinterpret_cast<const VWords*>(tp + T::CODES)[lane];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        kp[t][g] = reinterpret_cast<const uint4*>(tp + 2 * T::CODES)[gq * G + g];
        vp[t][g] = reinterpret_cast<const uint4*>(tp + 2 * T::CODES + T::PARAMS)[gq * G + g];
      }
    }
    // whether every column sees every position of the unit
    const bool whole = kv0 + UNIT - 1 <= p_lo &&
                       (a.window <= 0 || kv0 > p_hi - a.window || kv0 + UNIT <= a.sinks);
    uint4 kf[2][NS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&kw[t]);
#pragma unroll
      for (int s = 0; s < NS; ++s)
        kf[t][s] = make_uint4(w[s] & 0x000f000fu, w[s] & 0x00f000f0u, (w[s] >> 8) & 0x000f000fu,
                              (w[s] >> 8) & 0x00f000f0u);
    }
    float vmax = 0.f;
    if constexpr (!F16) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t* pw = reinterpret_cast<const uint32_t*>(&vp[t][g]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (kv0 + 16 * t + 4 * gq + r <= p_hi) vmax = fmaxf(vmax, bf16_bits_to_f32(pw[r] & 0xffffu));
        }
      vmax = fmaxf(vmax, __shfl_xor(vmax, 16, 64));
      vmax = fmaxf(vmax, __shfl_xor(vmax, 32, 64));
      // scales below 2^(e + 1) with e the largest one's exponent: P' < 2^15
      const int want = max(-126, min(126, 14 - ((int)(__float_as_uint(vmax) >> 23) - 127)));
      if (want < ve) {   // the same in every lane
        const float f = ldexpf(1.0f, want - ve);
#pragma unroll
        for (int n = 0; n < NCB; ++n)
#pragma unroll
          for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[n][g][j] *= f;
        ve = want;
      }
    }
    const float pf0 = pow2f(ve), pf1 = pf0 * 0.0625f;
#pragma unroll
    for (int n = 0; n < NCB; ++n) {
      float sc[2][4];
      bool vis[2][4];
      float mx = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        floatx4 acc[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
          acc[g] = floatx4{0.f, 0.f, 0.f, 0.f};
          acc[g] = mfma16x16x32<true>(kf[t][2 * g], qf[n][2 * g], acc[g]);
          acc[g] = mfma16x16x32<true>(kf[t][2 * g + 1], qf[n][2 * g + 1], acc[g]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = 0.f;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const uint32_t pw = reinterpret_cast<const uint32_t*>(&kp[t][g])[r];
            v = fmaf(act_bits_to_f32<F16>(pw & 0xffffu), acc[g][r], v);
            v = fmaf(act_bits_to_f32<F16>(pw >> 16), qs[n][g], v);
          }
          const int j = kv0 + 16 * t + 4 * gq + r;
          vis[t][r] = whole || (j <= pq[n] && (a.window <= 0 || j > pq[n] - a.window || j < a.sinks));
          sc[t][r] = vis[t][r] ? v : -__builtin_inff();
          mx = fmaxf(mx, sc[t][r]);
        }
      }
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      if (__any(mx > m[n])) {
        const float mn = fmaxf(m[n], mx);
        const float alpha = mn == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((m[n] - mn) * fl[n]);
        l[n] *= alpha;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          ol[n][g] *= alpha;
#pragma unroll
          for (int j = 0; j < 4; ++j) o[n][g][j] *= alpha;
        }
        m[n] = mn;
      }
      const float mu = m[n] == -__builtin_inff() ? 0.f : m[n];   // nothing above -inf yet
      float p[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[t][r] = vis[t][r] ? __builtin_amdgcn_exp2f((sc[t][r] - mu) * fl[n]) : 0.f;
          l[n] += p[t][r];
        }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float ps[2][4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t pw = reinterpret_cast<const uint32_t*>(&vp[t][g])[r];
            const float vs = act_bits_to_f32<F16>(pw & 0xffffu), vl = act_bits_to_f32<F16>(pw >> 16);
            // a position that is not seen may hold anything
            ol[n][g] = vis[t][r] ? fmaf(p[t][r], vl, ol[n][g]) : ol[n][g];
            ps[t][r] = vis[t][r] ? p[t][r] * vs * (r < 2 ? pf0 : pf1) : 0.f;
          }
        const uint4 pb = make_uint4(pack_act2<true>(ps[0][0], ps[0][1]), pack_act2<true>(ps[0][2], ps[0][3]),
                                    pack_act2<true>(ps[1][0], ps[1][1]), pack_act2<true>(ps[1][2], ps[1][3]));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t x = reinterpret_cast<const uint32_t*>(&vw[0])[2 * g + j / 2] >> (8 * (j & 1));
          const uint32_t y = reinterpret_cast<const uint32_t*>(&vw[1])[2 * g + j / 2] >> (8 * (j & 1));
          const uint4 vf = make_uint4(x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u);
          o[n][g][j] = mfma16x16x32<true>(vf, pb, o[n][g][j]);
        }
      }
    }
  }

  // join: each wave's outputs (times its own scale) in LDS, 16 columns at a time
#pragma unroll
  for (int n = 0; n < NCB; ++n) {
    float ls = l[n], os[G];
#pragma unroll
    for (int g = 0; g < G; ++g) os[g] = ol[n][g];
#pragma unroll
    for (int sft = 16; sft < 64; sft <<= 1) {
      ls += __shfl_xor(ls, sft, 64);
#pragma unroll
      for (int g = 0; g < G; ++g) os[g] += __shfl_xor(os[g], sft, 64);
    }
    if (n > 0) __syncthreads();
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float* dst = &s_o[wave][lq][KV4_GROUP * g + 16 * gq + 4 * r];
#pragma unroll
        for (int j = 0; j < 4; ++j) dst[j] = ldexpf(o[n][g][j][r], 24 - ve) + os[g];
      }
    if (gq == 0) {
      s_m[wave][lq] = m[n] == -__builtin_inff() ? m[n] : m[n] * fl[n];
      s_l[wave][lq] = ls;
    }
    __syncthreads();
    // 16 threads per column, D / 16 dims each
    constexpr int DT = D / 16;
    const int col = tid >> 4, part = tid & 15, c = c0 + 16 * n + col;
    if (c < cols) {
      float M = s_m[0][col];
#pragma unroll
      for (int w = 1; w < AW; ++w) M = fmaxf(M, s_m[w][col]);
      float L = 0.f, y[DT];
#pragma unroll
      for (int e = 0; e < DT; ++e) y[e] = 0.f;
#pragma unroll
      for (int w = 0; w < AW; ++w) {
        // a wave that saw nothing has weight 0 (its sums are 0 too)
        const float f = s_m[w][col] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(s_m[w][col] - M);
        L = fmaf(f, s_l[w][col], L);
#pragma unroll
        for (int e = 0; e < DT; ++e) y[e] = fmaf(f, s_o[w][col][DT * part + e], y[e]);
      }
      if (sg.nsplit == 1) {
        const float inv = 1.0f / L;
        uint16_t* out = static_cast<uint16_t*>(a.out) + ((int64_t)sg.row0 + c / rep) * a.ldo +
                        ((int64_t)kvh * rep + c % rep) * D + DT * part;
#pragma unroll
        for (int e = 0; e < DT; e += 4)
          *reinterpret_cast<uint2*>(out + e) = make_uint2(pack_act2<F16>(y[e] * inv, y[e + 1] * inv),
                                                          pack_act2<F16>(y[e + 2] * inv, y[e + 3] * inv));
      } else {
        float* pb = a.partial + ((int64_t)sg.part0 + (int64_t)block * sg.nsplit + split) * kv4_partial_floats(NCB, D) +
                    (int64_t)(16 * n + col) * (D + 2);
        if (part == 0) {
          pb[0] = M;
          pb[1] = L;
        }
#pragma unroll
        for (int e = 0; e < DT; ++e) pb[2 + DT * part + e] = y[e];
      }
    }
  }
}

// Joins a column's pieces in piece order: one wave per column, D / 64 dims a lane.
template <int D, bool F16>
__global__ __launch_bounds__(AT) void kv4_join_kernel(Kv4Args a, int ncb16) {
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * AW + (threadIdx.x >> 6);   // column among the items'
  const int item = (int)(id / ncb16), col = (int)(id % ncb16);
  if (item >= a.nitems) return;
  const CacheSeg& sg = a.seg[find_seg(a, item)];
  const int local = item - sg.item0;
  if (sg.nsplit == 1 || local % sg.nsplit) return;
  const int block = local / sg.nsplit;
  const int rep = a.rep, cols = sg.rows * rep, ncb = (cols + ncb16 - 1) / ncb16;
  const int c = block % ncb * ncb16 + col, slot = block / ncb;
  if (c >= cols) return;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const int64_t stride = (int64_t)ncb16 * (D + 2);
  const float* pb = a.partial + ((int64_t)sg.part0 + (int64_t)block * sg.nsplit) * stride + (int64_t)col * (D + 2);
  constexpr int DL = D / 64;
  float M = -__builtin_inff(), L = 0.f, y[DL];
#pragma unroll
  for (int e = 0; e < DL; ++e) y[e] = 0.f;
  // 64 pieces at a time: a lane weighs one, then the outputs are added with the
  // weights passed around, eight loads in flight (a load that waits for the one
  // before: 26 us for 78 pieces)
  for (int s0 = 0; s0 < sg.nsplit; s0 += 64) {
    const bool there = s0 + lane < sg.nsplit;
    const float m = there ? pb[(s0 + lane) * stride] : -__builtin_inff();
    const float l = there ? pb[(s0 + lane) * stride + 1] : 0.f;
    float mn = fmaxf(M, m);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor(mn, o, 64));
    const float f = m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    const float back = M == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(M - mn);
    L = fmaf(L, back, warp_sum(f * l));
#pragma unroll
    for (int e = 0; e < DL; ++e) y[e] *= back;
    M = mn;
    const int n = min(64, sg.nsplit - s0);
#pragma unroll 8
    for (int s = 0; s < n; ++s) {
      const float* p = pb + (s0 + s) * stride + 2 + DL * lane;
      const float fs = __shfl(f, s, 64);
#pragma unroll
      for (int e = 0; e < DL; ++e) y[e] = fmaf(fs, p[e], y[e]);
    }
  }
  const float inv = 1.0f / L;
  uint16_t* out = static_cast<uint16_t*>(a.out) + ((int64_t)sg.row0 + c / rep) * a.ldo +
                  ((int64_t)kvh * rep + c % rep) * D + DL * lane;
  if constexpr (DL == 2) *reinterpret_cast<uint32_t*>(out) = pack_act2<F16>(y[0] * inv, y[1] * inv);
  else *out = f32_to_act_bits<F16>(y[0] * inv);
}

template <int D, bool F16>
hipError_t launch_attn_ncb(const Kv4Args& a, int ncb, hipStream_t st) {
  switch (ncb) {
    case 1: kv4_attn_kernel<D, F16, 1><<<a.nitems, AT, 0, st>>>(a); break;
    case 2: kv4_attn_kernel<D, F16, 2><<<a.nitems, AT, 0, st>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Args& a, int32_t head_dim, bool f16, hipStream_t st) {
  if (a.nitems <= 0) return hipSuccess;
  const int grid = (a.nitems + 1) / 2;
  if (head_dim == 128) {
    if (f16) kv4_append_kernel<128, true><<<grid, NT, 0, st>>>(a);
    else kv4_append_kernel<128, false><<<grid, NT, 0, st>>>(a);
  } else if (head_dim == 64) {
    if (f16) kv4_append_kernel<64, true><<<grid, NT, 0, st>>>(a);
    else kv4_append_kernel<64, false><<<grid, NT, 0, st>>>(a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Args& a, int32_t head_dim, bool f16, hipStream_t st) {
  if (a.nitems <= 0) return hipSuccess;
  const int grid = (a.nitems + 1) / 2;
  if (head_dim == 128) {
    if (f16) kv4_read_kernel<128, true><<<grid, NT, 0, st>>>(a);
    else kv4_read_kernel<128, false><<<grid, NT, 0, st>>>(a);
  } else if (head_dim == 64) {
    if (f16) kv4_read_kernel<64, true><<<grid, NT, 0, st>>>(a);
    else kv4_read_kernel<64, false><<<grid, NT, 0, st>>>(a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_kv4_attention(const Kv4Args& a, int32_t head_dim, bool f16, int32_t ncb,
                                hipStream_t st) {
  if (a.nitems <= 0) return hipSuccess;
  if (head_dim == 128) return f16 ? launch_attn_ncb<128, true>(a, ncb, st) : launch_attn_ncb<128, false>(a, ncb, st);
  if (head_dim == 64) return f16 ? launch_attn_ncb<64, true>(a, ncb, st) : launch_attn_ncb<64, false>(a, ncb, st);
  return hipErrorInvalidValue;
}

hipError_t launch_kv4_join(const Kv4Args& a, int32_t head_dim, bool f16, int32_t ncb,
                           hipStream_t st) {
  if (a.nitems <= 0) return hipSuccess;
  const int grid = (int)(((int64_t)a.nitems * 16 * ncb + AW - 1) / AW);
  if (head_dim == 128) {
    if (f16) kv4_join_kernel<128, true><<<grid, AT, 0, st>>>(a, 16 * ncb);
    else kv4_join_kernel<128, false><<<grid, AT, 0, st>>>(a, 16 * ncb);
  } else if (head_dim == 64) {
    if (f16) kv4_join_kernel<64, true><<<grid, AT, 0, st>>>(a, 16 * ncb);
    else kv4_join_kernel<64, false><<<grid, AT, 0, st>>>(a, 16 * ncb);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace svl
