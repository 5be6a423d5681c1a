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

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

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

// The largest 16-bit value that is not above (hi - lo) / 15, as bits: the float32
// quotient is next to it, and 15 times a candidate is exact, so it is compared with
// the difference and its error.  Only bf16's range can overflow the difference.
template <bool F16>
__device__ __forceinline__ uint32_t step_bits(float lo, float hi) {
  const float d = hi - lo, back = d - hi;
  if (!F16 && __any(d == __builtin_inff())) {
    const double q = ((double)hi - lo) / 15.0;
    const uint32_t b = f32_to_act_bits<F16>((float)q);
    if ((double)act_bits_to_f32<F16>(b) > q) return b - 1;
    return (double)act_bits_to_f32<F16>(b + 1) <= q ? b + 1 : b;
  }
  const float err = (hi - (d - back)) - (lo + back);     // hi - lo = d + err
  const uint32_t b = f32_to_act_bits<F16>(d * (1.0f / 15.0f));
  auto above = [&](uint32_t x) { return (15.0f * act_bits_to_f32<F16>(x) - d) - err > 0.f; };
  return above(b) ? b - 1 : above(b + 1) ? b : b + 1;
}

constexpr int NT = 256;   // append and read: four waves, each the K or the V half of a tile

// One wave quantises the K or V half of a tile: lane = (row, quarter), the quarter
// holding the 16-byte pieces 4 i + quarter of its row, so a load takes 64 bytes a
// row and a lane's K words are neighbours in the cache.  2 d bytes in and d / 2 + d / 16 out
// per row; bound by the issue of some 24 instructions a value (82% of the cycles):
// 15211 rows of 32 heads of 128 in bf16 95 us, 3.4 TB/s, where a copy would take 63.
// A code is exact: k, the floor of the rounded quotient, is it or one below, and
// x - lo (with the error of its subtraction, where it has one) is compared with the
// border (k + 1/2) s, which float32 holds exactly.  (Float64 where float32 is near a
// border: ties are common among values of 8 bits, 163 us; the step in float64 and the
// subtraction's error always: 101.)
template <int D, bool F16>
__global__ __launch_bounds__(NT) void kv4_append_kernel(Kv4Args a) {
  typedef Tile<D> T;
  constexpr int NP = D / 32, G = T::G, PG = NP / G;   // pieces of a lane, of them in a group
  constexpr int CS = D + 8;                           // row stride of the codes in LDS
  __shared__ __attribute__((aligned(16))) uint8_t s_code[NT / 64][KV4_TILE][CS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  uint4 w[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) w[i] = make_uint4(0, 0, 0, 0);
  if (on) {
    const int64_t row = (int64_t)sg.row0 + (tile * KV4_TILE + r - sg.pos0);
    const uint16_t* src = static_cast<const uint16_t*>(is_v ? a.v : a.k) + row * (is_v ? a.ldv : a.ldk) + kvh * D + 8 * qd;
#pragma unroll
    for (int i = 0; i < NP; ++i) w[i] = *reinterpret_cast<const uint4*>(src + 32 * i);
  }
  uint8_t* tp = tile_ptr<D>(a, sg.sample, kvh, tile);
  uint32_t words[NP];       // eight codes of each piece
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float lo = __builtin_inff(), hi = -__builtin_inff();
    u16x2 tops = {0, 0}, lows = {0xffff, 0xffff};   // magnitudes as bits: the largest, the least but 0 less 1
#pragma unroll
    for (int i = g * PG; i < (g + 1) * PG; ++i) {
      const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x0 = act_bits_to_f32<F16>(v[e] & 0xffffu), x1 = act_bits_to_f32<F16>(v[e] >> 16);
        lo = fminf(lo, fminf(x0, x1));
        hi = fmaxf(hi, fmaxf(x0, x1));
        const u16x2 m = __builtin_bit_cast(u16x2, v[e] & 0x7fff7fffu);
        tops = __builtin_elementwise_max(tops, m);
        lows = __builtin_elementwise_min(lows, u16x2(m - u16x2{1, 1}));
      }
    }
    uint32_t top = max(tops[0], tops[1]), low = min(lows[0], lows[1]);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, o, 64));
      hi = fmaxf(hi, __shfl_xor(hi, o, 64));
      top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
      low = min(low, (uint32_t)__shfl_xor((int)low, o, 64));
    }
    const bool bad = top >= (F16 ? 0x7c00u : 0x7f80u);
    const uint32_t sb = bad ? (F16 ? 0x7e00u : 0x7fc0u) : step_bits<F16>(lo, hi);
    const uint32_t lb = bad ? (F16 ? 0x7e00u : 0x7fc0u) : f32_to_act_bits<F16>(lo);
    const float s = act_bits_to_f32<F16>(sb);
    const bool flat = bad || sb == 0;
    if (on && qd == g) {
      uint32_t* par = reinterpret_cast<uint32_t*>(tp + 2 * T::CODES + (is_v ? T::PARAMS : 0));
      par[((r >> 2) * G + g) * 4 + (r & 3)] = sb | (lb << 16);
    }
    // x and lo are multiples of the least magnitude's last place and their difference is
    // below four times the largest's power of two: within these many powers of two it
    // is exact in float32 (of 1024 normal values, 93% of the cases in bf16, two thirds
    // in fp16)
    constexpr uint32_t P = F16 ? 10 : 7;
    const bool wide = (top >> P) > max((low + 1) >> P, 1u) + 22 - P;
    // RARE: otherwise its error is taken along; a step below the type's normal range
    // may leave codes above 15; bf16's reciprocal or the range itself may overflow
    // (then all is scaled by 2^100).
    auto codes = [&]<bool RARE>() __attribute__((always_inline)) {
      const float big = !RARE || F16 ? 1.f : s < 0x1p-100f ? 0x1p100f : s > 0x1p100f ? 0x1p-100f : 1.f;
      const float sx = s * big, lx = lo * big, inv = 1.0f / sx, half = 0.5f * sx;
#pragma unroll
      for (int i = g * PG; i < (g + 1) * PG; ++i) {
        const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = act_bits_to_f32<F16>(e & 1 ? v[e / 2] >> 16 : v[e / 2] & 0xffffu);
          if constexpr (RARE) x *= big;
          const float d = x - lx;
          uint32_t c = (uint32_t)(d * inv);
          float over = d - fmaf((float)c, sx, half);
          if constexpr (RARE) {
            const float back = d - x;
            over += (x - (d - back)) - (lx + back);             // x - lo = d + that
          }
          // one more above the border, and on it if that makes c even (a sum that is 0 is +0)
          c += (int)(__float_as_uint(over) + (c & 1)) > 0 ? 1u : 0u;
          if constexpr (RARE) c = min(c, 15u);
          word |= c << (4 * e);
        }
        words[i] = flat ? 0u : word;
      }
    };
    if (__any(!flat & (wide | (s < (F16 ? 0x1p-14f : 0x1p-100f)) | (s > 0x1p100f)))) codes.template operator()<true>();
    else codes.template operator()<false>();
  }
  if (!is_v) {
    // place of row word 4 i + qd: the lane's words are neighbours
    if (!on) return;
    uint32_t* dst = reinterpret_cast<uint32_t*>(tp) + r * (D / 8) + qd * T::KW;
    if constexpr (NP == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(words[0], words[1], words[2], words[3]);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(words[0], words[1]);
    return;
  }
  // V words hold two dims of four positions: exchange through LDS, and keep the
  // nibbles of positions outside this call
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    // a nibble to a byte
    const uint32_t even = words[i] & 0x0f0f0f0fu, odd = (words[i] >> 4) & 0x0f0f0f0fu;
    *reinterpret_cast<uint2*>(&s_code[wave][r][8 * (4 * i + qd)]) =
        make_uint2(__builtin_amdgcn_perm(odd, even, 0x05010400u), __builtin_amdgcn_perm(odd, even, 0x07030602u));
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
      word |= two << sh;
      const int pos = 4 * quad + p;
      if (pos >= first && pos < last) mine |= 0x0f0fu << sh;
    }
    if (mine == 0) continue;
    if (mine != 0xffffffffu) word = (word & mine) | (vw[f] & ~mine);
    vw[f] = word;
  }
}

// One wave reads back the K or V half of a tile.  K: lane = (row, quarter) as in
// the append.  V: lane = (quad of positions, 4 dims of each group), whose words are
// neighbours.  Bound by memory: 15211 rows of 32 heads of 128 68 us, 4.6 TB/s.
template <int D, bool F16>
__global__ __launch_bounds__(NT) void kv4_read_kernel(Kv4Args a) {
  typedef Tile<D> T;
  constexpr int NP = D / 32, G = T::G, PG = NP / G;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x * (NT / 128) + (wave >> 1);
  if (item >= a.nitems) return;
  const CacheSeg& sg = a.seg[find_seg(a, item)];
  const int local = item - sg.item0;
  const int slot = local % sg.kv_cnt;
  const int tile = sg.pos0 / KV4_TILE + local / sg.kv_cnt;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const uint8_t* tp = tile_ptr<D>(a, sg.sample, kvh, tile);
  auto value = [](uint32_t pair, uint32_t c) {
    return fmaf(act_bits_to_f32<F16>(pair & 0xffffu), (float)c, act_bits_to_f32<F16>(pair >> 16));
  };
  if (wave & 1) {
    const int quad = lane >> 4, L = lane & 15;
    const uint32_t* vw = reinterpret_cast<const uint32_t*>(tp + T::CODES) + lane * T::VW;
    const uint4* par = reinterpret_cast<const uint4*>(tp + 2 * T::CODES + T::PARAMS) + quad * G;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint2 x = reinterpret_cast<const uint2*>(vw)[g];
      const uint4 pr = par[g];
      const uint32_t pairs[4] = {pr.x, pr.y, pr.z, pr.w};
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int pos = tile * KV4_TILE + 4 * quad + p, sh = 4 * (p >> 1) + 16 * (p & 1);
        if (pos < sg.pos0 || pos >= sg.pos0 + sg.rows) continue;
        uint16_t* dst = static_cast<uint16_t*>(a.v_out) + ((int64_t)sg.row0 + pos - sg.pos0) * a.ldv + kvh * D +
                        KV4_GROUP * g + 4 * L;
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(pack_act2<F16>(value(pairs[p], (x.x >> sh) & 15u), value(pairs[p], (x.x >> (sh + 8)) & 15u)),
                       pack_act2<F16>(value(pairs[p], (x.y >> sh) & 15u), value(pairs[p], (x.y >> (sh + 8)) & 15u)));
      }
    }
    return;
  }
  const int r = lane >> 2, qd = lane & 3;
  const int pos = tile * KV4_TILE + r;
  if (pos < sg.pos0 || pos >= sg.pos0 + sg.rows) return;
  const uint32_t* par = reinterpret_cast<const uint32_t*>(tp + 2 * T::CODES) + (r >> 2) * G * 4 + (r & 3);
  uint32_t words[NP];
  const uint32_t* kw = reinterpret_cast<const uint32_t*>(tp) + r * (D / 8) + qd * T::KW;
  if constexpr (NP == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(kw);
    words[0] = x.x, words[1] = x.y, words[2] = x.z, words[3] = x.w;
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(kw);
    words[0] = x.x, words[1] = x.y;
  }
  uint16_t* dst = static_cast<uint16_t*>(a.k_out) + ((int64_t)sg.row0 + pos - sg.pos0) * a.ldk + kvh * D + 8 * qd;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const uint32_t pair = par[i / PG * 4], x = words[i];
    uint32_t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      y[e] = pack_act2<F16>(value(pair, (x >> (8 * e)) & 15u), value(pair, (x >> (8 * e + 4)) & 15u));
    *reinterpret_cast<uint4*>(dst + 32 * i) = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

// ---------------------------------------------------------------- attention
// One workgroup: up to 16 columns (query row, head of the K/V head's group) of
// one K/V head, over one piece of the visible positions; four waves take 32
// positions (a unit) in turn, each with a running maximum and sum, and are joined
// at the end.  (32 columns share what is made of the codes but hold twice the sums,
// with half the waves: two chunks of 512 rows at 4096 and 3000 positions, 32 heads
// on 8, take 307 us in place of 232, and four of 64 at 900 53 in place of 20.)
//
// The products run on the codes themselves.  A nibble in the low ten bits of a
// half word is an fp16 subnormal, c 2^-24 (or c 2^-20 four bits higher), and the
// matrix cores keep subnormals, so one AND makes an operand pair of two codes.
// Scores: S^T = C Q^T per group of 64 dims, C the K codes (positions x dims), Q
// the query scaled by a power of two into fp16 (exact to 2^-35 of its largest
// value), then s S + lo sum(q) per position and group, in float32.
// Values: O^T = V^T P'^T per group with P' = p s, rounded to fp16 once, plus
// sum(p lo) in float32.  So neither K nor V is rounded to 16 bits on the way.
// What the rounding takes from P' is put back for the mean code, 7.5, in float32:
// what is left meets codes of mean 0 (error against float64 2.0 -> 1.35 times that
// of one rounding of the output, at no cost in time).
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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int N> struct Words;
template <> struct Words<4> { typedef u32x4 type; };
template <> struct Words<2> { typedef u32x2 type; };

template <int N>
__device__ __forceinline__ typename Words<N>::type load_words(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff) {
  if constexpr (N == 4) return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0));
  else return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, voff, soff, 0));
}

// Maximum over the four lanes of a column (lane, lane ^ 16, lane ^ 32, lane ^ 48).
__device__ __forceinline__ float column_max(float x) {
  const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Two codes of a word as fp16 subnormals: nibbles 0 and 4 (c 2^-24), 1 and 5 (c 2^-20).
__device__ __forceinline__ u32x4 four_pairs(uint32_t w) {
  return u32x4{w & 0x000f000fu, w & 0x00f000f0u, (w >> 8) & 0x000f000fu, (w >> 8) & 0x00f000f0u};
}

__device__ __forceinline__ floatx4 mfma_codes(const u32x4& a, const u32x4& b, const floatx4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t round_pair(float lo, float hi) { return pack_act2<true>(lo, hi); }

template <int D, bool F16>
__global__ __launch_bounds__(AT, 2) void kv4_attn_kernel(Kv4Args a) {
  typedef Tile<D> T;
  constexpr int G = T::G, NS = D / 32;
  typedef typename Words<T::KW>::type CodeWords;   // (K and V: as many words a lane)
  static_assert(T::KW == T::VW, "code words of a lane");
  __shared__ float s_o[AW][16][D + 4];
  __shared__ float s_m[AW][16], s_l[AW][16];
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const CacheSeg& sg = a.seg[find_seg(a, item)];
  const int rep = a.rep, cols = sg.rows * rep, ncb = (cols + KV4_COLS - 1) / KV4_COLS;
  const int local = item - sg.item0, split = local % sg.nsplit, block = local / sg.nsplit;
  const int cb = block % ncb, slot = block / ncb;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = lane >> 4, lq = lane & 15;
  const int c0 = cb * KV4_COLS;
  const int p_lo = sg.pos0 + c0 / rep, p_hi = sg.pos0 + (min(c0 + KV4_COLS, cols) - 1) / rep;
  const Units un = units_of(p_lo, p_hi, a.window, a.sinks);
  const int u0 = (int)((int64_t)un.n * split / sg.nsplit);
  const int u1 = (int)((int64_t)un.n * (split + 1) / sg.nsplit);

  // query fragments; a pair of codes is (dim i, dim i + 4) of a word, the pairs
  // 1 and 3 carry a factor 16
  const float sl2 = a.scale * 1.4426950408889634f;   // scores in log2 units
  u32x4 qf[NS];
  float qs[G], fl;
  int pq;                              // the column's position
  {
    const int c = c0 + lq;
    const bool on = c < cols;
    const int i = on ? c / rep : 0, h = kvh * rep + (on ? c % rep : 0);
    pq = on ? sg.pos0 + i : -1;
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((int64_t)sg.row0 + i) * a.ldq +
                         (int64_t)h * D + 8 * gq;
    float x[NS][8];
    float top = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) qs[g] = 0.f;
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
        qs[s / 2] += x[s][e];
        top = fmaxf(top, fabsf(x[s][e]));
      }
    }
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
      top = fmaxf(top, __shfl_xor(top, o, 64));
#pragma unroll
      for (int g = 0; g < G; ++g) qs[g] += __shfl_xor(qs[g], o, 64);
    }
    // 2^k brings the largest magnitude into [2^14, 2^15)
    const int k = top > 0.f ? max(-100, min(100, 141 - (int)(__float_as_uint(top) >> 23))) : 0;
    const float up = pow2f(k);
    fl = ldexpf(sl2, 24 - k);
#pragma unroll
    for (int g = 0; g < G; ++g) qs[g] *= pow2f(k - 24);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const float* y = x[s];
      const float up4 = up * 0.0625f;
      qf[s] = u32x4{round_pair(y[0] * up, y[4] * up), round_pair(y[1] * up4, y[5] * up4),
                    round_pair(y[2] * up, y[6] * up), round_pair(y[3] * up4, y[7] * up4)};
    }
  }

  float m = -__builtin_inff(), l = 0.f, ol[G];
  floatx4 o[G][4];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    ol[g] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[g][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  // P' = p s 2^ve follows the largest scale seen, so that it is in fp16's normal range for
  // weights down to 2^-24 whatever the size of V (a fixed factor of 4, which fits any
  // fp16 scale, loses the digits of small values and of long tails behind a first key)
  int ve = 126;

  // a head's cache is below 2^28 bytes; tiles past its end (the second of the last
  // unit) read as zeros
  const __amdgpu_buffer_rsrc_t head = make_rsrc(tile_ptr<D>(a, sg.sample, kvh, 0), (uint32_t)(a.tiles * T::BYTES));
  const uint32_t at_k = (lq * 4 + gq) * T::KW * 4, at_v = T::CODES + lane * T::VW * 4;
  const uint32_t at_p = 2 * T::CODES + gq * G * 16;
  const int wlim = a.window > 0 ? a.window : 1 << 30;   // (positions are below 2^20)

  struct Loaded {
    CodeWords kw[2], vw[2];
    u32x4 kp[2][G], vp[2][G];
  };
  auto load = [&](int unit) __attribute__((always_inline)) {
    Loaded x;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint32_t tile = (uint32_t)(2 * unit + t) * T::BYTES;
      x.kw[t] = load_words<T::KW>(head, at_k, tile);
#pragma unroll
      for (int g = 0; g < G; ++g) x.kp[t][g] = load_words<4>(head, at_p + 16 * g, tile);
      x.vw[t] = load_words<T::VW>(head, at_v, tile);
#pragma unroll
      for (int g = 0; g < G; ++g) x.vp[t][g] = load_words<4>(head, at_p + T::PARAMS + 16 * g, tile);
    }
    return x;
  };
  // One unit; PART: some column does not see some position of it.
  auto unit_of = [&](int u) { return u < un.us ? u : un.uw + (u - un.us); };
  auto add_unit = [&]<bool PART>(Loaded x, int kv0) __attribute__((always_inline)) {
    uint32_t vis = 0xffu;
    if constexpr (PART) {
      // a position that the column does not see may hold anything: neither its values
      // nor its scale may count
      vis = 0;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = kv0 + 16 * t + 4 * gq + r;
          const bool ok = (j <= pq) & ((j > pq - wlim) | (j < a.sinks));   // (no short cuts: branches)
          vis |= (uint32_t)ok << (4 * t + r);
#pragma unroll
          for (int g = 0; g < G; ++g) x.vp[t][g][r] = ok ? x.vp[t][g][r] : 0u;
        }
    }
    u32x4 kf[2][NS];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < NS; ++s) kf[t][s] = four_pairs(x.kw[t][s]);
    {
      float vmax = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r) vmax = fmaxf(vmax, act_bits_to_f32<F16>(x.vp[t][g][r] & 0xffffu));
      vmax = column_max(vmax);
      // scales below 2^(e + 1) with e the largest one's exponent: P' < 2^15
      const int want = max(-126, min(126, 14 - ((int)(__float_as_uint(vmax) >> 23) - 127)));
      if (__any(want < ve)) {   // (a column's own)
        const float f = ldexpf(1.0f, min(want - ve, 0));
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[g][j] *= f;
        ve = min(ve, want);
      }
    }
    const float pf0 = pow2f(ve), pf1 = pf0 * 0.0625f;
    const float back0 = -7.5f * pow2f(-ve), back1 = 16.f * back0;
    float sc[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx4 acc[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        acc[g] = mfma_codes(kf[t][2 * g], qf[2 * g], floatx4{0.f, 0.f, 0.f, 0.f});
        acc[g] = mfma_codes(kf[t][2 * g + 1], qf[2 * g + 1], acc[g]);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t pw = x.kp[t][g][r];
          v = fmaf(act_bits_to_f32<F16>(pw & 0xffffu), acc[g][r], v);
          v = fmaf(act_bits_to_f32<F16>(pw >> 16), qs[g], v);
        }
        sc[t][r] = v;
      }
    }
    if constexpr (PART) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[t][r] = (vis >> (4 * t + r)) & 1 ? sc[t][r] : -__builtin_inff();
    }
    float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                     fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
    mx = column_max(mx);
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f((m - mn) * fl);
      l *= alpha;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        ol[g] *= alpha;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[g][j] *= alpha;
      }
      m = mn;
    }
    const float mf = m == -__builtin_inff() ? 0.f : -m * fl;   // nothing above -inf yet: 0
    float p[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[t][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][r], fl, mf));
        l += p[t][r];
      }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float ps[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t pw = x.vp[t][g][r];
          const float vs = act_bits_to_f32<F16>(pw & 0xffffu);
          ol[g] = fmaf(p[t][r], fmaf(vs, 7.5f, act_bits_to_f32<F16>(pw >> 16)), ol[g]);
          ps[t][r] = p[t][r] * (r < 2 ? pf0 : pf1) * vs;
        }
      const u32x4 pb = {round_pair(ps[0][0], ps[0][1]), round_pair(ps[0][2], ps[0][3]),
                        round_pair(ps[1][0], ps[1][1]), round_pair(ps[1][2], ps[1][3])};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float back = i & 1 ? back1 : back0;
        ol[g] = fmaf(act_bits_to_f32<true>(pb[i] & 0xffffu), back, ol[g]);
        ol[g] = fmaf(act_bits_to_f32<true>(pb[i] >> 16), back, ol[g]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t y = x.vw[0][2 * g + j / 2] >> (8 * (j & 1)), z = x.vw[1][2 * g + j / 2] >> (8 * (j & 1));
        o[g][j] = mfma_codes(u32x4{y & 0x000f000fu, y & 0x00f000f0u, z & 0x000f000fu, z & 0x00f000f0u}, pb, o[g][j]);
      }
    }
  };
  // whether every column sees every position of a unit
  const int whole_hi = p_lo - UNIT + 1, whole_lo = a.window > 0 ? p_hi - a.window : -1, whole_sink = a.sinks - UNIT;
  int u = u0 + wave;
  if (u < u1) {
    Loaded next = load(unit_of(u));
    for (; u < u1; u += AW) {
      const Loaded x = next;
      const int kv0 = unit_of(u) * UNIT;
      // the next unit in flight meanwhile (8 x 8192 positions of 32 heads: 86 -> 71 us)
      next = load(unit_of(min(u + AW, u1 - 1)));
      if (kv0 <= whole_hi && (kv0 > whole_lo || kv0 <= whole_sink)) add_unit.template operator()<false>(x, kv0);
      else add_unit.template operator()<true>(x, kv0);
    }
  }

  // join: each wave's outputs (times its own scale) in LDS
  float ls = l, os[G];
#pragma unroll
  for (int g = 0; g < G; ++g) os[g] = ol[g];
#pragma unroll
  for (int sft = 16; sft < 64; sft <<= 1) {
    ls += __shfl_xor(ls, sft, 64);
#pragma unroll
    for (int g = 0; g < G; ++g) os[g] += __shfl_xor(os[g], sft, 64);
  }
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float* dst = &s_o[wave][lq][KV4_GROUP * g + 16 * gq + 4 * r];
#pragma unroll
      for (int j = 0; j < 4; ++j) dst[j] = ldexpf(o[g][j][r], 24 - ve) + os[g];
    }
  if (gq == 0) {
    s_m[wave][lq] = m == -__builtin_inff() ? m : m * fl;
    s_l[wave][lq] = ls;
  }
  __syncthreads();
  // 16 threads per column, D / 16 dims each
  constexpr int DT = D / 16;
  const int col = tid >> 4, part = tid & 15, c = c0 + col;
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
      float* pb = a.partial + ((int64_t)sg.part0 + (int64_t)block * sg.nsplit + split) * kv4_partial_floats(D) +
                  (int64_t)col * (D + 2);
      if (part == 0) {
        pb[0] = M;
        pb[1] = L;
      }
#pragma unroll
      for (int e = 0; e < DT; ++e) pb[2 + DT * part + e] = y[e];
    }
  }
}

// Joins the pieces of one column of a cut block, in piece order within each of four
// waves.  Bound by latency: the pieces' maxima are weighed at once, their outputs
// read eight at a time per wave (78 pieces by one wave, a load after the other: 26 us).
template <int D, bool F16>
__global__ __launch_bounds__(AT) void kv4_join_kernel(Kv4Args a) {
  constexpr int DL = D / 64;
  __shared__ float s_f[KV4_MAX_PIECES];
  __shared__ float s_red[2][AW], s_y[AW][D];
  int k = 0;
  for (int lo = 0, hi = a.nsegs - 1; lo <= hi;) {   // the last segment that begins at or before the block
    const int mid = (lo + hi) >> 1;
    if (a.seg[mid].join0 <= (int)blockIdx.x) k = mid, lo = mid + 1; else hi = mid - 1;
  }
  const CacheSeg& sg = a.seg[k];
  const int block = (int)blockIdx.x - sg.join0, n = sg.nsplit;
  const int rep = a.rep, cols = sg.rows * rep, ncb = (cols + KV4_COLS - 1) / KV4_COLS;
  const int col = blockIdx.y, c = block % ncb * KV4_COLS + col, slot = block / ncb;
  if (c >= cols) return;
  const int kvh = a.kv_table ? a.kv_table[sg.kv_off + slot] : slot;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t stride = (int64_t)KV4_COLS * (D + 2);
  const float* pb = a.partial + ((int64_t)sg.part0 + (int64_t)block * n) * stride + (int64_t)col * (D + 2);
  float M = -__builtin_inff();
  for (int s = tid; s < n; s += AT) {
    s_f[s] = pb[s * stride];
    M = fmaxf(M, s_f[s]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  if (lane == 0) s_red[0][wave] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < AW; ++w) M = fmaxf(M, s_red[0][w]);
  float L = 0.f;
  for (int s = tid; s < n; s += AT) {
    const float f = s_f[s] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(s_f[s] - M);
    s_f[s] = f;
    L = fmaf(f, pb[s * stride + 1], L);
  }
  L = warp_sum(L);
  if (lane == 0) s_red[1][wave] = L;
  __syncthreads();
  float y[DL];
#pragma unroll
  for (int e = 0; e < DL; ++e) y[e] = 0.f;
#pragma unroll 8
  for (int s = wave; s < n; s += AW) {
    const float* p = pb + s * stride + 2 + DL * lane;
    const float f = s_f[s];
#pragma unroll
    for (int e = 0; e < DL; ++e) y[e] = fmaf(f, p[e], y[e]);
  }
#pragma unroll
  for (int e = 0; e < DL; ++e) s_y[wave][DL * lane + e] = y[e];
  __syncthreads();
  if (wave) return;
  L = s_red[1][0] + s_red[1][1] + s_red[1][2] + s_red[1][3];
  const float inv = 1.0f / L;
#pragma unroll
  for (int e = 0; e < DL; ++e) {
    y[e] = 0.f;
#pragma unroll
    for (int w = 0; w < AW; ++w) y[e] += s_y[w][DL * lane + e];
    y[e] *= inv;
  }
  uint16_t* out = static_cast<uint16_t*>(a.out) + ((int64_t)sg.row0 + c / rep) * a.ldo +
                  ((int64_t)kvh * rep + c % rep) * D + DL * lane;
  if constexpr (DL == 2) *reinterpret_cast<uint32_t*>(out) = pack_act2<F16>(y[0], y[1]);
  else *out = f32_to_act_bits<F16>(y[0]);
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

hipError_t launch_kv4_attention(const Kv4Args& a, int32_t head_dim, bool f16, hipStream_t st) {
  if (a.nitems <= 0) return hipSuccess;
  if (head_dim == 128) {
    if (f16) kv4_attn_kernel<128, true><<<a.nitems, AT, 0, st>>>(a);
    else kv4_attn_kernel<128, false><<<a.nitems, AT, 0, st>>>(a);
  } else if (head_dim == 64) {
    if (f16) kv4_attn_kernel<64, true><<<a.nitems, AT, 0, st>>>(a);
    else kv4_attn_kernel<64, false><<<a.nitems, AT, 0, st>>>(a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_kv4_join(const Kv4Args& a, int32_t head_dim, bool f16, int32_t blocks,
                           int32_t columns, hipStream_t st) {
  if (blocks <= 0) return hipSuccess;
  const dim3 grid((unsigned)blocks, (unsigned)columns);
  if (head_dim == 128) {
    if (f16) kv4_join_kernel<128, true><<<grid, AT, 0, st>>>(a);
    else kv4_join_kernel<128, false><<<grid, AT, 0, st>>>(a);
  } else if (head_dim == 64) {
    if (f16) kv4_join_kernel<64, true><<<grid, AT, 0, st>>>(a);
    else kv4_join_kernel<64, false><<<grid, AT, 0, st>>>(a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace svl
