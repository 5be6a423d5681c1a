// Gradients of the windowed attention (window_attn.hip) on 16-bit MFMA, from the
// rows' log-sums: P = exp(scale q.k - lse), D = rowsum(dO * O), dP = dO V^T,
// dS = P (dP - D), then dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.  Sums,
// P, dP and dS are float32; P and dS are rounded to 16 bits once, as operands.
//
// Two launches, so that every sum has one owner and a fixed order (no atomics):
// the query gradient by tiles of query rows, the key and value gradients by
// tiles of keys; S and dP are formed in both.
//
// fp16: dS is scaled by a power of two into fp16's range, from the largest
// gradient of the row (dQ) or of the rows so far (dK), and further down where
// that does not hold it; the factor is taken out in float32.
//
// An inf or NaN of a row or key must not reach those that it is masked from (0
// times inf): in tiles that are partly masked, such values are 0 in the operands
// that mix rows or keys, and what sees them is made NaN by itself.
#include "window_attn.h"

namespace svl {
namespace {

constexpr int NT = 256;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Query gradient: four waves of 32 query rows against tiles of 64 keys.
// S^T = K Q^T and dP^T = V dO^T (keys x queries), dQ^T += K^T dS^T with K read
// transposed from LDS.
template <int D, bool F16>
__global__ __launch_bounds__(NT, 2) void window_dq_kernel(WinBwdArgs a) {
  constexpr int BQ = 128, BK = WIN_BK;
  constexpr int KS = D + 32, VS = D + 8;
  constexpr int NS = D / 16, NB = D / 32;
  constexpr int PR = D / 8, LD = BK * PR / NT;
  __shared__ __attribute__((aligned(16))) uint16_t Ks[BK * KS];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[BK * VS];
  __shared__ uint32_t s_bad[2][2];     // keys of a tile with an inf or NaN in K
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const WinBwdSeg& sg = a.seg[find_item_seg(a, item)];
  const int local = item - sg.item0;
  int h = local % a.n_heads;
  if (a.n_heads % 8 == 0) h = h % 8 * (a.n_heads / 8) + h / 8;   // as in the forward
  const int nqt = (sg.nq + BQ - 1) / BQ;
  const int qt = nqt - 1 - local / a.n_heads;
  const int kvh = h / (a.n_heads / a.n_kv_heads);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, lq = lane & 31;
  const int off = sg.nk - sg.nq;
  const int i0 = qt * BQ, qi = i0 + 32 * wave + lq;
  const bool on = qi < sg.nq;
  const int p = on ? off + qi : -1;
  const int p_lo = off + i0, p_hi = off + min(i0 + BQ, sg.nq) - 1;
  const int w_lo = off + i0 + 32 * wave, w_hi = min(w_lo + 31, p_hi);
  const int64_t row = (int64_t)sg.q0 + (on ? qi : 0);

  u32x4 qf[NS], gf[NS];
  float delta = 0.f;
  uint32_t top = 0;
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + row * a.ldq + (int64_t)h * D + 8 * half;
    const uint16_t* gp = static_cast<const uint16_t*>(a.grad) + row * a.ldg + (int64_t)h * D + 8 * half;
    const uint16_t* op = static_cast<const uint16_t*>(a.out) + row * a.ldo + (int64_t)h * D + 8 * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = load_piece(qp + 16 * s);
      gf[s] = load_piece(gp + 16 * s);
      const u32x4 o = load_piece(op + 16 * s);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        delta = fmaf(act_bits_to_f32<F16>(gf[s][e] & 0xffffu), act_bits_to_f32<F16>(o[e] & 0xffffu), delta);
        delta = fmaf(act_bits_to_f32<F16>(gf[s][e] >> 16), act_bits_to_f32<F16>(o[e] >> 16), delta);
        top = max(top, max(gf[s][e] & 0x7fffu, (gf[s][e] >> 16) & 0x7fffu));
      }
    }
  }
  delta += __shfl_xor(delta, 32, 64);
  top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
  const float lse2 = a.lse[row * a.n_heads + h] * kLog2e;
  // fp16: dS 2^-ex, which brings the row's largest gradient into [1, 2) (a row of
  // zeros, or with an inf or NaN, asks for nothing: fp16's smallest exponent)
  int ex = 0;
  if constexpr (F16)
    ex = top > 0 && top < kNonfinite<true> ? (int)(__float_as_uint(act_bits_to_f32<true>(top)) >> 23) - 127 : -24;
  if (on && half == 0) {
    a.delta[row * a.n_heads + h] = delta;
    if constexpr (F16) a.expo[row * a.n_heads + h] = ex;
  }
  int down = 0;                  // fp16: and 2^-down more, for the whole wave
  float fac = F16 ? pow2f(-ex) : 1.f;

  const uint16_t* kbase = static_cast<const uint16_t*>(a.k) + (int64_t)sg.k0 * a.ldk + (int64_t)kvh * D;
  const uint16_t* vbase = static_cast<const uint16_t*>(a.v) + (int64_t)sg.k0 * a.ldv + (int64_t)kvh * D;
  const uint8_t* mask = a.key_mask ? a.key_mask + sg.k0 : nullptr;
  const int start = a.window > 0 ? max(0, p_lo - a.window + 1) : 0;
  const int uw = start / BK, us = min((min(a.sinks, start) + BK - 1) / BK, uw);
  const int ntiles = us + p_hi / BK + 1 - uw;
  auto tile_of = [&](int u) { return (u < us ? u : uw + u - us) * BK; };
  u32x4 kr[LD], vr[LD];
  auto load = [&](int kv0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int task = tid + i * NT, r = min(kv0 + task / PR, sg.nk - 1), c = task % PR;
      kr[i] = load_piece(kbase + (int64_t)r * a.ldk + 8 * c);
      vr[i] = load_piece(vbase + (int64_t)r * a.ldv + 8 * c);
    }
  };
  floatx16 dq[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[b][r] = 0.f;
  const float sl2 = a.scale * kLog2e;
  bool poison = false;

  if (tid < 4) s_bad[tid >> 1][tid & 1] = 0;
  load(tile_of(0));
  for (int u = 0; u < ntiles; ++u) {
    const int kv0 = tile_of(u);
    const bool whole = kv0 + BK - 1 <= p_lo && (a.window <= 0 || kv0 > p_hi - a.window || kv0 + BK <= a.sinks);
    uint64_t seen = ~uint64_t(0);
    if (mask) seen = __ballot(mask[min(kv0 + lane, sg.nk - 1)] != 0);
    const bool partial = !whole || seen != ~uint64_t(0);
    __syncthreads();
    if (tid < 2) s_bad[(u + 1) & 1][tid] = 0;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int task = tid + i * NT, r = task / PR, c = task % PR;
      if (partial && any_nonfinite<F16>(kr[i])) {
        kr[i] = finite_part<F16>(kr[i]);
        atomicOr(&s_bad[u & 1][r >> 5], 1u << (r & 31));
      }
      *reinterpret_cast<u32x4*>(&Ks[r * KS + 8 * c]) = kr[i];
      *reinterpret_cast<u32x4*>(&Vs[r * VS + 8 * c]) = vr[i];
    }
    __syncthreads();
    load(tile_of(min(u + 1, ntiles - 1)));
    if (kv0 > w_hi || (a.window > 0 && kv0 + BK - 1 <= w_lo - a.window && kv0 >= a.sinks)) continue;

    const uint16_t* kt = &Ks[(4 * half + (lane & 15) / 4) * KS + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      floatx16 st, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = dp[r] = 0.f;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        st = mfma32x32x16<F16>(*reinterpret_cast<const u32x4*>(&Ks[(32 * kb + lq) * KS + 16 * s + 8 * half]), qf[s], st);
        dp = mfma32x32x16<F16>(*reinterpret_cast<const u32x4*>(&Vs[(32 * kb + lq) * VS + 16 * s + 8 * half]), gf[s], dp);
      }
      uint32_t see = 0xffffffffu, bad = 0;
      if (partial) {
        see = (uint32_t)(seen >> (32 * kb));
        bad = s_bad[u & 1][kb];
      }
      float big = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = exp2f(fmaf(st[r], sl2, -lse2)) * ((dp[r] - delta) * fac);
        if (partial) {
          const int jl = 8 * (r / 4) + 4 * half + r % 4, j = kv0 + 32 * kb + jl;
          const bool ok = j <= p && (a.window <= 0 || j > p - a.window || j < a.sinks) && ((see >> jl) & 1);
          x = ok ? x : 0.f;
          poison |= ok && ((bad >> jl) & 1);
        }
        st[r] = x;
        if constexpr (F16) big = fmaxf(big, fabsf(x));
      }
      if constexpr (F16) {
        if (__any(big > 32768.f)) {
          big = big < __builtin_inff() ? big : 0.f;   // an inf is its row's own
#pragma unroll
          for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
          const int more = max(0, min((int)(__float_as_uint(big) >> 23) - 127 - 10, 120));
          const float f = pow2f(-more);
          down += more;
          fac *= f;
#pragma unroll
          for (int r = 0; r < 16; ++r) st[r] *= f;
#pragma unroll
          for (int b = 0; b < NB; ++b) dq[b] *= f;
        }
      }
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const int t = 2 * kb + t2, r = 8 * t2;
        const u32x4 pb = {pack_act2<F16>(st[r], st[r + 1]), pack_act2<F16>(st[r + 2], st[r + 3]),
                          pack_act2<F16>(st[r + 4], st[r + 5]), pack_act2<F16>(st[r + 6], st[r + 7])};
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          const uint2 x = lds_read_tr(kt + 16 * t * KS + 32 * c), y = lds_read_tr(kt + (16 * t + 8) * KS + 32 * c);
          dq[c] = mfma32x32x16<F16>(u32x4{x.x, x.y, y.x, y.y}, pb, dq[c]);
        }
      }
    }
  }
  poison = poison || __shfl_xor((int)poison, 32, 64);
  if (!on) return;
  const float f = poison ? __builtin_nanf("") : a.scale;
  uint16_t* out = static_cast<uint16_t*>(a.dq) + row * a.lddq + (int64_t)h * D;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = F16 ? ldexpf(dq[b][4 * g + e] * f, ex + down) : dq[b][4 * g + e] * f;
      *reinterpret_cast<uint2*>(out + 32 * b + 8 * g + 4 * half) =
          make_uint2(pack_act2<F16>(y[0], y[1]), pack_act2<F16>(y[2], y[3]));
    }
}

// The (query head, tile of query rows) list of a key tile: heads of the group,
// each with the tiles [qt0, qt1) of its rows that see some key of the tile.
__device__ __forceinline__ void rows_of_tile(const WinBwdArgs& a, const WinBwdSeg& sg, int kt, int& qt0, int& qt1) {
  const int off = sg.nk - sg.nq, j0 = kt * WIN_DK, j1 = min(j0 + WIN_DK, sg.nk) - 1;
  const int first = max(0, j0 - off);
  int64_t end = sg.nq;
  if (a.window > 0 && j0 >= a.sinks) end = min(end, (int64_t)j1 + a.window - off);
  qt0 = first / WIN_DQ;
  qt1 = end > first ? (int)((end + WIN_DQ - 1) / WIN_DQ) : qt0;
}

// A work item of the key / value gradient: key tile, piece, and where its partial
// block is (-1: it has the whole list and writes the gradient itself).
struct DkvItem {
  int kvh, kt, piece, pieces;
  int64_t part;
};
__device__ __forceinline__ DkvItem dkv_item(const WinBwdArgs& a, const WinBwdSeg& sg, int local) {
  const int nkt = (sg.nk + WIN_DK - 1) / WIN_DK, sink = sg.nst * sg.ps, other = (nkt - sg.nst) * sg.po;
  DkvItem it;
  it.kvh = local % a.n_kv_heads;
  const int x = local / a.n_kv_heads;       // piece of the head, the long sink tiles first
  const bool is_sink = x < sink;
  const int y = is_sink ? x : x - sink;
  it.pieces = is_sink ? sg.ps : sg.po;
  it.kt = (is_sink ? 0 : sg.nst) + y / it.pieces;
  it.piece = y % it.pieces;
  it.part = it.pieces == 1 ? -1
            : is_sink      ? (int64_t)sg.part0 + (int64_t)it.kvh * sink + y
                           : (int64_t)sg.part1 + (int64_t)it.kvh * other + y;
  return it;
}

// Key and value gradients: four waves of 32 keys against tiles of 32 query rows.
// S = Q K^T and dP = dO V^T (queries x keys) with the wave's K and V in
// registers, then dV^T += dO^T P and dK^T += Q^T dS with the rows read transposed
// from LDS.
template <int D, bool F16>
__global__ __launch_bounds__(NT, 1) void window_dkv_kernel(WinBwdArgs a) {
  constexpr int RS = D + 32;           // row stride of the staged rows
  constexpr int NS = D / 16, NB = D / 32;
  constexpr int PR = D / 8, LD = WIN_DQ * PR / NT;
  __shared__ __attribute__((aligned(16))) uint16_t Qs[WIN_DQ * RS];
  __shared__ __attribute__((aligned(16))) uint16_t Gs[WIN_DQ * RS];
  __shared__ __attribute__((aligned(16))) float s_lse[WIN_DQ], s_delta[WIN_DQ];
  __shared__ int s_expo[WIN_DQ];
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const WinBwdSeg& sg = a.seg[find_item_seg(a, item)];
  const DkvItem it = dkv_item(a, sg, item - sg.item0);
  const int rep = a.n_heads / a.n_kv_heads, kvh = it.kvh;
  int qt0, qt1;
  rows_of_tile(a, sg, it.kt, qt0, qt1);
  const int ntq = qt1 - qt0;
  const int64_t total = (int64_t)rep * ntq;
  const int x0 = (int)(total * it.piece / it.pieces), x1 = (int)(total * (it.piece + 1) / it.pieces);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, lk = lane & 31;
  const int off = sg.nk - sg.nq;
  const int j0 = it.kt * WIN_DK, jw = j0 + 32 * wave, j = jw + lk;
  const bool on = j < sg.nk;
  const int64_t krow = (int64_t)sg.k0 + (on ? j : sg.nk - 1);
  const bool open = on && (!a.key_mask || a.key_mask[krow]);

  u32x4 kf[NS], vf[NS];
  {
    const uint16_t* kp = static_cast<const uint16_t*>(a.k) + krow * a.ldk + (int64_t)kvh * D + 8 * half;
    const uint16_t* vp = static_cast<const uint16_t*>(a.v) + krow * a.ldv + (int64_t)kvh * D + 8 * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      kf[s] = load_piece(kp + 16 * s);
      vf[s] = load_piece(vp + 16 * s);
    }
  }
  floatx16 dk[NB], dv[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.f;
  const float sl2 = a.scale * kLog2e;
  int ex = -126;                       // fp16: dS 2^-ex, the same in every lane of the wave
  float fac = 1.f;

  u32x4 qr[LD], gr[LD];
  float lse_r = 0.f, delta_r = 0.f;
  int expo_r = 0;
  auto load = [&](int x) __attribute__((always_inline)) {
    const int h = kvh * rep + x / ntq, i0 = (qt0 + x % ntq) * WIN_DQ;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int task = tid + i * NT, c = task % PR;
      const int64_t row = (int64_t)sg.q0 + min(i0 + task / PR, sg.nq - 1);
      qr[i] = load_piece(static_cast<const uint16_t*>(a.q) + row * a.ldq + (int64_t)h * D + 8 * c);
      gr[i] = load_piece(static_cast<const uint16_t*>(a.grad) + row * a.ldg + (int64_t)h * D + 8 * c);
    }
    if (tid < WIN_DQ) {
      const int64_t at = ((int64_t)sg.q0 + min(i0 + tid, sg.nq - 1)) * a.n_heads + h;
      lse_r = a.lse[at];
      delta_r = a.delta[at];
      if constexpr (F16) expo_r = a.expo[at];
    }
  };
  if (x0 < x1) load(x0);
  for (int x = x0; x < x1; ++x) {
    const int i0 = (qt0 + x % ntq) * WIN_DQ;
    const int p_lo = off + i0, p_hi = off + min(i0 + WIN_DQ, sg.nq) - 1;
    // whether every row sees every key of the workgroup
    const bool whole = i0 + WIN_DQ <= sg.nq && j0 + WIN_DK - 1 <= p_lo && j0 + WIN_DK <= sg.nk &&
                             (a.window <= 0 || j0 > p_hi - a.window || j0 + WIN_DK <= a.sinks) && !a.key_mask;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int task = tid + i * NT, r = task / PR, c = task % PR;
      if (!whole) {
        qr[i] = finite_part<F16>(qr[i]);
        gr[i] = finite_part<F16>(gr[i]);
      }
      *reinterpret_cast<u32x4*>(&Qs[r * RS + 8 * c]) = qr[i];
      *reinterpret_cast<u32x4*>(&Gs[r * RS + 8 * c]) = gr[i];
    }
    if (tid < WIN_DQ) {
      s_lse[tid] = lse_r * kLog2e;
      s_delta[tid] = delta_r;
      if constexpr (F16) s_expo[tid] = expo_r;
    }
    __syncthreads();
    load(min(x + 1, x1 - 1));
    // the wave's own keys may be seen by none of the rows
    if (jw > p_hi || (a.window > 0 && jw + 31 <= p_lo - a.window && jw >= a.sinks)) continue;
    floatx16 st, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = dp[r] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      st = mfma32x32x16<F16>(*reinterpret_cast<const u32x4*>(&Qs[lk * RS + 16 * s + 8 * half]), kf[s], st);
      dp = mfma32x32x16<F16>(*reinterpret_cast<const u32x4*>(&Gs[lk * RS + 16 * s + 8 * half]), vf[s], dp);
    }
    if constexpr (F16) {
      int e = s_expo[lk];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) e = max(e, __shfl_xor(e, o, 64));
      if (e > ex) {
        const float f = ldexpf(1.f, ex - e);
        ex = e;
        fac = pow2f(-ex);
#pragma unroll
        for (int b = 0; b < NB; ++b) dk[b] *= f;
      }
    }
    float big = 0.f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const floatx4 ls = *reinterpret_cast<const floatx4*>(&s_lse[8 * g + 4 * half]);
      const floatx4 de = *reinterpret_cast<const floatx4*>(&s_delta[8 * g + 4 * half]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e;
        float pr = exp2f(fmaf(st[r], sl2, -ls[e]));
        float x = pr * ((dp[r] - de[e]) * (F16 ? fac : 1.f));
        if (!whole) {
          const int pq = off + i0 + 8 * g + 4 * half + e;
          const bool ok = open && pq < sg.nk && j <= pq && (a.window <= 0 || j > pq - a.window || j < a.sinks);
          // a row with an inf or NaN in its operands has one in its log-sum or delta
          const float z = (ls[e] - ls[e]) + (de[e] - de[e]);
          pr = ok ? pr + z : 0.f;
          x = ok ? x + z : 0.f;
        }
        st[r] = pr;
        dp[r] = x;
        if constexpr (F16) big = fmaxf(big, fabsf(x));
      }
    }
    if constexpr (F16) {
      if (__any(big > 32768.f)) {
        big = big < __builtin_inff() ? big : 0.f;   // an inf is its key's own
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
        const int more = max(0, min((int)(__float_as_uint(big) >> 23) - 127 - 10, 100));
        const float f = pow2f(-more);
        ex += more;
        fac *= f;
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) dk[b] *= f;
      }
    }
    const int tr = (4 * half + (lane & 15) / 4) * RS + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int r = 8 * t;
      const u32x4 pb = {pack_act2<F16>(st[r], st[r + 1]), pack_act2<F16>(st[r + 2], st[r + 3]),
                        pack_act2<F16>(st[r + 4], st[r + 5]), pack_act2<F16>(st[r + 6], st[r + 7])};
      const u32x4 sb = {pack_act2<F16>(dp[r], dp[r + 1]), pack_act2<F16>(dp[r + 2], dp[r + 3]),
                        pack_act2<F16>(dp[r + 4], dp[r + 5]), pack_act2<F16>(dp[r + 6], dp[r + 7])};
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const uint2 x0 = lds_read_tr(&Gs[tr + 16 * t * RS + 32 * c]), y0 = lds_read_tr(&Gs[tr + (16 * t + 8) * RS + 32 * c]);
        dv[c] = mfma32x32x16<F16>(u32x4{x0.x, x0.y, y0.x, y0.y}, pb, dv[c]);
        const uint2 x1 = lds_read_tr(&Qs[tr + 16 * t * RS + 32 * c]), y1 = lds_read_tr(&Qs[tr + (16 * t + 8) * RS + 32 * c]);
        dk[c] = mfma32x32x16<F16>(u32x4{x1.x, x1.y, y1.x, y1.y}, sb, dk[c]);
      }
    }
  }
  if (it.part >= 0) {
    // float32 blocks [dk, dv][key][dim], the keys past the sample too (not read)
    float* pb = a.partial + it.part * (2 * WIN_DK * D) + (int64_t)(32 * wave + lk) * D;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        floatx4 y, z;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = F16 ? ldexpf(dk[b][4 * g + e] * a.scale, ex) : dk[b][4 * g + e] * a.scale;
          z[e] = dv[b][4 * g + e];
        }
        *reinterpret_cast<floatx4*>(pb + 32 * b + 8 * g + 4 * half) = y;
        *reinterpret_cast<floatx4*>(pb + WIN_DK * D + 32 * b + 8 * g + 4 * half) = z;
      }
    return;
  }
  if (!on) return;
  uint16_t* ko = static_cast<uint16_t*>(a.dk) + krow * a.lddk + (int64_t)kvh * D;
  uint16_t* vo = static_cast<uint16_t*>(a.dv) + krow * a.lddv + (int64_t)kvh * D;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = F16 ? ldexpf(dk[b][4 * g + e] * a.scale, ex) : dk[b][4 * g + e] * a.scale;
      const int c = 32 * b + 8 * g + 4 * half;
      *reinterpret_cast<uint2*>(ko + c) = make_uint2(pack_act2<F16>(y[0], y[1]), pack_act2<F16>(y[2], y[3]));
      *reinterpret_cast<uint2*>(vo + c) = make_uint2(pack_act2<F16>(dv[b][4 * g], dv[b][4 * g + 1]),
                                                     pack_act2<F16>(dv[b][4 * g + 2], dv[b][4 * g + 3]));
    }
}

// Adds the pieces of the cut key tiles, in piece order: one workgroup per work
// item that is a first piece, 32 bytes of a row per thread and pass.
template <int D, bool F16>
__global__ __launch_bounds__(NT) void window_dkv_join_kernel(WinBwdArgs a) {
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const WinBwdSeg& sg = a.seg[find_item_seg(a, item)];
  const DkvItem it = dkv_item(a, sg, item - sg.item0);
  if (it.part < 0 || it.piece != 0) return;
  const int rows = min(WIN_DK, sg.nk - it.kt * WIN_DK);
  const float* base = a.partial + it.part * (2 * WIN_DK * D);
  for (int t = threadIdx.x; t < 2 * rows * (D / 8); t += NT) {
    const int c = t % (D / 8) * 8, r = t / (D / 8) % rows, which = t / (D / 8) / rows;
    const float* src = base + ((int64_t)which * WIN_DK + r) * D + c;
    floatx4 y = {0.f, 0.f, 0.f, 0.f}, z = y;
    for (int s = 0; s < it.pieces; ++s) {
      y += *reinterpret_cast<const floatx4*>(src + (int64_t)s * 2 * WIN_DK * D);
      z += *reinterpret_cast<const floatx4*>(src + (int64_t)s * 2 * WIN_DK * D + 4);
    }
    const int64_t krow = (int64_t)sg.k0 + it.kt * WIN_DK + r;
    uint16_t* out = which ? static_cast<uint16_t*>(a.dv) + krow * a.lddv : static_cast<uint16_t*>(a.dk) + krow * a.lddk;
    *reinterpret_cast<uint4*>(out + (int64_t)it.kvh * D + c) =
        make_uint4(pack_act2<F16>(y[0], y[1]), pack_act2<F16>(y[2], y[3]), pack_act2<F16>(z[0], z[1]),
                   pack_act2<F16>(z[2], z[3]));
  }
}

}  // namespace

#define SVL_WIN_LAUNCH(kernel)                                               \
  if (a.nitems <= 0) return hipSuccess;                                      \
  if (head_dim == 128) {                                                     \
    if (f16) kernel<128, true><<<a.nitems, NT, 0, st>>>(a);                  \
    else kernel<128, false><<<a.nitems, NT, 0, st>>>(a);                     \
  } else if (head_dim == 64) {                                               \
    if (f16) kernel<64, true><<<a.nitems, NT, 0, st>>>(a);                   \
    else kernel<64, false><<<a.nitems, NT, 0, st>>>(a);                      \
  } else {                                                                   \
    return hipErrorInvalidValue;                                             \
  }                                                                          \
  return hipGetLastError();

hipError_t launch_window_dq(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st) {
  SVL_WIN_LAUNCH(window_dq_kernel)
}
hipError_t launch_window_dkv(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st) {
  SVL_WIN_LAUNCH(window_dkv_kernel)
}
hipError_t launch_window_dkv_join(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st) {
  SVL_WIN_LAUNCH(window_dkv_join_kernel)
}

}  // namespace svl
