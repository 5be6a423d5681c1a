// Gradients of the windowed attention (window_attn.hip) on 16-bit MFMA, from the
// rows' log-sums: P = exp(scale q.k - lse), D = rowsum(dO * O), dP = dO V^T,
// dS = P (dP - D), then dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.  Sums,
// P, dP and dS are float32 and rounded to 16 bits once, as operands.  D comes from
// an output that is rounded too; as sum(P) is 1, a row's sum(dS) is what that took
// off D, so the query gradient's kernel puts it right for the key gradient, and for
// itself, where its sums are begun by then, takes dS as two 16-bit terms instead.
// (Either error by itself is as large as the rounding of the result.)
//
// Two launches, so that every sum has one owner and a fixed order (no atomics):
// the query gradient by tiles of query rows, the key and value gradients by
// tiles of keys; S and dP are formed in both.
//
// fp16: dS is scaled by a power of two that brings the largest gradient of the row
// (dQ) or of the rows so far (dK) into [2^10, 2^11), and further down where dS
// passes 2^15: rows that give almost all of their weight to one key have dS far
// below their gradient.  The factor is taken out in float32.
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

// Query gradient: four waves of 32 query rows against tiles of 32 keys.
// S^T = K Q^T and dP^T = V dO^T (keys x queries), dQ^T += K^T dS^T with K read
// transposed from LDS.
template <int D, bool F16>
__global__ __launch_bounds__(NT, 2) void window_dq_kernel(WinBwdArgs a) {
  constexpr int BQ = 128, BK = 32;     // (64 keys' staging registers do not fit)
  constexpr int NS = D / 16, NB = D / 32;
  constexpr int PR = D / 8, LD = BK * PR / NT;
  __shared__ __attribute__((aligned(16))) uint16_t s_kv[2][2 * BK * D];   // as in the forward
  __shared__ uint32_t s_bad[3];        // keys of a tile with an inf or NaN in K
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const WinBwdSeg& sg = a.seg[find_item_seg(a, item)];
  const int local = item - sg.item0;
  int h = local % a.n_heads;
  if (a.n_heads % 8 == 0) h = h % 8 * (a.n_heads / 8) + h / 8;   // as in the forward
  const int nqt = (sg.nq + BQ - 1) / BQ;
  const int qt = nqt - 1 - local / a.n_heads;
  const int kvh = h / (a.n_heads / a.n_kv_heads);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  // (a lane past the sample has the operands of row 0: no weights, or those of keys that
  // row 0 does not see would set the wave's scale)
  const float lse2 = on ? a.lse[row * a.n_heads + h] * kLog2e : __builtin_inff();
  // fp16: dS 2^-ex, which brings the row's largest gradient into [2^10, 2^11) (a row of
  // zeros, or with an inf or NaN, asks for nothing: fp16's smallest exponent)
  int ex = 0;
  if constexpr (F16)
    ex = (top > 0 && top < kNonfinite<true> ? (int)(__float_as_uint(act_bits_to_f32<true>(top)) >> 23) - 127 : -24) - 10;
  if constexpr (F16)
    if (on && half == 0) a.expo[row * a.n_heads + h] = ex;
  float off_d = 0.f;             // sum(dS), times fac
  int down = 0;                  // fp16: and 2^-down more, for the whole wave
  float fac = F16 ? pow2f(-ex) : 1.f;

  const uint8_t* mask = a.key_mask ? a.key_mask + sg.k0 : nullptr;
  const KeyTiles<BK> tiles(p_lo, p_hi, a.window, a.sinks);
  static_assert(NT / PR % 16 == 0, "a thread's pieces of a tile");
  const int piece = lds_piece<D>(tid / PR, tid % PR);
  u32x4 kr[LD], vr[LD];
  uint8_t mr = 0;
  RowSource<D, NT / PR> ksrc(a.k, sg.k0, a.ldk, sg.nk, tid), vsrc(a.v, sg.k0, a.ldv, sg.nk, tid);
  auto load = [&](int kv0) __attribute__((always_inline)) {
    uint32_t ko, vo;
    ksrc.tile(kv0, ko, kvh * D * 2);
    vsrc.tile(kv0, vo, kvh * D * 2);
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      kr[i] = ksrc.load(ko, i);
      vr[i] = vsrc.load(vo, i);
    }
    if (mask) mr = mask[min(kv0 + lane, sg.nk - 1)];
  };
  struct Seen {
    bool whole;
    uint32_t keys;
  };
  auto seen_of = [&](int kv0) __attribute__((always_inline)) {
    Seen s{tiles.whole(kv0), ~0u};
    if (mask) s.keys = (uint32_t)__ballot(mr != 0);      // (of the tile loaded last)
    return s;
  };
  auto store = [&](int buf, int bad, const Seen& s) __attribute__((always_inline)) {
    uint16_t* dst = s_kv[buf];
    const bool partial = !s.whole || s.keys != ~0u;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int r = tid / PR + i * (NT / PR), at = piece + i * (NT / PR) * D;
      if (partial && any_nonfinite<F16>(kr[i])) {
        kr[i] = finite_part<F16>(kr[i]);
        atomicOr(&s_bad[bad], 1u << r);
      }
      *reinterpret_cast<u32x4*>(&dst[at]) = kr[i];
      *reinterpret_cast<u32x4*>(&dst[BK * D + at]) = vr[i];
    }
  };
  floatx16 dq[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[b][r] = 0.f;
  const float sl2 = a.scale * kLog2e;
  bool poison = false;

  const int fr = lds_frag<D>(lane), tr = lds_tr<D>(lane);
  const int wlim = a.window > 0 ? a.window : 1 << 30;
  if (tid < 3) s_bad[tid] = 0;
  __syncthreads();
  // a tile that the wave's own rows see nothing of
  const int skip_lo = a.window > 0 ? w_lo - a.window - BK + 1 : -1;
  int kv0 = tiles.first, next = tiles.n > 1 ? tiles.after(kv0) : kv0;
  load(kv0);
  Seen now = seen_of(kv0);
  store(0, 0, now);
  load(next);
  int bad0 = 0, bad1 = 1, bad2 = 2;     // s_bad of this tile, the next, the one after
  for (int u = 0; u < tiles.n; ++u) {
    __syncthreads();   // tile u is stored, and the readers of the tile before are done
    if (tid == 0) s_bad[bad2] = 0;
    const Seen here = now;
    const int kv = kv0, bad_at = bad0;
    bad0 = bad1, bad1 = bad2, bad2 = bad_at;
    if (u + 1 < tiles.n) {
      now = seen_of(next);
      store((u + 1) & 1, bad0, now);
      kv0 = next;
      if (u + 2 < tiles.n) next = tiles.after(next);
    }
    load(next);        // in flight meanwhile (past the last tile: not used)
    if (kv > w_hi || (kv <= skip_lo && kv >= a.sinks)) continue;
    const uint16_t* Ks = s_kv[u & 1];
    const uint16_t* Vs = Ks + BK * D;
    const bool partial = !here.whole || here.keys != ~0u;
    floatx16 st, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = dp[r] = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      st = mfma32x32x16<F16>(lds_read16(&Ks[fr ^ 16 * s]), qf[s], st);
      dp = mfma32x32x16<F16>(lds_read16(&Vs[fr ^ 16 * s]), gf[s], dp);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = exp2_raw(fmaf(st[r], sl2, -lse2)) * ((dp[r] - delta) * fac);
    if (partial) {
      const int j0 = kv + 4 * half;   // element r is key j0 + 8 (r / 4) + r % 4
      const uint32_t see = here.keys >> (4 * half), bad = __builtin_amdgcn_readfirstlane(s_bad[bad_at]);
      const int top = p - j0, low = top - wlim, sink = a.sinks - j0;
      // (no short cuts: they would be branches)
      auto ok = [&](int x) { return bool((x <= top) & ((x > low) | (x < sink)) & ((see >> x) & 1)); };
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = ok(8 * (r / 4) + r % 4) ? st[r] : 0.f;
      if (bad)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int x = 8 * (r / 4) + r % 4;
          poison |= ok(x) & ((bad >> (4 * half + x)) & 1);
        }
    }
    if constexpr (F16) {
      float big = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(st[r]));
      if (__any(big > 32768.f)) {
        big = big < __builtin_inff() ? big : 0.f;   // an inf is its row's own
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
        const int more = max(0, min((int)(__float_as_uint(big) >> 23) - 127 - 10, 120));
        const float f = pow2f(-more);
        down += more;
        fac *= f;
        off_d *= f;
#pragma unroll
        for (int r = 0; r < 16; ++r) st[r] *= f;
#pragma unroll
        for (int b = 0; b < NB; ++b) dq[b] *= f;
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) off_d += st[r];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4 hi = round8<F16>(st, 8 * t), lo = rest8<F16>(st, 8 * t, hi);
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        const u32x4 kt = lds_frag_tr<D>(Ks, tr, t, c);
        dq[c] = mfma32x32x16<F16>(kt, hi, dq[c]);
        dq[c] = mfma32x32x16<F16>(kt, lo, dq[c]);
      }
    }
  }
  poison = poison || __shfl_xor((int)poison, 32, 64);
  off_d += __shfl_xor(off_d, 32, 64);
  if (!on) return;
  // (a poisoned row's dS has 0 in place of an inf of K)
  if (half == 0) a.delta[row * a.n_heads + h] = poison ? delta : delta + ldexpf(off_d, ex + down);
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
          make_uint2(round2<F16>(y[0], y[1]), round2<F16>(y[2], y[3]));
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

// Key and value gradients: four groups of 32 keys against tiles of 64 query rows,
// two waves per group and 32 rows a step.  One forms S = Q K^T (queries x keys) and
// P, hands P over in LDS and adds dV^T += dO^T P; the other forms dP = dO V^T and, a
// step later, when P is there, dS, and adds dK^T += Q^T dS.  The rows are in LDS,
// read as they are and transposed; K or V stays in registers.  At 4096 + 3001 rows
// of 32 / 8 heads under a window of 1024: one wave for both gradients needs over
// 256 registers, 832 us alone on its SIMD, 589 us with V in LDS; two waves that
// both form S 467 us; this way 454 us.
constexpr int DKV_NT = 512;

template <int D, bool F16>
__global__ __launch_bounds__(DKV_NT, 2) void window_dkv_kernel(WinBwdArgs a) {
  constexpr int NS = D / 16, NB = D / 32;
  constexpr int PR = D / 8, LD = WIN_DQ * PR / DKV_NT, STEP = DKV_NT / PR;
  __shared__ __attribute__((aligned(16))) uint16_t s_qg[2][2 * WIN_DQ * D];   // two tiles in turn: Q, then dO
  __shared__ __attribute__((aligned(16))) float s_lse[2][WIN_DQ], s_delta[2][WIN_DQ];
  __shared__ int s_expo[2][WIN_DQ];
  __shared__ floatx4 s_p[2][4][4][64];                                        // two steps in turn: P of the groups
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
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave & 3;
  const bool for_k = wave >= 4;          // the wave's gradient: dK or dV
  const int half = lane >> 5, lk = lane & 31;
  const int off = sg.nk - sg.nq;
  const int j0 = it.kt * WIN_DK, jw = j0 + 32 * kg, j = jw + lk;
  const bool on = j < sg.nk;
  const int64_t krow = (int64_t)sg.k0 + (on ? j : sg.nk - 1);
  const bool seen = on && (!a.key_mask || a.key_mask[krow]), is_sink = j < a.sinks;

  u32x4 own[NS];                         // K of the group's keys, or V
  {
    const uint16_t* op = (for_k ? static_cast<const uint16_t*>(a.v) + krow * a.ldv
                                : static_cast<const uint16_t*>(a.k) + krow * a.ldk) + (int64_t)kvh * D + 8 * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) own[s] = load_piece(op + 16 * s);
    // wait here: left to the loop, the wait for these would also be one for the
    // loads that the loop keeps in flight
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
  }
  floatx16 sum[NB];                      // dK^T or dV^T
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[b][r] = 0.f;
  const float sl2 = a.scale * kLog2e;
  int ex = -126;                         // fp16: dS 2^-ex, the same in every lane of the wave
  // fp16: P is held 2^12 times larger, so that small weights keep their digits as an operand
  // (weights are 1 at most, but for the log-sum's rounding: the next 2^3 are for scores of
  // millions); dP - D takes it back: fac = 2^(-ex - UP)
  constexpr int UP = F16 ? 12 : 0;
  const float back = pow2f(-UP);
  float fac = 1.f;

  static_assert(STEP % 16 == 0, "a thread's pieces of a tile");
  const int piece = lds_piece<D>(tid / PR, tid % PR);
  u32x4 qr[LD], gr[LD];
  float lse_r = 0.f, delta_r = 0.f;
  int expo_r = 0;
  RowSource<D, STEP> qsrc(a.q, sg.q0, a.ldq, sg.nq, tid), gsrc(a.grad, sg.q0, a.ldg, sg.nq, tid);
  // An entry of the list: its head and its first row.
  struct Entry {
    int h, i0;
  };
  auto entry = [&](int x) { return Entry{kvh * rep + x / ntq, (qt0 + x % ntq) * WIN_DQ}; };
  auto after = [&](const Entry& e) {
    return e.i0 + WIN_DQ < qt1 * WIN_DQ ? Entry{e.h, e.i0 + WIN_DQ} : Entry{e.h + 1, qt0 * WIN_DQ};
  };
  auto load = [&](const Entry& en) __attribute__((always_inline)) {
    const int h = en.h, i0 = en.i0;
    uint32_t qo, go;
    qsrc.tile(i0, qo, h * D * 2);
    gsrc.tile(i0, go, h * D * 2);
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      qr[i] = qsrc.load(qo, i);
      gr[i] = gsrc.load(go, i);
    }
    if (tid < WIN_DQ) {
      const int64_t at = ((int64_t)sg.q0 + min(i0 + tid, sg.nq - 1)) * a.n_heads + h;
      lse_r = a.lse[at];
      delta_r = a.delta[at];
      if constexpr (F16) expo_r = a.expo[at];
    }
  };
  const int whole_from = j0 + WIN_DK <= sg.nk && !a.key_mask ? j0 + WIN_DK - 1 - off : INT_MAX;
  const int whole_to = a.window > 0 ? (int)min((int64_t)j0 + a.window - WIN_DQ - off, (int64_t)INT_MAX) : INT_MAX;
  auto whole_of = [&](int i0) __attribute__((always_inline)) {
    return i0 >= whole_from && (i0 <= whole_to || j0 + WIN_DK <= a.sinks) && i0 + WIN_DQ <= sg.nq;
  };
  auto store = [&](int buf, int i0) __attribute__((always_inline)) {
    uint16_t* dst = s_qg[buf];
    const bool whole = whole_of(i0);
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int at = piece + i * STEP * D;
      if (!whole) {
        qr[i] = finite_part<F16>(qr[i]);
        gr[i] = finite_part<F16>(gr[i]);
      }
      *reinterpret_cast<u32x4*>(&dst[at]) = qr[i];
      *reinterpret_cast<u32x4*>(&dst[WIN_DQ * D + at]) = gr[i];
    }
    if (tid < WIN_DQ) {
      s_lse[buf][tid] = lse_r * kLog2e - UP;
      s_delta[buf][tid] = delta_r;
      if constexpr (F16) s_expo[buf][tid] = expo_r;
    }
  };
  const int fr = lds_frag<D>(lane), tr = lds_tr<D>(lane);
  const int wlim = a.window > 0 ? a.window : 1 << 30;
  Entry now{kvh * rep, 0}, next = now;
  if (x0 < x1) {
    now = next = entry(x0);
    load(now);
    store(0, now.i0);
    if (x0 + 1 < x1) next = after(now);
    load(next);
  }
  const int steps = 2 * (x1 - x0);
  floatx16 dp;                           // for dK: dP - D of the step before
  const uint16_t* before = nullptr;      // and its rows, nullptr where the group's keys see none of them
  // one step more for the last dK
  for (int t = 0; t <= steps; ++t) {
    __syncthreads();   // tile and P of the step before are stored, their readers before that are done
    if (for_k && before) {
      const floatx4* pp = &s_p[(t - 1) & 1][kg][0][lane];
      floatx16 ds;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4 pr = pp[64 * g];
#pragma unroll
        for (int e = 0; e < 4; ++e) ds[4 * g + e] = pr[e] * dp[4 * g + e];
      }
      if constexpr (F16) {
        float big = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(ds[r]));
        if (__any(big > 32768.f)) {
          big = big < __builtin_inff() ? big : 0.f;   // an inf is its key's own
#pragma unroll
          for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o, 64));
          const int more = max(0, min((int)(__float_as_uint(big) >> 23) - 127 - 10, 100));
          const float f = pow2f(-more);
          ex += more;
          fac *= f;
#pragma unroll
          for (int r = 0; r < 16; ++r) ds[r] *= f;
#pragma unroll
          for (int b = 0; b < NB; ++b) sum[b] *= f;
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x4 pb = round8<F16>(ds, 8 * u);
#pragma unroll
        for (int c = 0; c < NB; ++c) sum[c] = mfma32x32x16<F16>(lds_frag_tr<D>(before, tr, u, c), pb, sum[c]);
      }
    }
    before = nullptr;
    if (t == steps) break;
    const int buf = (t >> 1) & 1, sub = 32 * (t & 1), i0 = now.i0;
    // whether every row of the tile sees every key of the workgroup
    const bool whole = whole_of(i0);
    if (sub) {         // the other tile's last step is done
      now = next;
      const int x = x0 + (t >> 1);
      if (x + 1 < x1) store(buf ^ 1, now.i0);
      if (x + 2 < x1) next = after(now);
      load(next);      // in flight meanwhile (past the last: not used)
    }
    const int p_lo = off + i0 + sub, p_hi = min(p_lo + 31, sg.nk - 1);
    // the group's keys may be seen by none of the rows (or there are none)
    if (p_lo >= sg.nk || jw > p_hi || (a.window > 0 && jw + 31 <= p_lo - a.window && jw >= a.sinks)) continue;
    const uint16_t* Qs = s_qg[buf] + sub * D;
    const uint16_t* Gs = Qs + WIN_DQ * D;
    const float* lses = &s_lse[buf][sub + 4 * half];
    const float* deltas = &s_delta[buf][sub + 4 * half];
    // rows of the elements: 8 (r / 4) + r % 4 from top on
    const int top = p_lo + 4 * half, end = sg.nk - top, low = j - top;
    floatx16 st;
#pragma unroll
    for (int r = 0; r < 16; ++r) st[r] = 0.f;
    const uint16_t* rows = for_k ? Gs : Qs;
#pragma unroll
    for (int s = 0; s < NS; ++s) st = mfma32x32x16<F16>(lds_read16(&rows[fr ^ 16 * s]), own[s], st);
    if (for_k) {
      if constexpr (F16) {
        int e = s_expo[buf][sub + lk];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) e = max(e, __shfl_xor(e, o, 64));
        if (e > ex) {
          const float f = ldexpf(1.f, ex - e);
          ex = e;
          fac = pow2f(-ex) * back;
#pragma unroll
          for (int b = 0; b < NB; ++b) sum[b] *= f;
        }
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4 de = *reinterpret_cast<const floatx4*>(&deltas[8 * g]);
#pragma unroll
        for (int e = 0; e < 4; ++e) st[4 * g + e] = (st[4 * g + e] - de[e]) * (F16 ? fac : 1.f);
      }
    } else {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4 ls = *reinterpret_cast<const floatx4*>(&lses[8 * g]);
#pragma unroll
        for (int e = 0; e < 4; ++e) st[4 * g + e] = exp2_raw(fmaf(st[4 * g + e], sl2, -ls[e]));
      }
    }
    if (!whole) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const floatx4 ls = *reinterpret_cast<const floatx4*>(&lses[8 * g]);
        const floatx4 de = *reinterpret_cast<const floatx4*>(&deltas[8 * g]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int y = 8 * g + e;
          const bool ok = seen & (y < end) & (y >= low) & ((y < low + wlim) | is_sink);
          // a row with an inf or NaN in its operands has one in its log-sum or delta
          st[4 * g + e] = ok ? st[4 * g + e] + ((ls[e] - ls[e]) + (de[e] - de[e])) : 0.f;
        }
      }
    }
    if (for_k) {
      dp = st;
      before = Qs;
    } else {
      floatx4* pp = &s_p[t & 1][kg][0][lane];
#pragma unroll
      for (int g = 0; g < 4; ++g) pp[64 * g] = floatx4{st[4 * g], st[4 * g + 1], st[4 * g + 2], st[4 * g + 3]};
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const u32x4 pb = round8<F16>(st, 8 * u);
#pragma unroll
        for (int c = 0; c < NB; ++c) sum[c] = mfma32x32x16<F16>(lds_frag_tr<D>(Gs, tr, u, c), pb, sum[c]);
      }
    }
  }
  const float f = for_k ? a.scale : 1.f;
  if (!F16 || !for_k) ex = -UP;
  if (it.part >= 0) {
    // float32 blocks [dk, dv][key][dim], the keys past the sample too (not read)
    float* pb = a.partial + it.part * (2 * WIN_DK * D) + (for_k ? 0 : WIN_DK * D) + (int64_t)(32 * kg + lk) * D;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        floatx4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = ldexpf(sum[b][4 * g + e] * f, ex);
        *reinterpret_cast<floatx4*>(pb + 32 * b + 8 * g + 4 * half) = y;
      }
    return;
  }
  if (!on) return;
  uint16_t* out = (for_k ? static_cast<uint16_t*>(a.dk) + krow * a.lddk : static_cast<uint16_t*>(a.dv) + krow * a.lddv) +
                  (int64_t)kvh * D;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = ldexpf(sum[b][4 * g + e] * f, ex);
      *reinterpret_cast<uint2*>(out + 32 * b + 8 * g + 4 * half) =
          make_uint2(round2<F16>(y[0], y[1]), round2<F16>(y[2], y[3]));
    }
}

// Adds the pieces of the cut key tiles, in piece order.  Bound by latency: the
// workgroups of a tile's pieces share its rows, 32 bytes of a row per thread and
// pass, four pieces in flight (16 sink tiles of some 15 pieces: 11 us, with one
// workgroup a tile 25).
template <int D, bool F16>
__global__ __launch_bounds__(NT) void window_dkv_join_kernel(WinBwdArgs a) {
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const WinBwdSeg& sg = a.seg[find_item_seg(a, item)];
  const DkvItem it = dkv_item(a, sg, item - sg.item0);
  if (it.part < 0) return;
  const int rows = min(WIN_DK, sg.nk - it.kt * WIN_DK);
  const float* base = a.partial + (it.part - it.piece) * (2 * WIN_DK * D);
  for (int t = it.piece * NT + threadIdx.x; t < 2 * rows * (D / 8); t += it.pieces * NT) {
    const int c = t % (D / 8) * 8, r = t / (D / 8) % rows, which = t / (D / 8) / rows;
    const float* src = base + ((int64_t)which * WIN_DK + r) * D + c;
    floatx4 y = {0.f, 0.f, 0.f, 0.f}, z = y;
#pragma unroll 4
    for (int s = 0; s < it.pieces; ++s) {
      y += *reinterpret_cast<const floatx4*>(src + (int64_t)s * 2 * WIN_DK * D);
      z += *reinterpret_cast<const floatx4*>(src + (int64_t)s * 2 * WIN_DK * D + 4);
    }
    const int64_t krow = (int64_t)sg.k0 + it.kt * WIN_DK + r;
    uint16_t* out = which ? static_cast<uint16_t*>(a.dv) + krow * a.lddv : static_cast<uint16_t*>(a.dk) + krow * a.lddk;
    *reinterpret_cast<uint4*>(out + (int64_t)it.kvh * D + c) =
        make_uint4(round2<F16>(y[0], y[1]), round2<F16>(y[2], y[3]), round2<F16>(z[0], z[1]),
                   round2<F16>(z[2], z[3]));
  }
}

}  // namespace

#define SVL_WIN_LAUNCH(kernel, threads)                                      \
  if (a.nitems <= 0) return hipSuccess;                                      \
  if (head_dim == 128) {                                                     \
    if (f16) kernel<128, true><<<a.nitems, threads, 0, st>>>(a);             \
    else kernel<128, false><<<a.nitems, threads, 0, st>>>(a);                \
  } else if (head_dim == 64) {                                               \
    if (f16) kernel<64, true><<<a.nitems, threads, 0, st>>>(a);              \
    else kernel<64, false><<<a.nitems, threads, 0, st>>>(a);                 \
  } else {                                                                   \
    return hipErrorInvalidValue;                                             \
  }                                                                          \
  return hipGetLastError();

hipError_t launch_window_dq(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st) {
  SVL_WIN_LAUNCH(window_dq_kernel, NT)
}
hipError_t launch_window_dkv(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st) {
  SVL_WIN_LAUNCH(window_dkv_kernel, DKV_NT)
}
hipError_t launch_window_dkv_join(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st) {
  SVL_WIN_LAUNCH(window_dkv_join_kernel, NT)
}

}  // namespace svl
