// Causal attention with a sliding window and sink positions over packed ragged
// rows, on 16-bit MFMA: query i of a sample, at position p = nk - nq + i, sees
// key j iff j <= p and (no window, or j > p - window, or j < sinks) and the key
// is not masked.  Scores, softmax statistics and sums are float32.
//
// One workgroup = one (sample, query head, tile of 32 query rows per wave);
// tiles of 64 keys go through LDS, only those that some row of the tile sees.
// S^T = K Q^T by 32 x 32 x 16 MFMA (keys x queries), so that a lane's sums all
// belong to one query and its probabilities are, in place, the operand of
// O^T = V^T P^T.  V is kept row by row in LDS and read transposed
// (ds_read_b64_tr_b16).
#include "attn_ops.h"
#include "device_util.h"
#include "plan_types.h"
#include "window_attn.h"

namespace svl {
namespace {

// Four waves: 4 / KP groups of 32 query rows; with KP = 2 (launches too short to
// fill the chip) two waves share a group's rows, one 32-key half of each tile
// each, and are joined at the end.
template <int D, bool F16, int KP>
__global__ __launch_bounds__(256, 2) void window_attn_kernel(WinArgs a) {
  constexpr int NT = 256, QG = 4 / KP, BQ = 32 * QG, BK = WIN_BK, KB = 2 / KP;
  constexpr int KS = D + 8;      // K row stride (elements): 16-byte reads of 32 rows spread over the banks
  constexpr int VS = D + 32;     // V row stride: the 4 x 32-byte rows of a transposed read spread over them
  constexpr int NS = D / 16, NB = D / 32;
  constexpr int PR = D / 8, LD = BK * PR / NT;    // 16-byte pieces of a row, and of a tile per thread
  __shared__ __attribute__((aligned(16))) uint16_t Ks[BK * KS];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[BK * VS];
  __shared__ uint32_t s_bad[2][2];                // keys of a tile with an inf or NaN in V, two tiles in turn
  const int item = blockIdx.x;
  if (item >= a.nitems) return;
  const WinSeg& sg = a.seg[find_item_seg(a, item)];
  const int local = item - sg.item0;
  int slot = local % sg.h_cnt;
  // workgroups go to the 8 XCDs in turn: neighbouring heads (which share K and V
  // in a group) onto one
  if (sg.h_cnt % 8 == 0) slot = slot % 8 * (sg.h_cnt / 8) + slot / 8;
  const int nqt = (sg.nq + BQ - 1) / BQ;
  const int qt = nqt - 1 - local / sg.h_cnt;      // longest tiles first
  const int h = a.head_table ? a.head_table[sg.h_off + slot] : slot;
  const int kvh = h / (a.n_heads / a.n_kv_heads);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int qg = wave % QG, part = wave / QG;
  const int half = lane >> 5, lq = lane & 31;
  const int off = sg.nk - sg.nq;
  const int i0 = qt * BQ, qi = i0 + 32 * qg + lq;
  const bool on = qi < sg.nq;
  const int p = on ? off + qi : -1;                                       // the lane's position
  const int p_lo = off + i0, p_hi = off + min(i0 + BQ, sg.nq) - 1;        // the workgroup's
  const int w_lo = off + i0 + 32 * qg, w_hi = min(w_lo + 31, p_hi);       // the wave's

  u32x4 qf[NS];
  {
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + ((int64_t)sg.q0 + (on ? qi : 0)) * a.ldq +
                         (int64_t)h * D + 8 * half;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = load_piece(qp + 16 * s);
  }
  const uint16_t* kbase = static_cast<const uint16_t*>(a.k) + (int64_t)sg.k0 * a.ldk + (int64_t)kvh * D;
  const uint16_t* vbase = static_cast<const uint16_t*>(a.v) + (int64_t)sg.k0 * a.ldv + (int64_t)kvh * D;
  const uint8_t* mask = a.key_mask ? a.key_mask + sg.k0 : nullptr;

  // key tiles: [0, us) for the sinks, then from uw on
  const int start = a.window > 0 ? max(0, p_lo - a.window + 1) : 0;
  const int uw = start / BK, us = min((min(a.sinks, start) + BK - 1) / BK, uw);
  const int ntiles = us + p_hi / BK + 1 - uw;
  auto tile_of = [&](int u) { return (u < us ? u : uw + u - us) * BK; };

  u32x4 kr[LD], vr[LD];
  auto load = [&](int kv0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int task = tid + i * NT, row = min(kv0 + task / PR, sg.nk - 1), c = task % PR;
      kr[i] = load_piece(kbase + (int64_t)row * a.ldk + 8 * c);
      vr[i] = load_piece(vbase + (int64_t)row * a.ldv + 8 * c);
    }
  };

  float m = -__builtin_inff(), l = 0.f;
  bool poison = false;           // the row sees an inf or NaN of V in a partly masked tile
  floatx16 o[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
  const float sl2 = a.scale * 1.4426950408889634f;   // scores in log2 units

  if (tid < 4) s_bad[tid >> 1][tid & 1] = 0;
  load(tile_of(0));
  for (int u = 0; u < ntiles; ++u) {
    const int kv0 = tile_of(u);
    // whether every row of the workgroup sees every key of the tile (by position)
    const bool whole = kv0 + BK - 1 <= p_lo && (a.window <= 0 || kv0 > p_hi - a.window || kv0 + BK <= a.sinks);
    uint64_t seen = ~uint64_t(0);                     // the key mask's bits of this tile
    if (mask) seen = __ballot(mask[min(kv0 + lane, sg.nk - 1)] != 0);
    const bool partial = !whole || seen != ~uint64_t(0);
    __syncthreads();   // the readers of the tile before are done
    if (tid < 2) s_bad[(u + 1) & 1][tid] = 0;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int task = tid + i * NT, row = task / PR, c = task % PR;
      *reinterpret_cast<u32x4*>(&Ks[row * KS + 8 * c]) = kr[i];
      if (partial && any_nonfinite<F16>(vr[i])) {
        // an inf or NaN must not reach rows that do not see it (0 times inf)
        vr[i] = finite_part<F16>(vr[i]);
        atomicOr(&s_bad[u & 1][row >> 5], 1u << (row & 31));
      }
      *reinterpret_cast<u32x4*>(&Vs[row * VS + 8 * c]) = vr[i];
    }
    __syncthreads();
    load(tile_of(min(u + 1, ntiles - 1)));   // in flight meanwhile (the last one is not used)
    // the wave's own rows may see nothing of it
    if (kv0 > w_hi || (a.window > 0 && kv0 + BK - 1 <= w_lo - a.window && kv0 >= a.sinks)) continue;

    floatx16 st[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const int kb = KP == 2 ? part : b;
#pragma unroll
      for (int r = 0; r < 16; ++r) st[b][r] = 0.f;
#pragma unroll
      for (int s = 0; s < NS; ++s)
        st[b] = mfma32x32x16<F16>(*reinterpret_cast<const u32x4*>(&Ks[(32 * kb + lq) * KS + 16 * s + 8 * half]),
                                  qf[s], st[b]);
    }
    if (partial) {
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const int kb = KP == 2 ? part : b;
        const uint32_t see = (uint32_t)(seen >> (32 * kb)), bad = s_bad[u & 1][kb];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int jl = 8 * (r / 4) + 4 * half + r % 4, j = kv0 + 32 * kb + jl;
          const bool ok = j <= p && (a.window <= 0 || j > p - a.window || j < a.sinks) && ((see >> jl) & 1);
          st[b][r] = ok ? st[b][r] : -__builtin_inff();
          poison |= ok && ((bad >> jl) & 1);
        }
      }
    }
    float mx = -__builtin_inff();
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[b][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * sl2;
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx);
      const float alpha = mn == -__builtin_inff() ? 1.f : exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int b = 0; b < NB; ++b) o[b] *= alpha;
      m = mn;
    }
    const float mu = m == -__builtin_inff() ? 0.f : m;   // nothing above -inf yet
    // V^T fragment of dims 32 b .. and keys 16 t ..: rows 16 t + 4 half and 8 further
    const uint16_t* vt = &Vs[(4 * half + (lane & 15) / 4) * VS + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        st[b][r] = exp2f(fmaf(st[b][r], sl2, -mu));
        l += st[b][r];
      }
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const int t = 2 * (KP == 2 ? part : b) + t2, r = 8 * t2;
        const u32x4 pb = {pack_act2<F16>(st[b][r], st[b][r + 1]), pack_act2<F16>(st[b][r + 2], st[b][r + 3]),
                          pack_act2<F16>(st[b][r + 4], st[b][r + 5]), pack_act2<F16>(st[b][r + 6], st[b][r + 7])};
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          const uint2 x = lds_read_tr(vt + 16 * t * VS + 32 * c), y = lds_read_tr(vt + (16 * t + 8) * VS + 32 * c);
          o[c] = mfma32x32x16<F16>(u32x4{x.x, x.y, y.x, y.y}, pb, o[c]);
        }
      }
    }
  }

  l += __shfl_xor(l, 32, 64);
  poison = poison || __shfl_xor((int)poison, 32, 64);
  if constexpr (KP == 2) {
    // part 1 hands its sums to part 0 (in the V buffer, 16 rows of a lane's sums at a time)
    static_assert(QG * 64 * 20 * 4 <= (int)sizeof(Vs), "join buffer");
    float* s_j = reinterpret_cast<float*>(&Vs[0]) + (qg * 64 + lane) * 20;
    float f0 = 1.f, f1 = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      __syncthreads();
      if (part == 1) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s_j[r] = o[b][r];
        s_j[16] = m;
        s_j[17] = l;
        s_j[18] = poison ? 1.f : 0.f;
      }
      __syncthreads();
      if (part == 0) {
        if (b == 0) {
          const float m1 = s_j[16], mn = fmaxf(m, m1);
          f0 = m == -__builtin_inff() ? 0.f : exp2f(m - mn);
          f1 = m1 == -__builtin_inff() ? 0.f : exp2f(m1 - mn);
          l = l * f0 + s_j[17] * f1;
          m = mn;
          poison |= s_j[18] != 0.f;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = o[b][r] * f0 + s_j[r] * f1;
      }
    }
    if (part == 1) return;
  }
  if (!on) return;
  // a row that sees no key: output 0, log-sum -inf
  const float inv = poison ? __builtin_nanf("") : l == 0.f ? 0.f : 1.0f / l;
  const int64_t row = (int64_t)sg.q0 + qi;
  uint16_t* out = static_cast<uint16_t*>(a.out);
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint2 w = make_uint2(pack_act2<F16>(o[b][4 * g] * inv, o[b][4 * g + 1] * inv),
                                 pack_act2<F16>(o[b][4 * g + 2] * inv, o[b][4 * g + 3] * inv));
      const int64_t col = (int64_t)h * D + 32 * b + 8 * g + 4 * half;
      *reinterpret_cast<uint2*>(out + (a.packed ? packed_index(row, col, a.ldo) : row * a.ldo + col)) = w;
    }
  if (a.lse && half == 0)
    a.lse[row * a.n_heads + h] = l == 0.f ? -__builtin_inff() : m * 0.6931471805599453f + logf(l);
}

template <int D, bool F16>
hipError_t launch_win(const WinArgs& a, int bq, hipStream_t st) {
  if (bq == 128) window_attn_kernel<D, F16, 1><<<a.nitems, 256, 0, st>>>(a);
  else if (bq == 64) window_attn_kernel<D, F16, 2><<<a.nitems, 256, 0, st>>>(a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace

hipError_t launch_window_attention(const WinArgs& a, int32_t head_dim, bool f16, int32_t bq,
                                   hipStream_t st) {
  if (a.nitems <= 0) return hipSuccess;
  if (head_dim == 128) return f16 ? launch_win<128, true>(a, bq, st) : launch_win<128, false>(a, bq, st);
  if (head_dim == 64) return f16 ? launch_win<64, true>(a, bq, st) : launch_win<64, false>(a, bq, st);
  return hipErrorInvalidValue;
}

}  // namespace svl
