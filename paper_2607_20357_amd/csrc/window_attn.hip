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
  constexpr int NS = D / 16, NB = D / 32;
  constexpr int PR = D / 8, LD = BK * PR / NT;    // 16-byte pieces of a row, and of a tile per thread
  __shared__ __attribute__((aligned(16))) uint16_t s_kv[2][2 * BK * D];   // two tiles in turn: K, then V
  __shared__ uint32_t s_bad[3][2];                // keys of a tile with an inf or NaN in V, three tiles in turn
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
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
  const uint8_t* mask = a.key_mask ? a.key_mask + sg.k0 : nullptr;

  const KeyTiles<BK> tiles(p_lo, p_hi, a.window, a.sinks);
  // (rows 16 apart have the same swizzle)
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
  // What the workgroup's rows see of a tile: all of it by position, and the key
  // mask's bits.
  struct Seen {
    bool whole;
    uint64_t keys;
  };
  auto seen_of = [&](int kv0) __attribute__((always_inline)) {
    Seen s{tiles.whole(kv0), ~uint64_t(0)};
    if (mask) s.keys = __ballot(mr != 0);      // (of the tile loaded last)
    return s;
  };
  auto store = [&](int buf, int bad, const Seen& s) __attribute__((always_inline)) {
    uint16_t* dst = s_kv[buf];
    const bool partial = !s.whole || s.keys != ~uint64_t(0);
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int row = tid / PR + i * (NT / PR), at = piece + i * (NT / PR) * D;
      *reinterpret_cast<u32x4*>(&dst[at]) = kr[i];
      if (partial && any_nonfinite<F16>(vr[i])) {
        // an inf or NaN must not reach rows that do not see it (0 times inf)
        vr[i] = finite_part<F16>(vr[i]);
        atomicOr(&s_bad[bad][row >> 5], 1u << (row & 31));
      }
      *reinterpret_cast<u32x4*>(&dst[BK * D + at]) = vr[i];
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
  // fp16: weights are held 2^7 times larger (2^15 at most, see the maximum below), so that
  // those of a long tail behind a first key are seldom subnormal: half a step of those is
  // 2^-32 of the row's largest weight
  constexpr float UP = F16 ? 7.f : 0.f;

  const int fr = lds_frag<D>(lane), tr = lds_tr<D>(lane);
  const int wlim = a.window > 0 ? a.window : 1 << 30;   // (positions are below 2^30)
  if (tid < 6) s_bad[tid >> 1][tid & 1] = 0;
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
    if (tid < 2) s_bad[bad2][tid] = 0;
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

    // 32 keys at a time
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const int kb = KP == 2 ? part : b;
      floatx16 st;
#pragma unroll
      for (int r = 0; r < 16; ++r) st[r] = 0.f;
#pragma unroll
      for (int s = 0; s < NS; ++s)
        st = mfma32x32x16<F16>(lds_read16(&Ks[(fr ^ 16 * s) + 32 * kb * D]), qf[s], st);
      if (!here.whole || here.keys != ~uint64_t(0)) {
        const int j0 = kv + 32 * kb + 4 * half;   // element r is key j0 + 8 (r / 4) + r % 4
        const uint32_t see = (uint32_t)(here.keys >> (32 * kb)) >> (4 * half);
        const uint32_t bad = __builtin_amdgcn_readfirstlane(s_bad[bad_at][kb]);
        if (here.whole) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            st[r] = (see >> (8 * (r / 4) + r % 4)) & 1 ? st[r] : -__builtin_inff();
          poison |= (see & (bad >> (4 * half)) & 0x0f0f0f0fu) != 0;
        } else {
          const int top = p - j0, low = top - wlim, sink = a.sinks - j0;
          // (no short cuts: they would be branches)
          auto ok = [&](int x) { return bool((x <= top) & ((x > low) | (x < sink)) & ((see >> x) & 1)); };
#pragma unroll
          for (int r = 0; r < 16; ++r) st[r] = ok(8 * (r / 4) + r % 4) ? st[r] : -__builtin_inff();
          if (bad)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int x = 8 * (r / 4) + r % 4;
              poison |= ok(x) & ((bad >> (4 * half + x)) & 1);
            }
        }
      }
      float mx = -__builtin_inff();
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, st[r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * sl2;
      // the maximum is followed at a distance: weights up to 2^8 lose nothing, and
      // rows seldom need their sums scaled again
      if (__any(mx > m + 8.f)) {
        const float mn = fmaxf(m, mx);
        const float alpha = mn == -__builtin_inff() ? 1.f : exp2_raw(m - mn);
        l *= alpha;
#pragma unroll
        for (int c = 0; c < NB; ++c) o[c] *= alpha;
        m = mn;
      }
      const float mu = m == -__builtin_inff() ? 0.f : m - UP;   // nothing above -inf yet: 0
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        st[r] = exp2_raw(fmaf(st[r], sl2, -mu));
        l += st[r];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int r = 8 * t;
        const u32x4 pb = round8<F16>(st, r);
#pragma unroll
        for (int c = 0; c < NB; ++c)
          o[c] = mfma32x32x16<F16>(lds_frag_tr<D>(Vs, tr, 2 * kb + t, c), pb, o[c]);
      }
    }
  }

  l += __shfl_xor(l, 32, 64);
  poison = poison || __shfl_xor((int)poison, 32, 64);
  if constexpr (KP == 2) {
    // part 1 hands its sums to part 0, 16 of a lane's at a time
    static_assert(QG * 64 * 20 * 4 <= (int)sizeof(s_kv), "join buffer");
    float* s_j = reinterpret_cast<float*>(&s_kv[0][0]) + (qg * 64 + lane) * 20;
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
          f0 = m == -__builtin_inff() ? 0.f : exp2_raw(m - mn);
          f1 = m1 == -__builtin_inff() ? 0.f : exp2_raw(m1 - mn);
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
      const uint2 w = make_uint2(round2<F16>(o[b][4 * g] * inv, o[b][4 * g + 1] * inv),
                                 round2<F16>(o[b][4 * g + 2] * inv, o[b][4 * g + 3] * inv));
      const int64_t col = (int64_t)h * D + 32 * b + 8 * g + 4 * half;
      *reinterpret_cast<uint2*>(out + (a.packed ? packed_index(row, col, a.ldo) : row * a.ldo + col)) = w;
    }
  if (a.lse && half == 0)
    a.lse[row * a.n_heads + h] = l == 0.f ? -__builtin_inff() : (m - UP) * 0.6931471805599453f + logf(l);
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
