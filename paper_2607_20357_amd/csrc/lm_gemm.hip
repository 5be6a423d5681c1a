// The three matrix products of the language-model loss:
//   logits  s = x w^T, whose tiles leave as exponentials and their slabs' maxima and sums
//   grad_x  P w        grad_w  P^T x
//
// C[n][m] = sum_k A[m][k] B[n][k] in tiles of 256 x 256, 64 of the sum a step.  Each
// operand comes as its memory has it: rows along k (fragments by 16-byte LDS
// reads), or rows along m or n (transposed LDS reads), so neither w, x nor P is
// ever laid out a second time.  Both go from memory to LDS without passing
// registers, two and three steps ahead, a whole line of memory at a time; the places of
// a step's 16-byte pieces are exchanged on the way (the lane asks for another piece,
// since its place in LDS is fixed), so that both kinds of fragment read are free of
// bank conflicts.
#include "device_util.h"
#include "lm_loss.h"
#include "svl_internal.h"
#include "window_attn.h"

namespace svl {
namespace {

constexpr int NT = 256;              // 4 waves, 2 along m and 2 along n, of W x W: tiles of 2 W x 2 W

// 16 bytes a lane from memory to LDS, from `to` on in lane order.  (The builtin would do, but
// for the compiler every transposed LDS read after it may be of what it brings: it waits
// for memory before each.  Here the waits are the turns' own, wait_loads().)
__device__ __forceinline__ void load_to_lds(const u32x4& rsrc, uint32_t voff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(to), "v"(voff), "s"(rsrc) : "memory");   // (nothing else here uses m0)
}

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// One operand's steps of T rows (or columns).  TR: rows along the sum; ENDS: they end inside a step.
template <bool TR, bool ENDS, int T>
struct Operand {
  static constexpr int LOADS = T / 32;      // of a wave a step
  static constexpr int PER = T == 256 ? 2 : 4;   // TR: rows of a load
  const uint16_t* p;      // of the tile's first row (TR: first column), first k
  int64_t ld;
  int32_t k;              // length of the sum, where rows along it end (TR)
  uint32_t voff[LOADS];
  u32x4 rs;
  int left;

  __device__ __forceinline__ void init(const uint16_t* base, int64_t ld_, int32_t first, int32_t count, int32_t k_) {
    const int w = wave_id(), lane = threadIdx.x & 63;
    ld = ld_;
    k = k_;
    p = base + (TR ? (int64_t)first : (int64_t)first * ld);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      if constexpr (TR) {
        // PER rows of T columns; pairs of pieces change places by the row
        const int r = (i * 4 + w) * PER + lane / (64 / PER), at = lane % (64 / PER);
        int piece = (((at >> 1) ^ ((r & 3) | ((r >> 3 & (T / 64 - 1)) << 2))) << 1) | (at & 1);
        const int most = (count - first) / 8 - 1;     // (widths are multiples of 8)
        piece = piece < most ? piece : most;
        voff[i] = (uint32_t)r * ((uint32_t)ld * 2) + piece * 16;
      } else {
        // 8 rows of 64: pieces change places by the pair of rows
        int r = (i * 4 + w) * 8 + (lane >> 3);
        const int piece = (lane & 7) ^ ((r >> 1) & 7);
        r = r < count - first ? r : count - first - 1;
        voff[i] = (uint32_t)r * ((uint32_t)ld * 2) + piece * 16;
      }
    }
  }

  // From here on the wave's loads are of step t.
  __device__ __forceinline__ void at_step(int t) {
    left = k - t * LM_BK;
    const uint64_t a = reinterpret_cast<uint64_t>(TR ? p + (int64_t)t * LM_BK * ld : p + t * LM_BK);
    rs = u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)) & 0xffffu, 0x7fffffffu, 0x00020000u};
  }
  // The wave's load i.  Rows behind the last of the sum are taken to be the last: P is 0 there.
  __device__ __forceinline__ void fetch(int i, uint32_t lds) const {
    uint32_t v = voff[i];
    if (ENDS && left < LM_BK) {
      const int over = (i * 4 + wave_id()) * PER + (int)(threadIdx.x & 63) / (64 / PER) - (left - 1);
      v -= over > 0 ? (uint32_t)over * ((uint32_t)ld * 2) : 0u;
    }
    load_to_lds(rs, v, lds + i * 4096);
  }
};

// Fragments of 16 rows (or columns) of a step, from `first` on, 32 of the sum each.
template <bool TR, int T>
struct Fragments {
  uint32_t at;          // bytes
  __device__ __forceinline__ void init(int first) {
    const int lane = threadIdx.x & 63, g = lane >> 4, l = lane & 15;
    if constexpr (TR)
      at = (uint32_t)((8 * g + l / 4) * T * 2 + (((first / 16) ^ (l / 4 | (g & (T / 64 - 1)) << 2)) * 32) + (l & 3) * 8);
    else
      at = (uint32_t)((first + l) * LM_BK * 2 + ((g ^ (l >> 1)) * 16));
  }
  // The lane's place in the step at LDS address `lds`.  (Opaque: the compiler would otherwise keep every
  // block's place of every buffer in registers.)
  __device__ __forceinline__ uint32_t place(uint32_t lds) const {
    uint32_t p = lds + at;
    asm volatile("" : "+v"(p));
    return p;
  }
  static __device__ __forceinline__ u32x4 read(uint32_t place, int block, int half) {
    if constexpr (TR) {
      const uint32_t q = (place ^ (block * 32)) + half * 64 * T;
      const uint2 a = read_tr(q), b = read_tr(q + 8 * T);
      return u32x4{a.x, a.y, b.x, b.y};
    } else {
      return *(__attribute__((address_space(3))) const u32x4*)(uintptr_t)((place ^ (half * 64)) + block * 32 * LM_BK);
    }
  }
  static __device__ __forceinline__ uint2 read_tr(uint32_t at) {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) shortx4*)(uintptr_t)at));
  }
};

// c += a b.  (In assembly so that all sums stay where they are, in the accumulation registers: the
// compiler moves some of 64 blocks of 4 to and fro.  What the hardware does not wait for by itself is
// kept apart: the fragments come from LDS, whose arrival is waited for, and no instruction of the vector
// unit writes an operand shortly before; a sum is used again by the product NB^2 later, and read after
// settle().  tests/test_lm_products_cpu.py looks at what the compiler makes of it.)
template <bool F16>
__device__ __forceinline__ void mfma(const u32x4& a, const u32x4& b, floatx4& c) {
  if constexpr (F16) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// Ends a turn: nothing moves over it, and all waves have come here.
__device__ __forceinline__ void turn() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xc07f); }     // lgkmcnt(0)
// Until at most N of the wave's loads are on their way (vmcnt).
template <int N>
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14); }

struct Tile {
  int m, n, piece, pieces, tiles, id;
};

// Workgroup -> tile: consecutive workgroups of an XCD take blocks of 8 x 4 tiles.
__device__ __forceinline__ bool tile_of(int mt, int nt, int nk, bool cut, Tile* t) {
  t->tiles = mt * nt;
  t->pieces = cut ? lm_pieces(t->tiles, nk) : 1;
  const int total = t->tiles * t->pieces, per = (total + 7) / 8;
  const int i = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || i >= total) return false;
  t->piece = i / t->tiles;
  t->id = i;
  const int j = i % t->tiles, group = j / (8 * nt), in = j % (8 * nt);
  const int gm = mt - group * 8 < 8 ? mt - group * 8 : 8;
  t->m = group * 8 + in % gm;
  t->n = in / gm;
  return true;
}

// Sizes of a product: m, n, k, and k's steps.
struct Sizes {
  int m, n, k, nk;
};
__device__ __forceinline__ Sizes sizes_of(const LmArgs& a, LmProduct p) {
  int rows = a.head->rows - a.chunk0;
  rows = rows < 0 ? 0 : rows < a.chunk ? rows : a.chunk;
  Sizes s;
  s.m = p == LM_LOGITS ? a.vocab : a.d;
  s.n = p == LM_GRAD_W ? a.vocab : rows;
  s.k = p == LM_LOGITS ? a.d : p == LM_GRAD_X ? a.vocab : rows;
  s.nk = (s.k + LM_BK - 1) / LM_BK;
  return s;
}

// Four elements of a gradient along d, from float32 to where they go: grad_x or grad_w.
template <bool F16>
__device__ __forceinline__ uint2 round_grad(floatx4 v, uint2 old, bool add) {
  if (add) {
    v[0] += act_bits_to_f32<F16>(old.x & 0xffffu);
    v[1] += act_bits_to_f32<F16>(old.x >> 16);
    v[2] += act_bits_to_f32<F16>(old.y & 0xffffu);
    v[3] += act_bits_to_f32<F16>(old.y >> 16);
  }
  return make_uint2(pack_act2<F16>(v[0], v[1]), pack_act2<F16>(v[2], v[3]));
}
// What a gradient's sums are multiplied by: the rows' gradient in fp16 by the row (n of `rows`), otherwise one for all.
template <LmProduct P, bool F16>
__device__ __forceinline__ float grad_scale(const LmArgs& a, int n, int rows) {
  const float most = a.head->weight, all = most * (F16 ? 1.f / LM_E_SCALE : 1.f);
  if (!F16 || P != LM_GRAD_X) return all;
  return n < rows ? lm_power(lm_part(a.weight[a.chunk0 + n], most)) * all : 0.f;
}

// N quads along d of one row of grad_w, 16 apart: sums of passes, and what is there already.
template <bool F16, int N>
__device__ __forceinline__ void add_grad_w(const LmArgs& a, int n, int m, float scale, floatx4 (&v)[N]) {
  if (a.sum_w) {
    float4* sum = reinterpret_cast<float4*>(a.sum_w + (int64_t)n * a.d + m);
    if (!a.first) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float4 s = sum[4 * i];
        v[i][0] += s.x; v[i][1] += s.y; v[i][2] += s.z; v[i][3] += s.w;
      }
    }
    if (!a.last) {
#pragma unroll
      for (int i = 0; i < N; ++i) sum[4 * i] = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
      return;
    }
  }
  uint2* out = reinterpret_cast<uint2*>(a.grad_w + (int64_t)n * a.ldgw + m);
  uint2 old[N];
#pragma unroll
  for (int i = 0; i < N; ++i) old[i] = a.accumulate ? out[4 * i] : make_uint2(0, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) out[4 * i] = round_grad<F16>(v[i] * scale, old[i], a.accumulate);
}

// A wave's W rows of W 16-bit results pass through its part of LDS, so that they leave in
// whole lines: 8 bytes (a half of the 16-byte piece) in, 16 bytes of a few rows out; pieces change
// places by the row against bank conflicts.
template <int W>
__device__ __forceinline__ void put(uint16_t* own, int row, int piece, int half, uint2 v) {
  *reinterpret_cast<uint2*>(own + row * W + (piece ^ (row & (W / 8 - 1))) * 8 + half * 4) = v;
}
template <int W>
__device__ __forceinline__ u32x4 get(const uint16_t* own, int row, int piece) {
  return *reinterpret_cast<const u32x4*>(own + row * W + (piece ^ (row & (W / 8 - 1))) * 8);
}

// Logits of W entries of the vocabulary (a wave's, a slab) become exponentials under their
// row's largest; a lane holds a quarter of the row's, three others the rest.
template <bool F16, int W>
__device__ __forceinline__ void store_logits(const LmArgs& a, int m0, int n, bool there, uint16_t* own, int row,
                                             floatx4 (&acc)[W / 16]) {
  const int g = (threadIdx.x & 63) >> 4;
  float top = -INFINITY;
  if (m0 + W > a.vocab) {
    const int end = a.vocab - m0 - 4 * g;
#pragma unroll
    for (int b = 0; b < W / 16; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (b * 16 + i >= end) acc[b][i] = -INFINITY;
  }
#pragma unroll
  for (int b = 0; b < W / 16; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, acc[b][i]);
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = fmaxf(top, __shfl_xor(top, 32, 64));
  const int label = there ? a.label[a.chunk0 + n] - m0 : -1;
  const bool here = label >= 0 && label < W && (label >> 2 & 3) == g;
  float sum = 0.f;
  if (__any(here)) {
    float mine = 0.f;
#pragma unroll
    for (int b = 0; b < W / 16; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (b * 16 + i == label - 4 * g) mine = acc[b][i];
    if (here) a.label_logit[n] = mine;
  }
  // 2^(log2(e) (s - top) + 14): what is kept.  The difference comes first: the largest is 2^14 whatever
  // its size (a product of top that is rounded by itself is off by parts of |top| 2^-24 of all values, and past
  // 2^24 leaves fp16's range).  (top -inf: nothing of the vocabulary here, or no probability)
  constexpr float LOG2E = 1.44269504088896340736f;
  const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int b = 0; b < W / 16; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      acc[b][i] = exp2_raw(fmaf(acc[b][i] - from, LOG2E, 14.f));
      sum += acc[b][i];
    }
  sum += __shfl_xor(sum, 16, 64);
  sum += __shfl_xor(sum, 32, 64);
  if (there && g == 0)
    a.stats[(int64_t)n * (a.vp / W) + m0 / W] = make_float2(top, sum * (1.f / LM_E_SCALE));
  if (!a.e) return;
#pragma unroll
  for (int b = 0; b < W / 16; ++b)
    put<W>(own, row, 2 * b + (g >> 1), g & 1,
        make_uint2(pack_act2<true>(acc[b][0], acc[b][1]), pack_act2<true>(acc[b][2], acc[b][3])));
}

template <LmProduct P, bool F16, int W>
__global__ __launch_bounds__(NT, W == 128 ? 1 : 2) void lm_product_kernel(LmArgs a) {
  constexpr int T = 2 * W, NB = W / 16, STEP = T * LM_BK;   // tile, a wave's blocks a side, elements of an operand's step
  static_assert(P != LM_GRAD_X || W == 128, "");            // (sums are cut in tiles of LM_TILE)
  constexpr bool TA = P != LM_LOGITS, TB = P == LM_GRAD_W;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[5 * STEP];   // three steps of one operand, two of the other: 160 or 80 KB
  const Sizes s = sizes_of(a, P);
  if (P == LM_GRAD_W && s.nk == 0 && !a.first && !a.last) return;   // nothing to add to the sums
  Tile t;
  if (!tile_of((s.m + T - 1) / T, (s.n + T - 1) / T, s.nk, P != LM_LOGITS && T == LM_TILE, &t)) return;
  const int m0 = t.m * T, n0 = t.n * T;
  const int kt0 = (int)((int64_t)s.nk * t.piece / t.pieces), kt1 = (int)((int64_t)s.nk * (t.piece + 1) / t.pieces);

  const uint16_t* xc = a.xc + (int64_t)a.chunk0 * a.d;
  Operand<TA, P == LM_GRAD_X, T> A;
  Operand<TB, false, T> B;
  constexpr int LOADS = Operand<TA, false, T>::LOADS;
  if constexpr (P == LM_LOGITS) {
    A.init(a.w, a.ldw, m0, a.vocab, a.d);
    B.init(xc, a.d, n0, s.n, a.d);
  } else if constexpr (P == LM_GRAD_X) {
    A.init(a.w, a.ldw, m0, a.d, a.vocab);
    B.init(a.e, a.vp, n0, s.n, a.vp);
  } else {
    A.init(xc, a.d, m0, a.d, s.nk * LM_BK);
    B.init(a.e, a.vp, n0, a.vp, s.nk * LM_BK);
  }
  const int w = wave_id(), wm = w & 1, wn = w >> 1;
  Fragments<TA, T> fa;
  Fragments<TB, T> fb;
  fa.init(wm * W);
  fb.init(wn * W);

  floatx4 acc[NB][NB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};

  // While half a step's fragments, in registers, are multiplied, the next half's are read and loads of
  // a later step go out: in the first half the deep operand's of two steps on, in the second the other's
  // of two steps on, into the buffer whose last fragments the first half has read.  One barrier a step.
  // The deep operand has three buffers: what streams from memory (w, P) in place of what the tiles of an
  // XCD share (x).  The sum's last steps ask for its last once more, so that all are alike.
  constexpr bool DEEP_A = P != LM_GRAD_W;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)lds;
  const uint32_t other = 3 * 2 * STEP;     // the other operand's buffers are behind the deep one's
  const uint32_t mine = __builtin_amdgcn_readfirstlane((int)(base + w * 1024));
  struct Frags {
    u32x4 a[NB], b[NB];
  };
  const auto at_step = [&](bool deep, int t) {
    t = t < kt1 ? t : kt1 - 1;
    if (deep == DEEP_A) A.at_step(t); else B.at_step(t);
  };
  const auto fetch = [&](bool deep, int i, uint32_t buf) {
    if (deep == DEEP_A) A.fetch(i, mine + buf); else B.fetch(i, mine + buf);
  };
  // Fragment i of a half, in the order in which the products take them.
  const auto read = [&](Frags& f, int i, uint32_t pa, uint32_t pb, int half) {
    if (i % 2 == 0) f.b[i / 2] = fb.read(pb, i / 2, half);
    else f.a[i / 2] = fa.read(pa, i / 2, half);
  };
  // Products of `f`, with the reads of half `half` of the step at pa, pb and the loads into `to` between them.
  const auto multiply = [&](const Frags& f, Frags& next, uint32_t pa, uint32_t pb, int half, bool deep, uint32_t to) {
#pragma unroll
    for (int i = 0; i < NB * NB; ++i) {
      mfma<F16>(f.a[i / NB], f.b[i % NB], acc[i % NB][i / NB]);
      if (i % (NB / 2) == 0) read(next, i / (NB / 2), pa, pb, half);
      if (i % NB == NB / 2 - 1) fetch(deep, i / NB, to);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_lds();
  };
  const auto places = [&](uint32_t deep, uint32_t shallow, uint32_t& pa, uint32_t& pb) {
    pa = fa.place(base + (DEEP_A ? deep : other + shallow));
    pb = fb.place(base + (DEEP_A ? other + shallow : deep));
  };
  Frags f0, f1;
  if (kt0 < kt1) {
    uint32_t pa, pb;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      at_step(true, kt0 + i);
      at_step(false, kt0 + i);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) fetch(true, j, i * 2 * STEP);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) fetch(false, j, other + i * 2 * STEP);
    }
    wait_loads<2 * LOADS>();
    turn();
    places(0, 0, pa, pb);
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) read(f0, i, pa, pb, 0);
    wait_lds();
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) asm volatile("" : "+a"(acc[i][j]));   // the zeros are written before
    settle();
    uint32_t deep = 0, shallow = 0;      // buffers of step t
#pragma unroll 1
    for (int t = kt0; t < kt1; ++t) {
      const uint32_t deep1 = deep == 4 * STEP ? 0 : deep + 2 * STEP, deep2 = deep1 == 4 * STEP ? 0 : deep1 + 2 * STEP;
      at_step(true, t + 2);
      multiply(f0, f1, pa, pb, 1, true, deep2);
      wait_loads<LOADS>();               // step t + 1 of both; what is on its way is of step t + 2
      turn();
      places(deep1, shallow ^ 2 * STEP, pa, pb);
      at_step(false, t + 2);
      multiply(f1, f0, pa, pb, 0, false, other + shallow);   // (behind the last step: reads that nothing uses)
      deep = deep1;
      shallow ^= 2 * STEP;
      if (t + 1 == kt1) settle();        // (in the loop: whatever leaves it finds the sums done)
    }
    wait_loads<0>();         // nothing may come into LDS that is another's by then
  }

  // Element i of a block's lane is 4 (lane / 16) + i along m, lane % 16 along n.
  const int lane = threadIdx.x & 63, g = lane >> 4, m = m0 + wm * W;
  if (P != LM_LOGITS && t.pieces > 1) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      float* part = a.parts + (int64_t)t.id * T * T + (int64_t)(wn * W + i * 16 + (lane & 15)) * T + wm * W + g * 4;
#pragma unroll
      for (int j = 0; j < NB; ++j) *reinterpret_cast<floatx4*>(part + j * 16) = acc[i][j];
    }
    return;
  }
  constexpr bool BY_ROW = P == LM_GRAD_X && F16;
  const float all = P == LM_LOGITS || BY_ROW ? 1.f : grad_scale<P, F16>(a, 0, 0);
  if (P == LM_GRAD_W && (a.accumulate || a.sum_w)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int n = n0 + wn * W + i * 16 + (lane & 15);
#pragma unroll
      for (int j = 0; j < NB; j += 4) {
        if (n >= s.n || m + j * 16 >= s.m) continue;         // (d is a multiple of 64)
        floatx4 v[4] = {acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]};
        add_grad_w<F16>(a, n, m + j * 16 + g * 4, all, v);
      }
    }
    return;
  }
  turn();                                  // all are done with the steps
  uint16_t* own = lds + w * (W * W);
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int row = i * 16 + (lane & 15), n = n0 + wn * W + row;
    if constexpr (P == LM_LOGITS) {
      store_logits<F16, W>(a, m, n, n < s.n, own, row, acc[i]);
    } else {
      const float scale = BY_ROW ? grad_scale<P, F16>(a, n, s.n) : all;
#pragma unroll
      for (int j = 0; j < NB; ++j)
        put<W>(own, row, 2 * j + (g >> 1), g & 1, round_grad<F16>(acc[i][j] * scale, make_uint2(0, 0), false));
    }
  }
  if (P == LM_LOGITS && !a.e) return;
  wave_lds_handoff();
  constexpr int ROWS = 512 / W;            // of a wave's store
  const int piece = lane % (W / 8), col = m + piece * 8;
  if (P != LM_LOGITS && col >= s.m) return;
#pragma unroll 8
  for (int i = 0; i < W / ROWS; ++i) {
    const int row = i * ROWS + lane / (W / 8), n = n0 + wn * W + row;
    if (n >= s.n) break;
    const u32x4 v = get<W>(own, row, piece);
    uint16_t* to;
    if constexpr (P == LM_LOGITS) to = a.e + (int64_t)n * a.vp + col;
    else if constexpr (P == LM_GRAD_X) to = a.grad_x + (int64_t)a.row_of[a.chunk0 + n] * a.ldgx + col;
    else to = a.grad_w + (int64_t)n * a.ldgw + col;
    *reinterpret_cast<u32x4*>(to) = v;
  }
}

// Joins the pieces of a cut product: 4 K of a tile's rows a workgroup, 64 lanes a row.
template <LmProduct P, bool F16, int K>
__global__ __launch_bounds__(256) void lm_join_kernel(LmArgs a) {
  constexpr int GROUPS = LM_TILE / (4 * K);
  const Sizes s = sizes_of(a, P);
  const int mt = (s.m + LM_TILE - 1) / LM_TILE, nt = (s.n + LM_TILE - 1) / LM_TILE, tiles = mt * nt;
  const int pieces = lm_pieces(tiles, s.nk), j = blockIdx.x / GROUPS;
  if (pieces <= 1 || j >= tiles) return;
  const int group = j / (8 * nt), in = j % (8 * nt), gm = mt - group * 8 < 8 ? mt - group * 8 : 8;
  const int c = (threadIdx.x & 63) * 4, m = (group * 8 + in % gm) * LM_TILE + c;
  if (m >= s.m) return;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int r = (blockIdx.x % GROUPS) * 4 * K + k * 4 + (threadIdx.x >> 6), n = in / gm * LM_TILE + r;
    if (n >= s.n) return;
    const float scale = grad_scale<P, F16>(a, n, s.n);
    const float* p = a.parts + ((int64_t)j * LM_TILE + r) * LM_TILE + c;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = 0; i < pieces; ++i) v += *reinterpret_cast<const floatx4*>(p + (int64_t)i * tiles * LM_TILE * LM_TILE);
    if constexpr (P == LM_GRAD_X) {
      *reinterpret_cast<uint2*>(a.grad_x + (int64_t)a.row_of[a.chunk0 + n] * a.ldgx + m) =
          round_grad<F16>(v * scale, make_uint2(0, 0), false);
    } else {
      floatx4 one[1] = {v};
      add_grad_w<F16>(a, n, m, scale, one);
    }
  }
}

template <LmProduct P, bool F16, int W>
hipError_t launch(const LmArgs& a, hipStream_t st) {
  // the most tiles that the rows with a label can need; workgroups without one end at once
  constexpr int T = 2 * W;
  const int64_t m = P == LM_LOGITS ? a.vocab : a.d, n = P == LM_GRAD_W ? a.vocab : a.chunk;
  const int64_t tiles = ((m + T - 1) / T) * ((n + T - 1) / T);
  const int64_t parts = P == LM_LOGITS || T != LM_TILE ? 0 : lm_parts(a, P);
  lm_product_kernel<P, F16, W><<<(uint32_t)(((tiles > parts ? tiles : parts) + 7) / 8 * 8), NT, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 0) return e;
  const int64_t cut = tiles < 2 * LM_CUS ? tiles : 2 * LM_CUS;      // tiles that may be cut
  // (few tiles have many pieces: a row a wave; 40 rows, 1024, 20000: 6 us against 18)
  if (cut <= 32) lm_join_kernel<P, F16, 1><<<(uint32_t)(cut * 64), 256, 0, st>>>(a);
  else lm_join_kernel<P, F16, 4><<<(uint32_t)(cut * 16), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t lm_parts(const LmArgs& a, LmProduct p) {
  const auto tiles_of = [](int64_t x) { return (int32_t)((x + LM_TILE - 1) / LM_TILE); };
  int64_t most = 0;
  if (p == LM_GRAD_X) {
    for (int32_t nt = 1; nt <= tiles_of(a.chunk); ++nt) {
      const int32_t tiles = tiles_of(a.d) * nt, s = lm_pieces(tiles, (a.vocab + LM_BK - 1) / LM_BK);
      if (s > 1 && (int64_t)tiles * s > most) most = (int64_t)tiles * s;
    }
  } else if (a.chunk > LM_SHORT) {
    const int64_t tiles = (int64_t)tiles_of(a.d) * tiles_of(a.vocab);
    if (tiles <= 2 * LM_CUS)
      for (int32_t nk = 1; nk <= (a.chunk + LM_BK - 1) / LM_BK; ++nk) {
        const int32_t s = lm_pieces((int32_t)tiles, nk);
        if (s > 1 && tiles * s > most) most = tiles * s;
      }
  }
  return most;
}

hipError_t launch_lm_product(const LmArgs& a, LmProduct p, bool f16, hipStream_t st) {
  if (p == LM_LOGITS && a.slab == 64)
    return f16 ? launch<LM_LOGITS, true, 64>(a, st) : launch<LM_LOGITS, false, 64>(a, st);
  if (p == LM_LOGITS) return f16 ? launch<LM_LOGITS, true, 128>(a, st) : launch<LM_LOGITS, false, 128>(a, st);
  if (p == LM_GRAD_X) return f16 ? launch<LM_GRAD_X, true, 128>(a, st) : launch<LM_GRAD_X, false, 128>(a, st);
  // Of a short sum the head's gradient is what costs, all of it written at once: two workgroups a CU, one
  // writing while the other multiplies
  if (a.chunk <= LM_SHORT)
    return f16 ? launch<LM_GRAD_W, true, 64>(a, st) : launch<LM_GRAD_W, false, 64>(a, st);
  return f16 ? launch<LM_GRAD_W, true, 128>(a, st) : launch<LM_GRAD_W, false, 128>(a, st);
}

}  // namespace svl
