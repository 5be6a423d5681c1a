// Device pieces shared by the forward and the backward of the windowed attention.
#pragma once

#include <climits>

#include "attn_ops.h"
#include "device_util.h"

namespace svl {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ u32x4 load_piece(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

template <bool F16>
__device__ __forceinline__ floatx16 mfma32x32x16(const u32x4& a, const u32x4& b, const floatx16& c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b),
                                                  c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                   c, 0, 0, 0);
}

// Four rows x 16 columns of 16-bit values per 16 lanes, transposed: lane l of
// the 16 gives the address of row l / 4, columns 4 (l % 4) .., and gets column l
// of the four rows.
__device__ __forceinline__ uint2 lds_read_tr(const uint16_t* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) shortx4*)p));
}

template <class A>
__device__ __forceinline__ int find_item_seg(const A& a, int item) {
  int lo = 0, hi = a.nsegs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.seg[mid].item0 <= item) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <bool F16> constexpr uint32_t kNonfinite = F16 ? 0x7c00u : 0x7f80u;

template <bool F16>
__device__ __forceinline__ bool any_nonfinite(const u32x4& v) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (v[i] & 0x7fffu) >= kNonfinite<F16> || ((v[i] >> 16) & 0x7fffu) >= kNonfinite<F16>;
  return bad;
}

// Infinities and NaNs to 0.
template <bool F16>
__device__ __forceinline__ u32x4 finite_part(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((v[i] & 0x7fffu) >= kNonfinite<F16>) v[i] &= 0xffff0000u;
    if (((v[i] >> 16) & 0x7fffu) >= kNonfinite<F16>) v[i] &= 0xffffu;
  }
  return v;
}

// 2^x; results below float32's normal range become 0.
__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// Rows of 16-bit values in LDS without padding: the 16-byte piece c of row r is at
// place c ^ lds_swizzle(r).  Both kinds of read are then free of bank conflicts:
// a fragment's (16 bytes of 16 consecutive rows per pass: 16 different places)
// and a transposed one's (64 bytes of 8 rows per pass: each block of 4 places
// twice).  With rows padded to suit one of them the other took 2-4 passes.
template <int D>
__device__ __forceinline__ int lds_swizzle(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

template <int D>
__device__ __forceinline__ int lds_piece(int r, int c) { return r * D + 8 * (c ^ lds_swizzle<D>(r)); }

// Fragment reads: element offset of the lane's row (r0 + lane % 32) and half; step
// s of the head dimension is at (it ^ 16 s), 32 rows further at + 32 D.
template <int D>
__device__ __forceinline__ int lds_frag(int lane) { return lds_piece<D>(lane & 31, lane >> 5); }

// Transposed reads of rows 16 t + 4 (lane / 32) .. and, second, 8 further: element
// offset of the first; columns 32 c .. at (it ^ 32 c), the second at (that ^ 16) + 8 D.
template <int D>
__device__ __forceinline__ int lds_tr(int lane) {
  const int r = 4 * (lane >> 5) + (lane & 15) / 4;
  return lds_piece<D>(r, 2 * ((lane >> 4) & 1) + (lane & 3) / 2) + 4 * (lane & 1);
}

// Loads of tiles of rows by the workgroup's threads: thread t takes the 16-byte
// piece t % (D / 8) of rows t / (D / 8) + STEP i of a tile.  Rows from `rows` on
// read as 0.  Descriptor, tile and step are scalar: a load costs no vector
// address, and where the rows span less than 2 GiB no new descriptor either.
template <int D, int STEP>
struct RowSource {
  __amdgpu_buffer_rsrc_t rsrc;
  const uint16_t* base;
  uint32_t ldb;         // bytes from row to row
  int rows;
  bool far;
  uint32_t lane;        // the thread's offset in a tile
  __device__ __forceinline__ RowSource(const void* p, int64_t row0, int64_t ld, int rows_, int tid)
      : base(static_cast<const uint16_t*>(p) + row0 * ld), ldb((uint32_t)ld * 2), rows(rows_) {
    const int64_t bytes = (int64_t)rows * ldb;
    far = bytes > 0x7fffffff;
    rsrc = make_rsrc(base, far ? 0u : (uint32_t)bytes);
    lane = (uint32_t)(tid / (D / 8)) * ldb + (tid % (D / 8)) * 16;
  }
  // Piece i of the tile at `row`, `col` bytes into its rows.
  __device__ __forceinline__ void tile(int row, uint32_t& soff, uint32_t col) {
    if (far) {
      const int64_t bytes = (int64_t)(rows - row) * ldb;
      rsrc = make_rsrc(base + (int64_t)row * (ldb / 2), (uint32_t)(bytes < 0x7fffffff ? bytes : 0x7fffffff));
      soff = col;
    } else {
      soff = (uint32_t)row * ldb + col;
    }
  }
  __device__ __forceinline__ u32x4 load(uint32_t soff, int i) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane, soff + i * STEP * ldb, 0));
  }
};

// The key tiles that rows at positions p_lo .. p_hi see: of the sinks, then of the
// window; and of them those that every one of these rows sees whole.
template <int BK>
struct KeyTiles {
  int first, n, jump_at, jump_to;
  int whole_hi, whole_lo, whole_sink;
  __device__ __forceinline__ KeyTiles(int p_lo, int p_hi, int window, int sinks) {
    const int start = window > 0 ? max(0, p_lo - window + 1) : 0;
    const int uw = start / BK, us = min((min(sinks, start) + BK - 1) / BK, uw);
    n = us + p_hi / BK + 1 - uw;
    jump_at = us * BK;
    jump_to = uw * BK;
    first = us > 0 ? 0 : jump_to;
    whole_hi = p_lo - BK + 1;
    whole_lo = window > 0 ? p_hi - window : -1;
    whole_sink = sinks - BK;
  }
  __device__ __forceinline__ int after(int kv0) const {
    kv0 += BK;
    return kv0 == jump_at ? jump_to : kv0;
  }
  __device__ __forceinline__ bool whole(int kv0) const {
    return kv0 <= whole_hi && (kv0 > whole_lo || kv0 <= whole_sink);
  }
};

__device__ __forceinline__ u32x4 lds_read16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

// The fragment of rows 16 t .. and columns 32 c .., transposed (tr: lds_tr).
template <int D>
__device__ __forceinline__ u32x4 lds_frag_tr(const uint16_t* rows, int tr, int t, int c) {
  const uint2 lo = lds_read_tr(&rows[(tr ^ 32 * c) + 16 * t * D]);
  const uint2 hi = lds_read_tr(&rows[(tr ^ 32 * c ^ 16) + (16 * t + 8) * D]);
  return u32x4{lo.x, lo.y, hi.x, hi.y};
}

// Two values rounded to 16 bits, in one instruction for either type.
template <bool F16>
__device__ __forceinline__ uint32_t round2(float lo, float hi) {
  if constexpr (F16) {
    return pack_act2<true>(lo, hi);
  } else {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
  }
}

// Elements r .. r + 7 as a fragment.
template <bool F16>
__device__ __forceinline__ u32x4 round8(const floatx16& x, int r) {
  return u32x4{round2<F16>(x[r], x[r + 1]), round2<F16>(x[r + 2], x[r + 3]), round2<F16>(x[r + 4], x[r + 5]),
               round2<F16>(x[r + 6], x[r + 7])};
}

// What rounding elements r .. r + 7 to `hi` took, as a second fragment.
template <bool F16>
__device__ __forceinline__ u32x4 rest8(const floatx16& x, int r, const u32x4& hi) {
  u32x4 lo;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    lo[i] = round2<F16>(x[r + 2 * i] - act_bits_to_f32<F16>(hi[i] & 0xffffu),
                        x[r + 2 * i + 1] - act_bits_to_f32<F16>(hi[i] >> 16));
  return lo;
}

}  // namespace svl
