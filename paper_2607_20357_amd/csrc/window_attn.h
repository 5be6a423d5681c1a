// Device pieces shared by the forward and the backward of the windowed attention.
#pragma once

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

}  // namespace svl
