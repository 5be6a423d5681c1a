// One AdamW step over many tensors, with states in 32 bits or in 8.
//
// Memory bounds it: each array is read once and written once.  A workgroup
// takes 4096 elements of one tensor, a thread 4 in a row at a time; the tensors
// travel in the kernel's arguments, so a launch serves 48 of them.
//
// 8-bit states hold a block of 256 under a power of two, so that scaling is exact
// and the codes are digits of the value itself: three bits after the point, 15
// binades for the first moment, 31 for the root of the second, below them
// evenly spaced down to 0.  A second moment that decays by a twentieth or a
// thousandth a step never leaves its code where codes are rounded to the nearest
// (a step is an eighth); rounded up or down by chance it does so on average.
#include "learn_ops.h"
#include "svl_internal.h"

namespace svl {
namespace {

constexpr int NT = 256, EL = 4;           // EL elements a thread: a wave's are a block of 256
constexpr int LOW_M = -13, LOW_V = -29;   // lowest exponent with all digits, of scale 1

__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;   // the digits of sqrt(2), sqrt(3) and the golden ratio: odd numbers without a pattern
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

// A code's value under scale 1: bits 0 .. 2 after the point, the exponent above.
__device__ __forceinline__ float code_value(uint32_t c, int low) {
  const float normal = __uint_as_float((c + ((uint32_t)(126 + low) << 3)) << 20);
  const float small = (float)(c & 7u) * __uint_as_float((uint32_t)(127 + low - 3) << 23);
  return c >= 8u ? normal : small;
}

// The code next to y >= 0 (under scale 1): above it with the chance that 16 random bits give.  (Both
// forms are computed and one is taken: a branch costs the wave more.)
__device__ __forceinline__ uint32_t code_of(float y, uint32_t r16, int low) {
  const uint32_t up = r16 << 4;
  const uint32_t normal = ((__float_as_uint(y) + up) >> 20) - ((uint32_t)(126 + low) << 3);
  const uint32_t small = ((uint32_t)(y * __uint_as_float((uint32_t)(127 + 23 - low) << 23)) + up) >> 20;
  return y >= __uint_as_float((uint32_t)(127 + low) << 23) ? normal : small;
}

// The largest magnitude's bits over a block, a wave's; NaN counts as the largest.
__device__ __forceinline__ uint32_t block_top(const float* x) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint32_t b = __shfl_xor(top, o, 64);
    top = b > top ? b : top;
  }
  return top;
}

// The scale of a block whose largest magnitude has these bits, and its reciprocal.
__device__ __forceinline__ float block_scale(uint32_t top, float* inverse) {
  if (top >= 0x7f800000u) {
    *inverse = 0.f;
    return __uint_as_float(0x7fc00000u);
  }
  if (top == 0) {
    *inverse = 0.f;
    return 0.f;
  }
  const uint32_t e = (top >> 23) > 37u ? top >> 23 : 37u;   // 2^-90
  *inverse = __uint_as_float((254u - e) << 23);
  return __uint_as_float(e << 23);
}

// FULL: all of the lane's elements are there, otherwise the first `valid`.
template <bool FULL>
__device__ __forceinline__ void load_codes(const void* p, int64_t i, int valid, uint32_t* c) {
  if constexpr (FULL) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p) + i);
#pragma unroll
    for (int k = 0; k < EL; ++k) c[k] = (w >> (8 * k)) & 255u;
  } else {
#pragma unroll
    for (int k = 0; k < EL; ++k) c[k] = k < valid ? static_cast<const uint8_t*>(p)[i + k] : 0u;
  }
}

template <bool FULL>
__device__ __forceinline__ void store_codes(void* p, int64_t i, int valid, const uint32_t* c) {
  if constexpr (FULL) {
    *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p) + i) = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
  } else {
#pragma unroll
    for (int k = 0; k < EL; ++k)
      if (k < valid) static_cast<uint8_t*>(p)[i + k] = (uint8_t)c[k];
  }
}

template <bool FULL>
__device__ __forceinline__ void load_some(const void* p, int32_t type, int64_t i, int valid, float* v) {
  if constexpr (FULL) {
    load4(p, type, i, v);
  } else {
#pragma unroll
    for (int k = 0; k < EL; ++k) v[k] = k < valid ? load1(p, type, i + k) : 0.f;
  }
}

template <bool FULL>
__device__ __forceinline__ void store_some(void* p, int32_t type, int64_t i, int valid, const float* v) {
  if constexpr (FULL) {
    store4(p, type, i, v);
  } else {
#pragma unroll
    for (int k = 0; k < EL; ++k)
      if (k < valid) store1(p, type, i + k, v[k]);
  }
}

// What a step's factors are, once a workgroup.
struct StepNow {
  float keep, lr, grad_scale, inverse1, inverse_root2;   // 1 - lr decay; 1 / correction1, 1 / sqrt(correction2)
  uint32_t seed;
};

// Elements i .. of a tensor: a wave's are a block of 256.
template <bool EIGHT, bool FULL>
__device__ __forceinline__ void adamw_block(const AdamwArgs& a, const AdamwTensor& t, const StepNow& now,
                                            uint32_t number, int64_t i) {
// the moments' products and sums are rounded one by one: 8-bit codes depend on every bit
#pragma clang fp contract(off)
  const int64_t left = t.n - i;
  const int valid = left >= EL ? EL : left > 0 ? (int)left : 0;
  float g[EL], p[EL], m[EL], v[EL];
  load_some<FULL>(t.grad, t.grad_type, i, valid, g);
  if (t.master) load_some<FULL>(t.master, SVL_TYPE_F32, i, valid, p);
  else load_some<FULL>(t.param, t.param_type, i, valid, p);
  if constexpr (EIGHT) {
    uint32_t cm[EL], cv[EL];
    load_codes<FULL>(t.m, i, valid, cm);
    load_codes<FULL>(t.v, i, valid, cv);
    const float sm = FULL || valid ? t.m_scale[i / ADAMW_BLOCK] : 0.f;
    const float sv = FULL || valid ? t.v_scale[i / ADAMW_BLOCK] : 0.f;
#pragma unroll
    for (int k = 0; k < EL; ++k) {
      const float x = sm * code_value(cm[k] & 127u, LOW_M), y = sv * code_value(cv[k], LOW_V);
      m[k] = cm[k] & 128u ? -x : x;
      v[k] = y * y;
    }
  } else {
    load_some<FULL>(t.m, SVL_TYPE_F32, i, valid, m);
    load_some<FULL>(t.v, SVL_TYPE_F32, i, valid, v);
  }
  float root[EL];
#pragma unroll
  for (int k = 0; k < EL; ++k) {
    const float x = g[k] * now.grad_scale;
    m[k] = a.beta1 * m[k] + a.rest1 * x;
    v[k] = a.beta2 * v[k] + (a.rest2 * x) * x;
    if (!FULL && k >= valid) m[k] = v[k] = 0.f;
    root[k] = sqrtf(v[k]);
    // (the quotient by the hardware's reciprocal: a last place of a step that is far smaller than p)
    p[k] = p[k] * now.keep -
           now.lr * ((m[k] * now.inverse1) * __builtin_amdgcn_rcpf(root[k] * now.inverse_root2 + a.eps));
  }
  if (t.master) store_some<FULL>(t.master, SVL_TYPE_F32, i, valid, p);
  store_some<FULL>(t.param, t.param_type, i, valid, p);
  if constexpr (EIGHT) {
    const uint32_t key = mix(now.seed + 0x9E3779B9u * (number + 1) + 0xBB67AE85u * (uint32_t)(i >> 32));
    float im, iv;
    const float sm = block_scale(block_top(m), &im), sv = block_scale(block_top(root), &iv);
    uint32_t cm[EL], cv[EL];
#pragma unroll
    for (int k = 0; k < EL; ++k) {
      const uint32_t r = mix((uint32_t)(i + k) * 0x9E3779B9u + key);
      cm[k] = im == 0.f ? 0u : code_of(fabsf(m[k]) * im, r & 0xffffu, LOW_M) | (m[k] < 0.f ? 128u : 0u);
      cv[k] = iv == 0.f ? 0u : code_of(root[k] * iv, r >> 16, LOW_V);
    }
    store_codes<FULL>(t.m, i, valid, cm);
    store_codes<FULL>(t.v, i, valid, cv);
    if ((FULL || valid) && (threadIdx.x & 63) == 0) {
      t.m_scale[i / ADAMW_BLOCK] = sm;
      t.v_scale[i / ADAMW_BLOCK] = sv;
    }
  } else {
    store_some<FULL>(t.m, SVL_TYPE_F32, i, valid, m);
    store_some<FULL>(t.v, SVL_TYPE_F32, i, valid, v);
  }
}

template <bool EIGHT>
__global__ __launch_bounds__(NT) void adamw_kernel(AdamwArgs a) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.t[mid].item0 <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const AdamwTensor& t = a.t[lo];
  const svl_adamw_dev d = a.dev ? *a.dev : a.now;
  const StepNow now = {1.f - d.lr * a.decay, d.lr, d.grad_scale, 1.f / d.correction1, 1.f / sqrtf(d.correction2), d.seed};
  const int64_t item = (int)blockIdx.x - t.item0 + (lo == 0 ? a.first_item : 0);
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll 1
  for (int it = 0; it < ADAMW_ITEM / (NT * EL); ++it) {
    const int64_t first = item * ADAMW_ITEM + it * (NT * EL) + w * ADAMW_BLOCK;
    if (first >= t.n) return;
    const int64_t i = first + (threadIdx.x & 63) * EL;
    if (first + ADAMW_BLOCK <= t.n) adamw_block<EIGHT, true>(a, t, now, (uint32_t)(a.number0 + lo), i);
    else adamw_block<EIGHT, false>(a, t, now, (uint32_t)(a.number0 + lo), i);
  }
}

// READS pieces of 4 a thread, a wave's in a row: what it writes leaves in whole lines.
constexpr int READS = 4;
__global__ __launch_bounds__(NT) void adamw_read_kernel(bool second, int64_t n, const uint8_t* codes,
                                                        const float* scales, float* out) {
#pragma clang fp contract(off)
  const int64_t i0 = ((int64_t)blockIdx.x * READS * NT + threadIdx.x) * 4;
  const auto value = [&](uint32_t c, float s) {
    const float x = s * code_value(second ? c : c & 127u, second ? LOW_V : LOW_M);
    return second ? x * x : c & 128u ? -x : x;
  };
  if (i0 + (int64_t)(READS - 1) * NT * 4 + 4 > n) {
    for (int j = 0; j < READS; ++j)
      for (int64_t i = i0 + (int64_t)j * NT * 4; i < i0 + (int64_t)j * NT * 4 + 4 && i < n; ++i)
        out[i] = value(codes[i], scales[i / ADAMW_BLOCK]);
    return;
  }
  uint32_t c[READS];
  float s[READS];
#pragma unroll
  for (int j = 0; j < READS; ++j) {
    const int64_t i = i0 + (int64_t)j * NT * 4;
    c[j] = *reinterpret_cast<const uint32_t*>(codes + i);
    s[j] = scales[i / ADAMW_BLOCK];
  }
#pragma unroll
  for (int j = 0; j < READS; ++j)
    *reinterpret_cast<float4*>(out + i0 + (int64_t)j * NT * 4) =
        make_float4(value(c[j] & 255u, s[j]), value(c[j] >> 8 & 255u, s[j]), value(c[j] >> 16 & 255u, s[j]),
                    value(c[j] >> 24, s[j]));
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, bool eight, int32_t items, hipStream_t st) {
  if (eight) adamw_kernel<true><<<items, NT, 0, st>>>(a);
  else adamw_kernel<false><<<items, NT, 0, st>>>(a);
  return hipGetLastError();
}

// (a launch's threads stay under 2^32)
hipError_t launch_adamw_read(bool second, int64_t n, const uint8_t* codes, const float* scales, float* out,
                             hipStream_t st) {
  constexpr int64_t PART = (int64_t)1 << 32;
  for (int64_t i = 0; i < n; i += PART) {
    const int64_t part = n - i < PART ? n - i : PART;
    adamw_read_kernel<<<(uint32_t)((part + READS * NT * 4 - 1) / (READS * NT * 4)), NT, 0, st>>>(second, part, codes + i,
                                                                               scales + i / ADAMW_BLOCK, out + i);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace svl
