// Kernel arguments of the operators around the decoder where it learns and
// answers (embedding, row norm, language-model loss, optimizer step), the
// geometry they share with the host, and rows of 32- or 16-bit values.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/svl.h"
#include "device_util.h"

namespace svl {

// ------------------------------------------------------------------ rows
// Eight values of a row as they are in memory: 32 bytes of float, or 16 in `a`.
struct Raw8 {
  uint4 a, b;
};

// The type is the same for all lanes: the branches are scalar.
__device__ __forceinline__ Raw8 load_raw8(const void* p, int32_t type, int64_t i) {
  Raw8 r;
  if (type == SVL_TYPE_F32) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
    r.a = q[0];
    r.b = q[1];
  } else {
    r.a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    r.b = make_uint4(0, 0, 0, 0);
  }
  return r;
}

__device__ __forceinline__ void widen8(const Raw8& r, int32_t type, float* v) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
  if (type == SVL_TYPE_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
  } else if (type == SVL_TYPE_BF16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_bits_to_f32<true>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
  }
}

__device__ __forceinline__ void store8(void* p, int32_t type, int64_t i, const float* v) {
  if (type == SVL_TYPE_F32) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
    return;
  }
  uint4 w;
  if (type == SVL_TYPE_BF16)
    w = make_uint4(pack_act2<false>(v[0], v[1]), pack_act2<false>(v[2], v[3]), pack_act2<false>(v[4], v[5]),
                   pack_act2<false>(v[6], v[7]));
  else
    w = make_uint4(pack_act2<true>(v[0], v[1]), pack_act2<true>(v[2], v[3]), pack_act2<true>(v[4], v[5]),
                   pack_act2<true>(v[6], v[7]));
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = w;
}

// Four values: of float, a wave's pieces follow one another without gaps (8 a lane leave
// its stores half lines: 153M floats 126 us in place of 197).
__device__ __forceinline__ void load4(const void* p, int32_t type, int64_t i, float* v) {
  if (type == SVL_TYPE_F32) {
    const float4 f = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    return;
  }
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
  const uint32_t h[4] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16};
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = type == SVL_TYPE_BF16 ? bf16_bits_to_f32(h[k]) : act_bits_to_f32<true>(h[k]);
}

__device__ __forceinline__ void store4(void* p, int32_t type, int64_t i, const float* v) {
  if (type == SVL_TYPE_F32)
    *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
  else if (type == SVL_TYPE_BF16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) =
        make_uint2(pack_act2<false>(v[0], v[1]), pack_act2<false>(v[2], v[3]));
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) =
        make_uint2(pack_act2<true>(v[0], v[1]), pack_act2<true>(v[2], v[3]));
}

__device__ __forceinline__ float load1(const void* p, int32_t type, int64_t i) {
  if (type == SVL_TYPE_F32) return static_cast<const float*>(p)[i];
  const uint32_t h = static_cast<const uint16_t*>(p)[i];
  return type == SVL_TYPE_BF16 ? bf16_bits_to_f32(h) : act_bits_to_f32<true>(h);
}

__device__ __forceinline__ void store1(void* p, int32_t type, int64_t i, float v) {
  if (type == SVL_TYPE_F32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = type == SVL_TYPE_BF16 ? f32_to_act_bits<false>(v) : f32_to_act_bits<true>(v);
}

// ------------------------------------------------------------------ row norm
struct RowNormArgs {
  const void* x;
  const void* gain;      // or nullptr
  const void* bias;      // or nullptr
  void* y;               // forward
  float* stats;          // forward: written or nullptr; backward: read
  const void* grad_y;    // backward
  void* grad_x;          // or nullptr
  float* partial;        // backward: [pieces][vectors][width], or nullptr
  int64_t ldx, ldy, ldgy, ldgx;
  int32_t rows, width;
  int32_t x_type, y_type, gain_type;
  bool layer;
  bool want_gain, want_bias;
  float eps;
};

// Pieces of the rows whose weight gradients are summed apart, a workgroup each.
constexpr int32_t NORM_PIECES = 512;
int32_t norm_pieces(int32_t rows, int32_t width);

hipError_t launch_row_norm(const RowNormArgs& a, hipStream_t st);
hipError_t launch_row_norm_backward(const RowNormArgs& a, hipStream_t st);
// grad0[c] (and grad1[c], where given) = (accumulate ? what it is : 0) + sum over pieces of
// partial[piece][vector][c]
hipError_t launch_norm_join(const float* partial, int32_t pieces, int32_t width, float* grad0, float* grad1,
                            bool accumulate, hipStream_t st);

// ------------------------------------------------------------------ embedding
struct EmbedArgs {
  const int32_t* tokens;
  const void* table;
  void* out;               // rows (forward) or the table's gradient
  const void* grad_rows;
  int64_t ldt, ldr;        // strides of the table or its gradient, of the rows
  int32_t rows, width, vocab;
  int32_t table_type, row_type;
  float scale;
  bool accumulate;
  // backward: rows ordered by token, and sums of 32 and of 1024 of them
  const uint32_t* key;
  const uint32_t* at;
  int32_t* run;            // [vocab + 1] first places of the tokens' runs
  float* sum32;            // [rows / 32][width], or nullptr
  float* sum1024;          // [rows / 1024][width], or nullptr
};

// The order of rows by token is a radix sort of 8 bits a pass over units of rows.
constexpr int32_t SORT_ALONE = 16384;     // rows that one workgroup sorts in one launch
constexpr int32_t SORT_UNIT = 1024;       // rows of a wave where several workgroups do
struct SortArgs {
  const int32_t* tokens;
  uint32_t* key[2];
  uint32_t* at[2];
  uint32_t* count;         // [256][units]
  int32_t rows, vocab, units, passes;
};

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st);
hipError_t launch_sort_tokens(const SortArgs& s, hipStream_t st);
hipError_t launch_embed_backward(const EmbedArgs& a, hipStream_t st);

// ------------------------------------------------------------------ optimizer
constexpr int32_t ADAMW_BLOCK = 256;      // elements that share an 8-bit state's scale
constexpr int32_t ADAMW_ITEM = 4096;      // elements of a workgroup
constexpr int32_t ADAMW_TENSORS = 48;     // of a launch: they travel in its arguments (under 4 KB)

struct AdamwTensor {
  void* param;
  const void* grad;
  float* master;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  int64_t n;
  int32_t item0;           // first work item
  int16_t param_type, grad_type;
};

struct AdamwArgs {
  AdamwTensor t[ADAMW_TENSORS];
  int32_t count, number0;  // tensors of the launch, and how many of the call came before
  int64_t first_item;      // of t[0], where a tensor is cut between launches
  float beta1, beta2, rest1, rest2, eps, decay;
  svl_adamw_dev now;
  const svl_adamw_dev* dev;
};

hipError_t launch_adamw(const AdamwArgs& a, bool eight, int32_t items, hipStream_t st);
hipError_t launch_adamw_read(bool second, int64_t n, const uint8_t* codes, const float* scales, float* out,
                             hipStream_t st);

}  // namespace svl
