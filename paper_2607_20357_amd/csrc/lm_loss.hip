// The language-model loss around its matrix products (lm_gemm.hip): the rows with
// a label packed together, log-sums and losses from the slabs' maxima and sums, and
// the exponentials turned into P.
//
// No float32 logits are in memory.  A product's tile leaves exponentials under the
// largest logit of 128 or 64 (a slab) as fp16, and per row and slab that largest and the sum
// in float32; once all slabs are known, e^(slab's - row's largest) / sum makes them the softmax.  That
// costs one pass over 16-bit values in place of a second product of the same size as the
// first, and no rounding that P would not have: fp16 digits under 2^14, before bf16's.
#include "learn_ops.h"
#include "lm_loss.h"
#include "svl_internal.h"

namespace svl {
namespace {

constexpr int NT = 256;

// Numbers the rows with a label in ascending order; their count and largest |weight|.
__global__ __launch_bounds__(1024) void lm_count_kernel(LmArgs a) {
  __shared__ int s_n[16];
  __shared__ float s_w[16];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int n = 0;
  float top = 0.f;
  for (int b = 0; b < a.rows; b += 1024) {
    const int i = b + tid;
    const int label = i < a.rows ? a.labels[i] : -1;
    const bool has = label >= 0 && label < a.vocab;
    const uint64_t all = __ballot(has);
    __syncthreads();
    if (lane == 0) s_n[w] = __popcll(all);
    __syncthreads();
    int before = n;
    for (int k = 0; k < 16; ++k) {
      if (k < w) before += s_n[k];
      n += s_n[k];
    }
    if (has) {
      const int to = before + __popcll(all & (((uint64_t)1 << lane) - 1));
      const float weight = a.row_weight ? a.row_weight[i] : 1.f;
      a.row_of[to] = i;
      a.label[to] = label;
      a.weight[to] = weight;
      top = fmaxf(top, fabsf(weight));
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if (lane == 0) s_w[w] = top;
  __syncthreads();
  if (tid == 0) {
    for (int k = 0; k < 16; ++k) top = fmaxf(top, s_w[k]);
    *a.head = LmHead{n, top};
  }
}

// A row a workgroup: labelled row i is copied to place i (rows behind the last, to a multiple
// of 64, are zeros); a row without a label gets its zeros.
__global__ __launch_bounds__(NT) void lm_pack_kernel(LmArgs a, int packed) {
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const int block = (int)(blockIdx.y * gridDim.x + blockIdx.x);
  if (block >= packed + a.rows) return;
  if (block < packed) {
    const int i = block, n = a.head->rows;
    if (i >= (n + LM_ROWS - 1) / LM_ROWS * LM_ROWS) return;
    const uint16_t* from = i < n ? a.x + (int64_t)a.row_of[i] * a.ldx : nullptr;
    for (int c = threadIdx.x * 8; c < a.d; c += NT * 8)
      *reinterpret_cast<uint4*>(a.xc + (int64_t)i * a.d + c) = from ? *reinterpret_cast<const uint4*>(from + c) : zero;
    return;
  }
  const int i = block - packed, label = a.labels[i];
  if (label >= 0 && label < a.vocab) return;
  if (threadIdx.x == 0) {
    a.loss[i] = 0.f;
    if (a.lse) a.lse[i] = 0.f;
  }
  if (a.grad_x)
    for (int c = threadIdx.x * 8; c < a.d; c += NT * 8)
      *reinterpret_cast<uint4*>(a.grad_x + (int64_t)i * a.ldgx + c) = zero;
}

// Both at once for a call of few rows: each workgroup counts the labels before its row by itself.
__global__ __launch_bounds__(NT) void lm_pack_few_kernel(LmArgs a) {
  __shared__ int s_n[NT / 64][2];
  __shared__ float s_w[NT / 64];
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  int before = 0, all = 0;
  float top = 0.f;
  for (int b = 0; b < a.rows; b += NT) {
    const int r = b + tid, label = r < a.rows ? a.labels[r] : -1;
    const bool has = label >= 0 && label < a.vocab;
    if (has && i == 0) top = fmaxf(top, a.row_weight ? fabsf(a.row_weight[r]) : 1.f);
    all += __popcll(__ballot(has));
    before += __popcll(__ballot(has && r < i));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if (lane == 0) {
    s_n[tid >> 6][0] = before;
    s_n[tid >> 6][1] = all;
    s_w[tid >> 6] = top;
  }
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int k = 0; k < NT / 64; ++k) {
    before += s_n[k][0];
    all += s_n[k][1];
    top = fmaxf(top, s_w[k]);
  }
  if (i == 0 && tid == 0) *a.head = LmHead{all, top};
  const uint4 zero = make_uint4(0, 0, 0, 0);
  if (i >= a.rows) {      // rows of zeros behind the last
    const int to = all + i - a.rows;
    if (to < (all + LM_ROWS - 1) / LM_ROWS * LM_ROWS)
      for (int c = tid * 8; c < a.d; c += NT * 8) *reinterpret_cast<uint4*>(a.xc + (int64_t)to * a.d + c) = zero;
    return;
  }
  const int label = a.labels[i];
  if (label >= 0 && label < a.vocab) {
    if (tid == 0) {
      a.row_of[before] = i;
      a.label[before] = label;
      a.weight[before] = a.row_weight ? a.row_weight[i] : 1.f;
    }
    for (int c = tid * 8; c < a.d; c += NT * 8)
      *reinterpret_cast<uint4*>(a.xc + (int64_t)before * a.d + c) =
          *reinterpret_cast<const uint4*>(a.x + (int64_t)i * a.ldx + c);
    return;
  }
  if (tid == 0) {
    a.loss[i] = 0.f;
    if (a.lse) a.lse[i] = 0.f;
  }
  if (a.grad_x)
    for (int c = tid * 8; c < a.d; c += NT * 8)
      *reinterpret_cast<uint4*>(a.grad_x + (int64_t)i * a.ldgx + c) = zero;
}

// A row a wave.
__global__ __launch_bounds__(NT) void lm_stats_kernel(LmArgs a) {
  const int i = blockIdx.x * (NT / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (i >= a.chunk || a.chunk0 + i >= a.head->rows) return;
  const int slabs = (a.vocab + a.slab - 1) / a.slab;
  const float2* st = a.stats + (int64_t)i * (a.vp / a.slab);
  float top = -INFINITY;
  for (int k = lane; k < slabs; k += 64) top = fmaxf(top, st[k].x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  float sum = 0.f;
  for (int k = lane; k < slabs; k += 64) {
    const float2 v = st[k];
    sum += v.x == -INFINITY ? v.y : v.y * expf(v.x - top);
  }
  sum = warp_sum(sum);
  if (lane != 0) return;
  // The largest and the sum stay apart: their log-sum is rounded at the logits' size (at 30 in steps of 2e-6),
  // which would be all that is left of a sure row's loss and P.
  const float log_sum = logf(sum);
  const int row = a.row_of[a.chunk0 + i];
  a.total[i] = make_float2(top, 1.f / sum);
  a.loss[row] = (top - a.label_logit[i]) + log_sum;
  if (a.lse) a.lse[row] = top + log_sum;
}

// P of a row's 2048 columns a workgroup; rows behind the last, to a multiple of 64, are zeros.
template <bool F16>
__global__ __launch_bounds__(NT) void lm_softmax_kernel(LmArgs a) {
  const int i = blockIdx.x, n = a.head->rows - a.chunk0;
  const int col = blockIdx.y * (NT * 8) + threadIdx.x * 8;
  if (i >= (n + LM_ROWS - 1) / LM_ROWS * LM_ROWS || col >= a.vp) return;
  uint16_t* p = a.e + (int64_t)i * a.vp + col;
  if (i >= n) {
    *reinterpret_cast<uint4*>(p) = make_uint4(0, 0, 0, 0);
    return;
  }
  // (what is known of the row is asked for first: its arrival is waited for once)
  const float2 total = a.total[i];
  const float most = a.head->weight, own = a.weight[a.chunk0 + i];
  const int label = a.label[a.chunk0 + i] - col;
  const float top = a.stats[(int64_t)i * (a.vp / a.slab) + col / a.slab].x;
  const Raw8 raw = {*reinterpret_cast<const uint4*>(p), make_uint4(0, 0, 0, 0)};
  float v[8];
  widen8(raw, SVL_TYPE_F16, v);
  const float under = expf(top - total.x) * total.y, factor = top == -INFINITY ? 1.f : under;
  const float part = lm_part(own, most), weight = F16 && a.grad_x ? part / lm_power(part) : part;
  const float in = factor * weight * (F16 ? 1.f : 1.f / LM_E_SCALE), one = weight * (F16 ? LM_E_SCALE : 1.f);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] *= in;
    if (k == label) v[k] -= one;
  }
  store8(p, F16 ? SVL_TYPE_F16 : SVL_TYPE_BF16, 0, v);
}

// fp16: the power of two of a row's part of the largest weight into its P, exact but for what falls below fp16's
// normal values there.  A row a workgroup; rows whose power is 1 (of equal weights: all) end at once.
__global__ __launch_bounds__(NT) void lm_weigh_kernel(LmArgs a) {
  const int i = blockIdx.x;
  if (i >= a.head->rows - a.chunk0) return;
  const float factor = lm_power(lm_part(a.weight[a.chunk0 + i], a.head->weight));
  if (factor == 1.f) return;
  uint16_t* p = a.e + (int64_t)i * a.vp;
#pragma unroll 4
  for (int c = threadIdx.x * 8; c < a.vp; c += NT * 8) {
    float v[8];
    widen8(Raw8{*reinterpret_cast<const uint4*>(p + c), make_uint4(0, 0, 0, 0)}, SVL_TYPE_F16, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= factor;
    store8(p, SVL_TYPE_F16, c, v);
  }
}

__global__ __launch_bounds__(NT) void lm_zero_w_kernel(uint16_t* w, int64_t ld, int d) {
  for (int c = threadIdx.x * 8; c < d; c += NT * 8)
    *reinterpret_cast<uint4*>(w + (int64_t)blockIdx.x * ld + c) = make_uint4(0, 0, 0, 0);
}

}  // namespace

hipError_t launch_lm_rows(const LmArgs& a, hipStream_t st) {
  if (a.rows <= LM_PACK) {
    lm_pack_few_kernel<<<a.rows + LM_ROWS, NT, 0, st>>>(a);
    return hipGetLastError();
  }
  lm_count_kernel<<<1, 1024, 0, st>>>(a);
  const int packed = (a.rows + LM_ROWS - 1) / LM_ROWS * LM_ROWS;
  // (a grid's first dimension times its threads stays under 2^32)
  const uint32_t blocks = (uint32_t)(packed + a.rows), nx = blocks < (1u << 22) ? blocks : 1u << 22;
  lm_pack_kernel<<<dim3(nx, (blocks + nx - 1) / nx), NT, 0, st>>>(a, packed);
  return hipGetLastError();
}

hipError_t launch_lm_stats(const LmArgs& a, hipStream_t st) {
  lm_stats_kernel<<<(a.chunk + NT / 64 - 1) / (NT / 64), NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_lm_softmax(const LmArgs& a, bool f16, hipStream_t st) {
  const dim3 grid((a.chunk + LM_ROWS - 1) / LM_ROWS * LM_ROWS, (a.vp + NT * 8 - 1) / (NT * 8));
  if (f16) lm_softmax_kernel<true><<<grid, NT, 0, st>>>(a);
  else lm_softmax_kernel<false><<<grid, NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_lm_weigh(const LmArgs& a, hipStream_t st) {
  lm_weigh_kernel<<<a.chunk, NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_lm_zero_w(const LmArgs& a, hipStream_t st) {
  lm_zero_w_kernel<<<a.vocab, NT, 0, st>>>(a.grad_w, a.ldgw, a.d);
  return hipGetLastError();
}

}  // namespace svl
