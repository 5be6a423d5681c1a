// RMS and layer norm of rows, forward and backward.
//
//   z = (x - m) r,  y = z gain + bias;  with h = grad_y gain
//   grad_x = r (h - z mean(h z) - [layer] mean(h)),  grad_gain = sum z grad_y,
//   grad_bias = sum grad_y.
//
// Memory bounds both: a row is read once, kept in registers between the sums
// over it and the result, and written once.  In the backward a workgroup takes
// every NORM_PIECES-th row (four rows at once where they are narrow) and keeps its sums
// of the weight gradients in registers; the pieces' sums are joined in order.
#include "learn_ops.h"
#include "svl_internal.h"

namespace svl {
namespace {

// Sums of two values over the row's T threads, the same bits in all of them.
// `s` has room for two calls in turn (`slot` 0 or 1): one barrier a call.
template <int T>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2 (*s)[T / 64], int slot) {
  a = warp_sum(a);
  b = warp_sum(b);
  if constexpr (T > 64) {
    if ((threadIdx.x & 63) == 0) s[slot][threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) {
      a += s[slot][i].x;
      b += s[slot][i].y;
    }
  }
  return make_float2(a, b);
}

template <int C>
__device__ __forceinline__ void load_row(const void* p, int32_t type, int64_t first, const int* col, int width,
                                         Raw8* raw) {
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (col[c] < width) raw[c] = load_raw8(p, type, first + col[c]);
    else raw[c] = Raw8{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
}

// T threads a row, C pieces of 8 values each.
template <int T, int C>
__global__ __launch_bounds__(T < 256 ? 256 : T) void row_norm_kernel(RowNormArgs a) {
  constexpr int PER = T < 256 ? 256 / T : 1;   // rows of a workgroup
  __shared__ float2 s[2][T / 64];
  const int t = threadIdx.x % T;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * PER + threadIdx.x / T;
  if (row >= a.rows) return;                   // (whole waves where PER > 1: no barrier then)
  int col[C];
#pragma unroll
  for (int c = 0; c < C; ++c) col[c] = (c * T + t) * 8;

  Raw8 raw[C], graw[C], braw[C];
  load_row<C>(a.x, a.x_type, row * a.ldx, col, a.width, raw);
  if (a.gain) load_row<C>(a.gain, a.gain_type, 0, col, a.width, graw);
  if (a.bias) load_row<C>(a.bias, a.gain_type, 0, col, a.width, braw);

  float v[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) widen8(raw[c], a.x_type, v[c]);
  float mean = 0.f;
  if (a.layer) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[c][i];
    mean = row_sum2<T>(sum, 0.f, s, 0).x / (float)a.width;
  }
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
    if (col[c] < a.width)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[c][i] -= mean;
        sq += v[c][i] * v[c][i];
      }
  const float r = 1.f / sqrtf(row_sum2<T>(sq, 0.f, s, 1).x / (float)a.width + a.eps);
  if (a.stats && t == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, r);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (col[c] >= a.width) continue;
    float g[8], b[8];
    if (a.gain) widen8(graw[c], a.gain_type, g);
    if (a.bias) widen8(braw[c], a.gain_type, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[c][i] *= r;
      if (a.gain) v[c][i] *= g[i];
      if (a.bias) v[c][i] += b[i];
    }
    store8(a.y, a.y_type, row * a.ldy + col[c], v[c]);
  }
}

// A workgroup takes every pieces-th group of PER rows; where PER > 1 its waves' sums of the weight
// gradients meet in LDS, so that narrow rows leave no more of them than wide ones.
template <int T, int C>
__global__ __launch_bounds__(T < 256 ? 256 : T) void row_norm_backward_kernel(RowNormArgs a, int32_t pieces) {
  constexpr int PER = T < 256 ? 256 / T : 1;
  __shared__ float2 s[2][T / 64];
  const int t = threadIdx.x % T;
  int col[C];
  float g[C][8], dg[C][8], db[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    col[c] = (c * T + t) * 8;
    Raw8 raw;
    const bool there = a.gain && col[c] < a.width;
    if (there) raw = load_raw8(a.gain, a.gain_type, col[c]);
    if (there) widen8(raw, a.gain_type, g[c]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (!there) g[c][i] = 1.f;
      dg[c][i] = db[c][i] = 0.f;
    }
  }
  const float inv = 1.f / (float)a.width;
  int slot = 0;
  for (int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / T; row < a.rows; row += (int64_t)pieces * PER, slot ^= 1) {
    Raw8 xr[C], yr[C];
    load_row<C>(a.x, a.x_type, row * a.ldx, col, a.width, xr);
    load_row<C>(a.grad_y, a.y_type, row * a.ldgy, col, a.width, yr);
    const float2 st = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    float z[C][8], h[C][8], hs = 0.f, hz = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (col[c] >= a.width) continue;
      widen8(xr[c], a.x_type, z[c]);
      widen8(yr[c], a.y_type, h[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        z[c][i] = (z[c][i] - st.x) * st.y;
        dg[c][i] += h[c][i] * z[c][i];
        db[c][i] += h[c][i];
        h[c][i] *= g[c][i];
        hs += h[c][i];
        hz += h[c][i] * z[c][i];
      }
    }
    if (!a.grad_x) continue;
    const float2 sum = row_sum2<T>(hs, hz, s, slot);
    const float shift = a.layer ? sum.x * inv : 0.f, along = sum.y * inv;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (col[c] >= a.width) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[c][i] = (h[c][i] - z[c][i] * along - shift) * st.y;
      store8(a.grad_x, a.x_type, row * a.ldgx + col[c], h[c]);
    }
  }
  if (!a.want_gain && !a.want_bias) return;
  if constexpr (PER > 1) {
    __shared__ float w[PER - 1][2 * C * 8][T];
    const int r = threadIdx.x / T;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r > 0) {
          w[r - 1][(c * 8 + i) * 2][t] = dg[c][i];
          w[r - 1][(c * 8 + i) * 2 + 1][t] = db[c][i];
        }
    __syncthreads();
    if (r > 0) return;
    for (int k = 0; k < PER - 1; ++k)
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dg[c][i] += w[k][(c * 8 + i) * 2][t];
          db[c][i] += w[k][(c * 8 + i) * 2 + 1][t];
        }
  }
  float* part = a.partial + (int64_t)blockIdx.x * (a.want_gain + a.want_bias) * a.width;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (col[c] >= a.width) continue;
    if (a.want_gain) store8(part, SVL_TYPE_F32, col[c], dg[c]);
    if (a.want_bias) store8(part + (a.want_gain ? a.width : 0), SVL_TYPE_F32, col[c], db[c]);
  }
}

// 16 columns a workgroup, 64 groups of pieces; a vector of the partial sums each grid row.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* partial, int32_t pieces, int32_t width,
                                                         float* grad0, float* grad1, bool accumulate) {
  __shared__ float s[64][17];
  const int c = blockIdx.x * 16 + threadIdx.x % 16, g = threadIdx.x / 16;
  const int64_t stride = (int64_t)gridDim.y * width;
  partial += (int64_t)blockIdx.y * width;
  float* grad = blockIdx.y ? grad1 : grad0;
  float sum = 0.f;
  if (c < width)
#pragma unroll 4
    for (int p = g; p < pieces; p += 64) sum += partial[(int64_t)p * stride + c];
  s[g][threadIdx.x % 16] = sum;
  __syncthreads();
  if (g != 0 || c >= width) return;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < 64; ++i) sum += s[i][threadIdx.x];
  grad[c] = accumulate ? grad[c] + sum : sum;
}

// The smallest of the shapes whose threads hold the row.
template <class F>
hipError_t by_width(int32_t width, const F& f) {
  if (width <= 512) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  if (width <= 1024) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  if (width <= 2048) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
  if (width <= 4096) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
  if (width <= 8192) return f(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}

}  // namespace

hipError_t launch_row_norm(const RowNormArgs& a, hipStream_t st) {
  return by_width(a.width, [&](auto t, auto c) {
    constexpr int T = decltype(t)::value, C = decltype(c)::value, PER = T < 256 ? 256 / T : 1;
    // (a grid's first dimension times its threads stays under 2^32)
    const uint32_t blocks = (a.rows + PER - 1) / PER, nx = blocks < (1u << 20) ? blocks : 1u << 20;
    row_norm_kernel<T, C><<<dim3(nx, (blocks + nx - 1) / nx), T * PER, 0, st>>>(a);
    return hipGetLastError();
  });
}

int32_t norm_pieces(int32_t rows, int32_t width) {
  const int32_t per = width <= 1024 ? 4 : 1, groups = (rows + per - 1) / per;
  return groups < NORM_PIECES ? groups : NORM_PIECES;
}

hipError_t launch_row_norm_backward(const RowNormArgs& a, hipStream_t st) {
  const int32_t pieces = norm_pieces(a.rows, a.width);
  return by_width(a.width, [&](auto t, auto c) {
    constexpr int T = decltype(t)::value, C = decltype(c)::value, PER = T < 256 ? 256 / T : 1;
    row_norm_backward_kernel<T, C><<<pieces, T * PER, 0, st>>>(a, pieces);
    return hipGetLastError();
  });
}

hipError_t launch_norm_join(const float* partial, int32_t pieces, int32_t width, float* grad0, float* grad1,
                            bool accumulate, hipStream_t st) {
  norm_join_kernel<<<dim3((width + 15) / 16, grad1 ? 2 : 1), 1024, 0, st>>>(partial, pieces, width, grad0, grad1,
                                                                          accumulate);
  return hipGetLastError();
}

}  // namespace svl
