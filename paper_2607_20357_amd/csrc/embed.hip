// Rows of an embedding table by token, and the table's gradient.
//
// The gradient is a sum over the rows of each token.  Rows are put in the order
// of their tokens by a radix sort that keeps the order of equal ones, then a
// workgroup per table row sums its run of rows in that order, so the result has
// the same bits on every call and no atomic touches a value.  A run's whole
// aligned pieces of 32 and of 1024 rows are summed before, side by side, so that a
// token that fills the batch costs no more than one that is rare.  Memory bounds
// it: every gradient row is read once, every table row written once.
#include "learn_ops.h"
#include "svl_internal.h"

namespace svl {
namespace {

constexpr int NT = 256;
constexpr int SLAB = NT * 8;   // columns of a workgroup

__global__ __launch_bounds__(NT) void embed_kernel(EmbedArgs a) {
  const int64_t row = blockIdx.x;
  const int col = blockIdx.y * SLAB + threadIdx.x * 8;
  if (col >= a.width) return;
  const int32_t tok = a.tokens[row];
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (tok >= 0 && tok < a.vocab) {
    widen8(load_raw8(a.table, a.table_type, (int64_t)tok * a.ldt + col), a.table_type, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= a.scale;
  }
  store8(a.out, a.row_type, row * a.ldr + col, v);
}

// ------------------------------------------------------------------ order
// A token outside the table counts as one behind it.
__device__ __forceinline__ uint32_t token_key(const SortArgs& s, int i) {
  const int32_t t = s.tokens[i];
  return t >= 0 && t < s.vocab ? (uint32_t)t : (uint32_t)s.vocab;
}

__device__ __forceinline__ void sort_source(const SortArgs& s, int pass, int i, uint32_t* key, uint32_t* at) {
  if (pass == 0) {
    *key = token_key(s, i);
    *at = (uint32_t)i;
  } else {
    *key = s.key[(pass - 1) & 1][i];
    *at = s.at[(pass - 1) & 1][i];
  }
}

// A wave's rows [i0, i1), at most SORT_UNIT, in registers: all loads at once, then LDS alone.
constexpr int EACH = SORT_UNIT / 64;
struct Unit {
  uint32_t key[EACH], at[EACH];
};
__device__ __forceinline__ void load_unit(const SortArgs& s, int pass, int i0, int i1, Unit& u) {
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int i = i0 + k * 64 + (int)(threadIdx.x & 63);
    u.key[k] = u.at[k] = 0;
    if (i < i1) sort_source(s, pass, i, &u.key[k], &u.at[k]);
  }
}

// Counts of the unit's digits into cnt[256] (LDS, cleared before).
__device__ __forceinline__ void count_unit(int pass, int i0, int i1, const Unit& u, uint32_t* cnt) {
#pragma unroll
  for (int k = 0; k < EACH; ++k)
    if (i0 + k * 64 + (int)(threadIdx.x & 63) < i1)
      atomicAdd(&cnt[(u.key[k] >> (8 * pass)) & 255u], 1u);   // whole numbers: any order
}

// Moves the unit's rows to where their digit's next place is (cnt: first places): put(place, key, at).
template <class Put>
__device__ __forceinline__ void move_unit(int pass, int i0, int i1, const Unit& u, uint32_t* cnt, const Put& put) {
  const int lane = threadIdx.x & 63;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int b = 0; b < EACH; ++b) {
    if (i0 + b * 64 >= i1) break;
    const bool there = i0 + b * 64 + lane < i1;
    const uint32_t digit = (u.key[b] >> (8 * pass)) & 255u;
    uint64_t same = __ballot(there);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint64_t one = __ballot((digit >> k) & 1u);
      same &= (digit >> k) & 1u ? one : ~one;
    }
    if (there) put(cnt[digit] + (uint32_t)__popcll(same & below), u.key[b], u.at[b]);
    wave_lds_handoff();
    if (there && (same & below) == 0) cnt[digit] += (uint32_t)__popcll(same);
    wave_lds_handoff();
  }
}

// Exclusive sums of v over the workgroup's threads (at most 16 waves).
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* s, uint32_t* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s[w] = x;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int i = 0; i < nw; ++i) {
    if (i < w) before += s[i];
    all += s[i];
  }
  *total = all;
  return before + x - v;
}

// One workgroup, the rows in LDS between the passes: 16384 rows of a vocabulary of 32000 41 us (8192 21,
// 1024 8), most of it the ballots of move_unit; several workgroups take six launches for it.
__global__ __launch_bounds__(1024) void sort_alone_kernel(SortArgs s) {
  __shared__ uint32_t cnt[16][256];
  __shared__ uint32_t sums[16];
  __shared__ uint32_t key[SORT_ALONE];
  __shared__ uint16_t at[SORT_ALONE];
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int seg = ((s.rows + 1023) / 1024) * 64;
  const int i0 = w * seg < s.rows ? w * seg : s.rows;
  const int i1 = i0 + seg < s.rows ? i0 + seg : s.rows;
  for (int pass = 0; pass < s.passes; ++pass) {
    for (int i = tid; i < 16 * 256; i += 1024) (&cnt[0][0])[i] = 0;
    Unit u;
    if (pass == 0) {
      load_unit(s, 0, i0, i1, u);
    } else {
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        const int i = i0 + k * 64 + lane;
        u.key[k] = i < i1 ? key[i] : 0;
        u.at[k] = i < i1 ? at[i] : 0;
      }
    }
    __syncthreads();
    count_unit(pass, i0, i1, u, cnt[w]);
    __syncthreads();
    uint32_t n = 0, all;
    if (tid < 256)
      for (int k = 0; k < 16; ++k) n += cnt[k][tid];
    uint32_t first = block_before(n, sums, &all);
    if (tid < 256)
      for (int k = 0; k < 16; ++k) {
        const uint32_t c = cnt[k][tid];
        cnt[k][tid] = first;
        first += c;
      }
    __syncthreads();
    move_unit(pass, i0, i1, u, cnt[w], [&](uint32_t to, uint32_t k, uint32_t a) {
      key[to] = k;
      at[to] = (uint16_t)a;
    });
    __syncthreads();   // the pass's rows are there before the next one reads them
  }
  uint32_t* to_key = s.key[(s.passes - 1) & 1];
  uint32_t* to_at = s.at[(s.passes - 1) & 1];
  for (int i = tid; i < s.rows; i += 1024) {
    to_key[i] = key[i];
    to_at[i] = at[i];
  }
}

__global__ __launch_bounds__(NT) void sort_count_kernel(SortArgs s, int pass) {
  __shared__ uint32_t cnt[4][256];
  const int tid = threadIdx.x, w = tid >> 6, unit = blockIdx.x * 4 + w;
  for (int i = tid; i < 4 * 256; i += NT) (&cnt[0][0])[i] = 0;
  __syncthreads();
  if (unit < s.units) {
    const int i0 = unit * SORT_UNIT, i1 = i0 + SORT_UNIT < s.rows ? i0 + SORT_UNIT : s.rows;
    Unit u;
    load_unit(s, pass, i0, i1, u);
    count_unit(pass, i0, i1, u, cnt[w]);
  }
  __syncthreads();
  for (int i = tid; i < 4 * 256; i += NT) {
    const int u = blockIdx.x * 4 + i / 256;
    if (u < s.units) s.count[(int64_t)(i % 256) * s.units + u] = cnt[i / 256][i % 256];
  }
}

// Counts [digit][unit] to first places.
__global__ __launch_bounds__(1024) void sort_scan_kernel(SortArgs s) {
  __shared__ uint32_t sums[16];
  const int64_t n = 256 * (int64_t)s.units;
  uint32_t carry = 0;
  for (int64_t b = 0; b < n; b += 4096) {
    const int64_t i = b + threadIdx.x * 4;   // (n is a multiple of 256)
    uint4 c = make_uint4(0, 0, 0, 0);
    if (i < n) c = *reinterpret_cast<const uint4*>(s.count + i);
    uint32_t all;
    uint32_t first = carry + block_before(c.x + c.y + c.z + c.w, sums, &all);
    if (i < n)
      *reinterpret_cast<uint4*>(s.count + i) =
          make_uint4(first, first + c.x, first + c.x + c.y, first + c.x + c.y + c.z);
    carry += all;
  }
}

__global__ __launch_bounds__(NT) void sort_move_kernel(SortArgs s, int pass) {
  __shared__ uint32_t cnt[4][256];
  const int tid = threadIdx.x, w = tid >> 6, unit = blockIdx.x * 4 + w;
  for (int i = tid; i < 4 * 256; i += NT) {
    const int u = blockIdx.x * 4 + i / 256;
    cnt[i / 256][i % 256] = u < s.units ? s.count[(int64_t)(i % 256) * s.units + u] : 0;
  }
  __syncthreads();
  if (unit >= s.units) return;
  const int i0 = unit * SORT_UNIT, i1 = i0 + SORT_UNIT < s.rows ? i0 + SORT_UNIT : s.rows;
  Unit u;
  load_unit(s, pass, i0, i1, u);
  move_unit(pass, i0, i1, u, cnt[w], [&](uint32_t to, uint32_t k, uint32_t a) {
    s.key[pass & 1][to] = k;
    s.at[pass & 1][to] = a;
  });
}

// ------------------------------------------------------------------ sums
// Where each token's run begins: the first place whose key is at least v, for v = 0 .. vocab.
__global__ __launch_bounds__(NT) void embed_runs_kernel(EmbedArgs a) {
  const int v = blockIdx.x * NT + threadIdx.x;
  if (v > a.vocab) return;
  int lo = 0, hi = a.rows;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.key[mid] < (uint32_t)v) lo = mid + 1; else hi = mid;
  }
  a.run[v] = lo;
}

// Rows of places [i0, i1): their numbers by the wave together, then FLIGHT rows at a time
// (behind the last one the last again, which is not added).
constexpr int FLIGHT = 8;
template <bool WIDE>
__device__ __forceinline__ void add_rows_of(const EmbedArgs& a, int i0, int i1, int col, float* sum) {
  const int lane = threadIdx.x & 63;
  const int32_t type = WIDE ? (int32_t)SVL_TYPE_F32 : a.row_type == SVL_TYPE_BF16 ? SVL_TYPE_BF16 : SVL_TYPE_F16;
  for (int b = i0; b < i1; b += 64) {
    const int n = i1 - b < 64 ? i1 - b : 64;
    const uint32_t at = lane < n ? a.at[b + lane] : 0;
#pragma unroll 1
    for (int i = 0; i < n; i += FLIGHT) {
      Raw8 raw[FLIGHT];
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        const int j = i + k < n ? i + k : n - 1;
        raw[k] = load_raw8(a.grad_rows, type, (int64_t)__builtin_amdgcn_readlane((int)at, j) * a.ldr + col);
      }
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        if (i + k >= n) break;
        float v[8];
        widen8(raw[k], type, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] += v[c];
      }
    }
  }
}
__device__ __forceinline__ void add_rows(const EmbedArgs& a, int i0, int i1, int col, float* sum) {
  if (a.row_type == SVL_TYPE_F32) add_rows_of<true>(a, i0, i1, col, sum);
  else add_rows_of<false>(a, i0, i1, col, sum);
}

__device__ __forceinline__ void add_pieces(const float* piece, int width, int i0, int i1, int col, float* sum) {
#pragma unroll 4
  for (int i = i0; i < i1; ++i) {
    const float4* p = reinterpret_cast<const float4*>(piece + (int64_t)i * width + col);
    const float4 x = p[0], y = p[1];
    sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
    sum[4] += y.x; sum[5] += y.y; sum[6] += y.z; sum[7] += y.w;
  }
}

// Sums of the aligned pieces of N places that lie inside one run (N = 32: of rows; 1024: of pieces of 32).
template <int N>
__global__ __launch_bounds__(NT) void embed_pieces_kernel(EmbedArgs a) {
  const int p = blockIdx.x;
  const int col = blockIdx.y * SLAB + threadIdx.x * 8;
  const uint32_t key = a.key[p * N];
  // (columns behind the last load the last: their wave reads places together)
  if (key >= (uint32_t)a.vocab || a.key[p * N + N - 1] != key) return;
  const int from = col < a.width ? col : a.width - 8;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if constexpr (N == 32) add_rows(a, p * N, p * N + N, from, sum);
  else add_pieces(a.sum32, a.width, p * 32, p * 32 + 32, from, sum);
  if (col < a.width) store8((N == 32 ? a.sum32 : a.sum1024) + (int64_t)p * a.width, SVL_TYPE_F32, col, sum);
}

// One table row a workgroup (BY_PLACE: a place of the order that begins a run).
template <bool BY_PLACE>
__global__ __launch_bounds__(NT) void embed_sum_kernel(EmbedArgs a) {
  const int col = blockIdx.y * SLAB + threadIdx.x * 8, from = col < a.width ? col : a.width - 8;
  uint32_t key = blockIdx.x;
  if constexpr (BY_PLACE) {
    const int i = blockIdx.x;
    key = a.key[i];
    if (key >= (uint32_t)a.vocab || (i > 0 && a.key[i - 1] == key)) return;
  }
  const int lo = a.run[key], hi = a.run[key + 1];
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int p0 = (lo + 31) / 32, p1 = hi / 32;           // whole pieces of 32
  if (!a.sum32 || p0 >= p1) {
    add_rows(a, lo, hi, from, sum);
  } else {
    add_rows(a, lo, p0 * 32, from, sum);
    const int q0 = (p0 + 31) / 32, q1 = p1 / 32;         // whole pieces of 1024
    if (!a.sum1024 || q0 >= q1) {
      add_pieces(a.sum32, a.width, p0, p1, from, sum);
    } else {
      add_pieces(a.sum32, a.width, p0, q0 * 32, from, sum);
      add_pieces(a.sum1024, a.width, q0, q1, from, sum);
      add_pieces(a.sum32, a.width, q1 * 32, p1, from, sum);
    }
    add_rows(a, p1 * 32, hi, from, sum);
  }
  if (col >= a.width) return;
  const int64_t to = (int64_t)key * a.ldt + col;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] *= a.scale;
  if (BY_PLACE) {
    float old[8];
    widen8(load_raw8(a.out, a.table_type, to), a.table_type, old);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] += old[i];
  }
  store8(a.out, a.table_type, to, sum);
}

}  // namespace

// A column slab is a grid's second dimension: the first times 256 stays under 2^32.
hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  embed_kernel<<<dim3(a.rows, (a.width + SLAB - 1) / SLAB), NT, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_sort_tokens(const SortArgs& s, hipStream_t st) {
  if (s.rows <= SORT_ALONE) {
    sort_alone_kernel<<<1, 1024, 0, st>>>(s);
    return hipGetLastError();
  }
  const int blocks = (s.units + 3) / 4;
  for (int pass = 0; pass < s.passes; ++pass) {
    sort_count_kernel<<<blocks, NT, 0, st>>>(s, pass);
    sort_scan_kernel<<<1, 1024, 0, st>>>(s);
    sort_move_kernel<<<blocks, NT, 0, st>>>(s, pass);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_embed_backward(const EmbedArgs& a, hipStream_t st) {
  const uint32_t slabs = (a.width + SLAB - 1) / SLAB;
  embed_runs_kernel<<<a.vocab / NT + 1, NT, 0, st>>>(a);
  if (a.sum32) embed_pieces_kernel<32><<<dim3(a.rows / 32, slabs), NT, 0, st>>>(a);
  if (a.sum1024) embed_pieces_kernel<1024><<<dim3(a.rows / 1024, slabs), NT, 0, st>>>(a);
  if (a.accumulate) embed_sum_kernel<true><<<dim3(a.rows, slabs), NT, 0, st>>>(a);
  else embed_sum_kernel<false><<<dim3(a.vocab, slabs), NT, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace svl
