// Kernel arguments and geometry of the language-model loss (lm_loss.hip,
// lm_gemm.hip), shared with the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace svl {

constexpr int32_t LM_TILE = 256;     // rows and columns of a product's tile
constexpr int32_t LM_BK = 64;        // of its sum a step
constexpr int32_t LM_ROWS = 64;      // labelled rows are filled up with zeros to a multiple
constexpr int32_t LM_SLAB = 128;     // vocabulary entries whose exponentials share a maximum, in whole tiles
// Rows up to which the head's gradient comes in tiles of a quarter the size (with the softmax before it, 4096,
// 32000: 320 rows 155 us against 169, 640 217 against 227, 1024 308 against 307), also where the sums of whole
// tiles would be cut (300 rows, 256, 3000: 7 us against 20).
constexpr int32_t LM_SHORT = 768;
// The logits come in tiles of a quarter the size, of which a CU holds two, where the call has at most
// LM_FEW rows (one such tile across: w is what there is to read, once, and twice the loads are on their way;
// vocabulary 65537, 1024, 128 rows: 47 us the call, of whole tiles 65; 151936, 5120, 8 rows: 321 against 368) and
// where whole tiles are at most LM_SMALL, half the CUs (32000, 4096: 24 rows 58 us against 89, 256 80 against
// 83; twice the tiles, 512 rows, 135 against 107).
constexpr int32_t LM_FEW = 128, LM_SMALL = 128;
constexpr int32_t LM_PACK = 1024;    // rows of a call that are packed in one launch
constexpr int32_t LM_CUS = 256;      // tiles at work at once
constexpr int32_t LM_CUT = 4;        // least steps of LM_BK of a piece of a sum (40 rows, 1024, 20000:
                                     // grad_x and its join 29 us, of 8 steps 44)
// Exponentials are held as fp16 under 2^14 (normal down to 2^-28 of their slab's largest), P
// in fp16 likewise, P over the largest weight of the call.  A row's part of it is 1 where weights are equal: the
// label's entry, most of a gradient's size, is then p - 1, just under 1, where a rounding is least of the value
// (times a weight over a power of two in its place, just over 1: gradients of 284 rows off by 38e-5 of themselves, not
// 23e-5).  fp16's range does not hold rows of small weight beside large ones, so for the rows' gradient the part's
// power of two (lm_power) is left out of P and multiplied in by the row; for the head's, whose sum runs over
// rows, it is in P.  (bf16 has float32's range: P over the largest weight for both.)
constexpr float LM_E_SCALE = 16384.f;

// A row's part of the largest weight, and the power of two at or below its size, at least 2^-126: the part over it is
// exact, and less than 2.
__device__ __forceinline__ float lm_part(float weight, float most) { return most == 0.f ? 0.f : weight / most; }
__device__ __forceinline__ float lm_power(float part) {
  const uint32_t e = __float_as_uint(part) & 0x7f800000u;
  return __uint_as_float(e ? e : 0x00800000u);
}

// What is known of a call's rows only on the device.
struct LmHead {
  int32_t rows;        // rows with a label
  float weight;        // their largest |weight|
};

struct LmArgs {
  LmHead* head;
  int32_t rows, d, vocab;       // of the call
  int32_t vp;                   // vocabulary rounded up to tiles: the stride of e and stats' slabs
  int32_t slab;                 // 128, or 64 in small tiles
  int32_t chunk0, chunk;        // labelled rows chunk0 .. + chunk of this pass
  const uint16_t* x;            // the call's rows
  int64_t ldx;
  const uint16_t* w;
  int64_t ldw;
  const int32_t* labels;
  const float* row_weight;      // or nullptr
  float* loss;
  float* lse;                   // or nullptr
  uint16_t* grad_x;             // or nullptr
  int64_t ldgx;
  uint16_t* grad_w;             // or nullptr
  int64_t ldgw;
  bool accumulate;
  // workspace; by labelled row in ascending order
  int32_t* row_of;              // [rows] the row it is
  int32_t* label;               // [rows]
  float* weight;                // [rows]
  uint16_t* xc;                 // [rows to a multiple of LM_ROWS][d]
  float* label_logit;           // [chunk]
  float2* total;                // [chunk] the row's largest logit, 1 / (sum of exponentials under it)
  float2* stats;                // [chunk][vp / slab] (maximum, sum of exponentials)
  uint16_t* e;                  // [chunk][vp] exponentials, then P; or nullptr
  float* parts;                 // tiles of a cut sum's pieces
  float* sum_w;                 // [vocab][d] the head's gradient of earlier passes, or nullptr
  bool first, last;             // pass of the call
};

enum LmProduct : int32_t { LM_LOGITS = 0, LM_GRAD_X = 1, LM_GRAD_W = 2 };

// Pieces of a product's sum of nk steps over `tiles` tiles: as many as fill the rounds of the CUs,
// up to three, where that shortens them by a tenth at least (a piece more is its tile written and read once in
// float32).  (grad_x of 500 steps, with the softmax before it: 144 tiles in three pieces 567 us,
// whole 686; 160 615 against 714.)
__host__ __device__ inline int32_t lm_pieces(int32_t tiles, int32_t nk) {
  if (tiles <= 0 || tiles > 2 * LM_CUS) return 1;
  const int32_t most = nk / LM_CUT;
  int32_t best = 1, rounds = (tiles + LM_CUS - 1) / LM_CUS;     // time: rounds / best
  for (int32_t r = 1; r <= 3; ++r) {
    int32_t s = r * LM_CUS / tiles;
    s = s < most ? s : most;
    if (s > best && 10 * r * best < 9 * rounds * s) {
      best = s;
      rounds = r;
    }
  }
  return best;
}

hipError_t launch_lm_rows(const LmArgs& a, hipStream_t st);                 // labelled rows, packed
hipError_t launch_lm_stats(const LmArgs& a, hipStream_t st);                // log-sums and losses
hipError_t launch_lm_softmax(const LmArgs& a, bool f16, hipStream_t st);    // exponentials to P
hipError_t launch_lm_weigh(const LmArgs& a, hipStream_t st);                // fp16: P of grad_x to P of grad_w
hipError_t launch_lm_product(const LmArgs& a, LmProduct p, bool f16, hipStream_t st);
// Most pieces of all tiles that a product is cut into, whatever rows have a label (0: it is never cut).
int64_t lm_parts(const LmArgs& a, LmProduct p);
hipError_t launch_lm_zero_w(const LmArgs& a, hipStream_t st);               // a call without rows

}  // namespace svl
