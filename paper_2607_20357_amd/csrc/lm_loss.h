// Kernel arguments and geometry of the language-model loss (lm_loss.hip,
// lm_gemm.hip), shared with the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace svl {

constexpr int32_t LM_TILE = 256;     // rows and columns of a product's tile
constexpr int32_t LM_BK = 64;        // of its sum a step
constexpr int32_t LM_ROWS = 64;      // labelled rows are filled up with zeros to a multiple
constexpr int32_t LM_SLAB = 128;     // vocabulary entries whose exponentials share a maximum
constexpr int32_t LM_FEW = 64;       // rows of a call whose logits a wave's products take straight from memory
constexpr int32_t LM_SHORT = 1024;   // rows up to which the head's gradient comes in tiles of a quarter the size
constexpr int32_t LM_PACK = 1024;    // rows of a call that are packed in one launch
constexpr int32_t LM_PARTS = 256;    // most workgroups (tiles x pieces) of a product whose sum is cut
constexpr int32_t LM_CUT = 8;        // least steps of LM_BK of a piece of a sum
// Exponentials are held as fp16 under 2^14 (normal down to 2^-28 of their slab's largest), P
// in fp16 likewise (of the largest weight).
constexpr float LM_E_SCALE = 16384.f;

// What is known of a call's rows only on the device.
struct LmHead {
  int32_t rows;        // rows with a label
  float weight;        // their largest |weight|
};

struct LmArgs {
  LmHead* head;
  int32_t rows, d, vocab;       // of the call
  int32_t vp;                   // vocabulary rounded up to tiles: the stride of e and stats' slabs
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
  float* log_sum;               // [chunk]
  float2* stats;                // [chunk][vp / LM_SLAB] (maximum, sum of exponentials)
  uint16_t* e;                  // [chunk][vp] exponentials, then P; or nullptr
  float* parts;                 // [LM_PARTS] tiles of a cut sum
  float* sum_w;                 // [vocab][d] the head's gradient of earlier passes, or nullptr
  bool first, last;             // pass of the call
};

enum LmProduct : int32_t { LM_LOGITS = 0, LM_GRAD_X = 1, LM_GRAD_W = 2 };

// Pieces of a product's sum of nk steps over `tiles` tiles.
__host__ __device__ inline int32_t lm_pieces(int32_t tiles, int32_t nk) {
  if (tiles <= 0 || tiles > LM_PARTS / 2) return 1;
  const int32_t s = LM_PARTS / tiles, most = nk / LM_CUT;
  return s < most ? s : (most > 1 ? most : 1);
}

hipError_t launch_lm_rows(const LmArgs& a, hipStream_t st);                 // labelled rows, packed
hipError_t launch_lm_stats(const LmArgs& a, hipStream_t st);                // log-sums and losses
hipError_t launch_lm_softmax(const LmArgs& a, bool f16, hipStream_t st);    // exponentials to P
hipError_t launch_lm_product(const LmArgs& a, LmProduct p, bool f16, hipStream_t st);
hipError_t launch_lm_few_logits(const LmArgs& a, bool f16, hipStream_t st); // logits of at most LM_FEW rows
hipError_t launch_lm_zero_w(const LmArgs& a, hipStream_t st);               // a call without rows

}  // namespace svl
