// Kernel arguments of the windowed attention operators and of the 4-bit K / V
// cache, and the geometry they share with the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace svl {

// ---------------------------------------------------------------- 4-bit cache
// One tile holds 16 positions of one K/V head: the K codes, the V codes, and
// the (scale, minimum) pairs of K and of V (layout: include/svl.h).
constexpr int KV4_TILE = 16;
constexpr int KV4_GROUP = 64;   // dims that share a pair
constexpr int64_t kv4_tile_bytes(int d) {
  return 2 * (int64_t)KV4_TILE * d / 2 + 2 * (int64_t)KV4_TILE * (d / KV4_GROUP) * 4;
}

// Segments travel in the kernel arguments (no copy to the device, so a
// captured launch keeps them); longer batches are several launches.
constexpr int SEGS_PER_LAUNCH = 64;

// One sample's rows of a launch: rows row0 .. row0 + rows - 1 are its positions
// pos0 .. pos0 + rows - 1.
struct CacheSeg {
  int32_t row0, rows, pos0, sample;
  int32_t kv_off, kv_cnt;   // K/V heads kv_table[kv_off .. kv_off + kv_cnt)
  int32_t item0;            // first work item of the segment
  int32_t nsplit;           // attention: pieces of its key range
  int32_t part0;            // attention: first partial block (nsplit > 1)
  int32_t join0;            // attention: blocks of earlier cut segments (the join's grid)
};

struct Kv4Args {
  CacheSeg seg[SEGS_PER_LAUNCH];
  int32_t nsegs, nitems;
  const int32_t* kv_table;  // nullptr: slot i is K/V head i
  int32_t n_kv_heads, rep;  // query heads per K/V head
  const void* k;            // append: 16-bit rows [row][K/V head][d], row stride ldk
  const void* v;
  void* k_out;              // read: the same
  void* v_out;
  int64_t ldk, ldv;
  uint8_t* cache;
  int64_t tiles;            // tiles of one head
  const void* q;            // attention: [row][head][d], row stride ldq
  void* out;                // row stride ldo
  int64_t ldq, ldo;
  float scale;
  int32_t window, sinks;
  float* partial;           // partial blocks (nsplit > 1)
};

// Columns (query row, head of the group) of an attention work item.
constexpr int KV4_COLS = 16;
constexpr int KV4_UNIT = 2 * KV4_TILE;     // positions that a wave takes at a time
// A launch is cut into about this many work items (256 CUs, two workgroups
// each), and a piece has this many units at least (two per wave).  With 1024 items
// sixteen samples in a window of 2048, 32 heads on 8, take 21 us in place of 17 and
// eight of 8192 positions 63 in place of 59; eight ragged ones up to 20001, 28 heads
// on 4, 15 in place of 17.  Pieces of 4 units are no faster.
constexpr int KV4_TARGET_ITEMS = 512, KV4_MIN_UNITS = 8;
constexpr int KV4_MAX_PIECES = KV4_TARGET_ITEMS + 1;   // of one block
// Floats of a partial block: per column the maximum, the sum and d outputs.
constexpr int64_t kv4_partial_floats(int d) { return (int64_t)KV4_COLS * (d + 2); }

hipError_t launch_kv4_append(const Kv4Args& a, int32_t head_dim, bool f16, hipStream_t st);
hipError_t launch_kv4_read(const Kv4Args& a, int32_t head_dim, bool f16, hipStream_t st);
hipError_t launch_kv4_attention(const Kv4Args& a, int32_t head_dim, bool f16, hipStream_t st);
// Joins the pieces of the segments with nsplit > 1: `blocks` of them, of up to
// `columns` columns each.
hipError_t launch_kv4_join(const Kv4Args& a, int32_t head_dim, bool f16, int32_t blocks,
                           int32_t columns, hipStream_t st);

// Positions are below 2^30: a wider window hides nothing, and the kernels' sums of a
// position and the window stay in 32 bits.
constexpr int32_t window_of(int32_t window) { return window < 1 << 30 ? window : 1 << 30; }

// ---------------------------------------------------------------- packed rows
// One sample: queries at rows q0 .. q0 + nq - 1, keys at rows k0 .. k0 + nk - 1;
// query i is at position nk - nq + i.
struct WinSeg {
  int32_t q0, nq, k0, nk;
  int32_t h_off, h_cnt;     // query heads head_table[h_off .. h_off + h_cnt)
  int32_t item0;            // first workgroup of the segment
  int32_t pad;
};

struct WinArgs {
  WinSeg seg[SEGS_PER_LAUNCH];
  int32_t nsegs, nitems;
  const int32_t* head_table;   // nullptr: slot i is head i
  int32_t n_heads, n_kv_heads;
  const void* q;               // [row][head][d], row strides ldq, ldk, ldv, ldo
  const void* k;
  const void* v;
  void* out;
  int64_t ldq, ldk, ldv, ldo;
  float* lse;                  // [query row][n_heads] or nullptr
  const uint8_t* key_mask;     // [key row] or nullptr
  float scale;
  int32_t window, sinks;
  int32_t packed;              // 1: out in the packed layout of the projections (K = ldo)
};

constexpr int WIN_BK = 64;     // keys of a tile

// bq: query rows of a workgroup, 128 or 64
hipError_t launch_window_attention(const WinArgs& a, int32_t head_dim, bool f16, int32_t bq,
                                   hipStream_t st);

// Backward.  The key / value gradient's work: key tiles of WIN_DK keys of a K/V
// head, each cut into pieces of its (query head, tile of WIN_DQ query rows)
// list; the first nst tiles (those with sink positions, seen by every later
// row) into ps pieces, the others into po.
constexpr int WIN_DK = 128, WIN_DQ = 64;
struct WinBwdSeg {
  int32_t q0, nq, k0, nk;
  int32_t nst, ps, po;
  int32_t item0;            // first workgroup of the segment
  int32_t part0, part1;     // first partial block of the cut sink tiles, of the other cut tiles
};

struct WinBwdArgs {
  WinBwdSeg seg[SEGS_PER_LAUNCH];
  int32_t nsegs, nitems;
  int32_t n_heads, n_kv_heads;
  const void* q;            // 16-bit rows [row][head][d] with their row strides
  const void* k;
  const void* v;
  const void* out;
  const void* grad;         // of out
  void* dq;
  void* dk;
  void* dv;
  int64_t ldq, ldk, ldv, ldo, ldg, lddq, lddk, lddv;
  const float* lse;         // [query row][n_heads]
  const uint8_t* key_mask;
  float* delta;             // [query row][n_heads]: rowsum(grad * out)
  int32_t* expo;            // [query row][n_heads]: exponent of the row's largest gradient (fp16)
  float* partial;           // blocks of [2][WIN_DK][d]
  float scale;
  int32_t window, sinks;
};
// One launch each; dq first (it writes delta and expo).
hipError_t launch_window_dq(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st);
hipError_t launch_window_dkv(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st);
hipError_t launch_window_dkv_join(const WinBwdArgs& a, int32_t head_dim, bool f16, hipStream_t st);

// ---------------------------------------------------------------- host side
// Cuts the segments that get(ctx, 0 .. n - 1) gives (their rows, positions and
// heads; empty ones are passed over) into work items and launches them, up to
// SEGS_PER_LAUNCH at a time.  `a` holds everything but the segments.
typedef CacheSeg (*CacheSegOf)(const void* ctx, int32_t i);
typedef WinSeg (*WinSegOf)(const void* ctx, int32_t i);
hipError_t kv4_append_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n, int32_t head_dim,
                               bool f16, hipStream_t st);
hipError_t kv4_read_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n, int32_t head_dim,
                             bool f16, hipStream_t st);
hipError_t kv4_attention_segments(Kv4Args& a, CacheSegOf get, const void* ctx, int32_t n,
                                  int32_t head_dim, bool f16, hipStream_t st);
hipError_t window_segments(WinArgs& a, WinSegOf get, const void* ctx, int32_t n, int32_t head_dim,
                           bool f16, hipStream_t st);
// Bytes of the partial blocks that kv4_attention_segments may need.
size_t kv4_partial_bytes(int32_t head_dim);

}  // namespace svl
