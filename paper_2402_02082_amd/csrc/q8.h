// The 8-bit key/value cache: its layout, and the interface of its kernels
// (q8_cache.hip, q8_attn.hip) and of the rotary positions (rope.hip) to the
// C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "attn.h"

namespace glide {

// Tokens of a block: whole blocks are held in 8 bits, K and V of a block and
// head with one scale each.  The tokens behind the last whole block, and the
// tree rows behind those, are bfloat16 rows of a ring: token j at row
// j % kQ8Tail.  A ring holds up to 31 accepted tokens and 64 tree rows.
constexpr int kQ8Block = 32;
constexpr int kQ8Tail = 128;
constexpr int kQ8PartBytes = kQ8Block * kHeadDim;    // K or V of a block
constexpr int kQ8BlockBytes = 2 * kQ8PartBytes;
constexpr int kQ8TailElems = 2 * kQ8Tail * kHeadDim;  // K and V ring of a head
constexpr int kQ8MaxBlocks = (1 << 22) / kQ8Block;

// Byte order of a block: the operands of v_mfma_f32_16x16x32, so that every
// load of the attention kernel is 1 KB in a row, one 16-byte unit a lane
// (lane 16 g + c).
//   K: load (kt, h): unit of lane (c, g) = token 16 kt + c, dims 64 h + 16 g + (0..15)
//   V: load u: unit of lane (c, g) = dims 8 c + 2 u + t (t = 0, 1), for each
//      the tokens 16 j + 4 g + i (j = 0, 1; i = 0..3) in bytes 8 t + 4 j + i
// (V is held transposed: the PV product takes eight tokens of a dim a lane.)
__host__ __device__ constexpr int q8_k_byte(int token, int dim) {
  return ((token >> 4) * 2 + (dim >> 6)) * 1024 + (((dim >> 4) & 3) * 16 + (token & 15)) * 16 + (dim & 15);
}
__host__ __device__ constexpr int q8_v_byte(int token, int dim) {
  return ((dim >> 1) & 3) * 1024 + (((token >> 2) & 3) * 16 + (dim >> 3)) * 16 + (dim & 1) * 8 + (token >> 4) * 4 +
         (token & 3);
}

struct Q8Cache {
  uint8_t* blocks;  // [B, H, n_blocks, kQ8BlockBytes]
  float* scales;    // [B, H, n_blocks, 2]: of K, of V
  uint16_t* tail;   // [B, H, 2, kQ8Tail, kHeadDim] bf16
};

// Rows written to a cache.  `hold`: to the ring alone (tree rows); else
// blocks that become whole are quantised.
struct Q8AppendArgs {
  const uint16_t* k;  // row (b, t, h) at b * sb + t * st + h * sh elements
  const uint16_t* v;
  Q8Cache cache;
  const int32_t* seq_lens;
  const int32_t* counts;  // nullable: T rows of every sequence
  int64_t sb, st, sh;
  int B, T, H, n_blocks;
};
hipError_t launch_q8_append(const Q8AppendArgs& a, bool int8, bool hold, hipStream_t stream);

struct Q8ReadArgs {
  Q8Cache cache;
  const int32_t* seq_lens;
  void* k_out;  // [B, H, T, D]: tokens start .. start + T - 1
  void* v_out;
  int B, H, n_blocks, start, T;
};
hipError_t launch_q8_read(const Q8ReadArgs& a, bool int8, bool out_bf16, hipStream_t stream);

constexpr int kQ8MaxLayers = 128;
struct Q8CommitArgs {
  const int32_t* seq_lens;
  const int32_t* accept_len;
  const int32_t* path;  // nullable: a chain, node d at depth d + 1
  int32_t* seq_lens_out;
  int B, H, N, n_blocks, layers;
  Q8Cache cache[kQ8MaxLayers];
};
hipError_t launch_q8_commit(const Q8CommitArgs& a, bool int8, hipStream_t stream);

// How the attention over an 8-bit cache is divided: workgroups of `waves` waves
// for `rows` query rows, `groups` of them over the rows of a cached head, and its
// keys in runs of units -- `splits` of every pair (sequence, cached head), or
// with splits == 0 up to `target` (half of it if they would be shorter than
// long_run units then) of about equal size in all, of at least min_units units
// each, pairs of up to whole_units in one, and no more runs of a pair than the root
// of its units times join_ratio.  runs: at most so many.
struct Q8AttnPlan {
  int rows, groups, waves, splits, target, min_units, whole_units, long_run;
  float join_ratio;
  long runs;
  size_t ws_bytes, part_ml_off, part_o_off;
};
Q8AttnPlan plan_q8_attn(int B, int N, int H, int H_kv, int n_blocks, int max_splits);

struct Q8AttnArgs {
  const uint16_t* q;
  Q8Cache cache;
  const int32_t* seq_lens;
  const int32_t* parents;  // nullptr: cross mode
  uint16_t* out;
  unsigned* counters;  // arrival counters of pairs that lie in several runs
  float* part_o;    // [runs, groups, rows, D]: normalised outputs
  float2* part_ml;  // [runs, groups, rows]: (max in log2 units, sum)
  int B, N, H, H_kv, G, n_blocks, groups, splits,  // G: query heads a cached one
      target, min_units, whole_units, long_run, runs;
  float join_ratio, scale_log2;
};
hipError_t launch_q8_attn(const Q8AttnArgs& a, bool int8, int rows, int waves, hipStream_t stream);

// Rotary positions of queries and keys.
struct RopeRows {
  const void* in;
  void* out;
  int64_t in_sb, in_st, in_sh, out_sb, out_st, out_sh;  // strides in elements
  int H;
};
struct RopeArgs {
  RopeRows q, k;          // k.H == 0: none
  const double* freqs;    // [rot / 2] angle per position
  const int32_t* positions;  // [B, T] or nullptr
  const int32_t* seq_lens;   // [B] or nullptr: first position (0)
  const int32_t* parents;    // [B, T] or nullptr: depth in the tree instead of t
  int B, T, rot;
  float mscale;
};
hipError_t launch_rope(const RopeArgs& a, bool bf16, bool interleaved, bool backward, hipStream_t stream);

}  // namespace glide
