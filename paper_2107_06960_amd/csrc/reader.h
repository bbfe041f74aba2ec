// reader.h -- argument blocks and launchers of the reader's operators
// (reader.cpp checks the calls; norm.hip, linear.hip and cross.hip hold the
// kernels).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/mafat_reader.h"

namespace mafat {

struct NormArgs {
  const void* x;
  const void* res;
  const float* gain;
  void* sum;
  void* y;
  float* y_scale;
  int64_t x_stride, res_stride, sum_stride, y_stride;
  int64_t rows;
  int32_t cols;
  float eps;
};
hipError_t launch_norm(int dtype, int out_dtype, const NormArgs& a, hipStream_t stream);


struct LinearArgs {
  const unsigned char* x;
  const unsigned char* w;
  const float* x_scale;
  const float* w_scale;
  const float* bias;
  void* y;
  // adapters (count 0: none); u = factor * x_scale * (a x) of every row as two
  // bfloat16 parts, [rows][2][rank_pad] with zeros past the rank
  const uint16_t* a;
  const uint16_t* b;
  const float* factor;
  const int32_t* of_row;
  uint16_t* u;
  int64_t x_stride, w_stride, y_stride;
  int64_t rows;
  int32_t in_cols, out_cols;
  int32_t count, rank, rank_pad;
};
hipError_t launch_linear(const LinearArgs& a, hipStream_t stream);

struct CrossArgs {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* q_offsets;
  const int32_t* k_lengths;
  const unsigned char* mask;
  void* y;
  float* lse;
  // several splits of the positions: per split, row and head the sum of the
  // values and, after all of these, largest score (base 2) and sum
  float* part;
  int64_t q_row, q_head, k_frame, k_pos, k_head, v_frame, v_pos, v_head, y_row, y_head, mask_row;
  int32_t frames, rows, positions, q_heads, kv_heads, group, head_dim;
  int32_t mask_by_row;
  int32_t splits;
  int32_t per_frame;   // query rows of a frame, without offsets
  int32_t row_blocks;  // blocks of query rows, of all frames together (at most)
  int32_t first_block;  // of this launch (see for_block_parts)
  float scale;         // times log2(e): scores are in base 2
};
// How a call is cut up, from its sizes alone (the workspace depends on it).
struct CrossPlan {
  int splits;  // of the positions, joined afterwards
  int few;     // 1: cross_few_kernel
  int waves;   // of cross_tile_kernel: 32 rows each
};
constexpr int kMaxCrossSplits = 64;  // one per lane of the joining wave
CrossPlan plan_cross(const mafat_cross& c);
// Waves of a block of cross_few_kernel, which share a split's positions: so
// many that their slots take 64 KB of LDS.
constexpr int cross_few_waves(int dtype, int head_dim) {
  const int row = head_dim * (dtype == MAFAT_F32 ? 4 : 2);
  return row <= 256 ? 4 : 2;
}
// A launch has fewer than 2^32 threads along an axis of its grid: more blocks
// than this along the first go in several, f(first block, blocks).  (A multiple
// of 8, so that xcd_remap finds the blocks of a launch on the XCDs it expects.)
constexpr int64_t kCrossLaunchBlocks = int64_t{1} << 22;
template <typename F>
hipError_t for_block_parts(int64_t blocks, F f) {
  for (int64_t at = 0; at < blocks; at += kCrossLaunchBlocks) {
    f(static_cast<int32_t>(at), static_cast<unsigned>(blocks - at < kCrossLaunchBlocks ? blocks - at : kCrossLaunchBlocks));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// Blocks of `tile` rows of all frames together, at most.
int64_t cross_row_blocks(const CrossArgs& a, int tile);
hipError_t launch_cross(int dtype, const CrossArgs& a, const CrossPlan& p, hipStream_t stream);
// Whole 16-byte pieces; in float32 heads up to 128.
hipError_t launch_cross_bf16(const CrossArgs& a, const CrossPlan& p, hipStream_t stream);
hipError_t launch_cross_f32(const CrossArgs& a, const CrossPlan& p, hipStream_t stream);

}  // namespace mafat
