// decay_launch.h -- the launches of linear attention with decays that decay.hip
// (any size) and decay_bf16.hip share.
#pragma once

#include "reader.h"

namespace mafat {

// What a launch of the chunked kernels does: what a segment adds to the state,
// or the outputs (and the last state).
enum { DECAY_ADDS = 0, DECAY_OUTPUTS = 1 };

// Whether sizes, strides and addresses are for decay_bf16.hip.
bool decay_bf16_fits(const DecayArgs& a);
hipError_t launch_decay_bf16(int mode, const DecayArgs& a, hipStream_t stream);

// f(arguments, blocks) for the blocks of all segments, heads and slices.
template <typename F>
hipError_t for_decay_blocks(DecayArgs a, F f) {
  const int64_t blocks = static_cast<int64_t>(a.segments) * a.kv_heads * a.slices;
  if (blocks >= (int64_t{1} << 31)) return hipErrorInvalidValue;
  a.blocks = static_cast<int32_t>(blocks);
  return for_block_parts(blocks, [&](int32_t from, unsigned n) {
    a.first_block = from;
    f(a, n);
  });
}

}  // namespace mafat
