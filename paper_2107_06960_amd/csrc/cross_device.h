// cross_device.h -- device helpers that the cross attention kernels share
// (cross.hip, cross_bf16.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "device_util.h"
#include "reader.h"

namespace mafat {
namespace {

enum { MASK_NONE = 0, MASK_KEYS = 1, MASK_ROWS = 2 };

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_t;

constexpr float kNone = -__builtin_huge_valf();

// n of the 16 bytes at p (the rest are zero); p need not be aligned.
template <typename T>
__device__ __forceinline__ u32x4 load16(const T* p, int n) {
  constexpr int V = 16 / sizeof(T);
  u32x4 v = {0, 0, 0, 0};
  if (n >= V) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0) {
    T t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = i < n ? p[i] : static_cast<T>(0);
    __builtin_memcpy(&v, t, 16);
  }
  return v;
}

// Key of a 32-key tile that accumulator register i of a lane of half h holds.
__device__ __forceinline__ int key_of(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// The i-th of n parts of `all` tiles, as even as they go: [first, last).  (One
// 32-bit division: these run ahead of a block's first load.)
__device__ __forceinline__ void part_of(int all, int i, int n, int* first, int* last) {
  const uint32_t per = static_cast<uint32_t>(all) / static_cast<uint32_t>(n);
  const int more = all - static_cast<int>(per) * n;  // the first `more` parts have one more
  *first = static_cast<int>(per) * i + min(i, more);
  *last = *first + static_cast<int>(per) + (i < more ? 1 : 0);
}

// A block's work: a row tile of a frame.
struct Place {
  int frame, row0, tile0, tile_rows, keys;  // first query row, first pair of the tile, pairs of the frame, valid positions
  bool any;
};

// Row block b of all frames together -> frame and row tile.  With offsets each
// wave scans the frames, 64 at a time.
template <int RT>
__device__ __forceinline__ Place find(const CrossArgs& a, int b) {
  Place p;
  p.any = true;
  p.keys = a.positions;
  if (!a.q_offsets) {
    const int per = a.per_frame, blocks = static_cast<int>((static_cast<uint32_t>(per * a.group) + RT - 1) / RT);
    p.frame = static_cast<int>(static_cast<uint32_t>(b) / static_cast<uint32_t>(blocks));
    p.row0 = p.frame * per;
    p.tile0 = (b - p.frame * blocks) * RT;
    p.tile_rows = per * a.group;
    p.any = p.frame < a.frames;
    if (p.any && a.k_lengths) p.keys = min(max(a.k_lengths[p.frame], 0), a.positions);
  } else {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    int before = 0;
    p.any = false;
    for (int f0 = 0; f0 < a.frames; f0 += 64) {
      const int f = f0 + lane;
      int lo = 0, n = 0, keys = a.positions;
      if (f < a.frames) {
        if (a.k_lengths) keys = min(max(a.k_lengths[f], 0), a.positions);
        lo = min(max(a.q_offsets[f], 0), a.rows);
        n = max(min(max(a.q_offsets[f + 1], 0), a.rows) - lo, 0);
      }
      // rows * q_heads < 2^31, and so are the pairs of all frames (if offsets
      // do not decrease; else the sums may wrap, and b matches some frame or none)
      const int pairs = static_cast<int>(static_cast<uint32_t>(n) * static_cast<uint32_t>(a.group));
      const int blocks = pairs > 0 ? (pairs - 1) / RT + 1 : 0;
      int upto = blocks;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int left = __shfl_up(upto, o, 64);
        upto = static_cast<int>(static_cast<uint32_t>(upto) + static_cast<uint32_t>(lane >= o ? left : 0));
      }
      const int from = before + upto - blocks;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(b >= from && b - from < blocks);
      if (hit) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        p.frame = f0 + l;
        p.row0 = __builtin_amdgcn_readlane(lo, l);
        p.keys = __builtin_amdgcn_readlane(keys, l);
        p.tile_rows = __builtin_amdgcn_readlane(pairs, l);
        p.tile0 = (b - __builtin_amdgcn_readlane(from, l)) * RT;
        p.any = true;
        break;
      }
      before = static_cast<int>(static_cast<uint32_t>(before) + static_cast<uint32_t>(__builtin_amdgcn_readlane(upto, 63)));
    }
  }
  return p;
}

// The products for one element type: operand fragments of a 32-wide tile from
// LDS rows and the 32x32 instruction.
//   bf16: 16 of the summed axis per instruction, 8 values a lane
//   f32:  2 per instruction, one value a lane; four of them make a 16-byte piece
template <int DT> struct Tile;
template <> struct Tile<MAFAT_BF16> {
  static constexpr int V = 8;  // values of a 16-byte piece
  static __device__ __forceinline__ void mul(f32x16& c, const u32x4& a, const u32x4& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct Tile<MAFAT_F32> {
  static constexpr int V = 4;
  static __device__ __forceinline__ void mul(f32x16& c, const u32x4& a, const u32x4& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
  }
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

}  // namespace
}  // namespace mafat
