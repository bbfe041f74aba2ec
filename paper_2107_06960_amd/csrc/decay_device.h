// decay_device.h -- device helpers that the kernels of linear attention with
// decays share (decay.hip, decay_bf16.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "device_util.h"
#include "reader.h"

namespace mafat {
namespace {

constexpr double kLog2e = 1.4426950408889634;

// A decay's logarithm in base 2, at most 0 and at least -200 (2^-200 is zero in
// float32); NaN stays.
__device__ __forceinline__ float decay_log2(float log_decay) {
  const float l = log_decay > 0.f ? 0.f : log_decay < -138.f ? -138.6f : log_decay;
  return static_cast<float>(static_cast<double>(l) * kLog2e);
}

// 2^x, its exponent's whole part apart: within float32's rounding for large x too, and
// with what is left of numbers below the least normal one, which large states and
// scores bring back.
template <typename F>
__device__ __forceinline__ float power2(F x) {
  const F whole = __builtin_elementwise_rint(x);
  // (the maximum is for NaN, which no integer has and the exponential keeps)
  const int by = static_cast<int>(__builtin_elementwise_max(whole, static_cast<F>(-1e6)));
  return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(x - whole)), by);
}

// Rows of request i: first and number.
__device__ __forceinline__ void rows_of(const DecayArgs& a, int i, int* first, int* n) {
  if (!a.offsets) {
    *first = i * a.per_request;
    *n = a.per_request;
    return;
  }
  *first = min(max(a.offsets[i], 0), a.rows);
  *n = max(min(max(a.offsets[i + 1], 0), a.rows) - *first, 0);
}

// Slot of request `lane`: asked for ahead of slot_of, beside what else a kernel
// starts with, since loads that wait for each other are what its start takes.
__device__ __forceinline__ int slots_ahead(const DecayArgs& a) {
  const int lane = static_cast<int>(threadIdx.x) & 63;
  return a.states && a.slots && lane < a.requests ? a.slots[lane] : -1;
}
// The state of a request's slot: NONE: starts from zeros and is not kept;
// TAKEN: an earlier request with rows has it.  The same in all lanes.
enum { SLOT_NONE = -1, SLOT_TAKEN = -2 };
__device__ __forceinline__ int64_t slot_of(const DecayArgs& a, int request, int ahead) {
  if (!a.states) return SLOT_NONE;
  int s = request;
  if (a.slots) s = request < 64 ? __builtin_amdgcn_readlane(ahead, request) : a.slots[request];
  if (s < 0 || s >= a.pool) return SLOT_NONE;
  if (a.slots) {
    // The requests before it, the first 64 of them from `ahead`, then 512 at a time.
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const auto has = [&](int e, int slot) {
      if (e >= request || slot != s) return false;
      int first, n;
      rows_of(a, e, &first, &n);
      return n > 0;
    };
    if (__builtin_amdgcn_ballot_w64(has(lane, ahead))) return SLOT_TAKEN;
    for (int e0 = 64; e0 < request; e0 += 512) {
      int slot[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) slot[i] = e0 + 64 * i + lane < request ? a.slots[e0 + 64 * i + lane] : -1;
      bool same = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) same |= has(e0 + 64 * i + lane, slot[i]);
      if (__builtin_amdgcn_ballot_w64(same)) return SLOT_TAKEN;
    }
  }
  return s;
}

// The segments of a request of n rows, and their length: as few as a segment's
// largest length allows, as even as whole chunks of 32 tokens go.
__device__ __forceinline__ int segments_of(const DecayArgs& a, int n, int* length) {
  const uint32_t rows = static_cast<uint32_t>(n), most = static_cast<uint32_t>(a.segment);
  if (rows <= most) {
    *length = a.segment;
    return rows > 0 ? 1 : 0;
  }
  const uint32_t count = (rows + most - 1) / most;
  const uint32_t len = ((rows + count - 1) / count + 31) & ~31u;
  *length = static_cast<int>(len);
  return static_cast<int>((rows + len - 1) / len);
}

// A block's work: a segment of a request.
struct Segment {
  int request, first, n;  // rows of the segment
  int index, count;       // of the request's segments
  bool any;
};

// Segment b of all requests together.  With offsets each wave scans the
// requests, 64 at a time.
__device__ __forceinline__ Segment find_segment(const DecayArgs& a, int b) {
  Segment s;
  s.any = true;
  int start, rows, length;
  if (!a.offsets) {
    rows = a.per_request;
    s.count = segments_of(a, rows, &length);
    s.request = static_cast<int>(static_cast<uint32_t>(b) / static_cast<uint32_t>(s.count));
    s.index = b - s.request * s.count;
    start = s.request * rows;
    s.any = s.request < a.requests;
  } else {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    uint32_t before = 0;
    s.any = false;
    s.request = s.index = s.count = start = rows = length = 0;
    for (int r0 = 0; r0 < a.requests; r0 += 64) {
      const int r = r0 + lane;
      int lo = 0, n = 0, len;
      if (r < a.requests) rows_of(a, r, &lo, &n);
      const uint32_t blocks = static_cast<uint32_t>(segments_of(a, n, &len));
      // (offsets that decrease may make the sums wrap: b then matches some request or none)
      uint32_t upto = blocks;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t left = static_cast<uint32_t>(__shfl_up(static_cast<int>(upto), o, 64));
        upto += lane >= o ? left : 0;
      }
      const uint32_t from = before + upto - blocks, mine = static_cast<uint32_t>(b) - from;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(mine < blocks);
      if (hit) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        s.request = r0 + l;
        start = __builtin_amdgcn_readlane(lo, l);
        rows = __builtin_amdgcn_readlane(n, l);
        length = __builtin_amdgcn_readlane(len, l);
        s.index = __builtin_amdgcn_readlane(static_cast<int>(mine), l);
        s.count = __builtin_amdgcn_readlane(static_cast<int>(blocks), l);
        s.any = true;
        break;
      }
      before += static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(upto), 63));
    }
  }
  s.first = start + s.index * length;
  s.n = min(length, rows - s.index * length);
  return s;
}

// n of the 4 values at p as floats (the rest are zero).
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p, int n) {
  T t[4];
  if (n >= 4) {
    __builtin_memcpy(t, p, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = i < n ? p[i] : static_cast<T>(0);
  }
  return f32x4{to_f(t[0]), to_f(t[1]), to_f(t[2]), to_f(t[3])};
}
template <typename T>
__device__ __forceinline__ void put4(T* p, int n, f32x4 v) {
  if (n >= 4) {
    T t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) store1(&t[i], v[i]);
    __builtin_memcpy(p, t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) store1(p + i, v[i]);
  }
}

}  // namespace
}  // namespace mafat
