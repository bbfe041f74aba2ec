// norm_device.h -- device helpers of the operators that norm rows (norm.hip,
// block_norm.hip): pieces of 16 bytes of a row, sums and maxima over the
// threads that share one, 8-bit scales.
#pragma once

#include <hip/hip_runtime.h>

#include "device_util.h"
#include "reader.h"

namespace mafat {
namespace {

template <int DT> struct Piece { static constexpr int V = 16 / sizeof(typename Elt<DT>::T); };

// The V values of a piece that starts at p, `n` of which are there (the rest are zero).
template <int DT>
__device__ __forceinline__ void load_piece(const typename Elt<DT>::T* p, int n, float (&v)[Piece<DT>::V]) {
  constexpr int V = Piece<DT>::V;
  typename Elt<DT>::T t[V];
  if (n >= V) {
    __builtin_memcpy(t, p, 16);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = i < n ? p[i] : static_cast<typename Elt<DT>::T>(0);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = to_f(t[i]);
}

template <int OUT> struct OutElt { using T = typename Elt<OUT>::T; };
template <> struct OutElt<MAFAT_F8> { using T = uint8_t; };

// V values of a piece to p, as OUT: bf16 rounds to nearest even, so does the
// hardware's conversion to 8 bits (inputs are at most 448 or NaN here).
template <int OUT, int V>
__device__ __forceinline__ void store_piece(typename OutElt<OUT>::T* p, int n, const float (&v)[V]) {
  typename OutElt<OUT>::T t[V];
  if constexpr (OUT == MAFAT_F8) {
    static_assert(V % 4 == 0, "four values a word");
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[i], v[i + 1], 0, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[i + 2], v[i + 3], w, true);
      __builtin_memcpy(t + i, &w, 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) store1(&t[i], v[i]);
  }
  if (n >= V) {
    __builtin_memcpy(p, t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = t[i];
  }
}

// Over the TEAM threads of a row; all of them get the result.  Teams of more
// than a wave join through LDS (the block is one team then).
template <int TEAM, typename T, typename F>
__device__ __forceinline__ T team_reduce(T v, F join, T* lds) {
#pragma unroll
  for (int o = (TEAM < 64 ? TEAM : 64) / 2; o > 0; o >>= 1) v = join(v, __shfl_xor(v, o, 64));
  if constexpr (TEAM > 64) {
    const int wave = static_cast<int>(threadIdx.x) >> 6;
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < TEAM / 64; ++w) v = join(v, lds[w]);
  }
  return v;
}

// The scale of a row from the bits of its largest magnitude, and what values
// are multiplied by.  (Bits of magnitudes compare like the numbers, a NaN
// above all: a maximum that lets no NaN pass unseen.)  Below 2^-100 the
// reciprocal could overflow and the row is zero in 8 bits whatever its scale
// is up to 1.
__device__ __forceinline__ float row_scale(uint32_t most, float* inverse) {
  const float m = __uint_as_float(most);
  if (m < 0x1p-100f) {
    *inverse = 1.f;
    return 1.f;
  }
  *inverse = 448.f / m;
  return m / 448.f;
}

struct Add {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct MaxBits {
  __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

// 4, 8 or 16 bytes at any address, read or written once: past the caches' usual
// replacement, so that a stream does not push itself out (16384 rows of 40 heads of
// 128 turned and written to others: from 88 to 61 us with both, 62 with the stores).
template <int BYTES> struct Words { typedef unsigned T __attribute__((ext_vector_type(BYTES / 4))); };
template <> struct Words<4> { typedef unsigned T; };
template <typename T, int V>
__device__ __forceinline__ void load_once(const T* p, T (&t)[V]) {
  typedef typename Words<sizeof(T) * V>::T W;
  typedef W __attribute__((aligned(1))) loose;
  const W w = __builtin_nontemporal_load(reinterpret_cast<const loose*>(p));
  __builtin_memcpy(t, &w, sizeof(t));
}
template <typename T, int V>
__device__ __forceinline__ void store_once(T* p, const T (&t)[V]) {
  typedef typename Words<sizeof(T) * V>::T W;
  typedef W __attribute__((aligned(1))) loose;
  W w;
  __builtin_memcpy(&w, t, sizeof(t));
  __builtin_nontemporal_store(w, reinterpret_cast<loose*>(p));
}

}  // namespace
}  // namespace mafat
