// norm.hip -- residual addition and root-mean-square norm, into float32,
// bfloat16 or 8 bits with a scale per row.
//
//   h = round(x + residual),  y = h * (mean(h^2) + eps)^(-1/2) * gain
//
// Bound by memory: x and the residual are read once and the sum and y written
// once, so a row stays in the registers of the threads that share it (a
// "team": part of a wave, a wave, or several waves), between the sum of
// squares, the maximum that fixes the 8-bit scale, and the store.  Only rows
// too long for that are read again (norm_long_kernel).  16384 rows of 4096
// bfloat16 values into 8 bits: 95 us, 4.9 TB/s, where a copy reaches 5.05.
//
// A row is cut into pieces of 16 bytes of its input type.  Rows need not be
// aligned: the pieces are read and written with unaligned vector accesses,
// and the last one, if it is short, value by value.
#include <hip/hip_runtime.h>

#include "norm_device.h"
#include "reader.h"

namespace mafat {
namespace {

// One row per team, NP pieces per thread at most.
template <int DT, int OUT, bool RES, int TEAM, int NP>
__global__ __launch_bounds__(TEAM > 256 ? TEAM : 256) void norm_kernel(const NormArgs a) {
  using T = typename Elt<DT>::T;
  constexpr int V = Piece<DT>::V;
  constexpr int TEAMS = TEAM >= 256 ? 1 : 256 / TEAM;
  __shared__ float lds_sum[TEAM > 64 ? TEAM / 64 : 1];
  __shared__ uint32_t lds_max[TEAM > 64 ? TEAM / 64 : 1];
  static_assert(TEAM <= 64 || TEAM >= 256, "a team is part of a wave, or the block");
  const int t = static_cast<int>(threadIdx.x) % TEAM;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * TEAMS + static_cast<int>(threadIdx.x) / TEAM;
  if (row >= a.rows) return;  // whole teams; a team of several waves is the block
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* res = RES ? static_cast<const T*>(a.res) + row * a.res_stride : nullptr;

  float h[NP][V];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = (k * TEAM + t) * V;
    load_piece<DT>(x + c, a.cols - c, h[k]);
  }
  if constexpr (RES) {
    float r[NP][V];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int c = (k * TEAM + t) * V;
      load_piece<DT>(res + c, a.cols - c, r[k]);
    }
    T* sum = static_cast<T*>(a.sum) + row * a.sum_stride;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int c = (k * TEAM + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] += r[k][i];
      if constexpr (DT == MAFAT_BF16) {  // the norm is that of the stored sum
#pragma unroll
        for (int i = 0; i < V; ++i) h[k][i] = static_cast<float>(static_cast<__bf16>(h[k][i]));
      }
      store_piece<DT>(sum + c, a.cols - c, h[k]);
    }
  }
  float sq = 0.f;
#pragma unroll
  for (int k = 0; k < NP; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) sq = fmaf(h[k][i], h[k][i], sq);
  sq = team_reduce<TEAM>(sq, Add{}, lds_sum);
  const float inv = 1.f / sqrtf(sq / static_cast<float>(a.cols) + a.eps);
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = (k * TEAM + t) * V;
    if (a.gain) {
      float g[4 * ((V + 3) / 4)];
      if (a.cols - c >= V) {
        __builtin_memcpy(g, a.gain + c, 4 * V);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = c + i < a.cols ? a.gain[c + i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= inv * g[i];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= inv;
    }
    if constexpr (OUT == MAFAT_F8) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < a.cols) most = MaxBits{}(most, __float_as_uint(h[k][i]) & 0x7fffffffu);
    }
  }
  using Y = typename OutElt<OUT>::T;
  Y* y = static_cast<Y*>(a.y) + row * a.y_stride;
  if constexpr (OUT == MAFAT_F8) {
    most = team_reduce<TEAM>(most, MaxBits{}, lds_max);
    float by;
    const float scale = row_scale(most, &by);
    if (t == 0) a.y_scale[row] = scale;
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= by;
  }
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = (k * TEAM + t) * V;
    store_piece<OUT>(y + c, a.cols - c, h[k]);
  }
}

// Rows of any length: a block of 1024 threads reads its row again for the
// maximum and for the outputs (from the caches, mostly).
template <int DT, int OUT, bool RES>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormArgs a) {
  using T = typename Elt<DT>::T;
  using Y = typename OutElt<OUT>::T;
  constexpr int V = Piece<DT>::V;
  constexpr int TEAM = 1024;
  __shared__ float lds_sum[TEAM / 64];
  __shared__ uint32_t lds_max[TEAM / 64];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* res = RES ? static_cast<const T*>(a.res) + row * a.res_stride : nullptr;
  T* sum = RES ? static_cast<T*>(a.sum) + row * a.sum_stride : nullptr;
  const T* again = RES ? sum : x;  // a thread reads back what it wrote itself
  Y* y = static_cast<Y*>(a.y) + row * a.y_stride;
  float h[V], sq = 0.f;
  for (int64_t c = static_cast<int64_t>(threadIdx.x) * V; c < a.cols; c += TEAM * V) {
    const int n = static_cast<int>(a.cols - c);
    load_piece<DT>(x + c, n, h);
    if constexpr (RES) {
      float r[V];
      load_piece<DT>(res + c, n, r);
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] += r[i];
      if constexpr (DT == MAFAT_BF16) {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = static_cast<float>(static_cast<__bf16>(h[i]));
      }
      store_piece<DT>(sum + c, n, h);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sq = fmaf(h[i], h[i], sq);
  }
  sq = team_reduce<TEAM>(sq, Add{}, lds_sum);
  const float inv = 1.f / sqrtf(sq / static_cast<float>(a.cols) + a.eps);
  auto normed = [&](int64_t c, int n) {
    load_piece<DT>(again + c, n, h);
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] *= a.gain ? inv * (i < n ? a.gain[c + i] : 0.f) : inv;
  };
  float by = 1.f;
  if constexpr (OUT == MAFAT_F8) {
    uint32_t most = 0;
    for (int64_t c = static_cast<int64_t>(threadIdx.x) * V; c < a.cols; c += TEAM * V) {
      const int n = static_cast<int>(a.cols - c);
      normed(c, n);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i < n) most = MaxBits{}(most, __float_as_uint(h[i]) & 0x7fffffffu);
    }
    most = team_reduce<TEAM>(most, MaxBits{}, lds_max);
    const float scale = row_scale(most, &by);
    if (threadIdx.x == 0) a.y_scale[row] = scale;
  }
  for (int64_t c = static_cast<int64_t>(threadIdx.x) * V; c < a.cols; c += TEAM * V) {
    const int n = static_cast<int>(a.cols - c);
    normed(c, n);
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] *= by;
    store_piece<OUT>(y + c, n, h);
  }
}

// A launch has fewer than 2^32 threads: where a row per block would pass
// that, `most` rows after another go in a launch of their own.
template <int DT, int OUT, typename F>
hipError_t by_rows(const NormArgs& a, int64_t most, F launch_rows) {
  using T = typename Elt<DT>::T;
  using Y = typename OutElt<OUT>::T;
  for (int64_t at = 0; at < a.rows; at += most) {
    NormArgs p = a;
    p.rows = a.rows - at < most ? a.rows - at : most;
    p.x = static_cast<const T*>(a.x) + at * a.x_stride;
    if (a.res) {
      p.res = static_cast<const T*>(a.res) + at * a.res_stride;
      p.sum = static_cast<T*>(a.sum) + at * a.sum_stride;
    }
    p.y = static_cast<Y*>(a.y) + at * a.y_stride;
    if (a.y_scale) p.y_scale = a.y_scale + at;
    launch_rows(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int DT, int OUT, bool RES>
hipError_t launch(const NormArgs& a, hipStream_t stream) {
  constexpr int V = Piece<DT>::V;
  constexpr int64_t kThreads = int64_t{1} << 31;  // of a launch, at most
  const int64_t pieces = (static_cast<int64_t>(a.cols) + V - 1) / V;
#define MAFAT_NORM(team_, np_)                                                                               \
  do {                                                                                                       \
    constexpr int teams = (team_) >= 256 ? 1 : 256 / (team_), block = (team_) > 256 ? (team_) : 256;         \
    return by_rows<DT, OUT>(a, teams * (kThreads / block), [&](const NormArgs& p) {                          \
      hipLaunchKernelGGL((norm_kernel<DT, OUT, RES, team_, np_>),                                            \
                         dim3(static_cast<unsigned>((p.rows + teams - 1) / teams)), dim3(block), 0, stream, p); \
    });                                                                                                      \
  } while (0)
  if (pieces <= 16) MAFAT_NORM(16, 1);
  if (pieces <= 64) MAFAT_NORM(64, 1);
  if (pieces <= 128) MAFAT_NORM(64, 2);
  if (pieces <= 256) MAFAT_NORM(256, 1);
  if (pieces <= 512) MAFAT_NORM(256, 2);
  if (pieces <= 1024) MAFAT_NORM(256, 4);
  if (pieces <= 2048) MAFAT_NORM(1024, 2);
  if (pieces <= 4096) MAFAT_NORM(1024, 4);
#undef MAFAT_NORM
  return by_rows<DT, OUT>(a, kThreads / 1024, [&](const NormArgs& p) {
    hipLaunchKernelGGL((norm_long_kernel<DT, OUT, RES>), dim3(static_cast<unsigned>(p.rows)), dim3(1024), 0, stream, p);
  });
}

template <int DT, int OUT>
hipError_t launch_out(const NormArgs& a, hipStream_t stream) {
  return a.res ? launch<DT, OUT, true>(a, stream) : launch<DT, OUT, false>(a, stream);
}

template <int DT>
hipError_t launch_in(int out_dtype, const NormArgs& a, hipStream_t stream) {
  switch (out_dtype) {
    case MAFAT_F32: return launch_out<DT, MAFAT_F32>(a, stream);
    case MAFAT_BF16: return launch_out<DT, MAFAT_BF16>(a, stream);
    default: return launch_out<DT, MAFAT_F8>(a, stream);
  }
}

}  // namespace

hipError_t launch_norm(int dtype, int out_dtype, const NormArgs& a, hipStream_t stream) {
  return dtype == MAFAT_BF16 ? launch_in<MAFAT_BF16>(out_dtype, a, stream) : launch_in<MAFAT_F32>(out_dtype, a, stream);
}

}  // namespace mafat
