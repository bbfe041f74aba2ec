// block_norm.hip -- the norm after a block, its gate, its residual scale, the
// residual addition and the norm before the next block, into float32, bfloat16
// or 8 bits with a scale per row.
//
//   u = x (mean_part x^2 + eps)^(-1/2) after_gain act(gate)
//   h = residual + scale u,  y = h (mean h^2 + eps)^(-1/2) before_gain
//
// Bound by memory: x, gate and residual are read once, sum and y written once.
// As in norm.hip a row stays in the registers of its team of threads; the
// norm after takes a sum over each of the row's parts, the one before a sum over
// the row, and 8 bits a maximum.  16384 rows of 4096 bfloat16 values with residual
// and gains into 8 bits: 100 us, 4.7 TB/s.
#include <hip/hip_runtime.h>

#include "norm_device.h"
#include "reader.h"

namespace mafat {
namespace {

// A norm's factor 1 / sqrt(sq / n + eps), each step rounded to nearest as norm.hip's
// divisions and root are.  Every thread of a row forms it for eight values, so where
// remainders are exact the steps are estimates (`per` is 1 / n) that one remainder
// corrects (Markstein), a third of the instructions: 16384 rows of 4096 bfloat16 values
// take 1.6 % more than with the hardware's estimates alone, and 4 % with divisions.  The
// last reciprocal's correction misses one root, all ones in its mantissa, which numbers
// of all ones, the last bit aside, have.
__device__ __forceinline__ float inverse_root(float sq, int n, float per, float eps) {
  const float count = static_cast<float>(n);
  if (sq >= 0x1p-60f && sq <= 0x1p100f) {
    const float q = sq * per;
    const float m = fmaf(fmaf(-q, count, sq), per, q) + eps;
    if (m < 0x1p126f && (__float_as_uint(m) & 0x7ffffe) != 0x7ffffe) {
      const float y = __builtin_amdgcn_rsqf(m), near = m * y;
      const float root = fmaf(fmaf(-near, near, m), 0.5f * y, near);
      return fmaf(fmaf(-root, y, 1.f), y, y);
    }
  }
  return 1.f / sqrtf(sq / count + eps);
}

// g or 1, times 1 / (1 + e^-g), as 2^-64 / (2^-64 + e^-g 2^-64): then neither the
// exponential nor the reciprocal leaves float32's normal numbers, which the hardware's
// instructions take, before the result does.  -g log2(e) in two parts, the second into
// the exponential as its derivative: within a few units down to where the result is
// zero.  (Below -110 the exponential counts as infinite: a gate times e^-110 is less than
// the least number.)
__device__ __forceinline__ float gate_of(float g, int silu) {
#pragma clang fp contract(off)  // (t is one rounded product wherever it is used)
  const float near = __builtin_amdgcn_fmed3f(g, -110.f, 110.f);
  const float t = near * -1.44269504f, down = t - 64.f;
  // (what `down` has of t: the sum is exact, as down's last bit is 2^-16 at most)
  const float rest = fmaf(near, -1.92596299e-8f, fmaf(near, -1.44269504f, -(down + 64.f)));
  float e = __builtin_amdgcn_exp2f(down);
  e = fmaf(e, rest * 0.693147181f, e);
  e = g >= -110.f ? e : g * -__builtin_huge_valf();  // (NaN stays)
  const float open = silu ? g : 1.f;
  return g > 110.f ? open : open * __builtin_amdgcn_rcpf(0x1p-64f + e) * 0x1p-64f;
}

// v of the lane that CONTROL names.
template <int CONTROL, typename T>
__device__ __forceinline__ T other_lane(T v) {
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, 15, 15, true));
}
// Over the TEAM threads of a row; all of them get the result.  Within a wave by
// exchanges of neighbours, quads, halves of 16 lanes, 16 lanes and halves.
template <int TEAM, typename T, typename F>
__device__ __forceinline__ T team_join(T v, F join, T* lds) {
  v = join(v, other_lane<0xb1>(v));
  v = join(v, other_lane<0x4e>(v));
  v = join(v, other_lane<0x141>(v));
  v = join(v, other_lane<0x140>(v));
  if constexpr (TEAM > 16) {
    const unsigned x = __builtin_bit_cast(unsigned, v);
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const unsigned a0 = a[0], a1 = a[1];  // (a bit cast of a vector's element takes the first one)
    v = join(__builtin_bit_cast(T, a0), __builtin_bit_cast(T, a1));
    const unsigned y = __builtin_bit_cast(unsigned, v);
    const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    const unsigned b0 = b[0], b1 = b[1];
    v = join(__builtin_bit_cast(T, b0), __builtin_bit_cast(T, b1));
  }
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

// n of the V floats at p (the rest are zero).
template <int V>
__device__ __forceinline__ void load_gain(const float* p, int n, float (&g)[V]) {
  if (n >= V) {
    __builtin_memcpy(g, p, 4 * V);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = i < n ? p[i] : 0.f;
  }
}

// As store_piece, past the caches.
template <int OUT, int V>
__device__ __forceinline__ void put_piece(typename OutElt<OUT>::T* p, int n, const float (&v)[V]) {
  if (n >= V) {
    typename OutElt<OUT>::T t[V];
    store_piece<OUT>(t, V, v);
    store_once(p, t);
  } else {
    store_piece<OUT>(p, n, v);
  }
}

// How the sums of a row's parts are formed: the row is one part; a part is a
// power of two of neighbouring lanes; parts of whole pieces, through LDS.
enum { PARTS_ROW = 0, PARTS_LANES = 1, PARTS_LDS = 2 };

// What a thread reads of a row, as it lies in memory.
template <typename T, int V, int NP>
struct RowPieces {
  T x[NP][V], gate[NP][V], res[NP][V];
};
template <typename T, int V, int NP>
__device__ __forceinline__ void load_pieces(const T* p, int cols, int first, int step, T (&t)[NP][V]) {
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = first + k * step, n = cols - c;
    if (n >= V) {
      load_once(p + c, t[k]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) t[k][i] = i < n ? p[c + i] : static_cast<T>(0);
    }
  }
}

// One row per team, NP pieces per thread at most: one, but for the longest rows,
// as many waves with all of their reads on the way at once are what hides the
// memory's latency (rows of 4096 bfloat16 values on 512 threads 113 us, on 256 with
// two pieces 125, and 181 row after row with the gains in registers; all of them before
// reads and writes went past the caches).
template <int DT, int OUT, int TEAM, int NP, int PARTS>
__global__ __launch_bounds__(TEAM > 64 ? TEAM : 256) void block_norm_kernel(const BlockArgs a) {
  using T = typename Elt<DT>::T;
  using Y = typename OutElt<OUT>::T;
  constexpr int V = Piece<DT>::V;
  constexpr int TEAMS = TEAM > 64 ? 1 : 256 / TEAM, WAVES = TEAM > 64 ? TEAM / 64 : 1;
  static_assert(PARTS != PARTS_LDS || TEAM > 64, "sums of parts in LDS are the block's");
  __shared__ float lds_a[WAVES], lds_b[WAVES];
  __shared__ uint32_t lds_max[WAVES];
  __shared__ float lds_part[PARTS == PARTS_LDS ? TEAM * NP : 1], lds_inv[PARTS == PARTS_LDS ? TEAM * NP : 1];
  const int t = static_cast<int>(threadIdx.x) % TEAM;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * TEAMS + static_cast<int>(threadIdx.x) / TEAM;
  if (row >= a.rows) return;  // whole teams; a team of several waves is the block
  // (Values past the row's last are zero all the way, or NaN where all of the row is.)
  RowPieces<T, V, NP> now;
  load_pieces(static_cast<const T*>(a.x) + row * a.x_stride, a.cols, t * V, TEAM * V, now.x);
  if (a.gate) load_pieces(static_cast<const T*>(a.gate) + row * a.gate_stride, a.cols, t * V, TEAM * V, now.gate);
  if (a.res) load_pieces(static_cast<const T*>(a.res) + row * a.res_stride, a.cols, t * V, TEAM * V, now.res);
  float after_gain[NP][V], scale[NP][V], before_gain[NP][V];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
#pragma unroll
    for (int i = 0; i < V; ++i) after_gain[k][i] = scale[k][i] = before_gain[k][i] = 1.f;
    const int c = (k * TEAM + t) * V;
    if (a.after_gain) load_gain<V>(a.after_gain + c, a.cols - c, after_gain[k]);
    if (a.scale) load_gain<V>(a.scale + c, a.cols - c, scale[k]);
    if (a.before_gain) load_gain<V>(a.before_gain + c, a.cols - c, before_gain[k]);
  }
  float h[NP][V];
#pragma unroll
  for (int k = 0; k < NP; ++k)
#pragma unroll
    for (int i = 0; i < V; ++i) h[k][i] = to_f(now.x[k][i]);
  if (a.after) {
    float inv[NP];
    if constexpr (PARTS == PARTS_ROW) {
      float sq = 0.f;
#pragma unroll
      for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) sq = fmaf(h[k][i], h[k][i], sq);
      sq = team_join<TEAM>(sq, Add{}, lds_a);
      const float one = inverse_root(sq, a.cols, a.per_col, a.eps);
#pragma unroll
      for (int k = 0; k < NP; ++k) inv[k] = one;
    } else {
      const int pieces = a.part / V;  // of a part
      float sq[NP];
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        sq[k] = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) sq[k] = fmaf(h[k][i], h[k][i], sq[k]);
      }
      if constexpr (PARTS == PARTS_LANES) {
        for (int o = pieces >> 1; o > 0; o >>= 1)
#pragma unroll
          for (int k = 0; k < NP; ++k) sq[k] += __shfl_xor(sq[k], o, 64);
#pragma unroll
        for (int k = 0; k < NP; ++k)  // (past the row's end there is no part: with an eps of 0 its factor would be infinite)
          inv[k] = (k * TEAM + t) * V < a.cols ? inverse_root(sq[k], a.part, a.per_part, a.eps) : 0.f;
      } else {
        const int lane = t & 63;
#pragma unroll
        for (int k = 0; k < NP; ++k) lds_part[k * TEAM + t] = sq[k];
        __syncthreads();
        for (int p = t >> 6; p < a.groups; p += TEAM / 64) {
          float s = 0.f;
          for (int i = lane; i < pieces; i += 64) s += lds_part[p * pieces + i];
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
          if (lane == 0) lds_inv[p] = inverse_root(s, a.part, a.per_part, a.eps);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NP; ++k) inv[k] = lds_inv[min((k * TEAM + t) / pieces, a.groups - 1)];
      }
    }
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] = h[k][i] * inv[k] * after_gain[k][i];
  }
  if (a.gate) {
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= gate_of(to_f(now.gate[k][i]), a.silu);
  }
  if (a.scale) {
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= scale[k][i];
  }
  if (a.res) {
    T* sum = static_cast<T*>(a.sum) + row * a.sum_stride;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int c = (k * TEAM + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] += to_f(now.res[k][i]);
      put_piece<DT>(sum + c, a.cols - c, h[k]);
    }
  }
  if (a.before) {
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
        sq = fmaf(h[k][i], h[k][i], sq);
    sq = team_join<TEAM>(sq, Add{}, lds_b);
    const float inv = inverse_root(sq, a.cols, a.per_col, a.eps);
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= inv * before_gain[k][i];
  }
  Y* y = static_cast<Y*>(a.y) + row * a.y_stride;
  if constexpr (OUT == MAFAT_F8) {
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
        most = MaxBits{}(most, __float_as_uint(h[k][i]) & 0x7fffffffu);
    most = team_join<TEAM>(most, MaxBits{}, lds_max);
    float by;
    const float y_scale = row_scale(most, &by);
    if (t == 0) a.y_scale[row] = y_scale;
#pragma unroll
    for (int k = 0; k < NP; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) h[k][i] *= by;
  }
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int c = (k * TEAM + t) * V;
    put_piece<OUT>(y + c, a.cols - c, h[k]);
  }
}

// Rows and parts of any length: a block of 1024 threads, value by value, reads
// its row again for every step (from the caches, mostly).
template <int DT, int OUT>
__global__ __launch_bounds__(1024) void block_norm_any_kernel(const BlockArgs a) {
  using T = typename Elt<DT>::T;
  using Y = typename OutElt<OUT>::T;
  constexpr int TEAM = 1024, WAVES = TEAM / 64;
  __shared__ float lds_inv[4096];
  __shared__ float lds_sum[2][WAVES];
  __shared__ uint32_t lds_max[WAVES];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63;
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + row * a.gate_stride : nullptr;
  const T* res = a.res ? static_cast<const T*>(a.res) + row * a.res_stride : nullptr;
  Y* y = static_cast<Y*>(a.y) + row * a.y_stride;
  if (a.after) {
    if (a.groups == 1) {
      float s = 0.f;
      for (int64_t i = tid; i < a.cols; i += TEAM) s = fmaf(to_f(x[i]), to_f(x[i]), s);
      s = team_reduce<TEAM>(s, Add{}, lds_sum[0]);
      if (tid == 0) lds_inv[0] = inverse_root(s, a.part, a.per_part, a.eps);
    } else {
      for (int p = tid >> 6; p < a.groups; p += WAVES) {
        float s = 0.f;
        const T* at = x + static_cast<int64_t>(p) * a.part;
        for (int i = lane; i < a.part; i += 64) s = fmaf(to_f(at[i]), to_f(at[i]), s);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
        if (lane == 0) lds_inv[p] = inverse_root(s, a.part, a.per_part, a.eps);
      }
    }
    __syncthreads();
  }
  const auto sum_at = [&](int64_t c) {
    float u = to_f(x[c]);
    if (a.after) {
      u *= lds_inv[static_cast<int>(c) / a.part];
      if (a.after_gain) u *= a.after_gain[c];
    }
    if (gate) u *= gate_of(to_f(gate[c]), a.silu);
    if (a.scale) u *= a.scale[c];
    return res ? u + to_f(res[c]) : u;
  };
  float inv = 1.f;
  if (a.before || res) {
    T* sum = static_cast<T*>(a.sum) + row * a.sum_stride;
    float s = 0.f;
    for (int64_t c = tid; c < a.cols; c += TEAM) {
      const float h = sum_at(c);
      if (res) store1(sum + c, h);
      s = fmaf(h, h, s);
    }
    if (a.before) inv = inverse_root(team_reduce<TEAM>(s, Add{}, lds_sum[1]), a.cols, a.per_col, a.eps);
  }
  const auto out_at = [&](int64_t c) {
    const float h = sum_at(c);
    return a.before ? h * (a.before_gain ? inv * a.before_gain[c] : inv) : h;
  };
  float by = 1.f;
  if constexpr (OUT == MAFAT_F8) {
    uint32_t most = 0;
    for (int64_t c = tid; c < a.cols; c += TEAM) most = MaxBits{}(most, __float_as_uint(out_at(c)) & 0x7fffffffu);
    most = team_reduce<TEAM>(most, MaxBits{}, lds_max);
    const float scale = row_scale(most, &by);
    if (tid == 0) a.y_scale[row] = scale;
  }
  for (int64_t c = tid; c < a.cols; c += TEAM) {
    if constexpr (OUT == MAFAT_F8) {
      y[c] = static_cast<Y>(__builtin_amdgcn_cvt_pk_fp8_f32(out_at(c) * by, 0.f, 0, false) & 0xff);
    } else {
      store1(y + c, out_at(c));
    }
  }
}

// A launch has fewer than 2^32 threads: where a row per block would pass
// that, `most` rows after another go in a launch of their own.
template <int DT, int OUT, typename F>
hipError_t by_rows(const BlockArgs& a, int64_t most, F launch_rows) {
  using T = typename Elt<DT>::T;
  using Y = typename OutElt<OUT>::T;
  for (int64_t at = 0; at < a.rows; at += most) {
    BlockArgs p = a;
    p.rows = a.rows - at < most ? a.rows - at : most;
    p.x = static_cast<const T*>(a.x) + at * a.x_stride;
    if (a.gate) p.gate = static_cast<const T*>(a.gate) + at * a.gate_stride;
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

template <int DT, int OUT>
hipError_t launch(const BlockArgs& a, hipStream_t stream) {
  constexpr int V = Piece<DT>::V;
  constexpr int64_t kThreads = int64_t{1} << 31;  // of a launch, at most
  const int64_t pieces = (static_cast<int64_t>(a.cols) + V - 1) / V;
  const int each = a.part / V;  // pieces of a part
  const bool one = !a.after || a.groups == 1, whole = a.part % V == 0;
  const bool lanes = whole && each <= 64 && (each & (each - 1)) == 0;
#define MAFAT_BLOCK(team_, np_, parts_)                                                                      \
  do {                                                                                                       \
    constexpr int teams = (team_) > 64 ? 1 : 256 / (team_), block = (team_) > 64 ? (team_) : 256;            \
    return by_rows<DT, OUT>(a, teams * (kThreads / block), [&](const BlockArgs& p) {                         \
      hipLaunchKernelGGL((block_norm_kernel<DT, OUT, team_, np_, parts_>),                                   \
                         dim3(static_cast<unsigned>((p.rows + teams - 1) / teams)), dim3(block), 0, stream, p); \
    });                                                                                                      \
  } while (0)
  if (one) {
    if (pieces <= 16) MAFAT_BLOCK(16, 1, PARTS_ROW);
    if (pieces <= 64) MAFAT_BLOCK(64, 1, PARTS_ROW);
    if (pieces <= 128) MAFAT_BLOCK(128, 1, PARTS_ROW);
    if (pieces <= 256) MAFAT_BLOCK(256, 1, PARTS_ROW);
    if (pieces <= 512) MAFAT_BLOCK(512, 1, PARTS_ROW);
    if (pieces <= 1024) MAFAT_BLOCK(1024, 1, PARTS_ROW);
    if (pieces <= 2048) MAFAT_BLOCK(1024, 2, PARTS_ROW);
  } else if (lanes) {
    if (pieces <= 64) MAFAT_BLOCK(64, 1, PARTS_LANES);
    if (pieces <= 256) MAFAT_BLOCK(256, 1, PARTS_LANES);
    if (pieces <= 512) MAFAT_BLOCK(512, 1, PARTS_LANES);
    if (pieces <= 1024) MAFAT_BLOCK(1024, 1, PARTS_LANES);
    if (pieces <= 2048) MAFAT_BLOCK(1024, 2, PARTS_LANES);
  } else if (whole) {
    if (pieces <= 256) MAFAT_BLOCK(256, 1, PARTS_LDS);
    if (pieces <= 512) MAFAT_BLOCK(512, 1, PARTS_LDS);
    if (pieces <= 1024) MAFAT_BLOCK(1024, 1, PARTS_LDS);
    if (pieces <= 2048) MAFAT_BLOCK(1024, 2, PARTS_LDS);
  }
#undef MAFAT_BLOCK
  return by_rows<DT, OUT>(a, kThreads / 1024, [&](const BlockArgs& p) {
    hipLaunchKernelGGL((block_norm_any_kernel<DT, OUT>), dim3(static_cast<unsigned>(p.rows)), dim3(1024), 0, stream, p);
  });
}

template <int DT>
hipError_t launch_in(int out_dtype, const BlockArgs& a, hipStream_t stream) {
  switch (out_dtype) {
    case MAFAT_F32: return launch<DT, MAFAT_F32>(a, stream);
    case MAFAT_BF16: return launch<DT, MAFAT_BF16>(a, stream);
    default: return launch<DT, MAFAT_F8>(a, stream);
  }
}

}  // namespace

hipError_t launch_block_norm(int dtype, int out_dtype, const BlockArgs& a, hipStream_t stream) {
  return dtype == MAFAT_BF16 ? launch_in<MAFAT_BF16>(out_dtype, a, stream) : launch_in<MAFAT_F32>(out_dtype, a, stream);
}

}  // namespace mafat
