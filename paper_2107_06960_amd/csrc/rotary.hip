// rotary.hip -- positions of queries and keys as rotations of pairs of values.
//
//   t = sum_a position_a * turns[a][i],  (x1, x2) -> m (x1 cos 2 pi t - x2 sin 2 pi t, x2 cos 2 pi t + x1 sin 2 pi t)
//
// Bound by memory: every value is read and written once.  A thread holds V
// pairs of a row (two pieces of 16 bytes of a head) and takes them through
// the heads, so that an angle's sine and cosine are computed once for all
// heads of q and k and stay in registers.
#include <hip/hip_runtime.h>

#include "norm_device.h"
#include "reader.h"

namespace mafat {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;  // heads whose loads are in flight together

// n of the V values at p, as they are (the rest are zero).
template <typename T, int V>
__device__ __forceinline__ void load_raw(const T* p, int n, T (&t)[V]) {
  if (n >= V) {
    __builtin_memcpy(t, p, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = i < n ? p[i] : static_cast<T>(0);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_raw(T* p, int n, const T (&t)[V]) {
  if (n >= V) {
    __builtin_memcpy(p, t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = t[i];
  }
}

template <int DT, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  using T = typename Elt<DT>::T;
  constexpr int V = Piece<DT>::V;
  const int tid = static_cast<int>(threadIdx.x);
  const int lr = div_small(tid, a.items), p = tid - lr * a.items;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / a.items) + lr;
  if (lr >= kThreads / a.items || row >= a.rows) return;
  const bool turning = p < a.turning;
  // the two pieces: first value and how many of them there are
  int at[2], n[2];
  if (!turning) {
    at[0] = 2 * a.pairs + 2 * V * (p - a.turning);
    at[1] = at[0] + V;
    n[0] = a.head_dim - at[0];
    n[1] = a.head_dim - at[1];
  } else if (INTERLEAVED) {
    at[0] = 2 * V * p;
    at[1] = at[0] + V;
    n[0] = 2 * a.pairs - at[0];
    n[1] = 2 * a.pairs - at[1];
  } else {
    at[0] = V * p;
    at[1] = a.pairs + V * p;
    n[0] = n[1] = a.pairs - V * p;
  }
  float cs[V], sn[V];
  if (turning) {
    int32_t pos[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) pos[x] = x < a.axes ? a.positions[row * a.axes + x] : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int pair = V * p + i;
      double t = 0.0;
      if (pair < a.pairs) {
        t = static_cast<double>(pos[0]) * a.turns[pair];
#pragma unroll
        for (int x = 1; x < 4; ++x)
          if (x < a.axes) t = fma(static_cast<double>(pos[x]), a.turns[x * a.pairs + pair], t);
      }
      // whole turns leave in float64, half a turn is 1 for sincospi
      sincospif(static_cast<float>(2.0 * (t - rint(t))), &sn[i], &cs[i]);
      cs[i] *= a.magnitude;
      sn[i] *= a.magnitude;
    }
  }
  const int first = static_cast<int>(blockIdx.y) * a.heads_each, last = min(first + a.heads_each, a.heads);
  for (int h0 = first; h0 < last; h0 += kAhead) {
    T v[kAhead][2][V];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = min(h0 + u, last - 1), of = h >= a.q_heads ? 1 : 0;
      const T* x = static_cast<const T*>(a.in[of]) + row * a.in_row[of] + (h - (of ? a.q_heads : 0)) * a.in_head[of];
      load_raw<T, V>(x + at[0], n[0], v[u][0]);
      load_raw<T, V>(x + at[1], n[1], v[u][1]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + u, of = h >= a.q_heads ? 1 : 0;
      if (h >= last) break;
      if (turning) {
        T w[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          // pair i of the thread: one value of each piece, or two in a row
          constexpr int H = V / 2;
          const float x1 = INTERLEAVED ? to_f(v[u][i / H][2 * (i % H)]) : to_f(v[u][0][i]);
          const float x2 = INTERLEAVED ? to_f(v[u][i / H][2 * (i % H) + 1]) : to_f(v[u][1][i]);
          const float y1 = x1 * cs[i] - x2 * sn[i], y2 = x2 * cs[i] + x1 * sn[i];
          store1(INTERLEAVED ? &w[i / H][2 * (i % H)] : &w[0][i], y1);
          store1(INTERLEAVED ? &w[i / H][2 * (i % H) + 1] : &w[1][i], y2);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) v[u][j][i] = w[j][i];
      }
      T* y = static_cast<T*>(a.out[of]) + row * a.out_row[of] + (h - (of ? a.q_heads : 0)) * a.out_head[of];
      store_raw<T, V>(y + at[0], n[0], v[u][0]);
      store_raw<T, V>(y + at[1], n[1], v[u][1]);
    }
  }
}

template <int DT>
hipError_t launch(bool interleaved, bool in_place, RotaryArgs a, hipStream_t stream) {
  using T = typename Elt<DT>::T;
  constexpr int V = Piece<DT>::V;
  a.turning = (a.pairs + V - 1) / V;
  a.items = a.turning + (in_place ? 0 : (a.head_dim - 2 * a.pairs + 2 * V - 1) / (2 * V));
  if (a.items == 0) return hipSuccess;  // nothing turns, in place
  const int rows_each = kThreads / a.items;
  const int64_t most = int64_t{rows_each} << 22;  // a launch has fewer than 2^32 threads along an axis
  for (int64_t from = 0; from < a.rows; from += most) {
    RotaryArgs p = a;
    p.rows = a.rows - from < most ? a.rows - from : most;
    p.positions = a.positions + from * a.axes;
    for (int i = 0; i < 2; ++i) {
      p.in[i] = static_cast<const T*>(a.in[i]) + from * a.in_row[i];
      p.out[i] = static_cast<T*>(a.out[i]) + from * a.out_row[i];
    }
    const int64_t blocks = (p.rows + rows_each - 1) / rows_each;
    // heads of a thread: all of them where rows alone fill the GPU
    int64_t each = a.heads * blocks / 1024;
    each = each < 1 ? 1 : each > a.heads ? a.heads : each;
    p.heads_each = static_cast<int32_t>(each);
    const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>((a.heads + each - 1) / each));
    if (interleaved) hipLaunchKernelGGL((rotary_kernel<DT, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((rotary_kernel<DT, false>), grid, dim3(kThreads), 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rotary(int dtype, bool interleaved, bool in_place, RotaryArgs a, hipStream_t stream) {
  return dtype == MAFAT_BF16 ? launch<MAFAT_BF16>(interleaved, in_place, a, stream)
                             : launch<MAFAT_F32>(interleaved, in_place, a, stream);
}

}  // namespace mafat
