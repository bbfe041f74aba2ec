// rotary.hip -- positions of queries and keys as rotations of pairs of values.
//
//   t = sum_a position_a * turns[a][i],  (x1, x2) -> m (x1 cos 2 pi t - x2 sin 2 pi t, x2 cos 2 pi t + x1 sin 2 pi t)
//
// Bound by memory: every value is read and written once.  A block has a few rows
// of q and k: it forms the sines and cosines of their pairs once for all heads,
// into LDS, and its threads then take the rows' pieces in the order that they lie
// in memory, V pairs (two pieces of 16 bytes) each.  (With the angles in a thread's
// registers and its heads one after another, a block read 256 bytes of each of 32
// rows at a time: 16384 rows of 40 heads of 128 took 87 us.)
#include <hip/hip_runtime.h>

#include "norm_device.h"
#include "reader.h"

namespace mafat {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 2;  // pieces of a thread whose loads are in flight together

// n of the V values at p, as they are (the rest are zero).  Fewer than V in at most
// three accesses, since other lanes of the wave wait for them: heads whose pairs
// are not whole pieces have such in every wave (4380 rows of 58 heads of 128, of
// which 24 turn: 67 us value by value).
template <typename T, int V>
__device__ __forceinline__ void load_raw(const T* p, int n, T (&t)[V]) {
  if (n >= V) {
    load_once(p, t);
    return;
  }
  n = n < 0 ? 0 : n;
  uint64_t w[2] = {0, 0};
  constexpr int BITS = 8 * sizeof(T);
  if constexpr (V == 8) {
    if (n & 4) __builtin_memcpy(&w[0], p, 4 * sizeof(T));
  }
  const int four = V == 8 ? n & 4 : 0;
  if (n & 2) {
    uint64_t two = 0;
    __builtin_memcpy(&two, p + four, 2 * sizeof(T));
    if (four) w[1] = two;
    else w[0] = two;
  }
  if (n & 1) {
    const int at = (n & ~1) * BITS;
    uint64_t one = 0;
    __builtin_memcpy(&one, p + (n & ~1), sizeof(T));
    one <<= at & 63;
    if (at >> 6) w[1] |= one;
    else w[0] |= one;
  }
  __builtin_memcpy(t, w, sizeof(t));
}
template <typename T, int V>
__device__ __forceinline__ void store_raw(T* p, int n, const T (&t)[V]) {
  if (n >= V) {
    store_once(p, t);
    return;
  }
  n = n < 0 ? 0 : n;
  uint64_t w[2];
  constexpr int BITS = 8 * sizeof(T);
  __builtin_memcpy(w, t, sizeof(w));
  if constexpr (V == 8) {
    if (n & 4) __builtin_memcpy(p, &w[0], 4 * sizeof(T));
  }
  const int four = V == 8 ? n & 4 : 0;
  if (n & 2) {
    const uint64_t two = four ? w[1] : w[0];
    __builtin_memcpy(p + four, &two, 2 * sizeof(T));
  }
  if (n & 1) {
    const int at = (n & ~1) * BITS;
    const uint64_t one = ((at >> 6) ? w[1] : w[0]) >> (at & 63);
    __builtin_memcpy(p + (n & ~1), &one, sizeof(T));
  }
}

template <int DT, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  using T = typename Elt<DT>::T;
  constexpr int V = Piece<DT>::V;
  extern __shared__ __align__(16) float trig[];  // cosines and sines: [rows][2][pairs, whole pieces of V]
  const int tid = static_cast<int>(threadIdx.x);
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.rows_each;
  const int rows = static_cast<int>(a.rows - row0 < a.rows_each ? a.rows - row0 : a.rows_each);
  const int padded = a.turning * V, in_row = a.heads * a.items, all = rows * in_row;

  T v[kAhead][2][V];
  // Piece `item` of the block's: where it is, which pairs, and its loads.
  struct Place {
    int row, of, head, at[2], n[2], pair;
  };
  const auto place = [&](int item) {
    Place w;
    w.row = div_small(item, in_row);
    const int rest = item - w.row * in_row, h = div_small(rest, a.items), p = rest - h * a.items;
    w.of = h >= a.q_heads ? 1 : 0;
    w.head = h - (w.of ? a.q_heads : 0);
    w.pair = p < a.turning ? V * p : -1;
    if (p >= a.turning) {  // behind the pairs
      w.at[0] = 2 * a.pairs + 2 * V * (p - a.turning);
      w.at[1] = w.at[0] + V;
      w.n[0] = a.head_dim - w.at[0];
      w.n[1] = a.head_dim - w.at[1];
    } else if (INTERLEAVED) {
      w.at[0] = 2 * V * p;
      w.at[1] = w.at[0] + V;
      w.n[0] = 2 * a.pairs - w.at[0];
      w.n[1] = 2 * a.pairs - w.at[1];
    } else {
      w.at[0] = V * p;
      w.at[1] = a.pairs + V * p;
      w.n[0] = w.n[1] = a.pairs - V * p;
    }
    return w;
  };
  const auto fetch = [&](const Place& w, T (&t)[2][V]) {
    const T* x = static_cast<const T*>(a.in[w.of]) + (row0 + w.row) * a.in_row[w.of] + w.head * a.in_head[w.of];
    load_raw<T, V>(x + w.at[0], w.n[0], t[0]);
    load_raw<T, V>(x + w.at[1], w.n[1], t[1]);
  };
  // The first pieces are on their way while the angles are formed.
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (tid + u * kThreads < all) fetch(place(tid + u * kThreads), v[u]);
  for (int i = tid; i < rows * padded; i += kThreads) {
    const int r = div_small(i, padded), pair = i - r * padded;
    double t = 0.0;
    if (pair < a.pairs) {
      const int32_t* pos = a.positions + (row0 + r) * a.axes;
      t = static_cast<double>(pos[0]) * a.turns[pair];
      for (int x = 1; x < a.axes; ++x) t = fma(static_cast<double>(pos[x]), a.turns[x * a.pairs + pair], t);
    }
    float sn, cs;
    // whole turns leave in float64, half a turn is 1 for sincospi
    sincospif(static_cast<float>(2.0 * (t - rint(t))), &sn, &cs);
    trig[2 * r * padded + pair] = cs * a.magnitude;
    trig[(2 * r + 1) * padded + pair] = sn * a.magnitude;
  }
  __syncthreads();
  for (int first = tid; first < all; first += kAhead * kThreads) {
    if (first != tid) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (first + u * kThreads < all) fetch(place(first + u * kThreads), v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (first + u * kThreads >= all) break;
      const Place w = place(first + u * kThreads);
      if (w.pair >= 0) {
        float cs[V], sn[V];
        __builtin_memcpy(cs, __builtin_assume_aligned(trig + 2 * w.row * padded + w.pair, 16), sizeof(cs));
        __builtin_memcpy(sn, __builtin_assume_aligned(trig + (2 * w.row + 1) * padded + w.pair, 16), sizeof(sn));
        T y[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          // pair i of the thread: one value of each piece, or two in a row
          constexpr int H = V / 2;
          const float x1 = INTERLEAVED ? to_f(v[u][i / H][2 * (i % H)]) : to_f(v[u][0][i]);
          const float x2 = INTERLEAVED ? to_f(v[u][i / H][2 * (i % H) + 1]) : to_f(v[u][1][i]);
          const float y1 = x1 * cs[i] - x2 * sn[i], y2 = x2 * cs[i] + x1 * sn[i];
          store1(INTERLEAVED ? &y[i / H][2 * (i % H)] : &y[0][i], y1);
          store1(INTERLEAVED ? &y[i / H][2 * (i % H) + 1] : &y[1][i], y2);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < V; ++i) v[u][j][i] = y[j][i];
      }
      T* y = static_cast<T*>(a.out[w.of]) + (row0 + w.row) * a.out_row[w.of] + w.head * a.out_head[w.of];
      store_raw<T, V>(y + w.at[0], w.n[0], v[u][0]);
      store_raw<T, V>(y + w.at[1], w.n[1], v[u][1]);
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
  // Rows of a block: a pair's angle for each thread, if there are rows for every CU; and no
  // more pieces than a quotient of theirs may have (see div_small).
  const int64_t padded = static_cast<int64_t>(a.turning) * V, in_row = static_cast<int64_t>(a.heads) * a.items;
  int64_t each = padded > 0 ? kThreads / padded : kThreads / in_row;
  if (each > a.rows / 512) each = a.rows / 512;
  if (each > 32) each = 32;
  a.rows_each = static_cast<int32_t>(each < 1 ? 1 : each);
  const size_t lds = static_cast<size_t>(a.rows_each) * 2 * padded * sizeof(float);
  const int64_t most = int64_t{a.rows_each} << 22;  // a launch has fewer than 2^32 threads
  for (int64_t from = 0; from < a.rows; from += most) {
    RotaryArgs p = a;
    p.rows = a.rows - from < most ? a.rows - from : most;
    p.positions = a.positions + from * a.axes;
    for (int i = 0; i < 2; ++i) {
      p.in[i] = static_cast<const T*>(a.in[i]) + from * a.in_row[i];
      p.out[i] = static_cast<T*>(a.out[i]) + from * a.out_row[i];
    }
    const dim3 grid(static_cast<unsigned>((p.rows + a.rows_each - 1) / a.rows_each));
    if (interleaved) hipLaunchKernelGGL((rotary_kernel<DT, true>), grid, dim3(kThreads), lds, stream, p);
    else hipLaunchKernelGGL((rotary_kernel<DT, false>), grid, dim3(kThreads), lds, stream, p);
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
