// decay.hip -- linear attention with a decay for each head: tokens of a request
// in order, a state of key_dim x value_dim per request and key/value head.
//
//   S_t = a_t S_{t-1} + k_t v_t^T,  y_t = scale q_t S_t
//
// Single tokens run token after token (decay_step_kernel), bound by reading and
// writing the states.  Prompts run in chunks of C tokens, with c_i the sum of log a
// over the chunk's tokens up to i:
//   y_i = scale (e^{c_i} q_i S_0 + sum_{j <= i} e^{c_i - c_j} (q_i . k_j) v_j)
//   S_C = e^{c_C} S_0 + sum_j e^{c_C - c_j} k_j v_j^T
// all of it products of matrices; exponents are differences of later and earlier
// sums, so none is above 0.  A block takes the chunks of one request and head in
// turn, its part of the state in the registers of the matrix accumulators.
// Where that leaves too few blocks, requests are cut into segments: a first launch
// forms what each segment adds to the state, a second one turns these into the
// states that the segments start from, the last one gives the outputs.
#include "decay_device.h"
#include "decay_launch.h"
#include "norm_device.h"

namespace mafat {
namespace {

// ------------------------------------------------------------ single tokens

// As load4 and put4 of float32, past the caches.
__device__ __forceinline__ f32x4 load4_once(const float* p, int n) {
  if (n < 4) return load4<float>(p, n);
  float t[4];
  load_once(p, t);
  return f32x4{t[0], t[1], t[2], t[3]};
}
__device__ __forceinline__ void put4_once(float* p, int n, f32x4 v) {
  if (n < 4) return put4<float>(p, n, v);
  const float t[4] = {v[0], v[1], v[2], v[3]};
  store_once(p, t);
}

// 64 columns of a state a block; a thread holds 4 of them in RPT of its rows, all
// of whose reads are on the way at once.  64 requests of 16 heads of 128: 27 us,
// 4.9 TB/s.
template <int DT, int RPT>
__global__ __launch_bounds__(256) void decay_step_kernel(const DecayArgs a) {
  using T = typename Elt<DT>::T;
  __shared__ f32x4 part[4][16];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int id = a.first_block + static_cast<int>(blockIdx.x);
  const int rh = static_cast<int>(static_cast<uint32_t>(id) / static_cast<uint32_t>(a.slices));
  const int slice = id - rh * a.slices;
  const int request = static_cast<int>(static_cast<uint32_t>(rh) / static_cast<uint32_t>(a.kv_heads));
  const int kv = rh - request * a.kv_heads;
  const int ahead = slots_ahead(a);
  int first, n;
  rows_of(a, request, &first, &n);
  if (n == 0) return;
  const int64_t slot = slot_of(a, request, ahead);
  const int c = 64 * slice + 4 * (tid & 15), nc = a.value_dim - c, r0 = tid >> 4;
  float* state = nullptr;
  f32x4 s[RPT];
  if (slot >= 0) {
    state = a.states + slot * a.state_slot + static_cast<int64_t>(kv) * a.key_dim * a.value_dim + c;
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = r0 + 16 * i;
      s[i] = load4_once(state + static_cast<int64_t>(r) * a.value_dim, r < a.key_dim ? nc : 0);
    }
  } else {
    const float f = slot == SLOT_TAKEN ? __builtin_nanf("") : 0.f;
#pragma unroll
    for (int i = 0; i < RPT; ++i) s[i] = f32x4{f, f, f, f};
  }
  for (int t = 0; t < n; ++t) {
    const int64_t row = first + t;
    const T* kp = static_cast<const T*>(a.k) + row * a.k_row + kv * a.k_head;
    const f32x4 v = load4<T>(static_cast<const T*>(a.v) + row * a.v_row + kv * a.v_head + c, nc);
    const float g = power2(decay_log2(a.log_decay[(a.decay_by_row ? row * a.decay_row : 0) + kv]));
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = r0 + 16 * i;
      const float k = r < a.key_dim ? to_f(kp[r]) : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = fmaf(k, v[j], g * s[i][j]);
    }
    for (int h = 0; h < a.group; ++h) {
      const int head = kv * a.group + h;
      const T* qp = static_cast<const T*>(a.q) + row * a.q_row + head * a.q_head;
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const int r = r0 + 16 * i;
        if (r < a.key_dim) {
          const float q = to_f(qp[r]);
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = fmaf(q, s[i][j], y[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] += __shfl_xor(y[j], 16, 64);
        y[j] += __shfl_xor(y[j], 32, 64);
      }
      if (lane < 16) part[wave][lane] = y;
      __syncthreads();
      if (tid < 16)
        put4<T>(static_cast<T*>(a.y) + row * a.y_row + head * a.y_head + c, nc,
                ((part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid])) * a.scale);
      __syncthreads();
    }
  }
  if (state) {
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int r = r0 + 16 * i;
      if (r < a.key_dim) put4_once(state + static_cast<int64_t>(r) * a.value_dim, nc, s[i]);
    }
  }
}

// ------------------------------------------------------------ prompts, any size

// Any size, stride, alignment and type: 32 tokens at a time as float32 in LDS
// and on the float32 matrix instructions (bfloat16 values are exact there).  A
// block has 64 columns of the state, a wave 16 of them in KT tiles of 16 rows.
// The 16x16x4 instruction's operands hold, in lane l, row (column) l % 16 and
// the summed axis' entry l / 16; its result column l % 16 and rows 4 (l / 16) + r.
// So the state's tile T is the operand of q S as it stands, if step r of the
// instruction sums over the keys' entries 16 T + 4 (l / 16) + r.  Bound by these
// instructions, a tenth of bfloat16's rate: 4131 rows of 16 heads of 128 in float32
// take 126 us, of 59 in bfloat16 73 (of 56, in decay_bf16.hip, 37).
template <int DT, int KT, int MODE>
__global__ __launch_bounds__(256) void decay_any_kernel(const DecayArgs a) {
  using T = typename Elt<DT>::T;
  constexpr int C = 32, KP = 16 * KT + 4, VP = 68, PP = 36;  // tokens; floats of a row of LDS
  __shared__ __align__(16) float sk[C * KP];
  __shared__ __align__(16) float sq[MODE == DECAY_OUTPUTS ? C * KP : 4];
  __shared__ __align__(16) float sv[C * VP];
  __shared__ __align__(16) float sp[MODE == DECAY_OUTPUTS ? C * PP : 4];
  __shared__ double sc[C];
  __shared__ int odd;  // whether the chunk's values are not all finite
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int l16 = lane & 15, h4 = lane >> 4;
  // (Slices last: workgroups go round the XCDs, and segments that are not there come
  // last, so that every XCD has as many that are.)
  const int id = a.first_block + static_cast<int>(blockIdx.x), all_bh = a.segments * a.kv_heads;
  const int slice = static_cast<int>(static_cast<uint32_t>(id) / static_cast<uint32_t>(all_bh));
  const int bh = id - slice * all_bh;
  const int b = static_cast<int>(static_cast<uint32_t>(bh) / static_cast<uint32_t>(a.kv_heads));
  const int kv = bh - b * a.kv_heads;
  const int ahead = slots_ahead(a);
  const Segment seg = find_segment(a, b);
  if (!seg.any || (MODE == DECAY_ADDS && seg.index + 1 == seg.count)) return;
  const int c0 = 64 * slice, col = c0 + 16 * wave + l16;  // of the state
  const int64_t slot = MODE == DECAY_OUTPUTS && (seg.index == 0 || seg.index + 1 == seg.count) ? slot_of(a, seg.request, ahead) : SLOT_NONE;
  float* const kept = slot >= 0 ? a.states + slot * a.state_slot + static_cast<int64_t>(kv) * a.key_dim * a.value_dim : nullptr;
  float* const part = a.part + (static_cast<int64_t>(b) * a.kv_heads + kv) * a.key_dim * a.value_dim;

  f32x4 s[KT];
  if (MODE == DECAY_OUTPUTS && (kept || seg.count > 1)) {
    const float* from = seg.count > 1 ? part : kept;
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * i + 4 * h4 + r;
        s[i][r] = row < a.key_dim && col < a.value_dim ? from[static_cast<int64_t>(row) * a.value_dim + col] : 0.f;
      }
  } else {
    const float f = slot == SLOT_TAKEN ? __builtin_nanf("") : 0.f;
#pragma unroll
    for (int i = 0; i < KT; ++i) s[i] = f32x4{f, f, f, f};
  }
  // The next chunk (and the next head's queries) are on their way in registers while
  // one is worked on.
  constexpr int KN = C * 4 * KT / 256, VN = C * 16 / 256;
  f32x4 next_k[KN], next_v[VN], next_q[MODE == DECAY_OUTPUTS ? KN : 1];
  float next_decay = 0.f;
  const auto ask = [&](int t0) {
    const int n = min(C, seg.n - t0);
    const int64_t row0 = seg.first + t0;
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int e = tid + 256 * i, r = e / (4 * KT), d = 4 * (e % (4 * KT));
      next_k[i] = load4<T>(static_cast<const T*>(a.k) + (row0 + r) * a.k_row + kv * a.k_head + d, r < n ? a.key_dim - d : 0);
    }
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int e = tid + 256 * i, r = e >> 4, d = 4 * (e & 15);
      next_v[i] = load4<T>(static_cast<const T*>(a.v) + (row0 + r) * a.v_row + kv * a.v_head + c0 + d, r < n ? a.value_dim - c0 - d : 0);
    }
    next_decay = lane < n ? a.log_decay[(a.decay_by_row ? (row0 + lane) * a.decay_row : 0) + kv] : 0.f;
  };
  const auto ask_q = [&](int t0, int h) {
    const int n = min(C, seg.n - t0);
    const int64_t row0 = seg.first + t0;
#pragma unroll
    for (int i = 0; i < (MODE == DECAY_OUTPUTS ? KN : 0); ++i) {
      const int e = tid + 256 * i, r = e / (4 * KT), d = 4 * (e % (4 * KT));
      next_q[i] = load4<T>(static_cast<const T*>(a.q) + (row0 + r) * a.q_row + (kv * a.group + h) * a.q_head + d,
                           r < n ? a.key_dim - d : 0);
    }
  };
  ask(0);
  ask_q(0, 0);
  double total = 0.0;
  for (int t0 = 0; t0 < seg.n; t0 += C) {
    const int n = min(C, seg.n - t0);
    const int64_t row0 = seg.first + t0;
    __syncthreads();
    if (tid == 0) odd = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KN; ++i) {
      const int e = tid + 256 * i;
      *reinterpret_cast<f32x4*>(&sk[e / (4 * KT) * KP + 4 * (e % (4 * KT))]) = next_k[i];
    }
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int e = tid + 256 * i;
      const f32x4 v = next_v[i];
      const float z = (v[0] - v[0]) + (v[1] - v[1]) + (v[2] - v[2]) + (v[3] - v[3]);
      if (!(z == 0.f)) odd = 1;
      *reinterpret_cast<f32x4*>(&sv[(e >> 4) * VP + 4 * (e & 15)]) = v;
    }
    const float decay = next_decay;
    if (t0 + C < seg.n) ask(t0 + C);
    if (wave == 0) {
      double g = 0.0;
      if (lane < n) g = decay_log2(decay);
#pragma unroll
      for (int o = 1; o < C; o <<= 1) {
        const double left = __shfl_up(g, o, 64);
        g += lane >= o ? left : 0.0;
      }
      if (lane < C) sc[lane] = g;
    }
    __syncthreads();
    if constexpr (MODE == DECAY_OUTPUTS) {
      for (int h = 0; h < a.group; ++h) {
        const int head = kv * a.group + h;
#pragma unroll
        for (int i = 0; i < KN; ++i) {
          const int e = tid + 256 * i;
          *reinterpret_cast<f32x4*>(&sq[e / (4 * KT) * KP + 4 * (e % (4 * KT))]) = next_q[i];
        }
        if (h + 1 < a.group) ask_q(t0, h + 1);
        else if (t0 + C < seg.n) ask_q(t0 + C, 0);
        __syncthreads();
        {  // scores: a tile of 16 x 16 per wave, none above the diagonal
          const int ti = wave >> 1, tj = wave & 1;
          f32x4 p = {0.f, 0.f, 0.f, 0.f}, p2 = p;  // two sums: an instruction's result takes several times its issue
          if (tj <= ti) {
#pragma unroll
            for (int i = 0; i < KT; ++i) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(&sq[(16 * ti + l16) * KP + 16 * i + 4 * h4]);
              const f32x4 y = *reinterpret_cast<const f32x4*>(&sk[(16 * tj + l16) * KP + 16 * i + 4 * h4]);
#pragma unroll
              for (int r = 0; r < 4; r += 2) {
                p = __builtin_amdgcn_mfma_f32_16x16x4f32(x[r], y[r], p, 0, 0, 0);
                p2 = __builtin_amdgcn_mfma_f32_16x16x4f32(x[r + 1], y[r + 1], p2, 0, 0, 0);
              }
            }
            p += p2;
          }
          const int j = 16 * tj + l16;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = 16 * ti + 4 * h4 + r;
            const float w = power2(static_cast<float>(sc[i] - sc[j]));
            sp[i * PP + j] = j <= i ? p[r] * w : 0.f;
          }
        }
        f32x4 o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < KT; ++i) {
          f32x4 x[2];
#pragma unroll
          for (int ti = 0; ti < 2; ++ti) x[ti] = *reinterpret_cast<const f32x4*>(&sq[(16 * ti + l16) * KP + 16 * i + 4 * h4]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int ti = 0; ti < 2; ++ti) o[ti] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[ti][r], s[i][r], o[ti], 0, 0, 0);
        }
#pragma unroll
        for (int ti = 0; ti < 2; ++ti)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[ti][r] *= power2(static_cast<float>(sc[16 * ti + 4 * h4 + r]));
        __syncthreads();
        if (odd) {  // a later token's value must not reach a row, not even times zero
#pragma unroll
          for (int ti = 0; ti < 2; ++ti)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int i = 16 * ti + 4 * h4 + r;
              for (int j = 0; j <= i; ++j) o[ti][r] = fmaf(sp[i * PP + j], sv[j * VP + 16 * wave + l16], o[ti][r]);
            }
        } else {
#pragma unroll
          for (int ti = 0; ti < 2; ++ti)
#pragma unroll
            for (int tj = 0; tj <= ti; ++tj) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(&sp[(16 * ti + l16) * PP + 16 * tj + 4 * h4]);
#pragma unroll
              for (int r = 0; r < 4; ++r)
                o[ti] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[r], sv[(16 * tj + 4 * h4 + r) * VP + 16 * wave + l16], o[ti], 0, 0, 0);
            }
        }
        if (col < a.value_dim) {
#pragma unroll
          for (int ti = 0; ti < 2; ++ti)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int i = 16 * ti + 4 * h4 + r;
              if (i < n) store1(static_cast<T*>(a.y) + (row0 + i) * a.y_row + head * a.y_head + col, o[ti][r] * a.scale);
            }
        }
        __syncthreads();
      }
    }
    // the state after the chunk
    total += sc[C - 1];
    const float down = power2(static_cast<float>(sc[C - 1]));
#pragma unroll
    for (int i = 0; i < KT; ++i) s[i] *= down;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * t + 4 * h4 + r;
        const float v = sv[j * VP + 16 * wave + l16] * power2(static_cast<float>(sc[C - 1] - sc[j]));
#pragma unroll
        for (int i = 0; i < KT; ++i) s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(sk[j * KP + 16 * i + l16], v, s[i], 0, 0, 0);
      }
  }
  float* const to = MODE == DECAY_ADDS ? part : seg.index + 1 == seg.count ? kept : nullptr;
  if (to) {
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 16 * i + 4 * h4 + r;
        if (row < a.key_dim && col < a.value_dim) to[static_cast<int64_t>(row) * a.value_dim + col] = s[i][r];
      }
  }
  if (MODE == DECAY_ADDS && slice == 0 && tid == 0)
    a.factor[static_cast<int64_t>(b) * a.kv_heads + kv] = power2(total);
}

// What segments add -> what they start from, for requests of several segments.
// A thread takes V entries of a head's state through the segments, with the next
// AHEAD of them on their way.  (121 segments of 4 heads of 128: 15 us at best with 32 ahead, 19 with 8.)
template <int V, int AHEAD>
__global__ __launch_bounds__(256) void decay_join_kernel(const DecayArgs a) {
  typedef float fv __attribute__((ext_vector_type(V)));
  const int64_t size = static_cast<int64_t>(a.key_dim) * a.value_dim;
  const int per = static_cast<int>((size + 256 * V - 1) / (256 * V));
  const int id = a.first_block + static_cast<int>(blockIdx.x);
  const int rh = static_cast<int>(static_cast<uint32_t>(id) / static_cast<uint32_t>(per));
  const int64_t e = V * (static_cast<int64_t>(id - rh * per) * 256 + threadIdx.x);
  const int request = static_cast<int>(static_cast<uint32_t>(rh) / static_cast<uint32_t>(a.kv_heads));
  const int kv = rh - request * a.kv_heads;
  // the request's first segment, and how many there are
  const int ahead = slots_ahead(a);
  int first, n, length;
  rows_of(a, request, &first, &n);
  const int count = segments_of(a, n, &length);
  if (count < 2) return;
  uint32_t b = static_cast<uint32_t>(request) * static_cast<uint32_t>(count);
  if (a.offsets) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    b = 0;
    for (int r = lane; r < request; r += 64) {
      int lo, m, len;
      rows_of(a, r, &lo, &m);
      b += static_cast<uint32_t>(segments_of(a, m, &len));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) b += static_cast<uint32_t>(__shfl_xor(static_cast<int>(b), o, 64));
  }
  const uint32_t room = static_cast<uint32_t>(a.segments);
  if (b > room || static_cast<uint32_t>(count) > room - b) return;  // (offsets that decrease)
  const int64_t slot = slot_of(a, request, ahead);
  if (e >= size) return;
  const float start = slot == SLOT_TAKEN ? __builtin_nanf("") : 0.f;
  fv s;
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = start;
  if (slot >= 0) __builtin_memcpy(&s, a.states + slot * a.state_slot + kv * size + e, sizeof(s));
  float* const part = a.part + (static_cast<int64_t>(b) * a.kv_heads + kv) * size + e;
  const float* const factor = a.factor + static_cast<int64_t>(b) * a.kv_heads + kv;
  const int64_t step = a.kv_heads * size;
  for (int i0 = 0; i0 < count; i0 += AHEAD) {
    fv adds[AHEAD];
    float by[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      by[i] = 0.f;
#pragma unroll
      for (int j = 0; j < V; ++j) adds[i][j] = 0.f;
      if (i0 + i + 1 < count) {  // (the last adds nothing to another's start)
        __builtin_memcpy(&adds[i], part + (i0 + i) * step, sizeof(s));
        by[i] = factor[static_cast<int64_t>(i0 + i) * a.kv_heads];
      }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (i0 + i < count) __builtin_memcpy(part + (i0 + i) * step, &s, sizeof(s));
#pragma unroll
      for (int j = 0; j < V; ++j) s[j] = fmaf(s[j], by[i], adds[i][j]);
    }
  }
}

template <int DT, int MODE>
hipError_t launch_chunks(DecayArgs a, hipStream_t stream) {
  if (DT == MAFAT_BF16 && decay_bf16_fits(a)) return launch_decay_bf16(MODE, a, stream);
  a.slices = (a.value_dim + 63) / 64;
  return for_decay_blocks(a, [&](const DecayArgs& p, unsigned n) {
    if (a.key_dim <= 64) hipLaunchKernelGGL((decay_any_kernel<DT, 4, MODE>), dim3(n), dim3(256), 0, stream, p);
    else if (a.key_dim <= 128) hipLaunchKernelGGL((decay_any_kernel<DT, 8, MODE>), dim3(n), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((decay_any_kernel<DT, 16, MODE>), dim3(n), dim3(256), 0, stream, p);
  });
}

template <int V, int AHEAD>
hipError_t launch_join(DecayArgs a, hipStream_t stream) {
  const int64_t size = static_cast<int64_t>(a.key_dim) * a.value_dim;
  const int64_t blocks = static_cast<int64_t>(a.requests) * a.kv_heads * ((size + 256 * V - 1) / (256 * V));
  if (blocks >= (int64_t{1} << 31)) return hipErrorInvalidValue;
  return for_block_parts(blocks, [&](int32_t from, unsigned n) {
    a.first_block = from;
    hipLaunchKernelGGL((decay_join_kernel<V, AHEAD>), dim3(n), dim3(256), 0, stream, a);
  });
}

template <int DT>
hipError_t launch_step(DecayArgs a, hipStream_t stream) {
  a.slices = (a.value_dim + 63) / 64;
  const int64_t blocks = static_cast<int64_t>(a.requests) * a.kv_heads * a.slices;
  if (blocks >= (int64_t{1} << 31)) return hipErrorInvalidValue;
  return for_block_parts(blocks, [&](int32_t from, unsigned n) {
    a.first_block = from;
    if (a.key_dim <= 64) hipLaunchKernelGGL((decay_step_kernel<DT, 4>), dim3(n), dim3(256), 0, stream, a);
    else if (a.key_dim <= 128) hipLaunchKernelGGL((decay_step_kernel<DT, 8>), dim3(n), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((decay_step_kernel<DT, 16>), dim3(n), dim3(256), 0, stream, a);
  });
}

template <int DT>
hipError_t launch(const DecayArgs& a, const DecayPlan& p, hipStream_t stream) {
  if (p.recurrent) return launch_step<DT>(a, stream);
  // (without offsets the requests' lengths are known)
  if (p.split && (a.offsets || a.per_request > a.segment)) {
    hipError_t e = launch_chunks<DT, DECAY_ADDS>(a, stream);
    // Entries four at a time where there are heads for a wave a SIMD; few heads have many
    // segments each.
    const bool many = static_cast<int64_t>(a.requests) * a.kv_heads * a.key_dim * a.value_dim >= 4 * 65536;
    if (e == hipSuccess)
      e = many && a.key_dim * a.value_dim % 4 == 0 ? launch_join<4, 8>(a, stream) : launch_join<1, 32>(a, stream);
    if (e != hipSuccess) return e;
  }
  return launch_chunks<DT, DECAY_OUTPUTS>(a, stream);
}

}  // namespace

DecayPlan plan_decay(const mafat_decay& c) {
  DecayPlan p{};
  // One token a request, if they are alike (two where the chunked kernel is the slow one):
  // a chunk would be nearly empty.  (64 requests, 16 heads of 128: one token each 28.5 us;
  // two in turn 31, in a chunk 28; four in a chunk 28.)
  // Segments that leave two blocks a CU, all of them at once: one
  // more would make the call take twice as long.  A request adds a segment that is not
  // full.  With that many requests alone, twice their mean length.
  const int columns = c.dtype == MAFAT_BF16 && c.key_dim % 8 == 0 && c.value_dim % 8 == 0 ? 128 : 64;  // of a block, mostly
  p.recurrent = c.rows <= (columns == 128 ? 1 : 2) * int64_t{c.requests};
  const int64_t slices = (c.value_dim + columns - 1) / columns;
  const int64_t room = c.key_dim > 128 ? 256 : 512;  // (one block a CU at larger heads)
  const int64_t most = room / (c.kv_heads * slices);
  int64_t len = most > 2 * int64_t{c.requests} ? c.rows / (most - c.requests) : 2 * (c.rows / c.requests);
  // A chunk takes 1 us in decay_bf16.hip, 3 to 7 here, and the two launches more 8: one request of
  // 1024 rows of 8 heads of 64 takes 30, 22 or 18 us in segments of 256, 128 or 64, of 4096 rows
  // 32, 26 or 29; one of 130 rows 11.5 whole and 18 in two (1 more since states enter outputs in two parts).
  const int64_t least = columns == 64 ? 64 : c.rows <= 256 ? 256 : 128;
  len = len < least ? least : len > 8192 ? 8192 : (len + 31) / 32 * 32;  // (extents of a segment are 31 bits wide)
  p.segment = len;
  p.segments = c.rows / len + c.requests;
  p.split = !p.recurrent && c.rows > len;
  return p;
}

hipError_t launch_decay(int dtype, const DecayArgs& a, const DecayPlan& p, hipStream_t stream) {
  return dtype == MAFAT_BF16 ? launch<MAFAT_BF16>(a, p, stream) : launch<MAFAT_F32>(a, p, stream);
}

}  // namespace mafat
