// cross.hip -- attention of query rows to the positions of the frames they
// are about.
//
//   s_j = scale q . k_j,  p_j = exp(s_j - max),  y = sum_j p_j v_j / sum_j p_j
//
// in one pass over the positions, with the largest score so far, the sum and
// the output's sums of every row held in float32 and rescaled when the largest
// score grows.  Scores are in base 2 (the scale carries log2(e)).
//
// The rows of a tile are the (query row, head) pairs of one frame that share a
// key/value head, so keys and values are read once for a whole group of heads
// and for all requests about the frame.  Both products run on 32x32 matrix
// instructions with the rows as columns:
//
//   S^T [key][row] = K Q^T      a lane: 16 keys of one row (and the lane 32
//                               further on the other 16 of the same row)
//   O^T [d][row]  += V^T P^T    a lane: sums of one row
//
// so a row's maximum takes one exchange between two lanes, rescaling is a
// multiplication by the lane's own factor, and the exponentials are the second
// product's B operand as they stand: the sum over keys may run in any order as
// long as V^T's fragment takes the same one.
#include <hip/hip_runtime.h>

#include "cross_device.h"

namespace mafat {
namespace {

// Any size, stride, alignment and type.  A block takes 64 rows and the
// positions of its split, 64 at a time through LDS: waves 0 and 1 (rows 0-31
// and 32-63) take the first 32 of them and waves 2 and 3 the others, and the
// two are joined at the end.  DP: head_dim rounded up; the values past it are
// zeros in LDS.  Bound by its loads, which go through registers and, unaligned,
// in small pieces: 4096 rows, 5776 positions and 16 heads of 127 take 1.40 ms
// (of 128, on cross_tile_kernel, 0.20), 64 rows of 8 frames of 1444 and 32/8 heads
// of 127 55 us (of 128 18).
constexpr int kRowTile = 64, kKeyTile = 64;

template <int DT, int DP>
struct AnyShape {
  using T = typename Elt<DT>::T;
  static constexpr int V = Tile<DT>::V;
  static constexpr int PIECES = DP / V;                       // of a row
  static constexpr int PITCH = DP * sizeof(T) + 16;           // bytes between LDS rows: 16 more spread the banks
  static constexpr int LDS = 2 * kKeyTile * PITCH;
  static constexpr int JOIN = kRowTile * (DP + 2) * 4;
  static constexpr int BYTES = LDS > JOIN ? LDS : JOIN;
};

template <int DT, int DP, int MASK>
__global__ __launch_bounds__(256) void cross_any_kernel(const CrossArgs a) {
  using S = AnyShape<DT, DP>;
  using T = typename S::T;
  constexpr int V = S::V, PIECES = S::PIECES, PITCH = S::PITCH, NT = DP / 32;
  __shared__ __align__(16) unsigned char smem[S::BYTES];
  unsigned char* const sk = smem;
  unsigned char* const sv = smem + kKeyTile * PITCH;
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int c = lane & 31, h = lane >> 5;
  const Place at = find<kRowTile>(a, a.first_block + static_cast<int>(blockIdx.x));
  if (!at.any) return;
  const int head0 = static_cast<int>(blockIdx.y) * a.group;
  const int split = static_cast<int>(blockIdx.z);
  const int D = a.head_dim;

  // This lane's row: pair r of the frame is query row r / group, head r % group.
  const int r = at.tile0 + 32 * (wave & 1) + c;
  const bool real = r < at.tile_rows;
  const int rr = real ? r : at.tile_rows - 1;
  const int in_frame = static_cast<int>(static_cast<uint32_t>(rr) / static_cast<uint32_t>(a.group));
  const int64_t row = at.row0 + in_frame;
  const int head = head0 + rr - in_frame * a.group;

  // Q^T fragments: piece t of lane half h holds values 2 V t + V h ...
  u32x4 qf[PIECES / 2];
  {
    const T* q = static_cast<const T*>(a.q) + row * a.q_row + static_cast<int64_t>(head) * a.q_head;
#pragma unroll
    for (int t = 0; t < PIECES / 2; ++t) {
      const int d = 2 * V * t + V * h;
      qf[t] = load16(q + d, D - d);
    }
  }
  f32x16 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
  float most = kNone, sum = 0.f;

  const int tiles = static_cast<int>((static_cast<uint32_t>(at.keys) + kKeyTile - 1) / kKeyTile);
  int first, last;
  part_of(tiles, split, a.splits, &first, &last);
  const T* kb = static_cast<const T*>(a.k) + at.frame * a.k_frame + static_cast<int64_t>(blockIdx.y) * a.k_head;
  const T* vb = static_cast<const T*>(a.v) + at.frame * a.v_frame + static_cast<int64_t>(blockIdx.y) * a.v_head;
  const unsigned char* frame_mask = MASK == MASK_KEYS ? a.mask + at.frame * a.mask_row : nullptr;
  const unsigned char* row_mask = MASK == MASK_ROWS ? a.mask + row * a.mask_row : frame_mask;

  for (int t = first; t < last; ++t) {
    const int key0 = t * kKeyTile;
    // A key that the length or the frame's mask excludes reads as zeros: what
    // it holds must not reach the second product, not even times zero.
    for (int e = tid; e < 2 * kKeyTile * PIECES; e += 256) {
      const int which = e / (kKeyTile * PIECES), f = e - which * (kKeyTile * PIECES);
      const int j = f / PIECES, d = (f - j * PIECES) * V, key = key0 + j;
      bool there = key < at.keys;
      if (MASK == MASK_KEYS && there) there = frame_mask[key] != 0;
      const T* src = which ? vb + key * a.v_pos : kb + key * a.k_pos;
      *reinterpret_cast<u32x4*>((which ? sv : sk) + j * PITCH + d * sizeof(T)) = load16(src + d, there ? D - d : 0);
    }
    __syncthreads();
    const int sub = 32 * (wave >> 1);  // this wave's keys of the tile
    if (key0 + sub < at.keys) {
      f32x16 s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int p = 0; p < PIECES / 2; ++p)
        Tile<DT>::mul(s, *reinterpret_cast<const u32x4*>(sk + (sub + c) * PITCH + (2 * p + h) * 16), qf[p]);
      float top = kNone;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + sub + key_of(i, h);
        bool ok = key < at.keys;
        if (MASK != MASK_NONE && ok) ok = row_mask[key] != 0;
        s[i] = ok ? s[i] * a.scale : kNone;
        top = fmaxf(top, s[i]);
      }
      top = fmaxf(most, fmaxf(top, __shfl_xor(top, 32, 64)));
      const float base = top == kNone ? 0.f : top;  // no key yet: every exponential is zero
      const float down = __builtin_amdgcn_exp2f(most - base);
      most = top;
      float add = 0.f;
      uint32_t used = 0;  // keys that some row of this wave reads
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (MASK == MASK_ROWS) {
          const uint64_t who = __builtin_amdgcn_ballot_w64(s[i] != kNone);
          used |= ((h ? static_cast<uint32_t>(who >> 32) : static_cast<uint32_t>(who)) != 0 ? 1u : 0u) << i;
        }
        s[i] = __builtin_amdgcn_exp2f(s[i] - base);
      }
      if constexpr (DT == MAFAT_BF16) {
        // Each exponential as the sum of two bfloat16 parts (see Rows in
        // cross_fast.h): matrix instructions are not what this kernel waits for.
        uint32_t pp[8], pl[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          add += s[2 * i] + s[2 * i + 1];  // as they are: the log-sum-exp is float32 whatever the second product takes
          pp[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
          pl[i] = pack_bf16(s[2 * i] - __uint_as_float(pp[i] << 16), s[2 * i + 1] - __uint_as_float(pp[i] & 0xffff0000u));
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[n][i] *= down;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            // V^T: this lane's column d = 32 n + lane % 32, keys in the order of
            // the exponentials' registers 8 u .. 8 u + 7.  The transposing read
            // gives lane i of 16 column i of 4 rows, of which lane i fetches 4
            // columns of row i / 4.
            const unsigned char* src = sv + (sub + 16 * u + 4 * h + ((lane & 15) >> 2)) * PITCH +
                                       (32 * n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
            s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(src));
            s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(src + 8 * PITCH));
            if (MASK == MASK_ROWS) {
              // a key that no row of this wave reads must not reach the product
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                lo[i] = (used >> (8 * u + i)) & 1 ? lo[i] : static_cast<short>(0);
                hi[i] = (used >> (8 * u + 4 + i)) & 1 ? hi[i] : static_cast<short>(0);
              }
            }
            const s16x4 vf[2] = {lo, hi};
            Tile<DT>::mul(acc[n], __builtin_bit_cast(u32x4, vf), u32x4{pp[4 * u], pp[4 * u + 1], pp[4 * u + 2], pp[4 * u + 3]});
            Tile<DT>::mul(acc[n], __builtin_bit_cast(u32x4, vf), u32x4{pl[4 * u], pl[4 * u + 1], pl[4 * u + 2], pl[4 * u + 3]});
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) add += s[i];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[n][i] *= down;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float vv = *reinterpret_cast<const float*>(sv + (sub + key_of(i, h)) * PITCH + (32 * n + c) * 4);
            if (MASK == MASK_ROWS) vv = (used >> i) & 1 ? vv : 0.f;
            acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(vv, s[i], acc[n], 0, 0, 0);
          }
        }
      }
      sum = sum * down + add;
    }
    __syncthreads();
  }
  sum += __shfl_xor(sum, 32, 64);

  // Waves 2 and 3 hand their part to waves 0 and 1.
  float* jo = reinterpret_cast<float*>(smem) + (wave & 1) * (32 * (DP + 2));
  if (wave >= 2) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) jo[(32 * n + key_of(i, h)) * 32 + c] = acc[n][i];
    if (h == 0) {
      jo[32 * DP + c] = most;
      jo[32 * DP + 32 + c] = sum;
    }
  }
  __syncthreads();
  if (wave >= 2) return;
  {
    const float most2 = jo[32 * DP + c], sum2 = jo[32 * DP + 32 + c];
    const float top = fmaxf(most, most2), base = top == kNone ? 0.f : top;
    const float w1 = __builtin_amdgcn_exp2f(most - base), w2 = __builtin_amdgcn_exp2f(most2 - base);
    most = top;
    sum = sum * w1 + sum2 * w2;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][i] = acc[n][i] * w1 + jo[(32 * n + key_of(i, h)) * 32 + c] * w2;
  }
  if (!real) return;
  if (a.splits > 1) {
    const int64_t at_pair = (static_cast<int64_t>(split) * a.rows + row) * a.q_heads + head;
    float* po = a.part + at_pair * D;
    float* stat = a.part + static_cast<int64_t>(a.splits) * a.rows * a.q_heads * D + at_pair * 2;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = 32 * n + key_of(i, h);
        if (d < D) po[d] = acc[n][i];
      }
    if (h == 0) {
      stat[0] = most;
      stat[1] = sum;
    }
    return;
  }
  const float over = sum == 0.f ? 0.f : 1.f / sum;  // no key: zeros
  T* y = static_cast<T*>(a.y) + row * a.y_row + static_cast<int64_t>(head) * a.y_head;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int d = 32 * n + key_of(i, h);
      if (d < D) store1(y + d, acc[n][i] * over);
    }
  if (a.lse && h == 0)
    a.lse[row * a.q_heads + head] = sum == 0.f ? kNone : (most + __log2f(sum)) * 0.6931471805599453f;
}

// Joins the splits' parts of a (query row, head) with W waves, each taking every
// W-th split: all four of a block where there are many splits, one where there
// are few (and then rather many pairs).  Bound by latency, so everything is
// asked for before anything is used: the parts of a wave's first four splits,
// and the statistics, of one split by each lane.
template <int DT, int W>
__global__ __launch_bounds__(256) void cross_join_kernel(const CrossArgs a) {
  using T = typename Elt<DT>::T;
  __shared__ float part[W > 1 ? W : 1][W > 1 ? 256 : 1];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int64_t pairs = static_cast<int64_t>(a.rows) * a.q_heads;
  const int64_t pair = W > 1 ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * 4 + wave;
  if (pair >= pairs) return;
  const int first = W > 1 ? wave : 0, D = a.head_dim;
  const float* stat = a.part + static_cast<int64_t>(a.splits) * pairs * D + pair * 2;
  const float* po = a.part + pair * D + lane;
  float v[4][4];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[j][k] = s0 + W * j < a.splits && lane + 64 * k < D ? po[(s0 + W * j) * pairs * D + 64 * k] : 0.f;
  };
  fetch(first);
  float most = kNone, sum = 0.f;
  if (lane < a.splits) {
    most = stat[lane * pairs * 2];
    sum = stat[lane * pairs * 2 + 1];
  }
  const int64_t row = static_cast<uint32_t>(pair) / static_cast<uint32_t>(a.q_heads);  // rows * q_heads < 2^31
  const int head = static_cast<int>(pair - row * a.q_heads);
  if (a.q_offsets) {
    // a row that no frame has is not written (its parts were not, either)
    const int lo = min(max(a.q_offsets[0], 0), a.rows), hi = min(max(a.q_offsets[a.frames], 0), a.rows);
    if (row < lo || row >= hi) return;
  }
  float top = most;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float weight = top == kNone ? 0.f : __builtin_amdgcn_exp2f(most - top);
  sum *= weight;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  float o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = first; s0 < a.splits; s0 += 4 * W) {
    if (s0 != first) fetch(s0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (s0 + W * j >= a.splits) break;
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), s0 + W * j));
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = fmaf(v[j][k], w, o[k]);
    }
  }
  const float over = sum == 0.f ? 0.f : 1.f / sum;  // no key: zeros
  T* y = static_cast<T*>(a.y) + row * a.y_row + static_cast<int64_t>(head) * a.y_head;
  if constexpr (W > 1) {
#pragma unroll
    for (int k = 0; k < 4; ++k) part[wave][lane + 64 * k] = o[k];
    __syncthreads();
    const int d = static_cast<int>(threadIdx.x);
    if (d < D) store1(y + d, ((part[0][d] + part[1][d]) + (part[2][d] + part[3][d])) * over);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 64 * k < D) store1(y + lane + 64 * k, o[k] * over);
  }
  if (a.lse && lane == 0 && first == 0)
    a.lse[pair] = sum == 0.f ? kNone : (top + __log2f(sum)) * 0.6931471805599453f;
}

template <int DT, int DP>
void launch_any(const CrossArgs& a, dim3 grid, hipStream_t stream) {
  if (!a.mask) hipLaunchKernelGGL((cross_any_kernel<DT, DP, MASK_NONE>), grid, dim3(256), 0, stream, a);
  else if (!a.mask_by_row) hipLaunchKernelGGL((cross_any_kernel<DT, DP, MASK_KEYS>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((cross_any_kernel<DT, DP, MASK_ROWS>), grid, dim3(256), 0, stream, a);
}

// Whole 16-byte pieces, offsets of a tile's 64 rows in 31 bits, heads whose
// sums fit the registers, and a scale other than zero (which cross_fast.h
// divides by; cross_any_kernel takes products that are not finite to NaN by it).
template <int DT>
bool fast(const CrossArgs& a) {
  constexpr int64_t esz = sizeof(typename Elt<DT>::T);
  const auto whole = [](const void* p, int64_t x, int64_t y, int64_t z) {
    return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(esz * (x | y | z))) & 15) == 0;
  };
  return a.scale != 0.f && a.head_dim * esz % 16 == 0 && (DT == MAFAT_BF16 || a.head_dim <= 128) &&
         a.k_pos < (1 << 22) && a.v_pos < (1 << 22) &&
         whole(a.k, a.k_frame, a.k_pos, a.k_head) && whole(a.v, a.v_frame, a.v_pos, a.v_head);
}

template <int DT>
hipError_t launch(const CrossArgs& a, const CrossPlan& p, hipStream_t stream) {
  hipError_t e;
  if (fast<DT>(a) && cross_row_blocks(a, 32) * a.kv_heads < (int64_t{1} << 31)) {
    e = DT == MAFAT_BF16 ? launch_cross_bf16(a, p, stream) : launch_cross_f32(a, p, stream);
  } else {
    const int64_t blocks = cross_row_blocks(a, kRowTile);
    if (blocks >= (int64_t{1} << 31)) return hipErrorInvalidValue;
    e = for_block_parts(blocks, [&](int32_t from, unsigned n) {
      CrossArgs p = a;
      p.first_block = from;
      const dim3 grid(n, static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.splits));
      if (a.head_dim <= 64) launch_any<DT, 64>(p, grid, stream);
      else if (a.head_dim <= 96) launch_any<DT, 96>(p, grid, stream);
      else if (a.head_dim <= 128) launch_any<DT, 128>(p, grid, stream);
      else launch_any<DT, 256>(p, grid, stream);
    });
  }
  if (e != hipSuccess || a.splits == 1) return e;
  const unsigned pairs = static_cast<unsigned>(a.rows) * static_cast<unsigned>(a.q_heads);
  if (a.splits > 8) hipLaunchKernelGGL((cross_join_kernel<DT, 4>), dim3(pairs), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((cross_join_kernel<DT, 1>), dim3((pairs + 3) / 4), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

int64_t cross_row_blocks(const CrossArgs& a, int tile) {
  const int64_t pairs = static_cast<int64_t>(a.rows) * a.group;
  if (a.q_offsets) return pairs / tile + a.frames;  // a frame's last tile may be short
  return a.frames * ((static_cast<int64_t>(a.rows / a.frames) * a.group + tile - 1) / tile);
}

CrossPlan plan_cross(const mafat_cross& c) {
  CrossPlan p{};
  p.splits = 1;
  p.waves = c.head_dim > 128 ? 8 : 4;
  if (c.rows < 1 || c.positions < 1) return p;
  const int64_t pairs = (c.rows + c.frames - 1) / c.frames * (c.q_heads / c.kv_heads);  // of a frame, if they are alike
  const int64_t each = static_cast<int64_t>(c.frames) * c.kv_heads;
  const auto blocks = [&](int64_t tile) { return each * ((pairs + tile - 1) / tile); };
  int64_t want, least;  // blocks that fill the GPU; positions that a split is worth
  if (pairs <= 64) {
    p.few = 1;
    // A block a CU; two where each still streams 512 positions.
    want = 256 / blocks(32);
    if (want > 0 && c.positions / want >= 1024) want *= 2;
    least = 64 * cross_few_waves(c.dtype, c.head_dim);
  } else {
    if (blocks(256) >= 256) p.waves = 8;
    want = (p.waves == 8 ? 256 : 512) / blocks(32 * p.waves);
    least = c.dtype == MAFAT_BF16 ? 256 : 64;  // float32 products take eight times as long
  }
  int64_t n = (c.positions + least - 1) / least;
  if (n > want) n = want;
  p.splits = n < 1 ? 1 : n > kMaxCrossSplits ? kMaxCrossSplits : static_cast<int>(n);
  return p;
}

hipError_t launch_cross(int dtype, const CrossArgs& a, const CrossPlan& p, hipStream_t stream) {
  return dtype == MAFAT_BF16 ? launch<MAFAT_BF16>(a, p, stream) : launch<MAFAT_F32>(a, p, stream);
}

}  // namespace mafat
