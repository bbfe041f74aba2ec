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

#include "device_util.h"
#include "reader.h"

namespace mafat {
namespace {

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
  if (!a.q_offsets) {
    const int per = a.rows / a.frames, blocks = static_cast<int>((static_cast<int64_t>(per) * a.group + RT - 1) / RT);
    p.frame = b / blocks;
    p.row0 = p.frame * per;
    p.tile0 = (b - p.frame * blocks) * RT;
    p.tile_rows = per * a.group;
    p.any = p.frame < a.frames;
  } else {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    int before = 0;
    p.any = false;
    for (int f0 = 0; f0 < a.frames; f0 += 64) {
      const int f = f0 + lane;
      int lo = 0, n = 0;
      if (f < a.frames) {
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
        p.tile_rows = __builtin_amdgcn_readlane(pairs, l);
        p.tile0 = (b - __builtin_amdgcn_readlane(from, l)) * RT;
        p.any = true;
        break;
      }
      before = static_cast<int>(static_cast<uint32_t>(before) + static_cast<uint32_t>(__builtin_amdgcn_readlane(upto, 63)));
    }
  }
  p.keys = 0;
  if (p.any) p.keys = a.k_lengths ? min(max(a.k_lengths[p.frame], 0), a.positions) : a.positions;
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

// Any size, stride, alignment and type.  A block takes 64 rows and the
// positions of its split, 64 at a time through LDS: waves 0 and 1 (rows 0-31
// and 32-63) take the first 32 of them and waves 2 and 3 the others, and the
// two are joined at the end.  DP: head_dim rounded up; the values past it are
// zeros in LDS.
constexpr int kRowTile = 64, kKeyTile = 64;
enum { MASK_NONE = 0, MASK_KEYS = 1, MASK_ROWS = 2 };

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
  const Place at = find<kRowTile>(a, static_cast<int>(blockIdx.x));
  if (!at.any) return;
  const int head0 = static_cast<int>(blockIdx.y) * a.group;
  const int split = static_cast<int>(blockIdx.z);
  const int D = a.head_dim;

  // This lane's row: pair r of the frame is query row r / group, head r % group.
  const int r = at.tile0 + 32 * (wave & 1) + c;
  const bool real = r < at.tile_rows;
  const int rr = real ? r : at.tile_rows - 1;
  const int64_t row = at.row0 + rr / a.group;
  const int head = head0 + rr % a.group;

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

  const int tiles = (at.keys + kKeyTile - 1) / kKeyTile;
  const int first = static_cast<int>(static_cast<int64_t>(tiles) * split / a.splits);
  const int last = static_cast<int>(static_cast<int64_t>(tiles) * (split + 1) / a.splits);
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
        uint32_t pp[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          pp[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
          // the sum is that of the rounded values: what is divided is what was added up
          add += __uint_as_float(pp[i] << 16) + __uint_as_float(pp[i] & 0xffff0000u);
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

// Joins the splits' parts: one wave per (query row, head).
template <int DT>
__global__ __launch_bounds__(256) void cross_join_kernel(const CrossArgs a) {
  using T = typename Elt<DT>::T;
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int64_t pairs = static_cast<int64_t>(a.rows) * a.q_heads;
  const int64_t pair = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (pair >= pairs) return;
  const int64_t row = pair / a.q_heads;
  const int head = static_cast<int>(pair - row * a.q_heads);
  if (a.q_offsets) {
    // a row that no frame has is not written (its parts were not, either)
    const int lo = min(max(a.q_offsets[0], 0), a.rows), hi = min(max(a.q_offsets[a.frames], 0), a.rows);
    if (row < lo || row >= hi) return;
  }
  const float* stat = a.part + static_cast<int64_t>(a.splits) * pairs * a.head_dim + pair * 2;
  float top = kNone;
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, stat[s * pairs * 2]);
  const float base = top == kNone ? 0.f : top;
  float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s) {
    const float w = __builtin_amdgcn_exp2f(stat[s * pairs * 2] - base);
    sum = fmaf(stat[s * pairs * 2 + 1], w, sum);
    const float* po = a.part + (s * pairs + pair) * a.head_dim;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 64 * k < a.head_dim) o[k] = fmaf(po[lane + 64 * k], w, o[k]);
  }
  const float over = sum == 0.f ? 0.f : 1.f / sum;
  T* y = static_cast<T*>(a.y) + row * a.y_row + static_cast<int64_t>(head) * a.y_head;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (lane + 64 * k < a.head_dim) store1(y + lane + 64 * k, o[k] * over);
  if (a.lse && lane == 0)
    a.lse[pair] = sum == 0.f ? kNone : (top + __log2f(sum)) * 0.6931471805599453f;
}

template <int DT, int DP>
void launch_any(const CrossArgs& a, dim3 grid, hipStream_t stream) {
  if (!a.mask) hipLaunchKernelGGL((cross_any_kernel<DT, DP, MASK_NONE>), grid, dim3(256), 0, stream, a);
  else if (!a.mask_by_row) hipLaunchKernelGGL((cross_any_kernel<DT, DP, MASK_KEYS>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((cross_any_kernel<DT, DP, MASK_ROWS>), grid, dim3(256), 0, stream, a);
}

template <int DT>
hipError_t launch(const CrossArgs& args, hipStream_t stream) {
  CrossArgs a = args;
  const int64_t pairs = static_cast<int64_t>(a.rows) * a.group;
  int64_t blocks;
  if (a.q_offsets) blocks = pairs / kRowTile + a.frames;  // a frame's last tile may be short
  else blocks = a.frames * ((static_cast<int64_t>(a.rows / a.frames) * a.group + kRowTile - 1) / kRowTile);
  if (blocks >= (int64_t{1} << 31)) return hipErrorInvalidValue;
  a.row_blocks = static_cast<int32_t>(blocks);
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.splits));
  if (a.head_dim <= 64) launch_any<DT, 64>(a, grid, stream);
  else if (a.head_dim <= 128) launch_any<DT, 128>(a, grid, stream);
  else launch_any<DT, 256>(a, grid, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t all = static_cast<int64_t>(a.rows) * a.q_heads;
  hipLaunchKernelGGL((cross_join_kernel<DT>), dim3(static_cast<unsigned>((all + 3) / 4)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

int cross_splits(const mafat_cross& c) {
  if (c.rows < 1 || c.positions < 1) return 1;
  const int64_t group = c.q_heads / c.kv_heads;
  const int64_t per = (c.rows + c.frames - 1) / c.frames;  // rows of a frame, if they are alike
  const int64_t blocks = c.frames * ((per * group + kRowTile - 1) / kRowTile) * c.kv_heads;
  const int64_t tiles = (c.positions + kKeyTile - 1) / kKeyTile;
  int64_t n = 512 / blocks;
  if (n > (tiles + 1) / 2) n = (tiles + 1) / 2;
  return n < 1 ? 1 : n > 64 ? 64 : static_cast<int>(n);
}

hipError_t launch_cross(int dtype, const CrossArgs& a, hipStream_t stream) {
  return dtype == MAFAT_BF16 ? launch<MAFAT_BF16>(a, stream) : launch<MAFAT_F32>(a, stream);
}

}  // namespace mafat
