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

#ifndef MAFAT_CROSS_R
#define MAFAT_CROSS_R 1
#define MAFAT_CROSS_NW 4
#endif

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

// ---------------------------------------------------------------- bfloat16, whole 16-byte pieces
//
// Keys and values go straight into LDS, fetched one tile ahead.  A row of
// either takes PITCH bytes there (128, 256 or 512), of which position p holds
// the 16-byte piece p ^ swizzle(row): keys are read a row per lane, so the 16
// lanes that are served at a time (of 32 rows) get 16 different places of the
// banks; values are read by the transposing read, 32 lanes at a time taking 64
// bytes each of four rows in a row, which get four different quarters (two
// halves, of 128-byte rows).
template <int DP>
struct Fast {
  static constexpr int PITCH = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;
  static constexpr int PER = PITCH / 16;             // positions of a row
  static constexpr int ROWS = 64 / PER > 0 ? 64 / PER : 1;  // rows of one wave's load
  static __device__ __forceinline__ int key_swizzle(int row) { return PER == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int value_swizzle(int row) {
    return PER == 8 ? ((row >> 1) & 1) << 2 : ((row & 3) << 2) | ((row >> 2) & 3);
  }
};

constexpr float kLazy = 8.f;  // the running maximum may lag by a factor of 2^8 of the sums before they are rescaled

// Many rows: NW waves of 32 R rows each, 64 keys at a time.
//
// Per 64 keys and 32 rows a wave spends 1024 cycles in matrix instructions (DP
// 128), about as many on the vector ALUs (of those half in the exponentials),
// and reads 32 KB from LDS, a quarter of which the CU gets through in the same
// time.
template <int DP, int R, int NW, bool SOME>
__global__ __launch_bounds__(64 * NW) void cross_tile_kernel(const CrossArgs a) {
  using F = Fast<DP>;
  constexpr int PITCH = F::PITCH, PER = F::PER, NT = DP / 32, QT = DP / 16;
  constexpr int KT = 64, HALF = KT * PITCH, SLOT = 2 * HALF;
  constexpr int LOADS = KT / F::ROWS / NW;  // of a wave, for keys and for values
  constexpr int RT = 32 * R * NW;
  static_assert(LOADS * F::ROWS * NW == KT, "whole loads per wave");
  __shared__ __align__(1024) unsigned char smem[2 * SLOT];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int c = lane & 31, h = lane >> 5;
  // head by head, so that the blocks that share keys and values share an XCD's cache
  const int id = xcd_remap(static_cast<int>(blockIdx.x), a.row_blocks * a.kv_heads);
  const int kv = id / a.row_blocks;
  const Place at = find<RT>(a, id - kv * a.row_blocks);
  if (!at.any) return;
  const int split = static_cast<int>(blockIdx.y);
  const int D = a.head_dim;
  const uint16_t* kb = static_cast<const uint16_t*>(a.k) + at.frame * a.k_frame + kv * a.k_head;
  const uint16_t* vb = static_cast<const uint16_t*>(a.v) + at.frame * a.v_frame + kv * a.v_head;
  const unsigned char* mask = SOME && a.mask ? a.mask + at.frame * a.mask_row : nullptr;
  const int tiles = (at.keys + KT - 1) / KT;
  const int first = static_cast<int>(static_cast<int64_t>(tiles) * split / a.splits);
  const int last = static_cast<int>(static_cast<int64_t>(tiles) * (split + 1) / a.splits);

  // This lane's loads: of tile row r = ROWS (g NW + wave) + lane / PER, position
  // lane % PER.  Rows past the last key end outside of the descriptor, pieces
  // past head_dim are put there.
  int lr[LOADS];
  unsigned ko[LOADS], vo[LOADS];
#pragma unroll
  for (int g = 0; g < LOADS; ++g) {
    const int r = F::ROWS * (g * NW + wave) + lane / PER, p = lane % PER;
    const int kd = 8 * (p ^ F::key_swizzle(r)), vd = 8 * (p ^ F::value_swizzle(r));
    lr[g] = r;
    ko[g] = kd < D ? static_cast<unsigned>((r * static_cast<int>(a.k_pos) + kd) * 2) : 0x80000000u;
    vo[g] = vd < D ? static_cast<unsigned>((r * static_cast<int>(a.v_pos) + vd) * 2) : 0x80000000u;
  }
  // Keys of tile t that may be read, as bits.
  auto valid = [&](int t) -> uint64_t {
    const int key = t * KT + lane;
    bool ok = key < at.keys;
    if (SOME && mask && ok) ok = mask[key] != 0;
    return __builtin_amdgcn_ballot_w64(ok);
  };
  auto issue = [&](int t, uint64_t ok) {
    unsigned char* slot = smem + (t & 1) * SLOT;
    const int key0 = t * KT, n = min(KT, at.keys - key0);
    const __amdgpu_buffer_rsrc_t rk =
        make_rsrc(kb + key0 * a.k_pos, static_cast<unsigned>(((n - 1) * static_cast<int>(a.k_pos) + D) * 2));
    const __amdgpu_buffer_rsrc_t rv =
        make_rsrc(vb + key0 * a.v_pos, static_cast<unsigned>(((n - 1) * static_cast<int>(a.v_pos) + D) * 2));
#pragma unroll
    for (int g = 0; g < LOADS; ++g)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_ptr_t)(slot + F::ROWS * (g * NW + wave) * PITCH), 16,
                                               static_cast<int>(ko[g]), 0, 0, 0);
    // values of keys that the mask excludes read as zeros: what they hold must
    // not reach the second product, not even times zero
#pragma unroll
    for (int g = 0; g < LOADS; ++g) {
      const unsigned bad = SOME && !((ok >> lr[g]) & 1) ? 0x80000000u : 0u;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_ptr_t)(slot + HALF + F::ROWS * (g * NW + wave) * PITCH), 16,
                                               static_cast<int>(vo[g] | bad), 0, 0, 0);
    }
  };

  int64_t row[R];
  int head[R];
  bool real[R];
  u32x4 qf[R][QT];
  uint64_t ok = 0;
  if (first < last) {
    ok = valid(first);
    issue(first, ok);
  }
  // A negative scale goes into the rows' sign, so that the largest product has
  // the largest score; a scale of zero makes them zero (minus infinity stands
  // for masked keys and must not meet it).
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : ~0u;
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale);
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int r = at.tile0 + 32 * (wave * R + j) + c;
    real[j] = r < at.tile_rows;
    const int rr = real[j] ? r : at.tile_rows - 1;
    row[j] = at.row0 + rr / a.group;
    head[j] = kv * a.group + rr % a.group;
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + row[j] * a.q_row + static_cast<int64_t>(head[j]) * a.q_head;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int d = 16 * t + 8 * h;
      qf[j][t] = load16(q + d, D - d);
#pragma unroll
      for (int i = 0; i < 4; ++i) qf[j][t][i] = (qf[j][t][i] ^ flip) & keep;
    }
  }
  f32x16 acc[R][NT];
  float most[R], sum[R];  // largest product so far that the sums are relative to; this lane's part of the sum
#pragma unroll
  for (int j = 0; j < R; ++j) {
    most[j] = kNone;
    sum[j] = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][n][i] = 0.f;
  }
  const int ksw = F::key_swizzle(c);  // of rows c and 32 + c alike
  const int vrow = 4 * h + ((lane & 15) >> 2);
  const int vcol = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);  // 16-byte piece within a 64-byte quarter
  const float lazy = kLazy / scale;

  for (int t = first; t < last; ++t) {
    wait_vmcnt<0>();
    wg_barrier();  // tile t is there, and nobody reads the other slot any more
    uint64_t next = 0;
    if (t + 1 < last) {
      next = valid(t + 1);
      issue(t + 1, next);
    }
    const unsigned char* sk = smem + (t & 1) * SLOT;
    const unsigned char* sv = sk + HALF;
    const uint64_t now = ok;
    ok = next;
    if (SOME && now == 0) continue;  // the same for all waves
    f32x16 s[R][2];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
      for (int j = 0; j < R; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[j][sub][i] = 0.f;
#pragma unroll
      for (int p = 0; p < QT; ++p) {
        const u32x4 kf = *reinterpret_cast<const u32x4*>(sk + (32 * sub + c) * PITCH + (((2 * p + h) ^ ksw) << 4));
#pragma unroll
        for (int j = 0; j < R; ++j) Tile<MAFAT_BF16>::mul(s[j][sub], kf, qf[j][p]);
      }
    }
    if (now != ~uint64_t{0}) {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const uint32_t bits = static_cast<uint32_t>(now >> (32 * sub)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int j = 0; j < R; ++j)
            s[j][sub][i] = (bits >> (8 * (i >> 2) + (i & 3))) & 1 ? s[j][sub][i] : kNone;
      }
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      float top = kNone;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(s[j][sub][i], s[j][sub][i + 1]));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      if (__builtin_amdgcn_ballot_w64(top > most[j] + lazy)) {
        const float up = fmaxf(most[j], top);
        const float down = up == kNone ? 0.f : __builtin_amdgcn_exp2f((most[j] - up) * scale);
        most[j] = up;
        sum[j] *= down;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[j][n][i] *= down;
      }
    }
    uint32_t pp[R][2][8];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const float base = most[j] == kNone ? 0.f : most[j] * scale;
      float add = 0.f;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float e0 = __builtin_amdgcn_exp2f(fmaf(s[j][sub][2 * i], scale, -base));
          const float e1 = __builtin_amdgcn_exp2f(fmaf(s[j][sub][2 * i + 1], scale, -base));
          add += e0 + e1;
          pp[j][sub][i] = pack_bf16(e0, e1);
        }
      sum[j] += add;
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int r = 32 * sub + 16 * u + vrow;  // and eight further on: the swizzles differ
          const int piece = 4 * n + vcol;
          const unsigned char* lo_at = sv + r * PITCH + ((piece ^ F::value_swizzle(r)) << 4) + 8 * (lane & 1);
          const unsigned char* hi_at = sv + (r + 8) * PITCH + ((piece ^ F::value_swizzle(r + 8)) << 4) + 8 * (lane & 1);
          const s16x4 vf[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(lo_at)),
                               __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(hi_at))};
#pragma unroll
          for (int j = 0; j < R; ++j)
            Tile<MAFAT_BF16>::mul(acc[j][n], __builtin_bit_cast(u32x4, vf),
                                  u32x4{pp[j][sub][4 * u], pp[j][sub][4 * u + 1], pp[j][sub][4 * u + 2], pp[j][sub][4 * u + 3]});
        }
  }

#pragma unroll
  for (int j = 0; j < R; ++j) {
    sum[j] += __shfl_xor(sum[j], 32, 64);
    if (!real[j]) continue;
    const float top = most[j] == kNone ? kNone : most[j] * scale;
    if (a.splits > 1) {
      const int64_t pair = (static_cast<int64_t>(split) * a.rows + row[j]) * a.q_heads + head[j];
      float* po = a.part + pair * D;
      float* stat = a.part + static_cast<int64_t>(a.splits) * a.rows * a.q_heads * D + pair * 2;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int d = 32 * n + 8 * g + 4 * h;
          const f32x4 part4 = {acc[j][n][4 * g], acc[j][n][4 * g + 1], acc[j][n][4 * g + 2], acc[j][n][4 * g + 3]};
          if (d < D) __builtin_memcpy(po + d, &part4, 16);
        }
      if (h == 0) {
        stat[0] = top;
        stat[1] = sum[j];
      }
      continue;
    }
    const float over = sum[j] == 0.f ? 0.f : 1.f / sum[j];  // no key: zeros
    uint16_t* y = static_cast<uint16_t*>(a.y) + row[j] * a.y_row + static_cast<int64_t>(head[j]) * a.y_head;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * n + 8 * g + 4 * h;
        if (d < D) {
          const uint2 v = {pack_bf16(acc[j][n][4 * g] * over, acc[j][n][4 * g + 1] * over),
                           pack_bf16(acc[j][n][4 * g + 2] * over, acc[j][n][4 * g + 3] * over)};
          __builtin_memcpy(y + d, &v, 8);
        }
      }
    if (a.lse && h == 0)
      a.lse[row[j] * a.q_heads + head[j]] = sum[j] == 0.f ? kNone : (top + __log2f(sum[j])) * 0.6931471805599453f;
  }
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

// Blocks of `tile` rows of all frames together, at most.
int64_t row_blocks(const CrossArgs& a, int tile) {
  const int64_t pairs = static_cast<int64_t>(a.rows) * a.group;
  if (a.q_offsets) return pairs / tile + a.frames;  // a frame's last tile may be short
  return a.frames * ((static_cast<int64_t>(a.rows / a.frames) * a.group + tile - 1) / tile);
}

template <int DP>
hipError_t launch_tile(const CrossArgs& args, hipStream_t stream) {
  constexpr int R = MAFAT_CROSS_R, NW = MAFAT_CROSS_NW;
  CrossArgs a = args;
  a.row_blocks = static_cast<int32_t>(row_blocks(a, 32 * R * NW));
  const dim3 grid(static_cast<unsigned>(a.row_blocks) * static_cast<unsigned>(a.kv_heads), static_cast<unsigned>(a.splits));
  if (a.mask) hipLaunchKernelGGL((cross_tile_kernel<DP, R, NW, true>), grid, dim3(64 * NW), 0, stream, a);
  else hipLaunchKernelGGL((cross_tile_kernel<DP, R, NW, false>), grid, dim3(64 * NW), 0, stream, a);
  return hipGetLastError();
}

// Whole 16-byte pieces, offsets of a tile's 64 rows in 31 bits, and no mask of its own for every row.
bool fast(const CrossArgs& a) {
  const auto whole = [](const void* p, int64_t x, int64_t y, int64_t z) {
    return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(2 * (x | y | z))) & 15) == 0;
  };
  return a.head_dim % 8 == 0 && a.k_pos < (1 << 23) && a.v_pos < (1 << 23) && whole(a.k, a.k_frame, a.k_pos, a.k_head) &&
         whole(a.v, a.v_frame, a.v_pos, a.v_head) && !(a.mask && a.mask_by_row);
}

template <int DT>
hipError_t launch(const CrossArgs& args, hipStream_t stream) {
  CrossArgs a = args;
  if constexpr (DT == MAFAT_BF16) {
    if (fast(a) && row_blocks(a, 32) * a.kv_heads < (int64_t{1} << 31) && a.splits == 1) {
      if (a.head_dim <= 64) return launch_tile<64>(a, stream);
      if (a.head_dim <= 128) return launch_tile<128>(a, stream);
    }
  }
  const int64_t blocks = row_blocks(a, kRowTile);
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
