// cross_fast.h -- cross attention with keys and values of whole 16-byte pieces:
// the kernels for many rows and for few, in bfloat16 and float32 (see cross.hip
// for the scheme of the two products, and for anything else).
//
// Both fetch keys and values straight into LDS and run the same code on a
// wave's 32 rows (struct Rows).  Many rows are bound by arithmetic, so the
// waves of a block hold different rows and share every tile; few rows are
// bound by reading keys and values once, so the waves hold the same rows and
// every wave streams positions of its own.
#pragma once

#include <hip/hip_runtime.h>

#include "cross_device.h"

namespace mafat {
namespace {

// A row of keys or values takes PITCH bytes of LDS, of which position p holds
// the 16-byte piece p ^ swizzle(row).  Keys are read a row per lane, so the 16
// lanes that are served at a time (of 32 rows) get 16 different places of the
// banks.  bfloat16 values are read by the transposing read, 32 lanes at a time
// taking 64 bytes each of four rows in a row, which get four different quarters
// (two halves, of 128-byte rows); float32 values 32 lanes taking 128 bytes of a
// row, the other 32 those of the row four further on, which get the other half.
template <int DT, int DP>
struct Fast {
  using T = typename Elt<DT>::T;
  static constexpr int BYTES = DP * static_cast<int>(sizeof(T)), V = Tile<DT>::V;  // of a row; values of a piece
  static constexpr int PITCH = BYTES <= 128 ? 128 : BYTES <= 256 ? 256 : 512;
  static_assert(BYTES <= PITCH, "rows fit");
  static constexpr int PER = PITCH / 16;  // positions of a row
  static constexpr int ROWS = 64 / PER;   // rows of one wave's load
  static constexpr int SUBS = BYTES <= 256 ? 2 : 1;  // 32 keys each, of a tile of the kernel for many rows
  static __device__ __forceinline__ int key_swizzle(int row) { return PER == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int value_swizzle(int row) {
    if (DT == MAFAT_F32) return ((row >> 2) & 1) << 3;
    return PER == 8 ? ((row >> 1) & 1) << 2 : ((row & 3) << 2) | ((row >> 2) & 3);
  }
};

// 16 bytes per lane from byte `off` of a descriptor's range (zeros past it)
// straight into LDS, lane after lane from byte `to`.  As assembly, because the
// compiler waits for every such load that it knows of before the next
// transposing read of LDS, whatever they touch: the loads of the next tile
// would be waited for at once.  The load has no register result; the kernel
// waits for it itself (wait_vmcnt) before the barrier that hands the tile on.
__device__ __forceinline__ void load_to_lds(const u32x4& range, unsigned off, unsigned to) {
  // (the same in all lanes, which the compiler has to know)
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(range[i])));
  to = static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(to)));
  // (The load needs five wait states after a vector instruction that wrote its
  // descriptor, which the compiler does not count into assembly.  m0 is a
  // register that assembly cannot declare as overwritten, so it is put back.)
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(to), "v"(off), "s"(r)
               : "memory");
}
// A descriptor of `bytes` bytes from p, as four words.
__device__ __forceinline__ u32x4 range_of(const void* p, unsigned bytes) {
  const uint64_t b = reinterpret_cast<uint64_t>(p);
  return u32x4{static_cast<unsigned>(b), static_cast<unsigned>(b >> 32) & 0xffffu, bytes, 0x00020000u};
}
__device__ __forceinline__ unsigned lds_offset(const void* p) {
  return static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_ptr_t)p));
}

// The running maximum may lag by a factor of 2^8 of the sums before they are
// rescaled, all rows of a wave together (rescaling a softmax's sums only past a
// threshold is published; float32 has room for the factor, and the bfloat16
// exponentials keep their relative accuracy).  A row's last bits so depend on
// its wave's other rows.
constexpr float kLazy = 8.f;

// Bytes of a mask as bits.  A lane holds those of 64 positions, so a wave looks
// 4096 ahead with four loads a lane.
struct MaskBits {
  static constexpr int SPAN = 64 * 64;
  uint64_t mine;
  // Bits of the `n` (at most 64 used) bytes at p.
  static __device__ __forceinline__ uint64_t of(const unsigned char* p, int n) {
    uint64_t bits = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u32x4 v = load16(p + 16 * g, n - 16 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t set = (((v[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | v[i]) & 0x80808080u;  // bytes that are not zero
        bits |= static_cast<uint64_t>(((set >> 7) * 0x01020408u) >> 24 & 15u) << (16 * g + 4 * i);
      }
    }
    return bits;
  }
  __device__ __forceinline__ void fill(const unsigned char* mask, int from, int keys) {
    // (unsigned: a span may look past 2^31 positions)
    const uint32_t at = static_cast<uint32_t>(from) + 64 * (threadIdx.x & 63), all = static_cast<uint32_t>(keys);
    mine = at < all ? of(mask + at, static_cast<int>(all - at)) : 0;
  }
  // Of 64 positions from 64 g after the first.
  __device__ __forceinline__ uint64_t get(int g) const {
    const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(mine)), g));
    const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(mine >> 32)), g));
    return static_cast<uint64_t>(hi) << 32 | lo;
  }
};
// The first n of 64 bits.
__device__ __forceinline__ uint64_t first_bits(int n) { return n >= 64 ? ~uint64_t{0} : n <= 0 ? 0 : (uint64_t{1} << n) - 1; }

// One wave's 32 rows: their fragments, sums and statistics, and the work on a
// tile of 32 SUBS keys: scores, softmax, outputs.  FINE: the exponentials enter
// the second product as the sum of two bfloat16 parts, so that a small output
// keeps the accuracy of its sums (where matrix instructions are not what a
// kernel waits for); otherwise rounded to bfloat16, an error of the size of the
// output's own rounding.
template <int DT, int DP, int SUBS, bool FINE>
struct Rows {
  using F = Fast<DT, DP>;
  using T = typename F::T;
  static constexpr int PITCH = F::PITCH, V = F::V, NT = DP / 32, QT = DP / V / 2;
  u32x4 qf[QT];
  f32x16 acc[NT];
  f32x16 s[SUBS];                       // scores of the tile, key by register
  uint32_t pp[SUBS][8], pl[SUBS][8];    // their exponentials, and what rounding left of them (FINE)
  float most, sum;    // largest product so far that the sums are relative to; this lane's part of the sum
  float scale, lazy;
  int64_t row;
  int head;
  bool real;
  int k_at[QT], v_lo[NT], v_hi[NT];  // LDS offsets of the fragments

  __device__ __forceinline__ void start(const CrossArgs& a, const Place& at, int kv, int tile_row) {
    const int lane = static_cast<int>(threadIdx.x) & 63, c = lane & 31, h = lane >> 5;
    const int r = at.tile0 + tile_row + c, D = a.head_dim;
    real = r < at.tile_rows;
    const int rr = real ? r : at.tile_rows - 1;
    const int in_frame = static_cast<int>(static_cast<uint32_t>(rr) / static_cast<uint32_t>(a.group));
    row = at.row0 + in_frame;
    head = kv * a.group + rr - in_frame * a.group;
    // A negative scale goes into the rows' sign, so that the largest product has
    // the largest score.  (A scale of zero is not for this kernel: minus infinity
    // stands for masked keys and must not meet it.)
    const uint32_t flip = a.scale < 0.f ? (DT == MAFAT_BF16 ? 0x80008000u : 0x80000000u) : 0u;
    scale = a.scale < 0.f ? -a.scale : a.scale;
    // Finite for any scale: plus infinity would make no product larger than a
    // maximum of minus infinity, and the first key would not be taken for one.
    lazy = fminf(kLazy / scale, 0x1.fffffep127f);
    const T* q = static_cast<const T*>(a.q) + row * a.q_row + static_cast<int64_t>(head) * a.q_head;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int d = V * (2 * t + h);  // pieces are whole: head_dim is a multiple of V
      qf[t] = u32x4{0, 0, 0, 0};
      if (d < D) __builtin_memcpy(&qf[t], q + d, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) qf[t][i] ^= flip;
    }
    most = kNone;
    sum = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
    const int ksw = F::key_swizzle(c);  // of rows c and 32 + c alike
#pragma unroll
    for (int p = 0; p < QT; ++p) k_at[p] = c * PITCH + (((2 * p + h) ^ ksw) << 4);
    if constexpr (DT == MAFAT_BF16) {
      // The transposing read gives lane i of 16 column i of 4 rows, of which it
      // fetches 4 columns of row i / 4.  Rows 16 further on have the same swizzle.
      const int vr = 4 * h + ((lane & 15) >> 2);
      const int vp = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);  // 16-byte piece of a 64-byte quarter
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        v_lo[n] = vr * PITCH + (((4 * n + vp) ^ F::value_swizzle(vr)) << 4) + 8 * (lane & 1);
        v_hi[n] = (vr + 8) * PITCH + (((4 * n + vp) ^ F::value_swizzle(vr + 8)) << 4) + 8 * (lane & 1);
      }
    } else {
      // One value a lane, of the key that register i holds; all of a lane's keys have one swizzle.
#pragma unroll
      for (int n = 0; n < NT; ++n) v_lo[n] = 4 * h * PITCH + (((8 * n + (c >> 2)) ^ F::value_swizzle(4 * h)) << 4) + 4 * (c & 3);
    }
  }

  // Scores of the tile's keys.
  __device__ __forceinline__ void scores(const unsigned char* sk) {
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[sub][i] = 0.f;
#pragma unroll
      for (int p = 0; p < QT; ++p)
        Tile<DT>::mul(s[sub], *reinterpret_cast<const u32x4*>(sk + k_at[p] + sub * 32 * PITCH), qf[p]);
    }
  }

  // Exponentials of the scores of the keys in `ok` (a lane's own bits, or the
  // wave's); `all`: those are all keys, for every lane.
  __device__ __forceinline__ void softmax(uint64_t ok, bool all) {
    if (!all) {
      const int h = (static_cast<int>(threadIdx.x) & 63) >> 5;
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub) {
        const uint32_t bits = static_cast<uint32_t>(ok >> (32 * sub)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[sub][i] = (bits >> (8 * (i >> 2) + (i & 3))) & 1 ? s[sub][i] : kNone;
      }
    }
    float top = kNone;
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
      for (int i = 0; i < 16; i += 2) top = fmaxf(top, fmaxf(s[sub][i], s[sub][i + 1]));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    if (__builtin_amdgcn_ballot_w64(top > most + lazy)) {
      const float up = fmaxf(most, top);
      const float down = up == kNone ? 0.f : __builtin_amdgcn_exp2f((most - up) * scale);
      most = up;
      sum *= down;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[n][i] *= down;
    }
    // Past float32: minus infinity is no key yet (every exponential is zero),
    // plus infinity makes the row NaN, as infinity minus infinity would.
    const float high = most * scale, base = high == kNone ? 0.f : high + (high - high);
    float add = 0.f;
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(s[sub][2 * i], scale, -base));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s[sub][2 * i + 1], scale, -base));
        add += e0 + e1;
        if constexpr (DT == MAFAT_F32) {
          s[sub][2 * i] = e0;
          s[sub][2 * i + 1] = e1;
          continue;
        }
        pp[sub][i] = pack_bf16(e0, e1);
        if (FINE)
          pl[sub][i] = pack_bf16(e0 - __uint_as_float(pp[sub][i] << 16), e1 - __uint_as_float(pp[sub][i] & 0xffff0000u));
      }
    sum += add;
  }

  // Adds the exponentials times the tile's values.  CHOSEN: values of keys that
  // are not in `used` count as zeros whatever they hold.
  template <bool CHOSEN>
  __device__ __forceinline__ void outputs(const unsigned char* sv, uint64_t used) {
    const int h = (static_cast<int>(threadIdx.x) & 63) >> 5;
    if constexpr (DT == MAFAT_F32) {
#pragma unroll
      for (int sub = 0; sub < SUBS; ++sub) {
        const uint32_t bits = static_cast<uint32_t>(used >> (32 * sub)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float v = *reinterpret_cast<const float*>(sv + v_lo[n] + (32 * sub + key_of(i, 0)) * PITCH);
            if (CHOSEN) v = (bits >> key_of(i, 0)) & 1 ? v : 0.f;
            acc[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[sub][i], acc[n], 0, 0, 0);
          }
      }
      return;
    }
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 keep;
        if (CHOSEN) {
          const uint32_t bits = static_cast<uint32_t>(used >> (32 * sub + 16 * u)) >> (4 * h);
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // registers 2 i and 2 i + 1: keys 8 (i / 2) + 2 (i % 2) and the next
            const uint32_t two = bits >> (8 * (i >> 1) + 2 * (i & 1));
            keep[i] = ((two & 1) ? 0xffffu : 0u) | ((two & 2) ? 0xffff0000u : 0u);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const unsigned char* base = sv + (32 * sub + 16 * u) * PITCH;
          const s16x4 vf[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(base + v_lo[n])),
                               __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(base + v_hi[n]))};
          u32x4 v = __builtin_bit_cast(u32x4, vf);
          if (CHOSEN) v &= keep;
          Tile<MAFAT_BF16>::mul(acc[n], v, u32x4{pp[sub][4 * u], pp[sub][4 * u + 1], pp[sub][4 * u + 2], pp[sub][4 * u + 3]});
          if (FINE)
            Tile<MAFAT_BF16>::mul(acc[n], v, u32x4{pl[sub][4 * u], pl[sub][4 * u + 1], pl[sub][4 * u + 2], pl[sub][4 * u + 3]});
        }
      }
  }

  // Outputs, or this split's part of them, of the 32-wide tiles n0, n0 + step,
  // ... of the head; `sum` is the whole one by now.
  __device__ __forceinline__ void finish(const CrossArgs& a, int split, int n0, int step) {
    const int h = (static_cast<int>(threadIdx.x) & 63) >> 5, D = a.head_dim;
    if (!real) return;
    const float top = most * scale;
    if (a.splits > 1) {
      const int64_t pair = (static_cast<int64_t>(split) * a.rows + row) * a.q_heads + head;
      float* po = a.part + pair * D;
      float* stat = a.part + static_cast<int64_t>(a.splits) * a.rows * a.q_heads * D + pair * 2;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          if (n % step != n0) continue;
          const int d = 32 * n + 8 * g + 4 * h;
          const f32x4 v = {acc[n][4 * g], acc[n][4 * g + 1], acc[n][4 * g + 2], acc[n][4 * g + 3]};
          if (d < D) __builtin_memcpy(po + d, &v, 16);
        }
      if (h == 0 && n0 == 0) {
        stat[0] = top;
        stat[1] = sum;
      }
      return;
    }
    const float over = sum == 0.f ? 0.f : 1.f / sum;  // no key: zeros
    T* y = static_cast<T*>(a.y) + row * a.y_row + static_cast<int64_t>(head) * a.y_head;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (n % step != n0) continue;
        const int d = 32 * n + 8 * g + 4 * h;
        const f32x4 o = f32x4{acc[n][4 * g], acc[n][4 * g + 1], acc[n][4 * g + 2], acc[n][4 * g + 3]} * over;
        if (d < D) {
          if constexpr (DT == MAFAT_BF16) {
            const uint2 v = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
            __builtin_memcpy(y + d, &v, 8);
          } else {
            __builtin_memcpy(y + d, &o, 16);
          }
        }
      }
    if (a.lse && h == 0 && n0 == 0) a.lse[row * a.q_heads + head] = sum == 0.f ? kNone : (top + __log2f(sum)) * 0.6931471805599453f;
  }
};

// The descriptors and offsets of a wave's loads of KT keys (or values) at a
// time: LOADS loads of ROWS rows each, rows STRIDE * ROWS apart, from row
// ROWS * `start`.  Rows past the last key end outside of the descriptor, pieces
// past head_dim are put there.
template <int DT, int DP, int KT, int LOADS, int STRIDE>
struct Fetch {
  using F = Fast<DT, DP>;
  using T = typename F::T;
  static constexpr int ESZ = static_cast<int>(sizeof(T));
  const T* base;
  int pos, D, keys;
  unsigned off[LOADS];
  int row[LOADS];
  template <bool VALUES>
  __device__ __forceinline__ void start(const void* p, int64_t offset, int64_t stride, int head_dim, int n_keys, int start) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    base = static_cast<const T*>(p) + offset;
    pos = static_cast<int>(stride);
    D = head_dim;
    keys = n_keys;
#pragma unroll
    for (int g = 0; g < LOADS; ++g) {
      const int r = F::ROWS * (g * STRIDE + start) + lane / F::PER, p16 = lane % F::PER;
      const int d = F::V * (p16 ^ (VALUES ? F::value_swizzle(r) : F::key_swizzle(r)));
      row[g] = r;
      off[g] = d < D ? static_cast<unsigned>((r * pos + d) * ESZ) : 0x80000000u;
    }
  }
  // Tile t into LDS from byte `slot`.  CHOSEN: rows that are not in `ok` read as
  // zeros (what they hold must not reach a product, not even times zero).
  template <bool CHOSEN>
  __device__ __forceinline__ void issue(int t, unsigned slot, int start, uint64_t ok) const {
    const int64_t key0 = static_cast<int64_t>(t) * KT;
    const int n = min(KT, static_cast<int>(keys - key0));
    const u32x4 range = range_of(base + key0 * pos, static_cast<unsigned>(((n - 1) * pos + D) * ESZ));
#pragma unroll
    for (int g = 0; g < LOADS; ++g) {
      const unsigned bad = CHOSEN && !((ok >> row[g]) & 1) ? 0x80000000u : 0u;
      load_to_lds(range, off[g] | bad, slot + F::ROWS * (g * STRIDE + start) * F::PITCH);
    }
  }
};

// Many rows: NW waves of 32 rows, 64 keys at a time (32 of heads above 128,
// whose sums take half of the registers), fetched one tile ahead.
//
// Per 64 keys a wave spends 1024 cycles in matrix instructions (DP 128) and
// about as many on the vector ALUs, a third of them in the exponentials; its LDS
// reads take 128.  The largest score lags (kLazy), so the sums are seldom
// rescaled.  2 frames x 2048 rows x 16 heads of 128, 5776 positions: 195 us,
// 994 TFLOP/s, where a large bfloat16 product of the library reaches 1590; matrix
// instructions are busy 39 % of the time, at a clock that both bring down to 2.1 GHz.
// Scores, softmax and outputs of a tile follow each other in every wave, and a
// barrier a tile keeps the waves of a SIMD together, so the two kinds of work
// seldom overlap.  With a mask by key 212 us; by row 443 (a lane reads its own
// mask, and registers spill from heads of 96 on); heads of 256 with a mask by
// row spill 300 registers: 4.9 ms, where without a mask they take 0.59.
template <int DT, int DP, int MASK, int NW>
__global__ __launch_bounds__(64 * NW, 2) void cross_tile_kernel(const CrossArgs a) {
  using F = Fast<DT, DP>;
  constexpr int SUBS = F::SUBS;
  constexpr int KT = 32 * SUBS, HALF = KT * F::PITCH;  // slots: keys and values of even tiles, of odd tiles
  constexpr int LOADS = KT / F::ROWS / NW;
  static_assert(LOADS * F::ROWS * NW == KT, "whole loads per wave");
  __shared__ __align__(1024) unsigned char smem[4 * HALF];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  // head by head, so that the blocks that share keys and values share an XCD's cache
  const int id = xcd_remap(a.first_block + static_cast<int>(blockIdx.x), a.row_blocks * a.kv_heads);
  const int kv = static_cast<int>(static_cast<uint32_t>(id) / static_cast<uint32_t>(a.row_blocks));
  const Place at = find<32 * NW>(a, id - kv * a.row_blocks);
  if (!at.any) return;
  const int split = static_cast<int>(blockIdx.y);
  const int tiles = static_cast<int>((static_cast<uint32_t>(at.keys) + KT - 1) / KT);
  int first, last;
  part_of(tiles, split, a.splits, &first, &last);
  Fetch<DT, DP, KT, LOADS, NW> fk, fv;
  fk.template start<false>(a.k, at.frame * a.k_frame + kv * a.k_head, a.k_pos, a.head_dim, at.keys, wave);
  fv.template start<true>(a.v, at.frame * a.v_frame + kv * a.v_head, a.v_pos, a.head_dim, at.keys, wave);
  const unsigned base = lds_offset(smem);

  constexpr uint64_t ALL = SUBS == 2 ? ~uint64_t{0} : 0xffffffffu;
  Rows<DT, DP, SUBS, false> w;
  w.start(a, at, kv, 32 * wave);
  const unsigned char* mask = nullptr;
  if (MASK == MASK_KEYS) mask = a.mask + at.frame * a.mask_row;
  if (MASK == MASK_ROWS) mask = a.mask + w.row * a.mask_row;
  MaskBits bits;
  // Keys of tile t that may be read: of this lane's row, or of all.
  auto valid = [&](int t) -> uint64_t {
    const int left = at.keys - t * KT;
    if (MASK == MASK_KEYS) {
      const int g = (t - first) % (MaskBits::SPAN / KT);
      if (g == 0) bits.fill(mask, t * KT, at.keys);
      return SUBS == 2 ? bits.get(g) : bits.get(g >> 1) >> (32 * (g & 1)) & ALL;
    }
    if (MASK == MASK_ROWS) return MaskBits::of(mask + static_cast<int64_t>(t) * KT, min(KT, left));
    return first_bits(left) & ALL;
  };
  uint64_t ok = 0;
  if (first < last) {
    ok = valid(first);
    fk.template issue<false>(first, base + (first & 1) * 2 * HALF, wave, 0);
    fv.template issue<MASK == MASK_KEYS>(first, base + (first & 1) * 2 * HALF + HALF, wave, ok);
  }
  for (int t = first; t < last; ++t) {
    wait_vmcnt<0>();
    wg_barrier();  // tile t is there, and nobody reads the other slot any more
    const uint64_t now = ok;
    if (t + 1 < last) {
      ok = valid(t + 1);
      fk.template issue<false>(t + 1, base + ((t + 1) & 1) * 2 * HALF, wave, 0);
      fv.template issue<MASK == MASK_KEYS>(t + 1, base + ((t + 1) & 1) * 2 * HALF + HALF, wave, ok);
    }
    const unsigned char* slot = smem + (t & 1) * 2 * HALF;
    if constexpr (MASK == MASK_ROWS) {
      if (__builtin_amdgcn_ballot_w64(now != 0) == 0) continue;
      uint64_t any = now;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) any |= __shfl_xor(any, o, 64);
      w.scores(slot);
      w.softmax(now, __builtin_amdgcn_ballot_w64(now == ALL) == ~uint64_t{0});
      if (__builtin_amdgcn_ballot_w64(any == ALL) == ~uint64_t{0}) w.template outputs<false>(slot + HALF, 0);
      else w.template outputs<true>(slot + HALF, any);
    } else {
      if (MASK == MASK_KEYS && now == 0) continue;
      w.scores(slot);
      w.softmax(now, now == ALL);
      w.template outputs<false>(slot + HALF, 0);
    }
  }
  w.sum += __shfl_xor(w.sum, 32, 64);
  w.finish(a, split, 0, 1);
}

// Few rows: 32 rows for all waves of a block, each wave streaming 32 keys at a
// time of a part of its own through SLOTS slots of its own: no wave waits for
// another before the end, where the parts are joined in LDS.  The slots of a
// block take at most 67 KB, so that two blocks share a CU: their waves fetch
// while others compute, and a ragged call's blocks run in one round (8 frames,
// 64 rows, 8 heads of 128, up to 1444 positions: 11.6 us and
// 4.0 for the join; 4 rows, 64980 positions, 4 heads of 128 for 16: 97 us, 5.5 TB/s,
// the rate of a copy).
template <int DT, int DP, int MASK>
__global__ __launch_bounds__(64 * cross_few_waves(DT, DP), 1) void cross_few_kernel(const CrossArgs a) {
  using F = Fast<DT, DP>;
  constexpr int NW = cross_few_waves(DT, DP), SLOTS = F::PITCH <= 128 ? 2 : 1;
  constexpr int KT = 32, HALF = KT * F::PITCH, LOADS = KT / F::ROWS;
  constexpr int NT = DP / 32, JOIN = 32 * DP + 64;  // floats of a wave's part: sums, statistics of 32 rows
  static_assert((SLOTS - 1) * 2 * LOADS <= 63, "loads in flight that a wave can count");
  constexpr int RING = NW * SLOTS * 2 * HALF, LDS = RING > NW * JOIN * 4 ? RING : NW * JOIN * 4;
  __shared__ __align__(1024) unsigned char smem[LDS];
  const int lane = static_cast<int>(threadIdx.x) & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int id = xcd_remap(a.first_block + static_cast<int>(blockIdx.x), a.row_blocks * a.kv_heads);
  const int kv = static_cast<int>(static_cast<uint32_t>(id) / static_cast<uint32_t>(a.row_blocks));
  const Place at = find<32>(a, id - kv * a.row_blocks);
  if (!at.any) return;
  const int split = static_cast<int>(blockIdx.y);
  const int tiles = static_cast<int>((static_cast<uint32_t>(at.keys) + KT - 1) / KT);
  int first, last;
  part_of(tiles, split * NW + wave, a.splits * NW, &first, &last);
  Fetch<DT, DP, KT, LOADS, 1> fk, fv;
  fk.template start<false>(a.k, at.frame * a.k_frame + kv * a.k_head, a.k_pos, a.head_dim, at.keys, 0);
  fv.template start<true>(a.v, at.frame * a.v_frame + kv * a.v_head, a.v_pos, a.head_dim, at.keys, 0);
  unsigned char* const mine = smem + wave * (SLOTS * 2 * HALF);
  const unsigned base = lds_offset(mine);
  const unsigned char* mask = MASK == MASK_KEYS ? a.mask + at.frame * a.mask_row : nullptr;
  MaskBits bits;
  // Keys of tile t that may be read, as they are asked for tile after tile.
  auto valid = [&](int t) -> uint64_t {
    if (MASK == MASK_KEYS) {
      const int g = (t - first) % 128;
      if (g == 0) bits.fill(mask, t * KT, at.keys);
      return bits.get(g >> 1) >> (32 * (g & 1)) & 0xffffffffu;
    }
    return first_bits(at.keys - t * KT) & 0xffffffffu;
  };
  auto issue = [&](int t, uint64_t ok) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot's last reads are done
    const unsigned slot = base + (t & (SLOTS - 1)) * 2 * HALF;
    fk.template issue<false>(t, slot, 0, 0);
    fv.template issue<MASK == MASK_KEYS>(t, slot + HALF, 0, ok);
  };
  uint64_t ok[SLOTS];  // of the tiles in flight, the oldest first
#pragma unroll
  for (int p = 0; p < SLOTS - 1; ++p) {
    ok[p] = first + p < last ? valid(first + p) : 0;
    if (first + p < last) issue(first + p, ok[p]);
  }
  Rows<DT, DP, 1, DT == MAFAT_BF16> w;
  w.start(a, at, kv, 0);
  const unsigned char* own_mask = MASK == MASK_ROWS ? a.mask + w.row * a.mask_row : nullptr;
  for (int t = first; t < last; ++t) {
    ok[SLOTS - 1] = 0;
    if (t + SLOTS - 1 < last) {
      ok[SLOTS - 1] = valid(t + SLOTS - 1);
      issue(t + SLOTS - 1, ok[SLOTS - 1]);
    }
    wait_stage<2 * LOADS, SLOTS - 1>(last - 1 - t);
    const unsigned char* slot = mine + (t & (SLOTS - 1)) * 2 * HALF;
    uint64_t now = ok[0];
#pragma unroll
    for (int p = 0; p + 1 < SLOTS; ++p) ok[p] = ok[p + 1];
    if constexpr (MASK == MASK_ROWS) {
      now = MaskBits::of(own_mask + static_cast<int64_t>(t) * KT, min(KT, at.keys - t * KT));
      if (__builtin_amdgcn_ballot_w64(now != 0) == 0) continue;
      uint64_t any = now;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) any |= __shfl_xor(any, o, 64);
      w.scores(slot);
      w.softmax(now, __builtin_amdgcn_ballot_w64(now == 0xffffffffu) == ~uint64_t{0});
      w.template outputs<true>(slot + HALF, any);
    } else {
      if (MASK == MASK_KEYS && now == 0) continue;
      w.scores(slot);
      w.softmax(now, now == 0xffffffffu);
      w.template outputs<false>(slot + HALF, 0);
    }
  }
  w.sum += __shfl_xor(w.sum, 32, 64);

  // Join: every wave puts its part down and takes every NW-th 32-wide tile of the head.
  wait_vmcnt<0>();
  __syncthreads();
  float* const parts_at = reinterpret_cast<float*>(smem);
  {
    float* p = parts_at + wave * JOIN;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) p[(32 * n + key_of(i, h)) * 32 + c] = w.acc[n][i];
    if (h == 0) {
      p[32 * DP + c] = w.most;
      p[32 * DP + 32 + c] = w.sum;
    }
  }
  __syncthreads();
  float top = kNone;
#pragma unroll
  for (int v = 0; v < NW; ++v) top = fmaxf(top, parts_at[v * JOIN + 32 * DP + c]);
  float by[NW], sum = 0.f;
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    by[v] = top == kNone ? 0.f : __builtin_amdgcn_exp2f((parts_at[v * JOIN + 32 * DP + c] - top) * w.scale);
    sum = fmaf(parts_at[v * JOIN + 32 * DP + 32 + c], by[v], sum);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if (n % NW != wave) continue;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float o = 0.f;
#pragma unroll
      for (int v = 0; v < NW; ++v) o = fmaf(parts_at[v * JOIN + (32 * n + key_of(i, h)) * 32 + c], by[v], o);
      w.acc[n][i] = o;
    }
  }
  w.most = top;
  w.sum = sum;
  if (wave < NT) w.finish(a, split, wave, NW);
}

template <int DT, int DP, int NW>
void launch_tile(const CrossArgs& a, dim3 grid, hipStream_t stream) {
  if (!a.mask) hipLaunchKernelGGL((cross_tile_kernel<DT, DP, MASK_NONE, NW>), grid, dim3(64 * NW), 0, stream, a);
  else if (!a.mask_by_row) hipLaunchKernelGGL((cross_tile_kernel<DT, DP, MASK_KEYS, NW>), grid, dim3(64 * NW), 0, stream, a);
  else hipLaunchKernelGGL((cross_tile_kernel<DT, DP, MASK_ROWS, NW>), grid, dim3(64 * NW), 0, stream, a);
}

template <int DT, int DP>
hipError_t launch_fast(CrossArgs a, const CrossPlan& p, hipStream_t stream) {
  constexpr int FEW = 64 * cross_few_waves(DT, DP);
  a.row_blocks = static_cast<int32_t>(cross_row_blocks(a, p.few ? 32 : 32 * p.waves));
  return for_block_parts(static_cast<int64_t>(a.row_blocks) * a.kv_heads, [&](int32_t from, unsigned n) {
    a.first_block = from;
    const dim3 grid(n, static_cast<unsigned>(a.splits));
    if (p.few) {
      if (!a.mask) hipLaunchKernelGGL((cross_few_kernel<DT, DP, MASK_NONE>), grid, dim3(FEW), 0, stream, a);
      else if (!a.mask_by_row) hipLaunchKernelGGL((cross_few_kernel<DT, DP, MASK_KEYS>), grid, dim3(FEW), 0, stream, a);
      else hipLaunchKernelGGL((cross_few_kernel<DT, DP, MASK_ROWS>), grid, dim3(FEW), 0, stream, a);
    } else if (DP > 128 || p.waves == 8) {
      launch_tile<DT, DP, 8>(a, grid, stream);
    } else {
      launch_tile<DT, DP <= 128 ? DP : 128, 4>(a, grid, stream);
    }
  });
}

}  // namespace
}  // namespace mafat
