// linear.hip -- projection of 8-bit rows by 8-bit weights, with low-rank
// adapters beside it.
//
//   y[i][j] = xs[i] ws[j] sum_k x[i][k] w[j][k] + bias[j] + sum_r u[i][r] b[a(i)][j][r]
//   u[i][r] = factor[a(i)] xs[i] sum_k x[i][k] a[a(i)][r][k]
//
// Two launches with adapters: u first (shrink_*), as two bfloat16 parts, then
// the product, whose epilogue adds the adapters.  The weights are the matrix
// instructions' A operand and the rows of x their B operand, so a lane ends up
// with consecutive output columns of one row of y.  Both operands are read
// along k and take it in the same order, so any order of k within an
// instruction will do: a lane takes 16-byte pieces.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "reader.h"

namespace mafat {
namespace {

// More rows than this take u on the matrix cores.
constexpr int64_t kShrinkRows = 64;

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ i32x8 pair8(const u32x4& lo, const u32x4& hi) {
  const u32x4 v[2] = {lo, hi};
  return __builtin_bit_cast(i32x8, v);
}

// c += a b^T over 128 k on 16 x 16 outputs, both operands e4m3.
__device__ __forceinline__ void mma8_16(f32x4& c, const i32x8& a, const i32x8& b) {
  c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// 16 bytes at p, of which `n` may be read (the rest are zero); p need not be
// aligned.  WHOLE: n is a multiple of 16 or negative.
template <bool WHOLE>
__device__ __forceinline__ u32x4 load16(const unsigned char* p, int n) {
  u32x4 v = {0, 0, 0, 0};
  if (n >= 16) {
    __builtin_memcpy(&v, p, 16);
  } else if (!WHOLE) {
    unsigned char t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = i < n ? p[i] : 0;
    __builtin_memcpy(&v, t, 16);
  }
  return v;
}

// Up to 8 bfloat16 values at p, `n` of which are there (the rest are zero), for
// rows of an adapter's matrix: ranks that are no multiple of 8 are rare, and
// their ends are put together one by one.
__device__ __forceinline__ u32x4 load_rank8(const uint16_t* p, int n) {
  u32x4 v = {0, 0, 0, 0};
  if (n >= 8) {
    __builtin_memcpy(&v, p, 16);
  } else if (n > 0) {
    uint64_t lo = 0, hi = 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const uint64_t e = static_cast<uint64_t>(p[i]) << (16 * (i & 3));
      if (i < 4) lo |= e;
      else hi |= e;
    }
    v = u32x4{static_cast<unsigned>(lo), static_cast<unsigned>(lo >> 32), static_cast<unsigned>(hi), static_cast<unsigned>(hi >> 32)};
  }
  return v;
}
// v as the sum of two bfloat16 parts (16 bits of it), to u and `pad` further on.
__device__ __forceinline__ void put_parts(uint16_t* u, int pad, float v) {
  const __bf16 hi = static_cast<__bf16>(v);
  store1(u, v);
  store1(u + pad, v - static_cast<float>(hi));
}

// The outputs of a block of 16 columns by 16 MT rows: one per thread and step,
// column n0 + e % 16 of row m0 + e / 16.  What does not depend on the product,
// the scale and what is added to it, is worked out first (start), while the
// product's loads are under way.
template <int MT, int NW>
struct FewOutputs {
  static constexpr int STEPS = (256 * MT + 64 * NW - 1) / (64 * NW);
  float scale[STEPS], add[STEPS];
  __device__ __forceinline__ void start(const LinearArgs& a, int n0, int64_t m0) {
    int ad[STEPS];
    float bias[STEPS];
    // places past the end repeat the last row or column; what they get is not stored
    const auto place = [&](int k, int64_t* m, int* j) {
      const int e = static_cast<int>(threadIdx.x) + 64 * NW * k;
      *m = min(m0 + (e >> 4), a.rows - 1);
      *j = min(n0 + (e & 15), a.out_cols - 1);
    };
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      int64_t m;
      int j;
      place(k, &m, &j);
      ad[k] = a.count ? a.of_row[m] : -1;
      scale[k] = a.x_scale[m] * a.w_scale[j];
      bias[k] = a.bias ? a.bias[j] : 0.f;
      add[k] = 0.f;
    }
    // sum_r u[r] b[r]: of eight ranks, everything for all places before its first use
    for (int r = 0; a.count && r < a.rank; r += 8) {
      u32x4 hi[STEPS], lo[STEPS], bv[STEPS];
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        int64_t m;
        int j;
        place(k, &m, &j);
        hi[k] = lo[k] = bv[k] = u32x4{0, 0, 0, 0};
        if (ad[k] >= 0 && ad[k] < a.count) {
          const uint16_t* u = a.u + m * 2 * a.rank_pad + r;
          __builtin_memcpy(&hi[k], u, 16);
          __builtin_memcpy(&lo[k], u + a.rank_pad, 16);
          bv[k] = load_rank8(a.b + (static_cast<int64_t>(ad[k]) * a.out_cols + j) * a.rank + r, a.rank - r);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const auto part = [&](const u32x4& v) { return __uint_as_float((i & 1) ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); };
          add[k] = fmaf(part(hi[k]) + part(lo[k]), part(bv[k]), add[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < STEPS; ++k) add[k] = bias[k] + add[k];
  }
  // part: the waves' sums, by register and lane of the matrix instruction.
  __device__ __forceinline__ void finish(const LinearArgs& a, const f32x4 (*part)[MT][64], int n0, int64_t m0) const {
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int e = static_cast<int>(threadIdx.x) + 64 * NW * k, col = e & 15, row = e >> 4;
      const int64_t m = m0 + row;
      if (e >= 256 * MT || m >= a.rows || n0 + col >= a.out_cols) continue;
      const int l = 16 * (col >> 2) + (row & 15);
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) s += part[w][row >> 4][l][col & 3];
      store1(static_cast<uint16_t*>(a.y) + m * a.y_stride + n0 + col, fmaf(s, scale[k], add[k]));
    }
  }
};

// Few rows: 16 output columns by 16 MT rows per block, every NW-th 128 k by each
// wave, through LDS slots of its own that are filled one or two stages ahead:
// no wave waits for another before the end, where their sums are joined.
// Bound by reading the weights, once; every row of x is read by every block,
// from the caches.  (Fragments read straight into registers take a line of the
// first-level cache per lane, 69 accesses a load: 11.8 us for 64 rows of 4096
// by 4096, that cache's rate; this one 7.4.)  Operands as for the tiles below.
constexpr int few_waves(int mt) { return mt == 4 ? 4 : 8; }
template <int MT>
__global__ __launch_bounds__(64 * few_waves(MT)) void linear_few_kernel(const LinearArgs a) {
  constexpr int NW = few_waves(MT), SLOTS = MT == 4 ? 3 : 2, LOADS = 2 + 2 * MT, SLOT = 1024 * LOADS;
  static_assert(NW * MT * 1024 <= NW * SLOTS * SLOT, "the sums fit");
  __shared__ __align__(1024) unsigned char smem[NW * SLOTS * SLOT];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int n0 = static_cast<int>(blockIdx.x) * 16;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (16 * MT);
  const int K = a.in_cols, ws = static_cast<int>(a.w_stride), xs = static_cast<int>(a.x_stride);
  const int rows_n = min(16, a.out_cols - n0), rows_m = static_cast<int>(min(static_cast<int64_t>(16 * MT), a.rows - m0));
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w + static_cast<int64_t>(n0) * ws, static_cast<unsigned>((rows_n - 1) * ws + K));
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x + m0 * xs, static_cast<unsigned>((rows_m - 1) * xs + K));
  // This lane's loads: row lane / 8 of 8-row group g, position lane % 8 (see linear_tile_kernel).
  unsigned off[LOADS];
  int lk[2];  // k of the piece: the groups' swizzles alternate
#pragma unroll
  for (int g = 0; g < LOADS; ++g) {
    const int r = 8 * g + (lane >> 3), k = 16 * ((lane & 7) ^ ((r >> 1) & 7));
    if (g < 2) {
      lk[g] = k;
      off[g] = r < rows_n ? static_cast<unsigned>(r * ws + k) : 0x80000000u;
    } else {
      off[g] = r - 16 < rows_m ? static_cast<unsigned>((r - 16) * xs + k) : 0x80000000u;
    }
  }
  unsigned char* const ring = smem + wave * (SLOTS * SLOT);
  const int steps = (K + 127) >> 7, mine = steps > wave ? (steps - wave - 1) / NW + 1 : 0;
  auto issue = [&](int s, int to) {
    const int k0 = (wave + NW * s) * 128;
#pragma unroll
    for (int g = 0; g < LOADS; ++g)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(g < 2 ? rw : rx, (lds_ptr_t)(ring + to * SLOT + g * 1024), 16,
                                               static_cast<int>((off[g] + k0) | (k0 + lk[g & 1] < K ? 0u : 0x80000000u)), 0, 0, 0);
  };
#pragma unroll
  for (int s = 0; s < SLOTS - 1; ++s)
    if (s < mine) issue(s, s);
  FewOutputs<MT, NW> out;
  out.start(a, n0, m0);
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int key = (c >> 1) & 7, p0 = c * 128 + 16 * (q ^ key), p1 = c * 128 + 16 * ((q + 4) ^ key);
  for (int s = 0, from = 0; s < mine; ++s) {
    if (s + SLOTS - 1 < mine) issue(s + SLOTS - 1, from == 0 ? SLOTS - 1 : from - 1);
    wait_stage<LOADS, SLOTS - 1>(mine - 1 - s);
    const unsigned char* slot = ring + from * SLOT;
    from = from == SLOTS - 1 ? 0 : from + 1;
    const i32x8 wf = pair8(*reinterpret_cast<const u32x4*>(slot + p0), *reinterpret_cast<const u32x4*>(slot + p1));
#pragma unroll
    for (int i = 0; i < MT; ++i)
      mma8_16(acc[i], wf, pair8(*reinterpret_cast<const u32x4*>(slot + 2048 * (i + 1) + p0),
                                *reinterpret_cast<const u32x4*>(slot + 2048 * (i + 1) + p1)));
  }
  __syncthreads();  // the slots are free
  f32x4(*const part)[MT][64] = reinterpret_cast<f32x4(*)[MT][64]>(smem);
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  out.finish(a, part, n0, m0);
}

// Any size and alignment: as linear_few_kernel with fragments read straight
// into registers, the last piece of a row byte by byte.  Bound by these reads, a
// line of the first-level cache per lane, and by every 16 columns reading x
// again: 8192 rows of 4090 by 4096 in 2.8 ms (4096 by 4096 on the tiles: 0.12),
// 64 rows in 23.5 us (7.4).
constexpr int kAnyWaves = 8, kAnyTiles = 4;
__global__ __launch_bounds__(64 * kAnyWaves) void linear_any_kernel(const LinearArgs a) {
  constexpr int MT = kAnyTiles;
  __shared__ f32x4 part[kAnyWaves][MT][64];
  const int lane = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6;
  const int c = lane & 15, q = lane >> 4;
  const int n0 = static_cast<int>(blockIdx.x) * 16;
  const int64_t m0 = static_cast<int64_t>(blockIdx.y) * (16 * MT);
  const int K = a.in_cols;
  // rows past the end repeat the last one; their outputs are not stored
  const int n = n0 + c < a.out_cols ? n0 + c : a.out_cols - 1;
  const unsigned char* wp = a.w + n * a.w_stride + 16 * q;
  const unsigned char* xp[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + 16 * i + c;
    xp[i] = a.x + (m < a.rows ? m : a.rows - 1) * a.x_stride + 16 * q;
  }
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k = 128 * wave; k < K; k += 128 * kAnyWaves) {
    const int left = K - k - 16 * q;
    const i32x8 wf = pair8(load16<false>(wp + k, left), load16<false>(wp + k + 64, left - 64));
#pragma unroll
    for (int i = 0; i < MT; ++i)
      mma8_16(acc[i], wf, pair8(load16<false>(xp[i] + k, left), load16<false>(xp[i] + k + 64, left - 64)));
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  FewOutputs<MT, kAnyWaves> out;
  out.start(a, n0, m0);
  out.finish(a, part, n0, m0);
}

// c += a b^T over 64 k on 32 x 32 outputs, both operands e4m3.
__device__ __forceinline__ void mma8_32(f32x16& c, const i32x8& a, const i32x8& b) {
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// Many rows: BN output columns by BM rows per block, WN x WM waves.  Stages of
// 128 k go through SLOTS LDS slots, fetched straight into LDS SLOTS - 1 stages ahead;
// rows of a slot are 128 bytes, of which position p holds the 16-byte piece
// p ^ (row / 2 % 8), so that the 16 lanes that are served at a time find
// their pieces in 16 different places of the banks.  A lane takes pieces q and
// q + 2 of a 64-byte half (q its half of the wave) for both operands.
// Operands, strides and in_cols in multiples of 16 bytes.  8192 rows of 4096 by
// 4096 without adapters: 111 us, 2.5 PFLOP/s (the library's 8-bit product 104).
constexpr int kStage = 128;
template <int BN, int BM, int WN, int WM, int SLOTS, bool ADAPT>
__global__ __launch_bounds__(64 * WN * WM) void linear_tile_kernel(const LinearArgs a, int tiles_n, int tiles_m) {
  constexpr int NW = WN * WM, NT = BN / WN / 32, MT = BM / WM / 32;
  constexpr int SLOT = (BN + BM) * kStage, LN = BN / 8 / NW, LM = BM / 8 / NW;
  static_assert(BN % (8 * NW) == 0 && BM % (8 * NW) == 0, "whole rows of eight per wave");
  static_assert((SLOTS - 1) * (LN + LM) <= 63, "loads in flight that a wave can count");
  __shared__ __align__(1024) unsigned char smem[SLOTS * SLOT];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int wn = wave / WM, wm = wave - wn * WM;
  // Tiles in bands of four row tiles, column by column: the blocks that run at
  // a time on an XCD share rows and columns in its cache.
  const int id = xcd_remap(static_cast<int>(blockIdx.x), tiles_n * tiles_m);
  const int band = id / (4 * tiles_n), in_band = id - band * 4 * tiles_n;
  const int high = min(4, tiles_m - 4 * band);
  const int tn = in_band / high, tm = 4 * band + in_band - tn * high;
  const int n0 = tn * BN;
  const int64_t m0 = static_cast<int64_t>(tm) * BM;
  const int K = a.in_cols;
  const int rows_n = min(BN, a.out_cols - n0), rows_m = static_cast<int>(min(static_cast<int64_t>(BM), a.rows - m0));
  const int ws = static_cast<int>(a.w_stride), xs = static_cast<int>(a.x_stride);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w + static_cast<int64_t>(n0) * ws, static_cast<unsigned>((rows_n - 1) * ws + K));
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x + m0 * xs, static_cast<unsigned>((rows_m - 1) * xs + K));
  // This lane's loads: row lane / 8 of 8-row group g of a tile, position lane % 8.
  const int lrow = lane >> 3;
  unsigned off_n[LN], off_m[LM];
  int k_n[LN], k_m[LM];
#pragma unroll
  for (int g = 0; g < LN; ++g) {
    const int row = 8 * (g * NW + wave) + lrow;
    k_n[g] = 16 * ((lane & 7) ^ ((row >> 1) & 7));
    off_n[g] = row < rows_n ? static_cast<unsigned>(row * ws + k_n[g]) : 0x80000000u;
  }
#pragma unroll
  for (int g = 0; g < LM; ++g) {
    const int row = 8 * (g * NW + wave) + lrow;
    k_m[g] = 16 * ((lane & 7) ^ ((row >> 1) & 7));
    off_m[g] = row < rows_m ? static_cast<unsigned>(row * xs + k_m[g]) : 0x80000000u;
  }
  // Past the last k both operands read as zeros.
  auto issue = [&](int s, int to) {
    unsigned char* slot = smem + to * SLOT;
    const int k0 = s * kStage;
#pragma unroll
    for (int g = 0; g < LN; ++g)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_ptr_t)(slot + 8 * (g * NW + wave) * kStage), 16,
                                               static_cast<int>((off_n[g] + k0) | (k0 + k_n[g] < K ? 0u : 0x80000000u)), 0, 0, 0);
#pragma unroll
    for (int g = 0; g < LM; ++g)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_ptr_t)(slot + (BN + 8 * (g * NW + wave)) * kStage), 16,
                                               static_cast<int>((off_m[g] + k0) | (k0 + k_m[g] < K ? 0u : 0x80000000u)), 0, 0, 0);
  };
  f32x16 acc[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.f;
  const int c = lane & 31, q = lane >> 5;
  const int key = (c >> 1) & 7;
  int at[4];  // this lane's four pieces of a row's 128 bytes: half 0's two, half 1's two
#pragma unroll
  for (int p = 0; p < 4; ++p) at[p] = 16 * ((2 * p + q) ^ key);
  const int rd_n = (wn * (BN / WN) + c) * kStage, rd_m = (BN + wm * (BM / WM) + c) * kStage;
  // Scale and adapter of this lane's rows (their latency is that of the first stage).
  float sx[MT];
  int mine[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int row = wm * (BM / WM) + 32 * m + c;
    const int64_t r = m0 + (row < rows_m ? row : rows_m - 1);
    sx[m] = a.x_scale[r];
    mine[m] = -1;
    if (ADAPT) {
      const int ad = a.of_row[r];
      mine[m] = row < rows_m && ad >= 0 && ad < a.count ? ad : -1;
    }
  }
  const int stages = (K + kStage - 1) / kStage;
#pragma unroll
  for (int s = 0; s < SLOTS - 1; ++s)
    if (s < stages) issue(s, s);
  for (int s = 0, from = 0; s < stages; ++s) {
    wait_stage<LN + LM, SLOTS - 2>(stages - 1 - s);
    wg_barrier();  // stage s is there, and nobody reads the slot before it any more
    if (s + SLOTS - 1 < stages) issue(s + SLOTS - 1, from == 0 ? SLOTS - 1 : from - 1);
    const unsigned char* slot = smem + from * SLOT;
    from = from == SLOTS - 1 ? 0 : from + 1;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      i32x8 fn[NT], fm[MT];
#pragma unroll
      for (int n = 0; n < NT; ++n)
        fn[n] = pair8(*reinterpret_cast<const u32x4*>(slot + rd_n + n * 32 * kStage + at[2 * half]),
                      *reinterpret_cast<const u32x4*>(slot + rd_n + n * 32 * kStage + at[2 * half + 1]));
#pragma unroll
      for (int m = 0; m < MT; ++m)
        fm[m] = pair8(*reinterpret_cast<const u32x4*>(slot + rd_m + m * 32 * kStage + at[2 * half]),
                      *reinterpret_cast<const u32x4*>(slot + rd_m + m * 32 * kStage + at[2 * half + 1]));
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) mma8_32(acc[n][m], fn[n], fm[m]);
    }
  }

  // Epilogue: a lane has, for each of its rows (32 m + c), columns 8 j + 4 q
  // .. + 3 of every 32.  The adapters' products are added on the matrix cores,
  // u as the sum of two bfloat16 parts (16 bits, below the output's 8), one
  // adapter of 32 rows after another, right before these rows leave, so that only
  // their sums are in use beside the operands; a lane takes what belongs to its row.
  // Each wave turns its 32 rows of outputs round in LDS, so that they leave as
  // whole lines.
  constexpr int WCOLS = BN / WN;             // columns of a wave
  constexpr int PITCH = WCOLS * 2 + 16;      // bytes of a staged row
  constexpr int PER = WCOLS / 8;             // 16-byte pieces of a row
  static_assert(2 * BN * 4 + NW * 32 * PITCH <= SLOTS * SLOT, "the staged rows fit");
  float* const s_scale = reinterpret_cast<float*>(smem);
  float* const s_bias = s_scale + BN;
  unsigned char* const stage = smem + 2 * BN * 4 + wave * 32 * PITCH;
  wg_barrier();  // nobody reads the slots any more
  for (int j = static_cast<int>(threadIdx.x); j < BN; j += 64 * NW) {
    const bool in = j < rows_n;
    s_scale[j] = in ? a.w_scale[n0 + j] : 0.f;
    s_bias[j] = in && a.bias ? a.bias[n0 + j] : 0.f;
  }
  __syncthreads();
  const int col0 = wn * WCOLS;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 sc = *reinterpret_cast<const f32x4*>(s_scale + col0 + 32 * n + 8 * g + 4 * q);
      const f32x4 bi = *reinterpret_cast<const f32x4*>(s_bias + col0 + 32 * n + 8 * g + 4 * q);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][m][4 * g + i] = fmaf(acc[n][m][4 * g + i], sx[m] * sc[i], bi[i]);
    }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if constexpr (ADAPT) {
      // One adapter of these 32 rows after another, 32 of its ranks at a time.
      const uint16_t* const u = a.u + (m0 + min(wm * (BM / WM) + 32 * m + c, rows_m - 1)) * 2 * a.rank_pad + 8 * q;
      uint64_t todo = __builtin_amdgcn_ballot_w64(mine[m] >= 0);
#pragma unroll 1
      while (todo) {
        const int ad = __builtin_amdgcn_readlane(mine[m], __ffsll(static_cast<unsigned long long>(todo)) - 1);
        const bool ours = mine[m] == ad;
        todo &= ~__builtin_amdgcn_ballot_w64(ours);
        const uint16_t* const b = a.b + static_cast<int64_t>(ad) * a.out_cols * a.rank + 8 * q;
#pragma unroll 1
        for (int r0 = 0; r0 < a.rank; r0 += 32) {
          u32x4 bf[2][NT], up[2][2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int r = r0 + 16 * t;
#pragma unroll
            for (int n = 0; n < NT; ++n)
              bf[t][n] = load_rank8(b + min(n0 + col0 + 32 * n + c, a.out_cols - 1) * a.rank + r, a.rank - r - 8 * q);
            up[t][0] = up[t][1] = u32x4{0, 0, 0, 0};
            if (ours && r < a.rank) {
              __builtin_memcpy(&up[t][0], u + r, 16);
              __builtin_memcpy(&up[t][1], u + a.rank_pad + r, 16);
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            f32x16 sum;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (r0 + 16 * t >= a.rank) break;
#pragma unroll
              for (int p = 0; p < 2; ++p)
                sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, bf[t][n]), __builtin_bit_cast(bf16x8, up[t][p]),
                                                              sum, 0, 0, 0);
            }
            // rows of other adapters keep what they have, whatever this one's matrix holds
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][m][i] += ours ? sum[i] : 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[n][m][4 * g], acc[n][m][4 * g + 1], acc[n][m][4 * g + 2], acc[n][m][4 * g + 3]};
        store4<MAFAT_BF16>(reinterpret_cast<uint16_t*>(stage + c * PITCH) + 32 * n + 8 * g + 4 * q, v);
      }
#pragma unroll
    for (int e = lane; e < 32 * PER; e += 64) {
      const int rr = e / PER, p = e - rr * PER;
      const int out_row = wm * (BM / WM) + 32 * m + rr, j = n0 + col0 + 8 * p;
      const u32x4 v = *reinterpret_cast<const u32x4*>(stage + rr * PITCH + 16 * p);
      if (out_row >= rows_m || j >= a.out_cols) continue;
      uint16_t* y = static_cast<uint16_t*>(a.y) + (m0 + out_row) * a.y_stride + j;
      if (j + 8 <= a.out_cols) {
        __builtin_memcpy(y, &v, 16);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (j + i < a.out_cols) y[i] = static_cast<uint16_t>(v[i >> 1] >> (16 * (i & 1)));
      }
    }
  }
}

// u of one row and 8 ranks per block, two ranks per wave; rows without an
// adapter leave theirs unwritten (and unread).
template <bool WHOLE>
__global__ __launch_bounds__(256) void shrink_rows_kernel(const LinearArgs a) {
  const int64_t m = blockIdx.x;
  const int ad = a.of_row[m];
  if (ad < 0 || ad >= a.count) return;
  const int lane = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6;
  const int r0 = static_cast<int>(blockIdx.y) * 8 + 2 * wave;
  if (r0 >= a.rank) {  // zeros past the rank
    if (lane == 0) {
      uint16_t* u = a.u + m * 2 * a.rank_pad + r0;
      u[0] = u[1] = u[a.rank_pad] = u[a.rank_pad + 1] = 0;
    }
    return;
  }
  const int K = a.in_cols;
  const unsigned char* xp = a.x + m * a.x_stride;
  const bool two = r0 + 1 < a.rank;
  const uint16_t* ap = a.a + (static_cast<int64_t>(ad) * a.rank + r0) * K;
  const uint16_t* bp = two ? ap + K : ap;
  float s0 = 0.f, s1 = 0.f;
  constexpr int AHEAD = WHOLE ? 4 : 1;  // pieces of 16 k that a lane asks for at a time
  for (int k0 = 16 * lane; k0 < K; k0 += AHEAD * 1024) {
    u32x4 xv[AHEAD], av[AHEAD][2], bv[AHEAD][2];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int k = k0 + 1024 * s, left = K - k;
      xv[s] = load16<WHOLE>(xp + k, left);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        av[s][p] = load16<WHOLE>(reinterpret_cast<const unsigned char*>(ap + k + 8 * p), 2 * left - 16 * p);
        bv[s][p] = load16<WHOLE>(reinterpret_cast<const unsigned char*>(bp + k + 8 * p), 2 * left - 16 * p);
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // all of these loads before the first use
#pragma unroll
    for (int s = 0; s < AHEAD; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int xw = static_cast<int>(xv[s][i >> 1]);
        const f32x2 x2 = (i & 1) ? __builtin_amdgcn_cvt_pk_f32_fp8(xw, true) : __builtin_amdgcn_cvt_pk_f32_fp8(xw, false);
        const uint32_t aw = av[s][i >> 2][i & 3], bw = bv[s][i >> 2][i & 3];
        s0 = fmaf(x2[0], __uint_as_float(aw << 16), s0);
        s0 = fmaf(x2[1], __uint_as_float(aw & 0xffff0000u), s0);
        s1 = fmaf(x2[0], __uint_as_float(bw << 16), s1);
        s1 = fmaf(x2[1], __uint_as_float(bw & 0xffff0000u), s1);
      }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    s0 += __shfl_xor(s0, o, 64);
    s1 += __shfl_xor(s1, o, 64);
  }
  if (lane == 0) {
    const float by = a.x_scale[m] * (a.factor ? a.factor[ad] : 1.f);
    uint16_t* u = a.u + m * 2 * a.rank_pad + r0;
    put_parts(u, a.rank_pad, r0 < a.rank ? by * s0 : 0.f);
    put_parts(u + 1, a.rank_pad, two ? by * s1 : 0.f);
  }
}

// u of 32 rows and 32 ranks per block on the matrix cores, for many rows: one
// adapter of those rows after another, its ranks by the rows' values as
// bfloat16 (exact).  Every fourth 128 k by each wave, through LDS slots of its
// own that are filled two stages ahead: read into registers, a fragment's 32
// rows would take 32 lines of the caches for 32 bytes each (29 us for 8192 rows
// of 4096 and rank 32).  Bound by reading x once, from memory, and an adapter's matrix per 32
// rows, from the caches.  The grid's second axis shares out the adapters of 32
// rows, where these are mixed (blocks without one end at once), its third the
// ranks.  x, its stride and a in whole 16-byte pieces, in_cols a multiple of 16.
constexpr int kShrinkWaves = 4, kShrinkSlots = 3;
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_tile_kernel(const LinearArgs a) {
  constexpr int NW = kShrinkWaves, SLOTS = kShrinkSlots, XB = 32 * 128, SLOT = XB + 32 * 256, LOADS = SLOT / 1024;
  __shared__ __align__(1024) unsigned char smem[NW * SLOTS * SLOT];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int c = lane & 31, h = lane >> 5;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * 32;
  const int rows = static_cast<int>(min(static_cast<int64_t>(32), a.rows - m0));
  const int64_t m = m0 + min(c, rows - 1);
  const int r_first = static_cast<int>(blockIdx.z) * 32, ranks = min(32, a.rank - r_first);
  const int K = a.in_cols, xs = static_cast<int>(a.x_stride);
  int mine = a.of_row[m];
  mine = c < rows && mine >= 0 && mine < a.count ? mine : -1;
  const float x_scale = a.x_scale[m];
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x + m0 * xs, static_cast<unsigned>((rows - 1) * xs + K));
  // This lane's loads.  x: row lane / 8 of 8-row group g, position lane % 8; a:
  // row lane / 16 of 4-row group g, position lane % 16; the piece at a position
  // as in linear_tile_kernel.
  unsigned xo[4], ao[8];
  int xk[4], ak[8];
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int r = 8 * g + (lane >> 3);
    xk[g] = 16 * ((lane & 7) ^ ((r >> 1) & 7));
    xo[g] = r < rows ? static_cast<unsigned>(r * xs + xk[g]) : 0x80000000u;
  }
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    const int r = 4 * g + (lane >> 4);
    ak[g] = 8 * ((lane & 15) ^ (r & 15));
    ao[g] = r < ranks ? static_cast<unsigned>((r * K + ak[g]) * 2) : 0x80000000u;
  }
  unsigned char* const ring = smem + wave * (SLOTS * SLOT);
  const int stages = (K + 127) >> 7, mine_stages = stages > wave ? (stages - wave - 1) / NW + 1 : 0;
  uint64_t todo = __builtin_amdgcn_ballot_w64(mine >= 0);
  for (int turn = 0; todo; ++turn) {  // the same for all waves
    const int ad = __builtin_amdgcn_readlane(mine, __ffsll(static_cast<unsigned long long>(todo)) - 1);
    const bool ours = mine == ad;
    todo &= ~__builtin_amdgcn_ballot_w64(ours);
    if (turn % static_cast<int>(gridDim.y) != static_cast<int>(blockIdx.y)) continue;
    const __amdgpu_buffer_rsrc_t ra =
        make_rsrc(a.a + (static_cast<int64_t>(ad) * a.rank + r_first) * K, static_cast<unsigned>(ranks * K * 2));
    auto issue = [&](int s, int to) {
      unsigned char* slot = ring + to * SLOT;
      const int k0 = (wave + NW * s) * 128;
#pragma unroll
      for (int g = 0; g < 4; ++g)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_ptr_t)(slot + g * 1024), 16,
                                                 static_cast<int>((xo[g] + k0) | (k0 + xk[g] < K ? 0u : 0x80000000u)), 0, 0, 0);
#pragma unroll
      for (int g = 0; g < 8; ++g)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr_t)(slot + XB + g * 1024), 16,
                                                 static_cast<int>((ao[g] + 2 * k0) | (k0 + ak[g] < K ? 0u : 0x80000000u)), 0, 0, 0);
    };
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int s = 0; s < SLOTS - 1; ++s)
      if (s < mine_stages) issue(s, s);
    for (int s = 0, from = 0; s < mine_stages; ++s) {
      if (s + SLOTS - 1 < mine_stages) issue(s + SLOTS - 1, from == 0 ? SLOTS - 1 : from - 1);
      wait_stage<LOADS, SLOTS - 1>(mine_stages - 1 - s);
      const unsigned char* slot = ring + from * SLOT;
      from = from == SLOTS - 1 ? 0 : from + 1;
      // A lane takes k 16 h .. + 15 of each 32, in two instructions.
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4 xv = *reinterpret_cast<const u32x4*>(slot + c * 128 + 16 * ((2 * j + h) ^ ((c >> 1) & 7)));
        bf16x8 xb[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(xv[i]), false);
          const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(xv[i]), true);
          xb[i >> 1][4 * (i & 1)] = static_cast<__bf16>(lo[0]);
          xb[i >> 1][4 * (i & 1) + 1] = static_cast<__bf16>(lo[1]);
          xb[i >> 1][4 * (i & 1) + 2] = static_cast<__bf16>(hi[0]);
          xb[i >> 1][4 * (i & 1) + 3] = static_cast<__bf16>(hi[1]);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const u32x4 av = *reinterpret_cast<const u32x4*>(slot + XB + c * 256 + 16 * ((4 * j + 2 * h + p) ^ (c & 15)));
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av), xb[p], acc, 0, 0, 0);
        }
      }
    }
    __syncthreads();  // the slots are free
    float* const part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < 16; ++i) part[(wave * 16 + i) * 64 + lane] = acc[i];
    __syncthreads();
    // Each wave adds up every fourth register of all waves: rank 8 (i / 4) + 4 h + i % 4 of the lane's row.
    const float by = x_scale * (a.factor ? a.factor[ad] : 1.f);
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const int i = wave + 4 * i4, r = 8 * (i >> 2) + 4 * h + (i & 3);
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) s += part[(w * 16 + i) * 64 + lane];
      if (ours && r_first + r < a.rank_pad)
        put_parts(a.u + m * 2 * a.rank_pad + r_first + r, a.rank_pad, r < ranks ? by * s : 0.f);
    }
    __syncthreads();
  }
}

bool whole(const void* p, int64_t stride_bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(stride_bytes)) & 15) == 0;
}

hipError_t launch_shrink(const LinearArgs& a, hipStream_t stream) {
  if (a.rows > kShrinkRows && a.in_cols % 16 == 0 && whole(a.x, a.x_stride) && whole(a.a, 0)) {
    // mixed adapters are shared out where the row tiles alone do not fill the GPU
    const int64_t tiles = (a.rows + 31) / 32, spare = tiles < 512 ? 512 / tiles : 1;
    const int64_t share = spare < a.count ? spare : a.count;
    const dim3 grid(static_cast<unsigned>(tiles), static_cast<unsigned>(share < 32 ? share : 32),
                    static_cast<unsigned>((a.rank + 31) / 32));
    hipLaunchKernelGGL(shrink_tile_kernel, grid, dim3(64 * kShrinkWaves), 0, stream, a);
  } else {
    const dim3 grid(static_cast<unsigned>(a.rows), static_cast<unsigned>(a.rank_pad / 8));
    if (a.in_cols % 16 == 0) hipLaunchKernelGGL(shrink_rows_kernel<true>, grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(shrink_rows_kernel<false>, grid, dim3(256), 0, stream, a);
  }
  return hipGetLastError();
}

template <int BN, int BM, int WN, int WM, int SLOTS>
void launch_tile(const LinearArgs& a, int tn, int tm, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(tn) * static_cast<unsigned>(tm)), block(64 * WN * WM);
  if (a.count) hipLaunchKernelGGL((linear_tile_kernel<BN, BM, WN, WM, SLOTS, true>), grid, block, 0, stream, a, tn, tm);
  else hipLaunchKernelGGL((linear_tile_kernel<BN, BM, WN, WM, SLOTS, false>), grid, block, 0, stream, a, tn, tm);
}

template <int MT>
void launch_few(const LinearArgs& a, dim3 grid, hipStream_t stream) {
  hipLaunchKernelGGL(linear_few_kernel<MT>, grid, dim3(64 * few_waves(MT)), 0, stream, a);
}

// Rows of one launch of each kernel, at most: it has fewer than 2^32 threads
// along the grid's first axis (shrink_rows_kernel has 256 a row) and 65535
// blocks of linear_any_kernel's 64 rows along its second.  Whole row tiles.
constexpr int64_t kLaunchRows = (int64_t{1} << 22) - 256;
static_assert(kLaunchRows <= int64_t{65535} * 16 * kAnyTiles && kLaunchRows % 256 == 0, "rows of a launch");

hipError_t launch_rows(const LinearArgs& a, hipStream_t stream) {
  if (a.count) {
    const hipError_t e = launch_shrink(a, stream);
    if (e != hipSuccess) return e;
  }
  const bool pieces = a.in_cols % 16 == 0 && whole(a.x, a.x_stride) && whole(a.w, a.w_stride);
  // More rows than linear_few_kernel takes at a time: tiles, as large as leaves
  // a block for every CU (8192 rows of 4096 by 4096, 8 adapters of rank 32: 131 us
  // by tiles of 256, 140 by tiles of 128; without adapters 111).
  if (pieces && a.rows > 64) {
    const auto tiles = [&](int64_t n, int64_t m) { return ((a.out_cols + n - 1) / n) * ((a.rows + m - 1) / m); };
    const int side = tiles(256, 256) >= 256 ? 256 : tiles(128, 128) >= 256 ? 128 : 64;
    if (tiles(side, side) >= (int64_t{1} << 23)) return hipErrorInvalidValue;  // 512 threads each (y would take a TB)
    const int tn = (a.out_cols + side - 1) / side, tm = static_cast<int>((a.rows + side - 1) / side);
    if (side == 256) launch_tile<256, 256, 4, 2, 2>(a, tn, tm, stream);
    else if (side == 128) launch_tile<128, 128, 2, 2, 2>(a, tn, tm, stream);
    else launch_tile<64, 64, 2, 2, 4>(a, tn, tm, stream);
    return hipGetLastError();
  }
  const unsigned nt = static_cast<unsigned>((a.out_cols + 15) / 16);
  if (pieces) {
    if (a.rows <= 16) launch_few<1>(a, dim3(nt), stream);
    else if (a.rows <= 32) launch_few<2>(a, dim3(nt), stream);
    else launch_few<4>(a, dim3(nt), stream);
    return hipGetLastError();
  }
  const dim3 grid(nt, static_cast<unsigned>((a.rows + 16 * kAnyTiles - 1) / (16 * kAnyTiles)));
  hipLaunchKernelGGL(linear_any_kernel, grid, dim3(64 * kAnyWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
  for (int64_t at = 0; at < a.rows; at += kLaunchRows) {
    LinearArgs p = a;
    p.rows = a.rows - at < kLaunchRows ? a.rows - at : kLaunchRows;
    p.x = a.x + at * a.x_stride;
    p.x_scale = a.x_scale + at;
    p.y = static_cast<uint16_t*>(a.y) + at * a.y_stride;
    if (a.count) {
      p.of_row = a.of_row + at;
      p.u = a.u + at * 2 * a.rank_pad;
    }
    const hipError_t e = launch_rows(p, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mafat
