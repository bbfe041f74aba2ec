// linear.hip -- projection of 8-bit rows by 8-bit weights, with low-rank
// adapters beside it.
//
//   y[i][j] = xs[i] ws[j] sum_k x[i][k] w[j][k] + bias[j] + sum_r u[i][r] b[a(i)][j][r]
//   u[i][r] = factor[a(i)] xs[i] sum_k x[i][k] a[a(i)][r][k]
//
// Two launches with adapters: u first (shrink_rows_kernel), then the product
// whose epilogue adds the adapters (linear_few_kernel).  The weights are the
// matrix instructions' A operand and the rows of x their B operand, so a lane
// ends up with consecutive output columns of one row of y.  Both operands are
// read along k and take it in the same order, so any order of k within an
// instruction will do: a lane takes 16-byte pieces.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "reader.h"

namespace mafat {
namespace {

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

// 16 bytes at p, of which `n` may be read (the rest are zero); p need not be aligned.
__device__ __forceinline__ u32x4 load16(const unsigned char* p, int n) {
  u32x4 v = {0, 0, 0, 0};
  if (n >= 16) {
    __builtin_memcpy(&v, p, 16);
  } else {
    unsigned char t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = i < n ? p[i] : 0;
    __builtin_memcpy(&v, t, 16);
  }
  return v;
}

// sum_r u[r] b[r] of one output column.
__device__ __forceinline__ float expand(const float* u, const uint16_t* b, int rank) {
  float s = 0.f;
  int r = 0;
  for (; r + 8 <= rank; r += 8) {
    uint16_t t[8];
    float v[8];
    __builtin_memcpy(t, b + r, 16);
    __builtin_memcpy(v, u + r, 32);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(v[i], to_f(t[i]), s);
  }
  for (; r < rank; ++r) s = fmaf(u[r], to_f(b[r]), s);
  return s;
}

// Few rows: 16 output columns by MT * 16 rows per block.  Bound by reading the
// weights (once), so nothing goes through LDS on the way in; the block's 8
// waves take every eighth 128 k each and join their sums at the end.  Every
// row of x is read by every block, from the caches.
constexpr int kFewWaves = 8;
template <int MT>
__global__ __launch_bounds__(64 * kFewWaves) void linear_few_kernel(const LinearArgs a) {
  __shared__ f32x4 part[kFewWaves][MT][64];
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
  for (int k = 128 * wave; k < K; k += 128 * kFewWaves) {
    const int left = K - k - 16 * q;
    const i32x8 wf = pair8(load16(wp + k, left), load16(wp + k + 64, left - 64));
#pragma unroll
    for (int i = 0; i < MT; ++i) mma8_16(acc[i], wf, pair8(load16(xp[i] + k, left), load16(xp[i] + k + 64, left - 64)));
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int e = static_cast<int>(threadIdx.x); e < 64 * MT; e += 64 * kFewWaves) {
    const int i = e >> 6, l = e & 63;
    const int64_t m = m0 + 16 * i + (l & 15);
    const int j0 = n0 + 4 * (l >> 4);
    if (m >= a.rows || j0 >= a.out_cols) continue;
    f32x4 s = part[0][i][l];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) s += part[w][i][l];
    const float xs = a.x_scale[m];
    const int ad = a.count ? a.of_row[m] : -1;
    const bool has = ad >= 0 && ad < a.count;
    uint16_t* y = static_cast<uint16_t*>(a.y) + m * a.y_stride + j0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = j0 + r;
      if (j >= a.out_cols) break;
      float v = s[r] * (xs * a.w_scale[j]);
      if (a.bias) v += a.bias[j];
      if (has) v += expand(a.u + m * a.rank, a.b + (static_cast<int64_t>(ad) * a.out_cols + j) * a.rank, a.rank);
      store1(y + r, v);
    }
  }
}

// c += a b^T over 64 k on 32 x 32 outputs, both operands e4m3.
__device__ __forceinline__ void mma8_32(f32x16& c, const i32x8& a, const i32x8& b) {
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

// Many rows: BN output columns by BM rows per block, WN x WM waves.  Stages of
// 128 k go through two LDS slots, fetched straight into LDS one stage ahead;
// rows of a slot are 128 bytes, of which position p holds the 16-byte piece
// p ^ (row / 2 % 8), so that the 16 lanes that are served at a time find
// their pieces in 16 different places of the banks.  A lane takes pieces q and
// q + 2 of a 64-byte half (q its half of the wave) for both operands.
// Operands, strides and in_cols in multiples of 16 bytes.
constexpr int kStage = 128;
template <int BN, int BM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM) void linear_tile_kernel(const LinearArgs a, int tiles_n, int tiles_m) {
  constexpr int NW = WN * WM, NT = BN / WN / 32, MT = BM / WM / 32;
  constexpr int SLOT = (BN + BM) * kStage, LN = BN / 8 / NW, LM = BM / 8 / NW;
  static_assert(BN % (8 * NW) == 0 && BM % (8 * NW) == 0, "whole rows of eight per wave");
  __shared__ __align__(1024) unsigned char smem[2 * SLOT];
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
  auto issue = [&](int s) {
    unsigned char* slot = smem + (s & 1) * SLOT;
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
  const int stages = (K + kStage - 1) / kStage;
  issue(0);
  for (int s = 0; s < stages; ++s) {
    wait_vmcnt<0>();
    wg_barrier();  // stage s is there, and nobody reads the other slot any more
    if (s + 1 < stages) issue(s + 1);
    const unsigned char* slot = smem + (s & 1) * SLOT;
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
  // adapter of the 32 rows after another; a lane takes what belongs to its row.
  // Each wave turns its 32 rows of outputs round in LDS, so that they leave as
  // whole lines.
  constexpr int WCOLS = BN / WN;             // columns of a wave
  constexpr int PITCH = WCOLS * 2 + 16;      // bytes of a staged row
  constexpr int PER = WCOLS / 8;             // 16-byte pieces of a row
  static_assert(2 * BN * 4 + NW * 32 * PITCH <= 2 * SLOT, "the staged rows fit");
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
  for (int m = 0; m < MT; ++m) {
    const int row = wm * (BM / WM) + 32 * m + c;  // of the tile
    const bool real = row < rows_m;
    const int64_t r = m0 + (real ? row : rows_m - 1);
    const float sx = a.x_scale[r];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 sc = *reinterpret_cast<const f32x4*>(s_scale + col0 + 32 * n + 8 * g + 4 * q);
        const f32x4 bi = *reinterpret_cast<const f32x4*>(s_bias + col0 + 32 * n + 8 * g + 4 * q);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][m][4 * g + i] = fmaf(acc[n][m][4 * g + i], sx * sc[i], bi[i]);
      }
    if (a.count) {
      int mine = a.of_row[r];
      mine = real && mine >= 0 && mine < a.count ? mine : -1;
      const float* u = a.u + r * a.rank;
      uint64_t todo = __builtin_amdgcn_ballot_w64(mine >= 0);
      while (todo) {
        const int ad = __builtin_amdgcn_readlane(mine, __ffsll(static_cast<unsigned long long>(todo)) - 1);
        const bool ours = mine == ad;
        todo &= ~__builtin_amdgcn_ballot_w64(ours);
        const uint16_t* b = a.b + static_cast<int64_t>(ad) * a.out_cols * a.rank;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int j = min(n0 + col0 + 32 * n + c, a.out_cols - 1);
          const uint16_t* bj = b + static_cast<int64_t>(j) * a.rank;
          f32x16 sum = acc[n][m];
          for (int r0 = 0; r0 < a.rank; r0 += 16) {
            const int rk = r0 + 8 * q, left = a.rank - rk;
            float uv[8];
            if (ours && left >= 8) {
              __builtin_memcpy(uv, u + rk, 32);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) uv[i] = ours && i < left ? u[rk + i] : 0.f;
            }
            bf16x8 hi, lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              hi[i] = static_cast<__bf16>(uv[i]);
              lo[i] = static_cast<__bf16>(uv[i] - static_cast<float>(hi[i]));
            }
            const bf16x8 bf = __builtin_bit_cast(bf16x8, load16(reinterpret_cast<const unsigned char*>(bj + rk), 2 * left));
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf, hi, sum, 0, 0, 0);
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf, lo, sum, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[n][m][i] = ours ? sum[i] : acc[n][m][i];
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
__global__ __launch_bounds__(256) void shrink_rows_kernel(const LinearArgs a) {
  const int64_t m = blockIdx.x;
  const int ad = a.of_row[m];
  if (ad < 0 || ad >= a.count) return;
  const int lane = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6;
  const int r0 = static_cast<int>(blockIdx.y) * 8 + 2 * wave;
  if (r0 >= a.rank) return;
  const int K = a.in_cols;
  const unsigned char* xp = a.x + m * a.x_stride;
  const bool two = r0 + 1 < a.rank;
  const uint16_t* ap = a.a + (static_cast<int64_t>(ad) * a.rank + r0) * K;
  const uint16_t* bp = two ? ap + K : ap;
  float s0 = 0.f, s1 = 0.f;
  for (int k = 16 * lane; k < K; k += 1024) {
    const u32x4 xv = load16(xp + k, K - k);
    const unsigned char* ab = reinterpret_cast<const unsigned char*>(ap + k);
    const unsigned char* bb = reinterpret_cast<const unsigned char*>(bp + k);
    const int left = 2 * (K - k);
    const u32x4 av[2] = {load16(ab, left), load16(ab + 16, left - 16)};
    const u32x4 bv[2] = {load16(bb, left), load16(bb + 16, left - 16)};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const f32x2 x2 = (i & 1) ? __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(xv[i >> 1]), true)
                               : __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(xv[i >> 1]), false);
      const uint32_t aw = av[i >> 2][i & 3], bw = bv[i >> 2][i & 3];
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
    float* u = a.u + m * a.rank + r0;
    u[0] = by * s0;
    if (two) u[1] = by * s1;
  }
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
  if (a.count) {
    hipLaunchKernelGGL(shrink_rows_kernel, dim3(static_cast<unsigned>(a.rows), static_cast<unsigned>((a.rank + 7) / 8)),
                       dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // More than 64 rows whose operands are whole 16-byte pieces: tiles through LDS.
  const auto whole = [](const void* p, int64_t stride) { return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(stride)) & 15) == 0; };
  if (a.rows > 64 && a.in_cols % 16 == 0 && whole(a.x, a.x_stride) && whole(a.w, a.w_stride)) {
    const auto tiles = [&](int64_t n, int64_t m) { return ((a.out_cols + n - 1) / n) * ((a.rows + m - 1) / m); };
    const int side = tiles(256, 256) >= 256 ? 256 : tiles(128, 128) >= 256 ? 128 : 64;
    if (tiles(side, side) < (int64_t{1} << 31)) {
      const int tn = (a.out_cols + side - 1) / side, tm = static_cast<int>((a.rows + side - 1) / side);
      const dim3 grid(static_cast<unsigned>(tn) * static_cast<unsigned>(tm));
      if (side == 256) hipLaunchKernelGGL((linear_tile_kernel<256, 256, 4, 2>), grid, dim3(512), 0, stream, a, tn, tm);
      else if (side == 128) hipLaunchKernelGGL((linear_tile_kernel<128, 128, 2, 2>), grid, dim3(256), 0, stream, a, tn, tm);
      else hipLaunchKernelGGL((linear_tile_kernel<64, 64, 2, 2>), grid, dim3(256), 0, stream, a, tn, tm);
      return hipGetLastError();
    }
  }
  const unsigned nt = static_cast<unsigned>((a.out_cols + 15) / 16);
  const int mt = a.rows <= 16 ? 1 : a.rows <= 32 ? 2 : 4;
  // the grid's second axis ends at 65535: more rows go in several launches
  constexpr int64_t kAxis = 65535;
  for (int64_t at = 0; at < a.rows; at += kAxis * 16 * mt) {
    LinearArgs p = a;
    p.rows = a.rows - at < kAxis * 16 * mt ? a.rows - at : kAxis * 16 * mt;
    p.x = a.x + at * a.x_stride;
    p.x_scale = a.x_scale + at;
    p.y = static_cast<uint16_t*>(a.y) + at * a.y_stride;
    if (a.count) {
      p.of_row = a.of_row + at;
      p.u = a.u + at * a.rank;
    }
    const dim3 grid(nt, static_cast<unsigned>((p.rows + 16 * mt - 1) / (16 * mt)));
    switch (mt) {
      case 1: hipLaunchKernelGGL(linear_few_kernel<1>, grid, dim3(64 * kFewWaves), 0, stream, p); break;
      case 2: hipLaunchKernelGGL(linear_few_kernel<2>, grid, dim3(64 * kFewWaves), 0, stream, p); break;
      default: hipLaunchKernelGGL(linear_few_kernel<4>, grid, dim3(64 * kFewWaves), 0, stream, p); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mafat
