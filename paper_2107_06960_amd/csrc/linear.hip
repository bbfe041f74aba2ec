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
