// reader.cpp -- C ABI of the reader's operators (include/mafat_reader.h):
// checks of the arguments, choice of the kernels' work split, launches.
#include <cmath>
#include <string>

#include "mafat_internal.h"
#include "reader.h"

namespace mafat {
namespace {

constexpr int64_t kMax31 = int64_t{1} << 31;

int fail(int status, const std::string& msg) {
  set_error(msg);
  return status;
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

size_t elt_size(int dtype) { return dtype == MAFAT_F32 ? 4 : dtype == MAFAT_BF16 ? 2 : 1; }

// Rows of `width` bytes every `pitch` bytes.
struct Span {
  const void* p;
  int64_t rows;
  int64_t width, pitch;
};

// Whether two tensors share a byte.  Tensors of one pitch may lie side by side
// in the rows of one buffer; others count as overlapping if their extents do.
bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t a1 = a0 + static_cast<uintptr_t>((a.rows - 1) * a.pitch + a.width);
  const uintptr_t b1 = b0 + static_cast<uintptr_t>((b.rows - 1) * b.pitch + b.width);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.pitch != b.pitch) return true;
  const int64_t d = static_cast<int64_t>(b0 >= a0 ? (b0 - a0) % a.pitch : (a.pitch - (a0 - b0) % a.pitch) % a.pitch);
  return d < a.width || d + b.width > a.pitch;
}

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? MAFAT_OK : fail(MAFAT_EHIP, std::string(what) + " launch failed: " + hipGetErrorString(e));
}

constexpr int64_t kMaxLinearCols = int64_t{1} << 22;  // 256 rows of a tile in 32-bit offsets
constexpr int kMaxRank = 128;

// The sizes and adapters of a projection; the workspace holds the adapters'
// inner products of every row.
int check_linear(int64_t rows, int64_t in_cols, int64_t out_cols, const mafat_adapters* ad, size_t* bytes) {
  if (rows < 0 || in_cols < 1 || out_cols < 1) return fail(MAFAT_EINVAL, "rows must be >= 0, in_cols and out_cols >= 1");
  if (rows >= kMax31 || in_cols >= kMaxLinearCols || out_cols >= kMaxLinearCols)
    return fail(MAFAT_EUNSUPPORTED, "2^31 or more rows, or 2^22 or more columns");
  *bytes = 0;
  if (ad) {
    if (ad->count < 1 || ad->rank < 1) return fail(MAFAT_EINVAL, "adapters: count and rank must be >= 1");
    if (ad->rank > kMaxRank) return fail(MAFAT_EUNSUPPORTED, "adapters: rank above 128");
    *bytes = (static_cast<size_t>(rows) * ad->rank * sizeof(float) + 255) & ~size_t{255};
  }
  return MAFAT_OK;
}

}  // namespace
}  // namespace mafat

using namespace mafat;

extern "C" int mafat_add_rms_norm(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t x_stride,
                                  const void* residual, int64_t residual_stride, const float* gain, float eps,
                                  void* sum, int64_t sum_stride, int32_t out_dtype, void* y, int64_t y_stride,
                                  float* y_scale, void* stream) {
  return guarded([&] {
    clear_error();
    if (dtype != MAFAT_F32 && dtype != MAFAT_BF16) return fail(MAFAT_EUNSUPPORTED, "dtype must be F32 or BF16");
    if (out_dtype != MAFAT_F32 && out_dtype != MAFAT_BF16 && out_dtype != MAFAT_F8)
      return fail(MAFAT_EUNSUPPORTED, "out_dtype must be F32, BF16 or F8");
    if (rows < 0 || cols < 1) return fail(MAFAT_EINVAL, "rows must be >= 0 and cols >= 1");
    if (rows >= kMax31 || cols >= kMax31) return fail(MAFAT_EUNSUPPORTED, "2^31 or more rows or columns");
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MAFAT_EINVAL, "eps must be finite and not negative");
    if (rows == 0) return static_cast<int>(MAFAT_OK);  // tensors of no rows may have no address
    if (!residual != !sum) return fail(MAFAT_EINVAL, "residual and sum go together");
    if ((out_dtype == MAFAT_F8) != (y_scale != nullptr))
      return fail(MAFAT_EINVAL, "y_scale goes with 8-bit output, and with no other");
    if (x_stride < cols || y_stride < cols || (residual && (residual_stride < cols || sum_stride < cols)))
      return fail(MAFAT_EINVAL, "a stride is smaller than cols");
    if (x_stride >= kMax31 || y_stride >= kMax31 || (residual && (residual_stride >= kMax31 || sum_stride >= kMax31)))
      return fail(MAFAT_EUNSUPPORTED, "a stride of 2^31 or more");
    const size_t in = elt_size(dtype), out = elt_size(out_dtype);
    if (!x || !y) return fail(MAFAT_EINVAL, "x and y must be non-NULL");
    if (!aligned(x, in) || !aligned(residual, in) || !aligned(sum, in) || !aligned(y, out) || !aligned(gain, 4) ||
        !aligned(y_scale, 4))
      return fail(MAFAT_EINVAL, "a pointer is not aligned to its elements");
    const int64_t isz = static_cast<int64_t>(in), osz = static_cast<int64_t>(out);
    const Span sx{x, rows, cols * isz, x_stride * isz}, sr{residual, rows, cols * isz, residual_stride * isz};
    const Span ss{sum, rows, cols * isz, sum_stride * isz}, sy{y, rows, cols * osz, y_stride * osz};
    const Span sc{y_scale, 1, 4 * rows, 4 * rows}, sg{gain, 1, 4 * cols, 4 * cols};
    const bool on_x = sum && sum == x && sum_stride == x_stride;
    const bool on_res = sum && sum == residual && sum_stride == residual_stride;
    if (overlap(sy, sx) || overlap(sy, sr) || overlap(sy, ss) || overlap(sy, sc) || overlap(sy, sg) || overlap(sc, sx) ||
        overlap(sc, sr) || overlap(sc, ss) || overlap(sc, sg) || overlap(ss, sg))
      return fail(MAFAT_EINVAL, "an output overlaps another tensor");
    if (sum && ((overlap(ss, sx) && !on_x) ||
                (overlap(ss, sr) && !on_res)))
      return fail(MAFAT_EINVAL, "sum overlaps x or residual without being it");
    NormArgs a{};
    a.x = x; a.res = residual; a.gain = gain; a.sum = sum; a.y = y; a.y_scale = y_scale;
    a.x_stride = x_stride; a.res_stride = residual_stride; a.sum_stride = sum_stride; a.y_stride = y_stride;
    a.rows = rows; a.cols = static_cast<int32_t>(cols); a.eps = eps;
    return launched(launch_norm(dtype, out_dtype, a, static_cast<hipStream_t>(stream)), "norm");
  });
}

extern "C" int mafat_linear_workspace(int64_t rows, int64_t in_cols, int64_t out_cols, const mafat_adapters* adapters,
                                      size_t* bytes) {
  return guarded([&] {
    clear_error();
    if (!bytes) return fail(MAFAT_EINVAL, "bytes is NULL");
    return check_linear(rows, in_cols, out_cols, adapters, bytes);
  });
}

extern "C" int mafat_linear(int64_t rows, int64_t in_cols, int64_t out_cols, const void* x, int64_t x_stride,
                            const float* x_scale, const void* w, int64_t w_stride, const float* w_scale,
                            const float* bias, const mafat_adapters* adapters, void* y, int64_t y_stride,
                            void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    clear_error();
    size_t need = 0;
    const int rc = check_linear(rows, in_cols, out_cols, adapters, &need);
    if (rc != MAFAT_OK) return rc;
    if (x_stride < in_cols || w_stride < in_cols || y_stride < out_cols)
      return fail(MAFAT_EINVAL, "a stride is smaller than its row");
    if (x_stride >= kMaxLinearCols || w_stride >= kMaxLinearCols || y_stride >= kMax31)
      return fail(MAFAT_EUNSUPPORTED, "a stride of 2^22 or more (y: 2^31)");
    if (rows == 0) return static_cast<int>(MAFAT_OK);  // tensors of no rows may have no address
    if (!x || !x_scale || !w || !w_scale || !y) return fail(MAFAT_EINVAL, "x, w, their scales and y must be non-NULL");
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(y, 2))
      return fail(MAFAT_EINVAL, "a pointer is not aligned to its elements");
    LinearArgs a{};
    const Span sy{y, rows, 2 * out_cols, 2 * y_stride};
    if (adapters) {
      const mafat_adapters& d = *adapters;
      if (!d.a || !d.b || !d.of_row) return fail(MAFAT_EINVAL, "adapters: a, b and of_row must be non-NULL");
      if (!aligned(d.a, 2) || !aligned(d.b, 2) || !aligned(d.factor, 4) || !aligned(d.of_row, 4))
        return fail(MAFAT_EINVAL, "adapters: a pointer is not aligned to its elements");
      if (ws_bytes < need)
        return fail(MAFAT_EWORKSPACE, "workspace " + std::to_string(ws_bytes) + " < " + std::to_string(need) + " bytes");
      if (!workspace || !aligned(workspace, 256))
        return fail(MAFAT_EINVAL, "workspace must be non-NULL and 256-byte aligned");
      const int64_t an = 2 * static_cast<int64_t>(d.count) * d.rank * in_cols, bn = 2 * static_cast<int64_t>(d.count) * d.rank * out_cols;
      const Span su{workspace, 1, static_cast<int64_t>(need), static_cast<int64_t>(need)};
      const Span others[] = {{d.a, 1, an, an}, {d.b, 1, bn, bn}, {d.factor, 1, 4 * d.count, 4 * d.count},
                             {d.of_row, 1, 4 * rows, 4 * rows}, {x, rows, in_cols, x_stride},
                             {w, out_cols, in_cols, w_stride}, {x_scale, 1, 4 * rows, 4 * rows},
                             {w_scale, 1, 4 * out_cols, 4 * out_cols}, {bias, 1, 4 * out_cols, 4 * out_cols}};
      for (const Span& o : others)
        if (overlap(sy, o) || overlap(su, o)) return fail(MAFAT_EINVAL, "y or the workspace overlaps an input");
      if (overlap(sy, su)) return fail(MAFAT_EINVAL, "y overlaps the workspace");
      a.a = static_cast<const uint16_t*>(d.a);
      a.b = static_cast<const uint16_t*>(d.b);
      a.factor = d.factor;
      a.of_row = d.of_row;
      a.u = static_cast<float*>(workspace);
      a.count = d.count;
      a.rank = d.rank;
    } else {
      const Span others[] = {{x, rows, in_cols, x_stride}, {w, out_cols, in_cols, w_stride},
                             {x_scale, 1, 4 * rows, 4 * rows}, {w_scale, 1, 4 * out_cols, 4 * out_cols},
                             {bias, 1, 4 * out_cols, 4 * out_cols}};
      for (const Span& o : others)
        if (overlap(sy, o)) return fail(MAFAT_EINVAL, "y overlaps an input");
    }
    a.x = static_cast<const unsigned char*>(x);
    a.w = static_cast<const unsigned char*>(w);
    a.x_scale = x_scale; a.w_scale = w_scale; a.bias = bias; a.y = y;
    a.x_stride = x_stride; a.w_stride = w_stride; a.y_stride = y_stride;
    a.rows = rows;
    a.in_cols = static_cast<int32_t>(in_cols);
    a.out_cols = static_cast<int32_t>(out_cols);
    return launched(launch_linear(a, static_cast<hipStream_t>(stream)), "linear");
  });
}
