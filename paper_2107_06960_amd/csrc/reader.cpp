// reader.cpp -- C ABI of the reader's operators (include/mafat_reader.h):
// checks of the arguments, choice of the kernels' work split, launches.
#include <cmath>
#include <initializer_list>
#include <string>
#include <utility>

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

// Whether n rows of a stride have an extent that byte arithmetic can hold.
bool fits(int64_t n, int64_t stride) { return n < 1 || stride < (int64_t{1} << 58) / n; }

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
constexpr int rank_padded(int rank) { return (rank + 15) & ~15; }  // whole matrix instructions

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
    *bytes = (static_cast<size_t>(rows) * 2 * rank_padded(ad->rank) * sizeof(uint16_t) + 255) & ~size_t{255};
  }
  return MAFAT_OK;
}

// What the kernels multiply products by: their exponentials are powers of two.
float base2_scale(float scale) { return static_cast<float>(static_cast<double>(scale) * 1.4426950408889634); }

// The sizes and strides of an attention call; the workspace holds the parts
// that the splits of the positions are joined from.
int check_cross(const mafat_cross* c, size_t* bytes) {
  if (!c) return fail(MAFAT_EINVAL, "c is NULL");
  if (c->dtype != MAFAT_F32 && c->dtype != MAFAT_BF16) return fail(MAFAT_EUNSUPPORTED, "dtype must be F32 or BF16");
  if (c->frames < 1 || c->rows < 0 || c->positions < 0) return fail(MAFAT_EINVAL, "frames must be >= 1, rows and positions >= 0");
  if (c->kv_heads < 1 || c->q_heads < 1 || c->q_heads % c->kv_heads)
    return fail(MAFAT_EINVAL, "q_heads must be a multiple of kv_heads");
  if (c->head_dim < 1) return fail(MAFAT_EINVAL, "head_dim must be >= 1");
  if (c->head_dim > 256) return fail(MAFAT_EUNSUPPORTED, "head_dim above 256");
  if (!std::isfinite(c->scale)) return fail(MAFAT_EINVAL, "scale must be finite");
  if (!std::isfinite(base2_scale(c->scale))) return fail(MAFAT_EUNSUPPORTED, "scale above 2.35e38");
  const int64_t d = c->head_dim;
  if (c->q_head < d || c->k_head < d || c->v_head < d || c->y_head < d)
    return fail(MAFAT_EINVAL, "a head stride is smaller than head_dim");
  if (c->q_row < d || c->y_row < d || c->k_pos < d || c->v_pos < d || c->k_frame < d || c->v_frame < d || c->mask_row < 0)
    return fail(MAFAT_EINVAL, "a row, position or frame stride is smaller than head_dim");
  const int64_t most = kMax31 / (c->dtype == MAFAT_F32 ? 4 : 2);
  if (c->rows >= kMax31 / c->q_heads || c->positions >= kMax31 || c->frames >= kMax31 / c->kv_heads || c->kv_heads > 65535)
    return fail(MAFAT_EUNSUPPORTED, "rows * q_heads, positions or frames * kv_heads of 2^31 or more, or more than 65535 kv_heads");
  if (c->q_row >= most || c->y_row >= most || c->k_pos >= most || c->v_pos >= most || c->q_head >= most || c->k_head >= most ||
      c->v_head >= most || c->y_head >= most)
    return fail(MAFAT_EUNSUPPORTED, "a row, position or head stride of 2^31 bytes or more");
  if (!fits(c->rows, c->q_row) || !fits(c->rows, c->y_row) || !fits(c->positions, c->k_pos) || !fits(c->positions, c->v_pos) ||
      !fits(c->frames, c->k_frame) || !fits(c->frames, c->v_frame) || !fits(c->mask_by_row ? c->rows : c->frames, c->mask_row))
    return fail(MAFAT_EUNSUPPORTED, "an extent of 2^58 or more");
  const int splits = plan_cross(*c).splits;
  *bytes = splits > 1 ? (static_cast<size_t>(splits) * static_cast<size_t>(c->rows) * c->q_heads * (c->head_dim + 2) * 4 + 255) & ~size_t{255}
                      : 0;
  return MAFAT_OK;
}

// Heads and rows as one extent (strides in any order).
Span extent(const void* p, int64_t esz, int64_t d, std::initializer_list<std::pair<int64_t, int64_t>> axes) {
  int64_t n = d;
  for (const auto& a : axes)
    if (a.first > 0) n += (a.first - 1) * a.second;
  return {p, 1, n * esz, n * esz};
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
    if (x_stride >= kMaxLinearCols || w_stride >= kMaxLinearCols || y_stride >= kMax31 || !fits(rows, y_stride))
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
      if (!workspace || !aligned(workspace, 256))
        return fail(MAFAT_EINVAL, "workspace must be non-NULL and 256-byte aligned");
      const int64_t an = 2 * static_cast<int64_t>(d.count) * d.rank * in_cols, bn = 2 * static_cast<int64_t>(d.count) * d.rank * out_cols;
      const Span su{workspace, 1, static_cast<int64_t>(need), static_cast<int64_t>(need)};
      const Span others[] = {{d.a, 1, an, an}, {d.b, 1, bn, bn}, {d.factor, 1, 4 * int64_t{d.count}, 4 * int64_t{d.count}},
                             {d.of_row, 1, 4 * rows, 4 * rows}, {x, rows, in_cols, x_stride},
                             {w, out_cols, in_cols, w_stride}, {x_scale, 1, 4 * rows, 4 * rows},
                             {w_scale, 1, 4 * out_cols, 4 * out_cols}, {bias, 1, 4 * out_cols, 4 * out_cols}};
      for (const Span& o : others)
        if (overlap(sy, o) || overlap(su, o)) return fail(MAFAT_EINVAL, "y or the workspace overlaps an input");
      if (overlap(sy, su)) return fail(MAFAT_EINVAL, "y overlaps the workspace");
      if (ws_bytes < need)
        return fail(MAFAT_EWORKSPACE, "workspace " + std::to_string(ws_bytes) + " < " + std::to_string(need) + " bytes");
      a.a = static_cast<const uint16_t*>(d.a);
      a.b = static_cast<const uint16_t*>(d.b);
      a.factor = d.factor;
      a.of_row = d.of_row;
      a.u = static_cast<uint16_t*>(workspace);
      a.rank_pad = rank_padded(d.rank);
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

extern "C" int mafat_cross_workspace(const mafat_cross* c, size_t* bytes) {
  return guarded([&] {
    clear_error();
    if (!bytes) return fail(MAFAT_EINVAL, "bytes is NULL");
    return check_cross(c, bytes);
  });
}

extern "C" int mafat_cross_attention(const mafat_cross* c, const void* q, const void* k, const void* v,
                                     const int32_t* q_offsets, const int32_t* k_lengths, const unsigned char* mask,
                                     void* y, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    clear_error();
    size_t need = 0;
    const int rc = check_cross(c, &need);
    if (rc != MAFAT_OK) return rc;
    if (c->rows == 0) return static_cast<int>(MAFAT_OK);  // tensors of no rows may have no address
    if (!q_offsets && c->rows % c->frames) return fail(MAFAT_EINVAL, "rows must divide by frames without q_offsets");
    if (!q || !y || (c->positions > 0 && (!k || !v))) return fail(MAFAT_EINVAL, "q, k, v and y must be non-NULL");
    if (mask && c->mask_row < c->positions) return fail(MAFAT_EINVAL, "mask_row is smaller than positions");
    const int64_t esz = static_cast<int64_t>(elt_size(c->dtype)), d = c->head_dim;
    const size_t es = elt_size(c->dtype);
    if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(y, es) || !aligned(q_offsets, 4) ||
        !aligned(k_lengths, 4) || !aligned(lse, 4))
      return fail(MAFAT_EINVAL, "a pointer is not aligned to its elements");
    if (ws_bytes < need)
      return fail(MAFAT_EWORKSPACE, "workspace " + std::to_string(ws_bytes) + " < " + std::to_string(need) + " bytes");
    if (need > 0 && (!workspace || !aligned(workspace, 256)))
      return fail(MAFAT_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    const int64_t mask_rows = c->mask_by_row ? c->rows : c->frames, lse_bytes = 4 * c->rows * c->q_heads;
    const Span ins[] = {extent(q, esz, d, {{c->rows, c->q_row}, {c->q_heads, c->q_head}}),
                        extent(c->positions ? k : nullptr, esz, d,
                               {{c->frames, c->k_frame}, {c->positions, c->k_pos}, {c->kv_heads, c->k_head}}),
                        extent(c->positions ? v : nullptr, esz, d,
                               {{c->frames, c->v_frame}, {c->positions, c->v_pos}, {c->kv_heads, c->v_head}}),
                        {q_offsets, 1, 4 * (c->frames + int64_t{1}), 4}, {k_lengths, 1, 4 * int64_t{c->frames}, 4},
                        extent(c->positions ? mask : nullptr, 1, c->positions, {{mask_rows, c->mask_row}})};
    const Span outs[] = {extent(y, esz, d, {{c->rows, c->y_row}, {c->q_heads, c->y_head}}),
                         {lse, 1, lse_bytes, lse_bytes},
                         {need ? workspace : nullptr, 1, static_cast<int64_t>(need), static_cast<int64_t>(need)}};
    for (int i = 0; i < 3; ++i) {
      for (const Span& s : ins)
        if (overlap(outs[i], s)) return fail(MAFAT_EINVAL, "y, lse or the workspace overlaps an input");
      for (int j = 0; j < i; ++j)
        if (overlap(outs[i], outs[j])) return fail(MAFAT_EINVAL, "y, lse and the workspace overlap");
    }
    CrossArgs a{};
    a.q = q; a.k = k; a.v = v; a.q_offsets = q_offsets; a.k_lengths = k_lengths;
    a.mask = c->positions ? mask : nullptr;
    a.y = y; a.lse = lse; a.part = static_cast<float*>(workspace);
    a.q_row = c->q_row; a.q_head = c->q_head; a.k_frame = c->k_frame; a.k_pos = c->k_pos; a.k_head = c->k_head;
    a.v_frame = c->v_frame; a.v_pos = c->v_pos; a.v_head = c->v_head; a.y_row = c->y_row; a.y_head = c->y_head;
    a.mask_row = c->mask_row;
    a.frames = c->frames; a.rows = static_cast<int32_t>(c->rows); a.positions = static_cast<int32_t>(c->positions);
    a.q_heads = c->q_heads; a.kv_heads = c->kv_heads; a.group = c->q_heads / c->kv_heads; a.head_dim = c->head_dim;
    a.mask_by_row = c->mask_by_row ? 1 : 0;
    a.per_frame = static_cast<int32_t>(c->rows / c->frames);
    const CrossPlan plan = plan_cross(*c);
    a.splits = plan.splits;
    a.scale = base2_scale(c->scale);
    return launched(launch_cross(c->dtype, a, plan, static_cast<hipStream_t>(stream)), "cross attention");
  });
}
