// tokens.cpp -- C ABI of the reader's operators among a request's tokens
// (include/mafat_reader.h): rotary positions, linear attention with decays, norms
// around a block.  Checks of the arguments, choice of the work split, launches.
#include <cmath>
#include <string>

#include "reader.h"
#include "reader_checks.h"

namespace mafat {
namespace {

constexpr int64_t kMaxHeads = 65535;

bool known(int dtype) { return dtype == MAFAT_F32 || dtype == MAFAT_BF16; }

// The sizes and strides of a call; the workspace holds the states and factors
// of the segments that long requests are cut into.
int check_decay(const mafat_decay* c, size_t* bytes) {
  if (!c) return fail(MAFAT_EINVAL, "c is NULL");
  if (!known(c->dtype)) return fail(MAFAT_EUNSUPPORTED, "dtype must be F32 or BF16");
  if (c->requests < 1 || c->rows < 0 || c->slots < 0) return fail(MAFAT_EINVAL, "requests must be >= 1, rows and slots >= 0");
  if (c->kv_heads < 1 || c->q_heads < 1 || c->q_heads % c->kv_heads)
    return fail(MAFAT_EINVAL, "q_heads must be a multiple of kv_heads");
  if (c->key_dim < 1 || c->value_dim < 1) return fail(MAFAT_EINVAL, "key_dim and value_dim must be >= 1");
  if (c->key_dim > 256 || c->value_dim > 256) return fail(MAFAT_EUNSUPPORTED, "key_dim or value_dim above 256");
  if (!std::isfinite(c->scale)) return fail(MAFAT_EINVAL, "scale must be finite");
  const int64_t k = c->key_dim, v = c->value_dim;
  if (c->q_head < k || c->q_row < k || c->k_head < k || c->k_row < k || c->v_head < v || c->v_row < v || c->y_head < v || c->y_row < v)
    return fail(MAFAT_EINVAL, "a row or head stride is smaller than its head");
  if (c->decay_by_row && c->decay_row < c->kv_heads) return fail(MAFAT_EINVAL, "decay_row is smaller than kv_heads");
  if (c->slots > 0 && c->state_slot < c->kv_heads * k * v) return fail(MAFAT_EINVAL, "state_slot is smaller than a state");
  if (c->rows >= kMax31 / c->q_heads || c->requests >= kMax31 / c->kv_heads || c->kv_heads > kMaxHeads || c->slots >= kMax31)
    return fail(MAFAT_EUNSUPPORTED, "rows * q_heads, requests * kv_heads or slots of 2^31 or more, or more than 65535 kv_heads");
  const int64_t most = kMax31 / static_cast<int64_t>(elt_size(c->dtype));
  for (int64_t s : {c->q_row, c->q_head, c->k_row, c->k_head, c->v_row, c->v_head, c->y_row, c->y_head})
    if (s >= most) return fail(MAFAT_EUNSUPPORTED, "a row or head stride of 2^31 bytes or more");
  if ((c->decay_by_row && c->decay_row >= kMax31) || !fits(c->slots, c->state_slot))
    return fail(MAFAT_EUNSUPPORTED, "a stride of the decays or states that is too large");
  const DecayPlan p = plan_decay(*c);
  *bytes = 0;
  if (p.split) {
    const int64_t states = p.segments * c->kv_heads;
    if (states >= kMax31) return fail(MAFAT_EUNSUPPORTED, "2^31 or more segments of requests and heads");
    // (states of 2^16 floats and a factor at most)
    *bytes = (static_cast<size_t>(states) * static_cast<size_t>(k * v + 1) * 4 + 255) & ~size_t{255};
  }
  return MAFAT_OK;
}

}  // namespace
}  // namespace mafat

using namespace mafat;

extern "C" int mafat_rotary(const mafat_turns* c, const int32_t* positions, const double* turns, const void* q, const void* k,
                            void* qy, void* ky, void* stream) {
  return guarded([&] {
    clear_error();
    if (!c) return fail(MAFAT_EINVAL, "c is NULL");
    if (!known(c->dtype)) return fail(MAFAT_EUNSUPPORTED, "dtype must be F32 or BF16");
    if (c->rows < 0 || c->q_heads < 1 || c->k_heads < 0) return fail(MAFAT_EINVAL, "rows and k_heads must be >= 0, q_heads >= 1");
    if (c->axes < 1 || c->axes > 4) return fail(MAFAT_EINVAL, "axes must be 1 .. 4");
    if (c->head_dim < 1 || c->pairs < 0 || c->pairs > c->head_dim / 2)
      return fail(MAFAT_EINVAL, "head_dim must be >= 1 and hold the pairs");
    if (c->head_dim > 1024) return fail(MAFAT_EUNSUPPORTED, "head_dim above 1024");
    if (!std::isfinite(c->magnitude)) return fail(MAFAT_EINVAL, "magnitude must be finite");
    if (c->rows >= kMax31 || c->q_heads > kMaxHeads || c->k_heads > kMaxHeads)
      return fail(MAFAT_EUNSUPPORTED, "rows of 2^31 or more, or more than 65535 heads");
    const int64_t d = c->head_dim;
    const bool has_k = c->k_heads > 0;
    if (c->q_row < d || c->q_head < d || c->qy_row < d || c->qy_head < d ||
        (has_k && (c->k_row < d || c->k_head < d || c->ky_row < d || c->ky_head < d)))
      return fail(MAFAT_EINVAL, "a row or head stride is smaller than head_dim");
    for (int64_t s : {c->q_row, c->q_head, c->qy_row, c->qy_head})
      if (s >= kMax31) return fail(MAFAT_EUNSUPPORTED, "a stride of 2^31 or more");
    if (has_k)
      for (int64_t s : {c->k_row, c->k_head, c->ky_row, c->ky_head})
        if (s >= kMax31) return fail(MAFAT_EUNSUPPORTED, "a stride of 2^31 or more");
    if (c->rows == 0) return static_cast<int>(MAFAT_OK);  // tensors of no rows may have no address
    if (!positions || !q || !qy || (c->pairs > 0 && !turns)) return fail(MAFAT_EINVAL, "positions, turns, q and qy must be non-NULL");
    if (has_k != (k != nullptr) || has_k != (ky != nullptr)) return fail(MAFAT_EINVAL, "k and ky go with k_heads, and with no others");
    const size_t es = elt_size(c->dtype);
    if (!aligned(q, es) || !aligned(k, es) || !aligned(qy, es) || !aligned(ky, es) || !aligned(positions, 4) || !aligned(turns, 8))
      return fail(MAFAT_EINVAL, "a pointer is not aligned to its elements");
    const int64_t esz = static_cast<int64_t>(es);
    const bool q_in = q == qy && (c->rows == 1 || c->q_row == c->qy_row) && (c->q_heads == 1 || c->q_head == c->qy_head);
    const bool k_in = has_k && k == ky && (c->rows == 1 || c->k_row == c->ky_row) && (c->k_heads == 1 || c->k_head == c->ky_head);
    const Heads hq{q, esz, d, c->rows, c->q_row, c->q_heads, c->q_head}, ho{qy, esz, d, c->rows, c->qy_row, c->q_heads, c->qy_head};
    const Heads hk{k, esz, d, c->rows, c->k_row, c->k_heads, c->k_head}, hy{ky, esz, d, c->rows, c->ky_row, c->k_heads, c->ky_head};
    const int64_t pn = 4 * c->rows * c->axes, tn = 8 * int64_t{c->axes} * c->pairs;
    const Span sp{positions, 1, pn, pn}, st{c->pairs ? turns : nullptr, 1, tn, tn};
    if ((!q_in && heads_overlap(ho, hq)) || overlap(ho.span(), sp) || overlap(ho.span(), st) ||
        (has_k && ((!k_in && heads_overlap(hy, hk)) || heads_overlap(ho, hk) || (!(q_in && k_in) && (heads_overlap(hy, hq) || heads_overlap(ho, hy))) ||
                   overlap(hy.span(), sp) || overlap(hy.span(), st))))
      return fail(MAFAT_EINVAL, "an output overlaps another tensor without being its own input");
    if (heads_collide(ho) || (has_k && heads_collide(hy))) return fail(MAFAT_EINVAL, "heads of an output overlap each other");
    RotaryArgs a{};
    a.positions = positions;
    a.turns = turns;
    a.in[0] = q; a.in[1] = k; a.out[0] = qy; a.out[1] = ky;
    a.in_row[0] = c->q_row; a.in_head[0] = c->q_head; a.out_row[0] = c->qy_row; a.out_head[0] = c->qy_head;
    if (has_k) {
      a.in_row[1] = c->k_row; a.in_head[1] = c->k_head; a.out_row[1] = c->ky_row; a.out_head[1] = c->ky_head;
    }
    a.rows = c->rows;
    a.axes = c->axes; a.q_heads = c->q_heads; a.heads = c->q_heads + c->k_heads; a.head_dim = c->head_dim; a.pairs = c->pairs;
    a.magnitude = c->magnitude;
    return launched(launch_rotary(c->dtype, c->interleaved != 0, q_in && (!has_k || k_in), a, static_cast<hipStream_t>(stream)),
                    "rotary");
  });
}

extern "C" int mafat_block_norm(const mafat_block* c, const void* x, const float* after_gain, const void* gate, const float* scale,
                                const void* residual, void* sum, const float* before_gain, void* y, float* y_scale,
                                void* stream) {
  return guarded([&] {
    clear_error();
    if (!c) return fail(MAFAT_EINVAL, "c is NULL");
    if (!known(c->dtype)) return fail(MAFAT_EUNSUPPORTED, "dtype must be F32 or BF16");
    if (!known(c->out_dtype) && c->out_dtype != MAFAT_F8) return fail(MAFAT_EUNSUPPORTED, "out_dtype must be F32, BF16 or F8");
    const int64_t rows = c->rows, cols = c->cols;
    if (rows < 0 || cols < 1) return fail(MAFAT_EINVAL, "rows must be >= 0 and cols >= 1");
    if (rows >= kMax31 || cols >= kMax31) return fail(MAFAT_EUNSUPPORTED, "2^31 or more rows or columns");
    if (c->groups < 1 || cols % c->groups) return fail(MAFAT_EINVAL, "groups must be >= 1 and divide cols");
    if (c->groups > 4096) return fail(MAFAT_EUNSUPPORTED, "more than 4096 groups");
    if (!(c->eps >= 0.f) || !std::isfinite(c->eps)) return fail(MAFAT_EINVAL, "eps must be finite and not negative");
    if (rows == 0) return static_cast<int>(MAFAT_OK);  // tensors of no rows may have no address
    if (!residual != !sum) return fail(MAFAT_EINVAL, "residual and sum go together");
    if ((after_gain && !c->after) || (before_gain && !c->before)) return fail(MAFAT_EINVAL, "a gain without its norm");
    if ((c->out_dtype == MAFAT_F8) != (y_scale != nullptr))
      return fail(MAFAT_EINVAL, "y_scale goes with 8-bit output, and with no other");
    if (c->x_stride < cols || c->y_stride < cols || (gate && c->gate_stride < cols) ||
        (residual && (c->residual_stride < cols || c->sum_stride < cols)))
      return fail(MAFAT_EINVAL, "a stride is smaller than cols");
    if (c->x_stride >= kMax31 || c->y_stride >= kMax31 || (gate && c->gate_stride >= kMax31) ||
        (residual && (c->residual_stride >= kMax31 || c->sum_stride >= kMax31)))
      return fail(MAFAT_EUNSUPPORTED, "a stride of 2^31 or more");
    const size_t in = elt_size(c->dtype), out = elt_size(c->out_dtype);
    if (!x || !y) return fail(MAFAT_EINVAL, "x and y must be non-NULL");
    if (!aligned(x, in) || !aligned(gate, in) || !aligned(residual, in) || !aligned(sum, in) || !aligned(y, out) ||
        !aligned(after_gain, 4) || !aligned(scale, 4) || !aligned(before_gain, 4) || !aligned(y_scale, 4))
      return fail(MAFAT_EINVAL, "a pointer is not aligned to its elements");
    const int64_t isz = static_cast<int64_t>(in), osz = static_cast<int64_t>(out);
    const Span ins[] = {{x, rows, cols * isz, c->x_stride * isz}, {gate, rows, cols * isz, c->gate_stride * isz},
                        {residual, rows, cols * isz, c->residual_stride * isz}, {after_gain, 1, 4 * cols, 4 * cols},
                        {scale, 1, 4 * cols, 4 * cols}, {before_gain, 1, 4 * cols, 4 * cols}};
    const Span outs[] = {{y, rows, cols * osz, c->y_stride * osz}, {sum, rows, cols * isz, c->sum_stride * isz},
                         {y_scale, 1, 4 * rows, 4 * rows}};
    for (int i = 0; i < 3; ++i) {
      for (const Span& s : ins)
        if (overlap(outs[i], s)) return fail(MAFAT_EINVAL, "an output overlaps an input");
      for (int j = 0; j < i; ++j)
        if (overlap(outs[i], outs[j])) return fail(MAFAT_EINVAL, "outputs overlap");
    }
    BlockArgs a{};
    a.x = x; a.gate = gate; a.res = residual; a.after_gain = after_gain; a.scale = scale; a.before_gain = before_gain;
    a.sum = sum; a.y = y; a.y_scale = y_scale;
    a.x_stride = c->x_stride; a.gate_stride = c->gate_stride; a.res_stride = c->residual_stride;
    a.sum_stride = c->sum_stride; a.y_stride = c->y_stride;
    a.rows = rows; a.cols = static_cast<int32_t>(cols);
    a.groups = c->after ? c->groups : 1;
    a.part = a.cols / a.groups;
    a.per_col = 1.f / static_cast<float>(a.cols);
    a.per_part = 1.f / static_cast<float>(a.part);
    a.after = c->after != 0; a.before = c->before != 0; a.silu = c->gate_act != 0; a.eps = c->eps;
    return launched(launch_block_norm(c->dtype, c->out_dtype, a, static_cast<hipStream_t>(stream)), "block norm");
  });
}

extern "C" int mafat_decay_workspace(const mafat_decay* c, size_t* bytes) {
  return guarded([&] {
    clear_error();
    if (!bytes) return fail(MAFAT_EINVAL, "bytes is NULL");
    return check_decay(c, bytes);
  });
}

extern "C" int mafat_decay_attention(const mafat_decay* c, const void* q, const void* k, const void* v, const float* log_decay,
                                     const int32_t* offsets, float* states, const int32_t* slots, void* y, void* workspace,
                                     size_t ws_bytes, void* stream) {
  return guarded([&] {
    clear_error();
    size_t need = 0;
    const int rc = check_decay(c, &need);
    if (rc != MAFAT_OK) return rc;
    if (c->rows == 0) return static_cast<int>(MAFAT_OK);  // tensors of no rows may have no address
    if (!offsets && c->rows % c->requests) return fail(MAFAT_EINVAL, "rows must divide by requests without offsets");
    if (!q || !k || !v || !log_decay || !y) return fail(MAFAT_EINVAL, "q, k, v, log_decay and y must be non-NULL");
    if (slots && !states) return fail(MAFAT_EINVAL, "slots without states");
    const size_t es = elt_size(c->dtype);
    if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(y, es) || !aligned(log_decay, 4) || !aligned(offsets, 4) ||
        !aligned(states, 4) || !aligned(slots, 4))
      return fail(MAFAT_EINVAL, "a pointer is not aligned to its elements");
    if (ws_bytes < need)
      return fail(MAFAT_EWORKSPACE, "workspace " + std::to_string(ws_bytes) + " < " + std::to_string(need) + " bytes");
    if (need > 0 && (!workspace || !aligned(workspace, 256)))
      return fail(MAFAT_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    const int64_t esz = static_cast<int64_t>(es), size = int64_t{c->kv_heads} * c->key_dim * c->value_dim;
    const int64_t dn = 4 * (c->decay_by_row ? (c->rows - 1) * c->decay_row + c->kv_heads : int64_t{c->kv_heads});
    const int64_t on = 4 * (c->requests + int64_t{1}), sn = 4 * int64_t{c->requests};
    const Heads heads[] = {{q, esz, c->key_dim, c->rows, c->q_row, c->q_heads, c->q_head},
                           {k, esz, c->key_dim, c->rows, c->k_row, c->kv_heads, c->k_head},
                           {v, esz, c->value_dim, c->rows, c->v_row, c->kv_heads, c->v_head}};
    const Heads hy{y, esz, c->value_dim, c->rows, c->y_row, c->q_heads, c->y_head};
    const Span ins[] = {heads[0].span(), heads[1].span(), heads[2].span(), {log_decay, 1, dn, dn}, {offsets, 1, on, on}, {slots, 1, sn, sn}};
    const Span outs[] = {hy.span(), {c->slots > 0 ? states : nullptr, c->slots, 4 * size, 4 * c->state_slot},
                         {need ? workspace : nullptr, 1, static_cast<int64_t>(need), static_cast<int64_t>(need)}};
    for (int i = 0; i < 3; ++i) {
      for (int j = 0; j < 6; ++j)
        if (i == 0 && j < 3 ? heads_overlap(hy, heads[j]) : overlap(outs[i], ins[j]))
          return fail(MAFAT_EINVAL, "y, the states or the workspace overlaps an input");
      for (int j = 0; j < i; ++j)
        if (overlap(outs[i], outs[j])) return fail(MAFAT_EINVAL, "y, the states and the workspace overlap");
    }
    if (heads_collide(hy)) return fail(MAFAT_EINVAL, "heads of y overlap each other");
    DecayArgs a{};
    const DecayPlan p = plan_decay(*c);
    a.q = q; a.k = k; a.v = v; a.log_decay = log_decay; a.offsets = offsets;
    a.states = c->slots > 0 ? states : nullptr; a.slots = slots; a.y = y;
    a.part = static_cast<float*>(workspace);
    a.q_row = c->q_row; a.q_head = c->q_head; a.k_row = c->k_row; a.k_head = c->k_head; a.v_row = c->v_row; a.v_head = c->v_head;
    a.y_row = c->y_row; a.y_head = c->y_head; a.decay_row = c->decay_row; a.state_slot = c->state_slot;
    a.pool = c->slots;
    a.requests = c->requests; a.rows = static_cast<int32_t>(c->rows); a.q_heads = c->q_heads; a.kv_heads = c->kv_heads;
    a.group = c->q_heads / c->kv_heads; a.key_dim = c->key_dim; a.value_dim = c->value_dim;
    a.per_request = static_cast<int32_t>(c->rows / c->requests);
    a.decay_by_row = c->decay_by_row != 0;
    a.segment = static_cast<int32_t>(p.split ? p.segment : c->rows);
    a.segments = static_cast<int32_t>(p.split ? p.segments : c->requests);
    if (!offsets)  // known, and no more than that
      a.segments = static_cast<int32_t>(c->requests * ((int64_t{a.per_request} + a.segment - 1) / a.segment));
    if (p.split) a.factor = a.part + p.segments * size;
    a.scale = c->scale;
    return launched(launch_decay(c->dtype, a, p, static_cast<hipStream_t>(stream)), "decay attention");
  });
}
