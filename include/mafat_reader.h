/*
 * mafat_reader.h -- C ABI of the operators of a reader: a decoder whose
 * tokens, of many requests at once, read the feature maps that a plan's
 * network (mafat.h) leaves on the device.  They are not part of the paper's
 * method; they consume its output where it lies.  Forward only.
 *
 *   mafat_add_rms_norm     residual addition and root-mean-square norm, into
 *                          float32, bfloat16 or 8 bits with a scale per row
 *   mafat_linear           projection of 8-bit rows by 8-bit weights, with
 *                          low-rank adapters of the requests beside it
 *   mafat_cross_attention  attention of the requests' tokens to the positions
 *                          of the frames they are about
 *   mafat_rotary           positions of queries and keys as rotations
 *   mafat_decay_attention  linear attention among the tokens of a request, with
 *                          a decay for each head and a state that is kept
 *   mafat_block_norm       norms after and before a block with its gate, its
 *                          residual scale and the residual addition
 *
 * Conventions of mafat.h hold: device buffers are the caller's, run functions
 * enqueue kernels on the given stream and return, no device memory is
 * allocated, nothing synchronises, no exception leaves, equal calls give
 * equal bits.  Strides are in elements and may leave gaps; the last axis is
 * contiguous.  Pointers need the alignment of their elements only; rows of
 * 16-byte alignment run fastest.  Sizes of zero rows are valid and enqueue
 * nothing.  Integer inputs on the device (lengths, offsets, adapter
 * numbers) are not read on the host: out-of-range values are clamped or
 * ignored as stated and never lead outside a buffer.
 *
 * MAFAT_F8 is the 8-bit float of 4 exponent and 3 mantissa bits with largest
 * value 448 and no infinities (OCP e4m3).
 */
#ifndef MAFAT_READER_H
#define MAFAT_READER_H

#include "mafat.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { MAFAT_F8 = 2 };

/* h = x + residual, rounded to dtype and written to sum; without a residual
 * (residual and sum NULL) h = x.  Then, per row,
 *   y = h * (mean(h^2) + eps)^(-1/2) * gain
 * with the mean over cols in float32.  out_dtype MAFAT_F8: y_scale[row] =
 * max |y| / 448 and y holds y / y_scale rounded to nearest even; a row whose
 * largest magnitude is below 2^-100 (one of zeros) gets scale 1.  A row with
 * a NaN gets NaN outputs and a NaN scale.
 *   x, residual, sum   rows x cols in dtype (MAFAT_F32 or MAFAT_BF16)
 *   gain               float32[cols], or NULL (ones)
 *   y                  rows x cols in out_dtype (MAFAT_F32, MAFAT_BF16, MAFAT_F8)
 *   y_scale            float32[rows] for MAFAT_F8, else NULL
 * sum may be x or residual itself (with its stride); otherwise outputs may
 * not overlap inputs or each other.  Errors: EINVAL (null or misaligned
 * pointer, negative size, cols < 1, stride below cols, one of residual and
 * sum without the other, a scale pointer that does not match out_dtype,
 * overlap, eps negative or not finite), EUNSUPPORTED (dtype; rows or cols of
 * 2^31 or more), EHIP. */
int mafat_add_rms_norm(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t x_stride,
                       const void* residual, int64_t residual_stride, const float* gain, float eps,
                       void* sum, int64_t sum_stride, int32_t out_dtype, void* y, int64_t y_stride,
                       float* y_scale, void* stream);

/* Low-rank adapters of mafat_linear: adapter i adds, to the rows that name
 * it, factor[i] * b[i] (a[i] x).
 *   a       bfloat16 [count][rank][in_cols], contiguous
 *   b       bfloat16 [count][out_cols][rank], contiguous
 *   factor  float32 [count], or NULL (ones)
 *   of_row  int32 [rows]: each row's adapter; any value outside
 *           [0, count) is none
 * All on the device; 1 <= rank <= 128. */
typedef struct {
  int32_t count, rank;
  const void* a;
  const void* b;
  const float* factor;
  const int32_t* of_row;
} mafat_adapters;

/* y[i][j] = x_scale[i] * w_scale[j] * sum_k x[i][k] w[j][k] + bias[j], plus
 * the row's adapter on the values x stands for, in bfloat16.
 *   x        8 bits [rows][in_cols], w 8 bits [out_cols][in_cols]
 *   x_scale  float32[rows], w_scale float32[out_cols]
 *   bias     float32[out_cols], or NULL
 *   adapters a host struct, read during the call, or NULL
 *   workspace  mafat_linear_workspace bytes, 256-byte aligned (NULL if 0)
 * Sums are float32.  The 8-bit matrix instructions align the products of a
 * step before they add them: a sum is 1.5e-5 from the exact one on average and
 * below 1e-4 singly, relative to the root of the sum of its squared products.
 * in_cols, strides and addresses of x and w in whole 16 bytes run an order of
 * magnitude faster than others where rows are many.  Errors: EINVAL
 * (null or misaligned pointer, negative size, in_cols or out_cols < 1,
 * stride below the row length, bad adapters, y overlapping an input),
 * EWORKSPACE, EUNSUPPORTED (rank > 128, sizes or a stride of 2^22 or more
 * columns, 2^31 or more rows), EHIP. */
int mafat_linear_workspace(int64_t rows, int64_t in_cols, int64_t out_cols,
                           const mafat_adapters* adapters, size_t* bytes);
int mafat_linear(int64_t rows, int64_t in_cols, int64_t out_cols, const void* x, int64_t x_stride,
                 const float* x_scale, const void* w, int64_t w_stride, const float* w_scale,
                 const float* bias, const mafat_adapters* adapters, void* y, int64_t y_stride,
                 void* workspace, size_t ws_bytes, void* stream);

/* Sizes and strides of mafat_cross_attention.  Query rows are those of all
 * requests about all frames, frame by frame; every query head h reads the
 * keys and values of head h / (q_heads / kv_heads). */
typedef struct {
  int32_t dtype;              /* MAFAT_F32 or MAFAT_BF16: q, k, v and y */
  int32_t frames;             /* key/value sequences */
  int64_t rows;               /* query rows of all frames together */
  int64_t positions;          /* positions of a frame's k and v */
  int32_t q_heads, kv_heads;  /* q_heads a multiple of kv_heads */
  int32_t head_dim;           /* 1 .. 256, of keys and of values */
  float scale;                /* of q . k */
  int64_t q_row, q_head;      /* strides of q */
  int64_t k_frame, k_pos, k_head;
  int64_t v_frame, v_pos, v_head;
  int64_t y_row, y_head;
  int64_t mask_row;           /* bytes between rows of the mask */
  int32_t mask_by_row;        /* 0: a mask row per frame; 1: per query row */
} mafat_cross;

/* For every query row i of frame f and head h, over the frame's valid
 * positions s (s < k_lengths[f], and allowed by the mask):
 *   p_s = softmax_s(scale * q[i][h] . k[f][s][h'])
 *   y[i][h] = sum_s p_s v[f][s][h'],  lse[i][h] = log sum_s exp(scale * ...)
 * A row that no position is valid for gets y = 0 and lse = -infinity.  Scores
 * (scale times product) are float32: one that is -infinity has p = 0, also
 * where a row has no other (y = 0 and lse = -infinity then), and one that is
 * +infinity or NaN makes its row NaN.  Keys
 * and values of positions that are not valid for any row of a frame by its
 * length or its mask may hold anything, NaN included.
 *   q_offsets  int32[frames + 1], not decreasing, each clamped to [0, rows]:
 *              frame f's rows are [q_offsets[f], q_offsets[f + 1]); rows that
 *              no frame has are not written.  (Offsets that decrease leave it
 *              open which rows are computed.)  NULL: rows / frames each (rows
 *              must divide)
 *   k_lengths  int32[frames], clamped to [0, positions]; NULL: positions
 *   mask       bytes, nonzero where a position may be read; [frames or
 *              rows][positions] by mask_by_row; or NULL
 *   y          [rows][q_heads][head_dim] in dtype;  lse float32 [rows][q_heads]
 *              contiguous, natural logarithm, or NULL
 *   workspace  mafat_cross_workspace bytes, 256-byte aligned (NULL if 0)
 * Softmax statistics and sums are float32.  In bfloat16 the exponentials enter
 * the second product as the sum of two bfloat16 parts (16 bits) where a frame
 * has up to 64 pairs of a row and a head that share a key/value head (rows /
 * frames counted alike), or where head_dim, or an address or stride of k or v,
 * is no multiple of 16 bytes, or scale is 0; else rounded to bfloat16, each by its own size.
 * So, and because rows of a wave rescale their sums together, the last bits of
 * a row may depend on the rows that share its call.  Errors: EINVAL
 * (null or misaligned pointer, bad size or stride, rows not divisible without
 * q_offsets, scale not finite, y overlapping an input), EWORKSPACE,
 * EUNSUPPORTED (dtype, head_dim > 256, sizes of 2^31 or more, strides of 2^31
 * bytes or more, a scale above 2.35e38 either way, which overflows in base 2),
 * EHIP. */
int mafat_cross_workspace(const mafat_cross* c, size_t* bytes);
int mafat_cross_attention(const mafat_cross* c, const void* q, const void* k, const void* v,
                          const int32_t* q_offsets, const int32_t* k_lengths, const unsigned char* mask,
                          void* y, float* lse, void* workspace, size_t ws_bytes, void* stream);

/* Sizes and strides of mafat_rotary.  y: where the turned values go. */
typedef struct {
  int32_t dtype;               /* MAFAT_F32 or MAFAT_BF16: q, k and their outputs */
  int32_t axes;                /* numbers of a position: 1 .. 4 */
  int64_t rows;
  int32_t q_heads, k_heads;    /* k_heads 0: no k */
  int32_t head_dim;            /* 1 .. 1024 */
  int32_t pairs;               /* the first 2 * pairs values of a head turn */
  int32_t interleaved;         /* pair i: 0: values i and pairs + i; 1: values 2 i and 2 i + 1 */
  float magnitude;             /* of the turned values */
  int64_t q_row, q_head, k_row, k_head;
  int64_t qy_row, qy_head, ky_row, ky_head;
} mafat_turns;

/* For every row r, head and pair i, with t = sum_a positions[r][a] * turns[a][i]
 * (in turns, so angles are 2 pi t):
 *   (x1, x2) -> magnitude * (x1 cos - x2 sin, x2 cos + x1 sin)
 * and the values of a head behind its pairs as they are.
 *   positions  int32 [rows][axes], contiguous; negative ones turn back
 *   turns      float64 [axes][pairs], contiguous: turns per step, for instance
 *              base^(-i / pairs) / (2 pi)
 *   qy, ky     may be q and k themselves (with their strides); otherwise outputs
 *              may not overlap inputs or each other.  Tensors of one pair of
 *              strides may lie between each other in any order
 * t is formed and brought below half a turn in float64, its sine and cosine in
 * float32: far positions keep the accuracy of near ones.  Errors: EINVAL (null
 * or misaligned pointer, negative rows or heads, axes outside 1 .. 4, pairs < 0
 * or 2 * pairs > head_dim, stride below head_dim, magnitude not finite,
 * overlap, also of an output's own heads), EUNSUPPORTED (dtype, head_dim > 1024, rows of 2^31 or more, more
 * than 65535 heads, strides of 2^31 or more), EHIP. */
int mafat_rotary(const mafat_turns* c, const int32_t* positions, const double* turns, const void* q, const void* k,
                 void* qy, void* ky, void* stream);

/* Sizes and strides of mafat_block_norm.  After and before: of the block whose
 * output is x, and of the next one. */
typedef struct {
  int32_t dtype;        /* MAFAT_F32 or MAFAT_BF16: x, gate, residual and sum */
  int32_t out_dtype;    /* MAFAT_F32, MAFAT_BF16 or MAFAT_F8: y */
  int64_t rows, cols;
  int32_t after;        /* norm x, in `groups` equal parts of a row */
  int32_t groups;       /* 1 .. 4096, divides cols */
  int32_t gate_act;     /* of the gate: 0 sigmoid, 1 gate * sigmoid(gate) */
  int32_t before;       /* norm the sum */
  float eps;
  int64_t x_stride, gate_stride, residual_stride, sum_stride, y_stride;
} mafat_block;

/* Per row:
 *   u = x * (mean of its part (x^2) + eps)^(-1/2) * after_gain    if after
 *   u = u * act(gate)                                             with a gate
 *   h = residual + scale * u          (scale 1 and residual 0 without them)
 *   y = h * (mean(h^2) + eps)^(-1/2) * before_gain                if before
 * in float32 throughout: sum is h rounded to dtype, y follows from h before that
 * rounding.  y and y_scale as in mafat_add_rms_norm.
 *   x, gate, residual, sum   rows x cols in dtype; gate NULL: none; residual
 *                            and sum go together, or are NULL
 *   after_gain, scale, before_gain   float32[cols], or NULL (ones)
 *   y, y_scale               rows x cols in out_dtype, float32[rows] for MAFAT_F8
 * Outputs may not overlap inputs or each other.  Errors: EINVAL (null or
 * misaligned pointer, negative rows, cols < 1, groups that do not divide cols, a
 * gain without its norm, stride below cols, one of residual and sum without
 * the other, a scale pointer that does not match out_dtype, overlap, eps
 * negative or not finite), EUNSUPPORTED (dtype; rows, cols or a stride of 2^31 or
 * more, groups > 4096), EHIP. */
int mafat_block_norm(const mafat_block* c, const void* x, const float* after_gain, const void* gate, const float* scale,
                     const void* residual, void* sum, const float* before_gain, void* y, float* y_scale, void* stream);

/* Sizes and strides of mafat_decay_attention.  Rows are the tokens of all
 * requests, request by request; every query head h reads the keys, values and
 * states of head h / (q_heads / kv_heads). */
typedef struct {
  int32_t dtype;              /* MAFAT_F32 or MAFAT_BF16: q, k, v and y */
  int32_t requests;
  int64_t rows;               /* tokens of all requests together */
  int64_t slots;              /* states in the pool */
  int32_t q_heads, kv_heads;  /* q_heads a multiple of kv_heads */
  int32_t key_dim, value_dim; /* 1 .. 256 each */
  float scale;
  int32_t decay_by_row;       /* 0: log_decay [kv_heads]; 1: [rows][kv_heads] */
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, y_row, y_head;
  int64_t decay_row;          /* between rows of log_decay, if by row */
  int64_t state_slot;         /* between states of the pool */
} mafat_decay;

/* For every request, its tokens t = 1, 2, ... in order, and every key/value head:
 *   S_t = exp(log_decay_t) S_{t-1} + k_t v_t^T      (key_dim x value_dim)
 *   y_t = scale * q_t S_t                           for the query heads of it
 * where S_0 is the request's state in the pool, which ends up as the last S.
 *   log_decay  float32; above 0 counts as 0, below -138 (a factor that float32
 *              ends at) as -138; NaN makes what follows NaN
 *   offsets    int32[requests + 1], not decreasing, each clamped to [0, rows]:
 *              request i's rows are [offsets[i], offsets[i + 1]); rows that no
 *              request has are not written, and requests without rows leave their
 *              state.  (Offsets that decrease leave it open which rows are
 *              computed.)  NULL: rows / requests each (rows must divide)
 *   states     float32 [slots][kv_heads][key_dim][value_dim], the last three
 *              contiguous, updated in place; NULL: every request starts from
 *              zeros and nothing is kept
 *   slots      int32[requests], each request's state; outside [0, slots): starts
 *              from zeros and is not kept.  A state belongs to the first request
 *              with rows that names it: later ones that name it too get y = NaN
 *              and do not change it.  NULL: request i has state i
 *   workspace  mafat_decay_workspace bytes, 256-byte aligned (NULL if 0)
 * States and sums are float32.  Long requests are cut into segments whose states
 * are joined, so the last bits of a row may depend on the sizes of the call.  What is
 * not finite in a token reaches its own request's rows from that token on, and its
 * state.  In bfloat16, where heads, addresses and strides are whole 16 bytes and
 * requests have more than one row, scores, and states and values where they end in
 * an output, enter products as two bfloat16 parts each, which leave 2^-16 of a
 * term: outputs are off by their own rounding, whatever else is in the call.  The
 * states that are kept have float32's accuracy, but for 2^-102 of a key that a
 * value may lose.  Errors:
 * EINVAL (null or misaligned pointer, bad size or stride, rows not divisible
 * without offsets, scale not finite, an output overlapping another tensor, or y's
 * heads each other),
 * EWORKSPACE, EUNSUPPORTED (dtype, key_dim or value_dim > 256, rows * q_heads or
 * requests * kv_heads of 2^31 or more, or segments of long requests that make it so,
 * more than 65535 kv_heads, strides of 2^31 bytes or more), EHIP. */
int mafat_decay_workspace(const mafat_decay* c, size_t* bytes);
int mafat_decay_attention(const mafat_decay* c, const void* q, const void* k, const void* v, const float* log_decay,
                          const int32_t* offsets, float* states, const int32_t* slots, void* y, void* workspace,
                          size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
