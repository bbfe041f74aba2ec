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

#ifdef __cplusplus
}
#endif
#endif
