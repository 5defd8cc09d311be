/*
 * rkc_packed.h -- C ABI of the rows of a paged KV cache, in 16 bits (rkc_cache.h) or held in 4, MI355X (gfx950).
 *
 *   rkc_store, rkc_packed_store   norm and rotation of new rows' queries and keys; keys and values into their slots
 *   rkc_read, rkc_packed_read     slots back into rows of 16 bits
 *   rkc_packed_attend             rkc_attend over a cache of 4 bits
 *
 * Ownership, errors, streams and the checks of what lies in device memory are those of rkc_cache.h.
 *
 * The 4 bits are a sign, two bits of exponent and one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4 and 6 for the codes 0 to 7, the
 * negatives for 8 to 15.  32 consecutive elements of a head share a scale 2^(b - 127), b a byte: the least scale with which
 * none of them is past 7, within b = 1 .. 252 (bfloat16) or 140 (float16); what is past 7 times the largest scale is held
 * as 6 times that.  Elements are rounded to the nearest value, halves to the even code.
 * A head of a slot of which a key's or value's element is not finite is marked by a scale byte of 255, the first of its
 * key: it is read back as NaN whole, and rows that see it get NaN for that head; rows that do not see it do not.
 */
#ifndef RKC_PACKED_H
#define RKC_PACKED_H

#include "rkc_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RKC_MAX_AXES 8

/* A cache in 4 bits: host struct.  Head h of block b is  page_tokens * (head_dim + head_dim / 16)  bytes from
 * b * block_stride + h * head_stride on: keys [slot][head_dim / 2] (the lower four bits are the earlier element), values
 * likewise, the keys' scales [slot][head_dim / 32], the values' scales. */
typedef struct rkc_packed {
  int32_t n_seqs;
  int32_t n_blocks;
  int32_t max_pages;
  int32_t page_tokens; /* 16, 32, 64, ... 1024                                                       */
  int32_t kv_heads;
  int32_t head_dim;    /* 64, 128 or 256                                                             */
  int32_t dtype;       /* enum rkc_dtype, of queries, rows and outputs                               */
  int32_t reserved;    /* must be 0                                                                  */
  int64_t block_stride, head_stride; /* bytes, multiples of 16; blocks < 2^32 apart                  */
  void* d_pool;                      /* 16-byte aligned                                              */
  const int32_t* d_block_table;      /* [n_seqs * max_pages]                                         */
  int32_t* d_status;                 /* [n_seqs], bits OR'ed in (the caller clears), or NULL         */
} rkc_packed;

/* Rows: host struct.  Rows of sequence s are [d_row_offset[s], d_row_offset[s+1]); with n of them they are those of its last
 * n slots of d_length[s].  Rows behind the last sequence, and those of a sequence told of by RKC_CS_LENGTH, are left alone.
 * Offsets go up: a sequence whose rows end before they begin is told of, and of rows that two others claim one has them.
 * A row of a block id outside the pool is not stored, and reads block 0 (RKC_CS_BLOCK).
 *
 * Stored rows: a head's queries and keys are multiplied by  norm[i] / sqrt(mean of squares + eps)  where there is a norm, then
 * pairs j < n_freq turn by the angle d_freq[j] * position: elements j and j + n_freq, or 2 j and 2 j + 1 where interleaved;
 * (a, b) becomes (a cos - b sin, a sin + b cos).  The position is that of axis d_axis[j] of the row, of one outside
 * [0, axes) that of axis 0; without d_position the slot's number.  Values, and elements from 2 n_freq on, do not turn.
 * Two rows of one call must not have the same slot.
 * Read rows: d_k and d_v are written; the fields of queries, norm and rotation are not used.
 * What is written shares no element with other rows of the call (d_k and d_v read, d_q_out and the rows stored). */
typedef struct rkc_rows {
  int32_t n_rows;
  int32_t q_heads;     /* where there are queries: any number up to 65536                            */
  int32_t max_len;     /* >= every sequence's length, <= max_pages * page_tokens                     */
  int32_t n_freq;      /* pairs that turn: a multiple of 8 up to head_dim / 2; 0: no rotation        */
  int32_t axes;        /* positions of a row, 1 .. RKC_MAX_AXES (with d_position)                    */
  int32_t interleaved; /* 0 or 1                                                                     */
  int32_t norm_f32;    /* the norms' weights are float (1) or of the cache's type (0)                */
  float eps;           /* >= 0                                                                       */
  int64_t k_row_stride, k_head_stride, v_row_stride, v_head_stride;         /* elements, multiples of 8 */
  int64_t q_row_stride, q_head_stride, q_out_row_stride, q_out_head_stride; /* elements, multiples of 8 */
  void* d_k;                   /* [n_rows][kv_heads][head_dim], 16-byte aligned; read by a store     */
  void* d_v;                   /* the same                                                           */
  const void* d_q;             /* [n_rows][q_heads][head_dim] or NULL, 16-byte aligned               */
  void* d_q_out;               /* the same; may be d_q with its strides                              */
  const int32_t* d_row_offset; /* [n_seqs + 1]                                                       */
  const int32_t* d_length;     /* [n_seqs]                                                           */
  const int32_t* d_position;   /* [axes][n_rows] or NULL                                             */
  const int32_t* d_axis;       /* [n_freq] or NULL (axes is 1)                                       */
  const float* d_freq;         /* [n_freq]                                                           */
  const void* d_q_norm;        /* [head_dim] or NULL                                                 */
  const void* d_k_norm;        /* [head_dim] or NULL                                                 */
} rkc_rows;

rkc_status rkc_store(const rkc_cache* c, const rkc_rows* r, void* s);
rkc_status rkc_read(const rkc_cache* c, const rkc_rows* r, void* s);
rkc_status rkc_packed_store(const rkc_packed* c, const rkc_rows* r, void* s);
rkc_status rkc_packed_read(const rkc_packed* c, const rkc_rows* r, void* s);

/* Attention over a cache of 4 bits: as rkc_attend.  There is no account (d_weight_in and d_weight must be NULL).
 * The products' operands have 16 bits, as there.  A value held is one of them (of float16: to the nearest multiple of 2^-24).  The
 * softmax's weights are rounded to the cache's type where max_rows x query heads of a key/value head is more than 16, and keep twice
 * its bits up to that; scores, maxima, sums and outputs up to the end are of 32 bits. */
size_t rkc_packed_attend_scratch_bytes(const rkc_packed* c, const rkc_attention* a);
rkc_status rkc_packed_attend(const rkc_packed* c, const rkc_attention* a, void* s);

#ifdef __cplusplus
}
#endif

#endif /* RKC_PACKED_H */
