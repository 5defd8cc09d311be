/*
 * rkc_cache.h -- C ABI of the operators on the contents of a paged KV cache, MI355X (gfx950).
 *
 * rkc.h replays what happens to the blocks of a pool; the functions here work on what the blocks hold:
 *   rkc_attend   attention of new rows over a cache: a prompt's chunk, or a tree of drafted tokens
 *   rkc_weigh    the account of a cache: how much attention each of its slots received
 *   rkc_evict    eviction by that account, which leaves a claim's leading slots alone
 *
 * A sequence's slots 0, 1, 2, ... lie in blocks of page_tokens slots, and the block table names the blocks in
 * order.  Keys are stored as attention reads them (position encodings applied), so the order of the slots
 * matters to the masks only.
 *
 * Ownership and errors are those of rkc.h: the caller owns every buffer, nothing is allocated, a call only
 * enqueues kernels on the stream, and a negative status means that nothing was enqueued (RKC_E_HIP, an error of
 * the runtime itself: that not all was).  A call whose launches would have 2^32 lanes or more (as the account of
 * 1,024 sequences and 8 heads with a max_len of 2^20) is RKC_E_UNSUPPORTED.  What the host cannot see (lengths,
 * offsets, block ids and parents in device memory) is checked on the device: nothing outside the buffers is read
 * or written, and RKC_CS_* bits are OR'ed into the sequence's word of d_status.
 *
 * Strides of what a call writes (outputs, accounts, and K and V where slots are evicted) may put the dimensions in any
 * order but must keep elements apart: strides of zero, as of a broadcast tensor, are for what is only read.
 */
#ifndef RKC_CACHE_H
#define RKC_CACHE_H

#include "rkc.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RKC_MAX_CACHE_LEN (1 << 26) /* slots of one sequence                                       */
#define RKC_MAX_TREE_ROWS 256       /* rows of one sequence when d_parent is given                  */

enum rkc_dtype { RKC_BF16 = 0, RKC_F16 = 1 };

enum rkc_cache_status {
  RKC_CS_LENGTH = 1, /* length or row count outside its limits, or more rows than slots: the sequence is
                        left out and its outputs are not written                                        */
  RKC_CS_BLOCK = 2,  /* a block id outside [0, n_blocks): block 0 was read instead; rkc_evict leaves out
                        the moves into or out of such a block                                           */
  RKC_CS_PARENT = 4  /* a parent that is not -1 or an earlier row of its sequence: -1 was taken     */
};

/* The cache: host struct.  K and V are [block][slot][head][dim] in any order of the first three (strides in
 * elements, multiples of 8, below 2^31 between blocks and 2^30 within one; the last dimension is contiguous); 16-byte
 * aligned. */
typedef struct rkc_cache {
  int32_t n_seqs;
  int32_t n_blocks;    /* blocks of the pool; table entries are < this                               */
  int32_t max_pages;   /* table entries per sequence                                                 */
  int32_t page_tokens; /* slots per block: 16, 32, 64, ... 1024                                      */
  int32_t kv_heads;
  int32_t head_dim;    /* 64, 128 or 256                                                             */
  int32_t dtype;       /* enum rkc_dtype, of the cache, the queries and the outputs                  */
  int32_t reserved;    /* must be 0                                                                  */
  int64_t k_block_stride, k_slot_stride, k_head_stride;
  int64_t v_block_stride, v_slot_stride, v_head_stride;
  void* d_k;
  void* d_v;
  const int32_t* d_block_table; /* [n_seqs * max_pages]                                              */
  int32_t* d_status;            /* [n_seqs], bits OR'ed in (the caller clears), or NULL              */
} rkc_cache;

/* Attention: host struct.  Rows of sequence s are [d_row_offset[s], d_row_offset[s+1]); with n of them, their
 * own keys and values are in its last n slots already.  Row i (of n, base = length - n) sees
 *   without d_parent   slots [row_start, base + i]           (row_start 0 without d_row_start)
 *   with d_parent      slots [row_start, base), its own slot base + i and those of its ancestors
 * and in both cases the slots below the sequence's prefix (with d_parent: below base).
 * The score of a row of query head h and a slot it sees is  x = scale q.k,  then softcap tanh(x / softcap) if
 * softcap > 0, then x - slope[h] |distance| if d_slope is given; the distance is that of the slots, drafted
 * slots counting as base + depth in the tree.  A row that sees nothing gets zeros and -inf.  Slots that no row
 * sees and slots behind the length may hold anything; an infinite value that a row sees makes its output infinite,
 * or NaN where its weight is below the range of 32 bits.  Query heads [g * h, g * (h + 1)) share key/value head h,
 * g = q_heads / kv_heads. */
typedef struct rkc_attention {
  int32_t n_rows;   /* rows of all sequences = d_row_offset[n_seqs]                                  */
  int32_t q_heads;  /* a multiple of kv_heads                                                        */
  int32_t max_rows; /* >= every sequence's rows                                                      */
  int32_t max_len;  /* >= every sequence's length, <= max_pages * page_tokens                        */
  float scale;
  float softcap;    /* >= 0                                                                          */
  float decay;      /* of the account, see d_weight                                                  */
  int32_t reserved; /* must be 0                                                                     */
  int64_t q_row_stride, q_head_stride;     /* elements, multiples of 8                               */
  int64_t out_row_stride, out_head_stride; /* elements, multiples of 8                               */
  int64_t weight_seq_stride, weight_head_stride; /* elements, of d_weight_in and d_weight            */
  const void* d_q;             /* [n_rows][q_heads][head_dim], 16-byte aligned                       */
  const int32_t* d_row_offset; /* [n_seqs + 1]                                                       */
  const int32_t* d_length;     /* [n_seqs]                                                           */
  const int32_t* d_row_start;  /* [n_rows] or NULL                                                   */
  const int32_t* d_prefix;     /* [n_seqs] or NULL                                                   */
  const int32_t* d_parent;     /* [n_rows] row within its sequence, -1 for a root; or NULL           */
  const float* d_slope;        /* [q_heads] or NULL                                                  */
  void* d_out;                 /* [n_rows][q_heads][head_dim], 16-byte aligned (rkc_attend); may be d_q with
                                  its strides where d_weight is NULL                                 */
  float* d_lse;                /* [n_rows][q_heads]: written by rkc_attend, read by rkc_weigh        */
  const float* d_weight_in;    /* [n_seqs][kv_heads][max_len] or NULL (zeros)                        */
  float* d_weight;             /* the same, may be d_weight_in; rkc_attend: or NULL.  Slots below the
                                  length become decay * in + the sum of exp(score - lse) over the rows and
                                  the head's queries; the others are not written                       */
  void* d_scratch;             /* >= rkc_attend_scratch_bytes, 256-byte aligned (rkc_attend)         */
  size_t scratch_bytes;
} rkc_attention;

/* Eviction: host struct.  Sequence s comes down to  new = min(length, max(budget, protect))  slots.  Of each
 * head, slots below protect stay where they are; of the others those with pos >= recent_from go before the rest,
 * then the larger account (NaN counts as lowest), then the lower slot.  What is kept beyond slot new moves, in
 * order, into the gaps before it; everything else stays in place.  K and V change in place (the blocks past
 * the new length are free afterwards); the account and the positions are written to d_weight_out and d_pos_out
 * up to slot new.  Blocks that sequences share must lie below protect in each of them. */
typedef struct rkc_eviction {
  int32_t max_len;  /* as in rkc_attention                                                           */
  int32_t reserved; /* must be 0                                                                     */
  int64_t weight_seq_stride, weight_head_stride; /* elements, of the four arrays below               */
  const int32_t* d_length;      /* [n_seqs]                                                          */
  const int32_t* d_budget;      /* [n_seqs], >= 0                                                    */
  const int32_t* d_protect;     /* [n_seqs] or NULL (0)                                              */
  const int32_t* d_recent_from; /* [n_seqs] or NULL (none is recent)                                 */
  const float* d_weight;        /* [n_seqs][kv_heads][max_len]                                       */
  const int32_t* d_pos;         /* the same, or NULL: a slot's position is its number                */
  float* d_weight_out;          /* the same, not d_weight                                            */
  int32_t* d_pos_out;           /* the same, not d_pos                                               */
  int32_t* d_length_out;        /* [n_seqs], none of the four above                                  */
  void* d_scratch;              /* >= rkc_evict_scratch_bytes, 256-byte aligned                      */
  size_t scratch_bytes;
} rkc_eviction;

/* Scratch of a call; read only the host structs, never fail (0 where the call would be refused). */
size_t rkc_attend_scratch_bytes(const rkc_cache* c, const rkc_attention* a);
size_t rkc_evict_scratch_bytes(const rkc_cache* c, const rkc_eviction* e);

/* s: a hipStream_t of the current device (NULL = the default stream). */
rkc_status rkc_attend(const rkc_cache* c, const rkc_attention* a, void* s);
rkc_status rkc_weigh(const rkc_cache* c, const rkc_attention* a, void* s);
rkc_status rkc_evict(const rkc_cache* c, const rkc_eviction* e, void* s);

#ifdef __cplusplus
}
#endif

#endif /* RKC_CACHE_H */
