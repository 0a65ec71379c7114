/*
 * lra_attn8.h - the layer path in 8 bits: projection of new tokens by 8-bit integers, a cache of 8-bit codes, and the
 * attention of lra_attn.h over it.  Conventions (ownership, streams, errors, re-entrance, determinism) are those of lra_attn.h.
 *
 *     lra_quantize_rows   hidden states -> codes, one scale per token
 *     lra_matmul_i8       codes x 8-bit weights -> Q, or [K | V | L] of the new tokens, in 16 or 32 bits
 *     lra_cache8_append   K, V (rotated on the way) and L of the new tokens -> the cache
 *     lra_attn_batch8     attention of a batch over the cache
 *     lra_cache8_gather   rows of the cache as 16 or 32-bit values, for the calls of lra_attn.h
 */
#ifndef LRA_ATTN8_H
#define LRA_ATTN8_H

#include "lra_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * 8-bit codes of K_base and V_base: LRA_E4M3, floating-point numbers of 4 exponent and 3 mantissa bits (OCP "e4m3fn", largest
 * 448, no infinities), or LRA_INT8, two's complement integers.  A code c stands for
 *     c * 2^(s - 127),
 * s the byte that its block of 16 tokens and its kv head have in k_scale or v_scale (255: not a number).  With a power of two
 * every value is a bf16 number exactly, for bytes from 3 (LRA_E4M3) or 0 (LRA_INT8) to 246: below, the smallest e4m3 codes lie
 * between bf16's denormal numbers and are rounded to them, above, the largest codes are beyond its range.  Integers are the closer
 * ones where the values of a block are of similar size, e4m3 where some channels are far larger than the others.
 */
typedef enum { LRA_E4M3 = 0, LRA_INT8 = 1 } lra_code;

/*
 * A cache of blocks of 16 tokens.  Token j of sequence t lies in block b = block_table[t*max_blocks_per_seq + j/16], slot j%16;
 * with block_table NULL there is one sequence, and b = j/16.  Its codes for kv head h are
 *     K: the head_dim bytes at  k + b*kv_block_stride + h*kv_head_stride + (j%16)*head_dim
 *     V: byte c*16 + j%16 at    v + b*kv_block_stride + h*kv_head_stride,  c = 0 .. head_dim-1
 * (V by dimension: a matrix instruction that sums over keys takes sixteen keys of one dimension as one 16-byte load.)
 * Scales: k_scale[b*scale_block_stride + h], v_scale alike.  The low-rank cache L, one for all agents, is that of lra_cache's
 * paged form in the type of lra_shape: row b*16 + j%16, l_row_stride elements apart (0: rank).
 *
 * What holds of a paged lra_cache holds here: entries of block_table past a sequence's last block are never read, those that
 * are read lie in [0, num_blocks); slots past seq_lens[t] may hold anything.  The scales of a block are read once it holds a
 * visible token.  Rows of one block share their scale: those that no query sees must be finite where the block holds others
 * that one sees.
 */
typedef struct {
  void* k;                    /* DEVICE, 16-byte aligned, as v and l */
  void* v;                    /* DEVICE */
  uint8_t* k_scale;           /* DEVICE */
  uint8_t* v_scale;           /* DEVICE */
  void* l;                    /* DEVICE */
  int64_t kv_block_stride;    /* bytes, multiples of 16, at most 2^40 */
  int64_t kv_head_stride;
  int64_t scale_block_stride; /* bytes, >= Hkv; 0: Hkv; at most 2^31 */
  int64_t l_row_stride;       /* elements; 0: rank.  A multiple of 8, or the rank; at most 2^24 */
  int32_t code;               /* lra_code */
  int32_t max_blocks_per_seq; /* row length of block_table (of no effect without one) */
  int32_t num_blocks;
  int32_t n_seqs;             /* 1 without a block table */
  const int32_t* block_table; /* DEVICE int32 [n_seqs][max_blocks_per_seq], or NULL */
  const int32_t* seq_lens;    /* DEVICE int32 [n_seqs], >= 0 */
  int32_t max_seq_len;        /* HOST-known upper bound, as in lra_cache */
} lra_cache8;

/*
 * New tokens of a batch of sequences: sequence t owns rows seq_start[t] .. seq_start[t+1]-1, c_t of them (none is fine), which
 * are the LAST c_t tokens of the sequence: its length in lra_cache8 counts them already.
 */
typedef struct {
  const void* k;             /* DEVICE [n_new][Hkv][head_dim], tokens k_token_stride elements apart; in lra_shape's type */
  const void* v;             /* DEVICE, alike */
  const void* l;             /* DEVICE [n_new][rank], or NULL: the L rows are left as they are */
  int64_t k_token_stride;    /* elements, at most 2^31; k_ and v_token_stride, like the addresses of k and v, multiples of 16 bytes */
  int64_t v_token_stride;
  int64_t l_token_stride;
  const int32_t* seq_start;  /* DEVICE int32 [n_seqs+1], non-decreasing, [0] = 0, [n_seqs] = n_new */
  const int32_t* positions;  /* DEVICE int32 [n_new], >= 0, or NULL: the token's index in its sequence */
  int32_t n_new;             /* >= 1 */
  int32_t max_new_per_seq;   /* HOST-known upper bound of every c_t */
  float rope_theta;          /* > 0: the keys are rotated by their positions (pairs i, i + head_dim/2, angle
                                position * theta^(-2i/head_dim)) before they are quantized; 0: taken as they are.
                                lra_projection's remark on evicted caches holds: give positions then */
} lra_new_rows;

/*
 * Write the new rows into the cache.  For every block and kv head that receives new tokens, the scale becomes the least power
 * of two (2^-126 at least) that brings the largest of the new values to 448 (LRA_E4M3) or 127 (LRA_INT8) at most, or stays
 * the old one if the block holds earlier tokens of the sequence and theirs is larger; where it grows, the codes of the earlier
 * tokens are rounded anew.  Rounding is to nearest, ties to even; rotation and scaling are done in fp32 before it.  Slots past
 * the end of a sequence are left as they were, and blocks without new tokens are not touched.  A block that receives tokens
 * belongs to one sequence (blocks that are full may be shared).  Calling again with the same rows changes nothing.
 * K and V must be finite: a value that is not makes the block's rows of that head unspecified.  (Above 3.29e38 the code may stand
 * for 2^128, which is read as infinite.)
 * Nothing is written for a sequence whose device-side length exceeds max_seq_len; tokens before the sequence's first (c_t
 * larger than its length) and blocks whose table entry is out of range are passed over.  More than 2^31 (block with new tokens,
 * pair of kv heads) of a sequence are LRA_ERR_UNSUPPORTED, and so are as many (sixteen rows, pair) in lra_cache8_gather.
 */
lra_status lra_cache8_append(const lra_shape* shape, const lra_cache8* cache, const lra_new_rows* rows, void* stream);

/*
 * Row i of sequence t of dst becomes the values of row kept[t][i] of src, for i < dst->seq_lens[t] (at most dst->max_seq_len):
 * what lra_evict_select keeps, or any choice.  kept NULL: the last rows of src, row i the token
 * src length - dst length + i; where dst's lengths are src's, the whole sequence.  dst is a cache of lra_attn.h (contiguous or
 * paged, any strides) whose k_base / v_base / l are WRITTEN although declared const; adapter 0's L rows are written.  bf16
 * values are exact where the scale byte allows it (lra_code), and the nearest elsewhere.  Rows behind, and those whose source is
 * not in [0, src length), are left as they are.
 * With the rotary key side (key_rope_theta > 0) a row must keep its index, by which lra_attn_batch rotates its adapter part: kept is
 * LRA_ERR_UNSUPPORTED then, as in lra_cache_gather, and without it dst's lengths must be src's, which is not checked (the last rows
 * alone would be attended to at other positions).  A caller that wants rows for something else leaves key_rope_theta 0.
 *   kept  DEVICE int32 [n_seqs][kept_stride], kept_stride >= dst->max_seq_len
 */
lra_status lra_cache8_gather(const lra_shape* shape, const lra_cache8* src, const int32_t* kept, int64_t kept_stride,
                             const lra_cache* dst, void* stream);

/*
 * lra_attn_batch (same batches, windows and sinks, adapters, outputs) over such a cache: the result is that of lra_attn_batch
 * on the values that the codes stand for.  bf16 with a rank that is a multiple of 8 runs on MFMA kernels, everything else on
 * vector-ALU kernels.  A rotated key-side adapter (key_rope_theta > 0 with a b_k) is LRA_ERR_UNSUPPORTED, and 2^24 query rows (queries
 * times n_q_heads) or more may be.  LRA_INT8 with 64 query rows per kv head or fewer: a block whose v_scale is 118 or more below the
 * largest one of its sequence (a factor of 2^118) may count as zeros.
 *   workspace  DEVICE, 256-byte aligned, >= lra_batch8_workspace_bytes(...), as for lra_attn_batch
 *   tuning     kernel_variant (1: vector-ALU kernels, 2: no kernel of its own for few query rows)
 */
lra_status lra_attn_batch8(const lra_shape* shape, const lra_cache8* cache, const lra_adapters* adapters, const lra_batch* batch,
                           const void* q, void* out, void* workspace, size_t workspace_bytes, const lra_tuning* tuning, void* stream);
/* (size_t)-1 when the arguments would be rejected. */
size_t lra_batch8_workspace_bytes(const lra_shape* shape, const lra_cache8* cache, const lra_batch* batch, const lra_tuning* tuning);

/*
 * Rows as 8-bit integers with a scale each: scales[i] = max_j |x[i][j]| / 127, codes[i][j] = x[i][j] * (127 / max) rounded to
 * nearest, ties to even, in fp32.  A row of zeros has scale 0 and codes 0; a row that is not finite gets the scale NaN, which
 * makes its row of a product NaN.  (Of rows whose largest value is below 127 * 2^-126, 1.5e-36, the scale is a denormal number: right to
 * 2^-150, and so with fewer bits.)  For activations (a row is a token) and for weights alike (a row is a feature).
 *   x      DEVICE [rows][cols] of dtype (lra_dtype), rows x_stride elements apart; x and the stride multiples of 16 bytes
 *   codes  DEVICE int8 [rows][cols], rows codes_stride bytes apart; both multiples of 16 bytes
 *   scales DEVICE float [rows]
 * cols a multiple of 16, at most 2^17; rows below 2^24 (a product takes 2^20 of them and fewer than 2^17 columns); strides at most
 * 2^40.
 */
lra_status lra_quantize_rows(const void* x, int32_t dtype, int64_t x_stride, int32_t rows, int32_t cols, int8_t* codes,
                             int64_t codes_stride, float* scales, void* stream);

/* Operands of lra_matmul_i8. */
typedef struct {
  const int8_t* x;       /* DEVICE [m][k], rows x_stride bytes apart: the tokens */
  const int8_t* w;       /* DEVICE [n][k], rows w_stride bytes apart: a linear layer's weight, one feature per row */
  const float* x_scale;  /* DEVICE [m] */
  const float* w_scale;  /* DEVICE [n] */
  int64_t x_stride;      /* strides and the addresses of x and w: multiples of 16 bytes; strides at most 2^31 */
  int64_t w_stride;
  int32_t m, n, k;       /* m and n at most 2^20; k a multiple of 16, below 2^17 (sums stay in 32 bits) */
} lra_i8_operands;

/*
 * y[i][j] = x_scale[i] * w_scale[j] * sum_c x[i][c] w[j][c]: the sum exact in 32-bit integers, scaled in fp32 (by x_scale first), rounded once.
 *   y          DEVICE [m][n] of dtype (lra_dtype), rows y_stride elements apart, 16-byte aligned; y_stride from n to 2^31
 *   workspace  as many bytes as lra_matmul_i8_workspace_bytes says: none for any size so far, NULL and 0 will do
 */
lra_status lra_matmul_i8(const lra_i8_operands* ops, void* y, int32_t dtype, int64_t y_stride, void* workspace,
                         size_t workspace_bytes, void* stream);
/* (size_t)-1 when the sizes would be rejected. */
size_t lra_matmul_i8_workspace_bytes(int32_t m, int32_t n, int32_t k, int32_t dtype);

#ifdef __cplusplus
}
#endif
#endif /* LRA_ATTN8_H */
