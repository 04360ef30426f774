/*
 * confspec_int4.h - generation and verification steps whose weights and paged cache are read in 4 bits.
 *
 * A step over few tokens (Algorithm 1's generate calls, the verification of a few drafted tokens) is bound by the bytes
 * of the weights and of the cached context.  The functions here are the 4-bit twins of confspec_op_gemm,
 * confspec_op_rope_split, the cache write-back and confspec_op_attention (confspec_ops.h, confspec_append.h): products
 * of up to 128 rows with 4-bit weights, the append of rotated keys and values to a 4-bit cache, the attention over it,
 * and its rows as the values they stand for.  One layer of such a step is, with confspec_op_rmsnorm between the parts:
 *     w4_gemm (QKV, store) -> kv4_append -> kv4_attention -> w4_gemm (O, residual) -> w4_gemm (gate/up, SwiGLU)
 *     -> w4_gemm (down, residual)
 *
 * Same conventions as confspec.h: dev pointers are caller-owned device memory, nothing is allocated, nothing
 * synchronises, every check that host-visible arguments allow is made before the first launch.  The calls can be
 * captured into HIP graphs: a graph keeps the host lengths and counts of its capture (launches and pieces come from them),
 * and the device arrays have to hold the same ones at every replay; block tables, cache and operands may change.  Calls on
 * different streams may run at the same time as long as their outputs, scratch and written cache rows differ.  Outputs
 * overlap no other operand unless a function says so.  All of them need a bf16 context (head_dim 128); other contexts get
 * CONFSPEC_E_UNSUPPORTED.
 */
#ifndef CONFSPEC_INT4_H
#define CONFSPEC_INT4_H

#include "confspec.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- paged cache in 4 bits ----
 * A cache row is one token of one kv head, 128 elements.  It stands for the values z + s * c: codes c in 0..15 and, per row,
 * two IEEE halves s and z.  A row x (bf16 values, clamped to +-65504) is stored as
 *     z = half(min x),  s = half(fp32((max x - z) / 15)),  c = (x - z) / s to the nearest whole number, ties to even,
 *     within 0..15 (0 where s is 0); a zero s or z is +0.
 * A row with a NaN among its elements stands for NaN throughout: s and z are 0x7E00, codes 0 (its finite elements are lost, and
 * the attention of the rows that see it is NaN, as it is with a NaN among bf16 keys or values).
 * Keys are stored rotated.  A page holds 16 tokens of one head, keys and values:
 *   byte    0  key codes: 32-bit word ((c * 16 + token) * 4 + i) has elements d = 32 i + 8 c + e, e = 0..7, the even
 *              e in bits 2 e .. 2 e + 3 and the odd ones in bits 2 e + 14 .. 2 e + 17
 *   byte 1024  value codes: word ((token / 4 * 16 + w) * 4 + token % 4) has elements 8 w + j in bits 4 j .. 4 j + 3
 *   byte 2048  (s, z) of the keys, two halves a token;  byte 2112  (s, z) of the values */
#define CONFSPEC_KV4_PAGE_BYTES 2176

/* pages: dev, 16-byte aligned, [n_layers][n_blocks][n_kv_heads][CONFSPEC_KV4_PAGE_BYTES]; block_size must be 16.
 * block_table and the clamping of its ids as in confspec_kv. */
typedef struct {
    void *pages;
    int32_t n_blocks, block_size;
    const int32_t *block_table;
    int32_t max_blocks_per_seq;
} confspec_kv4;

/* The front half of an attention block on a fp32 QKV projection: rotates q and k at positions L_b + t (half-split
 * pairing; angles and rotation in 64 bits, rounded to fp32 and then to bf16), writes q [T, Hq, 128], k and v
 * [T, Hkv, 128] in bf16, and stores the k and v rows so rounded of the tokens i < n_append[b] of every trace in rows
 * L_b + i of its cache (page block_table[b][(L_b + i) / 16], token (L_b + i) % 16).  Nothing else in the cache changes.
 *   dev_qkv      : fp32, row t at dev_qkv + t * qkv_stride: q heads, k heads, v heads; 16-byte aligned;
 *                  qkv_stride >= (Hq + 2 Hkv) * 128 elements, a multiple of 4
 *   dev_n_append / h_n_append : int32 [B] on the device and on the host (same values), 0 <= n_append[b] <= S_b;
 *                  both NULL: all tokens
 * The rows written must lie inside the block table's capacity, positions below 2^31 - 2^23, and no two traces may write the same
 * row. */
int confspec_op_kv4_append(confspec_ctx *ctx, const confspec_kv4 *kv, const confspec_batch *batch, int32_t layer,
                           const float *dev_qkv, int64_t qkv_stride, const int32_t *dev_n_append, const int32_t *h_n_append,
                           void *dev_q, void *dev_k, void *dev_v, confspec_stream stream);

/* The values cache rows stand for: rows L_b + i, i < S_b, of every trace (what confspec_op_kv4_append with the same
 * batch and no counts writes) into dev_k / dev_v, fp32 [T, Hkv, 128], 16-byte aligned. */
int confspec_op_kv4_read(confspec_ctx *ctx, const confspec_kv4 *kv, const confspec_batch *batch, int32_t layer, float *dev_k,
                         float *dev_v, confspec_stream stream);

/* Attention of one layer as confspec_op_attention has it, on a 4-bit context: softmax over the keys j <= L_b + t of
 * q . k_j / sqrt(128); rows 0..L_b-1 from the cache, the rest from dev_k_suffix / dev_v_suffix (bf16, what
 * confspec_op_kv4_append returned).  q [T, Hq, 128], out [T, Hq * 128], bf16; all 16-byte aligned.
 *   dev_scratch  : dev, 256-byte aligned, >= confspec_op_kv4_attention_scratch_bytes for this batch; its contents need
 *                  not be kept between calls, but two calls that may run at the same time need one each (NULL is fine
 *                  where the need is 0)
 * Numerics: q (below 2^116 in magnitude; taken as halves times a power of two of its row) and codes enter the score product
 * exactly, but for elements of q 2^-27 times their row's largest, which lose what is below 2^-38 of it; scores, softmax
 * statistics and sums are fp32; probabilities times the value row's s are rounded to IEEE half for the cached rows, carried
 * as two bf16 terms for the suffix.  Suffix values are below 2^90 in magnitude, or no finite numbers: a weight
 * is positive, so that an infinity makes its column infinite, and a NaN or infinities of both signs NaN, in the rows that see the
 * token, and in no other. */
int confspec_op_kv4_attention(confspec_ctx *ctx, const confspec_kv4 *kv, const confspec_batch *batch, int32_t layer,
                              const void *dev_q, const void *dev_k_suffix, const void *dev_v_suffix, void *dev_out,
                              void *dev_scratch, size_t scratch_bytes, confspec_stream stream);
int confspec_op_kv4_attention_scratch_bytes(const confspec_ctx *ctx, const confspec_batch *batch, size_t *out_bytes);

/* ---- products with 4-bit weights ----
 * A weight is s * (c - z): codes c in 0..15 and, for every row and every group of 32, 64 or 128 elements along k, two
 * IEEE halves s and z (z in units of the code and kept to 2^-21 of one; 8 where it is not given). */
#define CONFSPEC_W4_MAX_ROWS 128

/* Bytes confspec_w4_pack writes for an [N, K] matrix; 0 where the shape is not supported (N % 16 != 0, group not 32, 64
 * or 128, K % group != 0, K above 2^22, more than 2^34 elements with K rounded up to a multiple of 128). */
size_t confspec_w4_bytes(int32_t N, int32_t K, int32_t group);

/* Lays a quantised matrix out for confspec_op_w4_gemm, once per matrix.
 *   dev_codes  : uint8 [N, K / 2], element 2 j in the low and 2 j + 1 in the high four bits of byte j; 4-byte aligned
 *   dev_scales : half [N, K / group];  dev_zeros : half [N, K / group], or NULL (8 everywhere)
 *   gate_up    : 0, or 1 for a gate/up matrix (rows 0..N/2-1 gate, the rest up) that will be used with the SwiGLU epilogue
 *   dev_dst    : dev, 256-byte aligned, >= confspec_w4_bytes */
int confspec_w4_pack(confspec_ctx *ctx, const void *dev_codes, const void *dev_scales, const void *dev_zeros, int32_t N,
                     int32_t K, int32_t group, int32_t gate_up, void *dev_dst, size_t dst_bytes, confspec_stream stream);

/* out = A . W^T with an epilogue of confspec_ops.h: A bf16 [M, K] row-major, 1 <= M <= CONFSPEC_W4_MAX_ROWS, W as
 * confspec_w4_pack wrote it (same N, K, group).  Nothing in the packed bytes says how they were packed: with another group
 * or shape the result is wrong, and where that has more confspec_w4_bytes, bytes behind the matrix are read; a matrix
 * packed with gate_up = 1 goes with the SwiGLU epilogue, and only with it.
 *   CONFSPEC_EPI_STORE_F32 : out fp32 [M, N]
 *   CONFSPEC_EPI_RESID_F32 : out fp32 [M, N] = dev_residual + A . W^T (dev_residual may be dev_out: in place)
 *   CONFSPEC_EPI_SWIGLU    : W packed with gate_up = 1; out bf16 [M, N / 2] = silu(gate) * up
 * dev_residual is read by the residual epilogue only and must be NULL otherwise.  Operands are 16-byte aligned.
 * Products of codes and activations are exact, their sums within a group and over the groups fp32, added in an order
 * that only the shape decides.  A result that is no finite number so (infinite activations; sums of 31 times the activations beyond
 * fp32) is what the sum of activations times weights is, taken in fp32 group by group. */
int confspec_op_w4_gemm(confspec_ctx *ctx, const void *dev_A, const void *dev_W4, const float *dev_residual, void *dev_out,
                        int32_t M, int32_t N, int32_t K, int32_t group, int32_t epilogue, confspec_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* CONFSPEC_INT4_H */
