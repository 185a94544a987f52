/*
 * dllava, serving operators in 4 bits and with grouped heads: part of the same library as dllava.h, with its conventions
 * (device pointers, streams, status codes, messages, workspaces, nothing allocated, no host synchronisation).
 *   dllava_mx_quantize / dllava_mx_dequantize   rows to microscaled 4-bit floating point and back
 *   dllava_mx_linear                            linear layer, rows and weights in 4 bits (prompts)
 *   dllava_mx_linear_few                        linear layer, bfloat16 rows of a decode step, weights in 4 bits
 *   dllava_mx_cache_store / _load               keys and values into and out of a paged cache in 4 bits
 *   dllava_mx_decode_attn_append                one decode step over such a cache (Eq. 6), grouped heads
 *   dllava_group_prefill_attn                   causal attention of packed prompts (Eq. 1), grouped heads
 *
 * Microscaled 4-bit floating point: blocks of 32 consecutive elements share a power of two, stored as a byte s that stands for
 * 2^(s - 127); an element is a 4-bit code, sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0..7; 8..15 with a minus sign).
 * How a block is rounded: with 2^E <= amax < 2^(E+1) its largest magnitude, s = E - 2 + 127, one more where amax > 1.75 * 2^E
 * (seven would round to eight), at least 1 and at most 252 (all values are then finite in float32 and bfloat16); an element is the nearest code to x / 2^(s - 127), ties to the even
 * code, magnitudes beyond six to six.  A block that holds an infinity or a NaN has s = 255, and every element of it reads as NaN.  Signs are
 * kept, also those of zeros.  The rounding is exact arithmetic: the same input gives the same bytes everywhere.
 *
 * dllava_set_launch_override here (any other value: the call picks, and 0 gives it back):
 *   DLLAVA_LAUNCH_LINEAR_TILE     dllava_mx_linear: 8, 7, 6, 4 = 256 features x 256, 224, 192, 128 rows, 12 = 128 x 128, 2 = 64 x 32 with the
 *                                 columns shared out; dllava_mx_linear_few: 1, 2, 3 = 16, 32, 48 features per block
 *   DLLAVA_LAUNCH_DECODE_SPLITS   dllava_mx_decode_attn_append: blocks of the launch, at most as many as it would have
 *   DLLAVA_LAUNCH_PREFILL_WAVES, DLLAVA_LAUNCH_PREFILL_BLOCKS   dllava_group_prefill_attn, bfloat16: as for dllava_prefill_attn's long sequences
 */
#ifndef DLLAVA_MX_H
#define DLLAVA_MX_H

#include "dllava.h"

#ifdef __cplusplus
extern "C" {
#endif

/* dtype of a dllava_kv_cache whose pages are in 4 bits; only the calls of this header take such a cache.
 *   pages  [n_pages][H][17 * Dh] bytes, 16-byte aligned; per page and head:
 *            K codes  [16 tokens][Dh / 2]: byte i holds elements 2i (low half) and 2i + 1
 *            V codes  [4][16 columns c][4][Dh / 32 blocks m]: token 4g + j, elements 32m + c (low half) and 32m + 16 + c are
 *                     in byte ((16 g + c) * 4 + j) * (Dh / 32) + m (as the products of the attention read them)
 *            K scale bytes [16 tokens][Dh / 32], V scale bytes [16 tokens][Dh / 32]
 *   block_table, cache_len, page_size (16), Dh (64 or 128): as in dllava.h; H = heads of K and V. */
#define DLLAVA_MX 2

/*
 * A packed matrix [M, K] (K % 32 == 0) is one buffer of dllava_mx_bytes(M, K) bytes, 256-byte aligned.  With Kp = K rounded up to
 * 512 and Mp = M rounded up to 16:
 *   codes        [M][Kp / 2]: byte i of a row holds elements 2i (low half) and 2i + 1; elements K .. Kp-1 are zeros
 *   scale bytes  [Mp / 16][Kp / 512][4][16][4], behind the codes: the byte of row r and block c (of 32 elements) is at
 *                [r / 16][c / 16][c % 4][r % 16][c % 16 / 4]; 127 for rows and blocks that do not exist
 * (a wave of the products then reads the scales of its 16 x 512 piece as one line).
 */
size_t dllava_mx_bytes(int64_t M, int64_t K);   /* host, pure; 0 if a size is not supported */

/*
 * Rows to 4 bits.  x [M, K] dtype (DLLAVA_F32 or DLLAVA_BF16), row stride ldx; packed: out, fully written.
 * Sizes: K % 32 == 0, ldx * sizeof(dtype) % 16 == 0, ldx >= K, ceil(M / 16) * ceil(K / 512) < 2^24.  M == 0 is a no-op.
 */
int dllava_mx_quantize(const void* x, int64_t ldx, int64_t M, int64_t K, void* packed, size_t packed_bytes, int dtype, void* stream);

/* The values that a packed matrix stands for, y [M, K] dtype, row stride ldy.  They are exact in both types; of the scale bytes that
 * dllava_mx_quantize does not write, 0, 253 and 254 are read as the powers they stand for (a value beyond the type's range is an infinity). */
int dllava_mx_dequantize(const void* packed, size_t packed_bytes, int64_t M, int64_t K, void* y, int64_t ldy, int dtype, void* stream);

/*
 * dllava_linear with both matrices in 4 bits:  y = act(x W^T + bias) + residual (act 0, 1), or (x W^T + bias) * SiLU(residual) (act 2).
 *   xq  packed [M, K];  Wq  packed [N, K];  bias [N] float32 or NULL;
 *   residual [M, N] bfloat16 with y's row stride, or NULL (act 0, 1), may be y itself;  y [M, N] bfloat16, row stride ldy, out.
 * Products are exact, sums are float32, each result is rounded once.
 * Sizes: K % 32 == 0, N % 8 == 0, ldy % 8 == 0, K < 2^23, N < 2^27; ldy < 2^21, or ceil(N / 64) * ceil(M / 32) < 2^23.  dtype: DLLAVA_BF16.  M == 0 or N == 0 is a no-op.
 */
int dllava_mx_linear(const void* xq, size_t xq_bytes, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N,
                     int act, const void* residual, void* y, int64_t ldy, int dtype, void* stream);

/*
 * The same for few rows (M <= 64: one per sequence of a decode step) that stay in bfloat16: only the weights are in 4 bits, and their
 * bytes are the traffic.  x [M, K] bfloat16, row stride ldx.  ldx % 8 == 0, ldx < 2^24; otherwise as above.  No workspace.
 */
int dllava_mx_linear_few(const void* x, int64_t ldx, int64_t M, int64_t K, const void* Wq, size_t Wq_bytes, const float* bias, int64_t N,
                         int act, const void* residual, void* y, int64_t ldy, int dtype, void* stream);

/*
 * Keys and values into a cache in 4 bits: row i of sequence b goes to position start[b] + i,  i < n_b = off[b+1] - off[b], and
 * cache_len[b] = start[b] + n_b.
 *   K, V     [*, H, Dh] dtype (DLLAVA_F32 or DLLAVA_BF16), row stride ldkv elements (ldkv >= H * Dh, ldkv * sizeof(dtype) % 16 == 0)
 *   off      [B+1] int32 row offsets of the sequences (out_off of dllava_select_compact);  rows = host upper bound on off[B]
 *   start    [B] int32, or NULL (= 0).  Must not overlap cache_len (of which a copy can be passed).  start[b] < 0 is read as 0
 *   src_off, src_idx   both NULL: row i of sequence b is row off[b] + i of K and V.  Both given (seq_off and kept_idx of
 *            dllava_select_compact): it is row src_off[b] + src_idx[off[b] + i], so that only the kept rows are stored
 *   err_flag device int32, may be NULL: set to 1 if some sequence exceeds max_pages_per_seq * page_size; rows beyond it are
 *            not stored and cache_len[b] is clamped to it.  Never cleared by the library.
 * Only the slots of the stored tokens are written.  Positions before start[b] keep what they hold.  Sizes: rows / 16 + 2 B < 2^24.
 */
int dllava_mx_cache_store(const void* K, const void* V, int64_t ldkv, int32_t B, const int32_t* off, const int32_t* start, int64_t rows,
                          const int32_t* src_off, const int32_t* src_idx, const dllava_kv_cache* cache, int32_t* err_flag, int dtype,
                          void* stream);

/* The values of positions start[b] .. start[b] + n_b - 1 as the cache holds them, to rows off[b] .. off[b+1] - 1 of K and V [rows, H, Dh]
 * dtype, row stride ldkv; positions at or behind cache_len[b] give zeros.  K and V: outputs, neither NULL. */
int dllava_mx_cache_load(const dllava_kv_cache* cache, int32_t B, const int32_t* off, const int32_t* start, int64_t rows, void* K, void* V,
                         int64_t ldkv, int dtype, void* stream);

/*
 * dllava_decode_attn_append over a cache in 4 bits and with grouped heads: query head h attends to K/V head h / (Hq / H).
 *   o[b,h] = softmax(scale * [K_cache; k_new] q[b,h]) [V_cache; v_new], the current token as given (not rounded to 4 bits); the keep
 *   decision, keep_out, err_flag and the update of cache_len as there; a kept token's k_new, v_new are stored in 4 bits.
 *   q, o [B, Hq, Dh], k_new, v_new [B, H, Dh] bfloat16, contiguous;  Hq % H == 0
 *   workspace  dllava_mx_decode_workspace(B, Hq, H, Dh, max_pages_per_seq) bytes, 256-byte aligned, zero-filled once (counters, which every
 *              call leaves at zero).  It serves calls of any sizes that need no more bytes, one behind the other: calls that may
 *              run at the same time, captured ones too, each need their own.
 * Scores, softmax statistics and sums are float32; probabilities are rounded to bfloat16 before they meet the values.
 */
int dllava_mx_decode_attn_append(const void* q, const void* k_new, const void* v_new, int32_t B, int32_t Hq, const float* logits,
                                 float threshold, const uint8_t* keep_override, const dllava_kv_cache* cache, float scale, void* o,
                                 uint8_t* keep_out, int32_t* err_flag, void* workspace, size_t workspace_bytes, void* stream);
size_t dllava_mx_decode_workspace(int32_t B, int32_t Hq, int32_t H, int32_t Dh, int32_t max_pages_per_seq);

/*
 * dllava_prefill_attn in rows with grouped heads: for row i of sequence b and query head h, with g = h / (Hq / Hkv),
 *   O[i,h] = softmax_{j <= i}(scale * Q[i,h] . K[j,g]) V[j,g]      (rows of other sequences take no part)
 *   Q [rows, Hq, Dh] row stride ldq, K, V [rows, Hkv, Dh] row stride ldkv (elements; a fused projection's output can be passed as it is:
 *   ldq = ldkv = (Hq + 2 Hkv) * Dh), O [rows, Hq, Dh] contiguous, out; only rows < off[B] are written.  off, rows as in dllava_prefill_attn.
 * Scores, softmax statistics and sums are float32; with DLLAVA_BF16 probabilities are rounded to bfloat16 before they meet the values.
 * Sizes: Dh in {64, 128}, Hq % Hkv == 0, row strides in multiples of 16 bytes, a row at most 2^27 bytes, rows < 2^31 (float32: 2^24).  dtype DLLAVA_F32 or DLLAVA_BF16.
 */
int dllava_group_prefill_attn(const void* Q, int64_t ldq, const void* K, const void* V, int64_t ldkv, int32_t B, const int32_t* off, int64_t rows,
                              int32_t Hq, int32_t Hkv, int32_t Dh, float scale, void* O, int dtype, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DLLAVA_MX_H */
