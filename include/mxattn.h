/*
 * mxattn.h -- C ABI of libmxattn: MXFP4 attention forward for MI355X (gfx950).
 *
 * The library implements the hot path of "MXAttention: Data-Free Optimal
 * Scaling and Pre-Normalization Quantization for MXFP4 Attention":
 *
 *   1. an MXFP4 quantizer (32-element E2M1 blocks sharing one E8M0
 *      power-of-two scale) with either the OCP floor scale rule
 *      e = floor(log2 M) - 2 (Sec. 2, Eq. ocp_scale) or the Universal Optimal
 *      Scaling rule e = ceil(log2(M / 7.25)) (Sec. 4.1, Algorithm 1);
 *   2. a fused flash-style attention forward on MXFP4 Q, K, V: S = Q^K^T on
 *      block-scaled FP4 matrix cores, online softmax, in-register MXFP4
 *      quantization of the unnormalized exponential tile, and O~ += P^V^ on
 *      FP4 matrix cores (Algorithm 2 without its Hadamard rotation).
 *
 * Everything is asynchronous on the caller's HIP stream.  All tensor
 * pointers are device pointers owned by the caller; the library never frees
 * or retains them.  Arguments are validated before anything is launched; on
 * an error nothing is launched and a nonzero status is returned.  The library
 * never aborts, prints or throws.  Inputs must be finite (not checked).
 *
 * Layouts (row-major, bf16 = IEEE binary32 truncated to its top 16 bits):
 *   Q, K, V, O        bf16 [B, H, N, d], d = 128.
 *   head-dim blocks   (block_axis = 3, used for Q and K): 32 consecutive
 *                     channels of one token.
 *                     codes  uint8 [B, H, N, d/2]   element 2i in the low
 *                                                   nibble of byte i
 *                     scales uint8 [B, H, N, d/32]  E8M0 (bias 127)
 *   token blocks      (block_axis = 2, used for V): 32 consecutive tokens of
 *                     one channel; the last block of a row is padded with +0.
 *                     codes  uint8 [B, H, d, nb*16] nb = ceil(N/32), tokens
 *                                                   contiguous per channel
 *                     scales uint8 [B, H, d, nb]
 *   A 4-bit code is sign(1) | magnitude index(3) into the E2M1 grid
 *   {0, 0.5, 1, 1.5, 2, 3, 4, 6} (Sec. 2, "MXFP4 Block Quantization").
 *
 * Rounding of the quantizer (readings of the paper, which says only "round
 * to nearest with saturation at +-6"): ties go to the even code, magnitudes
 * above 6 saturate to 6, the code keeps the input's sign bit even for a zero
 * magnitude, the E8M0 exponent is clamped to [-127, 127], and an all-zero
 * block gets scale byte 127 (sigma = 1, as Algorithm 1 states).
 */
#ifndef MXATTN_H
#define MXATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Scale rule, row-sum placement and rotation (rows of the paper's
 * sequential ablation, Sec. 5.4):
 *   MXATTN_OCP_VANILLA  OCP floor rule for Q, K, V and P~; direct placement:
 *                       l accumulates the unquantized P~ (Eq.
 *                       direct_mxfp4_tile, Sec. 4.2).
 *   MXATTN_UOS          UOS rule (Algorithm 1) everywhere; direct placement.
 *   MXATTN_UOS_PNQ      UOS rule everywhere; Pre-Normalization Quantization:
 *                       l accumulates the quantized P^ that also feeds the PV
 *                       product (Eqs. pnq_tile_contribution and
 *                       pnq_online_update; Algorithm 2).
 *   MXATTN_UOS_PNQ_ROT  as MXATTN_UOS_PNQ, and Q and K are multiplied by the
 *                       fixed Hadamard rotation R_H = H/sqrt(128) before
 *                       quantization (Sec. 4.3; Algorithm 2, its first two
 *                       steps): Sylvester ordering, formed in fp32 by the
 *                       radix-2 fast Walsh-Hadamard transform (stages
 *                       h = 1, 2, ..., 64, pairs (a, b) -> (a + b, a - b)),
 *                       then one fp32 multiply by fp32(1/sqrt(128)); the
 *                       fp32 result is quantized directly.  V is not
 *                       rotated.  Since (Q R_H)(K R_H)^T = Q K^T, the
 *                       attention the operands represent is unchanged. */
typedef enum {
    MXATTN_OCP_VANILLA = 0,
    MXATTN_UOS = 1,
    MXATTN_UOS_PNQ = 2,
    MXATTN_UOS_PNQ_ROT = 3
} mxattn_mode;

typedef enum {
    MXATTN_OK = 0,
    MXATTN_ERR_NULL = 1,        /* a required pointer is NULL              */
    MXATTN_ERR_SHAPE = 2,       /* B, H or N < 1, beyond a size limit, or an
                                   output that overlaps an input            */
    MXATTN_ERR_ALIGN = 3,       /* a pointer is not 16-byte aligned, or a
                                   stride is no multiple of 8 elements      */
    MXATTN_ERR_MODE = 4,        /* mode is not an mxattn_mode value         */
    MXATTN_ERR_AXIS = 5,        /* block_axis is not 2 or 3                 */
    MXATTN_ERR_UNSUPPORTED = 6, /* d != 128                                 */
    MXATTN_ERR_OOM = 7,         /* workspace allocation failed              */
    MXATTN_ERR_HIP = 8,         /* a HIP call failed; see mxattn_last_error */
    MXATTN_ERR_BOUNDARY = 9,    /* a scale boundary q outside [4, 8], a
                                   boundary count outside [1, 64], or a
                                   pre-scale gamma not in (0, 3e38)         */
    MXATTN_ERR_SCRATCH = 10,    /* the problem needs more than the static
                                   scratch of mxattn_cross_attend_noalloc, or
                                   than the workspace that a call of attention
                                   over the cache was given (none, under graph
                                   capture)                                 */
    MXATTN_ERR_VALUE = 11       /* rot, pairs, eps, page_tokens, window, sinks,
                                   budget or recent outside what the call
                                   takes, Hq no multiple of Hkv or more than
                                   256 times as many                        */
} mxattn_status;

#define MXATTN_AXIS_TOKENS 2   /* blocks along N (V)      */
#define MXATTN_AXIS_HEAD_DIM 3 /* blocks along d (Q and K) */
#define MXATTN_MAX_BOUNDARIES 64 /* boundaries per mxattn_qmax_sse call */

/* MXFP4-quantize a bf16 tensor x [B, H, N, d] (Algorithm 1 with the scale
 * rule of `mode`: OCP floor for MXATTN_OCP_VANILLA, UOS otherwise).  With
 * MXATTN_UOS_PNQ_ROT and block_axis MXATTN_AXIS_HEAD_DIM the rows are first
 * rotated by R_H (Q and K of that mode); along MXATTN_AXIS_TOKENS that mode
 * quantizes like MXATTN_UOS_PNQ.
 *   x       device, bf16 [B, H, N, d], 16-byte aligned
 *   codes   device, layout of `block_axis` above, 16-byte aligned,
 *           mxattn_codes_bytes() bytes
 *   scales  device, layout of `block_axis` above, mxattn_scales_bytes() bytes
 *   stream  hipStream_t to run on (NULL: the null stream)
 * Returns MXATTN_OK or an error status; nothing is launched on error. */
int mxattn_quantize(const void* x, uint8_t* codes, uint8_t* scales, int block_axis, int mode,
                    int64_t B, int64_t H, int64_t N, int64_t d, void* stream);

/* MXFP4-quantize with the ceil scale rule of a general boundary q: each
 * block takes the smallest exponent e with M <= q 2^e (Eq. scale_definition,
 * Eq. uos_mapping), clamped to [-127, 127].  q = 6 is TFS, q = 7 the OAS rule
 * at 32-element blocks (App. "Relation to OAS and the OCP Endpoint
 * Convention"), q = 7.25 UOS (identical to mxattn_quantize in a UOS mode) and
 * q = 8 the ceil form of the OCP boundary (which differs from the floor rule
 * of MXATTN_OCP_VANILLA only where M is a power of two).  Layouts, rounding
 * and alignment as mxattn_quantize; no rotation.
 *   qmax    the boundary q, 4 <= q <= 8 (MXATTN_ERR_BOUNDARY otherwise)
 * Returns MXATTN_OK or an error status; nothing is launched on error. */
int mxattn_quantize_qmax(const void* x, uint8_t* codes, uint8_t* scales, int block_axis, double qmax,
                         int64_t B, int64_t H, int64_t N, int64_t d, void* stream);

/* Per-(batch, head) sum of squared MXFP4 quantization errors
 * sum_i (x_i - Q_q(x_i))^2 of x [B, H, N, d], blocked along block_axis, for
 * each boundary qs[j] of the ceil rule above: the per-tensor MSE sweep of
 * the paper's empirical check of the boundary (Sec. 5.5, Table
 * cx_distribution, which sweeps q from 6.00 to 8.00 in steps of 0.05).
 * Token blocks count their +0 padding, which adds no error.
 *   x       device bf16 [B, H, N, d], 16-byte aligned, finite
 *   qs      HOST array of nq boundaries, each 4 <= q <= 8, read before the
 *           call returns; 1 <= nq <= MXATTN_MAX_BOUNDARIES
 *   sse     device fp64 [B*H, nq], 8-byte aligned, written in full
 * Sums are formed in fp64 (each element's squared error exactly); the order
 * of additions within a workgroup is not fixed, so repeated calls may differ
 * in the last bits.  Uses stream-ordered workspace (the library's pool,
 * see mxattn_release_workspace): 2056 bytes per workgroup, at most 2048
 * workgroups or one per (batch, head) if there are more, so at most about
 * 2 KiB * max(B*H, 2048).
 * Returns MXATTN_OK, MXATTN_ERR_OOM, or another error status. */
int mxattn_qmax_sse(const void* x, int block_axis, const double* qs, int nq, double* sse, int64_t B,
                    int64_t H, int64_t N, int64_t d, void* stream);

/* Row-sum diagnostics of MXFP4-quantized attention probabilities (Sec. 5.5,
 * "Validation of Pre-Normalization Quantization", Fig. pnq_rowsum): what
 * direct block quantization of a materialized, normalized P does to the mass
 * of each row, which PNQ avoids.  Per row, stats holds 8 fp64 values
 *   [0] sum_j Q(x_j) / gamma        the row sum after quantization
 *   [1] sum_j p_j                    the row sum before
 *   [2] zeroing     sum of Q(x_j)/gamma - p_j over p_j > 0 with Q(x_j) = 0
 *   [3] saturation  ... over x_j / sigma > 6 (above the largest E2M1 value)
 *   [4] down        ... over the other entries with Q(x_j) < x_j
 *   [5] up          ... over Q(x_j) > x_j
 *   [6] exact       ... over Q(x_j) = x_j
 *   [7] entropy     -sum_{p_j > 0} p_j ln p_j (nats)
 * with x_j = fp32(gamma * p_j) quantized in blocks of 32 consecutive entries
 * of the row (the last block padded with +0) by the scale rule of `mode`
 * (OCP floor for MXATTN_OCP_VANILLA, UOS otherwise), and 1/gamma rounded to
 * fp64.  gamma is the single "pre-quant global scaling" factor of
 * Fig. pnq_rowsum (C); gamma = 1 quantizes P as it is.  [0] - [1] equals
 * [2] + ... + [6] up to rounding.  Sums are fp64 (each term exact but the
 * entropy's, which uses the fp32 base-2 logarithm); workgroup reductions run
 * in a fixed order.
 *
 * mxattn_softmax_rows materializes p = softmax(q k^T / sqrt(d)) for the query
 * rows [row0, row0 + rows) of every (batch, head): S on the bf16 matrix cores
 * with fp32 accumulation, p = 2^(s log2(e)/sqrt(d) - m) / L in fp32 (entries
 * below 2^-126 flush to 0).
 *   q       device bf16 [B, H, Nq, d]; k device bf16 [B, H, Nkv, d]
 *   p       device fp32 [B, H, rows, ld], ld >= Nkv, ld % 4 == 0; entries
 *           past Nkv up to the next multiple of 4 are set to 0, the rest of
 *           [Nkv, ld) is not written
 * mxattn_rowsum_diag quantizes given rows:
 *   p       device fp32 [rows, ld], entries >= 0 (first N of each row used),
 *           ld >= N, ld % 4 == 0, 16-byte aligned
 *           (an infinite entry makes [1] and [3] infinite, a NaN entry makes [1]
 *           and [6] NaN, for every gamma)
 *   stats   device fp64 [rows, 8]
 * mxattn_attention_rowsum_diag computes the same statistics for every query
 * row of q against k without materializing P: the probabilities are formed
 * exactly as mxattn_softmax_rows forms them and quantized in registers, so
 * the result equals mxattn_rowsum_diag applied to mxattn_softmax_rows up to
 * the order of the fp64 additions.  No workspace.
 *   stats   device fp64 [B, H, Nq, 8]
 * All three return MXATTN_OK or an error status; nothing is launched on
 * error. */
int mxattn_softmax_rows(const void* q, const void* k, float* p, int64_t B, int64_t H, int64_t Nq,
                        int64_t Nkv, int64_t d, int64_t row0, int64_t rows, int64_t ld, void* stream);
int mxattn_rowsum_diag(const float* p, int64_t rows, int64_t N, int64_t ld, int mode, float gamma,
                       double* stats, void* stream);
int mxattn_attention_rowsum_diag(const void* q, const void* k, int64_t B, int64_t H, int64_t Nq,
                                 int64_t Nkv, int64_t d, int mode, float gamma, double* stats,
                                 void* stream);

/* MXFP4 attention forward O = softmax(Q K^T / sqrt(d)) V with MXFP4 Q, K, V
 * and MXFP4 P~ (Algorithm 2, with its Hadamard rotation in mode
 * MXATTN_UOS_PNQ_ROT only; non-causal, no mask besides the sequence end).
 * Quantizes K along d and V along N into stream-ordered workspace (from
 * the library's pool on `stream`, see mxattn_release_workspace; about 0.53
 * bytes per element of each of K and V, the scales in whole tiles of 128 keys
 * and V too where there are more than 96; calls with few queries over many keys
 * take up to 34 MiB more, for partial results of runs of the keys, see
 * mxattn_cross_forward), then runs
 * the fused kernel, which quantizes Q along d in
 * its prologue with codes bit-identical to mxattn_quantize's; in
 * MXATTN_UOS_PNQ_ROT, Q is rotated and quantized into the workspace first
 * (0.53 bytes per element more).
 *   q, k, v  device bf16 [B, H, N, d], 16-byte aligned
 *   out      device bf16 [B, H, N, d], 16-byte aligned; MXATTN_ERR_SHAPE if
 *            it shares a byte with q, k or v
 * Size limits (MXATTN_ERR_SHAPE otherwise): N <= 2^24 keys (the kernel
 * addresses one head's quantized K and V with 32-bit byte offsets) and
 * B * H * ceil(N / 128) <= 2^30 query tiles.
 * Returns MXATTN_OK, MXATTN_ERR_OOM if the workspace cannot be allocated, or
 * another error status; nothing is launched on an argument error. */
int mxattn_forward(const void* q, const void* k, const void* v, void* out, int64_t B, int64_t H,
                   int64_t N, int64_t d, int mode, void* stream);

/* The fused attention kernel alone, on already quantized operands (the
 * layouts above: Q and K blocked along d, V blocked along N).  The scale rule
 * of `mode` applies to the in-kernel quantization of P~; `mode` also selects
 * direct or PNQ placement.  All pointers are device pointers; code arrays
 * and `out` are 16-byte aligned, k_scales 4-byte aligned, the other scale
 * arrays may have any alignment.  MXATTN_ERR_SHAPE if `out` shares a byte
 * with any code or scale array. */
int mxattn_attend(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                  const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                  void* out, int64_t B, int64_t H, int64_t N, int64_t d, int mode, void* stream);

/* Attention with different query and key/value lengths (cross-attention:
 * video queries attending to a short text sequence; the paper's Wan2.2 has
 * separate cross-attention modules, Sec. 5.1).  q and out are [B, H, Nq, d],
 * k and v are [B, H, Nkv, d]; the quantized variants take Q^ blocked along d
 * with Nq rows, K^ blocked along d with Nkv rows and V^ blocked along Nkv.
 * Otherwise as mxattn_forward / mxattn_attend, which are these calls with
 * Nq = Nkv = N; the key limit N <= 2^24 applies to Nkv.
 *
 * Calls whose query tiles (128 queries of one head) leave most of the chip idle
 * divide the keys of a head into runs; whether and into how many follows from
 * B * H, Nq and Nkv.  The running maximum, P~ and P^ are those of the undivided
 * sequence, but O~ and l are sums of fp32 partial sums: an output element may
 * differ by one bf16 unit in the last place (about one in 10 000 does) between
 * calls that divide the same head differently, as a call of all heads and one
 * of a few of them may.  Equal shapes give equal bits. */
int mxattn_cross_forward(const void* q, const void* k, const void* v, void* out, int64_t B,
                         int64_t H, int64_t Nq, int64_t Nkv, int64_t d, int mode, void* stream);
int mxattn_cross_attend(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                        const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                        void* out, int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d, int mode,
                        void* stream);

/* mxattn_cross_attend without any allocation, for callers that cannot
 * allocate device memory: code under HIP graph capture, tight serving loops,
 * and harnesses that forbid allocation.  Same arguments, checks and result
 * as mxattn_cross_attend (bit-identical output, the same kernels); it calls
 * no hipMalloc, hipMallocAsync, hipFree or any allocating routine.  Its one
 * buffer beyond the inputs and `out`, the K^ and V^ scales rearranged into
 * the kernel's operand order (1 KiB per (batch, head) and 128-key tile), is
 * a static device array of MXATTN_NOALLOC_SCRATCH_BYTES, followed by 34 MiB for
 * the partial results of calls with few queries over many keys, which a device
 * holds from the first such call on it until the process ends.  Limit: B * H *
 * ceil(Nkv / 128) <= 32768 (e.g. H = 40 heads of up to 104 832 keys), else
 * MXATTN_ERR_SCRATCH with a message in mxattn_last_error and nothing
 * launched.  The array is fully rewritten by every call before it is read,
 * but all calls on one device share it: calls that overlap in time on one
 * device (different streams without ordering between them) race and give
 * undefined results.  The first call on a device looks up the array's
 * device address (hipGetSymbolAddress); MXATTN_ERR_HIP if that fails. */
#define MXATTN_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)
int mxattn_cross_attend_noalloc(const uint8_t* q_codes, const uint8_t* q_scales, const uint8_t* k_codes,
                                const uint8_t* k_scales, const uint8_t* v_codes, const uint8_t* v_scales,
                                void* out, int64_t B, int64_t H, int64_t Nq, int64_t Nkv, int64_t d,
                                int mode, void* stream);

/* ---- Queries and keys before attention, and K and V kept between calls.
 *
 * Norm and rotation of a head's 128 channels x at a position, in fp32:
 *   y = x / sqrt(mean(x^2) + eps) * w         (w null: y = x)
 *   (a, b) -> (a cos - b sin, b cos + a sin)  for each pair of the first `rot`
 *                                             channels (rot 0: none)
 *   pairs     MXATTN_PAIRS_INTERLEAVED (2i, 2i+1) or MXATTN_PAIRS_HALVES
 *             (i, i + rot/2), i < rot/2
 *   rot       0, or a multiple of 16 up to 128
 *   cos, sin  device fp32 [table_rows, rot/2], 16-byte aligned: row p is the
 *             angles of position p.  A position outside [0, table_rows) makes the
 *             row's rotated channels NaN.
 *   w         device fp32 [128], 16-byte aligned
 *   eps       finite, >= 0 (used where w is given)
 * All strides are in elements, non-negative and multiples of 8; pointers of bf16
 * data are 16-byte aligned. */
#define MXATTN_PAIRS_INTERLEAVED 0
#define MXATTN_PAIRS_HALVES 1

/* Norm and rotation of Q [B, Hq, N, d] and K [B, Hkv, N, d] in one launch, each
 * rounded once to bf16: what a projection wrote, in any order of its axes, becomes
 * the operands of mxattn_forward or mxattn_cache_attend.
 *   q, k            device bf16; k (with k_out) may be NULL: Q alone
 *   *_strides       HOST int64[3], of batch, head and token; NULL: contiguous
 *                   [B, H, N, d].  Output rows must not overlap one another.
 *   positions       device int32 [B, N], or NULL: a token's index in its batch
 * MXATTN_ERR_SHAPE if the span of an output (first to last byte) shares a byte
 * with the span of an input or of the other output. */
int mxattn_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out, int64_t B, int64_t Hq,
                        int64_t Hkv, int64_t N, int64_t d, const int64_t* q_strides,
                        const int64_t* k_strides, const int64_t* q_out_strides,
                        const int64_t* k_out_strides, const float* q_weight, const float* k_weight,
                        float eps, const float* cos, const float* sin, const int32_t* positions,
                        int64_t table_rows, int64_t rot, int pairs, void* stream);

/* The paged cache.  K and V are held as 8-bit codes (E4M3: 4 exponent and 3
 * fraction bits, largest 448) with one E8M0 scale per block of 32 consecutive
 * tokens of a sequence and head.  Pages of `page_tokens` tokens (a power of two,
 * 32 to 4096) are given to sequences by a page table.
 *   k_codes   uint8 [pages, Hkv, page_tokens/32, 8, 32, 16]: channel 16 c + i of
 *             token t of a block at [c][t][i]
 *   v_codes   uint8 [pages, Hkv, page_tokens/32, 128, 32]: channel, token
 *   k_scales, v_scales  uint8 [pages, Hkv, page_tokens/32]
 * all on the device, codes 16-byte aligned.  A call's tokens belong to sequences:
 *   page_table  device int32 [seqs, max_pages]: the pages of a sequence in order;
 *               entries past its length are not read
 *   q_start     device int32 [seqs + 1], ascending from 0: sequence s owns the call's
 *               tokens q_start[s] .. q_start[s+1] - 1 (it may own none); tokens
 *               behind the last sequence are left alone
 *   kv_len      device int32 [seqs]: the sequence's length with these tokens, which
 *               are its last ones.  Token i of n has position kv_len - n + i.
 * These arrays are read by the kernels only (4-byte aligned).  Bad contents read
 * and write nothing out of range: a kv_len below 0 or past max_pages * page_tokens,
 * or a page outside [0, pages), appends nothing there and gives NaN to every query
 * that would see it; a q_start that does not ascend gives undefined results.
 * Limits (MXATTN_ERR_SHAPE otherwise): Hkv <= 65535, seqs <= 2^20,
 * max_pages * page_tokens <= 2^24, pages * Hkv * page_tokens <= 2^45. */

/* Append the call's tokens to the cache: K normed and rotated (w, eps, cos, sin,
 * table_rows, rot, pairs as above; positions: device int32 [tokens], or NULL: a
 * token's place in its sequence) and rounded once, V as it is.  A block's exponent
 * is the smallest e >= -127 with max|x| <= 448 2^e over its new tokens, and at
 * least that of the block if it holds older tokens; if it grew, those are rounded
 * again, code * 2^(e_old - e).  Rounding is to nearest, ties to even.  Values that
 * are not finite are stored as NaN and do not count towards the maximum.  Bytes of
 * tokens past the sequence's end are left as they were.  Tokens whose position is
 * negative (kv_len < n) are not stored.  A call's tokens must not reach one page
 * by two entries of the page table (which of them is stored is undefined).
 *   k, v   device bf16 [tokens, Hkv, d], heads contiguous, token strides
 * MXATTN_ERR_SHAPE if k or v shares a byte with the cache. */
int mxattn_cache_append(const void* k, const void* v, int64_t k_stride, int64_t v_stride, uint8_t* k_codes,
                        uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, int64_t pages,
                        int64_t page_tokens, const int32_t* page_table, const int32_t* q_start,
                        const int32_t* kv_len, int64_t seqs, int64_t max_pages, int64_t tokens, int64_t Hkv,
                        int64_t d, const float* k_weight, float eps, const float* cos, const float* sin,
                        const int32_t* positions, int64_t table_rows, int64_t rot, int pairs, void* stream);

/* Attention of the call's tokens over their sequences' cached keys (their own
 * among them, appended before): O = softmax(Q K^T / sqrt(d)) V with fp32 scores,
 * softmax and sums.  Query head i reads KV head i / (Hq / Hkv).  Four choices hold
 * less than fp32: scores are sums of the FP8 matrix cores (off by up to 2^-15 of
 * sum |q k|, as measured); P is rounded to f16 before its product with V (by 2^-11 of each p,
 * or 2^-36 of the row's largest below 2^-25 of that); Q is held to 2^-21 of its row's
 * largest magnitude; and blocks of V whose scale is below 2^-55 of the largest one of
 * their sequence lose digits.  Scores of 2^26 and more in magnitude, and keys of 2^112
 * and more, may give inf or NaN.
 * causal != 0: token i of n sees positions 0 .. kv_len - n + i, else all kv_len.
 * A query that sees no key gets 0.
 *   q     device bf16 [tokens, Hq, d], heads contiguous, token stride; Hq at most
 *         256 Hkv, (tokens * Hq / Hkv / 32 + seqs) * Hkv < 2^24
 *   out   device bf16 [tokens, Hq, d], likewise; tokens of no sequence are not
 *         written.  MXATTN_ERR_SHAPE if it shares a byte with q or the cache.
 *   max_q, max_kv  at least the new tokens and the keys of every sequence, as the
 *         caller knows them on the host; 0: unknown (tokens, and max_pages *
 *         page_tokens).  They choose how the work is divided: bounds that are too
 *         small or far too large cost time, not correctness.  Where the work is cut
 *         decides which running maximum each p is rounded under, and in what order
 *         fp32 sums are formed: other bounds, and other lengths of the call's other
 *         sequences, may change an output by these roundings (2^-11 of each p), so by
 *         its last bit or, where values cancel, by 2^-11 of sum p |v|.
 *   workspace  device memory of the caller, 16-byte aligned, of at least
 *         mxattn_cache_attend_workspace() bytes (else MXATTN_ERR_SCRATCH), for this
 *         call until it has run; what it holds before does not matter.  It shares no
 *         byte with q, out or the cache (MXATTN_ERR_SHAPE).  NULL: from the
 *         library's pool, which a stream under graph capture cannot use: there a
 *         call that needs workspace is refused (MXATTN_ERR_SCRATCH).
 * Equal arguments and contents give equal bits (a sequence's output may have others in
 * another batch, as said). */
int mxattn_cache_attend(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                        const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                        const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len,
                        int64_t seqs, int64_t max_pages, int64_t tokens, int64_t Hq, int64_t Hkv, int64_t d,
                        int causal, int64_t max_q, int64_t max_kv, void* out, int64_t out_stride,
                        void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace that mxattn_cache_attend needs: none where max_kv <= 1024 and
 * max_q * Hq / Hkv <= 128, else at most 65 MiB, and 8 bytes per KV head for each
 * sequence and each 32 query rows.  0 also for sizes that the call refuses. */
size_t mxattn_cache_attend_workspace(int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t tokens,
                                     int64_t Hq, int64_t Hkv, int64_t max_q, int64_t max_kv);

/* Attention of a call's tokens over part of their sequences' cached keys: as
 * mxattn_cache_attend (its arguments, limits, workspace and precision, the same keys
 * in the same order), but with T = kv_len - n + i + 1 (causal) or kv_len, a token
 * sees the last `window` keys before T, positions T - window .. T - 1, and positions
 * 0 .. sinks - 1 of those before T.  Page table entries whose pages no token of the
 * call sees are not read: a program may have given those pages away.
 *   window  >= 1, sinks >= 0 (MXATTN_ERR_VALUE otherwise)
 * mxattn_cache_attend_workspace() bytes with the same max_q and max_kv suffice. */
int mxattn_cache_attend_window(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                               const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages,
                               int64_t page_tokens, const int32_t* page_table, const int32_t* q_start,
                               const int32_t* kv_len, int64_t seqs, int64_t max_pages, int64_t tokens,
                               int64_t Hq, int64_t Hkv, int64_t d, int64_t window, int64_t sinks, int causal,
                               int64_t max_q, int64_t max_kv, void* out, int64_t out_stride, void* workspace,
                               size_t workspace_bytes, void* stream);

/* Attention for drafted tokens that form trees: as mxattn_cache_attend, but token i of n
 * sees positions 0 .. kv_len - n - 1, and of the n new ones (position kv_len - n + j)
 * those whose bit j is set in its mask: its ancestors and, where it is to see itself,
 * bit i.
 *   tree        device int32 [tokens, tree_words]: bit j & 31 of word j >> 5.  New tokens
 *               from 32 tree_words on are seen by none; bits from n on do not count.
 *   tree_words  1 .. 2^19
 * Rotation by depth is the caller's: give mxattn_cache_append the positions.
 * mxattn_cache_compact moves the tokens that were accepted to the sequence's end. */
int mxattn_cache_attend_tree(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                             const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages, int64_t page_tokens,
                             const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len,
                             int64_t seqs, int64_t max_pages, int64_t tokens, int64_t Hq, int64_t Hkv, int64_t d,
                             const int32_t* tree, int64_t tree_words, int64_t max_q, int64_t max_kv, void* out,
                             int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream);

/* mxattn_cache_attend that also weighs the keys: for every position j of a sequence
 * that owns tokens of the call, and every KV head,
 *   weights_out[j] = (j < kv_len - n ? weights[j] : 0) + sum of p over the n tokens and the
 *                    Hq / Hkv heads
 * in fp32, p the probabilities that O is made of (before they are rounded to f16).  Scores
 * are fp32 sums of exact products in this call, whatever its bounds: off by 2^-20 of
 * sum |q k| and less, and the p of a row add up to 1 but for the rounding of their fp32 sums
 * (2^-16 over 3000 keys).  Weights lie beside the cache, fp32 [pages, Hkv, page_tokens]; those
 * of other positions and sequences are not written.
 *   weights      NULL: zeros.  A key that was new to a call without weights has what lies there.
 *   weights_out  may be `weights`; must not overlap it otherwise
 *   max_kv       here a limit: a sequence that is longer counts as one of impossible
 *                length (its queries get NaN, its weights are not written).
 * A query that gets NaN (see above) makes the weights of the keys it sees NaN.  Equal
 * arguments and contents give equal bits.  Two sequences of a call must not share a page
 * (which one's weights are stored there is undefined).
 *   workspace    mxattn_cache_attend_weights_workspace() bytes: mxattn_cache_attend's, 8 for
 *                each token and head, and with few tokens the scores, 4 for each token,
 *                head and key of max_kv, at most 1 GiB (with many over few keys, up to
 *                256 KiB for partial sums). */
int mxattn_cache_attend_weights(const void* q, int64_t q_stride, const uint8_t* k_codes, const uint8_t* k_scales,
                                const uint8_t* v_codes, const uint8_t* v_scales, int64_t pages,
                                int64_t page_tokens, const int32_t* page_table, const int32_t* q_start,
                                const int32_t* kv_len, int64_t seqs, int64_t max_pages, int64_t tokens,
                                int64_t Hq, int64_t Hkv, int64_t d, const float* weights, float* weights_out,
                                int causal, int64_t max_q, int64_t max_kv, void* out, int64_t out_stride,
                                void* workspace, size_t workspace_bytes, void* stream);
size_t mxattn_cache_attend_weights_workspace(int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t tokens,
                                             int64_t Hq, int64_t Hkv, int64_t max_q, int64_t max_kv);

/* Which of a sequence's tokens stay when it is cut to `budget`, for every KV head: all
 * if there are no more; else the first `sinks`, the last `recent` and, of those between,
 * the ones of the largest weight (of equal ones the first; NaN and pages that do not
 * exist weigh less than every number).
 *   weights  device fp32 [pages, Hkv, page_tokens]
 *   kept     device int32 [seqs, Hkv, budget]: their positions, ascending, then -1
 *   counts   device int32 [seqs]: min(kv_len, budget); 0 for an impossible length
 *   budget   1 .. 2^24, sinks >= 0, recent >= 0, sinks + recent <= budget
 *            (MXATTN_ERR_VALUE otherwise); seqs * Hkv < 2^22
 * Kernels and workspace go by the table's width, max_pages * page_tokens: short sequences
 * are cut faster under a narrow table.
 *   workspace  as mxattn_cache_attend's, of mxattn_cache_select_workspace() bytes: none
 *            where max_pages * page_tokens <= 16384 (65536 from seqs * Hkv = 128 on), else at
 *            most 2.3 MB for each sequence and KV head.  It shares no byte with the other
 *            arguments.  NULL: from the library's pool, not under graph capture. */
int mxattn_cache_select(const float* weights, int64_t pages, int64_t page_tokens, const int32_t* page_table,
                        const int32_t* kv_len, int64_t seqs, int64_t max_pages, int64_t Hkv, int64_t budget,
                        int64_t sinks, int64_t recent, int32_t* kept, int32_t* counts, void* workspace,
                        size_t workspace_bytes, void* stream);
size_t mxattn_cache_select_workspace(int64_t page_tokens, int64_t seqs, int64_t max_pages, int64_t Hkv);

/* Move kept tokens together: position base + i of a sequence (i < counts) becomes what was
 * at position kept[i], K, V and weights; the sequence's length is then base + counts.
 * What is at positions below base stays (in the first block that is written, with the
 * others' scale).  A block takes the largest scale of the blocks that its tokens come
 * from, and code * 2^(e_old - e) is rounded to nearest, ties to even: exact unless it
 * falls below 2^-6.  A block's codes behind the last token become 0.
 *   kept       device int32 [seqs, kept_heads, width]; kept_heads is Hkv, or 1: the same for
 *              all heads.  A position that the page table does not have, or whose page
 *              does not exist, or whose scale is no number gives NaN codes (and weight 0
 *              without a page).
 *   counts     device int32 [seqs]; nothing is done for a sequence of a count outside
 *              1 .. width, or that does not fit the table
 *   base       device int32 [seqs], or NULL: 0
 *   out_table  device int32 [seqs, out_pages]: where the tokens go, on pages that hold
 *              none of the call's sources; nothing is written to a page that does not
 *              exist.  NULL or page_table (then of as many pages, MXATTN_ERR_SHAPE): in
 *              place, where kept ascends and kept[i] >= base + i (anything else gives
 *              undefined contents there; nothing out of range).
 *   weights    device fp32 [pages, Hkv, page_tokens], or NULL
 * Keys keep the rotation that they were stored with.  Where that is by position, tokens that
 * come later need theirs given (mxattn_cache_append's `positions`, and their queries'): a
 * token's place in its sequence, which the calls take without them, is no longer its position.
 * In place a head's K and V are two workgroups' work, 128 tokens a turn, one turn after
 * another: meant for a few blocks (accepted drafts of 16 sequences 10 us), right but slow for
 * many (118800 keys cut to 14850: 1.2 ms; into other pages 41 us, as all turns run at once there).
 * Sequences of a call must not share pages that are written.  seqs * Hkv < 2^22. */
int mxattn_cache_compact(uint8_t* k_codes, uint8_t* k_scales, uint8_t* v_codes, uint8_t* v_scales, int64_t pages,
                         int64_t page_tokens, const int32_t* page_table, int64_t seqs, int64_t max_pages,
                         const int32_t* out_table, int64_t out_pages, int64_t Hkv, int64_t d, const int32_t* kept,
                         int64_t kept_heads, int64_t width, const int32_t* counts, const int32_t* base,
                         float* weights, void* stream);

/* Sizes of the code and scale arrays of a [B, H, N, d] tensor blocked along
 * `block_axis`; 0 for invalid arguments. */
size_t mxattn_codes_bytes(int block_axis, int64_t B, int64_t H, int64_t N, int64_t d);
size_t mxattn_scales_bytes(int block_axis, int64_t B, int64_t H, int64_t N, int64_t d);

/* KV tile width B_c of the fused kernel: the running maximum is updated once
 * per B_c keys, in increasing key order (this fixes which exponentials are
 * quantized together; see Sec. 2, Eq. online_attention). */
int mxattn_kv_tile(void);

/* Query rows handled by one workgroup of the fused kernel. */
int mxattn_query_tile(void);

/* Static description of a status code. */
const char* mxattn_status_string(int status);

/* Detail of the last MXATTN_ERR_HIP, MXATTN_ERR_OOM or MXATTN_ERR_SCRATCH on
 * the calling thread ("" if none). */
const char* mxattn_last_error(void);

/* Workspace.  mxattn_forward, mxattn_cross_forward, mxattn_attend,
 * mxattn_cross_attend, mxattn_qmax_sse and the calls of attention over the cache
 * (where they are given none) take their workspace, stream-ordered, from a memory pool that belongs to the library (one per device,
 * created on first use; the device's default pool is left as it is).  The
 * pool keeps freed workspace for the next call rather than returning it to
 * the driver; one block of at most 64 MiB per device stays allocated for the
 * calls on the null stream that fit it.  mxattn_release_workspace returns all
 * of the current device's cached workspace that no call still uses, and waits
 * for none: call it after the streams that ran the library's calls have
 * completed, e.g. before a phase of a pipeline that needs the memory.  The
 * kept block stays while the null stream has work, or while a stream that
 * synchronizes with it is being captured.  Returns MXATTN_OK or
 * MXATTN_ERR_HIP. */
int mxattn_release_workspace(void);

/* ABI version (major * 100 + minor). */
int mxattn_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MXATTN_H */
