/*
 * int2kv.h -- C ABI of the rotated, key-centered INT2 KV cache and its decode attention
 * for AMD Instinct MI355X (gfx950).
 *
 * What is computed (Yun et al., "Output-Aware Rotation for INT2 KV-Cache Quantization"):
 *   cache write  (Sec. 4.1 key reparameterization; Sec. 6 efficiency analysis; appendix
 *                 "Key-mean estimation and application"):
 *       k_R = Q_2((k - mu) R_K) = Q_2(k R_K - mu R_K),   v_R = Q_2(v R_V)
 *   decode       (eq:int2_attention, eq:int2_residual_readout; appendix "Rotated-query
 *                 implementation" and "Equivalent inference implementation"):
 *       a_s = (q R_K) k_R,s^T / sqrt(d),  p = softmax_s(a),  o = (sum_s p_s v_R,s) R_V^T,
 *       y = concat_j(o_j) W_O^T   (optional)
 *   Query head j reads KV head h(j) = floor(j / G_q), G_q = H_q / H_kv (GQA, Sec. 3).
 *
 * Q_2 is group-wise affine INT2 (Sec. 5 implementation details, Table A) over groups of G = 32
 * or G = 128 (the paper's setting) consecutive rotated channels of one token. The arithmetic, fixed for bit-exactness, is
 * (all fp32, no contraction, round-to-nearest-even throughout):
 *       mn = min x, mx = max x;   if clip != 1: mn = clip*mn, mx = clip*mx
 *       s  = fp16(fp32(mx - mn) / 3),   z = fp16(mn)
 *       inv = s > 0 ? 1 / s : 0;        code = clamp(rint((x - z) * inv), 0, 3)
 *       dequantized value = code * s + z
 *
 * Conventions for every call:
 *   - All tensor pointers are DEVICE pointers owned by the caller; the library allocates
 *     nothing and never synchronizes. Work is enqueued on `stream` (0 = null stream).
 *   - bf16 and fp16 tensors are passed as uint16_t bit patterns; row-major, densely packed.
 *   - Return value: INT2KV_OK or a negative int2kv_status. On an argument error nothing is
 *     launched; int2kv_last_error() (thread-local) describes the last failure.
 *   - head_dim = 128, block_size = 16, group_size = 32 or 128 are the supported shapes.
 *
 * Packed cache (part of the bit-exact contract): with NG = 128 / group_size groups per token,
 * the pool holds one record of R = 1024 + 128 * NG bytes (1536 at G = 32, 1152 at G = 128; see
 * int2kv_record_bytes) per (physical block, KV head) at pool + (block * num_kv_heads + h) * R,
 * 16-byte aligned. Token row t (0..15) of a block and rotated channel c (0..127) are stored as
 *     [   0,  512) K codes, token-major: 16-bit half m of token t at byte 32*t + 2*m
 *     [ 512, 1024) V codes, half-major : 16-bit half m of token t at byte 512 + 32*m + 2*t
 *     [1024, 1024 + 64 NG) K scale/zero: token t, group g at 1024 + 4*NG*t + 4*g (fp16 s, fp16 z)
 *     [1024 + 64 NG, ...)  V scales: group g, token t at 1024 + 64*NG + 32*g + 2*t (fp16)
 *     [1024 + 96 NG, R)    V zeros : group g, token t at 1024 + 96*NG + 32*g + 2*t (fp16)
 *   where channel c = 16*p + m sits in half m at bits 2p..2p+1 (little endian), i.e. 2 bits
 *   per element plus 32 metadata bits per group: 3.0 bits per cached element at G = 32, 2.25 at
 *   G = 128. A cache slot is block * 16 + t.
 */
#ifndef INT2KV_H
#define INT2KV_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define INT2KV_HEAD_DIM 128
#define INT2KV_BLOCK_SIZE 16
#define INT2KV_GROUP_SIZE 32    /* default group size; 128 is also supported */
#define INT2KV_RECORD_BYTES 1536 /* record bytes at the default group size   */

typedef enum {
  INT2KV_OK = 0,
  INT2KV_EINVAL = -1,       /* bad pointer, shape or alignment                         */
  INT2KV_EUNSUPPORTED = -2, /* a shape the library does not implement                 */
  INT2KV_EWORKSPACE = -3,   /* workspace missing or smaller than required              */
  INT2KV_EHIP = -4          /* a HIP launch reported an error                          */
} int2kv_status;

/* The paged INT2 cache. `pool` points to num_blocks * num_kv_heads * int2kv_record_bytes(group_size)
 * bytes (device, 16-byte aligned). The caller zero-fills it once; every slot is rewritten in full
 * by an append, so no clearing is needed when blocks are reused. */
typedef struct int2kv_cache {
  void* pool;
  int32_t num_blocks;
  int32_t num_kv_heads;
  int32_t block_size; /* must be 16  */
  int32_t head_dim;   /* must be 128 */
  int32_t group_size; /* 32 or 128   */
} int2kv_cache;

/* Thread-local description of the last non-OK status ("" if none). */
const char* int2kv_last_error(void);

/* Library version string. */
const char* int2kv_version(void);

/* Bytes of the pool for the given shape: num_blocks * num_kv_heads * int2kv_record_bytes(group_size)
 * (0 for a group size other than 32 or 128, or a non-positive count). */
size_t int2kv_pool_bytes(int num_blocks, int num_kv_heads, int group_size);

/* Bytes of one (block, KV head) record: 1536 at group size 32, 1152 at 128, 0 otherwise. */
size_t int2kv_record_bytes(int group_size);

/* Rotated key mean mu_h R_{K,h}, precomputed once per KV head and subtracted right after the
 * key rotation in the cache write (Sec. 6 efficiency analysis; appendix key-mean
 * application: (k - mu) R_K = k R_K - mu R_K).
 *   R_k   : fp32 [H_kv, 128, 128], row-major, the row-vector rotation z -> z R_K
 *   mu    : fp32 [H_kv, 128]
 *   mu_rk : fp32 [H_kv, 128] (output)
 * Accumulates in fp32 in channel order. */
int int2kv_prepare_mu_rot(const float* R_k, const float* mu, float* mu_rk, int num_kv_heads,
                          hipStream_t stream);

/* Folded output projection W-bar_{O,j} = W_{O,j} R_{V,h(j)} (appendix "Equivalent inference
 * implementation"), so that y = concat_j(o'_j) W-bar_O^T with o'_j = o_j R_V needs no
 * un-rotation.
 *   W_o        : bf16 [d_model, H_q*128] row-major (W_{O,j} = columns j*128 .. j*128+127)
 *   R_v        : fp32 [H_kv, 128, 128]
 *   W_o_folded : bf16 [d_model, H_q*128] (output; fp32 accumulation, rounded once to bf16) */
int int2kv_fold_wo(const uint16_t* W_o, const float* R_v, uint16_t* W_o_folded, int d_model,
                   int num_q_heads, int num_kv_heads, hipStream_t stream);

/* Output-projection weights in the form the decode's projection streams best: fp16, stored as
 * 128-row x 32-column operand tiles, each 8 KiB tile contiguous (row blocks padded with zero
 * rows to a multiple of 128). With R_v given, the value rotation is folded in first, as in
 * int2kv_fold_wo (W-bar_{O,j} = W_{O,j} R_{V,h(j)}, appendix "Equivalent inference
 * implementation"), accumulated in fp32 and rounded once to fp16; without it the bf16 weights
 * are converted exactly. Weights must lie within the fp16 range (|w| <= 65504); values below
 * 2^-14 keep the fp16 subnormal spacing 2^-24. Done once per layer, like the fold.
 *   W_o        : bf16 [d_model, H_q*128] row-major
 *   R_v        : fp32 [H_kv, 128, 128], or NULL (no fold)
 *   W_prepared : int2kv_prepared_wo_bytes(d_model, H_q) bytes, 16-byte aligned (output); must
 *                not overlap W_o */
size_t int2kv_prepared_wo_bytes(int d_model, int num_q_heads);
int int2kv_prepare_wo(const uint16_t* W_o, const float* R_v, uint16_t* W_prepared, int d_model,
                      int num_q_heads, int num_kv_heads, hipStream_t stream);

/* Weight formats of the output projection in int2kv_decode (wo_format). */
enum {
  INT2KV_WO_PLAIN = 0,          /* W_O, bf16 row-major; the merge un-rotates o by R_V          */
  INT2KV_WO_FOLDED = 1,         /* W-bar_O from int2kv_fold_wo, bf16 row-major                */
  INT2KV_WO_PREPARED = 2,       /* int2kv_prepare_wo output without R_V (merge un-rotates)    */
  INT2KV_WO_PREPARED_FOLDED = 3 /* int2kv_prepare_wo output with R_V folded in                */
};

/* Quantize already rotated rows and store them (the quantizer and packer alone; results are
 * bit-exact with the arithmetic above).
 *   k_rot, v_rot : fp32 [n, H_kv, 128]: (k - mu) R_K and v R_V
 *   slot_mapping : int32 [n]; a negative slot skips the token; slots must be distinct
 *   clip_k/clip_v: clip ratios c_K, c_V in (0, 1] (1 = no clipping) */
int int2kv_quantize_pack_rotated(const int2kv_cache* cache, const float* k_rot, const float* v_rot,
                                 const int32_t* slot_mapping, int num_tokens, float clip_k,
                                 float clip_v, hipStream_t stream);

/* Cache write (Sec. 4.1; Sec. 6): per token and KV head, k R_K - mu R_K and v R_V with fp32
 * accumulation, then INT2 group quantization and packing into the slot given by slot_mapping.
 *   k, v         : bf16 [n, H_kv, 128] (post-RoPE keys; values), 16-byte aligned
 *   slot_mapping : int32 [n]; negative = skip; distinct slots
 *   R_k, R_v     : fp32 [H_kv, 128, 128], 16-byte aligned;  mu_rk: fp32 [H_kv, 128] from
 *                  int2kv_prepare_mu_rot, 16-byte aligned
 * The rotation runs on the matrix cores with R split into three bf16 terms (exact products, fp32
 * accumulation starting from -mu R_K), so codes may differ from an exact-arithmetic rotation only
 * where x sits at a rounding boundary of the quantizer. */
int int2kv_quantize_append(const int2kv_cache* cache, const uint16_t* k, const uint16_t* v,
                           const int32_t* slot_mapping, int num_tokens, const float* R_k,
                           const float* R_v, const float* mu_rk, float clip_k, float clip_v,
                           hipStream_t stream);

/* Flags of int2kv_quantize_append_rope: rotate keys (values) by the normalized Sylvester Hadamard
 * matrix H_128 / sqrt(128), entry (i, c) = (-1)^popcount(i & c) / sqrt(128), instead of R_K (R_V),
 * the QuaRot base rotation (Sec. 2; Sec. 5 baselines). The library applies it without reading a
 * matrix: the +-1 entries are exact matrix-core operands (one pass instead of the three of a dense
 * fp32 R) and the fp32 sum is scaled by RN(1 / sqrt(128)). Readers (decode, fold, mu_rot) take the
 * dense fp32 matrix with entries +-RN(1 / sqrt(128)), which is the same rotation. */
#define INT2KV_HADAMARD_K 1
#define INT2KV_HADAMARD_V 2

/* Cache write fed with pre-RoPE keys (appendix, key-mean estimation and application: the mean is
 * subtracted from the post-RoPE key, then rotated and quantized), fused in one kernel:
 *     k_rope = bf16(RoPE(k, positions[i])),  stored: Q2((k_rope - mu) R_K) and Q2(v R_V),
 * RoPE with rotate-half pairs (i, i + 64), i < 64, from the caller's table:
 *     y_i = x_i cos_i - x_{i+64} sin_i,   y_{i+64} = x_{i+64} cos_i + x_i sin_i,
 * each evaluated exactly in fp64 (bf16 x fp32 products) and rounded once to bf16, nearest even.
 *   positions   : int32 [num_tokens], the tokens' positions; NULL = keys are already post-RoPE (the
 *                 write then equals int2kv_quantize_append, or its Hadamard form with flags)
 *   cos_sin     : fp32 [max_pos, 128], row p = (cos theta_{p,0..63}, sin theta_{p,0..63})
 *   flags       : INT2KV_HADAMARD_K / INT2KV_HADAMARD_V (the matching R may then be NULL)
 *   k_rope_out  : optional bf16 [num_tokens, H_kv, 128]: the post-RoPE keys (for the BF16 window)
 * A token whose position lies outside [0, max_pos) is skipped: no cache write and no k_rope_out row.
 * Other arguments as int2kv_quantize_append (mu_rk = mu R_K, with the dense Hadamard under
 * INT2KV_HADAMARD_K). */
int int2kv_quantize_append_rope(const int2kv_cache* cache, const uint16_t* k, const uint16_t* v,
                                const int32_t* slot_mapping, const int32_t* positions, int num_tokens,
                                const float* cos_sin, int max_pos, const float* R_k, const float* R_v,
                                const float* mu_rk, float clip_k, float clip_v, int flags, uint16_t* k_rope_out,
                                hipStream_t stream);

/* int2kv_quantize_append that also reports each token's reconstruction error, for the diagnostics of
 * Sec. 3.2 (E_rec, eq:raw_reconstruction_objective): err[(i * H_kv + h) * 2 + 0] = ||x - x^||^2 of
 * the key and [... + 1] of the value of token i, KV head h, where x is the library's fp32 rotated
 * (and, for keys, centered) row and x^ its dequantized INT2 row; since R_K, R_V are orthogonal this
 * is ||k - k~||^2 (k~ = k^ R_K^T + mu) and ||v - v~||^2 in the model's basis. err: fp32
 * [num_tokens, H_kv, 2], written for every token (also for skipped slots). Cache bytes are those of
 * int2kv_quantize_append. */
int int2kv_quantize_append_error(const int2kv_cache* cache, const uint16_t* k, const uint16_t* v,
                                 const int32_t* slot_mapping, int num_tokens, const float* R_k,
                                 const float* R_v, const float* mu_rk, float clip_k, float clip_v,
                                 float* err, hipStream_t stream);

/* Workspace bytes int2kv_decode needs for these sizes (d_model = 0 when W_O is not applied). */
size_t int2kv_decode_workspace_bytes(int batch, int num_q_heads, int num_kv_heads, int max_ctx,
                                     int d_model);

/* Decode attention over the INT2 cache for one new query per sequence.
 *   q            : bf16 [B, H_q, 128] (post-RoPE), 16-byte aligned
 *   block_table  : int32 [B, max_blocks_per_seq]; entry i of sequence b is the physical
 *                  block of tokens 16i .. 16i+15
 *   ctx_lens     : int32 [B] cached tokens to attend (the current token is appended first);
 *                  lengths are clamped to [0, min(max_ctx, 16*max_blocks_per_seq)], and blocks
 *                  outside [0, num_blocks) are skipped
 *   max_ctx      : host-side upper bound of ctx_lens (sizes the split-context grid)
 *   R_k, R_v     : fp32 [H_kv, 128, 128], 16-byte aligned (R_v may be NULL with a folded W_o)
 *   W_o          : output-projection weights in the format wo_format names, 16-byte aligned, or
 *                  NULL (no output projection). Row-major bf16 weights are applied on the matrix
 *                  cores with o split into two bf16 terms (fp32-like precision); prepared fp16
 *                  weights with o rounded once to fp16 (relative error <= 2^-11 per element). The
 *                  K range is split in fixed slices summed in a fixed order (deterministic)
 *   wo_format    : INT2KV_WO_PLAIN, _FOLDED, _PREPARED or _PREPARED_FOLDED (with a folded format
 *                  R_v is not applied); ignored when W_o is NULL
 *   out          : fp32 [B, H_q, 128] if W_o is NULL, else fp32 [B, d_model]
 *   workspace    : device scratch of at least int2kv_decode_workspace_bytes(...) bytes
 * The context is split into fixed-size chunks scanned in parallel (online softmax per chunk),
 * then merged with a log-sum-exp reduction; sequences with ctx_len 0 produce zeros. */
int int2kv_decode(const int2kv_cache* cache, const uint16_t* q, int batch, int num_q_heads,
                  const int32_t* block_table, int max_blocks_per_seq, const int32_t* ctx_lens,
                  int max_ctx, const float* R_k, const float* R_v, const uint16_t* W_o, int d_model,
                  int wo_format, float* out, void* workspace, size_t workspace_bytes,
                  hipStream_t stream);

/* One decode step of a serving loop: the cache write of the current tokens
 * (int2kv_quantize_append with k, v, slot_mapping, num_tokens, R_k, R_v, mu_rk, clip_k, clip_v)
 * followed by int2kv_decode with the remaining arguments; the results are bit-identical to those
 * two calls made in that order. With the matrix-core decode and at most 256 tokens, the cache
 * write runs as extra work-groups of the decode's first launch, beside the query preparation
 * (which does not read the cache), instead of as a launch of its own. R_v is required when
 * num_tokens > 0 (the cache write uses it); num_tokens = 0 makes this int2kv_decode. Errors as
 * for the two calls; nothing is launched on an argument error. */
int int2kv_append_decode(const int2kv_cache* cache, const uint16_t* k, const uint16_t* v,
                         const int32_t* slot_mapping, int num_tokens, const float* mu_rk, float clip_k,
                         float clip_v, const uint16_t* q, int batch, int num_q_heads,
                         const int32_t* block_table, int max_blocks_per_seq, const int32_t* ctx_lens,
                         int max_ctx, const float* R_k, const float* R_v, const uint16_t* W_o,
                         int d_model, int wo_format, float* out, void* workspace,
                         size_t workspace_bytes, hipStream_t stream);

/* Bytes of the static scratch behind int2kv_append_decode_noalloc (64 MiB per GPU). */
#define INT2KV_NOALLOC_SCRATCH_BYTES (64u << 20)

/* int2kv_append_decode without a workspace argument, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that forbid allocation).
 * The decode's workspace is a static device array of INT2KV_NOALLOC_SCRATCH_BYTES inside the
 * library, one copy per GPU, held until the process ends; its device address is looked up once per
 * device on the first call made there (hipGetSymbolAddress with that device current). The call
 * allocates nothing and calls no allocating routine. Results, arguments and errors as
 * int2kv_append_decode; in addition a call whose workspace (int2kv_decode_workspace_bytes of its
 * sizes) exceeds the scratch returns INT2KV_EWORKSPACE without launching. Every call on a GPU shares
 * that GPU's scratch and leaves its contents behind (nothing in it needs to start at zero): calls
 * that overlap on one GPU (concurrent streams, or threads) race and must be serialized by the
 * caller. */
int int2kv_append_decode_noalloc(const int2kv_cache* cache, const uint16_t* k, const uint16_t* v,
                                 const int32_t* slot_mapping, int num_tokens, const float* mu_rk, float clip_k,
                                 float clip_v, const uint16_t* q, int batch, int num_q_heads,
                                 const int32_t* block_table, int max_blocks_per_seq, const int32_t* ctx_lens,
                                 int max_ctx, const float* R_k, const float* R_v, const uint16_t* W_o, int d_model,
                                 int wo_format, float* out, hipStream_t stream);

/* BF16 sink and recent windows (Sec. 4.1; Sec. 5 implementation details: the paper keeps the
 * first 64 and the last 256 tokens of a sequence out of INT2). Window tokens keep the key
 * centering and are held in BF16; their values are held unchanged. The window store is a caller
 * buffer of rows, each row one token for every KV head: win[(row * H_kv + h) * 128 + c], bf16,
 * 16-byte aligned; row b * win_cap + t is token t of sequence b in int2kv_decode_window.
 *
 * int2kv_window_write stores num_tokens tokens: win_k[row] = bf16_rne(fp32(k - mu)) (the key
 * mean mu in the model's basis, fp32 [H_kv, 128]), win_v[row] = v (bit copy).
 *   k, v     : bf16 [num_tokens, H_kv, 128]
 *   rows     : int32 [num_tokens]; a negative row, or one >= num_rows, skips the token; rows must
 *              be distinct
 * num_tokens = 0 launches nothing. Returns INT2KV_EINVAL on NULL or misaligned pointers. */
int int2kv_window_write(const uint16_t* k, const uint16_t* v, const int32_t* rows, int num_tokens,
                        int num_kv_heads, const float* mu, uint16_t* win_k, uint16_t* win_v,
                        int num_rows, hipStream_t stream);

/* int2kv_decode over the INT2 tokens (block_table, ctx_lens) together with each sequence's window
 * tokens (win_lens[b], clamped to [0, win_cap], rows b * win_cap .. of win_k / win_v): one softmax
 * over both sets (eq:int2_attention, with the window tokens' keys and values as stored). The order
 * of tokens does not matter, so the window may be a ring. Other arguments, results, workspace and
 * errors as int2kv_decode; in addition R_v is required (the window's output joins the INT2 part in
 * the R_V basis), win_cap must be in [1, 512], and win_k, win_v must be 16-byte aligned. */
int int2kv_decode_window(const int2kv_cache* cache, const uint16_t* q, int batch, int num_q_heads,
                         const int32_t* block_table, int max_blocks_per_seq, const int32_t* ctx_lens,
                         int max_ctx, const float* R_k, const float* R_v, const uint16_t* W_o,
                         int d_model, int wo_format, const uint16_t* win_k, const uint16_t* win_v,
                         const int32_t* win_lens, int win_cap, float* out, void* workspace,
                         size_t workspace_bytes, hipStream_t stream);

/* Output-error diagnostics of the INT2 cache (Sec. 3.2; appendix output-space error metrics):
 * for every sequence b and query head j, with p the attention of q_j over the full-precision keys
 * k, p~ over the cache's effective INT2 keys k~ = k^ R_K^T + mu, V the full-precision values and V~
 * the effective INT2 values v^ R_V^T,
 *     dy_K = ((p~ - p)^T V) W_{O,j}^T,   dy_V = (p~^T (V~ - V)) W_{O,j}^T,
 * so that y~_j - y_j = dy_K + dy_V exactly (the key- and value-induced output errors), and
 *     stats[(b * H_q + j) * 4 + {0, 1, 2, 3}] = ||dy_K + dy_V||^2 (E_out), ||dy_K||^2, ||dy_V||^2,
 *                                              <dy_K, dy_V>.
 *   k_rows, v_rows : bf16 full-precision keys (raw, not centered) and values, row b * row_cap + t
 *                    holding token t of sequence b for every KV head ([rows, H_kv, 128]), the
 *                    tokens the cache holds at block_table / ctx_lens (lengths are also clamped to
 *                    row_cap)
 *   W_o            : bf16 [d_model, H_q * 128] row-major (required)
 *   dy             : fp32 [B, H_q, 2, d_model] (dy_K, dy_V) or NULL
 *   workspace      : int2kv_output_error_workspace_bytes(...) bytes, 256-byte aligned
 * Other arguments as int2kv_decode; up to 16 query heads per KV head. Scores and sums run in fp32
 * (INT2 scores with the rotated query, as the vector-ALU decode). */
size_t int2kv_output_error_workspace_bytes(int batch, int num_q_heads, int num_kv_heads, int max_ctx,
                                           int d_model);
int int2kv_output_error(const int2kv_cache* cache, const uint16_t* q, int batch, int num_q_heads,
                        const int32_t* block_table, int max_blocks_per_seq, const int32_t* ctx_lens,
                        int max_ctx, const float* R_k, const float* R_v, const uint16_t* k_rows,
                        const uint16_t* v_rows, int row_cap, const uint16_t* W_o, int d_model,
                        float* stats, float* dy, void* workspace, size_t workspace_bytes,
                        hipStream_t stream);

/* ---- Around the decode step: a chunk's rotary positions, its attention, and rows read back.
 *
 * Rotary positions with several axes (time, height and width of image and video tokens) of a chunk's
 * queries and keys, in one launch. Rotate-half pairs (i, i + 64), i < 64; pair i turns by its axis'
 * position of the token:
 *     y_i = x_i cos - x_{i+64} sin,   y_{i+64} = x_{i+64} cos + x_i sin,
 *     (cos, sin) = cos_sin[positions[pair_axis[i]][token]][i], [... 64 + i],
 * each evaluated exactly in fp64 and rounded once to bf16, as in int2kv_quantize_append_rope (with
 * one axis the keys equal its k_rope_out). The turned keys go to int2kv_quantize_append and
 * int2kv_chunk_attention, the turned queries to the latter or to int2kv_decode.
 *   q, k         : bf16, head j of token t at t * stride + 128 j (elements); 16-byte aligned; either
 *                  may be NULL with 0 heads. The strides let them be views of a layer's fused
 *                  projection; multiples of 8, at least 128 * heads
 *   positions    : int32 [num_axes, num_tokens]; a token with a position outside [0, max_pos) on any
 *                  axis is skipped: its output rows are left as they were
 *   num_axes     : 1 .. 8;  pair_axis: HOST uint8 [64], the axis of each pair
 *   cos_sin      : fp32 [max_pos, 128], as in int2kv_quantize_append_rope; 16-byte aligned
 *   q_out, k_out : bf16 rows as q, k with strides of their own; may be q, k themselves (same stride),
 *                  otherwise no output row may overlap an input's or the other output's rows
 *   num_tokens   : at most 2^27 - 8 */
int int2kv_rope_axes(const uint16_t* q, int num_q_heads, int64_t q_stride, const uint16_t* k, int num_kv_heads,
                     int64_t k_stride, const int32_t* positions, int num_axes, const uint8_t* pair_axis,
                     int num_tokens, const float* cos_sin, int max_pos, uint16_t* q_out, int64_t q_out_stride,
                     uint16_t* k_out, int64_t k_out_stride, hipStream_t stream);

/* Row formats of int2kv_read_rows. */
enum {
  INT2KV_ROWS_BF16 = 0,
  INT2KV_ROWS_F32 = 1
};

/* Rows read back from the cache: the keys and values that the decode attends to, for another cache
 * (other rotations, group size or paging), a full-precision consumer, or diagnostics.
 *     k_out[i] = k^ R_K^T + mu,   v_out[i] = v^ R_V^T,   k^, v^ = code * s + z of slot slot_mapping[i];
 * without R_k (R_v) the row as stored, k^ (v^), in the rotated basis.
 *   slot_mapping : int32 [num_tokens], in any order, repeats allowed; a slot outside the cache (also a
 *                  negative one) leaves its output rows as they were; num_tokens * H_kv at most 2^28 - 16
 *   R_k, R_v     : fp32 [H_kv, 128, 128], 16-byte aligned, or NULL;  mu: fp32 [H_kv, 128] or NULL (keys
 *                  stay centered); mu needs R_k
 *   row_format   : INT2KV_ROWS_BF16 or INT2KV_ROWS_F32
 *   k_out, v_out : bf16 or fp32 [num_tokens, H_kv, 128], 16-byte aligned; one of them may be NULL; they
 *                  may not overlap
 * Stored rows are code * s + z in fp32 (exact unless s and z lie more than 2^11 apart), rounded once to
 * the format. The un-rotation runs on the matrix cores in
 * fp16 terms with fp32 sums: one term each for bf16 rows (about 3e-4 of the row's root mean square,
 * under the rounding of bf16), two for fp32 rows (below 1e-6). Dequantized values and rotations have
 * to lie within fp16's range (|x| <= 65504). */
int int2kv_read_rows(const int2kv_cache* cache, const int32_t* slot_mapping, int num_tokens, const float* R_k,
                     const float* R_v, const float* mu, int row_format, void* k_out, void* v_out,
                     hipStream_t stream);

/* Attention of several new tokens per sequence over the INT2 cache: a prompt or a chunk of one, a
 * turn after a cached history, drafted tokens. Token i (0 .. n_b - 1) of sequence b is row
 * q_starts[b] + i of q and out. Two forms:
 *   k_new given: the chunk's keys and values are the caller's bf16 rows, the cache holds what came
 *     before: token i sees the ctx_lens[b] cached tokens and the new tokens 0 .. i of its sequence,
 *       a_s = (q R_K) k^_s^T / sqrt(d),  a_t = q (k_t - mu)^T / sqrt(d),
 *       o = (sum_s p_s v^_s) R_V^T + sum_t p_t v_t,   one softmax over both;
 *   k_new NULL: the cache holds the new tokens too (appended first, as for int2kv_decode), ctx_lens[b]
 *     counts them: token i sees the cached tokens 0 .. ctx_lens[b] - n_b + i (for n_b = 1 this is
 *     int2kv_decode without W_O, up to rounding). n_b and ctx_lens[b] count here as they are given,
 *     also where max_q cuts the sequence or max_ctx or the table its context: a token's place does not
 *     move, it sees those of its tokens that are left.
 * A token that sees nothing gets zeros.
 *   q            : bf16, head j of token t at t * q_stride + 128 j (elements); post-RoPE; 16-byte
 *                  aligned; q_stride a multiple of 8, at least 128 * H_q
 *   q_starts     : int32 [batch + 1], ascending offsets into 0 .. total_q; rows of q and out outside
 *                  every sequence (padding behind the last one) are not written; a sequence may be empty
 *   total_q, max_q : rows of q and out; host-side upper bound of n_b (larger sequences are cut to it)
 *   block_table, max_blocks_per_seq, ctx_lens, max_ctx : as int2kv_decode (same clamping, blocks
 *                  outside the cache are skipped)
 *   R_k, R_v     : fp32 [H_kv, 128, 128], 16-byte aligned
 *   k_new, v_new : bf16 rows as q with H_kv heads and strides of their own (raw post-RoPE keys, not
 *                  centered; values), with mu: fp32 [H_kv, 128]; or NULL, NULL, NULL
 *   out          : bf16 [total_q, H_q, 128], 16-byte aligned, model basis; must not overlap q, k_new, v_new
 *   workspace    : int2kv_chunk_attention_workspace_bytes(...) bytes, 256-byte aligned; enough for every
 *                  call within the same bounds; nothing in it needs to be kept or cleared between calls,
 *                  calls that overlap need one each
 * Products run on the matrix cores with fp32 sums: queries and rotations, rotated queries, dequantized
 * rows, the probabilities over the INT2 tokens and the sums that R_V turns (each row scaled by a power
 * of two of its own) in fp16, the chunk's own rows and the probabilities over them in bf16, each rounded
 * once; softmax statistics in fp32. Queries (where the cache holds anything), rotated queries times
 * log2(e) / sqrt(128), rotations and dequantized values have to lie within fp16's range (|x| <= 65504).
 * A non-finite key or value reaches only the tokens that see it. Deterministic; no atomics on results. */
size_t int2kv_chunk_attention_workspace_bytes(int batch, int num_q_heads, int num_kv_heads, int total_q, int max_q,
                                              int max_ctx);
int int2kv_chunk_attention(const int2kv_cache* cache, const uint16_t* q, int64_t q_stride, const int32_t* q_starts,
                           int batch, int total_q, int max_q, int num_q_heads, const int32_t* block_table,
                           int max_blocks_per_seq, const int32_t* ctx_lens, int max_ctx, const float* R_k,
                           const float* R_v, const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new,
                           int64_t v_stride, const float* mu, uint16_t* out, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* Tokens of a drafted tree at most. */
#define INT2KV_MAX_TREE 256

/* Attention of the tokens of a drafted tree over the INT2 cache: a target model scoring every drafted
 * continuation in one pass, or a draft model growing the tree level by level. The tree's keys and
 * values are the caller's bf16 rows, tree_starts[b] .. tree_starts[b + 1] of k_tree and v_tree for
 * sequence b, T_b of them; the accepted ones are appended (int2kv_quantize_append, slot -1 for the
 * others) once they are known. parents[t] is the tree index (0 .. T_b - 1) of the token that token t
 * follows, a smaller one, or -1 where t follows the last cached token. The queries, n_b rows from
 * q_starts[b] of q, are the last n_b tokens of the tree: query i is token t = T_b - n_b + i and sees
 * the ctx_lens[b] cached tokens and its path t, parents[t], .. :
 *     a_s = (q R_K) k^_s^T / sqrt(d),  a_t = q (k_t - mu)^T / sqrt(d),
 *     o = (sum_s p_s v^_s) R_V^T + sum_t p_t v_t,   one softmax over both.
 * A token whose walk to -1 meets a parent outside [-1, own index) is absent, as is one with t < 0 or
 * t >= max_tree: it sees nothing, not even the cache, and gets zeros (places of a tree of a fixed
 * shape that stay empty take the parent -2). Rows of k_tree and v_tree on no query's path may hold
 * anything.
 *   q, q_starts, total_q, max_q, block_table, max_blocks_per_seq, ctx_lens, max_ctx, R_k, R_v, out :
 *                  as int2kv_chunk_attention
 *   tree_starts  : int32 [batch + 1], ascending offsets into 0 .. total_tree; the same as q_starts where
 *                  every token of the trees is a query
 *   total_tree, max_tree : rows of k_tree, v_tree and parents; host-side upper bound of T_b, at most
 *                  INT2KV_MAX_TREE
 *   k_tree, v_tree, mu : as k_new, v_new and mu of int2kv_chunk_attention (NULL, as parents, only where
 *                  total_tree is 0)
 *   workspace    : int2kv_tree_attention_workspace_bytes(...) bytes, 256-byte aligned; enough for every
 *                  call within the same bounds, nothing kept between calls, calls that overlap need one each
 * Numerics and ranges as int2kv_chunk_attention. Deterministic; no atomics on results. */
size_t int2kv_tree_attention_workspace_bytes(int batch, int num_q_heads, int num_kv_heads, int total_q, int max_q,
                                             int max_tree, int max_ctx);
int int2kv_tree_attention(const int2kv_cache* cache, const uint16_t* q, int64_t q_stride, const int32_t* q_starts,
                          int batch, int total_q, int max_q, int num_q_heads, const int32_t* tree_starts,
                          int total_tree, int max_tree, const int32_t* parents, const uint16_t* k_tree,
                          int64_t k_stride, const uint16_t* v_tree, int64_t v_stride, const float* mu,
                          const int32_t* block_table, int max_blocks_per_seq, const int32_t* ctx_lens, int max_ctx,
                          const float* R_k, const float* R_v, uint16_t* out, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);

/* Attention weight that every cached token receives, added to a running sum: what an eviction goes by.
 * The cache holds the new tokens too (appended first, as for int2kv_decode): query token i of n_b sees
 * the cached tokens 0 .. ctx_lens[b] - n_b + i, as the second form of int2kv_chunk_attention. For KV
 * head h and token s < ctx_lens[b]
 *     weights_out[b, h, s] = decay weights_in[b, h, s] + sum_i sum_{j in group h} p_ij(s),
 *     p_ij = softmax over what token i sees of (q_ij R_K) k^_s^T / sqrt(d).
 * One token a sequence: a decode step; the last tokens of a prompt: their vote on the rest; all of them.
 *   q .. max_ctx, R_k : as int2kv_chunk_attention (with max_q 0 the sums only decay; q, R_k may be NULL)
 *   weights_in   : fp32, KV head h of sequence b at (b H_kv + h) weights_stride, or NULL: zeros. The
 *                  entries of tokens that are new count too: zero, unless the caller wants otherwise
 *   decay        : factor of weights_in, finite
 *   weights_out  : fp32 as weights_in, which it may be, without otherwise overlapping it. Tokens from
 *                  min(ctx_lens[b], max_ctx) on are left as they were; tokens in blocks outside the
 *                  cache, or behind the table's end, receive nothing: their sums only decay
 *   weights_stride : at least max_ctx
 *   workspace    : int2kv_token_weights_workspace_bytes(...) bytes, 256-byte aligned; enough for every
 *                  call within the same bounds, nothing kept between calls, calls that overlap need one each.
 *                  Up to 8 rows (n_b H_q / H_kv, by max_q) of a KV head, which read the keys once: mostly
 *                  their scores, 4 bytes a row and token. More, which read the keys twice (64 sequences of
 *                  8,000 tokens, 4 KV heads: 8 rows 71 us, 12 or 16 rows 175): 17 KiB of operands for every
 *                  32 rows of a KV head and 8 bytes of statistics for each row and 256 tokens of max_ctx (a
 *                  prompt of 16,384 tokens, 32 + 8 heads: 0.6 GB); where that passes 1 GiB the rows are
 *                  taken in parts, one behind the other, so that it stays at 1 GiB or, if that is more,
 *                  what 1,024 rows of every sequence and KV head take
 * fp32 throughout: products run on the matrix cores in terms that keep fp32's precision, statistics and
 * sums in fp32 (a weight is off by about 1e-6 of itself and the scores' size times 1e-7). Queries and the
 * scales and zeros of the cached tokens have to be finite. Deterministic; no atomics on results. */
size_t int2kv_token_weights_workspace_bytes(int batch, int num_q_heads, int num_kv_heads, int total_q, int max_q,
                                            int max_ctx);
int int2kv_token_weights(const int2kv_cache* cache, const uint16_t* q, int64_t q_stride, const int32_t* q_starts,
                         int batch, int total_q, int max_q, int num_q_heads, const int32_t* block_table,
                         int max_blocks_per_seq, const int32_t* ctx_lens, int max_ctx, const float* R_k,
                         const float* weights_in, float decay, float* weights_out, int64_t weights_stride,
                         void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The tokens of every sequence and KV head that stay in a cache of `budget` tokens: the first `sink`
 * and the last `recent` ones, and of the others those of the largest weights (ties: the lower index;
 * NaN below every number), in ascending order. A sequence of at most `budget` tokens keeps them all.
 *   weights      : fp32, KV head h of sequence b at (b num_kv_heads + h) weights_stride, tokens
 *                  s < min(ctx_lens[b], max_ctx) (int2kv_token_weights)
 *   sink + recent at most budget
 *   kept         : int32, list of KV head h of sequence b at (b num_kv_heads + h) kept_stride;
 *                  kept_lens[b] = min(ctx_lens[b], max_ctx, budget) entries are written
 *   kept_stride  : at least min(budget, max_ctx)
 *   kept_lens    : int32 [batch]; neither it nor kept may overlap weights, ctx_lens or the other */
int int2kv_select_tokens(const float* weights, int64_t weights_stride, int batch, int num_kv_heads,
                         const int32_t* ctx_lens, int max_ctx, int budget, int sink, int recent, int32_t* kept,
                         int64_t kept_stride, int32_t* kept_lens, hipStream_t stream);

/* The kept tokens' rows, byte for byte, to the front of a sequence: token j < kept_lens[b] of KV head h
 * becomes the old token kept[b, h, j], whose place in block_table's blocks is written to token j's in
 * out_table's. Keys are stored after their rotary positions, so the readers see the kept tokens
 * as they were; the sequence's length is then kept_lens[b]. Lists come from int2kv_select_tokens, or
 * are the caller's, in any order, with repeats.
 *   block_table  : int32 [batch, max_blocks_per_seq]
 *   kept, kept_stride : as int2kv_select_tokens; max_kept: host-side upper bound of kept_lens (larger
 *                  ones are cut to it), at most kept_stride
 *   out_table    : int32 [batch, out_max_blocks], at least the pages of max_kept tokens: blocks that no
 *                  sequence of the call reads and no other writes. NULL (or block_table): in place, through the
 *                  workspace; no block may then belong to two sequences
 *   weights      : fp32 (as int2kv_token_weights) or NULL; moved along to out_weights, which in place may
 *                  be weights itself
 *   workspace    : in place int2kv_move_tokens_workspace_bytes(...) bytes, 16-byte aligned; else NULL
 * A row whose old token lies outside the table or in a block outside the cache is left as it was, as
 * are rows behind the last kept one, pages whose new block lies outside the cache, and weights beyond
 * a stride. In place that holds for weights behind the last kept one too: clear them before tokens are
 * appended there and int2kv_token_weights adds to their sums. */
size_t int2kv_move_tokens_workspace_bytes(int batch, int num_kv_heads, int group_size, int max_kept);
int int2kv_move_tokens(const int2kv_cache* cache, const int32_t* block_table, int max_blocks_per_seq,
                       const int32_t* kept, int64_t kept_stride, const int32_t* kept_lens, int batch,
                       int max_kept, const int32_t* out_table, int out_max_blocks, const float* weights,
                       int64_t weights_stride, float* out_weights, int64_t out_weights_stride, void* workspace,
                       size_t workspace_bytes, hipStream_t stream);

/* ---- OptR offline calibration (Sec. 4.2 - 4.5; Algorithm 1 of the appendix), fp64 on the GPU.
 * For every KV head h the corrected rotations R = R^0 exp(A - A^T) (eq:OptR_skew) are fitted to
 * calibration traces: first A_K on the key objective (eq:OptR_key_loss)
 *     L_K = mean over rows (t, j) of KL(p_t || p^K_t) + lambda_K ||((p^K_t - p_t)^T V) W_{O,j}^T||^2 / d_model,
 * then A_V on the value objective (eq:OptR_value_loss) under the selected key rotation's
 * probabilities p^K-hat:
 *     L_V = mean over rows of ||(p^K-hat_t^T (V~ - V)) W_{O,j}^T||^2 / d_model.
 * Rows: query heads j of the KV head's group at the final n_last positions t of each sequence,
 * attending causally (s <= t). Effective keys k~ = Q2((k - mu) R_K) R_K^T and values
 * v~ = Q2(v R_V) R_V^T use the cache's own quantizer on the fp32 rounding of the rotated rows
 * (group_size, clip ratios); tokens s < sink and s > t - recent stay in full precision (BF16
 * windows). Gradients pass the quantizer by the straight-through estimator of eq:OptR_ste: an
 * element's gradient passes when it lies inside its group's clipped range [c mn, c mx]; scale and
 * zero are held fixed. The optimizer is Adam (betas 0.9 / 0.999, eps 1e-8, learning rate lr); the
 * iterate with the lowest held-out objective among A = 0 and every eval_every-th step is kept.
 * All arithmetic is fp64; inputs stay as given (bf16 traces, fp32 R^0 and mu). Up to 16 query heads
 * per KV head. */
typedef struct int2kv_optr_traces {
  const uint16_t* k;          /* device bf16 [T, H_kv, 128]: keys (post-RoPE, raw); 16-byte aligned */
  const uint16_t* v;          /* device bf16 [T, H_kv, 128]: values; 16-byte aligned */
  const uint16_t* q;          /* device bf16 [T, H_q, 128]: queries (post-RoPE) */
  const int32_t* seq_starts;  /* HOST int32 [num_seqs + 1]: token offsets, seq_starts[0] = 0,
                                 sequences of 0 .. 4096 tokens */
  int num_seqs;
} int2kv_optr_traces;

typedef struct int2kv_optr_config {
  int num_kv_heads, num_q_heads, d_model, group_size; /* group_size 32 or 128 */
  float clip_k, clip_v;                               /* the paper's setting: 0.96, 0.92 */
  double lambda_k;                                    /* 1.0 */
  int n_last, sink, recent;                           /* 64, 64, 256 */
  int steps, eval_every;                              /* 80, 20 */
  double lr;                                          /* 0.02 */
} int2kv_optr_config;

/* Workspace bytes of the calls below (heldout may be NULL for the loss calls); 0 on bad arguments. */
size_t int2kv_optr_workspace_bytes(const int2kv_optr_config* cfg, const int2kv_optr_traces* calib,
                                   const int2kv_optr_traces* heldout);
/* Per-channel key mean per KV head (appendix, key-mean estimation): mu[h][c] = fp32(fp64 mean over
 * the num_tokens keys k [T, H_kv, 128] bf16). */
int int2kv_optr_key_mean(const uint16_t* k, int num_tokens, int num_kv_heads, float* mu, hipStream_t stream);
/* L_K of every KV head at generators A (device fp64 [H_kv, 128, 128]) into loss (device fp64 [H_kv]),
 * and dL_K/dA into grad (device fp64 [H_kv, 128, 128]) unless grad is NULL. R0_k: fp32 [H_kv, 128, 128];
 * mu: fp32 [H_kv, 128]; W_o: bf16 [d_model, H_q * 128]. */
int int2kv_optr_key_loss(const int2kv_optr_config* cfg, const int2kv_optr_traces* traces, const float* R0_k,
                         const float* mu, const uint16_t* W_o, const double* A, double* loss, double* grad,
                         void* workspace, size_t workspace_bytes, hipStream_t stream);
/* L_V at generators A_v under the key probabilities of generators A_k, and dL_V/dA_v. */
int int2kv_optr_value_loss(const int2kv_optr_config* cfg, const int2kv_optr_traces* traces, const float* R0_k,
                           const double* A_k, const float* mu, const float* R0_v, const uint16_t* W_o,
                           const double* A_v, double* loss, double* grad, void* workspace, size_t workspace_bytes,
                           hipStream_t stream);
/* Algorithm 1 for every KV head at once: R_k, R_v (device fp32 [H_kv, 128, 128]) receive the
 * selected R^0 exp(A - A^T); A_k, A_v (device fp64, may be NULL) the selected generators; history
 * (device fp64, may be NULL) [2][H_kv][steps + 1 + steps / eval_every]: for keys, then values, the
 * training objective before each step followed by the held-out objectives at A = 0 and every
 * eval_every-th step. The host tables of both trace sets are uploaded at the start (the call waits
 * for that copy); the rest runs asynchronously on stream. */
int int2kv_optr_calibrate(const int2kv_optr_config* cfg, const int2kv_optr_traces* calib,
                          const int2kv_optr_traces* heldout, const float* R0_k, const float* R0_v, const float* mu,
                          const uint16_t* W_o, float* R_k, float* R_v, double* A_k, double* A_v, double* history,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Measurement hook: when set (non-NULL), the calls this thread issues attach `before_scan` and
 * `after_scan` to the dispatch of their dominant kernel (hipExtLaunchKernel): the split-context scan
 * of int2kv_decode, int2kv_append_decode and int2kv_decode_window, the cache-write kernel of
 * int2kv_quantize_append(_error), the diagnostics scan of int2kv_output_error. They then mark that kernel's own start and end, and a caller can time it
 * alone with hipEventElapsedTime, without extra packets between the kernels. Pass NULLs to disable.
 * The setting is per calling thread. The events are owned by the caller and must outlive the calls
 * that record them. */
int int2kv_set_decode_events(hipEvent_t before_scan, hipEvent_t after_scan);

/* Tuning knobs for measurement sweeps: context chunk in tokens (multiple of 64, 0 = automatic)
 * and decode kernel variant (0 = automatic, 1 = vector ALU, 2 = matrix core; the matrix-core scan
 * serves at most 8 query heads per KV head, wider groups always use the vector-ALU scan). The
 * setting applies to the calls of the calling thread only (thread-local), including
 * int2kv_decode_workspace_bytes: size a workspace on the thread that decodes with it. Returns
 * INT2KV_EINVAL for out-of-range values. */
int int2kv_set_decode_tuning(int chunk_tokens, int variant);

#ifdef __cplusplus
}
#endif

#endif /* INT2KV_H */
