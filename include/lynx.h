/*
 * lynx.h -- C interface of the B200 (sm_100a) library for the data-parallel hot path of
 * Lynx's progressive speculative quantisation of the KV cache.
 *
 * The path (paper sections in brackets):
 *   1. split-quantise: BF16 K or V rows -> 8-bit linear per-group codes (Section 2.3,
 *      "Standard & Grouped Quantization": Q(X) = round(X/S + Z), S from the group's min-max
 *      range) split into an Anchor plane (top 4 bits) and a Residual plane (bottom 4 bits),
 *      two 4-bit values per byte, each stream contiguous, the scalars travelling with the
 *      Anchor stream (Section 4.1 stage 4; Section "Implementation", Compression Kernel).
 *   2. anchor attention: decode attention softmax(Q K^T / sqrt(d)) V (Section 2) evaluated on
 *      the Anchor plane alone, which is what the decode instance has when it starts drafting
 *      (Section 4.2, Anchor Phase).
 *   3. merge-verify attention: Anchor and Residual recombined into the full 8-bit state
 *      Q_full (Section 4.2, Residual Phase), the k drafted positions scored in one pass and the
 *      longest agreeing prefix reported (Section 4.3).
 *   4. recombine: the stand-alone Residual-phase refinement to full codes / BF16 pages.
 *
 * Group = one token's head vector of 128 elements (a "row").  Per row:
 *   mn = min, mx = max, range = fl(mx - mn), scale = fl(range/255), inv = fl(255/range),
 *   zero = mn (with -0 stored as +0); range < 2^-100 -> scale = inv = 0 (constant row);
 *   code = round-half-even of the exact product fl(x - mn) * inv, in [0, 255];
 *   anchor nibble a = code >> 4, residual nibble r = code & 15;
 *   byte j of a plane row = nibble of element 2j (low half) | nibble of element 2j+1 << 4.
 * Reconstruction: full state x^ = zero + scale * (16 a + r); Anchor-only state
 * x^ = zero + scale * (16 a + 8) (bucket mid-point).  Inputs must be finite.
 *
 * Memory layout of a quantised K (or V) cache of one layer, paged:
 *   anchor, residual : uint8 [num_blocks][num_kv_heads][block_tokens][64]
 *   meta             : float [num_blocks][num_kv_heads][block_tokens][2] = {scale, zero}
 * Token t of sequence b lives in row (t % block_tokens) of block
 * block_table[b][t / block_tokens].  A contiguous cache is the identity block table.
 * Several layers may be flattened into the batch dimension (each (layer, sequence) pair is an
 * independent problem with its own block-table row).
 *
 * Conventions for every call:
 *   - every pointer is a DEVICE pointer owned by the caller unless stated otherwise; the
 *     library never allocates, frees or synchronises (lynx_check is the one exception);
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream); calls
 *     only enqueue work and return;
 *   - arguments are validated on the host before any launch; an invalid call launches
 *     nothing and returns a status other than LYNX_OK;
 *   - device code never traps: block ids outside [0, num_blocks) are clamped and recorded in
 *     the workspace's status word, which lynx_check turns into LYNX_ERR_BAD_BLOCK_TABLE.
 */
#ifndef LYNX_H_
#define LYNX_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  LYNX_OK = 0,
  LYNX_ERR_NULL = 1,            /* a required pointer is NULL */
  LYNX_ERR_SHAPE = 2,           /* negative / zero / inconsistent size */
  LYNX_ERR_ALIGN = 3,           /* a pointer is not 16-byte aligned */
  LYNX_ERR_UNSUPPORTED = 4,     /* head_dim != 128, block_tokens % 16 != 0, too many columns */
  LYNX_ERR_WORKSPACE = 5,       /* workspace too small (see lynx_workspace_bytes) */
  LYNX_ERR_CUDA = 6,            /* a CUDA runtime call failed */
  LYNX_ERR_BAD_BLOCK_TABLE = 7, /* (lynx_check) a kernel saw a block id out of range */
  LYNX_ERR_TIMEOUT = 8,         /* (lynx_check) a bounded on-chip wait ran out */
  LYNX_ERR_RANGE = 9            /* (lynx_check) a value row outside the range a kernel can represent */
} lynx_status;

/* One of K or V of one layer (or of several flattened layers), quantised and paged. */
typedef struct {
  const uint8_t* anchor;   /* [num_blocks][Hkv][block_tokens][64] */
  const uint8_t* residual; /* same shape; ignored (may be NULL) by lynx_anchor_attention */
  const float* meta;       /* [num_blocks][Hkv][block_tokens][2] = {scale, zero} */
} lynx_plane;

typedef struct {
  int32_t num_q_heads;        /* Hq, a multiple of num_kv_heads; Hq/Hkv in 1..16 */
  int32_t num_kv_heads;       /* Hkv */
  int32_t head_dim;           /* must be 128 */
  int32_t block_tokens;       /* tokens per block, a multiple of 16 */
  int32_t num_blocks;         /* blocks in the pool the planes cover */
  int32_t max_blocks_per_seq; /* row length of block_table */
} lynx_shape;

/* Steps 1 (Section 2.3 quantiser; Section 4.1 stage 4 split; Compression Kernel packing).
 * src_bf16 : [n_rows][128] BF16, 16-byte aligned.  Row i of src produces row i of anchor
 *            ([n_rows][64] u8), residual ([n_rows][64] u8) and meta ([n_rows][2] float).
 * block_ids: NULL -> all rows 0..n_rows-1 are quantised.  Otherwise int32 [n_block_ids]:
 *            only rows block_ids[i]*rows_per_block .. +rows_per_block-1 are quantised (newly
 *            arrived blocks); ids outside [0, n_rows/rows_per_block) are skipped.  n_rows must
 *            then be a multiple of rows_per_block.
 * n_rows == 0 (or n_block_ids == 0) is a valid no-op. */
lynx_status lynx_split_quantize(const void* src_bf16, int64_t n_rows, const int32_t* block_ids,
                                int32_t n_block_ids, int32_t rows_per_block, uint8_t* anchor,
                                uint8_t* residual, float* meta, void* stream);

/* Step 4 (Section 4.2 Residual Phase refinement to Q_full).  For each of n_rows rows:
 * code = (a << 4) | r.  codes_u8 ([n_rows][128] u8) and dequant_bf16 ([n_rows][128] BF16 =
 * bf16_rne(fl(fma(code, scale, zero)))) are optional outputs; at least one must be given. */
lynx_status lynx_recombine(const uint8_t* anchor, const uint8_t* residual, const float* meta,
                           int64_t n_rows, uint8_t* codes_u8, void* dequant_bf16, void* stream);

/* Bytes of workspace the two attention calls need for `batch` sequences, `n_cols_q` query
 * positions (n_q or k) and sequences of at most max_blocks_per_seq * block_tokens tokens.
 * Returns 0 for an unsupported shape.  The workspace must be zero-filled once before its first
 * use (lynx_workspace_init, or cudaMemsetAsync of the whole buffer); each call leaves it ready
 * for the next, whatever the batch, heads and positions of either, as long as it is large enough
 * for both.  Calls sharing a workspace must be ordered on one stream.  It is not to be handed to
 * lynx_bf16_attention in between, whose scratch starts at its first byte.
 * A buffer smaller than this figure is rejected by the attention calls (LYNX_ERR_WORKSPACE): nothing
 * degrades silently.  It holds the status word, tickets, per-head deviations, log-sum-exps and the partial
 * results of split contexts. */
size_t lynx_workspace_bytes(const lynx_shape* shape, int32_t batch, int32_t n_cols_q);
lynx_status lynx_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

/* Step 2 (Section 2 attention equation on the Anchor-only state of Section 4.2).
 * q_bf16 : [batch][n_q][Hq][128] BF16; query head h reads KV head h / (Hq/Hkv).
 * Query j of sequence b attends tokens [0, seq_lens[b]) (causal == 0) or
 * [0, seq_lens[b] - n_q + j + 1) (causal != 0); a query that sees no token gets zeros.
 * softmax_scale 0 means 1/sqrt(128).  out : [batch][n_q][Hq][128] float.
 * n_q must be <= 64 (the cap on speculated positions of Section 5.1).  A kernel launch takes up to 32
 * query columns n_q * (Hq/Hkv); a call with more runs as slices of whole positions, each a pass of its own
 * over the planes, one after the other on the stream.  seq_lens[b] is clamped to the table's capacity.
 * Value rows of any finite scale are handled (the weights are fixed-point numbers relative to a
 * per-column reference exponent).  Queries enter as fixed-point numbers with 22 bits below the largest
 * |q| among the columns of a (sequence, KV head): whatever their magnitude, entries are exact to
 * 2^-22 of that largest one. */
lynx_status lynx_anchor_attention(const lynx_shape* shape, const void* q_bf16, int32_t batch,
                                  int32_t n_q, int32_t causal, lynx_plane K, lynx_plane V,
                                  const int32_t* block_table, const int32_t* seq_lens,
                                  float softmax_scale, float* out, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* Step 3 (Section 4.2 Residual Phase + Section 4.3 verification).  Same attention on the
 * recombined full codes for the k drafted positions in one pass over the context, then per
 * sequence   dev[b][j] = max over heads, dims of |out_full - draft| / (atol + rtol*|out_full|)
 * and first_reject[b] = smallest j with dev[b][j] > 1, or k if none (the longest agreeing
 * prefix; out_full at that position is the correction).
 * draft_out : [batch][k][Hq][128] float, the Anchor-state results being verified; may be NULL,
 * then dev / first_reject are not written (and may be NULL).  It needs the alignment of a float only (a view into a
 * larger buffer); 16-byte alignment is read faster.  out_full : same shape, float.
 * k must be <= 64.  Up to 16 columns k * (Hq/Hkv) are one launch of an integer kernel with exact sums;
 * 17..64 columns (up to 16 positions) are one launch of a kernel whose weights are two FP16 terms each
 * (22 bits), summed in FP32, or up to 32 columns on long contexts integers (steps of 2^-26 of the largest, rounded
 * without a bias), summed exactly; a longer window runs as slices of whole positions (a pass over the planes each).
 * Which of the two follows from the table's size (max_blocks_per_seq of more than 512 tokens, and 3072 per SM in all), so
 * that results may differ in their rounding between tables of different widths.  With several launches first_reject is
 * taken over the whole window from the deviations.
 * Value rows of any finite scale are handled with up to 32 columns.  With 33..64 columns per launch a value
 * row whose scale reaches 16 (a range of 4080 or more) is recorded in the status word and lynx_check
 * returns LYNX_ERR_RANGE: that is the range this width is specified and tested for. */
lynx_status lynx_merge_verify_attention(const lynx_shape* shape, const void* q_bf16,
                                        int32_t batch, int32_t k, int32_t causal, lynx_plane K,
                                        lynx_plane V, const int32_t* block_table,
                                        const int32_t* seq_lens, float softmax_scale,
                                        const float* draft_out, float atol, float rtol,
                                        float* out_full, int32_t* first_reject, float* dev,
                                        void* workspace, size_t workspace_bytes, void* stream);

/* Anchor attention without a caller workspace (the paper has no counterpart; this exists for
 * deployments where the calling code may not allocate device memory: a plug-in running inside
 * another framework's memory plan, a latency-critical serving loop that has frozen its
 * allocations, or a host that must not touch the allocator while other streams are being
 * captured).  Same computation, arguments and result as lynx_anchor_attention, but the scratch
 * memory is a fixed 8 MiB array inside the library image (every GPU that loads the library
 * holds it until the process exits); the call itself allocates nothing.
 *  - Problems whose scratch need (lynx_workspace_bytes for the same shape) exceeds 8 MiB are rejected
 *    with LYNX_ERR_WORKSPACE; nothing is launched and the array is not touched.
 *  - The first call on each device looks up the array's device address (a one-time set-up,
 *    done with that device current); make that first call before any stream capture begins.
 *  - All calls share the one array.  Each call clears the words that must start at zero, on
 *    `stream`; two calls that overlap on the GPU (different streams, or different host threads
 *    without ordering) race on it and produce wrong results.  Order them on one stream.
 *  - Out-of-range block ids are clamped as usual but cannot be reported (there is no workspace
 *    for lynx_check to read). */
lynx_status lynx_anchor_attention_static(const lynx_shape* shape, const void* q_bf16, int32_t batch,
                                         int32_t n_q, int32_t causal, lynx_plane K, lynx_plane V,
                                         const int32_t* block_table, const int32_t* seq_lens,
                                         float softmax_scale, float* out, void* stream);

/* The paper's own quantiser (Section 4.1, Algorithm 1 "Lynx Hierarchical Quantization"; inverse: the
 * inverse alpha-law of its stage 3, eq. 4) as a second scheme beside the linear one above.
 * src_bf16 : BF16 [n_pages][256][128]: pages of P = 256 consecutive tokens of one KV head (contiguous).
 * Per channel: page minimum and range (gamma_min, gamma_scale: float [n_pages][128]); per chunk of
 * C = 32 consecutive tokens its mean and largest deviation (mu, sigma: float [n_pages][8][128]);
 * magnitudes companded with the alpha-law (alpha = 255) to integers 0..120, split into a 4-bit
 * sign-aware two's-complement Anchor and a 4-bit centred Residual, packed two per byte like the linear
 * planes (q_anc, q_res: uint8 [n_pages][256][64], byte j = channel 2j | channel 2j+1 << 4).
 * Arithmetic is binary32; the readings of the algorithm's open points (alpha, epsilon = 1e-6, the scale
 * 120, the sign taken from the centred value) are stated in the library's design notes.  All pointers
 * 16-byte aligned (LYNX_ERR_ALIGN otherwise); n_pages == 0 is a valid no-op.
 * lynx_hier_dequantize reconstructs BF16 pages [n_pages][256][128] from both streams, or from the
 * Anchor alone when q_res is NULL (the Residual, a centred correction, taken as zero); the pages can be
 * attended to with lynx_bf16_attention (block_tokens = 256). */
lynx_status lynx_hier_quantize(const void* src_bf16, int64_t n_pages, uint8_t* q_anc, uint8_t* q_res,
                               float* gamma_min, float* gamma_scale, float* mu, float* sigma, void* stream);
lynx_status lynx_hier_dequantize(const uint8_t* q_anc, const uint8_t* q_res, int64_t n_pages,
                                 const float* gamma_min, const float* gamma_scale, const float* mu,
                                 const float* sigma, void* dst_bf16, void* stream);

/* Token-level verification of a speculated window (Section 4.3; the acceptance rule of speculative sampling
 * the paper builds on, Section 2.4).  The k draft tokens s_i were drawn from the Anchor-state distributions
 * p_i; the verification pass yields the distributions q_1 .. q_{k+1}.  Token i is accepted iff
 * u_i * p_i(s_i) < q_i(s_i), i.e. with probability min(1, q_i(s_i) / p_i(s_i)); n_accepted[b] is the length of
 * the accepted prefix.  next_token[b] is the correction drawn from norm(max(0, q_j - p_j)) at the first
 * rejected position j (from q_j itself should that residual be zero everywhere), or the bonus token drawn
 * from q_{k+1} when all k are accepted: the smallest vocabulary index whose cumulative weight exceeds
 * r[b] * total.  The outputs are then distributed as samples of q alone.
 * p_probs : float [batch][k][vocab]; q_probs : float [batch][k+1][vocab]; draft_tokens : int32 [batch][k]
 * (clamped to the vocabulary); u : float [batch][k] and r : float [batch], uniform in [0, 1), supplied by the
 * caller; n_accepted, next_token : int32 [batch].  1 <= k <= 64; vocab <= 1572864 (LYNX_ERR_UNSUPPORTED
 * beyond).  Sums are FP32: a decision within rounding of its threshold may differ from a higher-precision
 * evaluation. */
lynx_status lynx_token_verify(const float* p_probs, const float* q_probs, const int32_t* draft_tokens,
                              const float* u, const float* r, int32_t batch, int32_t k, int32_t vocab,
                              int32_t* n_accepted, int32_t* next_token, void* stream);

/* Decode attention over dequantised BF16 pages: the path the paper itself describes (Section 4.2: the
 * dequantisation kernel scatters BF16 pages into the paged KV memory, the engine's attention reads
 * them; Section 2 attention equation), here as the baseline the fused calls above are measured
 * against (256 bytes per row of K or V instead of 72 / 136).
 * k_pages_bf16, v_pages_bf16 : BF16 [num_blocks][Hkv][block_tokens][128], as lynx_recombine writes
 * them (dequant_bf16).  q_bf16, block_table, seq_lens, causal, softmax_scale, out as for
 * lynx_anchor_attention.  Hq/Hkv must be <= 8 and n_q <= 64; a launch takes up to 8 query columns
 * n_q * (Hq/Hkv), a call with more runs as slices of whole positions, each a pass of its own over the pages.
 * Any block_tokens.
 * workspace : lynx_bf16_workspace_bytes(shape, batch, n_q) bytes of scratch (split-K partials and the rows'
 * log-sum-exps), no initialisation needed.  Out-of-range block ids are clamped and not reported. */
size_t lynx_bf16_workspace_bytes(const lynx_shape* shape, int32_t batch, int32_t n_q);
lynx_status lynx_bf16_attention(const lynx_shape* shape, const void* q_bf16, int32_t batch, int32_t n_q,
                                int32_t causal, const void* k_pages_bf16, const void* v_pages_bf16,
                                const int32_t* block_table, const int32_t* seq_lens,
                                float softmax_scale, float* out, void* workspace,
                                size_t workspace_bytes, void* stream);

/* A quantised prefix followed by a BF16 tail (no paper counterpart as a call; Section 4.2 keeps the tokens the
 * decode node generates itself out of the quantiser, and Section 2's softmax runs over prefix and tail alike).
 * Every attention call above leaves, next to its output, the natural-log log-sum-exp of each output row's scaled
 * scores in its workspace: lse[b][j][h] = log sum_t exp(softmax_scale * q[b][j][h] . K_hat[t]) over the tokens the
 * query saw, -inf where it saw none.  lynx_workspace_lse / lynx_bf16_workspace_lse return the DEVICE address of
 * that array, float [batch][n_q][Hq], inside `workspace`, for the (shape, batch, n_q) of the call that wrote it
 * (NULL for an unsupported shape or a NULL workspace); it is valid once that call has completed on its stream and
 * until the next call on the workspace.  Nothing is launched, allocated or copied.
 *
 * lynx_lse_merge joins two results over disjoint key sets into the attention over their union:
 *   out[r] = (e^lse_a[r] out_a[r] + e^lse_b[r] out_b[r]) / (e^lse_a[r] + e^lse_b[r]),  lse_out[r] = log of that sum,
 * for n_rows rows of 128 floats (n_rows = batch * n_q * Hq for two attention calls on the same queries: the
 * prefix through lynx_anchor_attention or lynx_merge_verify_attention, non-causal, the tail through
 * lynx_bf16_attention, causal among the tail's own tokens).  A row with lse = -inf contributes nothing, whatever
 * its out row holds; two such rows give zeros and -inf.  All pointers are DEVICE pointers; out_* and out 16-byte
 * aligned; out may be out_a or out_b; lse_out may be NULL.  Asynchronous on `stream`.
 *
 * lynx_verify_decision is Section 4.3's agreement test on outputs that are already in memory -- the full-state
 * result of a window after it has been joined with the tail: out_full, draft_out float [batch][k][Hq][128],
 * dev[b][j] = max over heads and dims of |f - d| / (atol + rtol |f|), first_reject[b] = the smallest j with
 * dev[b][j] > 1, else k: the decision lynx_merge_verify_attention takes when it is given a draft.  k <= 64,
 * atol > 0, rtol >= 0; out_full and draft_out 16-byte aligned.  Asynchronous on `stream`. */
const float* lynx_workspace_lse(const lynx_shape* shape, int32_t batch, int32_t n_q, const void* workspace);
const float* lynx_bf16_workspace_lse(const lynx_shape* shape, int32_t batch, int32_t n_q, const void* workspace);
lynx_status lynx_lse_merge(const float* out_a, const float* lse_a, const float* out_b, const float* lse_b,
                           int64_t n_rows, float* out, float* lse_out, void* stream);
lynx_status lynx_verify_decision(const float* out_full, const float* draft_out, int32_t batch, int32_t k,
                                 int32_t num_q_heads, float atol, float rtol, int32_t* first_reject, float* dev,
                                 void* stream);

/* The Anchor / Residual split at other bit positions (Conclusion: splits other than INT4 + INT4; Section 4.1
 * stage 4 for the split itself, Section 2.3 for the code).  anchor_bits = A in {2, 4, 6}; R = 8 - A.  The 8-bit
 * code, scale and zero are exactly those of lynx_split_quantize; the Anchor plane holds the top A bits of every
 * code, the Residual plane the bottom R bits: (anchor << R) | residual is the code, and A = 4 writes the planes
 * lynx_split_quantize writes.  Packing per 128-element row and stream: element e's field occupies bits
 * [e w, (e + 1) w) of the row's 16 w bytes, least significant bit first (w = A or R).
 *   src_bf16 : [n_rows][128] BF16;  anchor : [n_rows][16 A] bytes;  residual : [n_rows][16 R] bytes;
 *   meta : [n_rows][2] float (scale, zero).  All DEVICE pointers, 16-byte aligned (meta: 8).
 * lynx_recombine_bits: levels = (anchor << R) | residual, or with residual NULL the middle of the Anchor's
 * bucket, (anchor << R) + 2^(R-1) (Section 4.2, Anchor phase); codes_u8 [n_rows][128] and / or dequant_bf16
 * [n_rows][128] BF16 = bf16(fl(level * scale + zero)), as lynx_recombine; at least one output.  The pages it
 * writes feed lynx_bf16_attention: that is how these splits reach attention (the fused attention calls read
 * the 4 + 4 planes only).  LYNX_ERR_UNSUPPORTED for any other anchor_bits. */
lynx_status lynx_split_quantize_bits(const void* src_bf16, int64_t n_rows, int32_t anchor_bits, uint8_t* anchor,
                                     uint8_t* residual, float* meta, void* stream);
lynx_status lynx_recombine_bits(const uint8_t* anchor, const uint8_t* residual, const float* meta, int64_t n_rows,
                                int32_t anchor_bits, uint8_t* codes_u8, void* dequant_bf16, void* stream);

/* Around the cache: rotary positions, tokens written into the planes and read back, and attention of a tree of drafted
 * tokens (the paper speculates on chains, Section 4.3; these serve decode nodes that draft trees, or that quantise the
 * tokens they accept instead of keeping them in BF16). */

/* The planes a call writes; as lynx_plane otherwise. */
typedef struct {
  uint8_t* anchor;
  uint8_t* residual;
  float* meta;
} lynx_plane_out;

/* Rotary positions on n_pairs pairs of channels, each turned by the angle of its axis' position: text has one axis, images
 * and video have time, height and width.  Pair i is (x[i], x[i + n_pairs]), or (x[2i], x[2i + 1]) if interleaved; with
 * p = positions[pair_axis[i]][token], c = cos_sin[p][i] and s = cos_sin[p][n_pairs + i]
 *     y1 = x1 c - x2 s,   y2 = x2 c + x1 s      (FP32);
 * channels from 2 n_pairs on stay as they are.  A position outside [0, n_positions) is taken as the nearest one inside. */
typedef struct {
  const int32_t* positions;   /* DEVICE int32 [n_axes][positions_stride]: positions[a * positions_stride + token] */
  const float* cos_sin;       /* DEVICE float [n_positions][2 n_pairs], 16-byte aligned */
  int64_t positions_stride;   /* at least the number of tokens */
  int32_t n_axes;             /* 1..8 */
  int32_t n_positions;        /* at least 1 */
  int32_t n_pairs;            /* 8, 16, ... 64 */
  int32_t interleaved;
  uint8_t pair_axis[64];      /* (read on the host) axis of each pair, below n_axes */
} lynx_rotary_spec;

/* q : BF16 [n_tokens][num_q_heads][128], k : BF16 [n_tokens][num_kv_heads][128], either may be NULL with 0 heads.  Strides
 * are elements from a token to the next, multiples of 8 and at least heads * 128: views of a fused projection's output can be
 * given.  The outputs have strides of their own and may be the inputs (with their strides: in place).  One rounding to BF16.
 * All pointers 16-byte aligned (positions: 4). */
lynx_status lynx_rotary(const lynx_rotary_spec* spec, const void* q, int64_t q_stride, int32_t num_q_heads, const void* k,
                        int64_t k_stride, int32_t num_kv_heads, int64_t n_tokens, void* q_out, int64_t q_out_stride,
                        void* k_out, int64_t k_out_stride, void* stream);

/* Quantises tokens' keys and values into a paged cache: the codes, planes and scalars that lynx_split_quantize gives, each
 * row in its place.  k, v : BF16 [n_src][num_kv_heads][128] with strides as for lynx_rotary.  Token i of n_tokens is source row
 * rows[i] (int32, e.g. the accepted nodes of a tree) or, with rows NULL, row i (n_src >= n_tokens); it goes to
 * slots[i] = block * block_tokens + offset (int64).  A token whose slot is outside [0, num_blocks * block_tokens) -- -1 for
 * padding -- or whose source row is outside [0, n_src) is left out.  Of several tokens with one slot, any one's values may
 * remain (K, V and planes not necessarily the same one's).  spec : NULL, or rotary positions (indexed by source row) for the
 * keys, which are turned in FP32 and quantised without a rounding in between.  Of the shape, num_kv_heads, head_dim (128),
 * block_tokens (any) and num_blocks are used.  n_tokens == 0 and, with rows, n_src == 0 are valid no-ops. */
lynx_status lynx_cache_append(const lynx_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                              int64_t n_src, const int32_t* rows, int64_t n_tokens, const int64_t* slots,
                              const lynx_rotary_spec* spec, lynx_plane_out K, lynx_plane_out V, void* stream);

/* Norms of heads: y = x / sqrt(mean x^2 + eps) * weight over a head's channels, FP32.  A tensor without weights is not normed. */
typedef struct {
  const void* q_weight;   /* DEVICE [channels of a head], BF16 or (weight_float) float, 16-byte aligned; or NULL */
  const void* k_weight;   /* likewise */
  float eps;              /* at least 0 */
  int32_t weight_float;
} lynx_head_norm;

/* Norms of queries and keys for each head and their rotary positions, in one pass: lynx_rotary's arguments, conventions and tensors
 * (in place or not), each head normed before it is turned, one rounding to BF16 behind both.  head_width : 64, 128 or 256 channels (strides at least
 * heads * head_width, weights of as many); 2 n_pairs <= head_width, and n_pairs <= 64 as always: of 256 channels at most 128 turn.  The heads of a token lie one
 * behind the other: rotary parts that lie between other channels of their heads (64 of every 192, say) are copied or projected apart first.  norm or spec may be
 * NULL: the rotation alone (of 64-wide rotary keys and queries, say), the norm alone, a copy. */
lynx_status lynx_norm_rotary(const lynx_head_norm* norm, const lynx_rotary_spec* spec, int32_t head_width, const void* q,
                             int64_t q_stride, int32_t num_q_heads, const void* k, int64_t k_stride, int32_t num_kv_heads,
                             int64_t n_tokens, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                             void* stream);

/* lynx_cache_append of keys that are normed first, by norm's k_weight (NULL norm or weight: none), then turned, then quantised: FP32 all the way,
 * no rounding in between. */
lynx_status lynx_norm_cache_append(const lynx_shape* shape, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                   int64_t n_src, const int32_t* rows, int64_t n_tokens, const int64_t* slots,
                                   const lynx_head_norm* norm, const lynx_rotary_spec* spec, lynx_plane_out K,
                                   lynx_plane_out V, void* stream);

/* Reads ranges of tokens back: output row i, offsets[b] <= i < offsets[b + 1], is token starts[b] + i - offsets[b] of sequence b,
 * BF16 bf16_rne(fl(fma(code, scale, zero))) as lynx_recombine writes it, but ordered by token:
 * k_out, v_out : BF16 [n_rows][num_kv_heads][128].  offsets : int32 [batch + 1], non-decreasing from 0; starts : int32 [batch], or
 * NULL (all 0).  Where K.residual and V.residual are NULL, the middle of the Anchor's bucket, 16 a + 8, stands for the code.
 * Rows from offsets[batch] on, tokens outside [0, max_blocks_per_seq * block_tokens) and tokens of a block id outside
 * [0, num_blocks) are zeros.  Any block_tokens.  n_rows == 0 is a valid no-op. */
lynx_status lynx_cache_read(const lynx_shape* shape, lynx_plane K, lynx_plane V, const int32_t* block_table, int32_t batch,
                            const int32_t* starts, const int32_t* offsets, int64_t n_rows, void* k_out, void* v_out,
                            void* stream);

/* Attention of drafted tokens that form a tree, over a quantised prefix and over each other, in one pass over the planes.
 * Node j of sequence b attends the tokens [0, seq_lens[b]) of the planes and the nodes i whose bit i is set in
 * tree_mask[b][j] (itself and its ancestors, say; bits from n_nodes on are ignored); a row that sees nothing gives zeros and
 * a log-sum-exp of -inf.  n_nodes <= 64, Hq/Hkv <= 16; sequences with fewer nodes leave the rest of their masks empty and
 * referenced by none: such a node's key and value enter no result, its rows attend to the prefix alone, and whatever its query holds the
 * other rows' results are what they are without it.  An infinity or a NaN in a query spoils the results of that row alone, one in a node's
 * key or value those of the rows that see the node, one in the scalars of a token of the prefix those of its sequence (all of a row's
 * channels may be NaN then).  A chain is a tree; n_nodes = 1 is a plain decode step.
 * q_bf16 : BF16 [batch][n_nodes][Hq][128];  k_nodes, v_nodes : BF16 [batch * n_nodes][Hkv][128], k_stride / v_stride elements from
 * a node to the next (multiples of 8, at least Hkv * 128: views of a fused projection's output);  tree_mask : uint64 [batch][n_nodes].
 * K, V with both residuals: the full codes; with both NULL: the Anchor's state.
 * out : [batch][n_nodes][Hq][128], BF16, or float where out_float is set (for lynx_lse_merge); lse : float [batch][n_nodes][Hq]
 * or NULL.  All pointers 16-byte aligned, the planes' meta among them
 * (tree_mask: 8; block_table, seq_lens, lse: 4).
 * Precision: scores, statistics and sums are FP32 or exact integers.  With more than 32 rows n_nodes * Hq/Hkv (and where the Anchor is short)
 * keys enter the scores exactly but for their middles zero + 128 scale (2^-22 of them) and scales below 2^-36 of the largest magnitude of their
 * 128 tokens; weights and values enter the second product as FP16 relative to exponents of their own (2^-12 of a term; value rows below 2^-29 of
 * the largest of their 128 tokens lose bits).  Queries are exact to 2^-24 (with fewer rows 2^-22) of the largest among the KV head's rows that
 * see a node, or of their own row's where that is larger; where no row sees a node, to 2^-14 and 2^-18 of their own row's at least.  With fewer rows
 * weights have 22 bits and more; a value row's scale counts as 2^-80, and as 2^-24 of its zero point, at least.
 * workspace : lynx_tree_workspace_bytes(shape, batch, n_nodes) bytes (0: unsupported shape), zero-filled once before its first use
 * (lynx_workspace_init); each call leaves it ready for the next, also of another batch, shape or number of nodes that it is large enough for:
 * one for a batch and a number of nodes is for smaller ones of both, of the same shape.
 * Calls that share one are ordered on a stream.  lynx_check reads its status word: block ids out of range are
 * clamped and recorded there.  block_tokens a multiple of 16; seq_lens[b] is clamped to the table's capacity. */
size_t lynx_tree_workspace_bytes(const lynx_shape* shape, int32_t batch, int32_t n_nodes);
lynx_status lynx_tree_attention(const lynx_shape* shape, const void* q_bf16, int32_t batch, int32_t n_nodes, lynx_plane K,
                                lynx_plane V, const int32_t* block_table, const int32_t* seq_lens, const void* k_nodes,
                                int64_t k_stride, const void* v_nodes, int64_t v_stride, const uint64_t* tree_mask,
                                float softmax_scale, int32_t out_float, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream);

/* Block tables, slots and positions from the lengths that requests have (old_lens) and are to have (new_lens), int32 [batch], on the device:
 * requests that grow take blocks from the pool's free ones, those that shrink (to 0: that end) give blocks back.  With bt = block_tokens,
 * have = ceil(old / bt) and want = ceil(new / bt) request b needs max(0, want - have) blocks.  It gets them where it needs none or where the sum
 * of all requests' needs up to and with its own is at most the number of free blocks; else it stays as it is (preempt it, and plan again).
 * block_table : int32 [batch][max_blocks_per_seq], of which entries [have, want) of a growing request are written and entries [want, have) of a
 *   shrinking one are given back (and left as they stand).
 * free_ring : int32 [num_blocks], pool_state : int32 [4] = {place of the first free block in the ring, number of free blocks, 0, 0}.  Free
 *   blocks are taken from the front, in the requests' order, and given back behind the last, in the requests' order and each request's: results
 *   do not depend on how the work is spread.  What is free and what requests hold must be at most num_blocks together, and a block held
 *   by one request at most (a block shared by several is not to be given back through this call).
 * lens : int32 [batch], the length each request has now: new_lens[b], or old_lens[b] where it did not get its blocks.  Not old_lens or new_lens.
 * Tokens [old, new) of the requests, one behind the other (a request that did not get its blocks has its rows, too), are rows of
 * offsets : int32 [batch + 1], or NULL: each request's first row, and their number;
 * slots : int64 [max_tokens], or NULL: block * bt + offset as lynx_cache_append takes it, -1 for tokens without a block;
 * positions : int32 [max_tokens], or NULL: the token's number in its sequence, as lynx_rotary_spec takes it.
 * Rows behind the last have slot -1 and position 0; rows from max_tokens on are left out.  With offsets and old_lens as its starts lynx_cache_read
 * reads the new tokens back.  Lengths are clamped to [0, max_blocks_per_seq * bt].  Any block_tokens; batch * max_blocks_per_seq * bt and
 * max_tokens below 2^31 - 8192 (LYNX_ERR_UNSUPPORTED otherwise).  Calls that share a pool are ordered on a stream. */
lynx_status lynx_plan_blocks(const lynx_shape* shape, const int32_t* old_lens, const int32_t* new_lens, int32_t batch,
                             int32_t* block_table, int32_t* free_ring, int32_t* pool_state, int64_t max_tokens, int32_t* lens,
                             int32_t* offsets, int64_t* slots, int32_t* positions, void* stream);

/* Caches of latents: models whose keys and values are expanded from one vector of 512 channels a token, next to a rotary key of 64 that all heads
 * share.  A latent is four rows of the planes -- num_kv_heads is 4 and head h holds channels [128 h, 128 (h + 1)) --, so that lynx_split_quantize,
 * lynx_recombine and the transfer of the streams take it as it is.  Rotary keys stay BF16 : rope_pages [num_blocks][block_tokens][64].
 *
 * lynx_latent_append: latents BF16 [n_src][512] and rope_keys BF16 [n_src][64], strides as for lynx_rotary (views of one projection's output).
 * rows, n_tokens, slots: as for lynx_cache_append (of several tokens with one slot, any one's rows and key may remain).  weight : NULL, or 512 BF16
 * (weight_float: float) weights of a norm over the latent's 512 channels, y = x / sqrt(mean x^2 + eps) * weight, FP32, quantised without a rounding
 * in between.  spec : NULL, or rotary positions of the keys, 2 n_pairs <= 64, one rounding to BF16.  Pointers 16-byte aligned (slots, meta: 8, rows: 4).
 * lynx_latent_read: ranges of tokens as lynx_cache_read's, latents_out BF16 [n_rows][512] (residual NULL: the middles of the Anchor's buckets)
 * and rope_out BF16 [n_rows][64]: what the expanded form of the attention multiplies by its projections.  Any block_tokens, both calls. */
lynx_status lynx_latent_append(const lynx_shape* shape, const void* latents, int64_t latent_stride, const void* rope_keys,
                               int64_t rope_stride, int64_t n_src, const int32_t* rows, int64_t n_tokens, const int64_t* slots,
                               const void* weight, int32_t weight_float, float eps, const lynx_rotary_spec* spec,
                               lynx_plane_out C, void* rope_pages, void* stream);
lynx_status lynx_latent_read(const lynx_shape* shape, lynx_plane C, const void* rope_pages, const int32_t* block_table,
                             int32_t batch, const int32_t* starts, const int32_t* offsets, int64_t n_rows, void* latents_out,
                             void* rope_out, void* stream);

/* Attention over a cache of latents, absorbed form: all heads of the queries, multiplied by their keys' projections beforehand, read the same latents,
 *   score = softmax_scale * (q_latent . latent_t + q_rope . rope_key_t),   out = sum_t softmax(score)_t latent_t,
 * whose rows the caller multiplies by the values' projections.  For row r = (b n_q + j) Hq + h, q_latent : BF16 [rows][512] with q_stride elements from a
 * row to the next, q_rope : BF16 [rows][64] with q_rope_stride (multiples of 8, at least 512 and 64: views of one [rows][576] can be given), rotated.  n_q <= 64
 * positions, Hq <= 128 heads, num_kv_heads 4 (see above), block_tokens a multiple of 16.  Position j of sequence b attends tokens [0, seq_lens[b]) (causal == 0) or
 * [0, seq_lens[b] - n_q + j + 1); one that sees no token gives zeros and a log-sum-exp of -inf.  softmax_scale 0 means 1/sqrt(192), of heads with 128 + 64
 * channels before they are absorbed.  C with its residual: the full codes; residual NULL: the Anchor's state.
 * out : [batch][n_q][Hq][512], BF16, or float where out_float is set; lse : float [batch][n_q][Hq] (natural log) or NULL.  Pointers 16-byte aligned (meta 8;
 * block_table, seq_lens, lse 4).
 * An infinity or a NaN in a query spoils that row alone, one in the scalars or the rotary key of a token the rows that see it (all of a sequence's may be NaN); what
 * lies behind a sequence's end, in blocks or in the table, is not looked at.
 * Precision: scores, statistics and sums are FP32.  A code's value, middle + scale (c - 128) with middle = zero + 128 scale, enters both products as FP16: scale and middle rounded (2^-11 of
 * each at most), then the value (2^-11 of it), relative to a power of two of the 128 tokens that the value's token is among (tokens [128 i, 128 i + 128) of a sequence), so that any finite scale is
 * handled.  Among such tokens rows lose bits of their scale where they hold less than 2^-21 of the largest value (2^-25 of it: seven bits are left, 2^-33: none), and values below 2^-29 of it lose bits.
 * Rotary keys enter as they are, queries relative to their row's largest (exact down to 2^-32 of it), weights as FP16 (2^-11 of one; below 2^-16 of a row's largest they lose bits,
 * below 2^-26 they are left out of the sum's numerator), whatever the sizes of other tokens' values; only where a set of 128 tokens holds less than 2^-64 of another's largest value its
 * weights may lose as many bits more as it holds less, and all of them beyond 2^-90.
 * Up to 64 rows n_q * Hq of a sequence take one pass over its planes.
 * workspace : lynx_latent_workspace_bytes(shape, batch, n_q) bytes (0: unsupported shape), zero-filled once before its first use (lynx_workspace_init); it serves
 * smaller batches and fewer positions of the same shape, too.  Calls that share one are ordered on a stream.  lynx_check reads its status word: block ids out of
 * range are clamped and recorded there.  seq_lens[b] is clamped to the table's capacity. */
size_t lynx_latent_workspace_bytes(const lynx_shape* shape, int32_t batch, int32_t n_q);
lynx_status lynx_latent_attention(const lynx_shape* shape, const void* q_latent, int64_t q_stride, const void* q_rope,
                                  int64_t q_rope_stride, int32_t batch, int32_t n_q, int32_t causal, lynx_plane C,
                                  const void* rope_pages, const int32_t* block_table, const int32_t* seq_lens,
                                  float softmax_scale, int32_t out_float, void* out, float* lse, void* workspace,
                                  size_t workspace_bytes, void* stream);

/* Synchronises `stream`, reads and clears the workspace's status word.  Test / debug use. */
lynx_status lynx_check(void* workspace, void* stream);

const char* lynx_status_string(lynx_status s);
int lynx_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LYNX_H_ */
