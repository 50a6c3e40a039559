/*
 * tilefuse.h -- C ABI of the fused weight-only quantized matmul for gfx950.
 *
 * The operation (TileFuse, Sections 2.1-2.2 and 4.2-4.3):
 *
 *     C[m, n] = sum_k A[m, k] * w_hat[k, n],      C = A x B (Section 2.1)
 *     w_hat[k, n] = s[g, n] * (q[k, n] - z[g, n]), g = floor(k / G)  (Eq. 2)
 *
 * A is fp16 [M, K] row-major, the weights are 4-bit (W4A16) or 8-bit (W8A16)
 * integer codes with one fp16 scale and one integer zero-point per group of G
 * consecutive k in one column n (Section 2.2), accumulation is fp32 and C is
 * fp16 [M, N] row-major, rounded to nearest even.  The weights never exist in
 * memory as fp16: each kernel unpacks and dequantizes them on the fly (Section
 * 4.3, fused unpack -> dequantize -> multiply-accumulate).
 *
 * Weights are first rearranged once, offline, into a device-private layout
 * (tf_pack_w4 / tf_pack_w8; the GPU counterpart of the offline pre-tiling of
 * Section 4.2).  The packed buffer is opaque; pass the same (K, N, group) to
 * the matmul calls that were given to the pack call.
 *
 * Conventions for every entry point:
 *  - All array pointers are DEVICE pointers (hipMalloc / torch CUDA tensors).
 *  - fp16 values travel as uint16_t bit patterns.
 *  - `stream` is a hipStream_t passed as void*; NULL means the null stream.  The
 *    current device of the calling thread has to be that of the stream and the
 *    arrays (the Python binding sees to it).
 *    Calls only enqueue work on `stream` and return; the caller synchronizes.
 *  - The caller allocates and frees every buffer; the library keeps no device
 *    memory.  Its only global state is a per-device cache of the compute-unit
 *    count (read atomically; the launch plans depend on it) and the locks that
 *    let calls with one workspace take turns, so calls are thread-safe: several
 *    threads may call on one stream with one workspace.  Calls on streams that
 *    run at the same time need workspaces of their own.  Plans are made for the
 *    device of the `stream` argument.
 *  - Arguments are validated before any HIP call; a rejected call enqueues
 *    nothing.  Only TF_ERR_HIP comes from the runtime (launch failure).
 *  - Outputs must not overlap inputs.
 *  - No C++ exception crosses this boundary.  The library prints nothing,
 *    except with the environment variable TF_LOG=1 (read once, at the first
 *    matmul call): each matmul call then writes one line to stderr naming the
 *    kernel it launched and its plan (tiles, K slices, stream-K blocks).
 */
#ifndef TILEFUSE_H
#define TILEFUSE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Status codes (returned as int; negative means failure). */
enum tf_status {
    TF_OK = 0,
    TF_ERR_NULL = -1,   /* a required pointer is NULL                          */
    TF_ERR_SHAPE = -2,  /* M < 1, K or N <= 0, K % group != 0, N % 8 != 0,
                           or a dimension above TF_MAX_DIM; heads, strides,
                           pages or batch out of range                          */
    TF_ERR_GROUP = -3,  /* group is not a positive multiple of 32              */
    TF_ERR_ALIGN = -4,  /* a pointer is not 16-byte aligned                    */
    TF_ERR_ARG = -5,    /* other bad argument: bits not 4/8, GEMV with M > 8,
                           unknown dtype, workspace too small                  */
    TF_ERR_HIP = -6     /* the HIP runtime reported an error at launch         */
};

/* Output dtypes of tf_dequant. */
enum tf_dtype { TF_F16 = 1, TF_F32 = 2, TF_BF16 = 3 };

/* Largest accepted K and N (each) and M; keeps every byte offset in int64
 * and every per-kernel index in 32 bits. */
#define TF_MAX_DIM 65536
#define TF_MAX_M (1 << 20)
/* Largest M accepted by the GEMV entry points (decode, Section 2.1). */
#define TF_GEMV_MAX_M 8

/* Library version of the packed layout; bumps whenever the layout changes. */
int tf_layout_version(void);

/* Human-readable text for a status code (static storage, never NULL). */
const char* tf_status_str(int status);

/*
 * Size in bytes of the packed buffer for a (bits, K, N, group) weight.
 * bits is 4 or 8.  Returns > 0, or a negative tf_status on bad arguments.
 */
int64_t tf_packed_bytes(int bits, int64_t K, int64_t N, int group);

/*
 * Offline pre-tiling of a 4-bit AWQ weight (Section 4.2: weights are known at
 * deployment, so the rearrangement is done once and is not on the timed path).
 *   qweight  int32 [K, N/8]   nibble i (bits 4i..4i+3) of word j = q[k, 8j+i]
 *   qzeros   int32 [K/G, N/8] same packing, z[g, 8j+i]
 *   scales   fp16  [K/G, N]   s[g, n]
 *   packed   tf_packed_bytes(4, K, N, group) bytes, written entirely
 * Requires N % 8 == 0, group % 32 == 0, K % group == 0, 16-byte aligned
 * pointers.  Integer rearrangement only: scales are copied bit for bit.
 */
int tf_pack_w4(const int32_t* qweight, const int32_t* qzeros, const uint16_t* scales,
               int64_t K, int64_t N, int group, void* packed, void* stream);

/*
 * Offline pre-tiling of an 8-bit weight with per-group zero-points.
 *   qweight  uint8 [K, N]     q[k, n]
 *   zeros    uint8 [K/G, N]   z[g, n]
 *   scales   fp16  [K/G, N]   s[g, n]
 *   packed   tf_packed_bytes(8, K, N, group) bytes
 * Same constraints as tf_pack_w4 (N % 8 == 0 keeps rows 8-byte aligned).
 * The symmetric form of Eq. 1 is the case z = 0 (pass a zero-filled array).
 */
int tf_pack_w8(const uint8_t* qweight, const uint8_t* zeros, const uint16_t* scales,
               int64_t K, int64_t N, int group, void* packed, void* stream);

/*
 * Offline pre-tiling of the W8A16 form of Section 2.2 (W8A16 paragraph):
 * signed INT8 weights with one scale per output channel and no zero-point,
 * dequantized by Eq. 1 as w_hat[k, n] = s[n] * q[k, n].
 *   qweight  int8  [K, N]     q[k, n] in -128..127
 *   scales   fp16  [N]        s[n]
 *   packed   tf_packed_bytes(8, K, N, group) bytes
 * Stored as the 8-bit layout with codes q + 128, zero-point 128 and the
 * column's scale repeated in every group of `group` rows, so the 8-bit
 * matmul and debug entry points (bits = 8, the same group) apply unchanged:
 * s * ((q + 128) - 128) = s * q exactly.  `group` only sets that internal
 * grouping (128 is the usual choice; it needs K % group == 0).  Same
 * constraints and errors as tf_pack_w8.
 */
int tf_pack_w8_sym(const int8_t* qweight, const uint16_t* scales, int64_t K, int64_t N, int group,
                   void* packed, void* stream);

/*
 * Workspace the matmul entry points can use for this problem, in bytes (0
 * when the kernels chosen for it need none).  Negative tf_status on bad
 * arguments.  The workspace holds per-K-slice partial sums (fp32) and, for
 * the decode GEMV and the weight-streaming matrix-core form, arrival counters;
 * it lets those kernels split K over more workgroups than there are output
 * panels, and the tiled GEMMs split K (partials summed by a second launch in
 * slice order) or share tiles between blocks (stream-K).
 *
 * Contract for every `workspace` argument below:
 *  - NULL selects kernels that need none (workspace_bytes is then ignored);
 *  - otherwise it is a device buffer of at least tf_workspace_bytes(...)
 *    bytes, 16-byte aligned and ZERO-FILLED before its first use; each call
 *    returns the arrival counters it used to zero, so the same buffer serves
 *    any later call (of any shape it is large enough for) without clearing;
 *  - calls that may run concurrently must not share one workspace.
 */
int64_t tf_workspace_bytes(int bits, int64_t M, int64_t K, int64_t N, int group);

/*
 * The same query under the name of the GEMM's workspace (the prefill GEMM
 * is the main user of a workspace: stream-K or split-K partial tiles).  It
 * returns exactly tf_workspace_bytes(bits, M, K, N, group), which already
 * covers every kernel the GEMM and GEMV entry points can choose for M rows,
 * so one buffer of that size serves either call.
 */
int64_t tf_gemm_workspace_bytes(int bits, int64_t M, int64_t K, int64_t N, int group);

/*
 * Prefill GEMM (Section 2.1: M grows with the prompt length):
 *   C_f16[M, N] = A_f16[M, K] x dequant(packed)[K, N], fp32 accumulate, RNE.
 * Any M >= 1.  M <= 3 runs the decode GEMV; 4 <= M <= 32 a weight-streaming
 * kernel on the matrix cores (16 or 32 row slots); larger M the tiled
 * matrix-core GEMMs, or, up to 64 rows of 8-bit weights with short K, the
 * streaming kernel with 64 row slots.  The tiled GEMMs and the 64-slot form
 * feed the matrix cores the dequantized fp16 weight RNE(s * (q - z)), rounded
 * once; up to 32 rows the streaming kernel feeds the codes themselves and
 * applies scale and zero-point to each group's sums (Eq. 2 summed over a
 * group), so no weight is rounded (as in the decode GEMV up to 4 rows).
 * workspace: see tf_workspace_bytes.
 */
int tf_w4a16_gemm(const uint16_t* A_f16, const void* packed, uint16_t* C_f16,
                  int64_t M, int64_t K, int64_t N, int group,
                  void* workspace, size_t workspace_bytes, void* stream);
int tf_w8a16_gemm(const uint16_t* A_f16, const void* packed, uint16_t* C_f16,
                  int64_t M, int64_t K, int64_t N, int group,
                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decode GEMV (Section 2.1: batch-1 generation turns linear layers into
 * matrix-vector products), 1 <= M <= TF_GEMV_MAX_M rows of A.
 * Same operands and result as the GEMM; vector ALU only, fp32 accumulate.
 * With a workspace (see tf_workspace_bytes) K is split over many
 * workgroups and the slices are added in a fixed order, so for a given
 * shape and workspace choice the result is bitwise identical run to run
 * (with and without a workspace the fp32 summation order differs).
 */
int tf_w4a16_gemv(const uint16_t* A_f16, const void* packed, uint16_t* C_f16,
                  int64_t M, int64_t K, int64_t N, int group,
                  void* workspace, size_t workspace_bytes, void* stream);
int tf_w8a16_gemv(const uint16_t* A_f16, const void* packed, uint16_t* C_f16,
                  int64_t M, int64_t K, int64_t N, int group,
                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * tf_w4a16_gemv without a workspace argument and without any allocation, for
 * callers that cannot allocate device memory (code under HIP graph capture,
 * serving loops that forbid hipMalloc).  Same operands, checks, kernels and
 * result as tf_w4a16_gemv with a workspace: where the decode GEMV splits K,
 * its partial sums and arrival counters live in a scratch array of 1 MiB in
 * the library's static device memory, one per GPU, held until the process
 * ends (every shape the GEMV entry points accept needs at most about 0.9 MiB;
 * a larger need returns TF_ERR_ARG).  The call allocates nothing: the first
 * call on a device looks up that device's copy of the array and enqueues one
 * small kernel on `stream` that zeroes its counters (again at the next call
 * outside stream capture if the first was captured); every call leaves the
 * counters at zero.  All calls on one GPU share its array, so calls that may
 * run concurrently on one GPU (different streams, not ordered by events)
 * race and must not overlap.
 */
int tf_w4a16_gemv_noalloc(const uint16_t* A_f16, const void* packed, uint16_t* C_f16,
                          int64_t M, int64_t K, int64_t N, int group, void* stream);

/*
 * BF16 activations and scales (the paper's dtype: Section 2.2 takes BF16
 * activations, Section 4.2 stores BF16 scales beside each weight tile,
 * Section 4.3 holds the dequantized weights in BF16 before the multiply):
 *   C_bf16[M, N] = A_bf16[M, K] x RNE_bf16(s_bf16 * (q - z))[K, N],
 * fp32 accumulate, C rounded to bfloat16, nearest even.
 * The packed buffer is the same format: tf_pack_w4 / tf_pack_w8 /
 * tf_pack_w8_sym copy the 16-bit scale patterns verbatim, so packing with
 * bfloat16 scale bits gives a buffer for these entry points (and packing
 * with fp16 bits one for the entry points above; the buffer does not record
 * which).  Same shapes, alignment, workspace contract and tf_workspace_bytes
 * as the fp16 entry points; the same kernels are chosen for each M.
 * s * (q - z) is formed exactly in fp32 and rounded once to bfloat16.
 */
int tf_w4a16_gemm_bf16(const uint16_t* A_bf16, const void* packed, uint16_t* C_bf16,
                       int64_t M, int64_t K, int64_t N, int group,
                       void* workspace, size_t workspace_bytes, void* stream);
int tf_w8a16_gemm_bf16(const uint16_t* A_bf16, const void* packed, uint16_t* C_bf16,
                       int64_t M, int64_t K, int64_t N, int group,
                       void* workspace, size_t workspace_bytes, void* stream);
int tf_w4a16_gemv_bf16(const uint16_t* A_bf16, const void* packed, uint16_t* C_bf16,
                       int64_t M, int64_t K, int64_t N, int group,
                       void* workspace, size_t workspace_bytes, void* stream);
int tf_w8a16_gemv_bf16(const uint16_t* A_bf16, const void* packed, uint16_t* C_bf16,
                       int64_t M, int64_t K, int64_t N, int group,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * Debug / test exports.  They read the packed buffer through the same device
 * unpack and dequantize code as the matmul kernels.
 *   tf_unpack : q_out uint8 [K, N] and z_out uint8 [K/G, N] (Section 4.3 unpack)
 *   tf_dequant: W_out [K, N] of s * (q - z) (Eq. 2), dtype TF_F16 (rounded
 *               once, nearest even) or TF_F32 (exact), both reading the
 *               scales as fp16; or TF_BF16: scales read as bfloat16, the
 *               weight rounded once to bfloat16 as the BF16 entry points do.
 */
int tf_unpack(int bits, const void* packed, int64_t K, int64_t N, int group,
              uint8_t* q_out, uint8_t* z_out, void* stream);
int tf_dequant(int bits, const void* packed, int64_t K, int64_t N, int group,
               int out_dtype, void* W_out, void* stream);

/*
 * Gated activation of a transformer MLP, for a layer-level composite around
 * the matmuls (gate/up GEMM -> this -> down GEMM); not part of the paper's
 * method:
 *   H[m, n] = silu(G[m, n]) * U[m, n],   silu(g) = g / (1 + exp(-g)),
 * where G = GU[:, 0:N] and U = GU[:, N:2N] are the two halves of one fp16
 * [M, 2N] row-major matrix (the output of a GEMM whose weight concatenates
 * the gate and up projections along N).  Computed in fp32; H is fp16 [M, N]
 * row-major, rounded to nearest even.  Requires N % 8 == 0 and 16-byte
 * aligned pointers; H must not overlap GU.
 */
int tf_silu_mul(const uint16_t* GU_f16, int64_t M, int64_t N, uint16_t* H_f16, void* stream);
/* The same with bfloat16 GU and H (the layer composite in the paper's dtype). */
int tf_silu_mul_bf16(const uint16_t* GU_bf16, int64_t M, int64_t N, uint16_t* H_bf16, void* stream);

/*
 * ---------------------------------------------------------------------------
 * The rest of a decoder layer around the quantized linear layers (not part of
 * the paper's method): the norm between two blocks, a 4-bit paged key/value
 * cache, attention of single tokens over it, and attention over whole prompts.
 * With the matmuls above they make a decoder layer run end to end.
 *
 * `dtype` is TF_F16 or TF_BF16, the type of every 16-bit tensor of a call.
 * Activations are [tokens, heads, head_dim] with head_dim contiguous, heads
 * head_dim apart and tokens `stride` elements apart (a multiple of 8, at least
 * heads * head_dim and at most 2^24), so that the parts of one packed q, k, v projection are
 * operands as they are.  head_dim is 64, 128 or 256; q_heads is a multiple of
 * kv_heads, and query head h reads key/value head h / (q_heads / kv_heads).
 * Sequences are packed one after the other: sequence b has the tokens
 * cu[b] .. cu[b + 1] - 1 (int32 [batch + 1] on the device, not decreasing).
 * Lengths, offsets and page tables stay on the device; the kernels check them
 * against the sizes given here and never leave the buffers.
 * ---------------------------------------------------------------------------
 */

/* Largest accepted numbers of sequences and heads. */
#define TF_MAX_BATCH 65536
#define TF_MAX_HEADS 1024

/*
 * The residual sum and the norms around it, in fp32 with one rounding per
 * output:
 *   y = X                     or  rms(X) * (post_weight + weight_offset)
 *   r = residual + scale * gate * y           -> residual_out
 *   Y = rms(r) * (weight + weight_offset),    rms(t) = t / sqrt(mean(t^2) + eps)
 * over rows of N.  Y is computed from r before r's rounding.  residual,
 * post_weight and gate may be NULL (absent); so may residual_out or (with
 * weight) Y, not both.  weights are [N]; gate is [N] (gate_stride 0) or [M, N]
 * with rows gate_stride apart.  residual_out may be residual itself and Y may
 * be X; nothing else may overlap.  N % 8 == 0, gate_stride % 8 == 0, 16-byte
 * aligned pointers.
 */
int tf_add_rms_norm(int dtype, const void* X, const void* residual, const void* post_weight, const void* gate,
                    int64_t gate_stride, float scale, const void* weight, float weight_offset, float eps,
                    int64_t M, int64_t N, void* residual_out, void* Y, void* stream);

/*
 * A 4-bit paged key/value cache.  Each key and each value of a head is a row
 * of head_dim codes of 4 bits with a scale s and a zero-point z of its own
 * (dtype, rounded to nearest even), standing for s * (q - z):
 *   s = (max - min) / 15,  z = -min / s,  q = round(x / s + z) within 0..15
 * in fp32 from the row's fp32 values, with s and z as rounded.  A row whose
 * values are one within the type's precision (s under 2^-100, or |min| over
 * 32768 s) is stored as its minimum, one with a value that is not finite reads
 * back as NaN.  `data` holds tf_kv4_cache_bytes(...) bytes, 256-byte aligned,
 * in `pages` pages of page_size positions (a multiple of 32); its layout is
 * opaque.  It needs no initial value: only appended positions are read.
 * Positions of sequence b live on the pages table[b * table_stride + p],
 * p = position / page_size < max_pages (int32; an entry outside 0..pages-1 is
 * no page: nothing is stored there, and attention leaves its positions out).
 */
typedef struct tf_kv4_cache {
    void* data;
    int64_t pages;
    int32_t page_size;
    int32_t kv_heads;
    int32_t head_dim;
    int32_t dtype;
    const int32_t* table;
    int64_t table_stride;
    int64_t max_pages;
} tf_kv4_cache;

/* Bytes of a cache of that many pages, or a negative tf_status. */
int64_t tf_kv4_cache_bytes(int64_t pages, int page_size, int kv_heads, int head_dim);

/*
 * Rotates the queries and keys of `tokens` packed tokens and appends keys and
 * values to the cache.  Token i of sequence b has the position starts[b] + i.
 * With cos and sin (fp32 [positions, head_dim / 2]) the pair (x[d],
 * x[d + head_dim / 2]) turns by the position's angle:
 *   (x1 cos - x2 sin, x2 cos + x1 sin) in fp32
 * and the cached key is quantized from that; NULL for both leaves q and k as
 * they are.  Q may be NULL (with Q_out, q_heads = 0); K_out may be NULL.  Q_out
 * [tokens, q_heads, head_dim] and K_out [tokens, kv_heads, head_dim]
 * (contiguous) receive the rotated rows rounded to dtype.  A token that no
 * sequence owns, or whose position is outside the tables of angles, has NaN in
 * Q_out and K_out and is not cached.  No two tokens of a call may share a position.
 */
int tf_kv4_append(const tf_kv4_cache* cache, const void* Q, int64_t q_stride, const void* K, int64_t k_stride,
                  const void* V, int64_t v_stride, const float* cos, const float* sin, int64_t positions,
                  const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens, int q_heads,
                  void* Q_out, void* K_out, void* stream);

/*
 * Reads the cached rows of positions starts[b] + i, i < cu[b + 1] - cu[b], back
 * as values s * (q - z) rounded to dtype: K_out and V_out are [tokens, kv_heads,
 * head_dim], packed as cu says.  A position without a page reads as NaN.
 */
int tf_kv4_read(const tf_kv4_cache* cache, const int32_t* cu, const int32_t* starts, int64_t batch, int64_t tokens,
                void* K_out, void* V_out, void* stream);

/*
 * Attention of the last q_len tokens of each sequence over its cache (decode;
 * q_len above 1 for speculated tokens, at most TF_KV4_MAX_Q):
 *   O[b, i, h] = sum_j softmax_j(scale * Q[b, i, h] . K[j]) V[j]
 * over the positions j <= lens[b] - q_len + i, j >= 0.  A query that sees none
 * gives zeros.  Q is [batch * q_len, q_heads, head_dim] with rows q_stride
 * apart, O contiguous.  lens[b] (int32) counts the appended tokens, the asking
 * ones among them; more than max_pages * page_size counts as that.  Codes are
 * multiplied as they are; scales and zero-points act in fp32, except that
 * softmax weights times the value's scale are rounded to dtype for the matrix
 * cores.  workspace: tf_kv4_attention_workspace_bytes(...) bytes, 16-byte
 * aligned and ZERO-FILLED before its first use; each call returns its counters
 * to zero, so that one buffer serves any later call of these sizes or smaller
 * need.  Calls that may run concurrently must not share one, and no matmul
 * call may use it.  The result is the same from run to run.
 */
#define TF_KV4_MAX_Q 8
int64_t tf_kv4_attention_workspace_bytes(int64_t batch, int q_len, int q_heads, int kv_heads, int head_dim);
int tf_kv4_attention(const tf_kv4_cache* cache, const void* Q, int64_t q_stride, const int32_t* lens, int64_t batch,
                     int q_len, int q_heads, float scale, void* O, void* workspace, size_t workspace_bytes,
                     void* stream);

/*
 * Attention over whole packed prompts:
 *   O[i, h] = sum_j softmax_j(scale * Q[i, h] . K[j]) V[j]
 * for query i of sequence b over its keys j; with causal, only j <= i + n_k - n_q
 * (the queries are the last n_q of n_k tokens).  A query that sees no key gives
 * zeros; keys and values that it does not see do not act on it, NaN and infinite
 * ones neither.  cu_q and cu_k: int32 [batch + 1].  Q, K, V strided as above, O
 * [tokens_q, q_heads, head_dim] contiguous.  Scores and sums in fp32, softmax
 * weights rounded to dtype for the matrix cores.  Rows of O that no sequence
 * owns are not written.  workspace: NULL, or at least
 * tf_prompt_attention_workspace_bytes(...) bytes (may be 0), 16-byte aligned, no
 * initial value: few queries on many keys are then split over the keys too,
 * their parts added in a fixed order.  Calls that may run concurrently must not
 * share one.
 */
int64_t tf_prompt_attention_workspace_bytes(int64_t batch, int64_t tokens_q, int64_t tokens_k, int q_heads,
                                            int kv_heads, int head_dim);
int tf_prompt_attention(int dtype, const void* Q, int64_t q_stride, const void* K, int64_t k_stride, const void* V,
                        int64_t v_stride, const int32_t* cu_q, const int32_t* cu_k, int64_t batch, int64_t tokens_q,
                        int64_t tokens_k, int q_heads, int kv_heads, int head_dim, float scale, int causal, void* O,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * ---------------------------------------------------------------------------
 * Linear layers whose activations are 8-bit integers too, and layers made of
 * experts (not part of the paper's method).  A row of activations stands as codes
 * q in -127..127 with a scale of its own, a weight's column as the signed INT8
 * codes of tf_pack_w8_sym with a scale of its own, and the product is one of
 * integers:
 *   C[m, n] = s_a[m] * s_w[n] * sum_k qa[m, k] * qw[k, n].
 * The sums are exact (int32).  An output is the sum as fp32 times the product of its
 * two scales in fp32, rounded once more to its type (four roundings in all); scales
 * may be as large or small as fp32 holds, and their product may leave it.  `dtype` is
 * TF_F16 or TF_BF16, the type of the 16-bit tensors of a call.
 * ---------------------------------------------------------------------------
 */

/* Largest accepted numbers of experts, of choices a token, and of rows of an
 * expert product (tokens times choices). */
#define TF_MAX_EXPERTS 1024
#define TF_MAX_TOP_K 32
#define TF_MAX_SLOTS (TF_MAX_M * TF_MAX_TOP_K)

/*
 * Codes of the rows of X [M, N], or with `gated` of H[m, n] = silu(X[m, n]) *
 * X[m, N + n], X being [M, 2 N] (H in fp32, not rounded between):
 *   scales[m] = max|row| / 127,   codes[m, n] = round(row[n] * (127 / max|row|)).
 * Rows of X are x_stride elements apart; codes [M, N] and scales fp32 [M] are
 * contiguous.  A row whose values are all under 2^-100 has the scale 0 and codes
 * 0, one with a value that is not finite the scale NaN and codes 0.  N % 16 == 0,
 * x_stride % 8 == 0, 16-byte aligned X and codes.
 */
int tf_quantize_rows(int dtype, const void* X, int64_t x_stride, int64_t M, int64_t N, int gated, int8_t* codes,
                     float* scales, void* stream);

/*
 * Pre-tiling of `experts` weights (1 for a dense layer): qweight int8
 * [experts, K, N] in -128..127, scales [experts, N] of scale_dtype (TF_F16,
 * TF_BF16 or TF_F32).  packed: experts * tf_w8a8_packed_bytes(K, N) bytes, 256-byte
 * aligned, one expert after the other; it serves outputs of either type.
 * K % 16 == 0, N % 8 == 0.  A weight whose signs and scales suit tf_pack_w8_sym
 * suits this call as it is.
 */
int64_t tf_w8a8_packed_bytes(int64_t K, int64_t N);
int tf_pack_w8a8(const int8_t* qweight, const void* scales, int scale_dtype, int64_t K, int64_t N, int64_t experts,
                 void* packed, void* stream);

/*
 * C [M, N] = the product above of codes A [M, K], their scales and a packed weight.
 * workspace: NULL, or at least tf_w8a8_workspace_bytes(...) bytes (may be 0), 16-byte
 * aligned, no initial value: few rows by few columns are then split over K too.  The
 * result is the same bit for bit.  Calls that may run concurrently must not share one.
 */
int64_t tf_w8a8_workspace_bytes(int64_t M, int64_t K, int64_t N);
int tf_w8a8_gemm(int dtype, const int8_t* A, const float* a_scales, const void* packed, void* C, int64_t M, int64_t K,
                 int64_t N, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The choice of experts for each of T tokens and the order in which their
 * products take the tokens.  From logits [T, experts] (TF_F16, TF_BF16 or TF_F32,
 * rows `stride` elements apart), in fp64:
 *   score  = softmax over the experts, or sigmoid (scoring 0 or 1),
 *   choice = score + bias (fp32 [experts], or NULL);
 * with groups > 1 (experts / groups neighbours each) only the experts of the
 * top_groups best groups take part, a group's value being the largest choice in it
 * or (group_score 1) the sum of its two largest; the top_k largest choices are the
 * token's experts, in that order.  Of equal groups or choices the lower index goes
 * first.  weights = score * scale, with `renormalize` divided by the sum of the
 * token's chosen scores before (zeros where that is 0).  An expert whose logit is
 * -infinity or NaN, or whose choice is, comes after all others, with weight 0 where it
 * is chosen for want of them, and is left out of a group's sum; infinite logits share
 * the softmax.  Outputs:
 *   weights fp32 [T, top_k], chosen int32 [T, top_k],
 *   offsets int32 [experts + 1]  expert e has the slots offsets[e] .. offsets[e+1] - 1,
 *   tokens  int32 [T * top_k]    the token of each slot, ascending within an expert,
 *   places  int32 [T, top_k]     the slot of each choice.
 * groups <= 64 divides experts; top_k is at most what the top groups hold.
 */
int tf_route_experts(int dtype, const void* logits, int64_t stride, const float* bias, int64_t T, int experts,
                     int top_k, int scoring, int groups, int top_groups, int group_score, int renormalize, float scale,
                     float* weights, int32_t* chosen, int32_t* offsets, int32_t* tokens, int32_t* places,
                     void* stream);

/*
 * The experts' products: row i of C [slots, N], offsets[e] <= i < offsets[e + 1], is
 * row rows[i] (rows NULL: i) of the codes A [a_rows, K] times weight e of `packed`.
 * offsets int32 [experts + 1] and rows int32 [slots] stay on the device; an offset
 * outside 0..slots counts as the nearer end, one below an earlier one as that.  Rows
 * of C that no expert has are not written; one whose row of A is outside 0..a_rows - 1
 * is zeros, whatever the columns' scales are.  With rows, A holds less than 2^32 - 256
 * bytes.
 */
int tf_w8a8_expert_gemm(int dtype, const int8_t* A, const float* a_scales, int64_t a_rows, const void* packed,
                        const int32_t* offsets, const int32_t* rows, void* C, int64_t slots, int64_t K, int64_t N,
                        int64_t experts, void* stream);

/*
 * out[t] = add[t] + sum_j weights[t, j] * Y[places[t, j]] in fp32, rounded once:
 * Y [slots, N] contiguous, weights fp32 and places int32 [T, top_k], add [T, N] or
 * NULL.  A choice of weight 0, or whose place is outside 0..slots - 1, adds nothing,
 * whatever is in Y.  out may be add itself.  N % 8 == 0.
 */
int tf_combine_experts(int dtype, const void* Y, int64_t slots, const float* weights, const int32_t* places,
                       const void* add, int64_t T, int top_k, int64_t N, void* out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TILEFUSE_H */
