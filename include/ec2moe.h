/*
 * ec2moe.h - C ABI of libec2moe.so, the GB300 (sm_103a) MoE-layer forward of
 * EC^2MoE (arXiv 2508.06024).
 *
 * The layer computes Eq. 1, y = sum_i G(x)_i E_i(x), with the gate G of the
 * hardware-aware lightweight group gate network (Eq. 4 local candidate set,
 * Eq. 5 per-group softmax gates, Eq. 6 global group gate, Eq. 7 fusion), Top-k
 * routing (Top-1 in the paper's evaluation), and the low-rank encoder/decoder
 * of the end-cloud pipeline (Z = U^T X V at the end, X_hat = U_hat Z V_hat^T in
 * the cloud) at the split between gate/routing and the experts.
 *
 * Conventions shared by every entry point:
 *  - Device pointers are CUDA device addresses owned by the caller; the library
 *    never allocates, frees or keeps them.  Host pointers are marked "host".
 *  - Matrices are row-major and dense.  Weights are stored [out, in], i.e. the
 *    reduction axis is contiguous.  Every device pointer handed to a bf16
 *    tensor-core GEMM must be 16-byte aligned and every row a multiple of 16
 *    bytes (d, d_ff, r multiples of 8 for bf16); violations return
 *    EC2MOE_ERR_MISALIGNED before any launch.
 *  - Storage type: desc->dtype selects bf16 (EC2MOE_BF16) or fp32 (EC2MOE_F32)
 *    for activations, expert weights and codec weights.  Gate weights and
 *    biases are always fp32.  bf16 GEMMs accumulate in fp32.
 *  - All work is enqueued on `stream` (a cudaStream_t; NULL = legacy default
 *    stream).  No call synchronises except ec2moe_last_device_error.
 *  - Arguments are validated on the host before any launch; a failed check
 *    returns its status and enqueues nothing.  Kernels never trap: waits inside
 *    the tensor-core kernels are bounded and report through a device error
 *    word that ec2moe_last_device_error reads.
 *  - Calls are thread-safe with respect to each other as long as they do not
 *    share output buffers or workspaces.
 */
#ifndef EC2MOE_H
#define EC2MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* ec2moe_stream_t; /* == cudaStream_t */

typedef enum ec2moe_status {
  EC2MOE_OK = 0,
  EC2MOE_ERR_INVALID_ARG = 1,      /* NULL pointer, non-positive size, E % n_groups != 0, ... */
  EC2MOE_ERR_ALL_MASKED = 2,       /* the local candidate set of Eq. 4 is empty */
  EC2MOE_ERR_TOO_FEW_EXPERTS = 3,  /* k > number of allowed experts */
  EC2MOE_ERR_UNSUPPORTED = 4,      /* a size beyond the limits below */
  EC2MOE_ERR_CUDA = 5,             /* a CUDA runtime call failed */
  EC2MOE_ERR_TIMEOUT = 6,          /* a bounded device wait gave up (see ec2moe_last_device_error) */
  EC2MOE_ERR_WORKSPACE = 7,        /* workspace NULL or smaller than ec2moe_workspace_size */
  EC2MOE_ERR_MISALIGNED = 8        /* pointer or row pitch not 16-byte aligned */
} ec2moe_status;

typedef enum ec2moe_dtype { EC2MOE_F32 = 0, EC2MOE_BF16 = 1 } ec2moe_dtype;

/* Expert FFN activation: GELU(u) = u Phi(u) (exact erf form), or SwiGLU
 * h = SiLU(W1 x) * (W3 x). */
typedef enum ec2moe_act { EC2MOE_GELU = 0, EC2MOE_SWIGLU = 1 } ec2moe_act;

#define EC2MOE_MAX_EXPERTS 128  /* E */
#define EC2MOE_MAX_GROUPS 16    /* K, n_groups */
#define EC2MOE_MAX_TOPK 8       /* k */
#define EC2MOE_MAX_SHARED 4     /* n_shared */

/* Shape of one MoE layer call.
 *  T            tokens (rows of X), >= 0 (T = 0 is a no-op)
 *  d            d_model
 *  E            routed experts (M of Eq. 5)
 *  d_ff         hidden width of each routed expert
 *  k            experts per token (Top-k)
 *  n_groups     K of Eq. 5-7; experts form K contiguous groups of E/K (group j
 *               owns experts [j*E/K, (j+1)*E/K)).  K = 1 is the plain softmax gate.
 *  act          ec2moe_act
 *  dtype        ec2moe_dtype
 *  r            codec rank; 0 = no codec (experts see X itself)
 *  n_shared     always-on shared experts (weight 1, not masked, not counted)
 *  d_ff_shared  hidden width of each shared expert
 *  renorm_topk  0: the combine weight is g_i itself (Eq. 1 with G = g);
 *               1: g_i divided by the sum of g over the token's top-k
 *  top_groups   0: every group takes part (Eq. 5-7).  G >= 1: top-group
 *               pruning, the group gate evaluated hierarchically -- per token
 *               only the G live groups (groups with an allowed expert) with
 *               the largest p_group of Eq. 6 keep their experts (ties to the
 *               lower group index, decided on the fp32 global logits), and
 *               p_group is renormalised over them, so the weights of Eq. 7
 *               still sum to 1 over the candidates.  G at or above the number
 *               of live groups (or K = 1) prunes nothing.  k above the allowed
 *               experts of the G live groups with the fewest returns
 *               EC2MOE_ERR_TOO_FEW_EXPERTS; G < 0 EC2MOE_ERR_INVALID_ARG. */
typedef struct ec2moe_layer_desc {
  int32_t T, d, E, d_ff, k, n_groups;
  int32_t act, dtype;
  int32_t r;
  int32_t n_shared, d_ff_shared;
  int32_t renorm_topk;
  int32_t top_groups;
} ec2moe_layer_desc;

/* Weights of one layer (device pointers, NULL where absent).
 *  W_local  fp32 [E, d]  the group gates W_k of Eq. 5 stacked in group order
 *  b_local  fp32 [E]     the b_k of Eq. 5 stacked likewise
 *  W_global fp32 [K, d]  Eq. 6 (NULL iff K == 1)
 *  b_global fp32 [K]     Eq. 6 (NULL iff K == 1)
 *  W1, W3   [E, d_ff, d] up projections (W3 only for SwiGLU)
 *  W2       [E, d, d_ff] down projection
 *  W1s, W3s [n_shared, d_ff_shared, d]; W2s [n_shared, d, d_ff_shared]
 *  V_enc    [r, d]       encoder: Z = X V_enc^T (V of the codec, U = I on tokens)
 *  V_dec    [d, r]       decoder: X_hat = Z V_dec^T (V_hat, U_hat = I) */
typedef struct ec2moe_layer_weights {
  const float* W_local;
  const float* b_local;
  const float* W_global;
  const float* b_global;
  const void* W1;
  const void* W3;
  const void* W2;
  const void* W1s;
  const void* W3s;
  const void* W2s;
  const void* V_enc;
  const void* V_dec;
} ec2moe_layer_weights;

/* Bytes of device workspace ec2moe_layer_forward needs for `desc` (0 on an
 * invalid desc).  The workspace holds the codec output Z, the decoded and
 * expert-ordered activations, the expert hidden activations, per-slot expert
 * outputs, the routing tables and the prepared gate rows; for decode-sized
 * bf16 calls (T <= 256) also the fp32 partial sums of the split-d_model gate,
 * the split-K encoder and the split-K down projection.  Its contents need no
 * initialisation and are not preserved between calls. */
size_t ec2moe_workspace_size(const ec2moe_layer_desc* desc);

/* Bytes of device workspace ec2moe_experts needs (hidden activations). */
size_t ec2moe_experts_workspace_size(const ec2moe_layer_desc* desc);

/* Bytes of device workspace ec2moe_route needs (per-block histograms). */
size_t ec2moe_route_workspace_size(const ec2moe_layer_desc* desc);

/* Steps 1-3a: local expert filter, group gate and Top-k.
 * Passage: Eq. 4 (the local candidate set E_local), Eq. 5 (per-group softmax
 * gates W_k x + b_k), Eq. 6 (global group gate W_global x + b_global), Eq. 7
 * (g_i = p_group^(k) p_local,i^(k)), and the Top-k selection of the gating
 * network that Eq. 1 sums over (Top-1 in the evaluation's parameter setup).
 *  X         [T, d] activations (dtype)
 *  mask      host uint8 [E]; 1 = expert in the local candidate set of Eq. 4.
 *            An all-zero mask returns EC2MOE_ERR_ALL_MASKED and fewer than k
 *            ones EC2MOE_ERR_TOO_FEW_EXPERTS.
 *  topk_idx  out int32 [T, k] expert ids, slot 0 = largest g, ties to the
 *            lower expert index
 *  topk_w    out fp32 [T, k] combine weights (g_i, or renormalised over the
 *            top-k when desc->renorm_topk)
 * Within a group the order is decided on the fp32 local logits; across groups
 * on the fp32 fused log-probability log p_group + log p_local. */
ec2moe_status ec2moe_gate(const ec2moe_layer_desc* desc, const void* X, const float* W_local,
                          const float* b_local, const float* W_global, const float* b_global,
                          const uint8_t* mask, int32_t* topk_idx, float* topk_w,
                          ec2moe_stream_t stream);

/* Step 3b: per-expert histogram, exclusive scan and stable permutation, plus
 * the optional gather of activation rows into expert order.
 * Passage: Eq. 1, whose sum runs only over the experts Top-k selected for each
 * token (Top-1 routing in the evaluation's parameter setup): the rows routed
 * to expert i are gathered so E_i runs once over all of them.
 *  topk_idx  int32 [T, k] (from ec2moe_gate)
 *  counts    out int32 [E]     tokens routed to each expert
 *  offsets   out int32 [E + 1] exclusive prefix sum of counts
 *  perm      out int32 [T * k] perm[p] = t * k + s for the p-th row in
 *            expert-major order; rows of one expert keep increasing (t, s)
 *  inv_perm  out int32 [T * k] or NULL: inv_perm[perm[p]] = p
 *  src, dst  NULL, or src [T, width] and dst [T * k, width] (dtype):
 *            dst[p] = src[perm[p] / k]
 *  workspace device scratch of ec2moe_route_workspace_size bytes
 * topk_idx is read on the device, so its ids cannot be checked before the
 * launch: an id outside [0, E) is skipped by the kernels (not counted, no perm
 * row, inv_perm = -1, no row gathered through it) and the next
 * ec2moe_last_device_error returns EC2MOE_ERR_INVALID_ARG; counts, offsets and
 * perm then describe the valid entries only. */
ec2moe_status ec2moe_route(const ec2moe_layer_desc* desc, const int32_t* topk_idx, int32_t* counts,
                           int32_t* offsets, int32_t* perm, int32_t* inv_perm, const void* src,
                           int32_t width, void* dst, void* workspace, size_t ws_bytes,
                           ec2moe_stream_t stream);

/* ec2moe_route without a workspace argument, for callers that cannot allocate
 * device memory: programs whose device memory is planned and reserved in full
 * before they start (a serving process that hands every byte to its own pool),
 * code in a latency-critical loop that must not hit cudaMalloc's implicit
 * device synchronisation, and bindings from languages that have no device
 * allocator of their own.  The paper has no counterpart; this is a library
 * convenience.
 *
 * Same arguments, results and errors as ec2moe_route except `workspace` and
 * `ws_bytes`.  The routing histograms live in a fixed 64 KiB device array
 * inside the library (EC2MOE_ROUTE_NOALLOC_MAX_CELLS int32 cells, one per
 * block of 1024 (token, slot) entries and expert), which every GPU that loads
 * the library holds until the process exits.  Sizes with
 * ceil(T * k / 1024) * E > EC2MOE_ROUTE_NOALLOC_MAX_CELLS (for E = 64: T * k >
 * 262144) return EC2MOE_ERR_UNSUPPORTED before any launch.  Nothing is
 * allocated or freed, by this call or by anything it calls.
 *
 * The first call on each device looks up the array's device address (with
 * that device current) and caches it, keyed on the device's current context;
 * make that first call before any stream capture.  After a cudaDeviceReset the
 * next call looks the address up again in the new context (so it, too, should
 * come before any capture), and the array's contents are gone.  All calls on a device share the array: every cell a call reads is
 * written earlier by the same call, but calls whose kernels overlap on the GPU
 * (different streams, or different host threads) race on it and must be
 * serialised by the caller. */
#define EC2MOE_ROUTE_NOALLOC_MAX_CELLS 16384
ec2moe_status ec2moe_route_noalloc(const ec2moe_layer_desc* desc, const int32_t* topk_idx, int32_t* counts,
                                   int32_t* offsets, int32_t* perm, int32_t* inv_perm, const void* src,
                                   int32_t width, void* dst, ec2moe_stream_t stream);

/* Steps 4-5a: routed expert FFNs on expert-ordered rows with the gate scale and
 * the unpermute fused into the down projection.
 * Passage: Eq. 1, each term G(x)_i E_i(x) with E_i a feed-forward expert
 * network (Preliminary, Mixture-of-Experts).
 *  X_perm    [T * k, d] rows in expert order (ec2moe_route's dst)
 *  offsets   int32 [E + 1] device (ec2moe_route)
 *  perm      int32 [T * k] device (ec2moe_route)
 *  topk_w    fp32 [T, k] (ec2moe_gate)
 *  slot_out  out [T * k, d]: slot_out[t * k + s] = topk_w[t, s] * E_e(x_t)
 *            for e = topk_idx[t, s]
 *  workspace ec2moe_experts_workspace_size bytes
 * offsets and perm are read on the device: a group whose range is not inside
 * [0, T * k] (or is decreasing) and a perm entry outside [0, T * k) are
 * skipped, with nothing written for them, and ec2moe_last_device_error then
 * reports EC2MOE_ERR_INVALID_ARG. */
ec2moe_status ec2moe_experts(const ec2moe_layer_desc* desc, const void* X_perm, const int32_t* offsets,
                             const void* W1, const void* W3, const void* W2, const float* topk_w,
                             const int32_t* perm, void* slot_out, void* workspace, size_t ws_bytes,
                             ec2moe_stream_t stream);

/* Always-on shared experts on every token: shared_out[s * T + t] = E_s(x_t).
 * Passage: Eq. 1's expert FFN E_i applied with weight 1 to every token; the
 * paper has no shared experts, the fine-grained layer shape adds them.
 *  X [T, d]; W1s/W3s/W2s as in ec2moe_layer_weights; shared_out out
 *  [n_shared * T, d]; workspace of ec2moe_experts_workspace_size bytes. */
ec2moe_status ec2moe_shared_experts(const ec2moe_layer_desc* desc, const void* X, const void* W1s,
                                    const void* W3s, const void* W2s, void* shared_out, void* workspace,
                                    size_t ws_bytes, ec2moe_stream_t stream);

/* Step 5b: y[t] = sum_s slot_out[t * k + s] + sum_j shared_out[j * T + t], in
 * that fixed order with an fp32 sum.  shared_out may be NULL.
 * Passage: Eq. 1, the sum over the selected experts of G(x)_i E_i(x). */
ec2moe_status ec2moe_combine(const ec2moe_layer_desc* desc, const void* slot_out, const void* shared_out,
                             void* Y, ec2moe_stream_t stream);

/* Step 6, end side: Z = X V_enc^T ([T, d] x [r, d]^T -> [T, r]).
 * Passage: the low-rank encoder of PO-ECC (Encoder-Decoder based on Low-Rank
 * Compression): Z = U^T X V, here with U = I on the token axis and
 * V = V_enc^T. */
ec2moe_status ec2moe_lr_encode(const ec2moe_layer_desc* desc, const void* X, const void* V_enc, void* Z,
                               ec2moe_stream_t stream);

/* Step 6, cloud side: X_hat = Z V_dec^T ([T, r] x [d, r]^T -> [T, d]).
 * Passage: the decoder of the same section, X_hat = U_hat Z V_hat^T, with
 * U_hat = I and V_hat = V_dec. */
ec2moe_status ec2moe_lr_decode(const ec2moe_layer_desc* desc, const void* Z, const void* V_dec,
                               void* X_hat, ec2moe_stream_t stream);

/* The fused layer: gate and routing on X, encode, decode into expert order,
 * routed and shared experts, combine.
 * Passage: Eq. 1 with the gate of Eq. 4-7 (HL-GGN) and the low-rank
 * encoder/decoder of PO-ECC at the end-cloud split between the gate and the
 * experts.
 *  Y         out [T, d] (dtype)
 *  topk_idx  out int32 [T, k]; topk_w out fp32 [T, k]; counts out int32 [E]
 *  Z         out [T, r] or NULL: the transmitted (encoded) activations
 *  workspace ec2moe_workspace_size(desc) bytes */
ec2moe_status ec2moe_layer_forward(const ec2moe_layer_desc* desc, const ec2moe_layer_weights* w,
                                   const void* X, const uint8_t* mask, void* Y, int32_t* topk_idx,
                                   float* topk_w, int32_t* counts, void* Z, void* workspace,
                                   size_t ws_bytes, ec2moe_stream_t stream);

/* Synchronises `stream`, then reads and clears the device error words of the
 * current device: EC2MOE_OK; EC2MOE_ERR_TIMEOUT when a bounded wait in a
 * tensor-core kernel gave up; EC2MOE_ERR_INVALID_ARG when a routing kernel met
 * (and skipped) an expert id outside [0, E) in a caller's topk_idx, or a
 * grouped expert GEMM met (and skipped) a group range in `offsets` outside
 * [0, T * k] or a destination in `perm` outside [0, T * k), or one of the 8-bit
 * and balance entry points an entry that its description names;
 * EC2MOE_ERR_CUDA
 * when the stream reports an error.  A timeout takes precedence. */
ec2moe_status ec2moe_last_device_error(ec2moe_stream_t stream);

/* Budget, in SM clock cycles, of every bounded wait inside the tensor-core
 * kernels of later calls (process-wide; default 4e9, about two seconds).  A
 * wait that runs out makes its CTA stop, wait (with a fixed one-second
 * budget) for the copies and MMAs it started, free its tensor memory and
 * return; ec2moe_last_device_error then reports EC2MOE_ERR_TIMEOUT and the
 * context stays usable.  With a budget of 0 a wait gives up when the hardware's
 * own try (which may suspend for a few microseconds) finds it unsatisfied, and
 * the fp32 GEMM's and the grouped products' waits for their accumulators, those of
 * the 8-bit products and the gate logits for their operands and the norm's for its rows at once; that is how failure handling is
 * exercised without a real fault.  Negative values return
 * EC2MOE_ERR_INVALID_ARG. */
ec2moe_status ec2moe_set_wait_budget(int64_t cycles);
int64_t ec2moe_get_wait_budget(void);

/* ---------------------------------------------------------------------------
 * The end/cloud pipeline of the paper's pipeline optimisation (PO-ECC: the end
 * runs the gate and the low-rank encoder, the cloud the decoder and the
 * experts, overlapped across requests), on one GPU with two CUDA streams.
 *
 * Same result as ec2moe_layer_forward, computed in n_micro contiguous
 * micro-batches of ceil(T / n_micro) tokens: stream_end runs the gate, the
 * routing and the encoder Z = X V_enc^T of micro-batch i + 1 while
 * stream_cloud runs the decoder (rows straight into expert order), the
 * experts, the shared experts and the combine of micro-batch i.  The
 * micro-batch's Z and routing tables are handed from the end to the cloud
 * through a CUDA event; counts is the sum of the micro-batches' histograms.
 * Y, topk_idx, topk_w and Z (optional) receive every token's rows in token
 * order, as for ec2moe_layer_forward; the order of rows inside each expert
 * (not an output) follows the micro-batches.
 *
 * Streams: stream_cloud first waits for everything enqueued on stream_end
 * before the call, and at the end stream_end waits for stream_cloud, so the
 * call as a whole is ordered on stream_end (synchronise or capture on
 * stream_end; stream_cloud is forked and joined inside the call).  Passing the
 * same stream twice runs the micro-batches back to back.
 *
 * workspace: ec2moe_pipelined_workspace_size(desc, n_micro) bytes, 16-byte
 * aligned; one region per micro-batch, so calls that overlap on the GPU must
 * not share it.  1 <= n_micro <= EC2MOE_MAX_MICRO (else
 * EC2MOE_ERR_INVALID_ARG); micro-batches beyond T tokens are empty and
 * skipped.  Other errors as ec2moe_layer_forward. */
#define EC2MOE_MAX_MICRO 64
size_t ec2moe_pipelined_workspace_size(const ec2moe_layer_desc* desc, int32_t n_micro);
ec2moe_status ec2moe_layer_forward_pipelined(const ec2moe_layer_desc* desc, const ec2moe_layer_weights* w,
                                             const void* X, const uint8_t* mask, void* Y, int32_t* topk_idx,
                                             float* topk_w, int32_t* counts, void* Z, void* workspace,
                                             size_t ws_bytes, int32_t n_micro, ec2moe_stream_t stream_end,
                                             ec2moe_stream_t stream_cloud);

/* ---------------------------------------------------------------------------
 * Experts in 8-bit floating point.  Values are e4m3 (1 sign, 4 exponent, 3
 * mantissa bits, largest 448, no infinities), one byte each, with one fp32 scale
 * for each block of EC2MOE_FP8_BLOCK columns: a stored value q stands for q times
 * its block's scale.  Activations have a scale per row and block
 * ([rows, ceil(cols / 128)]), weights one per 128 x 128 block
 * ([mats, ceil(rows / 128), ceil(cols / 128)]).  Scales need not be those of
 * ec2moe_fp8_quantize, but a row's scale and a weight block's are multiplied with each
 * other in fp32 before a block's sum is multiplied by them: where that product overflows
 * the result is an infinity or NaN (also of a sum of 0), where it is below 2^-126 it has
 * lost bits, even if the result itself would be an ordinary number.  (Quantised data
 * gets there when the largest magnitudes of a row's block and of a weight block multiply
 * to more than 2^145 or less than 2^-108.)  Rows are dense and multiples of 16 bytes
 * (cols, d, d_ff multiples of 16; others return EC2MOE_ERR_MISALIGNED); a last
 * block may be narrower than 128.  The paper has no counterpart: its experts
 * (Eq. 1) are computed from rounded inputs here, with fp32 sums. */
#define EC2MOE_FP8_BLOCK 128

/* X (dtype; rows of pitch ld >= cols elements) to e4m3 Q (dense) and its scales:
 *   a = max(2^-96, max |x| over the block), scale = a / 448, q = e4m3(x * (448 / a))
 * rounded to nearest, ties to even.  A NaN becomes e4m3's NaN and does not count
 * for its block's scale; an infinity makes its block's scale infinite.
 *  n_mats, rows  matrices of `rows` rows each, one behind the other in X and Q
 *  block_rows    1: a scale per row and 128 columns; 128: per 128 x 128 block,
 *                blocks starting anew in each matrix
 *  inv_perm, k   NULL and 0, or (block_rows = 1, n_mats = 1) device int32
 *                [rows, k] of ec2moe_route, 1 <= k <= EC2MOE_MAX_TOPK: row t is
 *                written to the rows inv_perm[t * k + s], s < k, of Q
 *                [rows * k, cols] and scale.  An entry of -1 is skipped; another
 *                one outside [0, rows * k) too, and ec2moe_last_device_error then
 *                reports EC2MOE_ERR_INVALID_ARG.
 * No rows is a no-op. */
ec2moe_status ec2moe_fp8_quantize(int32_t dtype, int32_t n_mats, int32_t rows, int32_t cols, int64_t ld,
                                  const void* X, int32_t block_rows, const int32_t* inv_perm, int32_t k, void* Q,
                                  float* scale, ec2moe_stream_t stream);

/* Bytes of device workspace ec2moe_fp8_gemm needs on the current device (0: none,
 * or an invalid size): partial sums of calls with few rows per group. */
size_t ec2moe_fp8_gemm_workspace_size(int32_t n_groups, int32_t rows, int32_t N, int32_t K);

/* C_g = A_g B_g^T of 8-bit operands: group g owns the rows [offsets[g],
 * offsets[g + 1]) of A [rows, K] and of C, and the weights B[g] [N, K].
 *  A_scale   fp32 [rows, ceil(K / 128)]
 *  offsets   device int32 [n_groups + 1], or NULL with n_groups = 1: all rows
 *  B_scale   fp32 [n_groups, ceil(N / 128), ceil(K / 128)]
 *  out_dtype EC2MOE_BF16 or EC2MOE_F32: type of C, rows of pitch ldc >= N
 *            elements (a multiple of 16 bytes)
 * Every block's products are summed in fp32 and the scaled sums of the blocks
 * added in fp32, rounded once to the output.  Rows of no group are not written; a
 * group whose range is not inside [0, rows], or which starts before the end of a group
 * before it, is skipped and ec2moe_last_device_error then reports
 * EC2MOE_ERR_INVALID_ARG.  No rows is a no-op; more than 2^31 - 256 of them
 * return EC2MOE_ERR_UNSUPPORTED. */
ec2moe_status ec2moe_fp8_gemm(int32_t n_groups, int32_t rows, int32_t N, int32_t K, const void* A,
                              const float* A_scale, const int32_t* offsets, const void* B, const float* B_scale,
                              int32_t out_dtype, void* C, int64_t ldc, void* workspace, size_t ws_bytes,
                              ec2moe_stream_t stream);

/* Expert weights in e4m3 with 128 x 128 scales, shapes as in ec2moe_layer_weights
 * (W3, S3 NULL for GELU): W1, W3 [E, d_ff, d], S1, S3 [E, ceil(d_ff / 128),
 * ceil(d / 128)]; W2 [E, d, d_ff], S2 [E, ceil(d / 128), ceil(d_ff / 128)]. */
typedef struct ec2moe_fp8_weights {
  const void* W1;
  const float* S1;
  const void* W3;
  const float* S3;
  const void* W2;
  const float* S2;
} ec2moe_fp8_weights;

/* Bytes of device workspace ec2moe_experts_fp8 needs on the current device (hidden
 * rows and their scales; partial sums where an expert's rows are few). */
size_t ec2moe_experts_fp8_workspace_size(const ec2moe_layer_desc* desc);

/* ec2moe_experts on 8-bit rows and weights.
 * Passage: Eq. 1, each term G(x)_i E_i(x).
 *  Xq, Xs    e4m3 [T * k, d] rows in expert order and their scales
 *            (ec2moe_fp8_quantize with the inv_perm of ec2moe_route)
 *  slot_out  out [T * k, d] in desc->dtype: slot_out[t * k + s] =
 *            topk_w[t, s] * E_e(x_t) for e = topk_idx[t, s]
 * The hidden rows are the activation of the fp32 sums (GELU to within 1e-6 |u|, SiLU to
 * within 1e-6 of itself for |u| <= 16), quantised like ec2moe_fp8_quantize's rows.  A sum
 * within its rounding error of a tie of that quantisation falls to either side, which
 * moves the hidden value by up to 2^-4 of it: an fp32 slot_out agrees with the same
 * formula in 64 bits to 1e-7 of its norm where none does, to about 3e-4 where some do.  offsets, perm, topk_w and what happens to entries
 * out of range as for ec2moe_experts; an expert whose rows start before the end of an
 * earlier one's is skipped and reported too. */
ec2moe_status ec2moe_experts_fp8(const ec2moe_layer_desc* desc, const void* Xq, const float* Xs,
                                 const int32_t* offsets, const ec2moe_fp8_weights* w, const float* topk_w,
                                 const int32_t* perm, void* slot_out, void* workspace, size_t ws_bytes,
                                 ec2moe_stream_t stream);

/* ---------------------------------------------------------------------------
 * Balance of the gate. */

/* Bytes of device workspace ec2moe_gate_logits needs (0 on an invalid desc). */
size_t ec2moe_gate_logits_workspace_size(const ec2moe_layer_desc* desc);

/* The gate's logits to fp32 accuracy: logits[t] = (W_local x_t + b_local,
 * W_global x_t + b_global), fp32 [T, E + K] (K = n_groups; [T, E] when it is 1).
 * Passage: Eq. 5 and Eq. 6 before their softmaxes.  Infinities and NaN in x_t, the gate
 * rows and the biases give what the definition gives; they reach the logits of their own
 * token or gate row alone. */
ec2moe_status ec2moe_gate_logits(const ec2moe_layer_desc* desc, const void* X, const float* W_local,
                                 const float* b_local, const float* W_global, const float* b_global, float* logits,
                                 void* workspace, size_t ws_bytes, ec2moe_stream_t stream);

/* Bytes of device workspace ec2moe_balance_loss needs (0 on an invalid desc or n_seg).
 * 1 <= n_seg <= 2^30, n_seg * E < 2^31. */
size_t ec2moe_balance_loss_workspace_size(const ec2moe_layer_desc* desc, int32_t n_seg);

/* Per-expert counts, the balance loss of the gate and its gradients.
 * With n_s the tokens of segment s that count, c_si the entries of their topk_idx
 * that name expert i, A the number of allowed experts, S' the number of segments
 * with n_s > 0 and g the gate's probabilities (Eq. 5-7 under mask and
 * desc->top_groups):
 *   f_si = c_si / (k n_s),  P_si = (1 / n_s) sum_t g_i(t),
 *   loss = coef / S' sum_s A sum_i f_si P_si
 * (coef when the experts are used evenly; 0 without such a segment).  The counts
 * are constants of the gradient.  The paper has no counterpart: it is the loss
 * that trains a gate of Eq. 5-7 towards even loads under a device's mask.
 *  logits      fp32 [T, E + K] of pitch ld >= E + K (ec2moe_gate_logits); those of
 *              masked experts and of groups without an allowed one are not used
 *  mask        host uint8 [E], as for ec2moe_gate
 *  topk_idx    int32 [T, k] (ec2moe_gate)
 *  valid       device uint8 [T]: 0 = a token that does not count (padding); NULL:
 *              all do
 *  seg_offsets device int32 [n_seg + 1], not decreasing, within [0, T]: segment s
 *              is the tokens [seg_offsets[s], seg_offsets[s + 1]), possibly none;
 *              tokens of no segment do not count.  NULL with n_seg = 1: all tokens
 *  d_loss      device fp32 scalar, the gradient that arrives at the loss (NULL: 1)
 *  loss        out fp32 scalar
 *  counts      out int32 [n_seg, E]: c_si
 *  d_logits    out fp32 [T, E + K] dense, or NULL: d_loss times the gradient; 0 for
 *              what is masked, pruned or does not count
 *  d_bias      out fp32 [E + K] or NULL: the gradient in (b_local, b_global), the
 *              sum of d_logits over the tokens.  The gate rows' gradients are the
 *              products d_logits^T X, the activations' d_logits (W_local; W_global).
 * The sums are in a fixed order: the same inputs give the same bits.  An id of
 * topk_idx outside [0, E) is skipped (not counted) and a segment bound outside
 * [0, T] or decreasing cuts no token that other bounds do not hold;
 * ec2moe_last_device_error then reports EC2MOE_ERR_INVALID_ARG.  With T = 0 loss,
 * counts and d_bias are 0. */
ec2moe_status ec2moe_balance_loss(const ec2moe_layer_desc* desc, const float* logits, int64_t ld,
                                  const uint8_t* mask, const int32_t* topk_idx, const uint8_t* valid,
                                  const int32_t* seg_offsets, int32_t n_seg, float coef, const float* d_loss,
                                  float* loss, int32_t* counts, float* d_logits, float* d_bias, void* workspace,
                                  size_t ws_bytes, ec2moe_stream_t stream);

/* ---------------------------------------------------------------------------
 * The norm in front of a layer and what its experts are trained with.  The paper
 * is about inference and has no counterpart of these; they are the formulas given
 * here. */

/* The residual's addition and the root-mean-square norm of the sum, row by row:
 *   h = x + residual,  rstd = 1 / sqrt(mean h^2 + eps),  y = h * rstd * weight
 * in fp32; y is taken from the sum before it is rounded to H's type.
 *  dtype, y_dtype  ec2moe_dtype of X, residual and H; of Y
 *  X, residual     [rows, cols], rows of pitch ld >= cols elements (a multiple of 16
 *                  bytes); residual NULL: none
 *  weight          fp32 [cols], or NULL: ones
 *  eps             finite, >= 0
 *  H               out, dense, or NULL: h; may be X or residual itself where ld = cols
 *  rstd            out fp32 [rows], or NULL (ec2moe_rmsnorm_backward needs it)
 *  Y               out, dense, or NULL
 *  Q, scale        out, or both NULL: y in 8 bits as ec2moe_fp8_quantize stores rows
 *                  (block_rows = 1), rounded once, from y itself: e4m3 [rows, cols],
 *                  dense, and fp32 [rows, ceil(cols / 128)]; what ec2moe_fp8_gemm and
 *                  ec2moe_experts_fp8 take
 * One output at least.  cols is a multiple of 8 (with Q of 16), at most 16384 (more
 * return EC2MOE_ERR_UNSUPPORTED).  The squares are summed in fp32: where that sum
 * overflows y is 0, as it is for a row with an infinity, whose infinite elements become NaN;
 * a NaN makes its row NaN.  Squares below 2^-150 count as 0: with eps = 0 a row of zeros
 * is NaN, and one of such values infinite.  Q is rounded from the exact quotient where a
 * block's largest |h * weight| is between 2^-80 and 2^100, else from y in fp32.  No rows is
 * a no-op. */
ec2moe_status ec2moe_rmsnorm(int32_t dtype, int32_t y_dtype, int32_t rows, int32_t cols, int64_t ld, const void* X,
                             const void* residual, const float* weight, float eps, void* H, float* rstd, void* Y,
                             void* Q, float* scale, ec2moe_stream_t stream);

/* Bytes of device workspace ec2moe_rmsnorm_backward needs for d_weight on the current
 * device (0: none, or an invalid size). */
size_t ec2moe_rmsnorm_backward_workspace_size(int32_t rows, int32_t cols);

/* The gradient of ec2moe_rmsnorm.  With g = dY * weight and xhat = H * rstd:
 *   dX = rstd * (g - xhat * mean(g * xhat)) + dH,  d_weight = sum over rows of dY * xhat
 *  dY        y_dtype [rows, cols] of pitch ld >= cols elements
 *  H, rstd   dense, as ec2moe_rmsnorm wrote them (without a residual H is its X)
 *  dH        dtype, dense, or NULL: the gradient that arrives at H itself (the residual
 *            stream behind the norm)
 *  dX        out, dtype, dense: the gradient of X and of residual; may be dH, H or (of
 *            the same type, ld = cols) dY itself
 *  d_weight  out fp32 [cols], or NULL (no workspace then); accumulate 1: it is added to
 * The sums are in a fixed order: the same inputs give the same bits.  No rows: d_weight
 * is 0 (accumulate: as it was). */
ec2moe_status ec2moe_rmsnorm_backward(int32_t dtype, int32_t y_dtype, int32_t rows, int32_t cols, int64_t ld,
                                      const void* dY, const void* H, const float* rstd, const float* weight,
                                      const void* dH, void* dX, float* d_weight, int32_t accumulate, void* workspace,
                                      size_t ws_bytes, ec2moe_stream_t stream);

/* The experts' activation of rows in expert order, with each row's gate weight:
 *   H[p] = row_scale[perm[p]] * a[p],  a = SiLU(U) * V  or  GELU(U)  (exact erf form)
 *  U, V       [rows, cols] (dtype), both of pitch ld >= cols elements, so that they may be
 *             the halves of one matrix (rows of W1 and W3 joined); V for EC2MOE_SWIGLU
 *  perm       device int32 [rows] (ec2moe_route), or NULL: perm[p] = p
 *  row_scale  fp32 [rows] (topk_w of ec2moe_gate), or NULL: 1
 *  H          out [rows, cols], dense
 * (Eq. 1's factor G(x)_i, applied before the linear down projection instead of behind
 * it.)  cols is a multiple of 8, at most 2^31 - 2049 (more return
 * EC2MOE_ERR_UNSUPPORTED).  A perm entry outside [0, rows) leaves its row as it
 * was and ec2moe_last_device_error then reports EC2MOE_ERR_INVALID_ARG.  No rows is a
 * no-op.
 * Accuracy of fp32 rows: SwiGLU within 10 2^-24 of itself where e^-U is finite (U > -88;
 * 0 below), its derivative in U within 18 2^-24 of |V| (1 + |U|) / (1 + e^-U); GELU within
 * 2.5e-7 and 2^-23 of itself, its derivative within 7e-7: absolute bounds, which leave few
 * digits of values below U = -4.  bf16 rows have SwiGLU within 2e-6 of itself for |U| <= 12
 * (fast exponentials) before it is rounded, and the same GELU. */
ec2moe_status ec2moe_activation(int32_t dtype, int32_t act, int32_t rows, int32_t cols, int64_t ld, const void* U,
                                const void* V, const int32_t* perm, const float* row_scale, void* H,
                                ec2moe_stream_t stream);

/* Its gradient, with s = row_scale[perm[p]]:
 *   dU = s dH da/dU,  dV = s dH SiLU(U),  d_row_scale[perm[p]] = sum over columns of dH * a
 *  dH           [rows, cols], dense
 *  dU, dV       out, pitch ld; may be U and V themselves
 *  H            out, dense, or NULL: the forward's H again (the weights' gradient needs
 *               it); may be dH itself
 *  d_row_scale  out fp32 [rows], or NULL
 * Rows with a perm entry out of range are skipped and reported as above; the others' entries
 * differ (two rows of one slot would both write its d_row_scale). */
ec2moe_status ec2moe_activation_backward(int32_t dtype, int32_t act, int32_t rows, int32_t cols, int64_t ld,
                                         const void* U, const void* V, const int32_t* perm, const float* row_scale,
                                         const void* dH, void* dU, void* dV, void* H, float* d_row_scale,
                                         ec2moe_stream_t stream);

/* Bytes of device workspace that any of the three products below needs on the current
 * device (0: none, or an invalid size): partial results of sums that are cut into ranges
 * where a call has few tiles. */
size_t ec2moe_grouped_gemm_workspace_size(int32_t n_groups, int32_t rows, int32_t N, int32_t K);

/* Products grouped by expert of bf16 operands, group g owning the rows [offsets[g],
 * offsets[g + 1]) of the row matrices and the weights B[g] [N, K] (dense):
 *   ec2moe_grouped_gemm        C_g  = A_g B_g^T     A [rows, K]   -> C [rows, N]
 *   ec2moe_grouped_gemm_dgrad  dA_g = dC_g B_g      dC [rows, N]  -> dA [rows, K]
 *   ec2moe_grouped_gemm_wgrad  dB_g = dC_g^T A_g    dC, A         -> dB [n_groups, N, K]
 *  offsets     device int32 [n_groups + 1], or NULL with n_groups = 1: all rows
 *  lda, lddc   row pitches in elements (multiples of 8)
 *  perm        device int32 [rows] or NULL: row p of the result is written to row perm[p]
 *              of C or dA (the token's slot: ec2moe_combine then adds them up); the
 *              destinations of different rows differ
 *  out_dtype   EC2MOE_BF16 or EC2MOE_F32: type of the result, rows of pitch ldc or ldda
 *              elements (a multiple of 16 bytes); dB is dense
 *  accumulate  1: dB is added to (EC2MOE_F32 only)
 * N and K are multiples of 8.  Sums are in fp32, rounded once to the result; the same
 * inputs give the same bits.  Rows of no group are not written and take no part, whatever
 * they hold; a group without rows has dB = 0 (accumulate: as it was).  A group whose
 * range is not inside [0, rows], or which starts before the end of a group before it,
 * counts as one without rows, and a destination outside [0, rows) is skipped;
 * ec2moe_last_device_error then reports EC2MOE_ERR_INVALID_ARG. */
ec2moe_status ec2moe_grouped_gemm(int32_t n_groups, int32_t rows, int32_t N, int32_t K, const void* A, int64_t lda,
                                  const int32_t* offsets, const void* B, const int32_t* perm, int32_t out_dtype, void* C,
                                  int64_t ldc, void* workspace, size_t ws_bytes, ec2moe_stream_t stream);
ec2moe_status ec2moe_grouped_gemm_dgrad(int32_t n_groups, int32_t rows, int32_t N, int32_t K, const void* dC, int64_t lddc,
                                        const int32_t* offsets, const void* B, const int32_t* perm, int32_t out_dtype,
                                        void* dA, int64_t ldda, void* workspace, size_t ws_bytes,
                                        ec2moe_stream_t stream);
ec2moe_status ec2moe_grouped_gemm_wgrad(int32_t n_groups, int32_t rows, int32_t N, int32_t K, const void* dC, int64_t lddc,
                                        const void* A, int64_t lda, const int32_t* offsets, int32_t out_dtype,
                                        int32_t accumulate, void* dB, void* workspace, size_t ws_bytes,
                                        ec2moe_stream_t stream);

/* Number of kernels the last successful call on this host thread enqueued. */
int32_t ec2moe_last_launch_count(void);

/* Per-launch timing.  While enabled, every kernel the library enqueues is
 * bracketed by a pair of CUDA events recorded on its stream; records
 * accumulate until ec2moe_profile_reset.  Reading a record synchronises on its
 * stop event.  `name` receives a static string naming the launch
 * ("gate_prep", "gate_topk", "gate_decide", "route_count", "route_scatter", "gather_rows",
 * "lr_encode", "lr_reduce", "lr_decode", "lr_codec", "expert_up", "expert_down", "shared_up",
 * "shared_down", "ffn_up", "ffn_down" (routed and shared experts in one launch),
 * "combine", "sum_counts", "quantize_rows", "quantize_blocks", "fp8_gemm", "fp8_up",
 * "fp8_down", "fp8_sum", "logits_prep", "logits_gemm", "logits_sum", "balance",
 * "balance_clear", "balance_count", "balance_main", "balance_final", "rmsnorm",
 * "rmsnorm_backward", "rmsnorm_dweight", "activation", "activation_backward",
 * "grouped_gemm", "grouped_dgrad", "grouped_wgrad", "grouped_join"); `ms` its device
 * duration.  Profiling is off by default and costs nothing when off. */
ec2moe_status ec2moe_profile_enable(int32_t enable);
/* Restricts profiling to one launch per call: with launch_index >= 0 only the
 * kernel that is the launch_index-th launch (0-based) of each later call is
 * bracketed, so its neighbours run without event records between them (which
 * would otherwise end the programmatic overlap of every launch with its
 * predecessor and add the records' own cost to every measured kernel);
 * -1 (the default) brackets every launch.  Values below -1 return
 * EC2MOE_ERR_INVALID_ARG. */
ec2moe_status ec2moe_profile_only(int32_t launch_index);
int32_t ec2moe_profile_count(void);
ec2moe_status ec2moe_profile_read(int32_t i, const char** name, float* ms);
void ec2moe_profile_reset(void);

/* ---------------------------------------------------------------------------
 * Route-aware heuristic pipeline scheduler (Eq. 9-11 of the paper's pipeline
 * optimisation).  Host code only: no device memory, no CUDA call, no stream.
 * Every pointer below is a host pointer.
 *
 * ec2moe_schedule places n tasks, task i with computational complexity
 * cost[i] = C(t_i) >= 0 and communication cost comm[i] = Comm(t_i) >= 0, on
 * the End (location[i] = EC2MOE_END) or the Cloud (EC2MOE_CLOUD):
 *   Eq. 10  P(t_i) = C(t_i) / (Comm(t_i) + eps)
 *   Eq. 11  End if Load_end + C(t_i) <= T_end and P(t_i) >= beta, else Cloud,
 * visiting the tasks in decreasing priority (ties to the lower index) and
 * adding C(t_i) to Load_end (starting at load_end) for each End task and to
 * Load_cloud (starting at load_cloud; reported only, Eq. 11 does not use it)
 * for each Cloud task.  order[j] receives the j-th visited task (may be NULL);
 * *load_end_out and *load_cloud_out the final loads (may be NULL).
 * Errors: EC2MOE_ERR_INVALID_ARG for n < 0, NULL cost/comm/location when
 * n > 0, a negative or NaN cost or comm, eps < 0 or NaN, or comm[i] + eps == 0
 * for some i.  T_end and beta may be +/-infinity. */
#define EC2MOE_END 0
#define EC2MOE_CLOUD 1
ec2moe_status ec2moe_schedule(int32_t n, const double* cost, const double* comm, double load_end,
                              double load_cloud, double T_end, double beta, double eps, int32_t* location,
                              int32_t* order, double* load_end_out, double* load_cloud_out);

/* Eq. 9, the heuristic's objective for a placement:
 *   sum_i alpha * ExecTime(t_i) + (1 - alpha) * Comm(t_i),
 * with ExecTime(t_i) = cost[i] / rate_end on the End and cost[i] / rate_cloud
 * on the Cloud, and Comm(t_i) paid by Cloud tasks only (a task run on the End
 * transmits nothing).  Sums in task order.  Errors: EC2MOE_ERR_INVALID_ARG for
 * n < 0, NULL arrays when n > 0, rates <= 0, a location other than
 * EC2MOE_END / EC2MOE_CLOUD, or NULL `objective`. */
ec2moe_status ec2moe_schedule_objective(int32_t n, const double* cost, const double* comm,
                                        const int32_t* location, double rate_end, double rate_cloud,
                                        double alpha, double* objective);

/* Route-aware tasks from a layer's routing histogram (counts, host copy of
 * the [E] output of ec2moe_route / ec2moe_layer_forward): one task per expert
 * with rows, in expert order.  expert_of_task[j] is the expert of task j,
 * cost[j] = 2 * rows * d * d_ff * (3 projections for SwiGLU, 2 for GELU) its
 * FFN flops, comm[j] = rows * (w_in + d) * bytes its transfer in bytes if it
 * runs in the Cloud (w_in = r encoded values per row, or d without a codec;
 * plus the d-wide output row; bytes = 2 for bf16, 4 for fp32).  All output
 * arrays hold desc->E entries; *n_tasks receives the task count.  Errors:
 * EC2MOE_ERR_INVALID_ARG for NULL pointers, an invalid desc, or a negative
 * count. */
ec2moe_status ec2moe_expert_tasks(const ec2moe_layer_desc* desc, const int32_t* counts, int32_t* expert_of_task,
                                  double* cost, double* comm, int32_t* n_tasks);

/* Human-readable name of a status code (static storage). */
const char* ec2moe_status_string(ec2moe_status status);

#ifdef __cplusplus
}
#endif

#endif /* EC2MOE_H */
