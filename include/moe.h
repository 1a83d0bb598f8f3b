/*
 * moe.h - C ABI of libmoe: one GPU's share of an expert-parallel MoE layer on
 * AMD Instinct MI355X (gfx950).
 *
 * ViBE (arXiv 2606.00735) balances per-GPU execution time of expert-parallel
 * MoE layers. What it balances is the work of this library: each GPU gates its
 * tokens, builds the per-expert token histogram (one row of the activation
 * matrix W, Section 4.2.2), runs its local experts on the tokens routed to them
 * (its token load n_g = sum of w_e over its experts S_g, Section 4.2.3) and
 * combines the results; the latency of that expert computation as a function
 * of the token load is the per-GPU performance model f_g(n) (Section 4.2.1,
 * Algorithm 1 Phase 1).
 *
 * Conventions shared by every entry point:
 *  - Array arguments are caller-owned DEVICE pointers unless marked "host".
 *    The library allocates no device memory and keeps no device state.
 *  - Matrices are row-major and dense. Weight matrices are stored
 *    out-features by in-features (the nn.Linear layout): row n of a matrix
 *    holds the input weights of output n, so every contraction reads its
 *    operands along contiguous rows.
 *  - bf16 data is IEEE bfloat16 (2 bytes); MOE_F32 data is IEEE binary32.
 *    Gate logits and weights are always fp32.
 *  - Calls are stream-ordered and asynchronous (except moe_load_sweep) and
 *    launch only on `stream`. Pointers must be 16-byte aligned.
 *  - Workspace: call with ws == NULL to receive the byte count in *ws_bytes
 *    (returns MOE_OK, launches nothing). With ws != NULL, *ws_bytes must be at
 *    least that count, else MOE_ERR_WORKSPACE.
 *  - Errors: every call returns a moe_status and never aborts. Arguments are
 *    validated on the host before anything is launched; launch failures are
 *    reported as MOE_ERR_HIP (hipGetLastError after each launch). Device
 *    data the host cannot see (ids, offsets, dest) is clamped inside the
 *    kernels so that no access leaves its buffer.
 *  - Thread safety: calls with distinct workspaces and streams are
 *    independent.
 */
#ifndef MOE_SHARD_MOE_H
#define MOE_SHARD_MOE_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define MOE_ABI_VERSION 3
#define MOE_MAX_EXPERTS 256 /* E and E_local limit */
#define MOE_MAX_TOPK 16

typedef enum moe_status {
  MOE_OK = 0,
  MOE_ERR_INVALID_ARG = 1, /* NULL pointer, negative size, k > E, misaligned */
  MOE_ERR_UNSUPPORTED = 2, /* valid but outside what the kernels handle */
  MOE_ERR_WORKSPACE = 3,   /* workspace smaller than the queried size */
  MOE_ERR_HIP = 4          /* a HIP launch or runtime call failed */
} moe_status;

typedef enum moe_dtype { MOE_F32 = 0, MOE_BF16 = 1 } moe_dtype;

/* Scores of moe_route and activations of moe_linear. */
typedef enum moe_score { MOE_SIGMOID = 0, MOE_SOFTMAX = 1 } moe_score;
typedef enum moe_act { MOE_ACT_NONE = 0, MOE_ACT_RELU = 1, MOE_ACT_SILU = 2, MOE_ACT_GELU = 3 } moe_act;

/* Short text for a status code (static storage, never NULL). */
const char* moe_status_string(moe_status s);

/* MOE_ABI_VERSION of the built library. */
int moe_abi_version(void);

/*
 * moe_gate_topk - router logits, top-k selection and renormalised gate weights.
 *
 * Section 2 (Mixture-of-Experts and Expert Parallelism): each token is routed
 * to a subset of experts. For token t:
 *   z[t,e]  = fl32( fl32(sum_h x[t,h] * w_router[e,h]) + bias[e] )
 *   ids[t,:] = the k experts with the largest z, ordered by (z descending,
 *              expert id ascending): equal logits go to the lower expert id
 *   w[t,j]  = exp(z_j - z_0) / sum_{j'<k} exp(z_j' - z_0)  (fp32, j ascending)
 *
 * x          [T, H]  dt          token activations
 * w_router   [E, H]  dt          row e = routing vector of expert e
 * bias       [E]     fp32        per-expert logit bias (may be NULL = 0)
 * logits_out [T, E]  fp32        optional (NULL to skip): z
 * topk_ids   [T, k]  int32       selected expert ids
 * topk_w     [T, k]  fp32        gate weights
 * Limits: 1 <= E <= 256, 1 <= k <= min(E, 16), H % 8 == 0 (bf16: H % 64 == 0).
 * ws         optional workspace: with ws == NULL and ws_bytes != NULL the
 *            call stores the byte count in *ws_bytes and launches nothing;
 *            with ws and ws_bytes both NULL the router runs in one pass
 *            without it. Given one (16-byte aligned, *ws_bytes at least the
 *            count, else MOE_ERR_WORKSPACE), bf16 routers compute the logits
 *            as fp32 partial sums over K ranges there and add them in a
 *            fixed order before the top-k:
 *              - batches of at most 256 tokens over at most 128 experts
 *                (when a 32-token block's distinct x and router rows reach
 *                192 KB), and batches over at most 64 experts whose
 *                32-token blocks would fill at most half the CUs: 32-token
 *                blocks times up to 8 K ranges;
 *              - 256 experts (any batch) or 128 experts (up to 4096 tokens;
 *                when H >= 4096, every batch whose 128-token blocks would
 *                fill at most half the CUs): 256-token tiles times K
 *                ranges, so a CU loads 256 tokens' rows and a K range of
 *                the router rows instead of every router row for each 64
 *                or 128 tokens.
 *            The count is 0 where no workspace is used (fp32 and every other
 *            case). It depends on the device's compute-unit count: query it
 *            with the device the call will run on current.
 * T == 0 is a no-op. The kernel accumulates in fp32; inputs whose products
 * and partial sums are exact in fp32 give order-independent logits (and the
 * same logits with or without the workspace).
 */
moe_status moe_gate_topk(const void* x, const void* w_router, const float* bias,
                         int T, int H, int E, int k, moe_dtype dt,
                         float* logits_out, int32_t* topk_ids, float* topk_w,
                         void* ws, size_t* ws_bytes, hipStream_t stream);

/*
 * moe_expert_histogram_scan - the activation profile and local offsets.
 *
 * counts[e] = #{(t,j) : topk_ids[t,j] == e} for all E experts (one row of the
 * activation matrix W of Section 4.2.2). expert_map (HOST array [E]) gives
 * the local slot of each expert on this GPU, or -1 for a remote expert; the
 * local slots must be exactly 0..E_local-1, each used once (the placement
 * S_g of Section 4.2.3). offsets[0] = 0 and offsets[l+1] = offsets[l] +
 * counts[expert in slot l]; offsets[E_local] is the GPU's token load.
 *
 * counts  [E]          int32 (device, written)
 * offsets [E_local+1]  int32 (device, written)
 * ws      per-block count table and per-block row bases; pass it unchanged
 *         to moe_permute. Size depends on T, E and E_local only.
 * Limits: 1 <= E <= 256, 0 <= E_local <= E, 1 <= k <= min(E, 16). Expert ids
 * outside [0, E) in topk_ids are ignored.
 */
moe_status moe_expert_histogram_scan(const int32_t* topk_ids, int T, int k, int E,
                                     const int32_t* expert_map, int E_local,
                                     int32_t* counts, int32_t* offsets,
                                     void* ws, size_t* ws_bytes, hipStream_t stream);

/*
 * moe_permute - dispatch: a stable counting sort of assignments by local slot.
 *
 * For flat assignment i = t*k + j in ascending order, if its expert is local
 * (slot l), it gets row pos = offsets[l] + (number of earlier assignments to
 * slot l): perm_src[pos] = i, dest[i] = pos and x_perm[pos,:] = x[t,:].
 * Remote assignments get dest[i] = -1. Under expert parallelism x_perm is the
 * send buffer of the dispatch all-to-all (Section 2).
 *
 * ws, ws_bytes  the workspace filled by moe_expert_histogram_scan (same T, k,
 *               E, E_local); expert_map is the same HOST array.
 * x_perm   [M_cap, H] dt   rows [0, offsets[E_local]) written; may be NULL,
 *          then only perm_src and dest are written (for
 *          moe_grouped_swiglu_ffn_gather, which reads the rows from x)
 * perm_src [M_cap]    int32 entries [0, offsets[E_local]) written
 * dest     [T*k]      int32 all written
 * Requires M_cap >= T*k (the worst case, so no host sync is needed).
 */
moe_status moe_permute(const void* x, const int32_t* topk_ids, const int32_t* expert_map,
                       const void* ws, size_t ws_bytes, int T, int H, int k, int E,
                       int E_local, int M_cap, moe_dtype dt, void* x_perm,
                       int32_t* perm_src, int32_t* dest, hipStream_t stream);

/*
 * moe_grouped_swiglu_ffn - every local expert on its rows of x_perm.
 *
 * For local slot l and rows R = [offsets[l], offsets[l+1]):
 *   G = x_perm[R] W_gate[l]^T, U = x_perm[R] W_up[l]^T   (fp32 accumulation)
 *   h = round_dt( silu(G) * U ),  silu(g) = g / (1 + exp(-g))   (fp32)
 *   y_perm[R] = round_dt( h W_down[l]^T )                  (fp32 accumulation)
 * This is the expert computation whose latency per token load is f_g(n)
 * (Section 4.2.1). Experts with no rows cost nothing and are not read.
 *
 * w_gate, w_up [E_local, I, H] dt with row stride ldw_gu elements (expert
 *              l's matrix starts at row l * I); w_down [E_local, H, I] dt with
 *              row stride ldw_dn (expert l at row l * H). A stride of 0 means
 *              dense (H, resp. I); otherwise it must be >= that, a multiple
 *              of 16 bytes and <= 2^20 (else MOE_ERR_INVALID_ARG). Padding
 *              the rows off a power of two (e.g. H + 64 for H = 4096) spreads
 *              a weight tile's rows over more HBM channels; padding elements
 *              are never read.
 * offsets      [E_local+1] int32 (device, from moe_expert_histogram_scan);
 *              clamped to [0, M_cap] inside the kernels
 * y_perm       [M_cap, H] dt, rows [0, offsets[E_local]) written
 * ws           holds h [M_cap, I] dt; for bf16 also work counters, the
 *              fp32 partial sums of tiles split along K (summed in a fixed
 *              order, so results are deterministic) and a split plan.
 *              bf16: the workspace's first 16 KiB are counters that must be
 *              zero before the first call that uses the workspace (allocate
 *              it zero-filled); every call leaves them zero again. Calls on
 *              one workspace must not overlap.
 *              Schedule (bf16): when no expert has more than 16 rows, or
 *              64 when no reduction launch follows (see below), or 128 in a
 *              GEMM launch with no more 128-column tiles than half its
 *              blocks, each GEMM's (tile, K chunk) units are dealt to the
 *              CUs in equal shares and tiles split between CUs are finished
 *              inside the GEMM launch; otherwise whole tiles run in rounds,
 *              with split-K for tile-starved launches and a split of a
 *              partly filled last round, whose partials a launch after each
 *              GEMM sums. When no expert can have more than 128 rows
 *              (M_cap <= 128; for the _gather variant min(T, M_cap) <= 128,
 *              since a token adds at most one row to an expert) those
 *              launches are left out (two kernel launches in all) and
 *              nothing is split outside the decode schedule. The first call on a device
 *              that is not under graph capture also launches a small
 *              one-time check of the GPU's workgroup-to-XCD assignment.
 * Limits: 0 <= E_local <= 256 (0 is a no-op); bf16: H % 128 == 0 and
 * I % 128 == 0; fp32: H % 4 == 0 and I % 4 == 0.
 */
moe_status moe_grouped_swiglu_ffn(const void* x_perm, const void* w_gate, const void* w_up,
                                  const void* w_down, const int32_t* offsets, int E_local,
                                  int H, int I, int ldw_gu, int ldw_dn, int M_cap, moe_dtype dt,
                                  void* y_perm, void* ws, size_t* ws_bytes, hipStream_t stream);

/*
 * moe_grouped_swiglu_ffn_gather - moe_grouped_swiglu_ffn with the dispatch
 * gather folded into the gate/up GEMM's operand loads.
 *
 * Computes what moe_permute followed by moe_grouped_swiglu_ffn computes
 * (bitwise the same y_perm and h whenever both take the same schedule; with
 * T <= 128 this one may finish split tiles in its GEMM launches where the
 * permuted call, bounded only by M_cap, splits differently, and results then
 * agree within the FFN's tolerance), but row r of the expert input is
 * read as x[perm_src[r] / k] (the token of flat assignment perm_src[r],
 * Section 2's dispatch) instead of from a permuted copy, so the x_perm write
 * and re-read are skipped: call moe_permute with x_perm = NULL for perm_src.
 *
 * x        [T, H] bf16 (the layer's input tokens); T >= 1, T*H*2 < 2^32
 * perm_src [M_cap] int32 from moe_permute; entries of rows outside
 *          [offsets[0], offsets[E_local]) are not read, the others are
 *          clamped to a token of x
 * k        the top-k of the routing (1..MOE_MAX_TOPK)
 * other arguments, workspace and limits: as moe_grouped_swiglu_ffn (bf16
 * only; fp32 returns MOE_ERR_UNSUPPORTED).
 */
moe_status moe_grouped_swiglu_ffn_gather(const void* x, const int32_t* perm_src, int T, int k,
                                         const void* w_gate, const void* w_up, const void* w_down,
                                         const int32_t* offsets, int E_local, int H, int I,
                                         int ldw_gu, int ldw_dn, int M_cap, moe_dtype dt,
                                         void* y_perm, void* ws, size_t* ws_bytes, hipStream_t stream);

/*
 * moe_grouped_swiglu_ffn_gather_of - moe_grouped_swiglu_ffn_gather in a layer
 * of E experts (E_local <= E <= MOE_MAX_EXPERTS; 0: not known, the same call).
 *
 * Same results, bit for bit. M_cap bounds the rows of the local experts, but
 * does not say what part of T*k they hold; with E the library expects T*k/E
 * rows an expert and launches the kernels that suit those, where it otherwise
 * launches two for a GEMM of many rows and lets the offsets choose.
 */
moe_status moe_grouped_swiglu_ffn_gather_of(const void* x, const int32_t* perm_src, int T, int k,
                                            const void* w_gate, const void* w_up, const void* w_down,
                                            const int32_t* offsets, int E, int E_local, int H, int I,
                                            int ldw_gu, int ldw_dn, int M_cap, moe_dtype dt,
                                            void* y_perm, void* ws, size_t* ws_bytes, hipStream_t stream);

/*
 * moe_grouped_swiglu_ffn_noalloc - moe_grouped_swiglu_ffn for callers that
 * cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation).
 *
 * Same arguments, results and limits as moe_grouped_swiglu_ffn, without the
 * workspace: the call allocates nothing (no hipMalloc, hipFree or
 * allocating library routine) and uses instead this library's scratch, a
 * device array of moe_ffn_scratch_bytes() bytes (128 MiB) in each GPU's copy
 * of the code object, held until the process ends. Its counters are cleared
 * on `stream` by the first call on a device; every call leaves them zero.
 * The scratch must hold the workspace's fixed part, the counters (16 KiB),
 * h [M_cap, I] and the split plan, i.e. roughly M_cap * I * sizeof(dt) +
 * 4 * max(M_cap, 64 E_local) + 16 KiB bytes (decode-sized batches: e.g.
 * M_cap <= 500 rows at I = 14336 in bf16); larger calls return
 * MOE_ERR_WORKSPACE and launch nothing. The rest of the scratch holds
 * partial sums of split tiles; where it is smaller than the workspace
 * moe_grouped_swiglu_ffn would use, fewer tiles are split (results stay
 * within the same tolerances, but need not be bitwise those of
 * moe_grouped_swiglu_ffn). All calls on one GPU share its scratch, whatever
 * their stream: calls that overlap in time on one GPU race, so serialise
 * them (one stream, or events).
 */
moe_status moe_grouped_swiglu_ffn_noalloc(const void* x_perm, const void* w_gate, const void* w_up,
                                          const void* w_down, const int32_t* offsets, int E_local,
                                          int H, int I, int ldw_gu, int ldw_dn, int M_cap, moe_dtype dt,
                                          void* y_perm, hipStream_t stream);

/* Bytes of the scratch that moe_grouped_swiglu_ffn_noalloc uses on each GPU. */
size_t moe_ffn_scratch_bytes(void);

/*
 * moe_unpermute_combine - gather and weighted sum back to token order.
 *
 * out[t,:] = round_dt( sum over j ascending with dest[t*k+j] >= 0 of
 *            topk_w[t,j] * y_perm[dest[t*k+j],:] ), fp32 accumulator.
 * Tokens with no local assignment get an exactly zero row, so summing the
 * partial outputs of all GPUs of an expert-parallel group gives the layer
 * output (the combine all-to-all of Section 2). dest entries outside
 * [0, M_cap) are treated as -1.
 *
 * out [T, H] dt (written completely).
 */
moe_status moe_unpermute_combine(const void* y_perm, const float* topk_w, const int32_t* dest,
                                 int T, int k, int H, int M_cap, moe_dtype dt, void* out,
                                 hipStream_t stream);

/*
 * MXFP8 expert FFN (FP8 experts).
 *
 * The paper serves its models in FP8 (Table 2a) without naming a scaling
 * scheme. These entry points use OCP Microscaling FP8 (MXFP8), the block
 * scaling gfx950's scaled MFMA consumes directly: elements are FP8 E4M3 (OCP
 * encoding: bias 7, no infinities, S.1111.111 NaN, largest finite 448), and
 * every 32 consecutive elements along the reduction dimension share one E8M0
 * scale code c, the power of two 2^(c - 127).
 *
 * Quantisation of a 32-element block v (OCP MX conversion): shared exponent
 * s = floor(log2(max |v_i|)) - 8 clamped to [-127, 127] (an all-zero block
 * takes -127), code c = s + 127, element q_i = E4M3 of v_i / 2^s clamped to
 * +-448 and rounded to nearest, ties to even (a value that rounds to zero
 * keeps its sign).
 *
 * Layout of an MXFP8 matrix with R rows and reduction length K (K % 128 == 0):
 *   codes  [R, K]        uint8, row-major (16-byte aligned)
 *   scales [K/128, R]    uint32, chunk-major: dword (k, r) holds the codes of
 *                        row r for elements [128 k, 128 k + 128), byte b
 *                        (little-endian) for elements [128 k + 32 b, +32)
 * A batch of B such matrices (expert weights) is codes [B, R, K] and scales
 * [B, K/128, R]. Weight codes may have padded rows: row r of matrix b at
 * byte (b * R + r) * ld, with ld >= K a multiple of 16 and <= 2^20 (0 means
 * ld = K); padding bytes are never read. Rows a multiple of 4 KiB long
 * (K = 4096) stream faster from HBM with 128 bytes of padding.
 * Activation codes (x, h, a) are always dense.
 */

/*
 * moe_mx_quantize - MXFP8 quantisation of `batch` matrices of `rows` x K.
 *
 * x         [batch, rows, K] dt (bf16 or fp32)
 * row_count DEVICE int32 or NULL (batch 1 only): quantise rows
 *           [0, min(rows, *row_count)) only, e.g. the routed rows of x_perm
 *           with row_count = offsets + E_local, without a host sync; the
 *           other rows' codes and scales are left untouched
 * codes     [batch, rows, K] uint8, rows ld_codes bytes apart (0: dense;
 *           otherwise as padded weight rows above, else MOE_ERR_INVALID_ARG)
 * scales    [batch, K/128, rows] uint32
 * Limits: K % 128 == 0; batch * rows * K <= 2^40.
 */
moe_status moe_mx_quantize(const void* x, moe_dtype dt, int batch, int rows, int K,
                           int ld_codes, const int32_t* row_count, uint8_t* codes,
                           uint32_t* scales, hipStream_t stream);

/*
 * moe_grouped_swiglu_mx - the gate/up half of the MXFP8 expert FFN.
 *
 * For local slot l and rows R = [offsets[l], offsets[l+1]) (clamped to
 * [0, M_cap]):
 *   G = X[R] Wg[l]^T, U = X[R] Wu[l]^T  from the MXFP8 operands (scaled MFMA,
 *                                        fp32 accumulation)
 *   h = silu(G) * U                      (fp32)
 *   (hq, hs)[R] = MXFP8 quantisation of h along I (rules above)
 * xq [M_cap, H], xs [H/128, M_cap]; wgq, wuq [E_local, I, H] (code rows ldw
 * bytes apart, 0: dense), wgs, wus [E_local, H/128, I]; hq [M_cap, I],
 * hs [I/128, M_cap]: rows R of every local expert written, the rest
 * untouched.
 * Limits: 0 <= E_local <= 256; H % 128 == 0, I % 128 == 0; H, I <= 2^20.
 */
moe_status moe_grouped_swiglu_mx(const uint8_t* xq, const uint32_t* xs, const uint8_t* wgq,
                                 const uint32_t* wgs, const uint8_t* wuq, const uint32_t* wus,
                                 const int32_t* offsets, int E_local, int H, int I, int ldw,
                                 int M_cap, uint8_t* hq, uint32_t* hs, hipStream_t stream);

/*
 * moe_grouped_gemm_mx - grouped MXFP8 GEMM with bf16 output: for local slot l,
 * c[R] = bf16( A[R] B[l]^T ) (fp32 accumulation), R as above.
 * aq [M_cap, K], as [K/128, M_cap]; bq [E_local, N, K] (code rows ldb bytes
 * apart, 0: dense), bs [E_local, K/128, N]; c [M_cap, N] bf16, rows R
 * written. The down projection of the MXFP8 FFN.
 * Limits: 0 <= E_local <= 256; N % 128 == 0, K % 128 == 0; N, K <= 2^20.
 */
moe_status moe_grouped_gemm_mx(const uint8_t* aq, const uint32_t* as, const uint8_t* bq,
                               const uint32_t* bs, const int32_t* offsets, int E_local, int N,
                               int K, int ldb, int M_cap, void* c, hipStream_t stream);

/*
 * moe_grouped_swiglu_ffn_mx - the MXFP8 expert FFN (the FP8 counterpart of
 * moe_grouped_swiglu_ffn): moe_grouped_swiglu_mx into the workspace, then
 * moe_grouped_gemm_mx with W_down (wdq [E_local, H, I], wds
 * [E_local, I/128, H]) into y_perm [M_cap, H] bf16. Weight code rows are
 * ldw_gu (W_gate, W_up) and ldw_dn (W_down) bytes apart (0: dense).
 * ws starts with 16 KiB of counters that must be zero before the first call
 * on the workspace (every call leaves them zero), then h codes [M_cap, I]
 * and, 256-byte aligned after them, their scales [I/128, M_cap], then the
 * split plan and the fp32 partial sums of tiles split along K (summed in a
 * fixed order, so results are deterministic). The schedules and launches
 * are those of moe_grouped_swiglu_ffn, with M_cap as the bound on an
 * expert's rows. Calls that share a workspace must not overlap.
 */
moe_status moe_grouped_swiglu_ffn_mx(const uint8_t* xq, const uint32_t* xs, const uint8_t* wgq,
                                     const uint32_t* wgs, const uint8_t* wuq, const uint32_t* wus,
                                     const uint8_t* wdq, const uint32_t* wds,
                                     const int32_t* offsets, int E_local, int H, int I,
                                     int ldw_gu, int ldw_dn, int M_cap, void* y_perm, void* ws,
                                     size_t* ws_bytes, hipStream_t stream);

/*
 * MXFP4 expert FFN (4-bit experts).
 *
 * OCP Microscaling FP4 (MXFP4): elements are E2M1 (+-0, 0.5, 1, 1.5, 2, 3, 4,
 * 6), 32 consecutive elements along the reduction dimension share one E8M0 scale
 * code c, the power of two 2^(c - 127). A weight takes 17/32 of a byte, a quarter
 * of bf16's traffic at decode, and the MFMA runs at four times the bf16 rate.
 *
 * Quantisation of a 32-element block v: shared exponent s = floor(log2(max
 * |v_i|)) - 2 clamped to at least -127 (an all-zero block takes -127), code
 * c = s + 127, element q_i = E2M1 of v_i / 2^s clamped to +-6 and rounded to
 * nearest, ties to even (a value that rounds to zero keeps its sign). A block
 * with a NaN or an infinity takes code 255 (NaN) and zero elements: whatever is
 * computed from it is NaN.
 *
 * Layout of an MXFP4 matrix with R rows and reduction length K (K % 32 == 0):
 * rows are padded with zero elements to C = ceil(K / 256) chunks of 256.
 *   codes  [R, 128 C]   uint8, row-major (16-byte aligned): byte j of a row holds
 *                       elements 2 j (low half) and 2 j + 1 (high half)
 *   scales [C, R, 2]    uint32, chunk-major: byte s of dword (k, r, h) is the code
 *                       of block 2 s + h of row r's chunk k, elements
 *                       [256 k + 64 s + 32 h, +32)
 * A batch of B such matrices is codes [B, R, 128 C] and scales [B, C, R, 2].
 * Weight codes may have padded rows, ld bytes apart (0: 128 C; otherwise at least
 * that, a multiple of 16 and <= 2^20); activation codes are dense. Operands of
 * the products need zero codes and scale codes below 255 in the chunk padding of
 * the weights (as moe_mx4_quantize writes them); in that of activations any
 * codes, with scale codes below 255.
 */

/*
 * moe_mx4_quantize - MXFP4 quantisation of `batch` matrices of `rows` x K.
 *
 * x         [batch, rows, K] dt (bf16 or fp32)
 * row_count DEVICE int32 or NULL (batch 1 only): quantise rows
 *           [0, min(rows, *row_count)) only; the others are left untouched
 * codes     [batch, rows, 128 C] uint8, rows ld_codes bytes apart (0: dense)
 * scales    [batch, C, rows, 2] uint32
 * Limits: K % 32 == 0, K <= 2^20; batch * rows * K <= 2^40.
 */
moe_status moe_mx4_quantize(const void* x, moe_dtype dt, int batch, int rows, int K,
                            int ld_codes, const int32_t* row_count, uint8_t* codes,
                            uint32_t* scales, hipStream_t stream);

/*
 * moe_mx4_dequantize - the values x [batch, rows, K] bf16 that MXFP4 codes stand
 * for (exact: every value of a code below 253 is a bf16; NaN for scale code 255).
 * Arguments and limits as moe_mx4_quantize.
 */
moe_status moe_mx4_dequantize(const uint8_t* codes, const uint32_t* scales, int batch, int rows,
                              int K, int ld_codes, void* x, hipStream_t stream);

/*
 * moe_grouped_swiglu_mx4 - the gate/up half of the MXFP4 expert FFN.
 *
 * For local slot l and rows R = [offsets[l], offsets[l+1]) (clamped to [0, M_cap]):
 *   G = X[R] Wg[l]^T, U = X[R] Wu[l]^T  from the MXFP4 operands (scaled MFMA,
 *                                        fp32 accumulation)
 *   h = silu(G) * U                      (fp32)
 *   (hq, hs)[R] = MXFP4 quantisation of h along I (rules above)
 * perm_src NULL: X has M_cap rows and T and k are not read. Otherwise (DEVICE
 * int32 [M_cap], from moe_permute) X has T rows and row r of the expert input is
 * row perm_src[r] / k of it, clamped to [0, T): tokens are quantised once each
 * and no permuted copy is made. Entries of rows outside the local experts' are
 * not read.
 * xq [M_cap or T, 128 C(H)], xs; wgq, wuq [E_local, I, 128 C(H)] (rows ldw bytes
 * apart, 0: dense), wgs, wus; hq [M_cap, 128 C(I)], hs: rows R written, the rest
 * untouched (and, for I % 256 != 0, the codes in the padding).
 * Limits: 0 <= E_local <= 256; H % 128 == 0, I % 128 == 0; H, I <= 2^20; with
 * perm_src T >= 1, 1 <= k <= 16 and T * 128 C(H) < 2^32.
 */
moe_status moe_grouped_swiglu_mx4(const uint8_t* xq, const uint32_t* xs, const int32_t* perm_src,
                                  int T, int k, const uint8_t* wgq, const uint32_t* wgs,
                                  const uint8_t* wuq, const uint32_t* wus, const int32_t* offsets,
                                  int E_local, int H, int I, int ldw, int M_cap, uint8_t* hq,
                                  uint32_t* hs, hipStream_t stream);

/*
 * moe_grouped_gemm_mx4 - grouped MXFP4 GEMM with bf16 output: for local slot l,
 * c[R] = bf16( A[R] B[l]^T ) (fp32 accumulation), R as above.
 * aq [M_cap, 128 C(K)], as; bq [E_local, N, 128 C(K)] (rows ldb bytes apart, 0:
 * dense), bs; c [M_cap, N] bf16, rows R written.
 * Limits: 0 <= E_local <= 256; N % 128 == 0, K % 128 == 0; N, K <= 2^20.
 */
moe_status moe_grouped_gemm_mx4(const uint8_t* aq, const uint32_t* as, const uint8_t* bq,
                                const uint32_t* bs, const int32_t* offsets, int E_local, int N,
                                int K, int ldb, int M_cap, void* c, hipStream_t stream);

/*
 * moe_grouped_swiglu_ffn_mx4 - the MXFP4 expert FFN: moe_grouped_swiglu_mx4 into
 * the workspace, then moe_grouped_gemm_mx4 with W_down (wdq [E_local, H,
 * 128 C(I)], wds) into y_perm [M_cap, H] bf16. Code rows are ldw_gu (W_gate,
 * W_up) and ldw_dn (W_down) bytes apart (0: dense).
 * ws starts with 16 KiB of counters that must be zero before the first call on
 * the workspace (every call leaves them zero), then h codes [M_cap, 128 C(I)]
 * and, 256-byte aligned after them, their scales, then the split plan and the
 * fp32 partial sums of tiles split along K (summed in a fixed order, so results
 * are deterministic). Calls that share a workspace must not overlap. Each of the
 * two products takes a kernel of its own for few rows where M_cap <= 128 and its
 * weight codes, an expert's once per 16 rows that it can have, are at most 128 MB;
 * otherwise one launch with the schedules of moe_grouped_swiglu_ffn, on 8 waves for
 * every load, and a reduction launch unless no expert can have more than 128 rows
 * (M_cap <= 128; with perm_src min(T, M_cap) <= 128).
 */
moe_status moe_grouped_swiglu_ffn_mx4(const uint8_t* xq, const uint32_t* xs,
                                      const int32_t* perm_src, int T, int k, const uint8_t* wgq,
                                      const uint32_t* wgs, const uint8_t* wuq, const uint32_t* wus,
                                      const uint8_t* wdq, const uint32_t* wds,
                                      const int32_t* offsets, int E_local, int H, int I,
                                      int ldw_gu, int ldw_dn, int M_cap, void* y_perm, void* ws,
                                      size_t* ws_bytes, hipStream_t stream);

/*
 * moe_load_sweep - per-expert latency versus token load.
 *
 * Algorithm 1 Phase 1 / Section 4.2.1: profile the expert computation over a
 * range of token counts to obtain f_g(n). For each M = Ms[i] (HOST array),
 * runs moe_grouped_swiglu_ffn on one expert with offsets [0, M]: `warmup`
 * untimed runs, then `iters` runs each bracketed by HIP events on `stream`.
 * Successive runs rotate through n_rot copies of the expert's weights so
 * that the 256 MB last-level cache does not hold them between runs.
 *
 * x        [maxM, H] dt        input rows (maxM = max of Ms)
 * w_gate, w_up [n_rot, I, H]; w_down [n_rot, H, I]   dt, rows strided by
 *          ldw_gu and ldw_dn as in moe_grouped_swiglu_ffn (0: dense)
 * y_scratch [maxM, H] dt       output rows (contents unspecified afterwards)
 * ws       workspace for maxM (query with ws == NULL); bf16: zero-filled
 *          before its first use, as for moe_grouped_swiglu_ffn
 * us_out   HOST [nM]: median microseconds per run
 * us_all   HOST [nM * iters] or NULL: every timed run, in order
 * Blocks the calling thread until the sweep is done. Limits: 1 <= nM <= 64,
 * 1 <= Ms[i] <= 1 << 20, 0 <= warmup, 1 <= iters <= 10000, n_rot >= 1.
 */
moe_status moe_load_sweep(const void* x, const void* w_gate, const void* w_up,
                          const void* w_down, int n_rot, int H, int I, int ldw_gu,
                          int ldw_dn, moe_dtype dt,
                          const int32_t* Ms, int nM, int warmup, int iters,
                          void* y_scratch, void* ws, size_t* ws_bytes,
                          float* us_out, float* us_all, hipStream_t stream);

/*
 * moe_load_sweep_mx - moe_load_sweep for the MXFP8 expert FFN (the FP8
 * kernel the paper's models run, Table 2a): f_g(n) profiled on
 * moe_grouped_swiglu_ffn_mx with one expert and offsets [0, M].
 *
 * xq [maxM, H], xs [H/128, maxM]   MXFP8 input rows (maxM = max of Ms)
 * wgq, wuq [n_rot, I, H], wgs, wus [n_rot, H/128, I];
 * wdq [n_rot, H, I], wds [n_rot, I/128, H]   MXFP8 weight copies, code rows
 *          ldw_gu / ldw_dn bytes apart (0: dense)
 * y_scratch [maxM, H] bf16; ws, us_out, us_all and limits as moe_load_sweep;
 * H % 128 == 0, I % 128 == 0.
 */
moe_status moe_load_sweep_mx(const uint8_t* xq, const uint32_t* xs, const uint8_t* wgq,
                             const uint32_t* wgs, const uint8_t* wuq, const uint32_t* wus,
                             const uint8_t* wdq, const uint32_t* wds, int n_rot, int H, int I,
                             int ldw_gu, int ldw_dn, const int32_t* Ms, int nM, int warmup, int iters, void* y_scratch,
                             void* ws, size_t* ws_bytes, float* us_out, float* us_all,
                             hipStream_t stream);

/* ------------------------------------------------------------------------
 * The router's training step: losses that balance the experts' loads, their
 * gradient to the router logits, and the gradients of the combine and of the
 * router's product. With the experts frozen (in 4 bits, say) this fine-tunes the
 * router:  moe_combine_backward -> dtopk_w, moe_balance_loss -> counts,
 * moe_gate_backward -> dlogits, moe_router_grad -> dW_router.
 * ---------------------------------------------------------------------- */

/*
 * moe_balance_loss - balance loss, z loss and per-expert counts of a router.
 *
 * Tokens form groups of seq_len consecutive rows (0: one group of all T), a
 * sequence each; mask (or NULL) marks the live ones (non-zero). With p[t,:] =
 * softmax(logits[t,:]), lse[t] = log sum_e exp(logits[t,e]), and for group s of
 * n_s live tokens c[s,e] = #{(t,j) live in s : topk_ids[t,j] == e}:
 *   loss[0] = mean over groups with n_s > 0 of E / (k n_s^2) sum_e c[s,e] sum_t p[t,e]
 *   loss[1] = mean over live tokens of lse[t]^2
 * (0 without live tokens). loss[0] is sum_e f_e P_e with f_e = E c_e / (k n) and
 * P_e the mean of p[:,e]: 1 for equal loads, up to E / k for the most skewed.
 * What masked rows hold is not used. A row that is -inf throughout has p = 0 and
 * lse = 0. Ids outside [0, E) are not counted.
 *
 * logits   [T, E] fp32 (moe_gate_topk's logits_out; 16-byte aligned)
 * topk_ids [T, k] int32
 * mask     [T] uint8 or NULL
 * loss     [2] fp32
 * counts   [groups, E] int32
 * live     [groups + 2] int32: n_s, then the sum of all, then the number of
 *          groups with live tokens
 * ws       its first 256 bytes must be zero before the first call on it (every call
 *          leaves them zero); calls that share one, of any sizes, must not overlap
 * Limits: 1 <= E <= 256, 1 <= k <= min(E, 16), T a multiple of seq_len, T * E <=
 * 2^40 and fewer than 2^23 blocks of 16 tokens or more of a group.
 * Sums are fp32 within a block, joined in fp64 in a fixed order: results do not
 * depend on timing.
 */
moe_status moe_balance_loss(const float* logits, const int32_t* topk_ids, const uint8_t* mask,
                            int T, int E, int k, int seq_len, float* loss, int32_t* counts,
                            int32_t* live, void* ws, size_t* ws_bytes, hipStream_t stream);

/*
 * moe_gate_backward - gradient to the router logits.
 *
 * dlogits[t,e] = (live t)  dloss[0] E / (S k n_s^2) p[t,e] (c[s,e] - sum_j c[s,j] p[t,j])
 *                        + dloss[1] 2 / n lse[t] p[t,e]
 *              + (every t) sum over j with topk_ids[t,j] == e of
 *                          topk_w[t,j] (dtopk_w[t,j] - sum_i topk_w[t,i] dtopk_w[t,i])
 * where n and S are the live tokens and the groups that have some: the gradients
 * of moe_balance_loss's losses (counts do not carry one) and of moe_gate_topk's
 * weights.
 *
 * counts, live  as moe_balance_loss wrote them; T, E, k, seq_len, mask as there
 * dloss         [2] fp32 (DEVICE): gradients of the two losses
 * topk_w, dtopk_w [T, k] fp32, both or neither (NULL: only the losses' part)
 * dlogits       [T, E] fp32, written completely (16-byte aligned)
 */
moe_status moe_gate_backward(const float* logits, const int32_t* topk_ids, const uint8_t* mask,
                             const int32_t* counts, const int32_t* live, const float* dloss,
                             const float* topk_w, const float* dtopk_w, int T, int E, int k,
                             int seq_len, float* dlogits, hipStream_t stream);

/*
 * moe_combine_backward - gradient of moe_unpermute_combine.
 *
 * dtopk_w[t,j] = sum_h dout[t,h] y_perm[dest[t*k+j],h]  (0 where dest is not in [0, M_cap))
 * dy_perm[dest[t*k+j],:] = round_dt( topk_w[t,j] dout[t,:] )
 * (fp32 products and sums). Arguments as moe_unpermute_combine; dtopk_w [T, k]
 * fp32; dy_perm [M_cap, H] dt or NULL: rows that no dest names are left alone.
 */
moe_status moe_combine_backward(const void* dout, const void* y_perm, const float* topk_w,
                                const int32_t* dest, int T, int k, int H, int M_cap, moe_dtype dt,
                                float* dtopk_w, void* dy_perm, hipStream_t stream);

/*
 * moe_router_grad - gradient of the router's product logits = x W_router^T + bias.
 *
 * dx        [T, H] dt or NULL  round_dt( dlogits W_router )
 * dw_router [E, H] fp32        dlogits^T x
 * dbias     [E]    fp32        sum_t dlogits[t,:]
 * dlogits [T, E] fp32; x [T, H], w_router [E, H] dt. bf16: dlogits enters the MFMA
 * as a sum of bf16 terms, all 24 bits of it for dw_router and rounded by at most 2^-17
 * of an element for dx; sums are fp32. T == 0 writes
 * zeros to dw_router and dbias. ws holds partial sums over ranges of tokens, added
 * in order (results do not depend on timing); its size depends on the device's
 * compute units. As in any such product, a row of x that is not finite makes dw_router
 * NaN even where its dlogits are 0: rows of masked tokens must hold numbers. An
 * infinite dlogits gives NaN in dw_router, and in bf16, where the other operand meets
 * each term of dlogits by itself, an infinite x or w_router gives NaN or an infinity.
 * Limits: 1 <= E <= 256, H % 8 == 0 (bf16: H % 64 == 0), H <= 2^20.
 */
moe_status moe_router_grad(const float* dlogits, const void* x, const void* w_router, int T, int E,
                           int H, moe_dtype dt, void* dx, float* dw_router, float* dbias, void* ws,
                           size_t* ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Around the routed experts: routing by scores, groups and a bias for balance
 * (in moe_gate_topk's place, on its logits), dense products with an epilogue
 * (a shared expert, added to the routed ones' output), dropout of the layer's
 * output, and their gradients.
 * ---------------------------------------------------------------------- */

/*
 * moe_route - experts and gate weights of a token from scores of its logits.
 *
 *   s_e = sigmoid(z_e), or exp(z_e) / sum_i exp(z_i)
 *   c_e = s_e + bias_e: what experts are selected by; the weights do not see bias
 *   Experts form n_group groups of E / n_group consecutive ones. A group's score is
 *   the sum of its two largest c (of its one c, where it has one to select); the
 *   topk_group groups of the largest scores are kept.
 *   ids[t,:] = the k experts of kept groups with the largest c, in that order; equal
 *              values go to the lower group and the lower expert id
 *   w[t,j]   = scale * s_j, or with norm scale * s_j / sum of the selected s (a ratio
 *              that selected scores have where they underflow, too)
 * Experts are selected as by s and c in 64 bits; w is computed in 64 bits and rounded to fp32
 * once.
 *
 * An expert whose logit is -inf, or whose c is -inf or NaN, is not selected (a -inf
 * takes part in a softmax with 0). A slot for which no expert is left, and every slot of a
 * token that mask marks as not live (0), gets id -1 and weight 0: moe_expert_histogram_scan
 * and moe_permute pass over it. A live row with a NaN logit (or, in a softmax, with +inf) has
 * NaN weights; its ids are of its other experts.
 *
 * logits [T, E] fp32; bias [E] fp32 or NULL; mask [T] uint8 or NULL (all live)
 * ids [T, k] int32, w [T, k] fp32: written completely; they may share memory neither with
 *   an input nor with each other
 * Limits: 1 <= E <= 256, n_group divides E, 1 <= topk_group <= n_group,
 * 1 <= k <= min(topk_group * E / n_group, 16), scale finite in fp32, T * E <= 2^40.
 */
moe_status moe_route(const float* logits, const float* bias, const uint8_t* mask, int T, int E, int k,
                     moe_score score, int n_group, int topk_group, int norm, double scale, int32_t* ids,
                     float* w, hipStream_t stream);

/*
 * moe_route_backward - gradient of moe_route's weights to the logits.
 *
 * With r_j = s_j / (sum of the selected s), sums over the slots j of a token, and
 * "slots of e" those with ids[t,j] == e (which carry no gradient of their own):
 *   sigmoid:         dlogits[t,e] = sum over slots of e of scale dw_j s_j (1 - s_j)
 *   sigmoid, norm:   ... of scale r_j (dw_j - sum_i r_i dw_i) (1 - s_j)
 *   softmax:         s_e scale (sum over slots of e of dw_j - sum_i s_i dw_i)
 *   softmax, norm:   sum over slots of e of scale r_j (dw_j - sum_i r_i dw_i)
 * in fp32. Slots whose id is outside [0, E) add nothing; a token of such slots alone has the
 * gradient 0, whatever its logits and dw hold. accumulate != 0 adds to what
 * dlogits holds (moe_gate_backward's gradient of the losses, say).
 *
 * logits [T, E], dw [T, k] fp32; ids [T, k] int32; dlogits [T, E] fp32, written completely;
 * it must not overlap logits, ids or dw. Limits: 1 <= E <= 256, 1 <= k <= min(E, 16), scale
 * finite in fp32, T * E <= 2^40.
 */
moe_status moe_route_backward(const float* logits, const int32_t* ids, const float* dw, int T, int E, int k,
                              moe_score score, int norm, double scale, int accumulate, float* dlogits,
                              hipStream_t stream);

/*
 * moe_linear - a dense product with an epilogue.
 *
 *   z = x w^T + bias                          (fp32 accumulation)
 *   y = round_dt( act(z) * mul + residual )   (fp32, rounded once)
 * act: none, max(z, 0), z / (1 + exp(-z)), or z times the normal distribution's integral
 * up to z. A gated projection is act and mul, a down projection added to the routed
 * experts' output is residual.
 *
 * x [M, K] dt; w [N, K] dt, rows ldw elements apart (0: K; otherwise as the expert
 * weights' strides); bias [N] fp32, mul and residual [M, N] dt: each may be NULL
 * y [M, N] dt; it may be mul or residual itself. z [M, N] dt or NULL: round_dt(z), what
 *   moe_linear_backward needs of a layer with an activation. Otherwise neither may share
 *   memory with an input or with the other
 * ws: partial sums of products of few tiles, split along K and joined in a fixed order
 *   (results do not depend on timing). The size that a query names for M serves every call of
 *   at most M rows with the same N, K and dt (a call of fewer rows may itself need more than
 *   one of M). It depends on the device's compute units; ws need not hold anything, and may share
 *   memory with no operand; calls that share one must not overlap.
 * Limits: N % 8 == 0, K % 8 == 0, 8 <= N, K <= 2^20, M <= 2^28, and M N, M K, N K <= 2^36
 * (fp32: 2^34). M == 0 is a no-op.
 */
moe_status moe_linear(const void* x, const void* w, const float* bias, const void* mul, const void* residual,
                      int M, int N, int K, int ldw, moe_act act, moe_dtype dt, void* y, void* z, void* ws,
                      size_t* ws_bytes, hipStream_t stream);

/*
 * moe_linear_backward - the gradients of moe_linear.
 *
 *   dmul  = round_dt( dy * act(z) )
 *   dz    = round_dt( dy * mul * act'(z) )      (dy itself without act and mul)
 *   dbias = sum over rows of dz, before it is rounded
 *   dx    = round_dt( dz w )                    (fp32 accumulation, of the rounded dz)
 *   dw    = round_dw_dt( dz^T x )
 * The residual's gradient is dy. act'(0) of max(z, 0) is 0.
 *
 * dy [M, N] dt; z [M, N] dt as moe_linear wrote it: required with an activation and
 *   for dmul, otherwise not read; mul [M, N] dt or NULL; x, w, ldw as moe_linear
 * dz [M, N] dt: required with an activation or mul (it may be dy itself), not written
 *   without; dmul [M, N] dt or NULL (NULL without mul; not dz, dy or mul)
 * dx [M, K] dt or NULL; dw [N, K] of dw_dt or NULL (fp32 data: fp32; bf16 data: either);
 * dbias [N] fp32 or NULL
 * No output may share memory with another, nor with an input; but dz may be dy itself, and dz
 * and dmul are written before the products, so that they may lie over x without dw and over
 * w without dx, and dx and dw over z or mul.
 * ws and limits as moe_linear. M == 0 writes zeros to dw and dbias.
 */
moe_status moe_linear_backward(const void* dy, const void* x, const void* w, const void* z, const void* mul,
                               int M, int N, int K, int ldw, moe_act act, moe_dtype dt, void* dz, void* dmul,
                               void* dx, void* dw, moe_dtype dw_dt, float* dbias, void* ws, size_t* ws_bytes,
                               hipStream_t stream);

/*
 * moe_dropout_add - dropout by a counter-based generator, and a residual.
 *
 *   out_i = round_dt( residual_i + (u_i < floor(2^32 p) ? 0 : x_i * fl32(1 / (1 - p))) )
 * u_i is word i % 4 of Philox4x32 with 10 rounds at counter offset + i / 4 (64 bits, modulo
 * 2^64; the counter's upper half is 0) under the 64-bit key seed. The mask is never stored:
 * the gradient to x is the same call on the gradient of out, without a residual. A call on n
 * elements uses ceil(n / 4) counters: the caller moves offset on between calls that are to
 * differ.
 *
 * x, residual (or NULL), out [n] dt; out may be x or residual itself, but not a part of
 *   either, nor of rng
 * rng [2] uint64 (DEVICE): seed, offset; read when the call runs, so a captured call takes
 *   what a replay finds there
 * Limits: 0 <= p < 1, n <= 2^40. n == 0 is a no-op.
 */
moe_status moe_dropout_add(const void* x, const void* residual, long long n, double p, const uint64_t* rng,
                           moe_dtype dt, void* out, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Placement control path (Section 4.2, Algorithms 1 and 2): the per-GPU
 * latency model f_g, the latency-aware greedy placement, the drift detector
 * and the incremental swap solver, for L MoE layers of E experts on G GPUs.
 *
 * Latency models: G models of nk knots each, knots_n [G, nk] and knots_t
 * [G, nk] fp64 (DEVICE arrays), knots_n strictly increasing and positive,
 * knots_t non-decreasing (moe_fit_latency_model builds them). f(n) = 0 for
 * n <= 0, knots_t[0] for 0 < n <= knots_n[0], linear between knots, and the
 * last segment's slope beyond the last knot (knots_t[0] n / knots_n[0] with
 * one knot). Knots that break these rules give unspecified placements but no
 * out-of-bounds access.
 *
 * Determinism: every decision is taken in fp64 with separately rounded
 * operations and sums in ascending index order; ties go to the lower GPU
 * index and, among experts, to the lower expert id. Limits: 1 <= E <= 1024,
 * 1 <= G <= 64, 1 <= nk <= 64, L >= 0 (0 is a no-op).
 * ---------------------------------------------------------------------- */

/*
 * moe_fit_latency_model - knots of f_g from measured points (HOST only,
 * launches nothing).
 *
 * Section 4.2.1: f_g(n) maps token load to kernel latency. loads [n] (HOST,
 * distinct, positive) and latencies [n] (HOST, finite) are the measured
 * points, e.g. one moe_load_sweep; the knots are the loads in ascending
 * order and the running maximum of the latencies in that order, so f is
 * monotone. knots_n, knots_t: HOST [n] outputs. 1 <= n <= 64.
 */
moe_status moe_fit_latency_model(const int32_t* loads, const float* latencies, int n,
                                 double* knots_n, double* knots_t);

/*
 * moe_place_greedy - initial latency-aware placement (Algorithm 1, Phase 2).
 *
 * Per layer l: N = sum_e w[l,e]; speeds s_g = 1 / f_g(N / E) (1 when N = 0);
 * token targets tau_g = N s_g / sum_h s_h; experts in descending load order
 * (ascending id among equal loads) each go to the GPU with the largest
 * tau_g - n_g among those holding fewer than `cap` experts (cap = 0: no
 * limit), whose load n_g then grows by the expert's load.
 *
 * w        [L, E] fp64 per-expert loads (DEVICE)
 * assign   [L, E] int32 (DEVICE): the GPU of each expert
 * loads    [L, G] fp64 (DEVICE) or NULL: final n_g
 * targets  [L, G] fp64 (DEVICE) or NULL: tau_g
 * cap: 0, or cap * G >= E.
 */
moe_status moe_place_greedy(const double* w, int L, int E, const double* knots_n,
                            const double* knots_t, int G, int nk, int cap, int32_t* assign,
                            double* loads, double* targets, hipStream_t stream);

/*
 * moe_place_incremental - incremental placement update (Algorithm 2).
 *
 * Per layer, starting from `assign` (DEVICE [L, E] int32, in/out; entries
 * outside [0, G) are read as GPU 0): while the largest f_g(n_g) exceeds
 * (1 + eps) times the mean of f_g(n_g) over the G GPUs, take the slowest GPU
 * g+ and the fastest g- and apply the swap of one expert of g+ with one of
 * g- that lowers max(f_g+(n_g+), f_g-(n_g-)) the most (first in ascending
 * expert ids on ties); stop when none lowers it or after max_swaps swaps.
 * Expert counts per GPU are kept.
 *
 * w        [L, E] fp64 loads (DEVICE)
 * n_swaps  [L] int32 (DEVICE) or NULL: swaps applied per layer
 * eps >= 0 finite; 0 <= max_swaps <= 1 << 20.
 */
moe_status moe_place_incremental(const double* w, int L, int E, const double* knots_n,
                                 const double* knots_t, int G, int nk, double eps, int max_swaps,
                                 int32_t* assign, int32_t* n_swaps, hipStream_t stream);

/*
 * moe_placement_cost - predicted cost of a placement (Section 4.2.3).
 *
 * Per layer l and GPU g: loads[l,g] = n_g = sum of w[l,e] over the experts
 * with assign[l,e] == g (ascending e), lat[l,g] = f_g(n_g), and
 * lat_grouped[l,g] = sum of f_g(w[l,e]) over the same experts (the reading
 * in which each expert runs as its own group). The layer latency the paper
 * minimises is max_g lat[l,g]. Experts with assign outside [0, G) count
 * nowhere.
 *
 * w [L, E] fp64, assign [L, E] int32, loads / lat_grouped [L, G] fp64 or
 * NULL, lat [L, G] fp64 (all DEVICE).
 */
moe_status moe_placement_cost(const double* w, const int32_t* assign, int L, int E,
                              const double* knots_n, const double* knots_t, int G, int nk,
                              double* loads, double* lat, double* lat_grouped, hipStream_t stream);

/*
 * moe_window_push - add one forward pass's per-layer expert counts to a
 * sliding window (Section 4.2.4: load vectors averaged over a window of
 * samples).
 *
 * ring [window, L, E] int32 and sums [L, E] fp64 (DEVICE) are the caller's
 * state, zeroed by the caller before the first push; slot = the ring entry
 * this pass replaces (the caller cycles it 0, 1, ..., window - 1, 0, ...).
 * sums += counts - ring[slot]; ring[slot] = counts. Exact for counts below
 * 2^53 / window. counts [L, E] int32 (DEVICE), e.g. the histogram's counts
 * of each layer. 1 <= window, 0 <= slot < window.
 */
moe_status moe_window_push(const int32_t* counts, int32_t* ring, double* sums, int L, int E,
                           int window, int slot, hipStream_t stream);

/*
 * moe_drift_distance - drift test (Section 4.2.4).
 *
 * d[l] = 1 - w_cur[l].w_ref[l] / (|w_cur[l]| |w_ref[l]|) (0 if both vectors
 * are zero, 1 if exactly one is), sums in ascending expert id; *trigger =
 * 1 if any d[l] > delta, else 0.
 *
 * w_cur, w_ref [L, E] fp64 (DEVICE; window sums or means: the distance does
 * not depend on scale); d [L] fp64 (DEVICE); trigger [1] int32 (DEVICE) or
 * NULL. delta finite. L <= 65536.
 */
moe_status moe_drift_distance(const double* w_cur, const double* w_ref, int L, int E, double delta,
                              double* d, int32_t* trigger, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MOE_SHARD_MOE_H */
