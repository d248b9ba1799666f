/* rom.h — C ABI of the B200 (sm_100a) forward pass of one Routing-Mamba (RoM) layer.
 *
 * Paper notation (Sections 3.1 and 4.2): X in R^{L x D_m} per sequence, D_e = d_inner,
 * D_s = d_state, k = d_conv, d_r = dt_rank, N experts = E, top-K.  T = B*L tokens in (b,t) order,
 * "assignment" a = t*K + k is slot k of token t.
 *
 * General rules
 *   - Every pointer is a DEVICE pointer unless marked "host".  The caller owns every buffer; the
 *     library allocates no device memory and keeps no state on the device between calls.  The one
 *     exception is rom_route_noalloc: its scratch is an array resident in the library's device image, so
 *     overlapping calls of it on one GPU must be serialised by the caller (see its own comment).
 *   - All tensors are dense, row-major, channels-last; device pointers must be 16-byte aligned.  The
 *     alignment of the elements (4 bytes) is enough for the fp32 vectors b_r, b_conv, dt_bias and D,
 *     for b_dt on the fp32 and plain-FMA paths and in rom_layer_step with the shared dt Proj, for h0 and h_last of rom_scan,
 *     for db_r and dD, and for routing outputs (topk_idx, gates, counts, offsets, perm, inv_perm, F, Pbar, loss).
 *   - "dtype" tensors are stored as ROM_F32 (float) or ROM_BF16 (bfloat16) as rom_config.dtype says.
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL = default stream);
 *     they neither synchronise the host nor copy device memory to the host.
 *   - Return value: a rom_status (0 = ok, negative = error).  Argument errors are found on the host
 *     before anything is launched.  Device-side problems (a bounded wait that expired) are latched
 *     in a status word at the head of the workspace and read with rom_get_status.
 *   - Outputs are fully overwritten; inputs are never written; workspace contents are scratch.
 *     Calls that use distinct workspaces and outputs are independent.
 */
#ifndef ROM_H_
#define ROM_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define ROM_API __attribute__((visibility("default")))
#else
#define ROM_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ROM_F32 = 0, ROM_BF16 = 1 } rom_dtype;

typedef enum {
  ROM_OK = 0,
  ROM_ERR_INVALID_ARG = -1,    /* NULL required pointer, bad size, misaligned pointer            */
  ROM_ERR_UNSUPPORTED = -2,    /* a legal problem the library does not cover (e.g. d_state != 16)  */
  ROM_ERR_WORKSPACE = -3,      /* ws_bytes smaller than rom_workspace_size                        */
  ROM_ERR_CUDA = -4,           /* a CUDA runtime/driver call failed (launch, tensor-map encode)   */
  ROM_ERR_ARCH = -5,           /* the current device is not sm_100                                */
  ROM_ERR_DEVICE_TIMEOUT = -6, /* a bounded device-side wait expired (reported by rom_get_status) */
  ROM_ERR_STATIC_SCRATCH = -7, /* the problem does not fit the built-in scratch of rom_route_noalloc */
  ROM_ERR_DEBUG_CHECK = -8     /* ROM_FLAG_DEBUG_CHECKS: a routing-table index out of range or a workspace canary
                                  overwritten (reported by rom_get_status)                          */
} rom_status;

typedef struct {
  int32_t B, L;               /* sequences, tokens per sequence                                   */
  int32_t d_model, d_inner;   /* D_m, D_e : multiples of 64                                       */
  int32_t d_state;            /* D_s : 16                                                         */
  int32_t d_conv;             /* k : 2, 3 or 4                                                    */
  int32_t dt_rank;            /* d_r : multiple of 16 (bf16) / of 4 (f32)                          */
  int32_t E, K;               /* experts (1..64), top-K (1..min(E,8))                             */
  int32_t dtype;              /* rom_dtype                                                        */
  int32_t gate_mode;          /* 0: R_i = P_i * 1[i in TopK] (Section 4.2, routing equation);
                                 1: P_i renormalised over the selected K (the sentence above it)   */
  int32_t disc_mode;          /* 0: zero-order hold B-bar (Section 3.1); 1: B-bar = Delta * B      */
  int32_t flags;              /* ROM_FLAG_* bits                                                  */
  int32_t small_proj_experts; /* 0 or 1: x Proj / dt Proj shared by all experts (Section 4.3, the method as
                                 proposed); E: one x Proj / dt Proj per expert under the same routing
                                 decision (the "(Conv, Gate, dt, x, Out)" ablation row of Section 5.3)      */
} rom_config;

#define ROM_FLAG_SIMT_GEMM 1  /* run every projection on the plain fp32-FMA kernels (bisecting aid;
                                 always the case for ROM_F32) instead of the tcgen05 tensor path   */
#define ROM_FLAG_DEBUG_CHECKS 2 /* rom_layer_forward / rom_layer_step only.  Every gather and scatter of the layer takes
                                 its row index from the routing tables: they are validated on the device before any
                                 kernel uses them (ranges, the two row <-> assignment maps agree, tile -> expert,
                                 padded offsets), and 256-byte canaries between the workspace sub-buffers are written
                                 before the first kernel and compared after the last.  A violation is latched as
                                 ROM_ERR_DEBUG_CHECK.  The workspace is larger with this flag (rom_workspace_size and
                                 rom_workspace_find take it into account); two more small launches per call.      */
#define ROM_FLAG_FUSED_SMALL 8 /* tensor path at top-1 with the shared x Proj / dt Proj: run the short conv, the x Proj and the
                                 dt Proj + softplus as ONE tcgen05 kernel (U written once and never re-read, delta kept on
                                 the SM) instead of three launches.  Same results up to rounding.  Off by default: as
                                 measured it is slower than the three launches (instruction-issue bound on one CTA per
                                 128 tokens); ignored where the sizes do not fit (d_r > 128, d_r + 2 D_s > 160) or b_conv
                                 is off a 16-byte boundary                                                      */
#define ROM_FLAG_TEST_STALL 4 /* fault injection for tests of the device-side timeout path (tensor path only, d_model > 64): the
                                 first grouped projection, and the shared x Proj and dt Proj after it, withhold the copies of one
                                 operand stage per CTA (or, on CTA pairs, in the x Proj and dt Proj kernels and
                                 in rom_layer_step, wait for more bytes than are copied) and every wait of them gives up after 2^14 polls
                                 instead of 2^22, so the call returns normally, produces no valid output, and rom_get_status reports
                                 ROM_ERR_DEVICE_TIMEOUT.  The workspace stays usable for the next call.  rom_ffn_moe_step in bf16: all stages
                                 of a block behind its first wait for more bytes than are copied, in both launches    */

typedef struct {                /* all read-only device pointers                                   */
  const void  *W_r;             /* [E, d_model]              dtype  router, W_r of Section 4.2 transposed */
  const float *b_r;             /* [E] or NULL               router bias (not in the paper)        */
  const void  *W_inz;           /* [E, 2*d_inner, d_model]   dtype  rows [0,D_e): Conv Proj W_in,i^T,
                                                                    rows [D_e,2D_e): Gate Proj W_g,i^T */
  const void  *w_conv;          /* [d_conv, d_inner]         dtype  tap d_conv-1 = current token   */
  const float *b_conv;          /* [d_inner] or NULL                                              */
  const void  *W_x;             /* [dt_rank+2*d_state, d_inner] dtype  rows delta | B | C (shared);
                                   [E, dt_rank+2*d_state, d_inner] when small_proj_experts == E      */
  const void  *W_dt;            /* [d_inner, dt_rank]        dtype  (shared); [E, d_inner, dt_rank]
                                   when small_proj_experts == E                                      */
  const float *b_dt;            /* [d_inner] or NULL                                              */
  const float *A;               /* [d_inner, d_state]        fp32, strictly negative              */
  const float *D;               /* [d_inner] or NULL         skip (not in the paper's equations)   */
  const void  *W_out;           /* [E, d_model, d_inner]     dtype  W_out,i^T                      */
} rom_weights;

/* Bytes of workspace rom_layer_forward / rom_route / rom_route_balance / rom_layer_step need for this
 * config (host out).                                                                              */
ROM_API int rom_workspace_size(const rom_config *cfg, size_t *bytes);

/* Bytes of workspace with which rom_scan cuts a long sequence into chunks that run in parallel (host out;
 * a few MB: two states and one sum of Delta per chunk, sequence and channel).  0 when batch x channels
 * already fill the GPU and the sequence is scanned in one pass.  Uses cfg->B, L, d_inner, d_state, dtype. */
ROM_API int rom_scan_workspace_size(const rom_config *cfg, size_t *bytes);

/* Router + top-K + dropless permutation (Section 4.2 routing equation; Section 5.1: no capacity
 * factor, no token dropping).
 *   logit[t,e] = b_r[e] + sum_d x[t,d] W_r[e,d], accumulated in fp64 (exact products; the same summation order
 *   for every expert, so equal weight rows give equal logits);
 *   P = softmax over all E; the K largest logits are selected, ties to the lowest expert id,
 *   slot k = k-th largest; gates per gate_mode.
 *   counts[e] = assignments of expert e; offsets = exclusive prefix sum (offsets[E] = T*K);
 *   inside an expert's segment assignments keep ascending a = t*K+k:
 *   perm[r] = a, inv_perm[a] = r.
 * Outputs: topk_idx[T,K] i32, gates[T,K] f32, counts[E], offsets[E+1], perm[T*K], inv_perm[T*K] i32.
 * Uses cfg->B, L, d_model, E, K, dtype, gate_mode.  Any output pointer may be NULL (not produced). */
ROM_API int rom_route(const rom_config *cfg, const void *x, const void *W_r, const float *b_r,
              int32_t *topk_idx, float *gates, int32_t *counts, int32_t *offsets,
              int32_t *perm, int32_t *inv_perm, void *ws, size_t ws_bytes, void *stream);

/* Load-balance statistic of the router of one layer (Appendix A.3, load balancing loss): runs the router
 * (same logits, top-K and tie rule as rom_route) and returns
 *   F[i]    = fraction of tokens dispatched to expert i = (assignments of i) / (B*L)   (sums to K),
 *   Pbar[i] = mean over tokens of Softmax(X W_r)_i,
 *   loss[0] = alpha * E * sum_i F[i] * Pbar[i]      (this layer's term; the paper uses alpha = 1e-3).
 * F, Pbar [E] and loss [1] are fp32 device outputs; each may be NULL.  Sums over tokens are taken in a fixed
 * order in fp64, so results are reproducible run to run.  Uses cfg->B, L, d_model, E, K, dtype.            */
ROM_API int rom_route_balance(const rom_config *cfg, const void *x, const void *W_r, const float *b_r, float alpha,
                      float *F, float *Pbar, float *loss, void *ws, size_t ws_bytes, void *stream);

/* rom_route for callers that cannot allocate device memory.  (The paper has no counterpart: this
 * is a deployment variant of the routing step above, with identical results.)
 *
 * Who needs it: a host that gives the library a fixed set of buffers and forbids cudaMalloc while
 * it runs -- a serving process whose memory pool belongs to another component, an allocator that
 * is locked after start-up, a latency-critical loop that cannot absorb an allocation's cost or its
 * failure.  Such a caller cannot provide the workspace rom_route asks for, so this entry point keeps
 * its scratch (about 2 MiB at the largest supported size) in a fixed 3 MiB array inside the library's
 * device image.  Every GPU that loads the library holds that array until the process exits.
 *
 * The caller passes inputs and outputs only; arguments, outputs and their meaning are those of
 * rom_route.  Limits: B*L <= 65536 tokens and B*L*K <= 131072 assignments (E <= 64, K <= 8 as
 * elsewhere); anything larger returns ROM_ERR_STATIC_SCRATCH and launches nothing -- use rom_route
 * with a caller-owned workspace instead.  The call itself allocates nothing, on the host or device.
 *
 * The first call on each GPU looks up the array's device address (once per device, with that
 * device current); make that first call before starting any stream capture.
 * All calls on one GPU share the array, and it keeps the previous call's contents.  Each call
 * rewrites what it reads, clears the one table that must start cleared and leaves its blocks-done
 * counter at zero, so back-to-back calls on one stream are safe; calls that overlap on the same GPU (other streams or
 * host threads) race on the scratch and must be serialised by the caller.                          */
ROM_API int rom_route_noalloc(const rom_config *cfg, const void *x, const void *W_r, const float *b_r,
                      int32_t *topk_idx, float *gates, int32_t *counts, int32_t *offsets,
                      int32_t *perm, int32_t *inv_perm, void *stream);

/* Selective scan (Section 3.1, linear recurrence h_t = A-bar h_{t-1} + B-bar U_t, Y_t = C h_t) with
 * A-bar = exp(Delta A), B-bar per disc_mode, optional skip D*U and optional gate y *= SiLU(z)
 * (output equation of Section 3.1).  State and arithmetic are fp32.
 *   u, z, y : [B, L, d_inner] dtype;  delta : [B, L, d_inner] fp32;  A : [d_inner, d_state] fp32;
 *   Bm, Cm : [B, L, d_state] fp32;  D : [d_inner] or NULL;  z NULL = no gate;
 *   h0 : [B, d_inner, d_state] fp32 or NULL (zeros);  h_last : same shape or NULL (not produced).
 *   ws : NULL (one pass per sequence, whatever its length; with few long bf16 sequences a kernel built for one warp per
 *        SM sub-partition is used) or at least rom_scan_workspace_size(cfg) bytes (few long sequences are then scanned in
 *        parallel along time, in chunks or in one launch; a larger buffer, e.g. the layer's workspace, is accepted; only its head is used).
 *        The result does not depend on the choice beyond fp32 rounding order.
 * Uses cfg->B, L, d_inner, d_state, dtype, disc_mode.                                             */
ROM_API int rom_scan(const rom_config *cfg, const void *u, const float *delta, const float *A,
             const float *Bm, const float *Cm, const float *D, const void *z, const float *h0,
             void *y, float *h_last, void *ws, size_t ws_bytes, void *stream);

/* Backward of rom_scan (Section 5.1 trains the layer end to end; the recurrence differentiated is that of Section
 * 3.1): given dy = dLoss/d(output of rom_scan), the gradients of every input of the same call.
 *   forward   h_t = a_t h_{t-1} + b_t u_t,  y_t = C_t h_t + D u_t,  out_t = y_t SiLU(z_t)  (a = exp(Delta A), b per disc_mode)
 *   reverse   g = dLoss/dh_t:  g += C_t e_t (e = dy SiLU(z));  dC_t = sum_c e_t h_t;  da = g h_{t-1};  db = g u_t;  g <- a_t g
 *   dy, u, z : [B, L, d_inner] dtype (z NULL = no gate);  delta : [B, L, d_inner] fp32;  A, Bm, Cm, D, h0 as in rom_scan;
 *   dh_last  : [B, d_inner, d_state] fp32 or NULL: gradient arriving at the final state.
 * Outputs: du, dz [B, L, d_inner] dtype (dz NULL exactly when z is);  ddelta [B, L, d_inner] fp32;  dA [d_inner, d_state],
 *   dBm, dCm [B, L, d_state], dD [d_inner] (NULL exactly when D is) fp32, each the sum over everything that shares the
 *   parameter (dA and dD over sequences and steps; dBm, dCm over channels) -- accumulated with floating-point atomics,
 *   so their last bits vary from run to run;  dh0 [B, d_inner, d_state] fp32 or NULL.
 * ws: rom_scan_backward_workspace_size(cfg) bytes (the state at the start of every 8 steps, plus the chunk states of the chunk-parallel form).  All arithmetic fp32.
 * Uses cfg->B, L, d_inner, d_state, dtype, disc_mode.                                                              */
ROM_API int rom_scan_backward_workspace_size(const rom_config *cfg, size_t *bytes);
ROM_API int rom_scan_backward(const rom_config *cfg, const void *dy, const void *u, const float *delta, const float *A,
                      const float *Bm, const float *Cm, const float *D, const void *z, const float *h0,
                      const float *dh_last, void *du, float *ddelta, float *dA, float *dBm, float *dCm, float *dD,
                      void *dz, float *dh0, void *ws, size_t ws_bytes, void *stream);

/* Forward pass of one RoM layer (Section 4.2 equations for G, H_t, O_t, E_i with the shared
 * Conv1D / x Proj / dt Proj / A / D of Section 4.3):
 *   route -> gather tokens by expert -> per-expert [Conv Proj | Gate Proj] -> un-permute, sum over
 *   the selected experts (indicator only) -> causal depthwise conv + SiLU -> x Proj, dt Proj +
 *   softplus -> selective scan -> * SiLU(gate) -> re-permute with the same routing -> per-expert
 *   Out Proj -> gate-weighted sum over the selected experts.
 *   x, out : [B, L, d_model] dtype.  topk_idx_out [T,K] i32, gates_out [T,K] f32, counts_out [E] i32
 *   may each be NULL.
 * With cfg->small_proj_experts == E the x Proj and dt Proj are per-expert layers under the same
 * routing (the paper prints no equation for this ablation; it is taken in the pattern of H_t and G):
 *   (delta_i, B_i, C_i) = U_t W_x,i;  B_t = sum_i 1_i B_i;  C_t = sum_i 1_i C_i;
 *   Delta_t = softplus(sum_i 1_i delta_i W_dt,i + b_dt)  -- indicator-only sums over the selected
 *   experts in ascending slot order, each expert's delta_i through its own dt Proj, b_dt shared.   */
ROM_API int rom_layer_forward(const rom_config *cfg, const rom_weights *w, const void *x, void *out,
                      int32_t *topk_idx_out, float *gates_out, int32_t *counts_out,
                      void *ws, size_t ws_bytes, void *stream);

/* Backward pass of one RoM layer (Section 5.1: the layer is trained end to end; Appendix A.3: the router is trained
 * through the gate values).  Given dout = dLoss/dO for the forward of rom_layer_forward on the same cfg, weights and
 * x, returns dx = dLoss/dX and the gradient of every weight.  The equations reversed are those of Sections 3.1 and
 * 4.2 as listed at rom_layer_forward.  Readings where the paper is silent: the top-K indicator is piecewise constant
 * and is held fixed, so the router receives gradient only through R_i (gate_mode decides which form), not through the
 * Conv/Gate projections, which carry the indicator alone; jitter noise and SparseMixer (Appendix A.3) are stochastic
 * training-time estimators and are not part of this call.  Only the shared x Proj / dt Proj wiring (Section 4.3) is
 * differentiated: cfg->small_proj_experts == E returns ROM_ERR_UNSUPPORTED.
 * The call recomputes the forward activations it needs from x (it does not read a forward workspace), then walks the
 * steps backwards: data gradients of the projections are grouped GEMMs on the weights as stored (the plain-FMA path
 * makes transposed copies of them in the workspace); weight gradients are sums over the tokens of each expert's segment.
 *   x, dout, dx : [B, L, d_model] dtype.
 *   g           : device pointers, fp32, fully overwritten: the shapes of the corresponding rom_weights fields;
 *                 db_r may be NULL (not produced); dD is NULL exactly when w->D is.
 *   ws          : rom_layer_backward_workspace_size(cfg) bytes.
 * Sums that cross thread blocks use floating-point atomics: the last bits of the gradients vary from run to run.  */
typedef struct {
  float *dW_r;      /* [E, d_model]                    */
  float *db_r;      /* [E] or NULL                     */
  float *dW_inz;    /* [E, 2*d_inner, d_model]         */
  float *dw_conv;   /* [d_conv, d_inner]               */
  float *db_conv;   /* [d_inner]                       */
  float *dW_x;      /* [dt_rank+2*d_state, d_inner]    */
  float *dW_dt;     /* [d_inner, dt_rank]              */
  float *db_dt;     /* [d_inner]                       */
  float *dA;        /* [d_inner, d_state]              */
  float *dD;        /* [d_inner] or NULL               */
  float *dW_out;    /* [E, d_model, d_inner]           */
} rom_grads;
ROM_API int rom_layer_backward_workspace_size(const rom_config *cfg, size_t *bytes);
ROM_API int rom_layer_backward(const rom_config *cfg, const rom_weights *w, const void *x, const void *dout, void *dx,
                       const rom_grads *g, void *ws, size_t ws_bytes, void *stream);

/* rom_layer_forward with HOST input and output: enqueues on `stream` the copy of x_host to x_dev, the
 * forward (x_dev -> out_dev) and the copy of out_dev to out_host, and returns without waiting.
 *   x_host, out_host : HOST pointers, [B, L, d_model] dtype; page-locked memory makes the copies
 *                      asynchronous (pageable memory works but serialises with the host)
 *   x_dev, out_dev   : device staging buffers of the same size, owned by the caller
 * out_host is valid once the stream has been synchronised.  Calls on different streams with their own
 * staging buffers and workspaces overlap one call's copies with another's kernels.               */
ROM_API int rom_layer_forward_host(const rom_config *cfg, const rom_weights *w, const void *x_host, void *out_host,
                           void *x_dev, void *out_dev, void *ws, size_t ws_bytes, void *stream);

/* Single-token step of the layer (recurrent inference; Section 3.1: the state-space model is a linear
 * recurrence, so a generated token costs the same whatever the context length).  Same equations and
 * routing as rom_layer_forward for one new token per sequence, with the state carried by the caller:
 *   x, out     : [B, d_model] dtype (cfg->L must be 1)
 *   conv_state : [B, d_conv-1, d_inner] fp32, in/out: H_t (the summed Conv Proj rows) of the previous
 *                d_conv-1 tokens, oldest first; zeros at the start of a sequence
 *   ssm_state  : [B, d_inner, d_state] fp32, in/out: h_{t-1}; zeros at the start of a sequence
 * Feeding a sequence token by token from zero states reproduces rom_layer_forward on the whole sequence
 * (up to the rounding of the storage dtype).  topk_idx_out [B,K], gates_out [B,K] may be NULL.
 * bf16 (small_proj_experts <= 1, no flags, d_r a multiple of 16, B <= 512, B*K <= 2048): a sequence's result does not depend on the
 * other sequences of the batch, to the last bit, among all calls of fewer than four assignments (B*K) and among all calls of
 * four and more; the two differ by fp32 rounding order.
 * ws: rom_workspace_size(cfg) bytes.                                                               */
ROM_API int rom_layer_step(const rom_config *cfg, const rom_weights *w, const void *x, float *conv_state,
                   float *ssm_state, void *out, int32_t *topk_idx_out, float *gates_out,
                   void *ws, size_t ws_bytes, void *stream);

/* Feed-forward SwiGLU mixture of experts that shares the routing decision of the preceding RoM layer
 * (Appendix A.2, the two equations of the hybrid RoM + FFN-MoE model):
 *   Y_t = sum_i R_i * 1[i in TopK] * f_i(X_t),   f_i(x) = W_down,i ( SiLU(W_gate,i x) * (W_up,i x) )
 * (the paper names f_i a SwiGLU expert without writing it out; the usual bias-free form is taken).
 * The selected experts and their gates are not recomputed: topk_idx [T,K] i32 and gates [T,K] f32 are
 * the outputs of that layer's rom_route / rom_layer_forward call (device pointers, read only).
 *   d_ff   : hidden width of an expert, a multiple of 128
 *   W_gu   : [E, 2*d_ff, d_model] dtype, rows [0,d_ff) = W_gate,i, rows [d_ff,2*d_ff) = W_up,i
 *   W_down : [E, d_model, d_ff]   dtype
 *   x, out : [B, L, d_model]      dtype (x is this layer's own input)
 *   ws     : rom_ffn_moe_workspace_size(cfg, d_ff) bytes of scratch, independent of the RoM layer's
 * Uses cfg->B, L, d_model, E, K, dtype, flags.  The K experts of a token must be distinct and in
 * [0, E); an index outside that range is clamped (every access stays in bounds, the result for that
 * token is unspecified) and rom_get_status then reports ROM_ERR_INVALID_ARG.                        */
ROM_API int rom_ffn_moe_workspace_size(const rom_config *cfg, int32_t d_ff, size_t *bytes);
ROM_API int rom_ffn_moe_forward(const rom_config *cfg, int32_t d_ff, const void *W_gu, const void *W_down,
                        const void *x, const int32_t *topk_idx, const float *gates, void *out,
                        void *ws, size_t ws_bytes, void *stream);

/* Routing Mamba on a Mamba2-style block (Section 5.2, "RoM on other linear recurrent architectures"; Section 5.4, first
 * insight: for blocks with a unified design all major projection layers become experts under the shared routing;
 * Appendix A.2: the deployment "follows the same logic" as on Mamba).  The paper prints no equations for this variant:
 * the block is the published Mamba2 block with one B/C group, and per token t
 *   [z | x | B | C | dt]_t = sum_i 1_i X_t W_in,i           (indicator only; widths D_e | D_e | N | N | heads)
 *   (x, B, C) <- SiLU(causal depthwise conv(x, B, C) + b_conv);   dt_h = softplus(dt_h + dt_bias_h)
 *   per head h (headdim channels):  H_t = exp(dt_h A_h) H_{t-1} + dt_h x_t (x) B_t,   y_t = C_t H_t + D_h x_t
 *   y^_t = (y_t * SiLU(z_t)) / sqrt(mean_c (y_t * SiLU(z_t))_c^2 + 1e-5) * w_norm
 *   O_t = sum_i R_i(X_t) y^_t W_out,i
 * with the router, top-K, gates and permutation of rom_route.  Shared by all experts: conv, A, D, dt_bias, w_norm.
 *   headdim : channels per head; d_inner / headdim heads, a multiple of 8.  cfg->dt_rank, disc_mode and
 *             small_proj_experts are not used; d_state must be 16, d_conv 2..4.
 *   x, out  : [B, L, d_model] dtype;  ws: rom_mamba2_workspace_size(cfg, headdim) bytes.                            */
typedef struct {                  /* read-only device pointers */
  const void  *W_r;               /* [E, d_model]                               dtype */
  const float *b_r;               /* [E] or NULL */
  const void  *W_in;              /* [E, 2*d_inner + 2*d_state + heads, d_model] dtype  rows z | x | B | C | dt */
  const void  *w_conv;            /* [d_conv, d_inner + 2*d_state]              dtype  tap d_conv-1 = current token */
  const float *b_conv;            /* [d_inner + 2*d_state] or NULL */
  const float *dt_bias;           /* [heads] or NULL */
  const float *A;                 /* [heads], strictly negative */
  const float *D;                 /* [heads] or NULL */
  const float *w_norm;            /* [d_inner] */
  const void  *W_out;             /* [E, d_model, d_inner]                      dtype */
} rom_mamba2_weights;
ROM_API int rom_mamba2_workspace_size(const rom_config *cfg, int32_t headdim, size_t *bytes);
ROM_API int rom_mamba2_layer_forward(const rom_config *cfg, int32_t headdim, const rom_mamba2_weights *w, const void *x,
                             void *out, int32_t *topk_idx_out, float *gates_out, int32_t *counts_out,
                             void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------------------------------------------------------------------
 * Serving: prompts and generated tokens of many sequences in one call.  Every live sequence has a slot in pools that the caller
 * owns: conv windows [n_slots, d_conv-1, d_inner] fp32 (oldest first) and scan states [n_slots, d_inner, d_state] fp32, the
 * layouts that rom_layer_step carries.  The recurrence and the short conv are those of Section 3.1; a prompt run by the ragged calls and
 * continued token by token gives what one call over the whole sequence gives, up to the rounding of the storage dtype.
 * Pools: a call reads the slots it names in the *_in pool and writes them in the *_out pool; the two may be one buffer (updated
 * in place) or two that do not overlap.  Slots that no sequence names are not touched.  Two sequences of a call must not name the same
 * slot: nothing is read or written out of bounds if they do, but what both yield is unspecified.  Pools, activations and weights are
 * 16-byte aligned; seq_start, slot, resume, Bm, Cm, D and b_conv need the alignment of their elements.  Rows of activations may lie ld
 * elements apart (ldx, ldz: at least d_inner, a multiple of 16 bytes; ld_bc: at least d_state). */
typedef struct {               /* sequences packed one behind the other in buffers of `rows` rows */
  int32_t n_seq;               /* sequences (0: nothing is done), at most 2^20                                    */
  int32_t rows;                /* rows of the packed buffers                                                      */
  int32_t n_slots;             /* states in each pool                                                             */
  const int32_t *seq_start;    /* device [n_seq+1], ascending: sequence i is rows [seq_start[i], seq_start[i+1]), none of them when the two
                                  are equal.  Outputs of the rows before the first and behind the last sequence are left as they are (their inputs
                                  may hold anything).  Offsets are cut to [0, rows]; what descending ones yield is unspecified, but in bounds.  */
  const int32_t *slot;         /* device [n_seq] or NULL (sequence i has slot i).  Outside [0, n_slots): the sequence starts
                                  from zeros and its state is not kept                                            */
  const int32_t *resume;       /* device [n_seq] or NULL.  0 (NULL: all): the sequence starts from zeros; else from its slot */
} rom_ragged;

/* Causal depthwise conv + SiLU over packed sequences: y_t = SiLU(b_conv + sum_j w_conv[j] x_{t-(d_conv-1)+j}), the rows before a sequence's first
 * one taken from its window (or zeros); afterwards the slot holds the sequence's last d_conv-1 rows.
 *   x : [rows, d_inner] dtype, pitch ldx;  w_conv : [d_conv, d_inner] dtype, tap d_conv-1 = current row;  b_conv : [d_inner] fp32 or NULL;
 *   win_in (NULL: every sequence starts from zeros), win_out (NULL: not kept);  y : [rows, d_inner] dtype, contiguous, not x.
 * Uses cfg->d_inner, d_conv, dtype (B and L are not used).                                                        */
ROM_API int rom_conv_ragged(const rom_config *cfg, const rom_ragged *seqs, const void *x, int64_t ldx, const void *w_conv,
                    const float *b_conv, const float *win_in, float *win_out, void *y, void *stream);

/* Selective scan over packed sequences: rom_scan's recurrence, skip and gate for each of them, states in slots.
 *   u, y : [rows, d_inner] dtype, contiguous;  delta : [rows, d_inner] fp32, contiguous;  Bm, Cm : [rows, d_state] fp32, pitch ld_bc;
 *   A, D as in rom_scan;  z : [rows, d_inner] dtype, pitch ldz, or NULL (no gate);
 *   h_in (NULL: every sequence starts from zeros), h_out (NULL: not kept).  y is none of the inputs.
 *   ws : rom_scan_ragged_workspace_size(cfg, n_seq, rows) bytes (host out); scratch of this call alone: overlapping calls, captured graphs
 *        that may run at the same time among them, need one each.  A buffer sized for some n_seq and rows does for all calls of no more of both.
 * State and arithmetic are fp32; in bf16 with zero-order hold a step's input may be 2^-10 of itself off (2^-19 in fp32), however small the step.
 * Uses cfg->d_inner, d_state, dtype, disc_mode (B and L are not used).                                              */
ROM_API int rom_scan_ragged_workspace_size(const rom_config *cfg, int32_t n_seq, int32_t rows, size_t *bytes);
ROM_API int rom_scan_ragged(const rom_config *cfg, const rom_ragged *seqs, const void *u, const float *delta, const float *A,
                    const float *Bm, const float *Cm, int64_t ld_bc, const float *D, const void *z, int64_t ldz, const float *h_in,
                    float *h_out, void *y, void *ws, size_t ws_bytes, void *stream);

/* The same for one token of cfg->B sequences (cfg->L must be 1): row b continues the sequence of slot[b] (NULL: slot b).  A row whose slot
 * is outside [0, n_slots) is padding: its output and all slots are left as they are.  Both pools are required.     */
ROM_API int rom_conv_step(const rom_config *cfg, const void *x, int64_t ldx, const void *w_conv, const float *b_conv, const int32_t *slot,
                  int32_t n_slots, const float *win_in, float *win_out, void *y, void *stream);
ROM_API int rom_scan_step(const rom_config *cfg, const void *u, const float *delta, const float *A, const float *Bm, const float *Cm,
                  int64_t ld_bc, const float *D, const void *z, int64_t ldz, const int32_t *slot, int32_t n_slots, const float *h_in,
                  float *h_out, void *y, void *stream);

/* rom_ffn_moe_forward for the few tokens of a generation step (B*L <= 64): same equation, inputs and layouts, in two launches that read
 * each chosen expert's weights once.  An expert index outside [0, E) contributes nothing; negative ones are the padding of a fixed
 * batch (a token with none but those gets a row of zeros), others are reported by rom_get_status as ROM_ERR_INVALID_ARG.  An expert that a
 * token names twice counts twice.
 *   ws : rom_ffn_moe_step_workspace_size(cfg, d_ff) bytes (host out); overlapping calls need one each.  A buffer sized for some
 *        B*L does for calls of fewer tokens (the rest of cfg and d_ff as they are).
 * Uses cfg->B, L, d_model, E, K, dtype (flags must be 0 but for ROM_FLAG_TEST_STALL).                               */
ROM_API int rom_ffn_moe_step_workspace_size(const rom_config *cfg, int32_t d_ff, size_t *bytes);
ROM_API int rom_ffn_moe_step(const rom_config *cfg, int32_t d_ff, const void *W_gu, const void *W_down, const void *x,
                     const int32_t *topk_idx, const float *gates, void *out, void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------------------------------------------------------------------
 * Linear attention with a decay for each head: the linear recurrence of Section 3.1 with a matrix state per head instead of d_state numbers per
 * channel, and a decay that is the head's alone.  (The architectures that Section 5.2 names, Mamba2 and Gated DeltaNet, decay by the token: they are not
 * this.)  Per value head h,
 *   S_t = lambda_h S_{t-1} + k_t v_t^T   [d_k, d_v],     o_t = scale * q_t S_t,     lambda_h = exp(log_decay[h]).
 * Value head h uses head h / (n_heads / n_qk_heads) of q and k.  Values wider than d_v = 128 are several heads that share q and k and their decay.
 *   q, k : [rows, n_qk_heads, d_k] dtype, pitches ldq, ldk;   v : [rows, n_heads, d_v] dtype, pitch ldv;   o : [rows, n_heads, d_v] dtype, contiguous;
 *   log_decay : [n_heads] fp32, finite and at most 0 (0: no decay; others are in bounds, their results unspecified);  a constant of the model: it has no gradient.
 *   State pools: [n_slots, n_heads, d_k, d_v] fp32, slots as in the serving calls above (rom_ragged; in place, or two that do not overlap).
 * Pitches: elements, at least the row's width and a multiple of 16 bytes.  log_decay needs the alignment of its elements, everything else 16 bytes.
 * States and sums are fp32.  In bf16 the scores (after their decay) and the state that a chunk of rows meets are operands of the matrix instructions as the sum
 * of two bf16 numbers (less than 2^-15 of each left out), and so are the keys in the backward's states, which only dq and dk meet; the keys that enter a state
 * that is a result are the sum of three, which are all of their bits.  A sum in the matrix instructions, which drop what is below its last bit, moves to fp32
 * registers after 512 rows at most, so that a state's error does not grow with its sequence (6e-7 of its norm measured, without decay).
 * A value that is not finite shows in its own row and later ones of its sequence and head, as infinity or NaN, in earlier rows never. */
typedef struct {
  int32_t n_heads;            /* value heads, 1..1024: one state and one decay each                            */
  int32_t n_qk_heads;         /* heads of q and k, a divisor of n_heads                                        */
  int32_t d_k, d_v;           /* multiples of 8, 8..128                                                        */
  int32_t dtype;              /* rom_dtype                                                                     */
  int32_t flags;              /* ROM_FLAG_SIMT_GEMM (bf16 on the plain fp32-FMA kernels), ROM_FLAG_TEST_STALL   */
  float scale;                /* of the outputs, d_k^-1/2 as a rule; finite                                    */
} rom_linattn_config;

/* Packed sequences.  s_in (NULL: every sequence starts from zeros), s_out (NULL: not kept).  o is none of the inputs.
 *   ws : rom_linattn_ragged_workspace_size(cfg, n_seq, rows) bytes (host out); scratch of this call alone: overlapping calls, captured graphs that may run at
 *        the same time among them, need one each.  A buffer sized for some n_seq and rows does for all calls of no more of both.  rom_get_status(ws) tells
 *        whether a device-side wait ran out.                                                                    */
ROM_API int rom_linattn_ragged_workspace_size(const rom_linattn_config *cfg, int32_t n_seq, int32_t rows, size_t *bytes);
ROM_API int rom_linattn_ragged(const rom_linattn_config *cfg, const rom_ragged *seqs, const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v,
                       int64_t ldv, const float *log_decay, const float *s_in, float *s_out, void *o, void *ws, size_t ws_bytes, void *stream);

/* One token of B sequences: row b continues the sequence of slot[b] (NULL: slot b).  A row whose slot is outside [0, n_slots) is padding: its output and all
 * slots are left as they are.  Both pools are required.                                                                 */
ROM_API int rom_linattn_step(const rom_linattn_config *cfg, int32_t B, const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv,
                     const float *log_decay, const int32_t *slot, int32_t n_slots, const float *s_in, float *s_out, void *o, void *stream);

/* Backward of rom_linattn_ragged on the same sequences and inputs: given dout = dLoss/do and ds_out = dLoss/d(s_out) (NULL: zeros),
 *   dq_t = scale * S_t dout_t,   R_t = lambda R_{t+1} + scale * q_t dout_t^T  (+ ds_out at a sequence's last row),   dk_t = R_t v_t,   dv_t = R_t^T k_t,
 * dq and dk summed over the value heads that share them, and ds_in = lambda R at a sequence's first row (of an empty one: ds_out), zeros for a sequence that
 * started from zeros (without s_in: all of them, whatever `resume` says).  The states are recomputed, not kept by the forward.
 *   dout : [rows, n_heads, d_v] contiguous;  dq, dk : [rows, n_qk_heads, d_k] contiguous;  dv : [rows, n_heads, d_v], pitch lddv;  all dtype, rows outside the
 *   sequences are left as they are;  ds_in (NULL: not produced): [n_slots, n_heads, d_k, d_v] fp32, slots that no sequence names are left as they are; does not
 *   overlap ds_out or s_in.  No output is an input.  Sums are taken in a fixed order: results are the same from run to run.
 *   ws : rom_linattn_backward_workspace_size(cfg, n_seq, rows) bytes, as above.                                         */
ROM_API int rom_linattn_backward_workspace_size(const rom_linattn_config *cfg, int32_t n_seq, int32_t rows, size_t *bytes);
ROM_API int rom_linattn_backward(const rom_linattn_config *cfg, const rom_ragged *seqs, const void *dout, const void *q, int64_t ldq, const void *k, int64_t ldk,
                         const void *v, int64_t ldv, const float *log_decay, const float *s_in, const float *ds_out, void *dq, void *dk, void *dv, int64_t lddv,
                         float *ds_in, void *ws, size_t ws_bytes, void *stream);

/* What prepares q and k of that recurrence: the RMS norm of every head and its rotation by the row's position, in one pass.
 *   n = x * (mean_c x_c^2 + eps)^-1/2 * w;   for the pair i of the first rot_dim places, with the angle pos[row] * inv_freq[i],
 *   (y_a, y_b) = (n_a cos - n_b sin, n_b cos + n_a sin),   (a, b) = (i, i + rot_dim/2), or (2i, 2i + 1) when interleaved;   the other places: y = n.
 * Prompts, training batches and single tokens are all rows of one call.
 *   q : [rows, n_q_heads, d_head] dtype, pitch ldq;  k : [rows, n_k_heads, d_head], pitch ldk;  q_out, k_out alike, with their own pitches; each output may be its
 *   input (same address and pitch), otherwise no output overlaps an input;
 *   w_q, w_k : [d_head] fp32, or NULL (ones);  pos : [rows] int32;  inv_freq : [rot_dim/2] fp32 (both NULL when rot_dim is 0).
 * The angle is the exact product of the two, reduced before it is rounded: positions up to 2^31 keep fp32 accuracy.  Norm and rotation are fp32, rounded once.
 * A value that is not finite may show in every place of its head in its row (and of its kind's dw in the backward), in no other row or head.
 * Pitches as above; w, pos and inv_freq need the alignment of their elements, everything else 16 bytes.                  */
typedef struct {
  int32_t n_q_heads, n_k_heads;   /* 1..1024                                                      */
  int32_t d_head;                 /* a multiple of 8, 8..256                                      */
  int32_t rot_dim;                /* places that are rotated: a multiple of 16, 0..d_head         */
  int32_t interleaved;            /* 0 or 1                                                       */
  int32_t dtype;                  /* rom_dtype                                                    */
  float eps;                      /* positive and finite                                          */
} rom_qk_config;
ROM_API int rom_qk_norm_rope(const rom_qk_config *cfg, int32_t rows, const void *q, int64_t ldq, const void *k, int64_t ldk, const float *w_q, const float *w_k,
                     const int32_t *pos, const float *inv_freq, void *q_out, int64_t ldq_out, void *k_out, int64_t ldk_out, void *stream);

/* Its backward, from the inputs of the forward and the gradients dq_out, dk_out of its outputs (contiguous):
 *   dn = the rotation back of dy;   dx = r (dn w - xhat mean_c(dn w xhat)),  r = (mean_c x_c^2 + eps)^-1/2, xhat = x r;   dw = sum over rows and heads of dn xhat.
 *   dq, dk : like q and k, pitches lddq, lddk, none of the inputs;  dw_q, dw_k : [d_head] fp32, NULL exactly when w_q, w_k are.  Sums in a fixed order.
 *   ws : rom_qk_norm_rope_backward_workspace_size(cfg, rows) bytes; one sized for more rows does for fewer.             */
ROM_API int rom_qk_norm_rope_backward_workspace_size(const rom_qk_config *cfg, int32_t rows, size_t *bytes);
ROM_API int rom_qk_norm_rope_backward(const rom_qk_config *cfg, int32_t rows, const void *dq_out, const void *dk_out, const void *q, int64_t ldq, const void *k,
                              int64_t ldk, const float *w_q, const float *w_k, const int32_t *pos, const float *inv_freq, void *dq, int64_t lddq, void *dk,
                              int64_t lddk, float *dw_q, float *dw_k, void *ws, size_t ws_bytes, void *stream);

/* Profiling aid: the same launch sequence as rom_layer_forward with a CUDA event recorded on
 * `stream` between stages; synchronises the stream and writes the device time of each stage in
 * milliseconds to stage_ms (host out, at least rom_num_stages() floats).  Stage i is named
 * rom_stage_name(i): route, gather, in_proj, conv, x_proj, dt_proj, scan, out_proj, combine.      */
ROM_API int rom_layer_forward_profile(const rom_config *cfg, const rom_weights *w, const void *x, void *out,
                              void *ws, size_t ws_bytes, void *stream, float *stage_ms, int n_stage_ms);
ROM_API int rom_num_stages(void);
ROM_API const char *rom_stage_name(int i);

/* Locate a named intermediate of the last rom_layer_forward inside the workspace (host-only
 * arithmetic; for tests and debugging).  Names: "U" [T,D_e] dtype, "delta_r" [T,d_r] dtype,
 * "Bm","Cm" [T,D_s] f32, "Delta" [T,D_e] dtype, "row_of_assign" [T*K] i32 (padded row of each
 * assignment), "XZp" [rows,2*D_e] dtype, "Ygp" [rows,D_e] dtype, "pad_offsets" [E+1] i32.
 * Returns ROM_ERR_INVALID_ARG for an unknown name.
 * After rom_layer_step on its own kernels (bf16, see there) "U", "delta_r", "Bm" and "Cm" hold the step's rows, and
 * "Ygp" its gated rows in token order ([B,D_e]); "row_of_assign", "pad_offsets", "Delta" and (top-1) the Conv half of
 * "XZp" are not filled: that path needs no permutation and keeps Delta in registers.               */
ROM_API int rom_workspace_find(const rom_config *cfg, const char *name, size_t *offset, size_t *bytes);

/* Re-run the checks of ROM_FLAG_DEBUG_CHECKS on a workspace that the last rom_layer_forward / rom_layer_step call
 * with that flag (same cfg) has filled: routing tables and canaries (a debugging aid; the paper has no counterpart).
 * Asynchronous on `stream`; the verdict is read with rom_get_status.  cfg->flags must carry the flag.  */
ROM_API int rom_debug_check(const rom_config *cfg, void *ws, size_t ws_bytes, void *stream);

/* Read and clear the device status word of a workspace.  `host_code` (host out) receives ROM_OK or the
 * rom_status a kernel latched: ROM_ERR_DEVICE_TIMEOUT (a bounded wait expired) or ROM_ERR_INVALID_ARG
 * (rom_ffn_moe_forward met an expert index out of range) or ROM_ERR_DEBUG_CHECK (ROM_FLAG_DEBUG_CHECKS; the second
 * and third int32 of the workspace then hold which check failed -- 10..15 a routing table, 20 a canary -- and the
 * offending index, until this call clears them).  This call synchronises `stream`.                  */
ROM_API int rom_get_status(void *ws, void *stream, int32_t *host_code);

/* Static string for a rom_status value.                                                           */
ROM_API const char *rom_status_string(int code);

/* Number of kernels the last call of rom_layer_forward launched on this host thread (host-only). */
ROM_API int rom_last_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* ROM_H_ */
