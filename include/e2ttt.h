/*
 * e2ttt.h -- C ABI of the MI355X (gfx950) E2-TTT chunk-parallel fast-weight update.
 *
 * Method: arxiv 2608.21308, "Rethinking Expressivity and Efficiency in
 * Test-Time Training".  The library computes, for every (batch, head) unit
 * independently, the chunk update of Algorithm 1:
 *   - chunk-start outputs  o_t = f_{W_0}(q_t)                  (eq. (6))
 *   - per-token gradients  G_t = -grad_W 1/2||f_{W_0}(k_t) - v_t||^2 at the
 *     chunk-start weights (Sec. 3.1)
 *   - the closed-form transition of Prop. 1 (eq. (10)-(11))
 *       M_C = b~_0 M_0 + sum_t K^M_t G_t
 *       W_C = g~_0 W_0 + b~_0 R_1 M_0 + sum_t K^W_t G_t
 *     which equals the per-token recurrence M_t = beta_t M_{t-1} + eta_t G_t,
 *     W_t = gamma_t W_{t-1} + M_t (eq. (7)) at every chunk end,
 * and the state (W, M) is carried from chunk to chunk.  The fast-weight net f
 * is the GELU MLP f(x) = x + LN(W2 GELU(W1 x)) or the SwiGLU net
 * f(x) = x + LN(Wd (SiLU(Wg x) * (Wu x))) of Sec. 4 (LayerNorm with biased
 * variance, eps = ln_eps, and optionally a learnable affine per head,
 * E2TTT_FLAG_LN_AFFINE).  GELU is x Phi(x) with the normal CDF; the
 * chunk kernels evaluate Phi through the rational erfc of Abramowitz & Stegun
 * eq. 7.1.26 (absolute error at most 1.5e-7, so a relative error of Phi that
 * grows for x << 0 where Phi itself is tiny), e2ttt_apply through erff.
 *
 * Conventions shared by every entry point:
 *   - Every tensor pointer is a DEVICE pointer (hipMalloc'd or equivalent) on
 *     the current HIP device; all work is enqueued on `stream` (a hipStream_t,
 *     NULL = the default stream) and the call returns without waiting.
 *   - The caller owns every buffer; the library never allocates, frees or
 *     keeps state between calls and is safe to call from several host threads
 *     on distinct streams.
 *   - Every argument check runs before anything is launched; on an error
 *     return nothing has been written.  Errors raised by kernels while they
 *     run surface on the stream as HIP errors.
 *   - Results are bitwise reproducible run to run (no floating-point atomics).
 *   - For the wider nets (d = 64: GELU MLP with dh > 128, SwiGLU with
 *     dh > 64; d = 128: dh > 64) each unit is split over two to eight
 *     workgroups that swap partial sums through the workspace (or the
 *     backward scratch); those
 *     kernels are launched cooperatively, so a call may wait for the whole
 *     device.  Calls that share a workspace or scratch buffer must not run
 *     concurrently.
 *
 * Tensor layouts (row-major, C order):
 *   q, k, v, out, d_out, dq, dk, dv : [B][H][T][d]   element type desc.io
 *   eta, beta, gamma, d_eta, ...    : [B][H][T]      float32
 *   w_*, m_*, d_w_*, d_m_*          : [B][H][P]      float32, P parameters per unit
 * Packing of the P fast-weight parameters of one unit (row-major, W x rule):
 *   GELU MLP : W1[dh][d], then W2[d][dh]                       P = 2 d dh
 *   SwiGLU   : Wg[dh][d], then Wu[dh][d], then Wd[d][dh]        P = 3 d dh
 *   (Wg, Wu, Wd are the paper's W1, W2, W3 of the SwiGLU net.)
 *
 * Supported shapes: io = BF16 with d = 64 (dh <= 256 for the MLP, <= 192 for
 * SwiGLU) or d = 128 (dh <= 512), or io = F32 with d = 16
 * (dh <= 128); dh is padded inside the library to a multiple of 16;
 * 1 <= chunk <= 512 (the paper's C = 512), forward and backward; a chunk
 * longer than the kernels' token tile (64 rows, 32 at d = 128) runs as
 * tiles that all take gradients and outputs at the chunk-start weights (one
 * after the other, or, where that is faster, all at once by two launches
 * per chunk); T >= 1 with a ragged last chunk of T mod chunk tokens allowed
 * (Prop. 1 holds for any chunk length).
 * bf16 tensors use MFMA bf16 operands with fp32 accumulation and fp32 state;
 * f32 tensors use fp32 MFMA throughout.  Anything else returns
 * E2TTT_ERR_UNSUPPORTED.
 */
#ifndef E2TTT_H
#define E2TTT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  E2TTT_OK = 0,
  E2TTT_ERR_NULL_ARG = 1,              /* a required pointer is NULL             */
  E2TTT_ERR_BAD_SHAPE = 2,             /* a size is <= 0 or inconsistent          */
  E2TTT_ERR_UNSUPPORTED = 3,           /* valid but outside the supported set     */
  E2TTT_ERR_WORKSPACE_TOO_SMALL = 4,   /* workspace / scratch smaller than needed */
  E2TTT_ERR_HIP = 5,                   /* a HIP launch failed                     */
  E2TTT_ERR_DEVICE = 6                 /* a bounded device-side wait expired      */
} e2ttt_status;
/* E2TTT_ERR_DEVICE: a bounded wait between the workgroups of a unit expired
 * (after 2 s, or the limit set by E2TTT_WAIT_LIMIT_US), the grid was drained
 * and the results of that call are undefined.  The kernels record it in a
 * status word of the workspace (forward) or scratch (backward) buffer;
 * e2ttt_wait_status reads it.  With the environment variable
 * E2TTT_DEBUG_SYNC=1 (read at every call) every call also waits for its
 * kernels and returns it. */

typedef enum { E2TTT_FW_GELU_MLP = 0, E2TTT_FW_SWIGLU = 1 } e2ttt_fw;

/* Element type of q, k, v, out, d_out, dq, dk, dv. */
typedef enum { E2TTT_DT_F32 = 0, E2TTT_DT_BF16 = 1 } e2ttt_dtype;

/* f(x) = y (the bare matrix net) instead of f(x) = x + LN(y). */
#define E2TTT_FLAG_NO_RESIDUAL_LN 0x1u
/* Chunk-averaged update rule instead of the closed form of Prop. 1: the
 * ablation baseline of Sec. 5 (Tables 4 and 5) that collapses the per-token
 * momentum and decay factors of a chunk to their means, after the chunk-level
 * momentum of eqs. (4)-(5).  Per chunk of L tokens, with beta_bar and
 * gamma_bar the means of beta_t and gamma_t over the chunk (gamma NULL:
 * gamma_bar = 1, which is eqs. (4)-(5) exactly):
 *   M_C = beta_bar M_0 + sum_t eta_t G_t,   W_C = gamma_bar W_0 + M_C,
 * that is K^W_t = K^M_t = eta_t and carry (gamma_bar, beta_bar, beta_bar).
 * Outputs, gradients and every other convention are unchanged (all entry
 * points that take a descriptor honour the flag). */
#define E2TTT_FLAG_CHUNK_AVERAGED 0x2u
/* Learnable LayerNorm affine of the fast-weight net (Sec. 4's LayerNorm with
 * an elementwise weight and bias per head, slow weights shared by the batch):
 *   f(x) = x + a * LN(y) + b,   a, b in R^d per head.
 * Calls with this flag take a and b (and return their gradients) through the
 * *_ln entry points below; the plain entry points return E2TTT_ERR_NULL_ARG
 * for it.  Not combinable with E2TTT_FLAG_NO_RESIDUAL_LN (E2TTT_ERR_BAD_SHAPE). */
#define E2TTT_FLAG_LN_AFFINE 0x4u
/* Post-chunk L2 normalisation of the fast weights (App. B.1, after LaCT): at
 * every chunk end, after the update of Prop. 1, each row of each fast-weight
 * matrix, taken over the matrix's input dimension (W1 / Wg / Wu: a hidden
 * unit's d weights; W2 / Wd: an output's dh weights), is rescaled to the norm
 * of the same row of the unit's initial weights w_in; a row of norm zero is
 * left as it is, the momentum is not normalised.  Chunk-start states, outputs
 * and w_out are then those of the normalised weights; the backward includes
 * the normalisation and its targets' dependence on w_in.  (The paper gives no
 * axis or target; this is the reading taken.  Off by default: with it the
 * closed form no longer equals the plain token recurrence.) */
#define E2TTT_FLAG_POST_NORM 0x8u

typedef struct {
  int32_t B, H, T;      /* batch, heads, tokens                        */
  int32_t d, dh;        /* head dim, fast-weight hidden width          */
  int32_t chunk;        /* chunk length C                              */
  int32_t fw;           /* e2ttt_fw                                    */
  int32_t io;           /* e2ttt_dtype                                 */
  uint32_t flags;       /* E2TTT_FLAG_*                                */
  float ln_eps;         /* LayerNorm epsilon (> 0 unless NO_RESIDUAL_LN) */
} e2ttt_desc;

/* Parameters per unit (P above), or 0 for a bad descriptor. */
size_t e2ttt_param_count(const e2ttt_desc* desc);

/* Bytes of `workspace` that e2ttt_chunk_forward needs.  With
 * save_for_backward != 0 the workspace also keeps what the backward reuses
 * (per-token scalar kernels, chunk-start checkpoints of W and M in the
 * operand precision, the LayerNorm outputs and inverse deviations of the key
 * and query passes, and either every chunk's W in the orders in which the
 * kernels multiply by it or, for the GELU MLP, the query-side activations and
 * GELU derivatives; the former, of up to 16 GiB, where that is faster), and the
 * same buffer, untouched, must then be passed to e2ttt_chunk_backward.  A
 * workspace of that size also serves calls that do not save.  Returns 0 for a
 * bad descriptor. */
size_t e2ttt_workspace_bytes(const e2ttt_desc* desc, int save_for_backward);

/* Bytes of `scratch` that e2ttt_chunk_backward needs (0 for a bad descriptor). */
size_t e2ttt_backward_scratch_bytes(const e2ttt_desc* desc);

/*
 * Forward: Algorithm 1 over every chunk of every unit.
 *   q, k, v   [B][H][T][d] io     queries, keys, values (k, v feed the inner
 *                                 loss, q the outputs)
 *   eta, beta [B][H][T]   f32     learning rate and momentum gates, eq. (7)
 *   gamma     [B][H][T]   f32     decay gate; NULL means gamma = 1
 *   w_in      [B][H][P]   f32     initial fast weights W (chunk-start state of chunk 0)
 *   m_in      [B][H][P]   f32     initial momentum M; NULL means zero
 *   out       [B][H][T][d] io     o_t = f_{W_0}(q_t) with W_0 the start state of t's chunk
 *   w_out, m_out [B][H][P] f32    state after the last token
 *   workspace, workspace_bytes    caller-owned device memory, at least
 *                                 e2ttt_workspace_bytes(desc, save_for_backward)
 * w_out / m_out may alias w_in / m_in only when save_for_backward == 0.
 * q, k, v, out and workspace must be 16-byte aligned (else E2TTT_ERR_BAD_SHAPE).
 */
e2ttt_status e2ttt_chunk_forward(const e2ttt_desc* desc, const void* q, const void* k,
                                 const void* v, const float* eta, const float* beta,
                                 const float* gamma, const float* w_in, const float* m_in,
                                 void* out, float* w_out, float* m_out, void* workspace,
                                 size_t workspace_bytes, int save_for_backward, void* stream);

/*
 * Backward of  sum_t <d_out_t, o_t> + <d_w_out, W_T> + <d_m_out, M_T>
 * with respect to every input of the forward (reverse mode through the chunk
 * chain; the paper trains with autograd through the same computation).
 *   q .. m_in         the forward's inputs, unchanged
 *   workspace         as left by e2ttt_chunk_forward(..., save_for_backward = 1)
 *   d_out             [B][H][T][d] io   gradient of the outputs
 *   d_w_out, d_m_out  [B][H][P] f32     gradient of the final state; NULL = zero
 *   dq, dk, dv        [B][H][T][d] io
 *   d_eta, d_beta     [B][H][T] f32
 *   d_gamma           [B][H][T] f32; must be NULL iff gamma is NULL
 *   d_w_in, d_m_in    [B][H][P] f32     gradient of the initial state
 *   scratch           at least e2ttt_backward_scratch_bytes(desc) bytes
 * q, k, v, workspace, d_out, dq, dk, dv and scratch must be 16-byte aligned
 * (else E2TTT_ERR_BAD_SHAPE).
 */
e2ttt_status e2ttt_chunk_backward(const e2ttt_desc* desc, const void* q, const void* k,
                                  const void* v, const float* eta, const float* beta,
                                  const float* gamma, const float* w_in, const float* m_in,
                                  const void* workspace, size_t workspace_bytes,
                                  const void* d_out, const float* d_w_out, const float* d_m_out,
                                  void* dq, void* dk, void* dv, float* d_eta, float* d_beta,
                                  float* d_gamma, float* d_w_in, float* d_m_in, void* scratch,
                                  size_t scratch_bytes, void* stream);

/*
 * Scalar kernels of every chunk (Prop. 1, eq. (9)-(11)), exposed on their own
 * so that callers (and tests) can inspect them:
 *   kw, km      [B][H][T] f32   K^W_t = eta_t b~_t R_t and K^M_t = eta_t b~_t
 *   carry       [B][H][NC][3] f32, NC = ceil(T / chunk): (g~_0, b~_0 R_1, b~_0)
 * gamma NULL means gamma = 1.
 */
e2ttt_status e2ttt_chunk_coeffs(const e2ttt_desc* desc, const float* eta, const float* beta,
                                const float* gamma, float* kw, float* km, float* carry,
                                void* stream);

/*
 * Net evaluation at a given state: out_t = f_W(q_t) for T tokens per unit, all
 * at the unit's one state W.  This is how a token's output is formed (eq. (6):
 * the net at the start state of the token's chunk, Table 1), exposed for
 * streaming decode: while a chunk fills, each arriving token is answered from
 * the current chunk-start state with this call (T = 1), and once C tokens have
 * arrived e2ttt_chunk_forward over those C tokens (w_in, m_in = the current
 * state) gives the next chunk-start state.  Outputs and states then agree
 * with those of one e2ttt_chunk_forward over the whole sequence within the
 * bf16 / fp32 tolerances (the two evaluate GELU's Phi differently, above).
 *   desc   as for the chunk calls (same supported set); desc.T is the number
 *          of tokens per unit to evaluate; desc.chunk is checked but unused
 *   q      [B][H][T][d] io
 *   w      [B][H][P]   f32, 16-byte aligned (else E2TTT_ERR_BAD_SHAPE)
 *   out    [B][H][T][d] io; may not overlap q or w
 * fp32 arithmetic on the fp32 state (GELU through erff); no workspace.
 */
e2ttt_status e2ttt_apply(const e2ttt_desc* desc, const void* q, const float* w, void* out,
                         void* stream);

/*
 * Gate parameterization of Sec. 4 ("Input-Dependent Dynamics", eqs. (12)-(14)):
 * per token, from the outputs l_eta, l_beta, l_alpha of the three linear heads,
 *   eta   = eta_base * sigmoid(l_eta)                       (12)
 *   beta  = sigmoid(l_beta)^(1 / tau)                       (13)
 *   alpha = alpha_base * sigmoid(l_alpha),  gamma = 1 - eta * alpha   (14)
 * (the paper trains with eta_base = 0.01, tau = 32, alpha_base = 0.1, App. B.1).
 * The outputs are the gate arrays e2ttt_chunk_forward takes, and the backward
 * maps the gate gradients e2ttt_chunk_backward returns to the logits.
 *   n                       number of tokens (B H T); 0 is a no-op
 *   l_eta, l_beta, l_alpha  [n] f32 device arrays; l_alpha NULL means no decay
 *                           gate (gamma = 1): gamma, d_gamma and d_l_alpha must
 *                           then be NULL too
 *   eta, beta, gamma        [n] f32 outputs
 * Errors: a required pointer NULL (or one of the alpha-side pointers given
 * without l_alpha) -> E2TTT_ERR_NULL_ARG; n < 0, tau <= 0 or a negative or
 * non-finite base -> E2TTT_ERR_BAD_SHAPE.  Caller-owned buffers, no workspace.
 */
typedef struct {
  float eta_base;    /* >= 0 */
  float alpha_base;  /* >= 0 */
  float tau;         /* > 0 */
} e2ttt_gate_params;

e2ttt_status e2ttt_gates_forward(const e2ttt_gate_params* params, int64_t n, const float* l_eta,
                                 const float* l_beta, const float* l_alpha, float* eta,
                                 float* beta, float* gamma, void* stream);

/* Backward of e2ttt_gates_forward: given d_eta, d_beta, d_gamma [n] f32 (for
 * example from e2ttt_chunk_backward), the gradients d_l_eta, d_l_beta,
 * d_l_alpha [n] f32 of the logits.  Same pointer rules as the forward. */
e2ttt_status e2ttt_gates_backward(const e2ttt_gate_params* params, int64_t n,
                                  const float* l_eta, const float* l_beta, const float* l_alpha,
                                  const float* d_eta, const float* d_beta, const float* d_gamma,
                                  float* d_l_eta, float* d_l_beta, float* d_l_alpha,
                                  void* stream);

/*
 * Status of the bounded waits between the workgroups of a unit in the last
 * e2ttt_chunk_forward that used `workspace` and the last e2ttt_chunk_backward
 * that used `scratch` (either may be NULL, not both).  Waits for `stream`
 * first (the calls must have been enqueued there or be complete), then reads
 * the status words: E2TTT_ERR_DEVICE when a wait of either call expired (its
 * results are undefined), E2TTT_OK otherwise (always for descriptors that run
 * one workgroup per unit).  Each call clears its buffer's word when it starts.
 * The wait limit is 2 s; the environment variable E2TTT_WAIT_LIMIT_US (a
 * decimal count of microseconds, read at every call) sets another; a limit of
 * 0 makes every wait give up before it reads the peer's flag, which lets a
 * test force the expiry without any kernel failing.
 */
e2ttt_status e2ttt_wait_status(const e2ttt_desc* desc, const void* workspace,
                               const void* scratch, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * e2ttt_chunk_forward with save_for_backward = 0 on a workspace the library
 * owns, a device array of E2TTT_STATIC_WORKSPACE_BYTES on each GPU it runs
 * on, held until the process ends.  Inputs, outputs and their rules are those
 * of e2ttt_chunk_forward.  Where the faster kernels' workspace
 * (e2ttt_workspace_bytes(desc, 0)) exceeds E2TTT_STATIC_WORKSPACE_BYTES, the
 * call runs on those that need least; a descriptor too large for them as well
 * returns E2TTT_ERR_WORKSPACE_TOO_SMALL before anything is launched.  The call
 * allocates nothing.  Every call on a GPU shares that GPU's array: calls that
 * overlap on one GPU race (enqueue them on one stream, or wait between them).
 * e2ttt_wait_status cannot read its status word (the array is the library's);
 * E2TTT_DEBUG_SYNC=1 reports an expired wait from the call itself.
 */
#define E2TTT_STATIC_WORKSPACE_BYTES ((size_t)64 << 20)
e2ttt_status e2ttt_chunk_forward_static(const e2ttt_desc* desc, const void* q, const void* k,
                                        const void* v, const float* eta, const float* beta,
                                        const float* gamma, const float* w_in, const float* m_in,
                                        void* out, float* w_out, float* m_out, void* stream);

/*
 * The chunk calls and the net evaluation with the learnable LayerNorm affine
 * (E2TTT_FLAG_LN_AFFINE in desc.flags): the same arguments as e2ttt_chunk_forward,
 * e2ttt_chunk_backward and e2ttt_apply, plus
 *   ln_weight, ln_bias    [H][d] f32 device arrays: a and b of each head (unit
 *                         (b, h) uses row h); required with the flag
 *   d_ln_weight, d_ln_bias [H][d] f32 (backward only): the gradients of a and b,
 *                         summed over the batch and all tokens (overwritten)
 * Without the flag every one of these pointers must be NULL, and the calls
 * equal the plain ones.  The backward's scratch (e2ttt_backward_scratch_bytes,
 * which reads the flag) then also holds, per token row, the adjoint the
 * affine's gradients are summed from, and one partial sum per block of 256
 * tokens; ln_weight and ln_bias must be 16-byte aligned (else E2TTT_ERR_BAD_SHAPE).
 */
e2ttt_status e2ttt_chunk_forward_ln(const e2ttt_desc* desc, const float* ln_weight,
                                    const float* ln_bias, const void* q, const void* k,
                                    const void* v, const float* eta, const float* beta,
                                    const float* gamma, const float* w_in, const float* m_in,
                                    void* out, float* w_out, float* m_out, void* workspace,
                                    size_t workspace_bytes, int save_for_backward, void* stream);
e2ttt_status e2ttt_chunk_backward_ln(const e2ttt_desc* desc, const float* ln_weight,
                                     const float* ln_bias, const void* q, const void* k,
                                     const void* v, const float* eta, const float* beta,
                                     const float* gamma, const float* w_in, const float* m_in,
                                     const void* workspace, size_t workspace_bytes,
                                     const void* d_out, const float* d_w_out,
                                     const float* d_m_out, void* dq, void* dk, void* dv,
                                     float* d_eta, float* d_beta, float* d_gamma, float* d_w_in,
                                     float* d_m_in, float* d_ln_weight, float* d_ln_bias,
                                     void* scratch, size_t scratch_bytes, void* stream);
e2ttt_status e2ttt_apply_ln(const e2ttt_desc* desc, const float* ln_weight, const float* ln_bias,
                            const void* q, const float* w, void* out, void* stream);

/*
 * Gated delta rule: the fast weight of a linear net f(x) = W x, updated by
 * every token at the weights the token before left (where the chunk calls take
 * a chunk's gradients at its start).  Per unit (sequence b, value head h), with
 * gamma_t = exp(log_gamma_t) and W [dv][dk]:
 *   e_t = v_t - gamma_t W_{t-1} k_t
 *   W_t = gamma_t W_{t-1} + eta_t e_t k_t^T
 *   o_t = scale W_t q_t                        (the state after the token)
 * H value heads share HK key heads in groups: value head h reads the queries
 * and keys of key head h / (H / HK).  Keys are expected of about unit length
 * with 0 <= eta <= 1 (eta |k|^2 <= 2): beyond that the rule itself diverges.
 *
 * Layouts: q, k [B][HK][T][dk] and v, out [B][H][T][dv] in desc.io; eta and
 * log_gamma [B][H][T] f32; states [B][H][dv][dk] f32, contiguous.  log_gamma
 * NULL: gamma = 1; -inf clears a finite state; growth (above 0) is taken while
 * its sums over neighbouring tokens stay below 88, where exp leaves fp32.  (The
 * chunk calls and e2ttt_gates_forward have gamma itself: its logarithm goes here.)
 * Token tensors and gates may have any non-negative strides
 * (e2ttt_delta_strides, in elements; the last dimension is contiguous), for
 * example those of a projection's [B][T][H][d]; strides NULL means C order.
 * Rows of the io type start on 16 bytes, tokens are at most 2^23 elements
 * apart, and elements of a written tensor do not overlap (else
 * E2TTT_ERR_BAD_SHAPE).
 * lengths [B] int32 (device; NULL: all T): tokens of sequence b at and after
 * lengths[b] (clamped to 0..T) are not read and do not touch the state; their
 * outputs and gradients are written as zero.
 * Supported: dk <= 128 and dv <= 256, multiples of 8, either io type, T >= 1,
 * B H up to 1.9 million units (more of dv <= 64) and 10^9 chunks of 64 tokens,
 * 7.8 million to train (else E2TTT_ERR_UNSUPPORTED).
 *
 * Precision: fp32 throughout, bf16 outputs rounded once.  (With bf16 tensors an
 * fp32 value enters the matrix products as the sum of three bf16 numbers, which
 * loses nothing; of a product of two such values at most 2^-23 is left out.)
 * Within a chunk of 64 tokens (0..63, 64..127, ...) a token with a non-finite
 * value may make the outputs of its whole chunk non-finite, as it does those
 * after it.
 */
typedef struct { int64_t b, h, t; } e2ttt_strides;

typedef struct {
  int32_t B;            /* sequences                                       */
  int32_t HK, H;        /* key heads, value heads (a multiple of HK)       */
  int32_t T;            /* tokens                                          */
  int32_t dk, dv;       /* head dims of keys and values                    */
  int32_t io;           /* e2ttt_dtype                                     */
  float scale;          /* of the outputs                                  */
} e2ttt_delta_desc;

/* The strides of each tensor of the delta calls (those of a call's other
 * tensors are not looked at). */
typedef struct {
  e2ttt_strides q, k, v, out, eta, log_gamma;
  e2ttt_strides d_out, dq, dk, dv, d_eta, d_log_gamma;
} e2ttt_delta_strides;

/* Bytes of `workspace` for e2ttt_delta_forward and of `scratch` for
 * e2ttt_delta_backward (0 for a bad descriptor).  Without save_for_backward at
 * most 704 MiB and one state per unit (more only where a single chunk of every
 * unit needs it); with it the workspace keeps, per unit and chunk, the
 * chunk-start state and what the backward reuses, and must be passed to
 * e2ttt_delta_backward untouched. */
size_t e2ttt_delta_workspace_bytes(const e2ttt_delta_desc* desc, int save_for_backward);
size_t e2ttt_delta_scratch_bytes(const e2ttt_delta_desc* desc);

/* The rule over T tokens of every unit from w_in (NULL: zero) to w_out (NULL:
 * not wanted; may be w_in itself). */
e2ttt_status e2ttt_delta_forward(const e2ttt_delta_desc* desc, const e2ttt_delta_strides* strides,
                                 const void* q, const void* k, const void* v, const float* eta,
                                 const float* log_gamma, const int32_t* lengths,
                                 const float* w_in, void* out, float* w_out, void* workspace,
                                 size_t workspace_bytes, int save_for_backward, void* stream);

/* Backward of  sum_t <d_out_t, o_t> + <d_w_out, W_T>  (d_w_out NULL: zero)
 * with the forward's inputs and its workspace (saved, untouched).  dq, dk are
 * summed over the value heads of a group.  d_log_gamma is NULL iff log_gamma
 * is; d_w_in [B][H][dv][dk] NULL: not wanted. */
e2ttt_status e2ttt_delta_backward(const e2ttt_delta_desc* desc,
                                  const e2ttt_delta_strides* strides, const void* q,
                                  const void* k, const void* v, const float* eta,
                                  const float* log_gamma, const int32_t* lengths,
                                  const void* workspace, size_t workspace_bytes,
                                  const void* d_out, const float* d_w_out, void* dq, void* dk,
                                  void* dv, float* d_eta, float* d_log_gamma, float* d_w_in,
                                  void* scratch, size_t scratch_bytes, void* stream);

/* The recurrent form, for decode: the T (few) arriving tokens of every
 * sequence, in fp32 arithmetic, on states w [n_slots][H][dv][dk] that are
 * updated in place.  Sequence b is at state slots[b] (int32, device; NULL: b,
 * with n_slots >= B).  A slot outside 0..n_slots-1 is skipped: its outputs are
 * zero.  Rows of the batch that name the same slot are taken in their order.
 * The state is read and written once whatever T; no workspace. */
e2ttt_status e2ttt_delta_step(const e2ttt_delta_desc* desc, const e2ttt_delta_strides* strides,
                              const void* q, const void* k, const void* v, const float* eta,
                              const float* log_gamma, float* w, const int32_t* slots,
                              int32_t n_slots, void* out, void* stream);

/*
 * Preparation of queries and keys (Sec. 4: SiLU and unit length before the
 * fast-weight net), with rotary positions, for the chunk calls and the delta
 * calls.  Per row x of d elements, each step optional:
 *   E2TTT_QK_SILU   s = x sigmoid(x)
 *   E2TTT_QK_UNIT   y = s / sqrt(sum s^2 + eps)
 *   rot > 0         the first rot (even) elements of y turn in pairs:
 *                     z_a = rot_scale (y_a cos - y_b sin)
 *                     z_b = rot_scale (y_b cos + y_a sin)
 *                   pair p of rot / 2 turns by position * inv_freq[p]; it is
 *                   (p, p + rot / 2), or (2 p, 2 p + 1) with
 *                   E2TTT_QK_INTERLEAVED.  The other elements pass.
 *   q [B][H][T][d], k [B][HK][T][d] io   (HK = 0: queries alone, k and k_out NULL)
 *   inv_freq [rot / 2] f32   frequencies, as scaled for the context (with
 *                   rot_scale its factor on the turned elements, else 1)
 *   positions [B][T] int64   NULL: 0 .. T - 1; angles are formed in 64 bits
 * Outputs may be the inputs themselves (same strides).  Strides as for the
 * delta calls.  Supported: d <= 256, a multiple of 8, either io type, up to 10^9
 * rows, and B T ceil((H + HK) / 8) L < 2^32 - 255 (else E2TTT_ERR_UNSUPPORTED).  L,
 * the lanes of a row, is d / (2 V) rounded up to a power of two, 64 at most; V, the
 * elements of an access, is the largest of 8 (bf16), 4, 2 and 1 that divides rot / 2.
 * (One head of bf16, d = rot = 128: 2^29 rows are too many.  An odd rot / 2 is
 * taken an element at a time: half as long again as its neighbours.)
 */
#define E2TTT_QK_SILU 0x1u
#define E2TTT_QK_UNIT 0x2u
#define E2TTT_QK_INTERLEAVED 0x4u

typedef struct {
  int32_t B, H, HK, T;  /* sequences, query heads, key heads, tokens */
  int32_t d, rot;       /* head dim, elements that turn              */
  int32_t io;           /* e2ttt_dtype                               */
  uint32_t flags;       /* E2TTT_QK_*                                */
  float eps;            /* at least 2^-126 with E2TTT_QK_UNIT        */
  float rot_scale;
} e2ttt_qk_desc;

typedef struct {
  e2ttt_strides q, k, q_out, k_out;
  e2ttt_strides d_q_out, d_k_out, dq, dk;
} e2ttt_qk_strides;

e2ttt_status e2ttt_qk_forward(const e2ttt_qk_desc* desc, const e2ttt_qk_strides* strides,
                              const void* q, const void* k, const float* inv_freq,
                              const int64_t* positions, void* q_out, void* k_out, void* stream);

/* Gradients of q and k from those of the outputs.  q and k are the forward's
 * inputs (not its outputs); without SILU and UNIT they are not read and may be
 * NULL. */
e2ttt_status e2ttt_qk_backward(const e2ttt_qk_desc* desc, const e2ttt_qk_strides* strides,
                               const void* q, const void* k, const float* inv_freq,
                               const int64_t* positions, const void* d_q_out,
                               const void* d_k_out, void* dq, void* dk, void* stream);

/* Static description of a status code. */
const char* e2ttt_status_str(e2ttt_status status);

#ifdef __cplusplus
}
#endif

#endif /* E2TTT_H */
