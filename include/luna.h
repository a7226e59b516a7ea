/*
 * luna.h — C ABI of the GB300 (sm_103a) LUNA attention library.
 *
 * LUNA (arXiv 2512.08061) is kernelized linear attention with a learned
 * feature map
 *
 *     phi(x) = (1/sqrt(M)) [ psi_l(w_i^T x + b_i) ]_{i<M, l<L}  in R^{D},  D = M*L
 *
 * (Eq. phi-def-scalarenv with the default envelope h = 1 of Sec. 5.4 /
 * Table 5; projection bias b and feature index i*L + l as in the appendix
 * listing), where each channel function is a scalar ReLU MLP
 *
 *     psi_l(u) = relu( sum_k w2[l,k] relu(w1[l,k] u + b1[l,k]) + b2[l] )
 *
 * (listing: ScalarMLP with hidden width `hidden`, act = ReLU, nonneg = True,
 * one MLP per channel).  Attention is Eq. (kernel-attn):
 *
 *     O_i = phi(q_i)^T S / (phi(q_i)^T z + eps),  S = sum_j phi(k_j) v_j^T,  z = sum_j phi(k_j)
 *
 * with the sums over all valid keys (non-causal) or over j <= i (the streaming
 * form named in the abstract and Sec. 3.2).  S and z are the key-side
 * sufficient statistics S_KV and S_K1 of Sec. 4.
 *
 * Conventions for every entry point:
 *   - All tensor pointers are DEVICE pointers owned by the caller.  The
 *     library never allocates device memory and keeps no state between calls
 *     except a per-process cache of the driver entry point it needs for TMA.
 *   - Q, K, dQ, dK are contiguous (B, H, n, d); V, O, dO, dV are contiguous
 *     (B, H, n, dv), element type `io` (fp32 or bf16).  Row-major, C order.
 *   - `lengths` is NULL (every sequence has n valid tokens) or a device array
 *     of B int32 valid lengths (right padding).  Values are clamped to [0, n].
 *     Keys at or beyond the length do not enter S and z; query rows at or
 *     beyond it produce O = 0 and receive dQ = dK = dV = 0.
 *   - `stream` is a cudaStream_t passed as void* (NULL = legacy default stream).
 *     Every call only enqueues work on it and returns without synchronising.
 *   - Argument errors are reported before anything is launched.  A failed
 *     launch returns LUNA_ERR_CUDA.  Device-side bounded waits that gave up
 *     are reported by luna_device_status().
 *   - Computation: the feature map is evaluated in fp32 for both io types
 *     (the listing casts the projections to float before the channel MLPs).
 *     Accumulations are fp32.  With io = bf16 the tensor-core contractions take
 *     bf16 operands; the normaliser phi(q)^T z is always an fp32 dot product.
 */
#ifndef LUNA_H
#define LUNA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LUNA_OK = 0,
    LUNA_ERR_INVALID_ARG = 1,    /* NULL pointer, negative size, bad enum            */
    LUNA_ERR_UNSUPPORTED = 2,    /* valid but outside the supported shape range     */
    LUNA_ERR_WORKSPACE = 3,      /* workspace / table / state buffer too small      */
    LUNA_ERR_CUDA = 4,           /* a CUDA runtime call or launch failed            */
    LUNA_ERR_DEVICE_TIMEOUT = 5  /* a bounded device-side wait gave up              */
} luna_status;

typedef enum { LUNA_F32 = 0, LUNA_BF16 = 1 } luna_dtype;

/* Hidden-unit activation of the channel MLPs (the listing's ScalarMLP `act`):
 * ReLU is the listing's default and the only one with the exact
 * piecewise-linear table; the others are evaluated directly.
 * GELU(a) = a Phi(a) (Phi: the standard normal distribution function, the erf
 * form), SiLU(a) = a / (1 + e^-a), tanh. */
typedef enum { LUNA_ACT_RELU = 0, LUNA_ACT_GELU = 1, LUNA_ACT_SILU = 2, LUNA_ACT_TANH = 3 } luna_act;

/* Shape of the feature map (Eq. phi-def-scalarenv; listing defaults hidden = 64).
 * shared_channels = 0: one scalar MLP per channel (the listing's default);
 * 1: one scalar MLP with L outputs serves all channels (the listing's
 * shared_channels = True: fc1 Linear(1, hidden) shared, fc2 Linear(hidden, L)).
 * ch_rms_target > 0 turns on the listing's channel RMS normalisation
 * (ch_rms): each application of the feature map, once to all queries and once
 * to all keys of the batch, scales channel l of the MLP outputs y_l by
 * s_l = min(target / (rms_l + 1e-6), 1), rms_l = sqrt(mean y_l^2 + 1e-6) over
 * every valid row (rows at or past a sequence's length excluded) and every
 * projection; the backward pass includes the dependence of s_l on every
 * sample.  0 = off (the listing's default); negative, NaN or infinite is
 * LUNA_ERR_INVALID_ARG.  With it on, luna_attn_fwd / luna_attn_bwd support
 * both forms (the streaming form runs on a copy of the table, in the
 * workspace, whose channel-l coefficients are scaled by sqrt(s^q_l s^k_l));
 * luna_featmap, luna_attn_decode and luna_attn_weights give
 * LUNA_ERR_UNSUPPORTED (a batch statistic has no single-row or single-token
 * form).
 * signed_outputs = 1 is the listing's ScalarMLP(nonneg = False): the channel
 * outputs are fc2(relu(fc1(u))) without the outer ReLU, so features (and kernel
 * values) of either sign; 0 keeps the outer ReLU (the listing's default).  The
 * table is the same for both (the flag is read from the descriptor by every
 * call, so pass the same descriptor to all calls of one problem); with
 * ch_rms_target > 0 it gives LUNA_ERR_UNSUPPORTED.
 * param_head_stride = 0: one parameter set serves every head (the listing's
 * "shared ... over tokens/heads").  > 0: per-head parameters, as in the
 * conversion of a pretrained model, where the feature map's parameters are
 * instantiated per layer and head (appendix, conversion of BERT and ViT):
 * `table` holds ad->H tables, head h's at table + h * param_head_stride bytes
 * (each prepared by luna_phi_prepare from head h's parameters; the stride is
 * at least luna_phi_table_size and a multiple of 256), and luna_attn_bwd
 * writes each head's parameter gradients, summed over the batch only, as
 * arrays with a leading head axis (dW [H][M][d], ..., db2 [H][L]).  The
 * attention calls then run one sub-problem per head index (the B sequences'
 * head h at a time).  Not with ch_rms_target > 0 (LUNA_ERR_UNSUPPORTED); for
 * luna_featmap pass head h's table with a stride of 0.
 * Feature-map variants (the kernel ablation of Sec. 5.4, Table 5; each 0 = off,
 * the paper's default "no gate" map psi):
 *   act (a luna_act): the channel MLPs' hidden activation.  Not ReLU: every
 *     (row, projection) evaluates the L channel MLPs unit by unit, and the
 *     backward pass sums the MLP parameter gradients sample by sample (the
 *     interval histogram needs a piecewise-linear MLP).
 *   envelope = 1: the envelope-gated map phi(x) = h(x) (.) psi(x), channel l
 *     of every projection multiplied by the tokenwise gate
 *     h_l(x) = sigmoid(We_l . x + be_l) in (0, 1) (We, be in luna_phi_params;
 *     their gradients dWe, dbe in luna_phi_grads).
 *   bank_coef = 1: Bank+Coef, channel l of every projection multiplied by a
 *     learned global coefficient c_l (coef; gradient dcoef): an input-agnostic
 *     reweighting of the bank of channel functions that keeps the feature
 *     dimension M*L (a negative c_l gives features of either sign).
 *   They combine with each other and with shared_channels and signed_outputs;
 *   any of them runs the attention calls on the generic (CUDA-core) kernels and
 *   gives LUNA_ERR_UNSUPPORTED with ch_rms_target > 0, with param_head_stride,
 *   and in luna_attn_decode and luna_attn_weights.  The
 *   table holds the gate and coefficient parameters, so pass the same
 *   descriptor to every call of one problem.
 * Supported: 1 <= M, 1 <= L <= 16, M*L <= 128, 1 <= hidden <= 128, L*hidden <= 512. */
typedef struct {
    int M;               /* number of projections w_i (rows of W)       */
    int L;               /* number of channel functions psi_l           */
    int hidden;          /* hidden width of each (or the shared) MLP     */
    int shared_channels; /* 0 or 1, see above                           */
    float ch_rms_target; /* channel RMS normalisation target, 0 = off   */
    int signed_outputs;  /* 0 or 1, see above                           */
    int64_t param_head_stride; /* bytes between heads' tables, 0 = shared  */
    int act;             /* luna_act of the channel MLPs' hidden units   */
    int envelope;        /* 0 or 1: envelope-gated map, see above        */
    int bank_coef;       /* 0 or 1: Bank+Coef channel coefficients       */
} luna_phi_desc;

/* Feature-map parameters, fp32 device arrays, row-major:
 *   W [M][d], b [M], w1 [L][hidden], b1 [L][hidden], w2 [L][hidden], b2 [L];
 *   with shared_channels, w1 and b1 are [hidden] (the one fc1).
 * w1[l][k], b1[l][k] are fc1 of channel l (Linear(1, hidden)); w2[l][k], b2[l]
 * are its fc2 (Linear(hidden, 1)), or row l of the shared fc2. The same
 * parameters serve queries and keys and are shared by all heads (listing:
 * "shared ... over tokens/heads").  The variants' parameters: We [L][d], be [L]
 * (envelope gate; read only with envelope = 1) and coef [L] (read only with
 * bank_coef = 1); NULL when their variant is off. */
typedef struct {
    const float *W, *b, *w1, *b1, *w2, *b2;
    const float *We, *be, *coef;
} luna_phi_params;

/* Gradients of the feature-map parameters, fp32 device arrays with the shapes
 * of luna_phi_params (dw1, db1 of [hidden] with shared_channels).  They are
 * OVERWRITTEN (not accumulated) by luna_attn_bwd.  dWe, dbe (envelope = 1) and
 * dcoef (bank_coef = 1) are required with their variant and ignored without. */
typedef struct {
    float *dW, *db, *dw1, *db1, *dw2, *db2;
    float *dWe, *dbe, *dcoef;
} luna_phi_grads;

/* Problem description (Sec. 3.1: Q, K in R^{n x d}; Sec. 4: values of width d_v).
 * Supported: 1 <= d, dv <= 128; B, H, n >= 0 (an empty problem is a no-op).
 * causal = 1 selects the streaming form (sums over j <= i).  chunk (0, or
 * 16..128 in steps of 16, else LUNA_ERR_INVALID_ARG) is accepted for the
 * interface and otherwise not used: the kernels choose their own tiles (128
 * rows in the tensor-core streaming forward, 64 in its backward, 16 in the
 * generic kernels), and results do not depend on it beyond rounding order.
 * eps >= 0 guards the row normaliser: O_i = num_i / (den_i + eps); a row
 * whose guarded normaliser is exactly 0 produces O_i = 0 and zero gradients. */
typedef struct {
    int B, H, n, d, dv;
    int causal;
    int chunk;
    float eps;
    luna_dtype io;
} luna_attn_desc;

/* Human-readable name of a status code (static string, never NULL). */
const char *luna_status_string(luna_status s);

/* Bytes of the prepared feature-map table for this descriptor and input width d
 * (written to *bytes).  The table is an opaque device blob produced by
 * luna_phi_prepare and consumed by every other call. */
luna_status luna_phi_table_size(const luna_phi_desc *pd, int d, size_t *bytes);

/* Builds the feature-map table from the parameters (Eq. phi-def-scalarenv,
 * listing ScalarMLP): a copy of W and b, and for every channel the exact
 * piecewise-linear form of psi_l.  A ReLU MLP of a scalar is linear between
 * the kinks t = -b1/w1 of its hidden units, so on the merged, sorted kink list
 * psi_l(u) = relu(alpha_{l,j} u + beta_{l,j}) on interval j.  Kinks are
 * placed at the exact fp32 thresholds of fma(w1, u, b1) > 0, so the interval
 * decides every hidden unit exactly as an fp32 evaluation of fc1 would.
 * With a non-ReLU act the table still holds the parameters (the calls
 * evaluate the MLPs from them) and the piecewise form is not used; with
 * envelope or bank_coef it also holds We, be or coef.
 * `table` is a device buffer of at least luna_phi_table_size bytes, 256-byte
 * aligned; it must not be modified while a call that reads it is in flight.
 * Parameters must be finite. */
luna_status luna_phi_prepare(const luna_phi_desc *pd, int d, const luna_phi_params *params, void *table,
                             size_t table_bytes, void *stream);

/* phi(X) for `rows` rows of width d (Eq. phi-def-scalarenv).
 * X: device, rows x d of type `xtype`; Phi: device fp32, rows x (M*L), feature
 * index i*L + l.  Debug / interoperability entry point: the attention calls
 * never materialise phi in memory. */
luna_status luna_featmap(const luna_phi_desc *pd, int d, const void *table, const void *X, luna_dtype xtype,
                         int64_t rows, float *Phi, void *stream);

/* Bytes of scratch memory the calls need (written to *bytes).  `backward`
 * selects the requirement of luna_attn_bwd (0 = luna_attn_fwd).  The caller
 * owns the workspace; its contents on entry are irrelevant and on exit are
 * unspecified.  Must be 256-byte aligned. */
luna_status luna_workspace_size(const luna_attn_desc *ad, const luna_phi_desc *pd, int backward, size_t *bytes);

/* Bytes of the optional forward state (the key statistics S, z of Sec. 4 per
 * head; for the causal form, the prefix statistics at every state segment). */
luna_status luna_state_size(const luna_attn_desc *ad, const luna_phi_desc *pd, size_t *bytes);

/* Forward pass, Eq. (kernel-attn) (causal: streaming form).
 * Q, K, V, lengths, O as in the conventions above.  `table` from
 * luna_phi_prepare.  `state` is NULL or a device buffer of luna_state_size
 * bytes that receives the key statistics for a later luna_attn_bwd.
 * `workspace` holds ws_bytes >= luna_workspace_size(ad, pd, 0). */
luna_status luna_attn_fwd(const luna_attn_desc *ad, const luna_phi_desc *pd, const void *table, const void *Q,
                          const void *K, const void *V, const int32_t *lengths, void *O, void *state,
                          void *workspace, size_t ws_bytes, void *stream);

/* Backward pass of luna_attn_fwd: given dO = dLoss/dO, writes dQ, dK, dV and
 * the parameter gradients `grads` (overwritten) of the same loss.
 * `state` is NULL (the key statistics are recomputed from K and V) or the
 * state written by luna_attn_fwd on the same Q, K, V, lengths and table.
 * The derivative of each ReLU at 0 is taken as 0.  Parameter gradients are
 * summed over all heads, rows and projections.  With pd->ch_rms_target > 0 the
 * channel statistics of Q and K are recomputed by every call, and a `state`
 * must come from luna_attn_fwd with the same descriptors (it holds the
 * normalised key statistics). */
luna_status luna_attn_bwd(const luna_attn_desc *ad, const luna_phi_desc *pd, const void *table, const void *Q,
                          const void *K, const void *V, const void *dO, const int32_t *lengths,
                          const void *state, void *dQ, void *dK, void *dV, const luna_phi_grads *grads,
                          void *workspace, size_t ws_bytes, void *stream);

/* Attention weights of query rows [row0, row0 + rows) of every (b, h), for the
 * conversion of a softmax model (appendix, "Stage 1: attention distillation":
 * the feature-map parameters are trained so that the attention distribution the
 * kernel induces matches the one of the original softmax module; the paper
 * does not fix the loss, so this call only produces the distributions).
 *   teacher = 0: the LUNA weights, Eq. (kernel-attn) read as a weighted average
 *       of the values,  a_ij = k(q_i, k_j) / (sum_j' k(q_i, k_j') + eps),
 *       k(x, y) = phi(x)^T phi(y), so that O_i = sum_j a_ij v_j exactly;
 *   teacher = 1: the softmax weights of the same queries and keys,
 *       p_ij = exp(q_i . k_j / sqrt(d)) / sum_j' exp(q_i . k_j' / sqrt(d))
 *       (`table` may then be NULL).
 * The sums run over the valid keys (j <= i with ad->causal = 1).  Keys outside
 * them, query rows at or past the valid length, and rows whose guarded sum is
 * exactly 0 get weight 0.  Q, K as in the conventions (ad->dv and ad->chunk are
 * ignored); A: fp32 device array (B, H, rows, n), every entry written.
 * 0 <= row0, 0 <= rows, row0 + rows <= n, else LUNA_ERR_INVALID_ARG;
 * pd->ch_rms_target > 0 gives LUNA_ERR_UNSUPPORTED.  No workspace: each block
 * of 32 rows writes its raw scores and normalises them in a second pass over
 * its own rows.  The feature map is fp32 for both io types; each row's sum
 * is accumulated in fp64. */
luna_status luna_attn_weights(const luna_attn_desc *ad, const luna_phi_desc *pd, const void *table, const void *Q,
                              const void *K, const int32_t *lengths, int row0, int rows, int teacher, float *A,
                              void *stream);

/* Location of the final state of a streaming-form forward pass (ad->causal = 1)
 * inside a `state` buffer written by luna_attn_fwd: the key statistics over all
 * valid tokens of each sequence, S = sum_j phi(k_j) v_j^T and z = sum_j phi(k_j)
 * (Eq. kernel-attn, streaming form of Sec. 3.2).  Head (b, h) holds S at
 * *S + (b*H + h) * *S_stride (D x dv fp32, row-major) and z at
 * *z + (b*H + h) * *z_stride (D fp32).  No device memory is touched; the
 * pointers are for luna_attn_decode, which continues each sequence after its
 * last valid token.  LUNA_ERR_INVALID_ARG for a non-causal descriptor or NULL
 * arguments. */
luna_status luna_state_final(const luna_attn_desc *ad, const luna_phi_desc *pd, void *state, float **S,
                             int64_t *S_stride, float **z, int64_t *z_stride);

/* One step of the streaming form (recurrent decode; the abstract and Sec. 3.2
 * name the associative streaming form of Eq. kernel-attn): for every (b, h)
 * and the new token's q, k, v,
 *     S <- S + phi(k) v^T,   z <- z + phi(k),   o = phi(q)^T S / (phi(q)^T z + eps)
 * i.e. the causal output of the token that follows the state's tokens.
 * q, k: (B, H, d); v, o: (B, H, dv), element type ad->io, one token per
 * (b, h); ad->n, ad->causal and ad->chunk are ignored.  S, z: fp32 device
 * arrays updated in place, head (b, h) at S + (b*H + h) * S_stride ([D][dv]
 * row-major) and z + (b*H + h) * z_stride ([D]); a stride of 0 selects the
 * dense layout (D*dv, D), a smaller nonzero stride is LUNA_ERR_INVALID_ARG.
 * A head whose guarded normaliser is exactly 0 produces o = 0.  No workspace;
 * B*H = 0 is a no-op. */
luna_status luna_attn_decode(const luna_attn_desc *ad, const luna_phi_desc *pd, const void *table, const void *q,
                             const void *k, const void *v, void *o, float *S, int64_t S_stride, float *z,
                             int64_t z_stride, void *stream);

/* ---------------------------------------------------------------------------
 * A block of linear attention with decay.  Next to the learned feature map the
 * library holds the three operators such a block is made of, forward and
 * backward: the attention itself (luna_decay_*), the norms before and after a
 * block with its gate and residual scale (luna_norm_*), and the projections
 * (luna_linear_*).  The paper has no counterpart of them.
 *
 * The conventions above hold (device pointers, asynchronous calls, checks before
 * any launch, fp32 sums).  Beyond them, tensors may be views: a stride or leading
 * dimension counts elements, the innermost dimension is contiguous, and inputs
 * may overlap each other or repeat (stride 0) while outputs may not: an output
 * whose strides let two of its elements share an address is
 * LUNA_ERR_INVALID_ARG.  With io = bf16 each output is rounded once. */

/* Strides of a (B, heads, n, width) tensor: batch entry, head, token.  All three
 * 0 stands for the contiguous layout. */
typedef struct {
    int64_t b, h, t;
} luna_strides;

/* Linear attention with a decay for each head.  With lambda_h =
 * exp(log_decay[h]) and the state S (d x dv, fp32) of each (b, h):
 *
 *     S_i = lambda_h S_{i-1} + k_i v_i^T,    o_i = scale * q_i^T S_i
 *
 * H query heads share Hkv heads of keys and values (H a multiple of Hkv): query
 * head h reads head h / (H / Hkv), and every query head has its own decay and
 * state.  log_decay is a device array of H fp32; -inf (lambda = 0: each token
 * sees only itself) and 0 (no decay) are valid, and values above 0 grow without
 * a check.  It takes no gradient.  Rows at or past a sequence's length neither
 * enter the state nor are read; their outputs and gradients are 0.  A value that
 * is not finite in a valid row may reach any valid row of the sequence.
 * Supported: 1 <= d, dv <= 128, n <= 2^24, B * H <= 2^24; empty problems are
 * no-ops (n = 0 copies the initial state).
 * bf16 with d and dv multiples of 8, and every tensor on 16-byte boundaries with
 * strides that are multiples of 8 elements, runs on tensor cores, where scores
 * and states enter products as bf16 roundings (outputs 2.3e-3 to 2.5e-3 off where
 * their own rounding alone leaves 1.7e-3) and the carried state itself stays
 * exact to fp32; everything else runs in fp32 on CUDA cores. */
typedef struct {
    int B, H, Hkv, n, d, dv;
    float scale;
    luna_dtype io;
    luna_strides q, k, v, o;      /* Q, K, V, O                                */
    luna_strides gq, gk, gv, go;  /* dQ, dK, dV, dO (luna_decay_bwd only)      */
} luna_decay_desc;

/* Bytes of scratch memory of luna_decay_fwd (backward = 0) or luna_decay_bwd
 * (1); the workspace must be 256-byte aligned.  The size does not depend on the
 * strides. */
luna_status luna_decay_workspace_size(const luna_decay_desc *dd, int backward, size_t *bytes);

/* Whole prompts.  S0: NULL (zero) or the initial states, fp32 [B][H][d][dv];
 * S1: NULL or the states after each sequence's last valid token, the same
 * layout (S1 may be S0 itself). */
luna_status luna_decay_fwd(const luna_decay_desc *dd, const float *log_decay, const void *Q, const void *K,
                           const void *V, const int32_t *lengths, const float *S0, void *O, float *S1,
                           void *workspace, size_t ws_bytes, void *stream);

/* Gradients of luna_decay_fwd on the same inputs.  dS1: NULL (zero) or the
 * gradient of the final states; dS0: NULL or the gradient of the initial states.
 * The gradients of shared keys and values are summed over their query heads in
 * fp32, in head order.  No atomics: equal inputs give equal bits. */
luna_status luna_decay_bwd(const luna_decay_desc *dd, const float *log_decay, const void *Q, const void *K,
                           const void *V, const void *dO, const int32_t *lengths, const float *S0, const float *dS1,
                           void *dQ, void *dK, void *dV, float *dS0, void *workspace, size_t ws_bytes,
                           void *stream);

/* One token of each of B sequences: S <- lambda S + k v^T, o = scale q^T S, in
 * place in a pool of states, fp32 [nslots][H][d][dv].  slots: NULL (sequence b
 * is slot b) or B int32 in device memory; a sequence whose slot is outside
 * [0, nslots) is idle (o = 0, no state is touched), and no two sequences may
 * share a slot.  q, k, v, o are one token for each head; the strides .b and .h
 * of the descriptor apply (all three 0: contiguous (B, heads, width)) and n and
 * .t are ignored. */
luna_status luna_decay_step(const luna_decay_desc *dd, const float *log_decay, const void *q, const void *k,
                            const void *v, const int32_t *slots, int nslots, float *S, void *o, void *stream);

/* The gated delta rule: linear attention whose state forgets by a gate of each
 * token and takes in the difference between a value and what the state already
 * gives for its key.  With a_t = exp(g_t) and the state S (d x dv, fp32) of each
 * (b, h):
 *
 *     S_t = a_t (S_{t-1} - beta_t k_t (k_t^T S_{t-1})) + beta_t k_t v_t^T,    o_t = scale * S_t^T q_t
 *
 * H heads of values, states and gates share Hk heads of queries and keys (H a
 * multiple of Hk): head h reads head h / (H / Hk).  log_decay (g) and beta are
 * (B, H, n) tensors of type io with strides of their own (g, beta; all three 0:
 * contiguous); g = -inf (a = 0: the state starts anew) is valid and takes a
 * gradient of 0; values above 0 grow without a check, and with bf16 tensors lose
 * their bits where they add up to more than about 10 within 64 tokens.  Keys are
 * meant to have length one and beta to lie in [0, 2]; with beta |k|^2 above 2 the
 * recurrence itself grows, and nothing checks that.
 * Rows at or past a sequence's length neither enter the state nor are read; their
 * outputs and gradients are 0.  A value that is not finite in a valid row may
 * reach any valid row of the sequence.
 * Supported: 1 <= d, dv <= 128, n <= 2^24, B * H <= 2^24, fewer than 2^31 chunks of
 * 64 rows in all; empty problems are no-ops (n = 0 copies the initial state).
 * bf16 runs on tensor cores, in chunks of 64 rows whose operands are scaled fp16
 * values: outputs and gradients are as near to their definition as their own
 * rounding lets them be (1.7e-3; their sums hold operands of 11 bits, some 3e-4),
 * states 3e-7 (one that all but vanishes within 64 tokens 2^-30 of what it and
 * their rows were); what is less than 2^-26 of the largest value of its kind in 64
 * tokens may lose bits.  Rows that start on 16-byte boundaries, with d and dv
 * multiples of 8, are read and written in vectors.
 * fp32 runs on CUDA cores. */
typedef struct {
    int B, H, Hk, n, d, dv;
    float scale;
    luna_dtype io;
    luna_strides q, k, v, o, g, beta;              /* Q, K, V, O, log_decay, beta */
    luna_strides gq, gk, gv, go, gg, gbeta;        /* dQ, dK, dV, dO, dlog_decay, dbeta (luna_delta_bwd only) */
} luna_delta_desc;

/* Bytes of scratch memory of luna_delta_fwd (backward = 0) or luna_delta_bwd
 * (1); the workspace must be 256-byte aligned.  The size does not depend on the
 * strides.  At d = dv = 128 with bf16 tensors it is 58 KB for each 64 tokens of a
 * head (3.6 times one of the tensors), with gradients 178 KB (11 times; up to 48 KB
 * more where heads share queries and keys); with fp32 tensors nothing, and 194 KB. */
luna_status luna_delta_workspace_size(const luna_delta_desc *dd, int backward, size_t *bytes);

/* Whole prompts.  S0: NULL (zero) or the initial states, fp32 [B][H][d][dv];
 * S1: NULL or the states after each sequence's last valid token, the same
 * layout (S1 may be S0 itself). */
luna_status luna_delta_fwd(const luna_delta_desc *dd, const void *log_decay, const void *beta, const void *Q,
                           const void *K, const void *V, const int32_t *lengths, const float *S0, void *O, float *S1,
                           void *workspace, size_t ws_bytes, void *stream);

/* Gradients of luna_delta_fwd on the same inputs.  dS1: NULL (zero) or the
 * gradient of the final states; dS0: NULL or the gradient of the initial states
 * (dS0 may be dS1 itself).  The gradients of shared queries and keys are summed
 * over their heads in fp32, in head order.  No atomics: equal inputs give equal
 * bits. */
luna_status luna_delta_bwd(const luna_delta_desc *dd, const void *log_decay, const void *beta, const void *Q,
                           const void *K, const void *V, const void *dO, const int32_t *lengths, const float *S0,
                           const float *dS1, void *dQ, void *dK, void *dV, void *dlog_decay, void *dbeta, float *dS0,
                           void *workspace, size_t ws_bytes, void *stream);

/* One token of each of B sequences, in place in a pool of states, fp32
 * [nslots][H][d][dv]; slots as in luna_decay_step.  q, k, v, o, log_decay and
 * beta are one token for each head; the strides .b and .h of the descriptor apply
 * (all three 0: contiguous) and n and .t are ignored. */
luna_status luna_delta_step(const luna_delta_desc *dd, const void *log_decay, const void *beta, const void *q,
                            const void *k, const void *v, const int32_t *slots, int nslots, float *S, void *o,
                            void *stream);

/* Beam search over recurrent states: K beams of each of B sequences, a
 * vocabulary of V tokens.
 *
 * luna_beam_select takes the logits of the next token, B * K rows of V (type io,
 * ld elements apart; 0 = V), and the beams' running log-probabilities `scores`
 * (fp32, B x K), and gives the K best of a sequence's candidates
 *
 *     scores[k] + logits[k][t] - log sum_t' exp(logits[k][t'])
 *
 * over all k and t, best first: their scores (fp32), tokens and parent beams
 * (int32, B x K).  Scores are compared in 64 bits; equal ones go by the lower
 * beam, then the lower token.  Within a beam that is the order of its logits as
 * they came.  A row's sum of exponentials is taken in fp32 (off by some 1e-6 in the
 * worst rows, and the same for rows of equal values), so that candidates of
 * different beams nearer to each other than that may come in either order.  A beam
 * of score -inf (one that is not in use yet), with a score or a logit that is NaN
 * or +inf, or whose logits are all -inf, has candidates of score -inf alone, which
 * come behind all others.
 * end: the token that ends a sequence, or -1 (none; done and done_out are then
 * NULL).  done: NULL (none) or B x K bytes, not 0 where a beam has ended: its
 * logits are not read, and its one candidate is itself with the token `end` and
 * the score it has.  done_out: NULL, or where the new beams have ended.
 * scores_out and done_out may be scores and done themselves.
 *
 * luna_beam_reorder lets the states in a pool follow their beams.  The pool has
 * nslots slots of slot_bytes each; slots (int32, B x K) says where each old
 * beam's state is, and new_slots (another array than these) receives where the
 * new beams' states are: the first child of a beam keeps its slot, further
 * children get copies in the slots of beams without a child, in order.  No two
 * beams may share a slot.  Slots outside [0, nslots) are neither read nor written; a parent
 * outside [0, K) stands for none (the beam takes a free slot as it is).  Several
 * pools are reordered by one call each with the same slots; pool may be NULL with
 * slot_bytes = 0 (new_slots alone).
 * Supported: K <= 32, V <= 2^24, B * K <= 65535; B = 0 is a no-op. */
typedef struct {
    int B, K, V;
    luna_dtype io;
    int64_t ld;
    int end;
} luna_beam_desc;

/* Bytes of the workspace of luna_beam_select (256-byte aligned). */
luna_status luna_beam_workspace_size(const luna_beam_desc *bd, size_t *bytes);

luna_status luna_beam_select(const luna_beam_desc *bd, const void *logits, const float *scores, const uint8_t *done,
                             float *scores_out, int32_t *tokens, int32_t *parents, uint8_t *done_out, void *workspace,
                             size_t ws_bytes, void *stream);

luna_status luna_beam_reorder(const luna_beam_desc *bd, const int32_t *parents, const int32_t *slots, int nslots,
                              void *pool, size_t slot_bytes, int32_t *new_slots, void *stream);

/* The norms after and before a block, fused with its gate and its residual
 * scale, over `rows` rows of `cols` values:
 *
 *     u  = norm(y) w_post + b_post    over each of `groups` equal groups of a row
 *     x' = x + alpha * u * act(gate)
 *     h  = norm(x') w_pre + b_pre     over the row
 *
 * norm(z) = z / sqrt(mean(z^2) + eps); the layer kind takes the mean of z out
 * first.  Parts are chosen by their pointers: x NULL (no residual: x' = alpha u
 * act(gate)), y NULL (x' = x, the norm before a first block), w_post NULL (u =
 * y), w_pre NULL (no h), each b NULL (0), and the gate by `gate`.  One call is
 * then a plain norm, the gated norm of an attention's heads (groups = H), or the
 * step from one block's output to the next block's input.
 * x, y, gate and their gradients, x' and h have the type io and a row stride
 * (ld*, in elements; 0 = cols) of at least cols; weights and biases are fp32
 * arrays of cols.  Statistics and sums are fp32; h is computed from x' before
 * its rounding.
 * Supported: cols <= 16384, rows < 2^31; rows = 0 is a no-op. */
typedef enum { LUNA_NORM_RMS = 0, LUNA_NORM_LAYER = 1 } luna_norm_kind;
typedef enum { LUNA_GATE_NONE = 0, LUNA_GATE_SIGMOID = 1, LUNA_GATE_SILU = 2 } luna_gate;

typedef struct {
    int64_t rows;
    int cols, groups;
    luna_norm_kind kind;
    luna_gate gate;
    float alpha, eps;
    luna_dtype io;
    int64_t ldx, ldy, ldgate, ldX, ldH;           /* x, y, gate, x', h            */
    int64_t lddX, lddH, lddx, lddy, lddgate;      /* their gradients (backward)   */
} luna_norm_desc;

/* Bytes of the workspace of luna_norm_bwd (256-byte aligned; the weight
 * gradients' partial sums). */
luna_status luna_norm_workspace_size(const luna_norm_desc *nd, size_t *bytes);

/* X (x') may be NULL where w_pre is given; H is required with w_pre and ignored
 * without.  X and H may be x and y themselves (same strides). */
luna_status luna_norm_fwd(const luna_norm_desc *nd, const void *x, const void *y, const void *gate,
                          const float *w_post, const float *b_post, const float *w_pre, const float *b_pre, void *X,
                          void *H, void *stream);

/* Gradients from dX = dLoss/dx' (NULL: zero; required without w_pre) and dH =
 * dLoss/dh (required with w_pre).  dx, dy, dgate are required where x, y, gate
 * are given; the weight gradients dw_post, db_post, dw_pre, db_pre (fp32, cols,
 * overwritten, summed over the rows in a fixed order) are written where not NULL
 * (db_* also where that bias is absent).  The workspace is not needed without
 * weight gradients. */
luna_status luna_norm_bwd(const luna_norm_desc *nd, const void *x, const void *y, const void *gate,
                          const float *w_post, const float *b_post, const float *w_pre, const void *dX, const void *dH,
                          void *dx, void *dy, void *dgate, float *dw_post, float *db_post, float *dw_pre,
                          float *db_pre, void *workspace, size_t ws_bytes, void *stream);

/* Linear layers with their epilogue in the product:
 *
 *     z = X W^T + bias,   Y = act(z) + R
 *
 * X: m x k, W: n x k, bias: n values, R, Y, Z: m x n, all of type io, rows a
 * leading dimension apart (ld*, in elements; 0 = the row's width, else at least
 * that).  bias and R may be NULL; R may be Y.  Z, where not NULL, receives the
 * pre-activation rounded to io, which luna_linear_bwd needs with an activation.  GELU is the
 * erf form.  Sums are fp32; the tensor cores' additions cut off instead of
 * rounding (1e-4 of a sum of 65536 positive products), so longer sums are joined
 * by rounded additions every 16384 products.
 * bf16 runs on tensor cores (with n or k that is not a multiple of 8 from
 * aligned copies of the operands in the workspace; a matrix that is off a
 * 16-byte boundary, or whose leading dimension is not a multiple of 8, although
 * n and k are, is multiplied on CUDA cores), up to eight rows of X on CUDA
 * cores.  fp32 products large enough to gain from it run on tensor cores too,
 * each operand written to the workspace as three bf16 values that sum to it
 * exactly (6 bytes a value); the result is as close as fp32 sums are (2e-7 of
 * its norm), and operands with an infinity or a NaN go to CUDA cores, where
 * these spread as in any fp32 product.  Small fp32 products run there always.
 * Supported: m <= 2^23, n, k <= 2^20; k = 0 sums nothing. */
typedef enum {
    LUNA_LINEAR_NONE = 0, LUNA_LINEAR_RELU = 1, LUNA_LINEAR_GELU = 2, LUNA_LINEAR_SILU = 3
} luna_linear_act;

typedef struct {
    int64_t m;
    int n, k;
    luna_linear_act act;
    luna_dtype io;
    int64_t ldx, ldw, ldy, ldr, ldz;  /* X, W, Y, R, Z        */
    int64_t lddy, lddx;               /* dY, dX (backward)    */
} luna_linear_desc;

/* Bytes of the workspace of luna_linear_fwd (backward = 0) or luna_linear_bwd
 * (1): partial sums, copies of the operands where the product needs them and,
 * with an activation, dLoss/dz.  256-byte aligned. */
luna_status luna_linear_workspace_size(const luna_linear_desc *ld, int backward, size_t *bytes);

luna_status luna_linear_fwd(const luna_linear_desc *ld, const void *X, const void *W, const void *bias, const void *R,
                            void *Y, void *Z, void *workspace, size_t ws_bytes, void *stream);

/* dX = dz W, dW = dz^T X (contiguous n x k), db = the column sums of dz (n), with
 * dz = dY act'(z); each is written where not NULL (the gradient of R is dY).
 * The bias gradient sums dz before dz is rounded to io for the products; bf16
 * layers of at most 64 rows whose products are short keep 16 bits of dz in them
 * instead of 8.  No atomics: equal inputs give equal bits. */
luna_status luna_linear_bwd(const luna_linear_desc *ld, const void *X, const void *W, const void *Z, const void *dY,
                            void *dX, void *dW, void *db, void *workspace, size_t ws_bytes, void *stream);

/* Synchronises `stream`, then reads and clears the device status word at the
 * start of `workspace`.  Every luna_attn_fwd / luna_attn_bwd call clears the
 * word when it starts; a device-side wait of that call that ran out of its
 * iteration limit sets it (the kernel then abandons its work and returns, so
 * the outputs of that call are undefined).  So this reports the LAST call that
 * used this workspace: LUNA_OK, LUNA_ERR_DEVICE_TIMEOUT, or LUNA_ERR_CUDA if
 * synchronising or the copy failed (including an earlier asynchronous fault). */
luna_status luna_device_status(void *workspace, void *stream);

/* Diagnostic of the failure path (not needed for computation): launches one
 * block that waits on a device-side barrier phase nothing ever completes,
 * gives up after limit_ns nanoseconds of wall time (1 <= limit_ns <= 1e9) and
 * sets the status word at the start of `workspace` exactly as a kernel of
 * luna_attn_fwd / luna_attn_bwd whose bounded wait ran out does.  A following
 * luna_device_status(workspace) then reports LUNA_ERR_DEVICE_TIMEOUT and clears
 * the word; the CUDA context stays usable and later calls run normally.
 * `workspace` as for luna_attn_fwd (256-byte aligned); LUNA_ERR_INVALID_ARG for
 * NULL or a limit out of range. */
luna_status luna_selftest_wait(void *workspace, int64_t limit_ns, void *stream);

/* Size of the library-owned scratch array used by luna_attn_fwd_noalloc. */
#define LUNA_NOALLOC_SCRATCH_BYTES (16u << 20)

/* luna_attn_fwd without a caller-provided workspace.  The paper has no
 * counterpart; this is a deployment convenience.
 *
 * Some callers hold only their input and output buffers and have no way to
 * obtain device scratch memory: a custom operator inside an inference engine
 * whose device-memory plan is fixed before it runs and that is handed nothing
 * but its tensors, or host code that must not call into an allocator while it
 * runs (fixed-latency loops).  For them this entry point allocates nothing:
 * no cudaMalloc, cudaFree or allocating library routine is called.  Its
 * scratch is one file-scope __device__ array of LUNA_NOALLOC_SCRATCH_BYTES
 * (16 MiB) that every GPU which loads the library holds until the process
 * exits; problems whose forward workspace (luna_workspace_size with
 * backward = 0) exceeds it are rejected with LUNA_ERR_WORKSPACE before
 * anything is launched.  Arguments and results are those of luna_attn_fwd
 * with state = NULL (no key statistics are kept for a backward pass).
 *
 * The first call on a device, with that device current, looks up the array's
 * device address (cudaGetSymbolAddress) and caches it; make that first call
 * before any stream capture.  All calls in the process share the one array
 * per device and leave their contents in it; each call clears what must start
 * at zero.  Calls whose executions overlap on the GPU (different streams, or
 * different host threads) race on the array and give undefined results: order
 * them on one stream.  The cached address is that of the device's primary
 * context: after cudaDeviceReset the array may move, and the library must not
 * be used on that device again in the same process.
 *
 * A bounded device-side wait of the call that ran out sets the status word at
 * the start of the array, as luna_attn_fwd does in its workspace (O is then
 * undefined); the next call clears it.  luna_noalloc_scratch gives the array's
 * address, so that luna_device_status(scratch, stream) reports the status of
 * the last call on the device. */
luna_status luna_attn_fwd_noalloc(const luna_attn_desc *ad, const luna_phi_desc *pd, const void *table,
                                  const void *Q, const void *K, const void *V, const int32_t *lengths, void *O,
                                  void *stream);

/* Device address and size of the scratch array of luna_attn_fwd_noalloc on the
 * current device (the same set-up as that call's first use: make the first call
 * before any stream capture).  Allocates nothing.  The address serves
 * luna_device_status, which reads and clears the status word of the last
 * luna_attn_fwd_noalloc call on this device, and luna_selftest_wait; the rest of
 * the array is the no-allocation call's scratch and must not be written while
 * such a call may be in flight.  The paper has no counterpart.
 * LUNA_ERR_INVALID_ARG for NULL arguments, LUNA_ERR_CUDA if the lookup fails. */
luna_status luna_noalloc_scratch(void **scratch, size_t *bytes);

/* Kernel timing (tracing aid, not needed for computation).  After
 * luna_profile_start(name), every launch of the library kernel `name` (e.g.
 * "bwd_query", "keystats"; the names are listed in the library's kernel
 * launch sites) is bracketed by two CUDA events recorded on the stream it is
 * launched on, up to 4096 launches.  luna_profile_stop waits for the recorded
 * events and returns the summed launch durations in milliseconds and the
 * number of launches, then stops recording.  Process-wide; one kernel name at
 * a time. */
luna_status luna_profile_start(const char *kernel);
luna_status luna_profile_stop(double *total_ms, int *launches);

/* Number of kernels this library has launched in this process since it was
 * loaded (all entry points, all streams). */
uint64_t luna_launch_count(void);

/* Library version, e.g. 100 for 0.1.0. */
int luna_version(void);

#ifdef __cplusplus
}
#endif

#endif /* LUNA_H */
