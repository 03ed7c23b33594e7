/*
 * dendsn.h - C ABI of libdendsn, the fused DendSN layer for NVIDIA GB300 (sm_103a).
 *
 * One DendSN layer (arXiv 2412.06355, Methods "Dendritic spiking neuron") maps the
 * branch input currents X[t, b, n, i] of B samples x N neurons x K compartments
 * over T time steps to somatic spikes S[t, b, n]:
 *
 *   V^d_i[t] = alpha_i V^d_i[t-1] + X_i[t]                 Eq. methods-compartment
 *   Y_j[t]   = psi( || (V^d_{C_j}[t] - xi_{C_j}) / zeta_j ||_2 )
 *                                                           Eq. methods-branch-aggregation
 *   psi(x)   = (1 - x^2) exp(-x^2 / 2)   or   psi(x) = x    Eq. methods-mexican-hat
 *   Z[t]     = sum_j kappa_j m_j Y_j[t]                     Eq. methods-soma-input,
 *                                                           Eq. methods-dbg-mask
 *   V^s[t]   = beta (1 - S[t-1]) V^s[t-1] + Z[t]            Eq. methods-lif-reset-charge
 *   S[t]     = Theta(V^s[t] - theta)                        Eq. methods-lif-fire
 *
 * and its backward is BPTT with the arctan surrogate dS/dV ~ 1/(1 + pi^2 (V - theta)^2)
 * (Eq. methods-sg). Branch j holds the G consecutive compartments j*G .. j*G+G-1
 * (G = P/B in the paper's notation); Kb = K / G branches.
 *
 * Conventions shared by every entry point
 *  - All tensor pointers are DEVICE pointers owned by the caller; the library never
 *    allocates, frees or copies between host and device.
 *  - Every call is asynchronous on the CUDA stream passed as `stream` (a
 *    cudaStream_t; NULL = legacy default stream). Argument errors are detected on
 *    the host before any launch and return a non-zero status with nothing enqueued.
 *    A failed launch returns DENDSN_ERR_CUDA. dendsn_last_error() describes the most
 *    recent failure of the calling thread.
 *  - Layouts are dense row-major:
 *      x, grad_x            [T, B, N, K] (or the PAPER layout, see dendsn_layout),
 *                           dtype x_dtype; base 16-byte aligned
 *      spikes, grad_spikes  [T, B, N]      dtype x_dtype (spikes are exactly 0 or 1)
 *      v_out, grad_v        [T, B, N]      float32
 *      alpha, xi            [C, K]         float32
 *      zeta, kappa          [C, Kb]        float32 (zeta > 0)
 *      mask                 [C, Kb] (mask_per_neuron = 0) or [N, Kb] (= 1), uint8 0/1,
 *                           base 4-byte aligned; NULL = all branches active
 *      grad_alpha, grad_xi  [C, K]         float32, OVERWRITTEN (not accumulated)
 *      grad_zeta, grad_kappa[C, Kb]        float32, OVERWRITTEN
 *    Neuron n of every sample uses parameter channel c(n) = (n / inner) % C, so the
 *    neurons at the spatial positions of a conv channel share parameters (Methods,
 *    "Dendritic spiking neural networks", constraint 3). N must be a multiple of
 *    C * inner. A layer-wide decay alpha (the paper's choice) is passed as a [C, K]
 *    array of equal values; its gradient is the sum of grad_alpha.
 *  - Supported: K in {1, 2, 4, 8, 16}; G in {1, 2, 4} with G dividing K;
 *    T >= 0; B * N < 2^31 * C * inner. Others return DENDSN_ERR_UNSUPPORTED.
 */
#ifndef DENDSN_H
#define DENDSN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DENDSN_OK = 0,
    DENDSN_ERR_INVALID_ARG = 1,   /* NULL pointer, bad size, bad enum value */
    DENDSN_ERR_UNSUPPORTED = 2,   /* valid but not compiled in (K, G, surrogate) */
    DENDSN_ERR_MISALIGNED = 3,    /* a pointer violates its alignment rule */
    DENDSN_ERR_CUDA = 4           /* a CUDA launch failed; see dendsn_last_error() */
} dendsn_status;

typedef enum { DENDSN_F32 = 0, DENDSN_BF16 = 1 } dendsn_dtype;
typedef enum { DENDSN_PSI_IDENTITY = 0, DENDSN_PSI_MEXHAT = 1 } dendsn_psi;
/* HARD: Eq. methods-lif-reset-charge. SOFT: V^s[t] = beta (V^s[t-1] - theta S[t-1]) + Z[t]. */
typedef enum { DENDSN_RESET_HARD = 0, DENDSN_RESET_SOFT = 1 } dendsn_reset;
/* ATAN: Eq. methods-sg, the only surrogate the paper uses. */
typedef enum { DENDSN_SG_ATAN = 0 } dendsn_surrogate;
/*
 * Layout of x and grad_x (spikes and the other [T, B, N] tensors are the same in both):
 *   KINNER: [T, B, N, K], a neuron's K compartments contiguous.
 *   PAPER : [T, B, N / inner, K, inner], i.e. a conv layer's output [T, B, C_o * P, H, W]
 *           read as (C_o, P, H, W) with inner = H * W (Methods, "Dendritic spiking neural
 *           networks"): compartment k of neuron n is (n / inner) * K * inner + k * inner
 *           + n % inner elements into the sample. No transpose is needed.
 */
typedef enum { DENDSN_LAYOUT_KINNER = 0, DENDSN_LAYOUT_PAPER = 1 } dendsn_layout;

typedef struct {
    int32_t T, B, N;        /* time steps, samples, neurons per sample */
    int32_t K, G;           /* compartments per neuron, compartments per branch */
    int32_t C, inner;       /* parameter channels; neurons per channel run */
    int32_t x_dtype;        /* dendsn_dtype of x, spikes, grad_spikes, grad_x */
    int32_t psi;            /* dendsn_psi */
    int32_t reset;          /* dendsn_reset */
    int32_t surrogate;      /* dendsn_surrogate */
    float theta;            /* firing threshold (1 in Eq. methods-lif-fire) */
    float beta;             /* somatic decay, 0 <= beta < 1 */
    int32_t detach_reset;   /* 1: no gradient through the reset term */
    int32_t mask_per_neuron;/* 0: mask is [C, Kb]; 1: mask is [N, Kb] */
    int32_t stateless;      /* 1: Stateless Dendrite, V^d = X (Methods, "Stateless compartment") */
    int32_t residual;       /* 1: Z += mean_i X_i (Eq. methods-residual) */
    int32_t layout;         /* dendsn_layout of x and grad_x */
} dendsn_config;

/*
 * Sizes of the two caller-owned device buffers a forward/backward pair needs.
 *   saved_bytes  : state the forward writes and the backward reads. For T > 8,
 *                  checkpoints of (V^d, V^s) every 8 steps (recompute with
 *                  checkpointing, Results "Constructing deep DendSNNs"). For layers
 *                  whose backward serves each 8-compartment neuron on one thread over
 *                  a single chunk (K = 8, G = 1, compartments innermost, no residual
 *                  term, T = 8, or T = 4 with bfloat16 x), V^s [T, B, N] float32, so
 *                  that the backward rescans only V^d; optional there (NULL in both
 *                  calls: the backward recomputes V^s from x, with the same bits).
 *                  Otherwise 0. 16-byte aligned. Must outlive the backward.
 *   scratch_bytes: per-block partial sums of the parameter gradients, used only by
 *                  dendsn_backward. 16-byte aligned. Contents need no initialisation.
 * Either output pointer may be NULL.
 */
dendsn_status dendsn_workspace_size(const dendsn_config *cfg, size_t *saved_bytes,
                                    size_t *scratch_bytes);

/*
 * Fused multi-step forward: compartment scan, L2 branch aggregation, psi, masked
 * kappa reduction and LIF soma, all T steps in one kernel with the state in
 * registers.
 *   x        [T,B,N,K] input currents (read)
 *   alpha..kappa, mask: parameters as above (read)
 *   spikes   [T,B,N] output (written)
 *   v_out    [T,B,N] float32 somatic potential V^s (written), or NULL
 *   saved    buffer of saved_bytes (written), or NULL when no backward will follow;
 *            ignored when saved_bytes == 0
 */
dendsn_status dendsn_forward(const dendsn_config *cfg, const void *x, const float *alpha,
                             const float *xi, const float *zeta, const float *kappa,
                             const uint8_t *mask, void *spikes, float *v_out, void *saved,
                             void *stream);

/*
 * Fused reverse-time backward (BPTT with the arctan surrogate, Eq. methods-sg). The
 * forward of each checkpoint interval is recomputed from x in registers.
 *   grad_spikes [T,B,N] dL/dS (read); grad_v [T,B,N] float32 dL/dV^s (read) or NULL
 *   saved       the buffer the forward of the same inputs filled (read); may be NULL
 *               when T <= 8 if it was NULL in the forward too (a buffer the forward did
 *               not fill gives wrong gradients, it is not detected)
 *   grad_x      [T,B,N,K] dL/dX (written)
 *   grad_alpha, grad_xi, grad_zeta, grad_kappa: parameter gradients summed over time,
 *               samples and the neurons of each channel (written, deterministic order).
 *               grad_alpha is all zero for a Stateless Dendrite. grad_kappa is the
 *               gradient w.r.t. the unmasked strength (zero where the mask is 0).
 *   scratch     scratch_bytes of device memory (contents are overwritten)
 */
dendsn_status dendsn_backward(const dendsn_config *cfg, const void *x, const float *alpha,
                              const float *xi, const float *zeta, const float *kappa,
                              const uint8_t *mask, const void *grad_spikes,
                              const float *grad_v, const void *saved, void *grad_x,
                              float *grad_alpha, float *grad_xi, float *grad_zeta,
                              float *grad_kappa, void *scratch, void *stream);

/*
 * dendsn_backward for a soma whose decay beta is learnable (the PLIF soma the paper cites
 * alongside LIF, read as Eq. methods-lif-reset-charge with beta a parameter). Same
 * arguments and outputs as dendsn_backward, plus
 *   grad_beta  [C] float32, OVERWRITTEN: dL/dbeta summed over time, samples and the
 *              neurons of each channel, where dV^s[t+1]/dbeta = (1 - S[t]) V^s[t] (hard
 *              reset) or V^s[t] - theta S[t] (soft). The gradient of the layer's single
 *              beta is the sum of the C entries (parameterisations such as
 *              beta = sigmoid(w) are applied by the caller).
 * Runs a separate build of the backward kernel that also accumulates dL/dbeta (one more
 * fused multiply-add per step); dendsn_backward does not pay for it.
 */
dendsn_status dendsn_backward_plif(const dendsn_config *cfg, const void *x, const float *alpha,
                                   const float *xi, const float *zeta, const float *kappa,
                                   const uint8_t *mask, const void *grad_spikes,
                                   const float *grad_v, const void *saved, void *grad_x,
                                   float *grad_alpha, float *grad_xi, float *grad_zeta,
                                   float *grad_kappa, float *grad_beta, void *scratch,
                                   void *stream);

/*
 * Same computation and outputs as dendsn_backward, without the caller's scratch buffer:
 * for callers that cannot allocate device memory for it, such as a C host that only
 * receives device pointers for the layer's tensors, or a runtime whose device memory is
 * budgeted in advance and that must not allocate per call. (The paper has no
 * counterpart; this is an interface convenience.)
 *   - The parameter-gradient partials go to a buffer compiled into the library:
 *     8 MiB of device memory on every GPU that loads the library, held until the
 *     process exits. A layer whose dendsn_workspace_size scratch_bytes exceeds 8 MiB
 *     is rejected with DENDSN_ERR_UNSUPPORTED before anything is enqueued.
 *   - The first call on a device looks up that buffer's device address (with that
 *     device current) and caches it; make that first call before any stream capture.
 *     The cached address belongs to the device's context at that time: after a
 *     cudaDeviceReset on that device (which unloads the library's device code) it is
 *     stale, so a process that resets a device must not call this entry point on it
 *     again.
 *   - All calls share the one buffer, which keeps the last call's contents. Nothing in
 *     it needs to start at zero. Calls whose executions overlap on the GPU (for example
 *     on two streams without ordering between them) race on it and give wrong results.
 *   - Allocates nothing: no cudaMalloc, cudaFree or allocating library call.
 * Arguments are those of dendsn_backward minus `scratch`.
 */
dendsn_status dendsn_backward_noalloc(const dendsn_config *cfg, const void *x,
                                      const float *alpha, const float *xi, const float *zeta,
                                      const float *kappa, const uint8_t *mask,
                                      const void *grad_spikes, const float *grad_v,
                                      const void *saved, void *grad_x, float *grad_alpha,
                                      float *grad_xi, float *grad_zeta, float *grad_kappa,
                                      void *stream);

/*
 * Point-neuron LIF layer: the baseline neuron the paper compares the DendSN layer's speed
 * with (Results, efficiency paragraph). It is the DendSN soma driven directly by one input
 * current per neuron (Eq. methods-lif-reset-charge with X[t] in place of Z[t],
 * Eq. methods-lif-fire; soft reset as above), trained with the same arctan surrogate
 * (Eq. methods-sg). Same conventions as the DendSN entry points (device pointers, async
 * on `stream`, host-side validation, dendsn_last_error()).
 *   x, grad_x, spikes, grad_spikes   [T, B, N]  dtype x_dtype, naturally aligned
 *   v_out, grad_v                    [T, B, N]  float32, 4-byte aligned; may be NULL
 *   saved   checkpoints (V at the end of every 8 steps), saved_bytes of 16-byte aligned
 *           device memory; needed (non-NULL) only when saved_bytes > 0, i.e. T > 8
 * Tensors whose neuron count B*N is a multiple of 4 and whose pointers are aligned to 4
 * elements (16 bytes for the float32 ones) take the vectorised kernels.
 */
typedef struct {
    int32_t T, B, N;        /* time steps, samples, neurons per sample */
    int32_t x_dtype;        /* dendsn_dtype of x, spikes, grad_spikes, grad_x */
    int32_t reset;          /* dendsn_reset */
    float theta, beta;      /* threshold, somatic decay (0 <= beta < 1) */
    int32_t detach_reset;   /* 1: no gradient through the reset term */
} dendsn_lif_config;

dendsn_status dendsn_lif_workspace_size(const dendsn_lif_config *cfg, size_t *saved_bytes);

/* Fused T-step LIF forward: writes spikes (and V if v_out), and the checkpoints to saved. */
dendsn_status dendsn_lif_forward(const dendsn_lif_config *cfg, const void *x, void *spikes,
                                 float *v_out, void *saved, void *stream);

/* Fused reverse-time LIF backward: dL/dX from dL/dS (and dL/dV if grad_v), recomputing V. */
dendsn_status dendsn_lif_backward(const dendsn_lif_config *cfg, const void *x,
                                  const void *grad_spikes, const float *grad_v,
                                  const void *saved, void *grad_x, void *stream);

/*
 * Token-sequence operators around a DendSN layer: the embedding that turns token ids into
 * input currents, a compartment scan whose decay is an input of its own, and the softmax
 * cross entropy of a linear readout of the spikes. Same conventions as above: device
 * pointers, dense row-major tensors, asynchronous on `stream`, host-side validation with
 * nothing enqueued on an error, caller-owned scratch whose contents need no initialisation,
 * dendsn_last_error(). All sums and states are float32; a bfloat16 output is rounded once.
 * Every result is the same for the same inputs from run to run (no floating-point atomics).
 * Tensors are naturally aligned (one element); rows whose addresses and lengths are multiples
 * of 16 bytes take wider loads. A scratch buffer serves one call at a time. Waits of the scan and
 * the cross entropy on other blocks or on copies give up after a second or more: the scan's block
 * goes on with NaN for the state that did not come (until a sequence starts), and the losses, or
 * grad_hidden with a grad_weight of no meaning, are NaN. The embedding's gradient meets at the
 * barriers of one cluster or of a cooperative grid, whose blocks all run at the same time.
 */
typedef enum { DENDSN_I32 = 0, DENDSN_I64 = 1 } dendsn_index;

/*
 * Embedding lookup with scaling, and its gradient.
 *   out[i, :]        = scale * table[ids[i], :]        for 0 <= ids[i] < V
 *   grad_table[v, :] = scale * sum of grad_out[i, :] over ids[i] = v, i ascending
 * A token equal to padding_id gives a row of zeros and takes no part in the gradient
 * (padding_id < 0: there is none). A token outside [0, V) gives a row of NaN and takes no
 * part in the gradient.
 *   table, grad_table [V, D], out, grad_out [n, D]   dtype x_dtype
 *   ids               [n]                            dtype ids_dtype
 *   grad_table is OVERWRITTEN: rows without tokens become zero. n >= 0, n < 2^31.
 */
typedef struct {
    int64_t n;              /* tokens */
    int64_t padding_id;     /* token id without a row, or negative: none */
    int32_t V, D;           /* vocabulary, row length */
    int32_t x_dtype;        /* dendsn_dtype of table, out, grad_out, grad_table */
    int32_t ids_dtype;      /* dendsn_index of ids */
    float scale;
} dendsn_embed_config;

/* scratch_bytes of the backward (the forward needs none). */
dendsn_status dendsn_embed_workspace_size(const dendsn_embed_config *cfg, size_t *scratch_bytes);
dendsn_status dendsn_embed_forward(const dendsn_embed_config *cfg, const void *table,
                                   const void *ids, void *out, void *stream);
dendsn_status dendsn_embed_backward(const dendsn_embed_config *cfg, const void *ids,
                                    const void *grad_out, void *grad_table, void *scratch,
                                    void *stream);

/*
 * Gated compartment scan: Eq. methods-compartment with a decay of its own for every channel
 * and step (channel = one of the B * N compartments).
 *   a[t] = gate[t] (DECAY) or 1 / (1 + exp(-gate[t])) (LOGIT)
 *   u[t] = x[t] (PLAIN) or (1 - a[t]) x[t] (COMPLEMENT)
 *   h[t] = a[t] h[t-1] + u[t],  h[-1] = h0
 * starts marks the first step of each packed sequence of a sample: where it is nonzero,
 * h[t] = u[t] whatever came before (also infinities and NaN), and no gradient passes back.
 *   x, gate, h, grad_h, grad_x, grad_gate   [T, B, N] or [B, T, N] (layout), dtype x_dtype
 *   starts        [T, B] or [B, T] uint8, or NULL: one sequence for each sample
 *   h0, grad_h0   [B, N] float32, or NULL (h0 NULL: zeros)
 *   h_last, grad_last [B, N] float32, or NULL; h_last may be h0 itself (a serving step)
 *   saved         saved_bytes, 16-byte aligned: the states at the end of every 64 steps, written
 *                 by the forward when not NULL and read by the backward (needed for T > 64)
 * The backward recomputes h from x and gate. grad_gate is the gradient of gate itself.
 * With T = 0, h_last = h0 and grad_h0 = grad_last (zeros where NULL).
 */
typedef enum { DENDSN_GATE_DECAY = 0, DENDSN_GATE_LOGIT = 1 } dendsn_gate;
typedef enum { DENDSN_MIX_PLAIN = 0, DENDSN_MIX_COMPLEMENT = 1 } dendsn_mix;
typedef enum { DENDSN_TIME_FIRST = 0, DENDSN_BATCH_FIRST = 1 } dendsn_scan_layout;

typedef struct {
    int32_t T, B, N;        /* steps, samples, channels per sample */
    int32_t x_dtype;        /* dendsn_dtype of x, gate, h and their gradients */
    int32_t gate;           /* dendsn_gate */
    int32_t mix;            /* dendsn_mix */
    int32_t layout;         /* dendsn_scan_layout */
} dendsn_scan_config;

dendsn_status dendsn_scan_workspace_size(const dendsn_scan_config *cfg, size_t *saved_bytes);
dendsn_status dendsn_scan_forward(const dendsn_scan_config *cfg, const void *x, const void *gate,
                                  const uint8_t *starts, const float *h0, void *h,
                                  float *h_last, void *saved, void *stream);
dendsn_status dendsn_scan_backward(const dendsn_scan_config *cfg, const void *x, const void *gate,
                                   const uint8_t *starts, const float *h0, const void *grad_h,
                                   const float *grad_last, const void *saved, void *grad_x,
                                   void *grad_gate, float *grad_h0, void *stream);

/*
 * Softmax cross entropy of a linear readout, in pieces of the vocabulary: the logits
 * hidden weight^T are never kept.
 *   l[r, v] = sum_d hidden[r, d] weight[v, d];  lse[r] = log sum_v exp l[r, v]
 *   loss[r] = lse[r] - l[r, labels[r]]
 * and, for an upstream gradient grad_loss of the row losses,
 *   G[r, v] = grad_loss[r] (exp(l[r, v] - lse[r]) - [v = labels[r]])
 *   grad_hidden = G weight;  grad_weight = G^T hidden
 * A row whose label is ignore_index has loss 0, lse 0 and zero gradient, whatever its hidden
 * values are (also infinities and NaN). A row with any other label outside [0, V) has loss,
 * lse and grad_hidden NaN and takes no part in grad_weight.
 * bfloat16 inputs: products are exact, sums float32 in the tensor cores (which cost the losses 8e-7
 * of their norm at D = 2048); the two products that take G have it as the sum of two bfloat16
 * terms (logit_grad SPLIT, within 2^-16), or rounded to one where the caller chooses so (logit_grad
 * BF16: two fifths fewer operations in the backward, and a rounding of up to 2^-8 of each logit's
 * gradient beside the output's own). float32 inputs: every operand is split into three bfloat16
 * terms, whose six leading products are summed (a relative error of about 2^-24 of each product);
 * the forward of up to 32 rows multiplies and adds in float32.
 * What the forward leaves in lse for the backward (statistics): LSE, lse [M] as above, whose
 * rounding is an error of up to 2^-24 |lse| of every probability in the backward; for up to 32
 * float32 rows the logits that the backward forms are also rounded otherwise than the forward's.
 * MAX_SUM, lse [2, M]: the largest logit and the sum of exp(l - largest), from which the backward
 * forms the probabilities without that rounding, and of the same logits at any size.
 *   hidden, grad_hidden [M, D], weight, grad_weight [V, D]   dtype x_dtype
 *   labels [M] dtype labels_dtype;  loss, grad_loss [M], lse [M] or [2, M] float32
 *   grad_hidden and grad_weight are OVERWRITTEN. V, D >= 1; M >= 0.
 *   scratch: 256-byte aligned; forward_bytes for the forward, backward_bytes for the backward.
 */
typedef enum { DENDSN_LOGIT_GRAD_SPLIT = 0, DENDSN_LOGIT_GRAD_BF16 = 1 } dendsn_logit_grad;
typedef enum { DENDSN_STATISTICS_LSE = 0, DENDSN_STATISTICS_MAX_SUM = 1 } dendsn_statistics;

typedef struct {
    int64_t ignore_index;
    int32_t M, V, D;        /* rows, vocabulary, row length */
    int32_t x_dtype;        /* dendsn_dtype of hidden, weight and their gradients */
    int32_t labels_dtype;   /* dendsn_index of labels */
    int32_t logit_grad;     /* dendsn_logit_grad; float32 inputs: SPLIT (three terms) */
    int32_t statistics;     /* dendsn_statistics of lse */
    int32_t weight_aligned; /* 1: weight is 16-byte aligned. Scratch then has no room for a copy of
                               bfloat16 weights with D a multiple of 8, which are read in place */
} dendsn_xent_config;

dendsn_status dendsn_xent_workspace_size(const dendsn_xent_config *cfg, size_t *forward_bytes,
                                         size_t *backward_bytes);
dendsn_status dendsn_xent_forward(const dendsn_xent_config *cfg, const void *hidden,
                                  const void *weight, const void *labels, float *loss,
                                  float *lse, void *scratch, void *stream);
dendsn_status dendsn_xent_backward(const dendsn_xent_config *cfg, const void *hidden,
                                   const void *weight, const void *labels, const float *lse,
                                   const float *grad_loss, void *grad_hidden,
                                   void *grad_weight, void *scratch, void *stream);

/* Static description of a status code. */
const char *dendsn_status_string(dendsn_status status);

/* Message describing the calling thread's most recent failed call ("" if none). */
const char *dendsn_last_error(void);

/* Number of kernels the library enqueued since load (all threads). */
uint64_t dendsn_launch_count(void);

#ifdef __cplusplus
}
#endif

#endif /* DENDSN_H */
