/*
 * hdet.h -- C ABI of the HDET (Hyperparameter-Divergent Ensemble Training) step for one
 * AMD MI355X (gfx950).
 *
 * The N data-parallel replicas of the paper live as a replica axis in one GPU's memory:
 * every per-replica tensor is an array of N planes, plane r starting `plane_stride`
 * elements after plane r-1.  The paper's AllReduce calls become reductions along that axis.
 *
 * One training step is (Algorithm 1 of the paper):
 *     hdet_forward_backward   loss and gradient of every replica          (model modes only)
 *     hdet_fanout_step        update t with per-replica rate eta_r        (Sec. 3.2, Eq. 1-2)
 *   (or hdet_train_step for both in one call, which lets the library fuse them)
 *   and, when t mod T == 0,
 *     hdet_converge           replica mean of the parameters              (Sec. 3.3, Eq. 3)
 *     hdet_autolr_update      controller on the interval losses           (Sec. 3.4, Eq. 4-9)
 *
 * General rules
 *   - Every pointer named *_dev is DEVICE memory, owned by the caller and borrowed for the
 *     lifetime of the handle; pointers named *_host are host memory read or written during
 *     the call only.  The library allocates one small device control block per handle
 *     (a few KiB) and nothing else on the device.
 *   - All device work is enqueued on the HIP stream given at creation; calls return without
 *     waiting for it unless stated otherwise.  Calls on one handle must not overlap.
 *   - Every function returns 0 (HDET_OK) or a negative HDET_E* code; after a failure
 *     hdet_last_error() gives a message.  No C++ exception crosses this boundary.
 *   - There is no CPU fallback: without a HIP device hdet_create fails with HDET_EHIP.
 */
#ifndef HDET_H
#define HDET_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define HDET_MAX_REPLICAS 64   /* one wavefront holds one replica per lane in the controller */
#define HDET_MAX_CH       8    /* explored hyperparameter channels (Remark 1)                */
#define HDET_MAX_GROUPS   4    /* parameter groups with a learning-rate channel each        */
#define HDET_MAX_LAYERS   16

enum { HDET_OK = 0, HDET_EINVAL = -1, HDET_ESTATE = -2, HDET_EHIP = -3,
       HDET_ENONFINITE = -4 };   /* an interval loss handed to hdet_autolr_update is not finite */

enum { HDET_SGDM = 0, HDET_ADAMW = 1 };                       /* optimizer                   */
enum { HDET_GRAD_SHARED = 0, HDET_GRAD_PER_REPLICA = 1 };     /* gradient exchange           */
enum { HDET_FP32 = 0, HDET_BF16_GEMM_FP32_MASTER = 1 };       /* precision of the model GEMMs */
enum { HDET_FLAT = 0, HDET_MLP = 1, HDET_TRANSFORMER = 2 };   /* model kind                  */
enum { HDET_CH_LR = 0, HDET_CH_DROPOUT = 1, HDET_CH_WD = 2,      /* channel kinds (Remark 1)   */
       HDET_CH_LABEL_SMOOTH = 3, HDET_CH_ATTN_TEMP = 4 };

/* flags of hdet_fanout_step and hdet_train_step */
#define HDET_FUSE_CONVERGE 1u  /* on a sync step, average inside the update kernel (Eq. 3)   */

typedef struct hdet_handle hdet_handle;

/* One explored scalar hyperparameter beside the learning rate (Remark 1): replica r uses
 * base * rho_{pi(r)} with rho from Eq. 1 at this channel's alpha and its own permutation. */
typedef struct {
  int32_t kind;        /* HDET_CH_DROPOUT, HDET_CH_WD, HDET_CH_LABEL_SMOOTH or HDET_CH_ATTN_TEMP */
  int32_t reserved;
  double  base;        /* initial centre value h_bar                                         */
  double  alpha;       /* spread ratio                                                       */
  double  lambda;      /* step of Eq. 7 for this channel                                     */
  double  lo, hi;      /* the centre value is clamped to [lo, hi] after each controller step.
                          Replica values range over centre * [1 - alpha, 1 + alpha] (Eq. 1), so
                          the whole range must stay meaningful: hi * (1 + alpha) < 1 for a
                          dropout rate, <= 1 for label smoothing, lo * (1 - alpha) > 0 for an
                          attention temperature; lo <= base <= hi.  HDET_EINVAL otherwise.    */
} hdet_channel;

typedef struct {
  int64_t n_params;                        /* HDET_FLAT: P, parameters per replica           */
  int32_t n_layers;                        /* HDET_MLP: number of Linear layers              */
  int32_t widths[HDET_MAX_LAYERS + 1];     /* HDET_MLP: d_in, hidden..., d_out               */
  int32_t batch;                           /* HDET_MLP: rows per replica and step;
                                              HDET_TRANSFORMER: sequences per replica and step */
  /* HDET_TRANSFORMER: decoder-only, pre-LayerNorm, learned positions, tanh-GELU MLP, causal
   * attention, biases on every Linear, untied output head, final LayerNorm (eps 1e-5).      */
  int32_t n_blocks, d_model, n_heads, d_ff, seq_len, vocab;
} hdet_model_dims;

/* Arguments of Algorithm 1 ("Require") plus what the paper leaves to the optimizer. */
typedef struct {
  int32_t  n_replicas;      /* N, 1..HDET_MAX_REPLICAS                                       */
  int32_t  sync_interval;   /* T >= 1                                                        */
  int64_t  total_steps;     /* S >= 1; hdet_fanout_step fails with HDET_ESTATE beyond it     */
  int64_t  warm_steps;      /* S_warm: the controller runs at sync steps with t >= S_warm    */
  double   lr_max;          /* one-cycle peak eta_max                                        */
  double   f_div;           /* initial rate = eta_max / f_div                                */
  double   f_final;         /* final rate   = eta_max / (f_div * f_final)                    */
  double   pct_start;       /* p: fraction of S spent rising                                 */
  int32_t  constant_lr;     /* nonzero: base schedule is eta_max at every step               */
  int32_t  autolr_enabled;  /* nonzero: run the controller of Sec. 3.4                       */
  double   alpha;           /* spread ratio of the learning rate (Eq. 1)                     */
  double   beta;            /* velocity momentum (Eq. 7)                                     */
  double   sigma;           /* softmax temperature (Eq. 4)                                   */
  double   lambda;          /* step of Eq. 7 for the learning rate                           */
  double   gamma_override;  /* >= 0 replaces the decay of Eq. 8; < 0 computes it             */
  int32_t  optimizer;       /* HDET_SGDM or HDET_ADAMW                                       */
  int32_t  grad_mode;       /* HDET_GRAD_SHARED: every replica applies the replica mean of
                               the gradients (the paper's gradient AllReduce);
                               HDET_GRAD_PER_REPLICA: replica r applies its own gradient    */
  int32_t  shared_opt_state;       /* 1 (HDET_ADAMW with HDET_GRAD_SHARED only): the moments
                               depend on the mean gradient alone, so they are the same for every
                               replica and are kept once: opt_m_dev and opt_v_dev are
                               [plane_stride] instead of [N][plane_stride], and a step moves
                               12 N + 16 bytes per element instead of 28 N                   */
  int32_t  reshuffle_every_sync;   /* 0: new permutations only when the controller runs
                               (Algorithm 1), numbered by the controller update k; 1: at every
                               sync step, also before warm_steps or with the controller off
                               (the caption of Fig. 1), numbered by the sync step t / T      */
  double   momentum;        /* SGDM                                                          */
  double   beta1, beta2, eps;      /* AdamW                                                  */
  double   weight_decay;    /* used by all replicas unless a HDET_CH_WD channel exists       */
  int32_t  precision;       /* HDET_FP32 or HDET_BF16_GEMM_FP32_MASTER                       */
  int32_t  model_kind;      /* HDET_FLAT, HDET_MLP or HDET_TRANSFORMER                       */
  hdet_model_dims dims;
  int32_t  n_extra_channels;           /* 0..HDET_MAX_CH - max(n_groups, 1)                  */
  int32_t  n_groups;        /* 0 or 1: one learning-rate channel for all parameters; G > 1:
                               parameter groups with a rate channel each (Sec. 3.4, "random
                               reassignment across hyperparameters": own base rate, velocity
                               and permutation per group, the same one-cycle until hand-over) */
  int64_t  group_end[HDET_MAX_GROUPS]; /* group g is the slice [group_end[g-1], group_end[g]) of a
                               parameter plane; ascending, multiples of 4, the last equals P  */
  hdet_channel extra[HDET_MAX_CH - 1];
  uint64_t seed;            /* keys the permutations of Eq. 9                                */
  void*    stream;          /* hipStream_t, borrowed; NULL = the default stream              */
} hdet_config;

/* Caller-owned device buffers.  Planes are `plane_stride` elements apart; plane_stride >= P
 * and a multiple of 4, every pointer 16-byte aligned (a stride that is a multiple of 64
 * elements and 256-byte aligned pointers put every plane on a cache-line boundary, which the
 * update stream rewards with about 8 % more bandwidth).  Parameter layout inside a plane for
 * HDET_MLP: [W_1 (d_out x d_in, row-major), b_1, W_2, b_2, ...].  For HDET_TRANSFORMER (all
 * row-major): tok_emb [V][d], pos_emb [S][d], then per block ln1_g, ln1_b [d], w_qkv [3d][d],
 * b_qkv [3d], w_o [d][d], b_o [d], ln2_g, ln2_b [d], w_1 [ff][d], b_1 [ff], w_2 [d][ff],
 * b_2 [d], then lnf_g, lnf_b [d], w_head [V][d], b_head [V]; rows 0..d-1 of w_qkv give q,
 * d..2d-1 k, 2d..3d-1 v and head h owns columns h*d/heads .. of each.                       */
typedef struct {
  float*    params_dev;       /* [N][plane_stride] fp32 master parameters, updated in place  */
  float*    grads_dev;        /* [N][plane_stride] fp32; written by hdet_forward_backward;
                                 may be NULL for HDET_FLAT (gradients are passed per step)   */
  float*    opt_m_dev;        /* [N][plane_stride] AdamW first moment / SGD momentum buffer;
                                 must be zero at t = 0 ([plane_stride] with shared_opt_state) */
  float*    opt_v_dev;        /* [N][plane_stride] AdamW second moment; NULL for HDET_SGDM
                                 ([plane_stride] with shared_opt_state)                      */
  uint16_t* params_bf16_dev;  /* [N][plane_stride] bfloat16 copy of the parameters, kept in
                                 step by the update and converge kernels; NULL unless
                                 precision == HDET_BF16_GEMM_FP32_MASTER                     */
  void*     workspace_dev;    /* activations and scratch for hdet_forward_backward           */
  size_t    workspace_bytes;
  int64_t   plane_stride;
} hdet_buffers;

/* Host-side snapshot of the schedule and controller state. */
typedef struct {
  int64_t t;                  /* updates done                                                */
  int64_t k;                  /* controller updates done                                     */
  int32_t controller_active;  /* the controller has taken the base rate over                 */
  int32_t nonfinite;          /* controller calls skipped because a loss was not finite      */
  int32_t n_replicas, n_channels;
  int32_t autolr_done;        /* t is a sync step and hdet_autolr_update has already run on it:
                                 a state saved between hdet_fanout_step and hdet_autolr_update
                                 has 0 here, and the resumed handle still accepts that call     */
  int32_t reserved;
  double  gamma;              /* decay in use for the learning-rate channel                  */
  double  base[HDET_MAX_CH];  /* centre value per channel (rate channels of the groups first,
                                 then the extra channels); rates are meaningful once active  */
  double  vel[HDET_MAX_CH];   /* velocity v of Eq. 7                                         */
  double  delta[HDET_MAX_CH]; /* last hypergradient (Eq. 6)                                  */
  double  w[HDET_MAX_REPLICAS];        /* last softmax weights (Eq. 4)                       */
  double  l_acc[HDET_MAX_REPLICAS];    /* loss accumulated since the last sync step          */
  double  l_last[HDET_MAX_REPLICAS];   /* interval losses L_r seen by the last sync step     */
  float   l_step[HDET_MAX_REPLICAS];   /* losses of the last hdet_forward_backward           */
  float   lr[HDET_MAX_REPLICAS];       /* rates used by the last hdet_fanout_step            */
  double  rho[HDET_MAX_CH][HDET_MAX_REPLICAS];   /* multipliers of Eq. 1 per channel         */
  int32_t perm[HDET_MAX_CH][HDET_MAX_REPLICAS];  /* pi_j(r): replica r uses rho_j[perm]      */
} hdet_state;

/* Bytes the caller must provide: one plane set (N * plane_stride elements) of fp32 for each
 * of params / grads / opt_m / opt_v, of bf16 for the shadow, and the workspace.  Any out
 * pointer may be NULL.  Returns HDET_EINVAL for an invalid configuration.                   */
int hdet_workspace_bytes(const hdet_config* cfg, int64_t plane_stride, size_t* plane_set_bytes,
                         size_t* shadow_bytes, size_t* workspace_bytes);

/* Validates the configuration, computes rho (Eq. 1) and gamma (Eq. 8), sets pi = identity,
 * v = 0, L_acc = 0, t = k = 0 (Algorithm 1, initialisation) and allocates the control block.
 * With HDET_BF16_GEMM_FP32_MASTER the bf16 copy of the parameters is (re)written from
 * params_dev.  Errors: HDET_EINVAL (bad argument, misaligned pointer), HDET_EHIP.           */
int hdet_create(const hdet_config* cfg, const hdet_buffers* buffers, hdet_handle** out);

/* Warm noisy initialisation (Sec. 3.5, Eq. 10): params_dev[r] <- theta0 + eps_r for every
 * replica r, eps_r ~ N(0, nu^2 ||theta0||^2 / P) independently per replica and element (the
 * paper uses nu = 0.01).  theta0_dev: [P] fp32 checkpoint in device memory, 16-byte aligned,
 * not overlapping params_dev.  The noise is a pure function of (seed, replica, index)
 * (Philox-4x32-10 + Box-Muller); the bf16 copy is refreshed.  Only before the first update:
 * HDET_ESTATE once t > 0.                                                                   */
int hdet_warm_init(hdet_handle* h, const float* theta0_dev, double nu, uint64_t seed);

/* For callers that cannot allocate device memory -- code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc: the initialisation of hdet_warm_init without a handle
 * (hdet_create allocates the control block that holds hdet_warm_init's partial sums).  Writes
 * params_dev[r][0..n_params) = theta0 + eps_r for r < n_replicas exactly as hdet_warm_init does
 * for the same (theta0, nu, seed), and, if params_bf16_dev is not NULL, the bfloat16 copy in the
 * same layout.  All pointers are device memory owned by the caller, 16-byte aligned, planes
 * plane_stride elements apart (>= n_params, a multiple of 4); theta0_dev [n_params] must not
 * overlap params_dev; stream: hipStream_t or NULL.  The partial sums of ||theta0||^2 live in a
 * fixed array of 8 KiB inside the library, one copy per GPU for the life of the process;
 * the call allocates and frees nothing and does not wait for the stream.  Every entry of that
 * array that a call reads it has written before, so nothing carries over from one call to the
 * next; but all calls on one GPU share the array: calls that overlap in time on the same GPU
 * (different streams or threads) race and must be serialised by the caller.
 * Limits: 1 <= n_params <= 2^34, 1 <= n_replicas <= HDET_MAX_REPLICAS; beyond them HDET_EINVAL.
 * Errors: HDET_EINVAL, HDET_EHIP; the message is that of hdet_last_error(NULL).              */
int hdet_warm_init_noalloc(const float* theta0_dev, float* params_dev, uint16_t* params_bf16_dev,
                           int64_t n_params, int64_t plane_stride, int32_t n_replicas, double nu,
                           uint64_t seed, void* stream);

/* Forward, mean cross-entropy and backward of all N replicas on x_dev [N][B][d_in]
 * (fp32; rounded to bf16 on load in bf16 precision) and labels y_dev [N][B] int32 -- for
 * HDET_TRANSFORMER x_dev is token ids [N][B][S] int32 and y_dev the next-token targets
 * [N][B][S] int32, the loss being the mean over the B*S positions
 * ("Forward + backward" of Algorithm 1; the loss is the one that Sec. 3.4 averages into
 * L_r).  With a HDET_CH_DROPOUT channel (Remark 1) replica r drops the two residual
 * branches of every transformer block at its own rate; the mask is a pure function of
 * (seed, step, replica, site, element) from Philox-4x32-10.  With a HDET_CH_LABEL_SMOOTH
 * channel replica r's targets are (1 - eps_r) onehot + eps_r / C (MLP and transformer); with
 * a HDET_CH_ATTN_TEMP channel its attention scores are q.k / (sqrt(d_head) tau_r).  Writes grads_dev, the per-replica losses of this step and adds them to L_acc.
 * If losses_host is not NULL the call waits for the stream and copies the N losses there.
 * HDET_ESTATE for HDET_FLAT handles.                                                        */
int hdet_forward_backward(hdet_handle* h, const void* x_dev, const int32_t* y_dev,
                          float* losses_host);

/* Update t <- t+1 of every replica (Eq. 2 generalised to SGD-momentum / AdamW) with
 * eta_r = eta_bar * rho_{pi(r)} (Eq. 1, Eq. 9), eta_bar being the one-cycle value of
 * schedule index t-1 until the controller has taken over and the controller's base
 * afterwards.  grads_dev: [N][plane_stride] fp32 gradients, or NULL to use the buffer given
 * at creation.  In shared mode the replica mean of the gradients is formed inside the same
 * kernel.  With HDET_FUSE_CONVERGE and t mod T == 0 the replica mean of the updated
 * parameters (Eq. 3) is written to all replicas by the same kernel, and the following
 * hdet_converge is a no-op.  HDET_ESTATE once t == total_steps.                             */
int hdet_fanout_step(hdet_handle* h, const float* grads_dev, uint32_t flags);

/* One whole step of Algorithm 1's inner loop in a single call: forward, loss and backward on
 * (x_dev, y_dev) as hdet_forward_backward does, then update t <- t+1 (Sec. 3.2, Eq. 1-2) as
 * hdet_fanout_step(h, NULL, flags) does.  Parameters, optimizer state, bfloat16 copy, losses and
 * schedule state after the call are those of the two separate calls, bit for bit.  The gradient
 * buffer given at creation is still required but is NOT a defined output of this call: with
 * HDET_BF16_GEMM_FP32_MASTER, HDET_ADAMW, HDET_GRAD_PER_REPLICA and per-replica moments the
 * update of a weight matrix is applied inside the product that forms its gradient (every
 * replica's tile of dW is complete in one block, so Eq. 2 can be applied to it at once), and
 * that gradient is never written to memory: 26 instead of 30 + 4 bytes per weight and replica.
 * Biases, LayerNorm parameters, embeddings and matrices too small for this to pay (see
 * hdet_set_launch_shape), and every configuration outside the one named, take the ordinary
 * update.  With HDET_FUSE_CONVERGE on a sync step the replica mean of Eq. 3
 * is formed after all updates (by the update kernel, or by the converge kernel when some
 * updates were applied inside products), and the following hdet_converge is a no-op.
 * losses_host as for hdet_forward_backward.  HDET_ESTATE for HDET_FLAT handles and once
 * t == total_steps.                                                                          */
int hdet_train_step(hdet_handle* h, const void* x_dev, const int32_t* y_dev, uint32_t flags,
                    float* losses_host);

/* theta_r <- (1/N) sum_r' theta_r' for all r (Eq. 3), summed in the order r' = 0..N-1;
 * optimizer state is left per replica.  May be called at any t (Algorithm 1 calls it when
 * t mod T == 0; a caller whose S is not a multiple of T ends with one more call).           */
int hdet_converge(hdet_handle* h);

/* Sync-step bookkeeping (Algorithm 1, inside "t mod T = 0"): L_r = L_acc / T -- or the N
 * host values given in interval_losses_host -- then L_acc <- 0; if the controller is
 * enabled and t >= S_warm: weights (Eq. 4), hypergradient per channel (Eq. 5-6), velocity
 * and base (Eq. 7-8), fresh permutations (Eq. 9).  Runs on the device in one wavefront.
 * A non-finite loss leaves the controller state untouched (L_acc is still reset, the sync
 * step still counts as processed) and increments hdet_state.nonfinite.  When the losses come
 * from the host (interval_losses_host != NULL, N doubles) and the controller was due, the
 * call then returns HDET_ENONFINITE; with device-accumulated losses the call does not wait
 * for the stream, so it returns HDET_OK and the caller sees the event in the counter of the
 * next hdet_get_state.  HDET_ESTATE off a sync step or twice on the same one.               */
int hdet_autolr_update(hdet_handle* h, const double* interval_losses_host);

/* Waits for the stream and copies the state out / overwrites it (resume).                   */
int hdet_get_state(hdet_handle* h, hdet_state* out);
int hdet_set_state(hdet_handle* h, const hdet_state* in);

/* Kernel selection, for measurements and tests.  variant 0 (default): the fastest update
 * kernel for the case (one thread per replica column, or -- when gradients or parameters
 * must cross the replica axis -- a wavefront for each one to four replicas with an LDS
 * exchange, or the general kernel where that is faster); variant 1: the general kernel in which one thread walks the replica axis (any
 * N).  `blocks` > 0 sets the grid of the grid-stride kernels (0: library default).
 * variant | 2: the transformer's attention runs as separate batched GEMMs and softmax
 * kernels (scores and probabilities in device memory) also where the fused kernels apply.
 * variant | 4: hdet_train_step applies the update inside every weight-gradient product that
 * can carry it; by default only inside products with at least one 256 x 256 tile per
 * compute unit (the update of a smaller matrix is faster as part of the plane-wide launch).  */
int hdet_set_launch_shape(hdet_handle* h, int32_t variant, int32_t blocks);

/* Message of the last failure on this handle (or of the last failed hdet_create if h is
 * NULL); owned by the library.                                                              */
const char* hdet_last_error(hdet_handle* h);

/* Releases the control block and the handle.  hdet_destroy(NULL) is a no-op.                */
int hdet_destroy(hdet_handle* h);

/* ---------------------------------------------------------------------------------------
 * Operators of language models
 *
 * What a program calls that forms its own forward and backward pass -- N replicas of a
 * residual network with a root-mean-square norm, linear layers whose inputs and weights are
 * held in 8 bits, and an output layer with its cross-entropy -- and hands the gradients to
 * hdet_fanout_step.  No handle: every call enqueues its kernels on `stream` (hipStream_t or
 * NULL), waits for nothing, allocates nothing and keeps nothing; scratch memory is the
 * caller's.  Errors: HDET_EINVAL for what the argument checks refuse (nothing has been
 * enqueued then), HDET_EHIP; the message is that of hdet_last_error(NULL).
 *
 * Matrices are hdet_rows: N replicas of a matrix of rows, columns next to each other.  Strides
 * are in elements; any that keep rows and replicas apart (of an output: no two elements may
 * share memory).  Rows of whole 16-byte pieces at 16-byte boundaries are the fastest, by a
 * factor of two and more.  Outputs may not lie over inputs unless stated otherwise.  With no
 * rows the sums over them (gradients of weights, mean losses) are written as 0, and no workspace
 * is needed.
 *
 * A matrix in 8 bits: codes -127 .. 127 and one fp32 scale a row; entry = code * scale.  The
 * codes of a row start 16-byte aligned (row and replica strides are multiples of 16) and are
 * followed by zeros up to the next multiple of 16 columns: hdet_rmsnorm and hdet_quantise_rows
 * write them so.  Those two choose as scale the smallest power of two, from 2^-126 on, that
 * takes the row's largest entry to 127 or less, and round to the nearest code, halves to even.  A
 * power of two costs up to one of the eight bits and makes code * scale a bfloat16 number: the
 * gradients below multiply the values themselves, with nothing rounded on the way.  A row with an
 * entry that is not finite has scale NaN and codes 0.  (The type's largest numbers read back as
 * infinity: the nearest code stands for 2^128.)
 * ------------------------------------------------------------------------------------- */
enum { HDET_TYPE_F32 = 0, HDET_TYPE_BF16 = 1 };               /* element type of a matrix    */
#define HDET_MAX_NORM_WIDTH 32768                             /* a row is held in registers  */
#define HDET_MAX_CODES_WIDTH 131056                           /* 32-bit sums of code products */

typedef struct {
  void*   dev;             /* element (replica r, row i, column j) at r * replica_stride +    */
  int64_t row_stride;      /* i * row_stride + j; NULL: absent                               */
  int64_t replica_stride;
} hdet_rows;

/* Root-mean-square norm of a residual sum:
 *   u = x + resid (u = x without resid),  total = u,  rstd = 1 / sqrt(mean_j u_j^2 + eps),
 *   y_j = u_j rstd gain_j,  codes and scale: y in 8 bits.
 * The sum of squares, the norm and what is rounded to codes are held in 64 bits (u of bfloat16
 * summands in fp32); the norm is that of u before it is rounded to `total`.  total, y, codes (with
 * scale) and rstd are written where they are given.  total may be x or resid itself.          */
typedef struct {
  int32_t   n_replicas;
  int32_t   dtype;         /* HDET_TYPE_* of x, resid, total and y                           */
  int64_t   rows;          /* per replica, 0 allowed                                         */
  int32_t   width;         /* 1 .. HDET_MAX_NORM_WIDTH                                       */
  int32_t   reserved;
  double    eps;           /* >= 0                                                           */
  hdet_rows x, resid, total, y;
  hdet_rows codes;         /* int8                                                           */
  float*    scale_dev;     /* [N][rows]; with codes                                          */
  float*    rstd_dev;      /* [N][rows]                                                      */
  const float* gain_dev;   /* [width] per replica, gain_stride apart                         */
  int64_t   gain_stride;
} hdet_norm_args;
int hdet_rmsnorm(const hdet_norm_args* args, void* stream);

/* Backward pass: dy is the gradient at y (or at the values the codes stand for: rounding to 8
 * bits counts as the identity), dtotal (optional) what arrives at `total` by the residual
 * stream.  With h = total as stored and xh_j = h_j rstd:
 *   dx_j = rstd (dy_j gain_j - xh_j mean_i(dy_i gain_i xh_i)) + dtotal_j     (of x and of resid)
 *   dgain_j = sum over the rows of dy_j xh_j                       (in a fixed order; optional)
 * dx may be dy or dtotal itself.  workspace: hdet_rmsnorm_backward_workspace bytes (needed for
 * dgain only), 16-byte aligned.                                                             */
typedef struct {
  int32_t   n_replicas, dtype;                 /* HDET_TYPE_* of total, dy, dtotal and dx    */
  int64_t   rows;
  int32_t   width, reserved;
  hdet_rows total, dy, dtotal, dx;
  const float* rstd_dev;   /* [N][rows]                                                      */
  const float* gain_dev;
  int64_t   gain_stride;
  float*    dgain_dev;     /* [width] per replica, dgain_stride apart, or NULL               */
  int64_t   dgain_stride;
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_norm_grad_args;
int hdet_rmsnorm_backward_workspace(int32_t n_replicas, int64_t rows, int32_t width, size_t* bytes);
int hdet_rmsnorm_backward(const hdet_norm_grad_args* args, void* stream);

/* Rows to 8 bits (weights for hdet_quantised_linear, activations kept for the backward pass)
 * and back.  Reading back multiplies code and scale and rounds to dtype.                    */
typedef struct {
  int32_t   n_replicas, dtype;                 /* HDET_TYPE_* of values                      */
  int64_t   rows;
  int32_t   width, reserved;                   /* 1 .. HDET_MAX_NORM_WIDTH to quantise, ..   */
  hdet_rows values, codes;                     /* .. HDET_MAX_CODES_WIDTH to restore         */
  float*    scale_dev;                         /* [N][rows]                                  */
} hdet_codes_args;
int hdet_quantise_rows(const hdet_codes_args* args, void* stream);      /* reads values       */
int hdet_restore_rows(const hdet_codes_args* args, void* stream);       /* writes values      */

/* y = X W^T + bias with X [rows][d_in] and W [d_out][d_in] in 8 bits: whole-number sums of code
 * products (exact in 32 bits), rounded to fp32 (from 2^24 on), times the fp32 product of both scales,
 * plus bias in one fused step, and rounded to y's type.  Scales may be any numbers here whose product
 * fp32 holds.                                                                               */
typedef struct {
  int32_t   n_replicas, y_dtype;               /* HDET_TYPE_* of y                           */
  int64_t   rows;
  int32_t   d_in, d_out;                       /* d_in up to HDET_MAX_CODES_WIDTH            */
  hdet_rows codes, w_codes;
  const float* scale_dev;                      /* [N][rows]                                  */
  const float* w_scale_dev;                    /* [N][d_out]                                 */
  const float* bias_dev;                       /* [d_out] per replica, bias_stride apart, or NULL */
  int64_t   bias_stride;
  hdet_rows y;
} hdet_linear_args;
int hdet_quantised_linear(const hdet_linear_args* args, void* stream);

/* Gradients of that layer from the 8-bit copies and dy (bfloat16):
 *   dx = dy W (bfloat16, optional),  dw = dy^T X (fp32, optional),  db = sum over the rows of dy (fp32, optional)
 * in bfloat16 products with fp32 sums.  The values code * scale are read as bfloat16 numbers: exact
 * for the scales that this library chooses, rounded for others.  X (for dw) and W (for dx) pass
 * through the workspace in bfloat16: hdet_quantised_linear_backward_workspace bytes, 16-byte aligned
 * (a call without some of the results needs no more).                                        */
typedef struct {
  int32_t   n_replicas, reserved;
  int64_t   rows;
  int32_t   d_in, d_out;
  hdet_rows dy, codes, w_codes;
  const float* scale_dev;
  const float* w_scale_dev;
  hdet_rows dx, dw;
  float*    db_dev;
  int64_t   db_stride;
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_linear_grad_args;
int hdet_quantised_linear_backward_workspace(int32_t n_replicas, int64_t rows, int32_t d_in, int32_t d_out, size_t* bytes);
int hdet_quantised_linear_backward(const hdet_linear_grad_args* args, void* stream);

/* Output layer with its softmax cross-entropy, in pieces of the vocabulary: neither the logits
 * z = h W^T + bias nor their gradient are held for more than `piece` classes.  A row counts if its
 * label is in 0 .. classes - 1; c = rows of the replica that count, at least 1.
 *   row_loss = log sum_v exp(z_v) - z_label, 0 for rows that do not count
 *   mean_loss = sum of row_loss / c
 *   dz_v = (softmax(z)_v - [v = label]) / c, 0 for rows that do not count
 *   dh = dz W,   dw = dz^T h,   db = sum over the rows of dz
 * h, W and dh are bfloat16; sums are fp32.  dw is bfloat16 or fp32.  dh and a bfloat16 dw are
 * formed from dz rounded to bfloat16, an fp32 dw from dz in three such parts (24 bits) and with two more
 * products.  dh, dw and db are optional: without them only the losses are formed.
 * A row that does not count takes part in nothing, whatever its row of h holds (NaN and infinity
 * too).  A bias of -inf takes a class of a finite row of W out of the sum; a row that counts and has
 * no class left is NaN.
 * piece: classes at a time (taken down to whole groups of 256 or, below that, of 8), or 0 for the
 * library's choice.  The workspace (16-byte aligned) depends on it and on the results:
 * hdet_vocab_loss_workspace with the same arguments, HDET_VOCAB_NO_DW for the type of a dw that is
 * absent, HDET_VOCAB_LOSSES where dh and db are too.  Without dw it is no more than with one of
 * either type, for the losses alone no more than that.                                       */
enum { HDET_VOCAB_NO_DW = -1, HDET_VOCAB_LOSSES = -2 };
typedef struct {
  int32_t   n_replicas, dw_dtype;              /* HDET_TYPE_* of dw                          */
  int64_t   rows;
  int32_t   width, classes;
  int32_t   piece, reserved;
  hdet_rows h, w;                              /* bfloat16: [rows][width], [classes][width]  */
  const float* bias_dev;                       /* [classes] per replica, bias_stride apart, or NULL */
  int64_t   bias_stride;
  const int32_t* labels_dev;                   /* [N][rows]                                  */
  float*    row_loss_dev;                      /* [N][rows]                                  */
  float*    mean_loss_dev;                     /* [N]                                        */
  hdet_rows dh, dw;
  float*    db_dev;                            /* or NULL                                    */
  int64_t   db_stride;
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_vocab_args;
int hdet_vocab_loss_workspace(int32_t n_replicas, int64_t rows, int32_t width, int32_t classes, int32_t dw_dtype, int32_t piece, size_t* bytes);
int hdet_vocab_loss(const hdet_vocab_args* args, void* stream);

/* Norm of every head of the queries and keys with the rotation by position, in one pass.  A row of q
 * is q_heads heads of head_dim columns, one of k k_heads; q and k may be slices of one matrix.
 *   xh = x rstd, rstd = 1 / sqrt(mean_c x_c^2 + eps) over the head's columns,  u = xh gain   (u = x where the gain is NULL)
 *   y: for each pair t of the head's first `rotated` columns, with a = position * freq_t,
 *      y_1 = magnitude (u_1 cos a - u_2 sin a),  y_2 = magnitude (u_1 sin a + u_2 cos a);  y = u in the other columns
 * Pair t is the columns t and t + rotated / 2 (HDET_ROTARY_HALVES) or 2 t and 2 t + 1 (HDET_ROTARY_PAIRS).
 * freq_dev holds rotated / 2 frequencies in radians a position, in 64 bits, as any stretching for long
 * contexts leaves them (hdet_rotary_frequencies makes the usual ones); angles are formed and reduced
 * in 64 bits, good for any 32-bit position.  Row i of a replica stands at positions_dev[replica][i] or, where
 * that is NULL, at i mod period (i where period is 0).  Sums are fp32; those of squares 64 bits where they leave its range.
 * q_out may be q itself, with its strides, and k_out k itself; otherwise outputs lie apart from one another and from what the call reads.  (Refused
 * where the library sees it: matrices of one start, and of the same strides.)  k absent (dev NULL): q alone; its norm and the keys' are
 * each left out where their gain is NULL.                                                    */
enum { HDET_ROTARY_HALVES = 0, HDET_ROTARY_PAIRS = 1 };
#define HDET_MAX_ROTARY_DIM 256
typedef struct {
  int32_t   n_replicas, dtype;                 /* HDET_TYPE_* of q, k and their outputs      */
  int64_t   rows;
  int32_t   head_dim;                          /* 1 .. HDET_MAX_ROTARY_DIM                   */
  int32_t   q_heads, k_heads;                  /* heads * head_dim up to 2^20                */
  int32_t   rotated;                           /* even, 0 .. head_dim                        */
  int32_t   layout;                            /* HDET_ROTARY_*                              */
  int32_t   period;                            /* >= 0                                       */
  double    eps, magnitude;
  hdet_rows q, k, q_out, k_out;
  const float*   q_gain_dev;                   /* [head_dim] per replica, stride apart, or NULL: no norm */
  int64_t        q_gain_stride;
  const float*   k_gain_dev;
  int64_t        k_gain_stride;
  const int32_t* positions_dev;                /* [N][rows] or NULL                          */
  const double*  freq_dev;                     /* [rotated / 2]                              */
} hdet_rotary_args;
int hdet_head_rotary(const hdet_rotary_args* args, void* stream);

/* Backward pass: dq_out and dk_out are the gradients at the outputs, q and k what the forward pass
 * took (needed with a gain only).  With w = dq_out rotated back (by -a, times magnitude):
 *   dq = rstd (w gain - xh mean_c(w_c gain_c xh_c))   (w where the gain is NULL)
 *   dgain_c = sum over rows and heads of w_c xh_c     (in a fixed order; optional)
 * dq may be dq_out itself or q, with their strides, dk dk_out or k; otherwise as above.  workspace: hdet_head_rotary_backward_workspace bytes (needed
 * for the gains' gradients only), 16-byte aligned.                                          */
typedef struct {
  int32_t   n_replicas, dtype;
  int64_t   rows;
  int32_t   head_dim, q_heads, k_heads, rotated, layout, period;
  double    eps, magnitude;
  hdet_rows q, k, dq_out, dk_out, dq, dk;
  const float*   q_gain_dev;
  int64_t        q_gain_stride;
  const float*   k_gain_dev;
  int64_t        k_gain_stride;
  const int32_t* positions_dev;
  const double*  freq_dev;
  float*    dq_gain_dev;                       /* [head_dim] per replica, stride apart, or NULL */
  int64_t   dq_gain_stride;
  float*    dk_gain_dev;
  int64_t   dk_gain_stride;
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_rotary_grad_args;
int hdet_head_rotary_backward_workspace(int32_t n_replicas, int64_t rows, int32_t head_dim, int32_t q_heads, int32_t k_heads, size_t* bytes);
int hdet_head_rotary_backward(const hdet_rotary_grad_args* args, void* stream);

/* freq_host[t] = b^(-2 t / rotated), t < rotated / 2, stretched for contexts longer than those of training (factor 1: not):
 *   HDET_STRETCH_POSITIONS  every frequency over factor
 *   HDET_STRETCH_BASE       b = base factor^(rotated / (rotated - 2)) (rotated > 2): the fastest pair stays, the slowest is over factor
 *   HDET_STRETCH_PARTS      pairs that turn `fast` times or more over `context` positions stay, those that turn `slow` times or
 *                           less are over factor, in between the two frequencies are mixed in proportion to the turns
 * On the host; context, slow and fast are read by HDET_STRETCH_PARTS only (0 < slow < fast).  */
enum { HDET_STRETCH_POSITIONS = 0, HDET_STRETCH_BASE = 1, HDET_STRETCH_PARTS = 2 };
int hdet_rotary_frequencies(int32_t rotated, double base, int32_t stretch, double factor, double context, double slow, double fast, double* freq_host);

/* Attention of `seqs` sequences a replica, each q_len queries over kv_len keys: query i of sequence b is row
 * b * q_len + i of q and out, key j row b * kv_len + j of k and v.  A row of q and out is `heads` heads of head_dim
 * columns, one of k and v kv_heads heads; query head h reads key head h / (heads / kv_heads).
 *   z_ij = scale q_i . k_j;  with softcap > 0, z_ij = softcap tanh(z_ij / softcap);  with slopes, z_ij -= slope_h |position_i - j|
 *   out_i = sum_j p_ij v_j,  p_i = softmax of z_i over the keys that query i attends,  lse_i = log sum_j exp(z_ij)
 * Query i stands at key position positions_dev[replica][row] or, where that is NULL, at i + kv_len - q_len.  It attends the keys
 * of its sequence from the largest of 0, first_dev[row] and, with window > 0, position - window + 1 on, and before the
 * smallest of kv_len, end_dev[row] and, with causal, position + 1.  (Packed documents: first = the document's start.
 * A prefix that all queries see: causal 0, end = the larger of position + 1 and the prefix.  Padding and caches with
 * room: end; rows of padding: end = 0.)  A query that attends no key has out 0, lse -infinity and gradient 0.
 * Keys, values and queries take part only in the pairs that are attended: whatever the others hold, NaN and infinity
 * too, leaves no trace.
 * Scores, statistics and sums are fp32; bfloat16 inputs: p (relative to some score of the row) is rounded to bfloat16 for the product with v.
 * out may not lie over the inputs.  workspace: hdet_attention_workspace bytes, 16-byte aligned (what few queries over many keys leave in
 * pieces; 0 otherwise).                                                                                      */
#define HDET_MAX_ATTENTION_DIM 128
typedef struct {
  int32_t   n_replicas, dtype;                 /* HDET_TYPE_* of q, k, v and out             */
  int32_t   seqs, q_len, kv_len;               /* seqs * q_len up to 2^21, seqs * kv_len up to 2^28, n_replicas * seqs * q_len * heads up to 2^31 */
  int32_t   heads, kv_heads, head_dim;         /* heads a multiple of kv_heads, heads * head_dim up to 2^20 */
  int32_t   causal, window;                    /* window 0: none                             */
  double    scale, softcap;                    /* softcap 0: none                            */
  hdet_rows q, k, v, out;
  float*    lse_dev;                           /* [N][heads][seqs * q_len] or NULL           */
  const float*   slopes_dev;                   /* [heads] per replica, slopes_stride apart, or NULL */
  int64_t        slopes_stride;
  const int32_t* positions_dev;                /* [N][seqs * q_len] or NULL                  */
  const int32_t* first_dev;
  const int32_t* end_dev;
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_attention_args;
int hdet_attention_workspace(int32_t n_replicas, int32_t seqs, int32_t q_len, int32_t kv_len, int32_t heads, int32_t kv_heads, int32_t head_dim, size_t* bytes);
int hdet_attention(const hdet_attention_args* args, void* stream);

/* Backward pass, from what the forward pass took, its out and lse, and dout (all with the same mask arguments):
 *   dv_j = sum_i p_ij dout_i,  dz_ij = p_ij (dout_i . v_j - dout_i . out_i),  times 1 - tanh^2 with softcap
 *   dq_i = scale sum_j dz_ij k_j,  dk_j = scale sum_i dz_ij q_i       (over the heads that share the key head; in a fixed order)
 * bfloat16 inputs: for their products p and, for dk, dz are rounded to bfloat16; dz for dq, and where few queries make dk and dv all of them, are
 * the sum of two bfloat16 numbers.  dq, dk and dv may not lie over the inputs.  workspace: hdet_attention_backward_workspace bytes, 16-byte aligned. */
typedef struct {
  int32_t   n_replicas, dtype;
  int32_t   seqs, q_len, kv_len, heads, kv_heads, head_dim, causal, window;
  double    scale, softcap;
  hdet_rows q, k, v, out, dout, dq, dk, dv;
  const float*   lse_dev;
  const float*   slopes_dev;
  int64_t        slopes_stride;
  const int32_t* positions_dev;
  const int32_t* first_dev;
  const int32_t* end_dev;
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_attention_grad_args;
int hdet_attention_backward_workspace(int32_t n_replicas, int32_t seqs, int32_t q_len, int32_t kv_len, int32_t heads, int32_t kv_heads, int32_t head_dim, size_t* bytes);
int hdet_attention_backward(const hdet_attention_grad_args* args, void* stream);

/* Gradients of many tensors, bounded by their common norm, on the way into the plane that hdet_fanout_step reads.
 *   norm_r = sqrt of the sum of g^2 over all tensors of replica r; with HDET_GRAD_SHARED that of the replicas' mean gradient, the same for all r
 *   out = g factor_r,  factor_r = max_norm / norm_r where norm_r > max_norm, else 1
 * Sums are 64 bits in a fixed order, the factor is rounded to fp32.  A norm that is not finite leaves factor 1: norm_dev says so to
 * the caller.  (A norm that is finite and beyond fp32 is written as infinity and bounds the gradients all the same.)  max_norm infinite: nothing is
 * bounded (and without `out` only the norm is formed).
 * tensors_host: read during the call only (the addresses in it are what a captured graph keeps).  Every tensor is an hdet_rows of rows x width;
 * `out` is fp32 in any strides, or absent: the gradients themselves are scaled, in their type.  No two elements of outputs (and of gradients that are
 * scaled in place) may share memory, within a tensor or between two, nor may what is written lie over another tensor's gradient; an output may be its
 * own gradient itself, an fp32 one, with its strides.  A tensor that is written where another one starts is refused, and so is an output that is seen
 * to lie over its own gradient otherwise.
 * Elements between the tensors of a plane are left as they are.
 * workspace: hdet_clip_gradients_workspace bytes, 16-byte aligned.                           */
#define HDET_MAX_GRAD_TENSORS 65536
typedef struct {
  hdet_rows grad, out;
  int64_t   rows;                              /* rows * width up to 2^40                    */
  int32_t   width;
  int32_t   dtype;                             /* HDET_TYPE_* of grad                        */
} hdet_grad_tensor;
typedef struct {
  int32_t   n_replicas, n_tensors;             /* 0 tensors: norm 0                          */
  const hdet_grad_tensor* tensors_host;
  int32_t   grad_mode, reserved;               /* HDET_GRAD_PER_REPLICA or HDET_GRAD_SHARED  */
  double    max_norm;                          /* >= 0                                       */
  float*    norm_dev;                          /* [N]                                        */
  void*     workspace_dev;
  size_t    workspace_bytes;
} hdet_clip_args;
int hdet_clip_gradients_workspace(int32_t n_replicas, int32_t n_tensors, size_t* bytes);
int hdet_clip_gradients(const hdet_clip_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HDET_H */
