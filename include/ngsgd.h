/*
 * ngsgd.h - C ABI of the MI355X NG-SGD minibatch-step library (libngsgd.so).
 *
 * One worker's natural-gradient SGD step from "Parallel training of DNNs with
 * Natural Gradient and Parameter Averaging" (Povey, Zhang, Khudanpur):
 * forward, objective, backward, online natural-gradient preconditioning of
 * both matrices that enter each layer's update, the rank-N update itself, and
 * on-device parameter averaging across replicas held on the same GPU.
 *
 * General conventions
 *   - All `dev_*` pointers are DEVICE pointers (HIP global memory on the
 *     current device).  Everything else is host memory.
 *   - Matrices are row-major fp32.  A leading dimension `ld` counts floats
 *     between consecutive rows; it must be a multiple of 4 and the base
 *     pointer 16-byte aligned.
 *   - The library allocates no device memory.  Every handle lives in a device
 *     workspace the caller allocates (size from the *_workspace_bytes call,
 *     256-byte aligned) and keeps alive until *_destroy.  Inputs and outputs
 *     stay caller-owned.
 *   - All work is enqueued on the HIP stream passed as `hip_stream` (a
 *     hipStream_t cast to void*; NULL is the default stream) and the calls
 *     return without waiting for it.  Scalars results are written to device
 *     memory.  Calls on the same handle must be issued in order on one stream.
 *     Handles are not thread-safe.
 *   - A network also owns up to three internal streams (default priority;
 *     ngsgd_config.side_streams): the factor updates of its preconditioners
 *     run there, each group of factors starting as soon as its matrix exists,
 *     so that they overlap the rest of the step and the following minibatch.
 *     Every call on the handle
 *     orders itself after whatever it depends on; a caller that wants the
 *     stream it passed to cover all of a step's work (to time it, or to read
 *     the handle's device memory directly) calls ngsgd_join first.
 *   - Every function returns NGSGD_OK (0) or a negative NGSGD_E* code.  After
 *     an error the handle's state is unchanged when the error is an argument
 *     error, and unspecified for NGSGD_EHIP.
 */
#ifndef NGSGD_H_
#define NGSGD_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NGSGD_OK 0
#define NGSGD_EINVAL (-1)    /* bad argument: NULL, size, alignment, rank >= dim, N > max_batch ... */
#define NGSGD_ENOMEM (-2)    /* workspace too small */
#define NGSGD_EHIP (-3)      /* a HIP runtime call failed; see ngsgd_last_hip_error() */
#define NGSGD_EUNSUPPORTED (-4)

#define NGSGD_TANH 0
#define NGSGD_PNORM 1
#define NGSGD_LAYERNORM 16   /* added to either: a layer norm follows, with a weight and a bias of its own */

/* Element types of the operators that take 16-bit data. */
#define NGSGD_FLOAT32 0
#define NGSGD_BFLOAT16 1
#define NGSGD_FLOAT16 2
/* Types of tokens and labels. */
#define NGSGD_INT32 3
#define NGSGD_INT64 4

#define NGSGD_MAX_LAYERS 16
#define NGSGD_MAX_RANK 96    /* the R x R update runs in one workgroup's LDS */

#define NGSGD_METHOD_ONLINE 0 /* Fisher factors from previous minibatches, App. B (the default)   */
#define NGSGD_METHOD_SIMPLE 1 /* Fisher factors from the other rows of the minibatch, App. A    */
#define NGSGD_METHOD_ADAMW 2  /* no factors: AdamW with the plain gradient, moments in fp32     */
#define NGSGD_METHOD_ADAMW8 3 /* the same with moments in 8 bits                                */

#define NGSGD_SIDE_INPUT 0   /* preconditioner of the layer-input matrix [X_l, 1]   */
#define NGSGD_SIDE_OUTPUT 1  /* preconditioner of the output-derivative matrix O_l  */

typedef struct ngsgd_net ngsgd_net;          /* one replica: weights + 2I preconditioners */
typedef struct ngsgd_precond ngsgd_precond;  /* one instance of the online method         */

/* Network description (host memory, copied by ngsgd_create).
 * dims[0] is the input dimension, dims[1..n_layers] the output dimension of each affine layer;
 * nonlin[l] (l < n_layers-1) follows affine layer l, the last affine layer feeds a log-softmax.
 * A p-norm layer (p = 2) maps groups of `pnorm_group` adjacent outputs to their 2-norm, so the
 * next layer's input dimension is dims[l+1] / pnorm_group (must divide).  Each affine layer keeps
 * its bias as the last column of its weight matrix: W_l is dims[l+1] x (in_dim_l + 1)
 * (Sec. 4.4 of the paper).  nonlin[l] | NGSGD_LAYERNORM puts a layer norm (epsilon 1e-5) between the nonlinearity
 * (renormalised or not) and the next layer; its weight and bias have no input and output side to precondition:
 * AdamW updates them with every method, at the step's learning rate (see ngsgd_set_adamw).  With the AdamW methods
 * max_change_per_sample has to be 0, and ranks and the other numbers of the preconditioner are not used.
 * Defaults of App. B.4/B.5: rank_in 20, rank_out 80, alpha 4,
 * num_samples_history 2000, epsilon 1e-10, update_period 4, always_update_first 10. */
typedef struct {
  int32_t n_layers;
  const int32_t* dims;
  const int32_t* nonlin;
  int32_t pnorm_group;
  int32_t max_batch;              /* largest minibatch a step will be given            */
  int32_t rank_in, rank_out;      /* 0 disables preconditioning on that side           */
  float alpha;                    /* identity smoothing, Sec. 4.8                      */
  float num_samples_history;      /* S in eta = 1 - exp(-N/S), App. B.4                */
  float epsilon;                  /* floor on rho and D, App. B.2-B.3                  */
  int32_t update_period;          /* J: factors updated when t < always_update_first   */
  int32_t always_update_first;    /*    or J divides t, App. B.4                       */
  int32_t renorm;                 /* 1: rows leave each p-norm layer with unit rms     */
  float max_change_per_sample;    /* App. C.3; 0 disables the limit (paper: 0.075)     */
  int32_t method;                 /* NGSGD_METHOD_ONLINE (App. B), _SIMPLE (App. A), _ADAMW or _ADAMW8 */
  float simple_epsilon;           /* floor on tr(X^T X) in beta, App. A.2 (1e-20)      */
  int32_t side_streams;           /* internal streams for the factor updates: 0 = chosen
                                   * by the layers, the ranks and the classes (1 or 2), else
                                   * 1..3.  One: all updates start after the backward pass;
                                   * two: the last layer's derivatives and the layer inputs
                                   * start after the forward pass, the other derivatives
                                   * after the backward pass (2 % shorter for deep networks
                                   * with a rank above 80 and ten times as many classes as
                                   * units in a layer, mostly 2 to 6 % longer for others);
                                   * three start the upper hidden layers in the middle of
                                   * the backward pass.  One is better when
                                   * many networks share the GPU, which has few hardware
                                   * queues per process                                    */
} ngsgd_config;

/* ---- one preconditioner instance (App. B) ------------------------------------------------- */

/* Device workspace needed by one instance for matrices of up to max_batch rows. */
int ngsgd_precond_workspace_bytes(int32_t dim, int32_t rank, int32_t max_batch, size_t* out_bytes);

/* Creates an instance in `dev_workspace`.  Requires 0 <= rank <= NGSGD_MAX_RANK, rank < dim.
 * The state (W_t = E_t^{1/2} R_t, D_t, rho_t) is built from the first matrix it is given
 * (App. B.3.2), which therefore needs more than `rank` rows. */
int ngsgd_precond_create(int32_t dim, int32_t rank, int32_t max_batch, float alpha,
                         float num_samples_history, float epsilon, int32_t update_period,
                         int32_t always_update_first, void* dev_workspace, size_t workspace_bytes,
                         ngsgd_precond** out);
int ngsgd_precond_destroy(ngsgd_precond* p);

/* Forgets the state: the next call re-initialises from its input, as a new process does. */
int ngsgd_precond_reset(ngsgd_precond* p);

/* The online natural-gradient call of Sec. 4.6 / App. B.5: overwrites the N x dim matrix dev_M
 * (leading dimension ld) with gamma_t * M * G_t^{-1}, which has the Frobenius norm of M, using
 * the factor estimated from the previous calls; then, when t < always_update_first or
 * update_period divides t, updates the factor with M.  t counts calls since creation / reset.
 *   dev_gamma     (optional, 1 float)  receives gamma_t (eq. gammat)
 *   dev_rownorm2  (optional, N floats) receives the squared 2-norm of each output row
 * Requires N <= max_batch; on the first call after creation/reset also N > rank. */
int ngsgd_precondition(ngsgd_precond* p, float* dev_M, int32_t N, int32_t ld, float* dev_gamma,
                       float* dev_rownorm2, void* hip_stream);

/* Copies the state out: dev_W (rank x dim floats, dense), dev_d (rank doubles, diag D_t),
 * dev_rho (1 double); *t_host receives the call counter.  Any pointer may be NULL. */
int ngsgd_precond_get_state(const ngsgd_precond* p, float* dev_W, double* dev_d, double* dev_rho,
                            int64_t* t_host, void* hip_stream);

/* Diagnostics of the latest factor update, copied to HOST memory after waiting for the stream:
 * flags (bit 0: orthogonality check still pending, 1: an eigenvalue of Z_t was floored, 2: the factor was
 * re-orthogonalised (App. B.3.1), 3: the eigen-solver hit its sweep limit; 4, of the latest first factor: its matrix was
 * reduced from memory, see ngsgd_set_wait_limit_us) and the Jacobi sweeps it used (1 where the direct solver served). */
int ngsgd_precond_diagnostics(const ngsgd_precond* p, int32_t* flags_host, int32_t* sweeps_host,
                              void* hip_stream);

/* Installs a state given in the definitional form of App. B.1: dev_R (rank x dim doubles, dense,
 * orthonormal rows), dev_d (rank doubles > 0), rho > 0, and the call counter t >= 1.
 * W_t = E_t^{1/2} R_t is formed on the device (eq. beta2, etii, wt:def). */
int ngsgd_precond_set_state(ngsgd_precond* p, const double* dev_R, const double* dev_d, double rho,
                            int64_t t, void* hip_stream);

/* ---- the simple method (App. A), stateless ---------------------------------------------------- */

/* Device workspace for matrices of up to max_rows rows and dim columns. */
int ngsgd_simple_workspace_bytes(int32_t max_rows, int32_t dim, size_t* out_bytes);

/* Overwrites the N x D matrix dev_M (leading dimension ld, a multiple of 4, 16-byte aligned rows)
 * with gamma * Xhat, where row i of Xhat is (beta I + F_i)^{-1} x_i, F_i = sum_{j != i} x_j x_j^T / (N-1)
 * is estimated from the other rows, beta = alpha max(tr(X^T X), epsilon) / (N D), and gamma restores
 * the Frobenius norm of the input (App. A.2).  Computed as in App. A.3: one inverse of size
 * min(N, D) (column space if N > D, row space otherwise) and a scalar correction per row.
 *   dev_workspace  caller-owned scratch of at least ngsgd_simple_workspace_bytes(N, D) bytes,
 *                  256-byte aligned; holds nothing between calls
 *   dev_gamma      (optional, 1 float)  receives gamma
 *   dev_rownorm2   (optional, N floats) receives the squared 2-norm of each output row
 * Requires N >= 2.  Returns NGSGD_EINVAL / NGSGD_ENOMEM before anything is enqueued. */
int ngsgd_precondition_simple(float* dev_M, int32_t N, int32_t D, int32_t ld, float alpha, float epsilon,
                              void* dev_workspace, size_t workspace_bytes, float* dev_gamma,
                              float* dev_rownorm2, void* hip_stream);

/* The same call for callers that cannot allocate device memory or bring a workspace (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the scratch is a fixed array of
 * NGSGD_SIMPLE_STATIC_BYTES in the library's device image, one copy per GPU, held until the process
 * ends.  Allocates nothing, on the device or through any library.  Same arguments, results and
 * errors as ngsgd_precondition_simple; in addition NGSGD_ENOMEM when
 * ngsgd_simple_workspace_bytes(N, D) exceeds NGSGD_SIMPLE_STATIC_BYTES (16 MiB: up to 512 x 5000, or
 * any shape whose scratch fits), before anything is enqueued.  All calls on one GPU share the array:
 * calls that overlap in time on the same GPU (different streams, different threads) race; issue them
 * on one stream or order them yourself.  Must be called with the target device current. */
#define NGSGD_SIMPLE_STATIC_BYTES (16 * 1024 * 1024)
int ngsgd_precondition_simple_static(float* dev_M, int32_t N, int32_t D, int32_t ld, float alpha,
                                     float epsilon, float* dev_gamma, float* dev_rownorm2,
                                     void* hip_stream);

/* ---- layer norm ------------------------------------------------------------------------------- */

/* y = xhat * weight + bias,  xhat = (x - mean) * rstd,  for each of the N rows of D numbers, with the row's mean
 * and rstd = (variance + epsilon)^(-1/2) (variance with divisor D, from the differences to the mean).
 *   type           of x and y (NGSGD_FLOAT32, NGSGD_BFLOAT16 or NGSGD_FLOAT16)
 *   weight_type    of weight and bias: `type` or NGSGD_FLOAT32
 *   dev_weight, dev_bias (optional, D numbers each): without them ones and zeros
 *   dev_mean, dev_rstd (optional, N floats each) receive what the backward pass needs
 * Statistics and sums are in fp32, outputs are rounded once.  Leading dimensions count elements, at least D and otherwise free:
 * rows need no alignment beyond an element's (rows on multiples of 16 bytes are faster).  dev_y may be dev_x with
 * the same leading dimension; other overlaps are not allowed.  N may be 0.  Rows do not mix: an infinity or NaN
 * stays in its row.  D is at most 2^25.  epsilon is finite and not negative; with 0 a row of equal numbers gives NaN, or
 * what rounding leaves of it.  A variance above what fp32 holds is infinite: rstd is 0. */
int ngsgd_layernorm_forward(const void* dev_x, int64_t ldx, int32_t type, const void* dev_weight,
                            const void* dev_bias, int32_t weight_type, int64_t N, int32_t D, float epsilon,
                            void* dev_y, int64_t ldy, float* dev_mean, float* dev_rstd, void* hip_stream);

/* Device workspace that ngsgd_layernorm_backward needs for the weight's and the bias' gradient of up to max_rows
 * rows; it holds nothing between calls. */
int ngsgd_layernorm_workspace_bytes(int64_t max_rows, int32_t D, size_t* out_bytes);

/* Gradients of the above for the derivative dy of a scalar, with the mean and rstd of the forward pass:
 *   dev_dx       (optional, N x D) = rstd * (g - mean(g) - xhat * mean(g * xhat)),  g = dy * weight
 *   dev_dweight  (optional, D, weight_type) = sum over the rows of dy * xhat
 *   dev_dbias    (optional, D, weight_type) = sum over the rows of dy
 * At least one of them.  The sums over the rows are in fp32 in an order that depends on the sizes alone: a call repeated
 * gives the same bits.  dev_dx may be dev_dy with the same leading dimension; other overlaps are not allowed.
 * With N = 0 the sums are zero.  dev_workspace (256-byte aligned) is only needed with dev_dweight or dev_dbias. */
int ngsgd_layernorm_backward(const void* dev_dy, int64_t lddy, const void* dev_x, int64_t ldx, int32_t type,
                             const void* dev_weight, int32_t weight_type, const float* dev_mean,
                             const float* dev_rstd, int64_t N, int32_t D, void* dev_dx, int64_t lddx,
                             void* dev_dweight, void* dev_dbias, void* dev_workspace, size_t workspace_bytes,
                             void* hip_stream);

/* ---- embedding -------------------------------------------------------------------------------- */

/* y_i = scale * table[token_i]: row token_i of a table of V rows of D numbers, for each of N tokens.
 *   dev_tokens     N of index_type (NGSGD_INT32 or NGSGD_INT64), dense.  One outside [0, V) is padding: its y is zeros
 *   table_type     NGSGD_FLOAT32, or `type`
 *   type           of y (NGSGD_FLOAT32, NGSGD_BFLOAT16 or NGSGD_FLOAT16)
 * The product is in fp32 and rounded once.  Leading dimensions as with layer norm: at least D, in elements, no alignment.  y
 * and the table do not overlap.  N may be 0 (with V >= 1).  N and V are at most 2^30, D at most 2^25. */
int ngsgd_embedding_forward(const void* dev_tokens, int32_t index_type, int64_t N, const void* dev_table, int64_t ldt,
                            int32_t table_type, int64_t V, int32_t D, float scale, void* dev_y, int64_t ldy,
                            int32_t type, void* hip_stream);

/* Device workspace that ngsgd_embedding_backward needs for up to max_tokens tokens; it holds nothing between calls. */
int ngsgd_embedding_workspace_bytes(int64_t max_tokens, int64_t V, int32_t D, size_t* out_bytes);

/* The table's gradient for the derivative dy of a scalar by y (N x D, `type`):
 *   dtable[v] = scale * sum of the dy_i with token_i = v          (V x D, table_type)
 * and zeros in rows that no token names; with accumulate = 1 the sums are added to what dtable holds, and rows that no token
 * names are neither read nor written (a table that is the last layer's weights too).  Tokens are sorted, and sums are in fp32 in an
 * order that depends on the tokens and sizes alone: a call repeated gives the same bits.  Rounded once.
 * dev_workspace is 256-byte aligned; calls that may run at the same time need one each. */
int ngsgd_embedding_backward(const void* dev_dy, int64_t lddy, int32_t type, const void* dev_tokens, int32_t index_type,
                             int64_t N, int64_t V, int32_t D, float scale, void* dev_dtable, int64_t lddt,
                             int32_t table_type, int32_t accumulate, void* dev_workspace, size_t workspace_bytes,
                             void* hip_stream);

/* ---- cross-entropy ---------------------------------------------------------------------------- */

/* loss_i = log sum_j exp(x_ij) - x_i,label_i  for each of N rows of V logits, and the gradient of
 * scale * (sum of the losses):  dlogits_ij = scale * (softmax_ij - [j = label_i]).
 *   dev_labels     N of index_type, dense.  A row whose label is outside [0, V) does not count: its loss and gradient are
 *                  zeros, its logits are not read
 *   dev_loss       (optional) N floats
 *   dev_dlogits    (optional) N x V of `type`; may be dev_logits with the same leading dimension, other overlaps are not allowed
 *   dev_scale      (optional, 1 float) is multiplied to scale: a loss scale, or one over a number of labels that only the device knows
 * One of loss and gradient at least.  Statistics are in fp32, and what the label's own term leaves of the sum is kept apart from it, so that
 * the loss and the label's gradient of a row that is as good as decided keep their digits; the gradient is rounded once.  A logit of -infinity is
 * a class that is not there: its probability is 0, and as the label's it gives a loss of infinity.  A row with a NaN or
 * +infinity, or with -infinity alone, has a loss and a gradient of NaN; finite logits of any size never do (where the largest of a row is
 * beyond 2^27, a term that is less than 2^-60 of its own may count as 0).  Sums are in an order that depends on the sizes alone.  Leading dimensions are
 * at least V.  N is at most 2^30 and V 2^29.  dev_workspace (256-byte aligned) holds nothing between calls; calls that may run at the
 * same time need one each. */
int ngsgd_cross_entropy_workspace_bytes(int64_t max_rows, int32_t V, size_t* out_bytes);
int ngsgd_cross_entropy(const void* dev_logits, int64_t ld, int32_t type, const void* dev_labels, int32_t index_type,
                        int64_t N, int32_t V, float* dev_loss, float scale, const float* dev_scale, void* dev_dlogits,
                        int64_t ldd, void* dev_workspace, size_t workspace_bytes, void* hip_stream);

/* ---- norm of all gradients, clipping ---------------------------------------------------------- */

/* Device workspace of the two calls below for up to so many tensors of any sizes; it holds nothing between calls. */
int ngsgd_grad_norm_workspace_bytes(int32_t n_tensors, size_t* out_bytes);

/* norm = sqrt(sum of the squares of all elements of all tensors), and factor = max_norm / norm where norm > max_norm, else 1.
 *   sizes, dev_grads (host arrays) elements and address of each tensor, dense, of `type`; one whose address is NULL or whose size is 0
 *                    does not count
 *   max_norm         not negative; infinity for the norm alone (factor 1)
 *   dev_norm, dev_factor (1 float each, either may be NULL)
 * Squares are summed in fp64, in an order that depends on the sizes alone, so no square overflows or vanishes; the norm is rounded to
 * fp32 and the factor formed before that (rounded to fp32 itself, with fewer digits below 2^-126).  An infinity among the elements gives the norm infinity and the factor 0 (max_norm
 * infinity: 1), a NaN gives NaN for both.  The factor is what ngsgd_adamw_step takes as dev_grad_scale.  At most 2^40 elements a tensor. */
int ngsgd_grad_norm(int32_t n_tensors, const int64_t* sizes, const void* const* dev_grads, int32_t type, double max_norm,
                    float* dev_norm, float* dev_factor, void* dev_workspace, size_t workspace_bytes, void* hip_stream);

/* The same, and every element times the factor, rounded once, to dev_out[i] (of the same type and size; NULL only where dev_grads[i] is or the
 * size is 0); dev_out NULL: in place, where with a factor of 1 nothing is read again or written.  dev_out[i] may be dev_grads[i]; where
 * outputs share memory with each other or with another gradient the call is refused (NGSGD_EINVAL). */
int ngsgd_grad_clip(int32_t n_tensors, const int64_t* sizes, const void* const* dev_grads, int32_t type, double max_norm,
                    void* const* dev_out, float* dev_norm, float* dev_factor, void* dev_workspace,
                    size_t workspace_bytes, void* hip_stream);

/* ---- AdamW over many tensors ------------------------------------------------------------------- */

typedef struct ngsgd_adamw ngsgd_adamw;  /* the moments and step count of a list of tensors */

/* Host memory, copied by ngsgd_adamw_create. */
typedef struct {
  int32_t n_tensors;
  void* const* dev_params;    /* each tensor dense; NULL only where its size is 0           */
  const int64_t* sizes;       /* elements; no two tensors may share memory                  */
  const float* weight_decay;  /* of each tensor; NULL: 0                                    */
  const float* rate;          /* factor of each tensor on the learning rate; NULL: 1        */
  int32_t param_type;         /* NGSGD_FLOAT32, _BFLOAT16 or _FLOAT16                       */
  int32_t grad_type;          /* that of the parameters, NGSGD_FLOAT32, or any with fp32 parameters */
  int32_t state_bits;         /* 32: moments in fp32; 8: codes with an exponent for every 256 elements */
  int32_t master;             /* 1: parameters in 16 bits are rounded from fp32 copies that are kept */
  double beta1, beta2;        /* in [0, 1)                                                  */
  float epsilon;              /* 0 or a positive normal number                              */
} ngsgd_adamw_config;

int ngsgd_adamw_workspace_bytes(const ngsgd_adamw_config* cfg, size_t* out_bytes);

/* Zero moments, step count 0, fp32 copies from the parameters.  The parameters stay where they are until
 * ngsgd_adamw_destroy.  Synchronises the device (so not under capture). */
int ngsgd_adamw_create(const ngsgd_adamw_config* cfg, void* dev_workspace, size_t workspace_bytes,
                       ngsgd_adamw** out);
int ngsgd_adamw_destroy(ngsgd_adamw* h);

/* One step, t = 1, 2, ...:
 *   g = grad_scale * gradient;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr * weight_decay) - lr * (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + epsilon)
 * in fp32, from the fp32 copy of p if there is one.
 *   dev_grads   (host array) the gradient of each tensor, dense, of grad_type; a tensor whose gradient is NULL is
 *               left as it is, while the step counts
 *   dev_lr, dev_grad_scale (optional, 1 float each) are multiplied to lr and grad_scale: a schedule or the
 *               factor of a clipped norm that only the device knows
 * The step count lives on the device, so a captured step counts on at each replay (with the gradients' addresses,
 * lr and grad_scale of its capture; the workspace has to be there as long as the graph).  At most 16 pieces of work (4096 elements
 * of a tensor, or its rest) in no more than 448 tensors take one launch; any other step takes one that counts it and one for every
 * 448 tensors.  Moments are fp32's: a v above what fp32 holds is infinite, and its element stays where it is (in 8 bits: NaN).
 * Moments in 8 bits: m as a sign, 4 bits of exponent and 3 behind the point, sqrt(v) as 5 and 3 bits, below an exponent that 256
 * elements share; p is updated from this step's moments before they are coded.  They are rounded down
 * after a share of a step has been added, frac(i A + t B) of the element's place i in the flat arrays and t (A, B = 0x9E3779B1,
 * 0x6A09E667 over 2^32, the upper 20 bits), so that over the steps changes much smaller than a code's step
 * add up.  An infinity or NaN makes its own element NaN, not its block; an m above 1.875 2^127 and a root above 1.875 2^63 are
 * held as those. */
int ngsgd_adamw_step(ngsgd_adamw* h, const void* const* dev_grads, float lr, const float* dev_lr,
                     float grad_scale, const float* dev_grad_scale, void* hip_stream);

/* The flat arrays: their length, and their addresses in the workspace (NULL for moments in 8 bits, or without fp32
 * copies).  Tensor k's elements start behind those of the tensors before it, each rounded up to a multiple of 256.  What lies
 * between the tensors is zero and no step changes it. */
int ngsgd_adamw_arrays(const ngsgd_adamw* h, int64_t* elements, float** dev_m, float** dev_v, float** dev_master);

/* The moments as values, to flat arrays in fp32 or bf16 (which holds those of 8-bit codes exactly, but for a v below
 * 2^-126; 16-byte aligned), and the step count.  Any of the three may be NULL. */
int ngsgd_adamw_get_state(const ngsgd_adamw* h, void* dev_m, void* dev_v, int32_t type, int64_t* dev_t,
                          void* hip_stream);

/* Installs moments (flat, zeros between the tensors, 16-byte aligned; NULL: zeros; in 8 bits rounded to the nearest code, which gives back what
 * ngsgd_adamw_get_state gave) and the step count t >= 0.  fp32 copies are taken from dev_master (flat), with the parameters
 * rounded from it, or with NULL from the parameters. */
int ngsgd_adamw_set_state(ngsgd_adamw* h, const float* dev_m, const float* dev_v, const float* dev_master,
                          int64_t t, void* hip_stream);

/* ---- one replica of the network -------------------------------------------------------------- */

int ngsgd_workspace_bytes(const ngsgd_config* cfg, size_t* out_bytes);

/* Creates a replica in `dev_workspace`; all weights start at zero (set them with
 * ngsgd_set_params; App. C.7 describes the initialisation the paper uses).  Synchronises the
 * device once. */
int ngsgd_create(const ngsgd_config* cfg, void* dev_workspace, size_t workspace_bytes,
                 ngsgd_net** out);
int ngsgd_destroy(ngsgd_net* net);

/* One NG-SGD minibatch step (Sec. 2, 4.5-4.7): maximises sum_i log p(y_i | x_i) by
 * W_l += lr * a_l * Obar_l^T Xbar_l for every layer (with the AdamW methods by an AdamW step along O_l^T X_l), gradients
 * summed over the minibatch.
 *   dev_x       N x dims[0] features, dense (ld = dims[0], which must be a multiple of 4)
 *   dev_labels  N class indices in [0, dims[n_layers])
 *   dev_logprob_sum (optional, 1 double) receives sum_i log p(y_i | x_i) evaluated before the update */
int ngsgd_step(ngsgd_net* net, const float* dev_x, const int32_t* dev_labels, int32_t N, float lr,
               double* dev_logprob_sum, void* hip_stream);

/* Makes hip_stream wait for what the network still has in flight on its internal streams (the latest
 * factor updates); enqueues nothing else. */
int ngsgd_join(ngsgd_net* net, void* hip_stream);

/* Parameter averaging of Sec. 3.1: every replica's weights are replaced by the arithmetic mean over
 * the n replicas (same configuration, same device), and so are their layer norms'.  With reset_preconditioners != 0 all
 * their preconditioners are reset, as the paper's re-spawned processes do (App. B.3.2), and AdamW's moments.
 * The replicas may have been stepped on other streams than hip_stream: the averaging kernel waits (on
 * the device) for each replica's latest ngsgd_step and factor updates, and each replica's next call
 * waits for the averaged weights, so the caller needs no synchronisation of its own.  (The call records an
 * event on the stream of each replica's latest ngsgd_step: those streams must still exist, and no other
 * host thread may be enqueuing a step of these replicas during the call.) */
int ngsgd_average(ngsgd_net* const* nets, int32_t n, int32_t reset_preconditioners, void* hip_stream);

/* Weights of one layer as a dense dims[layer+1] x (in_dim+1) row-major matrix, bias last. */
int ngsgd_get_params(const ngsgd_net* net, int32_t layer, float* dev_out, void* hip_stream);
int ngsgd_set_params(ngsgd_net* net, int32_t layer, const float* dev_in, void* hip_stream);

/* Weight (ones at first) and bias (zeros) of the layer norm behind hidden layer `layer`, as many as the next layer has
 * inputs; either pointer may be NULL.  NGSGD_EINVAL where there is none. */
int ngsgd_get_norm(const ngsgd_net* net, int32_t layer, float* dev_weight, float* dev_bias, void* hip_stream);
int ngsgd_set_norm(ngsgd_net* net, int32_t layer, const float* dev_weight, const float* dev_bias, void* hip_stream);

/* Numbers of the AdamW step over the layer norms' parameters and, with the AdamW methods, the weight matrices: its
 * learning rate is `rate` times the step's, weight_decay is of the matrices (bias column included) only.  Defaults: rate 1,
 * beta1 0.9, beta2 0.999, epsilon 1e-8 (not 0), weight_decay 0.  Forgets the moments and synchronises the device.
 * A step captured before keeps the numbers of its capture.  NGSGD_EINVAL for a network without AdamW; so does ngsgd_step where
 * rate * lr is above 1e18 or not a number. */
int ngsgd_set_adamw(ngsgd_net* net, float rate, double beta1, double beta2, float epsilon, float weight_decay);

/* Borrowed handle of a layer's preconditioner (side = NGSGD_SIDE_INPUT / NGSGD_SIDE_OUTPUT);
 * owned by the net, valid until ngsgd_destroy.  NULL result when that side's rank is 0. */
int ngsgd_net_precond(ngsgd_net* net, int32_t layer, int32_t side, ngsgd_precond** out);

/* Inspection of the latest step, for parity checks.  All outputs are dense row-major copies.
 *   ngsgd_last_preconditioned: the N x dim matrix Obar_l or Xbar_l (already rescaled by gamma)
 *   ngsgd_last_gradient:       a_l * Obar_l^T Xbar_l, dims[layer+1] x (in_dim+1), without lr
 *   ngsgd_last_max_change_scale: a_l of App. C.3 as one double (1 when the limit is disabled)
 *   ngsgd_last_norm_gradient:  of the layer norm behind hidden layer `layer`, by its weight and its bias */
int ngsgd_last_preconditioned(ngsgd_net* net, int32_t layer, int32_t side, float* dev_out,
                              void* hip_stream);
int ngsgd_last_gradient(ngsgd_net* net, int32_t layer, float* dev_out, void* hip_stream);
int ngsgd_last_max_change_scale(ngsgd_net* net, int32_t layer, double* dev_out, void* hip_stream);
int ngsgd_last_norm_gradient(ngsgd_net* net, int32_t layer, float* dev_dweight, float* dev_dbias, void* hip_stream);

/* ---- timing of kernel groups (for benchmarks) ------------------------------------------------
 * While enabled, every launch group of the categories below is bracketed by a pair of HIP events
 * recorded on the launch stream.  ngsgd_profile_read waits for the recorded events, adds the elapsed
 * milliseconds and the number of bracketed groups per category into ms_out / launches_out (arrays of
 * n_categories >= NGSGD_PROF_CATEGORIES entries, host memory) and clears the record.  Process-wide,
 * not thread-safe; at most 32768 groups are kept between reads (one whose work another group's kernel does is
 * not counted, but takes a place): if more were launched the call still
 * fills the arrays with what was kept and returns NGSGD_ENOMEM.
 * An updating ngsgd_precondition forms Xhat and finishes its output beside the R x R update and, up to rank 32,
 * the new factor: both are then in the time of those groups, and PRECOND_XHAT stays empty (large matrices aside).
 * So is B_t, and the check's W W^T, in that of W_{t+1}. */
#define NGSGD_PROF_GEMM_FWD 0        /* A_l = [X_l, 1] W_l^T, tanh                               */
#define NGSGD_PROF_GEMM_BWD 1        /* dX_l = O_l W_l, mostly with the derivative of tanh       */
#define NGSGD_PROF_GEMM_UPD 2        /* W_l += lr a_l Obar_l^T Xbar_l, max-change (one launch); AdamW */
#define NGSGD_PROF_PRECOND_H 3       /* H = X W^T and tr(X X^T)                                  */
#define NGSGD_PROF_PRECOND_J 4       /* J = H^T X                                                */
#define NGSGD_PROF_PRECOND_XHAT 5    /* Xhat = X - H W and row norms                             */
#define NGSGD_PROF_PRECOND_KL 6      /* K = J J^T, L = H^T H                                     */
#define NGSGD_PROF_PRECOND_SMALL 7   /* R x R update: Z_t, eigen-decomposition, A_t              */
#define NGSGD_PROF_PRECOND_WNEW 8    /* B_t, W_{t+1} = A_t B_t                                   */
#define NGSGD_PROF_ELEMENTWISE 9     /* nonlinearities behind no product, layer norms, log-softmax */
#define NGSGD_PROF_PRECOND_MISC 10   /* clears, gamma, orthogonality check, rescale              */
#define NGSGD_PROF_INIT 11           /* state initialisation from the first minibatch            */
#define NGSGD_PROF_SIMPLE_GRAM 12    /* simple method: X^T X or X X^T                            */
#define NGSGD_PROF_SIMPLE_INVERSE 13 /* simple method: (beta I + Gram / (N-1))^{-1}              */
#define NGSGD_PROF_SIMPLE_APPLY 14   /* simple method: Q, per-row factors, gamma                 */
#define NGSGD_PROF_PRECOND_FUSED 15  /* H, Xhat and row norms in one pass (calls without factor update) */
#define NGSGD_PROF_CATEGORIES 16
int ngsgd_profile_enable(int32_t on);
int ngsgd_profile_read(double* ms_out, int64_t* launches_out, int32_t n_categories);

/* ---- diagnostics -------------------------------------------------------------------------- */
const char* ngsgd_strerror(int code);
/* The fused apply kernel (Xhat = X - (X W^T) W in one pass, used by calls that do not update their
 * factor) lets the workgroups that share a block of rows wait for each other's part of X W^T.  The wait
 * is bounded: after this many microseconds (default 2000) a workgroup stops waiting and leaves its part
 * of the matrix to the (slow) completion step of the following kernel, so the kernel ends whatever else
 * occupies the GPU.  0 makes every workgroup take that route at once unless its partners have already
 * finished (used by the tests of that route).  The workgroups that share a matrix of 161 to 1024 rows while a
 * first factor is built wait for each other to be running: twice as long up to 512 rows, six times above.  Then they
 * leave, and the following kernel reduces that matrix from memory (a call with a first factor of 512 rows takes
 * 3.3 ms instead of 1.9, of 1024 rows 11.0 instead of 5.2).  0 sends every such matrix there.  Process-wide. */
int ngsgd_set_wait_limit_us(int64_t microseconds);
/* hipError_t value of the most recent failed HIP call on this thread (0 if none). */
int ngsgd_last_hip_error(void);
/* Library version: major * 10000 + minor * 100 + patch. */
int ngsgd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* NGSGD_H_ */
