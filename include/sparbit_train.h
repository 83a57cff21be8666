/*
 * sparbit_train.h - operators of a training step whose state is divided over the ranks of a
 * communicator, next to the allgather of sparbit.h that such a step has in its middle.
 *
 *   scan     a gated linear recurrence over long sequences, forward, backward and for single
 *            tokens.  A sequence divided by time over P ranks: each rank's slice maps a state h to
 *            decay * h + last; the block {decay, last} is what the ranks gather, and
 *            sparbit_scan_join folds the gathered blocks into each rank's first state.
 *   router   the choice of k experts a token with its weights, the per-expert counts, the balance
 *            loss and the gradient of all of them.  The counts are what the ranks gather: the
 *            balance term compares a rank's probabilities with the counts of ALL ranks (and the
 *            gathered counts are the block sizes of a following sparbit_plan_create_v).
 *   ortho    a matrix update orthogonalised by Newton-Schulz products, alone or with the momentum
 *            in front of it and the weight update behind it.  The ranks gather the rows of the
 *            matrix: a receive buffer of sparbit_allgather IS the matrix, row blocks in rank order.
 *
 * Conventions are those of sparbit.h: error codes, sparbit_strerror, sparbit_last_cuda_error;
 * plans are made on the host without a CUDA call; calls are asynchronous on `stream` (a
 * cudaStream_t as void*, NULL = the legacy default stream) and find every argument error on the
 * host before anything is launched; no call allocates device memory; a plan may be used by one
 * host thread and on one stream at a time and belongs to the device that was current when it got
 * its workspace.  All pointers without "host" in their comment are device pointers owned by the
 * caller.  All calls may be captured into a CUDA graph and replayed (scalars keep the captured
 * values).  Results do not change from run to run: no sum depends on the order in which CTAs run.
 *
 * Matrices are row-major with a row stride ("ld") in ELEMENTS, at least the row's width and at most
 * 2^46 divided by the number of rows (ERR_ARG).  Any
 * alignment that suits the element type gives the right answer; where pointers and strides are
 * multiples of 16 bytes the wide kernels run.  Outputs must overlap neither inputs nor each other
 * (ERR_ALIAS); row-interleaved halves of one buffer do not overlap.
 */
#ifndef SPARBIT_TRAIN_H
#define SPARBIT_TRAIN_H

#include "sparbit.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
enum { SPARBIT_F32 = 0, SPARBIT_BF16 = 1, SPARBIT_F16 = 2 };

/* ---- gated linear recurrence -----------------------------------------------------------------
 *
 *   a_t = 1 / (1 + exp(-gate_t)),   h_t = a_t h_{t-1} + (1 - a_t) x_t,   y_t = h_t
 *
 * independently for every channel; 1 - a_t is formed without cancellation and states are held in
 * 32 bits throughout.  With c_t the gradient that reaches step t from the steps after it,
 *
 *   g_t = dy_t + c_t,  c_{t-1} = a_t g_t,  dx_t = (1 - a_t) g_t,
 *   dgate_t = g_t (h_{t-1} - x_t) a_t (1 - a_t),  dh0 = c_0
 *
 * A NaN, or an infinite x, dy or first state, makes its channel NaN or infinite from there to the end
 * (beginning) of its sequence, and nothing else.
 *
 * A plan covers n sequences of given lengths (0 and 1 allowed) whose rows follow one another in
 * every matrix: sequence s has the lengths[s] rows from off[s] = the sum of the lengths before it.
 */
typedef struct sparbit_scan_plan_s sparbit_scan_plan_t;

/*
 * lengths: host array of n_seqs counts, copied.  Errors: ERR_ARG (null, n_seqs < 1, channels < 1,
 * unknown type), ERR_OVERFLOW (rows x channels beyond 2^46), ERR_LIMIT (more than 2^20 channels,
 * 65535 sequences or 2^30 pieces of up to 128 rows and 32 channels), ERR_NOMEM.  Host-only.
 */
int sparbit_scan_plan_create(int n_seqs, const size_t* lengths, size_t channels, int dtype,
                             sparbit_scan_plan_t** out);
int sparbit_scan_plan_destroy(sparbit_scan_plan_t* plan); /* NULL allowed; frees host memory only */

/* Bytes of device workspace the plan needs (16-byte aligned), and of the `carry` that the forward
 * pass leaves for the backward pass: the 32-bit state at every 128th step of each sequence. */
size_t sparbit_scan_plan_workspace_bytes(const sparbit_scan_plan_t* plan);
size_t sparbit_scan_plan_carry_bytes(const sparbit_scan_plan_t* plan);

/* Gives the plan its workspace, on the current device, and fills it with the plan's tables
 * (SYNCHRONISES).  The caller keeps it alive and unchanged while the plan is used.
 * ERR_WORKSPACE: null, misaligned or too small. */
int sparbit_scan_plan_set_workspace(sparbit_scan_plan_t* plan, void* dev, size_t bytes);

/*
 *   gate, x    [rows][channels] of the plan's type
 *   h0         [n_seqs][channels] 32-bit, row stride h0_ld; NULL = zero
 *   y          [rows][channels] of the plan's type; NULL = only the summary is wanted
 *   summary    [n_seqs][2][channels] 32-bit or NULL: the product of the sequence's a_t, and its
 *              last state (h0 for a sequence of no rows)
 *   carry      carry_bytes, 32-bit, or NULL: for sparbit_scan_backward
 * Errors: ERR_ARG, ERR_WORKSPACE (set no workspace yet), ERR_ALIAS, ERR_CUDA.
 */
int sparbit_scan_forward(sparbit_scan_plan_t* plan, const void* gate, size_t gate_ld, const void* x, size_t x_ld,
                         const float* h0, size_t h0_ld, void* y, size_t y_ld, float* summary, float* carry,
                         void* stream);

/*
 *   carry      what sparbit_scan_forward left for the same gate, x and h0
 *   dy         [rows][channels];  dlast [n_seqs][channels] 32-bit, row stride dlast_ld: gradient
 *              of the last states; NULL = zero
 *   dgate, dx  [rows][channels] of the plan's type
 *   dsummary   [n_seqs][2][channels] 32-bit or NULL: the product of the a_t, and dh0
 * With dgate and dx NULL (both or neither) only dsummary is computed; x and carry are then not
 * read and may be NULL.  Errors as above.
 */
int sparbit_scan_backward(sparbit_scan_plan_t* plan, const void* gate, size_t gate_ld, const void* x, size_t x_ld,
                          const float* carry, const void* dy, size_t dy_ld, const float* dlast, size_t dlast_ld,
                          void* dgate, size_t dgate_ld, void* dx, size_t dx_ld, float* dsummary, void* stream);

/* Synchronises the device; SPARBIT_OK, or SPARBIT_ERR_TIMEOUT if a wait inside a kernel of the plan
 * (for the state that an earlier piece of a sequence leaves) gave up since the last call; results of
 * that launch are then incomplete. */
int sparbit_scan_plan_status(sparbit_scan_plan_t* plan);

/* Test hook for that bounded wait: with `withhold` set, later launches never publish the states that
 * sequences of more than 2048 steps wait for, and give up after timeout_ns (0 = the default 2 s). */
int sparbit_scan_plan_set_wait_test(sparbit_scan_plan_t* plan, int withhold, uint64_t timeout_ns);

/*
 * One token for each of `rows` running sequences (serving).  Row i uses row slots[i] of the table
 * of states [n_slots][channels] (32-bit, row stride state_ld); slots NULL = row i itself, then
 * n_slots >= rows.  A slot outside 0 .. n_slots-1 marks a row without a sequence: no state is
 * touched and its y is 0.  Named slots must differ from one another.  state_out may be state_in;
 * where it is another table, only the named rows are written.  No plan, no workspace.
 */
int sparbit_scan_step(size_t rows, size_t channels, int dtype, const void* gate, size_t gate_ld, const void* x,
                      size_t x_ld, const int32_t* slots, size_t n_slots, const float* state_in, float* state_out,
                      size_t state_ld, void* y, size_t y_ld, void* stream);

/*
 * The first states of slices that follow one another in time, from the gathered summaries
 * (ERR_OVERFLOW where those pass 2^46 elements).  For
 * i in 0 .. n_ranks-1, rank r = first_rank + i:
 *   gathered   [n_ranks][P][2][channels]: what the allgather of [2][channels] blocks left in rank
 *              r's receive buffer (n_ranks = P, first_rank = 0: all virtual ranks of one GPU;
 *              n_ranks = 1: a process that is one rank)
 *   h0         [channels] or NULL = zero: the state before slice 0 (reverse: the gradient that
 *              enters after slice P-1)
 *   out        [n_ranks][channels], row stride out_ld: h0 carried through slices 0 .. r-1
 *              (reverse != 0: through slices P-1 down to r+1, for gathered dsummary blocks)
 */
int sparbit_scan_join(int P, int first_rank, int n_ranks, size_t channels, const float* gathered, const float* h0,
                      float* out, size_t out_ld, int reverse, void* stream);

/* ---- router: k experts a token, counts, balance loss ------------------------------------------
 *
 * For the logits l of a token: p = softmax(l); the k largest logits are chosen (of equal ones the
 * lowest index first); weights are the p of the chosen experts, divided by their sum where
 * `renormalize` is set.  A token whose mask byte is 0, or whose logits are all -inf, is left out:
 * indices -1, weights and lse 0, gradient 0, and whatever its logits hold (NaN included) reaches
 * nothing.  An expert whose logit is -inf or NaN is not chosen; where fewer than k are left the
 * places hold index -1 and weight 0.  Finite logits of any size are logits: a token all of whose
 * experts hold the type's lowest value takes part, with p = 1 / experts (and an lse^2 that 32 bits
 * may hold as inf only).  NaN or +inf in a token that takes part makes its weights, lse and gradient
 * NaN, and the sums of its rank; +inf can be chosen.
 *
 * With N the number of tokens that take part over all ranks and f_e = (tokens sent to e) / (N k):
 *   loss of rank r = alpha E sum_e f_e (sum of r's p_e) / N  +  beta (sum of r's lse^2) / N
 * whose sum over the ranks is the balance loss of the whole batch; f is a constant for gradients.
 */
typedef struct sparbit_router_plan_s sparbit_router_plan_t;

#define SPARBIT_ROUTER_MAX_EXPERTS 1024
#define SPARBIT_ROUTER_MAX_K 32

/*
 * tokens: host array of n_ranks counts, copied; the ranks' rows follow one another.  Errors:
 * ERR_ARG (null, n_ranks < 1, k < 1 or > experts, unknown type), ERR_LIMIT (experts or k beyond
 * the limits above, more than 65535 ranks or 2^31-1 rows), ERR_NOMEM.  Host-only.
 */
int sparbit_router_plan_create(int n_ranks, const size_t* tokens, int experts, int k, int dtype, int renormalize,
                               sparbit_router_plan_t** out);
int sparbit_router_plan_destroy(sparbit_router_plan_t* plan);
size_t sparbit_router_plan_workspace_bytes(const sparbit_router_plan_t* plan);
int sparbit_router_plan_set_workspace(sparbit_router_plan_t* plan, void* dev, size_t bytes);

/*
 *   logits   [rows][experts] of the plan's type       mask     [rows] bytes or NULL = all take part
 *   indices  [rows][k] int32                          weights  [rows][k] 32-bit
 *   lse      [rows] 32-bit: log of the sum of exp(l)
 *   counts   [n_ranks][experts + 1] int32: tokens sent to each expert, then tokens that take part
 *            (the block to gather: (experts + 1) * 4 bytes a rank)
 *   sums     [n_ranks][experts + 1] 32-bit: sum of each p_e, then sum of lse^2
 */
int sparbit_router_forward(sparbit_router_plan_t* plan, const void* logits, size_t ld, const uint8_t* mask,
                           int32_t* indices, float* weights, float* lse, int32_t* counts, float* sums,
                           void* stream);

/* gathered: [n_ranks][G][experts + 1] int32, rank r's receive buffer of the allgather of the counts
 * over a communicator of G ranks (1 <= G).  loss: [n_ranks] 32-bit. */
int sparbit_router_balance(sparbit_router_plan_t* plan, const int32_t* gathered, int G, const float* sums,
                           float alpha, float beta, float* loss, void* stream);

/*
 * Gradient of the logits: of sum(dweights * weights) (dweights [rows][k] 32-bit, NULL = zero) plus
 * dloss (one 32-bit value on the device, NULL = 1) times the balance loss.  indices, weights and
 * lse are the forward pass's.  dlogits: [rows][experts] of the plan's type.
 */
int sparbit_router_backward(sparbit_router_plan_t* plan, const void* logits, size_t ld, const uint8_t* mask,
                            const int32_t* indices, const float* weights, const float* lse,
                            const int32_t* gathered, int G, const float* dweights, float alpha, float beta,
                            const float* dloss, void* dlogits, size_t dlogits_ld, void* stream);

/* ---- orthogonalised update ---------------------------------------------------------------------
 *
 * X = U / (|U| + eps) in the Frobenius norm, then for every step with its coefficients (a, b, c)
 *   A = X X^T,  X = a X + (b A + c A A) X
 * (X^T X for a tall matrix): the singular vectors of U with every singular value driven towards
 * one.  A matrix that holds a NaN or an infinity gives NaN throughout; a zero matrix gives zeros.
 */
typedef struct sparbit_ortho_plan_s sparbit_ortho_plan_t;

/* Products of 16-bit operands that make up one product of the iteration.  ONE: error 0.3e-3 (4096 x
 * 8192, decaying singular values) to 1.9e-3 (64 x 64, random) of the result's norm; rounding to a
 * bf16 result makes 1.7e-3 beside it.  THREE, three times the work: where the result has 32 bits
 * 1e-6, of matrices of low rank 3e-6 to 7e-6 (plain 32-bit arithmetic: 1.4e-5).  AUTO: ONE for
 * SPARBIT_BF16 matrices with no side below 128; THREE for smaller ones, which ONE would leave more
 * than half as far off again as rounding does, and for the types with more bits.  The weights of a
 * Muon step do not enter: bf16 gradients of 32-bit weights have to ask for THREE where they want it. */
enum { SPARBIT_PRODUCTS_AUTO = 0, SPARBIT_PRODUCTS_ONE = 1, SPARBIT_PRODUCTS_THREE = 3 };

/*
 * A plan for `count` matrices of rows x cols, element type dtype.  coefficients: host array
 * [steps][3], copied; NULL = (3.4445, -4.7750, 2.0315) in every step (five steps are usual).
 * Errors: ERR_ARG (count, rows, cols or steps < 1, unknown type, eps negative or not finite, and
 * coefficients that what the steps hold has no room for: singular values that start in 0 .. 1 may
 * have magnitudes up to 6.9 where a step begins and 64 (less 2 %) after the last, and b s^2 + c s^4
 * up to 48, with and without -3/4 (b + c)), ERR_LIMIT (rows or cols > 65536, count > 4096, steps > 64, 2^31 tiles of work),
 * ERR_NOMEM.  Host-only.
 */
int sparbit_ortho_plan_create(int count, size_t rows, size_t cols, int dtype, int steps, const float* coefficients,
                              float eps, sparbit_ortho_plan_t** out);
int sparbit_ortho_plan_destroy(sparbit_ortho_plan_t* plan);
/* Before sparbit_ortho_plan_workspace_bytes: the plan forgets a workspace it had. */
int sparbit_ortho_plan_set_products(sparbit_ortho_plan_t* plan, int products);
size_t sparbit_ortho_plan_workspace_bytes(const sparbit_ortho_plan_t* plan);
int sparbit_ortho_plan_set_workspace(sparbit_ortho_plan_t* plan, void* dev, size_t bytes);

/* Synchronises the device; SPARBIT_OK, or SPARBIT_ERR_TIMEOUT if a wait inside a kernel of the plan
 * gave up since the last call (its results are then incomplete). */
int sparbit_ortho_plan_status(sparbit_ortho_plan_t* plan);

/* Test hook for those waits: with `withhold` set, later launches never announce a finished product to the
 * warps that write it out, and give up after timeout_ns (0 = the default 2 s) in each of their 3 kernels a step. */
int sparbit_ortho_plan_set_wait_test(sparbit_ortho_plan_t* plan, int withhold, uint64_t timeout_ns);

/* update and out: matrix i starts i * stride elements behind the first (stride is ignored for
 * count 1): one behind another, stride >= (rows - 1) * ld + cols, or side by side in the rows of one
 * buffer, stride >= cols and (count - 1) * stride + cols <= ld; ERR_ARG otherwise. */
int sparbit_orthogonalize(sparbit_ortho_plan_t* plan, const void* update, size_t ld, size_t stride, void* out,
                          size_t out_ld, size_t out_stride, void* stream);

/*
 * The update of the Muon optimiser, with X the orthogonalised U:
 *   M' = momentum * M + G;   U = nesterov ? G + momentum * M' : M'
 *   W' = (1 - lr * weight_decay) W - lr * scale * X
 * grad has the plan's type, the momentum is 32-bit, the weights have weight_dtype.  The outputs may
 * be the inputs (updated in place); other overlaps are ERR_ALIAS.  ld, stride: in and out alike.
 */
typedef struct {
    const void* grad;
    size_t grad_ld, grad_stride;
    const float* momentum_in;
    float* momentum_out;
    size_t momentum_ld, momentum_stride;
    const void* weight_in;
    void* weight_out;
    size_t weight_ld, weight_stride;
    int weight_dtype;
    int nesterov;
    float lr, momentum, weight_decay, scale;
} sparbit_muon;
int sparbit_muon_step(sparbit_ortho_plan_t* plan, const sparbit_muon* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPARBIT_TRAIN_H */
