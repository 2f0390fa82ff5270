/*
 * microadam.h -- C ABI of libmicroadam.so, a MicroAdam optimizer step for
 * AMD Instinct MI355X (gfx950).
 *
 * MicroAdam ("MicroAdam: Accurate Adaptive Optimization with Low Space
 * Overhead and Provable Convergence", Modoranu et al., 2024) keeps, per
 * parameter tensor:
 *   - a 4-bit error-feedback (EF) buffer e with per-bucket min/max metadata
 *     (delta, Delta) (Algorithm 1, the quantized EF; Section 3.1,
 *     "Quantization metadata");
 *   - a sliding window G = (I, V) of the last m sparse gradients, m rows of
 *     k block-relative uint16 indices and bf16 values (Section 3, notation;
 *     Section 3.1, "Top-K"; Section 3.2 for the 4-bytes-per-entry budget).
 * One step (Algorithm 1) decodes e and adds it to the gradient, keeps the
 * block-wise Top-K of |a| in a new window row, re-quantizes the residual
 * into e, rebuilds the Adam moments from the window (AdamStats, Algorithm 2)
 * and updates the parameters, with decoupled weight decay (Algorithm 4).
 *
 * Conventions for every call:
 *   - Return value: MICROADAM_OK (0) or a negative MICROADAM_ERR_* code.
 *     Arguments are validated before any device work is queued, so a call
 *     that fails leaves parameters and optimizer state untouched.
 *     microadam_error_string() names a code; microadam_last_error() gives the
 *     calling thread's most recent failure message in detail.
 *   - Device pointers are HIP device addresses owned by the caller.  Host
 *     pointers are plain host memory owned by the caller and only read
 *     during the call.
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     Device work is queued on it and the call returns without waiting.
 *   - A handle must be used by one host thread at a time.
 *   - No C++ exception crosses this interface.
 */
#ifndef MICROADAM_H
#define MICROADAM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  MICROADAM_OK = 0,
  MICROADAM_ERR_INVALID_ARG = -1, /* null pointer, value out of range, misaligned buffer */
  MICROADAM_ERR_UNSUPPORTED = -2, /* a valid but unimplemented configuration */
  MICROADAM_ERR_SHAPE = -3,       /* tensor count or sizes differ from microadam_init */
  MICROADAM_ERR_STATE_SIZE = -4,  /* state buffer smaller than microadam_state_bytes */
  MICROADAM_ERR_HIP = -5,         /* a HIP runtime call failed (see microadam_last_error) */
  MICROADAM_ERR_NO_MEMORY = -6    /* host or library-internal allocation failed */
};

/* Element types of parameters and gradients. */
enum { MICROADAM_F32 = 0, MICROADAM_BF16 = 1 };

/*
 * Hyper-parameters, in the paper's notation (Section 3, notation; Appendix B
 * gives the values the paper trains with: density 0.01, m = 10, b = 4,
 * bucket 64, beta1 0.9, beta2 0.999, eps 1e-8).
 *
 *   density      k/d in (0, 1].  A Top-K block of s elements keeps
 *                k_s = min(s, max(1, ceil(density * s - 1e-9))) entries.
 *   beta1,beta2  moment decay rates in [0, 1).
 *   eps          added to sqrt(v-hat) in the update (Algorithm 1); > 0 (an
 *                element without window entries then takes a zero step).
 *   lr           default step size eta (microadam_step may override it).
 *   weight_decay lambda of the decoupled decay theta *= (1 - eta*lambda)
 *                (Algorithm 4); >= 0.
 *   window       m, rows in the sliding window, 1..64.
 *   ef_bits      b, bits per EF code: 4 (the paper's choice, Section 3.1) or
 *                8 (a wider code for the same buckets).
 *   ef_rounding  how Q rounds: MICROADAM_ROUND_NEAREST (Algorithm 2, half to
 *                even) or MICROADAM_ROUND_RANDOMIZED (Lemma 1: floor((x -
 *                delta)/u + xi), xi ~ U[0, 1), which makes Q unbiased).
 *   seed         key of the randomized rounding's random stream: element i
 *                of tensor j at step t draws xi = (w >> 8) * 2^-24 from word
 *                i mod 4 of Philox4x32-10 (Salmon et al., SC 2011) at counter
 *                (i/4 low word, i/4 high word, j, t) under the key (seed low
 *                word, seed high word); j is the tensor's position in the
 *                numels list of microadam_init.  The floor is taken of the
 *                exact sum.  Unused with NEAREST.
 *   ef_bucket    B_q, elements sharing one (delta, Delta) pair: a power of
 *                two in [8, 512] dividing topk_block (buckets inside blocks),
 *                or any size >= topk_block (buckets of each tensor's
 *                elements [c*B_q, (c+1)*B_q), spanning blocks; Section 3.1
 *                names 100K), which runs the quantization as a second pass
 *                over the block.
 *   topk_block   B_d, Top-K block size; at most
 *                65536 (block-relative indices are uint16).  This build
 *                implements multiples of 16 and returns
 *                MICROADAM_ERR_UNSUPPORTED for other valid sizes.
 *   window_value_dtype  MICROADAM_BF16 (the paper's choice, Section 3.2) or
 *                MICROADAM_F32 (lossless window values, for checking the
 *                moment rebuild).
 *   fused        0: every step runs a select kernel (EF decode, block Top-K,
 *                new row, re-quantization) and then an update kernel (moment
 *                rebuild, parameter update), the faster form on MI355X; 1:
 *                where the configuration allows (see microadam_step_kernels),
 *                all of a step in one fused kernel, one workgroup per block.
 *                Both give the same results.
 *   reserved     0.
 */
/* Rounding of the error-feedback quantizer. */
enum { MICROADAM_ROUND_NEAREST = 0, MICROADAM_ROUND_RANDOMIZED = 1 };

typedef struct microadam_config {
  double density;
  double beta1;
  double beta2;
  double eps;
  double lr;
  double weight_decay;
  int32_t window;
  int32_t ef_bits;
  int32_t ef_bucket;
  int32_t topk_block;
  int32_t window_value_dtype;
  int32_t ef_rounding;
  uint64_t seed;
  int32_t fused;
  int32_t reserved;
} microadam_config;

typedef struct microadam_handle_s* microadam_handle;

/*
 * Where one tensor's optimizer state lives inside the state buffer (byte
 * offsets from its start).  The buffer holds three planes, EF codes, bucket
 * stats and window, each starting 256-byte aligned.  In each plane every
 * Top-K block owns a record of fixed size, at plane + g * stride for its
 * global block number g.  Full blocks (B_d elements) are numbered first,
 * tensor by tensor, then the ragged last blocks of the tensors whose numel is
 * not a multiple of B_d; a ragged block's record is padded to full size.
 * Block q of a tensor has global number first_block + q, except its last
 * block (q = num_blocks - 1), whose number is last_block.
 *
 *   EF codes   B_d/2 bytes per block: element 2j of the block in the low
 *              nibble of byte j, element 2j+1 in the high nibble (nibbles
 *              past the block's elements are 0).  With ef_bits = 8, B_d
 *              bytes per block, element i in byte i.
 *   stats      B_d/B_q pairs of float32 (delta, Delta) per block = (min,
 *              max) of the bucket's residual; pair b covers the block's
 *              elements [b*B_q, (b+1)*B_q); pairs past its elements are
 *              unused.  With buckets spanning blocks (ef_bucket >= B_d and
 *              not a power of two in [8, 512] dividing B_d) the buckets are
 *              the tensor's elements [c*B_q, (c+1)*B_q), and their pairs
 *              live in two tables of bucket_table_bytes: the pair of bucket
 *              c written at step t is at stats_plane + (t mod 2) *
 *              bucket_table_bytes + 8*c (stats_stride is 0).  A plane of 16
 *              bytes per block of partial (min, max) pairs follows them.
 *   window     m*k_full*entry_bytes per block, rounded up to a multiple
 *              of 128 bytes (the stride): row r (the row written at
 *              step s is r = (s-1) mod m) starts at r*k_q*entry_bytes within
 *              the record and holds the block's k_q entries in ascending
 *              index order (k_q = k_last for the last block).  With bf16
 *              values an entry is one little-endian uint32 (index |
 *              bf16_bits << 16); with float32 values it is a uint32 index
 *              followed by the float32 value.  For B_d > 4096 the record
 *              continues, after the m rows (at byte m*k_full*entry_bytes),
 *              with a table of m*ceil(B_d/1024) uint32: entry (r, j) is the
 *              position in row r of the first entry whose index is at least
 *              1024*j (the entries of the block's 1024-element quarter j
 *              are the positions [entry (r, j), entry (r, j+1)), the last
 *              ending at k_q).
 */
typedef struct microadam_layout {
  int64_t numel;
  int64_t num_blocks;
  int64_t num_buckets;
  int32_t k_full;      /* entries per row of a full block */
  int32_t k_last;      /* entries per row of the last block */
  int32_t entry_bytes; /* 4 (bf16 values) or 8 (float32 values) */
  int32_t reserved;
  int64_t first_block; /* global number of block 0 */
  int64_t last_block;  /* global number of block num_blocks - 1 */
  uint64_t ef_plane, ef_stride;
  uint64_t stats_plane, stats_stride;
  uint64_t window_plane, window_stride;
  uint64_t bucket_table_bytes; /* buckets spanning blocks: see stats above; else 0 */
} microadam_layout;

/*
 * Size in bytes of the device state buffer for tensors of the given element
 * counts (numels[0..n_tensors), each >= 1).  Pure host computation: per
 * Top-K block B_d/2 bytes of EF codes, 8*B_d/B_q bytes of bucket stats and
 * m*k_full*entry_bytes of window rounded up to 128 bytes, each plane
 * 256-byte aligned.  This is the
 * paper's 0.5d + 4mk (Section 3.2) plus the (delta, Delta) metadata of
 * Section 3.1, per-block rounding of k and the padding of each tensor's last
 * block.
 */
int microadam_state_bytes(const microadam_config* cfg, const int64_t* numels,
                          int32_t n_tensors, uint64_t* out_bytes);

/*
 * Creates a handle for the tensor list numels[0..n_tensors) and clears the
 * caller-owned device buffer `state` (>= microadam_state_bytes bytes, 256-byte
 * aligned) on `stream`: e = 0, delta = Delta = 0 as in the initialisation of
 * Algorithm 1.  The step counter starts at 0 (the next step is t = 1).
 * param_dtype / grad_dtype: MICROADAM_F32 or MICROADAM_BF16.
 * The library keeps small device tables of its own (freed by destroy:
 * the block -> tensor table, the window weights, and with Top-K blocks above
 * 4096 elements that are multiples of 4096 a 128-byte record per block
 * and a list of the blocks the threshold pass could not settle, 4 bytes per
 * block);
 * `state` stays owned by the caller and must outlive the handle.
 */
int microadam_init(const microadam_config* cfg, const int64_t* numels,
                   int32_t n_tensors, int32_t param_dtype, int32_t grad_dtype,
                   void* state, uint64_t state_bytes, void* stream,
                   microadam_handle* out);

/*
 * One MicroAdam step (Algorithm 1 with the decay of Algorithm 4) over all
 * tensors, queued on `stream` (microadam_step_kernels launches).  params[j] (updated in place)
 * and grads[j] (read only) are device pointers to numels[j] contiguous
 * elements of the init dtypes, 16-byte aligned.  lr: the step size eta for
 * this step, or NaN to use cfg.lr.  The step counter t advances by one.
 * Non-finite gradients (NaN, +-inf), which the method leaves undefined, give
 * unspecified parameters and state in the Top-K blocks that hold them (in
 * their buckets, when buckets span blocks); every other block is computed as
 * if they were absent, and no memory outside params, grads and the state is
 * touched.
 */
int microadam_step(microadam_handle h, void* const* params,
                   const void* const* grads, int32_t n_tensors, double lr,
                   void* stream);

/* Frees the handle and the library's device table (waits for nothing;
 * the caller must not destroy a handle whose step may still be running on
 * a stream it will not synchronize).  NULL is accepted. */
int microadam_destroy(microadam_handle h);

/* Steps taken so far (the t of the last step), or a negative error code. */
int64_t microadam_get_step(microadam_handle h);

/* Sets the step counter, e.g. after restoring a saved state buffer: the next
 * step is t + 1.  t >= 0. */
int microadam_set_step(microadam_handle h, int64_t t);

/* Layout of tensor `tensor`'s state (see microadam_layout). */
int microadam_tensor_layout(microadam_handle h, int32_t tensor,
                            microadam_layout* out);

/*
 * Test support: recomputes the dense float32 m-hat and v-hat of tensor
 * `tensor` from the window as it stands after the last step (AdamStats,
 * Algorithm 2, at the current t >= 1), into device buffers of numel floats.
 */
int microadam_debug_moments(microadam_handle h, int32_t tensor, float* mhat,
                            float* vhat, void* stream);

/*
 * Kernel launches per microadam_step (fixed at init), or a negative error
 * code: 1 where the step runs as one fused kernel (cfg.fused = 1, Top-K
 * blocks of 2049 to 4096 elements, at most 128 entries per row, m *
 * ceil(k/64) <= 16, parameters and gradients of one dtype, buckets inside
 * blocks); 2 (select, then update) otherwise; 4 with buckets spanning blocks
 * (select, bucket reduction, quantization, update); 4 with Top-K blocks
 * above 4096 elements that are multiples of 4096 and buckets inside blocks
 * (a threshold pass over each block, the select of its 4096-element
 * sub-blocks, the multi-wave select of the blocks whose threshold the first
 * pass left open, update).
 */
int microadam_step_kernels(microadam_handle h);

/*
 * Profiling.  With profiling on (off after init), every microadam_step
 * records HIP events on its stream around its kernels.  Events are
 * created on the first call that turns profiling on, with the init device
 * current.  Every call that turns it on starts a new total for
 * microadam_kernel_times_total.
 */
int microadam_set_profiling(microadam_handle h, int32_t on);

/*
 * Durations in milliseconds of the kernels of the last step, which must have
 * been taken with profiling on: out_ms[0] = select (EF decode, block Top-K,
 * new window row, EF re-quantisation), out_ms[1] = update (moment rebuild
 * from the window and parameter update); for a fused step (see
 * microadam_step_kernels) out_ms[0] is the fused kernel and out_ms[1] is 0.  Blocks until that step is done.
 * out_ms: 2 host floats.
 */
int microadam_kernel_times(microadam_handle h, float* out_ms);

/*
 * Summed kernel durations of every step profiled since profiling was last
 * switched on (or since the previous call of this function), without
 * synchronizing between steps: out_ms[0] = select, out_ms[1] = update, in
 * milliseconds (summed as microadam_kernel_times reports one step), and
 * *out_steps = the number of steps they cover; the totals then restart at 0.
 * The library keeps each profiled step's events in a ring of four sets and
 * reads a set when it is needed again, four profiled steps later.  Blocks
 * until the steps counted are done.  out_ms: 2 host floats; out_steps: one
 * host int64.  Errors: MICROADAM_ERR_INVALID_ARG for NULL outputs.
 */
int microadam_kernel_times_total(microadam_handle h, float* out_ms, int64_t* out_steps);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): step t
 * (>= 1) of the tensor list numels[0..n_tensors) on a caller-owned state
 * buffer laid out as microadam_init lays it out for the same cfg and numels
 * (>= microadam_state_bytes bytes, 256-byte aligned), holding the state
 * after step t - 1: all zero bytes before step 1, which the caller provides.
 * No handle is used and nothing is allocated: the tensor table and window
 * weights go to a static device array of the library, at most 4096 tensors
 * (393 KB; every GPU the library runs on holds its own copy until the
 * process ends), and the kernels are those of microadam_step, with the same
 * results.  params, grads, lr, stream as for microadam_step; param_dtype and
 * grad_dtype as for microadam_init.  Calls that overlap on one GPU (other
 * streams, other host threads) race on the shared array, and each call
 * overwrites what the last one left there; calls on one stream are ordered.
 * Errors: MICROADAM_ERR_UNSUPPORTED for more than 4096 tensors, else those
 * of microadam_init and microadam_step; nothing is queued on failure.
 */
int microadam_step_noalloc(const microadam_config* cfg, const int64_t* numels, int32_t n_tensors,
                           int32_t param_dtype, int32_t grad_dtype, void* state, uint64_t state_bytes,
                           int64_t t, void* const* params, const void* const* grads, double lr,
                           void* stream);

/*
 * ------------------------------------------------- matrix updates
 *
 * Orthogonalisation of an update by Newton-Schulz products, and the Muon
 * step built on it: the rule for weight matrices that is used beside an
 * Adam-type rule for a model's other parameters.
 *
 * For a rows x cols matrix G, with X0 = G / (||G||_F + eps), transposed when
 * rows > cols, each of `steps` steps takes
 *     A = X X^T,   B = a I + b A + c A A,   X <- B X,
 * which applies the odd polynomial a s + b s^3 + c s^5 to the singular values
 * of X and keeps its singular vectors.  The default coefficients (3.4445,
 * -4.7750, 2.0315) bring singular values above about 1e-2 of ||G||_F to
 * between 0.7 and 1.2 in 5 steps.
 *
 *   coefficients  host array of 3 * steps values, (a, b, c) step by step, or
 *                 NULL for the default.  Coefficients that let a singular
 *                 value grow beyond 7 overflow the intermediates.
 *   eps           added to the norm; > 0 (a zero matrix gives zeros).
 *   steps         1..16.
 *   precision     what the products' operands are held in, with binary32
 *                 accumulation in any case:
 *                 MICROADAM_PRECISION_F16    binary16, scaled by powers of two
 *                   (each rounding 2^-11, an eighth of bfloat16's at the same
 *                   rate of the matrix cores); results are good to 1e-3 to
 *                   3e-3 in the Frobenius norm.
 *                 MICROADAM_PRECISION_SPLIT  a sum of two binary16 numbers
 *                   (22 bits); three products for one; results are good to
 *                   1e-6 to 2e-6.
 *                 MICROADAM_PRECISION_AUTO   SPLIT for binary32 results or
 *                   parameters, else F16.
 */
enum { MICROADAM_PRECISION_AUTO = 0, MICROADAM_PRECISION_F16 = 1, MICROADAM_PRECISION_SPLIT = 2 };

typedef struct microadam_schulz_config {
  const double* coefficients;
  double eps;
  int32_t steps;
  int32_t precision;
} microadam_schulz_config;

/*
 * One matrix: rows of `cols` contiguous elements, *_ld elements apart (at
 * least cols, below 2^31).  Addresses are aligned to the element type; rows
 * that start at multiples of 16 bytes are read and written in vectors.
 *   grad      read only.
 *   momentum  updated in place (microadam_muon_step; else NULL).
 *   out       microadam_orthogonalize: the result, which may lie where grad
 *             does (grad has been read by then); microadam_muon_step: the
 *             parameter, updated in place.
 * At most 2^20 rows and columns and 2^33 elements.
 */
typedef struct microadam_matrix {
  const void* grad;
  void* momentum;
  void* out;
  int64_t rows, cols;
  int64_t grad_ld, momentum_ld, out_ld;
} microadam_matrix;

/*
 * Workspace for a list of matrices (only rows and cols are read): *min_bytes
 * is what the calls below accept, *useful_bytes what lets them take matrices
 * of the list together, at most 2 GiB or one matrix if that is larger.  The
 * list is worked off in batches of as many matrices as the workspace holds
 * (at most 96, of at most 8 shapes); a batch takes 2 + 3 * steps launches, and
 * one more per step where few rows against a long side have their products
 * summed in parts.
 * Either output may be NULL.  out_dtype as for the call it is meant for (the
 * parameters' dtype for microadam_muon_step).
 */
int microadam_matrix_workspace(const microadam_schulz_config* cfg, const microadam_matrix* matrices,
                               int32_t n_matrices, int32_t out_dtype, uint64_t* min_bytes,
                               uint64_t* useful_bytes);

/*
 * out = the orthogonalised grad, matrix by matrix, queued on `stream`.
 * Nothing is allocated on the device and no handle is kept: the workspace
 * (256-byte aligned, of any content) belongs to the caller and is in use
 * until the queued work is done.  The same list in a workspace of the same size
 * gives the same bits (batches of other matrices may be summed in another
 * order).
 * Outputs must not share bytes with each other, nor with any grad but their own
 * (interleaved rows do not): such a list is refused.
 * A matrix that holds NaN or an infinity gives NaN throughout; the others of
 * the list are not touched by it.
 */
int microadam_orthogonalize(const microadam_schulz_config* cfg, const microadam_matrix* matrices,
                            int32_t n_matrices, int32_t grad_dtype, int32_t out_dtype, void* workspace,
                            uint64_t workspace_bytes, void* stream);

/*
 * One Muon step over a list of matrices:
 *     V <- mu V + (1 - mu) G                       (momentum, in place)
 *     U  = mu V + (1 - mu) G with nesterov, else V (V before its rounding)
 *     W <- (1 - lr * weight_decay) W - lr * s * orthogonalised U
 * with s = 0.2 sqrt(max(rows, cols)) for MICROADAM_SCALE_MATCH_RMS (the root
 * mean square of an Adam update, so that Adam's learning rates carry over),
 * sqrt(max(1, rows / cols)) for MICROADAM_SCALE_SPECTRAL and 1 for
 * MICROADAM_SCALE_NONE.  V starts as zeros, which the caller provides.
 * Workspace, order and non-finite values as for microadam_orthogonalize.  A
 * parameter or momentum must not share bytes with anything else of the list,
 * but for a parameter and its own grad: such a list is refused.
 */
enum { MICROADAM_SCALE_MATCH_RMS = 0, MICROADAM_SCALE_SPECTRAL = 1, MICROADAM_SCALE_NONE = 2 };

typedef struct microadam_muon_config {
  microadam_schulz_config schulz;
  double momentum;     /* mu in [0, 1) */
  double weight_decay; /* >= 0 */
  int32_t nesterov;    /* 0 or 1 */
  int32_t scale;
} microadam_muon_config;

int microadam_muon_step(const microadam_muon_config* cfg, const microadam_matrix* matrices,
                        int32_t n_matrices, int32_t grad_dtype, int32_t momentum_dtype,
                        int32_t param_dtype, double lr, void* workspace, uint64_t workspace_bytes,
                        void* stream);

/*
 * ------------------------------------------------- token log probabilities
 *
 * `rows` rows of `vocab` logits x, ld elements apart (at least vocab), and one
 * token per row.  With group_rows > 0 (a divisor of rows) they come in groups
 * of as many, which start group_stride elements apart: the rows [:, :-1] of
 * sequences, say.  With z = x / temperature, lp_v = z_v - log sum exp z and
 * p = exp lp:
 *     logp = lp at the row's token,   entropy = -sum p lp  (0 where p = 0),
 * all sums in binary32 or more, each exponent taken from the row's maximum.  vocab is
 * at most 2^24, rows at most 2^20; addresses are aligned to their element
 * type (rows may start anywhere; 16 bytes at a time are read either way).
 *   - A row whose token is ignore_index is not read: logp and entropy 0,
 *     alternatives 0 and -1, gradient 0.
 *   - Logits of -inf (or so low that their p is 0) are tokens that cannot
 *     occur.  A row with no other: logp -inf, entropy 0, alternatives -inf at
 *     0, 1, .., gradient 0.
 *   - A row with NaN or +inf: logp, entropy and gradient NaN, alternatives NaN
 *     and -1.
 *   - A token outside [0, vocab) that is not ignore_index: logp NaN, gradient
 *     NaN, whatever the row holds (nothing outside the row is read).
 * The same call gives the same bits.  The order of a row's sums, and so their
 * last bits, goes by where the row starts within 16 bytes, by whether the call
 * has more than 128 rows, by top_k, and by which of the two functions it is.
 */
typedef struct microadam_logits {
  const void* data;
  const int64_t* targets; /* rows tokens */
  int64_t rows, vocab, ld;
  int64_t ignore_index;
  double temperature; /* finite, > 0 */
  int32_t dtype;      /* MICROADAM_F32 or MICROADAM_BF16 */
  int32_t reserved;   /* 0 */
  int64_t group_rows;   /* 0: rows at one stride */
  int64_t group_stride;
} microadam_logits;

/*
 * logp[rows], entropy[rows] (either may be NULL) and, with top_k > 0 (at most
 * 64 and vocab), the top_k most probable tokens of each row in order, ties to
 * the lowest index: top_logprobs and top_indices [rows][top_k].
 */
int microadam_token_logprobs(const microadam_logits* logits, int32_t top_k, float* logp,
                             float* entropy, float* top_logprobs, int64_t* top_indices, void* stream);

/*
 * logp and entropy (either may be NULL) and, in the same pass, the gradient of
 *     L = sum over rows of grad_logp * logp + grad_entropy * entropy
 * with respect to the logits: grad[rows][vocab] of the logits' dtype, grad_ld
 * elements from row to row.  grad_entropy may be NULL (zeros).  grad may be
 * the logits themselves when the row strides agree and group_rows is 0; any other overlap of its
 * rows with theirs is refused.
 */
int microadam_token_logprobs_grad(const microadam_logits* logits, const float* grad_logp,
                                  const float* grad_entropy, float* logp, float* entropy, void* grad,
                                  int64_t grad_ld, void* stream);

const char* microadam_error_string(int code);

/* The calling thread's most recent error message ("" if none). */
const char* microadam_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* MICROADAM_H */
