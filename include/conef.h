/*
 * libconef — one step of contractive error feedback (ConEF) on one GPU.
 *
 * C ABI.  Every pointer is either a HOST pointer or a DEVICE pointer and each
 * argument says which.  The library allocates no device memory: the caller
 * owns one device workspace whose size conef_workspace_bytes() reports, the
 * gradients and every output buffer.  All device work is enqueued on the
 * stream the caller passes (a cudaStream_t, typed void* here so that this
 * header needs no CUDA include); no call synchronises the device except
 * conef_last_status() and the copy helpers that say so.
 *
 * Every function returns CONEF_OK (0) or a negative CONEF_ERR_* code.  An
 * argument error is detected on the host before anything is launched and
 * leaves the context unchanged.
 *
 * What one step computes (Algorithm 2 of the paper, lines 5-9), for each of N
 * simulated workers i and each tensor of d = rows*cols elements:
 *     e   = decode(state_i)                       (line 5; e_0 = 0, line 1)
 *     p   = eta * g_i + e                          (line 5)
 *     D_i = Q(p)      -> all-reducible message     (line 6)
 *     r   = p - D_i                                (line 9)
 *     state_i = C(r)                               (line 9)
 * and conef_reduce_messages() forms the sum over workers of the messages
 * (line 7, "aggregate", before the division by N).  Algorithm 1 (EFSGD) is the
 * case C = identity.  Tensors with cols == 1 or compress == 0 pass through:
 * their message is eta*g and they keep no error state.
 */
#ifndef CONEF_H
#define CONEF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct conef_ctx conef_ctx;
typedef void *conef_stream; /* cudaStream_t */

enum {
    CONEF_OK = 0,
    CONEF_ERR_INVALID_ARG = -1,
    CONEF_ERR_BAD_PHASE = -2,           /* calls out of order, or a step index that does not advance */
    CONEF_ERR_WORKSPACE_TOO_SMALL = -3,
    CONEF_ERR_UNSUPPORTED = -4,
    CONEF_ERR_CUDA = -5,                /* a CUDA runtime call failed; see conef_error_string */
    CONEF_ERR_DEVICE_STATUS = -6,       /* a kernel recorded a consistency error (see conef_last_status) */
    CONEF_ERR_TOO_LARGE = -7            /* a size exceeds the fixed scratch of an allocation-free entry point */
};

/* gradient compressor Q (Alg. 2 line 6) */
enum { CONEF_Q_IDENTITY = 0, CONEF_Q_RANDK = 1, CONEF_Q_LOWRANK = 2, CONEF_Q_RANDBLOCK = 3 };
/* error compressor C (Alg. 2 line 9; Sec. 4.2) */
enum { CONEF_C_IDENTITY = 0, CONEF_C_INT8 = 1, CONEF_C_INT4 = 2, CONEF_C_COUNTSKETCH = 3,
       CONEF_C_ROWSKETCH = 4, CONEF_C_STOCHQUANT = 5, CONEF_C_MX4 = 6, CONEF_C_MX4_STOCHASTIC = 7 };
enum { CONEF_SCALE_FP32 = 0, CONEF_SCALE_FP16 = 1 };
/* element types of the matrix operators */
enum { CONEF_F32 = 0, CONEF_BF16 = 1, CONEF_F16 = 2 };
/* elements of 8-bit forms: four exponent bits and three of mantissa (largest value 448), or five and two (57344) */
enum { CONEF_E4M3 = 0, CONEF_E5M2 = 1 };
/* message kinds */
enum { CONEF_MSG_VALUES = 0, CONEF_MSG_P = 1, CONEF_MSG_Q = 2, CONEF_MSG_DENSE1D = 3 };

#define CONEF_MAX_WORKERS 64
#define CONEF_MAX_RANK 8

/* One parameter tensor, viewed as a rows x cols row-major matrix (a conv
 * weight as out x (in*kh*kw)).  rows*cols must be below 2^32. */
typedef struct {
    int64_t rows;
    int64_t cols;
    int32_t compress; /* 0: pass through */
    int32_t reserved;
} conef_tensor;

/* Q.  random-k (Sec. 1; remark after Assumption 4; Sec. 5.3): keep
 * k = max(1, floor(d*k_num/k_den)) coordinates, the same on every worker and
 * new at every step, no d/k rescaling.  random-block-k (Sec. 5.3): the k kept
 * coordinates are one contiguous block whose start is uniform on [0, d-k],
 * drawn from the shared (seed, tensor, step) stream.  low-rank (Sec. 5.2): rank
 * r = min(rank, rows, cols), one power iteration, warm-started. */
typedef struct {
    int32_t kind;
    int32_t rank;        /* low-rank: 1..CONEF_MAX_RANK */
    int64_t k_num, k_den;
    const float *q_init; /* DEVICE, low-rank only: concatenation over the compressed tensors,
                            in table order, of the cols x r row-major warm starts Q_0.
                            Copied during conef_init; the caller may free it afterwards
                            (after the stream has run). */
    uint64_t seed;       /* random-k, random-block-k: the seed shared by all workers */
} conef_q_cfg;

/* C.  int8/int4 (Sec. 4.2.1): symmetric absmax quantisation of blocks of
 * `block` consecutive elements of the row-major flattening (block in
 * {32,64,128,256}; int4 needs block >= 64), round to nearest even, one fp32
 * or fp16 scale per block; int4 packs element 2q in the low nibble of byte q.
 * count sketch (Sec. 4.2.2): cs_rows (odd, <= 7) rows of
 * w = max(1, floor(d/cs_col_div)) fp32 buckets, median decode.
 * row sketch (Sec. 4.2.2, the tensor trick; the form Sec. 5.4 runs): the
 * matrix view is hashed one row at a time, sketch row i is a w x cols fp32
 * matrix with w = max(1, floor(rows/cs_col_div)), T_i[h_i(a)][:] += s_i(a) R[a][:];
 * state per worker and tensor: cs_rows x w x cols floats, row-major; with
 * scale_dtype = CONEF_SCALE_FP16 the sketch itself is kept in binary16 (each
 * updated entry clamped to +-65504 and rounded to nearest even).
 * beta (Alg. 4, partial error feedback, 0 <= beta < 1; 0 is Alg. 2):
 * p = eta g + (1-beta) e and the stored error is C(beta e + p - Delta); the
 * row sketch, being linear, is updated as T <- beta T + sketch(p - Delta)
 * without decoding.
 * iconef = 1 (Alg. 3, version 1; identity, int8, int4 with beta = 0 only): a
 * second state q of the same kind and size is kept, p = (eta g + e~) + q,
 * e~ <- C(r), q <- C(r - decode(e~)) with r = p - Delta; conef_get_state2
 * reads it, conef_decompress_error returns e~ + q.  The tuned low-rank
 * kernels are switched off.
 * iconef = 2 (Alg. 3, version 2; Q random-k or random-block-k, C identity,
 * int8 or int4, beta = 0): e~ <- Q(r) by a second application of Q in the same
 * step, which draws its index set from the stream of step t + 2^62 (the first
 * draw would return zeros: r vanishes there); e~ is kept as its k fp32 values
 * in index order (conef_get_state2), the index set is recomputed when needed.
 * The stored state is q <- C(r - e~), and r - e~ is exactly 0 where e~ keeps a
 * value.  Next step p = (eta g + e~) + q.  conef_decompress_error returns
 * e~ + q.  A checkpoint also needs the step that stored e~
 * (conef_get_error_step / conef_set_error_step).
 * stochastic quantiser (Eq. 6 with the max-norm of Sec. 5.1, block-wise):
 * `levels` = s in 1..32767; per block a = max|r|, scale = a/s (fp32), the
 * stored level of r_j is floor(u) or floor(u)+1 with u = |r_j|/scale, up with
 * probability u - floor(u), signed; E[level * scale] = r_j.  Levels are kept
 * as int8 when s <= 127, else int16.  The uniform variate of (worker i, tensor,
 * step t, element j) is the top 24 bits of the library's 64-bit hash of j in
 * the stream (mix64(seed + i + 1), tensor, t), times 2^-24.
 * mx4, mx4-stochastic (a 4-bit float per element, see conef_mx4_quantise): the
 * row-major flattening of a tensor is quantised like one row of that many
 * elements, rounded to nearest even, or stochastically by the numbers that
 * conef_mx4_quantise draws for (seed, worker i, tensor, t).  (A context of one
 * rank's worker has worker 0 alone: seed + rank gives it, and the stochastic
 * quantiser's, the numbers of worker `rank`.)  State: two elements to a byte, then a
 * scale byte per block of 32; `block` and scale_dtype are not read.  Unlike the
 * other codes, a residual that is infinite or NaN makes its whole block NaN
 * (scale byte 255, codes 0), in this step's state and in those after it until a
 * step sends all of the block's elements (what is sent leaves zero, also where
 * p is not finite).  With beta > 0 or low-rank Q, which keep a part of what is
 * sent, such a block stays NaN.  A job clears it by writing 0 over its scale
 * byte (conef_get_state) between two steps.  iconef has to be 0.
 * cs_chunk (count sketch only; 0 = off): the sketch of Sec. 4.2.2 applied to
 * runs of a tensor, one level below the paper's layer-wise use.  A tensor of
 * d elements is cut into nc = max(1, floor(d / cs_chunk)) runs of cs_chunk
 * consecutive elements (the last run also takes the remainder); run c owns
 * the buckets [b(c), b(c+1)) of every sketch row, b(c) = floor(w c cs_chunk / d),
 * b(nc) = w, and element j of run c goes to bucket
 * b(c) + (((u >> 32) * (b(c+1) - b(c))) >> 32) with the hash u of j as before.
 * State size and layout are unchanged.  Runs never share a bucket, so the
 * library keeps a run's window in shared memory: coalesced reads and writes of
 * the sketch instead of gathers and atomic adds in L2.  Must be a multiple of
 * 256 and at least 4 cs_col_div, else CONEF_ERR_INVALID_ARG. */
typedef struct {
    int32_t kind;
    int32_t block;
    int32_t scale_dtype;
    int32_t cs_rows;
    int64_t cs_col_div;
    uint64_t seed; /* sketches: seed of the hash and sign functions */
    float beta;
    int32_t levels; /* stochastic quantiser: s */
    int32_t iconef; /* 1: iConEF-v1 (Alg. 3), see above; 0: off */
    int32_t cs_chunk; /* count sketch: elements per run, see above; 0: one run per tensor */
} conef_c_cfg;

/* Size in bytes of the device workspace for this configuration (HOST out). */
int conef_workspace_bytes(const conef_tensor *tensors /* HOST */, int n_tensors, int n_workers,
                          const conef_q_cfg *q /* HOST */, const conef_c_cfg *c /* HOST */,
                          size_t *out_bytes /* HOST */);

/* Create a context.  `workspace` is DEVICE memory, 256-byte aligned, of at
 * least conef_workspace_bytes() bytes; it stays the caller's and must outlive
 * the context.  Enqueues on `stream` the zeroing of all error state
 * (e_0 = 0, Alg. 2 line 1) and the copy of q_init.  `lr` is eta. */
int conef_init(conef_ctx **out /* HOST */, const conef_tensor *tensors /* HOST */, int n_tensors,
               int n_workers, const conef_q_cfg *q /* HOST */, const conef_c_cfg *c /* HOST */,
               float lr, void *workspace /* DEVICE */, size_t workspace_bytes,
               conef_stream stream);

/* Alg. 2 lines 5, 6, 9 for every worker and tensor.  grads is a HOST array of
 * n_workers DEVICE pointers; each points at one worker's gradient, the flat
 * fp32 concatenation of all tensors in table order (borrowed, read only,
 * 4-byte aligned; 32-byte alignment enables the vectorised kernels).
 * `step` is t; it must increase from call to call.  Identity and random-k Q
 * take phase 0 only.  Low-rank Q takes two phases because two reductions sit
 * inside Q: step(t,0) [P_i = M_i Q_{t-1}] -> reduce(MSG_P) [P_hat] ->
 * step(t,1) [Q_i = M_i^T P_hat; r; state = C(r)] -> reduce(MSG_Q) [Q_t].
 * Phase 1 may be given as phase 2 (Q_i only) followed by phase 3 (residual
 * and store only), which lets a caller read or replace the factors in
 * between; phase 4 is phase 3 computed by the fused kernel (conef_set_fused).
 * Another order returns CONEF_ERR_BAD_PHASE and launches nothing.
 * Non-finite gradients or states are not trapped and set no status: they
 * propagate IEEE-wise into p, the messages and the factors; a block maximum
 * skips NaN entries, and the stored code of a non-finite residual is
 * unspecified (but for mx4: see above conef_c_cfg). */
int conef_step(conef_ctx *ctx, int64_t step, const float *const *grads, int phase,
               conef_stream stream);

/* Alg. 2 line 7 without the division by N: out_sum[j] = ((m_0[j] + m_1[j]) +
 * m_2[j]) + ... in fp32, worker order.  out_sum is DEVICE memory of
 * conef_message_elems(which) floats, concatenated over tensors in table
 * order; it may be NULL for MSG_P and MSG_Q, whose results (the
 * orthonormalised P_hat, the warm start Q_t = sum/N) also stay inside the
 * context.  MSG_VALUES: the k selected values per compressed tensor in
 * ascending index order (all d values for Q = identity).  MSG_DENSE1D: the
 * pass-through tensors. */
int conef_reduce_messages(conef_ctx *ctx, int which, float *out_sum /* DEVICE */,
                          conef_stream stream);

/* Alg. 2 lines 7-8, x <- x - Delta_t with Delta_t the mean over workers of
 * Q's outputs.  x is DEVICE memory laid out like one worker's gradient (all
 * tensors, table order), read and written in place.  sum_values and
 * sum_dense1d are the DEVICE buffers conef_reduce_messages filled for this
 * step (MSG_VALUES; MSG_DENSE1D); either may be NULL when that message kind
 * is empty.  Identity Q and pass-through tensors: x[j] -= sum[j]/N.  Random-k:
 * x[idx[s]] -= sum[s]/N for the k shared indices of this step.  Low-rank:
 * x[a][b] -= fma-chain over c of P_hat[a][c] * Qmean[b][c], Qmean = (sum_i
 * Q_i)/N as left in the context by reduce(MSG_Q); the call must follow that
 * reduction (else CONEF_ERR_BAD_PHASE). */
int conef_apply_update(conef_ctx *ctx, float *x /* DEVICE */, const float *sum_values /* DEVICE */,
                       const float *sum_dense1d /* DEVICE */, conef_stream stream);

/* Error reset for a linear error compressor (Sec. 4.2.2 (ii); identity, count
 * sketch, row sketch): every worker's stored error becomes the mean over
 * workers, S_i <- (S_0 + S_1 + ...)/N (sum in worker order, one fp32
 * division).  Other compressors, and iconef = 2 (whose e~ is kept outside that
 * state), return CONEF_ERR_UNSUPPORTED.  Call it between steps. */
int conef_error_reset(conef_ctx *ctx, conef_stream stream);

/* Alg. 2 line 5's decode alone: the error e of one worker, concatenated over
 * the compressed tensors in table order, written to out (DEVICE,
 * conef_error_elems() floats). */
int conef_decompress_error(conef_ctx *ctx, int worker, float *out /* DEVICE */,
                           conef_stream stream);

/* Frees the host-side context and the side streams it created (the tuned low-rank passes run their
 * CTA-size classes on side streams that fork from and join into the caller's stream); the
 * workspace stays the caller's. */
void conef_destroy(conef_ctx *ctx);

/* ---- sizes ---- */
int64_t conef_message_elems(const conef_ctx *ctx, int which); /* floats per worker */
int64_t conef_error_elems(const conef_ctx *ctx);              /* sum of d over compressed tensors */
int64_t conef_state_bytes_per_worker(const conef_ctx *ctx);   /* compressed error state */

/* ---- inspection (tests, checkpoints); none is on the hot path ---- */

/* DEVICE pointer to worker's message buffer of the given kind. */
int conef_get_message(const conef_ctx *ctx, int which, int worker, float **ptr /* HOST out */);
/* DEVICE pointers to the stored error of (worker, tensor): a = codes (int8,
 * packed int4 or packed mx4), dense e (identity) or the sketch; b = scales (fp32,
 * fp16, or mx4's bytes in order) or NULL.  Sizes in bytes. */
int conef_get_state(const conef_ctx *ctx, int worker, int tensor, void **a, size_t *a_bytes,
                    void **b, size_t *b_bytes);
/* The same for the second state q of iConEF-v1, or for e~ of iConEF-v2 (a = k fp32 values, b =
 * NULL); CONEF_ERR_INVALID_ARG when iconef is 0. */
int conef_get_state2(const conef_ctx *ctx, int worker, int tensor, void **a, size_t *a_bytes,
                     void **b, size_t *b_bytes);
/* iConEF-v2: the step whose second draw of Q stored the current e~ (-1: none yet, e~ = 0), and a
 * setter for a context that resumes from a checkpoint (host only, nothing is launched;
 * CONEF_ERR_INVALID_ARG unless iconef = 2 and -1 <= step < 2^62). */
int64_t conef_get_error_step(const conef_ctx *ctx);
int conef_set_error_step(conef_ctx *ctx, int64_t step);
/* DEVICE pointer to this step's sorted random-k indices of a tensor (uint32[k]). */
int conef_get_indices(const conef_ctx *ctx, int tensor, uint32_t **idx, int64_t *k);
/* DEVICE pointers to the low-rank factors of a tensor: P_hat (rows x r), the
 * warm start Q (cols x r), and worker's local Q_i (cols x r) / P_i (rows x r). */
int conef_get_factors(const conef_ctx *ctx, int tensor, int worker, float **p_hat, float **q_prev,
                      float **q_i, float **p_i, int *rank);
/* Most recent consistency status written by the kernels (0 = none).
 * Synchronises `stream`. */
int conef_last_status(conef_ctx *ctx, conef_stream stream, int *status /* HOST out */);
/* Kernels launched by this context so far. */
int64_t conef_launch_count(const conef_ctx *ctx);
/* Rank-sharded runs (one process per GPU, the messages all-reduced across processes between
 * conef_step and conef_reduce_messages, Alg. 2 line 7): the N of the means (the warm start
 * Q_t = sum/N left by reduce(MSG_Q), the update x -= sum/N of conef_apply_update) is then the
 * number of workers of the whole job, not of this context.  total >= n_workers; the default is
 * n_workers. */
int conef_set_total_workers(conef_ctx *ctx, int total);
/* Choose kernels: 0 = generic kernels only, 1 = tuned kernels where the
 * tensor's shape and alignment allow (default). */
int conef_set_fast_path(conef_ctx *ctx, int enable);
/* For tests: has the random-k selection of every tensor above 1024 elements end as it otherwise does
 * for one tensor and step in 1e8: the window of hash values does not hold the threshold
 * (CONEF_SELECT_MISS), more elements lie inside it than its list has room for (CONEF_SELECT_FULL), or
 * the list holds something else (CONEF_SELECT_STALE, which conef_last_status reports as bit 0).
 * The index sets are the same.  CONEF_SELECT_NORMAL is the default.  Nothing is launched. */
enum { CONEF_SELECT_NORMAL = 0, CONEF_SELECT_MISS = 1, CONEF_SELECT_FULL = 2, CONEF_SELECT_STALE = 3 };
int conef_set_select(conef_ctx *ctx, int how);
/* Low-rank Q, phase 1 (Sec. 5.2; Alg. 2 line 9): on tensors whose shape allows it (rank 4 or 8,
 * cols a multiple of 32 and at least 256, int4 blocks of 128 or int8 blocks of 256) the two
 * halves of phase 1, Q_i = M_i^T P_hat and state = C(p - P_hat Q_i^T), run in ONE persistent
 * kernel whose CTAs take tiles of both halves from one list, ordered so that the second
 * half of a (worker, tensor) pair follows its first half while the gradient and the codes are
 * still in L2.  The kernel is launched cooperatively (all its CTAs resident) because a tile of
 * the second half waits for the tiles of the first; every wait is bounded, and one that runs
 * out is reported by conef_last_status.  enable = 0 (the default) keeps the separate kernels
 * (what phases 2 and 3 always run).  tile_periods = 0 takes the default tile length; a smaller number makes
 * small tensors span many tiles (tests) and is refused with CONEF_ERR_UNSUPPORTED where the
 * partial sums of a tensor would not fit the scratch.  ctas_per_sm (0 = default, or 2..4):
 * resident CTAs per SM the kernel is built for.  Nothing is launched. */
int conef_set_fused(conef_ctx *ctx, int enable, int tile_periods, int ctas_per_sm);
/* Whether phase 1 currently uses that kernel (HOST outs, any may be NULL): active, CTAs of the
 * launch, periods per tile, shared-memory slots per warp, tiles per step. */
int conef_fused_info(const conef_ctx *ctx, int *active, int *ctas, int *tile_periods, int *ring, int *tasks);
/* For tests: phase 4 of conef_step is phase 3 computed by that kernel: the residual is formed
 * with the Q_i found in the message buffer (which a caller may have replaced after phase 2),
 * and the Q_i the kernel itself computes on the way is left in a second buffer, to which this
 * returns the DEVICE pointer for (tensor, worker).  CONEF_ERR_INVALID_ARG for a tensor the
 * kernel does not take. */
int conef_get_fused_q(const conef_ctx *ctx, int tensor, int worker, float **q_i /* HOST out */);
const char *conef_error_string(int code);

/* ---- for callers that cannot allocate ----
 *
 * (The paper has no counterpart to this call: it is a packaging of step S3a,
 * the shared random-k index set, for a caller without a context.)
 *
 * The side that receives a random-k message has to know the index set S_t to
 * scatter the k values back into a dense update; S_t depends on (seed, tensor,
 * step) only.  A receiver of that kind (a parameter server, a rank that only
 * applies updates, a hook run inside another framework's step) often has no
 * ConEF context and may not use the device allocator: its memory pool is fixed
 * up front, and an allocation in the middle of a step would synchronise the
 * device or fail under memory pressure.  This call writes S_t (k indices,
 * ascending, bit-identical to what conef_step produces for the same seed,
 * tensor index and step) into idx_out (DEVICE, k uint32, caller-owned) and
 * allocates nothing: no cudaMalloc, no cudaFree, no allocating library call.
 *
 * Its scratch (one counter per 2048 elements and a list of the elements near
 * the threshold, about 290 KB) is a fixed array in the library's device image; every GPU that loads
 * the library holds it until the process exits.  Hence the limit
 * d <= CONEF_NOALLOC_MAX_ELEMS; a larger d returns CONEF_ERR_TOO_LARGE and
 * launches nothing.  The first call on a device looks up the array's device
 * address (cudaGetSymbolAddress); make that first call before any stream
 * capture.  All calls share the one array and it keeps the last call's
 * contents (each call leaves its counters zeroed), so two calls whose work
 * overlaps on the GPU -- different streams, or different host threads -- race:
 * issue them on one stream, or order them yourself.  Calls that did overlap may
 * have written wrong indices (still below d, and marked as below where the
 * threshold was not theirs); a call that starts after all of them have finished
 * is not affected.  Work is enqueued on `stream`; the call does not synchronise,
 * so a selection that fails on the device (more than 2304 elements sharing the
 * threshold's 32-bit hash: not observed, and excluded for practical purposes at
 * d <= 2^24) cannot be returned as a code: it is reported in the output instead,
 * idx_out[0] = 0xFFFFFFFF, a value no index can take, and no write ever goes
 * past idx_out[k-1].  A CUDA error pending from before the call makes it return
 * CONEF_ERR_CUDA without launching anything. */
#define CONEF_NOALLOC_MAX_ELEMS (1 << 24)
int conef_randk_indices_noalloc(uint64_t seed, int64_t tensor, int64_t step, int64_t d, int64_t k,
                                uint32_t *idx_out /* DEVICE */, conef_stream stream);
/* For tests: the same call ending as `how` says (see conef_set_select), or with the second of its two
 * kernels left out (CONEF_SELECT_HALF): what a call finds behind it is then what another's kernels
 * leave that ran between its own. */
enum { CONEF_SELECT_HALF = 4 };
int conef_randk_indices_noalloc_select(uint64_t seed, int64_t tensor, int64_t step, int64_t d, int64_t k,
                                       int how, uint32_t *idx_out /* DEVICE */, conef_stream stream);

/* ---- matrix operators: counter-based draws, dropout, microscaled 4-bit floats ----
 *
 * (The paper has no counterpart to these: they are what a training step does around the exchange of
 * gradients, on the same random streams and in the same kind of code as the error state.)
 *
 * A matrix argument is DEVICE memory: rows of `cols` elements of type CONEF_F32, CONEF_BF16 or CONEF_F16, `ld`
 * elements apart (ld >= cols where there is more than one row), aligned to its elements.  Sides and ld are below 2^31
 * (CONEF_ERR_UNSUPPORTED).  Sides of zero are allowed; nothing is launched for them.  What lies
 * between a row's end and the next row is neither read nor written.  No call allocates or synchronises; all may be captured into a graph.
 *
 * conef_draw names a set of random numbers.  Its stream is that of the step's own draws, with key mix64(seed +
 * worker + 1), tensor and step; element (r, c) of a matrix of C columns has, in the stream's hash of 2 (r ceil(C/4) +
 * floor(c/4)) (dropout) or of that + 1 (rounding), the 16 bits from 16 (c mod 4) on as its number u in 0..65535.
 * So the numbers depend on the draw, the number of columns and the element's place alone, and a
 * backward pass that names the draw of the forward pass has its numbers again.  A call captured into a graph draws the
 * numbers of the draw it was captured with in every replay. */
typedef struct {
    uint64_t seed;
    int64_t worker, tensor, step; /* >= 0 */
} conef_draw;

/* Dropout: out = x 65536 / (65536 - f) where u >= f = rint(65536 p), else 0, plus add (of the same type) unless that is
 * NULL; in fp32 with one rounding of the product and sum, then one to the type.  0 <= p <= 1.  A dropped element is
 * not read into the result, be it NaN.  The gradient of x is the same call on the gradient of out (add = NULL), that of
 * add is the gradient of out.  out may be x or add (with the same ld), else it does not overlap them. */
int conef_dropout(const void *x, const void *add, void *out, int dtype, int64_t rows, int64_t cols, int64_t x_ld,
                  int64_t add_ld, int64_t out_ld, double p, const conef_draw *draw /* HOST */, conef_stream stream);

/* A matrix in microscaled 4-bit floats (the OCP format MXFP4): blocks of 32 consecutive elements of a row, the last of a row
 * may be short; each element a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; a scale 2^E per block.  codes: for
 * each row ceil(cols/32) times 16 bytes, element 2q in the low and 2q + 1 in the high half of byte q, zero past the row's
 * end.  scales: bytes E + 127 (255: NaN) in tiles of 128 rows by 4 blocks; row r, block b has byte
 * 512 ((r/128) ceil(cols/128) + b/4) + 16 (r mod 32) + 4 (r mod 128 / 32) + b mod 4; those of rows and blocks that do not exist are zero.
 * Both are DEVICE memory, 16-byte aligned, of the sizes that conef_mx4_bytes gives. */
int conef_mx4_bytes(int64_t rows, int64_t cols, size_t *code_bytes /* HOST out */, size_t *scale_bytes /* HOST out */);

/* Quantise x: its rows into (codes, scales), and / or the rows of its transpose (cols x rows, blocks along x's columns)
 * into (codes_t, scales_t); a form not asked for is NULL.  E is the least, not below -127, for which no element is above
 * 6 2^E; a block that holds an infinity or a NaN has scale 255 and codes 0.  Elements are rounded to nearest even, or
 * (stochastic) up where floor(65536 f + 1/2) + u >= 65536, f the part of the step between the two values next to it that it lies
 * above the smaller one in size: off by 2^-17 at most from the unbiased probability.  With p > 0 what is quantised is x behind
 * the dropout above (rounded to fp32 once).  Both forms round an element by the same number.  draw may be NULL where
 * nothing is drawn. */
int conef_mx4_quantise(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, double p, int stochastic,
                       const conef_draw *draw /* HOST */, void *codes, void *scales, void *codes_t, void *scales_t,
                       conef_stream stream);
/* The values of a form, code 2^E, rounded to the type (in fp32 they are exact below 2^128, and infinite there: x above 1.75 2^127 in size
 * is rounded to that). */
int conef_mx4_dequantise(const void *codes, const void *scales, int64_t rows, int64_t cols, void *out, int dtype, int64_t ld,
                         conef_stream stream);
/* out[i][j] = sum over c < k of A[i][c] B[j][c] for forms A (m x k) and B (n x k), accumulated in fp32 and rounded once to the
 * type.  The bytes past a row's end and the scales of rows and blocks that do not exist have to be zero, as conef_mx4_quantise
 * leaves them.  k = 0 gives zeros.  The kernel's parts wait for one another, at a time for two seconds at most (for the sums of a tile of outputs
 * four microseconds more per 256 of k).  Should a wait run out (not observed), the kernel ends within two seconds more, conef_mx4_timeouts counts it, and the
 * outputs that were not computed are NaN. */
int conef_mx4_matmul(const void *a_codes, const void *a_scales, int64_t m, const void *b_codes, const void *b_scales, int64_t n,
                     int64_t k, void *out, int dtype, int64_t ld, conef_stream stream);
/* How many thread blocks of conef_mx4_matmul have had a wait run out on the current device since the library was loaded, the work
 * ahead in `stream` included.  Synchronises `stream`. */
int conef_mx4_timeouts(int64_t *count /* HOST out */, conef_stream stream);
/* For tests: the longest wait of the products that are enqueued from here on (0: two seconds), and the number of stages of 256 elements of k (8-bit forms:
 * 128, conef_orthogonalise: 64) that each thread block, or the first and the second one of a pair, brings before it stops, as one that hangs would
 * (-1: all of them).  For the products of all formats.  Nothing is launched. */
int conef_mx4_set_waits(int64_t nanoseconds, int64_t loads, int64_t loads_second);

/* ---- 8-bit floats with a scale per block of 128, root-mean-square norms, orthogonalised updates ----
 *
 * (The paper has no counterpart to these either: a layer's way in, its products and its update, beside the exchange of gradients.)  The rules for
 * matrix arguments above hold here too.
 *
 * A matrix in 8-bit floats with block scales: blocks of 128 consecutive elements of a row, the last of a row may be short; a code (CONEF_E4M3 or CONEF_E5M2) per
 * element; a scale 2^E per block.  codes: ceil(cols/128) times 128 bytes per row, zero past the row's end.  scales: bytes E + 127 (255: NaN) in
 * tiles of 128 rows by 4 blocks; row r, block b has byte 512 ((r/128) ceil(cols/512) + b/4) + 16 (r mod 32) + 4 (r mod 128 / 32) + b mod 4; those of rows
 * and blocks that do not exist are zero.  Both are DEVICE memory, 16-byte aligned, of the sizes that conef_f8_bytes gives. */
int conef_f8_bytes(int64_t rows, int64_t cols, size_t *code_bytes /* HOST out */, size_t *scale_bytes /* HOST out */);

/* Quantise x: its rows into (codes, scales), and / or the rows of its transpose (cols x rows, blocks along x's columns) into (codes_t, scales_t); a form not asked
 * for is NULL.  E is the least, not below -127, for which no element is above the type's largest value times 2^E; a block that holds an infinity or a NaN has
 * scale 255 and codes 0.  Elements are rounded to nearest even.  With `square`, 128 rows by 128 columns are a block (and have their scale once per row): both
 * forms then stand for the same values. */
int conef_f8_quantise(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int kind, int square, void *codes, void *scales, void *codes_t, void *scales_t,
                      conef_stream stream);
/* The values of a form, code 2^E, rounded to the type, nearest even: exact in fp32, and in bf16 where they are multiples of 2^-133 (all are where E >= -124, of
 * CONEF_E5M2 -117, and those of 2^-126 or more); 2^128 and more is infinite. */
int conef_f8_dequantise(const void *codes, const void *scales, int64_t rows, int64_t cols, int kind, void *out, int dtype, int64_t ld, conef_stream stream);
/* out[i][j] = sum over c < k of A[i][c] B[j][c] for forms A (m x k) and B (n x k) of either kind, accumulated in fp32 and rounded once to the type.  What
 * conef_mx4_matmul says of bytes past a row's end, of k = 0 and of waits holds here too; conef_f8_timeouts counts these. */
int conef_f8_matmul(const void *a_codes, const void *a_scales, int a_kind, int64_t m, const void *b_codes, const void *b_scales, int b_kind, int64_t n, int64_t k, void *out,
                    int dtype, int64_t ld, conef_stream stream);
int conef_f8_timeouts(int64_t *count /* HOST out */, conef_stream stream);

/* Root-mean-square norm of x's rows, behind the addition of a residual where `add` is not NULL: h = x + add, rounded to the type and written (without add, h is x
 * and the argument NULL); rstd[r] = 1 / sqrt(mean over the row of h^2 + eps), computed in 64 bits and rounded to fp32 (DEVICE, one per row); and h rstd weight,
 * either rounded to the type into y, or in 8-bit floats into (codes, scales) and / or (codes_t, scales_t) as conef_f8_quantise has them: the codes and scales are
 * those of the exact products (where these are above 2^-100 in size; fp32's 2^128 and more counts as infinite).  y and the forms may all be NULL.
 * weight: `cols` elements of the matrices' type or of CONEF_F32.  A row that holds an infinity or a NaN has rstd 0 or NaN, and what follows by IEEE rules.  h may be x or
 * add, y may be x, add or h (with the same ld); otherwise outputs do not overlap inputs. */
int conef_rms_norm(const void *x, const void *add, const void *weight, int dtype, int weight_dtype, int64_t rows, int64_t cols, int64_t x_ld, int64_t add_ld, double eps,
                   void *h, int64_t h_ld, float *rstd, void *y, int64_t y_ld, int kind, void *codes, void *scales, void *codes_t, void *scales_t, conef_stream stream);
/* Its gradient: with n = h rstd and g = dy weight, dx = rstd (g - n mean(g n)) + add, the gradient of x and of the residual (add: the gradient that reaches h
 * another way, or NULL), in fp32 and rounded once to the type; dweight[c] = sum over rows of dy n (fp32, DEVICE, or NULL), the same in every call.  dx may be
 * dy or add (with the same ld).  `workspace`: DEVICE, 4-byte aligned, of the size that conef_rms_norm_grad_bytes gives; it is the call's until that has
 * run on the stream. */
int conef_rms_norm_grad_bytes(int64_t rows, int64_t cols, size_t *bytes /* HOST out */);
int conef_rms_norm_grad(const void *dy, const void *h, const void *weight, const float *rstd, const void *add, int dtype, int weight_dtype, int64_t rows, int64_t cols,
                        int64_t dy_ld, int64_t h_ld, int64_t add_ld, void *dx, int64_t dx_ld, float *dweight, void *workspace, size_t workspace_bytes,
                        conef_stream stream);

/* Newton-Schulz orthogonalisation (Muon) of `batch` matrices of rows x cols (elements of a row are consecutive, rows `ld` apart, matrices `stride`, behind one another or
 * each between the others' rows, so that none share an element): X_0 = x / |x|, the Frobenius norm (a matrix of zeros stays one), `steps` (1..32) times
 * X <- (c0 + c1 A + c2 A^2) X with A = X X^T, the shorter side in front, and out = scale X, rounded once to CONEF_BF16 or CONEF_F16.  Operands of all products are held to 22 bits under a power of two and summed in fp32, which the
 * tensor cores cut off, not round, every 16 elements: ahead of the rounding to 16 bits the result is within 2^-12 of the exact one's size for up to ten steps of Muon's quintic and
 * sides of up to 16384 (of some hundred elements, and five steps, 1e-5).
 * coefficients: HOST, three; the polynomial s (c0 + c1 s^2 + c2 s^4) has to keep singular values below 10^4 in size over the steps (else
 * CONEF_ERR_INVALID_ARG).  A matrix that holds an infinity or a NaN becomes NaN.  out may be x (with the same distances).  `workspace`: DEVICE, 128-byte
 * aligned, of the size that conef_orthogonalise_bytes gives; it is the call's until that has run on the stream.  Waits are bounded as conef_mx4_matmul's,
 * conef_orthogonalise_timeouts counts these. */
int conef_orthogonalise_bytes(int64_t batch, int64_t rows, int64_t cols, size_t *bytes /* HOST out */);
int conef_orthogonalise(const void *x, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int steps, const double *coefficients /* HOST */,
                        double scale, void *out, int out_dtype, int64_t out_ld, int64_t out_stride, void *workspace, size_t workspace_bytes, conef_stream stream);
int conef_orthogonalise_timeouts(int64_t *count /* HOST out */, conef_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* CONEF_H */
