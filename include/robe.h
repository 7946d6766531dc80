/*
 * robe.h - C ABI of the B200 (sm_100a) ROBE-Z embedding library.
 *
 * ROBE (Random Offset Block Embedding array, arXiv 2108.02191) replaces all
 * embedding tables of a recommendation model by ONE circular array M of m learned
 * scalars.  The d-dimensional embedding of token x of table e is assembled from
 * ceil(d/Z) blocks of Z consecutive array elements; block c starts at the
 * universal-hash offset h(e,x,c) and wraps around the end of the array
 * (Section 3.1 "ROBE-D", Section 3.2 "ROBE-Z").  The backward pass adds the
 * output gradients back into the slots they were read from (Section 3.1,
 * backward equation).
 *
 * Conventions shared by every entry point
 *   - All sizes are in ELEMENTS unless a name says bytes.
 *   - "device pointer" = memory of the CUDA device that is current when the call
 *     is made; "host pointer" = ordinary host memory.  The library never
 *     allocates or frees device memory, and never synchronises, except where an
 *     entry point says otherwise.
 *   - Bags are sample-major.  With T tables and a batch of B samples there are
 *     B*T bags; bag k = n*T + e belongs to sample n and table e = k mod T and
 *     covers indices[offsets[k] .. offsets[k+1]).  offsets == NULL means one id
 *     per bag (one-hot): bag k is indices[k] and nnz must equal B*T.
 *   - Output / output-gradient element (n, e, i) lives at ((n*T + e)*d + i).
 *   - Every function returns a robe_status; invalid arguments launch nothing.
 *     No exception, abort or device trap crosses this boundary.
 *   - Launches are asynchronous on the given stream (a cudaStream_t passed as
 *     void*; NULL is the legacy default stream).
 */
#ifndef ROBE_H_
#define ROBE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct robe_ctx* robe_handle_t; /* opaque; host memory owned by the library */

typedef enum {
    ROBE_OK = 0,
    ROBE_ERR_INVALID_ARG = -1, /* null pointer, zero size, d > M, Z > d not a multiple of d, M + d > 2^32, ... */
    ROBE_ERR_NO_ARRAY = -2,    /* forward/backward before robe_attach_array            */
    ROBE_ERR_WORKSPACE = -3,   /* deterministic backward: workspace missing/too small  */
    ROBE_ERR_CUDA = -4,        /* the CUDA runtime reported an error at launch         */
    ROBE_ERR_UNSUPPORTED = -5  /* valid request that this build does not implement     */
} robe_status;

/* array element types */
#define ROBE_F32 0
#define ROBE_BF16 1

/* option keys for robe_set_option */
#define ROBE_OPT_SIGN 1     /* 0 (default) | 1: multiply by the sign hash g(e,x,i)        */
#define ROBE_OPT_BWD_MODE 2 /* ROBE_BWD_ATOMIC (default) | ROBE_BWD_DETERMINISTIC | ROBE_BWD_BINNED */
#define ROBE_OPT_VALIDATE 3 /* 0 (default) | 1: range-check ids/offsets on the device and
                               record the first violation in a status word instead of
                               using the bad value.  The word is sticky: while it is
                               non-zero EVERY kernel of EVERY later call on the handle
                               returns at once - robe_forward leaves `out` as it was
                               (not overwritten), robe_forward_keep keeps nothing, the
                               backward calls add nothing - and the host call still
                               returns ROBE_OK.  Read it with robe_last_device_status
                               and zero it yourself before going on.                      */
#define ROBE_OPT_FWD_KERNEL 4 /* forward kernel; every variant gives the same bits.
                                 0 automatic (default).  One-hot, sign off, block starts not kept: the
                                   rows kernel (repeats of an id gathered once) from 32768 rows on with
                                   more than 16 chunks per row (d <= 128, Z <= d); else, in large calls,
                                   the staged kernel for rows of 64 or 128 elements in blocks of 8 or 16
                                   and more (of 32 elements on arrays over 192 MB; of bf16 arrays with
                                   any block) and for most rows with a short last block; else the flat
                                   kernel (rows of any length as one run of elements).
                                   Pooled: the lane-hashed kernel for Z <= 2 on arrays of up to 192 MB,
                                   sign off; the pool kernel (a run of bags per warp) for many short
                                   bags, d <= 128.
                                   What is left: the staged kernel for d <= 128, else the direct one
                                 1 direct: any (Z, d); every lane hashes its element's chunk per id
                                 2 staged: d <= 128; block starts of a batch of ids through shared
                                   memory, 4-byte loads, lanes on consecutive slots of a block
                                 3 vector: 16-byte loads of the aligned pieces around a block, shifted
                                   in registers; fp32 array, d, Z and M multiples of 4, d <= 128, sign
                                   off (measured slower than 2 on every workload; kept for comparison)
                                 4 lane-hashed: d <= 128, Z <= d, sign off; chunks hashed in registers by
                                   the lane that owns the element, persistent warps
                                 A variant asked for a call it cannot take returns
                                 ROBE_ERR_UNSUPPORTED and launches nothing.                          */
#define ROBE_OPT_BWD_KERNEL 5 /* kernel of the ATOMIC backward (all within the atomic bound):
                                 0 automatic (default).  One-hot, sign off: the rows kernel (repeats of
                                   an id summed first) from 131072 rows on, from 32768 with more than 16
                                   chunks per row (d <= 128, Z <= d); else the flat kernel.
                                   Pooled: the pool kernel (a run of bags per warp) for many short bags,
                                   d <= 128.
                                   What is left: staged for d <= 128, else direct
                                 1 direct   2 staged (scalar red.global.add.f32, lanes on consecutive slots)
                                 3 vector: red.global.add.v4.f32 on the aligned middle of a block,
                                   scalar head and tail; d, Z, M multiples of 4, d <= 128, sign off
                                   (measured slower than 2; kept for comparison)
                                 4 vector, repeats of an id inside a staged batch merged first
                                 5 merged rows: one-hot input, sign off, d <= 128; a warp takes up to 64
                                   rows of ONE table, sums the gradient rows of repeated ids in
                                   registers and issues one reduction per element for all of them
                                   (skewed ids, Z = 128: 1.34 x over 2, 10-40 % slower on uniform ids;
                                   the rows kernel of the automatic choice, which looks for repeats
                                   among up to 512 rows, is faster on both)
                                 6 lane-hashed: d <= 128, Z <= d, sign off (the reductions, not the
                                   hashing, bound this pass: measured no faster than 2)              */

#define ROBE_OPT_INDEX_TYPE 6 /* ROBE_I64 (default) | ROBE_I32: element type of `indices` in the
                                 calls that follow (offsets stay int64)                   */

#define ROBE_OPT_BAG_LAYOUT 7 /* ROBE_BAGS_SAMPLE_MAJOR (default): bag k = n*T + e, out and grad_out are
                                 [batch, T, d];  ROBE_BAGS_TABLE_MAJOR: bag k = e*batch + n - the ids of
                                 table 0 for all samples, then table 1, ... (per-table id lists laid end
                                 to end) - and out and grad_out are [T, batch, d].  Applies to the calls
                                 that follow; offsets index bags in the chosen order.              */
#define ROBE_BAGS_SAMPLE_MAJOR 0
#define ROBE_BAGS_TABLE_MAJOR 1

#define ROBE_OPT_ARRAY_L2_KEEP 8 /* 0 (default) on | 1 off: the reductions of the atomic and the binned
                                    backward carry the L2 cache policy "evict these lines last"
                                    (createpolicy ... L2::evict_last), so that a gradient target about
                                    the size of the L2 stays there next to the streamed ids and gradient
                                    rows: 19-35 % faster on a 100 MB array, no slower elsewhere.  Results
                                    are unchanged.  (The same policy on the forward's loads measured no
                                    effect and is not offered.)                                      */

/* index element types */
#define ROBE_I64 0
#define ROBE_I32 1

#define ROBE_BWD_ATOMIC 0
#define ROBE_BWD_DETERMINISTIC 1
#define ROBE_BWD_BINNED 2

/* values of the device status word (robe_last_device_status) */
#define ROBE_DEV_OK 0
#define ROBE_DEV_BAD_INDEX 1  /* an id was negative                         */
#define ROBE_DEV_BAD_OFFSETS 2 /* offsets not monotone or out of [0, nnz]   */

/*
 * robe_create - make a handle for one ROBE array shape (Section 3.2).
 *   out         host pointer receiving the handle.
 *   M           array length m = |M| in elements; 1 <= d <= M and M + d <= 2^32.
 *   Z           block size.  1 <= Z <= d: Z = d is ROBE-D (one block per embedding,
 *               Section 3.1); Z = 1 hashes every element on its own (Section 3.3); if Z
 *               does not divide d the last block is short.  Z > d (Section 3.2, last
 *               paragraph: several embeddings clubbed into one chunk): Z must be a
 *               multiple of d and <= M; rows floor(x/R) R .. + R-1 of a table, R = Z/d,
 *               then share the block that starts at h(e, floor(x/R), 0), row x being the
 *               piece [(x mod R) d, (x mod R) d + d) of it.
 *   d           embedding dimension (one d per handle; several handles may share
 *               one array, Section 3.1 "Multiple embedding tables").
 *   num_tables  T >= 1; the table id e of bag k is k mod T (k / batch after
 *               ROBE_OPT_BAG_LAYOUT = ROBE_BAGS_TABLE_MAJOR).
 *   hash_seed   seeds the draw of the hash constants: P = 2^61 - 1 and, from a
 *               SplitMix64 stream, A_h B_h C_h D_h A_g B_g C_g D_g (61-bit draws,
 *               redrawn when outside [1,P-1] for multipliers / [0,P-1] for the
 *               additive terms), as the paper's hash family requires.
 * A handle holds options and, after the first deterministic backward, a CUDA stream and two
 * events of its own (no device memory) on the device that was current at that call; a
 * deterministic backward made later with another device current runs in the caller's stream
 * alone.  Calls on ONE handle must not overlap in time on the host; different handles are
 * independent.
 * Errors: ROBE_ERR_INVALID_ARG.
 */
int robe_create(robe_handle_t* out, uint64_t M, uint32_t Z, uint32_t d, uint32_t num_tables,
                uint64_t hash_seed);

/* robe_destroy - free the host handle (waits for the handle's own stream, if it has one).  Device
 * buffers stay the caller's. */
int robe_destroy(robe_handle_t h);

/* robe_set_option - see the ROBE_OPT_* keys.  ROBE_ERR_INVALID_ARG on a bad key/value. */
int robe_set_option(robe_handle_t h, int key, int64_t value);

/*
 * robe_attach_array - name the parameter array M (Section 3: the one array that holds the
 * learned parameters of all tables).
 *   dev_array  device pointer to M elements of `dtype`, 16-byte aligned, owned by the
 *              caller, read by forward and updated in place by the fused-SGD backward.
 *   dtype      ROBE_F32 or ROBE_BF16 (bf16 is read-only: widened exactly to fp32).
 */
int robe_attach_array(robe_handle_t h, void* dev_array, int dtype);

/*
 * robe_get_hash_constants - copy out {P, A_h, B_h, C_h, D_h, A_g, B_g, C_g, D_g}
 * (host pointer to 9 words) so that a checker can be handed numbers, not code.
 *   h(e,x,c) = ((A_h e + B_h x + C_h c + D_h) mod P) mod M           (Section 3.2)
 *   g(e,x,i) = 2 (((A_g e + B_g x + C_g i + D_g) mod P) mod 2) - 1   (Section 3.1)
 */
int robe_get_hash_constants(robe_handle_t h, uint64_t out[9]);

/*
 * robe_forward - embedding lookup with optional sum pooling (Section 3.2 forward).
 *   out[n,e,i] = sum over ids x_p of bag (n,e), in bag order, sequentially in fp32
 *                (first term initialises), of g(e,x_p,i) * M[(h(e,x_p,i/Z) + i%Z) mod M]
 *   indices  device pointer, int64 [nnz] (int32 [nnz] after ROBE_OPT_INDEX_TYPE = ROBE_I32),
 *            ids >= 0.
 *   offsets  device pointer, int64 [batch*T + 1], offsets[0] = 0, non-decreasing,
 *            offsets[batch*T] = nnz; or NULL for one-hot (then nnz == batch*T).
 *   batch    number of samples B >= 0;  nnz >= 0 total ids.
 *   out      device pointer, fp32 [batch, T, d] ([T, batch, d] with ROBE_BAGS_TABLE_MAJOR), fully
 *            overwritten; an empty bag gives +0.
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_NO_ARRAY, ROBE_ERR_CUDA.
 */
int robe_forward(robe_handle_t h, const void* indices, const int64_t* offsets, int64_t batch,
                 int64_t nnz, float* out, void* stream);

/*
 * robe_backward_workspace_bytes - bytes of caller-provided device scratch that
 * robe_backward needs in the handle's current backward mode for a call of this
 * size (0 in atomic mode; binned and deterministic mode need the same).  Returns 0 for a
 * bad handle.
 */
size_t robe_backward_workspace_bytes(robe_handle_t h, int64_t batch, int64_t nnz);

/*
 * robe_backward - scatter-add of the output gradient (Section 3.1 backward equation):
 *   delta[j] = sum over (p, i) with idx(e, x_p, i) = j of g(e,x_p,i) * grad_out[bag(p), i]
 * every occurrence of an id contributes, duplicates included.
 *   grad_out    device pointer, fp32 [batch, T, d].
 *   grad_array  device pointer, fp32 [M]: delta is ADDED to it (the caller zeroes it
 *               when a plain gradient is wanted).  NULL selects the fused SGD step
 *               M[j] <- M[j] - lr * delta[j] applied in place to the attached fp32
 *               array (the paper trains its DLRM with plain SGD, Section 5).
 *   lr          learning rate, used only when grad_array == NULL.
 *   workspace   device pointer to workspace_bytes bytes, 256-byte aligned; may be NULL
 *               in atomic mode.
 * Atomic mode adds with red.global (fp32, order not fixed).  Binned mode does the same adds
 * after grouping the blocks by array region (one radix pass on the top bits of the block
 * start), so that the read-modify-write of an array much larger than the L2 happens in L2; it
 * needs the workspace of the deterministic mode and gives atomic-mode accuracy, not
 * reproducible bits.  Deterministic mode sorts
 * the blocks by start offset (stable) and lets each array slot sum its terms in that
 * order in fp32 from +0, then applies ONE add (dense) or ONE fma (SGD) per touched
 * slot: results are bit-reproducible.
 * Errors: ROBE_ERR_INVALID_ARG (also: fused SGD on a bf16 array), ROBE_ERR_NO_ARRAY,
 * ROBE_ERR_WORKSPACE, ROBE_ERR_CUDA.
 */
int robe_backward(robe_handle_t h, const float* grad_out, const void* indices,
                  const int64_t* offsets, int64_t batch, int64_t nnz, float* grad_array, float lr,
                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * robe_forward_keep / robe_backward_kept - the forward and backward of one training step on
 * the same ids, sharing the hash work.  The block starts h(e, x_p, c) that the forward computes
 * (Section 3.2) are what the binned and the deterministic backward sort by; robe_forward_keep
 * is robe_forward that also stores them in `workspace`, and robe_backward_kept is
 * robe_backward that takes them from there instead of hashing every id again.  The paper has
 * no counterpart: it is a fusion across the two passes, results are those of robe_forward and
 * robe_backward bit for bit (deterministic mode) or within the same bound (binned mode).
 *   workspace  device pointer, 256-byte aligned, at least robe_backward_workspace_bytes(h,
 *              batch, nnz) bytes; owned by the caller, who leaves it untouched between the two
 *              calls.  The backward consumes what was kept: one robe_backward_kept per
 *              robe_forward_keep.
 *   The two calls get the same indices, offsets, batch and nnz, with the handle's sign,
 *   index-type and backward-mode options unchanged in between.  The backward trusts what the
 *   workspace holds: after anything else (other sizes, a workspace written to in between, no
 *   robe_forward_keep before) its behaviour is undefined, as for a wrong pointer.
 * In atomic mode nothing is sorted: the two calls are then robe_forward and robe_backward, and
 * workspace may be NULL.
 * Errors: those of robe_forward and robe_backward; ROBE_ERR_UNSUPPORTED and
 * ROBE_ERR_WORKSPACE already from robe_forward_keep.
 */
int robe_forward_keep(robe_handle_t h, const void* indices, const int64_t* offsets, int64_t batch,
                      int64_t nnz, float* out, void* workspace, size_t workspace_bytes, void* stream);
int robe_backward_kept(robe_handle_t h, const float* grad_out, const void* indices,
                       const int64_t* offsets, int64_t batch, int64_t nnz, float* grad_array, float lr,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * robe_backward_adam - deterministic backward with the Adam step fused in (the paper trains
 * five of its six Criteo-Kaggle models with Adam, Section 5; the update is Algorithm 1 of
 * Kingma & Ba, "Adam: a method for stochastic optimization").  For every array slot j that
 * receives at least one gradient term, with delta[j] summed in the deterministic order of
 * robe_backward:
 *     m1[j] = beta1 m1[j] + (1 - beta1) delta[j]
 *     m2[j] = beta2 m2[j] + (1 - beta2) delta[j]^2
 *     M[j]  = M[j] - lr * (m1[j] / (1 - beta1^step)) / (sqrt(m2[j] / (1 - beta2^step)) + eps)
 * each operation a separate round-to-nearest fp32 one; slots without a term keep M, m1 and m2
 * as they are (the "lazy" form that sparse embedding updates use).  Bit-reproducible.
 *   m1, m2   device pointers, fp32 [M], caller-owned, zeroed by the caller before step 1.
 *   step     t >= 1, the number of this update (used for the bias corrections only).
 *   workspace / workspace_bytes  as for robe_backward in deterministic mode; size it with
 *            robe_backward_workspace_bytes after ROBE_OPT_BWD_MODE = ROBE_BWD_DETERMINISTIC.
 * The handle's ROBE_OPT_BWD_MODE is not consulted.  The attached array must be fp32.
 * Errors: as robe_backward; ROBE_ERR_INVALID_ARG also for null moments, step < 1, beta outside
 * [0, 1) or eps < 0.
 */
int robe_backward_adam(robe_handle_t h, const float* grad_out, const void* indices,
                       const int64_t* offsets, int64_t batch, int64_t nnz, float* m1, float* m2,
                       float lr, float beta1, float beta2, float eps, int64_t step, void* workspace,
                       size_t workspace_bytes, void* stream);

/*
 * robe_backward_adagrad - deterministic backward with the Adagrad step fused in (Duchi, Hazan, Singer,
 * "Adaptive subgradient methods ..."; the optimizer recommendation models are commonly trained with,
 * beside the SGD and Adam of the paper's Section 5).  Embedding tables usually keep ONE accumulator
 * per row ("row-wise Adagrad"); the ROBE array has no rows - a slot is shared by elements of many
 * rows of many tables - so the accumulator is per slot.  For every array slot j that receives at
 * least one gradient term, with delta[j] summed in the deterministic order of robe_backward:
 *     sum_sq[j] = sum_sq[j] + delta[j]^2
 *     M[j]      = M[j] - lr * delta[j] / (sqrt(sum_sq[j]) + eps)
 * each operation a separate round-to-nearest fp32 one; other slots keep M and sum_sq.  Bit-reproducible.
 *   sum_sq   device pointer, fp32 [M], caller-owned, zeroed by the caller before the first step.
 *   workspace / workspace_bytes  as for robe_backward in deterministic mode.
 * The handle's ROBE_OPT_BWD_MODE is not consulted.  The attached array must be fp32.
 * Errors: as robe_backward; ROBE_ERR_INVALID_ARG also for a null sum_sq or eps < 0.
 */
int robe_backward_adagrad(robe_handle_t h, const float* grad_out, const void* indices,
                          const int64_t* offsets, int64_t batch, int64_t nnz, float* sum_sq, float lr,
                          float eps, void* workspace, size_t workspace_bytes, void* stream);

/*
 * robe_apply_sgd - the dense SGD apply of a data-parallel training step (Section 1 of the
 * paper, implications of the compression: the whole model fits every GPU, so training is plain
 * data-parallel and the ranks exchange one gradient the size of the array; Section 5: SGD).
 * A rank runs robe_backward with a dense grad_array on its shard of the batch, the caller
 * sums grad_array over the ranks (an all-reduce: 4 M bytes), and this call applies the sum
 *     M[j] <- fma(-lr, grad_array[j], M[j])       for every j < M
 * to the attached fp32 array in one streaming pass.  On one rank it gives the bits of the
 * fused step (robe_backward with grad_array == NULL) when grad_array held +0 before the
 * deterministic backward ran.
 *   grad_array  device pointer, fp32 [M], 16-byte aligned; with zero_grad = 1 it is left
 *               holding +0 everywhere, ready for the next step's robe_backward.
 *   zero_grad   0 or 1.
 * Errors: ROBE_ERR_INVALID_ARG (null or misaligned pointer, bf16 array), ROBE_ERR_NO_ARRAY,
 * ROBE_ERR_CUDA.
 */
int robe_apply_sgd(robe_handle_t h, float* grad_array, float lr, int zero_grad, void* stream);

/*
 * robe_backward_deterministic_static - the deterministic robe_backward for callers that
 * cannot supply scratch memory.  (The paper has no counterpart: this is a convenience of
 * this library, not part of the method.)
 *
 * Who needs it: code that runs where device allocation is off the table - for example a
 * serving process whose memory pool already owns the whole device, so a cudaMalloc would
 * fail or stall every stream while it synchronises the device, or an operator plugged
 * into a host framework that hands it input and output buffers and nothing else.  Such a
 * caller has no way to come up with the workspace robe_backward asks for in
 * deterministic mode.  Here the workspace is a fixed array of ROBE_STATIC_SCRATCH_BYTES
 * that is part of the library image itself: every device that loads librobe.so carries
 * it from load until the process exits, whether or not this function is ever called.
 *
 * Arguments and result are those of robe_backward in ROBE_BWD_DETERMINISTIC mode (the
 * handle's ROBE_OPT_BWD_MODE is ignored), minus workspace/workspace_bytes: the caller
 * still passes grad_out, indices, offsets and grad_array (or NULL for the fused SGD step),
 * and gets bit-identical output.  The function calls no cudaMalloc, cudaFree or other
 * allocating routine.
 *
 * Limit: the call must fit the fixed array, i.e. the value robe_backward_workspace_bytes
 * reports for it in deterministic mode (about 19 bytes per block, nnz * ceil(d/Z) blocks,
 * plus 4 bytes per id, 0.3 MB of counters and lists, and up to 0.25 MB more where a call
 * touches an array of up to 5.5 M slots densely) must not exceed
 * ROBE_STATIC_SCRATCH_BYTES; a larger call returns ROBE_ERR_WORKSPACE and launches nothing.
 *
 * First call on a device: the function looks up the device address of the array once per
 * device (with that device current) and remembers it.  Make that first call during
 * set-up, before any stream capture is begun.
 *
 * Sharing: all handles, streams and threads of the process use the same array on a given
 * device, and it keeps whatever the previous call left in it.  The function re-initialises
 * the parts that must start from zero on every call, so back-to-back calls on ONE stream
 * are safe; two calls that may overlap on the GPU (different streams without an ordering
 * between them) race on the array and give undefined results - order them yourself.
 *
 * Errors: as robe_backward, plus ROBE_ERR_WORKSPACE for a call beyond the limit and
 * ROBE_ERR_CUDA if the address lookup fails.
 */
#define ROBE_STATIC_SCRATCH_BYTES (32u << 20) /* 32 MiB per device */
int robe_backward_deterministic_static(robe_handle_t h, const float* grad_out,
                                       const void* indices, const int64_t* offsets,
                                       int64_t batch, int64_t nnz, float* grad_array, float lr,
                                       void* stream);

/*
 * robe_set_status_word - give the handle a device int32 (caller-owned, zeroed by the
 * caller) that kernels write a ROBE_DEV_* code into when ROBE_OPT_VALIDATE is on.  Only the
 * first violation is recorded (compare-and-swap from ROBE_DEV_OK), and a non-zero word turns
 * all later launches on the handle into no-ops until the caller zeroes it (see
 * ROBE_OPT_VALIDATE).
 * robe_last_device_status - synchronise `stream`, read that word (device-to-host copy)
 * and return it (>= 0), or a negative robe_status.
 */
int robe_set_status_word(robe_handle_t h, int32_t* dev_word);
int robe_last_device_status(robe_handle_t h, void* stream);

/*
 * robe_debug_status / robe_debug_selftest - the index-check build (librobe_debug.so: the same
 * sources compiled with -DROBE_DEBUG; it stands in for a memory checker on machines where none can
 * be run).  In that build every computed index of every kernel - array slots, sorted positions,
 * shared-memory offsets, positions in grad_out, window and hand-over record numbers - is compared
 * with its bound before use; a violation records a ROBE_DBG_* code (the first one sticks) and the
 * access is skipped: nothing traps, the context stays usable.  robe_debug_status synchronises
 * `stream`, returns the recorded code (0 = none; see the ROBE_DBG_* values below) and clears it.
 * robe_debug_selftest launches one kernel that fails a check on purpose WITHOUT touching memory
 * (code 99), to show that the reporting path works.  The release library performs no check and
 * returns ROBE_ERR_UNSUPPORTED from both.
 */
#define ROBE_DBG_ARRAY_SLOT 1
#define ROBE_DBG_SORT_POS 2
#define ROBE_DBG_SHARED 3
#define ROBE_DBG_GRAD_POS 4
#define ROBE_DBG_WINDOW 5
#define ROBE_DBG_LONG_WALK 6
#define ROBE_DBG_ROW_POS 7 /* position in a tensor of a row operator */
#define ROBE_DBG_SELFTEST 99
int robe_debug_status(void* stream);
int robe_debug_selftest(void* stream);

/* ------------------------------------------------------------------------------------------------
 * Row operators: what a model does next with the rows it looked up.  They take no ROBE handle.  Element
 * types are ROBE_F32 and ROBE_BF16 (`dtype`); everything is computed in fp32 and rounded once, to nearest
 * even, where a result is stored; results are bit-reproducible.  A matrix is a device pointer, aligned to
 * its elements, and a leading dimension `ld`: the distance of its rows in elements, at least their length
 * (not looked at for a single row).  16-byte aligned rows are the fastest, any alignment is served.  An output
 * overlaps no input and no other output unless an entry point says so (ROBE_ERR_INVALID_ARG); columns of
 * one wider matrix do not overlap.  What stands between the rows of an output is left as it was.
 * ROBE_ERR_UNSUPPORTED: more than a launch grid can hold.
 */

/*
 * robe_dropout - out[r,c] = kept(r,c) ? in[r,c] * s : +0.  The decisions come from a counter-based
 * generator and are never stored: the gradient of the call is the same call on the gradient of `out`.
 * With t = floor(65536 p + 1/2) (p to the nearest multiple of 2^-16, so that the expectation is exact)
 *     kept(r,c) = half(r,c) >= t,     s = 65536 / (65536 - t)
 * where half(r,c) is 16-bit half c mod 8 (low half of a word first) of the four words that Philox4x32
 * with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) makes
 * of the counter (floor(c / 8), r, low and high half of n) under the key (low, high half of seed), with
 * n = (offset + *step) mod 2^64.  A dropped NaN or infinity gives +0.  The decision does not depend on
 * dtype, ld or alignment.  t = 65536 drops everything.
 *   rows, cols  >= 0; rows <= 2^32, cols <= 2^31.   out may be `in` itself (same pointer, same ld).
 *   p           in [0, 1].
 *   seed        one per training run, say;  offset  one per call of a step (layer number).
 *   step        device pointer to one uint64 that the kernel reads when it runs, so that a captured
 *               graph draws anew in every replay once the caller counts it up; or NULL (0).
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_UNSUPPORTED, ROBE_ERR_CUDA.
 */
int robe_dropout(const void* in, int64_t in_ld, void* out, int64_t out_ld, int64_t rows, int64_t cols,
                 int dtype, float p, uint64_t seed, uint64_t offset, const uint64_t* step, void* stream);

typedef struct robe_bias_ctx* robe_bias_t; /* opaque; host memory owned by the library */

/*
 * robe_bias_create - a learned relative position bias: one learned number per head and bucket of
 * distances.  Of the S buckets of a side (S = num_buckets; half of it when two_sided) the first
 * E = floor(S / 2) hold one distance each, 0 .. E-1; bucket E + k, 0 <= k < L = S - E, begins at the
 * smallest distance n with n^L >= E^(L-k) max_distance^k (found in exact integers, no logarithm): equal
 * steps of the distance's logarithm from E to max_distance.  The last bucket takes all that is farther.  A
 * query at position p and a key at position j are r = j - p apart;
 *     one-sided   bucket(r) = that of max(-r, 0)      (later keys share bucket 0)
 *     two-sided   bucket(r) = that of |r|, + S for r > 0
 *   num_buckets   2 .. 128 one-sided; even, 4 .. 256, two-sided.
 *   max_distance  > E, < 2^30.
 * The handle is constant after creation: calls on one handle may overlap.
 */
int robe_bias_create(robe_bias_t* out, uint32_t num_buckets, uint32_t max_distance, int two_sided);
int robe_bias_destroy(robe_bias_t b);
/* robe_bias_num_buckets - num_buckets, or a negative robe_status. */
int robe_bias_num_buckets(robe_bias_t b);
/* robe_bias_get_edges - copy out the smallest distance |r| of each bucket (host pointer to num_buckets words; of a
 * bucket of later keys at least 1). */
int robe_bias_get_edges(robe_bias_t b, int64_t* edges);

/*
 * robe_bias_forward - out[n,h,i,j] = rows[bucket(j - (start_n + i)), h]
 *   rows      fp32 [num_buckets, heads], rows_ld apart: for instance the embeddings, d = heads, of the ids
 *             0 .. num_buckets-1 of one table, as robe_forward writes them (rows_ld = T*d).
 *   out       [batch, heads, q_len, k_len]: rows of k_len elements, out_ld apart.
 *   q_start   position of the first query of every sequence; q_starts, when not NULL, is a device pointer
 *             to batch positions, one per sequence (key j of every sequence stands at position j): one
 *             query each with q_starts = lengths - 1 is a decoding step.  Any value, negative ones too.
 *   causal    0, or 1: where the key is later than the query (r > 0) out is -infinity.
 *   q_len + k_len < 2^31;  batch < 2^31;  1 <= heads < 2^22.
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_UNSUPPORTED, ROBE_ERR_CUDA.
 */
int robe_bias_forward(robe_bias_t b, const float* rows, int64_t rows_ld, uint32_t heads, int64_t batch,
                      int64_t q_len, int64_t k_len, int64_t q_start, const int64_t* q_starts, int causal,
                      void* out, int64_t out_ld, int dtype, void* stream);

/*
 * robe_bias_backward - grad_rows[b,h] = sum of grad[n,h,i,j] over all n, i, j with bucket(j - (start_n + i)) = b
 * (and r <= 0 when causal: what stands in masked places has no effect, NaN included).
 *   grad        [batch, heads, q_len, k_len], rows grad_ld apart.
 *   grad_rows   fp32 [num_buckets, heads], grad_rows_ld apart, overwritten (+0 for an empty bucket): what
 *               robe_backward takes as grad_out.
 *   workspace   256-byte aligned, robe_bias_backward_workspace_bytes for these sizes (0 for bad arguments).
 * Errors: as above, and ROBE_ERR_WORKSPACE.
 */
size_t robe_bias_backward_workspace_bytes(robe_bias_t b, uint32_t heads, int64_t batch, int64_t q_len,
                                          int64_t k_len);
int robe_bias_backward(robe_bias_t b, const void* grad, int64_t grad_ld, uint32_t heads, int64_t batch,
                       int64_t q_len, int64_t k_len, int64_t q_start, const int64_t* q_starts, int causal,
                       int dtype, float* grad_rows, int64_t grad_rows_ld, void* workspace,
                       size_t workspace_bytes, void* stream);

#define ROBE_NORM_RMS 0   /* norm(v) = v / sqrt(mean(v^2) + eps)               */
#define ROBE_NORM_LAYER 1 /* norm(v) = (v - mean(v)) / sqrt(var(v) + eps)      */
#define ROBE_GATE_NONE 0   /* no gate (1)                                      */
#define ROBE_GATE_ROW 1    /* one number per row: gate is [rows, 1]            */
#define ROBE_GATE_VECTOR 2 /* [rows / gate_rows, d]: one vector for gate_rows rows in turn (1: a gate per element) */

/*
 * robe_residual_forward / robe_residual_backward - the join at which a block's output x enters the rows
 * again, norms before and after included:
 *     y      = norm(x) * w_post                        (x where w_post is NULL)
 *     out    = residual + scale * gate * dropout(y)    (residual NULL: nothing is added to)
 *     normed = norm(out) * w_pre                       (of out before its rounding; nothing where w_pre is NULL)
 * Dropout as in robe_dropout (row r, column c of x; p = 0: none).  A join with residual = NULL and
 * w_post = NULL is the entry of a model: dropout of looked-up rows and the norm before its first block.
 * out may be residual itself (same pointer, same ld).
 */
typedef struct robe_residual_t {
    int64_t rows, d;   /* rows >= 0, <= 2^32; 1 <= d <= 1048576 */
    int dtype;         /* of x, residual, gate, out, normed and their gradients; weights and their gradients are fp32 [d] */
    int norm;          /* ROBE_NORM_*, both norms */
    float eps, scale;  /* eps >= 0 */
    int gate;          /* ROBE_GATE_* */
    int64_t gate_rows; /* ROBE_GATE_VECTOR: divides rows; not looked at otherwise */
    float p;           /* in [0, 1] */
    uint64_t seed, offset;
    const uint64_t* step;
} robe_residual_t;
int robe_residual_forward(const robe_residual_t* c, const void* x, int64_t x_ld, const void* residual,
                          int64_t residual_ld, const void* gate, int64_t gate_ld, const float* w_post,
                          const float* w_pre, void* out, int64_t out_ld, void* normed, int64_t normed_ld,
                          void* stream);

/*
 * The gradients, from x, gate, out (as the forward call stored it; only looked at with w_pre) and the
 * gradients of out (NULL: zero) and normed (given exactly when w_pre is):
 *     t = grad_out + dnorm(out; grad_normed w_pre)     grad_residual = t         (NULL: not wanted)
 *     u = dropout(scale * gate * t)                    grad_x = dnorm(x; u w_post)   (u without w_post)
 *     grad_gate = sum of scale * dropout(y) * t over what a gate element was used for   (NULL: not wanted;
                    a dropped element adds +0, whatever t is there)
 *     grad_w_post = sum over rows of u norm(x)         grad_w_pre = sum over rows of grad_normed norm(out)
 * with dnorm(v; g) = rstd (g - [mean g] - n mean(g n)), n = norm(v), rstd its factor, [..] with layer norm.
 * grad_w_post and grad_w_pre are given exactly when their weights are; all outputs are overwritten (the
 * weights' gradients with +0 when rows is 0).  grad_residual may be grad_out itself (same pointer, same ld).
 *   gates      rows of the gate for ROBE_GATE_VECTOR, 0 otherwise
 *   workspace  256-byte aligned, robe_residual_backward_workspace_bytes(rows, d, gates)
 * Sums over rows are fp32 sums of at most 256 rows a thread, joined over at most 256 threads in fp32 and beyond in fp64.
 * Errors of both: ROBE_ERR_INVALID_ARG, ROBE_ERR_CUDA; of the backward also ROBE_ERR_WORKSPACE, ROBE_ERR_UNSUPPORTED.
 */
size_t robe_residual_backward_workspace_bytes(int64_t rows, int64_t d, int64_t gates);
int robe_residual_backward(const robe_residual_t* c, const void* grad_out, int64_t grad_out_ld,
                           const void* grad_normed, int64_t grad_normed_ld, const void* x, int64_t x_ld,
                           const void* out, int64_t out_ld, const void* gate, int64_t gate_ld,
                           const float* w_post, const float* w_pre, void* grad_x, int64_t grad_x_ld,
                           void* grad_residual, int64_t grad_residual_ld, void* grad_gate,
                           int64_t grad_gate_ld, float* grad_w_post, float* grad_w_pre, void* workspace,
                           size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Plain tables, as they stand beside the hashed array in a model: [vocab, d] rows of their own.
 */

/*
 * robe_table_forward - out[r,:] = scale * table[ids[r],:], +0 where ids[r] is not in 0 .. vocab-1 (a padding id of -1).
 *   table       fp32 or bf16 (table_dtype), rows table_ld apart;  out  fp32 or bf16 (out_dtype), whichever the table has.
 *   ids         device pointer to rows ids, ROBE_I64 or ROBE_I32 (index_type), aligned to their size.
 *   rows  >= 0, < 2^62;  0 <= vocab < 2^31;  1 <= d <= 1048576.
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_UNSUPPORTED, ROBE_ERR_CUDA.
 */
int robe_table_forward(const void* table, int64_t table_ld, int64_t vocab, int64_t d, int table_dtype, const void* ids,
                       int index_type, int64_t rows, float scale, void* out, int64_t out_ld, int out_dtype, void* stream);

/*
 * robe_table_backward - the gradient of a table: with S_v the sum of the rows of grad whose id is v, in fp32,
 *     accumulate 0    grad_table[v,:] = scale * S_v           (every row is written, +0 where no id is v)
 *     accumulate 1    grad_table[v,:] = fma(scale, S_v, grad_table[v,:])   (rows without an id keep their bits)
 * The second form also adds to what another use of the table has left (a tied output layer), and on an fp32 table itself, with
 * scale = -lr * (the forward's scale), it is the step of plain SGD.
 *   grad        [rows, d], fp32 or bf16 (dtype), grad_ld apart.
 *   skip        an id whose row gets no gradient (-1: none); ids outside the table never do.
 *   grad_table  fp32 [vocab, d], grad_table_ld apart.
 *   workspace   256-byte aligned, robe_table_backward_workspace_bytes(rows, vocab, d) (0 for bad arguments); the figure never falls
 *               as rows or d grows, so one for the largest call serves every smaller one.
 *   rows < 2^31.
 * A sum's order follows from the sizes and ids alone: fp32 sums of at most 256 rows in the order of the call, joined in fp64.
 * Errors: as above, and ROBE_ERR_WORKSPACE.
 */
size_t robe_table_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t d);
int robe_table_backward(const void* grad, int64_t grad_ld, int dtype, const void* ids, int index_type, int64_t rows,
                        float scale, int64_t skip, int accumulate, float* grad_table, int64_t grad_table_ld, int64_t vocab,
                        int64_t d, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Rows in 8 bits.  A row of d columns is codes, one byte each, and an fp32 scale for every `group` columns (the last group may be
 * shorter): what a code stands for is its own value times its group's scale.  With m the group's largest magnitude,
 *     scale = max(m, 2^-90) / Q,    code = round(v * (1 / scale))
 * where each operation is rounded to nearest even, in fp32 but for the last, so that codes and scales follow bit for
 * bit from the values.  ROBE_E4M3: Q = 448, codes are floats with four bits of exponent and three of fraction; ROBE_I8: Q = 127, whole
 * numbers.  A group that holds a NaN or an infinity reads back as NaN throughout.
 *   group   1 .. 256, or d (one scale a row; 0 means d).  Number of scales of a row: ceil(d / group).
 */
#define ROBE_E4M3 2
#define ROBE_I8 3

/*
 * robe_residual_quantize - robe_residual_forward without a norm of x, gate and dropout, whose `normed` leaves in 8 bits:
 *     out    = residual + scale * x              (residual NULL: nothing is added to; out NULL: not stored)
 *     normed = norm(out) * w_pre                 (of out before its rounding; w_pre NULL: out itself, no norm)
 *     codes, scales = normed in 8 bits
 * The gradient is robe_residual_backward's, from out as this call stored it, with the gradient of normed passed straight through
 * the rounding to codes.  out may be residual itself (same pointer, same ld).
 *   rows >= 0, <= 2^32;  1 <= d <= 1048576;  dtype  of x, residual and out;  norm  ROBE_NORM_*.
 *   codes   [rows, d] bytes, codes_ld apart;  scales  [rows, ceil(d / group)], scales_ld apart.
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_CUDA.
 */
int robe_residual_quantize(int64_t rows, int64_t d, int dtype, int norm, float eps, float scale, const void* x, int64_t x_ld,
                           const void* residual, int64_t residual_ld, const float* w_pre, void* out, int64_t out_ld, void* codes,
                           int64_t codes_ld, int code_type, int64_t group, float* scales, int64_t scales_ld, void* stream);

/*
 * A cache of rows in 8 bits, in pages of page_rows rows.  Row t of sequence s (t from 0) stands at position p = starts[s] + t and lies
 * in row p mod page_rows of page pages[s, floor(p / page_rows)]; it has no place where p is negative, beyond the page table, or
 * the page's number is not in 0 .. num_pages-1.  The call's rows are the sequences' one after the other: those of s
 * are offsets[s] .. offsets[s+1]-1 of them (offsets non-decreasing); without offsets every sequence has equally many.
 */
typedef struct robe_cache_t {
    void* codes;                      /* [num_pages, page_rows, d] bytes: rows codes_ld apart, pages codes_page */
    int64_t codes_ld, codes_page;
    float* scales;                    /* [num_pages, page_rows, ceil(d / group)] */
    int64_t scales_ld, scales_page;
    int64_t num_pages, page_rows;     /* < 2^31 each */
    int64_t d, group;                 /* as above */
    int code_type;                    /* ROBE_E4M3, ROBE_I8 */
    const int32_t* pages;             /* device [batch, max_pages], pages_ld apart */
    int64_t pages_ld, batch, max_pages;
    const int64_t* offsets;           /* device [batch + 1], or NULL */
    const int64_t* starts;            /* device [batch], or NULL: 0 */
} robe_cache_t;

/*
 * robe_cache_write - rows [n, d] into their places; rows without a place, before offsets[0] and from offsets[batch] on are
 * not written anywhere.  Two rows of a call with the same place (a page that two sequences write to) leave there some mixture
 * of the two: shared pages are for reading.
 * robe_cache_read  - the other way: out[r,:] = code * scale, +0 for a row without a place; rows before offsets[0] and from
 * offsets[batch] on are left as they were.
 *   rows / out   fp32 or bf16 (dtype), ld apart;  0 <= n <= 2^32 (a multiple of batch where offsets is NULL).
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_UNSUPPORTED, ROBE_ERR_CUDA.
 */
int robe_cache_write(const robe_cache_t* c, const void* rows, int64_t rows_ld, int64_t n, int dtype, void* stream);
int robe_cache_read(const robe_cache_t* c, void* out, int64_t out_ld, int64_t n, int dtype, void* stream);

/*
 * robe_cache_attention - attention of one new token of each sequence over its rows in two such caches.  The query of sequence s stands
 * at position starts[s] (its own key and value have been written there); query head h reads head h / (q_heads / heads) of the cache, which
 * is columns head * dim .. of a row:
 *     x_j = scale * q[s,h,:] . K_j + (bias ? bias_rows[bucket(j - starts[s]), h] : 0)      0 <= j <= starts[s]
 *     out[s,h,:] = sum_j exp(x_j) V_j / sum_j exp(x_j)
 * over the positions that have a place; +0 where there is none (starts[s] < 0, say).  bucket as in robe_bias_forward.
 *   keys, values   caches with the same code type, pages, sizes and strides; group = dim, d = heads * dim; offsets NULL;
 *                  codes 16-byte aligned (pointer, codes_ld and codes_page); scales as robe_cache_write leaves them.
 *   q, out         bf16 [batch, q_heads, dim]: heads ld apart, sequences seq (columns of a row that holds keys and values too, say).  dim 32,
 *                  64, 96, 128 or 256; heads divides q_heads.
 *   bias           handle or NULL;  bias_rows  fp32 [num_buckets, q_heads], bias_ld apart.
 *   workspace      256-byte aligned, robe_cache_attention_workspace_bytes(batch, heads, q_heads, dim, max_pages * page_rows)
 *                  bytes (0 for bad arguments); one call at a time.
 *   max_pages * page_rows < 2^31 - 2^16;  batch * q_heads < 2^31;  codes of a cache within 64 GB, scales within 16 (ROBE_ERR_UNSUPPORTED).
 * Scores, the divisor and the sums are fp32.  Weights are rounded to fp16 with their value's scale in them: with c_j = exp(x_j) times
 * V_j's scale and c the largest of a span's, c_j is off by at most 2^-11 of itself from 2^-14 c on and by at most 2^-25 c below,
 * so that a key of at most 2^-25 c adds nothing to the sum, while the divisor, in fp32, counts it.  A result is off by that times codes: small
 * next to the largest contribution to its row, not next to a column's own sum where the keys of large c_j have a code of 0 there.
 * How the sum over a sequence is cut follows from all lengths of the call; the same call gives the same bits.
 * Errors: ROBE_ERR_INVALID_ARG, ROBE_ERR_WORKSPACE, ROBE_ERR_UNSUPPORTED, ROBE_ERR_CUDA.
 */
size_t robe_cache_attention_workspace_bytes(int64_t batch, int64_t heads, int64_t q_heads, int64_t dim, int64_t positions);
int robe_cache_attention(const robe_cache_t* keys, const robe_cache_t* values, const void* q, int64_t q_ld, int64_t q_seq, int64_t q_heads,
                         float scale, robe_bias_t bias, const float* bias_rows, int64_t bias_ld, void* out, int64_t out_ld,
                         int64_t out_seq, void* workspace, size_t workspace_bytes, void* stream);

/* robe_status_string - static host string for a robe_status value. */
const char* robe_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* ROBE_H_ */
