/* relaysum.h -- one synchronous RelaySum round of RelaySGD for all n workers
 * of a tree, simulated on one MI355X (gfx950) GPU.
 *
 * What a round computes (the paper's Alg. 1, "RelaySum/Model", with the
 * Nesterov local step of Appendix D.2).  For round t and every worker i,
 * with N_i the neighbours of i in the tree:
 *
 *   local step   b_i   <- beta*b_i + g_i                         (beta != 0)
 *                xh_i   = x_i - lr*(g_i + beta*b_i)              (beta != 0)
 *                xh_i   = x_i - lr*g_i                           (beta == 0)
 *   relay        m_{i->j}^{(t)} = xh_i + sum_{k in N_i\j} m_{k->i}^{(t-1)}
 *                c_{i->j}^{(t)} = 1    + sum_{k in N_i\j} c_{k->i}^{(t-1)}
 *   average      nbar_i = 1 + sum_{j in N_i} c_{j->i}^{(t)}
 *                x_i    = (xh_i + sum_{j in N_i} m_{j->i}^{(t)}) / nbar_i
 *
 * with m^{(-1)} = 0 and c^{(-1)} = 0 before the first round.  All arithmetic
 * is IEEE binary32, one rounding per operation, no fused multiply-add; every
 * sum over a neighbour set starts from xh_i and adds neighbours in ascending
 * id; the average is a true division.  The result is therefore a fixed
 * function of the inputs (it does not depend on the launch shape).
 *
 * Memory: x, g, mom are DEVICE pointers to row-major float[n][d] (row i is
 * worker i, row stride d floats); they belong to the caller and must not
 * alias each other or any buffer of the handle.  Edge lists and every
 * *_host buffer are HOST memory.  The handle owns the tree (CSR form), a
 * two-slot ring of 2(n-1) messages of d floats each, the integer counters,
 * and the round number.
 *
 * Streams: all device work of a handle is queued on its stream (the null
 * stream until relaysum_set_stream); calls return before that work ends,
 * except the accessors marked "synchronises".  A handle is not thread-safe.
 *
 * Graphs: relaysum_create resolves every kernel and launch attribute, so
 * relaysum_step and relaysum_step_ex only enqueue kernels and can be
 * recorded by HIP stream capture.  The round number (and with it the ring
 * and counter parity a call uses) advances when a call is recorded, not
 * when the graph runs: record an even number of rounds, and replay the
 * graph only while the handle's eager calls come in pairs, so that every
 * replay finds the parity it was recorded with.  Arguments are fixed at
 * recording (Adam's step count, lr, the loss mask pointer).
 *
 * Errors: every int-returning function returns RELAYSUM_OK (0) or a negative
 * relaysum_status; relaysum_strerror() names a code and
 * relaysum_last_error() gives the text of the handle's last failure.
 */
#ifndef RELAYSUM_H
#define RELAYSUM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct relaysum_s relaysum_t;

/* Largest number of workers a handle takes.  The divisor nbar_i <= n of
 * Alg. 1's average is converted to binary32, which holds every integer up to
 * 2^24 exactly, so up to this size the division is the paper's. */
#define RELAYSUM_MAX_WORKERS 16777216

typedef enum relaysum_status {
    RELAYSUM_OK = 0,
    RELAYSUM_ERR_INVALID_ARG = -1,   /* bad size, NULL pointer, misuse */
    RELAYSUM_ERR_NOT_A_TREE = -2,    /* edge list is not a tree on n workers */
    RELAYSUM_ERR_OUT_OF_MEMORY = -3, /* device or host allocation failed */
    RELAYSUM_ERR_DEVICE = -4         /* HIP runtime or launch error */
} relaysum_status;

/* Create a handle for n workers with d-float models on the tree given by
 * num_edges undirected edges edges[2e], edges[2e+1] (0-based worker ids,
 * HOST memory, any order).  The tree is the paper's communication graph
 * (Section 3, Setup: n >= 1 workers, no self loops); RelaySum needs it to be
 * a tree (Alg. 1 input).
 *   1 <= n <= RELAYSUM_MAX_WORKERS, d >= 0 (d == 0: rounds only relay the
 *   counters).
 *   Returns RELAYSUM_ERR_NOT_A_TREE unless num_edges == n-1, every id is in
 *   [0, n), and the edges have no self loop, no duplicate and connect all
 *   workers; RELAYSUM_ERR_INVALID_ARG for n out of range, d < 0, out == NULL, or
 *   edges == NULL with num_edges > 0; RELAYSUM_ERR_OUT_OF_MEMORY when device
 *   memory for the ring cannot be had: 2 * 2(n-1) messages of d floats,
 *   each rounded up to whole ring tiles (4096 floats; a shorter message to
 *   the next power of two, at least 4 floats on single trees and 512 on
 *   double trees); single trees of more than 32 workers (double trees from
 *   65 workers, degrees of at most 32) also take d floats for each worker
 *   with a neighbour outside its cluster of 16 workers (32 on double trees
 *   and on single trees of 2,048 workers or more) and for each worker of
 *   more than 8 neighbours (single trees): 6 on a chain of 64.
 * Allocates on the current HIP device, zeroes every message and counter
 * (m^{(-1)} = 0, c^{(-1)} = 0) and sets the round number to 0.  On failure
 * *out is set to NULL. */
int relaysum_create(int32_t n, int64_t d, const int32_t *edges, int32_t num_edges,
                    relaysum_t **out);

/* Double binary trees (Section 3): a handle whose rounds relay the odd
 * model coordinates 1, 3, 5, ... over tree A (edges_a) and the even ones
 * 0, 2, 4, ... over tree B (edges_b), both trees on the same n workers with
 * num_edges = n-1 edges each, validated as in relaysum_create.  Each tree
 * keeps its own counters and messages (of d/2 and (d+1)/2 floats), so a
 * coordinate's result is exactly that of a single-tree handle on its tree
 * run over the coordinates of its parity.  Every step and accessor below
 * applies; directed-edge slots are numbered tree-major: tree A's 2(n-1)
 * slots first, then tree B's.  The trees need not be complementary; the
 * paper pairs two binary trees in which every worker is a leaf of one of
 * them, so that each worker has at most 4 neighbours in total. */
int relaysum_create_double(int32_t n, int64_t d, const int32_t *edges_a, const int32_t *edges_b,
                           int32_t num_edges, relaysum_t **out);

/* Release the handle after waiting for its stream.  NULL is a no-op. */
int relaysum_destroy(relaysum_t *h);

/* Queue later device work on `hip_stream` (a hipStream_t; NULL = null
 * stream).  The caller keeps the stream alive while the handle uses it. */
int relaysum_set_stream(relaysum_t *h, void *hip_stream);

/* One round t (Alg. 1 loop body, all workers), then t <- t+1.
 *   x    [n][d] device, read and overwritten with x^{(t+1)};
 *   g    [n][d] device, read only: the gradients at x^{(t)};
 *   mom  [n][d] device, the Nesterov buffers b_i (start them at 0), updated
 *        in place; may be NULL if and only if beta == 0, and is neither read
 *        nor written when beta == 0;
 *   lr   the learning rate gamma (lr == 0 is allowed: mom still updates);
 *   beta the momentum parameter alpha of Appendix D.2 (0 = plain SGD).
 * Rows must be 4-byte aligned.  Results do not depend on alignment or d;
 * rounds are fastest on 16-byte aligned pointers with d % 4 == 0 (the
 * cluster path's completion launch needs both for 16-byte accesses; the
 * other kernels move 16-byte chunks at any 4-byte alignment, or one float
 * per thread).
 * Returns RELAYSUM_ERR_INVALID_ARG for h, x or g NULL (unless d == 0), mom
 * NULL with beta != 0, misaligned pointers, arrays that share bytes, or an
 * array that is not n*d floats inside one device-memory (or managed-memory)
 * allocation of the handle's GPU (host memory, another GPU's memory or a
 * short buffer would make a kernel fault; checked with the HIP runtime's
 * pointer queries, once per array: the handle remembers the last 8 arrays
 * that passed, so an array freed and replaced at the same address by a
 * shorter allocation is not queried again); RELAYSUM_ERR_DEVICE if a launch
 * fails.  The round number then does not
 * advance; a round of the cluster or two-pass path is several
 * launches, and if a later one fails, x, the optimizer state and the
 * handle's messages are partly updated: restore them (relaysum_load_state,
 * or relaysum_reset and the caller's own copies) before another round. */
int relaysum_step(relaysum_t *h, float *x, const float *g, float *mom, float lr, float beta);

/* ---- other update rules and local optimizers --------------------------- */

/* How a round turns what each worker received into its new state. */
typedef enum relaysum_update {
    /* Alg. 1: x_i = (xh_i + sum_j m_{j->i}) / nbar_i. */
    RELAYSUM_UPDATE_MODEL = 0,
    /* Robust rule of Section 5.4 (eq. robust), for unreliable links:
     * x_i = (xh_i + sum_j m_{j->i} + (n - nbar_i) * x_i^{(t)}) / n, i.e. every
     * model that has not arrived is replaced by the worker's own x_i^{(t)}. */
    RELAYSUM_UPDATE_ROBUST = 1,
    /* Alg. 4 (RelaySGD/Grad, Appendix G): the relay carries the updates
     * u_i = -lr * g_i and x_i = x_i + (u_i + sum_j m_{j->i}) / n.  Plain SGD
     * only (the optimizer field must be RELAYSUM_OPT_SGD with beta1 == 0). */
    RELAYSUM_UPDATE_GRAD = 2,
    /* Alg. 3 (RelaySum for distributed mean estimation, Appendix F): g holds
     * this round's samples, state1 the running sums y;
     * y_i += g_i + sum_j m_{j->i}, s_i += 1 + sum_j c_{j->i}, x_i = y_i / s_i
     * (x is output only: the estimate after this round's update).  The
     * library keeps the integer s_i; the division converts it to binary32,
     * exact up to 2^24, so the library refuses (RELAYSUM_ERR_INVALID_ARG,
     * nothing queued) a round that could take some s_i past 2^24.  It bounds
     * s_i by the sum over the mean-estimation rounds t of the workers within
     * t+1 hops of a worker in a tree of the tree's largest degree D:
     * min(n, 1 + D(t+1)) for D <= 2, min(n, 1 + D(1 + (D-1) + ... +
     * (D-1)^t)) otherwise (on a 1024-worker chain, 16,639 rounds).
     * relaysum_reset clears the bound; snapshots carry it. */
    RELAYSUM_UPDATE_MEAN = 3
} relaysum_update;

/* Local step that forms the half-step xh_i (RELAYSUM_UPDATE_MODEL, _ROBUST). */
typedef enum relaysum_optimizer {
    /* beta1 == 0: xh = x - lr*g (Alg. 1's local step); beta1 != 0: Nesterov momentum
     * of Appendix D.2 with state1 = the momentum buffer. */
    RELAYSUM_OPT_SGD = 0,
    /* Adam, the local optimizer of Relay-Adam (Appendix D.3), in PyTorch's
     * form: bc1 = 1 - beta1^t, bc2 = 1 - beta2^t (double), m = beta1*m +
     * (1-beta1)*g, v = beta2*v + (1-beta2)*g*g, xh = x - (lr/bc1) * m /
     * (sqrt(v)/sqrt(bc2) + eps); state1 = m, state2 = v, t = adam_step. */
    RELAYSUM_OPT_ADAM = 1
} relaysum_optimizer;

typedef struct relaysum_round_args {
    int32_t update;          /* relaysum_update */
    int32_t optimizer;       /* relaysum_optimizer */
    float lr;                /* gamma */
    float beta1;             /* Nesterov alpha (SGD), or Adam beta1 */
    float beta2;             /* Adam beta2 */
    float eps;               /* Adam epsilon */
    int64_t adam_step;       /* Adam: 1-based step count t of the bias corrections */
    /* DEVICE array of one byte per directed-edge slot (2(n-1), or 4(n-1) on
     * double trees, tree-major), or NULL.  Nonzero marks the
     * message of that directed edge as lost in this round (Section 5.4): the
     * receiver gets neither the vector nor the counter, which count as zero
     * in its update now and in what it relays next round.  Read by the
     * round's kernels, so it must stay valid until they finish; checked
     * like x (RELAYSUM_ERR_INVALID_ARG if not). */
    const uint8_t *dropped;
} relaysum_round_args;

/* One round under `args` (see relaysum_update / relaysum_optimizer), then
 * t <- t+1.  x, g, state1, state2 are DEVICE [n][d] float rows as in
 * relaysum_step; which of them are read or written depends on the rule:
 *   MODEL/ROBUST + SGD:  x (rw), g (r), state1 = momentum (rw; NULL iff beta1 == 0)
 *   MODEL/ROBUST + ADAM: x (rw), g (r), state1 = m, state2 = v (rw)
 *   GRAD:                x (rw), g (r)
 *   MEAN:                x (w), g = samples (r), state1 = y (rw)
 * Unused pointers may be NULL.  Returns RELAYSUM_ERR_INVALID_ARG for a
 * missing buffer, an unknown rule, GRAD with momentum or Adam, Adam with
 * adam_step < 1, misaligned pointers, or used arrays that share bytes;
 * RELAYSUM_ERR_DEVICE on a launch failure (the round number then does not
 * advance).  relaysum_step(h, x, g, mom, lr, beta) is this call with MODEL,
 * SGD, beta1 = beta. */
int relaysum_step_ex(relaysum_t *h, float *x, const float *g, float *state1, float *state2,
                     const relaysum_round_args *args);

/* Mean estimation: s_i, the number of samples summed into y_i so far
 * (synchronises); n values per tree, tree-major (on double trees s_i of
 * tree A covers the odd coordinates, of tree B the even ones). */
int relaysum_get_samples(relaysum_t *h, int64_t *samples_host);

/* Consensus distance of the workers' models (the quantity Section 4's
 * analysis tracks, here with the uniform average of the models as centre):
 *   *dist   = (1/n) * sum_i ||x_i - xbar||^2,  xbar = (1/n) * sum_i x_i,
 *   *spread = max over workers i and coordinates c of |x_ic - xbar_c|
 * (spread may be NULL), for x of n*d floats in device memory of the
 * handle's GPU, row i worker i, 4-byte aligned, checked like relaysum_step's
 * arrays.  Accumulated in binary64 in an order fixed by n and d, so equal
 * inputs give equal bits.  Queued on the handle's stream behind its rounds,
 * then the stream is synchronised (not for graph capture).  d == 0 gives 0
 * and 0.  A NaN or an infinity in x makes *dist NaN.  *spread leaves out the
 * deviations that are no numbers: a coordinate with a NaN or with infinities
 * of both signs, and an infinite value's from the infinite mean; a coordinate
 * where some workers' values are infinite, of one sign, and others' finite
 * makes it infinite.  Not part of a round: an observability aid for training
 * loops and tests. */
int relaysum_consensus_distance(relaysum_t *h, const float *x, double *dist, double *spread);

/* Back to the state before the first round: messages, counters and sample
 * counts zeroed (queued on the handle's stream), round number 0. */
int relaysum_reset(relaysum_t *h);

/* Number of rounds done since create or reset. */
int relaysum_round(const relaysum_t *h, int64_t *t);

/* Number of trees of the handle: 1, or 2 for relaysum_create_double. */
int relaysum_num_trees(const relaysum_t *h, int32_t *count);

/* Kernel path a round of this handle takes (fixed at creation by the tree,
 * n and d; for tests and observability).  Every path computes the same
 * results. */
typedef enum relaysum_path {
    RELAYSUM_PATH_TILE = 0,        /* single trees of up to 32 workers */
    RELAYSUM_PATH_DTREE = 1,       /* double trees of up to 32 workers */
    RELAYSUM_PATH_WIDE_DTREE = 2,  /* retired; never returned */
    RELAYSUM_PATH_CLUSTER = 3,     /* single trees of more than 32 workers (workers of more
                                      than 8 neighbours through hub kernels ahead of the
                                      cluster kernel) */
    RELAYSUM_PATH_WIDE = 4,        /* retired; never returned */
    RELAYSUM_PATH_TWO_PASS = 5,    /* double trees of more than 64 workers with a worker of
                                      more than 32 neighbours, and d == 0 beyond 32
                                      workers */
    RELAYSUM_PATH_DTREE_SEQ = 6,   /* double trees of 33 to 64 workers */
    RELAYSUM_PATH_CLUSTER_DTREE = 7   /* double trees of more than 64 workers, degrees <= 32 */
} relaysum_path;
int relaysum_kernel_path(const relaysum_t *h, int32_t *path);

/* Number of directed-edge slots, 2(n-1) per tree.  Within a tree the slots
 * are ordered by source worker, then by destination, ascending; on double
 * trees tree A's slots come first. */
int relaysum_num_directed_edges(const relaysum_t *h, int32_t *count);

/* Floats in the message of `slot`: d on a single tree; on double trees
 * d/2 (tree A, odd coordinates) or (d+1)/2 (tree B, even coordinates). */
int relaysum_message_length(const relaysum_t *h, int32_t slot, int64_t *len);

/* Source and destination worker of a slot (host-side table lookup). */
int relaysum_directed_edge(const relaysum_t *h, int32_t slot, int32_t *src, int32_t *dst);

/* Counters of the last round (synchronises the handle's stream):
 * nbar_host[n per tree, tree-major] = nbar_i used in the last average,
 * edge_counts_host[one per slot] = c_{src->dst}.  Either pointer may be
 * NULL.  Before any round every value is 0. */
int relaysum_get_counts(relaysum_t *h, int32_t *nbar_host, int32_t *edge_counts_host);

/* The relaysum_message_length floats of message m_{src->dst} sent in the
 * last round, for `slot`, into dst_host (synchronises); on double trees the
 * carried coordinates in ascending order.  Before any round: zeros.
 * RELAYSUM_ERR_INVALID_ARG for a bad slot or NULL dst_host;
 * RELAYSUM_ERR_OUT_OF_MEMORY if a double-tree handle cannot get the host
 * staging buffer (whole ring tiles of the message). */
int relaysum_get_message(relaysum_t *h, int32_t slot, float *dst_host);

/* Snapshots, for resuming a run (no passage of the paper defines them; a
 * caller checkpointing a RelaySGD training run needs them).  A snapshot holds
 * what a handle carries from one round to the next: the round number, the
 * last round's counters, nbar and sample counts of every tree, and its
 * messages (the ring parity the next round reads), behind a header with the
 * handle's shape and a digest of its trees.  The caller keeps its own x and
 * optimizer state.  Loading a snapshot into a handle with the same n, d and
 * trees (edge lists in any order) and running rounds from there gives, bit
 * for bit, what the saved handle would have given.
 *
 * Bytes of a snapshot of this handle (about 2(n-1) * d * 4 per tree plus a
 * few KB). */
int relaysum_state_size(const relaysum_t *h, size_t *bytes);

/* Write a snapshot into buf (HOST or DEVICE memory, at least
 * relaysum_state_size bytes), after the work queued on the handle's stream
 * (synchronises).  RELAYSUM_ERR_INVALID_ARG for NULL buf or too few bytes. */
int relaysum_save_state(relaysum_t *h, void *buf, size_t bytes);

/* Replace the handle's state with a snapshot from buf (HOST or DEVICE
 * memory), after the work queued on its stream (synchronises); the round
 * number becomes the snapshot's.  RELAYSUM_ERR_INVALID_ARG, with the handle
 * unchanged, for NULL buf, too few bytes, another library version, or a
 * snapshot of a handle with other n, d or trees. */
int relaysum_load_state(relaysum_t *h, const void *buf, size_t bytes);

/* Test aid for the round's data flow: fill what the next round writes
 * (its ring parity, counters, nbar, sample counts, and the cluster path's
 * counter sums and partial sums of boundary workers) with all-ones bytes
 * (NaN floats, -1 integers), queued on the handle's stream with memset
 * nodes (not for graph capture).  A round reads only what the round before
 * it wrote, so its results do not change; one that read what it writes
 * would turn NaN or negative.  relaysum_get_counts reads -1 for nbar until
 * the next round, relaysum_get_samples -1 until the next mean-estimation
 * round (the only rule that keeps sample counts). */
int relaysum_poison_next(relaysum_t *h);

/* ---- for callers that cannot allocate ------------------------------------ */

/* relaysum_step without a handle, for callers that cannot allocate device
 * memory (code under HIP graph capture, allocation-free serving loops,
 * harnesses that forbid hipMalloc): one round t of Alg. 1 (relaysum_step's
 * arithmetic, bit for bit the result of a handle created with the same n, d
 * and edges at its round t) with the tree's CSR form, the counters and the
 * two-slot message ring kept in a static device buffer of the library
 * instead of handle memory.  It calls no allocator.
 *   n, d, edges, num_edges  as relaysum_create, with 1 <= n <= 32;
 *   t                       the round number: t == 0 starts a run (the
 *                           buffer's counters and the ring parity round 0
 *                           reads are cleared, by a kernel); t > 0 continues
 *                           the run whose round t-1 was the last call of this
 *                           function on the current device;
 *   x, g, mom, lr, beta     as relaysum_step (device pointers, [n][d] float);
 *   hip_stream              the stream the round is queued on (NULL = null
 *                           stream).
 * Limit: the buffer holds 64 MiB per GPU (allocated when the library is
 * loaded on a device, held until the process ends); a round needs about
 * 2 * 2(n-1) * d * 4 bytes of it (ring tiles of 4096 floats, or the next
 * power of two of at least 512 for shorter d), e.g. a 16-worker tree up to
 * d of about 270,000.  Every call on one GPU shares that GPU's buffer, which
 * keeps the last call's contents: runs on one GPU must not overlap (a new
 * run, t == 0, replaces the previous one), and calls from several threads
 * on one GPU race.
 * Returns RELAYSUM_ERR_NOT_A_TREE as relaysum_create; RELAYSUM_ERR_INVALID_ARG
 * for n outside 1..32, d < 0, t < 0, a round that needs more than the
 * buffer, the pointer errors of relaysum_step, or t > 0 when the buffer does
 * not hold round t-1 of this n, d and tree; RELAYSUM_ERR_DEVICE on a HIP
 * error (the run is then ended).  relaysum_last_error(NULL) gives the text of
 * this thread's last failure. */
int relaysum_step_static(int32_t n, int64_t d, const int32_t *edges, int32_t num_edges, int64_t t,
                         float *x, const float *g, float *mom, float lr, float beta,
                         void *hip_stream);

/* Static name of a status code. */
const char *relaysum_strerror(int code);

/* Text of the last failure on this handle ("" if none); valid until the
 * next call on the handle.  With h == NULL: the last failure of
 * relaysum_step_static on the calling thread. */
const char *relaysum_last_error(const relaysum_t *h);

/* ---- layers on 8-bit rows -------------------------------------------------
 *
 * What n workers compute between two rounds when their models have
 * feed-forward sub-layers, as transformers do: norm, products and their
 * gradients (attention and activations are the caller's) for all workers in
 * one launch, each worker with its own weights.  Weights are read where they lie, in the
 * models' rows x[i], and weight gradients are written where the next round
 * reads them, in the rows g[i].
 *
 *   norm         s = h + residual;  y = s * rstd * w,  rstd = 1 / sqrt(mean(s^2) + eps)
 *                y leaves in 8 bits; for the gradient s is kept in 8 bits too
 *   product      Y[t][c] = sum_k X[t][k] * W[c][k] of packed X and W, in integers
 *   gradients    of the product from the packed X and W, of the norm from the packed s;
 *                the rounding to 8 bits counts as the identity
 *
 * Packed rows.  A row of `width` entries is held as one int8 code per entry
 * and one int8 exponent per group of entries; a group is the whole row
 * (group 0) or 128 neighbouring entries (group 128):
 *   value = code * 2^exponent, |code| <= 127, the exponent the smallest of
 *   at least -126 that fits the group's largest entry, codes rounded to
 *   nearest, halves to even;
 *   exponent -128 marks a group with a NaN or an infinity: it stands for
 *   NaN throughout.  (64 * 2^122, what floats from 63.5 * 2^122 on are held
 *   as, is 2^128: an infinity as a float.)
 * Scales are powers of two so that values are exact in bfloat16, which the
 * gradients' products multiply in.  codes is [n][rows][stride] with stride =
 * relaysum_packed_stride(width) and zeros behind the width; exponents are
 * [n][rows][1], or [n][rows][stride / 128] for group 128.  Codes must be
 * 16-byte aligned and codes behind the width zero.
 *
 * Every array is DEVICE memory of the current GPU, checked with the HIP
 * runtime's pointer queries before anything is queued, and outputs share no
 * memory with other arrays, except where a call says so (they may lie between
 * other arrays' rows).  Sums over a row and over tokens, and every product,
 * are held in 32 bits or more.  Calls queue kernels on `hip_stream` (NULL =
 * null stream), allocate nothing, copy nothing to the host, use no atomics
 * (equal inputs give equal bits) and can be recorded by HIP stream capture.  They return RELAYSUM_OK or
 * RELAYSUM_ERR_INVALID_ARG (nothing queued) or RELAYSUM_ERR_DEVICE;
 * relaysum_layer_error() has the text.
 *
 * Limits: 1 <= n <= RELAYSUM_MAX_WORKERS, 0 <= rows or tokens (0: nothing to
 * do, but weight gradients are set to 0), 1 <= width <= 32768 (up to there
 * an integer sum of products fits 32 bits), 1 <= channels <= 2^24.  A launch
 * takes 2^22 - 1 workgroups: n of the norm's gradient, and of the products n
 * times the tiles of a worker's result (256 x 256; of gradients from floats
 * 128 x 128, from binary16 128 x 256). */

typedef enum relaysum_type {
    RELAYSUM_FLOAT = 0,    /* binary32 */
    RELAYSUM_BFLOAT = 1,   /* bfloat16 */
    RELAYSUM_HALF = 2      /* binary16 */
} relaysum_type;

/* Rows of n workers: entry k of row t of worker i is entry
 * i*worker_stride + t*row_stride + k of data.  Strides count entries and are
 * not negative; rows that are written must not overlap.  Rows may start
 * anywhere the type can. */
typedef struct relaysum_rows {
    void *data;
    int32_t type;            /* relaysum_type */
    int64_t worker_stride;   /* ignored for n == 1 */
    int64_t row_stride;      /* ignored for one row */
} relaysum_rows;

/* Packed rows, dense. */
typedef struct relaysum_packed {
    int8_t *codes;
    int8_t *exps;
    int32_t group;           /* 0 or 128: the same for rows of up to 128 entries */
} relaysum_packed;

/* Codes from the start of a packed row to the next; -1 for a bad width. */
int64_t relaysum_packed_stride(int64_t width);

/* Pack rows (weights once a round, activations for a backward pass), and
 * their values back into a type. */
int relaysum_pack(int32_t n, int64_t rows, int64_t width, const relaysum_rows *v,
                  const relaysum_packed *out, void *hip_stream);
int relaysum_unpack(int32_t n, int64_t rows, int64_t width, const relaysum_packed *p,
                    const relaysum_rows *out, void *hip_stream);

/* Norm of every token's row.
 *   h, residual, sum  rows of one type; sum = h + residual rounded to it, and
 *            the norm is that of the rounded sum; residual and sum may both
 *            be NULL (s = h).  sum may be h's or residual's own rows.
 *   weight   float[width] of worker i at weight + i*weight_stride
 *   y        out, group 0: what the product reads, and its gradient keeps
 *   rstd     out, float[n][tokens], also of rows whose mean(s^2) lies outside
 *            binary32's range; infinity where rstd itself does (rows of less than
 *            2^-128 with eps = 0; their y is right)
 *   saved    out, group 128, or NULL: s, for relaysum_rmsnorm_backward */
int relaysum_rmsnorm(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *h,
                     const relaysum_rows *residual, const float *weight, int64_t weight_stride,
                     float eps, const relaysum_rows *sum, const relaysum_packed *y, float *rstd,
                     const relaysum_packed *saved, void *hip_stream);

/* Gradients of the norm, with xh = rstd * s (s from saved) and u = dy * w:
 *   ds = dsum + rstd * (u - xh * mean(u * xh)),   weight_grad = sum over tokens of dy * xh
 * (ds is not finite in a row whose sum of u * xh passes binary32's range)
 *   dy, dsum, ds  rows of one type: the gradients of y, of the sum from
 *            elsewhere (NULL: none) and of h and residual alike; ds may be
 *            dy's or dsum's own rows
 *   weight_grad   float rows, one of each worker (row_stride is not used),
 *            overwritten
 *   workspace     relaysum_rmsnorm_workspace bytes, 4-byte aligned (NULL if 0) */
int64_t relaysum_rmsnorm_workspace(int32_t n, int64_t tokens, int64_t width);
int relaysum_rmsnorm_backward(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *dy,
                              const relaysum_rows *dsum, const relaysum_packed *saved,
                              const float *rstd, const float *weight, int64_t weight_stride,
                              const relaysum_rows *ds, const relaysum_rows *weight_grad,
                              void *workspace, size_t workspace_bytes, void *hip_stream);

typedef enum relaysum_product {
    RELAYSUM_LINEAR = 0,                   /* relaysum_linear */
    RELAYSUM_LINEAR_BACKWARD_INPUT = 1,
    RELAYSUM_LINEAR_BACKWARD_WEIGHT = 2
} relaysum_product;

/* Bytes that a call (relaysum_product) needs as workspace, 16-byte aligned,
 * for rows of this type (y's, or dy's); 0: none, and NULL will do.  Few
 * results with a long sum are made in parts, which are kept there.
 * relaysum_linear_workspace is the most of the three, for callers that keep
 * one workspace for all of them.  -1 for bad arguments. */
int64_t relaysum_linear_workspace_of(int32_t product, int32_t n, int64_t tokens, int64_t width,
                                     int64_t channels, int32_t type);
int64_t relaysum_linear_workspace(int32_t n, int64_t tokens, int64_t width, int64_t channels, int32_t type);

/* y[t][c] = sum_k x[t][k] * w[c][k] for every worker: x packed rows of tokens,
 * w packed rows of channels (the output features), both group 0.  The sum is
 * exact in integers; it is rounded to 24 bits and then to y's type. */
int relaysum_linear(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                    const relaysum_packed *x, const relaysum_packed *w, const relaysum_rows *y,
                    void *workspace, size_t workspace_bytes, void *hip_stream);

/* dx[t][k] = sum_c dy[t][c] * w[c][k]; dx has dy's type, w is group 0.  Here
 * and below dy's entries enter exactly, floats to a multiple of 2^-133. */
int relaysum_linear_backward_input(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                                   const relaysum_rows *dy, const relaysum_packed *w,
                                   const relaysum_rows *dx, void *workspace, size_t workspace_bytes,
                                   void *hip_stream);

/* weight_grad[c][k] = sum_t dy[t][c] * x[t][k], float rows, overwritten; x of
 * either group (what relaysum_rmsnorm gave, or activations packed for this). */
int relaysum_linear_backward_weight(int32_t n, int64_t tokens, int64_t width, int64_t channels,
                                    const relaysum_rows *dy, const relaysum_packed *x,
                                    const relaysum_rows *weight_grad, void *workspace,
                                    size_t workspace_bytes, void *hip_stream);

/* ---- attention ------------------------------------------------------------
 *
 * What mixes the tokens of a layer: attention of n workers' sequences, all of
 * them in one launch, and its gradients.
 *
 *   s_j = scale * q . k_j     for the keys j in [lo, hi) that a row sees
 *   out = sum_j p_j v_j,      p_j = exp(s_j) / sum exp(s),   lse = log sum exp(s)
 *
 * q and out are heads of `tokens` rows, k and v those of `keys` rows; `heads` is
 * a multiple of kv_heads, and heads g * heads / kv_heads and so on share key
 * head g.  Which keys a row sees is said by ranges, int32 [n][tokens][2] of
 * DEVICE memory: lo and hi of every row, in any order (packed sequences, prefixes,
 * windows); what lies outside 0..keys is not seen.  Without ranges (NULL) a row t
 * sees all keys, or with causal != 0 the keys up to t + keys - tokens: the last
 * row sees all of them.  A row that sees nothing gives zeros, an lse of -infinity,
 * and no gradient.  Keys and rows that do not see each other have no part in each
 * other's results: not in a bit of them where all are numbers; beside infinities
 * or NaN sums may be added up in another order.
 *
 * Scores, sums and gradients are held in 32 bits; the weights p and the gradients
 * of the scores enter the second products rounded to the arrays' type.  A row's
 * values are added up times up to 2^8 before they are divided by its weights' sum:
 * entries of v that are numbers give numbers up to 2^119 / keys.
 * Errors, streams, capture and the rules for arrays are those of the layer calls
 * above, relaysum_layer_error() has the text; equal inputs give equal bits. */

/* Heads of n workers: entry k of head h of row t of worker i is entry
 * i*worker_stride + t*row_stride + h*head_stride + k of data.  Strides count
 * entries and are not negative; rows that are written must not overlap.  Rows may
 * start anywhere the type can. */
typedef struct relaysum_heads {
    void *data;
    int32_t type;            /* relaysum_type */
    int64_t worker_stride;   /* ignored for n == 1 */
    int64_t row_stride;      /* ignored for one row */
    int64_t head_stride;     /* ignored for one head */
} relaysum_heads;

/* Ranges of packed sequences: sequence s of worker i has the rows starts[s] to
 * starts[s + 1] - 1 and the keys key_starts[s] to key_starts[s + 1] - 1, both
 * int32[count + 1] at + i * their stride (0: all workers have the same), in
 * ascending order.  A row sees its sequence's keys, with causal != 0 those up to
 * the one that is as far from their end as the row is from its own.  Rows in no
 * sequence see nothing.  ranges is int32 [tokens][2] of each worker, ranges_stride >= tokens rows
 * apart. */
int relaysum_attention_ranges(int32_t n, int64_t tokens, int64_t keys, int32_t count,
                              const int32_t *starts, int64_t starts_stride, const int32_t *key_starts,
                              int64_t key_starts_stride, int32_t causal, int32_t *ranges,
                              int64_t ranges_stride, void *hip_stream);

/*   q, k, v, out   heads of one type, 1 <= width <= 256
 *   ranges         8-byte aligned, or NULL; ranges_stride rows between workers'
 *                  (0: all have the same)
 *   scale          positive, at most 2^126
 *   lse            out, float[n][heads][tokens], or NULL: for the backward pass
 *   workspace      relaysum_attention_workspace bytes, 16-byte aligned (NULL if 0):
 *                  sums of few rows' keys that are shared out and join, or a mark
 *                  for each tile of many rows
 * tokens * heads and keys up to 2^30. */
int64_t relaysum_attention_workspace(int32_t n, int64_t tokens, int64_t keys, int32_t heads,
                                     int32_t kv_heads, int64_t width);
int relaysum_attention(int32_t n, int64_t tokens, int64_t keys, int32_t heads, int32_t kv_heads,
                       int64_t width, const relaysum_heads *q, const relaysum_heads *k,
                       const relaysum_heads *v, const int32_t *ranges, int64_t ranges_stride,
                       int32_t causal, float scale, const relaysum_heads *out, float *lse,
                       void *workspace, size_t workspace_bytes, void *hip_stream);

/* dq, dk and dv from dout, the gradient of out, and the forward pass's arguments,
 * out and lse; all of one type.  Every row of dq, dk and dv is written (dk and dv
 * sum over the heads that share a key head).  dq, dk and dv may be parts of the
 * rows of one array. */
int64_t relaysum_attention_backward_workspace(int32_t n, int64_t tokens, int64_t keys, int32_t heads,
                                              int32_t kv_heads, int64_t width, int32_t type);
int relaysum_attention_backward(int32_t n, int64_t tokens, int64_t keys, int32_t heads,
                                int32_t kv_heads, int64_t width, const relaysum_heads *dout,
                                const relaysum_heads *q, const relaysum_heads *k,
                                const relaysum_heads *v, const relaysum_heads *out, const float *lse,
                                const int32_t *ranges, int64_t ranges_stride, int32_t causal,
                                float scale, const relaysum_heads *dq, const relaysum_heads *dk,
                                const relaysum_heads *dv, void *workspace, size_t workspace_bytes,
                                void *hip_stream);

/* ---- recurrence -----------------------------------------------------------
 *
 * The other way to mix tokens: every channel carries a state along its sequence,
 *
 *   h_t = a_t h_(t-1) + (1 - a_t) x_t,   a = sigmoid(gate)
 *   dgate_t = dh_t (h_(t-1) - x_t) a_t (1 - a_t),  dx_t = (1 - a_t) dh_t
 *
 * where dh is the whole gradient of h_t: that of the output, and a_(t+1) times the
 * next token's.  A worker's rows hold `count` packed sequences: sequence s has the
 * rows starts[s] to starts[s + 1] - 1, int32[count + 1] of DEVICE memory at
 * + i * starts_stride (0: all workers have the same), ascending, within 0..tokens;
 * NULL: one sequence of all rows (count 1).  Each starts from its own state
 * (initial, or zeros) and leaves its last one; one of no rows leaves the state
 * that it has.  Rows in no sequence give zeros.  States are held in 32 bits, and
 * the gradients come from states in 32 bits, not from the rounded h.
 * Errors, streams, capture and the rules for arrays are those of the layer calls;
 * equal inputs give equal bits.  tokens up to 2^30, width up to 32768.
 *
 *   gate, x, h     rows of one type (of the gradients too)
 *   initial, last  float rows, `count` for each worker, or NULL
 *   saved          out, float[n][relaysum_recurrence_chunks(tokens)][width], for the
 *                  backward pass, or NULL
 *   workspace      relaysum_recurrence_workspace bytes, 8-byte aligned (NULL if 0) */
int64_t relaysum_recurrence_chunks(int64_t tokens);
int64_t relaysum_recurrence_workspace(int32_t n, int64_t tokens, int64_t width);
int relaysum_recurrence(int32_t n, int64_t tokens, int64_t width, int32_t count, const int32_t *starts,
                        int64_t starts_stride, const relaysum_rows *gate, const relaysum_rows *x,
                        const relaysum_rows *initial, const relaysum_rows *h, const relaysum_rows *last,
                        float *saved, void *workspace, size_t workspace_bytes, void *hip_stream);

/* dgate, dx and dinitial (NULL: not wanted) from dh, the gradient of h, and dlast,
 * that of last (NULL: none). */
int relaysum_recurrence_backward(int32_t n, int64_t tokens, int64_t width, int32_t count,
                                 const int32_t *starts, int64_t starts_stride, const relaysum_rows *dh,
                                 const relaysum_rows *dlast, const relaysum_rows *gate,
                                 const relaysum_rows *x, const relaysum_rows *initial, const float *saved,
                                 const relaysum_rows *dgate, const relaysum_rows *dx,
                                 const relaysum_rows *dinitial, void *workspace, size_t workspace_bytes,
                                 void *hip_stream);

/* ---- norms around a block ---------------------------------------------------
 *
 * The norm behind a block, with its gate and the scale of the residual branch,
 * and the norm in front of the next block, in one pass:
 *
 *   s = residual + scale * sigmoid(gate) * z * post_rstd * post_weight
 *   y = s * rstd * weight,    post_rstd and rstd = 1 / sqrt(mean^2 + eps) of z and s
 *
 * z, gate, residual and sum are rows of one type; s is rounded to it, and the
 * second norm is that of the rounded s.  gate may be NULL (1 in its place).
 * post_weight and weight are float[width] of each worker, scale one float, at
 * + i * their strides.  y leaves in 8 bits by whole rows, and s for the gradient
 * by 128 (saved, or NULL), as relaysum_rmsnorm's; the rounding to 8 bits counts
 * as the identity.  post_rstd and rstd are out, float[n][tokens].  sum may be
 * the own rows of z, gate or residual.  Rows whose mean square lies outside
 * binary32's range are treated as relaysum_rmsnorm's.  Limits, errors, streams
 * and capture are those of the calls on 8-bit rows. */
int relaysum_blocknorm(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *z,
                       const relaysum_rows *gate, const relaysum_rows *residual, const float *post_weight,
                       int64_t post_weight_stride, const float *scale, int64_t scale_stride,
                       const float *weight, int64_t weight_stride, float eps, const relaysum_rows *sum,
                       const relaysum_packed *y, float *post_rstd, float *rstd,
                       const relaysum_packed *saved, void *hip_stream);

/* The gradients of z (dz), gate (dgate, NULL if and only if gate is) and residual
 * (ds), and of the three parameters (float rows, one for each worker,
 * overwritten; scale_grad's has one entry), from dy, dsum (the gradient of the sum
 * from elsewhere, NULL: none) and what the forward pass gave.  dz, dgate and ds
 * may each be the own rows of one of the inputs.  Equal inputs give
 * equal bits.  workspace: relaysum_blocknorm_workspace
 * bytes, 4-byte aligned (NULL if 0). */
int64_t relaysum_blocknorm_workspace(int32_t n, int64_t tokens, int64_t width);
int relaysum_blocknorm_backward(int32_t n, int64_t tokens, int64_t width, const relaysum_rows *dy,
                                const relaysum_rows *dsum, const relaysum_rows *z,
                                const relaysum_rows *gate, const relaysum_packed *saved,
                                const float *post_rstd, const float *rstd, const float *post_weight,
                                int64_t post_weight_stride, const float *scale, int64_t scale_stride,
                                const float *weight, int64_t weight_stride, const relaysum_rows *dz,
                                const relaysum_rows *dgate, const relaysum_rows *ds,
                                const relaysum_rows *post_weight_grad, const relaysum_rows *scale_grad,
                                const relaysum_rows *weight_grad, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* Text of the calling thread's last failure in the layer calls (""
 * after a call that succeeded). */
const char *relaysum_layer_error(void);

#ifdef __cplusplus
}
#endif

#endif /* RELAYSUM_H */
