/*
 * klay.h -- C ABI of the MI355X (gfx950) layered arithmetic-circuit evaluator.
 *
 * The library evaluates a negation-normal-form circuit DAG (paper Section 2, Eq. 1: leaves
 * are literals, inner nodes AND / OR gates) on a batch of leaf-weight vectors, layer by
 * layer (Section 3.1, Eq. 2; Section 4, Alg. 1; Appendix C, Alg. 2-4), and differentiates
 * the root values with respect to the leaf weights.
 *
 * Conventions
 *   - Plain C, no exceptions.  Every call returns a klay_status; klay_last_error() gives a
 *     thread-local message for the last failing call on the calling thread.
 *   - "host" pointers are ordinary process memory, "device" pointers are HIP device memory on
 *     the circuit's device.  The library never takes ownership of caller buffers.
 *   - klay_forward / klay_backward only enqueue work on the caller's stream; they do not
 *     synchronise the host with the device.  A handle must not be used from two streams at
 *     once (its activation workspace is shared between calls).
 */
#ifndef KLAY_H
#define KLAY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct klay_circuit klay_circuit;   /* opaque; owns index arrays and (unless set) a workspace */

typedef enum {
    KLAY_OK = 0,
    KLAY_EINVAL = 1,   /* malformed argument or circuit (index out of range, empty gate, ...) */
    KLAY_ECYCLE = 2,   /* the node graph is not acyclic */
    KLAY_ENOMEM = 3,   /* host or device allocation failed, or caller workspace too small */
    KLAY_EHIP = 4,     /* a HIP runtime call failed */
    KLAY_ESTATE = 5    /* call order violated (backward before forward, host-only handle, ...) */
} klay_status;

/* Semiring of the evaluation (Section 4): REAL = (+, x) on probabilities, LOG = (logsumexp, +)
 * on log-probabilities (Alg. 4 with epsilon = 0).  Section 4 closes by noting that any semiring
 * whose operations are reductions will do; MAXLOG = (max, +) on log-probabilities is the one
 * offered beyond the paper's two: the log weight of the heaviest proof tree (for a smooth d-DNNF
 * the most probable model).  MAXLOG is evaluated forward only. */
typedef enum { KLAY_REAL = 0, KLAY_LOG = 1, KLAY_MAXLOG = 2 } klay_semiring;

/* node_type codes of the input DAG */
enum { KLAY_LIT = 0, KLAY_AND = 1, KLAY_OR = 2, KLAY_TRUE = 3, KLAY_FALSE = 4 };

/* Build-time options; zero-initialise and override.  0 means "library default". */
typedef struct klay_options {
    int32_t no_reorder;      /* 1: keep nodes of a layer in input-id order (no locality sort)     */
    int32_t heavy_fan;       /* rows with more sources than this are split (default 48); a pass that
                                splits rows anyway and whose unsplit rows are few (under 2e5 entries) with a
                                tenth or more of them in rows longer than half of it splits from half on */
    int32_t min_segment;     /* smallest split segment, in edges (default 24)                     */
    int32_t no_tail;         /* 1: one launch per layer also for the narrow top layers            */
    int32_t unary_chains;    /* 1: the paper's layerization throughout: an edge that skips layers goes through
                                one unary chain node per layer (Section 3.1).  Default (0): padding-free
                                below the narrow top of the circuit.  Chain nodes only copy a value, so in
                                the layers 1 .. A (A = klay_info_t.alias_top_layer) none are made and an edge
                                reads the child's own row wherever it lives; layer A is complete (it holds
                                a stand-in for every node read from above), and the layers above it, the
                                ones the persistent kernels may take, are as in the paper.  Same values
                                and gradients, fewer rows and edges.  klay_layer_csr returns, for the layers
                                up to A, rows of the whole activation buffer (layer 0 first).  A = 0 when
                                the whole circuit is narrow, A = L when no layer is (or with no_tail)   */
    int32_t no_merge;        /* 1: do not identify structurally identical gates (Section 3.2)         */
    int32_t small_batch_edges; /* 1: batches of at most 32 columns run the lanes = edges kernel (a wave takes
                                64 / B index entries per step and reduces the entries of a row across its
                                lanes with a segmented scan) instead of the default, a lane group per row,
                                which measures about twice as fast at B = 1 and B = 4; same results        */
    int32_t tail_rows_cap;   /* > 0: layers with more nodes than this are no candidates for the persistent
                                kernels (at most 20000, the default; smaller values move the boundary
                                between the two parts of the layerization up: for tests)                 */
    int32_t no_fusion;       /* 1: every AND node's value is written.  Default (0): in the padding-free part an
                                AND node with at most one child that is not a leaf, few children and parents,
                                and only short OR rows above it is fused into those rows when the batch has more
                                than 64 columns: they read its children and combine them themselves, so a forward
                                pass does not write its value.  klay_backward, which needs every value, evaluates
                                the fused rows first when it follows such a pass, and the forward pass of a handle
                                whose previous forward pass was followed by klay_backward writes every value.
                                Same results                                                              */
} klay_options;

typedef struct klay_info_t {
    int32_t num_vars;
    int32_t num_roots;
    int32_t num_layers;       /* L: gate layers 1..L above the leaf layer 0                        */
    int32_t device;           /* -1 for a host-only handle                                        */
    int64_t num_nodes;        /* nodes of the layered circuit, all layers, unary chain nodes incl. */
    int64_t num_edges;        /* edges of the layered circuit = sum over layers of |S_l|           */
    int64_t dag_nodes;        /* input nodes reachable from the roots                              */
    int64_t dag_edges;        /* their child edges                                                 */
    int64_t num_pad_nodes;    /* unary chain nodes inserted by layerization                        */
    int64_t max_layer_nodes;
    int64_t max_fan_in;
    int64_t max_fan_out;
    int64_t num_split_rows;   /* rows (forward) and columns (backward) evaluated by split passes   */
    int64_t index_bytes;      /* device bytes held by index arrays                                 */
    int64_t tail_first_layer; /* first layer that may run in the persistent top-of-circuit kernel
                                 (0: none); the layers actually taken depend on the batch size       */
    int64_t num_merged_nodes; /* input gates identified with a structurally identical gate          */
    int64_t alias_top_layer;  /* A: the layers 1 .. A are padding-free (see klay_options.unary_chains)  */
    int64_t num_fused_rows;   /* AND rows that the fused plans do not evaluate (see klay_options.no_fusion) */
} klay_info_t;

/* Per-kernel-class timing of the most recent forward / backward call, filled only while
 * profiling is enabled.  Durations come from HIP events recorded on the caller's stream around
 * every single launch.  FWD_x / BWD_x are the main-row launches of a layer, mostly with the segments of its
 * split rows (one kernel each: the generic row kernel up to 84 columns and, where most entries are segments, up
 * to 128, the streaming kernel otherwise), SPLIT segment launches of their own, COMBINE the
 * combine launches, MAIN_COMBINE (any operation) the launches that take the main rows and the combine
 * rows of a layer together (32 < B <= 64, where the segments run in a launch of their own first),
 * FWD_OR_FUSED the forward launches of OR layers that read the children of fused AND rows (klay_options.no_fusion),
 * PROD_EDGES the per-parent pass of the real-semiring reverse sweep over a product layer (adjoint
 * times the product of the non-zero children, in place), BWD_PROD the by-child pass that follows
 * it, BWD_SUM_MUL / BWD_PROD_MUL the passes into a product layer, whose rows leave multiplied by
 * the nodes' own values (so that PROD_EDGES only has to repair columns whose value is zero).
 * Log-semiring reverse sweep: BWD_SOFTMAX_ONE is the step through an OR layer that gathers one
 * row per edge, BWD_SUM_ENC the step through an AND layer that leaves the adjoints of the OR layer
 * below in the form that step reads; BWD_SOFTMAX, the two-gather step, only runs where that form
 * cannot be used. */
enum { KLAY_K_LEAF = 0, KLAY_K_FWD_SUM, KLAY_K_FWD_PROD, KLAY_K_FWD_LSE, KLAY_K_ROOT,
       KLAY_K_SEED, KLAY_K_BWD_SUM, KLAY_K_BWD_SOFTMAX, KLAY_K_BWD_LEAF, KLAY_K_TAIL_FWD,
       KLAY_K_TAIL_BWD, KLAY_K_SPLIT, KLAY_K_PROD_EDGES, KLAY_K_FWD_MAX, KLAY_K_BWD_SUM_ENC,
       KLAY_K_BWD_SOFTMAX_ONE, KLAY_K_BWD_PROD, KLAY_K_BWD_SUM_MUL, KLAY_K_BWD_PROD_MUL,
       KLAY_K_COMBINE, KLAY_K_MAIN_COMBINE, KLAY_K_FWD_OR_FUSED, KLAY_K_COUNT };
typedef struct klay_profile_t {
    float   ms[KLAY_K_COUNT];          /* summed device time of the class's launches       */
    int32_t launches[KLAY_K_COUNT];
    double  alg_bytes[KLAY_K_COUNT];   /* algorithmic bytes moved by those launches (no-reuse model:
                                          every index entry gathers its row from memory)             */
    double  min_bytes[KLAY_K_COUNT];   /* compulsory bytes of those launches: every distinct source row
                                          read once, every output row written once, plus the indices */
} klay_profile_t;

/*
 * klay_build -- layerize and tensorize a circuit (Section 3.1 Eq. 2, Section 3.2, Alg. 2, Alg. 3)
 * and upload the per-layer index arrays.
 *
 *   num_vars      V; literals name variables 0..V-1
 *   num_nodes     number of nodes of the input DAG
 *   node_type     host [num_nodes], KLAY_LIT .. KLAY_FALSE
 *   node_lit      host [num_nodes]; for KLAY_LIT +(v+1) (positive) or -(v+1) (negated), else ignored
 *   child_ptr     host [num_nodes+1]; children of node i are child_idx[child_ptr[i] .. child_ptr[i+1])
 *   child_idx     host [child_ptr[num_nodes]] node ids, in any order
 *   num_roots, roots   host [num_roots] node ids; out[:, r] of klay_forward is roots[r]'s value
 *   device        HIP device ordinal, or -1 for a host-only handle (layerization only: the
 *                 inspection calls work, forward/backward return KLAY_ESTATE)
 *   out           receives the handle
 *
 * All arrays are borrowed for the duration of the call only.  Nodes not reachable from a root
 * are dropped.  Leaves carrying the same literal and gates with the same type and the same
 * children are identified bottom-up (Section 3.2, Eq. 3, Theorem 1; child lists are compared on
 * a hash hit, so a collision never merges different gates); values are unchanged by it.  Gates of the wrong parity for their height (an OR directly over leaves, an AND
 * under an AND) are lifted one layer so that odd layers hold AND and even layers OR (Section 3.1).
 * Layer-skipping edges get one chain of unary nodes per (child, layer); all roots are extended to
 * the height of the tallest (Section 3.2).
 * Errors: KLAY_EINVAL (bad sizes, index or literal out of range, a gate without children, a gate of the
 * circuit that lists the same node id twice, a leaf with children, no roots), KLAY_ECYCLE, KLAY_ENOMEM,
 * KLAY_EHIP.  Two different leaf nodes with the same literal under one gate, or two gates that turn out
 * identical, are two children and count twice (Eq. 1).
 */
klay_status klay_build(int32_t num_vars, int64_t num_nodes, const uint8_t* node_type,
                       const int32_t* node_lit, const int64_t* child_ptr, const int32_t* child_idx,
                       int32_t num_roots, const int32_t* roots, int32_t device, klay_circuit** out);

/* Same with explicit options (opts may be NULL). */
klay_status klay_build_ex(int32_t num_vars, int64_t num_nodes, const uint8_t* node_type,
                          const int32_t* node_lit, const int64_t* child_ptr, const int32_t* child_idx,
                          int32_t num_roots, const int32_t* roots, int32_t device,
                          const klay_options* opts, klay_circuit** out);

/*
 * klay_forward -- evaluate all layers (Alg. 1 for KLAY_REAL, Alg. 4 for KLAY_LOG).
 *   leaf_weights  device [B, V] row-major fp32: p_v (REAL) or log p_v (LOG, MAXLOG).  The negated literal
 *                 of v gets 1 - p_v resp. log(1 - exp(x_v)).  LOG, MAXLOG: a child that is NaN (a NaN weight, or the
 *                 negated literal of x_v > 0) counts as impossible in an OR gate and makes an AND gate NaN.
 *   B             batch size >= 1
 *   out           device [B, R] row-major fp32; out[b, r] = value of roots[r] on sample b
 *   stream        hipStream_t (as void*), may be NULL for the default stream
 * Keeps the layers' values in the workspace for klay_backward (all but those of fused AND rows, which
 * klay_backward then evaluates itself: see klay_options.no_fusion).  Grows the library-owned
 * workspace (hipMalloc, which synchronises) when B exceeds what earlier calls needed, unless a
 * caller workspace was set.  Errors: KLAY_EINVAL, KLAY_ENOMEM, KLAY_EHIP, KLAY_ESTATE.
 */
klay_status klay_forward(klay_circuit* c, const float* leaf_weights, int32_t B, float* out,
                         klay_semiring semiring, void* stream);

/*
 * klay_forward_static -- klay_forward for callers that cannot allocate: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels, same results as
 * klay_forward, but the layer values, the partial rows of split rows and the transposed leaf weights
 * live in a fixed array in device memory that is part of the library image (KLAY_STATIC_WORKSPACE_BYTES
 * per GPU, held until the process ends) instead of the handle's workspace.  The call allocates
 * nothing (no hipMalloc / hipFree, no events: profiling is not recorded) and only enqueues kernels.
 *   - A circuit / batch size whose forward workspace, klay_workspace_bytes(c, B, 0), exceeds
 *     KLAY_STATIC_WORKSPACE_BYTES is refused with KLAY_ENOMEM before anything is launched.
 *   - Forward only: nothing is kept for klay_backward, and the handle's own state (a previous
 *     klay_forward that is still to be differentiated) is left untouched.
 *   - All handles on one GPU share the one array: calls that overlap in time on the same GPU (two
 *     streams, two threads, two handles) race.  Calls on one stream are ordered and safe; nothing in
 *     the array has to survive from one call to the next, and nothing is assumed to start at zero.
 * Errors: as klay_forward.
 */
#define KLAY_STATIC_WORKSPACE_BYTES ((size_t)64 << 20)
klay_status klay_forward_static(klay_circuit* c, const float* leaf_weights, int32_t B, float* out,
                                klay_semiring semiring, void* stream);

/*
 * klay_backward -- reverse-mode derivative of the most recent klay_forward on this handle
 * (the paper obtains it from autograd, Section 6; here it is a reverse sweep over the layers).
 *   dout          device [B, R] fp32, adjoint of `out`
 *   dleaf         device [B, V] fp32, receives sum_r dout[b,r] * d out[b,r] / d leaf_weights[b,v];
 *                 every entry is written (0 for variables the circuit does not use)
 * Uses B, the semiring and the activations of that forward call; the caller must not have run
 * another forward in between.  The first real-semiring call on a handle uploads extra index
 * arrays (hipMalloc, which synchronises); later calls only enqueue.
 * MAXLOG is not differentiated (KLAY_EINVAL).  A literal whose adjoint is exactly 0 contributes 0 even where the
 * derivative of its weight is infinite (log-domain negated literal at p = 1).
 * Errors: KLAY_ESTATE if no forward was run, KLAY_EINVAL, KLAY_EHIP.
 */
klay_status klay_backward(klay_circuit* c, const float* dout, float* dleaf, void* stream);

/*
 * klay_forward_lits / klay_backward_lits -- the same two passes with weights of their own for the
 * negated literals (weighted model counting with arbitrary literal weights, Section 2: every leaf
 * of the arithmetic circuit carries a weight).
 *   pos_weights   device [B, V]: weight of literal v (probability, or its log in the log-domain semirings)
 *   neg_weights   device [B, V]: weight of literal -v, same domain; NULL makes the call klay_forward
 *   dpos, dneg    device [B, V]: adjoints of the two arrays, treated as independent inputs; dneg may
 *                 be NULL when only dpos is wanted.  Every entry is written.
 * A forward pass with neg_weights must be differentiated by klay_backward_lits and one without by
 * klay_backward (KLAY_ESTATE otherwise).  Everything else is as for klay_forward / klay_backward.
 */
klay_status klay_forward_lits(klay_circuit* c, const float* pos_weights, const float* neg_weights, int32_t B,
                              float* out, klay_semiring semiring, void* stream);
klay_status klay_backward_lits(klay_circuit* c, const float* dout, float* dpos, float* dneg, void* stream);

/*
 * klay_forward_f64 / klay_backward_f64 -- the same evaluation in double precision, for circuits whose
 * log-values outgrow what fp32 resolves and as an on-device accuracy reference for the fp32 kernels.
 * Same launch plans, kernels of their own (a generic gather-reduce kernel, persistent kernels for the narrow
 * layers: klay_persistent_layers), the full-precision exp / log.
 *   pos_weights, neg_weights, out, dout, dpos, dneg   as for klay_forward_lits / klay_backward_lits,
 *                 in double; neg_weights = NULL derives the negated literals from pos_weights, and
 *                 dneg must then be NULL as well.
 * A NaN child makes an OR gate NaN here (LOG), unless every other child is impossible: then the gate is too.
 * All three semirings are evaluated; KLAY_LOG and KLAY_REAL are differentiated (KLAY_MAXLOG is not:
 * KLAY_EINVAL).  In double the real semiring reaches circuits whose values underflow fp32.
 * The activations live in a library-owned workspace of their own (klay_set_workspace and
 * klay_workspace_bytes do not cover it) and are independent of the fp32 state: a handle can hold
 * one fp32 and one double-precision forward pass at the same time.  Profiling does not cover
 * these calls.
 */
klay_status klay_forward_f64(klay_circuit* c, const double* pos_weights, const double* neg_weights, int32_t B,
                             double* out, klay_semiring semiring, void* stream);
klay_status klay_backward_f64(klay_circuit* c, const double* dout, double* dpos, double* dneg, void* stream);

/* Structure of the layered circuit. */
klay_status klay_info(const klay_circuit* c, klay_info_t* info);

/* nodes[l], edges[l] for l = 0..L (host arrays of num_layers+1 entries; edges[0] = 0). */
klay_status klay_layer_sizes(const klay_circuit* c, int64_t* nodes, int64_t* edges);

/*
 * Host copy of layer l's index vectors (Section 4 / Alg. 3), 1 <= l <= L, in CSR form:
 * row_ptr [n_l + 1], child [e_l].  child is the paper's S_l (position in layer l-1); the paper's
 * R_l is row_ptr expanded (edge j belongs to parent r iff row_ptr[r] <= j < row_ptr[r+1]).
 * For l <= klay_info_t.alias_top_layer child holds rows of the whole activation buffer instead
 * (the rows of layer 0, then those of layer 1, ...), always of a layer below l.
 */
klay_status klay_layer_csr(const klay_circuit* c, int32_t layer, int64_t* row_ptr, int32_t* child);

/*
 * Host copy of what each node of layer l (0 <= l <= L) stands for: origin[i] is the input node id
 * whose value row i holds (for a unary chain node: the id of the node the chain starts from),
 * is_pad[i] is 1 for chain nodes.
 */
klay_status klay_layer_nodes(const klay_circuit* c, int32_t layer, int32_t* origin, uint8_t* is_pad);

/*
 * position[r] (host array of num_roots entries) = row of the top layer L that holds roots[r]'s value
 * (Section 3.2: all roots sit in the last layer, a root of lower height through a stand-in).
 */
klay_status klay_root_positions(const klay_circuit* c, int32_t* position);

/* Bytes of device workspace a forward (and, if need_backward, backward) call with batch B needs.  A handle built
 * with device = -1 answers for a device that grants a workgroup the whole 160 KB LDS of a compute unit (the
 * persistent kernels' buffers depend on which layers fit). */
size_t klay_workspace_bytes(const klay_circuit* c, int32_t B, int need_backward);

/* Which layers a forward pass over B columns gives to the persistent kernels: *first_layer and all above it (0: none, every layer is
 * launched by itself), *plan = 1: the layers of the circuit as klay_layer_csr shows them, 2: the narrow top of a circuit with long
 * rows, whose chain nodes exist in those kernels only, 0 with *first_layer = 0.  double_precision: klay_forward_f64; training: the previous
 * forward pass of the handle was followed by a backward pass.  Handles built with device = -1 answer as for klay_workspace_bytes. */
klay_status klay_persistent_layers(const klay_circuit* c, int32_t B, klay_semiring semiring, int32_t double_precision, int32_t training,
                                   int32_t* first_layer, int32_t* plan);

/* Use caller device memory (256-byte aligned) as workspace instead of library-owned memory;
 * dev_ptr = NULL returns to library-owned memory.  The caller keeps ownership. */
klay_status klay_set_workspace(klay_circuit* c, void* dev_ptr, size_t bytes);

/* Enable (1) / disable (0) per-kernel-class event timing; klay_get_profile synchronises on the
 * recorded events and returns the figures of the most recent forward and backward calls. */
klay_status klay_set_profiling(klay_circuit* c, int32_t enable);
klay_status klay_get_profile(klay_circuit* c, klay_profile_t* profile);

/*
 * Incremental construction of a multi-rooted circuit (Section 3.2: circuits that share variables
 * are merged into one layered circuit, one after the other, and share every node they have in
 * common).  A builder collects circuits; klay_builder_finish layerizes all of them together, so
 * identical sub-circuits of different circuits become one set of rows and all roots reach the
 * height of the tallest circuit.
 *
 *   klay_builder_create   num_vars = V of the leaf-weight array all circuits are evaluated on.
 *   klay_builder_add      same arrays as klay_build (node ids are local to this circuit; borrowed
 *                         for the call).  first_root (may be NULL) receives the column of `out`
 *                         that this circuit's roots[0] will occupy; its roots take consecutive
 *                         columns, circuits in the order they were added.  Range errors are
 *                         reported here (KLAY_EINVAL) and leave the builder unchanged; structural
 *                         errors (cycle, empty gate, repeated child) are reported by finish.
 *   klay_builder_finish   layerize what has been added so far (as klay_build_ex).  The builder
 *                         stays valid: more circuits may be added and finish called again, each
 *                         call returning an independent handle.  KLAY_ESTATE if nothing was added.
 *   klay_builder_destroy  NULL is allowed.
 */
typedef struct klay_builder klay_builder;
klay_status klay_builder_create(int32_t num_vars, klay_builder** out);
klay_status klay_builder_add(klay_builder* b, int64_t num_nodes, const uint8_t* node_type,
                             const int32_t* node_lit, const int64_t* child_ptr, const int32_t* child_idx,
                             int32_t num_roots, const int32_t* roots, int32_t* first_root);
klay_status klay_builder_finish(const klay_builder* b, int32_t device, const klay_options* opts,
                                klay_circuit** out);
void klay_builder_destroy(klay_builder* b);

/* Frees index arrays and library-owned workspace.  NULL is allowed. */
void klay_destroy(klay_circuit* c);

/*
 * Operators between a network and a circuit's leaf weights.  They need no handle; every call enqueues kernels on `stream` of `device`
 * (of the calling thread's current device it makes no use, and leaves it as it was), allocates nothing and does not synchronise.
 * Two calls may overlap if they share no buffer that either writes.  An output must not overlap another one or an input (klay_scan_step's
 * state excepted); that dlogits is the logits, final the initial states, dinitial dfinal, or dgates or dinputs the states is refused.
 */

/* Types of the tensors that a network gives and takes: IEEE single, bfloat16, IEEE half.  All arithmetic is in single. */
typedef enum { KLAY_F32 = 0, KLAY_BF16 = 1, KLAY_F16 = 2 } klay_dtype;

/* Where row r (0 <= r < rows) of a tensor starts: (r / inner) * outer_stride + (r % inner) * inner_stride elements. */
typedef struct klay_rows {
    int64_t inner, outer_stride, inner_stride;
} klay_rows;

/*
 * klay_tokens_forward -- log probabilities of given tokens under rows of logits (the weights of literals "the network answers t"):
 *   p_j = exp(x_j) / sum_i exp(x_i);  logp_k = ln p_{t_k};  neg_k = ln(1 - p_{t_k}), the weight of the negated literal, from the other
 *   tokens' logits also where p rounds to 1 (-inf only where none of them is allowed: finite masks leave a finite weight);
 *   entropy = - sum_j p_j ln p_j;  the `top` largest logits (equal ones: the lowest index first).
 *   logits      device [rows, vocab] of `dtype`, the elements of a row next to each other, rows placed by logit_rows
 *   tokens      device [rows, num_tokens] int64, placed by token_rows and token_stride.  A negative token asks for nothing: its logp and
 *               neg are 0 and it has no gradient.  A token >= vocab gives NaN.  The same token may be asked for more than once.
 *   logp, neg   device [rows, num_tokens] fp32; neg may be NULL, logp only where num_tokens = 0
 *   entropy     device [rows] fp32, or NULL
 *   stats       device [rows, 4] fp32, what klay_tokens_backward needs of a row, or NULL
 *   top_logp, top_tokens   device [rows, top] fp32 / int64, best first; NULL where top = 0
 *   workspace   device, 16-byte aligned, klay_tokens_workspace_bytes(args) bytes; NULL where that is 0
 * A logit of -inf is a token that is not allowed.  A row of nothing else gives logp = -inf, neg = 0, entropy 0, and no gradient; a NaN or
 * +inf makes every value of its row NaN (and leaves top_tokens any tokens).
 * Errors: KLAY_EINVAL (sizes out of range: 1 <= vocab, 0 <= num_tokens <= 1024, 0 <= top <= min(vocab, 64), 0 <= rows < 2^31; null or
 * unknown arguments), KLAY_ENOMEM (workspace too small), KLAY_EHIP.
 */
typedef struct klay_tokens_args {
    int32_t dtype, device, vocab, num_tokens, top, reserved;
    int64_t rows;
    const void* logits;
    klay_rows logit_rows;
    const int64_t* tokens;
    klay_rows token_rows;
    int64_t token_stride;
} klay_tokens_args;
size_t klay_tokens_workspace_bytes(const klay_tokens_args* args);
klay_status klay_tokens_forward(const klay_tokens_args* args, float* logp, float* neg, float* entropy, float* stats, float* top_logp,
                                int64_t* top_tokens, void* workspace, size_t workspace_bytes, void* stream);

/*
 * klay_tokens_backward -- derivative of a klay_tokens_forward with respect to the logits, which must be as they were.
 *   stats       as written by the forward call (with entropy asked for if dentropy is given)
 *   dlogp, dneg, dentropy   device, shaped as the outputs; each may be NULL (no adjoint)
 *   dlogits     device [rows, vocab] contiguous, of `dtype`; every entry is written, rounded once.  An adjoint of exactly 0
 *               contributes 0, and a row all of whose adjoints are 0 gets zeros, whatever it holds; with any other adjoint a row
 *               that holds a NaN or +inf gets NaN.
 * The same inputs give the same bits.  Errors: as klay_tokens_forward.
 */
klay_status klay_tokens_backward(const klay_tokens_args* args, const float* stats, const float* dlogp, const float* dneg,
                                 const float* dentropy, void* dlogits, void* stream);

/*
 * klay_head_forward -- what klay_tokens_forward says of rows of logits, straight from the network's last layer: logit j of row i is
 * hidden_i . weight_j + bias_j, made in pieces on the chip (fp32 sums, not rounded) and never written.
 *   hidden      device [rows, width] of `dtype`, the elements of a row next to each other, rows placed by hidden_rows
 *   weight      device [vocab, width] of `dtype`, the elements of a row next to each other, rows weight_stride elements apart (>= 0)
 *   bias        device [vocab] fp32, or NULL.  -inf: a token that is not allowed, whatever its weights hold
 *   tokens      device [rows, num_tokens] int64, placed by token_rows and token_stride: as for klay_tokens_forward
 *   logp, neg, entropy   as for klay_tokens_forward
 *   kept        device, 16-byte aligned, klay_list_kept_bytes(rows, num_tokens) bytes: what klay_head_backward needs of the rows; NULL: not kept
 *   workspace   device, 16-byte aligned, klay_head_workspace_bytes(args, 0) bytes (for klay_head_backward: args, 1)
 * Rows are read where they lie if they have one stride, and their first and that stride are at multiples of 4 bytes; others are copied into the
 * workspace first.  A forward call's workspace holds the sums of tiles (64 MB, or those of 256 rows) and what `kept` would; a backward one's the
 * adjoints of a piece of the vocabulary (about 2^25 of them, 128 MB; of 256 tokens at least), fp32 sums of dhidden, a copy of hidden (two of 16
 * bits) and, with a bias, room for the piece's weights (of 256 rows or fewer those of 131072 tokens).
 * A row whose hidden state, or any allowed token's weights, holds a NaN or an infinity may get NaN in every value.
 * Errors: KLAY_EINVAL (sizes out of range: 1 <= vocab <= 2^31 - 4097, 1 <= width <= 2^20, 0 <= num_tokens <= 1024, 0 <= rows <= 2^20; null or
 * unknown arguments), KLAY_ENOMEM (workspace too small), KLAY_EHIP.
 */
typedef struct klay_head_args {
    int32_t dtype, device, width, vocab, num_tokens, reserved;
    int64_t rows;
    const void* hidden;
    klay_rows hidden_rows;
    const void* weight;
    int64_t weight_stride;
    const float* bias;
    const int64_t* tokens;
    klay_rows token_rows;
    int64_t token_stride;
} klay_head_args;
size_t klay_list_kept_bytes(int64_t rows, int32_t num_tokens);
size_t klay_head_workspace_bytes(const klay_head_args* args, int32_t backward);
klay_status klay_head_forward(const klay_head_args* args, float* logp, float* neg, float* entropy, void* kept, void* workspace,
                              size_t workspace_bytes, void* stream);

/*
 * klay_head_backward -- derivative of a klay_head_forward, which has kept its rows; hidden, weight, bias must be as they were.
 *   dlogp, dneg, dentropy   device, shaped as the outputs; each may be NULL (no adjoint)
 *   dhidden     device [rows, width] contiguous, of `dtype`; dweight device [vocab, width] contiguous, of `dtype`; dbias device [vocab]
 *               fp32; each may be NULL (not wanted); every entry is written (nothing where rows = 0)
 * The adjoints of the logits are made again in pieces of the vocabulary and go into the two products as two numbers of `dtype`, where it has 16 bits (fp16: under
 * a power of two common to all); sums are fp32, and the same inputs give the same bits.  A row all of whose adjoints are exactly 0, or that
 * allows nothing, has no gradient and gives none, whatever it holds.
 */
klay_status klay_head_backward(const klay_head_args* args, const void* kept, const float* dlogp, const float* dneg, const float* dentropy,
                               void* dhidden, void* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream);

/*
 * klay_distill_forward -- divergence of rows of logits from what a teacher says of its likeliest tokens (args->tokens, a list a row):
 *   p = softmax(x / temperature);  q = softmax(teacher / temperature) over the listed tokens
 *   loss = sum_k q_k (ln q_k - ln p_{t_k})
 *   rest: the teacher gives log probabilities, q_k = exp(teacher_k), and all tokens that are not listed are one more answer, q_r = 1 - sum q
 *   (0 where that is negative, or no such token is allowed: the q then add up to what the list has): + q_r (ln q_r - ln(1 - sum of p over the
 *   listed tokens))
 *   args        logits and tokens as for klay_tokens_forward, top = 0, num_tokens >= 1.  A negative token lists nothing; a token >= vocab
 *               gives NaN; of a token listed more than once the q add up in the gradient
 *   teacher     logits: device fp32 [rows, num_tokens], placed by rows and stride (elements); 0.001 <= temperature <= 1000
 *   loss        device [rows] fp32
 *   kept        as for klay_head_forward, for klay_distill_backward, and the call's own workspace: required
 * A row that lists nothing has loss 0 and no gradient.  A listed token that is not allowed and that the teacher gives mass to: +inf.  A NaN or +inf,
 * of a logit or of the teacher's, makes the loss of its row NaN.  Errors: as klay_tokens_forward.
 */
typedef struct klay_teacher {
    const float* logits;
    klay_rows rows;
    int64_t stride;
    double temperature;
    int32_t rest, reserved;
} klay_teacher;
klay_status klay_distill_forward(const klay_tokens_args* args, const klay_teacher* teacher, float* loss, void* kept, void* stream);

/*
 * klay_distill_backward -- its derivative with respect to the logits (the teacher is not differentiated), which must be as they were.
 *   dloss       device [rows] fp32;  dlogits device [rows, vocab] contiguous, of `dtype`; every entry is written, rounded once
 */
klay_status klay_distill_backward(const klay_tokens_args* args, const klay_teacher* teacher, const void* kept, const float* dloss,
                                  void* dlogits, void* stream);

/* The divergence straight from the network's last layer: logits, rows, workspace and gradients as for klay_head_forward and _backward. */
klay_status klay_head_distill_forward(const klay_head_args* args, const klay_teacher* teacher, float* loss, void* kept, void* workspace,
                                      size_t workspace_bytes, void* stream);
klay_status klay_head_distill_backward(const klay_head_args* args, const klay_teacher* teacher, const void* kept, const float* dloss,
                                       void* dhidden, void* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream);

/*
 * klay_scan_forward -- gated recurrence over sequences in a semiring (Section 4), the value of a chain of AND and OR gates of any length:
 *   h_t = a_t (x) h_{t-1} (+) x_t:  REAL: a h + x;  LOG: log(exp(a + h) + exp(x));  MAXLOG: max(a + h, x)
 *   gates, inputs   device [batch, time, channels] of `dtype` (KLAY_F32 in the log-domain semirings), channels next to each other,
 *               the two other strides in elements; at most 2^25 channels and 2^25 elements from one time step to the next
 *   offsets     NULL: `batch` sequences of `time` steps.  Otherwise batch = 1 and device int64 [sequences + 1]: sequence s is the rows
 *               offsets[s] .. offsets[s + 1] - 1, ascending, in 0 .. time; it may be empty.  Rows of no sequence get 0 as states.
 *   row_info    device int32 [time]; required with offsets, for klay_scan_backward, which reads what the forward call wrote
 *   initial     device fp32 [batch or sequences, channels]: the states before the first steps; NULL: 0 (LOG, MAXLOG: -inf)
 *   states      device [batch, time, channels] of `dtype`, contiguous: h, each rounded once from fp32
 *   final       device fp32 [batch or sequences, channels]: the states behind the last steps (of an empty sequence: its initial one); or NULL
 *   workspace   device, 16-byte aligned, klay_scan_workspace_bytes(args) bytes (for either direction); NULL where that is 0
 * Sums are in single.  Products of many gates, which may leave its range where the states themselves do not (gates above 1 behind a state of
 * 0), are held as mantissa and exponent then (REAL).
 * A state that is NaN or infinite (in the log domain: +inf) makes all behind it in its sequence and channel NaN or infinite.
 * Offsets that are none (descending, out of range) give undefined values, but no access outside the arrays.
 * Errors: KLAY_EINVAL, KLAY_ENOMEM (workspace too small), KLAY_EHIP.
 */
typedef struct klay_scan_args {
    int32_t dtype, semiring, device, channels;
    int64_t batch, time, sequences;
    const void* gates;
    const void* inputs;
    int64_t gates_batch_stride, gates_time_stride, inputs_batch_stride, inputs_time_stride;
    const int64_t* offsets;
    int32_t* row_info;
    const float* initial;
} klay_scan_args;
size_t klay_scan_workspace_bytes(const klay_scan_args* args);
klay_status klay_scan_forward(const klay_scan_args* args, void* states, float* final, void* workspace, size_t workspace_bytes, void* stream);

/*
 * klay_scan_backward -- derivative of a klay_scan_forward (REAL, LOG) with respect to gates, inputs and initial states.
 *   args        as for the forward call; REAL does not read inputs (may be NULL)
 *   states      as written by the forward call (16-bit types: dgates is made with the state before a step as it stands there, rounded)
 *   dstates     device [batch, time, channels] of `dtype`, contiguous, or NULL (no adjoint); dfinal fp32, or NULL
 *   dgates, dinputs   device [batch, time, channels] of `dtype`, contiguous; dinitial fp32; each may be NULL (not wanted)
 * A step whose value is log 0 passes nothing down.  Errors: as klay_scan_forward; MAXLOG is not differentiated (KLAY_EINVAL).
 */
klay_status klay_scan_backward(const klay_scan_args* args, const void* states, const void* dstates, const float* dfinal, void* dgates,
                               void* dinputs, float* dinitial, void* workspace, size_t workspace_bytes, void* stream);

/*
 * klay_scan_step -- one step for `rows` running sequences: state = gates (x) state (+) inputs, in place, and its copy in `dtype`.
 *   gates, inputs   device [rows, channels] of `dtype`;  state device fp32 [rows, channels];  out [rows, channels] of `dtype` or NULL
 * Channels next to each other, rows that many elements apart; rows of state and of out must not overlap.
 */
klay_status klay_scan_step(int32_t dtype, int32_t semiring, int32_t device, int64_t rows, int32_t channels, const void* gates,
                           int64_t gates_stride, const void* inputs, int64_t inputs_stride, float* state, int64_t state_stride, void* out,
                           int64_t out_stride, void* stream);

/* Message of the last failing call on this thread ("" if none). */
const char* klay_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* KLAY_H */
