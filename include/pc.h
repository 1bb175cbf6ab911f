/*
 * libpc -- forward (log-likelihood) and backward (PC flows) passes of a compiled probabilistic
 * circuit on one AMD gfx950 GPU.  Plain C ABI: raw pointers and sizes, no C++/torch types.
 *
 * Conventions used by every entry point
 *   - "device" pointers are hipMalloc-style GPU addresses owned by the caller; "host" pointers are
 *     ordinary CPU memory.  theta, tables, their flow arrays and the workspace must be 16-byte aligned
 *     (PC_ERR_ARG otherwise).  The handle (pc_circuit) owns only its compiled int32 tables and a few
 *     KB of reduction scratch.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Forward, backward
 *     and the EM step only enqueue kernels (no memset or copy nodes, no allocation); they never
 *     synchronise the device, so a caller may capture them into a HIP graph and replay it.  A kernel
 *     fault surfaces as PC_ERR_HIP from the next call that checks the runtime's error state.  Narrow layers share one launch
 *     whose workgroups wait for one another's results; should such a wait reach its limit of polls (pc_set_wait_limit),
 *     the launch ends, log-likelihoods and node flows that depend on the missing values are NaN, and every call on the
 *     handle that starts after that (forward, backward, EM step, profile read) returns PC_ERR_HIP.
 *   - Every call returns a pc_status; pc_last_error() gives a thread-local message for the last
 *     non-OK status.  No exceptions cross this boundary.
 *   - Node blocks hold K node slots.  The compiled node offset of user block u is (u+1)*K; rows
 *     0..K-1 are a reserved null block (log-probability 0, flow 0).  Parameter block p lives at
 *     theta[(p+1)*K*K ...]; theta[0 .. K*K) must be all zero (it backs the padding entries of the
 *     index tables, the "pseudo blocks with probability 0" of Sec. 4.3).  Inside a parameter block
 *     element (i, j) is at i*K + j, i = sum node in its block, j = child node in its block
 *     (the view(K_M, K_N) of Alg. 1).
 *   - tables[t][c][k]: probability of category c under node k of an input block that uses table t
 *     (category-major so that one (sample, variable) lookup reads K contiguous floats; the paper
 *     gives no input-layer layout).
 *   - Precision: fp32 data and fp32 accumulation everywhere.  Sum layers of K = 64 / 128 whose rows reduce over at least
 *     2048 child nodes, and parameter flows reduced over at least 4096 samples per parameter block, take each product
 *     as three bf16 MFMAs on operands split into a bf16 pair (hi + lo; the dropped lo x lo term is 2^-16 relative).
 *   - Environment switches, read once per process, for measurements and cross-checks (results stay within the same
 *     tolerances): PC_BF16=0 keeps every contraction on the fp32 matrix cores; PC_BF16_CT=1|2 forces the 64 x 32 or
 *     64 x 64 tile form of the bf16 sum kernels; PC_FORCE_GENERIC=1 (read by pc_compile) routes every block size
 *     through the one-thread-per-output kernels.
 */
#ifndef PC_H_
#define PC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pc_circuit pc_circuit;

typedef enum {
    PC_OK = 0,
    PC_ERR_ARG,              /* null pointer, negative size, id out of range, unsupported K      */
    PC_ERR_CYCLE,            /* the block graph is not a DAG                                    */
    PC_ERR_NOT_ALTERNATING,  /* sum block with a non-product child, product with a product child */
    PC_ERR_NOT_BLOCK_SPARSE, /* duplicate (parent, child) block pair, or an inner block w/o child */
    PC_ERR_TIE,              /* two sum blocks share some but not all of their parameter blocks  */
    PC_ERR_TOO_LARGE,        /* an index does not fit in int32                                  */
    PC_ERR_WORKSPACE,        /* workspace smaller than pc_workspace_bytes                       */
    PC_ERR_STATE,            /* pc_backward without a matching pc_forward                       */
    PC_ERR_HIP               /* the HIP runtime reported an error                               */
} pc_status;

/* Block-level DAG handed to pc_compile (all host pointers, read only, not retained).
 * Def. 1: input blocks carry a categorical distribution per node, product blocks multiply their
 * child blocks element-wise (node k of the block has node k of every child block as children),
 * sum blocks are fully connected to each of their child blocks through one K x K parameter block
 * (Sec. 4.2: every block pair is fully connected or unconnected). */
typedef struct {
    int32_t K;                 /* node block size K_M = K_N (Sec. 4.1), 1 <= K <= 128 (larger: PC_ERR_ARG); the matrix-core
                                  kernels serve K % 32 == 0, vector kernels every other K */
    int32_t n_blocks;
    int32_t root_block;        /* a sum block; its node 0 is the root n_r                        */
    const uint8_t *type;       /* [n_blocks] 0 input, 1 product, 2 sum                           */
    const int32_t *n_real;     /* [n_blocks] real nodes in the block, 1..K; slots n_real..K-1 are placeholders (Sec. 4.1
                                  footnote) of probability 0: the caller keeps their theta rows and table columns at 0.  A
                                  product node over a placeholder slot of any child has probability 0 as well, so a
                                  product block has no more useful nodes than its smallest child; equality of the
                                  counts is not required */
    const int64_t *child_ptr;  /* [n_blocks+1] CSR offsets into child / param_blk                */
    const int32_t *child;      /* [n_edges] child block ids                                      */
    const int32_t *param_blk;  /* [n_edges] parameter block id of a sum edge (equal ids = tied parameters,
                                  App. A.3); ignored for product edges                           */
    int32_t n_param_blocks;
    const int32_t *in_var;     /* [n_blocks] variable read by an input block                     */
    const int32_t *in_table;   /* [n_blocks] categorical table used by an input block            */
    int32_t n_vars, n_cats, n_tables;
    int32_t max_groups;        /* G of Alg. 2 (App. A.1)                                         */
    int32_t tol_permille;      /* tol of Alg. 2 in 1/1000                                        */
    int32_t product_scratch;   /* 0: every node's log-probability is kept for the backward pass.
                                  1: the memory-saving mode of Sec. 5 -- the log-probabilities of product blocks live in one
                                  scratch sized for the largest product layer and are recomputed in the backward pass just
                                  before the sum layer that reads them.  Needs the block order of pc_order_for_scratch. */
} pc_dag;

/* Compile once, reuse for every batch (Sec. 6.1).  Layers by longest-path depth (Sec. 3), groups by
 * the dynamic programme of App. A.1, forward index tensors sum_ids / prod_ids / param_ids (Sec. 4.3)
 * and backward index tensors ch_ids / par_ids / par_param_ids (App. A.2), for sum and product layers
 * alike.  Validation, depths and Alg. 2 run on the host; the graph transpose, the sorting of neighbour lists and
 * the filling of every table run as HIP kernels on `stream`; the call waits for them.  *out is set only on PC_OK. */
pc_status pc_compile(const pc_dag *dag, void *stream, pc_circuit **out);
/* The host half of pc_compile alone (validation, layering, Alg. 2, tables); touches no GPU.  The handle
 * serves pc_get_sizes / pc_get_layer / pc_copy_group / pc_workspace_*; forward, backward and the EM
 * step return PC_ERR_STATE on it, and pc_get_group reports NULL device pointers. */
pc_status pc_compile_host(const pc_dag *dag, pc_circuit **out);
void pc_destroy(pc_circuit *c);
const char *pc_last_error(void);

/* Collapse of consecutive sum / sum and product / product blocks (footnote to Def. 2): pc_compile accepts only DAGs
 * in which sum blocks have product children and product blocks have sum or input children (PC_ERR_NOT_ALTERNATING
 * otherwise); this optional pre-pass rewrites any other DAG of sum, product and input blocks into that form.  A
 * product block takes over the children of its product children; a sum block takes over the children of its sum
 * children with the K x K weight blocks multiplied (sum_j A[i][j] sum_k B[j][k] c_k = sum_k (A B)[i][k] c_k), several
 * paths to one child add up.  The circuit computes the same function; its parameters are those of the collapsed
 * circuit.  Host only; `theta` is a host array [n_param_blocks + 1][K][K].  Canonical form of the result:
 *   - edges keep the order of the original edges, a replaced edge expanding in place into its child's edges; a child
 *     reached twice keeps its first position (product blocks: PC_ERR_NOT_BLOCK_SPARSE);
 *   - blocks no longer reachable from the root are dropped, the others keep their order (block_map: old id -> new id, -1);
 *   - a sum block none of whose edges changed keeps its parameter blocks (and its ties), a changed one gets fresh
 *     blocks for all its edges; parameter blocks are renumbered in order of first use.
 * A sum block with an input child remains an error of pc_compile.  The handle owns every array it hands out
 * (pc_collapsed_dag: ready for pc_compile; max_groups, tol_permille, n_vars, n_cats, n_tables are copied). */
typedef struct pc_collapsed pc_collapsed;
pc_status pc_collapse(const pc_dag *dag, const float *theta, pc_collapsed **out);
/* Block order for product_scratch = 1 (Sec. 5, product values recomputed): the same DAG with its blocks renumbered --
 * input and sum blocks first (relative order kept), then the product blocks grouped by the depth of the sum blocks
 * that read them, so that the product blocks a sum layer reads are one contiguous range of ids.  A product block read
 * by sum blocks of several depths is copied, one copy per depth (it is then evaluated once for each of them; product
 * blocks carry no parameters, so log-likelihoods and parameter flows are those of the original circuit).  Parameter
 * block ids do not change; the result (pc_collapsed_dag; pc_collapsed_block_map: old id -> new id, for a copied block
 * its first copy; product_scratch already set) is owned by the handle. */
pc_status pc_order_for_scratch(const pc_dag *dag, pc_collapsed **out);
const pc_dag *pc_collapsed_dag(const pc_collapsed *r);
const float *pc_collapsed_theta(const pc_collapsed *r, int64_t *len);   /* [n_param_blocks + 1][K][K], block 0 zero */
const int32_t *pc_collapsed_block_map(const pc_collapsed *r);            /* [n_blocks of the input DAG]            */
void pc_collapsed_destroy(pc_collapsed *r);

typedef struct {
    int32_t K, n_blocks, n_layers;
    int64_t n_rows;            /* (n_blocks+1)*K rows of the node buffers                        */
    int64_t theta_len;         /* floats in theta / theta_flow: (n_param_blocks+1)*K*K           */
    int64_t tables_len;        /* floats in tables / table_flow: n_tables*n_cats*K               */
    int32_t n_vars, n_cats, n_tables;
} pc_sizes;
pc_status pc_get_sizes(const pc_circuit *c, pc_sizes *out);

/* Compiled layers, for inspection and bit-exact checks.  Layer 0 is the input layer. */
typedef struct {
    int32_t kind;              /* 0 input, 1 product, 2 sum                                      */
    int32_t depth;
    int32_t n_fwd_groups;      /* input layer: 1                                                 */
    int32_t n_bwd_groups;      /* input layer: 0                                                 */
} pc_layer_desc;
pc_status pc_get_layer(const pc_circuit *c, int32_t layer, pc_layer_desc *out);

/* One group of a layer.  dir 0 = forward tables, 1 = backward tables.
 *   sum / product layer, forward : ids = sum_ids [n_rows] (node offsets), nbr = prod_ids,
 *                                   par = param_ids [n_rows x width] (parameter offsets; product: zeros)
 *   sum / product layer, backward: ids = ch_ids, nbr = par_ids, par = par_param_ids
 *   input layer (dir 0, group 0) : ids = node offsets, nbr = variable per block, par = table per block, width 1
 * Pointers are device addresses owned by the handle. */
typedef struct {
    int32_t n_rows, width;
    const int32_t *ids, *nbr, *par;
} pc_group_desc;
pc_status pc_get_group(const pc_circuit *c, int32_t layer, int32_t dir, int32_t group, pc_group_desc *out);
/* Same tables copied to host arrays sized from pc_get_group (any of the three may be NULL). */
pc_status pc_copy_group(const pc_circuit *c, int32_t layer, int32_t dir, int32_t group,
                        int32_t *ids_host, int32_t *nbr_host, int32_t *par_host);

/* The kernel that serves a layer in a pass over B samples, as kernel traces name it with the template arguments that a rule
 * on sizes chooses ("k_chain<false>", "k_flow<1, 2, 1, true, false>"; of a layer in several launches, the first's), for inspection and tests.  dir 0:
 * the blocks of the layer are evaluated; dir 1: their flows go to their children, those of input blocks to the tables.  The
 * text is the calling thread's until its next such call. */
pc_status pc_get_kernel(const pc_circuit *c, int32_t layer, int32_t dir, int32_t B, const char **name);

/* Workspace (device, caller-owned) for batches of up to B samples.  It holds three node buffers
 * of n_rows x stride floats, row = node offset, samples contiguous (l in R^{N x B} of Sec. 4.3):
 *   l  log-probability residuals, F  node flows, N  log(F) - l of sum rows (the log_nf of Alg. 3 / 4; scratch otherwise),
 * one block buffer R of (n_blocks+1) x stride floats, row = node offset / K, and small per-batch
 * scratch.  The log-probability of node row n in sample b is  R[n / K][b] + l[n][b]  (R holds
 * integers; keeping the bulk of a large log-probability there leaves l accurate to ~1e-6).
 * stride = B rounded up to a multiple of 32; columns >= B behave as fully marginalised samples with
 * root flow 0. */
#define PC_MAX_BATCH 2097152   /* samples per call: kernels address a batch row with 32-bit byte offsets (else PC_ERR_TOO_LARGE) */
typedef struct {
    int64_t stride;            /* floats between consecutive rows                               */
    size_t l_offset, f_offset, n_offset, r_offset;   /* byte offsets into the workspace         */
    size_t total_bytes;
    int64_t l_rows;            /* rows of l and F: n_rows, or with product_scratch the null, input and sum blocks followed by
                                  the window of the largest product layer (product rows are not kept; N then has the
                                  null, input and sum rows only)                                           */
} pc_ws_layout;
pc_status pc_workspace_layout(const pc_circuit *c, int32_t B, pc_ws_layout *out);
pc_status pc_workspace_bytes(const pc_circuit *c, int32_t B, size_t *bytes);

/* Forward pass, Eq. (1) in log space: ll[b] = log p_root(x_b).
 *   theta  device [theta_len] fp32;  tables device [tables_len] fp32
 *   x      device int32 [B, n_vars] category per variable
 *   mask   device uint8 [B, n_vars] or NULL; non-zero marginalises that variable (Sec. 2)
 *   ll     device fp32 [B] (out).  A sample of probability 0 gives -inf.
 * Leaves every node's log-probability in the workspace for pc_backward. */
pc_status pc_forward(pc_circuit *c, const float *theta, const float *tables, const int32_t *x,
                     const uint8_t *mask, int32_t B, void *workspace, size_t workspace_bytes,
                     float *ll, void *stream);

/* pc_forward for callers that cannot allocate device memory or pass a workspace along: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments and same result as
 * pc_forward, but the workspace is a fixed array of PC_STATIC_SCRATCH_BYTES inside the library's device image (every
 * GPU the library runs on holds its copy until the process ends).  The call allocates nothing and records no timing
 * events; it only enqueues kernels on `stream`, pc_forward's but for one case: a circuit that is nothing but a chain of
 * single blocks of 32 or 64 nodes, with an input block of its own at each layer (an HMM of as many states), takes one
 * kernel with the same arithmetic while the batch is one at which pc_get_kernel names k_chain or k_walk64 for its sum
 * layers.  PC_ERR_WORKSPACE if pc_workspace_bytes(c, B) exceeds PC_STATIC_SCRATCH_BYTES.  All calls on one GPU share that
 * array: calls that overlap in time on one GPU (two streams, two threads, two circuits) race; every call writes what it reads.  It
 * leaves no state for pc_backward (which returns PC_ERR_STATE after it). */
#define PC_STATIC_SCRATCH_BYTES (64u << 20)
pc_status pc_forward_static(pc_circuit *c, const float *theta, const float *tables, const int32_t *x,
                            const uint8_t *mask, int32_t B, float *ll, void *stream);

/* Backward pass, Def. 2: node flows with F_root = 1, then
 *   theta_flow[param(n,c)] += sum_b theta_{n,c} p_c / p_n F_n        (Alg. 3; tied edges add up, App. A.3)
 *   table_flow[t][x_b,v][k] += sum_b F_n                              for observed variables
 * Both flow arrays are device fp32 with the layouts of theta / tables and are ACCUMULATED into
 * (mini-batch and full-batch EM, Sec. 6.1 / 6.3); either may be NULL to skip that part.
 * Must follow pc_forward on the same workspace, B, theta, tables, x, mask (else PC_ERR_STATE).
 * Samples of probability 0 contribute no flow. */
pc_status pc_backward(pc_circuit *c, const float *theta, const float *tables, const int32_t *x,
                      const uint8_t *mask, int32_t B, void *workspace, size_t workspace_bytes,
                      float *theta_flow, float *table_flow, void *stream);

/* EM update (Sec. 2; step size of App. C.3): per sum node, with Z = sum of its accumulated edge flows
 * and n_ch its number of real children,
 *   theta_new = (flow + pseudocount / n_ch) / (Z + pseudocount);  theta <- (1 - step) theta + step theta_new
 * (row unchanged if Z + pseudocount == 0; placeholder rows / columns unchanged); the same per table
 * column over the categories.  Sum blocks with tied parameters are normalised once over their summed
 * flows.  Zeroes theta_flow and table_flow afterwards. */
pc_status pc_em_step(pc_circuit *c, float *theta, float *tables, float *theta_flow, float *table_flow,
                     float step, float pseudocount, void *stream);

/* ---- Token models over circuits: predicting a variable, distilling from a teacher, decoding with beams ----
 * None of these calls but pc_get_mixture needs a handle: their operands are what the descriptors name, which is read before the call
 * returns and not retained.  They run on the device the calling thread has current.  Like the passes they only
 * enqueue kernels on `stream` and may be captured; a call with no rows (groups) does nothing and returns PC_OK.
 * Workspaces (16-byte aligned; NULL where none is needed) are scratch of one call: nothing in them is kept from call to call, calls
 * that overlap in time need one each.  Their bytes are those of the call that is asked about; a smaller batch may need more than a larger one.
 * Results do not depend on what a workspace holds, and are the same on every run. */
enum { PC_F32 = 0, PC_BF16 = 1, PC_F16 = 2 };   /* element types of rows of logits */

/* Input nodes of one variable with their weights in each sample: n_blocks blocks of K nodes; block j's weights are the rows
 * rows[j] .. rows[j] + K - 1 of `weights` (samples contiguous, `stride` floats between rows, stride >= B), its categorical
 * table is tables[table[j]].  rows / table are device arrays of n_blocks entries, or NULL: rows[j] = j * K, table[j] = j.  A
 * block whose rows or table lie outside [0, n_rows) / [0, n_tables) is left out.  K: 1 .. 128, n_rows >= K, n_cats <= 2^29 - 32.
 * Weights and table entries are not negative and at most 2^20 (probabilities).  Tables are 16-byte aligned; samples behind B are not used. */
typedef struct {
    int32_t K, n_blocks, n_cats, n_tables;
    int64_t n_rows, stride;
    const float *weights;
    const int32_t *rows, *table;
} pc_mixture;

/* The input blocks of variable `var` with their node flows F in a workspace that pc_backward has just filled (same
 * workspace and B as that call, else PC_ERR_STATE).  Where the variable is marginalised the flows are the probabilities of
 * its input nodes given the sample's evidence, so that pc_predict answers p(x_var | evidence).  (In a sample that observes
 * the variable they are the probabilities given that value too.)  Pointers stay valid until the workspace's next pass, as long as the handle. */
pc_status pc_get_mixture(const pc_circuit *c, int32_t var, int32_t B, const void *workspace, size_t workspace_bytes,
                         pc_mixture *out);

/* Predictive distribution:  logp[b][c] = log sum_j sum_k weights[rows[j] + k][b] * tables[table[j]][c][k],  b < B, c < n_cats,
 * ld >= n_cats floats between the rows of logp, which overlaps neither tables nor weights (PC_ERR_ARG).  A probability below FLT_MIN (a sample
 * without weights: all of them) gives -inf.  Sums are kept in fp32, products are off by at most 2^-22 of themselves, whatever batch a sample is in. */
pc_status pc_predict_workspace_bytes(const pc_mixture *m, int32_t B, size_t *bytes);
pc_status pc_predict(const pc_mixture *m, const float *tables, int32_t B, float *logp, int64_t ld, void *workspace,
                     size_t workspace_bytes, void *stream);

/* Its flows for a gradient dlogp of an objective with respect to logp, the weights held fixed (the responsibilities of an
 * EM step):
 *   flow[t][c][k] = tables[t][c][k] * sum over b and the blocks j of table t of weights[rows[j] + k][b] * dlogp[b][c] / exp(logp[b][c]),
 * which is the objective's gradient with respect to log tables[t][c][k];  table_flow = scale * flow for the tables that the mixture
 * names, added to what is there where `accumulate` is set.  With dlogp = -q (a loss -sum q logp, q >= 0) and scale = -1 these are
 * the flows of an EM step on soft targets, ready for pc_em_step.  Entries of logp below log FLT_MIN add nothing.  Sums are kept in
 * fp32, products weights * dlogp / exp(logp) are off by at most 2^-22 of themselves (by 2^-102 of the weight where that is more).
 * table_flow is 16-byte aligned, laid out like the tables, and overlaps neither them nor the weights, logp or dlogp (PC_ERR_ARG); flows of
 * tables that no block names stay as they are. */
pc_status pc_predict_backward_workspace_bytes(const pc_mixture *m, int32_t B, size_t *bytes);
pc_status pc_predict_backward(const pc_mixture *m, const float *tables, int32_t B, const float *logp, int64_t logp_ld,
                              const float *dlogp, int64_t dlogp_ld, float scale, int32_t accumulate, float *table_flow,
                              void *workspace, size_t workspace_bytes, void *stream);

/* Distillation from a teacher's top logits.  Per row, with temperature T:
 *   q_j  = softmax over the listed entries of teacher_j / T, or exp(teacher_j / T - teacher_lse) where the teacher's own
 *          log-normaliser (at T) over its whole vocabulary is given
 *   logp = log-softmax of student / T over its n_cats entries, or the row itself where `normalised` (log-probabilities, T = 1)
 *   loss = sum_j q_j (log q_j - logp[ids_j]);   dloss / dstudent_c = (p_c sum_j q_j - sum_{j: ids_j = c} q_j) / T,
 * without the p_c term where `normalised` (then -gradient is the soft target of pc_predict_backward).
 * ids outside [0, n_cats) are no entries (padding of short lists: -1), as are teacher logits of -inf; a category listed twice counts
 * twice.  A row without entries has loss 0 and gradient 0 whatever the student's row holds.  A student logit of -inf has p = 0;
 * loss is +inf where such a category, or any in a row of nothing else, is listed with q > 0.  NaN and +inf in a row make its
 * results NaN (a `normalised` row: its loss, where they are listed; its gradient is -q whatever it holds). */
#define PC_MAX_TOP 1024
typedef struct {
    int64_t rows;
    int32_t n_cats, top;                         /* entries of a student row; of a teacher's list, 1 .. PC_MAX_TOP */
    const void *student;  int32_t student_type;  int64_t student_ld;     /* ld: elements between rows              */
    const int32_t *ids;                          int64_t ids_ld;
    const void *teacher;  int32_t teacher_type;  int64_t teacher_ld;
    const float *teacher_lse;                    /* [rows] or NULL                                                  */
    float temperature;                           /* finite, and log2(e) / temperature too: at least 4.3e-39         */
    int32_t normalised;
} pc_distill;
pc_status pc_distill_workspace_bytes(const pc_distill *d, size_t *bytes);
/* loss: device fp32 [rows]; stats: device fp32 [rows][2], the row's maximum m and log sum exp((student - m) / T) (zeros where
 * `normalised`), for pc_distill_backward.  workspace: reserved; pc_distill_workspace_bytes says 0, the call reads neither and takes NULL. */
pc_status pc_distill_forward(const pc_distill *d, void *workspace, size_t workspace_bytes, float *loss, float *stats, void *stream);
/* dstudent[r][c] = scale * dloss[r] * gradient, rounded once to the student's type; dloss: device fp32 [rows] or NULL (ones);
 * dstudent_ld >= n_cats elements between rows; dstudent may be the student's rows themselves (same ld), else it does not overlap them (PC_ERR_ARG).  Rows whose scale * dloss is 0
 * get 0 whatever they hold. */
pc_status pc_distill_backward(const pc_distill *d, const float *stats, const float *dloss, float scale, void *dstudent,
                              int64_t dstudent_ld, void *stream);

/* Beam search: of all beams and categories of a group the n_out best.  Candidate (beam, c) has the score
 * running[beam] + z, z = scores[beam][c], minus log sum_c' exp(scores[beam][c']) where `normalise` (rows of logits), added in 64 bits.
 * The exponentials are fp32, their sum over a row and its logarithm 64 bits: the logarithm is off by at most 2^-17 (1e-7 for 50257 normal
 * logits), and candidates of different beams whose scores lie closer may change places.
 * A finished beam (done != 0) has the one candidate done_token with z = 0; its row is not read.  Order: higher score, then lower
 * beam, then (within a beam) higher z, then lower category.  Candidates that are no numbers or whose beam's running score is
 * no number below +inf count as -inf, as do all of a row whose log-normaliser is no finite number; candidates of -inf come last, by
 * beam and category.  So a group's output is complete and the same on every run. */
#define PC_MAX_BEAMS 64
#define PC_MAX_BEAM_OUT 64
typedef struct {
    int32_t groups, beams, n_cats, n_out;        /* beams 1 .. PC_MAX_BEAMS; n_out 1 .. PC_MAX_BEAM_OUT, at most beams * n_cats */
    const void *scores;  int32_t scores_type;  int64_t scores_ld;        /* [groups * beams][ld]                  */
    int32_t normalise;
    const float *running;                        /* [groups][beams] or NULL (zeros)                               */
    const uint8_t *done;                         /* [groups][beams] or NULL                                       */
    int32_t done_token;
} pc_beam;
pc_status pc_beam_workspace_bytes(const pc_beam *a, size_t *bytes);
/* out_scores (fp32), parents (beam within the group), tokens: device, [groups][n_out], best first.  workspace: 16-byte aligned.
 * Outputs overlap neither each other nor scores, running or done (PC_ERR_ARG), but out_scores may be `running` where n_out == beams. */
pc_status pc_beam_select(const pc_beam *a, void *workspace, size_t workspace_bytes, float *out_scores, int32_t *parents,
                         int32_t *tokens, void *stream);
/* What each survivor takes along: row g * n_out + i of dst = row g * beams + parents[g][i] of src, for up to PC_MAX_STATES arrays
 * of rows in one launch (evidence rows x and mask, hidden states, caches).  Strides are in bytes; a row's bytes behind row_bytes
 * are not touched.  dst, from its first row to its last, must not overlap any src or other dst (PC_ERR_ARG).  A parent outside [0, beams) leaves its row of dst as it was. */
#define PC_MAX_STATES 16
typedef struct {
    const void *src;
    void *dst;
    int64_t row_bytes, src_stride, dst_stride;
} pc_state;
pc_status pc_beam_reorder(const pc_state *states, int32_t n_states, const int32_t *parents, int32_t groups, int32_t beams,
                          int32_t n_out, void *stream);

/* Per-kernel timing for benchmarks (the measurement protocol, not an operation of the paper).  While enabled,
 * every kernel launch of forward / backward / EM is bracketed by two HIP events on the launch stream.
 * pc_profile_read waits for the recorded events (it synchronises with the work launched so far) and returns
 * the running totals per kernel class since pc_profile_enable; class names: pc_kernel_class_name(i),
 * i < n_classes ("sum_fwd", "sum_bwd_child", "sum_bwd_param", "prod_fwd", ...). */
#define PC_MAX_KERNEL_CLASSES 16
typedef struct {
    int32_t n_classes;
    int64_t launches[PC_MAX_KERNEL_CLASSES];
    double ms[PC_MAX_KERNEL_CLASSES];
    int64_t bf16_launches[PC_MAX_KERNEL_CLASSES];   /* of those, launches whose contraction ran as bf16-split products */
} pc_profile;
pc_status pc_profile_enable(pc_circuit *c, int32_t on);
pc_status pc_profile_read(pc_circuit *c, pc_profile *out);
const char *pc_kernel_class_name(int32_t cls);

/* Polls after which a wait inside a dataflow launch is given up (2^22 after pc_compile: some seconds).  The limit is the
 * handle's and applies from the next call on; 0 gives up on the first value that is not there yet, which is how the error
 * path is tested.  Any other limit than the first also sends chains of single blocks of 32 or 64 nodes, which are walked without waits
 * (k_chain, k_walk64), through a launch that waits; log-likelihoods and flows agree within the same tolerances. */
pc_status pc_set_wait_limit(pc_circuit *c, int32_t polls);

/* Achievable peaks of the device the calling thread has current, for quoting beside the published ones (measurement
 * protocol).  Both time `reps` launches of a plain kernel with HIP events on `stream` and wait for them.
 *   pc_measure_copy      16-byte streaming copy of `bytes` from src to dst (device, 16-byte aligned, not overlapping);
 *                        *gb_per_s = (bytes read + bytes written) / time
 *   pc_measure_mfma_f32  register-only loop of v_mfma_f32_32x32x2_f32 on every SIMD; `out` is a device buffer of at
 *                        least 2 MiB that receives the accumulators; *tflops = multiply-add flops / time */
pc_status pc_measure_copy(const void *src, void *dst, size_t bytes, int32_t reps, void *stream, double *gb_per_s);
pc_status pc_measure_mfma_f32(void *out, size_t out_bytes, int32_t reps, void *stream, double *tflops);

#ifdef __cplusplus
}
#endif
#endif /* PC_H_ */
