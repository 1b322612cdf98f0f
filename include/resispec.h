/*
 * resispec.h -- C ABI of libresispec.so, the MI355X (gfx950) verification step of
 * ResiSpec multi-candidate speculative sampling.
 *
 * What it computes (paper: "ResiSpec: Enhancing Multi-Candidate Speculative
 * Sampling via Residual Distribution Shaping"):
 *   for every node of a batch of draft trees, the temperature softmax of the
 *   target and draft logits over the whole vocabulary (Preliminary), the
 *   sequential accept/reject of the node's candidates with acceptance
 *   min(1, R(x)/D(x)) against the current residual R (Eq. 2, Algorithm 1), the
 *   residual update after each rejection -- the standard norm(max(R - D, 0))
 *   (Eq. 1/2, mode RS_MODE_SPECINFER) or ResiSpec's proxy-shaped residual
 *   norm(max(R - GetProxy(R, D, x), 0)) (Algorithm 1, mode RS_MODE_RESISPEC) --
 *   and the inverse-CDF draw from the final residual when every candidate is
 *   rejected; then a walk from each root that follows accepted children and
 *   returns the accepted tokens (Preliminary, tree-structured verification).
 * Around it: the draft step, sampling from rows of logits, beam search's step, and the pages,
 * slots and rows of a paged cache under a draft tree.
 *
 * Conventions shared by every entry point:
 *   - All array arguments are DEVICE pointers owned by the caller unless stated
 *     otherwise.  The library never allocates, frees or keeps them.
 *   - Calls are asynchronous on `stream` (a hipStream_t; NULL = the default
 *     stream).  Results are valid once the stream reaches the call.  No entry
 *     point synchronises the device.
 *   - Argument errors are returned synchronously as rs_status and nothing is
 *     launched.  Data faults found on the device (bad token ids, a candidate
 *     with zero draft probability, a malformed tree, out-of-range uniforms) are
 *     reported per row / per sequence in out_status (rs_seq_status); the outputs
 *     of such a row/sequence are -1.
 *   - Logits rows are contiguous over the vocabulary.  fp32 or bf16 (raw bf16,
 *     widened exactly to fp32 in the kernel).  Rows take 16-byte loads, whatever V
 *     and the base pointer's alignment (a byte length that is a multiple of 16 on a
 *     16-byte aligned base is somewhat faster); rows shorter than 16 bytes, and base
 *     pointers not aligned to their elements, are handled element by element.
 *   - Uniforms are fp32 in [0, 1).  The accept test is strict: u < ratio.
 *   - Thread safety: calls are re-entrant.  What the library keeps on each GPU between
 *     calls, the pool of resispec_verify below and the scratch of
 *     resispec_verify_tree_noalloc, does not affect results (the latter's calls must not
 *     overlap).
 */
#ifndef RESISPEC_H
#define RESISPEC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define RESISPEC_ABI_VERSION 3

/* Largest number of candidates (children) one node may have. */
#define RS_MAX_CANDIDATES 64
/* Largest supported vocabulary. */
#define RS_MAX_VOCAB (1 << 22)

typedef enum {
    RS_OK = 0,
    RS_ERR_INVALID_ARG = 1,  /* NULL pointer, non-positive size, T <= 0, unknown mode/dtype */
    RS_ERR_WORKSPACE = 2,    /* workspace NULL or smaller than resispec_workspace_bytes() */
    RS_ERR_UNSUPPORTED = 3,  /* size beyond RS_MAX_VOCAB / RS_MAX_CANDIDATES, or a row
                                group that cannot run on this device */
    RS_ERR_HIP = 4           /* a HIP launch error */
} rs_status;

/* Per-row / per-sequence device-side status (out_status). */
typedef enum {
    RS_SEQ_OK = 0,
    RS_SEQ_BAD_TOKEN = 1,        /* candidate id outside [0, V) */
    RS_SEQ_ZERO_DRAFT = 2,       /* a tested candidate has current draft probability 0 */
    RS_SEQ_UNDERFLOW = 3,        /* softmax or residual total is 0 (e.g. an all -inf row) */
    RS_SEQ_BAD_TREE = 4,         /* parent[.,0] != -1 or parent[n] not in [0, n) */
    RS_SEQ_BAD_UNIFORM = 5,      /* a used uniform outside [0, 1) */
    RS_SEQ_DEPTH_EXCEEDED = 6,   /* accepted path longer than max_depth */
    RS_SEQ_TOO_MANY_CHILDREN = 7, /* a node with more than RS_MAX_CANDIDATES children */
    RS_SEQ_GROUP_TIMEOUT = 8,    /* row groups: a workgroup did not receive the others'
                                    slot totals of a pass within 20 ms */
    RS_SEQ_DEFERRED = 9,         /* node outcomes of resispec_decide_nodes only: the node
                                    rejected its one candidate, or is a leaf, and its draw
                                    is left to the walk (resispec_walk_draw), which makes it
                                    only where a walk ends */
    RS_SEQ_BAD_PARAM = 10,       /* rows with sampling settings of their own (rs_filter): one
                                    of them is out of its range; a sequence's score, length,
                                    count or parent is */
    RS_SEQ_BAD_PAGE = 11,        /* a page number or slot outside the cache */
    RS_SEQ_NO_ROOM = 12          /* resispec_plan_cache: not enough free pages, or slots */
} rs_seq_status;

typedef enum { RS_MODE_RESISPEC = 0, RS_MODE_SPECINFER = 1 } rs_mode;
typedef enum { RS_F32 = 0, RS_BF16 = 1 } rs_dtype;

typedef struct {
    int32_t mode;                /* rs_mode */
    int32_t logits_dtype;        /* rs_dtype, same for target and draft */
    float   temperature;         /* > 0; softmax((l - max l) / T) for target and draft alike */
    int32_t without_replacement; /* 1: candidates of a node were drawn without replacement;
                                    each rejected id leaves the draft, which is renormalised
                                    before the next sibling is tested */
    int32_t bonus;               /* tree only: 1 = a walk that ends at a leaf draws one more
                                    token from that leaf's target distribution */
} rs_params;

/*
 * Flat verify: row b of the target/draft logits is one position with k candidates
 * (Eq. 2 / Algorithm 1 on a single node per row).
 *   target_logits, draft_logits : [B][V] fp32 or bf16 (prm->logits_dtype)
 *   cand_ids                    : [B][k] int32, verified in column order
 *   u_accept                    : [B][k] fp32, column i is the uniform of candidate i
 *   u_resample                  : [B]    fp32, uniform of the final draw
 *   out_token                   : [B] int32  accepted candidate id, or the id drawn
 *                                 from the final residual when all k are rejected
 *   out_accepted_len            : [B] int32  1 if a candidate was accepted, else 0
 *   out_status                  : [B] int32  rs_seq_status; may be NULL
 * k = 0 draws directly from the target distribution.  B = 0 is a no-op.
 * Batches of few long rows (up to 128 rows of at least 160 KiB, and the same for the node
 * rows of resispec_verify_tree and resispec_verify_nodes) take several workgroups a row,
 * whose exchange states come from a pool of 128 that the library keeps on each GPU; calls may
 * overlap on any streams and threads, and replay from graphs.  The results are the same bit
 * for bit, outputs are written with the outcomes and not before, and RS_SEQ_GROUP_TIMEOUT is
 * not reported: a row whose workgroups lose touch (20 ms), and every row of a call that
 * meets others of its kind and would not have a CU for each workgroup, is done by one
 * workgroup.
 */
rs_status resispec_verify(const void* target_logits, const void* draft_logits,
                          const int32_t* cand_ids, const float* u_accept,
                          const float* u_resample, int32_t B, int32_t V, int32_t k,
                          const rs_params* prm, int32_t* out_token,
                          int32_t* out_accepted_len, int32_t* out_status, void* stream);

/*
 * Tree verify over B sequences of N nodes each (node 0 = root): Algorithm 1 at every node
 * (accept test Eq. 2; residual update Eq. 1/2 or GetProxy by prm->mode), then the walk
 * down the accepted children of the tree-structured verification (§Preliminary).
 *   target_logits, draft_logits : [B][N][V]; row n is the target / draft distribution
 *                                 over the tokens that follow node n (the distribution
 *                                 node n's children were drawn from).  Draft rows of
 *                                 leaf nodes are never read.
 *   node_token                  : [B][N] int32 token of each node (entry 0 ignored)
 *   parent                      : [B][N] int32 parent node, parent[.,0] = -1 and
 *                                 parent[.,n] in [0, n) (topological numbering)
 *   u_accept                    : [B][N] fp32, entry n is used when node n is tested
 *   u_resample                  : [B][N] fp32, entry n is used when node n draws from its
 *                                 final residual (all children rejected) or its bonus
 *   max_depth                   : >= depth of the deepest node; out_tokens row width is
 *                                 max_depth + 1
 *   out_tokens                  : [B][max_depth+1] int32 accepted draft tokens followed by
 *                                 the drawn token, padded with -1
 *   out_accepted_len            : [B] int32 number of accepted draft tokens (-1 on a fault)
 *   out_status                  : [B] int32 rs_seq_status; may be NULL
 *   workspace                   : device buffer of at least resispec_workspace_bytes(B, N)
 *                                 bytes (per-node outcomes); contents on entry are ignored
 * Children of a node are tested in ascending node index.  Every node's outcome is
 * computed independently (each node owns its uniforms), then a walk from the root
 * follows accepted children; the result equals the sequential walk.
 */
rs_status resispec_verify_tree(const void* target_logits, const void* draft_logits,
                               const int32_t* node_token, const int32_t* parent,
                               const float* u_accept, const float* u_resample,
                               int32_t B, int32_t N, int32_t V, int32_t max_depth,
                               const rs_params* prm, int32_t* out_tokens,
                               int32_t* out_accepted_len, int32_t* out_status,
                               void* workspace, size_t workspace_bytes, void* stream);

/*
 * The all-nodes schedule of resispec_verify_tree with deferred draws (same arguments, same
 * results, bit for bit).  A node's draw from its final residual, and a leaf's bonus draw,
 * matter only where a walk ends (§Preliminary, tree-structured verification: the walk
 * draws once, at the node where it stops), so they are made there.  Two launches:
 *   - every node row with children takes pass 1 (the softmax statistics of Preliminary)
 *     and its tests (Eq. 2, Algorithm 1); a row with several candidates also takes the
 *     rejection passes its later tests need, and draws at once if it rejects them all; a
 *     row with one candidate that it rejects keeps its pass-1 slot totals in the
 *     workspace instead of drawing (no rejection pass re-reads its logits); a leaf's row,
 *     which serves only its bonus draw, is not read;
 *   - one workgroup per sequence walks the decisions and, where the walk ends at such a
 *     row, takes it up again: the residual pass of its rejection (Eq. 1/2 or GetProxy)
 *     over that row alone, or a leaf's pass 1, then the inverse-CDF draw, with the same
 *     arithmetic on the same values as resispec_verify_tree.
 *   workspace : device buffer of at least resispec_deferred_workspace_bytes(B, N) bytes,
 *               16-byte aligned (node outcomes, then 2 KiB of slot totals per node row);
 *               contents on entry are ignored.  Calls that overlap on one workspace race.
 * Errors and statuses as resispec_verify_tree.
 */
rs_status resispec_verify_tree_deferred(const void* target_logits, const void* draft_logits,
                                        const int32_t* node_token, const int32_t* parent,
                                        const float* u_accept, const float* u_resample,
                                        int32_t B, int32_t N, int32_t V, int32_t max_depth,
                                        const rs_params* prm, int32_t* out_tokens,
                                        int32_t* out_accepted_len, int32_t* out_status,
                                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * The two launches of resispec_verify_tree_deferred, for callers that schedule them
 * separately (same kernels, same results):
 *   resispec_decide_nodes: every node's tests into `workspace`; node outcomes (see
 *     resispec_node_outcomes, which reads this workspace too) are the accepted child,
 *     the drawn token of a row with several candidates that rejected them all, a fault,
 *     or RS_SEQ_DEFERRED;
 *   resispec_walk_draw: the walk from each root over those outcomes, with the deferred
 *     draw where a walk ends (same inputs, and the workspace written by
 *     resispec_decide_nodes with the same B and N, earlier on the same stream); it
 *     records the outcome of each node it draws for in the workspace.
 * resispec_walk over such a workspace draws nothing: a walk that ends at a deferred node
 * reports RS_SEQ_DEFERRED as its status.
 */
rs_status resispec_decide_nodes(const void* target_logits, const void* draft_logits,
                                const int32_t* node_token, const int32_t* parent,
                                const float* u_accept, const float* u_resample,
                                int32_t B, int32_t N, int32_t V, const rs_params* prm,
                                void* workspace, size_t workspace_bytes, void* stream);

rs_status resispec_walk_draw(const void* target_logits, const void* draft_logits,
                             const int32_t* node_token, const int32_t* parent,
                             const float* u_accept, const float* u_resample,
                             int32_t B, int32_t N, int32_t V, int32_t max_depth,
                             const rs_params* prm, void* workspace, size_t workspace_bytes,
                             int32_t* out_tokens, int32_t* out_accepted_len,
                             int32_t* out_status, void* stream);

/* Workspace bytes resispec_verify_tree_deferred needs for B sequences of N nodes (0 if
 * B <= 0 or N <= 0). */
size_t resispec_deferred_workspace_bytes(int32_t B, int32_t N);

/*
 * resispec_verify_tree without a caller workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc).  Same arguments, kernels and results as resispec_verify_tree; the
 * per-node outcomes go to a static device array of the library (one per GPU, held until
 * the process ends) sized for RS_NOALLOC_MAX_ROWS node rows (768 KiB).  The call
 * allocates nothing and nothing needs clearing: every call writes all B * N outcomes
 * before its walk reads them.  All calls on one GPU share that array, so the outcomes of
 * calls that overlap on one GPU (on different streams, or from different threads) race
 * (theirs alone: other calls are not affected); calls ordered on one stream do not.
 * RS_ERR_UNSUPPORTED when B * N > RS_NOALLOC_MAX_ROWS; RS_ERR_HIP if the array's device
 * address cannot be found; otherwise the errors of resispec_verify_tree.
 */
#define RS_NOALLOC_MAX_ROWS 65536
rs_status resispec_verify_tree_noalloc(const void* target_logits, const void* draft_logits,
                                       const int32_t* node_token, const int32_t* parent,
                                       const float* u_accept, const float* u_resample,
                                       int32_t B, int32_t N, int32_t V, int32_t max_depth,
                                       const rs_params* prm, int32_t* out_tokens,
                                       int32_t* out_accepted_len, int32_t* out_status,
                                       void* stream);

/*
 * Path-only schedule of resispec_verify_tree (same arguments without the workspace, same
 * results): one workgroup per sequence walks its tree from the root and verifies only
 * the nodes the walk reaches, one after another (Preliminary, tree-structured
 * verification: a node is verified only after its parent accepted it).  It reads the
 * rows of about accepted_len + 1 nodes per sequence instead of all N, and runs
 * B workgroups.  Per-node outcomes are the same functions of the node's rows and
 * uniforms as in the all-nodes schedule, so the tokens, lengths and statuses are
 * identical, faults included: both report only what the walk meets (a malformed
 * parent array is met at the root, whose row checks the whole array).
 */
rs_status resispec_verify_tree_path(const void* target_logits, const void* draft_logits,
                                    const int32_t* node_token, const int32_t* parent,
                                    const float* u_accept, const float* u_resample,
                                    int32_t B, int32_t N, int32_t V, int32_t max_depth,
                                    const rs_params* prm, int32_t* out_tokens,
                                    int32_t* out_accepted_len, int32_t* out_status, void* stream);

/*
 * The path-only schedule (§Preliminary walk, Algorithm 1 at each node it reaches) with row
 * groups, for batches too small to fill the device with one workgroup per sequence (same
 * results as resispec_verify_tree_path and resispec_verify_tree, bit for bit). Each
 * sequence gets `group_size` 512-thread workgroups that verify every row of its walk
 * together: each sweeps its share of the row's slots in every pass, and after a pass they
 * exchange their slots' totals through `workspace` (64-bit words tagged with the pass, so
 * a reader waits for the words of the current pass and no fence is needed).  The group
 * forms only when all its workgroups have started within 20 us of the first; otherwise
 * the first to give up waiting does the sequence alone (same results).  Every wait is
 * bounded: a workgroup that does not receive the others' totals within 20 ms reports
 * RS_SEQ_GROUP_TIMEOUT.
 *   group_size      : 0 = automatic (as many members as the device holds at once, up to
 *                     16 and to one per 4 slots of a row; 1 when that is under 2 or
 *                     workspace is NULL), 1 = one workgroup per sequence,
 *                     2..16 = that many (RS_ERR_UNSUPPORTED if B * group_size workgroups
 *                     cannot be resident at once or if a row has fewer slots than
 *                     members; rows that are not 16-byte aligned may be given as many
 *                     members as they have runs of 256 elements, and run with as many
 *                     as they have slots)
 *   workspace       : device buffer of at least resispec_path_workspace_bytes(B, V) bytes,
 *                     16-byte aligned, caller-owned; its counters and exchange words are
 *                     zeroed by the call itself (on `stream`) before the verification
 *                     kernel, and its residual rows need no initial contents; NULL allowed
 *                     when group_size is 0 or 1 (the later rejection passes then re-derive
 *                     the residual from the logits: same results; they also do so when B *
 *                     group_size exceeds the device's compute units, where the cache's
 *                     traffic costs more than it saves).  Calls that overlap on one
 *                     workspace race.
 * Other arguments, outputs and statuses as resispec_verify_tree_path.
 */
rs_status resispec_verify_tree_path_group(const void* target_logits, const void* draft_logits,
                                          const int32_t* node_token, const int32_t* parent,
                                          const float* u_accept, const float* u_resample,
                                          int32_t B, int32_t N, int32_t V, int32_t max_depth,
                                          const rs_params* prm, int32_t* out_tokens,
                                          int32_t* out_accepted_len, int32_t* out_status,
                                          int32_t group_size, void* workspace,
                                          size_t workspace_bytes, void* stream);

/*
 * resispec_verify_tree (Algorithm 1 at every node, §Preliminary walk) with row groups, for
 * batches of few rows (same results, bit for bit): every node row gets `group_size`
 * 512-thread workgroups that verify it together, exchanging slot totals through the
 * workspace with bounded waits like the path schedule's row groups (a group that does not
 * form within 20 us is done by one of its workgroups alone; RS_SEQ_GROUP_TIMEOUT after 20
 * ms without the others' totals), then the walk runs as in resispec_verify_tree.
 *   group_size : 0 = automatic (at most one workgroup per CU for B * N rows, up to 8
 *                members per row, one per 8 slots of a row and one per 40 KiB of a row's
 *                logits, none below 160 KiB; 1 = the ordinary one-workgroup row kernel
 *                when that is under 2),
 *                1 = the ordinary kernel,
 *                2..16 = that many (RS_ERR_UNSUPPORTED if B * N * group_size workgroups
 *                cannot be resident at once or a row has fewer slots than members; rows
 *                that are not 16-byte aligned may be given up to two workgroups a CU, and
 *                as many members as they have runs of 256 elements, and run with as many
 *                as there is room and slots for)
 *   workspace  : device buffer of at least resispec_tree_group_workspace_bytes(B, N)
 *                bytes, 16-byte aligned, caller-owned (node outcomes, then one group
 *                state per row; its counters are zeroed by the call itself on `stream`).
 *                Calls that overlap on one workspace race.
 * Other arguments, outputs and statuses as resispec_verify_tree.
 */
rs_status resispec_verify_tree_group(const void* target_logits, const void* draft_logits,
                                     const int32_t* node_token, const int32_t* parent,
                                     const float* u_accept, const float* u_resample, int32_t B,
                                     int32_t N, int32_t V, int32_t max_depth, const rs_params* prm,
                                     int32_t* out_tokens, int32_t* out_accepted_len,
                                     int32_t* out_status, int32_t group_size, void* workspace,
                                     size_t workspace_bytes, void* stream);

/* Workspace bytes resispec_verify_tree_group needs (0 if B <= 0 or N <= 0). */
size_t resispec_tree_group_workspace_bytes(int32_t B, int32_t N);

/* The group size resispec_verify_tree_group chooses with group_size = 0 for B * N rows
 * of V elements (16-byte aligned rows assumed), on the current device; -1 for invalid
 * arguments.  Host only: launches nothing. */
int32_t resispec_tree_group_size(int32_t B, int32_t N, int32_t V, const rs_params* prm);

/* Testing hook: the time limits of row groups in later launches of this process, in
 * ticks of the device's 100 MHz wall clock; UINT64_MAX restores a default.
 *   barrier_ticks   : every wait of a formed group for its members' totals (default
 *                     2,000,000 = 20 ms); a small limit makes groups report
 *                     RS_SEQ_GROUP_TIMEOUT instead of waiting, which is how the tests
 *                     exercise that path
 *   formation_ticks : the wait for a group's workgroups to start (default 2,000 = 20 us);
 *                     0 makes nearly every group fall back to one workgroup
 * Not for concurrent use with launches on other threads.  Always RS_OK. */
rs_status resispec_debug_set_group_waits(uint64_t barrier_ticks, uint64_t formation_ticks);

/* Testing hook: how many of the pool's group states (resispec_verify, above) are in use, and
 * workgroups counted, on the current device once it has been synchronised, which the call
 * does; 0 unless something went wrong, -1 for a HIP error. */
int32_t resispec_debug_pool_held(void);

/* Testing hook: the next n launches of the pool's groups in this process count as failed
 * (the calls return RS_ERR_HIP and their states go back); 0 ends that.  Always RS_OK. */
rs_status resispec_debug_fail_pool_launches(int32_t n);

/* Workspace bytes resispec_verify_tree_path_group needs for B sequences of V-element rows
 * (0 if B <= 0, V <= 0 or V > RS_MAX_VOCAB): one row-group state per sequence, then two
 * fp32 rows per sequence (V rounded up to a multiple of 1024 each), in which the ResiSpec
 * rejection passes after a row's second rejection keep the residual of the previous pass
 * and the draft's masses instead of re-deriving them from the logits through the chain
 * of earlier proxies (Algorithm 1 loop: each rejection updates R from the current R and
 * D). */
size_t resispec_path_workspace_bytes(int32_t B, int32_t V);

/* The group size resispec_verify_tree_path_group chooses with group_size = 0 for B
 * sequences of V-element rows (16-byte aligned rows assumed), on the current device;
 * -1 for invalid arguments.  Host only: launches nothing. */
int32_t resispec_path_group_size(int32_t B, int32_t V, const rs_params* prm);

/*
 * The draft step that precedes verification (Preliminary: candidates are drawn from the
 * draft distribution; Algorithm 1 draws x_i ~ D and r_i ~ Uniform(0, 1)), on the device:
 *   - every node's uniforms: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC'11) of
 *     counter (n, b, offset low word, offset high word) under key (seed low word, seed
 *     high word); word 0 -> u_accept[b][n], word 1 -> u_resample[b][n], word 2 -> the
 *     uniform that draws node n's own token; a word w maps to (w >> 8) * 2^-24;
 *   - every node's children's tokens, drawn from softmax(draft[b][n] / T) by inverse CDF
 *     in ascending vocabulary order, children in ascending node index; with
 *     prm->without_replacement each draw removes its token (and renormalises) before the
 *     next.
 *   draft_logits : [B][N][V] (prm->logits_dtype); draft rows of leaves are not read
 *   parent       : [B][N] int32, as for resispec_verify_tree
 *   node_token   : [B][N] int32 out; entry 0 = -1.  A node whose draft row has no usable
 *                  mass, or which has more than RS_MAX_CANDIDATES children, leaves its
 *                  children at -1; a malformed tree sets every entry of the sequence to -1.
 *   u_accept, u_resample : [B][N] fp32 out
 *   out_status   : [B] int32 out (RS_SEQ_OK or RS_SEQ_BAD_TREE), may be NULL
 * prm->mode and prm->bonus are ignored.  The outputs feed resispec_verify_tree directly.
 */
rs_status resispec_draft_candidates(const void* draft_logits, const int32_t* parent,
                                    int32_t B, int32_t N, int32_t V, const rs_params* prm,
                                    uint64_t seed, uint64_t offset, int32_t* node_token,
                                    float* u_accept, float* u_resample, int32_t* out_status,
                                    void* stream);

/*
 * The two stages of resispec_verify_tree, for callers that schedule them separately
 * (same kernels, same results): Algorithm 1 at every node, then the walk of §Preliminary.
 *   resispec_verify_nodes: every node's own outcome (accepted child or drawn token) into
 *     `workspace`, from the same inputs as resispec_verify_tree;
 *   resispec_walk: the walk from each root over the outcomes in `workspace` (written by
 *     resispec_verify_nodes with the same B and N, earlier on the same stream).
 * The workspace layout is private to the library.
 */
rs_status resispec_verify_nodes(const void* target_logits, const void* draft_logits,
                                const int32_t* node_token, const int32_t* parent,
                                const float* u_accept, const float* u_resample,
                                int32_t B, int32_t N, int32_t V, const rs_params* prm,
                                void* workspace, size_t workspace_bytes, void* stream);

rs_status resispec_walk(const int32_t* node_token, int32_t B, int32_t N, int32_t max_depth,
                        const void* workspace, size_t workspace_bytes, int32_t* out_tokens,
                        int32_t* out_accepted_len, int32_t* out_status, void* stream);

/*
 * Every node's own outcome as resispec_verify_nodes left it in `workspace` (the same
 * B and N, earlier on the same stream), copied into caller arrays (stream-ordered,
 * asynchronous; on the current device, the usual case, by one kernel, elsewhere by the
 * runtime's copies): the outcome of Algorithm 1 at each node, as the debug
 * entry below reports it.  The workspace of resispec_decide_nodes (and resispec_walk_draw)
 * is read the same way; there, nodes whose draw was deferred and not made report
 * RS_SEQ_DEFERRED.
 *   node_child, node_token_out, node_status : [B][N] int32 device out, as in
 *                 resispec_verify_tree_debug
 * RS_ERR_INVALID_ARG for B < 0, N <= 0 or NULL outputs (B > 0); RS_ERR_WORKSPACE for a
 * missing or short workspace.
 */
rs_status resispec_node_outcomes(const void* workspace, size_t workspace_bytes, int32_t B,
                                 int32_t N, int32_t* node_child, int32_t* node_token_out,
                                 int32_t* node_status, void* stream);

/* Workspace bytes resispec_verify_tree needs for B sequences of N nodes. */
size_t resispec_workspace_bytes(int32_t B, int32_t N);

/*
 * Host-side check of a tree batch (HOST pointers, synchronous, no device work).
 * Returns RS_OK when every sequence has parent[.,0] = -1, parent[.,n] in [0, n),
 * at most RS_MAX_CANDIDATES children per node and every node_token (n >= 1) in
 * [0, V); RS_ERR_INVALID_ARG otherwise.  If first_bad is not NULL it receives the
 * flat index b*N+n of the first offending entry (or -1).
 */
rs_status resispec_validate_tree_host(const int32_t* parent, const int32_t* node_token,
                                      int32_t B, int32_t N, int32_t V, int64_t* first_bad);

/*
 * Same as resispec_verify_tree, and also writes each node's own outcome (testing and
 * debugging; not the timed path):
 *   node_child  : [B][N] int32 accepted child node index, -1 if none
 *   node_token_out : [B][N] int32 token the node emits (accepted candidate, drawn token,
 *                 or -1)
 *   node_status : [B][N] int32 rs_seq_status of the node
 *   residual_out: [B][N][V] fp32 or NULL; for nodes that drew a token, the normalised
 *                 distribution of the draw (final residual, or the target for a bonus);
 *                 other rows are zero.  Costs one more pass over the logits.
 */
rs_status resispec_verify_tree_debug(const void* target_logits, const void* draft_logits,
                                     const int32_t* node_token, const int32_t* parent,
                                     const float* u_accept, const float* u_resample,
                                     int32_t B, int32_t N, int32_t V, int32_t max_depth,
                                     const rs_params* prm, int32_t* out_tokens,
                                     int32_t* out_accepted_len, int32_t* out_status,
                                     void* workspace, size_t workspace_bytes,
                                     int32_t* node_child, int32_t* node_token_out,
                                     int32_t* node_status, float* residual_out, void* stream);

/*
 * Sampling settings of rows of logits.  Each is one number for all rows, or (its array not
 * NULL, which wins) a device array with an entry for every `rows_per_entry` consecutive
 * rows: ceil(R / rows_per_entry) entries; the N node rows of a tree share a request's with
 * rows_per_entry = N.
 *
 * What they keep of a row l of V logits: with m its maximum and w_j = exp((l_j - m) / T),
 * order the finite elements by logit, equal ones by ascending index.  top_k keeps the first
 * top_k of that order; top_p, of what top_k keeps, the shortest prefix whose mass reaches
 * top_p times that of what top_k keeps; min_p those with w_j >= min_p (the maximum has w =
 * 1).  The first element is always kept.  All sums and comparisons are in 64 bits, the
 * exponentials to 4e-14 of their value; below 2^-1023, under the 64-bit type's normal range,
 * one may be zero, and its element then has no mass.
 */
typedef struct {
    int32_t logits_dtype;        /* rs_dtype */
    int32_t rows_per_entry;      /* >= 1 */
    float   temperature;         /* finite, > 0 */
    int32_t top_k;               /* >= 0; 0 = off */
    float   top_p;               /* in (0, 1]; 1 = off */
    float   min_p;               /* in [0, 1]; 0 = off */
    const float*   temperatures; /* device arrays; NULL = the number above for all rows */
    const int32_t* top_ks;
    const float*   top_ps;
    const float*   min_ps;
} rs_filter;

/*
 * Draws from rows of logits under sampling settings: the token of a position that has no
 * draft (k = 1), or the candidates that resispec_verify takes (k > 1, drawn with
 * replacement).
 *   logits      : R rows of V elements, `row_stride` (>= V) elements from row to row; what
 *                 lies between rows is not read
 *   u           : [R][k] fp32 in [0, 1), one for each draw
 *   out_token   : [R][k] int32: the smallest index j (vocabulary order) at which the kept
 *                 masses' running sum exceeds u times their total; the last kept index with
 *                 mass if rounding leaves none
 *   out_logprob : [R][k] fp32, may be NULL: the token's log-probability among what is kept
 *   out_kept    : [R] int32, may be NULL: how many elements are kept
 *   out_status  : [R] int32 rs_seq_status, may be NULL.  RS_SEQ_BAD_PARAM: a setting out of
 *                 its range; RS_SEQ_BAD_UNIFORM; RS_SEQ_UNDERFLOW: the row has no finite
 *                 logit, or a NaN or +inf.  Such a row's tokens and count are -1 and its
 *                 log-probabilities NaN.
 * RS_ERR_INVALID_ARG for a NULL pointer, R < 0, V <= 0, k <= 0, row_stride < V, or a number
 * in `filter` out of its range (a device array's entries are checked on the device);
 * RS_ERR_UNSUPPORTED for V > RS_MAX_VOCAB, k > RS_MAX_CANDIDATES or R >= 2^23.  R = 0 is a
 * no-op.  A row's outputs depend on that row, its settings and its uniforms alone, not on the
 * batch it is in.
 */
rs_status resispec_sample(const void* logits, int64_t row_stride, const float* u, int32_t R,
                          int32_t V, int32_t k, const rs_filter* filter, int32_t* out_token,
                          float* out_logprob, int32_t* out_kept, int32_t* out_status,
                          void* stream);

/*
 * Rows of logits cut to what their sampling settings keep: kept logits unchanged, every
 * other element -inf.  Target and draft rows cut this way go through
 * resispec_draft_candidates and every resispec_verify entry point as they are (-inf has
 * exactly zero mass there), at the same temperature: speculative decoding under top-k, top-p
 * and min-p.
 *   out, out_row_stride : R rows of V elements of the same type; may be `logits` itself with
 *                 the same stride; must not overlap it otherwise.  What lies between rows is
 *                 not written.
 *   out_kept, out_status: as resispec_sample (no uniforms here); a row with a status other
 *                 than RS_SEQ_OK is filled with -inf
 * Errors as resispec_sample.
 */
rs_status resispec_filter_logits(const void* logits, int64_t row_stride, int32_t R, int32_t V,
                                 const rs_filter* filter, void* out, int64_t out_row_stride,
                                 int32_t* out_kept, int32_t* out_status, void* stream);

/*
 * Log-probabilities and ranks of given tokens, such as those a verification returned, under
 * the temperature softmax of their rows (filtered rows give the filtered distribution's).
 *   tokens      : [R][k] int32; -1 = no token (the padding of resispec_verify_tree's
 *                 out_tokens): log-probability 0, rank 0
 *   filter      : the rows' type and temperature; its top_k, top_p and min_p must be off
 *   out_logprob : [R][k] fp32: (l_x - m) / T - ln sum_j exp((l_j - m) / T), its sum over
 *                 32-bit exponentials against the highest of a sample of the row and of the
 *                 row's tokens: 1e-7 or so off on rows of logits, 3e-6 at most where one of
 *                 these is the row's maximum, and 1.7e-5 at most where the maximum is far above
 *                 them all (resispec_sample's are from 64-bit sums); never above 0
 *   out_rank    : [R][k] int32, may be NULL: 1 + the number of elements before the token in
 *                 the order of rs_filter
 *   out_status  : [R] int32, may be NULL: RS_SEQ_BAD_TOKEN for an id outside [-1, V),
 *                 RS_SEQ_BAD_PARAM or RS_SEQ_UNDERFLOW as resispec_sample; such a row's
 *                 log-probabilities are NaN and its ranks -1
 * Errors as resispec_sample.
 */
rs_status resispec_token_logprobs(const void* logits, int64_t row_stride, const int32_t* tokens,
                                  int32_t R, int32_t V, int32_t k, const rs_filter* filter,
                                  float* out_logprob, int32_t* out_rank, int32_t* out_status,
                                  void* stream);

/*
 * Where rows of `row_bytes` bytes lie: the row of (o, p, i, t) starts at base +
 * o * outer_stride + p * page_stride + i * inner_stride + t * position_stride (bytes).  States
 * by beam: p is the beam, t its position.  A paged cache: p is the page, t the position in it,
 * and slot p * positions + t is the row's place in the cache.  `outer` are layers, keys and
 * values; `inner` what lies between a page and its positions (heads).  Strides may be larger
 * than what they step over; rows do not overlap.
 */
typedef struct {
    int64_t outer, pages, inner, positions, row_bytes;    /* >= 1 each */
    int64_t outer_stride, page_stride, inner_stride, position_stride;
} rs_rows;

/*
 * Beam search's choice: of all continuations of a sequence's W beams the k best.
 *   logits      : [B * W] rows of V elements, `row_stride` (>= V) elements from row to row; the
 *                 rows of beams that are not there or have ended are not read
 *   scores      : [B][W] fp32, the log-probability of each beam so far; -inf: there is no such
 *                 beam (a first step has one)
 *   ended       : [B][W] bytes, may be NULL; nonzero: the beam has ended
 *   end_token   : the token of an ended beam's continuation
 *   filter      : the rows' type and temperature; its top_k, top_p and min_p must be off (rows
 *                 cut by resispec_filter_logits are taken as they are)
 * A live beam w goes on with every token v whose logit is finite, at the score
 * (l_v - m) / T - ln sum_j exp((l_j - m) / T) + scores[w], m the row's maximum; an ended one
 * with end_token alone, at its own score.  The order is by score, equal ones by beam, within a
 * beam by logit and then by token.  It is decided in 64 bits: where sums of 32-bit exponentials
 * leave it open, by sums of 64-bit ones, to 7e-14 of their value at 151,936 elements a row and
 * 5e-13 at RS_MAX_VOCAB, and scores rounded a few times to 64 bits.  Rows with candidates within
 * 3e-6 of another beam's take a second pass each, one after another: give a first step one beam,
 * and -inf for the others, rather than W copies of it.
 *   out_parent, out_token : [B][k] int32, the best first: the beam, in [0, W), and the token; -1
 *                 past the last continuation
 *   out_score   : [B][k] fp32, its score; -inf past the last.  Besides its rounding it is off by
 *                 1.3e-6 at most, the 32-bit sum's error, which is gone where the row was summed
 *                 again, so it depends on the sequence's other beams too.  Given back as the next
 *                 step's scores the errors add up: n steps, n roundings and 1.3e-6 n at most.
 *   out_status  : [B] int32 rs_seq_status, may be NULL.  RS_SEQ_UNDERFLOW: a live beam's row has
 *                 no finite logit, or a NaN or +inf; RS_SEQ_BAD_PARAM: a score that is NaN or
 *                 +inf, or a temperature out of its range.  Such a sequence's parents and tokens
 *                 are -1 and its scores NaN.
 *   workspace   : device buffer of at least resispec_beam_workspace_bytes(B, W, V) bytes,
 *                 16-byte aligned; contents on entry are ignored.  Calls that overlap on one
 *                 workspace race.
 * RS_ERR_INVALID_ARG for a NULL pointer, B < 0, V, W or k <= 0, k > W * V, row_stride < V, or a
 * number in `filter` out of its range; RS_ERR_UNSUPPORTED for V > RS_MAX_VOCAB, W or k >
 * RS_MAX_CANDIDATES, B * W >= 2^23 or B >= 2^22; RS_ERR_WORKSPACE.  B = 0 is a no-op.  A sequence's
 * outputs depend on its rows, scores and ends alone, not on the batch.
 */
rs_status resispec_beam_select(const void* logits, int64_t row_stride, const float* scores,
                               const uint8_t* ended, int32_t end_token, int32_t B, int32_t W,
                               int32_t V, int32_t k, const rs_filter* filter,
                               int32_t* out_parent, int32_t* out_token, float* out_score,
                               int32_t* out_status, void* workspace, size_t workspace_bytes,
                               void* stream);

/* Workspace bytes resispec_beam_select needs (0 if a size is out of its range). */
size_t resispec_beam_workspace_bytes(int32_t B, int32_t W, int32_t V);

/*
 * The states of the chosen beams: for all k at once, dst[b][k] = src[b][parent[b][k]].
 *   src, src_rows : states of B * W beams (pages = B * W), of `positions` positions each
 *   dst, dst_rows : those of B * K beams; outer, inner, positions and row_bytes as src_rows.
 *                 `dst` may be `src` with the same layout (then K = W): the states change
 *                 places; it must not overlap it otherwise
 *   parent      : [B][K] int32 in [0, W); -1: that state of dst stays as it is
 *   lengths     : [B] int32, may be NULL: only the first lengths[b] positions are moved
 *   out_status  : [B] int32 rs_seq_status, may be NULL.  RS_SEQ_BAD_PARAM: a parent or a length
 *                 out of its range; nothing of that sequence is moved.
 * RS_ERR_INVALID_ARG for a NULL pointer, B < 0, W or K <= 0, or layouts that do not fit;
 * RS_ERR_UNSUPPORTED for W or K > RS_MAX_CANDIDATES, B >= 2^23, or a beam's state of 2^31 rows, or
 * pieces of 512 bytes, or more.  B = 0 is a no-op.
 */
rs_status resispec_beam_reorder(const void* src, const rs_rows* src_rows, void* dst,
                                const rs_rows* dst_rows, const int32_t* parent,
                                const int32_t* lengths, int32_t B, int32_t W, int32_t K,
                                int32_t* out_status, void* stream);

/*
 * The same for beams whose positions lie in the pages of a cache: position t of beam n is in
 * page table[n][t / P] at t % P, P = positions.
 *   src_table, dst_table : [B * W] and [B * K] rows of int32 page numbers, `src_table_stride`
 *                 and `dst_table_stride` entries from row to row, `max_pages` entries each
 *   dst         : may be `src` with the same layout, whatever W and K are (a first step's one
 *                 beam to K, W beams to 2 W).  A row of dst may then also be one of src,
 *                 if it is so at the same position of the same sequence (one table given twice;
 *                 beams that share the pages of their prompt), and not otherwise.  Beams that
 *                 share a row of dst must be given one and the same row.
 *   lengths     : [B] int32, at most max_pages * P
 *   out_status  : RS_SEQ_BAD_PARAM as above; RS_SEQ_BAD_PAGE: a page number outside the cache;
 *                 the rows that it is for are not moved
 * Errors as resispec_beam_reorder.
 */
rs_status resispec_beam_reorder_paged(const void* src, const rs_rows* src_rows,
                                      const int32_t* src_table, int64_t src_table_stride,
                                      void* dst, const rs_rows* dst_rows,
                                      const int32_t* dst_table, int64_t dst_table_stride,
                                      int32_t max_pages, const int32_t* parent,
                                      const int32_t* lengths, int32_t B, int32_t W, int32_t K,
                                      int32_t* out_status, void* stream);

/*
 * Pages and slots of a step's new rows in a paged cache.  Request r keeps its first kept[r]
 * positions and is given added[r] more; it needs want = ceil((kept + added) / page_size) pages
 * and holds the first held[r] entries of its row of the block table.  Pages past `want` go onto
 * the stack of free pages, requests in order and each request's in table order; then requests
 * in order take from its top what they lack.
 *   kept, added, held : [R] int32.  A finished request keeps 0 and is given 0; a new one holds 0.
 *   block_table : [R] rows of int32 page numbers, `table_stride` entries from row to row,
 *                 `max_pages` entries each; pages taken are entered, entries past those held
 *                 are left as they were
 *   free_pages  : [num_pages] int32 stack of page numbers in [0, num_pages), of which the first
 *                 free_count[0] are free; in and out
 *   out_held, out_free_count : [R], [1] int32; may be `held` and `free_count`
 *   out_starts  : [R + 1] int32, the running sum of added: request r's new rows are
 *                 out_starts[r] .. out_starts[r + 1] - 1
 *   out_slots   : [T] int32, the slot page * page_size + position % page_size of each new row;
 *                 -1 past the last row and where a request has been refused
 *   out_positions, out_requests : [T] int32, may be NULL: the position in its request of each
 *                 row, and the request; -1 as above
 *   out_status  : [R] int32 rs_seq_status, may be NULL.  RS_SEQ_NO_ROOM: there are not enough
 *                 free pages (for it and all requests before it), or its rows pass T;
 *                 RS_SEQ_BAD_PARAM: a negative number, more pages than max_pages, or a stack
 *                 that would hold more than num_pages.  Such a request is refused: it keeps what
 *                 it holds.  RS_SEQ_BAD_PAGE: a page number outside [0, num_pages); its rows'
 *                 slots are -1.
 * A request with RS_SEQ_BAD_PARAM for its own numbers counts as given no rows in out_starts; a
 * refused one counts with its rows.
 * RS_ERR_INVALID_ARG for a NULL pointer, R < 0, T < 0, page_size, num_pages or max_pages <= 0, or
 * table_stride < max_pages; RS_ERR_UNSUPPORTED for num_pages * page_size or max_pages *
 * page_size >= 2^31.  R = 0 sets out_starts[0], out_free_count and the padding.
 */
rs_status resispec_plan_cache(const int32_t* kept, const int32_t* added, const int32_t* held,
                              int32_t R, int32_t page_size, int32_t* block_table,
                              int64_t table_stride, int32_t max_pages, int32_t* free_pages,
                              const int32_t* free_count, int32_t num_pages, int32_t* out_held,
                              int32_t* out_free_count, int32_t* out_starts, int32_t T,
                              int32_t* out_slots, int32_t* out_positions,
                              int32_t* out_requests, int32_t* out_status, void* stream);

/*
 * The accepted nodes of verified trees: the way from the root down whose nodes carry the
 * accepted tokens.
 *   parent, node_token : [B][N] int32, as for resispec_verify_tree
 *   tokens, accepted_len : [B][max_depth + 1] and [B] int32, its outputs; accepted_len -1 (a
 *                 fault) gives no path
 *   out_path    : [B][max_depth + 1] int32: 0 (the root), then the accepted nodes, -1 after the
 *                 last.  Where nodes of several ways carry the same tokens, the way that ends at
 *                 the lowest node.
 *   out_status  : [B] int32 rs_seq_status, may be NULL.  RS_SEQ_BAD_TREE: a malformed parent
 *                 array, or no way carries the tokens; RS_SEQ_DEPTH_EXCEEDED: accepted_len
 *                 outside [-1, max_depth].  Such a sequence has no path.
 * RS_ERR_INVALID_ARG for a NULL pointer, B < 0, N <= 0 or max_depth < 0; RS_ERR_UNSUPPORTED for
 * N > RS_MAX_PATH_NODES or B >= 2^22.  B = 0 is a no-op.
 */
#define RS_MAX_PATH_NODES 8192
rs_status resispec_accepted_path(const int32_t* parent, const int32_t* node_token,
                                 const int32_t* tokens, const int32_t* accepted_len, int32_t B,
                                 int32_t N, int32_t max_depth, int32_t* out_path,
                                 int32_t* out_status, void* stream);

/*
 * The accepted rows at their places in the cache: node path[b][i] was given slot
 * slots[b][path[b][i]] for the verification and belongs at slots[b][i], behind the i accepted
 * nodes before it.  For every b and i up to the path's first -1:
 *   cache[slots[b][i]] = source row (page b, position path[b][i]), or, if source is NULL,
 *   cache[slots[b][i]] = cache[slots[b][path[b][i]]], all i at once.
 *   cache, cache_rows : the paged cache
 *   slots       : [B][N] int32; the slots of one call's nodes differ from each other
 *   path        : [B][depth] int32, nodes in ascending order, -1 after the last
 *   source, source_rows : NULL, or the rows of the trees' nodes outside the cache (pages = B,
 *                 positions = N; outer, inner and row_bytes as cache_rows); must not overlap it
 *   out_status  : [B] int32 rs_seq_status, may be NULL.  RS_SEQ_BAD_TREE: a path that does not
 *                 ascend or has a node outside [0, N); RS_SEQ_BAD_PAGE: a slot of it outside
 *                 the cache.  Nothing of that sequence is moved.
 * RS_ERR_INVALID_ARG for a NULL pointer, B < 0, N or depth <= 0, or layouts that do not fit;
 * RS_ERR_UNSUPPORTED for N or depth > RS_MAX_PATH_NODES, B >= 2^23, pages * positions or outer *
 * inner >= 2^31, or rows of 2^31 bytes or more.  B = 0 is a no-op.
 */
rs_status resispec_commit_path(void* cache, const rs_rows* cache_rows, const int32_t* slots,
                               const int32_t* path, const void* source,
                               const rs_rows* source_rows, int32_t B, int32_t N, int32_t depth,
                               int32_t* out_status, void* stream);

/* Static description of a status code. */
const char* resispec_status_string(int32_t status);

/* RESISPEC_ABI_VERSION of the loaded library. */
int32_t resispec_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* RESISPEC_H */
