/*
 * smore.h -- C ABI of the MI355X sampler for multi-hop query training data
 * (SMORE, arXiv 2110.14890: reverse directional sampling of queries, Sec. 3.1,
 * and bidirectional rejection sampling of verified negatives, Sec. 3.2).
 *
 * Conventions
 *  - Every call returns SMORE_OK (0) or a negative SMORE_E_* code; on error
 *    smore_last_error() returns a message for the calling thread.  No C++
 *    exception crosses this boundary.
 *  - Arguments are validated synchronously on the host before any launch;
 *    an invalid call launches nothing and writes nothing.
 *  - Pointers named *_host are host memory, all other buffers are device
 *    memory allocated by the caller (for example torch tensors on the same
 *    device).  The library never frees caller memory.
 *  - smore_sample is asynchronous on the caller's HIP stream and returns
 *    without synchronising; results are valid once that stream reaches them.
 *  - All ids and outputs are int32.  Entity ids are in [0, V), relation ids
 *    in [0, R') where R' = 2R when the graph adds inverse relations.
 */
#ifndef SMORE_H
#define SMORE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    SMORE_OK = 0,
    SMORE_E_INVALID_ARG = -1, /* null pointer, bad size, bad query plan */
    SMORE_E_RANGE = -2,       /* an id outside [0, V) or [0, R) */
    SMORE_E_UNSUPPORTED = -3, /* plan outside the fourteen shapes, limits */
    SMORE_E_NOMEM = -4,       /* device or host allocation failed */
    SMORE_E_HIP = -5,         /* a HIP runtime call failed */
    SMORE_E_OVERFLOW = -6     /* counts beyond the int32 / 32-bit query-id range, or
                                 batch x neg_tries of 2^31 or more */
};

/* flags of smore_build_graph */
#define SMORE_ADD_INVERSE 1u /* also insert (t, r + R, h) for every (h, r, t) */

/* Node operators of a query computation plan (Sec. 2, "Query computation
   plan"; appendix on the computation plan).  Each node is a set of
   entities; a projection node applies one relation to its single child, an
   intersection / union node combines its children, a complement node is
   V minus its single child, an anchor is a leaf. */
enum { SMORE_OP_ANCHOR = 0, SMORE_OP_PROJ = 1, SMORE_OP_AND = 2, SMORE_OP_OR = 3, SMORE_OP_NOT = 4 };

/* One plan node.  child[] index earlier nodes of the same plan (children
   before parents).  slot: the anchor slot (0..2) of an anchor, the relation
   slot (0..2) of a projection, -1 otherwise. */
typedef struct {
    int32_t op, n_child, child[3], slot;
} smore_dag_node;

/* A plan tree: n_nodes nodes, root = the answer node V_?. */
typedef struct {
    int32_t n_nodes, root;
    smore_dag_node node[16];
} smore_query_dag;

/* Arguments of one sampling call.
   batch        number of queries B (>= 1)
   n_neg        negatives wanted per query (>= 0)
   pos_tries    reverse-sampling attempts per query (>= 1)
   neg_tries    candidate draws per query (>= n_neg, <= SMORE_MAX_NEG_TRIES)
   max_fanout   0, or reject a grounding whose step (x, r) -> e has
                |A_r(x)| > max_fanout (the paper's per-relation expansion C)
   seed         64-bit key of the counter-based draws
   query_offset query q of this call has id query_offset + q; the result of
                a query depends only on (graph, plan, seed, id, counts), so a
                batch split over several calls gives identical rows
   flags        0 (reserved) */
typedef struct {
    int32_t batch, n_neg, pos_tries, neg_tries, max_fanout;
    uint64_t seed, query_offset;
    uint32_t flags;
} smore_sample_args;

#define SMORE_MAX_NEG_TRIES 4096

/* Caller-owned device outputs, int32, row-major.
   anchors   [B,3]   anchor entities by slot, -1 for unused slots
   relations [B,3]   relations by slot, -1 for unused slots
   positive  [B]     the answer entity grounded at the root
   negatives [B,n_neg] verified non-answers in draw order, -1 padded
   n_valid   [B]     number of negatives found; -1 if no positive was found
   pos_attempts [B]  attempts used (1-based); pos_tries when none succeeded
   neg_draws [B]     draws consumed: 1 + index of the n_neg-th accepted
                     draw, else neg_tries; 0 when n_neg = 0; -1 with no positive
   All seven pointers are required. */
typedef struct {
    int32_t *anchors, *relations, *positive, *negatives, *n_valid, *pos_attempts, *neg_draws;
} smore_sample_out;

typedef struct smore_graph smore_graph; /* opaque; owns its device arrays */

/* Build forward and reverse adjacency on the current HIP device from
   n_triples host triples (h, r, t) (int32 [n_triples, 3]).  The KG is a set
   of triples (Sec. 2), so duplicates are removed.  Adjacency is grouped by
   (entity, relation) with ascending relations per entity and ascending
   neighbours per group, as sorted lists (appendix on the optimal cut: sets
   kept as sorted lists).  Errors: SMORE_E_RANGE for an id outside
   [0, n_entities) / [0, n_relations); SMORE_E_OVERFLOW when the edge count
   (doubled with SMORE_ADD_INVERSE) reaches 2^31; SMORE_E_NOMEM; SMORE_E_HIP.
   Synchronous.  *out must be released with smore_free_graph. */
int smore_build_graph(const int32_t *triples_host, int64_t n_triples, int32_t n_entities,
                      int32_t n_relations, uint32_t flags, smore_graph **out);

/* Sizes of a built graph (any pointer may be NULL): entities, relations
   (after inverse), unique edges, forward and reverse (entity, relation)
   groups, device bytes held. */
int smore_graph_info(const smore_graph *g, int64_t *n_entities, int64_t *n_relations,
                     int64_t *n_edges, int64_t *n_seg_fwd, int64_t *n_seg_rev,
                     int64_t *device_bytes);

/* Copy one device array of the graph to host memory (for tests and
   inspection).  which: 0 fwd node_ptr [V+1], 1 fwd groups [2*(S_fwd+1)]
   (relation, first edge) pairs, 2 fwd neighbours [E], 3 rev node_ptr,
   4 rev groups, 5 rev neighbours, 6 active_in (entities with an in-edge,
   ascending), 7 in-edge mask [(V+31)/32] (bit v % 32 of word v / 32 set
   iff entity v has an in-edge), 8 coarse in-edge mask [(V+127)/128] (bit
   i % 32 of word i / 32 set iff one of entities 4i .. 4i+3 has an in-edge),
   9 in-relation signatures [(V+3)/4] (byte v % 4 of word v / 4, little
   endian, is entity v's: bit (r * 0x9E3779B1 mod 2^32) >> 29 set for each
   relation r of its in-edges, 0 for an entity without in-edges).
   count must equal the array length.
   Synchronous. */
int smore_graph_copy(const smore_graph *g, int32_t which, int32_t *host_dst, int64_t count);

/* Fill *out with one of the fourteen query structures of BetaE (Sec. 5.1):
   the nine without negation "1p" "2p" "3p" "2i" "3i" "ip" "pi" "2u" "up",
   and "2in" "3in" "inp" "pin" "pni", where one operand of the intersection
   is complemented (2in, 3in, inp, pin: the last one-hop operand; pni: the
   two-hop operand).  Anchor and relation slots follow branch order, and
   within a branch run from the anchor to the root. */
int smore_query_preset(const char *name, smore_query_dag *out);

/* Node cut of a plan tree minimising the worst per-anchor-path cost
   max(C^i, C^(t-i)) (Sec. 3.2, Def. "Node cut" and the optimal-scheduling
   equation), by the dynamic program of the appendix on the optimal cut
   (u = projections to the root, s = longest projection path to an anchor,
   o = best cost) and its top-down construction.  tie_break 0 adds a node
   when the children's best cost exceeds its own (as stated); 1 also adds it
   on equality, which caches as far forward as the same cost allows.
   cut_nodes receives up to 16 node indices; *n_cut their number. */
int smore_plan(const smore_query_dag *dag, int32_t tie_break, int32_t *cut_nodes, int32_t *n_cut);

/* Bytes of device workspace smore_sample / smore_sample_negatives need for
   these arguments (it grows with batch * neg_tries: per-draw states, the
   queues of long intersections, the list ranges of each query and the
   queries still short of n_neg; the same for every shape).  The caller allocates it; its contents need no
   initialisation and are scratch after the call.  Calls that may overlap on
   the device must not share a workspace.  A call with n_neg = 0 draws no
   candidates and needs no workspace (NULL and 0 are accepted). */
int smore_sample_workspace_bytes(const smore_graph *g, const smore_query_dag *dag,
                                 const smore_sample_args *args, size_t *bytes);

/* Sample args->batch queries of shape dag with one positive each and up to
   n_neg verified negatives (Sec. 3.1 reverse directional sampling; Sec. 3.2
   bidirectional rejection sampling with a constant candidate budget).
   Per query id q: attempt t grounds the root uniformly among entities with
   an in-edge, then walks from the root to the anchors in pre-order, each
   projection picking an in-relation uniformly and then an in-neighbour
   uniformly; the first attempt without a dead end, a repeated
   (anchor, relation) pair among single-projection siblings, or a step wider
   than max_fanout wins.  Candidate j (j < neg_tries) is uniform over all V
   entities and is kept iff it is not an answer of the query and was not
   drawn earlier; the first n_neg kept are returned.  Draws come from
   Philox4x32-10 with counter (j, t, q, tag) and key seed.
   A complemented operand of an intersection (the negation shapes) is
   grounded after the positive operands, from a sibling entity w drawn
   uniformly from A_r(x) of the first positive operand's step (x, r) -> e;
   the attempt is also rejected when e lies in the complemented set, so the
   root is always an answer.  Draws are numbered in grounding order (root,
   two per projection, one for w).  The plan must be one of the fourteen
   presets (SMORE_E_UNSUPPORTED otherwise).  hip_stream: a hipStream_t, or
   NULL for the default stream. */
int smore_sample(const smore_graph *g, const smore_query_dag *dag, const smore_sample_args *args,
                 const smore_sample_out *out, void *workspace, size_t ws_bytes, void *hip_stream);

/* smore_sample for callers that cannot allocate device memory (code under
   HIP graph capture, tight serving loops, harnesses that forbid
   allocation): the same arguments, validation, outputs and stream
   semantics, but no workspace argument.  The scratch is a fixed array of
   SMORE_NOALLOC_SCRATCH_BYTES in device memory, one per GPU the library
   runs on, held until the process ends; the call itself allocates and
   frees nothing.  Every call on one GPU shares that array, so calls that
   may overlap on a GPU (different streams, different threads) race and
   must be serialised by the caller; the array keeps the last call's
   contents, and each call initialises whatever it reads.  Errors as for
   smore_sample, and SMORE_E_UNSUPPORTED when the arguments need more
   scratch than the fixed size (smore_sample_workspace_bytes gives the
   need; about 15 KB per query at 512 negatives and 2,048 draws, e.g.
   4,096 such queries, or 16,384 queries with 64 negatives and 256
   draws). */
#define SMORE_NOALLOC_SCRATCH_BYTES (64u << 20)
int smore_sample_noalloc(const smore_graph *g, const smore_query_dag *dag,
                         const smore_sample_args *args, const smore_sample_out *out,
                         void *hip_stream);

/* The two stages of smore_sample, for callers that time or feed them
   separately.  Same arguments and validation as smore_sample.
   smore_sample_positives writes anchors, relations, positive, pos_attempts
   and n_valid (-1 for a query without a positive, else 0).
   smore_sample_negatives reads anchors, relations and positive (a row with
   positive < 0, or with an anchor or relation id used by the shape outside
   the graph's range, is skipped: negatives -1, n_valid -1, neg_draws -1) and
   writes negatives, n_valid and neg_draws; it may be run on queries built
   by the caller.  stats is NULL or a device int64 [batch, 4] array that
   receives, per query, the bytes and the 64-byte lines of graph data the
   verification read: [0], [1] by the wavefront that takes the draws
   (forward-cached lists once per query, then every read made from a
   candidate's side, whichever kernel takes the draw), [2], [3] in the
   intersections of lists too long for that wavefront to walk; lookups
   inside forward-cached lists are cache hits of the method and are not
   counted.  Counting makes
   the call slower and does not change any other output.  workspace /
   ws_bytes as for smore_sample (smore_sample_positives needs none). */
int smore_sample_positives(const smore_graph *g, const smore_query_dag *dag,
                           const smore_sample_args *args, const smore_sample_out *out,
                           void *hip_stream);
int smore_sample_negatives(const smore_graph *g, const smore_query_dag *dag,
                           const smore_sample_args *args, const smore_sample_out *out,
                           int64_t *stats, void *workspace, size_t ws_bytes, void *hip_stream);

/* smore_sample_negatives in three parts, for callers that schedule the
   candidate kernel (the draws, their verification and the selection of most
   queries, Sec. 3.2) apart from the rest, e.g. the candidate kernels of
   several calls back to back on one stream:
   part 0 the per-query preparation, part 1 the candidate kernel, part 2 the
   rest (long lists, and the queries that had some).
   Calling parts 0, 1 and 2 with the same arguments, outputs and workspace,
   each after the previous one has completed in stream order (on one stream,
   or ordered by the caller's events across streams), has exactly the effect
   of one smore_sample_negatives call; the outputs are final only after
   part 2.  The workspace carries state from part to part: it must not be
   used by any other call in between.  stats, the instrumentation hooks and
   errors as for smore_sample_negatives (smore_profile_kernel's candidate
   kernel and smore_wait_before_kernel act in part 1; any part disarms
   them).  SMORE_E_INVALID_ARG for another part. */
int smore_sample_negatives_part(const smore_graph *g, const smore_query_dag *dag,
                                const smore_sample_args *args, const smore_sample_out *out,
                                int64_t *stats, int32_t part, void *workspace, size_t ws_bytes,
                                void *hip_stream);

/* Caller-owned device outputs of smore_sample_shared, int32 unless noted.
   anchors [B,3], relations [B,3], positive [B], pos_attempts [B]
                     as in smore_sample_out
   shared   [n_neg]  the minibatch's candidate set N, in draw order, -1 padded
   n_shared [1]      |N|: n_neg, or fewer when neg_tries draws hold fewer
                     distinct entities
   mask     uint32 [B, (n_neg + 31) / 32]: bit k % 32 of word k / 32 of row i
                     is set iff N[k] is a verified non-answer of query i
   n_valid  [B]      set bits of row i; -1 for a query without a positive
                     (its row is zero)
   All pointers are required (shared and mask may be NULL when n_neg = 0). */
typedef struct {
    int32_t *anchors, *relations, *positive, *pos_attempts, *shared, *n_shared;
    uint32_t *mask;
    int32_t *n_valid;
} smore_shared_out;

/* A minibatch whose queries share one set of candidate negatives (Sec. 4.3,
   sharing negative samples): one candidate set N for all args->batch
   queries and a mask saying, per query, which members of N are negatives.
   The positives are exactly those of smore_sample with the same arguments.
   N holds the first n_neg distinct values of the draws
   pick(U(3, query_offset, 0, j), V), j < neg_tries (Philox counter
   (j, 0, low 32 bits of query_offset, 3)), so different minibatches
   (query_offset) draw different sets.  Every (query, member) pair is
   verified by the same bidirectional test as smore_sample.  Arguments,
   validation and workspace (smore_sample_workspace_bytes with the same
   args) as for smore_sample; asynchronous on hip_stream.  With n_neg = 0
   the set is empty (*n_shared = 0), no mask word exists, n_valid is 0 (or
   -1 without a positive) and no workspace is needed. */
int smore_sample_shared(const smore_graph *g, const smore_query_dag *dag,
                        const smore_sample_args *args, const smore_shared_out *out,
                        void *workspace, size_t ws_bytes, void *hip_stream);

/* Membership verification of caller-given candidates: for every query i
   (anchors / relations [B,3], device, as smore_sample writes them) and
   each of its n = args->n_neg candidates (device int32 [B, n]), is the
   candidate an entity outside the query's answer set?  This is the test
   behind rejection sampling (Sec. 3.2, bidirectional), run here on given
   pairs - for evaluation, where a query's answers differ between nested
   graphs G_train, G_valid, G_test (appendix on the task setup): verifying
   the positives of queries sampled on G_test against G_valid finds the
   answers missing from G_valid.
   mask  uint32 [B, (n + 31) / 32]: bit k % 32 of word k / 32 of row i set
         iff candidate k of query i is in [0, V) and not an answer
   n_valid [B]: set bits of row i; -1 when an anchor or relation the shape
         uses is out of range (row zero)
   Candidates outside [0, V) are never negatives and read no graph data.
   args: batch = B, n_neg = n, neg_tries >= n (workspace sizing as for
   smore_sample, see smore_sample_workspace_bytes); the other fields are
   checked as for smore_sample but unused.  With n = 0 only n_valid is
   written (0, or -1 as above) and candidates, mask and the workspace may
   be NULL.  Asynchronous on hip_stream. */
int smore_verify(const smore_graph *g, const smore_query_dag *dag, const smore_sample_args *args,
                 const int32_t *anchors, const int32_t *relations, const int32_t *candidates,
                 uint32_t *mask, int32_t *n_valid, void *workspace, size_t ws_bytes,
                 void *hip_stream);

/* Instrumentation: the next smore_sample or smore_sample_negatives call
   made by this thread records the caller's HIP events (hipEvent_t) on its
   stream immediately before and after one of its kernels: which = 0 the
   candidate kernel, 1 the kernels that intersect long lists (for 3p the
   batched long-list kernel and the kernel of its units, timed together; for
   the other shapes the finishing kernel), 2 the finishing kernel, which
   selects the negatives of the queries that had long lists (shapes made of
   edge tests alone have none of these: both events follow the candidate
   kernel).  Each `which` has
   its own arm, so one call can time several kernels.  One-shot: the
   next smore_sample, smore_sample_negatives or smore_sample_negatives_part
   call of this thread disarms all of them whether or not they recorded,
   also when that call fails validation.  Either event NULL disarms that
   `which`.  The events stay owned by the
   caller.  Returns SMORE_E_INVALID_ARG for another `which`. */
int smore_profile_kernel(void *start_event, void *stop_event, int32_t which);

/* Scheduling, for callers that run several sampling calls on different
   streams and want their candidate kernels one after another: the next
   smore_sample or smore_sample_negatives call made by this thread makes its
   stream wait on the caller's HIP event (hipEvent_t) right before its
   first candidate kernel (which = 0), after the per-query preparation, so
   the preparation does not wait.  One-shot: the next such call (or
   smore_sample_negatives_part) disarms it, also when it launches no
   candidate kernel (n_neg = 0) or fails validation.  NULL disarms.
   The event stays owned by the caller.  SMORE_E_INVALID_ARG for another
   `which`; SMORE_E_HIP if the wait cannot be enqueued (the call then
   launches nothing after the preparation). */
int smore_wait_before_kernel(void *event, int32_t which);

/* Instrumentation: n_reads random 4-byte reads from the device table of
   table_bytes (the first word of pseudo-randomly chosen 64-byte lines among
   the largest power-of-two number of lines that fits), eight independent
   reads in flight per lane, folded into sink (device uint32, at least
   (n_reads + 63) / 64 words, overwritten).  The rate of this kernel is the
   device's random-read ceiling that the sampler's gathers are compared
   with; it is not part of sampling.  Asynchronous on hip_stream.  Errors:
   SMORE_E_INVALID_ARG for null pointers, a table under 64 bytes, n_reads
   outside [1, 2^40] or a short sink. */
int smore_gather_probe(const void *table, int64_t table_bytes, int64_t n_reads, uint32_t *sink,
                       int64_t sink_words, void *hip_stream);

/* ---------------------------------------------------------------------
   Training on sampled batches: candidate scores, the preference loss of a
   positive against its verified negatives, and AdamW.  Like the sampling
   calls they validate on the host, launch on hip_stream and return; the
   device of the buffers must be the current one.  Strides count elements.
   Rows of any length and any alignment of a whole element are accepted.
   Sums are in fp32 in a fixed order: equal calls give equal bits. */

/* element types */
enum { SMORE_F32 = 0, SMORE_BF16 = 1, SMORE_F16 = 2 };

/* Sizes of smore_score / smore_score_grad.
   batch B (>= 1), n candidates per query (0 .. 2^30), dim (1 .. 2^20);
   n_rows        rows V of the table (>= 1)
   table_stride, query_stride (>= dim), candidate_stride, score_stride
                 (>= n): distance of two rows; the rows of the candidates
                 may coincide (candidate_stride 0: one set for all queries)
   table_type, query_type  SMORE_F32 or SMORE_BF16 */
typedef struct {
    int32_t batch, n, dim, n_rows;
    int64_t table_stride, query_stride, candidate_stride, score_stride;
    int32_t table_type, query_type;
} smore_score_args;

/* scores [B, n] (fp32): the product of each query's vector (queries
   [B, dim]) with the table rows (table [V, dim]) of its candidates (int32
   [B, n], as smore_sample writes them).  A candidate outside [0, V), such
   as the -1 of a short row, has score 0 and reads no row.  Errors:
   SMORE_E_INVALID_ARG, SMORE_E_UNSUPPORTED for another type,
   SMORE_E_OVERFLOW when B x ceil(n / 8) reaches 2^26. */
int smore_score(const smore_score_args *args, const void *table, const void *queries,
                const int32_t *candidates, float *scores, void *hip_stream);

/* Gradient of smore_score for the queries: grad_queries [B, dim] (of
   query_type, strides query_stride) = sum over k of grad_scores [B, n]
   (fp32, strides score_stride) times the row of candidate k.  Candidates
   outside [0, V) add nothing, whatever their grad_scores hold; n = 0 gives
   zeros.  Few queries with long lists are split over the chip and need a
   workspace (smore_score_grad_workspace_bytes, 0 where they are not; scratch
   after the call, not shared by calls that overlap).  The gradient for the
   table is taken by smore_adamw, row by row.  B below 2^24, else
   SMORE_E_OVERFLOW. */
int smore_score_grad_workspace_bytes(const smore_score_args *args, size_t *bytes);
int smore_score_grad(const smore_score_args *args, const void *table, const int32_t *candidates,
                     const float *grad_scores, void *grad_queries, void *workspace,
                     size_t ws_bytes, void *hip_stream);

/* Preference loss of paired log ratios.  For row b and its valid negatives
   k (c of them)
       z_k = beta ((positive - ref_positive) - (negatives[k] - ref_negatives[k]))
   SMORE_PREFERENCE_PAIRS    loss = 1/c sum_k (1 - smoothing) softplus(-z_k)
                                             + smoothing softplus(z_k)
   SMORE_PREFERENCE_SOFTMAX  loss = log(1 + sum_k exp(-z_k)), all negatives
                             against the positive at once (smoothing 0)
   With scores that are log probabilities up to a constant of the row the
   constant cancels. */
enum { SMORE_PREFERENCE_PAIRS = 0, SMORE_PREFERENCE_SOFTMAX = 1 };

/* batch B (>= 1, below 2^24), n negatives per row (0 .. 2^30), kind, score_type
   (SMORE_F32, _BF16, _F16: of the scores, the reference scores and the
   gradients), beta (finite, > 0), smoothing ([0, 1)), scale (finite: factor
   of the gradients), and the distances (>= 0) of two rows of each array; rows
   of the gradients must not overlap. */
typedef struct {
    int32_t batch, n, kind, score_type;
    float beta, smoothing, scale;
    int64_t positive_stride, negatives_stride, ref_positive_stride, ref_negatives_stride,
        grad_positive_stride, grad_negatives_stride;
} smore_preference_args;

/* positive [B], negatives [B, n]; ref_positive, ref_negatives the same of the
   reference model, both NULL for none.  Valid negatives of row b: the first
   n_valid[b] (int32 [B], as smore_sample writes it; -1 and 0: none, more
   than n: n), or those with bit k % 32 of word k / 32 of row b of mask set
   (uint32 [B, (n + 31) / 32], as smore_sample_shared and smore_verify write
   it), or all n where both are NULL; not both.  weight (fp32 [B] or NULL):
   factor of each row's gradient. */
typedef struct {
    const void *positive, *negatives, *ref_positive, *ref_negatives;
    const int32_t *n_valid;
    const uint32_t *mask;
    const float *weight;
} smore_preference_in;

/* loss [B] (fp32, unweighted; NULL: not wanted), and scale x weight[b] times
   the gradient of row b's loss: grad_positive [B], grad_negatives [B, n]
   (both NULL: not wanted).  A row without a valid negative has loss and
   gradients 0; places that are not valid are not used and get gradient 0.
   A valid score that is NaN makes its row NaN, as in the formula, and so does
   a z_k of -infinity (a negative at +infinity, a positive at -infinity) with
   SMORE_PREFERENCE_SOFTMAX; with SMORE_PREFERENCE_PAIRS a row's loss is infinite
   where the sum over its negatives passes fp32.  Outputs must not overlap inputs
   or each other. */
typedef struct {
    float *loss;
    void *grad_positive, *grad_negatives;
} smore_preference_out;

int smore_preference_loss(const smore_preference_args *args, const smore_preference_in *in,
                          const smore_preference_out *out, void *hip_stream);

/* Stable order of n entries (0 .. 2^26 - 1) by the table row they name: rows
   [n] receives ids (device int32 [n], any order) sorted, ids outside
   [0, n_rows) last, and order [n] the entry each came from, equal ids in
   their first order.  What smore_adamw takes as rows and order.  ids is not
   written and must not overlap the outputs.  The workspace
   (smore_sort_rows_workspace_bytes) is scratch after the call and not shared
   by calls that overlap. */
int smore_sort_rows_workspace_bytes(int64_t n, int32_t n_rows, size_t *bytes);
int smore_sort_rows(const int32_t *ids, int64_t n, int32_t n_rows, int32_t *rows, int64_t *order,
                    void *workspace, size_t ws_bytes, void *hip_stream);

/* AdamW with decoupled weight decay, for many tensors in one call:
       m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
       p = p (1 - lr decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
   Arithmetic is in fp32.

   A dense tensor (rows NULL) has n_rows x dim elements in a row, and so have
   its gradient and its moments.  A table (rows given) is stepped only in the
   rows that a batch touched: rows (int32 [n_entries], ascending but for
   entries outside [0, n_rows), which may come first or last; repeats allowed)
   names a row per entry, and the gradient of a row is the sum over
   its entries i of coef[o] x grad[o / per], o = order[i], where grad is
   [ceil(n_entries / per), dim], order (int64) is a permutation of the
   entries (NULL: o = i) and coef is fp32 (NULL: 1).  With ids, grad_scores
   and queries of smore_score flattened and sorted by id, per = n, this is
   smore_score's gradient for the table, never written out.  Entries outside
   [0, n_rows) are skipped; all other rows keep their values and moments,
   without decay.

   bits 32: m, v fp32.  bits 8: m and v are bytes, e4m3 codes of m and of
   sqrt(v) divided by the scale of their block of SMORE_ADAMW_BLOCK
   consecutive elements of a row (a dense tensor is one row): m_scale,
   v_scale fp32, [ceil(elements / block)], for tables [n_rows,
   ceil(dim / block)].  Moments that are all zero bytes are moments 0, a block
   whose moments are all below 2^-100 is held as 0, and one in which m or v is
   not finite keeps neither: both are NaN from then on.

   SMORE_ADAMW_STOCHASTIC: codes and bf16 parameters are rounded up or down
   at random by their remainder (nearest, ties to even, without it), from a
   hash of (seed, t, index, position): a step that is run again from the same
   values gives the same bits.  index tells the tensors of a model apart.
   Moments in 8 bits need it: a step changes v by 1 - beta2 of itself, a code is
   1/16 to 1/8 of its value wide, so rounded to the nearest a code stays where
   it is whatever the gradients do. */
#define SMORE_ADAMW_BLOCK 128
#define SMORE_ADAMW_STOCHASTIC 1u

typedef struct {
    void *param;        /* SMORE_F32 or SMORE_BF16 */
    const void *grad;   /* SMORE_F32, _BF16 or _F16 */
    void *m, *v;
    float *m_scale, *v_scale;
    const int32_t *rows;
    const int64_t *order;
    const float *coef;
    int64_t n_rows, dim, n_entries, per;
    int32_t param_type, grad_type, bits, index;
    float weight_decay;
} smore_adamw_tensor;

/* lr (finite, >= 0), beta1, beta2 in [0, 1), eps (finite, >= 0), step t (>= 1).
   With eps 0 the quotient of an element whose v is 0 is infinite or NaN: one
   without any gradient yet, or of gradients whose squares vanish in fp32 (below
   about 1e-21 in a first step with beta2 0.999).
   On the device, for steps captured into a graph (NULL: not used):
   step_device (int64, >= 1) and lr_device (fp32) replace step and lr;
   grad_scale (fp32) multiplies every gradient, and where it is not finite
   nothing is written. */
typedef struct {
    double lr, beta1, beta2, eps;
    int64_t step;
    const int64_t *step_device;
    const float *lr_device;
    const float *grad_scale;
    uint64_t seed;
    uint32_t flags;
} smore_adamw_args;

/* Steps n_tensors (host array) tensors.  Parameters and moments must not
   overlap, neither within a tensor nor between tensors: of the parameters
   this is checked (SMORE_E_INVALID_ARG).  That rows ascends is not: of a row
   that is named again after another one, some entries would be lost.  The
   workspace holds sums of long runs of equal rows (0 bytes without tables;
   scratch after the call, not shared by calls that overlap).
   SMORE_E_OVERFLOW: 2^26 or more entries, table rows of more than 2^20
   columns, or 2^34 or more elements of a dense tensor. */
int smore_adamw_workspace_bytes(const smore_adamw_tensor *tensors, int32_t n_tensors, size_t *bytes);
int smore_adamw(const smore_adamw_tensor *tensors, int32_t n_tensors, const smore_adamw_args *args,
                void *workspace, size_t ws_bytes, void *hip_stream);

/* Release a graph (NULL is a no-op). */
void smore_free_graph(smore_graph *g);

/* Message of the last failed call on this thread ("" if none). */
const char *smore_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SMORE_H */
