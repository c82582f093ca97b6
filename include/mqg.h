/*
 * mqg - mini-batch generation for sampled GNN training on one MI355X (gfx950).
 *
 * C ABI of the library.  The four operations are the per-mini-batch data path
 * that the MQ-GNN paper describes around its pipeline: node-wise neighbour
 * sampling, the mini-batch's topology and feature parts, the GPU feature
 * cache with host fallback, and the gather/aggregate (GA) step of GraphSAGE.
 * Beside them stand the calls of the layers that read what they produce: norms,
 * aggregation of 8-bit rows, and the steps of the weights.
 *
 * Conventions
 *   - Every pointer named *_dev / documented "device" must be dereferenceable
 *     by a GPU kernel of the current device (hipMalloc memory, or pinned host
 *     memory from hipHostMalloc where stated).  Pointers documented "host" are
 *     read by the CPU during the call only.
 *   - The caller owns every data buffer (graph, features, cache storage,
 *     block outputs, gathered rows).  A context owns only its private scratch.
 *     The library keeps no caller pointer after a call returns.
 *   - All calls only enqueue work on the given HIP stream and return; results
 *     (including the sizes that depend on the data) are complete when the
 *     stream has been synchronised.  One context serves one stream at a time;
 *     concurrent mini-batches use one context each.
 *   - Every function returns an mqg_status (0 = ok, negative = error).  Errors
 *     that the host can see (null pointers, bad enums, capacities below the
 *     bounds stated below) are returned before anything is enqueued.  No
 *     exception or abort crosses this boundary.
 *   - Blocks are indexed by the GNN layer they feed: block L-1 has the seed
 *     nodes as destinations, block 0 is the outermost and its source nodes
 *     are the rows whose input features are gathered.  fanouts[l] belongs to
 *     block l, so sampling (which walks outward from the seeds) uses
 *     fanouts[L-1] first.
 */
#ifndef MQG_H
#define MQG_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct mqg_ctx mqg_ctx;          /* opaque; owns scratch memory only            */
typedef void *mqg_stream;                /* a hipStream_t; NULL is the default stream    */

typedef enum {
    MQG_OK = 0,
    MQG_ERR_INVALID_ARG = -1,            /* null pointer, bad enum, negative size ...    */
    MQG_ERR_CAPACITY = -2,               /* an output buffer is below its stated bound   */
    MQG_ERR_HIP = -3,                    /* a HIP runtime call failed                    */
    MQG_ERR_UNSUPPORTED = -4             /* valid request outside the built limits       */
} mqg_status;

typedef enum { MQG_F32 = 0, MQG_F16 = 1, MQG_BF16 = 2 } mqg_dtype;   /* MQG_BF16: the calls of a layer only */
typedef enum { MQG_I32 = 0, MQG_I64 = 1 } mqg_itype;

#define MQG_MAX_FANOUT 64                /* per-node neighbour budget of one block       */
#define MQG_MAX_LAYERS 8

/*
 * Graph G = (V, E) in CSR form (paper Sec. III, notation paragraph).  Row v
 * lists the in-neighbours of v (the nodes whose features v aggregates); the
 * cache ranks nodes by this in-degree (Eq. 13).  Preconditions: rows hold no
 * duplicate entry (so distinct adjacency slots are distinct neighbours) and
 * every entry lies in [0, num_nodes); num_nodes < 2^31; every degree < 2^31.
 * Both arrays are device memory and are only read.
 */
typedef struct mqg_graph {
    int64_t num_nodes;
    int64_t num_edges;                   /* length of col_idx                            */
    int32_t ptr_type;                    /* mqg_itype of row_ptr                         */
    int32_t idx_type;                    /* mqg_itype of col_idx and of all node-id I/O  */
    const void *row_ptr;                 /* device [num_nodes + 1]                       */
    const void *col_idx;                 /* device [num_edges]                           */
} mqg_graph;

/*
 * Node feature storage F and the GPU-resident cache C of hot nodes (paper
 * Sec. III "Feature Cache"; Sec. IV "Mini-Batch Transfer To GPU").
 *   feats        the full feature matrix, row v at feats + v*feat_stride
 *                elements.  Pinned host memory (hipHostMalloc) or device
 *                memory; read by GPU kernels directly, so misses travel over
 *                the host link without a staging copy.
 *   cache_rows   device [num_cached x cache_stride]; slot s holds the row of
 *                node cached_ids[s].  NULL together with slot_of == NULL
 *                means "no cache": every row is read from feats (use this
 *                when feats itself is in HBM).
 *   slot_of      device [num_nodes]; cache slot of a node or -1.
 *   cached_ids   device [num_cached], graph idx_type; may be NULL if not wanted.
 * Strides are in elements of dtype.  Rows are moved as opaque bytes.
 */
typedef struct mqg_cache {
    int64_t num_nodes;
    int64_t num_cached;
    int32_t dim;
    int32_t dtype;                       /* mqg_dtype                                    */
    const void *feats;
    int64_t feat_stride;
    void *cache_rows;
    int64_t cache_stride;
    int32_t *slot_of;
    void *cached_ids;
} mqg_cache;

/*
 * One bipartite block (the topology part of a mini-batch, Sec. IV
 * "Mini-Batch Transfer To GPU").  Caller-allocated device buffers:
 *   src_ids  [cap_src]    global ids of the source nodes.  The first num_dst
 *                         entries are the destination nodes, in order, so a
 *                         destination's own previous-layer row (the second
 *                         half of the concatenation in Eq. 16) is row i of the
 *                         source matrix.  The remaining entries are the
 *                         sampled neighbours not among the destinations,
 *                         each once, ascending by id.
 *   indptr   [cap_dst+1]  CSR offsets of the sampled neighbours per destination.
 *   indices  [cap_nnz]    position in src_ids of each sampled neighbour; within
 *                         a row in ascending order of adjacency slot.
 *   sizes    [4]          int64, written on the device: num_dst, num_src, nnz,
 *                         and a flags word (0 = ok; in the innermost block bit 0
 *                         = some seed id was outside [0, num_nodes) and has been
 *                         replaced by node 0, bit 1 = a seed id occurs more
 *                         than once; the batch is then not a valid sample:
 *                         repeated ids keep their rows, the bounds below count
 *                         distinct ones, and the last of the sources that do
 *                         not fit are left out, edges to them point at 0).
 * Capacity bounds checked by mqg_sample_blocks (MQG_ERR_CAPACITY otherwise), with
 * need_dst(L-1) = num_seeds and need_dst(l) = need_src(l+1):
 *   cap_dst >= need_dst,  cap_nnz >= need_nnz = need_dst * fanouts[l],
 *   cap_src >= need_src = max(need_dst, min(num_nodes, need_dst + need_nnz)).
 */
typedef struct mqg_block {
    int64_t cap_dst;
    int64_t cap_src;
    int64_t cap_nnz;
    void *src_ids;
    int32_t *indptr;
    int32_t *indices;
    int64_t *sizes;
} mqg_block;

/* Library version (major*10000 + minor*100 + patch). */
int32_t mqg_version(void);

/*
 * Create a context for graphs of g's size and batches of at most max_seeds
 * seeds expanded with at most max_fanouts[l] (host array, length L) neighbours
 * per node in block l.  Allocates the private scratch on the current HIP
 * device (about 4.2 bytes per graph node plus a few words per sampled edge of
 * the largest batch).  g's array pointers are not read here and may be NULL.
 */
int mqg_ctx_create(mqg_ctx **out, const mqg_graph *g, int32_t max_seeds,
                   const int32_t *max_fanouts, int32_t num_layers);
int mqg_ctx_destroy(mqg_ctx *ctx);

/*
 * Allocate now what a context would otherwise allocate at the first use of an
 * optional path (with a stream synchronisation there), so that the calls
 * themselves only enqueue work.  `what` is a sum of:
 *   MQG_RESERVE_BACKWARD           scratch of the aggregations' backward, for blocks within the
 *                                  context's bounds (about 24 bytes per sampled edge)
 *   MQG_RESERVE_LAYERWISE          scratch of mqg_sample_layerwise and mqg_select_smallest_keys
 *                                  (about 32 bytes per graph node) for up to
 *                                  max(layerwise_rows, max_seeds) rows per block
 *   MQG_RESERVE_DEDUP_HASH         table and sort buffers of MQG_OPT_DEDUP_HASH
 *   MQG_RESERVE_SAMPLING_PRIORITY  tables of mqg_ctx_set_sampling_priority
 *   MQG_RESERVE_CACHE_BUILD        the temporaries of mqg_build_cache(_ex), about 75 bytes per
 *                                  graph node, kept until the context is destroyed.  With them a
 *                                  build allocates and frees nothing, and a build with
 *                                  MQG_CACHE_DEGREE_SAMPLED - the draw the paper repeats every
 *                                  epoch - returns as soon as its kernels are enqueued (builds on
 *                                  one context must then follow one another on one stream).
 *                                  MQG_CACHE_TOP_DEGREE still reads the maximum degree back and
 *                                  the random-walk policies the check of the training ids, so
 *                                  these wait for the stream; the push walk without
 *                                  graph_symmetric still allocates its transposed adjacency.
 * The call itself allocates and may synchronise the device; 0 for `what` does nothing.
 */
typedef enum { MQG_RESERVE_BACKWARD = 1, MQG_RESERVE_LAYERWISE = 2, MQG_RESERVE_DEDUP_HASH = 4,
               MQG_RESERVE_SAMPLING_PRIORITY = 8, MQG_RESERVE_CACHE_BUILD = 16 } mqg_reserve;
int mqg_ctx_reserve(mqg_ctx *ctx, int32_t what, int64_t layerwise_rows);

/* Message of the last failing call on ctx (or of the last failing
 * mqg_ctx_create on this thread when ctx is NULL).  Never NULL. */
const char *mqg_last_error(const mqg_ctx *ctx);

/* Tuning and test switches; see the MQG_OPT_* constants. */
typedef enum {
    MQG_OPT_FORCE_SLOW_SELECT = 1,       /* value != 0: every row with degree > fanout uses the
                                            repeated-minimum selection (test of the rare path) */
    MQG_OPT_PROFILE = 2,                 /* value != 0: bracket every kernel with HIP events
                                            (adds a few microseconds per kernel).  A gather
                                            through a cache then launches k_classify,
                                            k_gather_hit and k_gather_miss, as its two halves
                                            do, also where a call without profiling copies
                                            hits and misses in one launch                     */
    MQG_OPT_MISS_INFLIGHT_BYTES = 3,     /* bytes of host-memory reads the miss gather keeps
                                            outstanding (1 KiB..1 GiB, default 1 MiB): sizes
                                            its grid; enough to saturate the host link without
                                            crowding concurrent streams out of the memory system */
    MQG_OPT_HEAVY_DEGREE = 4,            /* destinations with more neighbours than this (>= 64,
                                            default 2048) are sampled by a whole workgroup
                                            instead of one wavefront; results do not change   */
    MQG_OPT_DEDUP_HASH = 5,              /* value != 0: frontier dedup and relabel through a hash
                                            table and a sort (memory proportional to the
                                            mini-batch) instead of the node-indexed bitmap and
                                            position table (4.2 bytes per graph node); same
                                            blocks, more kernel launches.  The first use
                                            allocates the table (synchronous)                */
    MQG_OPT_LAYERWISE_CANDIDATES = 6     /* how mqg_sample_layerwise finds the candidates of a
                                            layer: 0 = by graph size (default), 1 = a key slot per
                                            node, 2 = a list read off the masses, 3 = a list from
                                            bits set slot by slot; same blocks (test of the paths
                                            that only large graphs take)                      */
} mqg_option;
int mqg_ctx_set_option(mqg_ctx *ctx, int32_t option, int64_t value);

/*
 * With MQG_OPT_PROFILE on: sum of the HIP-event durations (milliseconds) and
 * number of launches of the kernel called `name` since the last reset.  The
 * call synchronises with the recorded events.  Unknown names give 0 launches.
 */
int mqg_ctx_kernel_time(mqg_ctx *ctx, const char *name, double *total_ms, int64_t *launches);
int mqg_ctx_reset_profile(mqg_ctx *ctx);
/* Names of the kernels seen so far, separated by '\n', into buf (host). */
int mqg_ctx_kernel_names(mqg_ctx *ctx, char *buf, int64_t buf_len);

/*
 * Feature cache (paper Sec. III "Feature Cache", Eq. 13: nodes enter the cache
 * by in-degree; here deterministically).  Ranks all nodes by (degree
 * descending, id ascending), assigns cache slot s to the s-th ranked node for
 * s < cache->num_cached, fills slot_of (-1 elsewhere), cached_ids (if not
 * NULL) and copies the cached rows from cache->feats into cache->cache_rows.
 * In: every field of *cache (buffers allocated by the caller).  Temporary
 * device memory (24 bytes per node, 8 per cached one) is allocated and freed inside the call,
 * which is therefore synchronous with respect to the host - unless
 * mqg_ctx_reserve(MQG_RESERVE_CACHE_BUILD) has set it aside beforehand.
 */
int mqg_build_cache(mqg_ctx *ctx, const mqg_graph *g, mqg_cache *cache, mqg_stream stream);

/*
 * The other ways the paper fills the cache (Sec. III "Feature Cache").
 *   MQG_CACHE_TOP_DEGREE      what mqg_build_cache does.
 *   MQG_CACHE_DEGREE_SAMPLED  Eq. 13 as stated: membership is drawn with probability proportional
 *                             to in-degree, without replacement - a fresh draw for every `seed`
 *                             (the paper rebuilds the cache every epoch).  Every adjacency slot j
 *                             of node v is a ticket with the uniform key
 *                             mix(mix(mix(mix(seed + G) ^ ~0) ^ v) ^ j); a node's key is the minimum
 *                             over its tickets (all ones without neighbours); the num_cached nodes
 *                             with the smallest (key, id) are cached, slot s = s-th smallest.
 *   MQG_CACHE_RANDOM_WALK     Eq. 14-15, for training sets that are a small part of the graph:
 *                             P(0) = 1/num_train on train_ids, 0 elsewhere, then num_steps steps with
 *                             the sampling ratio d_v = min(step_fanouts[l-1], deg_v) / deg_v (0 for an
 *                             empty row), deg_v the length of row v.  With A[v][u] = 1 for u in row(v)
 *                             (row v = the nodes v samples from) and D = diag(d), plan->walk_form
 *                             chooses how Eq. 15's matrix D A + I is applied:
 *                             MQG_WALK_PUSH (0, the default) along the direction in which sampling
 *                               moves, P(l) = (D A + I)^T P(l-1):
 *                                 P(l)[u] = P(l-1)[u] + sum over v with u in row(v) of d_v * P(l-1)[v],
 *                               the terms of u added in ascending order of v.  A node that holds mass
 *                               reaches each node of its row with probability d_v, so P(l)[u] is the
 *                               expected number of times u has entered the sampled frontier: the
 *                               nodes reached from the training set, which is what the cache wants.
 *                               The library transposes the adjacency for this (one stable sort of
 *                               the edges by column: about 24 bytes of temporary device memory per
 *                               edge, fewer than 2^31 edges) unless plan->graph_symmetric is set.
 *                             MQG_WALK_PRINTED (1) Eq. 15 exactly as printed, P a column vector,
 *                               P(l) = (D A + I) P(l-1):
 *                                 P(l)[i] = P(l-1)[i] + d_i * sum_{j in row(i)} P(l-1)[j],
 *                               the row summed in adjacency order, then scaled.  It moves mass
 *                               against the sampling direction; on a directed graph it scores nodes
 *                               that sampling from the training set never reaches, and after one
 *                               step from a uniform start every node of degree >= fanout scores alike.
 *                             On a graph that equals its transpose the push form is
 *                             P(l)[u] = P(l-1)[u] + sum_{v in row(u)} d_v * P(l-1)[v], (A D + I) P.
 *                             plan->graph_symmetric != 0 states that the graph equals its transpose
 *                             and that every row is in ascending order of id; the push form then sums
 *                             over the adjacency rows themselves and builds nothing.  The statement is
 *                             not checked: if it is false the result is that row-wise sum, not the
 *                             push form (no access leaves the arrays either way).
 *                             Double precision, products rounded on their own.  The num_cached nodes
 *                             of highest P(num_steps) are cached (ties: lower id).  scores_out
 *                             (device double [num_nodes], may be NULL) receives P(num_steps).
 *                             Membership is the deterministic top of the score, not a draw from it.
 *                             A training id outside [0, num_nodes) is never used as an index: it is
 *                             skipped and the call returns MQG_ERR_INVALID_ARG once the work is done.
 *   MQG_CACHE_RANDOM_WALK_SAMPLED  the same scores, membership drawn from them (the text after
 *                             Eq. 15 takes P(L) as the probability of entering the cache): weighted
 *                             sampling without replacement by an exponential race, key_i =
 *                             ticket_i / P(num_steps)[i] in double (+inf for a zero score),
 *                             ticket_i = -log2(r_i / 2^64) in fixed point with 32 fractional
 *                             bits, computed in integers by 32 squarings of the 64-bit mantissa
 *                             (truncated products), r_i = mix(mix(mix(mix(seed + G) ^ ~1) ^ i));
 *                             the num_cached smallest (key, id) are cached, slot s = s-th
 *                             smallest.
 * train_ids: device [num_train], graph idx_type, ids in [0, num_nodes); step_fanouts: host.
 */
typedef enum { MQG_CACHE_TOP_DEGREE = 0, MQG_CACHE_DEGREE_SAMPLED = 1, MQG_CACHE_RANDOM_WALK = 2,
               MQG_CACHE_RANDOM_WALK_SAMPLED = 3 } mqg_cache_policy;

typedef enum { MQG_WALK_PUSH = 0, MQG_WALK_PRINTED = 1 } mqg_walk_form;

typedef struct mqg_cache_plan {
    int32_t policy;                      /* mqg_cache_policy                             */
    int32_t num_steps;                   /* RANDOM_WALK: number of steps L, 0..MQG_MAX_LAYERS */
    uint64_t seed;                       /* DEGREE_SAMPLED, RANDOM_WALK_SAMPLED          */
    const void *train_ids;               /* RANDOM_WALK                                  */
    int64_t num_train;
    const int32_t *step_fanouts;         /* RANDOM_WALK: host [num_steps], each >= 1     */
    double *scores_out;                  /* RANDOM_WALK: optional                        */
    int32_t walk_form;                   /* RANDOM_WALK: mqg_walk_form                   */
    int32_t graph_symmetric;             /* RANDOM_WALK, push form: see above            */
} mqg_cache_plan;

/* mqg_build_cache with a choice of policy; plan == NULL means MQG_CACHE_TOP_DEGREE.  Otherwise as
 * mqg_build_cache (buffers in *cache, temporary device memory, synchronous with the host). */
int mqg_build_cache_ex(mqg_ctx *ctx, const mqg_graph *g, mqg_cache *cache, const mqg_cache_plan *plan,
                       mqg_stream stream);

/*
 * L-hop fixed-fanout node-wise neighbour sampling into blocks (paper Sec.
 * III-A, GraphSAGE paragraph: a fixed number of neighbours of every node of a
 * layer, drawn uniformly at random, a fresh draw per layer).
 *   seeds_dev  device [num_seeds], graph idx_type, distinct, in [0, num_nodes)
 *              (violations are flagged in blocks[L-1].sizes[3]; an id out of range
 *              is never used as an index)
 *   fanouts    host [num_layers], 1..MQG_MAX_FANOUT, indexed by block
 *   blocks     host array of num_layers descriptors (see mqg_block)
 * For each destination v of block l with adjacency row of length d: all d
 * neighbours if d <= fanouts[l]; otherwise the fanouts[l] adjacency slots j
 * with the smallest (key, j), key = mix(mix(mix(mix(rng_seed + G) ^ l) ^ v) ^ j)
 * with mix the SplitMix64 finaliser and G = 0x9E3779B97F4A7C15 - sampling
 * without replacement, a pure function of (rng_seed, l, v, j).
 */
int mqg_sample_blocks(mqg_ctx *ctx, const mqg_graph *g, const void *seeds_dev, int32_t num_seeds,
                      const int32_t *fanouts, int32_t num_layers, uint64_t rng_seed,
                      mqg_block *blocks, mqg_stream stream);

/*
 * mqg_sample_blocks with the sampling seed read from device memory when the
 * kernels run, for callers that record a mini-batch step into a HIP graph and
 * replay it: a recorded launch keeps its arguments, so what changes from one
 * replay to the next - the seeds in seeds_dev[0..num_seeds) and *rng_seed_dev -
 * has to live in buffers that the caller rewrites between replays.  Same
 * blocks as mqg_sample_blocks(..., rng_seed = *rng_seed_dev, ...).  With the
 * default dedup path and MQG_OPT_PROFILE off, this call, mqg_gather_features
 * and mqg_sage_mean_aggregate only enqueue kernels (no allocation, no memset,
 * no synchronisation) and can be captured.
 */
int mqg_sample_blocks_seed_dev(mqg_ctx *ctx, const mqg_graph *g, const void *seeds_dev, int32_t num_seeds,
                               const int32_t *fanouts, int32_t num_layers,
                               const uint64_t *rng_seed_dev, mqg_block *blocks, mqg_stream stream);

/*
 * Layer-wise sampling after LADIES (paper Sec. III-B, Eq. 6-9) into blocks of
 * the same layout, with edge weights.  blocks[L-1] has the seeds as rows; for
 * every block, from L-1 down to 0, with rows D:
 *   - column masses in integers: mass_i = sum over v in D with i in N(v) or
 *     i == v of floor(2^40 / (deg_v + 1)); q_i = mass_i / (deg_i + 1) is 2^40
 *     times the squared column norm ||R P_{*,i}||^2 of Eq. 7, P = D^-1/2 (A + I)
 *     D^-1/2 (Eq. 2); the candidates (Eq. 6) are the nodes with mass_i > 0;
 *   - layer_sizes[l] candidates are drawn without replacement with probability
 *     proportional to q_i (all of them if there are no more), by an
 *     exponential race: key_i = ticket_i * (deg_i + 1) / mass_i in doubles,
 *     ticket_i as for MQG_CACHE_RANDOM_WALK_SAMPLED from r_i =
 *     mix(mix(mix(mix(rng_seed + G) ^ (64 + l)) ^ i)); the smallest (key, id) win;
 *   - src_ids = the drawn nodes, ascending (they are the rows of block l-1;
 *     unlike mqg_sample_blocks the rows are not repeated among the sources);
 *     row v lists the drawn nodes among v itself and its adjacency row, the
 *     self edge first, then in slot order; edge_w[l][p] = P_vi / (s p_i) (Eq. 8),
 *     s the number of drawn nodes and p_i = q_i / sum_j q_j, divided by the
 *     row's sum if normalise != 0 (the normalisation of the sampled operator
 *     the paper mentions after Eq. 9; rows without an edge stay empty).
 * Which nodes are drawn is a pure function of the arguments (integer masses,
 * correctly rounded double operations); the weights are computed in double and
 * rounded to float.
 *   seeds_dev    device [num_seeds], graph idx_type, distinct; an id outside
 *                the graph is replaced by node 0 and flagged (sizes[3] bit 0)
 *   layer_sizes  host [num_layers], each >= 1
 *   blocks       host [num_layers]; block l needs cap_dst >= its number of rows
 *                (num_seeds for L-1, else min(N, layer_sizes[l+1])), cap_src >=
 *                min(N, layer_sizes[l]); edges beyond cap_nnz are dropped and
 *                flagged (sizes[3] bit 2; sizes[2] is then cap_nnz)
 *   edge_w       host array of num_layers device pointers, [cap_nnz] floats each
 * method MQG_LAYERWISE_FASTGCN (paper Sec. III-B, FastGCN paragraph, Eq. 4): the
 * masses are taken over all rows of the graph instead of the block's rows - the
 * squared column norms of P itself, computed at the first such call on the
 * context - so every node is a candidate and the draw does not depend on the
 * mini-batch; everything else is the same (drawn without replacement,
 * importance weights P_vu / (s p_u)).
 * method | MQG_LAYERWISE_DEBIAS (the "+debias" variants, paper Eq. 12): a drawn
 * node's column is scaled by its debiased coefficient beta instead of 1 / (s p),
 * edge_w = P_vi * beta_i (then the row normalisation, if asked for).  With the
 * drawn nodes in the order of the race (ascending (key, id)), n candidates,
 * a_r = n / ((n - r)(r + 1)) for the r-th draw (r from 0) and p_r = q_r / sum_j
 * q_j: the coefficient of a node is a_r (1 - p_0 - ... - p_{r-1}) / p_r when it
 * is drawn and becomes (1 - a_u) beta + a_u at every later draw u; when every
 * candidate is drawn, beta = 1.  Computed in double.
 * method | MQG_LAYERWISE_FLAT (the "+flat" variants, paper Eq. 10): nodes are
 * drawn with probability proportional to sqrt(q_i), the column norm itself
 * instead of its square - the distribution that minimises the variance of the
 * sampled product P (H W) when the rows of H W have equal norms, which is the
 * assumption the paper states (the printed right-hand side names the unknown
 * H W).  key_i = ((ticket_i * ticket_i) * (deg_i + 1)) / mass_i, the order of
 * ticket_i / sqrt(q_i); p_i = sqrt(q_i) / sum_j sqrt(q_j) in the weights and in
 * the debiased coefficients.  The three flags combine freely.
 * The first call allocates context scratch of about 32 bytes per graph node
 * (8 more for FastGCN) and synchronises the stream once.  Feed the blocks to
 * mqg_weighted_aggregate with self_w == NULL.
 */
typedef enum { MQG_LAYERWISE_LADIES = 0, MQG_LAYERWISE_FASTGCN = 1, MQG_LAYERWISE_DEBIAS = 2,
               MQG_LAYERWISE_FLAT = 4 } mqg_layerwise_method;

int mqg_sample_layerwise(mqg_ctx *ctx, const mqg_graph *g, const void *seeds_dev, int32_t num_seeds,
                         const int32_t *layer_sizes, int32_t num_layers, uint64_t rng_seed,
                         int32_t normalise, int32_t method, mqg_block *blocks,
                         float *const *edge_w, mqg_stream stream);

/*
 * The selection step of mqg_sample_layerwise on its own (the k smallest race
 * keys win the draw of Eq. 6-9): bit c of out_bitmap is set iff key c is among
 * the k smallest (key, index) pairs of keys[0..n) - all of them if n <= k; keys
 * that are exactly equal are taken in ascending index order.  A radix select:
 * two counting passes over the 25 leading bits, then the keys that share the
 * threshold's leading bits are settled as a short list.
 *   keys_dev        device [n] unsigned 64-bit keys
 *   out_bitmap_dev  device [ceil(n / 32)] words, written by the call
 * Uses the layer-wise sampler's context scratch (allocated at the first use; with
 * more keys than the graph has nodes, 12 more bytes per key, allocated and kept
 * at the first such call, after a stream synchronisation).
 */
int mqg_select_smallest_keys(mqg_ctx *ctx, const uint64_t *keys_dev, int64_t n, int64_t k,
                             uint32_t *out_bitmap_dev, mqg_stream stream);

/*
 * The selection step of mqg_sample_blocks for one row on its own (paper
 * Sec. III-A: s_node neighbours of a node drawn uniformly, here the k smallest
 * random keys): among `count` candidates, each a (key, slot word) pair, the k
 * first in the order (bit 31 of the slot word if `prioritised`, key, low 31
 * bits of the slot word) are chosen.  As the sampling kernels do it: by a bound
 * on the keys' upper 31 bits that exactly k lie below (prioritised: of the
 * candidates that compete, if those without bit 31 are fewer than k the others,
 * for the places that these leave), and where equal upper bits leave none, one
 * after the other by whole keys.  Exposed so that a test can feed it keys with
 * ties.
 *   keys_dev, slot_words_dev  device [count], 1 <= k <= count <= 256
 *   ordered         non-zero: the candidates are stored in ascending slot
 *                   order, so equal keys are resolved by position; zero: by
 *                   slot value
 *   out_mask_dev    device [8] words: bit c of the 256-bit mask = candidate c chosen
 */
int mqg_select_row_candidates(mqg_ctx *ctx, const uint64_t *keys_dev, const uint32_t *slot_words_dev,
                              int32_t count, int32_t k, int32_t prioritised, int32_t ordered,
                              uint32_t *out_mask_dev, mqg_stream stream);

/*
 * The ticket of the exponential races on its own (the draw from the random-walk
 * scores after Eq. 15 and the layer-wise draws of Eq. 6-10 race with key =
 * ticket / weight): tickets_dev[i] = ticket(r_i), r_i = mix(mix(mix(mix(seed + G)
 * ^ tag) ^ (first + i))) - slot 0 of node first + i in the key domain `tag` -
 * and ticket(r) = -log2(r / 2^64) in fixed point with 32 fractional bits as
 * described for MQG_CACHE_RANDOM_WALK_SAMPLED.  A pure integer function, exposed
 * so that a test can compare a long stretch of the stream, over thousands of
 * workgroups, with the same function computed on the CPU.
 *   tickets_dev  device [n] unsigned 64-bit
 */
int mqg_exp_tickets(mqg_ctx *ctx, uint64_t seed, int64_t tag, int64_t first, int64_t n,
                    uint64_t *tickets_dev, mqg_stream stream);

/*
 * Cache-prioritised neighbour sampling (paper Sec. I on global neighbour
 * sampling: the sampler prefers neighbours that are in the cache, which cuts
 * the number of distinct uncached rows a mini-batch needs).  After this call
 * every mqg_sample_blocks on `ctx` chooses, for a row with more neighbours than
 * the fanout k, the first k slots in the order (not cached, key, slot) with the
 * keys of mqg_sample_blocks: with c cached neighbours the row keeps min(k, c)
 * of them, uniformly, and fills up with uncached ones, uniformly.  Rows of at
 * most k neighbours are kept whole as before.
 * cache: membership is read from cache->slot_of (device, >= 0 = cached) into a
 * bitmap of num_nodes bits, and the number of cached neighbours of every node
 * of `graph` is tabulated (one pass over the adjacency, 4 bytes per node), both
 * owned by the context, on `stream`; call again after the cache has been
 * rebuilt.  cache == NULL switches back to the uniform draw (graph is then not
 * read).  The first call allocates the two tables.
 */
int mqg_ctx_set_sampling_priority(mqg_ctx *ctx, const mqg_graph *graph, const mqg_cache *cache,
                                  mqg_stream stream);

/*
 * Feature gather through the cache (paper Sec. IV "Mini-Batch Transfer To
 * GPU": rows of cached nodes come from GPU memory, the others from host
 * memory).  out[i, 0:dim] = F[ids[i], 0:dim] byte for byte.
 *   ids_dev      device [cap_ids], graph idx_type (normally blocks[0].src_ids)
 *   num_ids_dev  device int64: number of valid ids (normally &blocks[0].sizes[1]);
 *                values above cap_ids are clamped to cap_ids
 *   out_dev      device [cap_ids x out_stride] elements of cache->dtype; in a written row
 *                the elements from dim up to out_stride (padding) are unspecified: when
 *                source and destination rows are 64-byte (16-byte) aligned and long enough
 *                the copy is rounded up to whole 64-byte lines (16-byte words)
 *   stats_dev    device int64[2]: rows served from the cache, rows served
 *                from feats; may be NULL
 * An id outside [0, cache->num_nodes) is never used as an index: its output row
 * is left untouched and it counts in neither stat, so stats[0] + stats[1] below
 * the number of ids tells the caller that some were invalid.
 */
int mqg_gather_features(mqg_ctx *ctx, const mqg_cache *cache, int32_t idx_type,
                        const void *ids_dev, const int64_t *num_ids_dev, int64_t cap_ids,
                        void *out_dev, int64_t out_stride, int64_t *stats_dev, mqg_stream stream);

/*
 * The two halves of mqg_gather_features as calls of their own, for a pipeline
 * that keeps the host link busy (paper Sec. IV: transfer of one mini-batch
 * overlaps sampling and computation of others): the rows that come over the
 * host link are then copied on a stream that does nothing else, one
 * mini-batch after the other, while ids are classified and cached rows copied
 * elsewhere.
 *   mqg_gather_features_cached  looks the ids up, copies the rows found in the
 *       cache (HBM to HBM), writes both counts to stats_dev, and leaves the list
 *       of the other rows in the context;
 *   mqg_gather_features_missed  copies those rows from cache->feats.
 * Same arguments as mqg_gather_features; the pair, in this order, gives the
 * same rows and stats.  Every _cached call on a context must be followed by its
 * _missed call (same arguments) before the context gathers again, and the
 * caller orders the two (same stream, or an event) - the second reads what the
 * first left.  Without a cache (slot_of == NULL) every row belongs to the
 * second call and the first does nothing.
 */
int mqg_gather_features_cached(mqg_ctx *ctx, const mqg_cache *cache, int32_t idx_type,
                               const void *ids_dev, const int64_t *num_ids_dev, int64_t cap_ids,
                               void *out_dev, int64_t out_stride, int64_t *stats_dev, mqg_stream stream);
int mqg_gather_features_missed(mqg_ctx *ctx, const mqg_cache *cache, int32_t idx_type,
                               const void *ids_dev, const int64_t *num_ids_dev, int64_t cap_ids,
                               void *out_dev, int64_t out_stride, int64_t *stats_dev, mqg_stream stream);

/*
 * mqg_gather_features for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  It
 * takes no context (creating one allocates): the hit and miss lists and the
 * counters that mqg_gather_features keeps in its context live in a device array
 * of fixed size inside the library, MQG_GATHER_STATIC_MAX_IDS entries per list
 * (16 MiB + 64 bytes in all, held by every GPU the library runs on until the
 * process ends).  No call to hipMalloc, hipFree or any allocating routine is
 * made, at the first call or later; the first call on a device only looks up
 * the array's address there.  Same arguments, kernels, results and stats as
 * mqg_gather_features.  With a cache (slot_of != NULL) cap_ids above
 * MQG_GATHER_STATIC_MAX_IDS is refused with MQG_ERR_CAPACITY before anything
 * is enqueued; without a cache there is no limit (no list is used).  The
 * message of a failing call is read with mqg_last_error(NULL).  All calls on a
 * GPU share that GPU's array: two calls whose kernels can overlap there (two
 * streams, two threads) race, so keep them on one stream or order them with
 * events.
 */
#define MQG_GATHER_STATIC_MAX_IDS 1048576
int mqg_gather_features_static(const mqg_cache *cache, int32_t idx_type, const void *ids_dev,
                               const int64_t *num_ids_dev, int64_t cap_ids, void *out_dev,
                               int64_t out_stride, int64_t *stats_dev, mqg_stream stream);

/*
 * GraphSAGE mean aggregation over one block (paper Eq. 16,
 * Z_agg(v) = Mean(H(v)); the GA step "AH" of Sec. IV "Computation").
 *   out[i, c] = (1/n_i) * sum_{e in row i} x_src[indices[e], c],  n_i = row length;
 *   a destination with no sampled neighbour gets zeros.
 * x_src: device [num_src x x_stride]; out: device [cap_dst x out_stride];
 * strides in elements (columns from dim up to out_stride of a written row are
 * unspecified: with 16-byte aligned rows on both sides whole 16-byte words are
 * processed); sums are accumulated in fp32: partial sums (up to 64 for long rows of
 * few columns, up to four otherwise) take a row's entries by turns and are added up
 * at its end.  Rows with the same entries give the same bits, in this block or
 * another, with the same dim, dtype, strides and alignment; MQG_F16 rounds once, to
 * nearest even, at the store.
 */
int mqg_sage_mean_aggregate(mqg_ctx *ctx, const mqg_block *block, const void *x_src,
                            int64_t x_stride, void *out, int64_t out_stride, int32_t dim,
                            int32_t dtype, mqg_stream stream);

/*
 * Backward of the mean aggregation (paper Sec. IV "Computation": the gradient
 * of the GA step is the transposed product "AG", G the gradient matrix).  With
 * out = M x_src the forward operator of the block, M[i, s] = 1/n_i for every
 * edge of destination i that points to source s, this computes
 *   grad_x[s, c] = sum over edges (i -> s) of grad_out[i, c] / n_i
 * for all num_src sources (zeros where no edge points).
 * grad_out: device [num_dst x go_stride]; grad_x: device [cap_src x gx_stride];
 * strides in elements, padding columns of written rows unspecified as in the
 * forward.  The edges are first ordered by source, stably;
 * each source's terms come in ascending destination order and are summed as the
 * forward's entries are, so the result is reproducible bit for bit.  The first call (and any call with
 * larger block capacities than seen before) allocates context scratch of
 * about 20 bytes per edge and synchronises the stream once to do so.
 */
int mqg_sage_mean_aggregate_backward(mqg_ctx *ctx, const mqg_block *block, const void *grad_out,
                                     int64_t go_stride, void *grad_x, int64_t gx_stride, int32_t dim,
                                     int32_t dtype, mqg_stream stream);

/*
 * Weights of the sampled estimator of the graph convolution P H (paper Eq. 1-3),
 * P = D^-1/2 (A + I) D^-1/2 with D_ii = deg(v_i) + 1 (Eq. 2).  For block edge p
 * from destination i (node v_i) to source indices[p] (node v_j)
 *   edge_w[p] = deg(v_i) / n_i * 1 / sqrt((deg(v_i) + 1) (deg(v_j) + 1)),
 * n_i = the number of neighbours the block holds for v_i (Eq. 3 with s_node
 * read as the number actually drawn: a row kept whole has factor 1), and
 *   self_w[i] = P_ii = 1 / (deg(v_i) + 1)
 * is the diagonal term of A + I, which is never part of the sampled set.
 * deg is the length of the node's adjacency row in `graph`.  block->src_ids
 * must hold the sources' global ids, as mqg_sample_blocks writes them.
 * edge_w: device [cap_nnz] floats, self_w: device [cap_dst] floats; entries
 * 0..nnz-1 and 0..num_dst-1 are written (computed in double precision, rounded
 * once).  Enqueued on `stream`; nothing is allocated.
 */
int mqg_gcn_edge_weights(mqg_ctx *ctx, const mqg_graph *graph, const mqg_block *block,
                         float *edge_w, float *self_w, mqg_stream stream);

/*
 * Weighted aggregation over one block (the estimator of paper Eq. 1-3 with the
 * weights above, or any other per-edge weights, e.g. those of a layer-wise
 * sampler, Eq. 4-9):
 *   out[i, c] = self_w[i] * x_src[i, c] + sum over edges p of row i of
 *               edge_w[p] * x_src[indices[p], c]
 * self_w may be NULL (no diagonal term).  Layout, strides, dtype, padding and
 * accumulation as mqg_sage_mean_aggregate (fp32 sums, the diagonal term the
 * first of the row's terms).
 */
int mqg_weighted_aggregate(mqg_ctx *ctx, const mqg_block *block, const float *edge_w,
                           const float *self_w, const void *x_src, int64_t x_stride, void *out,
                           int64_t out_stride, int32_t dim, int32_t dtype, mqg_stream stream);

/*
 * Its backward (the transposed product, paper Sec. IV "Computation"):
 *   grad_x[s, c] = sum over edges p = (i -> s) of edge_w[p] * grad_out[i, c]
 *                  (+ self_w[s] * grad_out[s, c] for s < num_dst)
 * Buffers, ordering, reproducibility and scratch as
 * mqg_sage_mean_aggregate_backward (24 bytes of scratch per edge).
 */
int mqg_weighted_aggregate_backward(mqg_ctx *ctx, const mqg_block *block, const float *edge_w,
                                    const float *self_w, const void *grad_out, int64_t go_stride,
                                    void *grad_x, int64_t gx_stride, int32_t dim, int32_t dtype,
                                    mqg_stream stream);

/*
 * ---- The calls of a layer ------------------------------------------------------------------
 * What a training program does between two aggregations (the dense layer of Eq. 16's GraphSAGE
 * and its products are the caller's): the norm of the hidden rows with the residual's addition, the
 * aggregation of rows that are held in 8 bits, and the step of the weight matrices.  They take a
 * context for errors, profiling and scratch only; its graph is not used.  Rows and matrices may
 * be MQG_F32, MQG_F16 or MQG_BF16; strides are in elements, pointers need the alignment of an
 * element only, and, unlike in the calls above, nothing outside a row's dim columns is read or
 * written.  mqg_ctx_reserve_layer allocates now what mqg_rms_norm_backward and mqg_layer_norm_backward (for rows of up to norm_dim
 * columns) and mqg_orthogonalize and mqg_muon_step (for stacks of num_mats matrices of rows x cols) would
 * otherwise allocate when they are first called at that size, after a synchronisation of their stream
 * (it synchronises the device itself where it replaces smaller scratch, and is not for a time at which a stream is recorded):
 * up to 8 KiB per column for up to 2,048 columns, and for more 16 MiB or 2 KiB per column, whichever is more (the root-mean-square norm alone takes 2 KiB per column); 8 KiB per matrix, 12 bytes per element and 8 per element of the smaller side's square, sides rounded up to
 * multiples of 64 or 128, but nothing for matrices that one workgroup holds (with n and k sides in units of 32, n <= k, rounded up: n k <= 16
 * and 2 n k + n^2 <= 39, up to 32 x 512, 64 x 256 and 96 x 160).
 * While a stream is recorded into a HIP graph nothing is allocated: a call that would have to is
 * refused with MQG_ERR_UNSUPPORTED.  A recorded call goes on using the scratch that it was recorded with:
 * that stays allocated until mqg_ctx_destroy, also where later calls need more and get a larger one, and the graph may be
 * replayed until then (as any call on the context, by one stream at a time).  Pass 0 for what is not wanted.
 */
int mqg_ctx_reserve_layer(mqg_ctx *ctx, int32_t norm_dim, int32_t num_mats, int32_t rows, int32_t cols);

/*
 * Root-mean-square norm of rows, with the residual's addition:
 *   s = x + residual,  y = s * 1/sqrt(mean over the columns of s^2 + eps) * weight
 * computed in fp32 from the inputs (s * weight first, which has to stay within fp32's range); each output is rounded once.
 *   residual   may be NULL: s = x
 *   weight     device float [dim]; NULL = ones
 *   num_rows_dev  device int64, the number of rows (e.g. &blocks[l].sizes[1]); values above cap_rows
 *              are clamped to it, NULL = cap_rows
 *   sum        receives s (dtype), NULL if not wanted.  What the backward takes
 *   y          receives y (dtype), NULL if not wanted
 *   q, scale   receive y in 8 bits, NULL if not wanted (one of y and q is): one scale per row (group = 0) or per `group`
 *              columns (32, 64, 128; the last group of a row may be shorter),
 *              scale = max(max |y| / top, 2^-126), top = 448 for MQG_Q_E4M3 and 127 for MQG_Q_INT8,
 *              q = y / scale rounded to nearest, ties to even.  A group that holds a value that is
 *              not finite has the scale NaN, so that all its values read NaN.
 *              q: device bytes [cap_rows x q_stride], scale: device float [cap_rows x scale_stride]
 * A row of zeros gives zeros, with eps = 0 too, and so does a row whose 1/sqrt(...) is above fp32's numbers (a root mean square below
 * 2^-128); rows of any other size have their norm, whatever becomes of their squares in fp32.  sum and y may each be the buffer of x or of residual if its stride is the same.
 * dim <= MQG_NORM_MAX_DIM.
 */
#define MQG_NORM_MAX_DIM 16384
typedef enum { MQG_Q_E4M3 = 0, MQG_Q_INT8 = 1 } mqg_qtype;
int mqg_rms_norm(mqg_ctx *ctx, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight,
                 float eps, const int64_t *num_rows_dev, int64_t cap_rows, int32_t dim, int32_t dtype, void *sum, int64_t sum_stride,
                 void *y, int64_t y_stride, void *q, int64_t q_stride, int32_t q_type, int32_t group, float *scale, int64_t scale_stride,
                 mqg_stream stream);

/*
 * Its backward.  sum: the forward's s (its x where there was no residual); grad_y: the gradient of y (where y was
 * read in 8 bits: of the values that these stand for, the rounding is taken as the identity); grad_sum: the gradient that reaches s
 * by its other uses, NULL if it has none.  With R = 1/sqrt(mean(s^2) + eps), 0 where the forward gives zeros:
 *   grad_x = R (grad_y * weight - s * R^2 mean(grad_y * weight * s)) + grad_sum   (the gradient of x and of residual)
 *   grad_weight[c] = sum over the rows of grad_y * s * R    (device float [dim], written; NULL if not wanted)
 * Sums in fp32.  grad_weight is made of one sum per workgroup, added in a fixed order: the same bits in every call of the same
 * cap_rows, dim, dtype and number of rows.  grad_x may be the buffer of grad_y, grad_sum or sum if its stride is the same.
 */
int mqg_rms_norm_backward(mqg_ctx *ctx, const void *grad_y, int64_t gy_stride, const void *sum, int64_t sum_stride, const float *weight,
                          const void *grad_sum, int64_t gs_stride, float eps, const int64_t *num_rows_dev, int64_t cap_rows, int32_t dim,
                          int32_t dtype, void *grad_x, int64_t gx_stride, float *grad_weight, mqg_stream stream);

/*
 * Layer norm of rows, with the residual's addition:
 *   s = x + residual,  d = s - mean over the columns of s,  y = d * 1/sqrt(mean over the columns of d^2 + eps) * weight + bias
 * computed in fp32 from the inputs; each output is rounded once.  Arguments as mqg_rms_norm's, and
 *   bias   device float [dim]; NULL = zeros
 * A row of equal values gives the bias, with eps = 0 too, and so does a row whose 1/sqrt(...) is above fp32's numbers (one that spreads less than
 * 2^-128); rows of any other size and mean have their norm, whatever becomes of their sums and squares in fp32.  A row that holds a value that is not finite gives none that is.
 */
int mqg_layer_norm(mqg_ctx *ctx, const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight,
                   const float *bias, float eps, const int64_t *num_rows_dev, int64_t cap_rows, int32_t dim, int32_t dtype, void *sum,
                   int64_t sum_stride, void *y, int64_t y_stride, void *q, int64_t q_stride, int32_t q_type, int32_t group, float *scale,
                   int64_t scale_stride, mqg_stream stream);

/*
 * Its backward.  With d and R = 1/sqrt(mean(d^2) + eps) of the forward's s, 0 where that is above fp32's numbers (rows of equal values with eps = 0, and rows that spread
 * less than 2^-128), u = d R and h = grad_y * weight:
 *   grad_x = R (h - mean(h) - u mean(h u)) + grad_sum   (the gradient of x and of residual)
 *   grad_weight[c] = sum over the rows of grad_y * u,  grad_bias[c] = sum over the rows of grad_y    (device float [dim], written;
 *                    NULL if not wanted)
 * Arguments, sums, their order and buffers in place as mqg_rms_norm_backward's.
 */
int mqg_layer_norm_backward(mqg_ctx *ctx, const void *grad_y, int64_t gy_stride, const void *sum, int64_t sum_stride, const float *weight,
                            const void *grad_sum, int64_t gs_stride, float eps, const int64_t *num_rows_dev, int64_t cap_rows, int32_t dim,
                            int32_t dtype, void *grad_x, int64_t gx_stride, float *grad_weight, float *grad_bias, mqg_stream stream);

/*
 * mqg_sage_mean_aggregate of source rows in 8 bits with scales, as mqg_rms_norm writes them:
 *   out[i, c] = (1/n_i) * sum_{e in row i} scale[indices[e], c / group] * q[indices[e], c]
 *   (group = 0: one scale per row); a destination with no sampled neighbour gets zeros.
 * q: device bytes [num_src x q_stride]; scale: device float [num_src x scale_stride]; out: device [cap_dst x out_stride] of dtype.
 * Sums in fp32 (one that leaves its range is infinite), in an order that depends on the row's entries, dim and dtype alone; one rounding at the store.  Its backward, for the values that q
 * stands for, is mqg_sage_mean_aggregate_backward (of MQG_F32 and MQG_F16 gradients).
 */
int mqg_sage_mean_aggregate_q8(mqg_ctx *ctx, const mqg_block *block, const void *q, int64_t q_stride, int32_t q_type, int32_t group,
                               const float *scale, int64_t scale_stride, void *out, int64_t out_stride, int32_t dim, int32_t dtype,
                               mqg_stream stream);

/* A stack of num_mats matrices, element (r, c) of matrix i at data + i*mat_stride + r*row_stride + c. */
typedef struct mqg_matrices {
    int32_t num_mats, rows, cols;
    int32_t dtype;                       /* mqg_dtype                                    */
    void *data;                          /* device                                       */
    int64_t row_stride, mat_stride;
} mqg_matrices;

/* How an update is orthogonalised: `steps` steps (1..MQG_ORTH_MAX_STEPS) with coefficients (a, b, c) each (host float [3 * steps],
 * NULL = 3.4445, -4.7750, 2.0315 in all).  A plan of NULL means 5 such steps and eps = 1e-7. */
#define MQG_ORTH_MAX_STEPS 32
#define MQG_ORTH_MAX_SIDE 65536
#define MQG_ORTH_MAX_MATS 65535
typedef struct mqg_orth {
    int32_t steps;
    float eps;
    const float *coeffs;
} mqg_orth;

/*
 * The orthogonal factor of every matrix of a stack, by Newton-Schulz products: X = U / (|U|_F + eps), then per step
 *   A = X X^T,  X <- a X + (b A + c A^2) X          (with X^T X where U has more rows than columns)
 * which takes every singular value x to a x + b x^3 + c x^5 and keeps the singular vectors.  The usual coefficients take singular values
 * from about 0.001 up to 0.7 .. 1.2 in five steps; smaller ones stay smaller.  Rows and columns of zeros stay zeros, matrices of zeros with eps = 0 too; a matrix that holds a value that is not finite
 * gives one without a finite value.
 * Products are exact to about 22 bits with sums in fp32, whatever the types.  Coefficients that take singular values of up to
 * 1 above 256 are refused with MQG_ERR_UNSUPPORTED.
 *   update   any type;  out  any type, the same sizes; may be the update's buffer if the layout and the type are the same
 */
int mqg_orthogonalize(mqg_ctx *ctx, const mqg_matrices *update, const mqg_matrices *out, const mqg_orth *plan, mqg_stream stream);

/*
 * A step of the weights around it (the momentum's orthogonal factor as the update):
 *   momentum <- beta * momentum + grad;  U = nesterov ? grad + beta * momentum : momentum
 *   weight   <- (1 - lr * weight_decay) * weight - lr * scale * orthogonalize(U)
 * grad: any type; momentum, weight: MQG_F32, read and written in place.  `scale` is the caller's rule for the size of the step
 * (e.g. sqrt(max(1, rows / cols))).
 */
int mqg_muon_step(mqg_ctx *ctx, const mqg_matrices *grad, const mqg_matrices *momentum, const mqg_matrices *weight, float lr, float beta,
                  int32_t nesterov, float weight_decay, float scale, const mqg_orth *plan, mqg_stream stream);

/* How the moments of a parameter are held (mqg_adamw_step). */
typedef enum { MQG_STATE_F32 = 0, MQG_STATE_E4M3 = 1 } mqg_state_type;
#define MQG_ADAMW_BLOCK 128

/*
 * A tensor that an optimiser steps: numel elements, one after the other.  What is written (weight, copy, m, v and their scales) overlaps
 * no other buffer of the call (a step of tensors whose buffers do is refused); gradients may share memory with one another.  Any alignment of the element.
 */
typedef struct mqg_param {
    int64_t numel;
    void *weight;                        /* device [numel] of weight_type, read and written             */
    const void *grad;                    /* device [numel] of grad_type; NULL: the tensor is left alone */
    void *copy;                          /* device [numel] of copy_type, receives the weight rounded to it; NULL if not wanted */
    void *m, *v;                         /* device [numel]: the moments, float; or bytes with MQG_STATE_E4M3 */
    float *m_scale, *v_scale;            /* device [ceil(numel / MQG_ADAMW_BLOCK)]: MQG_STATE_E4M3 only */
    int32_t weight_type, grad_type, copy_type;   /* mqg_dtype                                           */
    int32_t state_type;                  /* mqg_state_type                                              */
    float lr_scale, decay_scale;         /* times the plan's lr and weight_decay: 1 in most, decay_scale 0 for biases and the like */
} mqg_param;

typedef struct mqg_adamw {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;                        /* the number of this step, 1, 2, ...                          */
    const int64_t *step_dev;             /* device; the same, read when the step runs (below 1: 1); NULL: step */
    const float *lr_dev;                 /* device; NULL: lr                                            */
    const float *grad_scale_dev;         /* device; what the gradients are multiplied by; NULL: 1       */
} mqg_adamw;

/*
 * The norm of all gradients of a list (their number, grad and grad_type are read; a grad of NULL counts as zeros), and the factor that clips them:
 *   n = mul * sqrt(sum over all gradients of g^2),   scale = mul * min(1, max_norm / n)
 * mul: what the gradients are to be multiplied by in any case (1, or one over a loss scale); max_norm: INFINITY = no limit.
 * norm, scale: device float, either may be NULL.  A norm that is not finite in fp32 gives the scale NaN, with which mqg_adamw_step steps nothing.
 * Squares are added in fp32 sixteen at a time and in double above, whatever the gradients' size, in an order that depends on the list's sizes, types
 * and addresses (their places in lines of 128 bytes) alone: the same bits in every call.  Nothing is allocated.
 */
int mqg_grad_norm(mqg_ctx *ctx, const mqg_param *params, int32_t num_params, float mul, float max_norm, float *norm, float *scale,
                  mqg_stream stream);

/*
 * An AdamW step of every tensor of a list, with g = grad_scale * grad:
 *   m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2
 *   weight <- (1 - lr weight_decay) weight - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * in fp32 (no change where the divisor is zero; an eps below 2^-126 counts as zero), each result rounded once, to nearest even.  Weights of 16 bits are rounded at every step, which loses steps of
 * less than half their last place: keep those in MQG_F32 and take a copy of 16 bits.
 *   MQG_STATE_E4M3   m = m_scale * value and sqrt(v) = v_scale * value, e4m3 values with a scale per MQG_ADAMW_BLOCK elements in order (the last block may be
 *              shorter), scale = max(max |.| / 448, 2^-126), values rounded to nearest, ties to even, a root above zero to 2^-9 at least.  The step itself
 *              has the moments before they are rounded.  Zeros (bytes and scales) are the moments before the first step.  Rounding to nearest
 *              means that a root follows its block's largest one exactly and changes against it once it is half a step (up to a 16th) away.
 *              A block with a moment that is not finite gets the scale NaN.
 * A grad_scale that is not finite leaves everything as it is.  A recorded call reads step_dev, lr_dev and grad_scale_dev at every replay; `step` and
 * `lr` are those it was recorded with.  The list is read during the call only; nothing is allocated.
 */
int mqg_adamw_step(mqg_ctx *ctx, const mqg_param *params, int32_t num_params, const mqg_adamw *plan, mqg_stream stream);

/*
 * Depth of the mini-batch queue, i.e. how many mini-batches to keep in flight
 * (paper Sec. IV "Determining Optimal Queue Size", Eq. 22 and 23):
 *   C = floor(M_Q / M_batch),  M_Q = total_mem - peak_mem * (1 + margin_percent/100)
 *   Q = min(C, max(2, ceil(max_prepare_ms / mean_compute_ms)))
 * max_prepare_ms is the largest observed sampling + transfer time of a
 * mini-batch, mean_compute_ms the mean time of the stage that consumes it,
 * peak_mem the measured peak device memory of one training epoch, margin the
 * paper's 5-10 % safety margin, mem_per_batch the device memory one queued
 * mini-batch holds.  Host arithmetic only (doubles for the times, integers
 * for the memory); no GPU is touched.  The rule presumes a pipeline that waits
 * for its consumer: where preparation is bound by something a deeper queue
 * cannot hide (here: the host link), the depth it gives is harmless but buys
 * nothing beyond the first few.  *cap_out (may be NULL) receives C,
 * *queue_size_out receives Q.  MQG_ERR_INVALID_ARG for non-positive times or
 * sizes, a margin outside 0..100, or peak memory above the total.
 */
int mqg_queue_size(double max_prepare_ms, double mean_compute_ms, int64_t total_mem_bytes,
                   int64_t peak_mem_bytes, int32_t margin_percent, int64_t mem_per_batch_bytes,
                   int64_t *cap_out, int64_t *queue_size_out);

#ifdef __cplusplus
}
#endif
#endif /* MQG_H */
