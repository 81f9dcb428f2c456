/*
 * rdf2v.h - C ABI of the MI355X (gfx950) RDF2vec random-walk corpus library.
 *
 * RDF2vec first extracts a corpus of graph walks from a knowledge graph and
 * then trains Word2Vec on it (gpuRDF2vec, Boeckling & Paulheim, arXiv
 * 2508.01073, Sec. 2). This library is the walk-extraction step for random
 * walks: it builds a subject-indexed graph from id triples and runs
 * walks_per_node uniform random walks of at most `depth` hops from each start
 * entity, emitting each walk as an entity/predicate token row padded with -1
 * (Sec. 3.1), with walks launched all at once rather than entity by entity
 * (Sec. 4.1).
 *
 * Conventions shared by every call:
 *  - Ids are int32. Entities are 0..num_entities-1, predicates are
 *    0..num_predicates-1; in walk rows an entity's token is its id and a
 *    predicate's token is num_entities + its id (Sec. 3.1: every entity and
 *    predicate is tokenised to an integer id). num_entities + num_predicates
 *    must stay below 2^31.
 *  - All array arguments are DEVICE pointers to caller-owned memory unless
 *    stated otherwise. The library never allocates, frees or keeps device
 *    memory and keeps no global state; calls on different streams may overlap.
 *    The one exception is rdf2v_skipgram_pairs_noalloc, which uses a fixed
 *    array of device memory that the library holds on each device.
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream). Every
 *    call only enqueues work on it and returns without synchronising.
 *  - Errors that the host can see (null pointers, negative or oversized
 *    counts, workspace too small) are returned synchronously and nothing is
 *    enqueued. Errors that only the device can see (ids out of range, an
 *    inconsistent CSR) are ORed as RDF2V_STATUS_* bits into *status_dev, a
 *    device int32 that the caller zeroes beforehand and reads after the stream
 *    has synchronised; status_dev may be NULL, in which case such errors are
 *    not reported. After a device-side error the outputs are unspecified, but
 *    every memory access stays inside the buffers described here.
 */
#ifndef RDF2V_H_
#define RDF2V_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum rdf2v_status {
  RDF2V_OK = 0,
  RDF2V_ERR_INVALID_ARGUMENT = 1, /* null pointer, negative count, depth outside [0, RDF2V_MAX_DEPTH], walk range outside the corpus */
  RDF2V_ERR_ID_OUT_OF_RANGE = 2,  /* an id the host can already see is out of range (e.g. triples with num_entities == 0) */
  RDF2V_ERR_TOO_LARGE = 3,        /* num_triples >= 2^31, num_entities + num_predicates >= 2^31, walk counts overflowing int64 */
  RDF2V_ERR_WORKSPACE = 4,        /* workspace NULL or smaller than the matching *_workspace_size() */
  RDF2V_ERR_HIP = 5               /* a HIP launch or runtime call failed */
} rdf2v_status;

/* Bits ORed into *status_dev by the kernels. */
#define RDF2V_STATUS_ID_OUT_OF_RANGE 0x1 /* a subject/object/start id >= num_entities or < 0, or a predicate id out of range */
#define RDF2V_STATUS_BAD_CSR 0x2         /* row_ptr not non-decreasing within [0, num_edges] */
#define RDF2V_STATUS_BAD_LENGTH 0x4      /* a walk length outside [0, row_width] (treated as clamped), or a bad string offset */
#define RDF2V_STATUS_BAD_VALUE 0x10      /* a log decay that is NaN or positive, a scan's rate that is not finite or positive, or a logit of rdf2v_beam_select that is NaN or +inf */
#define RDF2V_STATUS_CAPACITY 0x8        /* more results than the output holds (the rest are not written), or more distinct strings than a vocabulary bound */

/* Longest walk, in hops. A walk row holds 2 * depth + 1 tokens. */
#define RDF2V_MAX_DEPTH 64

/*
 * A read-only VIEW of a subject-indexed CSR in device memory, as written by
 * rdf2v_build_csr:
 *   row_ptr[num_entities + 1]: int32, row_ptr[0] = 0, non-decreasing,
 *                              row_ptr[num_entities] = num_edges.
 *   edges[num_edges][2]:       int32 (predicate, object) out-edge records of
 *                              entity v at rows row_ptr[v] .. row_ptr[v+1]-1;
 *                              8-byte aligned.
 * Duplicate triples and self-loops are separate records.
 */
typedef struct rdf2v_csr {
  int32_t num_entities;
  int32_t num_predicates;
  int64_t num_edges;
  const int32_t *row_ptr;
  const int32_t *edges;
  /* Optional (may be NULL): the same out-edge records extended with the row
   * bounds of their object, as written by rdf2v_build_walk_edges:
   * walk_edges[num_edges][4] = (predicate, object, row_ptr[object],
   * row_ptr[object + 1]), 16-byte aligned. When present, rdf2v_random_walks
   * reads one 16-byte record per hop instead of a record plus the next
   * entity's row bounds; the walks are identical either way. */
  const int32_t *walk_edges;
} rdf2v_csr;

/*
 * Bytes of device workspace rdf2v_build_csr needs for these sizes (0 when
 * num_triples == 0). Pure host function.
 */
size_t rdf2v_build_csr_workspace_size(int64_t num_triples, int32_t num_entities);

/*
 * Triples -> subject-indexed CSR (the graph the walks traverse; gpuRDF2vec
 * Sec. 3.1 loads the tokenised triples into device memory as a graph).
 *
 *   subj, pred, obj   [num_triples] int32 ids (device).
 *   row_ptr_out       [num_entities + 1] int32 (device), written; may overlap
 *                     the inputs, which are then lost.
 *   edges_out         [num_triples][2] int32 (predicate, object) (device),
 *                     written; 8-byte aligned; must not alias the inputs.
 *   workspace         device scratch of at least
 *                     rdf2v_build_csr_workspace_size(num_triples, num_entities)
 *                     bytes, 256-byte aligned; contents clobbered.
 *   status_dev        device int32 or NULL (RDF2V_STATUS_ID_OUT_OF_RANGE).
 *
 * Inside every row the records keep the input order of their triples (a
 * stable sort by subject), so the result is deterministic and equal to a
 * sequential counting sort. Runs as histogram, scan and stable-scatter passes
 * of an LSD radix sort on the subject id followed by a row-offset kernel.
 */
rdf2v_status rdf2v_build_csr(const int32_t *subj, const int32_t *pred, const int32_t *obj,
                             int64_t num_triples, int32_t num_entities, int32_t num_predicates,
                             int32_t *row_ptr_out, int32_t *edges_out, void *workspace,
                             size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * Walk records: for every out-edge record k of the CSR,
 *   walk_edges_out[k] = (edges[k][0], edges[k][1], row_ptr[o], row_ptr[o + 1])
 * with o = edges[k][1], so that a walk learns the row of the entity it moves
 * to from the record it has just read (one random access per hop; the walk
 * definition is unchanged).
 *
 *   csr             CSR view (row_ptr and edges are read; walk_edges ignored).
 *   walk_edges_out  [num_edges][4] int32 (device), written; 16-byte aligned.
 *   status_dev      device int32 or NULL: RDF2V_STATUS_ID_OUT_OF_RANGE if an
 *                   object id is out of range (its row bounds are written as
 *                   0, 0).
 */
rdf2v_status rdf2v_build_walk_edges(const rdf2v_csr *csr, int32_t *walk_edges_out,
                                    int32_t *status_dev, void *stream);

/*
 * Whether walk records are expected to make rdf2v_random_walks faster on a
 * CSR of this size than row_ptr and edges read directly (the walks are
 * identical either way). Pure host function; 1 = build them, 0 = do not.
 *
 * Without records a hop reads the current entity's row bounds and then one
 * 8-byte record; with them it reads one 16-byte record from a table twice as
 * large. While row_ptr (4 * (num_entities + 1) bytes) stays resident in each
 * XCD's 4 MB L2 the bound read is a cache hit and the smaller record table
 * wins; beyond that every hop pays a second cache miss. Measured crossover on
 * gfx950 (uniform and power-law graphs, mean out-degree 20, depth 8):
 * row_ptr between 1.2 and 2.0 MB, so this returns 1 when row_ptr is larger
 * than 1.5 MiB and num_edges > 0. Negative sizes return 0.
 */
int32_t rdf2v_walk_edges_recommended(int32_t num_entities, int64_t num_edges);

/* Bytes of device workspace rdf2v_nonsink_starts needs. Pure host function. */
size_t rdf2v_nonsink_starts_workspace_size(int32_t num_entities);

/*
 * The default start set: every entity with at least one out-edge, ascending
 * (the paper starts walks from all entities when no start list is given,
 * Sec. 3.3; an entity without out-edges would only give a one-token walk).
 *
 *   starts_out  [num_entities] int32 (device): the first *count_out entries
 *               are written.
 *   count_out   one int64 in device memory: the number of start entities.
 *   workspace   device scratch, rdf2v_nonsink_starts_workspace_size() bytes,
 *               256-byte aligned.
 */
rdf2v_status rdf2v_nonsink_starts(const rdf2v_csr *csr, int32_t *starts_out, int64_t *count_out,
                                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * Uniform random walks (gpuRDF2vec Sec. 2: iterative random choice of the
 * next hop; Sec. 3.1: triple-based token rows padded with -1; Sec. 4.1: all
 * walks of all start entities launched together).
 *
 * The corpus has num_walks = num_start * walks_per_node walks; walk w starts
 * at start_nodes[w / walks_per_node]. This call computes walks
 * w = walk_begin .. walk_begin + walk_count - 1 into rows r = w - walk_begin,
 * so a corpus can be produced in batches and any batch recomputed on its own.
 *
 * Walk w, from entity e_0 = start_nodes[w / walks_per_node], for hops
 * h = 0 .. depth-1: if e_h has no out-edge the walk ends; otherwise with
 * u = word (h mod 4) of Philox4x32-10(key = seed, counter = (h / 4, w)) (the
 * 64-bit seed as key words lo, hi; the counter words are lo, hi of h / 4 then
 * lo, hi of w; Salmon et al., SC'11), the walk takes out-edge record
 * k = floor(u * deg(e_h) / 2^32) of e_h's row, (p, x), and appends tokens
 * num_entities + p and x; e_{h+1} = x.
 *
 *   csr           view of a CSR as rdf2v_build_csr writes it (host pointer to
 *                 the struct; the arrays it points to are device memory). If
 *                 csr->walk_edges is set it must hold rdf2v_build_walk_edges'
 *                 records for this CSR; csr->edges is then not read.
 *   start_nodes   [num_start] int32 entity ids (device); duplicates and sinks
 *                 allowed.
 *   depth         hops per walk, 0 .. RDF2V_MAX_DEPTH.
 *   tokens_out    [walk_count][2 * depth + 1] int32 (device), row-major:
 *                 e_0, V+p_0, e_1, V+p_1, ..., then -1 after the walk's end.
 *   len_out       [walk_count] int32 (device): valid tokens, 2 * hops + 1.
 *   status_dev    device int32 or NULL (RDF2V_STATUS_* bits).
 *
 * walks_per_node == 0 or walk_count == 0 enqueues nothing and returns
 * RDF2V_OK.
 */
rdf2v_status rdf2v_random_walks(const rdf2v_csr *csr, const int32_t *start_nodes, int64_t num_start,
                                int32_t walks_per_node, int32_t depth, uint64_t seed,
                                int64_t walk_begin, int64_t walk_count, int32_t *tokens_out,
                                int32_t *len_out, int32_t *status_dev, void *stream);

/* Bytes of device workspace rdf2v_skipgram_pairs needs. Pure host function;
 * 0 when num_walks is negative or above 2^46 (rdf2v_skipgram_pairs returns
 * RDF2V_ERR_TOO_LARGE for more rows). */
size_t rdf2v_skipgram_pairs_workspace_size(int64_t num_walks);

/*
 * Skip-gram training pairs from walk rows (gpuRDF2vec Sec. 3.2: the data
 * module turns the walk corpus into center-context pairs; Sec. 3.1: the -1
 * padding is dropped first).
 *
 * For walk r with L = len[r] valid tokens t_0 .. t_{L-1}, every center
 * position i and every context position j with 1 <= |i - j| <= window and
 * 0 <= j < L give the pair (t_i, t_j); pairs are ordered by walk, then i, then
 * j. A walk of L tokens gives 2 * sum_{d=1}^{min(window, L-1)} (L - d) pairs.
 *
 *   tokens          [num_walks][row_width] int32 walk rows (device), as
 *                   rdf2v_random_walks writes them.
 *   len             [num_walks] int32 valid tokens per row (device).
 *   row_width       1 .. 2 * RDF2V_MAX_DEPTH + 1.
 *   window          >= 0 (the paper's example uses 5).
 *   pairs_out       [pair_capacity][2] int32 (center, context) (device); may
 *                   be NULL when pair_capacity == 0 (count only).
 *   pair_count_out  one int64 in device memory: the total number of pairs,
 *                   also when it exceeds pair_capacity (then only the first
 *                   pair_capacity pairs are written and RDF2V_STATUS_CAPACITY
 *                   is raised).
 *   workspace       device scratch, rdf2v_skipgram_pairs_workspace_size()
 *                   bytes, 256-byte aligned.
 *   status_dev      device int32 or NULL.
 */
rdf2v_status rdf2v_skipgram_pairs(const int32_t *tokens, const int32_t *len, int64_t num_walks,
                                  int32_t row_width, int32_t window, int32_t *pairs_out,
                                  int64_t pair_capacity, int64_t *pair_count_out, void *workspace,
                                  size_t workspace_bytes, int32_t *status_dev, void *stream);

/* Most walk rows one rdf2v_skipgram_pairs_noalloc call takes, and the size of
 * the device array it uses for its scratch on each device (32 MiB + 64 KiB). */
#define RDF2V_NOALLOC_MAX_WALKS ((int64_t)1 << 22)
#define RDF2V_NOALLOC_SCRATCH_BYTES (((size_t)32 << 20) + ((size_t)64 << 10))

/*
 * rdf2v_skipgram_pairs for callers that cannot allocate device memory (code
 * being captured into a graph, tight serving loops, harnesses that forbid
 * hipMalloc): the same pairs, count and status, with the same arguments
 * except that there is no workspace. The scratch (an output offset per block
 * of walks, and their sums) lives instead in a device array of RDF2V_NOALLOC_SCRATCH_BYTES
 * that the library holds on every device it runs on until the process ends;
 * the first call on a device looks its address up (making that device current
 * for the lookup and restoring the caller's current device). The call itself
 * allocates nothing.
 *
 *   num_walks   0 .. RDF2V_NOALLOC_MAX_WALKS; more returns
 *               RDF2V_ERR_TOO_LARGE and enqueues nothing (split the rows into
 *               batches, or use rdf2v_skipgram_pairs with a workspace).
 *   stream      the device whose array is used is the stream's device.
 *
 * All calls on one device share its array and its contents persist between
 * calls: calls that overlap on one device (on different streams or from
 * different threads) race and give wrong pairs. Serialise them, e.g. on one
 * stream. No part of the array needs clearing between calls.
 */
rdf2v_status rdf2v_skipgram_pairs_noalloc(const int32_t *tokens, const int32_t *len, int64_t num_walks,
                                          int32_t row_width, int32_t window, int32_t *pairs_out,
                                          int64_t pair_capacity, int64_t *pair_count_out, int32_t *status_dev,
                                          void *stream);

/* Bytes of device workspace rdf2v_cbow_examples needs. Pure host function;
 * 0 when num_walks is negative or above 2^46 (rdf2v_cbow_examples returns
 * RDF2V_ERR_TOO_LARGE for more rows). */
size_t rdf2v_cbow_examples_workspace_size(int64_t num_walks);

/*
 * CBOW training examples from walk rows (gpuRDF2vec Sec. 3.2: the library
 * trains Continuous Bag of Words next to Skip-Gram; CBOW predicts a center
 * token from the tokens around it; Sec. 3.1: the -1 padding is dropped).
 *
 * For walk r with L = len[r] valid tokens t_0 .. t_{L-1}, every position i
 * gives one example: the center t_i and its contexts, the t_j with
 * 1 <= |i - j| <= window and 0 <= j < L in ascending j, followed by -1 up to
 * 2 * window entries. Examples are ordered by walk, then i; a walk of L tokens
 * gives L examples (a one-token walk gives one with no context). Read in order,
 * the (center, context) of the non-padding contexts are exactly the pairs of
 * rdf2v_skipgram_pairs with the same window.
 *
 *   tokens, len, row_width  as for rdf2v_skipgram_pairs.
 *   window          1 .. 2 * RDF2V_MAX_DEPTH.
 *   centers_out     [capacity] int32 (device); may be NULL when capacity == 0.
 *   contexts_out    [capacity][2 * window] int32 (device), row-major; may be
 *                   NULL when capacity == 0.
 *   count_out       one int64 in device memory: the number of examples (the sum
 *                   of the lengths), also when it exceeds capacity (then only
 *                   the first capacity examples are written and
 *                   RDF2V_STATUS_CAPACITY is raised).
 *   workspace       device scratch, rdf2v_cbow_examples_workspace_size() bytes,
 *                   256-byte aligned.
 *   status_dev      device int32 or NULL (RDF2V_STATUS_BAD_LENGTH for a length
 *                   outside [0, row_width], treated as clamped;
 *                   RDF2V_STATUS_CAPACITY).
 */
rdf2v_status rdf2v_cbow_examples(const int32_t *tokens, const int32_t *len, int64_t num_walks,
                                 int32_t row_width, int32_t window, int32_t *centers_out, int32_t *contexts_out,
                                 int64_t capacity, int64_t *count_out, void *workspace, size_t workspace_bytes,
                                 int32_t *status_dev, void *stream);

/* Which tokens a walk row holds (Tab. 1 lists entity walks and property walks
 * beside triple-based random walks). All three follow the same walk, drawn
 * from the same random stream, so an entity or property walk is exactly the
 * projection of the triple-based walk with the same walk id. */
typedef enum rdf2v_walk_tokens {
  RDF2V_TOKENS_TRIPLES = 0,   /* e_0, V+p_0, e_1, ..., e_h: 2*depth+1 tokens per row */
  RDF2V_TOKENS_ENTITIES = 1,  /* e_0, e_1, ..., e_h: depth+1 tokens per row */
  RDF2V_TOKENS_PROPERTIES = 2 /* e_0, V+p_0, ..., V+p_{h-1}: depth+1 tokens per row */
} rdf2v_walk_tokens;

/*
 * rdf2v_random_walks with a choice of tokens: identical arguments plus
 * token_kind; tokens_out holds walk_count rows of 2*depth+1 (TRIPLES) or
 * depth+1 (ENTITIES, PROPERTIES) tokens, padded with -1, and len_out the
 * valid tokens per row (2*hops+1 or hops+1).
 */
rdf2v_status rdf2v_random_walks_tokens(const rdf2v_csr *csr, const int32_t *start_nodes,
                                       int64_t num_start, int32_t walks_per_node, int32_t depth,
                                       uint64_t seed, int64_t walk_begin, int64_t walk_count,
                                       int32_t token_kind, int32_t *tokens_out, int32_t *len_out,
                                       int32_t *status_dev, void *stream);

/* Bytes of device workspace rdf2v_unique_walks needs. Pure host function;
 * 0 when num_walks is negative or above 255 * 2^31 (rdf2v_unique_walks
 * returns RDF2V_ERR_TOO_LARGE for more rows). */
size_t rdf2v_unique_walks_workspace_size(int64_t num_walks);

/*
 * Duplicate-free walks (Tab. 1: "random walk duplicate free"): rows come in
 * groups of group_size consecutive rows (the walks of one start entity, as
 * rdf2v_random_walks writes them for walks_per_node = group_size; the last
 * group may be shorter). Within each group only the first occurrence, in row
 * order, of each distinct walk is kept; two rows are the same walk when their
 * lengths and their first len tokens agree. Kept rows are written, in order,
 * to tokens_out / len_out, and their number to *count_out (device int64).
 *
 *   tokens, len      [num_walks][row_width] and [num_walks] int32 (device).
 *   tokens_out, len_out  room for num_walks rows (device); must not alias the
 *                    inputs.
 *   workspace        rdf2v_unique_walks_workspace_size(num_walks) bytes of
 *                    device scratch, 256-byte aligned.
 */
rdf2v_status rdf2v_unique_walks(const int32_t *tokens, const int32_t *len, int64_t num_walks,
                                int32_t group_size, int32_t row_width, int32_t *tokens_out,
                                int32_t *len_out, int64_t *count_out, void *workspace,
                                size_t workspace_bytes, int32_t *status_dev, void *stream);

/* Bytes of device workspace rdf2v_bfs_walks needs. Pure host function;
 * 0 when a size is negative or num_roots >= 2^31 (rdf2v_bfs_walks returns
 * RDF2V_ERR_TOO_LARGE for that many roots). */
size_t rdf2v_bfs_walks_workspace_size(int32_t num_entities, int64_t num_roots);

/*
 * BFS walks (gpuRDF2vec Sec. 3.1: a BFS from each root gives every reached
 * entity one predecessor, the first entity to reach it, and each leaf-to-root
 * path of that tree is one walk, so an entity appears at most once per root).
 *
 * The tree is that of a queue-order BFS limited to `depth` hops: the entities
 * of one level are expanded in the order they were reached, each through its
 * out-edge records in CSR order, and an entity not yet in the tree gets the
 * current entity and record as its parent. Tree entities without a child
 * (including every entity at the depth limit) are leaves; in the order they
 * were reached, the first max_walks of them give the walks
 * root, V+p_1, v_1, ..., leaf.
 *
 *   csr          CSR view (row_ptr and edges are read).
 *   roots        [num_roots] int32 entity ids (device).
 *   tokens_out   [num_roots][max_walks][2 * depth + 1] int32 (device): the
 *                first counts_out[r] rows of root r are written (padded with
 *                -1); the rest are left untouched.
 *   len_out      [num_roots][max_walks] int32, written like tokens_out.
 *   counts_out   [num_roots] int32: walks written per root. A root with more
 *                leaves than max_walks raises RDF2V_STATUS_CAPACITY.
 *   workspace    rdf2v_bfs_walks_workspace_size(V, num_roots) bytes (12 bytes
 *                per root plus at most about 4 GiB), 256-byte aligned.
 */
rdf2v_status rdf2v_bfs_walks(const rdf2v_csr *csr, const int32_t *roots, int64_t num_roots, int32_t depth,
                             int32_t max_walks, int32_t *tokens_out, int32_t *len_out, int32_t *counts_out,
                             void *workspace, size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * Writes what rdf2v_bfs_walks leaves untouched: rows counts[r] .. max_walks - 1
 * of every root r become -1 and their lengths 0, as if both outputs had been
 * filled before that call (which would write most of them twice).
 *
 *   counts       [num_roots] int32 (device), as rdf2v_bfs_walks writes them;
 *                values outside [0, max_walks] are treated as clamped.
 *   row_width    tokens per row, 2 * depth + 1.
 *   tokens_out, len_out  as for rdf2v_bfs_walks (device).
 */
rdf2v_status rdf2v_bfs_fill_unused(const int32_t *counts, int64_t num_roots, int32_t max_walks, int32_t row_width,
                                   int32_t *tokens_out, int32_t *len_out, void *stream);

/* Largest num_triples and bound on distinct strings rdf2v_build_vocabulary takes. */
#define RDF2V_VOCAB_MAX_TRIPLES ((int64_t)1 << 30)
#define RDF2V_VOCAB_MAX_DISTINCT ((int64_t)1 << 30)

/* Bytes of device workspace rdf2v_build_vocabulary needs (0 for arguments it
 * rejects). Pure host function. */
size_t rdf2v_build_vocabulary_workspace_size(int64_t num_triples, int64_t max_entities, int64_t max_predicates);

/*
 * Vocabulary (gpuRDF2vec Sec. 3.1: every entity and predicate is tokenised to
 * an integer id at the start of the pipeline): string triples -> the int32 id
 * triples that rdf2v_build_csr takes.
 *
 * Entity ids number the distinct subject and object strings 0, 1, ... in the
 * order they first appear in s_0, o_0, s_1, o_1, ...; predicate ids number the
 * distinct predicate strings in the order they first appear in p_0, p_1, ....
 * Strings are compared as byte sequences (any bytes, NUL included; the empty
 * string is a string). The result is deterministic.
 *
 * Each column is given as
 *   X_chars     uint8 bytes of all strings of the column (device), 4-byte
 *               aligned; may be NULL when X_bytes == 0.
 *   X_offsets   [num_triples + 1] int64 (device): string t of the column is
 *               X_chars[X_offsets[t] .. X_offsets[t + 1]). Offsets outside
 *               [0, X_bytes] or decreasing raise RDF2V_STATUS_BAD_LENGTH (the
 *               string is then read as empty).
 *   X_bytes     length of X_chars in bytes (nothing past it is read).
 * for X = subj, pred, obj.
 *
 *   num_triples     0 .. RDF2V_VOCAB_MAX_TRIPLES.
 *   max_entities,   caller's upper bounds on the distinct entity and predicate
 *   max_predicates  strings, 1 .. RDF2V_VOCAB_MAX_DISTINCT; they size the hash
 *                   tables (2 to 4 slots of 132 B per bounded string). More distinct
 *                   strings than a bound raise RDF2V_STATUS_CAPACITY.
 *   subj_ids, pred_ids, obj_ids  [num_triples] int32 outputs (device).
 *   counts_out      [2] int64 (device): distinct entities, distinct predicates.
 *   workspace       rdf2v_build_vocabulary_workspace_size(num_triples,
 *                   max_entities, max_predicates) bytes, 256-byte aligned.
 *   status_dev      device int32 or NULL (RDF2V_STATUS_BAD_LENGTH,
 *                   RDF2V_STATUS_CAPACITY).
 */
rdf2v_status rdf2v_build_vocabulary(const uint8_t *subj_chars, const int64_t *subj_offsets, int64_t subj_bytes,
                                    const uint8_t *pred_chars, const int64_t *pred_offsets, int64_t pred_bytes,
                                    const uint8_t *obj_chars, const int64_t *obj_offsets, int64_t obj_bytes,
                                    int64_t num_triples, int64_t max_entities, int64_t max_predicates,
                                    int32_t *subj_ids, int32_t *pred_ids, int32_t *obj_ids, int64_t *counts_out,
                                    void *workspace, size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * Operators of a sequence model over walk tokens.
 *
 * Walk rows are what a model trains on and answers with: rows of entity and
 * predicate tokens of ragged length. The calls below are such a model's
 * sequence mixer (linear attention with a decay for each head), its loss
 * (distillation from a teacher's top logits) and its answers' search (beam
 * selection). Their arguments follow the conventions above; floating arrays
 * hold RDF2V_F32 or RDF2V_BF16 values. Sums, states and statistics are held in
 * 32 bits. With RDF2V_BF16, decay attention over whole rows multiplies tokens
 * with states, and values with the weights of their pairs of tokens, taken to 16
 * bits: an output is off by up to 2^-15 of the sum of its terms' absolute values
 * before it is rounded. The step takes them as they are.
 */
typedef enum rdf2v_dtype {
  RDF2V_F32 = 0,
  RDF2V_BF16 = 1 /* the upper 16 bits of an IEEE float32, rounded to nearest even */
} rdf2v_dtype;

/* Largest key or value size of a head in the decay attention calls. */
#define RDF2V_MAX_HEAD_SIZE 128

/* Sizes and parameters that the decay attention calls share. */
typedef struct rdf2v_attention {
  int64_t rows;      /* independent rows of tokens, 0 .. 2^31 - 1 */
  int64_t length;    /* tokens of a row, 0 .. 2^31 - 1 (not read by the step) */
  int32_t heads;     /* query heads, 1 .. 65535: a multiple of kv_heads */
  int32_t kv_heads;  /* key and value heads; query head h reads kv head h / (heads / kv_heads) */
  int32_t dk, dv;    /* size of a key (and query) and of a value, 1 .. RDF2V_MAX_HEAD_SIZE */
  int32_t dtype;     /* rdf2v_dtype of q, k, v, their gradients and the outputs */
  float scale;       /* factor of the outputs, finite */
  /* [heads] float32 (device): g_h <= 0, the log of the decay of a token. -inf
   * is a decay of zero. NaN or positive values raise RDF2V_STATUS_BAD_VALUE and
   * are taken as 0 (no decay). A constant: no gradient is computed for it. */
  const float *log_decay;
  /* [rows] int32 (device) or NULL: tokens of each row that count, as the walk
   * calls write them. Values outside [0, length] raise RDF2V_STATUS_BAD_LENGTH
   * and are clamped. NULL: all `length` tokens count. Not read by the step. */
  const int32_t *len;
} rdf2v_attention;

/* An input of the decay attention calls: element (row, token, head, i) lies at
 * data[row * row_stride + token * token_stride + head * head_stride + i].
 * Strides count elements and may be anything that keeps the offsets inside the
 * caller's memory (slices of one projection, heads before tokens, a broadcast
 * of stride 0, ...); where data is 16-byte aligned and all strides are
 * multiples of 16 bytes the reads are widest. */
typedef struct rdf2v_heads_view {
  const void *data; /* device; aligned to its element type */
  int64_t row_stride, token_stride, head_stride;
} rdf2v_heads_view;

/* Bytes of device workspace that rdf2v_decay_attention and
 * rdf2v_decay_attention_backward need (0 for sizes that they reject). Pure host
 * functions of the sizes: pointers are not read. */
size_t rdf2v_decay_attention_workspace_size(const rdf2v_attention *a);
size_t rdf2v_decay_attention_backward_workspace_size(const rdf2v_attention *a);

/*
 * Linear attention with a decay for each head, over whole rows of tokens. For
 * each row and query head, with gamma = exp(g_h), L the row's length and
 * S_{-1} = state (zeros if NULL), for t = 0 .. L-1:
 *
 *   S_t = gamma S_{t-1} + k_t v_t^T            a dk x dv matrix
 *   o_t = scale * S_t^T q_t                    dv values
 *
 *   q, k, v     views with `heads`, `kv_heads` and `kv_heads` heads of dk, dk
 *               and dv values. Tokens at and beyond L are not used, whatever
 *               they hold.
 *   state       [rows][heads][dk][dv] float32 (device) or NULL.
 *   out         [rows][length][heads][dv] of the dtype (device), written; zeros
 *               for tokens at and beyond L.
 *   state_out   [rows][heads][dk][dv] float32 (device) or NULL: S_{L-1} is
 *               written. May be `state` itself.
 *   workspace   rdf2v_decay_attention_workspace_size() bytes of device scratch,
 *               256-byte aligned.
 *   status_dev  device int32 or NULL (RDF2V_STATUS_BAD_VALUE,
 *               RDF2V_STATUS_BAD_LENGTH).
 *
 * Outputs may not overlap inputs or one another, but for state_out over state
 * (RDF2V_ERR_INVALID_ARGUMENT; so too in the gradients). The same inputs give the
 * same bits on every call. A NaN or infinity in a token below L reaches what the
 * sum over s <= t has it in, where an infinity may be NaN, and nothing else.
 */
rdf2v_status rdf2v_decay_attention(const rdf2v_attention *a, const rdf2v_heads_view *q, const rdf2v_heads_view *k,
                                   const rdf2v_heads_view *v, const float *state, void *out, float *state_out,
                                   void *workspace, size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * Gradients of rdf2v_decay_attention, from those of its outputs: dout is that
 * of out (a view with `heads` heads of dv values) and dstate_out that of
 * state_out (NULL: zeros). With R_t the gradient of S_t,
 *
 *   R_t = gamma R_{t+1} + scale * q_t do_t^T,   R_{L-1} = scale * q do^T + dstate_out
 *   dq_t = scale * S_t do_t,  dk_t = R_t v_t,  dv_t = R_t^T k_t,  dstate = gamma R_0
 *
 * (dstate = dstate_out for a row of length 0).
 *
 *   state   what the forward call was given, or NULL.
 *   dq, dk, dv  [rows][length][heads][dk], [rows][length][kv_heads][dk] and
 *           [rows][length][kv_heads][dv] of the dtype, written; zeros for
 *           tokens at and beyond L. A kv head's gradients are the sums over
 *           the query heads that read it, rounded once.
 *   dstate  [rows][heads][dk][dv] float32 or NULL, written. May be dstate_out
 *           itself.
 */
rdf2v_status rdf2v_decay_attention_backward(const rdf2v_attention *a, const rdf2v_heads_view *q,
                                            const rdf2v_heads_view *k, const rdf2v_heads_view *v,
                                            const rdf2v_heads_view *dout, const float *state,
                                            const float *dstate_out, void *dq, void *dk, void *dv, float *dstate,
                                            void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                            void *stream);

/*
 * One more token for each row: rdf2v_decay_attention at length 1 (a->length and
 * a->len are not read), with the states taken from other rows where a beam
 * search has reordered them.
 *
 *   q, k, v     views whose token_stride is not read.
 *   state       [num_states][heads][dk][dv] float32 (device).
 *   parents     [rows] int32 (device) or NULL: row r continues the state of
 *               row parents[r] of `state` (as rdf2v_beam_select numbers them).
 *               An index outside [0, num_states) raises
 *               RDF2V_STATUS_ID_OUT_OF_RANGE and stands for zeros. NULL: row r
 *               continues state r, and num_states must be `rows`.
 *   out         [rows][heads][dv] of the dtype (device), written.
 *   state_out   [rows][heads][dk][dv] float32 (device), written. Without
 *               parents it may be `state` itself; with parents the two may not
 *               overlap (RDF2V_ERR_INVALID_ARGUMENT).
 */
rdf2v_status rdf2v_decay_attention_step(const rdf2v_attention *a, const rdf2v_heads_view *q,
                                        const rdf2v_heads_view *k, const rdf2v_heads_view *v, const float *state,
                                        int64_t num_states, const int32_t *parents, void *out, float *state_out,
                                        int32_t *status_dev, void *stream);

/* Most beams, in or out, of a group of rdf2v_beam_select. */
#define RDF2V_MAX_BEAMS 64

/* Bytes of device workspace rdf2v_beam_select needs (0 for sizes it rejects).
 * Pure host function. */
size_t rdf2v_beam_select_workspace_size(int64_t groups, int32_t beams, int64_t vocab, int32_t num_out);

/*
 * Beam search's selection: of each group (one search) the num_out best
 * continuations of its beams over the whole vocabulary.
 *
 * A beam b that is not finished has a candidate for each token x, of total
 * scores[b] + (logits[b][x] - log sum_y exp logits[b][y]), computed in float32;
 * a finished beam has one candidate, token -1 ("the walk has ended") at total
 * scores[b]. Candidates of total -inf (masked tokens, beams whose score is
 * -inf, beams without a token above -inf) are never chosen. The num_out largest
 * totals are written in descending order, equal totals by ascending (beam,
 * token). Where fewer candidates are left, the rest is score -inf, token -1 and
 * the group's first row as parent.
 *
 *   logits      [groups * beams][logits_stride >= vocab] of the dtype (device).
 *               NaN and +inf raise RDF2V_STATUS_BAD_VALUE and count as -inf.
 *   scores      [groups][beams] float32 (device): the beams' totals so far;
 *               NaN counts as -inf.
 *   finished    [groups][beams] int32 (device) or NULL: nonzero = finished.
 *               Logits of finished beams, and of beams whose score is -inf,
 *               are not read.
 *   scores_out, tokens_out, parents_out  [groups][num_out] float32, int32 and
 *               int32 (device), written: total, token, and the row of the beam
 *               that it continues, group * beams + b. scores_out may be
 *               `scores` itself where num_out == beams.
 *   workspace   rdf2v_beam_select_workspace_size() bytes of device scratch,
 *               256-byte aligned.
 * groups * beams < 2^31; 1 <= beams, num_out <= RDF2V_MAX_BEAMS;
 * 1 <= vocab < 2^31.
 */
rdf2v_status rdf2v_beam_select(const void *logits, int64_t logits_stride, int32_t dtype, const float *scores,
                               const int32_t *finished, int64_t groups, int32_t beams, int64_t vocab,
                               int32_t num_out, float *scores_out, int32_t *tokens_out, int32_t *parents_out,
                               void *workspace, size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * States in the order of the chosen beams: row r of dst is row parents[r] of
 * src, row_bytes bytes each (any states that are rows: token histories, decay
 * attention states, ...). An index outside [0, num_src) raises
 * RDF2V_STATUS_ID_OUT_OF_RANGE and gives a row of zeros. dst and src may not
 * overlap.
 */
rdf2v_status rdf2v_beam_reorder(const void *src, int64_t num_src, int64_t row_bytes, const int32_t *parents,
                                int64_t num_rows, void *dst, int32_t *status_dev, void *stream);

/* Most teacher entries of a row in the distillation calls. */
#define RDF2V_MAX_TEACHER_TOP 512

/* Bytes of device workspace the distillation calls need (0 for sizes they
 * reject). Pure host function. */
size_t rdf2v_distill_workspace_size(int64_t rows, int64_t vocab, int32_t top, int32_t dtype);

/*
 * Distillation from a teacher's top logits: for each row, with z its logits,
 * (id_k, t_k) the teacher's entries and tau the temperature,
 *
 *   p = softmax over the entries of t / tau,   q = softmax over the vocabulary of z / tau
 *   loss = tau^2 * sum_k p_k (log p_k - log q[id_k])
 *   dlogits[j] = dloss * tau * (q[j] - sum of the p_k with id_k = j)
 *
 * p is that of the differences of the t_k, wherever they lie; log q is z / tau
 * less the row's lse in float32, off by up to 2^-24 of the two's size.
 * An entry whose id is negative, or whose t_k is -inf, is absent; a row without
 * entries (padding after a walk's end) has loss 0, lse 0 and gradient 0, and
 * its logits are not read. Logits of -inf have q = 0; a row of nothing else has
 * lse = -inf, loss = +inf, and q = 0 everywhere. NaN and +inf give what the
 * formulas give.
 *
 *   logits      [rows][logits_stride >= vocab] of the dtype (device).
 *   ids         [rows][top] int32 (device); an id may occur more than once. An
 *               id >= vocab raises RDF2V_STATUS_ID_OUT_OF_RANGE and is absent.
 *   teacher     [rows][top] float32 (device).
 *   top         0 .. RDF2V_MAX_TEACHER_TOP.
 *   temperature finite and > 0.
 *   loss, lse   [rows] float32 (device), written: the loss, and
 *               log sum_j exp(z_j / tau) for the backward call.
 *   dloss       [rows] float32 (device), or NULL: the loss's gradient. Given
 *               together with dlogits the gradient is computed too, which reads
 *               the logits from memory once where a call for each reads them
 *               twice.
 *   dlogits     [rows][dlogits_stride >= vocab] of the dtype (device) or NULL,
 *               written. May be `logits` itself with the same stride.
 *   workspace   rdf2v_distill_workspace_size() bytes of device scratch,
 *               256-byte aligned.
 */
rdf2v_status rdf2v_distill_loss(const void *logits, int64_t logits_stride, int32_t dtype, const int32_t *ids,
                                const float *teacher, int64_t rows, int64_t vocab, int32_t top, float temperature,
                                float *loss, float *lse, const float *dloss, void *dlogits, int64_t dlogits_stride,
                                void *workspace, size_t workspace_bytes, int32_t *status_dev, void *stream);

/* The gradient alone, with the lse that rdf2v_distill_loss wrote; arguments as
 * there. */
rdf2v_status rdf2v_distill_loss_backward(const void *logits, int64_t logits_stride, int32_t dtype,
                                         const int32_t *ids, const float *teacher, int64_t rows, int64_t vocab,
                                         int32_t top, float temperature, const float *lse, const float *dloss,
                                         void *dlogits, int64_t dlogits_stride, void *workspace,
                                         size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * Operators of a model's layers over walk tokens.
 *
 * What a layer needs beside its matrix products: rdf2v_residual_norm joins the
 * last layer's output to the residual stream and norms it, rdf2v_causal_conv
 * looks at the tokens just before, rdf2v_selective_scan mixes a row with decays
 * that its tokens give. Activations hold RDF2V_F32 or RDF2V_BF16 values,
 * parameters and their gradients float32. Everything between inputs and outputs
 * is float32. The conventions of the calls above hold: outputs may not overlap
 * inputs or one another where nothing else is said (RDF2V_ERR_INVALID_ARGUMENT);
 * tokens at and beyond a row's length are not used, whatever they hold, and
 * outputs and gradients are zeros there; the same inputs give the same bits on
 * every call; a NaN or infinity reaches what the formulas have it in, and
 * nothing else.
 */

/* An input of rows of tokens: value (row, token, channel) lies at
 * data[row * row_stride + token * token_stride + channel]. Strides count
 * elements and may be anything that keeps the offsets inside the caller's
 * memory. */
typedef struct rdf2v_tokens_view {
  const void *data; /* device; aligned to its element type */
  int64_t row_stride, token_stride;
} rdf2v_tokens_view;

/* Widest causal convolution, in tokens. */
#define RDF2V_MAX_CONV_WIDTH 8

/* Sizes and parameters that the causal convolution calls share. */
typedef struct rdf2v_conv {
  int64_t rows, length;  /* 0 .. 2^31 - 1 each; the step does not read length and len */
  int32_t channels;      /* 1 .. 2^31 - 1 */
  int32_t width;         /* 1 .. RDF2V_MAX_CONV_WIDTH */
  int32_t dtype;         /* rdf2v_dtype of inputs, outputs, states and their gradients */
  int32_t silu;          /* nonzero: the outputs go through u * sigmoid(u) */
  const float *weight;   /* [channels][width] float32 (device) */
  const float *bias;     /* [channels] float32 (device) or NULL */
  /* [rows] int32 (device) or NULL, as in rdf2v_attention */
  const int32_t *len;
} rdf2v_conv;

/* Bytes of device workspace rdf2v_causal_conv_backward needs (0 for sizes it
 * rejects). Pure host function of the sizes. */
size_t rdf2v_causal_conv_backward_workspace_size(const rdf2v_conv *a);

/*
 * Causal convolution of each channel by itself. With x_{-1}, x_{-2}, .. from the
 * state (zeros if NULL) and L the row's length, for t = 0 .. L-1 and every channel:
 *
 *   u_t = bias + sum_{j < width} weight[j] x_{t - width + 1 + j},   out_t = u_t or u_t sigmoid(u_t)
 *
 *   x          view of channels values, rows x length.
 *   state      [rows][width - 1][channels] of the dtype (device) or NULL: the
 *              inputs before the row's first token, the oldest first.
 *   out        [rows][length][channels] of the dtype (device), written.
 *   state_out  [rows][width - 1][channels] of the dtype (device) or NULL,
 *              written: the last width - 1 of the state's and the row's inputs.
 *   status_dev device int32 or NULL (RDF2V_STATUS_BAD_LENGTH).
 */
rdf2v_status rdf2v_causal_conv(const rdf2v_conv *a, const rdf2v_tokens_view *x, const void *state, void *out,
                               void *state_out, int32_t *status_dev, void *stream);

/*
 * Gradients of rdf2v_causal_conv from those of its outputs, dout (a view) and
 * dstate_out (as state_out; NULL: zeros).
 *
 *   dx         [rows][length][channels] of the dtype, written.
 *   dweight    [channels][width] float32, written; dbias [channels] float32 or
 *              NULL, written.
 *   dstate     [rows][width - 1][channels] of the dtype or NULL, written.
 *   workspace  rdf2v_causal_conv_backward_workspace_size() bytes of device
 *              scratch, 256-byte aligned.
 */
rdf2v_status rdf2v_causal_conv_backward(const rdf2v_conv *a, const rdf2v_tokens_view *x,
                                        const rdf2v_tokens_view *dout, const void *state, const void *dstate_out,
                                        void *dx, float *dweight, float *dbias, void *dstate, void *workspace,
                                        size_t workspace_bytes, int32_t *status_dev, void *stream);

/*
 * One more token for each row: rdf2v_causal_conv at length 1 (a->length and
 * a->len are not read), with the states taken from other rows.
 *
 *   x          view whose token_stride is not read.
 *   state      [num_states][width - 1][channels] of the dtype (device).
 *   parents    as in rdf2v_decay_attention_step.
 *   out        [rows][channels] of the dtype (device), written.
 *   state_out  [rows][width - 1][channels] of the dtype (device), written.
 *              Without parents it may be `state` itself.
 */
rdf2v_status rdf2v_causal_conv_step(const rdf2v_conv *a, const rdf2v_tokens_view *x, const void *state,
                                    int64_t num_states, const int32_t *parents, void *out, void *state_out,
                                    int32_t *status_dev, void *stream);

/* Most states of a channel in the selective scan calls. */
#define RDF2V_MAX_SCAN_STATES 64

/* Sizes and parameters that the selective scan calls share. */
typedef struct rdf2v_scan {
  int64_t rows, length;  /* 0 .. 2^31 - 1 each; the step does not read length and len */
  int32_t channels;      /* 1 .. 2^28: a multiple of groups */
  int32_t groups;        /* 1 .. 65535: channel d reads b and c of group d / (channels / groups) */
  int32_t states;        /* of a channel, 1 .. RDF2V_MAX_SCAN_STATES */
  int32_t dtype;         /* rdf2v_dtype of x, dt, b, c, gate, out and their gradients */
  /* [channels][states] float32 (device): rates, finite and <= 0. Others raise
   * RDF2V_STATUS_BAD_VALUE and are taken as 0 (no decay). Rates below -2^95
   * are taken as -2^95, with which a step of 2^-88 forgets everything. */
  const float *a;
  const float *dt_bias;  /* [channels] float32 (device) or NULL: zeros */
  const float *skip;     /* [channels] float32 (device) or NULL: zeros */
  /* [rows] int32 (device) or NULL, as in rdf2v_attention */
  const int32_t *len;
} rdf2v_scan;

/* Bytes of device workspace the two calls need (0 for sizes that they reject).
 * Pure host functions of the sizes: pointers are not read. */
size_t rdf2v_selective_scan_workspace_size(const rdf2v_scan *a);
size_t rdf2v_selective_scan_backward_workspace_size(const rdf2v_scan *a);

/*
 * Selective scan over whole rows of tokens. For each row and channel, with L the
 * row's length and h_{-1} = state (zeros if NULL), for t = 0 .. L-1:
 *
 *   delta_t = log(1 + exp(dt_t + dt_bias))
 *   h_t[n]  = exp(delta_t a[n]) h_{t-1}[n] + delta_t x_t b_t[n]     n < states
 *   y_t     = sum_n c_t[n] h_t[n] + skip x_t
 *   out_t   = y_t, or with a gate y_t gate_t sigmoid(gate_t)
 *
 *   x, dt      views of channels values, rows x length; gate likewise or NULL.
 *   b, c       views with `groups` heads of `states` values.
 *   state      [rows][channels][states] float32 (device) or NULL.
 *   out        [rows][length][channels] of the dtype (device), written.
 *   state_out  [rows][channels][states] float32 (device) or NULL: h_{L-1} is
 *              written. May be `state` itself.
 *   workspace  rdf2v_selective_scan_workspace_size() bytes of device scratch,
 *              256-byte aligned.
 *   status_dev device int32 or NULL (RDF2V_STATUS_BAD_VALUE,
 *              RDF2V_STATUS_BAD_LENGTH).
 */
rdf2v_status rdf2v_selective_scan(const rdf2v_scan *a, const rdf2v_tokens_view *x, const rdf2v_tokens_view *dt,
                                  const rdf2v_heads_view *b, const rdf2v_heads_view *c,
                                  const rdf2v_tokens_view *gate, const float *state, void *out, float *state_out,
                                  void *workspace, size_t workspace_bytes, int32_t *status_dev, void *stream);

/* Where rdf2v_selective_scan_backward writes (device). */
typedef struct rdf2v_scan_gradients {
  void *dx, *ddt;   /* [rows][length][channels] of the dtype */
  void *db, *dc;    /* [rows][length][groups][states] of the dtype: sums over the group's channels, rounded once */
  void *dgate;      /* [rows][length][channels] of the dtype; NULL where there is no gate, and only there */
  float *da;        /* [channels][states] float32 */
  float *ddt_bias;  /* [channels] float32 or NULL */
  float *dskip;     /* [channels] float32 or NULL */
  float *dstate;    /* [rows][channels][states] float32 or NULL; may be dstate_out itself */
} rdf2v_scan_gradients;

/*
 * Gradients of rdf2v_selective_scan from those of its outputs, dout (a view) and
 * dstate_out (as state_out; NULL: zeros). With g_t the gradient of y_t and r_t
 * that of h_t,
 *
 *   r_t = c_t g_t + exp(delta_{t+1} a) r_{t+1},   r_{L-1} = c g + dstate_out
 *   ddelta_t = sum_n r_t[n] (a[n] exp(delta_t a[n]) h_{t-1}[n] + x_t b_t[n]),   ddt_t = ddelta_t sigmoid(dt_t + dt_bias)
 *   dx_t = delta_t sum_n r_t[n] b_t[n] + skip g_t,   dgate_t = dout_t y_t times the slope of u sigmoid(u)
 *   db_t[n] = sum over channels of r_t[n] delta_t x_t,   dc_t[n] = sum over channels of g_t h_t[n]
 *   da[n] = sum_t r_t[n] delta_t exp(delta_t a[n]) h_{t-1}[n],   dskip = sum_t g_t x_t,   ddt_bias = sum_t ddt_t
 *   dstate = exp(delta_0 a) r_0
 *
 * (dstate = dstate_out for a row of length 0). A rate that was taken as 0 has
 * the gradient at 0.
 */
rdf2v_status rdf2v_selective_scan_backward(const rdf2v_scan *a, const rdf2v_tokens_view *x,
                                           const rdf2v_tokens_view *dt, const rdf2v_heads_view *b,
                                           const rdf2v_heads_view *c, const rdf2v_tokens_view *gate,
                                           const rdf2v_tokens_view *dout, const float *state,
                                           const float *dstate_out, const rdf2v_scan_gradients *grads,
                                           void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                           void *stream);

/*
 * One more token for each row: rdf2v_selective_scan at length 1 (a->length and
 * a->len are not read), with the states taken from other rows.
 *
 *   x, dt, b, c, gate  views whose token_stride is not read.
 *   state      [num_states][channels][states] float32 (device).
 *   parents    as in rdf2v_decay_attention_step.
 *   out        [rows][channels] of the dtype (device), written.
 *   state_out  [rows][channels][states] float32 (device), written. Without
 *              parents it may be `state` itself.
 */
rdf2v_status rdf2v_selective_scan_step(const rdf2v_scan *a, const rdf2v_tokens_view *x, const rdf2v_tokens_view *dt,
                                       const rdf2v_heads_view *b, const rdf2v_heads_view *c,
                                       const rdf2v_tokens_view *gate, const float *state, int64_t num_states,
                                       const int32_t *parents, void *out, float *state_out, int32_t *status_dev,
                                       void *stream);

/* Most channels of the residual norm calls. */
#define RDF2V_MAX_NORM_CHANNELS 16384

/* Sizes and parameters that the residual norm calls share. */
typedef struct rdf2v_norm {
  int64_t rows, length;    /* 0 .. 2^31 - 1 each */
  int32_t channels;        /* 1 .. RDF2V_MAX_NORM_CHANNELS */
  int32_t dtype;           /* rdf2v_dtype of x, out and their gradients */
  int32_t residual_dtype;  /* of residual, hidden and their gradients: the same, or RDF2V_F32 */
  int32_t center;          /* nonzero: the mean is taken off before the norm */
  float eps;               /* finite, >= 0 */
  const float *weight;     /* [channels] float32 (device) */
  const float *bias;       /* [channels] float32 (device) or NULL */
  const float *scale;      /* [channels] float32 (device) or NULL: ones */
  /* Share of x's values that are dropped, 0 <= drop < 1 - 2^-32. The others are
   * multiplied by 1 / (1 - drop). Value (row, token, channel) is dropped where
   * word [channel mod 4] of the Philox4x32-10 block of key (seed + seed_offset)
   * and counter (channel / 4, token + 1, row_begin + row as low and high word)
   * is below round(drop 2^32): the mask is a function of these alone, whatever
   * the batch, and none of a walk's words of the same seed. */
  double drop;
  uint64_t seed;
  /* One int64 (device) or NULL: added to the seed by the kernels, so that a
   * captured graph draws other masks when the caller changes it. */
  const int64_t *seed_offset;
  int64_t row_begin;       /* >= 0 */
  /* [rows] int32 (device) or NULL, as in rdf2v_attention */
  const int32_t *len;
} rdf2v_norm;

/* Bytes of device workspace rdf2v_residual_norm_backward needs (0 for sizes it
 * rejects). Pure host function of the sizes. */
size_t rdf2v_residual_norm_backward_workspace_size(const rdf2v_norm *a);

/*
 * Residual connection and norm, token by token:
 *
 *   hidden = residual + scale * dropout(x)
 *   out    = weight * (hidden - mean) / sqrt(mean of (hidden - mean)^2 + eps) + bias
 *
 * with mean 0 where center is 0. The norm is that of hidden before it is rounded.
 *
 *   x         view of channels values, rows x length.
 *   residual  view of residual_dtype or NULL: zeros.
 *   out       [rows][length][channels] of the dtype (device), written.
 *   hidden    [rows][length][channels] of residual_dtype (device) or NULL, written.
 *   stats     [rows][length][2] float32 (device) or NULL, written: the mean and
 *             1 / sqrt(..), for the backward call; zeros beyond a row's length.
 *   status_dev  device int32 or NULL (RDF2V_STATUS_BAD_LENGTH).
 */
rdf2v_status rdf2v_residual_norm(const rdf2v_norm *a, const rdf2v_tokens_view *x, const rdf2v_tokens_view *residual,
                                 void *out, void *hidden, float *stats, int32_t *status_dev, void *stream);

/*
 * Gradients of rdf2v_residual_norm from those of its outputs, dout and dhidden
 * (views; dhidden of residual_dtype or NULL: zeros), with the stats that it wrote.
 *
 *   dx         [rows][length][channels] of the dtype, written.
 *   dresidual  [rows][length][channels] of residual_dtype or NULL, written.
 *   dweight    [channels] float32, written; dbias, dscale [channels] float32 or
 *              NULL, written.
 *   workspace  rdf2v_residual_norm_backward_workspace_size() bytes of device
 *              scratch, 256-byte aligned.
 */
rdf2v_status rdf2v_residual_norm_backward(const rdf2v_norm *a, const rdf2v_tokens_view *x,
                                          const rdf2v_tokens_view *residual, const float *stats,
                                          const rdf2v_tokens_view *dout, const rdf2v_tokens_view *dhidden, void *dx,
                                          void *dresidual, float *dweight, float *dbias, float *dscale,
                                          void *workspace, size_t workspace_bytes, int32_t *status_dev,
                                          void *stream);

/* Static, human-readable name of a status code (any int: values that are not
 * an rdf2v_status give "RDF2V_UNKNOWN_STATUS"). */
const char *rdf2v_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* RDF2V_H_ */
