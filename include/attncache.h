/*
 * attncache.h -- C ABI of the MI355X (gfx950) AttnCache hot path.
 *
 * The library implements, on one GPU, the data-parallel part of AttnCache
 * (arXiv 2510.25979): similarity search over the feature-vector database,
 * reuse of a cached attention map (O = A_cached . V) and the exact causal
 * attention that serves queries without a hit.
 *
 * General rules
 *   - Plain C.  Every pointer argument says whether it is DEVICE memory
 *     (hipMalloc'd, e.g. a torch CUDA tensor's data_ptr()) or HOST memory.
 *   - Every function returns an int32_t status: AC_OK (0) or a negative
 *     AC_ERR_* code.  Nothing throws, aborts or prints.
 *   - The memory space of every pointer of a call is checked before anything
 *     is launched (AC_ERR_MEMSPACE: a host pointer never reaches a kernel and
 *     a device pointer is never dereferenced on the host).  The check is one
 *     driver query per pointer; it is skipped while `stream` is being
 *     captured into a graph, and attncache_set_pointer_checks(0) switches it
 *     off for loops that have validated their buffers once.
 *   - All GPU work is enqueued asynchronously on the caller's stream
 *     (`stream` is a hipStream_t passed as void*; NULL = the default
 *     stream).  A status covers argument validation and launch errors only.
 *   - The library never allocates or frees device memory.  Inputs, outputs,
 *     workspace and staging memory are owned by the caller; a database
 *     handle borrows the pointers it is given and the caller keeps that
 *     memory alive until attncache_destroy_db() and does not modify it
 *     behind the library's back (attncache_insert is the library's own
 *     way of writing it).
 *   - Tensors are dense, row-major, innermost index last, no padding.
 *     Every tensor base pointer must be 16-byte aligned.
 *   - Notation: B queries, N database feature vectors of dimension E,
 *     M map entries, L layers, Hq query heads, Hkv key/value heads
 *     (g = Hq / Hkv, query head h uses value head h / g), sequence length S,
 *     head dimension D.
 */
#ifndef ATTNCACHE_H
#define ATTNCACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ------------------------------------------------------ */
#define AC_OK 0
#define AC_ERR_NULL -1      /* a required pointer is NULL                      */
#define AC_ERR_SHAPE -2     /* a size is non-positive or unsupported           */
#define AC_ERR_DTYPE -3     /* unknown / unsupported element type or metric    */
#define AC_ERR_ALIGN -4     /* pointer not 16-byte aligned                     */
#define AC_ERR_K_RANGE -5   /* k outside 1..min(AC_MAX_K, N)                   */
#define AC_ERR_WORKSPACE -6 /* workspace / staging buffer too small            */
#define AC_ERR_INDEX -7     /* a hit index is outside [-1, M)                  */
#define AC_ERR_HIP -8       /* a HIP call failed, see attncache_last_hip_error */
#define AC_ERR_MEMSPACE -9  /* pointer is not in the memory space it must be   */
#define AC_ERR_NOMEM -10    /* a host-side allocation of the library failed     */

/* ---- element types, metrics ------------------------------------------- */
#define AC_F32 0
#define AC_F16 1  /* IEEE binary16 (feature vectors)                         */
#define AC_BF16 2 /* bfloat16 (maps, Q, K, V, O)                             */

#define AC_IP 0 /* similarity = inner product                               */
#define AC_L2 1 /* score = -||q - e||^2, similarity = 1 - ||q - e||          */

#define AC_LAYOUT_DENSE 0  /* each map is a row-major [S][S] matrix              */
#define AC_LAYOUT_PACKED 1 /* block-packed, see attncache_pack_maps (bf16 only)   */

#define AC_MAX_K 64

/* Size of the built-in search workspace of attncache_search_static. */
#define AC_STATIC_SCRATCH_BYTES (4u << 20)

/* ---- database ---------------------------------------------------------- */

/*
 * Description of the two stores of the paper's "Databases" paragraph
 * (Sec. 3.1): the feature-vector store that is searched and the
 * attention-map store that is fetched from.  Both share one index; when
 * several feature vectors refer to one map entry the optional table map_of
 * gives the entry of each vector.
 *
 * Supported: emb_dtype AC_F16 with emb_dim % 8 == 0 (16-byte rows) or AC_F32
 * with any emb_dim, either metric.  Inner products of fp16 rows run on the
 * matrix cores where emb_dim % 16 == 0 and emb_dim <= 512, and for more than
 * eight queries of other widths up to about 2,300 unless the database is small;
 * everything else (fp32, AC_L2) runs on the vector ALUs.  map_dtype AC_BF16
 * with seq_len % 32 == 0 and head_dim 64 or 128 (either layout), or map_dtype
 * AC_F32 with any seq_len and head_dim <= 256 (binary32 matrix instructions,
 * dense layout only).
 * n_q_heads % n_kv_heads == 0.
 */
typedef struct {
  int32_t n_emb;        /* N: feature vectors                                */
  int32_t emb_dim;      /* E                                                  */
  int32_t emb_dtype;    /* AC_F16 | AC_F32                                    */
  int32_t metric;       /* AC_IP | AC_L2                                      */
  int32_t n_entries;    /* M: map entries                                     */
  int32_t n_layers;     /* L                                                  */
  int32_t n_q_heads;    /* Hq                                                 */
  int32_t n_kv_heads;   /* Hkv                                                */
  int32_t head_dim;     /* D                                                  */
  int32_t seq_len;      /* S                                                  */
  int32_t map_dtype;    /* AC_BF16 | AC_F32                                   */
  int32_t causal;       /* 1: every map is exactly 0 above the diagonal and
                           those blocks are never read; 0: dense maps        */
  int32_t maps_on_host; /* 0: maps is DEVICE memory; 1: pinned HOST memory   */
  int32_t map_layout;   /* AC_LAYOUT_DENSE | AC_LAYOUT_PACKED                 */
} attncache_db_desc;

typedef struct attncache_db attncache_db; /* opaque, host-side */

/*
 * Bytes of DEVICE workspace attncache_search needs for up to max_batch
 * queries and top-k.  Written to *out.
 */
int32_t attncache_workspace_bytes(const attncache_db_desc *desc,
                                  int32_t max_batch, int32_t k, size_t *out);

/*
 * Bytes of one map entry (all layers and heads of one database item) in the
 * layout desc->map_layout.  Dense: L*Hq*S*S elements.  Packed causal:
 * L*Hq*(S/32)*(S/32+1)*512 elements (20 KiB instead of 32 KiB per head at
 * S = 128); packed non-causal: the same count as dense.
 */
int32_t attncache_map_entry_bytes(const attncache_db_desc *desc, size_t *out);

/*
 * Storage format conversion of the store step (Fig. 3, step 3): rewrite
 * n_entries dense maps into the packed layout the reuse kernel reads fastest.
 *
 *   dense   DEVICE [n_entries][L][Hq][S][S] bf16.
 *   packed  DEVICE, n_entries * attncache_map_entry_bytes(packed desc) bytes.
 *
 * Packed layout of one [S][S] map: rows are cut into blocks of 16, columns
 * into blocks of 32.  Row block r keeps its first nc(r) column blocks, nc(r) =
 * ceil((r+1)/2) for causal maps (everything above is zero by definition and is
 * dropped), S/32 otherwise.  Blocks are stored row-block-major; inside a block
 * (16 x 32 = 512 elements) element (i, 8q + e), q in 0..3, e in 0..7, sits at
 * offset (16q + i)*8 + e, which is the operand order of the 16x16x32 matrix
 * instruction.  desc->map_layout is ignored here (the result IS packed);
 * desc->map_dtype must be AC_BF16.  Entries can be converted in slices, so
 * the dense form never has to exist as a whole.
 */
int32_t attncache_pack_maps(const attncache_db_desc *desc, const void *dense,
                            int32_t n_entries, void *packed, void *stream);

/*
 * Store step of database building (Fig. 3, step 3): bind finished feature
 * vectors and attention maps into one searchable handle.
 *
 *   emb       DEVICE [N][E] of emb_dtype.
 *   map_of    DEVICE [N] int32 with values in [0, M), or NULL for the
 *             identity (requires N == M): map entry of each feature vector.
 *   maps      M entries of attncache_map_entry_bytes() each, of map_dtype, in
 *             the layout desc->map_layout (dense: [M][L][Hq][S][S]); DEVICE,
 *             or pinned HOST memory (hipHostMalloc) when desc->maps_on_host.
 *             Each row of each map sums to 1; with desc->causal the part
 *             above the diagonal is 0.  One entry is one contiguous block (all
 *             layers of one item lie together, as the paper's layer-adjacent
 *             layout).
 *   staging   DEVICE buffer of staging_bytes, used only when maps_on_host;
 *             must hold at least two entries.  NULL / 0 otherwise.  It is
 *             managed as a cache of whole entries (floor(staging_bytes /
 *             entry bytes) slots, least recently used slot replaced first;
 *             per call the entries that are already cached are served
 *             before the others, ascending entry number inside each class):
 *             an entry that an earlier attncache_apply left there is reused
 *             without a new copy, so spare HBM given here absorbs the popular
 *             entries of a skewed request stream (Sec. 3.1, locality of the
 *             stored maps).  The host maps must not change while the handle
 *             lives, or attncache_cache_reset() must be called.
 *   side_stream  hipStream_t on which host-to-device map copies are issued;
 *             used only when maps_on_host (must differ from the stream
 *             later passed to attncache_apply).
 *   out       receives the handle (host malloc; free with destroy).
 *
 * Validates sizes, types, alignment and the memory space of each pointer
 * (so a host pointer can never reach a kernel).  Copies nothing.
 */
int32_t attncache_build_db(const attncache_db_desc *desc, const void *emb,
                           const int32_t *map_of, const void *maps,
                           void *staging, size_t staging_bytes,
                           void *side_stream, attncache_db **out);

/* Releases the handle (and the events of the host-resident path).  The
 * caller must have synchronised the streams the handle was used on. */
int32_t attncache_destroy_db(attncache_db *db);

/*
 * Algorithm 1, search and threshold steps: exact top-k of the similarity
 * between each query and every database feature vector, then hit / miss
 * routing.
 *
 *   q         DEVICE [B][E] of the database's emb_dtype.
 *   k         1..min(AC_MAX_K, N).
 *   threshold theta: a query is a hit when the similarity of its best match
 *             is >= theta (compared in fp32).
 *   idx       DEVICE [B][k] int32 out: database rows, best first; equal
 *             scores are ordered by ascending row index.
 *   score     DEVICE [B][k] float out: fp32 scores (see AC_IP / AC_L2).
 *   hit       DEVICE [B] int32 out: map entry (map_of[idx[b][0]]) for a hit,
 *             -1 for a miss.
 *   ws        DEVICE workspace of ws_bytes >= attncache_workspace_bytes() for
 *             this or any larger max_batch.
 *
 * B == 0 is a no-op.  Scores are accumulated in fp32; the order of the
 * additions depends on the kernel that serves the shape, so two rows whose
 * exact scores differ by less than about 1e-6 relative may come out in
 * either order (rows with bit-identical feature vectors never do: the lower
 * index wins).  A query with a NaN component has no ordered scores: it is a
 * miss (hit -1), and its idx entries are -1 (score -inf) or name rows whose
 * score is NaN, depending on the kernel; nothing is read out of bounds.
 */
int32_t attncache_search(const attncache_db *db, const void *q, int32_t B,
                         int32_t k, float threshold, int32_t *idx,
                         float *score, int32_t *hit, void *ws, size_t ws_bytes,
                         void *stream);

/*
 * attncache_search for callers that cannot allocate or bring a workspace:
 * code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, same kernels and bit-identical results, but
 * the workspace is a fixed array of AC_STATIC_SCRATCH_BYTES (4 MiB) inside
 * the library's code object: every GPU the library runs on holds one copy
 * until the process ends.  The call allocates and frees nothing.
 *
 * Limit: batches that need more workspace than AC_STATIC_SCRATCH_BYTES
 * return AC_ERR_WORKSPACE (k = 1 fits up to about
 * 1,000 queries on a million-row index; large k on a large index does not).
 * All calls on one GPU share the one array: calls that overlap in time on
 * the same GPU (two streams, two threads, two handles) race and give wrong
 * results -- order them.  Nothing in it has to start at zero (every word
 * that is read was written by the same call before).  The array's device
 * address is looked up once per GPU, at attncache_build_db or at the first
 * call with that GPU current; when the first call of a process is to be
 * captured into a graph, build the handle beforehand (that is the norm).
 */
int32_t attncache_search_static(const attncache_db *db, const void *q,
                                int32_t B, int32_t k, float threshold,
                                int32_t *idx, float *score, int32_t *hit,
                                void *stream);

/*
 * Algorithm 2, reuse branch: O[b][l][h] = A[hit[b]][layer_begin+l][h] . V[b][l][h/g]
 * for l in [0, layer_count).  The maps are read in place from the database
 * (no gather copy) when they live in device memory.
 *
 *   hit       [B] int32 entry per query, -1 = miss.  DEVICE memory when the
 *             maps are in device memory; HOST memory when maps_on_host (the
 *             host schedules one copy per distinct entry and the indices
 *             are range-checked, AC_ERR_INDEX).
 *   V         DEVICE [B][layer_count][Hkv][S][D], element type = map_dtype.
 *   O         DEVICE [B][layer_count][Hq][S][D], element type = map_dtype.
 *             Rows of misses (hit[b] == -1) are not written.
 *
 * Device-resident maps: hit values outside [-1, M) are treated as misses by
 * the kernel (never dereferenced).  Host-resident maps: entries not yet in
 * the staging cache are copied on the side stream (one copy per distinct
 * entry, shared by all queries that hit it) and overlapped with the products
 * on `stream`; on return all work is enqueued, nothing is waited for.  Calls
 * on one handle must be issued in order (one stream, or ordered by the
 * caller): a slot remembers only its latest reader.
 * fp32 accumulation; bf16 results are rounded once (nearest even).
 */
int32_t attncache_apply(const attncache_db *db, const int32_t *hit,
                        const void *V, void *O, int32_t B, int32_t layer_begin,
                        int32_t layer_count, void *stream);

/*
 * Algorithm 2, recompute branch with the map of Sec. 4:
 * O = softmax(scale * Q K^T) V per (batch item, head); with causal != 0 keys
 * j > i are excluded.  Flash-style: the S x S map is never written.
 *
 *   Q         DEVICE [B][Hq][S][D]; K, V DEVICE [B][Hkv][S][D]; O DEVICE
 *             [B][Hq][S][D]; all of element type dtype (AC_BF16: S % 32 == 0,
 *             D 64 or 128; AC_F32: any S, D <= 256).  Q and K are taken as
 *             given (position encoding already applied).
 *   row_sel   NULL, or DEVICE [B] int32: items with row_sel[b] >= 0 are
 *             skipped and their O rows not written -- pass the hit array of
 *             attncache_search to compute only the misses.
 *   key_len   NULL, or DEVICE [B] int32: number of real tokens of sentence b
 *             in a batch padded on the right to S (values are clamped to
 *             [1, S]).  Keys j >= key_len[b] are hidden from every row (the
 *             attention mask of a padded batch, needed for non-causal
 *             models; with causal != 0 the rows inside the sentence never see
 *             the padding anyway) and chunks of keys that lie wholly in the
 *             padding are not read.  Rows i >= key_len[b] are padding
 *             themselves; they are computed by the same rule.
 *   scale     0 selects 1/sqrt(D).
 *
 * Softmax statistics and accumulators are fp32.
 */
int32_t attention_exact(const void *Q, const void *K, const void *V, void *O,
                        const int32_t *row_sel, const int32_t *key_len,
                        int32_t B, int32_t Hq,
                        int32_t Hkv, int32_t S, int32_t D, int32_t dtype,
                        int32_t causal, float scale, void *stream);

/*
 * Database building on the device (Fig. 3, steps 2 and 3: the attention maps
 * an input produced are stored under the input's feature vector): the
 * recompute branch for items that are to be remembered.  For every item b
 * with row_sel[b] < 0 (or row_sel == NULL)
 *
 *   O[b][l][h]                            = softmax(scale * Q K^T) V   (as attention_exact)
 *   maps[slot[b]][layer_begin + l][h]     = softmax(scale * Q K^T), rounded
 *                                           once to bf16, in the database's
 *                                           map layout (dense causal maps get
 *                                           their zeros above the diagonal)
 *   emb[slot[b]]                          = feat[b]
 *
 * for l in [0, layer_count), so that a later attncache_search hit on the slot
 * makes attncache_apply reproduce O from the stored map.  O is formed from
 * the ROUNDED map (what the reuse branch will read), fp32 accumulation.
 *
 *   db        map_dtype AC_BF16, maps in DEVICE memory (AC_ERR_DTYPE /
 *             AC_ERR_MEMSPACE otherwise).  This is the one entry point that
 *             WRITES the memory the handle borrows (feature rows and map
 *             entries of the named slots); the caller orders it against
 *             searches and reuses of the same slots (same stream, or events).
 *   feat      DEVICE [B][E] of emb_dtype, or NULL to store maps only (a
 *             layer-by-layer caller passes it once).  Requires map_of == NULL
 *             and N == M (one index for both stores) and E * sizeof(element)
 *             a multiple of 16.
 *   slot      DEVICE [B] int32: entry to overwrite, values outside [0, M)
 *             (e.g. -1) store nothing for that item.  NULL: nothing is stored
 *             at all.  Slots of one call must be distinct (equal slots race).
 *   row_sel   NULL or DEVICE [B] int32: items with row_sel[b] >= 0 are skipped
 *             entirely (pass the hit array to handle only the misses).
 *   key_len   NULL or DEVICE [B] int32: real tokens of sentence b in a batch
 *             padded on the right to S, as for attention_exact (clamped to
 *             [1, S]); keys in the padding get weight zero, and those zeros
 *             are what the stored map holds in their columns.
 *   Q         DEVICE [B][layer_count][Hq][S][D] bf16; K, V DEVICE
 *             [B][layer_count][Hkv][S][D]; O DEVICE like Q.
 *   scale     0 selects 1/sqrt(D).
 *
 * Two passes over the keys (row statistics first, then the normalised
 * weights), so it costs about twice the first product of attention_exact.
 */
int32_t attncache_insert(attncache_db *db, const void *feat,
                         const int32_t *slot, const int32_t *row_sel,
                         const int32_t *key_len, const void *Q, const void *K,
                         const void *V, void *O,
                         int32_t B, int32_t layer_begin, int32_t layer_count,
                         float scale, void *stream);

/*
 * Counters of the entry cache of a host-resident database since build /
 * reset: lookups = distinct entries requested, summed over attncache_apply
 * calls; copies = host-to-device entry copies issued.  HOST pointers.
 */
int32_t attncache_cache_stats(const attncache_db *db, uint64_t *lookups,
                              uint64_t *copies);

/* Forget every cached entry (after the host maps were modified) and zero the
 * counters.  The caller must have synchronised the streams the handle was
 * used on. */
int32_t attncache_cache_reset(attncache_db *db);

/*
 * Feature projector (Algorithm 1: f = feature_projector(h); Sec. 3.1
 * "Feature Projector": two MLP layers that map the input embedding to a
 * feature vector of lower dimension).  The step in front of
 * attncache_search: its output is a query block, or, for database building,
 * the `feat` argument of attncache_insert.  The paper fixes the two layers;
 * the pooling over tokens, the activation and the normalisation are this
 * library's reading:
 *
 *   x[b]    = mean of h[b][t] over the sentence's tokens t < seq_len[b]
 *   u[b]    = max(0, W1 x[b] + b1)
 *   f[b]    = W2 u[b] + b2,   divided by its Euclidean norm when `normalize`
 *             (a zero vector stays zero)
 *
 * All arithmetic is binary32 (fp32 matrix cores for the two layers).
 *
 *   h          DEVICE [B][S][model_dim], h_dtype AC_BF16 or AC_F32.
 *   seq_len    NULL (every sentence has S tokens) or DEVICE [B] int32; values
 *              are clamped to [1, S].  Tokens at and after seq_len[b] are not
 *              read.
 *   W1, b1     DEVICE fp32 [hidden_dim][model_dim] and [hidden_dim]
 *              (row j holds the weights of hidden unit j); b1 may be NULL.
 *   W2, b2     DEVICE fp32 [emb_dim][hidden_dim] and [emb_dim]; b2 may be NULL.
 *   feat       DEVICE [B][emb_dim], feat_dtype AC_F16 or AC_F32 (rounded to
 *              nearest even once, after normalisation).
 *   model_dim, hidden_dim, emb_dim   multiples of 8; emb_dim <= 2048;
 *              B <= 65535 (AC_ERR_SHAPE otherwise).  B == 0 is a no-op.
 *   workspace  DEVICE, attncache_project_workspace_bytes(...) bytes (0 is
 *              returned for non-positive sizes), 16-byte aligned; contents are
 *              scratch.  AC_ERR_WORKSPACE if too small.
 *
 * Two to four launches on `stream` by size; deterministic (partial sums are
 * added in a fixed order).  A workspace that is large enough, but smaller than
 * attncache_project_workspace_bytes(...) for these sizes, takes four.  Weights
 * and inputs are only read.
 */
size_t attncache_project_workspace_bytes(int32_t B, int32_t model_dim,
                                         int32_t hidden_dim, int32_t emb_dim);
int32_t attncache_project(const void *h, const int32_t *seq_len,
                          const float *W1, const float *b1, const float *W2,
                          const float *b2, void *feat, int32_t B, int32_t S,
                          int32_t model_dim, int32_t hidden_dim,
                          int32_t emb_dim, int32_t h_dtype, int32_t feat_dtype,
                          int32_t normalize, void *workspace,
                          size_t workspace_bytes, void *stream);

/* ---- generation after the prefill ---------------------------------------- */

/*
 * A paged K/V cache.  Reuse serves the prefill; a program that goes on
 * generating keeps K and V of the prompt and of every further token, and each
 * new token attends to all of them.  The cache is two arrays of pages,
 *
 *   k_pages, v_pages  [n_pages][heads][page_size][D], consecutive pages
 *                     page_stride elements apart (at least heads * page_size
 *                     * D; more where the cache holds further layers, whose
 *                     heads lie behind these, or K and V in one array).
 *                     Where a row of D elements is a whole number of 16-byte
 *                     pieces, page_stride must be one, too (AC_ERR_ALIGN).
 *
 * Token j of request b lies in page page_table[b][j / page_size] at place
 * j % page_size, in all heads; its slot is page * page_size + place.
 * n_pages * page_size must be below 2^31, max_pages * page_size at most 2^30.
 * Page numbers and slots that the kernels read are checked: what is outside
 * [0, n_pages) or [0, n_pages * page_size) is never followed.
 *
 * All pointers of these calls are to be memory of the current device
 * (AC_ERR_MEMSPACE for another device's, too).
 */

/*
 * The plan of a step: which pages the requests of a batch take and give back,
 * and where their new tokens go, from the requests' lengths, on the device.
 *
 *   seq_len    DEVICE [B] int32: tokens of each request that are in the cache
 *              (clamped to [0, max_pages * page_size]).
 *   new_len    DEVICE [B] int32: tokens to be added now (at most S are), 0 for
 *              none.  Negative: the request has ended and its pages go back.
 *   free_pages DEVICE [n_pages] int32: a ring of the pages that nobody has;
 *              free_state (DEVICE [2] int32) = index of the first, number.
 *   page_table DEVICE [B][max_pages] int32, in and out: entries below
 *              ceil(seq_len / page_size) are read, the new pages' entries
 *              written, all others left as they are.
 *   seq_len_out  DEVICE [B] int32 out: tokens after this step (0 for ended
 *              requests): what attention_paged takes once the rows are there.
 *   added      DEVICE [B] int32 out: tokens taken in, min(new_len, S) or 0.
 *   free_state_out  DEVICE [2] int32 out.
 *   slot       DEVICE [B][S] int32 out: slot of new token t, -1 from added[b]
 *              on: what attncache_page_append takes.
 *
 * Requests are served in their order.  One that needs more pages than the
 * ring has left takes nothing (added 0), and so do all after it that need a
 * page; those whose last page has room are served.  One that would outgrow
 * its max_pages takes nothing either.  Pages given back are the ring's for the
 * next call; they go behind its last one in order of request and place.  A
 * page is free or one request's: nothing may be in the ring or the tables
 * twice (attention_paged, which only reads, may be given shared pages).
 * The outputs seq_len_out, added, free_state_out may be seq_len, new_len,
 * free_state (a captured step then continues from where the last replay
 * ended); other arrays must not overlap.  B <= 2^22, S <= 2^25,
 * B * max_pages < 2^31 - 4096.  One launch, or two for many slots.  The
 * requests are looked through in order: 2^20 of one token take some 5 ms.
 */
int32_t attncache_page_plan(const int32_t *seq_len, const int32_t *new_len,
                            const int32_t *free_state, int32_t *free_pages,
                            int32_t *page_table, int32_t *seq_len_out,
                            int32_t *added, int32_t *free_state_out,
                            int32_t *slot, int32_t B, int32_t S,
                            int32_t max_pages, int32_t page_size,
                            int32_t n_pages, void *stream);

/*
 * Rows of K and V to their places: row t of head h of item b goes to slot
 * slot[b][t] of k_pages and v_pages; rows whose slot is outside
 * [0, n_pages * page_size), such as -1, are not read.
 *
 *   K, V       DEVICE [B][H][S][D] of dtype (AC_BF16: D 64 or 128; AC_F32:
 *              D <= 256), as attention_exact and attncache_insert take them
 *              (layers fold into heads); S = 1 for a generated token.
 *   slot       DEVICE [B][S] int32.  Slots of one call must be distinct
 *              (equal slots race).
 *   k_pages, v_pages  DEVICE, as above, with H heads.  Other places keep
 *              what they hold.
 * B * H * S below 2^31 - 4096.
 */
int32_t attncache_page_append(const void *K, const void *V,
                              const int32_t *slot, void *k_pages,
                              void *v_pages, int32_t B, int32_t H, int32_t S,
                              int32_t D, int32_t n_pages, int32_t page_size,
                              int64_t page_stride, int32_t dtype,
                              void *stream);

/*
 * Attention of one new token of each request to all tokens of its pages:
 * O[b][h] = softmax(scale * Q[b][h] K^T) V over the keys j < seq_len[b] of
 * K/V head h / (Hq / Hkv).
 *
 *   Q, O       DEVICE [B][Hq][D] of dtype (AC_BF16: D 64 or 128; AC_F32:
 *              D <= 256).
 *   page_table DEVICE [B][max_pages] int32.  Keys whose page is outside
 *              [0, n_pages) are hidden.
 *   seq_len    DEVICE [B] int32, clamped to [0, max_pages * page_size].  The
 *              new token's own K and V row is one of these keys if it has
 *              been appended before.  Places behind seq_len may hold anything.
 *              A request without a visible key gets zeros.
 *   scale      0 selects 1/sqrt(D).
 *   workspace  DEVICE, attention_paged_workspace_bytes(...) bytes (0 for sizes
 *              that are not positive), 16-byte aligned; scratch, and written
 *              by a call before it is read.  Its size depends on neither B nor
 *              the lengths.  Calls that may overlap in time need one each.
 *
 * fp32 statistics and sums; bf16 weights are rounded once before the product
 * with V and the result once; scores (scale * Q K^T) up to 2^30 in size, rows
 * with larger ones may be lost.  One launch, or two; deterministic.
 * B * Hkv * ceil(Hq / Hkv / 16) * (ceil(max_pages * page_size / 16) + 2) and
 * B * Hq below 2^31 - 65536.  Where the tables are wide, the lengths are looked
 * through by all workgroups: 16,384 requests of 16 tokens on one head take some
 * 0.5 ms, 2^20 of them 45 ms.
 */
size_t attention_paged_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv,
                                       int32_t D);
int32_t attention_paged(const void *Q, const void *k_pages,
                        const void *v_pages, const int32_t *page_table,
                        const int32_t *seq_len, void *O, int32_t B,
                        int32_t Hq, int32_t Hkv, int32_t D, int32_t n_pages,
                        int32_t page_size, int32_t max_pages,
                        int64_t page_stride, int32_t dtype, float scale,
                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention to another sequence's states (a decoder's to its encoder's):
 * O = softmax(scale * Q K^T) V with Sq query rows and Sk keys, any lengths,
 * nothing causal.
 *
 *   Q, O       DEVICE [B][Hq][Sq][D]; K, V DEVICE [B][Hkv][Sk][D]; all of
 *              dtype (AC_BF16: D 64 or 128; AC_F32: D <= 256).
 *   row_sel    NULL or DEVICE [B] int32: items with row_sel[b] >= 0 are
 *              skipped and their rows of O not written.
 *   key_len    NULL or DEVICE [B] int32: states of item b that are real,
 *              clamped to [0, Sk]; the others may hold anything.  An item of
 *              length 0 gets zeros.
 *   scale      0 selects 1/sqrt(D).
 *   workspace  DEVICE, attention_cross_workspace_bytes(...) bytes, as for
 *              attention_paged; may be NULL where that is 0 (calls of many
 *              rows, and sizes that attention_cross refuses).
 *
 * Arithmetic as in attention_paged.  bf16, D 128, 640 keys and more: 128 rows
 * among which a row's scores exceed the largest of its first 32 keys by some 41
 * or more (natural logarithm), or that meet an infinity or a NaN, take about
 * twice the time.  Hq / Hkv * Sq <= 2^24, B * Hkv <= 2^28,
 * Sk <= 2^30; AC_F32: B * Hkv * ceil(Hq / Hkv * Sq / 16) * (ceil(Sk / 16) + 2)
 * and B * Hq * Sq below 2^31 - 65536.
 */
size_t attention_cross_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv,
                                       int32_t Sq, int32_t Sk, int32_t D,
                                       int32_t dtype);
int32_t attention_cross(const void *Q, const void *K, const void *V, void *O,
                        const int32_t *row_sel, const int32_t *key_len,
                        int32_t B, int32_t Hq, int32_t Hkv, int32_t Sq,
                        int32_t Sk, int32_t D, int32_t dtype, float scale,
                        void *workspace, size_t workspace_bytes, void *stream);

/*
 * From a projection's product to Q, K and V: its rows are split into heads,
 * Q and K heads normalised and rotated by their positions, and each head goes
 * where the calls above want it, in one pass.
 *
 *   y = x / sqrt(mean(x^2) + eps) * weight     (where a weight is given)
 *   (a, b) -> amplitude * (a cos t - b sin t, b cos t + a sin t)
 *                      t = pos * freq[i], pair i of the first rot columns
 *
 *   X          DEVICE, B * S rows of dtype (AC_BF16: D 64 or 128; AC_F32:
 *              D <= 256): Hq heads of Q, Hkv of K, Hkv of V, D elements each.
 *              Rows lie row_stride elements apart (at least their size), items
 *              batch_stride (any, with B 1 not looked at); where D elements are
 *              a whole number of 16-byte pieces, both must be, too.
 *   q_weight, k_weight  NULL (no normalisation) or DEVICE [D] float.
 *   pos        DEVICE [B][S] int32.  Negative: the row is padding, and nothing
 *              of it is written anywhere.
 *   freq       DEVICE [rot / 2] double, radians a position, e.g. from
 *              attncache_rotary_frequencies.  rot even, 0 to D; columns from
 *              rot on are not rotated.  Angles are formed modulo one turn with
 *              64 bits and hold at any position; |freq| below 2^40.
 *   interleaved  0: pairs are columns (i, i + rot / 2), otherwise (2i, 2i + 1).
 *   Q          DEVICE [B][Hq][S][D] out.
 *   K, V       DEVICE [B][Hkv][S][D] out, or both NULL with slot.
 *   slot       NULL, or DEVICE [B][S] int32: K and V rows also go to these
 *              slots of k_pages and v_pages, as in attncache_page_append.
 *
 * binary32 inside, one rounding at the end.  eps >= 0.  The outputs may not
 * overlap X.  Hq + 2 Hkv <= 65535, B * S below 2^31 - 4096.
 */
int32_t attncache_rotate(const void *X, const float *q_weight,
                         const float *k_weight, const int32_t *pos,
                         const double *freq, const int32_t *slot, void *Q,
                         void *K, void *V, void *k_pages, void *v_pages,
                         int32_t B, int32_t S, int32_t Hq, int32_t Hkv,
                         int32_t D, int32_t rot, int64_t batch_stride,
                         int64_t row_stride, int32_t n_pages,
                         int32_t page_size, int64_t page_stride,
                         int32_t dtype, int32_t interleaved, float eps,
                         float amplitude, void *stream);

/*
 * freq[i] = base^(-2 i / rot), i < rot / 2, scaled for contexts `factor` times
 * as long as the model was trained on.  freq is HOST memory; nothing runs on
 * a GPU.  rot even, at least 2.
 *
 *   AC_ROTARY_PLAIN   not scaled (factor and what follows are not looked at)
 *   AC_ROTARY_LINEAR  freq / factor
 *   AC_ROTARY_BASE    base * factor^(rot / (rot - 2)) in the place of base: the
 *                     fastest pair stays, the slowest is stretched by factor
 *                     (rot at least 4)
 *   AC_ROTARY_RAMP    pairs with at most `low` turns within original_len are
 *                     stretched by factor, with at least `high` not at all,
 *                     between them freq is a weighted mean of both
 */
#define AC_ROTARY_PLAIN 0
#define AC_ROTARY_LINEAR 1
#define AC_ROTARY_BASE 2
#define AC_ROTARY_RAMP 3
int32_t attncache_rotary_frequencies(double *freq, int32_t rot, double base,
                                     int32_t scaling, double factor,
                                     double original_len, double low,
                                     double high);

/*
 * Rows of a paged cache become other rows: row b holds afterwards what row
 * from[b] held before.  Beams change places, several answers begin at one
 * prompt, requests end, and pages that a window has left behind go back.
 *
 *   from       DEVICE [B] int32.  b itself: the row goes on.  Outside [0, B),
 *              such as -1: the row ends and holds nothing.
 *   seq_len, free_state, free_pages  DEVICE, as in attncache_page_plan.
 *   page_table DEVICE [B][max_pages] int32: entries below
 *              ceil(seq_len / page_size) are read; those outside
 *              [0, n_pages) name no page and are taken over as -1 or as they
 *              are.
 *   page_table_out  DEVICE [B][max_pages] int32: the new rows' entries; others
 *              keep what they hold.
 *   seq_len_out  DEVICE [B] int32: seq_len[from[b]], 0 for a row that ends, -1
 *              for one that got no page (below), which holds nothing either.
 *   free_state_out  DEVICE [2] int32.
 *   k_pages, v_pages  DEVICE, with H heads (all layers: they fold into heads).
 *   sinks, window  window 0: nothing.  Otherwise pages of which every token
 *              j has j >= sinks and j < length - window go back, and their
 *              entries become -1: what attention_paged_window with this window
 *              sees of the row and of its later tokens stays.
 *
 * Full pages are shared among the rows that come from one.  A page that is
 * not full is kept by one (the row itself if it goes on, otherwise the first
 * that comes from it); each other takes a page from the ring, in order of
 * row, and its tokens are copied.  Rows for which the ring has none left get
 * nothing.  Pages that some row held and none holds afterwards go behind the
 * ring's last one, in order of their number, for the next call.
 *
 * Where the ring may run out, a call before, with from[b] = b for each row that
 * some row will come from and -1 for the others, gives back what nobody goes on
 * with; it takes no page.  Or give the call outputs of its own: it then leaves
 * the tables, lengths and states that it reads, the ring's entries in use and
 * the pages that rows hold as they were, so that a caller who finds a -1 can go
 * on from them in another way.
 *
 * All rows of the cache belong into one call: a page that a row outside it
 * holds would be given back.  attncache_page_plan goes on from the result (a
 * page it writes to is one row's), but does not know about sharing: rows that
 * share pages, or have lost some to a window, end here.
 * The outputs may be the inputs of the same meaning, or not overlap them.
 * workspace: DEVICE, attncache_page_fork_workspace_bytes(...) bytes, 16-byte
 * aligned; scratch, and written by a call before it is read.  Two launches up
 * to 1,024 rows, 8,192 entries of page_table and 65,536 pages, otherwise three.
 * Results do not depend on the order of threads.  B <= 2^22, B * max_pages below
 * 2^31 - 4096, page_size * D <= 2^30, otherwise as in attncache_page_plan.
 */
size_t attncache_page_fork_workspace_bytes(int32_t B, int32_t max_pages,
                                           int32_t n_pages);
int32_t attncache_page_fork(const int32_t *from, const int32_t *seq_len,
                            const int32_t *free_state, int32_t *free_pages,
                            const int32_t *page_table,
                            int32_t *page_table_out, int32_t *seq_len_out,
                            int32_t *free_state_out, void *k_pages,
                            void *v_pages, int32_t B, int32_t H, int32_t D,
                            int32_t max_pages, int32_t n_pages,
                            int32_t page_size, int64_t page_stride,
                            int32_t sinks, int32_t window, int32_t dtype,
                            void *workspace, size_t workspace_bytes,
                            void *stream);

/*
 * attention_paged for a batch in which requests share long prefixes (several
 * answers to one prompt, one instruction before many questions): K and V of a
 * prefix are read once for all its requests.  The result is that of
 * attention_paged.
 *
 *   share_first  DEVICE [G + 1] int32: group q is requests share_first[q] ...
 *              share_first[q + 1] - 1, which lie side by side in the batch; in
 *              ascending order (a smaller number counts as the largest before
 *              it), clamped to [0, B].  Other requests share nothing.
 *   share_len  DEVICE [G] int32: tokens that the group's requests have in
 *              common, clamped to [0, max_pages * page_size].  Any number: a
 *              prefix may end inside a page.  Requests with fewer tokens
 *              attend to theirs by themselves, as does a group of one.
 *   page_table, seq_len  as in attention_paged: a request's row names the
 *              pages of its prefix, too.  They are read through the first
 *              request of the group that has the whole prefix; the other
 *              rows' pages of the prefix must hold the same (be the same
 *              pages, or copies, as attncache_page_fork leaves them).
 *   workspace  DEVICE, attention_paged_shared_workspace_bytes(...) bytes,
 *              16-byte aligned; scratch, and written by a call before it is
 *              read.  Calls that may overlap in time need one each.
 *
 * G >= 0, and 0 groups need no share_len.  B and G at most 2^20, B * Hq at most
 * 2^25, Hkv * (B * ceil(g / 16) + B * g / 16 + G) * (ceil(max_pages * page_size /
 * 16) + 2) below 2^31 - 65536, with g = Hq / Hkv.  Two launches up to 256
 * requests and 255 groups, otherwise three, the first of which is one workgroup
 * that looks through the requests, 1,024 a step.  Without groups, where max_pages
 * * page_size is at most 128, and where K and V of B times as many tokens are at
 * most 64 MiB, each request is looked at by itself, as attention_paged does, and
 * its own row of the table is followed: by the launches of attention_paged, or,
 * where thousands of requests and heads have little each, by one launch that
 * gives each of them to a wave.
 * Deterministic.
 */
size_t attention_paged_shared_workspace_bytes(int32_t B, int32_t Hq,
                                              int32_t Hkv, int32_t D,
                                              int32_t G);
int32_t attention_paged_shared(const void *Q, const void *k_pages,
                               const void *v_pages, const int32_t *page_table,
                               const int32_t *seq_len,
                               const int32_t *share_first,
                               const int32_t *share_len, void *O, int32_t B,
                               int32_t Hq, int32_t Hkv, int32_t D, int32_t G,
                               int32_t n_pages, int32_t page_size,
                               int32_t max_pages, int64_t page_stride,
                               int32_t dtype, float scale, void *workspace,
                               size_t workspace_bytes, void *stream);

/*
 * Attention within a sliding window, with a few first tokens that stay
 * visible: row t of a prompt sees keys j <= t with j > t - window or j < sinks.
 *
 *   Q, O       DEVICE [B][Hq][S][D]; K, V DEVICE [B][Hkv][S][D]; all of dtype
 *              (AC_BF16: D 64 or 128; AC_F32: D <= 256), any S.
 *   row_sel    NULL or DEVICE [B] int32: items with row_sel[b] >= 0 are
 *              skipped and their rows of O not written (attncache_search's
 *              hits: only misses are computed.  The maps that hits reuse have
 *              to be of the same window; attncache_insert forms maps of causal
 *              or full attention, which serve a layer with a window only where
 *              this covers all S tokens).
 *   key_len    NULL or DEVICE [B] int32: tokens of item b that are real,
 *              clamped to [0, S]; the other keys are hidden and may hold
 *              anything.  Rows of padding are computed by the same rule; those
 *              that see no key get zeros.
 *   window     at least 1 (the token itself); S or more: causal attention.
 *   sinks      0 or more.
 *   scale      0 selects 1/sqrt(D).
 *
 * Arithmetic as in attention_paged, at scores of any size.  Keys that are hidden
 * from a row do not touch it, whatever K and V hold there: workgroups whose
 * blocks of keys hold an infinity or a NaN of V walk their keys four times,
 * which takes up to ten times as long; in Q or K they cost nothing.
 * Hq / Hkv * S <= 2^24, also with S rounded up to a multiple of 16;
 * B * Hkv <= 2^28, B * Hq below 2^31.
 */
int32_t attention_window(const void *Q, const void *K, const void *V, void *O,
                         const int32_t *row_sel, const int32_t *key_len,
                         int32_t B, int32_t Hq, int32_t Hkv, int32_t S,
                         int32_t D, int32_t dtype, int32_t window,
                         int32_t sinks, float scale, void *stream);

/*
 * The same for one new token of each request over its pages: of seq_len[b] = n
 * tokens those with j >= n - window or j < sinks are seen.  Everything else
 * is as in attention_paged, the workspace too
 * (attention_paged_workspace_bytes).  Pages of which no token is seen, and
 * their entries of page_table, are not looked at: attncache_page_fork gives
 * them back.  The limit counts window + sinks keys in the place of max_pages *
 * page_size.
 */
int32_t attention_paged_window(const void *Q, const void *k_pages,
                               const void *v_pages, const int32_t *page_table,
                               const int32_t *seq_len, void *O, int32_t B,
                               int32_t Hq, int32_t Hkv, int32_t D,
                               int32_t n_pages, int32_t page_size,
                               int32_t max_pages, int64_t page_stride,
                               int32_t dtype, int32_t window, int32_t sinks,
                               float scale, void *workspace,
                               size_t workspace_bytes, void *stream);

/*
 * Switches the per-call memory-space checks of pointers on (non-zero, the
 * default) or off for the whole process; returns the previous setting.
 * attncache_build_db always checks.
 */
int32_t attncache_set_pointer_checks(int32_t on);

/* Short constant description of a status code. */
const char *attncache_status_string(int32_t status);

/* hipError_t (as int) of the last failed HIP call on this thread, 0 if none. */
int32_t attncache_last_hip_error(void);

/* Library version, major * 1000 + minor. */
int32_t attncache_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ATTNCACHE_H */
