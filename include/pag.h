/*
 * pag.h -- C ABI of the MI355X (gfx950) PAG library.
 *
 * PAG (Projection-Augmented Graph) answers approximate K-nearest-neighbour
 * queries over a dataset D of n vectors in R^d (problem statement, Sec. 1) with
 * a best-first search over a proximity graph in which a projection-based test
 * (PRT, Eq. 3, with the Test-Feedback-Buffer threshold of Eq. 4) decides which
 * neighbours get an exact distance (Alg. 2).  The index is built by inserting
 * the vectors with that same search followed by RobustPrune (Alg. 1, Step 1;
 * Eq. 1).
 *
 * Conventions for every entry point
 *   - "dev" pointers are device (HBM) pointers of the GPU that was current when
 *     the index was created; "host" pointers are ordinary host memory.  All
 *     buffers are row-major, contiguous and owned by the caller: the library
 *     never frees them and copies whatever it keeps, so they may be released
 *     as soon as the call returns.
 *   - Work is enqueued on pag_params.stream (a hipStream_t, NULL = the null
 *     stream) and every call returns after that stream has been synchronised.
 *   - Return value: PAG_OK (0) or a negative pag_status; pag_last_error()
 *     returns a thread-local, human readable description of the last failure.
 *     No exception crosses this boundary.
 *   - Node ids are the row numbers of the vectors in insertion order.
 *   - A handle owns workspaces and counters: calls on one index must not overlap in time
 *     (different indexes are independent).  The exception is a pag_searcher, which has
 *     workspaces, counters and a stream of its own: pag_searcher_search may run while
 *     pag_insert, pag_search or other searchers work on the same index.
 */
#ifndef PAG_H
#define PAG_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pag_index pag_index; /* opaque; created by pag_build / pag_import, destroyed by pag_free */

typedef enum { PAG_L2 = 0, PAG_IP = 1, PAG_COS = 2 } pag_metric;

typedef enum {
    PAG_OK = 0,
    PAG_EINVAL = -1,       /* null / inconsistent argument, d % num_subspaces != 0, K == 0, K > n ... */
    PAG_ECAPACITY = -2,    /* pag_insert beyond pag_params.capacity */
    PAG_ENOMEM = -3,       /* host or device allocation failed */
    PAG_EHIP = -4,         /* a HIP call failed; text in pag_last_error() */
    PAG_EUNSUPPORTED = -5  /* a size outside what the kernels are built for (see pag_params) */
} pag_status;

/*
 * Index parameters (Alg. 1 inputs; Appendix D).  Names in brackets are the
 * paper's.  Limits of this build: d % 4 == 0, d <= 3072, num_subspaces <= 64,
 * d % num_subspaces == 0, max_degree <= 64, working-set size b <= 1024.
 */
typedef struct {
    uint32_t struct_size;     /* sizeof(pag_params), for ABI checking */
    int32_t  metric;          /* pag_metric.  PAG_IP expects unit-norm vectors (it ranks like PAG_COS
                                 without normalising); PAG_COS normalises base vectors and queries. */
    uint32_t max_degree;      /* [2M] maximum out-degree */
    uint32_t num_subspaces;   /* [L] number of subspaces of the rotated space; 16 projection vectors each */
    uint32_t ef_construction; /* [efC] nodes visited per insertion; W has min(efC, 100) nodes while indexing */
    uint32_t search_b;        /* working-set size b = |W| when searching; 0 = max(10, K) (Alg. 2) */
    uint32_t insert_subbatch; /* vectors inserted concurrently per step of the batch-synchronous build; 0 = auto;
                                 at most 2^20 */
    uint32_t flags;           /* PAG_FLAG_* */
    uint64_t capacity;        /* maximum number of vectors including later pag_insert calls; 0 = n */
    uint64_t seed;            /* seed of the random transform Q and of the codebooks */
    void*    stream;          /* hipStream_t; NULL = null stream */
} pag_params;

#define PAG_FLAG_NO_PRT 1u    /* ablation: skip the projection test, every unseen neighbour gets an exact distance */
#define PAG_FLAG_FP16_VECTORS 4u /* keep the rotated base vectors as 16-bit floats (the paper's payload, Sec. 4.2): halves the
                                   bytes per exact distance; the index then *is* the rounded data, and all arithmetic on it
                                   stays fp32/fp64.  Needs d % 8 == 0.  Build / import time only. */
#define PAG_FLAG_NO_PES 2u    /* ablation: index without the PES candidate buffers H(v) (Eq. 5; Alg. 1's last loop) */
#define PAG_FLAG_KEEP_ORDER 8u /* build / insert link the vectors in the order given (row 0 first) instead of a
                                  seeded shuffle: for input that is already in random order.  With
                                  insert_subbatch = 1 this is Alg. 1 as printed, one node after another, the
                                  PES buffer of a node verified right after its insertion. */
#define PAG_FLAG_EXACT_TEST_COUNT 16u /* diagnostic, search time: long searches resolve the seen set for every
                                  neighbour before the projection test instead of only for those that pass it,
                                  so that pag_counters.tests counts exactly the unseen neighbours (Sec. 4.2's
                                  gamma = passes / tests).  Results are unchanged; the search is a few % slower. */
#define PAG_FLAG_PERMUTATION_TRANSFORM 32u /* build time: Q is a random signed permutation (a coordinate shuffle with random
                                  signs) instead of a Haar-distributed rotation.  Still orthogonal, and its products are exact,
                                  so the stored vectors are the input's values bit for bit; it does not mix coordinates, so
                                  it suits data that is already isotropic (and comparisons that must not depend on rounding). */
#define PAG_FLAG_KEEP_QUERY_ORDER 64u /* search time: the queries of a call are taken as numbered.  By default a call with more
                                  queries than the GPU keeps waves resident takes them in the order of their projections onto
                                  the batch's direction of largest spread, so that searches running side by side visit the
                                  same part of the graph and share rows in the caches.  Results never depend on it. */

/*
 * Flat host view of an index (Alg. 1 output: node set, edge set E, inference
 * structure I, transform Q, codebooks).  Used by pag_export (the library fills
 * caller-allocated arrays) and pag_import (the library copies from them).
 */
typedef struct {
    uint32_t struct_size;
    int32_t  metric;
    uint64_t n;
    uint32_t d;
    uint32_t num_subspaces;   /* P */
    uint32_t max_degree;      /* deg */
    uint32_t n_entry;
    float*    vectors;   /* host [n*d]        base vectors after normalisation (COS) and rotation by Q (and rounding
                                              to 16-bit floats with PAG_FLAG_FP16_VECTORS), as fp32 */
    uint32_t* adj;       /* host [n*deg]      out-neighbour ids; 0xFFFFFFFF = free slot */
    float*    a;         /* host [n*deg]      a_i = ||w_i-u|| / cos(beta_i)            (Sec. 3.1) */
    float*    c;         /* host [n*deg]      c_i = ||w_i-u||^2 + 2 a_i sum_l <u_l, r*_il>  (stored offsets, Appendix C) */
    float*    e2;        /* host [n*deg]      ||w_i-u||^2 */
    uint8_t*  codes;     /* host [n*deg*P]    index (0..15) of the selected reference vector per subspace */
    float*    rotation;  /* host [d*d]        Q, row-major; rotated = Q x */
    float*    codebooks; /* host [P*16*(d/P)] projection vectors r_jl, norm 1/sqrt(P) */
    uint32_t* entry;     /* host [n_entry]    entry node ids; a search starts from the first b of them */
} pag_arrays;

/* Sums over all searches since creation or the last pag_reset_counters (Sec. 4.2's quantities); the searches
 * that pag_build and pag_insert run for their own vectors count as well. */
typedef struct {
    uint32_t struct_size;
    uint32_t adj_record_bytes;   /* size of one node's adjacency record in HBM */
    uint64_t queries;
    uint64_t hops;               /* expanded nodes (n' of Sec. 4.2) */
    uint64_t tests;              /* neighbours the projection test was evaluated for: the unseen ones; in long
                                    searches of large batches also already-seen ones that only the second
                                    level of the seen set would have recognised (it is consulted for passing
                                    neighbours only), unless PAG_FLAG_EXACT_TEST_COUNT is set.  A searcher beside an
                                    insertion can meet a record that lists a neighbour twice, and small batches then
                                    count it twice */
    uint64_t passes;             /* of those, how many passed (gamma = passes / tests) */
    uint64_t exact;              /* exact distances computed, entry nodes included */
    uint64_t rounds;             /* TFB rounds */
    uint64_t rf_overflow;        /* entries overwritten in the ring R_F */
    uint64_t rt_overflow;        /* entries overwritten in the ring R_T */
    uint64_t seen_spills;        /* seen-set insertions that went to the HBM bitmap (in long searches all of them, unless
                                    the batch is so small that the on-chip memory holds its seen sets) */
    double   last_search_kernel_ms; /* HIP-event time of the search kernel of the last pag_search */
    double   last_prepare_ms;       /* HIP-event time of rotation + projection tables of the last pag_search */
    double   last_build_ms;         /* wall time of the last pag_build / pag_insert */
    uint64_t phase_cycles[6];       /* diagnostic: per-phase clock ticks of the search kernel, summed over waves;
                                       all zero unless the library was compiled with -DPAG_PHASE_TIMERS */
    uint64_t relinked_batches;      /* insertion batches, since the index was created, that were found to crowd a
                                       region of their own and were linked a second time (see pag_insert) */
    double   last_build_phase_ms[4]; /* HIP-event times of the last pag_build / pag_insert, summed over its batches:
                                       [0] the search kernel in indexing mode, [1] candidate sort + RobustPrune,
                                       [2] pair sort + reverse edges and PES verification, [3] inference information */
} pag_counters;

/*
 * pag_build (Alg. 1, Step 1, batch-synchronous): creates an index over the n
 * vectors D (dev, float32 [n*d]).  D is normalised (PAG_COS), rotated by Q and
 * copied into the index.  *out receives the handle.  Node i is row i of D.  The
 * nodes are linked in batches drawn from a shuffle of the ids that
 * pag_params.seed fixes, so the order in which the rows arrive (sorted by
 * cluster, source or time) does not shape the graph; the first 1024 nodes of
 * that shuffle are the entry nodes.
 */
int pag_build(const float* D, uint64_t n, uint32_t d, const pag_params* params, pag_index** out);

/*
 * pag_search (Alg. 2): K approximate nearest neighbours of each of the nq
 * queries Q (dev, float32 [nq*d]).  efS is the paper's efS: the number of TFB
 * rounds is ceil(efS / b).  Outputs (dev): ids int64 [nq*K], dists float32
 * [nq*K], per query ascending by (dist, id).  dists holds squared Euclidean
 * distances for PAG_L2 and 1 - <q,x> (= ||q-x||^2 / 2 on unit vectors) for
 * PAG_IP / PAG_COS.  Slots beyond the number of nodes reached hold id -1,
 * dist +inf.
 */
int pag_search(const pag_index* ix, const float* Q, uint64_t nq, uint32_t K, uint32_t efS,
               int64_t* ids, float* dists);

/*
 * pag_search_static: pag_search for callers that cannot allocate device memory -- code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same results.  It calls
 * no hipMalloc, hipFree or other allocating routine: its workspaces (rotated queries, projection tables,
 * normalised copies, per-wave seen-set bitmaps) live in one 48 MB device array that is part of the library
 * and that every GPU the library runs on holds until the process ends (its address on a GPU is looked up
 * when an index is created there, so the call itself loads nothing either).  Limits (PAG_EUNSUPPORTED beyond
 * them, nothing is launched): nq * (d + 16 * S [+ d for PAG_COS]) <= 4,194,304 floats, where S is
 * num_subspaces rounded up to 16, 32 or 64; index capacity <= 4,194,304 vectors; working set b <= 128
 * (K <= 128).  With fewer bitmaps than the GPU could keep waves busy the call is slower than pag_search,
 * never different; it also takes the queries as numbered (see PAG_FLAG_KEEP_QUERY_ORDER).  All calls on one GPU share the array: calls that overlap in time on one GPU (from
 * any thread, on any index) race and must be serialised by the caller.  The call synchronises the
 * index's stream before it returns, like pag_search.
 */
int pag_search_static(const pag_index* ix, const float* Q, uint64_t nq, uint32_t K, uint32_t efS,
                      int64_t* ids, float* dists);

/*
 * pag_insert (online insertion, Sec. 4.1): appends the m vectors X (dev,
 * float32 [m*d]); they receive ids n .. n+m-1 and are linked in shuffled
 * batches like the vectors of pag_build.  The vectors of one batch do not see
 * each other while they are linked; a batch found to crowd a region of its
 * own (vectors inserted where the index has none yet) is therefore linked a
 * second time once its vectors are part of the graph.
 * PAG_ECAPACITY if n + m exceeds pag_params.capacity.
 * If the call fails half way (a HIP error, memory), the index keeps answering
 * searches over the n vectors it had, but some of their out-edges may already
 * point at the vectors that were being added: further pag_insert calls on it
 * are refused with PAG_EINVAL.
 */
int pag_insert(pag_index* ix, const float* X, uint64_t m);

/* Waits for the index's stream, releases everything the index owns.  NULL is accepted.  Free its searchers first. */
int pag_free(pag_index* ix);

/* Fills n, d, num_subspaces, max_degree, n_entry, metric of `out` (pointers untouched). */
int pag_describe(const pag_index* ix, pag_arrays* out);
/* Copies the index into the caller-allocated host arrays of `out` (sizes as reported by pag_describe). */
int pag_export(const pag_index* ix, pag_arrays* out);
/* Creates an index from host arrays (all of them required); params gives capacity, efC, search_b, seed, stream.
 * The graph is validated on the host: PAG_EINVAL for a neighbour or entry id >= n, a code above 15, a neighbour
 * listed twice by one node, or an entry id listed twice. */
int pag_import(const pag_arrays* in, const pag_params* params, pag_index** out);

/* Statistics summed over all searches since the last reset (set out->struct_size first), and the reset. */
int pag_get_counters(const pag_index* ix, pag_counters* out);
int pag_reset_counters(pag_index* ix);
/* Changes search-time settings of an existing index: working-set size (0 = max(10,K)) and the search-time
 * PAG_FLAG_* bits (PAG_FLAG_NO_PRT, PAG_FLAG_EXACT_TEST_COUNT, PAG_FLAG_KEEP_QUERY_ORDER); the bits fixed at build time stay. */
int pag_set_search_options(pag_index* ix, uint32_t search_b, uint32_t flags);
/* log2 of the slots of the per-query LDS seen-set table; 0 = choose from efS.  Small values exercise the HBM spill path. */
int pag_set_seen_capacity_log2(pag_index* ix, uint32_t log2_slots);

/*
 * Single steps of the search, exposed for kernel-level parity checks.
 *
 * pag_prepare_queries (Alg. 2, rotation step and projection-table step):
 *   q_rot (dev float32 [nq*d]) and tables (dev float32 [nq*P*16],
 *   tables[i][l][j] = <q_l, r_jl>) of the queries Q (dev).
 * pag_exact_distances (Alg. 2, exact-distance step):
 *   keys[i*m+j] = ||q_rot[i] - x[ids[i*m+j]]||^2 for already rotated queries;
 *   ids dev uint32 [nq*m] (each < n), keys dev float32 [nq*m].
 * pag_screen (Eq. 3 + Eq. 4 in estimate form): for query i expanding node
 *   u[i] at squared distance Du[i], est[i*deg+s] = Du + c_s - 2 a_s S_s for
 *   every neighbour slot s of u[i] (NaN for a free slot); a neighbour passes
 *   the test iff est < ||z_max - q||^2.  tables as produced above.
 * pag_edge_info (Sec. 3.1 / Appendix B): recomputes codes, a, c, e2 of every
 *   stored edge of nodes [node_begin, node_end) from the vectors; outputs are
 *   host arrays [(node_end-node_begin)*deg (*P)].
 * pag_insertion_candidates (Alg. 1, the search of one insertion; Eq. 5): what
 *   inserting each of the m vectors X (dev, float32 [m*d], raw like the input of
 *   pag_insert) into the index as it stands would start from, without changing
 *   the index: the list R_L (capacity efC, ascending by (dist, id)) and the PES
 *   buffer H(v) (capacity max_degree, ascending).  Outputs are host arrays:
 *   cand_ids / cand_keys [m*efC] with cand_count [m] valid entries per vector,
 *   pes_ids / pes_keys [m*max_degree] with pes_count [m]; keys are squared
 *   distances.  With PAG_FLAG_NO_PES the buffers come back empty.
 */
int pag_prepare_queries(const pag_index* ix, const float* Q, uint64_t nq, float* q_rot, float* tables);
int pag_exact_distances(const pag_index* ix, const float* q_rot, uint64_t nq, const uint32_t* ids,
                        uint32_t m, float* keys);
int pag_screen(const pag_index* ix, const float* tables, uint64_t nq, const uint32_t* u,
               const float* Du, float* est);
int pag_edge_info(const pag_index* ix, uint64_t node_begin, uint64_t node_end, uint8_t* codes,
                  float* a, float* c, float* e2);
int pag_insertion_candidates(const pag_index* ix, const float* X, uint64_t m, uint32_t* cand_ids,
                             float* cand_keys, uint32_t* cand_count, uint32_t* pes_ids, float* pes_keys,
                             uint32_t* pes_count);

/*
 * Diagnostic: how pag_search would lay out a call of nq queries now.  *waves: wavefronts that work on one query
 * (small batches get several, unless other calls of this process keep the GPU busy); *resident: queries that the GPU
 * works on at a time.  Nothing is launched.
 */
int pag_search_layout(const pag_index* ix, uint64_t nq, uint32_t K, uint32_t efS, uint32_t* waves, uint32_t* resident);

/*
 * Diagnostic for the roofline (no step of the method): reads `rows` whole rows of the index's vector
 * store, in order (scattered = 0) or in a scattered permutation (scattered = 1), four rows in flight
 * per wavefront, and reports the achieved rate in GB/s.  This is what the exact-distance step of
 * Alg. 2 could reach on this GPU if it did nothing but fetch its vectors.
 * scattered = 2 reproduces the traffic of whole hops of a long search instead: per seven random rows
 * one random adjacency record, eight random reads and seven random bit-sets in a per-wave seen-set
 * bitmap (the index's own workspace, cleared again afterwards); the rate counts rows and records only,
 * like the algorithmic bytes of the search do.
 */
int pag_measure_row_reads(const pag_index* ix, uint64_t rows, int scattered, double* gb_per_s);

/*
 * Searchers: searching while the index grows (the online-insertion setting of Sec. 5.2, D6).
 * A searcher is a view of an index with its own workspaces, counters and stream (a hipStream_t;
 * pass one that does not synchronise with the index's stream, else the calls just take turns).
 * pag_searcher_search is pag_search on that view: it sees the nodes whose insertion had completed when
 * the call began (pag_insert publishes its nodes after its last kernel has finished); nodes being inserted
 * are invisible.  While an insertion rewrites the out-edges of older nodes, a search may read an edge's
 * neighbour id and its inference information from different moments; that can change which neighbours
 * are tested in that hop, never a reported id/distance pair, which always comes from the stored vectors.
 * Results are therefore valid but, during an insertion, not reproducible bit for bit.
 * One searcher serves one call at a time; any number of searchers may share an index.  Free the
 * searchers before the index.  search_b, flags and the seen-set option are read from the index at each call.
 * For callers that insert and query at the same time from different host threads.
 */
typedef struct pag_searcher pag_searcher;
int pag_searcher_create(const pag_index* ix, void* stream, pag_searcher** out);
int pag_searcher_search(pag_searcher* s, const float* Q, uint64_t nq, uint32_t K, uint32_t efS,
                        int64_t* ids, float* dists);
int pag_searcher_get_counters(const pag_searcher* s, pag_counters* out);
int pag_searcher_free(pag_searcher* s);

/*
 * A memory that is searched: the keys and values of a language model's tokens in 8 or 4 bits, in pages, and attention over all of
 * them, over the tokens that a search returned (pag_search on an index over the keys; its ids, -1 where there is none, go
 * into pag_kv_attend_selected as they are), or over blocks of tokens that a cheap score selects.
 *
 * These calls belong into a decoding loop, many to a step, so they differ from the ones above in two points: they enqueue
 * their work on the stream that they are given and return without waiting for it, and they allocate nothing, so that a loop
 * can be captured into a HIP graph.  The stream belongs to the current GPU; its device pointers are that GPU's.  Arguments
 * that the host can see are checked before anything is launched; what only the GPU sees (lengths, page numbers, slots, ids)
 * is checked by the kernels: what is out of range counts as absent.
 *
 * A cache has a row of keys and a row of values side by side for every page, head and token, W = head_dim rounded up to a
 * multiple of 64 bytes each (zeros behind head_dim), and an exponent per block of 16 tokens, head and kind:
 *     data      uint8 [num_pages][kv_heads][page_tokens][2][W]
 *     exponents int8  [num_pages][kv_heads][page_tokens / 16][2]            number = code * 2^exponent, exponents of -126 to 126
 * Codes are signed integers (largest 127) or floats of 4 exponent and 3 mantissa bits without infinities (largest 448).
 * A power of two as scale means that a product with it never rounds and that a block which outgrows its exponent is rounded
 * again at most once per doubling.  slot = page * page_tokens + place in the page; a request's token p is in page table[p / page_tokens].
 * A cache of 4 bits a number (PAG_KV_FP4: a sign, 2 exponent and 1 mantissa bits: 0, 1/2, 1, 3/2, 2, 3, 4, 6) has rows of W / 2 bytes, number 2 i in the
 * low bits of byte i and number 2 i + 1 above it, and an exponent per 32 numbers of a row, those of 16 tokens side by side:
 *     data      uint8 [num_pages][kv_heads][page_tokens][2][W / 2]
 *     exponents int8  [num_pages][kv_heads][page_tokens / 16][2][W / 32][16]            exponents of -64 to 126
 */
typedef enum { PAG_KV_INT8 = 0, PAG_KV_FP8 = 1, PAG_KV_FP4 = 4 } pag_kv_format;
typedef enum { PAG_F32 = 0, PAG_F16 = 1, PAG_BF16 = 2 } pag_dtype;

typedef struct {
    uint32_t struct_size;
    uint32_t format;       /* pag_kv_format */
    uint32_t kv_heads;
    uint32_t head_dim;     /* a multiple of 8, at most 256 */
    uint32_t page_tokens;  /* a multiple of 16 */
    uint32_t reserved;     /* 0 */
    uint64_t num_pages;    /* num_pages * kv_heads * page_tokens < 2^32 */
    uint8_t* data;         /* dev, 16-byte aligned */
    int8_t*  exponents;    /* dev, 2-byte aligned (PAG_KV_FP4: 16-byte) */
} pag_kv_cache;

/* The block tables of `requests` requests and the pages that nobody holds (a stack: the last one is taken first).  All dev. */
typedef struct {
    uint32_t struct_size;
    uint32_t requests;
    uint32_t max_pages;    /* columns of table in use */
    uint32_t page_tokens;
    uint64_t table_stride; /* entries from row to row */
    uint64_t num_pages;    /* entries of free_pages: room for every page that may be given back */
    int32_t* table;        /* [requests * table_stride] */
    int32_t* lengths;      /* [requests] tokens held */
    int32_t* free_pages;   /* [num_pages] */
    int32_t* free_count;   /* [1] */
} pag_kv_tables;

/* One step of a batch: its new tokens, request after request.  Written by pag_kv_extend; the attention calls read it.  All dev. */
typedef struct {
    uint32_t struct_size;
    uint32_t requests;
    uint32_t max_pages;        /* as in pag_kv_tables */
    uint32_t max_new;          /* no request has more new tokens than this (0: not known); a hint: it decides how work is split, so the last bits of a result may differ with it */
    uint64_t table_stride;
    uint64_t tokens;           /* rows of the step's arrays, padding behind the last request included */
    const int32_t* table;
    int32_t* offsets;          /* [requests + 1] first new token of each request, ascending; rows before the first and behind the last are padding */
    int32_t* context;          /* [requests] tokens that it holds once the new ones are written; 0 if it was refused */
    int32_t* request;          /* [tokens] request of a token, -1 for padding (pag_kv_attend_selected reads it, pag_kv_attend does not) */
    int32_t* positions;        /* [tokens] position in the request, -1 for padding and for refused requests (likewise) */
    int64_t* slots;            /* [tokens] where its key and value go, -1 likewise (only pag_kv_extend uses the fields from here on) */
    int32_t* granted;          /* [requests] 1, or 0 if there were not enough pages, or not enough rows in the step */
    int32_t* lengths;          /* [requests] lengths after the step; may be pag_kv_tables.lengths itself */
    int32_t* free_count;       /* [1] likewise */
    int32_t* scratch;          /* [requests + 1] */
} pag_kv_step;

typedef struct {
    uint32_t struct_size;
    uint32_t dtype;            /* of q and out: PAG_F16 or PAG_BF16 */
    uint32_t heads;            /* query heads, a multiple of kv_heads: head h reads key/value head h * kv_heads / heads */
    uint32_t window;           /* a token reads the last `window` tokens, itself among them; 0: all (pag_kv_attend) or none (pag_kv_attend_selected) */
    float    scale;            /* scores are scale * <q, k> */
    float    softcap;          /* > 0: then softcap * tanh(score / softcap) */
    const float* slopes;       /* dev [heads] or null: then minus slopes[h] * (position of the query - position of the key) */
    const void* q;             /* dev [tokens][heads][head_dim], strides in elements; last dimension dense */
    int64_t  q_token_stride, q_head_stride;     /* multiples of 8; q 16-byte aligned */
    void*    out;              /* dev, like q */
    int64_t  out_token_stride, out_head_stride;
    float*   lse;              /* dev [tokens * heads]: log of the sum of exp(score); or null */
    void*    workspace;        /* dev, 16-byte aligned, pag_kv_workspace_bytes() bytes; calls that may overlap in time need one each */
    uint64_t workspace_bytes;
} pag_kv_attention;

/*
 * pag_kv_extend: request r gets add[r] (dev int32 [requests], negative counts as 0) new tokens.  Requests are served in order; one
 * that needs more pages than its row of the table or the stack has left is refused as a whole (granted 0, slots -1), and so
 * is every later one that needs a page once the stack could not serve one before it.  Refused as a whole is also a request whose new
 * tokens do not all have rows in the step (the sum of add up to it is above step->tokens), and with it every later one that gets tokens; it
 * takes no page and keeps its length.  offsets count the tokens of refused requests too.  Writes the new entries of the tables
 * and all arrays of `step`; the rest of `tables` changes only where step->lengths and step->free_count are its own arrays, so
 * a step can be looked at before it is taken over.
 * pag_kv_release: the requests with done[r] != 0 (dev int32 [requests]) give back their pages, first page first, in order of
 * their numbers, and hold nothing then.  Pages for which free_pages has no room (num_pages) are not put anywhere.
 */
int pag_kv_extend(const pag_kv_tables* tables, const int32_t* add, const pag_kv_step* step, void* stream);
int pag_kv_release(const pag_kv_tables* tables, const int32_t* done, void* stream);

/*
 * pag_kv_append: writes the keys and values of `tokens` tokens (dev, dtype PAG_F32 / F16 / BF16, [tokens][kv_heads][head_dim], strides in
 * elements, multiples of 16 bytes) into their slots (dev int64 [tokens]; -1 or out of range: left out).  The tokens of one block have to
 * follow each other in the call, in ascending order, with no other ones and none that are left out between them, as pag_kv_extend numbers them:
 * otherwise several waves write the block, and what it holds then is not defined.  A block that begins with the call (its
 * first token is among the new ones) is cleared first; its exponent is the smallest e >= -64 at which the largest code reaches the
 * largest finite magnitude.  Another block keeps its exponent unless the new tokens need a larger one; then what it held is
 * rounded again.  Rounding is to nearest even; infinities are held as the largest code, NaN as 0.
 * Of PAG_KV_FP4 the tokens of a call may come in any order, as long as no slot is there twice, and nothing but their own rows changes: each 32 numbers
 * get the smallest e >= -64 at which their largest finite magnitude is at most 7, which is rounded to the largest code by no more than half a step.
 * pag_kv_read: rows of the cache as numbers, [tokens][kv_heads][head_dim] with strides in elements (multiples of 16 bytes); k or v may be
 * null.  Slots -1 or out of range give zeros.  PAG_F32 and PAG_BF16 hold every number of the cache exactly, but for what a block near the end of
 * 32 bits rounds up to 2^128 and infinities held as the largest code there: that is read as the largest finite PAG_BF16, 255 * 2^120, where
 * attention's results end as well.
 * tokens * kv_heads of a call has to be below 2^27, and the tokens that pag_kv_append writes into a PAG_KV_FP4 cache below 2^25.
 */
int pag_kv_append(const pag_kv_cache* cache, uint32_t dtype, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                  const void* v, int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots, uint64_t tokens, void* stream);
int pag_kv_read(const pag_kv_cache* cache, const int64_t* slots, uint64_t tokens, uint32_t dtype, void* k, int64_t k_token_stride,
                int64_t k_head_stride, void* v, int64_t v_token_stride, int64_t v_head_stride, void* stream);

/*
 * pag_kv_append_rotated: pag_kv_append of keys that are turned by their positions, and of values as they are; and the same turn for queries.
 * Of the first `turned` numbers of a row at position p each pair (x, y), numbers i and i + turned / 2 or 2 i and 2 i + 1, becomes
 * (x cos a - y sin a, y cos a + x sin a) with the angle a = p * frequencies[i], a product in 64 bits.  Keys are turned in 64 bits where angles are below 2^31 in
 * magnitude, so that what is held is rounded once; queries in 32 bits, by cosines and sines of 64 bits that are rounded to 32, and rounded to their type.
 * A pair with an infinity or NaN becomes whatever these formulas give.  At most 2^24 tokens and 65536 heads a call, tokens * heads below 2^31.
 */
typedef enum { PAG_KV_HALVES = 0, PAG_KV_NEIGHBOURS = 1 } pag_kv_pairs;

typedef struct {
    uint32_t struct_size;
    uint32_t pairs;                /* pag_kv_pairs */
    uint32_t turned;               /* a multiple of 8, at most head_dim */
    uint32_t heads;                /* of q; 0: no q */
    const float* frequencies;      /* dev [turned / 2] */
    const int32_t* positions;      /* dev [tokens], of any sign; also those of tokens that are left out of the cache count, for q */
    const void* q;                 /* dev [tokens][heads][head_dim] of the call's dtype, strides in elements, multiples of 16 bytes */
    int64_t q_token_stride, q_head_stride;
    void* out;                     /* dev, like q: the turned rows; q itself, with q's strides, or apart from it; apart from k, v and each other */
    int64_t out_token_stride, out_head_stride;
} pag_kv_rotation;

int pag_kv_append_rotated(const pag_kv_cache* cache, uint32_t dtype, const void* k, int64_t k_token_stride, int64_t k_head_stride,
                          const void* v, int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots, uint64_t tokens,
                          const pag_kv_rotation* rotation, void* stream);

/*
 * pag_kv_workspace_bytes: the workspace of such a call of pag_kv_attend (selected = 0, id_heads and k are not looked at) or pag_kv_attend_selected;
 * often 0, then args->workspace may be null.  Of args it reads dtype, heads and window.
 * pag_kv_attend: every token of the step attends to the tokens of its request up to itself: out = sum softmax(score) v.
 * pag_kv_attend_selected: it attends to the last `window` tokens and to the tokens whose positions ids lists (dev int64
 * [tokens][id_heads][k], strides in elements, last dimension dense): id_heads is kv_heads (the heads of a group share a list), heads, or a
 * multiple of kv_heads that divides heads.  Ids below 0, in the window or beyond the token itself are passed over (the window's tokens count
 * once); an id listed twice counts twice.  tokens * heads and requests * kv_heads have to be below 2^23 there, below 2^31 in pag_kv_attend; k + window
 * below 2^30.
 * A token that finds nothing to attend to gets zeros and an lse of -inf; so does padding.
 * Sums, maxima and scores are held in 32 bits.  Rounded to 16-bit floats (11 bits) are the softmax weights for their product with the values,
 * together with the values' scale: what lies below 2^-31 of a row's largest weight * 2^exponent is lost from out, not from lse or from the sum
 * that out is divided by; and q, as multiples of 2^-32 of its row's largest magnitude at least.  Of PAG_KV_FP4 keys and values are multiples of 2^-24 of the largest
 * power of two among the parts of 16 tokens (of listed keys among their own): numbers whose part's power of two is within 2^-22 of that are held exactly.
 */
int pag_kv_workspace_bytes(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, int selected, uint32_t id_heads,
                           uint32_t k, uint64_t* bytes);
int pag_kv_attend(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, void* stream);
int pag_kv_attend_selected(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, const int64_t* ids,
                           int64_t ids_token_stride, int64_t ids_head_stride, uint32_t id_heads, uint32_t k, void* stream);

/*
 * Blocks of block_tokens tokens (a multiple of 16 that divides page_tokens; block b of a request holds its tokens b * block_tokens and on), of which
 * a token reads the k best.  A block's summary for a key/value head is, of each number of its keys as the cache holds them, the largest and the smallest, as integers with one
 * power of two: e is the smallest >= -64 at which 127 * 2^e reaches the largest magnitude, the largest is rounded up to a multiple of 2^e and the smallest down.
 * With a row of q as integers (nearest, at the smallest such power of two; infinities as 127, NaN as 0) a block's score for a query head is
 *     sum over the numbers of largest * max(q, 0) + smallest * min(q, 0),
 * which no key of the block exceeds, but for q's rounding; an integer below 2^23 times a power of two, so that which blocks are chosen is the same
 * on every run and by every path (scores beyond 32 bits count as equal).
 */
typedef struct {
    uint32_t struct_size;
    uint32_t block_tokens;
    int8_t* codes;             /* dev [num_pages][kv_heads][page_tokens / block_tokens][2: largest, smallest][W], 16-byte aligned */
    int8_t* exponents;         /* dev [num_pages][kv_heads][page_tokens / block_tokens] */
} pag_kv_blocks;

/*
 * pag_kv_blocks_update: after pag_kv_append of these slots (dev int64 [tokens]; -1 or out of range: left out): writes the summaries of the blocks that they lie in,
 * of all tokens from the block's first one to the last one in the call, which has to be the last one that the block holds.  The tokens of one of these blocks
 * have to follow each other in the call, in ascending order, with no other ones and none that are left out between them, as pag_kv_extend numbers them, also of a PAG_KV_FP4 cache:
 * otherwise several waves write its summary, and what it holds then is not defined.  tokens * kv_heads below 2^27.
 * pag_kv_blocks_select: for each token and list the k best of the blocks that begin before the token's window (args->window; 0: up to the token itself), of a list's heads by the
 * largest of their scores, of equal ones the first; their numbers in ascending order, -1 behind them (dev int32 [tokens][id_heads][k], strides in elements, last dimension dense).
 * Blocks in pages that are none are left out.  id_heads as in pag_kv_attend_selected.  Of args it reads dtype, heads, window, q and its strides,
 * and the workspace.  With `blocks` those that a row of the table has room for, max_pages * page_tokens / block_tokens: tokens * id_heads * blocks has to be at most 2^40 and
 * kv_heads * blocks / 256, rounded up for each head, below 2^24.  The workspace is 4 * id_heads * blocks bytes for each token of a launch, of as many tokens as 512 MB have room for (one
 * at least), or none where blocks and lists are few.
 * pag_kv_attend_blocks: pag_kv_attend_selected over the tokens of the listed blocks: those in the window or behind the token are passed over, a block listed twice counts
 * twice.  Both: tokens * heads and requests * kv_heads below 2^23, k * block_tokens + window below 2^30.
 * pag_kv_blocks_workspace_bytes: the workspaces of these two; either pointer may be null.
 */
int pag_kv_blocks_update(const pag_kv_cache* cache, const pag_kv_blocks* blocks, const int64_t* slots, uint64_t tokens, void* stream);
int pag_kv_blocks_select(const pag_kv_cache* cache, const pag_kv_blocks* blocks, const pag_kv_step* step, const pag_kv_attention* args, uint32_t id_heads,
                         uint32_t k, int32_t* ids, int64_t ids_token_stride, int64_t ids_head_stride, void* stream);
int pag_kv_attend_blocks(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, const int32_t* ids, int64_t ids_token_stride,
                         int64_t ids_head_stride, uint32_t id_heads, uint32_t k, uint32_t block_tokens, void* stream);
int pag_kv_blocks_workspace_bytes(const pag_kv_cache* cache, const pag_kv_step* step, const pag_kv_attention* args, uint32_t id_heads, uint32_t k,
                                  uint32_t block_tokens, uint64_t* select_bytes, uint64_t* attend_bytes);

const char* pag_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* PAG_H */
