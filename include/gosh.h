/* libgosh -- MI355X (gfx950) implementation of the GOSH graph-embedding training
 * path (Akyildiz, Aljundi, Kaya, "GOSH: Embedding Big Graphs on Small Hardware",
 * ICPP'20).  Plain C ABI: raw pointers and sizes only.
 *
 * Conventions
 *   - "device" pointers are HIP device memory of the current device; "host" pointers
 *     are ordinary host memory.  The library never frees or keeps caller arrays.
 *   - Graphs are CSR (Sec. 3.2.1 of the paper): adj holds the neighbour lists back to
 *     back, xadj holds n+1 offsets into it, xadj[n] == nnz.  Rows must be sorted
 *     ascending, without duplicates or self loops (gosh_csr_validate checks a host
 *     copy).  The training entry points do not verify this, but no array content can
 *     take their kernels outside the operands: a row whose offsets leave adj counts
 *     as empty, an entry that names no vertex (or, in the part-pair rotation, no vertex
 *     of the partner part) is no sample.  What such a graph trains is unspecified.
 *   - The embedding matrix M is n x d, row-major fp32, 16-byte aligned, d a multiple
 *     of 4 with 4 <= d <= 512.
 *   - Every function returns GOSH_OK (0) or a negative gosh_status; the message of the
 *     last failure on the calling thread is returned by gosh_last_error().  No
 *     exception crosses this boundary.
 *   - Device entry points are asynchronous: they enqueue work on the given HIP
 *     stream (a hipStream_t passed as void*, NULL = the default stream) and return.
 *     Faults inside a kernel surface at the caller's next synchronisation.
 */
#ifndef GOSH_H
#define GOSH_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  GOSH_OK = 0,
  GOSH_EINVAL = -1,  /* an argument violates a documented precondition */
  GOSH_ENOMEM = -2,  /* host or device allocation failed */
  GOSH_EHIP = -3,    /* a HIP runtime call failed */
  GOSH_EBUDGET = -4, /* device budget too small for the requested part layout */
  GOSH_EDIVERGED = -5 /* training finished, but the matrix it leaves holds non-finite values
                         (nothing in Alg. 1 bounds a row; a learning rate too large for the
                         graph's hubs makes rows grow until fp32 overflows) */
} gosh_status;

/* Borrowed view of a CSR graph.  All three arrays live on the same side (host or
 * device) as the entry point documents. */
typedef struct {
  int64_t n;          /* |V| : 1 <= n < 2^31 - 1 */
  int64_t nnz;        /* length of adj (= 2|E| for a symmetrised graph) */
  const void *xadj;   /* n+1 offsets; int32_t* if xadj_is64 == 0, else int64_t* */
  const int32_t *adj; /* neighbour ids */
  int32_t xadj_is64;
} gosh_csr;

#define GOSH_MAX_DIM 512
#define GOSH_MAX_NEG 15

/* gosh_train_epoch flags */
#define GOSH_FLAG_SEQUENTIAL 1u   /* debug: one wavefront walks the sources in ascending
                                     id, giving the sequential-order result */
#define GOSH_FLAG_PLAIN_STORES 2u /* concurrent mode: write every updated row back with
                                     plain stores (the paper's lock-free scheme as it
                                     stands: concurrent updates of one row can be lost) */
#define GOSH_FLAG_ATOMIC_ADDS 4u  /* concurrent mode: apply every update as atomic adds of
                                     the step (no update is ever lost; about 2x the cost) */

#define GOSH_FLAG_CONCURRENT_LAYOUT 64u /* debug, with GOSH_FLAG_SEQUENTIAL: the one lane group
                                     that walks the sources runs the concurrent kernel as it
                                     is shipped -- its lane-to-column layout, its device-scope
                                     row accesses, its hot-row rule with the atomic-add, plain-store
                                     and row-lock write paths -- instead of the plain 128-bit
                                     layout, so that exactly that code can be compared with a
                                     sequential reference.  No effect without
                                     GOSH_FLAG_SEQUENTIAL */

/* gosh_embed / gosh_embed_host only */
#define GOSH_FLAG_EDGE_EPOCHS 8u  /* an epoch is |E_i| sampled sources, the definition of the
                                     paper's experiments (Sec. 4.3), not the |V_i| of Alg. 3:
                                     level i runs e_i * ceil(|E_i| / |V_i|) passes of Alg. 3,
                                     |E_i| = nnz_i / 2, and the learning rate decays over all
                                     of them */

#define GOSH_FLAG_PAIR_LEVELS 32u /* a level that fits the device is trained in place with the
                                     pair scheme of Alg. 5 instead of Alg. 3 -- gosh_train_parts
                                     on the device matrix, B = 5 -- on the largest K of 16, 8,
                                     4, 2, 1 whose parts keep 2^22 vertices (pair_level_min_n of
                                     gosh_set_tuning) and whose whole
                                     rotations overshoot the level's epochs by at most an
                                     eighth; a level for which no K does keeps Alg. 3.  Not the
                                     paper's choice: see gosh_train_parts for what it buys */

/* gosh_train_parts / gosh_embed_host only */
#define GOSH_FLAG_BLOCKED_ORDER 16u /* visit the part pairs in the blocked order of
                                       gosh_pair_order_blocked (block = P_gpu - 2 parts, at
                                       least 1) instead of the paper's: the same pairs once
                                       per rotation, fewer parts over the host link */

const char *gosh_last_error(void);

/* ---- tuning record ------------------------------------------------------------------ */

/* Constants of this implementation that the paper does not have (Sec. 3.1 accepts lost
 * updates and only notes that too many of them hurt): how the training kernels are launched
 * and which rows count as "hot" (updated with atomic adds instead of plain stores, see
 * gosh_train_epoch).  One record per process, read at the start of every training call;
 * the library never reads the environment.  Meant for experiments and tests. */
typedef struct {
  int32_t plain_rows;        /* non-zero: plain 128-bit row accesses also in the concurrent
                                kernels (coherent inside one XCD only).  Default 0 */
  int64_t max_waves;         /* cap on the wavefronts that share the sources of one launch
                                (each then walks several sources, sampling ahead).
                                Default 2^18 */
  int64_t hot_inv_eps;       /* a vertex is hot if deg * C / nnz > 1 / hot_inv_eps, C = sources
                                in flight.  Default 64 */
  int64_t hot_all_inv_eps;   /* every row is hot if (k_neg + 1) * C / n > 1 / hot_all_inv_eps
                                (written under locks then where that pays, see
                                gosh_train_epoch); 0 switches that rule off.  Default 4 */
  int64_t hot_min_degree;    /* > 0: skip both rules; a vertex is hot iff its degree is at
                                least this.  Default 0 */
  int64_t pair_level_min_n;  /* GOSH_FLAG_PAIR_LEVELS: smallest part, in vertices.
                                Default 2^22 */
} gosh_tuning;

void gosh_tuning_defaults(gosh_tuning *t);
/* NULL restores the defaults.  GOSH_EINVAL for a value outside its range (max_waves,
 * hot_inv_eps, pair_level_min_n >= 1; the others >= 0); the record is unchanged then. */
int gosh_set_tuning(const gosh_tuning *t);
int gosh_get_tuning(gosh_tuning *t);

/* ---- schedule helpers (host, pure) ------------------------------------------------ */

/* Learning rate of epoch j (0-based) out of e_i at one level: lr0 * max(1 - j/e_i, 1e-4)
 * (Sec. 3, last paragraph before Alg. 2; Alg. 3 first line of the epoch loop).
 * Evaluated in double, rounded once.  Returns 0 if e_i <= 0. */
float gosh_lr(float lr0, int64_t j, int64_t e_i);

/* Epoch budget per level ("calculateEpochs", Sec. 3 paragraph on the smoothing ratio
 * p): a share p of e evenly over the D levels, the rest geometrically with each level
 * getting half of the next coarser one.  exact_i = p*e/D + (1-p)*e*2^i/(2^D-1); levels
 * i >= 1 get max(1, floor(exact_i)), level 0 the remainder, so sum(e_i) == e.
 * e_i: host array of D entries (written).  GOSH_EINVAL if D < 1, D > 62, p outside
 * [0,1] or e cannot give every level one epoch. */
int gosh_epoch_split(int64_t e, double p, int32_t D, int64_t *e_i);

/* The rule of GOSH_FLAG_PAIR_LEVELS (host, pure; not the paper's): parts for training a
 * resident level of n vertices for `epochs` epochs with the pair scheme in place -- the
 * largest K of 16, 8, 4, 2, 1 with K * min_n <= n whose whole rotations of B rounds overshoot
 * the epochs by at most an eighth (ceil(epochs / (B*K)) * B*K - epochs <= epochs / 8); 0 =
 * "train the level with Alg. 3". */
int32_t gosh_pair_level_parts(int64_t epochs, int64_t n, int64_t min_n, int32_t B);

/* ---- coarsening (host) -------------------------------------------------------------- */

/* Checks a host CSR graph against the conventions above (offsets start at 0, end at
 * nnz and never decrease; neighbour ids in range; rows strictly ascending; no self
 * loops).  GOSH_OK or GOSH_EINVAL with the first violation in gosh_last_error(). */
int gosh_csr_validate(const gosh_csr *g_host);

/* The set of coarsened graphs and the maps between them ("MultiEdgeCollapse", Alg. 4,
 * Sec. 3.2).  Opaque; owned by the library, released with gosh_hierarchy_free. */
typedef struct gosh_hierarchy gosh_hierarchy;

/* Alg. 4, sequential semantics.  Per level: vertices are visited by degree, largest
 * first (ties: smaller id first); an unmarked vertex v opens cluster number
 * (clusters so far) and takes every unmarked neighbour u, in neighbour-list order,
 * for which deg(v) <= delta or deg(u) <= delta, delta = nnz/n (tested as deg*n <= nnz).
 * G_{i+1} has the entry (a, b), a != b, iff some entry (x, y) of G_i has map[x] = a,
 * map[y] = b; rows ascending, parallel entries merged.
 * Levels are built while |V_i| > threshold (the paper's default is 100); building stops
 * after a level with |V_{i+1}| > min_shrink*|V_i| (that level is kept), at a level that
 * merged nothing (|V_{i+1}| == |V_i|: it would repeat G_i and is dropped), or when
 * max_levels graphs exist.  min_shrink in (0, 1]; 1.0 keeps only the no-progress guard.
 * n_threads <= 0 uses every available core (the result does not depend on the thread
 * count).
 * g0_host: host CSR, borrowed for the lifetime of the hierarchy (level 0 is a view of
 * it, not a copy).  *out receives the hierarchy; on failure it is NULL. */
int gosh_coarsen(const gosh_csr *g0_host, int64_t threshold, double min_shrink,
                 int32_t max_levels, int32_t n_threads, gosh_hierarchy **out);

/* MultiEdgeCollapse on the current HIP device: the same hierarchy, bit for bit (Alg. 4 has
 * one result), with the degree order a device radix sort, the marking sweep resolved in
 * parallel rounds, and "Coarsen" (the rebuild of the CSR of G_{i+1}, Sec. 3.2.1) a move of
 * the fine rows together by cluster and a merge of each coarse row.  g0 may be a host graph, which is uploaded
 * once, or a graph already in the current device's memory (detected from the pointers),
 * which is used where it is: in both cases it is borrowed for the lifetime of the
 * hierarchy, and its offsets and neighbour ids are range-checked on the device
 * (GOSH_EINVAL).  Every level then STAYS on
 * that device, where gosh_embed / gosh_embed_host read it without another upload, and the
 * host arrays behind gosh_hierarchy_graph / _map / _mult are downloaded on first request.
 * A graph whose marking does not resolve in a bounded number of rounds (long chains of
 * equal degrees) is marked on the host instead.  Device memory per entry of G_0 while running:
 * scratch of about 8 bytes (12 from 2^32 entries on), 16 more per entry of coarse rows that
 * are counted or 24 (32) of those that are radix-sorted -- both only rows of thousands of
 * entries, and only if there is room -- and up to 8 (12) for G_1, besides some 70 per vertex; afterwards
 * 8 (12) bytes per entry of all levels but the first, and the scratch blocks, which stay
 * with the hierarchy until gosh_hierarchy_trim_scratch, gosh_hierarchy_release_device or
 * gosh_hierarchy_free, because freeing them at once would slow the host link down for whatever
 * follows (the driver clears freed memory in the background).  For the same reason
 * gosh_hierarchy_free keeps device blocks for the next hierarchy, at most a 64th of the
 * device's memory per process, and up to 128 MB of pinned memory for the copies of pageable
 * arrays.  The blocks are given back when an allocation of this library needs them (other
 * allocators of the process cannot have them), and with the pinned memory by either of the other
 * two calls.
 * GOSH_ENOMEM / GOSH_EHIP if the device cannot.  Blocking; null stream. */
int gosh_coarsen_device(const gosh_csr *g0, int64_t threshold, double min_shrink,
                        int32_t max_levels, int32_t n_threads, gosh_hierarchy **out);

/* Returns to the driver the scratch blocks a device-built hierarchy still holds from its
 * construction and, whatever h is (NULL allowed), the blocks kept from freed hierarchies on the
 * current device, and the kept pinned memory.  The levels stay where they are. */
int gosh_hierarchy_trim_scratch(gosh_hierarchy *h);

/* Brings every array of a device-built hierarchy to the host and frees its device copies
 * (no-op for a host-built one).  Accessors and training keep working, from the host
 * copies.  Blocking. */
int gosh_hierarchy_release_device(gosh_hierarchy *h);

/* Accessors.  The arrays they hand out are host memory owned by the hierarchy (level 0:
 * by the caller) and stay valid until gosh_hierarchy_free.  For a device-built hierarchy
 * the first request for an array downloads it (blocking; the building device must be
 * current; GOSH_EHIP / GOSH_ENOMEM possible), so a hierarchy must not be used from two
 * threads at once. */

/* D, the number of graphs G_0..G_{D-1} (0 for NULL). */
int gosh_hierarchy_levels(const gosh_hierarchy *h);
/* |V_i| and the length of G_i's adj; either pointer may be NULL.  Never downloads. */
int gosh_hierarchy_shape(const gosh_hierarchy *h, int32_t i, int64_t *n, int64_t *nnz);
/* Borrowed host view of G_i (coarse levels have 64-bit offsets). */
int gosh_hierarchy_graph(const gosh_hierarchy *h, int32_t i, gosh_csr *view);
/* map_i: one entry per vertex of G_i, its super vertex in G_{i+1}; 0 <= i < D-1. */
int gosh_hierarchy_map(const gosh_hierarchy *h, int32_t i, const int32_t **map, int64_t *len);
/* Per entry of G_i's adj, how many entries of G_0 were merged into it (NULL and 0 for
 * level 0, where every entry counts once).  Not used by training; it makes edge-weight
 * conservation checkable: sum(mult_{i+1}) + (weight of entries inside clusters) =
 * sum(mult_i). */
int gosh_hierarchy_mult(const gosh_hierarchy *h, int32_t i, const int64_t **mult, int64_t *len);
/* Wall-clock milliseconds the three stages of Alg. 4 took when level i was coarsened
 * (0 <= i < D-1): ms3[0] degree sort, ms3[1] marking sweep, ms3[2] rebuilding the CSR of
 * G_{i+1} (Sec. 3.2.1 names these three stages). */
int gosh_hierarchy_times(const gosh_hierarchy *h, int32_t i, double *ms3);
void gosh_hierarchy_free(gosh_hierarchy *h);

/* ---- device entry points ---------------------------------------------------------- */
/* Every array these take must be memory a kernel can reach -- a device allocation, or
 * pinned host memory -- and must hold the documented number of elements inside the
 * allocation it starts in; both are checked before anything is launched (GOSH_EINVAL), so
 * that a wrong pointer or size becomes an error and not a memory fault on the device. */

/* "Randomly initialize M" (Alg. 2, second line).  Fills the device matrix M (n x d)
 * with values uniform in [-0.5/d, 0.5/d): entry (v, c) is word c%4 of
 * Philox4x32-10(counter = (v, c/4, 0xFFFFFFFF, level), key = seed), mapped as
 * ((w >> 8) * 2^-24 - 0.5) / d. */
int gosh_init_embedding(float *M_dev, int64_t n, int32_t d, uint64_t seed, uint32_t level,
                        void *hip_stream);

/* The sampler of Alg. 3 on its own (parity/debug): for every source src writes
 * out[src*(k_neg+1) + j], j = 0..k_neg.  j = 0 is the positive sample, a uniform member
 * of the neighbour list of src (Sec. 3.1; -1 if the list is empty); j >= 1 are the
 * negative samples, uniform over all n vertices.  Draw j of src is the low 64 bits of
 * Philox4x32-10(counter = (src, j, epoch, level), key = seed), reduced to an index
 * by multiply-high with the bound.  g_dev: CSR arrays on the device (the struct
 * itself on the host).  out_dev: device int32[n*(k_neg+1)]. */
int gosh_sample_epoch(const gosh_csr *g_dev, int32_t k_neg, uint64_t seed, uint32_t epoch,
                      uint32_t level, int32_t *out_dev, void *hip_stream);

/* One epoch of Alg. 3 ("TrainInGPU"): every vertex is the source of one positive and
 * k_neg negative updates of Alg. 1 ("UpdateEmbedding"), applied in that order:
 *   g = lr_epoch * (b - sigmoid(M[src] . M[v]));  M[src] += g*M[v];  M[v] += g*M[src]
 * (the second axpy uses the already updated source row; b = 1 for the positive, 0 for
 * negatives).  No positive update for a vertex without neighbours; a negative equal
 * to the source applies no update.  Sources run concurrently and no source waits for another's
 * turn (Sec. 3.1); the launch is the epoch barrier.  With GOSH_FLAG_SEQUENTIAL the sources are taken one
 * by one in ascending id, which is deterministic.  In concurrent mode the sources are
 * handed out in ascending id too (workgroups start in the order of their index and each walks
 * a block of consecutive sources), so an epoch sweeps the graph in the order of the sequential
 * one, a window of concurrently running sources wide.  The default write path is a
 * mix: rows likely to be held by several wavefronts at once (every row of a small
 * graph, high-degree vertices of a large one) receive atomic adds of the step, the
 * others plain stores.  Where every row would be added to and rows are long enough (d > 32) and
 * sources many enough, each row is written under a lock of its own instead, except those that
 * the epoch draws often, which are still added to; GOSH_FLAG_PLAIN_STORES / GOSH_FLAG_ATOMIC_ADDS
 * force one kind.  No update is lost to adds or locks (but an update whose lock cannot be had in
 * 2^14 tries is added without it).
 * The library owns the memory for this, per device: a bitmap (n bits) or lock words and counts
 * (12 bytes per vertex), allocated on first use and when a larger graph comes, smaller blocks
 * being kept.  All calls share it, so concurrent-mode calls on one device must not overlap on
 * different streams.  Without memory for lock words, and while the stream is being captured, the
 * launch adds.
 * g_dev: CSR arrays on the device.  M_dev: device matrix, updated in place.
 * (Where M_dev lies matters on this device: random row traffic inside one of the three HBM
 * ranks runs at about 5.2 TB/s, across two at about 6.2 TB/s; gosh_matrix_place allocates a
 * matrix that lies across two.)
 * lr_epoch: the already decayed learning rate (gosh_lr).  0 <= k_neg <= GOSH_MAX_NEG. */
int gosh_train_epoch(const gosh_csr *g_dev, float *M_dev, int32_t d, int32_t k_neg,
                     float lr_epoch, uint64_t seed, uint32_t epoch, uint32_t level,
                     uint32_t flags, void *hip_stream);

/* gosh_train_epoch for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  The same epoch with the
 * same arguments and error behaviour, except that it takes no row locks -- where
 * gosh_train_epoch does, this call adds: no update is lost either, and it takes up to twice as
 * long -- and that the hot-row bitmap lives in a fixed array inside the library's code
 * object: GOSH_STATIC_MAX_N bits = 8 MiB of device memory on every GPU the library is loaded
 * on, held until the process ends.  The
 * call allocates and frees nothing, on the device or the host, and takes graphs of at most
 * GOSH_STATIC_MAX_N vertices (GOSH_EINVAL beyond).  The bitmap is rewritten by every call
 * that uses it (nothing of a previous call is relied on), and all calls on one GPU share it:
 * calls that overlap on one GPU -- different streams, or threads -- race on it. */
#define GOSH_STATIC_MAX_N 67108864 /* 2^26 vertices */
int gosh_train_epoch_static(const gosh_csr *g_dev, float *M_dev, int32_t d, int32_t k_neg,
                            float lr_epoch, uint64_t seed, uint32_t epoch, uint32_t level,
                            uint32_t flags, void *hip_stream);

/* Divergence check (no passage of the paper: nothing in Alg. 1 bounds a row, and a learning
 * rate too large for a graph's hubs makes rows grow until fp32 overflows; the training calls
 * themselves are asynchronous and cannot tell).  Reads the n x d device matrix once and
 * returns the largest finite |entry| in *max_abs and the number of non-finite entries in
 * *nonfinite (either may be NULL).  Blocking: waits for the stream.  Uses a 16-byte
 * per-device result buffer owned by the library, so calls on one device must not overlap. */
int gosh_matrix_check(const float *M_dev, int64_t n, int32_t d, float *max_abs, int64_t *nonfinite,
                      void *hip_stream);

/* Row probe (no passage of the paper: the memory of the device, not the method): the row
 * traffic of the training kernels without their arithmetic, to be timed by the caller (HIP
 * events on the stream) -- to compare candidate locations for a matrix (on this device
 * random row traffic inside one of the three HBM ranks is slower than traffic that spans
 * two, see gosh_train_epoch), and to measure what the memory system allows a kernel that
 * moves rows of 4*d bytes at random.  A lane group of pow2ceil(d/4) lanes moves one row with
 * 128-bit accesses.  `accesses` units of work, drawn with Philox from `seed`:
 *   GOSH_PROBE_READ_WRITE  a uniformly random row is read and written back unchanged
 *   GOSH_PROBE_READ        a uniformly random row is read
 *   GOSH_PROBE_WRITE       a uniformly random row is overwritten with zeros
 *   GOSH_PROBE_EPOCH_MIX   the traffic of one source of Alg. 3 with three negatives: row
 *                          (i mod n) and four random rows are read, then all five written
 *                          back unchanged (5 + 5 row transfers per access)
 * Except in GOSH_PROBE_WRITE mode the matrix keeps its values, provided nothing else writes
 * it meanwhile.  Asynchronous on the stream. */
#define GOSH_PROBE_READ_WRITE 0
#define GOSH_PROBE_READ 1
#define GOSH_PROBE_WRITE 2
#define GOSH_PROBE_EPOCH_MIX 3
int gosh_row_probe(float *M_dev, int64_t n, int32_t d, int64_t accesses, uint64_t seed, int32_t mode,
                   void *hip_stream);

/* What gosh_matrix_place found (all sizes in bytes). */
typedef struct {
  uint64_t arena_bytes;          /* physical memory mapped for the search */
  uint64_t window_offset_bytes;  /* where in the arena the matrix starts */
  uint64_t kept_bytes;           /* what stays allocated: the 1 GiB pieces under the matrix */
  int32_t probes;                /* windows timed */
  float probe_ms_best, probe_ms_median;
  double search_ms;
} gosh_placement_info;

/* Allocates an n x d device matrix where random row traffic is fastest (no passage of the
 * paper: the memory of the device).  Maps an arena of arena_bytes (0: 120 GiB; never more
 * than what is free less 8 GiB; at least three times the matrix, else GOSH_ENOMEM) out of
 * 1 GiB pieces with the virtual-memory API, times gosh_row_probe on windows of it, returns
 * the fastest window in *M_dev -- in practice one that lies across two of the three HBM
 * ranks -- and gives the pieces outside it back before returning.  The matrix is
 * uninitialised.  Blocking; uses the null stream.  Free it with gosh_matrix_release (not
 * hipFree), after the work that uses it is done.  info may be NULL. */
int gosh_matrix_place(int64_t n, int32_t d, uint64_t arena_bytes, float **M_dev,
                      gosh_placement_info *info);
int gosh_matrix_release(float *M_dev);

/* "ExpandEmbedding" (Alg. 2; Sec. 3: the row of a vertex of G_{i-1} is the row of its
 * super vertex in G_i): M_fine[v,:] = M_coarse[map[v],:] for v < n_fine.  All pointers
 * are device memory; map holds n_fine ids in [0, n_coarse); an entry outside that range
 * gives a row of zeros.  M_fine and M_coarse must not overlap.  A slice of the fine level
 * can be projected by passing the matching slice of map and of M_fine. */
int gosh_project(const float *M_coarse_dev, int64_t n_coarse, const int32_t *map_dev,
                 int64_t n_fine, int32_t d, float *M_fine_dev, void *hip_stream);

/* ---- multilevel driver ---------------------------------------------------------------- */

typedef struct {
  int32_t level;     /* i */
  int64_t n, nnz;    /* size of G_i */
  int64_t epochs;    /* passes of Alg. 3 run on G_i: e_i, times ceil(|E_i|/|V_i|) with
                        GOSH_FLAG_EDGE_EPOCHS */
  double upload_ms;  /* host -> device copy of G_i (wall clock) */
  double train_ms;   /* the e_i epoch launches (HIP events on the stream) */
  double project_ms; /* projection to level i-1 (0 at level 0): HIP events around it where both matrices and
                        the map are on the device, else wall clock with the copies of map and rows */
  int32_t parts_K;   /* 0: trained with the epoch kernel; K > 0: trained with the part-pair
                        rotation on K parts (train_ms is then the wall time of that call) */
  float max_abs;     /* largest finite |entry| of M_i after training (levels trained by the
                        rotation on a host matrix: as met when parts were written back) */
  int64_t nonfinite; /* non-finite entries of M_i after training; 0 unless training diverged */
} gosh_level_stats;

/* Alg. 2 ("GOSH") for levels that fit the device: with D = levels of h and
 * e_i = gosh_epoch_split(epochs, p, D), for i = D-1 down to 0: copy G_i to the device,
 * (i = D-1: initialise M_{D-1} with gosh_init_embedding(seed, level D-1)), run e_i epochs
 * of gosh_train_epoch with lr = gosh_lr(lr0, j, e_i), epoch j and level i in the random
 * counter, then (i > 0) project to level i-1 with map_{i-1}.  The paper prints the loop
 * as "D-1 to 1"; the text trains until M_0 is obtained, which is what is done here.
 * h: hierarchy (host).  M0_dev: device matrix n_0 x d, receives the embedding of G_0.
 * flags: as for gosh_train_epoch, plus GOSH_FLAG_EDGE_EPOCHS and GOSH_FLAG_PAIR_LEVELS.
 * device_budget_bytes: if non-zero and the graph plus matrix of level 0 exceed it, the call is
 * refused with GOSH_EBUDGET (use gosh_embed_host, which keeps such levels on the host).
 * stats: NULL or host array of D entries; a call that fails at some level has filled those of the
 * levels that it finished before.
 * Blocking: returns after the last level finished; intermediate device buffers are
 * allocated and freed inside the call (without a budget those of up to 64 MB are blocks that the
 * library keeps for the next call, as it does those of freed hierarchies; gosh_hierarchy_trim_scratch
 * returns them).  The call waits for its own stream; it waits for the whole device only where it frees
 * buffers on the way or fails.  Every level is checked after its training
 * (gosh_matrix_check: one more read of the matrix): if any level ends with non-finite
 * entries the run is still completed, stats are filled, and GOSH_EDIVERGED is returned. */
int gosh_embed(const gosh_hierarchy *h, int32_t d, int32_t k_neg, int64_t epochs, double p,
               float lr0, uint64_t seed, uint32_t flags, uint64_t device_budget_bytes,
               float *M0_dev, gosh_level_stats *stats, void *hip_stream);

/* Alg. 2 including its "fits into GPU" branch, with the result on the host.  Levels whose
 * graph and matrix fit device_budget_bytes (0 = what the current device has free when the
 * call starts, less a sixteenth; graphs the hierarchy already keeps there are outside
 * that figure) are trained as in
 * gosh_embed; the others are trained with gosh_train_parts(level i, e_i epochs, the same
 * budget, P_gpu, S_gpu, B) on a host-resident matrix.  Projection runs on the device
 * (slice by slice when the finer level lives on the host); only when both levels live
 * on the host are the rows gathered there.  The initial matrix of a coarsest level that
 * does not fit is produced on the device slice by slice (same values as
 * gosh_init_embedding).  M0_host: host matrix n_0 x d (pinned memory recommended). */
int gosh_embed_host(const gosh_hierarchy *h, int32_t d, int32_t k_neg, int64_t epochs, double p,
                    float lr0, uint64_t seed, uint32_t flags, uint64_t device_budget_bytes,
                    int32_t P_gpu, int32_t S_gpu, int32_t B, float *M0_host,
                    gosh_level_stats *stats, void *hip_stream);

/* ---- graphs larger than a device budget (Sec. 3.3, Alg. 5 "LargeGraphGPU") -------------- */

typedef struct {
  int32_t K;             /* number of parts (contiguous ranges of ceil(n/K) vertices) */
  int64_t rotations;     /* ceil(epochs / (B*K)), at least 1 */
  int64_t pair_visits;   /* rotations * K(K+1)/2 pair kernels */
  int64_t updates;       /* updates of Alg. 1 attempted (sources * B * (k_neg+1) per visit) */
  uint64_t device_bytes; /* part slots + sample pools + hot-row bitmap (+ 12 bytes for each row
                            of two parts, if they are locked) */
  uint64_t bytes_h2d;    /* parts and pools copied to the device */
  uint64_t bytes_d2h;    /* parts copied back */
  double kernel_ms;      /* sum of the pair kernels' durations (HIP events) */
  double wall_ms;        /* whole call, host wall clock */
  double sampler_ms;     /* time the host sampler spent drawing positives (its own clock) */
  double sampler_wait_ms; /* time the driving thread waited for a pool of positives */
  float max_abs;         /* largest finite |entry| met when parts were written back (device
                            matrix: of the matrix after the last rotation) */
  int64_t nonfinite;     /* non-finite entries met there (a part that leaves the device several
                            times is counted each time); 0 unless training diverged */
} gosh_parts_stats;

/* Visiting order of the part pairs in one rotation (Sec. 3.3.1): (0,0), (1,0), (1,1),
 * (2,0), ... -- K(K+1)/2 pairs written to a[] and b[] (host arrays), a[j] >= b[j]. */
int gosh_pair_order(int32_t K, int32_t *a, int32_t *b);

/* A visiting order that is not the paper's, for hardware whose host link bounds the
 * rotation: the parts are cut into blocks of R consecutive parts; for every block in turn,
 * first the pairs inside the block in the order of gosh_pair_order, then for each later
 * part c the pairs (c, r) for every r of the block.  A device that keeps the block resident
 * and streams the later parts through meets R pairs per part it loads.  Every pair (a, b),
 * a >= b, occurs exactly once; R >= K gives gosh_pair_order.  GOSH_EINVAL if R < 1. */
int gosh_pair_order_blocked(int32_t K, int32_t R, int32_t *a, int32_t *b);

/* The part layout gosh_train_parts would use: the smallest K for which min(P_gpu, K) part
 * slots of ceil(n/K) rows, S_gpu sample pools of 2*ceil(n/K)*B ids and the hot-row bitmap
 * fit device_budget_bytes; rotations = ceil(epochs/(B*K)) (Alg. 5, first line).  Any of
 * the output pointers may be NULL.  GOSH_EBUDGET if no K up to min(n, 4096) fits. */
int gosh_parts_plan(int64_t n, int32_t d, int64_t epochs, uint64_t device_budget_bytes,
                    int32_t P_gpu, int32_t S_gpu, int32_t B, int32_t *K_out,
                    int64_t *rotations_out, uint64_t *device_bytes_out);

/* Parity/debug: the sample ids of one visit of the pair (pa, pb), pb <= pa, in the order
 * the sequential reference applies them: for every vertex of part pa, B rounds of
 * (positive, k_neg negatives), then -- if pa != pb -- the same for every vertex of part pb.
 * Positive of a vertex: uniform member of its neighbours inside the partner part, -1 if
 * none; negatives: uniform over the partner part.  Draw t of a source uses
 * Philox4x32-10(counter = (src, side*B*(k_neg+1) + t, rotation,
 * (level & 255) | (pair_index+1) << 8), key = seed).  Positives are drawn on the host,
 * negatives on the device, exactly as in training.  g_host: host CSR; out_host: host
 * int32[(size(pa) + size(pb))*B*(k_neg+1)] (only size(pa) sources if pa == pb). */
int gosh_parts_sample_pair(const gosh_csr *g_host, int32_t K, int32_t pa, int32_t pb, int32_t B,
                           int32_t k_neg, uint64_t seed, uint32_t rotation, uint32_t level,
                           uint32_t pair_index, int32_t *out_host);

/* Alg. 5 for one level: the matrix stays on the host, K parts rotate through P_gpu device
 * slots, every pair of parts is trained against each other once per rotation (in the
 * order of gosh_pair_order) for `rotations` rotations, with lr = gosh_lr(lr0, r, rotations)
 * in rotation r.  In a visit of (a, b) every vertex of a runs B rounds of one positive
 * update (a neighbour inside b, drawn on the host into a pool that is shipped to the
 * device) and k_neg negative updates (drawn on the device, uniform over b), and vice versa;
 * a vertex without a neighbour in the partner part gets no positive update there.
 * g_host: host CSR, or a CSR in the current device's memory (detected from the pointers;
 * what gosh_embed_host passes for a level of a device-built hierarchy): the pools of
 * positives are then filled by a kernel on the device, with the same values, and no host
 * sampler runs -- on this hardware the graph usually fits the device where the matrix
 * does not (one pool is enough then: S_gpu = 1 leaves more of the budget to the parts).
 * The graph is outside device_budget_bytes either way.
 * M_host: host matrix n x d, updated in place; pinned memory makes the
 * transfers asynchronous.  A matrix in the current device's memory (detected from the
 * pointer) is trained where it is: every part is its own slot, nothing is copied, P_gpu
 * only shapes the blocked pair order, the part count is force_K or else 16, and the budget
 * covers the pools and the bitmap alone.  What is left of Alg. 5 then is its visiting
 * order and its sampling rule, which on this hardware make an epoch's worth of samples
 * 1.2-1.4x cheaper than an epoch of Alg. 3 (a source row is loaded once per B rounds, and
 * the negatives of a visit fall into one part).
 * device_budget_bytes: cap for slots + pools + bitmap (0 only together with force_K > 0,
 * or with a device matrix); rows are locked, as in gosh_train_epoch, only where the words for
 * that fit under the cap too and can be had.  P_gpu >= 2 (paper: 3), S_gpu >= 1 (paper: 4), B >= 1
 * (paper: 5).  force_K > 0 overrides the part count.  flags as for gosh_train_epoch
 * (GOSH_FLAG_SEQUENTIAL: every pair kernel runs on one wavefront, sources in order), plus
 * GOSH_FLAG_BLOCKED_ORDER.
 * The library owns its streams, device buffers and sampler thread for the duration of
 * the call, which blocks until the matrix is back on the host.  stats_out may be NULL.
 * Every part is checked for non-finite entries on the device before it is written back (the
 * whole matrix at the end, if it lives on the device): GOSH_EDIVERGED, with the matrix as
 * training left it, if there were any. */
int gosh_train_parts(const gosh_csr *g_host, float *M_host, int32_t d, int32_t k_neg,
                     int64_t epochs, float lr0, uint64_t seed, uint32_t level,
                     uint64_t device_budget_bytes, int32_t P_gpu, int32_t S_gpu, int32_t B,
                     int32_t force_K, uint32_t flags, gosh_parts_stats *stats_out);

/* ---- a head on the embedding ------------------------------------------------------------- */
/* What is trained on the rows of an embedding, or on products of the rows of vertex pairs: layer norm, linear layers
 * with an activation and a residual, and 8-bit copies of activations kept between the two passes (no passage of the
 * paper: Sec. 4.1 fits a classifier on such products).  All entry points are asynchronous on the stream, allocate
 * nothing and give the same bits for the same arguments; a wrong pointer, size or type is GOSH_EINVAL before anything
 * is launched.  Sums, statistics and accumulators are kept in 32 bits and rounded once, to the type of the output. */

typedef enum { GOSH_F32 = 0, GOSH_BF16 = 1, GOSH_F16 = 2 } gosh_type;

/* Borrowed view of a rows x cols device matrix, entry (r, c) at data[r * ld + c]; ld in elements, ld >= cols.  Rows
 * need no alignment beyond that of their elements (they are read fastest where data and rows are 16-byte aligned).
 * 0 <= rows < 2^31 - 1, 1 <= cols <= GOSH_MAT_MAX_COLS, ld <= GOSH_MAT_MAX_LD; data may be NULL if rows = 0.
 * packed = 0: data holds entries of `type`; exps, ld_exps are ignored.
 * packed = 1: the 8-bit form of a matrix of `type`.  data holds int8 q, and entry (r, c) stands for
 * q * 2^(exps[r * ld_exps + c / 32] - 127), or NaN where that byte is 255; ld_exps >= ceil(cols / 32).  The exponent
 * of a group of 32 columns of a row (the last one of a row may be shorter) is the smallest e for which its largest
 * magnitude is at most 127 * 2^e, e >= -126 (GOSH_F16: -24, the unit of that type), and q = x / 2^e rounded to the
 * nearest whole number, ties to even: an error of half a unit at most, 1/127 of the group's largest magnitude or less
 * above that lowest e.
 * Every such value is exact in `type`.  Where rounding up would leave the type (a largest magnitude within 1.6 % of
 * its largest number) q stops at 63 units.  A group with an entry that is not finite in `type` stands for NaN. */
#define GOSH_MAT_MAX_COLS 65536
#define GOSH_MAT_MAX_LD 1048576
typedef struct {
  void *data;
  uint8_t *exps;
  int64_t rows, ld, ld_exps;
  int32_t cols;
  int32_t type; /* gosh_type */
  int32_t packed;
} gosh_mat;

/* x (not packed) to its 8-bit form q, and q back to x.  Same shape; pack: the same type; unpack: any. */
int gosh_pack8(const gosh_mat *x, const gosh_mat *q, void *hip_stream);
int gosh_unpack8(const gosh_mat *q, const gosh_mat *x, void *hip_stream);

/* Layer norm of each row: mean = sum x / cols, rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps), xhat = (x - mean) * rstd,
 * y = xhat * gamma + beta.  gamma, beta: cols floats.  mean, rstd: rows floats, or NULL.  xhat8, y8: packed matrices
 * of x's type for the backward pass, or NULL: xhat for gosh_layer_norm_backward, y for the x of a linear layer (both
 * from the values in 32 bits).  eps >= 0.  y may be x. */
int gosh_layer_norm(const gosh_mat *x, const float *gamma, const float *beta, float eps, const gosh_mat *y, float *mean,
                    float *rstd, const gosh_mat *xhat8, const gosh_mat *y8, void *hip_stream);

/* Its gradient: with g = dy * gamma and m(.) the mean over the columns,
 *   dx = rstd * (g - m(g) - xhat * m(g * xhat)) + add;  dgamma = sum over rows dy * xhat;  dbeta = sum over rows dy.
 * x: the rows that were normalised, with their mean; or packed, the xhat8 of gosh_layer_norm (mean is ignored then).
 * add: the gradient that reaches x beside the norm (a residual branch), or NULL.  dx may be dy or add.  dx, or both
 * dgamma and dbeta, may be NULL.  With rows = 0 dgamma and dbeta are zero.
 * workspace: device memory of at least gosh_layer_norm_workspace(rows, cols) bytes, 16-byte aligned, that no other
 * work uses until the call's is done (nothing is kept in it; NULL where that is 0 or dgamma is NULL).  The function is 0
 * for rows = 0 and for sizes that the call refuses. */
int gosh_layer_norm_backward(const gosh_mat *dy, const gosh_mat *x, const float *gamma, const float *mean,
                             const float *rstd, const gosh_mat *add, const gosh_mat *dx, float *dgamma, float *dbeta,
                             void *workspace, uint64_t workspace_bytes, void *hip_stream);
uint64_t gosh_layer_norm_workspace(int64_t rows, int32_t cols);

/* Activations: z; max(z, 0); z * s(2 sqrt(2/pi) (z + 0.044715 z^3)), GELU in its form with tanh; z * s(z).  s is the
 * logistic function.  The slope of RELU at 0 is 0. */
#define GOSH_ACT_NONE 0
#define GOSH_ACT_RELU 1
#define GOSH_ACT_GELU 2
#define GOSH_ACT_SILU 3

/* Linear layer: z = x w^T + bias, y = act(z) + residual.  x: rows x in; w: out x in; y: rows x out; all of one type,
 * not packed.  bias: out floats, or NULL.  residual: as y, or NULL; it may be y itself.  z, y8: what the backward pass
 * wants, or NULL: z as y, or packed; y8 packed, of y (both from the values in 32 bits).  y must not overlap x or w.
 * Products, here and in the gradient, are summed in 32 bits; those of GOSH_F32 have the accuracy of 32-bit products where
 * both entries are 0 or 2^-110 (7.7e-34) or more in magnitude; a smaller one may count as another, up to 2^-134 off.
 * Not-finite entries reach the results that they are part of and no others; an infinite one of GOSH_F32 (or one over
 * 3.39e38) may give NaN there. */
int gosh_linear(const gosh_mat *x, const gosh_mat *w, const float *bias, int32_t act, const gosh_mat *residual,
                const gosh_mat *y, const gosh_mat *z, const gosh_mat *y8, void *hip_stream);

/* Its gradient: dz = dy * act'(z), dx = dz w, dw = dz^T x, db = sum over rows dz (the residual's gradient is dy).
 * dy: rows x out.  x: rows x in, or packed.  w: out x in.  z: rows x out, or packed; NULL with GOSH_ACT_NONE.  dx:
 * rows x in; dw: out x in; db: out floats.  Any of the three may be NULL; w may be NULL if dx is, x if dw is.  All
 * of one type, but dw may be GOSH_F32.  dz is rounded to that type before the two products, not in db.  With rows = 0
 * dw and db are zero.  dx must not overlap dy, x, w or z.
 * workspace: as above, at least gosh_linear_backward_workspace bytes (where db is all that is asked for, those of any in). */
int gosh_linear_backward(const gosh_mat *dy, const gosh_mat *x, const gosh_mat *w, const gosh_mat *z, int32_t act,
                         const gosh_mat *dx, const gosh_mat *dw, float *db, void *workspace, uint64_t workspace_bytes,
                         void *hip_stream);
uint64_t gosh_linear_backward_workspace(int64_t rows, int32_t in, int32_t out, int32_t type, int32_t act);

/* ---- the head in 8-bit floating point ------------------------------------------------------- */
/* Linear layers whose operands are kept in 8 bits: half the bytes of 16, and for results of GOSH_BF16 twice the rate of 16 bits
 * on the matrix cores (131,072 x 1024 -> 4096 with GELU 0.71 ms with x put into 8 bits, gosh_linear 1.13).  Products for results of
 * GOSH_F16 and GOSH_F32, of layers with GOSH_ACT_RELU and with GOSH_FP8_EXACT run at the rate of 16 bits at most: 1.25, 1.43, 1.19 and
 * 1.24 ms, where gosh_linear takes 1.19 (GOSH_F16), 5.7 (GOSH_F32) and 1.07 (ReLU).  As above: asynchronous, nothing allocated, the
 * same bits for the same arguments.
 * Results are sums in 32 bits of exact products (an entry below 2^-133 may count as another, up to 2^-134 off); but for those of
 * GOSH_BF16 (not of a layer with GOSH_ACT_RELU, and not where there are so few results that their rate does not matter) the matrix
 * cores take eight products along the sum at a time and cut off what is below 2^-13 of the largest: together less than 2^-10 of the
 * magnitudes that are summed, typically 2^-16.  With GOSH_FP8_EXACT added to act they are exact too. */
#define GOSH_FP8_EXACT 256

/* Borrowed view of a rows x cols device matrix in 8-bit floating point.  data holds e4m3 entries q (a sign, 4 bits of
 * exponent, 3 of mantissa; largest 448, 0x7f and 0xff NaN), entry (r, c) at data[r * ld + c], and stands for
 * q * 2^(exps[r / block_rows * ld_exps + c / 128] - 127).  block_rows: 1 (128 columns of a row share a power of two) or
 * 128 (a square of 128 x 128; the last ones may be smaller).
 * 0 <= rows < 2^31 - 1, 0 <= cols <= GOSH_FP8_MAX_LD; data 16-byte aligned, exps 4-byte aligned, both may be NULL without
 * entries; ld a multiple of 128, cols <= ld <= GOSH_FP8_MAX_LD; ld_exps a multiple of 4, at least ceil(cols / 128), at most
 * GOSH_FP8_MAX_LD.  The bytes from cols to the next multiple of 128 of each row are zero: gosh_pack_fp8 writes them, and the
 * products take them for entries.  Exponent bytes are 1 to 254; those from ceil(cols / 128) to the next multiple of 4 of each
 * row of them are read, whatever they hold.
 * gosh_pack_fp8 takes the smallest power of two, at least 2^-126, at which the block's largest finite magnitude is at most
 * 448, and rounds once, to the nearest, ties to even: half of 2^-3 of an entry's magnitude at most down to 2^-6 of the unit,
 * 2^-10 of the unit below.  An entry that is not finite becomes NaN. */
#define GOSH_FP8_MAX_LD 8388608
typedef struct {
  void *data;
  uint8_t *exps;
  int64_t rows, cols, ld, ld_exps;
  int32_t block_rows;
} gosh_fp8;

/* x (not packed) to 8-bit floating point: as it is into q, transposed into qt (cols x rows; its blocks are 128 rows of a
 * column of x, or the squares of q), or both; one of them may be NULL.  With both, block_rows has to be the same. */
int gosh_pack_fp8(const gosh_mat *x, const gosh_fp8 *q, const gosh_fp8 *qt, void *hip_stream);
/* q back to x, a matrix of any type that is not packed; rounded once. */
int gosh_unpack_fp8(const gosh_fp8 *q, const gosh_mat *x, void *hip_stream);

/* Linear layer: z = x8 w^T + bias, y = act(z) + residual.  x: rows x in, of any type, is put into x8 first (block_rows 1),
 * as by gosh_pack_fp8; or NULL, and x8 holds it.  w: out x in, of either block_rows, out <= GOSH_MAT_MAX_COLS.  bias, act
 * (GOSH_FP8_EXACT may be added), residual, y and z (which may be packed) as for gosh_linear, of one type.  y must not overlap x, x8 or w. */
int gosh_linear_fp8(const gosh_mat *x, const gosh_fp8 *x8, const gosh_fp8 *w, const float *bias, int32_t act,
                    const gosh_mat *residual, const gosh_mat *y, const gosh_mat *z, void *hip_stream);

/* Its gradient: dz = dy * act'(z), dx = dz8 w, dw = dz8^T x8, db = sum over rows dz.  dz is formed in 32 bits and put into 8
 * twice, in blocks of 128 columns for dx and of 128 rows for dw; db sums it as it is.  dy: rows x out; z: as dy, or packed;
 * NULL with GOSH_ACT_NONE.  act: GOSH_FP8_EXACT may be added.  xt: in x rows, x transposed, block_rows 1 (gosh_pack_fp8's qt);
 * may be NULL if dw is.  wt: in x out, w transposed, of either block_rows; may be NULL if dx is.  dx: rows x in, of dy's type;
 * dw: out x in, of dy's type or GOSH_F32; db: out floats.  dx or dw may be NULL, db too (db alone: gosh_linear_backward).  in, out <= GOSH_MAT_MAX_COLS;
 * with dw rows <= GOSH_FP8_MAX_LD.  With rows = 0 dw and db are zero.  dx must not overlap dy, z, wt or xt,
 * nor dw wt or xt.
 * workspace: as above, at least gosh_linear_fp8_backward_workspace bytes (0 for sizes that the call refuses). */
int gosh_linear_fp8_backward(const gosh_mat *dy, const gosh_fp8 *xt, const gosh_fp8 *wt, const gosh_mat *z, int32_t act,
                             const gosh_mat *dx, const gosh_mat *dw, float *db, void *workspace, uint64_t workspace_bytes,
                             void *hip_stream);
uint64_t gosh_linear_fp8_backward_workspace(int64_t rows, int32_t in, int32_t out);

/* ---- losses and steps of a head ---------------------------------------------------------------- */

/* Softmax cross-entropy of each row of logits, rows x classes, of any type (not packed), against one class:
 *   loss = weight * (log(sum exp x) - x[target]),  dlogits = scale * weight * (softmax(x) - [class = target]).
 * targets: rows int32, or int64 with targets_are64 = 1.  A negative target is none: loss and gradient of the row are 0, as
 * they are for a row of weight 0 and for one all of whose logits are -infinity (which takes a class out).  A target of `classes` or more makes
 * both NaN, and so does a logit that is NaN or +infinity.  weight: rows floats, or NULL for 1.  loss: rows floats.
 * dlogits: as logits; may be logits, but must not overlap it otherwise (GOSH_EINVAL); NULL: the loss alone.  One reading of the logits; 32 bits within. */
int gosh_softmax_loss(const gosh_mat *logits, const void *targets, int32_t targets_are64, const float *weight, float scale,
                      float *loss, const gosh_mat *dlogits, void *hip_stream);

/* AdamW.  A parameter tensor of an optimiser: n entries p with their gradients g; state: gosh_adamw_state_bytes(n, bits)
 * bytes, 16-byte aligned, zero (as bytes) before the first step; copy: n entries of copy_type that receive the new
 * parameters rounded, or NULL.  Pointers need the alignment of their entries.  Flat arrays: tensors of any shape whose
 * memory has no gaps. */
typedef struct {
  float *p;
  const void *g;
  void *state;
  void *copy;
  int64_t n;           /* 0 <= n <= 2^40 */
  int32_t g_type;      /* gosh_type */
  int32_t copy_type;   /* GOSH_BF16 or GOSH_F16; ignored without copy */
  int32_t bits;        /* of a moment's entry: 8 or 32 */
  float weight_decay;  /* >= 0 */
} gosh_param;
/* bits = 32: n floats m and, from the next multiple of 16 bytes on, n floats v.  bits = 8, each from the next multiple of 16
 * bytes on: n bytes m, n bytes v, ceil(n / 128) exponent bytes of m, and of v.  128 entries of a tensor share an exponent.
 * m: a sign, 4 bits of exponent, 3 of mantissa, bias 15 (without infinities and NaN; exponent 0 has no leading one); v: 5
 * and 3 bits, bias 31; an entry stands for that number times 2^(byte - 127), or NaN where the byte is 255.  The exponent is
 * the smallest from 2^-95 on at which the block's largest magnitude is at most 1.875.  A block with an entry that is not
 * finite, or beyond 1.875 * 2^126, becomes NaN. */
uint64_t gosh_adamw_state_bytes(int64_t n, int32_t bits);

/* An optimiser over `count` tensors (host array, read by the call): checks them and puts their addresses into device memory
 * of the current device (waits for the device: for what any of its streams was given before).  The arrays stay the caller's and must live, where they are, as long as the
 * optimiser is used.  GOSH_EINVAL also where anything that a step writes overlaps another tensor's arrays. */
int gosh_adamw_create(const gosh_param *params, int32_t count, void **optimiser_out);
void gosh_adamw_free(void *optimiser); /* waits for the device's work */

/* One step, of all tensors in one launch: with g' = scale * g
 *   m = beta1 m + (1 - beta1) g',  v = beta2 v + ((1 - beta2) g') g',
 *   p = p (1 - lr weight_decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * from the moments as they are before they are put back into 8 bits.  t: step, from 1 on; or, where steps is not NULL (device memory),
 * *steps + 1, which the call leaves there.  lr_dev, scale: device floats in place of lr and of 1, or NULL.  Where *scale is
 * not finite nothing changes, *steps neither: a step with gradients that overflowed is left out.
 * 0 <= beta1, beta2 < 1, eps >= 0; lr and eps within the range of 32 bits (eps: 0, or 2^-149 or more).
 * Moments in 8 bits: the bits of a float below the third of its mantissa are cut off, after the addition of 20 bits
 * (i * 2654435769 + t * 1779033703 mod 2^32) / 2^12 (of the complement for v), i the entry's index: so that, over the steps,
 * the mean is right, and a v that shrinks by a thousandth of itself a step does not stay where it is.  A v over 0 does not
 * become 0, by which an update could grow without bound: it takes the smallest number of its block. */
typedef struct {
  double lr, beta1, beta2, eps;
  int64_t step;
  const float *lr_dev, *scale;
  int64_t *steps;
} gosh_adamw_options;
int gosh_adamw_step(void *optimiser, const gosh_adamw_options *options, void *hip_stream);

/* The moments of all tensors as values, to m and v, or from them (in 8 bits rounded to the nearest, v as above): flat arrays of `type`
 * (GOSH_F32; to: GOSH_BF16 too, which holds what 8 bits stand for exactly) in which a tensor begins at the sum of the sizes before it, each
 * rounded up to a multiple of 128; save writes zeros between.  `entries`: of m and of v each, gosh_adamw_entries or more. */
int64_t gosh_adamw_entries(const void *optimiser);
int gosh_adamw_save(void *optimiser, void *m, void *v, int64_t entries, int32_t type, void *hip_stream);
int gosh_adamw_load(void *optimiser, const float *m, const float *v, int64_t entries, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GOSH_H */
