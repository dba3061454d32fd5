/*
 * nms.h - C ABI of the MI355X (gfx950) data-parallel non-maximum suppression library.
 *
 * The library computes what the paper's two kernels compute ("Proposed Parallel
 * Algorithm": Algorithm 1, the all-pairs map kernel, and Algorithm 2, the row-AND
 * reduce kernel; "Algorithm Correctness": their postconditions):
 *
 *   box i survives  <=>  there is no box j that outranks i with overlap(i, j) >= theta
 *
 *   outranks:  score_j > score_i, or score_j == score_i and j < i        (total order;
 *              the paper's guard is the strict score test of Algorithm 1, the index
 *              tie-break is this library's addition)
 *   overlap:   iw = max(0, (min(x2_i, x2_j) - max(x1_i, x1_j)) + 1)
 *              ih = max(0, (min(y2_i, y2_j) - max(y1_i, y1_j)) + 1)
 *              overlap(i, j) = (iw * ih) / (((x2_j - x1_j) + 1) * ((y2_j - y1_j) + 1))
 *              i.e. intersection over the area of the OUTRANKING box, pixel-inclusive
 *              "+1" (Algorithm 1; MapKernel postcondition).  float32, every operation
 *              rounded to nearest-even on its own, in the order written.
 *
 * An eliminated box still eliminates others (ReduceKernel postcondition: V_i is the
 * AND of the whole row of B).  This is not the sequential greedy procedure.
 *
 * Conventions for every entry point
 *   - Pointers are DEVICE pointers unless a parameter says "host".  `stream` is a
 *     hipStream_t passed as void* (NULL = the default stream).
 *   - Calls only enqueue kernels on `stream` and return; they never allocate device
 *     memory, never synchronise, issue no memset or copy, and keep no state (except
 *     nms_init's pool, below), so they may be captured in a HIP graph.
 *   - The caller owns every buffer.  Buffers must stay valid until the stream has
 *     passed the call.  Inputs are never written.
 *   - Return value: NMS_OK or a negative nms_status.  Arguments are validated on the
 *     host before anything is launched; on error nothing has been enqueued.
 *     n == 0 (or frames == 0) is NMS_OK and enqueues nothing.
 *   - Preconditions that are NOT checked (results unspecified, memory-safe anyway):
 *     coordinates finite with |x| <= 2^40, x2 >= x1, y2 >= y1, scores not NaN.
 *   - Same inputs give the same bits, on any stream.
 *   - A box table ("sorted5") for n boxes is 5 * nms_padded_n(n) floats:
 *     first nms_padded_n(n) rows of (x1, y1, x2, y2) in rank order, then
 *     nms_padded_n(n) areas in rank order.  Rows at or beyond n hold the box (0,0,0,0), area 1.
 *   - An elimination mask for n boxes is nms_mask_words(n) 64-bit words laid out
 *     mask[w * nms_padded_n(n) + r]: bit b of that word is 1 iff the box of rank
 *     64*w + b eliminates the box of rank r.  Only words with w <= r / 64 are written
 *     (the ranked lower triangle; a box is only ever eliminated by a better-ranked
 *     one); bits at or above the diagonal and rows at or beyond n are written as 0.
 *   - Batched calls process `frames` independent frames.  Frame f uses
 *     boxes + f*n_max*4, scores + f*n_max, order + f*n_max, keep_out + f*n_max,
 *     sorted5 + f*5*nms_padded_n(n_max), mask + f*nms_mask_words(n_max).
 *     counts[f] (device, may be NULL = every frame holds n_max boxes) is clamped to
 *     [0, n_max]; keep_out entries at or beyond counts[f] are written 0.
 */
#ifndef NMS_MI355X_H
#define NMS_MI355X_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define NMS_VERSION 100          /* major*10000 + minor*100 + patch */
#define NMS_TILE 64              /* boxes per tile = wavefront width */
#define NMS_MAX_N 65536          /* largest n (and n_max) accepted */
#define NMS_MAX_FRAMES 65535     /* largest batch accepted */
#define NMS_MAX_MAP_WORKGROUPS 16777215  /* frames (rounded up to 8) x ceil(work units of a frame / 4) must not exceed this:
                                            the pair-test step of a batch is one launch.  A frame of n boxes has about
                                            (n/64)^2 / 8 work units; the limit only binds above some 5,600 boxes per frame
                                            (about 8,000 frames of 16,384 boxes, 500 of 65,536) */
#define NMS_SORT_CHUNK 4096      /* boxes ranked by one workgroup in LDS */
#define NMS_MAX_MATRIX 16384     /* largest capacity of the byte-matrix form (256 MiB of B) */
#define NMS_STATIC_SCRATCH_BYTES 4194304  /* scratch that the library itself holds on every GPU it is loaded on (4 MiB),
                                             used by nms_run_static_batched only */

typedef enum {
    NMS_OK = 0,
    NMS_ERR_INVALID_ARG = -1,   /* null pointer, negative size, NaN threshold, outputs over inputs (decoding calls) */
    NMS_ERR_TOO_LARGE = -2,     /* n > NMS_MAX_N, frames > NMS_MAX_FRAMES, the batch exceeds NMS_MAX_MAP_WORKGROUPS, or a size
                                   the limits of a decoding call */
    NMS_ERR_WORKSPACE = -3,     /* workspace missing, misaligned or too small; nms_run without nms_init */
    NMS_ERR_LAUNCH = -4         /* the HIP runtime refused a launch */
} nms_status;

/* Static, never freed.  Unknown codes give "unknown status". */
const char *nms_status_string(int status);
int nms_version(void);
/* HIP runtime's description of the calling thread's most recent NMS_ERR_LAUNCH (static string). */
const char *nms_last_launch_error(void);

/* Host-only size helpers (pure functions; 0 on invalid arguments). */
int nms_padded_n(int n);                                  /* n rounded up to a multiple of NMS_TILE */
size_t nms_mask_words(int n);                             /* ceil(n/64) * nms_padded_n(n) */
size_t nms_sort_workspace_bytes(int n_max, int frames);   /* scratch of nms_sort*: 0 when n_max <= NMS_SORT_CHUNK */
size_t nms_workspace_bytes(int n_max, int frames);        /* scratch of nms_run_ws / nms_run_batched */
/* Which kernels nms_run_batched launches for a batch shape at a threshold: one of NMS_ROUTE_*; -1 on invalid sizes or a NaN threshold. */
#define NMS_ROUTE_DIRECT 0
#define NMS_ROUTE_ALL_PAIRS 1
#define NMS_ROUTE_TWO_LAUNCH 2
#define NMS_ROUTE_EARLY_EXIT 3
#define NMS_ROUTE_SMALL_FRAMES 4
#define NMS_ROUTE_PLACE_FRAMES 5
#define NMS_ROUTE_PLACE_TABLE 6
int nms_route_at(int n_max, int frames, float threshold);
/* The same for thresholds that take the literal division (outside [2^-40, 2^20]); 0 .. 4, -1 on invalid sizes. */
int nms_route(int n_max, int frames);

/*
 * Step 1 - rank.  The total order that Algorithm 1 evaluates per pair as
 * "D[i].s < D[j].s", hoisted out of the pair loop so that only the ranked lower
 * triangle of B has to be evaluated.
 *   boxes   [n][4] (x1, y1, x2, y2)      in
 *   scores  [n]                           in
 *   order   [n] int32                     out: order[r] = input index of the box of rank r
 *   sorted5 5 * nms_padded_n(n) floats    out: box table (see above); area as in
 *                                              Algorithm 1's first assignment, per axis
 *   workspace  >= nms_sort_workspace_bytes(n, 1) bytes, 256-byte aligned; may be NULL when that is 0
 */
int nms_sort(const float *boxes, const float *scores, int n,
             int32_t *order, float *sorted5, void *workspace, size_t ws_bytes, void *stream);
int nms_sort_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                     int32_t *order, float *sorted5, void *workspace, size_t ws_bytes, void *stream);

/*
 * Step 2 - map.  Algorithm 1 on the ranked lower triangle, bit-packed and with the
 * polarity inverted (bit = 1 where the paper's B_ij is false).  One 64-bit word per
 * box per 64-box tile of outranking boxes.
 *   sorted5   box table from step 1      in
 *   threshold theta, any float but NaN (no clamping: theta <= 0 eliminates everything
 *             below the top rank, theta > 1 nothing)
 *   mask      nms_mask_words(n) words     out (layout above)
 */
int nms_overlap_mask(const float *sorted5, int n, float threshold, uint64_t *mask, void *stream);
int nms_overlap_mask_batched(const float *sorted5, const int32_t *counts, int n_max, int frames,
                             float threshold, uint64_t *mask, void *stream);

/*
 * Step 3 - reduce.  Algorithm 2's result (V_i = AND of row i of B), i.e. rank r
 * survives iff all its mask words are zero, scattered back to input order
 * (Equation 2 applies V to D index by index).
 *   keep_out [n] bytes, 1 = survives, 0 = eliminated
 */
int nms_reduce(const uint64_t *mask, const int32_t *order, int n, uint8_t *keep_out, void *stream);
int nms_reduce_batched(const uint64_t *mask, const int32_t *order, const int32_t *counts, int n_max, int frames,
                       uint8_t *keep_out, void *stream);

/*
 * The whole path in one call.  No mask is written to memory: the row AND is folded
 * into the pair tests, and the result is the same keep vector as steps 1-3 give.
 * The call picks its route by size and threshold (nms_route_at() names it); every route returns the same bits.
 *   NMS_ROUTE_PLACE_FRAMES  thresholds in [2^-40, 2^20], batches of frames of 449 to 4096 boxes: two frames of
 *                         2300 boxes or more, four of 2049 or more, 9000 boxes in frames beyond 1024 (8000 from 1640 on),
 *                         28,000 in frames beyond 512, 512 frames of 449 to 512.  One launch: the boxes in order of place
 *                         instead of rank, pairs of boxes that lie apart are left out.
 *   NMS_ROUTE_PLACE_TABLE the same thresholds, frames of more than NMS_SORT_CHUNK boxes: the same in two launches.
 * Other thresholds, and what these leave:
 *   NMS_ROUTE_DIRECT      small work (up to about 2^25 pair slots = frames * n_max^2): one launch.
 *   NMS_ROUTE_SMALL_FRAMES  batches of ten or more frames of 513 to 1024 boxes (of 128 or more
 *                         frames from 449 boxes on), and 2 to about 40
 *                         frames of 1025 to 4096 boxes (which batch sizes depends on the frame
 *                         length; nms_route_at() tells): one launch without a sort, every victim
 *                         against the two best-ranked of every sixteen input boxes, then the
 *                         victims still alive against the whole frame; rank order enters as a
 *                         compare of the two boxes' (score, index) keys.
 *   NMS_ROUTE_ALL_PAIRS   rank step, then every pair test of the ranked triangle.
 *   NMS_ROUTE_TWO_LAUNCH  frames beyond NMS_SORT_CHUNK boxes, 2^27 <= pair slots < 2^31: rank step,
 *                         every victim against the best 2048 ranks, then only the victims still
 *                         alive against the rest.
 *   NMS_ROUTE_EARLY_EXIT  large batches (frames of 1025 to NMS_SORT_CHUNK boxes from 2^28 pair
 *                         slots, larger frames from 2^31): nms_run_early_exit_batched below.
 * All but DIRECT and ALL_PAIRS skip pair tests of victims that already have an eliminator, so
 * their running time depends on the data.  Callers that want every pair evaluated whatever the
 * size (a fixed running time) call nms_run_ranked_batched.
 *   workspace >= nms_workspace_bytes(n or n_max, 1 or frames) bytes, 256-byte aligned
 *             (always required, whichever route is taken).
 * Two calls that share a workspace must be ordered on one stream.
 */
int nms_run_ws(const float *boxes, const float *scores, int n, float threshold,
               uint8_t *keep_out, void *workspace, size_t ws_bytes, void *stream);
int nms_run_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                    float threshold, uint8_t *keep_out, void *workspace, size_t ws_bytes, void *stream);

/*
 * The two all-pairs routes that nms_run_batched chooses between, callable on their own.
 *   ranked  rank step, then pair tests on the ranked lower triangle (each pair once).
 *           Needs the workspace.  Chosen for batches and large frames.
 *   direct  one launch, no workspace: Algorithm 1 on the full n x n grid of the unsorted
 *           input with the score guard evaluated per pair, row AND finished in the
 *           workgroup.  About 2.5x the arithmetic, so it is chosen only where launch
 *           latency dominates (n_max <= 4096 and frames * n_max^2 up to about 2^25).
 * Both give the same keep_out as nms_run_batched, bit for bit, for any sizes.
 */
int nms_run_ranked_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                           float threshold, uint8_t *keep_out, void *workspace, size_t ws_bytes, void *stream);
int nms_run_direct_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                           float threshold, uint8_t *keep_out, void *stream);

/*
 * The classic sequential greedy rule as a selectable reduce: rank r survives iff no
 * SURVIVING better-ranked box eliminates it (the procedure the paper's introduction and
 * related-work section describe; Algorithms 1 and 2 themselves let eliminated boxes
 * eliminate too).  Same mask, same overlap measure, same tie rule; every box kept by
 * nms_reduce is also kept here.
 *   nms_reduce_greedy*        step 3 alternative on the mask of step 2
 *   nms_run_greedy_batched    rank + map + greedy sweep; needs the mask in its workspace:
 *                             >= nms_greedy_workspace_bytes(n_max, frames) bytes, 256-byte aligned.
 *                             Batches of frames of at most NMS_SORT_CHUNK boxes with
 *                             frames * n_max >= 32 * 4096 take the route below instead (same
 *                             result, bit for bit).
 *   nms_run_greedy_fused_batched   rank, then one workgroup per frame walks the frame in rank
 *                             order, 64 rows a round, and tests only rows that are still alive
 *                             against boxes that survived; the rows left are packed together
 *                             after 2, 4, 8 ... rounds.  No mask, and most of the pair grid is
 *                             never evaluated.  n_max <= NMS_SORT_CHUNK (else NMS_ERR_TOO_LARGE);
 *                             workspace >= nms_workspace_bytes(n_max, frames).  A frame is one
 *                             compute unit's work, so it pays from a few dozen frames on.
 */
int nms_reduce_greedy(const uint64_t *mask, const int32_t *order, int n, uint8_t *keep_out, void *stream);
int nms_reduce_greedy_batched(const uint64_t *mask, const int32_t *order, const int32_t *counts, int n_max,
                              int frames, uint8_t *keep_out, void *stream);
size_t nms_greedy_workspace_bytes(int n_max, int frames);   /* host-only, pure; 0 on invalid arguments */
int nms_run_greedy_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                           float threshold, uint8_t *keep_out, void *workspace, size_t ws_bytes, void *stream);
int nms_run_greedy_fused_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max,
                                 int frames, float threshold, uint8_t *keep_out, void *workspace, size_t ws_bytes,
                                 void *stream);

/*
 * Selectable variants of the rule (the paper's closing section: the map/reduce pattern
 * carries over to the members of the greedy NMS family with changes in the merging step).
 * Every switch at its first value is the default path above.
 *   rule     NMS_RULE_PAPER   every outranking box counts (Algorithms 1 + 2)
 *            NMS_RULE_GREEDY  only outranking boxes that survive themselves count
 *   measure  NMS_MEASURE_OUTRANKING_AREA  intersection / area of the outranking box (Algorithm 1)
 *            NMS_MEASURE_IOU              intersection / ((area_i + area_j) - intersection)
 *   compare  NMS_COMPARE_GE   overlap >= theta eliminates (Algorithm 1: B = overlap < theta)
 *            NMS_COMPARE_GT   only overlap > theta eliminates
 *   ties     NMS_TIES_BY_INDEX  equal scores: the lower index outranks
 *            NMS_TIES_IGNORE    equal scores never eliminate each other (Algorithm 1's strict "<" as printed)
 *   pixel_offset  added to every extent before areas and intersections are formed:
 *            1.0f (the paper's pixel-inclusive convention) or 0.0f (continuous coordinates;
 *            then x2 > x1 and y2 > y1 is an unchecked precondition).  Other values: NMS_ERR_INVALID_ARG.
 *   classes  NULL, or device int32 [frames][n_max]: only boxes with equal labels interact.
 * float32, one rounding per operation, in the order written above; the division is IEEE.
 * nms_run_ex_batched: the paper's rule in order of place for most batches (frames beyond 1024 boxes,
 * smaller batches of shorter ones), else rank and the map step with the options and the row
 * reduction folded in; the greedy rule rank, mask (workspace) and sweep, on large batches the
 * mask-free walk, on frames of at most 192 boxes one launch, and under IoU in order of place on most
 * batches of frames of 2049 to 8192 boxes (its time then depends on the data: most where thousands of
 * candidates crowd around few objects).  With every option at its default the call is nms_run_batched /
 * nms_run_greedy_batched.
 *   options    HOST pointer, read before the call returns; NULL = all defaults
 *   workspace  >= nms_ex_workspace_bytes(n_max, frames) bytes, 256-byte aligned
 */
enum { NMS_RULE_PAPER = 0, NMS_RULE_GREEDY = 1 };
enum { NMS_MEASURE_OUTRANKING_AREA = 0, NMS_MEASURE_IOU = 1 };
enum { NMS_COMPARE_GE = 0, NMS_COMPARE_GT = 1 };
enum { NMS_TIES_BY_INDEX = 0, NMS_TIES_IGNORE = 1 };
typedef struct nms_options {
    int32_t rule;
    int32_t measure;
    int32_t compare;
    int32_t ties;
    float pixel_offset;
    int32_t reserved;          /* must be 0 */
    const int32_t *classes;    /* device, or NULL */
} nms_options;
size_t nms_ex_workspace_bytes(int n_max, int frames);   /* host-only, pure; 0 on invalid arguments */
int nms_run_ex_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                       float threshold, const nms_options *options, uint8_t *keep_out,
                       void *workspace, size_t ws_bytes, void *stream);

/*
 * The paper's rule with work skipped that cannot change the result (section "Algorithm
 * Correctness": V_i is the AND over all j, so it is settled by the first j that eliminates i):
 * a victim that has met an eliminator is dropped from all further tests, while it goes on
 * eliminating others.  Same keep vector as nms_run_batched, bit for bit, from a fraction of the
 * pair tests on clustered detections (a quarter on 4096-box frames of SSD-style anchors).  One
 * workgroup per frame, which ranks the frame, keeps its boxes and the list of undecided victims in
 * LDS and takes the outranking boxes in stages of doubling width (with fewer frames than compute
 * units a frame's victims are shared out among several workgroups; frames beyond NMS_SORT_CHUNK
 * boxes always are, and their workgroups fetch the outranking boxes from the ranked table in
 * memory); it pays from about 2^28 pair slots per batch (frames * n_max^2) on.  Sizes as
 * nms_run_batched; workspace >= nms_workspace_bytes(n_max, frames), 256-byte aligned (used
 * for the rank step's tables unless the rank step runs inside the kernel; required in either case).
 * Arguments, layout, ownership and errors as nms_run_batched.
 */
int nms_run_early_exit_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                               float threshold, uint8_t *keep_out, void *workspace, size_t ws_bytes, void *stream);

/*
 * The paper's own data layout, for measuring its form on this hardware: the boolean
 * matrix B as capacity x capacity BYTES over the UNSORTED input (Algorithm 1, one
 * matrix element per ordered pair, the score guard evaluated per pair), and
 * Algorithm 2's reduce with its k row partitions (a row gets capacity / k / 8 lanes --
 * capacity / k when that is not a multiple of 8 --, each of which folds its columns of all k
 * partitions; one combine per row instead of the paper's k block-wide ANDs).
 *   nms_map_matrix     B[i * capacity + j] = 0 iff j outranks i and overlap(i, j) >= theta,
 *                      else 1.  Every byte of B is written (the paper presets B to 1 with
 *                      a memset and rewrites the guarded entries; slots at or beyond n
 *                      never pass the guard there and come out as 1 here).
 *                      Outranking is this library's total order (index breaks score ties).
 *   nms_reduce_matrix  V[i] = AND over j of B[i * capacity + j], for all capacity rows
 *                      (rows of unused slots give 1, as in the paper).
 *   n <= capacity <= NMS_MAX_MATRIX, capacity a multiple of 64; k >= 1 divides capacity and
 *   capacity / k <= 1024; otherwise NMS_ERR_INVALID_ARG.
 */
int nms_map_matrix(const float *boxes, const float *scores, int n, int capacity, float threshold,
                   uint8_t *B, void *stream);
int nms_reduce_matrix(const uint8_t *B, int capacity, int k, uint8_t *V, void *stream);

/*
 * Profiling variant of the all-pairs routes (ranked or direct, chosen by size as in
 * nms_run_batched; never the early-exit route): identical work, and in addition records the
 * caller's HIP events on `stream`.  `events` is a HOST array of three hipEvent_t
 * (each may be NULL = skip): [0] before the rank step, [1] between rank and map,
 * [2] after the map step ([1] directly follows [0] on the direct route, which has no
 * rank step).  Event-record failures are reported as NMS_ERR_LAUNCH.
 */
int nms_run_batched_profiled(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                             float threshold, uint8_t *keep_out, void *workspace, size_t ws_bytes, void *stream,
                             void *const *events);

/*
 * nms_run: the same with the workspace taken from a pool registered once.
 * nms_init stores the pointer (caller-owned device memory, at least
 * nms_workspace_bytes(n_max, frames_max) bytes); nms_shutdown forgets it and never
 * frees it.  This pool is the library's only global state: one nms_run in flight at
 * a time, all on one stream.  nms_run before nms_init, or with n > the pool's n_max,
 * returns NMS_ERR_WORKSPACE.
 */
int nms_init(int n_max, int frames_max, void *workspace, size_t ws_bytes);
int nms_shutdown(void);
int nms_run(const float *boxes, const float *scores, int n, float threshold,
            uint8_t *keep_out, void *stream);

/*
 * nms_run_batched for callers that cannot allocate or bring scratch: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  The workspace is a static
 * device array of NMS_STATIC_SCRATCH_BYTES inside the library (one copy per GPU, resident from
 * the time the library is loaded there until the process ends); the call makes no allocation
 * of any kind.  Same result as nms_run_batched, bit for bit; the caller still passes inputs
 * and keep_out.
 *   sizes    nms_workspace_bytes(n_max, frames) must not exceed NMS_STATIC_SCRATCH_BYTES, else
 *            NMS_ERR_TOO_LARGE and nothing is enqueued.  That admits any single frame the library
 *            takes (65,536 boxes: 3.3 MiB), 4 frames of 16,384 boxes, 23 of 4096, 92 of 1024.
 *   sharing  every call on a GPU uses that GPU's one array, which keeps the previous call's
 *            contents (nothing in it has to start at zero: each call writes what it reads).
 *            Calls on the same GPU must therefore be ordered on one stream; calls that overlap
 *            race.  Calls on different GPUs are independent (the current device selects the copy).
 *   set-up   the first call on a device looks up the array's address (hipGetSymbolAddress,
 *            once per device, under a lock); make that call outside graph capture.
 * Other arguments, layout, ownership and errors as nms_run_batched.
 */
int nms_run_static_batched(const float *boxes, const float *scores, const int32_t *counts, int n_max, int frames,
                           float threshold, uint8_t *keep_out, void *stream);

/*
 * Host-only test hook: evaluates, on the CPU, the exact arithmetic the device pair
 * test uses for "does the outranking box eliminate the victim" (all pointers HOST:
 * victim[4], outranking[4]).  Every form of the test that a kernel may take for the pair is
 * evaluated (plain fast form; y-scaled; scaled late); returns 1/0, NMS_HOST_FORMS_DISAGREE if
 * they do not all give the same answer, or a negative status for a NaN threshold.
 * Lets the decision procedure be checked against plain division without a GPU.
 */
#define NMS_HOST_FORMS_DISAGREE (-100)
int nms_host_pair_test(const float *victim, const float *outranking, float threshold);

/*
 * Decoding: which candidates of a model that answers in tokens stand.  The two choices of one decoding step, with the
 * conventions above (device pointers, a stream, no state, nothing allocated, the same bits for the same inputs):
 * how many drafted tokens stand against the target's probabilities (nms_verify_batched), and which rows of a cache
 * stand by the attention weight that they gathered (nms_cache_keep_batched, nms_cache_move_batched, the whole path
 * nms_cache_evict_batched).  The first says how many of the rows that a step wrote to the cache are valid; the second
 * takes that as its counts, lengths and valid_tokens, and brings the cache back to its budget.
 */
enum { NMS_TYPE_F32 = 0, NMS_TYPE_F16 = 1, NMS_TYPE_BF16 = 2 };
#define NMS_MAX_DRAFTS 1024          /* largest drafts_max accepted */
#define NMS_MAX_VOCABULARY 4194304   /* largest vocabulary accepted */
#define NMS_MAX_SLOTS 1048576        /* largest number of slots of a cache accepted */
#define NMS_MAX_QUERY_ROWS 1048576   /* largest group * tokens of nms_cache_weights accepted */
#define NMS_CACHE_MAX_TENSORS 8      /* tensors that one call moves */

/*
 * Verification of drafted tokens by given random numbers.  Sequence s has c = counts[s] drafted tokens x_0 .. x_(c-1);
 * p_i and q_i are the target's and the draft's probabilities at place i, u its random numbers in [0, 1).
 *   accepted   a = the first i < c for which  u_i * q_i(x_i) < p_i(x_i)  does not hold; c when all hold
 *   weights    a < c:  w_j = max(p_a(j) - q_a(j), 0);   a = c:  w_j = p_c(j);   where all of them are 0:  w_j = p_a(j)
 *   token      the least j with  w_0 + .. + w_j  >  u_(drafts_max) * (w_0 + .. + w_(V-1))
 *   out        x_0 .. x_(a-1), token, -1 .. -1
 * so that the tokens out are distributed as the target's own.  Products are exact and sums are in 64 bits (their order
 * depends on the vocabulary alone, so a sequence's tokens do not depend on the batch); where rounding leaves no such j
 * it is the last with w_j > 0; where p_a has no positive entry the token is -1.  Entries that are not a number, infinite
 * or below 0 count as 0, and a drafted token outside the vocabulary has p = q = 0.
 *   target   [sequences][drafts_max + 1][vocabulary] of `type`, target_stride elements from row to row
 *   draft    [sequences][drafts_max][vocabulary] of `type`, draft_stride elements from row to row; NULL: the draft gave
 *            tokens alone, q_i is 1 at x_i and 0 elsewhere
 *   drafts   [sequences][drafts_max] int32 (may be NULL when drafts_max is 0: a plain draw from one row)
 *   counts   [sequences] int32, values above drafts_max count as drafts_max; NULL: drafts_max everywhere.  Below 0: no
 *            sequence at this place of the batch: accepted_out 0, tokens -1.  Its rows of target and draft are not read; its
 *            drafts and uniforms may be, whatever they hold (as may those behind a count)
 *   uniforms [sequences][drafts_max + 1] float: drafts_max for the tests, the last for the token
 *   tokens_out [sequences][drafts_max + 1] int32, accepted_out [sequences] int32; neither may overlap drafts, counts, uniforms or the
 *            other (else NMS_ERR_INVALID_ARG)
 *   workspace  >= nms_verify_workspace_bytes(vocabulary, sequences) bytes, 256-byte aligned; may be NULL when that is 0
 * sequences == 0 is NMS_OK; vocabulary must be at least 1, strides at least vocabulary.
 */
size_t nms_verify_workspace_bytes(int vocabulary, int sequences);   /* host-only, pure; 0 on invalid arguments */
int nms_verify_batched(const void *target, long long target_stride, const void *draft, long long draft_stride, int type,
                       const int32_t *drafts, const int32_t *counts, int drafts_max, int vocabulary, int sequences,
                       const float *uniforms, int32_t *tokens_out, int32_t *accepted_out, void *workspace, size_t ws_bytes,
                       void *stream);

/*
 * Eviction from a cache by accumulated attention weight.  A sequence has n = counts[s] cached rows in slots 0 .. n-1 (the
 * same number for each of its heads); per head and slot there are the weight gathered so far (sums) and the place of the
 * row's token in the text (positions).
 *   1  sums[i] += the step's attention weights of slot i, over the query heads that share the cached head and over the
 *      step's valid tokens.  Added in 64 bits, rounded once to float; weights that are not finite add nothing.
 *   2  the rows are ranked: protected rows first (position < first, or position >= lengths[s] - recent), then higher sums,
 *      then lower slots; sums that are not a number come last.  Rows of rank below k = min(n, budget) stay.
 *   3  the i-th row that stays in a slot at or beyond k moves to the i-th slot below k whose row does not: the rows that
 *      stay fill slots 0 .. k-1, and no other row is touched.  Slots keep no order of positions; whole pages at or beyond
 *      slot k are free.
 * nms_cache_keep_batched does 1 and 2 and names the moves of 3, nms_cache_move_batched moves rows of the caller's tensors,
 * and nms_cache_evict_batched does all of it, moves sums and positions as well and sets the sums of slots k .. n-1 to 0 (so
 * that the next rows written there start with none).  Slots at or beyond n are left as they are in every buffer but keep_out.
 *   sums       float [sequences][heads][n_max], in and out
 *   positions  int32 [sequences][heads][n_max] (out in the whole path), NULL: the slot's number (in the whole path only with
 *              recent == 0, since rows move)
 *   counts     [sequences] int32, clamped to [0, n_max]; NULL: n_max
 *   lengths    [sequences] int32, the tokens of the text so far; NULL: counts
 *   weights    HOST pointer, or NULL (nothing is added)
 *   keep_out   [sequences][heads][n_max] bytes, 1 = the row of this slot stays (slots as before any move), 0 = it goes or
 *              there is none; NULL: not wanted
 *   kept_out   [sequences] int32, k: the next step's rows are written behind it; NULL: not wanted
 *   moves_out  int32 [sequences][heads][nms_cache_moves_max(n_max, budget) + 1][2]: the number of moves and 0, then pairs
 *              (to, from), to ascending, from ascending; entries behind them are left as they are; NULL: not wanted
 *   workspace  >= nms_cache_workspace_bytes(n_max, heads, sequences, budget) bytes, 256-byte aligned
 * No buffer that is written may overlap counts, lengths or valid_tokens (else NMS_ERR_INVALID_ARG).
 * n_max <= NMS_MAX_SLOTS, sequences * heads <= NMS_MAX_FRAMES, group * tokens <= NMS_MAX_QUERY_ROWS; budget, first and recent >= 0.
 */
typedef struct nms_cache_weights {
    const void *weights;          /* device [sequences][heads][group][tokens][columns] of `type`, row_stride elements from row to row */
    long long row_stride;         /* >= columns */
    int32_t type;                 /* NMS_TYPE_* */
    int32_t group;                /* query heads that share a cached head */
    int32_t tokens;               /* query rows per query head */
    int32_t columns;              /* slots that have a weight; those at or beyond it get none (group, tokens or columns 0: nothing is added) */
    const int32_t *valid_tokens;  /* device [sequences]: how many of the query rows count, from the first (clamped to [0, tokens]); NULL: all */
} nms_cache_weights;
/* A tensor whose rows move with their slots: row (sequence, head, slot) begins at rows + sequence * sequence_stride +
 * head * head_stride + slot * slot_stride, all in bytes, none below 0, in any order of size; rows must not overlap.  With pages it begins at rows +
 * page * sequence_stride + head * head_stride + (slot % page_slots) * slot_stride, page = table[sequence * table_stride + slot / page_slots].  A page belongs to one
 * sequence: rows of pages that stand twice in the table, or in two sequences' tables, are not moved in any order. */
typedef struct nms_cache_tensor {
    void *rows;                /* device */
    long long row_bytes;       /* 1 .. 2^20 */
    long long sequence_stride; /* with pages: from page to page */
    long long head_stride;
    long long slot_stride;
} nms_cache_tensor;
typedef struct nms_cache_pages {
    const int32_t *table;      /* device [sequences][table_stride] page numbers; a move from or to a page outside 0 .. pages-1 is left out */
    int32_t table_stride;      /* >= ceil(n_max / page_slots) */
    int32_t page_slots;        /* >= 1 */
    int32_t pages;             /* pages that the tensors hold */
    int32_t reserved;          /* must be 0 */
} nms_cache_pages;
int nms_cache_moves_max(int n_max, int budget);   /* host-only, pure: min(budget, n_max - budget), at least 0; -1 on invalid arguments */
size_t nms_cache_workspace_bytes(int n_max, int heads, int sequences, int budget);   /* host-only, pure; 0 on invalid arguments */
int nms_cache_keep_batched(float *sums, const int32_t *positions, const int32_t *counts, const int32_t *lengths, int n_max,
                           int heads, int sequences, const nms_cache_weights *weights, int budget, int first, int recent,
                           uint8_t *keep_out, int32_t *kept_out, int32_t *moves_out, void *workspace, size_t ws_bytes, void *stream);
/* Moves rows as moves_out of nms_cache_keep_batched says (same n_max, heads, sequences and budget); a pair outside the slots that such a
 * list can name is left out, and so is what lies behind its nms_cache_moves_max entries; a number of moves below 0 is 0.  `tensors`
 * is a HOST array of n_tensors <= NMS_CACHE_MAX_TENSORS, `pages` a HOST pointer or NULL. */
int nms_cache_move_batched(const int32_t *moves, int n_max, int heads, int sequences, int budget, const nms_cache_tensor *tensors,
                           int n_tensors, const nms_cache_pages *pages, void *stream);
int nms_cache_evict_batched(float *sums, int32_t *positions, const int32_t *counts, const int32_t *lengths, int n_max,
                            int heads, int sequences, const nms_cache_weights *weights, int budget, int first, int recent,
                            const nms_cache_tensor *tensors, int n_tensors, const nms_cache_pages *pages,
                            uint8_t *keep_out, int32_t *kept_out, void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* NMS_MI355X_H */
