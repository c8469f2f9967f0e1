/*
 * redist -- array redistribution over a logical device mesh, executed on one NVIDIA B200.
 *
 * The method is the one of "Memory-efficient array redistribution through portable collective
 * communication" (arXiv 2112.01075): a multi-dimensional array is partitioned over a logical mesh
 * under a source distributed type and must reach a target distributed type through a sequence of
 * the collectives allgather, alltoall, dynslice and allpermute.  Here the N mesh devices are
 * *virtual*: every device's tile is its own buffer in the memory of one GPU, and each collective
 * step (or a fused run of adjacent steps) is one CUDA kernel that moves the tiles of all virtual
 * devices at once.
 *
 * Conventions
 *   - A distributed type lists, per array dimension, the mesh axes that partition it, ordered
 *     minor-to-major: the first listed axis varies fastest (Section 2.1, "Distributed array
 *     types").  Tile size = global size / product of the listed axis sizes; it must divide
 *     (rule wf-dim).  Axes a type does not list replicate the data.
 *   - Virtual device id = row-major index of the device's mesh coordinates over mesh_shape
 *     (last mesh axis fastest).  The paper leaves this numbering to the runtime (Section 2.1).
 *   - A tile is dense, row-major, last dimension contiguous, without padding.
 *   - All functions return a redist_status; nothing throws, aborts or prints across this
 *     boundary.  Output arguments are untouched on failure.
 *   - "host" / "device" on a pointer argument says which memory it must point to.
 */
#ifndef REDIST_H_
#define REDIST_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum redist_status {
    REDIST_OK = 0,
    REDIST_EINVAL = 1,       /* null pointer, bad rank / element size / flag / index                   */
    REDIST_EILLFORMED = 2,   /* rules wf-dim / wf-type: unknown axis, axis listed twice                */
    REDIST_ENOTDIV = 3,      /* tile size * product of axis sizes != global size (wf-dim)             */
    REDIST_EGLOBAL = 4,      /* source and target describe different global arrays (Section 2.5)      */
    REDIST_ESCRATCH = 5,     /* scratch buffer missing or smaller than redist_plan_scratch_bytes      */
    REDIST_EOVERLAP = 6,     /* destination / scratch ranges overlap each other or a source           */
    REDIST_EALIGN = 7,       /* a buffer is not aligned to redist_plan_alignment bytes                */
    REDIST_ENOMEM = 8,       /* host allocation failed                                                */
    REDIST_ECUDA = 9,        /* a CUDA call or kernel launch reported an error                        */
    REDIST_EUNSUPPORTED = 10,/* beyond a built-in limit (devices, rank, sizes); see redist_limits     */
    REDIST_EINTERNAL = 11    /* the synthesized plan failed its own end-state check (a bug)           */
} redist_status;

/*
 * A distributed type.  rank dimensions; global_shape[rank]; the axes of dimension k are
 * axes[axes_off[k] .. axes_off[k+1]) as indices into mesh_shape, minor-to-major.  All arrays are
 * host memory, read during the call only.
 */
typedef struct redist_type {
    int32_t rank;
    const int64_t *global_shape;
    const int32_t *axes_off;     /* rank + 1 entries, axes_off[0] == 0 */
    const int32_t *axes;         /* axes_off[rank] entries             */
} redist_type;

typedef struct redist_plan_s redist_plan_t;   /* opaque, host memory, immutable once created */

/* plan flags: exactly one execution mode, optionally or-ed with REDIST_NO_OVERPARTITION,
   REDIST_COST_PERMUTE and/or REDIST_NO_CACHE */
enum {
    REDIST_FUSE_ADJACENT = 0,    /* default: adjacent steps of the sequence run as one kernel wherever
                                    the fused copy keeps contiguous runs of at least 64 bytes         */
    REDIST_FUSE_NONE = 1,        /* one kernel per collective of the sequence; intermediates ping-pong
                                    between two scratch slots per virtual device                      */
    REDIST_FUSE_ALL = 2,         /* the whole sequence as a single kernel, no scratch                  */
    REDIST_NAIVE = 3,            /* comparison baseline only: gather the whole global array, then
                                    slice (the "easy" redistribution, Section 4.3)                    */
    REDIST_MODE_MASK = 3,
    REDIST_NO_OVERPARTITION = 16,/* forbid dynslice steps that partition the array over more mesh
                                    axes than the target type uses (over-partitioning, Section 7.2)  */
    REDIST_COST_PERMUTE = 32,    /* count the final allpermute when choosing the sequence.  The search
                                    of Section 7.3 weighs only dynslice / alltoall / allgather (the
                                    permutation carries no edge weight there) and appends the
                                    permutation afterwards; with this flag the sequences whose own cost
                                    lies below that plan's total are lowered too and the cheapest total
                                    (sequence plus permutation, cost model of Section 6.2) is kept.  The
                                    result never costs more than the default plan and obeys the same
                                    memory bound; planning takes longer.                              */
    REDIST_NO_CACHE = 64         /* synthesize afresh instead of consulting the plan cache             */
};

enum { REDIST_MAX_RANK = 8, REDIST_MAX_MESH_AXES = 16, REDIST_MAX_DEVICES = 1024 };

typedef enum redist_step_kind {
    REDIST_STEP_DYNSLICE = 0,
    REDIST_STEP_ALLTOALL = 1,
    REDIST_STEP_ALLGATHER = 2,
    REDIST_STEP_ALLPERMUTE = 3,
    REDIST_STEP_COPY = 4          /* only for an empty sequence (equal types): tiles are copied    */
} redist_step_kind;

/* One collective of the synthesized sequence (Sections 6 and 7). */
typedef struct redist_step_info {
    int32_t kind;                              /* redist_step_kind                                    */
    int32_t dim_i;                             /* dimension the axes leave (or are sliced into); -1   */
    int32_t dim_j;                             /* alltoall: dimension the axes move to; else -1       */
    int64_t factor;                            /* n = product of the sizes of the axes acted on       */
    int64_t local_before[REDIST_MAX_RANK];     /* localtype before the step                           */
    int64_t local_after[REDIST_MAX_RANK];      /* localtype after the step                            */
    int64_t cost;                              /* cost model of the paper, in elements per device     */
    int64_t localsize_after;                   /* elements per device after the step (for the height) */
} redist_step_info;

/* One kernel launch of the executor. */
typedef struct redist_launch_info {
    int32_t first_step, n_steps;   /* the collectives this launch covers                               */
    int32_t kernel;                /* 0 dynslice, 1 alltoall, 2 allgather, 3 allpermute, 4 copy,
                                      5 fused sequence, 6 naive gather, 7 naive slice                  */
    int32_t vector_bytes;          /* bytes per global memory access                                   */
    int64_t run_bytes;             /* shortest contiguous run                                          */
    int64_t bytes_read;            /* HBM bytes the launch reads (every source element once)          */
    int64_t bytes_written;         /* HBM bytes the launch writes                                      */
    int64_t n_items;               /* work items (thread-block sized pieces)                           */
    int32_t fanout;                /* destination replicas stored per element read                     */
    int32_t variant;               /* kernel variant: 0 rows, 1 chunks, 2 ragged chunks, 3 units (register
                                      kernels), 4 TMA bulk copies, 5 gather walk, 6 ragged rows loaded by
                                      TMA bulk copies, 7 zip through shared memory, 8 super-boxes through
                                      shared memory; the kernel is named
                                      redist_<collective>[_bulk|_gather|_ragged_bulk|_zip|_box]_kernel
                                      (variants 5, 7 and 8 on units of 1 or 2 bytes: redist_fused_..._kernel
                                      whatever the collective)                                        */
} redist_launch_info;

/*
 * redist_plan -- synthesize the sequence of collectives from src to dst (host only, no CUDA call).
 *
 * Follows Section 7: decompose the mesh into prime-sized axes (Principle 1, Section 3), search the
 * graph of weak types (nodes: local types with localsize <= max(localsize src, localsize dst);
 * edges: multi-axes dynslice / alltoall / allgather weighted by the cost model) for a shortest
 * path, lower it to device-map collectives (Lowering Theorem, Section 6.1), and append at most one
 * allpermute, placed before any trailing allgathers (Section 7.3).
 *
 *   n_mesh_axes, mesh_shape[n_mesh_axes]   host; the logical mesh, sizes >= 1
 *   src, dst                               host; distributed types over that mesh
 *   elem_bytes                             1, 2, 4, 8 or 16; elements are copied, never interpreted
 *   flags                                  see above
 *   out                                    host; receives the plan, owned by the caller until
 *                                          redist_plan_destroy
 * Plans are cached (the evaluation of Section 8 asks how long synthesis takes; a runtime asks for the
 * same few redistributions over and over): a second request for the same mesh, types, element size,
 * flags and tuning values returns a handle to the same immutable plan without searching again.  The
 * cache keeps the 256 most recently created plans; every handle must still be destroyed.
 * Errors: EINVAL, EILLFORMED, ENOTDIV, EGLOBAL, EUNSUPPORTED, ENOMEM, EINTERNAL.
 */
redist_status redist_plan(int32_t n_mesh_axes, const int64_t *mesh_shape, const redist_type *src,
                          const redist_type *dst, int32_t elem_bytes, uint32_t flags, redist_plan_t **out);

void redist_plan_destroy(redist_plan_t *plan);

/* Plan cache counters since the library was loaded or the cache was last cleared (any may be NULL). */
void redist_plan_cache_stats(int64_t *hits, int64_t *misses, int64_t *entries);
void redist_plan_cache_clear(void);

/*
 * Tuning values -- process-wide, copied into every plan created afterwards (existing plans keep theirs).
 * Defaults are the measured optima.  Names and ranges:
 *   "bulk"               0/1    1: aligned runs of 512 bytes and more move by TMA bulk copies (default);
 *                               0: register kernels only
 *   "gather"             0..2   gather walk: never / where measured faster (default 1) / wherever it applies
 *   "zip"                0..2   zip kernels: never / only where the gather walk is not chosen / wherever
 *                               they apply (default 2)
 *   "box"                0..2   super-box kernels (several interleaving dimensions staged through shared
 *                               memory at once): never / where the other short-run paths do badly
 *                               (default 1) / wherever they apply
 *   "box_width"          0..256 lanes that share one target range in the super-box kernels (a power of two; other
 *                               values are ignored); 0 (default): a warp or more as a rule, fewer where the units of
 *                               one range would fall into a few shared-memory banks
 *   "zip_walks"          0..7   chunk-to-unit maps the zip kernels may use: 1 periodic + 2 by range +
 *                               4 tabulated (default 7; the flat walk is always available)
 *   "zip_by_range_slots" >= 1   fewest chunk slots of a range for the by-range walk (default 256)
 *   "item_kb"            0..1024 KiB read per work item; 0 (default) = 32 / 16 / 8 by fan-out, and 20 / 12 / 6
 *                               in the bulk-copy kernels
 *   "l2_hint"            0..4   bulk copies of the plain bulk-copy kernels that carry an L2 evict-first policy: none /
 *                               loads / stores / both / stores where every segment goes to four or more replicas
 *                               (default 4)
 *   "piece"              0/1    1 (default): on units of 1 or 2 bytes and runs of 64 bytes and more the super-box
 *                               kernels read a chunk that lies inside one run as one unaligned 16-byte piece; 0: unit by unit
 *   "pdl"                0/1    1: kernels use programmatic dependent launch (default); 0: plain stream order
 *   "nvtx"               0/1    1: redist_execute and redist_execute_static wrap every kernel launch in an NVTX
 *                               range named after the collective, for timeline profilers (default 0)
 *   "step_latency"       >= 0   elements added to the cost of every collective while searching: small
 *                               transfers are bound by per-step latency, not by bytes (Section 8, the
 *                               third research question); 0 (default) is the paper's cost model
 *   "wait_polls"         >= 1   mbarrier polls before a bulk-copy block gives up (default 2^18); the operators'
 *                               matrix products take it from the values in force at the call, as they do "pdl" and
 *                               "test_extra_tx" (the wait for a whole sum gets it again for every 512 stages)
 *   "test_extra_tx"      >= 0   test only: makes every bounded wait run out (see redist_bulk_timeouts)
 *   "test_shrink_tiles"  >= 0   test only: the checked build takes every tile to be that many bytes shorter
 *                               (see redist_debug_bounds_report); no effect on the normal build
 *   "test_product_shape" 0..5   test only: the tile on which every matrix product of the operators runs, whatever its
 *                               size: 256 x 256 or 256 x 128 on a pair of SMs, 128 x 256, 128 x 128 or 128 x 64 on
 *                               one; 0 (default): chosen by size.  128 x 256 is not used where the result is symmetric
 *   "test_product_parts" 0..16  test only, with the former: into how many parts the sums are split (the
 *                               orthogonalisation's never are); 0 (default): one
 * Errors: EINVAL for an unknown name or a value out of range.
 */
redist_status redist_tuning_set(const char *name, int64_t value);
redist_status redist_tuning_get(const char *name, int64_t *value);
void redist_tuning_reset(void);

/*
 * redist_execute -- run the plan on the GPU (asynchronous on `stream`).
 *
 * Executes the collectives of the plan (typing rules T-AllGather, T-DynSlice, T-AllToAll and
 * T-Permute; low-level forms of Section 6) as strided copy kernels over all virtual devices.  The
 * result on every device is the tile its target type prescribes; data values never change.
 *
 *   src_shards[N]   host array of DEVICE pointers; src_shards[d] holds localsize(src)*elem_bytes
 *                   bytes.  Devices that replicate a tile must hold identical bytes (not checked);
 *                   source pointers may alias each other.  Read only.  When the tile size is not a
 *                   multiple of 16 bytes the kernels may read (never write) up to the next 16-byte
 *                   boundary past the tile's end -- always inside the allocation granule of any
 *                   CUDA allocator, and, as tiles start on 16-byte boundaries, never a byte of
 *                   another tile.
 *   dst_shards[N]   host array of DEVICE pointers; dst_shards[d] receives localsize(dst)*elem_bytes
 *                   bytes.  Every destination is written completely.
 *   scratch         DEVICE pointer to at least redist_plan_scratch_bytes(plan) bytes, or NULL when
 *                   that is 0.  Contents are undefined afterwards.
 *   cuda_stream     a cudaStream_t (NULL = default stream) on the current device
 * Ownership: all buffers and the stream belong to the caller.  The call allocates nothing, on the
 * host or on the device (pointer tables and the kernel parameter block live on the call's stack:
 * about 8 KiB for plans of up to 64 virtual devices, about 100 KiB beyond), copies no table to the device (tables travel as kernel parameters) and does not
 * synchronize.  A plan may be executed from several host threads at once on different streams and
 * buffers.
 * Errors: EINVAL, ESCRATCH, EALIGN (pointers must be multiples of redist_plan_alignment),
 * EOVERLAP (destination and scratch ranges must be disjoint from each other and from every
 * source; checked on the host), ECUDA (launch error; see redist_last_cuda_error).
 */
redist_status redist_execute(const redist_plan_t *plan, const void *const *src_shards,
                             void *const *dst_shards, void *scratch, size_t scratch_bytes,
                             void *cuda_stream);

/*
 * redist_bind / redist_bound_execute -- the same execution split in two for callers that run one
 * redistribution on the same buffers many times (every step of a training loop): binding validates
 * the buffers exactly as redist_execute does and prepares every kernel launch once (entry point,
 * launch shape, parameter block with both pointer tables); executing the bound plan is then the
 * kernel launches and nothing else -- no checks, no table building, no allocation.
 *
 *   redist_bind            arguments as redist_execute; *out receives the bound plan (host memory,
 *                          owned by the caller until redist_bound_destroy; it keeps the plan alive).
 *                          The buffers must stay valid and in place while the bound plan is used.
 *   redist_bound_execute   asynchronous on `cuda_stream`; may be called from several threads at once
 *                          (but the launches of all calls write the same buffers: order them)
 * Errors: redist_bind as redist_execute plus ENOMEM; redist_bound_execute EINVAL, ECUDA.
 */
typedef struct redist_bound_s redist_bound_t;
redist_status redist_bind(const redist_plan_t *plan, const void *const *src_shards, void *const *dst_shards,
                          void *scratch, size_t scratch_bytes, redist_bound_t **out);
redist_status redist_bound_execute(const redist_bound_t *bound, void *cuda_stream);
void redist_bound_destroy(redist_bound_t *bound);

/*
 * redist_execute_host -- the same redistribution for tiles that live in HOST memory.
 *
 * Copies every source tile to dev_src (one cudaMemcpyAsync per tile), runs redist_execute on the
 * staged tiles and copies every result tile back, all on `stream`; returns without synchronizing.
 *
 *   src_host[N], dst_host[N]   host arrays of HOST pointers (pinned memory gives true async copies)
 *   dev_src, dev_dst           DEVICE staging buffers of at least redist_plan_staging_bytes(plan, 0)
 *                              and (plan, 1) bytes: N tiles, each rounded up to 256 bytes
 *   scratch                    as for redist_execute
 * Errors: as redist_execute, plus ESCRATCH for staging buffers that are too small.
 */
redist_status redist_execute_host(const redist_plan_t *plan, const void *const *src_host,
                                  void *const *dst_host, void *dev_src, size_t dev_src_bytes,
                                  void *dev_dst, size_t dev_dst_bytes, void *scratch,
                                  size_t scratch_bytes, void *cuda_stream);

/*
 * redist_execute_static -- redist_execute for callers that cannot supply scratch memory.
 * (The paper has no counterpart: it is a property of this library, not of the method.)
 *
 * Some callers have tiles but no way to allocate: a plug-in inside a server that handed all device
 * memory to a pool at start-up and forbids cudaMalloc afterwards, or a latency-bound path on which
 * an allocation may fail or stall.  For them the ping-pong buffers of an unfused plan come from a
 * fixed array of REDIST_STATIC_SCRATCH_BYTES bytes built into the library image (every GPU that
 * loads the library holds those bytes until the process exits).  The call allocates nothing on
 * the device or the host and calls no allocating routine.
 *
 *   plan            any plan with redist_plan_scratch_bytes(plan) <= REDIST_STATIC_SCRATCH_BYTES;
 *                   a larger plan is refused with REDIST_ESCRATCH and nothing runs
 *   src_shards[N], dst_shards[N], cuda_stream    exactly as for redist_execute
 * Set-up: the first call on each device (with that device current) looks up the device address of
 * the built-in array; make that first call before any stream capture begins.  The address is kept
 * for the life of the process: it does not survive a cudaDeviceReset.
 * Sharing: all calls on a device use the same array.  It keeps whatever the previous call left;
 * nothing in it has to start at zero, because every byte a step reads from it was written by an
 * earlier step of the same call.  Two calls whose kernels may overlap on the GPU (different
 * streams without an ordering between them) race on the array: order them.
 * Errors: EINVAL, ESCRATCH (plan too large), EALIGN, EOVERLAP, EUNSUPPORTED (device index >= 64),
 * ECUDA.  Results are identical to redist_execute with a caller-provided scratch buffer.
 */
#define REDIST_STATIC_SCRATCH_BYTES (8u << 20)
redist_status redist_execute_static(const redist_plan_t *plan, const void *const *src_shards,
                                    void *const *dst_shards, void *cuda_stream);

/* ---- queries (host only) -------------------------------------------------------------------- */

int32_t redist_plan_num_devices(const redist_plan_t *plan);               /* N                        */
int32_t redist_plan_rank(const redist_plan_t *plan);
int64_t redist_plan_local_elems(const redist_plan_t *plan, int32_t which); /* 0: source, 1: target    */
size_t  redist_plan_scratch_bytes(const redist_plan_t *plan);             /* total to pass to execute */
size_t  redist_plan_scratch_bytes_per_device(const redist_plan_t *plan);  /* the per-virtual-device
                                               share; for REDIST_NAIVE the size of the global array,
                                               which the literal method would hold on every device   */
size_t  redist_plan_staging_bytes(const redist_plan_t *plan, int32_t which);
int32_t redist_plan_alignment(const redist_plan_t *plan);                 /* required pointer alignment */
int64_t redist_plan_height(const redist_plan_t *plan);   /* max localsize over the sequence (elements);
                                               the memory bound of Section 4.3 says
                                               height <= max(localsize src, localsize dst)            */
int64_t redist_plan_cost(const redist_plan_t *plan);     /* summed cost of the sequence (elements)    */
int32_t redist_plan_num_steps(const redist_plan_t *plan);    /* collectives in the sequence           */
int32_t redist_plan_num_launches(const redist_plan_t *plan); /* kernels redist_execute launches       */
redist_status redist_plan_step_info(const redist_plan_t *plan, int32_t step, redist_step_info *out);
redist_status redist_plan_launch_info(const redist_plan_t *plan, int32_t launch, redist_launch_info *out);

/*
 * redist_plan_describe -- the typed sequence and the launch descriptors as JSON (prime mesh, every
 * step with the axes acted on, the type and the device map after it, costs, and per launch the copy
 * descriptor the kernel receives).  Writes at most cap bytes including the terminating NUL and
 * returns the length the full text needs (excluding the NUL); call with cap = 0 to size a buffer.
 */
size_t redist_plan_describe(const redist_plan_t *plan, char *buf, size_t cap);

/*
 * redist_base_offsets -- base offset map T[[type]] (figure "Semantics for distributed dimensions
 * and types", part (a)): out_offsets[d*rank + k] is the lowest global index in dimension k of the
 * tile held by virtual device d; out_tile[rank] is the local tile shape.  Host only.
 */
redist_status redist_base_offsets(int32_t n_mesh_axes, const int64_t *mesh_shape, const redist_type *type,
                                  int64_t *out_tile, int64_t *out_offsets);

/*
 * redist_plan_gpu_split -- byte accounting for running the plan with its virtual devices spread over
 * several GPUs (host only; nothing in this library moves data between GPUs).  The paper executes its
 * collectives between real devices (Section 8) and discusses individual device-to-device transfers
 * derived from the base offset maps as the alternative (Section 9); this is that derivation for one
 * launch.  Virtual device d is placed on GPU d / (N / n_gpus): the leading mesh coordinates choose the
 * GPU, so n_gpus must be the product of the leading mesh axis sizes times a divisor of the next one.
 *
 *   launch          index of a kernel launch of the plan (redist_plan_num_launches)
 *   bytes           host; receives n_gpus * n_gpus numbers, row-major: bytes[s * n_gpus + t] = bytes that
 *                   GPU s reads from tiles it holds and writes into tiles that live on GPU t (a replicated
 *                   source tile is read on the receiving GPU when that GPU holds a replica, else from the
 *                   lowest-numbered holder).  The diagonal stays inside a GPU; the sum over the matrix is
 *                   the launch's bytes_written; with n_gpus = 1 it is that single number.
 * Errors: EINVAL (also for an n_gpus that is no prefix of the mesh), ENOMEM.
 */
redist_status redist_plan_gpu_split(const redist_plan_t *plan, int32_t n_gpus, int32_t launch, int64_t *bytes);

const char *redist_status_string(redist_status status);

/* The last CUDA error code (cudaError_t as int) seen by the calling thread inside this library. */
int32_t redist_last_cuda_error(void);

/*
 * redist_bulk_timeouts -- health counter of the bulk-copy kernels (not part of the paper's method).
 * Runs are staged in shared memory by TMA bulk copies whose completion a thread block awaits on an
 * mbarrier with a bounded number of polls ("wait_polls").  A block whose wait runs out stores
 * nothing, counts itself here, keeps polling (sleeping up to 256 ns between polls) for as many polls
 * again so that copies still in flight can land in shared memory it still owns, and returns: a
 * faulty copy engine shows up as a non-zero count and unwritten output instead of a hang.  Returns
 * the count for the current device since the library was loaded (0 in a healthy run), or -1 on a
 * CUDA error.  Synchronizes the device.  A non-zero count means the outputs of the run are invalid.
 * The tuning value "test_extra_tx" exists to test this path: it makes every block announce that
 * many bytes more than its copies deliver, so every copy lands but no wait ever completes.
 */
int64_t redist_bulk_timeouts(void);

/*
 * redist_debug_bounds_report -- checked build only (the library compiled with -DREDIST_BOUNDS, which
 * the tests load in place of the normal one).  There every global access of the kernels is tested
 * against the tiles of the launch and every dynamic shared-memory access against the launch's
 * shared-memory size; a failing access is skipped, not performed.  out[0] = number of failed tests
 * since the last call, out[1..4] = source line, thread block, side (1 read, 2 write, 3 shared memory)
 * and distance from the nearest tile base of the first one.  The call resets the record.
 * Synchronizes the device.  The normal build returns EUNSUPPORTED.
 */
redist_status redist_debug_bounds_report(int64_t out[5]);

/* ---- operators on a device's tiles ------------------------------------------------------------ */

/*
 * What runs on a tile between two redistributions (the paper's spmd_op, Section 2.2, is any function of
 * the local tiles): the linear layer and layer norm with their gradients, and the orthogonalisation of a
 * weight update.  All three are asynchronous on `cuda_stream`, allocate nothing and can be captured into
 * a CUDA graph.  Scratch comes from the caller: the matching ..._scratch_bytes query says how much (it
 * depends on sizes, strides and the alignment of the pointers), 256-byte aligned; NULL where it says 0;
 * its contents are undefined before and after.  Sums, means and norms are held in 32 bits or more.
 * Errors of all of them: EINVAL (null pointer, size, type, stride), EALIGN (a pointer off its element
 * size, scratch off 256 bytes), EOVERLAP (an output overlaps an input, scratch or another output, except
 * where said), ESCRATCH, EUNSUPPORTED (more than 2^31 - 512 rows or columns; in the orthogonalisation more than 2^22, or
 * more than 65535 matrices), ECUDA.
 */
typedef enum redist_dtype { REDIST_BF16 = 0, REDIST_F16 = 1, REDIST_F32 = 2 } redist_dtype;

typedef enum redist_activation {
    REDIST_ACT_NONE = 0,
    REDIST_ACT_RELU = 1,
    REDIST_ACT_GELU = 2,        /* z Phi(z), Phi by the error function                                 */
    REDIST_ACT_SILU = 3         /* z / (1 + exp(-z))                                                   */
} redist_activation;

/* A matrix in device memory: element (r, c) at data[r * row_stride + c * col_stride], strides in elements.
   "Row-major" below: col_stride 1 and row_stride >= the number of columns.  Inputs called "either order"
   may also be column-major (row_stride 1, col_stride >= the number of rows).  data NULL: absent. */
typedef struct redist_matrix {
    void *data;
    int64_t row_stride, col_stride;
} redist_matrix;

/*
 * redist_linear_forward -- out = activation(x w^T + bias) + residual.
 *
 *   rows >= 0, in_features >= 1, out_features >= 1
 *   type            REDIST_BF16 or REDIST_F16: x, w, residual, out and pre
 *   x               rows x in_features, either order;  w  out_features x in_features, either order
 *   bias            out_features elements of bias_type (any), or NULL
 *   residual        rows x out_features, row-major, or absent; may be `out` itself
 *   out             rows x out_features, row-major
 *   pre             rows x out_features, row-major, or absent: receives z = x w^T + bias for the backward pass
 * Products are accumulated (16 at a time, every sum cut off to 24 bits) and the epilogue computed in 32 bits; each
 * output is rounded once.  Operands whose lines do not start on 16-byte boundaries are laid out anew in scratch first.
 *
 * redist_linear_backward -- the gradients.  With dz = dy activation'(pre):
 *   dx = dz w  (rows x in_features)     dw = dz^T x  (out_features x in_features)     dbias = sum of dz's rows
 *   (the gradient of residual is dy itself).  dy, dx, dw row-major, of `type`; dbias out_features 32-bit
 *   floats; dx, dw and dbias may each be absent.  Of `op` the sizes, types and activation, x (unless dw is
 *   absent), w (unless dx is absent) and pre (unless the activation is NONE) are read.  dz is rounded to
 *   `type` where it becomes an operand of a product; dbias sums the unrounded values in a fixed order.
 *   rows = 0 gives zeros in dw and dbias.
 */
typedef struct redist_linear {
    int64_t rows, in_features, out_features;
    int32_t type, bias_type, activation, reserved;   /* reserved: 0 */
    redist_matrix x, w, residual, out, pre;
    const void *bias;
} redist_linear;

typedef struct redist_linear_grads {
    redist_matrix dy, dx, dw;
    float *dbias;
} redist_linear_grads;

size_t redist_linear_scratch_bytes(const redist_linear *op, const redist_linear_grads *grads); /* NULL: forward */
redist_status redist_linear_forward(const redist_linear *op, void *scratch, size_t scratch_bytes, void *cuda_stream);
redist_status redist_linear_backward(const redist_linear *op, const redist_linear_grads *grads, void *scratch,
                                     size_t scratch_bytes, void *cuda_stream);

/*
 * redist_layer_norm_forward -- y = (x - mean) rstd gamma + beta for every row, with mean and
 * rstd = 1 / sqrt(variance + eps) over the row (the variance is the mean squared difference from the mean).
 *
 *   rows >= 0, cols >= 1, eps >= 0
 *   type                 of x and y (and dy, dx): REDIST_BF16, REDIST_F16 or REDIST_F32
 *   x, y                 rows x cols, row-major
 *   gamma, beta          cols elements of weight_type (any), or NULL: 1 and 0
 *   mean, rstd           rows 32-bit floats each; the forward pass writes them (either may be NULL), the
 *                        backward pass reads them
 *
 * redist_layer_norm_backward -- with xh = (x - mean) rstd and c = dy gamma:
 *   dx = rstd (c - mean(c) - xh mean(c xh))     dgamma = sum of rows of dy xh     dbeta = sum of rows of dy
 *   dgamma and dbeta are cols 32-bit floats each, summed in a fixed order; either may be NULL.  y and beta
 *   are not read.  rows = 0 gives zeros in dgamma and dbeta.
 */
typedef struct redist_layer_norm {
    int64_t rows, cols;
    int32_t type, weight_type;
    float eps;
    int32_t reserved;                                 /* 0 */
    redist_matrix x, y;
    const void *gamma, *beta;
    float *mean, *rstd;
} redist_layer_norm;

typedef struct redist_layer_norm_grads {
    redist_matrix dy, dx;
    float *dgamma, *dbeta;
} redist_layer_norm_grads;

redist_status redist_layer_norm_forward(const redist_layer_norm *op, void *cuda_stream);
size_t redist_layer_norm_scratch_bytes(const redist_layer_norm *op, const redist_layer_norm_grads *grads);
redist_status redist_layer_norm_backward(const redist_layer_norm *op, const redist_layer_norm_grads *grads, void *scratch,
                                         size_t scratch_bytes, void *cuda_stream);

/*
 * redist_orthogonalize -- Newton-Schulz orthogonalisation of a stack of matrices, as the Muon optimiser
 * applies it to a momentum matrix: X <- X / (|X| + eps) (Frobenius norm), then per step, on the side on
 * which the Gram matrix is the smaller,
 *     A = X X^T,   X <- a X + (b A + c A A) X
 * and finally out = scale X.  The singular values move towards 1, the singular vectors stay.
 *
 *   batch, rows, cols >= 1;  1 <= steps <= 64;  eps >= 1e-30
 *   type            of x: REDIST_BF16, REDIST_F16 or REDIST_F32; out is REDIST_BF16
 *   x, out          row-major, matrix i at data + i * x_batch_stride (out_batch_stride) elements
 *   coefficients    host; steps triples (a, b, c), read during the call
 * The products run on 16-bit floats with 32-bit accumulation; X itself is carried from step to step in 22
 * bits, because small singular values grow by a factor of a per step and with them every error made in X.
 * How far results are off the exact iteration, in per cent of the norm (0.17 of it is the rounding of out), for the
 * coefficients of the Muon optimiser (3.4445, -4.7750, 2.0315) and five steps, the most seen in 64 matrices each (8 and 2 of the largest):
 *     min(rows, cols)                       1 to 4    8      16 to 32   64      128 and more
 *     Gaussian; low rank; one direction     0.7       0.45   0.32       0.26    0.22
 *     a part or all of the singular
 *     values equal, the rest noise          0.9       0.75   0.5        0.35    0.3
 * (equal singular values pass the same errors on, where others average), with sums of up to 2^18.  Longer ones lose more
 * in their 32-bit accumulation: 2^19 0.4, 2^20 0.6, 2^22 2.3.
 * Intermediates are scaled by powers of two found on the host from the coefficients; coefficients under
 * which a singular value could leave [0, 256] are refused (EINVAL).  A matrix with an infinity or NaN
 * gives NaN throughout, a zero matrix zeros.
 */
typedef struct redist_orthogonal {
    int64_t batch, rows, cols;
    int32_t type, steps;
    double eps;
    float scale;
    int32_t reserved;                                 /* 0 */
    redist_matrix x, out;
    int64_t x_batch_stride, out_batch_stride;
    const float *coefficients;
} redist_orthogonal;

size_t redist_orthogonalize_scratch_bytes(const redist_orthogonal *op);
redist_status redist_orthogonalize(const redist_orthogonal *op, void *scratch, size_t scratch_bytes, void *cuda_stream);

/* ---- a block of experts, and the bound on a step's gradients ------------------------------------ */

/*
 * A feed-forward layer whose weights are a set of experts of which every token uses a few: the router's choice and the order of
 * the rows, tokens moved to their experts' rows and back, and the linear layer with a weight per range of rows.  All sizes
 * are static (tokens * chosen rows, whatever the choice), only `offsets` and `position` depend on data and stay on the
 * device, so plans can move every array between shardings.  Rules and errors as above.
 *
 * redist_route_forward -- for every row of logits the `chosen` experts with the largest logits, in that order: equal ones by
 * the lower index, NaN before everything, minus infinity never (a row has empty places then; one of minus infinities only
 * goes nowhere).
 *
 *   tokens >= 0, 1 <= experts <= 1024, 1 <= chosen <= min(experts, 32), tokens * chosen < 2^31
 *   type            of logits (and dlogits): REDIST_BF16, REDIST_F16 or REDIST_F32
 *   logits          tokens x experts, row-major
 *   normalize       0: weights are softmax(logits) at the chosen experts; 1: softmax over the chosen ones only
 *   weights         tokens x chosen 32-bit floats, contiguous; 0 in empty places
 *   choice          tokens x chosen 32-bit integers: the expert; -1 in empty places
 *   position        tokens x chosen 32-bit integers: the row that this place gets when the rows are ordered by expert, within an
 *                   expert by token; -1 in empty places
 *   offsets         experts + 1 32-bit integers: rows offsets[e] ... offsets[e + 1] - 1 belong to expert e
 *
 * redist_route_backward -- the gradient of weights: with p = the softmax (0 outside the chosen with normalize) and s = sum over
 * the chosen of weight * dweight:  dlogits = p (dweight at chosen experts, 0 elsewhere, minus s).  What stands in dweights
 * at empty places does not count.  Of `op` the sizes, logits (unless normalize), weights and choice are read.
 */
typedef struct redist_route {
    int64_t tokens;
    int32_t experts, chosen, type, normalize;
    redist_matrix logits;
    float *weights;
    int32_t *choice, *position, *offsets;
} redist_route;

size_t redist_route_scratch_bytes(const redist_route *op);
redist_status redist_route_forward(const redist_route *op, void *scratch, size_t scratch_bytes, void *cuda_stream);
redist_status redist_route_backward(const redist_route *op, const float *dweights, const redist_matrix *dlogits, void *cuda_stream);

/*
 * redist_dispatch_forward, redist_combine_forward -- tokens to rows, and rows back to tokens:
 *   dispatch:  row[position[t, j]] = token[t]               combine:  token[t] = residual[t] + sum over j of weights[t, j] row[position[t, j]]
 * and their gradients:
 *   redist_dispatch_backward:  token[t] = sum over j of row[position[t, j]]   (row: the rows' gradient; token receives the tokens')
 *   redist_combine_backward:   drow[position[t, j]] = weights[t, j] token[t],  dweights[t, j] = <token[t], row[position[t, j]]>
 *                              (token: the output's gradient; that of residual is the same)
 *
 *   tokens, rows >= 0, 1 <= cols <= 33553920, 1 <= chosen <= 32
 *   type            of all matrices: REDIST_BF16, REDIST_F16 or REDIST_F32
 *   token, residual tokens x cols, row-major; residual may be absent, or `token` itself
 *   row, drow       rows x cols, row-major
 *   position        tokens x chosen 32-bit integers; a place outside 0 ... rows - 1 (as -1) is empty.  No row may be named twice
 *                   where rows are written (one of the two would win); rows that nobody names are left as they were
 *   weights         tokens x chosen 32-bit floats (dispatch: not read); dweights the same, 0 in empty places.  NULL in
 *                   redist_combine_forward: all 1
 * Sums are in 32 bits in the order of the places, each output is rounded once; dweights' sums have a fixed order.
 */
typedef struct redist_move {
    int64_t tokens, rows, cols;
    int32_t type, chosen;
    redist_matrix token, row, residual, drow;
    const int32_t *position;
    const float *weights;
    float *dweights;
} redist_move;

redist_status redist_dispatch_forward(const redist_move *op, void *cuda_stream);
redist_status redist_dispatch_backward(const redist_move *op, void *cuda_stream);
redist_status redist_combine_forward(const redist_move *op, void *cuda_stream);
redist_status redist_combine_backward(const redist_move *op, void *cuda_stream);

/*
 * redist_experts_forward -- the linear layer with a weight per range of rows: for offsets[e] <= r < offsets[e + 1]
 *   out[r] = activation(x[r] w[e]^T + bias[e])
 * Rows before offsets[0] and from offsets[experts] on are neither read for nor written to any output.
 *
 *   rows >= 0, in_features >= 1, out_features >= 1, 1 <= experts <= 65535
 *   type            REDIST_BF16 or REDIST_F16: x, w, out and pre
 *   x               rows x in_features, row-major
 *   w               experts matrices out_features x in_features, all row-major or all column-major, w_stride elements apart
 *   bias            experts vectors of out_features elements of bias_type (any), bias_stride elements apart, or NULL
 *   out, pre        rows x out_features, row-major; pre may be absent: receives z = x w^T + bias for the backward pass
 *   offsets         device; experts + 1 32-bit integers, not decreasing, 0 ... rows.  Others give results that are not defined, but
 *                   nothing outside the arrays is touched
 *
 * redist_experts_backward -- the gradients.  With dz = dy activation'(pre), over the rows of expert e:
 *   dx[r] = dz[r] w[e]     dw[e] = sum of dz[r]^T x[r]     dbias[e] = sum of dz[r]
 *   dy, dx row-major, dw a stack as w (row-major, dw_stride apart), all of `type`; dbias experts x out_features 32-bit floats,
 *   contiguous; dx, dw and dbias may each be absent.  Experts without rows get zeros in dw and dbias.  Of `op` the
 *   sizes, types, activation and offsets, x (unless dw is absent), w (unless dx is absent) and pre (unless the activation is NONE)
 *   are read.  Accumulation and roundings as in the linear layer; dbias sums the unrounded values in a fixed order.
 */
typedef struct redist_experts {
    int64_t rows, in_features, out_features;
    int32_t experts, type, bias_type, activation;
    redist_matrix x, w, out, pre;
    int64_t w_stride, bias_stride;
    const void *bias;
    const int32_t *offsets;
} redist_experts;

typedef struct redist_experts_grads {
    redist_matrix dy, dx, dw;
    int64_t dw_stride;
    float *dbias;
} redist_experts_grads;

size_t redist_experts_scratch_bytes(const redist_experts *op, const redist_experts_grads *grads); /* NULL: forward */
redist_status redist_experts_forward(const redist_experts *op, void *scratch, size_t scratch_bytes, void *cuda_stream);
redist_status redist_experts_backward(const redist_experts *op, const redist_experts_grads *grads, void *scratch,
                                      size_t scratch_bytes, void *cuda_stream);

/*
 * redist_clip -- the norm over all elements of a list of tensors, |g| = sqrt(sum of g^2), and the tensors times
 * min(1, max_norm / (|g| + eps)).
 *
 *   tensors         host; count entries, read during the call: data (contiguous, of type, at any element boundary) and out, which
 *                   receives the product (NULL or data itself: in place; tensors then stay untouched where the factor is 1).
 *                   Empty tensors are allowed
 *   max_norm        >= 0, or negative: the norm only (out is not written)
 *   eps             >= 0 (1e-6 is usual)
 *   norm            device; one 32-bit float, or NULL
 * Squares are summed in a fixed order and without overflow or underflow for every finite input (64 bits where 32 would not
 * hold them).  The factor follows the formula for all inputs, also where 32 bits hold neither it nor the norm (of which `norm`
 * receives infinity then): an infinite element gives 0 (and NaN where it stands), a NaN gives NaN throughout.  Errors: also EUNSUPPORTED for more than 2^40 elements in a tensor.
 */
typedef struct redist_tensor {
    void *data, *out;
    int64_t elements;
    int32_t type, reserved;                           /* reserved: 0 */
} redist_tensor;

typedef struct redist_clip_op {
    const redist_tensor *tensors;
    int64_t count;
    float max_norm, eps;
    float *norm;
} redist_clip_op;

size_t redist_clip_scratch_bytes(const redist_clip_op *op);
redist_status redist_clip(const redist_clip_op *op, void *scratch, size_t scratch_bytes, void *cuda_stream);

/*
 * redist_product_timeouts -- health counter of the matrix products, as redist_bulk_timeouts is of the bulk
 * copies: thread blocks whose bounded wait ("wait_polls") ran out on the current device.  Such a block
 * leaves its tiles unwritten and returns, although the call has returned REDIST_OK.  0 in a healthy run; -1 on a CUDA error.
 * Synchronizes the device.
 */
int64_t redist_product_timeouts(void);

#ifdef __cplusplus
}
#endif
#endif /* REDIST_H_ */
