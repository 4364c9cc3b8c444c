/*
 * sllm.h — C ABI of the MI355X checkpoint loader.
 *
 * The library converts a tensor checkpoint into a loading-optimized format
 * and streams it from pinned host DRAM into one preallocated HBM buffer
 * (ServerlessLLM, Sec. 4, fast multi-tier checkpoint loading).  Operators on
 * the loaded weights (4-bit matrices and products with them, embeddings) stand
 * at the end.
 *
 * Format (Sec. 4.1).  A checkpoint directory holds two files:
 *   sllm.part0  the partition for one GPU: the tensors' bytes only, in the
 *               caller's order, each at an offset aligned to A (a power of
 *               two), zero padding between tensors, zero-filled up to
 *               F = align_up(T, 4096) bytes, where T = sum align_up(s_i, A).
 *   sllm.index  the tensor index: name -> (dtype, shape, partition, offset,
 *               size), little-endian, closed by a CRC-32 (IEEE).  The exact
 *               byte layout is in docs/FORMAT.md.
 * A tensor's device address is base + offset (Sec. 4.1, direct tensor
 * addressing).
 *
 * Loading (Sec. 4.2).  Chunk k of a partition is the byte range
 * [kC, min(kC + C, T)).  Chunks move through a pool of fixed-size pinned host
 * chunks (the DRAM tier, with allocate/evict calls under application control)
 * and from there into device memory, either by the copy (SDMA) engines or by
 * a gfx950 kernel that reads the mapped host chunks directly.
 *
 * Conventions.
 *   - Every call returns an int32_t status: SLLM_OK (0) or a negative
 *     SLLM_E_* code; sllm_last_error() then gives a message for this thread.
 *   - No C++ exception crosses this interface.
 *   - "Device pointer" means an address in the HIP device's memory (for
 *     example a torch uint8 CUDA tensor's data_ptr()); "stream" is a
 *     hipStream_t passed as void* (NULL = the null stream).
 *   - The caller owns every buffer and stream it passes in.  The library
 *     owns its handles and everything reachable from them until the matching
 *     close/destroy call.
 *   - A handle may be used by one thread at a time; different handles may
 *     be used from different threads.
 *   - Copy streams (and their fork/join events) outlive the handles that
 *     used them: a closed handle leaves its idle streams to the next handle
 *     on the same device (at most 32 sets per process, kept until the
 *     process ends), so opening a handle per load costs no stream creation.
 *     A caller that resets a device must not use the library afterwards.
 *   - The device tables and HBM staging of a handle with a dev_alignment go
 *     back to the library at close and stay idle for the next handle (at most
 *     256 MiB in 32 blocks per device; the oldest are freed beyond that, and
 *     all of them when a handle's allocation finds no memory).
 *   - A load or repack may be captured into a HIP graph; the handle must stay
 *     open while the graph is replayed.  The device tables and staging of a
 *     handle used that way are freed at close, which waits for the device and
 *     so for replays under way.
 *   - Reader threads outlive the loads that start them: a finished reader
 *     waits idle (at most 64 per process, until the process ends) for the
 *     next load or pool fill, which then wakes it instead of starting a
 *     thread.
 *
 * Environment (read by the library; none is needed for normal use).
 *   SLLM_LOG_LEVEL        0 quiet (default), 1 info, 2 debug, on stderr.
 *   SLLM_TRACE_FILE       streamed loads append each chunk's read, move and
 *                         done times to this CSV file.
 *   SLLM_ROCTX=1          host stages become roctx ranges (rocprofv3
 *                         --marker-trace); the roctx library is loaded then.
 *   SLLM_READ_STREAM=0    buffered chunks are read straight into pinned
 *                         memory (default: through a 1 MiB per-thread buffer
 *                         copied on with streaming stores, so that the GPU
 *                         reads them from DRAM, not from dirty CPU caches).
 *   SLLM_READ_MAPPED=1    buffered files are mapped and chunks copied with
 *                         streaming stores instead of read with pread.
 *   SLLM_BATCH_TARGET_MB  bytes a streamed gather batch collects (64).
 *   SLLM_SPLIT_CHUNKS     leading chunks of a streamed load that all readers
 *                         read together in pieces (one per I/O thread; 0
 *                         reads every chunk whole).
 *   SLLM_IDLE_WORKERS     idle reader threads kept for later loads (64; 0
 *                         starts every reader on a new thread).
 *   SLLM_SDMA_MAX_COPY_MB largest merged copy-engine copy of cached chunks (256).
 *   SLLM_POOL_ARENA_MB    size of each pinned allocation a pool is cut from (1024).
 *   SLLM_K1_BLOCKS, SLLM_K1_STREAM_BLOCKS, SLLM_K1_UNROLL, SLLM_K1_NT,
 *   SLLM_K2_NT, SLLM_K2_MAX_GRID, SLLM_K2_UNROLL, SLLM_NOALLOC_PLAN_BLOCKS
 *                         kernel launch shapes, read at every launch (for
 *                         measurements and tests; the defaults are tuned, some
 *                         by the size of the image).
 */
#ifndef SLLM_H
#define SLLM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes -------------------------------------------------------- */
#define SLLM_OK          0
#define SLLM_E_INVAL    -1  /* bad argument or option                           */
#define SLLM_E_IO       -2  /* a file could not be opened, read or written      */
#define SLLM_E_FORMAT   -3  /* index or partition damaged or inconsistent       */
#define SLLM_E_NOMEM    -4  /* host or pool memory exhausted                    */
#define SLLM_E_HIP      -5  /* a HIP runtime call failed                        */
#define SLLM_E_RANGE    -6  /* destination buffer too small                     */
#define SLLM_E_BUSY     -7  /* object in use (load in progress, cached, opened) */
#define SLLM_E_NOTFOUND -8  /* no such tensor / checkpoint                      */

/* ---- dtypes (stored bytes are never converted) ---------------------------- */
#define SLLM_DTYPE_F32  0
#define SLLM_DTYPE_F16  1
#define SLLM_DTYPE_BF16 2
#define SLLM_DTYPE_I8   3
#define SLLM_MAX_NDIM   8

/* =========================================================================
 * Conversion (Sec. 4.1: checkpoints are converted once, loaded many times)
 * ========================================================================= */

/* One tensor of the source checkpoint.  `data` holds `nbytes` raw
 * little-endian bytes, and nbytes must equal prod(shape) * itemsize(dtype)
 * (a 0-d tensor has one element).  `name` is non-empty UTF-8 of at most
 * 65535 bytes, unique within the checkpoint. */
typedef struct sllm_src_tensor {
    const char*    name;
    uint32_t       dtype;   /* SLLM_DTYPE_* */
    uint32_t       ndim;    /* 0 .. SLLM_MAX_NDIM */
    const int64_t* shape;   /* ndim entries, each >= 0 (may be NULL if ndim == 0) */
    const void*    data;    /* host memory; may be NULL if nbytes == 0 */
    uint64_t       nbytes;
} sllm_src_tensor;

#define SLLM_CONVERT_FSYNC 1u   /* fsync both files before returning */

typedef struct sllm_convert_opts {
    uint64_t alignment;   /* A: power of two >= 1; 0 means 256            */
    uint64_t chunk_size;  /* default load chunk size C >= 1; 0 means 16 MiB */
    uint32_t flags;       /* SLLM_CONVERT_*                                */
    uint32_t reserved;    /* must be 0                                     */
} sllm_convert_opts;

/* Write out_dir/sllm.part0 and out_dir/sllm.index for the n tensors, in the
 * given order (out_dir must exist).  opts may be NULL (A = 256, C = 16 MiB).
 * The caller's tensor memory is only read during the call.  Existing files
 * are replaced; on error both files are removed.
 * Errors: INVAL (bad tensor or option; duplicate or empty name), IO. */
int32_t sllm_convert(const sllm_src_tensor* tensors, uint64_t n,
                     const char* out_dir, const sllm_convert_opts* opts);

/* Streaming form of sllm_convert for checkpoints that do not fit in host
 * memory twice: tensors are added one at a time and written immediately.
 * The files it produces are byte-identical to sllm_convert's.
 * sllm_writer_close writes the index and frees the writer (even on error);
 * sllm_writer_abort removes the partial files and frees the writer.
 * Errors: as sllm_convert; after a failed sllm_writer_add the writer only
 * accepts sllm_writer_abort or sllm_writer_close (which then removes the
 * files and returns the error). */
typedef struct sllm_writer sllm_writer;
int32_t sllm_writer_open(const char* out_dir, const sllm_convert_opts* opts,
                         sllm_writer** out);
int32_t sllm_writer_add(sllm_writer* w, const sllm_src_tensor* tensor);
int32_t sllm_writer_close(sllm_writer* w);
void    sllm_writer_abort(sllm_writer* w);

/* Convert safetensors shards (the format Hugging Face checkpoints ship in)
 * straight into out_dir: every tensor of every shard, in shard order and,
 * within a shard, in the order its bytes sit in the file, so each shard is
 * read front to back once.  Supported dtypes: F32, F16, BF16, I8.
 * Errors: INVAL (another dtype, more than 8 dimensions, a name repeated
 * across shards), IO, FORMAT (malformed header, data outside the file,
 * overlapping tensors, size != numel * itemsize).  On error no files remain. */
int32_t sllm_convert_safetensors(const char* const* paths, uint64_t n_paths, const char* out_dir,
                                 const sllm_convert_opts* opts);

/* =========================================================================
 * Pinned host chunk pool: the DRAM tier (Sec. 4.2, chunk-based data
 * management: fixed-size chunks, allocation and eviction under the
 * application's control)
 * ========================================================================= */

typedef struct sllm_pool sllm_pool;

/* Allocate n_chunks pinned, device-mapped host chunks of chunk_size bytes
 * (>= 1) for HIP device `device`.  Every chunk starts on a 4 KiB boundary
 * (chunks sit align_up(chunk_size, 4096) bytes apart), so direct file reads
 * can land in them.  Allocation is slow (pages are pinned); do it once,
 * outside the load path.
 * Errors: INVAL, HIP (pinned allocation failed). */
int32_t sllm_pool_create(uint64_t chunk_size, uint64_t n_chunks, int32_t device,
                         sllm_pool** out);

/* Free the pool.  BUSY while an open checkpoint handle still uses it. */
int32_t sllm_pool_destroy(sllm_pool* pool);

typedef struct sllm_pool_info {
    uint64_t chunk_size;
    uint64_t n_chunks;
    uint64_t free_chunks;
    uint64_t cached_checkpoints;
} sllm_pool_info;
/* Sizes and occupancy of the pool.  Errors: INVAL (NULL argument). */
int32_t sllm_pool_query(const sllm_pool* pool, sllm_pool_info* out);

/* Read the whole partition of checkpoint directory `dir` into pool chunks,
 * where it stays (cached in DRAM) until sllm_pool_evict.  Loads of handles
 * opened on this pool then copy from these chunks with no file I/O.
 * io_threads = 0 means 4.  flags: SLLM_OPEN_DIRECT_IO.
 * Errors: INVAL, IO, FORMAT, NOMEM (not enough free chunks), BUSY (already
 * cached).  The checkpoint is identified by the data file's device, inode,
 * size and modification time. */
int32_t sllm_pool_cache(sllm_pool* pool, const char* dir, uint32_t io_threads,
                        uint32_t flags);

/* Return a cached checkpoint's chunks to the pool.  NOTFOUND if not cached,
 * BUSY while an open handle loads from it. */
int32_t sllm_pool_evict(sllm_pool* pool, const char* dir);

/* =========================================================================
 * Open / load / index (Sec. 4.1 direct tensor addressing; Sec. 4.2 loading)
 * ========================================================================= */

#define SLLM_ENGINE_KERNEL 0u   /* gfx950 kernel reads mapped host chunks      */
#define SLLM_ENGINE_SDMA   1u   /* hipMemcpyAsync on the copy engines          */

#define SLLM_OPEN_DIRECT_IO 1u  /* O_DIRECT file reads (buffered if the file
                                   system refuses them; see stats.direct_io) */
#define SLLM_OPEN_TIMING    2u  /* time device work with HIP events (stats)   */
#define SLLM_OPEN_INDEX_ONLY 4u /* read and validate the index only: no data
                                   file, pool or device work; for processes
                                   that view a buffer another process loaded
                                   (sllm_load then returns SLLM_E_INVAL)      */
#define SLLM_OPEN_CACHE     8u  /* keep what the first load reads: it streams
                                   the file (storage -> pinned -> HBM,
                                   pipelined) into ceil(T/C) chunks of
                                   opts->pool, one per chunk, and once it has
                                   succeeded those chunks become the pool's
                                   cached copy of the checkpoint (the DRAM
                                   tier, Sec. 4.2), as after sllm_pool_cache.
                                   Needs a pool whose chunk size is C; NOMEM
                                   if it lacks free chunks.  No effect when
                                   the checkpoint is cached already.        */

typedef struct sllm_open_opts {
    uint64_t   chunk_size;     /* C for reads from the file; 0 = pool's chunk
                                  size if a pool is given, else the index's */
    uint64_t   dev_alignment;  /* 0: device layout = file layout.  Else A2, a
                                  power of two >= 16: tensor i goes to
                                  d_i = sum_{j<i} align_up(s_j, A2), zero
                                  padded, T2 = sum align_up(s_i, A2) bytes */
    sllm_pool* pool;           /* NULL: a private pool of ring_slots chunks
                                  is allocated by sllm_open                 */
    uint32_t   io_threads;     /* file-reading threads; 0 = 4               */
    uint32_t   n_streams;      /* copy streams for the SDMA engine; 0 = 2   */
    uint32_t   ring_slots;     /* chunks in flight when streaming from the
                                  file; 0 = 2 * io_threads                  */
    uint32_t   engine;         /* SLLM_ENGINE_*                             */
    uint32_t   flags;          /* SLLM_OPEN_*                               */
    int32_t    device;         /* HIP device ordinal                        */
} sllm_open_opts;

typedef struct sllm_ckpt sllm_ckpt;

/* Read and validate dir/sllm.index (magic, version, CRC, unique names,
 * sizes = numel * itemsize, aligned ordered non-overlapping offsets,
 * T = padded sum, file length F) and open dir/sllm.part0.  If `opts->pool`
 * caches this checkpoint, later loads copy from the cached chunks; else they
 * stream the file through ring_slots pool chunks.  opts may be NULL
 * (defaults above, device 0).  With a dev_alignment the handle keeps device
 * tables of 24 bytes per tensor plus 8 bytes per 16 KiB of the device image
 * (the repack kernel's plan), built here.
 * Errors: INVAL (also: direct reads where the chunk size or the padded file
 * length F is not a multiple of the file's direct-I/O alignment), IO,
 * FORMAT, NOMEM, HIP. */
int32_t sllm_open(const char* dir, const sllm_open_opts* opts, sllm_ckpt** out);

/* Bytes a load writes: T (file layout) or T2 (dev_alignment != 0); 0 for a
 * NULL handle. */
uint64_t sllm_total_bytes(const sllm_ckpt* h);

/* Load the checkpoint into device memory [dev_dst, dev_dst + total_bytes).
 * dev_dst must be 16-byte aligned.  All of [0, total) is written, padding
 * included (as zero); bytes past it are untouched.  Returns once every file
 * read has finished and every copy or kernel has been enqueued; completion is
 * ordered on `stream`: work queued there after this call sees every byte.
 * Errors: INVAL (dev_dst is not device memory of the handle's device, is
 * memory whose allocation range the runtime cannot report, or is not
 * 16-byte aligned), RANGE (dst_bytes < total, or the range runs past the
 * end of dev_dst's allocation), IO, HIP, BUSY (another load on this
 * handle).  On error, in-flight work is drained and the destination's
 * contents are unspecified; the handle stays usable. */
int32_t sllm_load(sllm_ckpt* h, void* dev_dst, uint64_t dst_bytes, void* stream);

/* On-device repack of a file-layout image into the device layout: src holds
 * the partition's first T bytes (as sllm_load writes them with
 * dev_alignment = 0) and dst receives T2 bytes laid out with the handle's
 * dev_alignment.  src and dst are device pointers, 16-byte aligned, and must
 * not overlap.  Enqueued on `stream`.
 * Errors: INVAL (handle opened without dev_alignment, overlap, a buffer that
 * is not device memory of the handle's device or whose allocation range the
 * runtime cannot report), RANGE, HIP. */
int32_t sllm_repack(const sllm_ckpt* h, const void* src_dev, uint64_t src_bytes,
                    void* dst_dev, uint64_t dst_bytes, void* stream);

/* sllm_repack for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same result, byte for byte, with no hipMalloc, hipFree or other
 * allocation.  Its device tables (sizes, file and device offsets, and the
 * repack plan for one window of the destination at a time) live in a fixed
 * library area of SLLM_NOALLOC_SCRATCH_BYTES per device, which each device
 * holds from the library's first kernel launch on it until the process
 * ends.  The sizes travel as kernel arguments; every table is rewritten by
 * each call, so nothing carries over between calls.
 *   h              any open handle, INDEX_ONLY included (its index gives the
 *                  layout); it may have been opened without a dev_alignment
 *   dev_alignment  A2, a power of two >= 16; 0 means the handle's own
 *   src_dev        the file-layout image, T = sllm_total_bytes of an
 *                  unaligned handle; src_bytes >= T
 *   dst_dev        receives T2 = sum align_up(s_i, A2) bytes; dst_bytes >= T2
 * Buffers are device memory of the handle's device, 16-byte aligned, and do
 * not overlap.  Enqueued on `stream`; the call returns without waiting.
 * Calls that overlap on one device (different streams or threads, or one
 * stream while another call's kernels still run elsewhere) race for the
 * area: order them, for example on one stream.
 * Errors: INVAL (no or bad alignment, overlap, a buffer that is not device
 * memory of the handle's device), RANGE (a buffer too small, or more than
 * SLLM_NOALLOC_MAX_TENSORS tensors), HIP. */
#define SLLM_NOALLOC_SCRATCH_BYTES (16ull << 20)
#define SLLM_NOALLOC_MAX_TENSORS   65536ull
int32_t sllm_repack_noalloc(const sllm_ckpt* h, uint64_t dev_alignment, const void* src_dev,
                            uint64_t src_bytes, void* dst_dev, uint64_t dst_bytes, void* stream);

/* One tensor of the index.  `offset` is relative to the device buffer:
 * the file offset o_i, or d_i when the handle has a dev_alignment.  `name`
 * stays valid until sllm_close. */
typedef struct sllm_tensor_info {
    const char* name;
    uint32_t    dtype;
    uint32_t    ndim;
    int64_t     shape[SLLM_MAX_NDIM];
    uint64_t    offset;
    uint64_t    nbytes;
} sllm_tensor_info;

/* Copy up to `cap` entries, in layout order, into out[] and set *n_total to
 * the number of tensors (cap = 0 with out = NULL asks for the count only).
 * Errors: INVAL (NULL handle, or out NULL with cap > 0). */
int32_t sllm_tensor_index(const sllm_ckpt* h, sllm_tensor_info* out, uint64_t cap,
                          uint64_t* n_total);

/* Look one tensor up by name.  Errors: INVAL (NULL argument), NOTFOUND. */
int32_t sllm_tensor_find(const sllm_ckpt* h, const char* name, sllm_tensor_info* out);

typedef struct sllm_stats {
    uint64_t bytes_loaded;      /* bytes written to the device by the last load  */
    uint64_t bytes_read;        /* bytes read from the file by the last load     */
    uint64_t n_chunks;          /* chunks moved by the last load                 */
    uint64_t n_launches;        /* kernel launches or copy calls of the last load */
    uint32_t engine;            /* engine used                                   */
    uint32_t direct_io;         /* 1 if the file is read with O_DIRECT           */
    uint32_t from_cache;        /* 1 if the last load came from cached chunks    */
    uint32_t io_threads;
    double   open_s;            /* wall time of sllm_open                        */
    double   load_s;            /* wall time of the last sllm_load call          */
    double   read_wait_s;       /* time the issue loop waited for file reads     */
    double   device_ms;         /* device time of the last load (TIMING flag), else -1 */
    uint64_t bytes_bounced;     /* direct-read bytes staged through a bounce buffer
                                   because the kernel refused direct transfers
                                   into the pinned chunks                      */
    double   reader_busy_s;     /* streamed loads: I/O-thread time spent reading
                                   (summed over threads)                       */
    double   reader_starved_s;  /* streamed loads: I/O-thread time spent waiting
                                   for a free slot (summed over threads)       */
} sllm_stats;
/* Counters of the handle's last load.  With SLLM_OPEN_TIMING this waits for
 * that load's device work to finish (to read its events).  Errors: INVAL, HIP. */
int32_t sllm_get_stats(const sllm_ckpt* h, sllm_stats* out);

/* =========================================================================
 * Handoff to another process (Sec. 4.1: the model manager loads, the
 * inference process receives the GPU base address as an IPC handle, computes
 * base + offset from the index and synchronizes with the manager)
 * ========================================================================= */

typedef struct sllm_ipc_desc {
    uint8_t  mem_handle[64];    /* IPC handle of the allocation holding the buffer */
    uint8_t  event_handle[64];  /* IPC handle of an event recorded after the load  */
    uint64_t offset;            /* start of the buffer inside that allocation      */
    uint64_t bytes;             /* length of the buffer                            */
    int32_t  device;
    uint32_t flags;             /* SLLM_IPC_*                                      */
} sllm_ipc_desc;

/* event_handle is valid: the importer's stream waits for it on the device.
 * Without it the exporter finished the load before filling the descriptor
 * (the runtime offers no interprocess events), and the importer waits for
 * nothing. */
#define SLLM_IPC_HAS_EVENT 1u

/* Largest allocation this library shares across processes: opening handles
 * of larger allocations does not complete on the MI355X systems it was
 * tested on, so export refuses them. */
#define SLLM_IPC_MAX_ALLOCATION ((2ull << 30) - 1)

typedef struct sllm_export sllm_export;
typedef struct sllm_import sllm_import;

/* Share [dev_ptr, dev_ptr + bytes) (inside one device allocation of at most
 * SLLM_IPC_MAX_ALLOCATION bytes) with other processes: fills *desc (plain
 * bytes, safe to send through a pipe or file) and records the handoff event
 * on `stream`, after the work already queued there (typically sllm_load).
 * Where the runtime has no interprocess events, it instead waits for that
 * work to finish and leaves SLLM_IPC_HAS_EVENT clear.
 * Keep the export alive while importers use the buffer.
 * Errors: INVAL (not device memory, allocation too large, range outside it), HIP. */
int32_t sllm_export_create(const void* dev_ptr, uint64_t bytes, int32_t device, void* stream,
                           sllm_ipc_desc* desc, sllm_export** out);
/* Release the export (its handoff event); importers must have closed their
 * mappings.  NULL is a no-op.  Always returns SLLM_OK. */
int32_t sllm_export_destroy(sllm_export* ex);

/* Map an exported buffer into this process: *dev_ptr is its start here, and
 * `stream` waits (on the device) for the exporter's handoff event, so work
 * queued on it afterwards sees the loaded bytes.  Errors: INVAL (unknown
 * flags, or offset + bytes past the end of the mapped allocation: nothing
 * stays mapped), HIP. */
int32_t sllm_import_open(const sllm_ipc_desc* desc, void* stream, void** dev_ptr, sllm_import** out);
/* Unmap; work that reads the buffer must have finished.  NULL is a no-op.
 * Errors: HIP (the mapping could not be closed; the import is freed anyway). */
int32_t sllm_import_close(sllm_import* im);

/* =========================================================================
 * Loading-time estimate (Sec. 6, estimating model loading time): a load of
 * n bytes queued behind other loads on this server finishes after q + n / b,
 * where q sums the estimates of the loads already queued (loads run one at a
 * time per server) and b is the bandwidth of the slowest tier the load
 * crosses (the tiers are pipelined).  Measured load times refine b.
 * Host-only; no device work.
 * ========================================================================= */

#define SLLM_TIER_DRAM    1u  /* pinned host DRAM -> HBM        */
#define SLLM_TIER_STORAGE 2u  /* local file -> pinned host DRAM */

typedef struct sllm_estimator sllm_estimator;

/* Initial bandwidths in bytes per second (> 0) and the weight in (0, 1] of a
 * new measurement in the running estimate (1 = keep only the latest).
 * Errors: INVAL, NOMEM. */
int32_t sllm_estimator_create(double dram_bytes_per_s, double storage_bytes_per_s, double weight,
                              sllm_estimator** out);
void    sllm_estimator_destroy(sllm_estimator* e);

/* q + n / b for a load of `bytes` crossing `tiers` (SLLM_TIER_* bits),
 * queued behind every load enqueued and not yet completed.  Errors: INVAL
 * (NULL argument, no or unknown tier bits). */
int32_t sllm_estimator_query(const sllm_estimator* e, uint64_t bytes, uint32_t tiers, double* eta_s);

/* Queue such a load: *eta_s is its estimate (as for query) and *task its id;
 * its own n / b joins q for the loads queued after it. */
int32_t sllm_estimator_enqueue(sllm_estimator* e, uint64_t bytes, uint32_t tiers, uint64_t* task,
                               double* eta_s);

/* The task's load took `seconds`: bytes / seconds updates the bandwidth of
 * its slowest tier and the task leaves the queue.  NOTFOUND for an unknown
 * task, INVAL for seconds <= 0. */
int32_t sllm_estimator_complete(sllm_estimator* e, uint64_t task, double seconds);

/* sllm_estimator_complete with the time the handle's last load took, from
 * its own counters (sllm_get_stats): open_s plus load_s, or plus the device
 * time of the load when the handle was opened with SLLM_OPEN_TIMING and that
 * is longer (a load from cached chunks returns once its work is enqueued,
 * so only the device time covers it).  With timing on, this waits for the
 * load's device work.  Errors: INVAL (NULL argument, nothing loaded yet),
 * NOTFOUND, HIP. */
int32_t sllm_estimator_complete_load(sllm_estimator* e, uint64_t task, const sllm_ckpt* h);

/* Current bandwidth estimate of one tier (bytes per second).  Errors: INVAL. */
int32_t sllm_estimator_bandwidth(const sllm_estimator* e, uint32_t tier, double* bytes_per_s);

/* Close the handle; waits for its in-flight device work first (the copy
 * streams' and, on the caller's streams, that of every load and repack the
 * handle enqueued), so that the pool chunks and device tables that work
 * reads may be reused as soon as it returns.  NULL is a no-op.
 * Errors: BUSY (a load is running on the handle). */
int32_t sllm_close(sllm_ckpt* h);

/* =========================================================================
 * Operators on loaded weights: matrices held in microscaled 4-bit floating
 * point (MX FP4), products with them, token embeddings, and what a decoder
 * layer has around them: norms and attention
 *
 * Every operator is enqueued on `stream` and returns without waiting; it
 * allocates nothing (a workspace, where one is needed, is the caller's) and may
 * be captured into a HIP graph.  Two calls may overlap if neither writes what
 * the other uses, workspaces included.  The same inputs give the same bytes.
 *
 * Buffers are memory of HIP device `device`, each inside one allocation.  An
 * output overlaps no other buffer of its call, a buffer being all from its first
 * byte to its last, with what lies between its rows.  A buffer of no bytes may be
 * NULL.  Sums are held in 32-bit floats and rounded once, to nearest even, to
 * the output's type.
 *
 * Errors of all of them: INVAL (NULL or inconsistent argument, a dtype other
 * than F32, F16 and BF16, sizes that do not fit together, a pointer that is
 * not aligned, not device memory or overlaps), RANGE (a buffer that runs past
 * the end of its allocation, a workspace too small, rows or columns of more
 * than SLLM_MAX_EXTENT), HIP.
 * ========================================================================= */

#define SLLM_MAX_EXTENT 0x7fff0000ull

/* A matrix in device memory, aligned to its element type: row r starts at
 * data + r * stride elements and its elements are adjacent. */
typedef struct sllm_matrix {
    void*    data;
    uint64_t rows;
    uint64_t cols;
    uint64_t stride;    /* elements, >= cols (any value for one row or none) */
    uint32_t dtype;     /* SLLM_DTYPE_F32, _F16 or _BF16 */
    uint32_t reserved;  /* must be 0 */
} sllm_matrix;

/* A matrix in MX FP4 (the OCP Microscaling formats' MXFP4): each row is cut
 * into blocks of 32 columns, the last one padded with zeros, and a block is one
 * E8M0 scale s (2^(s - 127); 255 makes the whole block NaN) and 32 E2M1 codes
 * (sign bit and 0, 0.5, 1, 1.5, 2, 3, 4, 6).  With blocks = ceil(cols / 32):
 *   codes   rows * blocks * 16 bytes; a block's column 2 i is the low half of
 *           its byte i and column 2 i + 1 the high half
 *   scales  rows * align_up(blocks, 16) bytes, the bytes past a row's blocks
 *           zero
 * Both are 16-byte aligned.  Rows are adjacent, so a run of rows is such a
 * matrix too. */
typedef struct sllm_mx {
    void*    codes;
    void*    scales;
    uint64_t rows;
    uint64_t cols;
} sllm_mx;

/* Token ids in device memory.  An id outside [0, table rows) names no row. */
typedef struct sllm_ids {
    const void* data;
    uint64_t    n;
    uint32_t    bits;      /* 32 or 64: signed, aligned to their size */
    uint32_t    reserved;  /* must be 0 */
} sllm_ids;

/* Bytes of the two buffers of a rows x cols matrix in MX FP4.  Host-only.
 * Errors: INVAL, RANGE. */
int32_t sllm_mx_sizes(uint64_t rows, uint64_t cols, uint64_t* codes_bytes, uint64_t* scales_bytes);

/* dst = src in MX FP4.  A block's scale is 2^(floor(log2 a) - 2), a its largest
 * magnitude, at least 2^-127 (and 2^-127 where a = 0); its elements divided by
 * the scale go to the nearest E2M1 value, ties to the even code, magnitudes
 * above 6 to 6.  A block with an infinity or a NaN gets scale 255 and codes 0. */
int32_t sllm_mx_quantize(const sllm_matrix* src, const sllm_mx* dst, int32_t device, void* stream);

/* dst = the values src stands for, rounded to dst's type. */
int32_t sllm_mx_dequantize(const sllm_mx* src, const sllm_matrix* dst, int32_t device, void* stream);

/* out = x * transpose(w): x has m rows of k elements, w is n x k, out m x n.
 * The products of x's elements, in their own type, with the values w stands
 * for are not rounded before they are summed; elements of x below 2^-110 in
 * magnitude count to within 2^-133. */
int32_t sllm_mx_linear(const sllm_matrix* x, const sllm_mx* w, const sllm_matrix* out, void* workspace,
                       uint64_t workspace_bytes, int32_t device, void* stream);

/* The same with x in MX FP4 too. */
int32_t sllm_mx_linear_mx(const sllm_mx* x, const sllm_mx* w, const sllm_matrix* out, void* workspace,
                          uint64_t workspace_bytes, int32_t device, void* stream);

/* dx = dy * w, the gradient of sllm_mx_linear by x, with the same sums: dy has
 * m rows of n elements, w is n x k, dx m x k. */
int32_t sllm_mx_linear_grad(const sllm_matrix* dy, const sllm_mx* w, const sllm_matrix* dx, void* workspace,
                            uint64_t workspace_bytes, int32_t device, void* stream);

/* The same with x in MX FP8 (see sllm_mx_octet_quantize).  Where out is in 16 bits, products
 * of eight neighbouring elements of x are added to within 2^-13 of the largest of them
 * each, and those sums in 32 bits; where it is F32, elements of x below 2^-126 count to within 2^-134,
 * and nothing is rounded before the sums in 32 bits. */
int32_t sllm_mx_linear_octet(const sllm_mx* x, const sllm_mx* w, const sllm_matrix* out, void* workspace,
                           uint64_t workspace_bytes, int32_t device, void* stream);

/* Workspace each of these needs for these operands (their data pointers'
 * alignment counts, the memory is not read); 0 means none, and workspace may
 * then be NULL.  A workspace is 16-byte aligned; its contents do not matter and
 * are overwritten.  Host-only. */
int32_t sllm_mx_linear_workspace(const sllm_matrix* x, const sllm_mx* w, uint64_t* bytes);
int32_t sllm_mx_linear_mx_workspace(const sllm_mx* x, const sllm_mx* w, uint64_t* bytes);
int32_t sllm_mx_linear_octet_workspace(const sllm_mx* x, const sllm_mx* w, uint32_t out_dtype, uint64_t* bytes);
int32_t sllm_mx_linear_grad_workspace(const sllm_matrix* dy, const sllm_mx* w, uint64_t* bytes);

/* out's row i = scale * row ids[i] of table, zeros where ids[i] names no row. */
int32_t sllm_embedding(const sllm_matrix* table, const sllm_ids* ids, float scale, const sllm_matrix* out,
                       int32_t device, void* stream);

/* The same from a table in MX FP4. */
int32_t sllm_embedding_mx(const sllm_mx* table, const sllm_ids* ids, float scale, const sllm_matrix* out,
                          int32_t device, void* stream);

#define SLLM_GRAD_ACCUMULATE 1u  /* add to grad instead of replacing it */

/* The gradient of a lookup by its table: grad's row v = scale * the sum, in the
 * order of positions, of dy's rows i with ids[i] = v; zeros where there are
 * none.  With SLLM_GRAD_ACCUMULATE that is added to what grad holds, in 32 bits,
 * and rows no id names are not touched.  At most 2^24 ids (RANGE). */
int32_t sllm_embedding_grad(const sllm_matrix* dy, const sllm_ids* ids, float scale, uint32_t flags,
                            const sllm_matrix* grad, void* workspace, uint64_t workspace_bytes, int32_t device,
                            void* stream);
int32_t sllm_embedding_grad_workspace(uint64_t n_ids, const sllm_matrix* grad, uint64_t* bytes);

/* A matrix in MX FP8 (the formats' MXFP8 with E4M3 elements; "octet" here), for activations: an sllm_mx
 * whose blocks have 32 code bytes each, a column a byte, and the same scales.  Sizes of the
 * two buffers; host-only.  Errors: INVAL, RANGE. */
int32_t sllm_mx_octet_sizes(uint64_t rows, uint64_t cols, uint64_t* codes_bytes, uint64_t* scales_bytes);

/* dst = src in MX FP8.  A block's scale is the smallest power of two from 2^-127 on whose
 * 448-fold is not below its largest magnitude, so nothing saturates; its elements divided by
 * the scale go to the nearest E4M3 value, ties to the even code.  A block with an infinity or
 * a NaN gets scale 255 and codes 0. */
int32_t sllm_mx_octet_quantize(const sllm_matrix* src, const sllm_mx* dst, int32_t device, void* stream);

/* dst = the values src stands for, rounded to dst's type. */
int32_t sllm_mx_octet_dequantize(const sllm_mx* src, const sllm_matrix* dst, int32_t device, void* stream);

/* h = x + residual, rounded to their dtype, and y = h / sqrt(mean h^2 + eps) * gain, the mean
 * over a row's columns.  x, residual, h and y are of one shape and dtype, gain is one row of
 * any dtype; residual and h are both NULL or both not: h is x where there is none.  eps is
 * not negative, and where it is 0 a row's root mean square is 2^-127 at least: its inverse has
 * to fit 32 bits.  inverse, if not NULL: each row's 1 / sqrt(mean h^2 + eps), for the gradient. */
int32_t sllm_rms_norm(const sllm_matrix* x, const sllm_matrix* residual, const sllm_matrix* gain, float eps,
                      const sllm_matrix* h, const sllm_matrix* y, float* inverse, int32_t device, void* stream);

/* The same with y, not rounded before, in MX FP8. */
int32_t sllm_rms_norm_octet(const sllm_matrix* x, const sllm_matrix* residual, const sllm_matrix* gain, float eps,
                          const sllm_matrix* h, const sllm_mx* y, int32_t device, void* stream);

/* The gradients of sllm_rms_norm from those by y and h (dh NULL: zero), and its h and
 * inverse: with f the inverse and s = dy * gain,
 *   dx = dh + f * (s - h * f^2 * mean(s * h)), the residual's gradient too, and
 *   dgain = the sum over rows of dy * h * f, in a fixed order, in gain's dtype. */
int32_t sllm_rms_norm_grad(const sllm_matrix* dy, const sllm_matrix* dh, const sllm_matrix* h, const sllm_matrix* gain,
                           const float* inverse, const sllm_matrix* dx, const sllm_matrix* dgain, void* workspace,
                           uint64_t workspace_bytes, int32_t device, void* stream);
int32_t sllm_rms_norm_grad_workspace(uint64_t rows, uint64_t cols, uint64_t* bytes);

/* Rows of tokens and heads in device memory, aligned to their element type: head h of
 * token t starts at data + t * token_stride + h * head_stride elements and its
 * `dim` elements are adjacent.  Rows do not overlap: either a token's heads lie within
 * its stride or a head's tokens do.  At most 2^30 rows of 128 elements each, and 2^16 heads
 * (RANGE). */
typedef struct sllm_heads {
    void*    data;
    uint64_t tokens, heads, dim;
    uint64_t token_stride, head_stride;  /* elements; any value for one token or head */
    uint32_t dtype;                      /* SLLM_DTYPE_F32, _F16 or _BF16 */
    uint32_t reserved;                   /* must be 0 */
} sllm_heads;

/* Causal attention with a sliding window and sinks, over packed sequences:
 *   out = softmax over the keys seen of (scale * q . key) times their values
 * The query at position i of its sequence sees the key at position j of the same one
 * where j <= i and (i - j < window or j < sinks); window 0: every j <= i.  q and out are
 * tokens x heads x dim, k and v tokens x kv_heads x dim, of one dtype; heads is a multiple
 * of kv_heads, and head h has the keys of head h / (heads / kv_heads).  Sequence s is
 * tokens offsets[s] to offsets[s + 1] - 1; NULL: all of them.  Offsets that go back, or lie
 * outside the tokens, are taken as the nearest that do not.  Tokens of no sequence have an
 * output of zeros.  At most 2^16 sequences, and 2^22 times the heads (RANGE).
 *
 * Scores, their running maximum and sum, and the output's sums are held in 32 bits;
 * weights are rounded to the dtype before they are multiplied with values, as the largest
 * weight of a row so far, or up to 2^8 times that, is one.  What a query does not see does
 * not count, infinities and NaN included.  scale is a positive number up to 2.3e38.
 *
 * lse, if not NULL: tokens x heads floats, the logarithm of the sum of exp(scale * q . key)
 * over the keys seen (zero for tokens of no sequence), for the gradient. */
int32_t sllm_attention(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v, const sllm_ids* offsets,
                       uint64_t window, uint64_t sinks, float scale, const sllm_heads* out, float* lse,
                       int32_t device, void* stream);

/* The gradients of sllm_attention by q, k and v, from dout (as out) and the out and lse of
 * that call: with p = exp(scale q . k - lse) and ds = p (dout . v - dout . out),
 *   dq = scale * sum ds k, dk = scale * sum ds q, dv = sum p dout,
 * the last two over all heads that share the key.  p is rounded to the dtype before it is
 * multiplied; ds goes as that and what the rounding leaves, two products (float16's times a
 * power of two that keeps it in float16's range); sums are held in 32 bits.  Where rows see
 * few keys, ds is freed of what out's rounding adds to its sum over a row, which is zero.  p
 * is off by |lse| * 2^-22 of itself, and where |lse| is past 350 by no more than there: such
 * rows' largest score and the sum against it are found again.  Tokens of no sequence have
 * gradients of zeros. */
int32_t sllm_attention_grad(const sllm_heads* dout, const sllm_heads* q, const sllm_heads* k, const sllm_heads* v,
                            const sllm_heads* out, const float* lse, const sllm_ids* offsets, uint64_t window,
                            uint64_t sinks, float scale, const sllm_heads* dq, const sllm_heads* dk,
                            const sllm_heads* dv, void* workspace, uint64_t workspace_bytes, int32_t device,
                            void* stream);
int32_t sllm_attention_grad_workspace(const sllm_heads* q, const sllm_heads* k, const sllm_ids* offsets,
                                      uint64_t window, uint64_t sinks, uint64_t* bytes);

/* Keys and values of sequences, each (sequences, heads, sinks + window, dim), contiguous:
 * position p is in slot p where p < sinks, and else in slot sinks + (p - sinks) % window,
 * which holds the last position that has been there. */
typedef struct sllm_kv_cache {
    void*    k;
    void*    v;
    uint64_t sequences, heads, dim;
    uint64_t window, sinks;  /* window at least 1, both at most 2^30 together (RANGE) */
    uint32_t dtype;
    uint32_t reserved;       /* must be 0 */
} sllm_kv_cache;

/* The same attention of new tokens behind those in the cache, with its window and sinks.
 * lengths[s] is how many tokens sequence s has had before; its new tokens are at the
 * positions from there on, see what they see in the cache and among themselves, and are
 * written into the cache.  Sequence s's new tokens are offsets[s] to offsets[s + 1] - 1, as
 * above, or token s alone where offsets is NULL: then at most 2^22 sequences times heads
 * (RANGE).  A sequence whose length is negative, or above 2^62, takes no part: its output is
 * zeros and its cache is left as it is.  lengths is only read. */
int32_t sllm_attention_cached(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v,
                              const sllm_kv_cache* cache, const sllm_ids* lengths, const sllm_ids* offsets,
                              float scale, const sllm_heads* out, void* workspace, uint64_t workspace_bytes,
                              int32_t device, void* stream);
int32_t sllm_attention_cached_workspace(const sllm_heads* q, const sllm_heads* k, const sllm_heads* v,
                                        const sllm_kv_cache* cache, const sllm_ids* lengths,
                                        const sllm_ids* offsets, uint64_t* bytes);

/* Message of the last failed call on this thread ("" if none). */
const char* sllm_last_error(void);
/* Static name of a status code. */
const char* sllm_strerror(int32_t code);

#ifdef __cplusplus
}
#endif
#endif /* SLLM_H */
