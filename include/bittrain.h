/*
 * libbittrain -- the sparse bitmap activation codec of BitTrain on one MI355X.
 *
 * The format (Section 3.2, "Bitmap Format"): an activation tensor of n
 * elements, flattened in place, is stored as
 *   (i)  a bitmap with one bit per element, set where the element is non-zero;
 *   (ii) the non-zero elements, in ascending flattened index order.
 * Compression runs in the forward pass (Algorithm 1), restoration in the
 * backward pass (Algorithm 2).  The footprint is M_b = width * nnz + n / 8
 * bytes against M_d = width * n dense.
 *
 * Conventions fixed here where the paper is silent:
 *   - "zero" is the all-zero bit pattern of the element.  -0.0, NaNs, denormals
 *     and infinities are kept as values, so Algorithm 2 after Algorithm 1
 *     reproduces the tensor bit for bit.  fp16 and bf16 are the same codec.
 *   - element i owns bit (i mod 32), least significant first, of the uint32
 *     word (i div 32).  The bitmap has ceil(n/32) words; the unused high bits
 *     of the last word are written as 0, so popcount(bitmap) == nnz.
 *   - a cleared bit restores +0 (all-zero bits) of the element width.
 *   - tensors are flat, contiguous buffers; the shape stays with the caller.
 *
 * Every pointer named d_* is DEVICE memory owned by the caller (d_nnz may also be pinned
 * host memory, see bt_compress).  The library
 * allocates nothing, frees nothing and never synchronises: each device call
 * enqueues its kernel(s) on `stream` and returns.  Argument errors are found on
 * the host before anything is launched; nothing is written in that case.
 * No exceptions, no errno, no logging: the return code is the only channel.
 */
#ifndef BITTRAIN_H
#define BITTRAIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BT_F32 = 0,  /* 4-byte elements */
    BT_F16 = 1,  /* 2-byte elements */
    BT_BF16 = 2, /* 2-byte elements; identical to BT_F16 at the byte level */
    BT_F64 = 3   /* 8-byte elements (the paper's formats are half, single and double precision) */
} bt_dtype;

typedef enum {
    BT_OK = 0,
    BT_ERR_NULL = 1,      /* a required pointer is NULL */
    BT_ERR_DTYPE = 2,     /* dtype is not one of bt_dtype */
    BT_ERR_ALIGN = 3,     /* a pointer is not aligned as documented */
    BT_ERR_WORKSPACE = 4, /* workspace smaller than bt_workspace_bytes(n, dtype) */
    BT_ERR_HIP = 5,       /* the HIP runtime refused the launch */
    BT_ERR_SIZE = 6,      /* n is beyond BT_MAX_ELEMENTS, or a size the call does not take */
    BT_ERR_UNSUPPORTED = 7, /* the call exists only in another build of the library */
    BT_ERR_ARGUMENT = 8   /* a number or a combination of arguments that the call does not take */
} bt_status;

/* Largest number of tensors in one batched call. */
#define BT_MAX_BATCH 64

/* Largest n any call accepts (2^37 elements). */
#define BT_MAX_ELEMENTS ((uint64_t)1 << 37)

/* A hipStream_t, passed as an opaque pointer so that this header needs no HIP
 * header.  NULL is the default stream. */
typedef void *bt_stream;

/* ---- host-only, pure functions (no device is touched) -------------------- */

/* M_b of Section 3.2, generalised to the element width and to whole 32-bit
 * bitmap words: 4 * ceil(n/32) + nnz * sizeof(dtype).  Equals the paper's
 * 4 * nnz + n / 8 for fp32 whenever 32 divides n (every row of Table 1).
 * Returns 0 for an unknown dtype or nnz > n. */
size_t bt_compressed_size(uint64_t n, uint64_t nnz, bt_dtype dtype);

/* M_d of Section 3.2: n * sizeof(dtype), the dense footprint.  0 for an unknown dtype. */
size_t bt_dense_size(uint64_t n, bt_dtype dtype);

/* M_c of Section 3.2, the footprint of the coordinate-list (COO) format the paper
 * compares with: (sizeof(dtype) + index_bytes * ndim) * nnz, index_bytes being 4
 * (integer indices) or 8 (long indices).  0 for an unknown dtype, ndim == 0 or
 * another index size. */
size_t bt_coo_size(uint64_t nnz, uint32_t ndim, uint32_t index_bytes, bt_dtype dtype);

/* 4 * ceil(n/32): the bytes d_bitmap must hold. */
size_t bt_bitmap_bytes(uint64_t n);

/* Bytes of scratch that bt_compress / bt_decompress need for a tensor of n
 * elements: a 256-byte header plus 24 bytes per tile of the single-pass grid
 * scan (a tile is 32 KiB of dense data: 4096 eight-byte, 8192 four-byte or 16384
 * two-byte elements), in blocks of 256 tiles.  Monotone in n; 0 for an unknown dtype. */
size_t bt_workspace_bytes(uint64_t n, bt_dtype dtype);

/* Size in bytes of one element, 0 for an unknown dtype. */
size_t bt_dtype_size(bt_dtype dtype);

const char *bt_status_str(bt_status status);

/* ---- device calls -------------------------------------------------------- */

/* What a caller may look at, or set, in a workspace: 32-bit words at the start of it.
 *   BT_WS_ERROR_WORD        0 in normal operation.  The one wait inside the kernels that can
 *                           fail, the grid scan waiting for the counts of a call's tiles, is
 *                           bounded; a kernel whose wait ran out sets this word to 1 and
 *                           ends normally, staying inside all buffers (read it with
 *                           bt_workspace_status).  The outputs of that call are not valid (nnz
 *                           in particular is not written), and later calls on the workspace
 *                           write nothing at all, until bt_workspace_init has been run on it again.
 *   BT_WS_WAIT_LIMIT_WORD   passes of the grid scan after which it gives up (where a call on a small
 *                           tensor has none: polls of its last tile); 0 (the initial
 *                           state) means the built-in limit of 2^20, far beyond what any
 *                           tensor needs.  Written by the caller only (a device-side store
 *                           or copy ordered before the call); meant for tests of the
 *                           failure path.
 *   BT_WS_PATIENCE_WORD     polls after which a tile's workgroup stops waiting for the grid
 *                           scan and counts what lies before its tile itself, from the
 *                           bitmap (restoration) or the input (compression): correct, only
 *                           slower; looked at every 256th poll; 0 means the built-in 4096.  Written by the caller only,
 *                           like the wait limit; meant for tests of that path.
 *   BT_WS_WIDE_WORD         non-zero: the grid scan of a call on one tensor writes every tile's
 *                           offset with 8-byte stores, which it otherwise does only once the
 *                           offsets reach 2^32 (below that it writes two neighbours' lower
 *                           halves in one store).  Same results; written by the caller only;
 *                           meant for tests of the wide path on tensors of ordinary size.
 *   BT_WS_MUTE_WORD         looked at in the instrumented build of the library only (-DBT_TIMELINE).  Non-zero:
 *                           the grid scan counts and ends the call as always but writes no offset, so that
 *                           every tile runs out of patience; in calls on small tensors, which have no grid scan,
 *                           1 keeps all counts from the tiles but the last, 2 from the last one too, whose wait
 *                           then runs out.  Written by the caller only; meant for tests of the paths behind the waits. */
#define BT_WS_ERROR_WORD 2
#define BT_WS_WAIT_LIMIT_WORD 3
#define BT_WS_PATIENCE_WORD 4
#define BT_WS_WIDE_WORD 5
#define BT_WS_MUTE_WORD 6

/* Put a workspace into its initial state (all zero bytes) by enqueueing a fill
 * kernel on `stream`.  Required once after allocating a workspace, before its
 * first use, and again if a kernel using it was aborted.  After that the
 * kernels leave the workspace ready for the next call themselves, so
 * bt_compress and bt_decompress are one launch each.
 * d_workspace: 128-byte aligned.  Errors: BT_ERR_NULL, BT_ERR_ALIGN, BT_ERR_HIP. */
bt_status bt_workspace_init(void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* Algorithm 1 (dense -> bitmap), as one fused pass over the input.
 *   d_in        n elements of `dtype`, 16-byte aligned, read once.
 *   d_bitmap    ceil(n/32) uint32 words, 4-byte aligned; every word is written.
 *   d_values    room for values_cap elements, element-aligned; on return
 *               elements [0, min(nnz, values_cap)) hold the non-zero elements in
 *               index order; the rest is untouched.
 *   values_cap  capacity of d_values in elements.  If nnz > values_cap nothing
 *               is written beyond the capacity, the bitmap and *d_nnz are still
 *               complete, and the caller sees the overflow as *d_nnz > values_cap.
 *               The worst case is n.
 *   d_nnz       one uint64, 8-byte aligned, written by the kernel: valid once
 *               `stream` has reached this call.  It may also be pinned host memory that the
 *               device can address (hipHostMalloc): the host may read it once it has waited for the
 *               stream or for an event behind the call.  A call that gives up a wait, or finds a
 *               workspace on which one was given up, leaves it as it was; others write it with one 8-byte
 *               store that is visible to the whole system.  So a host that has put a number there which no nnz
 *               is may also look for the change, if the memory is coherent (hipHostMalloc's is unless asked
 *               otherwise): it then has nnz, but not yet the rest of the call's outputs.
 *   d_workspace bt_workspace_bytes(n, dtype) bytes, 128-byte aligned, initialised
 *               once with bt_workspace_init.  A workspace must not be shared by
 *               two calls that can be in flight at the same time: calls that use
 *               one workspace must be ordered (same stream, or events).
 * Input and outputs must not overlap.  Algorithm 1's last step, giving up the
 * dense tensor, is the caller dropping d_in after this call is enqueued.  n == 0 only writes *d_nnz = 0.
 * Errors: BT_ERR_NULL, BT_ERR_DTYPE, BT_ERR_ALIGN, BT_ERR_SIZE, BT_ERR_WORKSPACE,
 * BT_ERR_HIP. */
bt_status bt_compress(const void *d_in, uint64_t n, bt_dtype dtype,
                      uint32_t *d_bitmap, void *d_values, uint64_t values_cap,
                      uint64_t *d_nnz,
                      void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* bt_compress for callers that cannot allocate device memory and have no workspace to pass: code
 * whose stream is being recorded into a HIP graph, tight serving loops, harnesses that forbid
 * allocation.  Same arguments and results as bt_compress, without the workspace: the library
 * uses a workspace of its own, a device array of 256 + 6144 * BT_STATIC_MAX_TILES / 256 bytes
 * (393,472) that exists once on every GPU the library is loaded on until the process ends.  The
 * call allocates and frees nothing; it enqueues a fill kernel that clears that workspace and then
 * the compression kernel.
 *   n           at most BT_STATIC_MAX_TILES tiles (bt_tile_elems(dtype) elements each),
 *               else BT_ERR_SIZE.
 * All calls on one GPU share the one array: two of them that can be in flight at the same time
 * (different streams without an event between them) race, and so do the processes' threads that
 * issue them.  Errors: as bt_compress, without BT_ERR_WORKSPACE; BT_ERR_HIP also if the array's
 * address cannot be had. */
#define BT_STATIC_MAX_TILES 16384
bt_status bt_compress_static(const void *d_in, uint64_t n, bt_dtype dtype,
                             uint32_t *d_bitmap, void *d_values, uint64_t values_cap,
                             uint64_t *d_nnz, bt_stream stream);

/* Activation pruning (Section 4.3) fused into Algorithm 1: one pass that stores an
 * element only where its value exceeds `threshold` and treats it as zero elsewhere
 * (the paper's thresholds are 0, 0.01, 0.05 and 0.1).  The comparison is strict and exact:
 * an element is kept where its value, as a real number, is greater than `threshold`, as a
 * real number.  (BT_F64 elements are compared in double precision; narrower ones, widened
 * exactly, in single precision with the largest single at or below `threshold`, which
 * decides the same.)  A NaN element exceeds nothing and is dropped; a NaN threshold drops
 * everything.  The result is exactly bt_compress of the pruned tensor (so a +0.0
 * that survives a negative threshold is still not stored).  The bitmap marks the kept
 * elements, d_values holds their original
 * bit patterns in index order, *d_nnz their number.  With threshold 0 on a
 * pre-activation tensor x this is compress(ReLU(x)) without ever writing ReLU(x):
 * bt_decompress then yields ReLU(x) and bt_relu_backward_from_bitmap its backward.
 * All arguments, requirements and errors as for bt_compress. */
bt_status bt_compress_pruned(const void *d_in, uint64_t n, bt_dtype dtype, double threshold,
                             uint32_t *d_bitmap, void *d_values, uint64_t values_cap,
                             uint64_t *d_nnz,
                             void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* The activation itself and its stash in one pass: as bt_compress_pruned, and in addition
 * the dense pruned tensor goes to d_dense_out (n elements, 16-byte aligned):
 *   d_dense_out[i] = x[i] where x[i] > threshold, +0 elsewhere,
 * i.e. y = ReLU(x) for threshold 0 -- what the next layer consumes -- while bitmap, values
 * and nnz are the compressed form of that same y, kept for the backward pass.  One read of
 * x serves both; run separately, ReLU and bt_compress read the activation three times and
 * write it once more.  d_dense_out may be d_in itself (in place) but must not partly
 * overlap it or any other argument.  Everything else as bt_compress_pruned. */
bt_status bt_activation_compress(const void *d_in, uint64_t n, bt_dtype dtype, double threshold,
                                 void *d_dense_out,
                                 uint32_t *d_bitmap, void *d_values, uint64_t values_cap,
                                 uint64_t *d_nnz,
                                 void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* Algorithm 2 (bitmap -> dense).
 *   d_bitmap    ceil(n/32) words as written by bt_compress (bits at positions
 *               >= n are ignored).
 *   d_values    the non-zero elements in index order, popcount(bitmap) of them,
 *               element-aligned.  nnz is not an argument: it is implied by the
 *               bitmap, so no host synchronisation is needed between the two calls.
 *   d_out       n elements, 16-byte aligned; every element is written (values at
 *               set bits, +0 at cleared bits).
 *   d_workspace as for bt_compress.
 * Errors: as bt_compress. */
bt_status bt_decompress(const uint32_t *d_bitmap, const void *d_values, uint64_t n,
                        bt_dtype dtype, void *d_out,
                        void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* ---- Algorithm 2 without the scan: the tile index ------------------------------
 *
 * Algorithm 2 carries one counter, j, the position in d_values of the next value.
 * bt_decompress has to find j for every tile of the tensor by a scan over the whole
 * bitmap before a tile can fetch its values.  bt_compress knows these numbers when it
 * writes the values: bt_compress_indexed also leaves them in d_index, entry t being j
 * at element t * bt_tile_elems(dtype) (the number of values stored before that
 * element), and bt_decompress_indexed starts every tile from its entry: no workspace,
 * no dependency between tiles.  The index is 8 bytes per 32 KiB of dense data, derived
 * from the bitmap alone; the compressed form proper (bitmap, values, nnz) is unchanged. */

/* Elements per tile: 32 KiB / sizeof(dtype).  0 for an unknown dtype. */
size_t bt_tile_elems(bt_dtype dtype);

/* Bytes d_index must hold: 8 * ceil(n / bt_tile_elems(dtype)). */
size_t bt_index_bytes(uint64_t n, bt_dtype dtype);

/* bt_compress, plus d_index (8-byte aligned, bt_index_bytes(n, dtype) bytes; every entry
 * is written).  Everything else as bt_compress. */
bt_status bt_compress_indexed(const void *d_in, uint64_t n, bt_dtype dtype,
                              uint32_t *d_bitmap, void *d_values, uint64_t values_cap,
                              uint64_t *d_nnz, uint64_t *d_index,
                              void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* Algorithm 2 with j taken from the tile index.
 *   d_values, values_cap   the stored values and how many elements d_values holds (at
 *                          least the number of set bits, for a correct result); nothing at
 *                          or beyond values_cap is read, whatever d_index says.
 *   d_index                as written by bt_compress_indexed for this bitmap.  Entries that
 *                          do not belong to the bitmap give a wrong d_out, never an access
 *                          outside the buffers.
 * d_bitmap, d_out, alignment and errors as bt_decompress (no workspace errors). */
bt_status bt_decompress_indexed(const uint32_t *d_bitmap, const void *d_values, uint64_t values_cap,
                                const uint64_t *d_index, uint64_t n, bt_dtype dtype, void *d_out,
                                bt_stream stream);

/* Backward of y = ReLU(x) from the bitmap of y alone.  Algorithm 1 sets bit i
 * exactly where y[i] != 0, i.e. where x[i] > 0, which is the ReLU derivative, so
 * the values array is not needed:
 *   grad_in[i] = bit(i) ? grad_out[i] : +0      (a select, never a multiply).
 *   d_grad_out, d_grad_in   n elements each, 16-byte aligned; they may be the
 *                           same buffer (in place) but must not partly overlap.
 * Errors: BT_ERR_NULL, BT_ERR_DTYPE, BT_ERR_ALIGN, BT_ERR_SIZE, BT_ERR_HIP. */
bt_status bt_relu_backward_from_bitmap(const uint32_t *d_bitmap, const void *d_grad_out,
                                       uint64_t n, bt_dtype dtype, void *d_grad_in,
                                       bt_stream stream);

/* The forward pass that the backward above belongs to, where nothing but the bitmap is kept: y = ReLU(x) and the
 * bitmap of y from one read of x, no values, no nnz, no workspace:
 *   out[i] = x[i] where x[i] > 0 or x[i] is a NaN (bit pattern kept), else +0;  bit(i) = out[i] != 0.
 *   d_in, d_out   n elements each, 16-byte aligned; they may be the same buffer but must not partly overlap.
 *   d_bitmap      ceil(n/32) words, bits at or beyond n are written as 0.
 * Errors: as bt_relu_backward_from_bitmap. */
bt_status bt_relu_forward(const void *d_in, uint64_t n, bt_dtype dtype, void *d_out, uint32_t *d_bitmap,
                          bt_stream stream);

/* Double-mask batch normalisation (Section 3.1, "Exploiting Sparsity"): the sparsity
 * pattern of a normalisation layer's input is applied to its output, so that the
 * output compresses as well as the input did.  d_bitmap is the bitmap of that input
 * (as written by bt_compress), d_in the layer's output:
 *   out[i] = bit(i) ? in[i] : +0.
 * The same select as bt_relu_backward_from_bitmap, under the name of this use; all
 * requirements and errors as there (d_out may be d_in). */
bt_status bt_mask_apply(const uint32_t *d_bitmap, const void *d_in, uint64_t n, bt_dtype dtype,
                        void *d_out, bt_stream stream);

/* ---- many tensors in one launch ------------------------------------------------
 *
 * A training step stores every layer's activation (Section 3.2 applies the format
 * to all of them; Table 1 lists a network's layers).  Compressing them one call
 * each pays one launch and one pipeline fill-and-drain per tensor, which dominates
 * for the small layers; the batched calls run Algorithm 1 / Algorithm 2 on all the
 * tensors of a list in one launch per BT_MAX_BATCH tensors (restoration) or 52 tensors
 * (compression, whose items are larger).  The result for each
 * tensor is exactly what the single-tensor call gives.  The item arrays are HOST
 * memory and are read before the call returns; the pointers inside them are device
 * pointers with the meaning, alignment and overlap rules of the single-tensor calls.
 * All tensors of a call share one dtype. */

typedef struct {
    const void *d_in;    /* n elements, 16-byte aligned (may be NULL when n == 0) */
    uint64_t n;
    uint32_t *d_bitmap;  /* ceil(n/32) words */
    void *d_values;      /* room for values_cap elements */
    uint64_t values_cap;
    uint64_t *d_nnz;     /* one uint64 per tensor, 8-byte aligned, required also when n == 0 */
    uint64_t *d_index;   /* NULL, or bt_index_bytes(n, dtype) bytes, 8-byte aligned: the tensor's tile index,
                            as bt_compress_indexed writes it */
    void *d_dense_out;   /* bt_compress_batch_pruned only, else NULL: the dense pruned tensor, as
                            bt_activation_compress writes it (n elements, 16-byte aligned, may be d_in);
                            given for every tensor of the call that has elements, or for none */
} bt_compress_item;

typedef struct {
    const uint32_t *d_bitmap;
    const void *d_values;
    uint64_t n;
    void *d_out;         /* n elements, 16-byte aligned */
    uint64_t values_cap; /* bt_decompress_batch_indexed only: elements d_values holds, as for bt_decompress_indexed */
    const uint64_t *d_index; /* bt_decompress_batch_indexed only: the tensor's tile index */
} bt_decompress_item;

/* Workspace bytes a batched call on tensors of n[0..count) elements needs (host
 * function; n is a host array).  Never less than bt_workspace_bytes(0, dtype); 0 for
 * an unknown dtype or n == NULL with count != 0. */
size_t bt_batch_workspace_bytes(const uint64_t *n, size_t count, bt_dtype dtype);

/* Algorithm 1 on every tensor of items[0..count).  All items are checked before
 * anything is launched.  d_workspace: bt_batch_workspace_bytes(...) bytes, 128-byte
 * aligned, initialised once with bt_workspace_init; the same workspace may serve
 * single-tensor and batched calls alike, in stream order.  count == 0 does nothing.
 * d_index of an item, if
 * given, receives that tensor's tile index.  Errors: as bt_compress (the first offending item
 * decides); BT_ERR_NULL also if an item has d_dense_out. */
bt_status bt_compress_batch(const bt_compress_item *items, size_t count, bt_dtype dtype,
                            void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* bt_compress_pruned on every tensor of items[0..count), one threshold for all; where the
 * items give d_dense_out, bt_activation_compress (the activations of a whole list of layers
 * pruned, handed on and stashed in one launch).  Otherwise as bt_compress_batch.
 * Errors: also BT_ERR_NULL if some tensors with elements have d_dense_out and others do not. */
bt_status bt_compress_batch_pruned(const bt_compress_item *items, size_t count, bt_dtype dtype,
                                   double threshold,
                                   void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* Algorithm 2 on every tensor of items[0..count); otherwise as bt_compress_batch and
 * bt_decompress.  values_cap and d_index of the items are not looked at. */
bt_status bt_decompress_batch(const bt_decompress_item *items, size_t count, bt_dtype dtype,
                              void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* bt_decompress_indexed on every tensor of items[0..count), each from the tile index that
 * bt_compress_indexed or a batched compression with d_index left for it: no scan, no
 * workspace, no dependency between tiles or tensors.  Errors: as bt_decompress_indexed. */
bt_status bt_decompress_batch_indexed(const bt_decompress_item *items, size_t count, bt_dtype dtype,
                                      bt_stream stream);

/* What became of the calls on a workspace, without knowing its layout: enqueues a kernel
 * that writes d_status[0] = 1 if a kernel gave up a wait on this workspace (the outputs of
 * that call and of every later one are not valid, and the workspace refuses work until
 * bt_workspace_init has been run on it again), else 0, and d_status[1] = the number of calls
 * completed on it since it was initialised.  d_status: two uint32 of device memory, valid
 * once `stream` has reached this call.  Errors: BT_ERR_NULL, BT_ERR_ALIGN, BT_ERR_HIP. */
bt_status bt_workspace_status(const void *d_workspace, uint32_t *d_status, bt_stream stream);

/* ---- the operators of a feed-forward sublayer -----------------------------------
 *
 * What stands around the activations that the codec keeps, in a step that trains such a sublayer or in a call that
 * answers with it: the gated projections whose output is the activation, the norms, gate and residual sum between two
 * sublayers, and the clipping of the step's gradients.  BT_F32, BT_F16 and BT_BF16.  All sums, statistics and
 * activations are computed in 32 bits or more and rounded once, to the tensors' type, where they are stored.  What a backward
 * pass takes from its forward pass is so rounded too (d_gate and d_up, d_out), and so are the factors that bt_gated_backward multiplies.
 *
 * Tensors are row-major and contiguous, and are aligned to their elements; those that are aligned to 16 bytes and whose
 * rows are whole 16-byte vectors go faster.  A workspace is scratch memory of the call: 128-byte aligned, of the size that the
 * call's size function gives, in any state, free again once the stream has passed the call; two calls that can be in
 * flight at the same time must not share one.  It may be NULL where that size is 0.  Results do not depend on
 * what else runs: equal inputs give equal bits. */

typedef enum {
    BT_ACT_RELU = 0,     /* act(g) = g where g > 0 (or g is a NaN), else 0 */
    BT_ACT_SILU = 1,     /* act(g) = g / (1 + exp(-g)) */
    BT_ACT_GELU_TANH = 2 /* act(g) = g / 2 * (1 + tanh(sqrt(2 / pi) * (g + 0.044715 g^3))); both are 0 at -infinity, with a slope of 0 */
} bt_activation;

/* Largest numbers of rows and of features that these calls accept. */
#define BT_MAX_ROWS (((uint64_t)1 << 31) - 1)
#define BT_MAX_FEATURES (((uint64_t)1 << 24))
/* Largest number of columns of the residual norms. */
#define BT_MAX_NORM_COLS 16384

/* Bytes of workspace for bt_gated_forward (backward == 0) or bt_gated_backward (else).  0 for an unknown dtype or sizes the calls refuse. */
size_t bt_gated_workspace_bytes(uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, int backward);

/* The gated projections: h = act(x w_gate^T) * (x w_up^T), in one kernel but where the sum over d is split (few rows) or rows that do not begin on 16-byte boundaries are
 * copied to some (128 rows and more).
 *   d_x               [rows, d]
 *   d_w_gate, d_w_up  [f, d] each
 *   d_h               [rows, f]
 *   d_gate, d_up      [rows, f] each, or NULL both: what bt_gated_backward needs of this pass, rounded to the
 *                     tensors' type: the pre-activations x w_gate^T and x w_up^T.  With BT_ACT_RELU act(x w_gate^T) and, where
 *                     that is not 0, x w_up^T, else +0: then h, gate and up are all +0 wherever a gate is closed and
 *                     compress as one.  (A gate that is open is kept as a number above 0, the smallest at the least, where
 *                     rounding would give 0.)
 * With BT_ACT_RELU h is +0 where the gate is closed, whatever the other factor is there (a select, never a multiply).
 * rows == 0 or f == 0 does nothing; with d == 0 the products are 0.  No output may overlap an input or another output.
 * Errors: BT_ERR_NULL, BT_ERR_DTYPE (BT_F64 too), BT_ERR_ALIGN, BT_ERR_SIZE, BT_ERR_WORKSPACE, BT_ERR_HIP, BT_ERR_ARGUMENT
 * (unknown activation, or only one of d_gate and d_up). */
bt_status bt_gated_forward(const void *d_x, const void *d_w_gate, const void *d_w_up,
                           uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, bt_activation activation,
                           void *d_h, void *d_gate, void *d_up,
                           void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* Its backward pass.  With g and u the two products, dg = grad_h * u * act'(g) and du = grad_h * act(g) (selects where a ReLU's gate
 * is closed), rounded to the tensors' type as the factors of the products (BT_F16: to an infinity beyond 65504, to fewer bits below 2^-14)
 *   grad_x = dg w_gate + du w_up      grad_w_gate = dg^T x      grad_w_up = du^T x
 *   d_gate, d_up                  as bt_gated_forward left them, for the same activation
 *   d_grad_x                      [rows, d], or NULL: not wanted (d_w_gate and d_w_up are not read then and may be NULL)
 *   d_grad_w_gate, d_grad_w_up    [f, d] each, or NULL both: not wanted (d_x is not read then and may be NULL)
 * Gradients are written, not added to.  rows == 0 writes zeros to the weights' gradients, f == 0 to grad_x.
 * Errors as for bt_gated_forward; BT_ERR_ARGUMENT also for only one of the weights' gradients. */
bt_status bt_gated_backward(const void *d_grad_h, const void *d_x, const void *d_w_gate, const void *d_w_up,
                            const void *d_gate, const void *d_up,
                            uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, bt_activation activation,
                            void *d_grad_x, void *d_grad_w_gate, void *d_grad_w_up,
                            void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* What stands between two blocks, in one pass over the rows:
 *   out = residual_scale * x + scale * gate * norm(block) * post_weight       y = norm(out) * pre_weight
 *   norm(t) = t / sqrt(mean(t^2) + eps) over a row of `cols`
 *   d_x            [rows, cols], the residual stream
 *   d_block        [rows, cols], the output of the block before; NULL: there is none, out is x itself and is not written
 *                  (d_out, d_post_weight and d_gate must be NULL then, and the two scales are not used)
 *   d_post_weight  [cols], or NULL: block goes in as it is, without its norm
 *   d_gate         [gate_rows, cols], or NULL: 1.  gate_rows divides rows: row r takes gate row r / (rows / gate_rows), so 1 is one
 *                  gate for all rows, the number of sequences one for each of them, and rows one for each row
 *   d_pre_weight   [cols], or NULL: y is not wanted (d_y must be NULL then)
 *   d_out, d_y     [rows, cols]; y is computed from out before out is rounded.  d_out may be d_x or d_block itself; else no overlap
 *   d_stats        NULL, or 2 * rows floats for bt_residual_norm_backward: 1 / sqrt(...) of block's rows (1 without
 *                  post_weight), then of out's
 * rows == 0 or cols == 0 does nothing.  Errors: BT_ERR_NULL, BT_ERR_DTYPE (BT_F64 too), BT_ERR_ALIGN, BT_ERR_SIZE, BT_ERR_HIP, BT_ERR_ARGUMENT
 * (a combination that is excluded above, gate_rows that does not divide rows, eps negative or not finite, a scale that is not finite). */
bt_status bt_residual_norm_forward(const void *d_x, const void *d_block, const void *d_post_weight, const void *d_gate,
                                   const void *d_pre_weight, uint64_t rows, uint64_t cols, uint64_t gate_rows, bt_dtype dtype,
                                   double eps, double scale, double residual_scale,
                                   void *d_out, void *d_y, float *d_stats, bt_stream stream);

/* Bytes of workspace for bt_residual_norm_backward; gate_rows 0 if there is no gate.  0 for an unknown dtype or sizes the call refuses. */
size_t bt_residual_norm_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t gate_rows, bt_dtype dtype);

/* The backward pass: the gradients of x, block, post_weight, gate and pre_weight from those of out and y.
 *   d_grad_out          [rows, cols], or NULL: 0
 *   d_grad_y            [rows, cols], or NULL: 0 (d_pre_weight and d_grad_pre_weight must be NULL then)
 *   d_out               out as the forward pass left it, rounded (x, if there was no block)
 *   d_block ... d_pre_weight, gate_rows, scale, residual_scale, d_stats    as in the forward pass
 *   d_grad_x            [rows, cols], or NULL: not wanted
 *   d_grad_block        [rows, cols]; d_grad_post_weight, d_grad_pre_weight [cols]; d_grad_gate [gate_rows, cols]: each NULL if not
 *                       wanted, and NULL if its tensor is
 * Gradients are written, not added to; d_grad_x may be d_grad_out itself, d_grad_block may be d_block or d_grad_y itself; else no
 * overlap.  A gradient that several rows share is summed in 32 bits, in an order that the sizes alone decide.
 * rows == 0 writes zeros to the weights' gradients.  Errors as for the forward pass, and BT_ERR_WORKSPACE. */
bt_status bt_residual_norm_backward(const void *d_grad_out, const void *d_grad_y, const void *d_out, const void *d_block,
                                    const void *d_post_weight, const void *d_gate, const void *d_pre_weight, const float *d_stats,
                                    uint64_t rows, uint64_t cols, uint64_t gate_rows, bt_dtype dtype, double scale, double residual_scale,
                                    void *d_grad_x, void *d_grad_block, void *d_grad_post_weight, void *d_grad_gate, void *d_grad_pre_weight,
                                    void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* A gradient among others (host memory, read before the call returns). */
typedef struct {
    const void *d_in;   /* n elements (may be NULL when n == 0) */
    void *d_out;        /* bt_clip_grads: n elements; d_in itself, or memory that overlaps no item's */
    uint64_t n;
    bt_dtype dtype;     /* BT_F32, BT_F16 or BT_BF16, of each item its own */
} bt_clip_item;

/* Bytes of workspace for bt_grad_norm and bt_clip_grads on `count` items, whatever their sizes. */
size_t bt_clip_workspace_bytes(size_t count);

/* *d_norm = sqrt(sum of the squares of all elements of all items), the sum in 64 bits, where no square overflows, in an order that the sizes alone decide.
 * (An infinity or a NaN among them makes it one.)  count == 0 writes 0.
 * Errors: BT_ERR_NULL, BT_ERR_DTYPE, BT_ERR_ALIGN, BT_ERR_SIZE (n beyond BT_MAX_ELEMENTS), BT_ERR_WORKSPACE, BT_ERR_HIP. */
bt_status bt_grad_norm(const bt_clip_item *items, size_t count, float *d_norm,
                       void *d_workspace, size_t workspace_bytes, bt_stream stream);

/* The same, and every gradient scaled so that their norm is at most max_norm: d_out = d_in * min(1, max_norm / (norm + eps)), the
 * product in 32 bits.  Nothing waits for the host: the factor stays on the device.  A norm of infinity makes the factor 0 and a NaN makes
 * it a NaN, as the formula has it; the caller sees either in *d_norm.  max_norm >= 0 (infinity: no clipping, whatever the norm), eps >= 0 (with both
 * 0 a norm of 0 leaves the zeros).
 * Errors: as bt_grad_norm, and BT_ERR_ARGUMENT. */
bt_status bt_clip_grads(const bt_clip_item *items, size_t count, double max_norm, double eps, float *d_norm,
                        void *d_workspace, size_t workspace_bytes, bt_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* BITTRAIN_H */
