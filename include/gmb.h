/*
 * gmb.h — C ABI of the mini-batch GNN hot path on MI355X (gfx950).
 *
 * The library implements the data-parallel part of one trainer's iteration
 * in DistDGL (arXiv 2010.05337): build a mini-batch by recursive fan-out
 * neighbour sampling (Section II-B), pull the feature rows of the sampled
 * vertices (the KVStore "pull" of Section III-C, here a local gather), and
 * run the GraphSAGE-mean forward pass (Section II-A, Eq. (1); model of
 * Section IV).
 *
 * Conventions shared by every entry point
 *   - Pointers documented "device" are HIP device pointers; "host" are host
 *     pointers.  Device buffers are owned by the caller; the library never
 *     allocates or frees device memory, and keeps none but the fixed scratch
 *     array of gmb_sample_blocks_noalloc (a static device array).
 *   - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *     All device work of a call is enqueued on that stream; a call returns
 *     as soon as the work is enqueued, unless it says it synchronises.
 *   - Return value: GMB_OK (0) or a negative gmb_status.  Argument errors are
 *     detected on the host before anything is enqueued, so nothing runs and
 *     no buffer is touched.  Errors in the data (a vertex id out of range, a
 *     duplicated seed) are found on the device; they set bits of a sticky
 *     status word that gmb_read_status() returns.  Outputs produced under a
 *     data error are unspecified, but every access stays in bounds.
 *   - gmb_last_error() returns a thread-local message for the last failing
 *     call on this thread.
 *   - Layer numbering: model layer l = 0 is the input layer; fanouts[l]
 *     belongs to layer l, so the first hop (from the seeds) uses
 *     fanouts[L-1], and blocks are returned in layer order.
 *   - Vertex ids are int32 (graphs up to 2^31 - 1 vertices); CSR row offsets
 *     may be int32 or int64.
 */
#ifndef GMB_H
#define GMB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GMB_MAX_LAYERS 8
#define GMB_ABI_VERSION 1

typedef enum {
  GMB_OK = 0,
  GMB_EINVAL = -1,   /* bad argument (null pointer, bad size, unsupported shape) */
  GMB_ENOSPC = -2,   /* workspace or state buffer too small */
  GMB_EDEVICE = -3,  /* a HIP runtime call failed */
  GMB_ERANGE = -4,   /* (device) a vertex id outside [0, num_nodes) */
  GMB_EDUP = -5      /* (device) the seed list holds a vertex twice */
} gmb_status;

typedef enum { GMB_F32 = 0, GMB_BF16 = 1 } gmb_dtype;

/* Microscaled formats, by the bits of an element. */
typedef enum { GMB_MXFP4 = 4, GMB_MXFP8 = 8 } gmb_mx_format;

/* Bits of the device status word. */
#define GMB_STATUS_ERANGE 1u
#define GMB_STATUS_EDUP 2u
#define GMB_STATUS_INTERNAL 4u   /* a bounded wait inside the relabel scan ran out */
#define GMB_STATUS_INVALID 8u    /* gmb_validate_blocks found an inconsistent block */

/* In-neighbour CSR of the input graph G(V, E) (Section II-A): row v lists
 * the sources u of the edges u -> v, so sampling row v samples the vertices
 * whose messages flow into v.  Rows must be sorted ascending and unique;
 * without that, sampled neighbour sets may hold duplicates.
 * All pointers are device pointers, read-only, owned by the caller. */
typedef struct {
  int64_t num_nodes;      /* |V|, 1 .. 2^31 - 1 */
  int64_t num_edges;      /* |E| = indptr[num_nodes] */
  const void* indptr;     /* [num_nodes + 1] int32 or int64 row offsets */
  int32_t indptr_bits;    /* 32 or 64 */
  int32_t reserved;
  const int32_t* indices; /* [num_edges] source vertex of each edge */
} gmb_csr;

/* One bipartite block of the sampled computation graph (Fig. 1(b)): the
 * messages of model layer l flow from the block's sources to its
 * destinations.  Filled in by gmb_sample_blocks with pointers into the
 * caller's workspace; sizes live on the device.
 *   indptr  [cap_dst + 1]  row offsets: edges of destination p are
 *                          [indptr[p], indptr[p+1]), k_p = min(deg, fanout)
 *   indices [cap_nnz]      local source id of each edge: a position in src_ids
 *   nbr     [cap_nnz]      the same edges as global vertex ids, each row in
 *                          ascending CSR-slot order
 *   src_ids [cap_src]      global ids of the sources; the first n_dst entries
 *                          are the destinations, in order, followed by the
 *                          new vertices in order of first appearance over
 *                          (destination position, slot).  All blocks of one
 *                          call share this array: block l uses its first
 *                          n_src(l) entries, and block 0's sources are the
 *                          input vertices whose features are gathered.
 *   sizes   [4]            device int32: n_dst, n_src, nnz, 0
 * cap_* are host-known upper bounds of the device-side sizes. */
typedef struct {
  int32_t* indptr;
  int32_t* indices;
  int32_t* nbr;
  int32_t* src_ids;
  int32_t* sizes;
  int64_t cap_dst, cap_src, cap_nnz;
  int32_t fanout;
  int32_t layer;
} gmb_block;

typedef struct {
  int32_t num_layers;
  int32_t num_seeds;
  gmb_block blk[GMB_MAX_LAYERS];   /* blk[l] = model layer l */
} gmb_blocks;

/* GraphSAGE-mean weights of an L-layer model (Section IV: 3 layers, hidden
 * 256).  Layer l maps dims[l] -> dims[l+1]:
 *   h_v' = act(h_v W_self[l] + mean_{u in sampled N(v)} h_u W_neigh[l] + bias[l])
 * with act = ReLU for l < L-1 and the identity for the last layer.
 * w_self[l], w_neigh[l]: device, [dims[l]][dims[l+1]] row-major, in `dtype`
 * (fp32, or bf16 bit patterns).  bias[l]: device, [dims[l+1]] fp32.  The
 * input features must have the same dtype as the matrices. */
typedef struct {
  int32_t num_layers;
  int32_t dtype;                       /* gmb_dtype */
  int32_t dims[GMB_MAX_LAYERS + 1];
  const void* w_self[GMB_MAX_LAYERS];
  const void* w_neigh[GMB_MAX_LAYERS];
  const float* bias[GMB_MAX_LAYERS];
} gmb_sage_weights;

/* ---- library ---------------------------------------------------------- */

/* GMB_ABI_VERSION of the loaded library. */
int32_t gmb_abi_version(void);

/* Message of the last failing call on this thread ("" if none). */
const char* gmb_last_error(void);

/* ---- sampler state ---------------------------------------------------- */

/* The sampler keeps one 32-bit slot per vertex (the dedup table of the
 * relabel step) plus a status word, in a caller-owned device buffer that
 * outlives calls: gmb_sampler_state_bytes() bytes for `num_nodes` vertices.
 * gmb_sampler_state_init() clears it (enqueued on `stream`); every
 * gmb_sample_blocks call leaves the table clear again.  One state serves
 * one call at a time: calls that share a state must be ordered on one
 * stream.  Returns 0 for num_nodes outside 1 .. 2^31 - 1. */
size_t gmb_sampler_state_bytes(int64_t num_nodes);
int gmb_sampler_state_init(void* state, size_t state_bytes, int64_t num_nodes, void* stream);

/* Device address of the state's status word (uint32, GMB_STATUS_* bits),
 * for passing to gmb_gather_features; NULL for a NULL state. */
uint32_t* gmb_state_status_word(void* state);

/* Synchronises `stream`, reads and clears the status word and returns the
 * matching status (GMB_ERANGE before GMB_EDUP before GMB_EDEVICE for
 * GMB_STATUS_INTERNAL or GMB_STATUS_INVALID), or GMB_OK.  After GMB_STATUS_INTERNAL it also
 * clears the state's table again (and synchronises once more), since the
 * failed call may have left slots behind. */
int gmb_read_status(void* state, void* stream);

/* ---- sampling (Section II-B, steps (i)-(ii), recursive per layer) ------- */

/* Bytes of workspace gmb_sample_blocks needs for these shapes (0 for bad
 * arguments). */
size_t gmb_sample_workspace_bytes(int32_t num_seeds, const int32_t* fanouts, int32_t num_layers,
                                  int64_t num_nodes);

/* Samples an L-layer mini-batch.
 *   seeds     device int32[num_seeds]: the target vertices, distinct, in
 *             [0, num_nodes) (a duplicate sets GMB_STATUS_EDUP, an id out of
 *             range GMB_STATUS_ERANGE).  num_seeds may be 0.
 *   fanouts   host int32[num_layers], each >= 1: at most fanouts[l]
 *             in-neighbours of each destination of layer l are picked,
 *             uniformly without replacement; a vertex with in-degree
 *             <= fanouts[l] keeps all of them.
 *   seed      64-bit key.  The sample of vertex v at layer l depends only on
 *             (seed, v, l) and the CSR row of v: Philox4x32-10 keyed by
 *             (lo32(seed), hi32(seed)) with counter (v, l, i, r) draws the
 *             i-th number of Floyd's algorithm by Lemire's
 *             multiply-and-reject on words x0..x3 of block r = 0, 1, ...
 *   state     the sampler state of this graph (see above).
 *   ws        device workspace of >= gmb_sample_workspace_bytes(...) bytes,
 *             256-byte aligned; the blocks point into it and stay valid
 *             until the workspace is reused.
 *   out       host struct filled with the blocks' pointers and capacities.
 * No host synchronisation: the sizes stay on the device (gmb_read_sizes). */
int gmb_sample_blocks(const gmb_csr* csr, const int32_t* seeds, int32_t num_seeds,
                      const int32_t* fanouts, int32_t num_layers, uint64_t seed,
                      void* state, size_t state_bytes, void* ws, size_t ws_bytes,
                      gmb_blocks* out, void* stream);

/* ---- sampling without allocation ---------------------------------------- */

/* Bytes of the fixed device scratch of gmb_sample_blocks_noalloc. */
#define GMB_NOALLOC_SCRATCH_BYTES (32u << 20)

/* For callers that cannot allocate device memory or cannot pass a
 * workspace: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  The same sampling as gmb_sample_blocks (same
 * kernels, the same blocks bit for bit), with the scratch that the call
 * needs besides its outputs (the relabel scans' look-back words and tickets,
 * the running edge counts, the dedup's routed pairs and answers) in a fixed
 * array of GMB_NOALLOC_SCRATCH_BYTES
 * that the library holds in device memory, one copy per GPU, from the first
 * call on that GPU until the process ends.  The call allocates nothing.
 *   out_buf    device buffer for the blocks, 256-byte aligned, caller-owned;
 *              gmb_sample_workspace_bytes(...) bytes for the same shapes
 *              always suffice (the blocks take its first part).  The blocks
 *              point into it and stay valid until it is reused.
 *   others     as for gmb_sample_blocks.
 * Errors: those of gmb_sample_blocks, and GMB_ENOSPC when the shapes need
 * more scratch than the fixed array holds (about 12 bytes per edge and per
 * destination of the last hop's capacity: 13 MB for 1000 seeds and fan-outs
 * 15, 10, 5); nothing is enqueued then.  The scratch is cleared by
 * the call's own first kernel.  Every call on one GPU shares that GPU's
 * array: calls that overlap in time on one GPU (other streams, other host
 * threads) race and give wrong blocks, so order them on one stream. */
int gmb_sample_blocks_noalloc(const gmb_csr* csr, const int32_t* seeds, int32_t num_seeds,
                              const int32_t* fanouts, int32_t num_layers, uint64_t seed,
                              void* state, size_t state_bytes, void* out_buf, size_t out_bytes,
                              gmb_blocks* out, void* stream);

/* Debug check of sampled blocks (run after every gmb_sample_blocks and
 * gmb_sample_blocks_noalloc call when the environment variable GMB_VALIDATE
 * is set to 1): enqueues on `stream` a device check of each block's
 * invariants (sizes within the capacities; row offsets rising from 0 to nnz
 * with at most `fanout` edges per row; every edge's local id below n_src and
 * naming the edge's sampled vertex in src_ids; every sampled vertex inside
 * the graph).  A violation sets GMB_STATUS_INVALID in the state's status
 * word, which gmb_read_status reports as GMB_EDEVICE.  The check reads only
 * within the blocks' capacities, whatever their size words hold.  It does
 * not check that src_ids is duplicate-free (the oracle tests do). */
int gmb_validate_blocks(const gmb_csr* csr, const gmb_blocks* blocks, void* state, void* stream);

/* Synchronises `stream` and copies the device sizes to host
 * sizes[num_layers][3] = {n_dst, n_src, nnz} (layer order). */
int gmb_read_sizes(const gmb_blocks* blocks, int64_t* sizes, void* stream);

/* ---- feature gather (KVStore pull, Section III-C) ---------------------- */

/* out[i, :] = feats[ids[i], :] bit for bit, for i < n, where n = *n_dev
 * (device int32, e.g. block 0's n_src) clamped to n_cap, or n = n_cap when
 * n_dev is NULL.  Rows at i >= n are not written.
 *   ids    device int32[n_cap]
 *   feats  device [num_nodes, dim] row-major, element size from dtype
 *   out    device [n_cap, dim]
 *   status device uint32 status word or NULL: an id outside [0, num_nodes)
 *          sets GMB_STATUS_ERANGE there and its output row is zero-filled. */
int gmb_gather_features(const int32_t* ids, const int32_t* n_dev, int64_t n_cap, const void* feats,
                        int64_t num_nodes, int32_t dim, int32_t dtype, void* out, uint32_t* status,
                        void* stream);

/* ---- GraphSAGE-mean forward (Eq. (1), Section IV model) ----------------- */

/* Bytes of workspace gmb_sage_forward needs (0 for bad arguments). */
size_t gmb_forward_workspace_bytes(const gmb_blocks* blocks, const gmb_sage_weights* weights);

/* Byte offset in the forward workspace of the output of layer l < L-1
 * (the hidden activations, [n_dst(l), dims[l+1]] in the weights' dtype);
 * -1 for a bad layer. */
int64_t gmb_forward_hidden_offset(const gmb_blocks* blocks, const gmb_sage_weights* weights,
                                  int32_t layer);

/* Runs the L layers over the blocks (the workspace keeps every layer's
 * mean and hidden output, which gmb_sage_backward reads).
 *   x       device [blocks->blk[0].cap_src, dims[0]] in weights->dtype: the
 *           gathered input features of block 0's sources (rows beyond
 *           n_src are not read).
 *   logits  device fp32 [num_seeds, dims[L]].
 *   ws      device workspace of >= gmb_forward_workspace_bytes() bytes,
 *           256-byte aligned.
 * Per layer: the mean of the sampled in-neighbours' rows (0 for a vertex
 * with none) accumulated in fp32, then the two products and the bias in
 * one matrix-core GEMM with fp32 accumulation.  In fp32 mode, where d_in and
 * the rows allow it, every operand is cut exactly into three bf16 parts and a
 * product is the sum of six of the nine part products (eight at some widths);
 * what is left out is below 2^-21 of the product, and the results' error is of
 * the order of an fp32 sum's.  In bf16 mode the mean and the hidden activations
 * are rounded to bf16 before the next product.
 * An empty batch (num_seeds == 0) has no rows in any layer: nothing is
 * enqueued, and x and logits may be NULL. */
int gmb_sage_forward(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                     float* logits, void* ws, size_t ws_bytes, void* stream);

/* The forward of gmb_sage_forward with the feature pull of Section III-C
 * folded into layer 0: instead of a gathered copy of every input row, the
 * layer-0 mean reads the sampled neighbours' rows straight from the feature
 * table by their global ids (block 0's nbr array), and only block 0's
 * destination rows, which its linear term h_v W_self needs, are gathered
 * into x_dst.  The results are bit for bit those of gmb_sage_forward on
 * the same blocks and weights (the same rows are summed in the same order).
 *   feats      device [num_nodes, dims[0]] in weights->dtype, read-only.
 *   num_nodes  rows of feats (1 .. 2^31 - 1).
 *   x_dst      device [blocks->blk[0].cap_dst, dims[0]] in weights->dtype,
 *              caller-owned, written with the destination rows; it stands
 *              for `x` in a later gmb_sage_backward (which reads layer 0's
 *              destination rows only).
 *   status     NULL or the sampler state's status word
 *              (gmb_state_status_word): an id outside [0, num_nodes) in
 *              the gather sets GMB_STATUS_ERANGE there and gives a zero row;
 *              in the mean it is read as row 0.
 *   others     as for gmb_sage_forward (same workspace size; with
 *              num_seeds == 0 nothing is enqueued and x_dst and logits
 *              may be NULL). */
int gmb_sage_forward_fused(const gmb_blocks* blocks, const void* feats, int64_t num_nodes, void* x_dst,
                           const gmb_sage_weights* weights, float* logits, void* ws, size_t ws_bytes,
                           uint32_t* status, void* stream);

/* ---- training step (the trainer's iteration of Section III-E) ---------- */

/* Gradient arrays of an L-layer model, one per weight array, fp32 and laid
 * out like the weights (d_self[l], d_neigh[l]: [dims[l]][dims[l+1]],
 * d_bias[l]: [dims[l+1]]).  Device pointers, caller-owned. */
typedef struct {
  int32_t num_layers;
  int32_t reserved;
  float* d_self[GMB_MAX_LAYERS];
  float* d_neigh[GMB_MAX_LAYERS];
  float* d_bias[GMB_MAX_LAYERS];
} gmb_sage_grads;

/* Bytes of workspace gmb_sage_backward needs (0 for bad arguments,
 * including a model the training step does not support: hidden dims not a
 * multiple of 4, a dims[l] above 640 for l >= 2).  For bf16 weights it
 * includes fp32 copies of what the backward reads. */
size_t gmb_backward_workspace_bytes(const gmb_blocks* blocks, const gmb_sage_weights* weights);

/* Gradients of the loss L = (1/B) sum over the B seeds of the softmax
 * cross-entropy of the seed's logits against its label, in every weight
 * and bias (the input features are not trained).  Node classification is
 * the task the paper trains (Section IV); its loss is not printed, this is
 * the standard one.  The backward follows Eq. (1) layer by layer from the
 * last: with dZ the gradient at a layer's pre-activation (ReLU passes it
 * where the layer's output is > 0), dW_self = H_dst^T dZ, dW_neigh = M^T dZ,
 * db = the column sums of dZ, and the layer input receives dZ W_self^T on
 * its destination rows plus, over every block edge (v <- u), its share
 * (dZ W_neigh^T)[v] / k_v of the mean.
 *   blocks, x, weights  as given to the gmb_sage_forward call that produced
 *                       `logits`, fp32 or bf16.  A bf16 model's backward
 *                       first widens the upper layers' rows (each layer
 *                       l >= 1: its destination rows and its kept mean) and
 *                       the matrices to fp32 (inside `ws`); layer 0's rows
 *                       and mean and every ReLU mask are read as bf16, a
 *                       value that fp32 holds exactly.  fp32 products, fp32
 *                       gradients (update with gmb_sgd_update_bf16).
 *   logits   device fp32 [num_seeds, dims[L]] from that call.
 *   labels   device int32 [num_seeds], the class of each seed in
 *            [0, dims[L]) (a label outside it is a data error: that row's
 *            loss term is 0 and its gradient unspecified, in bounds).
 *   fwd_ws   that call's workspace (it keeps every layer's mean and hidden
 *            output), unchanged since; fwd_ws_bytes its size.
 *   grads    where the gradients go (overwritten).
 *   loss     device fp32 scalar receiving L, or NULL.
 *   ws       device workspace of >= gmb_backward_workspace_bytes() bytes,
 *            256-byte aligned.
 * An empty batch (num_seeds == 0): the loss, a mean over no seeds, is
 * taken as 0, every gradient array is set to 0, and x, logits and labels
 * may be NULL.
 * Each weight gradient is summed over the rows in a fixed order (no
 * atomics), so the last layer's gradients are the same on every run.  The
 * gradient that flows into the input of layers >= 1 is pulled per source
 * vertex from a transpose of the block whose entries take their slots by
 * atomic counters, so each source's terms are summed in an order that can
 * change between runs, and the gradients of the layers below the last can
 * differ in their last bits.  The transpose's offsets come from a
 * single-pass scan whose tiles wait for their predecessors in a bounded
 * loop (about 4M short sleeps); only a GPU that stalls a running tile for
 * that long makes a wait give up.  The input gradients of that layer are
 * unknown then: the weight gradients of the layers below it are NaN, and so
 * is the loss (with loss NULL: the first entry of d_bias[0]). */
int gmb_sage_backward(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                      const float* logits, const int32_t* labels, const void* fwd_ws, size_t fwd_ws_bytes,
                      const gmb_sage_grads* grads, float* loss, void* ws, size_t ws_bytes, void* stream);

/* ---- learnable vertex embeddings (Section III-C, Section III-E) -------- */

/* Bytes of workspace gmb_sage_backward_embedding needs (0 for bad arguments,
 * including a model it does not support: those of gmb_sage_backward, and
 * dims[0] or dims[1] breaking the same limits as the hidden widths). */
size_t gmb_backward_embedding_workspace_bytes(const gmb_blocks* blocks, const gmb_sage_weights* weights);

/* gmb_sage_backward for a model whose layer-0 inputs are learnable vertex
 * embeddings (the transductive case of Section III-C): besides the weight
 * gradients it takes the gradient in layer 0's input rows,
 * dX = dZ_0 W_self^T on the destination rows plus, over every block-0 edge
 * (v <- u), (dZ_0 W_neigh^T)[v] / k_v on row u (no activation acts on the
 * input), and applies it at once as the sparse SGD step of the paper's
 * embeddings (Section III-E): table[src_ids[u]] -= emb_lr * dX[u] for every
 * input vertex u of block 0.  dX is never stored.
 *   x          as for gmb_sage_backward: the gathered input rows (those
 *              of table), or x_dst of gmb_sage_forward_fused run on table.
 *   table      device fp32 [num_nodes, dims[0]], 16-byte aligned, updated
 *              in place (rows of vertices outside the mini-batch are not
 *              touched).
 *   emb_lr     the embeddings' step size.
 *   ws         >= gmb_backward_embedding_workspace_bytes() bytes.
 * The rows of one mini-batch are distinct, so the update needs no atomics;
 * calls in flight together on several streams update the shared table
 * without locks (asynchronous SGD as in Hogwild, as the paper updates its
 * embeddings), and a gather running meanwhile may see old or new rows.
 * If a wait of block 0's transpose gives up (see gmb_sage_backward), no row
 * changes and the loss is NaN (with loss NULL: the first entry of d_bias[0]).
 * An empty batch changes no row (the gradients and the loss as for
 * gmb_sage_backward). */
int gmb_sage_backward_embedding(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                                const float* logits, const int32_t* labels, const void* fwd_ws, size_t fwd_ws_bytes,
                                const gmb_sage_grads* grads, float* loss, void* ws, size_t ws_bytes, float* table,
                                int64_t num_nodes, float emb_lr, void* stream);

/* One SGD step: every weight array W -= lr * dW, every bias b -= lr * db,
 * in place on the device arrays that `weights` points to (fp32). */
int gmb_sgd_update(const gmb_sage_weights* weights, const gmb_sage_grads* grads, float lr, void* stream);

/* One SGD step of a bf16 model (the trainer's update of Section III-E with
 * the dense parameters kept in fp32): the fp32 master weights `master`
 * (same dims, dtype GMB_F32) take W -= lr * dW and b -= lr * db, then
 * every bf16 matrix of `weights` becomes its master rounded to the nearest
 * bf16 (ties to even), and each bias of `weights`, when it is not the
 * master's own array, a copy of the master's.  All device arrays,
 * caller-owned, updated in place on `stream`. */
int gmb_sgd_update_bf16(const gmb_sage_weights* weights, const gmb_sage_weights* master, const gmb_sage_grads* grads,
                        float lr, void* stream);

/* ---- microscaled vertex store ------------------------------------------- */

/* The feature (or embedding) rows of the key-value store (Section III-C) in
 * 4 or 8 bits an element: a quarter to an eighth of the bytes that every
 * pull and every mean moves.  A row of `dim` elements is a record of
 * gmb_mx_row_bytes(dim, format) bytes:
 *   - its elements in nb = ceil(dim / 32) blocks of 32.  GMB_MXFP4: 16 bytes
 *     a block, element i in half i % 2 of byte i / 2 (0: the low half), sign
 *     bit, then the magnitudes 0 .5 1 1.5 2 3 4 6; GMB_MXFP8: 32 bytes, e4m3
 *     (bias 7, largest value 448, code 0x7F not a number).  Elements past dim
 *     are 0;
 *   - nb scale bytes c, the block's scale being 2^(c - 127), 255 not a number;
 *   - zeros up to a multiple of 16 bytes.
 * A table of records has an address and a row stride that are multiples of
 * 16 (the stride at least a record; bytes between record and stride are not
 * touched).  dim is 1 .. 65536, a table's rows 1 .. 2^31 - 1.
 * Quantising takes c = max(e - s, 0) with e the fp32 exponent field of the
 * block's largest magnitude and s = 2 (4 bits) or 8 (8 bits), and rounds
 * x / 2^(c - 127) to the nearest element, ties to even; what lies past the
 * largest element becomes it.  A block that holds an infinity or NaN gets
 * c = 255 and reads back as NaN.  Values of 4 or 8 bits are exact in fp32,
 * and in bf16 unless a bf16 denormal cannot hold them. */

/* Bytes of a record (0 for a bad dim or format). */
int64_t gmb_mx_row_bytes(int32_t dim, int32_t format);

/* Quantises rows into a table: record r_i = x[i, :] for i < n, where n = *n_dev
 * clamped to n_cap, or n_cap when n_dev is NULL; r_i = ids[i], or i when ids
 * is NULL (n_cap at most num_rows then).
 *   x       device, element (i, j) at i * row_stride + j * col_stride elements
 *           of `dtype` (strides >= 0): rows, or the columns of a weight matrix
 *           [d_in][d_out] (row_stride 1, col_stride d_out) that
 *           gmb_mx_linear wants as rows.  Rows need no alignment.
 *   ids     device int32[n_cap] or NULL.  An id outside [0, num_rows) sets
 *           GMB_STATUS_ERANGE and its row is not written.
 *   state   NULL: the ids are distinct (as a block's src_ids are); records of
 *           an id that comes twice are unspecified.  Else the sampler state
 *           of a graph of num_rows vertices: an id may come any number of
 *           times and its last row is what the record holds.  The state's
 *           table is left clear; calls that share it must be ordered on one
 *           stream.
 *   status  device status word or NULL (with a state: the state's). */
int gmb_mx_quantise(const void* x, int32_t dtype, int64_t row_stride, int64_t col_stride, const int32_t* ids,
                    const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t format, void* table, int64_t num_rows,
                    int64_t table_stride, void* state, size_t state_bytes, uint32_t* status, void* stream);

/* gmb_gather_features from a store: out[i, :] = the values of record ids[i]
 * (record i when ids is NULL), i < n as above, as fp32 or bf16 (`dtype`).
 *   out  device [n_cap, dim] row-major; rows at i >= n are not written; a row
 *        whose id is outside [0, num_rows) is zero-filled and sets
 *        GMB_STATUS_ERANGE in `status` (device word or NULL). */
int gmb_mx_gather(const int32_t* ids, const int32_t* n_dev, int64_t n_cap, const void* table, int64_t num_rows,
                  int64_t table_stride, int32_t dim, int32_t format, void* out, int32_t dtype, uint32_t* status,
                  void* stream);

/* The mean of Eq. (1) straight from a store: out[v, :] = (1 / k_v) times the
 * sum over e in [indptr[v], indptr[v + 1]) of the values of record ids[e], 0
 * for an empty range, fp32 sums.
 *   indptr  device int32[n_cap + 1], rising (a block's row offsets)
 *   ids     device int32, a record of the table for every e (a block's nbr);
 *           one outside [0, num_rows) is read as record 0
 *   n_dev   device int32 or NULL: destinations, clamped to n_cap (a block's
 *           sizes[0])
 *   out     device [n_cap, dim] of `dtype`. */
int gmb_mx_mean(const int32_t* indptr, const int32_t* ids, const int32_t* n_dev, int64_t n_cap, const void* table,
                int64_t num_rows, int64_t table_stride, int32_t dim, int32_t format, void* out, int32_t dtype,
                void* stream);

/* One operand of a product: GMB_MXFP4 records of d_in elements.
 *   rows     [num_rows], row i of the product being ids[i], or i without ids
 *            (an id outside the table counts as a row of zeros and sets
 *            GMB_STATUS_ERANGE)
 *   weights  [d_out]: output column j's weights, quantised along d_in. */
typedef struct {
  const void* rows;
  int64_t num_rows, row_stride;
  const int32_t* ids;
  const void* weights;
  int64_t weight_stride;
} gmb_mx_operand;

/* out = act(A W^T [+ A2 W2^T] + bias), the linear layer of Eq. (1) with
 * microscaled 4-bit rows and weights: exact products, fp32 sums on the
 * scaled matrix instructions.  No gradient: a model is trained on its fp32
 * masters (gmb_sage_backward on what the records stand for) and quantised
 * again.
 *   a, a2   the operands (a2 may be NULL; its ids must be)
 *   n_dev   device int32 or NULL: rows, clamped to n_cap (at most 2^31 - 1024)
 *   bias    device fp32 [d_out] or NULL; relu: nonzero for max(0, .)
 *   out     device [n_cap, d_out] of `dtype`. */
int gmb_mx_linear(const gmb_mx_operand* a, const gmb_mx_operand* a2, const int32_t* n_dev, int64_t n_cap,
                  int32_t d_in, int32_t d_out, const float* bias, int32_t relu, void* out, int32_t dtype,
                  uint32_t* status, void* stream);

/* A GraphSAGE-mean model in GMB_MXFP4: w_self[l], w_neigh[l] device records,
 * dims[l+1] rows of dims[l] elements at a stride of gmb_mx_row_bytes(dims[l])
 * (the transposes of gmb_sage_weights' matrices), bias[l] device fp32. */
typedef struct {
  int32_t num_layers;
  int32_t dims[GMB_MAX_LAYERS + 1];
  const void* w_self[GMB_MAX_LAYERS];
  const void* w_neigh[GMB_MAX_LAYERS];
  const float* bias[GMB_MAX_LAYERS];
} gmb_sage_mx_weights;

/* Bytes of workspace gmb_sage_forward_mx needs (0 for bad arguments), and the
 * byte offset there of layer l's mean records (hidden 0, [n_dst(l)] of
 * dims[l]) or hidden records (hidden 1, l < L-1, of dims[l+1]); -1 for a bad
 * layer. */
size_t gmb_mx_forward_workspace_bytes(const gmb_blocks* blocks, const gmb_sage_mx_weights* weights);
int64_t gmb_mx_forward_offset(const gmb_blocks* blocks, const gmb_sage_mx_weights* weights, int32_t layer,
                              int32_t hidden);

/* gmb_sage_forward_fused of such a model over a GMB_MXFP4 store: layer 0's
 * mean and its linear term read the store by the vertices' ids, and every
 * layer's mean and hidden output is quantised (GMB_MXFP4) as it is written.
 *   table   the store, num_nodes records of dims[0]
 *   logits  device fp32 [num_seeds, dims[L]]
 *   ws      device workspace, 256-byte aligned
 *   status  NULL or a status word: an id outside the store sets
 *           GMB_STATUS_ERANGE (zeros in the linear term, record 0 in the mean)
 * An empty batch enqueues nothing (logits may be NULL). */
int gmb_sage_forward_mx(const gmb_blocks* blocks, const void* table, int64_t num_nodes, int64_t table_stride,
                        const gmb_sage_mx_weights* weights, float* logits, void* ws, size_t ws_bytes,
                        uint32_t* status, void* stream);

/* ---- distillation -------------------------------------------------------- */

#define GMB_MAX_TEACHER 1024

/* A teacher's top logits, `top` (1 .. GMB_MAX_TEACHER) entries a row, and how
 * the student is held to them: temperature T (0.001 .. 1000) and weight alpha
 * (0 .. 1).
 *   logits   device fp32 [rows, top]
 *   classes  device int32 [rows, top], each entry's class.  An entry whose
 *            class is outside [0, C) (-1 pads a shorter list) or whose logit
 *            is -inf is left out; entries of one class add up. */
typedef struct {
  const float* logits;
  const int32_t* classes;
  int32_t top;
  float alpha;
  float temperature;
  int32_t reserved;
} gmb_teacher;

/* Bytes of workspace gmb_distill_loss needs (0 for bad arguments). */
size_t gmb_distill_workspace_bytes(int64_t rows, int32_t classes);

/* The mean over the rows of
 *   alpha T^2 KL(p || softmax(z / T)) + (1 - alpha) (-log softmax(z)_y)
 * and its gradient in the logits z, with p the softmax of the row's teacher
 * entries over T.  A row without entries lacks the first term, one whose
 * label is outside [0, classes) the second, and one whose logits are all
 * -inf both; their gradients are 0.  (A logit of -inf is a class that cannot
 * be: probability 0; the loss is infinite if the teacher gives it more.)
 * Sums and statistics are fp32, the mean over the rows 64 bits, in a fixed order.
 *   logits   device [rows, classes] fp32 or bf16 (`dtype`)
 *   labels   device int32 [rows] or NULL (no second term)
 *   dlogits  device [rows, classes] of `dtype`, or NULL for the loss alone;
 *            apart from the logits (GMB_EINVAL if they overlap)
 *   loss     device fp32 scalar (0 for no rows)
 *   ws       device workspace, 256-byte aligned. */
int gmb_distill_loss(const void* logits, int32_t dtype, int64_t rows, int32_t classes, const gmb_teacher* teacher,
                     const int32_t* labels, void* dlogits, float* loss, void* ws, size_t ws_bytes, void* stream);

/* gmb_sage_backward (table NULL), or gmb_sage_backward_embedding (table the
 * embeddings), from that loss instead of the cross-entropy: the same
 * workspaces (gmb_backward_workspace_bytes, or the embedding's) and
 * arguments; labels may be NULL; at most 32,768 classes. */
int gmb_sage_backward_distill(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                              const float* logits, const gmb_teacher* teacher, const int32_t* labels,
                              const void* fwd_ws, size_t fwd_ws_bytes, const gmb_sage_grads* grads, float* loss,
                              void* ws, size_t ws_bytes, float* table, int64_t num_nodes, float emb_lr,
                              void* stream);

/* ---- dropout, norm and loss of a residual model ------------------------- */

/* Rows of `dim` contiguous elements, row i at data + i * stride elements
 * (stride >= dim; no alignment beyond the element's own). */
typedef struct {
  void* data;
  int64_t stride;
} gmb_rows;

/* A dropout whose mask is never stored: it is drawn again wherever it is
 * needed, in the backward for instance.  Which elements are dropped is a
 * function of the seed, the row's key, the layer, the column and *step:
 * Philox4x32-10 keyed by (lo32(seed), hi32(seed)) with counter (key, 2^31 +
 * layer, column / 8, *step); columns 8 c .. 8 c + 7 take the low and high
 * halves of its words x0 .. x3 in order, and an element is dropped where its
 * 16 bits are below t = round(65536 p).  (The sampler's counters hold a layer
 * below 2^31 in their second word: one seed serves both.)  Dropped elements
 * become 0, whatever they hold; the others are multiplied by 65536 / (65536 -
 * t) in fp32.
 *   p      0 .. 1
 *   layer  0 .. 2^31 - 1: masks of different layers are independent
 *   step   device uint32 or NULL (0), read by the kernels: a captured graph
 *          whose step moves draws another mask at every replay. */
typedef struct {
  uint64_t seed;
  float p;
  int32_t layer;
  const uint32_t* step;
} gmb_dropout;

/* out[i, :] = [residual[i, :] +] dropout(x[i, :]) for i < n, where n = *n_dev
 * clamped to n_cap, or n_cap when n_dev is NULL; rows at i >= n are not
 * written.  Row i's key is ids[i] (a vertex: the same mask wherever it stands
 * in a batch), or i when ids is NULL.  fp32 sums, rounded once to `dtype`.  The
 * backward is the same call on the gradient (without residual).
 *   x, residual, out  rows of `dtype`; residual may be NULL; out may be x or
 *                     residual (the same address and stride), not overlap
 *                     them otherwise
 *   ids               device int32[n_cap] or NULL
 *   dim               1 .. 65536; n_cap 0 .. 2^31 - 1 */
int gmb_dropout_rows(const gmb_rows* x, const gmb_rows* residual, const gmb_dropout* drop, const int32_t* ids,
                     const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t dtype, const gmb_rows* out,
                     void* stream);

/* The root-mean-square norm of a sum, for rows i < n as above:
 *   r = [residual +] x, x dropped out first with `drop` (NULL: not),
 *   y = weight r / sqrt(mean(r^2) + eps),
 * with r rounded to `dtype` before it is normed (what `sum` holds is what y is
 * the norm of, and what gmb_rms_norm_backward takes); statistics fp32.
 *   weight  device fp32 [dim] or NULL (ones)
 *   eps     a positive normal number (>= 2^-126).  A row whose squares add up
 *           past fp32's range norms to 0
 *   sum     rows of `dtype` for r, or NULL; may be x or residual
 *   format  0: out is rows of `dtype` (out may be x or residual if sum is
 *           not); GMB_MXFP4 or GMB_MXFP8: out is records (a table of
 *           gmb_mx_quantise: 16-byte aligned, its stride in bytes, a multiple
 *           of 16), quantised from fp32. */
int gmb_rms_norm(const gmb_rows* x, const gmb_rows* residual, const gmb_dropout* drop, const int32_t* ids,
                 const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t dtype, const float* weight, float eps,
                 const gmb_rows* sum, int32_t format, const gmb_rows* out, void* stream);

/* Bytes of workspace gmb_rms_norm_backward needs for d_weight (0 for bad
 * arguments). */
size_t gmb_rms_norm_workspace_bytes(int64_t n_cap, int32_t dim);

/* The gradients of gmb_rms_norm with format 0, for rows i < n as above:
 * with s = 1 / sqrt(mean(r^2) + eps),
 *   dr = carry + s (weight dy - r s^2 mean(weight dy r)),
 * the gradient of the residual; that of x is dropout(dr); that of the weight
 * the sum over the rows of dy r s, in a fixed order (no atomics).  A row that
 * normed to 0 (see eps) passes the carry alone.
 *   dy, r        the gradient of y, and the sum (x itself if nothing was added)
 *   carry        the gradient that reaches r from elsewhere, or NULL
 *   d_residual   rows or NULL; may be dy, r or carry
 *   dx           rows or NULL; the same, and not d_residual
 *   d_weight     device fp32 [dim] or NULL (0 if there are no rows)
 *   ws           >= gmb_rms_norm_workspace_bytes() bytes, 256-byte aligned
 *                (NULL without d_weight). */
int gmb_rms_norm_backward(const gmb_rows* dy, const gmb_rows* r, const gmb_rows* carry, const gmb_dropout* drop,
                          const int32_t* ids, const int32_t* n_dev, int64_t n_cap, int32_t dim, int32_t dtype,
                          const float* weight, float eps, const gmb_rows* d_residual, const gmb_rows* dx,
                          float* d_weight, void* ws, size_t ws_bytes, void* stream);

/* A linear head over many classes (every vertex may be one: W is the
 * embedding table then): logits z = x W^T + bias.
 *   x       device [rows, d] of `dtype` at x_stride elements (>= d)
 *   w       device, element j of class c at c * w_row_stride + j *
 *           w_col_stride elements of `dtype` (strides >= 0): rows [classes][d],
 *           or the columns of a [d][classes] matrix
 *   bias    device fp32 [classes] or NULL (-inf: a class that cannot be; so is one
 *           below -2.35e38, as logits are held times log2(e): a mask of the type's
 *           lowest value is one of -inf)
 *   labels  device int32 [rows]; a row whose label is outside [0, classes)
 *           has no loss and no gradient, whatever x holds there
 *   rows 0 .. 2^22, d 1 .. 65536, classes 1 .. 2^27 */
typedef struct {
  const void* x;
  int64_t x_stride;
  const void* w;
  int64_t w_row_stride, w_col_stride;
  const float* bias;
  const int32_t* labels;
  int64_t rows;
  int32_t d, classes, dtype, reserved;
} gmb_linear_head;

/* Its gradients, each NULL if it is not wanted, apart from the inputs:
 *   dx    device [rows, d] of the head's dtype
 *   dw    device [classes, d] of the head's dtype, or with `turned` [d, classes]
 *   bias  device fp32 [classes] */
typedef struct {
  void* dx;
  void* dw;
  float* dbias;
  int32_t turned, reserved;
} gmb_linear_grads;

/* Bytes of workspace gmb_linear_loss needs (0 for bad arguments); of the
 * pointers of `grads` (NULL: the loss alone) only NULL or not counts, of w its
 * alignment.  It holds 16-bit copies of x and, unless it is bf16 in aligned rows
 * of a multiple of 64 values, of W (fp32: two of x; rows rounded up to 64 values),
 * and with gradients those of the logits, G = softmax(z) - onehot, of a piece of the
 * classes: 384 MB at most (more from 393,216 rows on), and that piece's sums where
 * they are split: of dw 128 MB at most, of dx 64 MB more than its own size in fp32,
 * of dbias a 32nd of G.  Few rows or classes: none of these, 64 MB of sums at most.
 * The logits are never stored.  0 too where the three extents together are more
 * than a launch takes. */
size_t gmb_linear_loss_workspace_bytes(const gmb_linear_head* head, const gmb_linear_grads* grads);

/* The mean over the rows (those without a label count as 0) of -log
 * softmax(z)_label, and its gradients.  A row whose logits are all -inf has
 * neither.  x and W are finite; with a NaN or an infinity among them the loss
 * is NaN, or the row of that x.  Logits are fp32; a row's sum of exponentials is
 * 64 bits from tile to tile, its loss and probabilities go by the distance to its
 * largest logit.  bf16: exact products, fp32 sums, softmax(z) - onehot rounded to
 * bf16 before its products (not for dbias).  fp32: few rows or
 * classes by fp32 products; else every operand is cut into two fp16 parts at a
 * power-of-two scale (x by rows for the logits; W, and x for dw, as a whole), a
 * product is three of the four part products; the error is of the order of an
 * fp32 sum's beside the operand's largest value (elements below 2^-16 of it lose
 * bits, below 2^-39 of it are lost; so are gradients of a logit below 2^-39).
 * Nothing is added by atomics: the same bits every time.  The mean is summed in
 * 64 bits.
 *   loss  device fp32 scalar
 *   ws    device workspace, 256-byte aligned. */
int gmb_linear_loss(const gmb_linear_head* head, const gmb_linear_grads* grads, float* loss, void* ws,
                    size_t ws_bytes, void* stream);

/* ---- a model trained with dropout, from a gradient at its outputs -------- */

/* gmb_sage_forward (feats NULL), or gmb_sage_forward_fused (feats the table, x
 * its x_dst), with `drop` on every hidden output: layer l < L-1's rows, after
 * the ReLU, are dropped out in place with layer drop->layer + l, keyed by their
 * vertices (in a bf16 model the scaled rows are rounded once more).  (Without it:
 * evaluation.)  Its backward is gmb_sage_backward_from with the same `drop`: the
 * workspace does not say that its rows were dropped out, and gmb_sage_backward,
 * _embedding and _distill, which take no dropout, would leave out its factor in
 * the layers below. */
int gmb_sage_forward_dropout(const gmb_blocks* blocks, void* x, const void* feats, int64_t num_nodes,
                             const gmb_sage_weights* weights, const gmb_dropout* drop, float* logits, void* ws,
                             size_t ws_bytes, uint32_t* status, void* stream);

/* gmb_sage_backward (table NULL), or gmb_sage_backward_embedding, from the
 * gradient at the model's outputs instead of a loss: d_logits device fp32
 * [num_seeds, dims[L]] (a loss of the caller's own, or layers behind the
 * model).  `drop`: as in the forward, or NULL.  If a bounded wait on the device
 * runs out, the first entry of d_bias[0] is NaN. */
int gmb_sage_backward_from(const gmb_blocks* blocks, const void* x, const gmb_sage_weights* weights,
                           const float* d_logits, const gmb_dropout* drop, const void* fwd_ws, size_t fwd_ws_bytes,
                           const gmb_sage_grads* grads, void* ws, size_t ws_bytes, float* table, int64_t num_nodes,
                           float emb_lr, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* GMB_H */
