/*
 * fusco.h - C boundary of the MI355X (gfx950) MoE token shuffle with the layout transformation
 * fused into the data movement.
 *
 * The library turns the router's token-expert matrix into a two-level layout descriptor
 * (fusco_plan), moves token rows straight to their final expert-major rows (fusco_dispatch) and
 * brings expert outputs back into token order with the gate weights (fusco_combine).
 *
 * Conventions for every entry point
 *   - Pointers named d_* are DEVICE pointers into memory owned by the caller.  The library never
 *     allocates, frees or keeps device memory, and never synchronises: each call only enqueues
 *     kernels on `stream` (a hipStream_t passed as void*; NULL is the default stream).
 *   - Device pointers must be 16-byte aligned.  Buffers must not overlap, except that the y
 *     argument of fusco_combine may be the expert buffer fusco_dispatch wrote.
 *   - Return value: FUSCO_OK (0) when the work was enqueued, a negative FUSCO_ERR_* otherwise.
 *     On an error nothing is launched.
 *   - A layout with N == 0 is valid everywhere: sizes are still checked, tensor pointers (all of
 *     them empty then) may be NULL, nothing is launched by the movers and FUSCO_OK is returned.
 *   - Expert-parallel devices are D virtual partitions of one GPU's buffers.  Expert e lives on
 *     device e / (E / D) (contiguous placement; E must be a multiple of D).
 *   - All row orders are deterministic: rows of one expert, and rows of one device's receive
 *     tensor, are in ascending token order.
 */
#ifndef FUSCO_H
#define FUSCO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FUSCO_VERSION 110

#define FUSCO_OK 0
#define FUSCO_ERR_INVALID_ARG (-1) /* null pointer, size out of range, misaligned pointer or row size */
#define FUSCO_ERR_WORKSPACE (-2)   /* caller-provided memory too small                               */
#define FUSCO_ERR_UNSUPPORTED (-3) /* dtype or flag combination not implemented                       */
#define FUSCO_ERR_HIP (-4)         /* the HIP runtime refused a launch                                */
#define FUSCO_ERR_STATIC_LIMIT (-5) /* fusco_plan_static: the input needs more scratch than the static buffer */

#define FUSCO_MAX_K 64   /* experts per token                    */
#define FUSCO_MAX_E 1024 /* experts (and therefore devices)      */
#define FUSCO_MAX_ROW_BYTES (1u << 20) /* one row of the movers, both planes of a dispatch together */
#define FUSCO_STATIC_SCRATCH_BYTES (4u << 20) /* planner scratch held by the library for fusco_plan_static */

/* element types of fusco_combine */
#define FUSCO_BF16 0
#define FUSCO_F32 1

/* scores of fusco_route */
#define FUSCO_SCORE_SOFTMAX 0
#define FUSCO_SCORE_SIGMOID 1
#define FUSCO_MAX_GROUPS 64 /* groups of experts */

/* gate of fusco_norm_after */
#define FUSCO_GATE_NONE 0
#define FUSCO_GATE_CHANNEL 1 /* one value per column, shared by all tokens */
#define FUSCO_GATE_TOKEN 2   /* one value per token, shared by all columns */
#define FUSCO_MAX_NORM_H 32768 /* columns of the norms */

/* flags of fusco_dispatch (no tensor flag means FUSCO_DISPATCH_EXPERT) */
#define FUSCO_DISPATCH_EXPERT 1u /* write the expert-activation tensor (level 2 result)       */
#define FUSCO_DISPATCH_WIRE 2u   /* write the deduplicated per-device receive tensors (level 1) */
#define FUSCO_DISPATCH_TWO_HOP 4u /* hop by hop: x -> receive tensors -> expert tensor (implies both) */
#define FUSCO_DISPATCH_STREAMING 8u /* modifier: write the rows past the memory-side cache (see fusco_dispatch) */

/*
 * Layout descriptor: the two-level descriptor lists of the paper's Communication Planner
 * (section 3.3, the paragraph on the descriptor-level plan) for fixed-size segments.  A segment is one
 * token row, so a segment descriptor (address, size) collapses to a row index.
 *
 * N tokens, k experts per token, E experts, D devices, P = N * k (token, expert) pairs.
 * Pair index p = t * k + j.  "slot" = row in the expert-activation tensor [P rows], ordered by
 * device, then expert, then token.  "send row" = row in the concatenated per-device receive
 * tensors [U rows, U = send_off[D]], ordered by device, then token; a token has one send row per
 * distinct destination device (first appearance of the device among its k entries).
 * All arrays live in device memory carved by fusco_layout_bind.
 */
typedef struct fusco_layout {
    int32_t N, k, E, D, P;
    int32_t send_cap;        /* rows reserved for send_src and a wire buffer: N * min(k, D)          */
    int32_t *exp_count;      /* [E]    rows per expert                                                */
    int32_t *exp_off;        /* [E+1]  exclusive prefix sum of exp_count; exp_off[E] == P             */
    int32_t *send_count;     /* [D]    send rows per device                                           */
    int32_t *send_off;       /* [D+1]  exclusive prefix sum of send_count; send_off[D] == U           */
    int32_t *pair_slot;      /* [P]    pair -> slot                 (level-2 receive descriptor)      */
    int32_t *slot_pair;      /* [P]    slot -> pair                                                   */
    int32_t *slot_token;     /* [P]    slot -> token                (source-token index)              */
    int32_t *send_src;       /* [send_cap] send row -> token; rows >= U are not written (level-1 send) */
    int32_t *pair_send_row;  /* [P]    pair -> send row of (t, device of its expert) (level-2 send)   */
    int32_t *slot_send_row;  /* [P]    slot -> send row holding its payload                           */
    uint8_t *pair_first;     /* [P]    1 iff the pair is the first appearance of its device in token t */
    int32_t *status;         /* [1]    number of expert ids outside [0, E) seen by the last fusco_plan */
    /* Transfer order (section 3.2: descriptor lists are dense arrays in transfer order).  The tokens are cut
     * into tile_count tiles of tile_tokens consecutive tokens (the last one may hold fewer); the entries
     * [i * tile_tokens * k, (i + 1) * tile_tokens * k) list the slots of tile i's (token, expert) pairs in
     * ascending order, i.e. expert by expert with ascending tokens inside an expert, followed by -1 up to the
     * tile's capacity (a ragged last tile, pairs with an invalid expert id).  fusco_dispatch moves the rows
     * in this order, tile by tile.  tile_tokens and tile_count depend on N and k only and are set by
     * fusco_layout_bind. */
    int32_t *tile_slots;     /* [tile_count * tile_tokens * k]                                        */
    int32_t tile_tokens, tile_count;
} fusco_layout;

/* Library version (FUSCO_VERSION of the build). */
int fusco_version(void);

/* Static text for a FUSCO_* return code. */
const char *fusco_status_string(int status);

/*
 * Bytes of device memory the descriptor arrays need for these sizes (0 if the sizes are
 * invalid: N < 0, k outside [1, FUSCO_MAX_K], E outside [1, FUSCO_MAX_E], D < 1, E % D != 0,
 * or N * k >= 2^31).
 */
size_t fusco_layout_bytes(int32_t N, int32_t k, int32_t E, int32_t D);

/* Bytes of planner scratch (partial counts per tile of 1024 or 2048 pairs and per chunk of tiles) for
 * these sizes; 0 if the sizes are invalid. */
size_t fusco_scratch_bytes(int32_t N, int32_t k, int32_t E, int32_t D);

/*
 * Fill *L (host struct) with the sizes and with pointers carved out of the caller's device
 * block d_mem of `bytes` bytes (256-byte aligned base).  Host-only: touches no device memory.
 * Errors: FUSCO_ERR_INVALID_ARG (null, bad sizes, misaligned), FUSCO_ERR_WORKSPACE (too small).
 */
int fusco_layout_bind(fusco_layout *L, int32_t N, int32_t k, int32_t E, int32_t D, void *d_mem, size_t bytes);

/*
 * Planner (section 3.3): per-expert histogram, prefix-scan offsets, stable expert-major slot of
 * every (t, e) pair, and removal of duplicate (token, device) sends with the resulting send rows.
 * d_topk_idx: [N, k] int32 row-major, the token-expert matrix A (may be NULL when N == 0).
 * Ids outside [0, E) are counted in L->status, get pair_slot = pair_send_row = -1 and are skipped
 * by dispatch and combine; the plan is then not a valid layout (slots at the end of the tensor
 * stay unassigned).
 * d_scratch: at least fusco_scratch_bytes() bytes, contents irrelevant before and after.
 * Every descriptor array is fully rewritten (send_src only in rows < U).  N == 0 is allowed.
 */
int fusco_plan(fusco_layout *L, const int32_t *d_topk_idx, void *d_scratch, size_t scratch_bytes, void *stream);

/*
 * fusco_plan for callers that cannot allocate device memory or pass a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same arguments and results as fusco_plan,
 * but the planner's scratch (per-tile and per-chunk counts) is a static array of FUSCO_STATIC_SCRATCH_BYTES
 * (4 MiB) inside the library, present on every GPU the library runs on until the process ends.  The call
 * allocates and frees nothing.  Inputs whose fusco_scratch_bytes() exceeds that size are refused with
 * FUSCO_ERR_STATIC_LIMIT and nothing is launched (4 MiB covers about 7.9 million (token, expert) pairs at
 * E + D = 264, e.g. 990 000 tokens with k = 8); use fusco_plan with a workspace of your own for those.
 * The first call on a device looks up the address of that device's copy of the array (no allocation; make
 * that first call outside a graph capture); the device current at the call must be the one `stream` belongs to.
 * All calls on one GPU share the one array: two fusco_plan_static calls that may overlap on the same GPU
 * (different streams, no ordering between them) race on it and give undefined descriptors; calls in one
 * stream, or ordered by events, are safe.  The array needs no clearing: every call writes all counts it reads.
 * Errors otherwise as fusco_plan; FUSCO_ERR_HIP also when the array's address cannot be resolved.
 */
int fusco_plan_static(fusco_layout *L, const int32_t *d_topk_idx, void *stream);

/*
 * Fused gather-pack (section 3.2, intra-node path: descriptor interpretation inlined into the
 * copy, no intermediate pass): every token row is read once and written to each of its slots,
 *     expert_buf[pair_slot[t*k+j]] = x[t]                          (FUSCO_DISPATCH_EXPERT)
 *     send_buf[pair_send_row[t*k+j]] = x[t] where pair_first       (FUSCO_DISPATCH_WIRE)
 * For large inputs the expert tensor is written tile by tile in the layout's transfer order (see
 * fusco_dispatch_in_transfer_order): every XCD of the GPU takes whole tiles of tokens and writes their rows
 * expert by expert with streaming stores, the tile's source rows being read from memory once and from the
 * XCD's L2 afterwards while they stay there.  A source tensor of more than 128 MiB is taken in chunks of tiles,
 * each chunk after a sequential read of its source rows (a few launches instead of one).  Where both tensors are
 * written, the tile's send rows follow its pairs, device by device (for few devices).  Otherwise every
 * token's row is read once and stored to its k rows at once (token walk).
 * Rows are opaque bytes.  d_x: [N, row_bytes], row_bytes a positive multiple of 16.  An optional
 * second plane (e.g. per-block scales of an fp8 payload) of aux_row_bytes (multiple of 16, or 0
 * with NULL aux pointers) follows the same descriptors; row_bytes + aux_row_bytes may not exceed
 * FUSCO_MAX_ROW_BYTES.  d_expert_buf: [P, row_bytes],
 * d_expert_aux: [P, aux_row_bytes]; d_send_buf: [send_cap, row_bytes], d_send_aux likewise; rows
 * >= U of the send buffers are not written.  Buffers of a plane that is not requested by `flags`
 * may be NULL.
 * FUSCO_DISPATCH_TWO_HOP executes the two descriptor levels one after the other, as the planner
 * describes them (section 3.3): first one row per (token, device) into the receive tensors, then
 *     expert_buf[s] = send_buf[slot_send_row[s]]
 * for every assigned slot.  Both tensors are written and hold the same bytes as in the fused mode;
 * the extra pass costs U + P more row reads.
 * FUSCO_DISPATCH_STREAMING may be added to the fused modes (not to FUSCO_DISPATCH_TWO_HOP): the token walk then
 * writes its rows with non-temporal stores, which do not stay in the GPU's 256 MB memory-side cache (the
 * transfer order always writes that way, and so does the token walk on its own when the tensors it writes
 * exceed that cache).  Choose it for smaller tensors when other traffic (an expert computation) comes between
 * this call and the first reader of the rows: a plain dispatch leaves its rows dirty in that cache, and whoever
 * streams through memory next pays for writing them back.  Results are identical either way.
 */
int fusco_dispatch(const fusco_layout *L, const void *d_x, size_t row_bytes, const void *d_x_aux,
                   size_t aux_row_bytes, void *d_expert_buf, void *d_expert_aux, void *d_send_buf,
                   void *d_send_aux, uint32_t flags, void *stream);

/*
 * Host-only: 1 if fusco_dispatch with these row sizes and flags moves the rows tile by tile in the layout's
 * transfer order (tile_slots), 0 if it walks the tokens, negative on invalid arguments.  The transfer order
 * is used when the expert tensor is written, k >= 2, the layout has at least 16 tiles, and the source
 * rows of one tile (tile_tokens * (row_bytes + aux_row_bytes)) fit the 4 MB L2 of an XCD whole (at most
 * 3840 KiB) or cut into up to eight column segments of at least 4 KiB each, which are then moved in as many
 * passes over the tile; and when the sizes make it pay: the expert tensor is larger than the 256 MB memory-side cache
 * (a smaller one is left there by the token walk's plain stores for its reader), rows shorter than 8 KiB
 * come with a source tensor of at most 128 MiB (less than 128 MiB for rows shorter than 4 KiB), and a source
 * tensor of more than 128 MiB comes with k >= 8, or with k >= 5 and rows that need no column segments.  Calls that
 * write the receive tensors as well have it on top of that with k >= 8, at most 8 devices and rows of at least 8 KiB,
 * or with at most 2 devices and rows that need no column segments (of at least 4 KiB for k < 8); with at least 4 devices and
 * 72 to 128 MiB of source rows in whole 64-byte units (112 to 128 MiB for rows that fill the lanes of their workgroups, as those of 8 and 12 KiB do and, with up to
 * 5 devices, those of 10 to 12 and 13.4 to 15 KiB) the receive
 * tensors are then written by a token walk of their own.  All ways write
 * the same bytes.
 */
int fusco_dispatch_in_transfer_order(const fusco_layout *L, size_t row_bytes, size_t aux_row_bytes, uint32_t flags);

/*
 * fusco_plan followed by fusco_dispatch (FUSCO_DISPATCH_EXPERT only) in a single launch, for inputs
 * that fit one planner tile: N <= floor(2048 / k) tokens (decode-sized batches, where a chain of
 * dependent launches costs more than the work; the planner's cost is fixed and shows at small
 * sizes, section 5.2).  Results are exactly those of the two calls: every descriptor array of *L is
 * written as by fusco_plan (no scratch is needed), d_expert_buf / d_expert_aux as by fusco_dispatch.
 * Arguments as in those two calls.  Returns FUSCO_ERR_UNSUPPORTED when the input needs more than
 * one tile; the caller then makes the two calls.
 */
int fusco_plan_dispatch(fusco_layout *L, const int32_t *d_topk_idx, const void *d_x, size_t row_bytes,
                        const void *d_x_aux, size_t aux_row_bytes, void *d_expert_buf, void *d_expert_aux,
                        void *stream);

/*
 * Weighted combine (reverse path of the shuffle: weighted sum of a token's expert outputs,
 * section 2.1):   out[t, :] = sum_{j=0..k-1} w[t, j] * y[pair_slot[t*k+j], :]
 * accumulated in fp32 with one fused multiply-add per term in ascending j from +0, then rounded
 * once (nearest even) when out_dtype is FUSCO_BF16.
 * d_y: [P, H] of y_dtype, d_w: [N, k] fp32, d_out: [N, H] of out_dtype.  H * sizeof(y element)
 * must be a multiple of 16 and at most FUSCO_MAX_ROW_BYTES.  `flags` must be 0.
 */
int fusco_combine(const fusco_layout *L, const void *d_y, int y_dtype, const float *d_w, void *d_out,
                  int out_dtype, int32_t H, uint32_t flags, void *stream);

/*
 * Combine along the two descriptor levels in reverse (mirror of FUSCO_DISPATCH_TWO_HOP; the paper
 * only says the reverse path is symmetric, the arithmetic is this library's reading):
 *   partial[r, :] = sum over the entries j of token send_src[r] whose send row is r of
 *                   w[t, j] * y[pair_slot[t*k+j], :]      fp32 fused multiply-adds, ascending j, from +0
 *   out[t, :]     = sum of the token's partial rows        fp32 additions from +0, in the order in which
 *                                                          the devices first appear among the k entries
 * so one fp32 row per (token, device) would cross the link instead of one row per (token, expert).
 * d_partial: [send_cap, H] fp32 scratch tensor, rows < U are overwritten.  H must be a multiple of 4
 * (and H * sizeof(y element) a multiple of 16).  The result differs from fusco_combine only by the
 * association of the sum: at most (k + D) * 2^-24 * sum_j |w_j y_j| from the exact value.
 */
int fusco_combine_two_hop(const fusco_layout *L, const void *d_y, int y_dtype, const float *d_w, float *d_partial,
                          void *d_out, int out_dtype, int32_t H, void *stream);

/*
 * Disaggregated baseline: the multi-stage shuffle the paper starts from (section 1: rearrange by
 * destination rank, all-to-all, rearrange by expert, and the symmetric reverse; section 5.4, the
 * "dComm-off" ablation, performs the rearrangements explicitly around the transfer).  Each stage is
 * a separate pass over the whole buffer; no deduplication (one row per (token, expert) pair).  It
 * exists to measure what fusing buys on this GPU and produces the same expert tensor / output.
 *
 * fusco_disaggregated_plan fills Lr, a second layout bound by the caller with
 * fusco_layout_bind(Lr, N, k, D, D, ...): the stable order of the pairs by destination device
 * ("rank-major": Lr->pair_slot is the pair's row, Lr->slot_token its token).  d_topk_dev: [N, k]
 * int32 scratch that receives the device of every pair.  d_scratch as for fusco_plan with (N,k,D,D).
 * L must already hold the plan of the same d_topk_idx.
 *
 * fusco_disaggregated_dispatch: stage_a[r] = x[token of rank row r]; stage_b = stage_a (the
 * exchange between virtual devices, a contiguous copy); expert_buf[s] = stage_b[rank row of slot s].
 * fusco_disaggregated_combine: stage_b[r] = y[slot of rank row r]; stage_a = stage_b;
 * out[t] = sum_j w[t,j] * stage_a[rank row of (t,j)] (same arithmetic as fusco_combine).
 * d_stage_a, d_stage_b: [P, row] scratch tensors, overwritten.
 */
int fusco_disaggregated_plan(fusco_layout *Lr, const fusco_layout *L, const int32_t *d_topk_idx, int32_t *d_topk_dev,
                             void *d_scratch, size_t scratch_bytes, void *stream);
int fusco_disaggregated_dispatch(const fusco_layout *L, const fusco_layout *Lr, const void *d_x, size_t row_bytes,
                                 void *d_stage_a, void *d_stage_b, void *d_expert_buf, void *stream);
int fusco_disaggregated_combine(const fusco_layout *L, const fusco_layout *Lr, const void *d_y, int y_dtype,
                                const float *d_w, void *d_stage_a, void *d_stage_b, void *d_out, int out_dtype,
                                int32_t H, void *stream);

/*
 * Input of the load balancer (section 3.4): the cross-node traffic load of the GPU that owns this plan,
 * i.e. the volume it must transmit to remote nodes.  The D destination devices are grouped into nodes of
 * devices_per_node consecutive devices (D must be a multiple); the GPU itself sits on node home_node.
 *     *d_load = row_bytes * sum of send_count[d] over the devices d with d / devices_per_node != home_node
 * in bytes, after duplicate removal (one send row per token and destination device; plan with D = number
 * of nodes for the paper's one copy per node).  d_load: one int64 in device memory, 8-byte aligned, e.g. the
 * GPU's cell of the [nodes, gpus] matrix that fusco_balance_groups takes once every GPU has filled its own.
 * Must follow the fusco_plan of the same layout in stream order.  One small launch.
 */
int fusco_cross_node_load(const fusco_layout *L, int32_t devices_per_node, int32_t home_node, size_t row_bytes,
                          int64_t *d_load, void *stream);

/*
 * Online Group-Balanced Assignment (Algorithm 1, section 3.4).  Host-only, no GPU work.
 * load: [nodes, gpus] row-major, cross-node traffic load of every GPU.  For every node the GPUs are
 * sorted by descending load (equal loads keep ascending GPU index), the sorted list is rotated by
 * the node index, and communication group i takes the GPU at position i of every node's rotated
 * list: group_gpu[i * nodes + n] = sorted_n[(i + n) mod gpus], for gpus groups of one GPU per node.
 * The direction of the rotation and the tie order are not fixed by the paper; these are this
 * library's readings.  O(gpus^2) per node (gpus is 4..8 in practice).
 * Errors: FUSCO_ERR_INVALID_ARG (null, sizes < 1 or nodes * gpus > 2^24), FUSCO_ERR_WORKSPACE (host allocation failed).
 */
int fusco_balance_groups(const int64_t *load, int32_t nodes, int32_t gpus, int32_t *group_gpu);

/*
 * Segment descriptor (section 3.2): where a logical segment lies, as a byte offset from a base
 * pointer, and its size in bytes.  Offsets and sizes must be multiples of 16.  A descriptor list is
 * a dense array in transfer order; the sender's and the receiver's lists map one to one.
 */
typedef struct fusco_segment {
    uint64_t offset;
    uint64_t size;
} fusco_segment;

/*
 * Cumulative bytes of a descriptor list: d_cum[0] = 0, d_cum[i+1] = d_cum[i] + size of segment i
 * (d_cum has n + 1 entries).  The engine finds the segment of a stream position from this array.
 * Descriptors with an offset or size that is not a multiple of 16 are counted in *d_status and take
 * part with size 0.  n <= 2^26.  One launch for up to 32768 segments, two for longer lists.
 */
int fusco_segments_scan(const fusco_segment *d_desc, int64_t n, uint64_t *d_cum, int32_t *d_status, void *stream);

/*
 * Descriptor-driven transfer of n segments (section 3.2): segment i is read at d_src + the
 * sender's offset and written at d_dst + the receiver's offset; its size comes from d_cum (built
 * by fusco_segments_scan from either list: the lists must agree on sizes).  A NULL descriptor list
 * means that side is the contiguous stream, i.e. segment i starts at d_cum[i]: with d_dst_desc ==
 * NULL the segments are gathered and packed into one buffer (sender side, slices for the network),
 * with d_src_desc == NULL a packed buffer is scattered to its final places (receiver side).
 * src_bytes / dst_bytes: sizes of the two buffers; a 16-byte unit that would fall outside, or is
 * misaligned, is skipped and counted in *d_status (which this call only adds to: it continues the
 * count of fusco_segments_scan).  stream_capacity: upper bound of the total size known on the
 * host (the exact total is read on the device from d_cum[n]).
 * Slices: if d_slice_fill is given, the contiguous stream is cut into slices of slice_bytes (a
 * multiple of 16384) and d_slice_fill[s] counts the bytes of slice s that have been written and are
 * visible: the data is stored write-through at system scope, every workgroup waits for its stores
 * and only then adds its bytes with a system-scope atomic.  A consumer (another stream, another
 * agent) takes slice s once the count reaches min(slice_bytes, total - s * slice_bytes); it must
 * read the counter with an acquire (or bypass its caches for the slice's bytes).  Units skipped for
 * being out of range are not counted, so a slice with holes never becomes ready.  The counters are
 * reset to 0 by a small kernel at the start of the call, in stream order: a consumer that is still
 * polling the counters of the previous call on the same d_slice_fill races with that reset; give
 * overlapping transfers counter arrays of their own.  A consumer kernel that polls while this call
 * runs must be able to run beside it: streams are dealt onto a few hardware queues, and two streams
 * on the same queue run one after the other, so a consumer launched first on such a stream would
 * poll for slices that cannot come.  Bound its polling, or launch it behind the producer.
 */
int fusco_segments_copy(const void *d_src, uint64_t src_bytes, const fusco_segment *d_src_desc, void *d_dst,
                        uint64_t dst_bytes, const fusco_segment *d_dst_desc, const uint64_t *d_cum, int64_t n,
                        uint64_t stream_capacity, uint64_t slice_bytes, uint32_t *d_slice_fill, int32_t *d_status,
                        void *stream);

/*
 * Gradient of fusco_combine (d_y, d_w and the layout as given to it, d_dout the gradient of its output):
 *     dy[pair_slot[t*k+j], :] = w[t, j] * dout[t, :]             rounded once when y_dtype is FUSCO_BF16
 *     dw[t, j] = sum over h of dout[t, h] * y[pair_slot[t*k+j], h]   held in fp32
 * d_dy: [P, H] of y_dtype, every assigned row is written; d_dw: [N, k] fp32, 0 for a pair without a slot.  d_dout: [N, H] of
 * dout_dtype.  H: a multiple of 8, at most 32768.  The gradient of fusco_dispatch needs no call of its own: it is fusco_combine with
 * weights of 1.
 */
int fusco_combine_backward(const fusco_layout *L, const void *d_y, int y_dtype, const float *d_w, const void *d_dout,
                           int dout_dtype, void *d_dy, float *d_dw, int32_t H, void *stream);

/*
 * Routing to experts: from a token's logits to the k experts and weights that fusco_plan and fusco_combine take.
 *     s[e] = 1 / (1 + exp(-l[e]))  (FUSCO_SCORE_SIGMOID)   or   exp(l[e] - max l) / sum exp(l - max l)  (FUSCO_SCORE_SOFTMAX)
 *     b[e] = s[e] + bias[e]        what experts compete by: a bias keeps the load balanced and does not enter the weights
 *     groups > 1: group g holds the E / groups experts from g * E / groups on and counts as much as its group_best (1 or 2) largest b
 *     together; only experts of the keep_groups best groups compete (with groups on devices: a token goes to few devices)
 *     topk_idx[j]: the expert with the j-th largest b, j = 0 .. k-1
 *     w[j] = scale * s[topk_idx[j]] / sum_i s[topk_idx[i]]  with renorm, scale * s[topk_idx[j]] without
 * Equal values go to the lower index, for groups as for experts.  Without a bias the softmax's denominator, the same for the whole
 * row, is left out where scores are compared.  Logits of -infinity (experts that are not allowed) have score 0; a row without any
 * allowed expert gets the experts that its ties name, with weights 0.  A NaN score ranks below every number; a softmax row with a NaN
 * or +infinity has weights NaN.  topk_idx always holds k distinct experts.
 * d_logits: [N, E] of logits_dtype (FUSCO_BF16 or FUSCO_F32), rows logits_stride elements apart (at least E; any alignment of its
 * type).  d_bias: [E] fp32 or NULL.  d_topk_idx: [N, k] int32, d_w: [N, k] fp32.  k <= keep_groups * (E / groups), E a multiple of
 * groups, group_best <= E / groups.
 */
typedef struct fusco_router {
    int32_t N, E, k;
    int32_t score;              /* FUSCO_SCORE_*                                    */
    int32_t groups, keep_groups, group_best;   /* 1, 1, 1 for a choice among all    */
    int32_t renorm;             /* 0 or 1                                           */
    int32_t logits_dtype;
    float scale;
    int64_t logits_stride;
} fusco_router;
int fusco_route(const fusco_router *R, const void *d_logits, const float *d_bias, int32_t *d_topk_idx, float *d_w, void *stream);

/*
 * Gradient of fusco_route's weights with respect to the logits (the choice itself has none, nor has the bias): d_dw [N, k] fp32 is
 * the gradient of the weights, d_dlogits [N, E] of logits_dtype (contiguous) is written whole.  Groups and bias play no part.
 */
int fusco_route_backward(const fusco_router *R, const void *d_logits, const int32_t *d_topk_idx, const float *d_dw, void *d_dlogits,
                         void *stream);

/*
 * Norms before and after a block (an attention or an MoE block) on a residual stream, inv(x) = 1 / sqrt(mean(x^2) + eps) per row:
 *     before:  out  = x * inv(x) * gain
 *     after:   out  = r + scale * gate * (y * inv(y) * gain)          and, if d_next is not NULL,
 *              next = out * inv(out) * next_gain                      (the norm before the next block, of the unrounded out)
 * y is the block's output, r the stream before it; gate is a value per column, a value per token or 1.  Sums are held in fp32, results
 * are rounded once.  Streams (r, x, out of fusco_norm_after and their gradients) are of stream_dtype, what goes into and comes out
 * of blocks (y, next, out of fusco_norm_before and their gradients) of block_dtype; gains and gate of gain_dtype; FUSCO_BF16 with a
 * block_dtype of FUSCO_F32 is not offered for the stream (FUSCO_ERR_UNSUPPORTED).  All tensors [N, H] contiguous, H a multiple of 8 and
 * at most FUSCO_MAX_NORM_H; eps > 0.  out may be the buffer of r, next that of y (where their types are the same).
 */
typedef struct fusco_norm {
    int32_t N, H;
    int32_t stream_dtype, block_dtype, gain_dtype;
    int32_t gate_kind;          /* FUSCO_GATE_*, fusco_norm_after and its gradient only */
    float scale, eps;
} fusco_norm;
int fusco_norm_before(const fusco_norm *n, const void *d_x, const void *d_gain, void *d_out, void *stream);
int fusco_norm_after(const fusco_norm *n, const void *d_r, const void *d_y, const void *d_gain, const void *d_gate, void *d_out,
                     const void *d_next_gain, void *d_next, void *stream);

/*
 * Their gradients.  Gradients of gains and gate are fp32, added up over the rows in a fixed order (two launches; partial sums in
 * d_scratch, fusco_norm_scratch_bytes() bytes, contents irrelevant before and after).
 * before:  dx = dres + gradient through the norm; d_dout is the gradient of out, d_dres [N, H] of stream_dtype (NULL: 0) what reaches x
 *          past the block; d_dgain [H].
 * after:   d_dout is the gradient of out (NULL: 0), d_dnext that of next (NULL if next was not asked for; then d_out, d_next_gain
 *          and d_dnext_gain are not used), d_out the out that fusco_norm_after wrote.  Results: d_dr, d_dy [N, H], d_dgain [H],
 *          d_dgate [H] or [N] by gate_kind, d_dnext_gain [H].
 */
size_t fusco_norm_scratch_bytes(int32_t N, int32_t H);
int fusco_norm_before_backward(const fusco_norm *n, const void *d_dout, const void *d_x, const void *d_gain, const void *d_dres,
                               void *d_dx, float *d_dgain, void *d_scratch, size_t scratch_bytes, void *stream);
int fusco_norm_after_backward(const fusco_norm *n, const void *d_dout, const void *d_dnext, const void *d_y, const void *d_out,
                              const void *d_gain, const void *d_gate, const void *d_next_gain, void *d_dr, void *d_dy,
                              float *d_dgain, float *d_dgate, float *d_dnext_gain, void *d_scratch, size_t scratch_bytes,
                              void *stream);

/*
 * Products of the experts, on the rows that fusco_dispatch wrote and a layout's plan describes: expert e has the rows
 * [exp_off[e], exp_off[e+1]) and weights of its own.  All tensors are bf16 and contiguous; sums are held in fp32 and rounded
 * once (nearest even).  Rows that no expert owns (a plan of invalid ids) are neither read nor written.  Every row size must
 * be a multiple of 16 bytes and at most FUSCO_MAX_ROW_BYTES, one expert's weights must lie below 2032 MiB.
 *
 * fusco_experts_gated: h[r, i] = silu(g) * u with g = sum_c x[r, c] w[e, i, c] and u = sum_c x[r, c] w[e, I + i, c],
 * silu(g) = g / (1 + exp(-g)).  d_x [P, H], d_w [E, 2 I, H], d_h [P, I].  d_pre, if not NULL, receives g and u,
 * [P, 2 I] with g first: what the gradient needs.
 *
 * fusco_experts_linear: y[r, m] = sum_c x[r, c] w[e, m, c].  d_x [P, C], d_w [E, M, C], d_y [P, M].
 */
int fusco_experts_gated(const fusco_layout *L, const void *d_x, const void *d_w, void *d_h, void *d_pre, int32_t H, int32_t I,
                        void *stream);
int fusco_experts_linear(const fusco_layout *L, const void *d_x, const void *d_w, void *d_y, int32_t C, int32_t M,
                         void *stream);

/*
 * Rows and weights in 8-bit floating point (e4m3: four significant bits, largest 448, NaN but no infinities) with a scale per block:
 *     s = 2^n, the smallest power of two with max |x| <= 448 s over the block (at least 2^-126; 1 for a block of zeros)
 *     q = x / s rounded to e4m3 (nearest even)
 * Infinities and NaN become NaN and take no part in the maximum.  A block is 128 columns of a row (matrix_rows 0: activations), or 128 rows by
 * 128 columns of a matrix (weights); the last ones of a row or matrix end with it.  d_x [rows, columns] of dtype, d_q [rows, columns] e4m3, both
 * contiguous; d_scale fp32: [rows, scale_stride] for rows (columns behind the last block's are left as they are: dispatch moves
 * them as its second plane, whose rows are multiples of 16 bytes), [rows / matrix_rows, ceil(matrix_rows / 128), ceil(columns / 128)]
 * for matrices.  fusco_from_fp8 writes x = q * s for any scales, rounded once; with the powers of two above, from 2^-124 on, bf16 holds it exactly.
 * columns: a multiple of 16, at most FUSCO_MAX_ROW_BYTES; less than 2^31 rows, at most 2^29 - 32 blocks of 128 columns of
 * rows (of matrices too), and less than 2^23 blocks of matrices.
 */
#define FUSCO_MAX_SCALE_STRIDE 65536
typedef struct fusco_fp8 {
    int64_t rows;
    int32_t columns;
    int32_t dtype;              /* of x: FUSCO_BF16 or FUSCO_F32                     */
    int32_t matrix_rows;        /* 0: scales per row; else rows per matrix           */
    int32_t scale_stride;       /* floats from one row of scales to the next; matrices: ceil(columns / 128) */
} fusco_fp8;
int fusco_to_fp8(const fusco_fp8 *f, const void *d_x, void *d_q, float *d_scale, void *stream);
int fusco_from_fp8(const fusco_fp8 *f, const void *d_q, const float *d_scale, void *d_x, void *stream);

/*
 * fusco_experts_gated and fusco_experts_linear on rows and weights of e4m3 with scales per block, which may be any fp32 numbers whose products are
 * ordinary ones (zero, or from 2^-126 to the largest):
 *     sum over blocks b of 128 columns of   (x_scale[r, b] * w_scale[e, m / 128, b]) * sum over c in b of x[r, c] w[e, m, c]
 * The product of the two scales is rounded to fp32 first: below 2^-126 it has fewer digits, and where it is infinite so is the result, or NaN for a sum of zero.
 * Sums and scales are fp32 and results are rounded once to bf16; the matrix instructions for e4m3 cut each product, before eight neighbours are added, to
 * a multiple of 2^-13 of the largest one's power of two (2^-16 of a result on the average, where its rounding to bf16 is 2^-9.7).  A result
 * that this carries over a border of e4m3 moves by a whole step when it is brought to e4m3 in turn: both products with fusco_to_fp8 between them
 * are 2.0e-3 to 2.1e-3 off in the norm, where exact products are 1.7e-3.  d_x [P, H] or [P, C] and d_x_scale [P, x_scale_stride] as
 * fusco_dispatch moves the two planes of such rows; weights [E, 2 I, H] or [E, M, C]; d_w_scale [E, 2 ceil(I / 128), ceil(H / 128)] (gate rows
 * and up rows begin blocks of their own: the weights are 2 E matrices of I rows) or [E, ceil(M / 128), ceil(C / 128)].  d_h, d_pre
 * and d_y are bf16 as there.  H (gated) and C (linear): multiples of 16.  I and M: multiples of 8.
 */
int fusco_experts_gated_fp8(const fusco_layout *L, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, const void *d_w,
                            const float *d_w_scale, void *d_h, void *d_pre, int32_t H, int32_t I, void *stream);
int fusco_experts_linear_fp8(const fusco_layout *L, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, const void *d_w,
                             const float *d_w_scale, void *d_y, int32_t C, int32_t M, void *stream);

/*
 * Gradients of these products (tensors, sizes and rounding as there).
 *
 * fusco_experts_input_grad: dx[r, c] = sum_m dy[r, m] w[e, m, c].  d_dy [P, M], d_w [E, M, C], d_dx [P, C].
 * With d_pre not NULL (the [P, 2 C] tensor of fusco_experts_gated with I = C, whose h was this product's input) the gradient
 * of the activation is taken as well, in fp32 before the only rounding, and d_dx is the gradient of pre, [P, 2 C]:
 *     dg = dh u sig(g) (1 + g (1 - sig(g))),   du = dh g sig(g),   sig(g) = 1 / (1 + exp(-g)).
 *
 * fusco_experts_weight_grad: dw[e, m, c] = sum over the expert's rows of dy[r, m] x[r, c]; zeros for an expert without rows.
 * d_dy [P, M], d_x [P, C], d_dw [E, M, C] of dw_dtype (FUSCO_BF16 or FUSCO_F32).
 */
int fusco_experts_input_grad(const fusco_layout *L, const void *d_dy, const void *d_w, void *d_dx, const void *d_pre,
                             int32_t M, int32_t C, void *stream);
int fusco_experts_weight_grad(const fusco_layout *L, const void *d_dy, const void *d_x, void *d_dw, int dw_dtype, int32_t M,
                              int32_t C, void *stream);

/*
 * The same gradients from activations that were kept in e4m3 with a scale per 128 columns of a row (fusco_to_fp8 of what the forward pass
 * wrote: half the bytes).
 *
 * fusco_experts_input_grad_fp8: fusco_experts_input_grad with pre-activations d_pre [P, 2 C] of e4m3, d_pre_scale [P, pre_scale_stride] (blocks of the
 * whole row of 2 C columns), used as fp32.  C: a multiple of 16.
 *
 * fusco_experts_weight_grad_fp8: fusco_experts_weight_grad with d_x [P, C] of e4m3, d_x_scale [P, x_scale_stride].  x * scale is rounded to bf16 before
 * the product, which changes nothing for scales that are powers of two, from 2^-124 on.  C: a multiple of 16.
 */
int fusco_experts_input_grad_fp8(const fusco_layout *L, const void *d_dy, const void *d_w, void *d_dpre, const void *d_pre, const float *d_pre_scale,
                                 int32_t pre_scale_stride, int32_t M, int32_t C, void *stream);
int fusco_experts_weight_grad_fp8(const fusco_layout *L, const void *d_dy, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, void *d_dw,
                                  int dw_dtype, int32_t M, int32_t C, void *stream);

/*
 * The experts of an MoE layer for a few tokens (one to FUSCO_MAX_FEW_TOKENS), from their rows and routing to the weighted sum, without a layout:
 *     out[t, :] = sum_j w[t, j] * W_out[e] (silu(g) * u),   g and u = gate and up rows of W_in[e] times x[t, :],   e = topk_idx[t, j]
 * as fusco_plan_dispatch, fusco_experts_gated, fusco_experts_linear and fusco_combine compute it, in two launches.  The first passes over w_in of a chosen expert once
 * for every 16 of its pairs (32 if N k >= 8 E), the second over w_out once for every 5 (15 if N k >= 3 E): up to some 8 tokens that is the faster way, from
 * 16 on the calls one by one are in most sizes.  Sums and silu(g) * u are fp32, the result is rounded once.  Pairs whose expert is not in [0, E) count
 * nothing; a token's equal experts count together.  An expert's weights reach only the tokens that chose it.
 * d_x [N, H] bf16, d_topk_idx and d_w [N, k], d_out [N, H] of out_dtype (FUSCO_BF16 or FUSCO_F32).  weight_dtype FUSCO_BF16: d_w_in [E, 2 I, H] and
 * d_w_out [E, H, I] as for fusco_experts_gated and fusco_experts_linear, H and I multiples of 8, scales NULL.  FUSCO_E4M3: weights and scales as for
 * fusco_experts_gated_fp8 and fusco_experts_linear_fp8, H and I multiples of 16.  An expert's w_in has less than 2^31 - 2^24 bytes, and
 * min(N k, E) I / 8 is less than 2^24 - 1, and 6 N k I bytes are below 2032 MiB.  Infinite weights of w_out give infinities or NaN.
 * d_scratch: fusco_moe_few_scratch_bytes() bytes, contents irrelevant before and after; calls that may run at the same time have scratch of their own.
 */
#define FUSCO_E4M3 2
#define FUSCO_MAX_FEW_TOKENS 64
typedef struct fusco_few {
    int32_t N, E, k, H, I;
    int32_t weight_dtype, out_dtype;
} fusco_few;
size_t fusco_moe_few_scratch_bytes(int32_t N, int32_t k, int32_t I);
int fusco_moe_few(const fusco_few *f, const void *d_x, const int32_t *d_topk_idx, const float *d_w, const void *d_w_in, const float *d_w_in_scale,
                  const void *d_w_out, const float *d_w_out_scale, void *d_out, void *d_scratch, size_t scratch_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FUSCO_H */
