/*
 * eaas.h -- C ABI of one stateless expert server's forward step on gfx950, and of
 * the separate products that train an expert layer or serve it in 8 bits.
 *
 * The operation (EaaS, §3.3 "Asynchronous Server Operation", and Fig. 5): the
 * server takes a batch of ready requests, reorganises the tokens by expert,
 * runs the grouped expert computation, and writes back for every token the
 * weighted sum of its experts' outputs.  The request payload (§3.2 "Data
 * Payload") carries the hidden states, an expert id per token slot and the
 * router score used for weighting; the header carries the batch size (§3.2
 * "Header").  The server is stateless (§2.4, §3.3): nothing survives between
 * calls, so every call is a pure function of its arguments.
 *
 * Symbols: T tokens (header batch_size), H hidden size, I expert intermediate
 * size, E resident experts on this server, k expert slots per token,
 * R = T*k slots.  Slot s = t*k + j.  A slot is valid iff 0 <= topk_ids[s] < E;
 * other ids (experts hosted by other servers) are skipped, not errors.
 *
 * Expert FFN (the paper names only "expert computations"; this library
 * implements the SwiGLU form without bias):
 *     y_e(x) = W_down[e] . ( silu(W_gate[e] . x) * (W_up[e] . x) )
 * with W_gate_up[e] = [W_gate[e]; W_up[e]] stacked by rows (gate rows [0,I),
 * up rows [I,2I)), W_gate_up[E,2I,H] and W_down[E,H,I], both [out,in]
 * row-major.  Accumulation is fp32; the intermediate h is rounded once to
 * bf16 (round to nearest even); the weighted sum is fp32, summed over valid
 * slots in ascending j starting from +0.
 *
 * Weights are bf16, or OCP fp8 e4m3fn with one fp32 scale per 128x128 block
 * of each expert matrix (W = q * s): scale arrays [E,2I/128,H/128] and
 * [E,H/128,I/128], row-major.
 *
 * Conventions for every entry point:
 *   - All array pointers are DEVICE pointers owned by the caller; the shape
 *     descriptor and the routing descriptor themselves live in host memory.
 *   - The library never allocates, frees or synchronises.  Scratch memory is
 *     the caller's workspace `ws` of at least eaas_workspace_bytes() bytes,
 *     256-byte aligned.  Its contents are undefined between calls.
 *   - `stream` is a hipStream_t passed as void* (NULL = null stream).  All work
 *     is enqueued on it with no host synchronisation and no device-to-host
 *     readback, so calls can be captured in a hipGraph.
 *   - Arguments are validated on the host before anything is enqueued; on any
 *     error a negative status is returned and nothing is enqueued.  T = 0 is
 *     a valid empty batch: EAAS_OK, nothing enqueued, outputs left untouched
 *     (pointers may then be NULL).  Device arrays must be 16-byte aligned
 *     (EAAS_ERR_INVALID_ARG otherwise).
 *   - Calls are re-entrant; concurrent calls must use distinct workspaces and
 *     outputs.
 *   - NaN and Inf in the data propagate; they are not errors.
 */
#ifndef EAAS_H
#define EAAS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct eaas_shape {
  int32_t T; /* tokens in the batch (>= 0)                              */
  int32_t H; /* hidden size, multiple of 128                             */
  int32_t I; /* expert intermediate size, multiple of 128                */
  int32_t E; /* resident experts, 1..1024                                */
  int32_t k; /* slots per token, 1..64                                   */
} eaas_shape;

enum eaas_status {
  EAAS_OK = 0,
  EAAS_ERR_INVALID_ARG = -1, /* null pointer, negative size, bad dtype, overlap
                                (k > E is valid: see eaas_route_permute) */
  EAAS_ERR_UNSUPPORTED = -2, /* H or I not a multiple of 128, E > 1024, k > 64,
                                or past the 32-bit element offsets the kernels
                                use: T*k, T*H, T*k*I or 4*I*H above 2^31 - 1 */
  EAAS_ERR_WORKSPACE = -3,   /* ws NULL, misaligned or smaller than the entry
                                point's eaas_workspace_bytes_for */
  EAAS_ERR_HIP = -4          /* a kernel launch was rejected by the runtime  */
};

enum eaas_dtype {
  EAAS_BF16 = 0,     /* bfloat16 bit patterns (uint16)                    */
  EAAS_FP8_E4M3 = 1, /* OCP fp8 e4m3fn bit patterns (uint8), weights only */
  EAAS_FP32 = 2,     /* IEEE binary32, outputs only                       */
  /* As a weight dtype: fp8 e4m3fn weights (as EAAS_FP8_E4M3) and fp8
   * activations.  The step quantizes x per token and h per row, per block of
   * 128 channels (s = amax/448, 1 for an all-zero block; q = e4m3(a/s),
   * nearest even, saturating at 448; fp32 arithmetic), and runs both grouped
   * GEMMs on fp8 x fp8 MFMAs with fp32 accumulation, scaling each 128-wide K
   * block's partial sums by its row scale times its weight block scale (the
   * block-scaled fp8 GEMM of the grouped-GEMM engine named in §4.1).  Needs
   * H a multiple of 256.  Accepted by every entry point that takes a
   * weight dtype. */
  EAAS_FP8_E4M3_A8 = 3,
  /* As a weight dtype: the fp8 e4m3fn weights of EAAS_FP8_E4M3 (same values,
   * same scales, same results bit for bit) stored in the tiled layout that
   * eaas_tile_weights_fp8 writes, which the decode-sized fp8 GEMMs stream as
   * contiguous blocks instead of rows K bytes apart.  Needs H a multiple of
   * 256.  Accepted by every entry point that takes a weight dtype. */
  EAAS_FP8_E4M3_TILED = 4,
  /* As the type of eaas_grouped_matmul_fp8's results: bf16, and sums in fewer bits than
   * fp32 where that is faster (see there). */
  EAAS_BF16_SHORT_SUMS = 5
};

/*
 * Routing of a batch: the token reorganisation of §3.3 plus the compacted
 * active-expert list of the group-shrink prefix scan (§4.1).  Device arrays:
 *   counts [E]    valid slots per expert
 *   offsets[E+1]  exclusive prefix sum of counts; offsets[E] = valid slots
 *   perm   [R]    row r -> slot s; rows are grouped by expert in ascending
 *                 expert id and, inside an expert, in ascending slot order
 *                 (the unique stable counting sort); rows >= offsets[E] hold -1
 *   inv    [R]    slot s -> row, or -1 for an invalid slot
 *   active [E+1]  active[0] = number of experts with counts > 0, then those
 *                 experts in ascending order, then zeros
 */
typedef struct eaas_routing {
  int32_t *counts;
  int32_t *offsets;
  int32_t *perm;
  int32_t *inv;
  int32_t *active;
} eaas_routing;

/* Bytes of workspace that every entry point below accepts for this shape and
 * weight dtype (the maximum over the entry points).  Returns 0 for a shape the
 * library rejects. */
size_t eaas_workspace_bytes(const eaas_shape *s, int w_dtype);

/* Bytes of workspace one entry point needs for this shape and weight dtype:
 *   EAAS_ENTRY_ROUTE_PERMUTE  eaas_route_permute (its histogram only; w_dtype
 *                             is ignored beyond validation)
 *   EAAS_ENTRY_FFN_GROUPED    eaas_expert_ffn_grouped (h, and for
 *                             EAAS_FP8_E4M3_A8 the quantized x; no staging)
 *   EAAS_ENTRY_FORWARD        eaas_expert_forward(_profiled), which is
 *                             eaas_workspace_bytes
 * Each is at most eaas_workspace_bytes(s, w_dtype).  Returns 0 for a shape or
 * dtype the library rejects and for an unknown entry. */
enum eaas_entry {
  EAAS_ENTRY_ROUTE_PERMUTE = 0, EAAS_ENTRY_FFN_GROUPED = 1, EAAS_ENTRY_FORWARD = 2
};
size_t eaas_workspace_bytes_for(const eaas_shape *s, int w_dtype, int entry);

/* Where a forward call leaves its intermediates inside the workspace (for
 * inspection and tests; the contents are those of the last call that used
 * the workspace, rows in the grouped order of the routing):
 *   EAAS_WS_H      h [R,I] bf16 (bf16 and fp8-weight modes)
 *   EAAS_WS_HQ     h quantized [R,I] e4m3fn codes   (EAAS_FP8_E4M3_A8)
 *   EAAS_WS_HS     its scales [R,I/128] fp32         (EAAS_FP8_E4M3_A8)
 *   EAAS_WS_XQ     x quantized [T,H] e4m3fn codes    (EAAS_FP8_E4M3_A8)
 *   EAAS_WS_XS     its scales [T,H/128] fp32         (EAAS_FP8_E4M3_A8)
 *   EAAS_WS_STAGE  expert outputs [R,H] fp32 (not yet weighted), row = slot
 *                  t*k+j (eaas_expert_forward; invalid slots untouched)
 * Writes the byte offset and size of the region.  Returns INVALID_ARG for a
 * null output pointer, an unknown region or one the dtype does not have,
 * UNSUPPORTED for a shape or dtype eaas_workspace_bytes rejects. */
enum eaas_ws_region {
  EAAS_WS_H = 0, EAAS_WS_HQ = 1, EAAS_WS_HS = 2, EAAS_WS_XQ = 3, EAAS_WS_XS = 4,
  EAAS_WS_STAGE = 5
};
int eaas_workspace_region(const eaas_shape *s, int w_dtype, int region, size_t *offset,
                          size_t *bytes);

/* Activation quantization of the EAAS_FP8_E4M3_A8 step, on its own:
 *   x [rows,K] bf16 (device), K a multiple of 128 and rows*K < 2^31
 *   q [rows,K] e4m3fn codes (device, written), s [rows,K/128] fp32 (device,
 *   written): per row and block of 128 channels, s = amax/448 (1 if the block
 *   is all zero), q = e4m3fn(x/s) rounded to nearest even and saturated at
 *   +-448, with s and x/s correctly rounded fp32.
 * x, q 16-byte aligned.  rows == 0 is a no-op.  Errors: INVALID_ARG (null or
 * misaligned pointer, rows < 0, K <= 0), UNSUPPORTED (K % 128, size), HIP. */
int eaas_quantize_rows_fp8(const void *x, int64_t rows, int32_t K, void *q, float *s,
                           void *stream);

/* The fp8 weight layout of EAAS_FP8_E4M3_TILED (weights stay resident on a
 * server, so they are rearranged once, when loaded).
 *   which    EAAS_GATE_UP: w is W_gate_up [E,2I,H] (N = 2I rows, K = H);
 *            EAAS_DOWN:    w is W_down    [E,H,I] (N = H rows, K = I)
 *   w        e4m3fn codes [E,N,K], row-major (device, read)
 *   w_tiled  E*N*K bytes (device, written), the same codes reordered: with
 *            BN = 512 for a gate/up matrix whose 2I is a multiple of 512 and
 *            256 otherwise, for expert e, N tile tn < N/BN, K tile kt < K/64,
 *            j < BN and b < 64,
 *              w_tiled[((e*(N/BN) + tn)*(K/64) + kt)*BN*64 + j*64 + b]
 *                = w[e][row(tn, j)][64*kt + b],
 *            row(tn, j) = tn*BN + j for W_down; for W_gate_up the tile's BN/2
 *            gate rows come first: row(tn, j) = tn*BN/2 + j for j < BN/2,
 *            I + tn*BN/2 + j - BN/2 otherwise.
 * The block scales are not moved.  s->T is not used (any valid value).
 * Errors: INVALID_ARG (unknown `which`, null, misaligned or overlapping
 * pointers), UNSUPPORTED (the shape, or H not a multiple of 256), HIP. */
enum eaas_matrix { EAAS_GATE_UP = 0, EAAS_DOWN = 1 };
int eaas_tile_weights_fp8(const eaas_shape *s, int which, const void *w, void *w_tiled,
                          void *stream);

/* Token reorganisation + group-shrink (§3.3 Fig. 5, §4.1).
 *   topk_ids [T,k] int32   expert id per slot (payload `expert_id`, §3.2)
 *   r                      all five arrays written, bit-exact and deterministic
 * Needs ws of eaas_workspace_bytes_for(s, EAAS_BF16, EAAS_ENTRY_ROUTE_PERMUTE)
 * bytes (a histogram of ceil(T*k/2048) x E ints); H and I only need to pass
 * validation.  k may exceed E: slots whose ids name other servers' experts are
 * skipped, so a server with fewer experts than a token has slots is valid. */
int eaas_route_permute(const eaas_shape *s, const int32_t *topk_ids,
                       const eaas_routing *r, void *ws, size_t ws_bytes,
                       void *stream);

/* Grouped expert FFN over the reorganised rows (§3.3 "grouped GEMM").
 *   x          [T,H] bf16 hidden states (payload, §3.2)
 *   r          routing produced by eaas_route_permute for the same ids
 *   w_gate_up  [E,2I,H] bf16 or fp8; w_gate_up_scale [E,2I/128,H/128] fp32
 *              for fp8, ignored (may be NULL) for bf16
 *   w_down     [E,H,I]  bf16 or fp8; w_down_scale [E,H/128,I/128] likewise
 *   y_perm     [R,H] fp32 output: row r = y_{e(r)}(x[perm[r]/k]), unweighted;
 *              rows >= offsets[E] are left untouched
 * Only experts listed in r->active are read.  Needs ws of
 * eaas_workspace_bytes_for(s, w_dtype, EAAS_ENTRY_FFN_GROUPED) bytes. */
int eaas_expert_ffn_grouped(const eaas_shape *s, const void *x,
                            const eaas_routing *r, const void *w_gate_up,
                            const float *w_gate_up_scale, const void *w_down,
                            const float *w_down_scale, int w_dtype,
                            float *y_perm, void *ws, size_t ws_bytes,
                            void *stream);

/* Weighted sum of expert outputs back into token order (§3.3 "the weighted sum
 * of expert outputs", weights = router_score of §3.2).
 *   out[t,:] = sum over ascending j with valid slot t*k+j of
 *              fp32(topk_weights[t,j] * y_perm[inv[t*k+j],:]), from +0
 *   out        [T,H] bf16 (round to nearest even of the fp32 sum) or fp32;
 *              tokens with no valid slot get zeros. */
int eaas_unpermute_combine(const eaas_shape *s, const float *y_perm,
                           const eaas_routing *r, const float *topk_weights,
                           void *out, int out_dtype, void *stream);

/* The whole step: route_permute, grouped FFN and weighted combine in one call,
 * result bitwise equal to calling the three entry points above in sequence.
 *   r      optional (NULL: routing lives in the workspace); when given it is
 *          written as by eaas_route_permute
 *   out    [T,H] bf16 or fp32.  out == x (exactly, bf16 out) is allowed: the
 *          result is written back into the request payload in place (§3.3);
 *          any other overlap of out with x is EAAS_ERR_INVALID_ARG. */
int eaas_expert_forward(const eaas_shape *s, const void *x,
                        const int32_t *topk_ids, const float *topk_weights,
                        const void *w_gate_up, const float *w_gate_up_scale,
                        const void *w_down, const float *w_down_scale,
                        int w_dtype, void *out, int out_dtype,
                        const eaas_routing *r, void *ws, size_t ws_bytes,
                        void *stream);

/* eaas_expert_forward, plus timing marks for measurement: events[0..4] are
 * hipEvent_t handles (passed as void*, NULL entries skipped) recorded on
 * `stream` before routing, before the gate/up GEMM, before the down GEMM,
 * before the combine and after it.  events itself may be NULL.  Same kernels,
 * same results as eaas_expert_forward.  (Small batches are routed inside the
 * gate/up launch: their routing interval is empty, and the gate/up interval
 * holds both.) */
int eaas_expert_forward_profiled(const eaas_shape *s, const void *x,
                                 const int32_t *topk_ids,
                                 const float *topk_weights,
                                 const void *w_gate_up,
                                 const float *w_gate_up_scale,
                                 const void *w_down, const float *w_down_scale,
                                 int w_dtype, void *out, int out_dtype,
                                 const eaas_routing *r, void *ws,
                                 size_t ws_bytes, void *stream,
                                 void *const *events);

/*
 * Dynamic batch of several clients' requests (§3.3: the server aggregates the
 * ready requests of its clients into one batch and writes each client's
 * results back into that client's payload; §3.2: a buffer slot's payload and
 * its header's batch size).
 *
 * One request, as laid out in a client's buffer slot (device pointers,
 * 16-byte aligned; only the first num_tokens[b] rows belong to the request):
 *   x            [n,H] bf16 hidden states
 *   topk_ids     [n,k] int32 expert ids (ids outside [0,E) are skipped)
 *   topk_weights [n,k] fp32 router scores
 *   out          [n,H] weighted sums, bf16 or fp32 per out_dtype.  out == x
 *                (bf16) writes the result back into the payload in place; out
 *                must not overlap any other request's arrays.
 */
typedef struct eaas_segment {
  const void *x;
  const int32_t *topk_ids;
  const float *topk_weights;
  void *out;
} eaas_segment;

/* Workspace bytes of eaas_expert_forward_segments for a capacity of s->T
 * tokens (0 for a shape the library rejects). */
size_t eaas_segments_workspace_bytes(const eaas_shape *s, int w_dtype);

/* The step on a dynamic batch of requests whose token counts are read on the
 * device, so the same call (or a captured graph of it) serves any mix of
 * batch sizes.  The tokens are walked with Algorithm 1 of §4 (a static grid
 * over requests of varying length that skips empty ones).
 *   s->T        capacity: grids and workspace are sized for at most s->T
 *               tokens in all requests together
 *   segs        [n_seg] eaas_segment, a DEVICE array
 *   num_tokens  [n_seg] int32, a DEVICE array: request b's batch size (header
 *               batch_size).  0 means no request from that client this step;
 *               negative counts count as 0.  Requests are batched in slot
 *               order; tokens past the capacity are not processed and their
 *               out rows are left untouched.
 *   n_seg       0..1024 (0: nothing enqueued)
 * For every request b, out rows [0, num_tokens[b]) receive exactly what
 * eaas_expert_forward writes for those tokens when run on the requests
 * concatenated in slot order; no other memory of the requests is written. */
int eaas_expert_forward_segments(const eaas_shape *s, const eaas_segment *segs,
                                 const int32_t *num_tokens, int n_seg,
                                 const void *w_gate_up,
                                 const float *w_gate_up_scale,
                                 const void *w_down, const float *w_down_scale,
                                 int w_dtype, int out_dtype, void *ws,
                                 size_t ws_bytes, void *stream);

/*
 * One server step over the clients' buffer slots (§3.2 "Shared Communication
 * Buffer Design", §3.3 "Asynchronous Server Operation", §3.4 offline clients).
 *
 * Every client owns one slot on the server, in device memory:
 *   flag      slot state, one of the eaas_slot_state values; the paper uses
 *             one byte, here it is a 32-bit word so that host and device can
 *             update it with naturally aligned atomic accesses
 *   header    [2] int32: layer_id, batch_size
 *   x         [capacity,H] bf16 hidden states; the step overwrites rows
 *             [0, n) with the request's weighted sums (the results are written
 *             back into the data payload, §3.3)
 *   topk_ids, topk_weights  [capacity,k] int32 / fp32 (payload, §3.2)
 * A server may hold several layers: layers[L] holds the weights of layer L
 * (the arrays and dtype of eaas_expert_forward), and requests of different
 * layers are batched into one grouped step (expert e of layer L is group
 * L*E + e).
 */
enum eaas_slot_state {
  EAAS_SLOT_EMPTY = 0,   /* the client may write a request                   */
  EAAS_SLOT_READY = 1,   /* client write done: the server may take it         */
  EAAS_SLOT_DONE = 2,    /* server computation done: the client may read      */
  EAAS_SLOT_OFFLINE = 3  /* client reported offline: the server leaves it alone */
};

typedef struct eaas_slot {
  int32_t *flag;
  const int32_t *header;
  void *x;
  const int32_t *topk_ids;
  const float *topk_weights;
  int64_t capacity;
} eaas_slot;

typedef struct eaas_layer_weights {
  const void *w_gate_up;
  const float *w_gate_up_scale;
  const void *w_down;
  const float *w_down_scale;
} eaas_layer_weights;

/* Workspace bytes of eaas_server_step (0 for a shape the library rejects). */
size_t eaas_server_workspace_bytes(const eaas_shape *s, int n_layers, int w_dtype);

/* One server step: snapshot the slot flags, take the ready slots (flag 1) in
 * slot order while their batch sizes (clamped to [0, capacity]) fit the step
 * capacity s->T, run them as one dynamic batch, write each request's weighted
 * sums (bf16) over its hidden states, then set the taken slots' flags to 2.
 *   s->E        experts per layer; n_layers * s->E <= 1024
 *   slots       [n_slots] eaas_slot, a DEVICE array; n_slots 0..1024
 *   layers      [n_layers] eaas_layer_weights, a DEVICE array, all of w_dtype
 * Slots in any other state, ready slots that do not fit (they stay ready for a
 * later step), and payload rows past a request are not written.  A taken
 * request whose layer_id names no layer of this server gets zeros.  Within a
 * taken request, every row equals eaas_expert_forward on the requests of its
 * layer concatenated in slot order.  The flags are written after all results,
 * behind a system-scope fence.  Two steps over the same slots must not
 * overlap in time (a later step runs on the same stream or after the first). */
int eaas_server_step(const eaas_shape *s, const eaas_slot *slots, int n_slots,
                     const eaas_layer_weights *layers, int n_layers, int w_dtype,
                     void *ws, size_t ws_bytes, void *stream);

/*
 * For callers that cannot allocate device memory: code under hipGraph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  eaas_expert_forward
 * with the caller's workspace replaced by a library-owned device array of
 * EAAS_NOALLOC_SCRATCH_BYTES bytes per GPU: static device memory that every
 * GPU the library is loaded on holds until the process ends.  The call itself
 * allocates and frees nothing.
 *   Same arguments and results as eaas_expert_forward (bitwise), without
 *   ws / ws_bytes.  The array used is that of the device current at the call
 *   (hipGetDevice), which must be the device `stream` belongs to.
 *   A shape that needs more, eaas_workspace_bytes(s, w_dtype) >
 *   EAAS_NOALLOC_SCRATCH_BYTES (80 MiB: it holds the 256-token, H 7168, I 2048,
 *   32-expert, top-8 decode step with fp8 or bf16 weights), returns
 *   EAAS_ERR_WORKSPACE and enqueues nothing; other errors as in
 *   eaas_expert_forward.
 *   Every call on one GPU shares that GPU's array, which keeps the last
 *   call's intermediates (each call rebuilds everything it reads, so nothing
 *   has to start at zero).  Calls that overlap in time on one GPU (on
 *   different streams, or from several host threads) race on the array and
 *   give undefined results: serialise them, e.g. on one stream.
 */
#define EAAS_NOALLOC_SCRATCH_BYTES (80u << 20)
int eaas_expert_forward_noalloc(const eaas_shape *s, const void *x,
                                const int32_t *topk_ids,
                                const float *topk_weights,
                                const void *w_gate_up,
                                const float *w_gate_up_scale,
                                const void *w_down, const float *w_down_scale,
                                int w_dtype, void *out, int out_dtype,
                                const eaas_routing *r, void *stream);

/*
 * The products of an expert layer on their own, for training the experts and
 * for serving them in 8-bit integers.  eaas_expert_forward fuses them into one
 * step; here each is a call, so that a caller can keep what a gradient needs.
 *
 * Rows are grouped by expert as by eaas_route_permute: group e holds the rows
 * [offsets[e], offsets[e+1]), which may be none, and rows from offsets[E] on
 * belong to no group: they are neither read into a result nor written.
 *   offsets  [E+1] int32 (device), ascending from 0, at most R; values outside
 *            are clamped to that range
 * A row array has rows ld elements apart (ld >= its width): rows cut out of a
 * wider array need no copy.  Its base needs no more alignment than an element;
 * sizes, strides and bases that are multiples of 16 bytes are faster.  Weights
 * W [E,N,K] are contiguous and 16-byte aligned.
 *   perm, k  perm == NULL: row r of the product reads row r of x.  Otherwise x
 *            is in token order, [R/k, K], R a multiple of k, and row r reads
 *            token perm[r]/k (the perm of the routing, values clamped to
 *            [0, R)): the reorganised copy of the tokens is never made.
 * bf16 operands, products of them exact, sums in fp32; 8-bit operands, sums in
 * int32.  Every sum is taken in a fixed order: equal calls give equal bits.
 */
typedef struct eaas_group_shape {
  int32_t R; /* rows of the grouped arrays, >= 0                        */
  int32_t E; /* groups, 1..1024                                         */
  int32_t N; /* outputs of an expert's matrix (its rows), >= 1          */
  int32_t K; /* inputs of an expert's matrix (its columns), >= 1        */
} eaas_group_shape;

/* Bytes of workspace that the grouped products of bf16 and of 8-bit integers accept for
 * this shape, those with an activation included (partial sums, where a long sum is split
 * over workgroups).  Conventions of `ws` as above.  0 for a shape the library rejects: see
 * the limits at eaas_grouped_matmul. */
size_t eaas_grouped_workspace_bytes(const eaas_group_shape *s);

/* y[r,:] = W[e] x[src(r),:] for the rows r of every group e.
 *   x [R or R/k, K] bf16 (ldx), w [E,N,K] bf16, y [R,N] bf16 or fp32 (ldy)
 * y must not overlap x or w (rows side by side in one wider array do not).
 * Errors: INVALID_ARG (null pointer, size below its least, ld below the width, k < 1
 * or R % k with perm, overlap, alignment), UNSUPPORTED (E > 1024, N*K or, with perm,
 * (R/k)*ldx above 2^31 - 1, an ld above 2^22), WORKSPACE, HIP.  R = 0: nothing is
 * enqueued. */
int eaas_grouped_matmul(const eaas_group_shape *s, const void *x, int64_t ldx,
                        const int32_t *perm, int32_t k, const int32_t *offsets,
                        const void *w, void *y, int64_t ldy, int y_dtype,
                        void *ws, size_t ws_bytes, void *stream);

/* Its gradient in the rows: dx[r,:] = W[e]^T dy[r,:].
 *   dy [R,N] bf16 (lddy), dx [R,K] bf16 or fp32 (lddx), in grouped order: with
 * weights of 1, eaas_unpermute_combine sums fp32 dx into the tokens' gradients.
 * Errors as eaas_grouped_matmul. */
int eaas_grouped_matmul_dx(const eaas_group_shape *s, const void *dy, int64_t lddy,
                           const int32_t *offsets, const void *w, void *dx, int64_t lddx,
                           int dx_dtype, void *ws, size_t ws_bytes, void *stream);

/* Its gradient in the weights: dW[e] = sum over the rows r of group e of
 * dy[r,:] x[src(r),:]^T; zeros for a group without rows.
 *   dw [E,N,K] bf16 or fp32, contiguous, 16-byte aligned
 *   accumulate != 0 (fp32 only): dw += that sum (micro-batches of one step)
 * R = 0 writes zeros (accumulate: nothing); dy, x and perm may then be NULL.
 * Errors as eaas_grouped_matmul; INVALID_ARG for accumulate with bf16. */
int eaas_grouped_matmul_dw(const eaas_group_shape *s, const void *dy, int64_t lddy,
                           const void *x, int64_t ldx, const int32_t *perm, int32_t k,
                           const int32_t *offsets, void *dw, int dw_dtype, int accumulate,
                           void *ws, size_t ws_bytes, void *stream);

/* Rows in 8-bit integers, one scale per row: s = amax * (1/127) with the constant
 * rounded to fp32 (1 where that is zero: rows of zeros, or below 2^-143), q = x/s to
 * the nearest integer, ties to even; product and quotients in fp32, correctly rounded.
 * A row that holds an infinity or a NaN gets a NaN scale and zero codes, so whatever is
 * computed from it is NaN.
 *   x [rows,K] bf16 (ldx), q [rows,K] int8 and s [rows] fp32, contiguous
 * Quantizes activations per token, and weights [E,N,K] per output channel
 * (rows = E*N).  rows = 0: nothing.  Errors: INVALID_ARG, UNSUPPORTED (rows or K
 * above 2^31 - 1, K above 2^22), HIP. */
int eaas_quantize_rows_int8(const void *x, int64_t ldx, int64_t rows, int32_t K, void *q,
                            float *s, void *stream);

/* The grouped product in 8-bit integers:
 *   y[r,n] = (sum_k xq[src(r),k] wq[e,n,k]) * xs[src(r)] * wscale[e,n]
 * with an exact int32 sum, rounded to fp32 before the two fp32 products (in this
 * order).  xq [R or R/k, K] int8 contiguous with xs fp32 per row of xq, wq
 * [E,N,K] int8, wscale [E,N] fp32, y [R,N] bf16 or fp32 (ldy).  K < 2^17 (the
 * sum fits).  Errors as eaas_grouped_matmul. */
int eaas_grouped_matmul_int8(const eaas_group_shape *s, const void *xq, const float *xs,
                             const int32_t *perm, int32_t k, const int32_t *offsets,
                             const void *wq, const float *wscale, void *y, int64_t ldy,
                             int y_dtype, void *ws, size_t ws_bytes, void *stream);

/* e4m3 codes with a scale for each block: 128 columns of a row, or 128 x 128 of a
 * matrix.
 *   x          [mats*rows,K] bf16 or fp32 (x_dtype), rows ldx elements apart: `mats`
 *              matrices of `rows` rows each
 *   block_rows 1: a scale for each 128 columns of a row (activations, per token);
 *              128: for each 128 x 128 block of a matrix, counted from its first row
 *              and column (weights [E,N,K]: mats = E, rows = N)
 *   q [mats*rows,K] e4m3fn codes, s [mats,ceil(rows/block_rows),ceil(K/128)] fp32,
 *              contiguous; the last block of a row or column may be narrower
 * s = amax * (1/448) with the constant rounded to fp32 (1 where that is zero), q =
 * e4m3fn(x/s) to the nearest, ties to even, saturated at +-448; product and quotients in
 * fp32, correctly rounded.  (eaas_quantize_rows_fp8 divides by 448: its scales differ by a
 * unit in the last place at most.)  A block that holds an infinity or a NaN gets a NaN
 * scale and zero codes, so whatever is computed from it is NaN.  rows or mats = 0:
 * nothing.  Errors: INVALID_ARG (also overlaps), UNSUPPORTED (mats*rows above 2^31 - 1, K
 * or ldx above 2^22), HIP. */
int eaas_quantize_blocks_fp8(const void *x, int x_dtype, int64_t ldx, int32_t mats, int64_t rows,
                             int32_t K, int32_t block_rows, void *q, float *s, void *stream);

/* Bytes of workspace of eaas_grouped_matmul_fp8 (0 for a shape the library rejects). */
size_t eaas_grouped_fp8_workspace_bytes(const eaas_group_shape *s);

/* The grouped product of e4m3 codes with the scales of eaas_quantize_blocks_fp8:
 *   y[r,n] = sum_b xs[src(r),b] wscale[e,n/128,b] (sum_{k in b} xq[src(r),k] wq[e,n,k])
 * over the blocks b of 128 columns (the last one may be narrower).
 *   xq [R or R/k, K] contiguous with xs [.., ceil(K/128)] fp32; wq [E,N,K], 16-byte
 *   aligned, with wscale [E,ceil(N/128),ceil(K/128)] fp32; y [R,N] bf16 or fp32 (ldy)
 * Products are exact and every sum is taken in fp32.  With y_dtype EAAS_BF16_SHORT_SUMS the
 * bf16 results of large groups come from the 8-bit floating matrix instructions, at up to
 * twice the rate: eight products at a time are added after each has been rounded to a
 * multiple of 2^-13 of the power of two under the largest of them, which moves a result by
 * at most 7 * 2^-14 of its terms' magnitudes in all (by 2^-16 of the results' norm for
 * normal data; the rounding to bf16 is 2^-8).  Whether a group is large depends on the
 * batch, and so do such results.  Products of a row's scale and a block's have to lie in
 * fp32's normal range (or be zero) there; otherwise results alone have to lie in fp32's.  The
 * sums of the blocks are added in fp32 either way.
 * Gradient in the rows: the same call with the transposed codes [E,K,N] and scales
 * [E,ceil(K/128),ceil(N/128)], and dy quantized as rows.
 * ws of eaas_grouped_fp8_workspace_bytes.  Errors as eaas_grouped_matmul. */
int eaas_grouped_matmul_fp8(const eaas_group_shape *s, const void *xq, const float *xs,
                            const int32_t *perm, int32_t k, const int32_t *offsets,
                            const void *wq, const float *wscale, void *y, int64_t ldy,
                            int y_dtype, void *ws, size_t ws_bytes, void *stream);

/* The gated half of the expert FFN in one product: for the rows r of every group e,
 *   h[r,:] = silu(W_gate[e] x[src(r),:]) * (W_up[e] x[src(r),:])
 * with s->N = 2I and w [E,2I,K] bf16, gate rows [0,I), up rows [I,2I).  Both sums are
 * fp32 and reach the activation unrounded; h is rounded once.
 *   x, perm, k, offsets  as in eaas_grouped_matmul
 *   h   [R,I] bf16 (ldh)
 *   gu  NULL, or [R,2I] bf16 (ldgu): the sums (gate, then up), rounded, which
 *       eaas_grouped_swiglu_backward and eaas_swiglu_backward read
 * h and gu overlap nothing (rows side by side in one wider array do not).  ws of
 * eaas_grouped_workspace_bytes(s).  Errors as eaas_grouped_matmul; INVALID_ARG also for
 * an odd N. */
int eaas_grouped_swiglu(const eaas_group_shape *s, const void *x, int64_t ldx,
                        const int32_t *perm, int32_t k, const int32_t *offsets, const void *w,
                        void *h, int64_t ldh, void *gu, int64_t ldgu, void *ws, size_t ws_bytes,
                        void *stream);

/* Its way back from the gradient of what follows it, the product y = W_down h:
 *   dh[r,:] = W_down[e]^T dy[r,:]                     (fp32, not stored)
 *   dgate = dh up t (1 + gate (1 - t)),  dup = dh gate t,  t = 1 / (1 + exp(-gate))
 *   w    [E,N,K] bf16: W_down, K = I;  dy [R,N] bf16 (lddy)
 *   gu   [R,2K] bf16 (ldgu): gate, then up
 *   dgu  [R,2K] bf16 (lddgu): dgate, then dup; may be gu itself (the same base and ldgu)
 *   h    NULL, or [R,K] bf16 (ldh): silu(gate) * up of the rounded gate and up, for
 *        W_down's gradient eaas_grouped_matmul_dw(dy, h)
 * The gradients of x and of W_gate_up are those of eaas_grouped_matmul for dgu.  No other
 * overlap.  ws of eaas_grouped_workspace_bytes(s).  Errors as eaas_grouped_matmul
 * (ldgu and lddgu too are at most 2^22). */
int eaas_grouped_swiglu_backward(const eaas_group_shape *s, const void *dy, int64_t lddy,
                                 const int32_t *offsets, const void *w, const void *gu,
                                 int64_t ldgu, void *dgu, int64_t lddgu, void *h, int64_t ldh,
                                 void *ws, size_t ws_bytes, void *stream);

/* The activation between the products, for rows of the grouped arrays:
 *   h = silu(gate) * up,  silu(g) = g / (1 + exp(-g)), in fp32
 *   gu      [rows,2I] bf16, contiguous: gate columns [0,I), up columns [I,2I)
 *   h       [rows,I] bf16 (rounded once), contiguous
 *   n_rows  NULL, or a device int32 (offsets + E of the routing): only the first
 *           min(rows, max(0, *n_rows)) rows are read and written
 * rows = 0: nothing.  Errors: INVALID_ARG (null, overlap of an output with an
 * input, element alignment), UNSUPPORTED (rows or I above 2^31 - 1, I above
 * 2^21), HIP. */
int eaas_swiglu(const void *gu, int64_t rows, int32_t I, const int32_t *n_rows, void *h,
                void *stream);

/* The same, quantized as by eaas_quantize_rows_int8 instead of rounded to bf16
 * (codes and scales are those of the fp32 h, which is within about two units in its
 * last place, for gates of any size): q [rows,I] int8, s [rows] fp32. */
int eaas_swiglu_int8(const void *gu, int64_t rows, int32_t I, const int32_t *n_rows, void *q,
                     float *s, void *stream);

/* The same as e4m3 codes with a scale for each 128 columns, as by
 * eaas_quantize_blocks_fp8 of h rounded once to fp32: q [rows,I], s
 * [rows,ceil(I/128)] fp32, contiguous. */
int eaas_swiglu_fp8(const void *gu, int64_t rows, int32_t I, const int32_t *n_rows, void *q,
                    float *s, void *stream);

/* Its gradient: with t = 1 / (1 + exp(-gate)),
 *   dgate = dh up t (1 + gate (1 - t)),  dup = dh gate t
 *   dh [rows,I] bf16, dgu [rows,2I] bf16 (dgate, then dup), contiguous.  dgu may
 *   be gu itself (exactly); no other overlap. */
int eaas_swiglu_backward(const void *gu, const void *dh, int64_t rows, int32_t I,
                         const int32_t *n_rows, void *dgu, void *stream);

/* Gradients of eaas_unpermute_combine: for every valid slot t*k+j at row r,
 *   dy_perm[r,:]      = topk_weights[t,j] * dout[t,:]        (bf16)
 *   dweights[t,j]     = sum over c of dout[t,c] * y_perm[r,c]   (fp32)
 * dweights of an invalid slot is 0; rows of dy_perm past the valid ones are left
 * untouched.
 *   dout [T,H] bf16 or fp32, y_perm [R,H] fp32, dy_perm [R,H] bf16, dweights
 *   [T,k] fp32; outputs overlap nothing.  Errors as eaas_unpermute_combine. */
int eaas_unpermute_combine_backward(const eaas_shape *s, const void *dout, int dout_dtype,
                                    const float *y_perm, const eaas_routing *r,
                                    const float *topk_weights, void *dy_perm, float *dweights,
                                    void *stream);

/* Static, human-readable name of a status code. */
const char *eaas_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* EAAS_H */
