/*
 * mmoe -- forward pass of one multi-model MoE layer on AMD MI355X (gfx950).
 *
 * Several fine-tuned variants of one MoE model are served from a single
 * consolidated pool of experts (paper, section 3.1: similar experts of the
 * variants are loaded once and shared; Algorithm 1 emits the expert map).  At
 * inference (Algorithm 2, the per-layer body; Figure 3) the requested variant's
 * own gate scores the token, the top experts are selected, each selected
 * (variant, expert) is looked up in the map, the resident expert for that
 * location is applied -- possibly another variant's when the location is
 * consolidated, the variant's own otherwise -- and the results are combined
 * with the gate's coefficients (section 3.2).
 *
 * This library evaluates that layer for a batch that mixes tokens of several
 * variants.  Every token carries its variant id; the map is the table
 * M[v][e] -> pool slot; the pool holds each resident expert once.
 *
 * Conventions
 *   T tokens, d = d_model, f = d_ff, V variants, E experts per variant,
 *   k = top_k, S pool slots, P = T*k (token, pick) pairs, pair id p = t*k + j.
 *   All tensors are dense and row-major.  "dtype" is the storage type of X, Wr,
 *   the pool, H and Y; every product is accumulated in fp32.  (fp32 batches with many rows per
 *   slot may run on the bf16 matrix instruction, every number as three bf16 parts that together
 *   hold all of its 24 bits over the whole range of fp32; products of the parts below 2^-24 of
 *   the term are left out.)
 *
 * Pointers
 *   Every pointer except mmoe_shape* is a DEVICE pointer owned by the caller.
 *   The library never allocates, frees or keeps device memory; scratch comes
 *   from the caller's workspace `ws` (at least mmoe_workspace_bytes(), 256-byte
 *   aligned).  Inputs are read-only, outputs are fully overwritten.  `stream`
 *   is a hipStream_t passed as void*; every call is asynchronous on it and
 *   never synchronises the host (mmoe_validate_inputs excepted).
 *
 * Errors
 *   0 on success, a negative mmoe_status otherwise.  Only host-checkable faults
 *   are detected: null pointers, bad dimensions, unsupported combinations,
 *   small workspace, misalignment, launch failures.  Device data is not
 *   validated on the hot path: vid[t] outside [0,V), M[v][e] outside [0,S) or
 *   non-finite logits give undefined results (use mmoe_validate_inputs).
 *
 * Limits
 *   d_model and d_ff multiples of 256; E <= 256; top_k <= min(E, 8); S <= 1024;
 *   P*max(d,f) < 2^35, and < 2^31 for bf16 batches large enough for the matrix-core expert
 *   kernels (P > 16*S, or 32*S when d*f <= 4 Mi): otherwise MMOE_ERR_LIMIT.  SWIGLU needs W3, RELU and GELU need W3 == NULL.
 */
#ifndef MMOE_H
#define MMOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { MMOE_F32 = 0, MMOE_BF16 = 1 } mmoe_dtype;
typedef enum { MMOE_RELU = 0, MMOE_SWIGLU = 1, MMOE_GELU = 2 } mmoe_act;
/*
 * How the gate's coefficients are formed (section 3.2: "the gate network generates weighted
 * averaging coefficients for each expert, and ... the top experts are selected"; the paper gives
 * no formula, and its two model families differ):
 *   MMOE_GATE_SELECTED  softmax over the k selected logits; the coefficients of a token sum to 1
 *                       (k = 1 gives exactly 1).  The Mixtral-style top-2 gate.
 *   MMOE_GATE_ALL       softmax over all E logits; every selected expert keeps its own probability,
 *                       nothing is renormalised, so the coefficients sum to less than 1 unless
 *                       k = E.  The Switch-style top-1 gate (section 4.3's model family).
 * The selection itself (k largest logits, ties to the lower index) is the same in both.
 */
typedef enum { MMOE_GATE_SELECTED = 0, MMOE_GATE_ALL = 1 } mmoe_gate;

typedef enum {
    MMOE_OK = 0,
    MMOE_ERR_NULL = -1,      /* a required pointer is NULL                               */
    MMOE_ERR_DIM = -2,       /* a dimension is not positive                              */
    MMOE_ERR_TOPK = -3,      /* top_k > E or top_k > 8                                   */
    MMOE_ERR_DTYPE = -4,     /* unknown dtype, activation or gate code                   */
    MMOE_ERR_W3 = -5,        /* W3 missing for SWIGLU, or given for RELU / GELU          */
    MMOE_ERR_WORKSPACE = -6, /* ws is NULL or ws_bytes too small                         */
    MMOE_ERR_ALIGN = -7,     /* a tensor pointer is not 16-byte (ws: 256-byte) aligned   */
    MMOE_ERR_MULTIPLE = -8,  /* d_model or d_ff is not a multiple of 256                 */
    MMOE_ERR_LIMIT = -9,     /* E, S or the problem size exceeds the limits above        */
    MMOE_ERR_LAUNCH = -10,   /* the HIP runtime refused a kernel launch                  */
    MMOE_ERR_STATIC_LIMIT = -11, /* the shape needs more than MMOE_STATIC_WORKSPACE_BYTES    */
    MMOE_ERR_HEAD = -12,     /* a head size, rotated part or number of heads is not supported */
    MMOE_ERR_STRIDE = -13,   /* a stride is too short or not a multiple of 16 bytes          */
    MMOE_ERR_FORMAT = -14    /* unknown cache format, rotary layout or scaling, or one that does not go with the type */
} mmoe_status;

typedef struct {
    int32_t T;       /* tokens in the batch                      */
    int32_t d_model; /* hidden size d                            */
    int32_t d_ff;    /* expert inner size f                      */
    int32_t V;       /* model variants                           */
    int32_t E;       /* experts per variant                      */
    int32_t S;       /* slots in the consolidated pool           */
    int32_t top_k;   /* experts selected per token               */
    int32_t dtype;   /* mmoe_dtype                               */
    int32_t act;     /* mmoe_act                                 */
    int32_t gate;    /* mmoe_gate                                */
    int32_t tile_rows; /* tuning, normally 0: token rows per tile of the matrix-core expert kernels.
                          0 chooses by shape: 128 rows (two workgroups per compute unit) when tiles are
                          short-lived (d_model <= 1536, or few rows per slot on average: under 100 up to
                          d_model 2048, under 64 beyond; the down product takes 256 rows there too where 128 would be
                          more tiles than compute units and 256 are not, with d_ff of 2048 and more and 64 rows per slot
                          and more), 256 rows otherwise.  128 or 256 forces that height for the call.  Either height sums
                          every output element in the same order: the results are bit-identical.  Any
                          other value: MMOE_ERR_DIM.  Ignored by fp32 and by shapes that use the streaming kernels. */
} mmoe_shape;

/* Host only, pure.  Workspace (bytes) sufficient for every call below, 0 if the shape is invalid. */
size_t mmoe_workspace_bytes(const mmoe_shape *shape);

/* Host only.  Text for a status code (static storage). */
const char *mmoe_strerror(int status);

/*
 * One-time repacking of the pool, done when the pool is loaded (the paper's
 * loader runs once, offline, before serving: section 3.1).  The boundary's
 * plain layout is "in x out": W1, W3 [S, d, f] and W2 [S, f, d].  The expert
 * kernels read the packed pool that this call writes; each packed matrix has as
 * many elements as the plain one.  With out[n] = sum_k x[k] W[k][n], N outputs, K inputs:
 *   fp32: the transpose [S, N, K] (reduction dimension contiguous);
 *   bf16: matrix-core fragments.  Element (n, k) of slot s is stored at
 *         ((((s*(N/32) + n/32)*(K/16) + ks)*64 + 32*h + n%32)*8 + k%8
 *         with m = k/64, h = (k%64)/32, kk = (k%32)/8, ks = 4*m + kk:
 *         the 64 pieces of 16 bytes that follow each other are exactly the 32-row x 16-k
 *         operand of v_mfma_f32_32x32x16_bf16 as its 64 lanes hold it.
 * W3/W3p are NULL for RELU and GELU.  Outputs must not overlap inputs.
 */
int mmoe_pack_weights(const mmoe_shape *shape, const void *W1, const void *W3, const void *W2,
                      void *W1p, void *W3p, void *W2p, void *stream);

/*
 * Step R -- gate of the requested variant (Algorithm 2, "gate(act)"; section 3.2).
 *   logit[t,e] = <X[t,:], Wr[vid[t],e,:]> (+ br[vid[t],e])
 *   the k largest logits are selected, ties to the lower expert index, listed in
 *   selection (descending) order; w[t,j] = softmax over the k selected logits
 *   (MMOE_GATE_SELECTED) or entry j's probability in the softmax over all E logits (MMOE_GATE_ALL).
 * The logit is an fp32 sum in a fixed order, so that the selected indices are
 * reproducible bit for bit: element i belongs to lane (i div 4) mod 64; a lane
 * accumulates its elements in ascending i with one fused multiply-add each,
 * starting from +0; the 64 partial sums are combined by the butterfly
 * "for off in 32,16,8,4,2,1: p[l] = p[l] + p[l xor off]"; the bias is added last.
 *   X [T,d] dtype; vid [T] int32; Wr [V,E,d] dtype; br [V,E] fp32 or NULL;
 *   topk_idx [T,k] int32 out; topk_w [T,k] fp32 out.
 */
int mmoe_route(const mmoe_shape *shape, const void *X, const int32_t *vid, const void *Wr,
               const float *br, int32_t *topk_idx, float *topk_w, void *stream);

/*
 * Steps M and G -- expert-map lookup and grouping by pool slot (Algorithm 2, the
 * "map[iL][iE]" lookup; section 3.2: a hit uses the resident expert whoever owns it,
 * a miss the requested variant's own, which here is a private slot).
 *   slot[p] = M[vid[t]][topk_idx[p]];  counts[s] = #{p : slot[p] = s};
 *   offsets = exclusive prefix sum of counts, offsets[S] = P;
 *   perm = pair ids sorted by (slot, p) (stable);  inv_perm[perm[r]] = r;
 *   Xg[r,:] = X[perm[r] / k, :].
 * Deterministic: no result depends on the order in which threads run.
 *   M [V,E] int32 in [0,S);  slot, perm, inv_perm [P];  counts [S];  offsets [S+1];
 *   Xg [P,d] dtype.  Uses `ws`.
 */
int mmoe_remap_permute(const mmoe_shape *shape, const void *X, const int32_t *vid,
                       const int32_t *topk_idx, const int32_t *M, int32_t *slot, int32_t *counts,
                       int32_t *offsets, int32_t *perm, int32_t *inv_perm, void *Xg, void *ws,
                       size_t ws_bytes, void *stream);

/*
 * Step F -- the resident experts applied to their groups (Algorithm 2,
 * "expert[iL][iE](act)"; section 3.2: a Mixtral expert has 3*d*f parameters).
 * For every slot s and row r in [offsets[s], offsets[s+1]):
 *   SWIGLU: Yg[r,:] = (silu(Xg[r,:] W1[s]) * (Xg[r,:] W3[s])) W2[s],  silu(a) = a/(1+exp(-a))
 *   RELU:   Yg[r,:] = relu(Xg[r,:] W1[s]) W2[s]
 *   GELU:   Yg[r,:] = gelu(Xg[r,:] W1[s]) W2[s],  gelu(a) = a/2 (1 + erf(a / sqrt 2))
 * Products accumulate in fp32; the hidden activation is stored in `dtype`
 * (rounded to nearest even for bf16) between the two products.
 *   Xg [P,d] dtype; offsets [S+1] int32 (device); W1p, W3p, W2p: PACKED pool
 *   (see mmoe_pack_weights);  Yg [P,d] fp32 out.  Uses `ws` for the hidden activation.
 */
int mmoe_expert_ffn(const mmoe_shape *shape, const void *Xg, const int32_t *offsets,
                    const void *W1p, const void *W3p, const void *W2p, float *Yg, void *ws,
                    size_t ws_bytes, void *stream);

/*
 * Step C -- combination with the gate's coefficients (section 3.2):
 *   Y[t,:] = sum_{j<k} topk_w[t,j] * Yg[inv_perm[t*k+j], :], fp32, ascending j,
 * rounded once to `dtype`.  Gather-side: no atomics, deterministic.
 *   Yg [P,d] fp32; inv_perm [P]; topk_w [T,k] fp32; Y [T,d] dtype out.
 */
int mmoe_combine(const mmoe_shape *shape, const float *Yg, const int32_t *inv_perm,
                 const float *topk_w, void *Y, void *stream);

/*
 * The whole layer, R -> M -> G -> F -> C, on one stream with no host
 * synchronisation; intermediates live in `ws`.  Arguments as above; the pool is
 * the PACKED one.  Y [T,d] dtype out.  The gathered copy Xg is not materialised: the
 * expert stage reads row perm[r] / k of X where the staged call reads row r of Xg; the
 * result is bit-identical to the staged calls'.
 */
int mmoe_layer_forward(const mmoe_shape *shape, const void *X, const int32_t *vid, const void *Wr,
                       const float *br, const int32_t *M, const void *W1p, const void *W3p,
                       const void *W2p, void *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * The layer with part of the pool in host memory: Algorithm 2's miss branch (section 3.2: on a
 * miss the requested variant's own expert is loaded from the host; section 5.1: the copy is what a
 * miss costs).  resident[s] (HOST array of S flags) says whether slot s of the DEVICE pool holds
 * its expert; for every other slot host_W1p[s], host_W3p[s], host_W2p[s] (HOST arrays of S
 * pointers) point to the slot's PACKED matrices in PINNED host memory (the layout
 * mmoe_pack_weights writes, one slot each).  The call
 *   - runs the gate, the map lookup and the grouping, then SYNCHRONISES `stream` once to learn
 *     which slots the batch touches (the copies to issue depend on the routing);
 *   - copies every touched non-resident slot into its place in the device pool on `copy_stream`
 *     (a second stream of the default priority, not `stream`);
 *   - applies the resident experts to their groups while the copies run, then the fetched ones,
 *     and combines: Y is bit-identical to mmoe_layer_forward on a fully resident pool.
 * The pool's non-resident slots are scratch until fetched; a fetched slot stays valid afterwards,
 * and fetched[s] (HOST out, may be NULL) tells the caller which ones arrived, so that it can mark
 * them resident for later calls (the paper leaves open what is evicted).  Returns the number
 * of slots fetched (>= 0) or a negative status.  Everything queued on `stream` before the call may
 * still read the pool: the copies wait for it.
 */
int mmoe_layer_forward_paged(const mmoe_shape *shape, const void *X, const int32_t *vid, const void *Wr,
                             const float *br, const int32_t *M, void *W1p, void *W3p, void *W2p,
                             const uint8_t *resident, const void *const *host_W1p,
                             const void *const *host_W3p, const void *const *host_W2p, void *Y, void *ws,
                             size_t ws_bytes, void *stream, void *copy_stream, uint8_t *fetched);

/*
 * mmoe_layer_forward for callers that cannot allocate device memory or hand over a workspace:
 * code that runs under HIP graph capture, tight serving loops (one decode step after the
 * other), harnesses that forbid allocation.  Same arguments without `ws`; same kernels, same
 * results bit for bit.  The intermediates live in a fixed array of
 * MMOE_STATIC_WORKSPACE_BYTES in device memory that belongs to the library's code object (each
 * GPU the library runs on holds its own copy until the process ends).  The call allocates and
 * frees nothing.  A shape with mmoe_workspace_bytes() up to that size is accepted; one above it is
 * refused with MMOE_ERR_STATIC_LIMIT before anything is launched, unless only its tile lists take it
 * there: the limit counts them as two lists per product of 16 bytes for every 32 rows, slot and 1024
 * features, and the array has the rest beside it.  (64 MiB covers decode-shaped batches: up to about
 * 700 tokens of the Mixtral shape, 6000 of the Switch shape.)
 * Every call on one GPU uses that GPU's one array, whatever the stream: two calls that overlap
 * in time on one GPU race; order them (same stream, or events).  Nothing in the array has to
 * start at zero: every intermediate is written before it is read, so the contents left by an
 * earlier call do not matter.  The array's address is looked up on the first call on each
 * device; make that call outside of any stream capture.
 */
#define MMOE_STATIC_WORKSPACE_BYTES (64u << 20)
int mmoe_layer_forward_static(const mmoe_shape *shape, const void *X, const int32_t *vid,
                              const void *Wr, const float *br, const int32_t *M, const void *W1p,
                              const void *W3p, const void *W2p, void *Y, void *stream);

/*
 * mmoe_layer_forward with timing marks, for benchmarks and profilers.  `events` is a HOST
 * array of MMOE_NUM_EVENTS hipEvent_t (as void*), created by the caller with timing
 * enabled; events[MMOE_EV_START] is recorded on `stream` before the first kernel and
 * events[i] right after the last kernel of stage i, so that the elapsed time between two
 * consecutive events is the duration of one stage (the expert stage is split into its up
 * product + activation and its down product: one kernel each).  A NULL entry is skipped (a
 * caller that wants one kernel's duration passes the two events around it); NULL `events`
 * makes this identical to mmoe_layer_forward.  The results do not depend on `events`.
 */
enum {
    MMOE_EV_START = 0,
    MMOE_EV_ROUTE = 1,    /* after step R                                         */
    MMOE_EV_PERMUTE = 2,  /* after steps M and G                                  */
    MMOE_EV_FFN_UP = 3,   /* after H = act(Xg W1 [, Xg W3])                       */
    MMOE_EV_FFN_DOWN = 4, /* after Yg = H W2                                      */
    MMOE_EV_COMBINE = 5,  /* after step C                                         */
    MMOE_NUM_EVENTS = 6
};
int mmoe_layer_forward_events(const mmoe_shape *shape, const void *X, const int32_t *vid,
                              const void *Wr, const float *br, const int32_t *M, const void *W1p,
                              const void *W3p, const void *W2p, void *Y, void *ws, size_t ws_bytes,
                              void *stream, void *const *events);

/*
 * Host only, pure: which expert-stage kernels
 * mmoe_expert_ffn and mmoe_layer_forward will use for this shape.  *streaming = 1: the
 * weight-streaming kernels (few rows per slot), *tile_rows = 32
 * (rows of a slot per pass over its weights); *streaming = 0: the matrix-core kernels with
 * tiles of up to *tile_rows (128 or 256; fp32: 96) token rows.  Where that is 128 and the shape's tile_rows is 0, tiles of
 * the down product may have up to 256.  The choice depends on the shape only.
 */
int mmoe_expert_plan(const mmoe_shape *shape, int *streaming, int *tile_rows);

/*
 * Measurement aid, SYNCHRONISES the stream; not part of the layer.  Measures what this GPU
 * delivers for the two resources that bound the expert stage: out[0] = GB/s of a pure
 * streaming read of `buf` (DEVICE memory, `bytes` >= 64 MiB, 256-byte aligned, zero-filled by
 * the caller; its last MiB is written), out[1] = TFLOP/s of a loop of
 * v_mfma_f32_16x16x32_bf16, the expert kernels' instruction, on random register operands with no
 * memory traffic.  `out` is a HOST array of two floats.  Benchmarks print these beside the data-sheet peaks.
 */
int mmoe_probe_ceilings(void* buf, size_t bytes, float* out, void* stream);

/*
 * The initial expert loader's table (Algorithm 1; section 3.1), run once, offline, before
 * serving.  V fine-tuned variants of one MoE model, L layers of E experts; the expert block of
 * a location (layer, expert) is the concatenation of its n_mats matrices.
 *   1. degree of similarity of a location: the L2 distance between the flattened experts that
 *      two variants hold there, summed over all variant-to-variant combinations (unordered pairs;
 *      the listing's sum over ordered pairs is twice this and ranks identically);
 *   2. locations are ranked, the lowest distance first (rank 1), ties to the lower l*E + e;
 *   3. from rank 1 on, while fewer than `capacity` locations are taken, the location is given to
 *      the variants in turn: rank r goes to variant (r - 1) mod V (the section's text: with two
 *      models the odd ranks go to the first model; the listing's "count mod |M|" read with
 *      0-based lists starts one variant later).  Such a location is CONSOLIDATED: one resident
 *      expert, the owner's, used by every variant;
 *   4. any other location keeps every variant's own expert (the paper loads it on a miss; here
 *      it is a private slot of the pool).
 * The per-layer table of the forward pass follows: variant 0's locations take slots 0..E-1
 * (shared or private alike), the private slots of variants 1.. follow in (variant, expert) order.
 */
typedef struct {
    int32_t V;            /* variants, 1..8                                             */
    int32_t L;            /* layers                                                     */
    int32_t E;            /* experts per layer; L*E <= 4096                             */
    int32_t n_mats;       /* matrices of an expert block, 1..3                          */
    int64_t mat_elems[3]; /* elements of each matrix per location, multiples of 256     */
    int32_t dtype;        /* mmoe_dtype                                                 */
    int32_t capacity;     /* expert capacity C: locations to consolidate (>= 0)         */
} mmoe_loader_shape;

/* Host only, pure.  Workspace (bytes) for mmoe_expert_distance, 0 if the shape is invalid. */
size_t mmoe_loader_workspace_bytes(const mmoe_loader_shape *shape);

/*
 * Step 1.  `mats` is a HOST array of V*n_mats DEVICE pointers: mats[v*n_mats + m] is matrix m of
 * variant v for every location, [L, E, mat_elems[m]] row-major, 16-byte aligned.
 * distance [L, E] float64 (DEVICE) out.  Differences and squares are fp32, sums fp64, in a fixed
 * order (no atomics).  Reads every stored element once.  Uses `ws`.
 */
int mmoe_expert_distance(const mmoe_loader_shape *shape, const void *const *mats, double *distance,
                         void *ws, size_t ws_bytes, void *stream);

/*
 * Steps 2 to 4, all DEVICE pointers.  distance [L, E] float64 in (finite).  Out: rank [L, E] int32
 * (1-based); owner [L, E] int32 (variant of a consolidated location, -1 otherwise); M [L, V, E]
 * int32 (the layer's table for mmoe_layer_forward); S [L] int32 (slots of each layer's pool);
 * slot_src [L, V*E, 2] int32: (variant, expert) whose weights fill each slot of the layer's pool,
 * rows past S[l] are (-1, -1).
 */
int mmoe_build_expert_map(const mmoe_loader_shape *shape, const double *distance, int32_t *rank,
                          int32_t *owner, int32_t *M, int32_t *S, int32_t *slot_src, void *stream);

/*
 * The loader's last step for one layer: the consolidated pool itself ("load M[idx].expert[iL][iE] to
 * GPU", Algorithm 1).  With the variants already in device memory the load is a device copy:
 * pool[m][s] (HOST array of n_mats DEVICE pointers, each [n_slots, mat_elems[m]] in the plain
 * layout) = matrix m of the (variant, expert) that slot_src names for slot s of `layer`.
 * slot_src is the whole [L, V*E, 2] array written by mmoe_build_expert_map (DEVICE); n_slots = S[layer]
 * (the caller reads S back to size the pool).  Follow with mmoe_pack_weights.
 */
int mmoe_assemble_pool(const mmoe_loader_shape *shape, const void *const *mats, const int32_t *slot_src,
                       int32_t layer, int32_t n_slots, void *const *pool, void *stream);

/*
 * Debugging aid, SYNCHRONISES the stream: checks on the device that every vid[t] is in
 * [0,V) and every M[v][e] in [0,S).  Returns 0 if so, 1 if not, a negative status on
 * argument errors.  `ws` needs 256 bytes.
 */
int mmoe_validate_inputs(const mmoe_shape *shape, const int32_t *vid, const int32_t *M, void *ws,
                         size_t ws_bytes, void *stream);

/*
 * ---- The attention half of a served layer -------------------------------------------------------
 *
 * What runs in front of the experts for the same batch of tokens of several variants: projections that
 * the variants share, each with its own low-rank adapter beside them; rotary positions; a paged cache of
 * keys and values, as they are or in 8 bits; attention of the tokens just added over that cache.  (The
 * paper calls everything but the experts a variant's non-expert layers, section 3.2.)  The conventions
 * above hold: device pointers, the caller's stream and workspace, no allocation, no host
 * synchronisation, negative codes for what the host can check.  Strides are in elements; 0 means dense.
 * Pointers and strides are multiples of 16 bytes unless a line says otherwise.
 */

/*
 * Projection with adapters.
 *   Y[t,:] = X[t,:] W + scale[a] (X[t,:] A[a]) B[a],  a = aid[t];  without the second term where aid[t]
 *   is outside [0, n_adapters) (-1 by convention) or n_adapters is 0.
 * All products accumulate in fp32.  With bf16 storage scale[a] (X A) goes into the second product as two
 * bf16 parts that together hold 16 bits of it, and Y is rounded once.
 */
typedef struct {
    int32_t T;          /* tokens                                                        */
    int32_t d_in;       /* inputs K, multiple of 256, up to 65536                        */
    int32_t d_out;      /* outputs N, multiple of 256, up to 262144                      */
    int32_t n_adapters; /* adapters, 0..1024                                             */
    int32_t rank;       /* rank R of the adapters, 1..128 (shorter ones padded with zeros); ignored without adapters */
    int32_t dtype;      /* mmoe_dtype of X, the weights and Y                            */
    int64_t ldx, ldy;   /* elements from one token's row to the next, up to 2^20; 0: d_in, d_out */
} mmoe_project_shape;

/* Host only, pure.  Workspace (bytes) of mmoe_project, never less for fewer tokens; 0 if the shape is invalid. */
size_t mmoe_project_workspace_bytes(const mmoe_project_shape *shape);

/* Host only, pure.  Elements of the packed adapters: the rank is padded to a multiple of 32 (fp32: 16).  0 if invalid. */
size_t mmoe_project_packed_rank(const mmoe_project_shape *shape);

/*
 * One-time packing, when the weights are loaded.  W [K, N], A [n, K, R], B [n, R, N] (in x out) to Wp (K*N
 * elements), Ap (n*Rp*K), Bp (n*N*Rp), Rp = mmoe_project_packed_rank().  A packed matrix with Q outputs and K
 * inputs is the sequence [Q/16][K/c][64 lanes] of 16-byte pieces, c = 32 (bf16) or 16 (fp32): piece
 * 16 g + r holds inputs c k + (c/4) g + [0, c/4) of output 16 q + r, which is what lane 16 g + r of a
 * matrix instruction holds.  Outputs must not overlap inputs.
 */
int mmoe_pack_projection(const mmoe_project_shape *shape, const void *W, void *Wp, void *stream);
int mmoe_pack_adapters(const mmoe_project_shape *shape, const void *A, const void *B, void *Ap, void *Bp, void *stream);

/*
 * X [T, d_in] (rows ldx apart), aid [T] int32, scale [n_adapters] fp32, Y [T, d_out] (rows ldy apart) out.  aid, Ap,
 * Bp and scale may be NULL when n_adapters is 0.  Y must not overlap X.  Results do not depend on the order in which
 * workgroups run.  Uses `ws`.
 */
int mmoe_project(const mmoe_project_shape *shape, const void *X, const int32_t *aid, const void *Wp, const void *Ap,
                 const void *Bp, const float *scale, void *Y, void *ws, size_t ws_bytes, void *stream);

/*
 * Rotary positions.  Pair i of a head, i < rot/2, is (x[i], x[i + rot/2]) (MMOE_ROTARY_HALVES) or (x[2i],
 * x[2i+1]) (MMOE_ROTARY_NEIGHBOURS) and turns by the angle pos[t] f_i:
 *   y0 = m (x0 cos - x1 sin),  y1 = m (x0 sin + x1 cos);   with `transpose` the sine's sign is swapped: the
 *   transposed map, which takes a gradient of y to the gradient of x.
 * Elements from rot on are copied.  Angles are kept in units of 2^-64 turn, where whole turns overflow, and rounded to fp32 as
 * fractions of a turn: within 2^-26 turn (that rounding) and |pos| 2^-55 (f_i is a double) of pos f_i at every position.
 *
 * f_i = base^(-2i/rot), changed for contexts longer than `original`, the one trained for, by `factor`:
 *   LINEAR  f_i / factor
 *   BASE    base * factor^(rot/(rot-2)) takes the place of base
 *   RAMP    between pair numbers lo = floor(p(32)) >= 0 and hi = ceil(p(1)) <= rot - 1, p(b) = rot ln(original / (2 pi b)) / (2 ln base)
 *           (the pair that makes b turns in `original` tokens): f_i up to lo, f_i / factor from hi on, a linear
 *           mixture between; m = 0.1 ln(factor) + 1
 *   BANDS   with u = original f_i / (2 pi) turns: f_i where u >= 4, f_i / factor where u <= 1, the linear mixture in u between
 * m = 1 but for RAMP.
 */
typedef enum { MMOE_ROTARY_HALVES = 0, MMOE_ROTARY_NEIGHBOURS = 1 } mmoe_rotary_layout;
typedef enum {
    MMOE_SCALE_NONE = 0,
    MMOE_SCALE_LINEAR = 1,
    MMOE_SCALE_BASE = 2,
    MMOE_SCALE_RAMP = 3,
    MMOE_SCALE_BANDS = 4
} mmoe_rotary_scaling;

typedef struct {
    int32_t T;         /* tokens                                                  */
    int32_t heads;     /* heads of a token                                        */
    int32_t head_dim;  /* D, multiple of 16, up to 512                            */
    int32_t rot;       /* rotated elements of a head, multiple of 16, up to D     */
    int32_t layout;    /* mmoe_rotary_layout                                      */
    int32_t dtype;     /* mmoe_dtype of X and Y                                   */
    int32_t transpose; /* 0 or 1                                                  */
    float magnitude;   /* m above                                                 */
    int64_t x_token, x_head, y_token, y_head; /* strides; 0: heads*D and D        */
} mmoe_rotary_shape;

/* Host only, pure.  steps [rot/2] (HOST out): f_i / (2 pi) in units of 2^-64, to be copied to the device; *magnitude (HOST
 * out) the m above. */
int mmoe_rotary_steps(int32_t rot, double base, int32_t scaling, double factor, int32_t original, uint64_t *steps,
                      float *magnitude);

/* X, Y [T, heads, D] (Y = X with equal strides: in place; otherwise they must not overlap); pos [T] int32, of either
 * sign; steps [rot/2] (8-byte aligned).  The arithmetic is fp32; Y is rounded once. */
int mmoe_rotary(const mmoe_rotary_shape *shape, const void *X, const int32_t *pos, const uint64_t *steps, void *Y, void *stream);

/*
 * Paged cache of keys and values.  A page holds MMOE_PAGE_TOKENS tokens; place p is row p mod 64 of page p / 64.  A
 * token's head is kept as it is (MMOE_CACHE_PLAIN) or as D codes of 8 bits with one fp32 scale:
 *   amax = max |x|;  inv = top / amax (0 where amax is 0);  scale = amax * (1 / top);
 *   INT8 (top 127): code = x inv rounded to the nearest integer, ties to even;
 *   FP8  (top 448): code = x inv in e4m3 (no infinities), to nearest, ties to even.
 * A head with a value that is not finite gets a scale of NaN and codes of zero, and reads back as NaN; one whose
 * amax is under 2^-100 gets zeros.
 *
 * Layout, for what reads pages directly.  K and V of a page and head are 64*D elements each, [n_pages, kv_heads, 64*D];
 * scales [n_pages, kv_heads, 64] fp32.  A piece is 16 bytes, E elements (8 bf16, 4 fp32, 16 codes).
 *   K, row r, element d:  ((r/16 * (D/(4E)) + d/(4E)) * 64 + (d mod 4E)/E * 16 + r mod 16) * E + d mod E
 *   V, row r, element d:  with q = r/16, g = (r mod 16)/4, j = 4q + r mod 4 (0..15):
 *                         ((d/16 * (16/E) + j/E) * 64 + g * 16 + d mod 16) * E + j mod E
 * INT8 codes are stored plus 128.
 */
#define MMOE_PAGE_TOKENS 64
typedef enum { MMOE_CACHE_PLAIN = 0, MMOE_CACHE_INT8 = 1, MMOE_CACHE_FP8 = 2 } mmoe_cache_format;

typedef struct {
    int32_t n_pages;
    int32_t kv_heads; /* 1..1024                                  */
    int32_t head_dim; /* D: 64, 128 or 256                        */
    int32_t dtype;    /* mmoe_dtype of what is appended and read  */
    int32_t format;   /* mmoe_cache_format                        */
} mmoe_cache_shape;

typedef struct {      /* DEVICE pointers; the scales are NULL for PLAIN */
    void *k, *v;
    float *k_scale, *v_scale;
} mmoe_cache;

/* Host only, pure.  Bytes of k (and of v); *scale_bytes (may be NULL) those of k_scale (and of v_scale).  0 if invalid. */
size_t mmoe_cache_bytes(const mmoe_cache_shape *shape, size_t *scale_bytes);

typedef struct {
    int32_t T;                                   /* tokens to append                                */
    int64_t k_token, k_head, v_token, v_head;    /* strides of K and V; 0: kv_heads*D and D         */
} mmoe_cache_rows;

/*
 * Appends K, V [T, kv_heads, D]: token t to place places[t] (int32; tokens whose place is outside the pages are skipped;
 * places must differ).  With `rotary` (and pos, steps) the keys are rotated first; what is kept is then what
 * mmoe_rotary's output, rounded to dtype, would give (its T, heads and strides are ignored, head_dim and dtype have to match).
 */
int mmoe_cache_append(const mmoe_cache_shape *shape, const mmoe_cache_rows *rows, const void *K, const void *V,
                      const int32_t *places, const mmoe_rotary_shape *rotary, const int32_t *pos, const uint64_t *steps,
                      const mmoe_cache *cache, void *stream);

/* Reads places[r], r < R, back to K, V [R, kv_heads, D] (dense): code * scale in fp32, rounded to dtype.  A place outside the
 * pages reads as zeros. */
int mmoe_cache_read(const mmoe_cache_shape *shape, const mmoe_cache *cache, int32_t R, const int32_t *places, void *K, void *V,
                    void *stream);

/*
 * Attention of drafted tokens over the cache.  Request b has ctx[b] committed tokens and the n = starts[b+1] - starts[b]
 * tokens starts[b] .. of Q, whose keys and values are in the cache already, behind the committed ones: token i of the
 * request is position ctx[b] + i, and position j lives in row j mod 64 of page pages[b, j/64].
 * Token i sees every committed position and
 *   with `tree`:  drafted token j < n where bit j mod 64 of tree[starts[b] + i, j/64] is set: the token itself, what it
 *                 descends from, or whatever else the caller asks for, itself not included if its bit is not;
 *   without:      drafted tokens j <= i (a chunk of a prompt, or a single token).
 * Query head h reads key head h / (heads / kv_heads).
 *   out[t,h] = sum_j softmax_j(scale <Q[t,h], K[j]>) V[j];  lse[t,h] = ln sum_j exp(scale <Q[t,h], K[j]>)
 * A token that sees nothing gets zeros and an lse of -infinity.  What a token does not see does not reach it, whatever it
 * holds: rows of a page past the end, infinities, NaN.  Scores, maxima, sums and outputs are fp32.  The probabilities are
 * rounded for the second product: to bf16 over PLAIN bf16 pages; with their value's scale to fp16 over 8-bit ones, 11 bits down to 2^-30 of
 * the token's largest, whose codes fp16 holds exactly (and queries there to fp16, relative to the row's largest; with fp32 nothing is
 * rounded).  The fp32 sums have room for scores of up to 2^28 and values of up to 2^100.  8-bit formats need dtype bf16 here.
 */
typedef struct {
    mmoe_cache_shape cache;
    int32_t T;          /* rows of Q, starts[n_requests]                                          */
    int32_t n_requests;
    int32_t heads;      /* query heads, a multiple of kv_heads, up to 64 to a key head            */
    int32_t max_pages;  /* columns of `pages`; positions from 64*max_pages on are not seen        */
    int32_t max_drafts; /* no request has more tokens in Q; what goes beyond is not written       */
                        /* (MMOE_ERR_LIMIT where n_requests * heads * max_drafts needs 2^24 workgroups, 64 or 128 rows each) */
    int32_t mask_words; /* 64-bit words of a row of `tree`                                        */
    int32_t max_keys;   /* hint: the longest ctx + n; 0: 64*max_pages.  Results do not depend on the hints beyond rounding */
    int64_t sum_keys;   /* hint: the sum of ctx + n; 0: n_requests * max_keys                     */
    float scale;        /* of the scores                                                          */
    int64_t q_token, q_head, o_token, o_head; /* strides of Q and out; 0: heads*D and D           */
} mmoe_attend_shape;

/* Host only, pure.  Workspace (bytes) of mmoe_attend, never less for fewer requests, tokens, drafts or pages, whatever the hints of those calls
 * (with a sum_keys here: for calls whose own, given or n_requests * max_keys, is up to that).  0 if the shape is invalid. */
size_t mmoe_attend_workspace_bytes(const mmoe_attend_shape *shape);

/* Q [T, heads, D], starts [n_requests + 1], ctx [n_requests], tree [T, mask_words] uint64 or NULL, pages [n_requests,
 * max_pages] int32 (entries outside [0, n_pages) are not seen); out [T, heads, D] dtype, lse [T, heads] fp32 or NULL.  Rows of Q
 * that belong to no request are left as they are in `out`.  Uses `ws`. */
int mmoe_attend(const mmoe_attend_shape *shape, const void *Q, const int32_t *starts, const int32_t *ctx, const uint64_t *tree,
                const int32_t *pages, const mmoe_cache *cache, void *out, float *lse, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MMOE_H */
