/* marlaas.h -- C ABI of the B200 multi-tenant LoRA linear layer.
 *
 * The layer is the one every adapted projection of the shared base model runs when many tenants
 * share one frozen base weight through lightweight LoRA adapters (paper: abstract; Introduction;
 * Methods, "Multi-Task Manager" -- per-task LoRA parameters theta_t^(v) with a version counter --
 * and "Multi-LoRA Rollout with Single-Task Training" -- rollouts batched across tasks by multi-LoRA
 * kernels; Algorithm 1 "Commit updated parameters").  For a token i routed to tenant slot t:
 *
 *     y_i  = x_i W + s_t (x_i A_t) B_t                              (forward: rollout decode and training)
 *     dx_i = dy_i W^T + s_t (dy_i B_t^T) A_t^T                      (backward)
 *     dA_t = s_t sum_{i:t(i)=t} x_i^T (dy_i B_t^T)      dB_t = s_t sum_{i:t(i)=t} (x_i A_t)^T dy_i
 *
 * W is d_in x d_out (K x N), A_t is K x r_t, B_t is r_t x N, s_t = alpha_t / r_t; everything is
 * row-major; x, W, A, B, y, dy, dx are bf16 (1-8-7, round-to-nearest-even on output), sums are
 * carried in fp32, dA_t and dB_t are fp32.  W is frozen: there is no dW.
 *
 * Conventions
 *  - All data pointers are DEVICE pointers on the pool's device unless a comment says HOST.
 *  - All work is enqueued on `cuda_stream` (a cudaStream_t passed as void*; NULL = the legacy default
 *    stream) and the calls return without synchronising unless MARLAAS_FLAG_VALIDATE_SYNC is given.
 *    The caller keeps every buffer alive and unmodified until the stream has passed the call.
 *  - The library never allocates or frees device memory: the adapter store and the per-call workspace
 *    are caller-provided (sizes from the *_bytes functions).
 *  - Every function returns MARLAAS_OK (0) or a negative marlaas_status_t; nothing throws or aborts.
 *    marlaas_last_error() gives a thread-local message for the last failure on this thread.
 *  - Arguments are validated on the host BEFORE anything is launched; a failing call launches nothing.
 *  - A pool may be used from one host thread at a time.
 *  - Required alignment: every bf16 pointer 16-byte aligned, every leading dimension a multiple of 8
 *    elements, d_in and d_out multiples of 8.
 */
#ifndef MARLAAS_H_
#define MARLAAS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct marlaas_pool marlaas_pool_t; /* opaque; one pool per adapted projection (d_in, d_out) */
typedef int32_t marlaas_status_t;

enum {
    MARLAAS_OK = 0,
    MARLAAS_ERR_INVALID_ARG = -1,        /* null / misaligned pointer, negative size, leading dim too small */
    MARLAAS_ERR_BAD_SEGMENT_TABLE = -2,  /* offsets not 0..T non-decreasing (host tables: before launch; device
                                            tables: reported by marlaas_check_status) */
    MARLAAS_ERR_UNKNOWN_TENANT = -3,
    MARLAAS_ERR_RANK_TOO_LARGE = -4,
    MARLAAS_ERR_POOL_FULL = -5,
    MARLAAS_ERR_UNSUPPORTED_DEVICE = -6, /* not an sm_100 device, or no CUDA device */
    MARLAAS_ERR_CUDA = -7,               /* a CUDA runtime / driver call failed */
    MARLAAS_ERR_DEVICE_TIMEOUT = -8,     /* a bounded wait inside a kernel ran out; results of that call are invalid */
    MARLAAS_ERR_DEVICE_BAD_INDEX = -9,   /* a device-side check met a slot outside [-1, capacity): that token was
                                            computed with the base weight only; or, in a policy call, a target outside the
                                            vocabulary: that row was ignored */
    MARLAAS_ERR_WORKSPACE_TOO_SMALL = -10
};

enum {
    MARLAAS_FLAG_ACCUMULATE = 1u,     /* backward: dA_t, dB_t += instead of overwrite; marlaas_policy_loss: stats += */
    MARLAAS_FLAG_HOST_TABLE = 2u,     /* seg_offsets / seg_slot are HOST arrays: validated on the host, then copied
                                         into the workspace in stream order (not while the stream is being captured:
                                         refused with MARLAAS_ERR_INVALID_ARG) */
    MARLAAS_FLAG_VALIDATE_SYNC = 4u,  /* synchronise the stream after the call and return the device status word */
    MARLAAS_FLAG_CUDA_CORE_PATH = 8u, /* diagnostics: run the plain CUDA-core kernels instead of the tcgen05 path */
    MARLAAS_FLAG_REUSE_PLAN = 16u,    /* the workspace still holds the plan of the previous call of the same kind
                                         (forward after forward, backward after backward) and that call had the same T,
                                         the same segment table contents and a pool of the same capacity and max_rank:
                                         the per-token slots and per-tile unit lists are not rebuilt.  For the
                                         projections of one decoder layer, which all see the same mixed batch.  The
                                         caller vouches for the condition; batches of at most 1024 tokens ignore the
                                         flag (their plan is built inside the first kernel anyway). */
    MARLAAS_FLAG_TOKEN_MEAN = 64u,    /* marlaas_group_advantages: every active token of a tenant weighs the same */
    MARLAAS_FLAG_NO_STD = 128u,       /* marlaas_group_advantages: rewards are centred, not divided by their deviation */
    MARLAAS_FLAG_RMS_NORM = 256u,     /* marlaas_layer_norm, _backward: the mean is not subtracted (RMS norm) */
    MARLAAS_FLAG_OVERLAP_PREVIOUS = 32u /* forward, decode-shaped batches (at most 1024 tokens): the caller states that the
                                         work submitted to the stream immediately before this call -- typically the same
                                         layer's call for another micro-batch of a serving loop that interleaves two --
                                         is independent of it: it does not produce this call's x, W or segment table,
                                         and it touches neither this call's workspace, y, h_save nor its pool.  The
                                         call's first kernel (the shrink) is then launched behind that work as a
                                         programmatic dependent that does not wait for it, and runs beside the end of
                                         it; a preceding marlaas_lora_forward lets it start once its own shrink has
                                         completed, so at most two consecutive calls are in flight together (two
                                         workspaces and two pools, used in turn, satisfy the condition).  Stream order
                                         holds for everything submitted after the call: it never completes before its
                                         predecessor.  Results are bit-identical with and without the flag.  Ignored
                                         for larger batches and with MARLAAS_FLAG_HOST_TABLE; refused by
                                         marlaas_lora_forward_multi and marlaas_lora_forward_static_ws.  If the
                                         condition does not hold the call races with its predecessor. */
};

/* Token-to-adapter segment table of one mixed batch: segment s covers tokens
 * [seg_offsets[s], seg_offsets[s+1]) and routes them to pool slot seg_slot[s] (-1 = base weight only).
 * seg_offsets[0] = 0, non-decreasing, seg_offsets[S] = T; zero-length segments are allowed; a slot may
 * recur in any number of non-adjacent segments.  An unsorted decode batch is T segments of one token.
 * The arrays are device memory unless MARLAAS_FLAG_HOST_TABLE is set. */
typedef struct {
    int32_t num_segments;       /* 0 <= S <= 2^30 */
    const int32_t* seg_offsets; /* [S+1] */
    const int32_t* seg_slot;    /* [S]   */
} marlaas_segments_t;

/* ---- pooled adapter store (the manager's per-task parameters theta_t^(v), "Multi-Task Manager") ---- */

/* Bytes of device memory a pool of `capacity` slots needs (0 if the arguments are invalid).
 * max_rank in [1,128]; ranks are stored padded to a multiple of 16 with zero rows (exact). */
size_t marlaas_adapter_pool_storage_bytes(int64_t d_in, int64_t d_out, int32_t max_rank, int32_t capacity);

/* Create a pool over caller-owned device memory `storage` (256-byte aligned, >= storage_bytes, on
 * `device`); clears it in stream order.  The pool object itself is host memory freed by _destroy; the
 * storage stays the caller's.  Fails with UNSUPPORTED_DEVICE unless `device` has compute capability 10.x. */
marlaas_status_t marlaas_adapter_pool_create(marlaas_pool_t** out, int device, int64_t d_in, int64_t d_out,
                                             int32_t max_rank, int32_t capacity, void* storage,
                                             size_t storage_bytes, void* cuda_stream);
marlaas_status_t marlaas_adapter_pool_destroy(marlaas_pool_t* pool);

/* One pool for several projections that read the same activations (q, k, v; gate, up), served as ONE layer of width
 * d_out = part_d_out[0] + ... + part_d_out[n_parts-1] whose weight is the projections' weights side by side,
 * W = [W_1 | ... | W_P] (paper: Methods, "Multi-LoRA Rollout with Single-Task Training" -- every adapted projection of
 * the shared base model serves all tenants' tokens at once; Introduction -- rollout dominates the run time, so the
 * decode-shaped pass over the projections of a decoder layer is what one such call shortens).  Tenant t holds one
 * adapter pair per projection, all of the tenant's rank r_t and scale s_t:
 *
 *     y_i[:, columns of projection p] = x_i W_p + s_t (x_i A_t,p) B_t,p
 *
 * The store keeps one block of A rows per projection and the B matrices side by side ([r_t][d_out]): nothing is stored
 * or streamed for the zero blocks that the projections' adapters would have as one block-diagonal adapter of rank P r_t.
 * 1 <= n_parts <= 4; every part_d_out[p] is a positive multiple of 256.  On such a pool
 *  - register / export / adamw_commit take A as n_parts blocks [d_in][rank] one after another and B as n_parts blocks
 *    [rank][part_d_out[p]] one after another (the projections' own matrices, concatenated in memory); the fp32 masters,
 *    moments and gradients of adamw_commit and the dA_t / dB_t of backward have the same block layout;
 *  - forward / backward take W with d_out columns (the projections' weights side by side, leading dimension ldw),
 *    y / dy with d_out columns, and dx sums over the projections;
 *  - h_save / h_saved are [n_parts][T][rank_stride] (one plane per projection);
 *  - marlaas_lora_forward_static_ws and MARLAAS_FLAG_REUSE_PLAN work as on any pool.
 * With n_parts = 1 the pool is an ordinary one (but for the multiple-of-256 rule). */
size_t marlaas_adapter_pool_storage_bytes_segmented(int64_t d_in, int32_t n_parts, const int64_t* part_d_out,
                                                    int32_t max_rank, int32_t capacity);
marlaas_status_t marlaas_adapter_pool_create_segmented(marlaas_pool_t** out, int device, int64_t d_in, int32_t n_parts,
                                                       const int64_t* part_d_out /* HOST */, int32_t max_rank,
                                                       int32_t capacity, void* storage, size_t storage_bytes,
                                                       void* cuda_stream);
/* Number of projections the pool holds (1 for a pool made by marlaas_adapter_pool_create). */
int32_t marlaas_adapter_pool_parts(const marlaas_pool_t* pool);

/* Commit adapter version `version` of tenant `tenant_id` into the pool ("Commit updated parameters to M",
 * Algorithm 1; Asynchronous Execution, training step).  A: bf16 [d_in][rank], B: bf16 [rank][d_out],
 * both row-major device memory, copied and re-laid-out in stream order (the caller may reuse them once the
 * stream has passed the call).  The layer uses s = alpha / rank formed in fp32.  A tenant that is already
 * registered keeps its slot and is overwritten in stream order; a new tenant takes the lowest free slot.
 * rank = 0 (A, B may be NULL) makes the slot behave as "no adapter".  *slot_out (HOST) receives the slot. */
marlaas_status_t marlaas_adapter_pool_register(marlaas_pool_t* pool, uint64_t tenant_id, uint64_t version,
                                               int32_t rank, float alpha, const void* A, const void* B,
                                               int32_t* slot_out, void* cuda_stream);
/* Free the tenant's slot (its rank becomes 0 in stream order). */
marlaas_status_t marlaas_adapter_pool_unregister(marlaas_pool_t* pool, uint64_t tenant_id, void* cuda_stream);
/* Host-side lookup: slot / rank / scale / version of a tenant (any out pointer may be NULL). */
marlaas_status_t marlaas_adapter_pool_lookup(const marlaas_pool_t* pool, uint64_t tenant_id, int32_t* slot_out,
                                             int32_t* rank_out, float* scale_out, uint64_t* version_out);
/* Copy a slot's adapter back out in the caller's layout (A_out bf16 [d_in][rank], B_out bf16 [rank][d_out],
 * device memory; either may be NULL).  Used to check the store's re-layout bit for bit. */
marlaas_status_t marlaas_adapter_pool_export(marlaas_pool_t* pool, int32_t slot, void* A_out, void* B_out,
                                             void* cuda_stream);
/* Policy update and commit of the updated parameters for n tenants in one launch (Algorithm 1: "PolicyUpdate",
 * then the commit of the new adapter version; Methods, Multi-Task Manager: per-task optimizer state and version
 * counter).  The paper names no optimizer; this is AdamW with decoupled weight decay, in fp32:
 *     g = grad_scale * grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *     theta = theta - lr * ( (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps) + weight_decay * theta )
 * applied to the fp32 master copies A [d_in][rank] and B [rank][d_out] of every listed tenant (moments m*, v* of the
 * same shapes, all updated in place), after which the bf16 rounding (round to nearest even) of the new masters
 * replaces the tenant's rows of the pooled store, as marlaas_adapter_pool_register would write them, and the
 * tenant's version becomes new_versions[i] (or its old version + 1 when new_versions is NULL).
 * tenant_ids / new_versions and the eight pointer tables are HOST arrays of n entries; the pointers in the tables are
 * device memory (4-byte aligned, caller-owned, gradients as marlaas_lora_backward wrote them: true rank, dense).
 * Stream-ordered like register.  Errors, before anything is launched: unknown tenant (MARLAAS_ERR_UNKNOWN_TENANT),
 * a tenant of rank 0 or listed twice, a NULL pointer, step < 1 (MARLAAS_ERR_INVALID_ARG). */
typedef struct marlaas_adamw {
    float lr, beta1, beta2, eps, weight_decay, grad_scale;
    int64_t step; /* >= 1: the step being taken */
} marlaas_adamw_t;
marlaas_status_t marlaas_adapter_pool_adamw_commit(marlaas_pool_t* pool, int32_t n, const uint64_t* tenant_ids,
                                                   const uint64_t* new_versions, const float* const* dA,
                                                   const float* const* dB, float* const* A, float* const* B,
                                                   float* const* m_A, float* const* v_A, float* const* m_B,
                                                   float* const* v_B, const marlaas_adamw_t* hp, void* cuda_stream);
/* Row stride (in floats) of the h_save / h_saved arrays: max_rank rounded up to a multiple of 16. */
int32_t marlaas_adapter_pool_rank_stride(const marlaas_pool_t* pool);

/* ---- the layer ---- */

/* Bytes of workspace forward/backward need for a batch of T tokens on this pool (device memory, 256-byte
 * aligned, contents need not be preserved between calls; two calls in flight need two workspaces).  The size does not
 * grow monotonically with T: the decode-shaped kernels chosen for small batches over large weights may use more exchange
 * scratch than those chosen for larger batches, so a workspace shared by calls of several batch sizes takes the largest
 * of their sizes (a call given less than its own full size still runs, see marlaas_lora_forward_workspace_min_bytes). */
size_t marlaas_lora_workspace_bytes(const marlaas_pool_t* pool, int64_t T);
/* The part of that workspace a forward call uses (its leading bytes): enough for marlaas_lora_forward alone. */
size_t marlaas_lora_forward_workspace_bytes(const marlaas_pool_t* pool, int64_t T);
/* The least a forward call accepts (also leading bytes).  The difference to the size above is scratch through which the
 * decode-shaped kernels for large weights pass partial sums between CTA pairs (up to about 20 MB); a call given less than
 * the full size runs the kernels that need no such scratch (slower on those shapes; every result still within the
 * layer's tolerance of the definition). */
size_t marlaas_lora_forward_workspace_min_bytes(const marlaas_pool_t* pool, int64_t T);

/* Forward: y[T][d_out] = x[T][d_in] W + s_t (x A_t) B_t with t from the segment table.
 * x (ldx >= d_in), W (ldw >= d_out), y (ldy >= d_out): bf16 row-major.  h_save: optional fp32
 * [T][rank_stride] that receives h_i = x_i A_t (zero beyond r_t) for reuse by backward; NULL = not kept.
 * T = 0 is a no-op. */
marlaas_status_t marlaas_lora_forward(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx,
                                      const void* W, int64_t ldw, void* y, int64_t ldy,
                                      const marlaas_segments_t* seg, float* h_save, void* workspace,
                                      size_t workspace_bytes, uint32_t flags, void* cuda_stream);

/* Several forward calls that do not depend on one another, as one call: the projections of a decoder layer that read
 * the same activations (q, k, v; gate, up) during rollout, when every adapted projection of the shared base model serves
 * all tenants' decode tokens at once (paper: Methods, "Multi-LoRA Rollout with Single-Task Training"; Introduction:
 * rollouts dominate the run time).  Each entry holds the arguments of one marlaas_lora_forward.  The caller states that
 * no call's output is another's input and that pools, outputs, h_save arrays and workspaces are pairwise distinct; the
 * library may then run the calls side by side (on streams it owns, forked from cuda_stream and joined to it before the
 * call returns; events only, so legal inside a stream capture), which lets one projection's epilogue overlap the next
 * one's pass over its weight.  Everything the call writes is ordered on cuda_stream as if issued there.  All entries are
 * validated before anything is launched.  MARLAAS_FLAG_VALIDATE_SYNC and MARLAAS_FLAG_REUSE_PLAN are refused. */
typedef struct {
    marlaas_pool_t* pool;
    int64_t T;
    const void* x; int64_t ldx;
    const void* W; int64_t ldw;
    void* y; int64_t ldy;
    const marlaas_segments_t* seg;
    float* h_save;
    void* workspace; size_t workspace_bytes;
} marlaas_forward_call_t;
marlaas_status_t marlaas_lora_forward_multi(int32_t n, const marlaas_forward_call_t* calls, uint32_t flags, void* cuda_stream);

/* The same forward pass for callers that cannot allocate device memory (no counterpart in the paper: an
 * addition for deployments, not part of the method).  Some hosts of this layer may not call cudaMalloc at all:
 * a serving loop whose memory pool was sized and frozen at start-up, a plug-in that is handed nothing but its
 * input and output buffers, a latency-critical path that cannot afford the device-wide synchronisation an
 * allocation implies or its failure under a full memory budget.  For them the per-call scratch comes from an
 * array built into the library (marlaas_lora_static_workspace_limit() bytes, 8 MiB, resident on every GPU that
 * loads the library until the process exits) instead of a caller workspace; x, W, y, the pool storage and h_save
 * are still the caller's.  The call itself allocates and frees nothing on the device.
 *  - Batches whose forward scratch (marlaas_lora_forward_workspace_min_bytes) exceeds the limit are rejected with
 *    MARLAAS_ERR_WORKSPACE_TOO_SMALL before anything is launched: 256 tokens on a pool of 32 slots of rank
 *    up to 64 fit.
 *  - The first call on each device looks up the array's device address.  That lookup is also the moment the CUDA
 *    runtime loads this part of the library onto the device and the device's copy of the array comes into being
 *    (8 MiB of device memory, taken once, which can fail if the device is full): make that first call at start-up,
 *    while memory may still be taken, and before starting any stream capture on that device.  Later calls on the
 *    device leave its free memory unchanged.
 *  - All calls on a device share the one array and it keeps the previous call's contents (nothing in it has to
 *    start at zero: each call writes what it later reads).  Two calls whose kernels overlap on the GPU -- different
 *    streams, or different pools on different streams -- race on it; keep such calls on one stream. */
size_t marlaas_lora_static_workspace_limit(void);
marlaas_status_t marlaas_lora_forward_static_ws(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx,
                                                const void* W, int64_t ldw, void* y, int64_t ldy,
                                                const marlaas_segments_t* seg, float* h_save, uint32_t flags,
                                                void* cuda_stream);

/* Backward for the policy-training stage: dx[T][d_in] bf16 (NULL = skip) and per-slot fp32 adapter gradients.
 * dA_slots / dB_slots: HOST arrays of `capacity` device pointers (either table, or any entry, may be NULL =
 * skip); dA_t is [d_in][r_t], dB_t is [r_t][d_out], row-major, at the slot's true rank.  Without
 * MARLAAS_FLAG_ACCUMULATE every non-NULL slot is overwritten (tenants with no token in the batch get exact
 * zeros); with it the batch's contribution is added.  The sums over a tenant's tokens run over all of its
 * segments.  h_saved: what forward wrote to h_save for the same batch and adapters, or NULL = recompute.
 * A row of x or dy with infinities or NaN may reach dA_t and dB_t of the other tenants that share a block of 64 tokens
 * with it (the call with dropout below keeps them apart).  All work is issued on cuda_stream.  Inside a
 * stream capture, pools of more than 64 slots copy dA_slots / dB_slots with a memcpy node that keeps the HOST pointers:
 * the caller's tables must then stay alive and unchanged for every replay.  Calls on one pool are not to be issued from
 * several host threads at once. */
marlaas_status_t marlaas_lora_backward(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx,
                                       const void* W, int64_t ldw, const void* dy, int64_t lddy,
                                       void* dx, int64_t lddx, float* const* dA_slots, float* const* dB_slots,
                                       const marlaas_segments_t* seg, const float* h_saved, void* workspace,
                                       size_t workspace_bytes, uint32_t flags, void* cuda_stream);

/* The indexing contract, bit-exact: tok_slot[T] (slot of the segment containing each token),
 * slot_count[capacity+1] (tokens per slot; the last entry counts slot -1), slot_offset[capacity+2]
 * (exclusive prefix sum in the order 0..capacity-1, then -1; last entry = T) and perm[T] (token indices
 * stably sorted by that key).  All four are device int32 arrays; any may be NULL. */
marlaas_status_t marlaas_lora_build_index(marlaas_pool_t* pool, int64_t T, const marlaas_segments_t* seg,
                                          int32_t* tok_slot, int32_t* slot_count, int32_t* slot_offset,
                                          int32_t* perm, void* workspace, size_t workspace_bytes,
                                          uint32_t flags, void* cuda_stream);

/* ---- the policy update around the layer (Algorithm 1, training branch; Experimental setup: GRPO) ----
 * rewards -> advantages and token weights -> clipped loss with KL term, whose gradient by the logits is the dy of the
 * output projection's marlaas_lora_backward -> AdamW with 8-bit moments committed into the pool.  The sequences of a
 * batch are the segments of its segment table; `pool` supplies the device, the slots and the status word. */

enum { MARLAAS_DTYPE_BF16 = 0, MARLAAS_DTYPE_F32 = 1 };    /* element type of logits and of their gradient */
enum { MARLAAS_MAX_VOCABULARY = 262144 };
enum { MARLAAS_POLICY_STATS = 8 };                         /* columns of marlaas_policy_loss's stats */

/* Bytes of workspace that marlaas_group_advantages and marlaas_policy_loss need for a batch of T tokens in num_segments
 * segments and num_groups groups (0 for the loss); 256-byte aligned, contents need not be preserved. */
size_t marlaas_policy_workspace_bytes(const marlaas_pool_t* pool, int64_t T, int32_t num_segments, int32_t num_groups);

/* Group-relative advantages and token weights.  Segment i of `seg` is sequence i with reward r_i; group g is the
 * sequences [group_offsets[g], group_offsets[g+1]) (the answers to one prompt).  With d_i = r_i - r_first(g), mean and
 * population variance over the group,
 *     a_i = (d_i - mean d) / (sqrt(var d) + eps)          (MARLAAS_FLAG_NO_STD: a_i = d_i - mean d)
 * A group whose rewards are all alike has advantages of exactly 0.  A token is active if its target is >= 0:
 *     adv = a_i,  weight = 1 / (N_t len_i)                (MARLAAS_FLAG_TOKEN_MEAN: weight = 1 / M_t)
 * with len_i the active tokens of its sequence, N_t the sequences of its tenant (slot) that have any, M_t the active
 * tokens of its tenant; slot -1 counts as one more tenant.  Inactive tokens get 0 and 0.  The weights of a tenant with an
 * active token sum to 1.  rewards fp32 [S], group_offsets int32 [G+1] (0 .. S, non-decreasing; on the device, or on the
 * HOST with MARLAAS_FLAG_HOST_TABLE like the segment table), targets int32 [T]; outputs fp32 seq_adv [S], adv [T],
 * weight [T], each may be NULL.  A device table that is not as described is reported by marlaas_check_status
 * (MARLAAS_ERR_BAD_SEGMENT_TABLE, MARLAAS_ERR_DEVICE_BAD_INDEX); the outputs are then unspecified. */
marlaas_status_t marlaas_group_advantages(marlaas_pool_t* pool, int64_t T, const marlaas_segments_t* seg,
                                          const float* rewards, int32_t num_groups, const int32_t* group_offsets,
                                          const int32_t* targets, float eps, float* seq_adv, float* adv, float* weight,
                                          void* workspace, size_t workspace_bytes, uint32_t flags, void* cuda_stream);

/* Log-probabilities of the target tokens under softmax(logits * inv_temperature), and the entropy of that distribution:
 * the behaviour policy's values at rollout, the reference policy's in training.  logits [T][V] of `dtype`, leading
 * dimension ld, rows on 16-byte boundaries (ld a multiple of 8 for bf16, of 4 for fp32; V is any number from 1 to
 * MARLAAS_MAX_VOCABULARY).  targets int32 [T]; logp fp32 [T]; entropy fp32 [T] or NULL.
 *  - A row with a negative target is ignored: it is not read, logp and entropy are 0.
 *  - Logits of -inf have probability 0.  A row whose logits are all -inf has no distribution: logp and entropy are 0.
 *  - A row with a NaN or +inf gets NaN.
 *  - A target >= V is reported by marlaas_check_status (MARLAAS_ERR_DEVICE_BAD_INDEX) and its row is ignored.
 *  - Sums run in an order that depends on T, V and dtype alone: on the same logits this call and marlaas_policy_loss give
 *    the same bits, so that the ratios of an update's first pass are exactly 1. */
marlaas_status_t marlaas_token_logprobs(marlaas_pool_t* pool, int64_t T, int64_t V, const void* logits, int64_t ld,
                                        int32_t dtype, const int32_t* targets, float inv_temperature, float* logp,
                                        float* entropy, uint32_t flags, void* cuda_stream);

/* The clipped policy loss with KL and entropy terms, and its gradient by the logits, in one pass over them.  With logp
 * and the entropy H of token i as above, A = adv[i], w = weight[i]:
 *     ratio = exp(logp - old_logp[i])      pg = -min(ratio A, clamp(ratio, 1 - clip_low, 1 + clip_high) A)
 *     d = ref_logp[i] - logp               kl = exp(d) - d - 1
 *     loss = sum_i w (pg + kl_coef kl - entropy_coef H)
 *     dlogits[i] = grad_scale * d loss / d logits[i]
 * where a clipped token's pg has no gradient.  dlogits: [T][V] of `dtype` with leading dimension lddl, rows on 16-byte
 * boundaries; NULL = not wanted; dlogits == logits with lddl == ld overwrites the logits, any other overlap is refused.
 * Columns from V to the leading dimension are left alone.  logp: fp32 [T] or NULL.
 * Rows that marlaas_token_logprobs ignores, and tokens of weight 0 whatever their other values, contribute nothing: their
 * gradient is 0.  ref_logp may be NULL if kl_coef is 0.
 * stats: fp32 [capacity + 1][MARLAAS_POLICY_STATS], per slot (last row: slot -1) the sums over its tokens of
 *     w (pg + kl_coef kl - entropy_coef H), w pg, w kl, w H, w ratio, w [clipped], w, 1
 * (with weights that sum to 1, the first six are the tenant's means; w kl is 0 without ref_logp, and filled with it also if
 * kl_coef is 0); written, or added to with MARLAAS_FLAG_ACCUMULATE, in a fixed order of the sums.  A token of an ill-formed
 * device table counts as slot -1 and is reported. */
typedef struct marlaas_policy_loss {
    float clip_low, clip_high, kl_coef, entropy_coef, inv_temperature, grad_scale;
} marlaas_policy_loss_t;
marlaas_status_t marlaas_policy_loss(marlaas_pool_t* pool, int64_t T, int64_t V, const void* logits, int64_t ld,
                                     int32_t dtype, const int32_t* targets, const marlaas_segments_t* seg,
                                     const float* old_logp, const float* ref_logp, const float* adv, const float* weight,
                                     const marlaas_policy_loss_t* hp, void* dlogits, int64_t lddl, float* logp,
                                     float* stats, void* workspace, size_t workspace_bytes, uint32_t flags,
                                     void* cuda_stream);

/* AdamW and commit as marlaas_adapter_pool_adamw_commit, with both moments held in 8 bits: 2.06 bytes per element
 * instead of 8, and 18 bytes moved per element instead of 30.  The moments of a matrix of n elements are
 * marlaas_adamw_compact_state_bytes(n) bytes: for every 256 consecutive elements a block of 528 bytes, 16-byte aligned:
 *     [0, 256) codes of m   [256, 512) codes of v   [512] exponent E_m   [513] E_v   [514, 528) unused
 * A code's low bits are the leading bits of an fp32 number (exponent and 3 mantissa bits) counted from the smallest
 * exponent the block can hold: m is a sign bit and 7 bits (15 binary orders below E_m), v is 8 bits (31 orders below E_v;
 * v is the square of what m averages, so both keep the same range of gradients).  Code 0 is 0.  All-zero bytes are zero
 * moments.  The update is done in fp32 on the decoded moments; the new moments are rounded stochastically with 16 random
 * bits each, so that their expected value is kept (at beta2 = 0.999 a moment moves by a thousandth per step, a hundredth of
 * what rounding to nearest would need to move it at all): a moment below the block's range becomes 0, except that a
 * positive v stays at the smallest code.  A moment that is not finite is stored as 0.  If the gradient itself was not finite,
 * the master then holds a NaN or an infinity.  If only its square left fp32's range (from about 6e20 at beta2 = 0.999), the
 * step leaves the master as it is but for the weight decay, and the next one starts both moments of the element anew from 0:
 * a step reads the m of an element whose v is 0 as 0 in blocks with E_m >= 127, where nothing else leaves the two like that
 * (the export gives the codes' values as they are).  The random bits depend on seed, hp->step, the tenant id, the matrix and
 * the element's index alone: the same call gives the same bits.
 * state_A[i] / state_B[i]: the tenant's state for A [d_in][rank] and B [rank][d_out]; on a pool over several projections,
 * the projections' states one after another, each of marlaas_adamw_compact_state_bytes of its own elements.
 * ranks: HOST [n], the ranks that the buffers were made for, or NULL; a tenant whose adapter has another rank by now is
 * refused (MARLAAS_ERR_INVALID_ARG).
 * Everything else, the errors included, as marlaas_adapter_pool_adamw_commit. */
size_t marlaas_adamw_compact_state_bytes(int64_t n);
marlaas_status_t marlaas_adapter_pool_adamw_compact_commit(marlaas_pool_t* pool, int32_t n, const uint64_t* tenant_ids,
                                                           const uint64_t* new_versions, const float* const* dA,
                                                           const float* const* dB, float* const* A, float* const* B,
                                                           void* const* state_A, void* const* state_B,
                                                           const int32_t* ranks, const marlaas_adamw_t* hp,
                                                           uint64_t seed, void* cuda_stream);
/* The values that `blocks` consecutive blocks of such a state stand for: fp32 m and v of 256 * blocks elements, 16-byte
 * aligned (for inspection, or to go on with marlaas_adapter_pool_adamw_commit); either may be NULL. */
marlaas_status_t marlaas_adamw_compact_state_export(marlaas_pool_t* pool, int64_t blocks, const void* state, float* m,
                                                    float* v, void* cuda_stream);
/* Device addresses of the pool's bf16 rows inside its storage: At [parts][capacity * rank_stride][d_in] (row
 * slot * rank_stride + j of block p is column j of A_t,p), Bs [capacity * rank_stride][d_out].  Read-only for the caller. */
marlaas_status_t marlaas_adapter_pool_store(const marlaas_pool_t* pool, const void** At, const void** Bs);

/* ---- around the adapted projections of a training step ---- */

enum { MARLAAS_MAX_NORM_WIDTH = 16384, MARLAAS_MAX_HEAD_WIDTH = 65536 };
enum { MARLAAS_HEAD_STATS = 4 };                           /* columns of marlaas_head_cross_entropy's stats */

/* The layer with dropout in its adapters, for training.  With m_i the mask of token i (a truth value per element of x_i),
 * t its slot, p_t the tenant's rate and s'_t = s_t / (1 - p_t):
 *     y_i  = x_i W + s'_t ((m_i o x_i) A_t) B_t
 *     dx_i = dy_i W^T + s'_t m_i o ((dy_i B_t^T) A_t^T)
 *     dA_t = s'_t sum (m_i o x_i)^T (dy_i B_t^T)           dB_t = s'_t sum ((m_i o x_i) A_t)^T dy_i
 * Masks are never stored: every pass computes them from the generator.  Philox-4x32 of seven rounds (Salmon, Moraes, Dror and
 * Shaw, 2011) with the key (low, high word of seed) and the counter (c, i, low, high word of offset) gives four words, whose
 * low and high halves in turn are the 16-bit numbers of the elements 8 c to 8 c + 7 of token i; an element is dropped if its
 * number is below round(65536 p_t), and p_t in the formulas is that number over 65536.  The backward pass takes the seed, the
 * offset and the rates of its forward pass; another step or another projection takes another offset.  A pool over several
 * projections drops the same elements for all of them.
 * rates: fp32 [capacity] on the device, per slot; a rate that is not above 0 (or a NaN) drops nothing, one of 1 or more drops
 * everything (the adapter then gives nothing and gets zero gradients).  What a dropped element holds does not matter to the
 * adapters, and what the rows of a tenant's tokens hold (infinities and NaN too) reaches no other tenant's rows and gradients.
 * With rates of 0 the results are marlaas_lora_forward's and marlaas_lora_backward's up to the order of sums; as there, s'_t h and
 * s'_t g are rounded to bf16 on their way into the second products, and from 512 tokens on h and g are the tensor cores' fp32 sums
 * (2e-6 relative) and enter dA and dB as the sum of two bf16 numbers each (2^-16 relative).
 * Meant for supervised tuning.  A policy that answers without dropout is another function than the one that trains with it: its
 * ratios are then not 1 in the first pass over a batch, and marlaas_head_cross_entropy's dx is not its policy gradient.
 * Otherwise as those two calls, with h_save = (m_i o x_i) A_t; of the flags, HOST_TABLE, VALIDATE_SYNC and (backward)
 * ACCUMULATE apply.  Workspace: marlaas_lora_dropout_workspace_bytes, for both; it has room for a copy of x beside the layer's
 * own, for batches whose tenants mix finely and for rows of more than 96 K elements.  Adapter gradients of pools of more than 64
 * slots cannot be captured. */
typedef struct marlaas_dropout {
    const float* rates;
    uint64_t seed, offset;
} marlaas_dropout_t;
size_t marlaas_lora_dropout_workspace_bytes(const marlaas_pool_t* pool, int64_t T);
marlaas_status_t marlaas_lora_forward_dropout(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx, const void* W, int64_t ldw, void* y,
                                              int64_t ldy, const marlaas_segments_t* seg, const marlaas_dropout_t* drop, float* h_save,
                                              void* workspace, size_t workspace_bytes, uint32_t flags, void* cuda_stream);
marlaas_status_t marlaas_lora_backward_dropout(marlaas_pool_t* pool, int64_t T, const void* x, int64_t ldx, const void* W, int64_t ldw,
                                               const void* dy, int64_t lddy, void* dx, int64_t lddx, float* const* dA_slots,
                                               float* const* dB_slots, const marlaas_segments_t* seg, const marlaas_dropout_t* drop,
                                               const float* h_saved, void* workspace, size_t workspace_bytes, uint32_t flags,
                                               void* cuda_stream);

/* Layer norm whose gain and bias are each tenant's own, over rows of d elements (d a multiple of 8 up to
 * MARLAAS_MAX_NORM_WIDTH; x and y are bf16 with leading dimensions ldx, ldy).  With t the slot of token i,
 *     y_i = (x_i - mean_i) rstd_i gain_t + bias_t,     rstd_i = 1 / sqrt(var_i + eps)
 * var the population variance; with MARLAAS_FLAG_RMS_NORM mean_i = 0.  gain and bias (NULL = none) are fp32
 * [capacity + 1][d], 16-byte aligned; row `capacity` serves slot -1, and the tokens that an ill-formed device table leaves out
 * (reported by marlaas_check_status).  mean and rstd: fp32 [T] for the backward pass, each may be NULL.  y may be x itself.
 * A row of infinities or NaN gives NaN and touches no other row; sums of a row's elements and of their squared deviations are fp32,
 * so that rows of elements beyond about 1e17 leave its range.  `pool` supplies the device, the slots and the status word.
 * The workspace is used with MARLAAS_FLAG_HOST_TABLE alone (marlaas_layer_norm_workspace_bytes with backward = 0). */
size_t marlaas_layer_norm_workspace_bytes(const marlaas_pool_t* pool, int64_t T, int64_t d, int32_t num_segments, int32_t backward);
marlaas_status_t marlaas_layer_norm(marlaas_pool_t* pool, int64_t T, int64_t d, const void* x, int64_t ldx,
                                    const marlaas_segments_t* seg, const float* gain, const float* bias, float eps, void* y,
                                    int64_t ldy, float* mean, float* rstd, void* workspace, size_t workspace_bytes,
                                    uint32_t flags, void* cuda_stream);
/* Its gradients: dx bf16 [T][d] (NULL = skip; may be dy or x itself), dgain and dbias fp32 [capacity + 1][d], 16-byte aligned
 * (each may be NULL), the sums over each tenant's tokens: exact zeros for a tenant without tokens, added to with
 * MARLAAS_FLAG_ACCUMULATE, in an order that depends on the sizes and the segment table alone.  mean (not read with
 * MARLAAS_FLAG_RMS_NORM) and rstd as the forward pass wrote them. */
marlaas_status_t marlaas_layer_norm_backward(marlaas_pool_t* pool, int64_t T, int64_t d, const void* x, int64_t ldx, const void* dy,
                                             int64_t lddy, const marlaas_segments_t* seg, const float* gain, const float* mean,
                                             const float* rstd, void* dx, int64_t lddx, float* dgain, float* dbias, void* workspace,
                                             size_t workspace_bytes, uint32_t flags, void* cuda_stream);

/* Cross entropy of the vocabulary head from the last hidden states, and its gradient by them, without the logits: what
 * marlaas_token_logprobs gives for logits = x W, and weighted sums of it, with x [T][d] and the frozen W [d][V] bf16 (ldx, ldw
 * multiples of 8; d a multiple of 8 up to MARLAAS_MAX_HEAD_WIDTH, V any number from 1 to MARLAAS_MAX_VOCABULARY).  With
 * z_i = inv_temperature x_i W in fp32, y_i = targets[i], w_i = weight[i] (NULL: 1):
 *     logp_i = z_i[y_i] - log sum exp z_i          loss = sum_i w_i (-logp_i)
 *     dx_i = grad_scale d loss / d x_i = grad_scale inv_temperature w_i (softmax(z_i) - e_y) W^T
 * Weights may have either sign: with w_i = weight_i adv_i of marlaas_group_advantages, dx is the gradient of
 * marlaas_policy_loss where all ratios are 1 (the first pass over a batch, without KL and entropy terms).
 *  - A token with a negative target or a weight of 0 is ignored whatever its row holds: logp 0, dx 0, nothing in the sums,
 *    and its part of the products is not computed.
 *  - A target >= V is reported by marlaas_check_status (MARLAAS_ERR_DEVICE_BAD_INDEX) and its token is ignored.
 *  - A row with a NaN or +inf logit gets NaN, and touches no other row; a logit of -inf has probability 0; a row whose logits
 *    are all -inf has no distribution: logp and dx are 0.
 * dx: bf16 [T][d] or NULL (no gradient: half the work and a smaller workspace); it may be x itself.  logp: fp32 [T] or NULL.
 * No output may overlap an input otherwise.
 * stats (or NULL; then seg is not read): fp32 [capacity + 1][MARLAAS_HEAD_STATS], per slot (last row: slot -1) the sums over its
 * tokens of  w (-logp), w, -logp, 1;  written, or added to with MARLAAS_FLAG_ACCUMULATE, in a fixed order.
 * The exponentials in the workspace are those of a piece of the batch (512 MB, or 256 rows where those are more); beside them it holds
 * the counted rows of the whole batch (2 T d bytes), and with a gradient up to 192 MB of partial sums.  Logits and the exponentials'
 * sums carry the tensor cores' fp32 sums and the hardware's exponential (about 2e-6 of a log-probability).  The probabilities
 * in the gradient's product are bf16, rounded twice on their way there (2^-8 relative each time); all sums are fp32. */
size_t marlaas_head_cross_entropy_workspace_bytes(const marlaas_pool_t* pool, int64_t T, int64_t d, int64_t V, int32_t num_segments,
                                                  int32_t with_gradient);
marlaas_status_t marlaas_head_cross_entropy(marlaas_pool_t* pool, int64_t T, int64_t d, int64_t V, const void* x, int64_t ldx,
                                            const void* W, int64_t ldw, const int32_t* targets, const marlaas_segments_t* seg,
                                            const float* weight, float inv_temperature, float grad_scale, void* dx, int64_t lddx,
                                            float* logp, float* stats, void* workspace, size_t workspace_bytes, uint32_t flags,
                                            void* cuda_stream);

/* Synchronise `cuda_stream`, read and clear the pool's device status word: MARLAAS_OK, or the first
 * device-side finding since the last check (BAD_SEGMENT_TABLE, DEVICE_BAD_INDEX, DEVICE_TIMEOUT). */
marlaas_status_t marlaas_check_status(marlaas_pool_t* pool, void* cuda_stream);

/* Diagnostic (no counterpart in the paper): every wait inside the tensor-core kernels is bounded, and a wait that runs
 * out makes its kernel drain and return with MARLAAS_ERR_DEVICE_TIMEOUT recorded in the pool's status word.  This call
 * exercises exactly that path without starving a real kernel: one small CTA waits, with the kernels' own wait routine,
 * on a barrier that nobody arrives on, gives up after limit_ns (at most 100 ms) and returns normally.  The next
 * marlaas_check_status on the pool then returns MARLAAS_ERR_DEVICE_TIMEOUT (and clears it); the pool stays usable. */
marlaas_status_t marlaas_debug_wait_runs_out(marlaas_pool_t* pool, uint64_t limit_ns, void* cuda_stream);

/* Message for the last non-OK status returned on the calling thread ("" if none). */
const char* marlaas_last_error(void);

/* Measurement aid (no counterpart in the paper): between _begin and _end the library brackets every launch of
 * the layer's dominant kernel (the base GEMM with the fused low-rank term, forward and dx) with CUDA events on
 * the launching stream.  _end synchronises those events and returns the summed device time in milliseconds
 * and the number of bracketed launches (either out pointer may be NULL). */
marlaas_status_t marlaas_kernel_timing_begin(marlaas_pool_t* pool);
marlaas_status_t marlaas_kernel_timing_end(marlaas_pool_t* pool, float* gemm_ms, int32_t* gemm_launches);

/* Number of kernels the library has launched in this process (all pools, all threads). */
uint64_t marlaas_kernel_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* MARLAAS_H_ */
