/*
 * psrl.h - C ABI of the tree-causal prefix-shared attention library (libpsrl.so).
 *
 * The library implements the attention step of training-time prefix sharing:
 * samples of a step-wise or tree-structured RL batch share decision prefixes;
 * every shared token span ("segment") is stored once, its K/V in a paged KV
 * store, and each token attends to all tokens of its ancestor segments plus
 * the causal part of its own segment, which reproduces per-sequence causal
 * attention exactly (paper Sec. 2.5, "Prefix sharing in training").  Backward
 * accumulates the adjoints of every consumer on the shared K/V (paper Sec. 6,
 * "Prefix-sharing training runtime") in a fixed order, so results are bitwise
 * reproducible run to run.
 *
 * Conventions
 *  - Every call returns a psrl_status_t; nothing throws, aborts or prints.
 *  - "host" / "device" is stated for every pointer.  The library never
 *    allocates device memory in the entry points below: tensors, pools, the
 *    plan's device mirror and the workspace are the caller's.
 *  - Kernels are launched on the caller's stream; no entry point synchronises
 *    except psrl_device_status().
 *  - Only sm_100a devices are supported; there is no CPU or other fallback.
 */
#ifndef PSRL_H_
#define PSRL_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PSRL_OK = 0,
  PSRL_ERR_INVALID_ARG = 1,    /* null / misaligned pointer, bad count, bad flag bits */
  PSRL_ERR_BAD_TREE = 2,       /* parent >= own index, length < 1, leaf that ends no sample */
  PSRL_ERR_BAD_BLOCK_SIZE = 3, /* block size not a power of two in [16, 256], or 0 =
                                      adaptive (Sec. 5.1): one extent per segment sized to its span at 16-slot
                                      granularity (bf16 path only) */
  PSRL_ERR_SHAPE = 4,          /* head counts do not divide, pool smaller than the plan needs */
  PSRL_ERR_UNSUPPORTED = 5,    /* dtype x head_dim outside {f32 x {64,128}, bf16 x 128} */
  PSRL_ERR_POOL_FULL = 6,      /* no free extent fits a page */
  PSRL_ERR_WORKSPACE = 7,      /* workspace / device buffer too small, or plan not uploaded */
  PSRL_ERR_HOST_OOM = 8,
  PSRL_ERR_CUDA = 9,           /* a CUDA runtime / driver call failed */
  PSRL_ERR_TIMEOUT = 10,       /* a bounded device-side wait ran out (read via psrl_device_status) */
  PSRL_ERR_INTERNAL = 11
} psrl_status_t;

typedef enum { PSRL_F32 = 0, PSRL_BF16 = 1 } psrl_dtype_t;

/* Segment flags. */
enum {
  PSRL_SEG_HAS_Q = 1,     /* the segment's tokens issue queries (rows of Q/O/dO/dQ exist) */
  PSRL_SEG_SAMPLE_END = 2 /* a training sample ends at this segment (root-to-here path) */
};

/*
 * Problem statement: a forest of token segments.  A sample is the path from a
 * root to a SAMPLE_END segment (tree sampling: leaves; step / tree-step
 * sampling: every node - paper Sec. 2.3).  Roots are independent prefix groups
 * (paper Sec. 4.2, semantic groups).  All pointers are HOST pointers, read
 * during psrl_plan_build only.
 */
typedef struct {
  int32_t n_segments;              /* >= 1 */
  const int32_t* parent;           /* [n_segments] -1 = root, else an index < own index */
  const int32_t* seg_len;          /* [n_segments] tokens, >= 1 */
  const uint8_t* seg_flags;        /* [n_segments] or NULL = HAS_Q everywhere, SAMPLE_END on leaves */
  const int32_t* group_block_size; /* one per root, in input order; power of two in [16, 256], or 0 =
                                      adaptive (Sec. 5.1): one extent per segment sized to its span at 16-slot
                                      granularity (bf16 path only) */
  int32_t n_groups;                /* must equal the number of roots */
  int32_t n_q_heads, n_kv_heads;   /* n_q_heads % n_kv_heads == 0 */
  int32_t head_dim;                /* 64 or 128 (f32), 128 (bf16) */
  psrl_dtype_t dtype;
  const int32_t* free_extents;     /* [2 * n_free] (start_slot, n_slots), multiples of 16; NULL = bump from 0 */
  int32_t n_free;
  /* Optional [n_segments] (input order) or NULL: where a segment's K/V already lives.  A value >= 0
   * (a multiple of 16) pins the segment: its pages are the consecutive runs of block-size slots starting
   * there and take nothing from the free extents; -1 allocates as usual.  This is how a prefix cached
   * by an earlier micro-batch is reused in place (paper Sec. 4.1 inter-batch / self-sequence sharing,
   * Sec. 5.2): the cache manager (psrl_cache.h) hands out these bases. */
  const int32_t* seg_slot_base;
} psrl_tree_desc_t;

typedef struct psrl_plan psrl_plan_t;

/*
 * Borrowed HOST pointers into the plan's canonical arrays (valid until
 * psrl_plan_destroy).  Segments are indexed in canonical order = DFS preorder,
 * roots and siblings in ascending input index.  The per-page fields are the
 * block metadata of the paper's KV manager (Sec. 6: base address, block size,
 * position of the token span in the full sequence, reference count); pages
 * follow reusable prefix spans and never cross a segment boundary (Sec. 5.1).
 */
typedef struct {
  int32_t n_seg, n_groups, n_pages, n_samples, max_depth;
  int32_t T;          /* tokens stored (each shared token once) */
  int32_t T_q;        /* tokens that issue queries */
  int32_t pool_slots; /* slots per KV head the pools must hold: max(page_slot + page_bs) */
  int64_t flat_tokens; /* sum of sample lengths (the unshared layout) */
  int64_t tree_pairs;  /* attended (query, key) pairs, shared:   sum len*anc + len(len+1)/2  (cf. Eq. 1) */
  int64_t flat_pairs;  /* attended pairs, unshared: sum L(L+1)/2 */
  int32_t n_anc, n_bt; /* lengths of anc_list and bt_pages */
  const int32_t *canon_of_input, *input_of_canon;               /* [n_seg] */
  const int32_t *seg_group, *seg_bs, *seg_parent, *seg_len, *seg_flags, *seg_depth;
  const int32_t *seg_anc_tokens; /* tokens of strict ancestors = position of the span in the sequence */
  const int32_t *seg_sub_end;    /* subtree = canonical indices [c, seg_sub_end[c]) */
  const int32_t *seg_tok_off;    /* exclusive prefix sum of seg_len */
  const int32_t *seg_q_off;      /* first row in Q/O/dO/dQ, -1 if the segment has no queries */
  const int32_t *seg_refcount;   /* samples that pass through the segment (Sec. 5.2) */
  const int32_t *anc_off, *anc_list;         /* CSR: strict ancestors root -> parent */
  const int32_t *seg_first_page, *seg_n_pages;
  const int32_t *page_seg, *page_bs, *page_valid, *page_pos, *page_refcount, *page_slot; /* [n_pages] */
  const int32_t *bt_off, *bt_pages;          /* CSR block table: ancestors' pages root -> parent, then own */
  const int32_t *tok_slot;                   /* [T] slot of every token in the pools */
  const int32_t *sample_end_seg, *sample_len; /* [n_samples] */
} psrl_plan_view_t;

/*
 * psrl_plan_build - host-side plan builder (paper Sec. 5.1 Adaptive Block
 * Allocation, Sec. 5.2 reference counts, Sec. 6 block metadata).
 * Turns the forest into the canonical plan (paged block table with a block
 * size per group) and a device work schedule.  Pure host code, no CUDA call.
 *   desc      HOST, read only during the call
 *   out_plan  HOST, receives a plan owned by the library (psrl_plan_destroy)
 * Errors: INVALID_ARG, BAD_TREE, BAD_BLOCK_SIZE, SHAPE, UNSUPPORTED,
 * POOL_FULL, HOST_OOM.  On error *out_plan is NULL.
 */
psrl_status_t psrl_plan_build(const psrl_tree_desc_t* desc, psrl_plan_t** out_plan);

/* Fills *out with borrowed host pointers.  INVALID_ARG on NULL. */
psrl_status_t psrl_plan_view(const psrl_plan_t* plan, psrl_plan_view_t* out);

/*
 * Borrowed HOST pointer to the device work schedule as psrl_plan_upload would
 * copy it (int32 words; *n_words = psrl_plan_device_bytes / 4).  The layout is
 * internal (a header of offsets, then the arrays: KV tiles, forward/dQ work
 * items with their KV-tile lists, dK/dV work items and splits, merge lists)
 * and not part of the bit-exact plan contract; it is exposed so that tests can
 * check its invariants - every (query row, key) pair of the tree covered
 * exactly once, every reduction a fixed total order (cf. the workload
 * estimate of Eq. 1 that the schedule balances) - without a GPU.
 * Valid until psrl_plan_destroy.  INVALID_ARG on NULL.
 */
psrl_status_t psrl_plan_schedule(const psrl_plan_t* plan, const int32_t** words, size_t* n_words);

/* Bytes of DEVICE memory psrl_plan_upload needs (0 for a NULL plan). */
size_t psrl_plan_device_bytes(const psrl_plan_t* plan);

/*
 * Copies the device schedule into caller-owned DEVICE memory (256-byte
 * aligned, >= psrl_plan_device_bytes) with cudaMemcpyAsync on `stream`
 * (a cudaStream_t passed as void*; NULL = default stream) and binds the plan
 * to that buffer.  The buffer must outlive every launch that uses the plan.
 * Errors: INVALID_ARG, WORKSPACE (too small), CUDA.
 */
psrl_status_t psrl_plan_upload(psrl_plan_t* plan, void* dev_buf, size_t bytes, void* stream);

/* Bytes of DEVICE workspace the forward / backward call needs (>= 256). */
size_t psrl_fwd_workspace_bytes(const psrl_plan_t* plan);
size_t psrl_bwd_workspace_bytes(const psrl_plan_t* plan);

/*
 * psrl_tree_attn_fwd - tree-causal attention forward (paper Sec. 2.5 attention
 * masking; Sec. 6: the attention backend locates K/V through block metadata).
 * For every query row i of a HAS_Q segment c and query head h (KV head
 * h / (Hq/Hkv)):  keys = all tokens of c's ancestors + tokens 0..i of c;
 *   O_i = softmax_j(scale * q_i . k_j) V,   LSE_i = ln sum_j exp(scale * q_i . k_j).
 * All tensor pointers are DEVICE pointers, 16-byte aligned, dtype = plan dtype (the Q-shaped ones may
 * be NULL when the plan has no query row at all, T_q = 0):
 *   q        [T_q, Hq, d]  read only; rows of segment c start at seg_q_off[c]
 *   k_pool   [Hkv, pool_capacity, d] read only; token t lives at slot tok_slot[t]
 *   v_pool   same layout.  Slots that hold no token (page pads, free slots)
 *            may contain anything, NaN included; they never reach an output.
 *   pool_capacity  slots per KV head in the caller's pools, >= plan pool_slots
 *   o        [T_q, Hq, d]  fully overwritten
 *   lse      [Hq, T_q] fp32 fully overwritten (natural log, scale inside)
 *   workspace, workspace_bytes  >= psrl_fwd_workspace_bytes(plan), 256-byte
 *            aligned; holds the device status word.  Concurrent launches need
 *            distinct workspaces.
 *   stream   cudaStream_t as void*
 * Errors: INVALID_ARG, SHAPE, WORKSPACE, CUDA.  Asynchronous.
 */
psrl_status_t psrl_tree_attn_fwd(const psrl_plan_t* plan, const void* q, const void* k_pool, const void* v_pool,
                                 int64_t pool_capacity, void* o, float* lse, float softmax_scale,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * psrl_tree_attn_bwd - backward of the above (paper Sec. 6: consumer adjoints
 * are accumulated on the shared prefix before one backward pass through its
 * producer).  Given dO (one row per shared token, already summed over the
 * samples that contain it):
 *   P = exp(S - LSE), dV = P^T dO, dP = dO V^T, D_i = dO_i . O_i,
 *   dS = P o (dP - D), dQ = scale dS K, dK = scale dS^T Q,
 * where dK/dV of a token sum over every query row that attends to it (its own
 * segment's later rows and all rows of all descendant segments) and over the
 * Hq/Hkv query heads of its KV head, in a fixed order.
 * DEVICE pointers, 16-byte aligned:
 *   q, k_pool, v_pool, o, lse   as in / as produced by the forward; read only
 *   d_o      [T_q, Hq, d] read only
 *   d_q      [T_q, Hq, d] fully overwritten
 *   dk_pool, dv_pool [Hkv, pool_capacity, d]: every slot of every page of the
 *            plan is overwritten (token slots: gradient; pad slots: 0); slots
 *            outside the plan's pages are not touched
 *   workspace >= psrl_bwd_workspace_bytes(plan): status word + D [Hq, T_q] fp32
 * Errors: INVALID_ARG, SHAPE, WORKSPACE, CUDA.  Asynchronous.
 */
psrl_status_t psrl_tree_attn_bwd(const psrl_plan_t* plan, const void* q, const void* k_pool, const void* v_pool,
                                 int64_t pool_capacity, const void* o, const float* lse, const void* d_o,
                                 void* d_q, void* dk_pool, void* dv_pool, float softmax_scale, void* workspace,
                                 size_t workspace_bytes, void* stream);

/*
 * psrl_tree_attn_bwd_static - the backward pass for callers that cannot
 * allocate device memory.  (The paper has no counterpart: this is a
 * convenience of this library.)
 *
 * psrl_tree_attn_bwd needs a caller-provided device workspace.  Callers that
 * must not call cudaMalloc - a latency-critical loop where an allocation would
 * synchronise the device, a plug-in inside a process whose GPU memory belongs
 * to another framework's pool, a process with a fixed memory budget - can use
 * this variant instead: its workspace is a fixed array inside the library
 * image (16 MiB + 256 bytes of device memory on every GPU that loads the
 * library, held until the process exits).  The call itself performs no
 * cudaMalloc / cudaFree and calls no allocating library routine.
 *
 * Same mathematics, same arguments (NULL Q-shaped pointers are accepted for a
 * plan without query rows, as there) and bit-identical results as
 * psrl_tree_attn_bwd, except:
 *   - no workspace arguments;
 *   - limit: the array stands in for the whole workspace, so a plan fits when
 *       psrl_bwd_workspace_bytes(plan) <= PSRL_BWD_STATIC_SCRATCH_BYTES,
 *     i.e. 256 bytes of header + D (one float per query row and head, so
 *     n_q_heads * T_q <= 4,194,304 at the very most) + the fp32 slabs of split
 *     KV tiles (n_kv_heads * 128 KiB each) + the partial dQ rows of cascaded
 *     prefixes (n_q_heads * 512 bytes each), the last two only for plans whose
 *     schedule has them.  Larger plans return PSRL_ERR_WORKSPACE and must use
 *     psrl_tree_attn_bwd;
 *   - status_workspace (HOST pointer, may be NULL) receives the DEVICE address
 *     of the array's status header; pass it to psrl_device_status to read the
 *     launch's device status.
 * Set-up: the first call on each device looks up the array's device address
 * (with that device current) and caches it.  Make that first call outside any
 * CUDA stream capture.
 * Sharing: every call on a device uses the same array, which keeps the
 * previous call's contents (the library clears what has to start at zero).
 * Two calls that overlap on the GPU - different streams, or different host
 * threads - race on it; serialise them, or use psrl_tree_attn_bwd with
 * separate workspaces.
 * Errors: INVALID_ARG, SHAPE, WORKSPACE (plan not uploaded, or over the
 * limit), CUDA.  Asynchronous.
 */
#define PSRL_BWD_STATIC_SCRATCH_BYTES ((size_t)16777472) /* 16 MiB + 256 */
psrl_status_t psrl_tree_attn_bwd_static(const psrl_plan_t* plan, const void* q, const void* k_pool,
                                        const void* v_pool, int64_t pool_capacity, const void* o, const float* lse,
                                        const void* d_o, void* d_q, void* dk_pool, void* dv_pool,
                                        float softmax_scale, void** status_workspace, void* stream);

/*
 * Synchronises `stream`, then reads the status word the last launch that used
 * `workspace` left: PSRL_OK, PSRL_ERR_TIMEOUT (a bounded wait gave up; outputs
 * are invalid) or PSRL_ERR_INTERNAL.  CUDA errors map to PSRL_ERR_CUDA.
 */
psrl_status_t psrl_device_status(const void* workspace, void* stream);

/*
 * psrl_kv_scatter / psrl_kv_gather - the neighbours of the attention calls: K and V leave the
 * projections token-major, the attention reads them through the paged pools (Sec. 6, KV manager), and
 * the gradients of the pools go back token-major.  scatter writes token t of the plan's tree (canonical
 * order, rows of `k_tok` / `v_tok`) to slot tok_slot[t] of every KV head; gather is the inverse read.
 * Slots that hold no token are neither written (scatter) nor read (gather).
 *   k_tok, v_tok  [T, Hkv, d] DEVICE, plan dtype, 16-byte aligned (either pair member may be NULL: skipped)
 *   k_pool, v_pool [Hkv, pool_capacity, d] DEVICE
 * Errors: INVALID_ARG, SHAPE, WORKSPACE (plan not uploaded), CUDA.  Asynchronous on `stream`.
 */
psrl_status_t psrl_kv_scatter(const psrl_plan_t* plan, const void* k_tok, const void* v_tok, void* k_pool,
                              void* v_pool, int64_t pool_capacity, void* stream);
psrl_status_t psrl_kv_gather(const psrl_plan_t* plan, const void* k_pool, const void* v_pool,
                             int64_t pool_capacity, void* k_tok, void* v_tok, void* stream);

/*
 * Rotary positions (the step between the projections and the attention).  Pair i of a head's first
 * `rotary_dim` elements is turned by the angle position * f_i:
 *   y1 = s (x1 cos - x2 sin),  y2 = s (x2 cos + x1 sin),   the other elements pass through.
 * A token's position is its place in its own sequence: the tokens of all ancestor segments, then its place in
 * the segment (seg_anc_tokens + i), so a token shared by many samples is rotated once.
 *   f_i = base^(-2 i / rotary_dim) radians per position, i < rotary_dim / 2, and with a scaling for contexts
 *   longer than `original_positions`:
 *   LINEAR  f_i / factor
 *   NTK     base replaced by base * factor^(rotary_dim / (rotary_dim - 2))
 *   YARN    pairs that make more than `high` turns over the original length keep f_i, pairs below `low` turns get
 *           f_i / factor, a linear ramp over the pair index between them; s = 0.1 ln(factor) + 1
 *           (Peng et al. 2023; low = 0 means 1, high = 0 means 32)
 *   BANDED  the same two ends with the ramp linear in the number of turns (low = 0 means 1, high = 0 means 4): the
 *           scaling by wavelength that open-weight long-context models published with their configurations in 2024
 * s is 1 unless YARN sets it; attention_scale > 0 replaces it.  Angles are computed exactly modulo a full turn
 * (64-bit fixed point), so far positions lose nothing.
 */
typedef enum { PSRL_ROPE_HALF = 0, PSRL_ROPE_INTERLEAVED = 1 } psrl_rope_layout_t; /* pairs (i, i + rotary_dim/2) | (2i, 2i + 1) */
typedef enum {
  PSRL_ROPE_UNSCALED = 0, PSRL_ROPE_LINEAR = 1, PSRL_ROPE_NTK = 2, PSRL_ROPE_YARN = 3, PSRL_ROPE_BANDED = 4
} psrl_rope_scaling_t;
typedef struct {
  int32_t head_dim;           /* multiple of 8, 8..256 */
  int32_t rotary_dim;         /* even, 2..head_dim */
  int32_t layout;             /* psrl_rope_layout_t */
  int32_t scaling;            /* psrl_rope_scaling_t */
  double base;                /* > 1 */
  double factor;              /* > 0, finite; read by every scaling but UNSCALED; YARN and BANDED: >= 1 */
  int32_t original_positions; /* YARN, BANDED: >= 1 */
  double low, high;           /* YARN, BANDED: turns, 0 <= low < high, 0 = the defaults above */
  double attention_scale;     /* 0 = as above */
} psrl_rope_desc_t;
typedef struct psrl_rope psrl_rope_t;

/* Host only.  Errors: INVALID_ARG, SHAPE (dimensions), HOST_OOM.  On error *out is NULL. */
psrl_status_t psrl_rope_create(const psrl_rope_desc_t* desc, psrl_rope_t** out);
/* Borrowed HOST pointer to the rotary_dim / 2 frequencies (radians per position) and the factor s. */
psrl_status_t psrl_rope_frequencies(const psrl_rope_t* rope, const double** freq, int32_t* n, double* scale);
void psrl_rope_destroy(psrl_rope_t* rope);

/*
 * psrl_rope_qkv_fwd - rotates the query rows and puts their keys and values into the pools, in one launch.
 * Row r is query row r of the plan (the tokens of the HAS_Q segments in canonical order; the K/V of other
 * segments is in the pools already, rotated, and is left alone).
 *   q  [T_q, Hq, d], k, v [T_q, Hkv, d]  DEVICE, plan dtype; row r at r * pitch elements, heads contiguous, so the
 *      three may be slices of one projection output
 *   q_out [T_q, Hq, d] contiguous: rotated Q (may be q itself when q is contiguous; INVALID_ARG when it is not)
 *   k_pool, v_pool [Hkv, pool_capacity, d]: rotated K and V of row r at the slot of its token; other slots untouched
 * A source may be NULL (with its destination ignored): skipped.  Pointers 16-byte aligned, pitches a multiple of
 * 16 bytes and at least a row.  Sources and destinations must not overlap otherwise.
 * Errors: INVALID_ARG, SHAPE (rope head_dim, pool size, pitches), WORKSPACE (plan not uploaded), CUDA.  Asynchronous.
 *
 * psrl_rope_qkv_bwd - the way back: the transposed (inverse) rotation of d_q and of the rows' slots of dk_pool, and the
 * rows' slots of dv_pool, to row-major dq_out, dk_out, dv_out with pitches (dq_out may be d_q with the pitch of a row).
 */
psrl_status_t psrl_rope_qkv_fwd(const psrl_plan_t* plan, const psrl_rope_t* rope, const void* q, int64_t q_pitch,
                                const void* k, int64_t k_pitch, const void* v, int64_t v_pitch, void* q_out,
                                void* k_pool, void* v_pool, int64_t pool_capacity, void* stream);
psrl_status_t psrl_rope_qkv_bwd(const psrl_plan_t* plan, const psrl_rope_t* rope, const void* d_q, const void* dk_pool,
                                const void* dv_pool, int64_t pool_capacity, void* dq_out, int64_t dq_pitch,
                                void* dk_out, int64_t dk_pitch, void* dv_out, int64_t dv_pitch, void* stream);

/*
 * psrl_rope_rows - the same rotation without a plan, for rows at positions of their own (one new token for each
 * sequence of a rollout).
 *   x, y  [n_rows, n_heads, d] DEVICE of `dtype`, rows at pitches as above; y may be x (equal pitches)
 *   positions [n_rows] DEVICE int32, any value;  inverse != 0: the transposed rotation
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED (dtype), CUDA.  n_rows = 0 does nothing.  Asynchronous.
 */
psrl_status_t psrl_rope_rows(const psrl_rope_t* rope, psrl_dtype_t dtype, const void* x, int64_t x_pitch,
                             const int32_t* positions, int64_t n_rows, int32_t n_heads, void* y, int64_t y_pitch,
                             int inverse, void* stream);

/*
 * psrl_plan_next_tokens - the targets of the tree's language-model loss.  A query row predicts the next token of its own
 * segment; the last row of a segment predicts the first token of every child (none at the end of a sample).  Row r's
 * targets are tokens next[off[r] .. off[r + 1]) - indices into the tree's tokens in canonical order (look their ids up to
 * get psrl_token_logprob_fwd's targets).  Only tokens of this plan are listed: where a later micro-batch continues a
 * segment, its first token is that plan's affair, and the caller's to add.
 *   off [T_q + 1], next [off[T_q]]  HOST, borrowed until psrl_plan_destroy
 */
psrl_status_t psrl_plan_next_tokens(const psrl_plan_t* plan, const int32_t** off, const int32_t** next);

/*
 * psrl_token_logprob_fwd / _bwd - the last step of the policy's forward pass and the first of its backward, over the
 * shared rows of the tree (each row once, however many samples run through it; paper Sec. 2.5, advantage masking: what
 * the samples' losses want of a shared token arrives as d_logprob of its targets).
 *   z = scale * hidden[r] . weight[v],   lse[r] = ln sum_v exp(z[r, v]),   logprob[t] = z[r, targets[t]] - lse[r]
 * for the targets t of row r: target_off[r] <= t < target_off[r + 1], or t = r when target_off is NULL (n_targets ==
 * n_rows).  Targets outside [0, vocab) are ignored: logprob 0, no gradient.  The logits are never stored.
 * Logits that are not finite: NaN or +inf makes the lse of its row and the logprob of the targets there NaN; -inf is an entry
 * of probability 0 (a row of nothing else has lse -inf, logprob NaN).  Other rows are not touched.
 * Backward: G_r = the sum of d_logprob over row r's targets,
 *   dz[r, v] = scale * (sum of d_logprob over r's targets equal to v  -  G_r exp(z[r, v] - lse[r]))
 *   d_hidden = dz weight,  d_weight = dz^T hidden
 * sums in fp32; bf16: dz rounded to bf16 as the tensor cores' operand (up to 128 rows in two parts), results rounded once;
 * f32: fp32 arithmetic throughout, as in the library's other fp32 paths (for parity; not tuned).  Bitwise reproducible.  A row
 * without a target, or whose d_logprob are all zero, contributes nothing (d_hidden row zero), whatever it holds, and costs
 * nothing but its place in the workspace.
 *   hidden   [n_rows, hidden_dim] DEVICE of `dtype`, row pitch in elements;  weight [vocab, hidden_dim] DEVICE of `dtype`
 *   targets  [n_targets] DEVICE int32;  target_off [n_rows + 1] DEVICE int32, not descending from 0 to n_targets, or NULL
 *   scale    finite, not 0 (1 / temperature)
 *   logprob, d_logprob [n_targets], lse [n_rows] DEVICE fp32 (backward: as produced by the forward)
 *   d_hidden, d_weight  DEVICE of `dtype` as their tensors, fully overwritten; NULL: not wanted
 *   workspace  DEVICE, >= psrl_token_logprob_workspace_bytes, 256-byte aligned; holds the device status word.  Forward:
 *              at most 16 bytes per row and 128 entries of the vocabulary (2 bytes where there are thousands of rows), and 8 MB;
 *              backward, with R = n_rows in whole 128s, at least 256: a piece of dz, 64 Mi numbers or 8192 per row of R if
 *              that is more; R rows of `hidden`; sums in fp32, R rows or 64 MB if that is more (bf16); 40 bytes per row and 24
 *              per target; whatever the vocabulary.  (Numbers and rows of `dtype`.)
 * hidden_dim is a multiple of 8, pitches are multiples of 16 bytes, tensors 16-byte aligned and apart from the outputs.
 * n_rows = 0 does nothing (backward: zeroes d_weight).  Rows, targets and vocabulary are at most 2^30.
 * Errors: INVALID_ARG, SHAPE, UNSUPPORTED (dtype), WORKSPACE, CUDA.  Asynchronous; calls that may overlap on the GPU need
 * distinct workspaces.
 */
size_t psrl_token_logprob_workspace_bytes(psrl_dtype_t dtype, int64_t n_rows, int32_t hidden_dim, int32_t vocab,
                                          int64_t n_targets, int backward);
psrl_status_t psrl_token_logprob_fwd(psrl_dtype_t dtype, int64_t n_rows, int32_t hidden_dim, int32_t vocab,
                                     const void* hidden, int64_t hidden_pitch, const void* weight, int64_t weight_pitch,
                                     const int32_t* targets, int64_t n_targets, const int32_t* target_off, float scale,
                                     float* logprob, float* lse, void* workspace, size_t workspace_bytes, void* stream);
psrl_status_t psrl_token_logprob_bwd(psrl_dtype_t dtype, int64_t n_rows, int32_t hidden_dim, int32_t vocab,
                                     const void* hidden, int64_t hidden_pitch, const void* weight, int64_t weight_pitch,
                                     const int32_t* targets, int64_t n_targets, const int32_t* target_off, float scale,
                                     const float* logprob, const float* lse, const float* d_logprob, void* d_hidden,
                                     int64_t d_hidden_pitch, void* d_weight, int64_t d_weight_pitch, void* workspace,
                                     size_t workspace_bytes, void* stream);

/*
 * Benchmark aid (no counterpart in the paper): psrl_tree_attn_bwd with a mask
 * of the backward kernels to launch, so that each can be timed on its own
 * with CUDA events.  Bit 0: D = rowsum(dO o O) pre-pass, bit 1: dQ kernel
 * (+ its merge), bit 2: dK/dV kernel (+ its reduce).  phases = 7 is exactly
 * psrl_tree_attn_bwd; with any other mask the outputs of the skipped kernels
 * are left untouched (and a skipped pre-pass leaves D as the previous call on
 * this workspace wrote it).  Stateless: the mask is an argument of the call.
 */
psrl_status_t psrl_bench_bwd_phases(const psrl_plan_t* plan, const void* q, const void* k_pool, const void* v_pool,
                                    int64_t pool_capacity, const void* o, const float* lse, const void* d_o,
                                    void* d_q, void* dk_pool, void* dv_pool, float softmax_scale, void* workspace,
                                    size_t workspace_bytes, void* stream, int phases);

/*
 * Number of kernels one psrl_tree_attn_fwd (backward == 0) or
 * psrl_tree_attn_bwd (backward != 0, all phases enabled) call launches for
 * this plan (no counterpart in the paper; bookkeeping for benchmarks).
 * Forward: 1, plus a merge when rows are assembled from partial results
 * (cascaded prefixes / split-KV).  Backward: D pre-pass + dQ + dK/dV, plus the
 * dQ merge, plus one fixed-order reduction when the bf16 schedule splits
 * heavy KV tiles.  0 for a NULL plan.
 */
int psrl_launch_count(const psrl_plan_t* plan, int backward);

/* Last CUDA error string seen by the library on this thread (HOST, static storage). */
const char* psrl_last_cuda_error(void);

void psrl_plan_destroy(psrl_plan_t* plan);
const char* psrl_status_string(psrl_status_t s);

#ifdef __cplusplus
}
#endif
#endif /* PSRL_H_ */
