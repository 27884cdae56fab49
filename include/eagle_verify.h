/*
 * eagle_verify.h - C ABI of the B200 (sm_100a) tree-verification library for EAGLE speculative decoding.
 *
 * The verification phase (Sec. 3.3, App. A.1 and A.2 of the EAGLE paper) scores every token of a
 * tree-structured draft in one target forward pass with tree attention, then walks the tree applying
 * multi-round speculative sampling (Algorithm 1) at every node.  This library implements, for one
 * attention layer and for the acceptance walk, exactly those two operations:
 *
 *   eagle_tree_verify_attn  tree-masked attention of the T draft-tree tokens against the committed
 *                           KV prefix plus the tree's own keys (a node sees the prefix, its ancestors
 *                           and itself)
 *   eagle_tree_accept       acceptance along the tree: greedy, or Algorithm 1 at every node
 *
 * Conventions shared by every call
 *   - Every pointer marked "device" is a device pointer owned by the caller; the library keeps none of
 *     them after the call returns, allocates no memory and never synchronises: work is enqueued on
 *     `stream` and the call returns.  Pointers marked "host" are ordinary host pointers.
 *   - Return value: EAGLE_OK, or a negative EAGLE_ERR_* when the host-side check of the arguments fails
 *     (nothing is launched) or a launch fails.  Problems only the device can see (a parent entry out of
 *     range, a prefix that does not fit the cache, a wait that ran out) are written to `*status`
 *     (device int32, first error wins, 0 = none); the affected sequence's rows are zeroed (attention)
 *     or its outputs set to "nothing accepted, bonus -1" (acceptance).  No trap is ever raised.
 *   - Tree: node i of sequence b has parent tree_parent[b, i] in [-1, i-1]; -1 means "child of the
 *     committed context".  At most 64 nodes per tree.  Entries at i >= tree size are ignored.
 */
#ifndef EAGLE_VERIFY_H_
#define EAGLE_VERIFY_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Opaque CUDA handles: a cudaStream_t / cudaEvent_t passed as a pointer-sized value. */
typedef void* eagle_stream_t;
typedef void* eagle_event_t;

enum {
  EAGLE_OK = 0,
  EAGLE_ERR_NULL = -1,       /* a required pointer is NULL */
  EAGLE_ERR_SHAPE = -2,      /* batch / heads / head_dim / max_tree / vocab out of the supported range */
  EAGLE_ERR_WORKSPACE = -3,  /* workspace missing, misaligned (256 B) or too small */
  EAGLE_ERR_LAUNCH = -4,     /* CUDA reported an error when launching */
  EAGLE_ERR_TREE = -5,       /* device-detected: parent entry outside [-1, i-1], or tree size out of range */
  EAGLE_ERR_SEQ = -6,        /* device-detected: seq_lens[b] < 0 or seq_lens[b] + tree size > kv_capacity */
  EAGLE_ERR_TOKEN = -7,      /* device-detected: draft token outside [0, vocab) */
  EAGLE_ERR_TIMEOUT = -8,    /* device-detected: a bounded wait inside a kernel ran out */
  EAGLE_ERR_DEVICE = -9,     /* the GPU is not an sm_100 device, or it lacks a required limit */
  EAGLE_ERR_PATH = -10,      /* device-detected: an accepted path that is not an increasing list of tree nodes whose slots exist */
  EAGLE_ERR_PAGE = -11,        /* device-detected: a block-table entry of a page in use outside [0, num_pages) */
  EAGLE_ERR_ROW = -12,         /* device-detected: a row of logits whose values are all -infinity or NaN: nothing can be drawn from it */
  EAGLE_ERR_SCALE = -13        /* device-detected: a scale of values in use that the attention does not take */
};

#define EAGLE_MAX_TREE 64

/*
 * Descriptor of one attention call.  Plain data, read during the call only.
 */
typedef struct eagle_attn_desc {
  int32_t batch;               /* B >= 0 */
  int32_t num_q_heads;         /* Hq; Hq % Hkv == 0, group size G = Hq / Hkv <= 16 */
  int32_t num_kv_heads;        /* Hkv */
  int32_t head_dim;            /* D: 64 or 128 */
  int32_t max_tree;            /* T_max <= 64: row stride of tree_parent, q and out */
  int32_t kv_capacity;         /* S_cap: slots per (sequence, KV head) of k_cache / v_cache */
  const int32_t* tree_sizes;   /* device int32 [B], or NULL: every tree has T_max nodes */
  float sm_scale;              /* softmax scale, > 0; 0 means 1/sqrt(D); negative or NaN is EAGLE_ERR_SHAPE */
  int32_t num_splits;          /* KV splits per sequence; 0 lets the device-side planner choose */
  void* workspace;             /* device, 256-byte aligned, >= eagle_tree_verify_attn_workspace() bytes */
  size_t workspace_bytes;
  int32_t* status;             /* device int32 or NULL */
  eagle_event_t ev_attn_begin; /* optional: recorded on `stream` right before / after the split-KV   */
  eagle_event_t ev_attn_end;   /* attention kernel (the dominant kernel), for timing it alone; or NULL */
  int32_t shared_tree;         /* nonzero: one tree for every sequence (the paper's experiments use one fixed tree shape,
                                  App. A.1): tree_parent is int32 [T_max] and tree_sizes NULL or int32 [1] */
} eagle_attn_desc;

/* Bytes of scratch one call with this descriptor needs (host function, no CUDA work).
 * Depends on batch, heads, head_dim, max_tree and num_splits only.  Returns 0 if the shape is unsupported.
 * With num_splits = 0 it is about 35 MB whatever the batch (plus some 100 bytes per (sequence, KV head, 256 query rows)). */
size_t eagle_tree_verify_attn_workspace(const eagle_attn_desc* desc);

/*
 * Tree-masked attention of one layer (tree attention of the verification pass: Sec. 3.3, App. A.1).
 *
 *   q        device bf16 [B, T_max, Hq, D]        queries of the tree tokens (already position-encoded)
 *   k_cache  device bf16 [B, Hkv, S_cap, D]       keys; slots [0, L_b) hold the committed prefix, slot
 *   v_cache  device bf16 [B, Hkv, S_cap, D]       L_b + m holds tree node m; later slots are never used
 *                                                 in the result, whatever they contain (NaN included)
 *   seq_lens device int32 [B]                     L_b, the committed prefix length (tree not included)
 *   tree_parent device int32 [B, T_max]           ([T_max] when desc->shared_tree is set)
 *   out      device bf16 [B, T_max, Hq, D]        out[b,i,h,:] = sum_j softmax_j(scale * q[b,i,h]·k[b,h/G,j]) v[b,h/G,j]
 *                                                 over j < L_b and j = L_b + m, m an ancestor of i or i itself;
 *                                                 rows of nodes i >= tree size are written as zeros
 *
 * Arithmetic: bf16 inputs, fp32 scores / softmax / accumulation, bf16 output (round to nearest even).  |scale * q.k| has to stay
 * below 2^20, 2^17 with an fp8 cache: the row maximum that the exponentials are relative to has 16 significant bits.  A score of a
 * visible key that is NaN or +infinite makes the rows that see it NaN.
 * q, k_cache and v_cache must be 16-byte aligned, out 32-byte aligned (else EAGLE_ERR_SHAPE).  Launches, in order on `stream`: the planner (tree masks +
 * work list), the split-KV attention kernel, the combine kernel.  The workspace must not be shared by
 * calls that can overlap on the GPU.
 */
int eagle_tree_verify_attn(const eagle_attn_desc* desc, const void* q, const void* k_cache, const void* v_cache,
                           const int32_t* seq_lens, const int32_t* tree_parent, void* out, eagle_stream_t stream);

/*
 * The same attention, for callers that cannot provide a workspace.  (The paper has no counterpart to this entry
 * point: it exists for the way the library is embedded, not for the method.)
 *
 * Who needs it: code that receives device pointers for its tensors but may not allocate device memory when it
 * runs - a serving backend whose memory pool is fixed at start-up, a plug-in living inside another engine's
 * execution context, a decode loop that must never call cudaMalloc because that call stalls the whole device.
 * Here the planner tables and the split partials live in a fixed array inside the library's device image,
 * eagle_tree_verify_attn_static_capacity() bytes (24 MiB) per GPU that loads the library, held until the
 * process ends.  `desc->workspace` and `desc->workspace_bytes` are ignored; everything else is as for
 * eagle_tree_verify_attn, and so are the results.
 *
 *   - No cudaMalloc, cudaFree or other allocating call is made, on any call.
 *   - Shapes whose tables and partials do not fit the array are refused with EAGLE_ERR_WORKSPACE and nothing is
 *     launched.  The need grows with batch * num_kv_heads * ceil(max_tree * G / 128), and steeply with a
 *     forced num_splits > 1; with num_splits = 0 the partials take (2 * (number of SMs) + 2 * batch if num_kv_heads is
 *     odd) * 128 * (D + 2) * 4 bytes (19.7 MB on a 148-SM B200 at D = 128), which leaves room for the tables of some 30 000
 *     (sequence, KV head, 256 query rows) units.
 *   - The first call on a device looks up the array's device address (once per device, with that device
 *     current).  Make that first call outside any stream capture.
 *   - All calls on one GPU share the one array, and it keeps the previous call's contents.  Nothing in it needs
 *     to start at zero (the planner kernel rewrites every table that is read, and each partial is written
 *     before it is merged), but two calls that can overlap on the GPU - different streams, or graphs replayed
 *     concurrently - would overwrite each other's plan: issue them on one stream, or order them yourself.
 */
int eagle_tree_verify_attn_static(const eagle_attn_desc* desc, const void* q, const void* k_cache, const void* v_cache,
                                  const int32_t* seq_lens, const int32_t* tree_parent, void* out, eagle_stream_t stream);

/* Size in bytes of the fixed array used by eagle_tree_verify_attn_static (host function). */
size_t eagle_tree_verify_attn_static_capacity(void);

/*
 * A KV cache kept in pages (a storage layout of the same cache: the verification pass of Sec. 3.3 reads the same keys
 * and values wherever a serving engine stores them).
 */
typedef struct eagle_paged_kv {
  const void* k_pages;          /* device bf16 [num_pages, Hkv, page_size, D], 16-byte aligned (uint8 codes for the _fp8 calls) */
  const void* v_pages;          /* device bf16 [num_pages, Hkv, page_size, D], 16-byte aligned */
  const int32_t* block_table;   /* device int32 [B, max_pages_per_seq]: slot j of sequence b is row j % page_size of page
                                   block_table[b, j / page_size]; entries of pages that hold no slot below
                                   seq_lens[b] + tree size are never read */
  int32_t num_pages;            /* pages in the pool, >= 1 */
  int32_t page_size;            /* slots per page: a power of two, >= 16 */
  int32_t max_pages_per_seq;    /* row length of block_table; a sequence holds at most max_pages_per_seq * page_size slots */
} eagle_paged_kv;

/*
 * eagle_tree_verify_attn over a paged cache.  Everything is as for that call (same planner, same kernels, same
 * arithmetic and results, same workspace size) except where the keys and values are read from: each 128-slot tile
 * is fetched page by page through the block table (one TMA box per page, or one box out of a page of 128 slots or
 * more).  desc->kv_capacity is ignored: the capacity is max_pages_per_seq * page_size.  A sequence whose prefix + tree
 * does not fit it reports EAGLE_ERR_SEQ, one with a block-table entry in use outside [0, num_pages) reports
 * EAGLE_ERR_PAGE; its output rows are zeros and no page is read for it.
 */
int eagle_tree_verify_attn_paged(const eagle_attn_desc* desc, const void* q, const eagle_paged_kv* kv,
                                 const int32_t* seq_lens, const int32_t* tree_parent, void* out, eagle_stream_t stream);

/*
 * The same call in two halves, for a verification pass over many layers.  The verification phase is one target
 * forward pass over every layer with the same draft tree and the same prefix lengths (Sec. 3.3, App. A.1); the tree
 * masks and the work split depend on nothing else, so they are made once per pass and reused by every layer:
 *
 *   eagle_tree_verify_plan          the planner alone: masks + work list into desc->workspace (one launch).
 *                                   `paged` is NULL for a contiguous cache; for a paged cache it names the block table
 *                                   (its page pointers are not read), so that the pages in use are validated.
 *   eagle_tree_verify_attn_planned  attention + combine of one layer over the plan in desc->workspace (two launches).
 *   eagle_tree_verify_attn_planned_paged   the same over a paged cache.
 *
 * The descriptor of the planned calls must equal the one the plan was made with (shape fields, num_splits, workspace),
 * on the same GPU; sm_scale, status and the events may differ.  Plan followed by planned gives bit for bit what
 * eagle_tree_verify_attn gives.  The plan stays valid until the workspace is written by another plan; the split
 * partials in the workspace are reused by every planned call, so planned calls that share a workspace must not overlap
 * on the GPU.  Arguments, results and errors as for eagle_tree_verify_attn (device-detected errors of the trees and
 * lengths are reported by the plan call; the planned calls then write zeros for the affected sequences).
 */
int eagle_tree_verify_plan(const eagle_attn_desc* desc, const int32_t* seq_lens, const int32_t* tree_parent,
                           const eagle_paged_kv* paged, eagle_stream_t stream);
int eagle_tree_verify_attn_planned(const eagle_attn_desc* desc, const void* q, const void* k_cache, const void* v_cache,
                                   void* out, eagle_stream_t stream);
int eagle_tree_verify_attn_planned_paged(const eagle_attn_desc* desc, const void* q, const eagle_paged_kv* kv, void* out,
                                         eagle_stream_t stream);

/*
 * The same attention over a cache STORED in fp8.  The decoding this method speeds up is bound by memory traffic (Sec. 4.4)
 * and the paper reports the method on a quantised deployment (Sec. 4.2); it fixes no quantisation scheme, so the
 * convention here is this library's: k_codes / v_codes are device uint8 [B, Hkv, S_cap, D] holding fp8 "e4m3" codes (1
 * sign, 4 exponent, 3 mantissa bits, bias 7, no infinities), and every (sequence, KV head) has one fp32 scale for its keys
 * and one for its values, k_scale / v_scale device fp32 [B, Hkv]:  key = value(code) * k_scale[b, h],  value =
 * value(code) * v_scale[b, h].  Only the storage changes: the codes are widened exactly (every e4m3 number is an fp16
 * number) on their way to the tensor cores, the keys' scale is folded into the softmax scale and the values' scale into
 * the output.  A tensor-core instruction takes one 16-bit type for both operands, so this form multiplies in fp16: the
 * bf16 queries are converted to fp16 (exact for magnitudes from 2^-14 to 65504; smaller ones are rounded to multiples of
 * 2^-24, larger ones become infinite) and the probabilities are rounded to fp16 instead of bf16.  Everything else (fp32
 * scores / softmax / accumulation, bf16 output, planner, work split, errors) is as for eagle_tree_verify_attn.  What it
 * saves is half of the cache bytes held and read.  head_dim must be 128 (else EAGLE_ERR_SHAPE).
 * Slots that are not visible may hold any code; one of the two NaN codes (0x7f, 0xff) in a VISIBLE slot makes the output
 * rows that see it NaN.
 * eagle_tree_verify_attn_planned_fp8 is the per-layer half over a plan made by eagle_tree_verify_plan (paged = NULL).
 */
int eagle_tree_verify_attn_fp8(const eagle_attn_desc* desc, const void* q, const void* k_codes, const void* v_codes,
                               const float* k_scale, const float* v_scale, const int32_t* seq_lens, const int32_t* tree_parent,
                               void* out, eagle_stream_t stream);
int eagle_tree_verify_attn_planned_fp8(const eagle_attn_desc* desc, const void* q, const void* k_codes, const void* v_codes,
                                       const float* k_scale, const float* v_scale, void* out, eagle_stream_t stream);

/*
 * The fp8 cache kept in pages: both storage choices of the same cache at once (Sec. 3.3 reads the same keys and values
 * wherever and however a serving engine stores them).  kv->k_pages / kv->v_pages are device uint8
 * [num_pages, Hkv, page_size, D] holding e4m3 codes, addressed through kv->block_table as for
 * eagle_tree_verify_attn_paged; k_scale / v_scale are device fp32 [B, Hkv] as for eagle_tree_verify_attn_fp8 (a page
 * belongs to one sequence, so the scales stay per (sequence, KV head)).  Arithmetic, errors and limits are those of the
 * two calls it combines: head_dim 128 (else EAGLE_ERR_SHAPE), fp16 x fp16 products, EAGLE_ERR_SEQ / EAGLE_ERR_PAGE per
 * sequence.  The planned form runs over a plan made by eagle_tree_verify_plan with the same `paged` description.
 */
int eagle_tree_verify_attn_paged_fp8(const eagle_attn_desc* desc, const void* q, const eagle_paged_kv* kv, const float* k_scale,
                                     const float* v_scale, const int32_t* seq_lens, const int32_t* tree_parent, void* out,
                                     eagle_stream_t stream);
int eagle_tree_verify_attn_planned_paged_fp8(const eagle_attn_desc* desc, const void* q, const eagle_paged_kv* kv,
                                             const float* k_scale, const float* v_scale, void* out, eagle_stream_t stream);


/*
 * Where a plan keeps its tree masks (host function, no CUDA work): device uint64 [B, T_max] inside desc->workspace,
 * bit m of entry [b, i] set iff node m is node i or one of its ancestors (the mask tree attention implies, Sec. 3.1 /
 * 3.3); entries of nodes >= tree size and of invalid sequences are 0.  Valid after eagle_tree_verify_plan or
 * eagle_tree_verify_attn on that workspace has run.  NULL if the descriptor is unusable.
 */
const uint64_t* eagle_tree_verify_plan_masks(const eagle_attn_desc* desc);

/*
 * How long a wait inside the attention kernel may go without progress before the kernel gives up, in nanoseconds
 * (host function; process-wide; applies to launches made after the call; 0 restores the default of two seconds).
 * Every wait in the kernels is bounded: when one runs out the kernel sets *status to EAGLE_ERR_TIMEOUT, releases what
 * it holds and returns, and the context stays usable.  Keep the limit far above the time a copy takes (milliseconds
 * are safe): a kernel that gives up while its own copies are still in flight would leave them writing into shared
 * memory it no longer owns.
 */
void eagle_set_wait_limit_ns(uint64_t ns);

/*
 * Test hook (fault injection for the time-out path; not for production use): attention launches (tree and chunk) made after this call
 * have their K/V producer stop issuing copies after `after_tiles` tiles per CTA, so the consumers' waits run out and
 * the kernel reports EAGLE_ERR_TIMEOUT.  Nothing is in flight when it returns.  A negative value switches it off.
 */
void eagle_test_stall_kv_producer(int32_t after_tiles);

/*
 * Descriptor of one acceptance call.
 */
typedef struct eagle_accept_desc {
  int32_t batch;               /* B >= 0 */
  int32_t max_tree;            /* T_max <= 64: row stride of the per-node arrays */
  int32_t vocab;               /* V >= 1 */
  int32_t path_cap;            /* entries per row of accepted_path; >= the deepest tree (T_max is always enough) */
  const int32_t* tree_sizes;   /* device int32 [B] or NULL */
  const uint8_t* greedy;       /* device uint8 [B] or NULL (= every sequence stochastic); 1: temperature-0 rule */
  int32_t* accept_len;         /* device int32 [B] or NULL: number of accepted nodes */
  int32_t* status;             /* device int32 or NULL */
  int32_t shared_tree;         /* nonzero: one tree for every sequence: tree_parent is int32 [T_max], tree_sizes NULL or int32 [1]
                                  (draft_tokens, the probability rows and the uniforms stay per sequence) */
} eagle_accept_desc;

/*
 * Acceptance along the draft tree: Algorithm 1 (multi-round speculative sampling, App. A.2) applied at
 * every node starting from the committed context (Sec. 3.3), or the greedy rule (Preliminaries).
 *
 *   target_probs device fp32 [B, T_max+1, V]   row 0: target distribution after the context;
 *                                              row i+1: target distribution after tree node i
 *   draft_probs  device fp32 [B, T_max, V]     row i: the distribution node i's token was drawn from
 *                                              (may be NULL when every sequence is greedy)
 *   draft_tokens device int32 [B, T_max]
 *   tree_parent  device int32 [B, T_max]      ([T_max] when desc->shared_tree is set)
 *   uniforms     device fp32 [B, T_max+1]      entry i: the uniform of node i's accept test; entry T_max:
 *                                              the uniform of the final draw (may be NULL when all greedy)
 *   accepted_path device int32 [B, path_cap]   accepted node indices from the top of the tree down, then -1
 *   bonus_token  device int32 [B]              the one extra token every step emits
 *
 * Per sequence: cur = context.  The children of cur, in ascending index, are Algorithm 1's candidates
 * against p = target row of cur: candidate i with token t is accepted iff r_i * p^_i(t) < p(t) (that is
 * r_i < p(t)/p^_i(t)); on rejection p <- norm(max(0, p - p^_i)) over the vocabulary (kept if its mass is
 * zero).  An accepted child becomes cur and starts again from its own target row.  When no child is
 * accepted (a leaf included) the bonus token is drawn from p by inverse CDF in ascending token id: the
 * smallest x with sum_{v<=x} p(v) > u * sum_v p(v).  Greedy sequences move to the lowest-index child whose
 * token equals argmax p (lowest id on ties), else emit that argmax.  Rows are used as given (not
 * renormalised).  Scalars and sums are fp64, so decisions agree with an fp64 reference except within
 * rounding of a boundary.
 */
int eagle_tree_accept(const eagle_accept_desc* desc, const float* target_probs, const float* draft_probs,
                      const int32_t* draft_tokens, const int32_t* tree_parent, const float* uniforms,
                      int32_t* accepted_path, int32_t* bonus_token, eagle_stream_t stream);

/*
 * How an acceptance call of this batch size and vocabulary is laid out on the current GPU (host function, launches
 * nothing): 0 when one warp walks each tree (vocabularies up to 4096), else the number of 512-thread CTAs, 1, 2, 4 or
 * 8, that form the thread-block cluster walking one tree (the fewer trees, the wider the cluster).  The result of
 * eagle_tree_accept does not depend on it; it is reported so that every variant can be told apart and exercised.
 * Negative EAGLE_ERR_* on a bad argument or when no sm_100 device is current.
 */
int eagle_tree_accept_cluster_width(int32_t batch, int32_t vocab);
/* The same for a call that passes draft_probs == NULL or uniforms == NULL, i.e. one whose sequences are all greedy (the
 * setting of most of the paper's tables, temperature 0): its walk is argmax sweeps only, and where eight CTAs per tree
 * would not fit the GPU at once it takes four. */
int eagle_tree_accept_cluster_width_greedy(int32_t batch, int32_t vocab);

/*
 * One whole verification step driven from HOST buffers (the two calls above, with the copies around them).
 *
 * Every input pointer below is a host pointer (pinned memory makes the copies asynchronous); the call enqueues on
 * `stream`: host->device copies of the inputs into `arena` (see eagle_tree_verify_step_host_bytes for what is copied),
 * eagle_tree_verify_attn, eagle_tree_accept, and
 * device->host copies of out, accepted_path, bonus_token and accept_len.  It allocates nothing: `arena` is device
 * memory provided by the caller, 256-byte aligned, at least eagle_tree_verify_step_host_arena() bytes (device copies
 * of all tensors plus the attention workspace).  The results are in the host buffers once `stream` has drained.
 * Verification phase: Sec. 3.3; acceptance: App. A.2, Algorithm 1.  Shapes and meanings as for the device calls.
 */
typedef struct eagle_host_step {
  int32_t batch, num_q_heads, num_kv_heads, head_dim, max_tree, kv_capacity, vocab, path_cap;
  float sm_scale;
  const void* q;                 /* host bf16 [B, T_max, Hq, D] */
  const void* k_cache;           /* host bf16 [B, Hkv, S_cap, D] */
  const void* v_cache;
  const int32_t* seq_lens;       /* host int32 [B] */
  const int32_t* tree_sizes;     /* host int32 [B] or NULL */
  const int32_t* tree_parent;    /* host int32 [B, T_max] */
  const float* target_probs;     /* host fp32 [B, T_max+1, V] */
  const float* draft_probs;      /* host fp32 [B, T_max, V] */
  const int32_t* draft_tokens;   /* host int32 [B, T_max] */
  const float* uniforms;         /* host fp32 [B, T_max+1] */
  const uint8_t* greedy;         /* host uint8 [B] or NULL */
  void* out;                     /* host bf16 [B, T_max, Hq, D] */
  int32_t* accepted_path;        /* host int32 [B, path_cap] */
  int32_t* bonus_token;          /* host int32 [B] */
  int32_t* accept_len;           /* host int32 [B] */
  int32_t* status;               /* host int32[1]: device-detected status of the step (0 = ok) */
  void* arena;                   /* device */
  size_t arena_bytes;
} eagle_host_step;

size_t eagle_tree_verify_step_host_arena(const eagle_host_step* step);
int eagle_tree_verify_step_host(const eagle_host_step* step, eagle_stream_t stream);

/*
 * Bytes one eagle_tree_verify_step_host call with these arguments copies host->device and device->host (host function,
 * no CUDA work; reads the host arrays seq_lens and tree_sizes).  Of k_cache / v_cache only the slots a sequence can see
 * (seq_lens[b] + tree size, clamped to the capacity; none for an empty tree) and of target_probs / draft_probs only the
 * rows of existing nodes are ever read by the kernels, so when that saves more than the extra copy calls cost the step
 * copies exactly those, sequence by sequence (2-D copies), and leaves the rest of the arena as it is; otherwise every
 * tensor is copied whole.  This function reports which of the two the call does.
 */
int eagle_tree_verify_step_host_bytes(const eagle_host_step* step, size_t* h2d_bytes, size_t* d2h_bytes);

/*
 * The same acceptance walk with the distributions given as LOGITS: every row the walk touches is taken as
 * softmax(logits / temperature) without being materialised (the target and draft probability tensors, [B, T_max+1, V]
 * and [B, T_max, V], are never written or read as a whole; only the rows on the walk are swept).  Sec. 4 runs the
 * method at temperature 1 (and at temperature 0, which is the per-sequence `greedy` flag of the descriptor: greedy
 * sequences use the argmax of the logits and ignore `temperature`).
 *
 *   target_logits device fp32 [B, T_max+1, V], draft_logits device fp32 [B, T_max, V]; temperature > 0 (else
 *   EAGLE_ERR_SHAPE); everything else as for eagle_tree_accept.
 *
 * Each row costs one more sweep (its maximum and its mass).  Exponentials are taken in fp32 (2^((z - max) * log2(e) /
 * temperature)), sums and scalars in fp64, so a decision can differ from an fp64 softmax only when it sits within
 * about 1e-6 of its boundary.
 */
int eagle_tree_accept_logits(const eagle_accept_desc* desc, const float* target_logits, const float* draft_logits,
                             const int32_t* draft_tokens, const int32_t* tree_parent, const float* uniforms,
                             float temperature, int32_t* accepted_path, int32_t* bonus_token, eagle_stream_t stream);

#define EAGLE_MAX_CHILDREN 16

typedef struct eagle_expand_desc {
  int32_t batch;               /* B >= 0 (at most 65535) */
  int32_t rows;                /* R >= 0: draft-tree nodes expanded per sequence in this call */
  int32_t vocab;               /* V >= 1 */
  int32_t max_children;        /* K <= EAGLE_MAX_CHILDREN: row stride of the per-child arrays */
  const uint8_t* greedy;       /* device uint8 [B] or NULL (= every sequence stochastic) */
  int32_t* status;             /* device int32 or NULL */
} eagle_expand_desc;

/*
 * Child tokens of draft-tree nodes (App. A.1, tree structure: in the greedy setting the k most probable tokens of a
 * node's draft distribution become its children, otherwise k tokens are sampled; k varies from node to node).
 *
 *   draft_probs  device fp32 [B, R, V]   the draft distribution at each node (used as given, not renormalised)
 *   num_children device int32 [B, R]     k of each node, 0 <= k <= K (greedy: also k <= V)
 *   uniforms     device fp32 [B, R, K]   one uniform in [0, 1) per draw (may be NULL when every sequence is greedy)
 *   child_tokens device int32 [B, R, K]  the k tokens, then -1
 *   child_probs  device fp32 [B, R, K] or NULL   draft_probs at those tokens, then 0
 *
 * Greedy sequences: descending probability, the lower token id first among equal values (exact).  Other sequences: k
 * independent draws (with replacement; the paper does not say), draw j = the smallest x with
 * sum_{v<=x} p(v) > uniforms[j] * sum_v p(v), prefix sums in fp64 (the last token with positive mass if rounding
 * leaves none).  A node whose k is out of range sets *status to EAGLE_ERR_SHAPE and gets no children.
 * One launch, asynchronous on `stream`; no workspace.
 */
int eagle_tree_expand(const eagle_expand_desc* desc, const float* draft_probs, const int32_t* num_children,
                      const float* uniforms, int32_t* child_tokens, float* child_probs, eagle_stream_t stream);

typedef struct eagle_commit_desc {
  int32_t batch;               /* B >= 0 (at most 65535) */
  int32_t num_kv_heads;        /* Hkv >= 0 */
  int32_t head_dim;            /* D: 64 or 128 */
  int32_t kv_capacity;         /* S_cap: slots per (sequence, KV head) of k_cache / v_cache */
  int32_t max_tree;            /* T_max <= 64: tree nodes are numbered 0 .. T_max-1; row count of features_in */
  int32_t path_cap;            /* entries per row of accepted_path */
  int32_t feature_dim;         /* F: elements per feature vector, a multiple of 8; 0 when no features are passed */
  int32_t* status;             /* device int32 or NULL */
} eagle_commit_desc;

/*
 * Commit of the accepted path: what the verification phase leaves behind for the next drafting phase (Sec. 3.3, last
 * sentence: the accepted tokens and their features are recorded).  The paper does not say where anything is stored;
 * with the cache layout of eagle_tree_verify_attn (tree node m at slot L_b + m) it is this:
 *
 *   k_cache, v_cache  device bf16 [B, Hkv, S_cap, D], updated IN PLACE (either may be NULL): for every sequence b with
 *                     accepted nodes path[0..a-1], slot L_b + j <- slot L_b + path[j] for all j < a at once (the
 *                     sources are read before any destination is written); all other slots keep their contents
 *   seq_lens          device int32 [B]          L_b, the committed prefix before the step
 *   accepted_path     device int32 [B, path_cap] node indices from the top of the tree down, then -1 (the output of
 *                                               eagle_tree_accept); entries after the first -1 are ignored
 *   features_in       device bf16 [B, T_max, F] or NULL   one vector per tree node (the target model's features)
 *   features_out      device bf16 [B, path_cap, F] or NULL  row j <- features_in row path[j] for j < a, zeros for j >= a
 *   new_seq_lens      device int32 [B] or NULL  L_b + a  (may alias seq_lens)
 *
 * One call serves one layer's cache; the token of the step's extra draw is not part of the path (its K/V do not
 * exist yet).  A row that is not strictly increasing, leaves [0, T_max), or points at a slot >= S_cap (or L_b < 0)
 * sets *status to EAGLE_ERR_PATH: nothing of that sequence is moved, its length is unchanged and its feature rows are
 * zeros.  All pointers must be 16-byte aligned.  One launch, asynchronous on `stream`; no workspace.
 * A cache of fp8 codes (uint8 [B, Hkv, S_cap, 128], see eagle_tree_verify_attn_fp8) is committed by the same call with
 * head_dim = 64: a row of 128 codes is a row of 64 16-bit elements and rows are moved as bytes (the scales do not change).
 */
int eagle_tree_commit(const eagle_commit_desc* desc, void* k_cache, void* v_cache, const int32_t* seq_lens,
                      const int32_t* accepted_path, const void* features_in, void* features_out,
                      int32_t* new_seq_lens, eagle_stream_t stream);

/*
 * eagle_tree_commit on a paged cache (see eagle_paged_kv): the pages named by kv->k_pages / kv->v_pages are updated IN
 * PLACE although the struct declares them const (either may be NULL).  Rows are copied between, or within, the pages
 * the sequence already owns; no page is allocated, freed or moved.  desc->kv_capacity is ignored (the capacity is
 * max_pages_per_seq * page_size).  A source or destination slot whose block-table entry is outside [0, num_pages)
 * sets *status to EAGLE_ERR_PAGE and the sequence is left alone, as for an invalid path.  Everything else as above.
 */
int eagle_tree_commit_paged(const eagle_commit_desc* desc, const eagle_paged_kv* kv, const int32_t* seq_lens,
                            const int32_t* accepted_path, const void* features_in, void* features_out,
                            int32_t* new_seq_lens, eagle_stream_t stream);

/*
 * Tree-mask builder alone (the mask "tree attention" implies: Sec. 3.1, Sec. 3.3): for every node the bit set
 * of its ancestors and itself, and its depth (top-level nodes: 1).
 *   tree_parent device int32 [B, T_max]; tree_sizes device int32 [B] or NULL;
 *   anc_mask device uint64 [B, T_max]; depth device uint8 [B, T_max] or NULL; status device int32 or NULL.
 * Entries of nodes >= tree size, and of sequences with an invalid tree, are 0.
 */
int eagle_tree_build_mask(const int32_t* tree_parent, const int32_t* tree_sizes, int32_t batch, int32_t max_tree,
                          uint64_t* anc_mask, uint8_t* depth, int32_t* status, eagle_stream_t stream);

/*
 * ---------------------------------------------------------------------------------------------------------------------
 * Around the verification step: rotary positions written into the cache, attention of a prompt's chunk, and penalties,
 * biases and grammar masks on the rows that acceptance reads.
 */

/*
 * A cache as the calls below take it, in any of its storage forms (see eagle_tree_verify_attn, eagle_paged_kv and
 * eagle_tree_verify_attn_fp8 for the layouts).
 */
typedef struct eagle_kv_store {
  void* k;                      /* device bf16, or uint8 e4m3 codes when the scales are set; 16-byte aligned:
                                   [B, Hkv, kv_capacity, D], or [num_pages, Hkv, page_size, D] with a block table */
  void* v;
  const float* k_scale;         /* device fp32 [B, Hkv], both or neither: the cache holds codes (head_dim 128) */
  const float* v_scale;
  int32_t kv_capacity;          /* slots per (sequence, KV head); ignored with a block table */
  const int32_t* block_table;   /* device int32 [B, max_pages_per_seq], or NULL: contiguous */
  int32_t num_pages;            /* pages in the pool, >= 1 */
  int32_t page_size;            /* a power of two, >= 16 */
  int32_t max_pages_per_seq;
} eagle_kv_store;

/* How rotary frequencies are stretched for contexts beyond the trained one. */
enum {
  EAGLE_ROPE_PLAIN = 0,         /* f_m = base^(-2m / R) */
  EAGLE_ROPE_LINEAR = 1,        /* f_m / factor */
  EAGLE_ROPE_NTK = 2,           /* base replaced by base * factor^(R / (R - 2)) */
  EAGLE_ROPE_YARN = 3,          /* f_m / factor below a band of wavelengths, f_m above it, a ramp between; amplitude 0.1 ln(factor) + 1 */
  EAGLE_ROPE_BANDED = 4         /* f_m / factor for wavelengths over context / low, f_m under context / high, blended between */
};
typedef struct eagle_rope_scaling {
  int32_t kind;                 /* EAGLE_ROPE_* */
  int32_t rotary_dim;           /* R: even, >= 2 (NTK: >= 4) */
  double base;                  /* > 1 */
  double factor;                /* >= 1 (all kinds but PLAIN) */
  double context;               /* the trained context, > 0 (YARN, BANDED) */
  double low, high;             /* YARN: turns over the trained context at the band's ends, high > low > 0 (32 and 1 are usual: high = 32,
                                   low = 1); BANDED: 0 < low < high (1 and 4 are usual) */
} eagle_rope_scaling;

/*
 * Rotary frequencies (host function, no CUDA work): freqs, host double [R / 2], in radians per position, and the amplitude
 * that sines and cosines are to be multiplied by (1 for all kinds but YARN).
 *   YARN: with d(t) = R ln(context / (2 pi t)) / (2 ln base), lo = max(floor(d(high)), 0), hi = min(ceil(d(low)), R - 1) (hi = lo + 0.001
 *   if they are equal), ramp = clamp((m - lo) / (hi - lo), 0, 1): f_m (1 - ramp) + f_m / factor * ramp.
 *   BANDED: with the wavelength w = 2 pi / f_m and s = (context / w - low) / (high - low) between the two borders: (1 - s) f_m / factor + s f_m.
 * EAGLE_ERR_NULL / EAGLE_ERR_SHAPE on bad arguments.
 */
int eagle_rope_frequencies(const eagle_rope_scaling* scaling, double* freqs, float* amplitude);

typedef struct eagle_rope_desc {
  int32_t batch;                /* B, 0 .. 65535 */
  int32_t num_tokens;           /* N >= 0: rows of q, k, v and q_out (chunk form) */
  int32_t max_tree;             /* T_max <= 64 (tree form; q, k, v and q_out have B * T_max rows) */
  int32_t num_q_heads;          /* Hq >= 0 (0: only the cache is written) */
  int32_t num_kv_heads;         /* Hkv >= 1 */
  int32_t head_dim;             /* D: 64 or 128 */
  int32_t rotary_dim;           /* R: a multiple of 16, <= D: the first R elements of each head turn, the others stay */
  int32_t interleaved;          /* 0: element m turns with m + R/2; nonzero: element 2m with 2m + 1 */
  float amplitude;              /* factor on sines and cosines; 0 means 1 */
  int64_t q_stride, k_stride, v_stride;   /* elements from one row to the next: multiples of 8, at least heads * D (slices of one
                                   projection's output need no copy); 0 means heads * D.  A row's heads are dense. */
  const double* freqs;          /* device double [R / 2], radians per position */
  const int32_t* positions;     /* chunk form: device int32 [N], or NULL: a token's position is its slot */
  const int32_t* tree_sizes;    /* tree form: device int32 [B] ([1] when shared_tree is set), or NULL */
  int32_t shared_tree;          /* tree form, nonzero: tree_parent is int32 [T_max], one tree for every sequence */
  int32_t* status;              /* device int32 or NULL */
} eagle_rope_desc;

/*
 * Rotary positions of new tokens, and their keys and values into the cache, in one launch.
 *
 *   q, k, v     device bf16 [N, Hq, D], [N, Hkv, D], [N, Hkv, D] with the descriptor's strides, 16-byte aligned
 *   seq_lens    device int32 [B]      L_b: slots of the cache that are in use already
 *   token_start device int32 [B + 1]  ascending: rows token_start[b] .. token_start[b + 1] - 1 are sequence b's new tokens, in order
 *   q_out       device bf16 [N, Hq, D] dense, 16-byte aligned; may be q itself when q is dense
 *
 * Token i of sequence b turns by position L_b + i (or positions[row]) and goes to slot L_b + i.  Pair (x, y) of frequency f at
 * position p becomes amplitude * (x cos pf - y sin pf, y cos pf + x sin pf); the angle is reduced in fp64, the rotation is
 * fp32, rounded once.  Keys of an fp8 cache are stored as the nearest e4m3 code of key / k_scale[b, h] in fp32 (ties go
 * to the even code, magnitudes above 448 become 448; scales are normal numbers of fp32), values likewise.  Nothing
 * else in the cache changes.  Rows outside every sequence (behind the last one) are not written.  A sequence with L_b < 0 or more tokens than its slots reports EAGLE_ERR_SEQ: its rows of q_out
 * are zeros and nothing of it is stored; starts that descend or leave [0, N] report it too, and rows that they do not place
 * are left alone.  A token whose page is outside the pool reports EAGLE_ERR_PAGE and is not stored.
 */
int eagle_rope_append(const eagle_rope_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                      const int32_t* seq_lens, const int32_t* token_start, eagle_stream_t stream);

/*
 * The same for the nodes of draft trees, in the layout of eagle_tree_verify_attn: q, k, v and q_out have rows [B, T_max], node i
 * of sequence b turns by position L_b + depth(i) - 1 (top-level nodes have depth 1: siblings share a position) and goes to slot
 * L_b + i.  Rows of nodes >= tree size are left alone.  An invalid tree reports EAGLE_ERR_TREE, a tree that does not fit
 * EAGLE_ERR_SEQ: the sequence's rows of q_out are zeros and nothing of it is stored.
 */
int eagle_tree_rope_append(const eagle_rope_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                           const int32_t* seq_lens, const int32_t* tree_parent, eagle_stream_t stream);

typedef struct eagle_chunk_desc {
  int32_t batch;                /* B, 0 .. 65535 */
  int32_t num_tokens;           /* N >= 0: rows of q and out */
  int32_t num_q_heads;          /* Hq; Hq % Hkv == 0, group size G = Hq / Hkv <= 16 */
  int32_t num_kv_heads;         /* Hkv */
  int32_t head_dim;             /* D: 64 or 128 */
  float sm_scale;               /* softmax scale, > 0; 0 means 1/sqrt(D) */
  void* workspace;              /* device, 256-byte aligned, >= eagle_chunk_attn_workspace() bytes */
  size_t workspace_bytes;
  int32_t* status;              /* device int32 or NULL */
} eagle_chunk_desc;

/* Bytes of scratch one call with this descriptor, or with fewer tokens, needs (host function, no CUDA work); 0 if the shape is unsupported. */
size_t eagle_chunk_attn_workspace(const eagle_chunk_desc* desc);

/*
 * Causal attention of one layer for chunks of new tokens: a prompt, a part of one, or single tokens, any mix in one call.
 *
 *   q           device bf16 [N, Hq, D], 16-byte aligned   queries, already position-encoded (q_out of eagle_rope_append)
 *   kv          the cache, bf16, contiguous or paged, with the chunk's own keys and values in it
 *   seq_lens    device int32 [B]      L_b: slots in use before the chunk
 *   token_start device int32 [B + 1]  as for eagle_rope_append
 *   out         device bf16 [N, Hq, D], 32-byte aligned   out[t,h,:] = sum_j softmax_j(scale * q[t,h]·k[b,h/G,j]) v[b,h/G,j], j <= L_b + i
 *                                     for token t = token_start[b] + i of sequence b
 *
 * A cache of fp8 codes is EAGLE_ERR_SHAPE.  bf16 inputs, fp32 scores / softmax / accumulation, probabilities rounded to bf16
 * for the tensor cores, bf16 output.  |scale * q.k| has to stay below 2^29 (beyond, a step of fp32 is wider than what an exponential spans:
 * a row may come out NaN).  Slots past the chunk may hold anything.  The values of slots in use have to be finite:
 * one that is not may reach rows of the same sequence that do not see it (its probability there is 0, and 0 * inf is NaN).
 * Rows outside every sequence are left as they were.  A sequence with L_b < 0 or L_b + n_b over its slots reports EAGLE_ERR_SEQ,
 * one with a block-table entry in use outside [0, num_pages) EAGLE_ERR_PAGE: its rows are zeros.  Starts that descend or
 * leave [0, N] report EAGLE_ERR_SEQ and no row is computed.  A wait inside the attention kernel that runs out reports EAGLE_ERR_TIMEOUT, and rows inside the
 * sequences may then hold anything (eagle_set_wait_limit_ns).  Three launches (planner, attention, merge), asynchronous on
 * `stream`; calls that share a workspace must not overlap on the GPU.  Calls with N <= B run a kernel made for single tokens (it is
 * right for any lengths, but reads a sequence's cache once for every 16 / G of its tokens).  A chunk of many tokens among as many empty
 * sequences is faster in the other kernel, up to five times at 200 tokens behind 8192 slots: leave empty sequences out, or pass a row
 * more than there are sequences; single tokens are up to 1.3 times faster without such a row.
 */
int eagle_chunk_attn(const eagle_chunk_desc* desc, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens,
                     const int32_t* token_start, void* out, eagle_stream_t stream);

#define EAGLE_MAX_BIAS 1024

typedef struct eagle_logits_desc {
  int32_t batch;                /* B, 0 .. 65535 */
  int32_t max_tree;             /* T_max <= 64; 0: one row per sequence, no trees */
  int32_t vocab;                /* V, 1 .. 2^30 */
  int32_t bf16;                 /* 0: logits are fp32; nonzero: bf16 */
  const int32_t* tree_sizes;    /* device int32 [B] ([1] when shared_tree is set), or NULL: T_max nodes each */
  int32_t shared_tree;          /* one tree for every sequence: tree_parent is [T_max] (draft_tokens stay per sequence) */
  int32_t history_cap;          /* row length of history */
  const int32_t* history;       /* device int32 [B, history_cap]: the sequence's tokens, prompt first; or NULL: nothing was there before */
  const int32_t* history_len;   /* device int32 [B] (with history) */
  const int32_t* prompt_len;    /* device int32 [B], or NULL: all of the history was generated */
  const float* repetition;      /* device fp32 [B] or NULL (1): rho > 0 */
  const float* presence;        /* device fp32 [B] or NULL (0): pi */
  const float* frequency;       /* device fp32 [B] or NULL (0): phi */
  int32_t max_bias;             /* row length of the bias lists, <= EAGLE_MAX_BIAS */
  const int32_t* bias_tokens;   /* device int32 [B, max_bias] or NULL */
  const float* bias_values;     /* device fp32 [B, max_bias] (with bias_tokens); a token listed twice gets the sum */
  const int32_t* bias_len;      /* device int32 [B], or NULL: max_bias entries each */
  const uint32_t* allowed;      /* device uint32 [B, T_max + 1, ceil(V / 32)] or NULL: bit v % 32 of word v / 32 is set where token v may follow */
  int32_t* status;              /* device int32 or NULL */
} eagle_logits_desc;

/*
 * Penalties for repeated tokens, biases and grammar masks on the target's rows of a draft tree (T_max = 0: on one row per
 * sequence, plain decoding), into the fp32 rows that eagle_tree_accept_logits reads.
 *
 *   logits       device fp32 or bf16 [B, T_max + 1, V]   row 0: after the context; row i + 1: after tree node i
 *   draft_tokens device int32 [B, T_max], tree_parent device int32 [B, T_max] ([T_max] when shared_tree is set); unused with T_max = 0
 *   out          device fp32 [B, T_max + 1, V]; may be `logits` itself when that is fp32
 *
 * With c the number of times token v was generated (in the history past the prompt, and on the path from the root to the row's
 * node, that node included) and seen = c > 0 or v in the prompt:
 *     z <- seen ? (z > 0 ? z / rho : z * rho) : z;   z <- z - phi c - (c > 0 ? pi : 0);   z <- z + bias(v);   not allowed: -inf
 * in fp32, z / rho as z times the rounded 1 / rho, and what is added to z summed up first.  A row whose mask allows nothing is all -inf (an acceptance walk that ends there still returns a token of the
 * vocabulary, which then means nothing).  Rows of nodes >= tree size are not written.  Lengths are clamped to
 * their rows; a token outside the vocabulary (history, bias list, draft) is ignored and reports EAGLE_ERR_TOKEN; an invalid
 * tree reports EAGLE_ERR_TREE and all T_max + 1 rows of its sequence become zeros.  One launch; no workspace.
 */
int eagle_tree_logits_adjust(const eagle_logits_desc* desc, const void* logits, const int32_t* draft_tokens, const int32_t* tree_parent,
                             float* out, eagle_stream_t stream);

/*
 * ---------------------------------------------------------------------------------------------------------------------
 * A cache in 8 bits with a scale for each block of slots and head; attention with a sliding window and a few first slots that stay
 * visible; sampling with temperature, top-k, top-p and min-p.
 */

/*
 * The block-scaled cache.  The calls below take an eagle_kv_store whose k and v hold e4m3 codes (as for eagle_tree_verify_attn_fp8,
 * head_dim 128) together with a block size in their descriptor: BS = 16, 32, 64 or 128 slots of one KV head share one fp32 scale,
 *     key = value(code) * k_scale[block],  value = value(code) * v_scale[block].
 *   contiguous: codes [B, Hkv, kv_capacity, 128], scales [B, Hkv, kv_capacity / BS], kv_capacity a multiple of BS
 *   paged:      codes [num_pages, Hkv, page_size, 128], scales [num_pages, Hkv, page_size / BS], page_size a multiple of BS
 * The range of a sequence's keys need not be known when it starts, as it has to be with one scale per (sequence, KV head): a block's
 * scale follows what is stored in it.  The append calls write the scales although the struct declares them const.
 */
typedef struct eagle_block_desc {
  int32_t batch;                /* B, 0 .. 65535 */
  int32_t num_tokens;           /* N >= 0: rows of q, k, v and q_out (chunk form) */
  int32_t max_tree;             /* T_max <= 64 (tree form; q, k, v and q_out have B * T_max rows) */
  int32_t num_q_heads;          /* Hq >= 0 (0: only the cache is written) */
  int32_t num_kv_heads;         /* Hkv >= 1 */
  int32_t rotary_dim;           /* R: a multiple of 16, <= 128, as for eagle_rope_append */
  int32_t interleaved;          /* 0: element m turns with m + R/2; nonzero: element 2m with 2m + 1 */
  int32_t block_size;           /* BS */
  float amplitude;              /* factor on sines and cosines; 0 means 1 */
  int64_t q_stride, k_stride, v_stride;   /* as for eagle_rope_append (head_dim is 128) */
  const double* freqs;          /* device double [R / 2], radians per position */
  const int32_t* positions;     /* chunk form: device int32 [N], or NULL: a token's position is its slot */
  const int32_t* tree_sizes;    /* tree form: device int32 [B] ([1] when shared_tree is set), or NULL */
  int32_t shared_tree;          /* tree form, nonzero: tree_parent is int32 [T_max], one tree for every sequence */
  int32_t* status;              /* device int32 or NULL */
} eagle_block_desc;

/*
 * Rotary positions of new tokens, and their keys and values into a block-scaled cache, in one launch.  Rows, positions, slots, strides,
 * q_out and what is reported are those of eagle_rope_append; what differs is how keys and values are stored.  Per KV head, for keys
 * and values alike, the new tokens of a block (rotated in fp32, not rounded before) with the largest finite magnitude a need the scale
 *     s(a) = 2^e, e the least whole number from -40 to 120 with a <= 448 * 2^e       (e = -40 where nothing is finite, or all is 0).
 * A block that begins at or behind slot L_b takes it.  The block that slot L_b lies inside of holds older slots: it keeps its scale if that is
 * at least s(a), and takes s(a) otherwise, its older codes then stored again as the nearest code of value(code) * old / new.  New codes are the
 * nearest e4m3 code of x / scale in fp32 (ties to the even code, magnitudes above 448 become 448, NaN stays NaN).
 * A power of two loses nothing against a finer scale, since codes are floating-point numbers, and storing older codes again costs them
 * at most the bits that leave the bottom of the range.  An old scale has to be a normal number above 0; blocks that hold no slot of a sequence
 * in use may have any.  No block may be shared by two sequences that append.  Values above 448 * 2^60 are stored, too, but their block's scale is one that
 * eagle_window_attn reports and does not take.
 */
int eagle_block_append(const eagle_block_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                       const int32_t* seq_lens, const int32_t* token_start, eagle_stream_t stream);

/*
 * The same for the nodes of draft trees, in the layout of eagle_tree_rope_append.  All blocks that a tree's slots L_b .. L_b + n_b - 1 lie in
 * take one scale per KV head: s(a) of the whole tree, or that of the block that holds older slots where it is larger.  So the accepted
 * path is committed by eagle_tree_commit / eagle_tree_commit_paged on the codes (head_dim 64 there), as for any cache of codes: rows move as bytes
 * between blocks of one scale.
 */
int eagle_tree_block_append(const eagle_block_desc* desc, const void* q, const void* k, const void* v, void* q_out, const eagle_kv_store* kv,
                            const int32_t* seq_lens, const int32_t* tree_parent, eagle_stream_t stream);

typedef struct eagle_window_desc {
  int32_t batch;                /* B, 0 .. 65535 */
  int32_t num_tokens;           /* N >= 0: rows of q and out (chunk form) */
  int32_t max_tree;             /* T_max, 0 .. 64 (tree form; q and out have B * T_max rows); ignored by the chunk form */
  int32_t num_q_heads;          /* Hq; Hq % Hkv == 0, group size G = Hq / Hkv <= 16 */
  int32_t num_kv_heads;         /* Hkv */
  int32_t head_dim;             /* D: 64 or 128; 128 with a block-scaled cache */
  int32_t block_size;           /* 0: a bf16 cache; else the block-scaled cache's BS */
  int32_t window;               /* W: 0 for no limit; tree form: 0 or at least EAGLE_MAX_TREE, so that a node's own path is always inside */
  int32_t sinks;                /* S >= 0: the first S slots stay visible (no effect with W = 0) */
  float sm_scale;               /* softmax scale, > 0; 0 means 1/sqrt(D) */
  const int32_t* tree_sizes;    /* tree form: device int32 [B] ([1] when shared_tree is set), or NULL */
  int32_t shared_tree;          /* tree form, nonzero: tree_parent is int32 [T_max], one tree for every sequence */
  void* workspace;              /* device, 256-byte aligned, >= eagle_window_attn_workspace() bytes */
  size_t workspace_bytes;
  int32_t* status;              /* device int32 or NULL */
} eagle_window_desc;

/* Bytes of scratch one call with this descriptor, or with fewer tokens, needs: of the chunk form with max_tree = 0, else of the tree form
 * (host function, no CUDA work); 0 if the shape is unsupported. */
size_t eagle_window_attn_workspace(const eagle_window_desc* desc);

/*
 * Attention of one layer for chunks of new tokens, as eagle_chunk_attn, with a sliding window and over a cache in either form.
 * The token at position p (its slot, L_b + i) sees the key of slot j iff
 *     j <= p  and  (W = 0  or  j > p - W  or  j < S).
 * kv holds bf16 (block_size 0, no scales) or block-scaled codes.  Keys and values of slots that no token of the call sees are not used,
 * pages that hold only such slots are not read and their block-table entries may be anything: pages that a window has left behind may go back
 * to the pool.  Work is proportional to what is visible.  A sequence may have up to 2^31 - 256 slots in use, the new tokens' among them; a longer one reports
 * EAGLE_ERR_SEQ.
 *
 * Arithmetic: as for eagle_chunk_attn over bf16.  Over codes the products are fp16 (every e4m3 number is one exactly): a query row is
 * scaled by a power of two so that its largest magnitude is in [1, 2), then rounded to fp16 (half a step is 2^-12 of an element, and 2^-25 of the
 * row's largest for those below 2^-14 of it); scores take their block's scale in fp32; a probability times its block's value scale is
 * rounded to fp16 (2^-11 of it, or 2^-32 of the row's largest such product); sums are fp32.  Scales of keys have to be normal numbers above 0, those of values from 2^-60 to 2^60: another one that is visible
 * reports EAGLE_ERR_SCALE, and rows that see it may hold anything.  (The row sum drops weights below 2^-133 of the largest probability times value scale, over
 * their own value scale.  With value scales within 2^100 of one another, as all are from 2^-40 to 2^60, no weight above 2^-33 of the largest is lost; with 2^60
 * and 2^-60 in one row those below 2^-13 can be.)
 * A visible score that is NaN or +infinite makes its row NaN.  Slots past the chunk may hold anything; what holds for slots in use and for the size of scores is
 * as for eagle_chunk_attn (values of slots in use have to be finite), with NaN codes in the place of values that are not.
 * Device-detected errors, rows outside every sequence, time-outs, launches and the rule N <= B are those of eagle_chunk_attn, too.
 */
int eagle_window_attn(const eagle_window_desc* desc, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens,
                      const int32_t* token_start, void* out, eagle_stream_t stream);

/*
 * The same for the nodes of draft trees, in the layout of eagle_tree_verify_attn: q and out are device bf16 [B, T_max, Hq, D], node i of
 * sequence b lies in slot L_b + i, at position p = L_b + depth(i) - 1, and sees the prefix's slots j < L_b with (W = 0 or j > p - W or j < S), its
 * ancestors and itself.  Rows of nodes >= tree size are written as zeros.  An invalid tree reports EAGLE_ERR_TREE, a tree that does not fit
 * EAGLE_ERR_SEQ: the sequence's rows are zeros.
 */
int eagle_tree_window_attn(const eagle_window_desc* desc, const void* q, const eagle_kv_store* kv, const int32_t* seq_lens,
                           const int32_t* tree_parent, void* out, eagle_stream_t stream);

#define EAGLE_MAX_SAMPLE_VOCAB (1 << 20)

typedef struct eagle_sample_desc {
  int32_t batch;                /* B, 0 .. 65535 */
  int32_t rows;                 /* R >= 0: rows per sequence (1: plain decoding; T_max + 1: the target's rows of a draft tree) */
  int32_t vocab;                /* V, 1 .. EAGLE_MAX_SAMPLE_VOCAB */
  int32_t bf16;                 /* 0: logits are fp32; nonzero: bf16 */
  const int32_t* num_rows;      /* device int32 [B], or NULL: R rows each (clamped to [0, R]); later rows are neither read nor written */
  const float* temperature;     /* device fp32 [B] or NULL (1); a temperature that is not above 0 is greedy */
  const int32_t* top_k;         /* device int32 [B] or NULL (off); k <= 0 or >= V is off */
  const float* top_p;           /* device fp32 [B] or NULL (off); 1 or more, and NaN, is off */
  const float* min_p;           /* device fp32 [B] or NULL (off); 0 or less, and NaN, is off */
  int32_t* status;              /* device int32 or NULL */
} eagle_sample_desc;

/*
 * Sampling with temperature, top-k, top-p and min-p: a token per row, and / or the distribution that it is drawn from.  The rows are those that
 * eagle_tree_logits_adjust leaves (or bf16 rows of the output layer); the distributions are what eagle_tree_accept takes as target_probs
 * and draft_probs and eagle_tree_expand as draft_probs, so that acceptance stays exact under these filters (Algorithm 1 returns exactly the
 * distribution that it is given).
 *
 *   logits   device fp32 or bf16 [B, R, V]
 *   uniforms device fp32 [B, R] in [0, 1), or NULL with tokens NULL
 *   tokens   device int32 [B, R] or NULL
 *   probs    device fp32 [B, R, V] or NULL; may not be `logits`
 *
 * With w(v) = exp((z(v) - max z) / temperature) and the tokens in descending order of z, equal ones in ascending order of their id:
 *   top-k   the first k tokens stay
 *   top-p   of these, a token stays if the w of those before it sum to less than p times the sum of all of these (the first always does)
 *   min-p   of these, those with w >= min(min_p, 1) stay
 * probs are w over the sum of what stays, 0 elsewhere; the token is the smallest v with sum_{x <= v} w(x) > u times that sum, over what
 * stays, in ascending order of the id.  A greedy row keeps the first token alone.  NaN logits count as -infinity; where some are +infinity these
 * share the mass.  A row without any value above -infinity reports EAGLE_ERR_ROW: token -1, probs 0.
 *
 * Orders are exact; w is taken in fp64 (relative error below 2^-45 for w of 2^-47 and more, which are those that sums see, and below 2^-41 down to 2^-980; smaller
 * ones count as 0) and summed as integers of at most 2^-46 of the largest w (V <= 2^17; 2^-43 at
 * V = 2^20), so results do not depend on how the work is split, and a decision can differ from the definition only where a boundary is nearer than
 * 1e-9 (1e-7 at V = 2^20) of the largest w at the worst, 1e-10 as a rule.  One launch; no workspace.
 */
int eagle_sample(const eagle_sample_desc* desc, const void* logits, const float* uniforms, int32_t* tokens, float* probs, eagle_stream_t stream);

/* Human-readable name of a return / status code (host function; never NULL). */
const char* eagle_status_string(int code);

/* Number of kernels this library has launched in this process so far (host counter, for accounting). */
uint64_t eagle_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* EAGLE_VERIFY_H_ */
