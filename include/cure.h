/*
 * cure.h — C ABI of the CURE repair-verify step on one GB300 (sm_103a).
 *
 * CURE ("Local Uncertainty Repair for Block-Parallel Speculative Decoding")
 * repairs a block-parallel draft at its low-margin positions and verifies the
 * draft and the repairs in one tree pass.  One decoding step of the method is
 * split into five calls (a sixth replaces the greedy argmax when verifying at
 * a temperature), each one CUDA kernel (or two) on the caller's stream:
 *
 *   cure_score_draft  Sec. 3.3, Eq. (2)     top-k ids, margin, top-1 log-prob
 *   cure_build_tree   Sec. 3.1 Eq. (1),     UFP gate + budgeted selection,
 *                     Sec. 3.3, 3.4         flattened repair tree + ancestor mask
 *   cure_tree_attn    Sec. 3.2, 3.4, 3.5    tree-masked GQA attention
 *   cure_accept       Sec. 3.5 Eq. (4)      target argmax + longest accepted path
 *   cure_lm_head_argmax Sec. 3.5, 4.1       the target's argmax per node straight from
 *                                           its hidden state (LM head + argmax fused)
 *   cure_sample_target Sec. 2 (T > 0)       the target's sampled token per node, for
 *                                           stochastic verification with cure_accept
 *   cure_resync_kv    Sec. 3.5, Alg. 1      write the path into the KV cache,
 *                                           realign the draft state
 *
 * Around the step, for the target model's own attention layers:
 *   cure_rope_qkv     Sec. 3.2, 3.4         head norms and rotary rotation of the tree's rows
 *                                           at their positions, as cure_tree_attn takes them
 *   cure_append_kv    Alg. 1 (input)        the same for prompt rows, K and V into the cache
 *   cure_prompt_attn  Alg. 1 (input)        causal attention of prompt rows over the cache
 * Each with several positions a token (cure_rope_qkv_axes, cure_append_kv_axes), and over a cache
 * held in 8 bits (cure_append_kv8, cure_prompt_attn8, cure_tree_attn8, cure_save_kv8,
 * cure_restore_kv8, cure_resync_kv8).
 *
 * Conventions shared by every call
 *  - Every pointer argument is a DEVICE pointer unless stated otherwise; the
 *    caller owns all memory (inputs, outputs, caches, workspace).  The library
 *    never allocates device memory.
 *  - `stream` is a cudaStream_t (NULL = the legacy default stream).  Calls are
 *    asynchronous; nothing waits on the host.
 *  - Arguments the host can check (sizes, null pointers, alignment) are
 *    checked before anything is launched; a bad one returns
 *    CURE_ERR_INVALID_ARG (or CURE_ERR_UNSUPPORTED for a valid but
 *    unimplemented shape) and launches nothing.
 *  - Conditions only the device can see (a cache slot past the capacity, a
 *    missing or out-of-range page id, a node count past n_max) make the kernel
 *    skip the offending access and raise a bit in a device error word;
 *    cure_device_error() reads and clears it.
 *  - Tensors are row-major, innermost dimension last.  bf16 is IEEE bfloat16.
 *  - Tie rule everywhere: equal values rank the lower index first.
 *  - Padding: entries of per-node outputs at j >= n_nodes[b] are -1 (ints) or
 *    0 (ancestor words); output rows of cure_tree_attn at j >= n_nodes[b] are
 *    left unwritten.
 */
#ifndef CURE_H_
#define CURE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CURE_OK = 0,
  CURE_ERR_INVALID_ARG = 1,   /* a host-checkable argument is wrong; nothing launched */
  CURE_ERR_CAPACITY = 2,      /* workspace too small for the shape; nothing launched */
  CURE_ERR_CUDA = 3,          /* a CUDA runtime call or launch failed */
  CURE_ERR_DEVICE_FAULT = 4,  /* returned by cure_device_error when a kernel flagged bad data */
  CURE_ERR_UNSUPPORTED = 5    /* valid but not implemented (e.g. head_dim != 128) */
} cure_status;

/* Bits of the device error word (cure_device_error). */
#define CURE_DEVERR_PAGE      0x1   /* block_table entry < 0 or >= num_pages */
#define CURE_DEVERR_SLOT      0x2   /* cache slot beyond the per-sequence capacity */
#define CURE_DEVERR_NODES     0x4   /* n_nodes[b] outside [1, n_max] or a bad path/parent index */
#define CURE_DEVERR_TOKEN     0x8   /* a token id outside [0, vocab) where one is required */
#define CURE_DEVERR_TIMEOUT   0x10  /* a pipeline wait inside a kernel gave up (the CTA drained and left) */
#define CURE_DEVERR_ALIGN     0x20  /* a kernel found its shared memory misaligned and did nothing */

/* Tree-construction parameters (Sec. 3.3 / 3.4 and Eq. 1). */
typedef struct {
  int32_t batch;         /* B, sequences */
  int32_t block;         /* K, draft positions per block, 1..32 */
  int32_t topk;          /* ranked candidates stored per position by cure_score_draft, 2..8 */
  float tau;             /* margin threshold: position i is a UFP iff margin_i < tau (float32 compare) */
  int32_t budget;        /* R, maximum repair nodes per sequence, >= 0; n_max = 1 + K + R <= 256 */
  int32_t branches;      /* candidates per UFP counting the draft token: ranks 2..branches are
                            the alternatives; 1..topk */
  int32_t repair_depth;  /* 1: alternative leaf; 2: alternative + its re-drafted successor */
  int32_t max_ufp;       /* 0 = no cap; else only the max_ufp lowest-margin UFPs are repaired */
  float margin_scale;    /* s of Eq. (3); 0 = fixed budget (every UFP offers branches-1
                            alternatives); > 0 and finite = dynamic budget (see cure_build_tree) */
  int32_t branch_min;    /* b_min of Eq. (3), 0..branches-1 (the paper: 1); used when
                            margin_scale > 0 */
  int32_t max_depth;     /* 0 = none; else no repair node deeper than max_depth (the paper: 15) */
  int32_t beam;          /* 0 = none; else at most `beam` nodes at any depth (the paper: 5) */
} cure_tree_params;

/* KV-cache geometry (one layer). */
typedef struct {
  int32_t layout;        /* 0: contiguous [B][max_len][heads_kv][head_dim]
                            1: paged [num_pages][page_size][heads_kv][head_dim] */
  int32_t heads_kv;      /* Hkv */
  int32_t head_dim;      /* D; 128 is implemented */
  int32_t page_size;     /* paged: tokens per page: 8, 16, 32 or 64; ignored when contiguous */
  int32_t max_len;       /* contiguous: rows per sequence; paged: entries per block_table row */
  int32_t num_pages;     /* paged: pages in the pool (bounds check); ignored when contiguous */
  const int32_t* block_table; /* paged: device int32 [B][max_len] physical page ids; else NULL */
} cure_kv_desc;

/*
 * Stage 1 — draft scores (Sec. 3.3, Eq. 2; Alg. 1 first step).
 * For each of `rows` rows (B*K draft positions) of `vocab` bf16 logits:
 *   top_ids[r][0..topk)  ids ranked by (logit desc, id asc)        int32
 *   top_vals[r][0..topk) their logits widened to float32            float
 *   margin[r]            top_vals[r][0] - top_vals[r][1] (Eq. 2; the log-softmax
 *                        normaliser cancels, so it is also the log-prob gap)
 *   logp1[r]             top_vals[r][0] - logsumexp(row)  (float32 accumulation)
 * logits: bf16 [rows][vocab], any alignment.  2 <= topk <= 8, topk <= vocab.
 * margin and logp1 may be NULL.  NaN logits are not supported (ranking undefined);
 * -inf is allowed.
 */
cure_status cure_score_draft(const void* logits, int32_t rows, int32_t vocab, int32_t topk,
                             int32_t* top_ids, float* top_vals, float* margin, float* logp1,
                             void* stream);

/*
 * Stages 2+3 — UFP selection and repair-tree construction (Sec. 3.1 Eq. 1,
 * Sec. 3.3, Sec. 3.4; Alg. 1 loop).  One warp per sequence.
 * Inputs:  top_ids int32 [B][K][topk] and margin float [B][K] (from stage 1),
 *          root_tok int32 [B] (last committed token), cache_len int32 [B] (L_b),
 *          redraft int32 [B][K][branches-1]: the successor token of each
 *          alternative (rank r at index r-2) when repair_depth == 2 (NULL
 *          otherwise).
 * Selection: positions with margin < tau, in ascending (margin, position)
 *   order; each alternative (i, r), r = 2..branches, costs min(repair_depth, K-i)
 *   nodes and is admitted while the repair nodes stay <= budget (an alternative
 *   that does not fit is skipped).
 * Dynamic branch budget (Sec. 3.3, Eq. 3), when margin_scale s > 0: UFP i
 *   offers the b_i alternatives of ranks 2..b_i+1 instead, with
 *   u_i = clip(1 - m_i / s, 0, 1) and
 *   b_i = clip(round(b_min + u_i (b_max - b_min)), b_min, b_max),
 *   b_min = branch_min, b_max = branches - 1; the quotient, the difference, the
 *   product and the sum are float32 operations rounded to nearest and round()
 *   takes halves away from zero.  The paper's (b_min, b_max) = (1, 5) is
 *   branch_min = 1, branches = 6 (topk >= 6).
 * Structural caps (Sec. 3.3, 3.4; repair branches only, branch 0 is never
 *   pruned): with max_depth > 0 an alternative at depth i+1 > max_depth is not
 *   spawned and a successor at depth i+2 > max_depth is dropped (the
 *   alternative then costs one node); with beam > 0 an alternative is admitted
 *   only while every depth it occupies holds fewer than `beam` nodes, the chain
 *   node included (one that does not fit is skipped, like the budget).
 * Tree (n_max = 1 + K + budget nodes per sequence, W = ceil(n_max/64)):
 *   node 0 root (root_tok, depth 0); nodes 1..K branch 0 (top-1 ids, chained);
 *   then repair nodes in (i, r, depth) order: the rank-r id at position i as a
 *   child of node i, and with depth-2 repairs (i < K-1) its successor.
 * Outputs: n_nodes [B]; tok, pos (= L_b + depth), parent (-1 for the root),
 *   depth: int32 [B][n_max]; anc uint64 [B][n_max][W] (bit a of node j set iff a
 *   is on the root-to-j path, j included); ufp_pos int32 [B][K] (repaired
 *   positions in selection order, then -1); n_ufp int32 [B].
 * `p` is a HOST pointer.
 */
cure_status cure_build_tree(const cure_tree_params* p, const int32_t* top_ids, const float* margin,
                            const int32_t* root_tok, const int32_t* cache_len, const int32_t* redraft,
                            int32_t* n_nodes, int32_t* tok, int32_t* pos, int32_t* parent,
                            int32_t* depth, uint64_t* anc, int32_t* ufp_pos, int32_t* n_ufp,
                            void* stream);

/*
 * Stage 4 — tree attention for one layer (Sec. 3.2 / 3.4 / 3.5: the target
 * verifies every tree path in one pass).  For sequence b, node j < n_nodes[b],
 * query head h (kv head h / (heads_q / heads_kv)):
 *   out[b][j][h] = softmax(scale * q k^T) v over the cached keys 0..L_b-1 and
 *                  the tree keys a with bit a of anc[b][j] set (0 where that
 *                  leaves no key).
 * q, out: bf16 [B][n_max][heads_q][D]; tree_k, tree_v: bf16 [B][n_max][heads_kv][D]
 * (this step's target keys/values of the tree tokens); k_cache, v_cache: one
 * layer in the layout of `kv` (a HOST pointer).
 * In-place layout: tree_k = tree_v = NULL means the tree rows were written
 * into the cache itself, node j of sequence b at slot L_b + j (a paged cache
 * then needs block_table entries up to slot L_b + n_b - 1).  The keys are then
 * one range 0..L_b+n_b-1 of the cache, in 64-key tiles; a tile past L_b
 * masks its tree part with the ancestor bits.  L_b + n_b past the capacity
 * sets CURE_DEVERR_SLOT.  Accumulation is float32; the
 * probabilities are rounded to bf16 before the PV product.  D = 128,
 * heads_q % heads_kv == 0, scale > 0 and finite (1/sqrt(D) in the paper's
 * models; otherwise CURE_ERR_INVALID_ARG), all tensor base pointers 16-byte
 * aligned.
 * workspace: device scratch of at least cure_tree_attn_workspace_size() bytes,
 * 256-byte aligned (split-KV partial results); its contents on entry do not
 * matter.  Calls that can overlap on the GPU must not share a workspace; after
 * CURE_DEVERR_TIMEOUT zero it before a captured call is replayed on it.
 * The kernel is launched as a programmatic dependent launch: it starts its
 * set-up while the previous kernel on the stream finishes and waits for that
 * kernel before reading any argument, so stream order is kept.
 */
cure_status cure_tree_attn(const void* q, const void* tree_k, const void* tree_v,
                           const void* k_cache, const void* v_cache, const cure_kv_desc* kv,
                           const int32_t* cache_len, const int32_t* n_nodes, const uint64_t* anc,
                           int32_t batch, int32_t n_max, int32_t heads_q, float scale, void* out,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace cure_tree_attn needs for this shape (0 on a bad argument). */
size_t cure_tree_attn_workspace_size(int32_t batch, int32_t n_max, int32_t heads_q,
                                     const cure_kv_desc* kv);

/* Size of the static device scratch behind cure_tree_attn_noalloc (64 MiB). */
#define CURE_NOALLOC_SCRATCH_BYTES (64u * 1024u * 1024u)

/*
 * cure_tree_attn without a caller-supplied workspace.  The paper has no
 * counterpart: this entry point exists for callers that cannot allocate
 * device memory — for instance a plugin in an inference server whose
 * allocator owns (and has nearly filled) HBM, or a host framework that hands
 * an extension only its input and output buffers.  It computes exactly what
 * cure_tree_attn computes, with the same arguments minus the workspace; the
 * split-KV partial results go to a 64 MiB array in the library's own static
 * device memory, which every GPU that loads that part of the library keeps
 * until the process exits.  It allocates nothing and calls no allocator.
 *  - Shapes whose cure_tree_attn_workspace_size() is larger than
 *    CURE_NOALLOC_SCRATCH_BYTES return CURE_ERR_CAPACITY and launch nothing.
 *  - The first call on each device looks up the device address of the array
 *    (cudaGetSymbolAddress); make that first call before any stream capture.
 *  - All calls share the one array and it keeps the last call's contents.
 *    Nothing in it needs to start at zero (each call writes every partial it
 *    reads), but two calls that can overlap on the GPU — on unordered streams
 *    or from different host threads — race on it and corrupt each other's
 *    outputs: order such calls on one stream.
 */
cure_status cure_tree_attn_noalloc(const void* q, const void* tree_k, const void* tree_v,
                                   const void* k_cache, const void* v_cache,
                                   const cure_kv_desc* kv, const int32_t* cache_len,
                                   const int32_t* n_nodes, const uint64_t* anc, int32_t batch,
                                   int32_t n_max, int32_t heads_q, float scale, void* out,
                                   void* stream);

/*
 * Stage 5 — acceptance walk (Sec. 3.5 Eq. 4, greedy decoding Sec. 4.1).
 * targ[b][j] = argmax_v target_logits[b][j][v] (lowest id on ties) for
 * j < n_nodes[b] (rows beyond are not read; their targ is -1).  Pass
 * target_logits (bf16 [B][n_max][vocab]) to have the argmax computed, or
 * target_logits = NULL and targ already filled with the target's tokens.
 * A non-root node j is verified when tok[j] == targ[parent[j]]; it is accepted
 * when every non-root node on its path is verified.  pi* = the deepest accepted
 * node (lowest index on ties), a = its depth.
 * Outputs (int32): accept_len [B] = a; best_node [B];
 *   path_nodes [B][K+2]: path node at each depth 0..a, then -1;
 *   out_tokens [B][K+2]: path tokens at depths 1..a, then targ[best] (the
 *                        token after the path), then -1;
 *   diverge_depth [B]: shallowest path depth whose node is a repair node
 *                      (index > K), or -1 when branch 0 wins.
 */
/*
 * Stage 5, stochastic verification (temperature > 0).  Speculative decoding is
 * lossless sampling from the target (Sec. 2); the paper's runs are greedy
 * (Sec. 4.1), where cure_accept's argmax fills targ.  This call fills targ
 * with samples instead, and cure_accept(target_logits = NULL, targ) then walks
 * the tree unchanged: a child is accepted when its token equals its parent's
 * sample.  Each sample is drawn independently of the drafted children, so the
 * emitted tokens follow the target's distribution.
 * For j < n_nodes[b]: targ[b][j] = the first id v with
 *   sum_{w <= v} softmax(target_logits[b][j] / temperature)_w > u,
 * u = uniforms[b][j] (float [B][n_max], clamped to [0, 1)), from float32
 * partial sums: within their rounding of the exact inverse CDF, never an id
 * of probability 0.  The probabilities are formed as 2^((l - l_max) log2(e)/T),
 * which cannot overflow: at temperatures so small that every logit below the
 * maximum underflows, the draw picks among the ids that hold the maximum
 * (the limit T -> 0).  A row of -inf logits gives 0; rows j >= n_nodes[b]
 * get -1.  target_logits bf16 [B][n_max][vocab], 2-byte aligned; temperature
 * > 0 with log2(e)/temperature finite (T >= about 4.2e-39, else
 * CURE_ERR_INVALID_ARG); 1 <= n_max <= 256.  One CTA of four warps per row,
 * each warp streaming a contiguous quarter of it.
 */
cure_status cure_sample_target(const void* target_logits, const float* uniforms, float temperature,
                               int32_t batch, int32_t n_max, int32_t vocab, const int32_t* n_nodes,
                               int32_t* targ, void* stream);

/*
 * Stage 5 fused with the target's LM head (Sec. 3.5, Eq. 4: the target scores
 * every tree node in one pass; greedy decoding, Sec. 4.1).  For each of `rows`
 * final hidden states (the tree nodes of all sequences, packed):
 *   targ[out_index ? out_index[r] : r] = the first v maximising hidden[r] . w_lm[v]
 * The contraction runs on the tensor cores with float32 accumulation and the
 * argmax is taken in its epilogue: the rows x vocab logits are never written.
 * Two ids whose logits lie within float32 accumulation error of each other may
 * be ranked either way (d_model products per logit; the bound is about
 * d_model/16 roundings of 2^-23 relative to sum_k |hidden[r][k] w_lm[v][k]|).
 * Then call cure_accept(target_logits = NULL, targ).
 * hidden: bf16 [rows][d_model]; w_lm: bf16 [vocab][d_model] (row-major, the
 * layout of an LM-head weight); both 16-byte aligned.  d_model a multiple of
 * 64 (else CURE_ERR_UNSUPPORTED).  out_index: int32 [rows] (NULL: identity),
 * e.g. b * n_max + j to fill cure_accept's targ [B][n_max] from rows packed over
 * the valid nodes; entries of targ that no row maps to are left unwritten.
 * workspace: at least cure_lm_head_workspace_size(rows, vocab) bytes (computed
 * for the current device), 256-byte aligned, contents on entry do not matter;
 * calls that can overlap on the GPU must not share one.  Two kernels: the
 * persistent tcgen05 contraction (one CTA per SM) and a per-row merge.
 */
cure_status cure_lm_head_argmax(const void* hidden, const void* w_lm, int32_t rows, int32_t d_model,
                                int32_t vocab, const int32_t* out_index, int32_t* targ, void* workspace,
                                size_t workspace_bytes, void* stream);

/* Bytes of workspace cure_lm_head_argmax needs on the current device (0 on a bad argument). */
size_t cure_lm_head_workspace_size(int32_t rows, int32_t vocab);

cure_status cure_accept(const void* target_logits, int32_t* targ, int32_t batch, int32_t n_max,
                        int32_t vocab, int32_t block, const int32_t* n_nodes, const int32_t* tok,
                        const int32_t* parent, const int32_t* depth, const uint64_t* anc,
                        int32_t* accept_len, int32_t* best_node, int32_t* path_nodes,
                        int32_t* out_tokens, int32_t* diverge_depth, void* stream);

/*
 * Stage 6 — repair resynchronisation (Sec. 3.5, Alg. 1 last step).
 * For every layer l and sequence b, the K/V rows of the accepted path's nodes
 * at depths 0..a are copied from tree_k/tree_v (bf16 [layers][B][n_max][Hkv][D])
 * into cache slots L_b..L_b+a of k_caches[l]/v_caches[l] (layout `kv`).
 * In-place layout (tree_k = tree_v = NULL, see cure_tree_attn): node j's rows
 * are read from cache slot L_b + j, so the rows of branch-0 nodes (j = depth)
 * are already in place and only the repair nodes past the divergence depth
 * are copied (nothing when branch 0 wins).
 * Then cache_len_out[b] = L_b + a + 1, draft_valid_len[b] = L_b + d when a
 * repair path wins at divergence depth d (else L_b + a + 1), and
 * replay_tokens[b] (int32 [B][K+2]) = the path tokens at depths d..a followed by
 * the token after the path (only that token on branch-0 wins), then -1;
 * n_replay[b] its length.  cache_len_out may alias cache_len_in; no other
 * output may overlap an input (the copies and the replay list are written by
 * one kernel, the lengths after it only when cache_len_out aliases).
 * k_caches, v_caches: HOST arrays of `layers` device pointers (layers <= 128).
 */
cure_status cure_resync_kv(int32_t layers, void* const* k_caches, void* const* v_caches,
                           const cure_kv_desc* kv, const void* tree_k, const void* tree_v,
                           int32_t batch, int32_t n_max, int32_t block, const int32_t* path_nodes,
                           const int32_t* accept_len, const int32_t* diverge_depth,
                           const int32_t* out_tokens, const int32_t* cache_len_in,
                           int32_t* cache_len_out, int32_t* draft_valid_len,
                           int32_t* replay_tokens, int32_t* n_replay, void* stream);

/*
 * The rotary rotation of a head (a HOST struct, made by cure_rope_init or
 * cure_rope_init_freqs).  Of a head's first rot_dim values, pair i (0 <= i <
 * rot_dim / 2) at position p turns by the angle p * f_i:
 *   a' = A (a cos(p f_i) - b sin(p f_i)),  b' = A (b cos(p f_i) + a sin(p f_i))
 * with A = amplitude and the pair (a, b) = values (i, i + rot_dim / 2) in style 0
 * (half), values (2i, 2i + 1) in style 1 (interleaved); the other values pass
 * through.
 */
typedef struct {
  int32_t style;        /* 0: half, 1: interleaved */
  int32_t rot_dim;      /* values of a head that are rotated: 0 (none) or a multiple of 16 up to 128 */
  float amplitude;      /* A; 1 without scaling for long contexts that asks for another */
  int32_t reserved;     /* 0 */
  uint64_t turns[64];   /* f_i / (2 pi) modulo 1, in units of 2^-64 */
} cure_rope;

/* Frequencies scaled for longer contexts than a model was trained on. */
typedef struct {
  int32_t kind;         /* 0: none
                           1 linear: f_i / factor
                           2 base:   f_i of the base  base * factor^(r / (r - 2)), r = rot_dim
                           3 bands:  with t_i = f_i original / (2 pi) turns within the original
                                     context: f_i where t_i >= high, f_i / factor where t_i <= low,
                                     between them g f_i + (1 - g) f_i / factor, g = (t_i - low) / (high - low)
                           4 ramp:   (1 - g) f_i + g f_i / factor, g = clip((i - i_0) / (i_1 - i_0), 0, 1),
                                     i_0 = max(floor(d(high)), 0), i_1 = min(ceil(d(low)), r - 1) (i_0 + 0.001 if
                                     that is not above i_0), d(t) = r ln(original / (2 pi t)) / (2 ln base) */
  int32_t reserved;     /* 0 */
  double factor;        /* > 0 */
  double low, high;     /* bands, ramp: turns, 0 < low < high */
  double original;      /* bands, ramp: the original context length in tokens, > 0 */
} cure_rope_scaling;

/*
 * Fills *out with the frequencies f_i = base^(-2i / rot_dim), scaled as `scaling`
 * says (NULL: not at all), in 64-bit arithmetic on the host.  base > 1 and finite
 * (CURE_ERR_INVALID_ARG otherwise, as for a rot_dim that is odd or outside
 * 2..128); rot_dim a multiple of 16 (CURE_ERR_UNSUPPORTED otherwise).
 */
cure_status cure_rope_init(cure_rope* out, int32_t style, int32_t rot_dim, double base,
                           const cure_rope_scaling* scaling, float amplitude);

/* The same from the caller's own frequencies: `freqs` is a HOST array of rot_dim / 2
 * finite values, in radians per position. */
cure_status cure_rope_init_freqs(cure_rope* out, int32_t style, int32_t rot_dim, const double* freqs,
                                 float amplitude);

/*
 * Per-head norms and the rotation, from the rows of a layer's Q/K/V projection
 * to the rows that cure_tree_attn takes (Sec. 3.2, 3.4: the target scores the
 * tree's nodes at their own positions).  For row r with pos[r] >= 0, every head
 * x of q and k:
 *   y = x * w / sqrt(mean(x^2) + eps)   (w = q_norm or k_norm, bf16 [D]; NULL: y = x)
 * then y is rotated to position pos[r] by `rope` (a HOST pointer; NULL: not at
 * all); heads of v are copied.  All in float32, rounded to bf16 once.  Rows with
 * pos[r] < 0 (the padding of cure_build_tree's `pos`) are left out, their outputs unwritten.
 * q [rows][heads_q][D], k and v [rows][heads_kv][D], bf16; row r of a tensor
 * starts ld values after row r - 1 (its heads lie end to end), so that the three
 * may be parts of one projection's rows.  A tensor and its output may both be
 * NULL (left out).  An output may be its input (same address and stride); any
 * other overlap is not allowed.  head_dim = 128; all pointers 16-byte aligned,
 * strides multiples of 8 values that hold a row's heads.  An angle is off by less
 * than 2^-25 of a turn (its fraction is rounded to a float at the end) and p times
 * what turns[i] is off by: below 2^-53 for the plain frequencies, as they are made
 * from 64-bit floats (p < 2^28: together below 2^-24; any p: below 2^-21).
 * eps >= 0 and finite.
 */
cure_status cure_rope_qkv(const void* q, const void* k, const void* v, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                          int32_t rows, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const int32_t* pos,
                          const cure_rope* rope, const void* q_norm, const void* k_norm, float eps, void* q_out,
                          void* k_out, void* v_out, int64_t ld_q_out, int64_t ld_k_out, int64_t ld_v_out,
                          void* stream);

/*
 * The same for packed rows whose K and V go into the cache (prompts, chunks of
 * prompts, single new tokens).  Sequence b has the rows row_start[b] ..
 * row_start[b+1] - 1 (device int32 [batch + 1], ascending; equal: none), and its
 * i-th row's K and V are written to slot cache_len[b] + i of its cache (one
 * layer, layout `kv`), behind the cache_len[b] tokens that it holds.  A row's
 * position is its slot, or pos[row] when `pos` is given (device int32 [rows]);
 * pos[row] < 0 leaves the row out.  With row_start = 0, n_max, 2 n_max, .. and
 * the tree's `pos` that is the in-place layout of cure_tree_attn.
 * q may be NULL (then q_out is not used); otherwise its rows go to q_out as in
 * cure_rope_qkv.  cache_len is not advanced: every layer of a model is appended
 * at the same lengths.  Rows outside row_start[0] .. row_start[batch] - 1 are
 * left out.  A slot past the capacity (CURE_DEVERR_SLOT) and a missing or bad page
 * (CURE_DEVERR_PAGE) leave the rows concerned out.  Where row_start does not ascend
 * from 0 or above, a row is written for a sequence whose range holds it or left out:
 * with CURE_DEVERR_NODES if entries of row_start lie on both sides of it, without
 * if it stands before row_start[0] or behind every other entry (cure_prompt_attn
 * reports every such sequence).  q, k, v, the norms, strides and alignment as in
 * cure_rope_qkv; caches 16-byte aligned; the inputs may not overlap the caches.
 * No two rows of a call may have the same slot of the same page.
 */
cure_status cure_append_kv(const void* q, const void* k, const void* v, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                           int32_t rows, int32_t heads_q, int32_t batch, const int32_t* row_start,
                           const int32_t* cache_len, const int32_t* pos, const cure_kv_desc* kv, void* k_cache,
                           void* v_cache, const cure_rope* rope, const void* q_norm, const void* k_norm, float eps,
                           void* q_out, int64_t ld_q_out, void* stream);

/*
 * Causal attention of packed rows over the cache, one layer (Alg. 1's input: the
 * target reads a prompt, a further chunk of one, or a single token, before the
 * next step).  Sequence b has the rows row_start[b] .. row_start[b+1] - 1
 * (device int32 [batch + 1], ascending; equal: none), which stand at positions
 * cache_len[b], cache_len[b] + 1, .. and whose K and V are in the cache at these
 * slots already (cure_append_kv).  For its i-th row r, head h (kv head
 * h / (heads_q / heads_kv)):
 *   out[r][h] = softmax(scale * q k^T) v over the cached keys 0 .. cache_len[b] + i
 * q, out: bf16 [rows][heads_q][D], out not overlapping any input; k_cache,
 * v_cache: one layer in the layout of `kv` (a HOST pointer).  Accumulation is
 * float32, with a rounding of up to 2^-24 of the sum for each 128 keys; the
 * probabilities are rounded to bf16 before the PV product.  A sequence of more than
 * 2^25 keys may be given up with CURE_DEVERR_TIMEOUT: what one CTA has to do of it
 * can outlast the limit of the kernel's waits.  What lies in the cache behind a
 * sequence's last key does not matter; the V rows of the sequence's own keys must be
 * finite (a key that a row does not see weighs 0 in the product, not nothing).  Rows
 * outside row_start[0] .. row_start[batch] - 1 are left unwritten, and so are the
 * rows of a sequence that does not fit its capacity (CURE_DEVERR_SLOT) or whose
 * row_start does not ascend within 0 .. rows (CURE_DEVERR_NODES).  A missing or bad
 * page counts as zeros (CURE_DEVERR_PAGE).  batch <= 256, rows <= 2^22, D = 128,
 * heads_q / heads_kv <= 128, scale > 0 and finite; all base pointers 16-byte
 * aligned.
 * workspace: device scratch of at least cure_prompt_attn_workspace_size() bytes,
 * 256-byte aligned (what parts of a long row group hand to the part that joins
 * them); its contents on entry do not matter.  Calls that can overlap on the GPU
 * must not share a workspace, captured ones included; after CURE_DEVERR_TIMEOUT zero
 * it before a captured call is replayed on it.  The same call on the same device
 * gives the same bits, call after call.  Where a long row group is cut into parts
 * depends on the other sequences of the batch and on the number of SMs, and a
 * row's last bits on where: it may differ within the rounding above between one
 * batch and another.
 */
cure_status cure_prompt_attn(const void* q, const void* k_cache, const void* v_cache, const cure_kv_desc* kv,
                             const int32_t* row_start, const int32_t* cache_len, int32_t rows, int32_t batch,
                             int32_t heads_q, float scale, void* out, void* workspace, size_t workspace_bytes,
                             void* stream);

/* Bytes of workspace cure_prompt_attn needs for this shape on the current device (0 on a bad argument). */
size_t cure_prompt_attn_workspace_size(int32_t rows, int32_t batch, int32_t heads_q, const cure_kv_desc* kv);

/*
 * Several positions a token (time, height and width of an image's or a video's
 * patches): pair i of a head turns by the angle p[axis[i]] * f_i.  A HOST struct.
 */
typedef struct {
  int32_t axes;         /* 1 .. 8 */
  int32_t reserved;     /* 0 */
  uint8_t axis[64];     /* 0 .. axes - 1: the axis whose position pair i turns by (read for i < rot_dim / 2) */
} cure_rope_axes;

/*
 * cure_rope_qkv and cure_append_kv with a position on each of several axes: pos is
 * device int32 [axes][rows], and a row is left out where any of its positions is
 * negative.  axes (a HOST pointer) NULL: one axis, exactly as those calls; else pos must
 * be given (cure_append_kv_axes: the slots are cache_len[b] + i as ever).
 */
cure_status cure_rope_qkv_axes(const void* q, const void* k, const void* v, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                               int32_t rows, int32_t heads_q, int32_t heads_kv, int32_t head_dim, const int32_t* pos,
                               const cure_rope_axes* axes, const cure_rope* rope, const void* q_norm,
                               const void* k_norm, float eps, void* q_out, void* k_out, void* v_out,
                               int64_t ld_q_out, int64_t ld_k_out, int64_t ld_v_out, void* stream);
cure_status cure_append_kv_axes(const void* q, const void* k, const void* v, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                int32_t rows, int32_t heads_q, int32_t batch, const int32_t* row_start,
                                const int32_t* cache_len, const int32_t* pos, const cure_rope_axes* axes,
                                const cure_kv_desc* kv, void* k_cache, void* v_cache, const cure_rope* rope,
                                const void* q_norm, const void* k_norm, float eps, void* q_out, int64_t ld_q_out,
                                void* stream);

/*
 * A cache held in 8 bits.  K and V of a layer lie as `kv` says, with e4m3 codes (one
 * byte: sign, 4 bits of exponent, 3 of mantissa; 448 at most, no infinity) in the place
 * of bf16 values, and a float scale for each block of CURE_KV8_BLOCK slots and head:
 *   k_scale, v_scale: [batch][ceil(max_len / 16)][heads_kv] (contiguous),
 *                     [num_pages][page_size / 16][heads_kv] (paged)
 *   value = code * scale
 * Pages hold 16, 32 or 64 tokens (CURE_ERR_UNSUPPORTED otherwise).  The calls that write
 * choose for a block s = 2^e, the least with |x| <= 448 s for every value x that it
 * then holds (2^-40 <= s <= 2^40; s = 2^-40 for a block of zeros), and the code nearest
 * to x / s (ties to even; values beyond 448 s saturate, a NaN stays one, and counts for
 * nothing in s).  What a block held before, its slots below cache_len[b], is
 * expressed anew where s changes: exactly, but for values below 2^-6 s, which are
 * rounded to steps of 2^-9 s (beside an infinity, s = 2^40, they are lost).  That
 * stays when s falls again: around rows that may not stay, as a tree's, what is held
 * is kept by cure_save_kv8 and cure_restore_kv8.  Slots of the block that hold nothing
 * may change their meaning with its scale.
 */
#define CURE_KV8_BLOCK 16

/*
 * cure_append_kv (cure_append_kv_axes) into a cache in 8 bits.  Arguments, and which rows
 * are left out with which error, are theirs; all values are computed in float32 and
 * rounded once.  A row that is left out does not count for its block's scale; one with
 * pos < 0 among others leaves its slot without meaning.  Caches 16-byte aligned, scales 4-byte.  No two rows of a call may lie in the
 * same block of the same page, unless they are of one sequence.  row_start must
 * ascend: where it does not, rows are left out with CURE_DEVERR_NODES, or written
 * for a sequence whose range holds them.
 */
cure_status cure_append_kv8(const void* q, const void* k, const void* v, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                            int32_t rows, int32_t heads_q, int32_t batch, const int32_t* row_start,
                            const int32_t* cache_len, const int32_t* pos, const cure_rope_axes* axes,
                            const cure_kv_desc* kv, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                            const cure_rope* rope, const void* q_norm, const void* k_norm, float eps, void* q_out,
                            int64_t ld_q_out, void* stream);

/*
 * cure_prompt_attn over a cache in 8 bits: the same formula with k = code * scale, and
 * the same rows, limits, errors and workspace rules.  Any scales from 2^-40 to 2^40
 * will do, not only powers of two; others (NaN, too) count as the nearer of those two.
 * Scores: q in two e4m3 parts, which hold it but for 2^-17 of its row's largest value
 * (2^-10 / 224 in the parts' units), products of e4m3 in float32; of single tokens and
 * the like (up to 16 / (heads_q / heads_kv) rows a sequence on average) q in fp16 under a
 * power of two a row, but for 2^-32 of the row's largest value, products in float32.  A probability times its block's scale is
 * rounded to fp16, by up to 2^-11 of itself, or 2^-32 of the row's largest such term.
 * q must be finite, and V's codes in a sequence's own slots must not be NaN (K's may be
 * where a row does not see them).
 */
cure_status cure_prompt_attn8(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                              const float* v_scale, const cure_kv_desc* kv, const int32_t* row_start,
                              const int32_t* cache_len, int32_t rows, int32_t batch, int32_t heads_q, float scale,
                              void* out, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace cure_prompt_attn8 needs for this shape on the current device (0 on a bad argument). */
size_t cure_prompt_attn8_workspace_size(int32_t rows, int32_t batch, int32_t heads_q, const cure_kv_desc* kv);

/*
 * cure_tree_attn over a cache in 8 bits, in the in-place layout: node j of sequence b
 * lies in slot cache_len[b] + j (cure_append_kv8 with row_start = 0, n_max, 2 n_max, ..
 * and the tree's positions).  out[b][j][h] = softmax(scale * q k^T) v over the cached
 * keys 0 .. L_b - 1 and the nodes a with bit a of anc[b][j] set (0 where that leaves
 * no key).  Rows j >= n_nodes[b] are left unwritten, and so are the rows of a sequence
 * with n_nodes[b] outside 1 .. n_max (CURE_DEVERR_NODES) or that does not fit its capacity
 * (CURE_DEVERR_SLOT); a missing or bad page counts as zeros (CURE_DEVERR_PAGE).  n_max <= 256,
 * batch <= 256, heads_q / heads_kv <= 128.  Roundings, workspace rules, and what q and V must
 * not hold (the tree's own slots included) as for cure_prompt_attn8.
 */
cure_status cure_tree_attn8(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                            const float* v_scale, const cure_kv_desc* kv, const int32_t* cache_len,
                            const int32_t* n_nodes, const uint64_t* anc, int32_t batch, int32_t n_max,
                            int32_t heads_q, float scale, void* out, void* workspace, size_t workspace_bytes,
                            void* stream);

/* Bytes of workspace cure_tree_attn8 needs for this shape on the current device (0 on a bad argument). */
size_t cure_tree_attn8_workspace_size(int32_t batch, int32_t n_max, int32_t heads_q, const cure_kv_desc* kv);

/*
 * Rows that may not stay (a tree's in place) behind the tokens that caches in 8 bits
 * hold: of every layer, cure_save_kv8 copies what sequence b holds of the block that
 * slot cache_len[b] lies in (nothing where that is a multiple of 16, or not from 1 up to
 * the capacity) and the block's scales to `saved`; cure_restore_kv8, at the same lengths
 * and with the same pages, puts them back, to the bit.  The slots from cache_len[b] on hold
 * nothing then.  In between only rows at or behind cache_len[b] may have been
 * written.  Before a tree's cure_append_kv8, and behind the last attention that reads its
 * rows, in front of cure_resync_kv8.  k_caches .. v_scales: HOST arrays of `layers`
 * device pointers (0 .. 128 layers), none twice; saved: device memory of at least
 * cure_save_kv8_size() bytes, 16-byte aligned.
 */
cure_status cure_save_kv8(int32_t layers, void* const* k_caches, void* const* v_caches, float* const* k_scales,
                          float* const* v_scales, const cure_kv_desc* kv, int32_t batch, const int32_t* cache_len,
                          void* saved, size_t saved_bytes, void* stream);
cure_status cure_restore_kv8(int32_t layers, void* const* k_caches, void* const* v_caches, float* const* k_scales,
                             float* const* v_scales, const cure_kv_desc* kv, int32_t batch, const int32_t* cache_len,
                             const void* saved, size_t saved_bytes, void* stream);

/* Bytes that cure_save_kv8 needs for this shape (0 on a bad argument). */
size_t cure_save_kv8_size(int32_t layers, int32_t batch, const cure_kv_desc* kv);

/*
 * cure_resync_kv for caches in 8 bits: the path's rows are taken from tree_k/tree_v (bf16
 * [layers][B][n_max][Hkv][D], not NULL: what the cache holds of the tree has been rounded
 * with other rows' scales) and written as cure_append_kv8 writes rows behind the
 * cache_len_in[b] tokens that a sequence holds.  k_scales, v_scales: HOST arrays of `layers`
 * device pointers, as the caches; no cache and no scales twice (CURE_ERR_INVALID_ARG: two
 * layers that share a block would give it two scales).  Lengths and replay lists as in
 * cure_resync_kv.
 */
cure_status cure_resync_kv8(int32_t layers, void* const* k_caches, void* const* v_caches, float* const* k_scales,
                            float* const* v_scales, const cure_kv_desc* kv, const void* tree_k, const void* tree_v,
                            int32_t batch, int32_t n_max, int32_t block, const int32_t* path_nodes,
                            const int32_t* accept_len, const int32_t* diverge_depth, const int32_t* out_tokens,
                            const int32_t* cache_len_in, int32_t* cache_len_out, int32_t* draft_valid_len,
                            int32_t* replay_tokens, int32_t* n_replay, void* stream);

/* Reads and clears the device error word of the current device after
 * synchronising `stream`.  *bits receives the CURE_DEVERR_* bits (may be NULL).
 * Returns CURE_ERR_DEVICE_FAULT when any bit was set, CURE_OK otherwise. */
cure_status cure_device_error(void* stream, int32_t* bits);

/*
 * Failure-detection self-test (no counterpart in the paper): runs the
 * library's bounded pipeline waits, the two that every kernel's barrier waits go
 * through, on a barrier that nothing ever completes: the compact one for 2^20 SM
 * clock cycles, then the other with a limit of `limit_cycles` (1 .. 2^30, the
 * kernels' own limit).  Each gives up; the last raises CURE_DEVERR_TIMEOUT in the
 * device error word and returns; cure_device_error() then reports it, and the
 * context stays usable.
 */
cure_status cure_selftest_wait_timeout(int64_t limit_cycles, void* stream);

/*
 * Failure-detection self-test: cure_lm_head_argmax with a wait that runs out
 * after `limit_cycles` cycles (1 .. 2^30) in one CTA (`rank` 0 or 1) of every
 * pair.  CURE_DEVERR_TIMEOUT is raised; the tokens are not the argmax, but
 * each is an id of the vocabulary.
 */
cure_status cure_selftest_lm_head_timeout(const void* hidden, const void* w_lm, int32_t rows, int32_t d_model,
                                          int32_t vocab, int32_t* targ, void* workspace, size_t workspace_bytes,
                                          int32_t rank, int64_t limit_cycles, void* stream);

/*
 * Failure-detection self-test: cure_prompt_attn with a wait that runs out, after 2^20
 * SM clock cycles, in one of the roles of its first CTA: the `wait`-th (from 1) of warp
 * `warp` (0 .. 15), if it comes to that many.  CURE_DEVERR_TIMEOUT is then raised, and
 * rows that the CTA had a part in may be left unwritten; the others are as ever, and so
 * is the next call, on the same workspace too.
 */
cure_status cure_selftest_prompt_timeout(const void* q, const void* k_cache, const void* v_cache,
                                         const cure_kv_desc* kv, const int32_t* row_start, const int32_t* cache_len,
                                         int32_t rows, int32_t batch, int32_t heads_q, float scale, void* out,
                                         void* workspace, size_t workspace_bytes, int32_t warp, int32_t wait,
                                         void* stream);

/*
 * The same of cure_prompt_attn8 (of few rows a sequence on average: warps 0 .. 11; else 0 .. 15) and cure_tree_attn8.
 */
cure_status cure_selftest_prompt8_timeout(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                                          const float* v_scale, const cure_kv_desc* kv, const int32_t* row_start,
                                          const int32_t* cache_len, int32_t rows, int32_t batch, int32_t heads_q,
                                          float scale, void* out, void* workspace, size_t workspace_bytes, int32_t warp,
                                          int32_t wait, void* stream);
cure_status cure_selftest_tree8_timeout(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                                        const float* v_scale, const cure_kv_desc* kv, const int32_t* cache_len,
                                        const int32_t* n_nodes, const uint64_t* anc, int32_t batch, int32_t n_max,
                                        int32_t heads_q, float scale, void* out, void* workspace,
                                        size_t workspace_bytes, int32_t warp, int32_t wait, void* stream);

/*
 * Self-test: the form a cure_tree_attn call of this shape takes (`kv` and
 * `route` are HOST pointers; in_place != 0: the in-place layout).  route[0] is
 * the number of CTAs in each unit's cluster (0: the persistent form), route[1]
 * is 1 if that takes its pieces in two tile slots in turn, route[2] the CTAs
 * of the grid.
 */
cure_status cure_selftest_attn_route(int32_t batch, int32_t n_max, int32_t heads_q, const cure_kv_desc* kv,
                                     int32_t in_place, int32_t* route);

/* Static description of a status code. */
const char* cure_status_string(cure_status s);

/* ABI version of this header (major * 100 + minor). */
int32_t cure_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* CURE_H_ */
