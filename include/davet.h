/*
 * davet.h -- C ABI of the DAVET per-denoising-step hot path on MI355X (gfx950).
 *
 * DAVET (Denoising-Aware Visual Evidence Trajectory Allocation) conditions each
 * denoising step of a diffusion vision-language model on one of K evidence views
 * built once from a single visual encoding, chosen per step by an allocation
 * policy.  This library implements, for one GPU:
 *
 *   davet_build_views    the ordered evidence hierarchy (Sec. 4.3)
 *   davet_denoise_step   one pass of the bidirectional denoiser over
 *                        [view | prompt | response] (Sec. 3.1, Eq. 1) with the
 *                        argmax / confidence decoding of masked positions
 *   davet_unmask         confidence-ranked commitment (Eq. 2)
 *   davet_policy_*       the allocation policy (Sec. 4.2, Eqs. 6-9): envelope
 *                        and step on the host, the per-step closed loop also
 *                        on the GPU (davet_policy_step_device)
 *   davet_run_schedule   the whole loop: views once, then T steps
 *   davet_cache_*        the attention of a denoiser (or decoder) that keeps
 *                        keys and values in a paged cache and computes only a
 *                        chunk of new tokens: entry into the cache, attention,
 *                        and with davet_evict_select eviction by weight
 *   davet_tree_plan      positions and ancestors of a tree of drafted tokens, and
 *                        with davet_cache_tree_attention its attention
 *   davet_cache_page_*   attention over the pages of a long cache that a cheap
 *                        score selects for each new token
 *   davet_token_logprobs log probabilities, entropy and top alternatives of
 *                        rows of logits
 *   davet_beam_select    the best continuations over beams and vocabulary, and with
 *                        davet_cache_reorder the cache that goes with them
 *   davet_rotary         rotary positions of any layout and scaling
 *
 * Conventions, for every entry point:
 *   - Pointers are DEVICE pointers unless the comment says host.  Arrays are
 *     dense and row-major.  The caller owns every buffer, including the
 *     workspace; the library never frees caller memory and allocates no device
 *     memory (davet_run_schedule uses small host-side vectors; its policy
 *     mode writes into a caller-owned mailbox made once by
 *     davet_mailbox_create).
 *   - Device work is enqueued asynchronously on the given HIP stream.  Only
 *     davet_run_schedule in policy mode synchronises: once per step, on the
 *     GPU kernel that writes the next levels (the next step's launch sizes
 *     depend on them); and davet_fp16_overflow_count, which reads a counter
 *     back to the host.
 *   - Every argument is validated before anything is enqueued; on an error the
 *     call returns a negative davet_status, enqueues nothing, and
 *     davet_last_error() describes the failure (thread-local string).
 *   - Element types: DAVET_F32 = IEEE float32, DAVET_BF16 = bfloat16 bit
 *     patterns, DAVET_F16 = IEEE binary16 bit patterns (both uint16).  The
 *     16-bit modes feed 16-bit operands of that type to the matrix cores with
 *     float32 accumulation; residual streams, softmax statistics and norms
 *     run in float32 in every mode.  A bf16 model is meant to run in the
 *     DAVET_F16 mode: davet_convert rounds its weights to fp16 (a bf16 value
 *     converts exactly when 2^-17 <= |w| <= 65504; smaller ones fall into
 *     fp16's subnormal range and lose bits, |w| <= 2^-25 becomes zero), and
 *     fp16 operands carry 3 more mantissa
 *     bits through the activations at the same matrix-core rate.  The
 *     DAVET_BF16 mode (bf16 activations into the matrix cores) is accurate
 *     to logits rel-RMS <= 1e-2 against a float64 evaluation only for
 *     shallow stacks: measured 6e-3 for one 8B-shaped layer and 2.2e-2 for
 *     32 layers, whose error exceeds that bound; use DAVET_F16 for deep
 *     stacks.
 */
#ifndef DAVET_H
#define DAVET_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum davet_status {
  DAVET_OK = 0,
  DAVET_EINVAL = -1,   /* bad scalar argument or null pointer              */
  DAVET_ESHAPE = -2,   /* unsupported or inconsistent shape                 */
  DAVET_EDTYPE = -3,   /* unsupported element type                          */
  DAVET_ENOMEM = -4,   /* workspace smaller than davet_workspace_bytes()   */
  DAVET_EHIP = -5      /* a HIP runtime call failed                         */
} davet_status;

typedef enum davet_dtype { DAVET_F32 = 0, DAVET_BF16 = 1, DAVET_F16 = 2 } davet_dtype;

/* Limits of this build. */
#define DAVET_MAX_SEQS 64        /* sequences per packed batch            */
#define DAVET_MAX_LEVELS 4       /* K                                     */
#define DAVET_MAX_RESP 1024      /* response length L                     */
#define DAVET_MAX_PAGE_SIZE 256  /* tokens of a cache page                */
#define DAVET_MAX_TOP 64         /* alternatives of davet_token_logprobs  */
#define DAVET_MAX_TREE 256       /* drafted tokens of a sequence          */
#define DAVET_MAX_BEAMS 64       /* beams of a request                    */

/* Evidence realizers (Sec. 4.3: any construction with an ordered
 * evidence-cost hierarchy; pooling is the paper's default, pruning varies
 * the retention ratio, merging the aggregation strength). */
typedef enum davet_realizer {
  DAVET_REALIZER_POOL = 0,   /* per-crop average pooling (and the mixed view) */
  DAVET_REALIZER_PRUNE = 1,  /* nested top-n by token L1 norm                 */
  DAVET_REALIZER_MERGE = 2   /* single-linkage merging by cosine similarity   */
} davet_realizer;
#define DAVET_MAX_REALIZER_GRID 64   /* grid limit of prune and merge */

/* Geometry of one sample's visual encoding v: n_crops crops of grid x grid
 * tokens, each token a d-vector; v is [n_crops*grid*grid, d], crop-major, then
 * row-major inside a crop.  K ordered levels, level K-1 being v itself.
 * mixed_stride: 0 for the pooling pyramid; S >= 2 (K = 3, pooling only) makes
 * level 1 the mixed view of Sec. 4.3 (see davet_build_views).
 * realizer: a davet_realizer; 0 (pooling) when the struct is zero-filled. */
typedef struct davet_view_geom {
  int32_t n_crops;
  int32_t grid;
  int32_t d;
  int32_t K;          /* 1..DAVET_MAX_LEVELS */
  int32_t dtype;      /* davet_dtype of v and of the pooled levels */
  int32_t mixed_stride;
  int32_t realizer;
} davet_view_geom;

/* Denoiser shape.  d = n_heads * head_dim, head_dim in {64, 128} (128 in the
 * 16-bit modes, where d must be a multiple of 128 and ffn of 64); d <= 8192;
 * mask_id in [0, vocab). */
typedef struct davet_model_cfg {
  int32_t n_layers;
  int32_t d;
  int32_t n_heads;
  int32_t head_dim;
  int32_t ffn;
  int32_t vocab;
  int32_t mask_id;
  float rms_eps;
  float rope_theta;
  int32_t dtype;      /* davet_dtype of weights, embeddings and views */
} davet_model_cfg;

/* One layer's parameters (element type = cfg.dtype, out = x W^T):
 *   wqkv [3d, d]  rows: query heads, key heads, value heads (head-major)
 *   wo   [d, d]
 *   wg   [ffn, d] gate, wu [ffn, d] up, wd [d, ffn] down (SwiGLU)
 *   attn_norm, ffn_norm: float32 [d] RMSNorm gains, or NULL for all-ones. */
typedef struct davet_layer_weights {
  const void* wqkv;
  const void* wo;
  const void* wg;
  const void* wu;
  const void* wd;
  const float* attn_norm;
  const float* ffn_norm;
} davet_layer_weights;

/* Layout of the vocabulary-head weights (davet_weights.head_layout).  Both
 * layouts give the same logits and argmaxes bit for bit; the confidences may
 * differ in their last bits (the tiled head sums the exponentials over
 * 256-column vocabulary slabs, the row-major one over 128-column slabs). */
typedef enum davet_head_layout {
  DAVET_HEAD_ROWS = 0,   /* [vocab, d] row-major */
  DAVET_HEAD_TILED = 1   /* 16-bit models only: the output of davet_pack_head */
} davet_head_layout;

/* embed [vocab, d] token embedding; head: untied output head, [vocab, d]
 * row-major or tiled (head_layout); final_norm float32 [d] or NULL; layers:
 * HOST array of n_layers entries. */
typedef struct davet_weights {
  const void* embed;
  const void* head;
  const float* final_norm;
  const davet_layer_weights* layers;
  int32_t head_layout;
} davet_weights;

/* Allocation policy parameters (Sec. 4.2): average budget B, reserve fraction
 * rho, risk strength alpha, operation demand d(o) in [0,1], phase orientation
 * (early != 0: p_t = 1-(t-0.5)/T; else p_t = (t-0.5)/T), K levels. */
typedef struct davet_policy {
  double B;
  double rho;
  double alpha;
  double demand;
  int32_t early;
  int32_t K;
} davet_policy;

const char* davet_last_error(void);
const char* davet_version(void);

/* ---------------------------------------------------------------- views -- */

/* Token counts of the K levels of a geometry (host out[K]).  Level l pools
 * windows of side 2^(K-1-l) per crop with ceil padding:
 * n_l = n_crops * ceil(grid / 2^(K-1-l))^2; the mixed level has
 * n_1 = n_crops * (ceil(grid / 4)^2 + m^2), m = #{o, o+S, ... < grid},
 * o = S / 2.  The prune and merge realizers keep the pooling counts n_l.
 * Errors: EINVAL, ESHAPE (bad K, grid, n_crops, stride or realizer). */
int davet_view_sizes(const davet_view_geom* g, int32_t* n_tokens /*host[K]*/);

/* Lengths of the K member lists of davet_build_views' index maps (host
 * out[K]): n_crops * grid^2 per pyramid or merge level (a partition of the
 * tokens), n_crops * (grid^2 + m^2) for the mixed level, n_l per prune level
 * (one member per kept token). */
int davet_view_map_sizes(const davet_view_geom* g,
                         int32_t* n_members /*host[K]*/);

/* Evidence hierarchy (Sec. 4.3, "Ordered evidence hierarchy"; Sec. 3.2: a full
 * budget leaves v unchanged).  Pooling: level l < K-1 token j is the mean of
 * the in-bounds tokens of its window (divisor = member count), accumulated in
 * float64 and rounded once to the view dtype.  Level K-1 is v itself: nothing
 * is written for it except its (identity) index map.  Prune and merge: the
 * levels given by davet_realizer_maps on davet_realizer_keys, each token the
 * float64 mean of its members in member order, rounded once (a kept token of
 * the prune realizer is copied unchanged).
 *   v            [n_crops*grid*grid, d] (dtype g.dtype), read only
 *   levels       HOST array of K device pointers; levels[l] receives
 *                [n_l, d] for l < K-1; levels[K-1] is ignored (may be NULL)
 *   idx_offsets  HOST array of K device pointers (int32 [n_l + 1]) or NULL;
 *   idx_members  HOST array of K device pointers (int32 [davet_view_map_sizes
 *                entry]) or NULL.  CSR map: token j of level l pools rows
 *                members[offsets[j] .. offsets[j+1]) of v, listed row-major in
 *                the window, ids c*grid*grid + r*grid + s.  Individual entries
 *                may be NULL to skip that level's map.
 * Mixed view (mixed_stride = S >= 2, K = 3; Sec. 4.3: the pooled view
 * augmented with a fixed subset of unpooled tokens): per crop, the level-0
 * tokens (windows of side 4) followed by the raw tokens at rows and columns
 * o, o+S, o+2S, ... (o = S/2), row-major, each a one-member window copied
 * bit for bit from v.
 * scratch: device memory of davet_views_scratch_bytes (NULL / 0 for pooling).
 * Errors: EINVAL (null v / levels entry, misaligned v or level, realizer
 * unknown), ENOMEM (scratch smaller than needed), ESHAPE (grid<1, n_crops<1,
 * K out of range, d % 8 != 0, mixed_stride 1 or < 0, or > 0 with K != 3 or a
 * realizer other than pooling, grid > DAVET_MAX_REALIZER_GRID for prune and
 * merge), EDTYPE. */
int davet_build_views(const davet_view_geom* g, const void* v,
                      void* const* levels, int32_t* const* idx_offsets,
                      int32_t* const* idx_members, void* scratch,
                      size_t scratch_bytes, hipStream_t stream);

/* Device scratch davet_build_views needs for a geometry (0 for pooling): the
 * realizer keys plus the index maps of levels < K-1.  v and the level
 * buffers must be 16-byte aligned; scratch 256-byte aligned.  The scratch is
 * overwritten; nothing is kept in it after the stream reaches the end of
 * the call. */
int davet_views_scratch_bytes(const davet_view_geom* g, size_t* bytes);

/* Number of keys of the prune (n_crops * grid^2, one per token) or merge
 * (n_crops * 2 * grid * (grid - 1), one per grid edge) realizer; 0 for
 * pooling.  Errors: EINVAL, ESHAPE. */
int davet_realizer_key_count(const davet_view_geom* g, int32_t* n_keys);

/* Realizer keys (Sec. 4.3, "Compatible evidence realizers"; the criteria
 * are readings, the paper gives none), float64, device out[n_keys]:
 *   prune  keys[c*grid^2 + i] = sum_j |v[c*grid^2 + i, j]|, the L1 norm of
 *          token i of crop c (exact in any order for fp16 v with d <= 8192);
 *   merge  keys[c*E + e] = cosine similarity of the two tokens of edge e of
 *          crop c, dot / sqrt(|a|^2 |b|^2) (0 if either norm is 0),
 *          E = 2*grid*(grid-1); edges (r,s)-(r,s+1) first at index
 *          r*(grid-1) + s, then (r,s)-(r+1,s) at grid*(grid-1) + r*grid + s.
 * v is [n_crops*grid^2, d] of g.dtype, 16-byte aligned, d % 8 == 0.
 * Errors: EINVAL (null, misaligned, pooling realizer), ESHAPE
 * (grid > DAVET_MAX_REALIZER_GRID), EDTYPE. */
int davet_realizer_keys(const davet_view_geom* g, const void* v,
                        double* keys, hipStream_t stream);

/* For callers that cannot allocate (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): davet_build_views with
 * the prune / merge realizers' scratch (davet_views_scratch_bytes: keys and
 * the maps of the pooled levels) in a device array the library holds, of
 * DAVET_STATIC_SCRATCH_BYTES per GPU, kept until the process ends.  Same
 * arguments and results as davet_build_views without scratch; the call
 * allocates nothing.  The first call on a device resolves the array's
 * address there (a one-time set-up step that may load the library's code
 * object: make it before capturing).  All calls on one device share its
 * array: calls that overlap on one device (other streams, other threads)
 * race; consecutive calls on one stream are safe (everything a call reads
 * from the array it first writes).  Pooling needs no scratch and never
 * touches the array.  Errors: as davet_build_views, and ENOMEM when the
 * geometry needs more scratch than the maximum (e.g. the merge realizer on
 * more than ~40 crops of a 64 x 64 grid). */
#define DAVET_STATIC_SCRATCH_BYTES (4u << 20)
int davet_build_views_static(const davet_view_geom* g, const void* v,
                             void* const* levels, int32_t* const* idx_offsets,
                             int32_t* const* idx_members, hipStream_t stream);

/* Index maps of all K levels from given keys (device float64 [n_keys]),
 * deterministic for identical keys.  Keys are ordered larger first, equal
 * keys by lower index, NaN as -inf, -0 as +0.  Per crop and level l with
 * n = ceil(grid / 2^(K-1-l))^2 tokens (the pooling counts):
 *   prune  the n tokens first in key order, listed by index, one member
 *          each (nested over levels);
 *   merge  edges are taken in key order and each edge joining two groups
 *          merges them until n groups remain, for l = K-2 down to 0
 *          (single linkage; coarser groups are unions of finer ones);
 *          groups listed by smallest member, members ascending.
 * Level K-1 gets the identity map.  idx_offsets[l] ([n_l + 1]) and
 * idx_members[l] (davet_view_map_sizes entry) are device pointers in HOST
 * arrays of K; a NULL entry skips that level.  Errors as
 * davet_realizer_keys. */
int davet_realizer_maps(const davet_view_geom* g, const double* keys,
                        int32_t* const* idx_offsets,
                        int32_t* const* idx_members, hipStream_t stream);

/* Element-type conversion of n values, rounding to nearest even (e.g. a bf16
 * checkpoint into the fp16 operand mode: a bf16 value converts exactly when
 * 2^-17 <= |x| <= 65504, smaller ones lose bits in fp16's subnormal range).  src and dst are device buffers of n elements of their
 * dtypes and must not overlap.  Errors: EINVAL (null, overlap), EDTYPE. */
int davet_convert(const void* src, int32_t src_dtype, void* dst,
                  int32_t dst_dtype, size_t n, hipStream_t stream);

/* Tiled copy of a 16-bit vocabulary head for the head kernel (a one-time
 * model-load transform; the logits are bit-identical to those of the
 * row-major head).  The tiled head is a sequence of 128 x 64 tiles, k-chunk
 * major, so that every vocabulary slab reads chunk c of its rows from one
 * contiguous region while all slabs stream chunk c at the same time:
 *   tiled[((c * S + s) * 128 + r) * 64 + j] = head[(128 s + r) * d + 64 c + j]
 * with S = ceil(vocab / 128) slabs, c < d / 64, r < 128, j < 64; rows past
 * vocab are zero.  src [vocab, d] and dst [davet_head_tiled_elems(vocab, d)]
 * are device buffers of dtype (DAVET_BF16 or DAVET_F16) and must not overlap.
 * Errors: EINVAL (null, overlap), ESHAPE (vocab < 1, d < 64, d % 64 != 0),
 * EDTYPE. */
size_t davet_head_tiled_elems(int32_t vocab, int32_t d);
int davet_pack_head(const void* src, void* dst, int32_t vocab, int32_t d,
                    int32_t dtype, hipStream_t stream);

/* ------------------------------------------------------------- denoiser -- */

/* Workspace bytes davet_denoise_step needs for at most max_tokens packed
 * tokens (sum over sequences of n_view + prompt + L), max_seqs sequences and
 * response length L.  The workspace must be 256-byte aligned. */
int davet_workspace_bytes(const davet_model_cfg* cfg, int32_t max_tokens,
                          int32_t max_seqs, int32_t L, size_t* bytes /*host*/);

/* One denoising step for a packed batch of n_seqs independent sequences
 * (Sec. 3.1, Eq. 1, with the view v_t of Sec. 3.2).  Sequence s is
 *   [ view_ptrs[s] (n_view[s] rows) | E[prompt ids cu_prompt[s]..cu_prompt[s+1]) |
 *     E[resp_ids[s*L + i]], or E[mask_id] where resp_masked[s*L + i] != 0 ]
 * at rotary positions 0..N_s-1, run through cfg.n_layers pre-norm layers with
 * NON-causal attention inside each sequence only (Sec. 1: bidirectional).
 * For every masked response position the final-normed hidden state is projected
 * on the vocabulary and decoded at temperature 0 (Sec. 5.1):
 *   argmax_out[s*L+i] = argmax over w != mask_id (lowest id on ties)
 *   conf_out[s*L+i]   = max softmax probability, [MASK] excluded from the
 *                       normaliser: 1 / sum_{w != mask} exp(l_w - l_argmax)
 * Committed (unmasked) positions get conf = -inf and argmax = -1.
 *   view_ptrs, n_view, cu_prompt: HOST arrays; view rows have dtype cfg.dtype.
 *   prompt_ids int32 [cu_prompt[n_seqs]]; resp_ids int32 [n_seqs*L];
 *   resp_masked uint8 [n_seqs*L]; conf_out float [n_seqs*L];
 *   argmax_out int32 [n_seqs*L];
 *   logits_out float [n_seqs*L, vocab] or NULL: when given, the logits of
 *   masked positions are stored in their rows (other rows untouched).
 *   Weight matrices, norm vectors and view rows are read with 16-byte
 *   vector loads: their pointers must be 16-byte aligned (EINVAL otherwise).
 * Errors: EINVAL, ESHAPE (head_dim, d, ffn, n_seqs, L or token counts out of
 * range), EDTYPE, ENOMEM (ws_bytes too small or workspace misaligned). */
int davet_denoise_step(const davet_model_cfg* cfg, const davet_weights* w,
                       int32_t n_seqs, const void* const* view_ptrs,
                       const int32_t* n_view, const int32_t* prompt_ids,
                       const int32_t* cu_prompt, const int32_t* resp_ids,
                       const uint8_t* resp_masked, int32_t L, float* conf_out,
                       int32_t* argmax_out, float* logits_out, void* workspace,
                       size_t ws_bytes, hipStream_t stream);

/* Number of non-finite values the 16-bit modes stored as GEMM outputs in the
 * last davet_denoise_step on this workspace, or over all the steps of the
 * last davet_run_schedule on it.  The counted stores are the projections'
 * 16-bit outputs: Q/K/V (after rotary embedding) and the SwiGLU product fed
 * to the down projection.  In DAVET_F16 a value beyond +-65504 becomes +-inf
 * there, so a nonzero count means the fp16 range was too small for this model
 * and input (run it in DAVET_F32, or DAVET_BF16 for a shallow stack).  The
 * other 16-bit tensors are bounded by these or by a norm: attention outputs
 * are convex combinations of V rows, and normed rows are at most
 * sqrt(d) * max|gain| in magnitude.  The residual stream and the logits are
 * float32 and not counted; a DAVET_F32 model always reads 0.
 *   workspace: the same 256-byte aligned workspace the step ran on (the
 *   counter is its first 4 bytes); count: HOST int32.
 * Enqueues a 4-byte read on `stream` and waits for it.  Errors: EINVAL (null
 * or misaligned pointer), EHIP (the copy or the wait failed). */
int davet_fp16_overflow_count(const void* workspace, int32_t* count /*host*/,
                              hipStream_t stream);

/* Key-range split of the 16-bit attention (process-wide setting).  A query
 * tile's workgroup normally sweeps every key of its sequence (Sec. 3.1:
 * bidirectional attention, every query sees every key).  When the ragged
 * last query tiles of a launch would run as a thin extra round behind the
 * full tiles, the library divides their keys among up to 8 workgroups, each
 * writing fp32 partial softmax statistics and outputs into the workspace,
 * and a merge kernel combines the pieces in a fixed order, so the result does
 * not depend on timing; only the summation order differs from the unsplit
 * launch.
 *   mode 0: automatic (default); 1: never split; 2..8: split every query
 *   tile into `mode` key ranges (a testing and tuning override; launches
 *   whose partials would not fit in the workspace stay unsplit).
 * Errors: EINVAL (mode outside [0, 8]). */
int davet_set_attention_split(int32_t mode);

/* --------------------------------------------------------------- unmask -- */

/* Confidence-ranked commitment, Eq. (2) (Sec. 5.1: confidence ranking).  Per
 * sequence s, among positions with resp_masked != 0, the k_s = min(k, |M|)
 * positions ranked first by (conf descending, position ascending) -- NaN ranks
 * with -inf, below every number -- are committed: resp_ids[i] = argmax[i],
 * resp_masked[i] = 0.  Other positions are untouched.
 *   conf float [n_seqs*L], argmax int32 [n_seqs*L] (read only)
 *   resp_ids int32 [n_seqs*L], resp_masked uint8 [n_seqs*L] (updated in place)
 *   selected int32 [n_seqs*k] or NULL: committed positions of each sequence in
 *   rank order, padded with -1.
 * Errors: EINVAL (k < 1, null pointers), ESHAPE (L out of range, n_seqs < 1). */
int davet_unmask(int32_t n_seqs, int32_t L, int32_t k, const float* conf,
                 const int32_t* argmax, int32_t* resp_ids, uint8_t* resp_masked,
                 int32_t* selected, hipStream_t stream);

/* ------------------------------------------------------ policy (host) -- */

/* Demand prior d(o) of Appendix A, Table A: category 0 lexical readout 1.000,
 * 1 numerical reasoning 0.941, 2 entity grounding 0.824, 3 binary decision
 * 0.647, 4 general understanding 0.529.  Returns a negative value for an
 * unknown category. */
double davet_demand_prior(int32_t category);

/* Operation parser g (App. A, "Operation Parser and Demand Prior"): the
 * category of a query text (NUL-terminated, any case), host only.  The
 * query is lowercased, generic conversation wrappers ("<image>", "answer
 * the question using a single word or phrase", "in the image", ...) are
 * dropped and the words are matched against the cue families in the
 * appendix's order -- binary decision (auxiliary- or modal-initial), numerical
 * reasoning, lexical readout, entity grounding -- the first match deciding;
 * otherwise general understanding.  The cue phrase lists are this library's
 * reading (the appendix describes the families, not the lists).  *category
 * uses the indices of davet_demand_prior.  Errors: EINVAL (null). */
int davet_parse_operation(const char* query, int32_t* category /*host*/);

/* Evidence envelope, Eq. (6): lower = N(p; (1-rho)B), upper = N(p;
 * [1-rho+rho d]B), with p the phase profile of Sec. 4.2 and N the rescale-and-
 * clip normaliser (exact scale: min(1, s p_t), mean = beta; beta >= 1 gives
 * ones, beta <= 0 zeros).  Double precision, evaluated without contraction.
 * lower, upper: HOST double [T].  Errors: EINVAL (T < 1, null, non-finite). */
int davet_policy_envelope(const davet_policy* pol, int32_t T,
                          double* lower, double* upper);

/* Budget and level of step t (1-based): r_t by Eq. (7) (r_1 = 1), b_t by
 * Eq. (8), level by Eq. (9) generalised to K levels (count of thresholds j/K,
 * j = 1..K-1, that are <= b_t).  lower/upper from davet_policy_envelope.
 * b_t, level, r_t: HOST outputs (r_t may be NULL). */
int davet_policy_step(const davet_policy* pol, int32_t t, int32_t T,
                      const double* lower, const double* upper,
                      double cbar_prev, double churn_prev, double* b_t,
                      int32_t* level, double* r_t);

/* Generation-state signals after a step (Sec. 4.2, before Eq. 7), all HOST
 * arrays of L entries.  cbar = mean of conf over positions still masked after
 * the step's commitment (masked_after != 0), summed in ascending position
 * order; churn = fraction of those positions whose argmax differs from
 * argmax_prev (0 on the first step: argmax_prev == NULL).  Empty set: 0, 0. */
int davet_step_stats(int32_t L, const float* conf, const int32_t* argmax,
                     const int32_t* argmax_prev, const uint8_t* masked_after,
                     double* cbar, double* churn);

/* The closed loop on the GPU (Sec. 4.2): davet_step_stats of every sample
 * after step t's commitment followed by davet_policy_step for step t+1, with
 * bit-identical results (the same float64 operations in the same order).
 *   n_seqs samples of L response positions; 1 <= t < T.
 *   pols, lower, upper: HOST (lower/upper [n_seqs * T] from
 *     davet_policy_envelope, sample s at s*T); every pols[s].K equal.
 *   conf, argmax (step t), argmax_prev (step t-1; NULL exactly when t = 1),
 *   masked_after: DEVICE [n_seqs * L], sample-major.
 *   level_out, budget_out (and r_out unless NULL): DEVICE or pinned host
 *     [n_seqs], the level, b_{t+1} and r_{t+1} of each sample.
 * Errors: EINVAL (null, t out of range, argmax_prev inconsistent with t, K
 * differs or out of range), ESHAPE (n_seqs, L). */
int davet_policy_step_device(int32_t n_seqs, int32_t L, int32_t t, int32_t T,
                             const davet_policy* pols, const double* lower,
                             const double* upper, const float* conf,
                             const int32_t* argmax, const int32_t* argmax_prev,
                             const uint8_t* masked_after, int32_t* level_out,
                             double* budget_out, double* r_out,
                             hipStream_t stream);

/* ------------------------------------------------------------- schedule -- */

/* Mailbox of the policy-mode loop (Sec. 4.2's closed loop): after every
 * step the GPU writes the next levels and budgets of each sample into it,
 * then a stamp the host waits for.  davet_mailbox_create is a one-time
 * set-up call: it allocates a few hundred bytes of pinned, host-coherent
 * memory (hipHostMalloc) that the caller owns until davet_mailbox_destroy,
 * which first synchronises the device (a policy step still queued may write
 * the mailbox) and then frees it.  A mailbox serves one davet_run_schedule
 * call at a time (calls that overlap on one mailbox race); each call uses
 * stamps no earlier call on that mailbox used.  Host only.
 * Errors: EINVAL (null out), ENOMEM, EHIP. */
typedef struct davet_mailbox davet_mailbox;
int davet_mailbox_create(davet_mailbox** out /*host*/);
int davet_mailbox_destroy(davet_mailbox* mailbox);   /* NULL: no-op */

/* Host-side limit (seconds, default 120) on each wait of davet_run_schedule
 * for a step's published levels; a longer wait returns DAVET_EHIP while the
 * stream may still be running (synchronise it before reusing the mailbox,
 * the workspace or the outputs).  Process-wide.  Errors: EINVAL (not
 * positive and finite). */
int davet_set_wait_limit(double seconds);

/* The whole DAVET loop for a packed batch (Sec. 3.1 and Sec. 4; Fig. 2):
 * davet_build_views once per sequence into view_bufs, then for t = 1..T:
 * choose each sequence's level -- fixed_levels[s*T + t-1] when fixed_levels is
 * given, else the policy pols[s] (Eqs. 7-9) from the signals of step t-1 --
 * davet_denoise_step, davet_unmask with k.  In policy mode each step but the
 * last ends with the device policy step (as davet_policy_step_device,
 * writing the next levels and budgets into the mailbox) and a host wait for
 * its stamp, bounded by davet_set_wait_limit; the levels and budgets equal
 * those of davet_step_stats + davet_policy_step on the same signals bit for
 * bit.  The call allocates and frees no host or device memory.
 *   geoms: HOST [n_seqs] (d and dtype must match cfg)
 *   visual: HOST [n_seqs] device pointers to each v
 *   view_bufs: HOST [n_seqs*(K-1)] device pointers, pooled level l of
 *              sequence s at view_bufs[s*(K-1) + l], sized by davet_view_sizes
 *   prompt_ids/cu_prompt as in davet_denoise_step (cu_prompt on the HOST)
 *   resp_ids / resp_masked: device, [n_seqs*L], in/out (normally all-masked
 *              on entry)
 *   pols: HOST [n_seqs] or NULL; fixed_levels: HOST [n_seqs*T] or NULL; exactly
 *         one of the two must be given.
 *   levels_out int32 / budgets_out double: HOST [n_seqs*T] or NULL
 *         (budgets are NaN in fixed mode)
 *   conf_trace float / argmax_trace int32: device [T, n_seqs*L] or NULL.
 *   mailbox: from davet_mailbox_create; required in policy mode with T > 1,
 *            ignored (may be NULL) otherwise.
 * Errors: as the calls it makes; EINVAL for a bad schedule argument or a
 * missing mailbox; EHIP when a wait for published levels fails or exceeds
 * the wait limit. */
int davet_run_schedule(const davet_model_cfg* cfg, const davet_weights* w,
                       int32_t n_seqs, const davet_view_geom* geoms,
                       const void* const* visual, void* const* view_bufs,
                       const int32_t* prompt_ids, const int32_t* cu_prompt,
                       int32_t L, int32_t T, int32_t k,
                       const davet_policy* pols, const int32_t* fixed_levels,
                       int32_t* resp_ids, uint8_t* resp_masked,
                       int32_t* levels_out, double* budgets_out,
                       float* conf_trace, int32_t* argmax_trace,
                       davet_mailbox* mailbox, void* workspace,
                       size_t ws_bytes, hipStream_t stream);

/* ---------------------------------------------------------- paged cache -- */

/* Keys and values of one layer in pages.  Element e of the key of cache index
 * j of sequence s, key head h, is
 *   k[((page * n_kv_heads + h) * page_size + j % page_size) * head_dim + e],
 *   page = page_table[s * max_pages + j / page_size]
 * and v alike.  An entry of the page table outside [0, n_pages) is a hole: it
 * holds no keys (nothing is read from it, nothing is written to it).  Sequences
 * may share pages that they only read.  page_size: a power of two in [16, 256];
 * head_dim 64 or 128; n_kv_heads up to 1024; every dtype.  k and v 16-byte
 * aligned; page_table is a DEVICE array, read when the call runs.
 *
 * A chunk on a cache: HOST arrays cu_q [n_seqs + 1] and kv_len [n_seqs].  Rows
 * cu_q[s] .. cu_q[s+1] of the chunk's tensors are the new tokens of sequence s,
 * the LAST ones of its kv_len[s] cached tokens: row i of n sits at cache index
 * kv_len[s] - n + i.  A sequence may have no new tokens, and no tokens at all.
 * Lengths are taken when the call is made: a captured graph replays those of
 * its capture.  Tensor rows have strides (ld, in elements) and start at 16-byte
 * boundaries; tensors that must not overlap may be columns side by side of one
 * buffer (one stride); query head h of [.., n_heads * head_dim] reads key head
 * h / (n_heads / n_kv_heads).  Rows past cu_q[n_seqs] are left as they are.
 * float32 and int32 arrays are aligned to their elements.
 * Errors of all: EINVAL (null, misaligned, bad scalar), ESHAPE (n_seqs, lengths,
 * strides, page or head counts; kv_len beyond max_pages * page_size), EDTYPE,
 * ENOMEM (workspace). */
typedef struct davet_kv_cache {
  void* k;
  void* v;                    /* may be NULL for davet_cache_weights          */
  const int32_t* page_table;  /* device [n_seqs, max_pages]                   */
  int32_t max_pages;          /* entries of a page table row                  */
  int32_t n_pages;            /* pages of k (and of v)                        */
  int32_t page_size;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t dtype;              /* of k, v and of the chunk's tensors           */
} davet_kv_cache;

/* A chunk's projected rows into the cache, in one pass:
 *   qkv [rows, (n_heads + 2 n_kv_heads) * head_dim], stride ld_qkv: query heads,
 *   key heads, value heads (the row order of davet_layer_weights.wqkv).
 *   norm 1: queries and keys of each head become x / sqrt(mean x^2 + eps) * gain
 *   first (q_gain, k_gain: device float32 [head_dim], 16-byte aligned, NULL for
 *   ones); 0: not.
 *   Then the rotary embedding: elements (i, i + head_dim/2) turn by
 *   p * theta^(-2i/head_dim), p = pos[row] (device int32 [rows]) or, with pos
 *   NULL, the row's cache index.  Angles are reduced in float64: every int32
 *   position is turned as exactly as a small one (theta >= 1).
 * Queries go to q_out [rows, n_heads * head_dim], stride ld_q, which may be qkv
 * itself (same address and, with more than one row, stride: the query columns in
 * place) and must not overlap it otherwise; keys to the cache; values are copied
 * to it bit for bit.  Norm and rotation run in float32 and round once.  The
 * chunk's cache slots must be distinct (no page shared among the sequences that
 * write it). */
int davet_cache_append(const davet_kv_cache* cache, int32_t n_seqs,
                       const int32_t* cu_q, const int32_t* kv_len,
                       const void* qkv, int64_t ld_qkv, int32_t n_heads,
                       const int32_t* pos, int32_t norm, const float* q_gain,
                       const float* k_gain, float eps, float theta, void* q_out,
                       int64_t ld_q, hipStream_t stream);

/* Workspace (256-byte aligned) that davet_cache_attention,
 * davet_cache_tree_attention, davet_cache_page_attention and
 * davet_cache_weights need for chunks of at most max_q tokens in all.  Calls
 * that may overlap in time need one each; its contents mean nothing between
 * calls. */
int davet_cache_workspace_bytes(int32_t n_heads, int32_t head_dim,
                                int32_t max_q, size_t* bytes /*host*/);

/* Attention of a chunk over the cache (which holds the chunk's own keys and
 * values already: davet_cache_append first):
 *   out[row, h] = sum_j softmax_j(scale * q[row, h] . k_j) v_j
 *   lse[row, h] = ln sum_j exp(scale * q[row, h] . k_j)
 * over the visible keys: every key of the sequence (block 0: the bidirectional
 * denoiser), or, with block B >= 1, all cached tokens before the chunk and the
 * chunk's own up to the end of the query's block, blocks of B counted from the
 * chunk's first token (B = 1: causal).  Holes hold no keys.  What is not visible
 * never contributes, whatever it holds (NaN and infinities included).  A row
 * that sees no key, or whose every score is -inf, gets zeros and lse -inf,
 * whatever the values; in any other row a visible value that is not finite makes
 * its element of out an infinity or NaN (it may not where its key scores -inf).
 *   scale: in [1e-30, 1e30], or 0 for 1 / sqrt(head_dim).
 *   q, out [rows, n_heads * head_dim] with strides, not overlapping; lse float32
 *   [rows, n_heads] or NULL.
 * The 16-bit modes round probabilities to 16 bits before they meet the values, or
 * to twice 16 where no chunk of the call has more than 32 rows a key head (queries
 * times heads that share it; so a sequence's results may differ by that rounding with
 * the chunks beside it).  Scores, sums and outputs are float32 until the store.  Results
 * do not depend on timing. */
int davet_cache_attention(const davet_kv_cache* cache, int32_t n_seqs,
                          const int32_t* cu_q, const int32_t* kv_len,
                          const void* q, int64_t ld_q, int32_t n_heads,
                          float scale, int32_t block, void* out, int64_t ld_out,
                          float* lse, void* workspace, size_t ws_bytes,
                          hipStream_t stream);

/* Attention weight that each cached key received from a chunk, over all its
 * queries and heads:
 *   weights[s, j] = prev[s, j] + sum_{row, h} exp(scale * q . k_j - lse[row, h])
 * for j < kv_len[s], with q, scale and block as given to the
 * davet_cache_attention call that wrote lse (rows with lse -inf give nothing).
 * prev and weights: device float32 rows of stride ld_weights; prev may be NULL
 * (zeros) or weights itself, to accumulate over layers and steps.  Entries past
 * kv_len[s] are left as they are; keys in holes receive nothing.
 * A term carries the roundings of its score and of the float32 lse: about 2^-22 of
 * their sizes, relative (0.5 % at 10^4, nothing to rely on beyond 10^6); where
 * |lse| is above 65536 no term counts more than 1. */
int davet_cache_weights(const davet_kv_cache* cache, int32_t n_seqs,
                        const int32_t* cu_q, const int32_t* kv_len,
                        const void* q, int64_t ld_q, int32_t n_heads,
                        float scale, int32_t block, const float* lse,
                        const float* prev, float* weights, int64_t ld_weights,
                        void* workspace, size_t ws_bytes, hipStream_t stream);

/* Which cache entries stay.  Of the n[s] entries of sequence s (HOST) keep[s]
 * (HOST, 0 <= keep <= n) stay: its first `first` and last `last` entries for
 * sure (first + last <= keep unless keep is 0), then those ranked first by
 * (weight descending, index ascending), NaN with -inf, -0 with +0.
 *   weights: device float32, rows of stride ld_weights.
 *   kept: device int32, rows of stride ld_kept: the keep[s] indices, ascending
 *   (entries past keep[s] are left as they are).
 *   weights_out: their weights in that order, rows of stride ld_weights_out, or
 *   NULL; it must not overlap weights.  Whole numbers only depend on the
 * weights: the same weights give the same indices. */
int davet_evict_select(int32_t n_seqs, const int32_t* n, const int32_t* keep,
                       const float* weights, int64_t ld_weights, int32_t first,
                       int32_t last, int32_t* kept, int64_t ld_kept,
                       float* weights_out, int64_t ld_weights_out,
                       hipStream_t stream);

/* Moves the entries that stay: cache index kept[s, j] under cache->page_table
 * becomes index j under dst_table (device [n_seqs, dst_max_pages], pages of the
 * same k and v) for j < keep[s], keys and values, every head.  Call it for each
 * layer, then free the old pages.  An index outside the source table, or in a
 * hole, gives zeros; a hole of dst_table takes nothing.  Destination pages must
 * be distinct and none of them a source page of the call (a page shared with
 * other sequences may be a source: it is only read). */
int davet_cache_gather(const davet_kv_cache* cache, int32_t n_seqs,
                       const int32_t* keep, const int32_t* kept,
                       int64_t ld_kept, const int32_t* dst_table,
                       int32_t dst_max_pages, hipStream_t stream);

/* ------------------------------------------- a tree of drafted tokens -- */

/* Positions and ancestors of drafted tokens that form trees, several continuations
 * of one history checked in one pass.  Rows cu_q[s] .. cu_q[s+1] (HOST, at most
 * DAVET_MAX_TREE of a sequence) are the drafted tokens, the last ones of the kv_len[s]
 * (HOST) cached ones; parent (device int32 [rows]) the token that each continues,
 * counted from its sequence's first drafted one, or a negative number: the last token
 * before the draft.  A parent comes before its children: an entry that is not below
 * the token's own number counts as negative.
 *   pos: device int32 [rows], or NULL: first_pos[s] (HOST, NULL for kv_len[s] less the
 *   drafted tokens) plus the number of drafted tokens above the row's; the `pos` of
 *   davet_cache_append.
 *   mask: device uint32 [rows, DAVET_MAX_TREE / 32], or NULL: bit j % 32 of word j / 32
 *   set where drafted token j is the row's own or above it.
 * kv_len may be NULL with first_pos.  Errors: EINVAL, ESHAPE. */
int davet_tree_plan(int32_t n_seqs, const int32_t* cu_q, const int32_t* kv_len,
                    const int32_t* first_pos, const int32_t* parent, int32_t* pos,
                    uint32_t* mask, hipStream_t stream);

/* davet_cache_attention (its formulas, arguments, workspace and numerics) where row i
 * of a sequence sees every cached token before the chunk, and of the chunk's own those
 * j whose bit in its row of `mask` (as davet_tree_plan's, but any bits will do) is
 * set; bits past the sequence's chunk are not looked at.  At most DAVET_MAX_TREE new
 * tokens a sequence.
 * The accepted tokens of a tree are moved to the front with davet_cache_gather: a
 * cache whose page tables start with the page of the first drafted token, `kept` what
 * of that page was there before and then the accepted ones, into fresh pages. */
int davet_cache_tree_attention(const davet_kv_cache* cache, int32_t n_seqs,
                               const int32_t* cu_q, const int32_t* kv_len,
                               const void* q, int64_t ld_q, int32_t n_heads,
                               float scale, const uint32_t* mask, void* out,
                               int64_t ld_out, float* lse, void* workspace,
                               size_t ws_bytes, hipStream_t stream);

/* --------------------------------------- attention over selected pages -- */

/* For caches of which a new token reads only the pages that matter to it.  Bounds:
 * of every page and key head the smallest and the largest value of each element of
 * its keys, as device array [n_pages, n_kv_heads, 2, head_dim] of the cache's type,
 * 16-byte aligned, which the caller keeps beside the pools (a page's bounds go with
 * the page: sequences that share one share them).
 *
 * This call brings up to date the bounds of the pages that hold the chunk's tokens,
 * over their tokens below kv_len: call it after davet_cache_append.  (A chunk of the
 * whole sequence, cu_q = 0, kv_len, does every page, for instance after
 * davet_cache_gather.)  Holes are left out, other pages' bounds as they are; a NaN
 * among the keys makes its bounds NaN.  A page must not belong to two sequences that
 * have new tokens in it.  cache->v may be NULL.  Errors: as for a chunk. */
int davet_cache_page_bounds(const davet_kv_cache* cache, int32_t n_seqs,
                            const int32_t* cu_q, const int32_t* kv_len, void* bounds,
                            hipStream_t stream);

/* Which pages each new token reads, for each key head: of the pages with keys that are
 * visible to it (as in davet_cache_attention, `block` too; holes apart) all, if there
 * are no more than `top`; else its first `first` and last `last` ones and then those
 * ranked first by (score descending, page ascending), NaN with -inf,
 *   score = sum_{heads of the key head} sum_e max(q_e lo_e, q_e hi_e),
 * no less than the sum of their scores (without the scale) with any key of the page.
 * The sum is taken in float64, in an order that goes by the sizes of the call, and
 * rounded to float32.  Where products and sums are exact in float64 (16-bit values whose
 * products lie within some 2^20 of each other) the order does not matter; elsewhere it
 * may seldom round a score to the neighbouring float32, and so decide between two pages
 * that close.
 *   pages: device int32 [rows, n_kv_heads, top]: indices in the sequence's page table,
 *   ascending, then -1.
 * top in [1, 32768], first + last <= top; sequences with new tokens have at most 32768
 * pages.  cache->k and v are not read.  Errors: as for a chunk. */
int davet_cache_page_select(const davet_kv_cache* cache, int32_t n_seqs,
                            const int32_t* cu_q, const int32_t* kv_len, const void* q,
                            int64_t ld_q, int32_t n_heads, int32_t block,
                            const void* bounds, int32_t first, int32_t last,
                            int32_t top, int32_t* pages, hipStream_t stream);

/* davet_cache_attention (its formulas, arguments, workspace and numerics; probabilities
 * are rounded to twice 16 bits) where each new token and key head sees, of the keys
 * that are visible there, those in the pages of its list: pages [rows, n_kv_heads, top]
 * as davet_cache_page_select writes it, or any other.  Entries outside the sequence's
 * pages are no pages, wherever they stand; of more entries than the sequence has pages
 * only as many are read; an order other than ascending changes no more than the sums'
 * order, and a page that is listed twice counts twice.  top in [1, 2^26]. */
int davet_cache_page_attention(const davet_kv_cache* cache, int32_t n_seqs,
                               const int32_t* cu_q, const int32_t* kv_len,
                               const void* q, int64_t ld_q, int32_t n_heads,
                               float scale, int32_t block, const int32_t* pages,
                               int32_t top, void* out, int64_t ld_out, float* lse,
                               void* workspace, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------ token log probabilities -- */

/* Log probabilities, entropy and top alternatives of rows of logits (for
 * instance davet_denoise_step's logits_out), temperature 1, natural logarithm:
 *   logp[r] = logits[r, targets[r]] - logsumexp(logits[r, :])
 *   entropy[r] = -sum_w p_w ln p_w
 *   top_ids, top_logp [rows, top]: the `top` (0 .. 64) largest logits' ids and
 *   log probabilities, by (logit descending, id ascending).
 * logits [rows, vocab] of dtype, row stride ld, aligned to their element.
 * exclude: a token left out of everything (probability 0; -1: none), as
 * davet_denoise_step leaves out [MASK].  A target outside [0, vocab) or excluded
 * has logp -inf.  Only logits above -inf are listed; where there are fewer than
 * `top`, ids are -1 and log probabilities -inf.  A row without any: logp -inf,
 * entropy 0.  A NaN or +inf logit makes the row's probabilities NaN; ids are
 * ranked all the same, NaN never listed.  logp (with targets), entropy may be
 * NULL.  workspace: davet_logprobs_workspace_bytes, 256-byte aligned (NULL / 0
 * where that is 0).  It says what exactly `rows` rows need, and fewer rows, each cut
 * into more slices, may need MORE (256 need nothing): a workspace kept for every
 * count of up to N rows holds (min(N, 255) + 255) * (8 * top + 12) bytes, which is
 * enough for each of them and for any vocab.
 * Errors: EINVAL, ESHAPE (rows, vocab, ld, top), EDTYPE, ENOMEM. */
int davet_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top,
                                   size_t* bytes /*host*/);
int davet_token_logprobs(int32_t rows, int32_t vocab, const void* logits,
                         int32_t dtype, int64_t ld, int32_t exclude,
                         const int32_t* targets, float* logp, float* entropy,
                         int32_t top, float* top_logp, int32_t* top_ids,
                         void* workspace, size_t ws_bytes, hipStream_t stream);

/* -------------------------------------------------------------- beams -- */

/* The best continuations of `groups` requests with `beams` beams each: row g beams + b
 * of logits (as davet_token_logprobs takes them, `exclude` too) belongs to beam b of
 * request g, which has the score scores[row] (device float32).  Candidates are the
 * pairs of a row and a token with a logit above -inf, of value
 *   scores[row] + logits[row, w] - logsumexp(logits[row, :]);
 * a row with done[row] other than 0 (device int32, NULL: none) has one candidate
 * instead, the token `pad` with the value scores[row], and its logits are not read.  A
 * row whose score or logsumexp is not finite has none.
 *   out_scores, out_rows, out_tokens [groups, top]: the values (rounded to float32),
 *   rows and tokens of the `top` (1 .. 64) best, by (value descending, row ascending,
 *   logit descending, token ascending); values are compared in float64, the sums of
 *   exponentials under them are float32.  Where there are fewer candidates: -inf, -1,
 *   -1.  out_scores may be scores where top is beams, and must not overlap it otherwise.
 * beams 1 .. DAVET_MAX_BEAMS, at most 2^22 rows.  workspace:
 * davet_beam_workspace_bytes for these sizes exactly (fewer requests may need more),
 * 256-byte aligned; (rows + 255) * (8 * top + 12) + 255 bytes are enough for any vocab
 * and fewer rows.
 * Errors: EINVAL, ESHAPE (sizes, ld), EDTYPE, ENOMEM. */
int davet_beam_workspace_bytes(int32_t groups, int32_t beams, int32_t vocab,
                               int32_t top, size_t* bytes /*host*/);
int davet_beam_select(int32_t groups, int32_t beams, int32_t vocab,
                      const void* logits, int32_t dtype, int64_t ld,
                      int32_t exclude, const float* scores, const int32_t* done,
                      int32_t pad, int32_t top, float* out_scores,
                      int32_t* out_rows, int32_t* out_tokens, void* workspace,
                      size_t ws_bytes, hipStream_t stream);

/* Moves the cache along with the beams: sequence s continues sequence parent[s]
 * (device int32 [n_seqs], rows of cache->page_table, which has n_seqs of them; the same
 * one may be continued several times).  Its row of dst_table (device [n_seqs,
 * dst_max_pages], not overlapping page_table) takes the pages of parent[s] that
 * kv_len[s] tokens (HOST: the parent's length) fill, which the two then share, and for
 * a last page that they fill in part fresh[s] (device int32), into which the keys and
 * values of its tokens are copied, every head.  Call it for each layer (the table comes
 * out the same), then let go of pages that no table has.  Entries behind are left as
 * they are.  Fresh pages must be distinct and hold no key that the call reads (fresh[s]
 * may be the parent's own last page: then it stays there, uncopied).  A parent outside
 * [0, n_seqs), a hole for a last page and a fresh page outside the pool make the
 * entries concerned -1.
 * n_seqs is at most DAVET_MAX_SEQS and parents count from this call's first row, while
 * davet_beam_select counts rows over its whole batch: a batch of more rows is moved in
 * several calls of whole requests, each on its rows of the page tables, with the first
 * of them taken off out_rows (on the device). */
int davet_cache_reorder(const davet_kv_cache* cache, int32_t n_seqs,
                        const int32_t* kv_len, const int32_t* parent,
                        const int32_t* fresh, int32_t* dst_table,
                        int32_t dst_max_pages, hipStream_t stream);

/* ----------------------------------------------------- rotary positions -- */

/* davet_cache_append turns whole heads in halves by unscaled frequencies.  For
 * models with another layout these calls turn queries and keys first; the append
 * then gets pos all zero, which turns no finite value (cos 0 = 1 and sin 0 = 0 exactly;
 * an infinity, 0 times which is NaN, makes its partner NaN there as in any turn). */
typedef enum davet_rotary_layout {
  DAVET_ROTARY_HALVES = 0,   /* pair i: elements i and i + dim / 2 */
  DAVET_ROTARY_PAIRS = 1     /* pair i: elements 2 i and 2 i + 1   */
} davet_rotary_layout;

/* Frequencies f_i of pair i, from f = theta^(-2 i / dim): */
typedef enum davet_rotary_scaling {
  DAVET_ROTARY_PLAIN = 0,    /* f                                                */
  DAVET_ROTARY_LINEAR = 1,   /* f / factor: positions interpolated               */
  DAVET_ROTARY_BASE = 2,     /* theta times factor^(dim / (dim - 2)): the fastest
                                pair as it was, the slowest one / factor         */
  DAVET_ROTARY_RAMP = 3      /* w f + (1 - w) f / factor, w the turns that the pair
                                makes in `trained` positions, from `slow` (0) to
                                `fast` (1), clamped: fast pairs as they were, slow
                                ones interpolated                                */
} davet_rotary_scaling;

/* turns[i] = f_i / (2 pi), the turns pair i makes a position (HOST, dim / 2 doubles;
 * copy them to the device once).  factor, trained, fast and slow are read by the
 * scalings that name them.  dim even in [2, 512]; theta >= 1, factor >= 1, trained
 * > 0, fast > slow >= 0.  Errors: EINVAL, ESHAPE. */
int davet_rotary_turns(int32_t dim, double theta, int32_t scaling, double factor,
                       double trained, double fast, double slow,
                       double* turns /*host*/);

/* Turns the first `dim` elements of each head of x [rows, n_heads * head_dim] (row
 * stride ld_x) to out (ld_out): pair (a, b) by t = 2 pi pos[row] turns[i],
 *   a' = gain (a cos t - b sin t),  b' = gain (b cos t + a sin t),
 * and copies the others.  inverse 1: by -t, which makes it the gradient of the call
 * with inverse 0 (dx from dout, the same gain).
 *   pos: device int32 [rows], any values, or NULL for the row numbers; turns: device
 *   double [dim / 2].  Whole turns are taken off in float64 without a rounding, so a
 *   far position adds only what its rate is off by, up to |pos| turns[i] 2^-53 turns
 *   (4e-8 for the fastest pair at 2^31).
 *   gain: finite (1; a scaled model's attention factor, once on queries and keys).
 *   out may be x (same address and, of several rows, stride) and must not overlap
 *   it otherwise.  Strides and addresses need no more than the elements' alignment;
 *   16-byte ones are the fastest.
 * Products run in float32 and round once.
 * Errors: EINVAL, ESHAPE (rows up to 2^24, n_heads in [1, 4096], head_dim even in
 * [2, 512], dim even in [2, head_dim], strides), EDTYPE. */
int davet_rotary(int32_t rows, int32_t n_heads, int32_t head_dim, int32_t dim,
                 int32_t layout, const void* x, int64_t ld_x, void* out,
                 int64_t ld_out, int32_t dtype, const int32_t* pos,
                 const double* turns, float gain, int32_t inverse,
                 hipStream_t stream);

/* ------------------------------------------------------------ profiling -- */

/* Per-kernel-class timing with HIP events recorded around every launch on the
 * launch stream (for the measurement harness).  davet_prof_enable(n) reserves
 * event pairs for n launches (host-side and HIP event objects, created here,
 * not in the steady state) and starts recording; davet_prof_enable(0) stops
 * and releases them.  davet_prof_read synchronises on the recorded events and
 * fills, per kernel class c < n_classes, the launch count and summed
 * milliseconds; names via davet_prof_class_name.  Returns the number of
 * classes, or a negative status.  davet_prof_only(c) restricts recording to
 * launches of class c (so that a timed run carries events around one kernel
 * class only); -1 records every class again. */
int davet_prof_enable(int32_t max_launches);
int davet_prof_reset(void);
int davet_prof_only(int32_t cls);
int davet_prof_read(int32_t n_classes, int64_t* counts /*host*/,
                    double* total_ms /*host*/);
const char* davet_prof_class_name(int32_t cls);

#ifdef __cplusplus
}
#endif
#endif /* DAVET_H */
