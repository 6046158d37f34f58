/*
 * lvlm.h - C ABI of the LightVLM token-reduction / KV-cache-compression kernels (sm_100a).
 *
 * The library implements the computation that LightVLM adds to a vision-language model:
 * pyramid token merging during encoding (paper Section 3.2.1) and KV-cache compression
 * followed by decoding over the shortened cache (Section 3.2.2), with the settings of
 * Appendix A.2.  It does not contain a model: callers hand in the tensors of one layer.
 *
 * Conventions for every entry point
 *   - Every data pointer is a DEVICE pointer owned by the caller.  The library never
 *     allocates, frees or keeps a pointer after the call returns.  `lvlm_dims` itself is a
 *     HOST struct, read during the call only.
 *   - Scratch memory comes from the caller: `ws` (device, 256-byte aligned) of at least
 *     `lvlm_workspace_bytes(op, dims)` bytes.  Its contents need not be preserved or zeroed.
 *   - All work is enqueued on `stream` (a cudaStream_t passed as void*; NULL = the legacy
 *     default stream) and the call returns without synchronising.  Calls that share `ws` or
 *     any in/out tensor must be ordered by the caller (same stream is enough).
 *   - Activations are bf16, scores fp32, indices int32.  The innermost dimension of every
 *     tensor is contiguous and 16-byte aligned.  Only D == 128 is supported.
 *   - A host-detectable error returns a non-zero `lvlm_status` and enqueues nothing.
 *     Conditions only the device can see (non-finite score, length beyond capacity) OR a
 *     `LVLM_DEV_*` bit into `*dev_status` (optional, caller-owned int32 on the device,
 *     never cleared by the library); the offending access is skipped and the kernel ends
 *     normally.  No kernel traps or asserts.
 *   - Results are bit-reproducible from run to run: no floating-point atomics are used.
 */
#ifndef LVLM_H_
#define LVLM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LVLM_OK = 0,
    LVLM_ERR_INVALID_ARG = 1,   /* NULL required pointer, size or range out of bounds */
    LVLM_ERR_UNSUPPORTED = 2,   /* D != 128, n or cache length beyond the built limits */
    LVLM_ERR_ALIGNMENT = 3,     /* pointer or stride not 16-byte aligned */
    LVLM_ERR_WORKSPACE = 4,     /* ws NULL, misaligned or smaller than lvlm_workspace_bytes */
    LVLM_ERR_CUDA = 5           /* a CUDA runtime call failed (launch, attribute, driver entry) */
} lvlm_status;

/* bits OR-ed into *dev_status by kernels */
enum { LVLM_DEV_NONFINITE = 1, LVLM_DEV_TIMEOUT = 2, LVLM_DEV_BOUNDS = 4 };

/* How the r+1 least important image tokens become one token (Section 3.2.1, paragraph 4).
 * p = 0 is the most important merged token; weights are divided by their sum.
 *   LINEAR_RANK   the stated weight list W_v = {r+1, r, ..., 1}                 (default)
 *   GEOMETRIC     (1/2, 1/4, ..., 2^-r, 2^-r): the literal result of repeatedly merging the
 *                 last two tokens of the queue with equal weights
 *   UNIFORM       1/(r+1) each
 *   CUSTOM        caller-supplied list w_custom[0..r]
 *   NEAREST_KEPT  not in the paper: each dropped token is averaged into the kept token with
 *                 the highest cosine similarity of the hidden rows (lower index wins ties),
 *                 weighted by the token masses; that layer's K and V rows are averaged with
 *                 the same assignment; no extra token.  Needs hidden_out (out of place),
 *                 1 <= k, n - k <= 65536, and a workspace sized with d->merge_mode set to it.
 *                 After the call the first B*(n-k) int32 of `ws` hold the assignment: for the
 *                 dropped tokens in ascending order, the index of their kept token in the
 *                 ascending list of kept tokens. */
typedef enum {
    LVLM_W_LINEAR_RANK = 0, LVLM_W_GEOMETRIC = 1, LVLM_W_UNIFORM = 2,
    LVLM_W_CUSTOM = 3, LVLM_W_NEAREST_KEPT = 4
} lvlm_merge_mode;

typedef enum {
    LVLM_OP_SCORE_TOKENS = 0, LVLM_OP_SELECT_TOPK = 1, LVLM_OP_MERGE_COMPACT = 2,
    LVLM_OP_KV_COMPRESS = 3, LVLM_OP_DECODE_ATTN = 4, LVLM_OP_PREFILL_ATTN = 5, LVLM_OP_TREE_ATTN = 6
} lvlm_op;

/* Problem sizes.  Each entry point lists the fields it reads; the others are ignored.
 * Strides are in ELEMENTS; 0 selects the packed default given beside the tensor. */
typedef struct lvlm_dims {
    int32_t B;        /* sequences in the batch */
    int32_t H;        /* query heads */
    int32_t Hkv;      /* key/value heads; H % Hkv == 0; query head h uses KV head h / (H/Hkv) */
    int32_t D;        /* head dimension (128) */
    int32_t N;        /* tokens per sequence before the call */
    int32_t C;        /* hidden channels, a multiple of 8 */
    int32_t cap;      /* rows allocated per (sequence, KV head) in a K or V cache */
    int32_t i0;       /* index of the first image token */
    int32_t n;        /* number of image tokens: the span is [i0, i0+n) */
    int32_t k;        /* image tokens kept intact (P_unmerged); the other n-k are merged */
    int32_t q_lo;     /* scoring: first query row (sequence position) of the window */
    int32_t q_hi;     /* scoring: one past the last query row of the window */
    int32_t causal;   /* scoring: 1 = row at position p sees keys j <= p; 0 = sees all N keys */
    int32_t recent;   /* kv_compress: this many newest entries of every head are never evicted */
    int32_t merge_mode; /* lvlm_workspace_bytes(LVLM_OP_MERGE_COMPACT): the lvlm_merge_mode to size for */
    int32_t cache_stable; /* decode_attn: 1 = Kc, Vc and len are neither written nor still being read by the
                             operation enqueued just before this call (see lvlm_decode_attn) */
    int64_t q_stride_b, q_stride_n, q_stride_h;  /* Q[b][i][h][D]; default packed [B][q_hi-q_lo][H][D] */
    int64_t kv_stride_b, kv_stride_h;            /* K,V[b][g][row][D], rows packed; default [B][Hkv][cap][D] */
    int64_t hid_stride_b;                        /* hidden[b][row][C], rows packed; default N*C */
    int64_t out_stride_b;                        /* hidden_out[b][row][C]; default (rows after the call)*C */
    int64_t head_stride;                         /* score_head[b][g] rows; default n */
    int32_t T;           /* rope_append, commit_rows: new rows of a sequence, the longest; tree_attn: drafted tokens, the most */
    int32_t page;        /* rows of a page of a paged cache: a power of two, at least 16; 0 = the cache is contiguous */
    int32_t n_pages;     /* pages in a paged cache */
    int32_t max_pages;   /* entries of a (sequence, KV head) in the page table */
    int32_t draft_cap;   /* rows allocated per (sequence, KV head) in Kd and Vd */
    int32_t rot;         /* rope_append: channels that are rotated, a multiple of 16 up to D; 0 = none */
    int32_t interleaved; /* rope_append: a pair is 0 = (i, i + rot/2), 1 = (2i, 2i + 1) */
    int32_t n_pos;       /* rope_append: rows of cos_sin */
    int32_t axes;        /* rope_append: positions of a token, 1 (or 0) or 3 */
    int32_t sect0;       /* rope_append, axes == 3: the first sect0 frequencies follow axis 0, */
    int32_t sect1;       /*                         the next sect1 axis 1, the others axis 2 */
    int32_t count_heads; /* commit_rows: 0 = count is [B], 1 = count is [B][Hkv] */
    int32_t mask_shared; /* tree_attn: 1 = one mask for all sequences */
    int64_t new_stride_b, new_stride_n, new_stride_h;  /* k_new,v_new[b][t][g][D]; default packed [B][T][Hkv][D] */
    int64_t page_stride;                         /* Kc,Vc[page][row][D] of a paged cache, rows packed; default page*D */
    int64_t draft_stride_b, draft_stride_h;      /* Kd,Vd[b][g][row][D], rows packed; default [B][Hkv][draft_cap][D] */
} lvlm_dims;

/* Library version string (static storage). */
const char* lvlm_version(void);

/* Text for a status code (static storage). */
const char* lvlm_status_string(lvlm_status s);

/* Bytes of device scratch `op` needs for `d` (0 if `d` is invalid for that op).  Host only. */
size_t lvlm_workspace_bytes(int op, const lvlm_dims* d);

/*
 * Importance of every image token: the attention it receives, summed over the query rows
 * of a window and averaged over heads (Section 3.2.1, paragraph 3: the per-key "cumsum
 * attention scores" A, "averaged ... across different heads").
 *
 *   s_head[b,h,j] = sum_{p in [q_lo,q_hi)} softmax_over_visible_keys(q[b,p,h] . K[b,h/G] * scale)[j]
 *   score[b,j-i0]          = (1/H) sum_h s_head[b,h,j]                     j in [i0, i0+n)
 *   score_head[b,g,j-i0]   = sum_{h in group g} s_head[b,h,j]   (what per-head KV compression uses)
 *
 * The softmax of row p is taken over ALL keys it can see (j <= p if d->causal, else all N),
 * not only over image keys.  The window [0,N) gives the column sums of the full causal
 * attention matrix; the window [i0+n, N) gives the attention of the instruction text only.
 *   Q          [B][q_hi-q_lo][H][D] bf16, row 0 = sequence position q_lo (strides d->q_stride_*)
 *   K          [B][Hkv][cap][D] bf16, rows 0..N-1 valid (strides d->kv_stride_*)
 *   lse        optional [B][H][q_hi-q_lo] fp32: natural-log sum-exp of each row's scaled
 *              logits as produced by the attention kernel that ran before; NULL = computed here
 *   score      [B][n] fp32 out;  score_head optional [B][Hkv] rows of n fp32 out, d->head_stride apart
 *              (a caller can point it at acc_score + i0 of a cache with head_stride = cap)
 * Reads d: B,H,Hkv,D,N,cap,i0,n,q_lo,q_hi,causal,q_stride_*,kv_stride_*,head_stride.
 * Errors: INVALID_ARG (NULL Q/K/score, i0+n>N, q_lo>=q_hi, q_hi>N, N>cap, H%Hkv), UNSUPPORTED
 * (D!=128), ALIGNMENT, WORKSPACE.  A non-finite score sets LVLM_DEV_NONFINITE.
 */
lvlm_status lvlm_score_tokens(const void* Q, const void* K, const float* lse,
                              const lvlm_dims* d, float scale,
                              float* score, float* score_head,
                              void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * The attention of a prefill layer with the importance scores as its by-product (Section 3.2.1, paragraph 3 and
 * its footnote: the per-key summed scores are what the attention kernel of the layer returns anyway, "to avoid
 * incurring additional massive computations").  Computes, for every sequence position p and query head h,
 *     out[b,p,h,:] = softmax_over_visible_keys(Q[b,p,h] . K[b,h/G] * scale) V[b,h/G]
 *     lse[b,h,p]   = natural log of the sum of the exponentials of row p's scaled logits
 * and, when `score` is given, exactly what lvlm_score_tokens computes for the window [q_lo, q_hi) of the same
 * rows - but from the normalisers this attention pass has just produced, so that only the column-sum pass
 * over the window is paid on top of the attention.
 *   Q          [B][N][H][D] bf16, row p = sequence position p (strides d->q_stride_*)
 *   K, V       [B][Hkv][cap][D] bf16, rows 0..N-1 valid (strides d->kv_stride_*)
 *   out        [B][N][H][D] bf16, packed        lse  [B][H][N] fp32
 *   score      optional [B][n] fp32; score_head optional [B][Hkv] rows of n fp32, d->head_stride apart
 *              (needs score); the workspace is only needed with score
 * Reads d: B,H,Hkv,D,N,cap,causal,q_stride_*,kv_stride_*, and with score also i0,n,q_lo,q_hi,head_stride.
 * Errors: INVALID_ARG (NULL Q/K/V/out/lse, N>cap, H%Hkv, scale<=0, score_head without score, a bad window),
 * UNSUPPORTED (D!=128), ALIGNMENT, WORKSPACE.  Contents of the outputs are undefined when a kernel gave up
 * on a wait and set LVLM_DEV_TIMEOUT (the same holds for lvlm_score_tokens, lvlm_merge_compact and out and acc_score
 * of lvlm_decode_attn, whose appended row and len are as without the timeout).
 */
lvlm_status lvlm_prefill_attn(const void* Q, const void* K, const void* V, const lvlm_dims* d, float scale,
                              void* out, float* lse, float* score, float* score_head,
                              void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * Split of the image tokens into P_unmerged and P_merged (Section 3.2.1, paragraph 4): the
 * total order of the n tokens by (score descending, index ascending).
 *   score     [B] rows of n fp32, row stride score_stride elements (0 = n)
 *   rank      [B][n] int32 out: position of token j in the order.  rank < k: kept intact;
 *             rank >= k: merged, and rank - k is its place in the merge queue
 *   kept_idx  optional [B][k] int32 out: the kept tokens, ascending
 *   near_tie  optional [B] int32 out: neighbours (p, p+1) of the order with p+1 >= k whose
 *             fp32 gap satisfies (s_p - s_{p+1}) < 1e-4 * |s_p|  (ties the caller may report)
 * -0 equals +0; NaN sorts last and sets LVLM_DEV_NONFINITE (so does an infinity).
 * Errors: INVALID_ARG (NULL score/rank, B<=0, n<=0, k outside [0,n]), UNSUPPORTED (n > 65536;
 * n > 51200 when kept_idx or near_tie is asked for).
 */
lvlm_status lvlm_select_topk(const float* score, int B, int n, int64_t score_stride, int k,
                             int32_t* rank, int32_t* kept_idx, int32_t* near_tie,
                             void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * Merge and compaction (Section 3.2.1, paragraph 4): P_new = W_v x P_merged and
 * P_compressed = [P_unmerged, P_new], written inside the full sequence:
 *     [ tokens before the image | kept image tokens, original order | P_new | tokens after ]
 * With r = n-k-1 the sequence shrinks from N to N-r rows; r <= 0 (k >= n-1) leaves every
 * tensor unchanged.  In mode NEAREST_KEPT there is no P_new row and the result has
 * N-(n-k) rows.
 *   hidden      [B][N][C] bf16 (batch stride d->hid_stride_b)
 *   hidden_out  [B][rows after][C] bf16, or NULL (or `hidden` itself) to compact `hidden` in place;
 *               any other overlap with `hidden` is INVALID_ARG
 *   Kc, Vc      optional [B][Hkv][cap][D] bf16: this layer's keys and values, rows 0..N-1
 *               valid; compacted IN PLACE with the same map, the merged row being the same
 *               weighted mean per KV head (pass both or neither)
 *   pos_ids     optional [B][N] int32, compacted in place; P_new takes the id of the most
 *               important merged token
 *   rank        [B][n] int32 from lvlm_select_topk (must be a permutation of 0..n-1)
 *   w_custom    [n-k] fp32 (device) when mode == CUSTOM, else NULL
 *   mass        NEAREST_KEPT only, optional [B][N] fp32 in/out: token masses (NULL = all 1),
 *               compacted in place like pos_ids; a kept token's mass grows by what it absorbs
 *   new_len     optional [B] int32 out: rows after the call
 * Reads d: B,N,C,Hkv,D,cap,i0,n,k,hid_stride_b,out_stride_b,kv_stride_*.
 * Errors: INVALID_ARG (NULL hidden/rank, i0+n>N, k outside [0,n], N>cap with Kc, only one of
 * Kc/Vc, CUSTOM without w_custom, C%8), UNSUPPORTED (D!=128 with Kc; C > 8192 with hidden_out;
 * NEAREST_KEPT without hidden_out), ALIGNMENT, WORKSPACE.
 */
lvlm_status lvlm_merge_compact(void* hidden, void* hidden_out, void* Kc, void* Vc,
                               int32_t* pos_ids, const int32_t* rank, const lvlm_dims* d,
                               lvlm_merge_mode mode, const float* w_custom, float* mass,
                               int32_t* new_len,
                               void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * KV-cache compression (Section 3.2.2, paragraph 2; Appendix A.2: threshold beta = 0.995,
 * layers after Layer 5), independently per (sequence, KV head): among the evictable entries
 *     E = [e_lo[b], min(e_hi[b], len - d->recent))
 * sort by (acc_score descending, index ascending), keep the shortest prefix whose cumulative
 * score reaches beta * (total score of E) - the entry that crosses the threshold is kept -
 * but at most budget - (entries outside E); drop the rest of E.  Survivors keep their order;
 * K, V, acc_score and pos are compacted in place and len is updated.
 * The count is exact: scores are taken in integer units of 2^-24 and beta in parts per
 * million; beta >= 1 disables the threshold (keep all, subject to the budget).  Where a head's scores sum to
 * 2^39 or more the unit is coarser, 2^-47 of the largest score's power of two (the sums are kept in 63 bits).
 *   Kc, Vc     [B][Hkv][cap][D] bf16 in/out        acc_score [B][Hkv][cap] fp32 in/out
 *   pos        optional [B][Hkv][cap] int32 in/out len [B][Hkv] int32 in/out
 *   e_lo,e_hi  optional [B] int32 (both or neither); NULL = every entry is evictable
 *   budget     maximum entries per head after the call; <= 0 means no budget
 * The paper's use: e = the image span, beta = 0.995, no budget, once before generation.
 * Periodic use during decoding: e = NULL, beta = 1, budget, d->recent protecting new entries.
 * Reads d: B,Hkv,D,cap,recent,kv_stride_*.
 * Errors: INVALID_ARG (NULL Kc/Vc/acc_score/len, beta outside (0,1], one of e_lo/e_hi),
 * UNSUPPORTED (D!=128, cap > 16384), ALIGNMENT, WORKSPACE.  len > cap sets LVLM_DEV_BOUNDS
 * and that head is left untouched.
 */
lvlm_status lvlm_kv_compress(void* Kc, void* Vc, float* acc_score, int32_t* pos, int32_t* len,
                             const int32_t* e_lo, const int32_t* e_hi, const lvlm_dims* d,
                             float beta, int budget,
                             void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * One decoding step of attention over the (ragged, compressed) cache (Section 3.2.2,
 * paragraph 1: the current token attends to every cached key and value).
 *   o[b,h,:] = softmax(q[b,h,:] . K[b,g,0:len[b,g],:]^T * scale) V[b,g,0:len[b,g],:],  g = h/(H/Hkv)
 *   q        [B][H][D] bf16            out [B][H][D] bf16
 *   Kc, Vc   [B][Hkv][cap][D] bf16     len [B][Hkv] int32
 *   k_new, v_new  optional [B][Hkv][D] bf16 (both or neither): appended at row len before
 *            attending, len += 1.  If len == cap the append is skipped, len stays and
 *            LVLM_DEV_BOUNDS is set.
 *   acc_score optional [B][Hkv][cap] fp32 in/out: entry j receives the probabilities of the
 *            group's query heads, acc_score[b,g,j] += sum_{h in g} p[b,h,j]
 * A head with len == 0 (and no append) outputs zeros.  A head whose len lies outside [0, cap]
 * is skipped: zeros are written, nothing is appended, its len is left alone and
 * LVLM_DEV_BOUNDS is set.
 * d->cache_stable = 1 promises that the operation enqueued on the stream just before this call
 * does not write Kc, Vc or len (true between the layers of a model: the cache of a layer was last
 * written in the previous decoding step; NOT true right after lvlm_kv_compress or
 * lvlm_merge_compact on the same cache).  The kernel then starts fetching the cache while that
 * operation is still draining; q, k_new, v_new and all writes wait for it as always.
 * Workspace: used when acc_score is given and the cache is so long that the scaled logits of a CTA's
 * own keys do not fit in its shared memory (they are then parked there between the pass over the keys and
 * the update of acc_score), and for the partial results where few heads with long caches are cut into parts
 * (two launches then); its contents need not be zeroed.  B * H * cap * 4 bytes (rounded up to 256) are needed; with less than
 * lvlm_workspace_bytes no head is cut.
 * d->N, optional: how many rows the caller expects a head to hold at most (0 = unknown).  Caches are compacted in
 * place, so their capacity says little about their length, and the length is only known on the device; with it
 * the faster form is taken.  It changes no result beyond rounding, and longer heads are handled all the same.
 * Reads d: B,H,Hkv,D,N,cap,kv_stride_*.
 * Errors: INVALID_ARG, UNSUPPORTED (D!=128, H/Hkv > 8), ALIGNMENT, WORKSPACE.
 */
lvlm_status lvlm_decode_attn(const void* q, void* Kc, void* Vc, int32_t* len,
                             const void* k_new, const void* v_new, float* acc_score,
                             const lvlm_dims* d, float scale, void* out,
                             void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

/*
 * lvlm_decode_attn without a workspace argument.  The paper has no counterpart: this entry
 * point exists for callers that cannot obtain device scratch memory at all - a plug-in inside a
 * serving engine that owns every byte of device memory in a pool sized at start-up, a binding
 * from a runtime that is handed raw tensor pointers but no allocator, or a decode loop that must
 * never meet the device-wide synchronisation cudaMalloc and cudaFree imply.  It computes exactly
 * what lvlm_decode_attn computes, with the same arguments minus `ws`/`ws_bytes`; inputs and
 * outputs are still the caller's.
 *
 * The scratch is a fixed array of LVLM_STATIC_SCRATCH_BYTES inside the library image: every GPU
 * on which the library is loaded carries it until the process exits.  A problem that needs more is
 * rejected with LVLM_ERR_WORKSPACE and nothing is enqueued (B * H * cap * 4 bytes are needed; B = 8, H = 32,
 * cap = 1152 takes about 1.2 MiB; long caches are cut into parts only where their results fit as well).
 *
 * The first call on each device looks up the array's device address (with that device current)
 * and remembers it; make that first call outside any stream capture.  No call allocates or frees
 * device memory, here or in a library underneath.
 *
 * All calls on one device share the one array, and it keeps whatever the previous call left in
 * it.  Nothing in it has to start at zero - every word a kernel reads was written earlier in the
 * same call - but two calls that overlap on the GPU (different streams, no ordering between
 * them) race on it and corrupt each other's results.  Keep calls on one stream, or order them.
 * Errors: as lvlm_decode_attn; LVLM_ERR_WORKSPACE when the problem does not fit; LVLM_ERR_CUDA
 * when the address lookup fails.
 */
#define LVLM_STATIC_SCRATCH_BYTES (4u << 20)
lvlm_status lvlm_decode_attn_static(const void* q, void* Kc, void* Vc, int32_t* len,
                                    const void* k_new, const void* v_new, float* acc_score,
                                    const lvlm_dims* d, float scale, void* out,
                                    int32_t* dev_status, void* stream);

/*
 * ---- several new tokens at a time, and paged caches --------------------------------------------------------------
 *
 * The three entry points below have no counterpart in the paper.  After lvlm_kv_compress every head has its own
 * length, but a contiguous cache still occupies cap rows a head; in a PAGED cache the memory that was freed can be used by
 * others.  And a step that takes a tree of drafted tokens reads the cache once for all of them.
 *
 * A cache argument (Kc, Vc, table) is
 *   contiguous  table == NULL, d->page == 0: [B][Hkv][d->cap][D] with strides d->kv_stride_*
 *   paged       Kc and Vc are [d->n_pages][d->page][D] (stride d->page_stride), table [B][Hkv][d->max_pages] int32 on the
 *               device: row j of head (b, g) lies in page table[b][g][j / page] at row j % page.  Its capacity is
 *               cap = max_pages * page.  Entries behind a head's length are not read.  Heads may share pages that are only read;
 *               a page that is appended to belongs to one head.
 * Drafted tokens are kept out of the cache: their keys and values lie in a small contiguous cache of their own,
 * Kd, Vd [B][Hkv][d->draft_cap][D], filled by lvlm_rope_append (len = NULL); after the verification lvlm_commit_rows appends
 * the accepted ones to the cache.  A rejected draft leaves nothing to undo.
 *
 * In all three, `count` (NULL = d->T everywhere) holds the new rows or drafts of each sequence, at most d->T; what
 * belongs to the others is neither read nor written.  A count outside [0, T] is taken as 0 and sets LVLM_DEV_BOUNDS.
 * A head whose len lies outside [0, cap] sets LVLM_DEV_BOUNDS, and so does an append that does not fit behind it: the two that append
 * skip it, nothing of that head is written and its length stays; lvlm_tree_attn gives out = 0 and lse = -inf for all of its rows
 * t < count, whatever drafts they see.  A page number outside [0, n_pages) sets it too; an append skips that row, lvlm_tree_attn takes
 * zeros for the rows of that page.
 */

/*
 * Rotary position embedding of new queries and keys, the keys and values appended to a cache on the way.
 * With c_i = cos_sin[p_i][i], s_i = cos_sin[p_i][rot/2 + i], i < rot/2, a pair (x, y) of channels becomes
 *     (x c_i - y s_i,  y c_i + x s_i)
 * in fp32, rounded once; channels from rot on stay as they are.  p_i is the token's position on the axis that frequency i follows.
 *   q_out[b,t,h]          = rot(q[b,t,h])           q optional [B][T][H][D] (strides d->q_stride_*); q_out [B][T][H][D]
 *                           packed, or q itself: rotated where it lies.  Any other overlap with q is INVALID_ARG
 *   K[b,g,len[b,g] + t]   = rot(k_new[b,t,g])       k_new, v_new [B][T][Hkv][D] (strides d->new_stride_*)
 *   V[b,g,len[b,g] + t]   = v_new[b,t,g]            for t < count[b]
 *   len_out[b,g]          = len[b,g] + count[b]
 * k_new and v_new may not overlap the cache.  A row that is skipped for its page counts in len_out all the same.
 *   pos        [axes][B][T] int32, positions of the tokens; one outside [0, n_pos) sets LVLM_DEV_BOUNDS and leaves the
 *              channels that follow it as they are
 *   cos_sin    [n_pos][rot] fp32, 16-byte aligned; cos_sin and pos are only needed with rot > 0
 *   len        [B][Hkv] int32, or NULL: all zero (a draft cache)
 *   len_out    optional [B][Hkv] int32, may be len itself (a second small launch then where T > 1); any other overlap with len,
 *              or with count, is INVALID_ARG (count may be both of them in one)
 *   acc_score  optional [B][Hkv][cap] fp32: the new entries become 0, as lvlm_decode_attn starts them
 *   pos_cache  optional [B][Hkv][cap] int32: the new entries take pos (of axis 0); needs pos
 * Reads d: B,H,Hkv,D,T,rot,interleaved,n_pos,axes,sect0,sect1,q_stride_*,new_stride_*, and the cache's fields.
 * Errors: INVALID_ARG (NULL k_new/v_new/Kc/Vc, q without q_out or the reverse, rot > 0 without pos or cos_sin, bad sections, a
 * table without pages or pages without a table), UNSUPPORTED (D != 128, rot % 16, a page that is no power of two or
 * below 16), ALIGNMENT.
 */
lvlm_status lvlm_rope_append(const void* q, const void* k_new, const void* v_new, const int32_t* pos,
                             const float* cos_sin, const int32_t* count, void* q_out, void* Kc, void* Vc,
                             const int32_t* table, const int32_t* len, int32_t* len_out, float* acc_score,
                             int32_t* pos_cache, const lvlm_dims* d, int32_t* dev_status, void* stream);

/*
 * Appends rows of a contiguous cache to another cache: the accepted path of a tree of drafts, or (index = NULL,
 * d->count_heads = 1, count = the lengths) a whole ragged cache that moves into pages.
 *   K[b,g,len[b,g] + i] = Kd[b,g,index[b,i]],  V the same,  i < count;   len_out[b,g] = len[b,g] + count
 *   index      optional [B][T] int32, any rows of Kd in any order (one outside [0, draft_cap) sets LVLM_DEV_BOUNDS and its row is
 *              skipped); NULL = rows 0, 1, 2, ...
 *   count      [B] int32, or with d->count_heads [B][Hkv]; NULL = T
 *   pos        optional [B][draft_cap] int32: positions of the rows of Kd, gathered into pos_cache (both or neither)
 *   len, len_out, acc_score, pos_cache: as in lvlm_rope_append.  Kd and Vd may not overlap Kc and Vc.
 * Reads d: B,Hkv,D,T,draft_cap,draft_stride_*,count_heads, and the cache's fields.
 * Errors: INVALID_ARG (also T > draft_cap without an index, Kd == Kc, Vd == Vc, pos without pos_cache or the reverse),
 * UNSUPPORTED, ALIGNMENT.
 */
lvlm_status lvlm_commit_rows(const void* Kd, const void* Vd, const int32_t* index, const int32_t* count,
                             const int32_t* pos, void* Kc, void* Vc, const int32_t* table, const int32_t* len,
                             int32_t* len_out, float* acc_score, int32_t* pos_cache, const lvlm_dims* d,
                             int32_t* dev_status, void* stream);

/*
 * Attention of the drafted tokens of every sequence over its cache and over one another.
 *   visible(b,g,t) = { cache rows j < len[b,g] } and { drafts u < count[b] : t sees u }
 *   out[b,t,h,:]   = softmax over visible of (q[b,t,h] . k * scale), applied to the values, g = h/(H/Hkv), t < count[b]
 *   lse[b,h,t]     = natural log of the sum of the exponentials of the scaled logits
 * A row that sees nothing gives out = 0 and lse = -inf.  With one draft a sequence this is decode attention over either kind
 * of cache.
 *   q        [B][T][H][D] bf16 (strides d->q_stride_*)     out  [B][T][H][D] bf16, packed; q itself where q is packed, any other
 *                                                          overlap with q is INVALID_ARG
 *   len      [B][Hkv] int32                                lse  optional [B][H][T] fp32
 *   Kd, Vd   [B][Hkv][draft_cap][D] bf16, the drafts' keys (rotated) and values, or both NULL: only the cache is seen
 *   mask     [B][T][(T+31)/32] uint32 ([T][(T+31)/32] with d->mask_shared): bit u % 32 of word u / 32 of row t set = t sees
 *            draft u (its ancestors and, as a rule, itself); NULL = a chain, t sees the drafts u <= t
 * Rows behind len and behind count may hold anything, NaN included; the rows in front of them are finite.
 * d->N, optional: how many rows the caller expects a head to hold at most (0 = unknown): how the work is split over the GPU then
 * goes by it instead of the capacity.  It changes no result beyond rounding.
 * Workspace: the partial results where a head's keys are split, 28.3 MB (2^20) and 8 bytes a head and 128 rows at most.
 * lvlm_workspace_bytes(LVLM_OP_TREE_ATTN, d) is enough for d and for every smaller problem; a call is refused less only where it would use
 * it, and one that splits nothing takes ws = NULL.  Calls that may overlap on the GPU need workspaces of their own.
 * Reads d: B,H,Hkv,D,N,T,draft_cap,mask_shared,q_stride_*,draft_stride_*, and the cache's fields.
 * Errors: INVALID_ARG (NULL q/Kc/Vc/len/out, one of Kd/Vd, a mask without drafts, draft_cap < T, scale <= 0), UNSUPPORTED
 * (D != 128, T > 256, H/Hkv > 64, cap / 128 x tiles of 128 query rows > 2^30), ALIGNMENT, WORKSPACE.  Contents of out and lse are undefined when a kernel gave up on a
 * wait and set LVLM_DEV_TIMEOUT.
 */
lvlm_status lvlm_tree_attn(const void* q, const void* Kc, const void* Vc, const int32_t* table, const int32_t* len,
                           const void* Kd, const void* Vd, const uint32_t* mask, const int32_t* count,
                           const lvlm_dims* d, float scale, void* out, float* lse,
                           void* ws, size_t ws_bytes, int32_t* dev_status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LVLM_H_ */
