/*
 * tkphi.h -- C ABI of libtkphi: decode-step Top-K+phi residual-mass attention
 * and its prefill summary build, and the append / attention calls of a paged cache,
 * as hand-written CUDA kernels for sm_100a.
 *
 * Method (arXiv 2604.05438, "Residual-Mass Accounting for Partial-KV Decoding"):
 * for one attention layer and each decode query head the library
 *   (1) scores the query against every mid-region key, s_i = q.k_i / sqrt(d_h)
 *       (Sec. 3, Eq. full_attention), and selects the K highest-scoring
 *       mid-region indices K(q) (exhaustive Top-K control selector, Sec. 5.1);
 *   (2) forms the exact unnormalised terms nu_E, Z_E over E = A U K(q), A the
 *       sink/tail anchors (Sec. 3, Eq. partition and Eq. exact_terms);
 *   (3) removes the retrieved tokens' feature contributions from the prefill
 *       summaries (S, u) (Sec. 4.2, Eq. subtraction);
 *   (4) evaluates the residual estimate nu_hat_R = S_R phi_q(q),
 *       Z_hat_R = phi_q(q)^T u_R (Sec. 4.3);
 *   (5) returns y = (nu_E + nu_hat_R) / (Z_E + Z_hat_R) (Sec. 4.3, Eq. hybrid_merge).
 * The prefill pass builds S = sum_{i in M} v_i phi_k(k_i)^T, u = sum_{i in M} phi_k(k_i)
 * over the mid-region M (Sec. 4.1, Eq. natural_cache).
 *
 * Feature maps: phi(x) = exp(W x + b - gamma ||x||^2) elementwise, W in R^{r x d};
 * one map per query head (phi_q) and one per KV head (phi_k) (Sec. 4.1; positivity
 * by exponentiation, App. C.1).
 *
 * General rules
 *  - Every tensor pointer is a DEVICE pointer unless its comment says "host".
 *    The caller owns all memory; the library allocates nothing, keeps nothing
 *    between calls, and enqueues its work on the caller's stream (a
 *    cudaStream_t passed as void*; NULL is the default stream).
 *  - Functions return after enqueuing.  The return value reports host-side
 *    validation and launch errors only; invalid arguments are rejected before
 *    anything is launched.  tkphi_last_error() gives a message for the last
 *    failing call of the calling thread.
 *  - Small per-sequence arrays (cu_seqlens, topk) are passed twice: a host copy
 *    (validated, used for sizing) and a device copy with the same contents (read
 *    by the kernels), so that no call needs a device-to-host synchronisation.
 *  - Inputs must be finite.  Results for NaN/Inf inputs are unspecified.
 *  - One call processes one attention layer; a model stack is a host loop.
 */
#ifndef TKPHI_H
#define TKPHI_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TKPHI_OK = 0,
  TKPHI_ERR_INVALID_ARG = -1,  /* bad pointer, size, stride or range */
  TKPHI_ERR_UNSUPPORTED = -2,  /* legal problem the library has no kernel for */
  TKPHI_ERR_WORKSPACE = -3,    /* workspace NULL, misaligned or too small */
  TKPHI_ERR_CUDA = -4,         /* a CUDA runtime/driver call failed */
  TKPHI_ERR_TIMEOUT = -5       /* a bounded device-side wait ran out (see tkphi_device_status) */
} tkphi_status;

/* Which entry point a workspace is sized for. */
enum { TKPHI_WS_BUILD = 0, TKPHI_WS_TOPK_DECODE = 1, TKPHI_WS_DECODE_STEP = 2, TKPHI_WS_MLP_KEY_FEATURES = 3 };

/* Flags of tkphi_decode_step. */
enum {
  TKPHI_FLAG_NONE = 0,
  TKPHI_FLAG_NOSUB = 1 /* skip the retrieved-token subtraction (the paper's NoSub ablation, Sec. 5.1) */
};

/*
 * One attention layer's K/V cache for `batch` ragged sequences (Sec. 3: keys and
 * values (k_i, v_i), i < L, per KV head).  Sequence b owns cache rows
 * cu_seqlens[b] .. cu_seqlens[b+1]-1; its prefill length is L_b = cu_seqlens[b+1]
 * - cu_seqlens[b] >= 1.  Element (head h, row t, dim c) of k is at
 * k + h*kv_stride_head + t*kv_stride_token + c (in bf16 elements); v uses the
 * same strides.  Requirements: 1 <= batch <= 1024; head_dim in {64, 128}; n_q_heads a multiple of
 * n_kv_heads with group size <= 8; n_feat in {64, 128}; k and v 16-byte aligned;
 * both strides multiples of 8 elements; kv_stride_token >= head_dim; total rows
 * < 2^31; at most 2,097,152 mid-region rows per sequence for the decode entry points.
 * With more than one KV head the heads must not share memory: either kv_stride_head >=
 * rows * kv_stride_token (head-major) or kv_stride_head >= head_dim and kv_stride_token >=
 * (n_kv_heads - 1) * kv_stride_head + head_dim (token-major); anything else, a zero head
 * stride included, is TKPHI_ERR_INVALID_ARG.
 * Query head h_q uses KV head h_q / (n_q_heads / n_kv_heads).
 * Any strides within these rules work.  Head-major caches (kv_stride_head a multiple of
 * kv_stride_token) and token-major ones (kv_stride_token a multiple of kv_stride_head) also
 * let the decode entry points fetch the rows of the exact support by TMA row gathers, which
 * calls with many retrieved rows (more 256-token pieces of support lists than SMs) use.
 * Anchors (Eq. partition): the first n_sink and the last n_tail rows of each
 * sequence (their union when L_b < n_sink + n_tail); the mid-region is what lies
 * between, |M_b| = max(0, L_b - n_sink - n_tail).
 * n_tail_seq_host / n_tail_seq_dev (optional; both NULL or both given, the same [batch]
 * values >= 0 on the host and on the device) give every sequence a tail-anchor count of its
 * own, which then replaces n_tail everywhere: sequences that have generated different
 * numbers of tokens share a decode call this way (see tkphi_decode_step).
 */
typedef struct {
  int32_t batch, n_q_heads, n_kv_heads, head_dim;
  int32_t n_feat;                 /* r = d_phi */
  int32_t n_sink, n_tail;         /* >= 0 */
  const int64_t* cu_seqlens_host; /* host,   [batch+1], cu[0] = 0, non-decreasing */
  const int64_t* cu_seqlens_dev;  /* device, same contents */
  const void* k;                  /* device, bf16 */
  const void* v;                  /* device, bf16 */
  int64_t kv_stride_head, kv_stride_token; /* in elements */
  const int32_t* n_tail_seq_host; /* host,   [batch] or NULL */
  const int32_t* n_tail_seq_dev;  /* device, [batch] or NULL */
} tkphi_kv_desc;

/* phi(x) = exp(W x + b - gamma ||x||^2); row-major fp32 parameters on the device; w_q and
 * w_k 16-byte aligned (as are S and u where a call takes them).
 *
 * phi_k_cache (optional, NULL to leave out) is the cached-feature variant that Sec. 4.2
 * names as a way to avoid recomputing the retrieved keys' feature maps at decode time:
 * device fp32 [n_kv_heads][T_total][n_feat], T_total = cu_seqlens[batch], 16-byte aligned,
 * owned by the caller.  tkphi_build_summaries, given a non-NULL pointer, also writes
 * phi_k(k_i) of every mid-region token i of every sequence to row cu_seqlens[b] + i of each
 * KV head (rows of anchor tokens are left untouched).  tkphi_decode_step, given a non-NULL
 * pointer, takes the retrieved tokens' feature rows from it instead of recomputing them from
 * the keys (Eq. subtraction is unchanged: the same phi_k(k_i) enter it); the rows must hold
 * what the build wrote for the same cache, anchors and parameters (w_k, b_k and gamma_k are
 * then not read by the decode step).  tkphi_topk_decode and the NoSub flag ignore it. */
typedef struct {
  const float* w_q; /* [n_q_heads][n_feat][head_dim] */
  const float* b_q; /* [n_q_heads][n_feat] */
  const float* w_k; /* [n_kv_heads][n_feat][head_dim] */
  const float* b_k; /* [n_kv_heads][n_feat] */
  float gamma_q, gamma_k;
  float* phi_k_cache; /* optional, [n_kv_heads][T_total][n_feat] */
} tkphi_phi_desc;

/*
 * Bytes of workspace the given entry point needs for this problem (0 on invalid
 * arguments; tkphi_last_error() then says why).  topk_host (host, [batch]) may be
 * NULL for TKPHI_WS_BUILD.  The workspace must be 256-byte aligned device memory.
 * Its contents on entry do not matter and are undefined on exit.
 */
size_t tkphi_workspace_bytes(const tkphi_kv_desc* kv, const int32_t* topk_host,
                             int32_t topk_max, int which);

/*
 * Prefill summary build (Sec. 4.1, Eq. natural_cache): for every sequence b and KV
 * head h, S[b][h] = sum_{i in M_b} v_i phi_k(k_i)^T (row-major [head_dim][n_feat],
 * fp32) and u[b][h] = sum_{i in M_b} phi_k(k_i) ([n_feat], fp32); both zero when the
 * mid-region is empty.  Only phi->w_k, b_k and gamma_k are read.
 * S: [batch][n_kv_heads][head_dim][n_feat], u: [batch][n_kv_heads][n_feat], written in full.
 */
tkphi_status tkphi_build_summaries(const tkphi_kv_desc* kv, const tkphi_phi_desc* phi,
                                   float* S, float* u,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Prefill summary build without any caller-provided workspace (the paper has no
 * counterpart; this serves a deployment constraint).  Some callers cannot obtain
 * device memory at call time: plug-ins of a serving process whose memory pool is sized
 * and handed out once at start-up, runtimes that forbid cudaMalloc (an implicit
 * device-wide synchronisation) on the latency-critical path, and hosts whose policy
 * allows allocation only during initialisation.  For them this entry point
 * computes exactly what tkphi_build_summaries computes, on the same kernel, but takes
 * its scratch from a fixed array of TKPHI_STATIC_SCRATCH_BYTES that is part of the
 * library's device image.  It calls no allocating routine of CUDA or of any library.
 *  - Limit: problems whose tkphi_workspace_bytes(kv, NULL, 0, TKPHI_WS_BUILD) exceeds
 *    TKPHI_STATIC_SCRATCH_BYTES are rejected with TKPHI_ERR_WORKSPACE before anything
 *    is enqueued (the message names both sizes); use tkphi_build_summaries for those.
 *  - Cost: the array is part of the library's device code.  Every GPU on which that code
 *    is loaded holds the array until the process exits.  The CUDA runtime loads it on a
 *    device when the library is first used there (at the latest by this function's first
 *    call on the device, which therefore is also where the device's free memory drops by
 *    the array's size).
 *  - First call on each device: looks up the array's device address (a host-side
 *    runtime query, done with that device current and cached).  Make that first call
 *    at initialisation, before any stream capture begins on the device.
 *  - Sharing: all calls on a device use the same array.  The array keeps the previous
 *    call's contents; the build needs none of it cleared (the kernel sets the status word
 *    at the head of the array itself and overwrites every partial sum before it is read).
 *    Two calls whose GPU work overlaps (different streams, or different host threads)
 *    race on it and give undefined results: serialise them.
 *  - Device-side errors: tkphi_static_device_status reads the status word of the last
 *    static call on the current device (the array's address is not exposed, so
 *    tkphi_device_status cannot be used): 0, or TKPHI_ERR_TIMEOUT if a bounded wait of the
 *    build kernel ran out, in which case (S, u) are not valid.  Waits for the stream;
 *    *status_out is a host int.  TKPHI_ERR_INVALID_ARG if no static call has been made on
 *    the device yet.
 * Arguments, outputs and error reporting otherwise as for tkphi_build_summaries;
 * tkphi_static_last_error() gives the message of the last failing call of the thread.
 */
#define TKPHI_STATIC_SCRATCH_BYTES (8u << 20)
tkphi_status tkphi_build_summaries_static(const tkphi_kv_desc* kv, const tkphi_phi_desc* phi,
                                          float* S, float* u, void* cuda_stream);
tkphi_status tkphi_static_device_status(void* cuda_stream, int32_t* status_out);
const char* tkphi_static_last_error(void);

/*
 * Selection-only Top-K decode (Sec. 3, Eq. exact_terms and y_TopK = nu_E / Z_E), steps
 * (1)-(2) above.
 *   q         bf16 [batch][n_q_heads][head_dim], one decode query per sequence and head.
 *   topk_host host int32 [batch]; topk_dev device copy.  0 <= topk[b] <= |M_b|
 *             (larger is TKPHI_ERR_INVALID_ARG); topk_max >= max_b topk[b].
 *   idx_out   int32 [batch][n_q_heads][topk_max] or NULL: the retrieved positions
 *             within the sequence (n_sink <= i < L_b - n_tail), ascending, padded
 *             with -1.  Equal scores are broken towards the lower index.
 *   y_out     fp32 [batch][n_q_heads][head_dim].
 * A sequence needs at least one anchor or one retrieved token (else INVALID_ARG).
 */
tkphi_status tkphi_topk_decode(const tkphi_kv_desc* kv, const void* q,
                               const int32_t* topk_host, const int32_t* topk_dev, int32_t topk_max,
                               int32_t* idx_out, float* y_out,
                               void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Length of one dbg_out row of tkphi_decode_step for a given head_dim. */
#define TKPHI_DBG_STRIDE(head_dim) (4 + (head_dim))

/*
 * Top-K+phi decode step (Sec. 4.2-4.3), steps (1)-(5) above, for summaries (S, u)
 * laid out as tkphi_build_summaries writes them.
 *   dbg_out   fp32 [batch][n_q_heads][TKPHI_DBG_STRIDE(head_dim)] or NULL.  Per query
 *             head: [0] m_E = max_{i in E} s_i, [1] sum_{i in E} exp(s_i - m_E),
 *             [2] log Z_hat_R (-inf when the residual was clamped away), [3] the
 *             common log-scale of the merge, [4..] nu_hat_R / Z_hat_R (zeros when clamped).
 *   flags     TKPHI_FLAG_*.
 * Clamp: a residual denominator Z_hat_R <= 0 (a finite-precision artefact of the
 * subtraction, App. C.1) drops both residual terms, so y falls back to nu_E / Z_E.
 * With no anchor and no retrieved token the output is nu_hat_R / Z_hat_R; if that is
 * clamped as well the output row is zero.
 * Generated tokens (Sec. 4.3, Eq. implemented_decode: tokens produced after the prefill
 * stay in the exact branch): append their rows to the cache and pass n_tail + n_gen as the
 * tail-anchor count of the decode call; the mid-region, and with it the meaning of (S, u)
 * built at prefill time with n_tail, is unchanged.  Sequences with different n_gen share a
 * call through n_tail_seq (entry b = n_tail + n_gen_b).
 * Other arguments as for tkphi_topk_decode.
 */
tkphi_status tkphi_decode_step(const tkphi_kv_desc* kv, const tkphi_phi_desc* phi, const void* q,
                               const int32_t* topk_host, const int32_t* topk_dev, int32_t topk_max,
                               const float* S, const float* u,
                               int32_t* idx_out, float* y_out, float* dbg_out, uint32_t flags,
                               void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The paper's own feature map (App. C.2, "Head-wise phi architecture"): a one-block ReZero MLP of
 * hidden width d_emb per head,
 *   g0 = W_s x + b_s;  Delta = W_2 GeLU(W_1 g0 + b_1) + b_2;  g1 = g0 + alpha Delta;  phi(x) = exp(W_o g1 + b_o),
 * GeLU(t) = t Phi(t) with the normal CDF (erf form).  One descriptor holds the maps of one side:
 * n_heads = n_q_heads for phi_q, n_kv_heads for phi_k.  Row-major fp32 device parameters, every
 * pointer 16-byte aligned; d_emb a multiple of 128, at most 512.
 */
typedef struct {
  int32_t d_emb, n_heads;
  const float* w_s; const float* b_s; /* [n_heads][d_emb][head_dim], [n_heads][d_emb] */
  const float* w_1; const float* b_1; /* [n_heads][d_emb][d_emb],    [n_heads][d_emb] */
  const float* w_2; const float* b_2; /* [n_heads][d_emb][d_emb],    [n_heads][d_emb] */
  const float* alpha;                 /* [n_heads] */
  const float* w_o; const float* b_o; /* [n_heads][n_feat][d_emb],   [n_heads][n_feat] */
} tkphi_mlp_desc;

/*
 * Key features of the MLP map (App. C.2) for a whole cache: phi_k(k_t) of EVERY cache row t of every
 * KV head (anchor rows included) is written to phi_k_cache, fp32 [n_kv_heads][T_total][n_feat]
 * (layout as in tkphi_phi_desc).  The four layers run as tensor-core GEMMs over all tokens with
 * bf16 operands (weights and the activations between the layers are rounded to bf16), fp32
 * accumulation, biases, residual and exponent.  Workspace: tkphi_workspace_bytes(kv, NULL, 0,
 * TKPHI_WS_MLP_KEY_FEATURES).  Feed the cache to tkphi_build_summaries_cached and
 * tkphi_decode_step_mlp.
 */
tkphi_status tkphi_mlp_key_features(const tkphi_kv_desc* kv, const tkphi_mlp_desc* mlp_k, float* phi_k_cache,
                                    void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Prefill summary build (Sec. 4.1, Eq. natural_cache) from stored key features: S[b][h] = sum_{i in M_b}
 * v_i phi_k(k_i)^T, u[b][h] = sum phi_k(k_i) with phi_k(k_i) read from row cu_seqlens[b] + i of
 * phi_k_cache (as tkphi_mlp_key_features, or tkphi_build_summaries with a cache, wrote it).  kv->k is
 * validated like every descriptor field (a valid device pointer) but its rows are not read.
 * Outputs, workspace (TKPHI_WS_BUILD) and errors as for tkphi_build_summaries.
 */
tkphi_status tkphi_build_summaries_cached(const tkphi_kv_desc* kv, const float* phi_k_cache, float* S, float* u,
                                          void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Top-K+phi decode step (Sec. 4.2-4.3) with the paper's MLP feature maps (App. C.2): phi_q(q) is
 * evaluated by the library from mlp_q (n_heads = n_q_heads), the retrieved keys' features are taken
 * from phi_k_cache (the MLP is never re-evaluated for keys at decode time).  With TKPHI_FLAG_NOSUB the
 * cache is not read and may be NULL.  Everything else as for tkphi_decode_step; workspace
 * TKPHI_WS_DECODE_STEP.
 */
tkphi_status tkphi_decode_step_mlp(const tkphi_kv_desc* kv, const tkphi_mlp_desc* mlp_q, const float* phi_k_cache,
                                   const void* q, const int32_t* topk_host, const int32_t* topk_dev, int32_t topk_max,
                                   const float* S, const float* u, int32_t* idx_out, float* y_out, float* dbg_out,
                                   uint32_t flags, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * ---------------------------------------------------------------------------------------------
 * Paged cache: writing it, attention over all of it, attention over selected pages.
 *
 * The calls above read a cache that somebody has filled and that lies in one piece per head.  The calls below serve
 * the rest of a serving step on a cache kept in pages: rotate and append the new tokens' keys and values, attend from
 * the new tokens to the whole cache (prefill, chunks of a prompt, decoding), or to the pages that a cheap bound selects.
 * (The paper has no counterpart; exact attention is its baseline y = nu / Z over all keys, Sec. 3, and page selection
 * is one more partial-KV selector beside the exhaustive Top-K of Sec. 5.1.)  A contiguous cache of this library is
 * also a paged one if its sequences start at multiples of page_size rows: page = row / page_size.
 *
 * One descriptor is one step of `batch` sequences.  kv_lens[b] is the sequence's cache length with this step's new
 * tokens, cu_q[b] .. cu_q[b+1]-1 are the rows of its new tokens in k_new, v_new, q and y; they are its last
 * q_len = cu_q[b+1] - cu_q[b] cache positions (q_len 0: the sequence takes no part).  Position t of sequence b is slot
 * t % page_size of page page_table[b][t / page_size]; element (page, head, slot, dim) of k and v is at
 * base + page*stride_page + head*stride_head + slot*stride_token + dim (16-bit elements).
 * Requirements: 1 <= batch <= 1024; head_dim 64 or 128; n_q_heads a multiple of n_kv_heads, at most 16 query heads per
 * KV head; page_size 16, 32, 64 or 128; k, v (and key_bounds) 16-byte aligned; strides multiples of 8 elements that
 * give every element memory of its own (in any order of page, head and slot); cu_q[0] = 0, non-decreasing;
 * 0 <= q_len <= kv_len <= max_pages * page_size (TKPHI_FLAG_FULL_CONTEXT lifts q_len <= kv_len), kv_len <= 2^30.
 * Host and device copies as in the general rules, with one addition for captured graphs: the launches are sized by
 * the host copy of kv_lens, and a replayed graph may find other device lengths as long as each is at most the captured
 * host value and still at least q_len; cu_q must be the captured one.
 *  - Page table: entries behind a sequence's last page are not read.  An entry outside [0, n_pages) is never followed:
 *    its rows are not written, or count as unspecified values, and *status is set to TKPHI_ERR_INVALID_ARG.  Pages that
 *    receive rows must belong to one sequence of the batch; pages that are only read may be shared.
 *  - status: a device int32 owned by the caller and set to 0 by it; the kernels store an error there (a bad page, or
 *    TKPHI_ERR_TIMEOUT) and never clear it.  Required.
 *  - A workspace serves one call at a time: calls that may overlap (other streams, captured graphs that are replayed side
 *    by side) need workspaces of their own.
 *  - Slots at or behind a sequence's length may hold anything, NaN included: nothing read from them reaches a result.  Nor
 *    does an infinity or NaN in the keys or values of a later new token reach the tokens before it.
 *  - key_bounds (optional; needed by tkphi_paged_block_attention): [n_pages][n_kv_heads][2][head_dim] in the cache's
 *    type, the element-wise minimum and maximum of each page's keys.
 */
enum { TKPHI_DTYPE_BF16 = 0, TKPHI_DTYPE_FP16 = 1 };
typedef struct {
  int32_t batch, n_q_heads, n_kv_heads, head_dim;
  int32_t dtype;                  /* TKPHI_DTYPE_*: of the cache, q, y, k_new, v_new and key_bounds */
  int32_t page_size, n_pages, max_pages;
  void* k;                        /* device; written by tkphi_paged_append only */
  void* v;
  int64_t stride_page, stride_head, stride_token;
  const int32_t* page_table;      /* device, [batch][max_pages] */
  const int64_t* kv_lens_host;    /* host,   [batch] */
  const int64_t* kv_lens_dev;     /* device, [batch] */
  const int64_t* cu_q_host;       /* host,   [batch+1] */
  const int64_t* cu_q_dev;        /* device, [batch+1] */
  void* key_bounds;               /* device or NULL */
  int32_t* status;                /* device */
} tkphi_paged_desc;

/* New tokens of one step.  Element (token row t, head h, dim c) of k_new is at t*stride_token + h*stride_head + c, and
 * so on; all pointers 16-byte aligned, all strides multiples of 8 elements (a fused projection's slices work as they
 * are), none of them overlapping the cache.  q and q_out (both or neither): the step's queries, rotated into q_out, which may be q itself (same strides)
 * and otherwise must not overlap it. */
typedef struct {
  const void* k_new; int64_t k_stride_token, k_stride_head;  /* [total_q][n_kv_heads][head_dim] */
  const void* v_new; int64_t v_stride_token, v_stride_head;
  const void* q;     int64_t q_stride_token, q_stride_head;  /* [total_q][n_q_heads][head_dim] or NULL */
  void* q_out;       int64_t o_stride_token, o_stride_head;
  const float* inv_freq;          /* device, [rot_dim / 2] angle per position; NULL if rot_dim is 0 */
  int32_t rot_dim;                /* dims rotated, from dim 0: a multiple of 16, at most head_dim; 0: none */
  int32_t pairs;                  /* 0: dim c turns with dim c + rot_dim/2; 1: dim 2c with dim 2c + 1 */
  const int64_t* positions;       /* device, [total_q] positions of the rotation, or NULL: the cache positions */
} tkphi_append_desc;

/*
 * Rotates the new keys (and queries) by their positions and writes keys and values into the cache's pages:
 * (a, c) -> (a cos w - c sin w, c cos w + a sin w) with w = position * inv_freq in 64 bits, the products in 32, rounded
 * once.  With key_bounds, the bounds of every page that receives a row are recomputed from its rows below the new
 * length (so they are right after a rollback of drafted tokens, too).  No workspace.
 */
tkphi_status tkphi_paged_append(const tkphi_paged_desc* kv, const tkphi_append_desc* step, void* cuda_stream);

/* Flag of tkphi_paged_attention: every new token sees all kv_len rows of its sequence instead of those up to its own
 * position.  A sequence may then be shorter than its number of new tokens, or empty. */
enum { TKPHI_FLAG_FULL_CONTEXT = 2 };

/* Workspace kinds of tkphi_paged_workspace_bytes. */
enum { TKPHI_WS_PAGED_ATTENTION = 4, TKPHI_WS_PAGED_BLOCK_ATTENTION = 5 };

/* Pages that tkphi_paged_block_attention reads for a token that sees n pages (its own is the last): the first
 * n_sink_pages, the last n_tail_pages (>= 1), and of those between the topk_pages with the largest bounds. */
typedef struct {
  int32_t n_sink_pages, n_tail_pages, topk_pages;
} tkphi_page_selection;

/* Bytes of workspace (256-byte aligned device memory, contents irrelevant) of the paged calls; selection may be NULL
 * for TKPHI_WS_PAGED_ATTENTION.  0 on invalid arguments.  The size goes by this step's cu_q and kv_lens (host copies): ask
 * for every step, or for those that the workspace has to serve; a call that finds it too small is refused. */
size_t tkphi_paged_workspace_bytes(const tkphi_paged_desc* kv, const tkphi_page_selection* selection, int which);

/*
 * Attention of the new tokens over their sequences' caches: y = softmax(scale q.k) v over the visible keys (the
 * token's own position included), all new tokens of all sequences in one call, whatever mix of lengths.
 * Scores, sums and products are accumulated in fp32.  A sequence whose new tokens have at most 16 query heads of one KV
 * head together (q_len * n_q_heads / n_kv_heads <= 16) has its probabilities multiplied as pairs of 16-bit numbers; with
 * more of them they are rounded to 16 bits once, fp16 ones by up to 2^-32 of the largest where they are below 2^-21 of it.
 * So a token's result differs in its last bits with the number of tokens that come with it.
 *   q     [total_q][n_q_heads][head_dim], y_out likewise, both in the cache's type, contiguous, 16-byte aligned.
 *         y_out may be q itself; otherwise they must not overlap.
 *   lse   fp32 [total_q][n_q_heads] or NULL: log of the softmax denominator, log sum exp(scale q.k), with which
 *         results over disjoint sets of keys can be joined.  A token that sees nothing (no keys, or none whose score
 *         is above -inf) gets y = 0, lse = -inf; one with a score that is no number or +inf gets NaN in both.
 *   scale 0 for 1/sqrt(head_dim), else finite and positive.
 *   flags TKPHI_FLAG_FULL_CONTEXT or 0.
 */
tkphi_status tkphi_paged_attention(const tkphi_paged_desc* kv, const void* q, void* y_out, float* lse_out, float scale,
                                   uint32_t flags, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Attention over selected pages.  For every new token and KV head the middle pages are ordered by the largest score
 * that a key within their bounds could have with one of the group's query heads,
 *   bound = max over the group of sum_c max(q_c lo_c, q_c hi_c)
 * (evaluated in 64 bits, 0 * inf as 0, heads whose sum is no number left out; equal bounds go to the lower page), and attention runs exactly over the rows of the selected
 * pages up to the token's position.  At most 131,072 pages per sequence.  A token that sees no more than n_sink_pages + n_tail_pages + topk_pages pages
 * gets plain attention.
 *   page_idx_out  int32 [total_q][n_kv_heads][n_sink_pages + n_tail_pages + topk_pages] or NULL: the selected pages
 *                 (indices into the sequence's page table row), ascending, padded with -1.
 * Other arguments as for tkphi_paged_attention.
 */
tkphi_status tkphi_paged_block_attention(const tkphi_paged_desc* kv, const tkphi_page_selection* selection,
                                         const void* q, void* y_out, float* lse_out, int32_t* page_idx_out, float scale,
                                         void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Reads the device status word that the kernels of the last call using this
 * workspace set (0 = fine; TKPHI_ERR_TIMEOUT if a bounded wait ran out).  Waits
 * for the stream.  *status_out is a host int.  (The workspaces of the paged calls
 * hold no such word: theirs is tkphi_paged_desc.status.)
 */
tkphi_status tkphi_device_status(const void* workspace, void* cuda_stream, int32_t* status_out);

/*
 * Self-test of the error path of the bounded device-side waits (no counterpart in the
 * paper).  Every wait inside the kernels (on a TMA copy, an MMA completion, a hand-off
 * between warps) gives up after a fixed number of polls, raises a flag that makes the
 * other warps of its CTA leave their loops, and the CTA stores TKPHI_ERR_TIMEOUT in the
 * status word at the head of the workspace before it returns.  This entry point runs a
 * one-CTA kernel through exactly that path: one warp waits, with a limit of 4096 polls, on
 * a barrier that nothing ever arrives on, a second warp waits on a barrier the first one
 * would have signalled.  The kernel returns by itself within microseconds; afterwards
 * tkphi_device_status(workspace) reads TKPHI_ERR_TIMEOUT, and the next ordinary call on
 * the same workspace sets the word back to 0.  workspace: device memory, 256-byte
 * aligned, at least 256 bytes.
 */
tkphi_status tkphi_selftest_timeout(void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Optional per-kernel timing for benchmarks (no counterpart in the paper).  While
 * enabled, every launch the library makes is bracketed by CUDA events on the caller's
 * stream (the events are host objects; no device memory is allocated).  Not
 * thread-safe; leave it off in production.  tkphi_kernel_timing_read waits for the
 * recorded events, adds up milliseconds and launch counts per kernel kind into the
 * two host arrays of TKPHI_KERNEL_KINDS entries, and clears the record.
 */
enum {
  TKPHI_KERNEL_SCORE = 0,           /* key scoring (streams the mid-region keys) */
  TKPHI_KERNEL_SELECT = 1,          /* exact Top-K over the score rows; query-side feature work */
  TKPHI_KERNEL_EXACT_RESIDUAL = 2,  /* exact branch, subtraction, residual, merge */
  TKPHI_KERNEL_BUILD = 3,           /* prefill summary build */
  TKPHI_KERNEL_MEMSET = 4,          /* clearing counters when there is nothing to score */
  TKPHI_KERNEL_CACHED_Z = 5,        /* <phi_q, cached phi_k row> of the retrieved tokens (phi_k_cache given) */
  TKPHI_KERNEL_MLP = 6,             /* the layers of the MLP key feature map (weight conversion included) */
  TKPHI_KERNEL_PAGED_APPEND = 7,    /* rotation and append to a paged cache */
  TKPHI_KERNEL_PAGED_SELECT = 8,    /* page bounds and selection */
  TKPHI_KERNEL_PAGED_ROWS = 9,      /* attention of few query rows over a paged cache, and its join */
  TKPHI_KERNEL_PAGED_TILES = 10,    /* attention of many query rows over a paged cache, and its join */
  TKPHI_KERNEL_KINDS = 11
};
void tkphi_kernel_timing_enable(int32_t on);
tkphi_status tkphi_kernel_timing_read(float* ms_out, int32_t* count_out);

/* Message for the last error returned on the calling thread ("" if none). */
const char* tkphi_last_error(void);

/* Library version, e.g. 100 for 0.1.0. */
int32_t tkphi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* TKPHI_H */
