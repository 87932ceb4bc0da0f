/*
 * lrqk.h — C ABI of the LRQK decode-step hot path for AMD MI355X (gfx950).
 *
 * LRQK ("Low Rank Query and Key" attention) keeps, per head, a rank-r key
 * factor A_K (l x r) on the GPU and the full-precision K/V rows in host
 * memory.  One decode step (Alg. 2, steps "proxy attention", "fetch missing",
 * "merge", followed by Attention(q, K_Omega, V_Omega) of Sec. 4.3) is:
 *
 *   a1  proxy scores   s = A_K q_hat^T                     (Alg. 2, top-k line)
 *   a2  selection      Omega_k = top(s, k) over [0, l-w),  Omega_l = [l-w, l)
 *                                                          (Sec. 4.1 "active" / "lite" tokens)
 *   a3  hit/miss       which of Omega_k already sit in the GPU cache, and where
 *                      the missing ones go                 (Sec. 4.1 hit-and-miss cache)
 *   a4  fetch          copy only the missing K/V rows host -> GPU cache
 *                                                          (Alg. 2 "Fetch missing", "merge")
 *   a5  attention      exact softmax attention of q over the k+w selected rows
 *                                                          (Sec. 4.3, last sentence)
 *
 * Conventions
 *   - Notation follows the paper: l context length, d head dimension, r rank,
 *     k active (top-k) tokens, w lite (recent) tokens.  B batch, Hq query heads,
 *     Hkv key/value heads, G = Hq/Hkv query heads per KV head, C cache slots
 *     per (batch, query head).
 *   - A_K, K, V and the lite rows are stored per (batch, KV head) and shared by
 *     the G query heads of the group; scores, selection, cache state, cache
 *     rows and outputs are per (batch, query head).  Query head h uses KV head
 *     h / G.
 *   - All arrays are dense, row-major, last index fastest, no padding.
 *   - "device" pointers are HIP device memory on the current device; "host"
 *     pointers are ordinary process memory; "pinned" is host memory allocated
 *     with hipHostMalloc (page-locked, device-visible).
 *   - Every buffer is allocated and owned by the caller.  The library keeps no
 *     pointer after a call returns, except inside an lrqk_plan.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     Unless stated otherwise a call only enqueues work and returns.
 *   - Every entry point returns an int status: LRQK_OK (0) or a negative
 *     lrqk_status.  Arguments are validated on the host before anything is
 *     enqueued; on a validation error nothing is written.
 *   - Device pointers must be 16-byte aligned.
 */
#ifndef LRQK_H
#define LRQK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LRQK_VERSION 200 /* major*10000 + minor*100 + patch */

typedef enum lrqk_status {
  LRQK_OK = 0,
  LRQK_EINVAL = -1, /* null or misaligned pointer, bad enum value, bad handle   */
  LRQK_ESHAPE = -2, /* sizes inconsistent or outside the supported range         */
  LRQK_EHIP = -3,   /* a HIP runtime call failed; see lrqk_last_hip_error()      */
  LRQK_ENOMEM = -4, /* workspace too small, or an allocation in plan_create failed */
  LRQK_ESTATE = -5  /* the cache state handed in is unusable (see lrqk_fetch_misses)   */
} lrqk_status;

enum { LRQK_KV_BF16 = 0, LRQK_KV_F32 = 1 };

/* How lrqk_decode_step / lrqk_fetch_misses move missing rows (step a4). */
enum {
  LRQK_FETCH_STAGED = 0, /* miss list -> host, host gathers rows into a pinned staging
                            buffer, one hipMemcpyAsync on the plan's side stream, then a
                            scatter kernel into the cache slots                        */
  LRQK_FETCH_DIRECT = 1, /* the GPU reads the rows straight out of the pinned host store
                            (device-visible host memory) and writes the cache slots; no host
                            synchronisation.  lrqk_fetch_misses does it in a kernel of its
                            own; lrqk_decode_step does it inside the attention kernel, so the
                            host-link reads overlap the HBM reads of the rows that hit      */
  LRQK_FETCH_GROUP = 2   /* as DIRECT, with the host link shared inside a KV group: K and V
                            exist once per KV head (Sec. 4, preliminaries), so a position that
                            several query heads of a group miss in the same step is one host
                            row; it is read once and written into the slot of each of those
                            heads.  The caches end up exactly as with the other modes; fewer
                            rows cross the link when the heads of a group want the same
                            tokens.  lrqk_decode_step: the shared fetch runs in one launch
                            with the attention over the rows that hit, the fetched rows are
                            attended by a second launch                                     */
};
/* May be OR-ed into the `mode` of lrqk_decode_step: estimate the candidate thresholds of the
 * selection from a sample of this step's proxy scores even though the layer carries thresholds
 * from its previous step (lrqk_layer.sel_thr).  For the first decode step of a sequence and
 * after anything that changes the score distribution wholesale.  Results never depend on it,
 * only speed does. */
#define LRQK_SELECT_FRESH 0x100

/*
 * Problem sizes of one layer's decode step.
 *   d        head dimension; only 128 is supported.
 *   r        rank of the factors, 4 <= r <= 128, multiple of 4.
 *   k        active tokens picked by proxy score, 1 <= k <= l - w, k <= 4096.
 *   w        lite tokens = the last w positions, always attended, 0 <= w <= 1024.
 *   C        cache slots per (batch, query head), k <= C <= 8192.
 *   kv_dtype element type of K/V rows (host store, cache, lite rows).
 *   scale    softmax scale applied to q.k (the usual 1/sqrt(d)).
 *   l_cap    rows allocated per head in the arrays that grow with the context (A_K, K_host,
 *            V_host, slot_of): their row stride.  0 means l (no room to grow); otherwise
 *            l <= l_cap < 2^24.  Where this header writes [.., l, ..] for one of those four
 *            arrays, read [.., l_cap, ..] with the first l rows in use.
 * Requirements: B >= 1, Hkv >= 1, Hq a multiple of Hkv, Hq/Hkv <= 8, l >= 1, l < 2^24.
 */
typedef struct lrqk_shape {
  int32_t B, Hq, Hkv, d, l, r, k, w, C;
  int32_t kv_dtype;
  float scale;
  int32_t l_cap;
} lrqk_shape;

/* Which call a workspace is sized for (lrqk_workspace_bytes). */
enum { LRQK_WS_SELECT = 1, LRQK_WS_ATTEND = 2, LRQK_WS_UPDATE = 3, LRQK_WS_PREFILL = 4 };

int lrqk_version(void);
const char* lrqk_status_string(int status);
/* Raw hipError_t of the most recent failing HIP call made by this library in
 * the calling thread (0 if none). */
int lrqk_last_hip_error(void);

/* Host-only check of a shape against the limits above. LRQK_OK / LRQK_EINVAL / LRQK_ESHAPE. */
int lrqk_validate_shape(const lrqk_shape* shape);

/* Bytes of device workspace the given call needs for this shape (0 on a bad
 * shape or selector).  Workspace contents need no initialisation. */
size_t lrqk_workspace_bytes(const lrqk_shape* shape, int which);

/*
 * a1 — proxy attention scores (Alg. 2, "compute proxy attention"; abstract: O(lr) per step).
 *   scores[b,h,i] = sum_{j<r} A_K[b, h/G, i, j] * q_hat[b, h, j],   i in [0, l)
 * accumulated in fp32 as one fused-multiply-add chain, j ascending, starting
 * from 0.0f, so the result is reproducible bit for bit.
 *   A_K     device, fp32 [B, Hkv, l, r]   read
 *   q_hat   device, fp32 [B, Hq, r]       read
 *   scores  device, fp32 [B, Hq, l]       written
 */
int lrqk_proxy_scores(const lrqk_shape* shape, const float* A_K, const float* q_hat,
                      float* scores, void* stream);

/*
 * a2 — active-token selection (Alg. 2, top(., k); Sec. 4.1: active + lite tokens).
 * For every (b,h): the k positions in [0, l-w) with the largest score; equal
 * scores are ordered by lower position first (-0.0f and +0.0f compare equal;
 * NaN scores are not supported).  Written in ascending position order.  The
 * lite set [l-w, l) is implicit and never listed.
 *   scores     device, fp32 [B, Hq, l]   read
 *   sel_idx    device, int32 [B, Hq, k]  written
 *   workspace  device, >= lrqk_workspace_bytes(shape, LRQK_WS_SELECT) bytes, 256-byte aligned
 * LRQK_ENOMEM if ws_bytes is too small.
 */
int lrqk_select_topk(const lrqk_shape* shape, const float* scores, int32_t* sel_idx,
                     void* workspace, size_t ws_bytes, void* stream);

/*
 * Cache state of one layer (all device memory):
 *   slot_of   int32 [B, Hq, l]  slot holding token i, or -1 if i is not on the GPU
 *   token_of  int32 [B, Hq, C]  token held by a slot, or -1 if the slot is empty
 *   last_used int32 [B, Hq, C]  step at which the slot's token was last selected, -1 if empty
 * slot_of and token_of are mutually inverse on the resident set.  Whether a token is resident is
 * read from slot_of alone: after slot_of[., i] = -1 (lrqk_append_token, or a caller that replaces
 * rows of a context it has cut back) the next step that selects i fetches its row, whatever
 * token_of says of the slot that held it.
 * lrqk_cache_init sets all three to -1 (an empty cache).
 */
int lrqk_cache_init(const lrqk_shape* shape, int32_t* slot_of, int32_t* token_of,
                    int32_t* last_used, void* stream);

/*
 * a3 — hit/miss resolution (Sec. 4.1: only tokens missing from the GPU cache are
 * fetched; Sec. 5.3 defines the miss rate as fetched rows / selected rows).
 * The paper's cache holds exactly the k active tokens; with C >= k slots a
 * replacement rule is needed and this library uses least-recently-selected:
 *   for each selected token, ascending position: resident -> hit, its slot's
 *   last_used becomes `step`; otherwise miss.  Victim slots are the slots whose
 *   last_used != step, ordered by (last_used ascending, slot ascending); the
 *   j-th miss (ascending position) takes the j-th victim; the evicted token's
 *   slot_of becomes -1; token_of / slot_of / last_used are updated.
 * With C == k this is the paper's behaviour (the cache ends up holding Omega_k).
 *   sel_idx   device int32 [B,Hq,k]  read; ascending, distinct, in [0, l-w)
 *   step      >= 0 and larger than every last_used currently stored
 *   slot_of, token_of, last_used     read and updated in place
 *   sel_slot  device int32 [B,Hq,k]  written: slot of sel_idx[..j] after the step
 *   hit       device uint8 [B,Hq,k]  written: 1 hit, 0 miss
 *   miss_tok, miss_slot device int32 [B,Hq,k]  written: first n_miss entries = the
 *             missing tokens (ascending) and the slots they were given; rest untouched
 *   n_miss    device int32 [B,Hq]    written
 * A head whose input breaks the contract (a position outside [0,l), or too
 * few victims because `step` was reused) does not fault: the offending entries
 * get sel_slot = -1 and that head's n_miss is written as -1.
 */
int lrqk_cache_resolve(const lrqk_shape* shape, const int32_t* sel_idx, int32_t step,
                       int32_t* slot_of, int32_t* token_of, int32_t* last_used,
                       int32_t* sel_slot, uint8_t* hit, int32_t* miss_tok, int32_t* miss_slot,
                       int32_t* n_miss, void* stream);

/*
 * a5 — exact attention over the selected rows (Sec. 4.3: Attention(q_t, K_Omega, V_Omega)
 * with the original q, K, V).
 *   out[b,h,:] = sum_{i in Omega} p_i V_i,  p = softmax_i(scale * q[b,h,:] . K_i)
 * Omega = the k cache rows named by sel_slot plus the w lite rows.  fp32
 * accumulation, max-subtracted softmax.  Entries of sel_slot outside [0, C)
 * are skipped.
 *   q                device fp32 [B,Hq,d]
 *   cacheK, cacheV   device kv_dtype [B,Hq,C,d]
 *   sel_slot         device int32 [B,Hq,k]
 *   liteK, liteV     device kv_dtype [B,Hkv,w,d]: the rows of positions l-w .. l-1, kept as a
 *                    ring: row j holds the position p of [l-w, l) with p mod w == j (the
 *                    attention does not depend on their order; may be NULL when w == 0)
 *   out              device fp32 [B,Hq,d]   written
 *   workspace        device, >= lrqk_workspace_bytes(shape, LRQK_WS_ATTEND), 256-byte aligned
 */
int lrqk_sparse_attend(const lrqk_shape* shape, const float* q, const void* cacheK,
                       const void* cacheV, const int32_t* sel_slot, const void* liteK,
                       const void* liteV, float* out, void* workspace, size_t ws_bytes,
                       void* stream);

/*
 * a5 for callers that cannot allocate: code under HIP graph capture, tight serving loops and
 * harnesses that forbid hipMalloc, which have no workspace to hand over either.  Same
 * arguments, kernels and results as lrqk_sparse_attend, without `workspace`: the partial
 * softmax states sit in a fixed array of LRQK_NOALLOC_SCRATCH_BYTES of device memory inside
 * the library (one copy per GPU, held until the process ends).  The call allocates and frees
 * nothing, on the host side of HIP or the device.
 *   LRQK_ENOMEM if lrqk_workspace_bytes(shape, LRQK_WS_ATTEND) exceeds the array (nothing is
 *   enqueued).  At the headline shape (32 heads, k = 2048, w = 64) the call needs 1.2 MB.
 * Every call on a GPU uses that GPU's one array: two calls whose work overlaps on the same
 * GPU (different streams, or threads) race.  Calls on one stream are ordered and safe.
 */
#define LRQK_NOALLOC_SCRATCH_BYTES (4u << 20)
int lrqk_sparse_attend_noalloc(const lrqk_shape* shape, const float* q, const void* cacheK,
                               const void* cacheV, const int32_t* sel_slot, const void* liteK,
                               const void* liteV, float* out, void* stream);

/*
 * A plan owns what the fused step and the fetch leg need beyond the caller's
 * buffers: device workspace, a side stream with events, and pinned staging
 * memory sized for `max_shape` (every later call must use a shape whose
 * B*Hq, l, k, w, C do not exceed it).  Created on the current device.
 */
typedef struct lrqk_plan lrqk_plan;
int lrqk_plan_create(const lrqk_shape* max_shape, lrqk_plan** plan_out);
int lrqk_plan_destroy(lrqk_plan* plan);

/*
 * a4 — fetch the missing rows (Alg. 2: "Fetch missing k_i, v_i from CPU K, V", "merge").
 * For every (b,h) and j < n_miss[b,h]:
 *   cacheK[b,h,miss_slot[b,h,j],:] = K_host[b,h/G,miss_tok[b,h,j],:]   (same for V), a bit copy.
 *   K_host, V_host  pinned host memory, kv_dtype [B,Hkv,l,d]
 *   miss_tok, miss_slot, n_miss  device, as written by lrqk_cache_resolve
 *   mode  LRQK_FETCH_STAGED: synchronises `stream` once to read the miss list on the
 *         host, then copies on the plan's side stream and makes `stream` wait for it.
 *         LRQK_FETCH_DIRECT, LRQK_FETCH_GROUP: one kernel on `stream`, no host
 *         synchronisation (GROUP needs the miss lists ascending, as lrqk_cache_resolve and
 *         lrqk_decode_step write them).
 *   total_miss_out  host int64*, optional: total rows fetched (STAGED only; the others write -1).
 * A head with n_miss < 0 (lrqk_cache_resolve could not place its misses): STAGED returns
 * LRQK_ESTATE after the synchronisation, with nothing copied; DIRECT and GROUP, which never see
 * the lists on the host, skip that head (its n_miss stays the only report).
 */
int lrqk_fetch_misses(lrqk_plan* plan, const lrqk_shape* shape, const void* K_host,
                      const void* V_host, const int32_t* miss_tok, const int32_t* miss_slot,
                      const int32_t* n_miss, void* cacheK, void* cacheV, int mode,
                      int64_t* total_miss_out, void* stream);

/* Buffers of one layer for the fused step. Device unless marked pinned. */
typedef struct lrqk_layer {
  float* A_K;          /* fp32 [B,Hkv,l,r]                       (written only by lrqk_append_token) */
  void* K_host;        /* pinned, kv_dtype [B,Hkv,l,d]           (likewise) */
  void* V_host;        /* pinned, kv_dtype [B,Hkv,l,d]           (likewise) */
  void* liteK;         /* kv_dtype [B,Hkv,w,d], ring of the last w rows (likewise) */
  void* liteV;         /* kv_dtype [B,Hkv,w,d]                   (likewise) */
  int32_t* slot_of;    /* int32 [B,Hq,l]  in/out */
  int32_t* token_of;   /* int32 [B,Hq,C]  in/out */
  int32_t* last_used;  /* int32 [B,Hq,C]  in/out */
  void* cacheK;        /* kv_dtype [B,Hq,C,d] in/out */
  void* cacheV;        /* kv_dtype [B,Hq,C,d] in/out */
  float* sel_thr;      /* fp32 [B,Hq] in/out, or NULL: candidate threshold of the selection
                          carried from one step of this layer to the next (see lrqk_decode_step);
                          set up with lrqk_select_state_init.  Only lrqk_decode_step uses it */
} lrqk_layer;

/*
 * Marks the carried selection thresholds of a layer as unknown (every entry NaN).
 *   sel_thr  device fp32 [B,Hq]  written
 */
int lrqk_select_state_init(const lrqk_shape* shape, float* sel_thr, void* stream);

/* Optional device outputs of the fused step (any may be NULL): the integer
 * results of a2/a3, bit-identical to what the separate calls produce. */
typedef struct lrqk_step_debug {
  int32_t* sel_idx;   /* [B,Hq,k] */
  int32_t* sel_slot;  /* [B,Hq,k] */
  uint8_t* hit;       /* [B,Hq,k] */
  int32_t* miss_tok;  /* [B,Hq,k] */
  int32_t* miss_slot; /* [B,Hq,k] */
  int32_t* n_miss;    /* [B,Hq]   */
  int32_t* link_rows; /* [B,Hkv]  LRQK_FETCH_GROUP only: rows read from the host store per KV
                         head = size of the union of its group's miss lists (cleared and
                         counted only when this pointer is given) */
} lrqk_step_debug;

/*
 * a1..a5 as one call (Alg. 2 from the proxy-attention line to the attention of
 * Sec. 4.3; Fig. 2: selection, then a small cache load overlapped with attention).
 * Scores never leave the library's workspace (for the shapes the filtered proxy-score
 * pass supports they are not even materialised).  STAGED: attention over the hit rows and
 * the lite rows runs on `stream` while the missing rows travel on the plan's side stream
 * and are attended afterwards; partial results are merged.  DIRECT: one attention launch
 * over all rows, the missing ones read from the host store and written to their slots on
 * the way.
 * Selection (shapes the filtered proxy-score pass supports): the pass over A_K keeps only the
 * positions whose score reaches a per-head candidate threshold, and the selection is made
 * exactly among those; a head whose candidates turn out unusable (fewer than k, or so many that
 * more than half of its positions, or more than 8192 equal scores, would have to be gone through)
 * is redone exactly from all its scores, so the threshold affects speed, never the result.  The
 * threshold is estimated from a sample of this step's scores (two small launches) when
 * layer->sel_thr is NULL or `mode` carries LRQK_SELECT_FRESH; otherwise it is
 * layer->sel_thr[b,h] * |q_hat[b,h]|, the value the previous step's selection left there (the
 * score at rank 1.5 k, per unit of |q_hat|), and every step rewrites sel_thr for the next one.
 * An entry that is NaN (lrqk_select_state_init) sends its head down the exact, slow route.
 *   q_hat  device fp32 [B,Hq,r];  q  device fp32 [B,Hq,d];  out  device fp32 [B,Hq,d]
 *   step   as in lrqk_cache_resolve
 *   mode   LRQK_FETCH_STAGED (one host synchronisation per call, to read the miss
 *          list), LRQK_FETCH_DIRECT or LRQK_FETCH_GROUP (fully asynchronous), optionally
 *          | LRQK_SELECT_FRESH
 *   dbg    optional
 *   total_miss_out  host int64*, optional (STAGED: rows fetched; DIRECT, GROUP: -1)
 */
int lrqk_decode_step(lrqk_plan* plan, const lrqk_shape* shape, int32_t step,
                     const lrqk_layer* layer, const float* q_hat, const float* q, float* out,
                     int mode, const lrqk_step_debug* dbg, int64_t* total_miss_out,
                     void* stream);

/*
 * u1 — decode-time update of the factors (Alg. 2, from the initial guess of k_hat to the two
 * gradient steps on B_Q and B_K; Sec. 4.2 decode objective and update rules; App. A.2 step
 * lengths).  Runs BEFORE the step's proxy scores: it produces the q_hat that lrqk_proxy_scores
 * / lrqk_decode_step take, and the k_hat that lrqk_append_token adds to A_K.
 * For the new projections q_t (per query head) and k_t (per KV head):
 *   k_hat <- k B_K^T (B_K B_K^T)^-1                                   (lambda_d1 = 0 guess)
 *   n_iter times:
 *     q_hat <- m_lq M_rq^-1 for every query head, with
 *        m_lq = q B_Q^T + lambda_d1 (q.k) k_hat + lambda_d2 (q K_Om^T) A_Om
 *        M_rq = B_Q B_Q^T + lambda_d1 k_hat^T k_hat + lambda_d2 A_Om^T A_Om
 *     k_hat <- (k B_K^T + lambda_d1 sum_g (q_g.k) q_hat_g)
 *              (B_K B_K^T + lambda_d1 sum_g q_hat_g^T q_hat_g)^-1     (sums over the G query
 *              heads that share the KV head; G = 1 gives the paper's rule)
 *   B_Q <- B_Q - eta_Q q_hat^T (q_hat B_Q - q),  B_K <- B_K - eta_K k_hat^T (k_hat B_K - k),
 *   each eta the exact minimiser along its gradient; a zero gradient leaves B unchanged.
 * Omega = the rows attended at the previous step: the previous selection (A_K rows at
 * sel_idx_prev, K rows in the cache slots sel_slot_prev) and the lite window [l-w, l) (A_K
 * rows l-w .. l-1, K rows in layer->liteK); q K_Om^T is the raw dot product.  Entries of the
 * previous selection with a position outside [0, l) or a slot outside [0, C) are left out.
 * The loop runs exactly n_iter rounds (the paper uses at most 2); there is no tolerance test.
 * Sums over rows are fp32 (App. B.1), the r x r systems fp64 (fp32 at r <= 16), results fp32.
 * Supported ranks: r in {8, 16, 32, 64}.
 *   layer          A_K, cacheK and liteK are read (device)
 *   sel_idx_prev, sel_slot_prev  device int32 [B,Hq,k], as written by the previous step
 *   q              device fp32 [B,Hq,d]
 *   k_new          device kv_dtype [B,Hkv,d]
 *   B_Q            device fp32 [B,Hq,r,d]   updated in place
 *   B_K            device fp32 [B,Hkv,r,d]  updated in place
 *   lambda_d1, lambda_d2  >= 0, finite;  1 <= n_iter <= 64
 *   q_hat          device fp32 [B,Hq,r]   written
 *   k_hat          device fp32 [B,Hkv,r]  written
 *   workspace      device, >= lrqk_workspace_bytes(shape, LRQK_WS_UPDATE), 256-byte aligned
 * LRQK_ESHAPE for an unsupported rank, LRQK_ENOMEM if ws_bytes is too small.
 */
int lrqk_factor_update(const lrqk_shape* shape, const lrqk_layer* layer,
                       const int32_t* sel_idx_prev, const int32_t* sel_slot_prev, const float* q,
                       const void* k_new, float* B_Q, float* B_K, float lambda_d1,
                       float lambda_d2, int32_t n_iter, float* q_hat, float* k_hat,
                       void* workspace, size_t ws_bytes, void* stream);

/*
 * u2 — the new token joins the context (Alg. 2: A_K <- [A_K; k_hat_t], K_Omega <- [K'; k_t],
 * V_Omega <- [V'; v_t], "Async k_t, v_t to CPU").  With l = shape->l the current length:
 *   A_K[b,kv,l,:] = k_hat[b,kv,:];  K_host[b,kv,l,:] = k_new[b,kv,:];  V_host likewise (bit
 *   copies, written by the GPU into the pinned store: asynchronous to the host, complete
 *   when the work enqueued on `stream` has finished);  the lite ring row l mod w (which held
 *   position l - w) receives k_new / v_new;  slot_of[b,h,l] = -1.
 * Afterwards the context has l + 1 rows: the caller passes shape->l + 1 to the following
 * calls (the new token is then inside the lite window [l+1-w, l+1), always attended).
 * Needs room for the row: shape->l_cap > shape->l, else LRQK_ESHAPE.
 *   layer   A_K, K_host, V_host, liteK, liteV, slot_of are written as described
 *   k_hat   device fp32 [B,Hkv,r]      (from lrqk_factor_update)
 *   k_new, v_new  device kv_dtype [B,Hkv,d]
 */
int lrqk_append_token(const lrqk_shape* shape, const lrqk_layer* layer, const float* k_hat,
                      const void* k_new, const void* v_new, void* stream);

/*
 * p1 — prefill factorisation (Alg. 1; Sec. 4.1 "Prefill": Q K^T ~ A_Q A_K^T with Q ~ A_Q B_Q,
 * K ~ A_K B_K, solved by alternating closed-form updates; App. A.1).  Produces the A_K that
 * the decode step scans and the B_Q, B_K that lrqk_factor_update continues from.
 * Starting from the A_Q, A_K handed in (the paper draws them from N(0,1); the caller draws),
 * n_iter rounds of
 *   B_Q <- (A_Q^T A_Q)^-1 A_Q^T Q                                  per query head
 *   B_K <- (A_K^T A_K)^-1 A_K^T K                                  per KV head
 *   A_K <- K (sum_g Q_g^T A_Q,g + lambda_pK B_K^T)
 *            (sum_g A_Q,g^T A_Q,g + lambda_pK B_K B_K^T)^-1        per KV head, sums over the
 *                                                                  G query heads of its group
 *   A_Q <- Q (K^T A_K + lambda_pQ B_Q^T)(A_K^T A_K + lambda_pQ B_Q B_Q^T)^-1   per query head
 * in this order (G = 1 gives the paper's rules).  B_Q, B_K are those computed at the top of
 * the last round.  Exactly n_iter rounds (the paper uses at most 2); no convergence test.
 * fp32 results (App. B.1): fp32 operands enter the matrix cores as sums of three bf16 terms,
 * d x d sums and the r x d algebra are fp64.  The sums over A_Q and A_K follow from the d x d sums
 * of Q and K; those are good enough for the result not to be further off than with fp32 sums over
 * A_Q and A_K themselves, also where queries and keys are strong in different directions.
 * Supported ranks: r in {8, 16, 32, 64}.
 * Of `shape`, B, Hq, Hkv, d, l, r, kv_dtype and l_cap are used.
 *   Q     device kv_dtype [B,Hq,l,d]     read
 *   K     device kv_dtype [B,Hkv,l,d]    read
 *   A_Q   device fp32 [B,Hq,l,r]         in: initial values, out: result
 *   A_K   device fp32 [B,Hkv,l_cap,r]    in: initial values, out: result (rows >= l untouched)
 *   B_Q   device fp32 [B,Hq,r,d]         written
 *   B_K   device fp32 [B,Hkv,r,d]        written
 *   lambda_pQ, lambda_pK  >= 0, finite;  1 <= n_iter <= 64
 *   workspace  device, >= lrqk_workspace_bytes(shape, LRQK_WS_PREFILL), 256-byte aligned
 * A_Q^T A_Q and A_K^T A_K must be positive definite (they are for generic inputs with l >= r).
 */
int lrqk_prefill_factorize(const lrqk_shape* shape, const void* Q, const void* K, float* A_Q,
                           float* A_K, float* B_Q, float* B_K, float lambda_pQ, float lambda_pK,
                           int32_t n_iter, void* workspace, size_t ws_bytes, void* stream);

/*
 * Paged K/V cache.  Before a prompt is factorised (p1) its tokens run through the model in chunks,
 * each chunk attending exactly to all positions up to its own; drafted tokens are verified in the
 * same way, and so is a sequence decoded that is too short for a selection to pay.  K and V of such
 * sequences lie in pages of a pool that several sequences share:
 *
 *   lrqk_pages_append   the new tokens' rows go into their pages, in 8 or 4 bits if the pages hold those
 *   lrqk_chunk_attend   exact attention of the new tokens over the paged rows
 *   lrqk_pages_read     rows of the pages as dense per-head arrays: what lrqk_prefill_factorize, the
 *                       host store (K_host, V_host) and the lite rows are made from
 *
 * Sequence b has kv_len[b] positions, the last n = start[b+1] - start[b] of which are its new tokens
 * (n >= 0; as long as start is ascending, each sequence may have another number).  Token i of them
 * is row start[b] + i of the packed arrays and position kv_len[b] - n + i.  Position p is row
 * p mod page of page table[b][p / page].
 *   - A table entry outside [0, n_pages) is no page: rows written to it are dropped, rows read from it
 *     are left alone in the output, positions on it take no part in an attention.  Several
 *     sequences may share a page (a common prefix).  A row that is written twice at a time (by two
 *     sequences of a call, by two entries of a table with the same page, by calls that overlap) holds
 *     parts of either, in 8 or 4 bits perhaps the codes of one under the scales of the other: it is only
 *     good if both write the same.
 *   - Positions below 0 or from l_max on do not exist (the same rules).
 *   - Rows of the packed arrays before start[0] and from start[B] on belong to no sequence: what
 *     they hold does not matter, and in outputs they stay as they were.
 *   - Rows of a page that no position reaches may hold anything, infinities and NaN included.
 * start, kv_len and table are device memory and are read by the kernels only: a captured call follows
 * what they hold when it is replayed.
 *
 * 8-bit and 4-bit pages: every 32 elements of a row share a scale 2^e, the smallest power of two with
 * e >= -110 for which none of them exceeds the largest code (448 for e4m3, 127 for i8, 6 for e2m1), kept as the
 * byte e + 127.  The codes of e2m1 are a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (0 to 7 in the low three
 * bits), two a byte: element 2 i of a row is the low half of byte i, so a row has 64 bytes.  Codes are x 2^-e rounded to the nearest, ties to even; since the scale is a power of
 * two that is the only rounding (of e2m1 a tie goes to the even one of the eight), and a code times its scale is exact in bf16 and fp32.  A finite
 * element is read back finite: where the nearest code would mean 2^128 (bf16's largest number does) the
 * next one below is taken.  32 elements with an infinity or a NaN among them get the scale byte 255 and
 * read as NaN.  Pools that are not written by lrqk_pages_append may hold other codes and scales, -128 and the
 * NaN of e4m3 too: a product that kv_dtype does not hold is an infinity.
 */
enum { LRQK_PAGE_BF16 = 0, LRQK_PAGE_F32 = 1, LRQK_PAGE_E4M3 = 2, LRQK_PAGE_I8 = 3, LRQK_PAGE_E2M1 = 8 };

/*
 *   T          rows of the packed arrays (q, out, k_new, v_new), 1 <= T < 2^24
 *   n_max      new tokens of any one sequence, at most; chooses between kernels, whose results
 *              differ by roundings
 *   l_max      positions of any one sequence, at most, 1 <= l_max < 2^24
 *   l_cap      rows allocated per head in the dense arrays of lrqk_pages_read; 0 means l_max
 *   page       positions per page: a power of two, 1 <= page <= 1024; from 16 on for prompts, whose
 *              attention takes twice as long over smaller ones, and for 4 bits (single tokens take 1.7 times as long over
 *              smaller ones, fp32 queries three to five times)
 *   n_pages    pages of the pool: at most 64 GiB of K rows and as much of V rows, without scales
 *   max_pages  entries of a sequence's row of the table, max_pages * page >= l_max
 *   kv_dtype   LRQK_KV_*: type of q, out, k_new, v_new and the dense arrays
 *   page_dtype LRQK_PAGE_*: type of the rows in the pool; BF16 and F32 need the same kv_dtype
 *   d = 128, Hq a multiple of Hkv, Hq/Hkv <= 8, B * Hq <= 65535, T * Hq < 2^31, scale finite
 */
typedef struct lrqk_pages_shape {
  int32_t B, Hq, Hkv, d, T, n_max, l_max, l_cap, page, n_pages, max_pages;
  int32_t kv_dtype, page_dtype;
  float scale;
} lrqk_pages_shape;

/* All device memory, 16-byte aligned. */
typedef struct lrqk_pages {
  void* K;              /* page_dtype [n_pages,Hkv,page,d] (e2m1: d/2 bytes a row) */
  void* V;              /* page_dtype [n_pages,Hkv,page,d] */
  uint8_t* K_scale;     /* 8-bit and 4-bit pages: [n_pages,Hkv,page,d/32]; else not looked at (may be NULL) */
  uint8_t* V_scale;     /* likewise */
  const int32_t* table;  /* [B,max_pages] */
  const int32_t* start;  /* [B+1] */
  const int32_t* kv_len; /* [B] */
} lrqk_pages;

/* Host-only check of a shape against the limits above. LRQK_OK / LRQK_EINVAL / LRQK_ESHAPE. */
int lrqk_validate_pages(const lrqk_pages_shape* shape);

/* Bytes of device workspace lrqk_chunk_attend needs for this shape (0 on a bad shape).  Contents
 * need no initialisation; calls that overlap, and graphs whose replays overlap, need one each. */
size_t lrqk_pages_workspace_bytes(const lrqk_pages_shape* shape);

/*
 * g1 — the new tokens' rows go into their pages.
 *   pages  K, V and, for 8-bit and 4-bit pages, K_scale, V_scale are written as described
 *   k_new, v_new  device kv_dtype [T,Hkv,d]
 */
int lrqk_pages_append(const lrqk_pages_shape* shape, const lrqk_pages* pages, const void* k_new,
                      const void* v_new, void* stream);

/*
 * g2 — rows of the pages as dense arrays: for every sequence b and first <= p < kv_len[b],
 *   K_out[b,kv,p,:] = the row of position p, V_out likewise; all other rows stay as they are.
 * With first = the length before a chunk only that chunk's rows are brought up to date.
 *   first >= 0
 *   K_out, V_out  kv_dtype [B,Hkv,l_cap,d], device memory or pinned host memory; one of them may
 *                 be NULL
 */
int lrqk_pages_read(const lrqk_pages_shape* shape, const lrqk_pages* pages, int32_t first, void* K_out,
                    void* V_out, void* stream);

/*
 * g3 — exact causal attention of the new tokens.  For token i of sequence b, at position
 * p0 = kv_len[b] - n + i:
 *   out[start[b]+i,h,:] = sum_{p <= p0} w_p V_p,   w = softmax_p(scale * q[start[b]+i,h,:] . K_p)
 * over the positions that exist (their pages too), K and V of KV head h / G.  A token that sees no
 * position, or only scores of -infinity, gets zeros.  What a token does not see does not reach its
 * output, whatever its rows hold.  An infinite element of V under a weight of 0 (a score of -infinity, or one
 * that far below the others) makes NaN or that infinity.  Finite elements of V from 2^92 on may make infinities (a weight is up to 2^12
 * before the sum of up to 2^24 of them divides it).  Products of bf16 operands are exact, sums fp32; with bf16 q the
 * weights are rounded to bf16 before they meet V and before they are summed.
 * (fp32 q over 4-bit pages of 16 positions and more: q and the weights are taken as three bf16 terms each that add up to
 * them exactly, but for terms below 2^-126.)
 *   q    device kv_dtype [T,Hq,d]
 *   out  device kv_dtype [T,Hq,d]  written
 *   workspace  device, >= lrqk_pages_workspace_bytes(shape), 256-byte aligned
 * The new tokens' own rows are read from their pages: lrqk_pages_append comes first, on the same
 * stream.  LRQK_ENOMEM if ws_bytes is too small.
 */
int lrqk_chunk_attend(const lrqk_pages_shape* shape, const lrqk_pages* pages, const void* q, void* out,
                      void* workspace, size_t ws_bytes, void* stream);

/*
 * Rotary positions.  Of a row of d elements the first `rot` are turned in pairs by angles that grow with
 * the token's position, the others stay as they are:
 *   pair j of rot/2 at position p:  a = 2 pi frac(p turns[j] / 2^64),
 *   y_u = amplitude (x_u cos a - x_v sin a),   y_v = amplitude (x_v cos a + x_u sin a)
 *   LRQK_ROPE_HALVES  u = j, v = j + rot/2;     LRQK_ROPE_PAIRS  u = 2 j, v = 2 j + 1
 * The fraction is exact for every position (an integer product mod 2^64): far positions lose nothing.  Sums are
 * fp32; a result is off by at most 8 2^-24 |amplitude| (|x_u| + |x_v|), and the rounding to its type.
 *   rot        even, 2 <= rot <= d
 *   back       0, or 1: by -a, the transposed map: what turns gradients back (and, up to amplitude^2, undoes it)
 *   amplitude  finite
 *   turns      device, [rot/2], as written by lrqk_rope_turns (copied to the device by the caller)
 */
enum { LRQK_ROPE_HALVES = 0, LRQK_ROPE_PAIRS = 1 };
typedef struct lrqk_rope {
  int32_t layout, rot, back;
  float amplitude;
  const uint64_t* turns;
} lrqk_rope;

/*
 * r0 -- the table of a rope: turns[j] = f_j / (2 pi) in units of 2^-64 turns, f_j radians a position.
 * Host only.  F_j = base^(-2 j / rot), and
 *   LRQK_ROPE_PLAIN   f = F
 *   LRQK_ROPE_LINEAR  f = F / factor
 *   LRQK_ROPE_BASE    f = F with base factor^(rot / (rot - 2)) for base (rot = 2: base)
 *   LRQK_ROPE_BANDS   f = F (s + (1 - s) / factor), s = (l_orig F / (2 pi) - low) / (high - low) within [0, 1]:
 *                     pairs that turn more than `high` times in the original length l_orig stay, those that turn less
 *                     than `low` times are stretched
 *   LRQK_ROPE_RAMP    the same with s = 1 - (j - j0) / max(j1 - j0, 0.001) within [0, 1], linear in j from the pair that
 *                     turns `high` times to the one that turns `low` times: j(n) = rot ln(l_orig / (2 pi n)) / (2 ln base),
 *                     j0 = max(floor(j(high)), 0), j1 = min(ceil(j(low)), rot - 1).  The pairs end at rot/2 - 1: if the last one
 *                     turns more than `low` times, j1 lies behind it and no pair is stretched fully
 *   base      > 1;  factor > 0 (not looked at by PLAIN);  0 < low < high and l_orig >= 1 (BANDS and RAMP)
 *   turns      host, [rot/2]  written
 *   amplitude  host, may be NULL: written with 0.1 ln(factor) + 1 for RAMP (factor >= 1), 1 otherwise
 */
enum { LRQK_ROPE_PLAIN = 0, LRQK_ROPE_LINEAR = 1, LRQK_ROPE_BASE = 2, LRQK_ROPE_BANDS = 3, LRQK_ROPE_RAMP = 4 };
int lrqk_rope_turns(int32_t rot, int32_t scaling, double base, double factor, double low, double high,
                    int32_t l_orig, uint64_t* turns, float* amplitude);

/*
 *   T                 tokens, 1 <= T < 2^24
 *   Hq, Hkv           heads of q and of k, 1 to 1024 each (that of an array that is not given is not looked at)
 *   q_type, q_out_type, k_type   LRQK_KV_*; k_out has the type of k
 *   q_stride, ...     elements from one token's rows to the next: 0 for dense rows (heads * d), else at least that
 *                     and a multiple of 16 bytes; so q and k may be parts of one projection's rows
 *   d = 128
 */
typedef struct lrqk_rotate_shape {
  int32_t T, Hq, Hkv, d;
  int32_t q_type, q_out_type, k_type;
  int32_t q_stride, q_out_stride, k_stride, k_out_stride;
} lrqk_rotate_shape;

/*
 * r1 -- queries and keys at positions of their own: what lrqk_factor_update, lrqk_append_token and
 * lrqk_decode_step take (q in fp32, k in kv_dtype), lrqk_chunk_attend and lrqk_pages_append; with rope->back their
 * gradients.
 *   pos        device int32 [T], any value
 *   q, q_out   device [T,Hq,d]    both or neither
 *   k, k_out   device [T,Hkv,d]   both or neither; one of q and k at least
 * In place if an output is its input, with the same type and stride; else they must not overlap.
 */
int lrqk_rotate(const lrqk_rotate_shape* shape, const lrqk_rope* rope, const int32_t* pos, const void* q,
                void* q_out, const void* k, void* k_out, void* stream);

/*
 * Rows of new tokens as a projection leaves them (lrqk_pages_rotate_append).
 *   q, k, v    device kv_dtype [T,Hq,d], [T,Hkv,d], [T,Hkv,d]; q may be NULL
 *   *_stride   as in lrqk_rotate_shape
 *   q_out      device kv_dtype [T,Hq,d], dense; NULL exactly if q is.  May be q where that is dense; must not overlap
 *              k, v or, else, q
 *   pos, slot  device int32 [T], both or neither: each row's position and the row of the pool it goes to, as
 *              written by lrqk_pages_advance.  Then start, kv_len and table are not looked at
 */
typedef struct lrqk_new_rows {
  const void *q, *k, *v;
  int32_t q_stride, k_stride, v_stride;
  void* q_out;
  const int32_t *pos, *slot;
} lrqk_new_rows;

/*
 * g4 -- a layer's new rows in one call: q_out is q turned; k, turned and rounded to kv_dtype, and v go into their pages as by
 * lrqk_pages_append.  The same bits as lrqk_rotate and lrqk_pages_append give.
 * A token at a position below 0 does not exist: nothing of it is written, q_out included.  One at l_max or beyond, or
 * without a page (a slot outside [0, n_pages * page)), has its q turned, its k and v are dropped.
 */
int lrqk_pages_rotate_append(const lrqk_pages_shape* shape, const lrqk_pages* pages, const lrqk_rope* rope,
                             const lrqk_new_rows* rows, void* stream);

/*
 * Tables of a paged cache that live on the device: what the calls above read, made from how many tokens each
 * request keeps and gets.  All device memory, 16-byte aligned.
 *   refs     how many table entries name a page; 0 (or less): it is free.  lrqk_pages_advance counts what it takes and gives
 *            back.  A caller that lets several sequences share a page, or keeps one for itself, counts that too
 *   table    sequence b holds the pages of its kv_len[b] positions in its first ceil(kv_len[b] / page) entries
 *   status   per sequence: LRQK_ADVANCE_*
 *   seq, pos, slot   per packed row: its sequence, its position, and the row of the pool (page * table[b][pos / page] +
 *            pos mod page); -1 for rows that belong to no sequence.  Each may be NULL
 * A sequence whose next row lies on a shared page (LRQK_ADVANCE_SHARED) goes on once the caller has given it a copy: a free page new for
 * the page old of its table, K, V and their scales of old copied to new in every layer's pool (whole pages, plain device copies), refs[old] one less,
 * refs[new] = 1, the table's entry new.  Prefixes that are whole pages need none.
 */
typedef struct lrqk_pages_tables {
  int32_t* refs;    /* [n_pages]      read and updated */
  int32_t* table;   /* [B,max_pages]  read and updated */
  int32_t* kv_len;  /* [B]            read and updated */
  int32_t* start;   /* [B+1]          written */
  int32_t* status;  /* [B]            written */
  int32_t* seq;     /* [T]            written */
  int32_t* pos;     /* [T]            written */
  int32_t* slot;    /* [T]            written */
} lrqk_pages_tables;

enum {
  LRQK_ADVANCE_OK = 0,
  LRQK_ADVANCE_LONG = 1,   /* more than n_max new tokens, or than l_max positions                     */
  LRQK_ADVANCE_SHARED = 2, /* its next row lies on a page that is counted more than once              */
  LRQK_ADVANCE_PAGES = 3,  /* not enough free pages for it and those before it                        */
  LRQK_ADVANCE_ROWS = 4    /* more than T rows, its and those of the sequences before it               */
};

/* An empty cache: refs and kv_len 0, table -1. */
int lrqk_pages_tables_init(const lrqk_pages_shape* shape, const lrqk_pages_tables* tables, void* stream);

/* Bytes of device workspace lrqk_pages_advance needs for this shape (0 on a bad shape). */
size_t lrqk_pages_advance_workspace_bytes(const lrqk_pages_shape* shape);

/*
 * g5 -- the tables of a step from those of the step before.  Sequence b is cut back to its first keep[b] positions
 * (drafts that were rejected; 0: the request has ended) and gets n_new[b] new ones:
 *   1. kept = min(max(keep[b], 0), kv_len[b]); the pages behind ceil(kept / page) are given back: their refs count one
 *      less, their table entries become -1
 *   2. a sequence with n = max(n_new[b], 0) > 0 is refused (status) if n > n_max or kept + n > l_max; else if kept is no
 *      multiple of page and the refs of the page of position kept are more than 1; else if the new pages that it
 *      and the sequences before it ask for are more than are free and it asks for any; else if its new rows and those of
 *      the sequences before it are more than T.  (One that is refused by the first two rules asks for nothing.)
 *      A refused sequence keeps its `kept` positions and gets no new one
 *   3. the j-th new page, counted through the sequences and their positions, is the j-th free page of the pool; its
 *      refs become 1
 *   4. kv_len = kept + n, start = the running sum of the n; seq, pos, slot of the T rows
 * Everything is decided on the device: a captured call follows keep and n_new, and what the tables hold.  Called again with the
 * same keep (none above kv_len) and n_new it gives the same tables.
 *   keep       device int32 [B], or NULL: everything is kept
 *   n_new      device int32 [B]
 *   workspace  device, >= lrqk_pages_advance_workspace_bytes(shape), 256-byte aligned
 * Table entries that are no pages are left out of the counting.  B, T, n_max, l_max, page, n_pages and max_pages of
 * the shape are used.
 */
int lrqk_pages_advance(const lrqk_pages_shape* shape, const lrqk_pages_tables* tables, const int32_t* keep,
                       const int32_t* n_new, void* workspace, size_t ws_bytes, void* stream);

/*
 * Instrumentation (not part of the method): GPU time of the kernels of lrqk_decode_step, each
 * taken from a pair of HIP events attached to the kernel itself (they hold its own start and
 * end, so neither the gaps between launches nor the events' own cost are included).
 * lrqk_plan_profile(plan, n) arms the next n calls of lrqk_decode_step on this plan (n = 0
 * switches it off); lrqk_plan_profile_read waits for the recorded steps, adds up every
 * slot's kernel time into ms_sum[LRQK_PROFILE_SLOTS] (milliseconds, summed over the steps;
 * 0 for kernels the steps did not launch) and re-arms.  Slots:
 */
enum {
  LRQK_SLOT_SAMPLE = 0,      /* threshold estimate: scores of the sampled rows          */
  LRQK_SLOT_THRESHOLD = 1,   /* threshold estimate: histogram of the samples            */
  LRQK_SLOT_PROXY = 2,       /* a1, the pass over A_K                                   */
  LRQK_SLOT_SELECT = 3,      /* a2 (+ a3 where one kernel does both; of the multi-launch
                                selection of very long contexts only the first kernel)  */
  LRQK_SLOT_RESOLVE = 4,     /* a3 as a kernel of its own                               */
  LRQK_SLOT_FETCH = 5,       /* STAGED: scatter of the copied rows into the cache slots */
  LRQK_SLOT_ATTEND = 6,      /* a5 partials (DIRECT: with the fetch; STAGED: hit rows)  */
  LRQK_SLOT_ATTEND_MISS = 7, /* STAGED: a5 partials over the rows that were fetched     */
  LRQK_SLOT_COMBINE = 8,     /* a5 merge of the partials                                */
  LRQK_PROFILE_SLOTS = 9
};
int lrqk_plan_profile(lrqk_plan* plan, int n_steps);
int lrqk_plan_profile_read(lrqk_plan* plan, double* ms_sum, int* n_steps_out);

/*
 * Instrumentation: time the dominant kernel alone.  Runs step a1's pass over A_K exactly as
 * lrqk_decode_step launches it for this shape (the filtered proxy-score kernel, its thresholds
 * taken from sel_thr [B,Hq] as in a step that carries them (device, a layer's array after a
 * step with this kind of q_hat), or, with sel_thr NULL, estimated once from a sample for q_hat;
 * the plain proxy-score kernel for shapes that do not use the filter), n_launches times back
 * to back on `stream`, cycling through the n_list
 * device arrays A_K_list[i] (each [B,Hkv,l,r] fp32, e.g. one per layer, so that no cache
 * holds them), bracketed by two HIP events: microseconds per launch, gaps between launches
 * included.  For the filtered kernel a second series of at most 64 launches attaches a pair
 * of events to every kernel (they hold that kernel's own start and end); the average of
 * those durations is reported instead when it is positive and not above the bracketed
 * figure.  Synchronises; *avg_us_out = microseconds per launch.  Results go to the plan's
 * workspace and are discarded.
 */
int lrqk_plan_time_proxy_pass(lrqk_plan* plan, const lrqk_shape* shape,
                              const float* const* A_K_list, int n_list, const float* q_hat,
                              const float* sel_thr, int n_launches, float* avg_us_out,
                              void* stream);

/*
 * Instrumentation: copy `bytes` (a multiple of 16) from src to dst, both device memory,
 * 16-byte aligned, with a plain one-load-one-store kernel.  Its HBM traffic is known
 * (bytes read + bytes written), which calibrates the hardware byte counters that the
 * measured traffic of the other kernels is scaled by.
 */
int lrqk_calib_copy(void* dst, const void* src, size_t bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LRQK_H */
