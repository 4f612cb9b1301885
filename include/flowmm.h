/*
 * flowmm.h - C ABI of the FlowMM KV-cache compression library for NVIDIA B200 (sm_100a).
 *
 * FlowMM (arXiv 2511.05534, Section 3.3) compresses each transformer layer's KV cache once,
 * after multimodal prefill, per KV head:
 *   1. score   - attention of the proxy tokens (the last W prompt positions) over all context
 *                keys gives every token an importance (Eq. 8); the same attention, split by
 *                modality, gives the layer's cross-modal interaction ratio rho (Eq. 6-7);
 *   2. flow    - rho against the threshold theta picks cross-modal or intra-modal merging;
 *   3. select  - the B most important tokens form the pivot set, the rest the non-pivot set;
 *   4. match   - each non-pivot finds the pivot of largest key cosine similarity (Eq. 9)
 *                among pivots whose importance does not exceed the sensitivity threshold
 *                tau (Eq. 10) and, in an intra-modal layer, that share its modality;
 *   5. merge   - non-pivots are folded into their pivots (Eq. 5) and the B merged rows are
 *                written out as the compressed cache.
 *
 * Conventions for every entry point
 *   - A "unit" is one (layer, sequence) pair; units are independent problems and a call
 *     processes n_units of them at once.  G = n_q_heads / n_kv_heads query heads share KV
 *     head h = g / G.  L = seq_len, W = window, B = n_keep, E = L - B.
 *   - Every tensor pointer is a DEVICE pointer owned by the caller; the library allocates
 *     and frees nothing.  Scratch memory comes from the caller as `ws` / `ws_bytes`
 *     (size from flowmm_workspace_bytes, 256-byte aligned); its first word is a sticky
 *     device status, so the caller zero-fills the first 256 bytes once after allocating
 *     it.  Inputs are never written; outputs must not alias inputs.
 *   - n_units * n_kv_heads must not exceed 4 194 304 per call, and that product times the number of
 *     128-token tiles of the context times the number of 128-row tiles of a KV head's proxy rows must
 *     stay below 2^31 (work items are counted in 32 bits); else FLOWMM_ERR_SHAPE.
 *   - Q, K, V and the outputs have the element type `dtype`, head_dim contiguous, and the
 *     element strides given in the params (unit, head, token).  Base pointers must be
 *     16-byte aligned and every stride a multiple of 8 elements, else FLOWMM_ERR_ALIGN.
 *     All other arrays are dense in the stated shape.
 *   - Calls enqueue work on `cuda_stream` (a cudaStream_t passed as void*, NULL = default
 *     stream) and return without waiting.  The return value reports host-side validation
 *     and launch errors.  Problems found on the device (a bounded wait that ran out) set
 *     the status word, which flowmm_last_device_status reads back.
 *   - There is no CPU fallback: on a device that is not compute capability 10.x every
 *     compute entry point returns FLOWMM_ERR_UNSUPPORTED_DEVICE.
 */
#ifndef FLOWMM_H_
#define FLOWMM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FLOWMM_OK = 0,
    FLOWMM_ERR_NULL = 1,               /* a required pointer is NULL */
    FLOWMM_ERR_SHAPE = 2,              /* sizes inconsistent (heads, head_dim, window, ...) */
    FLOWMM_ERR_BUDGET = 3,             /* n_keep outside [1, L], or below W with keep_window */
    FLOWMM_ERR_DTYPE = 4,
    FLOWMM_ERR_WORKSPACE = 5,          /* ws_bytes smaller than flowmm_workspace_bytes */
    FLOWMM_ERR_ALIGN = 6,
    FLOWMM_ERR_CUDA = 7,               /* a CUDA runtime call or launch failed */
    FLOWMM_ERR_TIMEOUT = 8,            /* device status: a bounded wait inside a kernel ran out */
    FLOWMM_ERR_UNSUPPORTED_DEVICE = 9,
    FLOWMM_ERR_INDEX = 10,             /* an index was out of range (index lists: debug build only; pages, slots and rows of the paged caches: always) */
    FLOWMM_ERR_POOL = 11               /* device status: the page pool, the block table or the slot map had no room for a unit's rows */
} flowmm_status;

typedef enum { FLOWMM_F32 = 0, FLOWMM_BF16 = 1 } flowmm_dtype;
typedef enum { FLOWMM_INTRA = 0, FLOWMM_CROSS = 1 } flowmm_strategy;
/* Eq. 5 leaves the merge functions open.  EXPSIM: pivot weight 1, non-pivot weight
 * exp(u - 1) with u its cosine similarity to the pivot; MEAN: all weights 1.  Weights are
 * normalised to sum to one per output row. */
typedef enum { FLOWMM_MERGE_EXPSIM = 0, FLOWMM_MERGE_MEAN = 1 } flowmm_merge_mode;
/* ABS: tau is compared with the importance directly.  REL: tau is in units of the
 * importance a uniform attention would give, tau_eff = tau * W / L. */
typedef enum { FLOWMM_TAU_ABS = 0, FLOWMM_TAU_REL = 1 } flowmm_tau_mode;
/* AUTO: the theta rule on rho (aligned merging).  FORCE_*: one strategy for every layer.  MISALIGNED: the
 * reverse of the rule (intra-modal where rho > theta, cross-modal elsewhere), the contrast case of the paper's
 * study of flow-aligned merging. */
typedef enum { FLOWMM_FLOW_AUTO = 0, FLOWMM_FLOW_FORCE_INTRA = 1, FLOWMM_FLOW_FORCE_CROSS = 2,
               FLOWMM_FLOW_MISALIGNED = 3 } flowmm_flow_mode;
/* Which kernels do the two dense contractions.  AUTO: tensor-core (tcgen05) kernels when
 * dtype is bf16 and head_dim is 128, SIMT fp32 kernels otherwise.  SIMT forces the latter. */
typedef enum { FLOWMM_PATH_AUTO = 0, FLOWMM_PATH_SIMT = 1 } flowmm_path;

typedef struct {
    int32_t n_units;                    /* independent (layer, sequence) problems */
    int32_t n_q_heads, n_kv_heads;      /* n_q_heads must be a multiple of n_kv_heads */
    int32_t head_dim;                   /* 64 or 128 */
    int32_t seq_len, window;            /* L, W with 1 <= W <= L */
    int32_t n_keep;                     /* B with 1 <= B <= L */
    int32_t dtype;                      /* flowmm_dtype of Q, K, V, K_out, V_out */
    float softmax_scale;                /* 0 selects 1/sqrt(head_dim) */
    float theta;                        /* cross-modal merging threshold of Section 3.3.1 */
    float tau;                          /* sensitivity threshold of Eq. 10; +inf disables it */
    int32_t tau_mode;                   /* flowmm_tau_mode */
    int32_t flow_mode;                  /* flowmm_flow_mode */
    int32_t merge_mode;                 /* flowmm_merge_mode */
    int32_t keep_window;                /* 1: the W proxy tokens are always pivots (needs B >= W) */
    int32_t path;                       /* flowmm_path */
    /* element strides of (unit, head, token); head_dim stride is 1 */
    int64_t q_stride[3];                /* Q_win [U, Hq,  W, D] */
    int64_t k_stride[3];                /* K     [U, Hkv, L, D] */
    int64_t v_stride[3];                /* V     [U, Hkv, L, D] */
    int64_t ko_stride[3];               /* K_out [U, Hkv, B, D] */
    int64_t vo_stride[3];               /* V_out [U, Hkv, B, D] */
} flowmm_params;

/* Scratch size in bytes that any entry point below needs for these params.  Host only; makes
 * no CUDA call.  Fails with the same validation errors as the compute entry points.  Never smaller
 * for more units or a longer context with all other fields alike, so a workspace serves those calls too. */
flowmm_status flowmm_workspace_bytes(const flowmm_params *p, size_t *bytes);

/*
 * Step 1, Eq. 8 (with the causal softmax of Eq. 4 on the proxy rows) and the masses of Eq. 7.
 *   q_win      [U, Hq, W, D]   queries of the last W prompt positions
 *   k          [U, Hkv, L, D]  layer keys
 *   modality   [U, L] uint8    0 = text token, 1 = visual token
 *   importance [U, Hkv, L] f32 out: I[h,i] = (1/G) sum_{g in h} sum_a alpha[g,a,i]
 *   cross_mass [U, Hq] f32     out: sum_a sum_{i: m_i != m_(p_a)} alpha[g,a,i]; the total mass
 *                              of a head is W because every softmax row sums to one.
 */
flowmm_status flowmm_score(const flowmm_params *p, const void *q_win, const void *k, const uint8_t *modality,
                           float *importance, float *cross_mass, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Step 2, Eq. 6 and the threshold rule after Eq. 7.
 *   rho      [U] f32   out: mean over query heads of cross_mass / W
 *   strategy [U] int32 out: FLOWMM_CROSS if rho > theta else FLOWMM_INTRA (or as flow_mode forces)
 */
flowmm_status flowmm_layer_flow(const flowmm_params *p, const float *cross_mass, float *rho, int32_t *strategy,
                                void *cuda_stream);

/*
 * Step 3, pivot selection of Section 3.3.1: the B largest importances per KV head, ties to the
 * lower index.
 *   retained_idx [U, Hkv, B] int32 out: pivot token positions, ascending; slot s holds r_s
 *   evicted_idx  [U, Hkv, E] int32 out: non-pivot token positions, ascending
 */
flowmm_status flowmm_select(const flowmm_params *p, const float *importance, int32_t *retained_idx,
                            int32_t *evicted_idx, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Step 4, Eq. 9 and Eq. 10.  For the j-th non-pivot e = evicted_idx[j]:
 *   match     [U, Hkv, E] int32 out: slot of the admissible pivot with the largest cosine
 *                                    similarity (ties to the lower slot), or -1 if none
 *   match_sim [U, Hkv, E] f32   out: that similarity, 0 where match is -1
 * A pivot r_s is admissible if importance[r_s] <= tau_eff and, when strategy[u] is
 * FLOWMM_INTRA, modality[r_s] == modality[e].  A key of zero norm has similarity 0.
 */
flowmm_status flowmm_match(const flowmm_params *p, const void *k, const float *importance, const uint8_t *modality,
                           const int32_t *retained_idx, const int32_t *evicted_idx, const int32_t *strategy,
                           int32_t *match, float *match_sim, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Step 5, Eq. 5 and compaction.  Output row s (s in [0, B), ascending token position) is
 *   (x[r_s] + sum_{j: match[j] = s} w_j x[e_j]) / (1 + sum w_j),  x in {K, V},
 * with w_j = exp(match_sim[j] - 1) (EXPSIM) or 1 (MEAN); non-pivots with match -1 are dropped.
 * Accumulation is fp32 in a fixed order (results are bit-reproducible), rounded once to dtype.
 *   k_out, v_out [U, Hkv, B, D]
 */
flowmm_status flowmm_merge(const flowmm_params *p, const void *k, const void *v, const int32_t *retained_idx,
                           const int32_t *evicted_idx, const int32_t *match, const float *match_sim,
                           void *k_out, void *v_out, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * flowmm_merge without a caller-provided workspace.  (The paper has no counterpart: this is a
 * packaging variant of step 5 for callers that cannot allocate device memory - a plugin running
 * inside another runtime's memory pool, code running while that pool is frozen, a host that is
 * handed fixed buffers only.  They still pass the inputs and the two output tensors; what they
 * cannot provide is the scratch flowmm_merge needs for its slot lists and partial sums.)
 *
 * The scratch is a fixed array of FLOWMM_MERGE_STATIC_BYTES inside the library image; every GPU
 * that loads the library holds one copy until the process exits.  The call makes no cudaMalloc
 * or cudaFree and calls no allocating routine.  Arguments, outputs and results are those of
 * flowmm_merge (same kernels, same fixed accumulation order, so the outputs are bit-identical).
 *
 * Limits and rules:
 *   - The scratch a problem needs, per (unit, KV head): 16 E + 16 (B + E / 64 + 1) + 12 (B + 1) + 4 B
 *     bytes of slot lists, piece table and counters, 8 L bytes of per-token (slot, weight) pairs,
 *     and (2 (E / 64) + 2) * (8 head_dim + 16) bytes of partial sums; every part is rounded up
 *     to 256 bytes and 768 bytes are fixed.  If that exceeds the array the call returns
 *     FLOWMM_ERR_WORKSPACE and launches nothing.
 *   - A problem found on the device (a bounded wait that ran out) is recorded in a status word
 *     inside the array, since there is no workspace to carry it: flowmm_merge_static_status
 *     waits for the stream, returns that word (FLOWMM_OK or the first error recorded by any
 *     call since the last read) and clears it.  Outputs of a call that reported an error are
 *     not valid.
 *   - The first call on a device looks up the array's device address (once per device, with
 *     that device current).  Make that first call outside any stream capture.
 *   - All calls on a device share the one array and it keeps the previous call's contents;
 *     nothing in it needs clearing between calls.  Two calls that overlap on the GPU (different
 *     streams, or graphs replayed concurrently) race on it: keep them ordered.
 */
#define FLOWMM_MERGE_STATIC_BYTES (8u << 20)
flowmm_status flowmm_merge_static(const flowmm_params *p, const void *k, const void *v, const int32_t *retained_idx,
                                  const int32_t *evicted_idx, const int32_t *match, const float *match_sim,
                                  void *k_out, void *v_out, void *cuda_stream);
flowmm_status flowmm_merge_static_status(void *cuda_stream);
/* Test aid for the reader above: waits for the stream and stores `word` in the array's status word
 * from the host, so that reading and clearing can be checked without making a kernel fail. */
flowmm_status flowmm_merge_static_poke_status(int32_t word, void *cuda_stream);

/*
 * Steps 1-5 in order on one stream: the whole per-layer FlowMM compression of Section 3.3.
 * The diagnostic outputs (importance ... match_sim, layouts as above) may each be NULL, in
 * which case the intermediate lives in the workspace only.
 */
flowmm_status flowmm_compress_layer(const flowmm_params *p, const void *q_win, const void *k, const void *v,
                                    const uint8_t *modality, void *k_out, void *v_out,
                                    float *importance, float *rho, int32_t *strategy,
                                    int32_t *retained_idx, int32_t *evicted_idx,
                                    int32_t *match, float *match_sim,
                                    void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Re-compression of a cache that has grown during decoding.  Eq. 3 appends one key / value row per decoded token;
 * the paper runs the compression of Section 3.3 once, after prefill, and does not say what follows.  The reading
 * offered here: the current cache of a KV head - the rows an earlier compression left, in order, then the rows
 * appended since - is treated as that head's context of L = seq_len rows, and steps 1-5 run on it again with the
 * proxy window taken from the W most recent queries.  A row that came out of an earlier merge is an ordinary token
 * with the modality of the pivot it was merged into; after a compression the heads of a layer no longer hold the
 * same tokens, so modality is given per head and row.  Importance is taken afresh from the window (the causal mask
 * follows the row order, exact once at least W rows have been appended); rho is still the layer's, the mean over
 * all query heads (Eq. 6), each head measured against its own rows; merge weights as in flowmm_merge.
 *   q_win            [U, Hq, W, D]   queries of the W most recent positions
 *   k_cache, v_cache [U, Hkv, L, D]  the cache rows, strides p->k_stride / p->v_stride
 *   row_modality     [U, Hkv, L] uint8
 *   k_out, v_out     [U, Hkv, B, D]; row_modality_out [U, Hkv, B] uint8 (the kept rows' modalities, for the next round)
 *   importance ... match_sim: optional diagnostics (may be NULL), shaped as in flowmm_compress_layer but per
 *   KV head throughout; rho, strategy [U].
 * The unit stride of q, k, v and the outputs must equal heads x head stride (dense over heads), else
 * FLOWMM_ERR_ALIGN.  Scratch: flowmm_recompress_workspace_bytes.  B == L returns the cache unchanged (the plain
 * append of Eq. 3).
 */
flowmm_status flowmm_recompress_workspace_bytes(const flowmm_params *p, size_t *bytes);
flowmm_status flowmm_recompress(const flowmm_params *p, const void *q_win, const void *k_cache, const void *v_cache,
                                const uint8_t *row_modality, void *k_out, void *v_out, uint8_t *row_modality_out,
                                float *importance, float *rho, int32_t *strategy, int32_t *retained_idx,
                                int32_t *evicted_idx, int32_t *match, float *match_sim,
                                void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The step before the compression path: the cross-modal interaction ratio of Eq. 6 and Eq. 7 taken
 * literally, over every query row of the prefill (both the text-to-visual and the visual-to-text
 * term), instead of over the proxy window that flowmm_score uses.  Causal softmax attention of all
 * L queries; per query head the attention mass that lands on keys of the other modality than the
 * query's, summed over the rows; rho = mean over heads of that mass / L; strategy by theta.
 *   q_full [U, Hq, L, D] with the element strides q_full_stride (unit, head, token); head_dim contiguous
 *   k      [U, Hkv, L, D] with p->k_stride
 *   cross_mass [U, Hq] f32 out;  rho [U] f32 out (may be NULL);  strategy [U] int32 out
 * Of p, the fields n_units, n_q_heads, n_kv_heads, head_dim, seq_len, dtype, softmax_scale, theta,
 * flow_mode, k_stride and path are used (window, n_keep, tau, q_stride are not).  Every query row
 * is scored against the keys up to itself, so the call
 * costs O(L^2 D) per head.  Scratch: flowmm_full_flow_workspace_bytes; its first word is the device status.
 */
flowmm_status flowmm_full_flow_workspace_bytes(const flowmm_params *p, size_t *bytes);
flowmm_status flowmm_full_flow(const flowmm_params *p, const void *q_full, const int64_t q_full_stride[3],
                               const void *k, const uint8_t *modality, float *cross_mass, float *rho,
                               int32_t *strategy, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The step after the compression path: decode-time attention of one new query per query head over a
 * cache of n_keys rows, Eq. 4 - o = softmax(q . K^T * scale) V - for the full cache or for the
 * compressed one that flowmm_compress_layer wrote.  Every cache row is read once for all G query
 * heads of its KV head.
 *   q   [U, Hq, D]  dense, element type `dtype`
 *   k,v [U, Hkv, n_keys, D] with the element strides given (unit, head, token); head_dim contiguous
 *   out [U, Hq, D]  f32
 * n_q_heads / n_kv_heads must be at most 8; head_dim 64 or 128.  Scratch: flowmm_decode_workspace_bytes
 * (its first word is a device status like the compression workspace's, see flowmm_last_device_status).
 * Every call starts the status at FLOWMM_OK by itself, so the scratch may hold anything beforehand; only replays of one
 * captured graph keep an error of an earlier replay until it is read.
 * `path` as in flowmm_params: AUTO runs both contractions on the tensor cores (tcgen05) when dtype is
 * bf16 and head_dim is 128, and SIMT fp32 kernels otherwise; SIMT forces the latter.
 * Same conventions as above (device pointers, caller-owned memory, asynchronous on the stream).
 */
typedef struct {
    int32_t n_units, n_q_heads, n_kv_heads, head_dim;
    int32_t n_keys;                     /* rows of the cache to attend to (L, or B after compression) */
    int32_t dtype;                      /* flowmm_dtype of q, k, v */
    float softmax_scale;                /* 0 selects 1/sqrt(head_dim) */
    int32_t path;                       /* flowmm_path */
    int64_t k_stride[3], v_stride[3];   /* element strides of (unit, head, token) */
} flowmm_decode_params;

flowmm_status flowmm_decode_workspace_bytes(const flowmm_decode_params *p, size_t *bytes);
flowmm_status flowmm_decode_attention(const flowmm_decode_params *p, const void *q, const void *k, const void *v,
                                      float *out, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The paged 8-bit cache: caches of units with lengths of their own, in pages of a common pool, with the decode attention that reads
 * them.  After compression every sequence keeps its own number of rows, and a decode step is bound by reading K and V: a row is held
 * in 8 bits instead of 16 or 32, and memory is given out by pages.  A cache is stored (flowmm_cache_store) from what
 * flowmm_compress_layer wrote or from dense caches, grows by a row a step, is attended to (flowmm_cache_attention) and, when it has
 * grown, is read back (flowmm_cache_load) for flowmm_recompress.  That takes units of one length and the modality of every row: it is called for
 * units of equal length at a time (their rows of the block table and of `rows`), and the rows' modalities, which the cache does not hold, are
 * the caller's to keep (flowmm_recompress gives back those of the rows it keeps).
 *
 *   k_pages, v_pages [n_pages, Hkv, page_size, D] e4m3 codes (4 exponent bits of bias 7, 3 mantissa bits, 127 and 255 NaN, no
 *                    infinity), dense
 *   k_scale, v_scale [n_pages, Hkv] f32: a code stands for code * scale.  flowmm_cache_store writes powers of two from 2^-96 on;
 *                    the readers take any positive scale up to 2^120.
 *   block_table      [U, max_pages] int32: the pages of a unit, in order; entries behind its last page are not read
 *   rows             [U] int32: rows that a unit holds, 0 to max_pages * page_size
 *   slots            [U, n_rows] int32: where each new row of a unit goes, page * page_size + place in the page; -1: nowhere
 *
 * `ws` as everywhere (flowmm_cache_workspace_bytes, first 256 bytes zeroed once); calls that share one are kept in order.  Page
 * numbers, slots and rows are checked before use in every build: a bad one sets the device status to FLOWMM_ERR_INDEX, nothing is
 * read or written out of bounds for it, and the outputs of its unit are not valid.  Heads (at most
 * 8 query heads a KV head), head_dim and dtype as in flowmm_decode_params.  n_pages * page_size and n_units * n_rows are
 * below 2^31, max_pages * page_size and n_rows at most 2^30, n_units * n_kv_heads at most 4 194 304.  Work is counted in 32 bits (FLOWMM_ERR_SHAPE
 * otherwise): the store takes fewer than 2^31 n_units * (2 n_kv_heads + 1) * pages that n_rows rows can reach, the load fewer than 2^30
 * n_units * n_kv_heads * n_rows / 64, the attention fewer than 2^31 n_units * n_q_heads * max_pages * page_size / 64.
 */
typedef struct {
    int32_t n_units, n_q_heads, n_kv_heads, head_dim;
    int32_t page_size;                  /* rows of a page: 16, 32, 64 or 128 */
    int32_t n_pages;                    /* pages of the pool */
    int32_t max_pages;                  /* entries of a unit in the block table */
    int32_t n_rows;                     /* slots (plan), rows of k and v (store, load) of a unit */
    int32_t dtype;                      /* flowmm_dtype of q and of the dense rows */
    float softmax_scale;                /* 0 selects 1/sqrt(head_dim) */
    int32_t path;                       /* flowmm_path of the attention */
    int64_t k_stride[3], v_stride[3];   /* element strides (unit, head, row) of the dense rows */
} flowmm_cache_params;

flowmm_status flowmm_cache_workspace_bytes(const flowmm_cache_params *p, size_t *bytes);

/*
 * Block tables and slot maps from the lengths of the requests, on the GPU (a step can be captured in a graph).
 * Unit u goes from rows[u] to max(0, rows[u] + grow[u]) rows: pages it needs more are taken from the ring of free pages, pages
 * it needs no longer go back to it (grow = -rows ends a request), the first grow[u] slots say where its new rows go, the others are -1.
 *   grow, rows [U] int32;  rows_out [U] out
 *   free_pages [n_pages] int32 in and out, a ring;  free_state {head, count}: the free pages are free_pages[(head + i) % n_pages],
 *              i < count;  free_state_out [2] out
 *   block_table in and out: entries of pages taken are written, all others left as they were
 *   slots [U, n_rows] out, or NULL: then any growth that the table has room for is planned, without slots
 * Units are served in order, pages in the ring's order; pages given back in a call are not given out in it, and go behind the
 * free ones, by unit and place.  A unit that asks for more than n_rows slots or max_pages pages, or that comes to need pages when
 * all units so far have asked for more than are free, is left as it was (rows_out = rows, slots -1) and the status becomes
 * FLOWMM_ERR_POOL; the others go on.  rows_out and free_state_out are arrays of their own: nothing that a call reads is changed
 * by it (places of the ring and the table that it writes held nothing), so a step that is not carried out is planned again from
 * the same rows and free_state.
 */
flowmm_status flowmm_cache_plan(const flowmm_cache_params *p, const int32_t *grow, const int32_t *rows, int32_t *rows_out,
                                int32_t *free_pages, const int32_t *free_state, int32_t *free_state_out, int32_t *block_table,
                                int32_t *slots, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Rows into pages.  Row t of unit u goes to slots[u][t].  The rows of a unit go to consecutive places (the rest of a page, then
 * whole pages from their first place on), as flowmm_cache_plan lays them out; -1 only behind the last row (a row with a place behind one without
 * is reported; where it is in a page whose first new row has none it is not stored).  No page is written for two units.  Per page, KV head and tensor:
 *   s = the smallest power of two, 2^-96 at least, with |x| <= 448 s for all finite new rows x of the page; where the page holds
 *       rows already (the first new row is not at its first place), not below its scale s_old
 *   new codes = e4m3(x / s), old codes = e4m3(code * s_old / s), round to nearest even; NaN and infinities become NaN
 * Places behind the new rows are left as they were.  A single new row per unit (n_rows = 1) is the decode step's form.
 *   k, v [U, Hkv, n_rows, D] with the element strides k_stride, v_stride
 */
flowmm_status flowmm_cache_store(const flowmm_cache_params *p, const void *k, const void *v, const int32_t *slots, void *k_pages,
                                 void *v_pages, float *k_scale, float *v_scale, void *ws, size_t ws_bytes, void *cuda_stream);

/* Pages into rows: k, v [U, Hkv, n_rows, D] out, code * scale in fp32 (exact with scales that flowmm_cache_store writes), rounded to the type, for the
 * first min(rows[u], n_rows) rows of each unit; the others are left as they were. */
flowmm_status flowmm_cache_load(const flowmm_cache_params *p, const void *k_pages, const void *v_pages, const float *k_scale,
                                const float *v_scale, const int32_t *block_table, const int32_t *rows, void *k, void *v, void *ws,
                                size_t ws_bytes, void *cuda_stream);

/*
 * flowmm_decode_attention over the paged cache: o = softmax(q . (k_scale K)^T * scale) (v_scale V) over the rows[u] rows of each
 * unit, zero for a unit without rows.  What stands behind a unit's last row (codes of NaN too) has no influence.  Several new
 * queries of a sequence are units that share a row of the block table and differ in rows.
 *   q [U, Hq, D] dense, element type `dtype`;  out [U, Hq, D] f32
 * `path`: AUTO runs both contractions on the tensor cores (tcgen05, the codes as operands) when dtype is bf16, and SIMT fp32 kernels
 * otherwise; SIMT forces the latter.  The workspace serves both.
 * Both sum in fp32, results without the division by the softmax's sum included: rows[u] * max |v| stays below 2^128.  The SIMT kernels multiply in fp32.  On
 * the tensor cores a query is two e4m3 numbers, exact for elements down to 2^-13 of its largest one, others within 2^-21 of that; a weight, the
 * softmax's times V's scale, is four, within 2^-16 of itself down to 2^-14 of the row's largest one, others within 2^-30 of that, so a page whose
 * V scale is 2^30 times smaller than another's of the head adds nothing.  The measured error on data like a cache's is 2e-7 of the result.
 */
flowmm_status flowmm_cache_attention(const flowmm_cache_params *p, const void *q, const void *k_pages, const void *v_pages,
                                     const float *k_scale, const float *v_scale, const int32_t *block_table, const int32_t *rows,
                                     float *out, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * The paged 4-bit cache: the same pools, block tables, slots and plans (flowmm_cache_plan) with rows held in 4.5 bits an element, a little over half of
 * the 8-bit cache's bytes, for decode steps that are bound by reading K and V and pools that are bound by memory.  Rows do not depend on one another: a
 * row that is stored changes no other one's codes.
 *
 *   k_pages, v_pages [n_pages, Hkv, page_size, D / 2] bytes of two e2m1 codes, the even channel's in the low half (sign, two exponent bits of bias 1, one
 *                    mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), dense
 *   k_scale, v_scale [n_pages, Hkv, page_size, D / 16] bytes, dense: a scale for 16 neighbouring channels of a row, five exponent bits of bias 15 and three
 *                    mantissa bits (an fp16 without sign and its lowest seven bits; 31 in the exponent: infinity and NaN).  A code stands for code *
 *                    scale.  flowmm_nibble_store writes 2^-14 to 10240 (bytes 8 to 226) and NaN (255); the readers take all bytes up to 226, and 255.
 *
 * Params, block_table, rows, slots, workspaces (of flowmm_nibble_workspace_bytes) and what is checked on the device as for the paged 8-bit cache;
 * `path` is not used.  Pages and scales are 16-byte aligned.  Work is counted in 32 bits (FLOWMM_ERR_SHAPE otherwise): the store takes fewer than 2^31
 * n_units * n_kv_heads * n_rows, the load fewer than 2^30 n_units * n_kv_heads * n_rows / 64, the attention fewer than 2^31
 * n_units * n_q_heads * max_pages * page_size / 64.
 */
flowmm_status flowmm_nibble_workspace_bytes(const flowmm_cache_params *p, size_t *bytes);

/*
 * Rows into pages.  Row t of unit u goes to slots[u][t], anywhere in the pool; -1: nowhere.  No place is written for two rows.  Per row, KV head, tensor and group of
 * 16 channels:
 *   s = max|x| / 6 rounded to four significant bits (to the nearest, ties to even), at least 2^-14, at most 10240
 *   codes = e2m1(x / s), to the nearest, ties to the even code, at most 6 in size (so elements beyond 61 440 become that), the sign of zeros kept
 * A group with an infinity or a NaN has the scale NaN and codes of zero.  Quotients are rounded as real numbers are: results do not depend on how they are formed.
 *   k, v [U, Hkv, n_rows, D] with the element strides k_stride, v_stride
 */
flowmm_status flowmm_nibble_store(const flowmm_cache_params *p, const void *k, const void *v, const int32_t *slots, void *k_pages,
                                  void *v_pages, void *k_scale, void *v_scale, void *ws, size_t ws_bytes, void *cuda_stream);

/* Pages into rows: k, v [U, Hkv, n_rows, D] out, code * scale, exactly (a product has six significant bits), for the first min(rows[u], n_rows) rows of each unit; the
 * others are left as they were. */
flowmm_status flowmm_nibble_load(const flowmm_cache_params *p, const void *k_pages, const void *v_pages, const void *k_scale,
                                 const void *v_scale, const int32_t *block_table, const int32_t *rows, void *k, void *v, void *ws,
                                 size_t ws_bytes, void *cuda_stream);

/*
 * flowmm_decode_attention over the paged 4-bit cache: o = softmax(scale * q . K^T) V over the rows[u] rows of each unit, zero for a unit without rows.  What
 * stands behind a unit's last row (scales of NaN too) has no influence.  Several new queries of a sequence are units that share a row of the block table
 * and differ in rows.  Logits may be as large as fp32 holds them (2^127 in units of log 2; beyond, outputs may be NaN).
 * Accuracy: sums and the softmax are fp32, both products go to the tensor cores as fp16 numbers.  K and V are that exactly.  A bf16 query is, down to 2^-31 of its
 * head's largest element; an fp32 one is two such numbers, within 2^-22 of itself or 2^-39 of the largest.  A weight is rounded to one fp16 number for bf16 rows,
 * within 2^-11 of itself down to 2^-24 of the largest weight, and to two for fp32, within 2^-21 down to 2^-18 of the largest; below that an error stays what it is
 * there.  The sum that weights are divided by takes them unrounded.  Matrix instructions cut their sums off: for fp32 rows these are 16 keys long and added to the
 * nearest, for bf16 as long as what a warp has of a sequence, 2^-23 of them at most for 16 keys (half a million rows of one warp to reach the output's rounding).  Random
 * keys and values, root mean square of the error relative to the output's: bf16 1.7e-3, its own last rounding; fp32 0.7e-7 to 2.5e-7, as with sums in fp32 throughout.
 *   q, out [U, Hq, D] dense, element type `dtype`
 */
flowmm_status flowmm_nibble_attention(const flowmm_cache_params *p, const void *q, const void *k_pages, const void *v_pages,
                                      const void *k_scale, const void *v_scale, const int32_t *block_table, const int32_t *rows,
                                      void *out, void *ws, size_t ws_bytes, void *cuda_stream);

/*
 * Rotary positions: queries and keys turned by their tokens' positions, before the keys are cached or scored.  A row's place in a cache that was
 * compressed is not its token's position any more, so positions are given for every row; image tokens may have three (time, height, width).
 * The first R = rotary_dim channels of a head are R / 2 pairs (a, b), pair i at angle t = position * f_i:
 *   (a, b) -> amplitude * (a cos t - b sin t, b cos t + a sin t);   the other D - R channels are copied
 *   f_i = base^(-2 i / R), by `scaling`: PLAIN as it is; LINEAR f_i / factor; BY_PARTS g f_i + (1 - g) f_i / factor with
 *         g = min(1, max(0, (trained * f_i / (2 pi) - low) / (high - low))): by how many turns the pair makes over the context that was trained on.
 *         Models whose g is a ramp over the pair's number i, between two rounded numbers, are not these: with a factor of 4, 1, 32 and 32 768 trained positions a middle
 *         frequency is up to 1.7 times the other.  For them, and for any other frequencies, the caller writes the table.
 * adjoint = 1 turns by -t: the gradient's way back, and for amplitude 1 the inverse (keys taken out of a cache and put to other positions).
 *
 * flowmm_rotary_table writes what the call needs of the frequencies, once for a model: table [R / 2] uint64, pair i's f_i / (2 pi) as a 64-bit fraction of a
 * turn, within 2^-63.  Positions are multiplied with it modulo whole turns, so any int32 position has its angle within 2^-31 turns (a factor below 1 divides both of
 * these); cos and sin and the products are fp32.  A table of the caller's own is as good: round(2^64 (f_i / (2 pi) mod 1)) for each pair; flowmm_rotary looks at
 * the table alone, not at base, scaling and what goes with it (which have to be valid all the same).
 *
 *   q, q_out [U, Hq, T, D], k, k_out [U, Hkv, T, D] with the element strides given, T = n_rows; q with q_out, or k with k_out, may be NULL (not both).
 *   q_out may be q (the same strides), k_out may be k; otherwise outputs must not overlap inputs.
 *   positions [U, n_axes, T] int32
 * rotary_dim is a multiple of 16 up to head_dim (0: head_dim).  n_axes is 1, or 3: then section[a] pairs go by position a, in order, R / 2 in all.
 * base at least 1, factor above 0, high above low, trained at least 0 are asked for where `scaling` uses them; amplitude 0 selects 1.
 * U * T is below 2^31, Hq + Hkv below 2^30.  No workspace: nothing on the device can fail.
 */
typedef enum { FLOWMM_ROTARY_HALVES = 0,        /* channels i and i + R / 2 are pair i */
               FLOWMM_ROTARY_PAIRS = 1          /* channels 2 i and 2 i + 1 are pair i */
} flowmm_rotary_layout;
typedef enum { FLOWMM_ROTARY_PLAIN = 0, FLOWMM_ROTARY_LINEAR = 1, FLOWMM_ROTARY_BY_PARTS = 2 } flowmm_rotary_scaling;

typedef struct {
    int32_t n_units, n_q_heads, n_kv_heads, head_dim;
    int32_t n_rows;                     /* T */
    int32_t dtype;                      /* flowmm_dtype of q, k and the outputs */
    int32_t rotary_dim;                 /* R */
    int32_t layout;                     /* flowmm_rotary_layout */
    int32_t adjoint;
    int32_t n_axes, section[3];
    int32_t scaling;                    /* flowmm_rotary_scaling */
    float amplitude;
    int32_t trained;                    /* positions of the context that was trained on */
    double base, factor, low, high;
    int64_t q_stride[3], k_stride[3];   /* element strides (unit, head, row) */
    int64_t q_out_stride[3], k_out_stride[3];
} flowmm_rotary_params;

flowmm_status flowmm_rotary_table(const flowmm_rotary_params *p, uint64_t *table, void *cuda_stream);
flowmm_status flowmm_rotary(const flowmm_rotary_params *p, const void *q, const void *k, const int32_t *positions, const uint64_t *table,
                            void *q_out, void *k_out, void *cuda_stream);

/* Waits for `cuda_stream`, then returns the device status word at the start of `ws`
 * (FLOWMM_OK, or the first error a kernel recorded) and clears it. */
flowmm_status flowmm_last_device_status(void *ws, void *cuda_stream);

/*
 * Self-test of the bounded device-side waits (every mbarrier wait inside the tensor-core kernels
 * gives up after about two seconds instead of hanging the GPU).  Enqueues one small kernel whose
 * threads wait for an event that never comes; it returns by itself after the limit and leaves
 * FLOWMM_ERR_TIMEOUT in the status word at the start of `ws`, which flowmm_last_device_status then
 * reports and clears.  The CUDA context stays usable.
 */
flowmm_status flowmm_selftest_wait_timeout(void *ws, void *cuda_stream);

/* Number of kernels the most recent compute entry point of this thread enqueued. */
int32_t flowmm_last_launch_count(void);

/*
 * 1 if the library was compiled with -DFLOWMM_DEBUG, else 0.  The debug build stands in for a memory checker:
 * flowmm_match, flowmm_merge and flowmm_merge_static first check the index lists they are given (inside
 * [0, L), strictly ascending; matches inside [-1, B)), wait for that check and return FLOWMM_ERR_INDEX without
 * launching anything else when a list is bad; inside the kernels every index taken from a list or computed for a
 * gather is range-checked before use, a bad one is skipped and recorded as FLOWMM_ERR_INDEX in the status word.
 * Results of good inputs are the same as the release build's.
 */
int32_t flowmm_debug_build(void);

/*
 * Profiling aid, per host thread, off by default.  While on, every compute entry point records
 * a CUDA event on its stream before its first kernel and after each kernel (one extra event
 * record per launch).  flowmm_profile_read waits for the last of them and fills, in launch
 * order, a static kernel name and the kernel's duration in milliseconds for the most recent
 * entry point; it returns the number of entries written (0 when off, -1 on a CUDA error).
 * The first enable creates the events.
 */
flowmm_status flowmm_profile_enable(int32_t on);
int32_t flowmm_profile_read(const char **names, float *ms, int32_t max_entries);

/* Static, human-readable name of a status code. */
const char *flowmm_status_string(flowmm_status s);

#ifdef __cplusplus
}
#endif
#endif /* FLOWMM_H_ */
