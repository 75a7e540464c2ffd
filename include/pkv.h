/*
 * pkv.h -- C ABI of libpkv: PyramidKV prefill-time KV-cache compression
 * (arXiv 2406.02069) for AMD MI355X (gfx950).
 *
 * For every transformer layer l the library keeps k^l of the n cached tokens
 * of each KV head: the last alpha "instruction" tokens, plus the k^l - alpha
 * prefix tokens that receive the most softmax attention from the instruction
 * queries (Sec. 4.2.2).  The per-layer budgets k^l follow the paper's
 * arithmetic "pyramid" (Sec. 4.2.1).  The kept K/V rows are copied, in
 * ascending position order, into a new smaller cache (appendix "Details of
 * Proposed Method": eviction by gather; appendix on rotary embeddings: kept
 * rows are not re-rotated and positions stay ascending).
 *
 * Conventions
 *  - Plain C, no C++/torch types.  Every function returns a pkv_status
 *    (0 = ok) except the pure size/string helpers.
 *  - Pointers marked DEVICE must be device memory owned by the caller and
 *    stay valid until the work queued on `stream` has finished.  Pointers
 *    marked HOST are read/written synchronously during the call.
 *  - Argument errors are detected on the host before anything is launched
 *    and leave all outputs untouched.
 *  - Launching calls are asynchronous on `stream` (a hipStream_t passed as
 *    void*; NULL = the default stream).  They never synchronise and never
 *    allocate or free memory.  Results are deterministic: the same inputs
 *    give bit-identical outputs.  A layer's do not depend on the number of
 *    layers in the call; the last bits of a sequence's scores can depend on
 *    the number of sequences and heads in it.
 *  - Inputs are never modified.
 *  - The library keeps no state between calls and reads no environment
 *    variables.  (The per-device attributes of its kernels are set on first
 *    use; pkv_compress_layer_noalloc has a built-in scratch buffer per device,
 *    see there.)
 *  - Exclusive use of the device.  Whenever a device with at least 256
 *    compute units is given a shape of G*alpha <= 512 and N <= 262144 without
 *    supplied softmax denominators, the workgroups of the scoring kernel
 *    (256 of a one-pass kernel, 512 of the register-resident one) exchange
 *    softmax sums with each other and must all be resident on the device at
 *    the same time; they fill it completely (registers and LDS of every
 *    compute unit).  (Some shapes of more than 128 query rows take a kernel
 *    without such waits; which ones is not part of the contract.)  The caller must therefore not run other kernels on the device
 *    while such a call executes: no second compress call on another stream,
 *    no other tenant.  Work queued behind it on the same stream is fine.
 *    If the workgroups cannot all be resident, the waits between them are
 *    given up after about 50 ms of wall-clock time each, the call completes,
 *    and every count_out of the call reads -1 (see pkv_compress_layer); it
 *    never hangs.  The variants with supplied denominators
 *    (pkv_compress_layers_lse) have no such waits and share the device
 *    freely.
 */
#ifndef PKV_H_
#define PKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PKV_OK = 0,
  PKV_ERR_INVALID_ARG = 1, /* NULL pointer, bad size, bad stride, bad enum   */
  PKV_ERR_UNSUPPORTED = 2, /* valid in the paper's terms, not built here     */
  PKV_ERR_WORKSPACE = 3,   /* workspace NULL, misaligned or too small        */
  PKV_ERR_HIP = 4,         /* a kernel launch was rejected by the runtime    */
  PKV_ERR_SCRATCH = 5      /* shape needs more than the built-in scratch
                              buffer of pkv_compress_layer_noalloc holds     */
} pkv_status;

typedef enum {
  PKV_POOL_NONE = 0,
  PKV_POOL_MAX = 1,
  PKV_POOL_AVG = 2
} pkv_pool;

/*
 * Per-layer budgets (Sec. 4.2.1, Eq. budget).  HOST only, pure.
 *
 * The alpha instruction tokens are kept in every layer; the pyramid is laid
 * over the remaining A = avg_budget - alpha entries per layer
 * (k_total = L*A): top layer A/beta, bottom layer 2A - A/beta, arithmetic
 * sequence in between.  The real-valued sequence is made integer by flooring
 * and handing the missing units to the layers with the largest fractional
 * parts (ties to the lower layer), so that
 *     sum_l k_out[l] == L * avg_budget   and   k_out[l] >= k_out[l+1].
 * k_out[l] INCLUDES the alpha instruction tokens.  L == 1 gives avg_budget;
 * beta == 1 gives a uniform budget.
 *
 * k_out: HOST, int32[L], written.
 * Errors: L < 1, beta < 1, alpha < 0, avg_budget < alpha, k_out NULL
 *         -> PKV_ERR_INVALID_ARG.
 */
int pkv_budgets(int32_t L, int32_t avg_budget, int32_t beta, int32_t alpha,
                int32_t* k_out);

/*
 * Other allocation strategies of the paper's ablation (appendix "Allocation
 * Strategies", which names a geometric and an exponential decay beside the
 * linear one without a formula; written in the layer index both are
 * r_l = C * q^l, so one schedule stands for the two).
 *   PKV_SCHEDULE_LINEAR     pkv_budgets
 *   PKV_SCHEDULE_GEOMETRIC  r_l = C * q^l over A = avg_budget - alpha, with the
 *                           linear pyramid's ratio of top to bottom layer,
 *                           q^(L-1) = 1/(2 beta - 1), and sum_l r_l = L*A
 *   PKV_SCHEDULE_UNIFORM    k_out[l] = avg_budget (SnapKV-style selection)
 * Integerisation, k_out, ownership and errors as pkv_budgets; an unknown
 * schedule -> PKV_ERR_INVALID_ARG.
 */
typedef enum {
  PKV_SCHEDULE_LINEAR = 0,
  PKV_SCHEDULE_GEOMETRIC = 1,
  PKV_SCHEDULE_UNIFORM = 2
} pkv_schedule;

int pkv_budgets_schedule(int32_t L, int32_t avg_budget, int32_t beta,
                         int32_t alpha, int32_t schedule, int32_t* k_out);

/*
 * Shape of one layer's compression problem.  Strides are in ELEMENTS (bf16);
 * the head dimension is always contiguous.
 */
typedef struct {
  int32_t B;      /* sequences in the batch, >= 1                            */
  int32_t Hq;     /* query heads; Hq % Hkv == 0                              */
  int32_t Hkv;    /* key/value heads                                         */
  int32_t d;      /* head dimension d_k: 64 or 128                           */
  int32_t N;      /* (padded) cached length of K and V, >= 1                 */
  int32_t alpha;  /* instruction-token window, 1 <= alpha <= 64              */
  int32_t k_l;    /* this layer's budget including the window, >= alpha      */
  int32_t pool;   /* pkv_pool                                                */
  int32_t pool_w; /* pooling width, odd, 1..63 (1 == no pooling)             */
  int32_t flags;  /* 0.  (Test and measurement switches, pkv_measure.h:
                     bits outside PKV_FLAG_ALL -> PKV_ERR_INVALID_ARG)       */
  int64_t q_sb, q_sh, q_st;    /* strides of Q_win [B, Hq, alpha, d]         */
  int64_t kv_sb, kv_sh, kv_st; /* strides of K and of V [B, Hkv, N, d]       */
  int64_t o_sb, o_sh, o_st;    /* strides of K_out and V_out
                                  [B, Hkv, k_cap, d], k_cap = min(k_l, N)    */
} pkv_layer_desc;

/*
 * Bytes of DEVICE workspace needed to compress L layers of this shape in one
 * call (L = 1 for pkv_compress_layer), whatever their budgets k_l.
 * HOST only, pure.  Returns 0 if the descriptor is invalid or L is not in
 * 1..1024.
 */
size_t pkv_workspace_bytes(const pkv_layer_desc* desc, int32_t L);

/*
 * Compress one layer (Sec. 4.2.2; gather per the appendix "Details of
 * Proposed Method").
 *
 * For each sequence b with n = seq_lens[b] valid tokens and each KV head g
 * (G = Hq/Hkv query heads h = g*G .. g*G+G-1 share it):
 *   1. if k_l >= n every token is kept;
 *   2. otherwise each window query t (absolute position n-alpha+t) attends
 *      causally: A = softmax over keys 0..n-alpha+t of q.k / sqrt(d)
 *      (Eq. Al), window keys included;
 *   3. s^h_i = sum_t A^{(h,t)}_i for prefix keys i < n-alpha (Eq. att_score),
 *      averaged over the G heads of the group;
 *   4. the scores are pooled along the sequence (stride 1, same length; max
 *      ignores out-of-range neighbours, avg counts them as zero and divides
 *      by pool_w);
 *   5. the k_l-alpha prefix positions with the largest pooled score are
 *      kept (equal scores: the lower position wins), in ascending order,
 *      followed by the window positions n-alpha .. n-1;
 *   6. K_out/V_out rows are bit copies of the kept K/V rows.
 * Arithmetic: bf16 inputs, fp32 accumulation and scores.
 *
 * desc       HOST.
 * Q_win      DEVICE bf16 [B,Hq,alpha,d]: queries of the LAST alpha valid
 *            tokens of each sequence (positions n_b-alpha .. n_b-1), as used
 *            by attention (after any rotary embedding).
 * K, V       DEVICE bf16 [B,Hkv,N,d], same strides.  Rows >= n_b are never
 *            read.  V is read only at the kept rows.
 * seq_lens   DEVICE int32[B] with 0 <= n_b <= N, or NULL (all n_b == N).
 *            Values outside the range are clamped on the device.
 *            If n_b <= k_l all n_b tokens are kept (this covers n_b < alpha).
 * K_out,V_out DEVICE bf16 [B,Hkv,k_cap,d], written.  Rows >= count are zero.
 * idx_out    DEVICE int32 [B,Hkv,k_cap] contiguous, written: kept positions,
 *            ascending; the last min(alpha,n_b) valid entries are the window;
 *            entries >= count are -1.
 * count_out  DEVICE int32 [B], written: min(k_l, n_b); or -1 for every
 *            sequence if the scoring kernel had to give up a wait between
 *            its workgroups (they exchange softmax statistics and rely on
 *            being resident on the device together; another tenant of the
 *            device can prevent that).  Every wait is bounded, so the call
 *            always completes; with count -1 the other outputs of the call
 *            are in range but meaningless and the call should be repeated.
 * scores_out DEVICE fp32 [B,Hkv,N] contiguous, or NULL: pooled scores before
 *            selection, defined for i < n_b-alpha when k_l < n_b; other
 *            entries are left untouched.
 * workspace  DEVICE, 256-byte aligned, >= pkv_workspace_bytes(desc, 1) bytes;
 *            contents on entry are irrelevant, contents on exit undefined
 *            (except as pkv_attention_recall uses them).
 *            Calls that may overlap in time need distinct workspaces (and
 *            see "Exclusive use of the device" above).
 * stream     hipStream_t.
 *
 * Errors: PKV_ERR_INVALID_ARG (NULL required pointer, shape/stride rules
 * above violated, unknown flags), PKV_ERR_UNSUPPORTED (d not 64/128,
 * alpha > 64, pool_w > 63), PKV_ERR_WORKSPACE, PKV_ERR_HIP.
 */
int pkv_compress_layer(const pkv_layer_desc* desc, const void* Q_win,
                       const void* K, const void* V, const int32_t* seq_lens,
                       void* K_out, void* V_out, int32_t* idx_out,
                       int32_t* count_out, float* scores_out, void* workspace,
                       size_t workspace_bytes, void* stream);

/*
 * pkv_compress_layer for callers that cannot hand over a workspace and must
 * not cause an allocation: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, results and errors as
 * pkv_compress_layer, without the workspace: the kernels use a scratch
 * buffer of PKV_NOALLOC_SCRATCH_BYTES that is part of the library's device
 * image (every device the library runs on holds one until the process ends).
 * The call allocates and frees nothing, on the host or on the device.
 *
 * A shape whose pkv_workspace_bytes(desc, 1) exceeds
 * PKV_NOALLOC_SCRATCH_BYTES -> PKV_ERR_SCRATCH, nothing launched.  (32 MiB
 * serve, e.g., B*Hkv = 8 heads of 262144 keys, or 64 heads of 32768.)
 * All calls on one device share that device's buffer: calls that may overlap
 * in time on one device race and give undefined results; serialise them (one
 * stream, or events).  The buffer keeps the last call's contents; the call
 * clears what it needs cleared itself.
 */
#define PKV_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)

int pkv_compress_layer_noalloc(const pkv_layer_desc* desc, const void* Q_win,
                               const void* K, const void* V,
                               const int32_t* seq_lens, void* K_out,
                               void* V_out, int32_t* idx_out,
                               int32_t* count_out, float* scores_out,
                               void* stream);

/*
 * Compress L layers of one request batch (the whole prefill-time step: every
 * layer has its own Q_win/K/V and its own budget descs[l].k_l, Sec. 4.2.1).
 * Same results as L calls of pkv_compress_layer, queued so that independent
 * stages of neighbouring layers can overlap on the device.
 *
 * descs      HOST, L descriptors.  All fields except k_l and the output
 *            strides must be equal across layers.
 * Q_win, K, V, K_out, V_out, idx_out, count_out, scores_out
 *            HOST arrays of L DEVICE pointers, each as in
 *            pkv_compress_layer (scores_out may be NULL, or hold NULLs).
 * seq_lens   DEVICE int32[B] or NULL; shared by all layers.
 * workspace  DEVICE, >= pkv_workspace_bytes(&descs[0], L) bytes.
 * Errors: as pkv_compress_layer; additionally L outside 1..1024 or differing
 * layer shapes -> PKV_ERR_INVALID_ARG.
 */
int pkv_compress_layers(int32_t L, const pkv_layer_desc* descs,
                        const void* const* Q_win, const void* const* K,
                        const void* const* V, const int32_t* seq_lens,
                        void* const* K_out, void* const* V_out,
                        int32_t* const* idx_out, int32_t* const* count_out,
                        float* const* scores_out, void* workspace,
                        size_t workspace_bytes, void* stream);

/*
 * pkv_compress_layers with the softmax denominators of the window queries
 * supplied by the caller.  The scores of Sec. 4.2.2 are taken from the
 * attention of the instruction tokens, which prefill has already computed;
 * an attention kernel that keeps its per-row log-sum-exp hands it over here,
 * and the keys are then swept once instead of twice (no statistics sweep, no
 * exchange between workgroups).
 *
 * lse        HOST array of L DEVICE pointers, each fp32 [B,Hq,alpha]
 *            contiguous: lse[b][h][t] = ln sum_{i <= n_b-alpha+t}
 *            exp(q_{b,h,t} . k_{b,g(h),i} / sqrt(d)), the natural log of the
 *            denominator of window query t's causal softmax (Eq. Al), window
 *            keys included.  The attention of step 2 becomes
 *            exp(q.k/sqrt(d) - lse) and is not renormalised: results equal
 *            pkv_compress_layers' to the accuracy of the supplied values.
 *            Entries of sequences with n_b <= k_l are not read.  Non-finite
 *            entries give meaningless (but in-range) selections.
 * Everything else, and the errors, as pkv_compress_layers; a NULL lse or a
 * NULL or misaligned lse[l] -> PKV_ERR_INVALID_ARG.  count_out is never -1
 * here (nothing waits).
 */
int pkv_compress_layers_lse(int32_t L, const pkv_layer_desc* descs,
                            const void* const* Q_win, const void* const* K,
                            const void* const* V, const float* const* lse,
                            const int32_t* seq_lens, void* const* K_out,
                            void* const* V_out, int32_t* const* idx_out,
                            int32_t* const* count_out,
                            float* const* scores_out, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * Per-layer paged output (appendix "PyramidKV Implementation at vLLM": every
 * layer keeps a different number of tokens, so every layer gets its own
 * block table and page pool instead of a share of one uniform paged cache).
 * As pkv_compress_layers (lse NULL) or pkv_compress_layers_lse (lse given),
 * except that the kept rows go straight into pages:
 *   kept row j (0 <= j < count_b) of sequence b, KV head g, layer l
 *     -> K_pages[l] / V_pages[l], page block_tables[l][b][j / page_size],
 *        head g, slot j % page_size.
 * Nothing else in the pools is written (a partly filled last page keeps its
 * old content behind the kept rows); descs[l].o_* are checked as usual but
 * not used.
 */
typedef struct {
  int32_t page_size; /* tokens per page, >= 1                                */
  int32_t num_pages; /* pages in each layer's pool                           */
  int32_t max_pages; /* entries per sequence in each block table,
                        >= ceil(min(k_l, N) / page_size) for every layer     */
  int32_t reserved;  /* must be 0                                            */
} pkv_paged_desc;

/*
 * paged        HOST.
 * K_pages, V_pages
 *              HOST arrays of L DEVICE pointers, each bf16
 *              [num_pages, Hkv, page_size, d] contiguous, 16-byte aligned.
 * block_tables HOST array of L DEVICE pointers, each int32 [B, max_pages]
 *              contiguous: page numbers in [0, num_pages).  Entries beyond
 *              ceil(count_b / page_size) are not read.  A page number out of
 *              range is never written through: the row is dropped and
 *              count_out[l][b] is set to -2.
 * idx_out, count_out, scores_out, seq_lens, workspace, stream: as
 * pkv_compress_layers.
 * Errors: as pkv_compress_layers(_lse); paged NULL or inconsistent (sizes
 * < 1, reserved != 0, max_pages too small for a layer's budget), a NULL or
 * misaligned table -> PKV_ERR_INVALID_ARG.
 */
int pkv_compress_layers_paged(int32_t L, const pkv_layer_desc* descs,
                              const void* const* Q_win, const void* const* K,
                              const void* const* V, const float* const* lse,
                              const int32_t* seq_lens,
                              const pkv_paged_desc* paged,
                              void* const* K_pages, void* const* V_pages,
                              const int32_t* const* block_tables,
                              int32_t* const* idx_out,
                              int32_t* const* count_out,
                              float* const* scores_out, void* workspace,
                              size_t workspace_bytes, void* stream);

/*
 * Attention recall rate of the kept sets (appendix, "Attention Recall Rate
 * Experiment"): the share of the window queries' attention over all keys
 * that falls on the kept keys, averaged over the G*alpha window queries of
 * a KV head: 1 - (window score mass on the dropped prefix keys) / alpha.
 *
 * Call it right after a pkv_compress_layers / _lse / _paged call, with the
 * same L, descs, seq_lens and workspace, on the same stream and before
 * anything else uses the workspace: it reads the un-pooled window scores
 * that the call left there, and the call's idx_out.
 *
 * lse_supplied 1 if the call was given lse, else 0.
 * idx_out      HOST array of L DEVICE pointers: the call's idx_out.
 * recall_out   HOST array of L DEVICE pointers, each fp32 [B,Hkv], written:
 *              1 for sequences that keep everything.
 * Errors: as pkv_compress_layers for descs, pointers and workspace.
 */
int pkv_attention_recall(int32_t L, const pkv_layer_desc* descs,
                         int32_t lse_supplied, const int32_t* seq_lens,
                         const int32_t* const* idx_out,
                         float* const* recall_out, const void* workspace,
                         size_t workspace_bytes, void* stream);

/*
 * The step after the path: decoding attention of one new query per sequence
 * over a layer's compacted cache (Sec. 3: after compression the model attends
 * over the kept keys and values only).  The kept rows carry the rotary phases
 * of their original positions, so q is taken as given (rotated at its own
 * position by the caller) and nothing is re-rotated.
 *   out[b][h] = sum_{j < count_b} softmax_j(q_bh . K_bgj / sqrt(d)) V_bgj,
 *   g = h / (Hq/Hkv);  fp32 accumulation and output.
 * The cache is what pkv_compress_layer(s) wrote (page_size 0: compact
 * [B,Hkv,k_cap,d] with strides c_*) or what pkv_compress_layers_paged wrote
 * (page_size > 0: pool [num_pages,Hkv,page_size,d] with this layer's block
 * table; a page number out of range makes its rows count as absent).
 */
typedef struct {
  int32_t B, Hq, Hkv; /* Hq % Hkv == 0, Hq/Hkv <= 8                          */
  int32_t d;          /* 64 or 128                                           */
  int32_t k_cap;      /* rows per sequence the cache can hold, <= 4096       */
  int32_t page_size;  /* 0: compact cache; > 0: paged                        */
  int32_t num_pages;  /* paged: pages in the pool                            */
  int32_t max_pages;  /* paged: entries per sequence in the block table,
                         >= ceil(k_cap / page_size)                          */
  int32_t reserved;   /* must be 0                                           */
  int32_t reserved2;  /* padding, ignored                                    */
  int64_t c_sb, c_sh, c_st; /* compact: element strides of K_cache/V_cache   */
} pkv_decode_desc;

/*
 * Bytes of DEVICE workspace pkv_decode_attention needs for this shape (0 for
 * shapes it serves with one workgroup per sequence and head; 0 as well if
 * the descriptor is invalid).  HOST only, pure.
 */
size_t pkv_decode_workspace_bytes(const pkv_decode_desc* desc);

/*
 * desc        HOST.
 * q           DEVICE bf16 [B,Hq,d] contiguous, 16-byte aligned.
 * K_cache, V_cache  DEVICE bf16, layouts above, 16-byte aligned.
 * block_table DEVICE int32 [B,max_pages] (paged) or NULL (compact).
 * count       DEVICE int32 [B]: valid rows per sequence (count_out of the
 *             compression call); values outside [0, k_cap] are clamped, so
 *             the error codes -1 / -2 read as an empty cache.
 * out         DEVICE fp32 [B,Hq,d] contiguous, written (zero rows for an
 *             empty cache).
 * lse_out     DEVICE fp32 [B,Hq] or NULL: natural log of the softmax
 *             denominator (-inf for an empty cache).
 * workspace   DEVICE, 256-byte aligned, >= pkv_decode_workspace_bytes(desc)
 *             bytes (may be NULL when that is 0); contents irrelevant on
 *             entry, undefined on exit; concurrent calls need distinct ones.
 * stream      hipStream_t.  Asynchronous, never allocates.
 * Errors: PKV_ERR_INVALID_ARG (NULL / misaligned pointers, shape or stride
 * rules violated), PKV_ERR_UNSUPPORTED (d, Hq/Hkv > 8, k_cap > 4096),
 * PKV_ERR_WORKSPACE, PKV_ERR_HIP.
 */
int pkv_decode_attention(const pkv_decode_desc* desc, const void* q,
                         const void* K_cache, const void* V_cache,
                         const int32_t* block_table, const int32_t* count,
                         float* out, float* lse_out, void* workspace,
                         size_t workspace_bytes, void* stream);

/*
 * pkv_decode_attention over the caches of L layers in one call (Sec. 3; the
 * per-layer budgets of Sec. 4.2.1 make the layers' caches unequal and, at
 * small batch, small: a launch per layer costs more than the rows it reads).
 * For callers that hold the queries of several layers at once; a decoder
 * that computes layer l+1's query from layer l's output calls
 * pkv_decode_attention per layer.
 *   descs[l]  HOST, L descriptors.  B, Hq, Hkv, d and page_size must be the
 *             same for all layers; k_cap, num_pages, max_pages and the c_*
 *             strides are per layer.
 *   q, K_cache, V_cache, block_tables, count, out, lse_out
 *             HOST arrays of L DEVICE pointers, each as in
 *             pkv_decode_attention.  block_tables may be NULL for compact
 *             caches; lse_out may be NULL (no log-sum-exp output), else all
 *             L entries are written through.
 *   workspace DEVICE, 256-byte aligned,
 *             >= pkv_decode_layers_workspace_bytes(L, descs) bytes (may be
 *             NULL when that is 0); contents irrelevant on entry, undefined
 *             on exit; concurrent calls need distinct ones.
 * Every layer's result is what pkv_decode_attention gives for it, up to the
 * order of the fp32 additions (the key ranges are cut differently).
 * Asynchronous on `stream`, never allocates.  Errors as for
 * pkv_decode_attention; layers that differ in B, Hq, Hkv, d or page_size ->
 * PKV_ERR_INVALID_ARG.
 */
size_t pkv_decode_layers_workspace_bytes(int32_t L,
                                         const pkv_decode_desc* descs);
int pkv_decode_attention_layers(int32_t L, const pkv_decode_desc* descs,
                                const void* const* q,
                                const void* const* K_cache,
                                const void* const* V_cache,
                                const int32_t* const* block_tables,
                                const int32_t* const* count,
                                float* const* out, float* const* lse_out,
                                void* workspace, size_t workspace_bytes,
                                void* stream);

/*
 * Element types of the operators below (rotary positions, prompt attention,
 * attention over long caches).  The compression calls take bf16.
 */
typedef enum { PKV_BF16 = 0, PKV_FP16 = 1 } pkv_dtype;

/* Which elements of a head turn together: (i, i + rot/2), or (2i, 2i + 1). */
typedef enum { PKV_ROTARY_HALF = 0, PKV_ROTARY_INTERLEAVED = 1 } pkv_rotary_layout;

/*
 * Frequencies of rotary positions, for contexts longer than the trained one
 * too.  HOST only, pure; in 64 bits.  With f_i = base^(-2i/rot), i < rot/2:
 *   PKV_ROTARY_PLAIN   f_i
 *   PKV_ROTARY_LINEAR  f_i / factor (positions are interpolated)
 *   PKV_ROTARY_BANDS   by the turns u_i = trained * f_i / 2 pi that fit into
 *                      the trained context: f_i / factor up to `low` turns,
 *                      f_i from `high` turns on, between them the blend
 *                      (1 - s) f_i / factor + s f_i, s = (u_i - low)/(high - low)
 *   PKV_ROTARY_RAMP    with c(u) = rot ln(trained / 2 pi u) / (2 ln base), the
 *                      pair that makes u turns: f_i / factor above
 *                      ceil(c(low)), f_i below floor(c(high)) (both clamped to
 *                      0 .. rot - 1), a ramp over the pairs' numbers between;
 *                      magnitude 0.1 ln(factor) + 1 where factor > 1
 * inv_freq_out  HOST, double[rot/2], written: radians per position.
 * magnitude_out HOST, written: factor for cosine and sine (1 but for RAMP).
 * Errors: rot odd or outside 2..256, base <= 1, factor < 1 or trained, low or
 * high not positive or low >= high where they are used, any of them not
 * finite, NULL -> PKV_ERR_INVALID_ARG.
 */
typedef enum {
  PKV_ROTARY_PLAIN = 0,
  PKV_ROTARY_LINEAR = 1,
  PKV_ROTARY_BANDS = 2,
  PKV_ROTARY_RAMP = 3
} pkv_rotary_scaling;

int pkv_rotary_frequencies(int32_t rot, int32_t scaling, double base,
                           double factor, double trained, double low,
                           double high, double* inv_freq_out,
                           float* magnitude_out);

/*
 * Rotary positions of new tokens, and their append to a cache: the step in
 * front of the compression (all tokens of a prompt; the calls above take
 * rotated queries and keys) and in front of each decoding step (one token per
 * sequence behind the rows that were kept; Sec. 3).
 *   y_a = m (x_a cos(p f_i) - x_b sin(p f_i)),
 *   y_b = m (x_b cos(p f_i) + x_a sin(p f_i))
 * for the pairs (a, b) of the first `rot` elements of a head; the other
 * elements are copied.  The angle is formed in 64 bits, the sums in fp32, one
 * rounding to the type at the end.
 * Token t < new_b of sequence b has row r = count_b - new_b + t of the cache
 * and position p = positions[b][t], or r if positions is NULL.  Its rotated
 * keys and its values go to row r of K_cache and V_cache.  A row outside
 * [0, k_cap), or one whose page number is out of range, is never written: it
 * is dropped and counted.  Nothing else of the caches is written.  A row that
 * two tokens are given (by a page that two sequences name) holds one of them
 * afterwards, not necessarily the same for every head.
 */
typedef struct {
  int32_t B, Hq, Hkv; /* sequences, query heads, key/value heads, >= 1       */
  int32_t d;          /* 64 or 128                                           */
  int32_t T;          /* tokens per sequence in q, k and v, >= 1             */
  int32_t rot;        /* elements of a head that turn: 8 .. d, a multiple
                         of 8                                                */
  int32_t layout;     /* pkv_rotary_layout                                   */
  int32_t dtype;      /* pkv_dtype                                           */
  int32_t k_cap;      /* rows per sequence the cache can hold                */
  int32_t page_size;  /* 0: compact cache; > 0: pages                        */
  int32_t num_pages;  /* pages in the pool                                   */
  int32_t max_pages;  /* entries per sequence in the block table,
                         >= ceil(k_cap / page_size)                          */
  float magnitude;    /* m, finite                                           */
  int32_t reserved;   /* must be 0                                           */
  int64_t q_sb, q_sh, q_st; /* element strides of q [B,Hq,T,d]               */
  int64_t k_sb, k_sh, k_st; /* of k [B,Hkv,T,d]                              */
  int64_t v_sb, v_sh, v_st; /* of v [B,Hkv,T,d]                              */
  int64_t o_sb, o_sh, o_st; /* of q_out [B,Hq,T,d]                           */
  int64_t c_sb, c_sh, c_st; /* of a compact K_cache and V_cache
                               [B,Hkv,k_cap,d]                               */
  int64_t p_sb, p_sh;       /* of pos_cache [B,Hkv,k_cap]                    */
} pkv_rotary_desc;

/*
 * desc        HOST.  Strides are >= 0 and multiples of 8 (p_*: any >= 0);
 *             those of tensors that are not given are not looked at.
 * q, q_out    DEVICE, 16-byte aligned, both or neither NULL.  q_out may be q
 *             with the same strides, and overlaps it in no other way.  Rows
 *             t >= new_b are neither read nor written.
 * k, v, K_cache, V_cache
 *             DEVICE, 16-byte aligned, all or none NULL; compact caches with
 *             strides c_*, or pools [num_pages,Hkv,page_size,d] contiguous.
 *             They overlap in one way at most: a compact cache may be k (and
 *             v) itself, same strides, where every row r is t.
 * inv_freq    DEVICE double[rot/2]: radians per position.
 * positions   DEVICE int32 [B,T] contiguous, or NULL.  Any value.
 * new_lens    DEVICE int32 [B]: new_b, clamped to 0..T; NULL: T.
 * count       DEVICE int32 [B]: rows of the cache that are valid once the new
 *             tokens are there (never written: a decoder adds 1 to all layers'
 *             counts before a step); NULL: new_b.
 * block_table DEVICE int32 [B,max_pages] contiguous (paged) or NULL.
 * pos_cache   DEVICE int32 [B,Hkv,k_cap] or NULL: the positions of the cache's
 *             rows (idx_out of a compression call, with room behind it);
 *             pos_cache[b][g][r] = p is written for every g.
 * dropped_out DEVICE int32 [B] or NULL, written: tokens of b that were dropped.
 * Asynchronous on `stream`, needs no workspace, never allocates.
 * Errors: PKV_ERR_INVALID_ARG, PKV_ERR_UNSUPPORTED (d not 64/128, rot not a
 * multiple of 8, B or B * T / 16 > 2^24 - 1, Hq + 2 Hkv > 65535), PKV_ERR_HIP.
 */
int pkv_rotary_append(const pkv_rotary_desc* desc, const void* q,
                      const void* k, const void* v, const double* inv_freq,
                      const int32_t* positions, const int32_t* new_lens,
                      const int32_t* count, const int32_t* block_table,
                      void* q_out, void* K_cache, void* V_cache,
                      int32_t* pos_cache, int32_t* dropped_out, void* stream);

/*
 * Attention of a prompt, or of the last part of one, over its keys: where the
 * window queries' softmax denominators that pkv_compress_layers_lse takes
 * come from, and the prompt's attention itself.
 * Query row t of sequence b has position p = q_start_b + t.  It is there if
 * 0 <= p < n_b, and sees the keys j with lo <= j <= hi,
 *   lo = max(doc_start[b][p], p - window + 1, 0),
 *   hi = max(p, prefix_end[b][p] - 1), and j < n_b
 * (without doc_start, window or prefix_end: without their part).
 *   s_j = q_p . k_j * scale;  cap > 0: s_j = cap tanh(s_j / cap);
 *   slopes: s_j -= slopes[h] |p - j|
 *   out[b][h][t] = sum_j softmax_j(s) V_j,  lse[b][h][t] = ln sum_j exp(s_j)
 * Rows that are not there, or see no key: zero and -inf.
 * fp32 scores, sums and accumulation; the softmax weights are rounded to the
 * input's type for the product with V (fp16: those below 2^-22 of the row's
 * largest are off by up to 2^-33 of it).  Rows >= n_b of K and V are never
 * read.  A key that a query does not see has no influence on its row beyond
 * rounding, whatever it holds (NaN and infinities included).  Where a query
 * sees values of V that are not finite, that element of out is their sum:
 * every weight is positive, however small.
 * The same call gives the same bits.  What a row is rounded to may depend on
 * the call's other rows and sequences: ranges of keys go by all lengths, and
 * rows of a tile are scaled anew together.
 */
typedef struct {
  int32_t B, Hq, Hkv; /* Hq % Hkv == 0                                       */
  int32_t d;          /* 64 or 128                                           */
  int32_t T;          /* query rows per sequence, >= 1                       */
  int32_t N;          /* (padded) length of K and V, >= 1                    */
  int32_t dtype;      /* pkv_dtype                                           */
  int32_t window;     /* 0: none; > 0: keys a query sees, itself included    */
  float scale;        /* > 0; 0: 1/sqrt(d)                                   */
  float cap;          /* 0: none; > 0                                        */
  int64_t q_sb, q_sh, q_st;    /* element strides of q [B,Hq,T,d]            */
  int64_t kv_sb, kv_sh, kv_st; /* of K and of V [B,Hkv,N,d]                  */
  int64_t o_sb, o_sh, o_st;    /* of out [B,Hq,T,d]                          */
} pkv_prefill_desc;

/*
 * Bytes of DEVICE workspace that pkv_prefill_attention needs for this shape
 * with whatever arguments (up to 204 MB for several long sequences, whose
 * ranges go by their lengths, up to 102 MB otherwise; 0 where one sequence's
 * query rows fill the device, and for short ones), and what it needs without
 * seq_lens and q_start (0 as well where all sequences' rows together fill the
 * device).  0 if the descriptor is invalid.  HOST only, pure.
 */
size_t pkv_prefill_workspace_bytes(const pkv_prefill_desc* desc);
size_t pkv_prefill_even_workspace_bytes(const pkv_prefill_desc* desc);

/*
 * desc       HOST.  Strides are >= 0 and multiples of 8.
 * q, K, V, out
 *            DEVICE, of the descriptor's type, 16-byte aligned; out overlaps
 *            nothing, and its rows not one another.
 * seq_lens   DEVICE int32 [B]: n_b, clamped to 0..N; NULL: N.
 * q_start    DEVICE int32 [B] or NULL (0).  Any value.
 * doc_start  DEVICE int32 [B,N] contiguous or NULL: where the document of
 *            position p begins.  Any value.
 * prefix_end DEVICE int32 [B,N] contiguous or NULL: the position behind the
 *            keys that p sees although they lie behind it.  Any value.
 * slopes     DEVICE fp32 [Hq] or NULL.  Finite.
 * lse_out    DEVICE fp32 [B,Hq,T] contiguous, or NULL.  With scale 0 and
 *            neither cap, slopes, window, doc_start nor prefix_end, the rows
 *            of the last alpha tokens are what pkv_compress_layers_lse takes.
 * workspace  DEVICE, 256-byte aligned, >= pkv_prefill_workspace_bytes(desc)
 *            bytes, or _even_workspace_bytes without seq_lens and q_start (may
 *            be NULL when that is 0); contents irrelevant on entry, undefined
 *            on exit; concurrent calls need distinct ones.
 * Asynchronous on `stream`, never allocates.
 * Errors: PKV_ERR_INVALID_ARG (also a scale, a cap, or a quotient of theirs
 * that is not a finite fp32 in units of log2), PKV_ERR_UNSUPPORTED (d not
 * 64/128, Hq/Hkv > 128, B > 65535, N or T > 2^30, T * Hq/Hkv > 2^31 - 256,
 * kv_st > 2^23, more than 2^24 - 1 workgroups of 128 rows),
 * PKV_ERR_WORKSPACE, PKV_ERR_HIP.
 */
int pkv_prefill_attention(const pkv_prefill_desc* desc, const void* q,
                          const void* K, const void* V,
                          const int32_t* seq_lens, const int32_t* q_start,
                          const int32_t* doc_start, const int32_t* prefix_end,
                          const float* slopes, void* out, float* lse_out,
                          void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * pkv_decode_attention for caches of any length and any number of query heads
 * per KV head: the single-token form of pkv_prefill_attention.  Rows of the
 * cache are keys 0 .. count_b - 1 with the positions positions[b][g][j] (the
 * kept rows of a compression call: its idx_out), or j if positions is NULL;
 * the query's position is q_pos_b, or count_b - 1 if q_pos is NULL.  A row is
 * seen if 0 <= position <= q's and, with a window, position > q's - window.
 * Scores, softmax, lse, rounding and values that are not finite as
 * pkv_prefill_attention has them; the softmax weights keep 16 bits and more
 * (fp16: those below 2^-22 of the row's largest are off by up to 2^-38 of it).
 * A page number out of range makes its rows count as absent.
 */
typedef struct {
  int32_t B, Hq, Hkv; /* Hq % Hkv == 0                                       */
  int32_t d;          /* 64 or 128                                           */
  int32_t k_cap;      /* rows per sequence the cache can hold                */
  int32_t page_size;  /* 0: compact cache; > 0: paged                        */
  int32_t num_pages;  /* paged: pages in the pool                            */
  int32_t max_pages;  /* paged: entries per sequence in the block table,
                         >= ceil(k_cap / page_size)                          */
  int32_t dtype;      /* pkv_dtype                                           */
  int32_t window;     /* 0: none; > 0                                        */
  float scale;        /* > 0; 0: 1/sqrt(d)                                   */
  float cap;          /* 0: none; > 0                                        */
  int64_t q_sb, q_sh;       /* element strides of q [B,Hq,d]                 */
  int64_t c_sb, c_sh, c_st; /* compact: of K_cache and V_cache
                               [B,Hkv,k_cap,d]                               */
  int64_t p_sb, p_sh;       /* of positions [B,Hkv,k_cap]                    */
} pkv_decode_long_desc;

/*
 * Bytes of DEVICE workspace pkv_decode_attention_long needs for this shape (0
 * for shapes it serves with one workgroup per sequence and head; 0 as well if
 * the descriptor is invalid).  HOST only, pure.
 */
size_t pkv_decode_long_workspace_bytes(const pkv_decode_long_desc* desc);

/*
 * desc        HOST.  Strides are >= 0 and multiples of 8 (p_*: any >= 0).
 * q           DEVICE, of the descriptor's type, 16-byte aligned.
 * K_cache, V_cache
 *             DEVICE, 16-byte aligned: compact with strides c_*, or pools
 *             [num_pages,Hkv,page_size,d] contiguous.
 * block_table DEVICE int32 [B,max_pages] contiguous (paged) or NULL.
 * count       DEVICE int32 [B], clamped to 0..k_cap.
 * positions   DEVICE int32 or NULL.
 * q_pos       DEVICE int32 [B] or NULL.
 * slopes      DEVICE fp32 [Hq] or NULL.  Finite.
 * out         DEVICE [B,Hq,d] contiguous, of the descriptor's type, 16-byte
 *             aligned, written (zero where no row is seen).
 * lse_out     DEVICE fp32 [B,Hq] contiguous, or NULL (-inf where no row is
 *             seen).
 * workspace   as pkv_decode_attention's, pkv_decode_long_workspace_bytes.
 * Asynchronous on `stream`, never allocates.
 * Errors: PKV_ERR_INVALID_ARG (also a scale, a cap, or a quotient of theirs
 * that is not a finite fp32 in units of log2), PKV_ERR_UNSUPPORTED (d not
 * 64/128, Hq/Hkv > 128, B or Hkv > 65535, B * Hq > 2^24 - 1, k_cap or c_st >
 * 2^30, a pool of more than 2^32 - 1 rows), PKV_ERR_WORKSPACE, PKV_ERR_HIP.
 */
int pkv_decode_attention_long(const pkv_decode_long_desc* desc, const void* q,
                              const void* K_cache, const void* V_cache,
                              const int32_t* block_table,
                              const int32_t* count, const int32_t* positions,
                              const int32_t* q_pos, const float* slopes,
                              void* out, float* lse_out, void* workspace,
                              size_t workspace_bytes, void* stream);

/*
 * ---- A cache in use ----
 *
 * What a decoder does with a cache besides pkv_decode_attention_long: several
 * drafted tokens at once, a record of how much attention each row has had with
 * the eviction of the rows that have had least, and steps that attend over a
 * part of the rows only.
 */

/*
 * Attention of drafted tokens over a cache: each sees the cache's rows and, of
 * the drafted tokens, those that its bits name (in a tree of guesses: its
 * ancestors and itself).  The drafted tokens are the last new_b rows of the
 * cache, where pkv_rotary_append has put them: token t < new_b has row
 * count_b - new_b + t.  What is verified is appended again behind the past rows
 * (pkv_rotary_append with the smaller count), which overwrites the rest.
 *   s_j = q_t . k_j * scale;  cap > 0: s_j = cap tanh(s_j / cap);
 *   slopes: s_j -= slopes[h] |q_pos_t - position_j|
 *   out[b][h][t] = sum_j softmax_j(s) V_j,  lse[b][h][t] = ln sum_j exp(s_j)
 * over the rows 0 <= j < count_b, position_j >= 0, of which token t sees
 *   of the past (j < count_b - new_b)  those with position_j <= q_pos_t,
 *   of the drafted tokens u            those with bit u of tree[b][t] set
 *                                      (tree NULL: u <= t),
 *   with a window                      of these those with position_j > q_pos_t - window.
 * Without positions and q_pos a past row's position is its number, a drafted
 * token's count_b - new_b + the number of drafted tokens that it sees besides
 * itself.  Rows t >= new_b, and rows that see nothing: zero and -inf.
 * Scores, softmax and lse as pkv_decode_attention_long has them, the softmax
 * weights' rounding too, or, where T * Hq/Hkv > 32, as pkv_prefill_attention
 * has it: a token's bits depend on how many there are beside it.  A key that a
 * token does not see has no influence on its row beyond rounding, whatever it
 * holds; where a token sees values of V that are not finite, that element of
 * out is their sum.  A page number out of range makes its rows count as absent.
 */
typedef struct {
  int32_t B, Hq, Hkv; /* Hq % Hkv == 0                                       */
  int32_t d;          /* 64 or 128                                           */
  int32_t T;          /* drafted tokens per sequence in q, 1..256            */
  int32_t k_cap;      /* rows per sequence the cache can hold                */
  int32_t page_size;  /* 0: compact cache; > 0: paged                        */
  int32_t num_pages;  /* paged: pages in the pool                            */
  int32_t max_pages;  /* paged: entries per sequence in the block table,
                         >= ceil(k_cap / page_size)                          */
  int32_t dtype;      /* pkv_dtype                                           */
  int32_t window;     /* 0: none; > 0                                        */
  int32_t reserved;   /* must be 0                                           */
  float scale;        /* > 0; 0: 1/sqrt(d)                                   */
  float cap;          /* 0: none; > 0                                        */
  int64_t q_sb, q_sh, q_st; /* element strides of q [B,Hq,T,d]               */
  int64_t c_sb, c_sh, c_st; /* compact: of K_cache and V_cache
                               [B,Hkv,k_cap,d]                               */
  int64_t p_sb, p_sh;       /* of positions [B,Hkv,k_cap]                    */
  int64_t o_sb, o_sh, o_st; /* of out [B,Hq,T,d]                             */
} pkv_tree_desc;

/*
 * Bits of a tree of T drafted tokens (1..256) from each one's parent: a token
 * in front of it, or -1 (it follows the past directly).
 * parents  HOST int32[T].
 * bits_out HOST int32[T][ceil(T / 32)], written: bit u % 32 of word u / 32 of
 *          row t is set for t itself and its ancestors.
 * HOST only, pure.  Errors: T outside 1..256, a parent outside -1..t-1, NULL
 * -> PKV_ERR_INVALID_ARG (nothing is written).
 */
int pkv_tree_bits(int32_t T, const int32_t* parents, int32_t* bits_out);

/* Bytes of DEVICE workspace that pkv_tree_attention needs for this shape; 0 if
 * the descriptor is invalid.  HOST only, pure. */
size_t pkv_tree_workspace_bytes(const pkv_tree_desc* desc);

/*
 * desc        HOST.  Strides are >= 0 and multiples of 8 (p_*: any >= 0).
 * q, out      DEVICE, of the descriptor's type, 16-byte aligned; out overlaps
 *             nothing, and its rows not one another: sorted by size, each of
 *             its strides reaches behind all that the smaller ones span.
 * K_cache, V_cache
 *             DEVICE, 16-byte aligned: compact with strides c_*, or pools
 *             [num_pages,Hkv,page_size,d] contiguous.
 * block_table DEVICE int32 [B,max_pages] contiguous (paged) or NULL.
 * count       DEVICE int32 [B]: valid rows, drafted tokens included.
 * new_lens    DEVICE int32 [B]: new_b, clamped to 0..T; NULL: T.
 * tree        DEVICE int32 [B,T,ceil(T / 32)] contiguous, or NULL.
 * positions, q_pos
 *             DEVICE int32 [B,Hkv,k_cap] and int32 [B,T] contiguous, both or
 *             neither NULL.  Any value.
 * slopes      DEVICE fp32 [Hq] or NULL.  Finite.
 * lse_out     DEVICE fp32 [B,Hq,T] contiguous, or NULL.
 * workspace   DEVICE, 256-byte aligned, >= pkv_tree_workspace_bytes(desc) bytes
 *             (may be NULL when that is 0); contents irrelevant on entry,
 *             undefined on exit; concurrent calls need distinct ones.
 * Asynchronous on `stream`, never allocates.
 * Errors: PKV_ERR_INVALID_ARG (also a scale, a cap, or a quotient of theirs
 * that is not a finite fp32 in units of log2), PKV_ERR_UNSUPPORTED (d not
 * 64/128, T > 256, Hq/Hkv > 128, B or Hkv > 65535, B * Hq * T > 2^24 - 1,
 * k_cap or c_st > 2^30, a pool of more than 2^32 - 1 rows), PKV_ERR_WORKSPACE,
 * PKV_ERR_HIP.
 */
int pkv_tree_attention(const pkv_tree_desc* desc, const void* q,
                       const void* K_cache, const void* V_cache,
                       const int32_t* block_table, const int32_t* count,
                       const int32_t* new_lens, const int32_t* tree,
                       const int32_t* positions, const int32_t* q_pos,
                       const float* slopes, void* out, float* lse_out,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * pkv_decode_attention_long that also adds each row's softmax weight, summed
 * over the query heads of its KV head, to a running sum:
 *   weights[b][g][j] += sum_{h of g} softmax_j(s_h)   for every seen row j.
 * Nothing else of weights is written.  Same descriptor, results and errors
 * (PKV_ERR_UNSUPPORTED also B * Hq > 2^23, or B * Hkv * ceil(k_cap / 1024) >=
 * 2^31).
 * weights   DEVICE fp32 [B,Hkv,k_cap], 4-byte aligned, with element strides w_sb
 *           and w_sh >= 0, in either order.  Sums do not overlap: where there
 *           are several sequences or heads, the smaller stride is >= k_cap and
 *           the larger one reaches behind all that the smaller one spans.
 * workspace DEVICE, 256-byte aligned,
 *           >= pkv_decode_accumulate_workspace_bytes(desc) bytes (the scores,
 *           4 * B * Hq * k_cap bytes, beside what the attention alone takes: as
 *           much as the cache itself where d heads share a KV head); contents
 *           irrelevant on entry, undefined on exit; concurrent calls need
 *           distinct ones.
 * A weight is exact to a few 2^-24 of itself times its score's size, and the
 * same call gives the same bits.
 */
size_t pkv_decode_accumulate_workspace_bytes(const pkv_decode_long_desc* desc);

int pkv_decode_attention_accumulate(
    const pkv_decode_long_desc* desc, const void* q, const void* K_cache,
    const void* V_cache, const int32_t* block_table, const int32_t* count,
    const int32_t* positions, const int32_t* q_pos, const float* slopes,
    float* weights, int64_t w_sb, int64_t w_sh, void* out, float* lse_out,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Eviction by those sums, in place: of n_b = count_b rows (clamped to
 * 0..k_cap) of sequence b every KV head keeps min(n_b, budget).
 * A row is protected if its position is >= 0 and either below `first` or among
 * the last `recent` ones (> newest - recent, newest: the largest position of
 * the head's rows).  Protected rows are kept first, then those with the largest
 * weight; of equal weights (and of protected rows, should they be more than the
 * budget) the lower row is kept.  A weight that is NaN counts as less than any
 * other, and a row with a negative position as less than that.
 * Rows behind the budget that are kept take the places of rows before it that
 * are not: the i-th of the former moves to the i-th of the latter.  So a step
 * that drops one row moves one at most, and rows are no longer in the order of
 * their positions (no call here needs that).
 */
typedef struct {
  int32_t B, Hkv;     /* >= 1                                                */
  int32_t d;          /* 64 or 128                                           */
  int32_t k_cap;      /* rows per sequence the cache can hold                */
  int32_t page_size;  /* 0: compact cache; > 0: paged                        */
  int32_t num_pages;  /* paged: pages in the pool                            */
  int32_t max_pages;  /* paged: entries per sequence in the block table,
                         >= ceil(k_cap / page_size)                          */
  int32_t budget;     /* rows that stay, >= 1                                */
  int32_t recent;     /* >= 0                                                */
  int32_t first;      /* >= 0, first + recent <= budget                      */
  int64_t c_sb, c_sh, c_st; /* compact: element strides of the caches        */
  int64_t p_sb, p_sh;       /* of positions [B,Hkv,k_cap]                    */
  int64_t w_sb, w_sh;       /* of weights                                    */
  int64_t po_sb, po_sh;     /* of positions_out                              */
  int64_t wo_sb, wo_sh;     /* of weights_out                                */
} pkv_evict_desc;

/* Bytes of DEVICE workspace that pkv_cache_evict needs for this shape; 0 if
 * the descriptor is invalid.  HOST only, pure. */
size_t pkv_evict_workspace_bytes(const pkv_evict_desc* desc);

/*
 * desc        HOST.  What is written has places of its own: of po_*, of wo_*
 *             and of c_* the smallest stride is >= k_cap (c_*: d), and each
 *             larger one reaches behind all that the smaller ones span, where
 *             there are several sequences, heads or rows.
 * K_cache, V_cache
 *             DEVICE, rows of d 16-bit elements, 16-byte aligned, compact or
 *             pools; rows behind the budget keep their content.  Pages that
 *             two sequences (or places of a table) name are not for this call.
 * block_table DEVICE int32 [B,max_pages] contiguous (paged) or NULL.  A page
 *             number out of range: nothing is read or written through it, and
 *             the position of a row that would have been moved there, or from
 *             there, is -1 afterwards.
 * count       DEVICE int32 [B].
 * positions   DEVICE int32 [B,Hkv,k_cap].
 * weights     DEVICE fp32 [B,Hkv,k_cap].
 * positions_out, weights_out
 *             DEVICE, as positions and weights, and may be these themselves
 *             with the same strides: the kept rows' values, and -1 and 0 for
 *             rows min(n_b, budget) .. n_b - 1.  Rows >= n_b are left as they
 *             were.
 * count_out   DEVICE int32 [B] or NULL, written: min(n_b, budget).  Overlaps
 *             nothing.
 * workspace   DEVICE, 256-byte aligned, >= pkv_evict_workspace_bytes(desc)
 *             bytes; contents irrelevant on entry, undefined on exit;
 *             concurrent calls need distinct ones.
 * Asynchronous on `stream`, never allocates.
 * Errors: PKV_ERR_INVALID_ARG, PKV_ERR_UNSUPPORTED (d not 64/128, B or Hkv >
 * 65535, B * Hkv > 2^22 - 1, k_cap or c_st > 2^30, a pool of more than 2^32 - 1
 * rows), PKV_ERR_WORKSPACE, PKV_ERR_HIP.
 */
int pkv_cache_evict(const pkv_evict_desc* desc, void* K_cache, void* V_cache,
                    const int32_t* block_table, const int32_t* count,
                    const int32_t* positions, const float* weights,
                    int32_t* positions_out, float* weights_out,
                    int32_t* count_out, void* workspace,
                    size_t workspace_bytes, void* stream);

/*
 * Steps that attend over a part of a whole cache: its rows in blocks, of which
 * each KV head takes `most` by a bound on their scores.  Three calls: bounds of
 * new rows, selection, attention over the blocks.
 */
typedef struct {
  int32_t B, Hq, Hkv; /* Hq % Hkv == 0 (pkv_block_bounds: Hq is not used)    */
  int32_t d;          /* 64 or 128                                           */
  int32_t k_cap;      /* rows per sequence the cache can hold                */
  int32_t page_size;  /* 0: compact cache; > 0: paged                        */
  int32_t num_pages;  /* paged: pages in the pool                            */
  int32_t max_pages;  /* paged: entries per sequence in the block table,
                         >= ceil(k_cap / page_size)                          */
  int32_t dtype;      /* pkv_dtype                                           */
  int32_t block;      /* rows of a block: 16, 32, 64, 128 or 256             */
  int32_t most;       /* blocks of a head that are taken, >= 1               */
  int32_t first;      /* blocks at the beginning that are taken in any case  */
  int32_t recent;     /* and at the end; both >= 0, together <= most         */
  int32_t reserved;   /* must be 0                                           */
  float scale;        /* > 0; 0: 1/sqrt(d)                                   */
  float cap;          /* 0: none; > 0                                        */
  int64_t q_sb, q_sh;       /* element strides of q [B,Hq,d]                 */
  int64_t c_sb, c_sh, c_st; /* compact: of K_cache and V_cache
                               [B,Hkv,k_cap,d]                               */
  int64_t b_sb, b_sh;       /* of bounds
                               [B,Hkv,ceil(k_cap / block),2,d]               */
} pkv_block_desc;

/*
 * Least and greatest value of each channel of K over the rows of a block: of
 * those blocks that hold any of the last new_b rows, from all of their rows <
 * n_b = count_b (clamped to 0..k_cap).
 *   bounds[b][g][blk][0][i] = min_j K_ji, bounds[b][g][blk][1][i] = max_j K_ji
 * exactly.  A channel of a block in which some value is NaN: -inf and +inf.
 * Rows on pages that are out of range are left out; a block without rows is 0.
 * Nothing else of bounds is written.
 * desc        HOST.  B, Hkv, d, k_cap, pages, dtype, block, c_* and b_* are used.
 * K_cache     DEVICE, 16-byte aligned, compact or pool.
 * block_table DEVICE int32 [B,max_pages] contiguous (paged) or NULL.
 * count       DEVICE int32 [B].
 * new_lens    DEVICE int32 [B]: new_b, clamped to 0..n_b; NULL: n_b (all).
 * bounds      DEVICE, of the descriptor's type, 16-byte aligned; strides
 *             multiples of 8, the last three dimensions contiguous; those of
 *             two heads do not overlap.
 * Asynchronous on `stream`, needs no workspace, never allocates.
 * Errors: PKV_ERR_INVALID_ARG, PKV_ERR_UNSUPPORTED (d not 64/128, block none of
 * the above, B or Hkv > 65535, B * Hkv > 2^22 - 1, k_cap or c_st > 2^30, a pool
 * of more than 2^32 - 1 rows), PKV_ERR_HIP.
 */
int pkv_block_bounds(const pkv_block_desc* desc, const void* K_cache,
                     const int32_t* block_table, const int32_t* count,
                     const int32_t* new_lens, void* bounds, void* stream);

/*
 * The blocks a step takes.  The score of block blk of KV head g,
 *   sum_{h of g} sum_i q_hi bounds[..][q_hi < 0 ? 0 : 1][i],
 * bounds the sum of the heads' products with any of the block's keys from
 * above.  It is formed in 64 bits and rounded to fp32 once; one that is NaN
 * counts as +inf.  Of the ceil(n_b / block) blocks the first `first` and the
 * last `recent` are taken, then those with the largest scores (of equal ones
 * the lower block) until there are `most`.
 * desc       HOST.  B, Hq, Hkv, d, k_cap, dtype, block, most, first, recent, q_*
 *            and b_* are used (cap and scale do not change the order).
 * q          DEVICE, of the descriptor's type, 16-byte aligned.  Strides are
 *            multiples of 8.
 * bounds     DEVICE, as pkv_block_bounds writes them.
 * count      DEVICE int32 [B].
 * blocks_out DEVICE int32 [B,Hkv,most] contiguous, written: ascending, -1 behind.
 * scores_out DEVICE fp32 [B,Hkv,ceil(k_cap / block)] contiguous or NULL: the
 *            scores; written below ceil(n_b / block).
 * workspace  DEVICE, 256-byte aligned, >= pkv_block_select_workspace_bytes(desc)
 *            bytes; contents irrelevant on entry, undefined on exit; concurrent
 *            calls need distinct ones.
 * Asynchronous on `stream`, never allocates.
 * Errors: as pkv_block_bounds, PKV_ERR_UNSUPPORTED also Hq/Hkv > 128 or most >
 * 2^30, PKV_ERR_WORKSPACE.
 */
size_t pkv_block_select_workspace_bytes(const pkv_block_desc* desc);

int pkv_block_select(const pkv_block_desc* desc, const void* q,
                     const void* bounds, const int32_t* count,
                     int32_t* blocks_out, float* scores_out, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * pkv_decode_attention_long over the rows of the listed blocks alone, without
 * positions, window and slopes.  Of a list the first min(most, ceil(n_b /
 * block)) entries are looked at; one outside 0 .. ceil(n_b / block) - 1 has no
 * rows, and one that is named twice counts twice.
 * desc        HOST.  first, recent and b_* are not used.
 * blocks      DEVICE int32 [B,Hkv,most] contiguous, in any order.
 * Everything else, and the errors, as pkv_decode_attention_long; most * block >
 * 2^30 -> PKV_ERR_UNSUPPORTED.
 */
size_t pkv_decode_blocks_workspace_bytes(const pkv_block_desc* desc);

int pkv_decode_attention_blocks(const pkv_block_desc* desc, const void* q,
                                const void* K_cache, const void* V_cache,
                                const int32_t* block_table,
                                const int32_t* count, const int32_t* blocks,
                                void* out, float* lse_out, void* workspace,
                                size_t workspace_bytes, void* stream);

/* Static, NUL-terminated description of a pkv_status value.  HOST only. */
const char* pkv_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* PKV_H_ */
