/*
 * dopr.h -- C ABI of the GB300-native DoPR online scoring library (libdopr.so).
 *
 * DoPR (Sec. 3.1 "Problem Formulation", Sec. 3.3 "Offline Compression",
 * Sec. 3.4 "Online Reranking") stores, for every document d, the multi-layer
 * key/value states C~_d of K_infer = m compressed prefix positions.  Online,
 * a pair (q, d) is scored by running the decoder over [q ; t_score] only,
 * each layer attending to d's stored prefix keys/values before the causal
 * online keys, and reading the score at t_score.  This library implements
 * that online pass on one GPU: a device-resident prefix store, a batch
 * packer that groups pairs by document, and the decoder kernels.
 *
 * Conventions for every entry point:
 *   - Plain C types only.  bf16 tensors are passed as `const void*` to
 *     16-bit bit patterns (IEEE bfloat16).  Matrices are row-major.
 *   - Inputs are borrowed for the duration of the call; the library copies
 *     what it keeps.  Outputs go to caller-owned buffers.  Library objects
 *     are opaque and released by the matching *_destroy.
 *   - Every argument is validated before any device work is launched; on an
 *     error nothing is written to caller buffers and the object is left as
 *     it was.  The status says what went wrong; dopr_last_error() returns a
 *     thread-local message for the last failing call on this thread.
 *   - Device work runs on the device that is current when the object is
 *     created; use the same device for all calls on that object.
 *   - Objects are not thread-safe: serialise calls on one object.
 */
#ifndef DOPR_H
#define DOPR_H

#include <stdint.h>

#if defined(__GNUC__)
#define DOPR_API __attribute__((visibility("default")))
#else
#define DOPR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DOPR_OK = 0,
    DOPR_ERR_INVALID_ARG = 1,   /* bad pointer, size, index or shape          */
    DOPR_ERR_UNKNOWN_DOC = 2,   /* a doc_id has no stored prefix              */
    DOPR_ERR_INCOMPLETE = 3,    /* a weight or a doc layer was never supplied */
    DOPR_ERR_OUT_OF_MEMORY = 4, /* device allocation or the store pool full   */
    DOPR_ERR_CUDA = 5,          /* a CUDA runtime/driver call failed          */
    DOPR_ERR_TIMEOUT = 6,       /* a bounded device wait ran out; the result
                                   of that call is invalid, the context is not */
    DOPR_ERR_UNSUPPORTED = 7,   /* a shape this build does not handle         */
    DOPR_ERR_INTERNAL = 8,      /* a checked build (DOPR_CHECKED) met an index
                                   outside its buffer and skipped the access:
                                   a library defect; the call's outputs are
                                   invalid, the context is not               */
    DOPR_ERR_RANGE = 9          /* a value the tensor cores take as an fp16
                                   operand (normed activations, q/k/v, the
                                   SwiGLU output, the attention output) or a
                                   score was not finite or exceeded 65504 in
                                   magnitude: the inputs leave the range the
                                   fp16 path computes on; the call's outputs
                                   are invalid, the context is not           */
} dopr_status;

/*
 * Decoder shape (Qwen3 family, the paper's backbone, Sec. 4.1).
 * Supported: head_dim == 128; n_q_heads % n_kv_heads == 0;
 * hidden % 256 == 0; ffn % 128 == 0; (n_q_heads + 2 n_kv_heads) * 128 % 256 == 0.
 * score_token_id is t_score (Sec. 3.1), appended by the library to every
 * query.  Positions m + j of online tokens must be < max_position.
 */
typedef struct {
    int32_t n_layers;
    int32_t hidden;
    int32_t n_q_heads;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t ffn;
    int32_t vocab;
    int32_t score_token_id;
    int32_t max_position;
    float rope_theta;   /* RoPE base, rotate-half pairs (i, i + head_dim/2) */
    float rms_eps;      /* RMSNorm epsilon                                  */
} dopr_model_config;

typedef struct dopr_model dopr_model;
typedef struct dopr_store dopr_store;

/* Weight kinds for dopr_model_put_weight; shapes are [rows][cols] bf16. */
typedef enum {
    DOPR_W_EMBED = 0,      /* [vocab][hidden]             (layer ignored) */
    DOPR_W_ATTN_NORM = 1,  /* [hidden]      input RMSNorm gain            */
    DOPR_W_Q = 2,          /* [n_q_heads*128][hidden]                     */
    DOPR_W_K = 3,          /* [n_kv_heads*128][hidden]                    */
    DOPR_W_V = 4,          /* [n_kv_heads*128][hidden]                    */
    DOPR_W_Q_NORM = 5,     /* [128]         per-head RMSNorm gain on q    */
    DOPR_W_K_NORM = 6,     /* [128]         per-head RMSNorm gain on k    */
    DOPR_W_O = 7,          /* [hidden][n_q_heads*128]                     */
    DOPR_W_MLP_NORM = 8,   /* [hidden]      post-attention RMSNorm gain   */
    DOPR_W_GATE = 9,       /* [ffn][hidden]                               */
    DOPR_W_UP = 10,        /* [ffn][hidden]                               */
    DOPR_W_DOWN = 11,      /* [hidden][ffn]                               */
    DOPR_W_FINAL_NORM = 12,/* [hidden]                    (layer ignored) */
    DOPR_W_SCORE_HEAD = 13 /* [2][hidden]: row 0 "yes", row 1 "no"
                              (layer ignored)                             */
} dopr_weight_kind;

/* Create a model: allocates device memory for all weights of `cfg` (left
 * unset until put).  *out receives the handle.  Errors: INVALID_ARG,
 * UNSUPPORTED, OUT_OF_MEMORY, CUDA. */
DOPR_API dopr_status dopr_model_create(const dopr_model_config *cfg, dopr_model **out);

/* Copy one weight tensor into the model (converted to the library's own
 * device layout).  `src` holds n_elems bf16 values in the layout listed
 * under dopr_weight_kind; src_on_device != 0 means `src` is a device
 * pointer.  Re-putting a weight replaces it.  Synchronous.  The
 * projection matrices (Q, K, V, O, gate, up, down) are held as fp16 for
 * the tensor cores: a value that is not finite or exceeds 65504 in
 * magnitude fails the put (the weight is then left as it was).
 * Errors: INVALID_ARG (kind, layer or n_elems wrong; a projection value
 * outside fp16's range), CUDA. */
DOPR_API dopr_status dopr_model_put_weight(dopr_model *model, int32_t kind, int32_t layer, const void *src,
                                  int64_t n_elems, int32_t src_on_device);

/*
 * Replace the yes/no score rows by the paper's lightweight MLP head on the
 * score token's state (Sec. 3.2.3, s = MLP(h_score); its shape is not given):
 * one hidden layer of `width` units over hn = RMSNorm(h) * final_norm,
 *   s = sum_j w2[j] * act(W1[j] . hn + b1[j]) + b2,
 * W1 bf16 [width][hidden], b1 and w2 bf16 [width]; activation 0 ReLU,
 * 1 GELU (erf form), 2 SiLU, 3 tanh.  src_on_device != 0: device pointers.
 * width == 0 restores the yes/no rows.  Synchronous.
 * Errors: INVALID_ARG, OUT_OF_MEMORY, CUDA.
 */
DOPR_API dopr_status dopr_model_set_mlp_head(dopr_model *model, int32_t width, int32_t activation, const void *w1,
                                            const void *b1, const void *w2, float b2, int32_t src_on_device);

/* Release a model and its device memory.  NULL is accepted. */
DOPR_API dopr_status dopr_model_destroy(dopr_model *model);

/*
 * Prefix store (Sec. 3.3: the offline store of C~_d; Sec. 3.4: fetched per
 * candidate).  Holds doc ids 0..max_doc_id in a device pool of pool_bytes
 * bytes; each document takes dopr_prefix_bytes(cfg, m) bytes of it.
 * Errors: INVALID_ARG, UNSUPPORTED, OUT_OF_MEMORY, CUDA.
 */
DOPR_API dopr_status dopr_store_create(const dopr_model_config *cfg, int64_t max_doc_id, int64_t pool_bytes,
                              dopr_store **out);

/*
 * Store one layer of a document's compressed prefix states (Sec. 3.4 and
 * its footnote: the multi-layer K/V obtained by forwarding the selected
 * representations as prefix inputs).
 *   k, v: bf16 [m][n_kv_heads][head_dim].  k is the key after the per-head
 *         RMSNorm and after RoPE at positions 0..m-1; v is the raw value.
 *   0 <= m <= 256 (the largest K_infer of the paper's settings, Tab. 8);
 *   m == 0 stores an empty prefix (the pass then equals a query-only forward).
 * The first put of a doc reserves its block; later puts must give the same
 * m (a different m is INVALID_ARG) and replace that layer.  A doc can be
 * scored once all n_layers layers were put.  The store keeps the values as
 * fp16 (exact for bf16 values in fp16's normal range); a value that is not
 * finite or exceeds 65504 in magnitude fails the put with INVALID_ARG and
 * leaves that layer marked missing.  Synchronous.
 * Errors: INVALID_ARG, OUT_OF_MEMORY (pool full), CUDA.
 */
DOPR_API dopr_status dopr_store_put(dopr_store *store, int64_t doc_id, int32_t m, int32_t layer, const void *k,
                           const void *v, int32_t src_on_device);

/* Release a store.  NULL is accepted. */
DOPR_API dopr_status dopr_store_destroy(dopr_store *store);

/*
 * Offline prefix construction (Sec. 3.3; Sec. 3.4's footnote): for each
 * document d, forward its selected representations c_1..c_m (the compressed
 * document inputs C~_d is built from) causally through the model as prefix
 * inputs at positions 0..m-1, and store every layer's key (after the q/k
 * norm and RoPE) and value as the document's prefix states -- the states
 * dopr_store_put would be given.  The last layer stops after its key/value
 * projection.
 *   doc_ids   [n_docs] int64, host; distinct, each in [0, max_doc_id].
 *   x_offsets [n_docs+1] int32, host: document d's representations are rows
 *             x_offsets[d] .. x_offsets[d+1]-1 of x; x_offsets[0] == 0,
 *             0 <= m_d <= 256 and m_d <= max_position.
 *   x         bf16 [x_offsets[n_docs]][hidden]; a device pointer when
 *             x_on_device != 0, else host memory (copied in by the call).
 *   cuda_stream: a cudaStream_t, or NULL for the default stream.
 * Documents are reserved (or must match an earlier reservation's m) before
 * any kernel runs; on success every layer of every document is present.
 * Synchronous.  Errors: INVALID_ARG, INCOMPLETE (model weights missing),
 * OUT_OF_MEMORY (pool full), CUDA, TIMEOUT.
 */
DOPR_API dopr_status dopr_build_prefixes(dopr_model *model, dopr_store *store, int32_t n_docs, const int64_t *doc_ids,
                                         const int32_t *x_offsets, const void *x, int32_t x_on_device,
                                         void *cuda_stream);

/*
 * Attention-based key token selection (Sec. 3.2.1), as the offline
 * construction of Sec. 3.3 applies it: encode each document alone (its
 * token ids at positions 0..n-1; no prefix, no score token), average the
 * last layer's attention weights over the q heads into A[n][n] (row =
 * attending token, causal), score token i by the mean of the top_p largest
 * entries of column i (of its min(top_p, n - i) causal entries), keep the
 * top_k most salient positions (equal salience to the lower position) and
 * return them in ascending order with their final-layer states after the
 * final RMSNorm -- the representations dopr_build_prefixes takes.  The paper
 * leaves p open; top_p >= n gives the column mean.
 *   doc_offsets [n_docs+1] int32, host: document d is doc_tokens[off[d] .. off[d+1]);
 *               off[0] == 0, 1 <= n_d <= 2048 and n_d <= max_position.
 *   doc_tokens  int32 token ids in [0, vocab), host.
 *   1 <= top_k <= 256, top_p >= 1.
 *   positions   [n_docs][top_k] int32, host: ascending, -1 past min(top_k, n_d).
 *   x_out       [n_docs][top_k][hidden] bf16, host: the states at `positions`
 *               (zero rows for -1).
 *   salience    [off[n_docs]] float, host, or NULL: u of every token.
 * Device memory of n^2 floats per document of a chunk is allocated for the
 * call.  Synchronous.  Errors: INVALID_ARG, INCOMPLETE (model weights
 * missing), OUT_OF_MEMORY, CUDA, TIMEOUT.
 */
DOPR_API dopr_status dopr_select_prefix_inputs(dopr_model *model, int32_t n_docs, const int32_t *doc_offsets,
                                               const int32_t *doc_tokens, int32_t top_k, int32_t top_p,
                                               int32_t *positions, void *x_out, float *salience, void *cuda_stream);

/*
 * A stored layer of one document, read back for testing: k_out and v_out
 * (host, fp16 bits [m][n_kv_heads][head_dim], the dopr_store_put layout).
 * A document with m == 0 writes nothing.  Synchronous.
 * Errors: INVALID_ARG, UNKNOWN_DOC (never stored), CUDA.
 */
DOPR_API dopr_status dopr_debug_store_read(const dopr_store *store, int64_t doc_id, int32_t layer, void *k_out,
                                           void *v_out);

/* Bytes of stored prefix state for one document of m prefix positions:
 * m * n_layers * 2 (K,V) * n_kv_heads * head_dim * 2 bytes.  This is the
 * document-side memory figure of Tab. 3 / Tab. 9.  Returns -1 on a bad cfg. */
DOPR_API int64_t dopr_prefix_bytes(const dopr_model_config *cfg, int32_t m);

/*
 * Score a batch of (query, document) pairs (Sec. 3.4).
 *   q_offsets [n_pairs+1] int32: query p is q_tokens[q_offsets[p] .. q_offsets[p+1]);
 *             q_offsets[0] == 0, non-decreasing; empty queries are allowed
 *             (the pair is then scored on the score token alone).
 *   q_tokens  int32 token ids in [0, vocab).
 *   doc_ids   [n_pairs] int64, each with a complete prefix in `store`.
 *   scores    [n_pairs] float, written in input order: the "yes" minus
 *             "no" logit at the score token.
 *   cuda_stream: a cudaStream_t, or NULL for the default stream.
 *   io_on_device: 0 = the four arrays are host memory (copied in and out by
 *             the call); 1 = device memory (read and written in place).
 * Arithmetic: the tensor-core operands (activations, projection weights,
 * q/k/v, attention probabilities) are fp16 -- the bf16 inputs widen to fp16
 * exactly in its normal range -- with fp32 accumulation, an fp32 residual
 * stream and fp32 norms, softmax and score head.
 * The call is synchronous in both modes: it synchronises `cuda_stream`
 * once after packing (to size the launches) and once after the last
 * kernel, reads the device error word, and only when it is clear copies
 * the scores into `scores` (a third synchronisation): a call that fails,
 * on the host or on the device, writes nothing.  Pairs of one doc_id are
 * grouped so that their prefix is staged once per group; scores do not
 * depend on batch order.  With io_on_device = 1 the inputs are validated
 * on the device and an invalid batch returns its error before any decoder
 * kernel runs.
 * Valid range: every fp16 operand must stay within +-65504 (the bf16
 * inputs are checked at put time; intermediates are checked as they are
 * written, see DOPR_ERR_RANGE).
 * Errors: INVALID_ARG, UNKNOWN_DOC, INCOMPLETE, OUT_OF_MEMORY, CUDA, TIMEOUT,
 * RANGE, INTERNAL (checked builds).
 */
DOPR_API dopr_status dopr_score(dopr_model *model, dopr_store *store, int32_t n_pairs, const int32_t *q_offsets,
                       const int32_t *q_tokens, const int64_t *doc_ids, float *scores, void *cuda_stream,
                       int32_t io_on_device);

/*
 * The packing plan dopr_score uses (its device packer), copied to host
 * arrays, for testing.  Inputs as in dopr_score (host memory).  Outputs,
 * all host int32:
 *   perm     [n_pairs]    input index of the pair in sorted position s;
 *                         pairs are ordered by (doc_id, input index)
 *   tok_off  [n_pairs+1]  first packed token of sorted pair s
 *   tok_pos  [T]          RoPE position of packed token t (m_doc + j)
 *   tok_id   [T]          token id of packed token t (score token last)
 *   tok_pair [T]          sorted pair index of packed token t
 * with T = q_offsets[n_pairs] - q_offsets[0] + n_pairs.
 * Errors: as dopr_score.
 */
DOPR_API dopr_status dopr_debug_pack_plan(dopr_model *model, dopr_store *store, int32_t n_pairs, const int32_t *q_offsets,
                                 const int32_t *q_tokens, const int64_t *doc_ids, int32_t *perm, int32_t *tok_off,
                                 int32_t *tok_pos, int32_t *tok_id, int32_t *tok_pair);

/*
 * The attention tile plan of one document's run of pairs, computed on the
 * host exactly as dopr_score plans it (no device work: usable without a GPU),
 * for testing the tiling rule of the prefix-plus-causal attention (Sec. 3.4).
 *   m              the document's prefix length (keys), >= 0;
 *   rows_per_tile  tokens per tile (128 / G for G q heads per kv head), 1..128;
 *   n_pairs        pairs of the run, >= 1; tok_len [n_pairs] int32 >= 1: the
 *                  packed tokens (query + score token) of each pair, laid out
 *                  consecutively in this order;
 *   out            [max_tiles][24] int32, caller-owned; tile t, in token order:
 *                  {kind (0 = tensor-core tile of at most 256 key columns, 1 =
 *                  long tile), tok_begin, n_tok, n_keys, n_seg, 0, 0, 0,
 *                  seg[0..15]}, seg[s] = (visible tokens << 16) | (uint16_t)
 *                  (first token of the pair - tok_begin), one per pair the tile
 *                  touches, in pair order.
 * Returns the number of tiles (>= 1), or -DOPR_ERR_INVALID_ARG for bad
 * arguments or when max_tiles is too small (nothing is written then).
 */
DOPR_API int32_t dopr_debug_attention_plan(int32_t m, int32_t rows_per_tile, int32_t n_pairs, const int32_t *tok_len,
                                           int32_t max_tiles, int32_t *out);

/*
 * The dense projection kernel alone, for testing: C = A * B^T with A fp16
 * [M][K], B fp16 [N][K] (IEEE half, device pointers), fp32 accumulation.
 *   epilogue 0: out fp16 [M][N] = C
 *   epilogue 1: out fp32 [M][N] += C            (residual add)
 *   epilogue 2: out fp16 [M][N/2] = silu(G) * U, where B's rows come in
 *               blocks of 256: rows 256b..256b+127 are gate rows 128b.., rows
 *               256b+128..256b+255 the matching up rows (SwiGLU, Sec. 4.1 backbone)
 * Requires K % 64 == 0 and N % 256 == 0.  Runs on cuda_stream (NULL = default)
 * and returns after completion.  Errors: INVALID_ARG, UNSUPPORTED, CUDA, TIMEOUT.
 */
DOPR_API dopr_status dopr_debug_gemm(int32_t M, int32_t N, int32_t K, const void *A, const void *B, void *out,
                            int32_t epilogue, void *cuda_stream);

/*
 * The launch or launches a projection of M rows takes on num_sms SMs (host
 * arithmetic only: usable without a GPU), for testing.  epilogue as in
 * dopr_debug_gemm, or 3 for the QKV projection.
 *   out [4] int32: {1 when few-row tiles take every row, rows per CTA of the
 *       pair, columns, W}; W > 0: the first W rows in wide tiles, the others
 *       in few-row tiles of that size by a launch beside.
 * Errors: INVALID_ARG, UNSUPPORTED (K % 64, N % 256).
 */
DOPR_API dopr_status dopr_debug_gemm_plan(int32_t epilogue, int32_t M, int32_t N, int32_t K, int32_t num_sms,
                                          int32_t *out);

/*
 * Runs one test kernel whose bounded waits, one on a barrier that nothing
 * completes and one at a gate that nothing opens, must give up after about
 * timeout_ms milliseconds.  Returns DOPR_ERR_TIMEOUT when the kernel reported
 * both waits as expired (the expected result), DOPR_OK if it did not.  Used to check the timeout path of the
 * device waits without hanging the GPU.
 */
DOPR_API dopr_status dopr_debug_wait_timeout(int32_t timeout_ms);

/*
 * Allocation-free packing (the paper has no counterpart; this is a service
 * entry point of this library).  For callers that cannot allocate device
 * memory while they score -- their GPU memory is owned by another allocator
 * (e.g. a framework's caching pool), or cudaMalloc/cudaFree would stall a
 * latency-critical loop by synchronising the device -- this runs the same
 * device packer ordering step as dopr_score (pairs ordered by (doc_id, input
 * index), packed token offsets) using only caller buffers and a fixed scratch
 * array compiled into the library.  It calls no cudaMalloc/cudaFree.
 *   q_offsets [n_pairs+1] int32, doc_ids [n_pairs] int64: DEVICE memory,
 *             same meaning as in dopr_score.
 *   perm      [n_pairs] int32 DEVICE output: input index of sorted pair s.
 *   tok_off   [n_pairs+1] int32 DEVICE output: first packed token of sorted
 *             pair s (query tokens + the score token per pair).
 * Validation is dopr_score's: unknown or incomplete documents, decreasing
 * offsets and m + query length + 1 > max_position (the store's, which
 * dopr_score requires to equal the model's) fail the call.  The C ABI carries
 * no buffer sizes: the caller guarantees the extents above.
 * Limits: n_pairs <= 32768 and store max_doc_id < 131072; larger requests
 * return DOPR_ERR_UNSUPPORTED with a message and launch nothing.  The scratch
 * array (about 256 KiB) is held by every GPU that loads the library until the
 * process exits.  The first call on a device looks the array's device address
 * up (cudaGetSymbolAddress) with that device current; make that first call
 * before any stream capture.  Every call shares the one array: calls that
 * overlap on the GPU (on different streams) race and must be serialised by
 * the caller; host threads may call on one stream, each call returns its own
 * status.  The call runs on cuda_stream (NULL = default)
 * and returns after its results are written (it synchronises the stream).
 * Errors: INVALID_ARG, UNKNOWN_DOC, INCOMPLETE, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_pack_order_noalloc(const dopr_store *store, int32_t n_pairs, const int32_t *q_offsets,
                                             const int64_t *doc_ids, int32_t *perm, int32_t *tok_off,
                                             void *cuda_stream);

/*
 * Paged prefix cache: operators for prefixes of any length (whole documents,
 * prefixes that grow) beside the store of compressed ones above (the paper has
 * no counterpart; Sec. 3.4's prefix-plus-causal attention is the same).  All
 * memory is the caller's, on the device that is current: one layer's keys and
 * values lie in two pools of pages, and a sequence (a table row) is a list of
 * pages.  A sequence may name a prefix sequence; any number may name the same.
 * A step of a program is
 *   dopr_cache_extend           pages, slots, positions for the new tokens
 *   dopr_shared_attention_plan  how the step's attention is split
 *   per layer: dopr_cache_append (rotary positions, keys and values into the
 *   pages) and dopr_shared_attention.
 * Unlike the calls above these return once their work is on cuda_stream: they
 * neither allocate, nor synchronise, nor read device memory on the host, and
 * can be captured into a graph.  Calls that share buffers (a cache, a plan, a
 * workspace) are ordered by the caller, as its own kernels would be.
 * Arguments on the host are checked before any launch.  What lies on the
 * device is checked there: nothing outside the stated extents is read or
 * written, and an error is stored in *status, a device int32 (NULL: dropped),
 * as a dopr_status, if *status is DOPR_OK; the caller clears it.  A call on no
 * rows (n_tokens or max_tokens 0) may pass NULL for the rows' buffers.
 */
typedef enum { DOPR_F16 = 0, DOPR_BF16 = 1, DOPR_F32 = 2 } dopr_dtype;

/*
 * k_pool, v_pool: [n_blocks][n_kv_heads][page][head_dim] of dtype, 16-byte
 * aligned.  block_tables: int32 [n_seqs][max_blocks]; entry p of a row is the
 * page of its positions p*page .. p*page + page - 1.
 * Supported: page 16, 32, 64 or 128; head_dim 64 or 128; dtype F16 or BF16;
 * n_seqs <= 16384; max_blocks * page < 2^31;
 * n_blocks * n_kv_heads * page < 2^31.
 */
typedef struct {
    int32_t n_blocks;
    int32_t page;
    int32_t n_kv_heads;
    int32_t head_dim;
    int32_t dtype;
    int32_t n_seqs;
    int32_t max_blocks;
} dopr_cache_layout;

/*
 * Block tables and slots of a step's new tokens, from lengths on the device.
 * Row i holds seq_lens[i] tokens and gets new_lens[i] >= 0 more; new_lens[i]
 * == -1 releases it (its pages return to the stack, its length becomes 0).
 *   seq_lens, new_lens [n_seqs] int32, prefix [n_seqs] int32 or NULL: the row
 *             that precedes row i's own tokens, -1 for none.  A row that is
 *             named as a prefix names none itself.
 *   free_blocks int32 [n_blocks], n_free [1] int32: a stack of unused pages,
 *             the top at n_free - 1.  Released pages are pushed first, row by
 *             row in page order; then rows in order take pages from the top,
 *             which become their next table entries.
 *   seq_lens_out [n_seqs], n_free_out [1]: lengths and stack height after the
 *             call; each may be the input itself.
 *   max_tokens extent of slots and positions; >= the new tokens in all.
 *   tok_off   [n_seqs+1] int32: row i's new tokens are tok_off[i] .. tok_off[i+1]-1.
 *   slots     [max_tokens] int64: page * layout->page + place of token t; -1
 *             behind the last token.
 *   positions [max_tokens] int32: length of the prefix row after the call +
 *             place in the row; -1 behind the last token.
 *   workspace dopr_cache_extend_workspace(layout) bytes, 16-byte aligned.
 * Device errors, which leave lengths, stack and tables as they were and give
 * no token a slot (tok_off all 0): INVALID_ARG (a length, new length or prefix
 * out of range, more than max_tokens new tokens, a position beyond 2^31 - 1),
 * OUT_OF_MEMORY (not enough free pages).  A page number outside the pool on
 * the stack or in a table is INVALID_ARG too: its tokens get slot -1, and that of
 * a released row goes onto the stack as it is.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_cache_extend(const dopr_cache_layout *layout, const int32_t *seq_lens, int32_t *block_tables,
                                       int32_t *free_blocks, const int32_t *n_free, const int32_t *prefix,
                                       const int32_t *new_lens, int32_t max_tokens, int32_t *seq_lens_out,
                                       int32_t *n_free_out, int32_t *tok_off, int64_t *slots, int32_t *positions,
                                       void *workspace, int32_t *status, void *cuda_stream);
/* Bytes of its workspace; -1 on a bad layout. */
DOPR_API int64_t dopr_cache_extend_workspace(const dopr_cache_layout *layout);

/* Rotary positions (RoPE): element pairs (x_a, x_b) of a head become
 *   (x_a cos - x_b sin, x_b cos + x_a sin), angle = position * f_i,
 * over the first rotary_dim = d elements; the others pass unchanged.
 * HALF pairs (i, i + d/2), INTERLEAVED pairs (2i, 2i + 1), i < d/2.
 * Frequencies, f_i = theta^(-2i/d) where PLAIN:
 *   LINEAR  f_i / factor;
 *   NTK     base theta * factor^(d / (d-2));
 *   BANDS   with turns n_i = original_max_position f_i / 2pi: f_i where n_i >= high,
 *           f_i / factor where n_i <= low, blended linearly in n_i between;
 *   RAMP    (YaRN, arXiv 2309.00071) f_i (1 - r_i) + f_i / factor r_i, r_i rising
 *           linearly from 0 to 1 between the indices floor(c(high)) and
 *           ceil(c(low)), c(n) = d ln(original_max_position / 2pi n) / (2 ln theta),
 *           kept within [0, d-1]; cos and sin times attention_factor (0: 0.1 ln(factor) + 1).
 */
typedef enum { DOPR_ROPE_HALF = 0, DOPR_ROPE_INTERLEAVED = 1 } dopr_rope_layout;
typedef enum {
    DOPR_ROPE_PLAIN = 0, DOPR_ROPE_LINEAR = 1, DOPR_ROPE_NTK = 2, DOPR_ROPE_BANDS = 3, DOPR_ROPE_RAMP = 4
} dopr_rope_scaling;
typedef struct {
    int32_t max_position;  /* positions 0 .. max_position - 1; at most 2^22      */
    int32_t rotary_dim;    /* even, 2 .. 256 (NTK: at least 4)                   */
    int32_t layout;
    int32_t scaling;
    double theta;          /* > 1                                                */
    double factor;         /* >= 1 (PLAIN: not used)                             */
    int32_t original_max_position;  /* BANDS, RAMP: > 0                          */
    double low, high;      /* BANDS, RAMP: turns, 0 < low < high                 */
    double attention_factor;        /* RAMP: >= 0                                */
} dopr_rope_config;
typedef struct dopr_rope dopr_rope;

/* The table of cos and sin (angles and functions in 64 bits, entries rounded
 * to 32) on the current device: 4 * rotary_dim * max_position bytes.
 * Synchronous.  Errors: INVALID_ARG, UNSUPPORTED, OUT_OF_MEMORY, CUDA. */
DOPR_API dopr_status dopr_rope_create(const dopr_rope_config *cfg, dopr_rope **out);
/* NULL is accepted.  No call that uses it may be pending. */
DOPR_API dopr_status dopr_rope_destroy(dopr_rope *rope);

/* A [tokens][n_heads][head_dim] view: strides in elements, head_dim contiguous.
 * Inputs may repeat a row for all tokens (token_stride 0); of an output all of a
 * token's heads, or all of a head's tokens, lie before those of the next. */
typedef struct {
    void *data;
    int64_t token_stride;
    int64_t head_stride;
    int32_t n_heads;
} dopr_heads;

/*
 * q_out = rotated q, k_out = rotated k (k, k_out NULL: q alone), of dtype F16,
 * BF16 or F32, computed in 32 bits and rounded once.  An output may be its
 * input; otherwise outputs overlap nothing.  inverse != 0 turns back (angle
 * -position f_i, the same attention_factor): the gradient of the rotation,
 * from that of its output.  Rows with positions[t] < 0 are left as they were.
 * head_dim even, rotary_dim <= head_dim <= 256.  Aligned views (data and
 * strides multiples of 16 bytes) are faster.
 * Device error: INVALID_ARG (a position >= max_position; its row is left).
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_rope_apply(const dopr_rope *rope, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                                     const int32_t *positions, const dopr_heads *q, const dopr_heads *q_out,
                                     const dopr_heads *k, const dopr_heads *k_out, int32_t inverse, int32_t *status,
                                     void *cuda_stream);

/*
 * One layer's new rows: k (rotated) and v into the pages at slots[t], and
 * q_out = rotated q (q, q_out NULL: keys and values alone).  rope NULL: k is
 * stored as it is, positions is not read, and q must be NULL.  Rows with
 * slots[t] < 0 are not stored; with positions[t] < 0 nothing of a row is
 * written.  Slots are distinct.  Device error: INVALID_ARG (a slot outside the
 * pool, a position >= max_position; that row is left).
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_cache_append(const dopr_cache_layout *layout, const dopr_rope *rope, int32_t n_tokens,
                                       const int32_t *positions, const int64_t *slots, const dopr_heads *q,
                                       const dopr_heads *q_out, const dopr_heads *k, const dopr_heads *v, void *k_pool,
                                       void *v_pool, int32_t *status, void *cuda_stream);

/*
 * How the attention of a step's tokens is split over the device: made once a
 * step, used by every layer.  tok_off, seq_lens (after dopr_cache_extend) and
 * prefix as there; tokens tok_off[n_seqs] .. max_tokens - 1 are behind the last.
 *   plan  dopr_shared_attention_plan_bytes(...) bytes, 16-byte aligned.  It serves
 *         attention with the same layout, n_q_heads and max_tokens on the same
 *         kind of device; with others that is INVALID_ARG and writes nothing.
 * 1 <= n_q_heads / n_kv_heads <= 64, a whole number.
 * Device errors: INVALID_ARG (offsets, a length or a prefix out of range),
 * UNSUPPORTED (2^29 units of work or more: for every kv head and group of up to
 * 256 rows that share keys, 6 a block of 128 keys that all of them see and 12
 * another; where 16 rows or fewer share them, 1 for every 16 keys.  90,000 tokens
 * of 32 heads on 8 over 2^20 keys are that many; or keys of such a group, its
 * rows' own together, beyond 2^31 - 129); the plan is then empty, and attention
 * writes nothing.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_shared_attention_plan(const dopr_cache_layout *layout, int32_t n_q_heads, int32_t max_tokens,
                                                const int32_t *tok_off, const int32_t *seq_lens, const int32_t *prefix,
                                                void *plan, int32_t *status, void *cuda_stream);
DOPR_API int64_t dopr_shared_attention_plan_bytes(const dopr_cache_layout *layout, int32_t n_q_heads,
                                                  int32_t max_tokens);

/*
 * out = softmax(scale q k^T) v for every token of the plan: token j of row i's
 * n_i tokens sees all seq_lens[prefix[i]] keys of the prefix and the row's own
 * keys 0 .. seq_lens[i] - n_i + j.  Rows that share a prefix read its pages
 * together, whatever their order; long keys are split and joined.  q head h
 * reads kv head h / (n_q_heads / n_kv_heads).
 *   plan     dopr_shared_attention_plan_bytes(...) bytes, of this call's sizes.
 *   q, out   views of layout->dtype, 16-byte aligned with strides multiples of
 *            16 bytes; out overlaps nothing.  Rows behind the last token are
 *            left as they were.
 *   lse      [max_tokens][n_q_heads] float or NULL: log of the sum of exponentials
 *            (natural).  A row that sees no key gives zeros and -infinity.
 *   workspace dopr_shared_attention_workspace(...) bytes, 32-byte aligned.
 * Keys and values past a row's end are never used, whatever the pages hold there.
 * Products take dtype operands with 32-bit sums; probabilities are rounded to
 * dtype (F16: those below 2^-25 of a row's largest to steps of 2^-35 of it),
 * statistics and sums are 32-bit.  A row's bits depend on the plan.
 * Device errors: INVALID_ARG (a page number outside the pool: page 0 is read
 * for it), TIMEOUT.  Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_shared_attention(const dopr_cache_layout *layout, const void *plan, int32_t max_tokens,
                                           const dopr_heads *q, const void *k_pool, const void *v_pool,
                                           const int32_t *block_tables, float scale, const dopr_heads *out, float *lse,
                                           void *workspace, int32_t *status, void *cuda_stream);
DOPR_API int64_t dopr_shared_attention_workspace(const dopr_cache_layout *layout, int32_t n_q_heads,
                                                 int32_t max_tokens);

/*
 * RMSNorm of each query and key head, and rotary positions, in one pass (Sec. 4.1's backbone norms q and k so):
 *   y_i = x_i g_i / sqrt(mean of x^2 over the head + eps), then dopr_rope_apply's turn of y.
 * Arguments as there; rope NULL: no turn, positions is not read.  eps > 0.  Gains [head_dim] of gain_dtype, one for all
 * heads of q, one for k; NULL: ones.  k, k_out NULL: q alone.  Computed in 32 bits, rounded once.  An output may be its input;
 * otherwise outputs overlap nothing.  Rows with positions[t] < 0 are left as they were.  Device error: INVALID_ARG (a
 * position >= max_position; its row is left).  Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_head_norm_rope(const dopr_rope *rope, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                                         const int32_t *positions, float eps, int32_t gain_dtype, const dopr_heads *q,
                                         const void *q_gain, const dopr_heads *q_out, const dopr_heads *k,
                                         const void *k_gain, const dopr_heads *k_out, int32_t *status,
                                         void *cuda_stream);

/*
 * Its gradients: from those of its outputs (dq_out, dk_out) and its inputs q, k, those of the inputs (dq, dk: views that may
 * be dq_out, dk_out or q, k themselves) and, where asked for, of the gains: dq_gain, dk_gain [head_dim] float, overwritten (the
 * sum over all rows with a position and all heads, in a fixed order).  An input that repeats a row (token_stride 0) gets a gradient
 * for each token.  dk_out, k, dk NULL: q alone.
 *   workspace dopr_head_norm_rope_workspace(head_dim) bytes, 16-byte aligned; NULL where no gain's gradient is asked for.
 */
DOPR_API dopr_status dopr_head_norm_rope_backward(const dopr_rope *rope, int32_t dtype, int32_t head_dim, int32_t n_tokens,
                                                  const int32_t *positions, float eps, int32_t gain_dtype,
                                                  const dopr_heads *dq_out, const dopr_heads *q, const void *q_gain,
                                                  const dopr_heads *dq, float *dq_gain, const dopr_heads *dk_out,
                                                  const dopr_heads *k, const void *k_gain, const dopr_heads *dk,
                                                  float *dk_gain, void *workspace, int32_t *status, void *cuda_stream);
/* Bytes of its workspace; -1 on a bad head_dim. */
DOPR_API int64_t dopr_head_norm_rope_workspace(int32_t head_dim);

/*
 * The same cache in 4 bits: pools of 4.25 bits an element in place of 16.  layout, tables, slots, plan and workspace are those
 * of the calls above; layout->dtype is the type of the rows (q, k, v and out).  32 elements of a head that follow one another
 * (a group) share a scale s and are held as whole numbers c, -7 .. 7, an element as c s.  A scale is a byte, five bits of
 * exponent above three of mantissa: s is the fp16 number of the bits byte << 7.  It is the smallest that is at least
 * max |x| / 7, at most 9216 (byte 0xe1); c = x / s to the nearest whole number, ties away from zero: |x - c s| <= s / 2 for
 * |x| <= 64512.  c s is exact in fp16 and bf16.  A group with a value that is not finite or above 65504 in magnitude is held as
 * NaN (byte 0xff) and stores DOPR_ERR_RANGE in *status; bytes above 0xe1 stand for NaN.
 * k_pool, v_pool: dopr_cache_4bit_pool_bytes(layout) bytes each, 16-byte aligned: [n_blocks][n_kv_heads] pages, each the codes
 * of its rows [page][head_dim / 2 bytes], then their scales [page][head_dim / 32].  Of eight codes c + 8 in a 32-bit word, element
 * 2 i is at bits 4 i and element 2 i + 1 at bits 16 + 4 i.  Memory that was never written must not be read as keys, so clear new pools.
 */
DOPR_API int64_t dopr_cache_4bit_pool_bytes(const dopr_cache_layout *layout);

/*
 * One layer's new rows into the pages at slots[t], as dopr_cache_append: v as it is; k, and q into q_out, normed where
 * eps > 0 (gains as in dopr_head_norm_rope; eps 0: not normed, gains NULL) and turned where rope is not NULL.  k is rounded to
 * layout->dtype, then held: the same bits as dopr_head_norm_rope and an append of its output.  q, q_out NULL: keys and
 * values alone; q needs a norm or a rope.  Views are 16-byte aligned with strides multiples of 16 bytes; rotary_dim is a
 * multiple of 16.  Rows with slots[t] < 0 are not stored; with positions[t] < 0 (and a rope) nothing of a row is written.  Slots
 * are distinct.  Device errors: INVALID_ARG (a slot outside the pool, a position >= max_position; that row is left), RANGE.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_cache_append_4bit(const dopr_cache_layout *layout, const dopr_rope *rope, int32_t n_tokens,
                                            const int32_t *positions, const int64_t *slots, float eps, int32_t gain_dtype,
                                            const dopr_heads *q, const void *q_gain, const dopr_heads *q_out,
                                            const dopr_heads *k, const void *k_gain, const dopr_heads *v, void *k_pool,
                                            void *v_pool, int32_t *status, void *cuda_stream);

/*
 * What the pages hold at slots[t], in layout->dtype (exact): k_out, v_out views of n_rows rows, 16-byte aligned with strides
 * multiples of 16 bytes.  Rows with slots[t] < 0 are left as they were; slots may repeat.  Groups whose scale byte stands for NaN come
 * as NaN, which is no error here.  Device error: INVALID_ARG (a slot outside the pool; its row is left).  Errors: INVALID_ARG,
 * UNSUPPORTED, CUDA.
 */
DOPR_API dopr_status dopr_cache_read_4bit(const dopr_cache_layout *layout, int32_t n_rows, const int64_t *slots,
                                          const void *k_pool, const void *v_pool, const dopr_heads *k_out,
                                          const dopr_heads *v_out, int32_t *status, void *cuda_stream);

/*
 * dopr_shared_attention over such pools: the same plan, arguments and arithmetic on the values that the pages hold.  A scale byte
 * above 0xe1 among a row's keys counts as zero: device error RANGE, which status alone tells: results stay finite.  Other errors as
 * there.  Where up to 8 rows share many keys, a
 * probability times a value's scale is rounded to 11 bits, or to steps of 2^-34 of the largest such product among the keys that the row
 * sees (scales below 2^-15 count as 2^-15 there), and a query's elements below 2^-27 of its head's largest to steps of 2^-37 of that.
 */
DOPR_API dopr_status dopr_shared_attention_4bit(const dopr_cache_layout *layout, const void *plan, int32_t max_tokens,
                                                const dopr_heads *q, const void *k_pool, const void *v_pool,
                                                const int32_t *block_tables, float scale, const dopr_heads *out, float *lse,
                                                void *workspace, int32_t *status, void *cuda_stream);

/*
 * Per-kernel accounting, for measurement.  Every dopr_score call counts its
 * kernel launches per kernel family (pack, embed, gemm_qkv, qknorm_rope,
 * attention, gemm_o, rmsnorm, gemm_gate_up, gemm_down, score, prefix_store;
 * dopr_build_prefixes counts into the same families) together with
 * the algorithmic floating-point operations and device-memory bytes of those
 * launches (the minimum the operation needs: each input read once, each output
 * written once).  While enabled, each launch is also bracketed with CUDA
 * events on the call's stream and the elapsed device time summed per family.
 * dopr_profile_enable clears all counters.  dopr_profile_read copies up to
 * max_entries families into `out` and returns the number of families
 * (or -1 on a NULL model).
 */
typedef struct {
    char name[24];
    int64_t launches;
    double time_ms;   /* summed event time while enabled, else 0 */
    double flops;     /* algorithmic FLOPs                        */
    double bytes;     /* algorithmic device-memory bytes           */
} dopr_kernel_stat;

DOPR_API dopr_status dopr_profile_enable(dopr_model *model, int32_t enable);
DOPR_API int32_t dopr_profile_read(const dopr_model *model, dopr_kernel_stat *out, int32_t max_entries);

/* Thread-local message describing the last failed call on this thread
 * ("" if none).  The pointer stays valid until the next call on the thread. */
DOPR_API const char *dopr_last_error(void);

/* Library version string. */
DOPR_API const char *dopr_version(void);

#ifdef __cplusplus
}
#endif

#endif /* DOPR_H */
