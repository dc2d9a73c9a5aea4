/*
 * nova.h -- C ABI of libnova: the single-GPU hot path of agentic VLM serving on MI355X (gfx950).
 *
 * A request is a screenshot plus an instruction (the paper's Sec. 2.1).  It passes through three
 * stages: vision encode (ViT + adapter), LLM prefill over [visual embeddings ; instruction
 * tokens] which builds the KV cache, and LLM decode, one greedy token per batched step
 * (Sec. 2.1, Sec. 2.2; in-flight decode batching, Sec. 3.4).  The stages run concurrently on
 * disjoint compute-unit partitions chosen before each forward pass (Sec. 3.2.2, Sec. 3.4), and
 * vision-encoder layers can be streamed from pinned host memory into K device slots (Sec. 3.5,
 * Eq. 7).
 *
 * Conventions for every call:
 *  - Return value: NOVA_OK (0) or a negative status; nova_last_error() then describes the failure
 *    (thread-local string).  Nothing is thrown across the ABI.
 *  - Pointers named "device" must point to GPU memory of the current device, 256-byte aligned.
 *    The caller owns all device and pinned-host memory (weights, KV pools, workspaces,
 *    inputs, outputs); the library never frees caller memory and never allocates device
 *    memory in the stage calls.  The library owns only its streams and events.
 *  - Stage calls are asynchronous on the given stream (0 = the null stream): errors in argument
 *    checks and kernel launches are reported at once; faults inside kernels surface at the
 *    caller's next synchronisation.
 *  - Element types: weights are bf16 (uint16 bit patterns).  Activations (stage inputs/outputs,
 *    KV cache) are bf16 when the model's act == NOVA_ACT_BF16 and fp32 when NOVA_ACT_F32.
 *    Logits are always fp32, token ids and block tables int32.
 *  - Threading: one thread per stage may call concurrently (vision, prefill, decode workers,
 *    Sec. 3.1).  A model object may be shared by the prefill and decode threads (they share
 *    weights, Sec. 3.1); nova_vit_encode with offload and nova_prefetch_layer on one nova_vit
 *    must come from one thread.
 */
#ifndef NOVA_H
#define NOVA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ihipStream_t* nova_stream_t; /* a hipStream_t */

enum {
  NOVA_OK = 0,
  NOVA_EINVAL = -1,       /* invalid argument (shape, pointer, alignment, range) */
  NOVA_ENOKV = -2,        /* block table does not cover the requested positions */
  NOVA_EHIP = -3,         /* a HIP runtime call or kernel launch failed */
  NOVA_EUNSUPPORTED = -4, /* configuration outside what the kernels implement */
  NOVA_ENOSPACE = -5      /* workspace smaller than nova_*_workspace_bytes() */
};
enum { NOVA_STAGE_ENCODE = 0, NOVA_STAGE_PREFILL = 1, NOVA_STAGE_DECODE = 2 };
enum { NOVA_ACT_BF16 = 0, NOVA_ACT_F32 = 1 };
enum { NOVA_KIND_GEMM = 0, NOVA_KIND_ATTN = 1, NOVA_KIND_GEMV = 2, NOVA_KIND_DECODE_ATTN = 3, NOVA_KIND_MISC = 4 };

/* Last error message of this thread ("" if none). */
const char* nova_last_error(void);
/* Select the device and create the library's streams/events; call once per process. */
int nova_init(int device);
/* Destroy the library's streams and events (partition streams included). */
void nova_shutdown(void);
/* Number of compute units of the initialised device (256 on MI355X). */
int nova_device_cus(void);

/* ------------------------------------------------------------------ vision encoder (Sec. 2.1)
 * Pre-LN ViT: x0 = patches W_p^T + b_p + E_pos; each layer h = x + Attn(LN1 x) W_o^T + b_o,
 * y = h + GELU(LN2 h W_1^T + b_1) W_2^T + b_2 with bidirectional attention over all patches;
 * adapter: LN per patch, concatenation of each merge x merge patch group, Linear to out_hidden.
 */
typedef struct {
  int hidden, heads, mlp, layers;
  int patch, merge, out_hidden;   /* merge 1 (LN + Linear) or 2 (2x2 patch merge) */
  int image_h, image_w;           /* multiples of patch (and of patch*merge) */
  float eps;                      /* LayerNorm epsilon */
  int act;                        /* NOVA_ACT_BF16 or NOVA_ACT_F32 */
} nova_vit_config;

/* Packed weight blobs.  Every tensor is bf16, row-major, at the returned byte offset (256-byte
 * aligned) of its blob.  Linear weights are [out, in]; "in" is zero-padded to kpad / ip where noted.
 *  embed blob: 0 patch.w [hidden, kpad] (kpad = 3*patch^2 rounded up to 64, zero tail),
 *              1 patch.b [hidden], 2 pos [n_patches, hidden]
 *  layer blob: 0 ln1.g, 1 ln1.b [hidden], 2 qkv.w [3*hidden, hidden] (q | k | v, head-major),
 *              3 qkv.b [3*hidden], 4 o.w [hidden, hidden], 5 o.b, 6 ln2.g, 7 ln2.b,
 *              8 fc1.w [ip, hidden], 9 fc1.b [ip], 10 fc2.w [hidden, ip], 11 fc2.b
 *              (ip = mlp rounded up to 256; padded rows/columns are zero)
 *  head blob:  0 merge.ln.g, 1 merge.ln.b [hidden], 2 merge.w [out_hidden, merge^2*hidden], 3 merge.b
 * offsets must have room for 3 / 12 / 4 entries; *bytes receives the blob size. */
int nova_vit_embed_layout(const nova_vit_config* cfg, size_t* offsets, size_t* bytes);
int nova_vit_layer_layout(const nova_vit_config* cfg, size_t* offsets, size_t* bytes);
int nova_vit_head_layout(const nova_vit_config* cfg, size_t* offsets, size_t* bytes);

typedef struct {
  nova_vit_config cfg;
  const void* embed;        /* device embed blob */
  const void* head;         /* device head blob */
  const void* layers;       /* device: cfg.layers layer blobs back to back (resident), or NULL */
  /* Layer offload (Sec. 3.5): all layer blobs in pinned host memory, n_slots device slots. */
  const void* host_layers;  /* pinned host (hipHostMalloc): cfg.layers blobs back to back, or NULL */
  void* slots;              /* device: n_slots layer blobs back to back */
  int n_slots;              /* K, 2 <= K < layers */
} nova_vit_desc;

typedef struct nova_vit nova_vit;
/* Validate a descriptor and build a model handle (no device memory is allocated; with
 * offload, one copy stream and 2K events are created). */
int nova_vit_create(const nova_vit_desc* desc, nova_vit** out);
void nova_vit_destroy(nova_vit* vit);
/* Bytes of device workspace nova_vit_encode needs for this batch size. */
size_t nova_vit_workspace_bytes(const nova_vit* vit, int batch);

/* Vision encode of `batch` images.
 *  pixels: device bf16 [batch, image_h, image_w, 3] (HWC, values fed as is)
 *  out:    device act-type [batch, n_patches / merge^2, out_hidden]
 * With offload, every layer waits for its slot's copy and, once done, its slot receives layer
 * (l + K) mod L (Eq. 7), so the next call's first K layers are loaded during this one.  When K
 * does not divide L the layer-to-slot map rotates from one call to the next. */
int nova_vit_encode(nova_vit* vit, const void* pixels, int batch, void* out, void* ws, size_t ws_bytes,
                    nova_stream_t stream);

/* Swap logical ViT layer `layer` into a physical slot from pinned host memory on copy_stream
 * (0: the model's own copy stream), after the last compute use of that slot has finished
 * (Sec. 3.5: one event per physical layer guards both the copy and the compute).  No-op if the
 * layer is already in a slot.  The slot is the one holding layer (layer - K) mod L (the Eq. 7
 * ring), else an empty one, else slot layer mod K.  nova_vit_encode queues layers 0..K-1 this
 * way itself; calling it earlier moves those copies ahead of the first encode.  Returns
 * NOVA_EINVAL without offload. */
int nova_prefetch_layer(nova_vit* vit, int layer, nova_stream_t copy_stream);

/* Offload ring state, host side: slot_layer (may be NULL) receives the n_slots logical layers
 * the physical slots hold or are receiving (-1: none yet), copies (may be NULL) the number of
 * host-to-device layer copies issued since creation.  Over repeated encodes the ring issues L
 * copies per call (Eq. 7).  Returns NOVA_EINVAL without offload. */
int nova_vit_offload_state(const nova_vit* vit, int* slot_layer, unsigned long long* copies);

/* ------------------------------------------------------------------ LLM (Sec. 2.1, Sec. 3.4)
 * Decoder layer: RMSNorm -> q, k, v (no bias) -> rotary embedding (half-split pairs) -> causal
 * grouped-query attention -> W_o + residual -> RMSNorm -> SwiGLU MLP + residual; final RMSNorm,
 * untied LM head, greedy argmax (ties to the lowest id).
 */
typedef struct {
  int hidden, n_q, n_kv, head_dim, inter, vocab, layers;
  int block;         /* tokens per KV block; must be 16 */
  float rope_theta;
  float eps;         /* RMSNorm epsilon */
  int act;
} nova_llm_config;

/* layer blob: 0 rms1.g [hidden], 1 qkv.w [(n_q+2n_kv)*head_dim, hidden] (q | k | v, head-major),
 *             2 o.w [hidden, n_q*head_dim], 3 rms2.g [hidden],
 *             4 gu.w [2*ip, hidden]: gate and up rows interleaved in blocks of 8
 *               (rows 16j..16j+7 = gate rows 8j..8j+7, rows 16j+8..16j+15 = up rows 8j..8j+7),
 *             5 down.w [hidden, ip]      (ip = inter rounded up to 256; padding is zero)
 * head blob:  0 norm.g [hidden], 1 lm_head.w [vocab, hidden]
 * The embedding table is a separate device bf16 [vocab, hidden] array. */
int nova_llm_layer_layout(const nova_llm_config* cfg, size_t* offsets, size_t* bytes);
int nova_llm_head_layout(const nova_llm_config* cfg, size_t* offsets, size_t* bytes);

typedef struct {
  nova_llm_config cfg;
  const void* embed;    /* device bf16 [vocab, hidden] */
  const void* layers;   /* device: cfg.layers layer blobs back to back */
  const void* head;     /* device head blob */
} nova_llm_desc;
typedef struct nova_llm nova_llm;
int nova_llm_create(const nova_llm_desc* desc, nova_llm** out);
void nova_llm_destroy(nova_llm* llm);

/* Paged KV cache (PagedAttention-style blocks of 16 tokens), caller-owned device memory:
 *  k: [layers][num_blocks][n_kv][16][head_dim]   (rotated keys)
 *  v: [layers][num_blocks][n_kv][head_dim][16]   (values, transposed within each block)
 * Element type follows the model's act.  nova_kv_bytes() gives the size of each of k and v. */
typedef struct {
  void* k;
  void* v;
  int num_blocks;
} nova_kv;
size_t nova_kv_bytes(const nova_llm* llm, int num_blocks);

/* Device workspace for prefill of up to `seq` tokens, or decode of `batch` sequences whose
 * context never exceeds max_ctx tokens. */
size_t nova_llm_prefill_workspace_bytes(const nova_llm* llm, int seq);
size_t nova_llm_decode_workspace_bytes(const nova_llm* llm, int batch, int max_ctx);

/* Prefill one request (no batching of prefill, Sec. 3.4).
 *  vis:   device act-type [n_vis, hidden] visual embeddings (may be NULL when n_vis == 0)
 *  ids:   device int32 [n_text] instruction tokens, appended after the visual embeddings
 *  block_table: device int32 [ceil((n_vis+n_text)/16)] physical block of each 16 positions
 *  Writes the rotated K and V of positions 0..S-1 into kv, the greedy next token into
 *  next_id (device int32 [1]) and, if logits != NULL, the last-row logits (device fp32 [vocab]). */
int nova_llm_prefill(const nova_llm* llm, const void* vis, int n_vis, const int32_t* ids, int n_text,
                     const int32_t* block_table, const nova_kv* kv, int32_t* next_id, float* logits, void* ws,
                     size_t ws_bytes, nova_stream_t stream);

/* One in-flight-batched decode step for `batch` sequences (batch <= 32).
 *  ids, pos:     device int32 [batch]: token fed and its position (context becomes pos + 1)
 *  block_tables: device int32 [batch, max_blocks] (row b covers positions 0..pos[b])
 *  max_ctx:      an upper bound of pos[b] + 1 over the batch (sizes the attention split); a
 *                position outside 0..max_ctx - 1 is clamped into it (garbage out, no access
 *                outside the sequence's block-table row)
 *  Appends each sequence's K/V at pos[b], writes next_ids (device int32 [batch]) and, if
 *  logits != NULL, device fp32 [batch, vocab]. */
int nova_llm_decode(const nova_llm* llm, const int32_t* ids, const int32_t* pos, const int32_t* block_tables,
                    int max_blocks, int batch, int max_ctx, const nova_kv* kv, int32_t* next_ids, float* logits,
                    void* ws, size_t ws_bytes, nova_stream_t stream);

/* Allocation-free decode step, for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the same step as
 * nova_llm_decode, same arguments and results, with its workspace (activations, split-K partial
 * sums, arrival counters, attention split partials) taken from a library-owned static device
 * array of NOVA_DECODE_SCRATCH_BYTES bytes, which each GPU the library runs on holds until the
 * process ends.  Calls no hipMalloc, hipFree or other allocating routine.  The step clears what
 * must start at zero (argmax keys, arrival counters) in its own first kernel; the array keeps the
 * last call's contents otherwise.  Every call on one GPU uses that GPU's single array: calls that
 * overlap in time on one GPU (two streams, two threads) race on it and give wrong results, so
 * the caller serialises them.  A step whose workspace (nova_llm_decode_workspace_bytes) exceeds
 * NOVA_DECODE_SCRATCH_BYTES returns NOVA_ENOSPACE and launches nothing; the 28-layer 3584-wide
 * decoder at batch 32 needs about 9 MB. */
#define NOVA_DECODE_SCRATCH_BYTES (32u << 20)
int nova_llm_decode_noalloc(const nova_llm* llm, const int32_t* ids, const int32_t* pos, const int32_t* block_tables,
                            int max_blocks, int batch, int max_ctx, const nova_kv* kv, int32_t* next_ids,
                            float* logits, nova_stream_t stream);

/* ------------------------------------------------------------------ operators over the paged cache
 * Calls below the stages, for programs that batch, draft or move requests themselves.  One layer at
 * a time, asynchronous on `stream`; device pointers are 16-byte aligned unless stated otherwise, and
 * rows are [n_heads][head_dim] contiguous at a pitch of their own (a multiple of 16 bytes, so q, k
 * and v may be views of one packed projection).  head_dim is 64 or 128.
 *
 * Of one call: at most 8192 heads, 2^25 rows and 2^30 tokens of a sequence.
 *
 * A cache layer of one of three types.  BF16 and F32 are a layer of a nova_kv pool.  E4M3 stores
 * 8 bits per value: token t of a KV head is D OCP e4m3 numbers and one byte e + 127, the values
 * being number * 2^e with the smallest e >= -100 that keeps |number| <= 448 (NaN and infinite values
 * are stored as NaN).  Values read back are exact in bf16, and appending them again stores the same
 * values (a largest one that rounded to 224 * 2^e becomes 448 * 2^(e-1)).  With the largest e, 120, a
 * number is at most 240, so that every finite value reads back finite. */
enum { NOVA_CACHE_BF16 = 0, NOVA_CACHE_F32 = 1, NOVA_CACHE_E4M3 = 2 };
typedef struct {
  void* k;          /* [num_blocks][n_kv][16][head_dim], 256-byte aligned */
  void* v;          /* [num_blocks][n_kv][head_dim][16], 256-byte aligned */
  uint8_t* k_exp;   /* E4M3: [num_blocks][n_kv][16]; else ignored */
  uint8_t* v_exp;
  int num_blocks, n_kv, head_dim, type;
} nova_cache;
/* Bytes of each of k and v of one layer (0 for invalid sizes); *exp_bytes (may be NULL): of each of
 * k_exp and v_exp. */
size_t nova_cache_bytes(int type, int num_blocks, int n_kv, int head_dim, size_t* exp_bytes);

/* A batch of sequences over a cache and the rows (tokens) that each brings.  Row j of sequence b is
 * row row_start[b] + j of the arrays and token ctx[b] + j of the sequence.  The arrays are read on
 * the device when the kernels run.  Row starts outside the rows are clamped into them; tokens outside
 * 0 .. max_ctx - 1 do not exist: such a row is not written to the cache, reads as zeros and is not seen
 * (its q is still rotated, and it still attends to what exists). */
typedef struct {
  const int32_t* row_start;  /* device int32 [batch + 1], ascending; NULL: max_rows rows each (rows == batch * max_rows) */
  const int32_t* ctx;        /* device int32 [batch]: tokens in the cache before these rows; NULL: 0 */
  const int32_t* tables;     /* device int32 [batch][max_blocks]: physical block of each 16 tokens; an
                                entry outside the pool names no block: its tokens are neither written nor seen */
  int max_blocks, batch;
  int rows;                  /* rows of the arrays; those behind row_start[batch] are left as they were */
  int max_rows;              /* upper bound of one sequence's rows; rows beyond it are left out */
  int max_ctx;               /* upper bound of ctx[b] plus its rows, at most 16 * max_blocks: see above */
} nova_rows;

/* Rotary embedding of the first `rot` dimensions (a multiple of 16, at most head_dim) of a head:
 * pairs (c, c + rot/2), or (2c, 2c + 1) when interleaved, turned by position * f_c with
 * f_c = theta^(-2c/rot).  Longer contexts: factor > 1 divides every f_c by it (linear interpolation);
 * with orig_ctx > 0 only as far as f_c turns fewer than `beta` times over orig_ctx tokens, wholly at
 * `alpha` turns and below (the "NTK-by-parts" interpolation of YaRN, arXiv 2309.00071, Eq. 18-20).
 * Sines and cosines are multiplied by mscale.  Angles are formed in 64 bits. */
typedef struct {
  int rot, interleaved;
  float theta, factor;
  int orig_ctx;
  float alpha, beta, mscale;
} nova_rope;

/* Append rows to a cache layer: q and k are rotated (rope NULL: not) at position pos[row] (device
 * int32 [rows]; NULL: the token's number in its sequence), the rotated q goes to q_out, k and v into
 * the cache (E4M3: quantised from the fp32 rotation, rounded once).
 *  q, k, v: device, all of in_type (NOVA_ACT_BF16 / NOVA_ACT_F32), rows of n_q, n_kv and n_kv heads at
 *           pitches in elements; q may be NULL (n_q 0): only k and v
 *  q_out:   device, q_out_type; may be q itself (same type and pitch)
 * No two rows may name the same slot of the same block (sequences that share a block append behind it). */
int nova_kv_append(const nova_cache* cache, const nova_rows* rows, const nova_rope* rope, const int32_t* pos,
                   int in_type, const void* q, int64_t q_pitch, int n_q, const void* k, int64_t k_pitch, const void* v,
                   int64_t v_pitch, void* q_out, int q_out_type, int64_t q_out_pitch, nova_stream_t stream);

/* Positions with several axes (time, row and column of an image's or video's tokens): pair c turns by the
 * position of one of n_axes axes (1 to 4), of which axis a gets pairs[a] pairs (their sum is rot / 2; 0: none):
 * runs of them in order, or when cyclic dealt one by one to the axes in turn, leaving out those that have theirs.
 * Pair c keeps the frequency theta^(-2c/rot) whatever its axis; with own_freqs the i-th of an axis' m pairs has
 * theta^(-i/m) (the axes' frequencies are alike).  Scaling for longer contexts applies to either. */
typedef struct {
  int n_axes;
  int pairs[4];
  int cyclic, own_freqs;
} nova_rope_axes;

/* nova_kv_append with positions of several axes: pos is device int32 [n_axes][rows] (NULL: the token's number on
 * every axis).  axes NULL: nova_kv_append; else rope is needed. */
int nova_kv_append_axes(const nova_cache* cache, const nova_rows* rows, const nova_rope* rope, const nova_rope_axes* axes,
                        const int32_t* pos, int in_type, const void* q, int64_t q_pitch, int n_q, const void* k,
                        int64_t k_pitch, const void* v, int64_t v_pitch, void* q_out, int q_out_type, int64_t q_out_pitch,
                        nova_stream_t stream);

/* Rotary embedding of dense rows [n_heads][head_dim] (a vision encoder's q and k, say): head_dim is a multiple of 8
 * up to 256, rot as in nova_rope up to head_dim; what is not turned is copied.
 *  pos:    device int32 [n_axes][rows], or [rows] with axes NULL
 *  x, out: device, in_type and out_type, pitches in elements; out may be x itself (same type and pitch) */
int nova_rotate(const nova_rope* rope, const nova_rope_axes* axes, const int32_t* pos, int rows, int n_heads, int head_dim,
                int in_type, const void* x, int64_t x_pitch, int out_type, void* out, int64_t out_pitch,
                nova_stream_t stream);

/* Read cached rows back as dense rows of out_type: row j of sequence b is token slots[row] (device
 * int32 [rows]; NULL: ctx[b] + j) of it.  Tokens of missing blocks read as zeros.  With the accepted
 * tokens of a tree as slots, a following nova_kv_append (no rope) moves them behind the context. */
int nova_kv_gather(const nova_cache* cache, const nova_rows* rows, const int32_t* slots, int out_type, void* k_out,
                   int64_t k_pitch, void* v_out, int64_t v_pitch, nova_stream_t stream);

/* Attention of each sequence's rows (drafted tokens, at most 64, already appended) over its cache:
 * row j sees every token below ctx[b], and token ctx[b] + i where bit i of mask[row] is set
 * (device uint64 [rows]; NULL: i <= j, a chain; one row per sequence is a decode step).  A row that
 * sees nothing gets zeros (one that sees scores of -infinity only has no softmax: NaN); what a row does
 * not see has no effect on it, whatever it holds.
 *  q, out: device, bf16 (F32 with an F32 cache), n_q heads (a multiple of n_kv); scale is applied to q.k
 *          (scores and the sums of p v, where p is up to 2^8, are fp32: scores up to 2^24 in magnitude and
 *          V up to 2^88 are safe)
 *  ws:     device, nova_tree_attention_workspace_bytes(), 256-byte aligned; contents need not be kept
 *          or cleared, but calls that may overlap in time need one each */
size_t nova_tree_attention_workspace_bytes(const nova_cache* cache, const nova_rows* rows, int n_q);
int nova_tree_attention(const nova_cache* cache, const nova_rows* rows, const uint64_t* mask, const void* q, int64_t q_pitch,
                        int n_q, float scale, void* out, int64_t out_pitch, void* ws, size_t ws_bytes,
                        nova_stream_t stream);

/* ------------------------------------------------------------------ log probabilities
 * From rows of logits (device, NOVA_ACT_BF16 / NOVA_ACT_F32, pitch in elements, any alignment of
 * their element; as the LLM calls return them), in fp32:
 *  given_lp[row][i] = log p(given[row][i]) (device int32 [rows][n_given]; -infinity for ids outside the
 *                     vocabulary), n_given 0: none
 *  entropy[row]     = -sum p log p; may be NULL
 *  top_lp, top_ids[row][n_top]: the most likely tokens, descending, equal ones by the lower id (NaN
 *                     counts as the largest); n_top <= 32 and <= vocab, 0: none
 * A logit of -infinity has probability 0.  A row with a NaN or +infinity, or with nothing but
 * -infinity, has NaN for every log probability of a token and for its entropy.  vocab <= 2^21, rows < 2^23.
 *  ws: device, nova_logprobs_workspace_bytes(), 256-byte aligned, as for nova_tree_attention */
size_t nova_logprobs_workspace_bytes(int rows, int vocab, int n_top);
int nova_logprobs(const void* logits, int type, int64_t pitch, int rows, int vocab, const int32_t* given, int n_given,
                  float* given_lp, float* entropy, int n_top, float* top_lp, int32_t* top_ids, void* ws,
                  size_t ws_bytes, nova_stream_t stream);

/* ------------------------------------------------------------------ between two model calls
 * What a program does with a verify step's logits and rows before the next one, on the device throughout, so that a
 * captured graph can hold the whole step.  Of `rows` the acceptance and the adapters read row_start, batch, rows and
 * max_rows only.
 *
 * Which drafted tokens are kept.  Row j of a sequence (at most 64) feeds token ids[row] and logits[row] are what the
 * target says after it; row 0 is the last token that is certain, the others are drafted.  With p a row's
 * probabilities at the sequence's temperature:
 *  - draft NULL: every row draws a token from p with its number u[row]; from row 0 the walk goes on in the first row
 *    that hangs under the present one and feeds the token drawn there, and ends where there is none.  mask (as for
 *    nova_tree_attention: a row hangs under the highest row below it that it sees) NULL: a chain.
 *  - draft (logits of the distributions that the drafted tokens were drawn from, row j's token from draft[row j]; row
 *    0's are not read; a chain, mask must be NULL): row j >= 1 is kept while u[row j] q(x) < p(x), p of the row before
 *    it.  Behind the last kept row the token is drawn with u[row 0]: from max(p - q, 0) where a row was not kept, else
 *    from p.  (Speculative sampling: the tokens are distributed as the target's own.)  A draft row without a
 *    distribution keeps nothing, and p is drawn from.
 * A draw is the first token whose running sum of probabilities exceeds u times their total (64-bit sums; u outside [0, 1)
 * is taken into it, NaN as 0).  Temperature 0 is greedy (the largest logit, of equal ones the lowest id; a drafted token
 * is kept if it is that).  A row with a NaN or +infinity, with nothing but -infinity, or of a sequence whose temperature
 * is negative, infinite or NaN has no distribution: its token is -1, its log probability NaN, and the walk ends there.
 *  logits, draft: device, NOVA_ACT_BF16 / NOVA_ACT_F32, pitch in elements, any alignment of their element
 *  temperature:   device fp32 [batch], or NULL: 1
 *  n_keep: device int32 [batch]: rows kept, row 0 among them (0: the sequence has no rows)
 *  path:   device int32 [batch][max_rows]: the kept rows' numbers in their sequence, ascending; -1 behind
 *  tokens: device int32 [batch][max_rows]: the token after each kept row (the last of them is new); -1 behind
 *  lp:     device fp32 [batch][max_rows]: their log probabilities under p (0 at temperature 0 and behind)
 * vocab <= 2^21, and rows (twice with draft) and batch times ceil(vocab / 8192) are below 2^24.
 *  ws: device, nova_accept_workspace_bytes(), 256-byte aligned, as for nova_tree_attention */
size_t nova_accept_workspace_bytes(const nova_rows* rows, int vocab, int with_draft);
int nova_accept(const nova_rows* rows, const int32_t* ids, const uint64_t* mask, const void* logits, int type, int64_t pitch,
                const void* draft, int draft_type, int64_t draft_pitch, int vocab, const float* temperature, const float* u,
                int32_t* n_keep, int32_t* path, int32_t* tokens, float* lp, void* ws, size_t ws_bytes, nova_stream_t stream);

/* Keep the accepted rows in `layers` layers of a cache (cache describes layer 0; layer l's arrays follow at l times
 * their size): token ctx[b] + path[b][i] of sequence b becomes its token ctx[b] + i, for i < n_keep[b] (as nova_accept
 * gives them; path NULL: the rows are in their places).  Everything is read before anything is written.  A path entry
 * outside the sequence's rows, or a token that does not exist, leaves its place as it was.
 *  ctx_out: device int32 [batch]: ctx[b] + n_keep[b] (n_keep taken into 0 .. the sequence's rows); not ctx itself; or NULL
 * At most 64 rows of a sequence; batch * layers * n_kv is at most 2^24. */
int nova_kv_keep(const nova_cache* cache, int layers, const nova_rows* rows, const int32_t* path, const int32_t* n_keep,
                 int32_t* ctx_out, nova_stream_t stream);

/* Blocks from[i] of one cache to blocks to[i] of another of the same type and heads, or of itself, in `layers` layers
 * (from, to: device int32 [n]).  Entries outside the pools copy nothing.  No block may be named twice in `to`, nor in both. */
int nova_kv_copy(const nova_cache* src, const nova_cache* dst, int layers, const int32_t* from, const int32_t* to, int n,
                 nova_stream_t stream);

/* The blocks of a pool: refs[block] is how many table entries name it; a block with 0 is free.  tables are device int32
 * [batch][max_blocks], an entry outside the pool names no block.  What is taken are always the lowest free blocks, in the
 * order of the requests; a request is served (done 1) if it and the requests before it find enough, and else left as it
 * was (done 0).  Calls on one pool are made one after the other (on one stream, say).  At most 65535 requests.
 * Rows share whole pages only, and none of these calls leaves a row ending inside a page that another names: rows append
 * behind what they share.  (A program that lowers a row's ctx by itself, or forks more tokens than the source holds, has
 * to see to that.)
 *  ws: device, nova_pages_workspace_bytes(), 256-byte aligned, as for nova_tree_attention */
typedef struct {
  int32_t* refs;    /* device [num_blocks], all 0 at first */
  int num_blocks;
} nova_pages;
size_t nova_pages_workspace_bytes(const nova_pages* pages, int batch, int n);
/* Give every sequence the blocks of its first tokens[b] tokens (device int32 [batch]; those that it lacks are taken);
 * done: device int32 [batch] (0 also where the table is too short). */
int nova_pages_extend(const nova_pages* pages, int32_t* tables, int max_blocks, int batch, const int32_t* tokens,
                      int32_t* done, void* ws, size_t ws_bytes, nova_stream_t stream);
/* Row dst[i] of the tables becomes the first tokens[i] tokens of row src[i] (device int32 [n] each): whole blocks are
 * shared, the last one, if tokens[i] fills it only in part, is copied in `layers` layers to a block that is taken.  What
 * row dst[i] named before is overwritten (give it up first).  Refused (done[i] 0): rows outside the tables, a target
 * that is a request's source (its own or another's: no source is overwritten) or an earlier request's target (served or
 * not), tokens beyond the source's blocks. */
int nova_pages_fork(const nova_pages* pages, const nova_cache* cache, int layers, int32_t* tables, int max_blocks, int batch,
                    const int32_t* src, const int32_t* dst, const int32_t* tokens, int n, int32_t* done, void* ws,
                    size_t ws_bytes, nova_stream_t stream);
/* Rows seqs[i] (device int32 [n]) give up everything; their entries become -1.  tokens: NULL (see nova_pages_trim). */
int nova_pages_free(const nova_pages* pages, int32_t* tables, int max_blocks, int batch, const int32_t* seqs,
                    const int32_t* tokens, int n, nova_stream_t stream);
/* Rows seqs[i] give up what lies behind their first tokens[i] tokens (device int32 [n] each); the entries become -1.  The
 * row goes on in the page that it keeps in part, so a request whose page is named by other entries too (counts as they
 * were before the call) is refused: done[i] 0, the row left as it was (device int32 [n]; 0 also for rows outside the
 * tables).  nova_pages_fork gives such tokens to another row with a copy of that page, after which this one can be freed. */
int nova_pages_trim(const nova_pages* pages, int32_t* tables, int max_blocks, int batch, const int32_t* seqs,
                    const int32_t* tokens, int n, int32_t* done, nova_stream_t stream);
/* Move the pool's used blocks to its front: of `live` of them those at live and above go to the free ones below, in order,
 * in `layers` layers, and tables and refs follow (refs_out, tables_out: of their shapes, or refs and tables themselves;
 * entries that name no used block become -1).  live_out: device int32 [1], or NULL.  Every table that names blocks of the
 * pool has to be among the tables. */
int nova_pages_compact(const nova_pages* pages, const nova_cache* cache, int layers, const int32_t* tables, int max_blocks,
                       int batch, int32_t* refs_out, int32_t* tables_out, int32_t* live_out, void* ws, size_t ws_bytes,
                       nova_stream_t stream);

/* ------------------------------------------------------------------ adapters
 * Low-rank adapters of many requests beside a projection that they share:
 *   out[row] = base[row] + scale[i] b[i] (a[i] x[row]),  i = which[sequence of the row]
 * (fp32 sums, a[i] x[row] taken on in all its 24 bits, rounded once; which outside 0 .. n - 1: no adapter, out is base;
 * an infinite weight gives infinity or NaN).  Rows outside the sequences are left as
 * they were.
 *  which: device int32 [batch];  x: device, x_type;  base: device, out_type, NULL: 0;  out: device, out_type, may be
 *         base itself (same pitch); pitches in elements, a multiple of 16 bytes
 * rank is a multiple of 8 up to 128; k and n_out are multiples of 8 up to 2^24. */
typedef struct {
  const void* a;       /* device bf16 [n][rank][k] */
  const void* b;       /* device bf16 [n][n_out][rank] */
  const float* scale;  /* device fp32 [n], or NULL: 1 */
  int n, rank, k, n_out;
} nova_adapters;
size_t nova_lora_workspace_bytes(const nova_adapters* adapters, const nova_rows* rows);
int nova_lora(const nova_adapters* adapters, const nova_rows* rows, const int32_t* which, int x_type, const void* x,
              int64_t x_pitch, int out_type, const void* base, int64_t base_pitch, void* out, int64_t out_pitch, void* ws,
              size_t ws_bytes, nova_stream_t stream);

/* ------------------------------------------------------------------ LLM on a cache of any type
 * nova_llm_prefill into a pool of nova_cache layers (cache describes layer 0; layer l's arrays follow
 * at l times their size): the prompt's attention reads K and V as computed, the cache keeps them in
 * its type.  The cache type is BF16 or E4M3 for a bf16 model, F32 for an fp32 one.  An E4M3 cache holds
 * what a BF16 one would, quantised: K is rounded to bf16 after its rotation and then to 8 bits. */
int nova_llm_prefill_cache(const nova_llm* llm, const void* vis, int n_vis, const int32_t* ids, int n_text,
                           const int32_t* block_table, const nova_cache* cache, int32_t* next_id, float* logits,
                           void* ws, size_t ws_bytes, nova_stream_t stream);

/* One decode step over drafted tokens (speculative decoding): the rows' tokens ids run through the
 * model together, each layer appending their K and V (in fp32 from the projection, rounded once) behind
 * its sequence's context and attending by mask, as nova_kv_append and nova_tree_attention do.  One row per
 * sequence is a plain decode step.
 *  ids, pos: device int32 [rows], rows <= 32: tokens and their rotary positions
 *  mask:     device uint64 [rows] or NULL (chains)
 *  next_ids [rows], logits [rows][vocab] or NULL: as for nova_llm_decode, one per row; rows behind
 *            the last sequence need valid ids too, and what they get means nothing
 * The sequences keep only the tokens that the caller accepts: the rest of the slots are overwritten
 * by the next step's rows. */
size_t nova_llm_verify_workspace_bytes(const nova_llm* llm, const nova_cache* cache, const nova_rows* rows);
int nova_llm_verify(const nova_llm* llm, const int32_t* ids, const int32_t* pos, const uint64_t* mask,
                    const nova_rows* rows, const nova_cache* cache, int32_t* next_ids, float* logits, void* ws,
                    size_t ws_bytes, nova_stream_t stream);

/* The same calls with rotary positions of the rows' own, for prompts with images or video: rope in place of the
 * model's (rope_theta over the whole head at the tokens' numbers), with axes (or NULL: one position a row), and pos
 * device int32 [n_axes][rows] ([n_axes][n_vis + n_text] of a prompt; [rows] with axes NULL).  What a row sees goes by
 * its place in the sequence as before.  Workspaces are those of nova_llm_prefill and nova_llm_verify. */
int nova_llm_prefill_axes(const nova_llm* llm, const void* vis, int n_vis, const int32_t* ids, int n_text,
                          const int32_t* block_table, const nova_cache* cache, const nova_rope* rope, const nova_rope_axes* axes,
                          const int32_t* pos, int32_t* next_id, float* logits, void* ws, size_t ws_bytes, nova_stream_t stream);
int nova_llm_verify_axes(const nova_llm* llm, const int32_t* ids, const nova_rope* rope, const nova_rope_axes* axes,
                         const int32_t* pos, const uint64_t* mask, const nova_rows* rows, const nova_cache* cache,
                         int32_t* next_ids, float* logits, void* ws, size_t ws_bytes, nova_stream_t stream);

/* ------------------------------------------------------------------ linear co-run study
 * The two-linear experiment behind the paper's choice of inter-CU partitioning (Sec. 3.2.1, its
 * linear co-run table, and Sec. 3.2.3): one linear layer out[M, N] += x[M, K] w[N, K]^T
 * (x, w device bf16 row-major, out device fp32, all 256-byte aligned), enqueued on `stream`,
 * with one of the kernels the stage calls use or the low-footprint pair of the intra-CU variant:
 *  NOVA_LINEAR_TILED       the encode / prefill GEMM (tiles chosen by size as for the stages;
 *                          K % 64 == 0, N % 128 == 0)
 *  NOVA_LINEAR_TILED_SMALL the same GEMM held to 128x128 tiles of 4 waves (64 KB of LDS), so a
 *                          CU keeps room for another kernel's workgroups
 *  NOVA_LINEAR_THIN        the decode thin GEMM on the matrix cores (M <= 32, K % 256 == 0,
 *                          N % 64 == 0, and N large enough that K is not split on the stream's CUs)
 *  NOVA_LINEAR_THIN_VALU   the decode linear on the vector ALUs without LDS (M <= 4, K % 512 == 0)
 * Returns NOVA_EUNSUPPORTED outside those shapes. */
enum { NOVA_LINEAR_TILED = 0, NOVA_LINEAR_TILED_SMALL = 1, NOVA_LINEAR_THIN = 2, NOVA_LINEAR_THIN_VALU = 3 };
int nova_linear(int variant, const void* x, int M, int K, const void* w, int N, float* out, nova_stream_t stream);

/* ------------------------------------------------------------------ CU partitions (Sec. 3.2.2)
 * gfx950 deals a kernel's workgroups round-robin over its 8 XCDs, and a CU-mask bit i selects
 * CU slot i/32 of shader engine (i/8)%4 of XCD i%8.  A partition therefore never confines a
 * stage to whole XCDs (the other XCDs' share of its workgroups could not run); it takes the
 * same CU slots on every XCD.  32 CUs = one mask word = 4 CUs on each XCD, one per engine. */

/* XCD-balanced mask of n_cus CUs (a positive multiple of 8, <= 256) starting at CU slot
 * first_slot (0..31, per shader engine): mask bits for slots first_slot .. first_slot +
 * n_cus/8 - 1 on every XCD, engines interleaved.  mask must have room for 8 words. */
int nova_make_cu_mask(int n_cus, int first_slot, uint32_t* mask);

/* Give `stage` the CUs in cu_mask (mask_words 32-bit words, bit i = CU i as above) and return
 * in *out_stream a library-owned stream restricted to them (created with
 * hipExtStreamCreateWithCUMask on first use of that mask, default priority, then cached).
 * A new mask's complement (when it keeps a CU on every XCD) gets its stream created right
 * after it, so that a stage pair on complementary masks sits on different hardware dispatch
 * pipes and runs concurrently; pairs of other masks carry no such guarantee.  Stages given the
 * same partial mask share its stream; the whole-GPU mask has a separate stream per stage
 * (the three are created together).
 * Work enqueued afterwards on *out_stream starts only after everything previously enqueued on
 * the stage's prior partition stream (ordering across the switch, Sec. 3.4: partitions change
 * only between forward passes).  Host-synchronous; does not wait for the device.
 * An empty mask, a mask with no CU on some XCD, or stage out of range gives NOVA_EINVAL. */
int nova_set_stage_partition(int stage, const uint32_t* cu_mask, int mask_words, nova_stream_t* out_stream);

/* Diagnostic: launch n_workgroups single-wave workgroups on `stream`; workgroup i writes
 * (xcd << 16) | (shader_engine << 8) | cu of the compute unit it ran on into out[i]
 * (device uint32 [n_workgroups]).  Used to check that a partition stream stays on its CUs. */
int nova_cu_probe(nova_stream_t stream, uint32_t* out, int n_workgroups);

/* ------------------------------------------------------------------ kernel timing
 * When on, every kernel family launch inside the stage calls is bracketed by HIP events on
 * its stream.  nova_timing_read waits for the recorded events of `kind` (NOVA_KIND_*), returns
 * the summed GPU time and number of launches since the last read, and clears them. */
int nova_timing_enable(int on);
int nova_timing_read(int kind, double* total_ms, int* launches);

#ifdef __cplusplus
}
#endif
#endif /* NOVA_H */
