/*
 * pq_attn — single-query decode attention over a product-quantized (PQ) KV cache,
 * and the nearest-centroid encode that appends tokens to it, for AMD MI355X (gfx950).
 *
 * Plain C ABI: every pointer argument says whether it is host or device memory,
 * every size is in elements unless it says bytes.  No call takes ownership of
 * caller memory; the context owns only its own scratch (re-packed codebooks,
 * split partials, tickets).  Calls are asynchronous on the HIP stream passed in
 * (a hipStream_t cast to void*, NULL = the default stream) and never synchronise
 * the host, except pq_attn_create / pq_attn_destroy / pq_attn_device_error.
 *
 * Notation (Section III-A, Eq. 4-6): B sequences, Hq query heads, Hkv KV heads
 * (query head h reads KV head h / (Hq/Hkv)), d = head_dim, M subspaces of width
 * ds = d / M, C = 256 centroids per subspace (8-bit codes), N_b quantized tokens
 * and R_b recent full-precision tokens of sequence b.
 *
 * Code tensors.  Logically Delta_K, Delta_V are [B][Hkv][N][M] uint8 (Eq. 4).  On the
 * device each is an opaque buffer of pq_attn_codes_bytes() bytes in a layout chosen
 * for the scan kernels (K and V use different layouts).  pq_encode_append writes
 * that layout directly; pq_pack_codes / pq_unpack_codes convert from / to the
 * logical token-major form.
 *
 * Every function returns a pq_status (0 = PQ_OK, negative = error) unless noted.
 * On an argument error nothing is launched.
 */
#ifndef PQ_ATTN_H
#define PQ_ATTN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pq_attn_ctx pq_attn_ctx;

typedef enum {
    PQ_OK = 0,
    PQ_ERR_NULL = -1,        /* a required pointer is NULL                               */
    PQ_ERR_SHAPE = -2,       /* sizes are inconsistent (Hq % Hkv, d % M, negative, ...)    */
    PQ_ERR_UNSUPPORTED = -3, /* a consistent shape this build has no kernel for          */
    PQ_ERR_CAPACITY = -4,    /* n_new / n_tokens exceeds the configured capacity         */
    PQ_ERR_HIP = -6,         /* a HIP runtime call failed                                */
    PQ_ERR_ALLOC = -7        /* device or host allocation failed                         */
} pq_status;

typedef enum { PQ_F16 = 0, PQ_F32 = 1, PQ_BF16 = 2 /* paged caches only */ } pq_dtype;
typedef enum { PQ_CODES_K = 0, PQ_CODES_V = 1 } pq_code_kind;

typedef struct {
    int32_t batch;        /* B >= 1                                                         */
    int32_t n_q_heads;    /* Hq                                                             */
    int32_t n_kv_heads;   /* Hkv, Hq % Hkv == 0                                             */
    int32_t head_dim;     /* d; supported: 128                                              */
    int32_t n_subspaces;  /* M; supported: 64 (ds = 2, 4 bits/dim) and 32 (ds = 4, 2 bits/dim) */
    int32_t n_centroids;  /* C; supported: 256 (nbits = 8), and 4096 (nbits = 12) with M = 32, fp16 */
    int32_t max_context;  /* token capacity of the code tensors per (sequence, KV head),    */
                          /* 1 .. 2^24                                                      */
    int32_t max_recent;   /* row capacity of the recent window tensors (0: no window), <= 2^24 */
    int32_t dtype;        /* pq_dtype of q, codebooks, recent K/V and new K/V               */
    int32_t device;       /* HIP device ordinal                                             */
    int32_t n_splits;     /* context splits per (sequence, query head); 0 = choose.         */
                          /* "0 = choose" with 2..64 sequences of 8-bit codes: the decode     */
                          /* kernel gives its workgroups to the sequences by their lengths   */
                          /* 4096-centroid contexts only: -k asks for the two-pass decode   */
                          /* (split by subspace group) with k token ranges; "0 = choose"    */
                          /* takes it by itself when (sequence, head) pairs are few         */
    int32_t reserved;     /* must be 0                                                      */
} pq_attn_config;

/* Checks the configuration on the host (no GPU needed): PQ_OK or the error
 * pq_attn_create would return for it. */
int pq_attn_validate_config(const pq_attn_config *cfg /* host */);

/* Bytes of ONE device code tensor (K or V) for this configuration: the token
 * capacity is rounded up to whole 64-token blocks.  Returns a negative pq_status
 * for an invalid configuration.  Host-only. */
int64_t pq_attn_codes_bytes(const pq_attn_config *cfg /* host */);

/* Creates a context on cfg->device: allocates the context-owned scratch and
 * synchronises.  *out is set only on PQ_OK.  The caller frees it with
 * pq_attn_destroy (which synchronises the device first). */
int pq_attn_create(const pq_attn_config *cfg /* host */, pq_attn_ctx **out /* host */);
int pq_attn_destroy(pq_attn_ctx *ctx);

/* Number of context splits the decode kernel uses (after "0 = choose"; a batch whose workgroups follow the
 * sequences' lengths has no such number: the one that fills the chip with equal lengths is returned). */
int pq_attn_n_splits(const pq_attn_ctx *ctx);

/* Kernels one pq_attn_decode call launches: 1 (fused), or 2 for a 4096-centroid
 * context that decodes in two passes (partial scores per subspace group, then
 * softmax and values). */
int pq_attn_n_passes(const pq_attn_ctx *ctx);

/* Query heads one decode workgroup serves: 1 for the kernels that build per-query
 * tables, 2..4 for the grouped-query kernels (one pass over a KV head's codes for
 * that many query heads: a KV head's Hq / Hkv >= 2 query heads are cut into
 * ceil(Hq / Hkv / 4) sub-groups of 2..4 heads, sizes as equal as possible, and the
 * largest is returned; chosen when the context is fp16 — for 4096-centroid contexts only where the shape is large
 * enough to pay for it: fewer than 5 compute units per (sequence, query head), or
 * a capacity of 1.5 M (query head, token) pairs, and n_splits >= 0). */
int pq_attn_heads_per_workgroup(const pq_attn_ctx *ctx);

/* Registers the codebooks trained offline (Section III-A, "Offline PQ Codebook
 * Training"): C_K, C_V as [Hkv][M][C][ds] in the context dtype, device memory.
 * The kernels launched by this call copy them into context-owned memory (a plain
 * copy for the encode kernels, a centroid-major image for the decode kernels); the
 * caller's tensors are read by those kernels only and may be freed, overwritten
 * or reused once they have run (i.e. after later work on the same stream, or a
 * stream synchronisation).  The library keeps no pointer to them.
 *
 * pq_attn_decode and pq_encode_append take codebook pointers too: non-NULL
 * pointers are registered by that call, on its stream, before its kernels (the
 * copy costs a few microseconds per call — register once and pass NULL in a
 * decoding loop).  A codebook changed in place has to be registered again.
 * Contexts of 64 subspaces keep what long appends look codes up in, from the first append on before which others
 * have paid for building it, for codebooks registered by this call, not by the other two: 3.3 MB of device memory per KV head (3.4 MB in
 * fp32), allocated by the first such append (never while a graph is recorded), freed with the context.
 * Registration must be stream-ordered with every other call on the context that
 * uses the codebooks: with two streams (asynchronous quantization), register
 * first, synchronise, then pass NULL on both. */
int pq_attn_set_codebooks(pq_attn_ctx *ctx, const void *k_codebook /* device */,
                          const void *v_codebook /* device */, void *hip_stream);

/* Decode attention for one new token per sequence over the quantized cache plus
 * the recent window (Eq. 6, evaluated as Eq. 7: per-head tables q^i.(C_K^i)^T are
 * sampled by the K codes, one softmax shared with the full-precision rows, values
 * aggregated through C_V by the V codes; Section III-B "Efficient Attention
 * Implementation" and steps 1-4 of Section III-C).
 *
 *   q           device [B][Hq][d]                 dtype
 *   k_codes     device, pq_attn_codes_bytes()     device layout (PQ_CODES_K)
 *   v_codes     device, pq_attn_codes_bytes()     device layout (PQ_CODES_V)
 *   ctx_len     device [B] int32                  N_b, clamped to [0, max_context]
 *   k_codebook  device [Hkv][M][C][ds] dtype      or NULL = the registered ones
 *   v_codebook  likewise
 *   recent_k/v  device [B][Hkv][max_recent][d]    dtype; both NULL = no window
 *   recent_len  device [B] int32                  R_b, clamped to [0, max_recent]; NULL = all 0
 *   scale       1/sqrt(d) of Eq. 1; must be finite (PQ_ERR_SHAPE otherwise)
 *   out         device [B][Hq][d] float32
 *
 * Rows >= R_b of the recent tensors and tokens >= N_b of the code tensors are never
 * used in the result.  A sequence with N_b + R_b == 0 gets a row of zeros.
 * Codebooks, q and the recent rows must be finite.  Calls on one context must be
 * stream-ordered with each other (they share the context's scratch). */
int pq_attn_decode(pq_attn_ctx *ctx, const void *q, const uint8_t *k_codes, const uint8_t *v_codes,
                   const int32_t *ctx_len, const void *k_codebook, const void *v_codebook, const void *recent_k,
                   const void *recent_v, const int32_t *recent_len, float scale, float *out, void *hip_stream);

/* pq_attn_decode for callers that cannot allocate device memory — code recorded into a HIP graph, tight
 * serving loops, harnesses that forbid hipMalloc — and therefore cannot hold a context: the same kernels, the
 * same result, with every piece of scratch (codebook images, split partials, tickets) in one array that is
 * part of the library's device code (4.5 MiB per GPU the library runs on, held until the process ends).  The call allocates and
 * frees nothing and does not synchronise.
 *
 *   cfg         host; as for pq_attn_create (cfg->device names the GPU).  The code tensors use the layout
 *               of a context created from the same configuration (pq_pack_codes / pq_encode_append of such a
 *               context produce them).
 *   k_codebook, v_codebook   device [Hkv][M][256][ds] dtype, required: re-packed into the scratch by every call
 *   all other arguments as in pq_attn_decode
 *
 * Limits (PQ_ERR_CAPACITY beyond them): 8-bit codes only (4096 centroids: PQ_ERR_UNSUPPORTED); one codebook
 * tensor at most 2 MiB (32 KV heads in fp16, 16 in fp32); batch * n_q_heads <= 1024; with an explicit
 * n_splits, batch * n_q_heads * n_splits <= 1024 ("0 = choose" never exceeds it).
 * Every call on a GPU uses that GPU's one array: calls that overlap in time on one GPU (two streams, two
 * threads, or with a call still in flight) race; stream-order them.  The first call on a device looks the array's
 * address up (no allocation, but a runtime query): make that call before any stream capture starts. */
int pq_attn_decode_noalloc(const pq_attn_config *cfg /* host */, const void *q, const uint8_t *k_codes,
                           const uint8_t *v_codes, const int32_t *ctx_len, const void *k_codebook,
                           const void *v_codebook, const void *recent_k, const void *recent_v,
                           const int32_t *recent_len, float scale, float *out, void *hip_stream);

/* Quantizes n_new full-precision tokens per (sequence, KV head) and appends their
 * codes (Eq. 4 with Section II-C's nearest-centroid assignment; step 5 of Section
 * III-C): for every sub-vector the index of the centroid at the smallest squared
 * Euclidean distance; equal distances go to the lowest index.  The distance is decided
 * in IEEE double as dist = fma(x_j - c_j, x_j - c_j, dist), j = 0 .. ds-1 in order.
 *
 *   new_k/new_v device [B][Hkv][n_new][d] dtype (finite values)
 *   k_codebook / v_codebook as in pq_attn_decode
 *   k_codes / v_codes       written at token positions ctx_len[b] .. ctx_len[b]+n_new-1
 *   ctx_len     device [B] int32, incremented by n_new on the stream
 *
 * The call may run on another stream concurrently with pq_attn_decode on the same context if the
 * two are given different length arrays and the decode does not attend over the positions being
 * written (asynchronous quantization, Section III-B); the caller publishes the new lengths afterwards.
 *
 * With 12-bit codes the call stages the codes in context-owned memory sized at pq_attn_create (except for
 * 8 or fewer new tokens per KV head over all sequences, which go straight into the code tensors); a long
 * append runs as several chunks through it (more launches, no allocation, no synchronisation).  Two appends
 * on one context must not overlap.
 *
 * 0 < n_new <= max_context, else PQ_ERR_CAPACITY.  Tokens that would land beyond
 * max_context for some sequence are dropped, that sequence's length saturates, and
 * bit 0 of the device error word is set (see pq_attn_device_error). */
int pq_encode_append(pq_attn_ctx *ctx, const void *new_k, const void *new_v, int32_t n_new, const void *k_codebook,
                     const void *v_codebook, uint8_t *k_codes, uint8_t *v_codes, int32_t *ctx_len, void *hip_stream);

/* Layout conversion of code tensors (device to device, asynchronous).
 *   token_major device [B][Hkv][n_tokens][M] uint8 (uint16 for 12-bit codes), n_tokens <= max_context
 *   packed      device, pq_attn_codes_bytes()
 * pack writes tokens 0..n_tokens-1 of every head; unpack reads them. */
int pq_pack_codes(pq_attn_ctx *ctx, int32_t kind /* pq_code_kind */, const void *token_major, int32_t n_tokens,
                  uint8_t *packed, void *hip_stream);
int pq_unpack_codes(pq_attn_ctx *ctx, int32_t kind, const uint8_t *packed, int32_t n_tokens, void *token_major,
                    void *hip_stream);

/* Offline codebook training (Section II-C, training phase; Section III-A, "Offline PQ Codebook Training"):
 * k-means per (KV head, subspace) on sampled key or value vectors, n_iters iterations of Lloyd's algorithm
 * from the caller's initial centroids.  Assignment: nearest centroid by the rule and arithmetic of
 * pq_encode_append (IEEE double, ties to the lowest index).  Update: a centroid with members becomes their
 * mean — exact member sum, divided in double, rounded to float and then to fp16 — and one without keeps its
 * value.  The result does not depend on the order in which samples are processed.
 *
 *   samples    device [Hkv][n_samples][d] fp16 (finite), 1 <= n_samples <= 2^20 (else PQ_ERR_CAPACITY)
 *   codebook   device [Hkv][M][C][ds] fp16: initial centroids in, trained centroids out (in place)
 *   workspace  device, 8-byte aligned, at least pq_kmeans_workspace_bytes(ctx) bytes (else PQ_ERR_CAPACITY);
 *              contents need not be initialised and are garbage afterwards
 *
 * fp16 contexts only (PQ_ERR_UNSUPPORTED otherwise); with 12-bit codes the codebook is [Hkv][32][4096][4].  Asynchronous on the stream.  Training a codebook that
 * is registered with the context in place requires pq_attn_set_codebooks afterwards. */
int64_t pq_kmeans_workspace_bytes(const pq_attn_ctx *ctx);
int pq_kmeans_fit(pq_attn_ctx *ctx, const void *samples /* device */, int32_t n_samples, void *codebook /* device */,
                  int32_t n_iters, void *workspace /* device */, int64_t workspace_bytes, void *hip_stream);

/* Measurement aid, not part of the method: one kernel that only reads `bytes` bytes (a multiple of
 * 16, 16-byte aligned, device memory) with the load instruction the decode kernels use for codes.
 * The benchmark times it to report what HBM delivers to a pure read on the box it runs on, beside
 * the nominal peak.  Asynchronous on the stream. */
int pq_stream_read_probe(pq_attn_ctx *ctx, const void *src /* device */, int64_t bytes, void *hip_stream);

/* Synchronises the device, returns the sticky device error word in *flags and
 * clears it.  Bit 0: an append overflowed max_context. */
int pq_attn_device_error(pq_attn_ctx *ctx, uint32_t *flags /* host */);

/* ---------------------------------------------------------------------------------------------------------------
 * The paged 8-bit cache: keys and values of many requests in blocks that any request can hold, one byte a value and
 * one scale for each block and KV head.  It serves what comes before and beside the PQ cache above: prompts are
 * attended and kept in 8 bits, their tokens read back (pq_paged_read gives what pq_encode_append takes) once they
 * are to be product-quantized.
 *
 * Blocks.  n_blocks blocks of block_tokens tokens.  Sequence b holds block_table[b][0 .. ceil(len / block_tokens) - 1];
 * its token at position p is in slot block_table[b][p / block_tokens] * block_tokens + p % block_tokens.  Requests may
 * name the same blocks (a shared prefix) as long as none of them appends to a shared one and the holders are counted:
 * pq_paged_plan gives back all blocks of a request that ends.  pq_paged_fork, pq_paged_free and pq_paged_compact keep that count.
 *
 * Values.  With x the values of one KV head's tokens in a block (K and V each for itself):
 *     scale = max(max |x|, 127 * 2^-40) / 127, rounded to fp32;  code = x / scale, rounded to the nearest integer, ties
 *     to the even one (the exact quotient decides);  the value that the cache holds is code * scale.
 * An append that brings a larger |x| to a block that has tokens already raises the block's scale from s to s', and the
 * older codes c become c * s / s', rounded in the same way.  If a value is not finite, the block's scale is NaN until
 * the block is begun anew: whoever attends over one of its tokens gets NaN.
 *
 * Layout.  k_cache, v_cache: pq_paged_cache_bytes() bytes each, every byte code + 128; k_scale, v_scale float32
 * [n_blocks][Hkv].  K is [n_blocks][Hkv][block_tokens][d]; V is [n_blocks][Hkv][block_tokens / 16] pieces of 16 tokens
 * as [d / 64][token / 4 % 4][d % 16][d / 16 % 4][token % 4], so that a lane's 16 bytes are what it multiplies.
 *
 * Device tensors are 16-byte aligned, token strides (in elements) multiples of 16 bytes (PQ_ERR_SHAPE otherwise).  A
 * block number or slot outside the cache is never followed: its tokens are left out (not written, not attended over, read
 * as nothing) and bit 1 of the device error word is set.  Lengths are clamped to [0, max_blocks * block_tokens].
 * Calls on one context must be stream-ordered with each other, replays of graphs that recorded them included (they
 * share the context's scratch); one context for each stream otherwise.
 * --------------------------------------------------------------------------------------------------------------- */
typedef struct pq_paged_ctx pq_paged_ctx;

typedef struct {
    int32_t max_seqs;     /* sequences of one call at most, 1 .. 4096                         */
    int32_t max_tokens;   /* new tokens of one call at most, over all sequences, 1 .. 2^20    */
    int32_t n_q_heads;    /* Hq, 1 .. 1024; max_tokens * Hq <= 2^28                          */
    int32_t n_kv_heads;   /* Hkv, Hq % Hkv == 0; query head h reads KV head h / (Hq / Hkv)    */
    int32_t head_dim;     /* d; supported: 64, 128                                           */
    int32_t block_tokens; /* supported: 16, 32, 64                                           */
    int32_t n_blocks;     /* blocks of the cache, n_blocks * block_tokens < 2^31              */
    int32_t max_blocks;   /* row length of the block tables, max_blocks * block_tokens <= 2^24 */
    int32_t dtype;        /* pq_dtype of q, new and read K/V, and out                         */
    int32_t device;       /* HIP device ordinal                                              */
    int32_t reserved;     /* must be 0                                                       */
} pq_paged_config;

/* As pq_attn_validate_config, pq_attn_codes_bytes, pq_attn_create and pq_attn_destroy: the bytes are those of
 * k_cache, or of v_cache.  A context is destroyed after the graphs that recorded its calls (they use its scratch), and not
 * while a graph is recorded. */
int pq_paged_validate_config(const pq_paged_config *cfg /* host */);
int64_t pq_paged_cache_bytes(const pq_paged_config *cfg /* host */);
int pq_paged_create(const pq_paged_config *cfg /* host */, pq_paged_ctx **out /* host */);
int pq_paged_destroy(pq_paged_ctx *ctx);

/* Blocks and slots for the next step of n_seqs requests, from their lengths, all on the device.
 *
 *   n_new        device [n_seqs] int32    tokens that request b brings; negative: it has ended, its blocks go back
 *   n_tokens     rows of the step's tensors: at least the sum of the n_new that are not negative
 *   seq_len      device [n_seqs] int32    tokens cached now
 *   free_list    device [n_blocks] int32  a stack of free blocks, the top at free_count - 1; changed in place
 *   free_count   device [1] int32         blocks on it
 *   block_table  device [n_seqs][max_blocks] int32; new blocks are written behind those that a request has
 *   new_seq_len, new_free_count           lengths and count after the step (may be the same arrays as seq_len, free_count)
 *   tok_start    device [n_seqs + 1] int32  row of request b's first new token: the requests' tokens lie one after another
 *   tok_len      device [n_seqs] int32    new tokens that have a place: n_new, or 0
 *   slot_map     device [n_tokens] int32  slot of each new token; -1 where it has none
 *
 * First the ended requests' blocks are pushed, in the order of the requests and of their tables, and their lengths become 0.
 * Then the requests take the blocks they need from the top, in order.  A request gets all its tokens or none: none if
 * it would be longer than max_blocks * block_tokens, if its rows end behind n_tokens, or if it needs blocks and there are not
 * enough for it and all that have asked before it (those that got none for this reason included); it keeps its length
 * then, and bit 0 of the device error word is set.
 * 1 <= n_seqs <= max_seqs, 0 <= n_tokens <= max_tokens, else PQ_ERR_CAPACITY (PQ_ERR_SHAPE if below). */
int pq_paged_plan(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_tokens, const int32_t *n_new, const int32_t *seq_len,
                  int32_t *free_list, const int32_t *free_count, int32_t *block_table, int32_t *new_seq_len,
                  int32_t *new_free_count, int32_t *tok_start, int32_t *tok_len, int32_t *slot_map, void *hip_stream);

/* Quantizes n_tokens rows of keys and values into their slots.
 *
 *   new_k/new_v  device, row t at t * kv_stride elements, [Hkv][d] dtype there (kv_stride >= Hkv * d)
 *   slot_map     device [n_tokens] int32; a row with a negative slot is passed over
 *
 * The slots of one block are those of rows in a row, ascending by one, as pq_paged_plan gives them (a block that is written
 * from two places of the map, or a slot that comes twice, leaves that block's contents unspecified, no other's).  Tokens of
 * the block in front of the first such slot are older ones and are kept, those behind the last are not; a block whose slot 0 is
 * written begins anew.
 * 0 <= n_tokens <= max_tokens; 0 does nothing. */
int pq_paged_append(pq_paged_ctx *ctx, int32_t n_tokens, const void *new_k, const void *new_v, int64_t kv_stride,
                    const int32_t *slot_map, uint8_t *k_cache, uint8_t *v_cache, float *k_scale, float *v_scale,
                    void *hip_stream);

/* Tokens of the cache in full precision: row r of sequence b is its token first[b] + r.
 *
 *   n_rows       rows per sequence, 0 .. 2^24; n_seqs * Hkv * (n_rows + 8) * d <= 2^36, else PQ_ERR_CAPACITY
 *   first        device [n_seqs] int32, >= 0; NULL: all 0
 *   out_k/out_v  device [n_seqs][Hkv][n_rows][d] dtype, what pq_encode_append takes; rows behind a sequence's last
 *                token are left as they were */
int pq_paged_read(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_rows, const uint8_t *k_cache, const uint8_t *v_cache,
                  const float *k_scale, const float *v_scale, const int32_t *block_table, const int32_t *seq_len,
                  const int32_t *first, void *out_k, void *out_v, void *hip_stream);

/* Attention of one query token per sequence over all its seq_len[b] tokens (its own, appended before, among them):
 * out = sum_t softmax_t(scale * q . k_t) v_t, with scores, weights and sums of both in fp32's range.  A weight is kept in units of the
 * largest v_scale * softmax of its row, down to 2^-126 of it: with values up to 2^48 in size every token counts whose softmax
 * weight is at least 2^-45 of the largest, also one of a block of zeros (scale 2^-40).  Larger values (bf16, fp32) take from that,
 * each doubling of them a factor of 2 for the tokens of the smallest blocks.
 *
 *   q            device, row b at b * q_stride elements, [Hq][d] dtype there (q_stride >= Hq * d)
 *   scale        finite, as is its product with log2(e) in fp32: up to 2.358e38 (PQ_ERR_SHAPE otherwise)
 *   out          device [n_seqs][Hq][d] dtype; a sequence without tokens gets a row of zeros */
int pq_paged_decode(pq_paged_ctx *ctx, int32_t n_seqs, const void *q, int64_t q_stride, const uint8_t *k_cache,
                    const uint8_t *v_cache, const float *k_scale, const float *v_scale, const int32_t *block_table,
                    const int32_t *seq_len, float scale, void *out, void *hip_stream);

/* Causal attention of the tokens that a step has brought (appended before): rows tok_start[b] .. tok_start[b] +
 * tok_len[b] - 1 of q are the last tok_len[b] tokens of sequence b, and row i of them attends over the first
 * seq_len[b] - tok_len[b] + i + 1 tokens (a row for which that is not positive gets zeros).
 *
 *   n_tokens             rows of q and out, >= the end of the last sequence's rows (the kernels are chosen by what they are
 *                        on average: a call padded to many times its tokens is right, but slower, and so is one that
 *                        has long prompts and requests of few tokens over very long caches: give those a call of their own)
 *   q                    as in pq_paged_decode, row t at t * q_stride elements
 *   seq_len              lengths after the step (pq_paged_plan's new_seq_len)
 *   tok_start, tok_len   device int32, as pq_paged_plan gives them (rows from n_tokens on are left out, a sequence whose
 *                        first row is outside [0, n_tokens) altogether; rows that two sequences claim hold nobody's result,
 *                        and where the sequences claim more than n_tokens rows in all, bit 2 of the device error word is
 *                        set and none of the call's rows is to be used)
 *   out                  device [n_tokens][Hq][d] dtype; rows of no sequence are left as they were
 *
 * 0 <= n_tokens <= max_tokens; 0 does nothing. */
int pq_paged_prefill(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_tokens, const void *q, int64_t q_stride,
                     const uint8_t *k_cache, const uint8_t *v_cache, const float *k_scale, const float *v_scale,
                     const int32_t *block_table, const int32_t *seq_len, const int32_t *tok_start, const int32_t *tok_len,
                     float scale, void *out, void *hip_stream);

/* Requests that hold blocks together.  holders[x] is the number of requests that hold block x besides the first: an array
 * of n_blocks int32 that the program sets to zero once, that pq_paged_fork, pq_paged_free and pq_paged_compact keep (never
 * negative between calls; a program that keeps blocks by itself, for prompts that may come again, adds and takes away 1 likewise), and
 * that pq_paged_plan need not know: a block that it gives or takes has 0.  Requests end by pq_paged_free then: pq_paged_plan with the
 * same n_new behind it finds them empty and gives back nothing twice.
 *
 * Requests that begin as copies of others: samples of one prompt, beams, chats with the same first part.
 *
 *   parent       device [n_seqs] int32  request whose tokens request b begins with; negative, or b: request b stays as it is
 *   keep         device [n_seqs] int32  tokens it takes of them at most (negative: none); NULL: all
 *   seq_len      device [n_seqs] int32  tokens cached now; a request that becomes a fork has 0
 *   free_list, free_count, block_table  as in pq_paged_plan (the list is only read)
 *   holders      device [n_blocks] int32, changed in place
 *   new_seq_len, new_free_count         after the call (may be the same arrays as seq_len, free_count)
 *   copy_src/dst device [n_seqs] int32  the block whose contents request b needs in a block of its own; -1 where it needs none
 *
 * With n = min(seq_len[parent[b]], keep[b]) request b holds the first n / block_tokens blocks of its parent with it.  Where n is not a
 * multiple of block_tokens it takes a free block from the top of the stack, in the order of the requests, and copy_src[b], copy_dst[b]
 * say what is to be copied, in the caches of every layer (pq_paged_copy), before anything is appended.  All
 * lengths are those before the call: a fork of a request that is itself empty is empty.  A request that is not empty, whose
 * parent is not one of the n_seqs, or that finds no block free for it and all that have asked before it stays as it
 * is, and bit 0 of the device error word is set. */
int pq_paged_fork(pq_paged_ctx *ctx, int32_t n_seqs, const int32_t *parent, const int32_t *keep, const int32_t *seq_len,
                  const int32_t *free_list, const int32_t *free_count, int32_t *block_table, int32_t *holders,
                  int32_t *new_seq_len, int32_t *new_free_count, int32_t *copy_src, int32_t *copy_dst, void *hip_stream);

/* Requests that end: each takes 1 from the holders of its blocks, and those that have no holder left go onto the stack of free
 * blocks, from the highest number down (the lowest is taken first).
 *
 *   n_new        device [n_seqs] int32  negative: request b ends, as for pq_paged_plan; the others stay as they are
 *   the others   as in pq_paged_fork; free_list is changed in place, block_table only read
 *
 * A block that more requests give back than hold it goes back once, and bit 3 of the device error word is set. */
int pq_paged_free(pq_paged_ctx *ctx, int32_t n_seqs, const int32_t *n_new, const int32_t *seq_len, int32_t *free_list,
                  const int32_t *free_count, const int32_t *block_table, int32_t *holders, int32_t *new_seq_len,
                  int32_t *new_free_count, void *hip_stream);

/* Live blocks (those that are not on the stack of free ones) moved together, so that with n_live of them no number from
 * n_live on is in use: a cache of n_live blocks or more can take their place, and what is free lies in a row.  The k-th highest
 * live block at or behind n_live goes to the k-th lowest free number in front of it; the others stay.
 *
 *   n_seqs                    all requests that hold blocks
 *   seq_len, block_table, holders, free_list, free_count  as in pq_paged_fork
 *   new_block_table, new_holders, new_free_list, new_free_count  after the call (may be the same arrays as the former).  Table
 *                             entries behind a request's blocks, and list entries behind the count, are left as they were; the
 *                             list is n_blocks - 1, n_blocks - 2, .., n_live
 *   moved_to      device [n_blocks] int32  each block's new number (for what else names blocks); -1 for a free one
 *   copy_src/dst  device [n_blocks] int32, n_copies device [1] int32  the blocks that move, and how many: for pq_paged_copy in the
 *                             caches of every layer, before anything else reads or writes them by the new numbers.  Entries
 *                             behind n_copies are left as they were
 *
 * A block that is on the list twice counts once.  A table's entry that is on the list, or outside the cache, sets bit 1 of the
 * device error word; the former becomes -1. */
int pq_paged_compact(pq_paged_ctx *ctx, int32_t n_seqs, const int32_t *seq_len, const int32_t *free_list,
                     const int32_t *free_count, const int32_t *block_table, const int32_t *holders, int32_t *new_free_list,
                     int32_t *new_free_count, int32_t *new_block_table, int32_t *new_holders, int32_t *moved_to,
                     int32_t *copy_src, int32_t *copy_dst, int32_t *n_copies, void *hip_stream);

/* Contents and scales of blocks src[i] of one cache into blocks dst[i] of another, or of the same: a fork's, a compacted cache's, or
 * requests on their way to a cache elsewhere and back (host memory that the device can address will do).
 *
 *   n_pairs       entries of src and dst (device int32), 0 ..; 0 does nothing.  A pair with a negative src is passed over
 *   count         device [1] int32  pairs to be looked at, if fewer; NULL: all
 *   n_from, n_to  blocks of the two caches, which have this context's heads, dims and block_tokens (n * block_tokens < 2^31,
 *                 PQ_ERR_CAPACITY otherwise).  A number outside sets bit 1 of the device error word, and its pair copies nothing
 *
 * A block that comes twice in dst holds parts of either source; one that is in dst and, of the same cache, in src of another pair leaves
 * that pair's block unspecified (pq_paged_fork and pq_paged_compact give no such pairs). */
int pq_paged_copy(pq_paged_ctx *ctx, int32_t n_pairs, const int32_t *src, const int32_t *dst, const int32_t *count,
                  int32_t n_from, const uint8_t *from_k, const uint8_t *from_v, const float *from_k_scale,
                  const float *from_v_scale, int32_t n_to, uint8_t *to_k, uint8_t *to_v, float *to_k_scale,
                  float *to_v_scale, void *hip_stream);

/* pq_paged_decode for groups of requests that begin with the same blocks: those are read once for a group, unless
 * that costs more than it saves.  It takes two or three launches, one where tables are short (max_blocks * block_tokens up to 1280, less for
 * many requests or wide values): calls of few tokens are faster by pq_paged_decode, whatever they share.  With 32 query and 8 KV heads that is so up to
 * some 2^15 tokens, those of all requests counted (4 of 1000 tokens 7.4 us there and 9.9 here, 4 of 8192 14.9 and 16.5, of 16384 23.7
 * and 21.4), but for many requests in short tables (32 of 512 tokens 10.6 us there and 7.4 here).
 *
 *   n_groups     1 .. n_seqs (PQ_ERR_SHAPE, PQ_ERR_CAPACITY otherwise); n_seqs * ceil(Hq / Hkv / 16) * max_blocks *
 *                block_tokens < 2^35 (PQ_ERR_CAPACITY)
 *   members      device [n_seqs] int32  requests, group after group, each at most once; NULL: 0, 1, .., n_seqs - 1
 *   group_start  device [n_groups + 1] int32  group g is members[group_start[g]] .. members[group_start[g + 1] - 1] (not
 *                ascending: a group that would begin before the one in front of it begins where that does)
 *   shared_len   device [n_groups] int32  tokens that all members of a group begin with, in the same blocks.  What counts is whole
 *                blocks, and no more than the first member has: they are read by its block table, or by each member's own where that is
 *                faster.  A member that is shorter attends over its own length of them
 *   workspace    device, 16-byte aligned, at least pq_paged_shared_workspace_bytes(ctx, n_seqs, n_groups) bytes (else
 *                PQ_ERR_CAPACITY); contents need not be initialised.  Calls that may run at the same time need one each
 *   out          device [n_seqs][Hq][d] dtype; rows of requests that are in no group are left as they were
 *
 * The others as in pq_paged_decode, and so is the result; a number in members that is no request sets bit 1 of the device error
 * word.  pq_paged_shared_workspace_bytes returns a negative pq_status for sizes that the call would refuse. */
int64_t pq_paged_shared_workspace_bytes(const pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_groups);
int pq_paged_shared_decode(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_groups, const void *q, int64_t q_stride,
                           const uint8_t *k_cache, const uint8_t *v_cache, const float *k_scale, const float *v_scale,
                           const int32_t *block_table, const int32_t *seq_len, const int32_t *members,
                           const int32_t *group_start, const int32_t *shared_len, float scale, void *workspace,
                           int64_t workspace_bytes, void *out, void *hip_stream);

/* As pq_attn_device_error.  Bit 0: pq_paged_plan or pq_paged_fork refused a request; bit 1: a block number, slot or request outside
 * the cache or the call; bit 2: the sequences of a pq_paged_prefill claimed more rows than it had; bit 3: pq_paged_free gave a block back
 * more often than it was held. */
int pq_paged_device_error(pq_paged_ctx *ctx, uint32_t *flags /* host */);

/* Static, never NULL. */
const char *pq_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* PQ_ATTN_H */
