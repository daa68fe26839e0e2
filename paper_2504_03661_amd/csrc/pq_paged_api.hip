// C ABI of the paged 8-bit cache: argument checks, context life cycle, launch plumbing.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <new>

#include "pq_paged.h"
#include "pq_paged_shared.h"

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

int validate(const pq_paged_config *c)
{
    if (c == nullptr)
        return PQ_ERR_NULL;
    if (c->max_seqs <= 0 || c->max_tokens <= 0 || c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 ||
        c->block_tokens <= 0 || c->n_blocks <= 0 || c->max_blocks <= 0 || c->device < 0 || c->reserved != 0)
        return PQ_ERR_SHAPE;
    if (c->n_q_heads % c->n_kv_heads != 0)
        return PQ_ERR_SHAPE;
    if (c->dtype != PQ_F16 && c->dtype != PQ_F32 && c->dtype != PQ_BF16)
        return PQ_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128)
        return PQ_ERR_UNSUPPORTED;
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64)
        return PQ_ERR_UNSUPPORTED;
    if (c->max_seqs > PQ_PAGED_MAX_SEQS || c->max_tokens > PQ_PAGED_MAX_TOKENS || c->n_q_heads > 1024)
        return PQ_ERR_UNSUPPORTED;
    // slots are int32, positions and blocks of a sequence are worked out in 32 bits
    if ((int64_t)c->n_blocks * c->block_tokens > INT32_MAX || (int64_t)c->max_blocks * c->block_tokens > PQ_MAX_TOKENS)
        return PQ_ERR_UNSUPPORTED;
    // launches have fewer than 2^32 threads: 8 for each row and head of it at most, and 2^31 for the sequences
    if ((int64_t)c->max_tokens * c->n_q_heads > (int64_t)1 << 28)
        return PQ_ERR_UNSUPPORTED;
    return PQ_OK;
}

bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }

// a row of `heads` heads at a stride of so many elements
bool stride_fits(const pq_paged_ctx *ctx, int64_t stride, int heads)
{
    const int64_t elem = ctx->cfg.dtype == PQ_F32 ? 4 : 2;
    return stride >= (int64_t)heads * ctx->cfg.head_dim && stride <= INT32_MAX && stride * elem % 16 == 0;
}

int check_seqs(const pq_paged_ctx *ctx, int32_t n_seqs)
{
    return n_seqs < 1 ? PQ_ERR_SHAPE : n_seqs > ctx->cfg.max_seqs ? PQ_ERR_CAPACITY : PQ_OK;
}

int check_tokens(const pq_paged_ctx *ctx, int32_t n_tokens)
{
    return n_tokens < 0 ? PQ_ERR_SHAPE : n_tokens > ctx->cfg.max_tokens ? PQ_ERR_CAPACITY : PQ_OK;
}

int check_groups(const pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_groups)
{
    const int rc = check_seqs(ctx, n_seqs);
    if (rc != PQ_OK || n_groups < 1)
        return rc != PQ_OK ? rc : PQ_ERR_SHAPE;
    // steps of 32 tokens for up to 16 query heads of a KV head are numbered in 30 bits
    const int64_t tiles = (ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads + 15) / 16, width = (int64_t)ctx->cfg.max_blocks << ctx->log_block;
    return n_groups > n_seqs || n_seqs * tiles * width >= (int64_t)1 << 35 ? PQ_ERR_CAPACITY : PQ_OK;
}

int check_attention(const pq_paged_ctx *ctx, const void *q, int64_t q_stride, const uint8_t *k, const uint8_t *v, float scale, const void *out)
{
    if (!aligned(q) || !aligned(out) || !aligned(k) || !aligned(v) || !stride_fits(ctx, q_stride, ctx->cfg.n_q_heads))
        return PQ_ERR_SHAPE;
    return fabsf(scale * LOG2E) <= FLT_MAX ? PQ_OK : PQ_ERR_SHAPE;  // NaN or infinite, or so in what the kernels multiply by
}

pq_paged_view view(const pq_paged_ctx *ctx, const uint8_t *k, const uint8_t *v, const float *k_scale, const float *v_scale,
                   const int32_t *table, const int32_t *seq_len)
{
    pq_paged_view c;
    c.k = k;
    c.v = v;
    c.k_scale = k_scale;
    c.v_scale = v_scale;
    c.table = table;
    c.seq_len = seq_len;
    c.n_blocks = ctx->cfg.n_blocks;
    c.max_blocks = ctx->cfg.max_blocks;
    c.log_block = ctx->log_block;
    c.Hkv = ctx->cfg.n_kv_heads;
    c.dev_err = ctx->dev_err;
    return c;
}

void free_ctx(pq_paged_ctx *ctx)
{
    (void)hipFree(ctx->scratch);
    delete ctx;
}

int attend(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_tokens, const void *q, int64_t q_stride, const pq_paged_view &c,
           const int32_t *tok_start, const int32_t *tok_len, float scale, void *out, void *hip_stream)
{
    const int rc = check_attention(ctx, q, q_stride, c.k, c.v, scale, out);
    if (rc != PQ_OK)
        return rc;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_attn_args a;
    a.c = c;
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.tok_start = tok_start;
    a.tok_len = tok_len;
    a.scale_log2e = scale * LOG2E;
    a.n_seqs = n_seqs;
    a.n_tokens = n_tokens;
    a.Hq = ctx->cfg.n_q_heads;
    a.G = ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads;
    const hipError_t e = tok_start == nullptr ? pq_launch_paged_decode(ctx, a, (hipStream_t)hip_stream)
                                              : pq_launch_paged_prefill(ctx, a, (hipStream_t)hip_stream);
    return e == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

}  // namespace

extern "C" {

int pq_paged_validate_config(const pq_paged_config *cfg) { return validate(cfg); }

int64_t pq_paged_cache_bytes(const pq_paged_config *cfg)
{
    const int rc = validate(cfg);
    if (rc != PQ_OK)
        return rc;
    return (int64_t)cfg->n_blocks * cfg->n_kv_heads * cfg->block_tokens * cfg->head_dim;
}

int pq_paged_create(const pq_paged_config *cfg, pq_paged_ctx **out)
{
    if (out == nullptr)
        return PQ_ERR_NULL;
    const int rc = validate(cfg);
    if (rc != PQ_OK)
        return rc;
    int n_dev = 0;
    if (hipGetDeviceCount(&n_dev) != hipSuccess || cfg->device >= n_dev) {
        (void)hipGetLastError();
        return PQ_ERR_HIP;
    }
    device_guard guard(cfg->device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    int n_cu = 0;
    if (hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, cfg->device) != hipSuccess || n_cu <= 0)
        return PQ_ERR_HIP;
    pq_paged_ctx *ctx = new (std::nothrow) pq_paged_ctx();
    if (ctx == nullptr)
        return PQ_ERR_ALLOC;
    ctx->cfg = *cfg;
    ctx->log_block = cfg->block_tokens == 16 ? 4 : cfg->block_tokens == 32 ? 5 : 6;
    ctx->n_cu = n_cu;
    ctx->decode = pq_paged_plan_decode(cfg, n_cu);
    ctx->prefill = pq_paged_plan_prefill(cfg, n_cu);
    // one allocation: what has to be zero first, then the rest
    const int64_t slots = pq_paged_decode_slots(cfg, ctx->decode);
    size_t bytes = 0;
    const auto room = [&](size_t n) { const size_t at = bytes; bytes += (n + 255) / 256 * 256; return at; };
    const size_t err_at = room(sizeof(unsigned int)), tickets_at = room(slots * sizeof(unsigned int));
    const size_t zeros = bytes;
    const int64_t of_plan = pq_paged_plan_scratch_bytes(), of_blocks = pq_paged_blocks_scratch_bytes();
    const size_t plan_at = room((size_t)(of_plan > of_blocks ? of_plan : of_blocks));
    const size_t decode_at = room((size_t)slots * pq_paged_decode_slot_floats(cfg, ctx->decode) * sizeof(float));
    const size_t prefill_at = room((size_t)pq_paged_prefill_floats(cfg, ctx->prefill) * sizeof(float));
    if (hipMalloc((void **)&ctx->scratch, bytes) != hipSuccess) {
        (void)hipGetLastError();
        delete ctx;
        return PQ_ERR_ALLOC;
    }
    ctx->dev_err = (unsigned int *)(ctx->scratch + err_at);
    ctx->decode.tickets = (unsigned int *)(ctx->scratch + tickets_at);
    ctx->plan = (int *)(ctx->scratch + plan_at);
    ctx->decode.partials = (float *)(ctx->scratch + decode_at);
    ctx->prefill.partials = (float *)(ctx->scratch + prefill_at);
    if (hipMemset(ctx->scratch, 0, zeros) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
        (void)hipGetLastError();
        free_ctx(ctx);
        return PQ_ERR_HIP;
    }
    *out = ctx;
    return PQ_OK;
}

int pq_paged_destroy(pq_paged_ctx *ctx)
{
    if (ctx == nullptr)
        return PQ_ERR_NULL;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    const bool ok = hipDeviceSynchronize() == hipSuccess;
    free_ctx(ctx);
    return ok ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_plan(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_tokens, const int32_t *n_new, const int32_t *seq_len,
                  int32_t *free_list, const int32_t *free_count, int32_t *block_table, int32_t *new_seq_len,
                  int32_t *new_free_count, int32_t *tok_start, int32_t *tok_len, int32_t *slot_map, void *hip_stream)
{
    if (ctx == nullptr || n_new == nullptr || seq_len == nullptr || free_list == nullptr || free_count == nullptr ||
        block_table == nullptr || new_seq_len == nullptr || new_free_count == nullptr || tok_start == nullptr ||
        tok_len == nullptr || (slot_map == nullptr && n_tokens != 0))
        return PQ_ERR_NULL;
    int rc = check_seqs(ctx, n_seqs);
    rc = rc == PQ_OK ? check_tokens(ctx, n_tokens) : rc;
    if (rc != PQ_OK)
        return rc;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_plan_args a;
    a.n_new = n_new;
    a.seq_len = seq_len;
    a.free_list = free_list;
    a.free_count = free_count;
    a.table = block_table;
    a.new_seq_len = new_seq_len;
    a.new_free_count = new_free_count;
    a.tok_start = tok_start;
    a.tok_len = tok_len;
    a.slot_map = slot_map;
    a.scratch = ctx->plan;
    a.n_seqs = n_seqs;
    a.n_tokens = n_tokens;
    a.n_blocks = ctx->cfg.n_blocks;
    a.max_blocks = ctx->cfg.max_blocks;
    a.log_block = ctx->log_block;
    a.dev_err = ctx->dev_err;
    return pq_launch_paged_plan(ctx, a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_append(pq_paged_ctx *ctx, int32_t n_tokens, const void *new_k, const void *new_v, int64_t kv_stride,
                    const int32_t *slot_map, uint8_t *k_cache, uint8_t *v_cache, float *k_scale, float *v_scale,
                    void *hip_stream)
{
    if (ctx == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr || v_scale == nullptr)
        return PQ_ERR_NULL;
    if (n_tokens != 0 && (new_k == nullptr || new_v == nullptr || slot_map == nullptr))
        return PQ_ERR_NULL;
    const int rc = check_tokens(ctx, n_tokens);
    if (rc != PQ_OK)
        return rc;
    if (!aligned(new_k) || !aligned(new_v) || !aligned(k_cache) || !aligned(v_cache) ||
        !stride_fits(ctx, kv_stride, ctx->cfg.n_kv_heads))
        return PQ_ERR_SHAPE;
    if (n_tokens == 0)
        return PQ_OK;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_append_args a;
    a.x[0] = new_k;
    a.x[1] = new_v;
    a.cache[0] = k_cache;
    a.cache[1] = v_cache;
    a.scale[0] = k_scale;
    a.scale[1] = v_scale;
    a.slot = slot_map;
    a.stride = kv_stride;
    a.n_tokens = n_tokens;
    a.n_blocks = ctx->cfg.n_blocks;
    a.log_block = ctx->log_block;
    a.Hkv = ctx->cfg.n_kv_heads;
    a.dev_err = ctx->dev_err;
    return pq_launch_paged_append(ctx, a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_read(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_rows, const uint8_t *k_cache, const uint8_t *v_cache,
                  const float *k_scale, const float *v_scale, const int32_t *block_table, const int32_t *seq_len,
                  const int32_t *first, void *out_k, void *out_v, void *hip_stream)
{
    if (ctx == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr || v_scale == nullptr ||
        block_table == nullptr || seq_len == nullptr || (n_rows != 0 && (out_k == nullptr || out_v == nullptr)))
        return PQ_ERR_NULL;
    const int rc = check_seqs(ctx, n_seqs);
    if (rc != PQ_OK)
        return rc;
    if (n_rows < 0 || !aligned(k_cache) || !aligned(v_cache) || !aligned(out_k) || !aligned(out_v))
        return PQ_ERR_SHAPE;
    if (n_rows > PQ_MAX_TOKENS || (int64_t)n_seqs * ctx->cfg.n_kv_heads * (n_rows + 8) * ctx->cfg.head_dim > (int64_t)1 << 36)
        return PQ_ERR_CAPACITY;  // (a thread has 32 elements)
    if (n_rows == 0)
        return PQ_OK;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_read_args a;
    a.c = view(ctx, k_cache, v_cache, k_scale, v_scale, block_table, seq_len);
    a.first = first;
    a.out[0] = out_k;
    a.out[1] = out_v;
    a.n_seqs = n_seqs;
    a.n_rows = n_rows;
    return pq_launch_paged_read(ctx, a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_decode(pq_paged_ctx *ctx, int32_t n_seqs, const void *q, int64_t q_stride, const uint8_t *k_cache,
                    const uint8_t *v_cache, const float *k_scale, const float *v_scale, const int32_t *block_table,
                    const int32_t *seq_len, float scale, void *out, void *hip_stream)
{
    if (ctx == nullptr || q == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr ||
        v_scale == nullptr || block_table == nullptr || seq_len == nullptr || out == nullptr)
        return PQ_ERR_NULL;
    const int rc = check_seqs(ctx, n_seqs);
    if (rc != PQ_OK)
        return rc;
    return attend(ctx, n_seqs, n_seqs, q, q_stride, view(ctx, k_cache, v_cache, k_scale, v_scale, block_table, seq_len),
                  nullptr, nullptr, scale, out, hip_stream);
}

int pq_paged_prefill(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_tokens, const void *q, int64_t q_stride,
                     const uint8_t *k_cache, const uint8_t *v_cache, const float *k_scale, const float *v_scale,
                     const int32_t *block_table, const int32_t *seq_len, const int32_t *tok_start, const int32_t *tok_len,
                     float scale, void *out, void *hip_stream)
{
    if (ctx == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr || v_scale == nullptr ||
        block_table == nullptr || seq_len == nullptr || tok_start == nullptr || tok_len == nullptr ||
        (n_tokens != 0 && (q == nullptr || out == nullptr)))
        return PQ_ERR_NULL;
    int rc = check_seqs(ctx, n_seqs);
    rc = rc == PQ_OK ? check_tokens(ctx, n_tokens) : rc;
    if (rc != PQ_OK)
        return rc;
    if (n_tokens == 0)
        return PQ_OK;
    return attend(ctx, n_seqs, n_tokens, q, q_stride, view(ctx, k_cache, v_cache, k_scale, v_scale, block_table, seq_len),
                  tok_start, tok_len, scale, out, hip_stream);
}

int pq_paged_fork(pq_paged_ctx *ctx, int32_t n_seqs, const int32_t *parent, const int32_t *keep, const int32_t *seq_len,
                  const int32_t *free_list, const int32_t *free_count, int32_t *block_table, int32_t *holders,
                  int32_t *new_seq_len, int32_t *new_free_count, int32_t *copy_src, int32_t *copy_dst, void *hip_stream)
{
    if (ctx == nullptr || parent == nullptr || seq_len == nullptr || free_list == nullptr || free_count == nullptr ||
        block_table == nullptr || holders == nullptr || new_seq_len == nullptr || new_free_count == nullptr ||
        copy_src == nullptr || copy_dst == nullptr)
        return PQ_ERR_NULL;
    const int rc = check_seqs(ctx, n_seqs);
    if (rc != PQ_OK)
        return rc;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_fork_args a;
    a.parent = parent;
    a.keep = keep;
    a.seq_len = seq_len;
    a.free_list = free_list;
    a.free_count = free_count;
    a.table = block_table;
    a.holders = holders;
    a.new_seq_len = new_seq_len;
    a.new_free_count = new_free_count;
    a.copy_src = copy_src;
    a.copy_dst = copy_dst;
    a.scratch = ctx->plan;
    a.n_seqs = n_seqs;
    a.n_blocks = ctx->cfg.n_blocks;
    a.max_blocks = ctx->cfg.max_blocks;
    a.log_block = ctx->log_block;
    a.dev_err = ctx->dev_err;
    return pq_launch_paged_fork(a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_free(pq_paged_ctx *ctx, int32_t n_seqs, const int32_t *n_new, const int32_t *seq_len, int32_t *free_list,
                  const int32_t *free_count, const int32_t *block_table, int32_t *holders, int32_t *new_seq_len,
                  int32_t *new_free_count, void *hip_stream)
{
    if (ctx == nullptr || n_new == nullptr || seq_len == nullptr || free_list == nullptr || free_count == nullptr ||
        block_table == nullptr || holders == nullptr || new_seq_len == nullptr || new_free_count == nullptr)
        return PQ_ERR_NULL;
    const int rc = check_seqs(ctx, n_seqs);
    if (rc != PQ_OK)
        return rc;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_free_args a;
    a.n_new = n_new;
    a.seq_len = seq_len;
    a.free_list = free_list;
    a.free_count = free_count;
    a.table = block_table;
    a.holders = holders;
    a.new_seq_len = new_seq_len;
    a.new_free_count = new_free_count;
    a.scratch = ctx->plan;
    a.n_seqs = n_seqs;
    a.n_blocks = ctx->cfg.n_blocks;
    a.max_blocks = ctx->cfg.max_blocks;
    a.log_block = ctx->log_block;
    a.dev_err = ctx->dev_err;
    return pq_launch_paged_free(a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_compact(pq_paged_ctx *ctx, int32_t n_seqs, const int32_t *seq_len, const int32_t *free_list,
                     const int32_t *free_count, const int32_t *block_table, const int32_t *holders, int32_t *new_free_list,
                     int32_t *new_free_count, int32_t *new_block_table, int32_t *new_holders, int32_t *moved_to,
                     int32_t *copy_src, int32_t *copy_dst, int32_t *n_copies, void *hip_stream)
{
    if (ctx == nullptr || seq_len == nullptr || free_list == nullptr || free_count == nullptr || block_table == nullptr ||
        holders == nullptr || new_free_list == nullptr || new_free_count == nullptr || new_block_table == nullptr ||
        new_holders == nullptr || moved_to == nullptr || copy_src == nullptr || copy_dst == nullptr || n_copies == nullptr)
        return PQ_ERR_NULL;
    const int rc = check_seqs(ctx, n_seqs);
    if (rc != PQ_OK)
        return rc;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_compact_args a;
    a.seq_len = seq_len;
    a.free_list = free_list;
    a.free_count = free_count;
    a.table = block_table;
    a.holders = holders;
    a.new_free_list = new_free_list;
    a.new_free_count = new_free_count;
    a.new_table = new_block_table;
    a.new_holders = new_holders;
    a.moved_to = moved_to;
    a.copy_src = copy_src;
    a.copy_dst = copy_dst;
    a.n_copies = n_copies;
    a.scratch = ctx->plan;
    a.n_seqs = n_seqs;
    a.n_blocks = ctx->cfg.n_blocks;
    a.max_blocks = ctx->cfg.max_blocks;
    a.log_block = ctx->log_block;
    a.dev_err = ctx->dev_err;
    return pq_launch_paged_compact(a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_copy(pq_paged_ctx *ctx, int32_t n_pairs, const int32_t *src, const int32_t *dst, const int32_t *count,
                  int32_t n_from, const uint8_t *from_k, const uint8_t *from_v, const float *from_k_scale,
                  const float *from_v_scale, int32_t n_to, uint8_t *to_k, uint8_t *to_v, float *to_k_scale,
                  float *to_v_scale, void *hip_stream)
{
    if (ctx == nullptr || from_k == nullptr || from_v == nullptr || from_k_scale == nullptr || from_v_scale == nullptr ||
        to_k == nullptr || to_v == nullptr || to_k_scale == nullptr || to_v_scale == nullptr ||
        (n_pairs != 0 && (src == nullptr || dst == nullptr)))
        return PQ_ERR_NULL;
    if (n_pairs < 0 || n_from < 1 || n_to < 1 || !aligned(from_k) || !aligned(from_v) || !aligned(to_k) || !aligned(to_v))
        return PQ_ERR_SHAPE;
    if (n_pairs > INT32_MAX / ctx->cfg.block_tokens || n_from > INT32_MAX / ctx->cfg.block_tokens ||
        n_to > INT32_MAX / ctx->cfg.block_tokens)
        return PQ_ERR_CAPACITY;
    if (n_pairs == 0)
        return PQ_OK;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    pq_paged_copy_args a;
    a.src = src;
    a.dst = dst;
    a.count = count;
    a.from[0] = from_k;
    a.from[1] = from_v;
    a.from_scale[0] = from_k_scale;
    a.from_scale[1] = from_v_scale;
    a.to[0] = to_k;
    a.to[1] = to_v;
    a.to_scale[0] = to_k_scale;
    a.to_scale[1] = to_v_scale;
    a.block_bytes = (int64_t)ctx->cfg.n_kv_heads * ctx->cfg.block_tokens * ctx->cfg.head_dim;
    a.n_pairs = n_pairs;
    a.n_from = n_from;
    a.n_to = n_to;
    a.Hkv = ctx->cfg.n_kv_heads;
    a.dev_err = ctx->dev_err;
    return pq_launch_paged_copy(a, ctx->n_cu, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int64_t pq_paged_shared_workspace_bytes(const pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_groups)
{
    if (ctx == nullptr)
        return PQ_ERR_NULL;
    const int rc = check_groups(ctx, n_seqs, n_groups);
    return rc != PQ_OK ? rc : pq_paged_shared_layout(ctx, n_seqs, n_groups, nullptr, nullptr);
}

int pq_paged_shared_decode(pq_paged_ctx *ctx, int32_t n_seqs, int32_t n_groups, const void *q, int64_t q_stride,
                           const uint8_t *k_cache, const uint8_t *v_cache, const float *k_scale, const float *v_scale,
                           const int32_t *block_table, const int32_t *seq_len, const int32_t *members,
                           const int32_t *group_start, const int32_t *shared_len, float scale, void *workspace,
                           int64_t workspace_bytes, void *out, void *hip_stream)
{
    if (ctx == nullptr || q == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr ||
        v_scale == nullptr || block_table == nullptr || seq_len == nullptr || group_start == nullptr ||
        shared_len == nullptr || workspace == nullptr || out == nullptr)
        return PQ_ERR_NULL;
    int rc = check_groups(ctx, n_seqs, n_groups);
    rc = rc == PQ_OK ? check_attention(ctx, q, q_stride, k_cache, v_cache, scale, out) : rc;
    if (rc != PQ_OK)
        return rc;
    if (!aligned(workspace))
        return PQ_ERR_SHAPE;
    pq_paged_shared_args a;
    if (workspace_bytes < pq_paged_shared_layout(ctx, n_seqs, n_groups, workspace, &a))
        return PQ_ERR_CAPACITY;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    a.c = view(ctx, k_cache, v_cache, k_scale, v_scale, block_table, seq_len);
    a.q = q;
    a.out = out;
    a.q_stride = q_stride;
    a.members = members;
    a.group_start = group_start;
    a.shared_len = shared_len;
    a.scale_log2e = scale * LOG2E;
    a.n_seqs = n_seqs;
    a.n_groups = n_groups;
    a.Hq = ctx->cfg.n_q_heads;
    a.G = ctx->cfg.n_q_heads / ctx->cfg.n_kv_heads;
    return pq_launch_paged_shared(ctx, a, (hipStream_t)hip_stream) == hipSuccess ? PQ_OK : PQ_ERR_HIP;
}

int pq_paged_device_error(pq_paged_ctx *ctx, uint32_t *flags)
{
    if (ctx == nullptr || flags == nullptr)
        return PQ_ERR_NULL;
    device_guard guard(ctx->cfg.device);
    if (!guard.ok)
        return PQ_ERR_HIP;
    unsigned int v = 0;
    if (hipDeviceSynchronize() != hipSuccess)
        return PQ_ERR_HIP;
    if (hipMemcpy(&v, ctx->dev_err, sizeof(v), hipMemcpyDeviceToHost) != hipSuccess)
        return PQ_ERR_HIP;
    if (v != 0 && hipMemset(ctx->dev_err, 0, sizeof(v)) != hipSuccess)
        return PQ_ERR_HIP;
    *flags = v;
    return PQ_OK;
}

}  // extern "C"
