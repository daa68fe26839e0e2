// pq_paged_decode: one query token per sequence over the paged 8-bit cache.
//
// A workgroup has one sequence, the up to 16 query heads of one KV head (more go to further workgroups) and a chunk of the
// sequence's tokens; its four wavefronts share the chunk out.  Scores are S^T = K Q^T, 16 tokens by 16 query heads per matrix
// instruction: in the result a lane holds four tokens of one head, which is what the second product, O^T = V^T W, takes as its
// right operand — weights go from one to the other in registers, and a head's maximum, sum and rescaling are its lanes' own.
// The dims of K and the tokens of V may come in any order as long as both operands of a product agree: K's rows are read 16
// bytes a lane as they lie in memory, V is stored so that a lane's 16 bytes are four dims' worth of its four tokens.
// No byte passes through LDS before the end.
//
// Chunks: all of a call's chunks are about equally long, so long sequences are cut into many and the chip is evenly filled
// whatever the lengths are.  Every workgroup works the cut out for itself from the lengths.  A sequence of several
// chunks is put together by the workgroup that finishes last (pq_device_utils.h, exchange of split partials).
//
// Bound by HBM, 2 d bytes per token and KV head: 8 sequences x 32 heads x 32K tokens in fp16 336 us, 6.4 TB/s.  Short calls by
// latency: a launch, lengths, block numbers, the bytes, the merge, each a trip to memory that waits for the one before — the
// queries and the scales travel beside them (32 heads x 1000 tokens 6.6 us).
#include <hip/hip_runtime.h>

#include "pq_paged_rows16.h"

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, ROWS = 16;
constexpr int AT_ONCE = 16;             // partials of a row on their way together
constexpr int STEP = STEP_16;           // tokens a wavefront takes at a time
constexpr int CHUNK_ALIGN = WAVES * STEP;

struct chunk_place {
    int b, len;        // sequence and its length; b < 0: no chunk for this workgroup
    int first, chunks; // the sequence's first chunk in the numbering, and how many it has
    int slot;          // of its first chunk among the chunks of sequences that have several
    int tokens;        // of a chunk
};

// Chunk number c of a call.  Sequence after sequence is cut into pieces of the same length, total / budget rounded up: that
// makes at most budget + n_seqs - 1 chunks (an empty sequence has one, somebody writes its zeros), and those of sequences
// with several are at most 2 budget.
__device__ inline chunk_place find_chunk(const pq_paged_attn_args &a, int budget, int c, int lane)
{
    chunk_place p;
    p.b = -1;
    if (a.n_seqs == 1) {
        p.len = paged_length(a.c, 0);
        p.tokens = piece_tokens((float)p.len, budget, CHUNK_ALIGN, CHUNK_ALIGN);
        p.chunks = p.len > 0 ? (p.len + p.tokens - 1) / p.tokens : 1;
        p.first = p.slot = 0;
        if (c < p.chunks)
            p.b = 0;
        return p;
    }
    float total = 0.0f;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64)
        total += b0 + lane < a.n_seqs ? (float)paged_length(a.c, b0 + lane) : 0.0f;
    p.tokens = piece_tokens(wave_sum(total), budget, CHUNK_ALIGN, CHUNK_ALIGN);
    int before = 0, slots = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int len = 0, n = 0;
        if (b0 + lane < a.n_seqs) {
            len = paged_length(a.c, b0 + lane);
            n = len > 0 ? (len + p.tokens - 1) / p.tokens : 1;
        }
        const int several = n > 1 ? n : 0, upto = before + lane_scan(n), slot = slots + lane_scan(several) - several;
        const uint64_t mine = __ballot(c >= upto - n && c < upto);
        if (mine != 0) {
            const int l = __builtin_ctzll(mine);
            p.b = b0 + l;
            p.len = __builtin_amdgcn_readlane(len, l);
            p.chunks = __builtin_amdgcn_readlane(n, l);
            p.first = __builtin_amdgcn_readlane(upto - n, l);
            p.slot = __builtin_amdgcn_readlane(slot, l);
            break;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        slots = __builtin_amdgcn_readlane(slot + several, 63);
    }
    return p;
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS, 2) void pq_paged_decode_kernel(pq_paged_attn_args a, pq_paged_decode_plan w)
{
    constexpr int DT = D / 16;
    __shared__ float part[WAVES][ROWS][D + 4];
    __shared__ float wave_base[WAVES][ROWS], wave_l[WAVES][ROWS], row_base[ROWS], row_l[ROWS];
    __shared__ int last_one;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int n_groups = a.c.Hkv * w.n_sub, group = blockIdx.x % n_groups, chunk = blockIdx.x / n_groups;
    const chunk_place p = find_chunk(a, w.budget, chunk, lane);
    if (p.b < 0)
        return;
    const int h = group / w.n_sub, sub = group - h * w.n_sub;
    const int head0 = h * a.G + sub * w.sub_rows;
    const int rows = a.G - sub * w.sub_rows < w.sub_rows ? a.G - sub * w.sub_rows : w.sub_rows;
    const int col = lane & 15, quad = lane >> 4;

    // this wavefront's tokens
    const int from = (chunk - p.first) * p.tokens, upto = from + p.tokens < p.len ? from + p.tokens : p.len;
    const int share = ((upto - from + WAVES - 1) / WAVES + STEP - 1) / STEP * STEP;
    const int t0 = from + wave * share, t1 = t0 + share < upto ? t0 + share : upto;
    const int32_t *table = a.c.table + (int64_t)p.b * a.c.max_blocks;
    const int last_block = (p.len + (1 << a.c.log_block) - 1) >> a.c.log_block;

    query_16<T, D> row;
    load_query((const T *)a.q + (int64_t)p.b * a.q_stride + (int64_t)(head0 + (col < rows ? col : 0)) * D, quad, row);
    step_data<D> now;
    block_batch batch;
    batch.first = -65;
    if (t0 < t1)
        load_step<D>(a.c, table, batch, last_block, h, t0, lane, now);

    rows_16<T, D> r;
    r.take(row, a.scale_log2e);
    r.attend(a.c, table, batch, last_block, h, t0, t1, lane, now);

    // the wavefronts' parts of the chunk
    const float l = r.sum();
    if (quad == 0) {
        wave_base[wave][col] = r.base;
        wave_l[wave][col] = l;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
        *(f32x4 *)&part[wave][col][16 * i + 4 * quad] = r.o[i];
    __syncthreads();
    if (threadIdx.x < ROWS) {
        const int r = threadIdx.x;
        float top = wave_base[0][r], sum = 0.0f;
#pragma unroll
        for (int i = 1; i < WAVES; ++i)
            top = fmaxf(top, wave_base[i][r]);
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float down = __builtin_amdgcn_exp2f(wave_base[i][r] - top);
            sum = fmaf(wave_l[i][r], down, sum);
            wave_base[i][r] = down;
        }
        row_base[r] = top;
        row_l[r] = sum;
    }
    __syncthreads();
    T *const out = (T *)a.out + ((int64_t)p.b * a.Hq + head0) * D;
    const int64_t slot0 = (int64_t)group * (2 * w.budget) + p.slot;
    float *const parts = w.partials + slot0 * w.sub_rows * (D + 2);  // of the sequence's first chunk
    const int per_chunk = w.sub_rows * (D + 2);
    float *const mine = parts + (int64_t)(chunk - p.first) * per_chunk;
    for (int i = threadIdx.x; i < rows * (D / 2); i += THREADS) {
        const int r = i / (D / 2), d = i % (D / 2) * 2;
        float x = 0.0f, y = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            x = fmaf(part[k][r][d], wave_base[k][r], x);
            y = fmaf(part[k][r][d + 1], wave_base[k][r], y);
        }
        if (p.chunks == 1) {
            const float sum = row_l[r], by = sum == 0.0f ? 0.0f : 1.0f / sum;
            out[r * D + d] = paged_elem<T>::down(x * by);
            out[r * D + d + 1] = paged_elem<T>::down(y * by);
        } else {
            publish(mine + r * (D + 2) + 2 + d, x, y);
        }
    }
    if (p.chunks == 1)
        return;
    if (threadIdx.x < rows)
        publish(mine + threadIdx.x * (D + 2), row_base[threadIdx.x], row_l[threadIdx.x]);
    publish_wait();
    __syncthreads();
    unsigned int *ticket = w.tickets + slot0;
    if (threadIdx.x == 0)
        last_one = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(p.chunks - 1);
    __syncthreads();
    if (!last_one)
        return;
    if (threadIdx.x == 0)
        ticket_reset(ticket);
    for (int i = threadIdx.x; i < rows * (D / 2); i += THREADS) {
        const int r = i / (D / 2), d = i % (D / 2) * 2;
        float top = LOWEST, sum = 0.0f, x = 0.0f, y = 0.0f;
        const float *from = parts + r * (D + 2);
        for (int c0 = 0; c0 < p.chunks; c0 += AT_ONCE, from += (int64_t)AT_ONCE * per_chunk) {
            float2 ml[AT_ONCE], v[AT_ONCE];
#pragma unroll
            for (int c = 0; c < AT_ONCE; ++c) {
                const float *piece = from + (c0 + c < p.chunks ? c : 0) * per_chunk;
                ml[c] = fetch(piece);
                v[c] = fetch(piece + 2 + d);
            }
#pragma unroll
            for (int c = 0; c < AT_ONCE; ++c) {
                const float m_c = c0 + c < p.chunks ? ml[c].x : -INFINITY;  // (a repeated one counts for nothing)
                const float high = fmaxf(top, m_c), old = __builtin_amdgcn_exp2f(top - high), by = __builtin_amdgcn_exp2f(m_c - high);
                top = high;
                sum = fmaf(ml[c].y, by, sum * old);
                x = fmaf(v[c].x, by, x * old);
                y = fmaf(v[c].y, by, y * old);
            }
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        out[r * D + d] = paged_elem<T>::down(x * by);
        out[r * D + d + 1] = paged_elem<T>::down(y * by);
    }
}

}  // namespace

// Chunks are as many as keep the chip busy, PER_CU workgroups a compute unit (8 x 32 heads x 32K: 348 us with one, 336 with two,
// 342 with three; 32 query / 8 KV heads x 128K 53, 54 and 59), and not more than the last workgroup reads in a few
// microseconds (16 query heads of one KV head x 100K: 46 us with up to 128, 40 with 64; 36 since scales are not waited for).
pq_paged_decode_plan pq_paged_plan_decode(const pq_paged_config *cfg, int n_cu)
{
    constexpr int PER_CU = 2, MOST = 64;
    pq_paged_decode_plan w;
    const int G = cfg->n_q_heads / cfg->n_kv_heads;
    w.n_sub = (G + ROWS - 1) / ROWS;
    w.sub_rows = (G + w.n_sub - 1) / w.n_sub;
    w.n_sub = (G + w.sub_rows - 1) / w.sub_rows;
    const int groups = cfg->n_kv_heads * w.n_sub, wanted = PER_CU * n_cu / groups;
    w.budget = wanted < 1 ? 1 : wanted > MOST ? MOST : wanted;
    w.partials = nullptr;
    w.tickets = nullptr;
    return w;
}

int64_t pq_paged_decode_slots(const pq_paged_config *cfg, const pq_paged_decode_plan &w)
{
    return (int64_t)cfg->n_kv_heads * w.n_sub * 2 * w.budget;
}

int64_t pq_paged_decode_slot_floats(const pq_paged_config *cfg, const pq_paged_decode_plan &w)
{
    return (int64_t)w.sub_rows * (cfg->head_dim + 2);
}

hipError_t pq_launch_paged_decode(const pq_paged_ctx *ctx, const pq_paged_attn_args &a, hipStream_t s)
{
    const pq_paged_decode_plan &w = ctx->decode;
    const unsigned grid = (unsigned)(a.c.Hkv * w.n_sub) * (unsigned)(w.budget + a.n_seqs - 1);
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_decode_kernel<T, D>), dim3(grid), dim3(THREADS), 0, s, a, w)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
