// pq_paged_prefill's other kernel, for sequences that bring few tokens — chunks, guessed tokens, the odd step among prompts — and
// for calls that are small as a whole.  And the merge of its pieces, and the launches.
//
// A workgroup has 32 rows (a token's query heads of a KV head side by side) and a piece of the keys that they see, of which each
// of its four wavefronts takes a part, as pq_paged_decode's do: bytes go from memory to the lanes that multiply them, with
// no LDS between.  The products are those of the kernel for many rows, 32x32x16, with K's dims in the order that 16-byte loads
// bring them and V's dims in that of its 16-byte words.
//
// Bound by latency and the merge where the work is small (12 tokens, 32 query / 8 KV heads, over 20K keys: 24 us for 41 MB), then by
// the conversion of bytes, which every tile of 32 rows does for itself: 1000 tokens over 8K keys 195 us, 663 TFLOP/s.
#include <hip/hip_runtime.h>

#include "pq_paged_work.h"

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, ROWS = PQ_PAGED_FEW_ROWS, STEP = 32;

// 32 keys as they lie in memory, and their blocks' scales
template <int D> struct step_bytes {
    u32x4 k[D / 32];
    uint32_t v[2][2][D / 32];  // [piece of 16 tokens][token quad half, half + 2][product]
    float k_scale[2], v_log[2], v_inv[2];
};

template <int D>
__device__ inline void load_bytes(const pq_paged_view &c, const int32_t *table, block_batch &batch, int last_block, int h, int t, int lane,
                                  step_bytes<D> &s)
{
    const int col = lane & 31, half = lane >> 5;
    // (t is a multiple of 32: both pieces are in one batch)
    const bool anew = (t >> c.log_block) >= batch.first + 64;
    if (anew)
        start_batch(c, table, t >> c.log_block, last_block, h, lane, batch);
    int at[2];
    int64_t base[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = t + 16 * i;
        at[i] = (p >> c.log_block) - batch.first;
        const int id = __builtin_amdgcn_readlane(batch.id, at[i]);
        base[i] = (((int64_t)id * c.Hkv + h) << c.log_block) * D + (p & ((1 << c.log_block) - 1)) * D;
    }
    const uint8_t *k = c.k + (col < 16 ? base[0] : base[1]) + (col & 15) * D + 16 * half;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
        s.k[x] = *(const u32x4 *)(k + 32 * x);
    // 128 dims: a lane's row is dim 64 (col / 16) + 16 k + col % 16 in product k, the four of a 16-byte word; 64 dims: 32 (col / 16)
    // + 16 k + col % 16, half a word
    const int v_at = (D == 128 ? (col >> 4) * 1024 : (col >> 4) * 8) + (col & 15) * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint8_t *v = c.v + base[i] + v_at + (half + 2 * q) * 256;
            if constexpr (D == 128) {
                const u32x4 w = *(const u32x4 *)v;
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    s.v[i][q][x] = w[x];
            } else {
                const u32x2 w = *(const u32x2 *)v;
                s.v[i][q][0] = w[0];
                s.v[i][q][1] = w[1];
            }
        }
    if (anew)
        finish_batch(batch);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        s.k_scale[i] = lane_of(batch.k_scale, at[i]);
        s.v_log[i] = lane_of(batch.v_log, at[i]);
        s.v_inv[i] = lane_of(batch.v_inv, at[i]);
    }
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS, sizeof(T) == 4 ? 1 : 2) void pq_paged_few_kernel(pq_paged_attn_args a, pq_paged_prefill_plan w)
{
    constexpr bool SPLIT = sizeof(T) == 4;  // two fp16 parts of queries and weights
    constexpr int PARTS = SPLIT ? 2 : 1, DT = D / 32;
    __shared__ float part[WAVES][ROWS][D + 4];
    __shared__ float wave_base[WAVES][ROWS], wave_l[WAVES][ROWS], row_base[ROWS], row_l[ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int h = blockIdx.x % a.c.Hkv, entry = blockIdx.x / a.c.Hkv;
    if (blockIdx.x == gridDim.x - 1) {  // (one more than the list has)
        if (wave == 0)
            check_claims(a, lane);
        return;
    }
    work_place p;
    if (!find_work(a, few_rule(w), entry, lane, p))
        return;
    const tile_place tile(p, a.G, ROWS);
    if (p.split >= tile.pieces)
        return;
    const int k0 = p.split * p.keys, k1 = k0 + p.keys < tile.sees ? k0 + p.keys : tile.sees;
    const int share = ((k1 - k0 + WAVES - 1) / WAVES + STEP - 1) / STEP * STEP;
    const int t0 = k0 + wave * share, t1 = t0 + share < k1 ? t0 + share : k1;
    const int32_t *table = a.c.table + (int64_t)p.b * a.c.max_blocks;
    const int last_block = (p.len + (1 << a.c.log_block) - 1) >> a.c.log_block;
    step_bytes<D> now, next;
    block_batch batch;
    batch.first = -65;
    if (t0 < t1)
        load_bytes<D>(a.c, table, batch, last_block, h, t0, lane, now);

    const int col = lane & 31, half = lane >> 5;
    const bool there = col < tile.rows;
    const int token = there ? (tile.row0 + col) / a.G : 0, head = there ? tile.row0 + col - token * a.G : 0;
    int sees = there ? p.past + token + 1 : 0;
    sees = sees < t1 ? sees : t1;
    const int least = __builtin_amdgcn_readfirstlane(tile.rows == ROWS ? p.past + tile.row0 / a.G + 1 : 0);  // (of the first row)
    half8v q[PARTS][D / 16];
    float per_score;
    {
        // dims 32 x + 16 half + 0 .. 15 of the row, as K's loads bring them
        float v[D / 2];
        float high = 0.0f;
        const T *src = (const T *)a.q + (int64_t)(p.first_row + token) * a.q_stride + (int64_t)(h * a.G + head) * D + 16 * half;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            paged_load8(src + 32 * x, v + 16 * x);
            paged_load8(src + 32 * x + 8, v + 16 * x + 8);
        }
#pragma unroll
        for (int i = 0; i < D / 2; ++i)
            high = fmaxf(high, fabsf(v[i]));
        high = fmaxf(high, __shfl_xor(high, 32, 64));
        const int e = query_exponent(high);
        per_score = ldexpf(a.scale_log2e, -e);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = ldexpf(v[8 * x + j], e);
                q[0][x][j] = (_Float16)f;
                if (SPLIT)
                    q[PARTS - 1][x][j] = (_Float16)(f - (float)q[0][x][j]);
            }
    }

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j)
            o[i][j] = 0.0f;
    float base = LOWEST, l = 0.0f;
    for (int t = t0; t < t1; t += STEP) {
        const bool more = t + STEP < t1;
        if (more)
            load_bytes<D>(a.c, table, batch, last_block, h, t + STEP, lane, next);
        f32x16 dot;
#pragma unroll
        for (int j = 0; j < 16; ++j)
            dot[j] = 0.0f;
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            const half8v k = codes8(now.k[x >> 1][2 * (x & 1)], now.k[x >> 1][2 * (x & 1) + 1]);
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
                dot = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[i][x], dot, 0, 0, 0);
        }
        float s[16];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float by = per_score * now.k_scale[i];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                s[8 * i + j] = fmaf(dot[8 * i + j], by, now.v_log[i]);
        }
        if (t + STEP > least || t + STEP > t1)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (t + 8 * (j >> 2) + 4 * half + (j & 3) >= sees)
                    s[j] = -INFINITY;
        float high = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j)
            high = fmaxf(high, s[j]);
        if (__ballot(high - base > MOST_BITS) != 0) {
            high = fmaxf(high, __shfl_xor(high, 32, 64));
            const float moved = fmaxf(base, weight_base(high)), down = __builtin_amdgcn_exp2f(base - moved);
            base = moved;
            l *= down;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    o[i][j] *= down;
        }
        half8v weights[PARTS][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = __builtin_amdgcn_exp2f(s[8 * i + j] - base);
                sum += x;
                weights[0][i][j] = (_Float16)x;
                if (SPLIT)
                    weights[PARTS - 1][i][j] = (_Float16)(x - (float)weights[0][i][j]);
            }
            l = fmaf(sum, now.v_inv[i], l);
        }
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const half8v v = codes8(now.v[x][0][i], now.v[x][1][i]);
#pragma unroll
                for (int j = 0; j < PARTS; ++j)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, weights[j][x], o[i], 0, 0, 0);
            }
        if (more)
            now = next;
    }

    // the wavefronts' parts
    l += __shfl_xor(l, 32, 64);
    if (half == 0) {
        wave_base[wave][col] = base;
        wave_l[wave][col] = l;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            const int d = (D == 128 ? 64 * (j >> 3) + 16 * i : 32 * (j >> 3) + 16 * i) + 8 * ((j >> 2) & 1) + 4 * half;
            *(f32x4 *)&part[wave][col][d] = f32x4{o[i][j], o[i][j + 1], o[i][j + 2], o[i][j + 3]};
        }
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
    float *const to = w.partials + ((int64_t)h * (2 * w.budget) + p.slot + p.split) * (ROWS * (D + 2));
    for (int i = threadIdx.x; i < tile.rows * (D / 2); i += THREADS) {
        const int r = i / (D / 2), d = i % (D / 2) * 2;
        float x = 0.0f, y = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            x = fmaf(part[k][r][d], wave_base[k][r], x);
            y = fmaf(part[k][r][d + 1], wave_base[k][r], y);
        }
        if (tile.pieces == 1) {
            const float by = row_l[r] == 0.0f ? 0.0f : 1.0f / row_l[r];
            const int row = tile.row0 + r, t = row / a.G;
            T *out = (T *)a.out + ((int64_t)(p.first_row + t) * a.Hq + h * a.G + (row - t * a.G)) * D + d;
            out[0] = paged_elem<T>::down(x * by);
            out[1] = paged_elem<T>::down(y * by);
        } else {
            *(float2 *)(to + r * (D + 2) + 2 + d) = make_float2(x, y);
            if (d == 0)
                *(float2 *)(to + r * (D + 2)) = make_float2(row_base[r], row_l[r]);
        }
    }
}

constexpr int MERGE_WAVES = 4, MERGE_GROUPS = ROWS / MERGE_WAVES;  // workgroups of a tile, a wavefront has one row

// Puts the pieces of a tile's keys together, two dims a lane.
template <typename T, int D>
__global__ __launch_bounds__(64 * MERGE_WAVES) void pq_paged_merge_kernel(pq_paged_attn_args a, pq_paged_prefill_plan w)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int group = blockIdx.x % MERGE_GROUPS, h = blockIdx.x / MERGE_GROUPS % a.c.Hkv;
    work_place p;
    if (!find_work<true>(a, few_rule(w), blockIdx.x / MERGE_GROUPS / a.c.Hkv, lane, p))
        return;
    const tile_place tile(p, a.G, ROWS);
    constexpr int64_t stride = ROWS * (D + 2);
    if (tile.pieces == 1)
        return;
    const int d = 2 * (lane % (D / 2)), r = group * MERGE_WAVES + wave;
    if (r < tile.rows) {
        const float *from = w.partials + ((int64_t)h * (2 * w.budget) + p.slot) * stride + r * (D + 2);
        float top = LOWEST, sum = 0.0f, x = 0.0f, y = 0.0f;
        for (int c0 = 0; c0 < tile.pieces; c0 += 64, from += 64 * stride) {
            // a lane has a piece's base and sum, and so its weight; one that is not there has the weight 0
            const int n = tile.pieces - c0 < 64 ? tile.pieces - c0 : 64;
            const float2 ml = lane < n ? *(const float2 *)(from + lane * stride) : make_float2(-INFINITY, 0.0f);
            const float high = fmaxf(top, wave_max(ml.x)), old = __builtin_amdgcn_exp2f(top - high), by = __builtin_amdgcn_exp2f(ml.x - high);
            top = high;
            sum = fmaf(sum, old, wave_sum(ml.y * by));
            x *= old;
            y *= old;
            constexpr int AT_ONCE = 16;  // loads on their way together
            for (int c1 = 0; c1 < n; c1 += AT_ONCE) {
                float2 v[AT_ONCE];
#pragma unroll
                for (int c = 0; c < AT_ONCE; ++c)
                    v[c] = *(const float2 *)(from + (c1 + c < n ? c1 + c : 0) * stride + 2 + d);
#pragma unroll
                for (int c = 0; c < AT_ONCE; ++c) {
                    const float weight = lane_of(by, c1 + c);
                    x = fmaf(v[c].x, weight, x);
                    y = fmaf(v[c].y, weight, y);
                }
            }
        }
        if (lane < D / 2) {
            const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int row = tile.row0 + r, token = row / a.G;
            T *out = (T *)a.out + ((int64_t)(p.first_row + token) * a.Hq + h * a.G + (row - token * a.G)) * D + d;
            out[0] = paged_elem<T>::down(x * by);
            out[1] = paged_elem<T>::down(y * by);
        }
    }
}

}  // namespace

// Pieces are as many as give every compute unit two workgroups.
pq_paged_prefill_plan pq_paged_plan_prefill(const pq_paged_config *cfg, int n_cu)
{
    pq_paged_prefill_plan w;
    w.budget = 2 * (n_cu / cfg->n_kv_heads > 1 ? n_cu / cfg->n_kv_heads : 1);
    w.few_rows = 256;
    w.partials = nullptr;
    return w;
}

int64_t pq_paged_prefill_floats(const pq_paged_config *cfg, const pq_paged_prefill_plan &w)
{
    return (int64_t)cfg->n_kv_heads * (2 * w.budget) * PQ_PAGED_FEW_ROWS * (cfg->head_dim + 2);
}

hipError_t pq_launch_paged_prefill(const pq_paged_ctx *ctx, const pq_paged_attn_args &a, hipStream_t s)
{
    pq_paged_prefill_plan w = ctx->prefill;
    const int64_t rows = (int64_t)a.n_tokens * a.G, seqs = a.n_seqs < a.n_tokens ? a.n_seqs : a.n_tokens;
    // Which kernels can have work.  The one for few rows has all of it where the other's tiles would not fill three quarters of the
    // chip (32 query / 8 KV heads over 8K keys: 1000 tokens 195 us here and 262 in tiles of 256 rows, 1500 tokens 277 and 277, 2000
    // tokens 359 and 278), and none where sequences have many rows on average (four ragged prompts of up to 2000 tokens x 32 heads:
    // 57 us, 62 with the launch that finds nothing).
    if (4 * rows * a.c.Hkv < 3 * (int64_t)PQ_PAGED_TILE_ROWS * ctx->n_cu)
        w.few_rows = INT32_MAX - 1;
    else if (rows >= 2 * (int64_t)w.few_rows * a.n_seqs)
        w.few_rows = 0;
    // tiles there can be: every sequence's last may be a part of one
    const int64_t each = rows / ROWS + seqs, most = seqs * ((w.few_rows + (int64_t)ROWS - 1) / ROWS), few_tiles = each < most ? each : most;
    // No tile is cut if no sequence can be long enough, nor one sequence's tiles, which are alike, where every compute unit has one
    // (250 tokens over 2000 keys 21 us, cut 34, over 10000 keys 78 and 85).
    if ((ctx->cfg.max_blocks << ctx->log_block) <= WHOLE_KEYS || (a.n_seqs == 1 && 2 * few_tiles >= w.budget))
        w.budget = 0;
    const int dtype = ctx->cfg.dtype, dim = ctx->cfg.head_dim;
    if (w.few_rows > 0) {
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_few_kernel<T, D>), dim3((unsigned)((few_tiles + w.budget) * a.c.Hkv) + 1), dim3(THREADS), 0, s, a, w)
        PQ_PAGED_BY_TYPE(dtype, dim, LAUNCH);
#undef LAUNCH
    }
    if (rows > w.few_rows) {
        const hipError_t e = pq_launch_paged_tiles(a, w, dtype, dim, rows / PQ_PAGED_TILE_ROWS + seqs, s);
        if (e != hipSuccess)
            return e;
    }
    if (w.few_rows > 0 && w.budget > 0) {
        const int64_t cut = few_tiles < w.budget ? few_tiles : w.budget;  // tiles that can have several pieces, of 2 budget in all
        const dim3 grid((unsigned)(cut * MERGE_GROUPS * a.c.Hkv));
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_merge_kernel<T, D>), grid, dim3(64 * MERGE_WAVES), 0, s, a, w)
        PQ_PAGED_BY_TYPE(dtype, dim, LAUNCH);
#undef LAUNCH
    }
    return hipGetLastError();
}
