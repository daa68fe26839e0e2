// pq_paged_prefill: causal attention of many query tokens per sequence over the paged 8-bit cache.
//
// A workgroup has one sequence, one KV head and a tile of query rows — a token's query heads of that KV head lie side by side,
// so a tile of 256 rows is 64 tokens of 4 heads — and walks the keys that the tile sees, 64 at a time.  Bytes become fp16 codes
// once per tile, on their way into LDS, and are then the left operands of 32x32x16 matrix instructions for all four
// wavefronts: S^T = K Q^T, and O^T = V^T W with the weights straight from the registers that the scores came in (V's
// tokens lie in LDS in the order in which the result of the first product holds them).  A lane has one query row per 32 columns:
// its maximum, sum, limit and rescaling are its own.
//
// Few rows over many keys: the keys of a tile are cut into pieces as well, put together by the workgroup that ends last.
//
// Bound by the matrix units and, nearly as much, by the exponentials beside them.
#include <hip/hip_runtime.h>

#include "pq_paged_tile.h"

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES;
constexpr int KEYS = 64;                      // tokens of a tile of keys
constexpr int K_PLANE = KEYS * 16 + 16;       // bytes of 8 dims of all keys, and a shift of 4 banks
constexpr int V_PLANE = 16;                   // bytes of 8 tokens of one dim

template <int D> struct tile_lds {
    unsigned char k[D / 8 * K_PLANE];         // [dim / 8][key][dim % 8]
    unsigned char v[KEYS / 16 * 2 * D * V_PLANE];  // [piece][half of its tokens][dim][8 tokens]
};

struct work_place {
    int b, len, first_row, rows;  // sequence, its length, its first row of the tensors, its rows there
    int past;                     // keys in front of its first row's own (negative: the first rows see nothing)
    int tile, split, keys;        // tile of its rows, piece of the keys, keys of a piece
    int slot;                     // of the tile's first piece among the call's
};

// Rows of sequence b that lie in the tensors
__device__ inline int rows_of(const pq_paged_attn_args &a, int b, int &start)
{
    start = a.tok_start[b];
    const int n = a.tok_len[b];
    if (start < 0 || start >= a.n_tokens || n <= 0)
        return 0;
    return n < a.n_tokens - start ? n : a.n_tokens - start;
}

// Entry e of the call's list of (sequence, tile, piece of keys); the tiles that see most come first.  With enough tiles there is
// one piece each; else the tokens-times-tiles of the call are cut into about `budget` pieces of the same length.
__device__ inline bool find_work(const pq_paged_attn_args &a, int tile_rows, int budget, int e, int lane, work_place &p)
{
    int64_t tiles = 0, work = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64)
        if (b0 + lane < a.n_seqs) {
            int start;
            const int n = (rows_of(a, b0 + lane, start) * a.G + tile_rows - 1) / tile_rows;
            tiles += n;
            work += (int64_t)n * paged_length(a.c, b0 + lane);
        }
    tiles = __shfl(lane_scan(tiles, lane), 63, 64);
    work = __shfl(lane_scan(work, lane), 63, 64);
    p.keys = PQ_MAX_TOKENS;
    if (tiles < budget) {
        const int64_t share = (work + budget - 1) / budget;
        const int n = share < PQ_MAX_TOKENS ? (int)share : PQ_MAX_TOKENS;
        p.keys = n > 4 * KEYS ? (n + KEYS - 1) / KEYS * KEYS : 4 * KEYS;
    }
    int before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int start = 0, rows = 0, len = 0, splits = 0, n = 0;
        if (b0 + lane < a.n_seqs) {
            rows = rows_of(a, b0 + lane, start);
            len = paged_length(a.c, b0 + lane);
            splits = len > 0 ? (len + p.keys - 1) / p.keys : 1;
            n = (rows * a.G + tile_rows - 1) / tile_rows * splits;
        }
        const int upto = before + (int)lane_scan(n, lane);
        const uint64_t mine = __ballot(e >= upto - n && e < upto);
        if (mine != 0) {
            const int l = __builtin_ctzll(mine);
            p.b = b0 + l;
            p.len = __builtin_amdgcn_readlane(len, l);
            p.first_row = __builtin_amdgcn_readlane(start, l);
            p.rows = __builtin_amdgcn_readlane(rows, l);
            p.past = p.len - a.tok_len[p.b];
            const int per_tile = __builtin_amdgcn_readlane(splits, l), all = __builtin_amdgcn_readlane(n, l);
            const int at = e - (__builtin_amdgcn_readlane(upto, l) - all);
            p.tile = all / per_tile - 1 - at / per_tile;
            p.split = at % per_tile;
            p.slot = e - p.split;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// A wavefront's share of a tile of keys, as bytes on their way to LDS
template <int D> struct key_bytes {
    u32x4 k[D / 64], v[D / 64];
};

// the piece of 16 tokens that part x of a wavefront's share lies in
template <int D> __device__ inline int piece_of(int wave, int x) { return D == 128 ? (wave >> 1) + 2 * x : wave; }

template <int D>
__device__ inline void load_keys(const pq_paged_view &c, const block_batch &batch, int h, int t, int wave, int lane, key_bytes<D> &to)
{
    const int tid = wave * 64 + lane;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
        const int piece = piece_of<D>(wave, x), p = t + 16 * piece;
        const int id = __builtin_amdgcn_readlane(batch.id, (p >> c.log_block) - batch.first);
        const int64_t base = (((int64_t)id * c.Hkv + h) << c.log_block) * D + (p & ((1 << c.log_block) - 1)) * D;
        const int at = (tid + THREADS * x) * 16 - piece * 16 * D;  // within the piece: K's 16-byte parts of rows, and V's words
        to.k[x] = *(const u32x4 *)(c.k + base + at);
        to.v[x] = *(const u32x4 *)(c.v + base + at);
    }
}

template <int D> __device__ inline void store_keys(tile_lds<D> &lds, int wave, int lane, const key_bytes<D> &from)
{
    const int tid = wave * 64 + lane;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
        const int id = tid + THREADS * x, key = id / (D / 16), part = id % (D / 16);
        *(half8v *)(lds.k + (2 * part) * K_PLANE + key * 16) = codes8(from.k[x][0], from.k[x][1]);
        *(half8v *)(lds.k + (2 * part + 1) * K_PLANE + key * 16) = codes8(from.k[x][2], from.k[x][3]);
        const int piece = piece_of<D>(wave, x), at = id - piece * D, quad = (at >> 4) & 3, dim0 = (at >> 6) * 64 + (at & 15);
        unsigned char *v = lds.v + (piece * 2 + (quad & 1)) * (D * V_PLANE) + (quad >> 1) * 8;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *(half4v *)(v + (dim0 + 16 * k) * V_PLANE) = codes4(from.v[x][k]);
    }
}

template <typename T, int D, int NT>
__global__ __launch_bounds__(THREADS, NT == 2 ? 1 : 2) void pq_paged_prefill_kernel(pq_paged_attn_args a, pq_paged_prefill_plan w)
{
    constexpr bool SPLIT = sizeof(T) == 4;  // two fp16 parts of queries and weights
    constexpr int PARTS = SPLIT ? 2 : 1, DT = D / 32, TILE_ROWS = WAVES * 32 * NT;
    __shared__ tile_lds<D> lds[2];
    __shared__ int last_one;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int h = blockIdx.x % a.c.Hkv, entry = blockIdx.x / a.c.Hkv;
    work_place p;
    if (!find_work(a, TILE_ROWS, w.budget, entry, lane, p))
        return;
    const int col = lane & 31, half = lane >> 5;
    const int past = p.past, row0 = p.tile * TILE_ROWS, all_rows = p.rows * a.G;
    const int last_row = (row0 + TILE_ROWS < all_rows ? row0 + TILE_ROWS : all_rows) - 1;
    int tile_sees = past + last_row / a.G + 1;                        // keys that the tile's last row sees
    tile_sees = tile_sees < 0 ? 0 : tile_sees;
    const int pieces = tile_sees > p.keys ? (tile_sees + p.keys - 1) / p.keys : 1;
    if (p.split >= pieces)
        return;
    const int k0 = p.split * p.keys, k1 = k0 + p.keys < tile_sees ? k0 + p.keys : tile_sees;

    // this lane's rows, and what they see
    int sees[NT], token[NT], head[NT];
    float per_score[NT];
    half8v q[NT][PARTS][D / 16];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = row0 + (wave * NT + n) * 32 + col;
        const bool there = r < all_rows;
        token[n] = there ? r / a.G : -1;
        head[n] = there ? r - token[n] * a.G : 0;
        sees[n] = there ? past + token[n] + 1 : 0;
        // dims 16 x + 8 half + 0 .. 7 of the row
        float v[D / 2];
        float high = 0.0f;
        const T *src = (const T *)a.q + (int64_t)(p.first_row + (there ? token[n] : 0)) * a.q_stride +
                       (int64_t)(h * a.G + head[n]) * D + 8 * half;
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
            paged_load8(src + 16 * x, v + 8 * x);
#pragma unroll
        for (int i = 0; i < D / 2; ++i)
            high = fmaxf(high, fabsf(v[i]));
        high = fmaxf(high, __shfl_xor(high, 32, 64));
        const int e = query_exponent(high);
        per_score[n] = ldexpf(a.scale_log2e, -e);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = ldexpf(v[8 * x + j], e);
                q[n][0][x][j] = (_Float16)f;
                if (SPLIT)
                    q[n][PARTS - 1][x][j] = (_Float16)(f - (float)q[n][0][x][j]);
            }
    }
    // what the wavefront's first and last rows see: keys below the one need no mask, keys from the other on no work
    const int wave_first = row0 + wave * NT * 32, wave_last = wave_first + NT * 32 - 1;
    const int wave_least = wave_last < all_rows ? past + wave_first / a.G + 1 : 0;
    int wave_sees = wave_first < all_rows ? past + (wave_last < all_rows ? wave_last : all_rows - 1) / a.G + 1 : 0;
    wave_sees = wave_sees < k1 ? wave_sees : k1;

    f32x16 o[DT][NT];
    float m[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        m[n] = LOWEST;
        l[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                o[i][n][j] = 0.0f;
    }

    const int32_t *table = a.c.table + (int64_t)p.b * a.c.max_blocks;
    const int last_block = (p.len + (1 << a.c.log_block) - 1) >> a.c.log_block, per_tile = KEYS >> a.c.log_block;
    key_bytes<D> bytes;
    block_batch batch, ahead;  // of the tile that is worked on, and of the one that is loaded
    if (k0 < k1) {
        ahead = load_batch(a.c, table, k0 >> a.c.log_block, last_block, h, lane);
        load_keys<D>(a.c, ahead, h, k0, wave, lane, bytes);
        store_keys<D>(lds[0], wave, lane, bytes);
    }
    int buffer = 0;
    for (int t = k0; t < k1; t += KEYS, buffer ^= 1) {
        __syncthreads();
        batch = ahead;
        const bool more = t + KEYS < k1;
        if (more) {
            const int j = (t + KEYS) >> a.c.log_block;
            if (j + per_tile > ahead.first + 64)
                ahead = load_batch(a.c, table, j, last_block, h, lane);
            load_keys<D>(a.c, ahead, h, t + KEYS, wave, lane, bytes);
        }
        if (t < wave_sees) {
            const tile_lds<D> &now = lds[buffer];
#pragma unroll
            for (int u = 0; u < 2; ++u) {  // 32 keys at a time
                f32x16 s[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        s[n][j] = 0.0f;
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const half8v k = *(const half8v *)(now.k + (2 * x + half) * K_PLANE + (32 * u + col) * 16);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < PARTS; ++i)
                            s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[n][i][x], s[n], 0, 0, 0);
                }
                float k_scale[2], v_log[2], v_inv[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int at = ((t + 32 * u + 16 * i) >> a.c.log_block) - batch.first;
                    k_scale[i] = lane_of(batch.k_scale, at);
                    v_log[i] = lane_of(batch.v_log, at);
                    v_inv[i] = lane_of(batch.v_inv, at);
                }
                half8v weights[NT][PARTS][2];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float by = per_score[n] * k_scale[i];
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            s[n][8 * i + j] = fmaf(s[n][8 * i + j], by, v_log[i]);
                    }
                    if (t + 32 * u + 32 > wave_least || t + 32 * u + 32 > k1)
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (t + 32 * u + 8 * (j >> 2) + 4 * half + (j & 3) >= (sees[n] < k1 ? sees[n] : k1))
                                s[n][j] = -INFINITY;
                    float high = s[n][0];
#pragma unroll
                    for (int j = 1; j < 16; ++j)
                        high = fmaxf(high, s[n][j]);
                    if (__ballot(high > m[n] + MAX_SLACK) != 0) {
                        high = fmaxf(high, __shfl_xor(high, 32, 64));
                        const float moved = fmaxf(m[n], high), down = __builtin_amdgcn_exp2f(m[n] - moved);
                        m[n] = moved;
                        l[n] *= down;
#pragma unroll
                        for (int i = 0; i < DT; ++i)
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                o[i][n][j] *= down;
                    }
                    const float base = m[n] - WEIGHT_BITS;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float sum = 0.0f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float x = __builtin_amdgcn_exp2f(s[n][8 * i + j] - base);
                            sum += x;
                            weights[n][0][i][j] = (_Float16)x;
                            if (SPLIT)
                                weights[n][PARTS - 1][i][j] = (_Float16)(x - (float)weights[n][0][i][j]);
                        }
                        l[n] = fmaf(sum, v_inv[i], l[n]);
                    }
                }
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const half8v v = *(const half8v *)(now.v + ((2 * u + x) * 2 + half) * (D * V_PLANE) + (32 * i + col) * V_PLANE);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < PARTS; ++j)
                                o[i][n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, weights[n][j][x], o[i][n], 0, 0, 0);
                    }
            }
        }
        if (more)
            store_keys<D>(lds[buffer ^ 1], wave, lane, bytes);
    }

    const int64_t slot0 = (int64_t)h * w.slots + p.slot;
    float *const parts = w.partials + slot0 * (TILE_ROWS * (D + 2));
    float *const mine = parts + (int64_t)p.split * (TILE_ROWS * (D + 2));
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float sum = l[n] + __shfl_xor(l[n], 32, 64);
        const int r = (wave * NT + n) * 32 + col;
        if (token[n] < 0)
            continue;
        if (pieces == 1) {
            const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
            T *out = (T *)a.out + ((int64_t)(p.first_row + token[n]) * a.Hq + h * a.G + head[n]) * D + 4 * half;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    T x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = paged_elem<T>::down(o[i][n][j + e] * by);
                    __builtin_memcpy(out + 32 * i + 2 * j, x, sizeof(x));
                }
        } else {
            float *to = mine + r * (D + 2);
            if (half == 0)
                publish(to, m[n], sum);
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; j += 2)
                    publish(to + 2 + 32 * i + 8 * (j >> 2) + 4 * half + (j & 3), o[i][n][j], o[i][n][j + 1]);
        }
    }
    if (pieces == 1)
        return;
    publish_wait();
    __syncthreads();
    unsigned int *ticket = w.tickets + slot0;
    if (threadIdx.x == 0)
        last_one = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(pieces - 1);
    __syncthreads();
    if (!last_one)
        return;
    if (threadIdx.x == 0)
        ticket_reset(ticket);
    const int rows = last_row - row0 + 1;
    for (int i = threadIdx.x; i < rows * (D / 2); i += THREADS) {
        const int r = i / (D / 2), d = i % (D / 2) * 2;
        float top = LOWEST, sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll 4
        for (int c = 0; c < pieces; ++c) {
            const float *from = parts + (int64_t)c * (TILE_ROWS * (D + 2)) + r * (D + 2);
            const float2 ml = fetch(from), v = fetch(from + 2 + d);
            const float high = fmaxf(top, ml.x), old = __builtin_amdgcn_exp2f(top - high), by = __builtin_amdgcn_exp2f(ml.x - high);
            top = high;
            sum = fmaf(ml.y, by, sum * old);
            x = fmaf(v.x, by, x * old);
            y = fmaf(v.y, by, y * old);
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int t = (row0 + r) / a.G;
        T *out = (T *)a.out + ((int64_t)(p.first_row + t) * a.Hq + h * a.G + (row0 + r - t * a.G)) * D + d;
        out[0] = paged_elem<T>::down(x * by);
        out[1] = paged_elem<T>::down(y * by);
    }
}

}  // namespace

// Rows of a tile: 256, in fp32 (queries in two parts) 128.
static int column_tiles(const pq_paged_config *cfg) { return cfg->dtype == PQ_F32 ? 1 : 2; }

// Pieces of keys are as many as give every compute unit a workgroup.
pq_paged_prefill_plan pq_paged_plan_prefill(const pq_paged_config *cfg, int n_cu)
{
    pq_paged_prefill_plan w;
    w.budget = n_cu / cfg->n_kv_heads > 1 ? n_cu / cfg->n_kv_heads : 1;
    w.slots = 2 * w.budget;
    w.partials = nullptr;
    w.tickets = nullptr;
    return w;
}

int64_t pq_paged_prefill_slot_floats(const pq_paged_config *cfg) { return (int64_t)WAVES * 32 * column_tiles(cfg) * (cfg->head_dim + 2); }

hipError_t pq_launch_paged_prefill(const pq_paged_ctx *ctx, const pq_paged_attn_args &a, hipStream_t s)
{
    const pq_paged_prefill_plan &w = ctx->prefill;
    const int tile_rows = WAVES * 32 * column_tiles(&ctx->cfg);
    // tiles there can be: every sequence's last may be a part of one
    const int64_t tiles = ((int64_t)a.n_tokens * a.G) / tile_rows + (a.n_seqs < a.n_tokens ? a.n_seqs : a.n_tokens);
    const int64_t entries = tiles < w.budget ? w.budget + tiles : tiles > 2 * w.budget ? tiles : 2 * w.budget;
    const dim3 grid((unsigned)(entries * a.c.Hkv));
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_prefill_kernel<T, D, sizeof(T) == 4 ? 1 : 2>), grid, dim3(THREADS), 0, s, a, w)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
