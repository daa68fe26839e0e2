// pq_paged_shared_decode: one query token per sequence, where groups of sequences begin with the same blocks.
//
// A group's query rows (a member's query heads of a KV head side by side, member after member) attend over the shared tokens in
// tiles of 32 rows, so that a block's bytes are read and converted for 32 rows at once; what a member has behind them it attends
// over by itself.  Both are the same work: a tile of rows over a piece of the keys of one block table, 32x32x16 products, the piece
// shared out over four wavefronts.  A first launch (one workgroup) cuts the call into such jobs of about equal length, a second does
// them, a third puts every row's pieces together:  with base_i, l_i, o_i of piece i,
//     m = max base_i,   out = sum 2^(base_i - m) o_i / sum 2^(base_i - m) l_i.
#include <hip/hip_runtime.h>

#include "pq_paged_scan.h"
#include "pq_paged_shared.h"
#include "pq_paged_step.h"

namespace {

constexpr int WAVES = 4, THREADS = 64 * WAVES, ROWS = PQ_PAGED_SHARED_ROWS, STEP = STEP_KEYS;
constexpr int KEY_ALIGN = WAVES * STEP, LEAST_KEYS = 256;

struct shared_sums {
    int start[PQ_PAGED_MAX_SEQS + 1];   // first position of each group
    int shared[PQ_PAGED_MAX_SEQS];      // tokens that its members share
    int length[PQ_PAGED_MAX_SEQS];      // of the sequence at a position; -1: none
    int group_jobs[PQ_PAGED_MAX_SEQS + 1], own_jobs[PQ_PAGED_MAX_SEQS + 1];
    int group_rows[PQ_PAGED_MAX_SEQS], own_rows[PQ_PAGED_MAX_SEQS];
};

__device__ inline int tiles_of(int rows) { return (rows + ROWS - 1) / ROWS; }

// The pieces that n tokens are cut into, none longer than `most`, and their length.  (KEY_ALIGN divides `most`, so the rounded
// length is no more than that, and n is behind (pieces - 1) * most: none is empty.)
__device__ inline int pieces_of(int n, int most) { return (n + most - 1) / most; }
__device__ inline int piece_length(int n, int pieces) { return ((n + pieces - 1) / pieces + KEY_ALIGN - 1) / KEY_ALIGN * KEY_ALIGN; }

// inclusive maximum over the workgroup's threads
__device__ inline int scan_max(int x, scan_room &room)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d, 64);
        x = lane >= d && y > x ? y : x;
    }
    if (lane == 63)
        room.wave[0][wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w)
        x = room.wave[0][w] > x ? room.wave[0][w] : x;
    __syncthreads();
    return x;
}

__device__ inline float sum_all(float x, float *room)
{
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0)
        room[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0f;
    for (int w = 0; w < SCAN_WAVES; ++w)
        x += room[w];
    __syncthreads();
    return x;
}

__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_shared_plan_kernel(pq_paged_shared_args a)
{
    __shared__ shared_sums s;
    __shared__ scan_room room;
    __shared__ float float_room[SCAN_WAVES];
    const int n_seqs = a.n_seqs, n_groups = a.n_groups, G = a.G;
    // where groups begin: as they are given, but never before the one in front
    int highest = 0;
    for (int g0 = 0; g0 <= n_groups; g0 += SCAN_THREADS) {
        const int g = g0 + threadIdx.x;
        int x = g <= n_groups ? between(a.group_start[g], n_seqs) : 0;
        x = x > highest ? x : highest;
        x = scan_max(x, room);
        if (g <= n_groups)
            s.start[g] = x;
        __syncthreads();
        highest = s.start[g0 + SCAN_THREADS - 1 < n_groups ? g0 + SCAN_THREADS - 1 : n_groups];
        __syncthreads();
    }
    bool range = false;
    for (int i = threadIdx.x; i < n_seqs; i += SCAN_THREADS) {
        const int b = a.members == nullptr ? i : a.members[i];
        const bool there = (unsigned)b < (unsigned)n_seqs;
        const bool in_group = i >= s.start[0] && i < s.start[n_groups];
        s.length[i] = in_group && there ? paged_length(a.c, b) : -1;
        range |= in_group && !there;
    }
    if (range)
        paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
    __syncthreads();
    float work = 0.0f;
    for (int g = threadIdx.x; g < n_groups; g += SCAN_THREADS) {
        const int first = s.start[g], n = s.start[g + 1] - first;
        int shared = 0;
        if (n > 1) {
            shared = a.shared_len[g];
            shared = shared < s.length[first] ? shared : s.length[first];
            shared = shared > 0 ? shared >> a.c.log_block << a.c.log_block : 0;
        }
        s.shared[g] = shared;
        work += (float)tiles_of(n * G) * (float)shared;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_seqs; i += SCAN_THREADS)
        if (s.length[i] > 0) {
            const int own = s.length[i] - s.shared[owner(s.start, n_groups, i)];
            work += own > 0 ? (float)tiles_of(G) * (float)own : 0.0f;
        }
    const int most = piece_tokens(sum_all(work, float_room), a.budget, KEY_ALIGN, LEAST_KEYS);

    // jobs and rows of partials: of the groups first, then of the members by themselves
    int jobs = 0, rows = 0;
    for (int g0 = 0; g0 < n_groups; g0 += SCAN_THREADS) {
        const int g = g0 + threadIdx.x;
        int n = 0, pieces = 0;
        if (g < n_groups) {
            n = (s.start[g + 1] - s.start[g]) * G;
            pieces = pieces_of(s.shared[g], most);
        }
        int upto = tiles_of(n) * pieces, upto_rows = n * pieces, all, all_rows;
        const int mine = upto, mine_rows = upto_rows;
        scan_two(upto, upto_rows, room, all, all_rows);
        if (g < n_groups) {
            s.group_jobs[g] = jobs + upto - mine;
            s.group_rows[g] = rows + upto_rows - mine_rows;
        }
        jobs += all;
        rows += all_rows;
    }
    const int of_groups = jobs;
    for (int i0 = 0; i0 < n_seqs; i0 += SCAN_THREADS) {
        const int i = i0 + threadIdx.x;
        int pieces = 0, g = 0;
        if (i < n_seqs && s.length[i] >= 0) {
            g = owner(s.start, n_groups, i);
            const int own = s.length[i] - s.shared[g];
            pieces = own > 0 ? pieces_of(own, most) : 0;
        }
        int upto = tiles_of(G) * pieces, upto_rows = G * pieces, all, all_rows;
        const int mine = upto, mine_rows = upto_rows;
        scan_two(upto, upto_rows, room, all, all_rows);
        if (i < n_seqs) {
            s.own_jobs[i] = upto - mine + jobs - of_groups;
            s.own_rows[i] = rows + upto_rows - mine_rows;
            pq_paged_shared_member m;
            m.b = s.length[i] < 0 ? -1 : a.members == nullptr ? i : a.members[i];
            m.own_row = s.own_rows[i];
            m.own_pieces = pieces;
            m.row = (i - s.start[g]) * G;
            m.rows = (s.start[g + 1] - s.start[g]) * G;
            m.group_row = s.group_rows[g];
            m.group_pieces = m.b < 0 ? 0 : pieces_of(s.shared[g], most);
            m.unused = 0;
            a.w.members[i] = m;
        }
        jobs += all;
        rows += all_rows;
    }
    if (threadIdx.x == 0) {
        s.group_jobs[n_groups] = of_groups;
        s.own_jobs[n_seqs] = jobs - of_groups;
        a.w.head[0] = jobs;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < jobs; e += SCAN_THREADS) {
        pq_paged_shared_job job;
        if (e < of_groups) {
            const int g = owner(s.group_jobs, n_groups, e), at = e - s.group_jobs[g];
            const int n = (s.start[g + 1] - s.start[g]) * G, tiles = tiles_of(n), pieces = pieces_of(s.shared[g], most);
            // tiles of one piece side by side: they read the same bytes
            const int piece = at / tiles, tile = at - piece * tiles, keys = piece_length(s.shared[g], pieces);
            job.position = s.start[g];
            job.table = s.start[g];
            job.row0 = tile * ROWS;
            job.rows = n - job.row0 < ROWS ? n - job.row0 : ROWS;
            job.k0 = piece * keys;
            job.k1 = job.k0 + keys < s.shared[g] ? job.k0 + keys : s.shared[g];
            job.partial = s.group_rows[g] + job.row0 * pieces + piece * job.rows;
        } else {
            const int i = owner(s.own_jobs, n_seqs, e - of_groups), at = e - of_groups - s.own_jobs[i];
            const int shared = s.shared[owner(s.start, n_groups, i)], own = s.length[i] - shared, tiles = tiles_of(G);
            const int pieces = pieces_of(own, most), piece = at / tiles, tile = at - piece * tiles, keys = piece_length(own, pieces);
            job.position = job.table = i;
            job.row0 = tile * ROWS;
            job.rows = G - job.row0 < ROWS ? G - job.row0 : ROWS;
            job.k0 = shared + piece * keys;
            job.k1 = job.k0 + keys < s.length[i] ? job.k0 + keys : s.length[i];
            job.partial = s.own_rows[i] + job.row0 * pieces + piece * job.rows;
        }
        job.table = a.members == nullptr ? job.table : a.members[job.table];
        a.w.jobs[e] = job;
    }
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS, sizeof(T) == 4 ? 1 : 2) void pq_paged_shared_kernel(pq_paged_shared_args a)
{
    constexpr bool SPLIT = sizeof(T) == 4;  // two fp16 parts of queries and weights
    constexpr int PARTS = SPLIT ? 2 : 1, DT = D / 32;
    __shared__ float part[WAVES][ROWS][D + 4];
    __shared__ float wave_base[WAVES][ROWS], wave_l[WAVES][ROWS], row_base[ROWS], row_l[ROWS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int h = blockIdx.x % a.c.Hkv, e = blockIdx.x / a.c.Hkv;
    if (e >= a.w.head[0])
        return;
    const pq_paged_shared_job job = a.w.jobs[e];
    const int share = ((job.k1 - job.k0 + WAVES - 1) / WAVES + STEP - 1) / STEP * STEP;
    const int t0 = job.k0 + wave * share, t1 = t0 + share < job.k1 ? t0 + share : job.k1;
    const int32_t *table = a.c.table + (int64_t)job.table * a.c.max_blocks;
    const int last_block = (job.k1 + (1 << a.c.log_block) - 1) >> a.c.log_block;
    step_bytes<D> now, next;
    block_batch batch;
    batch.first = -65;
    if (t0 < t1)
        load_bytes<D>(a.c, table, batch, last_block, h, t0, lane, now);

    const int col = lane & 31, half = lane >> 5;
    const int row = job.row0 + (col < job.rows ? col : 0), at = row / a.G, head = row - at * a.G;
    const int b = a.members == nullptr ? job.position + at : a.members[job.position + at];
    const bool there = (unsigned)b < (unsigned)a.n_seqs;
    // (columns behind the last row repeat the first one, and nobody takes what they find)
    int sees = col >= job.rows ? t1 : there ? paged_length(a.c, b) : 0;
    sees = sees < t1 ? sees : t1;
    const bool whole = __ballot(sees < t1) == 0;  // every row sees all of this wavefront's keys
    half8v q[PARTS][D / 16];
    float per_score;
    {
        // dims 32 x + 16 half + 0 .. 15 of the row, as K's loads bring them
        float v[D / 2];
        float high = 0.0f;
        const T *src = (const T *)a.q + (int64_t)(there ? b : 0) * a.q_stride + (int64_t)(h * a.G + head) * D + 16 * half;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            paged_load8(src + 32 * x, v + 16 * x);
            paged_load8(src + 32 * x + 8, v + 16 * x + 8);
        }
#pragma unroll
        for (int i = 0; i < D / 2; ++i)
            high = fmaxf(high, fabsf(v[i]));
        high = fmaxf(high, __shfl_xor(high, 32, 64));
        const int exponent = query_exponent(high);
        per_score = ldexpf(a.scale_log2e, -exponent);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = ldexpf(v[8 * x + j], exponent);
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
        if (!whole || t + STEP > t1)
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
    float *const to = a.w.partials + ((int64_t)h * a.w.most_rows + job.partial) * (D + 2);
    for (int i = threadIdx.x; i < job.rows * (D / 2); i += THREADS) {
        const int r = i / (D / 2), d = i % (D / 2) * 2;
        float x = 0.0f, y = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            x = fmaf(part[k][r][d], wave_base[k][r], x);
            y = fmaf(part[k][r][d + 1], wave_base[k][r], y);
        }
        *(float2 *)(to + r * (D + 2) + 2 + d) = make_float2(x, y);
        if (d == 0)
            *(float2 *)(to + r * (D + 2)) = make_float2(row_base[r], row_l[r]);
    }
}

// A row's pieces put together by a wavefront, D / 64 dims a lane.
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void pq_paged_shared_merge_kernel(pq_paged_shared_args a)
{
    constexpr int PER_LANE = D / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t at = (int64_t)blockIdx.x * WAVES + wave;
    const int i = (int)(at / a.Hq), head = (int)(at - (int64_t)i * a.Hq);
    if (i >= a.n_seqs)
        return;
    const pq_paged_shared_member m = a.w.members[i];
    if (m.b < 0)
        return;
    const int h = head / a.G, g = head - h * a.G;
    const float *const partials = a.w.partials + (int64_t)h * a.w.most_rows * (D + 2);
    float top = LOWEST, sum = 0.0f, o[PER_LANE] = {};
    // row r of `rows`, whose tile's pieces lie one after another
    const auto add = [&](int first, int r, int rows, int pieces) {
        const int tile = r / ROWS, in_tile = rows - tile * ROWS < ROWS ? rows - tile * ROWS : ROWS;
        const float *from = partials + (int64_t)(first + tile * ROWS * pieces + (r - tile * ROWS)) * (D + 2);
        const int64_t stride = (int64_t)in_tile * (D + 2);
        for (int c0 = 0; c0 < pieces; c0 += 64, from += 64 * stride) {
            // a lane has a piece's base and sum, and so its weight; one that is not there has the weight 0
            const int n = pieces - c0 < 64 ? pieces - c0 : 64;
            const float2 ml = lane < n ? *(const float2 *)(from + lane * stride) : make_float2(-INFINITY, 0.0f);
            const float high = fmaxf(top, wave_max(ml.x)), old = __builtin_amdgcn_exp2f(top - high), by = __builtin_amdgcn_exp2f(ml.x - high);
            top = high;
            sum = fmaf(sum, old, wave_sum(ml.y * by));
#pragma unroll
            for (int d = 0; d < PER_LANE; ++d)
                o[d] *= old;
            constexpr int AT_ONCE = 8;  // loads on their way together
            for (int c1 = 0; c1 < n; c1 += AT_ONCE) {
                float v[AT_ONCE][PER_LANE];
#pragma unroll
                for (int c = 0; c < AT_ONCE; ++c)
#pragma unroll
                    for (int d = 0; d < PER_LANE; ++d)
                        v[c][d] = from[(c1 + c < n ? c1 + c : 0) * stride + 2 + PER_LANE * lane + d];
#pragma unroll
                for (int c = 0; c < AT_ONCE; ++c) {
                    const float weight = lane_of(by, c1 + c);
#pragma unroll
                    for (int d = 0; d < PER_LANE; ++d)
                        o[d] = fmaf(v[c][d], weight, o[d]);
                }
            }
        }
    };
    add(m.group_row, m.row + g, m.rows, m.group_pieces);
    add(m.own_row, g, a.G, m.own_pieces);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    T *const out = (T *)a.out + ((int64_t)m.b * a.Hq + head) * D + PER_LANE * lane;
#pragma unroll
    for (int d = 0; d < PER_LANE; ++d)
        out[d] = paged_elem<T>::down(o[d] * by);
}

int64_t round_up(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// Jobs: `budget` pieces and a rest for each tile.  Rows of partials: as many as the tiles of those pieces have.
int64_t pq_paged_shared_layout(const pq_paged_ctx *ctx, int n_seqs, int n_groups, void *workspace, pq_paged_shared_work *w)
{
    const pq_paged_config &cfg = ctx->cfg;
    const int64_t G = cfg.n_q_heads / cfg.n_kv_heads, budget = pq_paged_shared_budget(ctx);
    const int64_t tiles = n_seqs * G / ROWS + n_groups + n_seqs * ((G + ROWS - 1) / ROWS);
    const int64_t jobs = budget + tiles, rows = ROWS * budget + 2 * n_seqs * G;
    int64_t bytes = 0;
    const auto room = [&](int64_t n) { const int64_t at = bytes; bytes += round_up(n); return at; };
    const int64_t head_at = room(sizeof(int)), members_at = room(n_seqs * sizeof(pq_paged_shared_member));
    const int64_t jobs_at = room(jobs * sizeof(pq_paged_shared_job));
    const int64_t partials_at = room(cfg.n_kv_heads * rows * (cfg.head_dim + 2) * sizeof(float));
    if (w != nullptr) {
        char *const at = (char *)workspace;
        w->head = (int *)(at + head_at);
        w->members = (pq_paged_shared_member *)(at + members_at);
        w->jobs = (pq_paged_shared_job *)(at + jobs_at);
        w->partials = (float *)(at + partials_at);
        w->most_jobs = (int)jobs;
        w->most_rows = rows;
    }
    return bytes;
}

// Pieces that a call's keys are cut into for each KV head: two workgroups a compute unit.
int pq_paged_shared_budget(const pq_paged_ctx *ctx)
{
    const int n = 2 * ctx->n_cu / ctx->cfg.n_kv_heads;
    return n > 1 ? n : 1;
}

hipError_t pq_launch_paged_shared(const pq_paged_ctx *ctx, const pq_paged_shared_args &a, hipStream_t s)
{
    hipLaunchKernelGGL(pq_paged_shared_plan_kernel, dim3(1), dim3(SCAN_THREADS), 0, s, a);
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_shared_kernel<T, D>), dim3((unsigned)a.w.most_jobs * (unsigned)a.c.Hkv), dim3(THREADS), 0, s, a)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    const int64_t rows = (int64_t)a.n_seqs * a.Hq;
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_shared_merge_kernel<T, D>), dim3((unsigned)((rows + WAVES - 1) / WAVES)), dim3(THREADS), 0, s, a)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
