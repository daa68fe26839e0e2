// Up to 32 query rows of a KV head against keys as they lie in memory, one wavefront, products of 32x32x16; and the parts of a
// workgroup's wavefronts put together (gfx950).
#pragma once

#include "pq_paged_tile.h"

namespace {

constexpr int STEP_32 = 32;  // keys a wavefront takes at a time

// With fp32 queries of 128 dims a wavefront's rows, keys and sums take nearly all of the 256 registers that let two workgroups share a compute
// unit.  What follows from x, which the compiler would else keep through all loops, is worked out where it is used: 288 registers become
// 256, and 32 samples of 8192 tokens 29.7 us instead of 37.1 (256 with what does not fit spilled: 32.1).
template <typename T, int D> __device__ inline void work_out_here(int &x)
{
    if constexpr (sizeof(T) == 4 && D == 128)
        asm volatile("" : "+v"(x));
}

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

// A query row: lane has that of its column, dims 32 x + 16 half + 0 .. 15, as K's loads bring them
template <typename T, int D> struct query_32 {
    paged_row8<T> x[D / 16];
};

template <typename T, int D> __device__ inline void load_query(const T *row, int half, query_32<T, D> &to)
{
    const T *src = row + 16 * half;
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
        to.x[x] = *(const paged_row8<T> *)(src + 32 * (x >> 1) + 8 * (x & 1));
}

template <typename T, int D> struct rows_32 {
    static constexpr bool SPLIT = sizeof(T) == 4;  // two fp16 parts of queries and weights
    static constexpr int PARTS = SPLIT ? 2 : 1, DT = D / 32, STEP = STEP_32;

    half8v q[PARTS][D / 16];
    float per_score;
    f32x16 o[DT];
    float base, l;

    __device__ inline void take(const query_32<T, D> &row, float scale_log2e)
    {
        float v[D / 2];
        float high = 0.0f;
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
            paged_up8(row.x[x], v + 8 * x);
#pragma unroll
        for (int i = 0; i < D / 2; ++i)
            high = fmaxf(high, fabsf(v[i]));
        high = fmaxf(high, __shfl_xor(high, 32, 64));
        const int e = query_exponent(high);
        per_score = ldexpf(scale_log2e, -e);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = ldexpf(v[8 * x + j], e);
                q[0][x][j] = (_Float16)f;
                if (SPLIT)
                    q[PARTS - 1][x][j] = (_Float16)(f - (float)q[0][x][j]);
            }
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                o[i][j] = 0.0f;
        base = LOWEST;
        l = 0.0f;
    }

    // The keys from t on: the lane's row attends over those in front of `sees`, and every row over those in front of `whole`
    __device__ inline void step(const step_bytes<D> &now, int t, int sees, int whole, int half)
    {
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
        if (t + STEP > whole) {
            asm volatile("");  // (else all steps are masked, without a branch)
            work_out_here<T, D>(half);
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (t + 8 * (j >> 2) + 4 * half + (j & 3) >= sees)
                    s[j] = -INFINITY;
        }
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
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const half8v v = codes8(now.v[x][0][i], now.v[x][1][i]);
#pragma unroll
                for (int j = 0; j < PARTS; ++j)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, weights[j][x], o[i], 0, 0, 0);
            }
    }

    // Keys t0 .. t1 - 1, the first STEP of which are in `now` already.  The lane's row attends over the first `sees` keys of its
    // sequence, no more than t1, and every row over the first `least`.
    __device__ inline void attend(const pq_paged_view &c, const int32_t *table, block_batch &batch, int last_block, int h, int t0, int t1,
                                  int sees, int least, int lane, step_bytes<D> &now)
    {
        const int half = lane >> 5, whole = least < t1 ? least : t1;
        step_bytes<D> next;
        for (int t = t0; t < t1; t += STEP) {
            const bool more = t + STEP < t1;
            if (more)
                load_bytes<D>(c, table, batch, last_block, h, t + STEP, lane, next);
            step(now, t, sees, whole, half);
            if (more)
                now = next;
        }
    }
};

// What a workgroup of four wavefronts puts its parts together in
constexpr int JOIN_WAVES = 4, JOIN_ROWS = 32;

template <int D> struct join_room {
    float part[JOIN_WAVES][JOIN_ROWS][D + 4];
    float base[JOIN_WAVES][JOIN_ROWS], l[JOIN_WAVES][JOIN_ROWS], row_base[JOIN_ROWS], row_l[JOIN_ROWS];

    // Row r's bases and sums, and its parts' factors (in `base`)
    template <typename T> __device__ inline void join(const rows_32<T, D> &x, int wave, int lane)
    {
        const int col = lane & 31, half = lane >> 5;
        const float sum_l = x.l + __shfl_xor(x.l, 32, 64);
        if (half == 0) {
            base[wave][col] = x.base;
            l[wave][col] = sum_l;
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const int d = (D == 128 ? 64 * (j >> 3) + 16 * i : 32 * (j >> 3) + 16 * i) + 8 * ((j >> 2) & 1) + 4 * half;
                *(f32x4 *)&part[wave][col][d] = f32x4{x.o[i][j], x.o[i][j + 1], x.o[i][j + 2], x.o[i][j + 3]};
            }
        __syncthreads();
        int r = threadIdx.x;
        work_out_here<T, D>(r);
        if (r < JOIN_ROWS) {
            float top = base[0][r], sum = 0.0f;
#pragma unroll
            for (int i = 1; i < JOIN_WAVES; ++i)
                top = fmaxf(top, base[i][r]);
#pragma unroll
            for (int i = 0; i < JOIN_WAVES; ++i) {
                const float down = __builtin_amdgcn_exp2f(base[i][r] - top);
                sum = fmaf(l[i][r], down, sum);
                base[i][r] = down;
            }
            row_base[r] = top;
            row_l[r] = sum;
        }
        __syncthreads();
    }

    // Dims d and d + 1 of row r
    __device__ inline float2 values(int r, int d) const
    {
        float x = 0.0f, y = 0.0f;
#pragma unroll
        for (int k = 0; k < JOIN_WAVES; ++k) {
            x = fmaf(part[k][r][d], base[k][r], x);
            y = fmaf(part[k][r][d + 1], base[k][r], y);
        }
        return make_float2(x, y);
    }
};

}  // namespace
