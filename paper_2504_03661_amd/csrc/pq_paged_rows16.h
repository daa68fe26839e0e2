// Up to 16 query rows of a KV head against keys as they lie in memory, one wavefront, products of 16x16x32 (gfx950).
//
// Scores are S^T = K Q^T, 16 tokens by 16 query rows per matrix instruction: in the result a lane holds four tokens of one row,
// which is what the second product, O^T = V^T W, takes as its right operand — weights go from one to the other in registers, and a
// row's maximum, sum and rescaling are its lanes' own.
#pragma once

#include "pq_paged_tile.h"

namespace {

constexpr int STEP_16 = 32;  // tokens a wavefront takes at a time

// Two pieces of 16 tokens as they lie in memory, and their blocks' scales
template <int D> struct step_data {
    u32x4 k[2][D / 64], v[2][D / 64];
    float k_scale[2], v_log[2], v_inv[2];
};

template <int D>
__device__ inline void load_step(const pq_paged_view &c, const int32_t *table, block_batch &batch, int last_block, int h, int t,
                                 int lane, step_data<D> &s)
{
    const int k_at = (lane & 15) * D + (lane >> 4) * 16, v_at = lane * 16;
    // (t is a multiple of 32: both pieces are in one batch)
    const bool anew = (t >> c.log_block) >= batch.first + 64;
    if (anew)
        start_batch(c, table, t >> c.log_block, last_block, h, lane, batch);
    int at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int p = t + 16 * i;
        at[i] = (p >> c.log_block) - batch.first;
        const int id = __builtin_amdgcn_readlane(batch.id, at[i]);
        const int64_t base = (((int64_t)id * c.Hkv + h) << c.log_block) * D + (p & ((1 << c.log_block) - 1)) * D;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
            s.k[i][x] = __builtin_nontemporal_load((const u32x4 *)(c.k + base + k_at + 64 * x));
            s.v[i][x] = __builtin_nontemporal_load((const u32x4 *)(c.v + base + v_at + 1024 * x));
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

// A query row: lane has that of its column, dims 64 x + 16 quad + 0 .. 15, as the instruction's k index takes K's bytes
template <typename T, int D> struct query_16 {
    paged_row8<T> x[D / 32];
};

template <typename T, int D> __device__ inline void load_query(const T *row, int quad, query_16<T, D> &to)
{
    const T *src = row + quad * 16;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
        to.x[i] = *(const paged_row8<T> *)(src + 64 * (i >> 1) + 8 * (i & 1));
}

template <typename T, int D> struct rows_16 {
    static constexpr bool SPLIT = sizeof(T) == 4;  // two fp16 parts of queries and weights
    static constexpr int PARTS = SPLIT ? 2 : 1, DT = D / 16, STEP = STEP_16;

    half8v q[PARTS][D / 32];
    float per_score;  // what a dot product of codes is multiplied by, but for the block's scale
    f32x4 o[DT];      // dims 16 i + 4 quad + 0 .. 3
    float base, l;

    __device__ inline void take(const query_16<T, D> &row, float scale_log2e)
    {
        float x[D / 4];
        float high = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
            paged_up8(row.x[i], x + 8 * i);
#pragma unroll
        for (int i = 0; i < D / 4; ++i)
            high = fmaxf(high, fabsf(x[i]));
        high = fmaxf(high, __shfl_xor(high, 16, 64));
        high = fmaxf(high, __shfl_xor(high, 32, 64));
        const int e = query_exponent(high);
        per_score = ldexpf(scale_log2e, -e);
#pragma unroll
        for (int s = 0; s < D / 32; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = ldexpf(x[8 * s + j], e);
                q[0][s][j] = (_Float16)v;
                if (SPLIT)
                    q[PARTS - 1][s][j] = (_Float16)(v - (float)q[0][s][j]);
            }
#pragma unroll
        for (int i = 0; i < DT; ++i)
            o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        base = LOWEST;
        l = 0.0f;
    }

    // Tokens t0 .. t1 - 1, the first STEP of which are in `now` already
    __device__ inline void attend(const pq_paged_view &c, const int32_t *table, block_batch &batch, int last_block, int h, int t0, int t1,
                                  int lane, step_data<D> &now)
    {
        const int quad = lane >> 4;
        step_data<D> next;
        for (int t = t0; t < t1; t += STEP) {
            const bool more = t + STEP < t1;
            if (more)
                load_step<D>(c, table, batch, last_block, h, t + STEP, lane, next);
            float s[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x4 dot = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    const half8v k = codes8(now.k[i][x >> 1][2 * (x & 1)], now.k[i][x >> 1][2 * (x & 1) + 1]);
#pragma unroll
                    for (int part_ = 0; part_ < PARTS; ++part_)
                        dot = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[part_][x], dot, 0, 0, 0);
                }
                const float by = per_score * now.k_scale[i];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[4 * i + j] = fmaf(dot[j], by, now.v_log[i]);
            }
            if (t + STEP > t1)  // the last step: tokens behind the end
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (t + 16 * (i >> 2) + 4 * quad + (i & 3) >= t1)
                        s[i] = -INFINITY;
            float high = s[0];
#pragma unroll
            for (int i = 1; i < 8; ++i)
                high = fmaxf(high, s[i]);
            if (__ballot(high - base > MOST_BITS) != 0) {
                high = fmaxf(high, __shfl_xor(high, 16, 64));
                high = fmaxf(high, __shfl_xor(high, 32, 64));
                const float moved = fmaxf(base, weight_base(high)), down = __builtin_amdgcn_exp2f(base - moved);
                base = moved;
                l *= down;
#pragma unroll
                for (int i = 0; i < DT; ++i)
                    o[i] *= down;
            }
            half8v weights[PARTS];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = __builtin_amdgcn_exp2f(s[4 * i + j] - base);
                    sum += x;
                    weights[0][4 * i + j] = (_Float16)x;
                    if (SPLIT)
                        weights[PARTS - 1][4 * i + j] = (_Float16)(x - (float)weights[0][4 * i + j]);
                }
                l = fmaf(sum, now.v_inv[i], l);
            }
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const half8v v = codes8(now.v[0][i >> 2][i & 3], now.v[1][i >> 2][i & 3]);
#pragma unroll
                for (int part_ = 0; part_ < PARTS; ++part_)
                    o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, weights[part_], o[i], 0, 0, 0);
            }
            if (more)
                now = next;
        }
    }

    // the sum of all lanes of a row
    __device__ inline float sum() const
    {
        float x = l;
        x += __shfl_xor(x, 16, 64);
        x += __shfl_xor(x, 32, 64);
        return x;
    }
};

}  // namespace
