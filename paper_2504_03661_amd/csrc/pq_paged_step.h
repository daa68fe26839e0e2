// 32 keys of a sequence from memory to the lanes that multiply them, for products of 32x32x16 (gfx950).
#pragma once

#include "pq_paged_tile.h"

namespace {

constexpr int STEP_KEYS = 32;

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

}  // namespace
