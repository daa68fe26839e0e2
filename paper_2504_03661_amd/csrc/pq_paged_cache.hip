// pq_paged_append and pq_paged_read: values in and out of the blocks of the paged 8-bit cache.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "pq_paged.h"

namespace {

constexpr float CODE_MAX = 127.0f;
constexpr float SMALLEST = 127.0f / 1099511627776.0f;  // 127 * 2^-40: no scale is below 2^-40, so no quotient overflows

// x / s to the nearest integer, ties to even, decided by the exact quotient: the product with the reciprocal names a candidate
// r at most one off; what is left, x - r s, is exact in one fma (it is a multiple of the smaller unit of x and s, and at
// most about s), and so is its comparison with s / 2.
__device__ inline float nearest_code(float x, float s, float inv)
{
    float r = rintf(x * inv);
    const float left = fmaf(-r, s, x), half = 0.5f * s;
    const bool odd = ((int)r & 1) != 0;
    if (left > half || (left == half && odd))
        r += 1.0f;
    else if (left < -half || (left == -half && odd))
        r -= 1.0f;
    return fminf(fmaxf(r, -CODE_MAX), CODE_MAX);
}

// an older code under a larger scale (in double: code * was is exact, and the quotient is far enough from a tie that it is not)
__device__ inline int regrown_code(int c, float was, float s) { return (int)rint((double)c * (double)was / (double)s); }

__device__ inline uint32_t stored(int c) { return (uint32_t)(c + 128); }

__device__ inline uint32_t wave_max_u32(uint32_t x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint32_t y = (uint32_t)__shfl_xor((int)x, d, 64);
        x = y > x ? y : x;
    }
    return x;
}

// One wavefront writes the tokens that a call brings to one block, for one KV head and K or V: it needs no other's results.
// A lane has four tokens by eight dims of a piece of 16 tokens — the four tokens are the bytes of V's words, the eight dims
// one load of a row.
//   A wavefront looks at `span` rows of the slot map and takes up every run that begins there.
template <typename T, int D>
__global__ __launch_bounds__(256) void pq_paged_append_kernel(pq_paged_append_args a, int span, int n_spans)
{
    constexpr int GROUPS = D / 8, LANES = 4 * GROUPS, PIECES = 64 / LANES;  // lanes of a piece, pieces at a time
    const int lane = threadIdx.x & 63;
    const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int kind = unit & 1, h = (unit >> 1) % a.Hkv, part = (unit >> 1) / a.Hkv;
    if (part >= n_spans)
        return;
    const int block_tokens = 1 << a.log_block, n_slots = a.n_blocks << a.log_block;
    const T *x = (const T *)a.x[kind] + (int64_t)h * D;
    const int t0 = part * span;

    bool begins = false;
    if (lane < span && t0 + lane < a.n_tokens) {
        const int t = t0 + lane, now = a.slot[t], before = t > 0 ? a.slot[t - 1] : -2;
        if (now >= n_slots)
            paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
        else
            begins = now >= 0 && (before != now - 1 || (now & (block_tokens - 1)) == 0);
    }
    uint64_t runs = __ballot(begins);
    const int piece0 = lane / LANES, quad = lane % LANES / GROUPS, d0 = lane % GROUPS * 8;
    while (runs != 0) {
        const int t = t0 + __builtin_ctzll(runs);
        runs &= runs - 1;
        const int slot = __builtin_amdgcn_readfirstlane(a.slot[t]);
        const int block = slot >> a.log_block, from = slot & (block_tokens - 1);
        const bool follows = lane < block_tokens - from && t + lane < a.n_tokens && a.slot[t + lane] == slot + lane;
        const uint64_t stops = ~__ballot(follows);
        const int n = stops != 0 ? __builtin_ctzll(stops) : 64;
        const int upto = from + n;  // tokens [from, upto) of the block are new, those before are older

        // the largest |x|; as bits, so that a NaN is larger than any number
        uint32_t high = 0;
        for (int p = piece0 + (from >> 4) / PIECES * PIECES; p * 16 < upto; p += PIECES)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = p * 16 + quad * 4 + i;
                if (r < from || r >= upto)
                    continue;
                float v[8];
                paged_load8(x + (int64_t)(t + r - from) * a.stride + d0, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t bits = __float_as_uint(v[e]) & 0x7fffffffu;
                    high = bits > high ? bits : high;
                }
            }
        const float largest = __uint_as_float(wave_max_u32(high));
        float *const scale_at = a.scale[kind] + (int64_t)block * a.Hkv + h;
        const float was = from > 0 ? *scale_at : 0.0f;
        float s;
        if (!(largest <= FLT_MAX) || !(was <= FLT_MAX))
            s = __uint_as_float(0x7fc00000u);  // (codes 0)
        else
            s = fmaxf(fmaxf(largest, SMALLEST) / CODE_MAX, was);
        const bool finite = s <= FLT_MAX, grown = from > 0 && s > was;
        const float inv = finite ? 1.0f / s : 0.0f;

        uint8_t *const bytes = a.cache[kind] + ((int64_t)block * a.Hkv + h) * ((int64_t)D << a.log_block);
        const int first_piece = grown ? 0 : (from >> 4) / PIECES * PIECES;
        for (int p = piece0 + first_piece; p * 16 < upto; p += PIECES) {
            const int r0 = p * 16 + quad * 4;
            const bool some = r0 < upto && (grown || r0 + 4 > from);
            if (!some)
                continue;
            // codes of the 4 tokens' 8 dims as bytes, a word per dim; those that are not written keep what is there
            uint32_t words[8];
            const bool whole = r0 >= from && r0 + 4 <= upto;
            if (!whole) {
                if (kind == 0) {
                    uint2 rows[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        rows[i] = *(const uint2 *)(bytes + (r0 + i) * D + d0);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        words[e] = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            words[e] |= (((e < 4 ? rows[i].x : rows[i].y) >> (8 * (e & 3))) & 0xffu) << (8 * i);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        words[e] = *(const uint32_t *)(bytes + pq_paged_v_offset(r0, d0 + e, D));
                }
                if (grown)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (r0 + i < from)
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int c = (int)((words[e] >> (8 * i)) & 0xffu) - 128;
                                words[e] = (words[e] & ~(0xffu << (8 * i))) | (stored(regrown_code(c, was, s)) << (8 * i));
                            }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    words[e] = 0;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i;
                if (r < from || r >= upto)
                    continue;
                float v[8];
                paged_load8(x + (int64_t)(t + r - from) * a.stride + d0, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int c = finite ? (int)nearest_code(v[e], s, inv) : 0;
                    words[e] = (words[e] & ~(0xffu << (8 * i))) | (stored(c) << (8 * i));
                }
            }
            if (kind == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (r0 + i >= upto)
                        continue;
                    uint2 row = make_uint2(0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        row.x |= ((words[e] >> (8 * i)) & 0xffu) << (8 * e);
                        row.y |= ((words[e + 4] >> (8 * i)) & 0xffu) << (8 * e);
                    }
                    *(uint2 *)(bytes + (r0 + i) * D + d0) = row;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    *(uint32_t *)(bytes + pq_paged_v_offset(r0, d0 + e, D)) = words[e];
            }
        }
        if (lane == 0)
            *scale_at = s;
    }
}

// A lane reads four tokens by eight dims, the four that V's words hold, and writes their rows.
template <typename T, int D> __global__ __launch_bounds__(256) void pq_paged_read_kernel(pq_paged_read_args a, int quads)
{
    constexpr int GROUPS = D / 8;
    const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t per_head = (int64_t)quads * GROUPS;
    const int64_t head = unit / per_head;
    const int rest = (int)(unit - head * per_head);
    const int h = (int)(head % a.c.Hkv), kind = blockIdx.y;
    const int64_t b = head / a.c.Hkv;
    if (b >= a.n_seqs)
        return;
    const int len = paged_length(a.c, (int)b);
    int first = a.first != nullptr ? a.first[b] : 0;
    if (first < 0)
        first = 0;
    const int64_t last = (int64_t)first + a.n_rows < len ? (int64_t)first + a.n_rows : len;
    const int64_t p0 = (int64_t)(first & ~3) + 4 * (int64_t)(rest / GROUPS);
    const int d0 = rest % GROUPS * 8;
    if (p0 >= last)
        return;
    const int block = a.c.table[b * a.c.max_blocks + (p0 >> a.c.log_block)];
    if ((unsigned)block >= (unsigned)a.c.n_blocks) {
        paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
        return;
    }
    const int r0 = (int)(p0 & ((1 << a.c.log_block) - 1));
    const int64_t at = (int64_t)block * a.c.Hkv + h;
    const float s = (kind == 0 ? a.c.k_scale : a.c.v_scale)[at];
    const uint8_t *bytes = (kind == 0 ? a.c.k : a.c.v) + at * ((int64_t)D << a.c.log_block);
    uint32_t words[8];  // V: a word per dim; K: two per token
    if (kind == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 w = *(const uint2 *)(bytes + (r0 + i) * D + d0);
            words[2 * i] = w.x;
            words[2 * i + 1] = w.y;
        }
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            words[e] = *(const uint32_t *)(bytes + pq_paged_v_offset(r0, d0 + e, D));
    T *out = (T *)a.out[kind] + (b * a.c.Hkv + h) * (int64_t)a.n_rows * D;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t p = p0 + i;
        if (p < first || p >= last)
            continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t byte = kind == 0 ? words[2 * i + e / 4] >> (8 * (e & 3)) : words[e] >> (8 * i);
            v[e] = (float)((int)(byte & 0xffu) - 128) * s;
        }
        paged_store8(out + (p - first) * D + d0, v);
    }
}

}  // namespace

hipError_t pq_launch_paged_append(const pq_paged_ctx *ctx, const pq_paged_append_args &a, hipStream_t s)
{
    const int64_t per_row = 2 * (int64_t)a.Hkv;
    const int span = a.n_tokens * per_row <= 64 * (int64_t)ctx->n_cu ? 1 : ctx->cfg.block_tokens;
    const int n_spans = (a.n_tokens + span - 1) / span;
    const int64_t units = n_spans * per_row;
#define LAUNCH(T, D) \
    hipLaunchKernelGGL((pq_paged_append_kernel<T, D>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a, span, n_spans)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}

hipError_t pq_launch_paged_read(const pq_paged_ctx *ctx, const pq_paged_read_args &a, hipStream_t s)
{
    const int quads = a.n_rows / 4 + 2;  // the first row may lie anywhere in its four
    const int64_t threads = (int64_t)a.n_seqs * a.c.Hkv * quads * (ctx->cfg.head_dim / 8);
#define LAUNCH(T, D) \
    hipLaunchKernelGGL((pq_paged_read_kernel<T, D>), dim3((unsigned)((threads + 255) / 256), 2), dim3(256), 0, s, a, quads)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
