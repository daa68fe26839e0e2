// Pieces that the two attention kernels over the paged 8-bit cache share (gfx950).
//
// Both form scores and values with fp16 matrix instructions.  A code is an integer of at most 7 bits and sign: exact in fp16.  A
// query row is multiplied by a power of two that brings its largest element to [2^13, 2^14) and rounded to fp16: what is 11 or
// fewer bits wide (fp16, bf16) stays exact down to 2^-27 of the row's largest element; fp32 rows are split into two fp16
// parts, 22 bits.  Products and sums are fp32.  A block's key scale multiplies the finished dot product; its value scale goes into
// the weights' exponent:
//     s_t = log2(e) scale q.k_t + log2(v_scale_t),   w_t = 2^(s_t - base),   out = sum_t w_t code_t / sum_t w_t / v_scale_t
// with the base 13 to 15 below the largest s_t, so that the weights that are multiplied by codes — rounded to fp16 (fp32 contexts: to two parts): a
// matrix instruction in fp32 has a sixteenth of the rate — keep 11 bits down to 2^-27 of the largest and never leave fp16's range.
// That is all the first sum needs, in which a weight counts by the size of its values.  In the second it counts by the softmax
// alone, however small its values are (a block of zeros has the scale 2^-40): that sum is taken of the weights in fp32, before they are
// rounded.  There they count down to 2^-126 of the largest (the range of the factors by which sums follow the maximum).
#pragma once

#include <cfloat>

#include "pq_device_utils.h"
#include "pq_paged.h"

namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half4v __attribute__((ext_vector_type(4)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float WEIGHT_BITS = 13.0f;  // log2 of the weight of the largest score when it sets a row's base
constexpr float MOST_BITS = 15.0f;    // .. and of one above which the base is moved: fp16 holds what is below 2^16
constexpr float LOWEST = -FLT_MAX;     // the base of a row that has seen nothing

// What a row's weights are measured from, 2^(s - base), if its largest score is s: 13 below it, and from 2^22 on, where s less 13
// is rounded — by more than fp16 leaves room for soon —, s itself.
__device__ inline float weight_base(float s) { return fabsf(s) < 0x1p22f ? s - WEIGHT_BITS : s; }

// Four bytes (code + 128) as fp16 codes: 0x6400 | byte is 1024 + byte, and 1152 less is the code.
__device__ inline half4v codes4(uint32_t w)
{
    const half2v bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    const half2v lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - bias;
    const half2v hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - bias;
    return half4v{lo.x, lo.y, hi.x, hi.y};
}

__device__ inline half8v codes8(uint32_t w0, uint32_t w1)
{
    const half4v a = codes4(w0), b = codes4(w1);
    return half8v{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}

// A block's value scale: never below 2^-40, which a block that nothing was written to would be (a NaN stays).
__device__ inline float value_scale(float v) { return v < 0x1p-40f ? 0x1p-40f : v; }

// The exponent by which a row of queries is scaled, from its largest |element|: that has 13 afterwards, subnormal or not.  (A row of
// zeros gets the largest there is: no scale then makes anything but 0 of its scores.)
__device__ inline int query_exponent(float largest)
{
    const uint32_t bits = __float_as_uint(largest);
    return (bits >> 23) != 0 ? 13 + 127 - (int)(bits >> 23) : 13 + 149 - 31 + __builtin_clz(bits | 1u);
}

// What a lane keeps of 64 blocks in a row of a sequence
struct block_batch {
    int first;  // number of the first one in the sequence
    int id;     // 0 where there is none
    float k_scale, v_log, v_inv;
};

// The first half: block numbers, and the scales on their way, which a block's bytes need not wait for (v_log has V's).
__device__ inline void start_batch(const pq_paged_view &c, const int32_t *table, int first, int last, int h, int lane, block_batch &x)
{
    x.first = first;
    const int j = first + lane;
    int id = j < last ? table[j] : -1;
    const bool there = (unsigned)id < (unsigned)c.n_blocks;
    if (j < last && !there)
        paged_error(c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
    x.id = there ? id : 0;
    x.k_scale = 0.0f;  // no such block: every score is -inf, every weight 0
    x.v_log = -INFINITY;
    if (there) {
        const int64_t at = (int64_t)id * c.Hkv + h;
        x.k_scale = c.k_scale[at];
        x.v_log = c.v_scale[at];
    }
}

// The second half
__device__ inline void finish_batch(block_batch &x)
{
    const bool there = x.v_log != -INFINITY;
    const float v = value_scale(x.v_log);
    x.v_log = there ? __log2f(v) : -INFINITY;
    x.v_inv = there && v <= FLT_MAX ? 1.0f / v : 0.0f;  // (a NaN is in v_log: a row that does not see the block adds 0 times this)
}

__device__ inline block_batch load_batch(const pq_paged_view &c, const int32_t *table, int first, int last, int h, int lane)
{
    block_batch x;
    start_batch(c, table, first, last, h, lane, x);
    finish_batch(x);
    return x;
}

__device__ inline float lane_of(float x, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); }

template <int CTRL, int ROW_MASK> __device__ inline int dpp_or_zero(int x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROW_MASK, 0xf, false);
}

// sum over the wavefront's lanes before this one and itself
__device__ inline int lane_scan(int x)
{
    x += dpp_or_zero<0x111, 0xf>(x);  // one lane up within the row of 16
    x += dpp_or_zero<0x112, 0xf>(x);
    x += dpp_or_zero<0x114, 0xf>(x);
    x += dpp_or_zero<0x118, 0xf>(x);
    x += dpp_or_zero<0x142, 0xa>(x);  // the last lane of rows 0 and 2 to rows 1 and 3
    x += dpp_or_zero<0x143, 0xc>(x);  // the last lane of row 1 to rows 2 and 3
    return x;
}

// Tokens of a piece if `total` is cut into `budget` pieces.  (The total is a sum in fp32: the length is taken a little larger, so
// that the pieces are not more.)
__device__ inline int piece_tokens(float total, int budget, int align, int least)
{
    const float share = total * 1.0001f / (float)budget;
    const int n = share < (float)PQ_MAX_TOKENS ? (int)share + 1 : PQ_MAX_TOKENS;
    return n > least ? (n + align - 1) / align * align : least;
}

}  // namespace
