// pq_paged_append and pq_paged_read: values in and out of the blocks of the paged 8-bit cache.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "pq_device_utils.h"
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

// Largest |x| of values as bits, in which NaN is larger than any number; two 16-bit types a word at a time.
template <typename T> struct largest_bits {
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    pair high = {0, 0};
    __device__ void add(const paged_row8<T> &r)
    {
        uint4 w;
        __builtin_memcpy(&w, &r, sizeof(w));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t bits = comp(w, i) & 0x7fff7fffu;
            high = __builtin_elementwise_max(high, __builtin_bit_cast(pair, bits));
        }
    }
    __device__ float all() const
    {
        const uint16_t bits = (uint16_t)wave_max_u32(high.x > high.y ? high.x : high.y);
        return paged_elem<T>::up(__builtin_bit_cast(T, bits));
    }
};
template <> struct largest_bits<float> {
    uint32_t high = 0;
    __device__ void add(const paged_row8<float> &r)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __float_as_uint(r.x[i]) & 0x7fffffffu;
            high = bits > high ? bits : high;
        }
    }
    __device__ float all() const { return __uint_as_float(wave_max_u32(high)); }
};

// Stored bytes of 8 values as whole numbers in fp32, x / s + 128 rounded.  In one fma the quotient is at most 2^-15 off: where none
// of the eight is that near a tie they are right as they are, else (one group of a wavefront's in thirty) all are decided exactly.
template <typename T> __device__ inline void stored8(const paged_row8<T> &row, float s, float inv, float *out)
{
    float far = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = fmaf(paged_elem<T>::up(row.x[e]), inv, 128.0f);
        out[e] = rintf(y);
        far = fmaxf(far, fabsf(y - out[e]));
    }
    if (far > 0.5f - 0x1p-15f)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            out[e] = nearest_code(paged_elem<T>::up(row.x[e]), s, inv) + 128.0f;
}

// PER wavefronts write the tokens that a call brings to one block, for one KV head and K or V: they need no others' results.
// Each has a piece of the block, 16 tokens (two pieces of 64 dims), and a lane of it four tokens by eight dims — the four tokens
// are the bytes of V's words, the eight dims one load of a row —, kept from the search for the largest to the rounding: a
// value is read once.  V's words go through LDS, from where they leave 16 bytes a lane in a row.  A unit of wavefronts looks
// at `span` rows of the slot map and takes up every run that begins there.
//   Bound by HBM: a value is 2 or 4 bytes read and one written.  32K tokens x 32 heads in fp16 at 16 tokens a block: 318 us where
// the rows were read twice and V's words stored 4 bytes at a time, 250 us without that, 210 us with the slots read in one go.
template <typename T, int D, int PER>
__global__ __launch_bounds__(PER == 1 ? 256 : 64 * PER) void pq_paged_append_kernel(pq_paged_append_args a, int span, int n_spans)
{
    constexpr int GROUPS = D / 8, LANES = 4 * GROUPS, PIECES = 64 / LANES;  // lanes of a piece, pieces of a wavefront
    constexpr int UNITS = PER == 1 ? 4 : 1;                                  // of a workgroup
    __shared__ uint32_t words_of[UNITS * PER][PIECES][4 * D];                // V's words of a wavefront's pieces
    __shared__ uint32_t largest_of[2][PER];  // (as bits: a NaN is the largest)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int unit = blockIdx.x * UNITS + wave / PER, member = wave % PER;
    const int kind = unit & 1, h = (unit >> 1) % a.Hkv, part = (unit >> 1) / a.Hkv;
    if (part >= n_spans)
        return;
    const int block_tokens = 1 << a.log_block, n_slots = a.n_blocks << a.log_block;
    const T *x = (const T *)a.x[kind] + (int64_t)h * D;
    const int t0 = part * span;

    // the rows' slots, and behind them those that a run may go on in: all that the search for runs needs, in one go
    const auto slot_of = [&](int t) { return t < a.n_tokens ? a.slot[t] : -2; };
    const int here = slot_of(t0 + lane), beyond = span > 1 && block_tokens == 64 ? slot_of(t0 + 64 + lane) : -2;
    int before = __shfl_up(here, 1, 64);
    if (lane == 0)
        before = t0 > 0 ? a.slot[t0 - 1] : -2;
    bool begins = lane < span && here >= 0 && (before != here - 1 || (here & (block_tokens - 1)) == 0);
    if (begins && here >= n_slots) {
        begins = false;
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
    }
    uint64_t runs = __ballot(begins);
    const int p = member * PIECES + lane / LANES, quad = lane % LANES / GROUPS, d0 = lane % GROUPS * 8, r0 = p * 16 + quad * 4;
    for (int turn = 0; runs != 0; turn ^= 1) {
        const int first = __builtin_ctzll(runs), t = t0 + first;
        runs &= runs - 1;
        const int slot = __builtin_amdgcn_readlane(here, first);
        const int block = slot >> a.log_block, from = slot & (block_tokens - 1);
        const int same = __shfl(here, (first + lane) & 63, 64), later = __shfl(beyond, (first + lane) & 63, 64);
        const bool follows = lane < block_tokens - from && (first + lane < 64 ? same : later) == slot + lane;
        const uint64_t stops = ~__ballot(follows);
        const int n = stops != 0 ? __builtin_ctzll(stops) : 64;
        const int upto = from + n;  // tokens [from, upto) of the block are new, those before are older

        float *const scale_at = a.scale[kind] + (int64_t)block * a.Hkv + h;
        const float was = from > 0 ? *scale_at : 0.0f;
        paged_row8<T> rows[4];
        largest_bits<T> high;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r0 + i >= from && r0 + i < upto)
                rows[i] = *(const paged_row8<T> *)(x + (int64_t)(t + r0 + i - from) * a.stride + d0);
            else
                rows[i] = paged_row8<T>{};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            high.add(rows[i]);
        float largest = high.all();
        if constexpr (PER > 1) {
            if (lane == 0)
                largest_of[turn][member] = __float_as_uint(largest);
            __syncthreads();  // (also: everybody has read the block's scale before it is written, below)
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                bits = largest_of[turn][i] > bits ? largest_of[turn][i] : bits;
            largest = __uint_as_float(bits);
        }
        float s;
        if (!(largest <= FLT_MAX) || !(was <= FLT_MAX))
            s = __uint_as_float(0x7fc00000u);  // (codes 0)
        else
            s = fmaxf(fmaxf(largest, SMALLEST) / CODE_MAX, was);
        const bool finite = s <= FLT_MAX, grown = from > 0 && s > was;
        const float inv = finite ? 1.0f / s : 0.0f;

        uint8_t *const bytes = a.cache[kind] + ((int64_t)block * a.Hkv + h) * ((int64_t)D << a.log_block);
        if (grown)  // (rare, and kept small: unrolled it took half of the registers)
#pragma unroll 1
            for (int k = 0; k < 8 && r0 < from; ++k) {
                uint32_t *const at = (uint32_t *)(bytes + (kind == 0 ? (r0 + k / 2) * D + d0 + k % 2 * 4 : pq_paged_v_offset(r0, d0 + k, D)));
                if (kind == 0 && r0 + k / 2 >= from)
                    break;
                const uint32_t old = *at;
                uint32_t w = old;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (kind == 0 || r0 + i < from) {
                        const int c = (int)((old >> (8 * i)) & 0xffu) - 128;
                        w = (w & ~(0xffu << (8 * i))) | (stored(regrown_code(c, was, s)) << (8 * i));
                    }
                *at = w;
            }
        if (kind == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i;
                if (r < from || r >= upto)
                    continue;
                uint2 w = make_uint2(0x80808080u, 0x80808080u);
                if (finite) {
                    float b[8];
                    stored8<T>(rows[i], s, inv, b);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w.x = __builtin_amdgcn_cvt_pk_u8_f32(b[e], e, w.x);
                        w.y = __builtin_amdgcn_cvt_pk_u8_f32(b[e + 4], e, w.y);
                    }
                }
                *(uint2 *)(bytes + r * D + d0) = w;
            }
        } else {
            // quads of four tokens with new ones among them; an older token beside them keeps its byte
            const auto written = [&](int r) { return r < upto && r + 4 > from; };
            uint32_t words[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                words[e] = 0x80808080u;
            if (written(r0)) {
                if (r0 < from)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        words[e] = *(const uint32_t *)(bytes + pq_paged_v_offset(r0, d0 + e, D));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (r0 + i >= from && r0 + i < upto) {
                        float b[8];
                        if (finite)
                            stored8<T>(rows[i], s, inv, b);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            words[e] = __builtin_amdgcn_cvt_pk_u8_f32(finite ? b[e] : 128.0f, i, words[e]);
                    }
            }
            uint32_t *const room = words_of[wave][lane / LANES];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                room[pq_paged_v_offset(quad * 4, d0 + e, D) / 4] = words[e];
            __builtin_amdgcn_wave_barrier();  // (a wavefront's own LDS operations are in order)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int chunk = k * LANES + lane % LANES;  // 16 bytes of one quad: four tokens, four dims
                const uint4 w = ((const uint4 *)room)[chunk];
                if (written(p * 16 + chunk % 64 / 16 * 4))
                    *(uint4 *)(bytes + p * (16 * D) + chunk * 16) = w;
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (lane == 0 && member == 0)
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

namespace {

template <typename T, int D, int PER> void launch_append(const pq_paged_append_args &a, int span, int n_spans, hipStream_t s)
{
    const int64_t units = n_spans * 2 * (int64_t)a.Hkv;
    const dim3 grid((unsigned)(PER == 1 ? (units + 3) / 4 : units)), threads(PER == 1 ? 256 : 64 * PER);
    hipLaunchKernelGGL((pq_paged_append_kernel<T, D, PER>), grid, threads, 0, s, a, span, n_spans);
}

template <typename T, int D> void launch_append(int block_tokens, const pq_paged_append_args &a, int span, int n_spans, hipStream_t s)
{
    const int per = block_tokens * D / 2048;  // (16 tokens of 64 dims: half a wavefront)
    if constexpr (D == 128)
        if (per == 4)
            return launch_append<T, D, 4>(a, span, n_spans, s);
    if (per == 2)
        launch_append<T, D, 2>(a, span, n_spans, s);
    else
        launch_append<T, D, 1>(a, span, n_spans, s);
}

}  // namespace

// A unit a row (of K or V of a head) where there are few, so that the blocks of a step's many sequences are written side by
// side; else a unit a block's worth of rows, most of which begin no run.
hipError_t pq_launch_paged_append(const pq_paged_ctx *ctx, const pq_paged_append_args &a, hipStream_t s)
{
    const int span = a.n_tokens * 2 * (int64_t)a.Hkv <= 64 * (int64_t)ctx->n_cu ? 1 : ctx->cfg.block_tokens;
    const int n_spans = (a.n_tokens + span - 1) / span;
#define LAUNCH(T, D) launch_append<T, D>(ctx->cfg.block_tokens, a, span, n_spans, s)
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
