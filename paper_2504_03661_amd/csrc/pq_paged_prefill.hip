// pq_paged_prefill: causal attention of many query tokens per sequence over the paged 8-bit cache.
//
// A workgroup has one sequence, one KV head and a tile of query rows — a token's query heads of that KV head lie side by side,
// so a tile of 256 rows is 64 tokens of 4 heads — and walks the keys that the tile sees, 64 at a time.  Bytes become fp16 codes
// once per tile, on their way into LDS, and are then the left operands of 32x32x16 matrix instructions for all of the
// workgroup's wavefronts, 32 rows each: S^T = K Q^T, and O^T = V^T W with the weights straight from the registers that the
// scores came in (V's tokens lie in LDS in the order in which the result of the first product holds them).  A lane has one query
// row: its maximum, sum, limit and rescaling are its own.
//
// Bound by the issue of matrix and vector instructions, which two wavefronts of a SIMD overlap only in part, and by waits: a
// prompt of 8K tokens, 32 query / 8 KV heads of 128 dims in bf16, takes 580 to 590 us (932 to 948 TFLOP/s; matrix units busy 42 % of
// the time, vector units 50 %, 40 % of the wavefronts' cycles are waits), in fp32, with operands in two parts, 963 us.
// Without its exponentials it would take 20 us less, without the conversion of bytes 61, without the search for the maximum
// 50, without the second product 156: no one of them stands out.  (Sums of weights before their rounding instead of after: no
// change, 580 and 583 us.  The way for scores beyond 2^22 costs the others 0.3 %.)
#include <hip/hip_runtime.h>

#include "pq_paged_work.h"

namespace {

constexpr int V_PLANE = 16;  // bytes of 8 tokens of one dim

// How a workgroup is made up: WAVES wavefronts of NT times 32 rows each, and tiles of KEYS keys
template <int D_, int NT_, int WAVES_, int KEYS_> struct shape {
    static constexpr int D = D_, NT = NT_, WAVES = WAVES_, KEYS = KEYS_, THREADS = 64 * WAVES, ROWS = 32 * NT * WAVES;
    static constexpr int LOADS = KEYS * D / (THREADS * 16);  // 16-byte loads a thread makes of K, and of V
    static constexpr int K_PLANE = KEYS * 16 + 16;           // bytes of 8 dims of all keys, and a shift of 4 banks
    static_assert(LOADS >= 1 && KEYS * D % (THREADS * 16) == 0 && (KEYS == 64 || KEYS == 128));
};

template <typename S> struct tile_lds {
    unsigned char k[S::D / 8 * S::K_PLANE];                  // [dim / 8][key][dim % 8]
    unsigned char v[S::KEYS / 16 * 2 * S::D * V_PLANE];      // [piece][half of its tokens][dim][8 tokens]
    float k_scale[S::KEYS / 16], v_log[S::KEYS / 16], v_inv[S::KEYS / 16];
};

// A wavefront's share of a tile of keys, as bytes on their way to LDS
template <typename S> struct key_bytes {
    u32x4 k[S::LOADS], v[S::LOADS];
};

// the piece of 16 tokens that load x of a wavefront lies in
template <typename S> __device__ inline int piece_of(int wave, int x) { return (wave * 64 + S::THREADS * x) / S::D; }

template <typename S>
__device__ inline void load_keys(const pq_paged_view &c, const block_batch &batch, int h, int t, int wave, int lane, key_bytes<S> &to)
{
#pragma unroll
    for (int x = 0; x < S::LOADS; ++x) {
        const int piece = piece_of<S>(wave, x), p = t + 16 * piece;
        const int id = __builtin_amdgcn_readlane(batch.id, (p >> c.log_block) - batch.first);
        const int64_t base = (((int64_t)id * c.Hkv + h) << c.log_block) * S::D + (p & ((1 << c.log_block) - 1)) * S::D;
        // within the piece: K's 16-byte parts of rows, and V's words
        const int at = (wave * 64 + S::THREADS * x - piece * S::D + lane) * 16;
        to.k[x] = *(const u32x4 *)(c.k + base + at);
        to.v[x] = *(const u32x4 *)(c.v + base + at);
    }
}

template <typename S>
__device__ inline void store_keys(tile_lds<S> &lds, const block_batch &batch, int log_block, int t, int wave, int lane,
                                  const key_bytes<S> &from)
{
    constexpr int D = S::D;
    if (wave == 0) {
        const int at = ((t + 16 * (lane & (S::KEYS / 16 - 1))) >> log_block) - batch.first;
        const float k_scale = __shfl(batch.k_scale, at, 64), v_log = __shfl(batch.v_log, at, 64), v_inv = __shfl(batch.v_inv, at, 64);
        if (lane < S::KEYS / 16) {
            lds.k_scale[lane] = k_scale;
            lds.v_log[lane] = v_log;
            lds.v_inv[lane] = v_inv;
        }
    }
#pragma unroll
    for (int x = 0; x < S::LOADS; ++x) {
        const int id = wave * 64 + lane + S::THREADS * x, key = id / (D / 16), part = id % (D / 16);
        *(half8v *)(lds.k + (2 * part) * S::K_PLANE + key * 16) = codes8(from.k[x][0], from.k[x][1]);
        *(half8v *)(lds.k + (2 * part + 1) * S::K_PLANE + key * 16) = codes8(from.k[x][2], from.k[x][3]);
        const int piece = piece_of<S>(wave, x), at = id - piece * D, quad = (at >> 4) & 3, dim0 = (at >> 6) * 64 + (at & 15);
        unsigned char *v = lds.v + (piece * 2 + (quad & 1)) * (D * V_PLANE) + (quad >> 1) * 8;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *(half4v *)(v + (dim0 + 16 * k) * V_PLANE) = codes4(from.v[x][k]);
    }
}

// What a wavefront keeps of its rows; a lane has row 32 n + lane % 32 of them, and dims or keys by its half
template <typename S, int PARTS> struct row_state {
    half8v q[S::NT][PARTS][S::D / 16];
    f32x16 o[S::D / 32][S::NT];
    float per_score[S::NT], base[S::NT], l[S::NT];
    float most[S::NT];  // the exponent of a weight above which the base is moved
    int sees[S::NT];  // keys that the row attends over
};

// K's rows of 32 keys, part u of a tile, against the queries: a lane gets keys 8 (j / 4) + 4 half + j % 4 for its query row
template <typename S, int PARTS>
__device__ inline void dots_32(const row_state<S, PARTS> &r, const tile_lds<S> &tile, int u, int col, int half, f32x16 (&dot)[S::NT])
{
#pragma unroll
    for (int n = 0; n < S::NT; ++n)
#pragma unroll
        for (int j = 0; j < 16; ++j)
            dot[n][j] = 0.0f;
#pragma unroll
    for (int x = 0; x < S::D / 16; ++x) {
        const half8v k = *(const half8v *)(tile.k + (2 * x + half) * S::K_PLANE + (32 * u + col) * 16);
#pragma unroll
        for (int n = 0; n < S::NT; ++n)
#pragma unroll
            for (int i = 0; i < PARTS; ++i)
                dot[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, r.q[n][i][x], dot[n], 0, 0, 0);
    }
}

template <typename S, int PARTS> struct part_weights {
    half8v w[S::NT][PARTS][2];
};

// .. and the weights of 32 keys times their values
template <typename S, int PARTS>
__device__ inline void values_32(row_state<S, PARTS> &r, const tile_lds<S> &tile, int u, int col, int half, const part_weights<S, PARTS> &w)
{
#pragma unroll
    for (int i = 0; i < S::D / 32; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const half8v v = *(const half8v *)(tile.v + ((2 * u + x) * 2 + half) * (S::D * V_PLANE) + (32 * i + col) * V_PLANE);
#pragma unroll
            for (int n = 0; n < S::NT; ++n)
#pragma unroll
                for (int j = 0; j < PARTS; ++j)
                    r.o[i][n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, w.w[n][j][x], r.o[i][n], 0, 0, 0);
        }
}

// One step of a wavefront: the weights of 32 keys (from key t of the sequence on) out of their dot products, while the matrix
// unit is at the dot products of the 32 keys after them and the values of those before — neither waits for this step's vector
// instructions, and so both units are kept busy by one instruction stream.
template <typename S, int PARTS, bool MASKED>
__device__ inline void step_32(row_state<S, PARTS> &r, const tile_lds<S> &next, int next_u, const tile_lds<S> &before, int before_u,
                               const tile_lds<S> &now, int u, int t, int col, int half, f32x16 (&dot)[S::NT],
                               part_weights<S, PARTS> &w)
{
    constexpr int D = S::D, NT = S::NT;
    f32x16 dot_next[NT];
    float k_scale[2], v_log[2], v_inv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        k_scale[i] = now.k_scale[2 * u + i];
        v_log[i] = now.v_log[2 * u + i];
        v_inv[i] = now.v_inv[2 * u + i];
    }
    // Exponents of the weights, s - base: one fma of a dot product, of which the largest decides whether the base stays.  The fma does
    // not round the product, as the score was that became the base.  Beyond 2^22 that is a matter of half a unit and more:
    // there every step goes the other way, by scores that are rounded, so that scores alike have weights alike.
    float e[NT][16];
    auto exponents = [&](int n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float by = r.per_score[n] * k_scale[i], off = v_log[i] - r.base[n];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                e[n][8 * i + j] = fmaf(dot[n][8 * i + j], by, off);
        }
        if (MASKED)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (t + 8 * (j >> 2) + 4 * half + (j & 3) >= r.sees[n])
                    e[n][j] = -INFINITY;
        float high = e[n][0];
#pragma unroll
        for (int j = 1; j < 16; ++j)
            high = fmaxf(high, e[n][j]);
        return high;
    };
    values_32<S, PARTS>(r, before, before_u, col, half, w);
    bool moves = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
        moves |= exponents(n) > r.most[n];
    if (__ballot(moves) != 0) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // (from the scores themselves: the base of a row that has seen nothing is too large to be subtracted and added again)
            const float was = r.base[n];
            r.base[n] = 0.0f;
            float high = exponents(n);
            high = fmaxf(high, __shfl_xor(high, 32, 64));
            const float base = fmaxf(was, weight_base(high)), down = __builtin_amdgcn_exp2f(was - base);
            r.base[n] = base;
            r.most[n] = fabsf(base) < 0x1p22f ? MOST_BITS : -INFINITY;
            r.l[n] *= down;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    r.o[i][n][j] *= down;
#pragma unroll
            for (int j = 0; j < 16; ++j)
                e[n][j] -= base;
        }
    }
    dots_32<S, PARTS>(r, next, next_u, col, half, dot_next);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float x = __builtin_amdgcn_exp2f(e[n][8 * i + j]), y = __builtin_amdgcn_exp2f(e[n][8 * i + j + 1]);
                // (before they are rounded: a weight is as large as its block's values are, and one that fp16 has no
                // number for counts in the sum as much as any other)
                sum += x + y;
                const half2v both = {(_Float16)x, (_Float16)y};
                w.w[n][0][i][j] = both.x;
                w.w[n][0][i][j + 1] = both.y;
                if (PARTS == 2) {
                    w.w[n][PARTS - 1][i][j] = (_Float16)(x - (float)both.x);
                    w.w[n][PARTS - 1][i][j + 1] = (_Float16)(y - (float)both.y);
                }
            }
            r.l[n] = fmaf(sum, v_inv[i], r.l[n]);
        }
#pragma unroll
    for (int n = 0; n < NT; ++n)
        dot[n] = dot_next[n];
}

template <typename T, typename S>
__global__ __launch_bounds__(S::THREADS, 2) void pq_paged_prefill_kernel(pq_paged_attn_args a, pq_paged_prefill_plan w)
{
    constexpr bool SPLIT = sizeof(T) == 4;  // two fp16 parts of queries and weights
    constexpr int PARTS = SPLIT ? 2 : 1, D = S::D, NT = S::NT, DT = D / 32, TILE_ROWS = S::ROWS, KEYS = S::KEYS;
    constexpr int BUFFERS = 3;
    __shared__ tile_lds<S> lds[BUFFERS];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int h = blockIdx.x % a.c.Hkv, entry = blockIdx.x / a.c.Hkv;
    if (blockIdx.x == gridDim.x - 1) {  // (one more than the list has)
        if (wave == 0)
            check_claims(a, lane);
        return;
    }
    work_place p;
    if (!find_work(a, tile_rule(w), entry, lane, p))
        return;
    const int col = lane & 31, half = lane >> 5;
    const tile_place tile(p, a.G, TILE_ROWS);
    const int past = p.past, row0 = tile.row0, all_rows = row0 + tile.rows, k1 = tile.sees;

    // this lane's rows
    row_state<S, PARTS> rows;
    int token[NT], head[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = row0 + (wave * NT + n) * 32 + col;
        const bool there = r < all_rows;
        token[n] = there ? r / a.G : -1;
        head[n] = there ? r - token[n] * a.G : 0;
        const int sees = there ? past + token[n] + 1 : 0;
        rows.sees[n] = sees < k1 ? sees : k1;
        rows.base[n] = LOWEST;
        rows.most[n] = MOST_BITS;
        rows.l[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                rows.o[i][n][j] = 0.0f;
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
        rows.per_score[n] = ldexpf(a.scale_log2e, -e);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = ldexpf(v[8 * x + j], e);
                rows.q[n][0][x][j] = (_Float16)f;
                if (SPLIT)
                    rows.q[n][PARTS - 1][x][j] = (_Float16)(f - (float)rows.q[n][0][x][j]);
            }
    }
    // what the wavefront's first and last rows see: keys below the one need no mask, keys from the other on no work
    const int wave_first = row0 + wave * NT * 32, wave_last = wave_first + NT * 32 - 1;
    const int wave_least = wave_last < all_rows ? past + wave_first / a.G + 1 : 0;
    int wave_sees = wave_first < all_rows ? past + (wave_last < all_rows ? wave_last : all_rows - 1) / a.G + 1 : 0;
    wave_sees = __builtin_amdgcn_readfirstlane(wave_sees < k1 ? wave_sees : k1);

    const int32_t *table = a.c.table + (int64_t)p.b * a.c.max_blocks;
    const int last_block = (p.len + (1 << a.c.log_block) - 1) >> a.c.log_block, per_tile = KEYS >> a.c.log_block;
    // Three tiles in LDS: the one whose keys are scored, the one whose values were not all used yet, the one that is filled.
    // A tile is stored after the barrier behind which nobody reads the tile it takes the place of, and read after the next.
    constexpr int PARTS_32 = KEYS / 32;
    key_bytes<S> bytes;
    block_batch batch;
    f32x16 dot[NT];
    part_weights<S, PARTS> weights;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                weights.w[n][i][0][j] = weights.w[n][i][1][j] = (_Float16)0.0f;
    auto load = [&](int t) {
        const int j = t >> a.c.log_block;
        if (j + per_tile > batch.first + 64)
            batch = load_batch(a.c, table, j, last_block, h, lane);
        load_keys<S>(a.c, batch, h, t, wave, lane, bytes);
    };
    if (k1 > 0) {
        batch.first = -65;
        load(0);
        store_keys<S>(lds[0], batch, a.c.log_block, 0, wave, lane, bytes);
        if (KEYS < k1)
            load(KEYS);
        __syncthreads();
        dots_32<S, PARTS>(rows, lds[0], 0, col, half, dot);
    }
    // (in a vector register, and so is the branch on it: as a uniform one the compiler moves so much across it that the kernel
    // takes 256 registers and spills 40 of them, 8K prompt 930 us instead of 597)
    int part_end = wave_least < k1 ? wave_least : k1;
    asm volatile("" : "+v"(part_end));
    int last = k1;
    asm volatile("" : "+v"(last));
    int at = 0, before = 0;  // the tile's place in LDS, and that of the tile in front of it
    // one step behind the last that the wavefront's rows see: it adds that one's values, and its own weights are all 0
    const int wave_end = wave_sees > 0 ? (wave_sees + 31) / 32 * 32 + 32 : 0;
    for (int t = 0; t < last; t += KEYS) {
        const int next = at == BUFFERS - 1 ? 0 : at + 1;
#pragma unroll
        for (int u = 0; u < PARTS_32; ++u) {
            const int part = t + 32 * u, next_u = u + 1 < PARTS_32 ? u + 1 : 0, before_u = u > 0 ? u - 1 : PARTS_32 - 1;
            const tile_lds<S> &of_next = lds[u + 1 < PARTS_32 ? at : next], &of_before = lds[u > 0 ? at : before];
            if (u + 1 == PARTS_32) {
                if (t + KEYS < k1)
                    store_keys<S>(lds[next], batch, a.c.log_block, t + KEYS, wave, lane, bytes);
                if (t + 2 * KEYS < k1)
                    load(t + 2 * KEYS);
                __syncthreads();
            }
            if (part + 32 <= part_end)
                step_32<S, PARTS, false>(rows, of_next, next_u, of_before, before_u, lds[at], u, part, col, half, dot, weights);
            else if (part < wave_end)
                step_32<S, PARTS, true>(rows, of_next, next_u, of_before, before_u, lds[at], u, part, col, half, dot, weights);
        }
        before = at;
        at = next;
    }
    if (k1 > 0)
        values_32<S, PARTS>(rows, lds[before], PARTS_32 - 1, col, half, weights);

#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float sum = rows.l[n] + __shfl_xor(rows.l[n], 32, 64);
        if (token[n] < 0)
            continue;
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        T *out = (T *)a.out + ((int64_t)(p.first_row + token[n]) * a.Hq + h * a.G + head[n]) * D + 4 * half;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                T x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = paged_elem<T>::down(rows.o[i][n][j + e] * by);
                __builtin_memcpy(out + 32 * i + 2 * j, x, sizeof(x));
            }
    }
}

}  // namespace

// Tiles of 256 rows, one workgroup a compute unit; 64 keys of 128 dims (128 of 64), 16 KiB of fp16 each of K and V.
hipError_t pq_launch_paged_tiles(const pq_paged_attn_args &a, const pq_paged_prefill_plan &w, int dtype, int dim, int64_t tiles, hipStream_t s)
{
#define LAUNCH(T, D)                                                                                                          \
    do {                                                                                                                      \
        using S = shape<D, 1, PQ_PAGED_TILE_ROWS / 32, 64 * 128 / D>;                                                         \
        hipLaunchKernelGGL((pq_paged_prefill_kernel<T, S>), dim3((unsigned)(tiles * a.c.Hkv) + 1), dim3(S::THREADS), 0, s, a, w); \
    } while (0)
    PQ_PAGED_BY_TYPE(dtype, dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
