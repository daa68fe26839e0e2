// What the translation units of the paged 8-bit cache share (gfx950 only).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pq_internal.h"

#define PQ_PAGED_MAX_SEQS 4096
#define PQ_PAGED_MAX_TOKENS (1 << 20)
#define PQ_PAGED_ERRFLAG_REFUSED 1u
#define PQ_PAGED_ERRFLAG_RANGE 2u
#define PQ_PAGED_ERRFLAG_CLAIMS 4u
#define PQ_PAGED_ERRFLAG_HOLDERS 8u

// how pq_paged_decode's workgroups are cut out, and what they exchange through
struct pq_paged_decode_plan {
    float *partials;        // [head group][2 budget slots][sub_rows][d + 2]: base, sum, sums of values
    unsigned int *tickets;  // one per slot, zero between calls
    int n_sub, sub_rows;    // head groups of a KV head, and query heads of one (the last may have fewer)
    int budget;             // chunks per head group that a call's tokens are cut into
};

// How pq_paged_prefill shares out a call: sequences of at most few_rows rows (tokens times query heads of a KV head) in tiles of
// PQ_PAGED_FEW_ROWS, whose keys are cut into about `budget` pieces per KV head (0: not cut), the others in tiles of
// PQ_PAGED_TILE_ROWS.  Partials: for each KV head [2 budget slots][PQ_PAGED_FEW_ROWS][d + 2]: base, sum, sums of values.
#define PQ_PAGED_TILE_ROWS 256
#define PQ_PAGED_FEW_ROWS 32
struct pq_paged_prefill_plan {
    float *partials;
    int budget, few_rows;
};

struct pq_paged_ctx {
    pq_paged_config cfg;
    int log_block;          // log2(block_tokens)
    int n_cu;
    char *scratch;          // the allocation that the pointers below and in the plans point into
    pq_paged_decode_plan decode;
    pq_paged_prefill_plan prefill;
    int *plan;              // what the launches of pq_paged_plan, fork, free and compact hand over
    unsigned int *dev_err;  // sticky error word
};

// a cache as the kernels see it
struct pq_paged_view {
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    const int32_t *table;  // [n_seqs][max_blocks]
    const int32_t *seq_len;
    int n_blocks, max_blocks, log_block, Hkv;
    unsigned int *dev_err;
};

struct pq_paged_plan_args {
    const int32_t *n_new, *seq_len;
    int32_t *free_list;
    const int32_t *free_count;
    int32_t *table, *new_seq_len, *new_free_count, *tok_start, *tok_len, *slot_map;
    int *scratch;
    int n_seqs, n_tokens, n_blocks, max_blocks, log_block;
    unsigned int *dev_err;
};

struct pq_paged_append_args {
    const void *x[2];
    uint8_t *cache[2];
    float *scale[2];
    const int32_t *slot;
    int64_t stride;
    int n_tokens, n_blocks, log_block, Hkv;
    unsigned int *dev_err;
};

struct pq_paged_read_args {
    pq_paged_view c;
    const int32_t *first;  // or NULL
    void *out[2];
    int n_seqs, n_rows;
};

struct pq_paged_fork_args {
    const int32_t *parent, *keep;  // keep: or NULL
    const int32_t *seq_len, *free_list, *free_count;
    int32_t *table, *holders, *new_seq_len, *new_free_count, *copy_src, *copy_dst;
    int *scratch;
    int n_seqs, n_blocks, max_blocks, log_block;
    unsigned int *dev_err;
};

struct pq_paged_free_args {
    const int32_t *n_new, *seq_len;
    int32_t *free_list;
    const int32_t *free_count, *table;
    int32_t *holders, *new_seq_len, *new_free_count;
    int *scratch;
    int n_seqs, n_blocks, max_blocks, log_block;
    unsigned int *dev_err;
};

struct pq_paged_compact_args {
    const int32_t *seq_len, *free_list, *free_count, *table, *holders;
    int32_t *new_free_list, *new_free_count, *new_table, *new_holders, *moved_to, *copy_src, *copy_dst, *n_copies;
    int *scratch;
    int n_seqs, n_blocks, max_blocks, log_block;
    unsigned int *dev_err;
};

struct pq_paged_copy_args {
    const int32_t *src, *dst, *count;  // count: or NULL
    const uint8_t *from[2];
    const float *from_scale[2];
    uint8_t *to[2];
    float *to_scale[2];
    int64_t block_bytes;  // of K, and of V
    int n_pairs, n_from, n_to, Hkv;
    unsigned int *dev_err;
};

struct pq_paged_attn_args {
    pq_paged_view c;
    const void *q;
    void *out;
    int64_t q_stride;
    const int32_t *tok_start, *tok_len;  // NULL: one row per sequence, at its end
    float scale_log2e;
    int n_seqs, n_tokens, Hq, G;
};

int64_t pq_paged_plan_scratch_bytes();
hipError_t pq_launch_paged_plan(const pq_paged_ctx *ctx, const pq_paged_plan_args &a, hipStream_t s);
hipError_t pq_launch_paged_append(const pq_paged_ctx *ctx, const pq_paged_append_args &a, hipStream_t s);
hipError_t pq_launch_paged_read(const pq_paged_ctx *ctx, const pq_paged_read_args &a, hipStream_t s);
int64_t pq_paged_blocks_scratch_bytes();
hipError_t pq_launch_paged_fork(const pq_paged_fork_args &a, hipStream_t s);
hipError_t pq_launch_paged_free(const pq_paged_free_args &a, hipStream_t s);
hipError_t pq_launch_paged_compact(const pq_paged_compact_args &a, hipStream_t s);
hipError_t pq_launch_paged_copy(const pq_paged_copy_args &a, int n_cu, hipStream_t s);
pq_paged_decode_plan pq_paged_plan_decode(const pq_paged_config *cfg, int n_cu);
int64_t pq_paged_decode_slots(const pq_paged_config *cfg, const pq_paged_decode_plan &w);
int64_t pq_paged_decode_slot_floats(const pq_paged_config *cfg, const pq_paged_decode_plan &w);
hipError_t pq_launch_paged_decode(const pq_paged_ctx *ctx, const pq_paged_attn_args &a, hipStream_t s);
pq_paged_prefill_plan pq_paged_plan_prefill(const pq_paged_config *cfg, int n_cu);
int64_t pq_paged_prefill_floats(const pq_paged_config *cfg, const pq_paged_prefill_plan &w);
hipError_t pq_launch_paged_tiles(const pq_paged_attn_args &a, const pq_paged_prefill_plan &w, int dtype, int dim, int64_t entries, hipStream_t s);
hipError_t pq_launch_paged_prefill(const pq_paged_ctx *ctx, const pq_paged_attn_args &a, hipStream_t s);

// Byte of token r (of its block) and dim d in the V bytes of one block and head: pieces of 16 tokens, in each
// [d / 64][r / 4][d % 16][d / 16 % 4][r % 4].  The 16 bytes that share all but the last two are four dims' worth of four tokens:
// one load of a lane that holds, for a matrix instruction over tokens, dims 16 apart.
__host__ __device__ inline int pq_paged_v_offset(int r, int d, int dim)
{
    return (r >> 4) * (16 * dim) + (d >> 6) * 1024 + ((r >> 2) & 3) * 256 + (d & 15) * 16 + ((d >> 4) & 3) * 4 + (r & 3);
}


namespace {

template <typename T> struct paged_elem;
template <> struct paged_elem<__half> {
    static __device__ float up(__half x) { return __half2float(x); }
    static __device__ __half down(float x) { return __float2half_rn(x); }
};
template <> struct paged_elem<__hip_bfloat16> {
    static __device__ float up(__hip_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __hip_bfloat16 down(float x) { return __float2bfloat16(x); }
};
template <> struct paged_elem<float> {
    static __device__ float up(float x) { return x; }
    static __device__ float down(float x) { return x; }
};

// 8 values in a row, 16-byte aligned
template <typename T> struct __align__(16) paged_row8 {
    T x[8];
};

template <typename T> __device__ inline void paged_up8(const paged_row8<T> &r, float *x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = paged_elem<T>::up(r.x[i]);
}

template <typename T> __device__ inline void paged_load8(const T *p, float *x) { paged_up8(*(const paged_row8<T> *)p, x); }

template <typename T> __device__ inline void paged_store8(T *p, const float *x)
{
    paged_row8<T> r;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        r.x[i] = paged_elem<T>::down(x[i]);
    *(paged_row8<T> *)p = r;
}

__device__ inline int paged_length(const pq_paged_view &c, int b)
{
    const int n = c.seq_len[b], most = c.max_blocks << c.log_block;
    return n < 0 ? 0 : n > most ? most : n;
}

__device__ inline void paged_error(unsigned int *word, unsigned int flag) { atomicOr(word, flag); }

}  // namespace

#define PQ_PAGED_BY_TYPE(dtype, dim, LAUNCH)                                                              \
    do {                                                                                                  \
        if ((dim) == 128) {                                                                               \
            if ((dtype) == PQ_F16) { LAUNCH(__half, 128); }                                               \
            else if ((dtype) == PQ_BF16) { LAUNCH(__hip_bfloat16, 128); }                                 \
            else { LAUNCH(float, 128); }                                                                  \
        } else {                                                                                          \
            if ((dtype) == PQ_F16) { LAUNCH(__half, 64); }                                                \
            else if ((dtype) == PQ_BF16) { LAUNCH(__hip_bfloat16, 64); }                                  \
            else { LAUNCH(float, 64); }                                                                   \
        }                                                                                                 \
    } while (0)
