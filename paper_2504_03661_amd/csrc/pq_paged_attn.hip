// Attention over the paged 8-bit cache: one wavefront per query row and head, a token per lane for the scores, dims per lane
// for the values.
#include <hip/hip_runtime.h>

#include "pq_device_utils.h"
#include "pq_paged.h"

namespace {

template <typename T, int D> __global__ __launch_bounds__(64) void pq_paged_attn_kernel(pq_paged_attn_args a)
{
    __shared__ float qs[D], weights[64];
    __shared__ int at[64];
    const int lane = threadIdx.x, head = blockIdx.y, h = head / a.G;
    int row = blockIdx.x, b = blockIdx.x;
    int n;
    if (a.tok_start != nullptr) {
        for (b = 0; b < a.n_seqs; ++b)
            if (row >= a.tok_start[b] && (int64_t)row < (int64_t)a.tok_start[b] + a.tok_len[b])
                break;
        if (b == a.n_seqs)
            return;
        n = paged_length(a.c, b) - a.tok_len[b] + (row - a.tok_start[b]) + 1;
    } else {
        n = paged_length(a.c, b);
    }
    const T *q = (const T *)a.q + (int64_t)row * a.q_stride + (int64_t)head * D;
    for (int d = lane; d < D; d += 64)
        qs[d] = paged_elem<T>::up(q[d]);
    __syncthreads();
    float top = NEG_BIG, sum = 0.0f, acc[D / 64] = {};
    for (int t0 = 0; t0 < n; t0 += 64) {
        const int t = t0 + lane;
        int block = -1;
        if (t < n)
            block = a.c.table[(int64_t)b * a.c.max_blocks + (t >> a.c.log_block)];
        if (t < n && (unsigned)block >= (unsigned)a.c.n_blocks) {
            paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
            block = -1;
        }
        const int r = t & ((1 << a.c.log_block) - 1);
        float score = -INFINITY, v_scale = 0.0f;
        if (block >= 0) {
            const int64_t place = (int64_t)block * a.c.Hkv + h;
            const uint8_t *k = a.c.k + (place << a.c.log_block) * D + r * D;
            float dot = 0.0f;
            for (int d = 0; d < D; ++d)
                dot += qs[d] * (float)((int)k[d] - 128);
            score = dot * a.c.k_scale[place] * a.scale_log2e;
            v_scale = a.c.v_scale[place];
        }
        const float high = fmaxf(top, wave_max(score));
        const float down = exp2f(top - high);
        const float p = block >= 0 ? exp2f(score - high) : 0.0f;
        top = high;
        sum = sum * down + wave_sum(p);
        weights[lane] = p * v_scale;
        at[lane] = block;
        __syncthreads();
        for (int i = 0; i < D / 64; ++i) {
            acc[i] *= down;
            const int d = lane + 64 * i;
            for (int j = 0; j < 64; ++j)
                if (at[j] >= 0) {
                    const int64_t place = (int64_t)at[j] * a.c.Hkv + h;
                    const int rr = (t0 + j) & ((1 << a.c.log_block) - 1);
                    const uint8_t *v = a.c.v + (place << a.c.log_block) * D;
                    acc[i] += weights[j] * (float)((int)v[pq_paged_v_offset(rr, d, D)] - 128);
                }
        }
        __syncthreads();
    }
    T *out = (T *)a.out + ((int64_t)row * a.Hq + head) * D;
    for (int i = 0; i < D / 64; ++i)
        out[lane + 64 * i] = paged_elem<T>::down(sum == 0.0f ? 0.0f : acc[i] / sum);
}

}  // namespace

hipError_t pq_launch_paged_attn(const pq_paged_ctx *ctx, const pq_paged_attn_args &a, hipStream_t s)
{
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_attn_kernel<T, D>), dim3(a.n_tokens, a.Hq), dim3(64), 0, s, a)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
