// pq_paged_plan: block tables, slots and the stack of free blocks from the requests' lengths.
//
// Two halves.  The first goes over the requests: running sums of the rows asked for and of the blocks given back, then (the
// sum of all blocks given back being known) of the blocks needed, which decide who gets them.  It is one workgroup's work,
// a chunk of 1024 requests at a time.  The second writes what is long — the blocks given back onto the stack, the new blocks
// into the tables, a slot per token —, every entry for itself: it finds its request by bisection of the running sums, which
// lie in LDS.  No entry that it reads is one that it writes: blocks pushed by this call and taken again by it are read where
// they come from, in the ended request's table.
//
// Bound by latency: a step of some hundred requests reads and writes a few KB.  Small calls run as one workgroup, one launch;
// calls with many tokens run the second half as a grid of its own.
#include <hip/hip_runtime.h>

#include "pq_paged.h"

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_WAVES = PLAN_THREADS / 64;

// inclusive sum over the workgroup's threads, and the total
__device__ int64_t scan_inclusive(int64_t x, int64_t *lds, int64_t &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(x, d, 64);
        if (lane >= d)
            x += y;
    }
    if (lane == 63)
        lds[wave] = x;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < PLAN_WAVES; ++w) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    __syncthreads();
    return x + before;
}

struct plan_shared {
    int64_t scan[PLAN_WAVES];
    int start[PQ_PAGED_MAX_SEQS + 1];
    int freed[PQ_PAGED_MAX_SEQS + 1];
    int taken[PQ_PAGED_MAX_SEQS + 1];
};

__device__ inline int clamp_length(int n, int most) { return n < 0 ? 0 : n > most ? most : n; }
__device__ inline int cap(int64_t x, int most) { return x > most ? most : (int)x; }

// The numbers of every request into the scratch arrays, and the outputs per request.
__device__ void plan_requests(const pq_paged_plan_args &a, plan_shared &s)
{
    const int most = a.max_blocks << a.log_block, round = (1 << a.log_block) - 1;
    int *old = a.scratch + PQ_PAGED_PLAN_OLD * a.scratch_stride;
    int *freed = a.scratch + PQ_PAGED_PLAN_FREED * a.scratch_stride;
    int *taken = a.scratch + PQ_PAGED_PLAN_TAKEN * a.scratch_stride;
    int *counts = a.scratch + PQ_PAGED_PLAN_COUNTS * a.scratch_stride;
    const int count = clamp_length(a.free_count[0], a.n_blocks);
    int64_t rows = 0, back = 0;  // of the requests before this chunk
    for (int b0 = 0; b0 < a.n_seqs; b0 += PLAN_THREADS) {
        const int b = b0 + threadIdx.x;
        int64_t asked = 0, gives = 0;
        int n = 0;
        if (b < a.n_seqs) {
            n = clamp_length(a.seq_len[b], most);
            asked = a.n_new[b] > 0 ? a.n_new[b] : 0;
            gives = a.n_new[b] < 0 ? (n + round) >> a.log_block : 0;
        }
        int64_t all_rows, all_back;
        const int64_t end = rows + scan_inclusive(asked, s.scan, all_rows);
        const int64_t given = back + scan_inclusive(gives, s.scan, all_back);
        if (b < a.n_seqs) {
            old[b] = n;
            freed[b] = cap(given - gives, a.n_blocks);
            a.tok_start[b] = cap(end - asked, a.n_tokens);
        }
        rows += all_rows;
        back += all_back;
    }
    const int there = cap(count + back, a.n_blocks);
    if (threadIdx.x == 0) {
        freed[a.n_seqs] = cap(back, a.n_blocks);
        a.tok_start[a.n_seqs] = cap(rows, a.n_tokens);
        counts[0] = count;
        counts[1] = there;
    }
    rows = 0;
    int64_t needed = 0;
    int highest = 0;  // blocks taken by the requests that this thread has granted, and all before them
    bool refused = false;
    for (int b0 = 0; b0 < a.n_seqs; b0 += PLAN_THREADS) {
        const int b = b0 + threadIdx.x;
        int64_t asked = 0, need = 0;
        int n = 0, n_new = 0;
        if (b < a.n_seqs) {
            n = old[b];  // (written by this thread)
            n_new = a.n_new[b];
            asked = n_new > 0 ? n_new : 0;
        }
        int64_t all_rows, all_need;
        const int64_t end = rows + scan_inclusive(asked, s.scan, all_rows);
        const bool fits = asked == 0 || (n + asked <= most && end <= a.n_tokens);
        if (fits)
            need = ((n + asked + round) >> a.log_block) - ((n + round) >> a.log_block);
        const int64_t upto = needed + scan_inclusive(need, s.scan, all_need);
        if (b < a.n_seqs) {
            const bool granted = fits && (need == 0 || upto <= there);
            if (granted && need > 0)
                highest = (int)upto;
            // no granted request follows a refused one that needs blocks, so the sums up to `there` are those of granted ones
            taken[b] = cap(upto - need, there);
            const int got = granted ? (int)asked : 0;
            a.tok_len[b] = got;
            a.new_seq_len[b] = n_new < 0 ? 0 : n + got;
            refused |= !granted;
        }
        rows += all_rows;
        needed += all_need;
    }
    // the largest `highest`
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_xor(highest, d, 64);
        highest = y > highest ? y : highest;
    }
    if ((threadIdx.x & 63) == 0)
        s.scan[threadIdx.x >> 6] = highest;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < PLAN_WAVES; ++w)
            highest = (int)s.scan[w] > highest ? (int)s.scan[w] : highest;
        taken[a.n_seqs] = highest;
        a.new_free_count[0] = there - highest;
    }
    if (refused)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_REFUSED);
}

// the last i of [0, n) with sums[i] <= x, for x >= sums[0] = 0
__device__ inline int owner(const int *sums, int n, int x)
{
    int low = 0, high = n;
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (sums[mid] <= x)
            low = mid;
        else
            high = mid;
    }
    return low;
}

// The i-th block that this call takes: it lies i below the top, among those pushed by this call or below them.
__device__ inline int nth_taken(const pq_paged_plan_args &a, const plan_shared &s, int i, int count, int there)
{
    const int e = there - 1 - i;
    if (e < count)
        return a.free_list[e];
    const int b = owner(s.freed, a.n_seqs, e - count);
    return a.table[(int64_t)b * a.max_blocks + (e - count - s.freed[b])];
}

// Threads first, first + step, .. of the second half; s.start, s.freed and s.taken are filled.
__device__ void plan_entries(const pq_paged_plan_args &a, const plan_shared &s, int first, int step)
{
    const int *old = a.scratch + PQ_PAGED_PLAN_OLD * a.scratch_stride;
    const int *counts = a.scratch + PQ_PAGED_PLAN_COUNTS * a.scratch_stride;
    const int count = counts[0], there = counts[1], round = (1 << a.log_block) - 1;
    for (int r = first; r < there - count; r += step) {
        const int b = owner(s.freed, a.n_seqs, r);
        a.free_list[count + r] = a.table[(int64_t)b * a.max_blocks + (r - s.freed[b])];
    }
    for (int i = first; i < s.taken[a.n_seqs]; i += step) {
        const int b = owner(s.taken, a.n_seqs, i);
        const int used = (old[b] + round) >> a.log_block;
        a.table[(int64_t)b * a.max_blocks + used + (i - s.taken[b])] = nth_taken(a, s, i, count, there);
    }
    bool range = false;
    for (int t = first; t < a.n_tokens; t += step) {
        int slot = -1;
        if (t < s.start[a.n_seqs]) {
            const int b = owner(s.start, a.n_seqs, t);
            if (a.tok_len[b] > 0) {
                const int p = old[b] + t - s.start[b], j = p >> a.log_block, used = (old[b] + round) >> a.log_block;
                const int block = j < used ? a.table[(int64_t)b * a.max_blocks + j]
                                           : nth_taken(a, s, s.taken[b] + j - used, count, there);
                if ((unsigned)block < (unsigned)a.n_blocks)
                    slot = (block << a.log_block) | (p & round);
                else
                    range = true;
            }
        }
        a.slot_map[t] = slot;
    }
    if (range)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
}

__device__ void load_sums(const pq_paged_plan_args &a, plan_shared &s)
{
    const int *freed = a.scratch + PQ_PAGED_PLAN_FREED * a.scratch_stride;
    const int *taken = a.scratch + PQ_PAGED_PLAN_TAKEN * a.scratch_stride;
    for (int b = threadIdx.x; b <= a.n_seqs; b += PLAN_THREADS) {
        s.start[b] = a.tok_start[b];
        s.freed[b] = freed[b];
        s.taken[b] = taken[b];
    }
    __syncthreads();
}

__global__ __launch_bounds__(PLAN_THREADS) void pq_paged_plan_kernel(pq_paged_plan_args a, bool entries)
{
    __shared__ plan_shared s;
    plan_requests(a, s);
    if (!entries)
        return;
    __syncthreads();  // (what this workgroup has written to memory is there for its own threads)
    load_sums(a, s);
    plan_entries(a, s, threadIdx.x, PLAN_THREADS);
}

__global__ __launch_bounds__(PLAN_THREADS) void pq_paged_plan_entries_kernel(pq_paged_plan_args a)
{
    __shared__ plan_shared s;
    load_sums(a, s);
    plan_entries(a, s, blockIdx.x * PLAN_THREADS + threadIdx.x, gridDim.x * PLAN_THREADS);
}

}  // namespace

hipError_t pq_launch_paged_plan(const pq_paged_ctx *ctx, const pq_paged_plan_args &a, hipStream_t s)
{
    const bool one = a.n_tokens <= 8 * PLAN_THREADS;
    hipLaunchKernelGGL(pq_paged_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, a, one);
    if (!one) {
        const int wanted = (a.n_tokens + PLAN_THREADS - 1) / PLAN_THREADS;
        hipLaunchKernelGGL(pq_paged_plan_entries_kernel, dim3(wanted < ctx->n_cu ? wanted : ctx->n_cu), dim3(PLAN_THREADS), 0, s, a);
    }
    return hipGetLastError();
}
