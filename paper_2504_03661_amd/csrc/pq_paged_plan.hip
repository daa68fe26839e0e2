// pq_paged_plan: block tables, slots and the stack of free blocks from the requests' lengths.
//
// Two halves.  The first goes over the requests: running sums of the rows asked for and of the blocks given back, then (the
// sum of all blocks given back being known) of the blocks needed, which decide who gets them.  It is one workgroup's work,
// a chunk of 1024 requests at a time.  The second writes what is long — the blocks given back onto the stack, the new blocks
// into the tables, a slot per token —, every entry for itself: it finds its request by bisection of the running sums, which
// lie in LDS.  No entry that it reads is one that it writes: blocks pushed by this call and taken again by it are read where
// they come from, in the ended request's table.
//
// Bound by latency: a step of some hundred requests reads and writes a few KB, one load after another.  A call of up to 8192
// tokens is one launch of one workgroup, whose wavefronts do the three kinds of entries side by side; with more tokens the
// second half is a grid of its own (64 requests, one token each: 5.2 us, 8.8 with the sums
// in memory and the entries one kind after another; 1000 requests with 114K tokens: 13.2 us).
#include <hip/hip_runtime.h>

#include "pq_paged_scan.h"

namespace {

constexpr int PLAN_THREADS = SCAN_THREADS;
constexpr int PLAN_WAVES = SCAN_WAVES;

// the numbers of every request, and behind the last one their sums
struct plan_sums {
    int old[PQ_PAGED_MAX_SEQS + 1];    // length before
    int start[PQ_PAGED_MAX_SEQS + 1];  // rows of the requests before this one
    int freed[PQ_PAGED_MAX_SEQS + 1];  // blocks given back by them
    int taken[PQ_PAGED_MAX_SEQS + 1];  // blocks taken by them
    int got[PQ_PAGED_MAX_SEQS];        // tokens that have a place
    int count, there;                  // free blocks before the call, and after the pushes
};

// The first half.  All sums are kept in 32 bits: what a request adds is limited to 2^20 + 1 (more rows than a call can have, all
// blocks of a sequence), a chunk of 1024 to 2^30, and the sums behind a chunk to what still decides the same.
__device__ void plan_requests(const pq_paged_plan_args &a, plan_sums &s, scan_room &room)
{
    const int most = a.max_blocks << a.log_block, round = (1 << a.log_block) - 1;
    const int count = between(a.free_count[0], a.n_blocks);
    int rows = 0, back = 0;  // of the requests before this chunk
    int n = 0, n_new = 0;    // of this thread's request (the only one, where there are up to 1024)
    for (int b0 = 0; b0 < a.n_seqs; b0 += PLAN_THREADS) {
        const int b = b0 + threadIdx.x;
        n = n_new = 0;
        if (b < a.n_seqs) {
            n = between(a.seq_len[b], most);
            n_new = a.n_new[b];
        }
        const int asks = between(n_new, a.n_tokens + 1), gives = n_new < 0 ? (n + round) >> a.log_block : 0;
        int end = asks, given = gives, all_rows, all_back;
        scan_two(end, given, room, all_rows, all_back);
        if (b < a.n_seqs) {
            s.old[b] = n;
            s.freed[b] = at_most(back + given - gives, a.n_blocks);
            s.start[b] = at_most(rows + end - asks, a.n_tokens);
            a.tok_start[b] = s.start[b];
        }
        rows = at_most(rows + all_rows, a.n_tokens + 1);
        back = at_most(back + all_back, a.n_blocks);
    }
    const int there = at_most(count + back, a.n_blocks);
    if (threadIdx.x == 0) {
        s.freed[a.n_seqs] = back;
        s.start[a.n_seqs] = a.tok_start[a.n_seqs] = at_most(rows, a.n_tokens);
        s.count = count;
        s.there = there;
    }
    rows = 0;
    int needed = 0;
    int highest = 0;  // blocks taken by the requests that this thread has granted, and all before them
    bool refused = false;
    for (int b0 = 0; b0 < a.n_seqs; b0 += PLAN_THREADS) {
        const int b = b0 + threadIdx.x;
        if (a.n_seqs > PLAN_THREADS) {
            n = b < a.n_seqs ? s.old[b] : 0;  // (written by this thread)
            n_new = b < a.n_seqs ? a.n_new[b] : 0;
        }
        const int asked = n_new > 0 ? n_new : 0, asks = at_most(asked, a.n_tokens + 1);
        int end = asks, nothing = 0, all_rows, all_need, unused;
        scan_two(end, nothing, room, all_rows, unused);
        // (a request that asks for no more than the rows left asks for less than 2^20: the sum does not pass 2^25)
        const bool fits = asked == 0 || (rows + end <= a.n_tokens && n + asked <= most);
        const int need = fits ? ((n + asked + round) >> a.log_block) - ((n + round) >> a.log_block) : 0;
        int upto = need;
        scan_two(upto, nothing, room, all_need, unused);
        upto += needed;
        if (b < a.n_seqs) {
            const bool granted = fits && (need == 0 || upto <= there);
            if (granted && need > 0)
                highest = upto;
            // no granted request follows a refused one that needs blocks, so the sums up to `there` are those of granted ones
            s.taken[b] = at_most(upto - need, there);
            s.got[b] = granted ? asked : 0;
            a.tok_len[b] = s.got[b];
            a.new_seq_len[b] = n_new < 0 ? 0 : n + s.got[b];
            refused |= !granted;
        }
        rows = at_most(rows + all_rows, a.n_tokens + 1);
        needed = at_most(needed + all_need, a.n_blocks + 1);
    }
    // the largest `highest`
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_xor(highest, d, 64);
        highest = y > highest ? y : highest;
    }
    if ((threadIdx.x & 63) == 0)
        room.wave[0][threadIdx.x >> 6] = highest;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < PLAN_WAVES; ++w)
            highest = room.wave[0][w] > highest ? room.wave[0][w] : highest;
        s.taken[a.n_seqs] = highest;
        a.new_free_count[0] = there - highest;
    }
    if (refused)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_REFUSED);
    __syncthreads();
}

// The i-th block that this call takes: it lies i below the top, among those pushed by this call or below them.
__device__ inline int nth_taken(const pq_paged_plan_args &a, const plan_sums &s, int i)
{
    const int e = s.there - 1 - i;
    if (e < s.count)
        return a.free_list[e];
    const int b = owner(s.freed, a.n_seqs, e - s.count);
    return a.table[(int64_t)b * a.max_blocks + (e - s.count - s.freed[b])];
}

// the second half: entries first, first + step, .. of each kind
__device__ void push_blocks(const pq_paged_plan_args &a, const plan_sums &s, int first, int step)
{
    for (int r = first; r < s.there - s.count; r += step) {
        const int b = owner(s.freed, a.n_seqs, r);
        a.free_list[s.count + r] = a.table[(int64_t)b * a.max_blocks + (r - s.freed[b])];
    }
}

__device__ void take_blocks(const pq_paged_plan_args &a, const plan_sums &s, int first, int step)
{
    const int round = (1 << a.log_block) - 1, all = s.taken[a.n_seqs];
    for (int i = first; i < all; i += step) {
        const int b = owner(s.taken, a.n_seqs, i), used = (s.old[b] + round) >> a.log_block;
        a.table[(int64_t)b * a.max_blocks + used + (i - s.taken[b])] = nth_taken(a, s, i);
    }
}

__device__ void map_slots(const pq_paged_plan_args &a, const plan_sums &s, int first, int step)
{
    const int round = (1 << a.log_block) - 1, all = s.start[a.n_seqs];
    bool range = false;
    for (int t = first; t < a.n_tokens; t += step) {
        int slot = -1;
        if (t < all) {
            const int b = owner(s.start, a.n_seqs, t);
            if (s.got[b] > 0) {
                const int p = s.old[b] + t - s.start[b], j = p >> a.log_block, used = (s.old[b] + round) >> a.log_block;
                const int block = j < used ? a.table[(int64_t)b * a.max_blocks + j] : nth_taken(a, s, s.taken[b] + j - used);
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

// entries: both halves.  Else the sums are left for the grid that does the second.
__global__ __launch_bounds__(PLAN_THREADS) void pq_paged_plan_kernel(pq_paged_plan_args a, bool entries)
{
    __shared__ plan_sums s;
    __shared__ scan_room room;
    plan_requests(a, s, room);
    if (entries) {
        // a quarter of the wavefronts pushes, a quarter takes, the others map: no kind waits for another's loads
        const int part = threadIdx.x / (PLAN_THREADS / 4), i = threadIdx.x % (PLAN_THREADS / 4);
        if (part == 0)
            push_blocks(a, s, i, PLAN_THREADS / 4);
        else if (part == 1)
            take_blocks(a, s, i, PLAN_THREADS / 4);
        else
            map_slots(a, s, threadIdx.x - PLAN_THREADS / 2, PLAN_THREADS / 2);
    } else {
        for (int i = threadIdx.x; i < (int)(sizeof(plan_sums) / sizeof(int)); i += PLAN_THREADS)
            a.scratch[i] = ((const int *)&s)[i];
    }
}

__global__ __launch_bounds__(PLAN_THREADS) void pq_paged_plan_entries_kernel(pq_paged_plan_args a)
{
    __shared__ plan_sums s;
    const plan_sums &from = *(const plan_sums *)a.scratch;
    for (int b = threadIdx.x; b <= a.n_seqs; b += PLAN_THREADS) {
        s.start[b] = from.start[b];
        s.freed[b] = from.freed[b];
        s.taken[b] = from.taken[b];
        if (b < a.n_seqs) {
            s.old[b] = from.old[b];
            s.got[b] = from.got[b];
        }
    }
    if (threadIdx.x == 0) {
        s.count = from.count;
        s.there = from.there;
    }
    __syncthreads();
    const int first = blockIdx.x * PLAN_THREADS + threadIdx.x, step = gridDim.x * PLAN_THREADS;
    push_blocks(a, s, first, step);
    take_blocks(a, s, first, step);
    map_slots(a, s, first, step);
}

}  // namespace

int64_t pq_paged_plan_scratch_bytes() { return sizeof(plan_sums); }

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
