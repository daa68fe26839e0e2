// pq_paged_fork, pq_paged_free, pq_paged_compact and pq_paged_copy: blocks that requests hold together.
//
// holders[x] is the number of requests that hold block x besides the first, so that a block that one request holds, and a free
// one, need no entry of their own: 0 is what pq_paged_plan finds and leaves.  A fork adds 1 for every block it shares; an end takes 1
// away, and the one that finds 0 leaves -1 behind: the block has no holder.  Sums of integers, so the order of the atomics
// does not matter; one that finds less than 0 takes its step back, and a block goes back once whatever the counts were.
//
// What goes onto the stack of free blocks is put in order by its number, not by who gave it: that is the same in every run, and
// the lowest numbers, on top, are taken first.
//
// Fork, free and compact are bound by latency: launches, and loads that need each other (four forks of a prompt of 1000 tokens 3 us, half
// of 1000 requests with up to 10K tokens ended 9 us in three launches, 2700 blocks compacted 6 us in two).  Copy is bound by HBM:
// 7200 blocks of 64 KiB for each of K and V, of a list of 8192 pairs, 378 us, 1.89 GB at 5.0 TB/s, 106 % of what a copy of 4 GiB reaches.
#include <hip/hip_runtime.h>

#include "pq_paged_scan.h"

namespace {

constexpr int SEGMENTS = 256;  // of the block numbers, at most, each a workgroup's
constexpr int ROW_THREADS = 256, LOADS = 4;  // entries of a thread on their way together
// Entries of all block tables together up to which one workgroup does a call, all its threads on all of them: with 4K of them a fork and its
// copy take 10.3 us, and 13.6 with a grid for the tables; an end, behind a copy of the counts, 10.8 and 15.2; with 7K 11.8 and 13.6,
// 13.4 and 14.8.  With 8K it is 13.7 and 13.3, 17.2 and 15.1: all atomics go through one compute unit.  (A wavefront a row, 256 requests
// of 16 blocks: 19.8, 19.4.)  It is the tables' width that counts, not what the rows hold: four forks of 1000 tokens 10.0 us, and 13.7 with
// room for 32K tokens a row; six of eight ends 8.2 and 16.0.
constexpr int ONE_ENTRIES = 7 * SCAN_THREADS;

// what a call's launches hand over, in the context's scratch
struct blocks_scratch {
    int shares[PQ_PAGED_MAX_SEQS];  // fork: blocks that a row shares with its parent
    int count[SEGMENTS];            // free, compact: of each segment
    int free_count;                 // free: before the call
    int n_live;                     // compact
};

__device__ inline bool in_range(int x, int n) { return (unsigned)x < (unsigned)n; }

__device__ inline int length_of(const int32_t *seq_len, int b, int most) { return between(seq_len[b], most); }

// ---------------------------------------------------------------------------------------------------------- fork

// Entries of the tables that become shared, and are counted, by threads first, first + step, .. of n: `from(e)` is where entry e comes from,
// or -1.  A row that gets blocks was empty: nobody reads it.  Whether all numbers were in range.
template <typename FROM> __device__ inline bool share(const pq_paged_fork_args &a, int32_t *to, int n, int first, int step, const FROM &from)
{
    bool range = false;
    for (int e0 = first; e0 < n; e0 += LOADS * step) {
        int x[LOADS];
        bool there[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            const int e = e0 + k * step;
            const int64_t at = e < n ? from(e) : -1;
            there[k] = at >= 0;
            x[k] = there[k] ? a.table[at] : 0;
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
            if (there[k]) {
                to[e0 + k * step] = x[k];
                if (in_range(x[k], a.n_blocks))
                    atomicAdd(a.holders + x[k], 1);
                else
                    range = true;
            }
    }
    return !range;
}

// Who becomes whose fork, and the block that it needs for itself: one workgroup, a chunk of 1024 rows at a time.  With `tables` the
// blocks that are shared as well, else they are left to a launch of their own.
__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_fork_kernel(pq_paged_fork_args a, bool tables)
{
    __shared__ int length[PQ_PAGED_MAX_SEQS], shares[PQ_PAGED_MAX_SEQS], parents[PQ_PAGED_MAX_SEQS];
    __shared__ scan_room room;
    blocks_scratch &s = *(blocks_scratch *)a.scratch;
    const int most = a.max_blocks << a.log_block, round = (1 << a.log_block) - 1;
    for (int b = threadIdx.x; b < a.n_seqs; b += SCAN_THREADS)
        length[b] = length_of(a.seq_len, b, most);
    const int count = between(a.free_count[0], a.n_blocks);
    __syncthreads();
    int before = 0;  // blocks asked for by the rows of the chunks before
    bool refused = false, range = false;
    for (int b0 = 0; b0 < a.n_seqs; b0 += SCAN_THREADS) {
        const int b = b0 + threadIdx.x;
        int n = 0, last = -1, p = -1;
        bool asks = false, fits = false;
        if (b < a.n_seqs) {
            p = a.parent[b];
            asks = p >= 0 && p != b;
            fits = asks && p < a.n_seqs && length[b] == 0;
            if (fits) {
                n = length[p];
                if (a.keep != nullptr)
                    n = between(a.keep[b], n);
                if ((n & round) != 0)
                    last = a.table[(int64_t)p * a.max_blocks + (n >> a.log_block)];
            }
        }
        const bool part = (n & round) != 0, needs = part && in_range(last, a.n_blocks);
        int upto = needs, unused = 0, all, all_unused;
        scan_two(upto, unused, room, all, all_unused);
        upto += before;
        before += all;
        if (b < a.n_seqs) {
            const bool granted = fits && (!needs || upto <= count);
            const int got = needs && granted ? a.free_list[count - upto] : -1;
            a.copy_src[b] = needs && granted ? last : -1;
            a.copy_dst[b] = got;
            a.new_seq_len[b] = granted ? n : length[b];
            if (tables) {
                shares[b] = granted ? n >> a.log_block : 0;
                parents[b] = p;
            } else {
                s.shares[b] = granted ? n >> a.log_block : 0;
            }
            if (granted && part)  // (a number outside the cache stays what it is: nobody follows it)
                a.table[(int64_t)b * a.max_blocks + (n >> a.log_block)] = needs ? got : last;
            refused |= asks && !granted;
            range |= granted && part && !needs;
        }
    }
    if (threadIdx.x == 0)
        a.new_free_count[0] = count - at_most(before, count);
    if (tables) {
        __syncthreads();
        range |= !share(a, a.table, a.n_seqs * a.max_blocks, threadIdx.x, SCAN_THREADS, [&](int e) {
            const int b = e / a.max_blocks, j = e - b * a.max_blocks;
            return j < shares[b] ? parents[b] * a.max_blocks + j : -1;
        });
    }
    if (refused)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_REFUSED);
    if (range)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
}

__global__ __launch_bounds__(ROW_THREADS) void pq_paged_fork_tables_kernel(pq_paged_fork_args a)
{
    const int b = blockIdx.x, n = ((const blocks_scratch *)a.scratch)->shares[b];
    if (n <= 0)
        return;
    const int64_t parent = (int64_t)a.parent[b] * a.max_blocks;
    if (!share(a, a.table + (int64_t)b * a.max_blocks, n, blockIdx.y * ROW_THREADS + threadIdx.x, gridDim.y * ROW_THREADS,
               [&](int j) { return parent + j; }))
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
}

// ---------------------------------------------------------------------------------------------------------- free

__device__ inline int used_blocks(const pq_paged_free_args &a, int b)
{
    return (length_of(a.seq_len, b, a.max_blocks << a.log_block) + (1 << a.log_block) - 1) >> a.log_block;
}

// Entries of the tables are given back, by threads first, first + step, .. of n, those for which `is` says so; `freed` hears of blocks that
// have no holder left.  What went wrong, as bits of the error word.
template <typename IS, typename FREED>
__device__ inline unsigned int release(const pq_paged_free_args &a, const int32_t *table, int n, int first, int step, const IS &is, const FREED &freed)
{
    unsigned int wrong = 0;
    for (int e0 = first; e0 < n; e0 += LOADS * step) {
        int x[LOADS], had[LOADS];
        bool there[LOADS];
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            there[k] = e0 + k * step < n && is(e0 + k * step);
            x[k] = there[k] ? table[e0 + k * step] : 0;
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k) {
            had[k] = 1;
            if (there[k]) {
                if (in_range(x[k], a.n_blocks))
                    had[k] = atomicSub(a.holders + x[k], 1);
                else
                    wrong |= PQ_PAGED_ERRFLAG_RANGE;
            }
        }
#pragma unroll
        for (int k = 0; k < LOADS; ++k)
            if (had[k] == 0) {
                freed(x[k]);
            } else if (had[k] < 0) {
                atomicAdd(a.holders + x[k], 1);
                wrong |= PQ_PAGED_ERRFLAG_HOLDERS;
            }
    }
    return wrong;
}

__device__ inline int new_length(const pq_paged_free_args &a, int b)
{
    return a.n_new[b] < 0 ? 0 : length_of(a.seq_len, b, a.max_blocks << a.log_block);
}

__global__ __launch_bounds__(ROW_THREADS) void pq_paged_release_kernel(pq_paged_free_args a)
{
    const int b = blockIdx.x;
    if (a.n_new[b] >= 0)
        return;
    const unsigned int wrong = release(a, a.table + (int64_t)b * a.max_blocks, used_blocks(a, b), blockIdx.y * ROW_THREADS + threadIdx.x,
                                       gridDim.y * ROW_THREADS, [](int) { return true; }, [](int) {});
    if (wrong != 0)
        paged_error(a.dev_err, wrong);
}

// A cache of up to so many blocks is a bit a block in LDS where one workgroup does the work: of those that are freed, or free.
constexpr int BIT_BLOCKS = 1 << 16, BIT_WORDS = BIT_BLOCKS / 32;

// All of a call whose tables are small, by one workgroup: all entries, then the words of the freed blocks.
__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_free_kernel(pq_paged_free_args a)
{
    __shared__ int gives[PQ_PAGED_MAX_SEQS];
    __shared__ unsigned int words[BIT_WORDS];
    __shared__ scan_room room;
    const int count = between(a.free_count[0], a.n_blocks), n_words = (a.n_blocks + 31) / 32;
    for (int b = threadIdx.x; b < a.n_seqs; b += SCAN_THREADS) {
        gives[b] = a.n_new[b] < 0 ? used_blocks(a, b) : 0;
        a.new_seq_len[b] = new_length(a, b);  // (nobody else reads this sequence's length)
    }
    for (int i = threadIdx.x; i < n_words; i += SCAN_THREADS)
        words[i] = 0;
    __syncthreads();
    const auto is = [&](int e) { const int b = e / a.max_blocks; return e - b * a.max_blocks < gives[b]; };
    const unsigned int wrong = release(a, a.table, a.n_seqs * a.max_blocks, threadIdx.x, SCAN_THREADS, is,
                                       [&](int x) { atomicOr(&words[x >> 5], 1u << (x & 31)); });
    if (wrong != 0)
        paged_error(a.dev_err, wrong);
    __syncthreads();
    // thread 0 has the highest blocks
    const int each = (n_words + SCAN_THREADS - 1) / SCAN_THREADS, last = n_words - 1 - (int)threadIdx.x * each;
    int mine = 0;
    for (int k = 0; k < each && last - k >= 0; ++k)
        mine += __builtin_popcount(words[last - k]);
    int upto = mine, unused = 0, all, all_unused;
    scan_two(upto, unused, room, all, all_unused);
    int place = count + upto - mine;
    for (int k = 0; k < each && last - k >= 0; ++k)
        for (unsigned int goes = words[last - k]; goes != 0; ++place) {
            const int at = 31 - __builtin_clz(goes), x = 32 * (last - k) + at;
            goes ^= 1u << at;
            a.holders[x] = 0;
            if (place < a.n_blocks)
                a.free_list[place] = x;
        }
    if (threadIdx.x == 0)
        a.new_free_count[0] = at_most(count + all, a.n_blocks);
}

// How many numbers of a segment are negative: blocks without a holder (free), free blocks (compact).
__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_count_kernel(const int32_t *x, int n, int per_segment, int *scratch, const int32_t *free_count)
{
    __shared__ scan_room room;
    blocks_scratch &s = *(blocks_scratch *)scratch;
    const int first = blockIdx.x * per_segment, end = n - first < per_segment ? n : first + per_segment;
    int found = 0, unused = 0, all, all_unused;
    for (int i = first + threadIdx.x; i < end; i += SCAN_THREADS)
        found += x[i] < 0;
    scan_two(found, unused, room, all, all_unused);
    if (threadIdx.x == 0) {
        s.count[blockIdx.x] = all;
        if (blockIdx.x == 0 && free_count != nullptr)
            s.free_count = between(free_count[0], n);
    }
}

// Sums of the segments before this workgroup's and of all.
__device__ inline void segment_sums(const blocks_scratch &s, int n_segments, scan_room &room, int &before, int &all)
{
    const int t = threadIdx.x, mine = t < n_segments ? s.count[t] : 0;
    int x = mine, y = t < (int)blockIdx.x ? mine : 0, all_x, all_y;
    scan_two(x, y, room, all_x, all_y);
    before = all_y;
    all = all_x;
}

__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_push_kernel(pq_paged_free_args a, int per_segment)
{
    __shared__ scan_room room;
    const blocks_scratch &s = *(const blocks_scratch *)a.scratch;
    int below, all;
    segment_sums(s, gridDim.x, room, below, all);
    const int first = blockIdx.x * per_segment, end = a.n_blocks - first < per_segment ? a.n_blocks : first + per_segment;
    int place = s.free_count + all - below - s.count[blockIdx.x];  // of the segment's highest block
    for (int e = end; e > first; e -= SCAN_THREADS) {
        const int x = e - 1 - (int)threadIdx.x;
        const bool goes = x >= first && a.holders[x] < 0;
        int upto = goes, unused = 0, found, all_unused;
        scan_two(upto, unused, room, found, all_unused);
        if (goes) {
            a.holders[x] = 0;
            if (place + upto - 1 < a.n_blocks)
                a.free_list[place + upto - 1] = x;
        }
        place += found;
    }
    for (int b = blockIdx.x * SCAN_THREADS + threadIdx.x; b < a.n_seqs; b += gridDim.x * SCAN_THREADS)
        a.new_seq_len[b] = new_length(a, b);
    if (blockIdx.x == 0 && threadIdx.x == 0)
        a.new_free_count[0] = at_most(s.free_count + all, a.n_blocks);
}

// ---------------------------------------------------------------------------------------------------------- compact

__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_mark_kernel(pq_paged_compact_args a, bool clear)
{
    const int first = blockIdx.x * SCAN_THREADS + threadIdx.x, step = gridDim.x * SCAN_THREADS;
    if (clear) {
        for (int i = first; i < a.n_blocks; i += step)
            a.moved_to[i] = 0;
        return;
    }
    const int count = between(a.free_count[0], a.n_blocks);
    bool range = false;
    for (int i = first; i < count; i += step) {
        const int x = a.free_list[i];
        if (in_range(x, a.n_blocks))
            a.moved_to[x] = -1;
        else
            range = true;
    }
    if (range)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
}

// The k-th highest live block at or behind n_live goes to the k-th lowest free number in front of it.  moved_to becomes the
// block's number where it stays, -1 where it is free, -2 - k where it moves.
__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_pair_kernel(pq_paged_compact_args a, int per_segment)
{
    __shared__ scan_room room;
    blocks_scratch &s = *(blocks_scratch *)a.scratch;
    int below, n_free;  // free numbers below this chunk's, and all
    segment_sums(s, gridDim.x, room, below, n_free);
    const int n_live = a.n_blocks - n_free;
    const int first = blockIdx.x * per_segment, end = a.n_blocks - first < per_segment ? a.n_blocks : first + per_segment;
    for (int i0 = first; i0 < end; i0 += SCAN_THREADS) {
        const int i = i0 + threadIdx.x;
        const bool there = i < end, is_free = there && a.moved_to[i] < 0;
        int upto = is_free, unused = 0, found, all_unused;
        scan_two(upto, unused, room, found, all_unused);
        upto += below;  // free numbers up to i
        below += found;
        if (!there)
            continue;
        if (i == n_live)
            a.n_copies[0] = upto - is_free;
        if (is_free) {
            if (i < n_live)
                a.copy_dst[upto - 1] = i;
        } else if (i < n_live) {
            a.moved_to[i] = i;
        } else {
            const int k = (a.n_blocks - 1 - i) - (n_free - upto);  // live blocks above it
            a.copy_src[k] = i;
            a.moved_to[i] = -2 - k;
        }
    }
    for (int i = blockIdx.x * SCAN_THREADS + threadIdx.x; i < n_free; i += gridDim.x * SCAN_THREADS)
        a.new_free_list[i] = a.n_blocks - 1 - i;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.new_free_count[0] = n_free;
        s.n_live = n_live;
        if (n_free == 0)
            a.n_copies[0] = 0;
    }
}

// Where a block goes, by moved_to as the kernel above leaves it.  (A number that is read while moved_to gets its last values is one or
// the other, which say the same.)
struct by_array {
    const pq_paged_compact_args &a;
    int n_live;
    __device__ by_array(const pq_paged_compact_args &args) : a(args), n_live(((const blocks_scratch *)args.scratch)->n_live) {}
    __device__ int operator()(int x) const
    {
        const int v = __hip_atomic_load(a.moved_to + x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return v < -1 ? a.copy_dst[-2 - v] : v;
    }
    __device__ void told(int, int) const {}
};

// Up to BIT_BLOCKS blocks: bits set where they are free, with the number of set bits in front of each word.  One
// workgroup makes them, of the list, and the list of numbers that are taken; all else is worked out from them.  With the copy
// 8K blocks take 13.9 us so and 24.6 by the four launches that larger caches need, 33K blocks 24 and 30, 83K blocks 219.6 and 217.2: the
// one workgroup reads the list alone.
struct bits_scratch {
    int n_free;
    unsigned int words[BIT_WORDS];
    int before[BIT_WORDS];
};

__global__ __launch_bounds__(SCAN_THREADS) void pq_paged_bits_kernel(pq_paged_compact_args a)
{
    __shared__ unsigned int words[BIT_WORDS];
    __shared__ scan_room room;
    bits_scratch &s = *(bits_scratch *)a.scratch;
    const int n_words = (a.n_blocks + 31) / 32;
    for (int i = threadIdx.x; i < n_words; i += SCAN_THREADS)
        words[i] = 0;
    const int count = between(a.free_count[0], a.n_blocks);
    __syncthreads();
    bool range = false;
    constexpr int AT_ONCE = 8;  // loads on their way together
    for (int i0 = 0; i0 < count; i0 += AT_ONCE * SCAN_THREADS) {
        int x[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int i = i0 + k * SCAN_THREADS + (int)threadIdx.x;
            x[k] = i < count ? a.free_list[i] : 0;
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (i0 + k * SCAN_THREADS + (int)threadIdx.x < count) {
                if (in_range(x[k], a.n_blocks))
                    atomicOr(&words[x[k] >> 5], 1u << (x[k] & 31));
                else
                    range = true;
            }
    }
    if (range)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
    __syncthreads();
    const int each = (n_words + SCAN_THREADS - 1) / SCAN_THREADS, first = threadIdx.x * each;
    int found = 0, unused = 0, n_free, all_unused;
    for (int i = first; i < first + each && i < n_words; ++i)
        found += __builtin_popcount(words[i]);
    int upto = found;
    scan_two(upto, unused, room, n_free, all_unused);
    const int n_live = a.n_blocks - n_free;
    int before = upto - found;
    for (int i = first; i < first + each && i < n_words; ++i) {
        const unsigned int word = words[i];
        s.words[i] = word;
        s.before[i] = before;
        const int front = n_live - 32 * i;  // of the word, the numbers below n_live
        unsigned int low = front >= 32 ? word : front <= 0 ? 0u : word & ((1u << front) - 1);
        if (i == n_live >> 5)
            a.n_copies[0] = before + __builtin_popcount(low);
        for (int k = before; low != 0; low &= low - 1, ++k)
            a.copy_dst[k] = 32 * i + __builtin_ctz(low);
        before += __builtin_popcount(word);
    }
    if (threadIdx.x == 0) {
        s.n_free = n_free;
        a.new_free_count[0] = n_free;
        if (n_live >> 5 >= n_words)  // nothing is free, and the last word is full
            a.n_copies[0] = 0;
    }
}

struct by_bits {
    const pq_paged_compact_args &a;
    const bits_scratch &s;
    int n_live;
    __device__ by_bits(const pq_paged_compact_args &args)
        : a(args), s(*(const bits_scratch *)args.scratch), n_live(args.n_blocks - s.n_free)
    {
    }
    // of a live block behind n_live, how many live ones are above it
    __device__ int from_top(int x) const
    {
        const int below = s.before[x >> 5] + __builtin_popcount(s.words[x >> 5] & ((1u << (x & 31)) - 1));
        return (a.n_blocks - 1 - x) - (s.n_free - below);
    }
    __device__ int operator()(int x) const
    {
        if (s.words[x >> 5] >> (x & 31) & 1)
            return -1;
        return x < n_live ? x : a.copy_dst[from_top(x)];
    }
    // what moved_to, the pairs and the new list say of it
    __device__ void told(int x, int to) const
    {
        a.moved_to[x] = to;
        if (to >= 0 && x >= n_live)
            a.copy_src[from_top(x)] = x;
        if (x < s.n_free)
            a.new_free_list[x] = a.n_blocks - 1 - x;
    }
};

// Tables and counts by the new numbers.
template <typename MOVED>
__global__ __launch_bounds__(ROW_THREADS) void pq_paged_renumber_kernel(pq_paged_compact_args a, int row_groups)
{
    const MOVED moved(a);
    if ((int)blockIdx.x < a.n_seqs * row_groups) {
        const int b = blockIdx.x / row_groups, group = blockIdx.x - b * row_groups;
        const int n = length_of(a.seq_len, b, a.max_blocks << a.log_block), used = (n + (1 << a.log_block) - 1) >> a.log_block;
        bool range = false;
        for (int j = group * ROW_THREADS + threadIdx.x; j < used; j += row_groups * ROW_THREADS) {
            const int64_t at = (int64_t)b * a.max_blocks + j;
            const int x = a.table[at];
            const int to = in_range(x, a.n_blocks) ? moved(x) : x;
            a.new_table[at] = to;
            range |= !in_range(to, a.n_blocks);
        }
        if (range)
            paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
        return;
    }
    const int groups = gridDim.x - a.n_seqs * row_groups;
    for (int x = (blockIdx.x - a.n_seqs * row_groups) * ROW_THREADS + threadIdx.x; x < a.n_blocks; x += groups * ROW_THREADS) {
        const int to = moved(x);
        moved.told(x, to);
        if (x < moved.n_live) {
            if (to >= 0)  // (a free one gets its count from the block that moves there)
                a.new_holders[x] = a.holders[x];
        } else {
            if (to >= 0) {
                a.new_holders[to] = a.holders[x];
                __hip_atomic_store(a.moved_to + x, to, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            a.new_holders[x] = 0;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------- copy

constexpr int COPY_THREADS = 256;
constexpr int COPY_LOADS = 4;  // 16-byte loads of a thread on their way together
constexpr int COPY_UNIT = COPY_THREADS * COPY_LOADS * 16;
// Workgroups a compute unit, one after another for the most part: with loads and stores that pass the caches 7200 blocks of 64 KiB
// for each of K and V (1.9 GB moved) take 382 us with 8 of them, 379 with 32, 377 with 64, and 19 000 pairs of a list of 83 000 206, 199 and 195; those that
// find nothing at the end of a short list cost about a microsecond for each eight.  (Through the caches 388 and 218 us, with 8.)
constexpr int COPY_PER_CU = 32;

__global__ __launch_bounds__(COPY_THREADS) void pq_paged_copy_kernel(pq_paged_copy_args a)
{
    const int count = a.count == nullptr ? a.n_pairs : between(a.count[0], a.n_pairs);
    const int parts = (int)((a.block_bytes + COPY_UNIT - 1) / COPY_UNIT);
    const int64_t units = (int64_t)count * 2 * parts;
    bool range = false;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int pair = (int)(u / (2 * parts)), rest = (int)(u - (int64_t)pair * (2 * parts)), kind = rest / parts, part = rest - kind * parts;
        const int src = a.src[pair], dst = a.dst[pair];
        if (src < 0)
            continue;
        if (src >= a.n_from || !in_range(dst, a.n_to)) {
            range = true;
            continue;
        }
        const uint8_t *from = a.from[kind] + src * a.block_bytes;
        uint8_t *to = a.to[kind] + dst * a.block_bytes;
        const int64_t at = (int64_t)part * COPY_UNIT + threadIdx.x * 16;
        u32x4 x[COPY_LOADS];
#pragma unroll
        for (int i = 0; i < COPY_LOADS; ++i)
            if (at + i * (COPY_THREADS * 16) < a.block_bytes)
                x[i] = __builtin_nontemporal_load((const u32x4 *)(from + at + i * (COPY_THREADS * 16)));
#pragma unroll
        for (int i = 0; i < COPY_LOADS; ++i)
            if (at + i * (COPY_THREADS * 16) < a.block_bytes)
                __builtin_nontemporal_store(x[i], (u32x4 *)(to + at + i * (COPY_THREADS * 16)));
        if (part == 0)
            for (int h = threadIdx.x; h < a.Hkv; h += COPY_THREADS)
                a.to_scale[kind][(int64_t)dst * a.Hkv + h] = a.from_scale[kind][(int64_t)src * a.Hkv + h];
    }
    if (range)
        paged_error(a.dev_err, PQ_PAGED_ERRFLAG_RANGE);
}

// blocks of a segment: a multiple of what a workgroup takes at a time
int per_segment(int n_blocks) { return (n_blocks / SEGMENTS / SCAN_THREADS + 1) * SCAN_THREADS; }
int segments(int n_blocks) { return (n_blocks + per_segment(n_blocks) - 1) / per_segment(n_blocks); }

// workgroups of a table's row: four entries a thread where it is that long
int groups_of_row(int max_blocks)
{
    const int n = (max_blocks + 4 * ROW_THREADS - 1) / (4 * ROW_THREADS);
    return n < 16 ? n : 16;
}

}  // namespace

int64_t pq_paged_blocks_scratch_bytes() { return sizeof(bits_scratch) > sizeof(blocks_scratch) ? sizeof(bits_scratch) : sizeof(blocks_scratch); }

hipError_t pq_launch_paged_fork(const pq_paged_fork_args &a, hipStream_t s)
{
    const bool tables = (int64_t)a.n_seqs * a.max_blocks <= ONE_ENTRIES;
    hipLaunchKernelGGL(pq_paged_fork_kernel, dim3(1), dim3(SCAN_THREADS), 0, s, a, tables);
    if (!tables)
        hipLaunchKernelGGL(pq_paged_fork_tables_kernel, dim3(a.n_seqs, groups_of_row(a.max_blocks)), dim3(ROW_THREADS), 0, s, a);
    return hipGetLastError();
}

hipError_t pq_launch_paged_free(const pq_paged_free_args &a, hipStream_t s)
{
    if ((int64_t)a.n_seqs * a.max_blocks <= ONE_ENTRIES && a.n_blocks <= BIT_BLOCKS) {
        hipLaunchKernelGGL(pq_paged_free_kernel, dim3(1), dim3(SCAN_THREADS), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(pq_paged_release_kernel, dim3(a.n_seqs, groups_of_row(a.max_blocks)), dim3(ROW_THREADS), 0, s, a);
    const int n = segments(a.n_blocks), per = per_segment(a.n_blocks);
    hipLaunchKernelGGL(pq_paged_count_kernel, dim3(n), dim3(SCAN_THREADS), 0, s, a.holders, a.n_blocks, per, a.scratch, a.free_count);
    hipLaunchKernelGGL(pq_paged_push_kernel, dim3(n), dim3(SCAN_THREADS), 0, s, a, per);
    return hipGetLastError();
}

hipError_t pq_launch_paged_compact(const pq_paged_compact_args &a, hipStream_t s)
{
    const int rows = groups_of_row(a.max_blocks), others = (a.n_blocks + ROW_THREADS - 1) / ROW_THREADS;
    const dim3 all(a.n_seqs * rows + (others < 1024 ? others : 1024));
    if (a.n_blocks <= BIT_BLOCKS) {
        hipLaunchKernelGGL(pq_paged_bits_kernel, dim3(1), dim3(SCAN_THREADS), 0, s, a);
        hipLaunchKernelGGL((pq_paged_renumber_kernel<by_bits>), all, dim3(ROW_THREADS), 0, s, a, rows);
        return hipGetLastError();
    }
    const int n = segments(a.n_blocks), per = per_segment(a.n_blocks), marks = (a.n_blocks + SCAN_THREADS - 1) / SCAN_THREADS;
    const dim3 grid(marks < 512 ? marks : 512);
    hipLaunchKernelGGL(pq_paged_mark_kernel, grid, dim3(SCAN_THREADS), 0, s, a, true);
    hipLaunchKernelGGL(pq_paged_mark_kernel, grid, dim3(SCAN_THREADS), 0, s, a, false);
    hipLaunchKernelGGL(pq_paged_count_kernel, dim3(n), dim3(SCAN_THREADS), 0, s, a.moved_to, a.n_blocks, per, a.scratch, (const int32_t *)nullptr);
    hipLaunchKernelGGL(pq_paged_pair_kernel, dim3(n), dim3(SCAN_THREADS), 0, s, a, per);
    hipLaunchKernelGGL((pq_paged_renumber_kernel<by_array>), all, dim3(ROW_THREADS), 0, s, a, rows);
    return hipGetLastError();
}

hipError_t pq_launch_paged_copy(const pq_paged_copy_args &a, int n_cu, hipStream_t s)
{
    const int64_t units = (int64_t)a.n_pairs * 2 * ((a.block_bytes + COPY_UNIT - 1) / COPY_UNIT), most = COPY_PER_CU * n_cu;
    hipLaunchKernelGGL(pq_paged_copy_kernel, dim3((unsigned)(units < most ? units : most)), dim3(COPY_THREADS), 0, s, a);
    return hipGetLastError();
}
