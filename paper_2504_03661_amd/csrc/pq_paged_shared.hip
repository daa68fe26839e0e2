// pq_paged_shared_decode: one query token per sequence, where groups of sequences begin with the same blocks.
//
// A group's query rows (a member's query heads of a KV head side by side, member after member) attend over the shared tokens in
// tiles of 32 rows, so that a block's bytes are read and converted for 32 rows at once: a workgroup has a tile and a piece of
// the keys, which its four wavefronts share out.  What the members have behind them they attend over by themselves, up to 16 rows
// a tile.  All sequences' own tokens are one line, 32 at a step, and a wavefront has a range of it: as many steps as any other,
// whatever the lengths are, and it goes from one sequence to the next where they end.  Both in one launch, cut so that
// the chip is filled once; a second one puts every row's pieces together:  with base_i, l_i, o_i of piece i,
//     m = max base_i,   out = sum 2^(base_i - m) o_i / sum 2^(base_i - m) l_i.
// Where the block tables are so narrow that a call is short whatever it holds, a workgroup does a sequence's rows of a KV head by itself, in
// one launch.
//
// Long own tokens are bound by HBM (256 chats of a shared prompt of 2048 tokens and 2000 of their own each, 32 query / 8 KV heads, bf16:
// 205 us, 5.2 TB/s over all; once the groups' jobs are done 6.8 TB/s), many rows over shared ones by the issue of vector and
// matrix instructions (512 x 4096 tokens: 60 us, 570 TFLOP/s; vector units busy half of the time, matrix units a fifth), small calls by
// latency: lengths, block numbers, bytes, and the same again in the merge (9 groups of up to 8 beams, 1000 tokens, fp32 16.7 us; 32 samples
// of 8192 tokens 24 us; four of 1000 12.2 us, of them 7 the first launch and 3 the second, and 10.5 in one launch).
#include <hip/hip_runtime.h>

#include "pq_paged_rows16.h"
#include "pq_paged_rows32.h"
#include "pq_paged_scan.h"
#include "pq_paged_shared.h"

namespace {

constexpr int WAVES = JOIN_WAVES, THREADS = 64 * WAVES, STEP = STEP_32;
constexpr int GROUP_ROWS = JOIN_ROWS, OWN_ROWS = 16;  // of a tile
// Workgroups of a compute unit that run together: what the kernel's registers and LDS leave room for, in every type and size (with 4, one after
// another, 32 samples of 8192 tokens 35 us instead of 27).
constexpr int PER_CU = 2;
// Who plans a call.  Up to SMALL_SEQS sequences every wavefront, with a lane for each: 1.7 us (four samples: 12.0 us, 14.4 where workgroups
// plan, 17.0 with a launch).  Up to MIDDLE_SEQS every workgroup, a thread each, sums in LDS (256 chats 205.1 us and with a launch 207.4,
// 128 requests of 500 tokens 18.6 and 21.8, as many of 40 13.6 and 16.8).  For more a launch of one workgroup: 6 to 9 us.
constexpr int SMALL_SEQS = 64, MIDDLE_SEQS = 256;
static_assert(STEP_16 == STEP);

__device__ inline int group_tiles(int rows) { return (rows + GROUP_ROWS - 1) / GROUP_ROWS; }
__host__ __device__ inline int own_tiles(int G) { return (G + OWN_ROWS - 1) / OWN_ROWS; }
__device__ inline int steps_of(int keys) { return (keys + STEP - 1) / STEP; }

// ---------------------------------------------------------------------------------------------------------- cutting

constexpr int GROUP_ALIGN = WAVES * STEP;
constexpr int LEAST_STEPS = 2;  // of a range (eight groups of four samples: 14.0 us, with 4 15.3)
// What a step of a group's job counts for beside one of the line: its bytes come from the L2 for all tiles but one (256 sequences of
// a shared prompt: 1.25 us and 2.45 us, with two wavefronts on a SIMD; 213.0 us where both count alike, 209.7 so).
constexpr float STEP_OF_GROUP = 0.5f;

// A sequence's place on the line, from the steps that it has: whole shortest ranges, so that in a call that has no more than those
// none goes from one sequence to the next.
__device__ inline int place_of(int steps) { return (steps + LEAST_STEPS - 1) / LEAST_STEPS * LEAST_STEPS; }

// Keys of a group's piece at most, from the keys over tiles of groups and sequences alike: a wavefront's share of all.  (The sum
// is one in fp32: the pieces are taken a little larger, so that they are not more.)
__device__ inline int group_piece(float keys, int workgroups)
{
    const int n = (int)fminf(keys * 1.0001f / (float)workgroups, (float)PQ_MAX_TOKENS) + 1;
    return (n + GROUP_ALIGN - 1) / GROUP_ALIGN * GROUP_ALIGN;
}

// Shared tokens that are read by a job of the group, or 0 where that costs more than it saves: a tile's job keeps a workgroup for some
// microseconds, and what it spares is the reading of the same tokens, from the L2 mostly, by the other members' own tiles.  Even at
// 128 to 450 tokens spared for each tile: 400 groups of two with 16 shared tokens 54 us so and 81 as jobs, with 128 tokens 92 both, with
// 256 tokens 133 and 112; 60 groups of eight with 32 tokens 40 and 44, with 128 tokens 52 and 46.
constexpr int SPARED_KEYS = 256;
__device__ inline int worth_sharing(int shared, int rows, int G)
{
    const int tiles = group_tiles(rows);
    return (int64_t)shared * (rows / G * own_tiles(G) - tiles) >= (int64_t)SPARED_KEYS * tiles ? shared : 0;
}

// How many pieces n keys are cut into, none longer than `most`, and their length.  (GROUP_ALIGN divides `most`, so the rounded
// length is no more than that, and n is behind (pieces - 1) * most: none is empty.)
__device__ inline int pieces_of(int n, int most) { return (n + most - 1) / most; }
__device__ inline int piece_length(int n, int pieces) { return ((n + pieces - 1) / pieces + GROUP_ALIGN - 1) / GROUP_ALIGN * GROUP_ALIGN; }

__device__ inline int range_begin(const pq_paged_shared_ranges &r, int w)
{
    return w <= r.n_longer ? w * r.longer : r.n_longer * r.longer + (w - r.n_longer) * r.shorter;
}

__device__ inline int range_of(const pq_paged_shared_ranges &r, int step)
{
    const int behind = step - r.n_longer * r.longer;
    return behind < 0 ? step / r.longer : r.n_longer + behind / r.shorter;
}

// The line's `steps` over the workgroups that the groups' jobs leave: those that run beside them get longer ranges, those that take
// their place when they are done shorter ones, by what the jobs' wavefronts have to do, so that all end together.  Where the ones
// beside them are done with all of it before others could be with a shortest range, there are only those.  Where the jobs are as many as
// the workgroups or more, all ranges are alike: those that have one job fewer than others end earlier.
__device__ inline pq_paged_shared_ranges cut_line(int steps, float group_keys, int group_jobs, int workgroups)
{
    pq_paged_shared_ranges r;
    const int beside = workgroups - group_jobs;
    const float of_job = group_jobs > 0 ? STEP_OF_GROUP * group_keys / (float)(WAVES * STEP * group_jobs) : 0.0f;
    const float least = (float)LEAST_STEPS;
    if (group_jobs > 0 && beside > 0 && (float)steps > (float)(WAVES * beside) * (of_job + least)) {
        const float all = (float)(WAVES * workgroups), even = ((float)steps + (float)(WAVES * group_jobs) * of_job) / all - of_job;
        const float shorter = even > least ? even : least;
        r.n_longer = WAVES * beside;
        r.longer = (int)((shorter + of_job) * 1.0001f) + 1;
        r.shorter = (int)(shorter * 1.0001f) + 1;
    } else {
        const int waves = WAVES * (beside > 0 ? beside : workgroups), each = (steps + waves - 1) / waves;
        r.longer = r.shorter = each > LEAST_STEPS ? each : LEAST_STEPS;
        r.n_longer = 0;
    }
    const int in_longer = r.n_longer * r.longer;
    r.count = steps <= in_longer ? (steps + r.longer - 1) / r.longer : r.n_longer + (steps - in_longer + r.shorter - 1) / r.shorter;
    return r;
}

// Job `at` of a group: `rows` query rows from position `first` on, over its shared tokens.  Tiles of one piece side by side: they read the
// same bytes.
__device__ inline void group_job(pq_paged_shared_job &job, int first, int rows, int shared, int pieces, int partial, int at)
{
    const int tiles = group_tiles(rows), piece = at / tiles, tile = at - piece * tiles, keys = piece_length(shared, pieces);
    job.position = job.table = first;
    job.row0 = tile * GROUP_ROWS;
    job.rows = rows - job.row0 < GROUP_ROWS ? rows - job.row0 : GROUP_ROWS;
    job.k0 = piece * keys;
    job.k1 = job.k0 + keys < shared ? job.k0 + keys : shared;
    job.partial = partial + job.row0 * pieces + piece * job.rows;
}

// -------------------------------------------------------------------------------------- the plan, by a workgroup

template <int MOST> struct shared_sums {
    int start[MOST + 1];     // first position of each group
    int shared[MOST];        // tokens that its members share
    int length[MOST];        // of the sequence at a position; -1: none
    int group[MOST];         // that the position is in
    int group_jobs[MOST + 1];
    int group_rows[MOST], group_pieces[MOST];
    int own[MOST];           // number of the sequence at a position among those that have tokens of their own; -1: none
    int begin[MOST];         // where such a one begins on the line
};

template <int PLAN_WAVES> struct plan_room {
    int sums[4][PLAN_WAVES];
    float2 keys[PLAN_WAVES];
};

// Inclusive sums of four numbers over the workgroup's threads, and their totals.
template <int PLAN_WAVES> __device__ inline void scan_four(int (&x)[4], int (&all)[4], plan_room<PLAN_WAVES> &room)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[k] = lane_scan(x[k]);
        if (lane == 63)
            room.sums[k][wave] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        all[k] = 0;
        int before = 0;
#pragma unroll
        for (int w = 0; w < PLAN_WAVES; ++w) {
            const int of_wave = room.sums[k][w];
            before += w < wave ? of_wave : 0;
            all[k] += of_wave;
        }
        x[k] += before;
    }
    __syncthreads();
}

__device__ inline int running_max(int x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d, 64);
        x = lane >= d && y > x ? y : x;
    }
    return x;
}

// All sums of a call.  Without COMPACT a sequence's number is its position, whether it has tokens of its own or not.
template <int PLAN_THREADS, int MOST, bool COMPACT>
__device__ inline pq_paged_shared_head plan_workgroup(const pq_paged_shared_args &a, shared_sums<MOST> &s, plan_room<PLAN_THREADS / 64> &room)
{
    constexpr int PLAN_WAVES = PLAN_THREADS / 64;
    const int n_seqs = a.n_seqs, n_groups = a.n_groups, G = a.G, tiles = own_tiles(G), lane = threadIdx.x & 63;
    bool range = false;
    for (int g = threadIdx.x; g <= n_groups; g += PLAN_THREADS) {
        s.start[g] = between(a.group_start[g], n_seqs);
        if (g < n_groups)
            s.shared[g] = a.shared_len[g];
    }
    for (int i = threadIdx.x; i < n_seqs; i += PLAN_THREADS) {
        const int b = a.members == nullptr ? i : a.members[i];
        s.length[i] = (unsigned)b < (unsigned)n_seqs ? paged_length(a.c, b) : -2;
    }
    __syncthreads();
    // where groups begin: as they are given, but never before the one in front
    bool falls = false;
    for (int g = threadIdx.x; g < n_groups; g += PLAN_THREADS)
        falls |= s.start[g] > s.start[g + 1];
    if (__syncthreads_or(falls)) {
        if (threadIdx.x < 64) {
            int highest = 0;
            for (int g0 = 0; g0 <= n_groups; g0 += 64) {
                int x = g0 + lane <= n_groups ? s.start[g0 + lane] : 0;
                x = running_max(x > highest ? x : highest, lane);
                if (g0 + lane <= n_groups)
                    s.start[g0 + lane] = x;
                highest = __builtin_amdgcn_readlane(x, 63);
            }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n_seqs; i += PLAN_THREADS) {
        const bool in_group = i >= s.start[0] && i < s.start[n_groups];
        range |= in_group && s.length[i] == -2;
        s.length[i] = in_group && s.length[i] >= 0 ? s.length[i] : -1;
        s.group[i] = s.length[i] >= 0 ? owner(s.start, n_groups, i) : 0;
    }
    if (range)
        paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
    __syncthreads();
    float of_groups = 0.0f, of_own = 0.0f;
    for (int g = threadIdx.x; g < n_groups; g += PLAN_THREADS) {
        const int first = s.start[g], n = s.start[g + 1] - first;
        int shared = 0;
        if (n > 1) {
            shared = s.shared[g];
            shared = shared < s.length[first] ? shared : s.length[first];
            shared = shared > 0 ? worth_sharing(shared >> a.c.log_block << a.c.log_block, n * G, G) : 0;
        }
        s.shared[g] = shared;
        of_groups += (float)group_tiles(n * G) * (float)shared;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n_seqs; i += PLAN_THREADS)
        if (s.length[i] > 0) {
            const int own = s.length[i] - s.shared[s.group[i]];
            of_own += own > 0 ? (float)tiles * (float)own : 0.0f;
        }
    of_groups = wave_sum(of_groups);
    of_own = wave_sum(of_own);
    if (lane == 0)
        room.keys[threadIdx.x >> 6] = make_float2(of_groups, of_own);
    __syncthreads();
    of_groups = of_own = 0.0f;
#pragma unroll
    for (int w = 0; w < PLAN_WAVES; ++w) {
        of_groups += room.keys[w].x;
        of_own += room.keys[w].y;
    }
    const int most = group_piece(of_groups + of_own, a.workgroups);

    // jobs and rows of partials of the groups; and the line of the sequences' own tokens
    int jobs = 0, rows = 0, line = 0, n_own = 0;
    for (int i0 = 0; i0 < n_seqs; i0 += PLAN_THREADS) {
        const int i = i0 + threadIdx.x;
        int n = 0, pieces = 0, own = 0;
        if (i < n_groups) {
            n = (s.start[i + 1] - s.start[i]) * G;
            pieces = pieces_of(s.shared[i], most);
        }
        if (i < n_seqs && s.length[i] >= 0)
            own = s.length[i] - s.shared[s.group[i]];
        const int steps = own > 0 ? steps_of(own) : 0;
        const int mine[4] = {group_tiles(n) * pieces, n * pieces, tiles * place_of(steps), !COMPACT || steps > 0};
        int upto[4] = {mine[0], mine[1], mine[2], mine[3]}, all[4];
        scan_four(upto, all, room);
        if (i < n_groups) {
            s.group_jobs[i] = jobs + upto[0] - mine[0];
            s.group_rows[i] = rows + upto[1] - mine[1];
            s.group_pieces[i] = pieces;
        }
        if (i < n_seqs) {
            s.own[i] = mine[3] ? n_own + upto[3] - 1 : -1;
            if (mine[3])
                s.begin[s.own[i]] = line + upto[2] - mine[2];
        }
        jobs += all[0];
        rows += all[1];
        line += all[2];
        n_own += all[3];
    }
    if (threadIdx.x == 0)
        s.group_jobs[n_groups] = jobs;
    pq_paged_shared_head head;
    head.group_jobs = jobs;
    head.group_rows = rows;
    head.n_own = n_own;
    head.ranges = cut_line(line, of_groups, jobs, a.workgroups);
    __syncthreads();
    return head;
}

// For the merge: the head, and where the partials of each position are.
template <int PLAN_THREADS, int MOST>
__device__ inline void write_members(const pq_paged_shared_args &a, const shared_sums<MOST> &s, const pq_paged_shared_head &head)
{
    if (threadIdx.x == 0)
        *a.w.head = head;
    for (int i = threadIdx.x; i < a.n_seqs; i += PLAN_THREADS) {
        const int g = s.group[i], own = s.length[i] - s.shared[g];
        pq_paged_shared_member m;
        m.b = s.length[i] < 0 ? -1 : a.members == nullptr ? i : a.members[i];
        m.row = (i - s.start[g]) * a.G;
        m.rows = (s.start[g + 1] - s.start[g]) * a.G;
        m.group_row = s.group_rows[g];
        m.group_pieces = m.b < 0 ? 0 : s.group_pieces[g];
        m.own = s.own[i];
        m.begin = m.own >= 0 ? s.begin[m.own] : 0;
        m.steps = m.b >= 0 && own > 0 ? steps_of(own) : 0;
        a.w.members[i] = m;
    }
}

// Job e of the groups' of a plan.
template <int MOST>
__device__ inline void plan_job(const pq_paged_shared_args &a, const shared_sums<MOST> &s, int e, pq_paged_shared_job &job)
{
    const int g = owner(s.group_jobs, a.n_groups, e);
    group_job(job, s.start[g], (s.start[g + 1] - s.start[g]) * a.G, s.shared[g], s.group_pieces[g], s.group_rows[g], e - s.group_jobs[g]);
    job.table = a.members == nullptr ? job.table : a.members[job.table];
}

// The plan of a call of many sequences.
constexpr int PLAN_THREADS = SCAN_THREADS;

__global__ __launch_bounds__(PLAN_THREADS) void pq_paged_shared_plan_kernel(pq_paged_shared_args a)
{
    __shared__ shared_sums<PQ_PAGED_MAX_SEQS> s;
    __shared__ plan_room<PLAN_THREADS / 64> room;
    const pq_paged_shared_head head = plan_workgroup<PLAN_THREADS, PQ_PAGED_MAX_SEQS, true>(a, s, room);
    write_members<PLAN_THREADS>(a, s, head);
    for (int i = threadIdx.x; i < a.n_seqs; i += PLAN_THREADS)
        if (s.own[i] >= 0) {
            pq_paged_shared_own o;
            o.b = a.members == nullptr ? i : a.members[i];
            o.k0 = s.shared[s.group[i]];
            o.k1 = s.length[i];
            o.begin = s.begin[s.own[i]];
            a.w.own[s.own[i]] = o;
        }
    for (int w = threadIdx.x; w < head.ranges.count; w += PLAN_THREADS)
        a.w.first[w] = owner(s.begin, head.n_own, range_begin(head.ranges, w));
    for (int e = threadIdx.x; e < head.group_jobs; e += PLAN_THREADS) {
        pq_paged_shared_job job;
        plan_job(a, s, e, job);
        a.w.jobs[e] = job;
    }
}

// ------------------------------------------------------------------------------- the plan of a small call, by a wavefront

// Lane g has group g, lane i the sequence at position i.
struct small_plan {
    int lo, rows, shared, group_pieces, group_job, group_row;  // first position, query rows, tokens, pieces, first job, first partial
    int b, length, group, steps, begin;                        // steps of its own, of one tile, and where they begin on the line
    pq_paged_shared_head head;
};

__device__ inline int of_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

__device__ inline small_plan plan_small(const pq_paged_shared_args &a, int lane)
{
    small_plan p;
    const int n_seqs = a.n_seqs, n_groups = a.n_groups, G = a.G, tiles = own_tiles(G);
    const bool is_group = lane < n_groups, is_seq = lane < n_seqs;
    int lo = is_group ? a.group_start[lane] : 0, hi = is_group ? a.group_start[lane + 1] : 0;
    int asked = is_group ? a.shared_len[lane] : 0;
    p.b = !is_seq ? -1 : a.members == nullptr ? lane : a.members[lane];
    const int length_of_lane = is_seq ? paged_length(a.c, lane) : -1;  // (asked for at once, and then looked up)
    const bool there = (unsigned)p.b < (unsigned)n_seqs;
    const int length = __shfl(length_of_lane, p.b & 63, 64);
    lo = between(lo, n_seqs);
    hi = between(hi, n_seqs);
    if (__ballot(is_group && hi < lo) != 0) {  // not ascending: no group begins before the one in front
        lo = running_max(lo, lane);
        hi = hi > lo ? hi : lo;
    }
    p.lo = lo;
    p.rows = is_group ? (hi - lo) * G : 0;
    const int begin = of_lane(lo, 0), end = of_lane(hi, n_groups - 1);
    // the last group that begins at or before the position
    p.group = 0;
    for (int g = 1; g < n_groups; ++g)
        p.group += of_lane(lo, g) <= lane;
    const bool in_group = is_seq && lane >= begin && lane < end;
    p.length = in_group && there ? length : -1;
    if (__ballot(in_group && !there) != 0 && lane == 0)
        paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
    const int of_first = __shfl(p.length, lo < 63 ? lo : 63, 64);
    asked = asked < of_first ? asked : of_first;
    p.shared = p.rows > G && asked > 0 ? worth_sharing(asked >> a.c.log_block << a.c.log_block, p.rows, G) : 0;
    const int own = p.length - __shfl(p.shared, p.group, 64);
    const float of_groups = wave_sum((float)group_tiles(p.rows) * (float)p.shared);
    const float of_own = wave_sum(own > 0 ? (float)tiles * (float)own : 0.0f);
    p.group_pieces = pieces_of(p.shared, group_piece(of_groups + of_own, a.workgroups));
    p.steps = own > 0 ? steps_of(own) : 0;
    const int jobs = group_tiles(p.rows) * p.group_pieces, rows = p.rows * p.group_pieces;
    const int place = tiles * place_of(p.steps);
    const int upto_jobs = lane_scan(jobs), upto_rows = lane_scan(rows), upto_steps = lane_scan(place);
    p.group_job = upto_jobs - jobs;
    p.group_row = upto_rows - rows;
    p.begin = upto_steps - place;
    p.head.group_jobs = of_lane(upto_jobs, 63);
    p.head.group_rows = of_lane(upto_rows, 63);
    p.head.n_own = n_seqs;  // (those without tokens of their own are numbered too)
    p.head.ranges = cut_line(of_lane(upto_steps, 63), of_groups, p.head.group_jobs, a.workgroups);
    return p;
}

// ---------------------------------------------------------------------------------------------------------- attention

// Row of the partials that the first row of a tile of a sequence's own is, in a range: both numbers only grow along the line.
__device__ inline int own_partial(const pq_paged_shared_head &head, int G, int tile_number, int range)
{
    return head.group_rows + (tile_number + range) * (G < OWN_ROWS ? G : OWN_ROWS);
}

// A tile of a sequence's query rows over keys of its own; `all`: there are no others, and the rows are done here: no partials and nothing
// to merge (800 sequences of a few hundred tokens each: 49.9 us; 54.5 where all rows went through the merge).
template <typename T, int D>
__device__ inline void attend_own(const pq_paged_shared_args &a, int h, int lane, int b, int row0, int k0, int k1, int partial, bool all)
{
    const int32_t *table = a.c.table + (int64_t)b * a.c.max_blocks;
    const int rows = a.G - row0 < OWN_ROWS ? a.G - row0 : OWN_ROWS;
    const int last_block = (k1 + (1 << a.c.log_block) - 1) >> a.c.log_block, col = lane & 15, quad = lane >> 4;
    block_batch batch;
    batch.first = -65;
    query_16<T, D> row;
    load_query((const T *)a.q + (int64_t)b * a.q_stride + (int64_t)(h * a.G + row0 + (col < rows ? col : 0)) * D, quad, row);
    step_data<D> now;
    load_step<D>(a.c, table, batch, last_block, h, k0, lane, now);
    rows_16<T, D> r;
    r.take(row, a.scale_log2e);
    r.attend(a.c, table, batch, last_block, h, k0, k1, lane, now);
    const float l = r.sum();
    if (col >= rows)
        return;
    if (all) {
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        T *const out = (T *)a.out + ((int64_t)b * a.Hq + h * a.G + row0 + col) * D + 4 * quad;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            T x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = paged_elem<T>::down(r.o[i][e] * by);
            __builtin_memcpy(out + 16 * i, x, sizeof(x));
        }
        return;
    }
    const int64_t to = (int64_t)h * a.w.most_rows + partial + col;
    if (quad == 0)
        a.w.sums[to] = make_float2(r.base, l);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
        *(f32x4 *)(a.w.partials + to * D + 16 * i + 4 * quad) = r.o[i];
}

// The part of range `range` that a sequence's own tokens, from step `begin` of the line on, have
template <typename T, int D>
__device__ inline void attend_range(const pq_paged_shared_args &a, const pq_paged_shared_head &head, int h, int lane, int range, int b, int k0,
                                    int k1, int begin, int number)
{
    const int steps = steps_of(k1 - k0), place = place_of(steps), tiles = own_tiles(a.G);
    const int from = range_begin(head.ranges, range) - begin, end = range_begin(head.ranges, range + 1) - begin;
    for (int tile = from > 0 ? from / place : 0; tile < tiles && tile * place < end; ++tile) {
        const int first = from > tile * place ? from - tile * place : 0, last = end - tile * place < steps ? end - tile * place : steps;
        if (first < last)
            attend_own<T, D>(a, h, lane, b, tile * OWN_ROWS, k0 + first * STEP, last < steps ? k0 + last * STEP : k1,
                             own_partial(head, a.G, number * tiles + tile, range), k0 == 0 && first == 0 && last == steps);
    }
}

// Who plans: every wavefront, every workgroup, or a launch before this one
enum { BY_WAVE, BY_WORKGROUP, BY_LAUNCH };

template <int BY> struct planned {};
template <> struct planned<BY_WORKGROUP> {
    shared_sums<MIDDLE_SEQS> s;
    plan_room<WAVES> room;
};

__device__ inline void make_uniform(int &x) { x = __builtin_amdgcn_readfirstlane(x); }

template <typename T, int D, int BY>
__global__ __launch_bounds__(THREADS, PER_CU) void pq_paged_shared_kernel(pq_paged_shared_args a)
{
    constexpr bool SMALL = BY == BY_WAVE;
    __shared__ join_room<D> room;
    __shared__ planned<BY> plan;
    const int of_thread = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int h = blockIdx.x % a.c.Hkv;
    small_plan p;
    if constexpr (SMALL) {
        const int lane = of_thread;
        p = plan_small(a, lane);
        if (blockIdx.x == 0 && wave == 0) {  // for the merge
            const int lo = __shfl(p.lo, p.group, 64), rows = __shfl(p.rows, p.group, 64);
            const int group_row = __shfl(p.group_row, p.group, 64), pieces = __shfl(p.group_pieces, p.group, 64);
            if (lane < a.n_seqs)
                a.w.members[lane] = pq_paged_shared_member{p.length < 0 ? -1 : p.b, (lane - lo) * a.G, rows, group_row, pieces,
                                                           lane, p.begin, p.steps};
            if (lane == 0)
                *a.w.head = p.head;
        }
    } else if constexpr (BY == BY_WORKGROUP) {
        p.head = plan_workgroup<THREADS, MIDDLE_SEQS, false>(a, plan.s, plan.room);
        make_uniform(p.head.group_jobs);
        make_uniform(p.head.group_rows);
        make_uniform(p.head.ranges.n_longer);
        make_uniform(p.head.ranges.longer);
        make_uniform(p.head.ranges.shorter);
        make_uniform(p.head.ranges.count);
        if (blockIdx.x == 0)
            write_members<THREADS>(a, plan.s, p.head);
    } else {
        p.head = *a.w.head;
    }
    // The groups' jobs first, then four ranges of the line at a time; the grid is what runs together
    const int stride = gridDim.x / a.c.Hkv, jobs = p.head.group_jobs + (p.head.ranges.count + WAVES - 1) / WAVES;
    for (int e = blockIdx.x / a.c.Hkv; e < jobs; e += stride) {
        int lane = of_thread;
        work_out_here<T, D>(lane);
        if (e >= p.head.group_jobs) {
            const int range = (e - p.head.group_jobs) * WAVES + wave;
            if (range >= p.head.ranges.count)
                continue;
            const int end = range_begin(p.head.ranges, range + 1);
            if constexpr (SMALL) {
                const int first = range_begin(p.head.ranges, range), upto = p.begin + own_tiles(a.G) * place_of(p.steps);
                const int shared = __shfl(p.shared, p.group, 64);
                // lanes whose sequences have a part of the range
                for (uint64_t mine = __ballot(p.begin < end && upto > first && p.steps > 0); mine != 0; mine &= mine - 1) {
                    const int i = __builtin_ctzll(mine);
                    attend_range<T, D>(a, p.head, h, lane, range, of_lane(p.b, i), of_lane(shared, i), of_lane(p.length, i),
                                       of_lane(p.begin, i), i);
                }
            } else if constexpr (BY == BY_WORKGROUP) {
                const int tiles = own_tiles(a.G);
                for (int step = range_begin(p.head.ranges, range); step < end;) {
                    int i = owner(plan.s.begin, a.n_seqs, step);  // (the last of those that begin there: it has tokens of its own)
                    make_uniform(i);
                    int b = a.members == nullptr ? i : a.members[i], k0 = plan.s.shared[plan.s.group[i]], k1 = plan.s.length[i], begin = plan.s.begin[i];
                    make_uniform(b);
                    make_uniform(k0);
                    make_uniform(k1);
                    make_uniform(begin);
                    const int after = k1 > k0 ? begin + tiles * place_of(steps_of(k1 - k0)) : step;
                    if (after <= step)  // (the last range may end behind the line)
                        break;
                    attend_range<T, D>(a, p.head, h, lane, range, b, k0, k1, begin, i);
                    step = after;
                }
            } else {
                int i = a.w.first[range];
                pq_paged_shared_own o = a.w.own[i];
                do {
                    const pq_paged_shared_own next = a.w.own[i + 1 < p.head.n_own ? i + 1 : i];  // (on its way beside the keys)
                    attend_range<T, D>(a, p.head, h, lane, range, o.b, o.k0, o.k1, o.begin, i);
                    o = next;
                    ++i;
                } while (i < p.head.n_own && o.begin < end);
            }
            continue;
        }
        const int col = lane & 31, half = lane >> 5;
        pq_paged_shared_job job;
        int row, at, b, length;  // this lane's query row, its member, and that one's sequence
        if constexpr (SMALL) {
            const int next = p.group_job + group_tiles(p.rows) * p.group_pieces;
            const int g = __builtin_ctzll(__ballot(e >= p.group_job && e < next));
            group_job(job, of_lane(p.lo, g), of_lane(p.rows, g), of_lane(p.shared, g), of_lane(p.group_pieces, g),
                      of_lane(p.group_row, g), e - of_lane(p.group_job, g));
            row = job.row0 + (col < job.rows ? col : 0);
            at = row / a.G;
            b = __shfl(p.b, job.position + at, 64);
            length = __shfl(p.length, job.position + at, 64);
            job.table = of_lane(p.b, job.table);
        } else {
            if constexpr (BY == BY_WORKGROUP) {
                plan_job(a, plan.s, e, job);
                make_uniform(job.table);
                make_uniform(job.position);
                make_uniform(job.row0);
                make_uniform(job.rows);
                make_uniform(job.k0);
                make_uniform(job.k1);
                make_uniform(job.partial);
            } else {
                job = a.w.jobs[e];
            }
            row = job.row0 + (col < job.rows ? col : 0);
            at = row / a.G;
            b = a.members == nullptr ? job.position + at : a.members[job.position + at];
            length = (unsigned)b < (unsigned)a.n_seqs ? paged_length(a.c, b) : -1;
        }
        query_32<T, D> query;
        load_query((const T *)a.q + (int64_t)(length < 0 ? 0 : b) * a.q_stride + (int64_t)(h * a.G + row - at * a.G) * D, half, query);
        const int share = ((job.k1 - job.k0 + WAVES - 1) / WAVES + STEP - 1) / STEP * STEP;
        const int t0 = job.k0 + wave * share, t1 = t0 + share < job.k1 ? t0 + share : job.k1;
        const int32_t *table = a.c.table + (int64_t)job.table * a.c.max_blocks;
        const int last_block = (job.k1 + (1 << a.c.log_block) - 1) >> a.c.log_block;
        step_bytes<D> now;
        block_batch batch;
        batch.first = -65;
        if (t0 < t1)
            load_bytes<D>(a.c, table, batch, last_block, h, t0, lane, now);
        // (columns behind the last row repeat the first one, and nobody takes what they find)
        int sees = col >= job.rows ? t1 : length;
        sees = sees < t1 ? sees : t1;
        const int least = __ballot(sees < t1) == 0 ? t1 : 0;
        rows_32<T, D> r;
        r.take(query, a.scale_log2e);
        r.attend(a.c, table, batch, last_block, h, t0, t1, sees, least, lane, now);
        room.join(r, wave, lane);
        const int64_t to = (int64_t)h * a.w.most_rows + job.partial;
        int thread = threadIdx.x;
        work_out_here<T, D>(thread);
        for (int i = thread; i < job.rows * (D / 2); i += THREADS) {
            const int r = i / (D / 2), d = i % (D / 2) * 2;
            *(float2 *)(a.w.partials + (to + r) * D + d) = room.values(r, d);
            if (d == 0)
                a.w.sums[to + r] = make_float2(room.row_base[r], room.row_l[r]);
        }
        __syncthreads();
    }
}

// A row's pieces put together by a wavefront, D / 64 dims a lane.
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void pq_paged_shared_merge_kernel(pq_paged_shared_args a)
{
    constexpr int PER_LANE = D / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t at = (int64_t)blockIdx.x * WAVES + wave;
    const int i = (int)(at / a.Hq), head = (int)(at - (int64_t)i * a.Hq);
    if (i >= a.n_seqs)
        return;
    const pq_paged_shared_member m = a.w.members[i];
    const pq_paged_shared_head whole = *a.w.head;
    if (m.b < 0)
        return;
    const int h = head / a.G, g = head - h * a.G;
    // the row's partials: the group's, then its own, each some rows apart
    int of_group = 0, group_first = 0, group_stride = 0, of_own = 0, own_first = 0;
    if (m.group_pieces > 0) {
        const int r = m.row + g, row0 = r / GROUP_ROWS * GROUP_ROWS;
        of_group = m.group_pieces;
        group_first = m.group_row + row0 * m.group_pieces + (r - row0);
        group_stride = m.rows - row0 < GROUP_ROWS ? m.rows - row0 : GROUP_ROWS;
    }
    const int own_stride = a.G < OWN_ROWS ? a.G : OWN_ROWS;
    if (m.steps > 0) {
        const int tile = g / OWN_ROWS, begin = m.begin + tile * place_of(m.steps), first = range_of(whole.ranges, begin);
        of_own = range_of(whole.ranges, begin + m.steps - 1) - first + 1;
        own_first = own_partial(whole, a.G, m.own * own_tiles(a.G) + tile, first) + g - tile * OWN_ROWS;
    }
    const int pieces = of_group + of_own;
    if (of_group == 0 && of_own == 1)  // (done by who had them)
        return;
    const int64_t of_head = (int64_t)h * a.w.most_rows;
    float top = LOWEST, sum = 0.0f, o[PER_LANE] = {};
    constexpr int AT_ONCE = 8;  // partials on their way together
    for (int c0 = 0; c0 < pieces; c0 += 64) {
        // a lane has a piece's base and sum, and so its weight; one that is not there has the weight 0
        const int c = c0 + lane, n = pieces - c0 < 64 ? pieces - c0 : 64;
        const int at = c < of_group ? group_first + c * group_stride : own_first + (c - of_group) * own_stride;
        const float2 ml = lane < n ? a.w.sums[of_head + at] : make_float2(-INFINITY, 0.0f);
        float v[AT_ONCE][PER_LANE];
        const auto ask = [&](int c1) {
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const float *from = a.w.partials + (of_head + of_lane(at, c1 + k < n ? c1 + k : 0)) * D + PER_LANE * lane;
#pragma unroll
                for (int d = 0; d < PER_LANE; ++d)
                    v[k][d] = from[d];
            }
        };
        ask(0);
        const float high = fmaxf(top, wave_max(ml.x)), old = __builtin_amdgcn_exp2f(top - high), by = __builtin_amdgcn_exp2f(ml.x - high);
        top = high;
        sum = fmaf(sum, old, wave_sum(ml.y * by));
#pragma unroll
        for (int d = 0; d < PER_LANE; ++d)
            o[d] *= old;
        for (int c1 = 0; c1 < n; c1 += AT_ONCE) {
            if (c1 > 0)
                ask(c1);
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const float weight = lane_of(by, c1 + k);
#pragma unroll
                for (int d = 0; d < PER_LANE; ++d)
                    o[d] = fmaf(v[k][d], weight, o[d]);
            }
        }
    }
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    T *const out = (T *)a.out + ((int64_t)m.b * a.Hq + head) * D + PER_LANE * lane;
#pragma unroll
    for (int d = 0; d < PER_LANE; ++d)
        out[d] = paged_elem<T>::down(o[d] * by);
}

// ------------------------------------------------------------------------------------------- calls that can only be small

// A workgroup has a tile of a sequence's rows over all its keys, wherever they come from; its wavefronts share those out and join through LDS.
// No plan, no partials and no merge; shared tokens are read by each member, from the L2 for the most part.
template <typename T, int D> __global__ __launch_bounds__(THREADS, 2) void pq_paged_shared_direct_kernel(pq_paged_shared_args a)
{
    __shared__ float part[WAVES][OWN_ROWS][D + 4];
    __shared__ float wave_base[WAVES][OWN_ROWS], wave_l[WAVES][OWN_ROWS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), col = lane & 15, quad = lane >> 4;
    const int h = blockIdx.x % a.c.Hkv, unit = blockIdx.x / a.c.Hkv, tiles = own_tiles(a.G);
    const int i = unit / tiles, row0 = (unit - i * tiles) * OWN_ROWS;
    const int b = a.members == nullptr ? i : a.members[i], begin = between(a.group_start[0], a.n_seqs);
    int end = begin;
    for (int g0 = 1; g0 <= a.n_groups; g0 += 64) {
        const int start = g0 + lane <= a.n_groups ? between(a.group_start[g0 + lane], a.n_seqs) : 0;
        end = start > end ? start : end;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const int other = __shfl_xor(end, d, 64);
        end = other > end ? other : end;
    }
    if (i < begin || i >= end)
        return;
    if ((unsigned)b >= (unsigned)a.n_seqs) {
        if (threadIdx.x == 0)
            paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_RANGE);
        return;
    }
    const int length = paged_length(a.c, b), share = ((length + WAVES - 1) / WAVES + STEP - 1) / STEP * STEP;
    const int t0 = wave * share, t1 = t0 + share < length ? t0 + share : length;
    const int32_t *table = a.c.table + (int64_t)b * a.c.max_blocks;
    const int rows = a.G - row0 < OWN_ROWS ? a.G - row0 : OWN_ROWS, last_block = (length + (1 << a.c.log_block) - 1) >> a.c.log_block;
    query_16<T, D> row;
    load_query((const T *)a.q + (int64_t)b * a.q_stride + (int64_t)(h * a.G + row0 + (col < rows ? col : 0)) * D, quad, row);
    step_data<D> now;
    block_batch batch;
    batch.first = -65;
    if (t0 < t1)
        load_step<D>(a.c, table, batch, last_block, h, t0, lane, now);
    rows_16<T, D> r;
    r.take(row, a.scale_log2e);
    r.attend(a.c, table, batch, last_block, h, t0, t1, lane, now);
    const float l = r.sum();
    if (quad == 0) {
        wave_base[wave][col] = r.base;
        wave_l[wave][col] = l;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
        *(f32x4 *)&part[wave][col][16 * i + 4 * quad] = r.o[i];
    __syncthreads();
    T *const out = (T *)a.out + ((int64_t)b * a.Hq + h * a.G + row0) * D;
    for (int e = threadIdx.x; e < rows * (D / 2); e += THREADS) {
        const int r = e / (D / 2), d = e % (D / 2) * 2;
        float top = wave_base[0][r], sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
            top = fmaxf(top, wave_base[w][r]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float by = __builtin_amdgcn_exp2f(wave_base[w][r] - top);
            sum = fmaf(wave_l[w][r], by, sum);
            x = fmaf(part[w][r][d], by, x);
            y = fmaf(part[w][r][d + 1], by, y);
        }
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
        out[r * D + d] = paged_elem<T>::down(x * by);
        out[r * D + d + 1] = paged_elem<T>::down(y * by);
    }
}

// Where the tables' width says that no call can be larger.  One launch of a few steps against two or three of many: 8 sequences of 1024
// tokens, 32 query / 8 KV heads, 10.8 us and 13.1, 64 of 256 7.8 and 13.0, 256 of 256 20.4 and 26.9, all of one prompt.  A workgroup gets
// through 45 GB/s: two sequences of 1280 tokens 11.4 and 12.0, of 1536 12.8 and 11.8, of 4096 29.3 and 13.6; fewer in fp32 with 128 dims,
// where the other way takes longer only for more sequences: of 1264 tokens one 13.0 and 12.0, two 13.1 and 12.4, four 13.2 and 13.0, eight
// 13.2 and 14.4; of 1136 one 12.2 and 12.0, two 12.3 both, four 12.3 and 13.1 (64 dims, 1264: one 9.6 and 9.9, two 9.6 and 10.1).
// And what is shared is read once for each member: 32 heads, 32 sequences of 512 17.5 and 13.7; of more than SMALL_SEQS, where the
// other way's plan takes longer, 128 of 512 17.2 and 18.6.  Many workgroups that have little to do cost more than a line of it:
// 1024 sequences of 32, 46.8 and 38.0.
constexpr int DIRECT_TOKENS = 1280, DIRECT_UNITS = 2048;
constexpr int DIRECT_FEW_SEQS = 4, DIRECT_FEW_TOKENS = 1152;  // fp32, 128 dims
constexpr int64_t DIRECT_SMALL = 1 << 18, DIRECT_LARGE = 1 << 19;  // tokens of all workgroups

bool is_direct(const pq_paged_config &cfg, const pq_paged_shared_args &a)
{
    const int64_t width = (int64_t)a.c.max_blocks << a.c.log_block, units = (int64_t)a.n_seqs * own_tiles(a.G) * a.c.Hkv;
    const bool few = cfg.dtype == PQ_F32 && cfg.head_dim == 128 && a.n_seqs <= DIRECT_FEW_SEQS;
    return width <= (few ? DIRECT_FEW_TOKENS : DIRECT_TOKENS) && units <= DIRECT_UNITS && units * width <= (a.n_seqs <= SMALL_SEQS ? DIRECT_SMALL : DIRECT_LARGE);
}

}  // namespace

// For each KV head: the groups' jobs are `workgroups` and a rest for each tile at most, the ranges of the line four for each workgroup, and
// two that rounding adds; partials of the line have a row's place for each tile and each range.
int64_t pq_paged_shared_layout(const pq_paged_ctx *ctx, int n_seqs, int n_groups, void *workspace, pq_paged_shared_args *a)
{
    const pq_paged_config &cfg = ctx->cfg;
    const int64_t G = cfg.n_q_heads / cfg.n_kv_heads;
    const int filled = PER_CU * ctx->n_cu / cfg.n_kv_heads, workgroups = filled > 1 ? filled : 1;
    const int64_t jobs = workgroups + n_seqs * G / GROUP_ROWS + n_groups, ranges = WAVES * workgroups + 2;
    const int64_t rows = GROUP_ROWS * workgroups + n_seqs * G + (n_seqs * own_tiles(G) + ranges) * (G < OWN_ROWS ? G : OWN_ROWS);
    int64_t bytes = 0;
    const auto room = [&](int64_t n) { const int64_t at = bytes; bytes += (n + 255) / 256 * 256; return at; };
    const int64_t head_at = room(sizeof(pq_paged_shared_head)), members_at = room(n_seqs * sizeof(pq_paged_shared_member));
    const int64_t jobs_at = room(jobs * sizeof(pq_paged_shared_job)), own_at = room(n_seqs * sizeof(pq_paged_shared_own));
    const int64_t first_at = room(ranges * sizeof(int)), sums_at = room(cfg.n_kv_heads * rows * sizeof(float2));
    const int64_t partials_at = room(cfg.n_kv_heads * rows * cfg.head_dim * sizeof(float));
    if (a != nullptr) {
        char *const at = (char *)workspace;
        a->w.head = (pq_paged_shared_head *)(at + head_at);
        a->w.members = (pq_paged_shared_member *)(at + members_at);
        a->w.jobs = (pq_paged_shared_job *)(at + jobs_at);
        a->w.own = (pq_paged_shared_own *)(at + own_at);
        a->w.first = (int *)(at + first_at);
        a->w.sums = (float2 *)(at + sums_at);
        a->w.partials = (float *)(at + partials_at);
        a->w.most_rows = rows;
        a->workgroups = workgroups;
    }
    return bytes;
}

hipError_t pq_launch_paged_shared(const pq_paged_ctx *ctx, const pq_paged_shared_args &a, hipStream_t s)
{
    if (is_direct(ctx->cfg, a)) {
        const dim3 units((unsigned)(a.n_seqs * own_tiles(a.G) * a.c.Hkv));
#define LAUNCH(T, D) hipLaunchKernelGGL((pq_paged_shared_direct_kernel<T, D>), units, dim3(THREADS), 0, s, a)
        PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
        return hipGetLastError();
    }
    if (a.n_seqs > MIDDLE_SEQS)
        hipLaunchKernelGGL(pq_paged_shared_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, a);
    const dim3 grid((unsigned)a.workgroups * (unsigned)a.c.Hkv), rows((unsigned)(((int64_t)a.n_seqs * a.Hq + WAVES - 1) / WAVES));
#define LAUNCH(T, D)                                                                                \
    do {                                                                                            \
        if (a.n_seqs <= SMALL_SEQS)                                                                        \
            hipLaunchKernelGGL((pq_paged_shared_kernel<T, D, BY_WAVE>), grid, dim3(THREADS), 0, s, a);      \
        else if (a.n_seqs <= MIDDLE_SEQS)                                                                  \
            hipLaunchKernelGGL((pq_paged_shared_kernel<T, D, BY_WORKGROUP>), grid, dim3(THREADS), 0, s, a); \
        else                                                                                               \
            hipLaunchKernelGGL((pq_paged_shared_kernel<T, D, BY_LAUNCH>), grid, dim3(THREADS), 0, s, a);    \
        hipLaunchKernelGGL((pq_paged_shared_merge_kernel<T, D>), rows, dim3(THREADS), 0, s, a);      \
    } while (0)
    PQ_PAGED_BY_TYPE(ctx->cfg.dtype, ctx->cfg.head_dim, LAUNCH);
#undef LAUNCH
    return hipGetLastError();
}
