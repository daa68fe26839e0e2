// How pq_paged_prefill's kernels share out a call: every workgroup finds its part of the list of work from the requests' rows and
// lengths, which are on the device only.
#pragma once

#include "pq_paged_tile.h"

namespace {

constexpr int KEY_ALIGN = 128, LEAST_KEYS = 512;  // of a piece of a tile's keys

struct work_place {
    int b, len, first_row, rows;  // sequence, its length, its first row of the tensors, its rows there
    int past;                     // keys in front of its first row's own (negative: the first rows see nothing)
    int tile, split, keys;        // tile of its rows, piece of the keys, keys of a piece
    int slot;                     // of the tile's first piece among the call's
};

// Rows of sequence b that lie in the tensors
__device__ inline int rows_there(const pq_paged_attn_args &a, int b, int &start)
{
    start = a.tok_start[b];
    const int n = a.tok_len[b];
    if (start < 0 || start >= a.n_tokens || n <= 0)
        return 0;
    return n < a.n_tokens - start ? n : a.n_tokens - start;
}

// Which sequences a kernel takes, and how it cuts them up
struct work_rule {
    int least, most;  // rows (tokens times query heads of a KV head) of its sequences
    int tile_rows;
    int budget;       // pieces that the keys of all tiles together are cut into at most, and a rest for each tile; 0: one a tile
};

__device__ inline int rows_of(const pq_paged_attn_args &a, const work_rule &rule, int b, int &start)
{
    const int n = rows_there(a, b, start);
    return n * a.G >= rule.least && n * a.G <= rule.most ? n : 0;
}

// The list of a kernel's work: sequence after sequence, tile after tile (those that see most first), the pieces of a tile's
// keys.  Finds the sequence for which `mine(entries before it, entries up to its end, first row, rows)` holds.
template <typename F>
__device__ inline bool find_sequence(const pq_paged_attn_args &a, const work_rule &rule, int lane, F mine, work_place &p, int &entries_before,
                                     int &tiles, int &per_tile)
{
    const int tile_rows = rule.tile_rows, budget = rule.budget;
    p.keys = PQ_MAX_TOKENS;
    if (budget > 0) {
        int64_t work = 0;
        for (int b0 = 0; b0 < a.n_seqs; b0 += 64)
            if (b0 + lane < a.n_seqs) {
                int start;
                const int n = (rows_of(a, rule, b0 + lane, start) * a.G + tile_rows - 1) / tile_rows;
                work += (int64_t)n * paged_length(a.c, b0 + lane);
            }
        work = __shfl(lane_scan(work, lane), 63, 64);
        const int64_t share = (work + budget - 1) / budget;
        const int n = share < PQ_MAX_TOKENS ? (int)share : PQ_MAX_TOKENS;
        p.keys = n > LEAST_KEYS ? (n + KEY_ALIGN - 1) / KEY_ALIGN * KEY_ALIGN : LEAST_KEYS;
    }
    int before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int start = 0, rows = 0, len = 0, splits = 1, n = 0;
        if (b0 + lane < a.n_seqs) {
            rows = rows_of(a, rule, b0 + lane, start);
            len = paged_length(a.c, b0 + lane);
            splits = len > 0 ? (len + p.keys - 1) / p.keys : 1;
            n = (rows * a.G + tile_rows - 1) / tile_rows * splits;
        }
        const int upto = before + (int)lane_scan(n, lane);
        const uint64_t found = __ballot(n > 0 && mine(upto - n, upto, start, rows));
        if (found != 0) {
            const int l = __builtin_ctzll(found);
            p.b = b0 + l;
            p.len = __builtin_amdgcn_readlane(len, l);
            p.first_row = __builtin_amdgcn_readlane(start, l);
            p.rows = __builtin_amdgcn_readlane(rows, l);
            p.past = p.len - __builtin_amdgcn_readfirstlane(a.tok_len[p.b]);
            per_tile = __builtin_amdgcn_readlane(splits, l);
            tiles = __builtin_amdgcn_readlane(n, l) / per_tile;
            entries_before = __builtin_amdgcn_readlane(upto - n, l);
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// entry e of the list
__device__ inline bool find_work(const pq_paged_attn_args &a, const work_rule &rule, int e, int lane, work_place &p)
{
    int before, tiles, per_tile;
    if (!find_sequence(a, rule, lane, [&](int from, int upto, int, int) { return e >= from && e < upto; }, p, before, tiles, per_tile))
        return false;
    p.tile = tiles - 1 - (e - before) / per_tile;
    p.split = (e - before) % per_tile;
    p.slot = e - p.split;
    return true;
}

// the first piece of the tile that query head g (of its KV head) of row t of the tensors is in
__device__ inline bool find_row(const pq_paged_attn_args &a, const work_rule &rule, int t, int g, int lane, work_place &p)
{
    int before, tiles, per_tile;
    if (!find_sequence(a, rule, lane, [&](int, int, int start, int rows) { return t >= start && t - start < rows; }, p, before, tiles, per_tile))
        return false;
    p.tile = ((t - p.first_row) * a.G + g) / rule.tile_rows;
    p.split = 0;
    p.slot = before + (tiles - 1 - p.tile) * per_tile;
    return true;
}

// A tile's rows of its sequence (token by token, query head by query head), and the pieces that the keys they see are in
struct tile_place {
    int row0, rows, sees, pieces;
    __device__ tile_place(const work_place &p, int G, int tile_rows)
    {
        const int all = p.rows * G;
        row0 = p.tile * tile_rows;
        rows = (row0 + tile_rows < all ? row0 + tile_rows : all) - row0;
        sees = p.past + (row0 + rows - 1) / G + 1;  // keys that the last row sees
        sees = __builtin_amdgcn_readfirstlane(sees < 0 ? 0 : sees);
        pieces = sees > p.keys ? (sees + p.keys - 1) / p.keys : 1;
    }
};

}  // namespace
