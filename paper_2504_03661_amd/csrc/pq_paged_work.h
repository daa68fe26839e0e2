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
__device__ inline int rows_there(const pq_paged_attn_args &a, int b, int &start, int &asked)
{
    start = a.tok_start[b];
    const int n = asked = a.tok_len[b];
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

__host__ __device__ inline work_rule few_rule(const pq_paged_prefill_plan &w)
{
    return work_rule{1, w.few_rows, PQ_PAGED_FEW_ROWS, w.few_budget};
}

__host__ __device__ inline work_rule tile_rule(const pq_paged_prefill_plan &w)
{
    return work_rule{w.few_rows + 1, INT32_MAX, w.tile_rows, w.tile_budget};
}

__device__ inline int rows_of(const pq_paged_attn_args &a, const work_rule &rule, int b, int &start, int &asked)
{
    const int n = rows_there(a, b, start, asked);
    return n * a.G >= rule.least && n * a.G <= rule.most ? n : 0;
}

// Entry e of the list of a kernel's work: sequence after sequence, tile after tile (those that see most first), the pieces of a
// tile's keys.  BY_TILE: tile e instead, its first piece.
template <bool BY_TILE = false>
__device__ inline bool find_work(const pq_paged_attn_args &a, const work_rule &rule, int e, int lane, work_place &p)
{
    const int tile_rows = rule.tile_rows;
    p.keys = PQ_MAX_TOKENS;
    if (rule.budget > 0) {
        float work = 0.0f;
        for (int b0 = 0; b0 < a.n_seqs; b0 += 64)
            if (b0 + lane < a.n_seqs) {
                int start, asked;
                const int n = (rows_of(a, rule, b0 + lane, start, asked) * a.G + tile_rows - 1) / tile_rows;
                work += (float)n * (float)paged_length(a.c, b0 + lane);
            }
        p.keys = piece_tokens(wave_sum(work), rule.budget, KEY_ALIGN, LEAST_KEYS);
    }
    int before = 0, tiles_before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int start = 0, asked = 0, rows = 0, len = 0, per_tile = 1, tiles = 0;
        if (b0 + lane < a.n_seqs) {
            rows = rows_of(a, rule, b0 + lane, start, asked);
            len = paged_length(a.c, b0 + lane);
            per_tile = len > 0 ? (len + p.keys - 1) / p.keys : 1;
            tiles = (rows * a.G + tile_rows - 1) / tile_rows;
        }
        const int n = tiles * per_tile, upto = before + lane_scan(n), tiles_upto = BY_TILE ? tiles_before + lane_scan(tiles) : 0;
        const bool mine = BY_TILE ? e >= tiles_upto - tiles && e < tiles_upto : e >= upto - n && e < upto;
        const uint64_t found = __ballot(mine);
        if (found != 0) {
            const int l = __builtin_ctzll(found);
            p.b = b0 + l;
            p.len = __builtin_amdgcn_readlane(len, l);
            p.first_row = __builtin_amdgcn_readlane(start, l);
            p.rows = __builtin_amdgcn_readlane(rows, l);
            p.past = p.len - __builtin_amdgcn_readlane(asked, l);
            const int each = __builtin_amdgcn_readlane(per_tile, l), all = __builtin_amdgcn_readlane(tiles, l);
            const int first = __builtin_amdgcn_readlane(upto - n, l);
            const int from_end = BY_TILE ? e - __builtin_amdgcn_readlane(tiles_upto - tiles, l) : (e - first) / each;
            p.tile = all - 1 - from_end;
            p.split = BY_TILE ? 0 : e - first - from_end * each;
            p.slot = first + from_end * each;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        tiles_before = __builtin_amdgcn_readlane(tiles_upto, 63);
    }
    return false;
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
