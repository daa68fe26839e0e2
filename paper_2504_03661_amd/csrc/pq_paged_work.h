// How pq_paged_prefill's kernels share out a call: every workgroup finds its part of the list of work from the requests' rows and
// lengths, which are on the device only.
#pragma once

#include "pq_paged_tile.h"

namespace {

// A piece of a tile's keys: a multiple of KEY_ALIGN, LEAST_KEYS at least.  Tiles of up to WHOLE_KEYS keys are not cut, where there
// are tiles for half of the compute units twice as many: pieces cost more than they save then (32 query / 8 KV heads, 187 tokens
// over 2000 keys: 24 us whole, 33 cut; four times 100 tokens over 2000: 38 and 51; but 12 tokens over 2000: 21 and 15).
constexpr int KEY_ALIGN = 128, LEAST_KEYS = 512, WHOLE_KEYS = 1024;

struct work_place {
    int b, len, first_row, rows;  // sequence, its length, its first row of the tensors, its rows there
    int past;                     // keys in front of its first row's own (negative: the first rows see nothing)
    int tile, split, keys;        // tile of its rows, piece of the keys, keys of a piece
    int slot;                     // of the tile's first piece among the pieces of tiles that are cut
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

// The grids are as large as sequences need whose rows are apart.  Where rows are claimed twice the list of work may be longer, and
// its end is left out; where all claims together are no more than the tensors have rows it is not.  One workgroup, of
// which the list asks nothing, says so.
__device__ inline void check_claims(const pq_paged_attn_args &a, int lane)
{
    int claimed = 0;  // (limited so that 64 lanes' sum fits 32 bits and decides the same)
    for (int b = lane; b < a.n_seqs; b += 64) {
        int start, asked;
        claimed += rows_there(a, b, start, asked);
        claimed = claimed > a.n_tokens ? a.n_tokens + 1 : claimed;
    }
    if (__builtin_amdgcn_readlane(lane_scan(claimed), 63) > a.n_tokens && lane == 0)
        paged_error(a.c.dev_err, PQ_PAGED_ERRFLAG_CLAIMS);
}

// Which sequences a kernel takes, and how it cuts them up
struct work_rule {
    int least, most;  // rows (tokens times query heads of a KV head) of its sequences
    int tile_rows;
    int budget;       // pieces that the keys of all tiles together are cut into at most, and a rest for each tile; 0: one a tile
};

__device__ inline work_rule few_rule(const pq_paged_prefill_plan &w) { return work_rule{1, w.few_rows, PQ_PAGED_FEW_ROWS, w.budget}; }
__device__ inline work_rule tile_rule(const pq_paged_prefill_plan &w) { return work_rule{w.few_rows + 1, INT32_MAX, PQ_PAGED_TILE_ROWS, 0}; }

__device__ inline int rows_of(const pq_paged_attn_args &a, const work_rule &rule, int b, int &start, int &asked)
{
    const int n = rows_there(a, b, start, asked);
    return n * a.G >= rule.least && n * a.G <= rule.most ? n : 0;
}

// Entry e of the list of a kernel's work: sequence after sequence, tile after tile (those that see most first), the pieces of a
// tile's keys.  All sequences are cut into pieces about as long as each other, each into equal ones.  That makes at most
// `budget` pieces and a rest for each tile, and those of tiles that have several are at most 2 `budget`.
// CUT_ONLY: e counts the tiles that have several pieces instead, and its first piece is given.
template <bool CUT_ONLY = false>
__device__ inline bool find_work(const pq_paged_attn_args &a, const work_rule &rule, int e, int lane, work_place &p)
{
    const int tile_rows = rule.tile_rows;
    int most_keys = PQ_MAX_TOKENS, whole_keys = PQ_MAX_TOKENS;
    if (rule.budget > 0) {
        float work = 0.0f, of_tiles = 0.0f;
        for (int b0 = 0; b0 < a.n_seqs; b0 += 64)
            if (b0 + lane < a.n_seqs) {
                int start, asked;
                const int n = (rows_of(a, rule, b0 + lane, start, asked) * a.G + tile_rows - 1) / tile_rows;
                of_tiles += (float)n;
                work += (float)n * (float)paged_length(a.c, b0 + lane);
            }
        most_keys = piece_tokens(wave_sum(work), rule.budget, KEY_ALIGN, LEAST_KEYS);
        whole_keys = 4.0f * wave_sum(of_tiles) < (float)rule.budget ? WHOLE_KEYS : 2 * WHOLE_KEYS;
    }
    int before = 0, slots = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        int start = 0, asked = 0, rows = 0, len = 0, keys = PQ_MAX_TOKENS, per_tile = 1, tiles = 0;
        if (b0 + lane < a.n_seqs) {
            rows = rows_of(a, rule, b0 + lane, start, asked);
            len = paged_length(a.c, b0 + lane);
            tiles = (rows * a.G + tile_rows - 1) / tile_rows;
            if (len > most_keys && len > whole_keys) {
                const int n = (len + most_keys - 1) / most_keys;
                keys = ((len + n - 1) / n + KEY_ALIGN - 1) / KEY_ALIGN * KEY_ALIGN;
                per_tile = (len + keys - 1) / keys;
            }
        }
        const int n = CUT_ONLY && per_tile == 1 ? 0 : CUT_ONLY ? tiles : tiles * per_tile, upto = before + lane_scan(n);
        const int several = per_tile > 1 ? tiles * per_tile : 0, slot = slots + lane_scan(several) - several;
        const uint64_t found = __ballot(e >= upto - n && e < upto);
        if (found != 0) {
            const int l = __builtin_ctzll(found);
            p.b = b0 + l;
            p.len = __builtin_amdgcn_readlane(len, l);
            p.first_row = __builtin_amdgcn_readlane(start, l);
            p.rows = __builtin_amdgcn_readlane(rows, l);
            p.past = p.len - __builtin_amdgcn_readlane(asked, l);
            p.keys = __builtin_amdgcn_readlane(keys, l);
            const int each = __builtin_amdgcn_readlane(per_tile, l), all = __builtin_amdgcn_readlane(tiles, l);
            const int at = e - __builtin_amdgcn_readlane(upto - n, l), from_end = CUT_ONLY ? at : at / each;
            p.tile = all - 1 - from_end;
            p.split = CUT_ONLY ? 0 : at - from_end * each;
            p.slot = __builtin_amdgcn_readlane(slot, l) + from_end * each;
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        slots = __builtin_amdgcn_readlane(slot + several, 63);
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
