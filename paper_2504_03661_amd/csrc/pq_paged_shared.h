// What pq_paged_shared_decode's host and device side share: the lists of work and the partials in the caller's workspace.
#pragma once

#include "pq_paged.h"

#define PQ_PAGED_SHARED_ROWS 32

// A tile of query rows over a piece of the keys of one block table
struct pq_paged_shared_job {
    int table;        // sequence whose blocks
    int position;     // of the group's first member, or the member's own
    int row0, rows;   // rows from there on: a member's query heads of the KV head, member after member
    int k0, k1;       // keys
    int partial;      // row of the partials that the tile's first is
    int unused;
};

// Where the partials of one sequence are: rows of its group's tiles, and of its own
struct pq_paged_shared_member {
    int b;                                    // the sequence; -1: none
    int row, rows, group_row, group_pieces;  // its first row of the group's, theirs, the group's first partial, pieces of a tile
    int own_row, own_pieces;
    int unused;
};

struct pq_paged_shared_work {
    int *head;  // number of jobs
    pq_paged_shared_member *members;
    pq_paged_shared_job *jobs;
    float *partials;  // [KV head][most_rows][d + 2]: base, sum, sums of values
    int most_jobs;
    int64_t most_rows;
};

struct pq_paged_shared_args {
    pq_paged_view c;
    const void *q;
    void *out;
    int64_t q_stride;
    const int32_t *members, *group_start, *shared_len;  // members: or NULL
    float scale_log2e;
    int n_seqs, n_groups, Hq, G, budget;
    pq_paged_shared_work w;
};

int pq_paged_shared_budget(const pq_paged_ctx *ctx);
// Bytes of the workspace; with `w`, where everything is in it.
int64_t pq_paged_shared_layout(const pq_paged_ctx *ctx, int n_seqs, int n_groups, void *workspace, pq_paged_shared_work *w);
hipError_t pq_launch_paged_shared(const pq_paged_ctx *ctx, const pq_paged_shared_args &a, hipStream_t s);
