// What pq_paged_shared_decode's host and device side share: the lists of work and the partials in the caller's workspace.
#pragma once

#include "pq_paged.h"

// A tile of a group's query rows over a piece of the tokens that its members share
struct pq_paged_shared_job {
    int table;        // sequence whose blocks
    int position;     // of the group's first member
    int row0, rows;   // rows from there on: a member's query heads of the KV head, member after member
    int k0, k1;       // keys
    int partial;      // row of the partials that the tile's first is
    int unused;
};

// What a sequence has behind the shared tokens: a part of the line of all such tokens, in steps of 32
struct pq_paged_shared_own {
    int b, k0, k1;    // the sequence, and its keys
    int begin;        // step of the line that its first tile of rows begins at; the other tiles follow
};

// Where the partials of the sequence at a position are
struct pq_paged_shared_member {
    int b;                                   // the sequence; -1: none
    int row, rows, group_row, group_pieces;  // its first row of the group's, theirs, the group's first partial, pieces of a tile
    int own;                                 // its number among those that have tokens of their own; -1: it has none
    int begin, steps;                        // where they begin on the line, and how many steps they are
};

// How the line is cut: into ranges of `longer` steps, and behind those into ranges of `shorter` ones
struct pq_paged_shared_ranges {
    int n_longer, longer, shorter, count;
};

struct pq_paged_shared_head {
    int group_jobs, group_rows;  // jobs of the groups, and rows of their partials
    int n_own;
    pq_paged_shared_ranges ranges;
};

struct pq_paged_shared_work {
    pq_paged_shared_head *head;
    pq_paged_shared_member *members;
    pq_paged_shared_job *jobs;    // of the groups
    pq_paged_shared_own *own;
    int *first;                   // the sequence of `own` that each range begins in
    float2 *sums;                 // [KV head][most_rows]: base, sum
    float *partials;              // [KV head][most_rows][d]: sums of values
    int64_t most_rows;
};

struct pq_paged_shared_args {
    pq_paged_view c;
    const void *q;
    void *out;
    int64_t q_stride;
    const int32_t *members, *group_start, *shared_len;  // members: or NULL
    float scale_log2e;
    int n_seqs, n_groups, Hq, G;
    int workgroups;  // for each KV head
    pq_paged_shared_work w;
};

// Bytes of the workspace; with `a`, where everything is in it, and how the call is cut.
int64_t pq_paged_shared_layout(const pq_paged_ctx *ctx, int n_seqs, int n_groups, void *workspace, pq_paged_shared_args *a);
hipError_t pq_launch_paged_shared(const pq_paged_ctx *ctx, const pq_paged_shared_args &a, hipStream_t s);
