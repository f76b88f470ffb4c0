// Internal definitions of the calls on a replica's rows: cache bookkeeping
// (wf_kv.cu) and beam selection (wf_beam.cu).
#pragma once

#include "wf_internal.cuh"

// The pool's ends before a call, and their places in the ring.
struct wf_ring {
    int64_t head, tail;
    uint32_t head_at, tail_at;
};

// Per-call scratch, one device allocation made by wf_decode_create.
struct wf_decode {
    int device;
    int sms;
    wf_decode_limits lim;
    void *mem;
    int *err;              // device error word (wf_decode_status)
    uint32_t *ticket;      // [1 + max_rows] arrivals of CTAs; every call leaves them 0
    int32_t *sums;         // [3 * max_rows + 3] extend's sums where shared memory does not hold them
    // reorder
    int32_t *freed;        // [max_rows][row blocks rounded up to a tile] ids of a tile's freed blocks
    int32_t *tile_freed;   // [groups][tiles] their count
    uint32_t *tile_copy;   // [groups][tiles] rows that need a copy of a block of this tile
    int2 *copy_from;       // [max_rows] the block that a row's copy is made from, its tokens
    int32_t *copy_rows;    // [max_rows] the rows with copies
    int32_t *n_copies;
    uint32_t *group_copy;  // [groups] rows with copies
    int4 *group_plan;      // [groups] {first place in the ring's tail, in its head, freed blocks used for copies, first copy}
    wf_ring *ring_was;
    // select
    float4 *part;          // [parts] a warp's part of a row: reference, sum of exponentials, maximum
    float *most;           // [units] the maximum of each unit of the rows
    int64_t parts, units;
};

constexpr int kTileCols = 256;     // columns of the tables that a CTA of the reorder takes
constexpr int kMaxGroup = 32;      // rows of a group, beams
constexpr int kMaxKeep = 64;

void wf_beam_scratch(int64_t rows, int64_t vocab, int sms, int64_t *parts, int64_t *units);
int wf_extend_setup();
int wf_launch_extend(wf_decode *d, const wf_kv *kv, const int32_t *add, const wf_kv_step *out, cudaStream_t st);
int wf_launch_reorder(wf_decode *d, const wf_kv *kv, int32_t group, const int32_t *parent, const wf_kv *to,
                      const wf_kv_cache *cache, int32_t *copies, uint32_t *status, cudaStream_t st);
int wf_launch_select(wf_decode *d, const wf_beam *in, const wf_beam_out *out, cudaStream_t st);
