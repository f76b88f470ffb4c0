// Attention over the paged cache: what its kernels share.  wf_attend.cu: rows with few
// new tokens; wf_prompt.cu: rows with many.
#pragma once

#include "wf_layer.cuh"

struct wf_attn {
    int device;
    int sms;
    wf_attn_limits lim;
    void *mem;
    int *err;            // device error word (wf_attn_status): 1 a block or a row, 2 a wait
    uint32_t *arrive;    // arrivals at units that several CTAs share, by the CTA that begins one; every call leaves them 0
    float *part;         // two parts a CTA
    size_t part_bytes;
    int grid[2][2];      // CTAs of attend_kernel by 8 bits or not, dim 64 or 128
};

struct AttendArgs {
    // rows
    const int32_t *table, *start, *len;
    int64_t table_stride, max_tokens;  // entries
    int32_t rows, row_blocks, bs, n_blocks;
    wf_div by_bs, by_group;
    // the layer
    const uint8_t *k, *v;
    int64_t block_stride, token_stride, head_stride;
    const float *k_scale, *v_scale;
    int32_t kv;
    // tensors
    const uint8_t *q;
    uint8_t *out;
    int64_t q_token, q_head, o_token, o_head;
    int32_t group;       // query heads of a key / value head
    float scale;         // log2(e) times the caller's
    // the rows that a launch takes: more than `above` and at most `most` new tokens times group
    int64_t above, most;
    int32_t tile_q;      // queries of a tile of wf_prompt.cu: whole tokens of the group, up to 128
    float *part;
    uint32_t *arrive;
    int *err;
};

struct Row {
    int32_t first, n, len;  // first token in the step, new tokens, tokens cached
};

// Row r, or no tokens where its numbers contradict each other.
__device__ __forceinline__ Row row_of(const AttendArgs &a, int32_t r)
{
    const int32_t s0 = a.start[r], s1 = a.start[r + 1], len = a.len[r];
    Row row = {s0, s1 - s0, len};
    if (s0 == s1) return {s0, 0, len};
    if (s0 < 0 || s1 < s0 || s1 > a.max_tokens || len < row.n || len > (int64_t)a.row_blocks * a.bs) {
        *a.err = 1;
        return {0, 0, 0};
    }
    return row;
}

// The new tokens of row r if this launch takes it, times group.
__device__ __forceinline__ int64_t taken(const AttendArgs &a, const Row &row)
{
    const int64_t m = (int64_t)row.n * a.group;
    return m > a.above && m <= a.most ? m : 0;
}

// A position's block, kept inside the cache.
__device__ __forceinline__ int32_t block_at(const AttendArgs &a, const int32_t *table, uint32_t j)
{
    const int32_t b = table[j];
    if ((uint32_t)b < (uint32_t)a.n_blocks) return b;
    *a.err = 1;
    return 0;
}

int wf_attend_setup(wf_attn *a);
void wf_attend_scratch(const wf_attn *a, size_t *part_bytes, int *ctas);
int wf_launch_attend(wf_attn *at, const AttendArgs &args, int dtype, int dim, bool eight, cudaStream_t st);
int wf_prompt_setup(wf_attn *a);
size_t wf_prompt_scratch(const wf_attn *a);
int wf_launch_prompt(wf_attn *at, const AttendArgs &args, int dtype, int dim, bool eight, cudaStream_t st);
