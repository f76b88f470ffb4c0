// Attention over the paged cache: what its kernels share.  wf_attend.cu: rows with few
// new tokens; wf_prompt.cu: rows with many.
#pragma once

#include "wf_layer.cuh"

struct wf_attn {
    int device;
    int sms;
    wf_attn_limits lim;
    int polls;           // of a bounded wait
    void *mem;
    size_t zeroed;       // bytes at its beginning that are 0 between calls: err and arrive
    int *err;            // device error words (wf_attn_status): not 0 after a bad block or row; after a wait that ran out
    // Of attend_kernel, of prompt_kernel, which may run side by side:
    uint32_t *arrive[2]; // arrivals at units that several CTAs share, by the CTA that begins one; a call whose waits do not run out leaves them 0
    float *part[2];      // two parts a CTA
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
    // Rows of up to `few` queries to a key head are attend_kernel's, the others prompt_kernel's; `both`: it runs beside the other.
    int64_t few;
    int32_t both, sms;
    int32_t pair_cost;   // cycles of a prompt_kernel's tile on an SM
    int32_t tile_cost;   // of an attend_kernel's on an SM of its own, and
    int32_t tile_share;  // 1 / 16 of the GPU's cycles that its bytes take at least
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
        a.err[0] = 1;
        return {0, 0, 0};
    }
    return row;
}

// Work.  attend_kernel: units of up to 16 queries, in tiles of 64 positions, each worth kFixed tiles more.  prompt_kernel: units of 2 tile_q
// queries; in 1 / (128 group) of a tile of 128 positions, unit i of a row's key head (queries 2 t i .., t = tile_q) sees `have` cached
// positions and up to 2 t (i + 1) / group of the step's, so that the sum over units 0 .. i - 1 is i W + t i (i + 1), W = group (128 kFixed + have).
constexpr int kFixed = 2;         // tiles that a unit's beginning and end are worth
constexpr int kShortQueries = 16, kShortTile = 64, kKeys = 128;

__device__ __forceinline__ int64_t queries_of(const AttendArgs &a, const Row &row) { return (int64_t)row.n * a.group; }

__device__ __forceinline__ int64_t unit_work(const Row &row) { return kFixed + (row.len + kShortTile - 1) / kShortTile; }
__device__ __forceinline__ int64_t short_work(const AttendArgs &a, const Row &row)
{
    const int64_t m = queries_of(a, row);
    return m <= a.few ? a.kv * ((m + kShortQueries - 1) / kShortQueries) * unit_work(row) : 0;
}

struct Line {
    int64_t w, tile_q;
    int64_t units;
    __device__ __forceinline__ int64_t upto(int64_t i) const { return i * w + tile_q * i * (i + 1); }
    __device__ __forceinline__ int64_t head() const { return upto(units); }
};

__device__ __forceinline__ Line line_of(const AttendArgs &a, const Row &row)
{
    const int64_t m = queries_of(a, row);
    return {(int64_t)a.group * (kKeys * kFixed + row.len - row.n), a.tile_q, m > a.few ? (m + 2 * a.tile_q - 1) / (2 * a.tile_q) : 0};
}
__device__ __forceinline__ int64_t long_work(const AttendArgs &a, const Row &row) { return a.kv * line_of(a, row).head(); }

// The SMs that prompt_kernel takes where both kernels run side by side, the others being attend_kernel's: as many as make both end at the
// same time.  Decoding alone cannot use them all (its bytes take tile_share / 16 of the whole GPU's cycles a tile), nor does a prompt's work shrink its bytes.
__device__ __forceinline__ int32_t prompt_sms(const AttendArgs &a, int64_t short_total, int64_t long_total)
{
    if (!a.both || !short_total) return a.sms;
    const double p = (double)long_total / ((double)kKeys * a.group) * a.pair_cost, d = (double)short_total * a.tile_cost;
    const double even = a.sms * p / (p + d), bytes = (double)short_total * a.tile_share / 16.0;  // cycles
    // With `even` SMs both take (p + d) / sms cycles; if the bytes take longer, prompts need only p / bytes SMs.
    const double want = (p + d) / a.sms >= bytes ? even : p / bytes;
    return max(1, min(a.sms - 1, (int32_t)ceil(want)));
}

// a / b for a >= 0, b > 0; in 32 bits where they fit, as they mostly do (a division in 64 bits is a hundred instructions).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b)
{
    return ((uint64_t)a | (uint64_t)b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// A line of work in equal stretches.
struct Span {
    int64_t total;
    int32_t ctas;
    __device__ __forceinline__ int64_t begin(int32_t c) const 
    {
        const int64_t q = quotient(total, ctas);
        return q * c + quotient((total - q * ctas) * c, ctas);
    }
    // The CTA whose stretch holds place p < total.
    __device__ __forceinline__ int32_t owner(int64_t p) const
    {
        int32_t c = (int32_t)max((int64_t)0, min((int64_t)(ctas - 1), (int64_t)((double)p * ctas / (double)total)));
        while (c > 0 && begin(c) > p) c--;
        while (c + 1 < ctas && begin(c + 1) <= p) c++;
        return c;
    }
};

// The line, how it is cut (by `cut`, from this kernel's and the other's totals), and the row (where it begins, its number, itself) that holds
// this CTA's first place; r = rows: this CTA has none.
struct Found {
    Span span;
    int64_t row_begin;
    int32_t r;
    Row row;
};

template <int THREADS, bool LONG, typename CUT> __device__ Found find_row(const AttendArgs &a, CUT cut)
{
    constexpr int kW = THREADS / 32;
    __shared__ int64_t sums[kW], others[kW];
    __shared__ Found found;
    const int32_t per = (a.rows + THREADS - 1) / THREADS, r0 = min(a.rows, (int32_t)threadIdx.x * per), r1 = min(a.rows, r0 + per);
    int64_t mine = 0, other = 0;
    Row row = {};
    for (int32_t r = r0; r < r1; r++) {
        row = row_of(a, r);
        mine += LONG ? long_work(a, row) : short_work(a, row);
        if (a.both) other += LONG ? short_work(a, row) : long_work(a, row);
    }
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int64_t incl = mine;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const int64_t x = __shfl_up_sync(~0u, incl, s);
        if (lane >= s) incl += x;
        other += __shfl_xor_sync(~0u, other, s);
    }
    if (lane == 31) sums[warp] = incl, others[warp] = other;
    __syncthreads();
    int64_t before = incl - mine, total = 0, rest = 0;
#pragma unroll
    for (int w = 0; w < kW; w++) {
        if (w < warp) before += sums[w];
        total += sums[w], rest += others[w];
    }
    const Span span = {total, cut(total, rest)};
    const int64_t at = blockIdx.x < span.ctas ? span.begin(blockIdx.x) : total;
    if (threadIdx.x == 0) found = {span, total, a.rows, {}};
    __syncthreads();
    if (mine && at >= before && at < before + mine && per == 1) {
        found = {span, before, r0, row};
    } else if (mine && at >= before && at < before + mine) {
        for (int32_t r = r0; r < r1; r++) {
            row = row_of(a, r);
            const int64_t w = LONG ? long_work(a, row) : short_work(a, row);
            if (at < before + w) {
                found = {span, before, r, row};
                break;
            }
            before += w;
        }
    }
    __syncthreads();
    return found;
}

// A position's block, kept inside the cache.
__device__ __forceinline__ int32_t block_at(const AttendArgs &a, const int32_t *table, uint32_t j)
{
    const int32_t b = table[j];
    if ((uint32_t)b < (uint32_t)a.n_blocks) return b;
    a.err[0] = 1;
    return 0;
}

// A weight of 0 does not undo a value that is no finite number.  So where some queries of a tile see a position and others do not, such values are taken
// out of the tile's products, and added here for the queries that do: positions begin .. end - 1, of N elements of the values v of type V, to x.  Their
// weights, whatever they are, leave an infinity what it is, and NaN.
template <typename V, int N>
__device__ __forceinline__ void add_unfit(const AttendArgs &a, const int32_t *table, const uint8_t *v, int32_t begin, int32_t end, float (&x)[N])
{
#pragma unroll 1
    for (int32_t p = begin; p < end; p++) {
        const uint32_t j = wf_quot(p, a.by_bs);
        const uint8_t *from = v + block_at(a, table, j) * a.block_stride + (p - (int32_t)j * a.bs) * a.token_stride;
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            if constexpr (sizeof(V) == 1) {
                const uint32_t w = wf_unfit<V>(*reinterpret_cast<const uint32_t *>(from + i));
#pragma unroll
                for (int k = 0; k < 4; k++)
                    if (w >> (8 * k + 7) & 1) x[i + k] = NAN;
            } else {
                const uint2 w = *reinterpret_cast<const uint2 *>(from + 2 * i);
                if (wf_unfit<V>(w.x) | wf_unfit<V>(w.y)) {
                    const float2 lo = wf_pair<V>::to_float(w.x), hi = wf_pair<V>::to_float(w.y);
                    const float y[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        if (!isfinite(y[k])) x[i + k] += y[k];
                }
            }
        }
    }
}

int wf_attend_setup(wf_attn *a);
void wf_attend_scratch(const wf_attn *a, size_t *part_bytes, int *ctas);
int wf_launch_attend(wf_attn *at, const AttendArgs &args, int dtype, int dim, bool eight, cudaStream_t st);
int wf_prompt_setup(wf_attn *a);
size_t wf_prompt_scratch(const wf_attn *a);
int wf_launch_prompt(wf_attn *at, const AttendArgs &args, int dtype, int dim, bool eight, cudaStream_t st);
