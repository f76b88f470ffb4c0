// Rows of a paged cache: block tables and slots of a step's tokens
// (wf_kv_extend), and rows put in the order of a beam selection
// (wf_kv_reorder).
//
// wf_kv_extend.  With nb(x) = ceil(x / block_tokens), row r needs
// nb(len + add) - nb(len) blocks and add places; both are summed over the rows
// in order, the row where a sum passes its limit ends the line, and the sums
// before a row say where its blocks lie in the ring and its tokens in the
// step.  A token then finds its row by bisecting the starts.
//
// It has to move 16 bytes a token (slot, position, row) and little else.  So
// the sums are made by every CTA for itself in shared memory (the rows'
// lengths come from L2) instead of by a kernel before: one launch.  2,000 rows
// decoding take 6.3 us and 12 rows 4.0, bound by the launch and two or three trips to L2 in
// turn; 35 M tokens of 2,000 rows 97 us, 5.96 TB/s, bound by the writes (a
// fill of the same arrays reaches 6.9), about 5 us of it the sums.
#include <algorithm>

#include "wf_decode.cuh"

namespace {

constexpr uint32_t kFull = 0xFFFFFFFFu;
constexpr uint32_t kSat = 0x7FFFFFFFu;  // sums stop here: above every limit (sizes are at most 2^31 - 2)

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kSat); }

// Arrival of one CTA; true for the last of n, which resets the count.  What
// the others wrote before it is visible to the caller's threads.
__device__ __forceinline__ bool last_arrival(uint32_t *ticket, uint32_t n)
{
    if (n == 1) return true;
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        last = atomicAdd(ticket, 1u) == n - 1;
        if (last) *ticket = 0;
    }
    __syncthreads();
    if (last) __threadfence();
    return last;
}

// ---------------------------------------------------------------------------
// Extend
// ---------------------------------------------------------------------------

constexpr int kExtThreads = 512;
constexpr int kTok = 2;         // consecutive tokens of a lane: its slots fill 16 bytes, so a warp's stores whole sectors
constexpr int kPer = 4;         // rows of a thread that are summed at once
constexpr int kSmemRows = 16384; // rows whose sums every CTA makes and holds (12 bytes each)

struct ExtendArgs {
    int32_t rows, width, bs, n_blocks, shift;  // shift: log2 of bs, or -1
    int32_t *table;
    int64_t stride;  // entries between table rows
    const int32_t *len, *add, *ring;
    const int64_t *ends;
    uint32_t max_tokens;
    wf_kv_step out;
    uint32_t *ticket;
    bool in_place;   // out.len is len or out.ends is ends
    bool wide;       // the outputs take a lane's tokens in one store each
};

// What a token needs of its row: the first token's place in the step, the
// row's length minus that place, and its blocks' place in the ring minus the
// blocks it had.
struct RowSums {
    int32_t *start;  // [rows + 1]
    int32_t *delta;  // [rows]
    int32_t *base;   // [rows]
};

// Their bytes.
constexpr size_t extend_smem(int rows) { return 4 * (3 * (size_t)rows + 1); }

__device__ __forceinline__ uint32_t blocks_of(uint32_t x, uint32_t bs, int shift)
{
    const uint32_t q = shift >= 0 ? x >> shift : x / bs;
    return q + (q * bs != x);
}

// What a row asks for: tokens (-1: the row is passed over) and blocks.
__device__ __forceinline__ int2 row_needs(const ExtendArgs &a, int32_t len, int32_t add)
{
    if (len < 0 || add < 0 || add > INT32_MAX - len) return make_int2(-1, 0);  // (a table row may hold more than a length counts)
    const uint32_t had = blocks_of((uint32_t)len, a.bs, a.shift), then = blocks_of((uint32_t)len + (uint32_t)add, a.bs, a.shift);
    return then <= (uint32_t)a.width ? make_int2(add, (int)(then - had)) : make_int2(-1, 0);
}

// The sums of every row, by one CTA, kPer consecutive rows a thread at a time;
// returns the step's tokens and blocks.  first: this CTA also writes the
// rows' outputs; write_len: the new lengths too.
__device__ __forceinline__ void row_sums(const ExtendArgs &a, const RowSums &s, uint32_t avail, bool first, bool write_len,
                                         uint32_t &tokens, uint32_t &blocks)
{
    __shared__ uint2 warp_sum[2][kExtThreads / 32];
    __shared__ uint2 cut;  // tokens and blocks before the row that ends the line
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t next_len[kPer], next_add[kPer];
    const auto load = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            next_len[i] = r0 + i < a.rows ? a.len[r0 + i] : 0;
            next_add[i] = r0 + i < a.rows ? a.add[r0 + i] : 0;
        }
    };
    load(tid * kPer);
    uint2 carry = make_uint2(0, 0);  // asked for by the rows so far
    bool over = false;
    int turn = 0;
    for (int lo = 0; lo < a.rows; lo += kPer * kExtThreads, turn ^= 1) {
        const int r0 = lo + tid * kPer;
        int32_t len[kPer];
        int2 need[kPer];
        uint2 sum = make_uint2(0, 0);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            len[i] = next_len[i];
            need[i] = row_needs(a, len[i], next_add[i]);
            sum.x = sat_add(sum.x, (uint32_t)max(need[i].x, 0));
            sum.y = sat_add(sum.y, (uint32_t)need[i].y);
        }
        if (lo + kPer * kExtThreads < a.rows) load(r0 + kPer * kExtThreads);
        uint2 inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(kFull, inc.x, o), y = __shfl_up_sync(kFull, inc.y, o);
            if (lane >= o) { inc.x = sat_add(inc.x, x); inc.y = sat_add(inc.y, y); }
        }
        uint2 before;
        before.x = __shfl_up_sync(kFull, inc.x, 1);
        before.y = __shfl_up_sync(kFull, inc.y, 1);
        if (lane == 0) before = make_uint2(0, 0);
        if (lane == 31) warp_sum[turn][warp] = inc;
        __syncthreads();
        // The warps' sums, scanned by every warp for itself.
        uint2 w = lane < kExtThreads / 32 ? warp_sum[turn][lane] : make_uint2(0, 0);
#pragma unroll
        for (int o = 1; o < kExtThreads / 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(kFull, w.x, o), y = __shfl_up_sync(kFull, w.y, o);
            if (lane >= o) { w.x = sat_add(w.x, x); w.y = sat_add(w.y, y); }
        }
        const uint2 here = make_uint2(__shfl_sync(kFull, w.x, kExtThreads / 32 - 1), __shfl_sync(kFull, w.y, kExtThreads / 32 - 1));
        if (warp) {
            before.x = sat_add(before.x, __shfl_sync(kFull, w.x, warp - 1));
            before.y = sat_add(before.y, __shfl_sync(kFull, w.y, warp - 1));
        }
        before.x = sat_add(before.x, carry.x);
        before.y = sat_add(before.y, carry.y);
        carry.x = sat_add(carry.x, here.x);
        carry.y = sat_add(carry.y, here.y);
        // The line ends at the one row that is the first past a limit.
        if (!over) {
            tokens = carry.x;
            blocks = carry.y;
            if (carry.x > a.max_tokens || carry.y > avail) {
                uint2 at = before;
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const uint2 next = make_uint2(sat_add(at.x, (uint32_t)max(need[i].x, 0)), sat_add(at.y, (uint32_t)need[i].y));
                    if ((next.x > a.max_tokens || next.y > avail) && at.x <= a.max_tokens && at.y <= avail) cut = at;
                    at = next;
                }
                __syncthreads();
                tokens = cut.x;
                blocks = cut.y;
                over = true;
            }
        }
        uint2 at = before;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + i;
            const uint2 next = make_uint2(sat_add(at.x, (uint32_t)max(need[i].x, 0)), sat_add(at.y, (uint32_t)need[i].y));
            const bool late_t = next.x > a.max_tokens, late_b = next.y > avail;
            const int32_t start = (int32_t)(late_t || late_b ? tokens : at.x);
            if (r < a.rows) {
                s.start[r] = start;
                s.delta[r] = len[i] - start;
                s.base[r] = (int32_t)(at.y - blocks_of((uint32_t)max(len[i], 0), a.bs, a.shift));
                if (first) {
                    if (write_len) a.out.len[r] = len[i] + (late_t || late_b ? 0 : max(need[i].x, 0));
                    a.out.start[r] = start;
                    a.out.status[r] = need[i].x < 0 ? WF_KV_LONG : (late_b ? WF_KV_BLOCKS : 0u) | (late_t ? WF_KV_TOKENS : 0u);
                }
            }
            at = next;
        }
    }
    if (tid == 0) {
        s.start[a.rows] = (int32_t)tokens;
        if (first) a.out.start[a.rows] = (int32_t)tokens;
    }
    __syncthreads();
}

// The row of token t < tokens: the last one whose start is at most t and
// that has tokens, found as the first whose successor starts after t.
__device__ __forceinline__ int row_of(const int32_t *start, int lo, int rows, int32_t t)
{
    int hi = rows - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

__device__ __forceinline__ void store_tokens(const ExtendArgs &a, uint32_t t0, const int64_t (&slot)[kTok], const int32_t (&pos)[kTok],
                                             const int32_t (&row)[kTok])
{
    if (a.wide && t0 + kTok <= a.max_tokens) {
        *(longlong2 *)(a.out.slot + t0) = make_longlong2(slot[0], slot[1]);
        *(int2 *)(a.out.pos + t0) = make_int2(pos[0], pos[1]);
        *(int2 *)(a.out.row + t0) = make_int2(row[0], row[1]);
    } else {
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            if (t0 + i >= a.max_tokens) break;
            a.out.slot[t0 + i] = slot[i];
            a.out.pos[t0 + i] = pos[i];
            a.out.row[t0 + i] = row[i];
        }
    }
}

// Where block blk of row r is named: in the table if it holds cached tokens
// (its first token comes before len), else at its place in the ring.
__device__ __forceinline__ const int32_t *block_name(const ExtendArgs &a, const RowSums &s, int r, uint32_t blk, uint32_t len, uint32_t h0)
{
    if (blk * (uint32_t)a.bs < len) return a.table + (r * a.stride + blk);
    uint32_t at = h0 + (uint32_t)s.base[r] + blk;
    if (at >= (uint32_t)a.n_blocks) at -= (uint32_t)a.n_blocks;
    return a.ring + at;
}

// kChunks times 64 tokens of row r, from this lane's first token t0 on: a
// lane's tokens lie in one block or two neighbouring ones, whose names are
// loaded for all chunks before any is used.
template <int kChunks>
__device__ __forceinline__ void row_chunks(const ExtendArgs &a, const RowSums &s, int r, uint32_t t0, uint32_t h0)
{
    constexpr uint32_t kChunk = 32 * kTok;
    const uint32_t bs = (uint32_t)a.bs, n = (uint32_t)a.n_blocks;
    const uint32_t p0 = t0 + (uint32_t)s.delta[r], len = (uint32_t)(s.start[r] + s.delta[r]);
    const uint32_t ring0 = h0 + (uint32_t)s.base[r];
    int32_t *const cells = a.table + r * a.stride;
    uint32_t off[kChunks];
    int32_t id[kChunks], id2[kChunks];
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
        const uint32_t p = p0 + u * kChunk, blk = a.shift >= 0 ? p >> a.shift : p / bs;
        off[u] = p - blk * bs;
        uint32_t at = ring0 + blk, at2 = ring0 + blk + 1;
        if (at >= n) at -= n;
        if (at2 >= n) at2 -= n;
        const bool two = off[u] + kTok > bs;  // the last tokens lie in the next block, a new one
        id[u] = *(blk * bs < len ? cells + blk : a.ring + at);  // (its first token cached: the table names it)
        id2[u] = two ? __ldg(&a.ring[at2]) : 0;
    }
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
        const uint32_t p = p0 + u * kChunk, blk = a.shift >= 0 ? p >> a.shift : p / bs;
        const bool two = off[u] + kTok > bs;
        const int next_at = (int)(bs - off[u]);
        if (off[u] == 0) cells[blk] = id[u];  // the block's first token: the table gets its name
        if (two) cells[blk + 1] = id2[u];
        const int64_t here = (int64_t)id[u] * bs + off[u], there = (int64_t)id2[u] * bs - next_at;
        int64_t slot[kTok];
#pragma unroll
        for (int i = 0; i < kTok; ++i) slot[i] = (two && i >= next_at ? there : here) + i;
        const uint32_t t = t0 + u * kChunk;
        *(longlong2 *)(a.out.slot + t) = make_longlong2(slot[0], slot[1]);
        *(int2 *)(a.out.pos + t) = make_int2((int)p, (int)p + 1);
        *(int2 *)(a.out.row + t) = make_int2(r, r);
    }
}

// The tokens of the step, 64 a warp at a time and kTok consecutive ones a
// lane; where they lie in one row, without a search.
__device__ __forceinline__ void write_tokens(const ExtendArgs &a, const RowSums &s, uint32_t tokens, uint32_t h0)
{
    constexpr uint32_t kChunk = 32 * kTok;
    constexpr int kFast = 4;  // chunks of a row at once
    const uint32_t bs = (uint32_t)a.bs, lane = threadIdx.x & 31;
    // All warps in turn kFast chunks (one, where that gives each warp some), so that what is written at a time lies
    // together: runs of a CTA's own took 105 us for 35 M tokens, this 98.
    const uint32_t chunks = (a.max_tokens + kChunk - 1) / kChunk;
    const uint32_t size = chunks >= gridDim.x * (kExtThreads / 32) * kFast ? kFast : 1, batches = (chunks + size - 1) / size;
    const uint32_t warps = gridDim.x * (kExtThreads / 32);
    int r = 0;
    for (uint32_t b = blockIdx.x * (kExtThreads / 32) + (threadIdx.x >> 5); b < batches; b += warps)
    for (uint32_t c = b * size, c1 = min(c + size, chunks); c < c1; ++c) {
        const uint32_t first = c * kChunk, t0 = first + lane * kTok;
        int64_t slot[kTok];
        int32_t pos[kTok], row[kTok];
        if (first >= tokens) {
#pragma unroll
            for (int i = 0; i < kTok; ++i) { slot[i] = -1; pos[i] = 0; row[i] = -1; }
        } else {
            if ((uint32_t)s.start[r + 1] <= first) r = row_of(s.start, r + 1, a.rows, (int32_t)first);  // (first < tokens: there is one)
            const uint32_t left = (uint32_t)s.start[r + 1] - first;
            if (left >= kFast * kChunk && c + kFast <= c1 && bs >= kTok && a.wide) {
                row_chunks<kFast>(a, s, r, first + lane * kTok, h0);
                c += kFast - 1;
                continue;
            }
            if (left >= kChunk && bs >= kTok && a.wide) {
                row_chunks<1>(a, s, r, first + lane * kTok, h0);
                continue;
            }
            {
                // Each token's row, then all their blocks' names at once.
                const int32_t *name[kTok];
                int32_t *cell[kTok];
                uint32_t off[kTok];
                int q = t0 < tokens ? row_of(s.start, r, a.rows, (int32_t)t0) : r;
#pragma unroll
                for (int i = 0; i < kTok; ++i) {
                    const uint32_t t = t0 + i;
                    name[i] = nullptr;
                    cell[i] = nullptr;
                    off[i] = 0;
                    pos[i] = 0;
                    row[i] = -1;
                    if (t >= tokens) continue;
                    while ((uint32_t)s.start[q + 1] <= t) ++q;
                    const uint32_t p = t + (uint32_t)s.delta[q], blk = a.shift >= 0 ? p >> a.shift : p / bs;
                    off[i] = p - blk * bs;
                    name[i] = block_name(a, s, q, blk, (uint32_t)(s.start[q] + s.delta[q]), h0);
                    if (off[i] == 0) cell[i] = a.table + (q * a.stride + blk);
                    pos[i] = (int32_t)p;
                    row[i] = q;
                }
                int32_t id[kTok];
#pragma unroll
                for (int i = 0; i < kTok; ++i) id[i] = name[i] ? *name[i] : 0;
#pragma unroll
                for (int i = 0; i < kTok; ++i) {
                    if (cell[i]) *cell[i] = id[i];
                    slot[i] = name[i] ? (int64_t)id[i] * bs + off[i] : -1;
                }
                r = __shfl_sync(kFull, q, 31);
            }
        }
        store_tokens(a, t0, slot, pos, row);
    }
}

__global__ void __launch_bounds__(kExtThreads) extend_kernel(const __grid_constant__ ExtendArgs a)
{
    extern __shared__ int32_t rows_sm[];
    const RowSums s{rows_sm, rows_sm + a.rows + 1, rows_sm + 2 * a.rows + 1};
    const int64_t head = a.ends[0], tail = a.ends[1];
    const uint32_t avail = (uint32_t)max(0ll, min((long long)(tail - head), (long long)a.n_blocks));
    uint32_t tokens, blocks;
    row_sums(a, s, avail, blockIdx.x == 0, !a.in_place, tokens, blocks);
    write_tokens(a, s, tokens, (uint32_t)((uint64_t)head % (uint32_t)a.n_blocks));
    if (!a.in_place) {
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            a.out.ends[0] = head + blocks;
            a.out.ends[1] = tail;
        }
        return;
    }
    // Every CTA has read the lengths and the ends once the last one is here: now they may be written in place.
    if (!last_arrival(a.ticket, gridDim.x)) return;
    for (int r = threadIdx.x; r < a.rows; r += kExtThreads) a.out.len[r] = s.start[r] + s.delta[r] + (s.start[r + 1] - s.start[r]);
    if (threadIdx.x == 0) {
        a.out.ends[0] = head + blocks;
        a.out.ends[1] = tail;
    }
}

// More rows than shared memory holds: one CTA makes the sums in global memory
// for the kernel after it.
__global__ void __launch_bounds__(kExtThreads) extend_sums_kernel(const __grid_constant__ ExtendArgs a, int32_t *sums)
{
    const RowSums s{sums + 2, sums + 3 + a.rows, sums + 3 + 2 * a.rows};
    const int64_t head = a.ends[0], tail = a.ends[1];
    const uint32_t avail = (uint32_t)max(0ll, min((long long)(tail - head), (long long)a.n_blocks));
    uint32_t tokens, blocks;
    row_sums(a, s, avail, true, true, tokens, blocks);  // (a row's length is read before it is written)
    if (threadIdx.x == 0) {
        sums[0] = (int32_t)tokens;
        sums[1] = (int32_t)((uint64_t)head % (uint32_t)a.n_blocks);
        a.out.ends[0] = head + blocks;
        a.out.ends[1] = tail;
    }
}

__global__ void __launch_bounds__(kExtThreads) extend_fill_kernel(const __grid_constant__ ExtendArgs a, int32_t *sums)
{
    const RowSums s{sums + 2, sums + 3 + a.rows, sums + 3 + 2 * a.rows};
    write_tokens(a, s, (uint32_t)sums[0], (uint32_t)sums[1]);
}

// ---------------------------------------------------------------------------
// Reorder
// ---------------------------------------------------------------------------
//
// 1. A CTA takes a group's rows over a tile of table columns: a thread per
//    column reads the old rows' entries into shared memory, writes the new
//    rows' in their place (all are read before any is written, so in place too),
//    and marks the entries that no new row holds: sharing stays within a
//    column, so a column decides alone.  The tile's freed ids are listed in
//    order, the rows whose last block lies in the tile say whether they need a
//    copy, and the last CTA to arrive sums freed blocks and copies over the
//    groups.
// 2. With the sums, a CTA per group gives its freed ids back and writes its rows'
//    lengths and last blocks, while other CTAs, which find a copy's blocks by
//    the same sums, copy.
//
// One group of 4 rows takes 7.8 us, 64 groups of 8 rows of 1,024 blocks 13.7 to 15.2:
// bound by L2 trips in turn (lengths, entries, arrivals, sums, lists), about
// 1,100 cycles each, and by code that is fetched once; 64 groups of 8 with 61 MB
// of tokens to copy 35.4 us, 27 of them the copies, 4.5 TB/s of reads and writes.  The
// second kernel is launched while the first runs and waits for it on the GPU, which hides most of a launch.  (Its CTAs could each make the sums for
// themselves and spare the first kernel its arrivals: 1 us less where nothing
// is copied, 2.5 us more where much is.)

constexpr int kColThreads = kTileCols;

struct ReorderArgs {
    int32_t rows, width, bs, n_blocks, group, groups, tiles;
    const int32_t *table, *len, *parent;
    const int64_t *ends;
    int32_t *to_table, *to_len, *ring;
    int64_t *to_ends;
    int64_t stride, to_stride;  // entries between table rows
    int32_t *copies;
    uint32_t *status;
    // scratch
    int32_t *freed, *tile_freed;
    int2 *copy_from;            // per row: the block that its copy is made from, its tokens
    int32_t *copy_rows, *n_copies;  // the rows with copies, in order
    uint32_t *tile_copy, *group_copy, *ticket;
    int4 *group_plan;           // {first place in the ring's tail, in its head, freed blocks used for copies, first copy}
    wf_ring *ring_was;
    int *err;
};

// Length of an old row within the table's width, and the blocks it holds.
__device__ __forceinline__ uint32_t row_len(const ReorderArgs &a, int64_t row)
{
    return (uint32_t)min((int64_t)max(a.len[row], 0), (int64_t)a.width * a.bs);
}

__device__ __forceinline__ int row_blocks(const ReorderArgs &a, uint32_t len) { return (int)((len + (uint32_t)a.bs - 1) / (uint32_t)a.bs); }

// The old row that row `row` of group g continues, counted in the group, or -1.
__device__ __forceinline__ int row_parent(const ReorderArgs &a, int g, int k, bool &bad)
{
    const int64_t p = (int64_t)a.parent[(int64_t)g * a.group + k] - (int64_t)g * a.group;
    const bool ok = p >= 0 && p < a.group;
    bad = !ok && a.parent[(int64_t)g * a.group + k] != -1;
    return ok ? (int)p : -1;
}

// Exclusive sums of v over the CTA's threads; total: the sums of all.
__device__ __noinline__ int3 block_before(int3 v, int3 &total)
{
    __shared__ int3 warps[kColThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int3 inc = v;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(kFull, inc.x, o), y = __shfl_up_sync(kFull, inc.y, o), z = __shfl_up_sync(kFull, inc.z, o);
        if (lane >= o) { inc.x += x; inc.y += y; inc.z += z; }
    }
    __syncthreads();
    if (lane == 31) warps[warp] = inc;
    __syncthreads();
    int3 before = make_int3(inc.x - v.x, inc.y - v.y, inc.z - v.z);
    total = make_int3(0, 0, 0);
#pragma unroll 1
    for (int w = 0; w < kColThreads / 32; ++w) {
        const int3 s = warps[w];
        if (w < warp) { before.x += s.x; before.y += s.y; before.z += s.z; }
        total.x += s.x;
        total.y += s.y;
        total.z += s.z;
    }
    return before;
}

// The groups' shares of the ring, by the last CTA of the tables' kernel; sums:
// two words a group for kTileCols / 2 * group groups at a time.
__device__ void plan_groups(const ReorderArgs &a, int32_t *sums)
{
    const int tid = threadIdx.x, chunk = kTileCols / 2 * a.group;
    const int64_t head = a.ends[0], tail = a.ends[1];
    int3 at = make_int3(0, 0, 0);  // given back, taken, copies
    for (int c0 = 0; c0 < a.groups; c0 += chunk) {
        const int n = min(chunk, a.groups - c0);
        __syncthreads();
        for (int i = tid; i < 2 * n; i += kColThreads) sums[i] = 0;
        __syncthreads();
        // Freed blocks and rows with copies: each row's last block lies in one tile.
        for (int i = tid; i < n * a.tiles; i += kColThreads) {
            const int freed = __ldcg(&a.tile_freed[(int64_t)c0 * a.tiles + i]);
            const uint32_t copy = __ldcg(&a.tile_copy[(int64_t)c0 * a.tiles + i]);
            const int g = a.tiles == 1 ? i : i / a.tiles;
            if (freed) atomicAdd(&sums[2 * g], freed);
            if (copy) atomicOr(&sums[2 * g + 1], (int)copy);
        }
        __syncthreads();
        const int per = (n + kColThreads - 1) / kColThreads, g0 = min(tid * per, n), g1 = min(g0 + per, n);
        int3 mine = make_int3(0, 0, 0), all;
#pragma unroll 1
        for (int g = g0; g < g1; ++g) {
            const int f = sums[2 * g], c = __popc((uint32_t)sums[2 * g + 1]);
            mine.x += max(f - c, 0);
            mine.y += max(c - f, 0);
            mine.z += c;
        }
        int3 here = block_before(mine, all);
        here.x += at.x;
        here.y += at.y;
        here.z += at.z;
#pragma unroll 1
        for (int g = g0; g < g1; ++g) {
            const uint32_t mask = (uint32_t)sums[2 * g + 1];
            const int f = sums[2 * g], c = __popc(mask);
            a.group_plan[c0 + g] = make_int4(here.x, here.y, min(f, c), here.z);
            a.group_copy[c0 + g] = mask;
            for (uint32_t m = mask; m; m &= m - 1) a.copy_rows[here.z++] = (c0 + g) * a.group + __ffs((int)m) - 1;
            here.x += max(f - c, 0);
            here.y += max(c - f, 0);
        }
        at.x += all.x;
        at.y += all.y;
        at.z += all.z;
    }
    if (tid == 0) {
        a.to_ends[0] = head + min((int64_t)at.y, max(tail - head, (int64_t)0));
        a.to_ends[1] = tail + at.x;
        *a.n_copies = at.z;
    }
}

__global__ void __launch_bounds__(kColThreads) reorder_tables_kernel(const __grid_constant__ ReorderArgs a)
{
    extern __shared__ int32_t cells[];  // [group][kTileCols]
    __shared__ int had[kMaxGroup], from[kMaxGroup], part[kMaxGroup];  // blocks, parent, tokens in a partly filled last block
    __shared__ int put[kMaxGroup];                                    // entries of the new row that are written here
    __shared__ uint32_t goes_on, copied;
    const int g = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, tid = threadIdx.x, K = a.group;
    const int64_t row0 = (int64_t)g * K;
    asm volatile("griddepcontrol.launch_dependents;");
    if (tid < 32) {
        bool bad;
        const int p = tid < K ? row_parent(a, g, tid, bad) : -1;
        if (tid < K) {
            const uint32_t len = row_len(a, row0 + tid);
            from[tid] = p;
            had[tid] = row_blocks(a, len);
            part[tid] = (int)(len % (uint32_t)a.bs);
        }
        const uint32_t on = __reduce_or_sync(kFull, p >= 0 ? 1u << p : 0u);
        if (tid == 0) goes_on = on;
    } else if (tid == 32 && blockIdx.x == 0) {
        const int64_t head = a.ends[0], tail = a.ends[1];
        *a.ring_was = {head, tail, (uint32_t)((uint64_t)head % (uint32_t)a.n_blocks), (uint32_t)((uint64_t)tail % (uint32_t)a.n_blocks)};
    }
    __syncthreads();
    const int j = tile * kTileCols + tid;
    const int32_t *column = a.table + row0 * a.stride + j;
#pragma unroll 4
    for (int k = 0; k < K; ++k, column += a.stride) {  // (copies, which no register waits for)
        int32_t *cell = &cells[k * kTileCols + tid];
        if (j < had[k])
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(cell)), "l"(column) : "memory");
        else
            *cell = -1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    // The rows whose last block lies here, is partly filled and is a lower row's too: they will get one of their own.
    if (tid < 32) {
        bool mine = false;
        int last = 0;
        int32_t id = -1, rest = 0;
        if (tid < K && from[tid] >= 0) {
            rest = part[from[tid]];
            last = had[from[tid]] - 1;
            mine = rest != 0 && last / kTileCols == tile;
            if (mine) id = cells[from[tid] * kTileCols + last % kTileCols];
        }
        const uint32_t in = __ballot_sync(kFull, mine);
        bool copy = false;
        if (mine) {
            const uint32_t same = __match_any_sync(in, (unsigned long long)(uint32_t)last << 32 | (uint32_t)id);
            copy = (same & ((1u << tid) - 1u)) != 0;
            if (copy) a.copy_from[row0 + tid] = make_int2(id, rest);
        }
        const uint32_t mask = __ballot_sync(kFull, copy);
        if (tid == 0) copied = mask;
        // A row that goes on in its own place needs no write; a block of its own is named later.
        if (tid < K) put[tid] = from[tid] < 0 || (a.table == a.to_table && from[tid] == tid) ? 0 : last + 1 - (int)copy;
    }
    __syncthreads();
    // The new rows.
    int32_t *to = a.to_table + row0 * a.to_stride + j;
#pragma unroll 4
    for (int k = 0; k < K; ++k, to += a.to_stride)
        if (j < put[k]) *to = cells[from[k] * kTileCols + tid];
    // Freed: an old row's entry that no row that goes on holds, and no lower one of those that end.
    uint32_t free_mask = 0;
#pragma unroll 1
    for (uint32_t ends = ~goes_on & (uint32_t)((1ull << K) - 1); ends; ends &= ends - 1) {
        const int k = __ffs((int)ends) - 1;
        const int32_t id = cells[k * kTileCols + tid];
        bool held = id < 0;  // no entry
#pragma unroll 2
        for (uint32_t others = goes_on | (ends ^ (ends - 1)) >> 1; others; others &= others - 1)
            held |= cells[(__ffs((int)others) - 1) * kTileCols + tid] == id;
        free_mask |= (uint32_t)!held << k;
    }
    int freed = 0;
    if (__syncthreads_or(free_mask != 0)) {
        int3 all;
        int at = block_before(make_int3(__popc(free_mask), 0, 0), all).x;
        freed = all.x;
        int32_t *list = a.freed + ((int64_t)g * a.tiles + tile) * kTileCols * K;
        for (uint32_t m = free_mask; m; m &= m - 1) list[at++] = cells[(__ffs((int)m) - 1) * kTileCols + tid];
    }
    if (tid == 0) {
        a.tile_copy[(int64_t)g * a.tiles + tile] = copied;
        a.tile_freed[(int64_t)g * a.tiles + tile] = freed;
    }
    if (last_arrival(a.ticket, (uint32_t)(a.groups * a.tiles))) plan_groups(a, cells);
}

constexpr int kFinishThreads = 256;
constexpr int kPiece = 16384;  // bytes of a plane's block that a CTA copies at once

// Freed block i of a group (i < 0: none), from the tiles' lists; a whole warp
// calls it, each lane for its own i.
__device__ __noinline__ int32_t freed_block(const ReorderArgs &a, int g, int i)
{
    const int32_t *tiles = a.tile_freed + (int64_t)g * a.tiles;
    const int lane = threadIdx.x & 31;
    int32_t id = -1;
    for (int t0 = 0, before = 0; t0 < a.tiles; t0 += 32) {
        const int n = t0 + lane < a.tiles ? tiles[t0 + lane] : 0;
        int inc = n;
#pragma unroll 1
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(kFull, inc, o);
            if (lane >= o) inc += x;
        }
        int tile = -1, at = 0;
#pragma unroll 1
        for (int t = 0; t < min(32, a.tiles - t0); ++t) {
            const int end = before + __shfl_sync(kFull, inc, t), begin = end - __shfl_sync(kFull, n, t);
            if (i >= begin && i < end) { tile = t0 + t; at = i - begin; }
        }
        if (tile >= 0) id = a.freed[((int64_t)g * a.tiles + tile) * kTileCols * a.group + at];
        before += __shfl_sync(kFull, inc, 31);
        if (!__any_sync(kFull, i >= before)) break;
    }
    return id;
}

// Place i from place `at` on of a ring of n (i below n in a pool that is in order).
__device__ __forceinline__ uint32_t ring_place(uint32_t at, uint64_t i, uint32_t n)
{
    if (i >= n) i %= n;
    const uint32_t p = at + (uint32_t)i;
    return p >= n ? p - n : p;
}

// The block that copy i of group g (i < 0: none) goes to, by a whole warp;
// false for the lanes without a copy or whose copy finds the ring run out.
__device__ __forceinline__ bool copy_block(const ReorderArgs &a, const int4 &plan, int g, int i, const wf_ring &ring, int32_t &to)
{
    to = freed_block(a, g, i < plan.z ? i : -1);
    if (i < plan.z) return i >= 0;
    const int64_t at = (int64_t)plan.y + i - plan.z;
    if (at >= ring.tail - ring.head) return false;
    to = a.ring[ring_place(ring.head_at, (uint64_t)at, (uint32_t)a.n_blocks)];
    return true;
}

// A row of a group: its parent (-1: none, bad: not of the group) and the parent's length.
struct RowFrom {
    int parent;
    bool bad;
    uint32_t len;
};

// A group: its freed blocks back to the ring, its rows' lengths, last blocks and outputs.
__device__ __forceinline__ void finish_group(const ReorderArgs &a, int g, const RowFrom &from)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.group;
    const uint32_t n = (uint32_t)a.n_blocks, mask = a.group_copy[g];
    const int4 plan = a.group_plan[g];
    const wf_ring ring = *a.ring_was;
    // What the copies do not use goes back; a warp takes every eighth tile.
    for (int t0 = 0, before = 0; t0 < a.tiles; t0 += 32) {
        const int c = t0 + lane < a.tiles ? a.tile_freed[(int64_t)g * a.tiles + t0 + lane] : 0;
        int inc = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(kFull, inc, o);
            if (lane >= o) inc += x;
        }
        for (int t = warp; t < min(32, a.tiles - t0); t += kFinishThreads / 32) {
            const int count = __shfl_sync(kFull, c, t), first = before + __shfl_sync(kFull, inc, t) - count - plan.z;
            const int32_t *list = a.freed + ((int64_t)g * a.tiles + t0 + t) * kTileCols * K;
            for (int i = lane; i < count; i += 32)
                if (first + i >= 0) a.ring[ring_place(ring.tail_at, (uint64_t)plan.x + first + i, n)] = list[i];
        }
        before += __shfl_sync(kFull, inc, 31);
    }
    if (warp) return;
    const bool here = lane < K, copies = here && (mask >> lane & 1u);
    const int64_t row = (int64_t)g * K + lane;
    uint32_t status = from.bad ? WF_KV_PARENT : 0, len = from.len;
    const int32_t block = copies ? a.copy_from[row].x : -1;
    int32_t to = -1;
    const bool found = copy_block(a, plan, g, copies ? __popc(mask & ((1u << lane) - 1u)) : -1, ring, to);
    if (!here) return;
    int2 move = make_int2(-1, -1);
    if (found) {
        a.to_table[row * a.to_stride + row_blocks(a, len) - 1] = to;  // left to this kernel
        if ((uint32_t)block < n && (uint32_t)to < n) move = make_int2(block, to);
        else *a.err = 1;
    } else if (copies) {
        status |= WF_KV_BLOCKS;
        len -= len % (uint32_t)a.bs;
    }
    a.to_len[row] = (int32_t)len;
    a.copies[2 * row] = move.x;
    a.copies[2 * row + 1] = move.y;
    a.status[row] = status;
}

// CTAs [0, groups) finish a group each; the others copy.  T: the widest type
// that the cache's addresses are aligned to.  A copying CTA takes a run of
// pieces, those of a copy one after the other.
template <class T>
__global__ void __launch_bounds__(kFinishThreads) reorder_finish_kernel(const __grid_constant__ ReorderArgs a,
                                                                        const __grid_constant__ wf_kv_cache c, int64_t block_bytes,
                                                                        int pieces)
{
    const int group = (int)blockIdx.x < a.groups ? (int)blockIdx.x : -1, lane = threadIdx.x & 31;
    // What the first kernel does not write is read while it runs.  (All parents' lengths are, before any is written: to_len may be len.)
    RowFrom from = {-1, false, 0};
    if (group >= 0 && threadIdx.x < 32 && lane < a.group) {
        from.parent = row_parent(a, group, lane, from.bad);
        if (from.parent >= 0) from.len = row_len(a, (int64_t)group * a.group + from.parent);
    }
    __syncwarp();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (group >= 0) {
        finish_group(a, group, from);
        return;
    }
    const int64_t each = (int64_t)c.planes * pieces, items = *a.n_copies * each, ctas = (int)gridDim.x - a.groups;
    const int64_t run = (items + ctas - 1) / ctas, it0 = ((int)blockIdx.x - a.groups) * run, it1 = min(it0 + run, items);
    const wf_ring ring = *a.ring_was;
    int copy = -1;
    int2 src = make_int2(0, 0);
    int32_t to = 0;
    int64_t bytes = 0;
    for (int64_t it = it0; it < it1; ++it) {
        if ((int)(it / each) != copy) {
            copy = (int)(it / each);
            const int row = a.copy_rows[copy], g = row / a.group;
            const int4 plan = a.group_plan[g];
            src = a.copy_from[row];
            const bool found = copy_block(a, plan, g, copy - plan.w, ring, to);
            bytes = found && (uint32_t)src.x < (uint32_t)a.n_blocks && (uint32_t)to < (uint32_t)a.n_blocks ? src.y * c.token_bytes : 0;
        }
        const int64_t rest = it - copy * each, plane = rest / pieces, first = (rest - plane * pieces) * kPiece;
        // (A piece past the copied bytes has nothing to copy; in 64 bits, since a block may have more than 2^31 bytes.)
        const int n = (int)(min(max(bytes - first, (int64_t)0), (int64_t)kPiece) / (int64_t)sizeof(T));
        uint8_t *base = (uint8_t *)c.base + plane * c.plane_stride + first;
        const T *from_at = (const T *)(base + src.x * block_bytes);
        T *to_at = (T *)(base + to * block_bytes);
        for (int i = threadIdx.x; i < n; i += 4 * kFinishThreads) {
            T v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * kFinishThreads < n) v[u] = from_at[i + u * kFinishThreads];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * kFinishThreads < n) to_at[i + u * kFinishThreads] = v[u];
        }
    }
}

template <class T>
int launch_finish(const ReorderArgs &a, const wf_kv_cache &c, int64_t block_bytes, int pieces, unsigned copiers, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.groups + copiers);
    cfg.blockDim = dim3(kFinishThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return wf_cuda_check(cudaLaunchKernelEx(&cfg, reorder_finish_kernel<T>, a, c, block_bytes, pieces), "reorder finish launch");
}

}  // namespace

int wf_launch_reorder(wf_decode *d, const wf_kv *kv, int32_t group, const int32_t *parent, const wf_kv *to,
                      const wf_kv_cache *cache, int32_t *copies, uint32_t *status, cudaStream_t st)
{
    ReorderArgs a;
    a.rows = kv->rows;
    a.width = kv->row_blocks;
    a.bs = kv->block_tokens;
    a.n_blocks = kv->n_blocks;
    a.group = group;
    a.groups = kv->rows / group;
    a.tiles = (a.width + kTileCols - 1) / kTileCols;
    a.table = kv->table;
    a.len = kv->len;
    a.parent = parent;
    a.ends = kv->ends;
    a.to_table = to->table;
    a.to_len = to->len;
    a.ring = kv->ring;
    a.to_ends = to->ends;
    a.stride = kv->table_stride / 4;
    a.to_stride = to->table_stride / 4;
    a.copies = copies;
    a.status = status;
    a.freed = d->freed;
    a.tile_freed = d->tile_freed;
    a.tile_copy = d->tile_copy;
    a.group_copy = d->group_copy;
    a.copy_from = d->copy_from;
    a.copy_rows = d->copy_rows;
    a.n_copies = d->n_copies;
    a.ticket = d->ticket;
    a.group_plan = d->group_plan;
    a.ring_was = d->ring_was;
    a.err = d->err;
    reorder_tables_kernel<<<(unsigned)(a.groups * a.tiles), kColThreads, 4 * (size_t)group * kTileCols, st>>>(a);
    int rc = wf_cuda_check(cudaGetLastError(), "reorder launch");
    if (rc) return rc;
    if (!cache) return launch_finish<uint32_t>(a, wf_kv_cache{}, 0, 0, 0, st);
    const int64_t block = cache->token_bytes * kv->block_tokens;
    const int pieces = (int)((block + kPiece - 1) / kPiece);
    const uint64_t bits = (uintptr_t)cache->base | (uint64_t)cache->token_bytes | (cache->planes > 1 ? (uint64_t)cache->plane_stride : 0);
    const unsigned copiers = (unsigned)std::min<int64_t>((int64_t)a.rows * cache->planes * pieces, 8 * d->sms);
    if (bits % 16 == 0) return launch_finish<uint4>(a, *cache, block, pieces, copiers, st);
    if (bits % 4 == 0) return launch_finish<uint32_t>(a, *cache, block, pieces, copiers, st);
    return launch_finish<uint8_t>(a, *cache, block, pieces, copiers, st);
}

// The most shared memory that extend_kernel takes, allowed once for a device: the limit is the kernel's there, not a
// call's, so one that a call set for its own rows would refuse the launches of handles on other threads.
int wf_extend_setup()
{
    return wf_cuda_check(cudaFuncSetAttribute(extend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)extend_smem(kSmemRows)),
                         "extend smem attribute");
}

int wf_launch_extend(wf_decode *d, const wf_kv *kv, const int32_t *add, const wf_kv_step *out, cudaStream_t st)
{
    ExtendArgs a;
    a.rows = kv->rows;
    a.width = kv->row_blocks;
    a.bs = kv->block_tokens;
    a.n_blocks = kv->n_blocks;
    a.shift = (a.bs & (a.bs - 1)) == 0 ? __builtin_ctz((unsigned)a.bs) : -1;
    a.table = kv->table;
    a.stride = kv->table_stride / 4;
    a.len = kv->len;
    a.add = add;
    a.ring = kv->ring;
    a.ends = kv->ends;
    a.max_tokens = (uint32_t)out->max_tokens;
    a.out = *out;
    a.ticket = d->ticket;
    a.in_place = out->len == kv->len || out->ends == kv->ends;
    a.wide = ((uintptr_t)out->slot & 15) == 0 && (((uintptr_t)out->pos | (uintptr_t)out->row) & 7) == 0;
    const int64_t ctas = ((int64_t)a.max_tokens + kTok * kExtThreads - 1) / (kTok * kExtThreads);
    const unsigned grid = (unsigned)std::min<int64_t>(ctas, 2 * d->sms);
    if (a.rows > kSmemRows) {
        extend_sums_kernel<<<1, kExtThreads, 0, st>>>(a, d->sums);
        extend_fill_kernel<<<grid, kExtThreads, 0, st>>>(a, d->sums);
        return wf_cuda_check(cudaGetLastError(), "extend launch");
    }
    extend_kernel<<<grid, kExtThreads, extend_smem(a.rows), st>>>(a);
    return wf_cuda_check(cudaGetLastError(), "extend launch");
}
