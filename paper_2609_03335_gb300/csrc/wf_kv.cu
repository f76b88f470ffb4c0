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
// What it has to move is 16 bytes a token (slot, position, row) and little
// else, so the sums are made by every CTA for itself in shared memory (the rows'
// lengths come from L2) instead of by a kernel before: one launch.
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
constexpr int kTok = 4;         // consecutive tokens of a thread
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
    bool wide;       // slot, pos and row take 16-byte stores
};

// What a token needs of its row: the first token's place in the step, the
// row's length minus that place, and its blocks' place in the ring minus the
// blocks it had.
struct RowSums {
    int32_t *start;  // [rows + 1]
    int32_t *delta;  // [rows]
    int32_t *base;   // [rows]
};

__device__ __forceinline__ uint32_t blocks_of(uint32_t x, uint32_t bs, int shift)
{
    const uint32_t q = shift >= 0 ? x >> shift : x / bs;
    return q + (q * bs != x);
}

// The sums of every row, by one CTA; returns the step's tokens and blocks.
// first: this CTA also writes the rows' outputs that no input may share.
__device__ void row_sums(const ExtendArgs &a, const RowSums &s, uint32_t avail, bool first, uint32_t &tokens,
                         uint32_t &blocks)
{
    __shared__ uint2 warp_sum[kExtThreads / 32];
    __shared__ uint2 cut;  // tokens and blocks before the row that ends the line
    __shared__ uint2 all;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // Needs, staged in place: start = tokens (negative: the row is passed over), base = blocks.
    for (int r = tid; r < a.rows; r += kExtThreads) {
        const int32_t len = a.len[r], add = a.add[r];
        int32_t t = -1, b = 0;
        if (len >= 0 && add >= 0) {
            const uint32_t had = blocks_of((uint32_t)len, a.bs, a.shift);
            const uint32_t then = blocks_of((uint32_t)len + (uint32_t)add, a.bs, a.shift);
            if (then <= (uint32_t)a.width) { t = add; b = (int32_t)(then - had); }
        }
        s.start[r] = t;
        s.base[r] = b;
        s.delta[r] = len;
    }
    if (tid == 0) cut = make_uint2(kSat, kSat);
    __syncthreads();
    const int per = (a.rows + kExtThreads - 1) / kExtThreads;
    const int r0 = min(tid * per, a.rows), r1 = min(r0 + per, a.rows);
    uint2 sum = make_uint2(0, 0);
    for (int r = r0; r < r1; ++r) {
        sum.x = sat_add(sum.x, (uint32_t)max(s.start[r], 0));
        sum.y = sat_add(sum.y, (uint32_t)s.base[r]);
    }
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
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    uint2 w = make_uint2(0, 0);
    for (int i = 0; i < warp; ++i) { w.x = sat_add(w.x, warp_sum[i].x); w.y = sat_add(w.y, warp_sum[i].y); }
    before.x = sat_add(before.x, w.x);
    before.y = sat_add(before.y, w.y);
    if (tid == kExtThreads - 1) all = make_uint2(sat_add(before.x, sum.x), sat_add(before.y, sum.y));
    // The line ends at the one row that is the first past a limit.
    uint2 at = before;
    for (int r = r0; r < r1; ++r) {
        const uint2 next = make_uint2(sat_add(at.x, (uint32_t)max(s.start[r], 0)), sat_add(at.y, (uint32_t)s.base[r]));
        if ((next.x > a.max_tokens || next.y > avail) && at.x <= a.max_tokens && at.y <= avail) cut = at;
        at = next;
    }
    __syncthreads();
    tokens = min(cut.x, all.x);
    blocks = min(cut.y, all.y);
    at = before;
    for (int r = r0; r < r1; ++r) {
        const int32_t t = s.start[r], b = s.base[r], len = s.delta[r];
        const uint2 next = make_uint2(sat_add(at.x, (uint32_t)max(t, 0)), sat_add(at.y, (uint32_t)b));
        const bool late_t = next.x > a.max_tokens, late_b = next.y > avail;
        const int32_t start = (int32_t)(late_t || late_b ? tokens : at.x);
        s.start[r] = start;
        s.delta[r] = len - start;
        s.base[r] = (int32_t)(at.y - blocks_of((uint32_t)max(len, 0), a.bs, a.shift));
        if (first) {
            a.out.start[r] = start;
            a.out.status[r] = t < 0 ? WF_KV_LONG : (late_b ? WF_KV_BLOCKS : 0u) | (late_t ? WF_KV_TOKENS : 0u);
        }
        at = next;
    }
    if (tid == 0) {
        s.start[a.rows] = (int32_t)tokens;
        if (first) a.out.start[a.rows] = (int32_t)tokens;
    }
    __syncthreads();
}

// The row of token t < tokens: the last one whose start is at most t and
// that has tokens, found as the first whose successor starts after t.
__device__ __forceinline__ int row_of(const int32_t *start, int rows, int32_t t)
{
    int lo = 0, hi = rows - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start[mid + 1] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// The tokens of the step, kTok consecutive ones a thread.
__device__ void write_tokens(const ExtendArgs &a, const RowSums &s, uint32_t tokens, uint32_t h0)
{
    const uint32_t n = (uint32_t)a.n_blocks, bs = (uint32_t)a.bs;
    const int64_t quads = ((int64_t)a.max_tokens + kTok - 1) / kTok;
    for (int64_t q = (int64_t)blockIdx.x * kExtThreads + threadIdx.x; q < quads;
         q += (int64_t)gridDim.x * kExtThreads) {
        const uint32_t t0 = (uint32_t)(q * kTok);
        int64_t slot[kTok];
        int32_t pos[kTok], row[kTok];
        int r = t0 < tokens ? row_of(s.start, a.rows, (int32_t)t0) : 0;
        uint32_t end = 0, blk = 0, off = 0, id = 0;
        bool fresh = true;
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
            const uint32_t t = t0 + i;
            if (t >= tokens) {
                slot[i] = -1;
                pos[i] = 0;
                row[i] = -1;
                continue;
            }
            if (i > 0 && t >= end) {
                do ++r; while ((uint32_t)s.start[r + 1] <= t);
                fresh = true;
            }
            const uint32_t p = t + (uint32_t)s.delta[r];
            bool load = true;
            if (fresh) {
                end = (uint32_t)s.start[r + 1];
                blk = a.shift >= 0 ? p >> a.shift : p / bs;
                off = p - blk * bs;
                fresh = false;
            } else if (++off == bs) {
                off = 0;
                ++blk;
            } else {
                load = false;
            }
            if (load) {
                // A block before the row's first new one holds cached tokens: it is in the table.  A new one's first
                // token has off 0 and is always new.
                const uint32_t len = (uint32_t)(s.start[r] + s.delta[r]);
                if (blk * bs < len) {
                    id = (uint32_t)a.table[r * a.stride + blk];
                } else {
                    uint32_t at = h0 + (uint32_t)s.base[r] + blk;
                    if (at >= n) at -= n;
                    id = (uint32_t)__ldg(&a.ring[at]);
                    if (off == 0) a.table[r * a.stride + blk] = (int32_t)id;
                }
            }
            slot[i] = (int64_t)(int32_t)id * bs + off;
            pos[i] = (int32_t)p;
            row[i] = r;
        }
        if (a.wide && t0 + kTok <= a.max_tokens) {
            *(longlong2 *)(a.out.slot + t0) = make_longlong2(slot[0], slot[1]);
            *(longlong2 *)(a.out.slot + t0 + 2) = make_longlong2(slot[2], slot[3]);
            *(int4 *)(a.out.pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
            *(int4 *)(a.out.row + t0) = make_int4(row[0], row[1], row[2], row[3]);
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
}

__global__ void __launch_bounds__(kExtThreads) extend_kernel(const __grid_constant__ ExtendArgs a)
{
    extern __shared__ int32_t rows_sm[];
    const RowSums s{rows_sm, rows_sm + a.rows + 1, rows_sm + 2 * a.rows + 1};
    const int64_t head = a.ends[0], tail = a.ends[1];
    const uint32_t avail = (uint32_t)max(0ll, min((long long)(tail - head), (long long)a.n_blocks));
    uint32_t tokens, blocks;
    row_sums(a, s, avail, blockIdx.x == 0, tokens, blocks);
    // Every CTA has read the lengths and the ends once the last one is here: they may be written, in place too.
    if (last_arrival(a.ticket, gridDim.x)) {
        for (int r = threadIdx.x; r < a.rows; r += kExtThreads)
            a.out.len[r] = s.start[r] + s.delta[r] + (s.start[r + 1] - s.start[r]);
        if (threadIdx.x == 0) {
            a.out.ends[0] = head + blocks;
            a.out.ends[1] = tail;
        }
    }
    write_tokens(a, s, tokens, (uint32_t)((uint64_t)head % (uint32_t)a.n_blocks));
}

// More rows than shared memory holds: one CTA makes the sums in global memory
// for the kernel after it.
__global__ void __launch_bounds__(kExtThreads) extend_sums_kernel(const __grid_constant__ ExtendArgs a, int32_t *sums)
{
    const RowSums s{sums + 2, sums + 3 + a.rows, sums + 3 + 2 * a.rows};
    const int64_t head = a.ends[0], tail = a.ends[1];
    const uint32_t avail = (uint32_t)max(0ll, min((long long)(tail - head), (long long)a.n_blocks));
    uint32_t tokens, blocks;
    row_sums(a, s, avail, true, tokens, blocks);
    for (int r = threadIdx.x; r < a.rows; r += kExtThreads)
        a.out.len[r] = s.start[r] + s.delta[r] + (s.start[r + 1] - s.start[r]);
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
// A CTA takes a group's rows over a tile of table columns: a thread per
// column reads the old rows' entries into shared memory, writes the new
// rows' in their place (all are read before any is written, so in place too),
// and marks the entries that no new row holds: sharing stays within a
// column, so a column decides alone.  The tile's freed ids are listed in
// order, the rows whose last block lies in the tile say whether they need a
// copy, and the last CTA to arrive sums freed blocks and copies over the
// groups.  A second kernel gives the freed ids back and names the copies' blocks, a
// third copies.

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
    int32_t *copy_from;
    uint32_t *tile_copy, *ticket, *n_pairs;
    int4 *group_plan, *pairs;
    int64_t *ring_was;
    int *err;
};

// Length of an old row within the table's width, and the blocks it holds.
__device__ __forceinline__ int64_t row_len(const ReorderArgs &a, int64_t row)
{
    return min((int64_t)max(a.len[row], 0), (int64_t)a.width * a.bs);
}

__device__ __forceinline__ int row_blocks(const ReorderArgs &a, int64_t len) { return (int)((len + a.bs - 1) / a.bs); }

// The old row that row `row` of group g continues, counted in the group, or -1.
__device__ __forceinline__ int row_parent(const ReorderArgs &a, int g, int k, bool &bad)
{
    const int64_t p = (int64_t)a.parent[(int64_t)g * a.group + k] - (int64_t)g * a.group;
    const bool ok = p >= 0 && p < a.group;
    bad = !ok && a.parent[(int64_t)g * a.group + k] != -1;
    return ok ? (int)p : -1;
}

// Exclusive sum of v over the CTA's threads; total: the sum of all.
__device__ __forceinline__ int block_before(int v, int &total)
{
    __shared__ int warps[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(kFull, inc, o);
        if (lane >= o) inc += x;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = inc;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) {
        if (w < warp) before += warps[w];
        total += warps[w];
    }
    return before + inc - v;
}

// The groups' shares of the ring, by the last CTA of the tables' kernel.
__device__ void plan_groups(const ReorderArgs &a)
{
    const int per = (a.groups + kColThreads - 1) / kColThreads;
    const int g0 = min((int)threadIdx.x * per, a.groups), g1 = min(g0 + per, a.groups);
    int give = 0, take = 0;
    for (int g = g0; g < g1; ++g) {
        int f = 0, c = 0;
        for (int t = 0; t < a.tiles; ++t) {
            f += __ldcg(&a.tile_freed[(int64_t)g * a.tiles + t]);
            c += __popc(__ldcg(&a.tile_copy[(int64_t)g * a.tiles + t]));
        }
        a.group_plan[g] = make_int4(0, 0, min(f, c), f);
        give += max(f - c, 0);
        take += max(c - f, 0);
        a.group_plan[g].x = f - c;
    }
    int gives, takes;
    int give_at = block_before(give, gives), take_at = block_before(take, takes);
    for (int g = g0; g < g1; ++g) {
        int4 p = a.group_plan[g];
        const int net = p.x;
        p.x = give_at;
        p.y = take_at;
        a.group_plan[g] = p;
        give_at += max(net, 0);
        take_at += max(-net, 0);
    }
    if (threadIdx.x == 0) {
        const int64_t head = a.ends[0], tail = a.ends[1];
        a.ring_was[0] = head;
        a.ring_was[1] = tail;
        a.to_ends[0] = head + min((int64_t)takes, max(tail - head, (int64_t)0));
        a.to_ends[1] = tail + gives;
        *a.n_pairs = 0;
    }
}

__global__ void __launch_bounds__(kColThreads) reorder_tables_kernel(const __grid_constant__ ReorderArgs a)
{
    extern __shared__ int32_t cells[];  // [group][kTileCols]
    __shared__ int had[kMaxGroup], from[kMaxGroup];
    __shared__ uint32_t goes_on, copied;
    const int g = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles, tid = threadIdx.x, K = a.group;
    const int64_t row0 = (int64_t)g * K;
    if (tid < 32) {
        bool bad;
        const int p = tid < K ? row_parent(a, g, tid, bad) : -1;
        if (tid < K) {
            from[tid] = p;
            had[tid] = row_blocks(a, row_len(a, row0 + tid));
        }
        const uint32_t on = __reduce_or_sync(kFull, p >= 0 ? 1u << p : 0u);
        if (tid == 0) goes_on = on;
    }
    __syncthreads();
    const int j = tile * kTileCols + tid;
    for (int k = 0; k < K; ++k) cells[k * kTileCols + tid] = j < had[k] ? a.table[(row0 + k) * a.stride + j] : -1;
    __syncthreads();
    // The rows whose last block lies here, is partly filled and is a lower row's too: they will get one of their own.
    if (tid < 32) {
        bool mine = false;
        int last = 0;
        int32_t id = -1;
        if (tid < K && from[tid] >= 0) {
            const int64_t n = row_len(a, row0 + from[tid]);
            last = had[from[tid]] - 1;
            mine = n % a.bs != 0 && last / kTileCols == tile;
            if (mine) id = cells[from[tid] * kTileCols + last % kTileCols];
        }
        const uint32_t in = __ballot_sync(kFull, mine);
        bool copy = false;
        if (mine) {
            const uint32_t same = __match_any_sync(in, (unsigned long long)(uint32_t)last << 32 | (uint32_t)id);
            copy = (same & ((1u << tid) - 1u)) != 0;
            if (copy) a.copy_from[row0 + tid] = id;
        }
        const uint32_t mask = __ballot_sync(kFull, copy);
        if (tid == 0) copied = mask;
    }
    __syncthreads();
    // The new rows.  A row that goes on in its own place needs no write.
    const bool in_place = a.table == a.to_table;
    for (int k = 0; k < K; ++k) {
        const int p = from[k];
        if (p < 0 || j >= had[p] || (in_place && p == k) || ((copied >> k & 1u) && j == had[p] - 1)) continue;
        a.to_table[(row0 + k) * a.to_stride + j] = cells[p * kTileCols + tid];
    }
    // Freed: an old row's entry that no row that goes on holds, and no lower one of those that end.
    uint32_t free_mask = 0;
    for (int k = 0; k < K; ++k) {
        if ((goes_on >> k & 1u) || j >= had[k]) continue;
        const int32_t id = cells[k * kTileCols + tid];
        bool held = false;
        for (int q = 0; q < K; ++q)
            held |= q != k && j < had[q] && ((goes_on >> q & 1u) || q < k) && cells[q * kTileCols + tid] == id;
        if (!held) free_mask |= 1u << k;
    }
    int freed;
    int at = block_before(__popc(free_mask), freed);
    int32_t *list = a.freed + ((int64_t)g * a.tiles + tile) * kTileCols * K;
    for (uint32_t m = free_mask; m; m &= m - 1) list[at++] = cells[(__ffs((int)m) - 1) * kTileCols + tid];
    if (tid == 0) {
        a.tile_copy[(int64_t)g * a.tiles + tile] = copied;
        a.tile_freed[(int64_t)g * a.tiles + tile] = freed;
    }
    if (last_arrival(a.ticket, (uint32_t)(a.groups * a.tiles))) plan_groups(a);
}

constexpr int kMoveThreads = 128;

// Freed block i of a group, from the tiles' lists.
__device__ __forceinline__ int32_t freed_id(const ReorderArgs &a, int g, int i)
{
    for (int t = 0; t < a.tiles; ++t) {
        const int n = a.tile_freed[(int64_t)g * a.tiles + t];
        if (i < n) return a.freed[((int64_t)g * a.tiles + t) * kTileCols * a.group + i];
        i -= n;
    }
    return -1;
}

__global__ void __launch_bounds__(kMoveThreads) reorder_moves_kernel(const __grid_constant__ ReorderArgs a)
{
    const int g = blockIdx.x, tid = threadIdx.x, K = a.group;
    const uint32_t n = (uint32_t)a.n_blocks;
    const int4 plan = a.group_plan[g];
    const int64_t head = a.ring_was[0], tail = a.ring_was[1];
    // Give back what the copies do not use.
    const uint32_t tail0 = (uint32_t)((uint64_t)tail % n);
    int before = 0;
    for (int t = 0; t < a.tiles; ++t) {
        const int c = a.tile_freed[(int64_t)g * a.tiles + t];
        const int32_t *list = a.freed + ((int64_t)g * a.tiles + t) * kTileCols * K;
        for (int i = tid; i < c; i += kMoveThreads) {
            const int rest = before + i - plan.z;
            if (rest < 0) continue;
            a.ring[((uint64_t)tail0 + plan.x + rest) % n] = list[i];
        }
        before += c;
    }
    if (tid >= 32) return;
    uint32_t copy = 0;
    for (int t = 0; t < a.tiles; ++t) copy |= a.tile_copy[(int64_t)g * a.tiles + t];
    if (tid >= K) return;
    const int64_t row = (int64_t)g * K + tid;
    bool bad;
    const int p = row_parent(a, g, tid, bad);
    uint32_t status = bad ? WF_KV_PARENT : 0;
    // The parents' lengths are read before any is written: to_len may be len.
    int64_t len = p >= 0 ? row_len(a, (int64_t)g * K + p) : 0;
    __syncwarp(K == 32 ? kFull : (1u << K) - 1u);
    int2 move = make_int2(-1, -1);
    if (copy >> tid & 1u) {
        const int i = __popc(copy & ((1u << tid) - 1u));
        int32_t *cell = &a.to_table[row * a.to_stride + row_blocks(a, len) - 1];  // left to this kernel
        const int64_t in_ring = (int64_t)plan.y + i - plan.z;
        if (i >= plan.z && in_ring >= tail - head) {
            status |= WF_KV_BLOCKS;
            len -= len % a.bs;
        } else {
            const int32_t src = a.copy_from[row];
            const int32_t dst = i < plan.z ? freed_id(a, g, i) : a.ring[((uint64_t)head + in_ring) % n];
            *cell = dst;
            if ((uint32_t)src < n && (uint32_t)dst < n) {
                move = make_int2(src, dst);
                a.pairs[atomicAdd(a.n_pairs, 1u)] = make_int4(src, dst, (int)(len % a.bs), 0);
            } else {
                *a.err = 1;
            }
        }
    }
    a.to_len[row] = (int32_t)len;
    a.copies[2 * row] = move.x;
    a.copies[2 * row + 1] = move.y;
    a.status[row] = status;
}

constexpr int kCopyThreads = 256;
constexpr int kPiece = 16384;  // bytes of a plane's block that a CTA copies at once

// T: the widest type that the cache's addresses are aligned to.
template <class T>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(wf_kv_cache c, int64_t block_bytes, int pieces, const int4 *pairs,
                                                            const uint32_t *n_pairs)
{
    const int64_t items = (int64_t)*n_pairs * c.planes * pieces;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int piece = (int)(it % pieces);
        const int64_t rest = it / pieces;
        const int4 m = pairs[rest / c.planes];
        const int64_t end = min((int64_t)m.z * c.token_bytes, (int64_t)(piece + 1) * kPiece);
        uint8_t *plane = (uint8_t *)c.base + (rest % c.planes) * c.plane_stride;
        const T *src = (const T *)(plane + m.x * block_bytes + (int64_t)piece * kPiece);
        T *dst = (T *)(plane + m.y * block_bytes + (int64_t)piece * kPiece);
        const int n = (int)((end - (int64_t)piece * kPiece) / (int64_t)sizeof(T));
        int i = threadIdx.x;
        for (; i + 3 * kCopyThreads < n; i += 4 * kCopyThreads) {
            T v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = src[i + u * kCopyThreads];
#pragma unroll
            for (int u = 0; u < 4; ++u) dst[i + u * kCopyThreads] = v[u];
        }
        for (; i < n; i += kCopyThreads) dst[i] = src[i];
    }
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
    a.copy_from = d->copy_from;
    a.ticket = d->ticket;
    a.n_pairs = d->n_pairs;
    a.group_plan = d->group_plan;
    a.pairs = d->pairs;
    a.ring_was = d->ring_was;
    a.err = d->err;
    reorder_tables_kernel<<<(unsigned)(a.groups * a.tiles), kColThreads, 4 * (size_t)group * kTileCols, st>>>(a);
    reorder_moves_kernel<<<(unsigned)a.groups, kMoveThreads, 0, st>>>(a);
    if (cache) {
        const int64_t block = cache->token_bytes * kv->block_tokens;
        const int pieces = (int)((block + kPiece - 1) / kPiece);
        const uint64_t bits = (uintptr_t)cache->base | (uint64_t)cache->token_bytes | (cache->planes > 1 ? (uint64_t)cache->plane_stride : 0);
        const int64_t most = (int64_t)a.rows * cache->planes * pieces;
        const unsigned ctas = (unsigned)std::min<int64_t>(most, 8 * d->sms);
        if (bits % 16 == 0) copy_kernel<uint4><<<ctas, kCopyThreads, 0, st>>>(*cache, block, pieces, a.pairs, a.n_pairs);
        else if (bits % 4 == 0) copy_kernel<uint32_t><<<ctas, kCopyThreads, 0, st>>>(*cache, block, pieces, a.pairs, a.n_pairs);
        else copy_kernel<uint8_t><<<ctas, kCopyThreads, 0, st>>>(*cache, block, pieces, a.pairs, a.n_pairs);
    }
    return wf_cuda_check(cudaGetLastError(), "reorder launch");
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
    a.wide = (((uintptr_t)out->slot | (uintptr_t)out->pos | (uintptr_t)out->row) & 15) == 0;
    const int64_t ctas = ((int64_t)a.max_tokens + kTok * kExtThreads - 1) / (kTok * kExtThreads);
    const unsigned grid = (unsigned)std::min<int64_t>(ctas, 2 * d->sms);
    if (a.rows > kSmemRows) {
        extend_sums_kernel<<<1, kExtThreads, 0, st>>>(a, d->sums);
        extend_fill_kernel<<<grid, kExtThreads, 0, st>>>(a, d->sums);
        return wf_cuda_check(cudaGetLastError(), "extend launch");
    }
    const size_t smem = 4 * (3 * (size_t)a.rows + 1);
    int rc = wf_cuda_check(cudaFuncSetAttribute(extend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem),
                           "extend smem attribute");
    if (rc) return rc;
    extend_kernel<<<grid, kExtThreads, smem, st>>>(a);
    return wf_cuda_check(cudaGetLastError(), "extend launch");
}
