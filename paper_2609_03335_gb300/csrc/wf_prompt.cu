// Attention over the paged cache for rows with many new tokens: prompts and their chunks.
//
// The sums of wf_attend.cu on the tensor cores' 128 x 128 tiles: S = Q K^T and O += P V with
// tcgen05.mma, S, P and O in TMEM, Q, K and V in shared memory in rows of 128 bytes (64 elements), swizzled.  A CTA (one an SM,
// TMEM and shared memory are full) holds two tiles A and B of 128 queries, each a new token and a head of the
// key head's group, so that what is loaded serves the whole group, and both tiles share what is loaded.
//
//   warps 0-3, 4-7   a thread per query of A, B: scores from TMEM, maximum, powers, weights back as 16-bit numbers;
//                    where a maximum has grown by more than 2^8, O is shrunk (not before: weights up to 2^8 lose nothing)
//   warps 8-11       copies of K, V and Q: the blocks' table, then 16 bytes at a time (8 bits: through registers, to halves)
//   warp 13          which units come next
//   warp 12          the products, in the order  S_A(0) S_B(0) | PV_A(j) S_A(j+1) PV_B(j) S_B(j+1) | ...
//                    so that one tile's powers run beside the other's products
//
// In order of issue is in order of execution: S_A(j+1)'s arrival says that PV_A(j) has read P and written O.
//
// Work is laid on a line and cut into equal stretches as in wf_attend.cu; a unit is the 256 queries, its weight grows with
// the positions that they see.  Every wait ends: after a limit it is reported (wf_attn_status) and the
// kernel runs to its end without waiting.
#include <algorithm>
#include <type_traits>

#include "wf_attend.cuh"
#include "wf_decode.cuh"

namespace {

constexpr int kThreads = 512;
constexpr int kQ = 128, kPair = 2 * kQ;   // queries of a tile, of a unit
constexpr int kKeys = 128;                // positions of a tile
constexpr int kLoaders = 128;
constexpr int kFixed = 2;                 // tiles that a unit's beginning and end are worth
constexpr float kSlack = 8.f;             // log2 of what a maximum may grow by before O is shrunk
constexpr float kLeastScale = 0x1p-64f;

template <bool E, int D> struct Shape {
    static constexpr int kRow = 2 * D;                       // bytes of a key or query in shared memory
    static constexpr int kHalf = kKeys * 128;                // bytes of 64 elements of a tile
    static constexpr int kTile = kKeys * kRow;
    static constexpr int kStages = E ? 4 : D == 128 ? 5 : 8;
    static constexpr int kScales = E ? 3 * kKeys * 4 : 0;    // of a stage: keys' scales, log2 and reciprocal of values'
    static constexpr int kQBytes = 2 * kTile;
    static constexpr int kSmem = 1024 + kQBytes + kStages * (kTile + kScales) + kKeys * 8;
    static_assert(kSmem + 1024 <= 227 * 1024, "shared memory");  // with what is static
};

constexpr int kUnits = 4;  // that the roles may be apart

enum { kBarQFull, kBarQEmpty, kBarS, kBarP = kBarS + 2, kBarO = kBarP + 2, kBarDrain = kBarO + 2, kBarFull, kBarUnit = kBarFull + 16, kBars = kBarUnit + 2 * kUnits };

__device__ __forceinline__ uint32_t smem_of(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{ .reg .pred p;\n"
                 "  mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000;\n"
                 "  selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done;
}

// Waits about 2 s at most; then (or when another thread has given up) on without waiting.
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up, int *err)
{
    if (bar_try(bar, parity)) return;
    for (int i = 0; i < 1 << 20 && !*gave_up; i++)
        if (bar_try(bar, parity)) return;
    if (!*gave_up) {
        *gave_up = 1;
        *err = 2;
    }
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int ID, int N> __device__ __forceinline__ void sync_some() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(N) : "memory"); }

__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit_to(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Both operands in shared memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool more)
{
    asm volatile("{ .reg .pred p;\n"
                 "  setp.ne.b32 p, %4, 0;\n"
                 "  tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)more) : "memory");
}
// The first operand in TMEM.
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t desc, bool more)
{
    asm volatile("{ .reg .pred p;\n"
                 "  setp.ne.b32 p, %4, 0;\n"
                 "  tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b), "r"(desc), "r"((uint32_t)more) : "memory");
}

#define R4(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3])
#define W4(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3])
#define LIST32 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}"
#define LIST32_1 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32}"

// 32 columns of the thread's lane.
__device__ __forceinline__ void tm_load(uint32_t *x, uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " LIST32 ", [%32];"
                 : R4(x, 0), R4(x, 4), R4(x, 8), R4(x, 12), R4(x, 16), R4(x, 20), R4(x, 24), R4(x, 28) : "r"(at) : "memory");
}
__device__ __forceinline__ void tm_store(uint32_t at, const uint32_t *x)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], " LIST32_1 ";" ::"r"(at),
                 W4(x, 0), W4(x, 4), W4(x, 8), W4(x, 12), W4(x, 16), W4(x, 20), W4(x, 24), W4(x, 28) : "memory");
}
__device__ __forceinline__ void tm_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Rows of 128 bytes, swizzled: eight rows are 1,024 bytes, `lead` the bytes to the next 64 elements where these run along rows.
__device__ __forceinline__ uint64_t matrix(uint32_t at, uint32_t lead)
{
    return (uint64_t)(at >> 4 & 0x3FFF) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ float power(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---------------------------------------------------------------------------
// The line of work
// ---------------------------------------------------------------------------

// Weights in 1 / (128 group) of a tile: unit i of a row's key head (queries 256 i ..) sees `have` cached positions and up to
// 256 (i + 1) / group of the step's; the sum over units 0 .. i - 1 is i W + 128 i (i + 1), W = group (128 kFixed + have).
struct Line {
    int64_t w;
    int64_t units;
    __device__ __forceinline__ int64_t upto(int64_t i) const { return i * w + 128 * i * (i + 1); }
    __device__ __forceinline__ int64_t head() const { return upto(units); }
};

__device__ __forceinline__ Line line_of(const AttendArgs &a, const Row &row)
{
    const int64_t m = taken(a, row);
    return {(int64_t)a.group * (kKeys * kFixed + row.len - row.n), (m + kPair - 1) / kPair};
}

struct Span {
    int64_t total;
    int32_t ctas;
    __device__ __forceinline__ int64_t begin(int32_t c) const { return total / ctas * c + total % ctas * c / ctas; }
    __device__ __forceinline__ int32_t owner(int64_t p) const
    {
        int32_t c = (int32_t)max((int64_t)0, min((int64_t)(ctas - 1), (int64_t)((double)p * ctas / (double)total)));
        while (c > 0 && begin(c) > p) c--;
        while (c + 1 < ctas && begin(c + 1) <= p) c++;
        return c;
    }
};

// A stretch is worth six tiles at least, so that only a unit's first and last CTA can find no tile in their part of it.
__device__ __forceinline__ Span span_of(const AttendArgs &a, int64_t total)
{
    return {total, (int32_t)max((int64_t)1, min((int64_t)gridDim.x, total / (6 * kKeys * (int64_t)a.group)))};
}

struct Found {
    int64_t total, row_begin;
    int32_t row;
};

__device__ Found find_row(const AttendArgs &a)
{
    constexpr int kW = kThreads / 32;
    __shared__ int64_t sums[kW];
    __shared__ Found found;
    const int32_t per = (a.rows + kThreads - 1) / kThreads, r0 = min(a.rows, (int32_t)threadIdx.x * per), r1 = min(a.rows, r0 + per);
    int64_t mine = 0;
    for (int32_t r = r0; r < r1; r++) mine += a.kv * line_of(a, row_of(a, r)).head();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int64_t incl = mine;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const int64_t x = __shfl_up_sync(~0u, incl, s);
        if (lane >= s) incl += x;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    int64_t before = incl - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kW; w++) {
        if (w < warp) before += sums[w];
        total += sums[w];
    }
    const Span span = span_of(a, total);
    const int64_t at = blockIdx.x < span.ctas ? span.begin(blockIdx.x) : total;
    if (threadIdx.x == 0) found = {total, total, a.rows};
    __syncthreads();
    if (mine && at >= before && at < before + mine)
        for (int32_t r = r0; r < r1; r++) {
            const int64_t w = a.kv * line_of(a, row_of(a, r)).head();
            if (at < before + w) {
                found = {total, before, r};
                break;
            }
            before += w;
        }
    __syncthreads();
    return found;
}

// A CTA's part of a unit; no tiles: the end.
struct Unit {
    Row row;
    int32_t r, head;        // row of the tables, key head
    int64_t q0;             // the first query: token * group + head of the group
    int32_t queries;        // up to 256
    int32_t t0, n;          // first tile of positions, tiles
    int32_t na, nb;         // of them those that A, B see
    int32_t seen;           // positions that the last query sees
    int32_t first, parts;   // the unit's CTAs
};

// Walks the CTA's stretch.
struct Walk {
    Span span;
    int64_t at, stop, row_begin;
    int32_t r;
    Row row;
    Line line;

    __device__ __forceinline__ Walk(const AttendArgs &a, const Found &f) : span(span_of(a, f.total)), row_begin(f.row_begin), r(f.row)
    {
        at = span.begin(blockIdx.x), stop = span.begin(blockIdx.x + 1);
        row = row_of(a, r), line = line_of(a, row);
    }

    __device__ __forceinline__ bool next(const AttendArgs &a, Unit &u)
    {
        while (at < stop) {
            const int64_t head = line.head();
            if (at >= row_begin + a.kv * head) {
                row_begin += a.kv * head;
                row = row_of(a, ++r), line = line_of(a, row);
                continue;
            }
            u.row = row, u.r = r;
            u.head = (int32_t)((at - row_begin) / head);
            const int64_t base = row_begin + u.head * head, x = at - base;
            // The unit that holds place x: i W + 128 i (i + 1) <= x.
            const double b = (double)line.w + 128.0;
            int64_t i = (int64_t)((sqrt(b * b + 512.0 * (double)x) - b) / 256.0);
            i = max((int64_t)0, min(line.units - 1, i));
            while (i > 0 && line.upto(i) > x) i--;
            while (i + 1 < line.units && line.upto(i + 1) <= x) i++;
            const int64_t begin = base + line.upto(i), end = base + line.upto(i + 1), m = (int64_t)row.n * a.group;
            const int32_t have = row.len - row.n;
            u.q0 = i * kPair;
            u.queries = (int32_t)min((int64_t)kPair, m - u.q0);
            auto sees = [&](int64_t q) { return have + (int32_t)wf_quot((uint32_t)q, a.by_group) + 1; };
            u.seen = sees(u.q0 + u.queries - 1);
            const int32_t tiles_a = (sees(u.q0 + min(u.queries, kQ) - 1) + kKeys - 1) / kKeys, tiles = (u.seen + kKeys - 1) / kKeys;
            const int64_t each = (int64_t)kKeys * a.group;
            auto tile = [&](int64_t p) { return p >= end ? tiles : (int32_t)max((int64_t)0, min((int64_t)tiles, (p - begin) / each - kFixed)); };
            const int32_t t0 = tile(max(at, begin)), t1 = tile(min(stop, end));
            const int64_t here = max(at, begin);
            at = min(stop, end);
            if (t1 <= t0) continue;
            u.t0 = t0, u.n = t1 - t0;
            u.na = max(0, min(t1, tiles_a) - t0), u.nb = u.queries > kQ ? u.n : 0;
            u.first = blockIdx.x, u.parts = 1;
            if (here != begin || at != end) {
                int32_t first = span.owner(begin), last = span.owner(end - 1);
                while (tile(span.begin(first + 1)) <= 0) first++;
                while (tile(span.begin(last)) >= tiles) last--;
                u.first = first, u.parts = last - first + 1;
            }
            return true;
        }
        return false;
    }
};

// ---------------------------------------------------------------------------
// Roles
// ---------------------------------------------------------------------------

struct Shared {
    Unit *units;           // [kUnits]
    uint8_t *q, *kv;       // on 1,024 bytes
    float *scales;
    int64_t *offset;       // [kKeys] of a tile's keys in the cache, -1: none
    uint32_t bars;         // address
    volatile int *gave_up;
    int *err;
    __device__ __forceinline__ uint32_t bar(int i) const { return bars + 8 * i; }
    __device__ __forceinline__ void wait(int i, uint32_t parity) const { bar_wait(bar(i), parity, gave_up, err); }
    // Unit i of the CTA.
    __device__ __forceinline__ const Unit &unit(uint32_t i) const
    {
        wait(kBarUnit + i % kUnits, i / kUnits & 1);
        return units[i % kUnits];
    }
    __device__ __forceinline__ void unit_done(uint32_t i) const { bar_arrive(bar(kBarUnit + kUnits + i % kUnits)); }
};

// One thread: the units, as room comes free.
__device__ __forceinline__ void unit_role(const AttendArgs &a, const Found &f, const Shared &sh)
{
    Walk walk(a, f);
    Unit u;
    for (uint32_t i = 0;; i++) {
        const bool more = walk.next(a, u);
        sh.wait(kBarUnit + kUnits + i % kUnits, (i / kUnits & 1) ^ 1);
        if (!more) u.n = 0;
        sh.units[i % kUnits] = u;
        bar_arrive(sh.bar(kBarUnit + i % kUnits));
        if (!more) return;
    }
}

// Bytes of 16-byte chunk c of row i in a tile.
__device__ __forceinline__ uint32_t place(int i, int c) { return c / 8 * (kKeys * 128) + i * 128 + ((c ^ i) & 7) * 16; }

// log2 of the power of two that a query of 8-bit products is divided by, so that halves hold it: its largest element becomes
// 2^13 .. 2^14.  0 where the queries are halves.
__device__ __forceinline__ int query_exponent(float most)
{
    return most > 0.f && most <= 3.402823466e38f ? min(max((__float_as_int(most) >> 23) - 127 - 13, -100), 127 - 13) : 0;
}

__device__ __forceinline__ const uint8_t *query(const AttendArgs &a, const Unit &u, int q)
{
    const uint32_t f = (uint32_t)(u.q0 + q), tok = wf_quot(f, a.by_group);
    return a.q + (int64_t)(u.row.first + tok) * a.q_token + (int64_t)(u.head * a.group + (f - tok * a.group)) * a.q_head;
}

template <typename T> __device__ __forceinline__ float largest(const uint4 &x)
{
    const float2 a = wf_pair<T>::to_float(x.x), b = wf_pair<T>::to_float(x.y), c = wf_pair<T>::to_float(x.z), d = wf_pair<T>::to_float(x.w);
    return fmaxf(fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(b.x), fabsf(b.y))), fmaxf(fmaxf(fabsf(c.x), fabsf(c.y)), fmaxf(fabsf(d.x), fabsf(d.y))));
}

template <typename T, bool E, int D> __device__ __forceinline__ void load_role(const AttendArgs &a, const Shared &sh)
{
    using S = Shape<E, D>;
    const int tid = threadIdx.x - 256;
    const uint32_t kv = smem_of(sh.kv), q = smem_of(sh.q);
    uint32_t it = 0, units = 0;
    int32_t waiting = 0;   // tiles whose copies are under way and not yet announced (16 bits)
    auto announce = [&](uint32_t i) {
        to_async();
        bar_arrive(sh.bar(kBarFull + i % S::kStages));
    };
    for (;; units++) {
        const Unit &u = sh.unit(units);
        if (!u.n) break;
        const int32_t *table = a.table + u.r * a.table_stride;
        const uint8_t *k = a.k + u.head * a.head_stride, *v = a.v + u.head * a.head_stride;
        const int32_t end = min(u.seen, (u.t0 + u.n) * kKeys);  // positions that count
        // The block of this thread's key of tile j.
        auto block = [&](int32_t j) {
            const int32_t p = min((u.t0 + j) * kKeys + tid, end - 1);
            return block_at(a, table, wf_quot(p, a.by_bs));
        };
        int32_t next = block(0);
        // What is under way belongs to the unit before, which must have it to come to its end.
        copies_wait<0>();
        for (; waiting; waiting--) announce(it - waiting);
        // Queries, once the products of the unit before have read theirs.
        sh.wait(kBarQEmpty, (units & 1) ^ 1);
        {
            constexpr int kPer = D / 8, kRows = kLoaders / kPer;  // 16-byte chunks of a query; queries at once
            const int c = tid % kPer;
            if (!E || std::is_same_v<T, __half>) {
#pragma unroll 4
                for (int i = tid / kPer; i < kPair; i += kRows) {
                    const bool there = i < u.queries;
                    copy16(q + i / kQ * S::kTile + place(i % kQ, c), query(a, u, there ? i : 0) + 16 * c, there);
                }
                copies_commit();
                copies_wait<0>();
            } else {
#pragma unroll 4
                for (int i = tid / kPer; i < kPair; i += kRows) {
                    const bool there = i < u.queries;
                    uint4 x = there ? *reinterpret_cast<const uint4 *>(query(a, u, i) + 16 * c) : make_uint4(0, 0, 0, 0);
                    float most = largest<T>(x);
#pragma unroll
                    for (int s = 1; s < kPer; s *= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, s));
                    const float down = __int_as_float((127 - query_exponent(most)) << 23);
                    uint32_t *w = &x.x;
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float2 y = wf_pair<T>::to_float(w[j]);
                        w[j] = wf_pair<__half>::of_float(y.x * down, y.y * down);
                    }
                    *reinterpret_cast<uint4 *>(sh.q + i / kQ * S::kTile + place(i % kQ, c)) = x;
                }
            }
            to_async();
            bar_arrive(sh.bar(kBarQFull));
        }
        for (int32_t j = 0; j < u.n; j++) {
            const int32_t p = (u.t0 + j) * kKeys + tid;
            int64_t *offset = sh.offset;
            sync_some<1, kLoaders>();
            offset[tid] = p < end ? next * a.block_stride + (int64_t)(p - (int32_t)wf_quot(p, a.by_bs) * a.bs) * a.token_stride : -1;
            const int32_t now = next;
            if (j + 1 < u.n) next = block(j + 1);
            sync_some<1, kLoaders>();
#pragma unroll 1
            for (int side = 0; side < 2; side++, it++) {  // keys, values
                const uint32_t s = it % S::kStages, to = kv + s * S::kTile;
                const uint8_t *from = side ? v : k;
                sh.wait(kBarFull + 8 + s, ((it / S::kStages) & 1) ^ 1);
                if constexpr (!E) {
                    constexpr int kPer = D / 8, kRows = kLoaders / kPer;
                    const int c = tid % kPer;
#pragma unroll 8
                    for (int i = tid / kPer; i < kKeys; i += kRows) {
                        const int64_t o = offset[i];
                        copy16(to + place(i, c), from + (o < 0 ? 0 : o) + 16 * c, o >= 0);
                    }
                    copies_commit();
                    // Two tiles under way; the one before them has landed.
                    if (waiting == 2) {
                        copies_wait<2>();
                        announce(it - 2);
                    } else {
                        waiting++;
                    }
                } else {
                    constexpr int kPer = D / 16, kRows = kLoaders / kPer, kTimes = kKeys / kRows;
                    const int c = tid % kPer;
                    uint4 x[kTimes];
#pragma unroll
                    for (int i = 0; i < kTimes; i++) {
                        const int64_t o = offset[i * kRows + tid / kPer];
                        x[i] = o >= 0 ? *reinterpret_cast<const uint4 *>(from + o + 16 * c) : make_uint4(0, 0, 0, 0);
                    }
                    if (side) {  // the scales of this tile, with its values: both stay until the weights are made
                        const int64_t at = (int64_t)now * a.kv + u.head;
                        const float f = p < end ? fmaxf(a.v_scale[at], kLeastScale) : 1.f;
                        float *sc = sh.scales + s * (S::kScales / 4) + tid;
                        sc[0] = p < end ? a.k_scale[at] : 1.f, sc[kKeys] = __log2f(f), sc[2 * kKeys] = __frcp_rn(f);
                    }
#pragma unroll
                    for (int i = 0; i < kTimes; i++) {
                        const int row = i * kRows + tid / kPer;
                        const uint2 h0 = wf_e4m3_halves(x[i].x), h1 = wf_e4m3_halves(x[i].y), h2 = wf_e4m3_halves(x[i].z), h3 = wf_e4m3_halves(x[i].w);
                        uint8_t *dst = sh.kv + s * S::kTile;
                        *reinterpret_cast<uint4 *>(dst + place(row, 2 * c)) = make_uint4(h0.x, h0.y, h1.x, h1.y);
                        *reinterpret_cast<uint4 *>(dst + place(row, 2 * c + 1)) = make_uint4(h2.x, h2.y, h3.x, h3.y);
                    }
                    announce(it);
                }
            }
        }
        sh.unit_done(units);
    }
    copies_wait<0>();
    for (; waiting; waiting--) announce(it - waiting);
}

template <typename T, bool E, int D> __device__ __forceinline__ void product_role(const Shared &sh, uint32_t tmem)
{
    using S = Shape<E, D>;
    using M = std::conditional_t<E, __half, T>;
    constexpr uint32_t kType = std::is_same_v<M, __nv_bfloat16> ? 1 : 0;
    // Sums in 32-bit floats, both operands of type M, 128 queries; S: 128 keys; O: D elements, the second operand's rows along keys.
    constexpr uint32_t kDescS = 1u << 4 | kType << 7 | kType << 10 | (kKeys / 8) << 17 | (kQ / 16) << 24;
    constexpr uint32_t kDescO = 1u << 4 | kType << 7 | kType << 10 | 1u << 16 | (D / 8) << 17 | (kQ / 16) << 24;
    const uint32_t kv = smem_of(sh.kv), q = smem_of(sh.q);
    uint32_t it = 0, units = 0, np[2] = {0, 0};
    auto full = [&](uint32_t i) { sh.wait(kBarFull + i % S::kStages, (i / S::kStages) & 1); };
    auto done = [&](uint32_t i) { commit_to(sh.bar(kBarFull + 8 + i % S::kStages)); };
    auto scores = [&](int x, uint32_t i) {
        const uint32_t key = kv + i % S::kStages * S::kTile;
#pragma unroll
        for (int s = 0; s < D / 16; s++) {
            const uint32_t at = s / 4 * S::kHalf + s % 4 * 32;
            mma_ss(tmem + x * kKeys, matrix(q + x * S::kTile + at, 16), matrix(key + at, 16), kDescS, s > 0);
        }
        commit_to(sh.bar(kBarS + x));
    };
    auto sums = [&](int x, uint32_t i, bool more) {
        const uint32_t value = kv + i % S::kStages * S::kTile;
#pragma unroll
        for (int s = 0; s < kKeys / 16; s++)
            mma_ts(tmem + 2 * kKeys + x * D, tmem + x * kKeys + 8 * s, matrix(value + s * 2048, S::kHalf), kDescO, more || s > 0);
    };
    for (;; units++) {
        const Unit &u = sh.unit(units);
        const int n[2] = {u.na, u.nb}, most = u.n;
        if (!most) break;
        sh.unit_done(units);
        sh.wait(kBarQFull, units & 1);
        full(it);
        after_sync();
#pragma unroll
        for (int x = 0; x < 2; x++)
            if (n[x] > 0) scores(x, it);
        done(it);
        if (most == 1) commit_to(sh.bar(kBarQEmpty));
        for (int j = 0; j < most; j++) {
            const bool go = j + 1 < most;
            full(it + 2 * j + 1);
            if (go) full(it + 2 * j + 2);
#pragma unroll
            for (int x = 0; x < 2; x++) {
                if (j >= n[x]) continue;
                sh.wait(kBarP + x, np[x] & 1);
                np[x]++;
                after_sync();
                sums(x, it + 2 * j + 1, j > 0);
                if (j + 1 < n[x]) scores(x, it + 2 * j + 2);
                else commit_to(sh.bar(kBarO + x));
            }
            done(it + 2 * j + 1);
            if (go) done(it + 2 * j + 2);
            if (j + 2 == most) commit_to(sh.bar(kBarQEmpty));
        }
        it += 2 * most;
    }
    // Nothing is under way when TMEM is given back.
    commit_to(sh.bar(kBarDrain));
    for (int i = 0; i < 1 << 20 && !bar_try(sh.bar(kBarDrain), 0); i++) {}
}

// Parts in scratch: D / 4 columns of [256 queries] four sums, then [256] references, [256] sums of weights.
template <int D> constexpr int kPart = kPair * (D + 2);

template <typename T, bool E, int D>
__device__ __forceinline__ void power_role(const AttendArgs &a, const Shared &sh, uint32_t tmem, int *last_one)
{
    using S = Shape<E, D>;
    using M = std::conditional_t<E, __half, T>;
    const int x = threadIdx.x / kQ, q = threadIdx.x % kQ, qq = threadIdx.x;  // tile, query of the tile, of the unit
    const uint32_t lane = tmem + ((uint32_t)(q / 32 * 32) << 16), st = lane + x * kKeys, ot = lane + 2 * kKeys + x * D;
    uint32_t ns = 0, no = 0, it = 0, units = 0;
    for (;; units++) {
        const Unit &u = sh.unit(units);
        if (!u.n) break;
        const int n = x ? u.nb : u.na;
        const bool there = qq < u.queries;
        const uint32_t flat = (uint32_t)(u.q0 + (there ? qq : 0)), tok = wf_quot(flat, a.by_group);
        const int32_t seen = u.row.len - u.row.n + (int32_t)tok + 1;
        const int32_t least = u.row.len - u.row.n + (int32_t)wf_quot((uint32_t)(u.q0 + min(u.queries - 1, qq / 32 * 32)), a.by_group) + 1;  // of the warp
        float scale = a.scale;
        if constexpr (E && std::is_same_v<T, __nv_bfloat16>) {
            const uint4 *p = reinterpret_cast<const uint4 *>(query(a, u, there ? qq : 0));
            float most = 0.f;
#pragma unroll 4
            for (int i = 0; i < D / 8; i++) most = fmaxf(most, largest<T>(p[i]));
            scale *= __int_as_float((127 + query_exponent(most)) << 23);
        }
        float ref = -INFINITY, sum = 0.f;
        for (int j = 0; j < n; j++) {
            float s[kKeys];
            uint32_t *w = reinterpret_cast<uint32_t *>(s);
            sh.wait(kBarS + x, ns & 1);
            ns++;
            after_sync();
#pragma unroll
            for (int i = 0; i < 4; i++) tm_load(w + 32 * i, st + 32 * i);
            const float *sc = nullptr;
            if constexpr (E) {
                const uint32_t i = it + 2 * j + 1;
                sh.wait(kBarFull + i % S::kStages, (i / S::kStages) & 1);
                sc = sh.scales + i % S::kStages * (S::kScales / 4);
            }
            tm_loaded();
            if constexpr (E) {
#pragma unroll
                for (int i = 0; i < kKeys; i += 4) {
                    const float4 ks = *reinterpret_cast<const float4 *>(sc + i), lg = *reinterpret_cast<const float4 *>(sc + kKeys + i);
                    s[i] = fmaf(s[i], scale * ks.x, lg.x), s[i + 1] = fmaf(s[i + 1], scale * ks.y, lg.y);
                    s[i + 2] = fmaf(s[i + 2], scale * ks.z, lg.z), s[i + 3] = fmaf(s[i + 3], scale * ks.w, lg.w);
                }
            }
            const int32_t p = (u.t0 + j) * kKeys;
            if (p + kKeys > least) {
#pragma unroll
                for (int i = 0; i < kKeys; i++)
                    if (p + i >= seen) s[i] = -INFINITY;
            }
            float most[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
            for (int i = 4; i < kKeys; i += 4)
#pragma unroll
                for (int k = 0; k < 4; k++) most[k] = fmaxf(most[k], s[i + k]);
            float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            if (!E) top *= scale;
            if (j == 0) {
                ref = top;
            } else if (__any_sync(~0u, top > ref + kSlack)) {
                const bool grow = top > ref + kSlack;
                const float less = grow ? power(ref - top) : 1.f;
                ref = grow ? top : ref;
                sum *= less;
                uint32_t o[32];
#pragma unroll 1
                for (int i = 0; i < D; i += 32) {
                    tm_load(o, ot + i);
                    tm_loaded();
#pragma unroll
                    for (int k = 0; k < 32; k++) o[k] = __float_as_uint(__uint_as_float(o[k]) * less);
                    tm_store(ot + i, o);
                }
            }
            const float base = ref == -INFINITY ? 0.f : ref;
            float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kKeys; i += 2) {
                const float y = power(E ? s[i] - base : fmaf(s[i], scale, -base)), z = power(E ? s[i + 1] - base : fmaf(s[i + 1], scale, -base));
                if constexpr (E) {
                    const float2 inv = *reinterpret_cast<const float2 *>(sc + 2 * kKeys + i);
                    sums[i % 4] = fmaf(y, inv.x, sums[i % 4]), sums[i % 4 + 1] = fmaf(z, inv.y, sums[i % 4 + 1]);
                } else {
                    sums[i % 4] += y, sums[i % 4 + 1] += z;
                }
                w[i / 2] = wf_pair<M>::of_float(y, z);
            }
            sum += (sums[0] + sums[1]) + (sums[2] + sums[3]);
            tm_store(st, w);
            tm_store(st + 32, w + 32);
            tm_stored();
            before_sync();
            bar_arrive(sh.bar(kBarP + x));
        }
        it += 2 * u.n;
        if (n > 0) {
            sh.wait(kBarO + x, no & 1);
            no++;
            after_sync();
        }
        uint8_t *out = a.out + (int64_t)(u.row.first + tok) * a.o_token + (int64_t)(u.head * a.group + (flat - tok * a.group)) * a.o_head;
        auto put = [&](int i, const float *y, float inv) {  // 32 elements
#pragma unroll
            for (int k = 0; k < 32; k += 8)
                *reinterpret_cast<uint4 *>(out + 2 * (i + k)) =
                    make_uint4(wf_pair<T>::of_float(y[k] * inv, y[k + 1] * inv), wf_pair<T>::of_float(y[k + 2] * inv, y[k + 3] * inv),
                               wf_pair<T>::of_float(y[k + 4] * inv, y[k + 5] * inv), wf_pair<T>::of_float(y[k + 6] * inv, y[k + 7] * inv));
        };
        float *part = a.part + (2 * (int64_t)blockIdx.x + (blockIdx.x == u.first)) * kPart<D>;
#pragma unroll 1
        for (int i = 0; i < D; i += 32) {
            float y[32];
            if (n > 0) {
                tm_load(reinterpret_cast<uint32_t *>(y), ot + i);
                tm_loaded();
            } else {
#pragma unroll
                for (int k = 0; k < 32; k++) y[k] = 0.f;
            }
            if (u.parts == 1) {
                if (there) put(i, y, 1.f / sum);
            } else {
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                    __stcg(reinterpret_cast<float4 *>(part) + (i + k) / 4 * kPair + qq, make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]));
            }
        }
        before_sync();
        if (u.parts > 1) {
            __stcg(part + kPair * D + qq, ref);
            __stcg(part + kPair * (D + 1) + qq, sum);
            __threadfence();
            sync_some<2, 256>();
            if (threadIdx.x == 0) {
                const bool last = atomicAdd(a.arrive + u.first, 1u) == (uint32_t)u.parts - 1;
                if (last) a.arrive[u.first] = 0;
                *last_one = last;
            }
            sync_some<2, 256>();
            const bool last = *last_one;
            sync_some<2, 256>();
            if (last) {  // the parts together, in their order
                __threadfence();
                auto part_of = [&](int i) { return a.part + (2 * (int64_t)(u.first + i) + (i == 0)) * kPart<D>; };
                float top = -INFINITY, all = 0.f;
                for (int i = 0; i < u.parts; i++) top = fmaxf(top, __ldcg(part_of(i) + kPair * D + qq));
                const float base = top == -INFINITY ? 0.f : top;
                for (int i = 0; i < u.parts; i++) all += power(__ldcg(part_of(i) + kPair * D + qq) - base) * __ldcg(part_of(i) + kPair * (D + 1) + qq);
#pragma unroll 1
                for (int i = 0; i < D; i += 32) {
                    float y[32];
#pragma unroll
                    for (int k = 0; k < 32; k++) y[k] = 0.f;
                    for (int c = 0; c < u.parts; c++) {
                        const float *from = part_of(c);
                        const float g = power(__ldcg(from + kPair * D + qq) - base);
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 z = __ldcg(reinterpret_cast<const float4 *>(from) + (i + k) / 4 * kPair + qq);
                            y[k] += g * z.x, y[k + 1] += g * z.y, y[k + 2] += g * z.z, y[k + 3] += g * z.w;
                        }
                    }
                    if (there) put(i, y, 1.f / all);
                }
            }
        }
        sh.unit_done(units);
    }
}

template <typename T, bool E, int D> __global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const AttendArgs a)
{
    using S = Shape<E, D>;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, last_one;
    __shared__ Unit units[kUnits];
    const Found f = find_row(a);
    if (f.row >= a.rows) return;
    Shared sh;
    sh.q = raw + (1024 - smem_of(raw) % 1024) % 1024;
    sh.kv = sh.q + S::kQBytes;
    sh.offset = reinterpret_cast<int64_t *>(sh.kv + S::kStages * S::kTile);
    sh.scales = reinterpret_cast<float *>(sh.offset + kKeys);
    sh.units = units, sh.bars = smem_of(bars), sh.gave_up = &gave_up, sh.err = a.err;
    const int warp = threadIdx.x / 32;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < kBars; i++) {
            const bool many = i == kBarQFull || (i >= kBarP && i < kBarO) || (i >= kBarFull && i < kBarFull + 8);
            bar_init(sh.bar(i), many ? 128 : i >= kBarUnit + kUnits ? 385 : 1);  // of a unit's end: 256 + 128 threads and the products'
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_of(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        before_sync();
    }
    __syncthreads();
    after_sync();
    const uint32_t tmem = tmem_at;
    // Registers: launched with 128 a thread; 2 x 128 x 176 + 128 x 88 + 128 x 72 = 65,536.
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        power_role<T, E, D>(a, sh, tmem, &last_one);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        load_role<T, E, D>(a, sh);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 12 && threadIdx.x % 32 == 0) product_role<T, E, D>(sh, tmem);
        if (warp == 13 && threadIdx.x % 32 == 0) unit_role(a, f, sh);
        __syncwarp();
    }
    before_sync();
    __syncthreads();
    after_sync();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <typename T, bool E, int D> int setup()
{
    return wf_cuda_check(cudaFuncSetAttribute(prompt_kernel<T, E, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<E, D>::kSmem), "prompt_kernel");
}

template <typename T, bool E, int D> int launch(const wf_attn *at, const AttendArgs &a, cudaStream_t st)
{
    prompt_kernel<T, E, D><<<at->sms, kThreads, Shape<E, D>::kSmem, st>>>(a);
    return wf_cuda_check(cudaGetLastError(), "prompt_kernel");
}

}  // namespace

int wf_prompt_setup(wf_attn *at)
{
    int rc = setup<__half, false, 64>();
    if (!rc) rc = setup<__nv_bfloat16, false, 64>();
    if (!rc) rc = setup<__half, false, 128>();
    if (!rc) rc = setup<__nv_bfloat16, false, 128>();
    if (!rc) rc = setup<__half, true, 64>();
    if (!rc) rc = setup<__nv_bfloat16, true, 64>();
    if (!rc) rc = setup<__half, true, 128>();
    if (!rc) rc = setup<__nv_bfloat16, true, 128>();
    return rc;
}

size_t wf_prompt_scratch(const wf_attn *at) { return sizeof(float) * 2 * (size_t)at->sms * (at->lim.dim == 64 ? kPart<64> : kPart<128>); }

int wf_launch_prompt(wf_attn *at, const AttendArgs &a, int dtype, int dim, bool eight, cudaStream_t st)
{
    if (dtype == WF_F16) {
        if (dim == 64) return eight ? launch<__half, true, 64>(at, a, st) : launch<__half, false, 64>(at, a, st);
        return eight ? launch<__half, true, 128>(at, a, st) : launch<__half, false, 128>(at, a, st);
    }
    if (dim == 64) return eight ? launch<__nv_bfloat16, true, 64>(at, a, st) : launch<__nv_bfloat16, false, 64>(at, a, st);
    return eight ? launch<__nv_bfloat16, true, 128>(at, a, st) : launch<__nv_bfloat16, false, 128>(at, a, st);
}
