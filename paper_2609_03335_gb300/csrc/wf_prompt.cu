// Attention over the paged cache for rows with many new tokens: prompts and their chunks.
//
// The sums of wf_attend.cu on the tensor cores' 128 x 128 tiles: S = Q K^T and O += P V with
// tcgen05.mma, S, P and O in TMEM, Q, K and V in shared memory in rows of 128 bytes (64 elements), swizzled.  A CTA (one an SM,
// TMEM and shared memory are full) holds two tiles A and B of 128 queries, each a new token and a head of the
// key head's group, so that what is loaded serves the whole group, and both tiles share what is loaded.
//
//   warps 0-3, 4-7   a thread per query of A, B: scores from TMEM, maximum, powers, weights back as 16-bit numbers;
//                    where a maximum has grown by more than 2^8, O is shrunk (not before: weights up to 2^8 lose nothing)
//   warp 14          copies of K, V and Q by tensor maps: the blocks' table, then a box of positions of one block at a time
//   warps 8-11       copies 16 bytes at a time where boxes do not fit (blocks that are no multiple of 8 positions), and 8 bits to halves
//   warp 15          8 bits: the scales
//   warp 13          which units come next
//   warp 12          the products, in the order  S_A(0) S_B(0) | PV_A(j) S_A(j+1) PV_B(j) S_B(j+1) | ...
//                    so that one tile's powers run beside the other's products
//
// In order of issue is in order of execution: S_A(j+1)'s arrival says that PV_A(j) has read P and written O.
//
// The products bound it: 64 cycles for each of a pair's 32 (heads of 128), 2,048 a turn of 128 positions, of about 2,950 that a turn takes.
// One prompt of 16,384 tokens (32 / 8 heads of 128) takes 1.34 ms, 1.65 PFLOP/s, of 8,192 0.38 ms; heads of 64 335 us for 8,192 (the tensor
// cores at work 36 % of the time: the powers' warps set the turn), over 8 bits 814 us (37 %: the conversions of one warp group bound it), over blocks
// that no box fits 582 us.  What the products' warp does between two of them counts most: weights
// handed over in halves, to begin sooner, cost 80 us of 1,420, a lane elected anew each turn 68, a second warp for tile B 280.  The roles that copy
// count next: a flag read after each wait there cost 3 %, an atomic report of bad blocks in place of a store 2 to 4 %.
//
// Weights are rounded once to the products' type, by 2^-9 relative in bfloat16 and 2^-12 in halves; sums of weights are not.  Outputs of a prompt
// of 2,000 are off by 2.0e-3 of their root mean square for it (bfloat16; their own rounding alone is 1.6e-3), 2.6e-4 in halves (2.0e-4).  The remainders' product, which
// attend_kernel has in bfloat16, would be half as many products again here, where these bound the work.
//
// Work is laid on a line and cut into equal stretches as in wf_attend.cu; a unit is the 256 queries, its weight grows with
// the positions that they see.  Every wait ends: after a limit it is reported (wf_attn_status) and the role that waited leaves, as the others of the
// CTA do at their next wait that finds nothing.  No unit is overwritten then, and no barrier without limit stands between roles; copies and products under
// way are awaited before the CTA ends, and wf_attn_status clears the arrivals that a join may be left with.
#include <algorithm>
#include <type_traits>

#include <cuda.h>

#include "wf_attend.cuh"
#include "wf_decode.cuh"

namespace {

constexpr int kThreads = 512;
constexpr int kQ = 128, kPair = 2 * kQ;   // queries of a tile, of a unit
constexpr int kLoaders = 128;
constexpr int kRaws = 3;                  // at most
constexpr int kFours = kKeys / 4, kSlots = 4;  // scales of a tile; tiles whose scales are held
constexpr float kSlack = 8.f;             // log2 of what a maximum may grow by before O is shrunk
constexpr float kLift = 15.f - kSlack;    // log2 of a half weight at the reference: half floats reach to 2^16, and what is 2^-32 of the reference still counts
constexpr float kLeastScale = 0x1p-64f;

template <bool E, int D> struct Shape {
    static constexpr int kRow = 2 * D;                       // bytes of a key or query in shared memory
    static constexpr int kHalf = kQ * 128;                   // bytes of 64 elements of the queries
    static constexpr int kEight = 8 * kRow;                  // bytes of eight keys: 64 elements of all, then the other 64
    static constexpr int kTile = kKeys * kRow;
    static constexpr int kStages = D == 64 ? 8 : 4;
    static constexpr int kRaw = D == 64 ? 3 : 2;             // tiles in 8 bits under way
    static constexpr int kScales = E ? kSlots * 3 * kFours * 4 : 0;  // keys' scales, log2 and reciprocal of values', for each four positions
    static constexpr int kQBytes = 2 * kTile;
    static constexpr int kRawBytes = E ? kRaw * kKeys * D : 0;
    static constexpr int kSmem = kQBytes + kRawBytes + kStages * kTile + kScales;
    static_assert(kSmem + 1024 <= 227 * 1024, "shared memory");  // with what is static, up to the next 1,024 bytes
};

struct PromptArgs {
    AttendArgs a;
    int32_t box;     // positions of a box of the maps k and v, 0: they are not used
    int32_t map_q;   // whether q is
    int32_t heads;   // the maps' last coordinate: block * heads + head
    int32_t beyond;  // the first that is not there
    int32_t polls, hint;  // of a wait before it gives up, nanoseconds of one
    CUtensorMap k, v, q;
};

constexpr int kUnits = 4;  // that the roles may be apart

enum { kBarQFull, kBarQEmpty, kBarS, kBarP = kBarS + 2, kBarO = kBarP + 2, kBarDrain = kBarO + 2, kBarFull, kBarUnit = kBarFull + 16, kBarRaw = kBarUnit + 2 * kUnits,
       kBarScale = kBarRaw + 2 * kRaws, kBarJoin = kBarScale + 2 * kSlots, kBarLast, kBars };

__device__ __forceinline__ uint32_t smem_of(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

// One arrival for the warp, once every lane has come.
__device__ __forceinline__ void warp_arrive(uint32_t bar)
{
    __syncwarp();
    if (threadIdx.x % 32 == 0) bar_arrive(bar);
}

// Whether the barrier's phase is over; the hardware may wait about `hint` nanoseconds for it.
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity, uint32_t hint = 1000)
{
    uint32_t done;
    asm volatile("{ .reg .pred p;\n"
                 "  mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
                 "  selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity), "r"(hint) : "memory");
    return done;
}

// Waits for so many polls more than one; false: that ran out, here or in another thread.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, int polls, uint32_t hint, volatile int *gave_up, int *err)
{
    if (bar_try(bar, parity, hint)) return true;
    for (int i = 0; i < polls && !*gave_up; i++)
        if (bar_try(bar, parity, hint)) return true;
    if (!*gave_up) {
        *gave_up = 1;
        err[1] = 1;
    }
    return false;
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
// A box of a tensor map from these coordinates; its bytes arrive at bar.
__device__ __forceinline__ void copy_box5(uint32_t to, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2, int c3, int c4)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(to),
                 "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}
__device__ __forceinline__ void copy_box3(uint32_t to, const CUtensorMap *map, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(to), "l"(map),
                 "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit_to(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// One lane of a whole warp: what it issues has operands that are the same in every lane, as the products' instructions want them.
__device__ __forceinline__ bool elected()
{
    uint32_t one;
    asm volatile("{ .reg .pred p;\n"
                 "  elect.sync _|p, 0xFFFFFFFF;\n"
                 "  selp.u32 %0, 1, 0, p; }" : "=r"(one)::"memory");
    return one;
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

// Rows of 128 bytes, swizzled, eight of them 1,024 bytes: `next` the bytes to the next eight rows, `lead` to the next 64 elements where these
// run along rows.
__device__ __forceinline__ uint64_t matrix(uint32_t at, uint32_t lead, uint32_t next)
{
    return (uint64_t)(at >> 4 & 0x3FFF) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(next >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ float power(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Two at once.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("{ .reg .b64 a, b, c, d;\n"
        "  mov.b64 a, {%2, %3};\n  mov.b64 b, {%4, %5};\n  mov.b64 c, {%6, %7};\n"
        "  fma.rn.f32x2 d, a, b, c;\n"
        "  mov.b64 {%0, %1}, d; }" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("{ .reg .b64 a, b, d;\n"
        "  mov.b64 a, {%2, %3};\n  mov.b64 b, {%4, %5};\n"
        "  add.rn.f32x2 d, a, b;\n"
        "  mov.b64 {%0, %1}, d; }" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// ---------------------------------------------------------------------------
// The line of work
// ---------------------------------------------------------------------------

// A CTA's part of a unit; no tiles: the end.
struct Unit {
    Row row;
    int32_t r, head;        // row of the tables, key head
    int64_t q0;             // the first query: token * group + head of the group
    int32_t queries;        // up to 2 tile_q
    int32_t t0, n;          // first tile of positions, tiles
    int32_t na, nb;         // of them those that A, B see
    int32_t seen;           // positions that the last query sees
    int32_t first, parts;   // the unit's CTAs
};

// Walks the CTA's stretch: from its first place (found by division and a root) unit by unit.
struct Walk {
    Span span;
    int64_t at, stop;
    int64_t begin;      // of the unit
    int64_t i;          // the unit of its key head
    int32_t r, head;
    Row row;
    Line line;

    __device__ __forceinline__ Walk(const AttendArgs &a, const Found &f) : span(f.span), r(f.r)
    {
        at = span.begin(blockIdx.x), stop = span.begin(blockIdx.x + 1);
        row = f.row, line = line_of(a, row);
        const int64_t each = line.head();
        head = (int32_t)quotient(at - f.row_begin, each);
        const int64_t base = f.row_begin + head * each, x = at - base;
        // The unit that holds place x: i W + t i (i + 1) <= x.
        const double t = (double)line.tile_q, b = (double)line.w + t;
        i = max((int64_t)0, min(line.units - 1, (int64_t)((sqrt(b * b + 4.0 * t * (double)x) - b) / (2.0 * t))));
        while (i > 0 && line.upto(i) > x) i--;
        while (i + 1 < line.units && line.upto(i + 1) <= x) i++;
        begin = base + line.upto(i);
    }

    __device__ __forceinline__ bool next(const AttendArgs &a, Unit &u)
    {
        while (at < stop) {
            while (i >= line.units) {  // the next key head, or the next row that has units
                i = 0;
                if (++head < a.kv && line.units) break;
                head = 0;
                row = row_of(a, ++r), line = line_of(a, row);
            }
            const int64_t end = begin + line.w + 2 * line.tile_q * (i + 1);
            const int32_t have = row.len - row.n;
            u.row = row, u.r = r, u.head = head;
            u.q0 = i * 2 * a.tile_q;
            u.queries = (int32_t)min((int64_t)2 * a.tile_q, (int64_t)row.n * a.group - u.q0);
            auto sees = [&](int64_t q) { return have + (int32_t)wf_quot((uint32_t)q, a.by_group) + 1; };
            u.seen = sees(u.q0 + u.queries - 1);
            const int32_t tiles_a = (sees(u.q0 + min(u.queries, a.tile_q) - 1) + kKeys - 1) / kKeys, tiles = (u.seen + kKeys - 1) / kKeys;
            const int64_t each = (int64_t)kKeys * a.group;
            auto tile = [&](int64_t p) {
                return p >= end ? tiles : p <= begin ? 0 : (int32_t)max((int64_t)0, min((int64_t)tiles, quotient(p - begin, each) - kFixed));
            };
            const int32_t t0 = tile(at), t1 = tile(stop);
            const bool split = at > begin || stop < end;
            const int64_t unit_begin = begin;
            at = min(stop, end);
            if (at == end) begin = end, i++;
            if (t1 <= t0) continue;
            u.t0 = t0, u.n = t1 - t0;
            u.na = max(0, min(t1, tiles_a) - t0), u.nb = u.queries > a.tile_q ? u.n : 0;
            u.first = blockIdx.x, u.parts = 1;
            if (split) {
                int32_t first = span.owner(unit_begin), last = span.owner(end - 1);
                auto part = [&](int64_t p) {
                    return p >= end ? tiles : p <= unit_begin ? 0 : (int32_t)max((int64_t)0, min((int64_t)tiles, quotient(p - unit_begin, each) - kFixed));
                };
                while (part(span.begin(first + 1)) <= 0) first++;
                while (part(span.begin(last)) >= tiles) last--;
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
    uint8_t *q, *kv, *raw; // on 1,024 bytes; raw: tiles in 8 bits as the cache has them
    float *scales;
    uint32_t bars;         // address
    int polls, hint, box;  // as in PromptArgs
    volatile int *gave_up;
    int *unfit;            // the last unit, from 1 on, out of whose products values that are no finite numbers were taken
    int *err;
    __device__ __forceinline__ uint32_t bar(int i) const { return bars + 8 * i; }
    // False: waiting was given up.  wait: every lane of the warp comes, and the answer is one for all.
    __device__ __forceinline__ bool wait_alone(int i, uint32_t parity) const { return bar_wait(bar(i), parity, polls, hint, gave_up, err); }
    __device__ __forceinline__ bool wait(int i, uint32_t parity) const { return __all_sync(~0u, wait_alone(i, parity)); }
    // Unit i of the CTA; null: there are no more, or waiting was given up.  It stays as it is until every role is done with it.
    __device__ __forceinline__ const Unit *unit(uint32_t i) const
    {
        if (!wait(kBarUnit + i % kUnits, i / kUnits & 1)) return nullptr;
        const Unit *u = units + i % kUnits;
        return u->n ? u : nullptr;
    }
    __device__ __forceinline__ void unit_done(uint32_t i) const { warp_arrive(bar(kBarUnit + kUnits + i % kUnits)); }
};

// One thread: the units, as room comes free.
__device__ __forceinline__ void unit_role(const AttendArgs &a, const Found &f, const Shared &sh)
{
    Walk walk(a, f);
    Unit u;
    for (uint32_t i = 0;; i++) {
        const bool more = walk.next(a, u);
        if (!sh.wait_alone(kBarUnit + kUnits + i % kUnits, (i / kUnits & 1) ^ 1)) return;
        if (!more) u.n = 0;
        sh.units[i % kUnits] = u;
        bar_arrive(sh.bar(kBarUnit + i % kUnits));
        if (!more) return;
    }
}

// Bytes of 16-byte chunk c of query i in its tile, of key i.
__device__ __forceinline__ uint32_t query_place(int i, int c) { return c / 8 * (kQ * 128) + i * 128 + ((c ^ i) & 7) * 16; }
template <int D> __device__ __forceinline__ uint32_t place(int i, int c) { return i / 8 * (16 * D) + c / 8 * 1024 + i % 8 * 128 + ((c ^ i) & 7) * 16; }

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

// A tile by boxes of `box` positions of one block, once there is room: one copy a lane, whose block (in the maps' last coordinate) and place in it are
// given.  False: waiting was given up.
template <bool E, int D>
__device__ __forceinline__ bool copy_boxes(const PromptArgs &pa, const Shared &sh, int room, uint32_t parity, const CUtensorMap *map, uint32_t to, int bar,
                                           int32_t block, int32_t place, int lane)
{
    constexpr int kRow = E ? D : 2 * D;
    const int box = pa.box;
    const bool there = sh.wait_alone(room, parity);
    if (there && lane == 0) bar_expect(sh.bar(bar), kKeys * kRow);
    if (!__all_sync(~0u, there)) return false;
    if (lane * box < kKeys) {
        if constexpr (E) copy_box3(to + lane * box * kRow, map, sh.bar(bar), 0, place, block);
        else copy_box5(to + lane * box * kRow, map, sh.bar(bar), 0, 0, 0, place / 8, block);
    }
    return true;
}

// Warp 14: copies by the tensor maps, where the layout allows them.
template <typename T, bool E, int D> __device__ __forceinline__ void box_role(const PromptArgs &pa, const Shared &sh)
{
    using S = Shape<E, D>;
    const AttendArgs &a = pa.a;
    const int lane = threadIdx.x % 32;
    const uint32_t kv = smem_of(sh.kv), raw = smem_of(sh.raw);
    uint32_t it = 0, units = 0, queries = 0;  // tiles, units, units' queries whose copies have begun
    auto unit = [&](const Unit &u) {
        if (pa.map_q) {
            if (!sh.wait(kBarQEmpty, (units & 1) ^ 1)) return false;
            const int tiles = u.nb ? 2 : 1;
            if (lane == 0) bar_expect(sh.bar(kBarQFull), tiles * (D / 64) * a.tile_q * 128);
            __syncwarp();
            if (lane < tiles * (D / 64)) {
                const int x = lane / (D / 64), g = lane % (D / 64);
                copy_box3(smem_of(sh.q) + x * S::kTile + g * S::kHalf, &pa.q, sh.bar(kBarQFull), g * 64, u.head * a.group,
                          u.row.first + (int32_t)wf_quot((uint32_t)u.q0 + x * a.tile_q, a.by_group));
            }
            queries++;
        }
        if (!pa.box) return true;
        const int32_t end = min(u.seen, (u.t0 + u.n) * kKeys);
        const int32_t *table = a.table + u.r * a.table_stride;
        // This lane's box of tile j: its block in the table, and in the maps.  Boxes behind `end` come from a block that is not there: zeros.
        auto position = [&](int32_t j) { return (u.t0 + j) * kKeys + min(lane * pa.box, kKeys - 1); };
        auto block = [&](int32_t j) { return block_at(a, table, wf_quot(min(position(j), end - 1), a.by_bs)); };
        int32_t next = block(0);
        for (int32_t j = 0; j < u.n; j++) {
            const int32_t p = (u.t0 + j) * kKeys, at = position(j);
            const int32_t b = at < end ? next * pa.heads + u.head : pa.beyond, place_in = at < end ? at - (int32_t)wf_quot(at, a.by_bs) * a.bs : 0;
            if (j + 1 < u.n) next = block(j + 1);
            // A box that the row ends in holds what lies behind the row, and a weight of 0 does not undo a NaN there.
            const bool ends = !E && u.row.len % pa.box && p + kKeys > u.row.len;
#pragma unroll 1
            for (int side = 0; side < 2; side++, it++) {
                const CUtensorMap *map = side ? &pa.v : &pa.k;
                if constexpr (E) {
                    const uint32_t s = it % S::kRaw;
                    if (!copy_boxes<E, D>(pa, sh, kBarRaw + kRaws + s, (it / S::kRaw & 1) ^ 1, map, raw + s * (kKeys * D), kBarRaw + s, b, place_in, lane))
                        return false;
                } else {
                    const uint32_t s = it % S::kStages, to = kv + s * S::kTile, empty = (it / S::kStages & 1) ^ 1;
                    if (!ends || !side) {
                        if (!copy_boxes<E, D>(pa, sh, kBarFull + 8 + s, empty, map, to, kBarFull + s, b, place_in, lane)) return false;
                    } else {
                        if (!sh.wait(kBarFull + 8 + s, empty)) return false;
                        constexpr int kPer = D / 8;
                        const uint8_t *v = a.v + u.head * a.head_stride;
#pragma unroll 1
                        for (int i = lane / kPer; i < kKeys; i += 32 / kPer) {
                            const int32_t key = min(p + i, end - 1);
                            const uint32_t in = wf_quot(key, a.by_bs);
                            const uint8_t *from = v + block_at(a, table, in) * a.block_stride + (key - (int32_t)in * a.bs) * a.token_stride;
                            copy16(to + place<D>(i, lane % kPer), from + lane % kPer * 16, p + i < end);
                        }
                        copies_commit();
                        copies_wait<0>();
                        to_async();
                        __syncwarp();
                        if (lane == 0) bar_arrive(sh.bar(kBarFull + s));
                    }
                }
            }
        }
        return true;
    };
    for (; const Unit *u = sh.unit(units); units++) {
        if (!unit(*u)) break;
        sh.unit_done(units);
    }
    // No copy is on its way into this CTA's shared memory when it ends, whatever the other roles have come to.
    if (lane == 0) {
        const int n = E ? S::kRaw : S::kStages, first = E ? kBarRaw : kBarFull;
        for (uint32_t i = it > (uint32_t)n ? it - n : 0; pa.box && i < it; i++)
            for (int k = 0; k < 1 << 16 && !bar_try(sh.bar(first + i % n), i / n & 1); k++) {}
        for (int k = 0; queries && k < 1 << 16 && !bar_try(sh.bar(kBarQFull), (queries - 1) & 1); k++) {}
    }
    __syncwarp();
}

// Positions that query q of the unit sees.
__device__ __forceinline__ int32_t seen_by(const AttendArgs &a, const Unit &u, int q)
{
    return u.row.len - u.row.n + (int32_t)wf_quot((uint32_t)(u.q0 + q), a.by_group) + 1;
}

// Warp 15, 8 bits: the scales of each four positions, which lie in one block.
__device__ __forceinline__ void scale_role(const AttendArgs &a, const Shared &sh)
{
    const int lane = threadIdx.x % 32;
    uint32_t t = 0;
    for (uint32_t units = 0; const Unit *now = sh.unit(units); units++) {
        const Unit &u = *now;
        const int32_t *table = a.table + u.r * a.table_stride;
        const int32_t end = min(u.seen, (u.t0 + u.n) * kKeys), n = u.n, p0 = u.t0 * kKeys + 4 * lane;
        const float *ks = a.k_scale + u.head, *vs = a.v_scale + u.head;
        // Blocks two tiles ahead, scales one.
        auto block = [&](int32_t j) { return (int64_t)block_at(a, table, wf_quot(min(p0 + j * kKeys, end - 1), a.by_bs)) * a.kv; };
        int64_t b = block(0);
        float k = ks[b], v = vs[b];
        b = block(min(1, n - 1));
        for (int32_t j = 0; j < n; j++, t++) {
            const float now_k = k, now_v = fmaxf(v, kLeastScale);
            if (j + 1 < n) k = ks[b], v = vs[b];
            if (j + 2 < n) b = block(j + 2);
            const uint32_t s = t % kSlots;
            if (!sh.wait(kBarScale + kSlots + s, (t / kSlots & 1) ^ 1)) return;
            float *to = sh.scales + s * 3 * kFours + lane;
            to[0] = now_k, to[kFours] = __log2f(now_v), to[2 * kFours] = __frcp_rn(now_v);
            warp_arrive(sh.bar(kBarScale + s));
        }
        sh.unit_done(units);
    }
}

// Warps 8 - 11: what tensor maps cannot copy: any blocks and alignment, queries of any group, and 8 bits to halves.
template <typename T, bool E, int D> __device__ __forceinline__ void load_role(const PromptArgs &pa, const Shared &sh)
{
    using S = Shape<E, D>;
    const AttendArgs &a = pa.a;
    const int tid = threadIdx.x - 256, lane = tid % 32;
    // Of a tile in 16 bits a warp copies kAt keys at once, kRows further on each time: 32 in all, of which each lane looks up one.
    constexpr int kChunks = D / 8, kAt = 32 / kChunks, kRows = kLoaders / kChunks;  // 16-byte chunks of a key or query; queries at once
    const int mine = lane / kAt * kRows + tid / 32 * kAt + lane % kAt;
    const uint32_t kv = smem_of(sh.kv), q = smem_of(sh.q);
    uint32_t it = 0, units = 0;
    bool on = true;
    int32_t waiting = 0;   // tiles whose copies are under way and not yet announced (16 bits)
    auto announce = [&](uint32_t i) {
        to_async();
        warp_arrive(sh.bar(kBarFull + i % S::kStages));
    };
    for (; on; units++) {
        const Unit *now = sh.unit(units);
        if (!now) break;
        const Unit &u = *now;
        const int32_t *table = a.table + u.r * a.table_stride;
        const uint8_t *k = a.k + u.head * a.head_stride, *v = a.v + u.head * a.head_stride;
        const int32_t end = min(u.seen, (u.t0 + u.n) * kKeys);  // positions that count
        // The block of this lane's key of tile j.
        auto block = [&](int32_t j) {
            const int32_t p = min((u.t0 + j) * kKeys + mine, end - 1);
            return block_at(a, table, wf_quot(p, a.by_bs));
        };
        const bool tiles = E || !pa.box;
        int32_t next = !E && tiles ? block(0) : 0;
        // What is under way belongs to the unit before, which must have it to come to its end.
        copies_wait<0>();
        for (; waiting; waiting--) announce(it - waiting);
        if (!pa.map_q) {  // queries, once the products of the unit before have read theirs
            on = sh.wait(kBarQEmpty, (units & 1) ^ 1);
            if (!on) break;
            const int c = tid % kChunks;
#pragma unroll 1
            for (int x = 0; x < (u.nb ? 2 : 1); x++) {
                const int queries = min(a.tile_q, u.queries - x * a.tile_q);
                if (!E || std::is_same_v<T, __half>) {
#pragma unroll 4
                    for (int i = tid / kChunks; i < kQ; i += kRows) {
                        const bool there = i < queries;
                        copy16(q + x * S::kTile + query_place(i, c), query(a, u, x * a.tile_q + (there ? i : 0)) + 16 * c, there);
                    }
                } else {
#pragma unroll 4
                    for (int i = tid / kChunks; i < kQ; i += kRows) {
                        const bool there = i < queries;
                        uint4 y = there ? *reinterpret_cast<const uint4 *>(query(a, u, x * a.tile_q + i) + 16 * c) : make_uint4(0, 0, 0, 0);
                        float most = largest<T>(y);
#pragma unroll
                        for (int s = 1; s < kChunks; s *= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, s));
                        const float down = __int_as_float((127 - query_exponent(most)) << 23);
                        uint32_t *w = &y.x;
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const float2 z = wf_pair<T>::to_float(w[j]);
                            w[j] = wf_pair<__half>::of_float(z.x * down, z.y * down);
                        }
                        *reinterpret_cast<uint4 *>(sh.q + x * S::kTile + query_place(i, c)) = y;
                    }
                }
            }
            copies_commit();
            copies_wait<0>();
            to_async();
            warp_arrive(sh.bar(kBarQFull));
        }
        for (int32_t j = 0; tiles && on && j < u.n; j++) {
            const int32_t p = (u.t0 + j) * kKeys, key = p + mine;
            // This lane's key in the cache, -1: none.
            const int64_t offset = !E && key < end ? next * a.block_stride + (int64_t)(key - (int32_t)wf_quot(key, a.by_bs) * a.bs) * a.token_stride : -1;
            if (!E && j + 1 < u.n) next = block(j + 1);
#pragma unroll 1
            for (int side = 0; on && side < 2; side++, it++) {  // keys, values
                const uint32_t s = it % S::kStages, to = kv + s * S::kTile;
                const uint8_t *from = side ? v : k;
                const uint32_t freed = ((it / S::kStages) & 1) ^ 1;
                // While there is no room, what has landed is announced at once: the warp's decision, as announcements are (its lanes' polls may differ).
                while (waiting && !__all_sync(~0u, bar_try(sh.bar(kBarFull + 8 + s), freed))) {
                    if (waiting == 2) copies_wait<1>();
                    else copies_wait<0>();
                    announce(it - waiting);
                    waiting--;
                }
                if constexpr (!E) {
                    on = sh.wait(kBarFull + 8 + s, freed);
                    if (!on) break;
                    const int c = tid % kChunks;
#pragma unroll 8
                    for (int i = 0; i < kKeys / kRows; i++) {
                        const int64_t o = __shfl_sync(~0u, offset, i * kAt + lane / kChunks);
                        copy16(to + place<D>(i * kRows + tid / kChunks, c), from + (o < 0 ? 0 : o) + 16 * c, o >= 0);
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
                    constexpr int kPer = D / 16, kStep = kLoaders / kPer, kTimes = kKeys / kStep;
                    const int c = tid % kPer;
                    const uint32_t rs = it % S::kRaw;
                    uint4 x[kTimes];
                    on = sh.wait(kBarRaw + rs, it / S::kRaw & 1);
                    if (!on) break;
#pragma unroll
                    for (int i = 0; i < kTimes; i++) {
                        const int row = i * kStep + tid / kPer;
                        x[i] = *reinterpret_cast<const uint4 *>(sh.raw + rs * (kKeys * D) + row * D + 16 * c);
                        if (p + row >= end) x[i] = make_uint4(0, 0, 0, 0);
                    }
                    warp_arrive(sh.bar(kBarRaw + kRaws + rs));
                    on = sh.wait(kBarFull + 8 + s, freed);
                    if (!on) break;
#pragma unroll
                    for (int i = 0; i < kTimes; i++) {
                        const int row = i * kStep + tid / kPer;
                        const uint2 h0 = wf_e4m3_halves(x[i].x), h1 = wf_e4m3_halves(x[i].y), h2 = wf_e4m3_halves(x[i].z), h3 = wf_e4m3_halves(x[i].w);
                        uint8_t *dst = sh.kv + s * S::kTile;
                        *reinterpret_cast<uint4 *>(dst + place<D>(row, 2 * c)) = make_uint4(h0.x, h0.y, h1.x, h1.y);
                        *reinterpret_cast<uint4 *>(dst + place<D>(row, 2 * c + 1)) = make_uint4(h2.x, h2.y, h3.x, h3.y);
                    }
                    announce(it);
                }
            }
        }
        if (on) sh.unit_done(units);
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
    const bool leader = elected();  // once: elected anew for each turn, one prompt of 16,384 took 1,370 us in place of 1,302
    // A lane whose wait was given up goes on at the unit's end, so that the warp leaves as one; the leader issues nothing more of the unit then.
    bool on = true;
    auto full = [&](uint32_t i) { return sh.wait_alone(kBarFull + i % S::kStages, (i / S::kStages) & 1); };
    auto commit = [&](int i) {
        if (leader) commit_to(sh.bar(i));
    };
    auto done = [&](uint32_t i) { commit(kBarFull + 8 + i % S::kStages); };
    auto scores = [&](int x, uint32_t i) {
        const uint64_t key = matrix(kv + i % S::kStages * S::kTile, 16, S::kEight), query = matrix(q + x * S::kTile, 16, 1024);
        if (leader) {
#pragma unroll
            for (int s = 0; s < D / 16; s++) {
                mma_ss(tmem + x * kKeys, query + ((s / 4 * S::kHalf + s % 4 * 32) >> 4), key + ((s / 4 * 1024 + s % 4 * 32) >> 4), kDescS, s > 0);
            }
            commit_to(sh.bar(kBarS + x));
        }
    };
    auto sums = [&](int x, uint32_t i, bool more) {
        const uint64_t value = matrix(kv + i % S::kStages * S::kTile, 1024, S::kEight);
        if (leader) {
#pragma unroll
            for (int s = 0; s < kKeys / 16; s++)
                mma_ts(tmem + 2 * kKeys + x * D, tmem + x * kKeys + 8 * s, value + s * (2 * S::kEight >> 4), kDescO, more || s > 0);
        }
    };
    for (; __all_sync(~0u, on); units++) {
        const Unit *u = sh.unit(units);
        if (!u) break;
        const int n[2] = {u->na, u->nb}, most = u->n;
        sh.unit_done(units);
        on = false;
        if (!sh.wait_alone(kBarQFull, units & 1) || !full(it)) continue;
        after_sync();
#pragma unroll
        for (int x = 0; x < 2; x++)
            if (n[x] > 0) scores(x, it);
        done(it);
        if (most == 1) commit(kBarQEmpty);
        for (int j = 0; j < most; j++) {
            if (!full(it + 2 * j + 1)) goto next;
            if (j + 1 < most && !full(it + 2 * j + 2)) goto next;
#pragma unroll
            for (int x = 0; x < 2; x++) {
                if (j < n[x]) {
                    if (!sh.wait_alone(kBarP + x, np[x] & 1)) goto next;
                    np[x]++;
                    after_sync();
                    sums(x, it + 2 * j + 1, j > 0);
                }
                if (x == 1) done(it + 2 * j + 1);
                if (j + 1 < n[x]) {
                    scores(x, it + 2 * j + 2);
                } else if (j < n[x]) {
                    commit(kBarO + x);
                }
            }
            if (j + 1 < most) done(it + 2 * j + 2);
            if (j + 2 == most) commit(kBarQEmpty);
        }
        it += 2 * most, on = true;
    next:;
    }
    // Nothing is under way when TMEM is given back.
    commit(kBarDrain);
    for (int i = 0; i < 1 << 20 && !bar_try(sh.bar(kBarDrain), 0); i++) {}
}

// Parts in scratch: D / 4 columns of [256 queries] four sums, then [256] references, [256] sums of weights.
template <int D> constexpr int kPart = kPair * (D + 2);

// Elements i .. i + 31 of the warp's queries, one a lane, times `by`.  Four lanes swap their 16-byte pieces (piece c of each query to lane c),
// so that a store fills 64 bytes of 8 queries in place of 16 bytes of 32: with those the end of a unit took 4,500 cycles.
template <typename T> __device__ __forceinline__ void put(uint8_t *const (&out)[4], int i, const float *y, float by)
{
    const int c = threadIdx.x % 4;
    uint32_t w[4][4];
#pragma unroll
    for (int k = 0; k < 16; k++) w[k / 4][k % 4] = wf_pair<T>::of_float(y[2 * k] * by, y[2 * k + 1] * by);
    // Two rounds: lanes 1 apart swap pieces whose numbers differ in bit 0, then lanes 2 apart those that differ in bit 1.
#pragma unroll
    for (int bit = 1; bit < 4; bit *= 2)
#pragma unroll
        for (int k = 0; k < 4; k++)
            if (!(k & bit)) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const bool up = c & bit;
                    const uint32_t got = __shfl_xor_sync(~0u, up ? w[k][j] : w[k | bit][j], bit);
                    if (up) w[k][j] = got;
                    else w[k | bit][j] = got;
                }
            }
#pragma unroll
    for (int k = 0; k < 4; k++)  // piece c of query k of the four
        if (out[k]) *reinterpret_cast<uint4 *>(out[k] + 2 * i + 16 * c) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
}

// Values of a tile (halves where the cache has 8 bits) from key `from` on, up to `to`, which some queries of the 128 do not see: what is no finite number becomes 0,
// and give_unfit's.  A thread looks through a key.  False: waiting was given up.  (Sixteen prompts of 512: 91 -> 97 us; after the powers, where more
// registers are spilled for it, one of 16,384 took 1,389 us for 1,333.)
template <typename T, bool E, int D> __device__ __forceinline__ bool take_unfit(const Shared &sh, uint32_t it, int32_t from, int32_t to, uint32_t unit)
{
    using S = Shape<E, D>;
    if (!sh.wait(kBarFull + it % S::kStages, it / S::kStages & 1)) return false;
    const int key = threadIdx.x % kQ;
    if (key < from || key >= to) return true;
    uint8_t *tile = sh.kv + it % S::kStages * S::kTile;
    auto at = [&](int c) { return reinterpret_cast<uint4 *>(tile + place<D>(key, c)); };
    uint32_t most[4] = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < D / 8; c++) {
        const uint4 y = *at(c);
        most[0] = wf_larger<T>(most[0], y.x), most[1] = wf_larger<T>(most[1], y.y), most[2] = wf_larger<T>(most[2], y.z), most[3] = wf_larger<T>(most[3], y.w);
    }
    if (wf_unfit<T>(make_uint4(most[0], most[1], most[2], most[3]))) {
        atomicMax(sh.unfit, (int)unit + 1);
        __threadfence_block();
#pragma unroll 1
        for (int c = 0; c < D / 8; c++) *at(c) = wf_fit<T>(*at(c));
        to_async();
    }
    return true;
}

// What take_unfit took, to a query's output or, where that is null, its sums.
template <typename T, bool E, int D> __device__ __noinline__ void give_unfit(const AttendArgs &a, const Unit &u, int32_t seen, uint8_t *out, float *sums)
{
    using V = std::conditional_t<E, __nv_fp8_e4m3, T>;
    const int32_t begin = max(seen_by(a, u, 0), u.t0 * kKeys), end = min(seen, (u.t0 + u.n) * kKeys);
#pragma unroll 1
    for (int i = 0; i < D; i += 4) {
        uint32_t *w = reinterpret_cast<uint32_t *>(out + 2 * i);
        float4 *s = reinterpret_cast<float4 *>(sums) + i / 4 * kPair;
        const float2 lo = out ? wf_pair<T>::to_float(w[0]) : make_float2(0.f, 0.f), hi = out ? wf_pair<T>::to_float(w[1]) : make_float2(0.f, 0.f);
        const float4 z = out ? make_float4(lo.x, lo.y, hi.x, hi.y) : __ldcg(s);
        float y[4] = {z.x, z.y, z.z, z.w};
        add_unfit<V>(a, a.table + u.r * a.table_stride, a.v + u.head * a.head_stride + i * (int)sizeof(V), begin, end, y);
        if (out) w[0] = wf_pair<T>::of_float(y[0], y[1]), w[1] = wf_pair<T>::of_float(y[2], y[3]);
        else __stcg(s, make_float4(y[0], y[1], y[2], y[3]));
    }
}

template <typename T, bool E, int D>
__device__ __forceinline__ void power_role(const AttendArgs &a, const Shared &sh, uint32_t tmem, int *last_one)
{
    using S = Shape<E, D>;
    using M = std::conditional_t<E, __half, T>;
    const int x = threadIdx.x / kQ, q = threadIdx.x % kQ, qq = x * a.tile_q + q;  // tile, query of the tile, of the unit
    const uint32_t lane = tmem + ((uint32_t)(q / 32 * 32) << 16), st = lane + x * kKeys, ot = lane + 2 * kKeys + x * D;
    uint32_t ns = 0, no = 0, ts = 0, joins = 0, units = 0;  // ts: tiles of the CTA, whichever are seen
    for (; const Unit *now = sh.unit(units); units++) {
        const Unit &u = *now;
        const int n = x ? u.nb : u.na;
        const bool there = q < a.tile_q && qq < u.queries;
        const uint32_t flat = (uint32_t)(u.q0 + (there ? qq : 0)), tok = wf_quot(flat, a.by_group);
        const int32_t seen = u.row.len - u.row.n + (int32_t)tok + 1;
        const int32_t least = seen_by(a, u, x * a.tile_q);  // what every query of the 128 sees (no more than that if there are none)
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
            const int32_t p = (u.t0 + j) * kKeys;
            // Tile A's threads do it for both where A sees the positions: B's product comes after A's.
            if (p + kKeys > least && (x == 0 || j >= u.na) && !take_unfit<M, E, D>(sh, 2 * ts + 1, least - p, u.seen - p + sh.box, units)) return;
            float s[kKeys];
            uint32_t *w = reinterpret_cast<uint32_t *>(s);
            if (!sh.wait(kBarS + x, ns & 1)) return;
            ns++;
            after_sync();
#pragma unroll
            for (int i = 0; i < 4; i++) tm_load(w + 32 * i, st + 32 * i);
            const float *sc = nullptr;
            bool on = true;
            if constexpr (E) {
                on = sh.wait(kBarScale + ts % kSlots, ts / kSlots & 1);
                sc = sh.scales + ts % kSlots * 3 * kFours;
            }
            tm_loaded();
            if (!on) return;
            if constexpr (E) {
#pragma unroll
                for (int i = 0; i < kFours; i += 4) {
                    const float4 ks = *reinterpret_cast<const float4 *>(sc + i), lg = *reinterpret_cast<const float4 *>(sc + kFours + i);
                    const float by[4] = {scale * ks.x, scale * ks.y, scale * ks.z, scale * ks.w}, plus[4] = {lg.x, lg.y, lg.z, lg.w};
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        const float2 y = fma2(make_float2(s[4 * i + k], s[4 * i + k + 1]), make_float2(by[k / 4], by[k / 4]), make_float2(plus[k / 4], plus[k / 4]));
                        s[4 * i + k] = y.x, s[4 * i + k + 1] = y.y;
                    }
                }
            }
            auto largest_of = [&] {
                float most[4] = {fmaxf(s[0], s[1]), fmaxf(s[2], s[3]), fmaxf(s[4], s[5]), fmaxf(s[6], s[7])};
#pragma unroll
                for (int i = 8; i < kKeys; i += 8)
#pragma unroll
                    for (int k = 0; k < 4; k++) most[k] = fmaxf(fmaxf(most[k], s[i + 2 * k]), s[i + 2 * k + 1]);
                const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
                return E ? top : top * scale;
            };
            float2 sums[2];
            const float2 by = make_float2(scale, scale);
            auto powers = [&](int half) {  // of 64 scores, packed in place
                const float base = ref == -INFINITY ? 0.f : std::is_same_v<M, __half> ? ref - kLift : ref;
                const float2 off = make_float2(-base, -base);
#pragma unroll
                for (int i = half * kKeys / 2; i < (half + 1) * kKeys / 2; i += 2) {
                    float2 y = make_float2(s[i], s[i + 1]);
                    y = E ? add2(y, off) : fma2(y, by, off);
                    y = make_float2(power(y.x), power(y.y));
                    if constexpr (E) {
                        const float inv = sc[2 * kFours + i / 4];
                        sums[i / 2 % 2] = fma2(y, make_float2(inv, inv), sums[i / 2 % 2]);
                    } else {
                        sums[i / 2 % 2] = add2(y, sums[i / 2 % 2]);
                    }
                    w[i / 2] = wf_pair<M>::of_float(y.x, y.y);
                }
            };
            sums[0] = sums[1] = make_float2(0.f, 0.f);
            if (p + kKeys > least) {
#pragma unroll
                for (int i = 0; i < kKeys; i++)
                    if (p + i >= seen) s[i] = -INFINITY;
            }
            const float top = largest_of();
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
#pragma unroll
            for (int half = 0; half < 2; half++) {
                powers(half);
                tm_store(st + half * 32, w + half * 32);
            }
            tm_stored();
            before_sync();
            warp_arrive(sh.bar(kBarP + x));
            if constexpr (E) warp_arrive(sh.bar(kBarScale + kSlots + ts % kSlots));
            ts++;
            sums[0] = add2(sums[0], sums[1]);
            sum += sums[0].x + sums[0].y;
        }
        if constexpr (E)  // tiles that this one does not see
            for (int j = n; j < u.n; j++, ts++) {
                if (!sh.wait(kBarScale + ts % kSlots, ts / kSlots & 1)) return;
                warp_arrive(sh.bar(kBarScale + kSlots + ts % kSlots));
            }
        else
            ts += u.n - n;
        if (n > 0) {
            if (!sh.wait(kBarO + x, no & 1)) return;
            no++;
            after_sync();
        }
        uint8_t *mine = there ? a.out + (int64_t)(u.row.first + tok) * a.o_token + (int64_t)(u.head * a.group + (flat - tok * a.group)) * a.o_head : nullptr;
        uint8_t *out[4];  // of the four queries whose elements this lane writes
#pragma unroll
        for (int i = 0; i < 4; i++)
            out[i] = reinterpret_cast<uint8_t *>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(mine), threadIdx.x % 32 / 4 * 4 + i));
        const int at = threadIdx.x;
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
                put<T>(out, i, y, 1.f / sum);
            } else {
#pragma unroll
                for (int k = 0; k < 32; k += 4)
                    __stcg(reinterpret_cast<float4 *>(part) + (i + k) / 4 * kPair + at, make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]));
            }
        }
        before_sync();
        if (__any_sync(~0u, n > 0 && *static_cast<volatile int *>(sh.unfit) > (int)units)) {
            __syncwarp();  // others have written this query's output, too
            if (there) give_unfit<T, E, D>(a, u, seen, u.parts == 1 ? mine : nullptr, part + 4 * at);
        }
        if (u.parts > 1) {
            __stcg(part + kPair * D + at, ref);
            __stcg(part + kPair * (D + 1) + at, sum);
            // The eight warps' parts are there; then one thread's answer.  Each warp reads it before it comes to the next join.
            __threadfence();
            warp_arrive(sh.bar(kBarJoin));
            if (threadIdx.x < 32) {
                if (!sh.wait(kBarJoin, joins & 1)) return;
                if (threadIdx.x == 0) {
                    const bool last = atomicAdd(a.arrive + u.first, 1u) == (uint32_t)u.parts - 1;
                    if (last) a.arrive[u.first] = 0;
                    *last_one = last;
                    bar_arrive(sh.bar(kBarLast));
                }
            }
            if (!sh.wait(kBarLast, joins & 1)) return;
            joins++;
            if (*last_one) {  // the parts together, in their order
                __threadfence();
                auto part_of = [&](int i) { return a.part + (2 * (int64_t)(u.first + i) + (i == 0)) * kPart<D>; };
                float top = -INFINITY, all = 0.f;
                for (int i = 0; i < u.parts; i++) top = fmaxf(top, __ldcg(part_of(i) + kPair * D + at));
                const float base = top == -INFINITY ? 0.f : top;
                for (int i = 0; i < u.parts; i++) all += power(__ldcg(part_of(i) + kPair * D + at) - base) * __ldcg(part_of(i) + kPair * (D + 1) + at);
#pragma unroll 1
                for (int i = 0; i < D; i += 32) {
                    float y[32];
#pragma unroll
                    for (int k = 0; k < 32; k++) y[k] = 0.f;
                    for (int c = 0; c < u.parts; c++) {
                        const float *from = part_of(c);
                        const float g = power(__ldcg(from + kPair * D + at) - base);
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 z = __ldcg(reinterpret_cast<const float4 *>(from) + (i + k) / 4 * kPair + at);
                            y[k] += g * z.x, y[k + 1] += g * z.y, y[k + 2] += g * z.z, y[k + 3] += g * z.w;
                        }
                    }
                    put<T>(out, i, y, 1.f / all);
                }
            }
        }
        sh.unit_done(units);
    }
}

template <typename T, bool E, int D> __global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const __grid_constant__ PromptArgs pa)
{
    const AttendArgs &a = pa.a;
    using S = Shape<E, D>;
    extern __shared__ __align__(1024) uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, last_one, unfit;
    __shared__ Unit units[kUnits];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // A stretch is worth six tiles at least, so that only a unit's first and last CTA can find no tile in their part of it.
    const Found f = find_row<kThreads, true>(a, [&](int64_t total, int64_t rest) {
        return (int32_t)max((int64_t)1, min((int64_t)prompt_sms(a, rest, total), total / (6 * kKeys * (int64_t)a.group)));
    });
    if (f.r >= a.rows) return;
    if (smem_of(raw) % 1024) {  // the swizzle's patterns would not lie as the products read them
        if (threadIdx.x == 0) a.err[1] = 1;
        return;
    }
    Shared sh;
    sh.q = raw;
    sh.kv = sh.q + S::kQBytes;
    sh.raw = sh.kv + S::kStages * S::kTile;
    sh.scales = reinterpret_cast<float *>(sh.raw + S::kRawBytes);
    sh.units = units, sh.bars = smem_of(bars), sh.polls = pa.polls, sh.hint = pa.hint, sh.box = pa.box, sh.gave_up = &gave_up, sh.unfit = &unfit, sh.err = a.err;
    const int warp = threadIdx.x / 32;
    if (threadIdx.x == 0) {
        gave_up = 0, unfit = 0;
        const bool loaders = E || !pa.box || !pa.map_q, boxes = pa.box || pa.map_q;
        for (int i = 0; i < kBars; i++) {
            uint32_t n = 1;  // a warp arrives once
            if (i == kBarQFull) n = pa.map_q ? 1 : 4;
            if (i >= kBarP && i < kBarO) n = 4;
            if (i >= kBarFull && i < kBarFull + 8) n = E || !pa.box ? 4 : 1;
            if (i >= kBarUnit + kUnits && i < kBarUnit + 2 * kUnits) n = 8 + 1 + (loaders ? 4 : 0) + (boxes ? 1 : 0) + (E ? 1 : 0);
            if (i >= kBarRaw + kRaws && i < kBarScale) n = 4;
            if (i >= kBarScale + kSlots && i <= kBarJoin) n = 8;
            bar_init(sh.bar(i), n);
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
        if (E || !pa.box || !pa.map_q) load_role<T, E, D>(pa, sh);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 12) product_role<T, E, D>(sh, tmem);
        if (warp == 13 && threadIdx.x % 32 == 0) unit_role(a, f, sh);
        if (warp == 14 && (pa.box || pa.map_q)) box_role<T, E, D>(pa, sh);
        if (E && warp == 15) scale_role(a, sh);
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

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled, or null; looked up once.
Encode encoder()
{
    static const Encode found = [] {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &how) != cudaSuccess ||
            how != cudaDriverEntryPointSuccess)
            fn = nullptr;
        cudaGetLastError();
        return (Encode)fn;
    }();
    return found;
}

// Whether these arrays can be read by boxes; else they are copied otherwise.
bool encode(CUtensorMap *map, CUtensorMapDataType type, int rank, const void *base, const cuuint64_t *sizes, const cuuint64_t *strides,
            const cuuint32_t *box, bool swizzle)
{
    const Encode f = encoder();
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i + 1 < rank; i++)
        if (!strides[i] || strides[i] >= 1ull << 40) return false;
    return f && f(map, type, rank, const_cast<void *>(base), sizes, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, bool E, int D> int launch(const wf_attn *at, const AttendArgs &args, cudaStream_t st)
{
    PromptArgs pa{};
    AttendArgs &a = pa.a;
    a = args, pa.polls = at->polls, pa.hint = at->polls ? 1000 : 0;
    const auto half = std::is_same_v<T, __half> ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    // Boxes of positions of one block, in whole rows of eight of the swizzle: the largest power of two up to 128 that divides a block, from 8
    // on.  A box is one request, [position / 8][64 elements' group][position % 8][64 elements], since requests are what the copies cost: with one
    // for each 64 elements blocks of 16 took 1,772 us where those of 128 took 1,496 (one prompt of 16,384).  Block and head share a
    // coordinate in steps of a head, which takes blocks that lie whole numbers of such steps apart.
    const int box = std::min(kKeys, a.bs & -a.bs);
    const int64_t step = a.kv == 1 ? a.block_stride : a.head_stride;
    const int64_t heads = step > 0 && a.block_stride % step == 0 ? a.block_stride / step : 0, places = (a.n_blocks - 1) * heads + a.kv;
    if (box >= (E ? 4 : 8) && heads && places < INT32_MAX) {
        const auto type = E ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : half;
        const cuuint64_t tok = (cuuint64_t)a.token_stride, sizes8[3] = {D, (cuuint64_t)a.bs, (cuuint64_t)places}, strides8[2] = {tok, (cuuint64_t)step};
        const cuuint32_t shape8[3] = {D, (cuuint32_t)box, 1};
        const cuuint64_t sizes[5] = {64, 8, D / 64, (cuuint64_t)a.bs / 8, (cuuint64_t)places}, strides[4] = {tok, 128, 8 * tok, (cuuint64_t)step};
        const cuuint32_t shape[5] = {64, 8, D / 64, (cuuint32_t)box / 8, 1};
        auto map = [&](CUtensorMap *m, const uint8_t *base) {
            return E ? encode(m, type, 3, base, sizes8, strides8, shape8, false) : encode(m, type, 5, base, sizes, strides, shape, true);
        };
        if (map(&pa.k, a.k) && map(&pa.v, a.v)) pa.box = box, pa.heads = (int32_t)heads, pa.beyond = (int32_t)places;
    }
    if (E && !pa.box) return -1;
    // Queries of whole tokens: a group's heads, then the next token's.  Over 8 bits bfloat16 queries are scaled first.
    if (a.group <= kQ && !(E && std::is_same_v<T, __nv_bfloat16>)) {
        const int tokens = kQ / a.group;
        const cuuint64_t sizes[3] = {D, (cuuint64_t)a.group * a.kv, (cuuint64_t)a.max_tokens};
        const cuuint64_t strides[2] = {(cuuint64_t)a.q_head, (cuuint64_t)a.q_token};
        const cuuint32_t shape[3] = {64, (cuuint32_t)a.group, (cuuint32_t)tokens};
        pa.map_q = a.q_head > 0 && a.q_token > 0 && encode(&pa.q, half, 3, a.q, sizes, strides, shape, true);
    }
    prompt_kernel<T, E, D><<<at->sms, kThreads, Shape<E, D>::kSmem, st>>>(pa);
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

// WF_OK, an error, or -1: not for this kernel (8 bits whose blocks do not come in fours of positions or lie anyhow).
int wf_launch_prompt(wf_attn *at, const AttendArgs &a, int dtype, int dim, bool eight, cudaStream_t st)
{
    if (dtype == WF_F16) {
        if (dim == 64) return eight ? launch<__half, true, 64>(at, a, st) : launch<__half, false, 64>(at, a, st);
        return eight ? launch<__half, true, 128>(at, a, st) : launch<__half, false, 128>(at, a, st);
    }
    if (dim == 64) return eight ? launch<__nv_bfloat16, true, 64>(at, a, st) : launch<__nv_bfloat16, false, 64>(at, a, st);
    return eight ? launch<__nv_bfloat16, true, 128>(at, a, st) : launch<__nv_bfloat16, false, 128>(at, a, st);
}
