// Attention over the paged cache for rows with few new tokens: decoding above all.
//
// For each query  o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(x_j - m),  x_j the scaled product with key j
// times log2(e), m the largest x_j so far: one pass over the keys and values, with o and the sum
// shrunk by 2^(m - m') whenever m grows.
//
// It has to read every key and value once, 2 (8 bits: 4) operations a byte and query: HBM bounds it.  So what counts
// is that 152 SMs always have enough copies under way, whatever the rows' lengths:
//  - The work is laid on one line: row by row, key head by key head, 16 queries (new tokens x heads of the
//    group) by 16, positions in tiles of 64.  Every CTA takes an equal stretch, wherever it begins.  What a CTA
//    does not hold of a unit alone goes to scratch, and the last of the unit's CTAs to arrive joins the parts in
//    their order.
//  - A warp has its own ring of stages of 16 positions, filled by 16-byte asynchronous copies, and meets the
//    others at the end of a unit only.
//  - Products are 16 x 8 x 16 matrix instructions on 16-bit floats.  A group of few heads leaves rows of the tile
//    empty; that costs nothing while copies bound it.
//
// 8 bits: E4M3 values are halves exactly, so keys and values go into the products unscaled, the queries as halves
// times a power of two of their own (exact but for what is 2^-29 of a row's largest element).  A key's scale multiplies its score.
// A value's scale f_j goes into the weight's exponent, w_j = 2^(x_j + log2 f_j - m), so that the largest
// weight of an unscaled value is 1 whatever the scales' range; the sum of weights takes w_j / f_j.
// 64 rows behind 9,200 tokens (32 / 8 heads of 128) take 369 us, 6.6 TB/s; 128 rows over 8 bits 425 us, 5.6 TB/s of the same bytes: there
// the conversions take half the issue slots.  The walk along the line is one thread's, in shared memory, since registers are what the
// kernels over 8 bits run short of.
// Weights are rounded to the values' type for the second product (by 2^-12 relative in half floats, 2^-9 in bfloat16, where a second
// product takes the remainder: below 2^-17 then), sums of weights are not.
#include <algorithm>
#include <type_traits>

#include "wf_attend.cuh"
#include "wf_decode.cuh"

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kSlice = 16;                // positions of a stage, queries of a unit
constexpr int kTile = kSlice * kWarps;    // positions of a unit of work
static_assert(kSlice == kShortQueries && kTile == kShortTile, "the line's units");
constexpr int kLeast = 6;                 // work that is not split further
constexpr float kLeastScale = 0x1p-64f;  // what a scale of 0 counts as

template <bool E, int D> struct Shape {
    static constexpr int kRow = E ? D : 2 * D;      // bytes of a key
    static constexpr int kChunks = kRow / 16;
    static constexpr int kStages = E ? 4 : D == 64 ? 4 : 3;
    static constexpr int kStage = 2 * kSlice * kRow + (E ? 2 * kSlice * 4 : 0);  // keys, values, scales
    static constexpr int kOutRow = D + 8;           // floats between rows of a warp's result, free of bank conflicts
    static constexpr int kWarpBytes = kStages * kStage;
    static constexpr int kSmem = kWarps * kWarpBytes;
    static constexpr int kCtas = E ? 3 : 2;
    static_assert(kSlice * kOutRow * 4 <= kWarpBytes, "a warp's result fits its stages");
};

// The place of 16-byte chunk c of key i in a stage: eight keys' chunks, and the chunks of a key, lie on different banks.
template <int ROW> __device__ __forceinline__ uint32_t place(int i, int c)
{
    return i * ROW + ((ROW == 64 ? c ^ (i >> 1 & 3) : c ^ (i & 7)) << 4);
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

__device__ __forceinline__ void copy4(uint32_t to, const void *from, bool there)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(there ? 4 : 0) : "memory");
}

__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void await() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldm(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

__device__ __forceinline__ void ldm_t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

template <typename T> __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float power(float x)  // 2^x, 0 for -inf
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float log2_of(float x)
{
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float one_over(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// ---------------------------------------------------------------------------
// A unit
// ---------------------------------------------------------------------------

// Up to 16 queries of a row and key head, and the positions that a CTA takes of them.
struct Unit {
    Row row;
    const int32_t *table;
    int32_t head;         // of keys
    int64_t q0;           // the first query: token * group + head of the group
    int32_t queries;
    int32_t begin, end;   // positions
    int32_t full;         // positions that every query sees
};

// A CTA's way along the line, and what it takes of a unit: positions u.begin .. u.end of it, one of `parts` whose first is CTA `first`'s.
struct Walk {
    Span span;
    int64_t at, stop, row_begin;
    int32_t r;
    Row row;
};
struct Part {
    Unit u;               // no queries: the end
    int32_t first, parts;
};

__device__ __forceinline__ void next_part(const AttendArgs &a, Walk &w, Part &p)
{
    Unit u;
    u.queries = 0;
    while (w.at < w.stop) {
        const int64_t work = short_work(a, w.row);
        if (w.at >= w.row_begin + work) {  // on to the next row
            w.row_begin += work;
            w.row = row_of(a, ++w.r);
            continue;
        }
        const int64_t each = unit_work(w.row), index = quotient(w.at - w.row_begin, each), begin = w.row_begin + index * each;
        const int64_t m = queries_of(a, w.row), tiles = (m + kSlice - 1) / kSlice;
        const int64_t body = begin + kFixed, t0 = max(w.at, body) - body, t1 = min(w.stop, begin + each) - body;
        w.at = min(w.stop, begin + each);
        if (t1 <= t0) continue;
        u.row = w.row, u.table = a.table + w.r * a.table_stride;
        u.head = (int32_t)quotient(index, tiles);
        u.q0 = (index - u.head * tiles) * kSlice;
        u.queries = (int32_t)min((int64_t)kSlice, m - u.q0);
        u.full = w.row.len - w.row.n + (int32_t)wf_quot((uint32_t)u.q0, a.by_group) + 1;
        const int32_t last = w.row.len - w.row.n + (int32_t)wf_quot((uint32_t)(u.q0 + u.queries - 1), a.by_group) + 1;
        u.begin = (int32_t)min((int64_t)last, t0 * kTile), u.end = (int32_t)min((int64_t)last, t1 * kTile);
        p.first = 0, p.parts = 1;
        if (t0 || t1 != each - kFixed) {
            p.first = w.span.owner(body);
            p.parts = w.span.owner(begin + each - 1) - p.first + 1;
        }
        break;
    }
    p.u = u;
}

// By warp: whether it has taken a value that is no finite number out of its part of the unit.
__device__ __forceinline__ volatile int *unfit_flags()
{
    __shared__ volatile int flags[kWarps];
    return flags;
}

template <typename T, bool E, int D> struct Kernel {
    using S = Shape<E, D>;
    using V = std::conditional_t<E, __nv_fp8_e4m3, T>;  // of the cache
    using M = std::conditional_t<E, __half, T>;  // of the products
    static constexpr int kSteps = D / 16, kTiles = D / 8;
    static constexpr bool kTwice = !E && std::is_same_v<T, __nv_bfloat16>;
    // Weights in half floats reach up to 2^15 in place of 1, sums of them likewise: so what is 2^-40 of the largest still counts (2^-25 else, and many
    // keys behind one that has most of the weight would be lost in the result, not in the sum).
    static constexpr float kLift = std::is_same_v<M, __half> ? 15.f : 0.f;

    float o[kTiles][4], m[2], l[2];
    uint32_t q[kSteps][4];
    float scale[2];
    int32_t seen[2];  // positions that the lane's two queries see

    // Queries as the first operand: step s holds elements 16s + 2c, +1, +8, +9 (c: lane % 4) of rows lane / 4 and + 8; in 8 bits
    // 16s + 4c .. 4c + 3, as a key's bytes come.
    __device__ __forceinline__ void load_queries(const AttendArgs &a, const Unit &u, int lane)
    {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int at = lane / 4 + 8 * i;
            const bool there = at < u.queries;
            const uint32_t f = (uint32_t)(u.q0 + (there ? at : 0)), tok = wf_quot(f, a.by_group);
            const uint8_t *p = a.q + (int64_t)(u.row.first + tok) * a.q_token + (int64_t)(u.head * a.group + (f - tok * a.group)) * a.q_head;
            seen[i] = u.row.len - u.row.n + (int32_t)tok + 1;
            scale[i] = a.scale;
#pragma unroll
            for (int s = 0; s < kSteps; s++) {
                if (E) {
                    const uint2 x = there ? *reinterpret_cast<const uint2 *>(p + 32 * s + 8 * (lane % 4)) : make_uint2(0, 0);
                    q[s][i] = x.x, q[s][2 + i] = x.y;
                } else {
                    const uint8_t *e = p + 32 * s + 4 * (lane % 4);
                    q[s][i] = there ? *reinterpret_cast<const uint32_t *>(e) : 0;
                    q[s][2 + i] = there ? *reinterpret_cast<const uint32_t *>(e + 16) : 0;
                }
            }
            if (E && std::is_same_v<T, __nv_bfloat16>) {
                float most = 0.f;
#pragma unroll
                for (int s = 0; s < kSteps; s++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const float2 x = wf_pair<T>::to_float(q[s][2 * j + i]);
                        most = fmaxf(most, fmaxf(fabsf(x.x), fabsf(x.y)));
                    }
#pragma unroll
                for (int s = 1; s < 4; s *= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, s));
                // The largest element to 2^13..2^14: halves hold what is 2^27 below it without loss.
                const int e = most > 0.f && most <= 3.402823466e38f ? min(max((__float_as_int(most) >> 23) - 127 - 13, -100), 127 - 13) : 0;
                const float down = __int_as_float((127 - e) << 23);
                scale[i] *= __int_as_float((127 + e) << 23);
#pragma unroll
                for (int s = 0; s < kSteps; s++)
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const float2 x = wf_pair<T>::to_float(q[s][2 * j + i]);
                        q[s][2 * j + i] = wf_pair<__half>::of_float(x.x * down, x.y * down);
                    }
            }
        }
    }

    // Copies of positions p .. p + 15 into a stage; b: the block of lane % 16's position.
    __device__ __forceinline__ void fill(const AttendArgs &a, const Unit &u, uint32_t stage, int32_t p, int32_t b, int lane)
    {
        const int32_t mine = p + lane % kSlice;
        const uint32_t j = wf_quot(min(mine, u.end - 1), a.by_bs);
        const int64_t off = b * a.block_stride + (int64_t)(min(mine, u.end - 1) - (int32_t)j * a.bs) * a.token_stride;
        const uint8_t *k = a.k + u.head * a.head_stride, *v = a.v + u.head * a.head_stride;
#pragma unroll
        for (int i = 0; i < S::kChunks / 2; i++) {
            const int id = 32 * i + lane, key = id / S::kChunks, c = id % S::kChunks;
            const int64_t from = __shfl_sync(~0u, off, key) + 16 * c;
            const bool there = p + key < u.end;
            copy16(stage + place<S::kRow>(key, c), k + from, there);
            copy16(stage + kSlice * S::kRow + place<S::kRow>(key, c), v + from, there);
        }
        if (E) copy4(stage + 2 * kSlice * S::kRow + 4 * lane, (lane < kSlice ? a.k_scale : a.v_scale) + (int64_t)b * a.kv + u.head, mine < u.end);
    }

    __device__ __forceinline__ int32_t block_of(const AttendArgs &a, const Unit &u, int32_t p, int lane)
    {
        return block_at(a, u.table, wf_quot(min(p + lane % kSlice, u.end - 1), a.by_bs));
    }

    // Values from `from` on of a stage, which some queries do not see: what is no finite number becomes 0, and add_unfit's.
    __device__ __forceinline__ void take_unfit(uint8_t *buf, int from, int lane)
    {
        bool found = false;
#pragma unroll
        for (int i = 0; i < S::kChunks / 2; i++) {
            const int id = 32 * i + lane, key = id / S::kChunks, c = id % S::kChunks;
            if (key < from) continue;
            uint4 *at = reinterpret_cast<uint4 *>(buf + kSlice * S::kRow + place<S::kRow>(key, c));
            const uint4 x = *at;
            if (wf_unfit<V>(x)) *at = wf_fit<V>(x), found = true;
        }
        if (found) unfit_flags()[threadIdx.x / 32] = 1;
        __syncwarp();
    }

    __device__ __forceinline__ void slice(const Unit &u, uint8_t *buf, uint32_t stage, int32_t p, int lane)
    {
        const int c = lane % 4;
        if (p + kSlice > u.full && u.full < u.end) take_unfit(buf, u.full - p, lane);
        float x[2][4] = {};
        if (!E) {
            const int key = lane / 16 * 8 + lane % 8, odd = lane / 8 % 2;
#pragma unroll
            for (int s = 0; s < kSteps; s++) {
                uint32_t b[4];
                ldm(b, stage + place<S::kRow>(key, 2 * s + odd));
                mma<M>(x[0], q[s], b[0], b[1]);
                mma<M>(x[1], q[s], b[2], b[3]);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int s = 0; s < kSteps; s += 4) {
                    uint32_t b[4];
                    ldm(b, stage + place<S::kRow>(8 * t + lane % 8, s + lane / 8));
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const uint2 h = wf_e4m3_halves(b[j]);
                        mma<M>(x[t], q[s + j], h.x, h.y);
                    }
                }
        }
        // Scores; the lane has positions p + 8t + 2c, + 1 of its two queries.
        float2 inv[2];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            float2 ks, log;
            if (E) {
                const float2 *sc = reinterpret_cast<const float2 *>(buf + 2 * kSlice * S::kRow) + 4 * t + c;
                const float2 f = make_float2(fmaxf(sc[kSlice / 2].x, kLeastScale), fmaxf(sc[kSlice / 2].y, kLeastScale));
                ks = sc[0], log = make_float2(log2_of(f.x), log2_of(f.y)), inv[t] = make_float2(one_over(f.x), one_over(f.y));
            }
#pragma unroll
            for (int i = 0; i < 2; i++) {
                x[t][2 * i] = E ? fmaf(x[t][2 * i], scale[i] * ks.x, log.x) : x[t][2 * i] * scale[i];
                x[t][2 * i + 1] = E ? fmaf(x[t][2 * i + 1], scale[i] * ks.y, log.y) : x[t][2 * i + 1] * scale[i];
            }
        }
        if (p + kSlice > u.full || p + kSlice > u.end) {
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (p + 8 * t + 2 * c + j % 2 >= min(seen[j / 2], u.end)) x[t][j] = -INFINITY;
        }
        float most[2] = {fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1])), fmaxf(fmaxf(x[0][2], x[0][3]), fmaxf(x[1][2], x[1][3]))};
#pragma unroll
        for (int s = 1; s < 4; s *= 2) {
            most[0] = fmaxf(most[0], __shfl_xor_sync(~0u, most[0], s));
            most[1] = fmaxf(most[1], __shfl_xor_sync(~0u, most[1], s));
        }
        if (__any_sync(~0u, most[0] > m[0] || most[1] > m[1])) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float now = fmaxf(m[i], most[i]);
                const float f = m[i] == now ? 1.f : power(m[i] - now);
                m[i] = now;
                l[i] *= f;
#pragma unroll
                for (int t = 0; t < kTiles; t++) o[t][2 * i] *= f, o[t][2 * i + 1] *= f;
            }
        }
        uint32_t w[4], rest[4];
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const float ref = m[i] == -INFINITY ? 0.f : m[i] - kLift;  // nothing seen yet
                const float a = power(x[t][2 * i] - ref), b = power(x[t][2 * i + 1] - ref);
                l[i] += E ? fmaf(a, inv[t].x, b * inv[t].y) : a + b;
                w[2 * t + i] = wf_pair<M>::of_float(a, b);
                if (kTwice) {
                    const float2 had = wf_pair<M>::to_float(w[2 * t + i]);
                    rest[2 * t + i] = wf_pair<M>::of_float(a - had.x, b - had.y);
                }
            }
        if (!E) {
            const int key = lane % 16, odd = lane / 16;
#pragma unroll
            for (int t = 0; t < kTiles; t += 2) {
                uint32_t b[4];
                ldm_t(b, stage + kSlice * S::kRow + place<S::kRow>(key, t + odd));
                mma<M>(o[t], w, b[0], b[1]);
                mma<M>(o[t + 1], w, b[2], b[3]);
                if (kTwice) {
                    mma<M>(o[t], rest, b[0], b[1]);
                    mma<M>(o[t + 1], rest, b[2], b[3]);
                }
            }
        } else {
            // The lane's column of tile t is element (D / 8) (lane / 4) + t: a key's D / 8 bytes from there on hold all of them.
            constexpr int kBytes = D / 8;
            uint32_t x4[4][kBytes / 4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int key = 2 * c + j % 2 + j / 2 * 8;
                const uint8_t *from = buf + kSlice * S::kRow + place<S::kRow>(key, lane / 4 * kBytes / 16) + lane / 4 * kBytes % 16;
                if (kBytes == 16) {
                    const uint4 r = *reinterpret_cast<const uint4 *>(from);
                    x4[j][0] = r.x, x4[j][1] = r.y, x4[j][kBytes / 4 - 2] = r.z, x4[j][kBytes / 4 - 1] = r.w;
                } else {
                    const uint2 r = *reinterpret_cast<const uint2 *>(from);
                    x4[j][0] = r.x, x4[j][1] = r.y;
                }
            }
#pragma unroll
            for (int t = 0; t < kTiles; t += 4) {
                uint2 h[4];
#pragma unroll
                for (int j = 0; j < 4; j++) h[j] = wf_e4m3_halves(x4[j][t / 4]);
                mma<M>(o[t], w, __byte_perm(h[0].x, h[1].x, 0x5410), __byte_perm(h[2].x, h[3].x, 0x5410));
                mma<M>(o[t + 1], w, __byte_perm(h[0].x, h[1].x, 0x7632), __byte_perm(h[2].x, h[3].x, 0x7632));
                mma<M>(o[t + 2], w, __byte_perm(h[0].y, h[1].y, 0x5410), __byte_perm(h[2].y, h[3].y, 0x5410));
                mma<M>(o[t + 3], w, __byte_perm(h[0].y, h[1].y, 0x7632), __byte_perm(h[2].y, h[3].y, 0x7632));
            }
        }
    }

    // The warp's share of the unit's positions, every kWarps-th slice.
    __device__ __forceinline__ void run(const AttendArgs &a, const Unit &u, uint8_t *buf, int warp, int lane)
    {
        const uint32_t base = (uint32_t)__cvta_generic_to_shared(buf);
        const int n = max(0, (u.end - u.begin - warp * kSlice + kTile - 1) / kTile);
        auto pos = [&](int i) { return u.begin + i * kTile + warp * kSlice; };
        int32_t next = n > 0 ? block_of(a, u, pos(0), lane) : 0;
        int in = 0;
#pragma unroll
        for (int i = 0; i < S::kStages - 1; i++) {
            if (in < n) {
                fill(a, u, base + i * S::kStage, pos(in), next, lane);
                if (++in < n) next = block_of(a, u, pos(in), lane);
            }
            commit();
        }
        load_queries(a, u, lane);
#pragma unroll
        for (int t = 0; t < kTiles; t++) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
        m[0] = m[1] = -INFINITY, l[0] = l[1] = 0.f;
        int s = 0;
        for (int i = 0; i < n; i++) {
            await<S::kStages - 2>();
            __syncwarp();
            const int free = s == 0 ? S::kStages - 1 : s - 1;
            if (in < n) {
                fill(a, u, base + free * S::kStage, pos(in), next, lane);
                if (++in < n) next = block_of(a, u, pos(in), lane);
            }
            commit();
            slice(u, buf + s * S::kStage, base + s * S::kStage, pos(i), lane);
            s = s + 1 == S::kStages ? 0 : s + 1;
        }
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int k = 1; k < 4; k *= 2) l[i] += __shfl_xor_sync(~0u, l[i], k);
        // The result in place of the stages.
        await<0>();
        __syncwarp();
        float *res = reinterpret_cast<float *>(buf);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            float *row = res + (lane / 4 + 8 * i) * S::kOutRow;
            const int c = lane % 4;
#pragma unroll
            for (int t = 0; t < kTiles; t++) {
                if (E) row[kTiles * 2 * c + t] = o[t][2 * i], row[kTiles * (2 * c + 1) + t] = o[t][2 * i + 1];
                else *reinterpret_cast<float2 *>(row + 8 * t + 2 * c) = make_float2(o[t][2 * i], o[t][2 * i + 1]);
            }
        }
    }
};

template <typename T, int D>
__device__ __forceinline__ void put_out(const AttendArgs &a, const Unit &u, int q, int e, const float (&x)[8])
{
    const uint32_t f = (uint32_t)(u.q0 + q), tok = wf_quot(f, a.by_group);
    uint8_t *p = a.out + (int64_t)(u.row.first + tok) * a.o_token + (int64_t)(u.head * a.group + (f - tok * a.group)) * a.o_head + 2 * e;
    *reinterpret_cast<uint4 *>(p) = make_uint4(wf_pair<T>::of_float(x[0], x[1]), wf_pair<T>::of_float(x[2], x[3]),
                                               wf_pair<T>::of_float(x[4], x[5]), wf_pair<T>::of_float(x[6], x[7]));
}

// Beside prompt_kernel this kernel ends after it, so that what follows on the stream finds both done.
__device__ __forceinline__ void leave(const AttendArgs &a)
{
    if (a.both && blockIdx.x == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Parts in scratch: [16 queries][D] sums, [16] references, [16] sums of weights.
template <int D> constexpr int kPart = kSlice * (D + 2);

template <typename T, bool E, int D> __global__ void __launch_bounds__(kThreads, Shape<E, D>::kCtas) attend_kernel(const AttendArgs a)
{
    using S = Shape<E, D>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float s_m[kWarps][kSlice], s_l[kWarps][kSlice], s_sum[kSlice];
    __shared__ bool s_last;
    __shared__ Walk s_walk;
    __shared__ Part s_part;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Found f = find_row<kThreads, false>(a, [&](int64_t total, int64_t rest) {
        const int64_t room = rest ? gridDim.x / a.sms * (a.sms - prompt_sms(a, total, rest)) : gridDim.x;
        return (int32_t)max((int64_t)1, min(room, total / kLeast));
    });
    if (f.r >= a.rows) {
        leave(a);
        return;
    }
    // The walk along the line is one thread's, and lies in shared memory: the others' registers are for the products.
    if (threadIdx.x == 0) s_walk = {f.span, f.span.begin(blockIdx.x), f.span.begin(blockIdx.x + 1), f.row_begin, f.r, f.row};
    for (;;) {
        if (threadIdx.x == 0) next_part(a, s_walk, s_part);
        __syncthreads();
        const Unit u = s_part.u;
        if (!u.queries) break;
        uint8_t *buf = smem + warp * S::kWarpBytes;
        if (u.full < u.end) {
            if (lane == 0) unfit_flags()[warp] = 0;
            __syncwarp();
        }
        {
            Kernel<T, E, D> k;
            k.run(a, u, buf, warp, lane);
            if (lane % 4 == 0) {
                s_m[warp][lane / 4] = k.m[0], s_m[warp][lane / 4 + 8] = k.m[1];
                s_l[warp][lane / 4] = k.l[0], s_l[warp][lane / 4 + 8] = k.l[1];
            }
        }
        __syncthreads();
        // The warps' results together: 8 elements of a query at a time.
        const int32_t first = s_part.first, n = s_part.parts;
        float *part = a.part + (2 * (int64_t)blockIdx.x + (blockIdx.x == first)) * kPart<D>;
        for (int i = threadIdx.x; i < u.queries * (D / 8); i += kThreads) {
            const int q = i / (D / 8), e = i % (D / 8) * 8;
            float ref = s_m[0][q], sum = 0.f, x[8] = {};
#pragma unroll
            for (int w = 1; w < kWarps; w++) ref = fmaxf(ref, s_m[w][q]);
            const float base = ref == -INFINITY ? 0.f : ref;
#pragma unroll
            for (int w = 0; w < kWarps; w++) {
                const float g = power(s_m[w][q] - base);
                const float4 *p = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem + w * S::kWarpBytes) + q * S::kOutRow + e);
                const float4 y = p[0], z = p[1];
                sum += g * s_l[w][q];
                x[0] += g * y.x, x[1] += g * y.y, x[2] += g * y.z, x[3] += g * y.w;
                x[4] += g * z.x, x[5] += g * z.y, x[6] += g * z.z, x[7] += g * z.w;
            }
            static_assert(kWarps == 4, "the flags");
            if (volatile int *f = unfit_flags(); u.full < u.end && (f[0] | f[1] | f[2] | f[3])) {
                const int32_t seen = u.row.len - u.row.n + (int32_t)wf_quot((uint32_t)(u.q0 + q), a.by_group) + 1;
                using V = typename Kernel<T, E, D>::V;
                add_unfit<V>(a, u.table, a.v + u.head * a.head_stride + e * (int)sizeof(V), max(u.begin, u.full), min(u.end, seen), x);
            }
            if (n == 1) {
                const float inv = 1.f / sum;
#pragma unroll
                for (int j = 0; j < 8; j++) x[j] *= inv;
                put_out<T, D>(a, u, q, e, x);
            } else {
                float4 *p = reinterpret_cast<float4 *>(part + q * D + e);
                __stcg(p, make_float4(x[0], x[1], x[2], x[3]));
                __stcg(p + 1, make_float4(x[4], x[5], x[6], x[7]));
                if (e == 0) __stcg(part + kSlice * D + q, ref), __stcg(part + kSlice * (D + 1) + q, sum);
            }
        }
        if (n > 1) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) {
                s_last = atomicAdd(a.arrive + first, 1u) == (uint32_t)n - 1;
                if (s_last) a.arrive[first] = 0;
            }
            __syncthreads();
            if (s_last) {
                __threadfence();
                // Part i: that of CTA first + i, the beginning unit's in its second place, the others' in their first.
                auto part_of = [&](int i) { return a.part + (2 * (int64_t)(first + i) + (i == 0)) * kPart<D>; };
                float *weight = reinterpret_cast<float *>(smem);  // [n][16]
                for (int q = warp; q < u.queries; q += kWarps) {
                    float ref = -INFINITY;
                    for (int i = lane; i < n; i += 32) ref = fmaxf(ref, __ldcg(part_of(i) + kSlice * D + q));
#pragma unroll
                    for (int s = 16; s; s /= 2) ref = fmaxf(ref, __shfl_xor_sync(~0u, ref, s));
                    const float base = ref == -INFINITY ? 0.f : ref;
                    float sum = 0.f;
                    for (int i = lane; i < n; i += 32) {
                        const float g = power(__ldcg(part_of(i) + kSlice * D + q) - base);
                        weight[i * kSlice + q] = g;
                        sum += g * __ldcg(part_of(i) + kSlice * (D + 1) + q);
                    }
#pragma unroll
                    for (int s = 16; s; s /= 2) sum += __shfl_xor_sync(~0u, sum, s);
                    if (lane == 0) s_sum[q] = 1.f / sum;
                }
                __syncthreads();
                for (int i = threadIdx.x; i < u.queries * (D / 8); i += kThreads) {
                    const int q = i / (D / 8), e = i % (D / 8) * 8;
                    float x[8] = {};
#pragma unroll 4
                    for (int j = 0; j < n; j++) {
                        const float4 *p = reinterpret_cast<const float4 *>(part_of(j) + q * D + e);
                        const float4 y = __ldcg(p), z = __ldcg(p + 1);
                        const float g = weight[j * kSlice + q];
                        x[0] += g * y.x, x[1] += g * y.y, x[2] += g * y.z, x[3] += g * y.w;
                        x[4] += g * z.x, x[5] += g * z.y, x[6] += g * z.z, x[7] += g * z.w;
                    }
#pragma unroll
                    for (int j = 0; j < 8; j++) x[j] *= s_sum[q];
                    put_out<T, D>(a, u, q, e, x);
                }
            }
        }
        __syncthreads();
    }
    leave(a);
}

template <typename T, bool E, int D> int setup(int sms, int *grid)
{
    using S = Shape<E, D>;
    int ctas = 0;
    int rc = wf_cuda_check(cudaFuncSetAttribute(attend_kernel<T, E, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem), "attend_kernel");
    if (!rc) rc = wf_cuda_check(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, attend_kernel<T, E, D>, kThreads, S::kSmem), "attend_kernel");
    *grid = sms * std::max(1, ctas);
    // The join's weights, one of 16 queries for each CTA, lie where the stages did.
    if (!rc && (size_t)*grid * kSlice * sizeof(float) > (size_t)S::kSmem) *grid = S::kSmem / (kSlice * sizeof(float));
    return rc;
}

template <typename T, bool E, int D> int launch(const wf_attn *at, const AttendArgs &a, cudaStream_t st)
{
    cudaLaunchConfig_t c{};
    c.gridDim = at->grid[E][D == 128], c.blockDim = kThreads, c.dynamicSmemBytes = Shape<E, D>::kSmem, c.stream = st;
    cudaLaunchAttribute beside{};
    beside.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    beside.val.programmaticStreamSerializationAllowed = 1;
    c.attrs = &beside, c.numAttrs = a.both ? 1 : 0;
    return wf_cuda_check(cudaLaunchKernelEx(&c, attend_kernel<T, E, D>, a), "attend_kernel");
}

}  // namespace

int wf_attend_setup(wf_attn *at)
{
    int rc = WF_OK, g = 0;
    auto both = [&](int r, int *grid) { rc = rc ? rc : r, *grid = *grid ? std::min(*grid, g) : g; };
    both(setup<__half, false, 64>(at->sms, &g), &at->grid[0][0]);
    both(setup<__nv_bfloat16, false, 64>(at->sms, &g), &at->grid[0][0]);
    both(setup<__half, false, 128>(at->sms, &g), &at->grid[0][1]);
    both(setup<__nv_bfloat16, false, 128>(at->sms, &g), &at->grid[0][1]);
    both(setup<__half, true, 64>(at->sms, &g), &at->grid[1][0]);
    both(setup<__nv_bfloat16, true, 64>(at->sms, &g), &at->grid[1][0]);
    both(setup<__half, true, 128>(at->sms, &g), &at->grid[1][1]);
    both(setup<__nv_bfloat16, true, 128>(at->sms, &g), &at->grid[1][1]);
    return rc;
}

// Scratch of attend_kernel for any of its launches: parts in bytes, CTAs.
void wf_attend_scratch(const wf_attn *at, size_t *part_bytes, int *ctas)
{
    const int g64 = std::max(at->grid[0][0], at->grid[1][0]), g128 = std::max(at->grid[0][1], at->grid[1][1]);
    *ctas = std::max(g64, g128);
    *part_bytes = sizeof(float) * 2 * std::max((size_t)g64 * kPart<64>, (size_t)g128 * kPart<128>);
}

int wf_launch_attend(wf_attn *at, const AttendArgs &a, int dtype, int dim, bool eight, cudaStream_t st)
{
    if (dtype == WF_F16) {
        if (dim == 64) return eight ? launch<__half, true, 64>(at, a, st) : launch<__half, false, 64>(at, a, st);
        return eight ? launch<__half, true, 128>(at, a, st) : launch<__half, false, 128>(at, a, st);
    }
    if (dim == 64) return eight ? launch<__nv_bfloat16, true, 64>(at, a, st) : launch<__nv_bfloat16, false, 64>(at, a, st);
    return eight ? launch<__nv_bfloat16, true, 128>(at, a, st) : launch<__nv_bfloat16, false, 128>(at, a, st);
}
