// Beam search's selection over beams and vocabulary (wf_beam_select).
//
// A candidate's sum is score + (x - m) - log Z, with a row's maximum m and
// Z = sum of exp(x - m).  One launch that reads the logits once:
//
//   1. The rows' logits, taken as one long run of units (a line of 512 bytes,
//      a warp's load, or several), are dealt out evenly to the warps.  A warp
//      sums the exponentials of its part of a row and keeps the maximum of
//      every unit; no barrier, no choice of candidates.
//   2. The last CTA of a search joins: m and Z of its rows, the sums of the
//      units' maxima, and a bound that at least `keep` of those reach.  Only the units that
//      reach it hold candidates that count, so only those are read again.
//
// The exponentials are summed relative to a value near the start of the
// warp's part: a sum relative to any value is as exact as one relative to
// the maximum as long as it stays within a float's range, and a row where it
// did not is summed again by the join.  Additions go in pairs and, where they
// are many, are compensated, so that a term passes through some 80 roundings in
// the streaming pass and 26 in the join's.
//
// The bound: the threads' maxima, over 32 or 64 classes of threads, have a
// keep-th largest.  The classes hold interleaved units, so few more than `keep`
// reach it, unless many are equal (a mask of one low value); then the keys that
// order equal sums by their place make the bound.
//
// Measured: 64 searches of 8 beams over 131,072 bf16 tokens (134 MB) take 32.2
// us; the last warp of step 1 ends at 22 us (6.1 TB/s; 63 warp instructions a
// line, 38 % of the issue slots: bound by HBM), the join takes 7 us more, the
// launch 2.  The join is bound by its chain (arrival, parts and units, the units
// read again: trips to L2 or HBM of 1,100 to 1,900 cycles) and by code that runs
// once a CTA, so what is not on its path stays out of line.  One search of 4
// beams over 32,000 tokens, all join, takes 8.7 to 9.0 us.  Lists of candidates that
// each CTA's part of a row kept, with a running bound, took 46 us for the large
// case: 10 K warp instructions a part, and barriers that leave the loads waiting.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "wf_decode.cuh"

namespace {

constexpr uint32_t kFull = 0xFFFFFFFFu;
constexpr int kCap = 512;      // keys gathered before they are ranked
constexpr int kStep = 4;       // lines that a warp has in flight, and as many in work
constexpr int kSum = 64;       // steps whose sums are added up before that sum joins the warp's
constexpr int kUnits = 4096 + kMaxGroup;  // units of a search, at most: shared memory holds their maxima
constexpr int kPick = 128;     // units that the join reads again, at most, before it orders them by key

// CTAs of 256 threads, three an SM (80 registers; with four and 64, spills:
// 0.4 us more for one search, 0.7 for 16), which stream best; or, where the
// join counts for more, of 512, one an SM.  deal() chooses.
constexpr int kSmall = 256, kBig = 512;
constexpr int per_sm(int threads) { return threads == kSmall ? 3 : 1; }

constexpr float kLog2e = 1.4426950408889634f;

// Whole numbers in the order of the floats; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }

// What candidates (and units, by their maxima) are ordered by, the larger
// key first: hi by sum, then lower beam; lo by logit, then lower place
// (token, or unit in the row).  hi = 0: none.
struct Key {
    uint64_t hi, lo;
};
__device__ __forceinline__ bool operator>(const Key &a, const Key &b) { return a.hi > b.hi || (a.hi == b.hi && a.lo > b.lo); }
__device__ __forceinline__ Key shuffle(const Key &k, int o)
{
    return {__shfl_xor_sync(kFull, k.hi, o), __shfl_xor_sync(kFull, k.lo, o)};
}

// The warp's keys in descending order, lane 0 the largest.
__device__ __noinline__ Key warp_sorted(Key v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll 1
        for (int o = size >> 1; o > 0; o >>= 1) {
            const Key w = shuffle(v, o);
            const bool first = (lane & o) == 0, down = size == 32 || (lane & size) == 0;
            if ((first == down) == (w > v)) v = w;
        }
    return v;
}

__device__ __forceinline__ float warp_sorted(float v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int o = size >> 1; o > 0; o >>= 1) {
            const float w = __shfl_xor_sync(kFull, v, o);
            const bool first = (lane & o) == 0, down = size == 32 || (lane & size) == 0;
            v = first == down ? fmaxf(v, w) : fminf(v, w);
        }
    return v;
}

// How a search's warps share its rows: each row is cut alike, so that equal rows
// that lie alike in memory have equal sums to the last bit.  Part q of the j-th row is number j * of_row + q.
struct Share {
    int of_row;  // warps of a row (1: a warp may have several rows)
    int units;   // units of a warp in a row
};

template <int kThreads>
struct Shared {
    static constexpr int kWarps = kThreads / 32;
    union {
        Key best[kWarps][32];  // the threads' best
        float most[kWarps][32];
    };
    Key got[kCap];           // gathered keys
    Key sorted[kMaxKeep];    // the best, in order; hi = 0 past the last
    union {
        float unit[kUnits];  // the units' maxima, then their sums
        struct {
            uint4 aside[kCap];           // vectors with a candidate that reaches the bound
            int2 aside_of[kCap];         // ... their beam and the token of their first element
        };
    };
    int32_t pick[kCap];      // units that reach the bound, counted over the search; at most kPick are read again
    float cut;               // the bound
    Key bound;
    uint32_t count, n_aside;
    uint32_t again;          // rows whose exponentials are summed again
    uint32_t live;           // the search's rows that have a score
    Share share;
    float score[kMaxGroup];
    float4 stat[kMaxGroup];  // a row's maximum, log Z and score
    float sum[kWarps];
    bool last;
};

// Each of the count keys in sm.got finds its place among them, four threads a
// key; the n best go to sm.sorted.
template <int kThreads>
__device__ __noinline__ void rank_keys(Shared<kThreads> &sm, int count, int n)
{
    const int tid = threadIdx.x;
    if (tid < n) sm.sorted[tid] = {0, 0};
    __syncthreads();
    for (int i = tid >> 2; i < (count + 7) / 8 * 8; i += kThreads / 4) {
        const Key k = i < count ? sm.got[i] : Key{0, 0};
        int ahead = 0;
#pragma unroll 4
        for (int j = tid & 3; j < count; j += 4) ahead += sm.got[j] > k;
        ahead += __shfl_xor_sync(kFull, ahead, 1);
        ahead += __shfl_xor_sync(kFull, ahead, 2);
        if (i < count && (tid & 3) == 0 && ahead < n) sm.sorted[ahead] = k;
    }
    __syncthreads();
}

// The n best of the CTA's keys, to sm.sorted: each(f) calls f with every key
// of this thread, and can be called again.
template <int kThreads, class Each>
__device__ __noinline__ void best_keys(Shared<kThreads> &sm, int n, const Each &each)
{
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    Key mine = {0, 0};
    each([&](const Key &k) { if (k > mine) mine = k; });
    __syncthreads();
    sm.best[warp][lane] = mine;
    __syncthreads();
    if (warp == 0) {
        Key even = sm.best[0][lane], odd = sm.best[1][lane];
        for (int w = 2; w < kWarps; w += 2) {
            const Key x = sm.best[w][lane], y = sm.best[w + 1][lane];
            if (x > even) even = x;
            if (y > odd) odd = y;
        }
        // The n-th best of 32 classes; of 64 (two sorted halves) from n = 17 on, the least of those beyond 32.
        Key sorted;
        if (n <= 16) {
            sorted = warp_sorted(even > odd ? even : odd);
        } else if (n <= 32) {
            const Key x = warp_sorted(even), y = warp_sorted(odd);
            const Key z = {__shfl_sync(kFull, y.hi, 31 - lane), __shfl_sync(kFull, y.lo, 31 - lane)};
            sorted = warp_sorted(x > z ? x : z);
        } else {
            sorted = warp_sorted(even > odd ? odd : even);
        }
        if (lane == min(n, 32) - 1) sm.bound = sorted;
        if (lane == 0) sm.count = 0;
    }
    __syncthreads();
    Key bound = sm.bound;
    for (int round = 0; round < 4; ++round) {
        each([&](const Key &k) {
            if (!k.hi || bound > k) return;
            const uint32_t at = atomicAdd(&sm.count, 1u);
            if (at < kCap) sm.got[at] = k;
        });
        __syncthreads();
        const int came = (int)sm.count;
        rank_keys(sm, min(came, kCap), n);
        if (came <= kCap) return;
        // An order that defeats the classes: the n-th of those that were kept is a better bound.
        bound = sm.sorted[n - 1];
        if (tid == 0) sm.count = 0;
        __syncthreads();
    }
    // Still too many: one after the other.
    Key last = {~0ull, ~0ull};
    for (int r = 0; r < n; ++r) {
        Key next = {0, 0};
        each([&](const Key &k) { if (last > k && k > next) next = k; });
#pragma unroll 1
        for (int o = 16; o > 0; o >>= 1) {
            const Key w = shuffle(next, o);
            if (w > next) next = w;
        }
        __syncthreads();
        if (lane == 0) sm.best[0][warp] = next;
        __syncthreads();
        last = {0, 0};
        for (int w = 0; w < kWarps; ++w)
            if (sm.best[0][w] > last) last = sm.best[0][w];
        if (tid == 0) sm.sorted[r] = last;
    }
    __syncthreads();
}

// The elements of a 16-byte vector as floats, and their maximum (NaN passed over).
template <int kType>
struct Elems;
template <>
struct Elems<WF_F32> {
    static constexpr int n = 4;
    using type = float;
    static __device__ __forceinline__ void get(const uint4 &v, float *x)
    {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float most(const uint4 &v)
    {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ uint32_t masked() { return 0xFF800000u; }  // -inf
};
template <>
struct Elems<WF_F16> {
    static constexpr int n = 8;
    using type = uint16_t;
    static __device__ __forceinline__ void get(const uint4 &v, float *x)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*(const __half2 *)&w[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float most(const uint4 &v)
    {
        const __half2 m = __hmax2(__hmax2(*(const __half2 *)&v.x, *(const __half2 *)&v.y),
                                  __hmax2(*(const __half2 *)&v.z, *(const __half2 *)&v.w));
        const float2 f = __half22float2(m);
        return fmaxf(f.x, f.y);
    }
    static __device__ __forceinline__ uint32_t masked() { return 0xFC00FC00u; }
};
template <>
struct Elems<WF_BF16> {
    static constexpr int n = 8;
    using type = uint16_t;
    static __device__ __forceinline__ void get(const uint4 &v, float *x)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ float most(const uint4 &v)
    {
        const __nv_bfloat162 m = __hmax2(__hmax2(*(const __nv_bfloat162 *)&v.x, *(const __nv_bfloat162 *)&v.y),
                                         __hmax2(*(const __nv_bfloat162 *)&v.z, *(const __nv_bfloat162 *)&v.w));
        const uint32_t w = *(const uint32_t *)&m;
        return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    }
    static __device__ __forceinline__ uint32_t masked() { return 0xFF80FF80u; }
};

// 2^x, 0 below the smallest normal number.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Sum: what is added to it passes through two roundings, however many additions follow (Kahan's compensated sum).
struct Sum {
    float s = 0, low = 0;
    __device__ __forceinline__ void add(float x)
    {
        const float y = x - low, t = s + y;
        low = (t - s) - y;
        s = t;
    }
};

// x[0] + ... + x[n - 1], pairs first: log2(n) roundings a term.
template <int n>
__device__ __forceinline__ float sum_pairs(float *x)
{
#pragma unroll
    for (int w = n / 2; w > 0; w >>= 1)
#pragma unroll
        for (int i = 0; i < w; ++i) x[i] += x[i + w];
    return x[0];
}

template <int kType>
__device__ __forceinline__ float element(const typename Elems<kType>::type *p)
{
    if (kType == WF_F32) return *(const float *)p;
    const uint32_t h = *(const uint16_t *)p;
    return kType == WF_F16 ? __half2float(__ushort_as_half((unsigned short)h)) : __uint_as_float(h << 16);
}

struct SelectArgs {
    wf_beam in;
    wf_beam_out out;
    int row_lines, unit_lines, row_units;
    int group_units;        // a search's units, and up to three more: a multiple of 16 bytes
    int ctas;               // of a search
    bool live_rows;         // the warps share the search's live rows, else all
    uint32_t unit_magic;    // i / row_units = (i * unit_magic) >> 32 for the units of a search
    int most_of_row;        // warps of a row, at most: each has the lines that it loads at once
    int parts;              // places for parts of a search
    float4 *part;           // [groups][parts] {reference, sum of exponentials, maximum}
    float *most;            // [groups][group_units] the units' maxima, a row's row_units side by side
    uint32_t *ticket;       // [groups]
};

__device__ __forceinline__ bool live_score(float s) { return s > -INFINITY; }  // neither -inf nor NaN

// A row's tokens; its first vector, on a 16-byte boundary, starts `lead` elements before them.
template <int kType>
__device__ __forceinline__ const typename Elems<kType>::type *row_base(const SelectArgs &a, int row, int &lead)
{
    const uint8_t *p = (const uint8_t *)a.in.logits + (int64_t)row * a.in.logits_stride;
    lead = (int)(((uintptr_t)p & 15) / sizeof(typename Elems<kType>::type));
    return (const typename Elems<kType>::type *)p;
}

// A vector that lies in its row in part, or not at all: masked where there is no token.
template <int kType>
__device__ __noinline__ uint4 load_edge(const typename Elems<kType>::type *base, int t0, int V)
{
    using E = Elems<kType>;
    uint32_t w[4] = {E::masked(), E::masked(), E::masked(), E::masked()};
#pragma unroll
    for (int e = 0; e < E::n; ++e) {
        if (t0 + e < 0 || t0 + e >= V) continue;
        if (E::n == 4) {
            w[e & 3] = ((const uint32_t *)base)[t0 + e];
        } else {
            const uint32_t h = ((const uint16_t *)base)[t0 + e];
            w[e >> 1] = e & 1 ? (w[e >> 1] & 0xFFFFu) | h << 16 : (w[e >> 1] & 0xFFFF0000u) | h;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float warp_max(float x)  // NaN passed over
{
    float y;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
    return y;
}

// Units [u0, u1) of a row, by one warp: their maxima and the sum of their
// exponentials.  kUnit: lines of a unit (1 or 2), or kStep for one or more
// steps.
template <int kType, int kUnit>
__device__ __forceinline__ void take_part(const SelectArgs &a, int row, int u0, int u1, float4 *part, float *most)
{
    using E = Elems<kType>;
    constexpr int kLine = 32 * E::n;
    const int lane = threadIdx.x & 31, V = a.in.vocab, unit_lines = kUnit < kStep ? kUnit : a.unit_lines;
    int lead;
    const auto *base = row_base<kType>(a, row, lead);
    const int i0 = u0 * unit_lines, i1 = min(u1 * unit_lines, a.row_lines);
    // Lines of tokens only; the row's first and last may hold fewer.
    const int whole0 = lead ? 1 : 0, whole1 = min(i1, (V + lead) / kLine);
    const auto *mine = base + (lane * E::n - lead);
    const auto load = [&](uint4 (&v)[kStep], int i) {
        if (i >= whole0 && i + kStep <= whole1) {
#pragma unroll
            for (int u = 0; u < kStep; ++u) v[u] = __ldcs((const uint4 *)(mine + (int64_t)i * kLine + u * kLine));
        } else {
#pragma unroll
            for (int u = 0; u < kStep; ++u) {
                if (i + u >= whole0 && i + u < whole1) v[u] = __ldcs((const uint4 *)(mine + (int64_t)(i + u) * kLine));
                else if (i + u < i1) v[u] = load_edge<kType>(base, (i + u) * kLine + lane * E::n - lead, V);
                else v[u] = make_uint4(E::masked(), E::masked(), E::masked(), E::masked());
            }
        }
    };
    uint4 v[kStep], next[kStep];
    load(v, i0);
    // exp(x - ref) = 2^(x log2e - c), c = ref log2e rounded: one operation each; what the rounding shifts is known to
    // the join.  Where the part starts with a mask (-inf, or a value so low that the others would leave a float's
    // range), 0 is the reference.
    float first = -INFINITY;
#pragma unroll
    for (int u = 0; u < kStep; ++u) first = fmaxf(first, E::most(v[u]));
    first = warp_max(first);
    const float c = first > -80.0f && first < 1e4f ? first * kLog2e : 0.0f;
    // A term's way into the sum: 5 additions in its step (4 in 32 bits), kSum of steps, the compensated sum over those.
    Sum sum;
    float all = -INFINITY, unit = -INFINITY;
    int left = unit_lines;
    for (int i = i0; i < i1;) {
        float steps = 0;
        const int until = min(i1, i + kSum * kStep);
#pragma unroll 1
        for (; i < until; i += kStep) {
            load(next, i + kStep);
            float top[kStep], line[kStep];
#pragma unroll
            for (int u = 0; u < kStep; ++u) {
                float x[E::n];
                E::get(v[u], x);
#pragma unroll
                for (int e = 0; e < E::n; ++e) x[e] = exp2_fast(fmaf(x[e], kLog2e, -c));
                line[u] = sum_pairs<E::n>(x);
                top[u] = E::most(v[u]);
                v[u] = next[u];
            }
            steps += sum_pairs<kStep>(line);
            if (kUnit < kStep) {
                constexpr int kHere = kStep / kUnit;  // units of a step
                float put = -INFINITY;
#pragma unroll
                for (int u = 0; u < kHere; ++u) {
                    float x = top[u * kUnit];
                    if (kUnit == 2) x = fmaxf(x, top[u * kUnit + 1]);
                    x = warp_max(x);
                    all = fmaxf(all, x);
                    put = lane == u ? x : put;
                }
                if (lane < kHere && i + lane * kUnit < i1) most[(i - i0) / kUnit + lane] = put;
            } else {
#pragma unroll
                for (int u = 0; u < kStep; ++u) unit = fmaxf(unit, top[u]);
                left -= kStep;
                if (left == 0 || i + kStep >= i1) {
                    unit = warp_max(unit);
                    if (lane == 0) *most = unit;
                    ++most;
                    all = fmaxf(all, unit);
                    unit = -INFINITY;
                    left = unit_lines;
                }
            }
        }
        sum.add(steps);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum.s += __shfl_xor_sync(kFull, sum.s, o);
    if (lane == 0) *part = make_float4(c, sum.s, all, 0.0f);
}

// The beam of a search's unit.
__device__ __forceinline__ int unit_beam(const SelectArgs &a, int i) { return a.row_units == 1 ? i : (int)__umulhi((uint32_t)i, a.unit_magic); }

// How a search's warps share `rows` of its rows.
template <int kThreads>
__device__ __forceinline__ Share share_rows(const SelectArgs &a, int rows)
{
    constexpr int kWarps = kThreads / 32;
    const int of_row = min(max(1, a.ctas * kWarps / max(rows, 1)), a.most_of_row);
    return {of_row, (a.row_units + of_row - 1) / of_row};
}

// The rows' maxima, log Z and scores, to sm.stat, and the units' maxima, to sm.unit.
template <int kType, int kThreads>
__device__ __forceinline__ void row_stats(const SelectArgs &a, Shared<kThreads> &sm, int group)
{
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, K = a.in.beams, V = a.in.vocab;
    if (tid == 0) { sm.again = 0; sm.count = 0; sm.n_aside = 0; }
    constexpr int kLoads = 4;  // parts that a lane loads at once
    const float4 none = make_float4(0.0f, 0.0f, -INFINITY, 0.0f), *parts = a.part + (int64_t)group * a.parts;
    const uint32_t live = sm.live;
    const Share share = sm.share;
    const int n_parts = (a.row_units + share.units - 1) / share.units;  // of a row
    const auto parts_of = [&](int k) {
        const int j = a.live_rows ? __popc(live & ((1u << k) - 1u)) : k;
        return live >> k & 1u ? make_int2(j * share.of_row, n_parts) : make_int2(0, 0);
    };
    // The first of them before the units' maxima, so that both are under way together.
    int2 at = warp < K ? parts_of(warp) : make_int2(0, 0);  // {first, count}
    float4 q[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) q[u] = lane + 32 * u < at.y ? __ldcg(&parts[at.x + lane + 32 * u]) : none;
    const int units = K * a.row_units;
    const float *most = a.most + (int64_t)group * a.group_units;
    for (int i = 4 * tid; i < units; i += 4 * kThreads)  // (all under way together: 0.2 to 0.5 us less than loads in fours)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(&sm.unit[i])), "l"(most + i) : "memory");
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
#pragma unroll 1
    for (int k = warp; k < K; k += kWarps) {
        if (k != warp) {
            at = parts_of(k);
#pragma unroll
            for (int u = 0; u < kLoads; ++u) q[u] = lane + 32 * u < at.y ? __ldcg(&parts[at.x + lane + 32 * u]) : none;
        }
        // Each lane's parts by their own maximum, then the lanes' by the row's.
        float m = -INFINITY, z = 0, doubt = -INFINITY;
#pragma unroll 1
        for (int p = lane; p < at.y; p += 32) {
            const float4 now = q[0];
            if (now.z > m) {
                z = m > -INFINITY ? z * exp2f((m - now.z) * kLog2e) : 0.0f;
                m = now.z;
            }
            // With 0 as the reference, a small sum may lack what fell below the smallest number.
            if (now.x == 0.0f && !(now.y > 1e-20f)) doubt = fmaxf(doubt, now.z);
            else z += now.y * exp2f(fmaf(-m, kLog2e, now.x));
#pragma unroll
            for (int u = 0; u + 1 < kLoads; ++u) q[u] = q[u + 1];
            q[kLoads - 1] = p + 32 * kLoads < at.y ? __ldcg(&parts[at.x + p + 32 * kLoads]) : none;
        }
        const float most_of = warp_max(m);
        if (m < most_of) z = m > -INFINITY ? z * exp2f((m - most_of) * kLog2e) : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(kFull, z, o);
        doubt = warp_max(doubt);
        if (lane == 0) {
            sm.stat[k] = make_float4(most_of, logf(z), sm.score[k], 0.0f);  // (an empty beam: a maximum of -inf)
            // The maximum alone gives Z = 1.  What a doubtful part lacks is nothing beside that if its maximum lies far below.
            if (most_of > -INFINITY && (!(z >= 0.5f && z < INFINITY) || doubt >= most_of - 60.0f)) atomicOr(&sm.again, 1u << k);
        }
    }
    __syncthreads();
    // Summed again, in the order of the tokens: rows with infinities, NaN or sums that left a float's range; and rows
    // that may be equal to another (same score and maximum) if that one is summed again, or if their sums are near each
    // other but not the same: where the rows' places in their 16 bytes differ, so do their parts' references and sums.
    uint32_t rows = sm.again;
    {
        // Each with every other, by rotation (a matching instruction takes longer for values that all differ).
        const float4 stat = sm.stat[lane < K ? lane : 0];
        const uint32_t mark = __float_as_uint(stat.z + 0.0f) * 0x9E3779B1u ^ __float_as_uint(stat.x + 0.0f);  // (-0 is 0)
        const float y = rows >> lane & 1u ? NAN : stat.y;  // (a row that is summed again takes its equals along)
        bool off = false;
#pragma unroll 1
        for (int d = 1; d < K; ++d) {
            const int from = lane + d < K ? lane + d : lane + d - K;
            const uint32_t its = __shfl_sync(kFull, mark, from);
            const float z = __shfl_sync(kFull, y, from);
            off |= its == mark && z != y && !(fabsf(z - y) >= 1e-3f);
        }
        rows |= __ballot_sync(kFull, off && lane < K && stat.x > -INFINITY);
    }
#pragma unroll 1
    for (; rows; rows &= rows - 1) {
        const int k = __ffs((int)rows) - 1;
        int lead;
        const auto *base = row_base<kType>(a, group * K + k, lead);
        const float m = sm.stat[k].x;
        Sum sum;
        for (int t0 = tid; t0 < V; t0 += 8 * kThreads) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = t0 + u * kThreads < V ? element<kType>(base + t0 + u * kThreads) : -INFINITY;
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = x[u] == m ? 1.0f : x[u] > -INFINITY ? exp2f((x[u] - m) * kLog2e) : 0.0f;
            sum.add(sum_pairs<8>(x));  // (up to 65,536 logits a thread)
        }
        float s = sum.s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
        if (lane == 0) sm.sum[warp] = s;
        __syncthreads();
        if (tid == 0) {
            float z = 0;
            for (int w = 0; w < kWarps; ++w) z += sm.sum[w];
            sm.stat[k].y = logf(z);
        }
        __syncthreads();
    }
}

// The sum of a logit of a beam.
__device__ __forceinline__ float sum_of(const float4 &stat, float x) { return stat.z + ((x == stat.x ? 0.0f : x - stat.x) - stat.y); }

// Its key: {0, 0} if it is no candidate.
template <int kThreads>
__device__ __forceinline__ Key key_of(const Shared<kThreads> &sm, int k, float x, uint32_t place)
{
    const float4 stat = sm.stat[k];
    const float sum = sum_of(stat, x);
    if (!(stat.x > -INFINITY) || !(x > -INFINITY) || !(sum > -INFINITY)) return {0, 0};
    return {(uint64_t)order_of(sum) << 32 | (uint32_t)~k, (uint64_t)order_of(x) << 32 | (uint32_t)~place};
}

// Item l of the picked units, kLines lines of one: the row's tokens, this
// lane's first token, its beam, and how many of the lines there are.
template <int kType, int kLines, int kThreads>
__device__ __forceinline__ const typename Elems<kType>::type *picked_lines(const SelectArgs &a, const Shared<kThreads> &sm, int group, int l,
                                                                           int &k, int &t0, int &lines)
{
    const int items = kLines < kStep ? 1 : a.unit_lines / kStep, j = items == 1 ? l : l / items;
    const int unit = sm.pick[j];
    k = unit_beam(a, unit);
    const int i = (unit - k * a.row_units) * a.unit_lines + (l - j * items) * kLines;
    lines = min(kLines, a.row_lines - i);
    int lead;
    const auto *base = row_base<kType>(a, group * a.in.beams + k, lead);
    t0 = (i * 32 + (int)(threadIdx.x & 31)) * Elems<kType>::n - lead;
    return base;
}

// A load without a branch around it, so that several stay in flight.
__device__ __forceinline__ void load_if(bool ok, const void *from, uint4 &v)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %4, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%5];\n\t}"
                 : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w) : "r"((int)ok), "l"(from));
}

// Calls f(beam, logit, token) for this lane's share of the picked units; a
// warp takes every kWarps-th of their items.
template <int kType, int kLines, int kThreads, class F>
__device__ __forceinline__ void each_token(const SelectArgs &a, const Shared<kThreads> &sm, int group, int items, const F &f)
{
    using E = Elems<kType>;
    constexpr int kWarps = kThreads / 32;
    for (int l = (int)threadIdx.x >> 5; l < items; l += kWarps) {
        int k, t0, lines;
        const auto *base = picked_lines<kType, kLines>(a, sm, group, l, k, t0, lines);
        for (int u = 0; u < lines; ++u, t0 += 32 * E::n) {
            float x[E::n];
            E::get(t0 >= 0 && t0 + E::n <= a.in.vocab ? *(const uint4 *)(base + t0) : load_edge<kType>(base, t0, a.in.vocab), x);
#pragma unroll
            for (int e = 0; e < E::n; ++e) f(k, x[e], (uint32_t)(t0 + e));
        }
    }
}

template <int kType, int kLines, int kThreads>
__device__ __forceinline__ void join(const SelectArgs &a, Shared<kThreads> &sm, int group)
{
    using E = Elems<kType>;
    constexpr int kWarps = kThreads / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.in.keep, units = a.in.beams * a.row_units;
    const float *most = a.most + (int64_t)group * a.group_units;
    row_stats<kType>(a, sm, group);
    // The bound, and the units that reach it.
    float top = -INFINITY;
#pragma unroll 4
    for (int i = tid; i < units; i += kThreads) {
        const float4 stat = sm.stat[unit_beam(a, i)];
        const float x = sm.unit[i], sum = stat.x > -INFINITY && x > -INFINITY ? sum_of(stat, x) : -INFINITY;
        sm.unit[i] = sum;
        top = fmaxf(top, sum);
    }
    sm.most[warp][lane] = top;
    __syncthreads();
    if (warp == 0) {
        float even = sm.most[0][lane], odd = sm.most[1][lane];
#pragma unroll
        for (int w = 2; w < kWarps; w += 2) {
            even = fmaxf(even, sm.most[w][lane]);
            odd = fmaxf(odd, sm.most[w + 1][lane]);
        }
        // The n-th largest of 32 classes; of 64 (the 32 largest of two sorted halves) from n = 17 on, the least of
        // those beyond 32.
        float sorted = warp_sorted(n <= 16 ? fmaxf(even, odd) : n <= 32 ? even : fminf(even, odd));
        if (n > 16 && n <= 32) sorted = warp_sorted(fmaxf(sorted, __shfl_sync(kFull, warp_sorted(odd), 31 - lane)));
        if (lane == min(n, 32) - 1) sm.cut = fmaxf(sorted, -3.402823466e38f);  // (a sum of -inf is no candidate)
    }
    __syncthreads();
    float cut = sm.cut;
    for (int i = tid; i < units; i += kThreads) {
        if (!(sm.unit[i] >= cut)) continue;
        const uint32_t at = atomicAdd(&sm.count, 1u);
        if (at < kCap) sm.pick[at] = i;
    }
    __syncthreads();
    int picked = (int)sm.count;
    if (picked > kPick && picked <= kCap) {
        // A loose bound (the least of 64 classes, for more than 32): the n-th largest of these sums is the bound.
        int mine[kCap / kThreads];
        bool keep[kCap / kThreads];
        float least = INFINITY;
#pragma unroll
        for (int u = 0; u < kCap / kThreads; ++u) {
            const int j = tid + u * kThreads;
            keep[u] = false;
            if (j >= picked) continue;
            mine[u] = sm.pick[j];
            const float sum = sm.unit[mine[u]];
            int ahead = 0;
#pragma unroll 4
            for (int i = 0; i < picked; ++i) ahead += sm.unit[sm.pick[i]] > sum;
            keep[u] = ahead < n;  // (equal sums stay together)
            if (keep[u]) least = fminf(least, sum);
        }
        __syncthreads();
        if (tid == 0) sm.count = 0;
        least = -warp_max(-least);
        if (lane == 0) sm.sum[warp] = least;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) least = fminf(least, sm.sum[w]);
#pragma unroll
        for (int u = 0; u < kCap / kThreads; ++u)
            if (keep[u]) sm.pick[atomicAdd(&sm.count, 1u)] = mine[u];
        __syncthreads();
        picked = (int)sm.count;
        cut = least;
    }
    if (picked > kPick) {  // many equal, or a loose bound for many: exactly the n best
        best_keys(sm, n, [&](auto f) {
            for (int i = tid; i < units; i += kThreads) {
                const int k = unit_beam(a, i);
                f(key_of(sm, k, __ldcg(&most[i]), (uint32_t)(i - k * a.row_units)));
            }
        });
        picked = 0;
        while (picked < n && sm.sorted[picked].hi) ++picked;
        if (tid < picked) sm.pick[tid] = (int)~(uint32_t)sm.sorted[tid].hi * a.row_units + (int)~(uint32_t)sm.sorted[tid].lo;
        if (picked == n) cut = value_of((uint32_t)(sm.sorted[n - 1].hi >> 32));
    }
    __syncthreads();
    if (tid == 0) sm.count = 0;
    // Their vectors that reach the bound, kBatch lines of a warp at once; then those vectors' candidates; those in order.
    constexpr int kBatch = kThreads == kSmall ? 8 : 4, kItems = kBatch / kLines;
    const int items = picked * (kLines < kStep ? 1 : a.unit_lines / kStep);
    for (int l0 = warp; l0 < items; l0 += kItems * kWarps) {
        uint4 v[kBatch];
        int k[kItems], t0[kItems], lines[kItems];
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            const int l = l0 + j * kWarps;
            const auto *base = picked_lines<kType, kLines>(a, sm, group, min(l, items - 1), k[j], t0[j], lines[j]);
            if (l >= items) lines[j] = 0;
#pragma unroll
            for (int u = 0; u < kLines; ++u) {
                const int t = t0[j] + u * 32 * E::n;
                v[j * kLines + u] = make_uint4(E::masked(), E::masked(), E::masked(), E::masked());
                load_if(u < lines[j] && t >= 0 && t + E::n <= a.in.vocab, base + t, v[j * kLines + u]);
            }
        }
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            const float4 stat = sm.stat[k[j]];
#pragma unroll
            for (int u = 0; u < kLines; ++u) {
                const int t = t0[j] + u * 32 * E::n;
                uint4 &w = v[j * kLines + u];
                int lead;
                if (u < lines[j] && t < a.in.vocab && (t < 0 || t + E::n > a.in.vocab))  // a row's end
                    w = load_edge<kType>(row_base<kType>(a, group * a.in.beams + k[j], lead), t, a.in.vocab);
                const float x = E::most(w);
                if (!(x > -INFINITY) || !(sum_of(stat, x) >= cut)) continue;
                const uint32_t at = atomicAdd(&sm.n_aside, 1u);
                if (at < kCap) { sm.aside[at] = w; sm.aside_of[at] = make_int2(k[j], t); }
            }
        }
    }
    __syncthreads();
    const int aside = (int)sm.n_aside;
    for (int i = tid; i < min(aside, kCap) * E::n; i += kThreads) {
        const float x = element<kType>((const typename E::type *)sm.aside + i);
        const int2 of = sm.aside_of[i / E::n];
        if (!(x > -INFINITY) || !(sum_of(sm.stat[of.x], x) >= cut)) continue;
        const uint32_t at = atomicAdd(&sm.count, 1u);
        if (at < kCap) sm.got[at] = key_of(sm, of.x, x, (uint32_t)(of.y + i % E::n));
    }
    __syncthreads();
    const int count = (int)sm.count;
    if (aside <= kCap && count <= kCap)
        rank_keys(sm, count, n);
    else
        best_keys(sm, n, [&](auto f) {
            each_token<kType, kLines>(a, sm, group, items, [&](int k, float x, uint32_t token) { f(key_of(sm, k, x, token)); });
        });
}

// A search's outputs, from sm.sorted, by warp 0.
template <int kThreads>
__device__ void write_group(const SelectArgs &a, const Shared<kThreads> &sm, int group)
{
    const int lane = threadIdx.x, n = a.in.keep, K = a.in.beams;
    const int64_t out = (int64_t)group * n, next = (int64_t)group * K;
    int put = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane;
        const Key key = i < n ? sm.sorted[i] : Key{0, 0};
        const float score = key.hi ? value_of((uint32_t)(key.hi >> 32)) : -INFINITY;
        const int32_t parent = key.hi ? group * K + (int32_t)~(uint32_t)key.hi : -1, token = key.hi ? (int32_t)~(uint32_t)key.lo : -1;
        if (i < n) {
            a.out.score[out + i] = score;
            a.out.parent[out + i] = parent;
            a.out.token[out + i] = token;
        }
        const bool goes = key.hi && token != a.in.eos;
        const uint32_t mask = __ballot_sync(kFull, goes);
        const int at = put + __popc(mask & ((1u << lane) - 1u));
        if (a.out.next_score && goes && at < K) {
            a.out.next_score[next + at] = score;
            a.out.next_parent[next + at] = parent;
            a.out.next_token[next + at] = token;
        }
        put += __popc(mask);
    }
    if (a.out.next_score && put + lane < K) {  // (K is at most 32)
        a.out.next_score[next + put + lane] = -INFINITY;
        a.out.next_parent[next + put + lane] = -1;
        a.out.next_token[next + put + lane] = -1;
    }
}

// Arrival of one CTA; true for the last of n, which resets the count.  The
// barrier hands what the CTA has written to the thread that makes it known
// to the others.
template <int kThreads>
__device__ __forceinline__ bool last_arrival(Shared<kThreads> &sm, uint32_t *ticket, uint32_t n)
{
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        sm.last = atomicAdd(ticket, 1u) == n - 1;
        if (sm.last) *ticket = 0;
        __threadfence();
    }
    __syncthreads();
    return sm.last;
}

template <int kType, int kUnit, int kThreads>
__global__ void __launch_bounds__(kThreads, per_sm(kThreads)) select_kernel(const __grid_constant__ SelectArgs a)
{
    constexpr int kWarps = kThreads / 32;
    __shared__ Shared<kThreads> sm;
    const int lane = threadIdx.x & 31, warp = (int)threadIdx.x >> 5, K = a.in.beams;
    const int group = (int)blockIdx.x / a.ctas, w = ((int)blockIdx.x % a.ctas) * kWarps + warp;
    const float score = lane < K ? a.in.score[group * K + lane] : -INFINITY;
    // With few units a warp the rows are shared out as they are, so that no load waits for the scores; with many, the
    // live ones are: a search's first step has one.
    uint32_t live = kFull;
    int rows = K;
    if (a.live_rows) {
        live = __ballot_sync(kFull, live_score(score));
        rows = __popc(live);
    }
    const Share share = share_rows<kThreads>(a, rows);
    float4 *parts = a.part + (int64_t)group * a.parts;
    float *most = a.most + (int64_t)group * a.group_units;
    const int u0 = share.of_row > 1 ? w % share.of_row * share.units : 0, u1 = min(u0 + share.units, a.row_units);
    for (int j = share.of_row > 1 ? w / share.of_row : w; j < rows && u0 < u1; j += a.ctas * kWarps) {
        const int k = a.live_rows ? (int)__fns(live, 0, j + 1) : j;
        take_part<kType, kUnit>(a, group * K + k, u0, u1, &parts[share.of_row > 1 ? w : j], most + k * a.row_units + u0);
    }
    if (warp == 0) {
        sm.score[lane] = score;
        live = __ballot_sync(kFull, live_score(score));
        if (lane == 0) { sm.live = live; sm.share = share; }
    }
    if (!last_arrival(sm, &a.ticket[group], (uint32_t)a.ctas)) return;
    join<kType, kUnit>(a, sm, group);
    if (warp == 0) write_group(a, sm, group);
}

// How the rows are cut.  CTAs: a search has its own, so that none is the last
// of two; no more in all than the machine holds at once (300 searches of 4
// beams over 32,000 tokens take 23 us on 300 CTAs, 29 on 600).  Warps: as many
// a row as that gives, rounded down (parts to be taken in two or three turns,
// which would leave fewer warps idle, cost 0.3 to 1 us more).  Units: a line
// where a warp has few; two where it has at least kLong and four from kLonger
// on, for half and a quarter of the reductions (four for two: 400 searches of 4
// over 32,000 26.8 -> 26.2 us, 64 of 5 over 100,000 20.7 -> 20.1, but 40 of 8
// over 131,072 24.3 -> 24.7); more where a search would have more than kUnits.
constexpr int kLong = 8, kLonger = 32;
// CTAs of 512 threads where every search has an SM and the logits are at most
// kShort lines (33 MB): twice the warps for the join, half the parts to join.
// us of 256 threads -> of 512: one search of 4 beams over 32,000 tokens 9.0 ->
// 8.6, 16 of 4 over 50,257 12.1 -> 10.5, 16 of 12 over 60,000 17.7 -> 15.1, one
// of 32 over 131,072 35.6 -> 25.3, 128 of 4 over 32,000 16.0 -> 15.2 (100 such
// 14.1 -> 14.6).  With more logits the fewer bytes in flight weigh more: 64 of
// 8 over 50,257 20.4 -> 20.2, 64 of 5 over 100,000 20.9 -> 22.4, 40 of 8 over
// 131,072 24.5 -> 26.5, 64 of 8 32.5 -> 35.9.
constexpr int64_t kShort = 65536;

bool deal(SelectArgs &a, int es, int sms, int &threads)
{
    const int64_t per = 16 / es, K = a.in.beams, groups = a.in.groups, rows = K * groups;
    const int64_t vectors = (a.in.vocab + 2 * (per - 1)) / per;  // a row may start inside a vector
    const int64_t row_lines = (vectors + 31) / 32, lines = K * row_lines;
    threads = groups <= sms && rows * row_lines <= kShort ? kBig : kSmall;
    const int64_t most = (int64_t)sms * per_sm(threads), kWarps = threads / 32;
    int64_t ctas = std::max<int64_t>(1, most / groups);
    const int64_t of_warp = lines / (ctas * kWarps);
    int64_t unit = std::max<int64_t>(of_warp >= kLonger ? 4 : of_warp >= kLong ? 2 : 1, (lines + kUnits - 1) / kUnits);
    if (unit > 2) unit = (unit + kStep - 1) / kStep * kStep;
    while (K * ((row_lines + unit - 1) / unit) > kUnits) unit = unit < kStep ? 2 * unit : unit + kStep;
    const int64_t row_units = (row_lines + unit - 1) / unit;
    // The warps that the rows, each cut alike, have a use for.
    const int64_t most_of_row = (row_lines + kStep - 1) / kStep;
    const int64_t of_row = std::min(std::max<int64_t>(1, ctas * kWarps / K), most_of_row), warp_units = (row_units + of_row - 1) / of_row;
    if (of_row == most_of_row || of_row > 1) ctas = std::min(ctas, (K * ((row_units + warp_units - 1) / warp_units) + kWarps - 1) / kWarps);
    a.row_lines = (int)row_lines;
    a.unit_lines = (int)unit;
    a.row_units = (int)row_units;
    a.group_units = (int)((K * row_units + 3) / 4 * 4);
    a.ctas = (int)ctas;
    a.most_of_row = (int)most_of_row;
    a.parts = (int)std::max<int64_t>(ctas * kWarps, K);
    a.live_rows = warp_units * unit >= kLong;
    // i * (2^32 / row_units, rounded up) is off by less than 1 / row_units for the units of a search, kUnits at most.
    a.unit_magic = (uint32_t)(((1ull << 32) + (uint64_t)row_units - 1) / (uint64_t)row_units);  // (row_units = 1: not used)
    return groups * a.ctas < INT32_MAX;
}

template <int kType, int kThreads>
int launch(const SelectArgs &a, cudaStream_t st)
{
    const unsigned ctas = (unsigned)(a.in.groups * a.ctas);
    if (a.unit_lines == 1) select_kernel<kType, 1, kThreads><<<ctas, kThreads, 0, st>>>(a);
    else if (a.unit_lines == 2) select_kernel<kType, 2, kThreads><<<ctas, kThreads, 0, st>>>(a);
    else select_kernel<kType, kStep, kThreads><<<ctas, kThreads, 0, st>>>(a);
    return wf_cuda_check(cudaGetLastError(), "select launch");
}

template <int kType>
int launch(const SelectArgs &a, int threads, cudaStream_t st)
{
    return threads == kSmall ? launch<kType, kSmall>(a, st) : launch<kType, kBig>(a, st);
}

}  // namespace

// Scratch of any call of at most these sizes.  Parts: a search's warps, or its
// rows; the searches' CTAs are at most what the machine holds of either size, or
// one each.  Units: a row's lines, or all that a search may have; up to three more a search.
void wf_beam_scratch(int64_t rows, int64_t vocab, int sms, int64_t *parts, int64_t *units)
{
    *parts = std::max({(int64_t)sms * per_sm(kSmall) * (kSmall / 32), rows * (kSmall / 32), (int64_t)sms * per_sm(kBig) * (kBig / 32)});
    *units = rows * (std::min<int64_t>((vocab + 6) / 128 + 1, kUnits) + 3);
}

int wf_launch_select(wf_decode *d, const wf_beam *in, const wf_beam_out *out, cudaStream_t st)
{
    SelectArgs a;
    a.in = *in;
    a.out = *out;
    int threads;
    const bool ok = deal(a, in->dtype == WF_F32 ? 4 : 2, d->sms, threads);
    a.part = d->part;
    a.most = d->most;
    a.ticket = d->ticket + 1;
    const int64_t parts = (int64_t)in->groups * a.parts;
    const int64_t units = (int64_t)in->groups * a.group_units;
    if (!ok || parts > d->parts || units > d->units)
        return wf_set_error(WF_EINVAL, "wf_beam_select: %lld parts and %lld units exceed the scratch", (long long)parts, (long long)units);
    if (in->dtype == WF_F32) return launch<WF_F32>(a, threads, st);
    if (in->dtype == WF_F16) return launch<WF_F16>(a, threads, st);
    return launch<WF_BF16>(a, threads, st);
}
