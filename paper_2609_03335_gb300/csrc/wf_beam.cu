// Beam search's selection over beams and vocabulary (wf_beam_select).
//
// A candidate's sum is score + (x - m) - log Z, with a row's maximum m and
// Z = sum of exp(x - m).  Within a row the order of the sums is that of the
// logits, so the row's `keep` best logits can be found in the pass that makes
// m and Z, before either is known:
//
//   1. a CTA takes a chunk of a row into registers (one read of the logits),
//      makes the chunk's maximum and sum of exponentials, and lists the
//      chunk's `keep` best logits;
//   2. the last CTA of a row joins its chunks: m, Z, the row's best;
//   3. the last CTA of a search joins its rows by their sums.
//
// All in one launch.  A list of the best n of many: the threads' own maxima,
// taken over 32 or 64 classes of threads, have a n-th largest; at least n
// values reach it and few more do (the classes hold interleaved values, so the
// n-th largest of their maxima is near the n-th largest of all).  Those are gathered
// and ranked by comparing each with all.  Where many values are equal (a mask of
// the type's lowest value) the gathering repeats with 64-bit keys that order
// equal values by their place, and where even that gathers too many the n-th
// largest key is found bit by bit.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "wf_decode.cuh"

namespace {

constexpr uint32_t kFull = 0xFFFFFFFFu;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCap = 512;      // values gathered before they are ranked
constexpr float kLog2e = 1.4426950408889634f;

// Whole numbers in the order of the floats; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }

// A key: the value's order above the complement of its place, so that the
// larger key is the larger value, of equal ones the first.  0: no value.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t place) { return (uint64_t)order_of(x) << 32 | (uint32_t)~place; }
__device__ __forceinline__ uint32_t place_of(uint64_t key) { return ~(uint32_t)key; }
__device__ __forceinline__ float value_of_key(uint64_t key) { return value_of((uint32_t)(key >> 32)); }

// The warp's values in descending order, lane 0 the largest.
template <class T>
__device__ __forceinline__ T warp_sorted(T v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int o = size >> 1; o > 0; o >>= 1) {
            const T w = __shfl_xor_sync(kFull, v, o);
            const bool first = (lane & o) == 0, down = size == 32 || (lane & size) == 0;
            v = first == down ? (v > w ? v : w) : (v > w ? w : v);
        }
    return v;
}

struct Shared {
    union {
        float f[kWarps][32];
        uint64_t k[kWarps][32];
    } best;                   // the threads' largest values
    uint64_t got[kCap];       // gathered keys
    uint64_t sorted[kMaxKeep];
    uint32_t count;
    uint32_t tally;
    float sum[kWarps];
    float2 stat[kMaxGroup];
    bool last;
};

// A value that at least n of the CTA's values reach (the lowest one, if there
// are fewer): v is each thread's largest.  top: the largest of all.
template <class T>
__device__ __forceinline__ T reached(T v, T (*best)[32], int n, T &top)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    best[warp][lane] = v;
    __syncthreads();
    T even = best[0][lane], odd = best[1][lane];
#pragma unroll
    for (int w = 2; w < kWarps; w += 2) {
        const T x = best[w][lane], y = best[w + 1][lane];
        even = x > even ? x : even;
        odd = y > odd ? y : odd;
    }
    const T both = warp_sorted(even > odd ? even : odd);
    top = __shfl_sync(kFull, both, 0);
    if (n <= 32) return __shfl_sync(kFull, both, n - 1);
    const T least = warp_sorted(even > odd ? odd : even);
    return __shfl_sync(kFull, least, 31);
}

// Ranks sm.got[0, count) and leaves the n largest keys, in order, in
// sm.sorted; what is missing is 0.
__device__ void rank_keys(Shared &sm, int count, int n)
{
    for (int i = threadIdx.x; i < n; i += kThreads) sm.sorted[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const uint64_t key = sm.got[i];
        int ahead = 0;
        for (int j = 0; j < count; ++j) ahead += sm.got[j] > key;
        if (ahead < n) sm.sorted[ahead] = key;
    }
    __syncthreads();
}

// Gathers the CTA's keys that are at least t (0 is no key); each(f) calls f
// with every key of this thread.  Returns how many there are; no more than
// kCap are kept.
template <class Each>
__device__ __forceinline__ int gather(Shared &sm, const Each &each, uint64_t t)
{
    if (threadIdx.x == 0) sm.count = 0;
    __syncthreads();
    each([&](uint64_t key) {
        if (key >= t && key) {
            const uint32_t at = atomicAdd(&sm.count, 1u);
            if (at < kCap) sm.got[at] = key;
        }
    });
    __syncthreads();
    return (int)sm.count;
}

// The n largest of the CTA's keys, in order, in sm.sorted.
template <class Each>
__device__ void best_keys(Shared &sm, const Each &each, int n)
{
    uint64_t mine = 0, top;
    each([&](uint64_t key) { mine = key > mine ? key : mine; });
    __syncthreads();
    uint64_t t = reached(mine, sm.best.k, n, top);
    int count = gather(sm, each, t);
    if (count > kCap) {
        // Bit by bit: the largest key that n keys reach.
        t = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t cand = t | 1ull << bit;
            uint32_t c = 0;
            each([&](uint64_t key) { c += key >= cand; });
            c = __reduce_add_sync(kFull, c);
            __syncthreads();
            if (threadIdx.x == 0) sm.tally = 0;
            __syncthreads();
            if ((threadIdx.x & 31) == 0) atomicAdd(&sm.tally, c);
            __syncthreads();
            if (sm.tally >= (uint32_t)n) t = cand;
        }
        count = gather(sm, each, t);
    }
    rank_keys(sm, count, n);
}

// Arrival of one CTA; true for the last of n, which resets the count.
__device__ __forceinline__ bool last_arrival(Shared &sm, uint32_t *ticket, uint32_t n)
{
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        sm.last = atomicAdd(ticket, 1u) == n - 1;
        if (sm.last) *ticket = 0;
    }
    __syncthreads();
    if (sm.last) __threadfence();
    return sm.last;
}

// The elements of a 16-byte vector as floats.
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
    static __device__ __forceinline__ uint32_t lowest() { return 0xFF800000u; }  // -inf
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
    static __device__ __forceinline__ uint32_t lowest() { return 0xFC00FC00u; }
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
    static __device__ __forceinline__ uint32_t lowest() { return 0xFF80FF80u; }
};

// 2^x, 0 below the smallest normal number.
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int kType>
__device__ __forceinline__ float element(const typename Elems<kType>::type *p)
{
    if (kType == WF_F32) return *(const float *)p;
    const uint32_t h = *(const uint16_t *)p;
    return kType == WF_F16 ? __half2float(__ushort_as_half((unsigned short)h)) : __uint_as_float(h << 16);
}

// The rare chunks, from memory once more (the registers of the common path
// stay few): its sum of exponentials with infinities, NaN or masks of the type's lowest value ...
template <int kType>
__device__ __noinline__ float chunk_sum(const typename Elems<kType>::type *base, int lo, int hi, float m)
{
    float s = 0;
    for (int t = lo + threadIdx.x; t < hi; t += kThreads) {
        const float x = element<kType>(base + t);
        s += x == m ? 1.0f : isnan(x) ? 0.0f : exp2f((x - m) * kLog2e);
    }
    return s;
}

// ... and its best where too many values reach the bound (equal values).
template <int kType>
__device__ __noinline__ void chunk_keys(Shared &sm, const typename Elems<kType>::type *base, int lo, int hi, int n)
{
    best_keys(sm, [&](auto f) {
        for (int t = lo + threadIdx.x; t < hi; t += kThreads) {
            const float x = element<kType>(base + t);
            f(x > -INFINITY ? key_of(x, (uint32_t)t) : 0ull);
        }
    }, n);
}

struct SelectArgs {
    wf_beam in;
    wf_beam_out out;
    int chunks;             // of a row
    float2 *part;
    uint64_t *list, *row_key;
    int32_t *row_token;
    uint32_t *row_ticket, *group_ticket;
};

__device__ __forceinline__ bool live_score(float s) { return s > -INFINITY; }  // neither -inf nor NaN

// Step 1: the chunk of kVecs vectors a thread.
template <int kType, int kVecs>
__device__ void chunk_best(const SelectArgs &a, Shared &sm, int row, int chunk)
{
    using E = Elems<kType>;
    using T = typename E::type;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.in.keep, V = a.in.vocab;
    const T *base = (const T *)((const uint8_t *)a.in.logits + (int64_t)row * a.in.logits_stride);
    // Vectors lie on 16-byte boundaries; element e of vector j is token j * E::n + e - lead.
    const int lead = (int)(((uintptr_t)base & 15) / sizeof(T));
    uint4 v[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int t0 = ((chunk * kVecs + i) * kThreads + tid) * E::n - lead;
        if (t0 >= 0 && t0 + E::n <= V) {
            v[i] = __ldcs((const uint4 *)(base + t0));
        } else {
            uint32_t w[4] = {E::lowest(), E::lowest(), E::lowest(), E::lowest()};
#pragma unroll
            for (int e = 0; e < E::n; ++e) {
                if (t0 + e < 0 || t0 + e >= V) continue;
                if (sizeof(T) == 4) {
                    w[e & 3] = ((const uint32_t *)base)[t0 + e];
                } else {
                    const uint32_t h = ((const uint16_t *)base)[t0 + e];
                    w[e >> 1] = e & 1 ? (w[e >> 1] & 0xFFFFu) | h << 16 : (w[e >> 1] & 0xFFFF0000u) | h;
                }
            }
            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    float mine = -INFINITY;  // fmaxf passes NaN over
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        float x[E::n];
        E::get(v[i], x);
#pragma unroll
        for (int e = 0; e < E::n; ++e) mine = fmaxf(mine, x[e]);
    }
    float m;
    const float t = reached(mine, sm.best.f, n, m);
    if (tid == 0) sm.count = 0;
    __syncthreads();
    // exp(x - m) = 2^(x log2e - c) * 2^(c - m log2e) with c = m log2e rounded: the first takes one operation, the second
    // is the same for all.
    const float c = m * kLog2e;
    const bool plain = fabsf(m) < 1e30f;
    const int t00 = (chunk * kVecs * kThreads + tid) * E::n - lead;
    float s = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        float x[E::n];
        E::get(v[i], x);
#pragma unroll
        for (int e = 0; e < E::n; ++e) {
            s += exp2_fast(fmaf(x[e], kLog2e, -c));
            if (x[e] >= t && x[e] > -INFINITY) {
                const uint32_t at = atomicAdd(&sm.count, 1u);
                if (at < kCap) sm.got[at] = key_of(x[e], (uint32_t)(t00 + i * kThreads * E::n + e));
            }
        }
    }
    s *= exp2f(-fmaf(m, kLog2e, -c));
    const int lo = max(chunk * kVecs * kThreads * E::n - lead, 0), hi = min((chunk + 1) * kVecs * kThreads * E::n - lead, V);
    // A NaN in one thread's values leaves its sum NaN; it then sums its share of the chunk's tokens again, so all do.
    if (__syncthreads_or(!plain || isnan(s))) s = m > -INFINITY ? chunk_sum<kType>(base, lo, hi, m) : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    if (lane == 0) sm.sum[warp] = s;
    __syncthreads();
    const int count = (int)sm.count;
    if (count > kCap) {  // many equal values
        chunk_keys<kType>(sm, base, lo, hi, n);
    } else {
        rank_keys(sm, count, n);
    }
    const int64_t at = (int64_t)row * a.chunks + chunk;
    for (int i = tid; i < n; i += kThreads) a.list[at * n + i] = sm.sorted[i];
    if (tid == 0) {
        float sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += sm.sum[w];
        a.part[at] = make_float2(m, sum);
    }
}

// Step 2: a row's maximum, log Z and best, from its chunks.
__device__ void row_best(const SelectArgs &a, Shared &sm, int row, float score)
{
    const int tid = threadIdx.x, n = a.in.keep, C = a.chunks;
    const int64_t at = (int64_t)row * C;
    if (tid < 32) {
        float m = -INFINITY, z = 0;
        for (int c = tid; c < C; c += 32) m = fmaxf(m, __ldcg(&a.part[at + c]).x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
        for (int c = tid; c < C; c += 32) {
            const float2 p = __ldcg(&a.part[at + c]);
            z += p.x == m ? p.y : p.y * exp2f((p.x - m) * kLog2e);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(kFull, z, o);
        if (tid == 0) sm.stat[0] = make_float2(m, logf(z));
    }
    // The lists' places interleave: neighbouring threads hold the same rank of neighbouring chunks.
    best_keys(sm, [&](auto f) {
        for (int i = tid; i < n * C; i += kThreads) f(__ldcg(&a.list[(at + i % C) * n + i / C]));
    }, n);
    const float2 stat = sm.stat[0];
    const int place0 = row % a.in.beams * n;
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t key = sm.sorted[i];
        uint64_t out = 0;
        if (key && live_score(score)) {
            const float x = value_of_key(key);
            const float sum = score + ((x == stat.x ? 0.0f : x - stat.x) - stat.y);
            if (sum > -INFINITY) out = key_of(sum, (uint32_t)(place0 + i));
        }
        a.row_key[(int64_t)row * n + i] = out;
        a.row_token[(int64_t)row * n + i] = (int32_t)place_of(key);
    }
}

// Step 3: a search's best and the next step's rows.
__device__ void group_best(const SelectArgs &a, Shared &sm, int group)
{
    const int tid = threadIdx.x, n = a.in.keep, K = a.in.beams;
    const int64_t first = (int64_t)group * K * n;
    best_keys(sm, [&](auto f) {
        for (int i = tid; i < n * K; i += kThreads) f(__ldcg(&a.row_key[first + (i % K) * n + i / K]));
    }, n);
    // Warp 0: two candidates a lane, `goes` those that do not end.
    if (tid >= 32) return;
    int put = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + tid;
        const uint64_t key = i < n ? sm.sorted[i] : 0;
        float score = -INFINITY;
        int32_t parent = -1, token = -1;
        if (key) {
            const uint32_t place = place_of(key);
            score = value_of_key(key);
            parent = group * K + (int32_t)(place / (uint32_t)n);
            token = __ldcg(&a.row_token[first + place]);
        }
        if (i < n) {
            a.out.score[(int64_t)group * n + i] = score;
            a.out.parent[(int64_t)group * n + i] = parent;
            a.out.token[(int64_t)group * n + i] = token;
        }
        const bool goes = key && token != a.in.eos;
        const uint32_t mask = __ballot_sync(kFull, goes);
        const int at = put + __popc(mask & ((1u << tid) - 1u));
        if (a.out.next_score && goes && at < K) {
            a.out.next_score[(int64_t)group * K + at] = score;
            a.out.next_parent[(int64_t)group * K + at] = parent;
            a.out.next_token[(int64_t)group * K + at] = token;
        }
        put += __popc(mask);
    }
    for (int at = put + tid; a.out.next_score && at < K; at += 32) {
        a.out.next_score[(int64_t)group * K + at] = -INFINITY;
        a.out.next_parent[(int64_t)group * K + at] = -1;
        a.out.next_token[(int64_t)group * K + at] = -1;
    }
}

template <int kType, int kVecs>
__global__ void __launch_bounds__(kThreads) select_kernel(SelectArgs a)
{
    __shared__ Shared sm;
    const int row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const float score = a.in.score[row];
    if (live_score(score)) {
        chunk_best<kType, kVecs>(a, sm, row, chunk);
    } else {  // an empty beam: nothing is read
        const int64_t at = (int64_t)row * a.chunks + chunk;
        for (int i = threadIdx.x; i < a.in.keep; i += kThreads) a.list[at * a.in.keep + i] = 0;
        if (threadIdx.x == 0) a.part[at] = make_float2(-INFINITY, 0.0f);
    }
    if (!last_arrival(sm, &a.row_ticket[row], (uint32_t)a.chunks)) return;
    row_best(a, sm, row, score);
    const int group = row / a.in.beams;
    if (!last_arrival(sm, &a.group_ticket[group], (uint32_t)a.in.beams)) return;
    group_best(a, sm, group);
}

constexpr int kMaxVecs = 8;
constexpr int64_t kFill = 304;  // CTAs that fill the machine (two an SM)

int chunks_of(int64_t vocab, int es, int vecs)
{
    const int64_t per = 16 / es, vectors = (vocab + 2 * (per - 1)) / per;  // a row may start inside a vector
    return (int)((vectors + (int64_t)vecs * kThreads - 1) / ((int64_t)vecs * kThreads));
}

// Vectors of a thread: as many as leave enough CTAs to fill the machine.
int vecs_of(int64_t rows, int64_t vocab, int es)
{
    int vecs = kMaxVecs;
    while (vecs > 1 && rows * chunks_of(vocab, es, vecs) < kFill) vecs >>= 1;
    return vecs;
}

template <int kType>
void launch(const SelectArgs &a, int vecs, cudaStream_t st)
{
    const unsigned ctas = (unsigned)(a.in.groups * a.in.beams * a.chunks);
    switch (vecs) {
    case 1: select_kernel<kType, 1><<<ctas, kThreads, 0, st>>>(a); break;
    case 2: select_kernel<kType, 2><<<ctas, kThreads, 0, st>>>(a); break;
    case 4: select_kernel<kType, 4><<<ctas, kThreads, 0, st>>>(a); break;
    default: select_kernel<kType, kMaxVecs><<<ctas, kThreads, 0, st>>>(a); break;
    }
}

}  // namespace

// Lists that any call of at most `rows` rows and `vocab` tokens needs: with
// kMaxVecs vectors a thread, its rows' chunks; with fewer, twice vecs would not have
// filled the machine, so at most twice that many CTAs and one more a row.
int64_t wf_beam_lists(int64_t rows, int64_t vocab)
{
    const int64_t full = rows * chunks_of(vocab, 4, kMaxVecs);
    return std::max(full, 2 * kFill + rows);
}

int wf_launch_select(wf_decode *d, const wf_beam *in, const wf_beam_out *out, cudaStream_t st)
{
    const int es = in->dtype == WF_F32 ? 4 : 2;
    const int64_t rows = (int64_t)in->groups * in->beams;
    const int vecs = vecs_of(rows, in->vocab, es);
    SelectArgs a;
    a.in = *in;
    a.out = *out;
    a.chunks = chunks_of(in->vocab, es, vecs);
    a.part = d->part;
    a.list = d->list;
    a.row_key = d->row_key;
    a.row_token = d->row_token;
    a.row_ticket = d->ticket + 1;
    a.group_ticket = d->ticket + 1 + d->lim.max_rows;
    if (rows * a.chunks > d->lists) return wf_set_error(WF_EINVAL, "wf_beam_select: %lld lists exceed the scratch", (long long)(rows * a.chunks));
    if (in->dtype == WF_F32) launch<WF_F32>(a, vecs, st);
    else if (in->dtype == WF_F16) launch<WF_F16>(a, vecs, st);
    else launch<WF_BF16>(a, vecs, st);
    return wf_cuda_check(cudaGetLastError(), "select launch");
}
