// A layer's keys and values into the paged cache, with rotary positions
// (wf_kv_write), and an 8-bit cache's scales after copies (wf_kv_copy_scales).
//
// A pair (a, b) of token t at angle x = pos * turn turns to
// m (a cos x - b sin x, b cos x + a sin x).  Turns are whole numbers of 2^-64,
// so pos * turn modulo 2^64 is the exact angle modulo a turn, whatever the
// position; its upper 32 bits, less whole quarters, go through sincospi.
//
// It has to read the step's tensors and write the queries and the cache, once
// each, and computes little: HBM bounds it, and launches where tokens are few.
// A lane takes 8 pairs of a head (two 16-byte loads, two 16-byte stores), a
// CTA some tokens with all their heads, so that the cosines of a token are made
// once, in shared memory, for every head.  18,360 tokens of 32 + 8 + 8 heads of 128 take 85 us, 5.3 TB/s; two rounds of loads under way
// together are best (77 us for 16,800 tokens; four 80: fewer warps fit).
#include <algorithm>

#include "wf_decode.cuh"
#include "wf_layer.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 64;   // tokens whose angles shared memory holds at once
constexpr int kMost16 = 32;  // tokens of a window over 8 bits and of a CTA that turns queries beside; 16 bits: 8 at most
constexpr int kMaxHeads = 4; // 8 bits: heads of a CTA

struct WriteArgs {
    const int64_t *slot;
    const int32_t *pos;
    int64_t tokens, n_slots;
    wf_div by_bs;
    int32_t few;        // slots fit 31 bits: a block by a multiplication
    int32_t rows, bs, kv, q_heads, pairs;  // pairs: of a head that turn
    const uint64_t *turn;
    float magnitude;
    const uint8_t *k, *v, *q;
    uint8_t *q_out;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;
    uint8_t *ck, *cv;
    int64_t block_stride, token_stride, head_stride;
    float *k_scale, *v_scale;
    int32_t per;        // tokens of a CTA (of an 8-bit window: whose blocks' parts it takes)
    int32_t windows;    // 8 bits: CTAs in x that write the cache; the others turn queries
    int32_t heads_per;  // 8 bits: heads of a CTA
    int *err;
};

template <int D> constexpr int kLanes = D / 16;  // lanes of a head: 8 pairs each

// 8 pairs of a lane: a and b as 4 packed words each.  HALF: pairs (i, i + dim/2), else neighbours.
struct Pairs {
    uint32_t a[4], b[4];
};

// Where lane u's pairs lie: HALF && turning: 8 elements from 8u and 8 from 8u + pairs; else 16 elements from 16u.
__device__ __forceinline__ bool halves_apart(bool half, int u, int pairs) { return half && 8 * u < pairs; }

template <bool HALF> __device__ __forceinline__ Pairs load_pairs(const uint8_t *head, int u, int pairs)
{
    const bool apart = halves_apart(HALF, u, pairs);
    const uint4 x = *reinterpret_cast<const uint4 *>(head + (apart ? 16 * u : 32 * u));
    const uint4 y = *reinterpret_cast<const uint4 *>(head + (apart ? 16 * u + 2 * pairs : 32 * u + 16));
    return {{x.x, x.y, x.z, x.w}, {y.x, y.y, y.z, y.w}};
}

template <bool HALF> __device__ __forceinline__ void store_pairs(uint8_t *head, int u, int pairs, const Pairs &p)
{
    const bool apart = halves_apart(HALF, u, pairs);
    *reinterpret_cast<uint4 *>(head + (apart ? 16 * u : 32 * u)) = make_uint4(p.a[0], p.a[1], p.a[2], p.a[3]);
    *reinterpret_cast<uint4 *>(head + (apart ? 16 * u + 2 * pairs : 32 * u + 16)) = make_uint4(p.b[0], p.b[1], p.b[2], p.b[3]);
}

// The same, element by element: any alignment, any even part of the head.  Pair i < pairs is (i, i + pairs) or
// (2i, 2i + 1), pair i >= pairs the elements 2i, 2i + 1 (which do not turn).
__device__ __forceinline__ int first_of(bool half, int i, int pairs) { return half && i < pairs ? i : 2 * i; }
__device__ __forceinline__ int second_of(bool half, int i, int pairs) { return half && i < pairs ? i + pairs : 2 * i + 1; }

template <bool HALF> __device__ __forceinline__ Pairs gather_pairs(const uint8_t *head, int u, int pairs)
{
    const uint16_t *x = reinterpret_cast<const uint16_t *>(head);
    Pairs p;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int i = 8 * u + 2 * j;
        p.a[j] = x[first_of(HALF, i, pairs)] | (uint32_t)x[first_of(HALF, i + 1, pairs)] << 16;
        p.b[j] = x[second_of(HALF, i, pairs)] | (uint32_t)x[second_of(HALF, i + 1, pairs)] << 16;
    }
    return p;
}

template <bool HALF> __device__ __forceinline__ void scatter_pairs(uint8_t *head, int u, int pairs, const Pairs &p)
{
    uint16_t *x = reinterpret_cast<uint16_t *>(head);
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const int i = 8 * u + j;
        x[first_of(HALF, i, pairs)] = (uint16_t)(p.a[j / 2] >> (16 * (j % 2)));
        x[second_of(HALF, i, pairs)] = (uint16_t)(p.b[j / 2] >> (16 * (j % 2)));
    }
}

// The lane's pairs turned by cs[8u ..] (cosine, sine, both times the magnitude) and rounded to T.  Of gathered pairs
// and of half pairs that lie apart, word j holds the firsts (a) and seconds (b) of pairs 2j, 2j + 1; of 16 neighbouring elements, a
// holds pairs 0..3 and b pairs 4..7, both elements of a pair in a word.
template <typename T, bool SPLIT> __device__ __forceinline__ void turn_pairs(Pairs &p, const float2 *cs, int u, int pairs)
{
    if (8 * u >= pairs) return;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const int i = SPLIT ? 8 * u + 2 * j : 8 * u + j, k = SPLIT ? i + 1 : i + 4;
        const float2 a = wf_pair<T>::to_float(p.a[j]), b = wf_pair<T>::to_float(p.b[j]);
        const float2 ci = i < pairs ? cs[i] : make_float2(1.f, 0.f), ck = k < pairs ? cs[k] : make_float2(1.f, 0.f);
        const float ix = a.x, iy = SPLIT ? b.x : a.y, kx = SPLIT ? a.y : b.x, ky = b.y;
        // One rounding of a product, one of the sum, the same in every layout.
        const float i0 = __fmaf_rn(ix, ci.x, -__fmul_rn(iy, ci.y)), i1 = __fmaf_rn(iy, ci.x, __fmul_rn(ix, ci.y));
        const float k0 = __fmaf_rn(kx, ck.x, -__fmul_rn(ky, ck.y)), k1 = __fmaf_rn(ky, ck.x, __fmul_rn(kx, ck.y));
        const uint32_t was_a = p.a[j], was_b = p.b[j];
        p.a[j] = SPLIT ? wf_pair<T>::of_float(i0, k0) : wf_pair<T>::of_float(i0, i1);
        p.b[j] = SPLIT ? wf_pair<T>::of_float(i1, k1) : wf_pair<T>::of_float(k0, k1);
        // Pairs behind the turning part keep their bits (0 times an infinity is none of them).
        if (SPLIT) {
            if (i >= pairs) p.a[j] = p.a[j] & 0xFFFF0000u | was_a & 0xFFFFu, p.b[j] = p.b[j] & 0xFFFF0000u | was_b & 0xFFFFu;
            if (k >= pairs) p.a[j] = p.a[j] & 0xFFFFu | was_a & 0xFFFF0000u, p.b[j] = p.b[j] & 0xFFFFu | was_b & 0xFFFF0000u;
        } else {
            if (i >= pairs) p.a[j] = was_a;
            if (k >= pairs) p.b[j] = was_b;
        }
    }
}

// VEC: tensors on 16-byte boundaries, and with HALF a turning part of a multiple of 16 elements.
template <typename T, bool HALF, bool VEC> __device__ __forceinline__ Pairs load_any(const uint8_t *head, int u, int pairs)
{
    return VEC ? load_pairs<HALF>(head, u, pairs) : gather_pairs<HALF>(head, u, pairs);
}

template <typename T, bool HALF, bool VEC>
__device__ __forceinline__ void turn_any(Pairs &p, const float2 *cs, int u, int pairs)
{
    if (VEC && !HALF) turn_pairs<T, false>(p, cs, u, pairs);
    else turn_pairs<T, true>(p, cs, u, pairs);
}

__device__ __forceinline__ int64_t block_of(const WriteArgs &a, int64_t slot)
{
    return a.few ? (int64_t)wf_quot((uint32_t)slot, a.by_bs) : slot / a.bs;
}

// The bytes from the cache's start to a slot's token, or -1.
__device__ __forceinline__ int64_t slot_offset(const WriteArgs &a, int64_t slot)
{
    if (slot < 0) return -1;
    if (slot >= a.n_slots) {
        *a.err = 1;
        return -1;
    }
    const int64_t block = block_of(a, slot);
    return block * a.block_stride + (slot - block * a.bs) * a.token_stride;
}

// cos and sin of n tokens from `first`, and where they go.
__device__ __forceinline__ void load_tokens(const WriteArgs &a, int64_t first, int n, float2 *cs, int64_t *at)
{
    for (int i = threadIdx.x; i < n; i += kThreads) at[i] = slot_offset(a, a.slot[first + i]);
    for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
        const int t = i / a.pairs, p = i - t * a.pairs;
        const uint32_t part = (uint32_t)(((uint64_t)(uint32_t)a.pos[first + t] * a.turn[p]) >> 32);  // of a turn, in 2^-32
        // The nearest quarter, and what is left: at most an eighth of a turn, so that 24 bits hold it to 2^-27 of a turn.
        const uint32_t quarter = (part + (1u << 29)) >> 30;
        float s, c;
        sincospif((float)(int32_t)(part - (quarter << 30)) * 0x1p-31f, &s, &c);
        if (quarter & 1) {
            const float was = c;
            c = -s, s = was;
        }
        if (quarter & 2) c = -c, s = -s;
        cs[i] = make_float2(c * a.magnitude, s * a.magnitude);
    }
}

// Tokens from `first`, n of them: keys, values (KV) and queries, each read once and written once.
template <typename T, int D, bool HALF, bool VEC, bool KV>
__device__ __forceinline__ void write_tokens(const WriteArgs &a, int64_t first, int n, float2 *cs)
{
    __shared__ int64_t at[kMost16];
    constexpr int kGroups = kThreads / kLanes<D>, kDeep = 2;  // heads at once; rounds whose loads are under way together
    const int u = threadIdx.x % kLanes<D>, heads = a.q_heads + (KV ? 2 * a.kv : 0);
    load_tokens(a, first, n, cs, at);
    __syncthreads();
    int t = 0, h = threadIdx.x / kLanes<D>;  // heads in the order queries, keys, values
    while (h >= heads) h -= heads, t++;
    while (t < n) {
        Pairs p[kDeep];
        int tt[kDeep], hh[kDeep];
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            tt[i] = t, hh[i] = h;
            if (t < n) {
                const uint8_t *from = h < a.q_heads ? a.q + (first + t) * a.q_token + h * a.q_head
                                      : h < a.q_heads + a.kv ? a.k + (first + t) * a.k_token + (h - a.q_heads) * a.k_head
                                                             : a.v + (first + t) * a.v_token + (h - a.q_heads - a.kv) * a.v_head;
                p[i] = load_any<T, HALF, VEC>(from, u, a.pairs);
            }
            h += kGroups;
            while (h >= heads) h -= heads, t++;
        }
#pragma unroll
        for (int i = 0; i < kDeep; i++) {
            if (tt[i] >= n || at[tt[i]] < 0) continue;
            const bool q = hh[i] < a.q_heads, v = hh[i] >= a.q_heads + a.kv;
            if (!v) turn_any<T, HALF, VEC>(p[i], cs + tt[i] * a.pairs, u, a.pairs);
            const int kh = hh[i] - a.q_heads - (v ? a.kv : 0);
            uint8_t *to = q ? a.q_out + (first + tt[i]) * a.o_token + hh[i] * a.o_head
                            : (v ? a.cv : a.ck) + at[tt[i]] + kh * a.head_stride;
            if (VEC) store_pairs<HALF>(to, u, a.pairs, p[i]);
            else scatter_pairs<HALF>(to, u, a.pairs, p[i]);
        }
    }
}

template <typename T, int D, bool HALF, bool VEC> __global__ void __launch_bounds__(kThreads) write16_kernel(const WriteArgs a)
{
    extern __shared__ float2 angles[];
    const int64_t first = (int64_t)blockIdx.x * a.per;
    write_tokens<T, D, HALF, VEC, true>(a, first, (int)min((int64_t)a.per, a.tokens - first), angles);
}

// ---------------------------------------------------------------------------
// 8 bits
//
// The scale of a block and head is known when its new tokens have been seen, so a block's part in the step is one CTA's: magnitudes, scale,
// elements.  That is a chain of loads, three barriers and a store, and what bounds it: 2,000 rows decoding (32 + 8 + 8 heads of 128) take
// 17 us where their bytes take 6.6, 8,660 prompt tokens in blocks of 64 30 us (9.2).  Elements stay in registers between magnitude and
// store where they fit (26 -> 17 us with blocks found by a multiplication in place of 64-bit divisions).
// ---------------------------------------------------------------------------

// The least e in -64..63 with 448 * 2^e >= x, x finite and >= 0; 448 = 0.875 * 2^9.
__device__ __forceinline__ float scale_of(float x)
{
    const int bits = __float_as_int(x), exp = bits >> 23;            // x = 1.f * 2^(exp - 127), 448 = 1.75 * 2^8
    const int e = exp - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000);    // subnormals lie below every limit
    return __int_as_float((min(max(e, -64), 63) + 127) << 23);
}

// A token is the first of its block's part in this step.
__device__ __forceinline__ bool begins(const WriteArgs &a, int64_t t, int64_t slot)
{
    return t == 0 || a.slot[t - 1] != slot - 1 || slot - block_of(a, slot) * a.bs == 0;
}

__device__ __forceinline__ float largest(float m, float x) { return fabsf(x) <= 3.402823466e38f ? fmaxf(m, fabsf(x)) : m; }

// The lane's 16 elements over a scale, to a token's head in the cache.
template <typename T, bool HALF, bool VEC> __device__ __forceinline__ void store8(const WriteArgs &a, const Pairs &p, float scale, uint8_t *to, int u)
{
    uint32_t w[8];  // a's 8 elements, b's 8, in twos
    const bool two = (__float_as_int(scale) & 0x7FFFFF) == 0;  // a power of two: the product with its inverse is the quotient
    const float inv = 1.f / scale;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        float2 f = wf_pair<T>::to_float(p.a[j]), g = wf_pair<T>::to_float(p.b[j]);
        if (two) f.x *= inv, f.y *= inv, g.x *= inv, g.y *= inv;
        else f.x /= scale, f.y /= scale, g.x /= scale, g.y /= scale;
        w[j] = wf_e4m3_of(f.x, f.y);
        w[4 + j] = wf_e4m3_of(g.x, g.y);
    }
    if (VEC) {
        const bool apart = halves_apart(HALF, u, a.pairs);
        *reinterpret_cast<uint2 *>(to + (apart ? 8 * u : 16 * u)) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
        *reinterpret_cast<uint2 *>(to + (apart ? 8 * u + a.pairs : 16 * u + 8)) = make_uint2(w[4] | w[5] << 16, w[6] | w[7] << 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            to[first_of(HALF, 8 * u + j, a.pairs)] = (uint8_t)(w[j / 2] >> (8 * (j % 2)));
            to[second_of(HALF, 8 * u + j, a.pairs)] = (uint8_t)(w[4 + j / 2] >> (8 * (j % 2)));
        }
    }
}

// A window of a.per <= 32 tokens, heads h0 .. h0 + n_heads: the parts of blocks that begin in it.  Largest magnitudes first, by part and
// head, then the scales, then the elements; where the parts are short (kKeep heads of a token for each group of lanes) these stay in registers
// between.
template <typename T, int D, bool HALF, bool VEC> __device__ __forceinline__ void write8_window(const WriteArgs &a, int64_t first, int h0, float2 *cs)
{
    constexpr int kL = kLanes<D>, kGroups = kThreads / kL, kKeep = 4;
    __shared__ int64_t at[kChunk], part_block[32];
    __shared__ int part_held[32];                    // tokens of the block before the part
    __shared__ int amax[32 * 2 * kMaxHeads];         // [32][combos], then the scales
    __shared__ float ratio[32 * 2 * kMaxHeads];      // [32][combos] old scale over new, 1: nothing to do
    __shared__ uint32_t s_begin;
    __shared__ int s_end;
    const int n_heads = min(a.heads_per, a.kv - h0), combos = 2 * n_heads;
    const int u = threadIdx.x % kL, group = threadIdx.x / kL;
    const int n = (int)min((int64_t)a.per, a.tokens - first);
    // The parts that begin here, and the end of the last one.
    if (threadIdx.x < 32) {
        const int64_t t = first + threadIdx.x;
        const int64_t slot = threadIdx.x < n ? a.slot[t] : -1;
        const bool live = slot >= 0 && slot < a.n_slots;
        if (slot >= a.n_slots) *a.err = 1;
        const uint32_t begin = __ballot_sync(~0u, live && begins(a, t, slot)), dead = __ballot_sync(~0u, !live && threadIdx.x < n);
        if (live && (begin >> threadIdx.x & 1)) {
            const int i = __popc(begin & ((1u << threadIdx.x) - 1));
            part_block[i] = block_of(a, slot);
            part_held[i] = (int)(slot - part_block[i] * a.bs);
        }
        if (threadIdx.x == 0) {
            s_begin = begin;
            const uint32_t after = begin ? dead & ~((2u << (31 - __clz(begin))) - 1) : 0;  // the last part ends in the window
            s_end = after ? __ffs(after) - 1 : 0x7FFFFFFF;
        }
    }
    for (int i = threadIdx.x; i < 32 * combos; i += kThreads) amax[i] = 0;
    __syncthreads();
    const uint32_t begin = s_begin;
    if (!begin) return;
    if (n == a.per && s_end > n) {  // on behind the window
        for (int64_t base = n; base < (int64_t)a.bs + n && s_end == 0x7FFFFFFF; base += kThreads) {
            __syncthreads();
            const int64_t t = first + base + threadIdx.x;
            const int64_t slot = t < a.tokens ? a.slot[t] : -1;
            if (slot < 0 || slot >= a.n_slots || begins(a, t, slot)) atomicMin(&s_end, (int)(base + threadIdx.x));
            __syncthreads();
        }
    }
    const int end = min((int64_t)s_end, a.tokens - first), from = __ffs(begin) - 1;
    const int parts = __popc(begin);
    // The part of token i of the range: how many begin at or before it.
    auto part_of = [&](int i) { return __popc(i >= 31 ? begin : begin & ((2u << i) - 1)) - 1; };
    auto load = [&](int t, int combo) {
        const int64_t tok = first + t;
        const bool v = combo >= n_heads;
        const int h = h0 + (v ? combo - n_heads : combo);
        return load_any<T, HALF, VEC>(v ? a.v + tok * a.v_token + h * a.v_head : a.k + tok * a.k_token + h * a.k_head, u, a.pairs);
    };
    auto head_at = [&](int combo) { return (combo >= n_heads ? a.cv : a.ck) + (h0 + (combo >= n_heads ? combo - n_heads : combo)) * a.head_stride; };
    auto scale_at = [&](int part, int combo) {
        const bool v = combo >= n_heads;
        return (v ? a.v_scale : a.k_scale) + part_block[part] * a.kv + h0 + (v ? combo - n_heads : combo);
    };
    auto most_of = [](const Pairs &p) {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float2 x = wf_pair<T>::to_float(p.a[j]), y = wf_pair<T>::to_float(p.b[j]);
            most = largest(largest(largest(largest(most, x.x), x.y), y.x), y.y);
        }
        return most;
    };
    // Every group of the warp comes; live: with a token and head of its own.
    auto put_most = [&](bool live, float most, int t, int combo) {
#pragma unroll
        for (int s = kL / 2; s; s /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, s));
        if (live && u == 0) atomicMax(&amax[part_of(t) * combos + combo], __float_as_int(most));
    };
    const float old = threadIdx.x < parts * combos ? *scale_at(threadIdx.x / combos, threadIdx.x % combos) : 0.f;  // under way early
    const int items = (end - from) * combos;
    const bool kept = end - from <= kChunk && items <= kKeep * kGroups;
    Pairs keep[kKeep];
    if (kept) {
#pragma unroll
        for (int r = 0; r < kKeep; r++) {
            const int i = group + r * kGroups, t = i / combos;
            if (i < items) keep[r] = load(from + t, i - t * combos);
        }
        load_tokens(a, first + from, end - from, cs, at);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kKeep; r++) {
            const int i = group + r * kGroups, t = i / combos, combo = i - t * combos;
            const bool live = i < items && at[t] >= 0;
            if (live && combo < n_heads) turn_any<T, HALF, VEC>(keep[r], cs + t * a.pairs, u, a.pairs);
            if (r * kGroups < items) put_most(live, live ? most_of(keep[r]) : 0.f, from + t, combo);
        }
    } else {
        for (int base = from; base < end; base += kChunk) {
            const int m = min(kChunk, end - base);
            __syncthreads();
            load_tokens(a, first + base, m, cs, at);
            __syncthreads();
            for (int i = group; i - group < m * combos; i += kGroups) {
                const int t = i / combos, combo = i - t * combos;
                const bool live = i < m * combos && at[t] >= 0;
                Pairs p = {};
                if (live) {
                    p = load(base + t, combo);
                    if (combo < n_heads) turn_any<T, HALF, VEC>(p, cs + t * a.pairs, u, a.pairs);
                }
                put_most(live, most_of(p), base + t, combo);
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < parts * combos; i += kThreads) {
        const int part = i / combos, combo = i - part * combos;
        float *scale = scale_at(part, combo);
        const float need = scale_of(__int_as_float(amax[i])), was = i == threadIdx.x ? old : *scale;
        const bool held = part_held[part] > 0;
        const float now = held && was > need ? was : need;
        *scale = now;
        amax[i] = __float_as_int(now);
        ratio[i] = held ? was / now : 1.f;
    }
    __syncthreads();
    // What the blocks held before, where a scale has grown.
    for (int i = group; i < parts * combos; i += kGroups) {
        const float r = ratio[i];
        if (r == 1.f) continue;
        const int part = i / combos, combo = i - part * combos;
        const int held = part_held[part];
        uint8_t *p = head_at(combo) + part_block[part] * a.block_stride + 16 * u;
        for (int j = 0; j < held; j += 4) {
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; k++)
                if (j + k < held) x[k] = *reinterpret_cast<const uint4 *>(p + (j + k) * a.token_stride);
#pragma unroll
            for (int k = 0; k < 4; k++) {
                if (j + k >= held) break;
                uint32_t *w = &x[k].x;
#pragma unroll
                for (int c = 0; c < 4; c++) {
                    const uint2 hv = wf_e4m3_halves(w[c]);
                    const float2 lo = wf_pair<__half>::to_float(hv.x), hi = wf_pair<__half>::to_float(hv.y);
                    w[c] = wf_e4m3_of(lo.x * r, lo.y * r) | wf_e4m3_of(hi.x * r, hi.y * r) << 16;
                }
                *reinterpret_cast<uint4 *>(p + (j + k) * a.token_stride) = x[k];
            }
        }
    }
    // The new tokens.
    if (kept) {
#pragma unroll
        for (int r = 0; r < kKeep; r++) {
            const int i = group + r * kGroups, t = i / combos, combo = i - t * combos;
            if (i < items && at[t] >= 0)
                store8<T, HALF, VEC>(a, keep[r], __int_as_float(amax[part_of(from + t) * combos + combo]), head_at(combo) + at[t], u);
        }
        return;
    }
    for (int base = from; base < end; base += kChunk) {
        const int m = min(kChunk, end - base);
        __syncthreads();
        load_tokens(a, first + base, m, cs, at);
        __syncthreads();
        for (int i = group; i < m * combos; i += kGroups) {
            const int t = i / combos, combo = i - t * combos;
            if (at[t] < 0) continue;
            Pairs p = load(base + t, combo);
            if (combo < n_heads) turn_any<T, HALF, VEC>(p, cs + t * a.pairs, u, a.pairs);
            store8<T, HALF, VEC>(a, p, __int_as_float(amax[part_of(base + t) * combos + combo]), head_at(combo) + at[t], u);
        }
    }
}

template <typename T, int D, bool HALF, bool VEC> __global__ void __launch_bounds__(kThreads, 4) write8_kernel(const WriteArgs a)
{
    extern __shared__ float2 angles[];
    const int split = (a.kv + a.heads_per - 1) / a.heads_per;
    const int64_t cta = blockIdx.x;
    if (cta < (int64_t)a.windows * split) {
        write8_window<T, D, HALF, VEC>(a, cta / split * a.per, (int)(cta % split) * a.heads_per, angles);
    } else {
        const int64_t first = (cta - (int64_t)a.windows * split) * a.per;
        write_tokens<T, D, HALF, VEC, false>(a, first, (int)min((int64_t)a.per, a.tokens - first), angles);
    }
}

// ---------------------------------------------------------------------------

__global__ void copy_scales_kernel(const int32_t *copies, int32_t rows, int32_t n_blocks, float *scale, int32_t planes, int64_t plane_stride,
                                   int32_t heads, int *err)
{
    const int64_t each = (int64_t)planes * heads;
    for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < rows * each; i += (int64_t)gridDim.x * blockDim.x) {
        const int32_t r = (int32_t)(i / each), j = (int32_t)(i - r * each), p = j / heads, h = j - p * heads;
        const int32_t from = copies[2 * (int64_t)r], to = copies[2 * (int64_t)r + 1];
        if (to < 0 && from < 0) continue;
        if (from < 0 || from >= n_blocks || to < 0 || to >= n_blocks) {
            *err = 1;
            continue;
        }
        scale[p * plane_stride + (int64_t)to * heads + h] = scale[p * plane_stride + (int64_t)from * heads + h];
    }
}

template <typename T, int D, bool HALF, bool VEC> int launch(const WriteArgs &args, bool f8, int sms, cudaStream_t st)
{
    WriteArgs a = args;
    // Tokens of a CTA: enough CTAs for every SM before a CTA's angles serve more than one token; 8 at most, from where on
    // nothing more is saved.
    if (!f8) {
        a.per = (int)std::min<int64_t>(8, std::max<int64_t>(1, a.tokens / (4 * sms)));
        write16_kernel<T, D, HALF, VEC><<<(unsigned)((a.tokens + a.per - 1) / a.per), kThreads, a.per * a.pairs * sizeof(float2), st>>>(a);
        return wf_cuda_check(cudaGetLastError(), "write16_kernel");
    }
    // 8 bits: a block's part is one CTA's, so that blocks, not tokens, are what there is to share out; heads are shared out too until
    // every SM has CTAs enough.
    a.per = (int)std::min<int64_t>(kMost16, std::max<int64_t>(1, a.tokens / (2 * sms)));
    a.windows = (int)((a.tokens + a.per - 1) / a.per);
    const int64_t parts = std::max((a.tokens + std::max(a.per, a.bs) - 1) / std::max(a.per, a.bs), std::min<int64_t>(a.rows, a.tokens) / a.per);
    a.heads_per = std::min(a.kv, kMaxHeads);
    while (a.heads_per > 1 && parts * ((a.kv + a.heads_per - 1) / a.heads_per) < 4 * sms) a.heads_per = (a.heads_per + 1) / 2;
    const int64_t split = (a.kv + a.heads_per - 1) / a.heads_per;
    const int64_t ctas = a.windows * split + (a.q_heads ? a.windows : 0);
    if (ctas > INT32_MAX) return wf_set_error(WF_EINVAL, "wf_kv_write: %lld tokens of %d heads", (long long)a.tokens, a.kv);
    const int most = (int)std::min<int64_t>(kChunk, (int64_t)a.per + a.bs);  // tokens whose angles a CTA holds
    write8_kernel<T, D, HALF, VEC><<<(unsigned)ctas, kThreads, most * a.pairs * sizeof(float2), st>>>(a);
    return wf_cuda_check(cudaGetLastError(), "write8_kernel");
}

template <typename T, int D> int launch_layout(const WriteArgs &a, bool half, bool vec, bool f8, int sms, cudaStream_t st)
{
    if (half) return vec ? launch<T, D, true, true>(a, f8, sms, st) : launch<T, D, true, false>(a, f8, sms, st);
    return vec ? launch<T, D, false, true>(a, f8, sms, st) : launch<T, D, false, false>(a, f8, sms, st);
}

}  // namespace

int wf_launch_write(wf_decode *d, const wf_kv *kv, const wf_kv_step *step, const wf_kv_layer *l, const wf_rope *rope,
                    const wf_kv_new *in, cudaStream_t st)
{
    WriteArgs a{};
    a.slot = step->slot, a.pos = step->pos;
    a.tokens = step->max_tokens, a.n_slots = (int64_t)kv->n_blocks * kv->block_tokens;
    a.by_bs = wf_make_div(kv->block_tokens), a.few = a.n_slots <= INT32_MAX;
    a.rows = kv->rows, a.bs = kv->block_tokens, a.kv = l->heads, a.q_heads = in->q_heads;
    a.pairs = rope ? rope->dim / 2 : 0;
    a.turn = rope ? rope->turn : nullptr, a.magnitude = rope ? rope->magnitude : 1.f;
    a.k = (const uint8_t *)in->k, a.v = (const uint8_t *)in->v, a.q = (const uint8_t *)in->q, a.q_out = (uint8_t *)in->q_out;
    a.k_token = in->k_token, a.k_head = in->k_head, a.v_token = in->v_token, a.v_head = in->v_head;
    a.q_token = in->q_token, a.q_head = in->q_head, a.o_token = in->q_out_token, a.o_head = in->q_out_head;
    a.ck = (uint8_t *)l->k, a.cv = (uint8_t *)l->v;
    a.block_stride = l->block_stride, a.token_stride = l->token_stride, a.head_stride = l->head_stride;
    a.k_scale = l->k_scale, a.v_scale = l->v_scale;
    a.err = d->err;
    const bool half = rope && rope->dim && !rope->interleaved, f8 = l->dtype == WF_E4M3;
    // 16 bytes at a time: every address a multiple of 16, and halves that a lane's 8 pairs do not straddle.
    int64_t bits = (int64_t)(uintptr_t)a.k | (int64_t)(uintptr_t)a.v | a.k_token | a.k_head | a.v_token | a.v_head;
    if (a.q_heads) bits |= (int64_t)(uintptr_t)a.q | (int64_t)(uintptr_t)a.q_out | a.q_token | a.q_head | a.o_token | a.o_head;
    const bool vec = bits % 16 == 0 && !(half && a.pairs % 8);
    if (in->dtype == WF_F16)
        return l->dim == 64 ? launch_layout<__half, 64>(a, half, vec, f8, d->sms, st) : launch_layout<__half, 128>(a, half, vec, f8, d->sms, st);
    return l->dim == 64 ? launch_layout<__nv_bfloat16, 64>(a, half, vec, f8, d->sms, st)
                        : launch_layout<__nv_bfloat16, 128>(a, half, vec, f8, d->sms, st);
}

int wf_launch_copy_scales(wf_decode *d, const wf_kv *kv, const int32_t *copies, float *scale, int32_t planes, int64_t plane_stride,
                          int32_t heads, cudaStream_t st)
{
    const int64_t n = (int64_t)kv->rows * planes * heads;
    const unsigned ctas = (unsigned)std::min<int64_t>((n + 255) / 256, 8 * d->sms);
    copy_scales_kernel<<<ctas, 256, 0, st>>>(copies, kv->rows, kv->n_blocks, scale, planes, plane_stride, heads, d->err);
    return wf_cuda_check(cudaGetLastError(), "copy_scales_kernel");
}
