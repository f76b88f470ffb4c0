// The calls on a layer's tensors, host side: the checks of their arguments.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>

#include "wf_attend.cuh"
#include "wf_decode.cuh"
#include "wf_layer.cuh"

#define REQUIRE(cond, ...) \
    do { if (!(cond)) return wf_set_error(WF_EINVAL, __VA_ARGS__); } while (0)

static int check_step(const wf_kv_step *step, const char *what)
{
    REQUIRE(step, "%s: the step is NULL", what);
    REQUIRE(step->max_tokens >= 1 && step->max_tokens <= INT32_MAX - 1, "%s: max_tokens %lld", what, (long long)step->max_tokens);
    return WF_OK;
}

static int check_layer(const wf_kv_layer *l, int32_t dtype, const char *what)
{
    REQUIRE(l, "%s: the layer is NULL", what);
    REQUIRE(l->dim == 64 || l->dim == 128, "%s: heads of %d elements; 64 or 128", what, l->dim);
    REQUIRE(l->heads >= 1 && l->heads <= 1024, "%s: %d key / value heads outside 1..1024", what, l->heads);
    REQUIRE(l->reserved == 0, "%s: reserved %d", what, l->reserved);
    REQUIRE(dtype == WF_F16 || dtype == WF_BF16, "%s: tensors of type %d", what, dtype);
    REQUIRE(l->dtype == dtype || l->dtype == WF_E4M3, "%s: a layer of type %d for tensors of type %d", what, l->dtype, dtype);
    REQUIRE(l->k && l->v, "%s: NULL keys or values", what);
    REQUIRE(wf_aligned(l->k, 16) && wf_aligned(l->v, 16), "%s: keys or values not on 16 bytes", what);
    REQUIRE(l->block_stride >= 0 && l->token_stride >= 0 && l->head_stride >= 0 &&
                (l->block_stride | l->token_stride | l->head_stride) % 16 == 0,
            "%s: strides %lld, %lld, %lld of the layer; multiples of 16, >= 0", what, (long long)l->block_stride,
            (long long)l->token_stride, (long long)l->head_stride);
    const bool scaled = l->dtype == WF_E4M3;
    REQUIRE(!!l->k_scale == scaled && !!l->v_scale == scaled, "%s: scales belong to layers of 8 bits, and to all of those", what);
    REQUIRE(wf_aligned(l->k_scale, 4) && wf_aligned(l->v_scale, 4), "%s: misaligned scales", what);
    return WF_OK;
}

static int check_heads(const void *p, int64_t token, int64_t head, const char *what, const char *name)
{
    REQUIRE(p, "%s: NULL %s", what, name);
    REQUIRE(wf_aligned(p, 2) && token % 2 == 0 && head % 2 == 0, "%s: %s or its strides %lld, %lld not on 2 bytes", what, name,
            (long long)token, (long long)head);
    return WF_OK;
}

// A tensor [tokens][heads][elements], strides in bytes.
struct Heads {
    const void *at;
    int64_t token, head;
    int32_t heads;
};

// Whether two of them have bytes in common.  Tensors that lie among each other (parts of one product's columns) need the same strides to be told
// apart; others have to have ranges of their own.
static bool meet(const Heads &a, const Heads &b, int64_t tokens, int64_t bytes)
{
    const int64_t n = tokens - 1;
    auto low = [&](const Heads &x) { return n * std::min<int64_t>(x.token, 0) + (x.heads - 1) * std::min<int64_t>(x.head, 0); };
    auto high = [&](const Heads &x) { return n * std::max<int64_t>(x.token, 0) + (x.heads - 1) * std::max<int64_t>(x.head, 0) + bytes; };
    const int64_t apart = (const uint8_t *)b.at - (const uint8_t *)a.at;
    if (apart + low(b) >= high(a) || apart + high(b) <= low(a)) return false;
    const int64_t head = a.heads == 1 ? b.head : a.head;  // one head's stride does not count
    if ((n && a.token != b.token) || (a.heads > 1 && b.heads > 1 && a.head != b.head)) return true;
    for (int64_t j = 1 - a.heads; j < b.heads; j++) {  // heads apart; then the token that lies nearest
        const int64_t at = apart + j * head, i = a.token ? std::clamp(-at / a.token, -n, n) : 0;
        for (int64_t k = std::max(-n, i - 1); k <= std::min(n, i + 1); k++)
            if (std::abs(at + k * a.token) < bytes) return true;
    }
    return false;
}

extern "C" int wf_kv_write(wf_decode *d, const wf_kv *kv, const wf_kv_step *step, const wf_kv_layer *layer, const wf_rope *rope,
                           const wf_kv_new *in, void *stream)
{
    const char *what = "wf_kv_write";
    REQUIRE(d, "NULL decode scratch");
    int rc = wf_check_rows(kv, d->lim.max_rows, what);
    if (!rc) rc = check_step(step, what);
    if (rc) return rc;
    REQUIRE(in, "%s: the tensors are NULL", what);
    rc = check_layer(layer, in->dtype, what);
    if (!rc) rc = check_heads(in->k, in->k_token, in->k_head, what, "keys");
    if (!rc) rc = check_heads(in->v, in->v_token, in->v_head, what, "values");
    if (rc) return rc;
    REQUIRE(in->q_heads >= 0 && in->q_heads <= 1024, "%s: %d query heads outside 0..1024", what, in->q_heads);
    if (in->q_heads) {
        rc = check_heads(in->q, in->q_token, in->q_head, what, "queries");
        if (!rc) rc = check_heads(in->q_out, in->q_out_token, in->q_out_head, what, "turned queries");
        if (rc) return rc;
        REQUIRE(in->q != in->q_out || (in->q_token == in->q_out_token && in->q_head == in->q_out_head),
                "%s: queries turned in place under other strides", what);
        const Heads out = {in->q_out, in->q_out_token, in->q_out_head, in->q_heads};
        const int64_t bytes = 2 * layer->dim;
        REQUIRE((in->q == in->q_out || !meet(out, {in->q, in->q_token, in->q_head, in->q_heads}, step->max_tokens, bytes)) &&
                    !meet(out, {in->k, in->k_token, in->k_head, layer->heads}, step->max_tokens, bytes) &&
                    !meet(out, {in->v, in->v_token, in->v_head, layer->heads}, step->max_tokens, bytes),
                "%s: turned queries in the memory of keys, values or other queries", what);
    }
    REQUIRE(step->slot && wf_aligned(step->slot, 8), "%s: NULL or misaligned slots", what);
    if (rope) {
        REQUIRE(rope->dim >= 0 && rope->dim <= layer->dim && rope->dim % 2 == 0, "%s: %d of %d elements turn; an even number", what,
                rope->dim, layer->dim);
        REQUIRE(rope->interleaved == 0 || rope->interleaved == 1, "%s: interleaved %d", what, rope->interleaved);
        REQUIRE(rope->reserved == 0 && std::isfinite(rope->magnitude), "%s: magnitude %g, reserved %d", what, rope->magnitude, rope->reserved);
        REQUIRE(!rope->dim || (rope->turn && wf_aligned(rope->turn, 8)), "%s: NULL or misaligned turns", what);
        REQUIRE(!rope->dim || (step->pos && wf_aligned(step->pos, 4)), "%s: NULL or misaligned positions", what);
    }
    rc = wf_cuda_check(cudaSetDevice(d->device), "cudaSetDevice");
    return rc ? rc : wf_launch_write(d, kv, step, layer, rope, in, (cudaStream_t)stream);
}

extern "C" int wf_kv_copy_scales(wf_decode *d, const wf_kv *kv, const int32_t *copies, float *scale, int32_t planes,
                                 int64_t plane_stride, int32_t heads, void *stream)
{
    const char *what = "wf_kv_copy_scales";
    REQUIRE(d, "NULL decode scratch");
    int rc = wf_check_rows(kv, d->lim.max_rows, what);
    if (rc) return rc;
    REQUIRE(copies && scale && wf_aligned(copies, 4) && wf_aligned(scale, 4), "%s: NULL or misaligned copies or scales", what);
    REQUIRE(planes >= 1 && heads >= 1 && heads <= 1024, "%s: %d planes of %d heads", what, planes, heads);
    REQUIRE((int64_t)planes * heads <= INT32_MAX, "%s: %d planes of %d heads", what, planes, heads);
    REQUIRE(planes == 1 || plane_stride >= (int64_t)kv->n_blocks * heads, "%s: plane_stride %lld below %lld", what,
            (long long)plane_stride, (long long)kv->n_blocks * heads);
    rc = wf_cuda_check(cudaSetDevice(d->device), "cudaSetDevice");
    return rc ? rc : wf_launch_copy_scales(d, kv, copies, scale, planes, plane_stride, heads, (cudaStream_t)stream);
}

// Polls of a bounded wait unless wf_attn_limit_waits says otherwise.
constexpr int32_t kPolls = 1 << 20;

extern "C" int wf_attn_create(const wf_attn_limits *lim, int device, wf_attn **out)
{
    REQUIRE(out, "out is NULL");
    *out = nullptr;
    REQUIRE(lim, "limits is NULL");
    REQUIRE(lim->max_rows >= 1 && lim->max_rows <= 65536, "max_rows %d outside 1..65536", lim->max_rows);
    REQUIRE(lim->max_heads >= 1 && lim->max_heads <= 1024, "max_heads %d outside 1..1024", lim->max_heads);
    REQUIRE(lim->dim == 64 || lim->dim == 128, "heads of %d elements; 64 or 128", lim->dim);
    REQUIRE(lim->reserved == 0, "reserved %d", lim->reserved);
    REQUIRE(device >= 0, "device %d", device);
    int rc = wf_cuda_check(cudaSetDevice(device), "cudaSetDevice");
    if (rc) return rc;
    wf_attn *a = (wf_attn *)calloc(1, sizeof(wf_attn));
    if (!a) return wf_set_error(WF_ENOMEM, "host allocation of the attention scratch");
    a->device = device;
    a->lim = *lim;
    a->polls = kPolls;
    rc = wf_cuda_check(cudaDeviceGetAttribute(&a->sms, cudaDevAttrMultiProcessorCount, device), "device attributes");
    if (!rc) rc = wf_attend_setup(a);
    if (!rc) rc = wf_prompt_setup(a);
    if (rc) { wf_attn_destroy(a); return rc; }
    int ctas = 0;
    size_t parts = 0;
    wf_attend_scratch(a, &parts, &ctas);
    parts = (parts + 255) / 256 * 256;
    const size_t arrivals = (4 * (size_t)std::max(ctas, a->sms) + 255) / 256 * 256, zeroed = 256 + 2 * arrivals;
    rc = wf_cuda_check(cudaMalloc(&a->mem, zeroed + parts + wf_prompt_scratch(a)), "cudaMalloc(attention scratch)");
    if (!rc) rc = wf_cuda_check(cudaMemset(a->mem, 0, zeroed), "clear the attention scratch");
    // The clearing runs on the default stream; the calls may use any other.
    if (!rc) rc = wf_cuda_check(cudaDeviceSynchronize(), "cudaDeviceSynchronize");
    if (rc) { wf_attn_destroy(a); return rc; }
    a->err = (int *)a->mem, a->zeroed = zeroed;
    for (int i = 0; i < 2; i++) {
        a->arrive[i] = (uint32_t *)((uint8_t *)a->mem + 256 + i * arrivals);
        a->part[i] = (float *)((uint8_t *)a->mem + zeroed + i * parts);
    }
    *out = a;
    return WF_OK;
}

extern "C" void wf_attn_destroy(wf_attn *a)
{
    if (!a) return;
    if (a->mem) {
        cudaSetDevice(a->device);
        cudaFree(a->mem);
    }
    free(a);
}

extern "C" int wf_attn_status(wf_attn *a, void *stream)
{
    REQUIRE(a, "NULL attention scratch");
    int rc = wf_cuda_check(cudaSetDevice(a->device), "cudaSetDevice");
    if (!rc) rc = wf_cuda_check(cudaStreamSynchronize((cudaStream_t)stream), "cudaStreamSynchronize");
    int err[2] = {0, 0};
    if (!rc) rc = wf_cuda_check(cudaMemcpy(err, a->err, sizeof(err), cudaMemcpyDeviceToHost), "read error words");
    if (rc || !(err[0] | err[1])) return rc;
    // With the arrivals: those of a call whose waits ran out were not all made.
    rc = wf_cuda_check(cudaMemset(a->mem, 0, a->zeroed), "clear error words");
    if (!rc) rc = wf_cuda_check(cudaDeviceSynchronize(), "cudaDeviceSynchronize");
    if (rc) return rc;
    if (err[1]) return wf_set_error(WF_ETIMEOUT, "a bounded wait expired; outputs of the calls since the last status are invalid");
    return wf_set_error(WF_EINVAL, "a table names a block outside the cache, or a row's lengths contradict each other");
}

extern "C" int wf_attn_limit_waits(wf_attn *a, int32_t polls)
{
    REQUIRE(a, "NULL attention scratch");
    REQUIRE(polls >= 0 && polls <= kPolls, "%d polls outside 0..%d", polls, kPolls);
    a->polls = polls;
    return WF_OK;
}

// Queries to a key head (new tokens times the group's heads) up to which a row goes to attend_kernel: one of its tiles.  Two tiles read the
// row's keys twice: 32 rows of 20 queries (32 / 8 heads of 128, bfloat16) behind 9,000 tokens take 398 us there and 242 in prompt_kernel, 64 rows of 20
// (16 / 4 heads of 64, halves) behind 3,000 107 us and 99.  Outputs in bfloat16 are further off there, as weights are rounded once: 2.3e-3 of their root mean square
// at 20 to 32 queries behind 9,000 tokens, 1.7e-3 in attend_kernel (the outputs' own rounding: 1.7e-3).
constexpr int64_t kFew = 16;

// Cycles of a tile of each kernel on an SM, as measured with full SMs (chunks of 500 behind 2,000 tokens; 161 rows behind 2,000), from which
// the SMs are shared out where both run.  tile_share: 64 positions' keys and values at 6.7 TB/s and 1.93 GHz.  Side by side against one after the other,
// us: 8 chunks of 500 and 161 rows behind 2,000 (28 / 4 heads of 128, bfloat16) 243, 279; the same over blocks that no box fits 298, 307; 12 of 300 and 108 rows
// behind 2,000 (24 / 8 of 64, bfloat16) 191, 214; 4 of 700 and 96 rows behind 4,000 (32 / 4 of 128, halves) 263, 318.  Over 8 bits instructions bound
// both kernels, and one after the other is faster: 9 of 700 and 51 rows behind 3,500 (24 / 8 of 64) 378, 351; 4 of 700 and 96 rows behind 4,000 (32 / 8 of 128) 519, 438.
static void wf_costs(int dim, AttendArgs *a)
{
    a->pair_cost = dim == 128 ? 4000 : 3000;
    a->tile_cost = dim == 128 ? 1100 : 900;
    a->tile_share = 16 * (64 * 2 * dim * 2) / 3470;
}

static int check_attn(const void *p, int64_t token, int64_t head, const char *what, const char *name)
{
    REQUIRE(p, "%s: NULL %s", what, name);
    REQUIRE(wf_aligned(p, 16) && token % 16 == 0 && head % 16 == 0, "%s: %s or its strides %lld, %lld not on 16 bytes", what, name,
            (long long)token, (long long)head);
    return WF_OK;
}

extern "C" int wf_attend(wf_attn *at, const wf_kv *kv, const wf_kv_step *step, const wf_kv_layer *layer, const wf_attn_in *in, void *stream)
{
    const char *what = "wf_attend";
    REQUIRE(at, "NULL attention scratch");
    int rc = wf_check_rows(kv, at->lim.max_rows, what);
    if (!rc) rc = check_step(step, what);
    if (rc) return rc;
    REQUIRE(in, "%s: the tensors are NULL", what);
    rc = check_layer(layer, in->dtype, what);
    if (rc) return rc;
    REQUIRE(layer->dim == at->lim.dim, "%s: heads of %d elements, scratch for %d", what, layer->dim, at->lim.dim);
    REQUIRE(in->heads >= 1 && in->heads <= at->lim.max_heads && in->heads % layer->heads == 0,
            "%s: %d query heads; a multiple of %d, up to %d", what, in->heads, layer->heads, at->lim.max_heads);
    REQUIRE(step->max_tokens * in->heads <= INT32_MAX, "%s: %lld tokens of %d heads", what, (long long)step->max_tokens, in->heads);
    REQUIRE(std::isfinite(in->scale) && in->scale >= 0, "%s: scale %g", what, in->scale);
    REQUIRE(in->new_tokens >= 0, "%s: new_tokens %d", what, in->new_tokens);
    REQUIRE(step->start && step->len && wf_aligned(step->start, 4) && wf_aligned(step->len, 4), "%s: NULL or misaligned start or len", what);
    rc = check_attn(in->q, in->q_token, in->q_head, what, "queries");
    if (!rc) rc = check_attn(in->out, in->out_token, in->out_head, what, "outputs");
    if (rc) return rc;
    REQUIRE(!meet({in->q, in->q_token, in->q_head, in->heads}, {in->out, in->out_token, in->out_head, in->heads}, step->max_tokens, 2 * layer->dim),
            "%s: outputs in the queries' memory", what);
    rc = wf_cuda_check(cudaSetDevice(at->device), "cudaSetDevice");
    if (rc) return rc;

    AttendArgs a{};
    a.table = kv->table, a.start = step->start, a.len = step->len;
    a.table_stride = kv->table_stride / 4, a.max_tokens = step->max_tokens;
    a.rows = kv->rows, a.row_blocks = kv->row_blocks, a.bs = kv->block_tokens, a.n_blocks = kv->n_blocks;
    a.k = (const uint8_t *)layer->k, a.v = (const uint8_t *)layer->v;
    a.block_stride = layer->block_stride, a.token_stride = layer->token_stride, a.head_stride = layer->head_stride;
    a.k_scale = layer->k_scale, a.v_scale = layer->v_scale, a.kv = layer->heads;
    a.q = (const uint8_t *)in->q, a.out = (uint8_t *)in->out;
    a.q_token = in->q_token, a.q_head = in->q_head, a.o_token = in->out_token, a.o_head = in->out_head;
    a.group = in->heads / layer->heads;
    a.by_bs = wf_make_div(a.bs), a.by_group = wf_make_div(a.group);
    // prompt_kernel masks scores before it scales them, and -inf * 0 is no number.  The least positive number in place of 0 keeps finite scores
    // within 2^-21 of each other (2^-149 times 2^128), so that the weights are equal; a finite scale stays finite.
    a.scale = std::clamp(in->scale * 1.4426950408889634f, FLT_TRUE_MIN, FLT_MAX);
    a.part = at->part[0], a.arrive = at->arrive[0], a.err = at->err, a.sms = at->sms;
    // Rows of up to kFew queries to a key head go to the kernel of 16-query tiles, the others to that of 128-query tiles.  Where no row is
    // expected to have more (or none can), one launch takes them all.
    const bool eight = layer->dtype == WF_E4M3;
    const int64_t expected = in->new_tokens ? std::min<int64_t>(in->new_tokens, step->max_tokens) : step->max_tokens;
    a.few = INT64_MAX, a.both = 0;
    if (expected * a.group > kFew) {
        a.tile_q = a.group <= kKeys ? kKeys / a.group * a.group : kKeys;
        a.few = kFew, a.both = !eight;
        wf_costs(layer->dim, &a);
        AttendArgs b = a;
        b.part = at->part[1], b.arrive = at->arrive[1];
        rc = wf_launch_prompt(at, b, in->dtype, layer->dim, eight, (cudaStream_t)stream);
        if (rc > 0) return rc;
        if (rc < 0) a.few = INT64_MAX, a.both = 0;
    }
    return wf_launch_attend(at, a, in->dtype, layer->dim, eight, (cudaStream_t)stream);
}
