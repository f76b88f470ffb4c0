// The calls on a layer's tensors, host side: the checks of their arguments.
#include <cmath>

#include "wf_decode.cuh"
#include "wf_layer.cuh"

#define REQUIRE(cond, ...) \
    do { if (!(cond)) return wf_set_error(WF_EINVAL, __VA_ARGS__); } while (0)

static int check_step(const wf_kv *kv, const wf_kv_step *step, const char *what)
{
    REQUIRE(step, "%s: the step is NULL", what);
    REQUIRE(step->max_tokens >= 1 && step->max_tokens <= INT32_MAX - 1, "%s: max_tokens %lld", what, (long long)step->max_tokens);
    (void)kv;
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

extern "C" int wf_kv_write(wf_decode *d, const wf_kv *kv, const wf_kv_step *step, const wf_kv_layer *layer, const wf_rope *rope,
                           const wf_kv_new *in, void *stream)
{
    const char *what = "wf_kv_write";
    REQUIRE(d, "NULL decode scratch");
    int rc = wf_check_rows(kv, d->lim.max_rows, what);
    if (!rc) rc = check_step(kv, step, what);
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
