// The calls on a replica's rows, host side: the scratch that they share and
// the checks of their arguments.
#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "wf_decode.cuh"

#define REQUIRE(cond, ...) \
    do { if (!(cond)) return wf_set_error(WF_EINVAL, __VA_ARGS__); } while (0)

static int select_device(const wf_decode *d)
{
    return wf_cuda_check(cudaSetDevice(d->device), "cudaSetDevice");
}

extern "C" int wf_decode_create(const wf_decode_limits *lim, int device, wf_decode **out)
{
    REQUIRE(out, "out is NULL");
    *out = nullptr;
    REQUIRE(lim, "limits is NULL");
    REQUIRE(lim->max_rows >= 1 && lim->max_rows <= 65536, "max_rows %d outside 1..65536", lim->max_rows);
    REQUIRE(lim->max_row_blocks >= 0 && (int64_t)lim->max_rows * lim->max_row_blocks < INT32_MAX,
            "max_rows * max_row_blocks = %d * %d", lim->max_rows, lim->max_row_blocks);
    REQUIRE(lim->max_vocab >= 0 && lim->max_vocab <= 1 << 24, "max_vocab %d outside 0..2^24", lim->max_vocab);
    REQUIRE(lim->max_keep >= 0 && lim->max_keep <= kMaxKeep, "max_keep %d outside 0..%d", lim->max_keep, kMaxKeep);
    REQUIRE(device >= 0, "device %d", device);
    int rc = wf_cuda_check(cudaSetDevice(device), "cudaSetDevice");
    if (rc) return rc;
    wf_decode *d = (wf_decode *)calloc(1, sizeof(wf_decode));
    if (!d) return wf_set_error(WF_ENOMEM, "host allocation of the decode scratch");
    d->device = device;
    d->lim = *lim;
    rc = wf_cuda_check(cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, device), "device attributes");
    if (!rc) rc = wf_extend_setup();
    if (rc) { wf_decode_destroy(d); return rc; }

    const int64_t rows = lim->max_rows;
    const int64_t tiles = (lim->max_row_blocks + kTileCols - 1) / kTileCols;
    if (lim->max_vocab && lim->max_keep) wf_beam_scratch(rows, lim->max_vocab, d->sms, &d->parts, &d->units);
    size_t at = 0;
    auto place = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const size_t o_err = place(64), o_ticket = place(4 * (1 + (size_t)rows));
    const size_t zeroed = at;
    const size_t o_sums = place(4 * (3 * (size_t)rows + 3));
    const size_t o_freed = place(4 * (size_t)(rows * tiles * kTileCols));
    const size_t o_tf = place(4 * (size_t)(rows * tiles)), o_tc = place(4 * (size_t)(rows * tiles));
    const size_t o_from = place(8 * (size_t)rows), o_rows = place(4 * (size_t)rows), o_gc = place(4 * (size_t)rows);
    const size_t o_plan = place(16 * (size_t)rows), o_was = place(sizeof(wf_ring)), o_nc = place(4);
    const size_t o_part = place(16 * (size_t)d->parts), o_most = place(4 * (size_t)d->units);
    rc = wf_cuda_check(cudaMalloc(&d->mem, at), "cudaMalloc(decode scratch)");
    if (!rc) rc = wf_cuda_check(cudaMemset(d->mem, 0, zeroed), "clear the decode scratch");
    if (rc) { wf_decode_destroy(d); return rc; }
    uint8_t *m = (uint8_t *)d->mem;
    d->err = (int *)(m + o_err);
    d->ticket = (uint32_t *)(m + o_ticket);
    d->sums = (int32_t *)(m + o_sums);
    d->freed = (int32_t *)(m + o_freed);
    d->tile_freed = (int32_t *)(m + o_tf);
    d->tile_copy = (uint32_t *)(m + o_tc);
    d->copy_from = (int2 *)(m + o_from);
    d->copy_rows = (int32_t *)(m + o_rows);
    d->n_copies = (int32_t *)(m + o_nc);
    d->group_copy = (uint32_t *)(m + o_gc);
    d->group_plan = (int4 *)(m + o_plan);
    d->ring_was = (wf_ring *)(m + o_was);
    d->part = (float4 *)(m + o_part);
    d->most = (float *)(m + o_most);
    // The clearing runs on the default stream; the calls may use any other.
    rc = wf_cuda_check(cudaDeviceSynchronize(), "cudaDeviceSynchronize");
    if (rc) { wf_decode_destroy(d); return rc; }
    *out = d;
    return WF_OK;
}

extern "C" void wf_decode_destroy(wf_decode *d)
{
    if (!d) return;
    if (d->mem) {
        cudaSetDevice(d->device);
        cudaFree(d->mem);
    }
    free(d);
}

extern "C" int wf_decode_status(wf_decode *d, void *stream)
{
    REQUIRE(d, "NULL decode scratch");
    int rc = select_device(d);
    if (rc) return rc;
    rc = wf_cuda_check(cudaStreamSynchronize((cudaStream_t)stream), "cudaStreamSynchronize");
    if (rc) return rc;
    int err = 0;
    rc = wf_cuda_check(cudaMemcpy(&err, d->err, sizeof(int), cudaMemcpyDeviceToHost), "read error word");
    if (rc) return rc;
    if (err) {
        const int zero = 0;
        rc = wf_cuda_check(cudaMemcpy(d->err, &zero, sizeof(int), cudaMemcpyHostToDevice), "clear error word");
        if (rc) return rc;
        return wf_set_error(WF_EINVAL, "a table, the ring, a slot or a copy names a block outside the cache; what was to be written there was left out");
    }
    return WF_OK;
}

static bool aligned(const void *p, size_t a) { return wf_aligned(p, a); }

// Two ranges are the same memory or have none in common.
static bool same_or_apart(const void *a, const void *b, size_t bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x == y || x + bytes <= y || y + bytes <= x;
}

int wf_check_rows(const wf_kv *kv, int32_t max_rows, const char *what)
{
    REQUIRE(kv, "%s: the rows are NULL", what);
    REQUIRE(kv->rows >= 1 && kv->rows <= max_rows, "%s: rows %d outside 1..%d", what, kv->rows, max_rows);
    REQUIRE(kv->row_blocks >= 1, "%s: row_blocks %d", what, kv->row_blocks);
    REQUIRE(kv->block_tokens >= 1, "%s: block_tokens %d", what, kv->block_tokens);
    REQUIRE(kv->n_blocks >= 1 && kv->n_blocks <= INT32_MAX - 1, "%s: n_blocks %d", what, kv->n_blocks);
    REQUIRE(kv->table && kv->len && kv->ring && kv->ends, "%s: NULL table, len, ring or ends", what);
    REQUIRE(kv->table_stride % 4 == 0 && kv->table_stride >= 4 * (int64_t)kv->row_blocks,
            "%s: table_stride %lld for %d blocks a row", what, (long long)kv->table_stride, kv->row_blocks);
    REQUIRE(aligned(kv->table, 4) && aligned(kv->len, 4) && aligned(kv->ring, 4) && aligned(kv->ends, 8),
            "%s: misaligned table, len, ring or ends", what);
    return WF_OK;
}

static int check_kv(const wf_decode *d, const wf_kv *kv, const char *what) { return wf_check_rows(kv, d->lim.max_rows, what); }

extern "C" int wf_kv_extend(wf_decode *d, const wf_kv *kv, const int32_t *add, const wf_kv_step *out, void *stream)
{
    REQUIRE(d, "NULL decode scratch");
    int rc = check_kv(d, kv, "wf_kv_extend");
    if (rc) return rc;
    REQUIRE(add && out, "wf_kv_extend: NULL add or out");
    REQUIRE(out->max_tokens >= 1 && out->max_tokens <= INT32_MAX - 1, "wf_kv_extend: max_tokens %lld",
            (long long)out->max_tokens);
    REQUIRE(out->slot && out->pos && out->row && out->start && out->len && out->ends && out->status,
            "wf_kv_extend: NULL output");
    REQUIRE(aligned(add, 4) && aligned(out->slot, 8) && aligned(out->pos, 4) && aligned(out->row, 4) &&
                aligned(out->start, 4) && aligned(out->len, 4) && aligned(out->ends, 8) && aligned(out->status, 4),
            "wf_kv_extend: misaligned array");
    REQUIRE(same_or_apart(kv->len, out->len, 4 * (size_t)kv->rows) && same_or_apart(kv->ends, out->ends, 16),
            "wf_kv_extend: len or ends overlap their inputs in part");
    rc = select_device(d);
    if (rc) return rc;
    return wf_launch_extend(d, kv, add, out, (cudaStream_t)stream);
}

extern "C" int wf_beam_select(wf_decode *d, const wf_beam *in, const wf_beam_out *out, void *stream)
{
    REQUIRE(d, "NULL decode scratch");
    REQUIRE(in && out, "wf_beam_select: NULL in or out");
    REQUIRE(in->beams >= 1 && in->beams <= kMaxGroup, "wf_beam_select: beams %d outside 1..%d", in->beams, kMaxGroup);
    REQUIRE(in->groups >= 1 && (int64_t)in->groups * in->beams <= d->lim.max_rows,
            "wf_beam_select: %d groups of %d beams, max_rows %d", in->groups, in->beams, d->lim.max_rows);
    REQUIRE(in->vocab >= 1 && in->vocab <= d->lim.max_vocab, "wf_beam_select: vocab %d outside 1..%d", in->vocab,
            d->lim.max_vocab);
    REQUIRE(in->keep >= 1 && in->keep <= d->lim.max_keep, "wf_beam_select: keep %d outside 1..%d", in->keep,
            d->lim.max_keep);
    REQUIRE(in->dtype == WF_F32 || in->dtype == WF_F16 || in->dtype == WF_BF16, "wf_beam_select: dtype %d", in->dtype);
    const size_t es = in->dtype == WF_F32 ? 4 : 2;
    REQUIRE(in->logits && in->score, "wf_beam_select: NULL logits or score");
    REQUIRE(aligned(in->logits, es) && aligned(in->score, 4), "wf_beam_select: misaligned logits or score");
    REQUIRE(in->logits_stride % (int64_t)es == 0 &&
                (in->logits_stride >= (int64_t)es * in->vocab || (int64_t)in->groups * in->beams == 1),
            "wf_beam_select: logits_stride %lld for %d tokens", (long long)in->logits_stride, in->vocab);
    REQUIRE(out->score && out->parent && out->token, "wf_beam_select: NULL output");
    const int given = !!out->next_score + !!out->next_parent + !!out->next_token;
    REQUIRE(given == 0 || given == 3, "wf_beam_select: next_score, next_parent and next_token go together");
    REQUIRE(aligned(out->score, 4) && aligned(out->parent, 4) && aligned(out->token, 4) && aligned(out->next_score, 4) &&
                aligned(out->next_parent, 4) && aligned(out->next_token, 4), "wf_beam_select: misaligned output");
    int rc = select_device(d);
    if (rc) return rc;
    return wf_launch_select(d, in, out, (cudaStream_t)stream);
}

extern "C" int wf_kv_reorder(wf_decode *d, const wf_kv *kv, int32_t group, const int32_t *parent, const wf_kv *to,
                             const wf_kv_cache *cache, int32_t *copies, uint32_t *status, void *stream)
{
    REQUIRE(d, "NULL decode scratch");
    int rc = check_kv(d, kv, "wf_kv_reorder");
    if (!rc) rc = check_kv(d, to, "wf_kv_reorder (to)");
    if (rc) return rc;
    REQUIRE(kv->row_blocks <= d->lim.max_row_blocks, "wf_kv_reorder: row_blocks %d above %d", kv->row_blocks,
            d->lim.max_row_blocks);
    REQUIRE(group >= 1 && group <= kMaxGroup && kv->rows % group == 0, "wf_kv_reorder: %d rows in groups of %d",
            kv->rows, group);
    REQUIRE(to->rows == kv->rows && to->row_blocks == kv->row_blocks && to->block_tokens == kv->block_tokens &&
                to->n_blocks == kv->n_blocks && to->ring == kv->ring, "wf_kv_reorder: sizes or ring of `to` differ");
    REQUIRE(parent && copies && status, "wf_kv_reorder: NULL parent, copies or status");
    REQUIRE(aligned(parent, 4) && aligned(copies, 4) && aligned(status, 4), "wf_kv_reorder: misaligned array");
    const size_t span = (size_t)(kv->rows - 1) * (size_t)std::max(kv->table_stride, to->table_stride) +
                        4 * (size_t)kv->row_blocks;
    REQUIRE(same_or_apart(kv->table, to->table, span) && (kv->table != to->table || kv->table_stride == to->table_stride),
            "wf_kv_reorder: the tables overlap in part");
    REQUIRE(same_or_apart(kv->len, to->len, 4 * (size_t)kv->rows) && same_or_apart(kv->ends, to->ends, 16),
            "wf_kv_reorder: len or ends overlap their inputs in part");
    if (cache) {
        REQUIRE(cache->base && cache->planes >= 1 && cache->token_bytes >= 1 && cache->reserved == 0,
                "wf_kv_reorder: NULL cache, %d planes of %lld bytes a token", cache->planes,
                (long long)cache->token_bytes);
        REQUIRE(cache->token_bytes <= (INT64_MAX / kv->n_blocks) / kv->block_tokens,
                "wf_kv_reorder: token_bytes %lld", (long long)cache->token_bytes);
        const int64_t plane = cache->token_bytes * kv->block_tokens * kv->n_blocks;
        REQUIRE(cache->planes == 1 || cache->plane_stride >= plane, "wf_kv_reorder: plane_stride %lld below %lld",
                (long long)cache->plane_stride, (long long)plane);
    }
    rc = select_device(d);
    if (rc) return rc;
    return wf_launch_reorder(d, kv, group, parent, to, cache, copies, status, (cudaStream_t)stream);
}
