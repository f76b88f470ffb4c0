"""Calls on a replica's rows against plain implementations: block tables and
slots, the beams' selection, the reordering of a paged cache."""
import ctypes
import math

import numpy as np
import pytest

import decode_ref as ref
from gpu_util import lib

pytestmark = pytest.mark.gpu


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def host(t):
    return t.cpu().numpy()


def same(got, want):
    for k, w in want.items():
        g = got[k]
        bad = np.argwhere(g != w)
        assert g.shape == w.shape and not len(bad), f"{k}: {len(bad)} differ, first at {bad[0]}: {g[tuple(bad[0])]}, not {w[tuple(bad[0])]}"


# ---------------------------------------------------------------------------
# Extend
# ---------------------------------------------------------------------------

def pool(rng, used, free, spare=3, base=None):
    n = max(1, used + free + spare)
    ids = rng.permutation(n).astype(np.int32)
    head = int(rng.integers(0, 5 * n)) if base is None else base
    ring = np.full(n, -9, np.int32)
    ring[(head + np.arange(free)) % n] = ids[used:used + free]
    return ids[:used], ring, np.array([head, head + free], np.int64)


def extend_inputs(rng, rows, bs, ctx, new, room=1.0, bad=False, base=None):
    length = rng.integers(0, ctx + 1, rows).astype(np.int32)
    add = rng.integers(0, new + 1, rows).astype(np.int32)
    width = -(-(ctx + new) // bs) + 1
    if bad:
        length[rng.integers(0, rows, 3)] = -1
        add[rng.integers(0, rows, 3)] = -5
        add[rng.integers(0, rows, 3)] = width * bs + 1
        add[rng.integers(0, rows, 2)] = np.iinfo(np.int32).max
    have = -(-np.maximum(length, 0).astype(np.int64) // bs)
    ok = (length >= 0) & (add >= 0)
    then = -(-(length.astype(np.int64) + add) // bs)
    need = int((then - have)[ok & (then <= width)].sum())
    ids, ring, ends = pool(rng, int(have.sum()), int(need * room), base=base)
    table = np.full((rows, width), -1, np.int32)
    table[np.arange(width) < have[:, None]] = ids
    return table, length, add, ring, ends


def run_extend(wf, table, length, add, ring, ends, bs, max_tokens, offset=0, stride=0, decode=None, stream=None):
    import torch
    d = decode or wf.Decode(max_rows=table.shape[0])
    full = torch.full((table.shape[0], table.shape[1] + stride), -1, dtype=torch.int32, device="cuda")
    full[:, :table.shape[1]] = dev(table)
    kv = wf.Kv(full[:, :table.shape[1]], dev(length), dev(ring), dev(ends), bs)
    out = wf.KvStep(kv.rows, max_tokens)
    if offset:  # outputs that are not on 16-byte boundaries
        out.slot, out.pos, out.row = (torch.empty(max_tokens + offset, dtype=t.dtype, device="cuda")[offset:]
                                      for t in (out.slot, out.pos, out.row))
        out.c.slot, out.c.pos, out.c.row = out.slot.data_ptr(), out.pos.data_ptr(), out.row.data_ptr()
    wf.wf_kv_extend(d, kv, dev(add), out, stream=stream)
    torch.cuda.synchronize()
    return dict(table=host(kv.table), slot=host(out.slot), pos=host(out.pos), row=host(out.row), start=host(out.start),
                len=host(out.len), ends=host(out.ends), status=host(out.status))


@pytest.mark.parametrize("rows,bs,ctx,new,tokens,room,bad", [
    (1, 16, 0, 1, 1, 1.0, False), (1, 16, 100, 0, 5, 1.0, False), (1, 1, 40, 33, 64, 1.0, False),
    (12, 16, 900, 1, 16, 1.0, False), (33, 7, 100, 50, 1000, 1.0, True), (169, 24, 3000, 128, 8192, 1.0, True),
    (512, 64, 1000, 3, 1024, 0.5, True), (513, 5, 60, 70, 20001, 0.8, True), (2000, 16, 300, 1, 2048, 1.0, True),
    (700, 1, 5, 9, 2999, 1.0, True), (1000, 128, 4000, 400, 65537, 0.9, True), (64, 1000, 9000, 5000, 170001, 1.0, True),
    (8192, 16, 200, 2, 8192, 1.0, True), (16384, 16, 40, 2, 20000, 1.0, True), (16385, 16, 40, 3, 40000, 1.0, True),
    (20000, 3, 10, 5, 30001, 0.9, True), (3, 16, 10, 0, 7, 1.0, False), (40, 16, 10, 300, 10, 1.0, False),
    (40, 16, 10, 300, 4000, 0.0, False)])
def test_extend_matches_the_row_by_row_form(rows, bs, ctx, new, tokens, room, bad):
    wf = lib()
    rng = np.random.default_rng(rows * 1000 + bs)
    args = extend_inputs(rng, rows, bs, ctx, new, room, bad)
    want = ref.extend(*args, bs, tokens)
    same(run_extend(wf, *args, bs, tokens), want)
    same(run_extend(wf, *args, bs, tokens, offset=1, stride=5), want)


def test_extend_counts_past_32_bits():
    """Ring positions past 2^40, slots past 2^32."""
    wf = lib()
    rng = np.random.default_rng(5)
    bs, n = 256, 20_000_000
    ring = np.arange(n, dtype=np.int32)[::-1].copy()
    head = (1 << 40) // n * n + n - 7  # wraps after 7 blocks; the first ids are the last in the pool
    ends = np.array([head, head + n // 2], np.int64)
    ring[:50] = n - 1 - np.arange(50, dtype=np.int32)
    table = np.full((9, 8), -1, np.int32)
    length = np.array([0, 0, 256, 300, 1, 0, 511, 512, 0], np.int32)
    table[2, 0], table[3, :2], table[4, 0], table[6, :2], table[7, :2] = n - 60, (n - 61, n - 62), n - 63, (n - 64, n - 65), (n - 66, n - 67)
    add = rng.integers(1, 1024, 9).astype(np.int32)
    want = ref.extend(table, length, add, ring, ends, bs, 10000)
    assert want["slot"].max() > 1 << 32
    same(run_extend(wf, table, length, add, ring, ends, bs, 10000), want)


def test_extend_sums_that_pass_31_bits_end_the_line():
    wf = lib()
    add = np.full(600, np.iinfo(np.int32).max, np.int32)
    add[0] = 3
    table = np.full((600, 8), -1, np.int32)
    length = np.zeros(600, np.int32)
    ring = np.arange(100, dtype=np.int32)
    bs = 1 << 30  # a table row holds 2^33 tokens
    want = ref.extend(table, length, add, ring, np.array([0, 100], np.int64), bs, 1000)
    assert (want["status"][1:] & wf.KV_TOKENS).all() and want["start"][-1] == 3
    same(run_extend(wf, table, length, add, ring, np.array([0, 100], np.int64), bs, 1000), want)


def test_extend_in_place_steps_streams_and_graph():
    """The state moves on over steps, on a stream of its own and replayed from a graph."""
    import torch
    wf = lib()
    rng = np.random.default_rng(11)
    rows, bs, width, n = 300, 16, 30, 4000
    d = wf.Decode(max_rows=rows)
    kv = wf.Kv.empty(rows, width, bs, n)
    step = wf.KvStep(rows, 4096, kv)
    add = torch.zeros(rows, dtype=torch.int32, device="cuda")
    state = dict(table=host(kv.table), len=host(kv.len), ends=host(kv.ends))
    ring = host(kv.ring)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        wf.wf_kv_extend(d, kv, add, step)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wf.wf_kv_extend(d, kv, add, step)
    torch.cuda.synchronize()
    for i in range(6):
        a = rng.integers(0, 25, rows).astype(np.int32) if i % 2 == 0 else np.ones(rows, np.int32)
        want = ref.extend(state["table"], state["len"], a, ring, state["ends"], bs, 4096)
        add.copy_(dev(a))
        torch.cuda.synchronize()
        if i < 3:
            with torch.cuda.stream(side):
                wf.wf_kv_extend(d, kv, add, step)
        else:
            graph.replay()
        torch.cuda.synchronize()
        same(dict(table=host(kv.table), slot=host(step.slot), pos=host(step.pos), row=host(step.row), start=host(step.start),
                  len=host(kv.len), ends=host(kv.ends), status=host(step.status)), want)
        state = want


# ---------------------------------------------------------------------------
# Select
# ---------------------------------------------------------------------------

def run_select(wf, logits, score, beams, keep, eos=-1, decode=None):
    import torch
    groups = logits.shape[0] // beams
    d = decode or wf.Decode(max_rows=logits.shape[0], max_vocab=logits.shape[1], max_keep=keep)
    out = wf.BeamOut(groups, beams, keep)
    wf.wf_beam_select(d, logits, score, out, eos=eos)
    torch.cuda.synchronize()
    return out


def check_select(logits, score, beams, keep, out, eos=-1):
    """The sums lie within the 32-bit form's rounding of the 64-bit ones, and candidates whose sums are further apart
    than that are in the right order.

    The bound: Z is a sum of at most 64 values in a thread, 5 + 8 across a CTA and 13 (two warps' steps of up to
    2^8 chunks) across chunks, so it is off by at most 90 * 2^-24, and each term by 2^-21 (the approximate 2^x and its
    argument); log, the differences and the two additions round at the size of what they return."""
    x = logits.float().cpu().numpy()
    s = score.float().cpu().numpy().reshape(-1)
    best = ref.select(x, s, beams, keep)
    got_s, got_p, got_t = host(out.score), host(out.parent), host(out.token)
    every = ref.sums(x, s)
    for g, want in enumerate(best):
        n = len(want)
        assert (got_t[g, n:] == -1).all() and (got_p[g, n:] == -1).all() and (got_s[g, n:] == -np.inf).all()
        mine = [(int(p), int(t)) for p, t in zip(got_p[g, :n], got_t[g, :n])]
        assert len(set(mine)) == n and all(g * beams <= p < (g + 1) * beams for p, _ in mine)
        for i, (c, p, t) in enumerate(want):
            far = 90 * 2.0 ** -24 + 2.0 ** -21 + 6 * 2.0 ** -24 * (abs(c) + 2 * abs(float(s[p])) + math.log(x.shape[1]) + 1)
            assert abs(every[mine[i]] - c) <= 2 * far, (g, i, mine[i], (p, t))
            assert got_s[g, i] == c or abs(got_s[g, i] - c) <= far, (g, i, got_s[g, i], c)
            apart = [abs(want[j][0] - c) > 2 * far for j in (i - 1, i + 1) if 0 <= j < n]
            if all(apart) and (i + 1 < n or n < keep):
                assert mine[i] == (p, t), (g, i, mine[i], (p, t))
        onward = [i for i in range(n) if mine[i][1] != eos][:beams]
        k = len(onward)
        assert [int(v) for v in host(out.next_parent)[g]] == [mine[i][0] for i in onward] + [-1] * (beams - k)
        assert [int(v) for v in host(out.next_token)[g]] == [mine[i][1] for i in onward] + [-1] * (beams - k)
        assert host(out.next_score)[g].tolist() == [got_s[g, i] for i in onward] + [-np.inf] * (beams - k)


def logits_of(rng, rows, vocab, dtype, scale=2.0):
    import torch
    x = rng.standard_normal((rows, vocab)) * scale
    for r in range(rows):
        at = rng.integers(0, vocab, min(vocab, 12))
        x[r, at] = 5 + 7 * rng.random(len(at))
    return torch.from_numpy(x.astype(np.float32)).cuda().to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("groups,beams,vocab,keep", [
    (1, 1, 1, 1), (1, 1, 1, 7), (2, 3, 2, 6), (1, 4, 17, 8), (5, 2, 255, 4), (3, 4, 2049, 8), (1, 4, 32000, 8),
    (7, 5, 4999, 10), (16, 4, 50257, 8), (2, 32, 8191, 64), (1, 32, 700, 64), (3, 8, 65536, 33), (40, 1, 3001, 2),
    (1, 2, 600_001, 32), (300, 3, 4100, 6)])
def test_select_matches_the_64_bit_form(groups, beams, vocab, keep, dtype):
    wf = lib()
    rng = np.random.default_rng(groups * 7 + vocab)
    logits = logits_of(rng, groups * beams, vocab, dtype)
    score = dev((-rng.random(groups * beams) * 20).astype(np.float32))
    eos = int(host(logits.float().argmax(1))[0])
    out = run_select(wf, logits, score, beams, keep, eos)
    check_select(logits, score, beams, keep, out, eos)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("offset", [1, 3, 6])
def test_select_rows_that_start_anywhere(dtype, offset):
    """A view into wider rows whose first element lies on no 16-byte boundary; NaN around it must not be read in."""
    import torch
    wf = lib()
    rng = np.random.default_rng(offset)
    for vocab in (5, 64, 1003):
        wide = torch.full((6, vocab + 11), math.nan, dtype=getattr(torch, dtype), device="cuda")
        logits = wide[:, offset:offset + vocab]
        logits.copy_(logits_of(rng, 6, vocab, dtype))
        score = dev((-rng.random(6) * 3).astype(np.float32))
        check_select(logits, score, 3, 6, run_select(wf, logits, score, 3, 6))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_select_masks_infinities_and_nan(dtype):
    import torch
    wf = lib()
    rng = np.random.default_rng(3)
    vocab, beams, keep = 9001, 4, 8
    t = getattr(torch, dtype)
    x = logits_of(rng, 40, vocab, dtype)
    score = -torch.rand(40, device="cuda") * 5
    low = torch.finfo(t).min
    some = torch.from_numpy(rng.random((40, vocab)) < 0.999).cuda()
    x[0:4][some[0:4]] = -math.inf           # most masked
    x[4:8][some[4:8]] = low                 # ... by the lowest value
    x[8:12] = -math.inf                     # all masked
    x[12:16] = low                          # all at the lowest value
    x[16] = -math.inf                       # one empty row
    x[17, ::7] = math.nan
    x[18] = math.nan
    x[19, 5:] = -math.inf
    x[20, [3, 4000, 8999]] = math.inf
    x[21, 17] = math.inf
    score[22] = -math.inf
    score[23] = math.nan
    score[24:28] = -math.inf                # an empty search
    x[28:32, 1:] = -math.inf                # one token each
    x[32] = -math.inf
    x[32, 8000] = low
    check_select(x, score, beams, keep, run_select(wf, x, score, beams, keep))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("keep", [1, 8, 33, 64])
def test_select_equal_values_go_to_the_first(dtype, keep):
    """Constant rows: equal sums go to the lower beam, then to the lower token."""
    import torch
    wf = lib()
    for vocab, beams in ((40, 2), (5000, 3), (70000, 2)):
        x = torch.full((2 * beams, vocab), 1.5, dtype=getattr(torch, dtype), device="cuda")
        x[beams:] = -0.0
        x[beams:, ::2] = 0.0  # the same value
        score = torch.full((2 * beams,), -2.0, device="cuda")
        out = run_select(wf, x, score, beams, keep)
        n = min(keep, vocab * beams)
        for g in range(2):
            assert host(out.parent)[g, :n].tolist() == [g * beams + i // vocab for i in range(n)]
            assert host(out.token)[g, :n].tolist() == [i % vocab for i in range(n)]
        # A lower beam goes first even where the other's token is lower.
        x[:] = -3
        x[0, 30], x[1, 7] = 4, 4
        out = run_select(wf, x, score, beams, keep)
        assert host(out.token)[0, 0] == 30 and host(out.parent)[0, 0] == 0
        if keep > 1:
            assert host(out.token)[0, 1] == 7 and host(out.parent)[0, 1] == 1


@pytest.mark.parametrize("groups,beams,vocab,dtype", [(1, 3, 4097, "bfloat16"), (2, 5, 50257, "float16"), (30, 7, 9001, "float32"),
                                                      (3, 32, 2000, "bfloat16"), (200, 6, 700, "bfloat16"), (9, 16, 40000, "bfloat16")])
def test_select_equal_rows_have_equal_sums(groups, beams, vocab, dtype):
    """Beams with the same logits and scores: to the last bit the same sums, so a logit's candidates go by beam, a
    beam's by token."""
    import torch
    wf = lib()
    rng = np.random.default_rng(vocab)
    x = logits_of(rng, groups, vocab, dtype).repeat_interleave(beams, 0).contiguous()
    score = torch.full((groups * beams,), -3.7, device="cuda")
    keep = min(64, 2 * beams)
    out = run_select(wf, x, score, beams, keep)
    parent, token, got = host(out.parent) % beams, host(out.token), host(out.score)
    for g in range(groups):
        row = host(x[g * beams].float())
        want = []
        for value in np.unique(row)[::-1]:
            want += [(k, int(t)) for k in range(beams) for t in np.flatnonzero(row == value)]
            if len(want) >= keep:
                break
        assert list(zip(parent[g].tolist(), token[g].tolist())) == want[:keep]
        at = row[token[g]]
        assert all(len(set(got[g][at == v].tolist())) == 1 for v in np.unique(at))


def test_select_orders_that_defeat_the_bound():
    """Values whose large ones all lie with a few threads: more reach the bound than are gathered."""
    import torch
    wf = lib()
    vocab = 30000
    ramp = torch.arange(vocab, device="cuda", dtype=torch.float32)
    for x in (ramp * 1e-3, -ramp * 1e-3, torch.where((ramp // 4) % 32 < 1, 10 + ramp * 1e-4, -ramp * 1e-4),
              torch.where((ramp // 128) % 2 == 0, (ramp % 128) * 1e-2 + 5, -ramp * 1e-4),
              torch.where(ramp % 1024 < 700, 3.0, ramp * 1e-6)):
        logits = torch.stack([x, x.flip(0)]).contiguous()
        score = torch.tensor([-1.0, -1.25], device="cuda")
        for keep in (4, 20, 64):
            check_select(logits, score, 2, keep, run_select(wf, logits, score, 2, keep))


@pytest.mark.parametrize("groups,beams,vocab", [(1, 3, 300), (40, 8, 30_000)])
def test_select_scores_in_place(groups, beams, vocab):
    """next_score may be the scores themselves, over steps."""
    import torch
    wf = lib()
    rng = np.random.default_rng(6)
    d = wf.Decode(max_rows=groups * beams, max_vocab=vocab, max_keep=2 * beams)
    score = dev((-rng.random(groups * beams)).astype(np.float32))
    here, apart = wf.BeamOut(groups, beams, 2 * beams, score), wf.BeamOut(groups, beams, 2 * beams)
    for _ in range(3):
        x = logits_of(rng, groups * beams, vocab, "float32")
        wf.wf_beam_select(d, x, score.clone(), apart)
        wf.wf_beam_select(d, x, score, here)
        for a, b in ((here.next_score.view(-1), apart.next_score.view(-1)), (here.token, apart.token), (here.next_parent, apart.next_parent)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("mask", [-40.0, -100.0, -1000.0, -9999.0, -1e9])
def test_select_masks_of_any_low_value(mask):
    """Parts of rows that start with a mask of a finite value."""
    wf = lib()
    rng = np.random.default_rng(31)
    for vocab in (3000, 60_000):
        x = logits_of(rng, 6, vocab, "float32")
        x[0, :vocab // 2] = mask
        x[1, vocab // 7:] = mask
        x[2, ::2] = mask
        x[3] = mask
        x[4, :vocab - 3] = mask
        score = dev((-rng.random(6)).astype(np.float32))
        check_select(x, score, 3, 6, run_select(wf, x, score, 3, 6))


def test_select_repeats_and_scratch_is_left_clean():
    """Calls of different sizes in turn on one scratch, twice with the same result to the last bit."""
    import torch
    wf = lib()
    rng = np.random.default_rng(8)
    d = wf.Decode(max_rows=64, max_vocab=20000, max_keep=16)
    seen = []
    for _ in range(2):
        rng = np.random.default_rng(8)
        for beams, groups, vocab, keep in ((4, 3, 20000, 8), (1, 64, 100, 16), (8, 8, 3333, 16), (2, 1, 19999, 1)):
            x = logits_of(rng, groups * beams, vocab, "bfloat16")
            s = dev(-rng.random(groups * beams).astype(np.float32))
            out = run_select(wf, x, s, beams, keep, decode=d)
            seen.append([host(v) for v in (out.score, out.parent, out.token, out.next_score, out.next_parent, out.next_token)])
    for a, b in zip(seen[:4], seen[4:]):
        assert all(np.array_equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("dtype,groups,beams,vocab,keep", [
    ("bfloat16", 1, 32, 200_003, 64), ("float32", 2, 16, 65537, 32), ("float16", 1, 1, 1 << 24, 8), ("float32", 500, 1, 999, 3),
    ("bfloat16", 700, 2, 513, 4), ("bfloat16", 5, 7, 30000, 17)])
def test_select_over_few_and_many_units(dtype, groups, beams, vocab, keep):
    """Searches cut into units of one line, of two, of many; more searches than the machine holds at once."""
    wf = lib()
    rng = np.random.default_rng(vocab)
    logits = logits_of(rng, groups * beams, vocab, dtype)
    score = dev((-rng.random(groups * beams) * 9).astype(np.float32))
    check_select(logits, score, beams, keep, run_select(wf, logits, score, beams, keep))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("vocab", [700, 70001])
def test_select_sums_that_leave_a_floats_range(dtype, vocab):
    """Exponentials relative to a value at the start of a row's part that says little about the rest: masked, far
    below it, far above it."""
    import torch
    wf = lib()
    rng = np.random.default_rng(17)
    x = logits_of(rng, 8, vocab, dtype)
    x[0] -= 200
    x[1, :vocab // 2] = -math.inf
    x[1] -= 95
    x[2, :vocab // 3] -= 60
    x[2, vocab // 2:] += 300
    x[3, :64] = -math.inf
    x[3, 64:] -= 93
    x[4] = -20000.0 + x[4]
    x[5, ::2] = torch.finfo(x.dtype).min
    x[6] += 9000
    x[7, vocab // 2:] = -math.inf
    score = torch.zeros(8, device="cuda")
    check_select(x, score, 2, 8, run_select(wf, x, score, 2, 8))


def test_select_first_step_reads_the_live_beams_alone():
    """One live beam of each search, the others empty with logits of NaN."""
    import torch
    wf = lib()
    rng = np.random.default_rng(2)
    for groups, beams, vocab in ((3, 4, 500), (20, 8, 40_000)):
        x = logits_of(rng, groups * beams, vocab, "bfloat16")
        score = torch.full((groups * beams,), -math.inf, device="cuda")
        score[beams // 2::beams] = -1.5
        x[~(score > -math.inf)] = math.nan
        out = run_select(wf, x, score, beams, 2 * beams)
        check_select(x, score, beams, 2 * beams, out)
        assert (host(out.parent) % beams == beams // 2).all()


@pytest.mark.parametrize("groups,beams,vocab,keep,dtype", [
    (160, 3, 1003, 6, "float16"), (160, 4, 8200, 8, "bfloat16"), (170, 2, 3001, 33, "float32"), (153, 1, 1, 2, "float32"),
    (152, 2, 257, 3, "bfloat16"), (10, 32, 60_001, 64, "bfloat16"), (6, 32, 100_001, 40, "float32"), (65, 8, 70_000, 16, "float16"),
    (64, 8, 65_520, 16, "bfloat16"), (63, 8, 65_520, 16, "bfloat16")])
def test_select_on_both_sides_of_the_ctas_sizes(groups, beams, vocab, keep, dtype):
    """More searches than SMs, or many logits, beside one less."""
    wf = lib()
    rng = np.random.default_rng(groups + vocab)
    logits = logits_of(rng, groups * beams, vocab, dtype)
    score = dev((-rng.random(groups * beams) * 9).astype(np.float32))
    check_select(logits, score, beams, keep, run_select(wf, logits, score, beams, keep))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("vocab,offset", [(700, 0), (1003, 3), (4097, 1)])
def test_select_of_many_searches_masks_infinities_and_order(dtype, vocab, offset):
    """More searches than SMs: views that start anywhere, masks, infinities, NaN, parts far apart, equal values, values
    whose large ones lie with a few threads."""
    import torch
    wf = lib()
    rng = np.random.default_rng(vocab)
    t, groups, beams, keep = getattr(torch, dtype), 165, 2, 8
    low = torch.finfo(t).min
    wide = torch.full((groups * beams, vocab + 8), math.nan, dtype=t, device="cuda")
    x = wide[:, offset:offset + vocab]
    x.copy_(logits_of(rng, groups * beams, vocab, dtype))
    score = dev((-rng.random(groups * beams) * 3).astype(np.float32))
    some = torch.from_numpy(rng.random((beams, vocab)) < 0.99).cuda()
    x[0:2][some] = -math.inf
    x[2:4][some] = low
    x[4:6] = -math.inf
    x[6:8] = low
    x[8, ::7] = math.nan
    x[9] = math.nan
    x[10, [3, 400]] = math.inf
    x[12, :vocab // 2] = -1000.0
    x[13, 5:] = -math.inf
    x[14] -= 200
    x[15, vocab // 2:] += 300
    score[16] = -math.inf
    score[17] = math.nan
    score[18:20] = -math.inf
    x[20:22, 1:] = -math.inf
    x[22:24] = torch.arange(vocab, device="cuda").to(t) * 1e-3
    x[24:26] = (-torch.arange(vocab, device="cuda") * 1e-3).to(t)
    x[26:28] = torch.where((torch.arange(vocab, device="cuda") // 4) % 32 < 1, 6.0, -1.0).to(t)
    check_select(x, score, beams, keep, run_select(wf, x, score, beams, keep))
    # Equal rows, equal values: by beam, then by token.
    x[:] = 1.5
    score[:] = -2.0
    out = run_select(wf, x, score, beams, keep)
    assert (host(out.parent) == np.arange(groups)[:, None] * beams).all()
    assert (host(out.token) == np.arange(keep)).all()


# ---------------------------------------------------------------------------
# Reorder
# ---------------------------------------------------------------------------

def beam_rows(rng, groups, beams, bs, width, lockstep=True):
    """Tables as a search leaves them: prefixes shared in growing subsets."""
    rows = groups * beams
    length = np.zeros(rows, np.int32)
    cells = [[None] * 0 for _ in range(rows)]
    fresh = 0
    for g in range(groups):
        n = int(rng.integers(0, width * bs + 1))
        for k in range(beams):
            r = g * beams + k
            length[r] = n if lockstep else int(rng.integers(0, width * bs + 1))
            nb = -(-int(length[r]) // bs)
            if k and rng.random() < 0.8:  # shares a prefix of a lower row
                q = g * beams + int(rng.integers(0, k))
                m = int(rng.integers(0, min(nb, len(cells[q])) + 1))
                if rng.random() < 0.3:
                    m = min(nb, len(cells[q]))
                cells[r] = cells[q][:m]
            else:
                cells[r] = []
            while len(cells[r]) < nb:
                cells[r].append(fresh)
                fresh += 1
    return length, cells, fresh


def reorder_inputs(rng, groups, beams, bs, width, free, lockstep=True, parents=None):
    length, cells, used = beam_rows(rng, groups, beams, bs, width, lockstep)
    ids, ring, ends = pool(rng, used, free)
    rows = groups * beams
    table = np.full((rows, width), -1, np.int32)
    for r, c in enumerate(cells):
        table[r, :len(c)] = ids[c]
    parent = np.repeat(np.arange(groups) * beams, beams) + rng.integers(0, beams, rows)
    if parents == "ended":
        parent[rng.random(rows) < 0.5] = -1
        parent[:beams] = -1
    elif parents == "wrong":
        parent[rng.integers(0, rows, 4)] = rows + 3
        parent[rng.integers(0, rows, 4)] = -2
        if groups > 1:
            parent[0], parent[-1] = rows - 1, 0
    elif parents == "same":
        parent = np.arange(rows)
    elif parents == "one":
        parent = np.repeat(np.arange(groups) * beams + beams - 1, beams)
    return table, length, ring, ends, parent.astype(np.int32)


def run_reorder(wf, table, length, ring, ends, bs, beams, parent, in_place, cache=None, stride=0):
    import torch
    rows, width = table.shape
    d = wf.Decode(max_rows=rows, max_row_blocks=width)
    full = torch.full((rows, width + stride), -1, dtype=torch.int32, device="cuda")
    full[:, :width] = dev(table)
    kv = wf.Kv(full[:, :width], dev(length), dev(ring), dev(ends), bs)
    to = kv if in_place else wf.Kv(dev(np.full((rows, width), -1, np.int32)), torch.empty_like(kv.len), kv.ring,
                                   torch.empty_like(kv.ends), bs)
    out = wf.KvMoves(rows)
    c = None if cache is None else dev(cache)
    wf.wf_kv_reorder(d, kv, beams, dev(parent), to, out, cache=c)
    wf.wf_decode_status(d)
    got = dict(table=host(to.table), len=host(to.len), ring=host(to.ring), ends=host(to.ends), copies=host(out.copies),
               status=host(out.status))
    if not in_place:
        assert np.array_equal(host(kv.table), table) and np.array_equal(host(kv.len), length)
    return got if cache is None else dict(got, cache=host(c))


@pytest.mark.parametrize("groups,beams,bs,width,free,lockstep,parents,token_bytes", [
    (1, 1, 16, 4, 5, True, None, 0), (1, 4, 16, 40, 8, True, None, 32), (16, 12, 16, 30, 200, True, None, 16),
    (5, 8, 16, 300, 50, True, None, 0), (3, 32, 4, 70, 100, True, None, 4), (2, 32, 16, 520, 64, True, "one", 48),
    (7, 3, 5, 11, 40, False, None, 6), (9, 5, 1, 20, 40, False, None, 3), (20, 4, 64, 3, 0, True, None, 20),
    (20, 4, 64, 3, 7, True, "one", 16), (11, 6, 16, 25, 80, True, "ended", 16), (11, 6, 16, 25, 80, False, "wrong", 16),
    (10, 4, 16, 260, 30, True, "same", 16), (700, 2, 8, 6, 900, True, None, 8), (1200, 1, 16, 3, 3, True, "ended", 0),
    (6, 4, 16, 257, 30, False, "ended", 64), (2, 5, 2000, 2, 20, True, None, 32)])
@pytest.mark.parametrize("in_place", [False, True])
def test_reorder_matches_the_row_by_row_form(groups, beams, bs, width, free, lockstep, parents, token_bytes, in_place):
    wf = lib()
    rng = np.random.default_rng(groups * 100 + beams + bs)
    table, length, ring, ends, parent = reorder_inputs(rng, groups, beams, bs, width, free, lockstep, parents)
    cache = rng.integers(0, 256, (3, ring.size, bs, token_bytes)).astype(np.uint8) if token_bytes else None
    want = ref.reorder(table, length, ring, ends, bs, beams, parent, table if in_place else np.full_like(table, -1), cache)
    same(run_reorder(wf, table, length, ring, ends, bs, beams, parent, in_place, cache, stride=3 if groups % 2 else 0), want)


def test_reorder_in_place_leaves_what_lies_past_a_row():
    """A row that gets shorter keeps its old entries past its blocks, in place."""
    wf = lib()
    table = np.array([[5, 6, 7], [8, -1, -1]], np.int32)
    args = (table, np.array([40, 10], np.int32), np.arange(12, dtype=np.int32), np.array([0, 0], np.int64), 16, 2,
            np.array([1, -1], np.int32))
    got = run_reorder(wf, *args, True)
    assert got["table"][0].tolist() == [8, 6, 7] and got["len"].tolist() == [10, 0]
    assert got["ring"][:3].tolist() == [5, 6, 7] and got["ends"].tolist() == [0, 3]


def test_reorder_names_blocks_outside_the_cache():
    """A corrupt entry: its copy is left out and the status says so; nothing out of range is touched."""
    wf = lib()
    import torch
    table = np.array([[1, 99], [1, 99]], np.int32)
    d = wf.Decode(max_rows=2, max_row_blocks=2)
    kv = wf.Kv(dev(table), dev(np.array([20, 20], np.int32)), dev(np.arange(4, dtype=np.int32)), dev(np.array([2, 4])), 16)
    cache = torch.zeros((1, 4, 16, 8), dtype=torch.uint8, device="cuda")
    out = wf.KvMoves(2)
    wf.wf_kv_reorder(d, kv, 2, dev(np.array([0, 1], np.int32)), kv, out, cache=cache)
    with pytest.raises(wf.WfError) as e:
        wf.wf_decode_status(d)
    assert e.value.code == wf.WF_EINVAL
    assert host(out.copies).tolist() == [[-1, -1], [-1, -1]] and not host(cache).any()
    wf.wf_decode_status(d)


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("beams,bs", [(1, 4), (3, 4), (4, 16), (8, 3)])
def test_search_over_a_paged_cache_keeps_every_hypothesis(beams, bs):
    """Select, reorder and extend in turn, in place: the tokens read through the block tables are the hypotheses'
    own, and every block is free or held in one group."""
    import torch
    wf = lib()
    rng = np.random.default_rng(beams * 10 + bs)
    groups, vocab, steps, prompt = 5, 211, 23, 10
    rows, width = groups * beams, -(-(prompt + steps) // bs) + 1
    n = rows * width + 8
    d = wf.Decode(max_rows=rows, max_row_blocks=width, max_vocab=vocab, max_keep=2 * beams)
    kv, moves = wf.Kv.empty(rows, width, bs, n), wf.KvMoves(rows)
    cache = torch.zeros((2, n, bs, 4), dtype=torch.int32, device="cuda")  # a token's id in place of its keys
    flat = cache.view(2, n * bs, 4)
    first = wf.KvStep(rows, rows * prompt, kv)
    step = wf.KvStep(rows, rows, kv)
    out = wf.BeamOut(groups, beams, 2 * beams)

    def write(st, tokens):
        flat[:, st.slot[:tokens.numel()]] = tokens[None, :, None].int()

    # The prompt lies in each group's first row; the first selection spreads it.
    texts = [[int(t) for t in rng.integers(0, vocab, prompt)] if r % beams == 0 else [] for r in range(rows)]
    wf.wf_kv_extend(d, kv, dev(np.array([prompt if r % beams == 0 else 0 for r in range(rows)], np.int32)), first)
    write(first, dev(np.array([t for x in texts for t in x])))
    score = dev(np.array([0.0 if r % beams == 0 else -math.inf for r in range(rows)], np.float32))
    one = torch.ones(rows, dtype=torch.int32, device="cuda")
    for s in range(steps):
        logits = dev(rng.standard_normal((rows, vocab)).astype(np.float32) * 2)
        wf.wf_beam_select(d, logits, score, out, eos=3)
        wf.wf_kv_reorder(d, kv, beams, out.next_parent.view(-1), kv, moves, cache=cache)
        wf.wf_kv_extend(d, kv, one, step)
        assert int(step.start[-1]) == rows and not host(step.status).any() and not host(moves.status).any()
        write(step, out.next_token.view(-1))
        score = out.next_score.view(-1).clone()
        parent, token = host(out.next_parent).reshape(-1), host(out.next_token).reshape(-1)
        texts = [texts[p] + [int(t)] for p, t in zip(parent, token)]
        table, length = host(kv.table), host(kv.len)
        held = {}
        for r in range(rows):
            assert length[r] == len(texts[r])
            p = np.arange(length[r])
            slots = table[r, p // bs].astype(np.int64) * bs + p % bs
            for plane in range(2):
                assert host(flat[plane, torch.from_numpy(slots).cuda(), 3]).tolist() == texts[r], (s, r)
            for b in table[r, :-(-length[r] // bs)]:
                assert held.setdefault(int(b), r // beams) == r // beams
        head, tail = host(kv.ends)
        free = host(kv.ring)[np.arange(head, tail) % n].tolist()
        assert sorted(free + list(held)) == list(range(n))
    # All searches end: every block comes back.
    wf.wf_kv_reorder(d, kv, beams, torch.full((rows,), -1, dtype=torch.int32, device="cuda"), kv, moves)
    head, tail = host(kv.ends)
    assert tail - head == n and sorted(host(kv.ring).tolist()) == list(range(n)) and not host(kv.len).any()
    wf.wf_decode_status(d)


# ---------------------------------------------------------------------------
# Refusals
# ---------------------------------------------------------------------------

def test_refusals():
    import torch
    wf = lib()
    L = wf.load_library()
    d = wf.Decode(max_rows=8, max_row_blocks=4, max_vocab=100, max_keep=8)
    kv = wf.Kv.empty(8, 4, 16, 40)
    step, moves, out = wf.KvStep(8, 16), wf.KvMoves(8), wf.BeamOut(2, 4, 8)
    add = torch.ones(8, dtype=torch.int32, device="cuda")
    by = ctypes.byref

    def einval(rc, what):
        assert rc == wf.WF_EINVAL, what
        assert wf.wf_last_error(), what

    def changed(struct, **kw):
        c = type(struct)()
        ctypes.memmove(by(c), by(struct), ctypes.sizeof(c))
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    ok = lambda k=kv.c, a=add.data_ptr(), o=step.c, h=d.ptr: L.wf_kv_extend(h, by(k), a, by(o), None)
    assert ok() == wf.WF_OK
    for kw in (dict(rows=0), dict(rows=9), dict(row_blocks=0), dict(block_tokens=0), dict(n_blocks=0), dict(table=None),
               dict(len=None), dict(ring=None), dict(ends=None), dict(table_stride=12), dict(table_stride=18),
               dict(table=kv.c.table + 2), dict(n_blocks=2 ** 31 - 1)):
        einval(ok(k=changed(kv.c, **kw)), kw)
    for kw in (dict(max_tokens=0), dict(max_tokens=2 ** 31 - 1), dict(slot=None), dict(pos=None), dict(row=None),
               dict(start=None), dict(len=None), dict(ends=None), dict(status=None), dict(slot=step.c.slot + 4),
               dict(len=kv.c.len + 4), dict(ends=kv.c.ends + 8)):
        einval(ok(o=changed(step.c, **kw)), kw)
    einval(ok(a=None), "add")
    einval(ok(h=None), "decode")

    logits = torch.zeros((8, 100), device="cuda")
    score = torch.zeros(8, device="cuda")
    b = wf.wf_beam(2, 4, 100, 8, wf._DTYPES["torch.float32"], -1, logits.data_ptr(), 400, score.data_ptr())
    sel = lambda i=b, o=out.c: L.wf_beam_select(d.ptr, by(i), by(o), None)
    assert sel() == wf.WF_OK
    for kw in (dict(groups=0), dict(groups=3), dict(beams=0), dict(beams=33), dict(vocab=0), dict(vocab=101), dict(keep=0),
               dict(keep=9), dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(score=None),
               dict(logits=logits.data_ptr() + 2), dict(logits_stride=396), dict(logits_stride=402)):
        einval(sel(i=changed(b, **kw)), kw)
    for kw in (dict(score=None), dict(parent=None), dict(token=None), dict(next_score=None), dict(next_parent=None, next_token=None),
               dict(score=out.c.score + 2)):
        einval(sel(o=changed(out.c, **kw)), kw)
    assert sel(o=changed(out.c, next_score=None, next_parent=None, next_token=None)) == wf.WF_OK

    parent = torch.full((8,), -1, dtype=torch.int32, device="cuda")
    cache = torch.zeros((2, 40, 16, 16), dtype=torch.uint8, device="cuda")
    cc = wf.wf_kv_cache(cache.data_ptr(), 2, 0, 40 * 16 * 16, 16)

    def re(k=kv.c, group=4, p=parent.data_ptr(), to=kv.c, c=cc, m=moves.copies.data_ptr(), s=moves.status.data_ptr()):
        return L.wf_kv_reorder(d.ptr, by(k), group, p, by(to), by(c) if c else None, m, s, None)
    assert re() == wf.WF_OK and re(c=None) == wf.WF_OK
    for kw in (dict(group=0), dict(group=3), dict(group=33), dict(p=None), dict(m=None), dict(s=None),
               dict(to=changed(kv.c, block_tokens=8)), dict(to=changed(kv.c, ring=kv.c.ring + 4)),
               dict(to=changed(kv.c, table=kv.c.table + 16)), dict(to=changed(kv.c, len=kv.c.len + 4)),
               dict(k=changed(kv.c, row_blocks=3)), dict(c=changed(cc, base=None)), dict(c=changed(cc, planes=0)),
               dict(c=changed(cc, token_bytes=0)), dict(c=changed(cc, plane_stride=100)),
               dict(c=changed(cc, token_bytes=2 ** 60)), dict(c=changed(cc, reserved=1))):
        einval(re(**kw), kw)
    wide = wf.Kv.empty(8, 5, 16, 40)
    einval(re(k=wide.c, to=wide.c), "wider than max_row_blocks")

    # The binding's own checks.
    for call in (lambda: wf.wf_kv_extend(d, kv, add.long(), step), lambda: wf.wf_kv_extend(d, kv, add[:4], step),
                 lambda: wf.wf_kv_extend(d, kv, add.cpu(), step), lambda: wf.wf_kv_extend(d, kv, add, wf.KvStep(4, 16)),
                 lambda: wf.wf_beam_select(d, logits.double(), score, out), lambda: wf.wf_beam_select(d, logits[:4], score, out),
                 lambda: wf.wf_beam_select(d, logits, score[:4], out), lambda: wf.wf_beam_select(d, logits.t(), score, out),
                 lambda: wf.wf_kv_reorder(d, kv, 4, parent[:4], kv, moves),
                 lambda: wf.wf_kv_reorder(d, kv, 4, parent, kv, moves, cache=cache[:, :30]),
                 lambda: wf.Kv(kv.table.t(), kv.len, kv.ring, kv.ends, 16), lambda: wf.Kv(kv.table, kv.len.long(), kv.ring, kv.ends, 16)):
        with pytest.raises(wf.WfError) as e:
            call()
        assert e.value.code == wf.WF_EINVAL
    torch.cuda.synchronize()
