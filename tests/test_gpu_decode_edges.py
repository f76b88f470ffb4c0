"""Calls on a replica's rows: what one prepared input gives in both forms of the measured calls, and the edges of sizes,
sums, devices and captures."""
import ctypes
import importlib.util
import math
import os
import random
import threading

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


def equal(a, b):
    return bool(((a == b) | ((a != a) & (b != b))).all())


# ---------------------------------------------------------------------------
# The measured calls on one input
# ---------------------------------------------------------------------------

@pytest.fixture(scope="module")
def measured():
    lib()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("measured_operators", os.path.join(root, "perf", "operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    yield m
    m.own = False


@pytest.mark.parametrize("seed", range(6))
def test_both_forms_agree_on_one_prepared_input(measured, seed):
    """Drawn cases: the library's calls, three passes that nothing waits between, and the plain form on the same
    tensors (two preparations of one seed need not be the same where likely tokens fall on one place).  Whole numbers
    and copies are equal.  A selection's are those of the 64-bit form too, and its sums near that form's: the inputs keep
    different sums at least 2^-8 / 17 apart, and 32-bit ones are off by less than 2^-16 there (values below 32:
    three roundings of up to 2^-19; log Z by up to 100 * 2^-24)."""
    import torch
    m, rng = measured, random.Random(seed)
    cases = [m.draw(rng) for _ in range(12)]
    for case in cases:
        m.own = True
        s, other = m.prepare(case, seed + 50), m.prepare(case, seed + 90)
        before = {k: v.clone() if torch.is_tensor(v) else v for k, v in s.items()}
        m.run(s)
        m.run(other)
        got = {k: v.clone() for k, v in m.run(s).items()}
        m.own = False
        want = m.run(before)
        for k, w in want.items():
            if case["kind"] != "select" or not w.is_floating_point():
                assert equal(got[k], w), (case, k, int((got[k] != w).sum()))
        if case["kind"] != "select":
            continue
        prepared, m._prepare_select = m._prepare_select, lambda c, g: before
        try:
            exact = m.exact(case, 0)
        finally:
            m._prepare_select = prepared
        for k, e in exact.items():
            g = got[k].cpu().reshape(e.shape)
            if not k.endswith("score"):
                assert equal(g, e), (case, k)
                continue
            there = torch.isfinite(e)
            assert equal(g.double()[~there], e[~there]), (case, k)
            assert not there.any() or float((g.double() - e)[there].abs().max()) < 2.0 ** -16, (case, k)


# ---------------------------------------------------------------------------
# Reorder: sizes of blocks, places of the cache
# ---------------------------------------------------------------------------

def test_reorder_copies_a_few_tokens_of_blocks_beyond_2_gib():
    """What lies past a copy's last byte is further than 31 bits from it, at one byte an access."""
    import torch
    wf = lib()
    bs, token, n = 70_001, 32_769, 3  # 2.29e9 bytes a block, on no 4-byte boundary
    assert bs * token > 2 ** 31 + 5 * token
    cache = torch.zeros((1, n, bs, token), dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache[0, 2, :7] = torch.randint(1, 256, (7, token), generator=gen, device="cuda", dtype=torch.uint8)
    d = wf.Decode(max_rows=2, max_row_blocks=1)
    kv = wf.Kv(dev(np.array([[2], [-1]], np.int32)), dev(np.array([5, 0], np.int32)), dev(np.array([1, 0, -1], np.int32)),
               dev(np.array([0, 2])), bs)
    out = wf.KvMoves(2)
    wf.wf_kv_reorder(d, kv, 2, dev(np.array([0, 0], np.int32)), kv, out, cache=cache)
    wf.wf_decode_status(d)
    assert host(out.copies).tolist() == [[-1, -1], [2, 1]] and host(kv.len).tolist() == [5, 5]
    assert torch.equal(cache[0, 1, :5], cache[0, 2, :5])
    assert not cache[0, 1, 5:].any() and not cache[0, 0].any() and not cache[0, 2, 7:].any()


# ---------------------------------------------------------------------------
# Refusals of the binding
# ---------------------------------------------------------------------------

def test_binding_refuses_outputs_and_scratch_of_another_device_or_size():
    """Nothing is launched for any of these: what the library would get are pointers of other memory."""
    import torch
    wf = lib()
    d = wf.Decode(max_rows=8, max_row_blocks=4, max_vocab=100, max_keep=8)
    kv, small = wf.Kv.empty(8, 4, 16, 40), wf.Kv.empty(4, 4, 16, 40)
    step, moves, out = wf.KvStep(8, 16), wf.KvMoves(8), wf.BeamOut(2, 4, 8)
    add = torch.ones(8, dtype=torch.int32, device="cuda")
    parent = torch.full((8,), -1, dtype=torch.int32, device="cuda")
    logits, score = torch.zeros((8, 100), device="cuda"), torch.zeros(8, device="cuda")
    elsewhere = wf.Decode(max_rows=8, max_row_blocks=4, max_vocab=100, max_keep=8)
    elsewhere.device = 1  # as if made there
    far = wf.Kv.empty(8, 4, 16, 40)
    far.device = 1
    for call in (lambda: wf.KvStep(8, 16, small),
                 lambda: wf.KvStep(8, 16, kv, device="cpu"),
                 lambda: wf.wf_kv_extend(d, kv, add, wf.KvStep(8, 16, device="cpu")),
                 lambda: wf.wf_kv_extend(elsewhere, kv, add, step),
                 lambda: wf.wf_beam_select(elsewhere, logits, score, out),
                 lambda: wf.wf_beam_select(d, logits, score, wf.BeamOut(2, 4, 8, device="cpu")),
                 lambda: wf.wf_beam_select(d, logits.cpu().numpy(), score, out),
                 lambda: wf.wf_kv_reorder(elsewhere, kv, 4, parent, kv, moves),
                 lambda: wf.wf_kv_reorder(d, kv, 4, parent, far, moves),
                 lambda: wf.wf_kv_reorder(d, kv, 4, parent, kv, wf.KvMoves(8, device="cpu")),
                 lambda: wf.wf_kv_reorder(d, kv, 4, parent, kv, moves, cache=np.zeros((1, 40, 16, 4), np.uint8)),
                 lambda: wf.wf_kv_reorder(d, kv, 4, parent, kv, moves, cache=torch.zeros((1, 40, 16, 4))),
                 lambda: wf.Kv(kv.table, kv.len, host(kv.ring), kv.ends, 16)):
        with pytest.raises(wf.WfError) as e:
            call()
        assert e.value.code == wf.WF_EINVAL
    # What fits goes through as before.
    wf.wf_kv_extend(d, kv, add, wf.KvStep(8, 16, kv))
    wf.wf_beam_select(d, logits, score, out)
    wf.wf_kv_reorder(d, kv, 4, parent, kv, moves)
    wf.wf_decode_status(d)
    assert int(kv.ends[1] - kv.ends[0]) == 40


# ---------------------------------------------------------------------------
# Extend: lengths, launches
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [5, 17_000])
def test_extend_passes_over_lengths_beyond_31_bits(rows):
    """A table row may hold more tokens than a 32-bit length counts: a row that would pass 2^31 - 1 is WF_KV_LONG, the
    others go on."""
    import torch
    wf = lib()
    most, bs = 2 ** 31 - 1, 1 << 30  # a table row of 4 blocks holds 2^32 tokens
    length, add = np.zeros(rows, np.int32), np.zeros(rows, np.int32)
    length[:5], add[:5] = [most - 5, most - 5, 0, most, most], [5, 6, 3, 0, most]
    table = np.full((rows, 4), -1, np.int32)
    table[[0, 1, 3, 4], :2] = np.arange(8).reshape(4, 2)
    ring, ends = np.arange(12, dtype=np.int32)[::-1].copy(), np.array([0, 4], np.int64)
    left_out = add.copy()
    left_out[[1, 4]] = -1  # the plain form passes these over for another reason, with the same outcome
    want = ref.extend(table, length, left_out, ring, ends, bs, 64)
    assert want["status"][:5].tolist() == [0, wf.KV_LONG, 0, 0, wf.KV_LONG] and want["len"][0] == most
    d = wf.Decode(max_rows=rows)
    kv, step = wf.Kv(dev(table), dev(length), dev(ring), dev(ends), bs), wf.KvStep(rows, 64)
    wf.wf_kv_extend(d, kv, dev(add), step)
    torch.cuda.synchronize()
    got = dict(table=kv.table, slot=step.slot, pos=step.pos, row=step.row, start=step.start, len=step.len, ends=step.ends,
               status=step.status)
    for k, w in want.items():
        assert np.array_equal(host(got[k]), w), k


def test_extend_of_different_sizes_from_two_threads():
    """Two handles on two host threads and streams: the rows' sums of one take four times the shared memory of the
    other's, and neither's call changes what the other may launch."""
    import torch
    wf = lib()
    failed, threads = [], []
    rng = np.random.default_rng(4)

    def work(rows, stream, d, kv, add, step, want):
        try:
            for _ in range(1500):
                wf.wf_kv_extend(d, kv, add, step, stream=stream)
            stream.synchronize()
            for k in ("slot", "start", "len", "ends", "status"):
                assert np.array_equal(host(getattr(step, k)), want[k]), (rows, k)
        except Exception as e:  # (an assertion of a thread is no failure of the test)
            failed.append(f"{rows} rows: {e!r}")

    for rows in (16_384, 4_000):
        add = rng.integers(0, 3, rows).astype(np.int32)
        kv = wf.Kv.empty(rows, 2, 16, rows)
        want = ref.extend(host(kv.table), host(kv.len), add, host(kv.ring), host(kv.ends), 16, 2 * rows)
        args = (rows, torch.cuda.Stream(), wf.Decode(max_rows=rows), kv, dev(add), wf.KvStep(rows, 2 * rows), want)
        threads.append(threading.Thread(target=work, args=args))
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed


# ---------------------------------------------------------------------------
# Select: equal beams, sums
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("low,level,spread", [(-1000.0, 85.0, 7.0), (-1000.0, -62.0, 2.0), (-200.0, 95.0, 4.0)])
@pytest.mark.parametrize("groups,beams,vocab", [(64, 2, 30_001), (40, 3, 50_257), (1, 5, 32_003)])
def test_select_equal_rows_have_equal_sums_where_one_leaves_a_floats_range(groups, beams, vocab, low, level, spread):
    """Equal rows that lie differently in their 16 bytes.  The first 1,023 tokens have a finite mask, so the four
    lines that give a part its reference hold the first token that says something in some rows and not in others:
    relative to that the sum fits a float, relative to 0 it passes its range (or nearly vanishes)."""
    import torch
    wf = lib()
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = (level + spread * (torch.rand((groups, vocab), generator=gen, device="cuda") - 0.5)).half()
    x[:, :1023] = low
    x[:, 1023] = level + 8  # so far above the others that log Z is small: a sum shows its last bits
    x = x.repeat_interleave(beams, 0).contiguous()
    assert vocab % 8 and x.stride(0) == vocab
    score = torch.zeros(groups * beams, device="cuda")
    keep = 2 * beams
    d = wf.Decode(max_rows=groups * beams, max_vocab=vocab, max_keep=keep)
    out = wf.BeamOut(groups, beams, keep)
    wf.wf_beam_select(d, x, score, out)
    parent, token, got = host(out.parent) % beams, host(out.token), host(out.score)
    for g in range(groups):
        row = host(x[g * beams].float())
        want = []
        for value in np.unique(row)[::-1]:
            want += [(k, int(t)) for k in range(beams) for t in np.flatnonzero(row == value)]
            if len(want) >= keep:
                break
        assert list(zip(parent[g].tolist(), token[g].tolist())) == want[:keep], g
        at = row[token[g]]
        assert all(len(set(got[g][at == v].tolist())) == 1 for v in np.unique(at)), g


def test_select_equal_rows_with_zeros_of_both_signs():
    """Scores and maxima of -0 and 0 are equal."""
    import torch
    wf = lib()
    vocab, beams, groups = 9001, 4, 30
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = (-20 * torch.rand((groups, vocab), generator=gen, device="cuda")).half()
    x[:, 77] = 0.0
    x = x.repeat_interleave(beams, 0).contiguous()
    x[1::2, 77] = -0.0
    score = torch.zeros(groups * beams, device="cuda")
    score[::3] = -0.0
    d = wf.Decode(max_rows=groups * beams, max_vocab=vocab, max_keep=beams)
    out = wf.BeamOut(groups, beams, beams)
    wf.wf_beam_select(d, x, score, out)
    assert (host(out.token) == 77).all() and (host(out.parent) % beams == np.arange(beams)).all()
    got = host(out.score)
    assert (got == got[:, :1]).all()


def z_bound(chain, levels, sizes):
    """How far a selection's sums may be from the 64-bit form's, by what is done in 32 bits (u = 2^-24):
      chain       additions that a term passes through on its way to Z, u each
      levels      distance of the terms that count from the maximum: the argument log2(e) x of 2^x is rounded
                  (u of it) and so is its factor log2(e) (2^-26 of it), twice, for a part's reference and the maximum's
      2^x         2^-22 for each of the two
      log, sum    an ulp of log Z, and half of one for each of two additions."""
    u = 2.0 ** -24
    log_z = math.log(sizes)
    ulp = 2.0 ** (math.floor(math.log2(max(log_z + levels, 1.0))) - 23)
    return chain * u + 2 * levels * (u + 2.0 ** -26) + 2 * 2.0 ** -22 + 2 * ulp


def check_two_levels(wf, x, score, keep, chain):
    """Rows of 5s and 0s (NaN masked): the best are the 5s, then the 0s."""
    import torch
    rows, vocab = x.shape
    d = wf.Decode(max_rows=rows, max_vocab=vocab, max_keep=keep)
    out = wf.BeamOut(rows, 1, keep)
    wf.wf_beam_select(d, x, score, out)
    got, token = host(out.score).astype(np.float64), host(out.token)
    high, none = host((x == 5).sum(1)), host(torch.isnan(x).sum(1))
    log_z = np.log(high + (vocab - high - none) * math.exp(-5.0))
    first = host(torch.where(torch.isnan(x), -1.0, x.float()).sort(dim=1, descending=True, stable=True).indices[:, :keep]) if vocab < 1 << 20 else None
    for r in range(rows):
        want = np.where(np.arange(keep) < high[r], 0.0, -5.0) - log_z[r]
        assert np.abs(got[r] - want).max() <= z_bound(chain, 5, vocab), (r, got[r] - want)
        if first is not None:
            assert token[r].tolist() == first[r].tolist()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_select_sums_of_long_parts(dtype):
    """More searches than are resident at once: a warp sums an eighth of a row.  Each step of a part holds one 5, so that is
    the part's reference; the others are 0, each term e^-5, and the roundings of its additions go one way.
    Chain: 5 additions to a step's sum, 64 steps, 2 for the compensated sum over those, 5 over the lanes, 1 part a lane,
    5 over the lanes of the join."""
    import torch
    wf = lib()
    vocab = 1 << (18 if dtype == "float32" else 19)
    x = torch.zeros((500, vocab), dtype=getattr(torch, dtype), device="cuda")
    x[:, ::512 if dtype == "float32" else 1024] = 5  # a step's tokens
    check_two_levels(wf, x, torch.zeros(500, device="cuda"), 12, 5 + 64 + 2 + 5 + 1 + 5)


@pytest.mark.parametrize("vocab", [600_001, 1 << 24])
@pytest.mark.parametrize("beams", [2])
def test_select_sums_of_rows_with_a_nan(vocab, beams):
    """A row with a NaN is summed again by the join, up to 65,536 logits a thread.  Chain: 3 additions to eight
    logits' sum, 2 for the compensated sum over those, 5 over the lanes, 16 over the warps; and for the row without, one
    step a part, 76 parts a lane at most."""
    import torch
    wf = lib()
    x = torch.zeros((beams, vocab), dtype=torch.float16, device="cuda")
    x[:, 1234] = 5
    x[0, vocab // 2 + 3] = math.nan
    for row, chain in ((0, 3 + 2 + 5 + 16), (1, 5 + 64 + 2 + 5 + 76 + 5)):
        check_two_levels(wf, x[row:row + 1], torch.zeros(1, device="cuda"), 4, chain)


# ---------------------------------------------------------------------------
# The example
# ---------------------------------------------------------------------------

@pytest.fixture(scope="module")
def example():
    import sys
    lib()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    import decode_window
    import wfgen
    prob = wfgen.config("tiny").problem
    return decode_window, prob, *decode_window.first_batch(prob, n_plans=64)


def test_example_decodes_what_lies_in_the_cache(example, monkeypatch):
    """With every cached vector's sign changed once, after the first step, other tokens follow."""
    ex, prob, device, batch = example
    plain = ex.decode(prob, device, batch, beams=3, steps=6)
    reorder, calls = ex.wf.wf_kv_reorder, []

    def and_change_signs(scratch, kv, group, parent, to, moves, cache=None, **kw):
        reorder(scratch, kv, group, parent, to, moves, cache=cache, **kw)
        calls.append(cache)
        if len(calls) == 1:
            cache.neg_()
    monkeypatch.setattr(ex.wf, "wf_kv_reorder", and_change_signs)
    other = ex.decode(prob, device, batch, beams=3, steps=6)
    assert plain["error"] < 1e-4 < other["error"]
    assert any(a[1:] != b[1:] for a, b in zip(plain["texts"], other["texts"]))


def test_example_ends_searches_that_find_no_block(example):
    """Blocks for the prompts and a few steps: searches end where a row finds none or waits, and all blocks come back."""
    ex, prob, device, batch = example
    all_of_it = ex.decode(prob, device, batch, beams=3, steps=40)
    assert all_of_it["steps"] == [40 if ok else 0 for ok in all_of_it["admitted"]]
    few = ex.decode(prob, device, batch, beams=3, steps=40, n_blocks=all_of_it["prompt_blocks"] + 2)
    assert few["admitted"].any() and few["left"] == few["n_blocks"] and few["error"] < 1e-4
    assert min(n for n, ok in zip(few["steps"], few["admitted"]) if ok) < 40
    assert [len(t) for t in few["texts"]] == [n if ok else 0 for n, ok in zip(few["steps"], few["admitted"])]
    assert all(0 < t < ex.VOCAB for text in few["texts"] for t in text)


# ---------------------------------------------------------------------------
# Captures, streams
# ---------------------------------------------------------------------------

def test_a_decoding_step_captured_and_on_a_stream_of_its_own():
    """Selection, reordering with copies and extension in place, as one step: eagerly on a side stream, then replayed
    from a graph; each step against the plain forms from the step's own state."""
    import torch
    wf = lib()
    rng = np.random.default_rng(12)
    groups, beams, vocab, bs, width = 6, 4, 3001, 4, 12
    rows, n = groups * beams, groups * beams * width + 4
    d = wf.Decode(max_rows=rows, max_row_blocks=width, max_vocab=vocab, max_keep=2 * beams)
    kv, moves, step = wf.Kv.empty(rows, width, bs, n), wf.KvMoves(rows), None
    step, first = wf.KvStep(rows, rows, kv), wf.KvStep(rows, rows * 10, kv)
    score = torch.full((rows,), -math.inf, device="cuda")
    score[::beams] = 0
    out = wf.BeamOut(groups, beams, 2 * beams, score)
    logits = torch.zeros((rows, vocab), device="cuda")
    one = torch.ones(rows, dtype=torch.int32, device="cuda")
    cache = dev(rng.integers(0, 256, (3, n, bs, 24)).astype(np.uint8))
    prompt = np.zeros(rows, np.int32)
    prompt[::beams] = rng.integers(1, 10, groups)
    wf.wf_kv_extend(d, kv, dev(prompt), first)

    def one_step():
        wf.wf_beam_select(d, logits, score, out, eos=2)
        wf.wf_kv_reorder(d, kv, beams, out.next_parent.view(-1), kv, moves, cache=cache)
        wf.wf_kv_extend(d, kv, one, step)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for i in range(12):
        x = rng.standard_normal((rows, vocab)).astype(np.float32) * 2
        logits.copy_(dev(x))
        torch.cuda.synchronize()
        if i == 6:
            with torch.cuda.graph(graph):  # (captured, not run)
                one_step()
        before = {k: host(v) for k, v in dict(table=kv.table, len=kv.len, ring=kv.ring, ends=kv.ends, cache=cache, score=score).items()}
        if i < 6:
            with torch.cuda.stream(side):
                one_step()
            side.synchronize()
        else:
            graph.replay()
            torch.cuda.synchronize()
        best = ref.select(x, before["score"], beams, 2 * beams)
        parent = host(out.next_parent).reshape(-1)
        for g, want in enumerate(best):  # (normal values: no two sums within their rounding)
            onward = [(p, t) for _, p, t in want if t != 2][:beams]
            assert list(zip(host(out.next_parent)[g].tolist(), host(out.next_token)[g].tolist())) == onward, (i, g)
        mid = ref.reorder(before["table"], before["len"], before["ring"], before["ends"], bs, beams, parent, before["table"], before["cache"])
        end = ref.extend(mid["table"], mid["len"], np.ones(rows, np.int32), mid["ring"], mid["ends"], bs, rows)
        got = dict(table=kv.table, len=kv.len, ends=kv.ends, slot=step.slot, pos=step.pos, row=step.row, start=step.start, status=step.status)
        for k, v in got.items():
            assert np.array_equal(host(v), end[k]), (i, k)
        assert np.array_equal(host(moves.copies), mid["copies"]) and np.array_equal(host(cache), mid["cache"]), i
        assert np.array_equal(host(kv.ring), mid["ring"]) and not host(moves.status).any()
    wf.wf_decode_status(d)


@pytest.mark.parametrize("offset,token_bytes,gap", [(0, 48, 0), (0, 48, 80), (4, 48, 4), (1, 48, 0), (8, 20, 16), (3, 7, 5)])
def test_reorder_of_a_cache_whose_planes_lie_apart_or_anywhere(offset, token_bytes, gap):
    """Planes further apart than their blocks, bases on no boundary: nothing between the planes changes."""
    import torch
    wf = lib()
    L, rng = wf.load_library(), np.random.default_rng(offset + gap)
    planes, n, bs, rows = 3, 9, 5, 4
    plane = n * bs * token_bytes
    raw = rng.integers(0, 256, offset + planes * (plane + gap) + 64).astype(np.uint8)
    buf = dev(raw)
    table = np.array([[0, 1, -1], [0, 2, -1], [0, 1, 3], [4, -1, -1]], np.int32)
    length, parent = np.array([8, 9, 11, 3], np.int32), np.array([1, 1, 3, 3], np.int32)
    ring, ends = np.array([5, 6, 7, 8, -1, -1, -1, -1, -1], np.int32), np.array([0, 4], np.int64)
    view = lambda a: np.stack([a[offset + p * (plane + gap):][:plane] for p in range(planes)]).reshape(planes, n, bs, token_bytes)
    want = ref.reorder(table, length, ring, ends, bs, rows, parent, table, view(raw))
    kv, out = wf.Kv(dev(table), dev(length), dev(ring), dev(ends), bs), wf.KvMoves(rows)
    d = wf.Decode(max_rows=rows, max_row_blocks=3)
    cc = wf.wf_kv_cache(buf.data_ptr() + offset, planes, 0, plane + gap, token_bytes)
    p = dev(parent)
    assert L.wf_kv_reorder(d.ptr, ctypes.byref(kv.c), rows, p.data_ptr(), ctypes.byref(kv.c), ctypes.byref(cc),
                           out.copies.data_ptr(), out.status.data_ptr(), torch.cuda.current_stream().cuda_stream or None) == wf.WF_OK
    wf.wf_decode_status(d)
    got = host(buf)
    assert np.array_equal(view(got), want["cache"]) and np.array_equal(host(out.copies), want["copies"])
    between = np.ones(raw.size, bool)
    for q in range(planes):
        between[offset + q * (plane + gap):][:plane] = False
    assert np.array_equal(got[between], raw[between])
