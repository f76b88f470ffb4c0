"""wf_attend against a plain implementation in 64 bits."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import lib
from test_gpu_write import HALF_STEP, LEAST, TYPES, Step, cache_of, f64, tensor

pytestmark = pytest.mark.gpu


def values(cache, scale):
    x = f64(cache)
    return x if scale is None else x * f64(scale)[:, :, None, :, None]


def attend(wf, st, cache, scale, q, scaling=None, new=0, out=None, attn=None):
    import torch
    out = torch.full_like(q, 7.0) if out is None else out
    layer = wf.KvLayer(cache[0], cache[1], *(() if scale is None else (scale[0], scale[1])))
    attn = attn or wf.Attn(max_rows=st.rows, heads=q.shape[1], dim=q.shape[2])
    wf.wf_attend(attn, st.kv, st.step, layer, q, out, scale=scaling, new=new)
    wf.wf_attn_status(attn)
    return out


def bound(size, small, want, q, dtype, eight, scaling, keys, k_most):
    """What an output may be off by.  Half a step for its rounding.  Of the sum of |weight * value| (size): half a step of the weights' type
    (half floats over 8 bits); a score is a sum of dim products in 32 bits, off by at most dim 2^-24 sum |q k|
    (the order of a matrix instruction's additions is not said) and 2^-23 relative by the scale in base 2, which is a
    weight's relative error, and the largest score's too; 2^-21 for powers and sums of weights per join, and n 2^-24 of a long sum.
    Weights in half floats are 2^-24 apart below 2^-14, where the largest (times its value's scale) is 1: each may be off by 2^-25 of that, times its
    value without the scale (small)."""
    dim = q.shape[-1]
    score = np.abs(scaling) * np.abs(q).sum(-1, keepdims=True) * k_most
    weight = HALF_STEP["float16" if eight else dtype] + 2 * score * (dim * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -19 + keys * 2.0 ** -24
    least = 0.0 if dtype == "bfloat16" and not eight else 2.0 ** -25
    return HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -8) + LEAST[dtype] + 2 * size * weight + small * least * (1 + 2.0 ** -8)


def check(st, cache, scale, q, got, scaling=None):
    scaling = q.shape[2] ** -0.5 if scaling is None else scaling
    x, dtype = values(cache, scale), str(q.dtype).split(".")[1]
    want, size, small = ref.attend(f64(q), x[0], x[1], st.table, st.start, st.len, st.bs, scaling, np.full(q.shape, 7.0),
                                   None if scale is None else f64(scale[1]))
    off, most = np.abs(f64(got) - want), bound(size, small, want, f64(q), dtype, scale is not None, scaling, int(st.len.max()), np.abs(x[0]).max())
    n = st.tokens
    assert (off[:n] <= most[:n]).all(), f"off by {np.max(off[:n] - most[:n])} more than allowed at {np.argwhere(off[:n] > most[:n])[0]} of {want.shape}"
    assert (got[n:] == 7).all()  # behind the last token


SHAPES = [  # have, add, block size, heads, key heads, dim
    ([0], [1], 16, 1, 1, 64), ([0], [1], 16, 4, 4, 128), ([63], [1], 16, 8, 2, 128), ([64], [1], 16, 8, 2, 64),
    ([0, 15, 16, 17, 300, 1], [1, 1, 1, 1, 1, 1], 16, 8, 2, 128), ([5, 0, 70, 129], [1, 0, 1, 0], 7, 6, 2, 64),
    ([0, 0, 3], [5, 16, 1], 16, 3, 1, 128), ([0], [130], 16, 4, 2, 64), ([100, 0, 17], [33, 64, 1], 24, 7, 1, 128),
    ([1000], [1], 1, 5, 5, 64), ([3000, 10], [1, 1], 128, 16, 1, 128), ([5000], [1], 100, 40, 2, 64),
    ([40] * 130, [1] * 130, 16, 4, 2, 64), ([0] * 5, [1, 2, 3, 4, 5], 3, 24, 8, 128), ([200, 90], [70, 300], 64, 8, 2, 128),
    ([700], [257], 16, 2, 2, 128)]


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("have,add,bs,heads,kv,dim", SHAPES, ids=range(len(SHAPES)))
def test_attend(have, add, bs, heads, kv, dim, dtype, eight):
    import torch
    wf = lib()
    rng = np.random.default_rng(len(have) * 100 + bs)
    st = Step(wf, rng, have, add, bs, spare=5)
    cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn" if eight else dtype)
    q = tensor(rng, (st.room, heads, dim), dtype, 1.5)
    got = attend(wf, st, cache, scale, q)
    check(st, cache, scale, q, got)
    # The hint changes nothing that is computed beyond rounding; the same call twice is the same.
    check(st, cache, scale, q, attend(wf, st, cache, scale, q, new=1))
    assert torch.equal(got, attend(wf, st, cache, scale, q))


LONG = [  # have, add, block size, heads, key heads, dim
    ([0], [700], 16, 1, 1, 128), ([0, 40], [300, 129], 7, 4, 2, 64), ([1000, 3], [64, 400], 100, 5, 1, 128), ([10] * 9, [33, 1, 40, 2, 90, 0, 127, 128, 129], 8, 6, 2, 64),
    ([0, 300], [40, 3], 64, 130, 1, 64), ([5], [260], 128, 7, 1, 128), ([2000], [64], 32, 64, 1, 128), ([130], [513], 1, 2, 1, 64), ([900], [37], 24, 24, 8, 128),
    ([0, 0, 0], [256, 255, 257], 48, 2, 2, 128)]


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("have,add,bs,heads,kv,dim", LONG, ids=range(len(LONG)))
def test_attend_prompts(have, add, bs, heads, kv, dim, dtype, eight):
    """Groups that fill a tile or do not, blocks of any size, chunks that end anywhere, NaN behind every row."""
    import torch
    wf = lib()
    rng = np.random.default_rng(len(have) * 1000 + bs)
    st = Step(wf, rng, have, add, bs, spare=5)
    cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn" if eight else dtype)
    used = np.concatenate([st.table[r, np.arange(n) // bs].astype(np.int64) * bs + np.arange(n) % bs for r, n in enumerate(st.len)])
    rest = torch.from_numpy(np.setdiff1d(np.arange(st.n_blocks * bs), used)).cuda()
    raw = cache.view(torch.uint8 if eight else torch.int16)
    raw.flatten(1, 2)[:, rest] = 0x7F if eight else (0x7E00 if dtype == "float16" else 0x7FC0)
    q = tensor(rng, (st.room, heads, dim), dtype, 1.5)
    got = attend(wf, st, cache, scale, q)
    clean = cache.clone()
    clean.view(torch.uint8).flatten(1, 2)[:, rest] = 0
    check(st, clean, scale, q, got)
    assert torch.equal(got, attend(wf, st, cache, scale, q))


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
def test_long_prompts_in_torch(eight):
    """Longer prompts, whose positions several blocks of the GPU share, against products in 64 bits on the GPU."""
    import torch
    wf = lib()
    rng = np.random.default_rng(31)
    for have, add, heads, kv, dim, bs in (([0, 3000], [3000, 700], 8, 2, 128, 16), ([20000], [130], 4, 1, 64, 32), ([11, 0, 5000], [1500, 2100, 1], 6, 2, 128, 24)):
        st = Step(wf, rng, have, add, bs)
        dtype = "bfloat16"
        cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn" if eight else dtype)
        q = tensor(rng, (st.room, heads, dim), dtype, 1.5)
        got = attend(wf, st, cache, scale, q).double()
        x = cache.double() if scale is None else cache.double() * scale.double()[:, :, None, :, None]
        for r, n in enumerate(st.len):
            blocks = torch.from_numpy(st.table[r, :-(-int(n) // bs)].astype(np.int64)).cuda()
            k, v = (x[i][blocks].flatten(0, 1)[:int(n)] for i in (0, 1))
            a, b = int(st.start[r]), int(st.start[r + 1])
            later = torch.arange(int(n), device="cuda") > torch.arange(int(have[r]), int(n), device="cuda")[:, None]
            for h in range(heads):
                w = torch.softmax((q[a:b, h].double() @ k[:, h * kv // heads].T * dim ** -0.5).masked_fill(later, -torch.inf), 1)
                want, size = w @ v[:, h * kv // heads], w @ v[:, h * kv // heads].abs()
                # As in bound(), with 2^-9 more for scores (dim 2^-24 times products up to 2^9 here) and for the subnormal weights over 8 bits.
                assert ((got[a:b, h] - want).abs() <= 2.0 ** -8 * want.abs() + size * (2 * 2.0 ** -8 + 2.0 ** -9)).all(), (r, h)


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
@pytest.mark.parametrize("have,heads,kv,dim", [([40000], 8, 1, 128), ([20000, 3, 9000, 1], 4, 2, 64), ([30000, 30000], 12, 4, 128)])
def test_long_rows_are_split(have, heads, kv, dim, eight):
    wf = lib()
    rng = np.random.default_rng(sum(have))
    st = Step(wf, rng, have, [1] * len(have), 16)
    cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn" if eight else "bfloat16")
    q = tensor(rng, (st.room, heads, dim), "bfloat16", 1.5)
    check(st, cache, scale, q, attend(wf, st, cache, scale, q, new=1))


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
@pytest.mark.parametrize("add", ([1, 1], [40, 300]), ids=("short", "long"))
@pytest.mark.parametrize("dtype", TYPES)
def test_attend_strides(dtype, add, eight):
    """Queries that are columns of one product, heads outermost, keys beside values, heads before places: the same outputs."""
    import torch
    wf = lib()
    rng = np.random.default_rng(21)
    st = Step(wf, rng, [300, 17], add, 16, spare=3)
    heads, kv, dim = 6, 2, 64
    cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn" if eight else dtype)
    q = tensor(rng, (st.room, heads, dim), dtype)
    want = attend(wf, st, cache, scale, q)
    whole = torch.cat([tensor(rng, (st.room, 2, dim), dtype), q, q], 1)
    assert torch.equal(attend(wf, st, cache, scale, whole[:, 2:2 + heads]), want)
    turn = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(attend(wf, st, cache, scale, turn(q), out=turn(torch.full_like(q, 7.0))), want)
    beside = cache.view(torch.uint8).view(2, st.n_blocks, st.bs, kv, -1).permute(1, 2, 3, 0, 4).contiguous().permute(3, 0, 1, 2, 4).view(cache.dtype)
    assert torch.equal(attend(wf, st, beside, scale, q), want)
    by_head = cache.transpose(2, 3).contiguous().transpose(2, 3)
    assert torch.equal(attend(wf, st, by_head, scale, q), want)


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
@pytest.mark.parametrize("have,add", [([37, 0, 5], [1, 1, 1]), ([37, 0, 5], [50, 130, 300])], ids=("short", "long"))
def test_what_lies_behind_a_row_does_not_count(have, add, eight):
    """NaN and infinities in places behind a row's tokens, in unused blocks, and blocks named there by no one."""
    import torch
    wf = lib()
    rng = np.random.default_rng(22)
    st = Step(wf, rng, have, add, 16)
    cache, scale = cache_of(rng, st, 2, 64, "float8_e4m3fn" if eight else "bfloat16")
    q = tensor(rng, (st.room, 4, 64), "bfloat16")
    want = attend(wf, st, cache, scale, q)
    used = np.concatenate([st.table[r, np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16 for r, n in enumerate(st.len)])
    rest = torch.from_numpy(np.setdiff1d(np.arange(st.n_blocks * 16), used)).cuda()
    raw = cache.view(torch.uint8 if eight else torch.int16)
    raw.flatten(1, 2)[:, rest] = 0x7F if eight else 0x7FC0
    if eight:
        free = np.setdiff1d(np.arange(st.n_blocks), st.table[st.table >= 0])
        scale[:, torch.from_numpy(free).cuda()] = float("nan")
    st.kv.table[st.kv.table < 0] = 1 << 30
    assert torch.equal(attend(wf, st, cache, scale, q), want)


@pytest.mark.parametrize("add", ([1, 1, 1], [200, 3, 140]), ids=("short", "long"))
@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
def test_large_and_equal_scores(add, eight):
    """Scores far apart (one key has all the weight), all equal (the mean), growing along the row; large and small scales of blocks."""
    import torch
    wf = lib()
    rng = np.random.default_rng(23)
    st = Step(wf, rng, [300, 150, 0], add, 16)
    dtype = "bfloat16"
    for spread, grow in ((40.0, False), (0.0, False), (3.0, True)):
        cache, scale = cache_of(rng, st, 2, 128, "float8_e4m3fn" if eight else dtype)
        if eight and not grow:
            scale.copy_(torch.from_numpy(2.0 ** rng.integers(-40, -5, scale.shape)).float())
        if grow:
            for r, n in enumerate(st.len):
                blocks = torch.from_numpy(st.table[r, :-(-int(n) // 16)]).cuda().long()
                if eight:
                    scale[:, blocks] = (2.0 ** (torch.arange(len(blocks), device="cuda") % 20 - 12.0))[None, :, None]
                else:
                    cache[0, blocks] = cache[0, blocks] * torch.linspace(0, 2, len(blocks), device="cuda", dtype=cache.dtype)[:, None, None, None]
        q = tensor(rng, (st.room, 8, 128), dtype, spread)
        check(st, cache, scale, q, attend(wf, st, cache, scale, q))


def test_scores_that_are_no_numbers():
    """An infinite or NaN key of a row makes its later outputs NaN and leaves other rows alone; a query of infinities its own."""
    import torch
    wf = lib()
    rng = np.random.default_rng(24)
    st = Step(wf, rng, [40, 40, 40], [1, 1, 1], 16)
    cache, _ = cache_of(rng, st, 1, 64, "float16")
    q = tensor(rng, (3, 2, 64), "float16")
    want = attend(wf, st, cache, None, q)
    cache[0, int(st.table[1, 1]), 3, 0, 5] = float("nan")
    q[2, 1, 7] = float("inf")
    got = attend(wf, st, cache, None, q)
    assert got[1].isnan().all() and got[2, 1].isnan().all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[2, 0], want[2, 0])


def test_bad_rows_are_reported_and_passed_over():
    import torch
    wf = lib()
    rng = np.random.default_rng(25)
    st = Step(wf, rng, [40, 40, 40, 40], [1, 1, 1, 1], 16)
    cache, _ = cache_of(rng, st, 1, 64, "float16")
    q = tensor(rng, (4, 2, 64), "float16")
    want = attend(wf, st, cache, None, q)
    attn = wf.Attn(max_rows=4, heads=2, dim=64)
    layer, out = wf.KvLayer(cache[0], cache[1]), torch.full_like(q, 7.0)
    length = st.kv.len.clone()
    st.kv.len[1], st.kv.len[2] = 0, 16 * st.table.shape[1] + 1
    wf.wf_attend(attn, st.kv, st.step, layer, q, out)
    with pytest.raises(wf.WfError, match="contradict"):
        wf.wf_attn_status(attn)
    wf.wf_attn_status(attn)
    assert torch.equal(out[[0, 3]], want[[0, 3]]) and (out[1:3] == 7).all()
    st.kv.len.copy_(length)
    st.kv.table[3, 1] = st.n_blocks
    wf.wf_attend(attn, st.kv, st.step, layer, q, out)
    with pytest.raises(wf.WfError, match="outside the cache"):
        wf.wf_attn_status(attn)
    assert torch.equal(out[:3], want[:3])
    st.step.start[4] = 5  # more tokens than the step has
    wf.wf_attend(attn, st.kv, st.step, layer, q, out)
    with pytest.raises(wf.WfError):
        wf.wf_attn_status(attn)


def test_attend_refuses():
    import torch
    wf = lib()
    rng = np.random.default_rng(26)
    st = Step(wf, rng, [40], [1], 16)
    cache, _ = cache_of(rng, st, 2, 64, "float16")
    layer, attn = wf.KvLayer(cache[0], cache[1]), wf.Attn(max_rows=1, heads=4, dim=64)
    q = tensor(rng, (1, 4, 64), "float16")
    ok = lambda **kw: wf.wf_attend(**{**dict(attn=attn, kv=st.kv, step=st.step, layer=layer, q=q, out=torch.empty_like(q)), **kw})
    ok()
    odd = torch.empty(257, dtype=torch.float16, device="cuda")[1:].view(1, 4, 64)
    for kw in (dict(q=q.float()), dict(q=q.bfloat16()), dict(q=q[:, :3]), dict(q=odd), dict(out=odd), dict(q=q.cpu()), dict(out=q[:, :2]),
               dict(q=q[0]), dict(scale=float("nan")), dict(new=-1), dict(attn=wf.Attn(max_rows=1, heads=4, dim=128)),
               dict(attn=wf.Attn(max_rows=1, heads=2, dim=64)), dict(layer=wf.KvLayer(cache[0, :-1], cache[1, :-1])),
               dict(layer=wf.KvLayer(cache[0].bfloat16(), cache[1].bfloat16())), dict(q=torch.cat([q, q])),
               dict(q=tensor(rng, (1, 5, 64), "float16"), out=tensor(rng, (1, 5, 64), "float16"))):
        with pytest.raises(wf.WfError):
            ok(**kw)


def test_cache_of_more_than_4_gib():
    import torch
    wf = lib()
    rng = np.random.default_rng(27)
    bs, n, kv, dim = 16, 140_000, 8, 128
    st = Step(wf, rng, [100, 20], [1, 130], bs, n_blocks=n)
    spots = n - 1 - np.arange(st.table.size).reshape(st.table.shape)
    cache = torch.zeros((2, n, bs, kv, dim), dtype=torch.bfloat16, device="cuda")
    cache[:, -100:] = tensor(rng, (2, 100, bs, kv, dim), "bfloat16")
    q = tensor(rng, (131, 16, dim), "bfloat16")
    st.kv.table.copy_(torch.from_numpy(spots.astype(np.int32)))
    got = attend(wf, st, cache, None, q)
    small = cache[:, -100:].contiguous()
    st.table = spots - (n - 100)
    check(st, small, None, q, got)


def test_attend_in_a_graph_and_on_another_stream():
    """A captured step replayed after the rows' state has moved on."""
    import torch
    wf = lib()
    rng = np.random.default_rng(28)
    st = Step(wf, rng, [500, 37, 0], [1, 140, 1], 16, spare=3)
    cache, _ = cache_of(rng, st, 2, 128, "bfloat16")
    q, layer, attn = tensor(rng, (st.room, 8, 128), "bfloat16"), wf.KvLayer(cache[0], cache[1]), wf.Attn(max_rows=3, heads=8, dim=128)
    want = attend(wf, st, cache, None, q, attn=attn)
    out, side, graph = torch.full_like(q, 7.0), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        wf.wf_attend(attn, st.kv, st.step, layer, q, out)
    assert (out == 7).all()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    st.kv.len[1] -= 5  # other lengths: the row's tokens lie 5 positions further up
    again = attend(wf, st, cache, None, q, attn=attn)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, again) and not torch.equal(out, want)
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        got = torch.full_like(q, 7.0)
        wf.wf_attend(attn, st.kv, st.step, layer, q, got)
    torch.cuda.synchronize()
    assert torch.equal(got, again)


def test_a_prompt_in_chunks_is_the_prompt():
    """Extend, write and attend, layer by layer as they are used: a prompt at once, in chunks and token by token, in 16 and 8 bits."""
    import torch
    wf = lib()
    rng = np.random.default_rng(29)
    bs, heads, kv, dim, total = 16, 4, 2, 64, 150
    dec, attn, rope = wf.Decode(max_rows=2), wf.Attn(max_rows=2, heads=heads, dim=dim), wf.Rope(dim)
    x = {name: tensor(rng, (total, h, dim), "bfloat16") for name, h in (("q", heads), ("k", kv), ("v", kv))}
    results = []
    for cuts in ([150], [64, 1, 85], [100] + [1] * 50):
        rows = wf.Kv.empty(2, 16, bs, 40)
        cache = torch.zeros((2, 40, bs, kv, dim), dtype=torch.bfloat16, device="cuda")
        layer, out, done = wf.KvLayer(cache[0], cache[1]), [], 0
        for n in cuts:
            step = wf.KvStep(2, n + 2, rows)
            wf.wf_kv_extend(dec, rows, torch.tensor([0, n], dtype=torch.int32, device="cuda"), step)
            pad = lambda t: torch.cat([t[done:done + n], torch.full_like(t[:2], float("nan"))])
            q, k, v = pad(x["q"]), pad(x["k"]), pad(x["v"])
            wf.wf_kv_write(dec, rows, step, layer, k, v, q=q, rope=rope)
            o = torch.zeros_like(q)
            wf.wf_attend(attn, rows, step, layer, q, o, new=n)
            out.append(o[:n])
            done += n
        wf.wf_decode_status(dec)
        wf.wf_attn_status(attn)
        results.append(torch.cat(out).double().cpu().numpy())
    freq = rope.freq
    turned = {n: ref.rotate(f64(x[n]), np.arange(total), freq, False, 1.0) for n in ("q", "k")}
    rounded = {n: torch.from_numpy(t).to(torch.bfloat16).double().numpy() for n, t in turned.items()}
    blocks = lambda t: np.concatenate([t, np.zeros((10, kv, dim))]).reshape(10, 16, kv, dim)
    want, size, _ = ref.attend(rounded["q"], blocks(rounded["k"]), blocks(f64(x["v"])), np.arange(10)[None], [0, total], [total], bs, dim ** -0.5,
                            np.zeros((total, heads, dim)))
    # The queries' and keys' own roundings may differ by a step here and there: a score by 2^-8 of its products.
    score = np.abs(rounded["q"]).sum(-1, keepdims=True) * np.abs(rounded["k"]).max() * dim ** -0.5
    for got in results:
        assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + size * (2.0 ** -7 + 2 * 2.0 ** -8 * score)).all()


@pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))
def test_beams_on_the_cache(eight):
    """A search as it runs: a prompt, rows that share its blocks, a reordering with copies of last blocks and their scales, a token each, attention."""
    import torch
    wf = lib()
    rng = np.random.default_rng(41)
    bs, heads, kv, dim, beams, prompt = 16, 4, 2, 64, 4, 43
    dtype = "bfloat16"
    dec, attn, rope = wf.Decode(max_rows=beams, max_row_blocks=8), wf.Attn(max_rows=beams, heads=heads, dim=dim), wf.Rope(dim)
    rows, moves = wf.Kv.empty(beams, 8, bs, 40), wf.KvMoves(beams)
    cache = torch.zeros((2, 40, bs, kv, dim), dtype=torch.float8_e4m3fn if eight else torch.bfloat16, device="cuda")
    scale = torch.ones((2, 40, kv), device="cuda") if eight else None
    layer = wf.KvLayer(cache[0], cache[1], *((scale[0], scale[1]) if eight else ()))
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    texts = [[] for _ in range(beams)]  # keys and values of each row, as given

    def step(add, new_max):
        s = wf.KvStep(beams, sum(add) + 1, rows)
        wf.wf_kv_extend(dec, rows, dev(add), s)
        t = {n: tensor(rng, (s.max_tokens, h, dim), dtype, spread) for n, h, spread in (("q", heads, 1.5), ("k", kv, rng.uniform(0.5, 8)), ("v", kv, 1))}
        q = torch.empty_like(t["q"])
        wf.wf_kv_write(dec, rows, s, layer, t["k"], t["v"], q=t["q"], q_out=q, rope=rope)
        out = torch.full_like(q, 7.0)
        wf.wf_attend(attn, rows, s, layer, q, out, new=new_max)
        at = 0
        for r, n in enumerate(add):
            texts[r] = texts[r] + [(t["k"][at + i], t["v"][at + i]) for i in range(n)]
            at += n
        return q, out, at

    step([prompt, 0, 0, 0], prompt)
    for parents in ([0, 0, 0, 0], [1, 1, 3, 0], [2, 0, 0, 3], [0, 1, 2, 3], [3, 3, 3, 3]):
        wf.wf_kv_reorder(dec, rows, beams, dev(parents), rows, moves, cache=cache.view(torch.uint8) if eight else cache, scale=scale)
        texts[:] = [list(texts[p]) for p in parents]
        q, out, n = step([1] * beams, 1)
        wf.wf_decode_status(dec)
        wf.wf_attn_status(attn)
        x, table, length = values(cache, scale), rows.table.cpu().numpy(), rows.len.cpu().numpy()
        want, size, small = ref.attend(f64(q), x[0], x[1], table, np.arange(beams + 1), length, bs, dim ** -0.5, np.full(q.shape, 7.0),
                                       None if scale is None else f64(scale[1]))
        off = np.abs(f64(out) - want)
        assert (off[:n] <= bound(size, small, want, f64(q), dtype, eight, dim ** -0.5, int(length.max()), np.abs(x[0]).max())[:n]).all()
        # What the blocks hold is each hypothesis's own keys and values: a rounding to E4M3 (2^-4, once more each time a block's scale grew; what is
        # small in its block to 2^-10 of the block's scale) where 8 bits hold them, as given where 16 do.
        for r in range(beams):
            p = np.arange(length[r])
            blocks, place = table[r, p // bs], p % bs
            held = x[1][blocks, place]
            given = np.stack([f64(v) for _, v in texts[r]])
            assert len(given) == length[r]
            if eight:
                unit = f64(scale[1])[blocks][:, :, None]
                assert (np.abs(held - given) <= np.abs(given) * (2 * 2.0 ** -4 + 2.0 ** -8) + 2 * 2.0 ** -10 * unit).all()
            else:
                assert np.array_equal(held, given)
