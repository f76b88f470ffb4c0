"""wf_kv_write and wf_kv_copy_scales against plain implementations in 64 bits."""
import numpy as np
import pytest

import layer_ref as ref
from gpu_util import lib

pytestmark = pytest.mark.gpu

TYPES = ("float16", "bfloat16")
HALF_STEP = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
LEAST = {"float16": 2.0 ** -25, "bfloat16": 0.0}  # half the distance of the subnormals


def f64(t):
    return t.float().cpu().double().numpy()


class Step:
    """Rows behind contexts `have` with `add` new tokens each, on shuffled blocks, and room for `spare` tokens more."""

    def __init__(self, wf, rng, have, add, bs, spare=0, n_blocks=None):
        import torch
        have, add = np.asarray(have, np.int64), np.asarray(add, np.int64)
        self.rows, self.bs, self.have, self.add = len(have), bs, have, add
        length = have + add
        nb = -(-length // bs)
        width = max(1, int(nb.max()))
        n = n_blocks or int(nb.sum()) + 3
        ids = rng.permutation(n).astype(np.int32)
        self.table = np.full((self.rows, width), -1, np.int32)
        self.table[np.arange(width) < nb[:, None]] = ids[:int(nb.sum())]
        self.start = np.concatenate([[0], np.cumsum(add)]).astype(np.int32)
        self.tokens, self.n_blocks = int(add.sum()), n
        self.room = max(1, self.tokens + spare)
        self.slot, self.pos = np.full(self.room, -1, np.int64), np.zeros(self.room, np.int32)
        self.row = np.full(self.room, -1, np.int32)
        for r in range(self.rows):
            p = np.arange(have[r], length[r])
            at = slice(int(self.start[r]), int(self.start[r + 1]))
            self.slot[at], self.pos[at], self.row[at] = self.table[r, p // bs].astype(np.int64) * bs + p % bs, p, r
        self.len = length.astype(np.int32)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        self.kv = wf.Kv(dev(self.table), dev(self.len), torch.zeros(n, dtype=torch.int32, device="cuda"),
                        torch.zeros(2, dtype=torch.int64, device="cuda"), bs)
        self.step = wf.KvStep(self.rows, self.room, self.kv)
        for name in ("slot", "pos", "row", "start"):
            getattr(self.step, name).copy_(dev(getattr(self, name)))
        self.decode = wf.Decode(max_rows=self.rows)


def tensor(rng, shape, dtype, spread=1.0):
    import torch
    return torch.from_numpy(rng.standard_normal(shape) * spread).to(getattr(torch, dtype)).cuda()


def cache_of(rng, st, kv, dim, dtype):
    """[2, n_blocks, bs, kv, dim] and scales (8 bits)."""
    import torch
    if dtype != "float8_e4m3fn":
        return tensor(rng, (2, st.n_blocks, st.bs, kv, dim), dtype), None
    cache = torch.from_numpy(ref.eight(rng.standard_normal((2, st.n_blocks, st.bs, kv, dim)) * 90)).to(torch.float8_e4m3fn).cuda()
    return cache, torch.from_numpy(2.0 ** rng.integers(-9, -5, (2, st.n_blocks, kv))).float().cuda()


def near(got, want, dtype, x, magnitude=1.0):
    """Half a step of the type for the rounding; before it, in 32 bits, cos and sin to 2^-22 (the angle to 2^-25 of a turn's
    6.3, sincospi to 2 steps, the product with the magnitude), two products and a sum, each to 2^-24."""
    size = np.abs(x).max(axis=-1, keepdims=True) * 2 * magnitude
    off = np.abs(got - want)
    most = HALF_STEP[dtype] * np.abs(want) * (1 + 2.0 ** -8) + LEAST[dtype] + size * 2.0 ** -21
    assert (off <= most).all(), f"off by {np.max(off - most)} more than allowed at {np.argwhere(off > most)[0]}"


ROPES = [dict(dim=0), dict(), dict(interleaved=True), dict(dim=48), dict(dim=32, interleaved=True), dict(dim=10), dict(dim=10, interleaved=True),
         dict(dim=2), dict(factor=8.0, context=4096, magnitude=1.2079), dict(factor=4.0, base=500000.0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", (64, 128))
@pytest.mark.parametrize("rope", ROPES, ids=lambda r: "-".join(f"{k}{v}" for k, v in r.items()) or "whole")
def test_write_16_bits(dtype, dim, rope):
    import torch
    wf = lib()
    rng = np.random.default_rng(dim + len(str(rope)))
    st = Step(wf, rng, [0, 5, 160, 31, 1000, 7, 70000], [33, 1, 1, 0, 18, 1, 3], 16, spare=9)
    heads, kv = 6, 2
    q, k, v = tensor(rng, (st.room, heads, dim), dtype), tensor(rng, (st.room, kv, dim), dtype), tensor(rng, (st.room, kv, dim), dtype)
    cache, _ = cache_of(rng, st, kv, dim, dtype)
    was = cache.clone()
    q_out = torch.full_like(q, 7.0)
    rp = wf.Rope(**{"dim": dim, **rope})
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1]), k, v, q=q, q_out=q_out, rope=rp)
    wf.wf_decode_status(st.decode)
    n = st.tokens
    turned = lambda x: ref.rotate(f64(x)[:n], st.pos[:n], rp.freq, rp.interleaved, rp.magnitude)
    near(f64(q_out)[:n], turned(q), dtype, f64(q)[:n], rp.magnitude)
    assert (q_out[n:] == 7).all()
    flat = cache.flatten(1, 2)
    near(f64(flat[0])[st.slot[:n]], turned(k), dtype, f64(k)[:n], rp.magnitude)
    assert np.array_equal(f64(flat[1])[st.slot[:n]], f64(v)[:n])
    rest = np.setdiff1d(np.arange(st.n_blocks * st.bs), st.slot[:n])
    assert torch.equal(flat[:, rest], was.flatten(1, 2)[:, rest])  # what is not a slot of the step stays
    if rp.dim < dim:  # and what does not turn keeps its bits
        assert torch.equal(q_out[:n, :, rp.dim:], q[:n, :, rp.dim:])
    # In place, the same.
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1]), k, v, q=q, rope=rp)
    assert torch.equal(q[:n], q_out[:n])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("eight", (False, True))
@pytest.mark.parametrize("rope", (dict(), dict(interleaved=True), dict(dim=10)), ids=("half", "interleaved", "part"))
def test_write_strides_and_alignment(dtype, eight, rope):
    """Tensors that are views: of one product for queries, keys and values, on 2-byte boundaries, heads before tokens; a cache whose
    keys and values lie side by side."""
    import torch
    wf = lib()
    rng = np.random.default_rng(3)
    dim, heads, kv = 64, 3, 2
    st = Step(wf, rng, [3, 0, 40], [20, 7, 1], 8, spare=2)
    q, k, v = tensor(rng, (st.room, heads, dim), dtype), tensor(rng, (st.room, kv, dim), dtype), tensor(rng, (st.room, kv, dim), dtype)
    rp = wf.Rope(**{"dim": dim, **rope})
    cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn" if eight else dtype)
    scales = lambda s: () if s is None else (s[0], s[1])

    def run(cache, scale, q, k, v, q_out):
        wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1], *scales(scale)), k, v, q=q, q_out=q_out, rope=rp)
        return q_out, cache, scale
    copy = lambda t: None if t is None else t.clone()
    want = run(cache.clone(), copy(scale), q, k, v, torch.zeros_like(q))
    bytes_of = lambda t: t.contiguous().view(torch.uint8)

    def same(got):
        assert torch.equal(got[0], want[0]) and torch.equal(bytes_of(got[1]), bytes_of(want[1]))
        assert scale is None or torch.equal(got[2], want[2])
    whole = torch.cat([q, k, v], 1)  # one product's columns
    same(run(cache.clone(), copy(scale), whole[:, :heads], whole[:, heads:heads + kv], whole[:, heads + kv:], torch.zeros_like(q)))
    odd = torch.zeros(whole.numel() + 1, dtype=whole.dtype, device="cuda")[1:].view_as(whole).copy_(whole)  # 2 bytes off
    same(run(cache.clone(), copy(scale), odd[:, :heads], odd[:, heads:heads + kv], odd[:, heads + kv:], torch.zeros_like(q)))
    turn = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # heads outermost
    same(run(cache.clone(), copy(scale), turn(q), turn(k), turn(v), turn(torch.zeros_like(q))))
    beside = cache.view(torch.uint8).view(2, st.n_blocks, st.bs, kv, -1).permute(1, 2, 3, 0, 4).contiguous().permute(3, 0, 1, 2, 4).view(cache.dtype)
    same(run(beside, copy(scale), q, k, v, torch.zeros_like(q)))
    by_head = cache.transpose(2, 3).contiguous().transpose(2, 3)  # [block][head][place]
    same(run(by_head, copy(scale), q, k, v, torch.zeros_like(q)))


def test_far_positions():
    """Angles at positions up to 2^31 - 1 are those of 64-bit arithmetic."""
    import torch
    wf = lib()
    rng = np.random.default_rng(5)
    dim = 128
    st = Step(wf, rng, [0], [40], 16)
    pos = np.concatenate([2 ** 31 - 1 - np.arange(20), rng.integers(2 ** 20, 2 ** 31, 20)]).astype(np.int32)
    st.step.pos.copy_(torch.from_numpy(pos))
    q, k = tensor(rng, (40, 1, dim), "float16"), tensor(rng, (40, 1, dim), "float16")
    cache, _ = cache_of(rng, st, 1, dim, "float16")
    rp = wf.Rope(dim)
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1]), k, k, q=q, rope=rp, q_out=(out := torch.empty_like(q)))
    # In 64 bits the angle itself (up to 2^31) is known to 2^-22 only: the reference reduces it in whole numbers.
    from fractions import Fraction
    two_pi = Fraction(2 * 3141592653589793238462643383279502884197, 10 ** 39)
    small = np.array([[float((int(p) * Fraction(f)) % two_pi) for f in rp.freq] for p in pos])
    x = f64(q)
    a, b, c, s = x[..., :64], x[..., 64:], np.cos(small)[:, None], np.sin(small)[:, None]
    near(f64(out), np.concatenate([a * c - b * s, b * c + a * s], -1), "float16", x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,kv,bs,have,add", [
    (64, 1, 16, [0], [1]), (128, 2, 16, [5, 16, 0, 31, 15], [1, 1, 1, 1, 1]), (128, 8, 16, [3, 0, 64, 7], [70, 33, 1, 0]),
    (64, 5, 1, [4, 0], [9, 3]), (64, 3, 24, [1000, 23, 24, 25], [1, 2, 30, 100]), (128, 2, 100, [99, 250], [250, 3]),
    (64, 9, 256, [100, 0], [700, 64]), (128, 1, 7, list(range(40)), [1] * 40), (64, 2, 64, [10] * 700, [1] * 700),
    (64, 2, 32, [0, 9], [4000, 5])])
def test_write_8_bits(dtype, dim, kv, bs, have, add):
    """Every scale and every element, given the keys and values as a cache in 16 bits has them."""
    import torch
    wf = lib()
    rng = np.random.default_rng(dim * bs + kv)
    st = Step(wf, rng, have, add, bs, spare=5)
    spread = 2.0 ** rng.integers(-6, 4, (st.room, 1, 1))  # so that scales grow, or do not
    k = tensor(rng, (st.room, kv, dim), dtype, spread)
    v = tensor(rng, (st.room, kv, dim), dtype, 2.0 ** rng.integers(-12, 1, (st.room, kv, 1)))
    q = tensor(rng, (st.room, 2 * kv, dim), dtype)
    rp = wf.Rope(dim)
    full, _ = cache_of(rng, st, kv, dim, dtype)
    q16, q8 = torch.zeros_like(q), torch.zeros_like(q)
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(full[0], full[1]), k, v, q=q, q_out=q16, rope=rp)
    cache, scale = cache_of(rng, st, kv, dim, "float8_e4m3fn")
    want, want_scale = f64(cache), f64(scale)
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1], scale[0], scale[1]), k, v, q=q, q_out=q8, rope=rp)
    wf.wf_decode_status(st.decode)
    live = st.slot >= 0
    for plane in range(2):
        x = np.zeros((st.room, kv, dim))
        x[live] = f64(full[plane].flatten(0, 1))[st.slot[live]]
        ref.write8(want[plane], want_scale[plane], st.slot, bs, x)
    assert np.array_equal(f64(scale), want_scale)
    assert np.array_equal(f64(cache), want)
    assert torch.equal(q8, q16)


def test_write_8_bits_extremes():
    """Zeros, the largest and least numbers, infinities and NaN: their places and the scale they leave the others."""
    import torch
    wf = lib()
    rng = np.random.default_rng(8)
    st = Step(wf, rng, [0] * 8, [3] * 8, 4)
    k = torch.zeros((24, 1, 64), dtype=torch.bfloat16, device="cuda")
    k[3:6] = 3e38
    k[6:9] = 1e-38
    k[9, 0, 0], k[10, 0, 1], k[11, 0, 2], k[9, 0, 3] = float("inf"), float("-inf"), float("nan"), 448.0
    k[12, 0, 0], k[13, 0, 0] = 448 * 2.0 ** 20, 1.0
    k[15, 0, 0] = 450 * 2.0 ** 20
    k[18:21] = float("nan")
    k[21, 0, 0], k[22, 0, :3] = 1.75, torch.tensor([1.0, 2.0 ** -17, 2.0 ** -18], dtype=torch.bfloat16)
    cache, scale = cache_of(rng, st, 1, 64, "float8_e4m3fn")
    want, want_scale = f64(cache), f64(scale)
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1], scale[0], scale[1]), k, k)
    for plane in range(2):
        ref.write8(want[plane], want_scale[plane], st.slot, 4, f64(k))
    assert np.array_equal(f64(scale), want_scale)
    assert np.array_equal(f64(cache), want, equal_nan=True)
    blocks = st.table[:, 0]
    assert scale[0, blocks[[0, 1, 3, 4, 5]], 0].tolist() == [2.0 ** -64, 2.0 ** 63, 1.0, 2.0 ** 20, 2.0 ** 21]


def test_write_twice_is_the_same():
    """A step written again leaves cache and scales as they are."""
    import torch
    wf = lib()
    rng = np.random.default_rng(9)
    st = Step(wf, rng, [5, 0, 37], [1, 40, 1], 16)
    k = tensor(rng, (st.room, 4, 128), "bfloat16", 30)
    cache, scale = cache_of(rng, st, 4, 128, "float8_e4m3fn")
    layer = wf.KvLayer(cache[0], cache[1], scale[0], scale[1])
    wf.wf_kv_write(st.decode, st.kv, st.step, layer, k, k, rope=wf.Rope(128))
    once = cache.view(torch.uint8).clone(), scale.clone()
    wf.wf_kv_write(st.decode, st.kv, st.step, layer, k, k, rope=wf.Rope(128))
    assert torch.equal(cache.view(torch.uint8), once[0]) and torch.equal(scale, once[1])


@pytest.mark.parametrize("eight", (False, True))
def test_slots_outside_the_cache(eight):
    import torch
    wf = lib()
    rng = np.random.default_rng(10)
    st = Step(wf, rng, [0], [8], 4)
    k = tensor(rng, (8, 1, 64), "float16")
    cache, scale = cache_of(rng, st, 1, 64, "float8_e4m3fn" if eight else "float16")
    slot = st.slot.copy()
    slot[[2, 5]] = st.n_blocks * 4 + np.array([0, 2 ** 40])
    st.step.slot.copy_(torch.from_numpy(slot))
    was = cache.view(torch.uint8).clone()
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1], *((scale[0], scale[1]) if eight else ())), k, k)
    with pytest.raises(wf.WfError, match="outside the cache"):
        wf.wf_decode_status(st.decode)
    wf.wf_decode_status(st.decode)  # reported once
    flat, was = cache.view(torch.uint8).flatten(1, 2), was.flatten(1, 2)
    # In 8 bits such a token cuts its block's part in two, which the call does not take: what the step's blocks then hold is open.
    rest = np.setdiff1d(np.arange(st.n_blocks * 4), st.slot) if eight else np.union1d(np.setdiff1d(np.arange(st.n_blocks * 4), st.slot), st.slot[[2, 5]])
    assert torch.equal(flat[:, rest], was[:, rest])
    ok = slot[np.delete(np.arange(8), [2, 5])]
    if not eight:
        assert np.array_equal(f64(cache.flatten(1, 2)[0])[ok], f64(k)[np.delete(np.arange(8), [2, 5])])


def test_cache_of_more_than_4_gib():
    """Slots whose bytes lie past 2^32."""
    import torch
    wf = lib()
    rng = np.random.default_rng(11)
    bs, n, kv, dim = 16, 140_000, 8, 128  # 4.6 GB a plane of 16 bits
    st = Step(wf, rng, [0, 20], [40, 1], bs, n_blocks=n)
    table = st.table.copy()
    table[:, :] = n - 1 - np.arange(table.size).reshape(table.shape)
    slot = np.concatenate([table[0, np.arange(40) // bs].astype(np.int64) * bs + np.arange(40) % bs, [int(table[1, 1]) * bs + 4]])
    st.step.slot.copy_(torch.from_numpy(slot))
    cache = torch.zeros((2, n, bs, kv, dim), dtype=torch.bfloat16, device="cuda")
    k = tensor(rng, (41, kv, dim), "bfloat16")
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1]), k, k)
    at = torch.from_numpy(slot).cuda()
    assert torch.equal(cache[0].flatten(0, 1)[at], k) and torch.equal(cache[1].flatten(0, 1)[at], k)
    assert int((cache[0, -100:] != 0).any(-1).any(-1).sum()) == 41 and not cache[0, :-100].any()


def test_copy_scales_follows_a_reordering():
    """Beams on an 8-bit cache: rows that copy a shared last block have its scales."""
    import torch
    wf = lib()
    rng = np.random.default_rng(12)
    bs, kv, dim, rows = 8, 3, 64, 4
    cache = torch.from_numpy(ref.eight(rng.standard_normal((2, 20, bs, kv, dim)) * 90)).to(torch.float8_e4m3fn).cuda()
    scale = torch.from_numpy(rng.random((2, 20, kv)).astype(np.float32)).cuda()
    dec = wf.Decode(max_rows=rows, max_row_blocks=4)
    kvr = wf.Kv.empty(rows, 4, bs, 20)
    step = wf.KvStep(rows, 64, kvr)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    wf.wf_kv_extend(dec, kvr, dev([21, 0, 0, 0]), step)
    moves, was, was8 = wf.KvMoves(rows), scale.clone(), cache.view(torch.uint8).clone()
    wf.wf_kv_reorder(dec, kvr, 4, dev([0, 0, 0, 0]), kvr, moves, cache=cache.view(torch.uint8), scale=scale)
    wf.wf_decode_status(dec)
    copies = moves.copies.cpu().numpy()
    assert (copies[1:] >= 0).all() and copies[0, 0] == -1
    for a, b in copies[1:]:
        assert torch.equal(scale[:, b], was[:, a]) and torch.equal(cache.view(torch.uint8)[:, b, :5], was8[:, a, :5])
    rest = np.setdiff1d(np.arange(20), copies[1:, 1])
    assert torch.equal(scale[:, rest], was[:, rest])
    bad = moves.copies.clone()
    bad[2, 1], bad[3, 0] = 20, -2
    before = scale.clone()
    wf.wf_kv_copy_scales(dec, kvr, bad, scale)
    with pytest.raises(wf.WfError, match="outside the cache"):
        wf.wf_decode_status(dec)
    assert torch.equal(scale, before)  # row 1's copy is as it was


def test_write_in_a_graph_and_on_another_stream():
    import torch
    wf = lib()
    rng = np.random.default_rng(13)
    st = Step(wf, rng, [5, 0, 37], [1, 40, 1], 16, spare=3)
    k, q = tensor(rng, (st.room, 4, 128), "bfloat16"), tensor(rng, (st.room, 8, 128), "bfloat16")
    rp = wf.Rope(128)
    for eight in (False, True):
        cache, scale = cache_of(rng, st, 4, 128, "float8_e4m3fn" if eight else "bfloat16")
        layers = []
        for _ in range(2):
            c, s = cache.clone(), None if scale is None else scale.clone()
            layers.append((c, s, wf.KvLayer(c[0], c[1], *(() if s is None else (s[0], s[1])))))
        outs = torch.zeros_like(q), torch.zeros_like(q)
        wf.wf_kv_write(st.decode, st.kv, st.step, layers[0][2], k, k, q=q, q_out=outs[0], rope=rp)
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            wf.wf_kv_write(st.decode, st.kv, st.step, layers[1][2], k, k, q=q, q_out=outs[1], rope=rp)
        assert not outs[1].any()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(layers[0][0].view(torch.uint8), layers[1][0].view(torch.uint8))
