"""wf_attend where scores, weights and values are extreme, and where a row's positions are shared among the GPU's blocks."""
import numpy as np
import pytest

from gpu_util import lib
from test_gpu_attend import attend, check
from test_gpu_write import HALF_STEP, TYPES, Step, cache_of, f64, tensor

pytestmark = pytest.mark.gpu
EIGHT = pytest.mark.parametrize("eight", (False, True), ids=("16", "8"))


def layer_type(eight, dtype):
    return "float8_e4m3fn" if eight else dtype


@EIGHT
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scaling", (0.0, 2.0 ** -140, 1.0, 4.0))
@pytest.mark.parametrize("have,add", [([300, 17], [1, 1]), ([300, 17], [40, 300]), ([6000], [70])], ids=("few", "many", "split"))
def test_scales(have, add, scaling, dtype, eight):
    """Any scale >= 0; with 0 every output is the mean of the values that its token sees."""
    wf = lib()
    rng = np.random.default_rng(51)
    st = Step(wf, rng, have, add, 16, spare=3)
    cache, scale = cache_of(rng, st, 2, 64, layer_type(eight, dtype))
    q = tensor(rng, (st.room, 6, 64), dtype)
    check(st, cache, scale, q, attend(wf, st, cache, scale, q, scaling=scaling), scaling)
    check(st, cache, scale, q, attend(wf, st, cache, scale, q, scaling=scaling, new=1), scaling)


@EIGHT
@pytest.mark.parametrize("n,value", [(200, 96), (60_000, 1)])
@pytest.mark.parametrize("add", (1, 40), ids=("few", "many"))
def test_the_tail_behind_one_key(add, n, value, eight):
    """The first key has nearly all the weight and a value of 0: what is left are n weights of 2^-26 of it.

    Weights in half floats lie 2^-24 apart below 2^-14, and the largest is 2^7 at least, so that each is off by 2^-25 of 2^7 at most, or by half a
    step; a score of 26 (in base 2) is off by 26 * 2^-23, sums of 60,000 by 2^-16 at most."""
    import torch
    wf = lib()
    rng = np.random.default_rng(52)
    st = Step(wf, rng, [n], [add], 16)
    cache = torch.zeros((2, st.n_blocks, 16, 1, 64), dtype=torch.float16, device="cuda")
    cache[1] = value
    first = int(st.table[0, 0])
    cache[0, first, 0, 0, 0], cache[1, first, 0] = 36, 0
    scale = torch.ones((2, st.n_blocks, 1), device="cuda") if eight else None
    if eight:
        cache = cache.to(torch.float8_e4m3fn)
    q = torch.zeros((add, 2, 64), dtype=torch.float16, device="cuda")
    q[:, :, 0] = 4
    rest = (n + np.arange(add)) * np.exp(-18.0)  # 4 * 36 / 8
    want = value * (rest / (1 + rest))[:, None, None]
    got = f64(attend(wf, st, cache, scale, q))
    least = 2.0 ** -32 * (n + add) * value
    assert (np.abs(got - want) <= want * (2 * HALF_STEP["float16"] + 26 * 2.0 ** -22 + 2.0 ** -15) + least * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("bs,kv,dim", [(7, 2, 64), (100, 1, 128), (1, 2, 64), (30, 4, 128)])
def test_blocks_that_no_box_fits_again_and_again(bs, kv, dim):
    """Prompts over blocks whose positions are copied one by one (no multiple of 8): many tiles under way, every call the same."""
    import torch
    wf = lib()
    rng = np.random.default_rng(55)
    st = Step(wf, rng, [900, 0, 40], [200, 700, 65], bs)
    cache, _ = cache_of(rng, st, kv, dim, "bfloat16")
    q = tensor(rng, (st.room, 2 * kv, dim), "bfloat16")
    attn = wf.Attn(max_rows=3, heads=2 * kv, dim=dim)
    first = attend(wf, st, cache, None, q, attn=attn)
    check(st, cache, None, q, first)
    for _ in range(30):
        assert torch.equal(first, attend(wf, st, cache, None, q, attn=attn))


@pytest.mark.parametrize("eight,dtype,bs,heads", [(False, "bfloat16", 16, 4), (False, "float16", 100, 4), (False, "bfloat16", 64, 130), (True, "float16", 16, 4),
                                                  (True, "bfloat16", 64, 4)], ids=("boxes", "no-boxes", "large-group", "8-half", "8-bfloat"))
def test_waits_that_run_out(eight, dtype, bs, heads):
    """A call whose waits give up, at the first or some later one, comes to its end and says so; the next one on the same scratch is right."""
    import torch
    wf = lib()
    rng = np.random.default_rng(56)
    st = Step(wf, rng, [3000, 0, 40], [300, 700, 65], bs, spare=2)
    cache, scale = cache_of(rng, st, 1, 64, layer_type(eight, dtype))
    q = tensor(rng, (st.room, heads, 64), dtype)
    want = attend(wf, st, cache, scale, q)
    attn = wf.Attn(max_rows=3, heads=heads, dim=64)
    layer, out = wf.KvLayer(cache[0], cache[1], *(() if scale is None else (scale[0], scale[1]))), torch.full_like(q, 7.0)
    for polls in (0, 0, 1, 2, 4, 8):
        wf.wf_attn_limit_waits(attn, polls)
        for _ in range(2):
            wf.wf_attend(attn, st.kv, st.step, layer, q, out)
        try:
            wf.wf_attn_status(attn)
            assert polls
        except wf.WfError as e:
            assert e.code == wf.WF_ETIMEOUT
        wf.wf_attn_status(attn)  # reported once
        assert (out[st.tokens:] == 7).all()
        wf.wf_attn_limit_waits(attn)
        for _ in range(2):
            assert torch.equal(attend(wf, st, cache, scale, q, attn=attn), want)
    for bad in (-1, (1 << 20) + 1):
        with pytest.raises(wf.WfError):
            wf.wf_attn_limit_waits(attn, bad)


LATER = [  # have, add, block size, heads, key heads, dim, tokens of the first row whose values are no numbers
    ([20, 5], [4, 1], 16, 4, 2, 64, (2,)), ([20, 5], [4, 1], 7, 8, 2, 128, (3,)), ([500], [16], 16, 1, 1, 64, (1, 9)),
    ([300, 0], [200, 90], 16, 8, 2, 128, (70,)), ([60], [600], 16, 2, 2, 64, (127, 130, 400)), ([0], [300], 24, 7, 1, 128, (0, 299)),
    ([90, 3], [250, 40], 7, 6, 2, 64, (33, 34)), ([5000], [80], 32, 4, 1, 128, (0, 41)), ([3], [70], 16, 130, 1, 64, (50,))]


def same(got, want):
    """Finite numbers alike, and the others in the same places."""
    import torch
    fine = want.isfinite()
    return torch.equal(got.isfinite(), fine) and torch.equal(got[fine], want[fine])


@EIGHT
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("have,add,bs,heads,kv,dim,at", LATER, ids=range(len(LATER)))
def test_a_value_reaches_no_earlier_token(have, add, bs, heads, kv, dim, at, dtype, eight):
    """Values that are infinite or no numbers reach the outputs of their token and those behind it, in their element and of their head, and no others.
    (Infinite or no number: the second product of attend_kernel in bfloat16 takes a weight's remainder, and 0 times an infinity is no number.)"""
    import torch
    wf = lib()
    rng = np.random.default_rng(53)
    st = Step(wf, rng, have, add, bs, spare=2)
    cache, scale = cache_of(rng, st, kv, dim, layer_type(eight, dtype))
    q = tensor(rng, (st.room, heads, dim), dtype, 0.5)
    for new in (0, 1):
        want = attend(wf, st, cache, scale, q, new=new)
        assert want.isfinite().all()
        for bad in ((float("nan"),) if eight else (float("inf"), float("-inf"), float("nan"))):
            held, expect = cache.clone(), want.clone()
            for i, token in enumerate(at):
                p, head, d = have[0] + token, i % kv, (5 + 9 * i) % dim
                block, place = int(st.table[0, p // bs]), p % bs
                if eight:
                    held.view(torch.uint8)[1, block, place, head, d] = 0xFF
                else:
                    held[1, block, place, head, d] = bad
                group = heads // kv
                expect[token:add[0], head * group:(head + 1) * group, d] = bad
            assert same(attend(wf, st, held, scale, q, new=new), expect), (new, bad)


def test_infinities_of_both_signs_and_whole_values():
    """An infinity of each sign in one element make NaN from the later one on; a token whose whole value is infinite leaves those before it alone."""
    import torch
    wf = lib()
    rng = np.random.default_rng(54)
    for add, new in ((4, 0), (150, 0), (150, 1)):
        st = Step(wf, rng, [33], [add], 16)
        cache, _ = cache_of(rng, st, 1, 64, "bfloat16")
        q = tensor(rng, (add, 2, 64), "bfloat16", 0.5)
        expect = attend(wf, st, cache, None, q, new=new)
        first, second, whole = add // 4, add // 2, add - 1
        put = lambda token: cache[1, int(st.table[0, (33 + token) // 16]), (33 + token) % 16, 0]
        put(first)[7], put(second)[7] = float("inf"), float("-inf")
        put(whole)[:] = float("inf")
        expect[first:second, :, 7] = float("inf")
        expect[whole] = float("inf")
        expect[second:, :, 7] = float("nan")
        assert same(attend(wf, st, cache, None, q, new=new), expect)


def test_outputs_in_the_queries_memory_are_refused():
    """In place, a head or a token further on, with other strides; two parts of one product's columns are apart."""
    import torch
    wf = lib()
    rng = np.random.default_rng(57)
    st = Step(wf, rng, [40, 3], [1, 30], 16)
    cache, _ = cache_of(rng, st, 2, 64, "float16")
    layer, attn = wf.KvLayer(cache[0], cache[1]), wf.Attn(max_rows=2, heads=4, dim=64)
    whole = torch.cat([tensor(rng, (st.room + 1, 4, 64), "float16"), torch.full((st.room + 1, 4, 64), 7.0, dtype=torch.float16, device="cuda")], 1)
    q = whole[:-1, :4]
    was = whole.clone()
    for out in (q, whole[:-1, 1:5], whole[:-1, 3:7], whole[1:, :4], whole.view(-1, 4, 64)[:st.room], whole.view(-1, 4, 64)[1:st.room + 1]):
        with pytest.raises(wf.WfError, match="queries' memory"):
            wf.wf_attend(attn, st.kv, st.step, layer, q, out)
    assert torch.equal(whole, was)
    check(st, cache, None, q.contiguous(), attend(wf, st, cache, None, q, out=whole[:-1, 4:]))
    assert torch.equal(whole[:, :4], was[:, :4])


def test_a_reordering_whose_scales_are_refused_changes_nothing():
    """Scales that wf_kv_copy_scales would not take are refused before the rows are reordered."""
    import torch
    wf = lib()
    dec, rows, moves = wf.Decode(max_rows=2, max_row_blocks=4), wf.Kv.empty(2, 4, 8, 20), wf.KvMoves(2)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    wf.wf_kv_extend(dec, rows, dev([21, 3]), wf.KvStep(2, 24, rows))
    was = rows.table.clone(), rows.len.clone()
    for scale in (torch.ones((2, 20, 1025), device="cuda"), torch.ones((2, 19, 4), device="cuda"), torch.ones((2, 20, 4), device="cuda").half()):
        with pytest.raises(wf.WfError):
            wf.wf_kv_reorder(dec, rows, 2, dev([1, 0]), rows, moves, scale=scale)
        assert torch.equal(rows.table, was[0]) and torch.equal(rows.len, was[1])


JOINS = [([40_000], [1], 8, 1, 128, 1), ([20_000, 7, 9_000], [1, 1, 2], 6, 2, 64, 0), ([20_000], [40], 8, 1, 64, 0), ([9_000, 30], [500, 2], 4, 2, 128, 0)]




@EIGHT
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("have,add,heads,kv,dim,new", JOINS, ids=("decode", "few", "many", "long"))
def test_every_tile_counts_once(have, add, heads, kv, dim, new, dtype, eight):
    """Equal scores, and values of 1 in one element for each 64 positions: an element is the share of the positions whose value it has.  No element has more than
    six such tiles, so that one that is lost, doubled or stale moves its element by a seventh at least.

    Weights are equal powers of two, their sums exact (whole numbers below 2^24 of them), the joins' factors 1; what is left are a division, a product
    and a rounding."""
    import torch
    wf = lib()
    rng = np.random.default_rng(58)
    st = Step(wf, rng, have, add, 16)
    cache = torch.zeros((2, st.n_blocks, 16, kv, dim), dtype=getattr(torch, dtype), device="cuda")
    for r, n in enumerate(st.len):
        p = np.arange(n)
        slot = torch.from_numpy(st.table[r, p // 16].astype(np.int64) * 16 + p % 16).cuda()
        one = torch.zeros((n, dim), dtype=cache.dtype, device="cuda")
        one[torch.from_numpy(p).cuda(), torch.from_numpy(p // 64 % dim).cuda()] = 1
        cache[1].flatten(0, 1)[slot] = one[:, None]
    scale = None
    if eight:
        cache, scale = cache.to(torch.float8_e4m3fn), torch.ones((2, st.n_blocks, kv), device="cuda")
    attn = wf.Attn(max_rows=st.rows, heads=heads, dim=dim)
    q = torch.zeros((st.room, heads, dim), dtype=getattr(torch, dtype), device="cuda")
    for _ in range(3):
        got = f64(attend(wf, st, cache, scale, q, new=new, attn=attn))
        for r, n in enumerate(st.len):
            for i in range(int(add[r])):
                seen = have[r] + i + 1
                want = np.bincount(np.arange(seen) // 64 % dim, minlength=dim) / seen
                off = np.abs(got[int(st.start[r]) + i] - want)
                assert (off <= want * (HALF_STEP[dtype] + 2.0 ** -22) + (2.0 ** -25 if dtype == "float16" else 0)).all(), (r, i)


@EIGHT
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("have,add,heads,new", [(20_000, 1, 16, 1), (20_000, 40, 8, 0)], ids=("few", "many"))
def test_one_key_has_all_the_weight(have, add, heads, new, dtype, eight):
    """The first and the last position of every tile of 64 (few queries) or 128 (many) in turn: each query's own key there has all the weight, and the output
    is its value, whichever part of the row it lies in.  The other weights are e^-64 of it."""
    import torch
    wf = lib()
    rng = np.random.default_rng(59)
    dim, tile = 64, 64 if add == 1 else 128
    st = Step(wf, rng, [have], [add], 16)
    n = have + add
    p = np.arange(n)
    slot = torch.from_numpy(st.table[0, p // 16].astype(np.int64) * 16 + p % 16).cuda()
    cache = torch.zeros((2, st.n_blocks, 16, 1, dim), dtype=getattr(torch, dtype), device="cuda")
    value = torch.from_numpy((p[:, None] * 7 + np.arange(dim) * 3) % 15 - 7).to(cache.dtype).cuda()
    cache[1].flatten(0, 1)[slot] = value[:, None]
    scale = torch.ones((2, st.n_blocks, 1), device="cuda") if eight else None
    attn = wf.Attn(max_rows=1, heads=heads, dim=dim)
    axis = np.arange(add * heads).reshape(add, heads) % dim  # a query looks along one element
    q = torch.zeros((add, heads, dim), dtype=cache.dtype, device="cuda")
    q.scatter_(2, torch.from_numpy(axis).cuda()[..., None], 8.0)
    spots = np.unique(np.concatenate([np.arange(0, have, tile), np.arange(tile - 1, have, tile), [have - 1]]))
    most = min(dim, add * heads)
    for i in range(0, len(spots), most):
        at = np.resize(spots[i:i + most], most)  # by element
        held = cache.clone()
        held[0].flatten(0, 1)[slot[torch.from_numpy(at).cuda()], 0, torch.arange(most, device="cuda")] = 8.0
        if eight:
            held = held.to(torch.float8_e4m3fn)
        got = attend(wf, st, held, scale, q, scaling=1.0, new=new, attn=attn)
        want = value[torch.from_numpy(at[axis]).cuda()]
        assert ((got.float() - want.float()).abs() <= 1e-6).all(), at


def test_two_scratches_at_once():
    """Prompts and decoding on two streams from two threads, each with a scratch of its own."""
    import threading
    import torch
    wf = lib()
    rng = np.random.default_rng(60)
    work = []
    for have, add, heads, dim, eight in (([3000, 0, 900], [200, 500, 1], 8, 128, False), ([8000, 40] * 3, [1, 300] * 3, 4, 64, True)):
        st = Step(wf, rng, have, add, 16)
        cache, scale = cache_of(rng, st, 2, dim, layer_type(eight, "bfloat16"))
        layer = wf.KvLayer(cache[0], cache[1], *(() if scale is None else (scale[0], scale[1])))
        q = tensor(rng, (st.room, heads, dim), "bfloat16")
        attn = wf.Attn(max_rows=st.rows, heads=heads, dim=dim)
        work.append((st, layer, q, attn, attend(wf, st, cache, scale, q, attn=attn), torch.cuda.Stream(), [torch.empty_like(q) for _ in range(20)]))
    torch.cuda.synchronize()

    def run(st, layer, q, attn, want, stream, outs):
        for out in outs:
            wf.wf_attend(attn, st.kv, st.step, layer, q, out, stream=stream)
    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for st, layer, q, attn, want, stream, outs in work:
        wf.wf_attn_status(attn)
        assert all(torch.equal(o, want) for o in outs)


def odd_scales(rng, scale):
    """No powers of two, and some 0."""
    import torch
    new = torch.from_numpy(rng.uniform(2.0 ** -9, 2.0 ** -5, scale.shape)).float().cuda()
    new[torch.from_numpy(rng.random(scale.shape) < 0.1).cuda()] = 0
    return new


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("have,add,new", [([300, 17], [1, 1], 1), ([300, 17], [40, 200], 0)], ids=("few", "many"))
def test_attention_over_scales_of_any_value(have, add, new, dtype):
    """A value's scale of 0 counts as 2^-64, a key's as 0."""
    wf = lib()
    rng = np.random.default_rng(61)
    st = Step(wf, rng, have, add, 16, spare=2)
    cache, scale = cache_of(rng, st, 2, 64, "float8_e4m3fn")
    scale = odd_scales(rng, scale)
    q = tensor(rng, (st.room, 4, 64), dtype, 1.5)
    got = attend(wf, st, cache, scale, q, new=new)
    least = scale.clone()
    least[1].clamp_(min=2.0 ** -64)
    check(st, cache, least, q, got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kv,bs,have,add", [(2, 16, [5, 16, 0, 31], [1, 3, 20, 1]), (3, 24, [1000, 23, 24], [1, 2, 60]), (1, 64, [10] * 100, [1] * 100)])
def test_writing_beside_scales_of_any_value(kv, bs, have, add, dtype):
    """Scales are the larger of what was and a power of two; elements, new ones and those that are scaled anew, are as near as any of their type to what
    they stand for, but for 2^-22 of a quotient or product in 32 bits; what need not change does not."""
    import layer_ref as ref
    wf = lib()
    rng = np.random.default_rng(62)
    st = Step(wf, rng, have, add, bs, spare=2)
    cache, scale = cache_of(rng, st, kv, 64, "float8_e4m3fn")
    scale = odd_scales(rng, scale) * 4
    k, v = (tensor(rng, (st.room, kv, 64), dtype, 2.0 ** rng.integers(-4, 6, (st.room, 1, 1))) for _ in range(2))
    was, want, want_scale = f64(cache), f64(cache), f64(scale)
    old_scale = want_scale.copy()
    wf.wf_kv_write(st.decode, st.kv, st.step, wf.KvLayer(cache[0], cache[1], scale[0], scale[1]), k, v)
    wf.wf_decode_status(st.decode)
    got, new_scale = f64(cache), f64(scale)
    for plane, x in enumerate((f64(k), f64(v))):
        ref.write8(want[plane], want_scale[plane], st.slot, bs, x)
        assert np.array_equal(new_scale[plane], want_scale[plane])
        with np.errstate(invalid="ignore"):  # blocks whose scale was 0 and stays so
            exact = was[plane] * (old_scale[plane] / new_scale[plane])[:, None, :, None]
        live = st.slot >= 0
        blocks = st.slot[live] // bs
        exact.reshape(-1, kv, 64)[st.slot[live]] = x[live] / new_scale[plane][blocks][:, :, None]
        changed = want[plane] != was[plane]
        near = np.abs(got[plane] - exact) <= np.abs(want[plane] - exact) + 2.0 ** -22 * np.abs(exact)
        assert np.where(changed, near, got[plane] == was[plane])[np.isfinite(exact)].all()


def test_turned_queries_in_other_memory_are_refused():
    """Into keys, values or the queries a head or a token further on; in place and beside them, as columns of one product, they go on."""
    import torch
    wf = lib()
    rng = np.random.default_rng(64)
    st = Step(wf, rng, [40, 3], [1, 30], 16)
    cache, _ = cache_of(rng, st, 2, 64, "float16")
    layer, rope = wf.KvLayer(cache[0], cache[1]), wf.Rope(64)
    whole = tensor(rng, (st.room + 1, 12, 64), "float16")
    q, k, v, free = whole[:-1, :4], whole[:-1, 4:6], whole[:-1, 6:8], whole[:-1, 8:]
    was = whole.clone()
    run = lambda out, q=q: wf.wf_kv_write(st.decode, st.kv, st.step, layer, k, v, q=q, q_out=out, rope=rope)
    for out in (whole[:-1, 1:5], whole[:-1, 3:7], whole[:-1, 5:9], whole[:-1, 7:11], whole[1:, :4], whole.view(-1, 4, 64)[:st.room]):
        with pytest.raises(wf.WfError, match="turned"):
            run(out)
    with pytest.raises(wf.WfError, match="turned"):
        run(whole[:-1, 4:5], q=whole[:-1, 8:9])  # one head, in the first key's place
    assert torch.equal(whole, was)
    apart = torch.empty_like(free)
    run(apart)
    run(free)
    run(None)
    assert torch.equal(free, apart) and torch.equal(q, apart) and torch.equal(whole[:-1, 4:8], was[:-1, 4:8])
