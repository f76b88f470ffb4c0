"""What a layer does with a step's tokens on a replica, over the range of sizes that it takes: what perf/operators.py is for the cache's bookkeeping.

  write    rotary positions of queries and keys, and the keys and values put into the paged cache's slots: in 16 bits, or in 8 with a scale for
           each block and head, where a block that is partly filled is scaled anew if a new token is too large for it
  attend   attention of the step's tokens over their rows' cached keys and values, causal, heads in groups: single tokens (decoding), whole
           prompts, chunks of prompts, and all of them in one step; over a cache in 16 bits or in 8

With `own` false, `run` computes them with elementary torch operations in 32 bits; with `own` true through the library's calls.  All inputs
are drawn from the seed on the GPU.  A step has room for `budget` tokens; the places behind the last one are padding, whose outputs stay as they were.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn


def listed():
    return [
        # One step of decoding for the activations of a tiny window: launches count.
        _write("write_tiny", rows=12, long=0, new=1, ctx=900, bs=16, heads=8, kv=2, dim=64, dtype="bf16", cache="16", rot=64),
        # A prompt batch of a large layer; positions scaled for a long context, keys already cached before.
        _write("write_prompt", rows=6, long=6, new=2800, ctx=9000, bs=16, heads=32, kv=8, dim=128, dtype="bf16", cache="16", rot=128, factor=8.0),
        # Chunked prefill beside decoding: interleaved pairs in a part of the head, odd block size, odd group of heads.
        _write("write_mixed", rows=169, long=12, new=500, ctx=3000, bs=24, heads=28, kv=4, dim=128, dtype="f16", cache="16", rot=48, inter=True),
        # A burst of rows decoding into an 8-bit cache: most blocks are partly filled.
        _write("write8_decode", rows=2000, long=0, new=1, ctx=150, bs=16, heads=32, kv=8, dim=128, dtype="bf16", cache="8", rot=128),
        # Prompts into an 8-bit cache with larger blocks; the first block of each continues a cached context.
        _write("write8_prompt", rows=7, long=7, new=1300, ctx=200, bs=64, heads=16, kv=8, dim=64, dtype="f16", cache="8", rot=64, inter=True),
        # Decoding of a few short rows: launches count.
        _attend("attend_tiny", rows=3, long=0, new=1, ctx=90, bs=16, heads=8, kv=2, dim=64, dtype="bf16", cache="16"),
        # One activation with a long context: the work is split over the positions.
        _attend("attend_one", rows=1, long=0, new=1, ctx=100_000, bs=32, heads=32, kv=8, dim=128, dtype="bf16", cache="16"),
        # A burst of 64 sessions decoding, ragged contexts around 9,000 tokens.
        _attend("attend_decode", rows=64, long=0, new=1, ctx=9000, bs=64, heads=32, kv=8, dim=128, dtype="bf16", cache="16"),
        # Whole prompts of different lengths, packed.
        _attend("attend_prompt", rows=3, long=3, new=4100, ctx=0, bs=16, heads=32, kv=8, dim=128, dtype="f16", cache="16"),
        # A mix window's step: chunks of eight prompts beside 161 rows that decode; odd block size, seven heads to a key.
        _attend("attend_mixed", rows=169, long=8, new=500, ctx=2000, bs=24, heads=28, kv=4, dim=128, dtype="bf16", cache="16"),
        # Decoding over an 8-bit cache, twice the rows for the same bytes.
        _attend("attend8_decode", rows=128, long=0, new=1, ctx=9000, bs=32, heads=32, kv=8, dim=128, dtype="bf16", cache="8"),
        # Chunks of prompts beside decoding over an 8-bit cache, narrow heads.
        _attend("attend8_mixed", rows=60, long=9, new=700, ctx=3500, bs=16, heads=24, kv=8, dim=64, dtype="f16", cache="8"),
    ]


def draw(rng):
    dim, kv = rng.choice((64, 128)), rng.choice((1, 2, 4, 8))
    heads = kv * rng.choice((1, 2, 3, 4, 5, 7, 8))
    common = dict(bs=rng.choice((8, 16, 16, 24, 32, 64, 100, 128)), heads=heads, kv=kv, dim=dim, dtype=rng.choice(("f16", "bf16", "bf16")),
                  cache=rng.choice(("16", "16", "8")))
    shape = rng.choice(("decode", "prompt", "mixed"))
    if rng.random() < 0.4:
        rows = _log(rng, 1, 2000) if shape == "decode" else _log(rng, 1, 160)
        long = 0 if shape == "decode" else rows if shape == "prompt" else max(1, rows // 10)
        new = _log(rng, 2, max(4, 12000 // long)) if long else 1
        return _write(None, rows=rows, long=long, new=new, ctx=_log(rng, 1, max(2, min(9000, 600_000 // rows))), rot=rng.choice((dim, dim, dim // 2, 48, 10)),
                      inter=rng.random() < 0.4, factor=rng.choice((1.0, 1.0, 4.0, 16.0)), **common)
    if shape == "decode":
        rows = _log(rng, 1, 512)
        return _attend(None, rows=rows, long=0, new=1, ctx=_log(rng, 1, min(60_000, 500_000 // rows)), **common)
    if shape == "prompt":
        rows = _log(rng, 1, 24)
        new = _log(rng, 2, 4000 / math.sqrt(rows))
        return _attend(None, rows=rows, long=rows, new=new, ctx=rng.choice((0, 0, _log(rng, 1, 3000 // rows + 2))), **common)
    rows, long = _log(rng, 4, 200), rng.randint(1, 4)
    return _attend(None, rows=rows, long=long, new=_log(rng, 2, 1500), ctx=_log(rng, 1, 3500), **common)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _case(name, kind, rows, long, new, ctx, bs, heads, kv, dim, dtype, cache, **more):
    """rows: `long` of them take about `new` tokens, the others one each, behind contexts of about `ctx` tokens."""
    c = dict(kind=kind, rows=rows, long=long, new=new, ctx=ctx, bs=bs, heads=heads, kv=kv, dim=dim, dtype=dtype, cache=cache, **more)
    return dict(c, name=name) if name else c


def _write(name, rot, inter=False, factor=1.0, **c):
    return _case(name, "write", rot=rot, inter=inter, factor=factor, **c)


def _attend(name, **c):
    return _case(name, "attend", **c)


def _around(mean):
    """The ends of the range that a ragged size of this mean is drawn from."""
    lo = max(1, mean // 2) if mean else 0
    return lo, 2 * mean - lo


def work(case):
    """Tokens and lengths at their means; of a product of two drawn sizes, the mean of the product."""
    rows, long, kv, dim = case["rows"], case["long"], case["kv"], case["dim"]
    tokens = long * case["new"] + rows - long
    size = 2 if case["cache"] == "16" else 1
    if case["kind"] == "write":
        scales = 0 if size == 2 else 8 * kv * (long * case["new"] / case["bs"] + rows)
        return {"bytes": tokens * dim * (4 * case["heads"] + kv * (4 + 2 * size)) + 16 * tokens + scales,
                "flops": 3 * tokens * case["rot"] * (case["heads"] + kv)}
    lo, hi = _around(case["new"])
    square = case["new"] ** 2 + ((hi - lo + 1) ** 2 - 1) / 12
    pairs = long * (case["new"] * case["ctx"] + (square + case["new"]) / 2) + (rows - long) * (case["ctx"] + 1)
    cached = long * (case["ctx"] + case["new"]) + (rows - long) * (case["ctx"] + 1)
    return {"bytes": cached * kv * dim * 2 * size + tokens * case["heads"] * dim * 4, "flops": 4 * dim * case["heads"] * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV)


def _inputs(case, seed):
    """The rows' tables and lengths, the step's tokens, the layer's cache and the tensors of the step."""
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    rows, long, bs, kv, dim, dtype = case["rows"], case["long"], case["bs"], case["kv"], case["dim"], TYPES[case["dtype"]]
    have = _ints(g, *_around(case["ctx"]), rows)
    add = torch.ones(rows, dtype=torch.int64, device=DEV)
    where = torch.randperm(rows, generator=g, device=DEV)[:long]  # rows of both kinds lie among each other
    add[where] = _ints(g, *_around(case["new"]), long)
    length = have + add
    budget = long * _around(case["new"])[1] + rows - long
    most = _around(case["ctx"])[1] + (_around(case["new"])[1] if long else 1)
    width = -(-most // bs)
    held = (length + bs - 1) // bs
    used = rows * width
    n_blocks = used + 3
    table = torch.randperm(n_blocks, generator=g, device=DEV)[:used].reshape(rows, width).int()
    table = torch.where(torch.arange(width, device=DEV) < held[:, None], table, -1)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), add.cumsum(0)])
    t = torch.arange(budget, device=DEV)
    live = t < start[-1]
    row = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp_(max=rows - 1)
    pos = have[row] + t - start[row]
    slot = table.long()[row, (pos // bs).clamp_(max=width - 1)] * bs + pos % bs
    s = dict(kind=case["kind"], bs=bs, long=where, n_long=long, most=most, new=_around(case["new"])[1], group=case["heads"] // kv,
             table=table, have=have, add=add, start=start.int(), len=length.int(), slot=torch.where(live, slot, -1),
             pos=torch.where(live, pos, 0).int(), row=torch.where(live, row, -1).int())
    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dtype)
    s["q"] = normal(budget, case["heads"], dim)
    if case["cache"] == "16":
        s["cache"], s["scale"] = normal(2, n_blocks, bs, kv, dim), None
    else:
        s["cache"] = normal(2, n_blocks, bs, kv, dim).mul_(90).clamp_(-448, 448).to(F8)
        s["scale"] = torch.exp2(torch.randint(-9, -5, (2, n_blocks, kv), generator=g, device=DEV).float())
    if case["kind"] == "attend":
        s["q"].mul_(1.5)
        s["out"] = torch.zeros_like(s["q"])
        return s
    # Keys have some channels that are far larger than others; a token in eight is larger than those before it.
    loud = torch.where(torch.rand((kv, dim), generator=g, device=DEV) < 0.05, 6.0, 1.0) * torch.where(torch.rand((budget, 1, 1), generator=g, device=DEV) < 0.12, 3.0, 1.0)
    s["k"], s["v"] = (normal(budget, kv, dim).float() * loud).to(dtype), normal(budget, kv, dim)
    s["rot"], s["inter"], s["factor"] = case["rot"], case["inter"], case["factor"]
    s["magnitude"] = 1.0 if case["factor"] == 1 else 0.1 * math.log(case["factor"]) + 1
    s["freq"] = _frequencies(case["rot"], case["factor"])
    s["q_out"] = torch.zeros_like(s["q"])
    return s


BASE, CONTEXT, SLOW, FAST = 10000.0, 4096, 1.0, 32.0


def _frequencies(rot, factor):
    """Radians a position, by pair: those that turn fewer than SLOW times in the context of the training are divided by the factor, those that turn
    more than FAST times stay, and between them it goes over linearly."""
    f = BASE ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    keep = ((CONTEXT * f / (2 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0, 1)
    return f * (keep + (1 - keep) / factor)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the handles and the views of these tensors that a user's program makes once
        from paper_2609_03335_gb300 import wf
        rows, n_blocks = s["table"].shape[0], s["cache"].shape[1]
        ring, ends = torch.zeros(n_blocks, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV)
        s["kv"] = wf.Kv(s["table"], s["len"], ring, ends, s["bs"])
        s["step"] = wf.KvStep(rows, s["slot"].numel(), s["kv"])
        for name in ("slot", "pos", "row", "start"):
            getattr(s["step"], name).copy_(s[name])
        s["layer"] = wf.KvLayer(s["cache"][0], s["cache"][1], *(() if s["scale"] is None else (s["scale"][0], s["scale"][1])))
        if s["kind"] == "write":
            s["decode"] = wf.Decode(max_rows=rows)
            s["rope"] = wf.Rope(s["rot"], base=BASE, interleaved=s["inter"], factor=s["factor"], context=CONTEXT, slow=SLOW, fast=FAST,
                                magnitude=s["magnitude"])
        else:
            s["attn"] = wf.Attn(max_rows=rows, heads=case["heads"], dim=case["dim"])
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain_write(s) if s["kind"] == "write" else _plain_attend(s)
    from paper_2609_03335_gb300 import wf
    if s["kind"] == "write":
        wf.wf_kv_write(s["decode"], s["kv"], s["step"], s["layer"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
        return dict(q=s["q_out"], cache=s["cache"], scale=s["scale"])
    # A step whose rows take one token each says so.
    wf.wf_attend(s["attn"], s["kv"], s["step"], s["layer"], s["q"], s["out"], new=s["new"] if s["n_long"] else 1)
    return s["out"]


def _rotated(x, s):
    """x, in 32 bits, with its first `rot` elements turned by their positions."""
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = (angle.cos() * s["magnitude"]).float()[:, None], (angle.sin() * s["magnitude"]).float()[:, None]
    x, half = x.float(), s["rot"] // 2
    part, rest = x[..., :s["rot"]], x[..., s["rot"]:]
    a, b = (part[..., 0::2], part[..., 1::2]) if s["inter"] else (part[..., :half], part[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack([a, b], -1).flatten(-2) if s["inter"] else torch.cat([a, b], -1)
    return torch.cat([part, rest], -1)


def _plain_write(s):
    live = s["slot"] >= 0
    dtype = s["q"].dtype
    q = torch.where(live[:, None, None], _rotated(s["q"], s).to(dtype), 0)
    k = _rotated(s["k"], s).to(dtype)
    if s["scale"] is None:
        return dict(q=q, cache=torch.stack([_put(s["cache"][0], s["slot"], k), _put(s["cache"][1], s["slot"], s["v"])]), scale=None)
    k, v = _plain_write8(s, 0, k.float()), _plain_write8(s, 1, s["v"].float())
    return dict(q=q, cache=torch.stack([k[0], v[0]]), scale=torch.stack([k[1], v[1]]))


def _put(cache, slot, x):
    """The cache with x in its slots; a slot of -1 is none."""
    flat = torch.cat([cache.flatten(0, 1), cache.new_empty((1,) + cache.shape[2:])])
    flat[torch.where(slot < 0, flat.shape[0] - 1, slot)] = x
    return flat[:-1].view_as(cache)


def _plain_write8(s, plane, x):
    cache, scale, bs = s["cache"][plane], s["scale"][plane], s["bs"]
    n, kv = scale.shape
    block = torch.where(s["slot"] < 0, n, s["slot"] // bs)
    amax = torch.zeros((n + 1, kv), device=DEV).scatter_reduce(0, block[:, None].expand(-1, kv), x.abs().amax(-1), "amax")[:n]
    # The least power of two whose 448-fold reaches amax: amax = m 2^e with m in [0.5, 1), 448 = 0.875 * 2^9.
    m, e = torch.frexp(amax)
    e = torch.where(amax == 0, -64, (e - 9 + (m > 0.875).int()).clamp(-64, 63))
    need = torch.ldexp(torch.ones_like(amax), e)
    # A row's first block may hold tokens already.
    part = s["have"] % bs
    first = torch.where(part > 0, s["table"].gather(1, (s["have"] // bs)[:, None].clamp(max=s["table"].shape[1] - 1))[:, 0].long(), n)
    written = torch.zeros(n + 1, dtype=torch.bool, device=DEV).index_fill_(0, block, True)[:n]
    kept = torch.zeros(n + 1, dtype=torch.bool, device=DEV).index_fill_(0, first, True)[:n]
    new = torch.where(written[:, None], torch.where(kept[:, None], torch.maximum(scale, need), need), scale)
    at = first.clamp(max=n - 1)
    was = cache.view(torch.uint8)[at].view(F8).float()
    old = (was * (scale[at] / new[at])[:, None, :, None]).clamp(-448, 448).to(F8)
    before = torch.arange(bs, device=DEV) < part[:, None]
    old = torch.where(before[:, :, None, None], old.float(), was).to(F8)
    blocks = torch.cat([cache, cache[:1]]).view(torch.uint8).index_copy_(0, torch.where(first == n, n, at), old.view(torch.uint8))[:n]
    value = x / torch.cat([new, new[:1]])[block][:, :, None]
    return _put(blocks, s["slot"], value.clamp(-448, 448).to(F8).view(torch.uint8)).view(F8), new


def _plain_attend(s):
    rows = s["table"].shape[0]
    out = torch.zeros((s["q"].shape[0] + 1,) + s["q"].shape[1:], dtype=s["q"].dtype, device=DEV)
    short = torch.ones(rows, dtype=torch.bool, device=DEV).index_fill_(0, s["long"], False)
    order = short.int().argsort(stable=True)
    if s["n_long"]:
        _plain_rows(s, out, order[:s["n_long"]], s["new"])
    if rows > s["n_long"]:
        _plain_rows(s, out, order[s["n_long"]:], 1)
    return out[:-1]


def _plain_rows(s, out, rows, most):
    """Rows with at most this many new tokens each, padded to it."""
    bs, g, budget = s["bs"], s["group"], s["q"].shape[0]
    length, add, start = s["len"].long()[rows], s["add"][rows], s["start"].long()[rows]
    p = torch.arange(s["most"], device=DEV)
    there = p < length[:, None]
    slot = torch.where(there, s["table"].long()[rows][:, (p // bs)] * bs + p % bs, 0)
    k, v = (_held(s, plane, slot) for plane in (0, 1))  # [rows, kv, positions, dim]
    n = torch.arange(most, device=DEV)
    token = torch.where(n < add[:, None], start[:, None] + n, budget)
    heads, dim = s["q"].shape[1:]
    q = s["q"][token.clamp(max=budget - 1)].float().reshape(len(rows), most, heads // g, g, dim).permute(0, 2, 3, 1, 4).reshape(len(rows), heads // g, g * most, dim)
    x = (q @ k.transpose(-1, -2)).mul_(dim ** -0.5).view(len(rows), heads // g, g, most, -1)
    last = (length - add)[:, None] + n
    x.masked_fill_((p > last[:, :, None])[:, None, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(len(rows), heads // g, g * most, -1) @ v).view(len(rows), heads // g, g, most, dim) / total
    out[token] = o.permute(0, 3, 1, 2, 4).reshape(len(rows), most, heads, dim).to(out.dtype)


def _held(s, plane, slot):
    """The values at these slots [rows, positions], in 32 bits, by head; 0 where a position is past its row."""
    x = s["cache"][plane].flatten(0, 1)[slot].float()
    if s["scale"] is not None:
        x *= s["scale"][plane][slot // s["bs"]][..., None]
    return x.transpose(1, 2)


# ---------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_write(case, s) if case["kind"] == "write" else _exact_attend(case, s)


def _exact_attend(case, s):
    if work(case)["flops"] > 2e12:
        return None
    bs, g, out = s["bs"], s["group"], torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    start, length = s["start"].tolist(), s["len"].tolist()
    for r in range(case["rows"]):
        a, b, n = start[r], start[r + 1], length[r]
        blocks = s["table"][r, :-(-n // bs)].long()
        k, v = s["cache"][0][blocks].double(), s["cache"][1][blocks].double()
        if s["scale"] is not None:
            k, v = k * s["scale"][0][blocks].double()[:, None, :, None], v * s["scale"][1][blocks].double()[:, None, :, None]
        k, v = k.reshape(-1, case["kv"], case["dim"])[:n], v.reshape(-1, case["kv"], case["dim"])[:n]
        later = torch.arange(n, device=DEV) > torch.arange(n - (b - a), n, device=DEV)[:, None]
        for h in range(case["heads"]):
            x = s["q"][a:b, h].double() @ k[:, h // g].T / math.sqrt(case["dim"])
            out[a:b, h] = torch.softmax(x.masked_fill_(later, -math.inf), 1) @ v[:, h // g]
    return out


def _exact_write(case, s):
    turn = torch.polar(torch.full_like(s["freq"], s["magnitude"]).expand(s["pos"].shape[0], -1), s["pos"].double()[:, None] * s["freq"])[:, None]

    def rotated(x):
        y = x.double()
        part = y[..., :s["rot"]]
        pair = part.reshape(*part.shape[:-1], -1, 2) if s["inter"] else part.reshape(*part.shape[:-1], 2, -1).transpose(-1, -2)
        pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        y[..., :s["rot"]] = (pair if s["inter"] else pair.transpose(-1, -2)).reshape(part.shape)
        return y
    live = s["slot"] >= 0
    slots, bs = s["slot"][live], s["bs"]
    q = rotated(s["q"])
    q[~live] = 0
    k, v = rotated(s["k"])[live], s["v"].double()[live]
    cache = s["cache"].double()
    if s["scale"] is None:
        for plane, x in enumerate((k, v)):
            cache[plane].flatten(0, 1)[slots] = x
        return dict(q=q, cache=cache)
    scale = s["scale"].double()
    blocks = torch.unique(slots // bs)
    first = torch.full((cache.shape[1],), bs, dtype=torch.int64, device=DEV).scatter_reduce(0, slots // bs, slots % bs, "amin")[blocks]
    for plane, x in enumerate((k.to(s["q"].dtype).double(), v)):
        most = torch.zeros(scale[plane].shape, dtype=torch.float64, device=DEV).index_reduce_(0, slots // bs, x.abs().amax(-1), "amax")[blocks]
        need = torch.full_like(most, 2.0 ** -64)
        for e in range(-64, 63):
            need = torch.where(most > 448 * 2.0 ** e, 2.0 ** (e + 1), need)
        was = scale[plane][blocks]
        now = torch.where((first > 0)[:, None], torch.maximum(was, need), need)
        scale[plane][blocks] = now
        old = _eight(cache[plane][blocks] * (was / now)[:, None, :, None])
        keep = torch.arange(bs, device=DEV) >= first[:, None]
        cache[plane][blocks] = torch.where(keep[:, :, None, None], cache[plane][blocks], old)
        cache[plane].flatten(0, 1)[slots] = _eight(x / scale[plane][slots // bs][:, :, None])
    return dict(q=q, cache=cache, scale=scale)


def _eight(x):
    """The nearest numbers with 4 bits from 2^-6 on (2^-9 apart below), up to 448; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)
