"""The calls that run admitted activations on a replica, over the range of sizes that they take: what perf/cases.py is for plans.

  extend    block tables and slot maps of a step's tokens, built on the GPU from the rows' lengths
  select    beam search's selection over beams and vocabulary
  reorder   the rows of a paged cache put in the order that a selection chose, shared last blocks copied, unused ones freed

With `own` false, `run` computes them with elementary torch operations; with `own` true through the library's calls.  All inputs are
drawn from the seed on the GPU.  `extend` and `reorder` give whole numbers (and copies); `select`'s sums are in 32 bits, and its inputs are such
that no two candidates' sums lie within their rounding, so that the tokens chosen have one right answer.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # One step of decoding for the activations of a tiny window: launches count.
        _extend("extend_tiny", 12, 16, ctx=900, new=1, budget=16),
        # The same for every activation of a burst window at once, long contexts in large blocks.
        _extend("extend_decode", 2000, 64, ctx=9000, new=1, budget=2048),
        # Chunked prefill beside decoding, odd block size; the token budget ends the line.
        _extend("extend_mixed", 169, 24, ctx=3000, new=128, budget=8192),
        # A burst window admitted whole: contexts of 2,048 to 32,768 tokens (256 to 4,096 MiB of cache at 128 KiB a token).
        _extend("extend_bulk", 2000, 16, ctx=0, new=17408, budget=35_000_000),
        # One activation that searches with four beams.
        _select("select_one", 1, 4, 32000, 8, "bf16"),
        # A mix window's sessions; an odd vocabulary, so rows start anywhere.
        _select("select_mix", 16, 4, 50257, 8, "f16"),
        # A burst of 64 sessions with eight beams each.
        _select("select_burst", 64, 8, 131072, 16, "bf16"),
        # Constrained decoding in 32 bits: most tokens masked, by -inf in some rows and the type's lowest value in others; dead beams.
        _select("select_masked", 40, 16, 65537, 32, "f32", mask=0.995, dead=0.1),
        # The four beams of one activation.
        _reorder("reorder_one", 1, 4, 16, blocks=40, planes=4, token_bytes=512),
        # A mix window's sessions, wide beams.
        _reorder("reorder_mix", 16, 12, 16, blocks=130, planes=8, token_bytes=1024),
        # A burst of 64 sessions, eight beams, contexts up to 16,384 tokens: tables count.
        _reorder("reorder_long", 64, 8, 16, blocks=1024, planes=0, token_bytes=0),
        # The same sessions with larger blocks and the cache of several layers: copies count.
        _reorder("reorder_copy", 64, 8, 64, blocks=9, planes=8, token_bytes=2048),
    ]


def draw(rng):
    kind = rng.choice(("extend", "select", "reorder"))
    if kind == "extend":
        rows, bs = _log(rng, 1, 8192), rng.choice((8, 16, 24, 32, 64, 128))
        if rng.random() < 0.4:
            return _extend(None, rows, bs, ctx=_log(rng, 16, 16000), new=1, budget=rows + rng.randint(0, 64))
        new = _log(rng, 4, max(8, min(20000, 16_000_000 // rows)))
        return _extend(None, rows, bs, ctx=_log(rng, 16, 16000), new=new, budget=max(16, int(rows * new * rng.uniform(0.5, 1.2))),
                       pool=rng.choice((1.0, 1.0, 0.7)))
    if kind == "select":
        groups, beams, dtype = _log(rng, 1, 64), rng.choice((1, 2, 4, 5, 8, 12, 16)), rng.choice(("f32", "f16", "bf16", "bf16"))
        vocab = _log(rng, 1000, max(2000, min(200_000, (1 << 26) // (groups * beams))))
        return _select(None, groups, beams, vocab, min(32, rng.choice((beams, 2 * beams, 2 * beams))), dtype,
                       mask=rng.choice((0.0, 0.0, 0.9)), dead=rng.choice((0.0, 0.0, 0.2)), first=rng.random() < 0.15)
    groups, beams, bs = _log(rng, 1, 64), rng.choice((1, 2, 3, 4, 6, 8, 12)), rng.choice((8, 16, 32, 64))
    blocks = _log(rng, 4, 600)
    tables_only = rng.random() < 0.4 or groups * beams * blocks > 12000
    return _reorder(None, groups, beams, bs, blocks=blocks, planes=0 if tables_only else rng.choice((2, 5, 8)),
                    token_bytes=0 if tables_only else rng.choice((256, 640, 1024)))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _named(name, c):
    return dict(c, name=name) if name else c


def _extend(name, rows, bs, ctx, new, budget, pool=1.0):
    """pool: the free blocks, as a share of those that all rows ask for."""
    return _named(name, dict(kind="extend", rows=rows, bs=bs, ctx=ctx, new=new, budget=budget, pool=pool))


def _select(name, groups, beams, vocab, keep, dtype, mask=0.0, dead=0.0, first=False):
    return _named(name, dict(kind="select", groups=groups, beams=beams, vocab=vocab, keep=keep, dtype=dtype, mask=mask, dead=dead, first=first))


def _reorder(name, groups, beams, bs, blocks, planes, token_bytes):
    return _named(name, dict(kind="reorder", groups=groups, beams=beams, bs=bs, blocks=blocks, planes=planes, token_bytes=token_bytes))


def work(case):
    if case["kind"] == "extend":
        rows, tokens = case["rows"], min(case["budget"], case["rows"] * case["new"] * case["pool"])
        taken = tokens / case["bs"]
        return {"bytes": 8 * rows + 16 + 16 * case["budget"] + 8 * taken + 12 * rows + 4 + 16, "flops": 0}
    if case["kind"] == "select":
        rows = case["groups"] * case["beams"]
        live = case["groups"] if case["first"] else rows * (1 - case["dead"])
        cells = live * case["vocab"]
        return {"bytes": cells * BYTES[case["dtype"]] + 4 * rows + 12 * (case["groups"] * case["keep"] + rows), "flops": 5 * cells}
    rows = case["groups"] * case["beams"]
    held = rows * case["blocks"] * 0.75  # contexts are between half and all of the table's width
    copied = case["groups"] * (case["beams"] - _parents(case["beams"])) * case["bs"] / 2 * case["planes"] * case["token_bytes"]
    return {"bytes": 8 * held + 2 * copied + 28 * rows, "flops": 0}


def _parents(beams):
    """Distinct parents of a group's new rows: beams continue about two in three of the old ones."""
    return max(1, (2 * beams + 2) // 3)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"extend": _prepare_extend, "select": _prepare_select, "reorder": _prepare_reorder}[case["kind"]](case, g)
    s["kind"] = case["kind"]
    if own:  # the handle and the views of these tensors that a user's program makes once
        from paper_2609_03335_gb300 import wf
        if case["kind"] == "select":
            s["decode"] = wf.Decode(max_rows=case["groups"] * case["beams"], max_vocab=case["vocab"], max_keep=case["keep"])
            s["out"] = wf.BeamOut(case["groups"], case["beams"], case["keep"])
        else:
            s["decode"] = wf.Decode(max_rows=s["table"].shape[0], max_row_blocks=s["table"].shape[1])
            s["kv"] = wf.Kv(s["table"], s["len"], s["ring"], s["ends"], case["bs"])
            if case["kind"] == "extend":
                s["out"] = wf.KvStep(case["rows"], case["budget"])
            else:
                s["to"] = wf.Kv(s["to_table"], torch.empty_like(s["len"]), s["ring"], torch.empty_like(s["ends"]), case["bs"])
                s["out"] = wf.KvMoves(s["table"].shape[0])
    return s


def _ints(g, lo, hi, n):
    return torch.randint(lo, hi + 1, (n,), generator=g, device=DEV)


def _pool(g, used, free, n):
    """Block ids of `used` cells of a pool of n blocks, and a ring that starts anywhere with `free` others."""
    ids = torch.randperm(n, generator=g, device=DEV).int()
    head = int(_ints(g, 0, n - 1, 1)) + 3 * n
    ring = torch.full((n,), -7, dtype=torch.int32, device=DEV)
    ring[(head + torch.arange(free, device=DEV)) % n] = ids[used:used + free]
    return ids[:used], ring, torch.tensor([head, head + free], dtype=torch.int64, device=DEV)


def _prepare_extend(case, g):
    rows, bs, ctx, new = case["rows"], case["bs"], case["ctx"], case["new"]
    length = _ints(g, ctx // 4, 2 * ctx - ctx // 4, rows) if ctx else torch.zeros(rows, dtype=torch.int64, device=DEV)
    if new == 1:
        add = torch.ones(rows, dtype=torch.int64, device=DEV)
    else:
        add = _ints(g, max(1, new // 8), 2 * new - max(1, new // 8), rows)
        add = torch.where(_ints(g, 0, 7, rows) == 0, torch.ones_like(add), add) if ctx else add  # some rows decode
    add = torch.where(_ints(g, 0, 63, rows) == 0, torch.zeros_like(add), add)  # some have nothing to do
    width = -(-(2 * ctx + 2 * new) // bs) + 1
    add = torch.where(_ints(g, 0, 299, rows) == 0, torch.full_like(add, width * bs + 1), add)  # some ask for more than a row holds
    have = (length + bs - 1) // bs
    need = ((length + add + bs - 1) // bs - have)[add <= width * bs]
    used = int(have.sum())
    free = int(case["pool"] * int(need.sum())) + 1
    ids, ring, ends = _pool(g, used, free, used + free + 5)
    table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV) < have[:, None]] = ids
    return dict(bs=bs, budget=case["budget"], table=table, len=length.int(), add=add.int(), ring=ring, ends=ends)


def _prepare_select(case, g):
    groups, beams, vocab, dtype = case["groups"], case["beams"], case["vocab"], TYPES[case["dtype"]]
    rows = groups * beams
    # Logits: a broad bell and, in each row, a few likely tokens, on a grid of 2^-5 (2^-8 in 32 bits).
    grid = 2.0 ** -8 if case["dtype"] == "f32" else 2.0 ** -5
    x = torch.randn((rows, vocab), generator=g, device=DEV).mul_(1.8)
    at = torch.randint(0, vocab, (rows, 24), generator=g, device=DEV)
    x.scatter_(1, at, 6 + 6 * torch.rand((rows, 24), generator=g, device=DEV))
    x = x.div_(grid).round_().mul_(grid)
    if case["mask"]:
        low = torch.where(torch.arange(rows, device=DEV) % 2 == 0, -math.inf, torch.finfo(dtype).min)
        keep = torch.rand((rows, vocab), generator=g, device=DEV) >= case["mask"]
        keep[:, :64] = True
        x = torch.where(keep, x, low[:, None])
        del keep
    x = x.to(dtype)
    # Scores: what a beam's sums start from lies on another offset of the grid for each beam of a group, so that sums of different beams
    # are at least grid / (beams + 1) apart.
    lse = torch.logsumexp(x.float(), 1).double()
    start = torch.rand((groups, beams), generator=g, device=DEV, dtype=torch.float64) * -6 - 4
    start = (start / grid).round() * grid + grid * torch.arange(beams, device=DEV) / (beams + 1)
    score = (start.reshape(-1) + lse).float()
    first = torch.arange(beams, device=DEV).repeat(groups) > 0
    dead = first if case["first"] else (torch.rand(rows, generator=g, device=DEV) < case["dead"]) & first
    score = torch.where(dead, torch.full_like(score, -math.inf), score)
    return dict(logits=x, score=score, groups=groups, beams=beams, keep=case["keep"], eos=int(at[0, 0]))


def _prepare_reorder(case, g):
    groups, beams, bs, blocks = case["groups"], case["beams"], case["bs"], case["blocks"]
    length = _ints(g, blocks * bs // 2, blocks * bs, groups)[:, None].expand(groups, beams)
    have = (length + bs - 1) // bs
    # A prompt that all beams share, then a stretch that pairs share, then blocks of a beam's own.
    col, k = torch.arange(blocks, device=DEV), torch.arange(beams, device=DEV)
    part = torch.rand((groups, 1, 1), generator=g, device=DEV) * 0.2 + 0.75
    owner = torch.where(col < part * have[:, :1, None] - 1, 0, torch.where(col < have[:, :1, None] - 2, k[:, None] // 2 * 2, k[:, None].expand(beams, blocks)))
    mine = (owner == k[:, None]) & (col < have[:, :, None])
    used = int(mine.sum())
    free = groups * beams + 3
    ids, ring, ends = _pool(g, used, free, groups * (blocks + -(-beams // 2) * (blocks // 4 + 2) + 2 * beams) + free)
    own_id = torch.full((groups, beams, blocks), -1, dtype=torch.int32, device=DEV)
    own_id[mine] = ids
    table = own_id.gather(1, owner.expand(groups, beams, blocks)).reshape(groups * beams, blocks).contiguous()
    # Parents: two in three beams go on; some groups have ended.
    alive = torch.rand((groups, beams), generator=g, device=DEV).argsort(1)[:, :_parents(beams)]
    pick = torch.cat([torch.arange(alive.shape[1], device=DEV).expand(groups, -1),
                      torch.randint(0, alive.shape[1], (groups, beams - alive.shape[1]), generator=g, device=DEV)], 1)
    pick = pick.gather(1, torch.rand((groups, beams), generator=g, device=DEV).argsort(1))
    parent = alive.gather(1, pick) + torch.arange(groups, device=DEV)[:, None] * beams
    ended = (torch.rand(groups, generator=g, device=DEV) < 0.05) & (torch.arange(groups, device=DEV) > 0)
    parent = torch.where(ended[:, None], torch.full_like(parent, -1), parent)
    s = dict(bs=bs, beams=beams, table=table, len=length.reshape(-1).int().contiguous(), ring=ring, ends=ends, parent=parent.reshape(-1).int(),
             to_table=torch.full_like(table, -1), cache=None)
    if case["planes"]:
        s["cache"] = torch.randn((case["planes"], ring.numel(), bs, case["token_bytes"] // 2), generator=g, device=DEV, dtype=torch.bfloat16)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(s):
    if not own:
        return {"extend": _plain_extend, "select": _plain_select, "reorder": _plain_reorder}[s["kind"]](s)
    from paper_2609_03335_gb300 import wf
    out = s["out"]
    if s["kind"] == "extend":
        wf.wf_kv_extend(s["decode"], s["kv"], s["add"], out)
        return dict(table=s["table"], slot=out.slot, pos=out.pos, row=out.row, start=out.start, len=out.len, ends=out.ends, status=out.status)
    if s["kind"] == "select":
        wf.wf_beam_select(s["decode"], s["logits"], s["score"], out, eos=s["eos"])
        return dict(score=out.score, parent=out.parent, token=out.token, next_score=out.next_score, next_parent=out.next_parent,
                    next_token=out.next_token)
    to = s["to"]
    wf.wf_kv_reorder(s["decode"], s["kv"], s["beams"], s["parent"], to, out, cache=s["cache"])
    got = dict(table=to.table, len=to.len, ring=to.ring, ends=to.ends, copies=out.copies, status=out.status)
    return got if s["cache"] is None else dict(got, cache=s["cache"])


def _blocks(x, bs):
    return (x + bs - 1) // bs


def _plain_extend(s):
    bs, budget, table, ring = s["bs"], s["budget"], s["table"], s["ring"]
    length, add = s["len"].long(), s["add"].long()
    head, tail = s["ends"][0], s["ends"][1]
    rows, width = table.shape
    have, then = _blocks(length, bs), _blocks(length + add, bs)
    ok = (length >= 0) & (add >= 0) & (then <= width)
    need, new = torch.where(ok, then - have, 0), torch.where(ok, add, 0)
    fits_blocks, fits_tokens = need.cumsum(0) <= tail - head, new.cumsum(0) <= budget
    admitted = ok & fits_blocks & fits_tokens
    status = (~ok).int() + (ok & ~fits_blocks).int() * 2 + (ok & ~fits_tokens).int() * 4
    new, need = torch.where(admitted, new, 0), torch.where(admitted, need, 0)
    end = new.cumsum(0)
    start, taken = end - new, need.cumsum(0)
    t = torch.arange(budget, device=table.device)
    live = t < end[-1]
    row = torch.searchsorted(end, t, right=True).clamp_(max=rows - 1)
    pos = length[row] + t - start[row]
    blk = pos // bs
    fresh = ring[(head + (taken - need)[row] + blk - have[row]).remainder(ring.numel())]
    block = torch.where(blk < have[row], table[row, blk.clamp(0, width - 1)], fresh).long()
    slot = torch.where(live, block * bs + pos % bs, -1)
    opens = live & (pos % bs == 0)  # a block's first token: the table gets its id
    flat = torch.cat([table.reshape(-1), table.new_empty(1)])
    flat[torch.where(opens, row * width + blk, rows * width)] = fresh
    return dict(table=flat[:-1].reshape(rows, width), slot=slot, pos=torch.where(live, pos, 0).int(), row=torch.where(live, row, -1).int(),
                start=torch.cat([start, end[-1:]]).int(), len=(length + new).int(), ends=torch.stack([head + taken[-1], tail]), status=status)


def _order(x):
    """Whole numbers in the order of the 32-bit floats."""
    b = (x + 0.0).view(torch.int32).long()
    return torch.where(b < 0, -(b & 0x7FFFFFFF), b)


def _best(key, n):
    """The n largest of distinct 64-bit keys in each row, largest first; rows that hold fewer are padded."""
    top = key.topk(min(n, key.shape[1]), 1).indices
    return torch.nn.functional.pad(top, (0, n - top.shape[1]), value=-1)


def _plain_select(s):
    groups, beams, n, eos = s["groups"], s["beams"], s["keep"], s["eos"]
    x = s["logits"].float()
    x = torch.where(x.isnan(), -math.inf, x)
    vocab = x.shape[1]
    m = x.amax(1, keepdim=True)
    d = torch.where(x == m, 0.0, x - m)
    logp = d - d.exp().sum(1, keepdim=True).log()
    c = s["score"][:, None] + logp
    c = torch.where((x > -math.inf) & (c > -math.inf), c, -math.inf)  # NaN drops out too
    # A row's best by logit, then the group's best by sum: equal sums go to the lower beam, then the larger logit, then the lower token.
    token = _best(_order(x) * vocab + torch.arange(vocab - 1, -1, -1, device=x.device), n)
    c = torch.where(token < 0, -math.inf, c.gather(1, token.clamp(min=0))).reshape(groups, beams * n)
    at = _best(_order(c) * (beams * n) + torch.arange(beams * n - 1, -1, -1, device=x.device), n)
    score, token = c.gather(1, at), token.reshape(groups, beams * n).gather(1, at).int()
    parent = (at // n + torch.arange(groups, device=x.device)[:, None] * beams).int()
    none = score == -math.inf
    parent, token = torch.where(none, -1, parent), torch.where(none, -1, token)
    # The first `beams` that do not end.
    goes = ~none & (token != eos)
    place = torch.where(goes, goes.cumsum(1) - 1, beams).clamp(max=beams)

    def put(v, fill):
        return torch.full((groups, beams + 1), fill, dtype=v.dtype, device=v.device).scatter(1, place, v)[:, :beams].contiguous()
    return dict(score=score, parent=parent, token=token, next_score=put(score, -math.inf), next_parent=put(parent, -1), next_token=put(token, -1))


def _plain_reorder(s):
    bs, beams, ring, old = s["bs"], s["beams"], s["ring"], s["table"]
    rows, width = old.shape
    groups, size = rows // beams, ring.numel()
    dev = old.device
    length, parent = s["len"].long(), s["parent"].long()
    first = torch.arange(rows, device=dev) // beams * beams
    ok = (parent >= first) & (parent < first + beams)
    status = ((parent != -1) & ~ok).int()
    src = torch.where(ok, parent, 0)
    new_len = torch.where(ok, length[src], 0)
    have, new_have = _blocks(length, bs), _blocks(new_len, bs)
    col = torch.arange(width, device=dev)
    table = torch.where(col < new_have[:, None], old[src], s["to_table"])
    # Freed: held by an old row, by no row that goes on and by no lower old row.
    cells, valid = old.reshape(groups, beams, width), (col < have[:, None]).reshape(groups, beams, width)
    goes = torch.zeros(rows + 1, dtype=torch.bool, device=dev).index_fill_(0, torch.where(ok, parent, rows), True)[:rows].reshape(groups, beams)
    lower = torch.ones((beams, beams), dtype=torch.bool, device=dev).tril(-1)
    same = (cells[:, :, None] == cells[:, None]) & valid[:, None] & (goes[:, None, :, None] | lower[None, :, :, None])
    freed = (valid & ~same.any(2)).transpose(1, 2).reshape(groups, width * beams)  # by position, then row
    # Last blocks that are written next and that a lower row holds too.
    last = torch.where(new_len % bs > 0, table.gather(1, (new_have - 1).clamp(min=0)[:, None])[:, 0].long(), -1).reshape(groups, beams)
    shared = ((last[:, :, None] == last[:, None]) & lower).any(2) & (last >= 0)
    n_freed, n_copy = freed.sum(1), shared.sum(1)
    keep, take = torch.minimum(n_freed, n_copy), (n_copy - n_freed).clamp(min=0)
    give = n_freed - keep
    rank = freed.cumsum(1) - 1
    ids = cells.transpose(1, 2).reshape(groups, width * beams)
    mine = torch.zeros((groups, width * beams + 1), dtype=torch.int32, device=dev).scatter(1, torch.where(freed, rank, width * beams), ids)
    i = shared.cumsum(1) - 1
    from_ring = (take.cumsum(0) - take)[:, None] + i - keep[:, None]
    short = shared & (i >= keep[:, None]) & (from_ring >= s["ends"][1] - s["ends"][0])
    to = torch.where(i < keep[:, None], mine.gather(1, i.clamp(min=0)), ring[(s["ends"][0] + from_ring).remainder(size)])
    copied = (shared & ~short).reshape(-1)
    short, to = short.reshape(-1), to.reshape(-1)
    copies = torch.where(copied[:, None], torch.stack([last.reshape(-1).int(), to], 1), -1)
    tail_at = (new_have - 1).clamp(min=0)[:, None]
    value = torch.where(copied[:, None], to[:, None], torch.where(short[:, None], s["to_table"].gather(1, tail_at), table.gather(1, tail_at)))
    table = table.scatter(1, tail_at, value)
    out_len = torch.where(short, new_len // bs * bs, new_len).int()
    status = status + short.int() * 2
    push = torch.where(freed & (rank >= keep[:, None]), (s["ends"][1] + (give.cumsum(0) - give)[:, None] + rank - keep[:, None]).remainder(size), size)
    ring = torch.cat([ring, ring.new_empty(1)]).scatter(0, push.reshape(-1), ids.reshape(-1))[:size]
    ends = torch.stack([s["ends"][0] + torch.minimum(take.sum(), s["ends"][1] - s["ends"][0]), s["ends"][1] + give.sum()])
    got = dict(table=table, len=out_len, ring=ring, ends=ends, copies=copies, status=status)
    if s["cache"] is None:
        return got
    a, b, fill = copies[copied, 0].long(), copies[copied, 1].long(), (new_len % bs)[copied]
    cache = s["cache"]
    cache[:, b] = torch.where((torch.arange(bs, device=dev) < fill[:, None])[None, :, :, None], cache[:, a], cache[:, b])
    return dict(got, cache=cache)


# ---------------------------------------------------------------------------
# The selection by its definition, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] != "select":
        return None  # whole numbers and copies
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = _prepare_select(case, g)
    groups, beams, n = case["groups"], case["beams"], case["keep"]
    got = {k: [] for k in ("score", "parent", "token", "next_score", "next_parent", "next_token")}
    for group in range(groups):
        x = s["logits"][group * beams:(group + 1) * beams].double()
        score = s["score"][group * beams:(group + 1) * beams].double()
        total = (x - torch.logsumexp(x, 1, keepdim=True) + score[:, None]).nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf).reshape(-1)
        order = torch.sort(total, descending=True, stable=True).indices[:n].tolist()
        best = [(float(total[i]), group * beams + i // case["vocab"], i % case["vocab"]) for i in order if float(total[i]) > -math.inf]
        onward = [b for b in best if b[2] != s["eos"]][:beams]
        for name, rows, most in (("", best, n), ("next_", onward, beams)):
            rows = rows + [(-math.inf, -1, -1)] * (most - len(rows))
            got[name + "score"].append([r[0] for r in rows])
            got[name + "parent"].append([r[1] for r in rows])
            got[name + "token"].append([r[2] for r in rows])
    return {k: torch.tensor(v, dtype=torch.float64 if k.endswith("score") else torch.int32) for k, v in got.items()}
