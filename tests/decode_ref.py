"""Plain implementations of the calls on a replica's rows (wf_kv_extend,
wf_beam_select, wf_kv_reorder): row by row, in Python integers and 64-bit
floats, written from their declarations in include/wf.h."""
import math

import numpy as np

LONG, BLOCKS, TOKENS, PARENT = 1, 2, 4, 1


def extend(table, length, add, ring, ends, bs, max_tokens):
    """Returns table, slot, pos, row, start, len, ends, status."""
    rows, width = table.shape
    table, n = table.copy(), ring.size
    slot = np.full(max_tokens, -1, np.int64)
    pos, row = np.zeros(max_tokens, np.int32), np.full(max_tokens, -1, np.int32)
    start, out_len, status = np.zeros(rows + 1, np.int64), length.copy(), np.zeros(rows, np.int32)
    head, tail = (int(x) for x in ends)
    blocks = tokens = 0  # asked for by the rows so far
    taken = placed = 0   # given to the admitted ones
    for r in range(rows):
        start[r] = placed
        have, want = int(length[r]), int(add[r])
        if have < 0 or want < 0 or -(-(have + want) // bs) > width:
            status[r] = LONG
            continue
        need = -(-(have + want) // bs) - -(-have // bs)
        blocks += need
        tokens += want
        status[r] = (BLOCKS if blocks > tail - head else 0) | (TOKENS if tokens > max_tokens else 0)
        if status[r]:
            continue
        for i in range(need):
            table[r, -(-have // bs) + i] = ring[(head + taken + i) % n]
        p = np.arange(have, have + want)
        slot[placed:placed + want] = table[r, p // bs].astype(np.int64) * bs + p % bs
        pos[placed:placed + want], row[placed:placed + want] = p, r
        out_len[r] = have + want
        taken += need
        placed += want
    start[rows] = placed
    return dict(table=table, slot=slot, pos=pos, row=row, start=start.astype(np.int32), len=out_len,
                ends=np.array([head + taken, tail], np.int64), status=status)


def reorder(table, length, ring, ends, bs, group, parent, to_table, cache=None):
    """Returns table, len, ring, ends, copies, status (and cache [planes, n_blocks, bs, ...])."""
    rows, width = table.shape
    out, ring, n = to_table.copy(), ring.copy(), ring.size
    out_len, status = np.zeros(rows, np.int32), np.zeros(rows, np.int32)
    copies = np.full((rows, 2), -1, np.int32)
    cache = None if cache is None else cache.copy()
    head, tail = (int(x) for x in ends)
    old_head, old_tail = head, tail
    held = [min(max(int(x), 0), width * bs) for x in length]
    nb = lambda x: -(-x // bs)
    asked = 0  # blocks asked of the ring so far
    for g in range(0, rows, group):
        par = []
        for r in range(g, g + group):
            ok = g <= parent[r] < g + group
            if not ok and parent[r] != -1:
                status[r] = PARENT
            par.append(int(parent[r]) if ok else -1)
        new = [[] if p < 0 else [int(x) for x in table[p, :nb(held[p])]] for p in par]
        size = [0 if p < 0 else held[p] for p in par]
        freed = []
        for j in range(width):
            still = {blocks[j] for blocks in new if len(blocks) > j}
            for r in range(g, g + group):
                if j < nb(held[r]) and int(table[r, j]) not in still:
                    still.add(int(table[r, j]))
                    freed.append(int(table[r, j]))
        owner, spare = set(), list(freed)
        for k in range(group):
            r = g + k
            if size[k] % bs:
                last = (len(new[k]) - 1, new[k][-1])
                if last in owner:
                    if spare:
                        dst = spare.pop(0)
                    else:
                        asked += 1
                        dst = int(ring[(old_head + asked - 1) % n]) if asked <= old_tail - old_head else None
                    if dst is None:
                        status[r] |= BLOCKS
                        size[k] -= size[k] % bs
                        new[k].pop()
                    else:
                        copies[r] = (last[1], dst)
                        if cache is not None:
                            cache[:, dst, :size[k] % bs] = cache[:, last[1], :size[k] % bs]
                        new[k][-1] = dst
                owner.add(last)
            out[r, :len(new[k])] = new[k]
            out_len[r] = size[k]
        for b in spare:
            ring[tail % n] = b
            tail += 1
    head += min(asked, max(old_tail - old_head, 0))
    got = dict(table=out, len=out_len, ring=ring, ends=np.array([head, tail], np.int64), copies=copies, status=status)
    return got if cache is None else dict(got, cache=cache)


def sums(logits, score):
    """Every candidate's sum in 64 bits, [rows, vocab]; -inf where it is none."""
    x = np.asarray(logits, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    out = np.full(x.shape, -np.inf)
    for r in range(x.shape[0]):
        m = x[r].max()
        if m == -np.inf or not score[r] > -np.inf:
            continue
        if m == np.inf:
            out[r, x[r] == m] = float(score[r]) - math.log(np.count_nonzero(x[r] == m))
            continue
        out[r] = float(score[r]) + (x[r] - m) - math.log(np.exp(x[r] - m).sum())
    return out


def select(logits, score, beams, keep):
    """The keep best (sum, parent, token) of each group, by (sum, beam, logit, token)."""
    c = sums(logits, score)
    vocab = c.shape[1]
    best = []
    for g in range(0, c.shape[0], beams):
        flat = c[g:g + beams].reshape(-1)
        order = np.argsort(-flat, kind="stable")[:keep]
        best.append([(flat[i], g + int(i) // vocab, int(i) % vocab) for i in order if flat[i] > -np.inf])
    return best
