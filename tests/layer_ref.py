"""Plain implementations of the calls on a layer's tensors (wf_kv_write,
wf_kv_copy_scales, wf_attend): token by token and head by head, in 64-bit floats,
written from their declarations in include/wf.h."""
import numpy as np


def rotate(x, pos, freq, interleaved, magnitude):
    """x [tokens, heads, dim]; freq [pairs] radians a position."""
    x, n = np.array(x, np.float64), len(freq)
    angle = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)
    cos, sin = np.cos(angle)[:, None] * magnitude, np.sin(angle)[:, None] * magnitude
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., first].copy(), x[..., second].copy()
    x[..., first], x[..., second] = a * cos - b * sin, b * cos + a * sin
    return x


def eight(x):
    """The nearest value of E4M3, ties to even; beyond 448 +-448, NaN stays."""
    x = np.asarray(x, np.float64)
    size = np.minimum(np.abs(x), 500.0)  # above 448 all the same
    exp = np.floor(np.log2(np.maximum(size, 2.0 ** -6)))
    step = 2.0 ** (exp - 3)
    return np.copysign(np.minimum(np.rint(size / step) * step, 448.0), x)


def need(x):
    """The least 2^e, -64 <= e <= 63, whose 448-fold reaches the largest finite magnitude."""
    x = np.abs(np.asarray(x, np.float64))
    most = x[np.isfinite(x)].max(initial=0.0)
    for e in range(-64, 63):
        if 448 * 2.0 ** e >= most:
            return 2.0 ** e
    return 2.0 ** 63


def write8(cache, scale, slot, bs, x):
    """cache [n_blocks, bs, heads, dim] values of E4M3, scale [n_blocks, heads], x [tokens, heads, dim] rounded to its
    type; changed in place."""
    parts = []
    for t, s in enumerate(slot):
        if s < 0:
            continue
        if t and slot[t - 1] == s - 1 and s % bs:
            parts[-1].append(t)
        else:
            parts.append([t])
    for part in parts:
        b, first = divmod(int(slot[part[0]]), bs)
        for h in range(x.shape[1]):
            now = need(x[part, h])
            if first:
                now = max(now, float(scale[b, h]))
                if now != scale[b, h]:
                    cache[b, :first, h] = eight(cache[b, :first, h] * (float(scale[b, h]) / now))
            scale[b, h] = now
            for i, t in enumerate(part):
                cache[b, first + i, h] = eight(x[t, h] / now)


def attend(q, k, v, table, start, length, bs, scale, out, v_scale=None):
    """q [tokens, heads, dim]; k, v [n_blocks, bs, kv heads, dim] values; out is filled in place and returned, and beside it what
    errors are relative to: the sum over a row's positions of |softmax| |v|, and the largest softmax times scale of the value's block
    (v_scale [n_blocks, kv heads] or 1) times the sum of |v| over that scale."""
    size, small = np.zeros(out.shape), np.zeros(out.shape)
    group = q.shape[1] // k.shape[2]
    for r in range(len(length)):
        n = int(start[r + 1] - start[r])
        if n <= 0:
            continue
        total = int(length[r])
        p = np.arange(total)
        blocks, place = table[r, p // bs], p % bs
        for h in range(q.shape[1]):
            kh, vh = k[blocks, place, h // group], v[blocks, place, h // group]
            f = np.ones(total) if v_scale is None else v_scale[blocks, h // group]
            bare = np.cumsum(np.abs(vh) / f[:, None], 0)
            for i in range(n):
                last = total - n + i + 1
                x = scale * (kh[:last] @ q[start[r] + i, h])
                w = np.exp(x - x.max())
                w /= w.sum()
                out[start[r] + i, h] = w @ vh[:last]
                size[start[r] + i, h] = w @ np.abs(vh[:last])
                small[start[r] + i, h] = (w * f[:last]).max() * bare[last - 1]
    return out, size, small
