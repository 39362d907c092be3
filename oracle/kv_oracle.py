"""64-bit forms of the attention block over a 4-bit paged cache, written from the definitions in include/mdbf.h
(test infrastructure only; shares no code with the library)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
SCALE_RANGE = {"f16": (-23, 13), "bf16": (-125, 125)}
BLOCK = 32


def slots(cached, fresh, table, free, taken, page_size, tokens):
    """One request after the other.  Returns a dict of what the call writes, table among it."""
    table = np.array(table)
    n, width = table.shape
    status = 0
    need = []
    for c, f in zip(cached, fresh):
        if c < 0 or f < 0 or c + f > 2 ** 31 - 1:
            status |= 1
            need.append((0, 0))
            continue
        before, after = -(-c // page_size), -(-(c + f) // page_size)
        status |= 2 if after > width else 0
        need.append((before, after))
    if sum(f for c, f in zip(cached, fresh) if c >= 0 and f >= 0 and c + f <= 2 ** 31 - 1) > tokens:
        status |= 4
    if taken < 0 or taken + sum(a - b for b, a in need) > len(free):
        status |= 8
    out = dict(status=status, slots=np.full(tokens, -1, np.int64), positions=np.full(tokens, -1, np.int32))
    if status:
        return dict(out, table=table, taken=taken, lengths=np.maximum(np.array(cached), 0), cu=np.zeros(n + 1, int))
    at, cu = 0, [0]
    for r, (c, f) in enumerate(zip(cached, fresh)):
        for i in range(*need[r]):
            table[r, i] = free[taken]
            taken += 1
        for pos in range(c, c + f):
            out["slots"][at] = int(table[r, pos // page_size]) * page_size + pos % page_size
            out["positions"][at] = pos
            at += 1
        cu.append(at)
    return dict(out, table=table, taken=taken, lengths=np.array(cached) + np.array(fresh), cu=np.array(cu))


def quantise(x, dtype):
    """x (..., multiple of 32): codes (uint8, one per entry) and scale bytes (one per block)."""
    x = np.asarray(x, np.float64)
    codes = np.zeros(x.shape, np.uint8)
    scales = np.zeros(x.shape[:-1] + (x.shape[-1] // BLOCK,), np.uint8)
    lo, hi = SCALE_RANGE[dtype]
    flat, fc, fs = x.reshape(-1, BLOCK), codes.reshape(-1, BLOCK), scales.reshape(-1)
    for b in range(flat.shape[0]):
        block = flat[b]
        if not np.isfinite(block).all():
            fs[b] = 255
            continue
        top, e = np.abs(block).max(), lo
        while e < hi and top > 7 * 2.0 ** e:
            e += 1
        mag = np.minimum(np.abs(block) / 2.0 ** e, 6.0)      # beyond the largest number: saturated
        dist = np.abs(mag[:, None] - LEVELS[None])
        near = dist.min(1, keepdims=True)
        tie = dist == near                      # two at a tie: the even code
        for i in range(BLOCK):
            c = np.flatnonzero(tie[i])
            fc[b, i] = c[0] if len(c) == 1 or c[0] % 2 == 0 else c[1]
            if block[i] < 0:
                fc[b, i] |= 8
        fs[b] = e + 127
    return codes, scales


def values(codes, scales):
    sign = np.where(codes & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return sign * LEVELS[codes & 7] * np.repeat(unit, BLOCK, -1)


def page_views(pool, pages, kv_heads, page_size, d):
    """Views of a pool's bytes: key codes, value codes, key scales, value scales (pages, heads, tokens, bytes)."""
    p = np.asarray(pool).reshape(pages, kv_heads, page_size * (d + d // 16))
    cb, sb = page_size * d // 2, page_size * d // 32
    cut = [0, cb, 2 * cb, 2 * cb + sb, 2 * cb + 2 * sb]
    return [p[:, :, a:b].reshape(pages, kv_heads, page_size, -1) for a, b in zip(cut, cut[1:])]


def unpack(nibbles):
    return np.stack([nibbles & 15, nibbles >> 4], -1).reshape(nibbles.shape[:-1] + (2 * nibbles.shape[-1],))


def norm_rope(x, weight, rope, positions, eps, interleaved):
    """x (T, heads, d) in 64 bits; rope (rows, rot): cosines, then sines."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if rope is not None:
        rot = rope.shape[1]
        y = x.copy()
        for t, pos in enumerate(positions):
            if pos < 0:
                continue
            for i in range(rot // 2):
                c, s = (float(rope[pos, i]), float(rope[pos, rot // 2 + i])) if pos < rope.shape[0] else (np.nan, np.nan)
                a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
                y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
                y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
        x = y
    if positions is not None:
        x[np.asarray(positions) < 0] = 0
    return x


def attention(q, k, v, positions, causal, window, scale):
    """One head of one request: q (rows, d) with the rows' positions, k and v (tokens, d).  Returns the result, the
    weighted sum of |v| (what the roundings of the weights are relative to) and the sum of the numerators."""
    out, mag, den = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1])), np.ones(len(q))
    for r, pos in enumerate(positions):
        lo, hi = 0, len(k)
        if causal:
            hi = min(hi, max(pos + 1, 0))
            lo = max(pos - window + 1, 0) if window else 0
        if hi <= lo:
            continue
        z = k[lo:hi] @ q[r] * scale
        e = np.exp(z - z.max())
        den[r] = e.sum()
        p = e / den[r]
        out[r], mag[r] = (p[:, None] * v[lo:hi]).sum(0), p @ np.abs(v[lo:hi])
    return out, mag, den
