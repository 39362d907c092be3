"""What stands around the projections of a serving step, in 64 bits (numpy): residual addition with norm, the tables that order rows by
adapter, the adapters' products, sampling.  Test infrastructure only."""
import numpy as np

TILE = 64
E4M3_MAX = 448.0


def add_norm(x, residual, weight, eps):
    """(y, h): h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, rows of float64."""
    h = x if residual is None else x + residual
    y = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return (y if weight is None else y * weight), h


def e4m3(v):
    """The nearest 8-bit number (four significant bits, subnormals of 2^-9), ties to even."""
    v = np.asarray(v, dtype=np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e, -5) - 4)
    return np.clip(np.round(v / step) * step, -E4M3_MAX, E4M3_MAX)


def block_scales(y):
    """Scale bytes of blocks of 32: the smallest power of two, from 2^-126, that leaves the largest at most 448; 255 for what is not finite."""
    T, n = y.shape
    out = np.zeros((T, -(-n // 32)), dtype=np.int64)
    for b in range(out.shape[1]):
        top = np.abs(y[:, 32 * b:32 * b + 32]).max(axis=1)
        for t in range(T):
            if not np.isfinite(top[t]):
                out[t, b] = 255
                continue
            e = -126
            while top[t] > E4M3_MAX * 2.0 ** e and e < 127:
                e += 1
            out[t, b] = e + 127
    return out


def adapter_tables(cu, adapter, adapters, T, room):
    """(rows, tiles, places), by going through the adapters and the requests."""
    rows, tiles, places = [], [], np.zeros(len(adapter), dtype=np.int64)
    of = [[] for _ in range(adapters + 1)]
    for r, a in enumerate(adapter):
        of[a if 0 <= a < adapters else adapters].append(r)
    at = 0
    for a, requests in enumerate(of):
        first = at
        for r in requests:
            places[r] = at
            n = cu[r + 1] - cu[r]
            if a < adapters:
                rows.extend(range(cu[r], cu[r + 1]))
            at += n
        if a < adapters:
            for done in range(0, at - first, TILE):
                tiles.append((a, first + done, min(TILE, at - first - done), 0))
    rows += [-1] * (T - len(rows))
    tiles += [(-1, 0, 0, 0)] * (room - len(tiles))
    return np.array(rows), np.array(tiles).reshape(room, 4), places


def adapters(x, of, A, B, scale):
    """What is added to y: scale[a] B[a] (A[a] x) of each row, a = of[t]; zeros where that is none."""
    out = np.zeros((x.shape[0], B.shape[1]))
    for t, a in enumerate(of):
        if 0 <= a < A.shape[0]:
            out[t] = (1.0 if scale is None else scale[a]) * (B[a] @ (A[a] @ x[t]))
    return out


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, share) of one row, from the definition: an ordered list of tokens, cut three times, and a walk along it."""
    z = np.asarray(logits, dtype=np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    top = z.max()
    if top == -np.inf:
        return -1, 0.0
    order = np.argsort(-z, kind="stable")
    if not temperature > 0:
        return int(order[0]), 1.0
    u = 0.0 if np.isnan(u) else min(max(float(u), 0.0), 1 - 2.0 ** -24)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(z == top, 1.0, np.exp((z - top) / np.float64(temperature)))
    w = np.where((z == -np.inf) | ((top == np.inf) & (z != top)), 0.0, w)[order]
    n = len(w)
    if 0 < top_k < n:
        n = int(top_k)
    if top_p < 1:
        mass = np.concatenate(([0.0], np.cumsum(w[:n])))
        n = max(1, int(np.sum(mass[:-1] < np.float64(top_p) * mass[-1])))
    if min_p > 0:
        n = max(1, int(np.sum(w[:n] >= np.float64(min_p))))
    mass = np.cumsum(w[:n])
    at = int(np.sum(mass <= u * mass[-1]))
    return int(order[at]), float(w[at] / mass[-1])
