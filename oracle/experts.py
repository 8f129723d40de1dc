"""Oracle of the operators around dense experts (numpy, float64, written from their definitions): rows in 8 bits,
routing lists, ragged products and the weighted sum.  Test infrastructure only."""
import numpy as np

LOW = -100   # least exponent of a row's scale


def e4m3_values() -> np.ndarray:
    """The value of each E4M3 byte: 1 sign, 4 exponent (bias 7), 3 mantissa bits; 127 and 255 are NaN."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = np.nan if (b & 127) == 127 else -v if b & 128 else v
    return out


def e4m3_codes(v: np.ndarray) -> np.ndarray:
    """The nearest E4M3 byte of finite values of magnitude <= 448, ties to the even byte."""
    grid = e4m3_values()[:127]
    a = np.abs(np.asarray(v, np.float64))
    hi = np.clip(np.searchsorted(grid, a), 0, 126)   # first byte whose value is >= a
    lo = np.maximum(hi - 1, 0)
    mid = (grid[lo] + grid[hi]) / 2                  # exact
    up = (a > mid) | ((a == mid) & (hi % 2 == 0))
    return (np.where(up, hi, lo) + 128 * np.signbit(v)).astype(np.uint8)


def rowscale(x: np.ndarray):
    """Codes (uint8) and scales (float32) of the rows of x."""
    x = np.asarray(x, np.float64)
    codes = np.zeros(x.shape, np.uint8)
    scales = np.empty(x.shape[0], np.float32)
    for r, row in enumerate(x):
        if not np.isfinite(row).all():
            scales[r] = np.nan
            continue
        a, e = np.abs(row).max() if row.size else 0.0, LOW
        while a > 448.0 * 2.0 ** e:
            e += 1
        scales[r] = 2.0 ** e
        codes[r] = e4m3_codes(row / 2.0 ** e)
    return codes, scales


def route(logits: np.ndarray, k: int, renormalize: bool = True):
    """(experts, weights, offsets, pairs, places) of the rows of logits."""
    T, E = logits.shape
    experts = np.full((T, k), -1, np.int32)
    weights = np.zeros((T, k))
    for t in range(T):
        v = np.asarray(logits[t], np.float64)
        can = [e for e in range(E) if not np.isnan(v[e]) and v[e] != -np.inf]
        best = sorted(can, key=lambda e: (-v[e], e))[:k]
        if not best:
            continue
        experts[t, :len(best)] = best
        w = np.exp(v[best] - v[best[0]])
        weights[t, :len(best)] = w / (w if renormalize else np.exp(v[can] - v[best[0]])).sum()
    lists = [[t * k + j for t in range(T) for j in range(k) if experts[t, j] == e] for e in range(E)] if T * E <= 4096 else None
    if lists is None:
        flat = experts.reshape(-1)
        order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
        n = int((flat >= 0).sum())
        pairs, counts = order[:n], np.bincount(flat[flat >= 0], minlength=E)
    else:
        pairs, counts = np.array(sum(lists, []), np.int64), np.array([len(x) for x in lists])
    places = np.full(T * k, -1, np.int32)
    places[pairs] = np.arange(len(pairs))
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    pairs = np.concatenate([pairs, np.full(T * k - len(pairs), -1)]).astype(np.int32)
    return experts, weights, offsets, pairs, places.reshape(T, k)


def product(w, x, offsets, index=None, fan=1, up=None):
    """(y, sums) with NaN rows where no expert has one; sums: for each result the sums of the products' magnitudes, of
    w and of up (what a rounding error is measured by), and the two products."""
    E = w.shape[0]
    P = len(index) if index is not None else x.shape[0]
    y = np.full((P, w.shape[1]), np.nan)
    parts = []
    for p in range(P):
        e = int(np.searchsorted(offsets, p, side="right")) - 1
        if e < 0 or e >= E:
            parts.append(None)
            continue
        q = int(index[p]) // fan if index is not None else p
        if q < 0 or q >= x.shape[0] or (index is not None and index[p] < 0):
            parts.append("bad")
            continue
        g = w[e] @ x[q]
        mg = np.abs(w[e]) @ np.abs(x[q])
        if up is None:
            y[p] = g
            parts.append((g, mg, None, None))
        else:
            u = up[e] @ x[q]
            y[p] = g / (1 + np.exp(-g)) * u
            parts.append((g, mg, u, np.abs(up[e]) @ np.abs(x[q])))
    return y, parts


def combine(y, places, weights, base=None):
    T, k = places.shape
    out = np.zeros((T, y.shape[1])) if base is None else base.copy()
    for t in range(T):
        for j in range(k):
            if 0 <= places[t, j] < y.shape[0]:
                out[t] += weights[t, j] * y[places[t, j]]
    return out
