"""CPU oracle of the microscaled 4-bit matrices and of the norms between blocks, in numpy fp64.

Written from the formats' definitions (E2M1 elements; E8M0 scales over 32 columns or E4M3 scales over
16) and the operators' formulas; shares nothing with the GPU path.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {"e8m0": 32, "e4m3": 16}


def _e4m3_table() -> np.ndarray:
    v = np.empty(128)
    for c in range(128):
        e, m = c >> 3, c & 7
        v[c] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    v[127] = np.nan
    return v


E4M3 = _e4m3_table()


def scale_values(byte: np.ndarray, fmt: str) -> np.ndarray:
    if fmt == "e8m0":
        return np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127.0))
    return E4M3[byte & 127]


def nearest_even(v: np.ndarray, table: np.ndarray) -> np.ndarray:
    """Index of the nearest entry of an ascending table, ties to the even index, clipped at both ends."""
    hi = np.clip(np.searchsorted(table, v), 1, len(table) - 1)
    lo = hi - 1
    a, b = v - table[lo], table[hi] - v
    return np.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def quantize(x: np.ndarray, fmt: str, scale: float):
    """(codes rows x cols in 0..15, scale bytes rows x blocks) of x (fp32 values), scale a power of two."""
    rows, cols = x.shape
    blk = BLOCK[fmt]
    nb = -(-cols // blk)
    v = np.zeros((rows, nb * blk))
    v[:, :cols] = x.astype(np.float64) / scale
    v = v.reshape(rows, nb, blk)
    bad = ~np.isfinite(v).all(axis=2) | (np.abs(v).max(axis=2) > np.finfo(np.float32).max)
    v = np.where(bad[:, :, None], 0.0, v)
    top = np.abs(v).max(axis=2)
    if fmt == "e8m0":
        e = np.frexp(top)[1] - 3                       # floor(log2 top) - 2
        byte = np.where(top > 0, np.clip(e, -127, 125), -127) + 127
    else:
        byte = nearest_even(np.minimum(top / 6.0, 448.0), E4M3[:127])
    sc = scale_values(byte, fmt)[:, :, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(sc > 0, np.abs(v) / sc, 0.0)
    codes = nearest_even(q, E2M1) + 8 * (np.signbit(v) & (sc > 0))
    byte = np.where(bad, 255 if fmt == "e8m0" else 127, byte)
    codes = np.where(bad[:, :, None], 0, codes)
    return codes.reshape(rows, -1)[:, :cols].astype(np.uint8), byte.astype(np.uint8)


def values(codes: np.ndarray, byte: np.ndarray, fmt: str, scale: float) -> np.ndarray:
    e = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes & 7]
    sc = np.repeat(scale_values(byte, fmt), BLOCK[fmt], axis=1)[:, :codes.shape[1]]
    return e * sc * scale


def pack_codes(codes: np.ndarray) -> np.ndarray:
    """Stored bytes: rows x 16 ceil(cols / 32), even column in the lower half."""
    rows, cols = codes.shape
    c = np.zeros((rows, 32 * (-(-cols // 32))), np.uint8)
    c[:, :cols] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def tile_scales(byte: np.ndarray) -> np.ndarray:
    """Scale bytes in the stored order, one by one from the layout's formula."""
    rows, nb = byte.shape
    tiles = -(-nb // 4)
    out = np.zeros(-(-rows // 128) * tiles * 512, np.uint8)
    r, b = np.meshgrid(np.arange(rows), np.arange(nb), indexing="ij")
    out[((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4] = byte
    return out


def silu(v: np.ndarray) -> np.ndarray:
    with np.errstate(over="ignore"):
        return v / (1.0 + np.exp(-v))


def product(w: np.ndarray, x: np.ndarray, up: np.ndarray | None = None):
    """(y, sum |w||x|, and with up also u and its sum) for w rows x cols, x T x cols in fp64."""
    y, a = x @ w.T, np.abs(x) @ np.abs(w).T
    if up is None:
        return y, a
    return y, a, x @ up.T, np.abs(x) @ np.abs(up).T


def block_norm(h, y=None, post=None, gate=None, channel=None, branch_scale=1.0, residual_scale=1.0,
               pre=None, post_eps=1e-6, pre_eps=1e-6):
    """(h', branch, x): post None: no post-norm, else the gains (D); gate broadcastable to T x D; pre: gains."""
    b = np.zeros_like(h)
    if y is not None:
        b = y.copy()
        if post is not None:
            b = b / np.sqrt((b * b).mean(axis=1, keepdims=True) + post_eps) * post
        if gate is not None:
            b = b * gate
        if channel is not None:
            b = b * channel
        b = b * branch_scale
    hn = residual_scale * h + b
    x = hn / np.sqrt((hn * hn).mean(axis=1, keepdims=True) + pre_eps)
    return hn, b, x if pre is None else x * pre
