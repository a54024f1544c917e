"""The 8-bit paged KV cache in fp64: appending, and attention over it.

Written from the definitions: a tile is 32 slots of one page and KV head and
holds e4m3 numbers with one power-of-two scale for the keys and one for the
values.  The cache here is a dict of plain arrays indexed by page, head and
slot, not the library's layout:

    k, v       [pages, Hkv, slots, dh] fp64: the e4m3 numbers
    k_exp, v_exp [pages, Hkv, slots / 32] int: their tiles' exponents
"""

from __future__ import annotations

import numpy as np

E_MIN = -110


def _e4m3_values() -> np.ndarray:
    """The 127 finite non-negative e4m3 numbers, by their codes."""
    code = np.arange(127)
    e, m = code >> 3, code & 7
    return np.where(e == 0, m / 8.0 * 2.0**-6, (1 + m / 8.0) * 2.0 ** (e - 7.0))


E4M3 = _e4m3_values()


def e4m3_decode(code: np.ndarray) -> np.ndarray:
    code = np.asarray(code, dtype=np.int64)
    mag = np.append(E4M3, np.nan)[code & 127]
    return np.where(code & 128, -mag, mag)


def e4m3_round(x: np.ndarray) -> np.ndarray:
    """The nearest e4m3 number (ties to the even code); beyond the range the
    largest, a NaN stays one."""
    a = np.abs(np.nan_to_num(x, nan=0.0, posinf=1e300, neginf=-1e300))
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    pick = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(x), np.nan, np.copysign(E4M3[pick], x))


def tile_exponent(x: np.ndarray) -> int:
    """The smallest e >= E_MIN with |x| <= 448 * 2^e for the finite values."""
    x = np.abs(x[np.isfinite(x)])
    top = x.max() if x.size else 0.0
    e = E_MIN
    while top > 448.0 * 2.0**e:
        e += 1
    return e


def empty(pages: int, heads: int, page: int, dh: int) -> dict:
    exps = lambda: np.full((pages, heads, page // 32), E_MIN, dtype=np.int64)  # noqa: E731
    return dict(k=np.zeros((pages, heads, page, dh)), v=np.zeros((pages, heads, page, dh)), k_exp=exps(), v_exp=exps())


def rotate(k: np.ndarray, pos: int, base: float) -> np.ndarray:
    """Rotate-half of [..., dh] by position `pos`."""
    half = k.shape[-1] // 2
    w = pos * base ** (-np.arange(half) / half)
    a, b = k[..., :half], k[..., half:]
    return np.concatenate([a * np.cos(w) - b * np.sin(w), b * np.cos(w) + a * np.sin(w)], -1)


def append(cache: dict, table, length: int, k: np.ndarray, v: np.ndarray, base=None):
    """Append rows k, v [n, Hkv, dh] behind `length` cached slots of one
    sequence (table: its pages).  Returns the unrounded numbers that the new
    slots hold, in units of their tiles' scales: (k, v) [n, Hkv, dh]."""
    n, heads, _ = k.shape
    page = cache["k"].shape[2]
    if base:
        k = np.stack([rotate(k[j], length + j, base) for j in range(n)])
    raw = []
    for name, x in (("k", k), ("v", v)):
        num, exps = cache[name], cache[name + "_exp"]
        out = np.zeros(x.shape)
        for t in range(length // 32, (length + n + 31) // 32):
            lo, hi = max(length, 32 * t), min(length + n, 32 * t + 32)
            pg, s0 = table[32 * t // page], 32 * t % page
            for h in range(heads):
                rows = x[lo - length:hi - length, h]
                e = tile_exponent(rows)
                old = max(0, length - 32 * t)
                if old > 0:
                    was = int(exps[pg, h, s0 // 32])
                    e = max(e, was)
                    num[pg, h, s0:s0 + old] = e4m3_round(num[pg, h, s0:s0 + old] * 2.0 ** (was - e))
                exps[pg, h, s0 // 32] = e
                out[lo - length:hi - length, h] = rows * 2.0**-e
                num[pg, h, s0 + lo - 32 * t:s0 + hi - 32 * t] = e4m3_round(rows * 2.0**-e)
        raw.append(out)
    return raw


def read(cache: dict, table, n: int):
    """The first n slots of a sequence: (k, v) [Hkv, n, dh]."""
    page = cache["k"].shape[2]
    out = []
    for name in ("k", "v"):
        num, exps = cache[name], cache[name + "_exp"]
        x = np.zeros((num.shape[1], n, num.shape[3]))
        for s in range(n):
            pg, at = table[s // page], s % page
            x[:, s] = num[pg, :, at] * 2.0 ** exps[pg, :, at // 32][:, None]
        out.append(x)
    return out


def visible(length: int, anc, window: int = 0, sinks: int = 0) -> np.ndarray:
    """sees[i, x]: whether node i sees key x (the cached slots, then the
    nodes); anc[i]: bits of the nodes that node i sees."""
    n = len(anc)
    sees = np.zeros((n, length + n), dtype=bool)
    for i in range(n):
        up = [j for j in range(n) if int(anc[i]) >> j & 1]
        pos = length + sum(j != i for j in up)
        ok = lambda at: window == 0 or pos - at < window or at < sinks  # noqa: E731
        for s in range(length):
            sees[i, s] = ok(s)
        for r, j in enumerate(up):
            sees[i, length + j] = ok(length + r)
    return sees


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, ck: np.ndarray, cv: np.ndarray, sees: np.ndarray,
              scale=None):
    """q [N, Hq, dh], the nodes' own k, v [N, Hkv, dh], the cached ck, cv
    [Hkv, len, dh], sees [N, len + N].  Returns o [N, Hq, dh] and, for bounds
    of its rounding, the weighted magnitudes sum p |v| [N, Hq, dh] and the
    largest sum of a score's magnitudes, sum |q| |k| * scale.  What is not
    seen does not enter; a node that sees nothing gets zeros."""
    n, hq, dh = q.shape
    group = hq // k.shape[1]
    scale = dh**-0.5 if scale is None else scale
    o, mag, top = np.zeros(q.shape), np.zeros(q.shape), 0.0
    for h in range(hq):
        keys = np.concatenate([ck[h // group], k[:, h // group]])
        vals = np.concatenate([cv[h // group], v[:, h // group]])
        for i in range(n):
            at = np.nonzero(sees[i])[0]
            if not len(at):
                continue
            s = keys[at] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o[i, h] = p @ vals[at]
            mag[i, h] = p @ np.abs(vals[at])
            top = max(top, float((np.abs(keys[at]) @ np.abs(q[i, h])).max() * scale))
    return o, mag, top
