"""A plain paged cache of 8-bit numbers in 64 bits, and the bounds that its operators are held to (not collected by pytest).

e4m3: sign, 4 bits of exponent with bias 7, 3 of mantissa; 0x7f and 0xff are NaN, 0x7e is 448, below 2^-6 steps of 2^-9.
"""
import numpy as np

import operators_reference as ref

_BYTE = np.arange(127)
_EXP, _MAN = _BYTE >> 3, _BYTE & 7
VALUES = np.where(_EXP > 0, (1 + _MAN / 8) * 2.0 ** (_EXP - 7), _MAN * 2.0 ** -9)          # of 0x00 .. 0x7e
_BETWEEN = (VALUES[1:] + VALUES[:-1]) / 2


def decode(codes):
    codes = np.asarray(codes, np.uint8)
    size = np.concatenate([VALUES, [np.nan]])[codes & 0x7f]
    return np.where(codes & 0x80, -size, size)


def nearest(x):
    """Each value's nearest 8-bit number, ties to even, as a value; not finite: NaN; past 448: 448."""
    x = np.asarray(x, np.float64)
    size = np.where(np.isfinite(x), np.abs(x), 0.0)
    up, down = np.searchsorted(_BETWEEN, size, "right"), np.searchsorted(_BETWEEN, size, "left")
    k = np.where(up == down, up, np.where(up % 2 == 0, up, down))         # on a border the two differ by one: the even code
    return np.where(np.isfinite(x), np.copysign(VALUES[k], x), np.nan)


def power_for(m):
    """The least power of two between 2^-96 and 2^119 by which values up to m lie within 448."""
    if m == 0:
        return 2.0 ** -96
    e = int(np.floor(np.log2(m))) - 9
    while m > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** min(max(e, -96), 119)


def turned(x, at, frequencies, interleaved=False, magnitude=1.0):
    """x [rows, heads, dh] at positions, the angle reduced to a turn in extended precision, as positions may be far."""
    y, n = np.array(x, np.float64), len(frequencies)
    turns = np.asarray(at, np.longdouble)[:, None] * (np.asarray(frequencies) / (2 * np.pi)).astype(np.longdouble)
    angle = (2 * np.pi * (turns - np.rint(turns)).astype(np.float64))[:, None]
    c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    u, w = np.array(x[..., first], np.float64), np.array(x[..., second], np.float64)
    y[..., first], y[..., second] = u * c - w * s, u * s + w * c
    return y


class Cache:
    """numbers[page][head][row] in units of scale[page][head], values (not codes); NaN where nothing is known."""

    def __init__(self, pages, page, Hkv, dh):
        self.page, self.Hkv, self.dh = page, Hkv, dh
        self.numbers = {n: np.full((pages, Hkv, page, dh), np.nan) for n in "kv"}
        self.scale = {n: np.full((pages, Hkv), np.nan) for n in "kv"}

    def append(self, table, held, new, k, v):
        """k, v [rows, Hkv, dh]: the rows of sequence s are the last new[s] of its held[s] tokens."""
        row, P, pages = 0, self.page, len(self.scale["k"])
        for s, (length, n) in enumerate(zip(held, new)):
            at = length - n + np.arange(n)
            for p in np.unique(at[(at >= 0) & (at < P * table.shape[1])] // P):
                page = table[s, p]
                if not 0 <= page < pages:
                    continue
                mine = np.flatnonzero((at // P == p) & (at >= 0))
                a, b = at[mine[0]] - p * P, at[mine[-1]] - p * P + 1
                for name, x in (("k", k), ("v", v)):
                    for h in range(self.Hkv):
                        z = x[row + mine, h]
                        now = power_for(np.abs(z[np.isfinite(z)]).max(initial=0.0))
                        held_here, scale = self.numbers[name][page, h], self.scale[name]
                        if a > 0:
                            if now > scale[page, h]:
                                held_here[:a] = nearest(held_here[:a] * scale[page, h] / now)
                            now = max(now, scale[page, h])
                        held_here[a:b] = nearest(z / now)
                        scale[page, h] = now
            row += n

    def rows(self, name, table, s, length):
        """[length, Hkv, dh] of a sequence; tokens on no page are NaN."""
        out = np.full((length, self.Hkv, self.dh), np.nan)
        for j in range(length):
            page = table[s, j // self.page] if j // self.page < table.shape[1] else -1
            if 0 <= page < len(self.scale["k"]):
                out[j] = self.numbers[name][page, :, j % self.page] * self.scale[name][page][:, None]
        return out


def attention(cache, table, held, new, q, causal=True, window=0, scale=None, cap=0.0, slopes=None, dtype="bf16"):
    """{name: (value, bound)} for o [rows, H, dh] and lse [H, rows].  The bounds are those of attention over key ranges, three times as wide in float32, where
    queries and probabilities go through the matrix cores as three numbers each and sums have three times the terms."""
    H, dh = q.shape[1], q.shape[2]
    o, lse = [np.zeros(q.shape), np.zeros(q.shape)], [np.full((H, len(q)), -np.inf), np.zeros((H, len(q)))]
    row = 0
    for s, (length, n) in enumerate(zip(held, new)):
        length = min(length, cache.page * table.shape[1])
        k, v = cache.rows("k", table, s, length), cache.rows("v", table, s, length)
        there = np.array([j // cache.page < table.shape[1] and 0 <= table[s, j // cache.page] < len(cache.scale["k"]) for j in range(length)], bool)
        at = held[s] - n + np.arange(n)
        for r in range(n):                                   # (row by row: pages that are missing make holes in what it sees)
            hi = min(at[r] + 1, length) if causal else length
            lo = max(at[r] + 1 - window, 0) if window else 0
            see = np.flatnonzero(there[:max(hi, 0)])
            see = see[see >= lo]
            if len(see) == 0:
                continue
            kk, vv = k[see], v[see]
            if slopes is not None:
                got = _biased(q[row + r][None], kk, vv, at[r] - see, scale, cap, slopes, dtype)
            else:
                got = ref.attention(q[row + r][None], kk, vv, [0], [len(see)], None, scale, cap, None, None, dtype)
            o[0][row + r], o[1][row + r] = got["o"][0][0], got["o"][1][0]
            lse[0][:, row + r], lse[1][:, row + r] = got["lse"][0][:, 0], got["lse"][1][:, 0]
        row += n
    wide = 3.0 if dtype == "f32" else 1.0
    return {"o": (o[0], o[1] * wide), "lse": (lse[0], lse[1] * wide)}


def _biased(q, k, v, distance, scale, cap, slopes, dtype):
    """The same with a distance per key: keys are put where their distance from row 0 is what it should be."""
    order = np.argsort(distance)[::-1]                       # far ones first; holes between them are keys that nobody sees
    far = int(distance.max())
    near = min(int(distance.min()), 0)
    m = far - near + 1
    kk, vv = np.full((m,) + k.shape[1:], np.nan), np.full((m,) + v.shape[1:], np.nan)
    place = far - distance[order]
    kk[place], vv[place] = k[order], v[order]
    if len(place) == m:
        return ref.attention(q, kk, vv, [0], [m], [far], scale, cap, slopes, None, dtype)
    assert False, "a bias over missing pages is not tested"


def quantized(x):
    """Codes and scale of rows, the scale a 32-bit number and the quotient exact."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(1, initial=0.0)
    with np.errstate(invalid="ignore"):
        scale = (top / 127).astype(np.float32).astype(np.float64)
    scale[scale < 2.0 ** -126] = 0.0
    bad = ~np.isfinite(top)
    unit = np.where((scale > 0) & ~bad, scale, 1.0)
    codes = np.rint(np.where((bad | (scale == 0))[:, None], 0.0, x) / unit[:, None])      # (a quotient of two 32-bit numbers never rounds onto a half in 64 bits)
    scale[bad] = np.nan
    return codes, scale
