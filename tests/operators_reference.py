"""Float64 references of the operators for attention layers, with error bounds worked out from the arithmetic that the
kernels document (not collected by pytest).

Bounds.  u is half a step of the storage type (bf16 2^-8, float32 2^-24), e = 2^-24.  A score is a float32 sum of dh products: it
is off by at most (dh + 8) e sum |q k| scale, its cap by cap 2^-21 more (the bf16 kernels' tanh; the full one: 8 e of the score), its bias by 2 e slope distance.
A probability is off by twice that (its own score, the row's sum), by (n + 16) e for the exponential and the sum of n
terms, and in bf16 by u as an operand of the matrix cores: rel.  Hence o: rel sum p |v| and u |o| for its own
rounding; dv likewise over the queries.  D = <o, dO> inherits the error of o; ds = p (dP - D) is off by rel |ds|
(rounded to an operand as well), by p times the errors of D and of dP; dq and dk sum those, and are rounded themselves.
"""
import numpy as np

E32 = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": E32}


def ranges(q_lens, k_lens=None, causal=True, window=0, prefix=None, Tq=None):
    """lo, hi, at of packed documents (rows past the last document see nothing)."""
    k_lens = q_lens if k_lens is None else k_lens
    prefix = prefix or [0] * len(q_lens)
    Tq = sum(q_lens) if Tq is None else Tq
    lo, hi, at = np.zeros(Tq, int), np.zeros(Tq, int), np.zeros(Tq, int)
    i = k0 = 0
    for nq, nk, p in zip(q_lens, k_lens, prefix):
        for r in range(nq):
            a = k0 + nk - nq + r
            l, h = k0, k0 + nk
            if causal:
                h = min(max(a + 1, k0 + p), k0 + nk)
                if window:
                    l = max(l, a + 1 - window)
            l, h = max(l, 0), max(h, 0)
            lo[i], hi[i], at[i] = (l, h, a) if l < h else (0, 0, a)
            i += 1
        k0 += nk
    return lo, hi, at


def attention(q, k, v, lo, hi, at=None, scale=None, cap=0.0, slopes=None, do=None, dtype="bf16"):
    """q [n, H, dh], k, v [m, Hkv, dh]; returns {name: (value, bound)} for o, lse and, with do, dq, dk, dv."""
    n, H, dh = q.shape
    m, Hkv = k.shape[0], k.shape[1]
    G, u = H // Hkv, HALF[dtype]
    p_round = u if dtype == "bf16" else 0.0
    scale = 1.0 / np.sqrt(dh) if scale is None else scale
    at = np.arange(n) if at is None else at
    j = np.arange(m)
    sees = (j >= np.asarray(lo)[:, None]) & (j < np.asarray(hi)[:, None])
    zero = lambda *s: (np.zeros(s), np.zeros(s))
    out = {"o": zero(n, H, dh), "lse": zero(H, n), "dq": zero(n, H, dh), "dk": zero(m, Hkv, dh), "dv": zero(m, Hkv, dh)}
    for h in range(H):
        qh, kh, vh = q[:, h], k[:, h // G], v[:, h // G]
        # what a query doesn't see stays out of it, whatever it holds
        kz, vz = np.where(np.isfinite(kh), kh, 0.0), np.where(np.isfinite(vh), vh, 0.0)
        qz = np.where(np.isfinite(qh), qh, 0.0)
        z = qz @ kz.T * scale
        e_s = (dh + 8) * E32 * (np.abs(qz) @ np.abs(kz).T) * abs(scale)
        t = np.tanh(z / cap) if cap else 0.0
        s = t * cap if cap else z
        if cap:
            e_s = e_s + (cap * 2.0 ** -21 if dtype == "bf16" and cap <= 4096 else 8 * E32 * np.abs(s))
        if slopes is not None:
            d = np.abs(np.asarray(at)[:, None] - j) * slopes[h]
            s = s - d
            e_s = e_s + 2 * E32 * np.abs(d)
        s = np.where(sees, s, -np.inf)
        top = s.max(1, initial=-np.inf)
        live = top > -np.inf
        p = np.exp(s - np.where(live, top, 0.0)[:, None])
        tot = p.sum(1)
        p = p / np.where(live, tot, 1.0)[:, None]
        with np.errstate(divide="ignore"):
            lse = np.where(live, top + np.log(np.where(live, tot, 1.0)), -np.inf)
        e_s = np.where(sees, e_s, 0.0)
        e_row = e_s.max(1, initial=0.0)
        rel = 2 * e_row[:, None] + (sees.sum(1)[:, None] + 16) * E32 + p_round
        o = p @ vz
        e_o = rel * (p @ np.abs(vz)) + u * np.abs(o)
        out["o"][0][:, h], out["o"][1][:, h] = o, e_o
        out["lse"][0][h] = lse
        out["lse"][1][h] = np.where(live, e_row + (sees.sum(1) + 16) * E32 * (1 + np.abs(np.where(live, lse, 0.0))), 0.0)
        if do is None:
            continue
        g = np.where(np.isfinite(do[:, h]), do[:, h], 0.0)
        D = (o * g).sum(1, keepdims=True)
        e_D = (e_o * np.abs(g)).sum(1, keepdims=True) + (dh + 8) * E32 * (np.abs(o) * np.abs(g)).sum(1, keepdims=True)
        dp = g @ vz.T
        e_dp = (dh + 8) * E32 * (np.abs(g) @ np.abs(vz).T)
        keep = 1 - t * t if cap else 1.0
        ds = p * (dp - D) * keep
        e_ds = (rel + (8 * 2.0 ** -21 if cap else 0.0)) * np.abs(p * (dp - D)) + p * (e_D + e_dp)
        r = lambda a, b: a @ b * scale
        size = lambda a, b: a @ b * abs(scale)              # (of errors: whatever the sign of the scale)
        dq = r(ds, kz)
        out["dq"][0][:, h], out["dq"][1][:, h] = dq, size(e_ds + (m + 8) * E32 * np.abs(ds), np.abs(kz)) + u * np.abs(dq)
        out["dk"][0][:, h // G] += r(ds.T, qz)
        out["dk"][1][:, h // G] += size((e_ds + (n * G + 8) * E32 * np.abs(ds)).T, np.abs(qz))
        out["dv"][0][:, h // G] += p.T @ g
        out["dv"][1][:, h // G] += (p * (rel + (n * G + 8) * E32)).T @ np.abs(g)
    for name in ("dk", "dv"):
        out[name] = (out[name][0], out[name][1] + u * np.abs(out[name][0]))
    return out


def outside(got, want, bound):
    """The largest error as a multiple of its bound (0 where both are the same, infinities among them)."""
    got = np.asarray(got, np.float64)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want) / np.maximum(bound, 1e-30))
    return float(np.where(np.isnan(off), np.inf, off).max(initial=0.0))


def rotary(x, pos, freq, interleaved, magnitude=1.0, transposed=False):
    """x [T, H, dh] float64; turns the first 2 len(freq) columns of every head."""
    y, n = x.copy(), len(freq)
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(freq)[None]
    c, s = (np.cos(a) * magnitude)[:, None], (np.sin(a) * (-magnitude if transposed else magnitude))[:, None]
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    u, w = x[..., first], x[..., second]
    y[..., first], y[..., second] = u * c - w * s, u * s + w * c
    return y


def layernorm(x, gain, bias, eps, dy=None):
    g = 1.0 if gain is None else gain
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    y = xh * g + (0.0 if bias is None else bias)
    if dy is None:
        return y, mean, rstd
    d = dy * g
    dx = rstd[:, None] * (d - d.mean(1, keepdims=True) - xh * (d * xh).mean(1, keepdims=True))
    return y, mean, rstd, dx, (dy * xh).sum(0), dy.sum(0)
