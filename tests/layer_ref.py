"""Plain 64-bit forms of the gated linear recurrence and the block norms, token by
token and row by row, with bounds on what the fp32 kernels may differ by.

Every ``*_bound`` follows the same reckoning, made before the kernels ran.  One
fp32 rounding costs half of EPS = 2^-23 relative.  A gate's decay and its
complement are off by (|g| + 5) EPS relative: |g| EPS from the rounded exponent, an
ulp each from the exponential and the reciprocal, and for 1 - e^g beyond the
series up to 5 EPS by cancellation.  An error then travels the way its value
does, so its bound obeys the value's own recurrence or formula over magnitudes;
the kernels' regrouping of a recurrence into tiles at most doubles it.  A sum of n
terms costs (n / 64 + 24) EPS times the sum of magnitudes (64 partial sums at
least, then a tree and a few products), one over rows (rows + 64) EPS.  bf16
results are rounded once more, 2^-8 relative at most.
"""

import numpy as np

EPS = 2.0 ** -23
ROUND = {"bf16": 2.0 ** -8, "f32": EPS}


def gate(g, raw):
    """(a, 1 - a, d log a / d gate)."""
    with np.errstate(over="ignore"):
        if raw:
            t = np.exp(-np.abs(g))
            r = 1.0 / (1.0 + t)
            a, f = np.where(g > 0, t * r, r), np.where(g > 0, r, t * r)
            return a, f, -f
        return np.exp(g), -np.expm1(g), np.ones_like(g)


def glr(x, g, lens, s0=None, raw=False, convex=False, dh=None, dfinal=None):
    """Values and error bounds: {"h", "final"} and, from dh, {"dx", "dg", "ds0"}; each a
    pair (value, bound without the result's own rounding)."""
    x, g = np.asarray(x, np.float64), np.asarray(g, np.float64)
    T, D = x.shape
    a, f, slope = gate(g, raw)
    w = f if convex else np.ones_like(a)
    ga = (np.where(np.isfinite(g), np.abs(g), 0.0) + 5) * EPS
    out = {k: (np.zeros((T, D)), np.zeros((T, D))) for k in ("h", "dx", "dg")}
    out.update({k: (np.zeros((len(lens), D)), np.zeros((len(lens), D))) for k in ("final", "ds0")})
    prev, eprev = np.zeros((T, D)), np.zeros((T, D))
    t = 0
    with np.errstate(invalid="ignore", over="ignore"):
        for n, length in enumerate(lens):
            s = np.zeros(D) if s0 is None else np.asarray(s0[n], np.float64)
            e = np.zeros(D)
            for i in range(t, t + length):
                prev[i], eprev[i] = s, e
                new = a[i] * s + w[i] * x[i]
                e = a[i] * e + (ga[i] + EPS) * (a[i] * np.abs(s) + w[i] * np.abs(x[i])) + EPS * np.abs(new)
                s = new
                out["h"][0][i], out["h"][1][i] = s, 2 * e
            out["final"][0][n], out["final"][1][n] = s, 2 * e
            if dh is not None:
                q = np.zeros(D) if dfinal is None else np.asarray(dfinal[n], np.float64)
                eq = np.zeros(D)
                for i in range(t + length - 1, t - 1, -1):
                    d = dh[i] + q
                    ed = eq + EPS * (np.abs(dh[i]) + np.abs(q))
                    q = a[i] * d
                    eq = a[i] * ed + (ga[i] + EPS) * np.abs(q)
                    u = prev[i] - x[i] if convex else prev[i]
                    mu = np.abs(prev[i]) + (np.abs(x[i]) if convex else 0.0)
                    out["dx"][0][i] = w[i] * d
                    out["dx"][1][i] = 2 * (w[i] * ed + (ga[i] + EPS) * np.abs(w[i] * d))
                    out["dg"][0][i] = slope[i] * q * u
                    out["dg"][1][i] = np.abs(slope[i]) * (2 * eq * mu + 2 * np.abs(q) * eprev[i] +
                                                          (ga[i] + 4 * EPS) * np.abs(q) * mu)
                out["ds0"][0][n], out["ds0"][1][n] = q, 2 * eq
            t += length
    return out


def _sum(v):
    return v.sum(-1, keepdims=True)


def add_norm(x, res, w, scale, post, eps):
    """(y, r') with bounds."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    D = x.shape[1]
    k = (D / 64 + 24) * EPS
    rx = 1 / np.sqrt(_sum(x * x) / D + eps) if post is not None else 1.0
    u = x * rx * (post if post is not None else 1.0)
    res = np.zeros_like(x) if res is None else np.asarray(res, np.float64)
    r = res + scale * u
    er = k * (np.abs(res) + np.abs(scale * u)) if post is not None else 2 * EPS * (np.abs(res) + np.abs(scale * u))
    rr = 1 / np.sqrt(_sum(r * r) / D + eps)
    y = r * rr * w
    # an error er of r reaches y directly and through the root mean square
    ey = np.abs(w) * rr * (er + np.abs(r) * rr * rr * _sum(np.abs(r) * er) / D) + k * np.abs(y)
    return {"y": (y, ey), "res": (r, er)}


def _norm_back(x, r, g, k):
    """Gradient of x r g's sum through r = 1 / rms(x), and its bound, for an incoming
    weight-multiplied gradient g known to within k of its magnitude."""
    D = x.shape[1]
    d = r * (g - x * (r * r * _sum(x * g) / D))
    m = r * (np.abs(g) + np.abs(x) * (r * r * _sum(np.abs(x * g)) / D))
    return d, 3 * k * m, m


def add_norm_back(dy, dres, res, x, w, scale, post, eps):
    dy, res = np.asarray(dy, np.float64), np.asarray(res, np.float64)
    T, D = dy.shape
    k, kt = (D / 64 + 24) * EPS, (T + 64) * EPS
    rr = 1 / np.sqrt(_sum(res * res) / D + eps)
    d, ed, m = _norm_back(res, rr, w * dy, k)
    if dres is not None:
        d, m = d + dres, m + np.abs(dres)
        ed = ed + EPS * np.abs(dres)
    out = {"dres": (d, ed), "dw": ((dy * res * rr).sum(0), (kt + k) * np.abs(dy * res * rr).sum(0))}
    du, mu = scale * d, np.abs(scale) * m
    if x is None:
        out["dx"] = (du, np.abs(scale) * ed + EPS * mu)
        return out
    x = np.asarray(x, np.float64)
    if post is None:
        out["dx"] = (du, np.abs(scale) * ed + EPS * mu)
        out["dscale"] = ((d * x).sum(0), (kt + 4 * k) * (m * np.abs(x)).sum(0))
        return out
    rx = 1 / np.sqrt(_sum(x * x) / D + eps)
    xn = x * rx
    out["dscale"] = ((d * xn * post).sum(0), (kt + 8 * k) * (m * np.abs(xn * post)).sum(0))
    out["dpost"] = ((du * xn).sum(0), (kt + 8 * k) * (mu * np.abs(xn)).sum(0))
    dx = _norm_back(x, rx, post * du, k)[0]
    out["dx"] = (dx, 8 * k * _norm_back(x, rx, np.abs(post) * mu, k)[2])
    return out


def act(z, silu):
    t = np.exp(-np.abs(z))
    s = np.where(z > 0, 1 / (1 + t), t / (1 + t))
    return (z * s, s * (1 + z * (1 - s))) if silu else (s, s * (1 - s))


def gate_norm(o, z, w, silu, eps, dy=None):
    """{"y"} or, from dy, {"do", "dz", "dw"}, with bounds; o, z, dy [rows, d]."""
    o, z = np.asarray(o, np.float64), np.asarray(z, np.float64)
    rows, d = o.shape
    kz = (np.abs(z) + 8) * EPS  # of an activation or its slope, relative to 1 + |z|
    k = (d / 64 + 24) * EPS
    r = 1 / np.sqrt(_sum(o * o) / d + eps)
    f, df = act(z, silu)
    n = o * r * w
    if dy is None:
        return {"y": (n * f, (k + 2 * kz) * np.abs(n * f))}
    dy = np.asarray(dy, np.float64)
    dn = dy * f
    do, edo, m = _norm_back(o, r, w * dn, k + 2 * kz.max())
    mag = np.abs(dy * n)
    return {"do": (do, edo), "dz": (dy * n * df, k * mag * np.abs(df) + 4 * kz * mag * (1 + np.abs(z))),
            "dw": ((dn * o * r).sum(0), ((rows + 64) * EPS + k + 2 * kz.max()) * np.abs(dn * o * r).sum(0))}


def excess(got, want, dtype):
    """How far got is beyond its bound, as a multiple of it (<= 1: inside).  got: a
    tensor; want: a pair (value, bound).  NaN and infinities must agree."""
    v, b = want
    got = got.detach().double().cpu().numpy().reshape(v.shape)
    tiny = 2.0 ** -126  # results below the least normal number may be flushed
    limit = b + ROUND[dtype] * np.abs(v) + tiny
    same = np.isfinite(v)
    assert np.array_equal(np.isfinite(got), same), "finite and other values differ in place"
    assert np.array_equal(np.isnan(got), np.isnan(v)), "NaN in other places"
    with np.errstate(invalid="ignore"):
        off = np.where(same, np.abs(got - v) / limit, 0.0)
    return float(off.max()) if off.size else 0.0
