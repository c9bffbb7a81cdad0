"""Plain 64-bit forms of the short causal convolution and the selective state space scan,
token by token, with bounds on what the fp32 kernels may differ by, in the manner of
layer_ref.py.

The reckoning, from the kernels' arithmetic.  One fp32 rounding costs half of EPS = 2^-23
relative.  A logistic function is off by (|v| + 5) EPS relative (the exponent's product,
an ulp each of exponential and reciprocal), its product or slope by 3 EPS more.  A step
size log(1 + e^v) is off by (2 |v| + 8) EPS relative: v's own sum, the exponential, the
logarithm (an ulp) with its product, what rounding 1 + e^v loses, added back, and the sum.  A decay e^(dt A) takes |dt A| times its exponent's error; where
chunks of at most 520 tokens are folded, the exponent is a sum of so many step sizes, 260
EPS more.  An error travels the way its value does, so its bound obeys the value's own
recurrence over magnitudes; regrouping a recurrence into chunks at most doubles it.  A sum of n
terms costs n EPS of the sum of magnitudes, one over 64 lanes and columns (D / 64 + 24) EPS,
one over tokens (T + 64) EPS.  Results in bf16 are rounded once more (layer_ref.excess).
"""

import numpy as np

from layer_ref import EPS, excess  # noqa: F401


def logistic(v):
    with np.errstate(over="ignore"):
        t = np.exp(-np.abs(v))
    return np.where(v > 0, 1 / (1 + t), t / (1 + t))


def silu(v):
    """(value, slope, what the slope's error is relative to)."""
    s = logistic(v)
    return v * s, s * (1 + v * (1 - s)), s * (1 + np.abs(v) * (1 - s))


# --------------------------------------------------------------- convolution
def conv(x, w, b, lens, w0=None, act=True, dy=None, dfinal=None):
    """{"y", "final"} and, from dy, {"dx", "dw", "db", "dw0"}: pairs (value, bound)."""
    T, D = x.shape
    W = w.shape[1]
    N = len(lens)
    out = {"y": (np.zeros((T, D)), np.zeros((T, D))), "final": (np.zeros((N, W - 1, D)), np.zeros((N, W - 1, D)))}
    if dy is not None:
        out.update(dx=(np.zeros((T, D)), np.zeros((T, D))), dw0=(np.zeros((N, W - 1, D)), np.zeros((N, W - 1, D))))
        dw, mw, db, mb = np.zeros((D, W)), np.zeros((D, W)), np.zeros(D), np.zeros(D)
    t = 0
    for n, length in enumerate(lens):
        window = np.zeros((W - 1, D)) if w0 is None else np.asarray(w0[n], np.float64)
        seen = np.concatenate([window, x[t:t + length]])
        out["final"][0][n] = seen[length:]
        p = np.tile(np.zeros(D) if b is None else b, (length, 1))
        m = np.abs(p)
        for j in range(W):
            p = p + seen[j:j + length] * w[:, j]
            m = m + np.abs(seen[j:j + length] * w[:, j])
        ep = (W + 2) * EPS * m
        y, slope, size = silu(p)
        if act:
            out["y"][0][t:t + length] = y
            out["y"][1][t:t + length] = 1.1 * ep + (np.abs(p) + 8) * EPS * np.abs(y)
        else:
            out["y"][0][t:t + length], out["y"][1][t:t + length] = p, ep
        if dy is not None:
            g = dy[t:t + length]
            # |silu''| <= 1/2
            dp = g * slope if act else g
            edp = np.abs(g) * (2 * (np.abs(p) + 8) * EPS * size + 0.5 * ep) if act else np.zeros_like(g)
            dseen, eseen = np.zeros_like(seen), np.zeros_like(seen)
            for j in range(W):
                dseen[j:j + length] += w[:, j] * dp
                eseen[j:j + length] += np.abs(w[:, j]) * (edp + (W + 2) * EPS * np.abs(dp))
                dw[:, j] += (dp * seen[j:j + length]).sum(0)
                mw[:, j] += ((edp + (T + 64) * EPS * np.abs(dp)) * np.abs(seen[j:j + length])).sum(0)
            db += dp.sum(0)
            mb += (edp + (T + 64) * EPS * np.abs(dp)).sum(0)
            if dfinal is not None:
                dseen[length:] += dfinal[n]
                eseen[length:] += EPS * (np.abs(dseen[length:]) + 2 * np.abs(dfinal[n]))
            out["dw0"][0][n], out["dw0"][1][n] = dseen[:W - 1], eseen[:W - 1]
            out["dx"][0][t:t + length], out["dx"][1][t:t + length] = dseen[W - 1:], eseen[W - 1:]
        t += length
    if dy is not None:
        out["dw"], out["db"] = (dw, mw), (db, mb)
    return out


# ---------------------------------------------------------------------- scan
def step_sizes(dt, bias, raw):
    """(step sizes, relative errors, slopes, |v|)."""
    if not raw:
        return dt, np.zeros_like(dt), np.ones_like(dt), np.abs(dt)
    v = dt + (0.0 if bias is None else bias)
    # (a step of zero, from a value of -infinity, is exact)
    size = np.where(np.isfinite(v), np.abs(v), 0.0)
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v))), (2 * size + 8) * EPS, logistic(v), size


def ssm(x, dt, A, B, C, lens, skip=None, z=None, bias=None, s0=None, raw=False, dy=None, dfinal=None):
    """{"y", "final"} and, from dy, {"dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "dbias",
    "ds0"}: pairs (value, bound).  B, C [T, G, S]."""
    T, D = x.shape
    S, G = A.shape[1], B.shape[1]
    group = np.arange(D) // (D // G)
    step, rstep, slope, v = step_sizes(dt, bias, raw)
    Bd, Cd = B[:, group], C[:, group]
    rate = step[..., None] * A
    a = np.exp(rate)
    ga = np.abs(rate) * (rstep[..., None] + 262 * EPS) + 3 * EPS
    u = step * x
    eu = (rstep + EPS) * np.abs(u)
    h, eh = np.zeros((T, D, S)), np.zeros((T, D, S))
    kept, ekept = np.zeros((T, D, S)), np.zeros((T, D, S))  # a_t h_{t-1}
    N = len(lens)
    final, efinal = np.zeros((N, D, S)), np.zeros((N, D, S))
    t = 0
    for n, length in enumerate(lens):
        s = np.zeros((D, S)) if s0 is None else np.asarray(s0[n], np.float64)
        e = np.zeros((D, S))
        for i in range(t, t + length):
            in_ = u[i][:, None] * Bd[i]
            kept[i] = a[i] * s
            ekept[i] = a[i] * e + (ga[i] + EPS) * np.abs(kept[i])
            new = kept[i] + in_
            e = ekept[i] + eu[i][:, None] * np.abs(Bd[i]) + EPS * np.abs(in_) + EPS * np.abs(new)
            s = new
            h[i], eh[i] = s, 2 * e
        final[n], efinal[n] = s, 2 * e
        t += length
    y = (Cd * h).sum(-1)
    my = np.abs(Cd * h).sum(-1)
    ey = (np.abs(Cd) * eh).sum(-1)
    if skip is not None:
        y, my = y + skip * x, my + np.abs(skip * x)
    ey = ey + (S + 6) * EPS * my
    out = {"final": (final, efinal)}
    gate, dgate, size = silu(z) if z is not None else (1.0, 0.0, 0.0)
    kz = (np.abs(z) + 8) * EPS if z is not None else 0.0
    out["y"] = (y * gate, ey * np.abs(gate) + kz * np.abs(y * gate) + EPS * np.abs(y * gate))
    if dy is None:
        return out
    ekept = 2 * ekept
    d = dy * gate
    ed = (kz + EPS) * np.abs(d)
    if z is not None:
        out["dz"] = (dy * y * dgate, np.abs(dy) * (ey * np.abs(dgate) + np.abs(y) * 2 * (kz + EPS) * size))
    dh, edh = np.zeros((T, D, S)), np.zeros((T, D, S))
    ds0, eds0 = np.zeros((N, D, S)), np.zeros((N, D, S))
    t = T
    for n in range(N - 1, -1, -1):
        E = np.zeros((D, S)) if dfinal is None else np.asarray(dfinal[n], np.float64)
        eE = np.zeros((D, S))
        for i in range(t - 1, t - lens[n] - 1, -1):
            in_ = Cd[i] * d[i][:, None]
            dh[i] = E + in_
            err = eE + np.abs(Cd[i]) * ed[i][:, None] + EPS * (np.abs(E) + np.abs(in_))
            edh[i] = 2 * err
            E = a[i] * dh[i]
            eE = a[i] * err + (ga[i] + EPS) * np.abs(E)
        ds0[n], eds0[n] = E, 2 * eE
        t -= lens[n]
    out["ds0"] = (ds0, eds0)
    kl, kt = (D / 64 + 24) * EPS, (T + 64) * EPS
    by_group = lambda q: q.reshape(T, G, D // G, S).sum(2)
    out["dC"] = (by_group(d[..., None] * h),
                 by_group(ed[..., None] * np.abs(h) + np.abs(d)[..., None] * (eh + kl * np.abs(h))))
    out["dB"] = (by_group(dh * u[..., None]),
                 by_group(edh * np.abs(u)[..., None] + np.abs(dh) * (eu + kl * np.abs(u))[..., None]))
    w, mw = (dh * Bd).sum(-1), np.abs(dh * Bd).sum(-1)
    ew = (edh * np.abs(Bd)).sum(-1) + (S + 4) * EPS * mw
    p = dh * kept
    ep = edh * np.abs(kept) + np.abs(dh) * ekept + EPS * np.abs(p)
    ds, ms = (A * p).sum(-1), np.abs(A * p).sum(-1)
    eds = (np.abs(A) * ep).sum(-1) + (S + 6) * EPS * ms
    dstep = x * w + ds
    edstep = np.abs(x) * ew + eds + 3 * EPS * (np.abs(x) * mw + ms)
    dv = dstep * slope
    edv = edstep * slope + ((v + 6) * EPS if raw else 0.0) * np.abs(dv)
    out["ddt"] = (dv, edv)
    dx = step * w + (skip * d if skip is not None else 0.0)
    edx = step * ew + (rstep + 2 * EPS) * np.abs(step * w)
    if skip is not None:
        edx = edx + np.abs(skip) * ed + 2 * EPS * np.abs(skip * d)
        out["dskip"] = ((d * x).sum(0), (np.abs(x) * (ed + kt * np.abs(d))).sum(0))
    out["dx"] = (dx, edx)
    sp = step[..., None]
    out["dA"] = ((sp * p).sum(0), (sp * ep + (rstep[..., None] + kt) * np.abs(sp * p)).sum(0))
    out["dbias"] = (dv.sum(0), (edv + kt * np.abs(dv)).sum(0))
    return out
