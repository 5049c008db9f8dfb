"""64-bit oracle of the sequence operators (include/rocket.h has the formulas).

Plain numpy loops over series and steps, written from the definitions, with
bounds on what fp32 arithmetic may differ by: every function that has one
returns, beside each result, an array `tol` of the same shape.  A bound runs
the operator's own recurrence on errors: it adds, for every operation, a few
units of 2^-24 of that operation's operands.
"""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24          # half a unit in the last place of fp32, relative
TYPE_U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -126, "bfloat16": 2.0 ** -126, "float16": 2.0 ** -25}
EVERY = 128
_erf = np.vectorize(math.erf)


def rounded(tol, value, dtype: str):
    """A bound after one rounding of a value within tol to dtype."""
    return tol * (1 + TYPE_U[dtype]) + np.abs(value) * TYPE_U[dtype] * 1.0001 + TINY[dtype]


def logistic(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def lengths_of(n, L, lengths):
    return np.full(n, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)


# -------------------------------------------------------------- group norm
def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z * logistic(z)
    if name == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    return z.copy()


def act_slope(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        s = logistic(z)
        return s + z * s * (1.0 - s)
    if name == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return np.ones_like(z)


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, activation="none", lengths=None, dtype="float32"):
    """dict y, mean, rstd and their tolerances (y_tol, mean_tol, rstd_tol)."""
    x = np.asarray(x, np.float64)
    n, L, C = x.shape
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    width = C // groups
    out = dict(y=np.zeros((n, L, C)), mean=np.zeros((n, groups)), rstd=np.zeros((n, groups)))
    out.update({k + "_tol": np.zeros_like(v) for k, v in list(out.items())})
    for i, T in enumerate(lengths_of(n, L, lengths)):
        for g in range(groups if T else 0):
            cs = slice(g * width, (g + 1) * width)
            v = x[i, :T, cs]
            m = v.mean()
            var = ((v - m) ** 2).mean()
            r = 1.0 / math.sqrt(var + eps)
            # a sum of N terms in a tree of chains of at most 256 additions
            m_tol = 256 * U * np.abs(v).mean()
            # squares about a mean that is off by m_tol, summed the same way
            var_tol = 256 * U * var + m_tol ** 2
            r_tol = r * (0.5 * var_tol / (var + eps) + 4 * U)
            out["mean"][i, g], out["rstd"][i, g] = m, r
            out["mean_tol"][i, g], out["rstd_tol"][i, g] = m_tol, r_tol
            xh = (v - m) * r
            z = xh * w[cs] + b[cs]
            z_tol = np.abs(w[cs]) * (r * m_tol + np.abs(v - m) * r_tol + 8 * U * np.abs(xh)) + 8 * U * (
                np.abs(z) + np.abs(b[cs]))
            y = act(z, activation)
            out["y"][i, :T, cs] = y
            # slopes are at most 1.13; the activations' own roundings
            out["y_tol"][i, :T, cs] = 1.2 * z_tol + 8 * U * np.abs(z)
    out["y_tol"] = rounded(out["y_tol"], out["y"], dtype)
    return out


def group_norm_backward(dy, x, groups, mean, rstd, weight=None, bias=None, activation="none", lengths=None,
                        dtype="float32"):
    """dict dx, dweight, dbias and their tolerances, from given mean and rstd."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    mean, rstd = np.asarray(mean, np.float64), np.asarray(rstd, np.float64)
    n, L, C = x.shape
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    b = np.zeros(C) if bias is None else np.asarray(bias, np.float64)
    width = C // groups
    out = dict(dx=np.zeros((n, L, C)), dweight=np.zeros(C), dbias=np.zeros(C))
    out.update({k + "_tol": np.zeros_like(v) for k, v in list(out.items())})
    for i, T in enumerate(lengths_of(n, L, lengths)):
        if not T:
            continue
        m, r = np.repeat(mean[i], width), np.repeat(rstd[i], width)
        xh = (x[i, :T] - m) * r
        z = xh * w + b
        # x - m of given fp32 numbers is rounded to its own size, whatever the level
        xh_tol = 4 * U * np.abs(xh)
        z_tol = np.abs(w) * xh_tol + 4 * U * (np.abs(z) + np.abs(b) + np.abs(xh * w))
        slope = act_slope(z, activation)
        dz = dy[i, :T] * slope
        # second derivatives are below 1; the slopes' own roundings
        dz_tol = np.abs(dy[i, :T]) * (z_tol + 16 * U * (1 + np.abs(z)))
        if activation == "relu":   # the slope jumps where z may change its sign
            dz_tol = np.abs(dy[i, :T]) * (np.abs(z) <= z_tol)
        g, g_tol = dz * w, np.abs(w) * dz_tol + 2 * U * np.abs(dz * w)
        shape = (T, groups, width)

        def mean_of(t):
            return np.repeat(t.reshape(shape).mean(axis=(0, 2)), width)

        mg, mgx = mean_of(g), mean_of(g * xh)
        # sums in chains of at most 256 additions
        mg_tol = mean_of(g_tol) + 256 * U * mean_of(np.abs(g))
        mgx_tol = mean_of(g_tol * np.abs(xh) + np.abs(g) * xh_tol) + 256 * U * mean_of(np.abs(g * xh))
        out["dx"][i, :T] = r * (g - mg - xh * mgx)
        out["dx_tol"][i, :T] = r * (g_tol + mg_tol + np.abs(xh) * mgx_tol + xh_tol * np.abs(mgx)
                                    + 8 * U * (np.abs(g) + np.abs(mg) + np.abs(xh * mgx)))
        out["dbias"] += dz.sum(0)
        out["dweight"] += (dz * xh).sum(0)
        out["dbias_tol"] += dz_tol.sum(0) + 256 * U * np.abs(dz).sum(0)
        out["dweight_tol"] += (dz_tol * np.abs(xh) + np.abs(dz) * xh_tol).sum(0) + 256 * U * np.abs(dz * xh).sum(0)
    out["dx_tol"] = rounded(out["dx_tol"], out["dx"], dtype)
    return out


# -------------------------------------------------------------- recurrence
K = 16   # units of 2^-24 of the operands that a step may add


def recurrence(v, f, o=None, h0=None, lengths=None, dtype="float32"):
    """dict y, h_last, states (before the steps 0, EVERY, ...), all states
    [n, L + 1, C] as "all", and tolerances."""
    v, f = np.asarray(v, np.float64), np.asarray(f, np.float64)
    n, L, C = v.shape
    T = lengths_of(n, L, lengths)
    h = np.zeros((n, C)) if h0 is None else np.asarray(h0, np.float64).copy()
    err = U * np.abs(h)
    every, tols = np.zeros((n, L + 1, C)), np.zeros((n, L + 1, C))
    every[:, 0], tols[:, 0] = h, err
    y, y_tol = np.zeros((n, L, C)), np.zeros((n, L, C))
    for t in range(L):
        on = (T > t)[:, None]
        a, keep = logistic(f[:, t]), logistic(-f[:, t])
        new = a * h + keep * v[:, t]
        new_err = a * err + K * U * (a * np.abs(h) + keep * np.abs(v[:, t]))
        h, err = np.where(on, new, h), np.where(on, new_err, err)
        every[:, t + 1], tols[:, t + 1] = h, err
        q = np.ones_like(h) if o is None else logistic(np.asarray(o, np.float64)[:, t])
        y[:, t] = np.where(on, q * h, 0.0)
        y_tol[:, t] = np.where(on, q * err + K * U * np.abs(q * h), 0.0)
    y_tol = rounded(y_tol, y, dtype)
    return dict(y=y, y_tol=y_tol, h_last=h, h_last_tol=err + TINY["float32"], states=every[:, 0:L:EVERY],
                states_tol=tols[:, 0:L:EVERY] + TINY["float32"], all=every, all_tol=tols)


def recurrence_backward(dy, v, f, o=None, h0=None, dh_last=None, lengths=None, dtype="float32"):
    """dict dv, df, do, dh0 and tolerances."""
    fwd = recurrence(v, f, o, h0, lengths)
    dy, v, f = (np.asarray(t, np.float64) for t in (dy, v, f))
    n, L, C = v.shape
    T = lengths_of(n, L, lengths)
    e = np.zeros((n, C)) if dh_last is None else np.asarray(dh_last, np.float64).copy()
    err = np.zeros((n, C))
    names = ("dv", "df") + (() if o is None else ("do",))
    out = {k: np.zeros((n, L, C)) for k in names}
    out.update({k + "_tol": np.zeros((n, L, C)) for k in names})
    for t in range(L - 1, -1, -1):
        on = (T > t)[:, None]
        a, keep = logistic(f[:, t]), logistic(-f[:, t])
        before, h = fwd["all"][:, t], fwd["all"][:, t + 1]
        before_tol, h_tol = fwd["all_tol"][:, t], fwd["all_tol"][:, t + 1]
        q = np.ones_like(e) if o is None else logistic(np.asarray(o, np.float64)[:, t])
        g = dy[:, t] * q
        dh = g + e
        dh_err = err + K * U * (np.abs(g) + np.abs(e))
        d = before - v[:, t]
        res = dict(dv=dh * keep, df=dh * d * a * keep)
        tol = dict(dv=dh_err * keep + K * U * np.abs(dh * keep),
                   df=a * keep * (dh_err * np.abs(d) + np.abs(dh) * (before_tol + K * U * (
                       np.abs(before) + np.abs(v[:, t])))))
        if o is not None:
            p = logistic(-np.asarray(o, np.float64)[:, t])
            res["do"] = dy[:, t] * h * q * p
            tol["do"] = np.abs(dy[:, t]) * q * p * (h_tol + K * U * (np.abs(h) + a * np.abs(before)
                                                                      + keep * np.abs(v[:, t])))
        for k in names:
            out[k][:, t] = np.where(on, res[k], 0.0)
            out[k + "_tol"][:, t] = np.where(on, tol[k], 0.0)
        e = np.where(on, a * dh, e)
        err = np.where(on, a * dh_err + K * U * np.abs(a * dh), err)
    for k in names:
        out[k + "_tol"] = rounded(out[k + "_tol"], out[k], dtype)
    out["dh0"], out["dh0_tol"] = e, err + TINY["float32"]
    return out


# ----------------------------------------------------------------- dropout
def philox(counter, key, rounds=10):
    """Philox4x32 of Salmon, Moraes, Dror and Shaw (SC 2011) on Python
    integers: four 32-bit words."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_numbers(indices, seed, call):
    """The 16-bit numbers of the given element indices."""
    seed, call = seed % 2 ** 64, call % 2 ** 64
    out, blocks = [], {}
    for i in indices:
        blk = int(i) // 8
        if blk not in blocks:
            blocks[blk] = philox((blk & 0xFFFFFFFF, blk >> 32, call & 0xFFFFFFFF, call >> 32),
                                 (seed & 0xFFFFFFFF, seed >> 32))
        k = int(i) % 8
        out.append(blocks[blk][k // 2] >> (16 * (k % 2)) & 0xFFFF)
    return np.array(out, dtype=np.int64)


def dropout_threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))
