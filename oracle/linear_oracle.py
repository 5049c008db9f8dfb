"""64-bit oracle of the operators around linear layers (include/rocket.h has the
formulas): RMS norm, 8-bit rows and their product, checkpoints and the weight
gradient.

Plain numpy from the definitions, on rows [rows, channels]; `live` says which
rows hold data.  What is defined by single fp32 operations (8-bit values and
their scales, sums rounded to a type) is computed by these and compared for
equality; every other result comes with a bound `*_tol` on what fp32 arithmetic
may differ by: a sum of n terms in any order is off by at most n units U of its
terms' magnitudes, an operation by U of its result.
"""
from __future__ import annotations

import numpy as np

from oracle.sequence_oracle import U, rounded

BLOCK = 128   # rows that share a channel's scale in a checkpoint
PAD = 64      # columns of 8-bit rows come in multiples
F = np.float32


def to_type(a, dtype: str):
    """float32 values rounded to nearest even to dtype, as float32."""
    a = np.asarray(a, F)
    if dtype == "float16":
        return a.astype(np.float16).astype(F)
    if dtype == "bfloat16":
        bits = a.view(np.uint32)
        out = ((bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(F)
        return np.where(np.isfinite(a), out, a).astype(F)
    return a


def pad(channels: int) -> int:
    return -(-channels // PAD) * PAD


def live_rows(n: int, steps: int, lengths) -> np.ndarray:
    t = np.arange(steps)[None, :] < np.clip(np.full(n, steps) if lengths is None else lengths, 0, steps)[:, None]
    return t.reshape(-1)


def _sum_units(C: int) -> float:
    """Roundings that a term of a row's sum meets: at most C / 1024 in a thread of
    a looped row, 32 in one that holds its row, and 40 where threads meet."""
    return C / 1024 + 72


# ---------------------------------------------------------------- RMS norm
def rms_norm(x, weight=None, residual=None, eps=1e-5, live=None, dtype="float32"):
    """dict total, y, rstd with y_tol, rstd_tol."""
    x = np.asarray(x, F)
    rows, C = x.shape
    live = np.ones(rows, bool) if live is None else live
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    total = x if residual is None else to_type(x + np.asarray(residual, F), dtype)
    total = np.where(live[:, None], total, 0)
    s = total.astype(np.float64)
    k = 1.0 / np.sqrt((s * s).sum(1) / C + eps) * live
    k_tol = k * (_sum_units(C) / 2 + 4) * U
    y = s * k[:, None] * w
    y_tol = np.abs(y) * ((_sum_units(C) / 2 + 4) + 3) * U
    return dict(total=total, rstd=k, rstd_tol=k_tol, y=y, y_tol=rounded(y_tol, y, dtype))


def rms_norm_backward(dy, total, rstd, weight=None, dtotal=None, live=None, dtype="float32"):
    """dict dx, dweight with dx_tol, dweight_tol; of the given rstd."""
    dy, s = np.asarray(dy, np.float64), np.asarray(total, np.float64)
    rows, C = s.shape
    live = np.ones(rows, bool) if live is None else live
    dy, s = np.where(live[:, None], dy, 0), np.where(live[:, None], s, 0)
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    k = np.asarray(rstd, np.float64)[:, None] * live[:, None]
    g, xh = dy * w, s * k
    mean = (g * xh).mean(1, keepdims=True)
    mean_tol = np.abs(g * xh).mean(1, keepdims=True) * (_sum_units(C) + 5) * U
    dx = k * (g - xh * mean)
    tol = k * (np.abs(g) * U + np.abs(xh) * mean_tol + np.abs(xh * mean) * U) + 2 * U * np.abs(dx)
    if dtotal is not None:
        dx = dx + np.where(live[:, None], np.asarray(dtotal, np.float64), 0)
        tol = tol + U * np.abs(dx)
    terms = np.abs(dy * xh)
    return dict(dx=dx, dx_tol=rounded(tol * 1.001, dx, dtype), dweight=(dy * xh).sum(0),
                dweight_tol=terms.sum(0) * (rows + 2) * U)


# ------------------------------------------------------------- 8-bit values
def _quotients(v, top, axis):
    """127 / top, one fp32 division, and round(v * that); 0 for tiny or non-finite tops."""
    kept = np.isfinite(top) & (top >= F(2.0 ** -100))
    inverse = np.where(kept, F(127) / np.where(kept, top, F(1)), F(0)).astype(F)
    inv = np.expand_dims(inverse, axis)
    return np.ascontiguousarray(np.where(inv == 0, 0, np.rint(np.where(inv == 0, F(0), v) * inv)), np.int8)


def _steps(top):
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(top), np.where(top >= F(2.0 ** -100), top / F(127), F(0)), F(np.nan)).astype(F)


def _top(v, axis):
    """The largest magnitude, NaN where one is not finite."""
    m = np.abs(v).max(axis=axis, initial=0)
    return np.where(np.isfinite(v).all(axis=axis), m, F(np.nan)).astype(F)


def quantize_rows(x, live=None):
    """(q [rows, padded], scale [rows]) by single fp32 operations."""
    x = np.asarray(x, F)
    live = np.ones(len(x), bool) if live is None else live
    x = np.where(live[:, None], x, F(0))
    top = _top(x, 1)
    q = np.zeros((x.shape[0], pad(x.shape[1])), np.int8)
    q[:, :x.shape[1]] = _quotients(x, top, 1)
    return q, _steps(top)


def linear8(q, scale, wq, wscale, bias=None, live=None, dtype="float32"):
    """(y, y_tol): the sum is exact; its conversion, the scales' product, their
    product and the bias' addition round once each."""
    q, wq = np.asarray(q, np.float64), np.asarray(wq, np.float64)
    s = np.asarray(scale, np.float64)[:, None] * np.asarray(wscale, np.float64)[None, :]
    product = (q @ wq.T) * s
    y = product + (0 if bias is None else np.asarray(bias, np.float64)[None, :])
    tol = 3 * U * np.abs(product) + U * np.abs(y)
    if live is not None:
        y, tol = np.where(live[:, None], y, 0), np.where(live[:, None], tol, 0)
    return y, rounded(tol, y, dtype)


# -------------------------------------------------------------- checkpoints
def checkpoint(x, live=None):
    """(q [blocks, channels, BLOCK], scale [blocks, channels]) by single fp32 operations."""
    x = np.asarray(x, F)
    rows, C = x.shape
    live = np.ones(rows, bool) if live is None else live
    blocks = -(-rows // BLOCK)
    v = np.zeros((blocks * BLOCK, C), F)
    v[:rows] = np.where(live[:, None], x, F(0))
    v = v.reshape(blocks, BLOCK, C).transpose(0, 2, 1)
    top = _top(v, 2)
    return _quotients(v, top, 2), _steps(top)


def restore(q, scale, rows, live=None, dtype="float32"):
    """float32 values of that type."""
    x = (q.astype(F) * np.asarray(scale, F)[:, :, None]).transpose(0, 2, 1).reshape(-1, q.shape[1])[:rows]
    x = to_type(x, dtype)
    return x if live is None else np.where(live[:, None], x, F(0))


def linear_weight_gradient(dy, q, scale, live=None):
    """dict dweight, dbias and their bounds.  The matrix unit may cut off where it
    adds, which counts two units."""
    dy = np.asarray(dy, np.float64)
    rows = dy.shape[0]
    if live is not None:
        dy = np.where(live[:, None], dy, 0)
    x = (q.astype(np.float64) * np.asarray(scale, np.float64)[:, :, None]).transpose(0, 2, 1)
    x = x.reshape(-1, q.shape[1])[:rows]
    units = 2 * min(rows, 3 * BLOCK) + rows / BLOCK + 16
    return dict(dweight=dy.T @ x, dweight_tol=(np.abs(dy).T @ np.abs(x)) * units * U, dbias=dy.sum(0),
                dbias_tol=np.abs(dy).sum(0) * (3 * rows + 2) * U)
