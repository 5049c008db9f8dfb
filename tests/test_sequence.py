"""Sequence operators without a GPU: the 64-bit oracle against published
vectors and against differences, the C ABI's refusals (all before any device
work) and the Python binding's."""
import ctypes
import os

import numpy as np
import pytest

from oracle import sequence_oracle as so
from paper_2601_17091_amd import rocket as rb

DUMMY = 0x10000   # never dereferenced: every call below is refused, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rb.LIB_PATH):
        from paper_2601_17091_amd import build_lib
        build_lib.build()
    return rb.library()


# ------------------------------------------------------------------ oracle
def test_philox_published_vectors():
    """The known answers published with the generator."""
    ones = 0xFFFFFFFF
    assert so.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert so.philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert so.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def _difference(fn, x, d, h=1e-5):
    return (fn(x + h * d) - fn(x - h * d)) / (2 * h)


@pytest.mark.parametrize("activation", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("lengths", [None, [3, 0, 5]])
def test_oracle_group_norm_gradient_is_the_difference(activation, lengths):
    rng = np.random.default_rng(5)
    n, L, C, G = 3, 5, 6, 2
    x, dy = rng.standard_normal((n, L, C)) + 0.5, rng.standard_normal((n, L, C))
    w, b = rng.standard_normal(C), rng.standard_normal(C)
    if lengths is not None:
        for i, t in enumerate(lengths):
            dy[i, t:] = 0.0

    def loss(x, w, b):
        return (so.group_norm(x, G, w, b, activation=activation, lengths=lengths)["y"] * dy).sum()

    f = so.group_norm(x, G, w, b, activation=activation, lengths=lengths)
    g = so.group_norm_backward(dy, x, G, f["mean"], f["rstd"], w, b, activation=activation, lengths=lengths)
    for _ in range(4):
        d = rng.standard_normal(x.shape)
        assert abs(_difference(lambda t: loss(t, w, b), x, d) - (g["dx"] * d).sum()) < 1e-6
        dc = rng.standard_normal(C)
        assert abs(_difference(lambda t: loss(x, t, b), w, dc) - (g["dweight"] * dc).sum()) < 1e-6
        assert abs(_difference(lambda t: loss(x, w, t), b, dc) - (g["dbias"] * dc).sum()) < 1e-6


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("lengths", [None, [4, 0, 7]])
def test_oracle_recurrence_gradient_is_the_difference(gate, lengths):
    rng = np.random.default_rng(6)
    n, L, C = 3, 7, 4
    v, f, o, dy = (rng.standard_normal((n, L, C)) for _ in range(4))
    h0, dl = rng.standard_normal((n, C)), rng.standard_normal((n, C))

    def loss(v, f, o, h0):
        r = so.recurrence(v, f, o if gate else None, h0, lengths)
        return (r["y"] * dy).sum() + (r["h_last"] * dl).sum()

    g = so.recurrence_backward(dy, v, f, o if gate else None, h0, dl, lengths)
    d = rng.standard_normal((n, L, C))
    assert abs(_difference(lambda t: loss(t, f, o, h0), v, d) - (g["dv"] * d).sum()) < 1e-7
    assert abs(_difference(lambda t: loss(v, t, o, h0), f, d) - (g["df"] * d).sum()) < 1e-7
    if gate:
        assert abs(_difference(lambda t: loss(v, f, t, h0), o, d) - (g["do"] * d).sum()) < 1e-7
    d0 = rng.standard_normal((n, C))
    assert abs(_difference(lambda t: loss(v, f, o, t), h0, d0) - (g["dh0"] * d0).sum()) < 1e-7


# ---------------------------------------------------------------- refusals
def shape(n=2, steps=5, channels=8, dtype=0, lengths=None):
    return rb.CSequenceShape(n, steps, channels, dtype, lengths)


def seq(data=DUMMY, series=40, step=8):
    return rb.CSequence(data, series, step)


def norm(lib, s=None, groups=2, x=None, w=None, b=None, eps=1e-5, act=0, y=None, mean=DUMMY, rstd=DUMMY, ws=DUMMY,
         size=1 << 40):
    p = ctypes.byref
    return lib.rocket_group_norm_forward(p(s or shape()), groups, p(x or seq()), w, b, eps, act, p(y or seq()), mean,
                                         rstd, ws, size, None)


BAD_SHAPES = [dict(n=-1), dict(steps=-1), dict(channels=0), dict(dtype=3), dict(dtype=-1), dict(n=2 ** 31),
              dict(steps=2 ** 31), dict(channels=2 ** 24 + 1), dict(n=2 ** 30, steps=2 ** 30)]
# outputs that would overlap themselves, or whose address is no element's
BAD_OUTPUTS = [seq(step=7), seq(series=7, step=8), seq(series=16, step=8), seq(data=DUMMY + 1), seq(data=None),
               seq(step=-8), seq(series=2 ** 60)]
BAD_INPUTS = [seq(data=DUMMY + 2), seq(data=None), seq(step=-8), seq(series=-40), seq(series=2 ** 60)]


@pytest.mark.parametrize("over", BAD_SHAPES)
def test_refused_shapes(lib, over):
    s = shape(**over)
    size = ctypes.c_int64()
    assert norm(lib, s) == rb.ROCKET_ERR_INVALID_ARG
    assert lib.rocket_group_norm_workspace(ctypes.byref(s), 1, 0, ctypes.byref(size)) == rb.ROCKET_ERR_INVALID_ARG
    assert lib.rocket_recurrence_workspace(ctypes.byref(s), ctypes.byref(size)) == rb.ROCKET_ERR_INVALID_ARG
    assert rec(lib, s) == rb.ROCKET_ERR_INVALID_ARG
    assert rec_back(lib, s) == rb.ROCKET_ERR_INVALID_ARG
    assert norm_back(lib, s) == rb.ROCKET_ERR_INVALID_ARG


def norm_back(lib, s=None, groups=2, dy=None, x=None, act=0, mean=DUMMY, rstd=DUMMY, dx=None, dw=None, db=None,
              ws=DUMMY, size=1 << 40):
    p = ctypes.byref
    return lib.rocket_group_norm_backward(p(s or shape()), groups, p(dy or seq()), p(x or seq()), None, None, act,
                                          mean, rstd, p(dx or seq()), dw, db, ws, size, None)


def rec(lib, s=None, v=None, f=None, o=None, h0=None, y=None, h_last=DUMMY, states=None, ws=DUMMY, size=1 << 40):
    p = ctypes.byref
    return lib.rocket_recurrence_forward(p(s or shape()), p(v or seq()), p(f or seq()), p(o) if o else None, h0,
                                         p(y or seq()), h_last, states, ws, size, None)


def rec_back(lib, s=None, dy=None, v=None, f=None, o=None, states=DUMMY, dh_last=None, dv=None, df=None, do=None,
             dh0=DUMMY, ws=DUMMY, size=1 << 40):
    p = ctypes.byref
    return lib.rocket_recurrence_backward(p(s or shape()), p(dy or seq()), p(v or seq()), p(f or seq()),
                                          p(o) if o else None, states, dh_last, p(dv or seq()), p(df or seq()),
                                          p(do) if do else None, dh0, ws, size, None)


@pytest.mark.parametrize("k", range(len(BAD_OUTPUTS)))
def test_refused_outputs(lib, k):
    bad = BAD_OUTPUTS[k]
    for st in (norm(lib, y=bad), norm_back(lib, dx=bad), rec(lib, y=bad), rec_back(lib, dv=bad),
               rec_back(lib, df=bad), rec_back(lib, o=seq(), do=bad)):
        assert st == rb.ROCKET_ERR_INVALID_ARG


@pytest.mark.parametrize("k", range(len(BAD_INPUTS)))
def test_refused_inputs(lib, k):
    bad = BAD_INPUTS[k]
    for st in (norm(lib, x=bad), norm_back(lib, x=bad), norm_back(lib, dy=bad), rec(lib, v=bad), rec(lib, f=bad),
               rec(lib, o=bad), rec_back(lib, dy=bad), rec_back(lib, v=bad), rec_back(lib, f=bad),
               rec_back(lib, o=bad, do=seq())):
        assert st == rb.ROCKET_ERR_INVALID_ARG


def test_refused_group_norm_arguments(lib):
    INV = rb.ROCKET_ERR_INVALID_ARG
    for groups in (0, -1, 3, 9, 16):
        assert norm(lib, groups=groups) == INV and norm_back(lib, groups=groups) == INV
    for act in (-1, 4):
        assert norm(lib, act=act) == INV and norm_back(lib, act=act) == INV
    for eps in (-1e-5, float("nan"), float("inf")):
        assert norm(lib, eps=eps) == INV
    for miss in (dict(mean=None), dict(rstd=None), dict(mean=DUMMY + 2), dict(rstd=DUMMY + 1)):
        assert norm(lib, **miss) == INV and norm_back(lib, **miss) == INV
    assert norm(lib, w=DUMMY + 2) == INV and norm(lib, b=DUMMY + 2) == INV
    assert norm(lib, s=shape(lengths=DUMMY + 2)) == INV
    assert norm_back(lib, dw=DUMMY + 2) == INV and norm_back(lib, db=DUMMY + 2) == INV
    assert lib.rocket_group_norm_forward(None, 1, None, None, None, 0.0, 0, None, None, None, None, 0, None) == INV
    # a series longer than a workgroup holds needs a workspace; so does any gradient
    long = shape(steps=100000)
    size = ctypes.c_int64()
    assert lib.rocket_group_norm_workspace(ctypes.byref(long), 2, 0, ctypes.byref(size)) == rb.ROCKET_OK
    assert size.value > 0
    wide = seq(series=800000)
    assert norm(lib, s=long, x=wide, y=wide, size=size.value - 1) == INV
    assert norm(lib, s=long, x=wide, y=wide, size=size.value, ws=None) == INV
    assert norm(lib, s=long, x=wide, y=wide, size=size.value, ws=DUMMY + 4) == INV
    assert lib.rocket_group_norm_workspace(ctypes.byref(shape()), 2, 0, ctypes.byref(size)) == rb.ROCKET_OK
    assert size.value == 0
    assert lib.rocket_group_norm_workspace(ctypes.byref(shape()), 2, 1, ctypes.byref(size)) == rb.ROCKET_OK
    assert size.value > 0
    assert norm_back(lib, size=size.value - 1) == INV
    assert lib.rocket_group_norm_workspace(ctypes.byref(shape()), 2, 0, None) == INV


def test_refused_recurrence_arguments(lib):
    INV = rb.ROCKET_ERR_INVALID_ARG
    assert rec(lib, h_last=None) == INV
    assert rec(lib, h_last=DUMMY + 2) == INV and rec(lib, h0=DUMMY + 2) == INV and rec(lib, states=DUMMY + 2) == INV
    assert rec_back(lib, dh0=None) == INV and rec_back(lib, states=None) == INV
    assert rec_back(lib, dh_last=DUMMY + 2) == INV
    assert rec_back(lib, o=seq()) == INV and rec_back(lib, do=seq()) == INV   # both or neither
    long, wide, size = shape(steps=100000), seq(series=800000), ctypes.c_int64()
    assert lib.rocket_recurrence_workspace(ctypes.byref(long), ctypes.byref(size)) == rb.ROCKET_OK
    assert size.value > 0
    for ws, n in ((DUMMY, size.value - 1), (None, size.value), (DUMMY + 4, size.value)):
        assert rec(lib, s=long, v=wide, f=wide, y=wide, ws=ws, size=n) == INV
        assert rec_back(lib, s=long, dy=wide, v=wide, f=wide, dv=wide, df=wide, ws=ws, size=n) == INV
    assert lib.rocket_recurrence_workspace(ctypes.byref(long), None) == INV
    assert lib.rocket_recurrence_workspace(None, ctypes.byref(size)) == INV


def step(lib, n=2, C=8, dtype=0, v=DUMMY, vs=8, f=DUMMY, fs=8, o=None, os_=8, h=DUMMY, h_out=DUMMY, y=DUMMY, ys=8):
    return lib.rocket_recurrence_step(n, C, dtype, v, vs, f, fs, o, os_, h, h_out, y, ys, None)


@pytest.mark.parametrize("over", [dict(n=-1), dict(C=0), dict(dtype=5), dict(v=None), dict(f=None), dict(y=None),
                                  dict(h=None), dict(h_out=None), dict(v=DUMMY + 1), dict(o=DUMMY + 1),
                                  dict(ys=7), dict(vs=-1), dict(h=DUMMY + 2)])
def test_refused_steps(lib, over):
    assert step(lib, **over) == rb.ROCKET_ERR_INVALID_ARG


def drop(lib, x=DUMMY, r=None, y=DUMMY, rows=2, cols=8, xs=8, rs=8, ys=8, dtype=0, p=0.5):
    return lib.rocket_dropout(x, r, y, rows, cols, xs, rs, ys, dtype, p, 1, 0, None)


@pytest.mark.parametrize("over", [dict(p=-0.1), dict(p=1.1), dict(p=float("nan")), dict(rows=-1), dict(cols=-1),
                                  dict(dtype=7), dict(x=None), dict(y=None), dict(x=DUMMY + 2), dict(r=DUMMY + 1),
                                  dict(xs=7), dict(ys=7), dict(r=DUMMY, rs=7), dict(rows=2 ** 31, cols=2 ** 31),
                                  dict(rows=2 ** 40, cols=2 ** 40, xs=2 ** 40, ys=2 ** 40)])
def test_refused_dropout(lib, over):
    assert drop(lib, **over) == rb.ROCKET_ERR_INVALID_ARG


def test_nothing_to_do_touches_nothing(lib):
    """No series (or no elements): accepted without a device."""
    none = rb.CSequence(None, 0, 0)
    assert norm(lib, s=shape(n=0), x=none, y=none, mean=None, rstd=None, ws=None, size=0) == rb.ROCKET_OK
    assert rec(lib, s=shape(n=0), v=none, f=none, y=none, h_last=None, ws=None, size=0) == rb.ROCKET_OK
    assert rec_back(lib, s=shape(n=0), dy=none, v=none, f=none, dv=none, df=none, states=None, dh0=None) == rb.ROCKET_OK
    assert step(lib, n=0, v=None, f=None, h=None, h_out=None, y=None) == rb.ROCKET_OK
    assert drop(lib, rows=0, x=None, y=None) == rb.ROCKET_OK
    assert drop(lib, cols=0, x=None, y=None) == rb.ROCKET_OK


def test_binding_refuses_host_tensors(lib):
    import torch

    from paper_2601_17091_amd import sequence
    x, h = torch.zeros(2, 3, 4), torch.zeros(2, 4)
    for call in (lambda: sequence.group_norm(x, 2), lambda: sequence.group_norm_backward(x, x, 2, h, h),
                 lambda: sequence.recurrence(x, x), lambda: sequence.recurrence_backward(x, x, x, h),
                 lambda: sequence.recurrence_step(h, h, h), lambda: sequence.dropout(x, 0.5, 1),
                 lambda: sequence.dropout_backward(x, 0.5, 1)):
        with pytest.raises(TypeError):
            call()
    assert sequence.EVERY == so.EVERY == 128


def test_package_imports_without_torch():
    """The generator, planner and fit do not wait for torch; `sequence` brings it."""
    import subprocess
    import sys
    code = ("import sys, paper_2601_17091_amd as rk; rk.library(); assert 'torch' not in sys.modules; "
            "rk.sequence.EVERY; assert 'torch' in sys.modules")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([sys.executable, "-c", code], cwd=root, check=True)
