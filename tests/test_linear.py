"""Operators around linear layers without a GPU: the 64-bit oracle against
differences and worked values, the C ABI's refusals (all before any device work)
and the Python binding's."""
import ctypes
import os

import numpy as np
import pytest

from oracle import linear_oracle as lo
from paper_2601_17091_amd import rocket as rb

DUMMY = 0x10000   # never dereferenced: every call below is refused, or has nothing to do
INV = rb.ROCKET_ERR_INVALID_ARG
byref = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rb.LIB_PATH):
        from paper_2601_17091_amd import build_lib
        build_lib.build()
    return rb.library()


# ------------------------------------------------------------------ oracle
@pytest.mark.parametrize("weighted", [False, True])
def test_oracle_rms_norm_gradient_is_the_difference(weighted):
    rng = np.random.default_rng(3)
    s, dy, dt = (rng.standard_normal((4, 7)) for _ in range(3))
    w = 1 + 0.3 * rng.standard_normal(7) if weighted else np.ones(7)
    live = np.array([True, True, False, True])

    def loss(s, w):
        k = 1 / np.sqrt((s * s).mean(1, keepdims=True) + 1e-5)
        return ((s * k * w * dy + s * dt) * live[:, None]).sum()

    k = 1 / np.sqrt((s * s).mean(1) + 1e-5)
    g = lo.rms_norm_backward(dy, s, k, w, dt, live)
    for _ in range(4):
        d, e, h = rng.standard_normal(s.shape), rng.standard_normal(7), 1e-5
        assert abs((loss(s + h * d, w) - loss(s - h * d, w)) / (2 * h) - (g["dx"] * d).sum()) < 1e-7
        assert abs((loss(s, w + h * e) - loss(s, w - h * e)) / (2 * h) - (g["dweight"] * e).sum()) < 1e-7
    assert (g["dx"][2] == 0).all()


def test_oracle_rounding():
    a = np.array([1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8 - 2.0 ** -20, np.inf, np.nan, 3e38], np.float32)
    want = [1.0, 1.0, 1 + 4 * 2.0 ** -8, -1 - 2.0 ** -7, np.inf, np.nan]
    assert np.array_equal(lo.to_type(a, "bfloat16")[:6], np.array(want, np.float32), equal_nan=True)
    assert np.array_equal(lo.to_type(a[:4], "float16"), a[:4].astype(np.float16).astype(np.float32))


def test_oracle_8_bit_values():
    """127 at the largest, ties to even, zeros past the channels; rows that hold
    nothing finite or nothing at all."""
    x = np.array([[127, 0.5, 1.5, -2.5, -127], [254, 1, -3, 0, 5], [0, 0, 0, 0, 0], [1, np.nan, 0, 0, 0],
                  [1, np.inf, 0, 0, 0], [1e-38, 0, 0, 0, 0]], np.float32)
    q, scale = lo.quantize_rows(x)
    assert q.shape == (6, 64) and (q[:, 5:] == 0).all()
    assert q[0, :5].tolist() == [127, 0, 2, -2, -127] and q[1, :5].tolist() == [127, 0, -2, 0, 2]
    assert (q[2:] == 0).all()
    assert scale[:3].tolist() == [1, 2, 0] and np.isnan(scale[3:5]).all() and scale[5] == 0
    kq, ks = lo.checkpoint(x.T)
    assert kq.shape == (1, 6, 128) and (kq[0, :, 5:] == 0).all() and (kq[0, :, :5] == q[:, :5]).all()
    assert np.array_equal(ks[0], scale, equal_nan=True)
    back = lo.restore(kq, ks, 5)
    assert np.array_equal(back[:, 0], [127, 0, 2, -2, -127])
    r = np.random.default_rng(1).standard_normal((300, 9)).astype(np.float32)
    kq, ks = lo.checkpoint(r, np.arange(300) != 7)
    assert kq.shape == (3, 9, 128)
    apart = np.abs(lo.restore(kq, ks, 300) - r)
    assert (apart[np.arange(300) != 7] <= np.repeat(ks, 128, 0)[:300][np.arange(300) != 7] * 0.5001).all()


def test_oracle_weight_gradient_is_the_product():
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((200, 6)).astype(np.float32), rng.standard_normal((200, 3))
    live = rng.random(200) < 0.7
    q, s = lo.checkpoint(x, live)
    g = lo.linear_weight_gradient(dy, q, s, live)
    assert np.allclose(g["dweight"], (dy * live[:, None]).T @ lo.restore(q, s, 200), atol=1e-5)
    assert np.allclose(g["dbias"], (dy * live[:, None]).sum(0))


# ---------------------------------------------------------------- refusals
def shape(n=2, steps=5, channels=8, dtype=0, lengths=None):
    return rb.CSequenceShape(n, steps, channels, dtype, lengths)


def seq(data=DUMMY, series=40, step=8):
    return rb.CSequence(data, series, step)


def opt(s):
    return None if s is None else byref(s)


def norm(lib, s=None, x=None, r=None, w=None, eps=1e-5, y=None, total=None, rstd=DUMMY):
    return lib.rocket_rms_norm_forward(byref(s or shape()), byref(x or seq()), opt(r), w, eps, byref(y or seq()),
                                       opt(total), rstd, None)


def norm8(lib, s=None, x=None, r=None, w=None, eps=1e-5, q=DUMMY, scale=DUMMY, total=None, rstd=DUMMY):
    return lib.rocket_rms_norm_bytes_forward(byref(s or shape()), byref(x or seq()), opt(r), w, eps, q, scale, opt(total),
                                        rstd, None)


def norm_back(lib, s=None, dy=None, t=None, w=None, rstd=DUMMY, dt=None, dx=None, dw=DUMMY, ws=DUMMY, size=1 << 40):
    return lib.rocket_rms_norm_backward(byref(s or shape()), byref(dy or seq()), byref(t or seq()), w, rstd, opt(dt),
                                        byref(dx or seq()), dw, ws, size, None)


def quantize(lib, s=None, x=None, q=DUMMY, scale=DUMMY):
    return lib.rocket_quantize_rows(byref(s or shape()), byref(x or seq()), q, scale, None)


def product(lib, s=None, columns=64, q=DUMMY, scale=DUMMY, w=DUMMY, ws=DUMMY, bias=None, y=None, at=DUMMY,
            size=1 << 40):
    return lib.rocket_linear_bytes(byref(s or shape()), columns, q, scale, w, ws, bias, byref(y or seq()), at, size, None)


def keep(lib, s=None, x=None, q=DUMMY, scale=DUMMY):
    return lib.rocket_checkpoint(byref(s or shape()), byref(x or seq()), q, scale, None)


def restore(lib, s=None, q=DUMMY, scale=DUMMY, x=None):
    return lib.rocket_restore(byref(s or shape()), q, scale, byref(x or seq()), None)


def gradient(lib, s=None, channels=16, dy=None, q=DUMMY, scale=DUMMY, dw=DUMMY, db=DUMMY, ws=DUMMY, size=1 << 40):
    return lib.rocket_linear_weight_gradient(byref(s or shape()), channels, byref(dy or seq()), q, scale, dw, db, ws,
                                             size, None)


ALL = (norm, norm8, norm_back, quantize, product, keep, restore, gradient)
BAD_SHAPES = [dict(n=-1), dict(steps=-1), dict(channels=0), dict(dtype=3), dict(dtype=-1), dict(n=2 ** 31),
              dict(steps=2 ** 31), dict(channels=2 ** 24 + 1), dict(n=2 ** 30, steps=2 ** 30)]
BAD_OUTPUTS = [seq(step=7), seq(series=7, step=8), seq(series=16, step=8), seq(data=DUMMY + 1), seq(data=None),
               seq(step=-8), seq(series=2 ** 60)]
BAD_INPUTS = [seq(data=DUMMY + 2), seq(data=None), seq(step=-8), seq(series=-40), seq(series=2 ** 60)]


@pytest.mark.parametrize("over", BAD_SHAPES)
@pytest.mark.parametrize("call", ALL)
def test_refused_shapes(lib, call, over):
    assert call(lib, shape(**over)) == INV


@pytest.mark.parametrize("over", BAD_SHAPES)
def test_refused_workspace_shapes(lib, over):
    size, s = ctypes.c_int64(), shape(**over)
    assert lib.rocket_rms_norm_workspace(byref(s), byref(size)) == INV
    assert lib.rocket_linear_bytes_workspace(byref(s), 64, byref(size)) == INV
    assert lib.rocket_linear_weight_gradient_workspace(byref(s), 64, byref(seq()), byref(size)) == INV


@pytest.mark.parametrize("bad", BAD_OUTPUTS)
def test_refused_outputs(lib, bad):
    for st in (norm(lib, y=bad), norm(lib, r=seq(), total=bad), norm8(lib, r=seq(), total=bad), norm_back(lib, dx=bad),
               product(lib, y=bad), restore(lib, x=bad)):
        assert st == INV


@pytest.mark.parametrize("bad", BAD_INPUTS)
def test_refused_inputs(lib, bad):
    for st in (norm(lib, x=bad), norm(lib, r=bad, total=seq()), norm8(lib, x=bad), norm8(lib, r=bad, total=seq()),
               norm_back(lib, dy=bad), norm_back(lib, t=bad), norm_back(lib, dt=bad), quantize(lib, x=bad),
               keep(lib, x=bad), gradient(lib, dy=bad)):
        assert st == INV


def test_refused_operands(lib):
    nan, inf = float("nan"), float("inf")
    for call in (norm, norm8):
        for over in (dict(r=seq()), dict(total=seq()), dict(rstd=None), dict(w=DUMMY + 1), dict(eps=-1e-9),
                     dict(eps=nan), dict(eps=inf)):
            assert call(lib, **over) == INV
    for call in (norm8, quantize, keep, restore, gradient, product):
        for over in (dict(q=None), dict(q=DUMMY + 8), dict(scale=None), dict(scale=DUMMY + 2)):
            assert call(lib, **over) == INV
    for over in (dict(rstd=None), dict(dw=DUMMY + 2), dict(w=DUMMY + 2)):
        assert norm_back(lib, **over) == INV
    for over in (dict(w=None), dict(w=DUMMY + 4), dict(ws=None), dict(ws=DUMMY + 1), dict(bias=DUMMY + 1),
                 dict(columns=0), dict(columns=-64), dict(columns=63), dict(columns=96), dict(columns=131072 + 64)):
        assert product(lib, **over) == INV
    for over in (dict(dw=None), dict(dw=DUMMY + 2), dict(db=DUMMY + 2), dict(channels=0), dict(channels=-1),
                 dict(channels=2 ** 24 + 1), dict(s=shape(channels=2 ** 20), channels=2 ** 20)):
        assert gradient(lib, **over) == INV


def test_refused_workspaces(lib):
    size = ctypes.c_int64()
    long = shape(n=64, steps=1000, channels=256)
    wide = seq(series=256000, step=256)
    assert lib.rocket_rms_norm_workspace(byref(long), byref(size)) == 0 and size.value > 0 and size.value % 8 == 0
    for ws, n in ((None, size.value), (DUMMY + 4, size.value), (DUMMY, size.value - 1)):
        assert norm_back(lib, long, wide, wide, dx=wide, ws=ws, size=n) == INV
    assert lib.rocket_linear_weight_gradient_workspace(byref(long), 100, byref(wide), byref(size)) == 0 and size.value > 0
    for ws, n in ((None, size.value), (DUMMY + 4, size.value), (DUMMY, size.value - 1)):
        assert gradient(lib, long, 100, wide, ws=ws, size=n) == INV
    for call in (lambda s, p: lib.rocket_rms_norm_workspace(s, p),
                 lambda s, p: lib.rocket_linear_bytes_workspace(s, 64, p),
                 lambda s, p: lib.rocket_linear_weight_gradient_workspace(s, 64, byref(wide), p)):
        assert call(byref(long), None) == INV and call(None, byref(size)) == INV
    assert lib.rocket_linear_bytes_workspace(byref(long), 96, byref(size)) == INV
    for channels, view in ((0, byref(wide)), (64, None), (64, byref(seq(data=None)))):
        assert lib.rocket_linear_weight_gradient_workspace(byref(long), channels, view, byref(size)) == INV


@pytest.mark.parametrize("none", [dict(n=0), dict(steps=0)])
def test_nothing_to_do_touches_nothing(lib, none):
    """No rows: accepted without a device (the sums of no rows are not wanted)."""
    s, v = shape(**none), rb.CSequence(None, 0, 0)
    assert norm(lib, s, v, y=v, rstd=None) == 0
    assert norm8(lib, s, v, q=None, scale=None, rstd=None) == 0
    assert norm_back(lib, s, v, v, rstd=None, dx=v, dw=None, ws=None, size=0) == 0
    assert quantize(lib, s, v, None, None) == 0 and keep(lib, s, v, None, None) == 0
    assert restore(lib, s, None, None, v) == 0
    assert product(lib, s, q=None, scale=None, w=None, ws=None, y=v, at=None, size=0) == 0


def test_binding_refuses_host_tensors(lib):
    import torch

    from paper_2601_17091_amd import sequence as sq
    x, r, w = torch.zeros(2, 3, 4), torch.zeros(2, 3), torch.zeros(4)
    q, k = torch.zeros(2, 3, 64, dtype=torch.int8), torch.zeros(1, 4, 128, dtype=torch.int8)
    for call in (lambda: sq.rms_norm(x), lambda: sq.rms_norm8(x, w), lambda: sq.rms_norm_backward(x, x, r),
                 lambda: sq.quantize_rows(x), lambda: sq.linear8(q, r, q[0], w), lambda: sq.checkpoint(x),
                 lambda: sq.restore(k, torch.zeros(1, 4), (2, 3)),
                 lambda: sq.linear_weight_gradient(x, k, torch.zeros(1, 4))):
        with pytest.raises(TypeError):
            call()
    assert sq.ROWS8_PAD == lo.PAD == 64 and sq.CHECKPOINT_ROWS == lo.BLOCK == 128
