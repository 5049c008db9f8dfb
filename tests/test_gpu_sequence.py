"""Sequence operators on the GPU against the 64-bit oracle, within the bounds
that the oracle derives from the operations' roundings: types, odd sizes, one
step to several tiles, strides, ragged and empty series, and what must not
change results (alignment, streams, graphs, repeated calls)."""
import math

import numpy as np
import pytest

from oracle import sequence_oracle as so

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")
ALL_ACTS = ("none", "relu", "silu", "gelu")


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2601_17091_amd as rk
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    rk.library()
    return torch, rk.sequence


def typed(torch, a, dtype):
    """(GPU tensor of that type, its values in 64 bits)."""
    t = torch.from_numpy(np.asarray(a, np.float32)).to(getattr(torch, dtype)).cuda()
    return t, t.double().cpu().numpy()


def f32(torch, a):
    return None if a is None else torch.from_numpy(np.asarray(a, np.float32)).cuda()


def host(t):
    return t.double().cpu().numpy()


def close(got, want, tol, what):
    got = host(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - tol
    assert over.max(initial=-1.0) <= 0, "%s: off by %.3g beyond the bound at %s" % (
        what, over.max(), np.unravel_index(over.argmax(), over.shape))


def ragged(rng, n, L):
    t = rng.integers(0, L + 1, size=n).astype(np.int32)
    t[0] = L
    if n > 1:
        t[1] = 0
    if n > 2:
        t[2] = 1
    return t


def blank(a, lengths):
    """NaN past every series' length."""
    if lengths is not None:
        for i, t in enumerate(lengths):
            a[i, t:] = np.nan
    return a


def cleaned(a):
    return np.nan_to_num(a, nan=0.0)


# ---------------------------------------------------------------- group norm
# n, L, C, groups: one element; one step; narrow rows; groups of odd widths;
# one group; one channel a group; each size of workgroup; several chunks;
# groups wider than a workgroup's columns; more series than workgroups keep
NORM_SHAPES = [(1, 1, 1, 1), (3, 1, 2000, 20), (2, 9, 3, 3), (5, 7, 5, 1), (3, 129, 33, 3), (2, 40, 24, 24),
               (3, 100, 132, 4), (2, 257, 64, 8), (1, 700, 40, 5), (2, 1100, 64, 4), (1, 2100, 36, 2),
               (2, 3, 5000, 2), (1, 5, 4100, 1), (40, 4, 16, 2), (2500, 2, 12, 3)]


def norm_inputs(torch, seed, n, L, C, dtype, with_lengths):
    rng = np.random.default_rng(seed)
    lengths = ragged(rng, n, L) if with_lengths else None
    level, spread = rng.standard_normal(C), np.exp(0.3 * rng.standard_normal(C))
    x, xv = typed(torch, blank(rng.standard_normal((n, L, C)) * spread + level, lengths), dtype)
    dy, dyv = typed(torch, blank(rng.standard_normal((n, L, C)), lengths), dtype)
    w, b = 1 + 0.2 * rng.standard_normal(C), 0.2 * rng.standard_normal(C)
    w, b = w.astype(np.float32), b.astype(np.float32)
    return x, cleaned(xv), dy, cleaned(dyv), w, b, lengths


def check_norm(torch, seq, n, L, C, G, dtype, act, with_lengths, affine=True):
    x, xv, dy, dyv, w, b, lengths = norm_inputs(torch, n * 1000 + L + C, n, L, C, dtype, with_lengths)
    if not affine:
        w = b = None
    lt = None if lengths is None else torch.from_numpy(lengths).cuda()
    tw, tb = f32(torch, w), f32(torch, b)
    y, mean, rstd = seq.group_norm(x, G, tw, tb, activation=act, lengths=lt)
    want = so.group_norm(xv, G, w, b, activation=act, lengths=lengths, dtype=dtype)
    close(mean, want["mean"], want["mean_tol"], "mean")
    close(rstd, want["rstd"], want["rstd_tol"], "rstd")
    close(y, want["y"], want["y_tol"], "y")
    dx, dw, db = seq.group_norm_backward(dy, x, G, mean, rstd, tw, tb, activation=act, lengths=lt)
    want = so.group_norm_backward(dyv, xv, G, host(mean), host(rstd), w, b, activation=act, lengths=lengths,
                                  dtype=dtype)
    close(dx, want["dx"], want["dx_tol"], "dx")
    close(dw, want["dweight"], want["dweight_tol"], "dweight")
    close(db, want["dbias"], want["dbias_tol"], "dbias")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C,G", NORM_SHAPES)
def test_group_norm_shapes(env, n, L, C, G, dtype):
    check_norm(*env, n, L, C, G, dtype, "silu", False)


@pytest.mark.parametrize("act", ALL_ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C,G", [(6, 37, 33, 3), (5, 1100, 48, 6)])
def test_group_norm_activations_and_lengths(env, n, L, C, G, dtype, act):
    check_norm(*env, n, L, C, G, dtype, act, True)


@pytest.mark.parametrize("L", [11, 2100])
def test_group_norm_without_weights(env, L):
    check_norm(*env, 3, L, 40, 5, "float32", "none", True, affine=False)


@pytest.mark.parametrize("L,C", [(20, 32), (5000, 32)])
def test_group_norm_level_far_above_the_spread(env, L, C):
    """Values at 1,000 with a spread of 1: the variance loses no digits."""
    torch, seq = env
    rng = np.random.default_rng(9)
    x, xv = typed(torch, 1000 + rng.standard_normal((2, L, C)), "float32")
    y, mean, rstd = seq.group_norm(x, 4)
    want = so.group_norm(xv, 4)
    close(rstd, want["rstd"], want["rstd_tol"], "rstd")
    close(y, want["y"], want["y_tol"], "y")
    # a constant group: variance 0, rstd 1 / sqrt(eps), y = bias
    bias = torch.arange(C, dtype=torch.float32, device="cuda")
    y, mean, rstd = seq.group_norm(torch.full((2, L, C), 3.0, device="cuda"), 4, None, bias, eps=1e-4)
    assert torch.equal(y, bias.expand(2, L, C)) and torch.allclose(rstd, torch.full_like(rstd, 100.0))


def test_group_norm_infinities_and_nan_stay_in_their_group(env):
    torch, seq = env
    x = torch.randn(3, 50, 64, device="cuda")
    clean = seq.group_norm(x, 4, activation="silu")[0]
    x[1, 7, 20] = float("nan")
    x[2, 7, 40] = float("inf")
    y = seq.group_norm(x, 4, activation="silu")[0]
    assert torch.equal(y[0], clean[0])
    assert y[1, :, 16:32].isnan().all() and torch.equal(y[1, :, :16], clean[1, :, :16])
    assert y[2, :, 32:48].isnan().all() and torch.equal(y[2, :, 48:], clean[2, :, 48:])


@pytest.mark.parametrize("L", [30, 1500])
def test_group_norm_gradient_is_the_difference(env, L):
    torch, seq = env
    rng = np.random.default_rng(4)
    n, C, G = 3, 24, 3
    x, xv = typed(torch, rng.standard_normal((n, L, C)), "float32")
    dy, dyv = typed(torch, rng.standard_normal((n, L, C)), "float32")
    w, b = rng.standard_normal(C).astype(np.float32), rng.standard_normal(C).astype(np.float32)
    y, mean, rstd = seq.group_norm(x, G, f32(torch, w), f32(torch, b), activation="gelu")
    dx, dw, db = seq.group_norm_backward(dy, x, G, mean, rstd, f32(torch, w), f32(torch, b), activation="gelu")

    def loss(x, w, b):
        return (so.group_norm(x, G, w, b, activation="gelu")["y"] * dyv).sum()

    h = 1e-4   # the difference's own error is of order h^2
    d = rng.standard_normal((n, L, C))
    dc = rng.standard_normal(C)
    w64, b64 = w.astype(np.float64), b.astype(np.float64)
    for fn, grad, direction in ((lambda e: loss(xv + e * d, w64, b64), dx, d),
                                (lambda e: loss(xv, w64 + e * dc, b64), dw, dc),
                                (lambda e: loss(xv, w64, b64 + e * dc), db, dc)):
        slope = (fn(h) - fn(-h)) / (2 * h)
        size = math.sqrt((host(grad) ** 2).sum() * (direction ** 2).sum())
        assert abs(slope - (host(grad) * direction).sum()) < 2e-5 * size + 1e-6


# ---------------------------------------------------------------- recurrence
# n, L, C: one element; one step; runs of less than a thread's; tiles that end
# inside a run; several tiles; lanes over 1 channel to several blocks
REC_SHAPES = [(1, 1, 1), (3, 1, 70), (2, 15, 2), (2, 16, 3), (2, 17, 5), (3, 128, 64), (2, 129, 66), (1, 300, 131),
              (2, 640, 9), (1, 1025, 130), (1, 9000, 1), (1, 4200, 2), (30, 33, 8), (1, 2000, 260)]


def rec_inputs(torch, seed, n, L, C, dtype, gate, with_lengths, packed):
    rng = np.random.default_rng(seed)
    lengths = ragged(rng, n, L) if with_lengths else None
    parts = 3 if gate else 2
    raw = rng.standard_normal((n, L, parts, C))
    raw[:, :, 1] += np.linspace(-2.0, 5.0, C)   # gates from forgetting to memories of hundreds of steps
    p, pv = typed(torch, blank(raw.reshape(n, L, parts * C), lengths), dtype)
    pv = cleaned(pv)
    views = [p[:, :, k * C:(k + 1) * C] for k in range(parts)]
    if not packed:
        views = [t.contiguous() for t in views]
    vals = [pv[:, :, k * C:(k + 1) * C] for k in range(parts)]
    if not gate:
        views.append(None)
        vals.append(None)
    dy, dyv = typed(torch, blank(rng.standard_normal((n, L, C)), lengths), dtype)
    h0 = rng.standard_normal((n, C)).astype(np.float32)
    dl = rng.standard_normal((n, C)).astype(np.float32)
    return views, vals, dy, cleaned(dyv), h0, dl, lengths


def check_rec(torch, seq, n, L, C, dtype, gate, with_lengths=False, packed=False, state=True):
    (v, f, o), (vv, fv, ov), dy, dyv, h0, dl, lengths = rec_inputs(torch, n + 10 * L + C, n, L, C, dtype, gate,
                                                                  with_lengths, packed)
    if not state:
        h0 = dl = None
    lt = None if lengths is None else torch.from_numpy(lengths).cuda()
    y, h_last, states = seq.recurrence(v, f, o, h0=f32(torch, h0), lengths=lt, keep_states=True)
    want = so.recurrence(vv, fv, ov, h0, lengths, dtype)
    close(y, want["y"], want["y_tol"], "y")
    close(h_last, want["h_last"], want["h_last_tol"], "h_last")
    close(states, want["states"], want["states_tol"], "states")
    bare = seq.recurrence(v, f, o, h0=f32(torch, h0), lengths=lt)
    assert torch.equal(bare[0], y) and torch.equal(bare[1], h_last) and bare[2] is None
    out = None
    if packed:
        parts = 3 if gate else 2
        d = torch.full((n, L, parts * C + 1), 7.0, dtype=v.dtype, device="cuda")
        out = [d[:, :, k * C:(k + 1) * C] for k in range(parts)]
    dv, df, do, dh0 = seq.recurrence_backward(dy, v, f, states, o, dh_last=f32(torch, dl), lengths=lt, out=out)
    want = so.recurrence_backward(dyv, vv, fv, ov, h0, dl, lengths, dtype)
    close(dv, want["dv"], want["dv_tol"], "dv")
    close(df, want["df"], want["df_tol"], "df")
    close(dh0, want["dh0"], want["dh0_tol"], "dh0")
    if gate:
        close(do, want["do"], want["do_tol"], "do")
    else:
        assert do is None
    if packed:
        assert bool((d[:, :, -1] == 7.0).all())   # the column beside the gradients


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C", REC_SHAPES)
def test_recurrence_shapes(env, n, L, C, dtype, gate):
    check_rec(*env, n, L, C, dtype, gate)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C", [(7, 40, 33), (5, 500, 130), (4, 300, 1)])
def test_recurrence_lengths_and_column_blocks(env, n, L, C, dtype, gate):
    check_rec(*env, n, L, C, dtype, gate, with_lengths=True, packed=True)


@pytest.mark.parametrize("L", [5, 700])
def test_recurrence_without_states(env, L):
    check_rec(*env, 3, L, 40, "bfloat16", True, state=False)


@pytest.mark.parametrize("lowest", [False, True])
def test_recurrence_closed_and_open_gates(env, lowest):
    """Gates at the ends of the range: f of the type's lowest value (or -inf)
    takes v as it is, of its highest (or inf) keeps the state to the bit."""
    torch, seq = env
    big = float("inf") if not lowest else torch.finfo(torch.float32).max
    n, L, C = 2, 300, 70
    v = torch.randn(n, L, C, device="cuda")
    f = torch.full_like(v, -big)
    f[:, :, 35:] = big
    h0 = torch.randn(n, C, device="cuda")
    y, h_last, states = seq.recurrence(v, f, h0=h0, keep_states=True)
    assert torch.equal(y[:, :, :35], v[:, :, :35]) and torch.equal(h_last[:, 35:], h0[:, 35:])
    assert torch.equal(y[:, :, 35:], h0[:, None, 35:].expand(n, L, 35))
    dv, df, _, dh0 = seq.recurrence_backward(torch.ones_like(v), v, f, states)
    assert torch.equal(dv[:, :, :35], torch.ones_like(dv[:, :, :35])) and bool((dv[:, :, 35:] == 0).all())
    assert bool((df == 0).all()) and bool((dh0[:, :35] == 0).all()) and bool((dh0[:, 35:] == L).all())


def test_recurrence_nan_stays_in_its_channel(env):
    torch, seq = env
    n, L, C = 2, 300, 66
    v, f = torch.randn(n, L, C, device="cuda"), torch.randn(n, L, C, device="cuda")
    clean = seq.recurrence(v, f)[0]
    v[1, 200, 5] = float("nan")
    f[1, 100, 6] = float("nan")
    y = seq.recurrence(v, f)[0]
    assert y[1, 200:, 5].isnan().all() and y[1, 100:, 6].isnan().all()
    assert torch.equal(y[1, :200, 5], clean[1, :200, 5]) and torch.equal(y[1, :100, 6], clean[1, :100, 6])
    keep = [c for c in range(C) if c not in (5, 6)]
    assert torch.equal(y[:, :, keep], clean[:, :, keep]) and torch.equal(y[0], clean[0])


def test_recurrence_of_no_steps(env):
    torch, seq = env
    h0, dl = torch.randn(3, 10, device="cuda"), torch.randn(3, 10, device="cuda")
    x = torch.empty(3, 0, 10, device="cuda")
    y, h_last, states = seq.recurrence(x, x, h0=h0, keep_states=True)
    assert y.shape == (3, 0, 10) and torch.equal(h_last, h0) and states.shape == (3, 0, 10)
    assert torch.equal(seq.recurrence_backward(x, x, x, states, dh_last=dl)[3], dl)
    y, mean, rstd = seq.group_norm(x, 2)
    assert y.shape == (3, 0, 10) and bool((mean == 0).all()) and bool((rstd == 0).all())
    dx, dw, db = seq.group_norm_backward(x, x, 2, mean, rstd)
    assert dx.shape == (3, 0, 10) and bool((dw == 0).all()) and bool((db == 0).all())
    e = torch.empty(0, 4, 10, device="cuda")
    assert seq.group_norm(e, 2)[0].shape == (0, 4, 10) and seq.recurrence(e, e)[1].shape == (0, 10)
    assert bool((seq.group_norm_backward(e, e, 2, torch.empty(0, 2, device="cuda"),
                                         torch.empty(0, 2, device="cuda"))[1] == 0).all())
    assert seq.dropout(e, 0.5, 1).shape == (0, 4, 10)
    assert seq.recurrence_step(e[:, 0], e[:, 0], torch.empty(0, 10, device="cuda"))[0].shape == (0, 10)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", [(1, 1), (3, 7), (64, 512), (5, 331)])
def test_recurrence_step(env, n, C, dtype, gate):
    """A step is the recurrence over one step, and steps in a row are the
    recurrence over a sequence."""
    torch, seq = env
    (v, f, o), (vv, fv, ov), _, _, h0, _, _ = rec_inputs(torch, n + C, n, 4, C, dtype, gate, False, True)
    h, ys = f32(torch, h0), []
    for t in range(4):
        y, h2 = seq.recurrence_step(v[:, t], f[:, t], h, None if o is None else o[:, t], h_out=h)
        assert h2 is h
        ys.append(y)
    want = so.recurrence(vv, fv, ov, h0, None, dtype)
    close(torch.stack(ys, 1), want["y"], want["y_tol"], "y")
    close(h, want["h_last"], want["h_last_tol"], "h")


def test_recurrence_gradient_is_the_difference(env):
    torch, seq = env
    n, L, C = 2, 400, 20
    (v, f, o), (vv, fv, ov), dy, dyv, h0, dl, _ = rec_inputs(torch, 3, n, L, C, "float32", True, False, False)
    states = seq.recurrence(v, f, o, h0=f32(torch, h0), keep_states=True)[2]
    grads = seq.recurrence_backward(dy, v, f, states, o, dh_last=f32(torch, dl))
    rng = np.random.default_rng(8)
    h = 1e-4
    at = [vv, fv, ov, h0.astype(np.float64)]
    for k in range(4):
        d = rng.standard_normal(at[k].shape)

        def loss(e):
            a = list(at)
            a[k] = a[k] + e * d
            r = so.recurrence(a[0], a[1], a[2], a[3])
            return (r["y"] * dyv).sum() + (r["h_last"] * dl).sum()

        slope, g = (loss(h) - loss(-h)) / (2 * h), host(grads[k])
        size = math.sqrt((g ** 2).sum() * (d ** 2).sum())
        assert abs(slope - (g * d).sum()) < 2e-5 * size + 1e-6


# ------------------------------------------------------------------- dropout
def expected_dropout(torch, x, residual, p, seed, call, indices):
    """The formula's fp32 operations, one rounding each, at flat indices."""
    d = so.dropout_threshold(p)
    u = torch.from_numpy(so.dropout_numbers(indices, seed, call))
    scale = np.float32(65536.0 / (65536.0 - d)) if d < 65536 else np.float32(0)
    ix = torch.as_tensor(indices)
    y = torch.where(u < d, torch.zeros(()), x.reshape(-1)[ix].float().cpu() * float(scale))
    if residual is not None:
        y = y + residual.reshape(-1)[ix].float().cpu()
    return y.to(x.dtype)


@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,p,call", [((1,), 0.5, 0), ((7,), 0.3, 1), ((8,), 0.3, 2 ** 40 + 1), ((3, 5, 7), 0.1, 9),
                                          ((2, 129, 33), 0.75, 2 ** 64 - 1), ((2050,), 0.0, 3), ((300,), 1.0, 4)])
def test_dropout(env, shape, p, call, dtype, with_residual):
    torch, seq = env
    seed = 0x123456789ABCDEF0
    x = torch.randn(shape, device="cuda").to(getattr(torch, dtype))
    r = torch.randn(shape, device="cuda").to(getattr(torch, dtype)) if with_residual else None
    y = seq.dropout(x, p, seed, call, residual=r)
    want = expected_dropout(torch, x, r, p, seed, call, np.arange(x.numel()))
    assert torch.equal(y.reshape(-1).cpu(), want)
    assert torch.equal(seq.dropout_backward(x, p, seed, call).reshape(-1).cpu(),
                       expected_dropout(torch, x, None, p, seed, call, np.arange(x.numel())))
    again = seq.dropout(x, p, seed, call, residual=r, out=x)   # in place
    assert again is x and torch.equal(again, y)


def test_dropout_masks_do_not_leak_and_differ(env):
    torch, seq = env
    x = torch.full((4096,), float("nan"), device="cuda")
    y = seq.dropout(x, 0.5, 1, 0)
    masks = [y.isnan()]
    assert bool((y[~masks[0]] == 0).all())
    for seed, call in ((1, 1), (2, 0), (1, 2 ** 32), (1 + 2 ** 32, 0)):
        masks.append(seq.dropout(x, 0.5, seed, call).isnan())
    for i in range(len(masks)):
        # 4096 fair draws: 2048 +- 6 standard deviations
        assert abs(int(masks[i].sum()) - 2048) < 192
        for j in range(i):
            assert abs(int((masks[i] == masks[j]).sum()) - 2048) < 192


@pytest.mark.parametrize("dtype", DTYPES)
def test_dropout_in_rows(env, dtype):
    """Column blocks: the element's number is that of the dense tensor."""
    torch, seq = env
    dt = getattr(torch, dtype)
    big = torch.randn(6, 9, 70, device="cuda").to(dt)
    for c0, c1 in ((0, 64), (3, 36), (69, 70), (5, 12)):
        x = big[:, :, c0:c1]
        dense = seq.dropout(x.contiguous(), 0.4, 77, 5, residual=x.contiguous())
        assert torch.equal(seq.dropout(x, 0.4, 77, 5, residual=x), dense)
        out = torch.full((6, 9, 80), 3.0, device="cuda", dtype=dt)
        seq.dropout(x.contiguous(), 0.4, 77, 5, residual=x, out=out[:, :, 1:1 + c1 - c0])
        assert torch.equal(out[:, :, 1:1 + c1 - c0], dense)
        assert bool((out[:, :, :1] == 3).all()) and bool((out[:, :, 1 + c1 - c0:] == 3).all())


def test_dropout_past_32_bits(env):
    """Elements past 2^32: the counter and the offsets are 64 bits wide."""
    torch, seq = env
    n = (1 << 32) + 1003
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = seq.dropout(x, 0.25, 11, 3, out=x)
    ix = np.concatenate([np.arange(40), np.arange((1 << 31) - 20, (1 << 31) + 20),
                         np.arange((1 << 32) - 20, (1 << 32) + 20), np.arange(n - 30, n)])
    want = expected_dropout(torch, torch.ones(1, dtype=torch.bfloat16).expand(n), None, 0.25, 11, 3, ix)
    assert torch.equal(y[torch.from_numpy(ix).cuda()].cpu(), want)


# ------------------------------------------- layouts, streams, graphs, repeats
def all_calls(torch, seq, x, f, o, lengths=None):
    """Outputs of every sequence call on [n, L, C] operands."""
    w = torch.linspace(0.5, 1.5, x.shape[2], device="cuda")
    y, mean, rstd = seq.group_norm(x, 3, w, w, activation="silu", lengths=lengths)
    grads = seq.group_norm_backward(o, x, 3, mean, rstd, w, w, activation="silu", lengths=lengths)
    r, h, states = seq.recurrence(x, f, o, lengths=lengths, keep_states=True)
    back = seq.recurrence_backward(x, x, f, states, o, dh_last=h, lengths=lengths)
    return [y, mean, rstd, *grads, r, h, states, *back]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C", [(3, 50, 33), (2, 1300, 30)])
def test_strides_and_alignment_change_nothing(env, n, L, C, dtype):
    torch, seq = env
    dt = getattr(torch, dtype)
    x, f, o = (torch.randn(n, L, C, device="cuda").to(dt) for _ in range(3))
    want = all_calls(torch, seq, x, f, o)

    def columns(t, at):       # a block of columns at any offset
        big = torch.full((n, L, C + 9), float("nan"), device="cuda").to(dt)
        big[:, :, at:at + C] = t
        return big[:, :, at:at + C]

    def steps_first(t):       # [L, n, C] in memory
        return t.transpose(0, 1).contiguous().transpose(0, 1)

    def flat(t, at):          # a storage offset of any element
        big = torch.full((t.numel() + 16,), float("nan"), device="cuda").to(dt)
        big[at:at + t.numel()] = t.reshape(-1)
        return big[at:at + t.numel()].view(n, L, C)

    for move in (lambda t: columns(t, 1), lambda t: columns(t, 8), steps_first, lambda t: flat(t, 1),
                 lambda t: flat(t, 3)):
        got = all_calls(torch, seq, move(x), move(f), move(o))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_repeated_rows_as_inputs(env):
    """An input that is one row for every series or step (strides of 0)."""
    torch, seq = env
    for row in (torch.randn(1, 40, 30, device="cuda"), torch.randn(2, 1, 30, device="cuda")):
        x = row.expand(2, 40, 30)
        got = all_calls(torch, seq, x, x, x)
        want = all_calls(torch, seq, x.contiguous(), x.contiguous(), x.contiguous())
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("L", [60, 1500])
def test_outputs_in_place(env, L):
    torch, seq = env
    n, C = 2, 33
    x, f, o = (torch.randn(n, L, C, device="cuda").to(torch.bfloat16) for _ in range(3))
    y, mean, rstd = seq.group_norm(x, 3)
    r, h, states = seq.recurrence(x, f, o, keep_states=True)
    dx = seq.group_norm_backward(o, x, 3, mean, rstd)[0]
    dv, df, do, _ = seq.recurrence_backward(o, x, f, states, o)
    for k in range(2):
        a, b = x.clone(), o.clone()
        seq.group_norm_backward(b, a, 3, mean, rstd, out=(a, b)[k])
        assert torch.equal((a, b)[k], dx)
    a = x.clone()
    assert torch.equal(seq.group_norm(a, 3, out=a)[0], y)
    for k in range(3):
        t = [x.clone(), f.clone(), o.clone()]
        assert torch.equal(seq.recurrence(*t, out=t[k])[0], r)
    t = [x.clone(), f.clone(), o.clone(), o.clone()]
    seq.recurrence_backward(t[3], t[0], t[1], states, t[2], out=t[:3])
    assert torch.equal(t[0], dv) and torch.equal(t[1], df) and torch.equal(t[2], do)


@pytest.mark.parametrize("dtype", DTYPES)
def test_nothing_is_written_outside(env, dtype):
    """Outputs inside a larger buffer, odd sizes: the rest of it stays."""
    torch, seq = env
    dt = getattr(torch, dtype)
    for n, L, C in ((2, 19, 33), (1, 1200, 9), (3, 130, 131)):
        x = torch.randn(n, L, C, device="cuda").to(dt)
        for call, m in ((lambda out: seq.group_norm(x, 1, out=out), n),
                        (lambda out: seq.recurrence(x, x, x, out=out), n),
                        (lambda out: seq.dropout(x[:1], 0.5, 1, out=out), 1)):   # rows of equal distance
            big = torch.full((n + 1, L + 2, C + 5), 9.0, device="cuda").to(dt)
            call(big[:m, 1:L + 1, 3:C + 3])
            outside = torch.ones_like(big, dtype=torch.bool)
            outside[:m, 1:L + 1, 3:C + 3] = False
            assert bool((big[outside] == 9.0).all()) and not bool((big[~outside] == 9.0).any())


def test_other_streams(env):
    """A call on a stream that is not the current one, after work queued there."""
    torch, seq = env
    x, f, o = (torch.randn(8, 700, 66, device="cuda") for _ in range(3))
    want = seq.recurrence(x, f, o)[0]
    norm = seq.group_norm(x, 3)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            late = torch.zeros_like(x)
            late.add_(x)          # queued on the side stream, before the calls
        got = seq.recurrence(late, f, o, stream=side)[0]
        got2 = seq.group_norm(late, 3, stream=side)[0]
        filler = [torch.full((700, 66), 5.0, device="cuda") for _ in range(20)]   # the current stream goes on
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(got2, norm)
        del filler


def test_graph_replays(env):
    """Captured once, replayed with new inputs between eager work."""
    torch, seq = env
    x, f, o = (torch.randn(2, 1200, 66, device="cuda") for _ in range(3))
    step = torch.randn(2, 66, device="cuda")
    all_calls(torch, seq, x, f, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = all_calls(torch, seq, x, f, o)
        out += [seq.dropout(x, 0.3, 5, 6, residual=f), *seq.recurrence_step(step, step, step)]
    for k in range(4):
        for t in (x, f, o, step):
            t.normal_()
        want = all_calls(torch, seq, x, f, o)
        want += [seq.dropout(x, 0.3, 5, 6, residual=f), *seq.recurrence_step(step, step, step)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_repeated_calls_agree_bitwise(env):
    torch, seq = env
    x, f, o = (torch.randn(5, 2000, 130, device="cuda").to(torch.bfloat16) for _ in range(3))
    x = x[:, :, :129]
    f, o = f[:, :, :129], o[:, :, :129]
    lengths = torch.tensor([2000, 0, 1, 999, 128], dtype=torch.int32, device="cuda")
    want = all_calls(torch, seq, x, f, o, lengths)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(all_calls(torch, seq, x, f, o, lengths), want))


def test_lengths_outside_the_range_are_taken_into_it(env):
    torch, seq = env
    x, f, o = (torch.randn(3, 20, 12, device="cuda") for _ in range(3))
    a = all_calls(torch, seq, x, f, o, torch.tensor([-3, 999, 7], dtype=torch.int32, device="cuda"))
    b = all_calls(torch, seq, x, f, o, torch.tensor([0, 20, 7], dtype=torch.int32, device="cuda"))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_offsets_past_32_bits(env):
    """Series 2^31 and more elements apart, in one buffer."""
    torch, seq = env
    far, L, C = (1 << 31) + 24, 200, 40
    big = torch.zeros(2 * far + L * C, dtype=torch.bfloat16, device="cuda")
    views = big.as_strided((3, L, C), (far, C, 1))
    x = torch.randn(3, L, C, device="cuda").to(torch.bfloat16)
    views.copy_(x)
    want = [seq.group_norm(x, 5)[0], seq.recurrence(x, x, x)[0]]
    assert torch.equal(seq.group_norm(views, 5)[0], want[0])
    assert torch.equal(seq.recurrence(views, views, views)[0], want[1])
    seq.recurrence(x, x, x, out=views)
    assert torch.equal(views, want[1])
    seq.group_norm(x, 5, out=views)
    assert torch.equal(views, want[0])


def test_binding_refusals(env):
    torch, seq = env
    x = torch.zeros(2, 6, 8, device="cuda")
    h = torch.zeros(2, 8, device="cuda")
    bad_value = [
        lambda: seq.group_norm(x[0], 2), lambda: seq.group_norm(x.double(), 2), lambda: seq.group_norm(x, 2, h[0, :4]),
        lambda: seq.group_norm(x, 2, activation="tanh"), lambda: seq.group_norm(x, 2, out=x[:, :3]),
        lambda: seq.group_norm(x.transpose(1, 2), 2),
        lambda: seq.group_norm(x, 2, lengths=torch.zeros(2, device="cuda")),
        lambda: seq.group_norm(x, 2, lengths=torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: seq.recurrence(x, x[:, :5]), lambda: seq.recurrence(x, x.half()), lambda: seq.recurrence(x, x, h0=h[:1]),
        lambda: seq.recurrence_backward(x, x, x, h), lambda: seq.recurrence_backward(x, x, x, h[:, None], out=[x]),
        lambda: seq.recurrence_step(x, x, h), lambda: seq.recurrence_step(h, h, h.half()),
        lambda: seq.dropout(x.transpose(1, 2), 0.5, 1), lambda: seq.dropout(x.long(), 0.5, 1),
        lambda: seq.dropout(x, 0.5, 1, residual=x[:1])]
    for k, call in enumerate(bad_value):
        with pytest.raises(ValueError):
            call()
            print(k)
    for call in (lambda: seq.group_norm(x.cpu(), 2), lambda: seq.group_norm(x, 2, lengths=[6, 6]),
                 lambda: seq.recurrence(x, x.cpu()), lambda: seq.recurrence_backward(x, x, x, None),
                 lambda: seq.group_norm_backward(x, x, 2, None, None), lambda: seq.recurrence_step(h, h, None)):
        with pytest.raises(TypeError):
            call()
    from paper_2601_17091_amd import RocketError
    for call in (lambda: seq.group_norm(x, 3), lambda: seq.group_norm(x, 0), lambda: seq.dropout(x, 1.5, 1),
                 lambda: seq.group_norm(x, 2, eps=-1.0)):
        with pytest.raises(RocketError):
            call()
