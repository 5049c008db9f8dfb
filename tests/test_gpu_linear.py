"""The operators around linear layers on the GPU against the 64-bit oracle, within
the bounds that the oracle derives from the operations' roundings, and bit for
bit where single fp32 operations define the result: types, one row to many, odd
sizes, strides, ragged and empty series, NaN and infinities, streams, graphs."""
import numpy as np
import pytest

from oracle import linear_oracle as lo

pytestmark = pytest.mark.gpu

DTYPES = ("float32", "bfloat16", "float16")


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2601_17091_amd as rk
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    rk.library()
    return torch, rk.sequence


def host(t):
    return t.double().cpu().numpy()


def cuda(torch, a, dtype="float32"):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(getattr(torch, dtype)).cuda()


def values(t):
    return t.float().cpu().numpy()


def close(got, want, tol, what):
    got = host(got).reshape(want.shape)
    assert np.isfinite(got).all(), what
    over = np.abs(got - want) - tol
    assert over.max(initial=-1.0) <= 0, "%s: off by %.3g beyond the bound at %s" % (
        what, over.max(), np.unravel_index(over.argmax(), over.shape))


def same(got, want, what):
    got = got.float().cpu().numpy().reshape(want.shape)
    assert np.array_equal(got, want.astype(np.float32), equal_nan=True), (what, np.argwhere(got != want)[:5])


def ragged(rng, n, L):
    t = rng.integers(0, L + 1, size=n).astype(np.int32)
    t[0] = L
    if n > 1:
        t[1] = 0
    if n > 2:
        t[2] = 1
    return t


class Sample:
    """Sequences [n, L, C] of a type with NaN past every series' length."""

    def __init__(self, torch, seed, n, L, dtype, with_lengths):
        self.torch, self.rng, self.n, self.L, self.dtype = torch, np.random.default_rng(seed), n, L, dtype
        self.lengths = ragged(self.rng, n, L) if with_lengths else None
        self.on_gpu = None if self.lengths is None else torch.from_numpy(self.lengths).cuda()
        self.live = lo.live_rows(n, L, self.lengths)

    def blank(self, a):
        a = np.asarray(a, np.float32).reshape(self.n * self.L, -1)
        a[~self.live] = np.nan
        return a.reshape(self.n, self.L, -1)

    def normal(self, C, scale=1.0, level=0.0, dtype=None):
        """(tensor, its values [rows, C])."""
        t = cuda(self.torch, self.blank(level + scale * self.rng.standard_normal((self.n * self.L, C))),
                 dtype or self.dtype)
        return t, values(t).reshape(-1, C)

    def floats(self, *shape, scale=1.0, shift=0.0):
        a = (shift + scale * self.rng.standard_normal(shape)).astype(np.float32)
        return cuda(self.torch, a), a


# ---------------------------------------------------------------- RMS norm
# one element; narrow rows; each number of threads and chunks with odd rests; rows
# that a workgroup loops over; more rows than a launch's workgroups take at once
NORM_SHAPES = [(1, 1, 1), (2, 3, 7), (3, 5, 64), (3, 5, 67), (2, 9, 129), (2, 9, 255), (1, 7, 331), (2, 3, 513),
               (3, 3, 924), (2, 2, 2000), (1, 3, 2051), (1, 3, 4100), (2, 1, 8195), (1, 2, 12345), (1, 2, 20000),
               (1, 2, 24576), (1, 2, 24577), (1, 2, 50001), (3000, 3, 20), (2500, 1, 260)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n,L,C", NORM_SHAPES)
def test_rms_norm(env, n, L, C, residual, dtype):
    check_norm(*env, n, L, C, residual, dtype, False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n,L,C", [(1, 1, 5), (7, 37, 33), (40, 9, 300), (5, 11, 924), (3, 4, 20001), (3, 2, 30000)])
def test_rms_norm_lengths(env, n, L, C, residual, dtype):
    check_norm(*env, n, L, C, residual, dtype, True)


# of each width more rows than the workgroups of a launch, with empty rows between
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C", [(4500, 1, 900), (9000, 3, 33), (13000, 1, 200), (4000, 2, 256), (400, 5, 1400), (401, 5, 2047), (330, 3, 2049), (270, 3, 4001),
                                   (150, 2, 7001), (140, 2, 8193), (140, 2, 12001), (130, 2, 16400)])
def test_rms_norm_many_wide_rows(env, n, L, C, dtype):
    check_norm(*env, n, L, C, True, dtype, True)


@pytest.mark.parametrize("C", [40, 30000])
def test_rms_norm_without_weights(env, C):
    check_norm(*env, 3, 5, C, True, "float32", True, weighted=False)


def check_norm(torch, seq, n, L, C, residual, dtype, with_lengths, weighted=True):
    s = Sample(torch, n * 1000 + L + C, n, L, dtype, with_lengths)
    level = s.rng.standard_normal(C)
    x, xv = s.normal(C, level=level)
    r, rv = s.normal(C, scale=2.0) if residual else (None, None)
    w, wv = s.floats(C, scale=0.2, shift=1.0) if weighted else (None, None)
    want = lo.rms_norm(xv, wv, rv, live=s.live, dtype=dtype)
    y, total, rstd = seq.rms_norm(x, w, residual=r, lengths=s.on_gpu)
    if residual:
        same(total, want["total"], "total")
    else:
        assert total is x
    close(rstd, want["rstd"], want["rstd_tol"], "rstd")
    close(y, want["y"], want["y_tol"], "y")
    # 8-bit rows of the same: q to the nearest whole number of what it stands for
    q, scale, total8, rstd8 = seq.rms_norm8(x, w, residual=r, lengths=s.on_gpu)
    assert q.shape == (n, L, lo.pad(C)) and torch.equal(rstd8, rstd)
    if residual:
        assert torch.equal(total8, total)
    q, v = host(q).reshape(n * L, -1), want["total"].astype(np.float64) * (1.0 if wv is None else wv)
    top = np.abs(v).max(1)
    close(scale, want["rstd"] * top / 127, want["rstd_tol"] * top / 127 + want["rstd"] * top / 127 * 4 * lo.U, "scale")
    assert (q[:, C:] == 0).all()
    unit = np.where(top > 0, top / 127, 1)[:, None]
    # s w, 127 / a and their product round once each
    assert (np.abs(q[:, :C] - v / unit) <= 0.5 + 127 * 3 * lo.U).all()
    assert (np.abs(q).max(1) == np.where(top > 0, 127, 0)).all()
    # the gradient
    dy, dyv = s.normal(C)
    dt, dtv = s.normal(C) if residual else (None, None)
    dx, dw = seq.rms_norm_backward(dy, total, rstd, w, dtotal=dt, lengths=s.on_gpu)
    want = lo.rms_norm_backward(dyv, want["total"], values(rstd).reshape(-1), wv, dtv, s.live, dtype)
    close(dx, want["dx"], want["dx_tol"], "dx")
    close(dw, want["dweight"], want["dweight_tol"], "dweight")


@pytest.mark.parametrize("dtype", DTYPES)
def test_rms_norm_in_place_and_in_strides(env, dtype):
    """Columns of a wider matrix, rows turned about, every allowed aliasing."""
    torch, seq = env
    n, L, C = 4, 6, 77
    wide = torch.randn(L, n, 3 * C + 1, device="cuda").to(getattr(torch, dtype))
    w = torch.randn(C, device="cuda")
    x, r = wide[:, :, 1:C + 1].transpose(0, 1), wide[:, :, C + 1:2 * C + 1].transpose(0, 1)
    xc, rc = x.contiguous(), r.contiguous()
    want, total, rstd = seq.rms_norm(xc, w, residual=rc)
    for outs in ((None, None), (0, 1), (1, 0)):
        a = wide.clone()
        ops = [a[:, :, 1:C + 1].transpose(0, 1), a[:, :, C + 1:2 * C + 1].transpose(0, 1)]
        y, t, k = seq.rms_norm(ops[0], w, residual=ops[1], out=None if outs[0] is None else ops[outs[0]],
                               total_out=None if outs[1] is None else ops[outs[1]])
        assert torch.equal(y, want) and torch.equal(t, total) and torch.equal(k, rstd)
        assert torch.equal(a[:, :, 0], wide[:, :, 0]) and torch.equal(a[:, :, 2 * C + 1:], wide[:, :, 2 * C + 1:])
    dy, dt = torch.randn_like(xc), torch.randn_like(xc)
    dx, dw = seq.rms_norm_backward(dy, total, rstd, w, dtotal=dt)
    for k in range(3):
        ops = [dy.clone(), total.clone(), dt.clone()]
        got, dw2 = seq.rms_norm_backward(ops[0], ops[1], rstd, w, dtotal=ops[2], out=ops[k])
        assert got is ops[k] and torch.equal(got, dx) and torch.equal(dw, dw2)
    # rows as a matrix
    y2, _, k2 = seq.rms_norm(xc.view(n * L, C), w, residual=rc.view(n * L, C))
    assert torch.equal(y2.view(n, L, C), want) and k2.shape == (n * L,)


def test_rms_norm_wide_gradient_in_place(env):
    """Rows too wide for registers: dweight is summed before dx is written over dy."""
    torch, seq = env
    x, dy = torch.randn(2, 3, 30000, device="cuda"), torch.randn(2, 3, 30000, device="cuda")
    _, _, rstd = seq.rms_norm(x)
    dx, dw = seq.rms_norm_backward(dy, x, rstd)
    for k in range(2):
        ops = [dy.clone(), x.clone()]
        got, dw2 = seq.rms_norm_backward(*ops, rstd, out=ops[k])
        assert torch.equal(got, dx) and torch.equal(dw, dw2)


def test_rms_norm_rows_do_not_meet(env):
    """NaN and infinities stay in their rows; a row of zeros is finite."""
    torch, seq = env
    x = torch.randn(1, 40, 33, device="cuda")
    bad = x.clone()
    bad[0, 3, 5], bad[0, 9, 32], bad[0, 11] = float("nan"), float("inf"), 0.0
    y, _, _ = seq.rms_norm(x)
    z, _, k = seq.rms_norm(bad)
    rest = [i for i in range(40) if i not in (3, 9, 11)]
    assert torch.equal(y[0, rest], z[0, rest]) and (z[0, 11] == 0).all() and z[0, 3].isnan().all()
    q, scale, _, _ = seq.rms_norm8(bad)
    good = seq.rms_norm8(x)
    assert torch.equal(q[0, rest], good[0][0, rest]) and torch.equal(scale[0, rest], good[1][0, rest])
    assert (q[0, [3, 9, 11]] == 0).all() and scale[0, [3, 9]].isnan().all() and scale[0, 11] == 0


# -------------------------------------------------------------- 8-bit rows
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,L,C,with_lengths", [(1, 1, 1, False), (3, 5, 64, True), (7, 3, 331, True), (2, 9, 924, False),
                                                (1, 2, 20000, False), (2, 2, 30000, True)])
def test_quantize_rows(env, n, L, C, with_lengths, dtype):
    torch, seq = env
    s = Sample(torch, C, n, L, dtype, with_lengths)
    x, xv = s.normal(C, level=3 * s.rng.standard_normal(C))
    q, scale = seq.quantize_rows(x, lengths=s.on_gpu)
    wq, wscale = lo.quantize_rows(xv, s.live)
    same(q, wq, "q")
    same(scale, wscale, "scale")


def test_quantize_rows_extremes(env):
    torch, seq = env
    x = torch.tensor([[127, 0.5, 1.5, -2.5, -127], [254, 1, -3, 0, 5], [0, 0, 0, 0, 0], [1, float("nan"), 0, 0, 0],
                      [1, float("inf"), 0, 0, 0], [1e-38, 0, 0, 0, 0], [3e38, -3e38, 1e38, 0, 1], [1e-30, 5e-31, 0, 0, 0]],
                     device="cuda")
    q, scale = seq.quantize_rows(x)
    wq, wscale = lo.quantize_rows(x.cpu().numpy())
    same(q, wq, "q")
    same(scale, wscale, "scale")


# ----------------------------------------------------------------- product
# one row and one channel to several tiles each way, odd sizes, few and many columns
PRODUCTS = [(1, 1, 64, 1), (1, 3, 64, 5), (2, 8, 128, 16), (1, 17, 192, 33), (5, 13, 320, 64), (1, 64, 2048, 192),
            (3, 43, 960, 131), (1, 130, 64, 993), (9, 31, 448, 257), (1, 700, 384, 300), (1, 5, 20032, 77),
            (1, 300, 4096, 16)]


def product_inputs(s, columns, N, whole=False):
    torch, rng = s.torch, s.rng
    q = rng.integers(-127, 128, size=(s.n, s.L, columns)).astype(np.int8)
    p = rng.integers(-127, 128, size=(N, columns)).astype(np.int8)
    scale = (0.5 + rng.random((s.n, s.L))).astype(np.float32)
    scale.reshape(-1)[~s.live] = np.nan
    ws, b = (0.01 + 0.01 * rng.random(N)).astype(np.float32), rng.standard_normal(N).astype(np.float32)
    return [q, scale, p, ws, b], [torch.from_numpy(a).cuda() for a in (q, scale, p, ws, b)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("with_lengths", [False, True])
@pytest.mark.parametrize("n,L,columns,N", PRODUCTS)
def test_linear8(env, n, L, columns, N, with_lengths, dtype):
    torch, seq = env
    s = Sample(torch, n + L + columns + N, n, L, dtype, with_lengths)
    (q, scale, p, ws, b), on_gpu = product_inputs(s, columns, N)
    flat = np.where(s.live, scale.reshape(-1), 0)
    for bias in (True, False):
        y = seq.linear8(*on_gpu[:4], on_gpu[4] if bias else None, dtype=getattr(torch, dtype), lengths=s.on_gpu)
        assert y.shape == (n, L, N)
        want, tol = lo.linear8(q.reshape(n * L, -1), flat, p, ws, b if bias else None, s.live, dtype)
        close(y, want, tol, "y")
    again = seq.linear8(*on_gpu[:4], dtype=getattr(torch, dtype), lengths=s.on_gpu)
    assert torch.equal(again, y)


# rows, columns, channels where each size of tile, and tiles whose columns are shared out,
# cost least; last stages of 64 and of 128 columns, one stage, more tiles than run at once
WAYS = [(20000, 192, 1100), (70001, 64, 513), (70000, 2048, 250), (6000, 2048, 1530), (9000, 320, 1000),
        (1000, 1984, 1536), (30000, 256, 768), (100000, 128, 60), (1000, 20032, 190), (130, 20032, 70),
        (65, 4096, 2000), (300, 8192, 33), (16100, 1984, 1536), (33000, 1984, 1030), (65000, 64, 2000)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("with_lengths", [False, True])
@pytest.mark.parametrize("rows,columns,N", WAYS)
def test_linear8_large(env, rows, columns, N, with_lengths, dtype):
    """Against 64-bit products on the GPU, of the roundings that the oracle counts."""
    torch, seq = env
    g = torch.Generator(device="cuda").manual_seed(rows + columns + N)
    rand8 = lambda *s: torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    n = next(k for k in (7, 5, 4, 3, 2, 1) if rows % k == 0)
    L = rows // n
    q, p, scale, ws, b = rand8(n, L, columns), rand8(N, columns), 0.5 + rand(n, L), 0.01 + rand(N), rand(N) - 0.5
    lengths, live = None, torch.ones(n, L, 1, dtype=torch.bool, device="cuda")
    if with_lengths:
        lengths = torch.randint(0, L + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        live = (torch.arange(L, device="cuda")[None, :] < lengths[:, None])[:, :, None]
        scale = scale.masked_fill(~live[:, :, 0], float("nan"))
    y = seq.linear8(q, scale, p, ws, b, dtype=getattr(torch, dtype), lengths=lengths)
    product = (q.view(rows, columns).double() @ p.double().t().contiguous()).view(n, L, N)
    product = product * scale.double()[:, :, None] * ws.double()
    want = product + b
    tol = (3 * product.abs() + want.abs()) * lo.U
    tol = tol * 1.01 + want.abs() * (2.0 ** -8 if dtype == "bfloat16" else lo.U) * 1.001 + 1e-30
    ok = ((y.double() - want).abs() <= tol) & live | (y == 0) & ~live
    assert ok.all(), torch.nonzero(~ok)[:4]


def row_lengths(kind, n, L, g):
    """Lengths [n]: any, none, all, one row of one series, past both ends, all or nothing."""
    import torch
    any_ = torch.randint(0, L + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "none":
        return torch.zeros_like(any_)
    if kind == "all":
        return torch.full_like(any_, L)
    if kind == "one row":
        any_.zero_()[n - 2] = 1
    elif kind == "past both ends":
        any_[::3], any_[1::3] = -5, L + 7
    elif kind == "all or nothing":
        any_ = (any_ > L // 2).int() * L
    return any_


# (series, steps, columns, channels) of large products whose live rows are listed first: the
# most series, the least columns, last stages of 64 columns, a launch's last tiles of each
# number, of each size; and those past what is listed: more series, more bytes, fewer
# stages, less work
LISTED = [(4096, 20, 256, 768), (777, 129, 960, 993), (2, 33000, 256, 1000), (3000, 30, 320, 1000),
          (64, 1000, 2048, 1536), (333, 50, 2048, 1536), (200, 1000, 192, 512), (300, 1000, 256, 130)]
UNLISTED = [(4097, 30, 256, 768), (2, 33000, 32768, 768), (50, 1000, 128, 1024), (777, 129, 192, 200)]


@pytest.mark.parametrize("kind", ["any", "none", "all", "one row", "past both ends", "all or nothing"])
@pytest.mark.parametrize("n,L,columns,N", LISTED + UNLISTED)
def test_linear8_of_listed_rows(env, n, L, columns, N, kind):
    """Rows that hold data have the very results of a call without lengths, the others are
    zeros, and nothing is written beside them."""
    torch, seq = env
    rows, listed = n * L, (n, L, columns, N) in LISTED
    assert (seq._linear8_size(n, L, N, 2, columns) == (rows * 4 + 11) // 8 * 8) == listed
    g = torch.Generator(device="cuda").manual_seed(rows + columns + N)
    q = torch.randint(-127, 128, (n, L, columns), generator=g, device="cuda", dtype=torch.int8)
    p = torch.randint(-127, 128, (N, columns), generator=g, device="cuda", dtype=torch.int8)
    scale, ws, b = (torch.rand(k, generator=g, device="cuda") + 0.5 for k in ((n, L), (N,), (N,)))
    ws *= 2.0 ** -12   # results that float16 holds
    lengths = row_lengths(kind, n, L, g)
    live = (torch.arange(L, device="cuda")[None, :] < lengths[:, None])
    want = seq.linear8(q, scale, p, ws, b, dtype=torch.float16).masked_fill(~live[:, :, None], 0)
    scale = scale.masked_fill(~live, float("nan"))
    wide = torch.full((n, L, N + 5), 7.0, dtype=torch.float16, device="cuda")
    out = wide[:, :, 3:N + 3]
    seq.linear8(q, scale, p, ws, b, lengths=lengths, out=out)
    assert torch.equal(out, want)
    assert (wide[:, :, :3] == 7).all() and (wide[:, :, N + 3:] == 7).all()


def test_linear8_of_listed_rows_in_a_graph(env):
    """A captured call lists the rows anew in every replay."""
    torch, seq = env
    n, L, columns, N = LISTED[1]
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randint(-127, 128, (n, L, columns), generator=g, device="cuda", dtype=torch.int8)
    p = torch.randint(-127, 128, (N, columns), generator=g, device="cuda", dtype=torch.int8)
    scale, ws = torch.rand(n, L, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    lengths = row_lengths("any", n, L, g)
    call = lambda: seq.linear8(q, scale, p, ws, lengths=lengths)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call()
    for kind in ("any", "one row", "all", "none", "past both ends"):
        lengths.copy_(row_lengths(kind, n, L, g))
        graph.replay()
        got = y.clone()
        assert torch.equal(got, call())
        live = torch.arange(L, device="cuda")[None, :] < lengths[:, None]
        assert (got[~live] == 0).all()


def test_linear8_is_exact(env):
    """Whole numbers below 2^24 come out as they are: no rounding anywhere."""
    torch, seq = env
    rng = np.random.default_rng(5)
    q = rng.integers(-127, 128, size=(333, 576)).astype(np.int8)
    p = rng.integers(-127, 128, size=(211, 576)).astype(np.int8)
    one = lambda k: torch.ones(k, device="cuda")  # noqa: E731
    y = seq.linear8(torch.from_numpy(q).cuda(), one(333), torch.from_numpy(p).cuda(), one(211), dtype=torch.float32)
    assert np.array_equal(y.cpu().numpy(), (q.astype(np.int64) @ p.astype(np.int64).T).astype(np.float32))
    # the largest sums that 32 bits hold
    q = torch.full((3, 131072), -128, dtype=torch.int8, device="cuda")
    q[1], q[2] = 127, -127
    w = torch.full((2, 131072), 127, dtype=torch.int8, device="cuda")
    y = seq.linear8(q, one(3), w, one(2), dtype=torch.float32)
    assert y[:, 0].tolist() == [float(np.float32(-128 * 127 * 131072)), 127.0 * 127 * 131072, -127.0 * 127 * 131072]


def test_linear8_into_columns(env):
    """Results into columns of a wider matrix, rows turned about; what lies beside stays."""
    torch, seq = env
    s = Sample(torch, 8, 5, 9, "float16", True)
    _, ops = product_inputs(s, 256, 75)
    want = seq.linear8(*ops, dtype=torch.float16, lengths=s.on_gpu)
    wide = torch.full((9, 5, 200), 7.0, dtype=torch.float16, device="cuda")
    out = wide[:, :, 101:176].transpose(0, 1)
    got = seq.linear8(*ops, lengths=s.on_gpu, out=out)
    assert got is out and torch.equal(out, want)
    assert (wide[:, :, :101] == 7).all() and (wide[:, :, 176:] == 7).all()


def test_linear8_of_a_row_that_is_nothing(env):
    torch, seq = env
    q = torch.zeros(3, 64, dtype=torch.int8, device="cuda")
    scale = torch.tensor([1.0, float("nan"), 0.0], device="cuda")
    w, ws, b = torch.ones(5, 64, dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda"), torch.arange(5.).cuda()
    y = seq.linear8(q, scale, w, ws, b, dtype=torch.float32)
    assert torch.equal(y[0], b) and y[1].isnan().all() and torch.equal(y[2], b)


# ------------------------------------------------------------- checkpoints
KEEPS = [(1, 1, 1), (1, 3, 5), (2, 64, 64), (1, 128, 3), (1, 129, 65), (7, 37, 331), (777, 1, 20), (3, 100, 924),
         (1, 300, 20001)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("with_lengths", [False, True])
@pytest.mark.parametrize("n,L,C", KEEPS)
def test_checkpoint(env, n, L, C, with_lengths, dtype):
    torch, seq = env
    s = Sample(torch, n + L + C, n, L, dtype, with_lengths)
    x, xv = s.normal(C, level=3 * s.rng.standard_normal(C))
    q, scale = seq.checkpoint(x, lengths=s.on_gpu)
    wq, wscale = lo.checkpoint(xv, s.live)
    same(q, wq, "q")
    same(scale, wscale, "scale")
    for out in DTYPES:
        back = seq.restore(q, scale, (n, L), dtype=getattr(torch, out), lengths=s.on_gpu)
        assert back.shape == (n, L, C)
        same(back, lo.restore(wq, wscale, n * L, s.live, out), out)


def test_checkpoint_strides_and_extremes(env):
    torch, seq = env
    wide = torch.randn(6, 50, 200, device="cuda")
    x = wide[:, :, 3:80].transpose(0, 1)
    x[1, 2, 5], x[40, 3, 6], x[:, :, 7], x[:, :, 8] = float("nan"), float("inf"), 0.0, 1e-36
    q, scale = seq.checkpoint(x)
    wq, wscale = lo.checkpoint(x.reshape(300, 77).cpu().numpy())
    same(q, wq, "q")
    same(scale, wscale, "scale")
    into = torch.full((6, 50, 200), 7.0, device="cuda")
    out = seq.restore(q, scale, (50, 6), out=into[:, :, 3:80].transpose(0, 1))
    same(out, lo.restore(wq, wscale, 300).reshape(50, 6, 77), "restored")
    assert (into[:, :, :3] == 7).all() and (into[:, :, 80:] == 7).all()
    assert out[1, 2, 5].isnan() and (out[:, :, 7] == 0).all()
    # steps past a length stay 0 where their channel's scale is NaN
    lengths = torch.tensor([3] * 50, dtype=torch.int32, device="cuda")
    out = seq.restore(q, scale, (50, 6), dtype=torch.float32, lengths=lengths)
    assert (out[:, 3:] == 0).all() and out[0, 0, 5].isnan()


# --------------------------------------------------------- weight gradient
GRADIENTS = [(1, 1, 1, 1), (1, 3, 2, 7), (2, 64, 64, 64), (1, 129, 65, 33), (7, 37, 131, 331), (3, 100, 192, 924),
             (1, 1000, 17, 300), (40, 70, 300, 40), (1, 64, 192, 2000), (2, 700, 2, 5000), (30, 129, 40, 530),
             (1, 9000, 5, 6)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("with_lengths", [False, True])
@pytest.mark.parametrize("n,L,N,C", GRADIENTS)
def test_weight_gradient(env, n, L, N, C, with_lengths, dtype):
    torch, seq = env
    s = Sample(torch, n + L + C + N, n, L, dtype, with_lengths)
    dy, dyv = s.normal(N, level=0.3)
    x, xv = s.normal(C, level=3 * s.rng.standard_normal(C), dtype="float32")
    q, scale = lo.checkpoint(xv, s.live)
    ops = torch.from_numpy(q).cuda(), torch.from_numpy(scale).cuda()
    dw, db = seq.linear_weight_gradient(dy, *ops, lengths=s.on_gpu)
    want = lo.linear_weight_gradient(dyv, q, scale, s.live)
    close(dw, want["dweight"], want["dweight_tol"], "dweight")
    close(db, want["dbias"], want["dbias_tol"], "dbias")
    dw2, db2 = seq.linear_weight_gradient(dy, *ops, lengths=s.on_gpu)
    assert torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient_keeps_every_digit(env, dtype):
    """Whole numbers whose sums stay below 2^24 come out exactly, 24-bit dy included."""
    torch, seq = env
    rng = np.random.default_rng(4)
    rows, N, C = 512, 70, 90
    dy = rng.integers(-3, 4, size=(rows, N)).astype(np.float32)
    q = rng.integers(-127, 128, size=(4, C, 128)).astype(np.int8)
    scale = 2.0 ** rng.integers(-2, 3, size=(4, C)).astype(np.float32)
    x = (q * scale[:, :, None]).transpose(0, 2, 1).reshape(rows, C)
    dw, db = seq.linear_weight_gradient(cuda(torch, dy, dtype), torch.from_numpy(q).cuda(), cuda(torch, scale))
    assert np.array_equal(host(dw), dy.T.astype(np.float64) @ x) and np.array_equal(host(db), dy.sum(0))
    if dtype == "float32":   # single products: 17 bits times 7
        dy = np.zeros((128, N), np.float32)
        dy[5] = (rng.integers(2 ** 16, 2 ** 17, size=N) * rng.choice([-1, 1], N)).astype(np.float32)
        q = np.zeros((1, C, 128), np.int8)
        q[0, :, 5] = rng.integers(-127, 128, size=C)
        dw, db = seq.linear_weight_gradient(cuda(torch, dy), torch.from_numpy(q).cuda(), torch.ones(1, C).cuda())
        assert np.array_equal(host(dw), np.outer(dy[5].astype(np.float64), q[0, :, 5]))
        assert np.array_equal(host(db), dy[5])


def test_weight_gradient_strides_and_extremes(env):
    torch, seq = env
    wide = torch.randn(20, 30, 99, device="cuda")
    dy = wide[:, :, 7:40].transpose(0, 1)
    q, scale = seq.checkpoint(torch.randn(600, 50, device="cuda"))
    want = seq.linear_weight_gradient(dy.contiguous(), q, scale)
    got = seq.linear_weight_gradient(dy, q, scale)
    rows = seq.linear_weight_gradient(dy.reshape(600, 33), q, scale)
    for a, b, c in zip(want, got, rows):
        assert torch.equal(a, b) and torch.equal(a, c)
    # a NaN channel of x is a NaN column, an infinite dy its channel's row
    scale[2, 11] = float("nan")
    bad = dy.contiguous()
    bad[3, 4, 9] = float("inf")
    dw, db = seq.linear_weight_gradient(bad, q, scale)
    assert dw[:, 11].isnan().all() and torch.isinf(db[9]) and not torch.isfinite(dw[9]).any()
    rest_m, rest_c = [m for m in range(33) if m != 9], [c for c in range(50) if c != 11]
    assert torch.equal(dw[rest_m][:, rest_c], want[0][rest_m][:, rest_c]) and torch.equal(db[rest_m], want[1][rest_m])


@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient_scales_far_apart(env, dtype):
    """Blocks whose scales differ by 2^100 and more, scales of 0 over values that are
    not, a channel's scales all 0, negative ones: each as the formula has it."""
    torch, seq = env
    rng = np.random.default_rng(6)
    blocks, N, C = 12, 70, 90
    rows = blocks * 128 - 50
    q = rng.integers(-127, 128, size=(blocks, C, 128)).astype(np.int8)
    scale = (2.0 ** rng.integers(-60, 60, size=(blocks, C)) * rng.choice([-1, 1], (blocks, C))).astype(np.float32)
    scale[rng.random((blocks, C)) < 0.3] = 0.0
    scale[:, 7] = 0.0
    scale[:, :5] = (0.5 + rng.random((blocks, 5))).astype(np.float32)
    dy = cuda(torch, rng.standard_normal((rows, N)), dtype)
    dyv = values(dy)
    dw, db = seq.linear_weight_gradient(dy, torch.from_numpy(q).cuda(), cuda(torch, scale))
    want = lo.linear_weight_gradient(dyv, q, scale)
    close(dw, want["dweight"], want["dweight_tol"], "dweight")
    assert (dw[:, 7] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient_error_of_many_rows(env, dtype):
    """20,000 rows: off by less than 1e-6 of the whole in the 2-norm (terms add at random
    signs, each partial sum rounds to 2^-24 of what it has come to)."""
    torch, seq = env
    dy = torch.randn(20000, 64, device="cuda").to(getattr(torch, dtype))
    q, scale = seq.checkpoint(torch.randn(20000, 96, device="cuda"))
    dw, db = seq.linear_weight_gradient(dy, q, scale)
    x = (q.double() * scale.double()[:, :, None]).transpose(1, 2).reshape(-1, 96)[:20000]
    want = dy.double().t() @ x
    assert float((dw.double() - want).norm() / want.norm()) < 1e-6
    want = dy.double().sum(0)
    assert float((db.double() - want).norm() / want.norm()) < 1e-6


# many rows: staged tiles of 32, 64, 128 and 256 channels of dy, whole and cut off; dy laid
# out anew (odd channels, fp32)
MANY = [(40000, 20, 3000), (40000, 50, 3000), (30000, 128, 2000), (30000, 300, 1000), (30009, 301, 999),
        (40005, 17, 3001), (50001, 63, 2000), (20001, 129, 2500)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["plain", "ragged", "far"])
@pytest.mark.parametrize("rows,N,C", MANY)
def test_weight_gradient_many_rows(env, rows, N, C, kind, dtype):
    """Against 64-bit products on the GPU, within the oracle's bound.  far: blocks whose
    scales differ by 2^60 and more, scales of 0 over values that are not."""
    torch, seq = env
    g = torch.Generator(device="cuda").manual_seed(rows + N + C)
    n = next(k for k in (8, 7, 3, 1) if rows % k == 0) if kind == "ragged" else 1
    L, blocks = rows // n, -(-rows // 128)
    q = torch.randint(-127, 128, (blocks, C, 128), generator=g, device="cuda", dtype=torch.int8)
    scale = torch.rand(blocks, C, generator=g, device="cuda") + 0.5
    if kind == "far":
        scale *= 2.0 ** torch.randint(-40, 40, (blocks, C), generator=g, device="cuda").float()
        scale[torch.rand(blocks, C, generator=g, device="cuda") < 0.2] = 0.0
        scale[:, C // 2:] = 1.0 + scale[:, C // 2:].clamp(max=1.0)
    dy = torch.randn(n, L, N, generator=g, device="cuda").to(getattr(torch, dtype))
    lengths, live = None, torch.ones(n, L, 1, dtype=torch.bool, device="cuda")
    if kind == "ragged":
        lengths = torch.randint(0, L + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        live = (torch.arange(L, device="cuda")[None, :] < lengths[:, None])[:, :, None]
        dy.masked_fill_(~live, float("nan"))
    dw, db = seq.linear_weight_gradient(dy, q, scale, lengths=lengths)
    d = torch.where(live, dy.double(), 0.0).view(rows, N)
    x = (q.double() * scale.double()[:, :, None]).transpose(1, 2).reshape(-1, C)[:rows]
    want = d.t().contiguous() @ x
    # a product enters a block's sum of at most 384, rounded or cut off, then at most
    # `blocks` sums and multiplications and as many joins
    units = 2 * 384 + 4 * blocks
    tol = (d.abs().t().contiguous() @ x.abs()) * units * lo.U
    assert ((dw.double() - want).abs() <= tol).all()
    if kind != "far":   # and by far less as a whole: each rounding at random
        assert float((dw.double() - want).norm() / want.norm()) < 1e-6
    want = d.sum(0)
    assert ((db.double() - want).abs() <= d.abs().sum(0) * 3 * rows * lo.U).all()
    assert float((db.double() - want).norm() / want.norm()) < 1e-6
    again = seq.linear_weight_gradient(dy, q, scale, lengths=lengths)
    assert torch.equal(dw, again[0]) and torch.equal(db, again[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("first,N", [(0, 300), (1, 300), (2, 301), (7, 299)])
def test_weight_gradient_many_rows_of_wider_ones(env, first, N, dtype):
    """dy as columns of a wider matrix, rows turned about: aligned to a value only, as they
    stand or laid out anew; NaN beside them does not reach the result."""
    torch, seq = env
    wide = torch.full((200, 150, 312), float("nan"), device="cuda").to(getattr(torch, dtype))
    dy = wide[:, :, first:first + N]
    dy.copy_(torch.randn(200, 150, N, device="cuda"))
    q, scale = seq.checkpoint(torch.randn(30000, 520, device="cuda"))
    want = seq.linear_weight_gradient(dy.contiguous(), q, scale)
    for a, b in zip(want, seq.linear_weight_gradient(dy, q, scale)):
        assert torch.equal(a, b)
    turned = dy.transpose(0, 1)
    want = seq.linear_weight_gradient(turned.contiguous(), q, scale)
    for a, b in zip(want, seq.linear_weight_gradient(turned, q, scale)):
        assert torch.equal(a, b)
    # one row for all of them
    same_row = dy[3, 4].expand(200, 150, N)
    for a, b in zip(seq.linear_weight_gradient(same_row.contiguous(), q, scale),
                    seq.linear_weight_gradient(same_row, q, scale)):
        assert torch.equal(a, b)


def test_weight_gradient_many_rows_nothing_finite(env):
    """NaN scales and infinite dy reach their column and row, and no others."""
    torch, seq = env
    dy = torch.randn(30000, 256, device="cuda").bfloat16()
    q, scale = seq.checkpoint(torch.randn(30000, 512, device="cuda"))
    want = seq.linear_weight_gradient(dy, q, scale)
    scale[100, 11], scale[0, 12], scale[234, 13] = float("nan"), float("nan"), float("nan")
    dy[20000, 9] = float("inf")
    dw, db = seq.linear_weight_gradient(dy, q, scale)
    assert dw[:, 11:14].isnan().all() and torch.isinf(db[9]) and not torch.isfinite(dw[9]).any()
    rest_m, rest_c = [m for m in range(256) if m != 9], [c for c in range(512) if not 11 <= c <= 13]
    assert torch.equal(dw[rest_m][:, rest_c], want[0][rest_m][:, rest_c]) and torch.equal(db[rest_m], want[1][rest_m])


# -------------------------------------------------------------- all of them
def block(seq, x, r, w, wq, ws, b, lengths=None, dtype=None):
    """Norm in 8 bits, product, checkpoint of the sum: a layer's forward pass."""
    q, scale, total, rstd = seq.rms_norm8(x, w, residual=r, lengths=lengths)
    y = seq.linear8(q, scale, wq, ws, b, dtype=dtype or x.dtype, lengths=lengths)
    return y, total, rstd, seq.checkpoint(total, lengths=lengths)


def layer(torch, n, L, C, N, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    t = getattr(torch, dtype)
    return rand(n, L, C).to(t), rand(n, L, C).to(t), 1 + 0.1 * rand(C), rand(N, C) / C ** 0.5, rand(N)


@pytest.mark.parametrize("n,L,C,N", [(1, 1, 2000, 192), (6, 33, 257, 100), (2, 500, 924, 331)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_layer_forward_and_backward(env, n, L, C, N, dtype):
    """The operators in a row against 64-bit autograd of the layer without 8 bits: what
    8 bits lose is half a step of 1 / 127 of a row's (a channel's) largest value."""
    torch, seq = env
    x, r, w, W, b = layer(torch, n, L, C, N, dtype)
    wq, ws = seq.quantize_rows(W)
    lengths = torch.tensor([max(0, L - 7 * i) for i in range(n)], dtype=torch.int32, device="cuda")
    y, total, rstd, (kq, ks) = block(seq, x, r, w, wq, ws, b, lengths)
    live = (torch.arange(L, device="cuda")[None, :] < lengths[:, None])[:, :, None]
    xd, wd, Wd, bd = (t.double().requires_grad_(True) for t in (total, w, W, b))
    norm = xd * (xd.square().mean(2, keepdim=True) + 1e-5).rsqrt() * wd
    want = norm @ Wd.t() + bd
    # |error| of a product of C terms: half a step a factor, all of one sign at worst
    top, wtop = norm.abs().amax(2, keepdim=True), Wd.abs().amax(1)
    tol = (norm.abs().sum(2, keepdim=True) * wtop + top * Wd.abs().sum(1)) * 0.5 / 127 * 1.01
    tol = tol + want.abs() * torch.finfo(y.dtype).eps + 1e-6
    assert (((y.double() - want).abs() <= tol) | ~live).all() and (y[~live.expand_as(y)] == 0).all()
    dy = torch.randn(n, L, N, device="cuda").to(y.dtype)
    want.backward(torch.where(live, dy.double(), 0.0))
    dnorm = (torch.where(live, dy, torch.zeros_like(dy)).float() @ W).to(x.dtype)
    dx, dw = seq.rms_norm_backward(dnorm, total, rstd, w, lengths=lengths)
    # dnorm was rounded to its type
    scale = float(xd.grad.abs().max()) + 1e-30
    assert float((dx.double() - xd.grad).abs().max()) <= scale * (0.02 if dtype != "float32" else 1e-4)
    # a checkpoint of the normalised rows gives W's gradient
    normed, _, _ = seq.rms_norm(total, w, lengths=lengths)
    kq, ks = seq.checkpoint(normed, lengths=lengths)
    dW, db = seq.linear_weight_gradient(dy, kq, ks, lengths=lengths)
    step = ks.double().repeat_interleave(128, 0)[:n * L] * 0.51 + normed.abs().double().view(n * L, C) * 2 ** -8
    tol = torch.where(live, dy, torch.zeros_like(dy)).double().abs().view(n * L, N).t() @ step + 1e-4
    assert ((dW.double() - Wd.grad).abs() <= tol).all()
    assert float((db.double() - bd.grad).abs().max()) <= 1e-4 * (1 + float(bd.grad.abs().max()))


def test_captured_calls_replay(env):
    """Two graphs of a layer that share no memory of theirs but the inputs, replayed in
    turn with eager work between, and new inputs in the captured places."""
    torch, seq = env
    ops = layer(torch, 5, 70, 300, 90, "bfloat16")
    wq, ws = seq.quantize_rows(ops[3])
    dy = torch.randn(5, 70, 90, device="cuda").bfloat16()

    def run():
        y, total, rstd, kept = block(seq, *ops[:3], wq, ws, ops[4])
        dx, dw = seq.rms_norm_backward(ops[0], total, rstd, ops[2], dtotal=ops[1])
        return (y, total, rstd, dx, dw, seq.restore(*kept, (5, 70))) + tuple(seq.linear_weight_gradient(dy, *kept))

    run()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = run()
        graphs.append((g, got))
    for turn in range(4):
        new = layer(torch, 5, 70, 300, 90, "bfloat16", seed=turn + 1)
        for a, b in zip(ops[:3], new[:3]):
            a.copy_(b)
        want = run()
        torch.cuda.synchronize()
        for g, got in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            for a, b in zip(got, want):
                assert torch.equal(a, b)


def test_calls_on_a_stream(env):
    torch, seq = env
    ops = layer(torch, 3, 40, 200, 60, "float32")
    wq, ws = seq.quantize_rows(ops[3])
    want = block(seq, *ops[:3], wq, ws, ops[4])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    q, scale, total, rstd = seq.rms_norm8(ops[0], ops[2], residual=ops[1], stream=side)
    y = seq.linear8(q, scale, wq, ws, ops[4], dtype=torch.float32, stream=side)
    kq, ks = seq.checkpoint(total, stream=side)
    back = seq.restore(kq, ks, (3, 40), dtype=torch.float32, stream=side)
    dx, dw = seq.rms_norm_backward(ops[0], total, rstd, ops[2], stream=side)
    dW, db = seq.linear_weight_gradient(y, kq, ks, stream=side)
    q2, s2 = seq.quantize_rows(ops[3], stream=side)
    n1, _, _ = seq.rms_norm(ops[0], ops[2], stream=side)
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(total, want[1]) and torch.equal(kq, want[3][0])
    assert torch.equal(back, seq.restore(*want[3], (3, 40), dtype=torch.float32))
    assert torch.equal(q2, wq) and torch.equal(n1, seq.rms_norm(ops[0], ops[2])[0])
    assert torch.equal(dW, seq.linear_weight_gradient(y, kq, ks)[0])
    assert torch.equal(dx, seq.rms_norm_backward(ops[0], total, rstd, ops[2])[0])


def test_no_rows(env):
    torch, seq = env
    for leading in ((0, 5), (5, 0), (0,)):
        x = torch.zeros(*leading, 9, device="cuda")
        assert seq.rms_norm(x)[0].shape == x.shape
        q, scale, _, rstd = seq.rms_norm8(x)
        w, ws = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
        assert seq.linear8(q, scale, w, ws).shape == (*leading, 4)
        dx, dw = seq.rms_norm_backward(x, x, rstd)
        assert dx.shape == x.shape and (dw == 0).all()
        kq, ks = seq.checkpoint(x)
        assert kq.shape == (0, 9, 128) and seq.restore(kq, ks, leading).shape == x.shape
        dW, db = seq.linear_weight_gradient(x, kq, ks)
        assert dW.shape == (9, 9) and (dW == 0).all() and (db == 0).all()


def test_operands_that_require_gradients_are_refused(env):
    torch, seq = env
    x, w, r = torch.randn(2, 6, 8, device="cuda"), torch.ones(8, device="cuda"), torch.ones(2, 6, device="cuda")
    q, s, _, _ = seq.rms_norm8(x)
    wq, ws = seq.quantize_rows(torch.randn(8, 8, device="cuda"))
    kq, ks = seq.checkpoint(x)
    for call, operands in ((lambda x, r, w: seq.rms_norm(x, w, residual=r), (x, x, w)),
                           (lambda x, r, w: seq.rms_norm8(x, w, residual=r), (x, x, w)),
                           (lambda dy, t, k, w, dt: seq.rms_norm_backward(dy, t, k, w, dtotal=dt), (x, x, r, w, x)),
                           (lambda x: seq.quantize_rows(x), (x,)),
                           (lambda s, ws, b: seq.linear8(q, s, wq, ws, b), (s, ws, w)),
                           (lambda x: seq.checkpoint(x), (x,)), (lambda s: seq.restore(kq, s, (2, 6)), (ks,)),
                           (lambda dy, s: seq.linear_weight_gradient(dy, kq, s), (x, ks))):
        call(*operands)
        for k in range(len(operands)):
            wanting = [t.clone().requires_grad_(True) if i == k else t for i, t in enumerate(operands)]
            with pytest.raises(ValueError, match="requires gradients"):
                call(*wanting)
            with torch.no_grad():
                call(*wanting)


def test_refusals_of_the_binding(env):
    torch, seq = env
    x, r = torch.randn(2, 6, 8, device="cuda"), torch.ones(2, 6, device="cuda")
    q, s, _, _ = seq.rms_norm8(x)
    wq, ws = seq.quantize_rows(torch.randn(8, 8, device="cuda"))
    kq, ks = seq.checkpoint(x)
    t = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    for call in (lambda: seq.rms_norm(x[0], lengths=t), lambda: seq.rms_norm(x, residual=x.half()),
                 lambda: seq.rms_norm(x, torch.ones(9, device="cuda")), lambda: seq.rms_norm(x, total_out=x.clone()),
                 lambda: seq.rms_norm(x, out=x.half()), lambda: seq.rms_norm(x.double()),
                 lambda: seq.rms_norm(x.transpose(1, 2)), lambda: seq.rms_norm(x[0, 0]),
                 lambda: seq.rms_norm_backward(x, x, r[:1]), lambda: seq.rms_norm_backward(x.half(), x, r),
                 lambda: seq.linear8(q.float(), s, wq, ws), lambda: seq.linear8(q, s[:1], wq, ws),
                 lambda: seq.linear8(q, s, wq, ws[:4]), lambda: seq.linear8(q[:, :, :32].contiguous(), s, wq, ws),
                 lambda: seq.linear8(q, s, wq, ws, dtype=torch.float64), lambda: seq.linear8(q[:, ::2], s[:, ::2], wq, ws),
                 lambda: seq.linear8(q[0], s[0], wq, ws, lengths=t), lambda: seq.linear8(q, s, wq, ws, lengths=t[:1]),
                 lambda: seq.linear8(q, s, wq, ws, out=x.half()[:, :, :7]),
                 lambda: seq.restore(kq, ks, (3, 60)), lambda: seq.restore(kq, ks, (2, 3, 4)),
                 lambda: seq.restore(kq, ks, (12,), lengths=t), lambda: seq.restore(kq, ks[:, :3], (2, 6)),
                 lambda: seq.linear_weight_gradient(x.view(1, 12, 8).expand(20, 12, 8), kq, ks),
                 lambda: seq.linear_weight_gradient(x, kq, ks.half())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: seq.rms_norm_backward(x, x, None), lambda: seq.linear8(q, None, wq, ws),
                 lambda: seq.linear8(q, s, None, ws), lambda: seq.restore(kq, None, (2, 6)),
                 lambda: seq.restore(ks, ks, (2, 6)), lambda: seq.checkpoint(x.cpu())):
        with pytest.raises(TypeError):
            call()


def test_outputs_over_saved_tensors_are_noticed(env):
    torch, seq = env
    x = torch.randn(2, 6, 8, device="cuda")
    _, _, rstd = seq.rms_norm(x)
    q, s, _, _ = seq.rms_norm8(x)
    wq, ws = seq.quantize_rows(torch.randn(8, 8, device="cuda"))
    kq, ks = seq.checkpoint(x)
    for call in (lambda t: seq.rms_norm(x, out=t), lambda t: seq.rms_norm(x, residual=x, total_out=t),
                 lambda t: seq.rms_norm8(x, residual=x, total_out=t), lambda t: seq.rms_norm_backward(x, x, rstd, out=t),
                 lambda t: seq.linear8(q, s, wq, ws, out=t), lambda t: seq.restore(kq, ks, (2, 6), out=t)):
        saved = x.clone()
        w = torch.ones_like(x, requires_grad=True)
        loss = (saved * w).sum()
        call(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
