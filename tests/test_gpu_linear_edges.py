"""Operators around linear layers on the GPU at the limits of what their definitions
promise: values halfway between two 8-bit ones."""
import numpy as np
import pytest

from oracle import linear_oracle as lo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2601_17091_amd as rk
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    rk.library()
    return torch, rk.sequence


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_8_bit_values_halfway_between_two(env, dtype):
    """Rows whose largest value is a multiple of 127, so that many others lie halfway, and half
    the largest of any: the oracle's operations to the bit, in rows and in checkpoints."""
    torch, seq = env
    rng = np.random.default_rng(12)
    bits = 8 if dtype == "bfloat16" else 11
    top = rng.integers(1, 2 ** bits // 127 + 1, size=(300, 1)) * 127
    top[150:] = rng.integers(1, 2 ** bits, size=(150, 1))
    v = np.concatenate([rng.integers(-2 * top, 2 * top + 1, size=(300, 126)) / 2, top / 2, top], 1).astype(np.float32)
    v = np.clip(lo.to_type(v, dtype), -top, top).astype(np.float32)
    x = torch.from_numpy(v).to(getattr(torch, dtype)).cuda()
    q, scale = seq.quantize_rows(x)
    want, wscale = lo.quantize_rows(v)
    assert np.array_equal(q.cpu().numpy(), want) and np.array_equal(scale.cpu().numpy(), wscale)
    kq, ks = seq.checkpoint(x.t().contiguous())   # 128 rows, 300 channels
    want, wscale = lo.checkpoint(np.ascontiguousarray(v.T))
    assert np.array_equal(kq.cpu().numpy(), want) and np.array_equal(ks.cpu().numpy(), wscale)
    q = q.cpu().numpy()[:, :128].astype(np.int64)
    assert (np.abs(127 * np.rint(2 * v).astype(np.int64) - 2 * q * top) <= top).all()


# threads of a row from 128 to 1,024, held in registers, summed aside, and read twice
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("C", [1500, 2500, 5000, 10000, 20000, 25000])
def test_rms_norm_rows_without_data_between_others(env, C, dtype):
    """Workgroups that go from row to row, with any number of rows without data between two
    that hold some: each row's results are those of a call without such rows."""
    torch, seq = env
    g = torch.Generator(device="cuda").manual_seed(C)
    rows = 2500
    lengths = torch.randint(0, 2, (rows,), generator=g, device="cuda", dtype=torch.int32)
    live = lengths.bool()
    rand = lambda: torch.randn(rows, 1, C, generator=g, device="cuda").to(getattr(torch, dtype))  # noqa: E731
    x, r, dy, dt = rand(), rand(), rand(), rand()
    x *= 1 + torch.rand(rows, 1, 1, generator=g, device="cuda").to(x.dtype) * 9   # no row's sum is another's
    w = 1 + 0.2 * torch.randn(C, generator=g, device="cuda")
    own = [t[live].clone() for t in (x, r, dy, dt)]
    for t in (x, r, dy, dt):
        t[~live] = float("nan")
    for _ in range(3):
        y, total, rstd = seq.rms_norm(x, w, residual=r, lengths=lengths)
        q, scale, _, rstd8 = seq.rms_norm8(x, w, residual=r, lengths=lengths)
        qx, sx = seq.quantize_rows(x, lengths=lengths)
        dx, dw = seq.rms_norm_backward(dy, total, rstd, w, dtotal=dt, lengths=lengths)
        y1, total1, rstd1 = seq.rms_norm(own[0], w, residual=own[1])
        q1, scale1, _, _ = seq.rms_norm8(own[0], w, residual=own[1])
        qx1, sx1 = seq.quantize_rows(own[0])
        dx1, dw1 = seq.rms_norm_backward(own[2], total1, rstd1, w, dtotal=own[3])
        for got, want in ((y, y1), (total, total1), (rstd, rstd1), (q, q1), (scale, scale1), (rstd8, rstd1), (qx, qx1),
                          (sx, sx1), (dx, dx1)):
            assert torch.equal(got[live], want) and (got[~live] == 0).all()
        # sums of at most 2,500 terms in two orders, 2^-24 of the terms for each
        terms = (own[2].double() * total1.double() * rstd1.double()[:, :, None]).abs().sum((0, 1))
        assert ((dw.double() - dw1.double()).abs() <= 2 * (rows + 2) * lo.U * terms).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("N,C", [(2000, 6000), (4096, 4096), (1536, 20000)])
def test_weight_gradient_of_no_rows_of_a_large_layer(env, N, C, dtype):
    """Zeros, and nothing is read: the checkpoint of no rows has no memory."""
    torch, seq = env
    q, scale = torch.empty(0, C, 128, dtype=torch.int8, device="cuda"), torch.empty(0, C, device="cuda")
    for leading in ((0, 5), (5, 0), (0,)):
        dy = torch.empty(*leading, N, dtype=getattr(torch, dtype), device="cuda")
        ways = [None] if len(leading) == 1 else [None, torch.zeros(leading[0], dtype=torch.int32, device="cuda")]
        for lengths in ways:
            dw, db = seq.linear_weight_gradient(dy, q, scale, lengths=lengths)
            assert dw.shape == (N, C) and (dw == 0).all() and (db == 0).all()


# staged tiles of 32, 64, 128 and 256 channels of dy (as they lie and laid out anew), and the
# direct way
DRIFTS = [(40000, 20, 3000), (40000, 50, 3000), (30000, 128, 2000), (30000, 300, 1000), (30009, 301, 999), (1536, 40, 90)]


def drifting(torch, kind, blocks):
    """Scales [blocks, 1] that move by less than 2^40 a block, by 2^117 and more in a few."""
    b = torch.arange(blocks, device="cuda")
    turns = {"falls": 60 - 39 * (b % 4), "rises": 39 * (b % 4) - 60, "falls slowly": 100 - 19 * (b % 11),
             "to and fro": torch.where(b % 8 < 4, 60 - 39 * (b % 4), 39 * (b % 4) - 57)}
    return (2.0 ** turns[kind].float())[:, None]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["falls", "rises", "falls slowly", "to and fro"])
@pytest.mark.parametrize("rows,N,C", DRIFTS)
def test_weight_gradient_of_drifting_scales(env, rows, N, C, kind, dtype):
    """A channel that fades along the rows, or grows: what an early block gave stays, also
    where no later one adds to it."""
    torch, seq = env
    g = torch.Generator(device="cuda").manual_seed(rows + N + C)
    blocks = -(-rows // 128)
    q = torch.randint(-127, 128, (blocks, C, 128), generator=g, device="cuda", dtype=torch.int8)
    scale = (torch.rand(blocks, C, generator=g, device="cuda") * 0.25 + 1) * drifting(torch, kind, blocks)
    scale[:, C // 2:] = 1.0 + scale[:, C // 2:].clamp(max=1.0)   # ordinary ones beside them
    dy = torch.randn(rows, N, generator=g, device="cuda").to(getattr(torch, dtype))
    for m in range(0, N, 3):   # channels that only every 16th block reaches
        dy[:, m] *= ((torch.arange(rows, device="cuda") // 128 + m // 3) % 16 == 0).to(dy.dtype)
    dw, db = seq.linear_weight_gradient(dy, q, scale)
    d = dy.double()
    x = (q.double() * scale.double()[:, :, None]).transpose(1, 2).reshape(-1, C)[:rows]
    want = d.t().contiguous() @ x
    # a product enters a block's sum of at most 384, rounded or cut off, then at most
    # `blocks` sums and multiplications and as many joins
    tol = (d.abs().t().contiguous() @ x.abs()) * (2 * 384 + 4 * blocks) * lo.U
    assert ((dw.double() - want).abs() <= tol).all()
    assert ((db.double() - d.sum(0)).abs() <= d.abs().sum(0) * 3 * rows * lo.U).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["even", "far", "falls"])
def test_weight_gradient_keeps_infinities(env, kind, dtype):
    """An infinite dy gives infinities of its products' signs (NaN where it meets a 0), whatever
    the scales of later blocks are; a finite channel is not touched."""
    torch, seq = env
    rows, N, C = 30000, 300, 1000
    g = torch.Generator(device="cuda").manual_seed(9)
    blocks = -(-rows // 128)
    q = torch.randint(-127, 128, (blocks, C, 128), generator=g, device="cuda", dtype=torch.int8)
    scale = torch.rand(blocks, C, generator=g, device="cuda") + 0.5
    if kind == "far":
        scale *= 2.0 ** (60.0 * (torch.arange(blocks, device="cuda") % 2))[:, None]
    elif kind == "falls":
        scale *= drifting(torch, kind, blocks)
    dy = torch.randn(rows, N, generator=g, device="cuda").to(getattr(torch, dtype))
    want = seq.linear_weight_gradient(dy, q, scale)
    at = {7: (130, float("inf")), 100: (5 * 128 + 3, float("-inf")), 299: (0, float("inf"))}
    for m, (row, value) in at.items():
        dy[row, m] = value
    dw, db = seq.linear_weight_gradient(dy, q, scale)
    for m, (row, value) in at.items():
        met = q[row // 128, :, row % 128].float() * value   # NaN for 0
        assert torch.equal(dw[m].isnan(), met.isnan()) and torch.equal(dw[m][met != 0].nan_to_num(0.0, 1.0, -1.0),
                                                                       met[met != 0].nan_to_num(0.0, 1.0, -1.0))
        assert db[m] == value
    rest = [m for m in range(N) if m not in at]
    assert torch.equal(dw[rest], want[0][rest]) and torch.equal(db[rest], want[1][rest])


@pytest.mark.parametrize("N", [2 ** 24, 2 ** 24 - 7, 2 ** 24 - 8])
def test_weight_gradient_of_the_widest_rows(env, N):
    """A stage of rows that are laid out 2^25 bytes apart reaches 2^31."""
    torch, seq = env
    rows, C = 130, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    dy = torch.randn(rows, N, generator=g, device="cuda", dtype=torch.bfloat16)
    q, scale = seq.checkpoint(torch.randn(rows, C, generator=g, device="cuda"))
    dw, db = seq.linear_weight_gradient(dy, q, scale)
    x = (q.double() * scale.double()[:, :, None]).transpose(1, 2).reshape(-1, C)[:rows]
    for part in (slice(0, 300), slice(N // 2 - 300, N // 2 + 300), slice(N - 300, N)):
        d = dy[:, part].double()
        tol = (d.abs().t().contiguous() @ x.abs()) * (2 * rows + 18) * lo.U
        assert ((dw[part].double() - d.t().contiguous() @ x).abs() <= tol).all()
        assert ((db[part].double() - d.sum(0)).abs() <= d.abs().sum(0) * (3 * rows + 2) * lo.U).all()


# rows and channels of each way that takes the most columns: few rows, columns shared out,
# tiles of 128 and of 64 channels; live rows listed and not
@pytest.mark.parametrize("n,L,N", [(1, 1, 1), (1, 64, 33), (1, 130, 70), (1, 300, 192), (2, 900, 192), (1, 7000, 513),
                                   (2, 3500, 1300), (5, 700, 2000), (1, 20000, 17)])
def test_linear8_of_the_largest_sums(env, n, L, N):
    """-128 by -128 at 131,072 columns is 2^31, one more than 32 bits hold; with one value
    less, or at 131,008 columns, it is not."""
    torch, seq = env
    most = 131072
    one = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    q = torch.full((n, L, most), -128, dtype=torch.int8, device="cuda")
    p = torch.full((N, most), -128, dtype=torch.int8, device="cuda")
    q[:, 1::5] = 127
    p[1::3] = 127
    q[:, 2::5, 99] = -127
    lengths = torch.full((n,), L, dtype=torch.int32, device="cuda")
    lengths[0] = L // 2 + 1
    live = (torch.arange(L, device="cuda")[None, :] < lengths[:, None])[:, :, None]
    for columns in (most, most - 64):
        # whole numbers below 2^53 whatever their order
        kinds = q[0, :3, :columns].double() @ p[:2, :columns].double().t().contiguous()
        row, col = torch.arange(L, device="cuda") % 5, torch.arange(N, device="cuda") % 3
        row = torch.where(row > 2, torch.zeros_like(row), row)
        want = kinds[row.clamp(max=kinds.shape[0] - 1)][:, (col == 1).long().clamp(max=kinds.shape[1] - 1)]
        y = seq.linear8(q[:, :, :columns].contiguous(), one(n, L), p[:, :columns].contiguous(), one(N), dtype=torch.float32)
        assert torch.equal(y, want.float().expand(n, L, N))
        y = seq.linear8(q[:, :, :columns].contiguous(), one(n, L), p[:, :columns].contiguous(), one(N),
                        dtype=torch.bfloat16, lengths=lengths)
        assert torch.equal(y, torch.where(live, want.float().bfloat16().expand(n, L, N), 0))
    assert float(seq.linear8(q[:, :1].contiguous(), one(n, 1), p, one(N), dtype=torch.float32)[0, 0, 0]) == 2.0 ** 31


def test_a_norm_and_its_sum_in_one_tensor_are_refused(env):
    from paper_2601_17091_amd.rocket import RocketError
    torch, seq = env
    x, r = torch.randn(3, 5, 8, device="cuda"), torch.randn(3, 5, 8, device="cuda")
    for t in (torch.empty_like(x), x, r):
        with pytest.raises(RocketError):
            seq.rms_norm(x, residual=r, out=t, total_out=t)


def test_a_norm_in_place_gives_no_sum(env):
    """x is written over, so that it is not what was normalised; the gradient's call says so."""
    torch, seq = env
    x = torch.randn(3, 5, 8, device="cuda")
    want, total, rstd = seq.rms_norm(x)
    assert total is x
    for view in (x.clone(), x.clone().view(15, 8)):
        for out in (view, view.view(view.shape)):
            kept = view.clone()
            y, total, k = seq.rms_norm(view, out=out)
            assert y is out and total is None and torch.equal(y.view(3, 5, 8), want) and torch.equal(k.view(3, 5), rstd)
            with pytest.raises(TypeError):
                seq.rms_norm_backward(y, total, k)
            view.copy_(kept)
    # with a residual the sum has a place of its own
    r = torch.randn(3, 5, 8, device="cuda")
    y, total, _ = seq.rms_norm(x.clone(), residual=r)
    z = x.clone()
    y2, total2, _ = seq.rms_norm(z, residual=r, out=z)
    assert torch.equal(y, y2) and torch.equal(total, total2)
    empty = torch.empty(0, 5, 8, device="cuda")
    assert seq.rms_norm(empty)[1] is empty
