"""Group norm's backward pass where groups or levels differ: what one group
holds does not reach another's gradients, on every way a call is cut."""
import numpy as np
import pytest

from oracle import sequence_oracle as so
from test_gpu_sequence import close, env, f32, host, typed  # noqa: F401

pytestmark = pytest.mark.gpu

# n, L, C, groups: held, groups of whole columns; held, columns in two groups;
# held, rows of less than 16 bytes; chunks of several groups; chunks of narrow
# rows; groups wider than a workgroup's columns
CUTS = [(3, 50, 64, 4), (3, 50, 33, 11), (4, 40, 6, 3), (2, 5000, 64, 16), (2, 5000, 6, 3), (2, 300, 4100, 2)]


def backward(torch, seq, x, dy, G, w, b, act):
    _, mean, rstd = seq.group_norm(x, G, w, b, activation=act)
    return (mean, rstd) + seq.group_norm_backward(dy, x, G, mean, rstd, w, b, activation=act)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("group", [0, -1])
@pytest.mark.parametrize("dtype,act", [("float32", "silu"), ("bfloat16", "relu"), ("float16", "gelu")])
@pytest.mark.parametrize("n,L,C,G", CUTS)
def test_infinities_and_nan_stay_in_their_group(env, n, L, C, G, dtype, act, group, bad):  # noqa: F811
    torch, seq = env
    dt, width = getattr(torch, dtype), C // G
    x, dy = (torch.randn(n, L, C, device="cuda").to(dt) for _ in range(2))
    w, b = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-0.2, 0.2, C, device="cuda")
    _, _, *clean = backward(torch, seq, x, dy, G, w, b, act)
    at = group % G * width
    own = torch.zeros(C, dtype=torch.bool, device="cuda")
    own[at:at + width] = True
    for t in (x, dy):   # in x the group's mean is lost, in dy its gradients only
        was = t[1, L // 2, at + width // 2].clone()
        t[1, L // 2, at + width // 2] = bad
        _, _, dx, dw, db = backward(torch, seq, x, dy, G, w, b, act)
        t[1, L // 2, at + width // 2] = was
        assert torch.equal(dx[:, :, ~own], clean[0][:, :, ~own])
        assert torch.equal(dw[~own], clean[1][~own]) and torch.equal(db[~own], clean[2][~own])
        others = [i for i in range(n) if i != 1]
        assert torch.equal(dx[others], clean[0][others])
        assert not torch.isfinite(dx[1, :, own]).any() if t is x else not torch.isfinite(dw[own]).all()


@pytest.mark.parametrize("level", [1e4, 1e6])
@pytest.mark.parametrize("dtype,act", [("float32", "silu"), ("float32", "relu"), ("bfloat16", "gelu")])
@pytest.mark.parametrize("n,L,C,G", CUTS)
def test_groups_of_unequal_levels(env, n, L, C, G, dtype, act, level):  # noqa: F811
    """The first group at a level far above the others', which lie near 0: their
    gradients are as near to the formula's as without it."""
    torch, seq = env
    rng = np.random.default_rng(n + L + C)
    width = C // G
    raw = rng.standard_normal((n, L, C))
    raw[:, :, :width] += level
    x, xv = typed(torch, raw, dtype)
    dy, dyv = typed(torch, rng.standard_normal((n, L, C)), dtype)
    w = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    b = (0.2 * rng.standard_normal(C)).astype(np.float32)
    mean, rstd, dx, dw, db = backward(torch, seq, x, dy, G, f32(torch, w), f32(torch, b), act)
    want = so.group_norm_backward(dyv, xv, G, host(mean), host(rstd), w, b, activation=act, dtype=dtype)
    near = slice(width, C)
    close(dx[:, :, near], want["dx"][:, :, near], want["dx_tol"][:, :, near], "dx")
    close(dw[near], want["dweight"][near], want["dweight_tol"][near], "dweight")
    close(db[near], want["dbias"][near], want["dbias_tol"][near], "dbias")


@pytest.mark.parametrize("dtype,level", [("float32", 1e3), ("float32", 1e4), ("float32", 1e5), ("float16", 1e3)])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("n,L,C,G", CUTS)
def test_level_far_above_the_spread(env, n, L, C, G, act, dtype, level):  # noqa: F811
    """All values far above their spread of 1: x - m loses nothing, and neither
    do the gradients."""
    torch, seq = env
    rng = np.random.default_rng(n + L + C + 1)
    x, xv = typed(torch, level + rng.standard_normal((n, L, C)), dtype)
    dy, dyv = typed(torch, rng.standard_normal((n, L, C)), dtype)
    w = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    b = (0.2 * rng.standard_normal(C)).astype(np.float32)
    mean, rstd, dx, dw, db = backward(torch, seq, x, dy, G, f32(torch, w), f32(torch, b), act)
    want = so.group_norm_backward(dyv, xv, G, host(mean), host(rstd), w, b, activation=act, dtype=dtype)
    close(dx, want["dx"], want["dx_tol"], "dx")
    close(dw, want["dweight"], want["dweight_tol"], "dweight")
    close(db, want["dbias"], want["dbias_tol"], "dbias")


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("n,L,C,G", [(3, 6000, 99, 3), (2, 300, 4100, 2), (2, 5000, 33, 1), (50, 30, 99, 3)])
def test_channels_of_two_columns_have_one_value(env, n, L, C, G, act, dtype):  # noqa: F811
    """Channels that two threads compute, and either may write last: the same
    bits from both, over the input or beside it, call after call."""
    torch, seq = env
    torch.manual_seed(1)
    x, dy = (torch.randn(n, L, C, device="cuda").to(getattr(torch, dtype)) for _ in range(2))
    w, b = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-0.2, 0.2, C, device="cuda")
    y, mean, rstd = seq.group_norm(x, G, w, b, activation=act)
    dx = seq.group_norm_backward(dy, x, G, mean, rstd, w, b, activation=act)[0]
    for _ in range(5):
        assert torch.equal(seq.group_norm(x, G, w, b, activation=act)[0], y)
        assert torch.equal(seq.group_norm_backward(dy, x, G, mean, rstd, w, b, activation=act)[0], dx)
    t = x.clone()
    assert torch.equal(seq.group_norm(t, G, w, b, activation=act, out=t)[0], y)
    t = dy.clone()
    assert torch.equal(seq.group_norm_backward(t, x, G, mean, rstd, w, b, activation=act, out=t)[0], dx)
