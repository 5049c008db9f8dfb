"""Calls that one launch cannot hold (2^32 threads or more): several launches,
the same results."""
import numpy as np
import pytest

from test_gpu_sequence import env, expected_dropout  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back(env):  # noqa: F811
    """The memory of these tests is not kept for the others."""
    yield
    env[0].cuda.empty_cache()


def test_dropout_of_more_elements_than_a_launch(env):  # noqa: F811
    torch, seq = env
    n = (1 << 35) + 1003
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = seq.dropout(x, 0.25, 11, 3, out=x)
    ix = np.concatenate([np.arange(40), np.arange((1 << 35) - 2100, (1 << 35) - 2000),
                         np.arange((1 << 35) - 20, (1 << 35) + 20), np.arange(n - 30, n)])
    want = expected_dropout(torch, torch.ones(1, dtype=torch.bfloat16).expand(n), None, 0.25, 11, 3, ix)
    assert torch.equal(y[torch.from_numpy(ix).cuda()].cpu(), want)


def test_recurrence_of_more_series_than_a_launch(env):  # noqa: F811
    """2^26 series of one step and channel and a few more, a wavefront each: all
    of them against the formula, in fp32 on the way."""
    torch, seq = env
    n = (1 << 26) + 5
    v, f, dy = (torch.randn(n, 1, 1, device="cuda").to(torch.bfloat16) for _ in range(3))
    h0 = torch.randn(n, 1, device="cuda")
    y, h, states = seq.recurrence(v, f, h0=h0, keep_states=True)
    assert torch.equal(states[:, 0], h0)
    a, keep = torch.sigmoid(f.float())[:, 0], torch.sigmoid(-f.float())[:, 0]
    want = a * h0 + keep * v.float()[:, 0]
    # a few roundings of fp32 operands of up to 6
    assert float((h - want).abs().max()) < 1e-5
    assert float((y[:, 0].float() - want).abs().sub_(want.abs() * 2.0 ** -8).max()) < 2e-5
    dv, df, _, dh0 = seq.recurrence_backward(dy, v, f, states, dh_last=h0)
    dh = dy.float()[:, 0] + h0
    assert float((dh0 - a * dh).abs().max()) < 1e-5
    for got, want in ((dv, dh * keep), (df, dh * (h0 - v.float()[:, 0]) * a * keep)):
        assert float((got[:, 0].float() - want).abs().sub_(want.abs() * 2.0 ** -8).max()) < 5e-5


def test_recurrence_step_of_more_words_than_a_launch(env):  # noqa: F811
    """2^32 words of channels and more: 1,025 channels of 2^23 series, the inputs
    a few rows repeated."""
    torch, seq = env
    n, C = (1 << 23) + 7, 1025
    v, f = (torch.randn(1, C, device="cuda").to(torch.bfloat16) for _ in range(2))
    h = torch.ones(n, C, device="cuda")
    y, h = seq.recurrence_step(v.expand(n, C), f.expand(n, C), h, h_out=h)
    small_y, small_h = seq.recurrence_step(v, f, torch.ones(1, C, device="cuda"))
    per = ((1 << 32) - 256) // 513   # series of a launch
    for at in (0, per - 3, n - 1000):
        assert torch.equal(h[at:at + 1000], small_h.expand(len(h[at:at + 1000]), C))
        assert torch.equal(y[at:at + 1000], small_y.expand(len(y[at:at + 1000]), C))
    assert float(h.sum(0, dtype=torch.float64).sub_(small_h[0].double() * n).abs().max()) < 1e-6 * n


@pytest.mark.parametrize("n,C,G,dtype", [((1 << 24) + 3, 4, 2, "float16"), ((1 << 26) + 3, 9, 3, "bfloat16")])
def test_group_norm_of_more_series_than_a_launch(env, n, C, G, dtype):  # noqa: F811
    """A workgroup a series, some of no steps: all against the formula in fp32."""
    torch, seq = env
    x = torch.randn(n, 1, C, device="cuda").to(getattr(torch, dtype))
    lengths = (torch.rand(n, device="cuda") < 0.9).int()
    w, b = torch.linspace(0.5, 1.5, C, device="cuda"), torch.linspace(-1.0, 1.0, C, device="cuda")
    y, mean, rstd = seq.group_norm(x, G, w, b, activation="relu", lengths=lengths)
    live = lengths.bool()[:, None]
    v = x.float().view(n, G, C // G)
    m = v.mean(2)
    r = 1 / torch.sqrt(((v - m[:, :, None]) ** 2).mean(2) + 1e-5)
    # a few roundings of sums of two or three values of up to 6, and of a rstd of up to 316
    assert float((mean - m * live).abs().max()) < 5e-6
    assert float((rstd - r * live).abs().div_(r).max()) < 1e-3
    z = ((v - m[:, :, None]) * r[:, :, None]).view(n, C) * w + b
    want = z.clamp_(min=0.0).mul_(live)
    unit = 2.0 ** -11 if dtype == "float16" else 2.0 ** -8
    assert float((y[:, 0].float() - want).abs().sub_(want * unit).max()) < 3e-3


def test_group_norm_chunks_of_more_series_than_a_launch(env):  # noqa: F811
    """Two chunks a series, 2^24 chunks and more, in place: forward and backward
    against calls of some of the series, the bias's gradient against the sum."""
    torch, seq = env

    def some(n):
        per = (((1 << 32) - 1) // 256) // 2   # series of a launch
        return [slice(0, 50), slice(per - 25, per + 25), slice(n - 50, n)]

    n, L = (1 << 23) + 3, 4097
    x = torch.empty(n, L, 1, dtype=torch.bfloat16, device="cuda").normal_()
    before = [x[at].clone() for at in some(n)]
    y, mean, rstd = seq.group_norm(x, 1, activation="silu", out=x)
    for at, t in zip(some(n), before):
        want = seq.group_norm(t, 1, activation="silu")
        assert torch.equal(y[at], want[0]) and torch.equal(mean[at], want[1]) and torch.equal(rstd[at], want[2])
    del x, y, before
    torch.cuda.empty_cache()

    n, L = (1 << 23) + 5, 2049
    x = torch.empty(n, L, 1, dtype=torch.bfloat16, device="cuda").normal_()
    dy = torch.empty_like(x).uniform_()
    mean, rstd = torch.zeros(n, 1, device="cuda"), torch.ones(n, 1, device="cuda")
    before = [dy[at].clone() for at in some(n)]
    total = sum(float(dy[i:i + (1 << 20)].sum(dtype=torch.float64)) for i in range(0, n, 1 << 20))
    dx, dw, db = seq.group_norm_backward(dy, x, 1, mean, rstd, out=dy)
    for at, t in zip(some(n), before):
        assert torch.equal(dx[at], seq.group_norm_backward(t, x[at], 1, mean[at], rstd[at])[0])
    # chains of up to 8,192 additions of positive numbers
    assert abs(float(db[0]) - total) < 8192 * 2.0 ** -24 * total
