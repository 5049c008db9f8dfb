"""The activations of the group norm and their slopes, value by value: with a
weight of 0 and the values as biases the output is act(z), and the gradient of
the bias of one row is act'(z)."""
import numpy as np
import pytest

from oracle import sequence_oracle as so
from test_gpu_sequence import close, env, f32, typed  # noqa: F401

pytestmark = pytest.mark.gpu
C = 4096


def values(low, high):
    """fp32 numbers over the range, dense around 0 and at its ends."""
    z = np.concatenate([np.linspace(low, high, C // 2), -np.geomspace(1e-6, -low, C // 4),
                        np.geomspace(1e-6, high, C // 4)])
    return z.astype(np.float32)


def normal_tail(z):
    """The normal distribution function, to the last digits of its lower tail."""
    import math
    return np.array([0.5 * math.erfc(-t / math.sqrt(2.0)) for t in z])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("act,low,high", [("gelu", -12.5, 12.5), ("gelu", -4.0, 1.0), ("silu", -80.0, 80.0),
                                          ("silu", -5.0, 5.0)])
def test_activations_and_slopes(env, act, low, high, dtype):  # noqa: F811
    """Relative errors: fp32 32 units of 2^-24 (the exponential, the reciprocal
    and a polynomial's last operations, each a few); 16 bits 1.2e-4 before the
    type's own rounding, and never more than 16 units of 2^-24 of 1 + |z|."""
    torch, seq = env
    z = values(low, high)
    x, _ = typed(torch, np.random.default_rng(1).standard_normal((1, 1, C)), dtype)
    zero, bias = torch.zeros(C, device="cuda"), f32(torch, z)
    y, mean, rstd = seq.group_norm(x, 1, zero, bias, activation=act)
    ones = torch.ones_like(x)
    _, _, slope = seq.group_norm_backward(ones, x, 1, mean, rstd, zero, bias, activation=act)
    z = z.astype(np.float64)
    if act == "gelu":
        cdf, density = normal_tail(z), np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
        want, want_slope, size = z * cdf, cdf + z * density, cdf + np.abs(z) * density
    else:
        s, rest = so.logistic(z), so.logistic(-z)
        want, want_slope, size = z * s, s + z * s * rest, s + np.abs(z) * s * rest
    part = 32 * so.U if dtype == "float32" else 1.2e-4
    most = 16 * so.U * (1 + np.abs(z))
    tol = np.minimum(part * np.abs(want), most * np.abs(z))
    close(y[0, 0], want, so.rounded(tol, want, dtype), "activation")
    close(slope, want_slope, np.minimum(part * size, most) + 2.0 ** -126, "slope")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_activations_of_infinities_and_nan(env, act, dtype):  # noqa: F811
    torch, seq = env
    x = torch.randn(1, 1, 16, device="cuda").to(getattr(torch, dtype))
    bias = torch.zeros(16, device="cuda")
    bias[0], bias[1], bias[2], bias[3] = float("inf"), float("nan"), 1e30, -1e30
    y, mean, rstd = seq.group_norm(x, 1, torch.zeros(16, device="cuda"), bias, activation=act)
    y = y[0, 0].float()
    assert y[0] == float("inf") and y[1].isnan() and bool((y[4:] == 0).all())
    assert y[2] > 6e4 and (act == "none" or y[3] == 0)
    slope = seq.group_norm_backward(torch.ones_like(x), x, 1, mean, rstd, torch.zeros(16, device="cuda"), bias,
                                    activation=act)[2]
    assert slope[2] == 1 and (act == "none" or slope[3] == 0)
