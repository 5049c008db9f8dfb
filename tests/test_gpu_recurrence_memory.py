"""The recurrence over thousands of steps that keep: the gates' roundings must
not lean to one side, since their product carries them all."""
import numpy as np
import pytest

from test_gpu_sequence import env  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("low,high", [(3.0, 6.0), (4.0, 8.0)])
@pytest.mark.parametrize("L", [2000, 400])
def test_product_of_many_gates_does_not_drift(env, L, low, high):  # noqa: F811
    """4,096 products of L gates, forward and as the gradient of the first state.
    A gate's rounding is a unit of 2^-24 or less either way, so that the mean of
    the products' errors has a deviation of sqrt(L / 4096) units or less: 6 of
    them, and 0.005 units a gate for what leans."""
    torch, seq = env
    rng = np.random.default_rng(L)
    f = rng.uniform(low, high, (1, L, 4096)).astype(np.float32)
    want = np.exp(-np.log1p(np.exp(-f.astype(np.float64))).sum(1))
    t = torch.from_numpy(f).cuda()
    zero, one = torch.zeros_like(t), torch.ones(1, 4096, device="cuda")
    _, h, states = seq.recurrence(zero, t, h0=one, keep_states=True)
    dh0 = seq.recurrence_backward(zero, zero, t, states, dh_last=one)[3]
    for got in (h, dh0):
        error = (got.double().cpu().numpy() / want - 1) / U
        assert abs(error.mean()) < 6 * np.sqrt(L / 4096) + 0.005 * L
