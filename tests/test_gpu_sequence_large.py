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
