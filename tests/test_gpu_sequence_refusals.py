"""Refusals of the sequence binding that its C types do not make by themselves."""
import pytest

from test_gpu_sequence import env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups", [2 ** 32 + 2, -2 ** 32 + 2, 2 ** 64 + 4])
def test_groups_past_32_bits(env, groups):  # noqa: F811
    torch, seq = env
    x = torch.zeros(2, 6, 8, device="cuda")
    _, mean, rstd = seq.group_norm(x, groups % 2 ** 32)
    with pytest.raises(ValueError):
        seq.group_norm(x, groups)
    with pytest.raises(ValueError):
        seq.group_norm_backward(x, x, groups, mean, rstd)
