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
