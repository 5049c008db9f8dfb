"""Operators around linear layers, without a GPU: limits of what their definitions
promise, and rules of the code that no run can show."""
import numpy as np
import pytest

from oracle import linear_oracle as lo


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_8_bit_values_of_16_bit_ones_are_nearest(dtype):
    """|127 v - q a| <= a / 2 in whole numbers: never the farther neighbour.  Of values that
    lie exactly halfway some go to the odd one, which is what the header says."""
    rng = np.random.default_rng(11)
    bits = 8 if dtype == "bfloat16" else 11
    # 254 v = a (2 k + 1) asks for 127 in a (halves are common then, but bfloat16 holds
    # no such a but 127 2^e, whose quotient is exact) or in 2 k + 1: v = a / 2, 63.5 steps
    top = np.concatenate([rng.integers(1, 2 ** bits // 127 + 1, size=2000) * 127, rng.integers(1, 2 ** bits, size=2000)])
    twice = rng.integers(-2 * top[:, None], 2 * top[:, None] + 1, size=(4000, 60))   # of v
    # v = twice / 2 as the type holds it
    v = lo.to_type(twice.astype(np.float32) / 2, dtype)
    v = np.concatenate([np.clip(v, -top[:, None], top[:, None])[:, :59], top[:, None] / 2, top[:, None]], 1)
    v = v.astype(np.float32)
    assert np.array_equal(lo.to_type(v, dtype), v)
    q, scale = lo.quantize_rows(v)
    q, v2 = q[:, :61].astype(np.int64), np.rint(2 * v).astype(np.int64)
    apart = np.abs(127 * v2 - 2 * q * top[:, None])   # twice the distance, in units of a
    assert (apart <= top[:, None]).all()
    halfway = apart == top[:, None]
    assert halfway.any() and (q[halfway] % 2 != 0).any() and (q[halfway] % 2 == 0).any()


# ---------------------------------------------------------------- the C ABI
@pytest.fixture(scope="module")
def lib():
    import os

    from paper_2601_17091_amd import rocket as rb
    if not os.path.exists(rb.LIB_PATH):
        from paper_2601_17091_amd import build_lib
        build_lib.build()
    return rb.library()


def gradient_workspace(lib, n, steps, m, c, dtype, lengths=None, data=0x10000, step=None):
    """Bytes that rocket_linear_weight_gradient asks for; rows at a distance of `step` values (m)."""
    import ctypes

    from paper_2601_17091_amd import rocket as rb
    shape = rb.CSequenceShape(n, steps, m, dtype, lengths)
    view = rb.CSequence(data, steps * (step or m), step or m)
    size = ctypes.c_int64(-1)
    assert lib.rocket_linear_weight_gradient_workspace(ctypes.byref(shape), c, ctypes.byref(view), ctypes.byref(size)) == 0
    return size.value


LARGE_LAYERS = [(1536, 20000), (2000, 6000), (1000, 12000), (600, 20000), (4096, 4096)]


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("m,c", LARGE_LAYERS)
def test_a_gradient_of_no_rows_stages_nothing(lib, m, c, dtype):
    """The staged kernel reads its first block's scales at once: without a block it must not
    be the one chosen, which its workspace (the biases' sums at least) tells."""
    assert gradient_workspace(lib, 8, 1000, m, c, dtype) > 0   # with rows it is
    for n, steps in ((0, 5), (5, 0), (0, 0)):
        for lengths in (None, 0x10000):
            assert gradient_workspace(lib, n, steps, m, c, dtype, lengths, data=None) == 0


def test_a_norm_and_its_sum_in_one_place_are_refused(lib):
    """Whichever were written last would be both."""
    import ctypes

    from paper_2601_17091_amd import rocket as rb
    byref = ctypes.byref
    shape, at = rb.CSequenceShape(2, 5, 8, 0, None), 0x10000
    x, r, y = rb.CSequence(at, 40, 8), rb.CSequence(2 * at, 40, 8), rb.CSequence(3 * at, 40, 8)
    for total in (rb.CSequence(3 * at, 40, 8), rb.CSequence(3 * at, 80, 16)):
        assert lib.rocket_rms_norm_forward(byref(shape), byref(x), byref(r), None, 1e-5, byref(y), byref(total), at,
                                           None) == rb.ROCKET_ERR_INVALID_ARG
    # no rows: nothing is written, and an empty tensor's address is no one's
    none, empty = rb.CSequence(None, 0, 0), rb.CSequenceShape(0, 5, 8, 0, None)
    assert lib.rocket_rms_norm_forward(byref(empty), byref(none), byref(none), None, 1e-5, byref(none), byref(none),
                                       None, None) == 0
