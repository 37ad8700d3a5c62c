"""Temperatures next to zero, refused on the host (no GPU needed)."""
import ctypes
import math

import numpy as np
import pytest

from tests.test_operators_host import ctx, distill, distill_grad, err, lib, logprobs, logprobs_grad  # noqa: F401


@pytest.mark.parametrize("call", [logprobs, logprobs_grad, distill, distill_grad])
def test_the_factor_of_the_exponent_is_finite(lib, ctx, call):  # noqa: F811
    """The kernels take log2(e) / T: where that is not a float32 any more, 0 times it is NaN and every sum with it."""
    most = float(np.finfo(np.float32).max)
    for T in (1.05 / most, 1.3 / most, 1.44 / most):                        # 1 / T is finite, log2(e) / T is not
        t = ctypes.c_float(T).value
        assert math.isfinite(float(np.float32(1.0) / np.float32(t)))
        assert call(lib, ctx, T=t) == -1 and "temperature" in err(lib, ctx), T
    assert call(lib, ctx, n=0, T=ctypes.c_float(1.5 / most).value) == 0
