"""The gated delta rule where 32 columns go to a workgroup, close in norm: sums over many terms are nearer than their worst case.

The bounds are those of 16 columns a workgroup (test_gradients_are_close_in_norm), whose products are the same: numbers of 24 bits (2^-24 of a term) and sums of up to 128 of them, as often
rounded up as down, twice there and twice back: 4 sqrt(2 * 128) 2^-24 = 4e-6, half of it on one way; 2^-14 where the squares of a chunk have 16 bits; decays' gradients are sums over
all positions of differences of such sums."""
import pytest
import torch

import sequence_reference as R
from test_gpu_gated_delta import BF16, F16, F32, _backward, _forward, _make, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,key_dim", [(F32, 64), (F16, 128), (F16, 64), (BF16, 128), (BF16, 48)])
def test_close_in_norm(dtype, key_dim):
    c = _make(95, 2, 200, 3, 9, key_dim, 240, dtype, state=True)
    assert 15 * 9 * 2 > 256                        # tiles of 16 columns, and CUs
    want, got = _reference(c, grad=True), _backward(c)
    y, state = _forward(c)
    far = lambda a, b: float((R.wide(a) - b).norm() / b.norm())  # noqa: E731
    rounding = {F32: 0.0, F16: 2.0 ** -11, BF16: 2.0 ** -8}[dtype]
    assert far(y, want["y"]) < 2e-6 + rounding and far(state, want["state"]) < 2e-6
    assert far(got.dstate, want["dstate"]) < 2e-6
    for name in ("dq", "dk", "dv", "dbeta", "ddelta"):
        assert far(getattr(got, name), want[name]) < (4e-6 if dtype == F32 else 2.0 ** -14) + rounding, name
    for name in ("dA", "ddelta_bias"):
        assert far(getattr(got, name), want[name]) < 1e-5, name
