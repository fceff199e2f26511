"""The gated delta rule on both sides of where short sequences go a position at a time: up to 10 positions in bf16, 12 in wider types, 20 where there are more heads than CUs."""
import ctypes

import pytest

from paper_2010_15884_amd import binding as B
from paper_2010_15884_amd import sequence as S
from test_gpu_gated_delta import BF16, F16, F32, _check_forward, _make

BORDERS = [(BF16, 1, 10), (F16, 1, 12), (F32, 1, 12), (BF16, 64, 20), (F16, 64, 20), (F32, 64, 20)]
name = lambda v: str(v).replace("torch.", "")  # noqa: E731


@pytest.mark.parametrize("dtype,batch,most", BORDERS, ids=name)
def test_a_position_at_a_time_needs_no_workspace(dtype, batch, most):
    code = {F32: B.SYS_F32, F16: B.SYS_F16, BF16: B.SYS_BF16}[dtype]

    def size(length):
        packed = S._DELTA.pack(code, 1, 1, batch, length, 2, 4, 40, 24, 0, 1.0, 0, *[length * 96, 96] * 3, *[length * 4, 4] * 2, length * 96, 96)
        return S._entry_points().sys_gated_delta_rule_workspace(ctypes.c_char_p(packed))
    assert size(most) == 0 < size(most + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("more", [0, 1])
@pytest.mark.parametrize("dtype,batch,most", BORDERS, ids=name)
def test_both_sides(dtype, batch, most, more):
    _check_forward(_make(84 + most, batch, most + more, 2, 4, 40, 24, dtype, state=True))
