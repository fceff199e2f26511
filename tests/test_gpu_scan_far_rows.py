"""The selective scan with rows of its output so far apart that one chunk spans more than 4 GiB, and channels that fill no workgroup: the rows
hold what a packed output holds, and what lies between them is not touched."""
import pytest
import torch

from paper_2010_15884_amd import binding as B
from test_gpu_selective_scan import BF16, F32, _forward, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length,channels,states,dtype", [(32, 70, 16, F32), (75, 70, 5, BF16), (40, 3, 1, F32)])
def test_gaps_between_far_rows_of_the_output_stay(length, channels, states, dtype):
    c = _make(length, 1, length, channels, states, dtype)
    want = _forward(c)[0]
    apart = (1 << 26) - 5
    far = torch.full(((length - 1) * apart + channels,), 7.0, dtype=dtype, device="cuda")
    y = far.as_strided((1, length, channels), (far.numel(), apart, 1))
    _forward(c, d_y=y)
    assert torch.equal(y, want)
    for r in range(length - 1):
        assert (far[r * apart + channels:(r + 1) * apart] == 7.0).all(), r
