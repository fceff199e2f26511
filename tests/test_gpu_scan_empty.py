"""The selective scan of sequences without a position, whose inputs have rows that are used again: nothing is read through their pointers."""
import pytest
import torch

from paper_2010_15884_amd import binding as B
from test_gpu_selective_scan import BF16, F32, _inputs, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("channels,states,dtype,row", [(20, 16, BF16, 0), (70, 1, F32, 0), (33, 5, F32, 7)])
def test_no_length_and_rows_used_again(channels, states, dtype, row):
    c = _make(1, 2, 0, channels, states, dtype, state=True)
    for k in ("u", "delta", "z", "dy"):
        c[k] = torch.empty(0, dtype=dtype, device="cuda").as_strided((2, 0, channels), (0, row, 1))
    for k in ("B", "C"):
        c[k] = torch.empty(0, dtype=dtype, device="cuda").as_strided((2, 0, 1, states), (0, row, states, 1))
    out = torch.full_like(c["state"], float("nan"))
    assert B.sys_selective_scan(*_inputs(c), softplus=True, d_state=c["state"], d_state_out=out).shape == (2, 0, channels)
    assert torch.equal(out, c["state"])
    g = B.sys_selective_scan_backward(c["dy"], *_inputs(c), softplus=True, d_state=c["state"], d_dstate_out=c["dstate_out"])
    assert g.du.shape == (2, 0, channels) and torch.equal(g.dstate, c["dstate_out"]) and not g.dA.any() and not g.dD.any()
