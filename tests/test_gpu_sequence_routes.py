"""The kernels that large calls of the operators on sequences take: many rows a lane in the causal convolution, several spans a chunk in the
gradients of the scan (test_sequence_routes.py checks that these calls take them).

Tolerances as in sequence_reference.py; the references run on the GPU here, in 64 bits.  A sigmoid is off by (|pre| + 8) u of its value.
"""
import contextlib

import pytest
import torch

import sequence_reference as R
from paper_2010_15884_amd import binding as B
from test_gpu_selective_scan import _inputs, _make

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16

# batch, length, channels, type: every width below with lanes of 16 bytes and with lanes of one channel; the lengths of the sequences (or None)
WIDE = [(3, 8341, 1003, BF16, [8341, 0, 5003]), (2, 12511, 1005, F16, None), (2, 6301, 1003, F32, [17, 6301]), (3, 349603, 3, BF16, None), (2, 524309, 3, F16, [500000, 1]),
        (3, 349609, 3, F32, None)]
WIDTHS = [2, 3, 4, 5, 6, 7, 8]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("batch,length,channels,dtype,lengths", WIDE, ids=lambda v: str(v).replace("torch.", "") if not isinstance(v, list) else "lengths")
def test_convolution_of_many_rows(batch, length, channels, dtype, lengths, width):
    g = torch.Generator(device="cuda").manual_seed(length + width)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = rand(batch, length, channels + 2).to(dtype)[..., 1:-1]
    w, bias, state = (0.5 * rand(channels, width)).to(dtype), (0.3 * rand(channels)).to(dtype), rand(batch, width - 1, channels).to(dtype)
    silu = width % 2 == 0
    ends = [length] * batch if lengths is None else lengths
    for b, n in enumerate(ends):
        x[b, n:] = float("nan")
    after = torch.full_like(state, float("nan"))
    y = B.sys_causal_conv1d(x, w, bias, activation="SILU" if silu else "NONE", d_state=state, d_state_out=after,
                            d_lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    for b, n in enumerate(ends):
        rows = torch.cat([state[b], x[b, :n]]).double()
        pre, size = bias.double().expand(n, channels).clone(), bias.double().abs().expand(n, channels).clone()
        for j in range(width):
            pre += rows[j:j + n] * w[:, j].double()
            size += (rows[j:j + n] * w[:, j].double()).abs()
        want = pre * torch.sigmoid(pre) if silu else pre
        room = (1.1 * (width + 2) + pre.abs() + 8) * R.U * size if silu else (width + 2) * R.U * size
        relative, absolute = R.ROUNDING[dtype]
        off = (y[b, :n].double() - want).abs()
        assert (off <= room * (1 + relative) + relative * want.abs() + absolute).all(), (b, float((off - room).max()))
        assert not y[b, n:].any() and torch.isfinite(y[b, n:]).all()
        assert torch.equal(after[b].double(), rows[n:])


# spans a chunk; batch, length, channels, states, type, groups, gate, skip, bias, state, lengths
SPANS = [
    (8, (4, 300, 3441, 16, BF16, 1, True, True, True, False, None)),
    (2, (3, 75, 4422, 13, F32, 2, True, True, True, True, [75, 33, 0])),
    (3, (2, 130, 2931, 27, F16, 3, False, True, False, True, None)),
    (5, (2, 61, 5101, 64, BF16, 1, True, False, True, True, [61, 22])),
    (6, (5, 200, 3050, 3, F32, 1, True, True, True, True, [200, 129, 1, 97, 180])),
    (4, (2, 513, 2041, 7, BF16, 1, False, True, True, False, None)),
    (7, (7, 230, 2180, 16, F32, 4, True, True, True, True, None)),
    (8, (2, 1025, 2112, 30, BF16, 3, True, True, True, False, [1024, 700])),
]


@contextlib.contextmanager
def _references_on_the_gpu():
    was, R.wide = R.wide, lambda t: None if t is None else t.detach().double()
    try:
        with torch.device("cuda"):
            yield
    finally:
        R.wide = was


@pytest.mark.parametrize("spans,case", SPANS, ids=lambda v: str(v) if isinstance(v, int) else "-".join(str(k) for k in v[:6]).replace("torch.", ""))
def test_scan_gradients_in_chunks_of_several_spans(spans, case):
    batch, length, channels, states, dtype, groups = case[:6]
    lengths = case[10]
    c = _make(sum(case[:4]), *case[:10], lengths)
    g = B.sys_selective_scan_backward(c["dy"], *_inputs(c), softplus=True, d_state=c["state"], d_lengths=c["lengths"], d_dstate_out=c["dstate_out"])
    with _references_on_the_gpu():
        args = dict(state=c["state"], lengths=lengths, dy=c["dy"], dstate_out=c["dstate_out"])
        want, bound = R.scan(*_inputs(c), **args), R.scan(*_inputs(c), bound=True, **args)
        # as in test_gpu_selective_scan; sums over a group's channels are of 64 a workgroup, then of the workgroups, and those over
        # positions of a chunk's (at most 128), then of the chunks and sequences
        chain = (length + 2) * (12 * want["sA"] + 6) * R.U
        both = 2 * chain + (states + 4 + 20 + 20) * R.U
        over_channels = both + (64 + channels // groups // 64 + 1) * R.U
        over_positions = both + (128 + batch * (length // 4 + 1)) * R.U
        for name, allowed in (("du", both), ("ddelta", both), ("dz", both), ("dstate", both), ("dB", over_channels), ("dC", over_channels),
                              ("dA", over_positions), ("dD", over_positions), ("ddelta_bias", over_positions)):
            got = getattr(g, name)
            needs = {"dz": "z", "dD": "D", "ddelta_bias": "delta_bias", "dstate": "state"}.get(name)
            if needs and c[needs] is None:
                assert got is None
            else:
                R.check(got, want[name], allowed * bound[name], name)
