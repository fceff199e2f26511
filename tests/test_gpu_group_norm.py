"""Group norm with an activation against its definition in 64 bits.

Tolerances (u = 2^-24).  mean: of values that are off by nothing, summed eight at a time and merged in at most 40 steps that each round
by 2u of the values' spread and of the mean: 100 u (|mean| + spread), spread = sqrt(var + eps).  rstd: the sum of squared distances is off by as much
relative to itself, plus what the means' errors add (their square): 150 u.  hat = (x - mean) rstd: the difference is off by 100 u (|mean| + spread) + u |x - mean|, so
hat by (102 |mean| / spread + 102 + 152 |hat|) u.  y follows with w, and SiLU multiplies by at most 1.1 and adds (|pre| + 8) u |pre|.
The gradients are computed from statistics that are given, so hat is off by (|x| + |mean|) rstd u + 3 u |hat| only; dx and the sums over at most 16
levels of 64 values follow from it (below).
"""
import pytest
import torch

import sequence_reference as R
from paper_2010_15884_amd import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _make(seed, batch, rows, channels, dtype, affine=True, params=None, shift=0.5, offset=0):
    g = _gen(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = (rand(batch, rows, channels + offset + 2) + shift).to(dtype)[..., offset:offset + channels]
    return {"x": x, "w": (1 + 0.3 * rand(channels)).to(params or dtype) if affine else None, "b": (0.3 * rand(channels)).to(params or dtype) if affine else None,
            "dy": rand(batch, rows, channels + 1).to(dtype)[..., 1:]}


def _check_all(c, groups, activation, eps=1e-5):
    x = c["x"]
    batch, rows, channels = x.shape
    want = R.group_norm(x, groups, c["w"], c["b"], eps, activation)
    mean, rstd = (torch.full((batch, groups), float("nan"), device="cuda") for _ in range(2))
    y = B.sys_group_norm(x, groups, c["w"], c["b"], eps=eps, activation=activation, d_mean=mean, d_rstd=rstd)
    wide = lambda s: s[:, None, :, None].expand(batch, rows, groups, channels // groups).reshape(batch, rows, channels)  # noqa: E731
    spread = 1.0 / want["rstd"]
    R.check(mean, want["mean"], 100 * R.U * (want["mean"].abs() + spread), "mean")
    R.check(rstd, want["rstd"], 150 * R.U * want["rstd"], "rstd")
    w = torch.ones(channels, dtype=torch.float64) if c["w"] is None else R.wide(c["w"]).abs()
    hat = R.U * (102 * wide(want["mean"].abs() * want["rstd"]) + 102 + 152 * want["hat"].abs())
    pre = hat * w + 2 * R.U * (want["pre"].abs() + want["hat"].abs() * w)
    room = 1.1 * pre + (want["pre"].abs() + 8) * R.U * want["pre"].abs() if activation == "SILU" else pre
    R.check(y, want["y"], room, "y")

    # gradients from the statistics that the call left
    want = R.group_norm(x, groups, c["w"], c["b"], eps, activation, dy=c["dy"], mean=mean, rstd=rstd)
    dx, dw, db = B.sys_group_norm_backward(c["dy"], x, groups, mean, rstd, c["w"], c["b"], activation=activation)
    dy, xw = R.wide(c["dy"]).abs(), R.wide(x).abs()
    hat = R.U * ((xw + wide(R.wide(mean).abs())) * wide(R.wide(rstd)) + 3 * want["hat"].abs())
    pre = hat * w + 2 * R.U * (want["pre"].abs() + want["hat"].abs() * w)
    f_size = dy * (1.1 if activation == "SILU" else 1.0)
    # the derivative of SiLU: its own is at most 0.5, its evaluation is off by (2 |pre| + 20) u of s (1 + |pre|)
    f = dy * (0.5 * pre + (2 * want["pre"].abs() + 20) * R.U * R.act_grad(want["pre"], "SILU", True)) + R.U * f_size if activation == "SILU" else R.U * f_size
    if activation == "RELU":
        # a value that close to zero may fall on either side
        f = f + torch.where(want["pre"].abs() <= pre, dy, torch.zeros_like(dy))
    sums = 100 * R.U
    grouped = lambda t: t.view(batch, rows, groups, channels // groups)  # noqa: E731
    over = lambda t: grouped(t).mean(dim=(1, 3), keepdim=True).expand(batch, rows, groups, channels // groups).reshape(x.shape)  # noqa: E731
    size_hat = want["hat"].abs()
    f_hat = f * size_hat + f_size * hat
    if c["w"] is not None:
        R.check(dw, want["dw"], (f_hat + sums * f_size * size_hat).sum(dim=(0, 1)), "dw")
        R.check(db, want["db"], (f + sums * f_size).sum(dim=(0, 1)), "db")
    else:
        assert dw is None and db is None
    m1, m2 = over((f + sums * f_size) * w), over((f_hat + sums * f_size * size_hat) * w)
    size = f_size * w + over(f_size * w) + size_hat * over(f_size * size_hat * w)
    allowed = wide(R.wide(rstd)) * (f * w + m1 + hat * over(f_size * size_hat * w) + size_hat * m2 + 6 * R.U * size)
    R.check(dx, want["dx"], allowed, "dx")


CASES = [
    # batch, rows, channels, groups, dtype, activation, affine, parameters' type, column offset
    (2, 64, 64, 8, BF16, "SILU", True, None, 0),
    (5, 1, 128, 4, BF16, "NONE", True, None, 0),
    (3, 1, 4096, 64, F16, "SILU", True, F32, 0),
    (1, 300, 30, 3, F32, "SILU", True, None, 1),
    (2, 77, 320, 32, F16, "SILU", True, None, 0),
    (2, 9, 7, 7, F32, "RELU", True, None, 1),
    (3, 33, 63, 1, BF16, "NONE", False, None, 1),
    (1, 1, 24, 2, F32, "RELU", True, None, 0),
    (2, 1025, 12, 2, F32, "SILU", False, None, 0),
    (1, 5000, 16, 4, BF16, "SILU", True, None, 0),
    (2, 20, 2600, 26, BF16, "SILU", True, F32, 0),
    (1, 3, 2050, 2, F32, "NONE", True, None, 0),
    (300, 1, 96, 1, F16, "RELU", True, None, 2),
    (3, 2, 1, 1, F32, "NONE", True, None, 0),
    (1, 4099, 40, 4, F16, "NONE", True, None, 3),
    (2, 256, 512, 32, BF16, "SILU", True, None, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c[:6]).replace("torch.", ""))
def test_forward_and_gradients(case):
    batch, rows, channels, groups, dtype, activation, affine, params, offset = case
    _check_all(_make(sum(case[:4]), batch, rows, channels, dtype, affine, params, offset=offset), groups, activation)


LAYOUTS = [
    # groups of every width a lane may hold (1, 2, 4, 8 channels), few and many units, whole and ragged last rows, from 1 to 32 rows a lane
    (2, 1024, 70, 10, F16, "SILU"), (1, 1023, 70, 10, BF16, "NONE"), (3, 31, 70, 10, F32, "RELU"),
    (4, 1024, 320, 32, F16, "SILU"), (1, 700, 320, 32, BF16, "RELU"), (9, 1023, 160, 16, F16, "NONE"), (2, 4096, 60, 6, F32, "SILU"),
    (3, 2047, 24, 2, BF16, "SILU"), (40, 130, 60, 5, F16, "NONE"), (130, 97, 20, 5, F32, "SILU"), (64, 513, 12, 1, F16, "SILU"),
    (2, 4096, 64, 2, BF16, "SILU"), (1, 4097, 64, 2, BF16, "NONE"), (70, 255, 128, 4, F16, "RELU"), (5, 1000, 40, 5, BF16, "SILU"),
    # rows of many lanes
    (3, 1, 8192, 1, BF16, "SILU"), (2, 5, 4096, 1, F16, "NONE"), (1, 3, 6000, 2, F32, "SILU"), (1, 4, 8000, 1, F32, "NONE"),
    # tokens, several entries a unit: units in a wavefront, of one, of several
    (20000, 1, 256, 64, BF16, "SILU"), (2101, 1, 4096, 1, F16, "NONE"), (16387, 1, 500, 1, BF16, "RELU"),
]


@pytest.mark.parametrize("case", LAYOUTS, ids=lambda c: "-".join(str(v) for v in c).replace("torch.", ""))
def test_layouts(case):
    batch, rows, channels, groups, dtype, activation = case
    _check_all(_make(sum(case[:4]), batch, rows, channels, dtype), groups, activation)


def test_variances_of_every_size():
    """Without eps the results are the same at every power of two; the square of the smallest is 2^-120."""
    for rows, channels, groups in ((50, 24, 3), (1, 256, 4), (6000, 40, 4)):
        c = _make(rows, 2, rows, channels, F32)
        for exponent in (-60, -30, 40):
            _check_all(dict(c, x=c["x"] * 2.0 ** exponent), groups, "SILU", eps=0.0)


def test_means_far_from_zero():
    """Squares summed as they come would lose the variance: 4096^2 2^-24 = 1."""
    for rows, channels, groups in ((500, 24, 3), (1, 256, 4), (64, 16, 2)):
        _check_all(_make(rows, 2, rows, channels, F32, shift=4096.0), groups, "NONE")
    x = _make(3, 2, 200, 16, F32)["x"].contiguous()
    x[0, 0] = 1e6                                           # the first row is an outlier
    _check_all({"x": x, "w": None, "b": None, "dy": torch.randn_like(x)}, 2, "NONE")


def test_constant_groups():
    x = torch.full((2, 50, 32), 3.0, device="cuda")
    mean, rstd = (torch.empty((2, 4), device="cuda") for _ in range(2))
    assert not B.sys_group_norm(x, 4, eps=1e-6, d_mean=mean, d_rstd=rstd).any()
    assert (mean == 3).all() and ((rstd - 1000).abs() < 1e-2).all()


def test_empty_batch():
    x = torch.empty((0, 5, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    assert B.sys_group_norm(x, 4, w, w).shape == (0, 5, 16)
    stats = torch.empty((0, 4), device="cuda")
    dx, dw, db = B.sys_group_norm_backward(x, x, 4, stats, stats, w, w)
    assert dx.shape == (0, 5, 16) and not dw.any() and not db.any()


def test_what_is_not_finite_stays_in_its_group():
    for rows, channels in ((40, 64), (1, 512), (3000, 64)):
        c = _make(rows, 3, rows, channels, F32)
        clean = B.sys_group_norm(c["x"], 8, c["w"], c["b"], activation="SILU")
        c["x"][1, rows // 2, 3] = float("nan")
        y = B.sys_group_norm(c["x"], 8, c["w"], c["b"], activation="SILU")
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[1, :, :channels // 8] = True
        assert not torch.isfinite(y[bad]).any() and torch.equal(y[~bad], clean[~bad])


def test_strides():
    c = _make(7, 1, 60, 48, F32)
    y = B.sys_group_norm(c["x"], 6, c["w"], c["b"])
    x = c["x"].contiguous()
    assert torch.equal(B.sys_group_norm(x, 6, c["w"], c["b"]), y)
    assert torch.equal(B.sys_group_norm(x.expand(4, 60, 48), 6, c["w"], c["b"]), y.expand(4, 60, 48))
    out = torch.full((2, 60, 50), 5.0, device="cuda")
    B.sys_group_norm(x.expand(2, 60, 48), 6, c["w"], c["b"], d_y=out[..., 1:49])
    assert torch.equal(out[..., 1:49], y.expand(2, 60, 48)) and (out[..., 0] == 5).all() and (out[..., 49] == 5).all()
    far = torch.empty(1 << 32, dtype=BF16, device="cuda")
    rows = far.as_strided((2, 9, 48), ((1 << 31) - 100, (1 << 27) + 1, 1))
    rows.copy_(torch.randn((2, 9, 48), generator=_gen(1), device="cuda"))
    w = c["w"].to(BF16)
    assert torch.equal(B.sys_group_norm(rows, 6, w), B.sys_group_norm(rows.contiguous(), 6, w))


def test_gradients_against_differences():
    """Central differences of L = <y, r>, e = 2^-6: cut off at e^2/6 times a third derivative, rounded by 2^-24 / e."""
    for rows, channels, groups in ((30, 24, 3), (1, 64, 4)):
        c = _make(rows, 2, rows, channels, F32)
        point = [c["x"].contiguous(), c["w"], c["b"]]
        mean, rstd = (torch.empty((2, groups), device="cuda") for _ in range(2))

        def loss(x, w, b):
            return float((B.sys_group_norm(x, groups, w, b, activation="SILU", d_mean=mean, d_rstd=rstd).double() * c["dy"].double()).sum())

        loss(*point)
        grads = B.sys_group_norm_backward(c["dy"], point[0], groups, mean.clone(), rstd.clone(), c["w"], c["b"], activation="SILU")
        g = _gen(3)
        for i, grad in enumerate(grads):
            v, e = torch.randn(point[i].shape, generator=g, device="cuda"), 2.0 ** -6
            up, down = ([p + s * e * v if k == i else p for k, p in enumerate(point)] for s in (1, -1))
            slope = (loss(*up) - loss(*down)) / (2 * e)
            assert abs(slope - float((grad.double() * v.double()).sum())) <= 2e-3 * float((grad.double() * v.double()).abs().sum()), i


def test_same_bits_every_time_on_any_stream_and_from_a_graph():
    for rows, channels, groups in ((700, 320, 32), (1, 1024, 16)):
        c = _make(rows, 3, rows, channels, BF16)
        mean, rstd = (torch.empty((3, groups), device="cuda") for _ in range(2))

        def calls():
            y = B.sys_group_norm(c["x"], groups, c["w"], c["b"], activation="SILU", d_mean=mean, d_rstd=rstd)
            return [y, mean, rstd, *B.sys_group_norm_backward(c["dy"], c["x"], groups, mean, rstd, c["w"], c["b"], activation="SILU")]

        want = [t.clone() for t in calls()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        y = B.sys_group_norm(c["x"], groups, c["w"], c["b"], activation="SILU", stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(y, want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = calls()
        for _ in range(3):
            for t in got:
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, want))
            assert all(torch.equal(p, q) for p, q in zip(calls(), want))
