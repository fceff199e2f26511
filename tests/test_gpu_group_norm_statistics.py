"""Statistics of the group norm where they are hardest to keep: a first value that is an outlier, and groups of many rows and channels.

Tolerances (u = 2^-24).  The mean: 100 u (|mean| + spread), spread = sqrt(var + eps), as in test_gpu_group_norm.  rstd of groups that are
summed up in chunks: what a chunk leaves of a channel (a sum of squared distances of some tens of values) is off by at most some 40 u of itself,
either way; these are at least 2^14 here, so their sum is off by less than u, and everything from there on is worked out in 64 bits.  The
variance is rounded to 32 bits, eps is added, and the instruction is off by 2 u: 4 u in all; 8 u are allowed.
"""
import pytest
import torch

import sequence_reference as R
from paper_2010_15884_amd import binding as B
from paper_2010_15884_amd import sequence as S

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
EPS = 1e-5


def _call(x, groups):
    batch, rows, channels = x.shape
    mean, rstd = (torch.full((batch, groups), float("nan"), device="cuda") for _ in range(2))
    y = B.sys_group_norm(x, groups, eps=EPS, d_mean=mean, d_rstd=rstd)
    xg = x.double().view(batch, rows, groups, channels // groups)
    want = xg.mean(dim=(1, 3))
    away = xg - want[:, None, :, None]
    return y, mean.double(), rstd.double(), want, 1.0 / torch.sqrt(away.square().mean(dim=(1, 3)) + EPS), away.reshape(x.shape)


def _x(seed, batch, rows, channels, dtype):
    return torch.randn((batch, rows, channels), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("outlier", [1000.0, -3e4])
@pytest.mark.parametrize("batch,rows,channels,groups", [(1, 16384, 64, 1), (2, 2048, 64, 1), (3, 8192, 96, 3), (1, 32768, 8, 1), (2, 65536, 3, 1), (3, 1, 16384, 1),
                                                        (2, 1, 8192, 2), (1, 1 << 20, 1, 1), (16, 4096, 512, 32), (4, 1024, 256, 4), (2, 500, 40, 1), (70, 255, 128, 4),
                                                        (2048, 65536, 1, 1), (300, 100000, 3, 1)])
def test_the_first_value_is_an_outlier(batch, rows, channels, groups, outlier):
    x = _x(rows, batch, rows, channels, F32)
    x[:, 0, ::channels // groups] = outlier
    _, mean, rstd, want, want_rstd, _ = _call(x, groups)
    assert ((mean - want).abs() <= 100 * R.U * (want.abs() + 1.0 / want_rstd)).all(), float(((mean - want).abs() * want_rstd).max() / R.U)
    assert ((rstd - want_rstd).abs() <= 150 * R.U * want_rstd).all()


@pytest.mark.parametrize("value", [0.1, -3.7e5])
@pytest.mark.parametrize("batch,rows,channels,groups", [(2, 50, 33, 3), (5, 1, 512, 4), (3, 4096, 512, 32), (1, 1023, 70, 10), (2, 16384, 24, 2), (3, 1, 16384, 1)])
def test_equal_values_leave_nothing(batch, rows, channels, groups, value):
    """Every mean is the value itself and every distance 0, so y is 0 and rstd that of eps alone."""
    x = torch.full((batch, rows, channels), value, device="cuda")
    y, mean, rstd, *_ = _call(x, groups)
    assert not y.any() and (mean == x[0, 0, 0].double()).all()
    assert ((rstd * EPS ** 0.5 - 1.0).abs() <= 4 * R.U).all()


CHUNKED = [(1, 16384, 2048, 1), (4, 4096, 2048, 1), (4, 4096, 2048, 4), (2, 8192, 1024, 32), (1, 65536, 64, 2), (1, 131072, 24, 1), (3, 1, 1 << 20, 2)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("batch,rows,channels,groups", CHUNKED)
def test_variances_of_groups_in_chunks(batch, rows, channels, groups, dtype):
    code = {F32: B.SYS_F32, F16: B.SYS_F16, BF16: B.SYS_BF16}[dtype]
    packed = S._NORM.pack(code, code, 0, groups, batch, channels, EPS, 0, rows, rows * channels, channels, rows * channels, channels)
    assert S._entry_points().sys_group_norm_workspace(packed) > 0          # in chunks
    x = _x(batch + rows, batch, rows, channels, dtype) + 0.25
    _, mean, rstd, want, want_rstd, _ = _call(x, groups)
    assert ((mean - want).abs() <= 8 * R.U * (want.abs() + 1.0 / want_rstd)).all()
    assert ((rstd - want_rstd).abs() <= 8 * R.U * want_rstd).all(), float(((rstd - want_rstd) / want_rstd).abs().max() / R.U)
