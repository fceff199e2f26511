"""The gated delta rule on rows that are used again, that lie in one another, or whose distance means nothing: the same as on copies of them, bit for bit."""
import pytest
import torch

from test_gpu_gated_delta import BF16, F16, F32, INPUTS, _backward, _forward, _make

pytestmark = pytest.mark.gpu

STRIDED = ("q", "k", "v", "delta", "beta", "dy")


def _same(c):
    """The calls on c are those on contiguous copies of what it has."""
    plain = {n: t.contiguous() if n in STRIDED else t for n, t in c.items()}
    for n, (a, b) in zip(("y", "state"), zip(_forward(c), _forward(plain))):
        assert torch.equal(a, b), n
    got, want = _backward(c), _backward(plain)
    for n in got._fields:
        a, b = getattr(got, n), getattr(want, n)
        assert (a is None and b is None) or torch.equal(a, b), n
    assert all(torch.isfinite(t).all() for t in got if t is not None)


def _repeated(t):
    """The first position's row for all of them, without a copy."""
    return t[:, :1].expand(t.shape)


def _within(t, apart):
    """Rows of [batch, length, heads, dim] (or [batch, length, heads]) that begin `apart` elements after one another, less than they are long."""
    batch, length = t.shape[:2]
    heads = t.shape[2:]
    room = torch.randn((batch, (length - 1) * apart + heads.numel()), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")
    inner = (heads[1], 1) if len(heads) == 2 else (1,)
    return (0.05 * room).to(t.dtype).as_strided(t.shape, (room.shape[1], apart, *inner))


# the last chunk is whole, or has one position, or some; value heads apart and together
CASES = [
    # batch, length, key heads, heads, key dim, value dim, dtype, bias, state, lengths
    (2, 65, 1, 2, 64, 32, F32, True, True, None),
    (2, 130, 2, 4, 128, 64, BF16, True, False, None),
    (2, 20, 1, 1, 40, 24, F16, True, True, None),
    (1, 1, 2, 2, 64, 64, BF16, True, False, None),
    (1, 128, 1, 1, 128, 128, F32, True, True, None),
]
RAGGED = [(3, 130, 1, 2, 64, 48, BF16, True, True, [130, 0, 67]), (4, 70, 2, 2, 128, 32, F32, True, False, [1, 64, 70, 9])]


@pytest.mark.parametrize("which", [*STRIDED, "q dy", "q k v delta beta dy"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c[:7]).replace("torch.", ""))
def test_one_row_for_all_positions(case, which):
    c = _make(sum(case[:6]) + 5, *case)
    _same(dict(c, **{n: _repeated(c[n]) for n in which.split()}))


@pytest.mark.parametrize("case", RAGGED, ids=lambda c: "-".join(str(v) for v in c[:7]).replace("torch.", ""))
def test_one_row_for_all_positions_of_unequal_lengths(case):
    c = _make(sum(case[:6]) + 6, *case[:9])
    c["lengths"] = torch.tensor(case[9], dtype=torch.int32, device="cuda")
    for which in (("q", "dy"), ("k", "v"), STRIDED):
        _same(dict(c, **{n: _repeated(c[n]) for n in which}))


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_within_one_another(dtype, odd):
    c = _make(91, 2, 70, 1, 2, 64, 32, dtype, state=True)
    for which in (("q", "dy"), STRIDED):
        _same(dict(c, **{n: _within(c[n], 8 + odd if c[n].dim() == 4 else 1) for n in which}))


def test_a_broadcast_query_and_a_sum_over_positions():
    """One position alone: the gradients are those of the formula, not those of the 64 that a chunk has room for."""
    c = _make(92, 2, 1, 1, 2, 64, 32, F32)
    q, dy = (c[n][:, :1, :, :].expand(c[n].shape) for n in ("q", "dy"))
    q, dy = q.as_strided(q.shape, (q.stride(0), 0, *q.stride()[2:])), dy.as_strided(dy.shape, (dy.stride(0), 0, *dy.stride()[2:]))
    _same(dict(c, q=q, dy=dy))


@pytest.mark.parametrize("apart", [0, 1, 1 << 30, 1 << 40])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distances_that_mean_nothing(dtype, apart):
    """From a row to the next where there is one row."""
    c = _make(93, 2, 1, 2, 4, 64, 48, dtype, state=True)
    _same(dict(c, **{n: c[n].as_strided(c[n].shape, (c[n].stride(0), apart, *c[n].stride()[2:])) for n in STRIDED}))


def test_what_is_not_finite_in_a_row_within_another():
    """The last row's last columns hold what is not finite: in the columns in front of them nothing of it is seen."""
    c = _make(94, 1, 70, 1, 1, 64, 64, F32, state=True)
    room = torch.randn(69 * 8 + 64, device="cuda")
    room[-8:] = float("nan")
    v = room.as_strided(c["v"].shape, (room.numel(), 8, 64, 1))
    y, state = _forward(dict(c, v=v))
    assert torch.isfinite(y[..., :56]).all() and torch.isfinite(state[..., :56]).all() and torch.isnan(state[..., 56:]).all()
