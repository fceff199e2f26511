"""The norm of queries and keys with the rotation of positions against its formulas in 64 bits (tests/delta_reference.py has the tolerances' derivation)."""
import pytest
import torch

import delta_reference as D
import sequence_reference as R
from paper_2010_15884_amd import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _make(seed, batch, length, q_heads, k_heads, dim, rotary, dtype, weights=True, param=None, positions=True, lengths=None, table=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    row = rand(batch, length, (q_heads + 2 * k_heads) * dim + 3).to(dtype)
    split = lambda t, at, h: t[..., at:at + h * dim].unflatten(-1, (h, dim))  # noqa: E731
    c = {"q": split(row, 3, q_heads), "k": split(row, 3 + q_heads * dim, k_heads) if k_heads else None}
    dy = rand(batch, length, (q_heads + k_heads) * dim + 1).to(dtype)
    c["dyq"], c["dyk"] = split(dy, 1, q_heads), split(dy, 1 + q_heads * dim, k_heads) if k_heads else None
    param = dtype if param is None else param
    c["wq"] = (1.0 + 0.3 * rand(dim)).to(param) if weights else None
    c["wk"] = (1.0 + 0.3 * rand(dim)).to(param) if weights and k_heads else None
    c["cos"] = c["sin"] = c["positions"] = None
    if rotary:
        n = table or length + 5
        angle = 6.3 * torch.rand((n, rotary // 2), generator=g, device="cuda")
        c["cos"], c["sin"] = torch.cos(angle), torch.sin(angle)
        if positions:
            c["positions"] = torch.randint(0, n, (batch, length), generator=g, device="cuda", dtype=torch.int32)
    if lengths is not None:
        for b, m in enumerate(lengths):
            for t in (c["q"], c["k"], c["dyq"], c["dyk"]):
                if t is not None:
                    t[b, max(m, 0):] = float("nan")
    c["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    return c


def _shared(c):
    return [c[n] for n in ("cos", "sin", "positions")]


def _check(c, **how):
    yq, yk = B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c), d_lengths=c["lengths"], **how)
    dq, dk, dwq, dwk = B.sys_head_norm_backward(c["dyq"], c["dyk"], c["q"], c["k"], c["wq"], c["wk"], *_shared(c), d_lengths=c["lengths"], **how)
    for x, w, dy, y, dx, dw in ((c["q"], c["wq"], c["dyq"], yq, dq, dwq), (c["k"], c["wk"], c["dyk"], yk, dk, dwk)):
        if x is None:
            assert y is None and dx is None and dw is None
            continue
        want = D.head_norm(x, w, *_shared(c), lengths=c["lengths"], dy=dy, **how)
        R.check(y, want["y"], want["room"]["y"], "y")
        R.check(dx, want["dx"], want["room"]["dx"], "dx")
        if w is None:
            assert dw is None
        else:
            R.check(dw, want["dw"], want["room"]["dw"], "dw")


CASES = [
    # batch, length, q heads, k heads, dim, rotary, dtype
    (1, 1, 1, 1, 1, 0, F32),
    (1, 1, 1, 1, 2, 2, F32),
    (2, 3, 4, 2, 64, 64, BF16),
    (2, 5, 3, 1, 128, 128, F16),
    (3, 7, 5, 3, 128, 64, F32),
    (1, 9, 6, 6, 96, 0, BF16),
    (2, 4, 2, 1, 50, 22, F32),
    (1, 6, 3, 2, 33, 10, BF16),
    (1, 70, 1, 1, 40, 40, F16),
    (2, 3, 17, 5, 72, 72, BF16),
    (1, 3, 2, 2, 127, 126, F16),
    (1, 4, 2, 1, 129, 2, F32),
    (1, 5, 2, 2, 255, 254, BF16),
    (1, 5, 3, 0, 256, 64, BF16),
    (2, 2, 2, 1, 512, 512, F32),
    (1, 2, 1, 1, 511, 0, F16),
    (1, 2, 2, 1, 510, 34, BF16),
    (1, 2, 70, 9, 16, 8, F16),
    (1, 3, 40, 2, 8, 8, F32),
]


@pytest.mark.parametrize("norm,interleaved", [("RMS", False), ("L2", True)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace("torch.", ""))
def test_forward_and_gradients(case, norm, interleaved):
    _check(_make(sum(case[:6]), *case), norm=norm, interleaved=interleaved)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_lengths_positions_and_weights(dtype, interleaved):
    c = _make(3, 4, 9, 6, 2, 64, 32, dtype, param=F32, lengths=[9, 0, 4, -2])
    _check(c, interleaved=interleaved)
    _check(dict(c, positions=None), interleaved=interleaved)
    _check(_make(4, 2, 9, 3, 3, 48, 16, dtype, weights=False), interleaved=interleaved, eps=1e-3)
    one = _make(5, 2, 5, 3, 3, 48, 16, dtype)
    _check(dict(one, wk=None), interleaved=interleaved)
    _check(dict(one, wq=None), interleaved=interleaved)


def test_tokens_that_are_not_there():
    c = _make(6, 2, 8, 3, 1, 64, 64, BF16)
    c["positions"][0, 3], c["positions"][1, 0], c["positions"][1, 7] = -1, c["cos"].shape[0], 2 ** 31 - 1
    for t in (c["q"], c["k"], c["dyq"], c["dyk"]):
        t[0, 3], t[1, 0] = float("nan"), float("inf")
    _check(c)
    yq, _ = B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c))
    assert (yq[0, 3] == 0).all() and (yq[1, 0] == 0).all() and (yq[1, 7] == 0).all()
    empty = dict(c, cos=c["cos"][:0].contiguous(), sin=c["sin"][:0].contiguous())
    yq, yk = B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(empty))
    assert (yq == 0).all() and (yk == 0).all()


def test_many_tokens_and_heads():
    """Sums of the weights over several workgroups, and wavefronts with several turns."""
    _check(_make(7, 3, 700, 4, 2, 64, 64, BF16))
    _check(_make(8, 1, 2500, 9, 3, 24, 8, F32), interleaved=True)


def test_outputs_given_and_strided():
    c = _make(9, 2, 5, 4, 2, 64, 64, BF16)
    wide_q, wide_k = torch.full((2, 5, 5, 64), 7.0, device="cuda", dtype=BF16), torch.full((3, 5, 2, 64), 7.0, device="cuda", dtype=BF16)
    B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c), d_yq=wide_q[:, :, :4], d_yk=wide_k[:2])
    yq, yk = B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c))
    assert torch.equal(wide_q[:, :, :4], yq) and torch.equal(wide_k[:2], yk)
    assert (wide_q[:, :, 4] == 7).all() and (wide_k[2] == 7).all()


def test_values_that_are_not_finite_stay_in_their_head():
    c = _make(10, 1, 4, 4, 1, 128, 128, F32)
    clean, _ = B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c))
    c["q"][0, 1, 2, 5], c["q"][0, 2, 0, 0] = float("nan"), float("inf")
    y, _ = B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c))
    bad = torch.zeros(y.shape[:3], dtype=torch.bool, device="cuda")
    bad[0, 1, 2] = bad[0, 2, 0] = True
    assert torch.equal(y[~bad], clean[~bad]) and torch.isnan(y[0, 1, 2]).all() and torch.isnan(y[0, 2, 0, 0])


def test_empty():
    c = _make(11, 2, 3, 2, 1, 16, 8, F32)
    yq, yk = B.sys_head_norm(c["q"][:0], c["k"][:0], c["wq"], c["wk"], c["cos"], c["sin"])
    assert yq.shape[0] == 0 == yk.shape[0]
    dq, dk, dwq, dwk = B.sys_head_norm_backward(c["dyq"][:, :0], c["dyk"][:, :0], c["q"][:, :0], c["k"][:, :0], c["wq"], c["wk"], c["cos"], c["sin"])
    assert dq.shape[1] == 0 and (dwq == 0).all() and (dwk == 0).all()


def test_runs_repeat_and_capture():
    c = _make(12, 2, 300, 6, 2, 64, 64, BF16)
    call = lambda: (*B.sys_head_norm(c["q"], c["k"], c["wq"], c["wk"], *_shared(c)),  # noqa: E731
                    *B.sys_head_norm_backward(c["dyq"], c["dyk"], c["q"], c["k"], c["wq"], c["wk"], *_shared(c)))
    first = call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for turn in range(3):
        c["q"].mul_(-1.0 if turn else 1.0)
        want = call()
        for o in out:
            o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert torch.equal(first[1], out[1])
