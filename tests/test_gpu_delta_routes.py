"""The gated delta rule and the norm of heads by the routes that sizes, alignment and strides choose: aligned rows, many columns, rows far apart,
caches beyond 32 bits, several streams, the operators one after the other."""
import pytest
import torch

import delta_reference as D
import sequence_reference as R
import test_gpu_head_norm as H
from paper_2010_15884_amd import binding as B
from test_gpu_gated_delta import BF16, F16, F32, INPUTS, _backward, _check_forward, _check_gradients, _forward, _make, _reference, _step, ids

pytestmark = pytest.mark.gpu

# rows that start at 16 bytes: wide loads of keys and values
ALIGNED = [
    # batch, length, key heads, heads, key dim, value dim, dtype, bias, state, lengths
    (2, 130, 2, 4, 64, 64, BF16, True, True, [130, 77]),
    (1, 192, 2, 2, 128, 128, BF16, True, False, None),
    (9, 129, 1, 1, 64, 32, F32, True, True, [0, 1, 16, 17, 63, 64, 65, 128, 129]),
    (9, 129, 1, 2, 128, 40, F16, False, True, [129, 128, 65, 64, 63, 17, 16, 1, 0]),
    (1, 100, 1, 8, 72, 24, BF16, True, True, None),
    (2, 70, 1, 2, 128, 64, F32, True, True, [70, 3]),
    (1, 17, 1, 1, 8, 8, F16, True, True, None),
]
# more than 256 tiles of 16 columns: 32 columns a workgroup
MANY = [
    (4, 70, 2, 8, 24, 144, F32, True, True, None),
    (3, 66, 1, 3, 128, 1023, BF16, True, True, [66, 64, 2]),
    (2, 129, 5, 10, 64, 216, F16, True, False, None),
    (5, 65, 3, 6, 128, 148, F16, True, True, [65, 0, 31, 64, 1]),
    (2, 80, 1, 3, 128, 1024, F32, True, True, None),
    (4, 70, 8, 8, 64, 136, BF16, True, True, [70, 69, 0, 64]),
]


@pytest.mark.parametrize("case", ALIGNED, ids=ids)
def test_aligned_rows(case):
    c = _make(sum(case[:6]) + 2, *case, odd=0)
    _check_forward(c)
    c["dy"] = c["dy"].contiguous()
    _check_gradients(c)


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("case", MANY, ids=ids)
def test_many_columns(case, odd):
    c = _make(sum(case[:6]) + 3, *case, odd=odd)
    _check_forward(c)
    _check_gradients(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_far_apart(dtype):
    """As far as is taken, a chunk's rows over nearly 4 GiB in fp32; what lies between the rows of y stays as it was."""
    c = _make(71, 1, 70, 1, 2, 32, 24, dtype, state=True)
    apart = (1 << 24) - 1
    columns, results = (torch.full((69 * apart + 2000,), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    at = 1

    def far(t):
        nonlocal at
        view = columns.as_strided(t.shape, (columns.numel(), apart, *([t.shape[3], 1] if t.dim() == 4 else [1])), at)
        at += t[0, 0].numel() + 1
        return view
    apart_too = dict(c)
    for n in ("q", "k", "v", "delta", "beta", "dy"):
        apart_too[n] = far(c[n])
        apart_too[n].copy_(c[n])
    y = results.as_strided(c["v"].shape, (results.numel(), apart, c["v"].shape[3], 1))
    want = _forward(c)[0]
    _forward(apart_too, d_y=y)
    assert torch.equal(y, want)
    for a, b in zip(_backward(apart_too), _backward(c)):
        assert torch.equal(a, b)
    for r in range(69):
        assert (results[r * apart + y[0, 0].numel():(r + 1) * apart] == 7.0).all(), r
    # one element further is refused
    c["q"] = columns.as_strided((1, 3, 1, 32), (columns.numel(), apart + 1, 32, 1))
    with pytest.raises(B.SysconvError):
        B.sys_gated_delta_rule(*[t if t is None or t.dim() == 1 else t[:, :3] for t in (c[n] for n in INPUTS)])


def test_caches_beyond_32_bits():
    c = _make(72, 3, 1, 1, 2, 64, 64, BF16, state=True)
    slots = (1 << 32) // (2 * 64 * 64) + 7         # the last states begin behind 2^32 elements
    cache = torch.empty((slots, 2, 64, 64), device="cuda")
    order = [slots - 1, 0, slots - 3]
    cache[order] = c["state"]
    cache[slots - 2] = 5.0
    want = _reference(c)
    allowed = D.delta_allowed(dict(c, dy=None), want, 1, BF16)
    y = _step(c, cache, d_slots=torch.tensor(order, dtype=torch.int32, device="cuda"))
    R.check(y, want["y"][:, 0], allowed["y"][:, 0], "y")
    R.check(cache[order], want["state"], allowed["state"], "state")
    assert (cache[slots - 2] == 5.0).all()


def test_heads_beyond_32_bits():
    """Rows of the norm's tensors that begin behind 2^31 and 2^32 elements."""
    c = H._make(73, 2, 3, 4, 2, 64, 32, BF16)
    apart = (1 << 30) + 8
    room, results = (torch.full((5 * apart + 2000,), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    far = lambda of, at: of.as_strided(c["q"].shape, (3 * apart - 64, apart, 64, 1), at)  # noqa: E731
    q, dyq, yq = far(room, 0), far(room, 400), far(results, 0)
    q.copy_(c["q"])
    dyq.copy_(c["dyq"])
    shared = [c["wq"], c["wk"], *H._shared(c)]
    want, _ = B.sys_head_norm(c["q"], c["k"], *shared)
    B.sys_head_norm(q, c["k"], *shared, d_yq=yq)
    assert torch.equal(yq, want)
    for a, b in zip(B.sys_head_norm_backward(dyq, c["dyk"], q, c["k"], *shared), B.sys_head_norm_backward(c["dyq"], c["dyk"], c["q"], c["k"], *shared)):
        assert torch.equal(a, b)
    assert (results[256:apart] == 7.0).all() and (results[apart + 256:2 * apart] == 7.0).all() and (results[2 * apart + 256:3 * apart - 64] == 7.0).all()


def test_calls_side_by_side():
    """Two streams at once, each with its own outputs and workspaces."""
    cs = [_make(74 + i, 2, 300, 2, 4, 64, 64, BF16, state=True) for i in range(2)]
    want = [(*_forward(c), *_backward(c)) for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    got = []
    for _ in range(3):
        got.append([(*_forward(c, stream=s.cuda_stream), *_backward(c, stream=s.cuda_stream)) for c, s in zip(cs, streams)])
    torch.cuda.synchronize()
    for turn in got:
        assert all(torch.equal(a, b) for g, w in zip(turn, want) for a, b in zip(g, w))


def test_states_that_are_not_finite_stay_in_their_column():
    c = _make(76, 2, 90, 2, 2, 64, 64, F32, state=True)
    clean, clean_state = _forward(c)
    c["state"][1, 0, 7, 20] = float("inf")
    y, state = _forward(c)
    others = torch.arange(64, device="cuda") != 20
    assert torch.equal(y[0], clean[0]) and torch.equal(y[1, :, 1], clean[1, :, 1]) and torch.equal(y[1, :, 0][:, others], clean[1, :, 0][:, others])
    assert not torch.isfinite(y[1, 1:, 0, 20]).any() and torch.equal(state[1, 0][:, others], clean_state[1, 0][:, others])


@pytest.mark.parametrize("dtype,key_dim", [(F32, 64), (F16, 40), (BF16, 128)])
def test_many_sequences(dtype, key_dim):
    """More chunks of key heads than CUs: a workgroup goes through the value heads that share keys, instead of one of them."""
    lengths = [(0, 1, 2, 3)[b % 4] for b in range(150)]
    lengths[7], lengths[31], lengths[149] = 70, 64, 65
    c = _make(79, 150, 70, 2, 6, key_dim, 16, dtype, state=True, lengths=lengths)
    _check_forward(c)
    _check_gradients(c)


@pytest.mark.parametrize("batch,length", [(1, 12), (1, 13), (64, 20), (64, 21)])
def test_lengths_between_the_routes(batch, length):
    _check_forward(_make(80 + length, batch, length, 2, 4, 40, 24, BF16, state=True))


@pytest.mark.parametrize("length", [9, 100])
def test_rows_behind_a_sequence_are_zero_whatever_the_state_is(length):
    c = _make(78, 3, length, 1, 2, 64, 48, BF16, state=True, lengths=[length - 4, 0, 5])
    c["state"][:, 0, 3, 7], c["dstate_out"][:, 1, 2, 9] = float("inf"), float("nan")
    y, _ = _forward(c)
    grads = _backward(c)
    for b, n in enumerate([length - 4, 0, 5]):
        for t in (y, grads.dq, grads.dk, grads.dv, grads.ddelta, grads.dbeta):
            assert (t[b, n:] == 0).all()
    assert not torch.isfinite(y[0, :length - 4, 0, 7]).any()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_operators_in_a_row(dtype):
    """Convolution, norm of queries and keys, delta rule, norm of the results: each of what the one before left, over ragged prompts and one token more."""
    g = torch.Generator(device="cuda").manual_seed(77)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    batch, length, hk, h, dk, dv, taps, ns = 3, 90, 2, 4, 48, 40, 4, [89, 1, 64]
    columns = 2 * hk * dk + h * dv
    x = rand(batch, length, columns + 2 * h).to(dtype)
    w, bias, norm_w = (0.5 * rand(columns, taps)).to(dtype), 0.1 * rand(columns).to(dtype), (1.0 + 0.2 * rand(dv)).to(dtype)
    A, step_bias = -torch.rand(h, generator=g, device="cuda"), rand(h) - 2.0

    def heads(t):
        return t[..., :hk * dk].unflatten(-1, (hk, dk)), t[..., hk * dk:2 * hk * dk].unflatten(-1, (hk, dk)), t[..., 2 * hk * dk:].unflatten(-1, (h, dv))

    def run(x, lengths):
        rows = torch.empty((batch, taps - 1, columns), device="cuda", dtype=dtype)
        state = torch.empty((batch, h, dk, dv), device="cuda")
        mixed = B.sys_causal_conv1d(x[..., :columns], w, bias, activation="SILU", d_state_out=rows, d_lengths=lengths)
        q, k, v = heads(mixed)
        q, k = B.sys_head_norm(q, k, norm="L2", d_lengths=lengths)
        y = B.sys_gated_delta_rule(q, k, v, x[..., columns:columns + h], A, x[..., columns + h:], step_bias, softplus=True, sigmoid=True, d_state_out=state,
                                   d_lengths=lengths)
        return B.sys_head_norm(y, d_wq=norm_w, d_lengths=lengths)[0], rows, state
    whole, _, _ = run(x, None)
    lengths = torch.tensor(ns, dtype=torch.int32, device="cuda")
    padded = x.clone()
    for b, n in enumerate(ns):
        padded[b, n:] = float("nan")
    y, rows, state = run(padded, lengths)
    for b, n in enumerate(ns):
        assert torch.equal(y[b, :n], whole[b, :n]) and (y[b, n:] == 0).all()
    at = (torch.arange(batch, device="cuda"), lengths.long())
    token = x[at]
    q, k, v = heads(B.sys_causal_conv1d_update(token[:, :columns], w, bias, rows, activation="SILU"))
    q, k = B.sys_head_norm(q[:, None], k[:, None], norm="L2")
    t = B.sys_gated_delta_rule_update(q[:, 0], k[:, 0], v, token[:, columns:columns + h], A, token[:, columns + h:], state, step_bias, softplus=True, sigmoid=True)
    got = B.sys_head_norm(t[:, None], d_wq=norm_w)[0][:, 0].double()
    # The delta rule's results are rounded to the type on both sides, and by a position at a time or a chunk (here a thousand times less in fp32: 100 * 2^-24 of a
    # result's largest entries); a root of a mean square divides by no less than the entries are, and multiplies their error by at most 1 + sqrt(dv) on the way.
    eps = torch.finfo(dtype).eps / 2
    assert float((got - whole[at].double()).abs().max()) <= (3 * eps + 300 * 2.0 ** -24) * (1 + dv ** 0.5) * float(whole[at].abs().max())
