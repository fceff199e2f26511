"""The selective scan against its recurrence in 64 bits (tests/sequence_reference.py has the tolerances' derivation)."""
import pytest
import torch

import sequence_reference as R
from paper_2010_15884_amd import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _make(seed, batch, length, channels, states, dtype, groups=1, gate=True, skip=True, bias=True, state=False, lengths=None, rank=3):
    g = _gen(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    bc = rand(batch, length, rank + 2 * groups * states).to(dtype)
    c = {"u": rand(batch, length, channels).to(dtype), "delta": (0.5 * rand(batch, length, channels)).to(dtype),
         "A": -torch.rand((channels, states), generator=g, device="cuda") * 4.0,
         "B": bc[..., rank:rank + groups * states].unflatten(-1, (groups, states)), "C": bc[..., rank + groups * states:].unflatten(-1, (groups, states)),
         "D": rand(channels) if skip else None, "z": rand(batch, length, 2 * channels).to(dtype)[..., channels:] if gate else None,
         "delta_bias": 0.5 * rand(channels) - 2.0 if bias else None, "state": rand(batch, channels, states) if state else None,
         "dy": rand(batch, length, channels + 1).to(dtype)[..., 1:], "dstate_out": rand(batch, channels, states) if state else None}
    if lengths is not None:
        for b, n in enumerate(lengths):
            for k, bad in (("u", float("nan")), ("delta", float("inf")), ("z", float("nan")), ("dy", float("-inf")), ("B", float("nan")), ("C", float("inf"))):
                if c[k] is not None:
                    c[k][b, max(n, 0):] = bad
    c["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    return c


def _inputs(c):
    return [c[k] for k in ("u", "delta", "A", "B", "C", "D", "z", "delta_bias")]


def _forward(c, softplus=True, **more):
    out = torch.full((c["u"].shape[0], *c["A"].shape), float("nan"), device="cuda")
    y = B.sys_selective_scan(*_inputs(c), softplus=softplus, d_state=c["state"], d_state_out=out, d_lengths=c["lengths"], **more)
    return y, out


def _check_all(c, lengths, softplus=True):
    batch, length, channels = c["u"].shape
    args = dict(softplus=softplus, state=c["state"], lengths=lengths, dy=c["dy"], dstate_out=c["dstate_out"])
    want, bound = R.scan(*_inputs(c), **args), R.scan(*_inputs(c), bound=True, **args)
    y, state = _forward(c, softplus)
    # L decays, each off by (12 |sA| + 6) u, the sum over the states, the skip and the gate (|z| < 6: (6 + 8) u) behind them
    chain = (length + 2) * (12 * want["sA"] + 6) * R.U
    sums = (c["A"].shape[1] + 4 + 20) * R.U
    R.check(state, want["state"], chain * bound["state"], "state")
    R.check(y, want["y"], (chain + sums) * bound["y"], "y")
    g = B.sys_selective_scan_backward(c["dy"], *_inputs(c), softplus=softplus, d_state=c["state"], d_lengths=c["lengths"], d_dstate_out=c["dstate_out"])
    both = 2 * chain + sums + 20 * R.U
    wide_sums = both + (64 + 64 + 16) * R.U
    for name, allowed in (("du", both), ("ddelta", both), ("dz", both), ("dstate", both), ("dA", wide_sums), ("dB", wide_sums), ("dC", wide_sums),
                          ("dD", wide_sums), ("ddelta_bias", wide_sums)):
        got = getattr(g, name)
        needs = {"dz": "z", "dD": "D", "ddelta_bias": "delta_bias", "dstate": "state"}.get(name)
        if needs and c[needs] is None:
            assert got is None
        else:
            R.check(got, want[name], allowed * bound[name], name)


CASES = [
    # batch, length, channels, states, dtype, groups, gate, skip, bias, state, lengths
    (2, 40, 64, 16, BF16, 1, True, True, True, False, None),
    (1, 1, 1, 1, F32, 1, True, True, True, True, None),
    (3, 1, 130, 16, F16, 2, False, True, True, True, None),
    (2, 17, 65, 2, F32, 1, True, False, True, True, None),
    (1, 65, 3, 3, BF16, 3, True, True, False, False, None),
    (2, 64, 96, 5, F32, 2, False, False, False, True, None),
    (2, 33, 70, 9, F32, 1, True, True, True, True, None),
    (1, 70, 66, 33, F16, 2, True, True, True, False, None),
    (2, 18, 10, 64, BF16, 1, True, True, True, True, None),
    (1, 130, 20, 48, F32, 2, False, True, True, True, None),
    (4, 81, 72, 16, F32, 1, True, True, True, True, [81, 0, 1, 64]),
    (3, 66, 36, 7, BF16, 3, True, True, True, False, [65, -5, 99]),
    (2, 20, 9, 64, F16, 1, True, False, True, True, [3, 20]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c[:6]).replace("torch.", ""))
def test_forward_and_gradients(case):
    lengths = case[10]
    _check_all(_make(sum(case[:4]), *case[:10], lengths), lengths)


def test_step_sizes_as_they_come():
    c = _make(3, 2, 30, 40, 16, F32, state=True)
    c["delta"], c["delta_bias"] = c["delta"].abs() * 0.2, None
    _check_all(c, None, softplus=False)


def test_long_sequences_in_chunks():
    """Few channels and many positions: chunks that run side by side, forwards and backwards."""
    c = _make(21, 1, 1111, 20, 16, F32, groups=2, state=True)
    _check_all(c, None)
    lengths = [700, 0]
    c = _make(22, 2, 1000, 5, 3, BF16, gate=True, state=True, lengths=lengths)
    _check_all(c, lengths)


@pytest.mark.parametrize("case", [
    # thousands of channels in few sequences
    (1, 83, 3300, 16, BF16, 1, True, True, True, False, None),
    (1, 81, 3211, 5, F32, 1, False, True, False, True, None),
    (3, 70, 1100, 16, F32, 2, True, False, True, True, [70, 0, 33]),
    (2, 66, 1650, 33, F16, 3, True, True, True, True, [17, 65]),
    (1, 97, 3203, 17, BF16, 1, True, True, True, True, None),
], ids=lambda c: "-".join(str(v) for v in c[:6]).replace("torch.", ""))
def test_many_channels(case):
    c = _make(sum(case[:4]), *case[:10], case[10])
    args = dict(state=c["state"], lengths=case[10])
    want, bound = R.scan(*_inputs(c), **args), R.scan(*_inputs(c), bound=True, **args)
    y, state = _forward(c)
    chain = (case[1] + 2) * (12 * want["sA"] + 6) * R.U
    R.check(state, want["state"], chain * bound["state"], "state")
    R.check(y, want["y"], (chain + (case[3] + 24) * R.U) * bound["y"], "y")


def test_step_sizes_of_every_size():
    """softplus far out on both sides: results keep their relative accuracy where e^delta is all that is left."""
    delta = torch.tensor([-100.0, -80.0, -40.0, -20.0, -10.0, -5.0, -1e-4, 0.0, 1e-4, 1.0, 5.0, 15.0, 30.0, 80.0], device="cuda")[None, :, None].contiguous()
    u, one = torch.ones_like(delta), torch.ones((1, 14, 1, 1), device="cuda")
    out = torch.empty((1, 1, 1), device="cuda")
    y = B.sys_selective_scan(u, delta, torch.full((1, 1), -1e30, device="cuda"), one, one, softplus=True, d_state_out=out)
    want = torch.logaddexp(delta.double(), torch.zeros_like(delta.double())).cpu()         # nothing is remembered: y = s
    # (e^-100 and e^-80 are below or near the smallest normal number and may be 0)
    assert ((y.double().cpu() - want).abs() <= 10 * R.U * want + 1e-34).all()


def test_empty_length_and_batch():
    c = _make(1, 2, 0, 20, 16, BF16, state=True)
    y, out = _forward(c)
    assert y.shape == (2, 0, 20) and torch.equal(out, c["state"])
    g = B.sys_selective_scan_backward(c["dy"], *_inputs(c), softplus=True, d_state=c["state"], d_dstate_out=c["dstate_out"])
    assert g.du.shape == (2, 0, 20) and torch.equal(g.dstate, c["dstate_out"]) and not g.dA.any() and not g.dD.any() and not g.ddelta_bias.any()
    c = _make(1, 0, 7, 20, 16, BF16)
    assert _forward(c)[0].shape == (0, 7, 20)
    assert not B.sys_selective_scan_backward(c["dy"], *_inputs(c), softplus=True).dA.any()


@pytest.mark.parametrize("states,dtype,groups", [(16, BF16, 1), (1, F32, 2), (5, F16, 1), (64, BF16, 3), (36, F32, 1)])
def test_prompts_in_pieces_and_tokens(states, dtype, groups):
    """A prompt in two pieces, then token by token out of a cache of states, against the whole in 64 bits."""
    c = _make(states, 3, 24, 42, states, dtype, groups, state=True)
    want, bound = R.scan(*_inputs(c), state=c["state"]), R.scan(*_inputs(c), state=c["state"], bound=True)
    cut = lambda a, b: [c[k][:, a:b] if k in ("u", "delta", "B", "C", "z") else c[k] for k in ("u", "delta", "A", "B", "C", "D", "z", "delta_bias")]  # noqa: E731
    mid, end = torch.empty_like(c["state"]), torch.empty_like(c["state"])
    got = [B.sys_selective_scan(*cut(0, 7), softplus=True, d_state=c["state"], d_state_out=mid),
           B.sys_selective_scan(*cut(7, 20), softplus=True, d_state=mid, d_state_out=end)]
    cache = torch.zeros((6, 42, states), device="cuda")
    slots = torch.tensor([5, 1, 2], dtype=torch.int32, device="cuda")
    cache[slots.long()] = end
    for t in range(20, 24):
        u, delta, A, Bt, Ct, D, z, bias = cut(t, t + 1)
        got.append(B.sys_selective_scan_update(u[:, 0], delta[:, 0], A, Bt[:, 0], Ct[:, 0], cache, D, z[:, 0], bias, softplus=True, d_slots=slots)[:, None])
    chain = 26 * (12 * want["sA"] + 6) * R.U
    R.check(torch.cat(got, dim=1), want["y"], (chain + (states + 24) * R.U) * bound["y"], "y")
    R.check(cache[slots.long()], want["state"], chain * bound["state"], "state")
    assert not cache[[0, 3, 4]].any()


def test_tokens_skip_slots_that_are_not_there():
    c = _make(4, 4, 1, 12, 16, F32)
    cache = torch.randn((3, 12, 16), generator=_gen(2), device="cuda")
    before, other = cache.clone(), torch.full_like(cache, 7)
    slots = torch.tensor([1, -1, 3, 0], dtype=torch.int32, device="cuda")
    args = [c[k][:, 0] for k in ("u", "delta")] + [c["A"]] + [c[k][:, 0] for k in ("B", "C")]
    rest = [c["D"], c["z"][:, 0], c["delta_bias"]]
    y = B.sys_selective_scan_update(*args, cache, *rest, softplus=True, d_slots=slots, d_state_out=other)
    assert torch.equal(cache, before)
    assert torch.equal(B.sys_selective_scan_update(*args, cache, *rest, softplus=True, d_slots=slots), y)
    assert not y[[1, 2]].any() and torch.equal(cache[2], before[2]) and (other[2] == 7).all()
    assert torch.equal(other[:2], cache[:2]) and not torch.equal(cache[:2], before[:2])


def test_offsets_beyond_32_bits():
    c = _make(6, 2, 20, 70, 16, BF16)
    want = _forward(c)[0]
    far = torch.empty(1 << 32, dtype=BF16, device="cuda")
    u = far.as_strided((2, 20, 70), ((1 << 31) + 5, (1 << 25) + 3, 1))
    u.copy_(c["u"])
    assert torch.equal(_forward(dict(c, u=u))[0], want)
    grads, far_grads = (B.sys_selective_scan_backward(c["dy"], v, *_inputs(c)[1:], softplus=True) for v in (c["u"], u))
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(grads, far_grads))
    del far, u
    cache = torch.zeros(((1 << 31) // (70 * 16) + 3, 70, 16), device="cuda")
    slots = torch.tensor([cache.shape[0] - 1, 1], dtype=torch.int32, device="cuda")
    args = [c[k][:, 0] for k in ("u", "delta")] + [c["A"]] + [c[k][:, 0] for k in ("B", "C")]
    small = torch.zeros((2, 70, 16), device="cuda")
    rest = [c["D"], c["z"][:, 0], c["delta_bias"]]
    y = B.sys_selective_scan_update(*args, cache, *rest, softplus=True, d_slots=slots)
    assert torch.equal(y, B.sys_selective_scan_update(*args, small, *rest, softplus=True))
    assert torch.equal(cache[slots.long()], small)


def test_rows_beyond_32_bits_and_the_widest_that_are_taken():
    far = torch.empty(75 << 25, dtype=BF16, device="cuda")
    for channels, states in ((70, 16), (3300, 5)):
        c = _make(8, 1, 75, channels, states, BF16)
        u = far.as_strided((1, 75, channels), (far.numel(), 1 << 25, 1))
        u.copy_(c["u"])
        assert torch.equal(_forward(dict(c, u=u))[0], _forward(c)[0])
        grads, far_grads = (B.sys_selective_scan_backward(c["dy"], v, *_inputs(c)[1:], softplus=True) for v in (c["u"], u))
        assert all(p is q is None or torch.equal(p, q) for p, q in zip(grads, far_grads))
    c = _make(9, 1, 2, 70, 16, BF16)
    u = far.as_strided((1, 2, 70), (far.numel(), (1 << 26) - 1, 1))
    u.copy_(c["u"])
    assert torch.equal(_forward(dict(c, u=u))[0], _forward(c)[0])
    with pytest.raises(B.SysconvError):
        _forward(dict(c, u=far.as_strided((1, 2, 70), (far.numel(), 1 << 26, 1))))


def test_gradients_against_differences():
    """As in test_gpu_causal_conv: central differences of L = <y, r> + <state_out, r'>, e = 2^-7."""
    c = _make(31, 2, 21, 12, 5, F32, groups=2, state=True, lengths=[21, 13])
    for k in ("u", "delta", "z", "dy", "B", "C"):
        c[k][1, 13:] = 0.0
    names = ["u", "delta", "A", "B", "C", "D", "z", "delta_bias", "state"]
    point = {k: c[k].contiguous() for k in names}

    def loss(p):
        y, out = _forward(dict(c, **p))
        return float((y.double() * c["dy"].double()).sum() + (out.double() * c["dstate_out"].double()).sum())

    g = B.sys_selective_scan_backward(c["dy"], *[point[k] for k in names[:8]], softplus=True, d_state=point["state"], d_lengths=c["lengths"],
                                      d_dstate_out=c["dstate_out"])
    rng = _gen(32)
    for name in names:
        grad = getattr(g, "d" + name)
        v = torch.randn(point[name].shape, generator=rng, device="cuda")
        e = 2.0 ** -7
        slope = (loss({**point, name: point[name] + e * v}) - loss({**point, name: point[name] - e * v})) / (2 * e)
        size = float((grad.double() * v.double()).abs().sum())
        assert abs(slope - float((grad.double() * v.double()).sum())) <= 2e-3 * size, name


def test_what_is_not_finite_stays_where_it_belongs():
    """A NaN in one channel of one sequence: other channels and sequences as without it, and positions before it."""
    c = _make(41, 2, 40, 70, 16, F32)
    clean, _ = _forward(c)
    c["u"][0, 20, 5] = float("nan")
    y, state = _forward(c)
    bad = ~torch.isfinite(y)
    assert bad[0, 20:, 5].all() and int(bad.sum()) == 20
    assert torch.equal(y[~bad], clean[~bad]) and int((~torch.isfinite(state)).sum()) == 16


def test_same_bits_every_time_on_any_stream_and_from_a_graph():
    c = _make(51, 2, 600, 130, 16, BF16, state=True)

    def calls():
        y, out = _forward(c)
        return [y, out, *B.sys_selective_scan_backward(c["dy"], *_inputs(c), softplus=True, d_state=c["state"])]

    want = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, out = _forward(c, stream=side.cuda_stream)
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
