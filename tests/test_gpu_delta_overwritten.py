"""Values that are written over much larger ones: what a key gives back is the new value, whose digits do not go by the old one's size.

With strength 1 and a query that is the position's key (of length one) y = scale v: S^T k is taken out and v put in.  In a chunk y is the sum of scale e^G S^T q, of the size of
the old value, and of what the chunk's positions write, which takes it back.  Let m be the root of the mean square of S^T k over the positions and columns of a head.  What the numbers
that are multiplied are rounded to and the terms left out are worth 2^-24 of a term each and as often up as down, and so is a sum's rounding; a result is made of four products
(K S, the inverse times what misses, Q S, P U) of up to key_dim or 64 terms, whose squares add up to m^2 for K S and Q S and to at most 64 m^2 for the others: in norm
sqrt(2 key_dim + 2 * 64) 2^-24 m for the sums' roundings and no more for the numbers', 2 sqrt(2 * 128 + 2 * 64) 2^-24 m = 2.4e-6 m together.  On top of it comes the rounding to the
type, at most half a step of each value.
"""
import pytest
import torch

import delta_reference as D
import sequence_reference as R
from paper_2010_15884_amd import binding as B

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("length", [5, 64, 150])
@pytest.mark.parametrize("key_dim,value_dim,heads", [(64, 48, 2), (128, 32, 2), (128, 256, 18)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_new_values_over_large_ones(dtype, key_dim, value_dim, heads, length):
    g = torch.Generator(device="cuda").manual_seed(key_dim + length)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    # keys of length one in every type: four entries of one half, each with a sign
    k = torch.zeros((1, length, heads, key_dim), device="cuda")
    at = torch.argsort(torch.rand((1, length, heads, key_dim), generator=g, device="cuda"), dim=-1)[..., :4]
    k.scatter_(3, at, 0.5 * torch.sign(rand(1, length, heads, 4)))
    k, v = k.to(dtype), rand(1, length, heads, value_dim).to(dtype)
    state = 3000.0 * rand(1, heads, key_dim, value_dim)
    delta, beta, A = (torch.full((1, length, heads), x, device="cuda").to(dtype) for x in (0.01, 1.0, 0.0))
    A = torch.zeros(heads, device="cuda")          # nothing is forgotten
    y = B.sys_gated_delta_rule(k, k, v, delta, A, beta, scale=1.0, d_state=state)
    want = D.gated_delta(k, k, v, delta, A, beta, scale=1.0, softplus=False, sigmoid_beta=False, state=state)
    assert float((want["y"] - R.wide(v)).abs().max()) < 1e-9                       # the new value
    sizes, held = torch.zeros(heads, dtype=torch.float64), R.wide(state)[0]
    for t in range(length):
        old = torch.einsum("hkv,hk->hv", held, R.wide(k)[0, t])
        held = held + R.wide(k)[0, t, :, :, None] * (R.wide(v)[0, t] - old)[:, None]
        sizes += old.square().sum(dim=1)
    size = lambda x: (x.square().sum(dim=(1, 3)) / (length * value_dim)).sqrt()    # noqa: E731
    error = size(R.wide(y) - want["y"])[0]
    allowed = 2.4e-6 * (sizes / (length * value_dim)).sqrt() + (torch.finfo(dtype).eps / 2) * size(want["y"])[0]
    assert (error <= allowed).all(), (error / allowed).max()


@pytest.mark.parametrize("length", [64, 150])
@pytest.mark.parametrize("key_dim,shared", [(16, 1), (32, 2)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_gradients_of_queries_behind_an_overwritten_state(dtype, key_dim, shared, length):
    """dq = scale S dy, with S the state behind the position: small where its chunk has written over all that was there, though the state before the chunk was large.

    The first key_dim positions have the unit vectors as keys and strength 1, so that the state behind them has nothing of the old one's m = 3000 a column and entry left.  In
    the chunk dq is the sum of scale e^G S dy over value_dim columns and of B K, which takes it back: products of numbers of 24 bits (2^-24 of a term, as often up as down)
    and sums of value_dim and of two times 64 terms (U, B, and B K), whose squares add up to value_dim (m |dy|)^2 / value_dim each, in norm over the entries: sqrt(2 value_dim + 4 * 64) 2^-24
    m |dy| for the sums and no more for the numbers.  On top of it comes the rounding to the type."""
    g = torch.Generator(device="cuda").manual_seed(key_dim + length)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    value_dim, heads = 48, 2
    k = torch.nn.functional.normalize(rand(1, length, heads // shared, key_dim), dim=-1) * 0.99
    k[0, :key_dim] = torch.eye(key_dim, device="cuda")[:, None]
    k, q, v = k.to(dtype), rand(1, length, heads // shared, key_dim).to(dtype), rand(1, length, heads, value_dim).to(dtype)
    dy = rand(1, length, heads, value_dim)
    dy[0, :key_dim] = 0.0                          # (what was large is not asked for)
    dy = dy.to(dtype)
    state = 3000.0 * rand(1, heads, key_dim, value_dim)
    delta, A = torch.full((1, length, heads), 0.01, device="cuda").to(dtype), torch.zeros(heads, device="cuda")
    beta = torch.full((1, length, heads), 0.5, device="cuda").to(dtype)
    beta[0, :key_dim] = 1.0
    got = B.sys_gated_delta_rule_backward(dy, q, k, v, delta, A, beta, scale=1.0, d_state=state)
    want = D.gated_delta(q, k, v, delta, A, beta, scale=1.0, softplus=False, sigmoid_beta=False, state=state, dy=dy)["dq"]
    error = (R.wide(got.dq) - want).norm(dim=3)[0, key_dim:].norm(dim=1)           # of a position, over heads and entries
    size = R.wide(dy).norm(dim=3)[0, key_dim:].norm(dim=1)
    allowed = 2 * (2 * value_dim + 4 * 64) ** 0.5 * 2.0 ** -24 * 3000.0 * key_dim ** 0.5 * size + (torch.finfo(dtype).eps / 2) * want[0, key_dim:].flatten(1).norm(dim=1)
    assert float(want[0, key_dim:].abs().max()) < 100.0
    assert (error <= allowed).all(), (error / allowed).max()
