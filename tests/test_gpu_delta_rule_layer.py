"""The example layer: runs, serves what it computes over whole sequences, and its gradients are those of the formulas and of differences."""
import os
import runpy

import pytest
import torch

pytestmark = pytest.mark.gpu

EXAMPLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "delta_rule_layer.py")


def test_example_layer(capsys):
    runpy.run_path(EXAMPLE, run_name="__main__")
    assert "all good" in capsys.readouterr().out


def _in_64_bits(layer, p, h):
    """The layer's output from its formulas, on the CPU."""
    x, z, delta, beta = (h @ p["into"].T).split(layer.sizes, dim=-1)
    taps = p["w"].shape[1]
    padded = torch.nn.functional.pad(x, (0, 0, taps - 1, 0))
    x = torch.nn.functional.silu(p["bias"] + sum(p["w"][:, j] * padded[:, j:j + x.shape[1]] for j in range(taps)))
    unit = lambda t: t / torch.sqrt((t * t).sum(-1, keepdim=True) + 1e-6)  # noqa: E731
    q, k, v = layer._heads(x)
    group = layer.value_heads // layer.key_heads
    q, k = (unit(t).repeat_interleave(group, dim=2) for t in (q, k))
    decay = torch.exp(-torch.exp(p["log_a"]) * torch.nn.functional.softplus(delta + p["step_bias"], threshold=100.0))
    state, rows = torch.zeros((h.shape[0], layer.value_heads, layer.key_dim, layer.value_dim), dtype=torch.float64), []
    for t in range(h.shape[1]):
        state = decay[:, t, :, None, None] * state
        u = torch.sigmoid(beta[:, t, :, None]) * (v[:, t] - (state * k[:, t, ..., None]).sum(2))
        state = state + k[:, t, ..., None] * u[:, :, None]
        rows.append(layer.key_dim ** -0.5 * (state * q[:, t, ..., None]).sum(2))
    y = torch.stack(rows, dim=1)
    y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * p["norm_w"]
    return (y.flatten(-2) * torch.nn.functional.silu(z)) @ p["out"].T


def test_gradients_of_the_layer():
    torch.manual_seed(3)
    layer = runpy.run_path(EXAMPLE)["Layer"](width=24)
    h, dy = torch.randn((2, 70, 24), device="cuda"), torch.randn((2, 70, 24), device="cuda")
    (layer(h) * dy).sum().backward()
    got = {n: t.grad.cpu().double() for n, t in layer.named_parameters()}
    p = {n: t.detach().cpu().double().requires_grad_() for n, t in layer.named_parameters()}
    loss = lambda q: (_in_64_bits(layer, q, h.cpu().double()) * dy.cpu().double()).sum()  # noqa: E731
    loss(p).backward()
    # In norm: a gradient passes up to eight operators there and back, each of whose results is off by less than some 300 roundings of the size of what made it (sums
    # of 140 rows, 128 columns and 32 entries of a head), and the norms divide by lengths that are not far from one: 16 * 300 * 2^-24 = 3e-4.
    for n, t in p.items():
        assert float((got[n] - t.grad).norm()) <= 3e-4 * float(t.grad.norm()), n
    # and along a direction in each parameter, from differences in 64 bits (whose own error is the third derivative's, e^2)
    e = 1e-5
    for n in p:
        v = torch.randn_like(p[n])
        with torch.no_grad():
            up, down = (loss({**p, n: p[n] + s * e * v}) for s in (1, -1))
        assert float((up - down) / (2 * e) - (got[n] * v).sum()) == pytest.approx(0.0, abs=3e-4 * float(p[n].grad.norm() * v.norm())), n
