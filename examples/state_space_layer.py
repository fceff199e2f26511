#!/usr/bin/env python3
"""A state-space mixer layer from the library's operators: trained, run over prompts of unequal lengths, and continued token by token
(needs an MI355X and a built libsysconv.so).

    python -m paper_2010_15884_amd.build && python examples/state_space_layer.py

The layer projects its input to a signal x and a gate z, runs x through a short causal convolution with SiLU, scans it with step sizes and
B, C that are projected from it, gates it with z, normalises every token over groups of channels, and projects back.  The projections are torch's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2010_15884_amd import binding as sysconv  # noqa: E402


class CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias):
        ctx.save_for_backward(x, w, bias)
        return sysconv.sys_causal_conv1d(x, w, bias, activation="SILU")

    @staticmethod
    def backward(ctx, dy):
        return sysconv.sys_causal_conv1d_backward(dy.contiguous(), *ctx.saved_tensors, activation="SILU")[:3]


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, *inputs):                     # u, delta, A, B, C, D, z, delta_bias
        ctx.save_for_backward(*inputs)
        return sysconv.sys_selective_scan(*inputs, softplus=True)

    @staticmethod
    def backward(ctx, dy):
        return tuple(sysconv.sys_selective_scan_backward(dy.contiguous(), *ctx.saved_tensors, softplus=True)[:8])


class TokenNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, groups, w, b):             # x: [tokens, 1, channels]
        mean, rstd = (torch.empty((x.shape[0], groups), device=x.device) for _ in range(2))
        y = sysconv.sys_group_norm(x, groups, w, b, d_mean=mean, d_rstd=rstd)
        ctx.save_for_backward(x, w, b, mean, rstd)
        ctx.groups = groups
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, b, mean, rstd = ctx.saved_tensors
        dx, dw, db = sysconv.sys_group_norm_backward(dy.contiguous(), x, ctx.groups, mean, rstd, w, b)
        return dx, None, dw, db


class Layer(torch.nn.Module):
    def __init__(self, width, channels, states=16, taps=4, groups=4, rank=8):
        super().__init__()
        make = lambda *s: torch.nn.Parameter(torch.randn(s, device="cuda") * s[-1] ** -0.5)  # noqa: E731
        self.states, self.groups, self.rank, self.channels = states, groups, rank, channels
        self.into, self.out = make(2 * channels, width), make(width, channels)
        self.select, self.step = make(rank + 2 * states, channels), make(channels, rank)
        self.w, self.bias = make(channels, taps), torch.nn.Parameter(torch.zeros(channels, device="cuda"))
        self.log_a = torch.nn.Parameter(torch.log(torch.arange(1.0, states + 1, device="cuda")).repeat(channels, 1))
        self.skip = torch.nn.Parameter(torch.ones(channels, device="cuda"))
        self.step_bias = torch.nn.Parameter(torch.linspace(-6.0, -2.0, channels, device="cuda"))
        self.norm_w, self.norm_b = torch.nn.Parameter(torch.ones(channels, device="cuda")), torch.nn.Parameter(torch.zeros(channels, device="cuda"))

    def _selected(self, x):
        """Step sizes, B and C of the convolved signal; B and C stay columns of one projection."""
        s = x @ self.select.t()
        b, c = (t.unflatten(-1, (1, self.states)) for t in s[..., self.rank:].split(self.states, dim=-1))
        return s[..., :self.rank] @ self.step.t(), -torch.exp(self.log_a), b, c

    def forward(self, v):
        x, z = (v @ self.into.t()).split(self.channels, dim=-1)              # two halves of one tensor: strided rows
        x = CausalConv.apply(x, self.w, self.bias)
        delta, a, b, c = self._selected(x)
        y = Scan.apply(x, delta, a, b, c, self.skip, z, self.step_bias)
        return TokenNorm.apply(y.reshape(-1, 1, self.channels), self.groups, self.norm_w, self.norm_b).view(y.shape) @ self.out.t()

    @torch.no_grad()
    def prompt(self, v, lengths):
        """Outputs of a padded batch of prompts, and the states behind each of them."""
        x, z = (v @ self.into.t()).split(self.channels, dim=-1)
        rows = torch.empty((v.shape[0], self.w.shape[1] - 1, self.channels), device="cuda")
        x = sysconv.sys_causal_conv1d(x, self.w, self.bias, activation="SILU", d_state_out=rows, d_lengths=lengths)
        delta, a, b, c = self._selected(x)
        h = torch.empty((v.shape[0], self.channels, self.states), device="cuda")
        y = sysconv.sys_selective_scan(x, delta, a, b, c, self.skip, z, self.step_bias, softplus=True, d_state_out=h, d_lengths=lengths)
        y = sysconv.sys_group_norm(y.view(-1, 1, self.channels), self.groups, self.norm_w, self.norm_b).view(y.shape)
        return y @ self.out.t(), rows, h

    @torch.no_grad()
    def token(self, v, rows, h, slots):
        """One token for each of the requests whose states lie at `slots` of the two caches, which are updated in place."""
        x, z = (v @ self.into.t()).split(self.channels, dim=-1)
        x = sysconv.sys_causal_conv1d_update(x, self.w, self.bias, rows, activation="SILU", d_slots=slots)
        delta, a, b, c = self._selected(x)
        y = sysconv.sys_selective_scan_update(x, delta, a, b, c, h, self.skip, z, self.step_bias, softplus=True, d_slots=slots)
        y = sysconv.sys_group_norm(y.view(-1, 1, self.channels), self.groups, self.norm_w, self.norm_b).view(y.shape)
        return y @ self.out.t()


def main():
    torch.manual_seed(0)
    layer = Layer(width=32, channels=64)

    # training: the signal two steps ago, smoothed
    optimizer = torch.optim.Adam(layer.parameters(), lr=1e-2)
    losses = []
    for _ in range(60):
        v = torch.randn((8, 96, 32), device="cuda")
        target = torch.zeros_like(v)
        target[:, 2:] = v[:, :-2]
        loss = (layer(v) - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    print(f"training: loss {losses[0]:.3f} -> {losses[-1]:.3f}")

    # serving: prompts of unequal lengths in one call, their states into caches, then token by token
    lengths = [40, 7, 1, 23]
    v = torch.randn((4, 50, 32), device="cuda")
    with torch.no_grad():
        whole = layer(v)
    y, rows, h = layer.prompt(v[:, :40], torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    slots = torch.tensor([3, 0, 5, 2], dtype=torch.int32, device="cuda")
    row_cache, state_cache = torch.zeros((6, *rows.shape[1:]), device="cuda"), torch.zeros((6, *h.shape[1:]), device="cuda")
    row_cache[slots.long()], state_cache[slots.long()] = rows, h
    worst = max(float((y[b, :n] - whole[b, :n]).abs().max()) for b, n in enumerate(lengths))
    for step in range(10):
        at = torch.tensor([n + step for n in lengths], device="cuda")
        got = layer.token(v[torch.arange(4, device="cuda"), at], row_cache, state_cache, slots)
        worst = max(worst, float((got - whole[torch.arange(4, device="cuda"), at]).abs().max()))
    print(f"serving: prompts and 10 tokens each, largest difference from the whole sequences {worst:.1e}")
    assert losses[-1] < 0.5 * losses[0] and worst < 1e-4
    print("all good")


if __name__ == "__main__":
    main()
