#!/usr/bin/env python3
"""A gated delta rule layer from the library's operators: trained, run over prompts of unequal lengths, and continued token by token
(needs an MI355X and a built libsysconv.so).

    python -m paper_2010_15884_amd.build && python examples/delta_rule_layer.py

The layer projects its input to queries, keys and values, which go through a short causal convolution with SiLU, to a gate z and to the step sizes
and strengths of the heads.  Queries and keys are brought to length one, the gated delta rule writes the values under the keys and reads them
with the queries, every head's result is normalised and gated with z, and all of it is projected back.  The projections and the gate are torch's.
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


class UnitHeads(torch.autograd.Function):
    """Queries and keys of length one."""
    @staticmethod
    def forward(ctx, q, k):
        ctx.save_for_backward(q, k)
        return sysconv.sys_head_norm(q, k, norm="L2")

    @staticmethod
    def backward(ctx, dyq, dyk):
        q, k = ctx.saved_tensors
        return sysconv.sys_head_norm_backward(dyq.contiguous(), dyk.contiguous(), q, k, norm="L2")[:2]


class HeadNorm(torch.autograd.Function):
    """One tensor of heads, by the root of each head's mean square, and a weight."""
    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return sysconv.sys_head_norm(x, d_wq=w)[0]

    @staticmethod
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        dx, _, dw, _ = sysconv.sys_head_norm_backward(dy.contiguous(), None, x, d_wq=w)
        return dx, dw


class DeltaRule(torch.autograd.Function):
    @staticmethod
    def forward(ctx, *inputs):                     # q, k, v, delta, A, beta, delta_bias
        ctx.save_for_backward(*inputs)
        return sysconv.sys_gated_delta_rule(*inputs, softplus=True, sigmoid=True)

    @staticmethod
    def backward(ctx, dy):
        return tuple(sysconv.sys_gated_delta_rule_backward(dy.contiguous(), *ctx.saved_tensors, softplus=True, sigmoid=True)[:7])


class Layer(torch.nn.Module):
    def __init__(self, width, key_heads=2, value_heads=4, key_dim=32, value_dim=32, taps=4):
        super().__init__()
        make = lambda *s: torch.nn.Parameter(torch.randn(s, device="cuda") * s[-1] ** -0.5)  # noqa: E731
        self.key_heads, self.value_heads, self.key_dim, self.value_dim = key_heads, value_heads, key_dim, value_dim
        values = value_heads * value_dim
        self.sizes = [2 * key_heads * key_dim + values, values, value_heads, value_heads]
        self.into, self.out = make(sum(self.sizes), width), make(width, values)
        self.w, self.bias = make(self.sizes[0], taps), torch.nn.Parameter(torch.zeros(self.sizes[0], device="cuda"))
        self.log_a = torch.nn.Parameter(torch.log(torch.linspace(1.0, 8.0, value_heads, device="cuda")))
        self.step_bias = torch.nn.Parameter(torch.linspace(-5.0, -2.0, value_heads, device="cuda"))
        self.norm_w = torch.nn.Parameter(torch.ones(value_dim, device="cuda"))

    def _heads(self, x):
        """Queries, keys and values, columns of the convolved rows."""
        keys, dim = self.key_heads * self.key_dim, (self.key_heads, self.key_dim)
        return x[..., :keys].unflatten(-1, dim), x[..., keys:2 * keys].unflatten(-1, dim), x[..., 2 * keys:].unflatten(-1, (self.value_heads, self.value_dim))

    def _gated(self, y, z):
        return (y.flatten(-2) * torch.nn.functional.silu(z)) @ self.out.t()

    def forward(self, h):
        x, z, delta, beta = (h @ self.into.t()).split(self.sizes, dim=-1)     # columns of one tensor: strided rows
        q, k, v = self._heads(CausalConv.apply(x, self.w, self.bias))
        q, k = UnitHeads.apply(q, k)
        y = DeltaRule.apply(q, k, v, delta, -torch.exp(self.log_a), beta, self.step_bias)
        return self._gated(HeadNorm.apply(y, self.norm_w), z)

    @torch.no_grad()
    def prompt(self, h, lengths):
        """Outputs of a padded batch of prompts, and the states behind each of them."""
        x, z, delta, beta = (h @ self.into.t()).split(self.sizes, dim=-1)
        rows = torch.empty((h.shape[0], self.w.shape[1] - 1, self.sizes[0]), device="cuda")
        x = sysconv.sys_causal_conv1d(x, self.w, self.bias, activation="SILU", d_state_out=rows, d_lengths=lengths)
        q, k, v = self._heads(x)
        q, k = sysconv.sys_head_norm(q, k, norm="L2", d_lengths=lengths)
        state = torch.empty((h.shape[0], self.value_heads, self.key_dim, self.value_dim), device="cuda")
        y = sysconv.sys_gated_delta_rule(q, k, v, delta, -torch.exp(self.log_a), beta, self.step_bias, softplus=True, sigmoid=True, d_state_out=state,
                                         d_lengths=lengths)
        return self._gated(sysconv.sys_head_norm(y, d_wq=self.norm_w, d_lengths=lengths)[0], z), rows, state

    @torch.no_grad()
    def token(self, h, rows, state, slots):
        """One token for each of the requests whose states lie at `slots` of the two caches, which are updated in place."""
        x, z, delta, beta = (h @ self.into.t()).split(self.sizes, dim=-1)
        x = sysconv.sys_causal_conv1d_update(x, self.w, self.bias, rows, activation="SILU", d_slots=slots)
        q, k, v = self._heads(x)
        q, k = sysconv.sys_head_norm(q[:, None], k[:, None], norm="L2")       # (a request is a sequence of one)
        y = sysconv.sys_gated_delta_rule_update(q[:, 0], k[:, 0], v, delta, -torch.exp(self.log_a), beta, state, self.step_bias, softplus=True,
                                                sigmoid=True, d_slots=slots)
        return self._gated(sysconv.sys_head_norm(y[:, None], d_wq=self.norm_w)[0][:, 0], z)


def main():
    torch.manual_seed(0)
    layer = Layer(width=32)

    # training: the signal two steps ago
    optimizer = torch.optim.Adam(layer.parameters(), lr=1e-2)
    losses = []
    for _ in range(60):
        h = torch.randn((8, 96, 32), device="cuda")
        target = torch.zeros_like(h)
        target[:, 2:] = h[:, :-2]
        loss = (layer(h) - target).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    print(f"training: loss {losses[0]:.3f} -> {losses[-1]:.3f}")

    # serving: prompts of unequal lengths in one call, their states into caches, then token by token
    lengths = [100, 7, 1, 64]
    h = torch.randn((4, 110, 32), device="cuda")
    with torch.no_grad():
        whole = layer(h)
    y, rows, state = layer.prompt(h[:, :100], torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    slots = torch.tensor([3, 0, 5, 2], dtype=torch.int32, device="cuda")
    row_cache, state_cache = torch.zeros((6, *rows.shape[1:]), device="cuda"), torch.zeros((6, *state.shape[1:]), device="cuda")
    row_cache[slots.long()], state_cache[slots.long()] = rows, state
    worst = max(float((y[b, :n] - whole[b, :n]).abs().max()) for b, n in enumerate(lengths))
    for step in range(10):
        at = torch.tensor([n + step for n in lengths], device="cuda")
        got = layer.token(h[torch.arange(4, device="cuda"), at], row_cache, state_cache, slots)
        worst = max(worst, float((got - whole[torch.arange(4, device="cuda"), at]).abs().max()))
    print(f"serving: prompts and 10 tokens each, largest difference from the whole sequences {worst:.1e}")
    assert worst < 1e-4
    print("all good")


if __name__ == "__main__":
    main()
