"""The operators on channels-last sequences written out in 64 bits, a position at a time, and how far a 32-bit computation may be off.

Every function takes tensors on any device, widens them and returns a dict.  With ``bound=True`` each product and sum is taken of
absolute values (decays stay as they are): the result bounds what passes through the sums, and errors are measured against it.

Tolerances.  u = 2^-24 is the unit of a 32-bit rounding; the exponential, reciprocal, logarithm and square root instructions are off by at most
2u, their arguments by u.
  sigmoid(x): e^-x is off by (|x| + 3) u relative (argument 2 roundings), the sum and the reciprocal add 3u: (|x| + 6) u.
  softplus(x): max(x, 0) + log(1 + e): e is off by (|x| + 3) u of itself and e |x| <= 0.37, the logarithm and the sums add 4u: at
  most 8u of the result.
  causal convolution: width + 1 multiply-adds: (width + 2) u of the bound; SiLU adds (|pre| + 8) u and multiplies by at most 1.1.
  scan: s = softplus is off by 8u (+ 1 for the bias), so e^(sA) by (12 |sA| + 4) u; a state is a sum of products of at most L of them:
  a term is off by L (12 |sA| + 6) u, which is also what a gradient through the recurrence from the other end costs.  A product of a state and
  a gradient of one has both.
  sums over m values: at most m u, and in the kernels' tree order far less; m is bounded by 64 per level here.
  group norm: see test_gpu_group_norm.
A result is rounded when it is stored, by at most half a unit of the last place: 2^-8 of it in bf16 (8 significant bits), 2^-11 in fp16 (11; plus
2^-25 where it is subnormal), u in fp32.
"""
import torch

U = 2.0 ** -24
ROUNDING = {torch.float32: (U, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 0.0)}


def wide(t):
    return None if t is None else t.detach().double().cpu()


def sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def act(x, kind, bound=False):
    if kind == "SILU":
        return x.abs() * sigmoid(x) if bound else x * sigmoid(x)
    return torch.clamp_min(x, 0.0) if kind == "RELU" else x


def act_grad(x, kind, bound=False):
    if kind == "SILU":
        s = sigmoid(x)
        return s * (1.0 + (x.abs() if bound else x) * (1.0 - s))
    return (x > 0).double() if kind == "RELU" else torch.ones_like(x)


def causal_conv(x, w, bias=None, activation="NONE", state=None, lengths=None, dy=None, dstate_out=None, bound=False):
    """y, state and, with dy, dx, dw, dbias, dstate."""
    x, w, bias, state, dy, dstate_out = map(wide, (x, w, bias, state, dy, dstate_out))
    batch, length, channels = x.shape
    k = w.shape[1]
    a = torch.abs if bound else (lambda t: t)
    out = {"y": torch.zeros(x.shape, dtype=torch.float64), "state": torch.zeros((batch, k - 1, channels), dtype=torch.float64),
           "dx": torch.zeros(x.shape, dtype=torch.float64), "dw": torch.zeros(w.shape, dtype=torch.float64),
           "dbias": torch.zeros(channels, dtype=torch.float64), "dstate": torch.zeros((batch, k - 1, channels), dtype=torch.float64)}
    for b in range(batch):
        n = length if lengths is None else min(max(int(lengths[b]), 0), length)
        rows = torch.cat([torch.zeros((k - 1, channels), dtype=torch.float64) if state is None else state[b], x[b, :n]])
        drows = torch.zeros_like(rows)
        if dstate_out is not None:
            drows[n:] += a(dstate_out[b])
        for t in range(n):
            pre = (rows[t:t + k].t() * w).sum(dim=1) + (0.0 if bias is None else bias)
            most = (rows[t:t + k].t() * w).abs().sum(dim=1) + (0.0 if bias is None else bias.abs())
            out["y"][b, t] = (1.1 * most if activation == "SILU" else most) if bound else act(pre, activation)
            if dy is not None:
                # in the bound: what an error of pre does to the derivative, whose own derivative is at most 0.5
                slope = act_grad(pre, activation, bound) + (0.5 * most if bound and activation == "SILU" else 0.0)
                dpre = a(dy[b, t]) * slope
                drows[t:t + k] += (a(w) * dpre[:, None]).t()
                out["dw"] += a(rows[t:t + k]).t() * dpre[:, None]
                out["dbias"] += dpre
        out["state"][b] = rows[n:]
        out["dx"][b, :n] = drows[k - 1:]
        out["dstate"][b] = drows[:k - 1]
    return out


def scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=True, state=None, lengths=None, dy=None, dstate_out=None, bound=False):
    """y, state and, with dy, du, ddelta, dA, dB, dC, dD, dz, ddelta_bias, dstate; "sA": the largest |s A|."""
    u, delta, A, B, C, D, z, delta_bias, state, dy, dstate_out = map(wide, (u, delta, A, B, C, D, z, delta_bias, state, dy, dstate_out))
    batch, length, d = u.shape
    g, n = B.shape[2], A.shape[1]
    a = torch.abs if bound else (lambda t: t)
    of = torch.arange(d) // (d // g)
    full = lambda *shape: torch.zeros(shape, dtype=torch.float64)  # noqa: E731
    out = {"y": full(batch, length, d), "state": full(batch, d, n), "du": full(batch, length, d), "ddelta": full(batch, length, d),
           "dz": full(batch, length, d), "dA": full(d, n), "dB": full(batch, length, g, n), "dC": full(batch, length, g, n), "dD": full(d),
           "ddelta_bias": full(d), "dstate": full(batch, d, n), "sA": 0.0}
    for b in range(batch):
        m = length if lengths is None else min(max(int(lengths[b]), 0), length)
        h = full(d, n) if state is None else a(state[b])
        hs, parts = [h], []
        for t in range(m):
            pre = delta[b, t] + (0.0 if delta_bias is None else delta_bias)
            s = torch.logaddexp(pre, torch.zeros_like(pre)) if softplus else pre
            decay = torch.exp(s[:, None] * A)
            out["sA"] = max(out["sA"], float((s[:, None] * A).abs().max()))
            sa = a(s)
            h = decay * h + (sa * a(u[b, t]))[:, None] * a(B[b, t, of])
            yr = (h * a(C[b, t, of])).sum(dim=1) + (0.0 if D is None else a(D) * a(u[b, t]))
            gate = torch.ones(d, dtype=torch.float64) if z is None else act(z[b, t], "SILU", bound)
            out["y"][b, t] = yr * gate
            hs.append(h)
            parts.append((pre, s, sa, decay, yr, gate))
        out["state"][b] = h
        if dy is None:
            continue
        carry = full(d, n) if dstate_out is None else a(dstate_out[b])
        for t in range(m - 1, -1, -1):
            pre, s, sa, decay, yr, gate = parts[t]
            bt, ct, ut = a(B[b, t, of]), a(C[b, t, of]), a(u[b, t])
            if z is not None:
                out["dz"][b, t] = a(dy[b, t]) * yr * act_grad(z[b, t], "SILU", bound)
            e = a(dy[b, t]) * gate
            gt = carry + e[:, None] * ct
            q = gt * decay * hs[t]
            gb = (gt * bt).sum(dim=1)
            ds = ut * gb + (q * a(A)).sum(dim=1)
            out["du"][b, t] = sa * gb + (0.0 if D is None else a(D) * e)
            out["ddelta"][b, t] = ds * (sigmoid(pre) if softplus else 1.0)
            out["dA"] += q * sa[:, None]
            out["dB"][b, t] = (gt * (sa * ut)[:, None]).view(g, d // g, n).sum(dim=1)
            out["dC"][b, t] = (hs[t + 1] * e[:, None]).view(g, d // g, n).sum(dim=1)
            out["dD"] += e * ut
            out["ddelta_bias"] += out["ddelta"][b, t]
            carry = gt * decay
        out["dstate"][b] = carry
    return out


def group_norm(x, groups, w=None, b=None, eps=1e-5, activation="NONE", dy=None, mean=None, rstd=None):
    """y, mean, rstd and, with dy (and the statistics to use), dx, dw, db."""
    x, w, b, dy, mean, rstd = map(wide, (x, w, b, dy, mean, rstd))
    batch, rows, c = x.shape
    per = c // groups
    xg = x.view(batch, rows, groups, per)
    w = torch.ones(c, dtype=torch.float64) if w is None else w
    b = torch.zeros(c, dtype=torch.float64) if b is None else b
    if mean is None:
        mean = xg.mean(dim=(1, 3))
        rstd = 1.0 / torch.sqrt(((xg - mean[:, None, :, None]) ** 2).mean(dim=(1, 3)) + eps)
    hat = ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(x.shape)
    pre = hat * w + b
    out = {"y": act(pre, activation), "mean": mean, "rstd": rstd, "hat": hat, "pre": pre}
    if dy is not None:
        f = dy * act_grad(pre, activation)
        fw = (f * w).view(xg.shape)
        m1, m2 = fw.mean(dim=(1, 3), keepdim=True), (fw * hat.view(xg.shape)).mean(dim=(1, 3), keepdim=True)
        out["dx"] = (rstd[:, None, :, None] * (fw - m1 - hat.view(xg.shape) * m2)).reshape(x.shape)
        out["dw"], out["db"] = (f * hat).sum(dim=(0, 1)), f.sum(dim=(0, 1))
        out["f"], out["fw"] = f, fw
    return out


def check(got, want, allowed, what):
    """|got - want| <= allowed + the rounding of got's type, element by element; NaN and infinities at the same places."""
    got_w, (relative, absolute) = wide(got), ROUNDING[got.dtype]
    assert got_w.shape == want.shape, (what, got_w.shape, want.shape)
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got_w), finite), f"{what}: NaN or infinity at other places"
    off = (got_w - want).abs()[finite]
    room = (allowed.expand_as(want)[finite] if isinstance(allowed, torch.Tensor) else allowed) * (1 + relative) + relative * want.abs()[finite] + absolute
    if off.numel():
        worst = (off - room).argmax()
        assert (off <= room).all(), f"{what}: off by {off[worst]:.3e}, allowed {room[worst]:.3e}, value {want[finite][worst]:.3e}"
