"""The gated delta rule and the norm of queries and keys written out in 64 bits, a position at a time, and how far a 32-bit computation may be off.

Tolerances of the rule.  u = 2^-24.  With keys of length one at most and strengths in [0, 1] a position multiplies each column of the state by a (I - b k k^T),
which makes no vector longer, so what a position gets wrong is added to what the others do and does not grow.  Let M[c] be the largest |S_t[., c]| + |v_t[c]|
of a head over its positions (2-norms), and N[c] the largest |dS_t[., c]| + scale |q_t| |dy_t[c]| of the gradients' recurrence, which has the same
factors.  A position at a time: S^T k is a sum of key_dim products, off by (key_dim + 2) u M at most, the factors b and a by 16 u and
(12 |s A| + 4) u (sequence_reference), the update by 3 u: (key_dim + 64) u M a position while |s A| <= 3.  In blocks of up to 64 positions a block instead does K S (key_dim
products), the inverse of I + A, whose entries are products of such factors and thus at most 1 in magnitude, by sums of at most 64 products twice over, its product with R
(64), and K^T U (64); the ratios of decays within a block are differences of sums in 64 bits, off by what the step sizes are off, 8u |G| e^-|G| <= 4u and
the exponential's own 2u: (key_dim + 4 * 64) u M a block.  ``steps`` counts positions or blocks, whichever computes; a gradient meets the
errors of both recurrences.  From there:
  y = scale S^T q: scale |q| M, and in 16-bit types products within a block are taken of numbers of 16 bits (2^-17 of each factor, 64 terms of at most scale |q| M).
  dv = b k^T dS: N.  dq = scale S dy: sum of M |dy| scale over the columns.  dk, dbeta, d(sA): sums over the columns of products of something at most M and something
  at most N (each the 2-norm over the key entries), of which there are at most four.  ddelta = A d(sA) sigmoid; dA, ddelta_bias: sums of them over the positions.
  In 16-bit types the products that make dq, dk, dbeta and d(sA) are taken of numbers of 16 bits as well: 4 * 2^-17 of the same bounds for each of at most
  six factors in a chain, 2^-12.
Tolerances of the norm: see head_norm.
"""
import torch

from sequence_reference import U, sigmoid, wide


def gated_delta(q, k, v, delta, A, beta, delta_bias=None, scale=None, softplus=True, sigmoid_beta=True, state=None, lengths=None, dy=None, dstate_out=None):
    """y, state and, with dy, dq, dk, dv, ddelta, dA, dbeta, ddelta_bias, dstate; and the sizes M, N [batch, heads, value_dim]."""
    q, k, v, delta, A, beta, delta_bias, state, dy, dstate_out = map(wide, (q, k, v, delta, A, beta, delta_bias, state, dy, dstate_out))
    batch, length, hk, dk = q.shape
    h, dv = v.shape[2:]
    of = torch.arange(h) // (h // hk)
    scale = dk ** -0.5 if scale is None else scale
    full = lambda *shape: torch.zeros(shape, dtype=torch.float64)  # noqa: E731
    out = {"y": full(batch, length, h, dv), "state": full(batch, h, dk, dv), "dq": full(*q.shape), "dk": full(*q.shape), "dv": full(*v.shape),
           "ddelta": full(*delta.shape), "dA": full(h), "dbeta": full(*beta.shape), "ddelta_bias": full(h), "dstate": full(batch, h, dk, dv),
           "M": full(batch, h, dv), "N": full(batch, h, dv), "sA": 0.0, "absA": full(h), "abs_bias": full(h)}
    for b in range(batch):
        n = length if lengths is None else min(max(int(lengths[b]), 0), length)
        s = full(h, dk, dv) if state is None else state[b]
        out["M"][b] = s.norm(dim=1)
        kept = []
        for t in range(n):
            pre = delta[b, t] + (0.0 if delta_bias is None else delta_bias)
            step = torch.logaddexp(pre, torch.zeros_like(pre)) if softplus else pre
            a = torch.exp(step * A)
            strength = sigmoid(beta[b, t]) if sigmoid_beta else beta[b, t]
            held = a[:, None, None] * s
            miss = v[b, t] - torch.einsum("hkv,hk->hv", held, k[b, t, of])
            u = strength[:, None] * miss
            kept.append((s, held, miss, u, pre, step, a, strength))
            s = held + k[b, t, of][:, :, None] * u[:, None]
            out["y"][b, t] = scale * torch.einsum("hkv,hk->hv", s, q[b, t, of])
            out["M"][b] = torch.maximum(out["M"][b], s.norm(dim=1) + v[b, t].abs())
            out["sA"] = max(out["sA"], float((step * A).abs().max()))
        out["state"][b] = s
        if dy is None:
            continue
        g = full(h, dk, dv) if dstate_out is None else dstate_out[b]
        out["N"][b] = g.norm(dim=1)
        news = [x[0] for x in kept[1:]] + [s]
        for t in range(n - 1, -1, -1):
            before, held, miss, u, pre, step, a, strength = kept[t]
            kt, qt = k[b, t, of], q[b, t, of]
            g = g + scale * qt[:, :, None] * dy[b, t][:, None]
            out["N"][b] = torch.maximum(out["N"][b], g.norm(dim=1) + scale * qt.norm(dim=1)[:, None] * dy[b, t].abs())
            du = torch.einsum("hkv,hk->hv", g, kt)
            dmiss = strength[:, None] * du
            dheld = g - kt[:, :, None] * dmiss[:, None]
            by_head = scale * torch.einsum("hkv,hv->hk", news[t], dy[b, t])
            out["dq"][b, t] = by_head.view(hk, h // hk, dk).sum(dim=1)
            by_head = torch.einsum("hkv,hv->hk", g, u) - torch.einsum("hkv,hv->hk", held, dmiss)
            out["dk"][b, t] = by_head.view(hk, h // hk, dk).sum(dim=1)
            out["dv"][b, t] = dmiss
            db = (du * miss).sum(dim=1)
            out["dbeta"][b, t] = db * strength * (1.0 - strength) if sigmoid_beta else db
            dlog = a * (dheld * before).sum(dim=(1, 2))
            ds = dlog * A * (sigmoid(pre) if softplus else 1.0)
            out["ddelta"][b, t] = ds
            out["dA"] += dlog * step
            out["ddelta_bias"] += ds
            out["absA"] += step.abs()
            out["abs_bias"] += A.abs()
            g = a[:, None, None] * dheld
        out["dstate"][b] = g
    return out


def delta_allowed(c, want, steps, dtype):
    """What each result may be off by before it is rounded."""
    q, dy, A = wide(c["q"]).clone(), wide(c.get("dy")), wide(c["A"])
    dy = None if dy is None else dy.clone()
    for b, n in enumerate([] if c["lengths"] is None else c["lengths"].tolist()):
        for t in (q, dy):                          # what lies behind a sequence is 0 there, exactly
            if t is not None:
                t[b, min(max(n, 0), t.shape[1]):] = 0.0
    hk, h, dk = q.shape[2], A.shape[0], q.shape[3]
    scale = dk ** -0.5 if c.get("scale") is None else abs(c["scale"])
    dv = want["M"].shape[2]
    narrow = 2.0 ** -12 if dtype != torch.float32 else 0.0
    one = steps * (dk + 256) * U
    two = 2 * one + (dv + 64) * U + narrow
    M, N = want["M"], want["N"]
    MN = 4 * (M * N).sum(dim=2)                                        # [batch, heads]
    per_key = lambda x: x.view(x.shape[0], hk, h // hk).sum(dim=2)     # noqa: E731
    size = scale * q.norm(dim=3).repeat_interleave(h // hk, dim=2)     # [batch, length, heads]
    allowed = {"state": one * M[:, :, None], "y": (one + 64 * 2 * (2.0 ** -17 if narrow else 0.0)) * size[..., None] * M[:, None]}
    if dy is not None:
        dq = scale * (M[:, None] * dy.abs()).sum(dim=3).flatten(0, 1)
        mn = lambda x: two * x                                         # noqa: E731
        allowed |= {"dv": (one + narrow) * N[:, None], "dstate": one * N[:, :, None],
                    "dq": mn(per_key(dq).view(*q.shape[:2], hk, 1)), "dk": mn(per_key(MN)[:, None, :, None]), "dbeta": mn(MN[:, None]),
                    "ddelta": mn(MN[:, None] * A.abs()), "dA": mn(MN.amax(dim=0) * want["absA"]), "ddelta_bias": mn(MN.amax(dim=0) * want["abs_bias"])}
    return allowed


def head_norm(x, w=None, cos=None, sin=None, positions=None, norm="RMS", eps=1e-6, interleaved=False, lengths=None, dy=None):
    """y and, with dy, dx and dw of one tensor [batch, length, heads, dim]; "room": what each may be off by, in 32-bit units of its parts' sizes.

    The mean is a sum of dim squares, off by (dim + 2) u, its root and quotient by half of that and 3u: r by (dim / 2 + 5) u.  y = x r w turned: each of two
    products by 4u more.  The gradient: n . dn is a sum of dim products with two factors r; dx = r (dn - n share (n . dn)): (2 dim + 16) u of its parts.
    dw: sums over tokens and heads of terms off by (dim / 2 + 10) u, m of them at most m u of their sizes on top."""
    x, w, cos, sin, dy = map(wide, (x, w, cos, sin, dy))
    batch, length, heads, dim = x.shape
    there = torch.ones((batch, length), dtype=torch.bool)
    rows = torch.arange(length)[None].expand(batch, length) if positions is None else positions.cpu().long()
    if lengths is not None:
        for b in range(batch):
            there[b, min(max(int(lengths[b]), 0), length):] = False
    half = 0 if cos is None else cos.shape[1]
    if half:
        there &= (rows >= 0) & (rows < cos.shape[0])
        rows = torch.where(there, rows, torch.zeros_like(rows))
        c, s = cos[rows][:, :, None], sin[rows][:, :, None]
    at = torch.arange(half)
    first, second = (2 * at, 2 * at + 1) if interleaved else (at, at + half)

    def turn(z, sign, most=False):
        z = z.clone()
        if half:
            p, r = z[..., first], z[..., second]
            if most:
                z[..., first], z[..., second] = p.abs() * c.abs() + r.abs() * s.abs(), r.abs() * c.abs() + p.abs() * s.abs()
            else:
                z[..., first], z[..., second] = p * c - sign * r * s, r * c + sign * p * s
        return z
    keep = there[:, :, None, None]
    x = torch.where(keep, x, torch.zeros_like(x))
    share = 1.0 / dim if norm == "RMS" else 1.0
    r = 1.0 / torch.sqrt((x * x).sum(dim=3, keepdim=True) * share + eps)
    n = x * r
    ww = torch.ones(dim, dtype=torch.float64) if w is None else w
    zero = lambda t: torch.where(keep, t, torch.zeros_like(t))         # noqa: E731
    out = {"y": zero(turn(n * ww, 1.0)), "room": {"y": (dim / 2 + 10) * U * zero(turn((n * ww).abs(), 1.0, True))}}
    if dy is not None:
        dz = zero(turn(torch.where(keep, dy, torch.zeros_like(dy)), -1.0))
        most = zero(turn(torch.where(keep, dy, torch.zeros_like(dy)).abs(), -1.0, True))
        dn = dz * ww
        out["dx"] = zero(r * (dn - n * share * (n * dn).sum(dim=3, keepdim=True)))
        out["dw"] = (dz * n).sum(dim=(0, 1, 2))
        parts = r * (most * ww.abs() + n.abs() * share * (n.abs() * most * ww.abs()).sum(dim=3, keepdim=True))
        out["room"]["dx"] = (2 * dim + 16) * U * zero(parts)
        out["room"]["dw"] = (dim / 2 + 10 + batch * length * heads) * U * (most * n.abs()).sum(dim=(0, 1, 2))
    return out
