"""The operators of a state-space mixer layer, as cases that can be timed and checked.

Three operators on [batch, length, channels] tensors, each in the forms a program needs of it: the short causal
convolution (prompt, gradient, single token), the selective scan (prompt, gradient, single token), and the group norm
with an activation (forward, gradient).  A pass is one call of the public Python entry points (``own``), or the same in
elementary torch operations in 32 bits (the plain forms).

Values are what such a layer meets: activations about normal, step sizes between 0.001 and 0.1 before the data moves
them, decays -1 .. -N as they are usually initialised.  Prompts of unequal lengths are padded on the right.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def _conv(name, batch, length, channels, width, dtype, act="SILU", bias=True, state=False, ragged=False, sliced=False, grad=False):
    c = {"op": "conv_grad" if grad else "conv", "batch": batch, "length": length, "channels": channels, "width": width,
         "dtype": dtype, "act": act, "bias": bias, "state": state, "ragged": ragged, "sliced": sliced}
    return dict(c, name=name) if name else c


def _conv_step(name, requests, slots, channels, width, dtype, act="SILU", bias=True):
    c = {"op": "conv_step", "requests": requests, "slots": slots, "channels": channels, "width": width, "dtype": dtype,
         "act": act, "bias": bias}
    return dict(c, name=name) if name else c


def _scan(name, batch, length, channels, states, dtype, groups=1, gate=True, state=False, ragged=False, grad=False):
    c = {"op": "scan_grad" if grad else "scan", "batch": batch, "length": length, "channels": channels, "states": states,
         "groups": groups, "dtype": dtype, "gate": gate, "state": state, "ragged": ragged}
    return dict(c, name=name) if name else c


def _scan_step(name, requests, slots, channels, states, dtype, groups=1, gate=True):
    c = {"op": "scan_step", "requests": requests, "slots": slots, "channels": channels, "states": states,
         "groups": groups, "dtype": dtype, "gate": gate}
    return dict(c, name=name) if name else c


def _norm(name, batch, rows, channels, groups, dtype, act="SILU", affine=True, grad=False):
    c = {"op": "norm_grad" if grad else "norm", "batch": batch, "rows": rows, "channels": channels, "groups": groups,
         "dtype": dtype, "act": act, "affine": affine}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the convolution of two long prompts; x is one half of a wider projection, so its rows are strided
        _conv("conv_prompt_bf16", 2, 4096, 4096, 4, "bf16", sliced=True),
        # continued prompts of unequal lengths (one of them empty), an odd number of channels, three taps
        _conv("conv_ragged_f16", 5, 1021, 1001, 3, "f16", state=True, ragged=True),
        # a training step of the convolution: gradients of input, taps and bias
        _conv("conv_train_bf16", 4, 2048, 4096, 4, "bf16", grad=True),
        # one token for a few requests out of a cache of states: launch and host time
        _conv_step("conv_step_bf16", 8, 12, 2048, 4, "bf16"),
        # the scan of one long prompt
        _scan("scan_prompt_bf16", 1, 4096, 4096, 16, "bf16"),
        # continued prompts of unequal lengths, channels that fill no block, four groups of B and C
        _scan("scan_ragged_f16", 7, 517, 1000, 16, "f16", groups=4, state=True, ragged=True),
        # a training step of the scan
        _scan("scan_train_bf16", 4, 2048, 2048, 16, "bf16", grad=True),
        # a small training step in full precision, odd sizes, no gate
        _scan("scan_train_f32", 2, 333, 510, 9, "f32", groups=2, gate=False, grad=True),
        # one token for a full batch of requests: the states are read and written once
        _scan_step("scan_step_bf16", 64, 80, 4096, 16, "bf16"),
        # feature maps of 64 x 64 in a convolutional network
        _norm("norm_image_bf16", 16, 4096, 512, 32, "bf16"),
        # one row a token, a group a head: the norm behind the scan
        _norm("norm_tokens_bf16", 8192, 1, 4096, 64, "bf16", act="NONE"),
        # a training step of the norm, ten channels a group
        _norm("norm_train_f16", 8, 4096, 320, 32, "f16", grad=True),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    op = rng.choice(["conv", "conv_grad", "conv_step", "scan", "scan", "scan_grad", "scan_step", "norm", "norm", "norm_grad"])
    if op in ("conv", "conv_grad"):
        channels, most = _log_uniform(rng, 8, 8192), 32 << 20
        if rng.random() < 0.6:
            channels = (channels + 7) // 8 * 8
        batch = _log_uniform(rng, 1, 16)
        length = _log_uniform(rng, 1, max(1, min(8192, most // (batch * channels))))
        return _conv(None, batch, length, channels, rng.choice([2, 3, 4, 4, 4, 5, 8]), dtype, rng.choice(["SILU", "SILU", "NONE"]),
                     rng.random() < 0.7, rng.random() < 0.4, rng.random() < 0.4, rng.random() < 0.5, op == "conv_grad")
    if op == "conv_step":
        requests = _log_uniform(rng, 1, 256)
        return _conv_step(None, requests, requests + rng.randint(0, 32), _log_uniform(rng, 8, 8192), rng.choice([2, 3, 4, 4, 5]), dtype)
    if op in ("scan", "scan_grad", "scan_step"):
        states = rng.choice([1, 4, 8, 16, 16, 16, 16, 32, 64, rng.randint(1, 64)])
        groups = rng.choice([1, 1, 1, 2, 3])
        channels = groups * _log_uniform(rng, 8, 4096 // groups)
        if op == "scan_step":
            requests = _log_uniform(rng, 1, 128)
            channels = min(channels, groups * max(1, (64 * 4096 * 16) // (requests * states * groups)))
            return _scan_step(None, requests, requests + rng.randint(0, 16), channels, states, dtype, groups, rng.random() < 0.7)
        batch = _log_uniform(rng, 1, 16)
        channels = min(channels, groups * max(1, (1 << 28) // (batch * states * groups)))
        length = _log_uniform(rng, 1, max(1, min(8192, (1 << 28) // (batch * channels * states))))
        return _scan(None, batch, length, channels, states, dtype, groups, rng.random() < 0.7, rng.random() < 0.4,
                     rng.random() < 0.4, op == "scan_grad")
    groups = rng.choice([1, 4, 8, 16, 32, 32, 64])
    # eight values a group or more: the gradient of a group of one or two is zero but for rounding
    tokens = rng.random() < 0.35
    channels = groups * _log_uniform(rng, 8 if tokens else 1, 4096 // groups)
    rows = 1 if tokens else _log_uniform(rng, 8, 16384)
    rows = min(rows, (32 << 20) // channels)
    batch = _log_uniform(rng, 1, max(1, min(16384 if tokens else 32, (32 << 20) // (rows * channels))))
    return _norm(None, batch, rows, channels, groups, dtype, rng.choice(["SILU", "SILU", "RELU", "NONE"]), rng.random() < 0.8,
                 op == "norm_grad")


def _lengths(case):
    """Unequal lengths, the first whole and the last empty: a property of the case, so that its work can be stated."""
    full = case["length"]
    if not case["ragged"]:
        return [full] * case["batch"]
    r = random.Random(case["batch"] * 1000003 + full)
    got = [r.randint(0, full) for _ in range(case["batch"])]
    got[0] = full
    if case["batch"] > 1:
        got[-1] = 0
    return got


class _Values:
    """Seeded values on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed))

    def normal(self, shape, scale=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=self.gen, device="cuda").mul_(scale).to(dtype)

    def uniform(self, shape, low, high):
        return torch.rand(shape, generator=self.gen, device="cuda").mul_(high - low).add_(low)


def prepare(case, seed):
    v, dtype, op = _Values(seed), DTYPES[case["dtype"]], case["op"]
    s = {"case": case}
    if op in ("conv", "conv_grad", "conv_step"):
        k, c = case["width"], case["channels"]
        s["w"] = v.normal((c, k), k ** -0.5, dtype)
        s["bias"] = v.normal((c,), 0.2, dtype) if case["bias"] else None
        if op == "conv_step":
            _slots(s, case, seed)
            s["x"] = v.normal((case["requests"], c), 1.0, dtype)
            s["state"] = v.normal((case["slots"], k - 1, c), 1.0, dtype)
            s["state_out"] = torch.zeros_like(s["state"])
            return s
        b, n = case["batch"], case["length"]
        s["x"] = v.normal((b, n, 2 * c if case["sliced"] else c), 1.0, dtype)[..., :c]
        s["state"] = v.normal((b, k - 1, c), 1.0, dtype) if case["state"] else None
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        if op == "conv_grad":
            s["dy"] = v.normal((b, n, c), 1.0, dtype)
            s["dstate_out"] = v.normal((b, k - 1, c), 1.0, dtype) if case["state"] else None
        else:
            s["state_out"] = torch.empty((b, k - 1, c), dtype=dtype, device="cuda")
        return s
    if op in ("scan", "scan_grad", "scan_step"):
        d, n, g = case["channels"], case["states"], case["groups"]
        lead = (case["requests"],) if op == "scan_step" else (case["batch"], case["length"])
        # B and C are columns of one projection, behind the columns that the step sizes are made from
        rank = (d + 15) // 16
        bc = v.normal(lead + (rank + 2 * g * n,), 1.0, dtype)
        s["B"] = bc[..., rank:rank + g * n].unflatten(-1, (g, n))
        s["C"] = bc[..., rank + g * n:].unflatten(-1, (g, n))
        s["u"] = v.normal(lead + (d,), 0.7, dtype)
        s["delta"] = v.normal(lead + (d,), 0.5, dtype)
        # the gate is the second half of a wider projection
        s["z"] = v.normal(lead + (2 * d,), 1.0, dtype)[..., d:] if case["gate"] else None
        s["A"] = -torch.arange(1, n + 1, dtype=torch.float32, device="cuda") * v.uniform((d, n), 0.8, 1.2)
        s["D"] = v.uniform((d,), 0.5, 1.5)
        dt = torch.exp(v.uniform((d,), math.log(0.001), math.log(0.1)))
        s["delta_bias"] = dt + torch.log(-torch.expm1(-dt))
        if op == "scan_step":
            _slots(s, case, seed)
            s["state"] = v.normal((case["slots"], d, n), 0.5)
            s["state_out"] = torch.zeros_like(s["state"])
            return s
        s["state"] = v.normal((case["batch"], d, n), 0.5) if case["state"] else None
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        if op == "scan_grad":
            s["dy"] = v.normal(lead + (d,), 1.0, dtype)
            s["dstate_out"] = v.normal((case["batch"], d, n), 1.0) if case["state"] else None
        else:
            s["state_out"] = torch.empty((case["batch"], d, n), dtype=torch.float32, device="cuda")
        return s
    b, r, c, g = case["batch"], case["rows"], case["channels"], case["groups"]
    # channels have means and sizes of their own
    x = v.normal((b, r, c)).mul_(v.uniform((c,), 0.5, 2.0)).add_(v.normal((c,), 0.5))
    s["x"] = x.to(dtype)
    s["w"] = v.uniform((c,), 0.5, 1.5).to(dtype) if case["affine"] else None
    s["b"] = v.normal((c,), 0.3, dtype) if case["affine"] else None
    if op == "norm_grad":
        # the statistics that the forward pass left
        xf = s["x"].float().view(b, r, g, c // g)
        s["mean"] = xf.mean(dim=(1, 3))
        s["rstd"] = torch.rsqrt((xf - s["mean"][:, None, :, None]).square().mean(dim=(1, 3)) + EPS)
        s["dy"] = v.normal((b, r, c), 1.0, dtype)
    else:
        s["mean"], s["rstd"] = (torch.empty((b, g), dtype=torch.float32, device="cuda") for _ in range(2))
    return s


def _slots(s, case, seed):
    order = list(range(case["slots"]))
    random.Random(int(seed)).shuffle(order)
    s["slots"] = torch.tensor(order[:case["requests"]], dtype=torch.int32, device="cuda")


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    from paper_2010_15884_amd import binding
    case, op = s["case"], s["case"]["op"]
    if op == "conv":
        y = binding.sys_causal_conv1d(s["x"], s["w"], s["bias"], activation=case["act"], d_state=s["state"],
                                      d_state_out=s["state_out"], d_lengths=s["lengths"])
        return {"y": y, "state": s["state_out"]}
    if op == "conv_grad":
        dx, dw, db, ds = binding.sys_causal_conv1d_backward(s["dy"], s["x"], s["w"], s["bias"], activation=case["act"],
                                                            d_state=s["state"], d_dstate_out=s["dstate_out"],
                                                            d_lengths=s["lengths"])
        return {"dx": dx, "dw": dw, "db": db, "ds": ds}
    if op == "conv_step":
        y = binding.sys_causal_conv1d_update(s["x"], s["w"], s["bias"], s["state"], activation=case["act"],
                                             d_slots=s["slots"], d_state_out=s["state_out"])
        return {"y": y, "state": s["state_out"]}
    if op == "scan":
        y = binding.sys_selective_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"], s["delta_bias"],
                                       softplus=True, d_state=s["state"], d_state_out=s["state_out"], d_lengths=s["lengths"])
        return {"y": y, "state": s["state_out"]}
    if op == "scan_grad":
        g = binding.sys_selective_scan_backward(s["dy"], s["u"], s["delta"], s["A"], s["B"], s["C"], s["D"], s["z"],
                                                s["delta_bias"], softplus=True, d_state=s["state"],
                                                d_dstate_out=s["dstate_out"], d_lengths=s["lengths"])
        return {"du": g.du, "ddelta": g.ddelta, "dA": g.dA, "dB": g.dB, "dC": g.dC, "dD": g.dD, "dz": g.dz,
                "ddelta_bias": g.ddelta_bias, "ds": g.dstate}
    if op == "scan_step":
        y = binding.sys_selective_scan_update(s["u"], s["delta"], s["A"], s["B"], s["C"], s["state"], s["D"], s["z"],
                                              s["delta_bias"], softplus=True, d_slots=s["slots"], d_state_out=s["state_out"])
        return {"y": y, "state": s["state_out"]}
    if op == "norm":
        y = binding.sys_group_norm(s["x"], case["groups"], s["w"], s["b"], eps=EPS, activation=case["act"],
                                   d_mean=s["mean"], d_rstd=s["rstd"])
        return {"y": y, "mean": s["mean"], "rstd": s["rstd"]}
    dx, dw, db = binding.sys_group_norm_backward(s["dy"], s["x"], case["groups"], s["mean"], s["rstd"], s["w"], s["b"],
                                                 activation=case["act"])
    return {"dx": dx, "dw": dw, "db": db}


# ---------------------------------------------------------------- the same in elementary operations, 32 bits

def _run_plain(s):
    return {"conv": _plain_conv, "conv_grad": _plain_conv_grad, "conv_step": _plain_conv_step, "scan": _plain_scan,
            "scan_grad": _plain_scan_grad, "scan_step": _plain_scan_step, "norm": _plain_norm,
            "norm_grad": _plain_norm_grad}[s["case"]["op"]](s)


def _activate(pre, act):
    if act == "SILU":
        return pre * torch.sigmoid(pre)
    return torch.clamp_min(pre, 0.0) if act == "RELU" else pre


def _activate_grad(pre, act):
    if act == "SILU":
        sig = torch.sigmoid(pre)
        return sig * (1.0 + pre * (1.0 - sig))
    return (pre > 0).to(pre.dtype) if act == "RELU" else torch.ones_like(pre)


def _inside(s):
    """True where a position lies within its sequence, [batch, length, 1]; None where all do."""
    if s["lengths"] is None:
        return None
    return (torch.arange(s["case"]["length"], device="cuda")[None, :] < s["lengths"][:, None])[..., None]


def _keep(x, inside):
    return x if inside is None else torch.where(inside, x, torch.zeros((), dtype=x.dtype, device=x.device))


def _rows(s):
    """state ++ x in 32 bits, [batch, width - 1 + length, channels], zero behind the sequences' ends."""
    case, x = s["case"], _keep(s["x"].float(), _inside(s))
    head = torch.zeros((x.shape[0], case["width"] - 1, x.shape[2]), device="cuda") if s["state"] is None else s["state"].float()
    return torch.cat([head, x], dim=1)


def _last_rows(s, rows):
    k1 = s["case"]["width"] - 1
    if s["lengths"] is None:
        return rows[:, rows.shape[1] - k1:]
    at = s["lengths"].long()[:, None] + torch.arange(k1, device="cuda")[None, :]
    return torch.gather(rows, 1, at[..., None].expand(-1, -1, rows.shape[2]))


def _pre(s, rows):
    k, n, w = s["case"]["width"], s["case"]["length"], s["w"].float()
    pre = rows[:, :n] * w[:, 0]
    for j in range(1, k):
        pre = pre + rows[:, j:j + n] * w[:, j]
    return pre if s["bias"] is None else pre + s["bias"].float()


def _plain_conv(s):
    rows = _rows(s)
    y = _keep(_activate(_pre(s, rows), s["case"]["act"]), _inside(s))
    return {"y": y.to(s["x"].dtype), "state": _last_rows(s, rows).to(s["x"].dtype)}


def _plain_conv_grad(s):
    case, dtype = s["case"], s["x"].dtype
    k, n, w = case["width"], case["length"], s["w"].float()
    rows = _rows(s)
    dpre = _keep(s["dy"].float(), _inside(s)) * _activate_grad(_pre(s, rows), case["act"])
    drows = torch.zeros_like(rows)
    dw = torch.empty_like(w)
    for j in range(k):
        drows[:, j:j + n] += dpre * w[:, j]
        dw[:, j] = (dpre * rows[:, j:j + n]).sum(dim=(0, 1))
    if s["dstate_out"] is not None:
        if s["lengths"] is None:
            drows[:, n:] += s["dstate_out"].float()
        else:
            at = s["lengths"].long()[:, None] + torch.arange(k - 1, device="cuda")[None, :]
            drows.scatter_add_(1, at[..., None].expand(-1, -1, drows.shape[2]), s["dstate_out"].float())
    return {"dx": drows[:, k - 1:].to(dtype), "dw": dw.to(s["w"].dtype),
            "db": None if s["bias"] is None else dpre.sum(dim=(0, 1)).to(dtype),
            "ds": None if s["state"] is None else drows[:, :k - 1].to(dtype)}


def _plain_conv_step(s):
    case, at = s["case"], s["slots"].long()
    rows = torch.cat([s["state"][at].float(), s["x"].float()[:, None]], dim=1)
    pre = (rows * s["w"].float().t()[None]).sum(dim=1)
    if s["bias"] is not None:
        pre = pre + s["bias"].float()
    s["state_out"][at] = rows[:, 1:].to(s["state"].dtype)
    return {"y": _activate(pre, case["act"]).to(s["x"].dtype), "state": s["state_out"]}


def _softplus(x):
    return torch.clamp_min(x, 0.0) + torch.log1p(torch.exp(-x.abs()))


def _per_channel(m, channels):
    """[..., groups, states] -> [..., channels, states]."""
    return m.float().repeat_interleave(channels // m.shape[-2], dim=-2)


def _recur(a, x, h):
    """h_t = a_t h_{t-1} + x_t along dim 1 by doubling within blocks of 128 steps."""
    got = []
    for at in range(0, a.shape[1], 128):
        ab, xb = a[:, at:at + 128], x[:, at:at + 128]
        k = 1
        while k < ab.shape[1]:
            xb = torch.cat([xb[:, :k], xb[:, k:] + ab[:, k:] * xb[:, :-k]], dim=1)
            ab = torch.cat([ab[:, :k], ab[:, k:] * ab[:, :-k]], dim=1)
            k *= 2
        hb = xb + ab * h[:, None]
        h = hb[:, -1]
        got.append(hb)
    return torch.cat(got, dim=1)


def _scan_parts(s):
    d, inside = s["case"]["channels"], _inside(s)
    u = _keep(s["u"].float(), inside)
    pre = _keep(s["delta"].float(), inside) + s["delta_bias"]
    dt = _keep(_softplus(pre), inside)
    b, c = (_keep(m, None if inside is None else inside[..., None]) for m in (_per_channel(s["B"], d), _per_channel(s["C"], d)))
    a = torch.exp(dt[..., None] * s["A"])
    h0 = torch.zeros((u.shape[0], d, s["case"]["states"]), device="cuda") if s["state"] is None else s["state"]
    return inside, u, pre, dt, b, c, a, h0, _recur(a, (dt * u)[..., None] * b, h0)


def _plain_scan(s):
    inside, u, _, _, _, c, _, _, h = _scan_parts(s)
    y = (h * c).sum(dim=-1) + s["D"] * u
    if s["z"] is not None:
        y = y * _activate(_keep(s["z"].float(), inside), "SILU")
    return {"y": y.to(s["u"].dtype), "state": h[:, -1].clone()}


def _plain_scan_grad(s):
    case, dtype = s["case"], s["u"].dtype
    g = case["groups"]
    inside, u, pre, dt, b, c, a, h0, h = _scan_parts(s)
    dy = _keep(s["dy"].float(), inside)
    dz = None
    if s["z"] is not None:
        z = _keep(s["z"].float(), inside)
        dz = (dy * ((h * c).sum(dim=-1) + s["D"] * u) * _activate_grad(z, "SILU")).to(dtype)
        dy = dy * _activate(z, "SILU")
    tail = torch.zeros_like(h0) if s["dstate_out"] is None else s["dstate_out"]
    # gh_t = c_t dy_t + a_{t+1} gh_{t+1}: the same recurrence from the end
    x = dy[..., None] * c
    x[:, -1] += tail
    later = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], dim=1)
    gh = _recur(later.flip(1), x.flip(1), torch.zeros_like(h0)).flip(1)
    before = torch.cat([h0[:, None], h[:, :-1]], dim=1)
    q = gh * a * before
    gb = (gh * b).sum(dim=-1)
    ddt = (q * s["A"]).sum(dim=-1) + gb * u
    ddelta = ddt * torch.sigmoid(pre)
    split = lambda m: m.unflatten(2, (g, case["channels"] // g)).sum(dim=3)  # noqa: E731
    return {"du": _keep(gb * dt + dy * s["D"], inside).to(dtype), "ddelta": _keep(ddelta, inside).to(dtype),
            "dA": (q * dt[..., None]).sum(dim=(0, 1)), "dB": split(gh * (dt * u)[..., None]).to(dtype),
            "dC": split(h * dy[..., None]).to(dtype), "dD": (dy * u).sum(dim=(0, 1)), "dz": dz,
            "ddelta_bias": _keep(ddelta, inside).sum(dim=(0, 1)), "ds": None if s["state"] is None else a[:, 0] * gh[:, 0]}


def _plain_scan_step(s):
    d, at = s["case"]["channels"], s["slots"].long()
    u, dt = s["u"].float(), _softplus(s["delta"].float() + s["delta_bias"])
    h = torch.exp(dt[..., None] * s["A"]) * s["state"][at] + (dt * u)[..., None] * _per_channel(s["B"], d)
    y = (h * _per_channel(s["C"], d)).sum(dim=-1) + s["D"] * u
    if s["z"] is not None:
        y = y * _activate(s["z"].float(), "SILU")
    s["state_out"][at] = h
    return {"y": y.to(s["u"].dtype), "state": s["state_out"]}


def _norm_parts(s):
    case = s["case"]
    b, r, c, g = case["batch"], case["rows"], case["channels"], case["groups"]
    x = s["x"].float().view(b, r, g, c // g)
    w = torch.ones(c, device="cuda") if s["w"] is None else s["w"].float()
    bias = torch.zeros(c, device="cuda") if s["b"] is None else s["b"].float()
    return x, w.view(g, c // g), bias.view(g, c // g)


def _plain_norm(s):
    x, w, b = _norm_parts(s)
    mean = x.mean(dim=(1, 3), keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(dim=(1, 3), keepdim=True) + EPS)
    y = _activate((x - mean) * rstd * w + b, s["case"]["act"])
    return {"y": y.view(s["x"].shape).to(s["x"].dtype), "mean": mean[:, 0, :, 0], "rstd": rstd[:, 0, :, 0]}


def _plain_norm_grad(s):
    x, w, b = _norm_parts(s)
    rstd = s["rstd"][:, None, :, None]
    hat = (x - s["mean"][:, None, :, None]) * rstd
    dpre = s["dy"].float().view(x.shape) * _activate_grad(hat * w + b, s["case"]["act"])
    dhat = dpre * w
    dx = rstd * (dhat - dhat.mean(dim=(1, 3), keepdim=True) - hat * (dhat * hat).mean(dim=(1, 3), keepdim=True))
    affine = s["w"] is not None
    return {"dx": dx.view(s["x"].shape).to(s["x"].dtype), "dw": (dpre * hat).sum(dim=(0, 1)).flatten().to(s["w"].dtype) if affine else None,
            "db": dpre.sum(dim=(0, 1)).flatten().to(s["b"].dtype) if affine else None}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op, e = case["op"], BYTES[case["dtype"]]
    if op in ("conv", "conv_grad"):
        k, c = case["width"], case["channels"]
        rows, full = sum(_lengths(case)), case["batch"] * case["length"]
        states = case["batch"] * (k - 1) * c * e
        taps = c * (k + (1 if case["bias"] else 0)) * e
        if op == "conv":
            return {"bytes": (rows + full) * c * e + taps + states * (2 if case["state"] else 1), "flops": 2 * k * rows * c}
        return {"bytes": (2 * rows + full) * c * e + 2 * taps + (3 * states if case["state"] else 0), "flops": 6 * k * rows * c}
    if op == "conv_step":
        k, c, n = case["width"], case["channels"], case["requests"]
        return {"bytes": n * c * e * (2 + 2 * (k - 1)) + c * (k + 1) * e, "flops": 2 * k * n * c}
    if op in ("scan", "scan_grad", "scan_step"):
        d, n, bc = case["channels"], case["states"], 2 * case["groups"] * case["states"]
        params, gate = d * (n + 2) * 4, 1 if case["gate"] else 0
        if op == "scan_step":
            r = case["requests"]
            return {"bytes": r * (d * (3 + gate) + bc) * e + 2 * r * d * n * 4 + params, "flops": 7 * r * d * n}
        rows, full = sum(_lengths(case)), case["batch"] * case["length"]
        states = case["batch"] * d * n * 4
        if op == "scan":
            return {"bytes": rows * (d * (2 + gate) + bc) * e + full * d * e + params + states * (2 if case["state"] else 1),
                    "flops": 7 * rows * d * n}
        return {"bytes": rows * (d * (3 + gate) + bc) * e + full * (d * (2 + gate) + bc) * e + 2 * params
                + (3 * states if case["state"] else 0), "flops": 20 * rows * d * n}
    values, c = case["batch"] * case["rows"] * case["channels"], case["channels"]
    stats, affine = 8 * case["batch"] * case["groups"], 2 * c * e if case["affine"] else 0
    if op == "norm":
        return {"bytes": 2 * values * e + stats + affine, "flops": 8 * values}
    return {"bytes": 3 * values * e + stats + 2 * affine, "flops": 16 * values}


# ---------------------------------------------------------------- the definitions in 64 bits, a position at a time

def exact(case, seed):
    s = prepare(case, seed)
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    return {"conv": _exact_conv, "conv_grad": _exact_conv, "conv_step": _exact_conv_step, "scan": _exact_scan,
            "scan_grad": _exact_scan, "scan_step": _exact_scan_step, "norm": _exact_norm, "norm_grad": _exact_norm}[case["op"]](case, s)


def _d_act(pre, act):
    if act == "SILU":
        e = torch.exp(-pre)
        return 1.0 / (1.0 + e) + pre * e / (1.0 + e) ** 2
    return torch.where(pre > 0, 1.0, 0.0).double() if act == "RELU" else torch.ones_like(pre)


def _act(pre, act):
    return pre / (1.0 + torch.exp(-pre)) if act == "SILU" else torch.relu(pre) if act == "RELU" else pre


def _exact_conv(case, s):
    k, c, n = case["width"], case["channels"], case["length"]
    grad = case["op"] == "conv_grad"
    y = torch.zeros((case["batch"], n, c), dtype=torch.float64, device="cuda")
    dw, db = torch.zeros_like(s["w"]), torch.zeros(c, dtype=torch.float64, device="cuda")
    states = []
    for i, m in enumerate(_lengths(case)):
        head = s["state"][i] if s["state"] is not None else torch.zeros((k - 1, c), dtype=torch.float64, device="cuda")
        ext = torch.cat([head, s["x"][i, :m]])
        pre = torch.zeros((m, c), dtype=torch.float64, device="cuda") if s["bias"] is None else s["bias"].expand(m, c).clone()
        for j in range(k):
            pre.addcmul_(ext[j:j + m], s["w"][:, j].expand(m, c))
        if not grad:
            y[i, :m] = _act(pre, case["act"])
            states.append(ext[m:])
            continue
        dpre = s["dy"][i, :m] * _d_act(pre, case["act"])
        dext = torch.zeros_like(ext)
        if s["dstate_out"] is not None:
            dext[m:] += s["dstate_out"][i]
        for j in range(k):
            dext[j:j + m].addcmul_(dpre, s["w"][:, j].expand(m, c))
            dw[:, j] += (dpre * ext[j:j + m]).sum(dim=0)
        db += dpre.sum(dim=0)
        y[i, :m] = dext[k - 1:]
        states.append(dext[:k - 1])
    if not grad:
        return {"y": y, "state": torch.stack(states)}
    return {"dx": y, "dw": dw, "db": db if case["bias"] else None, "ds": torch.stack(states) if case["state"] else None}


def _exact_conv_step(case, s):
    y = torch.zeros_like(s["x"])
    out = s["state_out"]
    for i, slot in enumerate(s["slots"].tolist()):
        rows = torch.cat([s["state"][slot], s["x"][i:i + 1]])
        pre = (rows.t() * s["w"]).sum(dim=1)
        y[i] = _act(pre if s["bias"] is None else pre + s["bias"], case["act"])
        out[slot] = rows[1:]
    return {"y": y, "state": out}


def _step_size(pre):
    return torch.logaddexp(pre, torch.zeros_like(pre))


def _exact_scan(case, s):
    b, n, d, g = case["batch"], case["length"], case["channels"], case["groups"]
    grad = case["op"] == "scan_grad"
    full = dict(dtype=torch.float64, device="cuda")
    h = torch.zeros((b, d, case["states"]), **full) if s["state"] is None else s["state"].clone()
    lens = torch.tensor(_lengths(case), device="cuda")
    of = torch.arange(d, device="cuda") // (d // g)
    y, kept = torch.zeros((b, n, d), **full), []
    for t in range(n):
        on = (t < lens)[:, None]
        dt = _step_size(s["delta"][:, t] + s["delta_bias"])
        new = torch.exp(dt[..., None] * s["A"]) * h + (dt * s["u"][:, t])[..., None] * s["B"][:, t, of]
        if grad:
            kept.append(h)
        h = torch.where(on[..., None], new, h)
        y[:, t] = torch.where(on, (h * s["C"][:, t, of]).sum(dim=-1) + s["D"] * s["u"][:, t], 0.0)
    if not grad:
        return {"y": y if s["z"] is None else y * _act(s["z"], "SILU"), "state": h}
    out = {k: torch.zeros((b, n, d), **full) for k in ("du", "ddelta", "dz")}
    out["dB"], out["dC"] = (torch.zeros((b, n, g, case["states"]), **full) for _ in range(2))
    dA, dD, dbias = torch.zeros_like(s["A"]), torch.zeros(d, **full), torch.zeros(d, **full)
    gh = torch.zeros_like(h) if s["dstate_out"] is None else s["dstate_out"].clone()
    for t in range(n - 1, -1, -1):
        on = (t < lens)[:, None]
        u, pre, bt, ct, before = s["u"][:, t], s["delta"][:, t] + s["delta_bias"], s["B"][:, t, of], s["C"][:, t, of], kept.pop()
        dt = _step_size(pre)
        a = torch.exp(dt[..., None] * s["A"])
        dy = torch.where(on, s["dy"][:, t], 0.0)
        if s["z"] is not None:
            out["dz"][:, t] = dy * y[:, t] * _d_act(s["z"][:, t], "SILU")
            dy = dy * _act(s["z"][:, t], "SILU")
        now = a * before + (dt * u)[..., None] * bt
        gt = torch.where(on[..., None], gh + dy[..., None] * ct, 0.0)
        ga = gt * a * before
        d_dt = (ga * s["A"]).sum(dim=-1) + u * (gt * bt).sum(dim=-1)
        out["du"][:, t] = dt * (gt * bt).sum(dim=-1) + s["D"] * dy
        out["ddelta"][:, t] = d_dt / (1.0 + torch.exp(-pre))
        dA += (ga * dt[..., None]).sum(dim=0)
        dD += (dy * u).sum(dim=0)
        dbias += out["ddelta"][:, t].sum(dim=0)
        out["dB"][:, t] = (gt * (dt * u)[..., None]).view(b, g, d // g, -1).sum(dim=2)
        out["dC"][:, t] = (now * dy[..., None]).view(b, g, d // g, -1).sum(dim=2)
        gh = torch.where(on[..., None], gt * a, gh)
    return {"du": out["du"], "ddelta": out["ddelta"], "dA": dA, "dB": out["dB"], "dC": out["dC"], "dD": dD,
            "dz": out["dz"] if case["gate"] else None, "ddelta_bias": dbias, "ds": gh if case["state"] else None}


def _exact_scan_step(case, s):
    d, out, y = case["channels"], s["state_out"], torch.zeros_like(s["u"])
    of = torch.arange(d, device="cuda") // (d // case["groups"])
    for i, slot in enumerate(s["slots"].tolist()):
        dt = _step_size(s["delta"][i] + s["delta_bias"])
        h = torch.exp(dt[:, None] * s["A"]) * s["state"][slot] + (dt * s["u"][i])[:, None] * s["B"][i, of]
        y[i] = (h * s["C"][i, of]).sum(dim=1) + s["D"] * s["u"][i]
        if case["gate"]:
            y[i] *= _act(s["z"][i], "SILU")
        out[slot] = h
    return {"y": y, "state": out}


def _exact_norm(case, s):
    b, c, g = case["batch"], case["channels"], case["groups"]
    per = c // g
    rows = s["x"].view(b, case["rows"], g, per).transpose(1, 2).reshape(b, g, -1)          # a group's values in one line
    w = (s["w"] if case["affine"] else torch.ones(c, dtype=torch.float64, device="cuda")).view(g, 1, per)
    bias = (s["b"] if case["affine"] else torch.zeros(c, dtype=torch.float64, device="cuda")).view(g, 1, per)
    back = lambda m: m.reshape(b, g, case["rows"], per).transpose(1, 2).reshape(s["x"].shape)  # noqa: E731
    if case["op"] == "norm":
        mean = rows.mean(dim=2)
        rstd = 1.0 / torch.sqrt(rows.var(dim=2, unbiased=False) + EPS)
        hat = ((rows - mean[..., None]) * rstd[..., None]).view(b, g, -1, per)
        return {"y": back(_act(hat * w + bias, case["act"])), "mean": mean, "rstd": rstd}
    hat = ((rows - s["mean"][..., None]) * s["rstd"][..., None]).view(b, g, -1, per)
    dy = s["dy"].view(b, case["rows"], g, per).transpose(1, 2)
    dpre = dy * _d_act(hat * w + bias, case["act"])
    dhat = dpre * w
    m1, m2 = dhat.mean(dim=(2, 3), keepdim=True), (dhat * hat).mean(dim=(2, 3), keepdim=True)
    dx = back((dhat - m1 - hat * m2) * s["rstd"][..., None, None])
    return {"dx": dx, "dw": (dpre * hat).sum(dim=(0, 2)).reshape(-1) if case["affine"] else None,
            "db": dpre.sum(dim=(0, 2)).reshape(-1) if case["affine"] else None}
