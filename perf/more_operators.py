"""The operators of a gated delta rule layer, as cases that can be timed and checked.

Two operators on [batch, length, heads, dim] tensors, each in the forms a program needs of it: the gated delta rule (prompt, gradient,
single token), and the norm of queries and keys for each head with the rotation of their positions (forward, gradient; a single
token is a row of its own).  A pass is one call of the public Python entry points (``own``), or the same in elementary torch operations in 32
bits (the plain forms).

Values are what such layers meet: queries and keys that were convolved, activated and brought to length one; step sizes between 0.001 and
0.1 before the data moves them, decays 1 .. 16; q, k and v as columns of one projection, so that their rows are strided.  Prompts of unequal
lengths are padded on the right.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6
CHUNK = 64            # of the plain form


def _delta(name, batch, length, key_heads, heads, key_dim, value_dim, dtype, state=False, ragged=False, grad=False):
    c = {"op": "delta_grad" if grad else "delta", "batch": batch, "length": length, "key_heads": key_heads, "heads": heads,
         "key_dim": key_dim, "value_dim": value_dim, "dtype": dtype, "state": state, "ragged": ragged}
    return dict(c, name=name) if name else c


def _delta_step(name, requests, slots, key_heads, heads, key_dim, value_dim, dtype):
    c = {"op": "delta_step", "requests": requests, "slots": slots, "key_heads": key_heads, "heads": heads, "key_dim": key_dim,
         "value_dim": value_dim, "dtype": dtype}
    return dict(c, name=name) if name else c


def _norm(name, batch, length, q_heads, k_heads, dim, rotary, dtype, norm="RMS", interleaved=False, weights=True, ragged=False, grad=False):
    c = {"op": "norm_grad" if grad else "norm", "batch": batch, "length": length, "q_heads": q_heads, "k_heads": k_heads, "dim": dim,
         "rotary": rotary, "dtype": dtype, "norm": norm, "interleaved": interleaved, "weights": weights, "ragged": ragged}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one long prompt: 32 heads whose queries and keys are shared by two
        _delta("delta_prompt_bf16", 1, 4096, 16, 32, 128, 128, "bf16"),
        # a batch of continued prompts of unequal lengths (one of them empty), heads of 64
        _delta("delta_ragged_f16", 5, 1021, 8, 8, 64, 128, "f16", state=True, ragged=True),
        # a short prompt in full precision with odd sizes: key and value dimensions that fill no tile
        _delta("delta_odd_f32", 2, 333, 3, 6, 40, 72, "f32", state=True),
        # a training step
        _delta("delta_train_bf16", 4, 2048, 8, 16, 128, 128, "bf16", grad=True),
        # a small training step in full precision, odd sizes, unequal lengths, with states before and behind
        _delta("delta_train_f32", 3, 250, 2, 4, 64, 100, "f32", state=True, ragged=True, grad=True),
        # one token for a full batch of requests: the states are read and written once
        _delta_step("delta_step_bf16", 64, 80, 16, 32, 128, 128, "bf16"),
        # one token for a few requests: launch and host time
        _delta_step("delta_step_f32", 3, 8, 4, 4, 64, 64, "f32"),
        # queries and keys of two long prompts of an attention layer, eight heads of queries to one of keys
        _norm("norm_prompt_bf16", 2, 4096, 32, 4, 128, 128, "bf16"),
        # queries and keys of a delta rule layer brought to length one: no weights, no positions; unequal lengths
        _norm("norm_length_f16", 5, 1021, 12, 12, 96, 0, "f16", norm="L2", weights=False, ragged=True),
        # a training step: heads of 256, a quarter of each turned, neighbouring entries paired
        _norm("norm_train_bf16", 4, 2048, 16, 2, 256, 64, "bf16", interleaved=True, grad=True),
        # a training step in full precision with a dimension that fills no vector
        _norm("norm_train_f32", 2, 777, 6, 3, 50, 22, "f32", grad=True),
        # one token for a batch of requests, each at a position of its own
        _norm("norm_step_bf16", 32, 1, 32, 8, 128, 128, "bf16"),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    op = rng.choice(["delta", "delta", "delta_grad", "delta_grad", "delta_step", "norm", "norm", "norm_grad", "norm_grad"])
    if op.startswith("delta"):
        key_dim, value_dim = (rng.choice([32, 64, 64, 128, 128, 128, rng.randint(8, 128)]) for _ in range(2))
        value_dim = rng.choice([value_dim, value_dim, value_dim, 192, 256])
        shared = rng.choice([1, 1, 2, 2, 4])
        key_heads = _log_uniform(rng, 1, 32 // shared)
        heads = key_heads * shared
        if op == "delta_step":
            most = (64 * 32 * 128 * 128) // (heads * key_dim * value_dim)
            requests = _log_uniform(rng, 1, max(1, min(256, most)))
            return _delta_step(None, requests, requests + rng.randint(0, 16), key_heads, heads, key_dim, value_dim, dtype)
        # at most the positions x heads x state of the largest listed case, a half of it where elements are wider than 16 bits
        most = (1 << (30 if dtype == "f32" else 31)) // (heads * key_dim * value_dim)
        batch = _log_uniform(rng, 1, 16)
        length = _log_uniform(rng, 1, max(1, min(8192, most // batch)))
        return _delta(None, batch, length, key_heads, heads, key_dim, value_dim, dtype, rng.random() < 0.4, rng.random() < 0.4, op == "delta_grad")
    dim = rng.choice([64, 64, 128, 128, 128, 256, rng.randint(8, 256)])
    rotary = rng.choice([0, dim // 2 * 2, dim // 2 * 2, dim // 8 * 2])
    k_heads = _log_uniform(rng, 1, 16)
    q_heads = k_heads * rng.choice([1, 1, 2, 4, 8])
    batch = _log_uniform(rng, 1, 32)
    most = (36 << 20) // (dim * (q_heads + k_heads)) // (2 if dtype == "f32" else 1)
    length = _log_uniform(rng, 1, max(1, min(8192, most // batch)))
    return _norm(None, batch, length, q_heads, k_heads, dim, rotary, dtype, rng.choice(["RMS", "RMS", "L2"]), rng.random() < 0.4,
                 rng.random() < 0.7, rng.random() < 0.4, op == "norm_grad")


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
    if op in ("delta", "delta_grad", "delta_step"):
        hk, h, dk, dv = case["key_heads"], case["heads"], case["key_dim"], case["value_dim"]
        lead = (case["requests"],) if op == "delta_step" else (case["batch"], case["length"])
        row = v.normal(lead + (2 * hk * dk + h * dv,))
        qk = row[..., :2 * hk * dk].unflatten(-1, (2 * hk, dk))
        qk.copy_(qk * torch.sigmoid(qk))
        qk.mul_(torch.rsqrt(qk.square().sum(dim=-1, keepdim=True) + EPS))
        row = row.to(dtype)
        s["q"], s["k"] = (t.unflatten(-1, (hk, dk)) for t in row[..., :2 * hk * dk].split(hk * dk, dim=-1))
        s["v"] = row[..., 2 * hk * dk:].unflatten(-1, (h, dv))
        # step sizes and strengths are the two halves of another projection
        gates = v.normal(lead + (2 * h,), 0.7, dtype)
        s["delta"], s["beta"] = gates.split(h, dim=-1)
        s["A"] = -v.uniform((h,), 1.0, 16.0)
        dt = torch.exp(v.uniform((h,), math.log(0.001), math.log(0.1)))
        s["delta_bias"] = dt + torch.log(-torch.expm1(-dt))
        if op == "delta_step":
            order = list(range(case["slots"]))
            random.Random(int(seed)).shuffle(order)
            s["slots"] = torch.tensor(order[:case["requests"]], dtype=torch.int32, device="cuda")
            s["state"] = v.normal((case["slots"], h, dk, dv), 0.3)
            s["state_out"] = torch.zeros_like(s["state"])
            return s
        s["state"] = v.normal((case["batch"], h, dk, dv), 0.3) if case["state"] else None
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        if op == "delta_grad":
            s["dy"] = v.normal(lead + (h, dv), 1.0, dtype)
            s["dstate_out"] = v.normal((case["batch"], h, dk, dv), 0.3) if case["state"] else None
        else:
            s["state_out"] = torch.empty((case["batch"], h, dk, dv), dtype=torch.float32, device="cuda")
        return s
    b, n, hq, hk, d = case["batch"], case["length"], case["q_heads"], case["k_heads"], case["dim"]
    # queries, keys and values of one projection; its entries have sizes of their own
    row = v.normal((b, n, (hq + 2 * hk) * d)).mul_(v.uniform(((hq + 2 * hk) * d,), 0.3, 3.0)).to(dtype)
    s["q"], s["k"] = row[..., :hq * d].unflatten(-1, (hq, d)), row[..., hq * d:(hq + hk) * d].unflatten(-1, (hk, d))
    s["wq"], s["wk"] = (v.uniform((d,), 0.5, 1.5).to(dtype) if case["weights"] else None for _ in range(2))
    s["cos"] = s["sin"] = s["positions"] = None
    if case["rotary"]:
        # a program keeps one table for all its positions; each sequence begins where its cache ends
        half = case["rotary"] // 2
        turns = torch.arange(2 * n + 4096, dtype=torch.float64, device="cuda")[:, None]
        angle = turns * torch.pow(10000.0, -torch.arange(half, dtype=torch.float64, device="cuda") / half)
        s["cos"], s["sin"] = torch.cos(angle).float(), torch.sin(angle).float()
        begin = (v.uniform((b, 1), 0.0, 1.0) * (n + 4096)).to(torch.int32)
        s["positions"] = begin + torch.arange(n, dtype=torch.int32, device="cuda")
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    if op == "norm_grad":
        s["dyq"], s["dyk"] = v.normal((b, n, hq, d), 1.0, dtype), v.normal((b, n, hk, d), 1.0, dtype)
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---------------------------------------------------------------- the framework's calls

def _run_own(s):
    from paper_2010_15884_amd import binding
    case, op = s["case"], s["case"]["op"]
    if op == "delta":
        y = binding.sys_gated_delta_rule(s["q"], s["k"], s["v"], s["delta"], s["A"], s["beta"], s["delta_bias"], softplus=True,
                                         sigmoid=True, d_state=s["state"], d_state_out=s["state_out"], d_lengths=s["lengths"])
        return {"y": y, "state": s["state_out"]}
    if op == "delta_grad":
        g = binding.sys_gated_delta_rule_backward(s["dy"], s["q"], s["k"], s["v"], s["delta"], s["A"], s["beta"], s["delta_bias"],
                                                  softplus=True, sigmoid=True, d_state=s["state"], d_dstate_out=s["dstate_out"],
                                                  d_lengths=s["lengths"])
        return {"dq": g.dq, "dk": g.dk, "dv": g.dv, "ddelta": g.ddelta, "dA": g.dA, "dbeta": g.dbeta, "ddelta_bias": g.ddelta_bias,
                "ds": g.dstate}
    if op == "delta_step":
        y = binding.sys_gated_delta_rule_update(s["q"], s["k"], s["v"], s["delta"], s["A"], s["beta"], s["state"], s["delta_bias"],
                                                softplus=True, sigmoid=True, d_slots=s["slots"], d_state_out=s["state_out"])
        return {"y": y, "state": s["state_out"]}
    how = dict(norm=case["norm"], eps=EPS, interleaved=case["interleaved"], d_lengths=s["lengths"])
    if op == "norm":
        q, k = binding.sys_head_norm(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], **how)
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = binding.sys_head_norm_backward(s["dyq"], s["dyk"], s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"],
                                                      s["positions"], **how)
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


# ---------------------------------------------------------------- the same in elementary operations, 32 bits

def _run_plain(s):
    return {"delta": _plain_delta, "delta_grad": _plain_delta_grad, "delta_step": _plain_delta_step, "norm": _plain_norm,
            "norm_grad": _plain_norm_grad}[s["case"]["op"]](s)


def _inside(s, axes):
    """True where a position lies within its sequence, [batch, length, 1, ..]; None where all do."""
    if s["lengths"] is None:
        return None
    inside = torch.arange(s["case"]["length"], device="cuda")[None, :] < s["lengths"][:, None]
    return inside.view(inside.shape + (1,) * axes)


def _keep(x, inside):
    return x if inside is None else torch.where(inside, x, torch.zeros((), dtype=x.dtype, device=x.device))


def _softplus(x):
    return torch.clamp_min(x, 0.0) + torch.log1p(torch.exp(-x.abs()))


def _inverse(a):
    """(I + a)^-1 of strictly lower triangular matrices of CHUNK rows: blocks of 2, 4, .. rows from pairs of half their size."""
    at = torch.arange(CHUNK, device="cuda")
    x = torch.eye(CHUNK, device="cuda").expand_as(a)
    m = 1
    while m < CHUNK:
        block = at // m
        pair = (block[:, None] == block[None, :] + 1) & (block[:, None] % 2 == 1)
        x = x - x @ torch.where(pair, a, torch.zeros((), device="cuda")) @ x
        m *= 2
    return x


def _chunks(x):
    """[batch, length, heads, ..] -> [batch, heads, chunks, CHUNK, ..], zeros past the end."""
    short = -x.shape[1] % CHUNK
    if short:
        x = torch.cat([x, torch.zeros((x.shape[0], short) + x.shape[2:], dtype=x.dtype, device=x.device)], dim=1)
    return x.unflatten(1, (-1, CHUNK)).movedim(3, 1)


def _delta_forward(case, inside, q, k, v, delta, A, beta, bias, state):
    """The rule on chunks of 64 positions, inputs in 32 bits; sums of logarithms of decays in 64."""
    shared = case["heads"] // case["key_heads"]
    inside4 = None if inside is None else inside[..., None]
    q, k = (_chunks(_keep(t, inside4)).repeat_interleave(shared, dim=1) for t in (q, k))
    v = _chunks(_keep(v, inside4))
    g = _chunks(_keep(_softplus(_keep(delta, inside) + bias) * A, inside))
    b = _chunks(_keep(torch.sigmoid(_keep(beta, inside)), inside))[..., None]
    G = g.double().cumsum(dim=-1)
    lower = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device="cuda").tril()
    ratio = torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], float("-inf"))).float()
    whole, left = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]
    kt = k.transpose(-1, -2)
    x = _inverse((b * ratio * (k @ kt)).tril(-1))
    mixed = ratio * (q @ kt)
    u0, w = x @ (b * v), x @ (b * whole * k)
    qw, kl = q * whole, (k * left).transpose(-1, -2)
    h = torch.zeros((q.shape[0], case["heads"], case["key_dim"], case["value_dim"]), device="cuda") if state is None else state
    ys = []
    for i in range(q.shape[2]):
        u = u0[:, :, i] - w[:, :, i] @ h
        ys.append(qw[:, :, i] @ h + mixed[:, :, i] @ u)
        h = whole[:, :, i, -1:] * h + kl[:, :, i] @ u
    y = torch.stack(ys, dim=2).flatten(2, 3)[:, :, :case["length"]].transpose(1, 2)
    return _keep(y * case["key_dim"] ** -0.5, inside4), h


def _delta_inputs(s):
    return [s[n].float() for n in ("q", "k", "v", "delta", "A", "beta", "delta_bias")]


def _plain_delta(s):
    y, h = _delta_forward(s["case"], _inside(s, 1), *_delta_inputs(s), s["state"])
    return {"y": y.to(s["q"].dtype), "state": h.clone()}


def _plain_delta_grad(s):
    leaves = [t.detach().clone().requires_grad_() for t in _delta_inputs(s)]
    state = None if s["state"] is None else s["state"].clone().requires_grad_()
    y, h = _delta_forward(s["case"], _inside(s, 1), *leaves, state)
    outputs, seeds = [y], [s["dy"].float()]
    if state is not None:
        outputs, seeds, leaves = outputs + [h], seeds + [s["dstate_out"]], leaves + [state]
    got = torch.autograd.grad(outputs, leaves, seeds)
    dtype = s["q"].dtype
    return {"dq": got[0].to(dtype), "dk": got[1].to(dtype), "dv": got[2].to(dtype), "ddelta": got[3].to(dtype), "dA": got[4],
            "dbeta": got[5].to(dtype), "ddelta_bias": got[6], "ds": None if state is None else got[7]}


def _plain_delta_step(s):
    case, at = s["case"], s["slots"].long()
    q, k, v, delta, A, beta, bias = _delta_inputs(s)
    q, k = (t.repeat_interleave(case["heads"] // case["key_heads"], dim=1) for t in (q, k))
    h = torch.exp(_softplus(delta + bias) * A)[..., None, None] * s["state"][at]
    u = torch.sigmoid(beta)[..., None] * (v - (h * k[..., None]).sum(dim=2))
    h = h + k[..., None] * u[:, :, None]
    s["state_out"][at] = h
    y = (h * q[..., None]).sum(dim=2) * case["key_dim"] ** -0.5
    return {"y": y.to(s["q"].dtype), "state": s["state_out"]}


def _turn(case, x, cos, sin):
    """Pairs of the first `rotary` entries turned; cos, sin: [batch, length, 1, rotary / 2]."""
    n = case["rotary"]
    if not n:
        return x
    head, rest = x[..., :n], x[..., n:]
    a, b = (head[..., 0::2], head[..., 1::2]) if case["interleaved"] else (head[..., :n // 2], head[..., n // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    head = torch.stack([a, b], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([head, rest], dim=-1)


def _angles(s):
    if s["positions"] is None:
        return None, None
    at = s["positions"].long()
    return s["cos"][at][:, :, None], s["sin"][at][:, :, None]


def _inverse_size(case, x):
    square = x.square()
    return torch.rsqrt((square.mean(dim=-1, keepdim=True) if case["norm"] == "RMS" else square.sum(dim=-1, keepdim=True)) + EPS)


def _plain_norm(s):
    case, inside, (cos, sin) = s["case"], _inside(s, 2), _angles(s)

    def one(x, w):
        z = _keep(x.float(), inside)
        z = z * _inverse_size(case, z)
        return _turn(case, z if w is None else z * w.float(), cos, sin).to(x.dtype)
    return {"q": one(s["q"], s["wq"]), "k": one(s["k"], s["wk"])}


def _plain_norm_grad(s):
    case, inside, (cos, sin) = s["case"], _inside(s, 2), _angles(s)

    def one(dy, x, w):
        xf = _keep(x.float(), inside)
        r = _inverse_size(case, xf)
        n = xf * r
        dz = _turn(case, _keep(dy.float(), inside), cos, None if sin is None else -sin)
        dn = dz if w is None else dz * w.float()
        along = (dn * n).sum(dim=-1, keepdim=True) / (case["dim"] if case["norm"] == "RMS" else 1)
        return (r * (dn - n * along)).to(x.dtype), None if w is None else (dz * n).sum(dim=(0, 1, 2)).to(w.dtype)
    dq, dwq = one(s["dyq"], s["q"], s["wq"])
    dk, dwk = one(s["dyk"], s["k"], s["wk"])
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op, e = case["op"], BYTES[case["dtype"]]
    if op in ("delta", "delta_grad", "delta_step"):
        hk, h, dk, dv = case["key_heads"], case["heads"], case["key_dim"], case["value_dim"]
        row_in, params, one = (2 * hk * dk + h * dv + 2 * h) * e, 8 * h, h * dk * dv
        if op == "delta_step":
            r = case["requests"]
            return {"bytes": r * (row_in + h * dv * e + 8 * one) + params, "flops": 7 * r * one}
        rows, full = sum(_lengths(case)), case["batch"] * case["length"]
        states = case["batch"] * one * 4
        if op == "delta":
            return {"bytes": rows * row_in + full * h * dv * e + params + states * (2 if case["state"] else 1), "flops": 7 * rows * one}
        return {"bytes": rows * (row_in + h * dv * e) + full * row_in + 2 * params + (3 * states if case["state"] else 0),
                "flops": 20 * rows * one}
    rows, full = sum(_lengths(case)), case["batch"] * case["length"]
    values, turned = (case["q_heads"] + case["k_heads"]) * case["dim"], rows * (case["rotary"] * 4 + 4) if case["rotary"] else 0
    weights = 2 * case["dim"] * e if case["weights"] else 0
    if op == "norm":
        return {"bytes": (rows + full) * values * e + turned + weights, "flops": 8 * rows * values}
    return {"bytes": (2 * rows + full) * values * e + turned + 2 * weights, "flops": 16 * rows * values}


# ---------------------------------------------------------------- the definitions in 64 bits, a position at a time

def exact(case, seed):
    s = prepare(case, seed)
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    return {"delta": _exact_delta, "delta_grad": _exact_delta, "delta_step": _exact_delta_step, "norm": _exact_norm,
            "norm_grad": _exact_norm}[case["op"]](case, s)


def _exact_delta(case, s):
    b, n, hk, h, dk, dv = (case[k] for k in ("batch", "length", "key_heads", "heads", "key_dim", "value_dim"))
    full, of, scale = dict(dtype=torch.float64, device="cuda"), torch.arange(h, device="cuda") // (h // hk), 1.0 / math.sqrt(dk)
    lens = torch.tensor(_lengths(case), device="cuda")
    state = torch.zeros((b, h, dk, dv), **full) if s["state"] is None else s["state"].clone()
    grad = case["op"] == "delta_grad"
    y, kept = torch.zeros((b, n, h, dv), **full), []

    def at(t):
        on = (t < lens)[:, None]
        pre = torch.where(on, s["delta"][:, t] + s["delta_bias"], 0.0)
        dt = torch.logaddexp(pre, torch.zeros_like(pre))
        strength = 1.0 / (1.0 + torch.exp(-s["beta"][:, t]))
        return on, pre, dt, torch.exp(dt * s["A"]), strength, s["q"][:, t, of], s["k"][:, t, of], s["v"][:, t]

    for t in range(n):
        on, _, _, a, strength, q, k, v = at(t)
        kept.append(state if grad else None)
        held = a[..., None, None] * state
        u = strength[..., None] * (v - (k[..., None, :] @ held)[..., 0, :])
        new = held + k[..., :, None] * u[..., None, :]
        state = torch.where(on[..., None, None], new, state)
        y[:, t] = torch.where(on[..., None], scale * (q[..., None, :] @ new)[..., 0, :], 0.0)
    if not grad:
        return {"y": y, "state": state}
    out = {"dq": torch.zeros((b, n, hk, dk), **full), "dk": torch.zeros((b, n, hk, dk), **full), "dv": torch.zeros((b, n, h, dv), **full),
           "ddelta": torch.zeros((b, n, h), **full), "dbeta": torch.zeros((b, n, h), **full)}
    dA, dbias = torch.zeros(h, **full), torch.zeros(h, **full)
    gs = torch.zeros((b, h, dk, dv), **full) if s["dstate_out"] is None else s["dstate_out"].clone()
    for t in range(n - 1, -1, -1):
        on, pre, dt, a, strength, q, k, v = at(t)
        before = kept.pop()
        on1, on2 = on[..., None], on[..., None, None]
        held = a[..., None, None] * before
        miss = v - (k[..., None, :] @ held)[..., 0, :]
        u = strength[..., None] * miss
        dy = torch.where(on1, s["dy"][:, t], 0.0)
        new = held + k[..., :, None] * u[..., None, :]
        g = gs + scale * q[..., :, None] * dy[..., None, :]
        du = (k[..., None, :] @ g)[..., 0, :]
        dmiss = strength[..., None] * du
        dheld = g - k[..., :, None] * dmiss[..., None, :]
        dq = scale * (new @ dy[..., :, None])[..., 0]
        dkey = (g @ u[..., :, None])[..., 0] - (held @ dmiss[..., :, None])[..., 0]
        dg = a * (dheld * before).sum(dim=(2, 3))
        dpre = dg * s["A"] / (1.0 + torch.exp(-pre))
        out["dq"][:, t] = torch.where(on1, dq, 0.0).view(b, hk, h // hk, dk).sum(dim=2)
        out["dk"][:, t] = torch.where(on1, dkey, 0.0).view(b, hk, h // hk, dk).sum(dim=2)
        out["dv"][:, t] = torch.where(on1, dmiss, 0.0)
        out["dbeta"][:, t] = torch.where(on, (du * miss).sum(dim=-1) * strength * (1.0 - strength), 0.0)
        out["ddelta"][:, t] = torch.where(on, dpre, 0.0)
        dA += torch.where(on, dg * dt, 0.0).sum(dim=0)
        dbias += out["ddelta"][:, t].sum(dim=0)
        gs = torch.where(on2, a[..., None, None] * dheld, gs)
    return {**out, "dA": dA, "ddelta_bias": dbias, "ds": gs if case["state"] else None}


def _exact_delta_step(case, s):
    h, dk = case["heads"], case["key_dim"]
    of, out, y = torch.arange(h, device="cuda") // (h // case["key_heads"]), s["state_out"], torch.zeros_like(s["v"])
    for i, slot in enumerate(s["slots"].tolist()):
        pre = s["delta"][i] + s["delta_bias"]
        a = torch.exp(torch.logaddexp(pre, torch.zeros_like(pre)) * s["A"])
        held = a[:, None, None] * s["state"][slot]
        q, k = s["q"][i, of], s["k"][i, of]
        u = (s["v"][i] - torch.matmul(k[:, None], held)[:, 0]) / (1.0 + torch.exp(-s["beta"][i]))[:, None]
        out[slot] = held + k[:, :, None] * u[:, None]
        y[i] = torch.matmul(q[:, None], out[slot])[:, 0] / math.sqrt(dk)
    return {"y": y, "state": out}


def _exact_norm(case, s):
    b, n, d, half = case["batch"], case["length"], case["dim"], case["rotary"] // 2
    inside = (torch.arange(n, device="cuda")[None] < torch.tensor(_lengths(case), device="cuda")[:, None])[..., None, None]
    grad = case["op"] == "norm_grad"
    at = torch.arange(half, device="cuda")
    first, second = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + half)
    if half:
        turn = torch.complex(s["cos"], s["sin"])[s["positions"].long()][:, :, None]

    def turned(x, by):
        x = x.clone()
        if half:
            z = torch.complex(x[..., first], x[..., second]) * by
            x[..., first], x[..., second] = z.real, z.imag
        return x

    def one(x, w, dy):
        m = 1.0 / torch.sqrt((x * x).sum(dim=-1, keepdim=True) / (d if case["norm"] == "RMS" else 1) + EPS)
        if not grad:
            z = x * m * (1.0 if w is None else w)
            return torch.where(inside, turned(z, turn if half else None), 0.0)
        dz = torch.where(inside, turned(dy, turn.conj() if half else None), 0.0)
        dn = dz * (1.0 if w is None else w)
        share = m ** 3 / (d if case["norm"] == "RMS" else 1)
        dx = m * dn - share * x * (x * dn).sum(dim=-1, keepdim=True)
        return torch.where(inside, dx, 0.0), None if w is None else (dz * x * m).sum(dim=(0, 1, 2))
    if not grad:
        return {"q": one(s["q"], s["wq"], None), "k": one(s["k"], s["wk"], None)}
    (dq, dwq), (dk, dwk) = one(s["q"], s["wq"], s["dyq"]), one(s["k"], s["wk"], s["dyk"])
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
