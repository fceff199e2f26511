"""The operators of a gated delta rule layer where no GPU is needed: what the C entry points and the binding refuse, the sizes of workspaces, and the
64-bit references' gradients against differences."""
import os
import shutil
import subprocess

import pytest
import torch

import delta_reference as D
from paper_2010_15884_amd import binding as B
from paper_2010_15884_amd import sequence as S

OK, NULL, SIZE, ALIAS, UNSUPPORTED = B.SYS_OK, B.SYS_ERR_NULL, B.SYS_ERR_SIZE, B.SYS_ERR_ALIAS, B.SYS_ERR_UNSUPPORTED
# fake "device" addresses far apart: validation never dereferences them
P = [0x100000000 * (i + 1) for i in range(24)]

HEADS = dict(dtype=B.SYS_BF16, param_dtype=B.SYS_F32, norm=0, rotary=8, interleaved=0, batch=2, length=10, q_heads=4, k_heads=2, dim=16, positions=30, eps=1e-6,
             q_batch=640, q_row=64, k_batch=320, k_row=32, yq_batch=640, yq_row=64, yk_batch=320, yk_row=32)
DELTA = dict(dtype=B.SYS_BF16, softplus=1, sigmoid=1, batch=2, length=70, key_heads=2, value_heads=4, key_dim=16, value_dim=8, slots=5, scale=0.25, reserved=0,
             q_batch=2240, q_row=32, k_batch=2240, k_row=32, v_batch=2240, v_row=32, delta_batch=280, delta_row=4, beta_batch=280, beta_row=4, y_batch=2240, y_row=32)
STRUCTS = {"sys_head_norm": (S._HEADS, HEADS), "sys_gated_delta_rule": (S._DELTA, DELTA)}
# pointers by name, in order; [] marks what may be NULL
ARGUMENTS = {
    "sys_head_norm": "q k [wq] [wk] cos sin [positions] [lengths] yq yk",
    "sys_head_norm_backward": "dyq dyk q k [wq] [wk] cos sin [positions] [lengths] dq dk [dwq] [dwk] workspace",
    "sys_gated_delta_rule": "q k v delta A beta [delta_bias] [state] [lengths] y [state_out] workspace",
    "sys_gated_delta_rule_backward": "dy q k v delta A beta [delta_bias] [state] [lengths] [dstate_out] dq dk dv ddelta dA dbeta [ddelta_bias] [dstate] workspace",
    "sys_gated_delta_rule_update": "q k v delta A beta [delta_bias] state [slots] y state_out",
}
OUTPUTS = {
    "sys_head_norm": "yq yk", "sys_head_norm_backward": "dq dk dwq dwk workspace", "sys_gated_delta_rule": "y state_out workspace",
    "sys_gated_delta_rule_backward": "dq dk dv ddelta dA dbeta ddelta_bias dstate workspace", "sys_gated_delta_rule_update": "y state_out",
}


def _call(name, change=None, pointers=None):
    packer, fields = STRUCTS[name.replace("_backward", "").replace("_update", "")]
    fields = dict(fields, **(change or {}))
    names = [a.strip("[]") for a in ARGUMENTS[name].split()]
    at = dict(zip(names, P))
    at.update(pointers or {})
    return getattr(S._entry_points(), name)(packer.pack(*fields.values()), *[at[n] for n in names], None)


def _refused(name, want, change=None, pointers=None):
    got = _call(name, change, pointers)
    assert got == want, (name, change, pointers, B.status_string(got))


def test_structs_have_the_header_s_sizes():
    assert (S._HEADS.size, S._DELTA.size) == (112, 144)


@pytest.mark.parametrize("name", ARGUMENTS)
def test_required_pointers(name):
    for a in ARGUMENTS[name].split():
        if not a.startswith("["):
            _refused(name, NULL, pointers={a: None})
    assert getattr(S._entry_points(), name)(None, *P[:len(ARGUMENTS[name].split())], None) == NULL


@pytest.mark.parametrize("name", ARGUMENTS)
def test_outputs_meet_nothing(name):
    names = [a.strip("[]") for a in ARGUMENTS[name].split()]
    for out in OUTPUTS[name].split():
        for other in names:
            if other == out or {out, other} == {"state", "state_out"} and name.endswith("update"):
                continue
            _refused(name, ALIAS, pointers={out: P[names.index(other)]})
    if name.endswith("update"):                    # in place or apart, not in between
        _refused(name, ALIAS, pointers={"state_out": P[names.index("state")] + 4})


def test_results_end_where_others_begin():
    # 64 columns of the last of 2 x 10 rows, in bf16
    q, y = P[0], P[8]
    _refused("sys_head_norm", ALIAS, pointers={"yq": q + 2 * 640 * 2 - 2})
    _refused("sys_head_norm", ALIAS, pointers={"yk": y + 2 * 640 * 2 - 2})
    _refused("sys_gated_delta_rule", ALIAS, pointers={"y": q - 2 * 2240 * 2 + 2})
    _refused("sys_gated_delta_rule_update", ALIAS, dict(y_batch=32), pointers={"y": P[7] + 5 * 4 * 16 * 8 * 4 - 2})


@pytest.mark.parametrize("name", ARGUMENTS)
def test_alignment(name):
    for a in ARGUMENTS[name].split():
        _refused(name, UNSUPPORTED, pointers={a.strip("[]"): P[20] + 1})


BAD = [-1, (1 << 40) + 1]                          # of a stride
SIZES = {
    "sys_head_norm": [(dict(batch=-1), SIZE), (dict(length=-1), SIZE), (dict(q_heads=0), SIZE), (dict(k_heads=-1), SIZE), (dict(dim=0), SIZE), (dict(positions=-1), SIZE),
                      (dict(eps=-1.0), SIZE), (dict(eps=float("nan")), SIZE), (dict(rotary=-2), SIZE), (dict(rotary=7), SIZE), (dict(rotary=18), SIZE),
                      (dict(dim=513, yq_row=1 << 20, yk_row=1 << 20), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
                      (dict(param_dtype=B.SYS_F16), UNSUPPORTED), (dict(norm=2), UNSUPPORTED), (dict(norm=-1), UNSUPPORTED), (dict(interleaved=2), UNSUPPORTED),
                      (dict(q_heads=(1 << 20) + 1), UNSUPPORTED), (dict(k_heads=(1 << 20) + 1), UNSUPPORTED), (dict(q_heads=(1 << 31) - 1, dim=512), UNSUPPORTED),
                      *[({s: v}, SIZE) for s in ("q_batch", "q_row", "k_batch", "k_row", "yq_batch", "yq_row", "yk_batch", "yk_row") for v in BAD]],
    "sys_gated_delta_rule": [(dict(batch=-1), SIZE), (dict(length=-1), SIZE), (dict(key_heads=0), SIZE), (dict(value_heads=0), SIZE), (dict(key_heads=3), SIZE),
                             (dict(value_heads=1), SIZE), (dict(key_dim=0), SIZE), (dict(value_dim=0), SIZE), (dict(key_dim=129), UNSUPPORTED),
                             (dict(value_dim=1025), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(softplus=2), UNSUPPORTED),
                             (dict(sigmoid=-1), UNSUPPORTED), (dict(reserved=1), UNSUPPORTED), (dict(value_heads=(1 << 21) + 2, value_dim=8), UNSUPPORTED),
                             (dict(key_heads=(1 << 30), value_heads=(1 << 30)), UNSUPPORTED),
                             *[({s + "_batch": v}, SIZE) for s in ("q", "k", "v", "delta", "beta", "y") for v in BAD],
                             *[({s + "_row": v}, SIZE) for s in ("q", "k", "v", "delta", "beta", "y") for v in BAD]],
}


@pytest.mark.parametrize("name", ARGUMENTS)
def test_sizes_and_types(name):
    base = name.replace("_backward", "").replace("_update", "")
    for change, want in SIZES[base]:
        _refused(name, want, change)
    if name.endswith("update"):
        _refused(name, SIZE, dict(slots=-1))
        _refused(name, SIZE, dict(slots=1), pointers={"slots": None})
        _refused(name, SIZE, dict(y_batch=31))
    elif base == "sys_gated_delta_rule":
        for s in ("q", "k", "v", "delta", "beta", "y"):
            _refused(name, UNSUPPORTED, {s + "_row": 1 << 24, "y_batch": 1 << 40})
        _refused(name, UNSUPPORTED, dict(length=(1 << 30) + 1, y_batch=1 << 40))
    else:
        _refused(name, UNSUPPORTED, dict(length=(1 << 30) + 1, yq_batch=1 << 40, yk_batch=1 << 40))
        _refused(name, SIZE, dict(positions=9), pointers={"positions": None})
    if name == "sys_gated_delta_rule":
        _refused(name, SIZE, dict(y_row=31))
        _refused(name, SIZE, dict(y_batch=2239))
    if name == "sys_head_norm":
        for change in (dict(yq_row=63), dict(yk_row=31), dict(yq_batch=639), dict(yk_batch=319)):
            _refused(name, SIZE, change)


def test_gradients_need_what_they_are_of():
    for of in ("delta_bias", "state"):
        _refused("sys_gated_delta_rule_backward", NULL, pointers={of: None})
    for of in ("wq", "wk"):
        _refused("sys_head_norm_backward", NULL, pointers={of: None})
    _refused("sys_head_norm_backward", NULL, dict(k_heads=0))              # dwk without keys


def test_empty_calls_need_no_tensors():
    none = lambda names: {n: None for n in names.split()}  # noqa: E731
    for empty in (dict(batch=0), dict(length=0, q_batch=0)):
        assert _call("sys_head_norm", empty, none("q k cos sin yq yk")) == OK
        assert _call("sys_head_norm_backward", empty, none("dyq dyk q k cos sin dq dk dwq dwk workspace")) == OK
    assert _call("sys_gated_delta_rule", dict(batch=0), none("q k v delta beta y")) == OK
    assert _call("sys_gated_delta_rule_update", dict(batch=0), none("q k v delta beta y")) == OK
    # no turning: no tables; a table without rows holds no token
    _refused("sys_head_norm", ALIAS, dict(rotary=0), dict(none("cos sin"), yq=P[0]))
    _refused("sys_head_norm", ALIAS, dict(positions=0), dict(none("cos sin"), yq=P[0]))
    _refused("sys_head_norm", NULL, pointers=none("cos"))


def test_workspaces_grow_with_the_call_and_are_0_where_it_is_refused():
    c = S._entry_points()
    for name, (packer, fields) in STRUCTS.items():
        for form in ("_workspace", "_backward_workspace"):
            f = getattr(c, name + form, None)
            if f is None:
                continue
            assert f(packer.pack(*dict(fields, dtype=7).values())) == 0 == f(None)
            small, large = (f(packer.pack(*dict(fields, batch=b).values())) for b in (2, 200))
            assert 0 < small <= large < 1 << 30 and small % 4 == 0
    size = lambda **change: c.sys_gated_delta_rule_workspace(S._DELTA.pack(*dict(DELTA, **change).values()))  # noqa: E731
    assert size(length=1) == 0                     # a position at a time needs none
    # beyond 32 bits, and in full
    long = dict(batch=64, length=1 << 20, key_heads=16, value_heads=64, key_dim=128, value_dim=128, q_row=2048, k_row=2048, v_row=8192, y_row=8192, y_batch=1 << 33)
    f = c.sys_gated_delta_rule_backward_workspace
    assert f(S._DELTA.pack(*dict(DELTA, **long).values())) > 64 * (1 << 14) * 64 * 2 * 128 * 128 * 4


def test_binding_refuses_before_the_library_is_looked_for(monkeypatch):
    monkeypatch.setattr(B, "LIB_PATH", "/nowhere/libsysconv.so")
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(S, "_calls", None)
    x, w = torch.zeros((2, 5, 2, 8)), torch.zeros(2)
    gates = torch.zeros((2, 5, 2))
    for call in (lambda: B.sys_head_norm(x), lambda: B.sys_head_norm(None), lambda: B.sys_head_norm(x, x, w, w), lambda: B.sys_head_norm_backward(x, None, x),
                 lambda: B.sys_gated_delta_rule(x, x, x, gates, w, gates), lambda: B.sys_gated_delta_rule(None, x, x, gates, w, gates),
                 lambda: B.sys_gated_delta_rule_backward(x, x, x, x, gates, w, gates),
                 lambda: B.sys_gated_delta_rule_update(x[:, 0], x[:, 0], x[:, 0], gates[:, 0], w, gates[:, 0], x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_binding_refuses_shapes_types_and_strides():
    zeros = lambda *s, **how: torch.zeros(s, device="cuda", **how)  # noqa: E731
    q, k, w, table = zeros(2, 5, 4, 8), zeros(2, 5, 2, 8), zeros(8), zeros(9, 4)
    positions, lengths = zeros(2, 5, dtype=torch.int32), zeros(2, dtype=torch.int32)
    ok = dict(d_q=q, d_k=k, d_wq=w, d_wk=w, d_cos=table, d_sin=table, d_positions=positions, d_lengths=lengths)
    B.sys_head_norm(**ok)
    for error, change in ((ValueError, dict(d_q=q[0])), (ValueError, dict(d_q=q.transpose(1, 2).contiguous().transpose(1, 2))), (ValueError, dict(d_k=k[:1])),
                          (TypeError, dict(d_k=k.half())), (ValueError, dict(d_k=zeros(2, 5, 2, 6))), (ValueError, dict(d_wq=w[:7])), (TypeError, dict(d_wq=w.half())),
                          (ValueError, dict(d_sin=None)), (ValueError, dict(d_sin=table[:8])), (TypeError, dict(d_cos=table.half())), (ValueError, dict(d_cos=None, d_sin=None)),
                          (ValueError, dict(d_positions=positions[:1])), (TypeError, dict(d_positions=positions.long())), (TypeError, dict(d_lengths=lengths.float())),
                          (ValueError, dict(d_yq=k)), (KeyError, dict(norm="MAX")), (B.SysconvError, dict(eps=-1.0)), (B.SysconvError, dict(d_yq=q)),
                          (ValueError, dict(d_k=None)), (TypeError, dict(d_q=q.cpu())), (ValueError, dict(d_q=zeros(2, 5, 4, 16)[..., ::2])),
                          (B.SysconvError, dict(d_positions=None, d_cos=table[:4].contiguous(), d_sin=table[:4].contiguous()))):
        with pytest.raises(error):
            B.sys_head_norm(**dict(ok, **change))
    with pytest.raises(TypeError):
        B.sys_head_norm_backward(q, None, **ok)
    v, gates, A, state = zeros(2, 5, 4, 6), zeros(2, 5, 4), zeros(4), zeros(2, 4, 8, 6)
    ok = dict(d_q=k, d_k=k, d_v=v, d_delta=gates, d_A=A, d_beta=gates, d_delta_bias=A, d_state=state, d_lengths=lengths)
    B.sys_gated_delta_rule(**ok)
    wrong = ((ValueError, dict(d_q=k[0])), (ValueError, dict(d_k=q)), (ValueError, dict(d_v=v[:, :4])), (TypeError, dict(d_v=v.half())), (ValueError, dict(d_delta=gates[..., :3])),
             (TypeError, dict(d_beta=gates.half())), (TypeError, dict(d_A=A.half())), (ValueError, dict(d_A=A[:3])), (TypeError, dict(d_A=None)),
             (ValueError, dict(d_delta_bias=A[:3])), (ValueError, dict(d_state=state[:1])), (TypeError, dict(d_state=state.half())), (ValueError, dict(d_lengths=lengths[:1])),
             (B.SysconvError, dict(d_q=zeros(2, 5, 3, 8), d_k=zeros(2, 5, 3, 8))), (B.SysconvError, dict(d_q=zeros(2, 5, 2, 129), d_k=zeros(2, 5, 2, 129), d_state=None)))
    for error, change in (*wrong, (ValueError, dict(d_y=v[:1])), (B.SysconvError, dict(d_y=v)), (ValueError, dict(d_state_out=state[:1])), (B.SysconvError, dict(d_state_out=state))):
        with pytest.raises(error):
            B.sys_gated_delta_rule(**dict(ok, **change))
    for error, change in (*wrong, (TypeError, dict(d_dy=v.half())), (ValueError, dict(d_dy=v[:1])), (ValueError, dict(d_dstate_out=state[:1]))):
        with pytest.raises(error):
            B.sys_gated_delta_rule_backward(**{**ok, "d_dy": v, **change})
    ok = dict(d_q=k[:, 0], d_k=k[:, 0], d_v=v[:, 0], d_delta=gates[:, 0], d_A=A, d_beta=gates[:, 0], d_state=state, d_slots=lengths)
    B.sys_gated_delta_rule_update(**ok)
    for error, change in ((ValueError, dict(d_q=k)), (ValueError, dict(d_state=state[:, :2])), (TypeError, dict(d_state=state.half())), (TypeError, dict(d_slots=lengths.long())),
                          (ValueError, dict(d_slots=lengths[:1])), (B.SysconvError, dict(d_slots=None, d_state=state[:1])), (ValueError, dict(d_state_out=state[:1])),
                          (ValueError, dict(d_y=v)), (B.SysconvError, dict(d_y=v[:, 0]))):
        with pytest.raises(error):
            B.sys_gated_delta_rule_update(**dict(ok, **change))


# ---------------------------------------------------------------- the references themselves

def _slope(loss, point, key, v, e=1e-5):
    up, down = (loss({**point, key: point[key] + s * e * v}) for s in (1, -1))
    return float(up - down) / (2 * e)


@pytest.mark.parametrize("softplus,sigmoid", [(True, True), (False, False)])
def test_reference_gradients_of_the_rule_against_differences(softplus, sigmoid):
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    point = {"q": rand(2, 9, 2, 3), "k": 0.5 * rand(2, 9, 2, 3), "v": rand(2, 9, 4, 5), "delta": rand(2, 9, 4), "A": -rand(4).abs(), "beta": rand(2, 9, 4),
             "delta_bias": rand(4), "state": rand(2, 4, 3, 5)}
    dy, ds, how = rand(2, 9, 4, 5), rand(2, 4, 3, 5), dict(softplus=softplus, sigmoid_beta=sigmoid, lengths=[9, 4], scale=0.7)

    def loss(p):
        o = D.gated_delta(**p, **how)
        return (o["y"] * dy).sum() + (o["state"] * ds).sum()
    got = D.gated_delta(**point, **how, dy=dy, dstate_out=ds)
    for k in point:
        v = rand(*point[k].shape)
        assert _slope(loss, point, k, v) == pytest.approx(float((got["d" + k] * v).sum()), rel=1e-6, abs=1e-6), k


@pytest.mark.parametrize("norm,interleaved", [("RMS", False), ("L2", True)])
def test_reference_gradients_of_the_norm_against_differences(norm, interleaved):
    g = torch.Generator().manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    point, dy, angle = {"x": rand(2, 5, 3, 8), "w": rand(8)}, rand(2, 5, 3, 8), rand(7, 3)
    how = dict(cos=torch.cos(angle), sin=torch.sin(angle), positions=torch.tensor([[0, 6, 2, 7, 1], [3, -1, 4, 4, 5]]), norm=norm, interleaved=interleaved, lengths=[5, 4])
    got = D.head_norm(**point, **how, dy=dy)
    for k in point:
        v = rand(*point[k].shape)
        assert _slope(lambda p: (D.head_norm(**p, **how)["y"] * dy).sum(), point, k, v) == pytest.approx(float((got["d" + k] * v).sum()), rel=1e-6, abs=1e-7), k


def test_chunks_are_the_recurrence():
    """The formulas of a chunk, in 64 bits: (I + A) U = b (V - G K S), Y = scale (G Q S + P U), S' = G_end S + K^T (E U)."""
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    n, dk, dv, scale = 64, 12, 7, 0.3
    q, k, v, s = rand(n, dk), rand(n, dk), rand(n, dv), rand(dk, dv)
    k = k / k.norm(dim=1, keepdim=True)
    decay, b = -0.1 * rand(n).abs(), torch.sigmoid(rand(n))
    total = torch.cumsum(decay, 0)
    ratio = torch.exp(total[:, None] - total[None]).tril()
    a = b[:, None] * (ratio * (k @ k.T)).tril(-1)
    u = torch.linalg.solve_triangular(torch.eye(n, dtype=torch.float64) + a, b[:, None] * (v - total.exp()[:, None] * (k @ s)), upper=False)
    y = scale * (total.exp()[:, None] * (q @ s) + (ratio * (q @ k.T)) @ u)
    end = total[-1].exp() * s + k.T @ ((total[-1] - total).exp()[:, None] * u)
    want = D.gated_delta(q[None, :, None], k[None, :, None], v[None, :, None], decay[None, :, None], torch.ones(1, dtype=torch.float64), b[None, :, None], scale=scale,
                         softplus=False, sigmoid_beta=False, state=s[None, None])
    assert float((y - want["y"][0, :, 0]).abs().max()) < 1e-12 and float((end - want["state"][0, 0]).abs().max()) < 1e-12


def test_host_code_under_sanitizers():
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc is not installed")
    from paper_2010_15884_amd import build
    exe = build.build_host_sanitized(verbose=False, driver="delta_san_driver")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert res.returncode == 0 and "clean" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr
