"""The operators on channels-last sequences where no GPU is needed: what the C entry points and the binding refuse, the sizes of workspaces, and the
64-bit references' gradients against differences."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import sequence_reference as R
from paper_2010_15884_amd import binding as B
from paper_2010_15884_amd import sequence as S

OK, NULL, SIZE, ALIAS, UNSUPPORTED = B.SYS_OK, B.SYS_ERR_NULL, B.SYS_ERR_SIZE, B.SYS_ERR_ALIAS, B.SYS_ERR_UNSUPPORTED
# fake "device" addresses far apart: validation never dereferences them
P = [0x100000000 * (i + 1) for i in range(24)]

CONV = dict(dtype=B.SYS_BF16, param_dtype=B.SYS_BF16, activation=1, width=4, batch=2, length=10, channels=16, slots=5, x_batch=160, x_row=16, y_batch=160,
            y_row=16)
SCAN = dict(dtype=B.SYS_BF16, softplus=1, batch=2, length=10, channels=16, states=16, groups=2, slots=5, u_batch=160, u_row=16, delta_batch=160, delta_row=16,
            z_batch=160, z_row=16, b_batch=320, b_row=32, c_batch=320, c_row=32, y_batch=160, y_row=16)
NORM = dict(dtype=B.SYS_BF16, param_dtype=B.SYS_F32, activation=1, groups=4, batch=2, channels=16, eps=1e-5, reserved=0, rows=10, x_batch=160, x_row=16,
            y_batch=160, y_row=16)
STRUCTS = {"sys_causal_conv1d": (S._CONV, CONV), "sys_selective_scan": (S._SCAN, SCAN), "sys_group_norm": (S._NORM, NORM)}
# pointers by name, in order; [] marks what may be NULL
ARGUMENTS = {
    "sys_causal_conv1d": "x w [bias] [state] [lengths] y [state_out]",
    "sys_causal_conv1d_backward": "dy x w [bias] [state] [lengths] [dstate_out] dx dw [dbias] [dstate] workspace",
    "sys_causal_conv1d_update": "x w [bias] state [slots] y state_out",
    "sys_selective_scan": "u delta A B C [D] [z] [delta_bias] [state] [lengths] y [state_out] [workspace]",
    "sys_selective_scan_backward": "dy u delta A B C [D] [z] [delta_bias] [state] [lengths] [dstate_out] du ddelta dA dB dC [dD] [dz] [ddelta_bias] [dstate] workspace",
    "sys_selective_scan_update": "u delta A B C [D] [z] [delta_bias] state [slots] y state_out",
    "sys_group_norm": "x [w] [b] y [mean] [rstd] [workspace]",
    "sys_group_norm_backward": "dy x [w] [b] mean rstd dx [dw] [db] workspace",
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


@pytest.mark.parametrize("name", ARGUMENTS)
def test_required_pointers(name):
    for a in ARGUMENTS[name].split():
        if not a.startswith("["):
            _refused(name, NULL, pointers={a: None})
    assert getattr(S._entry_points(), name)(None, *P[:len(ARGUMENTS[name].split())], None) == NULL


@pytest.mark.parametrize("name", ARGUMENTS)
def test_outputs_meet_nothing(name):
    names = [a.strip("[]") for a in ARGUMENTS[name].split()]
    outputs = [n for n in names if n in ("y", "state_out", "mean", "rstd", "workspace") or (n[0] == "d" and n not in ("dy", "delta", "delta_bias", "dstate_out"))]
    if name == "sys_group_norm_backward":
        outputs = [n for n in outputs if n not in ("mean", "rstd")]
    if name == "sys_selective_scan":
        outputs.remove("workspace")                # (none at this size)
    for out in outputs:
        for other in names:
            if other == out or (other == "workspace" and name == "sys_selective_scan") or {out, other} == {"state", "state_out"} and name.endswith("update"):
                continue
            _refused(name, ALIAS, pointers={out: P[names.index(other)]})
    if name.endswith("update"):                    # in place or apart, not in between
        _refused(name, ALIAS, pointers={"state_out": P[names.index("state")] + 4})


@pytest.mark.parametrize("name", ARGUMENTS)
def test_alignment(name):
    for a in ARGUMENTS[name].split():
        if a == "[workspace]" and name == "sys_selective_scan":
            continue
        _refused(name, UNSUPPORTED, pointers={a.strip("[]"): P[20] + 1})


SIZES = {
    "sys_causal_conv1d": [(dict(batch=-1), SIZE), (dict(length=-1), SIZE), (dict(channels=0), SIZE), (dict(x_row=-1), SIZE), (dict(x_batch=1 << 41), SIZE),
                          (dict(width=1), UNSUPPORTED), (dict(width=9), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
                          (dict(param_dtype=B.SYS_F16), UNSUPPORTED), (dict(activation=2), UNSUPPORTED), (dict(length=(1 << 30) + 1, y_batch=1 << 35), UNSUPPORTED),
                          (dict(channels=(1 << 24) + 1, y_row=1 << 25, y_batch=1 << 30), UNSUPPORTED)],
    "sys_selective_scan": [(dict(batch=-1), SIZE), (dict(length=-1), SIZE), (dict(channels=0), SIZE), (dict(states=0), SIZE), (dict(groups=0), SIZE),
                           (dict(groups=3), SIZE), (dict(z_row=-1), SIZE), (dict(c_batch=1 << 41), SIZE), (dict(states=65), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED),
                           (dict(softplus=2), UNSUPPORTED)],
    "sys_group_norm": [(dict(batch=-1), SIZE), (dict(rows=0), SIZE), (dict(channels=0), SIZE), (dict(groups=0), SIZE), (dict(groups=3), SIZE),
                       (dict(eps=-1.0), SIZE), (dict(eps=float("nan")), SIZE), (dict(x_row=-1), SIZE), (dict(dtype=3), UNSUPPORTED),
                       (dict(param_dtype=B.SYS_F16), UNSUPPORTED), (dict(activation=3), UNSUPPORTED), (dict(activation=-1), UNSUPPORTED), (dict(reserved=1), UNSUPPORTED)],
}


@pytest.mark.parametrize("name", ARGUMENTS)
def test_sizes_and_types(name):
    base = name.replace("_backward", "").replace("_update", "")
    for change, want in SIZES[base]:
        if name.endswith("update") and "length" in change and "y_batch" in change:
            change = dict(length=(1 << 30) + 1)
        _refused(name, want, change)
    if not name.endswith("backward"):
        _refused(name, SIZE, dict(y_batch=15) if name.endswith("update") else dict(y_row=15))
        if not name.endswith("update"):
            _refused(name, SIZE, dict(y_batch=159))
    if name.endswith("update"):
        _refused(name, SIZE, dict(slots=-1))
        _refused(name, SIZE, dict(slots=1), pointers={"slots": None})


def test_gradients_need_what_they_are_of():
    _refused("sys_causal_conv1d_backward", NULL, pointers={"bias": None})
    _refused("sys_causal_conv1d_backward", NULL, pointers={"state": None})
    for of in ("D", "z", "delta_bias", "state", "dz"):
        _refused("sys_selective_scan_backward", NULL, pointers={of: None})
    for of in ("w", "b"):
        _refused("sys_group_norm_backward", NULL, pointers={of: None})


def test_empty_calls_need_no_tensors():
    empty = dict(batch=0)
    assert _call("sys_causal_conv1d", empty, dict(x=None, y=None)) == OK
    assert _call("sys_causal_conv1d_update", empty, dict(x=None, y=None)) == OK
    assert _call("sys_selective_scan", empty, dict(u=None, delta=None, B=None, C=None, y=None)) == OK
    assert _call("sys_selective_scan_update", empty, dict(u=None, delta=None, B=None, C=None, y=None)) == OK
    assert _call("sys_group_norm", empty, dict(x=None, y=None)) == OK


def test_workspaces_grow_with_the_call_and_are_0_where_it_is_refused():
    c = S._entry_points()
    for name, (packer, fields) in STRUCTS.items():
        for form in ("_workspace", "_backward_workspace"):
            f = getattr(c, name + form, None)
            if f is None:
                continue
            assert f(packer.pack(*dict(fields, dtype=7).values())) == 0 == f(None)
            small, large = (f(packer.pack(*dict(fields, batch=b).values())) for b in (2, 200))
            assert small <= large < 1 << 30 and small % 4 == 0
    # beyond 32 bits
    long = dict(SCAN, batch=64, length=1 << 20, channels=4096, u_row=4096, u_batch=1 << 32, y_row=4096, y_batch=1 << 32)
    assert c.sys_selective_scan_backward_workspace(S._SCAN.pack(*long.values())) > 1 << 40


def test_binding_refuses_before_the_library_is_looked_for(monkeypatch):
    monkeypatch.setattr(B, "LIB_PATH", "/nowhere/libsysconv.so")
    monkeypatch.setattr(B, "_lib", None)
    monkeypatch.setattr(S, "_calls", None)
    x, w = torch.zeros((2, 5, 8)), torch.zeros((8, 4))
    for call in (lambda: B.sys_causal_conv1d(x, w), lambda: B.sys_causal_conv1d(None, w), lambda: B.sys_causal_conv1d_backward(x, x, w),
                 lambda: B.sys_causal_conv1d_update(x[:, 0], w, None, x), lambda: B.sys_selective_scan(x, x, w, x, x),
                 lambda: B.sys_selective_scan_backward(x, x, x, w, x, x), lambda: B.sys_selective_scan_update(x, x, w, x, x, x),
                 lambda: B.sys_group_norm(x, 2), lambda: B.sys_group_norm_backward(x, x, 2, w, w)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_binding_refuses_shapes_types_and_strides():
    x, w, bias = torch.zeros((2, 5, 8), device="cuda"), torch.zeros((8, 4), device="cuda"), torch.zeros(8, device="cuda")
    states, lengths = torch.zeros((2, 3, 8), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ok = dict(d_x=x, d_w=w, d_bias=bias, d_state=states, d_lengths=lengths)
    B.sys_causal_conv1d(**ok)
    for error, change in ((ValueError, dict(d_x=x[0])), (ValueError, dict(d_x=torch.zeros((2, 8, 5), device="cuda").transpose(1, 2))), (ValueError, dict(d_w=w[:7])),
                          (TypeError, dict(d_w=w.half())), (TypeError, dict(d_x=x.double())), (ValueError, dict(d_w=w.t().contiguous().t())),
                          (ValueError, dict(d_bias=bias[:7])), (ValueError, dict(d_state=states[:1])), (TypeError, dict(d_state=states.half())),
                          (TypeError, dict(d_lengths=lengths.long())), (ValueError, dict(d_lengths=lengths[:1])), (ValueError, dict(d_y=x[:1])),
                          (TypeError, dict(d_y=x.half())), (KeyError, dict(activation="TANH")), (B.SysconvError, dict(activation="RELU")),
                          (B.SysconvError, dict(d_w=torch.zeros((8, 9), device="cuda"), d_state=None)), (B.SysconvError, dict(d_y=x))):
        with pytest.raises(error):
            B.sys_causal_conv1d(**dict(ok, **change))
    A, bc, D = torch.zeros((8, 16), device="cuda"), torch.zeros((2, 5, 2, 16), device="cuda"), torch.zeros(8, device="cuda")
    ok = dict(d_u=x, d_delta=x, d_A=A, d_B=bc, d_C=bc, d_D=D, d_z=x, d_delta_bias=D)
    B.sys_selective_scan(**ok)
    for error, change in ((ValueError, dict(d_delta=x[:, :4])), (TypeError, dict(d_A=A.half())), (ValueError, dict(d_A=A[:7])), (ValueError, dict(d_C=bc[:, :, :1])),
                          (ValueError, dict(d_B=bc[:, :, 0])), (TypeError, dict(d_B=bc.half())), (ValueError, dict(d_D=D[:7])), (TypeError, dict(d_z=x.half())),
                          (ValueError, dict(d_B=torch.zeros((2, 5, 2, 32), device="cuda")[..., :16])), (ValueError, dict(d_state=A)),
                          (B.SysconvError, dict(d_B=torch.zeros((2, 5, 3, 16), device="cuda"), d_C=torch.zeros((2, 5, 3, 16), device="cuda")))):
        with pytest.raises(error):
            B.sys_selective_scan(**dict(ok, **change))
    for error, change in ((ValueError, dict(d_x=x[0])), (ValueError, dict(d_w=D[:7])), (TypeError, dict(d_w=D.half())), (B.SysconvError, dict(groups=3)),
                          (B.SysconvError, dict(eps=-1.0)), (ValueError, dict(d_mean=A)), (B.SysconvError, dict(d_y=x))):
        with pytest.raises(error):
            B.sys_group_norm(**dict(dict(d_x=x, groups=2, d_w=D, d_b=D), **change))


# ---------------------------------------------------------------- the references themselves

def _slope(loss, point, key, v, e=1e-5):
    up, down = (loss({**point, key: point[key] + s * e * v}) for s in (1, -1))
    return float(up - down) / (2 * e)


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    point = {"x": rand(2, 9, 3), "w": rand(3, 4), "bias": rand(3), "state": rand(2, 3, 3)}
    dy, ds = rand(2, 9, 3), rand(2, 3, 3)

    def conv(p):
        o = R.causal_conv(**p, activation="SILU", lengths=[9, 4])
        return (o["y"] * dy).sum() + (o["state"] * ds).sum()
    got = R.causal_conv(**point, activation="SILU", lengths=[9, 4], dy=dy, dstate_out=ds)
    for k in point:
        v = rand(*point[k].shape)
        assert _slope(conv, point, k, v) == pytest.approx(float((got["d" + k] * v).sum()), rel=1e-6, abs=1e-7), k

    point = {"u": rand(2, 7, 4), "delta": rand(2, 7, 4), "A": -rand(4, 3).abs(), "B": rand(2, 7, 2, 3), "C": rand(2, 7, 2, 3), "D": rand(4), "z": rand(2, 7, 4),
             "delta_bias": rand(4), "state": rand(2, 4, 3)}
    dy, ds = rand(2, 7, 4), rand(2, 4, 3)

    def scan(p):
        o = R.scan(**p, lengths=[7, 5])
        return (o["y"] * dy).sum() + (o["state"] * ds).sum()
    got = R.scan(**point, lengths=[7, 5], dy=dy, dstate_out=ds)
    for k in point:
        v = rand(*point[k].shape)
        assert _slope(scan, point, k, v) == pytest.approx(float((got["d" + k] * v).sum()), rel=1e-6, abs=1e-7), k

    point = {"x": rand(2, 5, 6), "w": rand(6), "b": rand(6)}
    dy = rand(2, 5, 6)
    got = R.group_norm(point["x"], 2, point["w"], point["b"], activation="SILU", dy=dy)
    for k in point:
        v = rand(*point[k].shape)
        norm = lambda p: (R.group_norm(p["x"], 2, p["w"], p["b"], activation="SILU")["y"] * dy).sum()  # noqa: E731
        assert _slope(norm, point, k, v) == pytest.approx(float((got["d" + k] * v).sum()), rel=1e-6, abs=1e-7), k


def test_reference_bounds_are_bounds():
    g = torch.Generator().manual_seed(2)
    rand = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    c = [rand(1, 12, 4), rand(1, 12, 4), -rand(4, 3).abs(), rand(1, 12, 2, 3), rand(1, 12, 2, 3), rand(4), rand(1, 12, 4), rand(4)]
    args = dict(state=rand(1, 4, 3), dy=rand(1, 12, 4), dstate_out=rand(1, 4, 3))
    want, bound = R.scan(*c, **args), R.scan(*c, **args, bound=True)
    for k in want:
        if k != "sA":
            assert (want[k].abs() <= bound[k] * (1 + 1e-12)).all(), k


def test_host_code_under_sanitizers():
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc is not installed")
    from paper_2010_15884_amd import build
    exe = build.build_host_sanitized(verbose=False, driver="sequence_san_driver")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert res.returncode == 0 and "clean" in res.stdout, res.stdout[-2000:] + res.stderr[-4000:]
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr


def test_structs_have_the_header_s_sizes():
    assert (S._CONV.size, S._SCAN.size, S._NORM.size) == (64, 128, 72)
    assert ctypes.sizeof(ctypes.c_int) == 4
