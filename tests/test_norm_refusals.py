"""What the norm calls refuse on the host: nothing is launched by anything here."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


A, B, C, D, E, F = (ctypes.c_void_p(4096 * i) for i in range(1, 7))      # never dereferenced


def norm(r3, **kw):
    base = dict(T=4, d=64, act_dtype=1, w_dtype=1, gate_kind=0, eps=1e-6, residual_scale=1.0,
                branch_scale=1.0)
    base.update(kw)
    return r3.Norm(**base)


def fwd(r3, s, x=A, y=B, w_post=C, gate=None, w_pre=C, x_out=D, h=E):
    return r3.lib.r3_norm_residual(ctypes.byref(s) if s else None, x, y, w_post, gate, w_pre, x_out, h, None)


def bwd(r3, s, x_out=A, y=B, w_post=C, gate=None, w_pre=C, dx_out=A, dh=B, dx=D, dy=E, dw_post=F,
        dgate=None, dw_pre=F, ws=None, n=0):
    return r3.lib.r3_norm_residual_bwd(ctypes.byref(s) if s else None, x_out, y, w_post, gate, w_pre,
                                       dx_out, dh, dx, dy, dw_post, dgate, dw_pre, ws, n, None)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(T=0x7f000001), dict(T=(1 << 30) + 1), dict(d=0), dict(d=60), dict(act_dtype=2),
                                dict(w_dtype=7), dict(gate_kind=4), dict(gate_kind=-1), dict(eps=0.0),
                                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                dict(residual_scale=float("inf")), dict(branch_scale=float("nan"))])
def test_bad_shapes(r3, kw):
    s = norm(r3, **kw)
    assert fwd(r3, s) == r3.R3_ERR_INVALID_ARG and bwd(r3, s) == r3.R3_ERR_INVALID_ARG
    assert r3.lib.r3_norm_residual_bwd_workspace_bytes(ctypes.byref(s)) == 0


def test_too_wide(r3):
    for kw in (dict(d=16392), dict(d=8200, act_dtype=0)):
        assert fwd(r3, norm(r3, **kw)) == r3.R3_ERR_UNSUPPORTED
        assert bwd(r3, norm(r3, **kw)) == r3.R3_ERR_UNSUPPORTED


def test_bad_arguments(r3):
    s, bad = norm(r3), r3.R3_ERR_INVALID_ARG
    assert fwd(r3, None) == bad and bwd(r3, None) == bad
    assert fwd(r3, s, x=None) == bad
    assert fwd(r3, s, y=None, w_post=None, x_out=None, w_pre=None, h=None) == bad    # nothing to do
    assert fwd(r3, s, y=None, x_out=None) == bad                                     # w_post without y
    assert fwd(r3, s, y=None, w_post=None) == bad                                    # x_out without y
    assert fwd(r3, s, x_out=None) == bad
    assert fwd(r3, s, gate=A) == bad                                                 # kind NONE
    assert fwd(r3, norm(r3, gate_kind=1)) == bad                                     # kind without gate
    assert fwd(r3, s, h=None) == bad and fwd(r3, s, w_pre=None) == bad
    assert fwd(r3, s, h=D) == bad                                                    # h is x_out
    assert fwd(r3, s, x=ctypes.c_void_p(4104)) == bad                                # 8-byte aligned
    assert fwd(r3, norm(r3, gate_kind=2), gate=ctypes.c_void_p(4098)) == bad
    assert bwd(r3, s, dx=None) == bad and bwd(r3, s, dy=None) == bad and bwd(r3, s, dy=D) == bad
    assert bwd(r3, s, dw_post=None) == bad and bwd(r3, s, dw_pre=None) == bad
    assert bwd(r3, s, x_out=None) == bad and bwd(r3, s, dh=None) == bad
    assert bwd(r3, s, w_pre=None, dw_pre=None) == bad                                # dh without w_pre
    assert bwd(r3, s, w_pre=None, dw_pre=None, dh=None, dx_out=None) == bad          # no gradient at all
    assert bwd(r3, s, dgate=F) == bad
    assert bwd(r3, norm(r3, gate_kind=3), gate=A) == bad
    assert bwd(r3, s, dy=ctypes.c_void_p(8)) == bad
    assert bwd(r3, s) == r3.R3_ERR_WORKSPACE
    assert bwd(r3, s, ws=ctypes.c_void_p(4096 + 16), n=1 << 30) == r3.R3_ERR_WORKSPACE
    empty = norm(r3, T=0)
    assert fwd(r3, empty, x=None, y=None, x_out=None, h=None) == r3.R3_OK


def test_python_checks(r3):
    with pytest.raises(ValueError):
        r3.norm_residual(torch.zeros(2, 8), w_pre=torch.ones(8))                     # host tensors
    with pytest.raises(TypeError):
        r3.norm_residual(None)


def kind_of(r3, rows, d, gate, weights=None, said=None):
    """The gate kind that the binding takes for a call (checked against host tensors here)."""
    like = None if weights is None else torch.ones(d, dtype=weights)
    return r3._norm_shape(rows, d, torch.bfloat16, like, gate, None, 1e-6, 1.0, 1.0, torch.device("cpu"),
                          said)[0].gate_kind


def test_gate_kinds_by_shape(r3):
    f32, bf = torch.float32, torch.bfloat16
    assert kind_of(r3, 4, 64, torch.ones(64), f32) == r3.R3_GATE_CHANNEL
    assert kind_of(r3, 4, 64, torch.ones(64)) == r3.R3_GATE_CHANNEL
    assert kind_of(r3, 4, 64, torch.ones(4), f32) == r3.R3_GATE_TOKEN
    assert kind_of(r3, 4, 64, torch.ones(4), bf) == r3.R3_GATE_TOKEN
    assert kind_of(r3, 4, 64, torch.ones(4, 1), bf) == r3.R3_GATE_TOKEN
    assert kind_of(r3, 1, 64, torch.ones(1), bf) == r3.R3_GATE_TOKEN
    assert kind_of(r3, 4, 64, torch.ones((4, 64), dtype=bf), f32) == r3.R3_GATE_FULL
    for bad in (torch.ones(5), torch.ones(1, 64), torch.ones(64, 1), torch.ones(4, dtype=bf), torch.ones(())):
        with pytest.raises(ValueError):
            kind_of(r3, 4, 64, bad, f32)


def test_a_vector_with_as_many_rows_as_columns(r3):
    """[T] = [d]: the types tell a gate per channel (the weights') from one per token (float32), or the
    caller does."""
    f32, bf = torch.float32, torch.bfloat16
    assert kind_of(r3, 64, 64, torch.ones(64, dtype=bf), bf) == r3.R3_GATE_CHANNEL
    assert kind_of(r3, 64, 64, torch.ones(64, dtype=bf)) == r3.R3_GATE_CHANNEL
    assert kind_of(r3, 64, 64, torch.ones(64), bf) == r3.R3_GATE_TOKEN
    assert kind_of(r3, 64, 64, torch.ones(64, 1), f32) == r3.R3_GATE_TOKEN
    for weights in (f32, None):
        with pytest.raises(ValueError, match="gate_kind"):
            kind_of(r3, 64, 64, torch.ones(64), weights)
        assert kind_of(r3, 64, 64, torch.ones(64), weights, "channel") == r3.R3_GATE_CHANNEL
        assert kind_of(r3, 64, 64, torch.ones(64), weights, "token") == r3.R3_GATE_TOKEN
    with pytest.raises(ValueError):
        kind_of(r3, 64, 64, torch.ones(64), f32, "row")
    for said, gate in (("channel", torch.ones(4)), ("token", torch.ones(64)), ("full", torch.ones(64)),
                       ("channel", torch.ones(4, 64))):
        with pytest.raises(ValueError):
            kind_of(r3, 4, 64, gate, f32, said)


def test_scratch_of_another_device_is_refused(r3, monkeypatch):
    """A caller's workspace is looked at like every other tensor: its address would be written to (a stand-in
    for the library here, host tensors for the device's)."""
    calls = []

    class Library:
        def __getattr__(self, name):
            def call(*a):
                calls.append(name)
                return 0
            return call
    monkeypatch.setattr(r3, "lib", Library())
    monkeypatch.setattr(r3, "_device_of", lambda name, t: t.device)
    monkeypatch.setattr(r3, "_stream", lambda stream=None: None)
    x, w = torch.zeros((4, 64)), torch.ones(64)
    room = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (room.to("meta"), room[::2], 4096):
        with pytest.raises((ValueError, TypeError)):
            r3.norm_residual_bwd(x, x, x, x, w_post=w, w_pre=w, ws=bad)
    assert "r3_norm_residual_bwd" not in calls
    r3.norm_residual_bwd(x, x, x, x, w_post=w, w_pre=w, ws=room)
    r3.norm_residual_bwd(x, x, x, x, w_post=w, w_pre=w)
    assert calls.count("r3_norm_residual_bwd") == 2
