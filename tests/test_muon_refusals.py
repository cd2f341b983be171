"""What the orthogonalised update refuses on the host: nothing is launched by anything here."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


def doubles(*v):
    return ctypes.cast((ctypes.c_double * len(v))(*v), ctypes.c_void_p)


def ortho(r3, **kw):
    cfg = dict(batch=2, rows=16, cols=24, in_dtype=0, out_dtype=0, steps=5, products=1, eps=1e-7, coefs=None)
    at = dict(x=1 << 20, out=2 << 20, ws=3 << 20, ws_bytes=1 << 30, status=None)
    for k, v in kw.items():
        (cfg if k in cfg else at)[k] = v
    return r3.lib.r3_orthogonalize(ctypes.byref(r3.Orthogonal(**cfg)), *at.values(), None)


BAD = [dict(steps=0), dict(steps=17), dict(products=2), dict(products=0), dict(eps=-1e-9), dict(eps=math.nan),
       dict(eps=math.inf), dict(steps=1, coefs=doubles(math.nan, 0, 0)), dict(steps=1, coefs=doubles(1, math.inf, 0)),
       dict(steps=1, coefs=doubles(20.0, 0, 0)), dict(steps=1, coefs=doubles(1, -90.0, 30.0)),
       dict(steps=3, coefs=doubles(*[4.0, 0, 0] * 3))]


@pytest.mark.parametrize("kw", BAD + [
    dict(batch=-1), dict(rows=0), dict(cols=0), dict(rows=16385), dict(cols=16385), dict(batch=(1 << 24) + 1),
    dict(in_dtype=2), dict(out_dtype=-1), dict(x=None), dict(out=None), dict(x=(1 << 20) + 8),
    dict(out=(2 << 20) + 8), dict(status=4097), dict(out=1 << 20, out_dtype=1), dict(out=(1 << 20) + 3056),
    dict(x=(2 << 20) + 3056), dict(x=(2 << 20) - 1520, in_dtype=1)])
def test_orthogonalize_refused(r3, kw):
    assert ortho(r3, **kw) == r3.R3_ERR_INVALID_ARG


def test_orthogonalize_workspace(r3):
    for kw in (dict(ws=None), dict(ws=(3 << 20) + 128), dict(ws_bytes=255), dict(ws_bytes=1 << 20, rows=300, cols=300)):
        assert ortho(r3, **kw) == r3.R3_ERR_WORKSPACE
    assert ortho(r3, batch=0, x=None, out=None, ws=None) == r3.R3_OK
    assert r3.lib.r3_orthogonalize(None, None, None, None, 0, None, None) == r3.R3_ERR_INVALID_ARG
    assert r3.lib.r3_orthogonalize_workspace_bytes(None) == 0


def muon(r3, stacks=None, grad_scale=None, lr_now=None, n=None, ws=1 << 40, ws_bytes=1 << 32, status=None, **kw):
    cfg = dict(param_dtype=0, grad_dtype=0, master=0, nesterov=1, steps=5, products=1, lr=0.1, momentum=0.9,
               eps=1e-7, coefs=None)
    cfg.update(kw)
    rows = []
    for i, t in enumerate([{}] if stacks is None else stacks):
        row = dict(param=(1 + 8 * i) << 20, master=None, grad=(2 + 8 * i) << 20, momentum=(3 + 8 * i) << 20, batch=2,
                   rows=8, cols=16, weight_decay=0.0, scale=1.0)
        row.update(t)
        rows.append(r3.MuonStack(**row))
    table = (r3.MuonStack * max(1, len(rows)))(*rows)
    return r3.lib.r3_muon_step(ctypes.byref(r3.MuonConfig(**cfg)), table, len(rows) if n is None else n, grad_scale,
                               lr_now, ws, ws_bytes, status, None)


A = 1 << 20                                                    # the first entry's param; 256 elements


@pytest.mark.parametrize("kw", BAD + [
    dict(param_dtype=2), dict(grad_dtype=5), dict(master=1), dict(lr=-1.0), dict(lr=math.nan), dict(momentum=1.0),
    dict(momentum=-0.1), dict(n=-1), dict(param_dtype=1, master=1), dict(stacks=[dict(master=9 << 20)]),
    dict(stacks=[dict(batch=-1)]), dict(stacks=[dict(rows=0)]), dict(stacks=[dict(cols=16385)]),
    dict(stacks=[dict(weight_decay=-1.0)]), dict(stacks=[dict(weight_decay=math.nan)]),
    dict(stacks=[dict(scale=-1.0)]), dict(stacks=[dict(scale=math.inf)]), dict(stacks=[dict(param=None)]),
    dict(stacks=[dict(grad=None)]), dict(stacks=[dict(momentum=None)]), dict(stacks=[dict(param=A + 8)]),
    dict(stacks=[dict(momentum=(3 << 20) + 4)]), dict(grad_scale=4097), dict(lr_now=4098), dict(status=4098),
    # the same memory twice
    dict(stacks=[{}, dict(param=A)]), dict(stacks=[{}, dict(param=A + 1008)]), dict(stacks=[dict(momentum=A)]),
    dict(stacks=[{}, dict(momentum=3 << 20)]), dict(stacks=[dict(grad=A)]), dict(stacks=[dict(grad=(3 << 20) + 1008)]),
    dict(stacks=[{}, dict(grad=A)]), dict(grad_scale=A + 4), dict(lr_now=(3 << 20) + 1020),
    dict(param_dtype=1, master=1, stacks=[dict(master=9 << 20, grad=9 << 20)]),
])
def test_muon_refused(r3, kw):
    assert muon(r3, **kw) == r3.R3_ERR_INVALID_ARG


def test_muon_workspace_and_nothing_to_do(r3):
    for kw in (dict(ws=None), dict(ws=(1 << 40) + 128), dict(ws_bytes=255),
               dict(stacks=[dict(rows=300, cols=300, param=1 << 36, momentum=2 << 36)], ws_bytes=1 << 20)):
        assert muon(r3, **kw) == r3.R3_ERR_WORKSPACE
    assert muon(r3, stacks=[], ws=None) == r3.R3_OK
    assert muon(r3, stacks=[dict(batch=0, param=None, grad=None, momentum=None)] * 2, ws=None) == r3.R3_OK
    assert r3.lib.r3_muon_step(None, None, 0, None, None, None, 0, None, None) == r3.R3_ERR_INVALID_ARG
    shared = [dict(grad=9 << 30), dict(grad=9 << 30)]            # one gradient for two stacks is only read
    assert muon(r3, stacks=shared, ws=None) == r3.R3_ERR_WORKSPACE


def test_struct_layouts(r3):
    assert ctypes.sizeof(r3.Orthogonal) == 48 and ctypes.sizeof(r3.MuonStack) == 56
    assert ctypes.sizeof(r3.MuonConfig) == 56


@pytest.mark.parametrize("bad", ["size", "dtype", "layout", "kind", "count", "none"])
def test_refused_gradients_leave_the_handle_as_it_was(r3, monkeypatch, bad):
    monkeypatch.setattr(r3, "_ptr", lambda t: ctypes.c_void_p(t.data_ptr()) if t.is_contiguous() else
                        (_ for _ in ()).throw(ValueError("tensor must be contiguous")))
    monkeypatch.setattr(r3, "_device_of", lambda name, t: t.device)
    params = [torch.zeros(4, 8), torch.zeros(2, 4, 8)]
    opt = r3.Muon(params, [torch.zeros_like(p) for p in params])
    before = [row.grad for row in opt._table]
    new = [torch.zeros(p.shape, dtype=torch.bfloat16) for p in params]
    new[1] = {"size": new[1][:1], "dtype": params[1], "layout": torch.zeros(2, 8, 4, dtype=torch.bfloat16).mT,
              "kind": [0.0], "count": new[1], "none": None}[bad]
    with pytest.raises((ValueError, TypeError)):
        opt.set_grads(new[:1] if bad == "count" else new)
    assert [row.grad for row in opt._table] == before and opt._config.grad_dtype == r3.R3_F32
    assert (opt._table[1].batch, opt._table[1].rows, opt._table[1].cols) == (2, 4, 8)


def test_binding_refuses(r3, monkeypatch):
    with pytest.raises(ValueError):
        r3.Muon([torch.zeros(4, 8)])
    monkeypatch.setattr(r3, "_device_of", lambda name, t: t.device)
    monkeypatch.setattr(r3, "_ptr", lambda t: ctypes.c_void_p(t.data_ptr()))
    w = torch.zeros(4, 8)
    for args, kw in ((([],), {}), (([torch.zeros(8)],), {}), (([w.half()],), {}), (([w],), dict(masters=True)),
                     (([w],), dict(scale="big")), (([w],), dict(scale=[1.0, 2.0])),
                     (([w],), dict(weight_decay=[0.0, 0.1])), (([w],), dict(products=2)),
                     (([w],), dict(coefficients=[(1, 2)])), (([w],), dict(coefficients=[(1.0, 0, 0)] * 3)),
                     (([w],), dict(momentum_buffers=[w.double()])), (([w, w.bfloat16()],), {})):
        with pytest.raises((ValueError, TypeError)):
            r3.Muon(*args, **kw)
    for args, kw in (((w.half(),), {}), ((w[0],), {}), ((w,), dict(out_dtype=torch.float16)),
                     ((w, torch.zeros(8, 4)), {}), ((w,), dict(products=5)), ((w,), dict(coefficients=(1, 2)))):
        with pytest.raises(ValueError):
            r3.orthogonalize(*args, **kw)
