"""What the AdamW step refuses on the host: nothing is launched by anything here."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


def call(r3, tensors=None, grad_scale=None, scalars=None, n=None, **kw):
    cfg = dict(param_dtype=0, grad_dtype=0, master=0, state_bits=32, step=1, lr=0.1, beta1=0.9,
               beta2=0.99, eps=1e-8)
    cfg.update(kw)
    if tensors is None:
        tensors = [{}]
    rows = []
    for i, t in enumerate(tensors):
        row = dict(param=(1 + 8 * i) << 20, master=None, grad=(2 + 8 * i) << 20, exp_avg=(3 + 8 * i) << 20,
                   exp_avg_sq=(4 + 8 * i) << 20, exp_avg_scale=None, exp_avg_sq_scale=None, n=100,
                   weight_decay=0.0)
        row.update(t)
        rows.append(r3.AdamWTensor(**row))
    table = (r3.AdamWTensor * max(1, len(rows)))(*rows)
    return r3.lib.r3_adamw_step(ctypes.byref(r3.AdamWConfig(**cfg)), table, len(rows) if n is None else n,
                                grad_scale, scalars, None)


@pytest.mark.parametrize("kw", [
    dict(param_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(master=1), dict(step=0),
    dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1),
    dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=-1e-8), dict(eps=float("inf")),
    dict(n=-1), dict(state_bits=8),                                       # no scales
    dict(param_dtype=1, master=1),                                        # no master buffer
    dict(tensors=[dict(master=9 << 20)]),                                 # a master that is not used
    dict(tensors=[dict(n=-5)]), dict(tensors=[dict(n=(1 << 40) + 1)]), dict(tensors=[dict(param=None)]),
    dict(tensors=[dict(grad=None)]), dict(tensors=[dict(exp_avg=None)]), dict(tensors=[dict(exp_avg_sq=None)]),
    dict(tensors=[dict(param=(1 << 20) + 8)]), dict(tensors=[dict(grad=(1 << 20) + 4)]),
    dict(tensors=[dict(weight_decay=-0.1)]), dict(tensors=[dict(weight_decay=float("nan"))]),
    dict(tensors=[{}, {}, dict(param=1 << 20)]),                          # the same tensor twice
    dict(tensors=[{}, dict(param=(1 << 20) + 384)]),                      # overlapping tensors
    dict(grad_scale=ctypes.c_void_p(4097)), dict(scalars=ctypes.c_void_p(4098)),
])
def test_refused(r3, kw):
    assert call(r3, **kw) == r3.R3_ERR_INVALID_ARG


A, B = 1 << 20, 100 * 4                                        # the first entry's param, its bytes


@pytest.mark.parametrize("kw", [
    dict(tensors=[{}, dict(exp_avg=3 << 20)]),                            # one state for two tensors
    dict(tensors=[{}, dict(exp_avg_sq=(4 << 20) + 384)]),
    dict(tensors=[dict(exp_avg_sq=3 << 20)]),                             # both states of a tensor
    dict(tensors=[dict(exp_avg=A + 16 * (B // 16 - 1))]),                 # the param's last elements
    dict(param_dtype=1, master=1, tensors=[dict(master=9 << 21), dict(master=9 << 21)]),
    dict(state_bits=8, tensors=[dict(exp_avg_scale=5 << 20, exp_avg_sq_scale=5 << 20)]),
    dict(state_bits=8, n=2, tensors=[dict(n=257, exp_avg_scale=5 << 20, exp_avg_sq_scale=6 << 20),
                                     dict(n=1, exp_avg_scale=(5 << 20) + 4, exp_avg_sq_scale=7 << 20)]),
])
def test_shared_memory_is_refused(r3, kw):
    assert call(r3, **kw) == r3.R3_ERR_INVALID_ARG


def test_null_and_nothing_to_do(r3):
    assert r3.lib.r3_adamw_step(None, None, 0, None, None, None) == r3.R3_ERR_INVALID_ARG
    assert call(r3, tensors=[]) == r3.R3_OK
    assert call(r3, tensors=[dict(n=0, param=None, grad=None)] * 3) == r3.R3_OK


def test_struct_layouts(r3):
    assert ctypes.sizeof(r3.AdamWTensor) == 72 and ctypes.sizeof(r3.AdamWConfig) == 56
    assert ctypes.sizeof(r3.Norm) == 32 and ctypes.sizeof(r3.Logits) == 32


def test_host_tensors_are_refused(r3):
    with pytest.raises(ValueError):
        r3.AdamW([torch.zeros(8)], [torch.zeros(8)])


@pytest.mark.parametrize("bad", ["size", "dtype", "layout", "device", "kind", "count"])
def test_refused_gradients_leave_the_handle_as_it_was(r3, monkeypatch, bad):
    """A list of gradients of which one is refused changes none of the handle's addresses, its list or its
    type (host tensors here: no step is taken)."""
    monkeypatch.setattr(r3, "_ptr", lambda t: ctypes.c_void_p(t.data_ptr()) if t.is_contiguous() else
                        (_ for _ in ()).throw(ValueError("tensor must be contiguous")))
    monkeypatch.setattr(r3, "_device_of", lambda name, t: t.device)
    params = [torch.zeros(8), torch.zeros(16)]
    old = [torch.zeros(8), torch.zeros(16)]
    opt = r3.AdamW(params, old)
    before = [row.grad for row in opt._table]
    assert before == [g.data_ptr() for g in old]
    new = [torch.zeros(8, dtype=torch.bfloat16), torch.zeros(16, dtype=torch.bfloat16)]
    new[1] = {"size": new[1][:4], "dtype": torch.zeros(16), "layout": torch.zeros(32, dtype=torch.bfloat16)[::2],
              "device": torch.zeros(16, dtype=torch.bfloat16, device="meta"), "kind": [0.0] * 16,
              "count": new[1]}[bad]
    with pytest.raises((ValueError, TypeError)):
        opt.set_grads(new[:1] if bad == "count" else new)
    assert [row.grad for row in opt._table] == before
    assert opt._config.grad_dtype == r3.R3_F32 and all(a is b for a, b in zip(opt.grads, old))
    new = [torch.ones(8, dtype=torch.bfloat16), torch.ones(16, dtype=torch.bfloat16)]
    opt.set_grads(new)
    assert [row.grad for row in opt._table] == [g.data_ptr() for g in new]
    assert opt._config.grad_dtype == r3.R3_BF16


FAR = 1 << 34


@pytest.mark.parametrize("kw", [
    dict(tensors=[dict(grad=A)]),                                         # a param as its own gradient
    dict(tensors=[dict(grad=3 << 20)]), dict(tensors=[dict(grad=4 << 20)]),
    dict(tensors=[dict(grad=A + 16 * (B // 16 - 1))]),                    # the last elements alone
    dict(tensors=[{}, dict(grad=A)]), dict(tensors=[dict(grad=9 << 20), {}]),       # another entry's param
    dict(tensors=[dict(param=FAR), dict(grad=3 << 20), {}]),              # lists that do not ascend
    dict(tensors=[dict(param=FAR), dict(grad=FAR)]),
    dict(param_dtype=1, master=1, tensors=[dict(master=9 << 20, grad=9 << 20)]),
    dict(state_bits=8, tensors=[dict(exp_avg_scale=5 << 20, exp_avg_sq_scale=6 << 20, grad=6 << 20)]),
    dict(grad_scale=ctypes.c_void_p(A + 396)), dict(scalars=ctypes.c_void_p(A + 396)),
    dict(grad_scale=ctypes.c_void_p((4 << 20) + 8)), dict(scalars=ctypes.c_void_p((4 << 20) - 8)),
])
def test_reading_what_is_written_is_refused(r3, kw):
    assert call(r3, **kw) == r3.R3_ERR_INVALID_ARG
