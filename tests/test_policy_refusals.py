"""What the policy loss and the balance loss refuse on the host: nothing is launched by anything here."""
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


def policy(r3, **kw):
    cfg = dict(T=100, S=2, ratio=0, reduce=0, adv_per_token=1, clip_low=0.2, clip_high=0.2, dual_clip=0.0,
               infer_cap=2.0, kl_coef=0.0, entropy_coef=0.0, denominator=0.0)
    at = dict(logp=1 << 20, old=2 << 20, adv=3 << 20, cu=4 << 20, mask=None, infer=None, ref=None,
              entropy=None, dloss=None, loss=5 << 20, dlogp=6 << 20, dentropy=None, metrics=7 << 20,
              counts=8 << 20, ws=9 << 20, ws_bytes=1 << 20, status=None)
    for k, v in kw.items():
        (cfg if k in cfg else at)[k] = v
    return r3.lib.r3_policy_loss(ctypes.byref(r3.Policy(**cfg)), *at.values(), None)


@pytest.mark.parametrize("kw", [
    dict(T=-1), dict(S=-1), dict(T=(1 << 30) + 1), dict(S=(1 << 28) + 1), dict(ratio=2), dict(reduce=-1),
    dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=math.nan), dict(clip_high=-0.1),
    dict(clip_high=math.nan), dict(dual_clip=1.0), dict(dual_clip=-2.0), dict(dual_clip=math.nan),
    dict(infer_cap=0.0), dict(infer_cap=math.nan), dict(kl_coef=math.inf), dict(kl_coef=math.nan),
    dict(entropy_coef=math.nan), dict(denominator=-1.0), dict(denominator=math.inf),
    dict(denominator=math.nan), dict(logp=None), dict(old=None), dict(adv=None), dict(loss=None),
    dict(cu=None), dict(cu=None, S=0), dict(dentropy=10 << 20), dict(logp=(1 << 20) + 2),
    dict(dlogp=(6 << 20) + 1), dict(loss=(5 << 20) + 2), dict(cu=(4 << 20) + 1), dict(status=4097),
])
def test_policy_refused(r3, kw):
    assert policy(r3, **kw) == r3.R3_ERR_INVALID_ARG


def test_policy_workspace(r3):
    for kw in (dict(ws=None), dict(ws=(9 << 20) + 128), dict(ws_bytes=255)):
        assert policy(r3, **kw) == r3.R3_ERR_WORKSPACE
    bad = r3.Policy(T=-1, S=1, infer_cap=1.0)
    assert r3.lib.r3_policy_loss_workspace_bytes(ctypes.byref(bad)) == 0
    assert r3.lib.r3_policy_loss_workspace_bytes(None) == 0
    assert r3.lib.r3_policy_loss(None, *[None] * 15, 0, None, None) == r3.R3_ERR_INVALID_ARG


def balance(r3, shape=None, L=2, **kw):
    cfg = dict(balance_coef=1.0, z_coef=0.0, accumulate=0, counts_given=0)
    at = dict(logits=1 << 20, idx=2 << 20, mask=None, counts=3 << 20, loss=4 << 20, dlogits=5 << 20,
              ws=6 << 20, ws_bytes=1 << 24, status=None)
    for k, v in kw.items():
        (cfg if k in cfg else at)[k] = v
    s = shape or r3.make_shape(64, 8, 16, 2, 8)
    return r3.lib.r3_balance_loss(ctypes.byref(s), L, ctypes.byref(r3.Balance(**cfg)), *at.values(), None)


@pytest.mark.parametrize("kw", [
    dict(L=-1), dict(L=65536), dict(balance_coef=math.nan), dict(z_coef=math.inf), dict(logits=None),
    dict(idx=None), dict(loss=None), dict(counts=None, counts_given=1), dict(accumulate=1, dlogits=None),
    dict(logits=(1 << 20) + 8), dict(idx=(2 << 20) + 8), dict(dlogits=(5 << 20) + 8),
    dict(counts=(3 << 20) + 2), dict(loss=(4 << 20) + 2), dict(status=4097),
])
def test_balance_refused(r3, kw):
    assert balance(r3, **kw) == r3.R3_ERR_INVALID_ARG


def test_balance_shapes_and_workspace(r3):
    i16 = torch.int16
    assert balance(r3, r3.make_shape(64, 8, 300, 2, 8)) == r3.R3_ERR_INVALID_ARG       # uint8 record
    assert balance(r3, r3.make_shape(64, 8, 1025, 2, 8, idx=i16)) == r3.R3_ERR_UNSUPPORTED
    assert balance(r3, r3.make_shape(64, 8, 4, 5, 8)) == r3.R3_ERR_INVALID_ARG         # K > E
    assert balance(r3, r3.make_shape(-1, 8, 4, 2, 8)) == r3.R3_ERR_INVALID_ARG
    for kw in (dict(ws=None), dict(ws=(6 << 20) + 64), dict(ws_bytes=16)):
        assert balance(r3, **kw) == r3.R3_ERR_WORKSPACE
    assert balance(r3, L=0) == r3.R3_OK
    assert r3.lib.r3_balance_loss(None, 1, None, *[None] * 7, 0, None, None) == r3.R3_ERR_INVALID_ARG


def test_struct_layouts(r3):
    assert ctypes.sizeof(r3.Policy) == 80 and ctypes.sizeof(r3.Balance) == 24


def test_binding_refuses(r3, monkeypatch):
    monkeypatch.setattr(r3, "_device_of", lambda name, t: t.device)
    x, s = torch.zeros(8), r3.make_shape(4, 8, 8, 2, 8)
    cu = torch.tensor([0, 8], dtype=torch.int32)
    for kw in (dict(), dict(advantages=x, seq_advantages=x[:1]), dict(advantages=x[:4]),
               dict(seq_advantages=x), dict(advantages=x.double()), dict(advantages=x, mask=x),
               dict(advantages=x, ratio="word"), dict(advantages=x, reduce=None),
               dict(advantages=x, logp_infer=x[::2]), dict(advantages=x, dloss=torch.ones(2)),
               dict(advantages=x, entropy=x.bfloat16())):
        with pytest.raises(ValueError):
            r3.policy_loss(x, x, cu, **kw)
    with pytest.raises(ValueError):
        r3.policy_loss(x.view(2, 4), x.view(2, 4), cu, advantages=x)
    with pytest.raises(ValueError):
        r3.policy_loss(x, x, cu.long(), advantages=x)
    z, idx = torch.zeros(1, 4, 8), torch.zeros(1, 4, 2, dtype=torch.uint8)
    for args, kw in (((z,), {}), ((z[0], idx), {}), ((z, idx.short()), {}), ((z, idx[:, :2]), {}),
                     ((z, idx), dict(accumulate=True)), ((z, idx), dict(mask=torch.ones(3, dtype=torch.bool))),
                     ((z,), dict(counts=torch.zeros(1, 8))), ((z, idx), dict(dlogits=z.bfloat16()))):
        with pytest.raises(ValueError):
            r3.balance_loss(s, 1, *args, **kw)
