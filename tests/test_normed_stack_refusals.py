"""What the normed-stack calls refuse on the host: nothing is launched by anything here."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


P = [ctypes.c_void_p(i << 20) for i in range(1, 24)]           # never dereferenced
T, D, E, K, F, L = 16, 64, 4, 2, 64, 2


def norms(r3, **kw):
    base = dict(w_pre=1 << 30, w_post=2 << 30, gate=None, dw_pre=3 << 30, dw_post=4 << 30, dgate=None,
                w_dtype=0, eps=1e-6, residual_scale=1.0, branch_scale=1.0)
    base.update(kw)
    return r3.BlockNorms(**base)


def fwd(r3, n=None, s=None, layers=L, ws=None, size=0, drop=None):
    s = s if s is not None else r3.make_shape(T, D, E, K, F)
    a = [None if i == drop else P[i] for i in range(7)]
    n = norms(r3) if n is None else n
    return r3.lib.r3_normed_stack(ctypes.byref(s), layers, ctypes.byref(n), *a, ws, size, None, None)


def train(r3, n=None, s=None, layers=L, adamw=None, states=None, grads=True, drop=None, ws=None, size=0):
    s = s if s is not None else r3.make_shape(T, D, E, K, F)
    n = norms(r3) if n is None else n
    a = [None if i == drop else P[i] for i in range(14)]
    if not grads:
        a[11] = a[12] = a[13] = None
    return r3.lib.r3_normed_stack_train(
        ctypes.byref(s), layers, ctypes.byref(n), *a, ctypes.addressof(adamw) if adamw else None,
        ctypes.addressof(states) if states is not None else None, None, None, ws, size, None, None)


@pytest.mark.parametrize("kw", [dict(w_pre=None), dict(w_pre=(1 << 30) + 4), dict(w_post=8), dict(w_dtype=3),
                                dict(eps=0.0), dict(eps=float("nan")), dict(residual_scale=float("inf")),
                                dict(branch_scale=float("nan"))])
def test_bad_norms(r3, kw):
    assert fwd(r3, norms(r3, **kw)) == r3.R3_ERR_INVALID_ARG
    assert train(r3, norms(r3, **kw)) == r3.R3_ERR_INVALID_ARG


def test_bad_gradients_and_sizes(r3):
    bad = r3.R3_ERR_INVALID_ARG
    for kw in (dict(dw_pre=None), dict(dw_post=None), dict(w_post=None), dict(dgate=5 << 30), dict(gate=5 << 30)):
        assert train(r3, norms(r3, **kw)) == bad
    assert fwd(r3, layers=0) == bad and train(r3, layers=-1) == bad
    wide = r3.make_shape(T, 16392, E, K, F)
    assert fwd(r3, s=wide) == r3.R3_ERR_UNSUPPORTED and train(r3, s=wide) == r3.R3_ERR_UNSUPPORTED
    import torch
    assert train(r3, s=r3.make_shape(T, D, E, K, F, act=torch.float32)) == r3.R3_ERR_UNSUPPORTED
    for i in range(7):
        assert fwd(r3, drop=i) == bad, i
    for i in range(14):
        assert train(r3, drop=i) == bad, i
    assert fwd(r3) == r3.R3_ERR_WORKSPACE and train(r3) == r3.R3_ERR_WORKSPACE
    assert train(r3, grads=False) == r3.R3_ERR_WORKSPACE                 # legal without expert gradients
    none = r3.make_shape(0, D, E, K, F)
    assert fwd(r3, s=none) == r3.R3_OK and train(r3, s=none) == r3.R3_OK


def test_bad_optimisers(r3):
    bad = r3.R3_ERR_INVALID_ARG
    block = E * F * D

    def states(**kw):
        rows = []
        for l in range(L):
            for k in range(3):
                at = (4 + k << 20) + l * block * 2
                row = dict(param=at, master=None, grad=None, exp_avg=(40 + 3 * l + k) << 24,
                           exp_avg_sq=(60 + 3 * l + k) << 24, exp_avg_scale=None, exp_avg_sq_scale=None,
                           n=block, weight_decay=0.0)
                row.update(kw)
                rows.append(r3.AdamWTensor(**row))
        return (r3.AdamWTensor * len(rows))(*rows)

    def config(**kw):
        base = dict(param_dtype=1, grad_dtype=0, master=0, state_bits=32, step=1, lr=0.1, beta1=0.9, beta2=0.99,
                    eps=1e-8)
        base.update(kw)
        return r3.AdamWConfig(**base)

    assert train(r3, adamw=config(), states=states()) == r3.R3_ERR_WORKSPACE       # all right but the workspace
    assert train(r3, adamw=config(), states=None) == bad
    assert train(r3, adamw=config(), states=states(), grads=False) == bad
    assert train(r3, adamw=config(param_dtype=0), states=states()) == bad
    assert train(r3, adamw=config(grad_dtype=1), states=states()) == bad
    assert train(r3, adamw=config(step=0), states=states()) == bad
    assert train(r3, adamw=config(state_bits=8), states=states()) == bad            # no scales
    assert train(r3, adamw=config(), states=states(n=block - 8)) == bad
    assert train(r3, adamw=config(), states=states(param=1 << 28)) == bad           # not the block's weights
    assert train(r3, adamw=config(), states=states(exp_avg=None)) == bad

    shared = states()
    shared[3].exp_avg = shared[0].exp_avg                                           # another block's state
    assert train(r3, adamw=config(), states=shared) == bad


def test_the_binding_checks_every_layers_tensors(r3, monkeypatch):
    """Routers, records and expert weights of another type than the shape says, or with fewer layers, would
    be read as raw bytes, past their ends: refused before the library is called (a stand-in here)."""
    import torch
    calls = []

    class Library:
        def __getattr__(self, name):
            def call(*a):
                calls.append(name)
                return 0
            return call
    monkeypatch.setattr(r3, "lib", Library())
    monkeypatch.setattr(r3, "_device_of", lambda name, t: t.device)
    monkeypatch.setattr(r3, "_ptr", lambda t, host=False: None if t is None else ctypes.c_void_p(t.data_ptr()))
    monkeypatch.setattr(r3, "_stream", lambda stream=None: None)
    s = r3.make_shape(T, D, E, K, F)
    bf = torch.bfloat16
    x = torch.zeros((T, D), dtype=bf)
    w_pre = torch.ones((L, D))
    good = dict(w_router=torch.zeros((L, E, D)), idx=torch.zeros((L, T, K), dtype=torch.uint8),
                w_gate=torch.zeros((L, E, F, D), dtype=bf), w_up=torch.zeros((L, E, F, D), dtype=bf),
                w_down=torch.zeros((L, E, D, F), dtype=bf))
    bad = [dict(idx=good["idx"].to(torch.int16)), dict(idx=good["idx"].to(torch.int64)),
           dict(w_router=good["w_router"].to(bf)), dict(w_gate=good["w_gate"].float()),
           dict(w_router=None), dict(w_up=good["w_up"].transpose(2, 3)),
           dict(w_down=good["w_down"].to("meta"))]
    bad += [{k: good[k][:1]} for k in good] + [{k: torch.cat([good[k]] * 2)} for k in good]
    for kw in bad:
        with pytest.raises((ValueError, TypeError)):
            r3.normed_stack(s, L, x, **{**good, **kw}, w_pre=w_pre)
        with pytest.raises((ValueError, TypeError)):
            r3.normed_stack_train(s, L, x, **{**good, **kw}, dy=x, w_pre=w_pre)
    assert not [c for c in calls if not c.endswith("_bytes")]
    r3.normed_stack(s, L, x, **good, w_pre=w_pre)
    r3.normed_stack_train(s, L, x, **good, dy=x, w_pre=w_pre)
    assert [c for c in calls if not c.endswith("_bytes")] == ["r3_normed_stack", "r3_normed_stack_train"]


def test_random_layouts_against_every_pair(r3):
    """States of small blocks at random places (in order, list by list, interleaved or overlapping) and three
    gradients among them: refused exactly where a written buffer meets another buffer.  What is not refused
    gets as far as the workspace, which is missing."""
    import random
    rng = random.Random(3)
    s = r3.make_shape(16, 8, 1, 1, 8)
    n = 64                                                               # elements of a block's weight
    found = {True: 0, False: 0}
    for trial in range(1500):
        layers, bits, master = rng.choice([1, 2, 3, 4, 12, 30]), rng.choice([8, 32]), rng.random() < 0.4
        count = 3 * layers
        fields = ["exp_avg", "exp_avg_sq"] + (["master"] if master else [])
        fields += ["exp_avg_scale", "exp_avg_sq_scale"] if bits == 8 else []
        size = dict(exp_avg=n * bits // 8, exp_avg_sq=n * bits // 8, master=4 * n, exp_avg_scale=4,
                    exp_avg_sq_scale=4)
        keys = [(i, f) for i in range(count) for f in fields] + [(i, "grad") for i in range(3)]
        if rng.random() < 0.5:                                           # list by list
            keys.sort(key=lambda k: (k[1], k[0]))
        places = rng.sample(range(1, rng.choice([len(keys) + 8, 10 * len(keys), 4000])), len(keys))
        if rng.random() < 0.6:
            places.sort()
        unit = rng.choice([128, 256, 256])
        at = {k: (1 << 30) + p * unit for k, p in zip(keys, places)}
        weights = [(1 << 29) + k * 4096 for k in range(3)]
        if rng.random() < 0.3:                                           # the weights among the states
            weights[rng.randrange(3)] = (1 << 30) + rng.randrange(max(places) + 1) * unit
        written = [(at[i, f], size[f]) for i in range(count) for f in fields]
        written += [(weights[i % 3] + i // 3 * 2 * n, 2 * n) for i in range(count)]
        read = [(at[k, "grad"], 4 * n) for k in range(3)]
        scale = (1 << 30) + rng.randrange(max(places) + 1) * unit + 64 if rng.random() < 0.2 else None
        if scale:
            read.append((scale, 4))
        rows = [r3.AdamWTensor(param=weights[i % 3] + i // 3 * 2 * n, n=n, weight_decay=0.0,
                               **{f: at[i, f] for f in fields}) for i in range(count)]
        table = (r3.AdamWTensor * count)(*rows)
        config = r3.AdamWConfig(param_dtype=1, grad_dtype=0, master=int(master), state_bits=bits, step=1, lr=0.1,
                                beta1=0.9, beta2=0.99, eps=1e-8)
        a = P[:3] + [ctypes.c_void_p(w) for w in weights] + P[6:11]
        a += [ctypes.c_void_p(at[k, "grad"]) for k in range(3)]
        got = r3.lib.r3_normed_stack_train(
            ctypes.byref(s), layers, ctypes.byref(norms(r3)), *a, ctypes.addressof(config),
            ctypes.addressof(table), ctypes.c_void_p(scale) if scale else None, None, None, 0, None, None)

        def meet(p, q):
            return p[0] < q[0] + q[1] and q[0] < p[0] + p[1]
        bad = any(meet(p, q) for i, p in enumerate(written) for q in written[:i] + read)
        found[bad] += 1
        assert got == (r3.R3_ERR_INVALID_ARG if bad else r3.R3_ERR_WORKSPACE), (trial, bad, got)
    assert min(found.values()) > 200, found
