"""Pins of oracle/r3_update_oracle.py: closed forms, brute force and central finite differences."""
import math

import numpy as np
import pytest

from oracle import r3_update_oracle as U


def fd(f, x, h=1e-6):
    """Central differences of the scalar f in every element of x."""
    g = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        keep = x[i]
        x[i] = keep + h
        hi = f()
        x[i] = keep - h
        lo = f()
        x[i] = keep
        g[i] = (hi - lo) / (2 * h)
    return g


def test_logprobs_closed_forms():
    # logits ln 1, ln 2, ln 5: probabilities 1/8, 2/8, 5/8
    z = np.log(np.array([[1.0, 2.0, 5.0]]))
    r = U.token_logprobs(z, [1], n_top=3)
    assert abs(r["logp"][0] - math.log(0.25)) < 1e-15
    h = -sum(p * math.log(p) for p in (0.125, 0.25, 0.625))
    assert abs(r["entropy"][0] - h) < 1e-15
    assert r["top_ids"].tolist() == [[2, 1, 0]]
    assert abs(r["stats"][0, 0] + r["stats"][0, 1] - math.log(8.0)) < 1e-15
    # temperature 1/2 squares the weights: 1/30, 4/30, 25/30
    r = U.token_logprobs(z, [1], temperature=0.5)
    assert abs(r["logp"][0] - math.log(4.0 / 30.0)) < 1e-15
    # uniform rows, whatever the level: log p = -ln V, entropy ln V
    for level in (0.0, -3e38, 88.0):
        r = U.token_logprobs(np.full((1, 7), level), [3], n_top=2)
        assert abs(r["logp"][0] + math.log(7)) < 1e-15 and abs(r["entropy"][0] - math.log(7)) < 1e-14
        assert r["top_ids"].tolist() == [[0, 1]]


def test_logprobs_special_rows():
    z = np.array([[0.0, 1.0, -np.inf], [-np.inf] * 3, [0.0, np.nan, 0.0], [0.0, np.inf, 0.0],
                  [1.0, 2.0, 3.0]])
    r = U.token_logprobs(z, [2, 0, 0, 0, -1], n_top=2)
    assert r["logp"][0] == -np.inf and np.isfinite(r["entropy"][0])
    assert r["logp"][1] == -np.inf and r["entropy"][1] == 0 and r["top_ids"][1].tolist() == [0, 1]
    assert np.isnan(r["logp"][2]) and np.isnan(r["entropy"][3]) and r["top_ids"][3].tolist() == [-1, -1]
    assert r["logp"][4] == 0 and r["top_ids"][4].tolist() == [-1, -1]


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_logprobs_gradient_by_differences(temperature):
    rng = np.random.default_rng(3)
    z = rng.normal(size=(4, 9)) * 2
    ids = np.array([0, 8, -1, 3])
    dl, de = rng.normal(size=4), rng.normal(size=4)

    def loss():
        r = U.token_logprobs(z, ids, temperature)
        return float((dl * r["logp"] + de * r["entropy"]).sum())

    g = U.token_logprobs_bwd(z, ids, dl, de, temperature)
    assert np.abs(g - fd(loss, z)).max() < 1e-8
    assert np.abs(g.sum(1)).max() < 1e-13            # the softmax does not see a common shift
    assert not g[2].any()


# ---- norms around a block ------------------------------------------------------------------------
def test_norm_closed_forms():
    # a row of equal magnitudes a has rms a: the norm gives its signs
    y = np.array([[3.0, -3.0, 3.0, 3.0], [0.0, 0.0, 0.0, 0.0]])
    w = np.array([1.0, 2.0, 3.0, 4.0])
    assert np.allclose(U.rms_norm(y, w, 1e-300)[0], [1, -2, 3, 4], rtol=0, atol=1e-15)
    assert not U.rms_norm(y, w, 1e-6)[1].any()
    x = np.ones((2, 4))
    x_out, h = U.norm_residual(x, y, w_post=np.ones(4), gate=np.array([[0.5], [2.0]]), eps=1e-300,
                               residual_scale=2.0, branch_scale=4.0)
    assert np.allclose(x_out[0], [4, 0, 4, 4], rtol=0, atol=1e-14) and np.allclose(x_out[1], 2.0)
    assert h is None
    none, h = U.norm_residual(x * 5, None, w_pre=w, eps=1e-300)
    assert none is None and np.allclose(h, np.stack([w, w]), rtol=0, atol=1e-14)


@pytest.mark.parametrize("kind", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_norm_gradients_by_differences(kind, post, pre):
    rng = np.random.default_rng(5)
    T, d = 3, 8
    x, y = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    p = dict(w_post=1 + 0.3 * rng.normal(size=d) if post else None,
             w_pre=1 + 0.3 * rng.normal(size=d) if pre else None,
             gate={"none": None, "channel": rng.normal(size=d), "token": rng.normal(size=(T, 1)),
                   "full": rng.normal(size=(T, d))}[kind])
    kw = dict(eps=0.1, residual_scale=1.3, branch_scale=0.7)
    a, b = rng.normal(size=(T, d)), rng.normal(size=(T, d))

    def loss():
        x_out, h = U.norm_residual(x, y, **p, **kw)
        return float((a * x_out).sum() + ((b * h).sum() if pre else 0.0))

    x_out = U.norm_residual(x, y, **p, **kw)[0]
    g = U.norm_residual_bwd(x_out, y, a, b if pre else None, **p, **kw)
    for name, v in (("dx", x), ("dy", y), ("dw_post", p["w_post"]), ("dw_pre", p["w_pre"]),
                    ("dgate", p["gate"])):
        if v is None:
            assert name not in g
        else:
            assert g[name].shape == v.shape and np.abs(g[name] - fd(loss, v)).max() < 1e-8, name


def test_norm_gradient_in_front_of_the_first_block():
    rng = np.random.default_rng(6)
    x, w, b = rng.normal(size=(3, 8)), rng.normal(size=8), rng.normal(size=(3, 8))
    g = U.norm_residual_bwd(x, None, None, b, w_pre=w, eps=0.1)

    def loss():
        return float((b * U.norm_residual(x, None, w_pre=w, eps=0.1)[1]).sum())
    assert np.abs(g["dx"] - fd(loss, x)).max() < 1e-8 and np.abs(g["dw_pre"] - fd(loss, w)).max() < 1e-8


# ---- AdamW ----------------------------------------------------------------------------------------
def test_adamw_closed_forms():
    # first step from zero states: m-hat = g, v-hat = g^2, so the step is lr sign(g) (eps aside)
    w, m, v = U.adamw(np.array([1.0, 2.0]), np.array([3.0, -4.0]), 0.0, 0.0, 1, 0.1, (0.9, 0.99), 0.0, 0.0)
    assert np.allclose(w, [0.9, 2.1], rtol=0, atol=1e-14)
    assert np.allclose(m, [0.3, -0.4]) and np.allclose(v, [0.09, 0.16])
    # a zero gradient leaves the decay alone
    w, _, _ = U.adamw(np.array([1.0]), np.array([0.0]), 0.0, 0.0, 1, 0.1, (0.9, 0.99), 1e-8, 0.5)
    assert abs(w[0] - 0.95) < 1e-15


def test_adamw_agrees_with_torch():
    import torch
    g = torch.Generator().manual_seed(0)
    p = torch.randn(50, generator=g, dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.8, 0.9), eps=1e-6, weight_decay=0.3)
    w, m, v = p.detach().numpy().copy(), 0.0, 0.0
    for step in range(1, 6):
        p.grad = torch.randn(50, generator=g, dtype=torch.float64)
        w, m, v = U.adamw(w, p.grad.numpy(), m, v, step, 0.01, (0.8, 0.9), 1e-6, 0.3)
        opt.step()
        assert np.abs(w - p.detach().numpy()).max() < 1e-14


def test_e4m3_values_and_scales():
    import torch
    vals = U.e4m3_values()
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    assert np.array_equal(vals, codes.double().numpy()) and vals[-1] == 448.0 and vals[1] == U.E4M3_MIN
    rng = np.random.default_rng(1)
    q = np.concatenate([rng.uniform(-448, 448, 5000), vals, -vals, (vals[1:] + vals[:-1]) / 2,
                        2.0 ** rng.uniform(-14, 8, 5000)]).astype(np.float32)
    want = torch.from_numpy(q).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(U.nearest_e4m3(q), want)
    for top, scale in ((448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -126)):
        assert U.block_scale(np.array([[0.0, -top]]))[0] == scale


# ---- stacks with norms --------------------------------------------------------------------------------
@pytest.mark.parametrize("post,gated", [(True, True), (False, False), (True, False)])
def test_normed_stack_gradients_by_differences(post, gated):
    rng = np.random.default_rng(9)
    T, d, E, K, F, L = 3, 8, 4, 2, 8, 2
    x0, dy = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    layers = [[rng.normal(size=(E, d)) * 0.5, np.argsort(rng.random((T, E)), axis=1)[:, :K],
               rng.normal(size=(E, F, d)) * 0.5, rng.normal(size=(E, F, d)) * 0.5,
               rng.normal(size=(E, d, F)) * 0.5] for _ in range(L)]
    norms = [(1 + 0.3 * rng.normal(size=d), 1 + 0.3 * rng.normal(size=d) if post else None,
              rng.normal(size=d) if gated else None) for _ in range(L)]
    kw = dict(eps=0.05, residual_scale=0.9, branch_scale=0.6)

    def loss():
        return float((dy * U.normed_stack_bwd(x0, layers, norms, dy, **kw)["x_out"]).sum())

    g = U.normed_stack_bwd(x0, layers, norms, dy, expert_grads=True, **kw)
    assert np.abs(g["dx0"] - fd(loss, x0)).max() < 1e-7
    for l in range(L):
        assert np.abs(g["dw_r"][l] - fd(loss, layers[l][0])).max() < 1e-7
        assert np.abs(g["dw_pre"][l] - fd(loss, norms[l][0])).max() < 1e-7
        if post:
            assert np.abs(g["dw_post"][l] - fd(loss, norms[l][1])).max() < 1e-7
        if gated:
            assert np.abs(g["dgate"][l] - fd(loss, norms[l][2])).max() < 1e-7
        down = np.stack([g["dw_experts"][l][e][2] for e in range(E)])
        assert np.abs(down - fd(loss, layers[l][4])).max() < 1e-7


def test_normed_stack_without_blocks_output_is_the_residual_alone():
    rng = np.random.default_rng(2)
    x0, dy = rng.normal(size=(3, 8)), rng.normal(size=(3, 8))
    layers = [[rng.normal(size=(4, 8)), np.argsort(rng.random((3, 4)), axis=1)[:, :2],
               rng.normal(size=(4, 8, 8)), rng.normal(size=(4, 8, 8)), np.zeros((4, 8, 8))]] * 2
    g = U.normed_stack_bwd(x0, layers, [(np.ones(8), None, None)] * 2, dy, residual_scale=0.5)
    assert np.allclose(g["x_out"], 0.25 * x0) and np.allclose(g["dx0"], 0.25 * dy)
