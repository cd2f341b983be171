"""The losses' oracle against differences of its own loss and against closed forms."""
import numpy as np
import pytest

from oracle import r3_loss_oracle as O


def inputs(seed=0, T=40):
    rng = np.random.default_rng(seed)
    old = -rng.random(T) * 4
    return rng, dict(logp=old + 0.3 * rng.standard_normal(T), logp_old=old,
                     logp_infer=old + 0.5 * rng.standard_normal(T),
                     logp_ref=old + 0.4 * rng.standard_normal(T), entropy=rng.random(T),
                     mask=rng.random(T) < 0.8, cu_seqlens=[0, 7, 7, 8, 30, 38])


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("reduce", ["token", "sequence"])
@pytest.mark.parametrize("per_sequence", [False, True])
@pytest.mark.parametrize("dual", [0.0, 1.3])
def test_policy_gradient_is_that_of_the_loss(ratio, reduce, per_sequence, dual):
    rng, kw = inputs()
    adv = rng.standard_normal(5).view(O.PerSequence) if per_sequence else rng.standard_normal(40)
    kw.update(advantages=adv, ratio=ratio, reduce=reduce, dual_clip=dual, kl_coef=0.3, entropy_coef=0.2,
              clip_low=0.05, clip_high=0.1)
    ref = O.policy_loss(**kw)
    h = 1e-6
    for name, grad in (("logp", "dlogp"), ("entropy", "dentropy")):
        for t in range(40):
            up, down = dict(kw), dict(kw)
            up[name], down[name] = kw[name].copy(), kw[name].copy()
            up[name][t] += h
            down[name][t] -= h
            slope = (O.policy_loss(**up)["loss"] - O.policy_loss(**down)["loss"]) / (2 * h)
            assert abs(slope - ref[grad][t]) < 1e-8
    assert (ref["dlogp"][38:] == 0).all() and (ref["dlogp"][~kw["mask"]] == 0).all()


def test_policy_closed_forms():
    z = np.zeros(4)
    ref = O.policy_loss(z, z, np.array([1.0, -2, 3, 0]), [0, 4])          # on policy: -A, gradient -A / N
    assert ref["loss"] == -0.5 and np.array_equal(ref["dlogp"], [-0.25, 0.5, -0.75, 0])
    logp = np.log([1.5, 1.5, 0.5, 0.5])
    ref = O.policy_loss(logp, z, np.array([1.0, -1, 1, -1]), [0, 4])
    assert np.allclose(ref["loss"], (-1.2 + 1.5 - 0.5 + 0.8) / 4)
    assert np.allclose(ref["dlogp"], [0, 1.5 / 4, -0.5 / 4, 0]) and ref["clipped"] == 2
    logp = np.log([4.0, 0.25])                                              # the geometric mean is 1
    ref = O.policy_loss(logp, z[:2], np.ones(2), [0, 2], ratio="sequence", reduce="sequence")
    assert np.allclose(ref["loss"], -1) and np.allclose(ref["dlogp"], -0.5)


def test_balance_gradient_is_that_of_the_loss():
    rng = np.random.default_rng(1)
    z, idx = rng.standard_normal((12, 7)), np.argsort(rng.random((12, 7)), 1)[:, :3]
    mask = rng.random(12) < 0.7
    ref = O.balance_loss(z, idx, mask, balance_coef=0.4, z_coef=0.1)
    for t in range(12):
        for e in range(7):
            up, down = z.copy(), z.copy()
            up[t, e] += 1e-6
            down[t, e] -= 1e-6
            a, b = O.balance_loss(up, idx, mask), O.balance_loss(down, idx, mask)
            slope = (0.4 * (a[0] - b[0]) + 0.1 * (a[1] - b[1])) / 2e-6
            assert abs(slope - ref[3][t, e]) < 1e-8


def test_balance_closed_forms():
    idx = np.arange(8).reshape(4, 2)
    balance, z, counts, d, *_ = O.balance_loss(np.zeros((4, 8)), idx)
    assert balance == 1.0 and np.allclose(z, np.log(8) ** 2) and (counts == 1).all() and np.allclose(d, 0)
    one = np.full((3, 4), -np.inf)
    one[:, 2] = 5.0
    balance, z, counts, *_ = O.balance_loss(one, np.full((3, 1), 2))        # all on one expert: E
    assert balance == 4.0 and z == 25.0 and counts[2] == 3
