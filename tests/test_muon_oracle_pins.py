"""The orthogonalised update's oracle against the singular value decomposition: the iteration acts on
singular values alone."""
import numpy as np
import pytest

from oracle import r3_muon_oracle as O


def scalar(s, steps=5, coefs=None):
    for k in range(steps):
        a, b, c = O.QUINTIC if coefs is None else coefs[k]
        s = a * s + b * s ** 3 + c * s ** 5
    return s


@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (7, 1), (5, 5), (12, 30), (30, 12)])
def test_iteration_acts_on_singular_values(shape):
    x = np.random.default_rng(0).standard_normal(shape)
    U, s, V = np.linalg.svd(x, full_matrices=False)
    want = (U * scalar(s / (np.sqrt((s ** 2).sum()) + 1e-7))) @ V
    assert np.allclose(O.iterate(x), want, atol=1e-12)
    coefs = [(2.0, -1.5, 0.5)] * 12
    assert np.allclose(O.iterate(x, 12, coefs), (U * scalar(s / (np.sqrt((s ** 2).sum()) + 1e-7), 12, coefs)) @ V)


def test_singular_values_end_near_one():
    x = np.random.default_rng(1).standard_normal((64, 200))
    s = np.linalg.svd(O.iterate(x), compute_uv=False)
    assert s.min() > 0.6 and s.max() < 1.3
    assert not O.iterate(np.zeros((3, 4))).any()


def test_fp16_operands_lose_no_more_than_a_bf16_result():
    """The claim behind one fp16 product with X carried in full: the error stays near that of rounding the
    result to bf16 (2^-9 / sqrt(3) of an element's magnitude, 1.7e-3 measured), whatever the spectrum."""
    rng = np.random.default_rng(2)
    U, _, V = np.linalg.svd(rng.standard_normal((96, 256)), full_matrices=False)
    for s in (np.ones(96), np.exp(-np.arange(96) / 12.0), np.where(np.arange(96) < 4, 1.0, 1e-4)):
        x = (U * s) @ V
        want = O.iterate(x)
        err = np.sqrt(((O.iterate(x, operand=O.half_operand) - want) ** 2).mean() / (want ** 2).mean())
        assert err < 4e-3


def test_step_by_hand():
    w, m = O.step(np.full((1, 1), 2.0), np.full((1, 1), 3.0), np.full((1, 1), 4.0), lr=0.1, momentum=0.5,
                  decay=0.2, scale=3.0, grad_scale=0.5)
    assert m[0, 0] == 3.5                                     # 0.5 * 3 + 2; the direction is its sign
    assert np.isclose(w[0, 0], 2.0 * 0.98 - 0.3 * scalar(1.0 / (1 + 1e-7 / 3.75)))
