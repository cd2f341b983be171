"""The oracle's models of what the orthogonalised update's number formats lose: without the loss they are the iteration,
and what two planes hold is what the header says."""
import numpy as np
import pytest

from oracle import r3_muon_oracle as O


@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (7, 3), (12, 30), (40, 40)])
@pytest.mark.parametrize("steps", [1, 5, 9])
def test_models_without_their_loss(shape, steps):
    x = np.random.default_rng(3).standard_normal(shape)
    want = O.iterate(x, steps)
    assert np.allclose(O.iterate_planes(x, steps, split=lambda v: (v, 0 * v)), want, rtol=0, atol=1e-11)
    assert np.allclose(O.iterate_short(x, steps, part=0.0), want, rtol=0, atol=1e-11)
    assert np.allclose(O.iterate(x, steps, operand=lambda v: v), want, rtol=0, atol=1e-11)
    assert 0 < np.abs(O.iterate_f32(x, steps) - want).max() < 1e-4


def test_two_planes_hold_22_bits_down_to_small_elements():
    rng = np.random.default_rng(4)
    for scale, small, within in ((2.0 ** 14, 2.0 ** -28, 2.0 ** -50), (2.0 ** 10, 2.0 ** -24, 2.0 ** -46)):
        x = rng.choice([-1, 1], 20000) * 10.0 ** rng.uniform(-16, 0, 20000) * 3.4
        hi, lo = O.planes(x, scale)
        off = np.abs(hi + lo - x)
        assert (off <= np.where(np.abs(x) >= small, 2.0 ** -22 * np.abs(x), within)).all()
        one = np.abs(O.scaled_operand(x, scale) - x)
        assert (one <= np.where(np.abs(x) >= small, 2.0 ** -11 * np.abs(x), within * 2.0 ** 11)).all()
