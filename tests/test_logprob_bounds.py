"""The bound that gradients to the logits are held to tells a wrong gradient at the vocabularies in use:
mistakes planted in the oracle's own gradient (on the CPU)."""
import numpy as np
import pytest

from oracle import r3_update_oracle as U
from tests.helpers import logits_gradient_bound


@pytest.mark.parametrize("V,temperature", [(50257, 1.0), (151936, 1.0), (50257, 0.6)])
def test_planted_mistakes_are_found(V, temperature):
    rng = np.random.default_rng(V)
    T = 3
    z = (rng.standard_normal((T, V)) * 2.5).astype(np.float32).astype(np.float64)
    z[:, 0] += 3.0
    ids = rng.integers(0, V, T)
    dlogp, dent = rng.standard_normal(T) + 2.0, rng.standard_normal(T) + 2.0
    for d in (None, dent):
        ref = U.token_logprobs_bwd(z, ids, dlogp, d, temperature)
        for eps in (2.0 ** -7, 2.0 ** -23):                         # bfloat16, float32
            bound = logits_gradient_bound(z, ids, dlogp, d, temperature, ref, eps)

            def wrong(got):
                return (np.abs(got - ref) > bound).mean()
            assert wrong(ref * (1 + eps / 2 - 2.0 ** -40)) == 0      # a rounding
            assert wrong(np.zeros_like(ref)) > 0.999                 # elements left out
            assert wrong(np.roll(ref, 1, axis=1)) > 0.9              # one place off
            # 1% off (but for elements next to a change of sign: log p near -H)
            assert wrong(1.01 * ref) > 0.98
            part = ref.copy()
            part[:, -5:] = 0                                         # the ragged end left out
            assert (np.abs(part - ref) > bound)[:, -5:].mean() > 0.99
        # the token's own term left out
        bare = ref.copy()
        bare[np.arange(T), ids] -= dlogp / temperature
        assert (np.abs(bare - ref) > bound).any(axis=1).all()
    # the entropy's term left out
    full = U.token_logprobs_bwd(z, ids, dlogp, dent, temperature)
    less = U.token_logprobs_bwd(z, ids, dlogp, None, temperature)
    bound = logits_gradient_bound(z, ids, dlogp, dent, temperature, full, 2.0 ** -7)
    assert (np.abs(full - less) > bound).mean() > 0.9
