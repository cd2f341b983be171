"""Sizes at the ends of what the Update step's losses take, on the host: nothing is launched by anything here."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


def balance(r3, T, ws_bytes):
    """Addresses that nothing stands behind: the call has to end at its checks."""
    s, c = r3.make_shape(T, 8, 1, 1, 8), r3.Balance(1.0, 0.0, 0, 0)
    code = r3.lib.r3_balance_loss(s, 1, ctypes.byref(c), 1 << 40, 2 << 40, None, None, 3 << 40, 4 << 40, 5 << 40,
                                  ws_bytes, None, None)
    return code, r3.lib.r3_balance_loss_workspace_bytes(s, 1)


def test_balance_tokens_whose_numbers_would_pass_32_bits(r3):
    for T in ((1 << 30) + 1, (1 << 31) - 1):
        assert balance(r3, T, 1 << 40) == (r3.R3_ERR_UNSUPPORTED, 0)
    code, need = balance(r3, 1 << 30, 0)
    assert code == r3.R3_ERR_WORKSPACE and need > 0
