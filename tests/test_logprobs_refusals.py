"""What the log-probability calls refuse on the host: nothing is launched by anything here."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


FAKE = ctypes.c_void_p(4096)       # never dereferenced: the calls fail before any launch


def fwd(r3, s, logits=FAKE, ids=FAKE, logp=FAKE, ent=None, stats=None, n=0, tid=None, tlp=None):
    return r3.lib.r3_token_logprobs(ctypes.byref(s) if s else None, logits, ids, logp, ent, stats, n,
                                    tid, tlp, None, None)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(V=0), dict(V=-5), dict(ld=99), dict(dtype=2),
                                dict(id_bytes=2), dict(temperature=0.0), dict(temperature=-1.0),
                                dict(temperature=float("nan")), dict(temperature=float("inf")),
                                dict(temperature=1e-7), dict(temperature=1e21)])
def test_bad_shapes(r3, kw):
    base = dict(T=4, V=100, ld=100, dtype=0, id_bytes=8, temperature=1.0)
    base.update(kw)
    s = r3.Logits(**base)
    assert fwd(r3, s) == r3.R3_ERR_INVALID_ARG
    assert r3.lib.r3_token_logprobs_bwd(ctypes.byref(s), FAKE, FAKE, FAKE, None, FAKE, None, FAKE,
                                        128, None, None) == r3.R3_ERR_INVALID_ARG


def test_bad_arguments(r3):
    s = r3.Logits(4, 100, 100, 0, 8, 1.0)
    bad = r3.R3_ERR_INVALID_ARG
    assert fwd(r3, None) == bad
    assert fwd(r3, s, logits=None) == bad
    assert fwd(r3, s, logits=ctypes.c_void_p(4098)) == bad          # not a float's alignment
    assert fwd(r3, s, ids=ctypes.c_void_p(4100)) == bad             # not an int64's
    assert fwd(r3, s, ids=None) == bad                              # logp without ids
    assert fwd(r3, s, logp=None) == bad                             # nothing asked for
    assert fwd(r3, s, logp=ctypes.c_void_p(4098)) == bad            # not a float's alignment
    assert fwd(r3, s, ent=ctypes.c_void_p(4097)) == bad
    assert fwd(r3, s, n=3) == bad                                   # no room for the alternatives
    assert fwd(r3, s, n=-1) == bad
    assert fwd(r3, s, n=101, tid=FAKE, tlp=FAKE) == bad             # more than the vocabulary
    assert fwd(r3, s, n=33, tid=FAKE, tlp=FAKE) == r3.R3_ERR_UNSUPPORTED
    assert fwd(r3, r3.Logits(0, 100, 100, 0, 8, 1.0), logits=None, ids=None) == r3.R3_OK

    def bwd(logits=FAKE, ids=FAKE, stats=FAKE, ent=None, dlogp=FAKE, dent=None, out=FAKE, ld=100):
        return r3.lib.r3_token_logprobs_bwd(ctypes.byref(s), logits, ids, stats, ent, dlogp, dent,
                                            out, ld, None, None)
    assert bwd(logits=None) == bad and bwd(stats=None) == bad and bwd(out=None) == bad
    assert bwd(dlogp=None) == bad                                   # neither gradient
    assert bwd(ids=None) == bad                                     # dlogp without ids
    assert bwd(dent=FAKE) == bad                                    # dentropy without the entropy
    assert bwd(ld=99) == bad
    assert bwd(stats=ctypes.c_void_p(4098)) == bad and bwd(dlogp=ctypes.c_void_p(2)) == bad
    assert bwd(ld=128) == bad                                       # in place with another stride


def test_host_tensors_are_refused(r3):
    with pytest.raises(ValueError):
        r3.token_logprobs(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError):
        r3.token_logprobs([[0.0]], None)
