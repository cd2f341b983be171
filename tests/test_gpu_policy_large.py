"""The policy loss on batches of more units than warps are resident (each warp takes several), on units longer than
128 tokens, and with bounds of sequences that make no sense.  Bounds and oracle: test_gpu_policy's."""
import ctypes

import numpy as np
import pytest
import torch

from tests.test_gpu_policy import call, check, lengths, make, oracle

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def runs(ratio):
    beyond = dict(clip_low=0.01, clip_high=0.02) if ratio == "sequence" else dict(clip_low=0.2, clip_high=0.28)
    return dict(ratio=ratio, dual_clip=1.5, infer_cap=1.3, kl_coef=0.1, entropy_coef=0.01, **beyond)


def many(seed):
    """Short responses around one of 20000 tokens (more than 64 units, each of which a CTA shares) and empty ones."""
    rng = np.random.default_rng(seed)
    n = np.concatenate([rng.integers(0, 25, 4600), [20000], rng.integers(0, 25, 600), [9000, 0, 0, 8500]])
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("reduce", ["token", "sequence"])
def test_more_units_than_warps(r3, ratio, reduce):
    for cu in (many(1), lengths(70000, 8192, 2)):
        T = int(cu[-1])
        for seed, kw in enumerate([dict(per_sequence=True, infer=True, ref=True, entropy=True, mask=0.3), dict(infer=True)]):
            t = make(T, cu, seed, **kw)
            args = dict(reduce=reduce, **runs(ratio))
            out = call(r3, t, cu, **args)
            check(out, t, oracle(t, cu, **args))
            bare = call(r3, t, cu, want_grad=False, **args)
            assert torch.equal(bare[0], out[0]) and torch.equal(bare[4], out[4])


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("reduce", ["token", "sequence"])
@pytest.mark.parametrize("T,S", [(300001, 3), (1000003, 900)])
def test_units_of_more_than_128_tokens(r3, ratio, reduce, T, S):
    cu = lengths(T, S, 4)
    t = make(T, cu, 2, per_sequence=True, infer=True, ref=True, entropy=True, mask=0.2)
    args = dict(reduce=reduce, **runs(ratio))
    check(call(r3, t, cu, **args), t, oracle(t, cu, **args))


GARBAGE = [[0, 50, 40, 100], [1, 50, 100], [0, 50, 1 << 30], [0, -5, 100], [-(1 << 31), (1 << 31) - 1, 0], [0, 30000, 0, 30000],
           [30000] * 40, [0] + [30000, 0] * 300 + [30000]]


@pytest.mark.parametrize("T", [100, 30000])
@pytest.mark.parametrize("ratio,reduce", [("token", "token"), ("sequence", "sequence"), ("token", "sequence")])
def test_bad_bounds_leave_what_lies_around_the_outputs(r3, T, ratio, reduce):
    """Every output and the workspace lie between margins of one buffer, which keep what they held."""
    rows = GARBAGE + [np.random.default_rng(i).integers(-(1 << 31), 1 << 31, 700).tolist() for i in range(4)]
    t = {k: v.cuda() for k, v in make(T, [0, T], 3, entropy=True, infer=True, ref=True).items()}
    for row in rows:
        cu = torch.tensor(row, dtype=torch.int32).cuda()
        c = r3.Policy(T, len(row) - 1, r3._RATIO[ratio], r3._REDUCE[reduce], 1, 0.2, 0.2, 1.5, 2.0, 0.1, 0.1, 0.0)
        need = r3.lib.r3_policy_loss_workspace_bytes(ctypes.byref(c))
        sizes = dict(loss=4, dlogp=4 * T, dentropy=4 * T, metrics=12, counts=12, ws=need)
        margin, at, places = 8192, 8192, {}
        for k, n in sizes.items():
            places[k] = (at, n)
            at += (n + 255) // 256 * 256 + margin
        buf = torch.full((at,), 0x5a, dtype=torch.uint8, device="cuda")
        st = r3.new_status("cuda")
        p = lambda k: buf.data_ptr() + places[k][0]
        code = r3.lib.r3_policy_loss(
            ctypes.byref(c), t["logp"].data_ptr(), t["logp_old"].data_ptr(), t["advantages"].data_ptr(), cu.data_ptr(), None,
            t["logp_infer"].data_ptr(), t["logp_ref"].data_ptr(), t["entropy"].data_ptr(), None, p("loss"), p("dlogp"),
            p("dentropy"), p("metrics"), p("counts"), p("ws"), need, st.data_ptr(), r3._stream())
        good = row[0] == 0 and all(a <= b for a, b in zip(row, row[1:])) and row[-1] <= T
        assert code == r3.R3_OK and st.item() == (r3.DEV_OK if good else r3.DEV_BAD_INDEX)
        for at, n in places.values():
            buf[at:at + n] = 0x5a
        assert (buf == 0x5a).all()
