"""The policy loss on the GPU against the float64 oracle.

Tolerances, relative to each part of a token's gradient.  A ratio is the float32 exponential (2^-22) of a
difference rounded to float32 (2^-24 of it, which moves the ratio by 2^-24 |d|), the correction w the
same with x = logp_old - logp_infer; advantage, ratio, w and the weight meet in three products and the
weight is rounded once: 4 2^-24.  Together 2^-21 (1 + 1/2 + |d| + |x|) and less than 2^-20 (1 + |d| + |x|).
The KL part: its x is rounded (which moves expm1 by 2^-24 (1 + |x|) of itself), expm1 2^-22, weight and
product: 2^-21 (1 + |x|).  One rounding of the sum.  The loss is the 64-bit sum of such terms."""
import numpy as np
import pytest
import torch

from oracle import r3_loss_oracle as O
from tests.helpers import f64

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -20


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def lengths(T, S, seed):
    """S lengths that add up to T, some of them 0."""
    rng = np.random.default_rng(seed)
    cut = np.sort(rng.integers(0, T + 1, S - 1)) if S > 1 else np.zeros(0, dtype=int)
    return np.concatenate([[0], cut, [T]]).astype(np.int32)


def make(T, cu, seed=0, per_sequence=False, infer=False, ref=False, entropy=False, mask=0.0):
    g = torch.Generator().manual_seed(seed + T)

    def rn(n=T):
        return torch.randn(n, generator=g)
    old = -torch.rand(T, generator=g) * 5
    t = dict(logp=old + 0.2 * rn(), logp_old=old)
    if infer:
        t["logp_infer"] = old + 0.4 * rn()
    if ref:
        t["logp_ref"] = old + 0.5 * rn()
    if entropy:
        t["entropy"] = torch.rand(T, generator=g) * 3
    if mask:
        t["mask"] = torch.rand(T, generator=g) >= mask
        for k in ("logp", "logp_old", "logp_infer", "logp_ref", "entropy"):
            if k in t:                                     # nothing of a masked token may be used
                t[k] = torch.where(t["mask"], t[k], float("nan") if seed % 2 else float("inf"))
    adv = rn(len(cu) - 1 if per_sequence else T)
    adv[:1] = 0
    t["seq_advantages" if per_sequence else "advantages"] = adv
    return t


def oracle(t, cu, **kw):
    kw.pop("dloss", None)
    args = {k: f64(v) for k, v in t.items() if k not in ("mask", "seq_advantages", "advantages")}
    adv = f64(t["advantages"]) if "advantages" in t else f64(t["seq_advantages"]).view(O.PerSequence)
    return O.policy_loss(advantages=adv, cu_seqlens=cu, mask=t["mask"].numpy() if "mask" in t else None,
                         **args, **kw)


def call(r3, t, cu, **kw):
    dev = {k: v.cuda() for k, v in t.items()}
    st = r3.new_status("cuda")
    cu = None if cu is None else torch.as_tensor(cu, dtype=torch.int32).cuda()
    out = r3.policy_loss(dev.pop("logp"), dev.pop("logp_old"), cu, dev_status=st, **dev, **kw)
    assert st.item() == 0
    return out


def check(out, t, ref, scale=1.0):
    loss, dlogp, dentropy, metrics, counts = out
    x = np.abs(ref["x"])
    pol = np.maximum(np.abs(ref["policy_grad"]), ref["seq_size"])
    kl = np.abs(ref["kl_grad"])
    xr = np.abs(f64(t["logp_ref"]) - f64(t["logp"])) if "logp_ref" in t else 0.0
    worst = x.max() if x.size else 0.0
    bound = EPS * ((1 + np.abs(ref["d"]) + (worst if ref["seq_size"].any() else x)) * pol
                   + np.nan_to_num(1 + xr, posinf=0) * kl) + 2.0 ** -24 * np.abs(ref["dlogp"])
    assert (np.abs(f64(dlogp) - scale * ref["dlogp"]) <= abs(scale) * bound + 1e-37).all()
    if dentropy is not None:
        assert (np.abs(f64(dentropy) - scale * ref["dentropy"])
                <= 2.0 ** -22 * abs(scale) * np.abs(ref["dentropy"]) + 1e-37).all()
    far = EPS * (1 + (np.abs(ref["d"]).max() if x.size else 0) + worst)
    got = f64(metrics)
    assert abs(got[0] - ref["policy"]) <= far * ref["size"] + 1e-37
    assert abs(got[1] - ref["kl"]) <= 2.0 ** -19 * ref["kl"] + 1e-37
    assert abs(got[2] - ref["entropy"]) <= 2.0 ** -22 * abs(ref["entropy"]) + 1e-37
    whole = ref["size"] + abs(ref["kl"]) + abs(ref["entropy"])
    assert abs(float(loss) - ref["loss"]) <= far * whole + 1e-37
    assert counts.tolist() == [ref["tokens"], ref["clipped"], ref["cut"]]


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("reduce", ["token", "sequence"])
@pytest.mark.parametrize("T,S", [(1, 1), (1, 3), (31, 2), (255, 1), (256, 1), (257, 5), (1531, 12), (3000, 40),
                                 (9000, 1), (20011, 300), (20011, 4)])
def test_against_oracle(r3, T, S, ratio, reduce):
    cu = lengths(T, S, T)
    for seed, kw in enumerate([dict(), dict(per_sequence=True, infer=True, ref=True, entropy=True, mask=0.3),
                               dict(infer=True, mask=0.9), dict(per_sequence=True, ref=True)]):
        t = make(T, cu, seed, **kw)
        args = dict(ratio=ratio, reduce=reduce, clip_low=0.01 if ratio == "sequence" else 0.2,
                    clip_high=0.02 if ratio == "sequence" else 0.28, dual_clip=[0.0, 1.5][seed % 2],
                    infer_cap=1.3, kl_coef=0.1, entropy_coef=0.01)
        check(call(r3, t, cu, **args), t, oracle(t, cu, **args))


@pytest.mark.parametrize("T,S", [(900, 7), (30000, 90)])
def test_tokens_behind_the_last_sequence_and_padded_rows(r3, T, S):
    """cu_seqlens may end before T; a padded batch [B, R] is B sequences of R tokens with a mask."""
    cu = lengths(T - 100, S, 3)
    t = make(T, cu, 2, per_sequence=True, infer=True, ref=True, entropy=True)
    for k in t:
        if t[k].numel() == T:
            t[k][T - 100:] = float("nan")
    args = dict(ratio="sequence", reduce="sequence", clip_low=0.01, clip_high=0.01, kl_coef=0.1,
                entropy_coef=0.1)
    out = call(r3, t, cu, **args)
    assert (out[1][T - 100:] == 0).all() and (out[2][T - 100:] == 0).all()
    short = {k: v[:T - 100] if v.numel() == T else v for k, v in t.items()}
    ref = oracle(short, cu, **args)
    check((out[0], out[1][:T - 100], out[2][:T - 100], *out[3:]), short, ref)


def test_no_sequence_no_token_and_no_bounds(r3):
    t = make(500, [0, 500], 1)
    ref = oracle(t, [0, 500])
    check(call(r3, t, None), t, ref)                             # one sequence
    empty = {k: v[:0] for k, v in t.items()}
    for cu in (None, [0], [0, 0, 0]):
        loss, dlogp, _, _, counts = call(r3, empty, cu)
        assert loss.item() == 0 and dlogp.numel() == 0 and counts.tolist() == [0, 0, 0]
    t["mask"] = torch.zeros(500, dtype=torch.uint8)
    for ratio in ("token", "sequence"):
        for reduce in ("token", "sequence"):
            loss, dlogp, _, metrics, counts = call(r3, t, [0, 200, 500], ratio=ratio, reduce=reduce)
            assert loss.item() == 0 and not dlogp.any() and not metrics.any() and counts.tolist() == [0, 0, 0]
    t.pop("mask")
    loss, dlogp, *_ = call(r3, {**t, "advantages": t["advantages"]}, [0])      # all behind the last
    assert loss.item() == 0 and not dlogp.any()


def test_borders_are_inside(r3):
    """A ratio exactly on a border takes its gradient, the next float beyond it does not."""
    up = np.float32(np.log1p(0.2))
    if float(up) > np.log1p(0.2):
        up = np.nextafter(up, np.float32(0))
    d = torch.tensor([float(up), float(np.nextafter(up, np.float32(9))), 0.0, 0.0])
    t = dict(logp=d, logp_old=torch.zeros(4), advantages=torch.tensor([1.0, 1.0, 2.0, -2.0]))
    _, dlogp, _, _, counts = call(r3, t, [0, 4])
    assert dlogp[0] != 0 and dlogp[1] == 0 and dlogp[2] == -0.5 and dlogp[3] == 0.5
    assert counts.tolist() == [4, 1, 0]


@pytest.mark.parametrize("T", [64, 30000])
def test_what_is_not_finite_stays_with_its_token(r3, T):
    cu = np.array([0, T // 2, T], dtype=np.int32)
    t = make(T, cu, 4, ref=True)
    t["logp"][3] = float("nan")
    t["logp"][T - 2] = -float("inf")                    # a sampled token that the mask of logits shut
    t["advantages"][T - 2] = 1.0
    t["logp"][T // 2] = 200.0                           # the ratio overflows; no advantage, no term
    t["advantages"][T // 2] = 0.0
    t["logp_ref"][T // 2] = 200.0
    clean = {k: v.clone() for k, v in t.items()}
    loss, dlogp, *_ = call(r3, t, cu, kl_coef=0.0)
    assert torch.isnan(loss) and torch.isnan(dlogp[3])
    assert torch.isfinite(dlogp[:3]).all() and torch.isfinite(dlogp[4:T - 2]).all() and dlogp[T // 2] == 0
    _, dlogp, *_ = call(r3, t, cu, ratio="sequence", kl_coef=0.0)
    assert torch.isnan(dlogp[:T // 2]).all() and not torch.isnan(dlogp[T // 2:T - 2]).any()
    clean["mask"] = torch.isfinite(clean["logp"])
    args = dict(clip_low=0.3)
    check(call(r3, clean, cu, **args), clean, oracle(clean, cu, **args))


def test_upstream_gradient_denominator_and_no_gradient(r3):
    cu = lengths(5000, 9, 1)
    t = make(5000, cu, 2, infer=True, ref=True, entropy=True, mask=0.2)
    for reduce in ("token", "sequence"):
        args = dict(reduce=reduce, kl_coef=0.2, entropy_coef=0.1, denominator=123.0)
        ref = oracle(t, cu, **args)
        check(call(r3, t, cu, dloss=torch.full((1,), -3.0).cuda(), **args), t, ref, scale=-3.0)
        loss, dlogp, dentropy, *_ = call(r3, t, cu, want_grad=False, **args)
        assert dlogp is None and dentropy is None
        assert loss.item() == call(r3, t, cu, **args)[0].item()
    # parts of a batch with the whole batch's denominator add up to the whole
    whole = call(r3, t, cu, kl_coef=0.2)
    n = int(whole[4][0])
    part = 0.0
    for i in range(9):
        some = {k: v[cu[i]:cu[i + 1]] for k, v in t.items()}
        if len(some["logp"]):
            part += call(r3, some, None, kl_coef=0.2, denominator=float(n))[0].item()
    assert abs(part - whole[0].item()) < 1e-5


def test_unaligned_views_infinite_borders_and_repeats(r3):
    cu = lengths(7000, 33, 5)
    t = make(7000, cu, 6, infer=True)
    args = dict(clip_high=float("inf"), clip_low=1.0, infer_cap=float("inf"))
    ref = oracle(t, cu, **args)
    assert ref["clipped"] == 0 and ref["cut"] == 0
    views = {k: torch.cat([torch.zeros(1), v]).cuda()[1:] for k, v in t.items()}
    ws = r3.workspace(1 << 20, "cuda")
    ws.fill_(255)
    kw = dict(ws=ws, **args)
    c = torch.as_tensor(cu).cuda()
    first = r3.policy_loss(views["logp"], views["logp_old"], c, advantages=views["advantages"],
                           logp_infer=views["logp_infer"], **kw)
    check(first, t, ref)
    for _ in range(3):
        again = r3.policy_loss(views["logp"], views["logp_old"], c, advantages=views["advantages"],
                               logp_infer=views["logp_infer"], **kw)
        assert all(torch.equal(a, b) for a, b in zip(first, again) if a is not None)


@pytest.mark.parametrize("T,S", [(1000, 4), (40000, 100)])
def test_captured_and_on_another_stream(r3, T, S):
    cu = lengths(T, S, 8)
    t = {k: v.cuda() for k, v in make(T, cu, 8, per_sequence=True, infer=True, entropy=True).items()}
    c = torch.as_tensor(cu).cuda()
    rest = {k: t[k] for k in ("seq_advantages", "logp_infer", "entropy")}

    def run(**kw):
        return r3.policy_loss(t["logp"], t["logp_old"], c, ratio="sequence", clip_low=0.01, clip_high=0.01,
                              entropy_coef=0.1, **rest, **kw)
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for _ in range(2):
        t["logp"].add_(0.01)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(run(), held))


@pytest.mark.parametrize("cu", [[0, 50, 40, 100], [1, 50, 100], [0, 50, 200], [0, -5, 100], [0, 1 << 30, 100],
                                [0, 100, 0, 100]])
@pytest.mark.parametrize("T", [100, 20000])
def test_bad_bounds_are_reported_and_stay_in_range(r3, cu, T):
    t = {k: v.cuda() for k, v in make(T, [0, T], 3, entropy=True).items()}
    st = r3.new_status("cuda")
    guard = torch.full((T + 64,), 7.0, device="cuda")
    dlogp = r3.policy_loss(t["logp"], t["logp_old"], torch.tensor(cu, dtype=torch.int32).cuda(),
                           advantages=t["advantages"], entropy=t["entropy"], ratio="sequence",
                           reduce="sequence", dev_status=st)[1]
    bad = not (cu[0] == 0 and all(a <= b for a, b in zip(cu, cu[1:])) and cu[-1] <= T)
    assert st.item() == (r3.DEV_BAD_INDEX if bad else 0) and dlogp.shape == (T,)
    assert (guard == 7.0).all()


@pytest.mark.parametrize("T,S", [(700, 5), (300000, 50), (40000, 400)])
def test_ratios_of_sequences_without_other_terms(r3, T, S):
    """Nothing but the mask is read again: terms, clipped and capped tokens come from the first pass, whole
    sequences beyond a border and such without a token among them."""
    cu = lengths(T, S, 7)
    for seed, per_sequence in enumerate((True, False, True)):
        t = make(T, cu, seed, per_sequence=per_sequence, infer=seed > 0, mask=0.2 * seed)
        for i in range(0, S, 3):                            # far below, far above
            t["logp"][cu[i]:cu[i + 1]] += 0.7 if i % 2 else -0.7
        for reduce in ("token", "sequence"):
            args = dict(ratio="sequence", reduce=reduce, clip_low=0.2, clip_high=0.3, dual_clip=1.6, infer_cap=1.2)
            ref = oracle(t, cu, **args)
            assert 0 < ref["clipped"] < ref["tokens"]
            check(call(r3, t, cu, **args), t, ref)
            bare = call(r3, t, cu, want_grad=False, **args)
            assert torch.equal(bare[0], call(r3, t, cu, **args)[0])
