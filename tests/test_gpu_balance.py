"""The balance loss on the GPU against the float64 oracle.

Tolerances.  A probability is exp(s - top) / sum: the difference is rounded (2^-24 |s - top| of p), the
exponential 2^-22, the sum of E positive terms at most (V + 5) 2^-24 with V <= 32 of them per lane, quotient
and product 2^-23: p is within D = 2^-24 (|s - top| + 50) of itself, and so is sum f p (positive terms, as
many roundings again).  The gradient's terms are p f, p sum f p and p lse, four roundings each."""
import numpy as np
import pytest
import torch

from oracle import r3_loss_oracle as O
from tests.helpers import f64, random_record

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def make(r3, L, T, E, K, idx=torch.uint8, seed=0, std=1.5):
    g = torch.Generator().manual_seed(seed + T + E)
    rng = np.random.default_rng(seed + T)
    logits = torch.randn((L, T, E), generator=g) * std + torch.randn((L, 1, E), generator=g)
    rec = torch.stack([random_record(rng, T, E, K, idx) for _ in range(L)]) if T else \
        torch.zeros((L, 0, K), dtype=idx)
    return r3.make_shape(T, 8, E, K, 8, idx=idx), logits, rec


def check(out, logits, rec, mask=None, counts=None, bc=1.0, zc=0.0, base=None):
    loss, got_counts, dlogits = out
    for l in range(logits.shape[0]):
        balance, z, n, d, p, lse, f = O.balance_loss(
            f64(logits[l]), rec[l].long().numpy(), None if mask is None else mask.numpy(),
            None if counts is None else counts[l].numpy(), bc, zc)
        assert np.array_equal(got_counts[l].cpu().numpy(), n)
        x = f64(logits[l])
        top = x.max(1, keepdims=True)
        far = np.where(p > 0, top - x, 0)
        near = 2.0 ** -24 * (far + 50)
        tokens = max(1, int(mask.sum()) if mask is not None else logits.shape[1])
        along = (p * f).sum(1, keepdims=True)
        size = p * (abs(bc) * (f + along) + 2 * abs(zc) * (np.abs(lse) + 1)) / tokens
        bound = size * (2 * near + 2.0 ** -24 * 60) + 2.0 ** -140
        want = d if base is None else d + f64(base[l])
        if base is not None:
            bound = bound + 2.0 ** -24 * np.abs(want)
        if dlogits is not None:
            assert (np.abs(f64(dlogits[l]) - want) <= bound).all()
        adds = 2.0 ** -24 * (logits.shape[1] / 8 + 80 + np.abs(far).max(initial=0))
        assert abs(float(loss[l, 0]) - balance) <= adds * balance
        assert abs(float(loss[l, 1]) - z) <= 2.0 ** -20 * (z + 1)


@pytest.mark.parametrize("E,K,idx", [(1, 1, torch.uint8), (3, 2, torch.uint8), (8, 2, torch.uint8),
                                     (16, 16, torch.int16), (17, 3, torch.uint8), (60, 4, torch.uint8),
                                     (64, 6, torch.uint8), (128, 8, torch.uint8), (130, 8, torch.int16),
                                     (256, 8, torch.uint8), (301, 6, torch.int16), (512, 10, torch.int16),
                                     (1021, 3, torch.int16), (1024, 8, torch.int16)])
@pytest.mark.parametrize("L,T", [(1, 1), (2, 63), (3, 129), (1, 4097)])
def test_against_oracle(r3, L, T, E, K, idx):
    s, logits, rec = make(r3, L, T, E, K, idx)
    st = r3.new_status("cuda")
    check(r3.balance_loss(s, L, logits.cuda(), rec.cuda(), balance_coef=0.7, z_coef=0.2, dev_status=st),
          logits, rec, bc=0.7, zc=0.2)
    mask = torch.rand(T, generator=torch.Generator().manual_seed(1)) < 0.6
    bad = torch.where(mask[None, :, None], logits, float("nan"))
    loose = rec.clone()
    loose[:, ~mask] = -1 if idx == torch.int16 else 255        # a masked token's record is not looked at
    check(r3.balance_loss(s, L, bad.cuda(), loose.cuda(), mask=mask.cuda(), balance_coef=-0.3, dev_status=st),
          torch.where(mask[None, :, None], logits, 0.0), torch.where(mask[None, :, None], rec, 0 * rec),
          mask, bc=-0.3)
    assert st.item() == 0


def test_large_skewed(r3):
    s, logits, rec = make(r3, 1, 30000, 128, 8)
    rec[:, :20000, 0] = 5                                     # an expert that most tokens chose
    rec[:, :20000, 1:] = torch.arange(6, 13, dtype=torch.uint8)
    check(r3.balance_loss(s, 1, logits.cuda(), rec.cuda()), logits, rec)


def test_given_counts_accumulate_and_forward_alone(r3):
    s, logits, rec = make(r3, 2, 700, 128, 8)
    dev, idx = logits.cuda(), rec.cuda()
    loss, counts, none = r3.balance_loss(s, 2, dev, idx, want_grad=False)
    assert none is None
    check((loss, counts, None), logits, rec)
    more = counts * 3 + torch.randint(0, 50, counts.shape, device="cuda", dtype=torch.int32)   # other ranks'
    kept = more.clone()
    base = torch.randn(2, 700, 128)
    dl = base.cuda()
    out = r3.balance_loss(s, 2, dev, counts=more, dlogits=dl, accumulate=True, balance_coef=0.5, z_coef=0.1)
    assert out[2] is dl and torch.equal(more, kept)
    check(out, logits, rec, counts=more.cpu(), bc=0.5, zc=0.1, base=base)
    huge = torch.full((2, 128), 1 << 30, dtype=torch.int32, device="cuda")     # their sum passes 32 bits
    check(r3.balance_loss(s, 2, dev, counts=huge), logits, rec, counts=huge.cpu().long())
    mask = torch.zeros(700, dtype=torch.uint8)
    mask[:5] = 2
    dl = base.cuda()
    out = r3.balance_loss(s, 2, dev, idx, mask=mask.cuda(), dlogits=dl, accumulate=True)
    assert torch.equal(dl[:, 5:].cpu(), base[:, 5:])
    check(out, logits, rec, mask.bool(), base=base)
    same = dev.clone()                                        # the gradient in the logits' buffer
    out = r3.balance_loss(s, 2, same, idx, dlogits=same)
    check(out, logits, rec)


def test_empty_masked_and_bad_records(r3):
    s, logits, rec = make(r3, 2, 0, 16, 2)
    loss, counts, d = r3.balance_loss(s, 2, logits.cuda(), rec.cuda())
    assert not loss.any() and not counts.any() and d.shape == (2, 0, 16)
    s, logits, rec = make(r3, 2, 300, 16, 2)
    loss, counts, d = r3.balance_loss(s, 2, logits.cuda(), rec.cuda(), mask=torch.zeros(300, dtype=torch.bool).cuda(),
                                      z_coef=1.0)
    assert not loss.any() and not counts.any() and not d.any()
    st = r3.new_status("cuda")
    wrong = rec.clone()
    wrong[0, 7, 1] = 16
    loss, counts, d = r3.balance_loss(s, 2, logits.cuda(), wrong.cuda(), dev_status=st)
    assert st.item() == r3.DEV_BAD_INDEX and counts[0].sum() == 599 and counts[1].sum() == 600
    assert torch.isfinite(d).all()


def test_infinities_and_nan(r3):
    s, logits, rec = make(r3, 1, 200, 64, 4)
    logits[0, :, 5] = -float("inf")                           # an expert that is shut
    logits[0, 7] = -float("inf")                              # a token without any
    logits[0, 9, 3] = torch.finfo(torch.float32).min
    check(r3.balance_loss(s, 1, logits.cuda(), rec.cuda(), z_coef=0.1), logits, rec, zc=0.1)
    clean = r3.balance_loss(s, 1, logits.cuda(), rec.cuda())[2]
    for v in (float("nan"), float("inf")):
        logits[0, 11, 60] = v
        loss, _, d = r3.balance_loss(s, 1, logits.cuda(), rec.cuda())
        assert torch.isnan(loss).all() and torch.isnan(d[0, 11]).all()
        rest = torch.arange(200) != 11
        assert torch.equal(d[0, rest.cuda()], clean[0, rest.cuda()])


def test_repeats_streams_and_graphs(r3):
    s, logits, rec = make(r3, 3, 5000, 128, 8)
    dev, idx = logits.cuda(), rec.cuda()
    ws = r3.workspace(r3.lib.r3_balance_loss_workspace_bytes(s, 3), "cuda")
    ws.fill_(255)
    want = r3.balance_loss(s, 3, dev, idx, z_coef=0.1, ws=ws)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, r3.balance_loss(s, 3, dev, idx, z_coef=0.1, ws=ws)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = r3.balance_loss(s, 3, dev, idx, z_coef=0.1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = r3.balance_loss(s, 3, dev, idx, z_coef=0.1)
    for _ in range(2):
        dev.mul_(1.1)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(r3.balance_loss(s, 3, dev, idx, z_coef=0.1), held))


@pytest.mark.parametrize("L,T,E,K,idx", [(1, 1024, 8, 2, torch.uint8), (1, 1025, 8, 2, torch.uint8),
                                         (5, 64, 128, 8, torch.int16), (5, 65, 128, 8, torch.int16),
                                         (3, 8, 1024, 10, torch.int16), (2, 8192, 1, 1, torch.uint8)])
def test_blocks_around_a_single_ctas_size(r3, L, T, E, K, idx):
    """Both sides of the size up to which a CTA counts its block's choices itself: masks, given counts, sums onto
    a gradient, invalid records."""
    s, logits, rec = make(r3, L, T, E, K, idx, 4)
    dev, record = logits.cuda(), rec.cuda()
    mask = (torch.rand(T, generator=torch.Generator().manual_seed(2)) < 0.5).to(torch.uint8) * 3
    base = torch.randn(L, T, E)
    dl = base.cuda()
    out = r3.balance_loss(s, L, dev, record, mask=mask.cuda(), dlogits=dl, accumulate=True, z_coef=0.1)
    check(out, logits, rec, mask.bool(), zc=0.1, base=base)
    assert torch.equal(dl[:, ~mask.bool()].cpu(), base[:, ~mask.bool()])
    given = torch.randint(0, 1 << 29, (L, E), dtype=torch.int32).cuda()
    check(r3.balance_loss(s, L, dev, counts=given, mask=mask.cuda()), logits, rec, mask.bool(), counts=given.cpu().long())
    wrong, st = rec.clone(), r3.new_status("cuda")
    wrong[L - 1, T - 1, K - 1] = E
    if idx == torch.int16:
        wrong[0, 0, 0] = -3
    _, counts, d = r3.balance_loss(s, L, dev, wrong.cuda(), dev_status=st)
    assert st.item() == r3.DEV_BAD_INDEX and torch.isfinite(d).all()
    assert counts.sum() == L * T * K - (2 if idx == torch.int16 else 1)
    loss, counts, none = r3.balance_loss(s, L, dev, record, want_grad=False)
    want = r3.balance_loss(s, L, dev, record)
    assert none is None and torch.equal(loss, want[0]) and torch.equal(counts, want[1])
