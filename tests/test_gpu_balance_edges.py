"""The balance loss where its numbers are large or many.

Tolerances: test_gpu_balance's, D = 2^-24 (|s - top| + 50) of a probability and of sum f p."""
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


LARGE = [9e5, 2e6, 5e9, 1e10, 3e20, 3e38, -2e6, -1e9, -1e10, -1e30, float(torch.finfo(torch.float32).min)]


@pytest.mark.parametrize("E,K", [(8, 2), (60, 4), (128, 8), (301, 6), (1021, 3), (1024, 8)])
def test_large_finite_logits(r3, E, K):
    """Finite fills of masked experts, of whole rows too, and tops far from zero: softmax and its gradient are those
    of the differences."""
    T = 6 * len(LARGE) + 3
    g = torch.Generator().manual_seed(E)
    x = torch.randn((1, T, E), generator=g)
    for i, m in enumerate(LARGE):
        rows = x[0, 6 * i:6 * i + 6]
        rows[0] = m                                            # evenly
        rows[1], rows[1, E // 2:] = m, -float("inf")
        rows[2, E // 3:] = -abs(m)                             # a fill beside ordinary logits
        rows[3, 1:], rows[3, 0] = m, float(np.nextafter(np.float32(m), np.float32(-abs(m) / 2)))
        rows[4] = m + 4 * rows[4] if abs(m) < 1e9 else m * (1 - rows[4].abs() / 8)
        rows[5, 0] = abs(m)
    rec = random_record(np.random.default_rng(E), T, E, K, torch.int16)[None]
    s = r3.make_shape(T, 8, E, K, 8, idx=torch.int16)
    loss, _, d = r3.balance_loss(s, 1, x.cuda(), rec.cuda(), balance_coef=0.7)
    balance, _, _, want, p, _, f = O.balance_loss(f64(x[0]), rec[0].long().numpy(), None, None, 0.7, 0.0)
    far = np.where(p > 0, f64(x[0]).max(1, keepdims=True) - f64(x[0]), 0)
    near = 2.0 ** -24 * (far + 50)
    size = p * 0.7 * (f + (p * f).sum(1, keepdims=True)) / T
    assert np.isfinite(f64(d)).all()
    assert (np.abs(f64(d[0]) - want) <= size * (2 * near + 2.0 ** -24 * 60) + 2.0 ** -140).all()
    assert abs(loss[0, 0].item() - balance) <= 2.0 ** -24 * (T / 8 + 80 + far.max()) * balance
    # the logarithm of the sum, by the z loss of tokens one by one; its square may pass float32
    for t in (0, 6, 12, 6 * LARGE.index(-1e9)):
        one = r3.make_shape(1, 8, E, K, 8, idx=torch.int16)
        z = r3.balance_loss(one, 1, x[:, t:t + 1].contiguous().cuda(), rec[:, t:t + 1].contiguous().cuda())[0][0, 1].item()
        lse = O.balance_loss(f64(x[0, t:t + 1]), rec[0, t:t + 1].long().numpy())[5][0, 0]
        assert abs(z - lse ** 2) <= 2.0 ** -20 * lse ** 2


@pytest.mark.parametrize("seed", [0, 6])
def test_sums_of_many_tokens(r3, seed):
    """2^26 equal tokens: added one after the other in float32, 1771 a lane on 148 SMs, p_0 would be 317 (327) and the
    square 142 (186) times 2^-24 off, since equal terms are rounded the same way again and again.  In runs of 64
    at most, those in 64 bits: half of 64 steps of 2^-24, and what each term is off by (a probability 53, the square of
    the logarithm 12)."""
    T, E = 1 << 26, 3
    x = np.random.default_rng(seed).standard_normal(E).astype(np.float32)
    logits = torch.from_numpy(x).cuda().expand(1, T, E).contiguous()
    counts = torch.tensor([[1, 0, 0]], dtype=torch.int32).cuda()
    loss = r3.balance_loss(r3.make_shape(T, 8, E, 1, 8), 1, logits, counts=counts, want_grad=False)[0]
    p = np.exp(x.astype(np.float64))
    lse = np.log(p.sum())
    assert abs(loss[0, 0].item() / (E * p[0] / p.sum()) - 1) <= 2.0 ** -24 * (32 + 53 + 8)
    assert abs(loss[0, 1].item() / lse ** 2 - 1) <= 2.0 ** -24 * (32 + 12 / min(1.0, abs(lse)) + 8)


def test_gradient_to_router_and_block_input(r3):
    """From a block's input through its logits to the losses and back: the dense products with the block's input and
    its router's weight are the gradients of the formula, by autograd in 64 bits.  Logits are float32 sums of 256
    products of a bf16 and a float32 number, off by 2^-19 at most, which moves a probability and what is formed of it
    by as much; with sums of 600 tokens in float32 1e-4 of the largest element covers them.  What only the recorded
    experts' columns hold of it is far from that."""
    T, d, E, K, bc, zc = 600, 256, 32, 4, 0.3, 0.02
    g = torch.Generator().manual_seed(9)
    x = (torch.randn((T, d), generator=g)).to(torch.bfloat16)
    w = torch.randn((E, d), generator=g) * 0.06
    s = r3.make_shape(T, d, E, K, 8)
    idx, logits = r3.capture_topk(s, x.cuda(), w.cuda(), want_logits=True)
    loss, counts, dl = r3.balance_loss(s, 1, logits[None], idx[None], balance_coef=bc, z_coef=zc)
    xd, wd = x.double().requires_grad_(), w.double().requires_grad_()
    z = xd @ wd.T
    f = E * counts[0].cpu().double() / (T * K)
    want = bc * (f * torch.softmax(z, 1).mean(0)).sum() + zc * (torch.logsumexp(z, 1) ** 2).mean()
    want.backward()
    assert abs(bc * loss[0, 0].item() + zc * loss[0, 1].item() - want.item()) < 1e-5 * want.item()
    dw, dx = dl[0].T @ x.cuda().float(), dl[0] @ w.cuda()
    for got, ref in ((dw, wd.grad), (dx, xd.grad)):
        assert (got.cpu().double() - ref).abs().max() <= 1e-4 * ref.abs().max()
    kept = torch.zeros_like(dl[0]).scatter_(1, idx.long(), dl[0].gather(1, idx.long()))
    assert ((kept @ w.cuda()).cpu().double() - xd.grad).abs().max() > 0.1 * xd.grad.abs().max()
