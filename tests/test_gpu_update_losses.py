"""The policy loss, the routers' balance loss and the matrix optimiser where an Update step uses them: between
the log probabilities and their gradient, on the dlogits of a stack's exact backward chain, and on its
expert-weight gradients; eager and as one captured graph.

Tolerances.  The gradient to the vocabulary's logits is dlogp (p - onehot) with dlogp within 2^-19 (1 + |d|)
of itself (the policy loss) and p within 2e-5 (the log probabilities' float32 sums over the vocabulary):
together 1e-4 of the row's largest element.  The balance gradient is added to dlogits in float32: 1e-5 of the
largest element.  A weight's step is the oracle's on the same gradients, within its own tests' bound."""
import numpy as np
import pytest
import torch

from oracle import r3_loss_oracle as O
from oracle import r3_muon_oracle as M
from tests.helpers import f64
from tests.test_gpu_normed_stack import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def responses(seed, lengths, V, ratio_noise):
    g = torch.Generator().manual_seed(seed)
    T = sum(lengths)
    logits = torch.randn((T, V), generator=g) * 2
    ids = torch.randint(0, V, (T,), generator=g)
    ids[torch.rand(T, generator=g) < 0.2] = -1                    # prompt and padding
    lp = torch.log_softmax(logits.double(), 1).gather(1, ids.clamp(min=0)[:, None])[:, 0]
    noise = lambda std: (lp + std * torch.randn(T, generator=g)).float()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32)
    return dict(logits=logits, ids=ids, cu=cu, old=noise(ratio_noise), infer=noise(0.1), ref=noise(0.3),
                adv=torch.randn(len(lengths), generator=g), T=T)


def test_from_logits_to_their_gradient(r3):
    V, kl, ent_c = 1003, 0.05, 0.02
    t = responses(1, [40, 1, 0, 130, 77, 300], V, 0.15)
    dev = {k: v.cuda() for k, v in t.items() if k != "T"}
    for ratio, reduce in (("token", "token"), ("sequence", "sequence"), ("token", "sequence")):
        logp, entropy, stats, _, _ = r3.token_logprobs(dev["logits"], dev["ids"], want_entropy=True, want_stats=True)
        loss, dlogp, dent, metrics, counts = r3.policy_loss(
            logp, dev["old"], dev["cu"], seq_advantages=dev["adv"], mask=dev["ids"] >= 0, logp_infer=dev["infer"],
            logp_ref=dev["ref"], entropy=entropy, ratio=ratio, reduce=reduce, kl_coef=kl, entropy_coef=ent_c)
        got = r3.token_logprobs_bwd(dev["logits"], dev["ids"], stats, dlogp, entropy=entropy, dentropy=dent)
        # the same in 64 bits, the loss's parts from its oracle, the rest by autograd
        z = t["logits"].double().requires_grad_()
        lsm = torch.log_softmax(z, 1)
        lp = lsm.gather(1, t["ids"].clamp(min=0)[:, None])[:, 0]
        H = -(lsm.exp() * lsm).sum(1)
        ref = O.policy_loss(f64(lp), f64(t["old"]), f64(t["adv"]).view(O.PerSequence), t["cu"].tolist(),
                            (t["ids"] >= 0).numpy(), f64(t["infer"]), f64(t["ref"]), f64(H), ratio, reduce,
                            kl_coef=kl, entropy_coef=ent_c)
        ((lp * torch.from_numpy(ref["dlogp"])).sum() + (H * torch.from_numpy(ref["dentropy"])).sum()).backward()
        want = f64(z.grad)
        assert abs(loss.item() - ref["loss"]) < 1e-5 * (ref["size"] + ref["kl"] + ref["entropy"])
        assert counts.tolist() == [ref["tokens"], ref["clipped"], ref["cut"]]
        bound = 1e-4 * np.abs(want).max(1, keepdims=True) + 1e-12
        assert (np.abs(f64(got) - want) <= bound).all()


def test_balance_loss_on_a_stacks_router_gradients(r3):
    """dlogits of the exact backward chain plus the balance loss's, as one gradient of the routers."""
    w, x0, dy, w_r, idx, ex, norms = build(192, 256, 16, 2, 128, 2)
    s = r3.shape_of(w)
    out = r3.normed_stack_train(s, 2, x0, w_r, idx, *ex, dy, **norms)
    dlogits = out[1]
    plain = dlogits.clone()
    h = torch.randn(2, 192, 256, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    _, logits = r3.capture_topk_batched(s, 2, h, w_r, want_idx=False, want_logits=True)
    loss, counts, same = r3.balance_loss(s, 2, logits, idx, balance_coef=0.3, z_coef=0.01, dlogits=dlogits,
                                         accumulate=True)
    assert same is dlogits
    for l in range(2):
        balance, z, n, d, *_ = O.balance_loss(f64(logits[l]), idx[l].cpu().long().numpy(), None, None, 0.3, 0.01)
        want = f64(plain[l]) + d
        assert np.abs(f64(dlogits[l]) - want).max() <= 1e-5 * np.abs(want).max()
        assert np.array_equal(counts[l].cpu().numpy(), n) and abs(loss[l, 0].item() - balance) < 1e-5 * balance


def test_expert_weights_take_orthogonalised_steps(r3):
    """Gradients of a stack's experts as they lie, into one step over all of them and the routers' beside."""
    w, x0, dy, w_r, idx, ex, norms = build(256, 256, 8, 2, 136, 1, seed=2)
    s = r3.shape_of(w)
    grads = list(r3.normed_stack_train(s, 1, x0, w_r, idx, *ex, dy, expert_grads=True, **norms)[-3:])
    assert [g.shape for g in grads] == [e.shape for e in ex]
    before = [e.clone() for e in ex]
    opt = r3.Muon(ex, grads, momentum=0.9, scale="rms", weight_decay=0.01)
    opt.step(0.05)
    for e, old, g in zip(ex, before, grads):
        rows, cols = e.shape[-2:]
        for j in (0, 3, 7):
            u = 1.9 * f64(g[0, j])
            o = M.iterate(u)
            hard = 2 * np.abs(M.iterate(u, operand=M.half_operand) - o).max() + 2.0 ** -20 * np.abs(o).max()
            rate = 0.05 * 0.2 * max(rows, cols) ** 0.5
            want = f64(old[0, j]) * (1 - 0.05 * 0.01) - rate * o
            slack = rate * hard + 2.0 ** -20 * np.abs(want).max()
            assert (np.abs(f64(e[0, j]) - want) <= slack + 2.0 ** -8 * (np.abs(want) + slack)).all()


def test_one_graph_of_the_whole_step(r3):
    """Log probabilities, loss, gradient and the weights' step captured once and replayed give what the eager
    calls give, twice in a row."""
    t = responses(3, [200, 57, 400], 515, 0.05)
    d = {k: v.cuda() for k, v in t.items() if k != "T"}
    g = torch.Generator().manual_seed(4)
    x = torch.randn((t["T"], 96), generator=g).cuda()
    weights = [(torch.randn((515, 96), generator=g) * 0.1).cuda() for _ in range(2)]
    grads = [torch.zeros_like(w) for w in weights]
    opts = [r3.Muon([w], [gr]) for w, gr in zip(weights, grads)]
    weights[1].copy_(weights[0])

    def step(i):
        logits = x @ weights[i].T
        logp, _, stats, _, _ = r3.token_logprobs(logits, d["ids"], want_stats=True)
        loss, dlogp, *_ = r3.policy_loss(logp, d["old"], d["cu"], seq_advantages=d["adv"], mask=d["ids"] >= 0)
        dlogits = r3.token_logprobs_bwd(logits, d["ids"], stats, dlogp, dlogits=logits)
        torch.mm(dlogits.T, x, out=grads[i])
        opts[i].step(0.01)
        return loss
    start, buf = weights[0].clone(), opts[0].momentum_buffers[0]
    step(0)                                                        # libraries' own set-up, before the capture
    weights[0].copy_(start)
    buf.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(0)
    for _ in range(3):
        graph.replay()
        loss = step(1)
        assert torch.equal(held, loss) and torch.equal(weights[0], weights[1])


def test_calls_on_two_streams_at_once_and_two_graphs_of_them(r3):
    """Every operator on two streams without a wait between them, and replayed from two graphs side by side, gives
    what it gives alone: workspaces are each call's own."""
    g = torch.Generator().manual_seed(5)
    T, L, E, K = 9000, 3, 128, 8
    shape = r3.make_shape(T, 8, E, K, 8)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]

    def inputs():
        rn = lambda *s: torch.randn(s, generator=g).cuda()
        return dict(lp=rn(T), old=rn(T), adv=rn(T), cu=torch.tensor([0, 4000, 4001, T], dtype=torch.int32).cuda(),
                    logits=rn(L, T, E), rec=torch.randint(0, E, (L, T, K), generator=g, dtype=torch.uint8).cuda(),
                    small=rn(5, 96, 700), wide=rn(2, 300, 520), bf=rn(12, 512, 768).bfloat16())

    def run(t):
        out = []
        for _ in range(3):
            out += [r3.policy_loss(t["lp"], t["old"], t["cu"], advantages=t["adv"], ratio="sequence")[1],
                    *r3.balance_loss(shape, L, t["logits"], t["rec"], z_coef=0.1),
                    r3.orthogonalize(t["small"]), r3.orthogonalize(t["wide"]), r3.orthogonalize(t["bf"])]
        return out

    both = [inputs(), inputs()]
    want = [run(t) for t in both]
    torch.cuda.synchronize()
    got = []
    for t, side in zip(both, sides):
        with torch.cuda.stream(side):
            got.append(run(t))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    graphs, held = [], []
    for t in both:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held.append(run(t))
        graphs.append(graph)
    for _ in range(2):
        for graph, side in zip(graphs, sides):
            with torch.cuda.stream(side):
                graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, held):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
