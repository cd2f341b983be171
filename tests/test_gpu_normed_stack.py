"""Stacks of replayed blocks with norms around them on the GPU against the float64 oracle, and the
operators of an Update step run together: forward, log probabilities, their gradient, the exact backward
chain and the optimiser's steps.

Tolerances.  Rows and gradients between the blocks are stored in bfloat16 (2^-8 of a value each), the
layers keep their intermediates in bfloat16 too; the bar is the one every block of this library is held
to, max|err| <= 2e-2 max|ref| (1e-5 for float32 layers; here twice that for two chained blocks)."""
import numpy as np
import pytest
import torch

from oracle import r3_diag_oracle as D
from oracle import r3_update_oracle as U
from paper_2510_11370_b200 import synth
from tests.helpers import f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def bf16_store(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(BF).to(torch.float64).numpy()


def build(T, d, E, K, F, L, act="bf16", w_dtype=F32, post=True, gated=True, seed=0):
    w = synth.scaled(synth.WORKLOADS["c2_layer_bf16"], name="normed", T=T, d=d, E=E, K=K, F=F, act=act,
                     layers=L, seed=seed)
    g = torch.Generator().manual_seed(seed + T)
    x0 = synth.activations(w).cuda()
    dy = synth.upstream_grad(w).cuda()
    w_r = torch.stack([synth.router_weight(w, layer=l) for l in range(L)]).cuda()
    ex = [torch.stack(t).cuda() for t in zip(*(synth.expert_weights(w, layer=l) for l in range(L)))]
    rng = np.random.default_rng(seed)
    idx = torch.from_numpy(np.argsort(rng.random((L, T, E)), axis=2)[:, :, :K].copy()).to(torch.uint8).cuda()
    vec = lambda spread: (1 + spread * torch.randn((L, d), generator=g)).to(w_dtype).cuda()
    norms = dict(w_pre=vec(0.2), w_post=vec(0.2) if post else None, gate=vec(0.4) if gated else None)
    return w, x0, dy, w_r, idx, ex, norms


def oracle(x0, dy, w_r, idx, ex, norms, store, **kw):
    L = w_r.shape[0]
    pick = lambda t, l: None if t is None else f64(t[l])
    layers = [(f64(w_r[l]), idx[l].cpu().to(torch.int64).numpy(), *(f64(e[l]) for e in ex)) for l in range(L)]
    return U.normed_stack_bwd(f64(x0), layers, [tuple(pick(norms[k], l) for k in ("w_pre", "w_post", "gate"))
                                                for l in range(L)], f64(dy), store=store, expert_grads=True, **kw)


def rel(got, want):
    want = np.asarray(want)
    return float(np.abs(f64(got) - want).max() / np.abs(want).max())


KW = dict(eps=1e-5, residual_scale=0.9, branch_scale=0.5)


@pytest.mark.parametrize("T,d,E,K,F,L,post,gated,w_dtype", [
    (1, 64, 4, 1, 64, 1, True, True, F32), (33, 128, 8, 2, 136, 3, True, True, BF),
    (260, 256, 16, 4, 128, 2, False, False, F32), (70, 520, 8, 8, 64, 2, True, False, F32)])
def test_forward_and_exact_chain(r3, T, d, E, K, F, L, post, gated, w_dtype):
    w, x0, dy, w_r, idx, ex, norms = build(T, d, E, K, F, L, post=post, gated=gated, w_dtype=w_dtype)
    s, st = r3.shape_of(w), r3.new_status("cuda")
    ref = oracle(x0, dy, w_r, idx, ex, norms, bf16_store, **KW)
    fwd = r3.normed_stack(s, L, x0, w_r, idx, *ex, dev_status=st, **norms, **KW)
    out = r3.normed_stack_train(s, L, x0, w_r, idx, *ex, dy, expert_grads=True, dev_status=st, **norms, **KW)
    assert st.item() == 0
    x_out, dlogits, dx0, dw_r, dw_pre, dw_post, dgate, dwg, dwu, dwd = out
    assert torch.equal(fwd, x_out)
    assert rel(x_out, ref["x_out"]) < 2e-2 and rel(dx0, ref["dx0"]) < 2e-2
    for l in range(L):
        if K > 1:
            assert rel(dlogits[l], ref["ds"][l]) < 2e-2 and rel(dw_r[l], ref["dw_r"][l]) < 2e-2
        assert rel(dw_pre[l], ref["dw_pre"][l]) < 2e-2
        if post:
            assert rel(dw_post[l], ref["dw_post"][l]) < 2e-2
        if gated:
            assert rel(dgate[l], ref["dgate"][l]) < 2e-2
        for k, got in enumerate((dwg, dwu, dwd)):
            want = np.stack([ref["dw_experts"][l][e][k] for e in range(E)])
            assert rel(got[l], want) < 2e-2
    assert (dw_post is None) == (not post) and (dgate is None) == (not gated)


def test_float32_forward(r3):
    w, x0, dy, w_r, idx, ex, norms = build(40, 128, 8, 2, 64, 2, act="f32")
    s = r3.shape_of(w)
    ref = oracle(x0, dy, w_r, idx, ex, norms, None, **KW)
    assert rel(r3.normed_stack(s, 2, x0, w_r, idx, *ex, **norms, **KW), ref["x_out"]) < 2e-5
    with pytest.raises(r3.R3Error) as e:
        r3.normed_stack_train(s, 2, x0, w_r, idx, *ex, dy, **norms, **KW)
    assert e.value.code == r3.R3_ERR_UNSUPPORTED


def handle(r3, ex, L, **kw):
    return r3.AdamW([e[l] for l in range(L) for e in ex], **kw)


@pytest.mark.parametrize("kw", [dict(state_bits=8), dict(state_bits=32, masters=True)])
def test_optimiser_in_the_chain_is_the_optimiser_behind_it(r3, kw):
    """The expert weights' steps block by block give the bits of one step over all blocks' gradients."""
    T, d, E, K, F, L = 90, 128, 8, 2, 64, 3
    w, x0, dy, w_r, idx, ex, norms = build(T, d, E, K, F, L)
    s = r3.shape_of(w)
    other = [e.clone() for e in ex]
    one, two = handle(r3, ex, L, weight_decay=0.1, **kw), handle(r3, other, L, weight_decay=0.1, **kw)
    gs = torch.tensor([0.5], device="cuda")
    for step in (1, 2):
        a = r3.normed_stack_train(s, L, x0, w_r, idx, *ex, dy, optimiser=one, step=step, lr=1e-2,
                                  grad_scale=gs, **norms)
        b = r3.normed_stack_train(s, L, x0, w_r, idx, *other, dy, expert_grads=True, **norms)
        for p, q in zip(a[:7], b[:7]):
            assert torch.equal(p, q)
        for p, q in zip(a[7:], b[7:]):
            assert torch.equal(p, q[0])                       # block 0's gradients are the last
        two.set_grads([q[l] for l in range(L) for q in b[7:]])
        two.step(step, 1e-2, grad_scale=gs)
        for p, q in zip(ex, other):
            assert torch.equal(p, q)
        for p, q in zip(one.exp_avg + one.exp_avg_sq, two.exp_avg + two.exp_avg_sq):
            assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))


def test_update_step_end_to_end(r3):
    """One Update step: rollout record, forward, head, log probabilities, their gradient, the chain with
    the experts' optimiser, and one for the router, the norms and the head.  Gradients against float64."""
    T, d, E, K, F, L, V = 120, 128, 8, 2, 64, 2, 517
    w, x0, _, w_r, idx, ex, norms = build(T, d, E, K, F, L, seed=4)
    s = r3.shape_of(w)
    g = torch.Generator().manual_seed(8)
    head = (torch.randn((V, d), generator=g) * 0.1).to(BF).cuda()
    ids = torch.randint(0, V, (T,), generator=g).cuda()
    ids[::7] = -1                                             # prompt tokens
    adv = torch.randn(T, generator=g).cuda()
    n = int((ids >= 0).sum())
    x_l = r3.normed_stack(s, L, x0, w_r, idx, *ex, **norms)
    logits = x_l.float() @ head.float().T
    logp, ent, stats, _, _ = r3.token_logprobs(logits, ids, want_entropy=True, want_stats=True)
    dlogp = torch.where(ids >= 0, -adv / n, torch.zeros_like(adv))
    dent = torch.full_like(adv, -0.01 / n)
    dlogits = r3.token_logprobs_bwd(logits, ids, stats, dlogp, entropy=ent, dentropy=dent)
    dy = (dlogits @ head.float()).to(BF)
    opt = handle(r3, ex, L, state_bits=8)
    small = [w_r, norms["w_pre"], norms["w_post"], norms["gate"]]
    before = [e.clone() for e in ex + small]
    x_out, ds, dx0, dw_r, dw_pre, dw_post, dgate, *_ = r3.normed_stack_train(
        s, L, x0, w_r, idx, *ex, dy, optimiser=opt, step=1, lr=1e-3, **norms)
    rest = r3.AdamW(small, [dw_r, dw_pre, dw_post, dgate], weight_decay=[0.1, 0.0, 0.0, 0.0])
    rest.step(1, 1e-3)
    assert torch.equal(x_out, x_l)
    # ---- the same in float64, from the inputs alone
    snap = dict(zip(("w_pre", "w_post", "gate"), before[4:]))
    ref = oracle(x0, dy, before[3], idx, before[:3], snap, bf16_store)
    z = ref["x_out"] @ f64(head).T
    f = U.token_logprobs(z, ids.cpu().numpy())
    # a logit is off by the head's row times x_L's error (2e-2 of its largest, over d columns at random)
    far = 2e-2 * np.abs(ref["x_out"]).max() * 0.1 * np.sqrt(d) * 5
    assert np.abs(f64(logp) - f["logp"]).max() < 2 * far and np.abs(f64(ent) - f["entropy"]).max() < 2 * far
    dz = U.token_logprobs_bwd(f64(logits), ids.cpu().numpy(), f64(dlogp), f64(dent))
    # within a float32 gradient's own error (see the log-probability tests) and dy's rounding
    assert np.abs(f64(dlogits) - dz).max() < 4e-5 * (np.abs(f64(dlogp)).max() + 50 * 0.01 / n)
    assert rel(dy, dz @ f64(head)) < 2.0 ** -7
    assert rel(dx0, ref["dx0"]) < 2e-2
    for l in range(L):
        assert rel(dw_r[l], ref["dw_r"][l]) < 2e-2 and rel(dw_post[l], ref["dw_post"][l]) < 2e-2
    # every weight with a gradient has moved, by at most the first step's lr (1 + eps) and the decay
    for p, q in zip(ex + small, before):
        moved = (p.float() - q.float()).abs()
        assert moved.max() > 0
        assert moved.max() <= 1e-3 * 1.01 + 1e-4 * q.float().abs().max() + 2.0 ** -8 * q.float().abs().max()
    # the step's new log probabilities against the old ones: what Eq. (kl) is fed
    again = r3.normed_stack(s, L, x0, w_r, idx, *ex, **norms).float() @ head.float().T
    new = r3.token_logprobs(again, ids)[0]
    kept = ids >= 0
    pa, pb = new[kept].exp(), logp[kept].exp()
    kl, _ = r3.prob_discrepancy(pa, pb, [2.0])
    want = D.kl_k3(f64(pa), f64(pb))
    assert abs(kl.item() - want) <= 1e-5 * want + 1e-12       # the estimate's own error


def test_captured_step_replays(r3):
    T, d, E, K, F, L = 64, 128, 8, 2, 64, 2
    w, x0, dy, w_r, idx, ex, norms = build(T, d, E, K, F, L)
    s = r3.shape_of(w)
    other = [e.clone() for e in ex]
    one, two = handle(r3, ex, L, state_bits=8), handle(r3, other, L, state_bits=8)
    ws = r3.workspace(r3.lib.r3_normed_stack_train_workspace_bytes(__import__("ctypes").byref(s), L), "cuda")
    scalars = torch.tensor(one.scalars(1, 1e-2), device="cuda")
    warm = [e.clone() for e in ex]                            # the first call outside a capture
    r3.normed_stack_train(s, L, x0, w_r, idx, *warm, dy, ws=ws, **norms)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = r3.normed_stack_train(s, L, x0, w_r, idx, *ex, dy, optimiser=one, step=1, lr=0.0,
                                    scalars=scalars, ws=ws, **norms)
    for step, lr in ((1, 1e-2), (2, 5e-3)):
        scalars.copy_(torch.tensor(one.scalars(step, lr)))
        graph.replay()
        want = r3.normed_stack_train(s, L, x0, w_r, idx, *other, dy, optimiser=two, step=step, lr=lr, **norms)
        torch.cuda.synchronize()
        for p, q in zip(out[:7], want[:7]):
            assert torch.equal(p, q)
        for p, q in zip(ex, other):
            assert torch.equal(p, q)


def test_one_block_of_the_stack_workload(r3):
    """A block of 4096 tokens at the paper-like layer shape against the operators called one by one."""
    w = synth.WORKLOADS["c2_layer_bf16"]
    x0, dy = synth.activations(w, "cuda"), synth.upstream_grad(w, "cuda")
    w_r = synth.router_weight(w, "cuda")
    ex = synth.expert_weights(w, "cuda")
    rng = np.random.default_rng(0)
    idx = torch.from_numpy(np.argsort(rng.random((w.T, w.E)), axis=1)[:, :w.K].copy()).to(torch.uint8).cuda()
    pre, post, gate = (1 + 0.2 * torch.randn(w.d, device="cuda") for _ in range(3))
    s = r3.shape_of(w)
    out = r3.normed_stack_train(s, 1, x0, w_r[None], idx[None], *(e[None] for e in ex), dy, w_pre=pre[None],
                                w_post=post[None], gate=gate[None])
    _, h = r3.norm_residual(x0, w_pre=pre)
    y = r3.replay_layer(s, h, w_r, idx, *ex, dy)[0]
    x1, _ = r3.norm_residual(x0, y, w_post=post, gate=gate)
    assert torch.equal(out[0], x1)
    dres, dyl, dw_post, dgate, _ = r3.norm_residual_bwd(x1, y, dy, w_post=post, gate=gate)
    _, ds, dh, dw_r = r3.replay_layer_train(s, h, w_r, idx, *ex, dyl)
    dx, _, _, _, dw_pre = r3.norm_residual_bwd(x0, None, dres, dh, w_pre=pre)
    for a, b in zip((out[1][0], out[2], out[3][0], out[4][0], out[5][0], out[6][0]),
                    (ds, dx, dw_r, dw_pre, dw_post, dgate)):
        assert torch.equal(a, b)


def test_wrong_optimisers_are_refused(r3):
    w, x0, dy, w_r, idx, ex, norms = build(20, 64, 4, 2, 64, 2)
    s = r3.shape_of(w)
    run = lambda opt: r3.normed_stack_train(s, 2, x0, w_r, idx, *ex, dy, optimiser=opt, step=1, lr=1e-3, **norms)
    keep = [e.clone() for e in ex]
    with pytest.raises(ValueError):
        run(handle(r3, ex, 1))
    swapped = r3.AdamW([e[l] for l in (1, 0) for e in ex])
    with pytest.raises(r3.R3Error) as e:
        run(swapped)                                          # block 1's weights in block 0's place
    assert e.value.code == r3.R3_ERR_INVALID_ARG
    with pytest.raises(r3.R3Error):
        run(handle(r3, [e.clone() for e in ex], 2))           # other tensors
    assert all(torch.equal(a, b) for a, b in zip(ex, keep))


def test_without_rows(r3):
    """A rank whose batch is empty: gradients of zero, untouched weights and states."""
    T, d, E, K, F, L = 8, 64, 4, 2, 64, 2
    w, x0, dy, w_r, idx, ex, norms = build(T, d, E, K, F, L)
    s = r3.make_shape(0, d, E, K, F)
    o = handle(r3, ex, L, state_bits=32)
    before = [e.clone() for e in ex]
    none = torch.empty((0, d), dtype=BF, device="cuda")
    junk = torch.full((1 << 20,), 7.0, device="cuda")         # what an allocation may find
    del junk
    assert r3.normed_stack(s, L, none, w_r, idx[:, :0], *ex, **norms).shape == (0, d)
    for kw in (dict(expert_grads=True), dict(optimiser=o, step=1, lr=0.1)):
        out = r3.normed_stack_train(s, L, none, w_r, idx[:, :0], *ex, none, **kw, **norms)
        for t in out:
            assert not t.float().any()
    for p, q in zip(ex, before):
        assert torch.equal(p, q)
    assert not any(t.any() for t in o.exp_avg + o.exp_avg_sq)


def test_wrong_rows_are_refused(r3):
    w, x0, dy, w_r, idx, ex, norms = build(12, 64, 4, 2, 64, 1)
    s = r3.shape_of(w)
    for bad in (x0[:11], x0.float(), x0.cpu()):
        with pytest.raises(ValueError):
            r3.normed_stack(s, 1, bad, w_r, idx, *ex, **norms)
        with pytest.raises(ValueError):
            r3.normed_stack_train(s, 1, x0, w_r, idx, *ex, bad, **norms)
    with pytest.raises(ValueError):
        r3.normed_stack(s, 1, x0, w_r, idx, *ex, x_out=x0[:11], **norms)


@pytest.mark.parametrize("kw", [dict(state_bits=8), dict(state_bits=32, masters=True)])
@pytest.mark.parametrize("case", ["word from before", "bad record", "bad record, no word"])
def test_no_step_after_an_error(r3, case, kw):
    """An error that stands in dev_status, or that a block reports in this call, leaves weights, masters and
    states as they were; the same call without it steps."""
    T, d, E, K, F, L = 50, 128, 8, 2, 64, 2
    w, x0, dy, w_r, idx, ex, norms = build(T, d, E, K, F, L)
    s, opt = r3.shape_of(w), handle(r3, ex, L, **kw)
    held = ex + opt.exp_avg + opt.exp_avg_sq + (opt.masters or []) + (opt.exp_avg_scale or [])
    held = [t.detach().view(torch.uint8) for t in held]
    before = [t.clone() for t in held]
    st = r3.new_status("cuda")
    record = idx.clone()
    if case == "word from before":
        st.fill_(r3.DEV_TIMEOUT)
    else:
        record[0, 7, 1] = E                                   # the first block's: its backward is the last
    word = None if case.endswith("no word") else st
    r3.normed_stack_train(s, L, x0, w_r, record, *ex, dy, optimiser=opt, step=1, lr=1e-2, dev_status=word, **norms)
    if word is not None:
        assert st.item() == (r3.DEV_TIMEOUT if case == "word from before" else r3.DEV_BAD_INDEX)
    assert all(torch.equal(p, q) for p, q in zip(before, held))
    st.zero_()
    r3.normed_stack_train(s, L, x0, w_r, idx, *ex, dy, optimiser=opt, step=1, lr=1e-2, dev_status=word, **norms)
    assert st.item() == 0 and not any(torch.equal(p, q) for p, q in zip(before, held))
