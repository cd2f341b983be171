"""Calls with stream= another stream than the current one: what the binding allocates for them is that
stream's memory, and new outputs are known to the stream that was current."""
import contextlib
import inspect
import re

import pytest
import torch


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import build
    build.build()
    from paper_2510_11370_b200 import r3 as mod
    return mod


class FakeTensor(torch.Tensor):
    @staticmethod
    def __new__(cls, log):
        t = torch.Tensor._make_subclass(cls, torch.zeros(1))
        t.log = log
        return t

    def record_stream(self, stream):
        self.log.append((id(self), stream))


class FakeStream:
    device = torch.device("cpu")


def test_allocations_belong_to_the_given_stream(r3, monkeypatch):
    now = [FakeStream()]
    home, side, used = now[0], FakeStream(), []

    @contextlib.contextmanager
    def enter(stream):
        now.append(stream)
        yield
        now.pop()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.cuda, "stream", enter)
    made_on = []

    @r3._in_order
    def by_name(given, *, want=True, stream=None):
        made_on.append(now[-1])
        return given, FakeTensor(used), None

    @r3._in_order
    def by_place(given, stream=None):
        made_on.append(now[-1])
        return FakeTensor(used)

    given = FakeTensor(used)
    by_name(given)
    by_place(given)
    by_name(given, stream=home)
    assert made_on == [home] * 3 and not used
    _, new, _ = by_name(given, stream=side)
    assert made_on[-1] is side and used == [(id(new), home)]       # not the caller's own tensor
    other = by_place(given, side)
    assert made_on[-1] is side and used[1:] == [(id(other), home)]
    by_place(given, stream=side)
    assert made_on[-1] is side and now == [home]


def test_every_call_that_allocates_is_ordered(r3):
    allocates = re.compile(r"torch\.(empty|zeros|full|as_tensor)|workspace\(|new_empty|\bnew\(")
    seen = 0
    for name, fn in inspect.getmembers(r3, inspect.isfunction):
        if name.startswith("_") or "stream" not in inspect.signature(fn).parameters:
            continue
        if allocates.search(inspect.getsource(fn)):
            seen += 1
            assert hasattr(fn, "__wrapped__"), name
    assert seen >= 30


# ---------------------------------------------------------------------------------------------
def side_stream_kept_busy():
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                             # 0.1 s at the highest clock
    return side


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["norm_residual_bwd", "normed_stack", "normed_stack_train", "replay_layer"])
def test_scratch_is_not_handed_out_while_it_is_in_use(r3, monkeypatch, call):
    """A call on a stream that is behind: what the current stream allocates next, and writes at once, is
    not the call's scratch."""
    from paper_2510_11370_b200 import synth
    T, d, E, K, F, L = 300, 256, 8, 2, 128, 2
    w = synth.scaled(synth.WORKLOADS["c2_layer_bf16"], name="streams", T=T, d=d, E=E, K=K, F=F, layers=L)
    g = torch.Generator().manual_seed(3)
    x, dy = synth.activations(w).cuda(), synth.upstream_grad(w).cuda()
    w_r = torch.stack([synth.router_weight(w, layer=l) for l in range(L)]).cuda()
    ex = [torch.stack(t).cuda() for t in zip(*(synth.expert_weights(w, layer=l) for l in range(L)))]
    idx = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(L * T)])
    idx = idx.view(L, T, K).to(torch.uint8).cuda()
    vec = (1 + 0.2 * torch.randn((L, d), generator=g)).cuda()
    s = r3.shape_of(w)

    def run(**kw):
        if call == "norm_residual_bwd":
            return r3.norm_residual_bwd(x, dy, x, dy, w_post=vec[0], gate=vec[1], w_pre=vec[1], **kw)
        if call == "normed_stack":
            return (r3.normed_stack(s, L, x, w_r, idx, *ex, w_pre=vec, w_post=vec, gate=vec, **kw),)
        if call == "normed_stack_train":
            return r3.normed_stack_train(s, L, x, w_r, idx, *ex, dy, w_pre=vec, w_post=vec, gate=vec,
                                         expert_grads=True, **kw)
        return r3.replay_layer(s, x, w_r[0], idx[0], *(e[0] for e in ex), dy, **kw)

    want = [t.clone() for t in run()]
    make, scratch = r3.workspace, []

    def workspace(*a):
        t = make(*a)
        scratch.append((t.data_ptr(), t.numel()))
        return t
    monkeypatch.setattr(r3, "workspace", workspace)
    side = side_stream_kept_busy()
    got = run(stream=side)
    (at, size), = scratch
    later = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(t.data_ptr() + size <= at or at + size <= t.data_ptr() for t in later)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.gpu
def test_new_memory_is_free_of_the_current_streams_work(r3):
    """Outputs of a call on another stream are not memory that the current stream still writes."""
    logits = torch.randn((64, 1000), device="cuda")
    ids = torch.arange(64, device="cuda")
    want = r3.token_logprobs(logits, ids)[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    old = [torch.zeros(64, device="cuda") for _ in range(16)]      # written late, given back at once
    del old
    got = r3.token_logprobs(logits, ids, stream=side)[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
