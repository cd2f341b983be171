"""The momentum step over matrices that go through memory between their products (a side above 128, or one above
2048): every type, rows of any length, several shapes and many stacks in a launch, options and graphs.

Tolerances.  The momentum goes through three roundings, a weight through four and that of its type.  The update: three
products as in test_gpu_muon_precision (twice what its model of the planes loses, twice the error of float32 products,
and the drift of sums that drop their last places); one product 1.5 times its model's root mean square, and a bf16
weight without a master has X rounded in front of the last step, which that step's a multiplies."""
import numpy as np
import pytest
import torch

from oracle import r3_muon_oracle as O
from tests.helpers import f64
from tests.test_gpu_muon import flat, make, state

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def rms(x):
    return float(np.sqrt((np.asarray(x) ** 2).mean()))


def check_step(opt, before, lr, scales, decays, nesterov=True, mu=0.95, gs=1.0):
    p0, m0, g0, master0 = before
    for i, p in enumerate(opt.params):
        for j in {0, flat(p).shape[0] - 1}:
            w0 = f64(flat(master0[i] if master0 else p0[i])[j])
            m, g = f64(flat(m0[i])[j]), f64(flat(g0[i])[j]) * gs
            want_m = mu * m + g
            assert (np.abs(f64(flat(opt.momentum_buffers[i])[j]) - want_m) <= 2.0 ** -22 * (mu * np.abs(m) + np.abs(g))).all()
            u = g + mu * want_m if nesterov else want_m
            o = O.iterate(u)
            want = w0 * (1 - lr * decays[i]) - lr * scales[i] * o
            if opt._config.products == 3:
                loss = 2 * rms(O.iterate_planes(u) - o) + 2 * rms(O.iterate_f32(u) - o) + rms(O.iterate_short(u) - o)
            else:
                last = O.iterate(u, 4)
                loss = 1.5 * rms(O.iterate(u, operand=O.scaled_operand) - o) + O.QUINTIC[0] * rms(O.scaled_operand(last) - last)
            loss = lr * scales[i] * (loss + 2.0 ** -20 * rms(o)) + 2.0 ** -22 * rms(np.abs(w0) + lr * scales[i] * np.abs(o))
            if master0:
                assert rms(f64(flat(opt.masters[i])[j]) - want) <= loss
                assert torch.equal(flat(p)[j], flat(opt.masters[i])[j].to(p.dtype))
            else:
                assert rms(f64(flat(p)[j]) - want) <= loss + torch.finfo(p.dtype).eps / 2 * (rms(want) + loss)


SHAPES = [(3, 136, 264), (201, 333), (2, 333, 201), (129, 130), (2, 2, 136, 264), (520, 130), (4, 2056), (8, 8), (300, 1000)]
DECAYS = [0.0, 0.1, 0.2, 0.0, 0.3, 0.0, 0.1, 0.1, 0.0]
SCALES = [1.0, 2.0, 0.5, 1.0, 3.0, 1.0, 1.0, 1.0, 0.7]


@pytest.mark.parametrize("dtype,grad,masters", [(F32, F32, False), (F32, BF, False), (BF, F32, False),
                                                (BF, BF, False), (BF, F32, True), (BF, BF, True)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step_against_oracle(r3, dtype, grad, masters, nesterov):
    """Seven shapes, more than a launch takes, in stacks that lie apart; a second step with a gradient's scale."""
    opt = make(r3, SHAPES, dtype, grad, masters, 13, nesterov=nesterov, weight_decay=DECAYS, scale=SCALES)
    for lr, gs in ((0.02, None), (1.0, 0.37)):
        before = state(opt)
        st = r3.new_status("cuda")
        opt.step(lr, grad_scale=None if gs is None else torch.full((1,), gs).cuda(), dev_status=st)
        assert st.item() == 0
        check_step(opt, before, lr, SCALES, DECAYS, nesterov, gs=1.0 if gs is None else float(np.float32(gs)))


@pytest.mark.parametrize("dtype,masters", [(F32, False), (BF, True), (BF, False)])
def test_more_stacks_and_matrices_than_a_round_takes(r3, dtype, masters):
    for shapes in ([(130, 140)] * 70 + [(140, 130)] * 3, [(40, 770, 1000), (30, 1000, 770), (130, 130)]):
        opt = make(r3, shapes, dtype, F32, masters, 15, scale=1.0)
        before = state(opt)
        opt.step(0.1)
        check_step(opt, before, 0.1, [1.0] * len(shapes), [0.0] * len(shapes))


@pytest.mark.parametrize("dtype,masters", [(F32, False), (BF, True), (BF, False)])
def test_skipped_step_and_learning_rate_on_the_device(r3, dtype, masters):
    opt = make(r3, [(2, 150, 296), (301, 150)], dtype, F32, masters, 16, scale=1.0)
    before = state(opt)
    for bad in (float("inf"), float("nan")):
        opt.step(0.1, grad_scale=torch.full((1,), bad).cuda())
    for a, b in zip(before, state(opt)):
        assert a is None or all(torch.equal(x, y) for x, y in zip(a, b))
    opt.step(123.0, lr_tensor=torch.full((1,), 0.1).cuda())
    check_step(opt, before, float(np.float32(0.1)), [1.0, 1.0], [0.0, 0.0])


def test_gradient_that_is_not_finite_stays_in_its_matrix(r3):
    for bad in (float("nan"), float("inf")):
        opt, clean = (make(r3, [(3, 150, 200), (200, 136)], F32, F32, False, 17) for _ in range(2))
        opt.grads[0][1, 149, 199] = bad
        opt.step(0.1)
        clean.step(0.1)
        assert torch.isnan(opt.params[0][1]).all()
        for i in (0, 2):
            assert torch.equal(opt.params[0][i], clean.params[0][i])
        assert torch.equal(opt.params[1], clean.params[1])


def test_captured_step_matches_eager_ones_and_repeats(r3):
    a, b = (make(r3, [(3, 136, 264), (264, 140), (301, 513), (40, 64)], BF, BF, True, 18, weight_decay=0.1) for _ in range(2))
    lr = torch.full((1,), 0.05).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(0.0, lr_tensor=lr)
    for value in (0.05, 0.02):
        lr.fill_(value)
        graph.replay()
        b.step(value)
        for x, y in zip(state(a), state(b)):
            assert all(torch.equal(s, t) for s, t in zip(x, y))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.step(0.01, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    b.step(0.01)
    assert all(torch.equal(s, t) for s, t in zip(a.params, b.params))


@pytest.mark.parametrize("coefs", [(3.74, 0, 0), (3.76, 0, 0), (16.0, 0, 0), (1.0, -30.0, 20.0), (1.0, 50.0, -37.0)])
@pytest.mark.parametrize("rows,cols", [(8, 8), (100, 300), (140, 150), (300, 130)])
def test_coefficients_up_to_what_fp16_holds(r3, coefs, rows, cols):
    """A matrix of one element, whose singular value is one, and a full one: the operands' scale leaves room for the
    largest iterates that are taken."""
    x = torch.zeros((2, rows, cols))
    x[0, rows - 1, cols // 2] = 3.0
    x[1] = torch.randn((rows, cols), generator=torch.Generator().manual_seed(rows))
    for products in (1, 3):
        got = r3.orthogonalize(x.cuda(), steps=1, coefficients=coefs, products=products).cpu()
        for i in range(2):
            want = O.iterate(f64(x[i]), 1, [coefs])
            # to first order: X is rounded twice in A, A once, so seven roundings stand in A A, one in B, one in X, each
            # 2^-11 of the value at most; of two planes 2^-22, and 2^-22 for the lo lo terms of four products; the sums
            # of four products drop 2^-21 of themselves each
            size = O.iterate(np.abs(f64(x[i])), 1, [np.abs(coefs)])
            off = (9.0 * 2.0 ** -11 if products == 1 else 13.0 * 2.0 ** -22) * 1.01 + 2.0 ** -19
            assert (np.abs(f64(got[i]) - want) <= off * size + 2.0 ** -30).all()
