"""The orthogonalised update on the GPU against the float64 oracle.

Tolerances.  One fp16 product (products = 1): the kernel rounds operands where the oracle's fp16 model rounds
them, so its error is the model's, which the oracle gives for each input; sums in float32 move a value across
a rounding border now and then, which exchanges one rounding error for another of the same size.  Bound:
1.5 times the model's root mean square, twice its maximum, and half a step of the result's type.
Three products: the errors stand at the same places, in the operands and sums of the same products, and reach
the result in the same way (to first order linearly: a step's error in a weak direction grows up to 3.4445
fold per later step, which for a square matrix of full rank is 100 times its share of the result, so no bound
relative to the result alone holds).  What differs is their size: an fp16 operand is off by 2^-11 at most and
2^-13 at least in root mean square (a relative rounding error is uniform within 2^-12 to 2^-11 of the value),
two planes by 2^-22, the dropped lo lo term by 2^-22; accumulation adds 16 products at a time to a running sum
of 24 bits and drops what lies below: 2^-23 for the sum and, their signs being mixed, sqrt(16) 2^-24 for the
products, less than 2^-22 for each of K / 16 additions: together e = 2^-20 + K 2^-26.  So the bound is that of
one product times e / 2^-13.  What the model leaves out is X's own rounding as it is carried, which only counts
here: per step an element's two terms, up to 3.4445 and 2.8 of it, are added in float32 and kept in two planes,
7 2^-24 + 2^-22 < 2^-20.5 of X's rms, spread over all directions, and a later step lets an error grow by the
largest slope of a s + b s^3 + c s^5 at most: the sum of 2^-20.5 rms(X_k) times the slopes behind step k, and
eight times that for the largest of an array of such errors (a million normal ones stay below five)."""
import numpy as np
import pytest
import torch

from oracle import r3_muon_oracle as O
from tests.helpers import f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def matrix(rows, cols, seed=0, kind="full", B=1):
    g = torch.Generator().manual_seed(seed + 7 * rows + cols)
    x = torch.randn((B, rows, cols), generator=g)
    if kind == "full":
        return x * 1e-3
    r = max(1, min(rows, cols) // 16)
    low = torch.randn((B, rows, r), generator=g) @ torch.randn((B, r, cols), generator=g)
    return (low + (0.01 if kind == "decay" else 1e-4) * x) * 1e-3


def rms(x):
    return float(np.sqrt((np.asarray(x) ** 2).mean()))


def carried(x, steps, coefs, eps):
    grown = 0.0
    for k in range(steps):
        a, b, c = O.QUINTIC if coefs is None else coefs[k]
        s2 = np.linspace(0, 1.3, 200) ** 2
        grown = grown * np.abs(a + 3 * b * s2 + 5 * c * s2 * s2).max()
        grown += 2.0 ** -20.5 * rms(O.iterate(x, k + 1, coefs, eps))
    return grown


def check(got, x, products, steps=5, coefs=None, eps=1e-7):
    """got, x: [rows, cols] tensors."""
    want = O.iterate(f64(x), steps, coefs, eps)
    err = f64(got) - want
    model = O.iterate(f64(x), steps, coefs, eps, operand=O.half_operand) - want
    share = 1.0 if products == 1 else 2.0 ** 13 * (2.0 ** -20 + max(x.shape) * 2.0 ** -26)
    soft, hard = share * 1.5 * rms(model), share * 2 * np.abs(model).max()
    if products == 3:
        own = carried(f64(x), steps, coefs, eps)
        soft, hard = soft + own, hard + 8 * own
    half = torch.finfo(got.dtype).eps / 2
    soft = np.hypot(soft, half * rms(want)) + 2.0 ** -22 * rms(want)
    assert rms(err) <= soft
    assert (np.abs(err) <= hard + half * np.abs(want) + 2.0 ** -20 * np.abs(want).max()).all()


SHAPES = [(1, 1), (1, 9), (9, 1), (2, 3), (8, 8), (31, 33), (64, 64), (65, 127), (128, 520), (520, 128), (129, 256),
          (256, 257), (300, 300), (301, 513), (513, 301), (640, 264)]


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize_against_oracle(r3, rows, cols, products):
    for kind, B in (("full", 1), ("decay", 3)):
        x = matrix(rows, cols, 1, kind, B)
        for dtype in (F32, BF):
            st = r3.new_status("cuda")
            given = x.to(dtype)
            got = r3.orthogonalize(given.cuda(), out_dtype=F32, products=products, dev_status=st)
            assert st.item() == 0
            for i in range(B):
                check(got[i].cpu(), given[i], products)
    got = r3.orthogonalize(x[0].to(BF).cuda())                    # a matrix without a batch, bf16 to bf16
    assert got.dtype == BF and got.shape == (rows, cols)
    check(got.cpu(), x[0].to(BF), 1)


def test_low_rank_steps_coefficients_and_eps(r3):
    x = matrix(200, 320, 2, "low")
    for steps, coefs in ((1, None), (5, None), (3, [(2.0, -1.5, 0.5)] * 3), (6, [(4.0, -6.8, 2.9)] + [(2, -1.5, 0.5)] * 5)):
        for products in (1, 3):
            got = r3.orthogonalize(x.cuda(), steps=steps, coefficients=coefs, products=products, eps=1e-3)
            check(got[0].cpu(), x[0], products, steps, coefs, 1e-3)


@pytest.mark.parametrize("steps,coefs", [(1, None), (2, None), (5, None), (2, [(2.0, -1.5, 0.5), (5.0, -6.0, 2.0)]),
                                         (4, [(2.0, -1.5, 0.5)] * 4)])
@pytest.mark.parametrize("rows,cols", [(200, 320), (320, 200), (96, 100)])
def test_bf16_results_whose_last_step_needs_less(r3, rows, cols, steps, coefs):
    """A bf16 result takes the last step from X rounded to fp16, where that step's a is at most 4: a 2^-11 of an
    element at most, a 2^-13 rms at least and 2^-12 at most, against the rounding's 2^-9 and 2^-9 / sqrt(3)."""
    for kind in ("full", "low"):
        x = matrix(rows, cols, 14, kind).to(BF)
        got = r3.orthogonalize(x.cuda(), steps=steps, coefficients=coefs)[0].cpu()
        want = O.iterate(f64(x[0]), steps, coefs)
        model = O.iterate(f64(x[0]), steps, coefs, operand=O.half_operand) - want
        before = O.iterate(f64(x[0]), steps - 1, coefs) if steps > 1 else 0 * want
        err, half = f64(got) - want, torch.finfo(BF).eps / 2
        assert rms(err) <= np.sqrt((1.5 * rms(model)) ** 2 + (half * rms(want)) ** 2 + (4 * 2.0 ** -12 * rms(before)) ** 2)
        assert (np.abs(err) <= (2 * np.abs(model).max() + 4 * 2.0 ** -11 * np.abs(before).max()) * (1 + half)
                + half * np.abs(want) + 2.0 ** -20 * np.abs(want).max()).all()


def test_many_small_matrices_and_one_large(r3):
    x = matrix(24, 40, 3, "full", 700)
    got = r3.orthogonalize(x.cuda(), products=3)
    for i in (0, 1, 333, 699):
        check(got[i].cpu(), x[i], 3)
    x = matrix(1100, 900, 4)
    for products in (1, 3):
        check(r3.orthogonalize(x.cuda(), products=products)[0].cpu(), x[0], products)


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("B,rows,cols", [(24, 300, 520), (24, 769, 500), (12, 769, 513), (40, 249, 2000),
                                         (40, 2000, 249), (8, 300, 6001), (8, 6001, 300)])
def test_enough_tiles_for_wide_ones(r3, B, rows, cols, products):
    """So many matrices take tiles of 256 columns, the long ones with their sums in parts; the first and the last
    are compared, and all of them with what they give elsewhere in the batch."""
    x = matrix(rows, cols, 13, "decay", B)
    x[B // 2] = x[0]
    st = r3.new_status("cuda")
    got = r3.orthogonalize(x.cuda(), products=products, dev_status=st)
    assert st.item() == 0 and torch.equal(got[B // 2], got[0])
    for i in (0, B - 1):
        check(got[i].cpu(), x[i], products)


def test_batches_in_parts(r3):
    """More matrices than the workspace holds at once give what each gives alone."""
    x = matrix(768, 1024, 5, "decay", 90).cuda()
    need = r3.lib.r3_orthogonalize_workspace_bytes(r3.Orthogonal(90, 768, 1024, 1, 1, 5, 1, 1e-7, None))
    assert need < 90 * 768 * 1024 * 12
    got = r3.orthogonalize(x.to(BF))
    for i in (0, 40, 89):
        assert torch.equal(got[i], r3.orthogonalize(x[i].to(BF)))


def test_zeros_and_what_is_not_finite(r3):
    x = matrix(70, 130, 6, "full", 5)
    x[1] = 0
    x[2, 3, 4] = float("nan")
    x[3, 69, 129] = float("inf")
    clean = r3.orthogonalize(x[:1].cuda()), r3.orthogonalize(x[4:].cuda())
    for products in (1, 3):
        got = r3.orthogonalize(x.cuda(), products=products)
        assert not got[1].any() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    got = r3.orthogonalize(x.cuda())
    assert torch.equal(got[0], clean[0][0]) and torch.equal(got[4], clean[1][0])
    for size in (1e-30, 1e30):                                    # squares beyond float32
        check(r3.orthogonalize((x[0] * size).cuda(), eps=0.0).cpu(), x[0], 3, eps=0.0)
    assert r3.orthogonalize(torch.zeros(0, 4, 8).cuda()).shape == (0, 4, 8)


def test_in_place_repeats_streams_and_graphs(r3):
    x = matrix(264, 392, 7, "decay", 3).cuda()
    want = r3.orthogonalize(x, products=1)
    ws = r3.workspace(1 << 26, "cuda")
    ws.fill_(255)                                                 # NaN in whatever is not written first
    for _ in range(3):
        assert torch.equal(want, r3.orthogonalize(x, products=1, ws=ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = r3.orthogonalize(x, products=1, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(want, got)
    y = x.clone()
    assert r3.orthogonalize(y, y, products=1) is y and torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = r3.orthogonalize(x, products=1)
    for _ in range(2):
        x.add_(1e-4)
        graph.replay()
        assert torch.equal(held, r3.orthogonalize(x, products=1))


# ---- the step -----------------------------------------------------------------------------------------
def make(r3, shapes, dtype, grad, masters, seed=0, **kw):
    g = torch.Generator().manual_seed(seed)
    w = [torch.randn(s, generator=g) * 0.05 for s in shapes]
    grads = [matrix(s[-2], s[-1], seed, "decay", int(np.prod(s[:-2]))).reshape(s).to(grad).cuda() for s in shapes]
    bufs = [matrix(s[-2], s[-1], seed + 1, "full", int(np.prod(s[:-2]))).reshape(s).cuda() for s in shapes]
    return r3.Muon([x.to(dtype).cuda() for x in w], grads, masters=[x.cuda() for x in w] if masters else None,
                   momentum_buffers=bufs, **kw)


def flat(t):
    return t.reshape(-1, *t.shape[-2:]).cpu()


def check_step(opt, before, lr, scales, decays, nesterov=True, mu=0.95, gs=1.0):
    """Against the oracle's step on the state before.  The iteration's error is bounded as above; the momentum
    goes through three roundings, the weight through four and that of its type."""
    p0, m0, g0, master0 = before
    products = opt._config.products
    for i, p in enumerate(opt.params):
        for j in range(flat(p).shape[0]):
            w0 = f64(flat(master0[i] if master0 else p0[i])[j])
            rows, cols = w0.shape
            want_m = mu * f64(flat(m0[i])[j]) + f64(flat(g0[i])[j]) * gs
            got_m = f64(flat(opt.momentum_buffers[i])[j])
            size = mu * np.abs(f64(flat(m0[i])[j])) + np.abs(f64(flat(g0[i])[j]) * gs)
            assert (np.abs(got_m - want_m) <= 2.0 ** -22 * size).all()
            want, _ = O.step(w0, f64(flat(m0[i])[j]), f64(flat(g0[i])[j]), lr, mu, nesterov, decays[i], scales[i], gs)
            u = f64(flat(g0[i])[j]) * gs + mu * want_m if nesterov else want_m
            o = O.iterate(u)
            hard = 2 * np.abs(O.iterate(u, operand=O.half_operand) - o).max()
            if products == 3:
                hard = hard * 2.0 ** 13 * (2.0 ** -20 + max(rows, cols) * 2.0 ** -26) + 8 * carried(u, 5, None, 1e-7)
            slack = lr * scales[i] * (hard + 2.0 ** -20 * np.abs(o).max()) + 2.0 ** -22 * (np.abs(w0) + lr * scales[i] * np.abs(o))
            if master0:
                assert (np.abs(f64(flat(opt.masters[i])[j]) - want) <= slack).all()
                assert torch.equal(flat(p)[j], flat(opt.masters[i])[j].to(p.dtype))
            else:
                half = torch.finfo(p.dtype).eps / 2
                assert (np.abs(f64(flat(p)[j]) - want) <= slack + half * (np.abs(want) + slack)).all()


def state(opt):
    return tuple([t.clone() for t in ts] if ts is not None else None
                 for ts in (opt.params, opt.momentum_buffers, opt.grads, opt.masters))


@pytest.mark.parametrize("dtype,grad,masters", [(F32, F32, False), (F32, BF, False), (BF, F32, False),
                                                (BF, BF, False), (BF, F32, True), (BF, BF, True)])
@pytest.mark.parametrize("nesterov", [True, False])
def test_step_against_oracle(r3, dtype, grad, masters, nesterov):
    shapes = [(3, 128, 264), (40, 72), (3, 264, 128), (2, 2, 128, 264), (33, 7), (40, 72), (1, 1), (0, 8, 8)]
    decays = [0.0, 0.1, 0.2, 0.0, 0.3, 0.0, 0.1, 0.0]
    opt = make(r3, shapes, dtype, grad, masters, 3, nesterov=nesterov, weight_decay=decays,
               scale=["spectral", "rms", "spectral", 2.0, 0.5, "spectral", 1.0, 1.0])
    scales = [1.0, 0.2 * 72 ** 0.5, (264 / 128) ** 0.5, 2.0, 0.5, 1.0, 1.0, 1.0]
    for lr, gs in ((0.02, None), (0.1, 0.37)):
        before = state(opt)
        st = r3.new_status("cuda")
        opt.step(lr, grad_scale=None if gs is None else torch.full((1,), gs).cuda(), dev_status=st)
        assert st.item() == 0
        check_step(opt, before, lr, scales, decays, nesterov,
                   gs=1.0 if gs is None else float(np.float32(gs)))


def test_more_stacks_than_a_launch_takes(r3):
    shapes = [(16, 24)] * 150 + [(24, 16)] * 3
    opt = make(r3, shapes, F32, F32, False, 5)
    before = state(opt)
    opt.step(0.1)
    check_step(opt, before, 0.1, [1.0] * 150 + [1.5 ** 0.5] * 3, [0.0] * 153)


def test_skipped_step_and_learning_rate_on_the_device(r3):
    for dtype, masters in ((F32, False), (BF, True)):
        opt = make(r3, [(2, 64, 96), (30, 50)], dtype, F32, masters, 6)
        before = state(opt)
        for bad in (float("inf"), float("nan")):
            opt.step(0.1, grad_scale=torch.full((1,), bad).cuda())
        for a, b in zip(before, state(opt)):
            assert a is None or all(torch.equal(x, y) for x, y in zip(a, b))
        opt.step(123.0, lr_tensor=torch.full((1,), 0.1).cuda())
        check_step(opt, before, float(np.float32(0.1)), [1.0, 1.0], [0.0, 0.0])


def test_gradient_that_is_not_finite_stays_in_its_matrix(r3):
    opt = make(r3, [(3, 64, 96)], F32, F32, False, 7)
    clean = make(r3, [(3, 64, 96)], F32, F32, False, 7)
    opt.grads[0][1, 5, 5] = float("nan")
    opt.step(0.1)
    clean.step(0.1)
    assert torch.isnan(opt.params[0][1]).all()
    for i in (0, 2):
        assert torch.equal(opt.params[0][i], clean.params[0][i])


def test_captured_step_matches_eager_ones(r3):
    a, b = (make(r3, [(3, 128, 264), (264, 40)], BF, BF, True, 8, weight_decay=0.1) for _ in range(2))
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


@pytest.mark.parametrize("rows,cols,size", [(8, 8, 1e-34), (129, 256, 1e-35)])
def test_norms_whose_inverse_passes_float32(r3, rows, cols, size):
    """eps below 4e-36 counts as that: 2^10 over the norm alone would be infinite."""
    x = (matrix(rows, cols, 12)[0].double() * size).float()
    assert 1024 / np.linalg.norm(f64(x)) > 3.4e38
    check(r3.orthogonalize(x.cuda(), eps=0.0).cpu(), x, 3, eps=float(np.float32(4e-36)))
