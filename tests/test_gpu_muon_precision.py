"""How close float32 results of the orthogonalised update come to float32 products, and what becomes of rows and
columns that are far smaller than the others.

Tolerances, all root mean squares over the rows that are looked at.  Three products lose what the planes lose, which
the oracle's model of them gives for each input (twice that is allowed), and what sums in float32 lose.  The kernel
adds 16 products at a time and drops what lies below the sum's last place, less than 2^-23 of it, where a float32 product
rounds, 2^-24.  So of the errors of mixed signs it has twice those of the iteration in float32.  But what is dropped has
one sign: four additions make 64 of k, which are then added up in registers, so a sum of terms of one sign (the Gram
matrix's diagonal) may be short of up to 4 2^-23 = 2^-21 of itself, all of them alike, and an iteration lets that drift
grow by the slopes of its polynomial, the more the more steps there are: what it comes to is computed in 64 bits with
every product short by that much, and added.  2^-20 of the result besides, since a float32 run of few numbers may be
right by luck.  All of that is a tenth at most of what one product loses by its own model, which each test states.
One product: 1.5 times its model, the rounding of the result, and of X in front of the last step, times its a."""
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


def rms(x):
    return float(np.sqrt((np.asarray(x) ** 2).mean()))


def matrix(rows, cols, seed, B=1):
    g = torch.Generator().manual_seed(seed + 3 * rows + cols)
    return torch.randn((B, rows, cols), generator=g) * 1e-3


def three(got, x, steps, parts):
    want = O.iterate(f64(x), steps)
    loss, f32 = O.iterate_planes(f64(x), steps) - want, O.iterate_f32(f64(x), steps) - want
    drift = O.iterate_short(f64(x), steps) - want
    one = O.iterate(f64(x), steps, operand=O.scaled_operand) - want
    for part in parts:
        bound = 2 * rms(loss[part]) + 2 * rms(f32[part]) + rms(drift[part]) + 2.0 ** -20 * rms(want[part])
        assert bound < rms(one[part]) / 10
        assert rms((f64(got) - want)[part]) <= bound


@pytest.mark.parametrize("rows,cols,B", [(8, 8, 1), (31, 33, 1), (65, 127, 3), (128, 520, 1), (520, 128, 2), (40, 2048, 1),
                                         (129, 256, 1), (300, 300, 1), (301, 513, 2), (513, 301, 1), (24, 2500, 1),
                                         (769, 500, 24), (300, 2001, 12), (700, 1100, 1)])
def test_float32_results_are_those_of_float32_products(r3, rows, cols, B):
    x = matrix(rows, cols, 1, B)
    st = r3.new_status("cuda")
    got = r3.orthogonalize(x.cuda(), dev_status=st)
    assert st.item() == 0
    for i in {0, B - 1}:
        three(got[i].cpu(), x[i], 5, [np.s_[:]])


WEAK = [1e-3, 1e-5, 1e-6, 1e-7, 1e-8]


@pytest.mark.parametrize("steps", [5, 16])
@pytest.mark.parametrize("rows,cols,B", [(96, 200, 1), (200, 96, 1), (64, 1500, 2), (300, 600, 1), (600, 300, 1),
                                         (300, 520, 24)])
def test_weak_rows_keep_their_bits(r3, rows, cols, B, steps):
    """Rows (columns of a tall matrix) scaled down: float32 results hold them to float32's precision as far as 2^-49
    of the norm is below it."""
    for size in WEAK:
        x = matrix(rows, cols, 2, B)
        weak = np.s_[:9] if rows <= cols else np.s_[:, :9]
        for i in range(B):
            x[i][weak] *= size
        got = r3.orthogonalize(x.cuda(), steps=steps)
        three(got[B - 1].cpu(), x[B - 1], steps, [weak, np.s_[:]])


@pytest.mark.parametrize("rows,cols", [(96, 200), (200, 96), (300, 600), (600, 300)])
def test_weak_rows_of_bf16_results(r3, rows, cols):
    for size in WEAK:
        x = matrix(rows, cols, 3)[0]
        weak = np.s_[:9] if rows <= cols else np.s_[:, :9]
        x[weak] *= size
        x = x.to(BF)
        want, before = O.iterate(f64(x)), O.iterate(f64(x), 4)
        got = f64(r3.orthogonalize(x.cuda()))
        model = O.iterate(f64(x), operand=O.scaled_operand) - want
        last = O.QUINTIC[0] * (O.scaled_operand(before) - before)
        half = torch.finfo(BF).eps / 2
        for part in (weak, np.s_[:]):
            bound = np.sqrt((1.5 * rms(model[part])) ** 2 + (half * rms(want[part])) ** 2 + rms(last[part]) ** 2)
            assert rms((got - want)[part]) <= bound


def test_step_keeps_weak_rows(r3):
    """The same by the momentum step, on the chip and larger, float32 weights: of size zero, so that they show the
    update alone."""
    shapes = [(2, 96, 200), (2, 300, 600), (600, 300)]
    grads = [matrix(s[-2], s[-1], 4, int(np.prod(s[:-2]))).reshape(s) for s in shapes]
    for g in grads[:2]:
        g[:, :9] *= 1e-6
    grads[2][:, :9] *= 1e-6
    weights = [torch.zeros(s).cuda() for s in shapes]
    opt = r3.Muon(weights, [g.cuda() for g in grads], momentum=0.5, scale=1.0)
    opt.step(1.0)
    for w, g, weak in zip(weights, grads, (np.s_[:9], np.s_[:9], np.s_[:, :9])):
        u = g.reshape(-1, *g.shape[-2:])[0] * 1.5
        three(-w.reshape(-1, *w.shape[-2:])[0].cpu(), u, 5, [weak, np.s_[:]])


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (3, 1), (2, 3), (4, 64), (3, 500), (500, 3), (8, 8), (15, 300),
                                       (9, 2500), (2500, 15)])
def test_short_sides_take_three_products(r3, rows, cols):
    """The errors of one product even out over many operands, of which these have few: asked for one, they take
    three, and a bf16 result is off by its rounding."""
    x = matrix(rows, cols, 5, 3).to(BF)
    got, rounded = r3.orthogonalize(x.cuda(), out_dtype=F32, products=1).cpu(), r3.orthogonalize(x.cuda()).cpu()
    assert torch.equal(got, r3.orthogonalize(x.cuda(), out_dtype=F32, products=3).cpu())
    assert torch.equal(got.to(BF), rounded)
    for i in range(3):
        want = O.iterate(f64(x[i]))
        bound = 2 * rms(O.iterate_planes(f64(x[i])) - want) + 2 * rms(O.iterate_f32(f64(x[i])) - want) + \
            rms(O.iterate_short(f64(x[i])) - want) + 2.0 ** -20 * rms(want)
        assert rms(f64(got[i]) - want) <= bound < 1e-4 * rms(want)


def test_one_step_over_short_and_long_sides(r3):
    """Stacks that take one product and such that take three, on the chip (there each as by itself) and larger, in
    one call."""
    shapes = [(2, 8, 40), (2, 40, 80), (12, 2600), (24, 2600), (300, 500), (2600, 15), (3, 16, 16), (1, 15, 15), (8, 40)]
    grads = [matrix(s[-2], s[-1], 6, int(np.prod(s[:-2]))).reshape(s).to(BF) for s in shapes]
    weights = [torch.zeros(s, dtype=BF).cuda() for s in shapes]
    r3.Muon(weights, [g.cuda() for g in grads], momentum=0.0, scale=1.0).step(1.0)
    half = torch.finfo(BF).eps / 2
    for w, g in zip(weights, grads):
        rows, cols = g.shape[-2:]
        u = g.reshape(-1, rows, cols)
        if max(rows, cols) <= 256 and min(rows, cols) <= 128:
            assert torch.equal(-w, r3.orthogonalize(u.cuda()).reshape(w.shape))
        want, before = O.iterate(f64(u[0])), O.iterate(f64(u[0]), 4)
        loss = rms(O.iterate(f64(u[0]), operand=O.scaled_operand) - want) if min(rows, cols) >= 16 else 2.0 ** -16 * rms(want)
        last = O.QUINTIC[0] * rms(O.scaled_operand(before) - before)
        err = rms(f64(-w.reshape(-1, rows, cols)[0]) - want)
        assert err <= np.sqrt((1.5 * loss) ** 2 + (half * rms(want)) ** 2 + last ** 2)
