"""The AdamW step on the GPU against the float64 oracle.

Tolerances.  A 32-bit state goes through at most 5 roundings of 2^-24 of terms that do not exceed
the sum of its terms' magnitudes (v: of positive terms): 2^-21 of that.  The weight's update is
m / (sqrt(v) bias + eps): errors of m (2^-21 of its terms), half of v's, the root, the approximate
quotient (2^-22) and constants rounded to float32: together 2^-19 of the update formed from the
magnitudes, and 2^-22 of the weight itself, then half a step of the weight's type.  An 8-bit state is
the e4m3 value nearest to the float32 state: off by at most half a step of that value (2^-4 of it, or
half of 2^-9 below 2^-6), widened by the state's own 2^-21."""
import numpy as np
import pytest
import torch

from oracle import r3_update_oracle as U
from tests.helpers import f64

pytestmark = pytest.mark.gpu
BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
BETAS = (0.9, 0.95)


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def make(r3, sizes, dtype, grad, master, bits, seed=0, **kw):
    g = torch.Generator().manual_seed(seed + sum(sizes))

    def rn(n, std):
        return torch.randn(n, generator=g) * std * torch.exp(torch.randn(1, generator=g))
    w = [rn(n, 0.05) for n in sizes]
    params = [x.to(dtype).cuda() for x in w]
    grads = [rn(n, 1e-3).to(grad).cuda() for n in sizes]
    masters = [x.cuda() for x in w] if master else None
    m, v = [rn(n, 5e-4) for n in sizes], [rn(n, 1e-3).square() for n in sizes]
    if bits == 32:
        state = dict(exp_avg=[x.cuda() for x in m], exp_avg_sq=[x.cuda() for x in v])
    else:
        state = dict(exp_avg=[], exp_avg_sq=[], exp_avg_scale=[], exp_avg_sq_scale=[])
        for a, b in ((m, "exp_avg"), ([x.sqrt() for x in v], "exp_avg_sq")):
            for x in a:
                scale = U.block_scale(blocks(x.numpy()))
                q = U.nearest_e4m3(blocks(x.numpy()) / scale[:, None]).reshape(-1)[:x.numel()]
                state[b].append(torch.from_numpy(q).to(E4).cuda())
                state[b + "_scale"].append(torch.from_numpy(scale).float().cuda())
    return r3.AdamW(params, grads, masters=masters, state_bits=bits, betas=BETAS, **state, **kw)


def blocks(x):
    """[n] -> [ceil(n / 256), 256], zeros behind the end."""
    n = x.shape[0]
    out = np.zeros((-(-n // U.BLOCK), U.BLOCK), dtype=x.dtype)
    out.reshape(-1)[:n] = x
    return out


def state64(opt, i):
    m, v = f64(opt.exp_avg[i]), f64(opt.exp_avg_sq[i])
    if opt.state_bits == 8:
        m = (blocks(m) * f64(opt.exp_avg_scale[i])[:, None]).reshape(-1)[:m.size]
        v = (blocks(v) * f64(opt.exp_avg_sq_scale[i])[:, None]).reshape(-1)[:v.size] ** 2
    return m, v


def check_codes(value, code, scale, root):
    """code [blocks, 256] and scale [blocks] hold value (64 bits) to the nearest code."""
    slack = 2.0 ** -20
    want = U.block_scale(value)
    border = np.abs(np.abs(value).max(1) / (U.E4M3_MAX * want) - 1) < slack
    border |= np.abs(np.abs(value).max(1) / (U.E4M3_MAX * want / 2) - 1) < slack
    assert np.array_equal(scale[~border], want[~border])
    assert (np.abs(np.log2(scale / want)) <= border).all()
    q = value / scale[:, None]
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6))) - 3)
    err = np.abs(code - q)
    if root:
        least = (value > 0) & (np.abs(q) <= 2.0 ** -10 * (1 + slack))
        assert ((code == U.E4M3_MIN) | (code == 0))[least].all()
        # nothing above zero, as float32 holds it, is kept as zero: a root above 1e-20 has a second
        # moment above 1e-40, formed from a square above 1e-40, both far above the least float32
        # (2^-149 = 1.4e-45); below, the square itself may round to zero
        assert (code[value > 1e-20] > 0).all()
        err[least] = 0
    # the step above a value just below a power of two is twice its own
    assert (err <= step / 2 * (1 + 2 ** -3 * (np.abs(q) > 440)) + slack * np.abs(q)).all()


def check_step(r3, opt, step=7, lr=1e-2, grad_scale=None, **kw):
    before = []
    for i in range(len(opt.params)):
        w = opt.params[i] if opt.masters is None else opt.masters[i]
        before.append((f64(w), f64(opt.grads[i]), *state64(opt, i)))
    gs = None if grad_scale is None else torch.tensor([grad_scale], device="cuda")
    opt.step(step, lr, grad_scale=gs, **kw)
    s = 1.0 if grad_scale is None else float(np.float32(grad_scale))
    for i, (w0, g, m0, v0) in enumerate(before):
        decay = float(opt._table[i].weight_decay)
        w, m, v = U.adamw(w0, g, m0, v0, step, lr, BETAS, opt._config.eps, decay, s)
        mm = BETAS[0] * np.abs(m0) + (1 - BETAS[0]) * np.abs(g * s)
        tiny = 1e-44                                      # below float32's smallest steps
        if opt.state_bits == 32:
            assert (np.abs(f64(opt.exp_avg[i]) - m) <= 2.0 ** -21 * mm + tiny).all()
            assert (np.abs(f64(opt.exp_avg_sq[i]) - v) <= 2.0 ** -21 * v + tiny).all()
        else:
            check_codes(blocks(m), blocks(f64(opt.exp_avg[i])), f64(opt.exp_avg_scale[i]), False)
            check_codes(blocks(np.sqrt(v)), blocks(f64(opt.exp_avg_sq[i])), f64(opt.exp_avg_sq_scale[i]), True)
        bias1, bias2 = 1 - BETAS[0] ** step, 1 - BETAS[1] ** step
        upd = lr * (mm / bias1) / (np.sqrt(v / bias2) + opt._config.eps)
        far = 2.0 ** -19 * upd + 2.0 ** -22 * np.abs(w0) + tiny
        if opt.masters is not None:
            assert (np.abs(f64(opt.masters[i]) - w) <= far).all()
            assert torch.equal(opt.params[i], opt.masters[i].to(opt.params[i].dtype))
        else:
            half = torch.finfo(opt.params[i].dtype).eps / 2
            assert (np.abs(f64(opt.params[i]) - w) <= far * (1 + half) + half * np.abs(w)).all()


SIZES = [1, 3, 255, 256, 257, 1000, 8192, 8193, 20000, 100003]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad,master", [(F32, F32, False), (F32, BF, False), (BF, F32, False),
                                               (BF, BF, False), (BF, F32, True), (BF, BF, True)])
def test_step(r3, dtype, grad, master, bits):
    opt = make(r3, SIZES, dtype, grad, master, bits, weight_decay=[0.1 * (i % 3) for i in range(len(SIZES))])
    check_step(r3, opt)
    check_step(r3, opt, step=8, grad_scale=0.37)


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(r3, bits):
    """More than one launch (over 400 tensors), and empty ones among them."""
    rng = np.random.default_rng(0)
    sizes = [int(n) for n in rng.integers(0, 700, 930)]
    check_step(r3, make(r3, sizes, BF, F32, bits == 32, bits, weight_decay=0.2), grad_scale=2.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_fresh_states_and_several_steps(r3, bits):
    w = torch.randn(5000, generator=torch.Generator().manual_seed(1)).cuda()
    opt = r3.AdamW([w], [torch.zeros_like(w)], state_bits=bits)
    for step in range(1, 6):
        opt.set_grads([torch.randn(5000, generator=torch.Generator().manual_seed(step)).cuda()])
        check_step(r3, opt, step=step)
    before = w.clone()
    opt.set_grads([torch.zeros_like(w)])
    for step in range(6, 200):                          # states fade without becoming NaN
        opt.step(step, 1e-3)
    assert torch.isfinite(w).all() and (w - before).abs().max() < 0.05


def test_8_bit_states_are_a_function_of_the_inputs(r3):
    """The stored codes equal those of the same operations, each rounded to float32 (on the CPU).  A root's
    code may be the neighbouring one where the root is within 2^-22 of the middle between two codes (the
    kernel's root is an approximation): none of these inputs is."""
    n = 256 * 400
    opt = make(r3, [n], F32, F32, False, 8, seed=3)
    g = opt.grads[0].cpu().numpy()
    f = np.float32
    m0 = blocks(opt.exp_avg[0].float().cpu().numpy()) * opt.exp_avg_scale[0].cpu().numpy()[:, None]
    r0 = blocks(opt.exp_avg_sq[0].float().cpu().numpy()) * opt.exp_avg_sq_scale[0].cpu().numpy()[:, None]
    gs = f(0.37)
    opt.step(5, 1e-3, grad_scale=torch.tensor([0.37], device="cuda"))
    gb = blocks(g) * gs
    m = f(0.9) * m0 + f(1 - 0.9) * gb
    v = f(0.95) * (r0 * r0) + f(1 - 0.95) * (gb * gb)
    assert m.dtype == v.dtype == np.float32
    root = np.sqrt(v)
    for x, code, scale in ((m, opt.exp_avg[0], opt.exp_avg_scale[0]),
                           (root, opt.exp_avg_sq[0], opt.exp_avg_sq_scale[0])):
        s = U.block_scale(x)
        q = U.nearest_e4m3(x.astype(np.float64) / s[:, None])
        if x is root:
            q[(x > 0) & (q == 0)] = U.E4M3_MIN
        assert np.array_equal(f64(scale), s) and np.array_equal(blocks(f64(code)), q)


def test_wide_ranges_in_a_block(r3):
    """Blocks whose largest value dwarfs the rest: small roots are kept above zero, and a weight with a
    tiny state takes no wild step."""
    n = 512
    g = torch.full((n,), 1e-12)
    g[0] = 1e3
    g[300] = 0.0
    g[257:300] = 1e-30
    w = torch.ones(n).cuda()
    opt = r3.AdamW([w], [g.cuda()], state_bits=8)
    check_step(r3, opt, step=1, lr=1e-3)
    for step in range(2, 30):
        opt.step(step, 1e-3)
    assert torch.isfinite(w).all() and (1 - w).abs().max() < 0.06
    assert (opt.exp_avg_sq[0].float()[:256] > 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_not_finite(r3, bits):
    opt = make(r3, [700], F32, F32, False, bits)
    keep = [t.clone() for t in (opt.params[0], opt.exp_avg[0].view(torch.uint8), opt.exp_avg_sq[0].view(torch.uint8))]
    for bad in (float("nan"), float("inf")):
        opt.step(3, 0.1, grad_scale=torch.tensor([bad], device="cuda"))
    now = (opt.params[0], opt.exp_avg[0].view(torch.uint8), opt.exp_avg_sq[0].view(torch.uint8))
    assert all(torch.equal(a, b) for a, b in zip(keep, now))          # skipped
    other = make(r3, [700], F32, F32, False, bits)
    opt.grads[0][5] = float("nan")
    opt.grads[0][300] = float("inf")
    opt.step(3, 0.1)
    other.step(3, 0.1)
    hit = torch.zeros(700, dtype=torch.bool, device="cuda")
    hit[[5, 300]] = True
    assert torch.isnan(opt.params[0][hit]).all()
    assert torch.equal(opt.params[0][~hit], other.params[0][~hit])
    m = opt.exp_avg[0].float()
    assert torch.isfinite(m[~hit]).all() and not torch.isfinite(m[hit]).any()
    if bits == 8:
        assert torch.isfinite(opt.exp_avg_scale[0]).all() and torch.isnan(m[hit]).all()


def test_views_of_a_flat_buffer_leave_the_rest(r3):
    """Tensors inside larger buffers: what lies behind each stays as it was."""
    flat = [torch.full((4096,), 3.0, device="cuda") for _ in range(4)]
    views = [[f[0:777], f[1024:1024 + 513]] for f in flat]
    opt = r3.AdamW(views[0], views[1], exp_avg=views[2], exp_avg_sq=views[3])
    check_step(r3, opt)
    for f in (flat[0], flat[2], flat[3]):
        assert (f[777:1024] == 3.0).all() and (f[1024 + 513:] == 3.0).all()


def test_captured_step_with_device_scalars(r3):
    a = make(r3, [5000, 300], BF, F32, True, 8, weight_decay=0.1)
    b = make(r3, [5000, 300], BF, F32, True, 8, weight_decay=0.1)
    scalars = torch.tensor(a.scalars(4, 1e-2), device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(1, 0.0, scalars=scalars)
    for step, lr in ((4, 1e-2), (5, 3e-3)):
        scalars.copy_(torch.tensor(a.scalars(step, lr)))
        graph.replay()
        b.step(step, lr)
    torch.cuda.synchronize()
    for x, y in zip(a.masters + a.params + a.exp_avg_scale, b.masters + b.params + b.exp_avg_scale):
        assert torch.equal(x, y)


def test_large_tensor(r3):
    """Offsets beyond 2^31 bytes and elements: the last block of a tensor of 2^31 + 300 elements."""
    n = (1 << 31) + 300
    w = torch.zeros(n, dtype=BF, device="cuda")
    g = torch.zeros(n, dtype=BF, device="cuda")
    g[-400:] = 1.0
    g[:100] = -1.0
    opt = r3.AdamW([w], [g], state_bits=8, eps=1e-8)
    opt.step(1, 0.5)
    assert (w[-400:] == -0.5).all() and (w[:100] == 0.5).all() and not w[100:1000].any()
    assert not w[-1000:-400].any()


def test_python_refusals(r3):
    w = torch.zeros(512, device="cuda")
    g = torch.zeros(512, device="cuda")
    with pytest.raises(ValueError):
        r3.AdamW([w], [g[:100]])
    with pytest.raises(ValueError):
        r3.AdamW([w], [g.half()])
    with pytest.raises(ValueError):
        r3.AdamW([w], [g], masters=True)
    with pytest.raises(ValueError):
        r3.AdamW([w], [g], state_bits=16)
    with pytest.raises(ValueError):
        r3.AdamW([w], [g.cpu()])
    with pytest.raises(ValueError):
        r3.AdamW([w[::2]], [g[::2]])
    with pytest.raises(ValueError):
        r3.AdamW([], [])
    with pytest.raises(r3.R3Error):
        r3.AdamW([w]).step(1, 0.1)                                     # no gradients yet
    same = r3.AdamW([w, w], [g, g])
    with pytest.raises(r3.R3Error) as e:
        same.step(1, 0.1)
    assert e.value.code == r3.R3_ERR_INVALID_ARG and not w.any()
    with pytest.raises(r3.R3Error):
        r3.AdamW([w[:300], w[256:]], [g[:300], g[256:]]).step(1, 0.1)
    with pytest.raises(r3.R3Error):
        r3.AdamW([w[1:]], [g[1:]]).step(1, 0.1)                        # 4-byte aligned only
    with pytest.raises(r3.R3Error):
        r3.AdamW([w], [g]).step(0, 0.1)                                # steps count from 1


def test_exchanged_data_leaves_the_handle_its_memory(r3):
    p = torch.nn.Parameter(torch.ones(1000, device="cuda"))
    g = torch.ones(1000, device="cuda")
    o = r3.AdamW([p], [g])
    p.data = torch.zeros(1000, device="cuda")
    others = [torch.full((1000,), 5.0, device="cuda") for _ in range(8)]
    o.step(1, 0.1)
    assert all((t == 5.0).all() for t in others) and not p.any()


def test_a_step_after_refused_gradients_takes_the_old_ones(r3):
    a = make(r3, [700, 300], F32, F32, False, 32)
    b = make(r3, [700, 300], F32, F32, False, 32)
    for bad in ([torch.ones(700, device="cuda"), torch.ones(299, device="cuda")],
                [torch.ones(700, dtype=BF, device="cuda"), torch.ones(300, device="cuda")]):
        with pytest.raises(ValueError):
            a.set_grads(bad)
    a.step(2, 1e-2)
    b.step(2, 1e-2)
    for p, q in zip(a.params + a.exp_avg + a.exp_avg_sq, b.params + b.exp_avg + b.exp_avg_sq):
        assert torch.equal(p, q)


def midpoints():
    """Values around the middle between any two neighbouring positive e4m3 values, and their float32
    neighbours, with 448 in front of every block (so that the scale is 1)."""
    codes = np.arange(0x7f, dtype=np.uint8)
    at = torch.from_numpy(codes).view(E4).to(torch.float32).numpy()
    mid = ((at[1:] + at[:-1]) / 2).astype(np.float32)
    out = [mid]
    for direction in (np.float32(0), np.float32(1e9)):
        near = mid
        for _ in range(6):
            near = np.nextafter(near, direction)
            out.append(near)
    out = np.concatenate(out)
    out = np.concatenate([out, np.zeros(-len(out) % 255, dtype=np.float32)]).reshape(-1, 255)
    return np.concatenate([np.full((len(out), 1), 448, dtype=np.float32), out], axis=1)


@pytest.mark.parametrize("exponent", [0, 40, -61, -66])
@pytest.mark.parametrize("dtype,master", [(F32, False), (BF, False), (BF, True)])
def test_codes_of_roots_between_two_codes(r3, dtype, master, exponent):
    """Without averaging (betas 0) the second moment is the gradient's square: the stored code is that of
    its correctly rounded root also next to the middle between two codes, and in it (ties to even).  The
    lowest exponents take the smaller squares below float32's normal range, and to zero."""
    unit = np.float32(2.0) ** np.float32(exponent)
    g = midpoints() * unit
    w = torch.zeros(g.size, dtype=dtype, device="cuda")
    opt = r3.AdamW([w], [torch.from_numpy(g.reshape(-1)).cuda()], state_bits=8, betas=(0.0, 0.0),
                   masters=True if master else None)
    opt.step(1, 1e-3)
    root = np.sqrt(g * g)
    assert root.dtype == np.float32
    want = U.nearest_e4m3(root.astype(np.float64) / float(unit))
    want[(root > 0) & (want == 0)] = U.E4M3_MIN
    assert (opt.exp_avg_sq_scale[0] == float(unit)).all()
    assert np.array_equal(blocks(f64(opt.exp_avg_sq[0])), want)


@pytest.mark.parametrize("dtype,master,bits", [(F32, False, 32), (F32, False, 8), (BF, True, 32), (BF, True, 8),
                                               (BF, False, 32)])
def test_the_update_is_rounded_operation_by_operation(r3, dtype, master, bits):
    """Without averaging, from weights of zero and with a rate of 1 the step is one quotient: the bits of
    float32 square, root, sum and division, each rounded to the last bit (half a step of 2^-24)."""
    g = torch.randn(30000, generator=torch.Generator().manual_seed(5)) * torch.logspace(-12, 6, 30000)
    w = torch.zeros(30000, dtype=dtype, device="cuda")
    eps = 1e-3
    opt = r3.AdamW([w], [g.cuda()], state_bits=bits, betas=(0.0, 0.0), eps=eps, masters=True if master else None)
    opt.step(1, 1.0)
    x = g.numpy()
    want = -(x / (np.sqrt(x * x) + np.float32(eps)))
    assert want.dtype == np.float32
    held = opt.masters[0] if master else w
    assert torch.equal(held.cpu(), torch.from_numpy(want).to(held.dtype))
    assert torch.equal(w, held.to(dtype))
