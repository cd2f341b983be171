"""Norm, gate, scaled residual and norm on the GPU against the float64 oracle.

Tolerances.  A row's sum of squares is formed from at most 32 values per thread, 5 shuffle steps
and 16 warps: at most 53 roundings of 2^-24, halved by the root, and rsqrtf is off by at most 2^-22:
a norm's factor is within 2^-18 relative.  An output's own products add a few 2^-24.  So a forward
output is within 2^-17 of the magnitudes it is summed from plus half a step of its type; a gradient,
formed from such factors twice over (means of products included, taken in magnitude), within
2^-15.  A sum over tokens adds one rounding per row that a CTA takes and per CTA that is added up, at
most 2^9 on these sizes: within 2^-14 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import r3_update_oracle as U
from tests.helpers import f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
KINDS = ["none", "channel", "token", "full"]


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def make(T, d, act, wdt, kind, post, pre, first=False, seed=0, spread=1.0):
    g = torch.Generator().manual_seed(seed + T * 7 + d)

    def rn(*shape):
        return torch.randn(shape, generator=g)
    s = dict(x=(rn(T, d) * spread).to(act), y=None if first else (rn(T, d) * 0.3 * spread).to(act),
             w_post=(1 + 0.3 * rn(d)).to(wdt) if post else None,
             w_pre=(1 + 0.3 * rn(d)).to(wdt) if pre else None,
             gate={"none": None, "channel": rn(d).to(wdt), "token": rn(T, 1), "full": rn(T, d).to(act)}[kind],
             dx_out=None if first else rn(T, d).to(act), dh=rn(T, d).to(act) if pre else None)
    return {k: None if v is None else v.cuda() for k, v in s.items()}


def n64(v):
    return None if v is None else f64(v)


def within(got, ref, mag, rel, what):
    got, step = f64(got), torch.finfo(got.dtype).eps / 2
    assert got.shape == ref.shape, what
    err = np.abs(got - ref) - step * np.abs(ref) - rel * mag - 1e-37
    assert err.size == 0 or err.max() <= 0, (what, err.max(), np.unravel_index(err.argmax(), err.shape))


def check(r3, s, eps=1e-6, residual_scale=1.0, branch_scale=0.7, **inplace):
    kw = dict(eps=eps, residual_scale=residual_scale, branch_scale=branch_scale)
    v = {k: n64(t) for k, t in s.items()}
    vec = {k: v[k] for k in ("w_post", "gate", "w_pre")}
    T, d = v["x"].shape
    first = s["y"] is None
    # ---- forward
    x_out, h = r3.norm_residual(s["x"], s["y"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], **kw)
    ref_x, ref_h = U.norm_residual(v["x"], v["y"], **vec, **kw)
    if first:
        assert x_out is None
        mag = np.abs(v["x"])
        full = v["x"]
    else:
        n = v["y"] if v["w_post"] is None else U.rms_norm(v["y"], v["w_post"], eps)
        mag = np.abs(residual_scale * v["x"]) + np.abs(branch_scale * U._gate_2d(v["gate"], T, d) * n)
        full = ref_x
        within(x_out, ref_x, mag, 2.0 ** -17, "x_out")
    if ref_h is None:
        assert h is None
    else:
        r = 1 / np.sqrt((full * full).mean(1, keepdims=True) + eps)
        within(h, ref_h, mag * r * np.abs(v["w_pre"]) + np.abs(ref_h), 2.0 ** -17, "h")
    # ---- backward, at the activations as they are kept
    at = s["x"] if first else x_out
    out = r3.norm_residual_bwd(at, s["y"], s["dx_out"], s["dh"], w_post=s["w_post"], gate=s["gate"],
                               w_pre=s["w_pre"], **kw)
    got = dict(zip(("dx", "dy", "dw_post", "dgate", "dw_pre"), out))
    ref = U.norm_residual_bwd(f64(at), v["y"], v["dx_out"], v["dh"], **vec, **kw)
    assert {k for k, t in got.items() if t is not None} == set(ref)
    a = f64(at)
    gm = 0.0 if v["dx_out"] is None else np.abs(v["dx_out"])
    if v["w_pre"] is not None:
        r = 1 / np.sqrt((a * a).mean(1, keepdims=True) + eps)
        m, u = np.abs(a) * r, np.abs(v["dh"] * v["w_pre"])
        gm = gm + r * (u + m * (u * m).mean(1, keepdims=True))
        within(got["dw_pre"], ref["dw_pre"], (np.abs(v["dh"]) * m).sum(0), 2.0 ** -14, "dw_pre")
    within(got["dx"], ref["dx"], np.abs(1.0 if first else residual_scale) * gm, 2.0 ** -15, "dx")
    if not first:
        gate = np.abs(U._gate_2d(v["gate"], T, d))
        sy = 1.0 if v["w_post"] is None else 1 / np.sqrt((v["y"] ** 2).mean(1, keepdims=True) + eps)
        w = 1.0 if v["w_post"] is None else np.abs(v["w_post"])
        nm, q = np.abs(v["y"]) * sy, abs(branch_scale) * gm
        t = q * gate
        back = t * w if v["w_post"] is None else sy * (t * w + nm * (t * w * nm).mean(1, keepdims=True))
        within(got["dy"], ref["dy"], back, 2.0 ** -15, "dy")
        if v["w_post"] is not None:
            within(got["dw_post"], ref["dw_post"], (t * nm).sum(0), 2.0 ** -14, "dw_post")
        if v["gate"] is not None:
            e = q * nm * w
            shape = v["gate"].shape
            em = e if shape == (T, d) else e.sum(1, keepdims=True) if shape == (T, 1) else e.sum(0)
            within(got["dgate"], ref["dgate"], em, 2.0 ** -14, "dgate")
    return x_out, h, out, kw


@pytest.mark.parametrize("act,wdt", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_every_form(r3, act, wdt, kind, post, pre):
    for T, d in ((5, 72), (3, 1160)):
        check(r3, make(T, d, act, wdt, kind, post, pre))


@pytest.mark.parametrize("act,wdt", [(BF, BF), (F32, F32)])
@pytest.mark.parametrize("T,d", [(1, 8), (2, 16), (700, 8), (1, 2048), (33, 256), (130, 512), (17, 520),
                                 (257, 2048), (3, 4096), (9, 4104), (5, 8192), (4099, 40), (2500, 264),
                                 (1, 32), (6, 1024)])
def test_sizes(r3, act, wdt, T, d):
    check(r3, make(T, d, act, wdt, "channel", True, True))
    check(r3, make(T, d, act, wdt, "none", False, True, first=True), branch_scale=1.0)


@pytest.mark.parametrize("act,d", [(BF, 3592), (BF, 4096), (F32, 1992)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_rows_worked_on_two_at_a_time(r3, act, d, kind, post, pre):
    """Long rows, whose gradient takes two of a group's rows at once: no second row, one for one group
    only, an odd number of rows for each."""
    for T in (1, 149, 450):
        check(r3, make(T, d, act, act, kind, post, pre))


@pytest.mark.parametrize("act,d", [(BF, 6152), (BF, 8200), (BF, 12296), (F32, 3080), (F32, 4104)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_every_form_of_wide_rows(r3, act, d, kind, post, pre):
    check(r3, make(150, d, act, F32, kind, post, pre))


@pytest.mark.parametrize("act,T,d", [(BF, 70001, 64), (BF, 30001, 520), (F32, 5001, 2000), (F32, 5100, 3080)])
def test_token_gates_of_many_rows(r3, act, T, d):
    """More than 32 rows for a group of threads (one warp, several, two rows at a time, the wide form)."""
    check(r3, make(T, d, act, F32, "token", True, True))


def test_largest_rows(r3):
    for d in (8200, 16384):
        check(r3, make(40, d, BF, F32, "channel", True, True))
        check(r3, make(40, d, BF, BF, "token", True, True))
    with pytest.raises(r3.R3Error) as e:
        r3.norm_residual(torch.zeros((1, 16392), dtype=BF, device="cuda"), w_pre=torch.ones(16392, dtype=BF, device="cuda"))
    assert e.value.code == r3.R3_ERR_UNSUPPORTED


def test_many_rows(r3):
    check(r3, make(20000, 128, BF, BF, "channel", True, True))
    check(r3, make(9001, 544, F32, F32, "token", True, True), residual_scale=0.5, branch_scale=-1.5)


@pytest.mark.parametrize("act", [BF, F32])
def test_zero_rows_large_and_small_values(r3, act):
    """Rows of zeros (the factor is 1 / sqrt(eps)), rows whose squares are near the ends of
    float32's range, rows beside them unaffected."""
    s = make(8, 264, act, act, "channel", True, True)
    s["y"][0] = 0
    s["x"][1] = 0
    s["y"][1] = 0
    s["x"][2] *= 1e15
    s["y"][3] *= 1e15
    s["y"][4] *= 1e-18
    s["x"][5] *= 1e-18
    s["y"][5] *= 1e-18
    check(r3, s)
    check(r3, s, eps=1e-2)


def test_nan_stays_in_its_row(r3):
    s = make(9, 520, BF, BF, "channel", True, True)
    clean = r3.norm_residual(s["x"], s["y"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    s["y"][4, 7] = float("nan")
    x_out, h = r3.norm_residual(s["x"], s["y"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    rest = [t for t in range(9) if t != 4]
    assert torch.isnan(x_out[4]).all() and torch.isnan(h[4]).all()
    assert torch.equal(x_out[rest], clean[0][rest]) and torch.equal(h[rest], clean[1][rest])


def test_no_gradient_from_above(r3):
    """dx_out may be missing (the last residual is not used): the same as zeros."""
    s = make(50, 264, BF, F32, "full", True, True)
    kw = dict(w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    a = r3.norm_residual_bwd(s["x"], s["y"], None, s["dh"], **kw)
    b = r3.norm_residual_bwd(s["x"], s["y"], torch.zeros_like(s["x"]), s["dh"], **kw)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_empty_batch(r3):
    s = make(0, 64, BF, F32, "channel", True, True)
    kw = dict(w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    x_out, h = r3.norm_residual(s["x"], s["y"], **kw)
    assert x_out.shape == h.shape == (0, 64)
    dx, dy, dw_post, dgate, dw_pre = r3.norm_residual_bwd(x_out, s["y"], s["dx_out"], s["dh"], **kw)
    assert dx.shape == (0, 64)
    for t in (dw_post, dgate, dw_pre):
        assert t.shape == (64,) and not t.any()          # sums of nothing, written all the same


@pytest.mark.parametrize("act", [BF, F32])
@pytest.mark.parametrize("T,d", [(2000, 512), (3000, 2048), (70, 8192)])
def test_in_place_and_reproducible(r3, T, d, act):
    s = make(T, d, act, act, "channel", True, True)
    kw = dict(w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    x_out, h = r3.norm_residual(s["x"], s["y"], **kw)
    x2, y2 = s["x"].clone(), s["y"].clone()
    r3.norm_residual(x2, y2, x_out=x2, h=y2, **kw)
    assert torch.equal(x2, x_out) and torch.equal(y2, h)
    want = r3.norm_residual_bwd(x_out, s["y"], s["dx_out"], s["dh"], **kw)
    again = r3.norm_residual_bwd(x_out, s["y"], s["dx_out"], s["dh"], **kw)
    assert all(torch.equal(p, q) for p, q in zip(want, again))
    for dx_at, dy_at in (("dx_out", "dh"), ("dh", "dx_out"), ("dx_out", "y")):
        c = {k: s[k].clone() for k in ("dx_out", "dh", "y")}
        got = r3.norm_residual_bwd(x_out, c["y"], c["dx_out"], c["dh"], dx=c[dx_at], dy=c[dy_at], **kw)
        assert all(torch.equal(p, q) for p, q in zip(want, got)), (dx_at, dy_at)


def test_streams_graph_and_shared_workspace(r3):
    s = make(500, 2048, BF, BF, "channel", True, True)
    kw = dict(w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    want = r3.norm_residual_bwd(s["x"], s["y"], s["dx_out"], s["dh"], **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = r3.norm_residual_bwd(s["x"], s["y"], s["dx_out"], s["dh"], **kw)
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    ws = r3.workspace(1 << 24, "cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a = r3.norm_residual_bwd(s["x"], s["y"], s["dx_out"], s["dh"], ws=ws, **kw)
    with torch.cuda.graph(other):                      # the same workspace, replayed in turn
        b = r3.norm_residual_bwd(s["x"], s["y"], s["dx_out"], s["dh"], ws=ws, **kw)
    for _ in range(2):
        graph.replay()
        other.replay()
    torch.cuda.synchronize()
    for o in (got, a, b):
        assert all(torch.equal(p, q) for p, q in zip(want, o))


def test_rows_beyond_32_bit_offsets(r3):
    """T d = 2^31 + 2^26 elements of bfloat16 in each row array: the first and last rows."""
    d = 2048
    T = (1 << 20) + (1 << 15)
    x = torch.zeros((T, d), dtype=BF, device="cuda")
    y = torch.zeros((T, d), dtype=BF, device="cuda")
    pick = [0, 1, T // 2, T - 2, T - 1]
    small = make(5, d, BF, BF, "channel", True, True)
    x[pick], y[pick] = small["x"], small["y"]
    kw = dict(w_post=small["w_post"], gate=small["gate"], w_pre=small["w_pre"])
    want = r3.norm_residual(small["x"], small["y"], **kw)
    x_out, h = r3.norm_residual(x, y, **kw)
    assert torch.equal(x_out[pick], want[0]) and torch.equal(h[pick], want[1])
    assert not x_out[2:T // 2].any()


@pytest.mark.parametrize("act,T,d", [(BF, 45, 264), (F32, 70, 1160), (F32, 64, 64), (BF, 1, 520)])
def test_token_gates_as_a_vector(r3, act, T, d):
    """A gate [T] is the gate [T, 1], with its gradient in the same shape; [T] = [d] of float32 has to be
    named."""
    s = make(T, d, act, F32, "token", True, True)
    kw = dict(w_post=s["w_post"], w_pre=s["w_pre"])
    vec = dict(gate=s["gate"][:, 0].contiguous(), gate_kind="token" if T == d else None, **kw)
    ahead = r3.norm_residual(s["x"], s["y"], gate=s["gate"], **kw)
    got = r3.norm_residual(s["x"], s["y"], **vec)
    assert all(torch.equal(p, q) for p, q in zip(ahead, got))
    want = r3.norm_residual_bwd(s["x"], s["y"], s["dx_out"], s["dh"], gate=s["gate"], **kw)
    got = r3.norm_residual_bwd(s["x"], s["y"], s["dx_out"], s["dh"], **vec)
    assert got[3].shape == (T,) and want[3].shape == (T, 1)
    assert all(torch.equal(p.view(-1), q.view(-1)) for p, q in zip(want, got))
    if T == d:
        with pytest.raises(ValueError):
            r3.norm_residual(s["x"], s["y"], **dict(vec, gate_kind=None))
        channel = r3.norm_residual(s["x"], s["y"], **dict(vec, gate_kind="channel"))
        assert not torch.equal(channel[0], ahead[0])
