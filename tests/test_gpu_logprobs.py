"""Token log probabilities, entropy, alternatives and the logits' gradient on the GPU against the
float64 oracle.

Tolerances, in units of 2^-24 (half a float32 step): a term's exponent u = c x - M carries one
rounding of at most |u| (terms below 2^-40 do not matter, so 40), the constant c one of |u| again,
the approximate exponential 2 steps = 4 and its conversion ln2 of that; a sum of up to 2^18 positive
terms is formed in partial sums of at most 2^10 terms with a random walk of roundings, at most 2^10
in the worst case but below 64 on the data used here; together below 200 units = 1.2e-5 relative in
S, absolute in L = ln S.  logp and entropy add a few steps of their own magnitude (at most 30 here).
The bound used is 2e-5 + 2^-22 |value|.  A gradient is a product of p (relative error as S plus the
exponent's) and a factor of size |dlogp| + |dentropy| (|log p| + H), rounded once to its type."""
import numpy as np
import pytest
import torch

from oracle import r3_update_oracle as U
from tests.helpers import f64, logits_gradient_bound

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def r3():
    from paper_2510_11370_b200 import r3 as mod
    return mod


def make(T, V, dtype, seed, pad=0, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn((T, V + pad), generator=g) * scale
    buf[:, 0] += 3.0
    logits = buf.to(dtype).cuda()[:, :V]
    ids = torch.randint(0, V, (T,), generator=g)
    if T > 3:
        ids[::5] = -1
    return logits, ids.cuda()


def close(got, ref, what, rel=2.0 ** -22, ab=2e-5):
    got = f64(got)
    ref = np.asarray(ref, dtype=np.float64)
    assert got.shape == ref.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]) and np.array_equal(np.isinf(got), inf), what
    ok = np.isfinite(ref)
    err = np.abs(got[ok] - ref[ok]) - rel * np.abs(ref[ok])
    assert err.size == 0 or err.max() <= ab, (what, err.max())


def check_forward(r3, logits, ids, temperature=1.0, n_top=0):
    st = r3.new_status("cuda")
    logp, ent, stats, tid, tlp = r3.token_logprobs(
        logits, ids, temperature=temperature, n_top=n_top, want_entropy=True, want_stats=True,
        dev_status=st)
    ref = U.token_logprobs(f64(logits), ids.cpu().numpy(), temperature, n_top)
    assert st.item() == 0
    close(logp, ref["logp"], "logp")
    close(ent, ref["entropy"], "entropy")
    close(stats, ref["stats"], "stats")
    if n_top:
        assert np.array_equal(tid.cpu().numpy(), ref["top_ids"])
        close(tlp, ref["top_logp"], "top_logp")
    # without the entropy and the alternatives other kernels run: the same numbers within rounding
    l2, e2, s2, t2, _ = r3.token_logprobs(logits, ids, temperature=temperature)
    assert e2 is None and s2 is None and t2 is None
    close(l2, ref["logp"], "logp alone")
    again = r3.token_logprobs(logits, ids, temperature=temperature, n_top=n_top, want_entropy=True,
                              want_stats=True)
    assert all(a is b or torch.equal(a, b) for a, b in zip(again, (logp, ent, stats, tid, tlp))
               if a is None or not torch.isnan(a.float()).any())       # reproducible
    return ref


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,n_top,pad", [
    (1, 1, 1, 0), (1, 7, 7, 0), (3, 31, 5, 1), (5, 33, 32, 0), (17, 700, 20, 0), (9, 1000, 32, 7),
    (6, 8191, 3, 0), (300, 8193, 1, 0), (2, 50257, 20, 0), (40, 20011, 32, 13), (1, 151936, 20, 0),
    (7, 131072, 32, 64)])
def test_forward(r3, T, V, n_top, pad, dtype):
    logits, ids = make(T, V, dtype, T * V, pad)
    check_forward(r3, logits, ids, n_top=n_top)


@pytest.mark.parametrize("temperature", [0.3, 0.7, 2.0])
def test_temperature_and_int32_ids(r3, temperature):
    logits, ids = make(33, 5003, F32, 5)
    check_forward(r3, logits, ids.to(torch.int32), temperature, 4)


@pytest.mark.parametrize("temperature", [1e-6, 1e-3, 1e4, 1e20])
def test_extreme_temperatures(r3, temperature):
    """Nearly greedy (every exponent is huge: the sums go by differences to the top) and uniform rows.
    float32 logits apart by one step of 2^-23 are 0.1 apart after division by 1e-6, so log probabilities
    are compared relative to their size."""
    logits, ids = make(24, 3001, F32, 77)
    ref = U.token_logprobs(f64(logits), ids.cpu().numpy(), temperature, 5)
    logp, ent, stats, tid, tlp = r3.token_logprobs(logits, ids, temperature=temperature, n_top=5,
                                                   want_entropy=True, want_stats=True)
    close(logp, ref["logp"], "logp")
    close(ent, ref["entropy"], "entropy")
    close(stats, ref["stats"], "stats")
    close(tlp, ref["top_logp"], "top_logp")
    assert np.array_equal(tid.cpu().numpy(), ref["top_ids"])
    check_backward(r3, logits, ids, temperature)
    # masked values and the padding of a thread's pieces count nothing at any temperature
    logits[:, 5:2000] = float("-inf")
    ids = ids.clamp(max=4)
    ref = U.token_logprobs(f64(logits), ids.cpu().numpy(), temperature)
    logp, ent, _, _, _ = r3.token_logprobs(logits, ids, temperature=temperature, want_entropy=True)
    close(logp, ref["logp"], "logp")
    close(ent, ref["entropy"], "entropy")


@pytest.mark.parametrize("T", [1, 30, 700])
@pytest.mark.parametrize("V", [400, 3001, 40000])
def test_ties_and_adversarial_orders(r3, T, V):
    """Constant rows, rows of few distinct values, rows whose largest values all fall to the same
    thread, ascending and descending rows: the alternatives are the first of the largest values."""
    col = torch.arange(V)
    kinds = [torch.zeros(V), torch.full((V,), -0.0), (col % 3).float(), (col // 700 % 2).float(),
             col.float() / 64, -col.float() / 64, torch.where(col % 4096 < 8, 5.0, 0.0),
             torch.where(col % 2048 < 4, 5.0 + col / V, torch.zeros(V)),
             torch.where(col % 2 == 0, 0.0, -0.0), torch.where(col == V - 1, 1.0, 0.0)]
    x = torch.stack([kinds[t % len(kinds)] for t in range(T)])
    ids = torch.arange(T) % V
    for dtype in (BF, F32):
        rows = x.to(dtype).cuda()
        if T > 40:                                      # the oracle is slow: the rows repeat
            _, _, _, tid, tlp = r3.token_logprobs(rows, ids.cuda(), n_top=32)
            ref = U.token_logprobs(f64(rows[:len(kinds)]), ids[:len(kinds)].numpy(), n_top=32)
            pick = torch.arange(T) % len(kinds)
            assert np.array_equal(tid.cpu().numpy(), ref["top_ids"][pick.numpy()])
            close(tlp, ref["top_logp"][pick.numpy()], "top_logp")
        else:
            check_forward(r3, rows, ids.cuda(), n_top=32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [40, 5000, 66000])
def test_masks_and_special_rows(r3, V, dtype):
    """-inf and the lowest value as masks, one token left, nothing left, NaN, +inf, very large
    and very small logits."""
    g = torch.Generator().manual_seed(V)
    low = torch.finfo(dtype).min
    x = torch.randn((14, V), generator=g) * 3
    x[0, 5:] = -np.inf
    x[1, 5:] = low
    x[2, :] = -np.inf
    x[3, :] = low
    x[4, :] = -np.inf
    x[4, V - 1] = 2.0
    x[5, 3] = np.nan
    x[6, V // 2] = np.inf
    x[7] = x[7] * 1e4
    x[8] = x[8] + 3e5
    x[9] = x[9] - 3e7
    x[10] = x[10] * 1e36
    x[11, ::2] = -np.inf
    x[12, 1::2] = low
    x[12, 0] = 1e30
    x[13, :] = 1e-30
    ids = torch.tensor([1, 2, 0, 3, 0, 1, 1, 4, 5, 6, 7, 1, 1, 2])
    ids[4] = V - 1
    ids[11] = 2                                     # a masked token: log probability -inf
    logits = x.to(dtype).cuda()
    with np.errstate(over="ignore"):
        check_forward(r3, logits, ids.cuda(), n_top=6)
    check_backward(r3, logits[:5], ids[:5].cuda())
    check_backward(r3, logits[7:], ids[7:].cuda())
    # rows with NaN or +inf give NaN everywhere, and rows beside them stay clean
    stats = r3.token_logprobs(logits, ids.cuda(), want_stats=True)[2]
    d = r3.token_logprobs_bwd(logits, ids.cuda(), stats, torch.ones(14, device="cuda"))
    bad = torch.isnan(d).all(1).cpu()
    assert bad.tolist() == [t in (5, 6) for t in range(14)]
    assert not torch.isnan(d[~bad.cuda()]).any()


def check_backward(r3, logits, ids, temperature=1.0, with_entropy=True, inplace=False):
    T, V = logits.shape
    g = torch.Generator().manual_seed(T + V)
    dlogp, dent = torch.randn(T, generator=g), torch.randn(T, generator=g)
    _, ent, stats, _, _ = r3.token_logprobs(logits, ids, temperature=temperature, want_entropy=True,
                                            want_stats=True)
    with np.errstate(over="ignore"):
        ref = U.token_logprobs_bwd(f64(logits), ids.cpu().numpy(), dlogp.numpy().astype(np.float64),
                                   dent.numpy().astype(np.float64) if with_entropy else None,
                                   temperature)
    src = logits.clone() if inplace else logits
    kw = dict(entropy=ent, dentropy=dent.cuda()) if with_entropy else {}
    d = r3.token_logprobs_bwd(src, ids, stats, dlogp.cuda(), temperature=temperature,
                              dlogits=src if inplace else None, **kw)
    step = torch.finfo(logits.dtype).eps / 2
    # 2e-5 relative in p, times a factor that the largest of dlogp and dentropy |log p| bounds
    size = (np.abs(dlogp.numpy()) + (np.abs(dent.numpy()) * 50 if with_entropy else 0)) / temperature
    err = np.abs(f64(d) - ref) - step * np.abs(ref)
    assert (err <= 4e-5 * size[:, None]).all(), err.max()
    # and relative to each element where p is small (the exponent's rounding, up to 60 units there)
    return d


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V,pad", [(1, 1, 0), (3, 31, 1), (17, 700, 0), (9, 1000, 7),
                                     (6, 8193, 0), (5, 50257, 0), (2, 151936, 64)])
def test_backward(r3, T, V, pad, dtype):
    logits, ids = make(T, V, dtype, T * V + 1, pad)
    for with_entropy in (True, False):
        for temperature in (1.0, 0.6):
            check_backward(r3, logits, ids, temperature, with_entropy)
    a = check_backward(r3, logits, ids)
    b = check_backward(r3, logits, ids, inplace=True)
    assert torch.equal(a, b)


def test_backward_of_the_entropy_alone_and_by_differences(r3):
    """A directional difference of the kernel's own forward, in float32 logits."""
    logits, ids = make(8, 600, F32, 11)
    ids = ids.clamp(min=0)
    g = torch.Generator().manual_seed(1)
    direction = torch.randn((8, 600), generator=g).cuda()
    _, ent, stats, _, _ = r3.token_logprobs(logits, ids, want_entropy=True, want_stats=True)
    one, zero = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    for dlogp, dent, pick in ((one, None, 0), (None, one, 1), (zero, one, 1)):
        d = r3.token_logprobs_bwd(logits, ids if dlogp is not None else None, stats, dlogp,
                                  entropy=ent, dentropy=dent)
        h = 1e-2
        up = r3.token_logprobs(logits + h * direction, ids, want_entropy=True)[pick]
        dn = r3.token_logprobs(logits - h * direction, ids, want_entropy=True)[pick]
        want = ((up - dn) / (2 * h)).double()
        got = (d.double() * direction.double()).sum(1)
        # truncation: h^2 / 6 times a third derivative below 30; rounding: 2e-5 / h
        assert (want - got).abs().max().item() < 30 * h * h / 6 + 2 * 2e-5 / h


def test_skipped_rows_padding_columns_and_bad_ids(r3):
    logits, ids = make(12, 300, F32, 2, pad=20)
    ids[3] = 300
    st = r3.new_status("cuda")
    logp, ent, stats, tid, tlp = r3.token_logprobs(logits, ids, n_top=3, want_entropy=True,
                                                   want_stats=True, dev_status=st)
    assert st.item() == r3.DEV_BAD_INDEX
    for t in (0, 3, 5, 10):
        assert logp[t] == 0 and ent[t] == 0 and not stats[t].any() and (tid[t] == -1).all()
        assert not tlp[t].any()
    buf = torch.full((12, 320), 7.0, device="cuda")
    d = r3.token_logprobs_bwd(logits, ids, stats, torch.ones(12, device="cuda"),
                              dlogits=buf[:, :300], dev_status=st)
    assert d.data_ptr() == buf.data_ptr() and (buf[:, 300:] == 7.0).all()
    assert not buf[[0, 3, 5, 10], :300].any() and buf[1, :300].any()
    # rows that are skipped are not read: NaN there changes nothing
    other = logits.clone()
    other[0] = float("nan")
    assert torch.equal(r3.token_logprobs(other, ids)[0], logp)


def test_misaligned_rows_of_different_strides(r3):
    """bfloat16 rows at odd strides, gradient into a dense buffer (no common alignment)."""
    buf = torch.randn((9, 1003)).to(BF).cuda()
    logits = buf[:, 1:1002]                         # starts 2 bytes off
    ids = torch.arange(9, device="cuda")
    check_forward(r3, logits, ids, n_top=4)
    check_backward(r3, logits, ids)


def test_rows_beyond_32_bit_offsets(r3):
    """Rows whose offset passes 2^31 elements."""
    T, V = 20000, 120000                            # 2.4e9 elements, 4.8 GB of bfloat16
    logits = torch.zeros((T, V), dtype=BF, device="cuda")
    ids = torch.full((T,), -1, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    for t in (0, T - 2, T - 1):
        logits[t] = (torch.randn(V, generator=g, device="cuda") * 2).to(BF)
        ids[t] = t % V
    logp, ent, stats, tid, _ = r3.token_logprobs(logits, ids, n_top=5, want_entropy=True,
                                                 want_stats=True)
    rows = [0, T - 2, T - 1]
    ref = U.token_logprobs(f64(logits[rows]), ids[rows].cpu().numpy(), n_top=5)
    close(logp[rows], ref["logp"], "logp")
    close(ent[rows], ref["entropy"], "entropy")
    assert np.array_equal(tid[rows].cpu().numpy(), ref["top_ids"])
    dlogp = torch.ones(T, device="cuda")
    want = U.token_logprobs_bwd(f64(logits[rows]), ids[rows].cpu().numpy(), np.ones(3))
    d = r3.token_logprobs_bwd(logits, ids, stats, dlogp, dlogits=logits)
    assert np.abs(f64(d[rows]) - want).max() < 2.0 ** -9 + 4e-5
    assert not d[1:T - 2].any()


def test_no_ids_streams_and_graphs(r3):
    logits, ids = make(20, 3000, BF, 9)
    _, ent, stats, tid, _ = r3.token_logprobs(logits, None, n_top=2, want_entropy=True,
                                              want_stats=True)
    ref = U.token_logprobs(f64(logits), np.zeros(20, dtype=int), n_top=2)
    close(ent, ref["entropy"], "entropy")
    assert np.array_equal(tid.cpu().numpy(), ref["top_ids"])
    # two streams at once and a captured, replayed call: the same bits
    want = r3.token_logprobs(logits, ids, n_top=2)
    torch.cuda.synchronize()
    outs = []
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            outs.append(r3.token_logprobs(logits, ids, n_top=2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        outs.append(r3.token_logprobs(logits, ids, n_top=2))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], want[0]) and torch.equal(o[3], want[3]) and torch.equal(o[4], want[4])


def test_feeds_the_discrepancy_measures(r3):
    """The probabilities that Eq. (kl) takes are exp of these log probabilities."""
    from oracle import r3_diag_oracle as D
    logits, ids = make(64, 4000, F32, 21)
    keep = ids >= 0
    other = logits + 0.05 * torch.randn(logits.shape, device="cuda")
    pa = r3.token_logprobs(logits, ids)[0][keep].exp()
    pb = r3.token_logprobs(other, ids)[0][keep].exp()
    kl, _ = r3.prob_discrepancy(pa, pb, [2.0])
    i = ids.cpu().numpy()
    ra = np.exp(U.token_logprobs(f64(logits), i)["logp"][i >= 0])
    rb = np.exp(U.token_logprobs(f64(other), i)["logp"][i >= 0])
    # d(k3)/d(log ratio) = r - 1, and a log ratio is off by at most 2 (2e-5 + 30 * 2^-22)
    far = 2 * (2e-5 + 30 * 2.0 ** -22) * np.abs(ra / rb - 1).mean()
    assert abs(kl.item() - D.kl_k3(ra, rb)) <= far + 1e-9 + 1e-5 * kl.item()


def check_every_element(r3, logits, ids, temperature=1.0, with_entropy=True, dlogits=None):
    """The gradient held to a bound relative to each element's own probability, so that the small ones of a
    long row count."""
    T, V = logits.shape
    g = torch.Generator().manual_seed(3 * T + V)
    dlogp, dent = torch.randn(T, generator=g), torch.randn(T, generator=g)
    _, ent, stats, _, _ = r3.token_logprobs(logits, ids, temperature=temperature, want_entropy=True,
                                            want_stats=True)
    kw = dict(entropy=ent, dentropy=dent.cuda()) if with_entropy else {}
    z, at = f64(logits), ids.cpu().numpy()
    d64 = [dlogp.numpy().astype(np.float64), dent.numpy().astype(np.float64) if with_entropy else None]
    with np.errstate(over="ignore"):
        ref = U.token_logprobs_bwd(z, at, *d64, temperature)
    bound = logits_gradient_bound(z, at, *d64, temperature, ref, torch.finfo(logits.dtype).eps)
    d = r3.token_logprobs_bwd(logits, ids, stats, dlogp.cuda(), temperature=temperature, dlogits=dlogits, **kw)
    far = np.abs(f64(d) - ref) - bound
    assert (far <= 0).all(), (far.max(), np.unravel_index(far.argmax(), far.shape))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("with_entropy", [True, False])
@pytest.mark.parametrize("T,V,pad", [(1, 1, 0), (4, 31, 1), (17, 700, 0), (9, 1003, 7), (6, 8193, 0),
                                     (5, 50257, 0), (5, 50257, 15), (4, 131072, 0), (3, 151936, 64)])
def test_every_element_of_the_gradient(r3, T, V, pad, with_entropy, dtype):
    logits, ids = make(T, V, dtype, T * V + 2, pad)
    for temperature in (1.0, 0.6):
        check_every_element(r3, logits, ids, temperature, with_entropy)
    # in place, and into rows that start elsewhere in their 16-byte pieces
    room = torch.empty((T, V + pad + 9), dtype=dtype, device="cuda")
    for off in (0, 1, 5):
        check_every_element(r3, logits, ids, 1.0, with_entropy, dlogits=room[:, off:off + V])
    check_every_element(r3, logits, ids, 1.0, with_entropy, dlogits=logits)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_every_element_of_masked_rows(r3, dtype):
    """Masks of -inf and of the lowest value in every other row of a real vocabulary."""
    logits, ids = make(6, 50257, dtype, 8)
    shut = torch.rand((6, 50257), generator=torch.Generator().manual_seed(2)).cuda() < 0.25
    shut[::2] = False
    ids = ids.clamp(min=0)
    shut.scatter_(1, ids[:, None], False)
    logits[shut & (torch.arange(6, device="cuda") % 4 == 1)[:, None]] = float("-inf")
    logits[shut & (torch.arange(6, device="cuda") % 4 == 3)[:, None]] = torch.finfo(dtype).min
    for with_entropy in (True, False):
        check_every_element(r3, logits, ids, 0.8, with_entropy)


def test_every_element_beyond_32_bit_offsets(r3):
    """Rows whose offset passes 2^31 elements, gradient in place."""
    T, V = 20000, 120000
    logits = torch.zeros((T, V), dtype=BF, device="cuda")
    ids = torch.full((T,), -1, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = [0, T - 2, T - 1]
    for t in rows:
        logits[t] = (torch.randn(V, generator=g, device="cuda") * 2).to(BF)
        ids[t] = t % V
    stats = r3.token_logprobs(logits, ids, want_stats=True)[2]
    z, at = f64(logits[rows]), ids[rows].cpu().numpy()
    ref = U.token_logprobs_bwd(z, at, np.ones(3))
    bound = logits_gradient_bound(z, at, np.ones(3), None, 1.0, ref, torch.finfo(BF).eps)
    d = r3.token_logprobs_bwd(logits, ids, stats, torch.ones(T, device="cuda"), dlogits=logits)
    assert (np.abs(f64(d[rows]) - ref) <= bound).all()
    assert not d[1:T - 2].any()


def plan_of(T, row_bytes, sms):
    """(threads, CTAs per row) that a call takes: the rule of r3_token_logprobs."""
    resident = {32: 24, 128: 8, 256: 4}
    waves = {n: -(-T // (resident[n] * sms)) for n in resident}
    threads = (32 if row_bytes <= 16384 else 128 if row_bytes <= 49152 else
               256 if waves[128] <= 4 and waves[256] < 2 * waves[128] else 128)
    split = 1
    while split < 8 and T * split <= sms and row_bytes // (split * 2) >= 32 * threads:
        split *= 2
    return threads, split


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,n_top", [(149, 20), (300, 0), (590, 5)])
def test_long_rows_on_one_block_of_256_threads(r3, T, n_top, dtype):
    """A few hundred long rows: too many to share, too few for blocks of 128 threads.  The oracle's rows
    repeat."""
    V, kinds = 25013, 7                             # 50 and 100 KB
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert sms != 148 or plan_of(T, V * torch.finfo(dtype).bits // 8, sms) == (256, 1)
    few, _ = make(kinds, V, dtype, 17)
    few[2, 5:9000] = float("-inf")
    few[3] = torch.finfo(dtype).min
    pick = torch.arange(T) % kinds
    ids = torch.arange(T) * 83 % V
    ids[::11] = -1
    ids[pick == 2] = 3
    logits = few[pick.cuda()]
    got = r3.token_logprobs(logits, ids.cuda(), n_top=n_top, want_entropy=True, want_stats=True)
    ref = U.token_logprobs(f64(logits), ids.numpy(), n_top=n_top)
    for name, t in zip(("logp", "entropy", "stats"), got):
        close(t, ref[name], name)
    if n_top:
        assert np.array_equal(got[3].cpu().numpy(), ref["top_ids"])
        close(got[4], ref["top_logp"], "top_logp")
