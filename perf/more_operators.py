"""The losses and the matrix optimiser of an Update step, as they are timed and compared.

  policy_loss     clipped policy loss over packed responses, its correction for the rollout engine's
                  probabilities, its KL term and its entropy bonus, with the gradients to both
  balance_loss    balance and z loss of the routers of L blocks with the counts per expert, and the
                  gradient to the router logits
  orthogonalize   Newton-Schulz iteration that brings a matrix's singular values near one
  Muon.step       momentum, orthogonalised update and weight decay of stacks of matrices

`run` gives the plain form (elementary torch operations) where `own` is false and the framework's
entry points where it is true."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
QUINTIC = (3.4445, -4.7750, 2.0315)     # the iteration's usual coefficients


# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # a handful of short responses, PPO's loss with one clip range
        dict(name="policy_few", op="policy", T=1531, S=12, ratio="token", reduce="token",
             per_token=True, infer=False, ref=False, entropy=False, mask=0.2, dual=0.0, high=0.2),
        # one batch of the Update stage: 256 responses packed to the replayed token count; clip-higher,
        # rollout correction, KL term and entropy bonus
        dict(name="policy_update", op="policy", T=65536, S=256, ratio="token", reduce="token",
             per_token=False, infer=True, ref=True, entropy=True, mask=0.1, dual=3.0, high=0.28),
        # a whole rollout batch with ratios of whole sequences
        dict(name="policy_rollout_sequence", op="policy", T=1000003, S=1024, ratio="sequence",
             reduce="sequence", per_token=False, infer=True, ref=False, entropy=False, mask=0.1,
             dual=0.0, high=4e-4),
        # the smallest block: 8 experts, 2 of them per token
        dict(name="balance_tiny", op="balance", L=1, T=512, E=8, K=2, idx="u8", mask=0.0, z=1e-3),
        # three blocks over a padded batch, an odd number of experts in 16-bit records
        dict(name="balance_odd", op="balance", L=3, T=4097, E=301, K=6, idx="i16", mask=0.3, z=1e-3),
        # the replayed batch of one block
        dict(name="balance_replay", op="balance", L=1, T=65536, E=128, K=8, idx="u8", mask=0.0, z=0.0),
        # all routers of the 48-block stack
        dict(name="balance_stack", op="balance", L=48, T=16384, E=128, K=8, idx="u8", mask=0.0,
             z=1e-3),
        # the router weight of one block
        dict(name="ortho_router", op="ortho", B=1, rows=128, cols=2048, dtype="f32"),
        # matrices of odd sizes
        dict(name="ortho_odd", op="ortho", B=5, rows=1163, cols=501, dtype="bf16"),
        # the expert weights of the smallest block: gate, up and down
        dict(name="muon_tiny", op="muon", stacks="8x256x128,8x256x128,8x128x256", dtype="f32",
             grad="f32", master=False, nesterov=True, decay=0.0, clip=False),
        # square and oblong projections of some blocks, float32 masters, bf16 gradients
        dict(name="muon_masters", op="muon",
             stacks="4x2048x2048,1x512x2048,1x512x2048,1x512x2048,2x1163x501", dtype="bf16",
             grad="bf16", master=True, nesterov=True, decay=0.1, clip=True),
        # all expert weights of one 128-expert block, float32 gradients as its backward leaves them
        dict(name="muon_experts", op="muon", stacks="128x768x2048,128x768x2048,128x2048x768",
             dtype="bf16", grad="f32", master=False, nesterov=True, decay=0.1, clip=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["policy", "balance", "ortho", "muon"])
    if op == "policy":
        T = _log_int(rng, 1, 1000000)
        ratio = rng.choice(["token", "sequence"])
        high = rng.choice([0.2, 0.28]) if ratio == "token" else rng.choice([4e-4, 2e-3])
        return dict(op=op, T=T, S=_log_int(rng, 1, max(1, min(2048, T // 8))), ratio=ratio,
                    reduce=rng.choice(["token", "sequence"]), per_token=rng.random() < 0.5,
                    infer=rng.random() < 0.5, ref=rng.random() < 0.5, entropy=rng.random() < 0.5,
                    mask=rng.choice([0.0, 0.1, 0.5]), dual=rng.choice([0.0, 3.0]), high=high)
    if op == "balance":
        E = rng.choice([8, 16, 60, 64, 128, 160, 256, rng.randint(3, 512)])
        L = rng.choice([1, 1, 2, rng.randint(3, 48)])
        T = _log_int(rng, 1, min(65536, 100000000 // (L * E)))
        return dict(op=op, L=L, T=T, E=E, K=rng.randint(1, min(E, 10)),
                    idx="i16" if E > 256 else rng.choice(["u8", "i16"]),
                    mask=rng.choice([0.0, 0.0, 0.3]), z=rng.choice([0.0, 1e-3]))
    if op == "ortho":
        rows, cols = _log_int(rng, 1, 4096), _log_int(rng, 1, 4096)
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["bf16", "f32"]),
                    B=_log_int(rng, 1, max(1, min(64, 60000000 // (rows * cols)))))
    left, stacks = 60000000, []
    for _ in range(rng.randint(1, 4)):
        rows, cols = _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
        if rows * cols > left:
            break
        B = _log_int(rng, 1, max(1, min(128, left // (rows * cols))))
        left -= B * rows * cols
        stacks.append("%dx%dx%d" % (B, rows, cols))
    dtype = rng.choice(["bf16", "f32"])
    return dict(op=op, stacks=",".join(stacks) or "1x1024x1024", dtype=dtype,
                grad=rng.choice(["bf16", "f32"]), master=dtype == "bf16" and rng.random() < 0.5,
                nesterov=rng.random() < 0.7, decay=rng.choice([0.0, 0.1]), clip=rng.random() < 0.5)


def _stacks(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["stacks"].split(",")]


# ---------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _prepare_policy(case, seed):
    g = _gen(seed)
    T, S = case["T"], case["S"]

    def randn(n=T):
        return torch.randn(n, generator=g, device="cuda")

    # response lengths spread over two decades
    share = torch.exp(1.2 * randn(S)).cumsum(0)
    cut = (share / share[-1] * T).round().to(torch.int32)
    cut[-1] = T
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), cut])
    # a policy a few steps away from the one that sampled, the rollout engine's rounding in between
    old = -torch.rand(T, generator=g, device="cuda").pow(3) * 9.0
    s = dict(case=case, cu=cu, old=old, logp=(old + 0.12 * randn()).clamp(max=-1e-7), infer=None,
             ref=None, entropy=None, mask=None, adv=None, seq_adv=None)
    if case["infer"]:
        far = torch.where(torch.rand(T, generator=g, device="cuda") < 0.01, 1.0, 0.05)
        s["infer"] = (old + far * randn()).clamp(max=-1e-7)
    if case["ref"]:
        s["ref"] = (old + 0.2 * randn()).clamp(max=-1e-7)
    if case["entropy"]:
        s["entropy"] = torch.rand(T, generator=g, device="cuda") * 2.0
    if case["mask"]:
        s["mask"] = torch.rand(T, generator=g, device="cuda") >= case["mask"]
        # what stands in prompt and padding is no probability of anything
        for k in ("logp", "old", "infer", "ref", "entropy"):
            if s[k] is not None:
                s[k] = torch.where(s["mask"], s[k], math.nan)
    # rewards within a group of responses, less their mean and over their deviation
    if case["per_token"]:
        s["adv"] = randn()
    else:
        s["seq_adv"] = randn(S)
    return s


def _prepare_balance(case, seed):
    g = _gen(seed)
    L, T, E, K = case["L"], case["T"], case["E"], case["K"]
    # some experts are liked by all tokens, as in a router that has begun to lean
    lean = torch.randn((L, 1, E), generator=g, device="cuda") * 0.6
    logits = torch.randn((L, T, E), generator=g, device="cuda").add_(lean)
    # the record of a rollout engine whose logits differ a little
    idx = torch.empty((L, T, K), dtype=torch.uint8 if case["idx"] == "u8" else torch.int16,
                      device="cuda")
    for i in range(L):
        noise = torch.randn((T, E), generator=g, device="cuda") * 0.02
        idx[i] = (logits[i] + noise).topk(K, dim=1).indices.to(idx.dtype)
    s = dict(case=case, logits=logits, idx=idx, mask=None)
    if case["mask"]:
        s["mask"] = torch.rand(T, generator=g, device="cuda") >= case["mask"]
        s["mask"][0] = True
    return s


def _matrices(g, B, rows, cols, std):
    """[B, rows, cols] as gradients are: some strong directions over a floor of noise."""
    r = min(rows, cols, 24)
    strong = torch.randn((B, rows, r), generator=g, device="cuda")
    strong *= torch.exp(-0.3 * torch.arange(r, device="cuda"))
    x = torch.bmm(strong, torch.randn((B, r, cols), generator=g, device="cuda"))
    noise = torch.randn((B, rows, cols), generator=g, device="cuda")
    return noise.mul_(0.3).add_(x).mul_(std)


def _prepare_ortho(case, seed):
    return dict(case=case, x=_matrices(_gen(seed), case["B"], case["rows"], case["cols"],
                                       1e-3).to(DTYPES[case["dtype"]]))


def _prepare_muon(case, seed):
    g = _gen(seed)
    s = dict(case=case, lr=0.02, momentum=0.95, param=[], master=[], grad=[], buf=[], grad_scale=None)
    for B, rows, cols in _stacks(case):
        w = torch.randn((B, rows, cols), generator=g, device="cuda") * 0.02
        s["param"].append(w.to(DTYPES[case["dtype"]]))
        if case["master"]:
            s["master"].append(w)
        s["grad"].append(_matrices(g, B, rows, cols, 1e-3).to(DTYPES[case["grad"]]))
        s["buf"].append(_matrices(g, B, rows, cols, 1e-2))
    if case["clip"]:
        s["grad_scale"] = torch.full((1,), 0.37, device="cuda")
    return s


def prepare(case, seed):
    return {"policy": _prepare_policy, "balance": _prepare_balance, "ortho": _prepare_ortho,
            "muon": _prepare_muon}[case["op"]](case, seed)


# ---------------------------------------------------------------------------------------------
INFER_CAP, CLIP_LOW, KL_COEF, ENTROPY_COEF = 2.0, 0.2, 0.02, 0.001


def _low(case):
    return CLIP_LOW if case["ratio"] == "token" else 0.75 * case["high"]


def _plain_policy(s):
    c = s["case"]
    T, S = c["T"], c["S"]
    cu = s["cu"].long()
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), cu[1:] - cu[:-1], output_size=T)
    kept = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]

    def value(k):
        return torch.where(kept, s[k], 0.0).double()

    def per_seq(v):
        return torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, seq, v)

    n = per_seq(kept.double())
    count = n.sum()
    d = value("logp") - value("old")
    if c["ratio"] == "sequence":
        d = (per_seq(d) / n.clamp(min=1))[seq]
    # the borders of the clip ranges are those of the logarithm, in 64 bits
    adv = (s["adv"] if c["per_token"] else s["seq_adv"][seq]).float()
    up, down = adv > 0, adv < 0
    high = kept & up & (d > math.log1p(c["high"]))
    low = kept & down & (d < math.log1p(-_low(c)))
    far = kept & down & (d > math.log(c["dual"])) if c["dual"] else torch.zeros_like(kept)
    ratio = d.float().exp()
    w = torch.ones(T, device="cuda")
    cut = torch.zeros_like(kept)
    if s["infer"] is not None:
        x = value("old") - value("infer")
        cut = kept & (x > math.log(INFER_CAP))
        w = torch.where(cut, INFER_CAP, x.float().exp())
    used = torch.where(high, 1 + c["high"], torch.where(low, 1 - _low(c), torch.where(
        far, c["dual"], ratio)))
    wa = w * adv * kept
    term = -wa * used
    slope = torch.where(high | low | far, 0.0, -wa * ratio)
    if c["reduce"] == "token":
        weight = kept / count.clamp(min=1)
    else:
        weight = kept / (n.clamp(min=1) * (n > 0).sum().clamp(min=1))[seq]
    if c["ratio"] == "sequence":
        slope = (per_seq(slope * weight) / n.clamp(min=1))[seq] * kept
    else:
        slope = slope * weight
    total = (term * weight).sum()
    metrics = [total]
    if s["ref"] is not None:
        x = value("ref") - value("logp")
        kl = ((torch.expm1(x) - x) * weight).sum()
        slope = slope - KL_COEF * torch.expm1(x) * weight
        total = total + KL_COEF * kl
        metrics.append(kl)
    else:
        metrics.append(torch.zeros_like(total))
    out = {}
    if s["entropy"] is not None:
        ent = (value("entropy") * weight).sum()
        total = total - ENTROPY_COEF * ent
        metrics.append(ent)
        out["dentropy"] = (-ENTROPY_COEF * weight).float()
    else:
        metrics.append(torch.zeros_like(total))
    out["loss"] = total.float()[None]
    out["dlogp"] = slope.float()
    out["metrics"] = torch.stack(metrics).float()
    out["counts"] = torch.stack([kept.sum(), (high | low | far).sum(), cut.sum()]).to(torch.int32)
    return out


def _own_policy(s):
    from paper_2510_11370_b200 import r3
    c = s["case"]
    loss, dlogp, dentropy, metrics, counts = r3.policy_loss(
        s["logp"], s["old"], s["cu"], advantages=s["adv"], seq_advantages=s["seq_adv"],
        mask=s["mask"], logp_infer=s["infer"], logp_ref=s["ref"], entropy=s["entropy"],
        ratio=c["ratio"], reduce=c["reduce"], clip_low=_low(c), clip_high=c["high"],
        dual_clip=c["dual"], infer_cap=INFER_CAP, kl_coef=KL_COEF, entropy_coef=ENTROPY_COEF)
    out = {"loss": loss, "dlogp": dlogp, "metrics": metrics, "counts": counts}
    if dentropy is not None:
        out["dentropy"] = dentropy
    return out


BALANCE_COEF = 0.01


def _plain_balance(s):
    c = s["case"]
    L, T, E, K = c["L"], c["T"], c["E"], c["K"]
    kept = torch.ones(T, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"]
    n = kept.sum().clamp(min=1).float()
    loss = torch.empty((L, 2), device="cuda")
    counts = torch.empty((L, E), dtype=torch.int32, device="cuda")
    dlogits = torch.empty((L, T, E), device="cuda")
    for i in range(L):
        z = s["logits"][i]
        top = z.amax(1, keepdim=True)
        e = (z - top).exp()
        whole = e.sum(1, keepdim=True)
        p = e / whole
        lse = top + whole.log()
        hits = torch.zeros(E, dtype=torch.float64, device="cuda")
        hits.index_add_(0, s["idx"][i].reshape(-1).long(),
                        kept.double()[:, None].expand(T, K).reshape(-1))
        share = (hits / (n * K) * E).float()
        mean = (p * kept[:, None]).double().sum(0) / n
        loss[i, 0] = (share * mean).sum()
        loss[i, 1] = (lse[:, 0].square() * kept).double().sum() / n
        counts[i] = hits.to(torch.int32)
        d = BALANCE_COEF * p * (share - (p * share).sum(1, keepdim=True))
        if c["z"]:
            d += 2 * c["z"] * lse * p
        dlogits[i] = torch.where(kept[:, None], d / n, 0.0)
    return {"loss": loss, "counts": counts, "dlogits": dlogits}


def _own_balance(s):
    from paper_2510_11370_b200 import r3
    c = s["case"]
    shape = r3.make_shape(c["T"], 8, c["E"], c["K"], 8, idx=s["idx"].dtype)
    loss, counts, dlogits = r3.balance_loss(shape, c["L"], s["logits"], s["idx"], mask=s["mask"],
                                            balance_coef=BALANCE_COEF, z_coef=c["z"])
    return {"loss": loss, "counts": counts, "dlogits": dlogits}


def _newton_schulz(u, steps=5):
    """[B, rows, cols] float32 -> the iteration's result, float32."""
    flip = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if flip else u
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt().float()
    x = x / (norm + 1e-7)
    a, b, c = QUINTIC
    for _ in range(steps):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)
    return x.transpose(1, 2) if flip else x


def _plain_ortho(s):
    return {"out": _newton_schulz(s["x"].float()).to(s["x"].dtype)}


def _own_ortho(s):
    from paper_2510_11370_b200 import r3
    return {"out": r3.orthogonalize(s["x"])}


def _scale(rows, cols):
    """What the orthogonal factor is multiplied with: tall matrices map to longer vectors."""
    return math.sqrt(max(1.0, rows / cols))


def _muon_outputs(s):
    names = ["param", "buf"] + (["master"] if s["master"] else [])
    return {"%s%d" % (k, i): t for k in names for i, t in enumerate(s[k])}


def _plain_muon(s):
    c = s["case"]
    for i, (B, rows, cols) in enumerate(_stacks(c)):
        g = s["grad"][i].float()
        if s["grad_scale"] is not None:
            g = g * s["grad_scale"]
        s["buf"][i].mul_(s["momentum"]).add_(g)
        u = g + s["momentum"] * s["buf"][i] if c["nesterov"] else s["buf"][i]
        w = s["master"][i] if c["master"] else s["param"][i].float()
        w = w * (1 - s["lr"] * c["decay"]) - s["lr"] * _scale(rows, cols) * _newton_schulz(u)
        if c["master"]:
            s["master"][i].copy_(w)
        s["param"][i].copy_(w)
    return _muon_outputs(s)


def _own_muon(s):
    if "optimiser" not in s:
        # the handle that a training program keeps beside its parameters
        from paper_2510_11370_b200 import r3
        c = s["case"]
        s["optimiser"] = r3.Muon(s["param"], s["grad"], masters=s["master"] if c["master"] else None,
                                 momentum_buffers=s["buf"], momentum=s["momentum"],
                                 nesterov=c["nesterov"], weight_decay=c["decay"])
    s["optimiser"].step(s["lr"], grad_scale=s["grad_scale"])
    return _muon_outputs(s)


PLAIN = {"policy": _plain_policy, "balance": _plain_balance, "ortho": _plain_ortho,
         "muon": _plain_muon}
OWN = {"policy": _own_policy, "balance": _own_balance, "ortho": _own_ortho, "muon": _own_muon}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
def _products(rows, cols, steps=5):
    """Operations of the iteration: the Gram matrix and its square are symmetric, half of each is
    enough; their product with the matrix is whole."""
    m, n = min(rows, cols), max(rows, cols)
    return steps * (m * m * n + m ** 3 + 2 * m * m * n)


def work(case):
    op = case["op"]
    if op == "policy":
        read = 8 + sum(4 for k in ("infer", "ref", "entropy", "per_token") if case[k])
        read += 1 if case["mask"] else 0
        kept = 1 - case["mask"]
        return {"bytes": case["T"] * (read + 4 + (4 if case["entropy"] else 0)) + 8 * case["S"],
                "flops": 40 * kept * case["T"]}
    if op == "balance":
        rows = case["L"] * case["T"]
        moved = rows * (4 * case["E"] * (2 - case["mask"])
                        + case["K"] * (1 if case["idx"] == "u8" else 2))
        return {"bytes": moved, "flops": rows * (1 - case["mask"]) * case["E"] * 20}
    if op == "ortho":
        n = case["B"] * case["rows"] * case["cols"]
        return {"bytes": n * (4 if case["dtype"] == "bf16" else 8),
                "flops": case["B"] * _products(case["rows"], case["cols"])}
    p, g = (2 if case["dtype"] == "bf16" else 4), (2 if case["grad"] == "bf16" else 4)
    # momentum read and written; with masters the stored parameter is written only
    moved = 8 + g + ((8 + p) if case["master"] else 2 * p)
    return {"bytes": sum(B * r * c for B, r, c in _stacks(case)) * moved,
            "flops": sum(B * _products(r, c) for B, r, c in _stacks(case))}


# ---------------------------------------------------------------------------------------------
# The definitions once more, in 64 bits.
def _exact_policy(s):
    """By differentiating the loss as it is written down."""
    c = s["case"]
    cu = s["cu"].tolist()
    T, S = c["T"], c["S"]
    live = torch.arange(T, device="cuda") if s["mask"] is None else s["mask"].nonzero()[:, 0]
    owner = torch.bucketize(live, s["cu"][1:].long(), right=True)
    lp = s["logp"][live].double().requires_grad_()
    old = s["old"][live].double()
    length = torch.bincount(owner, minlength=S).double()
    ratio = torch.exp(lp - old)
    if c["ratio"] == "sequence":
        mean = torch.zeros(S, dtype=torch.float64, device="cuda").index_add(0, owner, lp - old)
        ratio = torch.exp(mean / length.clamp(min=1))[owner]
    adv = (s["adv"][live] if c["per_token"] else s["seq_adv"][owner]).double()
    inner = torch.clamp(ratio, 1 - _low(c), 1 + c["high"])
    gain = torch.minimum(ratio * adv, inner * adv)
    bound = (inner != ratio) & (inner * adv < ratio * adv)
    if c["dual"]:
        floor = torch.maximum(gain, c["dual"] * adv)
        bound = bound | ((adv < 0) & (floor > gain))
        gain = torch.where(adv < 0, floor, gain)
    cut = torch.zeros_like(bound)
    if s["infer"] is not None:
        w = torch.exp(old - s["infer"][live].double())
        cut = w > INFER_CAP
        gain = gain * w.clamp(max=INFER_CAP)
    if c["reduce"] == "token":
        weight = torch.full_like(old, 1.0 / max(1, live.numel()))
    else:
        weight = 1.0 / (length[owner] * int((length > 0).sum()))
    policy = -(gain * weight).sum()
    loss, kl, ent = policy, torch.zeros_like(policy), torch.zeros_like(policy)
    if s["ref"] is not None:
        x = s["ref"][live].double() - lp
        kl = ((torch.exp(x) - 1 - x) * weight).sum()
        loss = loss + KL_COEF * kl
    if s["entropy"] is not None:
        h = s["entropy"][live].double().requires_grad_()
        ent = (h * weight).sum()
        loss = loss - ENTROPY_COEF * ent
    grads = torch.autograd.grad(loss, [lp] + ([h] if s["entropy"] is not None else []))

    def spread(v):
        return torch.zeros(T, dtype=torch.float64, device="cuda").index_copy(0, live, v)

    out = {"loss": loss.detach()[None], "dlogp": spread(grads[0]),
           "metrics": torch.stack([policy, kl, ent]).detach(),
           "counts": torch.stack([torch.tensor(live.numel(), device="cuda"), bound.sum(), cut.sum()])}
    if s["entropy"] is not None:
        out["dentropy"] = spread(grads[1])
    return out if cu[-1] == T else None


def _exact_balance(s):
    c = s["case"]
    L, T, E, K = c["L"], c["T"], c["E"], c["K"]
    kept = torch.arange(T, device="cuda") if s["mask"] is None else s["mask"].nonzero()[:, 0]
    loss, counts, grads = [], [], []
    for i in range(L):
        z = s["logits"][i][kept].double().requires_grad_()
        hits = torch.bincount(s["idx"][i][kept].long().flatten(), minlength=E)
        logp = torch.log_softmax(z, 1)
        balance = E / (K * kept.numel()) * (hits * logp.exp().mean(0)).sum()
        zed = torch.logsumexp(z, 1).square().mean()
        (d,) = torch.autograd.grad(BALANCE_COEF * balance + c["z"] * zed, z)
        loss.append(torch.stack([balance, zed]).detach())
        counts.append(hits)
        grads.append(torch.zeros((T, E), dtype=torch.float64, device="cuda").index_copy(0, kept, d))
    return {"loss": torch.stack(loss), "counts": torch.stack(counts), "dlogits": torch.stack(grads)}


def _exact_iteration(u):
    """One matrix [rows, cols] float64; the side of the smaller dimension is the Gram matrix's."""
    x = u / (torch.linalg.matrix_norm(u) + 1e-7)
    a, b, c = QUINTIC
    eye = torch.eye(min(x.shape), dtype=x.dtype, device=x.device)
    for _ in range(5):
        if x.shape[0] <= x.shape[1]:
            gram = x @ x.T
            x = (a * eye + gram @ (b * eye + c * gram)) @ x
        else:
            gram = x.T @ x
            x = x @ (a * eye + gram @ (b * eye + c * gram))
    return x


def _exact_muon(s):
    c, out = s["case"], {}
    for i, (B, rows, cols) in enumerate(_stacks(c)):
        names = ["param", "buf"] + (["master"] if c["master"] else [])
        for k in names:
            out["%s%d" % (k, i)] = torch.empty((B, rows, cols), dtype=torch.float64, device="cuda")
        scale = 1.0 if s["grad_scale"] is None else s["grad_scale"].double()
        for j in range(B):
            g = s["grad"][i][j].double() * scale
            m = s["momentum"] * s["buf"][i][j].double() + g
            o = _exact_iteration(g + s["momentum"] * m if c["nesterov"] else m)
            w = (s["master"] if c["master"] else s["param"])[i][j].double()
            w = w - s["lr"] * (c["decay"] * w + _scale(rows, cols) * o)
            for k, v in zip(names, (w, m, w)):
                out["%s%d" % (k, i)][j] = v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "policy":
        return _exact_policy(s)
    if case["op"] == "balance":
        return _exact_balance(s)
    if case["op"] == "ortho":
        return {"out": torch.stack([_exact_iteration(x.double()) for x in s["x"]])}
    return _exact_muon(s)
