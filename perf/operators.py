"""The operators of an Update step around the replayed MoE block, as they are timed and compared.

  token_logprobs, token_logprobs_bwd   log probabilities of the sampled tokens, entropy and top
                                       alternatives of each row of logits, and the logits' gradient
  norm_residual, norm_residual_bwd     RMSNorm after a block, its gate, the scaled residual and the
                                       RMSNorm in front of the next block, and the gradients
  AdamW.step                           one AdamW step over many tensors, states in 32 or in 8 bits

`run` gives the plain form (elementary torch operations) where `own` is false and the framework's
entry points where it is true."""
import itertools
import math
import random

import torch

own = False

BLOCK = 256           # elements that share one scale of an 8-bit optimiser state
E4M3_MAX = 448.0      # largest finite value of the 8-bit states' type
E4M3_MIN = 2.0 ** -9  # smallest positive one
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------
def listed():
    return [
        # a decode step of a rollout engine that reports the 20 best alternatives of each token
        dict(name="logprobs_decode", op="logprobs", T=16, V=131072, dtype="bf16", n_top=20,
             entropy=True, temperature=0.7, ignored=0.0, masked=0.25, pad=0),
        # scoring a short batch of responses from float32 logits, a vocabulary of odd size
        dict(name="logprobs_score_odd", op="logprobs", T=1023, V=50257, dtype="f32", n_top=5,
             entropy=True, temperature=1.0, ignored=0.1, masked=0.0, pad=0),
        # one micro-batch of the Update stage: the training engine's log probabilities
        dict(name="logprobs_update", op="logprobs", T=8192, V=151936, dtype="bf16", n_top=0,
             entropy=True, temperature=1.0, ignored=0.1, masked=0.0, pad=0),
        # gradient of a short batch with an entropy bonus
        dict(name="logprobs_bwd_odd", op="logprobs_bwd", T=257, V=50257, dtype="f32",
             entropy=True, temperature=0.8, ignored=0.1, masked=0.25, pad=0),
        # gradient of the Update stage's micro-batch
        dict(name="logprobs_bwd_update", op="logprobs_bwd", T=8192, V=151936, dtype="bf16",
             entropy=False, temperature=1.0, ignored=0.1, masked=0.0, pad=0),
        # the decode batch of the capture workload between two blocks
        dict(name="norm_decode", op="norm", T=256, d=2048, dtype="bf16", w_dtype="bf16",
             gate="channel", post=True, pre=True, first=False),
        # the token batch of one block of the 48-block stack
        dict(name="norm_stack", op="norm", T=16384, d=2048, dtype="bf16", w_dtype="bf16",
             gate="channel", post=True, pre=True, first=False),
        # float32 activations, odd token count, gate per token
        dict(name="norm_bwd_odd", op="norm_bwd", T=4097, d=1160, dtype="f32", w_dtype="f32",
             gate="token", post=True, pre=True, first=False),
        # the replayed batch of 65536 tokens going back through one block
        dict(name="norm_bwd_replay", op="norm_bwd", T=65536, d=2048, dtype="bf16", w_dtype="bf16",
             gate="channel", post=True, pre=True, first=False),
        # the small parameters of one block: the router weight and four norm weights
        dict(name="adamw_router", op="adamw", sizes="262144,2048,2048,2048,2048", dtype="f32",
             grad="f32", master=False, bits=32, clip=True, decay=0.0),
        # many odd tensors with float32 master weights and 32-bit states
        dict(name="adamw_ragged", op="adamw", sizes="ragged:150:120000000", dtype="bf16",
             grad="bf16", master=True, bits=32, clip=True, decay=0.1),
        # the expert weights of one 128-expert block, float32 gradients, 8-bit states
        dict(name="adamw_experts_8bit", op="adamw", sizes="201326592,201326592,201326592",
             dtype="bf16", grad="f32", master=False, bits=8, clip=True, decay=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs_bwd", "norm", "norm_bwd", "adamw"])
    if op in ("logprobs", "logprobs_bwd"):
        dtype = rng.choice(["bf16", "f32"])
        V = _log_int(rng, 700, 200000)
        n_top = rng.choice([0, 0, 1, rng.randint(2, 32)]) if op == "logprobs" else 0
        cells = (1 << 27) if n_top else (1200000000 if dtype == "bf16" else 600000000)
        T = _log_int(rng, 1, max(1, min(8192, cells // (V + 64))))
        case = dict(op=op, T=T, V=V, dtype=dtype, entropy=rng.random() < 0.6,
                    temperature=rng.choice([1.0, 0.6, 1.3]), ignored=rng.choice([0.0, 0.1, 0.4]),
                    masked=rng.choice([0.0, 0.25, 0.9]), pad=rng.choice([0, 0, 7, 64]))
        if op == "logprobs":
            case["n_top"] = n_top
        return case
    if op in ("norm", "norm_bwd"):
        dtype = rng.choice(["bf16", "f32"])
        d = 8 * _log_int(rng, 8, 1024)
        T = _log_int(rng, 1, 134000000 // d if dtype == "bf16" else 67000000 // d)
        post, pre = rng.choice([(True, True), (True, True), (False, True), (True, False)])
        first = pre and rng.random() < 0.15
        return dict(op=op, T=min(T, 65536), d=d, dtype=dtype, w_dtype=rng.choice(["bf16", "f32"]),
                    gate="none" if first else rng.choice(["none", "channel", "token", "full"]),
                    post=post and not first, pre=pre, first=first)
    total = _log_int(rng, 3000, 250000000)
    count = min(_log_int(rng, 1, 400), total // 100)
    dtype = rng.choice(["bf16", "f32"])
    return dict(op=op, sizes="ragged:%d:%d" % (count, total), dtype=dtype,
                grad=rng.choice(["bf16", "f32"]), master=dtype == "bf16" and rng.random() < 0.5,
                bits=rng.choice([8, 32]), clip=rng.random() < 0.5, decay=rng.choice([0.0, 0.1]))


def _sizes(case):
    """Element counts of the tensors of an optimiser case."""
    text = case["sizes"]
    if not text.startswith("ragged:"):
        return [int(n) for n in text.split(",")]
    count, total = (int(n) for n in text.split(":")[1:])
    rng = random.Random(total)
    share = [rng.random() ** 3 + 1e-3 for _ in range(count)]
    whole = sum(share)
    return [max(1, int(total * s / whole)) for s in share]


# ---------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _prepare_logits(case, seed):
    g = _gen(seed)
    T, V, dtype = case["T"], case["V"], DTYPES[case["dtype"]]
    z = torch.randn((T, V), generator=g, device="cuda") * 2.5
    # a trained model's rows: some peaked on one token, others broad
    best = torch.randint(0, V, (T, 1), generator=g, device="cuda")
    z.scatter_add_(1, best, torch.rand((T, 1), generator=g, device="cuda") * 16.0)
    if case["masked"]:
        # a sampler's or a grammar's mask: the same share of the vocabulary shut in every other
        # row, by infinity or by the type's lowest value
        shut = torch.rand((T, V), generator=g, device="cuda") < case["masked"]
        shut &= (torch.arange(T, device="cuda") % 2 == 1)[:, None]
        shut.scatter_(1, best, False)
        low = torch.where(torch.arange(T, device="cuda") % 4 == 1, -math.inf,
                          torch.finfo(dtype).min)[:, None]
        z = torch.where(shut, low, z)
    logits = torch.empty((T, V + case["pad"]), dtype=dtype, device="cuda")[:, :V]
    logits.copy_(z)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    likely = torch.rand(T, generator=g, device="cuda") < 0.7
    ids = torch.where(likely, logits.argmax(1), ids)
    ids = torch.where(logits.gather(1, ids[:, None])[:, 0] < -1e30, logits.argmax(1), ids)
    ids[torch.rand(T, generator=g, device="cuda") < case["ignored"]] = -1   # prompt and padding
    return g, logits, ids


def _prepare_norm(case, seed):
    g = _gen(seed)
    T, d, dtype, w_dtype = case["T"], case["d"], DTYPES[case["dtype"]], DTYPES[case["w_dtype"]]
    shape = {"none": None, "channel": (d,), "token": (T,), "full": (T, d)}[case["gate"]]
    s = dict(case=case, x=_randn(g, (T, d), dtype), y=_randn(g, (T, d), dtype, 0.3), gate=None,
             w_post=None, w_pre=None, residual_scale=1.0, branch_scale=0.7, eps=1e-6)
    if shape:
        s["gate"] = (torch.rand(shape, generator=g, device="cuda") + 0.25).to(
            torch.float32 if case["gate"] == "token" else dtype if case["gate"] == "full" else w_dtype)
    if case["post"]:
        s["w_post"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(w_dtype)
    if case["pre"]:
        s["w_pre"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(w_dtype)
    if case["first"]:
        s["y"] = None
    if case["op"] == "norm_bwd":
        # x_out of the forward is what a training step keeps beside y
        s["x_out"] = s.pop("x")
        s["dx_out"] = None if case["first"] else _randn(g, (T, d), dtype)
        s["dh"] = _randn(g, (T, d), dtype) if case["pre"] else None
    return s


def _quantise(v):
    """[blocks, BLOCK] float32 -> (float8 values, scale [blocks]): the scale is the smallest power
    of two (at least 2^-126) that brings the block's largest magnitude to at most 448."""
    mantissa, exponent = torch.frexp(v.abs().amax(1))
    k = (exponent - 9 + (mantissa > 0.875).to(torch.int32)).clamp(min=-126)
    k = torch.where(mantissa == 0, torch.full_like(k, -126), k)
    scale = ((k + 127) << 23).view(torch.float32)
    return (v / scale[:, None]).to(torch.float8_e4m3fn), scale


def _quantise_root(v):
    """The same for the second moment, held as its square root; a root above zero is never held
    as zero (the update divides by it)."""
    root = v.sqrt()
    code, scale = _quantise(root)
    tiny = (root > 0) & (code.float() == 0)
    return torch.where(tiny, E4M3_MIN, code.float()).to(torch.float8_e4m3fn), scale


def _prepare_adamw(case, seed):
    g = _gen(seed)
    sizes = _sizes(case)
    # the tensors lie one behind the other in flat buffers, each from a multiple of BLOCK on
    blocks = [-(-n // BLOCK) for n in sizes]
    starts = [0, *itertools.accumulate(blocks)]
    total = starts.pop()
    of_tensor = torch.repeat_interleave(torch.arange(len(sizes)), torch.tensor(blocks)).cuda()
    place = torch.arange(total * BLOCK, device="cuda").view(total, BLOCK)
    place -= BLOCK * torch.tensor(starts, device="cuda")[of_tensor][:, None]
    live = place < torch.tensor(sizes, device="cuda")[of_tensor][:, None]
    size = torch.exp(torch.randn((total, 1), generator=g, device="cuda"))   # layers differ in scale

    def normal(std):
        return torch.randn((total, BLOCK), generator=g, device="cuda") * std * live

    s = dict(case=case, sizes=sizes, starts=starts, blocks=blocks, step=37, lr=3e-4,
             betas=(0.9, 0.95), eps=1e-8, grad_scale=None)
    w = normal(0.02)
    s["param"] = w.to(DTYPES[case["dtype"]])
    s["master"] = w if case["master"] else None
    s["grad"] = (normal(2e-3) * size).to(DTYPES[case["grad"]])
    m = normal(5e-4) * size
    v = (normal(1e-3) * size).square() + (3e-4 * size * live).square()
    if case["bits"] == 8:
        s["exp_avg"], s["exp_avg_scale"] = _quantise(m)
        s["exp_avg_sq"], s["exp_avg_sq_scale"] = _quantise_root(v)
    else:
        s["exp_avg"], s["exp_avg_sq"] = m, v
    if case["clip"]:
        s["grad_scale"] = torch.full((1,), 0.37, device="cuda")
    # weight decay for every tensor but the small ones (norms, biases)
    s["decay"] = [case["decay"] if n > 4096 else 0.0 for n in sizes]
    s["decay_of_block"] = torch.tensor(s["decay"], device="cuda")[of_tensor][:, None]
    return s


def prepare(case, seed):
    op = case["op"]
    if op.startswith("norm"):
        return _prepare_norm(case, seed)
    if op == "adamw":
        return _prepare_adamw(case, seed)
    g, logits, ids = _prepare_logits(case, seed)
    s = dict(case=case, logits=logits, ids=ids)
    if op == "logprobs_bwd":
        T = case["T"]
        # what the forward of the training step left: the largest logit of each row, the logarithm
        # of the sum of exponentials above it, and the entropy
        stats = torch.zeros((T, 2), device="cuda")
        ent = torch.zeros(T, device="cuda")
        slab = max(1, (1 << 27) // case["V"])
        for lo in range(0, T, slab):
            z = logits[lo:lo + slab].double()
            top = z.amax(1, keepdim=True)
            z = (z - top) / case["temperature"]
            total = z.exp().sum(1, keepdim=True).log()
            stats[lo:lo + slab, 0] = top[:, 0].float()
            stats[lo:lo + slab, 1] = total[:, 0].float()
            p = (z - total).exp()
            ent[lo:lo + slab] = -torch.where(p > 0, p * (z - total), 0.0).sum(1).float()
        kept = ids >= 0
        s["stats"] = torch.where(kept[:, None], stats, 0.0)
        s["entropy"] = torch.where(kept, ent, 0.0)
        s["dlogp"] = torch.randn(T, generator=g, device="cuda") / T
        s["dentropy"] = torch.full((T,), -0.01 / T, device="cuda") if case["entropy"] else None
    return s


# ---------------------------------------------------------------------------------------------
def _top(logits, n):
    """Indices of the n largest of each row, ties to the lowest index: one key per element holds
    its value's order above its index's."""
    bits = (logits.float() + 0.0).view(torch.int32).to(torch.int64)    # + 0.0: both zeros alike
    order = torch.where(bits >= 0, bits, -(bits & 0x7fffffff) - 1)
    V = logits.shape[1]
    key = order * (1 << 32) + (V - 1 - torch.arange(V, device=logits.device))
    return V - 1 - (key.topk(n, dim=1).values & 0xffffffff)


def _plain_logprobs(s):
    c = s["case"]
    kept = s["ids"] >= 0
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    z = (z - top) / c["temperature"]
    total = z.exp().sum(1, keepdim=True).log()
    z -= total
    out = {"logp": torch.where(kept, z.gather(1, s["ids"].clamp(min=0)[:, None])[:, 0], 0.0),
           "stats": torch.where(kept[:, None], torch.cat([top, total], 1), 0.0)}
    if c["entropy"]:
        p = z.exp()
        out["entropy"] = torch.where(kept, -torch.where(p > 0, p * z, 0.0).sum(1), 0.0)
    if c["n_top"]:
        best = _top(s["logits"], c["n_top"])
        out["top_ids"] = torch.where(kept[:, None], best, -1).to(torch.int32)
        out["top_logp"] = torch.where(kept[:, None], z.gather(1, best), 0.0)
    return out


def _own_logprobs(s):
    from paper_2510_11370_b200 import r3
    c = s["case"]
    logp, entropy, stats, top_ids, top_logp = r3.token_logprobs(
        s["logits"], s["ids"], temperature=c["temperature"], n_top=c["n_top"],
        want_entropy=c["entropy"], want_stats=True)
    out = {"logp": logp, "stats": stats}
    if c["entropy"]:
        out["entropy"] = entropy
    if c["n_top"]:
        out["top_ids"], out["top_logp"] = top_ids, top_logp
    return out


def _plain_logprobs_bwd(s):
    c = s["case"]
    kept = (s["ids"] >= 0)[:, None]
    z = (s["logits"].float() - s["stats"][:, :1]) / c["temperature"] - s["stats"][:, 1:]
    p = z.exp()
    dlogp = s["dlogp"][:, None]
    d = -dlogp * p
    if c["entropy"]:
        d -= torch.where(p > 0, s["dentropy"][:, None] * p * (z + s["entropy"][:, None]), 0.0)
    d.scatter_add_(1, s["ids"].clamp(min=0)[:, None], dlogp)
    return {"dlogits": torch.where(kept, d / c["temperature"], 0.0).to(s["logits"].dtype)}


def _own_logprobs_bwd(s):
    from paper_2510_11370_b200 import r3
    c = s["case"]
    return {"dlogits": r3.token_logprobs_bwd(
        s["logits"], s["ids"], s["stats"], s["dlogp"], entropy=s["entropy"] if c["entropy"] else None,
        dentropy=s["dentropy"], temperature=c["temperature"])}


def _gate(s, like):
    if s["gate"] is None:
        return 1.0
    return s["gate"].to(like.dtype)[:, None] if s["case"]["gate"] == "token" else s["gate"].to(like.dtype)


def _normed(v, w, eps):
    return v * torch.rsqrt(v.square().mean(1, keepdim=True) + eps) * w.to(v.dtype)


def _norm(s, kind):
    """The forward in the given type, not rounded."""
    x = s["x"].to(kind)
    if s["y"] is None:
        return {"h": _normed(x, s["w_pre"], s["eps"])}
    y = s["y"].to(kind)
    b = y if s["w_post"] is None else _normed(y, s["w_post"], s["eps"])
    x = s["residual_scale"] * x + s["branch_scale"] * (_gate(s, y) * b)
    out = {"x_out": x}
    if s["w_pre"] is not None:
        out["h"] = _normed(x, s["w_pre"], s["eps"])
    return out


def _plain_norm(s):
    out = _norm(s, torch.float32)
    return {k: v.to(s["x"].dtype) for k, v in out.items()}


def _own_norm(s):
    from paper_2510_11370_b200 import r3
    x_out, h = r3.norm_residual(s["x"], s["y"], w_post=s["w_post"], gate=s["gate"],
                                w_pre=s["w_pre"], eps=s["eps"], residual_scale=s["residual_scale"],
                                branch_scale=s["branch_scale"])
    out = {} if s["y"] is None else {"x_out": x_out}
    if s["w_pre"] is not None:
        out["h"] = h
    return out


def _plain_norm_bwd(s):
    c, act = s["case"], s["x_out"].dtype
    out = {}
    g = 0.0 if s["dx_out"] is None else s["dx_out"].float()
    if s["w_pre"] is not None:
        x, dh = s["x_out"].float(), s["dh"].float()
        r = torch.rsqrt(x.square().mean(1, keepdim=True) + s["eps"])
        n, u = x * r, dh * s["w_pre"].float()
        out["dw_pre"] = (dh * n).sum(0)
        g = g + r * (u - n * (u * n).mean(1, keepdim=True))
    if s["y"] is None:
        return {**out, "dx": g.to(act)}
    out["dx"] = (s["residual_scale"] * g).to(act)
    q = s["branch_scale"] * g
    y = s["y"].float()
    dn = q * _gate(s, q)
    if s["w_post"] is not None:
        r = torch.rsqrt(y.square().mean(1, keepdim=True) + s["eps"])
        n, u = y * r, dn * s["w_post"].float()
        b = n * s["w_post"].float()
        out["dw_post"] = (dn * n).sum(0)
        dn = r * (u - n * (u * n).mean(1, keepdim=True))
    else:
        b = y
    out["dy"] = dn.to(act)
    if c["gate"] == "channel":
        out["dgate"] = (q * b).sum(0)
    elif c["gate"] == "token":
        out["dgate"] = (q * b).sum(1)
    elif c["gate"] == "full":
        out["dgate"] = (q * b).to(act)
    return out


def _own_norm_bwd(s):
    from paper_2510_11370_b200 import r3
    dx, dy, dw_post, dgate, dw_pre = r3.norm_residual_bwd(
        s["x_out"], s["y"], s["dx_out"], s["dh"], w_post=s["w_post"], gate=s["gate"],
        w_pre=s["w_pre"], eps=s["eps"], residual_scale=s["residual_scale"],
        branch_scale=s["branch_scale"])
    out = {"dx": dx, "dy": dy, "dw_post": dw_post, "dgate": dgate, "dw_pre": dw_pre}
    return {k: v for k, v in out.items() if v is not None}


def _adamw_outputs(s):
    keys = ["param", "master", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale"]
    return {k: s[k] for k in keys if s.get(k) is not None}


def _plain_adamw(s):
    b1, b2 = s["betas"]
    g = s["grad"].float()
    if s["grad_scale"] is not None:
        g = g * s["grad_scale"]
    m, v = s["exp_avg"], s["exp_avg_sq"]
    if s["case"]["bits"] == 8:
        m = m.float() * s["exp_avg_scale"][:, None]
        v = (v.float() * s["exp_avg_sq_scale"][:, None]).square()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    if s["case"]["bits"] == 8:
        code, scale = _quantise(m)
        s["exp_avg"].copy_(code)
        s["exp_avg_scale"].copy_(scale)
        code, scale = _quantise_root(v)
        s["exp_avg_sq"].copy_(code)
        s["exp_avg_sq_scale"].copy_(scale)
    else:
        s["exp_avg"].copy_(m)
        s["exp_avg_sq"].copy_(v)
    w = s["param"].float() if s["master"] is None else s["master"]
    root = v.sqrt() * (1 / math.sqrt(1 - b2 ** s["step"])) + s["eps"]
    w = w * (1 - s["lr"] * s["decay_of_block"]) - s["lr"] / (1 - b1 ** s["step"]) * (m / root)
    if s["master"] is not None:
        s["master"].copy_(w)
    s["param"].copy_(w)
    return _adamw_outputs(s)


def _own_adamw(s):
    if "optimiser" not in s:
        # the handle that a training program keeps beside its parameters
        from paper_2510_11370_b200 import r3

        def views(name, unit=BLOCK):
            flat = s[name].view(-1)
            return [flat[a * unit:a * unit + (n if unit > 1 else b)]
                    for a, n, b in zip(s["starts"], s["sizes"], s["blocks"])]

        kw = {}
        if s["case"]["bits"] == 8:
            kw = dict(exp_avg_scale=views("exp_avg_scale", 1),
                      exp_avg_sq_scale=views("exp_avg_sq_scale", 1))
        s["optimiser"] = r3.AdamW(
            views("param"), views("grad"), masters=views("master") if s["case"]["master"] else None,
            exp_avg=views("exp_avg"), exp_avg_sq=views("exp_avg_sq"), state_bits=s["case"]["bits"],
            betas=s["betas"], eps=s["eps"], weight_decay=s["decay"], **kw)
    s["optimiser"].step(s["step"], s["lr"], grad_scale=s["grad_scale"])
    return _adamw_outputs(s)


PLAIN = {"logprobs": _plain_logprobs, "logprobs_bwd": _plain_logprobs_bwd, "norm": _plain_norm,
         "norm_bwd": _plain_norm_bwd, "adamw": _plain_adamw}
OWN = {"logprobs": _own_logprobs, "logprobs_bwd": _own_logprobs_bwd, "norm": _own_norm,
       "norm_bwd": _own_norm_bwd, "adamw": _own_adamw}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "adamw":
        n = sum(_sizes(case))
        p, g = (2 if case["dtype"] == "bf16" else 4), (2 if case["grad"] == "bf16" else 4)
        state = 2 * (case["bits"] / 8 + (4 / BLOCK if case["bits"] == 8 else 0))
        # with master weights the stored parameter is written only
        moved = 2 * state + g + ((8 + p) if case["master"] else 2 * p)
        return {"bytes": n * moved, "flops": 16 * n}
    size = 2 if case["dtype"] == "bf16" else 4
    if op.startswith("norm"):
        T, d = case["T"], case["d"]
        back = op == "norm_bwd"
        full = T * d * size
        if case["first"]:
            rows = 3 if back else 2
        elif back:
            rows = 4 + (2 if case["pre"] else 0)            # y, dx_out, dx, dy; x_out, dh
        else:
            rows = 3 + (1 if case["pre"] else 0)
        if back and case["gate"] == "none" and not case["post"] and not case["first"]:
            rows -= 1                                       # y is not needed
        if case["gate"] == "full":
            rows += 2 if back else 1
        other = 4 * d * ((case["pre"] + case["post"] + (case["gate"] == "channel")) * (2 if back else 1))
        return {"bytes": rows * full + other, "flops": (24 if back else 10) * T * d}
    rows = case["T"] * (1 - case["ignored"])
    moved = rows * case["V"] * size
    if op == "logprobs_bwd":
        moved += case["T"] * case["V"] * size
    return {"bytes": moved + case["T"] * (24 + 8 * case.get("n_top", 0)),
            "flops": rows * case["V"] * (8 if case["entropy"] else 5)}


# ---------------------------------------------------------------------------------------------
# The definitions once more, in 64 bits.
def _exact_logprobs(s, lo, hi):
    c = s["case"]
    ids = s["ids"][lo:hi]
    z = s["logits"][lo:hi].double()
    top = z.max(1).values
    e = ((z - top[:, None]) / c["temperature"])
    weight = torch.exp(e)
    whole = weight.sum(1)
    out = {"logp": torch.stack([e[i, t] - whole[i].log() if t >= 0 else whole.new_zeros(())
                                for i, t in enumerate(ids.tolist())]),
           "stats": torch.stack([top, whole.log()], 1) * (ids >= 0)[:, None]}
    if c["entropy"]:
        h = whole.log() - (weight * e.clamp(min=-1e5)).sum(1) / whole
        out["entropy"] = h * (ids >= 0)
    if c["n_top"]:
        best, at = torch.sort(z, dim=1, descending=True, stable=True)
        best, at = best[:, :c["n_top"]], at[:, :c["n_top"]]
        lp = (best - top[:, None]) / c["temperature"] - whole.log()[:, None]
        out["top_ids"] = torch.where((ids >= 0)[:, None], at, -1)
        out["top_logp"] = torch.where((ids >= 0)[:, None], lp, 0.0)
    return out


def _exact_logprobs_bwd(s, lo, hi):
    c = s["case"]
    ids = s["ids"][lo:hi]
    z = (s["logits"][lo:hi].double() - s["stats"][lo:hi, :1].double()) / c["temperature"]
    logp = z - s["stats"][lo:hi, 1:].double()
    p = torch.exp(logp)
    onehot = torch.zeros_like(p)
    rows = (ids >= 0).nonzero()[:, 0]
    onehot[rows, ids[rows]] = 1.0
    d = s["dlogp"][lo:hi, None].double() * (onehot - p)
    if c["entropy"]:
        lean = logp.clamp(min=-1e5) + s["entropy"][lo:hi, None].double()
        d = d - s["dentropy"][lo:hi, None].double() * p * lean
    return {"dlogits": d / c["temperature"] * (ids >= 0)[:, None]}


def _exact_norm_bwd(s):
    """By differentiating the forward's definition at the point that reproduces x_out."""
    f = {k: s[k].double() for k in ("x_out", "y", "gate", "w_post", "w_pre", "dx_out", "dh")
         if s[k] is not None}
    live = {k: f[k].clone().requires_grad_() for k in ("y", "gate", "w_post", "w_pre") if k in f}
    names = dict(s, **{k: live.get(k) for k in ("y", "gate", "w_post", "w_pre")})
    if s["y"] is None:
        x = f["x_out"].requires_grad_()
        out = _norm(dict(names, x=x), torch.float64)
        loss = (out["h"] * f["dh"]).sum()
    else:
        with torch.no_grad():
            branch = _norm(dict(s, x=torch.zeros_like(f["x_out"]), w_pre=None), torch.float64)["x_out"]
            x = (f["x_out"] - branch) / s["residual_scale"]
        x.requires_grad_()
        out = _norm(dict(names, x=x), torch.float64)
        loss = (out["x_out"] * f["dx_out"]).sum()
        if "h" in out:
            loss = loss + (out["h"] * f["dh"]).sum()
    wanted = {"dx": x, **{"d" + k: v for k, v in live.items()}}
    grads = torch.autograd.grad(loss, list(wanted.values()), allow_unused=True)
    return {k: v for k, v in zip(wanted, grads) if v is not None}


def _exact_code(v, scale):
    """The 8-bit value nearest to v / scale (ties to even), in 64 bits."""
    q = v / scale
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(q / step) * step


def _exact_scale(v):
    k = torch.ceil(torch.log2(v.abs().amax(1, keepdim=True).clamp(min=1e-300) / E4M3_MAX))
    return torch.exp2(k.clamp(min=-126))


def _exact_adamw(s, lo, hi):
    b1, b2 = s["betas"]
    g = s["grad"][lo:hi].double()
    if s["grad_scale"] is not None:
        g = g * s["grad_scale"].double()
    m, v = s["exp_avg"][lo:hi].double(), s["exp_avg_sq"][lo:hi].double()
    if s["case"]["bits"] == 8:
        m = m * s["exp_avg_scale"][lo:hi, None].double()
        v = (v * s["exp_avg_sq_scale"][lo:hi, None].double()) ** 2
    m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g * g - v)
    w = (s["param"] if s["master"] is None else s["master"])[lo:hi].double()
    mh, vh = m / (1 - b1 ** s["step"]), v / (1 - b2 ** s["step"])
    w = w - s["lr"] * (mh / (vh.sqrt() + s["eps"]) + s["decay_of_block"][lo:hi].double() * w)
    out = {"param": w, "exp_avg": m, "exp_avg_sq": v}
    if s["master"] is not None:
        out["master"] = w
    if s["case"]["bits"] == 8:
        ms, vs = _exact_scale(m), _exact_scale(v.sqrt())
        code = _exact_code(v.sqrt(), vs)
        out["exp_avg"], out["exp_avg_scale"] = _exact_code(m, ms), ms[:, 0]
        out["exp_avg_sq"] = torch.where((v > 0) & (code == 0), E4M3_MIN, code)
        out["exp_avg_sq_scale"] = vs[:, 0]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _norm(s, torch.float64)
    if case["op"] == "norm_bwd":
        return _exact_norm_bwd(s)
    if case["op"] == "adamw":
        part, rows, width = _exact_adamw, s["param"].shape[0], BLOCK
    else:
        part = _exact_logprobs if case["op"] == "logprobs" else _exact_logprobs_bwd
        rows, width = case["T"], case["V"]
    step = max(1, (1 << 28) // width)
    parts = [part(s, lo, min(rows, lo + step)) for lo in range(0, rows, step)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
