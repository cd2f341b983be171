"""Float64 oracle of the Update step's losses: the clipped policy loss over packed responses and the
routers' balance loss, written from their formulas.  Test infrastructure only."""
import numpy as np


def policy_loss(logp, logp_old, advantages, cu_seqlens, mask=None, logp_infer=None, logp_ref=None,
                entropy=None, ratio="token", reduce="token", clip_low=0.2, clip_high=0.2, dual_clip=0.0,
                infer_cap=2.0, kl_coef=0.0, entropy_coef=0.0, denominator=0.0):
    """Returns a dict: loss, policy, kl, entropy (weighted sums), tokens, clipped, cut, dlogp, dentropy, and
    what bounds are made of: policy_grad, kl_grad (dlogp's parts), size (weighted sum of |term|), d."""
    T = len(logp)
    adv = np.asarray(advantages, dtype=np.float64)
    seqs = [np.arange(a, b) for a, b in zip(cu_seqlens[:-1], cu_seqlens[1:])]
    on = np.ones(T, dtype=bool) if mask is None else np.asarray(mask).astype(bool)
    seqs = [s[on[s]] for s in seqs]
    n_tokens, n_seqs = sum(map(len, seqs)), sum(len(s) > 0 for s in seqs)
    D = denominator if denominator > 0 else max(1, n_tokens if reduce == "token" else n_seqs)
    out = dict(policy=0.0, kl=0.0, entropy=0.0, tokens=n_tokens, clipped=0, cut=0, size=0.0,
               dlogp=np.zeros(T), dentropy=np.zeros(T), policy_grad=np.zeros(T), kl_grad=np.zeros(T),
               seq_size=np.zeros(T), d=np.zeros(T), x=np.zeros(T))
    with np.errstate(all="ignore"):
        for i, s in enumerate(seqs):
            if len(s) == 0:
                continue
            weight = 1.0 / D if reduce == "token" else 1.0 / (D * len(s))
            A = adv[s] if adv.shape[0] == T and not getattr(advantages, "per_sequence", False) else \
                np.full(len(s), adv[i])
            d = logp[s] - logp_old[s]
            if ratio == "sequence":
                d = np.full(len(s), d.sum() / len(s))
            w, cut = np.ones(len(s)), np.zeros(len(s), dtype=bool)
            if logp_infer is not None:
                x = logp_old[s] - logp_infer[s]
                cut = x > np.log(infer_cap)
                w = np.where(cut, infer_cap, np.exp(x))
                out["x"][s] = x
            rho = np.exp(d)
            high = (A > 0) & (d > np.log1p(clip_high))
            low = (A < 0) & (d < np.log1p(-clip_low))
            far = (A < 0) & (d > np.log(dual_clip)) if dual_clip else np.zeros_like(cut)
            used = np.where(high, 1 + clip_high, np.where(low, 1 - clip_low, np.where(far, dual_clip, rho)))
            term = np.where(A == 0, 0.0, -w * used * A)
            slope = np.where(high | low | far | (A == 0), 0.0, -w * A * rho)
            out["policy"] += weight * term.sum()
            out["size"] += weight * np.abs(term).sum()
            out["clipped"] += int((high | low | far).sum())
            out["cut"] += int(cut.sum())
            if ratio == "sequence":
                out["seq_size"][s] = weight * np.abs(slope).sum() / len(s)
                slope = np.full(len(s), slope.sum() / len(s))
            out["policy_grad"][s] = weight * slope
            out["d"][s] = d
            if logp_ref is not None:
                x = logp_ref[s] - logp[s]
                out["kl"] += weight * (np.expm1(x) - x).sum()
                out["kl_grad"][s] = -kl_coef * weight * np.expm1(x)
            if entropy is not None:
                out["entropy"] += weight * entropy[s].sum()
                out["dentropy"][s] = -entropy_coef * weight
    out["dlogp"] = out["policy_grad"] + out["kl_grad"]
    out["loss"] = out["policy"] + kl_coef * out["kl"] - entropy_coef * out["entropy"]
    return out


class PerSequence(np.ndarray):
    """Advantages of whole sequences (their number may equal that of the tokens)."""
    per_sequence = True


def balance_loss(logits, idx, mask=None, counts=None, balance_coef=1.0, z_coef=0.0):
    """logits [T, E], idx [T, K]: (balance, z, counts [E], dlogits [T, E], p, lse, f)."""
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    on = np.ones(T, dtype=bool) if mask is None else np.asarray(mask).astype(bool)
    n = max(1, int(on.sum()))
    if counts is None:
        counts = np.bincount(np.asarray(idx)[on].ravel(), minlength=E) if on.any() else np.zeros(E, dtype=int)
    f = E * counts / max(1, counts.sum())
    top = logits.max(1, keepdims=True)
    top = np.where(np.isneginf(top), 0.0, top)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.exp(logits - top)
        whole = e.sum(1, keepdims=True)
        p = np.where(whole == 0, 0.0, e / np.where(whole == 0, 1.0, whole))
        lse = np.where(whole == 0, 0.0, top + np.log(np.where(whole == 0, 1.0, whole)))
    p, lse = np.where(on[:, None], p, 0.0), np.where(on[:, None], lse, 0.0)
    balance = float((f * p.sum(0)).sum() / n)
    z = float((lse ** 2).sum() / n)
    d = balance_coef * p * (f - (p * f).sum(1, keepdims=True)) / n + 2 * z_coef * lse * p / n
    return balance, z, counts, d, p, lse, f
