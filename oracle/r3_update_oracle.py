"""CPU oracle (numpy float64) of the operators around the replayed block in an Update step: token
log probabilities and their gradient, the norms around a block and their gradient, and one AdamW
step.  Each function is the operator's definition written out; nothing is shared with the product."""
from __future__ import annotations

import numpy as np


# ---- log probabilities of given tokens --------------------------------------------------------
def token_logprobs(logits, token_ids, temperature=1.0, n_top=0):
    """logits [T, V], token_ids [T] (negative: the row is skipped).  Returns a dict of logp [T],
    entropy [T], stats [T, 2] (largest logit, log of the sum of exponentials above it), top_ids
    [T, n_top] (ties to the lower id), top_logp [T, n_top]."""
    z = np.asarray(logits, dtype=np.float64)
    T, V = z.shape
    out = dict(logp=np.zeros(T), entropy=np.zeros(T), stats=np.zeros((T, 2)),
               top_ids=np.full((T, n_top), -1, dtype=np.int64), top_logp=np.zeros((T, n_top)))
    for t in range(T):
        i = int(token_ids[t])
        if i < 0 or i >= V:
            continue
        row = z[t]
        if np.isnan(row).any() or np.isposinf(row).any():
            for k in ("logp", "entropy", "stats", "top_logp"):
                out[k][t] = np.nan
            continue
        order = np.argsort(-row, kind="stable")[:n_top]
        out["top_ids"][t] = order
        top = row.max()
        if np.isneginf(top):
            out["logp"][t] = -np.inf
            out["top_logp"][t] = -np.inf
            out["stats"][t] = (-np.inf, 0.0)
            continue
        e = (row - top) / temperature
        total = np.log(np.exp(e).sum())
        lp = e - total
        p = np.exp(lp)
        out["logp"][t] = lp[i]
        out["entropy"][t] = -np.sum(p[p > 0] * lp[p > 0])
        out["stats"][t] = (top, total)
        out["top_logp"][t] = lp[order]
    return out


def token_logprobs_bwd(logits, token_ids, dlogp, dentropy=None, temperature=1.0):
    """d/dlogits of sum_t dlogp[t] logp[t] + dentropy[t] entropy[t]."""
    z = np.asarray(logits, dtype=np.float64)
    f = token_logprobs(z, token_ids, temperature)
    out = np.zeros_like(z)
    for t in range(z.shape[0]):
        i = int(token_ids[t])
        top, total = f["stats"][t]
        if i < 0 or i >= z.shape[1] or np.isneginf(top):
            continue
        lp = (z[t] - top) / temperature - total
        p = np.exp(lp)
        d = -dlogp[t] * p
        d[i] += dlogp[t]
        if dentropy is not None:
            live = p > 0
            d[live] -= dentropy[t] * p[live] * (lp[live] + f["entropy"][t])
        out[t] = d / temperature
    return out


# ---- norm, gate, scaled residual, norm ---------------------------------------------------------
def _gate_2d(gate, T, d):
    """gate None, [d], [T, 1] or [T, d] as a factor over [T, d]."""
    return np.ones((T, d)) if gate is None else np.broadcast_to(np.asarray(gate, dtype=np.float64), (T, d))


def rms_norm(v, w, eps):
    v = np.asarray(v, dtype=np.float64)
    return v / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps) * w


def norm_residual(x, y, w_post=None, gate=None, w_pre=None, eps=1e-6, residual_scale=1.0,
                  branch_scale=1.0):
    """(x_out or None, h or None)."""
    x = np.asarray(x, dtype=np.float64)
    if y is None:
        return None, rms_norm(x, w_pre, eps)
    y = np.asarray(y, dtype=np.float64)
    n = y if w_post is None else rms_norm(y, w_post, eps)
    x_out = residual_scale * x + branch_scale * _gate_2d(gate, *x.shape) * n
    return x_out, None if w_pre is None else rms_norm(x_out, w_pre, eps)


def rms_norm_bwd(v, w, eps, dn):
    """(dv, dw) of rms_norm for the upstream gradient dn."""
    r = 1.0 / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)
    u = dn * w
    return r * u - v * r ** 3 * (u * v).mean(axis=1, keepdims=True), (dn * v * r).sum(axis=0)


def norm_residual_bwd(x_out, y, dx_out, dh=None, w_post=None, gate=None, w_pre=None, eps=1e-6,
                      residual_scale=1.0, branch_scale=1.0):
    """dict of dx, dy, dw_post, dgate (in the gate's shape), dw_pre; x_out is x where y is None."""
    out = {}
    g = 0.0 if dx_out is None else np.asarray(dx_out, dtype=np.float64)
    if w_pre is not None:
        through, out["dw_pre"] = rms_norm_bwd(x_out, w_pre, eps, dh)
        g = g + through
    if y is None:
        out["dx"] = g
        return out
    T, d = y.shape
    out["dx"] = residual_scale * g
    n = y if w_post is None else rms_norm(y, w_post, eps)
    q = branch_scale * g
    dgate, dn = q * n, q * _gate_2d(gate, T, d)
    if gate is not None:
        shape = np.asarray(gate).shape
        out["dgate"] = dgate if shape == (T, d) else (dgate.sum(axis=1, keepdims=True)
                                                      if shape == (T, 1) else dgate.sum(axis=0))
    if w_post is None:
        out["dy"] = dn
    else:
        out["dy"], out["dw_post"] = rms_norm_bwd(y, w_post, eps, dn)
    return out


# ---- AdamW -----------------------------------------------------------------------------------------
BLOCK = 256
E4M3_MAX, E4M3_MIN = 448.0, 2.0 ** -9


def adamw(w, g, m, v, step, lr, betas, eps, decay, grad_scale=1.0):
    """One step on float64 arrays: (w, m, v)."""
    g = np.asarray(g, dtype=np.float64) * grad_scale
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    mh, vh = m / (1 - betas[0] ** step), v / (1 - betas[1] ** step)
    return w - lr * decay * w - lr * mh / (np.sqrt(vh) + eps), m, v


def block_scale(x):
    """[blocks, 256] -> the smallest power of two >= 2^-126 that brings each block to at most 448."""
    top = np.abs(np.asarray(x, dtype=np.float64)).max(axis=1)
    out = np.empty_like(top)
    for b, t in enumerate(top):
        k = -126
        while t > E4M3_MAX * 2.0 ** k:
            k += 1
        out[b] = 2.0 ** k
    return out


def e4m3_values():
    """The non-negative finite values of the type, by code."""
    vals = []
    for code in range(127):
        e, f = code >> 3, code & 7
        vals.append(f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return np.array(vals)


def nearest_e4m3(q):
    """The nearest e4m3 value of each element (|q| <= 448), ties to the even code."""
    vals = e4m3_values()
    a = np.abs(np.asarray(q, dtype=np.float64))
    hi = np.searchsorted(vals, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    up, down = vals[hi] - a, a - vals[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(vals[code], q)


# ---- stacks of replayed blocks with norms around every block ----------------------------------------
def normed_stack_bwd(x0, layers, norms, dy, eps=1e-6, residual_scale=1.0, branch_scale=1.0, store=None,
                     expert_grads=False):
    """h_l = RMSNorm(x_l) w_pre,l; x_{l+1} = residual_scale x_l + branch_scale gate_l RMSNorm(y_l) w_post,l
    with y_l the replayed layer at h_l; then the gradient of <dy, x_L>.  layers[l] = (w_r, idx, w_gate,
    w_up, w_down), norms[l] = (w_pre, w_post or None, gate or None).  store: rounding of kept rows.
    Returns a dict of x_out, dx0 and lists ds, dw_r, dw_pre, dw_post, dgate, dw_experts."""
    from oracle import r3_oracle as O
    keep = store or (lambda v: v)
    kw = dict(eps=eps, residual_scale=residual_scale, branch_scale=branch_scale)
    L = len(layers)
    xs, hs, ys = [np.asarray(x0, dtype=np.float64)], [], []
    h = rms_norm(xs[0], norms[0][0], eps)
    for l in range(L):
        h = keep(h)
        w_r, idx, wg, wu, wd = layers[l]
        y = O.replay_output(h, O.router_logits(h, w_r), idx, wg, wu, wd)[0]
        hs.append(h)
        ys.append(keep(y))
        w_next = norms[l + 1][0] if l + 1 < L else None
        x, h = norm_residual(xs[l], ys[l], norms[l][1], norms[l][2], w_next, **kw)
        xs.append(keep(x))
    out = dict(x_out=xs[L], ds=[None] * L, dw_r=[None] * L, dw_pre=[None] * L, dw_post=[None] * L,
               dgate=[None] * L, dw_experts=[None] * L)
    around, dh = np.asarray(dy, dtype=np.float64), None
    for l in range(L - 1, -1, -1):
        w_next = norms[l + 1][0] if l + 1 < L else None
        g = norm_residual_bwd(xs[l + 1], ys[l], around, dh, norms[l][1], norms[l][2], w_next, **kw)
        if w_next is not None:
            out["dw_pre"][l + 1] = g["dw_pre"]
        out["dw_post"][l], out["dgate"][l] = g.get("dw_post"), g.get("dgate")
        around, dyl = g["dx"], g["dy"]
        w_r, idx, wg, wu, wd = layers[l]
        b = O.layer_bwd_input(hs[l], w_r, idx, wg, wu, wd, dyl)
        out["ds"][l], out["dw_r"][l] = b["ds"], b["dw_r"]
        if expert_grads:
            out["dw_experts"][l] = O.layer_bwd_weights(hs[l], w_r, idx, wg, wu, wd, dyl)
        dh = b["dx"]
    g = norm_residual_bwd(xs[0], None, around, dh, w_pre=norms[0][0], eps=eps)
    out["dw_pre"][0], out["dx0"] = g["dw_pre"], g["dx"]
    return out
