"""Shared test helpers: build a synthetic case on the CPU, widen it for the oracle."""
import numpy as np
import torch

from oracle import r3_oracle as O
from paper_2510_11370_b200 import synth


def f64(t: torch.Tensor) -> np.ndarray:
    """Exact widening of a stored tensor (bf16 / f32) to float64 numpy."""
    return t.detach().to("cpu").to(torch.float64).numpy()


def f32(t: torch.Tensor) -> np.ndarray:
    """Exact widening of a stored tensor (bf16 / f32) to float32 numpy (halves oracle memory)."""
    return t.detach().to("cpu").to(torch.float32).numpy()


class Case:
    """Inputs of one replayed layer (CPU tensors) plus the oracle's logits and the record."""

    def __init__(self, w: synth.Workload, layer: int = 0, device="cpu"):
        self.w = w
        self.x = synth.activations(w, device, layer).cpu()
        self.dy = synth.upstream_grad(w, device, layer).cpu()
        self.w_r = synth.router_weight(w, device, layer).cpu()
        self.w_gate, self.w_up, self.w_down = (t.cpu() for t in synth.expert_weights(w, device, layer))
        self.s = O.router_logits(f64(self.x), f64(self.w_r))
        self.idx = synth.make_record(w, torch.from_numpy(self.s), layer).cpu()

    def idx_np(self) -> np.ndarray:
        return self.idx.to(torch.int64).numpy()

    def oracle_layer(self):
        return O.layer_fwd_bwd(f64(self.x), f64(self.w_r), self.idx_np(), f32(self.w_gate),
                               f32(self.w_up), f32(self.w_down), f64(self.dy))

    def cuda(self):
        return {k: getattr(self, k).cuda() for k in
                ("x", "dy", "w_r", "w_gate", "w_up", "w_down", "idx")}


def rel_err(got, ref) -> float:
    """max |err| / max |ref| - the tolerance measure of the benchmark brief."""
    got = np.asarray(got, dtype=np.float64)
    ref = np.asarray(ref, dtype=np.float64)
    denom = np.abs(ref).max()
    return float(np.abs(got - ref).max() / (denom if denom > 0 else 1.0))


def random_record(rng: np.random.Generator, T: int, E: int, K: int, dtype) -> torch.Tensor:
    """K distinct experts per token, uniformly random, random slot order."""
    keys = rng.random((T, E))
    idx = np.argsort(keys, axis=1)[:, :K]
    return torch.from_numpy(idx.astype(np.int64)).to(dtype)


def logits_gradient_bound(logits, token_ids, dlogp, dentropy, temperature, ref, eps):
    """How far a float32 kernel's gradient to the logits may be from `ref` (float64, the oracle's), element by
    element.  An element is p k plus, at the token, g = dlogp / temperature, with k = -g - ge (log p + H) and
    ge = dentropy / temperature; it is rounded once, by eps / 2 of itself.
      p = 2^u, u from z = (x - top) / temperature and L: the difference, the constant and L's product are off
      by 2^-24 of |z|, |z|, L and L, the sum by 2^-24 of |log p|, which |z| + L is (L >= 0, z <= 0); L itself by
      the forward's 2e-5; the exponential by 2^-22.  Together p is within 2e-5 + 2^-22 (|log p| + 1).
      k: log p as above, H within 2e-5 + 2^-22 H, three roundings of the terms: within
      |ge| (4e-5 + 2^-21 (|log p| + H)) + 2^-22 |g|, the last within p's share of |g|.
      g: two roundings, 2^-23.
    Probabilities below float32's normal range count as 0."""
    z = np.asarray(logits, dtype=np.float64)
    top = z.max(axis=1, keepdims=True)
    with np.errstate(invalid="ignore", over="ignore"):
        z = np.where(np.isneginf(top), -np.inf, (z - np.where(np.isneginf(top), 0, top)) / temperature)
        total = np.exp(z).sum(axis=1, keepdims=True)
        lp = z - np.log(np.where(total > 0, total, 1))
    p = np.exp(lp)
    size = np.where(p > 0, np.maximum(lp, -1e4), 0) * -1                       # |log p| where it counts
    g = np.abs(np.asarray(dlogp, dtype=np.float64))[:, None]
    ge = 0.0 if dentropy is None else np.abs(np.asarray(dentropy, dtype=np.float64))[:, None]
    H = (p * size).sum(axis=1, keepdims=True)
    factor = g + ge * (size + H)
    bound = p * ((2e-5 + 2.0 ** -22 * (size + 1)) * factor + ge * (4e-5 + 2.0 ** -21 * (size + H)))
    bound += 2.0 ** -126 * (1 + factor)
    at = np.asarray(token_ids)
    rows = np.nonzero((at >= 0) & (at < z.shape[1]))[0]
    bound[rows, at[rows]] += 2.0 ** -23 * g[rows, 0]
    return bound / temperature + eps / 2 * np.abs(ref) + 2.0 ** -126
