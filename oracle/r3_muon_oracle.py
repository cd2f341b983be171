"""Float64 oracle of the orthogonalised update: the Newton-Schulz iteration and the momentum step around
it, and a model of the iteration with fp16 operands (what a product loses by them, nothing else).  Test
infrastructure only."""
import numpy as np

QUINTIC = (3.4445, -4.7750, 2.0315)


def iterate(u, steps=5, coefs=None, eps=1e-7, operand=None):
    """u [rows, cols] -> X after `steps`.  operand: rounds what enters a product (and the Gram matrix as it is
    stored); the last product is (a I + b A + c A^2) X, and what X loses as its operand is added, times a: X
    itself is carried without rounding."""
    u = np.asarray(u, dtype=np.float64)
    flip = u.shape[0] > u.shape[1]
    x = u.T if flip else u
    norm = np.sqrt((x ** 2).sum())
    x = x / (norm + eps) if norm > 0 else x * 0
    for k in range(steps):
        a, b, c = QUINTIC if coefs is None else coefs[k]
        h = x if operand is None else operand(x)
        A = h @ h.T
        if operand is not None:
            A = operand(A)
        B = a * np.eye(A.shape[0]) + b * A + c * (A @ A)
        if operand is not None:
            B = operand(B)
        x = B @ h + a * (x - h)
    return x.T if flip else x


def half_operand(x):
    """To fp16 with the library's power of two."""
    return (x * 1024.0).astype(np.float16).astype(np.float64) / 1024.0


def step(w, m, g, lr, momentum=0.95, nesterov=True, decay=0.0, scale=1.0, grad_scale=1.0, **kw):
    """One matrix: (w, m) after the step."""
    g = np.asarray(g, dtype=np.float64) * grad_scale
    m = momentum * np.asarray(m, dtype=np.float64) + g
    u = g + momentum * m if nesterov else m
    w = np.asarray(w, dtype=np.float64)
    return w * (1 - lr * decay) - lr * scale * iterate(u, **kw), m
